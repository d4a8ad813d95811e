// What attention's kernels share: tiles of rows in shared memory and how the matrix instructions read them, masks, the bias.
//
// Scores are formed with the pair's two sides such that probabilities stay in registers.  A 32 x 32 product leaves a lane with one column (lane % 32) and
// 16 rows (8 a + 4 (lane / 32) + 0 .. 3, a = 0 .. 3); as the right operand of the next product it wants one column and eight values along the
// sum.  Which eight is free as long as the left operand has the same: those of a = 2 m and 2 m + 1 for the m-th sixteen of the sum, so that
// the left operand's two reads take rows 16 m + 4 (lane / 32) + 0 .. 3 and eight further.  Nothing is exchanged between lanes.
#pragma once

#include "../../include/leap_networks.h"
#include "act_product.h"

namespace net {

using namespace act;

constexpr int TILE = 64;                   // rows of a tile: keys, or queries in the gradient of keys and values
constexpr int WAVE = 64, WAVES = 4, BLOCK = WAVE * WAVES;
constexpr int COLS = 32 * WAVES;           // queries (or keys) of a block, 32 to a wave
constexpr float LOG2E = 1.4426950408889634f;

// An array [item][row][head][width] of bfloat16.
struct rows_of {
    const uint16_t *data;
    int64_t item, row, head;
};

// Positions of a tile's rows: the least and the largest, whether every four (from a multiple of four on) are consecutive, and whether each is larger than the one before.
struct place_range {
    int32_t low, high, fours, rising;
};

struct attention_args {
    rows_of q, k, v;
    int32_t batch, queries, keys, heads, kv_heads, width;
    const uint8_t *mask;
    int64_t mask_item;
    const void *table;
    const int32_t *bucket_of, *query_positions, *key_positions;
    int32_t table_type, offsets, buckets;
    float scale;
    // in the workspace, with a table: a number for every difference of positions, in units of log2, heads `line` apart; its bucket; the positions of each TILE rows
    float *lines;
    uint16_t *line_buckets;
    uint8_t *line_rising;                  // of every 64 of them: each is larger than the one before
    place_range *query_places, *key_places;
    int32_t line;
};

// A tile of TILE rows of DEEP values in shared memory, in 16-byte pieces.  The order of a row's pieces lets 16 neighbouring rows be read at one piece, and
// four rows at four neighbouring pieces (the transposing read), each from all banks once.  96 values lie in rows of 128.
template <int DEEP> struct rows_tile {
    static constexpr int CHUNKS = DEEP / 8, ROW = DEEP <= 32 ? 64 : DEEP <= 64 ? 128 : 256, BYTES = TILE * ROW;
    static constexpr int EACH = TILE * CHUNKS / BLOCK;                     // pieces a thread brings
    static_assert(TILE * CHUNKS % BLOCK == 0, "");

    static __device__ inline int place(int r, int chunk)
    {
        const int turn = ROW == 256 ? r % 4 * 4 + r / 4 % 4 : ROW == 128 ? r / 2 % 2 * 4 + r / 4 % 4 : r / 4 % 4;
        return r * ROW + (chunk ^ turn) * 16;
    }
    // Eight values of row first + lane % 32 from 16 step + 8 (lane / 32) on: a side of a product along the width.
    static __device__ inline bf16x8 along(const lds_byte *from, int first, int step, int lane)
    {
        return *(const __attribute__((address_space(3))) bf16x8 *)(from + place(first + lane % 32, step * 2 + lane / 32));
    }
    // The values of column 32 block + lane % 32 in rows first + 4 (lane / 32) + 0 .. 3 and eight further.
    static __device__ inline bf16x8 across(const lds_byte *from, int first, int block, int lane)
    {
        const int row = first + lane / 32 * 4 + lane % 16 / 4, col = block * 32 + lane / 16 % 2 * 16 + lane % 4 * 4;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(from + place(row, col / 8) + col % 8 * 2));
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(from + place(row + 8, col / 8) + col % 8 * 2));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// Eight values of a row of `width` from 8 chunk on, zeros beyond its end.  Nothing beyond the row is read: the last piece of a row
// that does not end with it is the row's last eight values, moved.
__device__ inline u32x4 moved(const u32x4 &v, int values)
{
    const uint64_t low = (uint64_t)v[1] << 32 | v[0], high = (uint64_t)v[3] << 32 | v[2];
    const int s = values * 16;                                             // 16 .. 112
    const uint64_t a = s < 64 ? low >> s | high << (64 - s) : high >> (s - 64), b = s < 64 ? high >> s : 0;
    return u32x4{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
}
__device__ inline u32x4 row_piece(const uint16_t *row, int width, int chunk)
{
    const int left = width - chunk * 8;
    u32x4 v = {0, 0, 0, 0};
    if (width >= 8) {
        if (left > 0) {
            const int back = left < 8 ? 8 - left : 0;
            __builtin_memcpy(&v, row + chunk * 8 - back, 16);
            if (width % 8) v = back ? moved(v, back) : v;
        }
    } else if (left > 0) {
        uint16_t e[8] = {};
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left) e[i] = row[i];
        __builtin_memcpy(&v, e, 16);
    }
    return v;
}

// Where a product's side along the width lies in a lane: eight values of its row a step.
template <int STEPS> __device__ inline void load_side(bf16x8 (&side)[STEPS], const uint16_t *row, int width, bool there, int lane)
{
#pragma unroll
    for (int s = 0; s < STEPS; ++s) side[s] = __builtin_bit_cast(bf16x8, there ? row_piece(row, width, s * 2 + lane / 32) : u32x4{0, 0, 0, 0});
}

// Tiles of one head's rows on their way to shared memory.  DIRECT: past the registers, where rows begin at multiples of 16 bytes, are whole
// multiples of 8 values or followed by zeros, and a tile spans less than 2^31 bytes.  Otherwise through them, so that land() puts down what fetch() has asked for.
template <int DEEP, bool DIRECT> struct source;
template <int DEEP> struct source<DEEP, true> {
    using tile = rows_tile<DEEP>;
    static constexpr int PIECES = tile::BYTES / 1024, EACH = PIECES / WAVES;           // 1 KiB: a wave's fetch
    static_assert(PIECES % WAVES == 0, "");
    const uint8_t *base;
    int64_t stride, end;                   // bytes from row to row; of the array from its first row on
    uint32_t offset[EACH];                 // of a lane's 16 bytes from its tile's first row on; NOWHERE: not of the row

    __device__ inline source(const uint16_t *rows, int64_t stride_, int64_t count, int width, int wave, int lane) : base((const uint8_t *)rows), stride(stride_ * 2)
    {
        end = (count - 1) * stride + whole(width * 2, 16);                  // (rows whose width is no multiple of 8 have zeros up to one, from lay_out)
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int slot = (e * WAVES + wave) * 64 + lane, r = slot * 16 / tile::ROW, chunk = (tile::place(r, 0) - r * tile::ROW) / 16 ^ slot % (tile::ROW / 16);
            offset[e] = chunk * 8 < width ? (uint32_t)(r * stride) + chunk * 16 : NOWHERE;
        }
    }
    __device__ inline void fetch(int64_t first, uint64_t there, lds_byte *to, int wave, int lane) const
    {
        const u32x4 from = window{base + first * stride, end - first * stride, 0}.buffer();
        if (!~there) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) fetch16(from, offset[e], to + (e * WAVES + wave) * 1024);
            return;
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int piece = e * WAVES + wave, r = (piece * 64 + lane) * 16 / tile::ROW;
            fetch16(from, there >> r & 1 ? offset[e] : NOWHERE, to + piece * 1024);
        }
    }
    __device__ inline void land(lds_byte *) const {}
};
template <int DEEP> struct source<DEEP, false> {
    using tile = rows_tile<DEEP>;
    const uint16_t *base;
    int64_t stride;
    int width;
    u32x4 piece[tile::EACH];

    __device__ inline source(const uint16_t *rows, int64_t stride_, int64_t, int width_, int, int) : base(rows), stride(stride_), width(width_) {}
    __device__ inline void fetch(int64_t first, uint64_t there, lds_byte *, int, int)
    {
#pragma unroll
        for (int e = 0; e < tile::EACH; ++e) {
            const int id = e * BLOCK + threadIdx.x, r = id / tile::CHUNKS, chunk = id % tile::CHUNKS;
            piece[e] = there >> r & 1 ? row_piece(base + (first + r) * stride, width, chunk) : u32x4{0, 0, 0, 0};
        }
    }
    __device__ inline void land(lds_byte *to) const
    {
#pragma unroll
        for (int e = 0; e < tile::EACH; ++e) {
            const int id = e * BLOCK + threadIdx.x, r = id / tile::CHUNKS, chunk = id % tile::CHUNKS;
            *(__attribute__((address_space(3))) u32x4 *)(to + tile::place(r, chunk)) = piece[e];
        }
    }
};

// All that fetch16 has asked for is in shared memory, of this wave; a barrier makes it so for the block.
__device__ inline void fetched() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Which of the rows first .. first + TILE - 1 there are: within `rows`, and in the mask (null: all).
__device__ inline uint64_t rows_there(const uint8_t *mask, int64_t first, int64_t rows, int lane)
{
    const bool in = first + lane < rows;
    return __ballot(in && (!mask || mask[first + lane]));
}

// The tiles of an item's keys that have any, one after the other; the mask's bytes are asked for a tile ahead.
struct key_walk {
    const uint8_t *mask;
    int64_t keys, first;
    uint64_t bits;
    uint8_t ahead;

    __device__ inline uint8_t ask(int64_t at, int lane) const { return at + lane < keys ? mask ? mask[at + lane] : 1 : 0; }
    // From `begin`, a multiple of TILE, to `end`.
    __device__ inline key_walk(const uint8_t *mask_, int64_t begin, int64_t end, int lane) : mask(mask_), keys(end), first(begin - TILE)
    {
        ahead = ask(begin, lane);
        next(lane);
    }
    __device__ inline void next(int lane)
    {
        do {
            first += TILE;
            bits = __ballot(ahead != 0);
            ahead = ask(first + TILE, lane);
        } while (!bits && first < keys);
    }
    __device__ inline bool done() const { return first >= keys; }
};

// Numbers of the table in units of log2; what is finite stays so.
__device__ inline float table_value(const attention_args &A, int head, int bucket)
{
    const int64_t at = (int64_t)head * A.buckets + bucket;
    const float v = A.table_type == LEAP_F32    ? ((const float *)A.table)[at]
                    : A.table_type == LEAP_BF16 ? element<LEAP_BF16>::to_float(((const uint16_t *)A.table)[at])
                                                : element<LEAP_F16>::to_float(((const uint16_t *)A.table)[at]);
    const float most = element<LEAP_F32>::LARGEST, scaled = v * LOG2E;
    return finite_magnitude(v) && !finite_magnitude(scaled) && scaled != 0.0f ? copysignf(most, v) : scaled;
}

__device__ inline int query_position(const attention_args &A, int i) { return A.query_positions ? A.query_positions[i] : i; }
__device__ inline int key_position(const attention_args &A, int j) { return A.key_positions ? A.key_positions[j] : j; }

// The bucket of a line's number.
__device__ inline int bucket_at(const attention_args &A, int64_t at)
{
    const int b = A.bucket_of[at];
    return b < 0 ? 0 : b >= A.buckets ? A.buckets - 1 : b;
}

// Register r of a lane's 32 rows stands for row row_of(r) + 4 (lane / 32).
__device__ inline constexpr int row_of(int r) { return r / 4 * 8 + r % 4; }

// Where in a line the difference of two positions is.
__device__ inline int line_at(const attention_args &A, int key, int query)
{
    const int64_t at = (int64_t)key - query + A.offsets / 2;
    return at < 0 ? 0 : at >= A.offsets ? A.offsets - 1 : (int)at;
}

// The part of a line that the pairs of two tiles' rows take: the numbers from `first` (a multiple of eight) on, `count` of them.  `inside`: it is within the line and
// MOST numbers, so that shared memory has it; otherwise pairs look theirs up in memory.
struct line_window {
    int first, count;
    bool inside;
};
__device__ inline line_window window_of(const attention_args &A, const place_range &keys, const place_range &queries, int most)
{
    const int64_t low = (int64_t)keys.low - queries.high + A.offsets / 2, high = (int64_t)keys.high - queries.low + A.offsets / 2;
    const int64_t first = low / 8 * 8;
    return {(int)first, (int)(high - first + 1), low >= 0 && high < A.offsets && high - first < most};
}
__device__ inline place_range both(const place_range &a, const place_range &b) { return {a.low < b.low ? a.low : b.low, a.high > b.high ? a.high : b.high, a.fours & b.fours, 0}; }

// Brings a window of SIZE-byte numbers to shared memory, a KiB a wave.
template <int SIZE> __device__ inline void fetch_window(const void *line, int length, const line_window &w, lds_byte *to, int wave, int lane)
{
    const u32x4 from = window{(const uint8_t *)line, whole((int64_t)length * SIZE, 16), 0}.buffer();
    for (int piece = wave; piece * (1024 / SIZE) < w.count; piece += WAVES) fetch16(from, (uint32_t)w.first * SIZE + piece * 1024 + lane * 16, to + piece * 1024);
}

// Where in shared memory a window's number is for a row at position 0: the window is at `to`, and the lane's position counts with the sign.  Modulo 2^32, as over_places
// goes on: positions are up to 2^30, so four times one passes 31 bits, and the sum of both is in the window again.
__device__ inline uint32_t origin_of(const lds_byte *to, const attention_args &A, const line_window &w, int position, bool added)
{
    return (uint32_t)(uintptr_t)to + 4u * ((uint32_t)(A.offsets / 2) - (uint32_t)w.first + (added ? (uint32_t)position : 0u - (uint32_t)position));
}

// f(r, p) for the sixteen pairs of a lane's position with the rows 8 a + 4 (lane / 32) + c of `places`: *p is the pair's number.  The rows are keys (SIGN 1) or queries
// (-1).  at: origin_of.
template <int SIGN, class T, class F> __device__ inline void over_places(const int *places, bool fours, uint32_t at, int lane, F &&f)
{
    typedef __attribute__((address_space(3))) T *numbers;
    if (fours) {
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const numbers begin = (numbers)(uintptr_t)(at + 4u * SIGN * ((uint32_t)places[a * 8 + lane / 32 * 4] + (SIGN < 0 ? 3 : 0)));
#pragma unroll
            for (int c = 0; c < 4; ++c) f(a * 4 + c, begin + (SIGN < 0 ? 3 - c : c));
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) f(r, (numbers)(uintptr_t)(at + 4u * SIGN * (uint32_t)places[row_of(r) + lane / 32 * 4]));
    }
}

__device__ inline bf16x8 eight(const f32x16 &v, int m)
{
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)v[m * 8 + i];
    return r;
}

// v's m-th eight as the sum of PARTS bfloat16, each of what those before leave (nothing here is infinite).  A difference is one instruction, v - (1, 0).(part, its neighbour) or with (0, 1): exact, as the
// difference is.  The constants come from registers: of those in an instruction the compiler makes others.
template <int PARTS> __device__ inline void parts_of_eight(const f32x16 &v, int m, bf16x8 (&part)[PARTS])
{
    uint32_t low = 0x0000bf80u, high = 0xbf800000u;                        // (-1, 0), (0, -1)
    if constexpr (PARTS > 1) asm("" : "+s"(low), "+s"(high));
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float a = v[m * 8 + i], b = v[m * 8 + i + 1];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const bf16x2 both = {(__bf16)a, (__bf16)b};
            part[p][i] = both[0], part[p][i + 1] = both[1];
            if (p + 1 == PARTS) break;
            a = __builtin_amdgcn_fdot2_f32_bf16(both, __builtin_bit_cast(bf16x2, low), a, false);
            b = __builtin_amdgcn_fdot2_f32_bf16(both, __builtin_bit_cast(bf16x2, high), b, false);
        }
    }
}

// Inside a branch that is seldom taken: it stays one, instead of selections that are always made.
__device__ inline void seldom() { asm volatile(""); }

__device__ inline f32x16 product(const bf16x8 &a, const bf16x8 &b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

__device__ inline f32x16 zeros()
{
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}

// The two lanes of a column, which hold its two sets of rows, as one.
template <class F> __device__ inline float both_halves(float v, F &&f)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float column_sum(float v)
{
    return both_halves(v, [](float a, float b) { return a + b; });
}
__device__ inline float column_max(float v)
{
    return both_halves(v, [](float a, float b) { return fmaxf(a, b); });
}

// A lane's column of a [width][32] result, times `by`, to a row of `width` bfloat16; BLOCKS of 32 values.
template <int BLOCKS> __device__ inline void store_column(uint16_t *row, int width, f32x16 (&v)[BLOCKS], float by, int lane, bool there)
{
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        uint32_t run[4][2];
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            run[a][0] = two_bf16(v[b][a * 4] * by, v[b][a * 4 + 1] * by);
            run[a][1] = two_bf16(v[b][a * 4 + 2] * by, v[b][a * 4 + 3] * by);
        }
        join_runs<2>(run);                     // sixteen neighbours
        const int at = b * 32 + lane / 32 * 16;
        if (!there) continue;
#pragma unroll
        for (int p = 0; p < 2; ++p)
            if (at + p * 8 < width)
                store_piece<2>((uint8_t *)(row + at + p * 8), (int64_t)(width - at - p * 8) * 2,
                               u32x4{run[p * 2][0], run[p * 2][1], run[p * 2 + 1][0], run[p * 2 + 1][1]});
    }
}

// A number that a wave's lanes have in common, as the compiler is to know.
__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Unit u of `units`, such that neighbouring units (which share keys, or queries) run on the same of the eight parts of the chip: blocks go round over those.
__device__ inline int64_t unit_of(int64_t block, int64_t units)
{
    const int64_t each = units / 8, more = units % 8, part = block % 8, turn = block / 8;
    return part * each + (part < more ? part : more) + turn;
}

// ---- host side ----

// f(the width up to a multiple of 32, as a constant)
template <class F> inline int by_width(int64_t width, F &&f)
{
    if (width <= 32) return f(std::integral_constant<int, 32>{});
    if (width <= 64) return f(std::integral_constant<int, 64>{});
    if (width <= 96) return f(std::integral_constant<int, 96>{});
    return f(std::integral_constant<int, 128>{});
}

// f(flags as constants)
template <class F> inline int by_flags(F &&f) { return f(); }
template <class F, class... R> inline int by_flags(F &&f, bool flag, R... rest)
{
    if (flag) return by_flags([&](auto... c) { return f(std::true_type{}, c...); }, rest...);
    return by_flags([&](auto... c) { return f(std::false_type{}, c...); }, rest...);
}

constexpr const char *TOO_MANY_BLOCKS = "2^24 or more of an item's 128 queries, or keys, of a head: items times heads times those";
// Null if fine: an array's strides; a description.
const char *bad_array(int64_t items, int64_t item, int64_t rows, int64_t row, int64_t heads, int64_t head);
const char *bad_attention(const leap_attention_desc *d);
attention_args arguments_of(const leap_attention_desc *d, const void *q, const void *k, const void *v);

// Whether every row of an array is a whole number of aligned 16 bytes and a tile of them within a buffer's reach.
bool direct_array(const void *p, int64_t item, int64_t row, int64_t head, int64_t width);
// Rows whose width is no multiple of 8 as rows that are, with zeros behind them: bytes, and what writes them.  Pays (18414 patches of 49: a step of 9.3 ms, 12.4 without)
// where a row is read again and again: by more than LAID_OUT rows of the other side.
constexpr int64_t LAID_OUT = 512;
int64_t laid_out_bytes(int64_t items, int64_t rows, int64_t heads, int64_t width);
int lay_out(rows_of &array, int64_t items, int64_t rows, int64_t heads, int64_t width, void *to, hipStream_t st);
// The lines' workspace, and what writes it; nothing without a table.
int64_t lines_bytes(const leap_attention_desc *d);
int write_lines(attention_args &A, void *work, hipStream_t st);

}  // namespace net
