// The tiled product behind leap_linear8 and its kin: D[j][i] = sum over k of P(i, k) Q(j, k).
//
// A block owns TI x TJ of D and walks over k in steps of 64; a step's tiles of P and Q are fetched into shared memory (mostly straight
// from memory, past the registers) while the one or two steps before are multiplied: two or three buffers, one barrier a step.  i runs along a lane's
// registers and j across lanes, so a lane ends with runs of neighbouring i: what a row of an output, and a group of 32 that
// shares a scale, is made of.
//
// Which k a lane's eight values stand for is free as long as P and Q agree: of each 32, lane half h takes 16 h .. 16 h + 15
// in two turns of eight, so that 16 codes are one shared-memory read.
#pragma once

#include "act_common.h"

namespace act {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(3))) uint8_t lds_byte;

constexpr uint32_t NOWHERE = 0x80000000u;  // an offset beyond every buffer: reads as zeros

// How an operand lies in memory: rows of bfloat16 along k; rows of k; codes along k; rows of k of codes.
enum { WIDE_ALONG, WIDE_ACROSS, CODES_ALONG, CODES_ACROSS };

// `rows` rows (i or j) of `depth` values of k.  Memory rows are `stride` elements apart; every one begins at a multiple of 16
// bytes and has memory up to one, zeros beyond its end.
struct operand {
    const uint8_t *data, *scales;
    int64_t stride, groups;                // groups: scale bytes of a memory row
    int64_t rows, depth;
};

// What of an operand lies from the current k on: a buffer that moves along it, and ends where the operand does (reads beyond
// give zeros).
struct window {
    const uint8_t *base;
    int64_t left;              // bytes
    uint32_t step;             // bytes from one step to the next

    __device__ inline u32x4 buffer() const
    {
        const uint64_t at = (uint64_t)base;
        const auto uniform = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };    // it is; the compiler has to see it
        return u32x4{uniform((uint32_t)at), uniform((uint32_t)(at >> 32) & 0xffffu),
                     uniform(left <= 0 ? 0u : left < 0x7ffffff0 ? (uint32_t)left : 0x7ffffff0u), 0x00020000u};
    }
    // The same for the compiler's own loads.
    __device__ inline __amdgpu_buffer_rsrc_t resource() const
    {
        return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, left <= 0 ? 0 : left < 0x7ffffff0 ? (int)left : 0x7ffffff0, 0x00020000);
    }
    __device__ inline void advance() { base += step, left -= step; }
};

// n in whole pieces of 16 bytes: a fetch that ends inside a word reads nothing of it.
__device__ inline int64_t whole(int64_t n, int piece) { return (n + piece - 1) / piece * piece; }

// Starts a fetch of 16 bytes a lane, from `offset` of the buffer to 16 * lane beyond `to`.  In assembly, because the compiler would
// wait for the fetch before the next read of any shared memory; it has no result but shared memory, and every step begins by waiting for it.  m0, through
// which the address goes, cannot be declared as overwritten: it gets back what it held.
__device__ inline void fetch16(const u32x4 &from, uint32_t offset, lds_byte *to)
{
    uint32_t m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0)
                 : "s"(__builtin_amdgcn_readfirstlane((int)(uintptr_t)to)), "v"(offset), "s"(from)
                 : "memory");
}

// A tile of T rows and STEP values of k of an operand in shared memory, by KIND.  ALONG: T rows of 2 * STEP (codes: STEP)
// bytes, their 16-byte pieces in an order that spreads 16 neighbouring rows over all banks; ACROSS: STEP rows of 2 T bytes,
// pieces likewise spread for the transposing read, which takes four of them at once.
template <int KIND, int T, int STEP, int THREADS> struct tile {
    static constexpr int BYTES = KIND == CODES_ALONG ? T * STEP : T * STEP * 2;
    static constexpr int WAVES = THREADS / 64, PIECES = BYTES / 1024, EACH = PIECES / WAVES;       // 1 KiB pieces: a wave's fetch
    static_assert(PIECES % WAVES == 0, "a tile is fetched by all waves alike");
    static constexpr int VALUE = KIND == CODES_ALONG ? 1 : 2;                // bytes
    static constexpr int ROW = STEP * VALUE, CHUNKS = ROW / 16;              // ALONG: bytes and 16-byte pieces of a row
    static constexpr int ROWS = 1024 / ROW;                                  // and rows of a 1 KiB piece

    // Where piece `chunk` of row r goes (and what is found there): rows 256 / ROW apart begin in the same bank.
    static __device__ inline int place(int r, int chunk) { return chunk ^ (r / (256 / ROW) % CHUNKS); }

    // A wave's part in fetching tiles of the operand, k after k.  HALVES 2: the tile's rows are, span by span, the same rows of
    // two operands, `apart` bytes apart (the gate's and the other half).
    template <int HALVES, int SPAN> struct stream {
        uint32_t offset[EACH];
        window at;
        const uint8_t *other;                  // where the second half's window begins
        static_assert(HALVES == 1 || (KIND == WIDE_ALONG && WAVES * ROWS <= SPAN / 2), "all waves fetch of one half at a time");
        static constexpr int half_of(int e) { return HALVES == 1 ? 0 : e * WAVES * ROWS % SPAN / (SPAN / 2); }

        __device__ inline void init(const operand &O, int wave, int lane)
        {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const int piece = e * WAVES + wave;
                if constexpr (KIND == WIDE_ACROSS) {
                    constexpr int DEEP = 512 / T;                            // rows of k in a piece
                    const int k = piece * DEEP + lane / (T / 8), chunk = (lane % (T / 8)) ^ (k % 4 * 4);
                    offset[e] = (uint32_t)k * (uint32_t)O.stride * 2 + chunk * 16;
                } else {
                    const int r = piece * ROWS + lane / CHUNKS, row = HALVES == 1 ? r : r / SPAN * (SPAN / 2) + r % (SPAN / 2);
                    offset[e] = (uint32_t)row * (uint32_t)O.stride * VALUE + place(r, lane % CHUNKS) * 16;
                }
            }
        }

        // Rows from row0 on, k from `first` on, of an operand that ends at `rows` and at k = `last`.
        __device__ inline void aim(const operand &O, int64_t rows, int64_t row0, int64_t first, int64_t last, int64_t apart, int every)
        {
            if constexpr (KIND == WIDE_ACROSS)
                at = {O.data + (first * O.stride + row0) * 2, ((last - 1 - first) * O.stride + whole(rows, 8) - row0) * 2, (uint32_t)(every * STEP * O.stride * 2)};
            else
                at = {O.data + (row0 * O.stride + first) * VALUE, ((rows - 1 - row0) * O.stride + whole(last, 16 / VALUE) - first) * VALUE, (uint32_t)(every * STEP * VALUE)};
            other = at.base + apart;
        }

        // Makes the next tile's fetch ready, `k` values of k from the operand's end: pieces beyond that read as zeros.
        u32x4 from[HALVES];
        uint32_t dead;
        __device__ inline void ready(int64_t k, int wave, int lane)
        {
            from[0] = at.buffer();
            if constexpr (HALVES == 2) from[1] = window{other, at.left, 0}.buffer(), other += at.step;
            at.advance();
            dead = 0;
            // (the pieces a lane fetches are of the same place in their rows)
            static_assert(KIND == WIDE_ACROSS || WAVES * ROWS / (256 / ROW) % CHUNKS == 0, "");
            if constexpr (KIND != WIDE_ACROSS) dead = place(wave * ROWS + lane / CHUNKS, lane % CHUNKS) * (16 / VALUE) < k ? 0u : NOWHERE;
        }
        // Starts the fetch of its piece e.
        __device__ inline void fetch(int e, int wave, lds_byte *to) const { fetch16(from[half_of(e)], offset[e] | dead, to + (e * WAVES + wave) * 1024); }
    };

    // The eight values of turn s of 32-run `run` of the tile's rows first .. first + 31.
    static __device__ inline bf16x8 read(const lds_byte *from, int first, int run, int s, int lane)
    {
        const int half = lane / 32;
        if constexpr (KIND == WIDE_ALONG) {
            const int r = first + lane % 32;
            return *(const __attribute__((address_space(3))) bf16x8 *)(from + r * ROW + place(r, run * 4 + half * 2 + s) * 16);
        } else {
            const int k = run * 32 + half * 16 + s * 8 + lane % 16 / 4, col = first + lane / 16 % 2 * 16 + lane % 4 * 4;
            const lds_byte *at = from + k * (T * 2) + ((col / 8) ^ (k % 4 * 4)) * 16 + col % 8 * 2;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at);
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + 4 * T * 2));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }

    // The 16 codes of both turns.
    static __device__ inline u32x4 read_codes(const lds_byte *from, int first, int run, int lane)
    {
        const int r = first + lane % 32;
        return *(const __attribute__((address_space(3))) u32x4 *)(from + r * ROW + place(r, run * 2 + lane / 32) * 16);
    }

    // Eight codes as bfloat16; `scale` counts by its exponent alone.
    static __device__ inline bf16x8 widen(uint32_t lo, uint32_t hi, float scale)
    {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
        return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
};

// Codes across k on their way through the registers: widened between fetch and store, eight at a time.
template <int T, int STEP, int THREADS> struct staged_codes {
    static constexpr int EACH = T * STEP / 8 / THREADS, ROWS = THREADS / (T / 8);       // rows of k the block takes at once
    uint2 codes[EACH];
    uint32_t byte[EACH];
    uint32_t offset, scale_offset, stride, groups;
    window at, scales;

    int thread;                                        // of the group

    __device__ inline void init(const operand &O, int thread_)
    {
        thread = thread_;
        const uint32_t k = thread / (T / 8), i = thread % (T / 8) * 8;
        stride = (uint32_t)O.stride * ROWS, groups = (uint32_t)O.groups * ROWS;
        offset = k * (uint32_t)O.stride + i, scale_offset = k * (uint32_t)O.groups + i / GROUP;
    }

    __device__ inline void aim(const operand &O, int64_t row0, int64_t first, int64_t last, int every)
    {
        at = {O.data + first * O.stride + row0, (last - 1 - first) * O.stride + whole(O.rows, 16) - row0, (uint32_t)(every * STEP * O.stride)};
        scales = {O.scales + first * O.groups + row0 / GROUP, (last - first) * O.groups - row0 / GROUP, (uint32_t)(every * STEP * O.groups)};
    }

    __device__ inline void fetch()
    {
        const __amdgpu_buffer_rsrc_t from = at.resource(), with = scales.resource();
        at.advance(), scales.advance();
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            codes[e] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(from, offset + e * stride, 0, 0));
            byte[e] = __builtin_amdgcn_raw_buffer_load_b8(with, scale_offset + e * groups, 0, 0);
        }
    }

    __device__ inline void store(lds_byte *to) const
    {
        using as = tile<WIDE_ACROSS, T, STEP, THREADS>;
        const int k = thread / (T / 8), chunk = thread % (T / 8);
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            *(__attribute__((address_space(3))) bf16x8 *)(to + (k + e * ROWS) * (T * 2) + (chunk ^ ((k + e * ROWS) % 4 * 4)) * 16) =
                as::widen(codes[e].x, codes[e].y, __uint_as_float(byte[e] << 23));
    }
};

// Exchanges between lane halves so that the runs of four a lane holds of 32 neighbouring i (8 q + 4 half + 0 .. 3, q = 0 .. 3)
// become 16 neighbours: half 0 gets 0 .. 15, half 1 16 .. 31.  W words a run.
template <int W> __device__ inline void join_runs(uint32_t (&run)[4][W])
{
#pragma unroll
    for (int w = 0; w < W; ++w) {
        // the upper half of the first changes places with the lower half of the second
        const auto a = __builtin_amdgcn_permlane32_swap(run[0][w], run[2][w], false, false);
        const auto b = __builtin_amdgcn_permlane32_swap(run[1][w], run[3][w], false, false);
        run[0][w] = a[0], run[1][w] = a[1], run[2][w] = b[0], run[3][w] = b[1];
    }
}

// And back, a word a run.
__device__ inline void split_runs(uint32_t (&run)[4])
{
    const auto a = __builtin_amdgcn_permlane32_swap(run[0], run[1], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(run[2], run[3], false, false);
    run[0] = a[0], run[2] = a[1], run[1] = b[0], run[3] = b[1];
}

__device__ inline uint32_t two_bf16(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); }

// A wave's shared memory between its results, 32 rows (j, a lane each, twice) of which a lane holds pieces, and memory, which
// wants runs of a row from neighbouring lanes: with a lane a row every store would touch 32 lines.  Rows of PITCH bytes whose
// 16-byte pieces are in an order that keeps 16 lanes, of neighbouring rows or of one, in different banks.
template <int PITCH> struct exchange {
    static constexpr int CHUNKS = PITCH / 16, ROWS = 64 / CHUNKS, TURNS = 32 / ROWS;     // pieces a row, rows a turn of all lanes
    lds_byte *room;

    __device__ inline lds_byte *place(int row, int chunk) const
    {
        constexpr int A_LINE = PITCH >= 256 ? 1 : 256 / PITCH;
        return room + row * PITCH + ((chunk ^ (row / A_LINE % CHUNKS)) * 16);
    }
    __device__ inline void put(int row, int chunk, const u32x4 &v) const { *(__attribute__((address_space(3))) u32x4 *)place(row, chunk) = v; }
    __device__ inline u32x4 get(int row, int chunk) const { return *(const __attribute__((address_space(3))) u32x4 *)place(row, chunk); }

    // Half a piece; the halves change places every 16 rows, for the banks' sake.
    __device__ inline void put_half(int row, int chunk, int half, uint32_t a, uint32_t b) const
    {
        *(__attribute__((address_space(3))) uint64_t *)(place(row, chunk) + (half ^ (row / 16)) * 8) = (uint64_t)b << 32 | a;
    }
    __device__ inline u32x4 get_halves(int row, int chunk) const
    {
        const u32x4 v = get(row, chunk);
        return row / 16 ? u32x4{v[2], v[3], v[0], v[1]} : v;
    }
    // The lanes' stores are there for its loads: a wave's accesses are carried out in order.
    __device__ static inline void turn() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }
};

// The first n of 16 bytes; SIZE bytes a value.
template <int SIZE> __device__ inline void store_piece(uint8_t *to, int64_t n, const u32x4 &v)
{
    if (n >= 16) {
        __builtin_memcpy(to, &v, 16);
    } else {
        uint8_t b[16];
        __builtin_memcpy(b, &v, 16);
#pragma unroll
        for (int x = 0; x < 16; x += SIZE)
            if (x < n) __builtin_memcpy(to + x, b + x, SIZE);
    }
}

__device__ inline u32x4 load_piece(const uint8_t *from, int64_t n)
{
    u32x4 v = {0, 0, 0, 0};
    if (n >= 16) {
        __builtin_memcpy(&v, from, 16);
    } else {
        uint8_t b[16] = {};
#pragma unroll
        for (int x = 0; x < 15; ++x)
            if (x < n) b[x] = from[x];
        __builtin_memcpy(&v, b, 16);
    }
    return v;
}

// Rows of an array in memory from (j, i) on, `left` of them, that a wave writes (or reads) in pieces of 16 bytes.  `whole`: all its
// columns are there, and the buffer's end keeps the rows apart that are not.
struct landing {
    uint8_t *base;
    int64_t left, bytes;                   // rows; bytes of a row
    uint32_t pitch;                        // bytes between rows
    bool whole, past;                      // past: stores go past the caches, which pays where they fill whole lines of memory
    __amdgpu_buffer_rsrc_t buffer;

    __device__ inline landing(const void *array, int64_t j, int64_t rows, int64_t pitch_, int64_t i, int64_t end, int width)
        : base((uint8_t *)array + j * pitch_ + i), left(rows - j), bytes(end - i), pitch((uint32_t)pitch_), whole(end - i >= width),
          past((pitch_ | (int64_t)(uintptr_t)base) % 64 == 0)
    {
        const int64_t all = left * pitch_ - i;
        buffer = __builtin_amdgcn_make_buffer_rsrc(base, 0, left <= 0 || all <= 0 ? 0 : all < 0x7ffffff0 ? (int)all : 0x7ffffff0, 0x00020000);
    }
    // What `room` holds, to row `first` on, byte `at` on.
    template <int SIZE, bool HALVES, class ROOM> __device__ inline void write(const ROOM &room, int first, int at, int lane) const
    {
        const int row = lane / ROOM::CHUNKS, chunk = lane % ROOM::CHUNKS;
        if (whole) {
            const uint32_t offset = (first + row) * pitch + at + chunk * 16;
            const auto rows = [&](auto hint) {
#pragma unroll
                for (int turn = 0; turn < ROOM::TURNS; ++turn) {
                    const int r = turn * ROOM::ROWS + row;
                    __builtin_amdgcn_raw_buffer_store_b128(HALVES ? room.get_halves(r, chunk) : room.get(r, chunk), buffer,
                                                           offset + turn * ROOM::ROWS * pitch, 0, decltype(hint)::value);
                }
            };
            if (past) rows(std::integral_constant<int, 2>{});
            else rows(std::integral_constant<int, 0>{});
        } else {
#pragma unroll 1
            for (int turn = 0; turn < ROOM::TURNS; ++turn) {
                const int r = turn * ROOM::ROWS + row;
                store_piece<SIZE>(base + (int64_t)(first + r) * pitch + at + chunk * 16, first + r < left ? bytes - at - chunk * 16 : 0,
                                  HALVES ? room.get_halves(r, chunk) : room.get(r, chunk));
            }
        }
    }
    template <class ROOM> __device__ inline void read(u32x4 (&to)[ROOM::TURNS], int first, int lane) const
    {
        const int row = lane / ROOM::CHUNKS, chunk = lane % ROOM::CHUNKS;
        if (whole) {
            const uint32_t offset = (first + row) * pitch + chunk * 16;
#pragma unroll
            for (int turn = 0; turn < ROOM::TURNS; ++turn)
                to[turn] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer, offset + turn * ROOM::ROWS * pitch, 0, 0));
        } else {
#pragma unroll
            for (int turn = 0; turn < ROOM::TURNS; ++turn) {
                const int r = first + turn * ROOM::ROWS + row;
                to[turn] = load_piece(base + (int64_t)r * pitch + chunk * 16, r < left ? bytes - chunk * 16 : 0);
            }
        }
    }
};

// The largest magnitude of the finite values among the 16 that a lane holds and the 16 of the other half's lane, as bits.
__device__ inline uint32_t group_magnitude(const f32x16 &v)
{
    float most = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) most = __builtin_fmaxf(most, __builtin_fabsf(v[r]));       // passes over NaN
    uint32_t amax = __float_as_uint(most);
    if (amax >= 0x7f800000u) {                                                              // an infinity: without it
        amax = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const uint32_t m = finite_magnitude(v[r]);
            amax = m > amax ? m : amax;
        }
    }
    const auto other = __builtin_amdgcn_permlane32_swap(amax, amax, false, false);
    return other[0] > other[1] ? other[0] : other[1];
}

// Codes of a group of 32 that two lanes hold of a row: 16 neighbours each.
__device__ inline u32x4 encode_group(const f32x16 &v, uint32_t byte)
{
    const float inverse = scale_inverse(byte);
    uint32_t w[4][1];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * q] * inverse, v[4 * q + 1] * inverse, 0, false);
        w[q][0] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * q + 2] * inverse, v[4 * q + 3] * inverse, lo, true);
    }
    join_runs(w);
    return u32x4{w[0][0], w[1][0], w[2][0], w[3][0]};
}

// And back.
__device__ inline f32x16 decode_group(const u32x4 &codes, uint32_t byte)
{
    uint32_t w[4] = {codes[0], codes[1], codes[2], codes[3]};
    split_runs(w);
    const float scale = scale_value(byte);
    f32x16 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w[q], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w[q], true);
        v[4 * q] = a[0] * scale, v[4 * q + 1] = a[1] * scale, v[4 * q + 2] = b[0] * scale, v[4 * q + 3] = b[1] * scale;
    }
    return v;
}

// The scale bytes of a row's next 16 groups, a register a four: read every 512 values of k.
struct scale_run {
    uint32_t w[4];
    __device__ inline void load(const uint8_t *p, int64_t n)
    {
        if (n >= 16) {
            __builtin_memcpy(w, p, 16);
        } else {
            uint8_t b[16] = {};
#pragma unroll
            for (int i = 0; i < 15; ++i)
                if (i < n) b[i] = p[i];
            __builtin_memcpy(w, b, 16);
        }
    }
    __device__ inline uint32_t byte(int i) const { return w[0] >> (8 * i) & 255u; }
    template <int N> __device__ inline void pass()               // over N of them
    {
        static_assert(N <= 4, "");
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t above = i < 3 ? w[i + 1] : 0u;
            w[i] = N == 4 ? above : __builtin_amdgcn_alignbyte(above, w[i], N);
        }
    }
};

// What becomes of D: rows of bfloat16; of float (of its part of k, `part` floats apart); gate and the other half packed, and
// their gated product; the gradient of those two from D and what is kept of them, and the same beside what its rounding leaves.
enum { TO_WIDE, TO_FULL, TO_GATED, TO_GATE_GRAD, TO_GATE_GRAD_FINE };

template <int TO> constexpr bool gate_grad() { return TO == TO_GATE_GRAD || TO == TO_GATE_GRAD_FINE; }

// Whether a block goes on to further tiles; where not, all of its shared memory is write()'s.
template <int TO> constexpr bool stays() { return !gate_grad<TO>(); }

struct result {
    void *out;
    int64_t stride, part;
    int64_t columns;                       // gated: of `out`
    int64_t low;                           // from a value of a fine gradient to what its rounding leaves
    uint8_t *gated_codes, *gated_scales, *kept_codes, *kept_scales;
};

// WI x WJ waves share TI x TJ of D.  Tiles: `across` of i, `along` of j, `parts` of depth_part values of k.  A block takes
// tile after tile (but for the gate's gradient), and its fetches run ahead of its products across their borders.
//
// A step is multiplied in turns of 16 values of k.  What a turn takes is read while the turn before is multiplied; the next
// step's fetches are started while the first turn's operands are on their way from shared memory.
//
// Where tiles are few, GROUPS of WI x WJ waves share one: each takes every GROUPS-th step, by itself but for the meetings, and
// their sums are added through shared memory at the end.  A wave alone on its unit spends two thirds of a step waiting.  A step of
// one block a compute unit still lasts as long as its fetch (1.6 us), hence DEPTH 3 there, where shared memory allows: two fetches under way.
// It gains nothing where two blocks a unit hide the fetch, nor for the large tiles (262144 x 512 -> 1024: 318 us, 301 with two).
template <int PKIND, int QKIND, int TO, int TI, int TJ, int WI, int WJ, int GROUPS, int DEPTH>
__global__ __launch_bounds__(WI * WJ * GROUPS * 64, WI * WJ * GROUPS > 4 ? 1 : 2) void k_product(operand P, operand Q, result R, uint32_t across, uint32_t along, uint32_t parts,
                                                                               int64_t depth_part)
{
    constexpr bool THROUGH = PKIND == CODES_ACROSS, STAYS = stays<TO>() && GROUPS == 1;
    constexpr int THREADS = WI * WJ * 64 /* of a group */, FI = TI / WI / 32, FJ = TJ / WJ / 32, STEP = 64, TURNS = STEP / 16;
    constexpr int PWIDE = THROUGH ? WIDE_ACROSS : PKIND;
    using ptile = tile<PWIDE, TI, STEP, THREADS>;
    using qtile = tile<QKIND, TJ, STEP, THREADS>;
    constexpr int TILES = ptile::BYTES + qtile::BYTES, AREA = 4096;            // a step's; what a wave's results go through
    constexpr int BUFFER = TILES > WI * WJ * AREA ? TILES : WI * WJ * AREA;
    static_assert(DEPTH == 2 || !THROUGH, "what goes through the registers is one step ahead");
    __shared__ __attribute__((aligned(1024))) uint8_t room[DEPTH * GROUPS * BUFFER];
    const int lane = threadIdx.x % 64, in_block = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int group = in_block / (WI * WJ), wave = in_block % (WI * WJ);
    lds_byte *const lds = (lds_byte *)room + group * (DEPTH * BUFFER);
    const int wi = wave % WI, wj = wave / WI;

    // Blocks go round the eight dies; each die has a run of neighbouring tiles, so that what they share comes from its cache.
    const uint32_t all = across * along * parts, die = blockIdx.x % 8, share = all / 8, more = all % 8;
    const uint32_t tiles_end = (die + 1) * share + (die < more ? die + 1 : more), stride = (gridDim.x - die + 7) / 8;
    const uint32_t tile_first = die * share + (die < more ? die : more) + blockIdx.x / 8;
    if (tile_first >= tiles_end) return;
    struct place {
        int64_t i, j, first, length;
        uint32_t part;
    };
    const auto place_of = [&](uint32_t tile) {
        place at;
        at.part = tile / (across * along);
        const uint32_t in = tile % (across * along);
        at.i = (int64_t)(in % across) * (TO == TO_GATED ? TI / 2 : TI), at.j = (int64_t)(in / across) * TJ;
        at.first = at.part * depth_part;
        at.length = P.depth - at.first < depth_part ? P.depth - at.first : depth_part;
        return at;
    };

    typename ptile::template stream<TO == TO_GATED ? 2 : 1, TI / WI> pstream;
    typename qtile::template stream<1, TJ> qstream;
    staged_codes<TI, STEP, THREADS> through;
    if constexpr (THROUGH) through.init(P, threadIdx.x % THREADS);
    else pstream.init(P, wave, lane);
    qstream.init(Q, wave, lane);

    // What is fetched next: k_left values of k, the groups' together, of tile `tile_ahead` (none: no tiles are left).
    uint32_t tile_ahead = tile_first;
    int64_t k_left = 0;
    const auto aim = [&] {
        const place at = place_of(tile_ahead);
        const int64_t first = at.first + group * STEP, last = at.first + at.length;
        if constexpr (THROUGH) through.aim(P, at.i, first, last, GROUPS);
        else pstream.aim(P, TO == TO_GATED ? R.columns : P.rows, at.i, first, last, R.columns * P.stride * 2, GROUPS);
        qstream.aim(Q, Q.rows, at.j, first, last, 0, GROUPS);
        k_left = at.length;
    };
    // The next step's fetch, made ready, in FETCHES pieces, and done.
    constexpr int FETCHES = THROUGH ? 1 + qtile::EACH : ptile::EACH + qtile::EACH;
    static_assert(FETCHES < 16, "counted by four bits");
    const auto ready = [&] {
        if constexpr (!THROUGH) pstream.ready(k_left - group * STEP, wave, lane);
        qstream.ready(k_left - group * STEP, wave, lane);
    };
    const auto fetch = [&](int piece, int to) {
        constexpr int OF_P = THROUGH ? 1 : ptile::EACH;
        if (piece >= OF_P) {
            qstream.fetch(piece - OF_P, wave, lds + to + ptile::BYTES);
        } else {
            if constexpr (THROUGH) through.fetch();
            else pstream.fetch(piece, wave, lds + to);
        }
    };
    const auto fetched = [&] {
        k_left -= GROUPS * STEP;
        if (k_left <= 0) {
            tile_ahead += stride;
            k_left = 0;
            if (STAYS && tile_ahead < tiles_end) aim();
        }
    };
    aim();

    f32x16 acc[FI][FJ];
    scale_run bytes[FJ];
    const auto scales_of = [&](int64_t j, int64_t g) {
        if constexpr (QKIND == CODES_ALONG) {
#pragma unroll
            for (int t = 0; t < FJ; ++t) {
                const int64_t row = j + (wj * FJ + t) * 32 + lane % 32;
                bytes[t].load(Q.scales + (row < Q.rows ? row : Q.rows - 1) * Q.groups + g, Q.groups - g);
            }
        }
    };
    const auto clear = [&] {
#pragma unroll
        for (int f = 0; f < FI; ++f)
#pragma unroll
            for (int t = 0; t < FJ; ++t) acc[f][t] = f32x16{};
    };
    bf16x8 p[2][FI], q[2][FJ];
    u32x4 codes[FJ];
    const auto read = [&](int turn, int at) {
        const int run = turn / 2, s = turn % 2;
#pragma unroll
        for (int f = 0; f < FI; ++f) p[s][f] = ptile::read(lds + at, (wi * FI + f) * 32, run, s, lane);
#pragma unroll
        for (int t = 0; t < FJ; ++t) {
            const int first = (wj * FJ + t) * 32;
            if constexpr (QKIND == CODES_ALONG) {
                if (s == 0) codes[t] = qtile::read_codes(lds + at + ptile::BYTES, first, run, lane);
                q[s][t] = qtile::widen(codes[t][2 * s], codes[t][2 * s + 1], __uint_as_float(bytes[t].byte(run) << 23));
            } else {
                q[s][t] = qtile::read(lds + at + ptile::BYTES, first, run, s, lane);
            }
        }
    };
    // A tile's results, through the buffer that was multiplied last.  A wave's: rows j_wave .. , columns i_wave .. .
    const auto write = [&](const place &of, lds_byte *area) {
        const int64_t j_wave = of.j + wj * FJ * 32, i_wave = of.i + wi * (TO == TO_GATED ? FI / 2 : FI) * 32, groups = groups_of(R.columns);
        area += wave * (gate_grad<TO>() ? FI * 4096 : AREA);
        // addresses are formed here: worked out ahead of the tiles they would take registers from the products
        int lane = threadIdx.x % 64;
        asm volatile("" : "+v"(lane));
        const int half = lane / 32;
        if constexpr (TO == TO_WIDE || TO == TO_FULL) {
            using room = exchange<128>;                              // 64 values of 16 bits, or 32 of 32
            constexpr int SIZE = TO == TO_WIDE ? 2 : 4, AT_ONCE = 4 / SIZE;
            const room x{area};
            landing to((uint8_t *)R.out + (TO == TO_FULL ? of.part * R.part * SIZE : 0), j_wave, Q.rows, R.stride * SIZE, i_wave * SIZE,
                       P.rows * SIZE, FI * 32 * SIZE);
            if (parts > 1 || (TO == TO_FULL && Q.rows * R.stride * SIZE <= READ_NEXT)) to.past = false;      // they are read again at once
#pragma unroll
            for (int t = 0; t < FJ; ++t)
#pragma unroll
                for (int f0 = 0; f0 < FI; f0 += AT_ONCE) {
#pragma unroll
                    for (int f = 0; f < AT_ONCE; ++f) {
                        const f32x16 &v = acc[f0 + f][t];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            if constexpr (TO == TO_WIDE) {
                                x.put_half(lane % 32, f * 4 + q, half, two_bf16(v[4 * q], v[4 * q + 1]), two_bf16(v[4 * q + 2], v[4 * q + 3]));
                            } else {
                                x.put(lane % 32, f * 8 + q * 2 + half, u32x4{__float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]),
                                                                            __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3])});
                            }
                        }
                    }
                    x.turn();
                    to.template write<SIZE, TO == TO_WIDE>(x, t * 32, f0 * 32 * SIZE, lane);
                    x.turn();
                    __builtin_amdgcn_sched_barrier(0);
                }
        } else if constexpr (TO == TO_GATED) {
            using room = exchange<FI * 16>;                          // FI / 2 * 32 codes
            constexpr int COLUMNS = FI / 2 * 32, ARRAY = 32 * FI * 16;
            const landing gated(R.gated_codes, j_wave, Q.rows, R.columns, i_wave, R.columns, COLUMNS);
            const landing kept_g(R.kept_codes, j_wave, Q.rows, 2 * R.columns, i_wave, R.columns, COLUMNS);
            const landing kept_p(R.kept_codes, j_wave, Q.rows, 2 * R.columns, R.columns + i_wave, 2 * R.columns, COLUMNS);
            static_assert(2 * ARRAY <= AREA, "two arrays of a group of rows at a time");
#pragma unroll
            for (int t = 0; t < FJ; ++t) {
                const int64_t j = j_wave + t * 32 + lane % 32, g0 = i_wave / GROUP;
                // columns beyond the end hold zeros: their rows of the weight read as such
                const auto pack = [&](const f32x16 &v, int f, int slot, uint8_t *scales, bool mine) {
                    const uint32_t byte = scale_byte(group_magnitude(v));
                    room{area + slot * ARRAY}.put(lane % 32, f * 2 + half, encode_group(v, byte));
                    if (mine && j < Q.rows && g0 + f < groups) scales[g0 + f] = (uint8_t)byte;
                };
#pragma unroll
                for (int f = 0; f < FI / 2; ++f) {
                    const f32x16 &g = acc[f][t], &p = acc[f + FI / 2][t];
                    f32x16 a;
#pragma unroll
                    for (int x = 0; x < 16; ++x) a[x] = g[x] * sigmoid(g[x]) * p[x];
                    pack(a, f, 0, R.gated_scales + j * groups, half == 0);
                    if (R.kept_codes) pack(g, f, 1, R.kept_scales + 2 * j * groups, half == 1);
                }
                room::turn();
                gated.template write<1, false>(room{area}, t * 32, 0, lane);
                if (R.kept_codes) {
                    kept_g.template write<1, false>(room{area + ARRAY}, t * 32, 0, lane);
                    room::turn();
#pragma unroll
                    for (int f = 0; f < FI / 2; ++f) pack(acc[f + FI / 2][t], f, 0, R.kept_scales + (2 * j + 1) * groups, half == 0);
                    room::turn();
                    kept_p.template write<1, false>(room{area}, t * 32, 0, lane);
                }
                room::turn();
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            using room = exchange<FI * 32>;                          // FI * 32 codes of each half
            using wide = exchange<FI * 64>;
            constexpr int ARRAY = 32 * FI * 32;
            const landing kept_g(R.kept_codes, j_wave, Q.rows, 2 * R.columns, i_wave, R.columns, FI * 32);
            const landing kept_p(R.kept_codes, j_wave, Q.rows, 2 * R.columns, R.columns + i_wave, 2 * R.columns, FI * 32);
            landing to_g(R.out, j_wave, Q.rows, 2 * R.stride, 2 * i_wave, 2 * R.columns, FI * 64);
            landing to_p(R.out, j_wave, Q.rows, 2 * R.stride, 2 * (R.columns + i_wave), 4 * R.columns, FI * 64);
            constexpr bool FINE = TO == TO_GATE_GRAD_FINE;
            landing rest_g(R.out, j_wave, Q.rows, 2 * R.stride, 2 * (R.low + i_wave), 2 * (R.low + R.columns), FI * 64);
            landing rest_p(R.out, j_wave, Q.rows, 2 * R.stride, 2 * (R.low + R.columns + i_wave), 2 * (R.low + 2 * R.columns), FI * 64);
            if (Q.rows * R.stride * 2 <= READ_NEXT) to_g.past = to_p.past = rest_g.past = rest_p.past = false;
            u32x4 raw[2][room::TURNS];
            uint32_t bytes_of[2];                                    // a byte a group: at most four
            const auto load = [&](int t) {
                kept_g.template read<room>(raw[0], t * 32, lane);
                kept_p.template read<room>(raw[1], t * 32, lane);
                const int64_t j = j_wave + t * 32 + lane % 32, g0 = i_wave / GROUP, n = j < Q.rows ? groups - g0 : 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint8_t *from = R.kept_scales + (2 * j + h) * groups + g0;
                    bytes_of[h] = 0;
                    if (n >= FI) {
                        __builtin_memcpy(&bytes_of[h], from, FI);
                    } else {
#pragma unroll
                        for (int f = 0; f < FI - 1; ++f)
                            if (f < n) bytes_of[h] |= (uint32_t)from[f] << (8 * f);
                    }
                }
            };
            load(0);
#pragma unroll
            for (int t = 0; t < FJ; ++t) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int turn = 0; turn < room::TURNS; ++turn)
                        room{area + h * ARRAY}.put(turn * room::ROWS + lane / room::CHUNKS, lane % room::CHUNKS, raw[h][turn]);
                const uint32_t bytes_now[2] = {bytes_of[0], bytes_of[1]};
                room::turn();
                __builtin_amdgcn_sched_barrier(0);
                if (t + 1 < FJ) load(t + 1);
                const wide x{area + 2 * ARRAY};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    [[maybe_unused]] f32x16 rest[FINE ? FI : 1];
#pragma unroll
                    for (int f = 0; f < FI; ++f) {
                        f32x16 v = acc[f][t];                        // the other half's gradient waits in acc
                        if (h == 0) {
                            const f32x16 g = decode_group(room{area}.get(lane % 32, f * 2 + half), bytes_now[0] >> (8 * f) & 255u);
                            const f32x16 p = decode_group(room{area + ARRAY}.get(lane % 32, f * 2 + half), bytes_now[1] >> (8 * f) & 255u);
#pragma unroll
                            for (int x = 0; x < 16; ++x) {
                                const float s = sigmoid(g[x]), ds = v[x] * s;
                                acc[f][t][x] = ds * g[x];
                                v[x] = ds * p[x] * (1.0f + g[x] * (1.0f - s));
                            }
                        }
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            x.put_half(lane % 32, f * 4 + q, half, two_bf16(v[4 * q], v[4 * q + 1]), two_bf16(v[4 * q + 2], v[4 * q + 3]));
                        if constexpr (FINE) {
#pragma unroll
                            for (int y = 0; y < 16; ++y) rest[f][y] = rest_of_bf16(v[y]);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    x.turn();
                    (h ? to_p : to_g).template write<2, true>(x, t * 32, 0, lane);
                    x.turn();
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (FINE) {
#pragma unroll
                        for (int f = 0; f < FI; ++f)
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                x.put_half(lane % 32, f * 4 + q, half, two_bf16(rest[f][4 * q], rest[f][4 * q + 1]),
                                           two_bf16(rest[f][4 * q + 2], rest[f][4 * q + 3]));
                        x.turn();
                        (h ? rest_p : rest_g).template write<2, true>(x, t * 32, 0, lane);
                        x.turn();
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        }
    };

    const auto after = [](uint32_t at) { return at + BUFFER == DEPTH * BUFFER ? 0u : at + BUFFER; };
    int under_way = 0;                               // steps fetched and not multiplied
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d) {
        const bool more_of_it = k_left > 0;
        ready();                                     // (of nothing, where no step is left: it is not fetched)
        if (more_of_it) {
#pragma unroll
            for (int e = 0; e < FETCHES; ++e) fetch(e, d * BUFFER);
            fetched();
            ++under_way;
        }
    }
    if constexpr (THROUGH) through.store(lds);
    place now = place_of(tile_first);
    constexpr int SCALES = GROUPS * STEP / GROUP;    // of a row, from one of a group's steps to its next
    scales_of(now.j, now.first / GROUP + group * (STEP / GROUP));
    for (uint32_t tile = tile_first, at = 0;;) {
        clear();
        for (int64_t k = 0; k < now.length; k += GROUPS * STEP, at = after(at)) {
            // What this wave fetched and stored for this step has arrived (lgkmcnt(0), and vmcnt(0) or as many as a later step's
            // fetches are: loads arrive in order, and whatever else is under way was started after this step's).
            if (DEPTH > 2 && under_way > 1) __builtin_amdgcn_s_waitcnt(0x0070 | FETCHES);
            else __builtin_amdgcn_s_waitcnt(0x0070);
            __syncthreads();
            const bool ahead = k_left > 0;           // the buffer before this one, which every wave is done with, takes the next tiles
            const int other = DEPTH == 2 ? after(at) : after(after(at));
            --under_way;
            read(0, at);
            if (ahead) ready();
            __builtin_amdgcn_sched_barrier(0);
            if (ahead) {
#pragma unroll
                for (int e = 0; e < FETCHES; ++e) fetch(e, other);
            }
#pragma unroll
            for (int turn = 0; turn < TURNS; ++turn) {
                if (turn + 1 < TURNS) read(turn + 1, at);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int f = 0; f < FI; ++f)
#pragma unroll
                    for (int t = 0; t < FJ; ++t) acc[f][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p[turn % 2][f], q[turn % 2][t], acc[f][t], 0, 0, 0);
            }
            if (ahead) {
                fetched();
                ++under_way;
                if constexpr (THROUGH) through.store(lds + other);
            }
            if constexpr (QKIND == CODES_ALONG) {
                const int64_t g = (now.first + k + GROUPS * STEP) / GROUP;
                if (k + GROUPS * STEP < now.length) {
                    if (g % 16 == 0) scales_of(now.j, g + group * (STEP / GROUP));
                    else {
#pragma unroll
                        for (int t = 0; t < FJ; ++t) bytes[t].template pass<SCALES>();
                    }
                }
            }
        }
        const place done = now;
        tile += stride;
        const bool on = STAYS && tile < tiles_end;
        if (on) {
            now = place_of(tile);
            scales_of(now.j, now.first / GROUP);
        }
        __syncthreads();
        if constexpr (GROUPS > 1) {
            // a fragment's 16 sums of a lane beside those of its neighbours
            static_assert(GROUPS * FI * FJ * 4096 * WI * WJ <= DEPTH * GROUPS * BUFFER, "the groups' sums fit");
            typedef float f32x4 __attribute__((ext_vector_type(4)));
            const auto sums = [&](int g, int f, int t, int q) {
                return (__attribute__((address_space(3))) f32x4 *)((lds_byte *)room + ((((g * WI * WJ + wave) * FI + f) * FJ + t) * 4 + q) * 1024 + lane * 16);
            };
#pragma unroll
            for (int f = 0; f < FI; ++f)
#pragma unroll
                for (int t = 0; t < FJ; ++t)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (group > 0) *sums(group - 1, f, t, q) = f32x4{acc[f][t][4 * q], acc[f][t][4 * q + 1], acc[f][t][4 * q + 2], acc[f][t][4 * q + 3]};
            __syncthreads();
            if (group > 0) return;
#pragma unroll
            for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
                for (int f = 0; f < FI; ++f)
#pragma unroll
                    for (int t = 0; t < FJ; ++t)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const f32x4 v = *sums(g, f, t, q);
#pragma unroll
                            for (int x = 0; x < 4; ++x) acc[f][t][4 * q + x] += v[x];
                        }
        }
        write(done, STAYS ? lds + (at == 0 ? DEPTH - 1 : at / BUFFER - 1) * BUFFER : lds + (GROUPS - 1) * (FI * FJ * 4096 * WI * WJ));
        if (!on) break;
    }
}

}  // namespace act
