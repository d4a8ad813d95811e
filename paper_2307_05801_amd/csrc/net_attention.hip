// Attention, forward: o = sum over keys of exp(x) v / sum of exp(x), x = scale q.k + bias, in one pass over the keys.
//
// A block has 128 queries of a head, 32 to a wave, whose values stay in registers; it walks over the keys in tiles of 64, which all four waves
// read from shared memory.  A wave forms x for 32 keys by 32 queries with a lane a query (net_attention.h says why), keeps the largest so far, m, and
// the sum of exp2(x - m) of each query in that lane, and multiplies the values summed so far by exp2(m before - m now) where m has grown.  m follows the largest only when a
// query's has got 2^8 ahead of it: sums of exp2 up to 2^8 are as good, and one of 32 queries has a new largest in nearly every tile.
//
// What bounds it: at width 64 the vector instructions (with a table 12 to 16 a pair, counted; 512 windows of 512 patches, 8 heads, kept for a backward pass: 1.05 ms, 262 TFLOP/s, twice as many flops with
// the probabilities' other two parts), at width 128 those (8 a pair) and the matrix instructions about alike (32768 patches, 8 heads: 6.0 ms, 730 TFLOP/s, half as many flops again with the second part).
// Three blocks share a compute unit at width 64 (the windows, with probabilities in two parts: 0.95 ms, with two blocks 1.16).
#include "net_attention.h"

namespace {

using namespace net;

// Numbers of a line in shared memory for a tile's pairs: 191 are enough for rows one after the other, a few hundred on a grid, and 1500 where a tile has the end of one plane
// of 27 x 22 patches and the next one's beginning.  As many as leave a compute unit room for two blocks.
constexpr int window_of_tile(int deep) { return deep > 64 ? 1024 : 2048; }

struct forward_args {
    attention_args a;
    uint16_t *o;
    float *stats;                          // [item][head][query][2], or null
    uint16_t *rest;                        // what o's rounding leaves
    // Where queries are few: so many of a block's waves are heads that share keys, not more queries; the keys go to `parts` blocks, `length` of them each (whole
    // tiles), whose sums (of a query [parts][width], and [parts][2]: m and the sum of exp2) k_join puts together.
    int32_t abreast, parts, length;
    float *part_sums, *part_stats;
    int64_t first;                         // block of this launch of k_join
};

// What rounding v to bfloat16 leaves, as it is kept: the difference of the two numbers' bits, of 16 bits and a sign, whatever v's size.  (2^15 is one where v lies just
// between two and the lower is taken; one less than that is a unit of 32 bits off.)
__device__ inline uint16_t rest_of(float v)
{
    const int rest = (int)(__float_as_uint(v) - ((uint32_t)element<LEAP_BF16>::from_float(v) << 16));
    return finite_magnitude(v) ? (uint16_t)(rest < 0x7fff ? rest : 0x7fff) : 0;
}

// The second of a query's statistics where there is no table: exponents are lowered by it too, in every tile of k_grad_key.
__device__ inline float log_of(float sum) { return sum != 0.0f ? __builtin_amdgcn_logf(sum) : INFINITY; }

// BIAS: with a table.  FINE: for a backward pass, which takes delta = grad.o off every product grad.v of a query: an o with its rounding, or with the probabilities',
// would spoil all of the query's alike, and in grad_q that adds up along what the keys have in common (keys and values with a common part as large as what
// differs, 512 keys: grad_q was 0.020 of its norm off, with four times as large a part 0.34; now 0.003 and 0.007, which is the rounding of ds).  So there the
// probabilities are the sum of two bfloat16, and o's other 16 bits are kept.  With a table they are the sum of three, their 24 bits: its gradient is 32 bits, and what delta lacks is in every pair of a
// query, which a bucket that has most of them adds up (of two, from 8 patches to 5397, the gradient is 0.4e-6 to 6e-6 of its norm off, of three 1.4e-7 to 1.3e-6, all in 32 bits 1.4e-7 to 1.2e-6; the forward
// pass of 512 windows 0.95 ms, with three 1.04).  Otherwise they are rounded to bfloat16 once: o is 0.0022 to 0.0024 of its norm off, 0.0017 of it by its own rounding (of two parts
// 32768 patches, 8 heads of 128, take 5.5 instead of 4.1 ms, 2 x 16 queries over 262144 keys 89 instead of 74 us).
template <int DEEP, bool DIRECT, bool BIAS, bool FINE> __global__ __launch_bounds__(BLOCK, DEEP > 64 || !DIRECT ? 2 : 3) void k_attention(forward_args F)
{
    using tile = rows_tile<DEEP>;
    constexpr int STEPS = DEEP / 16, BLOCKS = DEEP / 32, WINDOW = window_of_tile(DEEP), PARTS = !FINE ? 1 : BIAS ? 3 : 2;
    const attention_args &A = F.a;
    __shared__ __attribute__((aligned(16))) uint8_t room[4 * tile::BYTES + (BIAS ? 2 * WINDOW * 4 : 0)];
    __shared__ int places[BIAS ? 2 : 1][TILE];
    lds_byte *const lds = (lds_byte *)room;
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int cols = COLS / F.abreast, tiles = (A.queries + cols - 1) / cols, across = A.heads / F.abreast;
    int64_t unit = unit_of(blockIdx.x, gridDim.x);
    const int part = uniform((int)(unit % F.parts));
    unit /= F.parts;
    const int64_t item = uniform((int)(unit / tiles / across));
    const int head = uniform((int)(unit / tiles % across) * F.abreast + wave % F.abreast), kv_head = uniform(head / (A.heads / A.kv_heads));
    const int query0 = uniform((int)(unit % tiles) * cols), query = query0 + uniform(wave / F.abreast) * 32 + lane % 32;
    const bool there = query < A.queries;
    source<DEEP, DIRECT> k(A.k.data + item * A.k.item + kv_head * A.k.head, A.k.row, A.keys, A.width, wave, lane);
    source<DEEP, DIRECT> v(A.v.data + item * A.v.item + kv_head * A.v.head, A.v.row, A.keys, A.width, wave, lane);

    bf16x8 q[STEPS];
    load_side<STEPS>(q, A.q.data + item * A.q.item + head * A.q.head + query * A.q.row, A.width, there, lane);
    const float *const line = BIAS ? A.lines + (int64_t)head * A.line : nullptr;
    const int position = BIAS ? query_position(A, there ? query : A.queries - 1) : 0;
    place_range mine;
    if constexpr (BIAS) mine = both(A.query_places[query0 / TILE], A.query_places[query0 + TILE < A.queries ? query0 / TILE + 1 : query0 / TILE]);
    const float scale = A.scale * LOG2E;
    f32x16 o[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) o[b] = zeros();
    float m = -INFINITY, sum = 0.0f;

    const int64_t end = (int64_t)(part + 1) * F.length;
    key_walk at(A.mask ? A.mask + item * A.mask_item : nullptr, (int64_t)part * F.length, end < A.keys ? end : A.keys, lane);
    const bool idle = !__any(there);                   // a wave without queries brings tiles alone
    line_window window, coming;
    bool fours = false, coming_fours = false;
    int place = 0;
    const auto fetch = [&](int to) {                   // the walk's tile
        lds_byte *const kt = lds + to * 2 * tile::BYTES;
        k.fetch(at.first, at.bits, kt, wave, lane);
        v.fetch(at.first, at.bits, kt + tile::BYTES, wave, lane);
        if constexpr (BIAS) {
            const place_range keys = A.key_places[at.first / TILE];
            coming = window_of(A, keys, mine, WINDOW), coming_fours = keys.fours;
            if (coming.inside) fetch_window<4>(line, A.offsets, coming, lds + 4 * tile::BYTES + to * WINDOW * 4, wave, lane);
            if (wave == 0) place = key_position(A, at.first + lane < A.keys ? (int)at.first + lane : A.keys - 1);
        }
    };
    if (!at.done()) fetch(0);
    // A tile; which of the two pairs it lies in is a constant, so that addresses in shared memory are.
    const auto one = [&](auto which) {
        constexpr int turn = decltype(which)::value;
        lds_byte *const kt = lds + turn * 2 * tile::BYTES, *const vt = kt + tile::BYTES;
        const uint64_t bits = at.bits;
        k.land(kt), v.land(vt);
        if constexpr (BIAS) {
            if (wave == 0) places[turn][lane] = place;
            window = coming, fours = coming_fours;
        }
        if constexpr (DIRECT || BIAS) fetched();
        __syncthreads();                               // two pairs of tiles: the one written next was read before this
        at.next(lane);
        if (!at.done()) fetch(turn ^ 1);
        if (idle) return;

        f32x16 x[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            x[h] = zeros();
#pragma unroll
            for (int s = 0; s < STEPS; ++s) x[h] = product(tile::along(kt, h * 32, s, lane), q[s], x[h]);
        }
        if constexpr (BIAS) {
            const uint32_t from = origin_of(lds + 4 * tile::BYTES + turn * WINDOW * 4, A, window, position, false);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (window.inside)
                    over_places<1, const float>(places[turn] + h * 32, fours, from, lane, [&](int r, auto number) { x[h][r] = __builtin_fmaf(x[h][r], scale, *number); });
                else
#pragma unroll
                    for (int r = 0; r < 16; ++r) x[h][r] = __builtin_fmaf(x[h][r], scale, line[line_at(A, places[turn][h * 32 + row_of(r) + lane / 32 * 4], position)]);
        }
        if (~bits) {
            seldom();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t held = (uint32_t)(bits >> (h * 32)) >> (lane / 32 * 4);
#pragma unroll
                for (int r = 0; r < 16; ++r) x[h][r] = held >> row_of(r) & 1 ? x[h][r] : -INFINITY;
            }
        }
        float most = x[0][0];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, x[h][r]);
        most = column_max(most);
        const float now = fmaxf(m, BIAS ? most : most * scale);
        if (__any(now > m + 8.0f)) {                   // (the first keys of a query among them: m is -inf before)
            const float by = now == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - now);
            sum *= by;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) o[b] *= by;
            m = now;
        }
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[h][r] = __builtin_amdgcn_exp2f(BIAS ? x[h][r] - base : __builtin_fmaf(x[h][r], scale, -base));
                sum += x[h][r];
            }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                bf16x8 p[PARTS];
                parts_of_eight(x[h], t, p);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    const bf16x8 values = tile::across(vt, h * 32 + t * 16, b, lane);
#pragma unroll
                    for (int i = 0; i < PARTS; ++i) o[b] = product(values, p[i], o[b]);
                }
            }
    };
    while (!at.done()) {
        one(std::integral_constant<int, 0>{});
        if (at.done()) break;
        one(std::integral_constant<int, 1>{});
    }
    sum = column_sum(sum);
    if (F.parts > 1) {
        if (!there) return;
        const int64_t row = ((item * A.heads + head) * (int64_t)A.queries + query) * F.parts + part;
        if (lane < 32) F.part_stats[row * 2] = m, F.part_stats[row * 2 + 1] = sum;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int at = b * 32 + row_of(r) + lane / 32 * 4;
                if (at < A.width) F.part_sums[row * A.width + at] = o[b][r];
            }
        return;
    }
    const float by = sum != 0.0f ? 1.0f / sum : 0.0f;                 // (a sum that is not a number: so is o)
    const int64_t row = (item * A.queries + query) * A.heads + head;
    store_column<BLOCKS>(F.o + row * A.width, A.width, o, by, lane, there);
    if (FINE && there && lane < 32) {
        float *const to = F.stats + ((item * A.heads + head) * (int64_t)A.queries + query) * 2;
        to[0] = sum != 0.0f ? m : 0.0f, to[1] = BIAS ? sum : log_of(sum);
    }
    if constexpr (FINE) {
        if (there)
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = b * 32 + row_of(r) + lane / 32 * 4;
                    if (at < A.width) F.rest[row * A.width + at] = rest_of(o[b][r] * by);
                }
    }
}

// A query of a head from its parts, a block each: every wave adds up a fourth of them.
__global__ __launch_bounds__(BLOCK) void k_join(forward_args F)
{
    const attention_args &A = F.a;
    __shared__ float values[WAVES][LEAP_ATTENTION_WIDEST], sums[WAVES];
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    const int64_t row = F.first + blockIdx.x;                                              // (item, head, query)
    const float *const stats = F.part_stats + row * F.parts * 2, *const from = F.part_sums + row * F.parts * A.width;
    float m = -INFINITY;
    for (int p = lane; p < F.parts; p += WAVE) m = fmaxf(m, stats[p * 2]);
#pragma unroll
    for (int d = 1; d < WAVE; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    const float base = m == -INFINITY ? 0.0f : m;
    float sum = 0.0f, o[2] = {};
#pragma unroll 8
    for (int p = wave; p < F.parts; p += WAVES) {
        const float by = __builtin_amdgcn_exp2f(stats[p * 2] - base);
        sum += stats[p * 2 + 1] * by;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (lane + i * WAVE < A.width) o[i] += from[(int64_t)p * A.width + lane + i * WAVE] * by;
    }
    values[wave][lane] = o[0], values[wave][lane + WAVE] = o[1];
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = sums[0] + sums[1] + sums[2] + sums[3];
    const float by = sum != 0.0f ? 1.0f / sum : 0.0f;
    const int64_t query = row % A.queries, head = row / A.queries % A.heads, item = row / A.queries / A.heads, to = (item * A.queries + query) * A.heads + head;
    if (const int at = threadIdx.x; at < A.width) {
        const float v = (values[0][at] + values[1][at] + values[2][at] + values[3][at]) * by;
        F.o[to * A.width + at] = element<LEAP_BF16>::from_float(v);
        if (F.rest) F.rest[to * A.width + at] = rest_of(v);
    }
    if (F.stats && threadIdx.x == 0) F.stats[row * 2] = base, F.stats[row * 2 + 1] = A.table ? sum : log_of(sum);
}

// Rows of `width` to rows of whole 16 bytes, a piece a thread.
__global__ __launch_bounds__(BLOCK) void k_lay_rows(rows_of from, int rows, int heads, int width, int64_t pieces, int64_t first, uint8_t *to)
{
    const int each = (width + 7) / 8;
    const int64_t id = (first + blockIdx.x) * BLOCK + threadIdx.x;
    if (id >= pieces) return;
    const int64_t row = id / each, head = row % heads, at = row / heads % rows, item = row / heads / rows;
    const u32x4 v = row_piece(from.data + item * from.item + at * from.row + head * from.head, width, (int)(id % each));
    __builtin_memcpy(to + id * 16, &v, 16);
}

// A head's number for every difference of positions; and what positions each tile of queries and of keys has.
__global__ __launch_bounds__(BLOCK) void k_lines(attention_args A)
{
    const int64_t id = (int64_t)blockIdx.x * BLOCK + threadIdx.x;
    if ((int)blockIdx.y < A.heads) {
        if (id < A.offsets) {
            const int bucket = bucket_at(A, id);
            A.lines[(int64_t)blockIdx.y * A.line + id] = table_value(A, blockIdx.y, bucket);
            if (blockIdx.y == 0) {
                A.line_buckets[id] = (uint16_t)bucket;
                const bool rising = __all(id + 1 >= A.offsets || bucket_at(A, id + 1) > bucket);
                if (id % WAVE == 0) A.line_rising[id / WAVE] = rising;
            }
        }
        return;
    }
    const int64_t query_tiles = (A.queries + TILE - 1) / TILE, key_tiles = (A.keys + TILE - 1) / TILE, tile = id / WAVE;
    if (tile >= query_tiles + key_tiles) return;
    const bool keys = tile >= query_tiles;
    const int lane = threadIdx.x % WAVE, first = (int)(keys ? tile - query_tiles : tile) * TILE, rows = keys ? A.keys : A.queries, row = first + lane < rows ? first + lane : rows - 1;
    const int place = keys ? key_position(A, row) : query_position(A, row);
    int low = place, high = place;
#pragma unroll
    for (int d = 1; d < WAVE; d *= 2) {
        const int a = __shfl_xor(low, d), b = __shfl_xor(high, d);
        low = a < low ? a : low, high = b > high ? b : high;
    }
    const int begin = __shfl(place, lane / 4 * 4);
    const bool fours = __all(place == begin + lane % 4);               // (not so where the rows end: what there is not has the last one's place)
    const bool rising = __all(place > __shfl_up(place, 1) || lane == 0 || first + lane >= rows);
    if (lane == 0) (keys ? A.key_places : A.query_places)[keys ? tile - query_tiles : tile] = {low, high, fours, rising};
}

}  // namespace

namespace net {

bool direct_array(const void *p, int64_t item, int64_t row, int64_t head, int64_t width)
{
    return width % 8 == 0 && (uintptr_t)p % 16 == 0 && item % 8 == 0 && row % 8 == 0 && head % 8 == 0 && row < (int64_t)1 << 24;
}

int64_t laid_out_bytes(int64_t items, int64_t rows, int64_t heads, int64_t width) { return width % 8 ? items * rows * heads * ((width + 7) / 8) * 16 : 0; }

int lay_out(rows_of &array, int64_t items, int64_t rows, int64_t heads, int64_t width, void *to, hipStream_t st)
{
    const int64_t pieces = items * rows * heads * ((width + 7) / 8), row = (width + 7) / 8 * 8;
    const int rc = over_blocks((pieces + BLOCK - 1) / BLOCK, [&](int64_t first, unsigned n) {
        hipLaunchKernelGGL(k_lay_rows, dim3(n), dim3(BLOCK), 0, st, array, (int)rows, (int)heads, (int)width, pieces, first, (uint8_t *)to);
    });
    array = {(const uint16_t *)to, rows * heads * row, heads * row, row};
    return rc;
}

static int64_t line_length(int64_t offsets) { return (offsets + 7) / 8 * 8; }
static int64_t rising_bytes(int64_t offsets) { return (offsets + WAVE * 16 - 1) / (WAVE * 16) * 16; }
static int64_t tiles_of(int64_t rows) { return (rows + TILE - 1) / TILE; }

int64_t lines_bytes(const leap_attention_desc *d)
{
    if (!d->d_table) return 0;
    return d->heads * line_length(d->offsets) * 4 + line_length(d->offsets) * 2 + rising_bytes(d->offsets) + (tiles_of(d->queries) + tiles_of(d->keys)) * (int64_t)sizeof(place_range);
}

int write_lines(attention_args &A, void *work, hipStream_t st)
{
    const int64_t length = line_length(A.offsets), tiles = tiles_of(A.queries) + tiles_of(A.keys);
    A.line = (int32_t)length;
    A.lines = (float *)work;
    A.line_buckets = (uint16_t *)(A.lines + A.heads * length);
    A.line_rising = (uint8_t *)(A.line_buckets + length);
    A.query_places = (place_range *)(A.line_rising + rising_bytes(A.offsets));
    A.key_places = A.query_places + tiles_of(A.queries);
    const int64_t threads = A.offsets > tiles * WAVE ? A.offsets : tiles * WAVE;
    hipLaunchKernelGGL(k_lines, dim3((unsigned)((threads + BLOCK - 1) / BLOCK), (unsigned)(A.heads + 1)), dim3(BLOCK), 0, st, A);
    return launched();
}

const char *bad_array(int64_t items, int64_t item, int64_t rows, int64_t row, int64_t heads, int64_t head)
{
    const int64_t most = (int64_t)1 << 58;
    if (item < 0 || row < 0 || head < 0 || item > most / (items + 1) || row > most / (rows + 1) || head > most / (heads + 1)) return "a stride is negative or reaches beyond what addresses hold";
    return nullptr;
}

const char *bad_attention(const leap_attention_desc *d)
{
    const int64_t most = (int64_t)1 << 30;
    if (!d) return "null description";
    if (d->batch < 0 || d->queries < 0 || d->keys < 0) return "sizes must not be negative";
    if (d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads) return "heads must be a multiple of the heads of keys";
    if (d->width < 1 || d->width > LEAP_ATTENTION_WIDEST) return "rows of 1 to 128 values";
    if (d->queries > most || d->keys > most || d->heads > 65536 || d->batch > most || d->batch * d->heads > most) return "more than 2^30 queries, keys or heads of items";
    if (!(d->scale > 0.0f) || d->scale > 1e30f) return "the scale must be positive";
    const char *why = bad_array(d->batch, d->q_item, d->queries, d->q_row, d->heads, d->q_head);
    if (!why) why = bad_array(d->batch, d->k_item, d->keys, d->k_row, d->kv_heads, d->k_head);
    if (!why) why = bad_array(d->batch, d->v_item, d->keys, d->v_row, d->kv_heads, d->v_head);
    if (why) return why;
    if (d->d_mask && (d->mask_item < 0 || d->mask_item > ((int64_t)1 << 58) / (d->batch + 1))) return "a stride is negative or reaches beyond what addresses hold";
    if (d->d_table) {
        if (!known_type(d->table_type)) return "unknown element type";
        if (d->buckets < 1 || d->buckets > LEAP_ATTENTION_BUCKETS) return "1 to 4096 buckets";
        if (!d->d_bucket_of || d->offsets < 1 || d->offsets > LEAP_ATTENTION_OFFSETS || d->offsets * d->heads > most) return "the table needs the buckets of 1 to 2^24 differences, 2^30 for all heads";
        if (d->heads >= 65535) return "more than 65534 heads with a table";
    }
    return nullptr;
}

attention_args arguments_of(const leap_attention_desc *d, const void *q, const void *k, const void *v)
{
    return {{(const uint16_t *)q, d->q_item, d->q_row, d->q_head}, {(const uint16_t *)k, d->k_item, d->k_row, d->k_head},
            {(const uint16_t *)v, d->v_item, d->v_row, d->v_head}, (int32_t)d->batch, (int32_t)d->queries, (int32_t)d->keys, (int32_t)d->heads,
            (int32_t)d->kv_heads, (int32_t)d->width, d->d_mask, d->mask_item, d->d_table, d->d_bucket_of, d->d_query_positions, d->d_key_positions,
            d->table_type, (int32_t)d->offsets, (int32_t)d->buckets, d->scale};
}

}  // namespace net

namespace {

// How the queries and keys of a call are dealt out to blocks.
struct shares {
    int32_t abreast, parts, length;
    int64_t units;                         // blocks that have all keys
};
shares shares_of(const leap_attention_desc *d)
{
    shares S;
    const int64_t group = d->heads / d->kv_heads, tiles = (d->keys + TILE - 1) / TILE;
    S.abreast = d->d_table ? 1 : d->queries <= 32 && group % 4 == 0 ? 4 : d->queries <= 64 && group % 2 == 0 ? 2 : 1;
    S.units = d->batch * (d->heads / S.abreast) * ((d->queries + COLS / S.abreast - 1) / (COLS / S.abreast));
    // Half the chip without work and at least sixteen tiles of keys: parts of four tiles and more, as many as fill it. One query, 8 heads of 64, a call: 8 tiles 11 us (16 in two parts),
    // 15 tiles 17, 16 to 64 tiles in parts 15, which is the host's time for two launches; between 8 and 15 the two sides meet, and what that leaves is 2 us
    int64_t parts = 1;
    if (S.units > 0 && S.units <= 128 && tiles >= 16) {
        parts = 512 / S.units;
        parts = parts < tiles / 4 ? parts : tiles / 4;
    }
    const int64_t each = tiles ? (tiles + parts - 1) / parts : 1;
    S.parts = (int32_t)(tiles ? (tiles + each - 1) / each : 1);
    S.length = (int32_t)(each * TILE);
    return S;
}
int64_t part_bytes(const leap_attention_desc *d, const shares &S)
{
    return S.parts > 1 ? (d->batch * d->heads * d->queries * S.parts * (d->width + 2) * 4 + 15) / 16 * 16 : 0;
}

// Of keys, and of values, laid out.
int64_t laid_out(const leap_attention_desc *d) { return d->queries > LAID_OUT ? laid_out_bytes(d->batch, d->keys, d->kv_heads, d->width) : 0; }

}  // namespace

extern "C" int64_t leap_attention_work(const leap_attention_desc *desc)
{
    return bad_attention(desc) ? 0 : lines_bytes(desc) + part_bytes(desc, shares_of(desc)) + 2 * laid_out(desc);
}

extern "C" int leap_attention(const leap_attention_desc *desc, const void *d_q, const void *d_k, const void *d_v, void *d_o, float *d_stats, void *d_rest,
                              void *d_work, void *hip_stream)
{
    if (const char *why = bad_attention(desc)) return refuse(why);
    if (!desc->batch || !desc->queries) return LEAP_OK;
    if (!d_q || !d_o || (desc->keys && (!d_k || !d_v))) return refuse("null data pointer");
    if (!d_rest != !d_stats) return refuse("statistics and what o's rounding leaves: both or neither");
    const shares S = shares_of(desc);
    const int64_t lines = lines_bytes(desc), parts = part_bytes(desc, S), laid = laid_out(desc);
    if (lines + parts + laid && unaligned(d_work)) return refuse(NO_WORK);
    forward_args F{arguments_of(desc, d_q, d_k, d_v), (uint16_t *)d_o, d_stats, (uint16_t *)d_rest, S.abreast, S.parts, S.length, nullptr, nullptr, 0};
    const int64_t blocks = S.units * S.parts, rows = desc->batch * desc->heads * desc->queries;
    if (blocks >= (int64_t)1 << 24) return refuse(TOO_MANY_BLOCKS);
    F.part_sums = (float *)((char *)d_work + lines);
    F.part_stats = F.part_sums + rows * S.parts * desc->width;
    const hipStream_t st = stream_of(hip_stream);
    if (desc->d_table) {
        const int rc = write_lines(F.a, d_work, st);
        if (rc != LEAP_OK) return rc;
    }
    if (laid) {
        char *const to = (char *)d_work + lines + parts;
        int rc = lay_out(F.a.k, desc->batch, desc->keys, desc->kv_heads, desc->width, to, st);
        if (rc == LEAP_OK) rc = lay_out(F.a.v, desc->batch, desc->keys, desc->kv_heads, desc->width, to + laid, st);
        if (rc != LEAP_OK) return rc;
    }
    const bool direct = laid || (direct_array(d_k, desc->k_item, desc->k_row, desc->k_head, desc->width) && direct_array(d_v, desc->v_item, desc->v_row, desc->v_head, desc->width));
    const int rc = by_width(desc->width, [&](auto w) {
        return by_flags([&](auto straight, auto bias, auto fine) {
            hipLaunchKernelGGL((k_attention<decltype(w)::value, decltype(straight)::value, decltype(bias)::value, decltype(fine)::value>), dim3((unsigned)blocks), dim3(BLOCK), 0, st, F);
            return launched();
        }, direct, desc->d_table != nullptr, d_rest != nullptr);
    });
    if (rc != LEAP_OK || S.parts == 1) return rc;
    return over_blocks(rows, [&](int64_t first, unsigned n) {
        F.first = first;
        hipLaunchKernelGGL(k_join, dim3(n), dim3(BLOCK), 0, st, F);
    });
}
