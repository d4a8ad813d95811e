// Attention's gradients.  With p the probabilities, formed again from the scores and each query's statistics, and
// dp = grad.v:  delta = grad.o (the sum of p dp over a query's keys),  ds = p (dp - delta),  grad_v = sum over queries of p grad,  grad_q = scale times the
// sum over keys of ds k,  grad_k = scale times the sum over queries of ds q,  and a bucket's number gets the sum of ds over its pairs.
//
// Two kernels, each the owner of what it writes, so that no sum depends on an order of arrival: k_grad_query has queries in its lanes and
// walks over keys as the forward pass does; k_grad_key has keys in its lanes and walks over queries.  Both form the scores and dp: seven products instead
// of the five of one kernel, which would have to add up grad_q over blocks.
//
// p and ds are 32 bits until they are a side of the products that sum over them, where they are rounded to bfloat16: gradients are 0.0022 to 0.0026 of their norm off, 0.0017 of it by their own
// rounding.  In two bfloat16 each, as p is in the forward pass, the two kernels took 3.18 ms instead of 2.87 in 512 windows of 512 patches of 64, and 23.3 instead of 16.4 ms for 32768 patches of 128 (three
// products more of seven).
//
// Neither kernel deals out the side that it walks over: few queries, or few keys, are few blocks (2 x 16 queries over 262144 keys of 8 heads: 16).
//
// 32768 patches, 8 heads of 128: queries 6.3 ms, keys and values 9.7 to 10.3 ms (1040, and 860 to 900 TFLOP/s of matrix instructions; the latter's sums leave room for one wave a SIMD).
// 512 windows of 512 patches, 8 heads of 64 with a table: 1.70 and 1.17 ms, bound by vector instructions (21 and 14 a pair, counted) and, for the table's gradient, adds to shared
// memory (those to differences took 0.27 ms: without the buckets' 1.58 ms, without either 1.30).
#include "net_attention.h"

namespace {

using namespace net;

struct grad_args {
    attention_args a;
    rows_of grad;
    const uint16_t *o, *rest;
    const float *stats;
    float *delta;
    uint16_t *grad_q, *grad_k, *grad_v;
    float *part;                       // [heads][parts][buckets]
    int32_t parts;
    int64_t first;                     // block of this launch
};

// A query's statistics: probabilities are exp2(x - most) / sum, without a table (BIAS) exp2(x - most - log), and zeros where it has no keys.
struct query_stats {
    float most, second;
};
__device__ inline query_stats stats_of(const grad_args &G, int64_t row)
{
    return {G.stats[row * 2], G.stats[row * 2 + 1]};
}
template <bool BIAS> constexpr query_stats NO_KEYS = {0.0f, BIAS ? 0.0f : INFINITY};
template <bool BIAS> __device__ inline float log_of(const query_stats &s) { return !BIAS ? s.second : s.second != 0.0f ? __builtin_amdgcn_logf(s.second) : INFINITY; }

constexpr int DELTA_LANES = LEAP_ATTENTION_WIDEST / 8, DELTA_ROWS = BLOCK / DELTA_LANES;

// The sum of grad o over eight values of a row; o is what it was before its rounding: its bits and what is to be added to them.
__device__ inline float grad_dot_o(const u32x4 &g, const u32x4 &o, const u32x4 &rest)
{
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t gi = i % 2 ? g[i / 2] & 0xffff0000u : g[i / 2] << 16, oi = i % 2 ? o[i / 2] & 0xffff0000u : o[i / 2] << 16;
        sum += __uint_as_float(gi) * __uint_as_float(oi + (uint32_t)(int32_t)(int16_t)(rest[i / 2] >> (i % 2 * 16)));
    }
    return sum;
}

// delta by itself, where k_grad_query does not run: sixteen lanes a row.  Summed as there, so that the gradient of keys has the same bits whether that of queries is wanted or not: the
// even pieces one after the other, the odd ones, then both.
__global__ __launch_bounds__(BLOCK) void k_delta(grad_args G)
{
    const attention_args &A = G.a;
    const int lane = threadIdx.x % DELTA_LANES;
    const int64_t row = (G.first + blockIdx.x) * DELTA_ROWS + threadIdx.x / DELTA_LANES;
    if (row >= (int64_t)A.batch * A.queries * A.heads) return;
    const int head = (int)(row % A.heads);
    const int64_t query = row / A.heads % A.queries, item = row / A.heads / A.queries;
    const u32x4 g = row_piece(G.grad.data + item * G.grad.item + query * G.grad.row + head * G.grad.head, A.width, lane);
    const float piece = grad_dot_o(g, row_piece(G.o + row * A.width, A.width, lane), row_piece(G.rest + row * A.width, A.width, lane));
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < DELTA_LANES; s += 2) sum += __shfl(piece, s + lane % 2, DELTA_LANES);
    sum += __shfl_xor(sum, 1);
    if (lane == 0) G.delta[(item * A.heads + head) * (int64_t)A.queries + query] = sum;
}

// Numbers of a line in shared memory (see net_attention.hip): as many as leave a compute unit room for two blocks, up to width 64; above, the tiles and a table's sums leave it one
// (93 to 117 KB), and without a table's gradient two.
constexpr int window_of_tile(int deep, int buckets) { return deep > 64 || buckets > 1024 ? 1024 : 2048; }

// A table's gradient.  Adds of integers to shared memory take a wave 4 cycles, those of floats 192 (3 a lane), and integers' order does not matter.  So a tile's ds are added as
// integers to two numbers for every difference that its pairs have: whole multiples of 2^-22 of the largest of them's power of two, which scales without a rounding, and what is left in multiples of 2^-46.  (With the
// first alone sums were 0.6e-5 to 6e-5 of the table's norm off, since a bucket that nearly all of a query's keys are in has a sum far smaller than its terms.)  Keys rise, so a
// difference has at most one pair of each of the block's 128 queries, and 128 times 2^23 fits 32 bits.
// In the next tile's time the sums go to their buckets, which the block keeps in 64 bits where shared memory has room for them (a bucket of most of a query's keys is a small difference of large tiles'
// sums: 16 x 211 rows 1.4e-7 of the norm off, with floats twice that; no slower), for more than 1024 of width 64 as floats: without atomic adds where the window's buckets rise (one of its own to
// every difference: in 512 windows 0.39 ms of 1.97 were such adds), otherwise a wave to every fourth bucket.
// Where the differences are too far apart or keys do not rise, ds go to the buckets as one integer of 64 bits, of 2^-48 of that power: 8192 of them fit.
template <int BUCKETS, int WINDOW, class SUM> struct table_sums {
    SUM bucket[BUCKETS];
    union {
        struct {
            int32_t upper[WINDOW], lower[WINDOW];
        };
        uint64_t total[WINDOW];
    };
    uint16_t which[WINDOW];                                // the buckets of the window
    uint32_t peak[WAVES];                                  // the largest ds of each wave's, its bits
};
template <int WINDOW, class SUM> struct table_sums<0, WINDOW, SUM> {};

// Shared memory's writes of all waves are there for all; what comes from memory is not waited for.
__device__ inline void shared_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The largest of a wave, of magnitudes as integers: what is not a number is larger than infinity there.
constexpr uint32_t INFINITE = 0x7f800000u;
__device__ inline uint32_t wave_max(uint32_t v)
{
    const auto with = [&](int other) { v = (uint32_t)other > v ? (uint32_t)other : v; };
    with(__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false));        // the neighbour, the other pair,
    with(__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false));
    with(__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));       // the other four of eight, the other eight of sixteen
    with(__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, false));
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = a[0] > a[1] ? a[0] : a[1];
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return b[0] > b[1] ? b[0] : b[1];
}

template <int DEEP, bool DIRECT, bool BIAS, int BUCKETS> __global__ __launch_bounds__(BLOCK, BUCKETS && DEEP > 64 ? 1 : 2) void k_grad_query(grad_args G)
{
    using tile = rows_tile<DEEP>;
    constexpr int STEPS = DEEP / 16, BLOCKS = DEEP / 32, WINDOW = window_of_tile(DEEP, BUCKETS);
    const attention_args &A = G.a;
    __shared__ __attribute__((aligned(16))) uint8_t room[4 * tile::BYTES + (BIAS ? 2 * WINDOW * 4 : 0)];
    using sum_of_bucket = std::conditional_t<BUCKETS == LEAP_ATTENTION_BUCKETS && DEEP == 64, float, double>;
    __shared__ __attribute__((aligned(16))) table_sums<BUCKETS, WINDOW, sum_of_bucket> sums;
    __shared__ int places[BIAS ? 2 : 1][TILE];
    lds_byte *const lds = (lds_byte *)room;
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int tiles = (A.queries + COLS - 1) / COLS;
    const int64_t units = (int64_t)A.batch * tiles;
    if constexpr (BUCKETS != 0) {
        for (int b = threadIdx.x; b < BUCKETS; b += BLOCK) sums.bucket[b] = 0;
        for (int b = threadIdx.x; b < WINDOW; b += BLOCK) sums.upper[b] = sums.lower[b] = 0;
    }

    const int64_t block = unit_of(blockIdx.x, gridDim.x);
    // a block a unit, the heads of an item apart; with a table the same head for all units of a block
    const int head = BUCKETS ? (int)(block / G.parts) : (int)(block / tiles % A.heads), kv_head = head / (A.heads / A.kv_heads);
    int64_t unit = BUCKETS ? block % G.parts : block / tiles / A.heads * tiles + block % tiles;
    const float *const line = BIAS ? A.lines + (int64_t)head * A.line : nullptr;
    const float scale = A.scale * LOG2E;
    if (unit < units) do {
        int width = A.width;                               // (what follows from it alone is not to be kept for the next unit: it would fill the registers)
        asm volatile("" : "+s"(width));
        const int64_t item = unit / tiles;
        const int query0 = (int)(unit % tiles) * COLS, query = query0 + wave * 32 + lane % 32;
        const bool there = query < A.queries;
        source<DEEP, DIRECT> k(A.k.data + item * A.k.item + kv_head * A.k.head, A.k.row, A.keys, width, wave, lane);
        source<DEEP, DIRECT> v(A.v.data + item * A.v.item + kv_head * A.v.head, A.v.row, A.keys, width, wave, lane);
        bf16x8 q[STEPS], g[STEPS];
        load_side<STEPS>(q, A.q.data + item * A.q.item + head * A.q.head + query * A.q.row, width, there, lane);
        load_side<STEPS>(g, G.grad.data + item * G.grad.item + head * G.grad.head + query * G.grad.row, width, there, lane);
        const int64_t row = (item * A.heads + head) * (int64_t)A.queries + query;
        const query_stats stats = there ? stats_of(G, row) : NO_KEYS<BIAS>;
        float delta = 0.0f;
        {
            const int64_t at = ((item * A.queries + query) * A.heads + head) * width;
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
                if (there) delta += grad_dot_o(__builtin_bit_cast(u32x4, g[s]), row_piece(G.o + at, width, s * 2 + lane / 32), row_piece(G.rest + at, width, s * 2 + lane / 32));
            delta = column_sum(delta);
            if (there && lane < 32) G.delta[row] = delta;          // for k_grad_key
        }
        // With a table scores can be so large that the logarithm of their sum would be lost in what they are lowered by, and the table's gradient is 32 bits, of which the rounding of exponents
        // takes the fewer the nearer they are to 0: so there they are lowered by the largest alone, and the sum is a factor of dp's and delta's.
        const float base = !BIAS ? stats.most + stats.second : stats.second != 0.0f ? stats.most : INFINITY;
        const float factor = BIAS && stats.second != 0.0f ? 1.0f / stats.second : 0.0f, lowered = factor * delta;
        const int position = BIAS ? query_position(A, there ? query : A.queries - 1) : 0;
        place_range mine;
        if constexpr (BIAS) mine = both(A.query_places[query0 / TILE], A.query_places[query0 + TILE < A.queries ? query0 / TILE + 1 : query0 / TILE]);
        f32x16 sum[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) sum[b] = zeros();

        key_walk at(A.mask ? A.mask + item * A.mask_item : nullptr, 0, A.keys, lane);
        line_window window{}, coming{}, before{};
        bool fours = false, coming_fours = false, rising = false, coming_rising = false, pending = false, apart = false;
        uint8_t coming_apart = 0;
        int place = 0;
        float unscale = 0.0f;
        const auto fetch = [&](int to) {
            lds_byte *const kt = lds + to * 2 * tile::BYTES;
            k.fetch(at.first, at.bits, kt, wave, lane);
            v.fetch(at.first, at.bits, kt + tile::BYTES, wave, lane);
            if constexpr (BIAS) {
                const place_range keys = A.key_places[at.first / TILE];
                coming = window_of(A, keys, mine, WINDOW), coming_fours = keys.fours, coming_rising = keys.rising;
                if (coming.inside) fetch_window<4>(line, A.offsets, coming, lds + 4 * tile::BYTES + to * WINDOW * 4, wave, lane);
                if (wave == 0) place = key_position(A, at.first + lane < A.keys ? (int)at.first + lane : A.keys - 1);
                if constexpr (BUCKETS != 0)        // (a window spans less than 64 times 64)
                    coming_apart = coming.inside && coming.first / WAVE + lane <= (coming.first + coming.count - 1) / WAVE ? A.line_rising[coming.first / WAVE + lane] : 1;
            }
        };
        // The sums of the tile before: every wave has the buckets of its own, and each of those its order.
        const auto settle = [&] {
            if constexpr (BUCKETS != 0) {
                if (pending && apart)              // no two of a bucket
                    for (int i = threadIdx.x; i < before.count; i += BLOCK) {
                        sums.bucket[sums.which[i]] += ((sum_of_bucket)sums.upper[i] + (sum_of_bucket)sums.lower[i] * (sum_of_bucket)0x1p-24) * unscale;
                        sums.upper[i] = sums.lower[i] = 0;
                    }
                else if (pending)
                    for (int i = lane; i < before.count; i += WAVE) {
                        const int bucket = sums.which[i];
                        if (bucket % WAVES != wave) continue;
                        const int upper = sums.upper[i], lower = sums.lower[i];
                        if (!(upper | lower)) continue;                                    // a float's add takes the 3 cycles for every lane that makes one
                        sums.upper[i] = sums.lower[i] = 0;
                        __hip_atomic_fetch_add(&sums.bucket[bucket], ((sum_of_bucket)upper + (sum_of_bucket)lower * (sum_of_bucket)0x1p-24) * unscale, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                    }
            }
        };
        __syncthreads();                                   // the unit before has read its tiles
        if (!at.done()) fetch(0);
        const auto one = [&](auto pair) {
            const int turn = pair;
            lds_byte *const kt = lds + turn * 2 * tile::BYTES, *const vt = kt + tile::BYTES;
            const uint64_t bits = at.bits;
            k.land(kt), v.land(vt);
            if constexpr (BIAS) {
                if (wave == 0) places[turn][lane] = place;
                window = coming, fours = coming_fours, rising = coming_rising;
            }
            const bool window_apart = BUCKETS && __all(coming_apart != 0);
            if constexpr (DIRECT || BIAS) fetched();
            __syncthreads();
            at.next(lane);
            if (!at.done()) fetch(turn ^ 1);
            settle();
            const uint32_t from_line = origin_of(lds + 4 * tile::BYTES + turn * WINDOW * 4, A, window, position, false);
            f32x16 x[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                x[h] = zeros();
                f32x16 dp = zeros();
#pragma unroll
                for (int s = 0; s < STEPS; ++s) x[h] = product(tile::along(kt, h * 32, s, lane), q[s], x[h]);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) dp = product(tile::along(vt, h * 32, s, lane), g[s], dp);
                const uint32_t held = (uint32_t)(bits >> (h * 32)) >> (lane / 32 * 4);
                const auto ds_of = [&](int r, float exponent) {
                    x[h][r] = __builtin_amdgcn_exp2f(exponent) * (BIAS ? __builtin_fmaf(dp[r], factor, -lowered) : dp[r] - delta);
                };
                if constexpr (BIAS) {
                    if (window.inside)
                        over_places<1, const float>(places[turn] + h * 32, fours, from_line, lane,
                                                    [&](int r, auto number) { ds_of(r, __builtin_fmaf(x[h][r], scale, *number) - base); });
                    else
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            ds_of(r, __builtin_fmaf(x[h][r], scale, line[line_at(A, places[turn][h * 32 + row_of(r) + lane / 32 * 4], position)]) - base);
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r) ds_of(r, __builtin_fmaf(x[h][r], scale, -base));
                }
                if (~bits) {
                    seldom();
#pragma unroll
                    for (int r = 0; r < 16; ++r) x[h][r] = held >> row_of(r) & 1 ? x[h][r] : 0.0f;
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bf16x8 ds = eight(x[h], t);
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b) sum[b] = product(tile::across(kt, h * 32 + t * 16, b, lane), ds, sum[b]);
                }
            }
            const bool near = window.inside && rising;
            if constexpr (BUCKETS != 0) {
                float largest = 0.0f;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 16; ++r) largest = __builtin_elementwise_maximum(largest, fabsf(x[h][r]));
                const auto of_block = [&] {                // and the sums before are settled
                    const uint32_t mine = wave_max(__float_as_uint(largest));
                    if (lane == 0) sums.peak[wave] = mine;
                    shared_barrier();
                    uint32_t most = __float_as_uint(1e-30f);
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) most = sums.peak[w] > most ? sums.peak[w] : most;
                    return (uint32_t)uniform((int)most);
                };
                uint32_t most = of_block();
                if (most >= INFINITE) {                    // ds that are not finite go to the buckets of their pairs by themselves
                    seldom();
                    largest = 0.0f;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const bool finite = (__float_as_uint(x[h][r]) & 0x7fffffffu) < INFINITE;
                            if (!finite && there)
                                __hip_atomic_fetch_add(&sums.bucket[A.line_buckets[line_at(A, places[turn][h * 32 + row_of(r) + lane / 32 * 4], position)]], (sum_of_bucket)x[h][r], __ATOMIC_RELAXED,
                                                       __HIP_MEMORY_SCOPE_WORKGROUP);
                            x[h][r] = finite ? x[h][r] : 0.0f;
                            largest = fmaxf(largest, fabsf(x[h][r]));
                        }
                    shared_barrier();                      // all have read the peaks
                    most = of_block();
                }
                const uint32_t power = most >> 23;         // of two, of the largest, + 127: 27 to 254
                if (near) {
                    fetch_window<2>(A.line_buckets, A.offsets, window, (lds_byte *)sums.which, wave, lane);
                    const float by = __uint_as_float((276 - power) << 23);                     // 2^22 for the power
                    unscale = __uint_as_float((power - 22) << 23);
                    const uint32_t to_sums = origin_of((lds_byte *)sums.upper, A, window, position, false);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        over_places<1, int>(places[turn] + h * 32, fours, to_sums, lane, [&](int r, auto sum_of) {
                            const float v = x[h][r] * by, whole = rintf(v);
                            __hip_atomic_fetch_add(sum_of, (int)whole, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                            __hip_atomic_fetch_add(sum_of + WINDOW, (int)((v - whole) * 0x1p24f), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                        });
                } else {
                    constexpr int AT_ONCE = WINDOW;
                    float by = __uint_as_float((270 - power) << 23);                           // 2^16
                    const float unit = __uint_as_float(power << 23);
                    for (int first = 0; first < A.buckets; first += AT_ONCE) {
                        asm volatile("" : "+v"(by));       // (the terms are not to be kept from one turn to the next: it would fill the registers)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const int b = A.line_buckets[line_at(A, places[turn][h * 32 + row_of(r) + lane / 32 * 4], position)] - first;
                                const float v = x[h][r] * by, whole = rintf(v);
                                const int64_t term = ((int64_t)(int)whole << 32) + (int)((v - whole) * 0x1p32f);
                                if (b >= 0 && b < AT_ONCE) __hip_atomic_fetch_add(&sums.total[b], (uint64_t)term, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                            }
                        shared_barrier();
                        for (int b = threadIdx.x; b < AT_ONCE && first + b < A.buckets; b += BLOCK) {
                            sums.bucket[first + b] += (sum_of_bucket)(int64_t)sums.total[b] * (sum_of_bucket)0x1p-48 * unit;
                            sums.total[b] = 0;
                        }
                        shared_barrier();
                    }
                }
            }
            pending = near, before = window, apart = window_apart;
        };
        for (int turn = 0; !at.done(); turn ^= 1) one(turn);
        if constexpr (BUCKETS != 0) {
            fetched();                                     // the last tile's buckets
            __syncthreads();
            settle();
        }
        if (G.grad_q) store_column<BLOCKS>(G.grad_q + ((item * A.queries + query) * A.heads + head) * width, width, sum, A.scale, lane, there);
        unit += G.parts;
    } while (BUCKETS && unit < units);
    if constexpr (BUCKETS != 0) {
        __syncthreads();
        for (int b = threadIdx.x; b < A.buckets; b += BLOCK) G.part[block * A.buckets + b] = (float)sums.bucket[b];
    }
}

// grad_table <- the sum of the parts.
__global__ __launch_bounds__(BLOCK) void k_join_table(const float *__restrict__ part, int parts, int buckets, float *__restrict__ out)
{
    const int b = blockIdx.x * BLOCK + threadIdx.x;
    if (b >= buckets) return;
    const float *const from = part + (int64_t)blockIdx.y * parts * buckets + b;
    double sum = 0.0;
#pragma unroll 8
    for (int p = 0; p < parts; ++p) sum += from[(int64_t)p * buckets];
    out[(int64_t)blockIdx.y * buckets + b] = (float)sum;
}

template <int DEEP, bool DIRECT, bool BIAS> __global__ __launch_bounds__(BLOCK, DEEP > 64 ? 1 : 2) void k_grad_key(grad_args G)
{
    using tile = rows_tile<DEEP>;
    constexpr int STEPS = DEEP / 16, BLOCKS = DEEP / 32, WINDOW = 2048;
    const attention_args &A = G.a;
    __shared__ __attribute__((aligned(16))) uint8_t room[4 * tile::BYTES + (BIAS ? 2 * WINDOW * 4 : 0)];
    __shared__ __attribute__((aligned(16))) float most[2][TILE], log[2][TILE], delta[2][TILE];
    __shared__ int places[BIAS ? 2 : 1][TILE];
    lds_byte *const lds = (lds_byte *)room;
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int blocks = (A.keys + COLS - 1) / COLS, group = A.heads / A.kv_heads, tiles = (A.queries + TILE - 1) / TILE;
    const int64_t unit = unit_of(blockIdx.x, gridDim.x), item = unit / blocks / A.kv_heads;
    const int kv_head = (int)(unit / blocks % A.kv_heads), key0 = (int)(unit % blocks) * COLS, key = key0 + wave * 32 + lane % 32;
    const bool there = key < A.keys;
    const uint8_t *const mask = A.mask ? A.mask + item * A.mask_item : nullptr;
    const bool held = there && (!mask || mask[key]);
    const bool any = rows_there(mask, key0, A.keys, lane) | rows_there(mask, key0 + TILE, A.keys, lane);        // of all waves alike
    const float scale = A.scale * LOG2E;
    f32x16 gk[BLOCKS], gv[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) gk[b] = gv[b] = zeros();

    if (any) {
        bf16x8 k[STEPS], v[STEPS];
        load_side<STEPS>(k, A.k.data + item * A.k.item + kv_head * A.k.head + key * A.k.row, A.width, held, lane);
        load_side<STEPS>(v, A.v.data + item * A.v.item + kv_head * A.v.head + key * A.v.row, A.width, held, lane);
        const int position = BIAS ? key_position(A, there ? key : A.keys - 1) : 0;
        place_range mine;
        if constexpr (BIAS) mine = both(A.key_places[key0 / TILE], A.key_places[key0 + TILE < A.keys ? key0 / TILE + 1 : key0 / TILE]);
        // the group's heads one after the other, each head's queries in tiles
        for (int head = kv_head * group; head < (kv_head + 1) * group; ++head) {
            source<DEEP, DIRECT> q(A.q.data + item * A.q.item + head * A.q.head, A.q.row, A.queries, A.width, wave, lane);
            source<DEEP, DIRECT> g(G.grad.data + item * G.grad.item + head * G.grad.head, G.grad.row, A.queries, A.width, wave, lane);
            const float *const line = BIAS ? A.lines + (int64_t)head * A.line : nullptr;
            const int64_t row0 = (item * A.heads + head) * (int64_t)A.queries;
            query_stats stats;
            float nd;
            int place = 0;
            line_window window{}, coming{};
            bool fours = false, coming_fours = false;
            const auto fetch = [&](int at, int to) {
                const int first = at * TILE;
                const uint64_t bits = A.queries - first >= TILE ? ~(uint64_t)0 : ((uint64_t)1 << (A.queries - first)) - 1;
                lds_byte *const qt = lds + to * 2 * tile::BYTES;
                q.fetch(first, bits, qt, wave, lane);
                g.fetch(first, bits, qt + tile::BYTES, wave, lane);
                if constexpr (BIAS) {
                    const place_range queries = A.query_places[at];
                    coming = window_of(A, mine, queries, WINDOW), coming_fours = queries.fours;
                    if (coming.inside) fetch_window<4>(line, A.offsets, coming, lds + 4 * tile::BYTES + to * WINDOW * 4, wave, lane);
                }
                if (wave == 0) {
                    const bool in = first + lane < A.queries;
                    stats = in ? stats_of(G, row0 + first + lane) : NO_KEYS<BIAS>;
                    nd = in ? G.delta[row0 + first + lane] : 0.0f;
                    if (BIAS) place = query_position(A, in ? first + lane : A.queries - 1);
                }
            };
            __syncthreads();                               // the head before has read its tiles
            if (tiles) fetch(0, 0);
            const auto one = [&](int at, auto pair) {
                const int turn = pair;
                lds_byte *const qt = lds + turn * 2 * tile::BYTES, *const gt = qt + tile::BYTES;
                q.land(qt), g.land(gt);
                if (wave == 0) {
                    most[turn][lane] = BIAS ? stats.most : stats.most + stats.second;
                    log[turn][lane] = log_of<BIAS>(stats);
                    delta[turn][lane] = nd;
                    if constexpr (BIAS) places[turn][lane] = place;
                }
                if constexpr (BIAS) window = coming, fours = coming_fours;
                if constexpr (DIRECT || BIAS) fetched();
                __syncthreads();
                if (at + 1 < tiles) fetch(at + 1, turn ^ 1);
                const uint32_t from_line = origin_of(lds + 4 * tile::BYTES + turn * WINDOW * 4, A, window, position, true);
                // Half a tile's scores and dp are multiplied while the other half's probabilities are formed: x[h] becomes p, dp[h] ds.
                f32x16 x[2], dp[2];
                const auto scores = [&](int h) {
                    x[h] = zeros(), dp[h] = zeros();
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) {
                        x[h] = product(tile::along(qt, h * 32, s, lane), k[s], x[h]);
                        dp[h] = product(tile::along(gt, h * 32, s, lane), v[s], dp[h]);
                    }
                };
                const auto probabilities = [&](int h) {
                    const auto p_of = [&](int r, float exponent) {
                        x[h][r] = __builtin_amdgcn_exp2f(exponent);
                        dp[h][r] = x[h][r] * (dp[h][r] - delta[turn][h * 32 + row_of(r) + lane / 32 * 4]);
                    };
                    const auto lowered = [&](int r, float score) {
                        const int row = h * 32 + row_of(r) + lane / 32 * 4;
                        return score - most[turn][row] - log[turn][row];
                    };
                    if constexpr (BIAS) {
                        if (window.inside)
                            over_places<-1, const float>(places[turn] + h * 32, fours, from_line, lane,
                                                         [&](int r, auto number) { p_of(r, lowered(r, __builtin_fmaf(x[h][r], scale, *number))); });
                        else
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                p_of(r, lowered(r, __builtin_fmaf(x[h][r], scale, line[line_at(A, position, places[turn][h * 32 + row_of(r) + lane / 32 * 4])])));
                    } else {
#pragma unroll
                        for (int r = 0; r < 16; ++r) p_of(r, __builtin_fmaf(x[h][r], scale, -most[turn][h * 32 + row_of(r) + lane / 32 * 4]));
                    }
                };
                const auto gradients = [&](int h) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const bf16x8 p = eight(x[h], t), ds = eight(dp[h], t);
#pragma unroll
                        for (int b = 0; b < BLOCKS; ++b) {
                            gv[b] = product(tile::across(gt, h * 32 + t * 16, b, lane), p, gv[b]);
                            gk[b] = product(tile::across(qt, h * 32 + t * 16, b, lane), ds, gk[b]);
                        }
                    }
                };
                if constexpr (DEEP > 64) {
                    scores(0);
                    scores(1);
                    probabilities(0);
                    gradients(0);
                    probabilities(1);
                    gradients(1);
                    // A wave has its SIMD to itself: reads of shared memory go ahead of the products that want them, and the probabilities' vector instructions between products.
                    constexpr int MFMA = 0x8, VECTOR = 0x2, READ = 0x100;
                    const auto products = [&](auto count, auto reads, auto vectors) {
#pragma unroll
                        for (int i = 0; i < decltype(count)::value; ++i) {
                            __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
                            __builtin_amdgcn_sched_group_barrier(READ, decltype(reads)::value, 0);
                            if constexpr (decltype(vectors)::value) __builtin_amdgcn_sched_group_barrier(VECTOR, decltype(vectors)::value, 0);
                        }
                    };
                    using std::integral_constant;
                    __builtin_amdgcn_sched_group_barrier(READ, 6, 0);
                    products(integral_constant<int, 2 * STEPS + 10>{}, integral_constant<int, 1>{}, integral_constant<int, 0>{});
                    products(integral_constant<int, 2 * STEPS - 10>{}, integral_constant<int, 2>{}, integral_constant<int, 0>{});
                    products(integral_constant<int, 4 * BLOCKS>{}, integral_constant<int, 2>{}, integral_constant<int, 6>{});
                    products(integral_constant<int, 4 * BLOCKS>{}, integral_constant<int, 2>{}, integral_constant<int, 0>{});
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) scores(h), probabilities(h), gradients(h);
                }
            };
            // Two tiles a turn, so that addresses in shared memory are constants: pays (12.3 to 10.4 ms for 32768 patches of 128) where a wave has its SIMD's registers to
            // itself, not where their number decides (512 windows of 512 patches of 64: 1.42 ms, 1.14 so)
            if constexpr (DEEP > 64)
                for (int at = 0; at < tiles; at += 2) {
                    one(at, std::integral_constant<int, 0>{});
                    if (at + 1 < tiles) one(at + 1, std::integral_constant<int, 1>{});
                }
            else
                for (int at = 0; at < tiles; ++at) one(at, at % 2);
        }
    }
    // a key that is left out has whatever its zeros gave
    if (!held)
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) gk[b] = gv[b] = zeros();
    const int64_t row = ((item * A.keys + key) * A.kv_heads + kv_head) * A.width;
    if (G.grad_k) store_column<BLOCKS>(G.grad_k + row, A.width, gk, A.scale, lane, there);
    if (G.grad_v) store_column<BLOCKS>(G.grad_v + row, A.width, gv, 1.0f, lane, there);
}

// Gradients that no query has a part in, eight values of 16 bits a thread.
__global__ __launch_bounds__(BLOCK) void k_zeros(uint16_t *to, int64_t values, int64_t first)
{
    const int64_t at = ((first + blockIdx.x) * BLOCK + threadIdx.x) * CHUNK;
    if (at < values) store_piece<2>((uint8_t *)(to + at), (values - at) * 2, u32x4{0, 0, 0, 0});
}

int zeros_to(void *to, int64_t values, hipStream_t st)
{
    if (!to) return LEAP_OK;
    return over_blocks((values + BLOCK * CHUNK - 1) / (BLOCK * CHUNK), [&](int64_t first, unsigned blocks) {
        hipLaunchKernelGGL(k_zeros, dim3(blocks), dim3(BLOCK), 0, st, (uint16_t *)to, values, first);
    });
}

// Blocks that a head's units are dealt out to where the table's gradient is formed: each has room of its own for it.
int64_t table_parts(const leap_attention_desc *d)
{
    const int64_t units = d->batch * ((d->queries + COLS - 1) / COLS), most = d->heads < 1024 ? 2048 / d->heads : 2;
    return units < 1 ? 1 : units < most ? units : most;
}

// Of keys (and of values), and of queries (and of grad), laid out for the kernel that walks over them.
int64_t laid_keys(const leap_attention_desc *d) { return d->queries > LAID_OUT ? laid_out_bytes(d->batch, d->keys, d->kv_heads, d->width) : 0; }
int64_t laid_queries(const leap_attention_desc *d) { return d->keys > LAID_OUT ? laid_out_bytes(d->batch, d->queries, d->heads, d->width) : 0; }

int64_t delta_bytes(const leap_attention_desc *d) { return (d->batch * d->heads * d->queries * 4 + 15) / 16 * 16; }

}  // namespace

extern "C" int64_t leap_attention_backward_work(const leap_attention_desc *desc, int32_t with_table)
{
    if (bad_attention(desc)) return 0;
    return delta_bytes(desc) + lines_bytes(desc) + 2 * laid_keys(desc) + 2 * laid_queries(desc) + (with_table && desc->d_table ? desc->heads * table_parts(desc) * desc->buckets * 4 : 0);
}

extern "C" int leap_attention_backward(const leap_attention_desc *desc, const void *d_grad, int64_t grad_item, int64_t grad_row, int64_t grad_head, const void *d_q,
                                       const void *d_k, const void *d_v, const void *d_o, const float *d_stats, const void *d_rest, void *d_grad_q,
                                       void *d_grad_k, void *d_grad_v, float *d_grad_table, void *d_work, void *hip_stream)
{
    if (const char *why = bad_attention(desc)) return refuse(why);
    if (const char *why = bad_array(desc->batch, grad_item, desc->queries, grad_row, desc->heads, grad_head)) return refuse(why);
    if (d_grad_table && !desc->d_table) return refuse("the gradient of a table that is not there");
    const int64_t rows = desc->batch * desc->heads * desc->queries, kept = desc->batch * desc->kv_heads * desc->keys;
    if (rows && (!d_grad || !d_q || !d_o || !d_stats || !d_rest || (desc->keys && (!d_k || !d_v)))) return refuse("null data pointer");
    if (rows && unaligned(d_work)) return refuse(NO_WORK);
    const int64_t tiles = (desc->queries + COLS - 1) / COLS, key_tiles = (desc->keys + COLS - 1) / COLS;
    if (desc->batch * desc->heads * tiles >= (int64_t)1 << 24 || desc->batch * desc->kv_heads * key_tiles >= (int64_t)1 << 24) return refuse(TOO_MANY_BLOCKS);
    if ((int64_t)desc->heads / desc->kv_heads * ((desc->queries + TILE - 1) / TILE) >= (int64_t)1 << 31) return refuse("more than 2^37 queries share a key");
    const hipStream_t st = stream_of(hip_stream);
    if (!rows) {                                           // nothing is read, the workspace is not written
        const int rc = zeros_to(d_grad_k, kept * desc->width, st);
        const int status = rc == LEAP_OK ? zeros_to(d_grad_v, kept * desc->width, st) : rc;
        return status == LEAP_OK ? zeros_to(d_grad_table, desc->heads * desc->buckets * 2, st) : status;
    }
    grad_args G{arguments_of(desc, d_q, d_k, d_v), {(const uint16_t *)d_grad, grad_item, grad_row, grad_head}, (const uint16_t *)d_o, (const uint16_t *)d_rest,
                d_stats, (float *)d_work, (uint16_t *)d_grad_q, (uint16_t *)d_grad_k, (uint16_t *)d_grad_v, (float *)((char *)d_work + delta_bytes(desc) + lines_bytes(desc) + 2 * laid_keys(desc) + 2 * laid_queries(desc)),
                (int32_t)table_parts(desc), 0};
    int rc = LEAP_OK;
    if (!d_grad_q && !d_grad_table && (d_grad_k || d_grad_v))
        rc = over_blocks((rows + DELTA_ROWS - 1) / DELTA_ROWS, [&](int64_t first, unsigned blocks) {
            G.first = first;
            hipLaunchKernelGGL(k_delta, dim3(blocks), dim3(BLOCK), 0, st, G);
        });
    if (rc != LEAP_OK) return rc;
    if (desc->d_table) rc = write_lines(G.a, (char *)d_work + delta_bytes(desc), st);
    if (rc != LEAP_OK) return rc;
    const int64_t laid_k = laid_keys(desc), laid_q = laid_queries(desc);
    const bool keys_walked = d_grad_table || d_grad_q, queries_walked = d_grad_k || d_grad_v;
    grad_args of_keys = G;                                 // for k_grad_key, which has its keys as they are
    char *const to = (char *)d_work + delta_bytes(desc) + lines_bytes(desc);
    if (laid_k && keys_walked) {
        rc = lay_out(G.a.k, desc->batch, desc->keys, desc->kv_heads, desc->width, to, st);
        if (rc == LEAP_OK) rc = lay_out(G.a.v, desc->batch, desc->keys, desc->kv_heads, desc->width, to + laid_k, st);
    }
    if (laid_q && queries_walked && rc == LEAP_OK) {
        rc = lay_out(of_keys.a.q, desc->batch, desc->queries, desc->heads, desc->width, to + 2 * laid_k, st);
        if (rc == LEAP_OK) rc = lay_out(of_keys.grad, desc->batch, desc->queries, desc->heads, desc->width, to + 2 * laid_k + laid_q, st);
    }
    if (rc != LEAP_OK) return rc;
    const bool keys_direct = laid_k || (direct_array(d_k, desc->k_item, desc->k_row, desc->k_head, desc->width) && direct_array(d_v, desc->v_item, desc->v_row, desc->v_head, desc->width));
    const bool queries_direct = laid_q || (direct_array(d_q, desc->q_item, desc->q_row, desc->q_head, desc->width) && direct_array(d_grad, grad_item, grad_row, grad_head, desc->width));
    return by_width(desc->width, [&](auto w) {
        constexpr int W = decltype(w)::value;
        int status = LEAP_OK;
        if (d_grad_table) {
            const dim3 grid((unsigned)(desc->heads * G.parts));
            by_flags([&](auto direct, auto few) {
                hipLaunchKernelGGL((k_grad_query<W, decltype(direct)::value, true, decltype(few)::value ? 1024 : LEAP_ATTENTION_BUCKETS>), grid, dim3(BLOCK), 0, st, G);
                return LEAP_OK;
            }, keys_direct, desc->buckets <= 1024);
            if ((status = launched()) != LEAP_OK) return status;
            const dim3 across((unsigned)((desc->buckets + BLOCK - 1) / BLOCK), (unsigned)desc->heads);
            hipLaunchKernelGGL(k_join_table, across, dim3(BLOCK), 0, st, G.part, G.parts, (int)desc->buckets, d_grad_table);
            status = launched();
        } else if (d_grad_q) {
            const dim3 grid((unsigned)(desc->batch * desc->heads * tiles));
            status = by_flags([&](auto direct, auto bias) {
                hipLaunchKernelGGL((k_grad_query<W, decltype(direct)::value, decltype(bias)::value, 0>), grid, dim3(BLOCK), 0, st, G);
                return launched();
            }, keys_direct, desc->d_table != nullptr);
        }
        if (status != LEAP_OK || !kept || !(d_grad_k || d_grad_v)) return status;
        const dim3 grid((unsigned)(desc->batch * desc->kv_heads * key_tiles));
        return by_flags([&](auto direct, auto bias) {
            hipLaunchKernelGGL((k_grad_key<W, decltype(direct)::value, decltype(bias)::value>), grid, dim3(BLOCK), 0, st, of_keys);
            return launched();
        }, queries_direct, desc->d_table != nullptr);
    });
}
