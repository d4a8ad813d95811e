// Attention's gradients.  With p the probabilities, formed again from the scores and each query's statistics, and
// dp = grad.v:  delta = grad.o (the sum of p dp over a query's keys),  ds = p (dp - delta),  grad_v = sum over queries of p grad,  grad_q = scale times the
// sum over keys of ds k,  grad_k = scale times the sum over queries of ds q,  and a bucket's number gets the sum of ds over its pairs.
//
// Two kernels, each the owner of what it writes, so that no sum depends on an order of arrival: k_grad_query has queries in its lanes and
// walks over keys as the forward pass does; k_grad_key has keys in its lanes and walks over queries.  Both form the scores and dp: seven products instead
// of the five of one kernel, which would have to add up grad_q over blocks.
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

// A query's statistics, and what its scores are lowered by: together where scores have no bias, which can be far larger than the logarithm.
struct query_stats {
    float most, log;
};
__device__ inline query_stats stats_of(const grad_args &G, int64_t row)
{
    return {G.stats[row * 2], G.stats[row * 2 + 1]};
}

constexpr int DELTA_LANES = LEAP_ATTENTION_WIDEST / 8, DELTA_ROWS = BLOCK / DELTA_LANES;

// delta: sixteen lanes a row.
__global__ __launch_bounds__(BLOCK) void k_delta(grad_args G)
{
    const attention_args &A = G.a;
    const int lane = threadIdx.x % DELTA_LANES;
    const int64_t row = (G.first + blockIdx.x) * DELTA_ROWS + threadIdx.x / DELTA_LANES;
    if (row >= (int64_t)A.batch * A.queries * A.heads) return;
    const int head = (int)(row % A.heads);
    const int64_t query = row / A.heads % A.queries, item = row / A.heads / A.queries;
    const auto halves = [](const u32x4 &v, int i) { return __uint_as_float(i % 2 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16); };
    const u32x4 g = row_piece(G.grad.data + item * G.grad.item + query * G.grad.row + head * G.grad.head, A.width, lane);
    const u32x4 o = row_piece(G.o + row * A.width, A.width, lane), rest = row_piece(G.rest + row * A.width, A.width, lane);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += halves(g, i) * (halves(o, i) + element<LEAP_F16>::to_float((uint16_t)(rest[i / 2] >> (i % 2 * 16))) * 0x1p-8f);
#pragma unroll
    for (int d = 1; d < DELTA_LANES; d *= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) G.delta[(item * A.heads + head) * (int64_t)A.queries + query] = sum;
}

// BUCKETS: room for the gradient of a table of up to so many (0: not wanted).
template <int DEEP, bool BIAS, int BUCKETS> __global__ __launch_bounds__(BLOCK) void k_grad_query(grad_args G)
{
    using tile = rows_tile<DEEP>;
    constexpr int STEPS = DEEP / 16, BLOCKS = DEEP / 32;
    const attention_args &A = G.a;
    __shared__ __attribute__((aligned(16))) uint8_t room[4 * tile::BYTES];
    __shared__ float table[BUCKETS ? WAVES * BUCKETS : 1];
    lds_byte *const lds = (lds_byte *)room;
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    const int tiles = (A.queries + COLS - 1) / COLS;
    const int64_t units = (int64_t)A.batch * tiles;
    float *const mine = table + wave * BUCKETS;
    if constexpr (BUCKETS != 0)
        for (int b = threadIdx.x; b < WAVES * BUCKETS; b += BLOCK) table[b] = 0.0f;

    const int64_t block = unit_of(blockIdx.x, gridDim.x);
    // a block a unit, the heads of an item apart; with a table the same head for all units of a block
    const int head = BUCKETS ? (int)(block / G.parts) : (int)(block / tiles % A.heads), kv_head = head / (A.heads / A.kv_heads);
    const int64_t from = BUCKETS ? block % G.parts : block / tiles / A.heads * tiles + block % tiles, step = BUCKETS ? G.parts : units;
    for (int64_t unit = from; unit < units; unit += step) {
        const int64_t item = unit / tiles;
        const int query = (int)(unit % tiles) * COLS + wave * 32 + lane % 32;
        const bool there = query < A.queries;
        const uint16_t *const k = A.k.data + item * A.k.item + kv_head * A.k.head, *const v = A.v.data + item * A.v.item + kv_head * A.v.head;
        const uint8_t *const mask = A.mask ? A.mask + item * A.mask_item : nullptr;
        bf16x8 q[STEPS], g[STEPS];
        {
            const uint16_t *const row = A.q.data + item * A.q.item + head * A.q.head + query * A.q.row;
            const uint16_t *const grad = G.grad.data + item * G.grad.item + head * G.grad.head + query * G.grad.row;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                q[s] = __builtin_bit_cast(bf16x8, there ? row_piece(row, A.width, s * 2 + lane / 32) : u32x4{0, 0, 0, 0});
                g[s] = __builtin_bit_cast(bf16x8, there ? row_piece(grad, A.width, s * 2 + lane / 32) : u32x4{0, 0, 0, 0});
            }
        }
        const int64_t row = (item * A.heads + head) * (int64_t)A.queries + query;
        const query_stats stats = there ? stats_of(G, row) : query_stats{0.0f, INFINITY};
        const float delta = there ? G.delta[row] : 0.0f, scale = A.scale * LOG2E, base = stats.most + stats.log;
        const int position = BIAS && there ? query_position(A, query) : 0;
        f32x16 sum[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) sum[b] = zeros();

        staged<DEEP> nk, nv;
        uint64_t bits = rows_there(mask, 0, A.keys, lane);
        if (bits) nk.fetch(k, A.k.row, 0, bits, A.width), nv.fetch(v, A.v.row, 0, bits, A.width);
        int turn = 0;
        __syncthreads();                                   // the unit before has read its tiles
        for (int64_t first = 0; first < A.keys; first += TILE) {
            const uint64_t next = rows_there(mask, first + TILE, A.keys, lane);
            if (!bits) {                                   // of all waves alike
                bits = next;
                if (bits) nk.fetch(k, A.k.row, first + TILE, bits, A.width), nv.fetch(v, A.v.row, first + TILE, bits, A.width);
                continue;
            }
            lds_byte *const kt = lds + turn * 2 * tile::BYTES, *const vt = kt + tile::BYTES;
            nk.store(kt), nv.store(vt);
            __syncthreads();
            turn ^= 1;
            if (next) nk.fetch(k, A.k.row, first + TILE, next, A.width), nv.fetch(v, A.v.row, first + TILE, next, A.width);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x16 x = zeros(), dp = zeros();
#pragma unroll
                for (int s = 0; s < STEPS; ++s) x = product(tile::along(kt, h * 32, s, lane), q[s], x);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) dp = product(tile::along(vt, h * 32, s, lane), g[s], dp);
                const uint32_t held = (uint32_t)(bits >> (h * 32)) >> (lane / 32 * 4);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float p;
                    int bucket = 0;
                    if constexpr (BIAS) {
                        const int64_t key = first + h * 32 + row_of(r) + lane / 32 * 4;
                        bucket = key < A.keys ? bucket_at(A, key_position(A, (int)key) - position) : 0;
                        p = __builtin_amdgcn_exp2f(x[r] * scale + table_value(A, head, bucket) - stats.most - stats.log);
                    } else {
                        p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], scale, -base));
                    }
                    if (~bits) p = held >> row_of(r) & 1 ? p : 0.0f;
                    x[r] = p * (dp[r] - delta);
                    if constexpr (BUCKETS != 0) __hip_atomic_fetch_add(&mine[bucket], x[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bf16x8 ds = eight(x, t);
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b) sum[b] = product(tile::across(kt, h * 32 + t * 16, b, lane), ds, sum[b]);
                }
            }
            bits = next;
        }
        if (G.grad_q) store_column<BLOCKS>(G.grad_q + ((item * A.queries + query) * A.heads + head) * A.width, A.width, sum, A.scale, lane, there);
    }
    if constexpr (BUCKETS != 0) {
        __syncthreads();
        for (int b = threadIdx.x; b < A.buckets; b += BLOCK) {
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += table[w * BUCKETS + b];
            G.part[block * A.buckets + b] = sum;
        }
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

template <int DEEP, bool BIAS> __global__ __launch_bounds__(BLOCK) void k_grad_key(grad_args G)
{
    using tile = rows_tile<DEEP>;
    constexpr int STEPS = DEEP / 16, BLOCKS = DEEP / 32;
    const attention_args &A = G.a;
    __shared__ __attribute__((aligned(16))) uint8_t room[4 * tile::BYTES];
    __shared__ __attribute__((aligned(16))) float most[2][TILE], log[2][TILE], delta[2][TILE];
    __shared__ __attribute__((aligned(16))) int place[2][TILE];
    lds_byte *const lds = (lds_byte *)room;
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
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
        const uint16_t *const krow = A.k.data + item * A.k.item + kv_head * A.k.head + key * A.k.row, *const vrow = A.v.data + item * A.v.item + kv_head * A.v.head + key * A.v.row;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            k[s] = __builtin_bit_cast(bf16x8, held ? row_piece(krow, A.width, s * 2 + lane / 32) : u32x4{0, 0, 0, 0});
            v[s] = __builtin_bit_cast(bf16x8, held ? row_piece(vrow, A.width, s * 2 + lane / 32) : u32x4{0, 0, 0, 0});
        }
        const int position = BIAS && there ? key_position(A, key) : 0;
        staged<DEEP> nq, ng;
        query_stats stats;
        float nd;
        int np = 0;
        // Step `at` of group * tiles: tile at % tiles of head at / tiles.
        const auto fetch = [&](int at) {
            const int head = kv_head * group + at / tiles;
            const int64_t first = (int64_t)(at % tiles) * TILE;
            const uint64_t bits = rows_there(nullptr, first, A.queries, lane);
            nq.fetch(A.q.data + item * A.q.item + head * A.q.head, A.q.row, first, bits, A.width);
            ng.fetch(G.grad.data + item * G.grad.item + head * G.grad.head, G.grad.row, first, bits, A.width);
            if (wave == 0) {
                const bool in = first + lane < A.queries;
                const int64_t row = (item * A.heads + head) * (int64_t)A.queries + first + lane;
                stats = in ? stats_of(G, row) : query_stats{0.0f, INFINITY};
                nd = in ? G.delta[row] : 0.0f;
                if (BIAS) np = in ? query_position(A, (int)first + lane) : 0;
            }
        };
        const int steps = group * tiles;
        if (steps) fetch(0);
        for (int at = 0; at < steps; ++at) {
            const int turn = at % 2, head = kv_head * group + at / tiles;
            lds_byte *const qt = lds + turn * 2 * tile::BYTES, *const gt = qt + tile::BYTES;
            nq.store(qt), ng.store(gt);
            if (wave == 0) {
                most[turn][lane] = BIAS ? stats.most : stats.most + stats.log;
                log[turn][lane] = stats.log;
                delta[turn][lane] = nd;
                place[turn][lane] = np;
            }
            __syncthreads();
            if (at + 1 < steps) fetch(at + 1);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x16 x = zeros(), dp = zeros();
#pragma unroll
                for (int s = 0; s < STEPS; ++s) x = product(tile::along(qt, h * 32, s, lane), k[s], x);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) dp = product(tile::along(gt, h * 32, s, lane), v[s], dp);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = h * 32 + row_of(r) + lane / 32 * 4;
                    float p;
                    if constexpr (BIAS)
                        p = __builtin_amdgcn_exp2f(x[r] * scale + table_value(A, head, bucket_at(A, position - place[turn][row])) - most[turn][row] - log[turn][row]);
                    else
                        p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], scale, -most[turn][row]));
                    x[r] = p;
                    dp[r] = p * (dp[r] - delta[turn][row]);
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bf16x8 p = eight(x, t), ds = eight(dp, t);
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b) {
                        gv[b] = product(tile::across(gt, h * 32 + t * 16, b, lane), p, gv[b]);
                        gk[b] = product(tile::across(qt, h * 32 + t * 16, b, lane), ds, gk[b]);
                    }
                }
            }
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

// Blocks that a head's units are dealt out to where the table's gradient is formed: each has room of its own for it.
int64_t table_parts(const leap_attention_desc *d)
{
    const int64_t units = d->batch * ((d->queries + COLS - 1) / COLS), most = d->heads < 1024 ? 2048 / d->heads : 2;
    return units < 1 ? 1 : units < most ? units : most;
}

int64_t delta_bytes(const leap_attention_desc *d) { return (d->batch * d->heads * d->queries * 4 + 15) / 16 * 16; }

}  // namespace

extern "C" int64_t leap_attention_backward_work(const leap_attention_desc *desc, int32_t with_table)
{
    if (bad_attention(desc)) return 0;
    return delta_bytes(desc) + (with_table && desc->d_table ? desc->heads * table_parts(desc) * desc->buckets * 4 : 0);
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
    if ((rows || d_grad_table) && unaligned(d_work)) return refuse(NO_WORK);
    const int64_t tiles = (desc->queries + COLS - 1) / COLS, key_tiles = (desc->keys + COLS - 1) / COLS;
    if (desc->batch * desc->heads * tiles >= (int64_t)1 << 24 || desc->batch * desc->kv_heads * key_tiles >= (int64_t)1 << 24) return refuse("more than 2^31 rows of heads");
    if ((int64_t)desc->heads / desc->kv_heads * ((desc->queries + TILE - 1) / TILE) >= (int64_t)1 << 31) return refuse("more than 2^37 queries share a key");
    const hipStream_t st = stream_of(hip_stream);
    grad_args G{arguments_of(desc, d_q, d_k, d_v), {(const uint16_t *)d_grad, grad_item, grad_row, grad_head}, (const uint16_t *)d_o, (const uint16_t *)d_rest,
                d_stats, (float *)d_work, (uint16_t *)d_grad_q, (uint16_t *)d_grad_k, (uint16_t *)d_grad_v, (float *)((char *)d_work + delta_bytes(desc)),
                (int32_t)table_parts(desc), 0};
    int rc = LEAP_OK;
    if (rows && (d_grad_q || d_grad_k || d_grad_v || d_grad_table))
        rc = over_blocks((rows + DELTA_ROWS - 1) / DELTA_ROWS, [&](int64_t first, unsigned blocks) {
            G.first = first;
            hipLaunchKernelGGL(k_delta, dim3(blocks), dim3(BLOCK), 0, st, G);
        });
    if (rc != LEAP_OK) return rc;
    return by_width(desc->width, [&](auto w) {
        constexpr int W = decltype(w)::value;
        int status = LEAP_OK;
        if (d_grad_table) {
            const dim3 grid((unsigned)(desc->heads * G.parts));
            if (desc->buckets <= 512) hipLaunchKernelGGL((k_grad_query<W, true, 512>), grid, dim3(BLOCK), 0, st, G);
            else hipLaunchKernelGGL((k_grad_query<W, true, LEAP_ATTENTION_BUCKETS>), grid, dim3(BLOCK), 0, st, G);
            if ((status = launched()) != LEAP_OK) return status;
            const dim3 across((unsigned)((desc->buckets + BLOCK - 1) / BLOCK), (unsigned)desc->heads);
            hipLaunchKernelGGL(k_join_table, across, dim3(BLOCK), 0, st, G.part, G.parts, (int)desc->buckets, d_grad_table);
            status = launched();
        } else if (d_grad_q && rows) {
            const dim3 grid((unsigned)(desc->batch * desc->heads * tiles));
            if (desc->d_table) hipLaunchKernelGGL((k_grad_query<W, true, 0>), grid, dim3(BLOCK), 0, st, G);
            else hipLaunchKernelGGL((k_grad_query<W, false, 0>), grid, dim3(BLOCK), 0, st, G);
            status = launched();
        }
        if (status != LEAP_OK || !kept || !(d_grad_k || d_grad_v)) return status;
        const dim3 grid((unsigned)(desc->batch * desc->kv_heads * key_tiles));
        if (desc->d_table) hipLaunchKernelGGL((k_grad_key<W, true>), grid, dim3(BLOCK), 0, st, G);
        else hipLaunchKernelGGL((k_grad_key<W, false>), grid, dim3(BLOCK), 0, st, G);
        return launched();
    });
}
