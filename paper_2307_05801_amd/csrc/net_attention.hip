// Attention, forward: o = sum over keys of exp(x) v / sum of exp(x), x = scale q.k + bias, in one pass over the keys.
//
// A block has 128 queries of a head, 32 to a wave, whose values stay in registers; it walks over the keys in tiles of 64, which all four waves
// read from shared memory.  A wave forms x for 32 keys by 32 queries with a lane a query (net_attention.h says why), keeps the largest so far, m, and
// the sum of exp2(x - m) of each query in that lane, and multiplies the values summed so far by exp2(m before - m now) where a query's m has grown.
#include "net_attention.h"

namespace {

using namespace net;

// What becomes of a query beside o.
struct forward_args {
    attention_args a;
    uint16_t *o;
    float *stats;
    uint16_t *rest;
};

// BIAS: with a table.  FINE: for a backward pass, which takes delta = grad.o off every product grad.v of a query: an o with its rounding, or with the probabilities',
// would spoil all of the query's alike, and in grad_q that adds up along what the keys have in common (keys and values with a common part as large as what
// differs, 512 keys: grad_q was 0.020 of its norm off, with four times as large a part 0.34; now 0.003 and 0.007, which is the rounding of ds).  So there the
// probabilities are the sum of two bfloat16, and what o's rounding leaves is kept.
template <int DEEP, bool BIAS, bool FINE> __global__ __launch_bounds__(BLOCK) void k_attention(forward_args F)
{
    using tile = rows_tile<DEEP>;
    constexpr int STEPS = DEEP / 16, BLOCKS = DEEP / 32;
    const attention_args &A = F.a;
    __shared__ __attribute__((aligned(16))) uint8_t room[4 * tile::BYTES];
    lds_byte *const lds = (lds_byte *)room;
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    const int tiles = (A.queries + COLS - 1) / COLS;
    const int64_t unit = unit_of(blockIdx.x, gridDim.x), item = unit / tiles / A.heads;
    const int head = (int)(unit / tiles % A.heads), kv_head = head / (A.heads / A.kv_heads);
    const int query = (int)(unit % tiles) * COLS + wave * 32 + lane % 32;
    const bool there = query < A.queries;
    const uint16_t *const k = A.k.data + item * A.k.item + kv_head * A.k.head, *const v = A.v.data + item * A.v.item + kv_head * A.v.head;
    const uint8_t *const mask = A.mask ? A.mask + item * A.mask_item : nullptr;

    bf16x8 q[STEPS];
    {
        const uint16_t *const row = A.q.data + item * A.q.item + head * A.q.head + query * A.q.row;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) q[s] = __builtin_bit_cast(bf16x8, there ? row_piece(row, A.width, s * 2 + lane / 32) : u32x4{0, 0, 0, 0});
    }
    const int position = BIAS && there ? query_position(A, query) : 0;
    const float scale = A.scale * LOG2E;
    f32x16 o[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) o[b] = zeros();
    float m = -INFINITY, sum = 0.0f;

    staged<DEEP> nk, nv;
    uint64_t bits = rows_there(mask, 0, A.keys, lane);
    if (bits) nk.fetch(k, A.k.row, 0, bits, A.width), nv.fetch(v, A.v.row, 0, bits, A.width);
    int turn = 0;
    for (int64_t first = 0; first < A.keys; first += TILE) {
        const uint64_t next = rows_there(mask, first + TILE, A.keys, lane);
        if (!bits) {                                   // of all waves alike
            bits = next;
            if (bits) nk.fetch(k, A.k.row, first + TILE, bits, A.width), nv.fetch(v, A.v.row, first + TILE, bits, A.width);
            continue;
        }
        lds_byte *const kt = lds + turn * 2 * tile::BYTES, *const vt = kt + tile::BYTES;
        nk.store(kt), nv.store(vt);
        __syncthreads();                               // two pairs of tiles: the one written next was read before the last barrier
        turn ^= 1;
        if (next) nk.fetch(k, A.k.row, first + TILE, next, A.width), nv.fetch(v, A.v.row, first + TILE, next, A.width);

        f32x16 x[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            x[h] = zeros();
#pragma unroll
            for (int s = 0; s < STEPS; ++s) x[h] = product(tile::along(kt, h * 32, s, lane), q[s], x[h]);
        }
        if constexpr (BIAS) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int64_t key = first + h * 32 + row_of(r) + lane / 32 * 4;
                    x[h][r] = key < A.keys ? x[h][r] * scale + table_value(A, head, bucket_at(A, key_position(A, (int)key) - position)) : 0.0f;
                }
        }
        if (~bits) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t mine = (uint32_t)(bits >> (h * 32)) >> (lane / 32 * 4);
#pragma unroll
                for (int r = 0; r < 16; ++r) x[h][r] = mine >> row_of(r) & 1 ? x[h][r] : -INFINITY;
            }
        }
        float most = x[0][0];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, x[h][r]);
        most = column_max(most);
        const float now = fmaxf(m, BIAS ? most : most * scale), base = now == -INFINITY ? 0.0f : now;
        if (__any(now > m)) {
            const float by = __builtin_amdgcn_exp2f(m - base);
            sum *= by;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) o[b] *= by;
        }
        m = now;
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
                const bf16x8 p = eight(x[h], t), low = FINE ? rest_of_eight(x[h], t) : p;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    const bf16x8 values = tile::across(vt, h * 32 + t * 16, b, lane);
                    o[b] = product(values, p, o[b]);
                    if constexpr (FINE) o[b] = product(values, low, o[b]);
                }
            }
        bits = next;
    }
    sum = column_sum(sum);
    const float by = sum != 0.0f ? 1.0f / sum : 0.0f;                 // (a sum that is not a number: so is o)
    const int64_t row = (item * A.queries + query) * A.heads + head;
    store_column<BLOCKS>(F.o + row * A.width, A.width, o, by, lane, there);
    if (FINE && there && lane < 32) {
        float *const to = F.stats + ((item * A.heads + head) * (int64_t)A.queries + query) * 2;
        to[0] = sum != 0.0f ? m : 0.0f;
        to[1] = sum != 0.0f ? __builtin_amdgcn_logf(sum) : INFINITY;
    }
    if constexpr (FINE) {
        if (there)
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = b * 32 + row_of(r) + lane / 32 * 4;
                    if (at < A.width) F.rest[row * A.width + at] = element<LEAP_F16>::from_float(rest_of_bf16(o[b][r] * by) * 256.0f);
                }
    }
}

}  // namespace

namespace net {

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
        if (!d->d_bucket_of || d->offsets < 1 || d->offsets > most) return "the table needs the buckets of 1 to 2^30 differences";
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

extern "C" int64_t leap_attention_work(const leap_attention_desc *desc)
{
    (void)desc;
    return 0;
}

extern "C" int leap_attention(const leap_attention_desc *desc, const void *d_q, const void *d_k, const void *d_v, void *d_o, float *d_stats, void *d_rest,
                              void *d_work, void *hip_stream)
{
    (void)d_work;
    if (const char *why = bad_attention(desc)) return refuse(why);
    if (!desc->batch || !desc->queries) return LEAP_OK;
    if (!d_q || !d_o || (desc->keys && (!d_k || !d_v))) return refuse("null data pointer");
    if (!d_rest != !d_stats) return refuse("statistics and what o's rounding leaves: both or neither");
    const forward_args F{arguments_of(desc, d_q, d_k, d_v), (uint16_t *)d_o, d_stats, (uint16_t *)d_rest};
    const int64_t blocks = desc->batch * desc->heads * ((desc->queries + COLS - 1) / COLS);
    if (blocks >= (int64_t)1 << 24) return refuse("more than 2^31 rows of heads");
    return by_width(desc->width, [&](auto w) {
        constexpr int W = decltype(w)::value;
        const dim3 grid((unsigned)blocks), block(BLOCK);
        const hipStream_t st = stream_of(hip_stream);
        if (desc->d_table && d_rest) hipLaunchKernelGGL((k_attention<W, true, true>), grid, block, 0, st, F);
        else if (desc->d_table) hipLaunchKernelGGL((k_attention<W, true, false>), grid, block, 0, st, F);
        else if (d_rest) hipLaunchKernelGGL((k_attention<W, false, true>), grid, block, 0, st, F);
        else hipLaunchKernelGGL((k_attention<W, false, false>), grid, block, 0, st, F);
        return launched();
    });
}
