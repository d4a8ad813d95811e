// Group norm with an activation, channels last, and its gradients.
//
// A thread has eight neighbouring values of an item at a time and steps from voxel to voxel such that they are always the same channels, whose
// mean, weight, ... stay in its registers.  Where rows have no gaps and the channels are no multiple of 8, the values are cut in eights regardless of rows: after
// `positions` eights the channels begin anew, so that no length costs more than its values.
//
// Sums over a group are formed in three stages that depend on the sizes alone: a thread's values (means and squares about them, a piece of eight voxels exactly in two
// passes over registers, pieces joined by their means; 512 voxels at most), a block's threads, and in 64 bits the blocks of an item.  Memory bounds it all: x is read
// twice forward, x and the gradient twice backward.  So a few items (or one) at a time are read for their sums and, in the opposite order, again, before the next: the second time
// part of them comes from the cache of 256 MB.  (Rows with gaps whose channels are no multiple of 8 are read value by value at their ends, and registers spill in the sums: 5.9 million voxels of 20
// channels, bfloat16, a step 836 us, 436 without gaps.) An item of 2^21 voxels of 64 channels in bfloat16: moments 53 us (5.0 TB/s), activation 97 (5.5), sums 118 (4.5), gradient 161 (5.0).
#include "../../include/leap_networks.h"
#include "act_common.h"

namespace {

using namespace act;

constexpr int BLOCK = 256;
constexpr int PIECE = 8;                    // voxels a thread takes at once for their moments,
template <int TYPE> constexpr int AT_ONCE = TYPE == LEAP_F32 ? 2 : 4;      // and x and a gradient (of 32 bytes or 16): as many as leave room for four blocks a compute unit

// How an item's values are dealt out to threads.
struct dealing {
    int64_t voxels, periods;                // periods of `positions` eights: a voxel, or as many as whole eights need
    int64_t length;                         // periods of a block
    int32_t channels, groups, size;         // size: channels of a group
    int32_t positions, strips, segments;    // eights of a period; blocks along the voxels, across a period
    int32_t rows;                           // voxels of a period
};

struct array {
    const void *data;
    int64_t item, row;                      // distances in elements
};

// A thread's part in it.
struct part {
    int position, turn, turns, count;       // which eight of a period, which of the block's periods at once; values there
    int64_t from, to, whole;                // periods; up to which they are known to be complete
    int64_t item, strip;                    // item: of those at once, which the arrays' addresses begin with

    __device__ inline part(const dealing &D, bool backwards)
    {
        int64_t block = backwards ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
        const int segment = (int)(block % D.segments);
        block /= D.segments;
        strip = block % D.strips, item = block / D.strips;
        turns = D.positions < BLOCK ? BLOCK / D.positions : 1;
        position = D.segments > 1 ? segment * BLOCK + (int)threadIdx.x : (int)threadIdx.x % D.positions;
        turn = D.segments > 1 ? 0 : (int)threadIdx.x / D.positions;
        const bool there = position < D.positions && turn < turns;
        count = !there ? 0 : D.rows > 1 || D.channels - position * CHUNK >= CHUNK ? CHUNK : D.channels - position * CHUNK;
        from = strip * D.length + turn, to = (strip + 1) * D.length < D.periods ? (strip + 1) * D.length : D.periods;
        if (!there) from = to;
        whole = D.rows > 1 && to == D.periods ? to - 1 : to;
    }
    __device__ inline int channel(const dealing &D, int i) const { return D.rows > 1 ? (position * CHUNK + i) % D.channels : position * CHUNK + i; }
    // Values from one period to the next in an item of rows `row` apart; where its eight of a period begin, and how many there are.
    __device__ inline int64_t step(const dealing &D, int64_t row) const { return D.rows > 1 ? (int64_t)D.positions * CHUNK : row; }
    __device__ inline int64_t at(const dealing &D, int64_t period, int64_t row) const { return period * step(D, row) + position * CHUNK; }
    __device__ inline int there(const dealing &D, int64_t period) const
    {
        if (D.rows == 1) return count;
        const int64_t left = D.voxels * D.channels - at(D, period, 0);
        return left >= CHUNK ? CHUNK : left > 0 ? (int)left : 0;
    }
};

// Eight values as memory has them.
template <int TYPE> struct eight_of {
    using raw = typename element<TYPE>::raw;
    raw r[CHUNK];
    // FULL: all of them are there.
    template <bool FULL> __device__ inline void load(const raw *p, int n)
    {
        if (FULL || n >= CHUNK) {
            __builtin_memcpy(r, p, sizeof r);
        } else {
#pragma unroll
            for (int i = 0; i < CHUNK; ++i) r[i] = i < n ? p[i] : raw(0);
        }
    }
    __device__ inline float operator[](int i) const { return element<TYPE>::to_float(r[i]); }
};

// step(periods at once, the first of them, values there) for all of a thread's periods: AT_ONCE of them, and one at a time what is left.
template <int AT_ONCE, class F> __device__ inline void over_periods(const dealing &D, const part &P, F &&f)
{
    int64_t p = P.from;
    for (; p + (AT_ONCE - 1) * P.turns < P.whole; p += AT_ONCE * P.turns) f(std::integral_constant<int, AT_ONCE>{}, p, P.count);
    for (; p < P.to; p += P.turns) f(std::integral_constant<int, 1>{}, p, P.there(D, p));
}

__device__ inline float value_at(const void *p, int type, int64_t i)
{
    return type == LEAP_F32 ? ((const float *)p)[i] : type == LEAP_BF16 ? element<LEAP_BF16>::to_float(((const uint16_t *)p)[i]) : element<LEAP_F16>::to_float(((const uint16_t *)p)[i]);
}

struct group_args {
    dealing deal;
    array x, grad;
    const void *weight, *bias;
    int32_t weight_type;
    float eps;
    float *stats;                           // [items][groups][2]
    const float *coefficients;              // [items][groups][2]
    float *parts;
    void *out;
    int64_t first;
    bool past;                              // outputs past the caches
};

struct moments {
    float n, mean, square;                  // square: sum of squares about the mean
    __device__ inline void join(const moments &o)
    {
        const float all = n + o.n;
        if (o.n == 0.0f) return;
        const float share = o.n / all, d = o.mean - mean, far = n > 0.0f ? d * d : 0.0f;       // (the first values' square may be beyond what a float holds)
        mean += d * share;
        square += o.square + far * (n * share);
        n = all;
    }
};

// Each slot (eight * 8 + value) of a period: its moments over the block's voxels, to parts [items][strips][slots].
template <int TYPE, bool FULL> __global__ __launch_bounds__(BLOCK, 4) void k_group_moments(group_args A)
{
    const dealing &D = A.deal;
    const part P(D, false);
    using raw = typename element<TYPE>::raw;
    const raw *const x = (const raw *)A.x.data + P.item * A.x.item + P.position * CHUNK;
    const int64_t step = P.step(D, A.x.row);
    float n = 0.0f, mean[CHUNK] = {}, square[CHUNK] = {};
    int64_t p = P.from;
    for (; p + (PIECE - 1) * P.turns < P.whole; p += PIECE * P.turns) {
        eight_of<TYPE> v[PIECE];
#pragma unroll
        for (int u = 0; u < PIECE; ++u) v[u].template load<FULL>(x + (p + u * P.turns) * step, P.count);
        const float all = n + PIECE, share = PIECE / all, weight = n * share;
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) {
            float m = 0.0f, s = 0.0f;
#pragma unroll
            for (int u = 0; u < PIECE; ++u) m += v[u][i];
            m *= 1.0f / PIECE;
#pragma unroll
            for (int u = 0; u < PIECE; ++u) s += (v[u][i] - m) * (v[u][i] - m);
            const float d = m - mean[i], far = n > 0.0f ? d * d : 0.0f;
            mean[i] += d * share;
            square[i] += s + far * weight;
        }
        n = all;
    }
    moments all[CHUNK];
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) all[i] = {n, mean[i], square[i]};
    for (; p < P.to; p += P.turns) {
        const int there = P.there(D, p);
        eight_of<TYPE> v;
        v.template load<false>(x + p * step, there);
#pragma unroll
        for (int i = 0; i < CHUNK; ++i)
            if (i < there) all[i].join({1.0f, v[i], 0.0f});
    }
    // the threads that have the same eight, two by two
    __shared__ moments room[CHUNK][BLOCK];
    int half = 1;
    while (half < P.turns) half *= 2;
    for (half /= 2; half > 0; half /= 2) {
        __syncthreads();
        if (P.turn >= half && P.turn < 2 * half)
#pragma unroll
            for (int i = 0; i < CHUNK; ++i) room[i][threadIdx.x] = all[i];
        __syncthreads();
        if (P.turn < half && P.turn + half < P.turns)
#pragma unroll
            for (int i = 0; i < CHUNK; ++i) all[i].join(room[i][threadIdx.x + half * D.positions]);
    }
    if (P.turn == 0 && P.position < D.positions) {
        moments *const to = (moments *)A.parts + ((P.item * D.strips + P.strip) * D.positions + P.position) * CHUNK;
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) to[i] = all[i];
    }
}

constexpr int WIDE = 1024;                 // threads of a block that joins parts

__device__ inline double block_sum(double v, double *room)
{
    room[threadIdx.x] = v;
    __syncthreads();
    for (int half = WIDE / 2; half > 0; half /= 2) {
        if ((int)threadIdx.x < half) room[threadIdx.x] += room[threadIdx.x + half];
        __syncthreads();
    }
    v = room[0];
    __syncthreads();
    return v;
}

// mean and rstd of a group, a block each.
__global__ __launch_bounds__(WIDE) void k_group_stats(group_args A)
{
    const dealing &D = A.deal;
    __shared__ double room[WIDE];
    const int64_t unit = A.first + blockIdx.x, item = unit / D.groups, slots = (int64_t)D.positions * CHUNK;
    const int group = (int)(unit % D.groups), each = D.rows * D.size;           // slots of a strip
    const moments *const from = (const moments *)A.parts + item * D.strips * slots + group * D.size;
    // f(moments) for a thread's share: some of a strip's slots of every few strips
    const auto over = [&](auto &&f) {
        const int wide = each < WIDE ? each : WIDE, high = WIDE / wide;
        if ((int)threadIdx.x >= wide * high) return;
        for (int e = threadIdx.x % wide; e < each; e += wide) {
            const moments *const at = from + e / D.size * D.channels + e % D.size;
#pragma unroll 4
            for (int s = threadIdx.x / wide; s < D.strips; s += high) f(at[s * slots]);
        }
    };
    double sum = 0.0, square = 0.0;
    over([&](const moments &m) { sum += (double)m.n * m.mean; });
    const double values = (double)D.voxels * D.size, mean = block_sum(sum, room) / values;
    over([&](const moments &m) { square += m.square + m.n * (m.mean - mean) * (m.mean - mean); });
    square = block_sum(square, room) / values;
    if (threadIdx.x == 0) A.stats[unit * 2] = (float)mean, A.stats[unit * 2 + 1] = (float)(1.0 / sqrt(square + A.eps));
}

// What a thread knows of its eight channels: u = (x - mean) by + bias, by = rstd weight.
struct known {
    float mean[CHUNK], by[CHUNK], bias[CHUNK];
    __device__ inline known(const group_args &A, const part &P)
    {
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) {
            const bool there = i < P.count;
            const int c = there ? P.channel(A.deal, i) : 0;
            mean[i] = there ? A.stats[group_of(A, P, i) * 2] : 0.0f;
            by[i] = !there ? 0.0f : A.stats[group_of(A, P, i) * 2 + 1] * (A.weight ? value_at(A.weight, A.weight_type, c) : 1.0f);
            bias[i] = there && A.bias ? value_at(A.bias, A.weight_type, c) : 0.0f;
        }
    }
    static __device__ inline int64_t group_of(const group_args &A, const part &P, int i) { return P.item * A.deal.groups + (i < P.count ? P.channel(A.deal, i) : 0) / A.deal.size; }
    // the activation's argument, in both passes from the same steps
    __device__ inline float argument(float v, int i) const { return __builtin_fmaf(v - mean[i], by[i], bias[i]); }
};

template <int TYPE> __device__ inline float gate(float u) { return TYPE == LEAP_F32 ? fine_sigmoid(u) : sigmoid(u); }
template <int TYPE, int ACTIVATION> __device__ inline float activated(float u) { return ACTIVATION == LEAP_SILU ? u * gate<TYPE>(u) : ACTIVATION == LEAP_RELU ? (u < 0.0f ? 0.0f : u) : u; }
template <int TYPE, int ACTIVATION> __device__ inline float slope(float u)
{
    if (ACTIVATION == LEAP_SILU) {
        const float s = gate<TYPE>(u);
        return s * __builtin_fmaf(u, 1.0f - s, 1.0f);
    }
    return ACTIVATION == LEAP_RELU && !(u > 0.0f) ? 0.0f : 1.0f;
}

template <int TYPE, bool FULL, int ACTIVATION> __global__ __launch_bounds__(BLOCK, 4) void k_group_apply(group_args A)
{
    const dealing &D = A.deal;
    const part P(D, true);
    using raw = typename element<TYPE>::raw;
    const raw *const x = (const raw *)A.x.data + P.item * A.x.item + P.position * CHUNK;
    raw *const y = (raw *)A.out + P.item * D.voxels * D.channels + P.position * CHUNK;
    const int64_t step = P.step(D, A.x.row), out = P.step(D, D.channels);
    const known K(A, P);
    over_periods<AT_ONCE<TYPE> * 2>(D, P, [&](auto at_once, int64_t p, int n) {
        constexpr int N = decltype(at_once)::value;
        eight_of<TYPE> v[N];
#pragma unroll
        for (int u = 0; u < N; ++u) v[u].template load<FULL && N != 1>(x + (p + u * P.turns) * step, n);
#pragma unroll
        for (int u = 0; u < N; ++u) {
            float o[CHUNK];
#pragma unroll
            for (int i = 0; i < CHUNK; ++i) o[i] = activated<TYPE, ACTIVATION>(K.argument(v[u][i], i));
            store8<TYPE>(y, (p + u * P.turns) * out, FULL && N != 1 ? CHUNK : n, o, A.past);
        }
    });
}

// Few values, whole groups of eights: a block has a group of an item in its registers, which takes one launch instead of three (256 voxels of 64 channels: 6.8 us instead of 22).
constexpr int SMALL_EIGHTS = 8;            // of a thread
constexpr int64_t SMALL_GROUP = (int64_t)BLOCK * SMALL_EIGHTS * CHUNK, SMALL = (int64_t)1 << 20;        // values of a group, and of all: neighbouring groups share lines of memory

// The same over a block of BLOCK threads.
__device__ inline double small_sum(double v, double *room)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    __syncthreads();
    if (threadIdx.x % 64 == 0) room[threadIdx.x / 64] = v;
    __syncthreads();
    return (room[0] + room[1]) + (room[2] + room[3]);
}

template <int TYPE, int ACTIVATION> __global__ __launch_bounds__(BLOCK) void k_group_small(group_args A)
{
    const dealing &D = A.deal;
    using raw = typename element<TYPE>::raw;
    __shared__ double room[BLOCK / 64];
    const int64_t unit = A.first + blockIdx.x, item = unit / D.groups;
    const int group = (int)(unit % D.groups), each = D.size / CHUNK, all = (int)D.voxels * each;
    const raw *const x = (const raw *)A.x.data + item * A.x.item + group * D.size;
    raw *const y = (raw *)A.out + item * D.voxels * D.channels + group * D.size;
    eight_of<TYPE> v[SMALL_EIGHTS];
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < SMALL_EIGHTS; ++j) {
        const int id = j * BLOCK + (int)threadIdx.x;
        if (id >= all) continue;
        v[j].template load<true>(x + id / each * A.x.row + id % each * CHUNK, CHUNK);
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) sum += v[j][i];
    }
    const double values = (double)D.voxels * D.size, exact = small_sum(sum, room) / values;
    double square = 0.0;
#pragma unroll
    for (int j = 0; j < SMALL_EIGHTS; ++j)
        if (j * BLOCK + (int)threadIdx.x < all) {
#pragma unroll
            for (int i = 0; i < CHUNK; ++i) square += (v[j][i] - exact) * (v[j][i] - exact);
        }
    const float mean = (float)exact, rstd = (float)(1.0 / sqrt(small_sum(square, room) / values + A.eps));
    if (A.stats && threadIdx.x == 0) A.stats[unit * 2] = mean, A.stats[unit * 2 + 1] = rstd;
#pragma unroll
    for (int j = 0; j < SMALL_EIGHTS; ++j) {
        const int id = j * BLOCK + (int)threadIdx.x, c = group * D.size + id % each * CHUNK;
        if (id >= all) continue;
        float o[CHUNK];
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) {
            const float by = rstd * (A.weight ? value_at(A.weight, A.weight_type, c + i) : 1.0f), bias = A.bias ? value_at(A.bias, A.weight_type, c + i) : 0.0f;
            o[i] = activated<TYPE, ACTIVATION>(__builtin_fmaf(v[j][i] - mean, by, bias));         // as known::argument has it
        }
        store8<TYPE>(y, (int64_t)(id / each) * D.channels + id % each * CHUNK, CHUNK, o);
    }
}

// Each slot's sums of du and of du h over the block's voxels, to parts [items][strips][slots][2].
template <int TYPE, bool FULL, int ACTIVATION> __global__ __launch_bounds__(BLOCK, 4) void k_group_sums(group_args A)
{
    const dealing &D = A.deal;
    const part P(D, false);
    using raw = typename element<TYPE>::raw;
    const raw *const x = (const raw *)A.x.data + P.item * A.x.item + P.position * CHUNK, *const grad = (const raw *)A.grad.data + P.item * A.grad.item + P.position * CHUNK;
    const int64_t step = P.step(D, A.x.row), grad_step = P.step(D, A.grad.row);
    const known K(A, P);
    float one[CHUNK] = {}, two[CHUNK] = {};                   // two: of du (x - mean), rstd comes at the end
    over_periods<TYPE == LEAP_F32 && ACTIVATION == LEAP_SILU ? 2 : 4>(D, P, [&](auto at_once, int64_t p, int n) {
        constexpr int N = decltype(at_once)::value;
        eight_of<TYPE> v[N], g[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            v[u].template load<FULL && N != 1>(x + (p + u * P.turns) * step, n);
            g[u].template load<FULL && N != 1>(grad + (p + u * P.turns) * grad_step, n);
        }
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int i = 0; i < CHUNK; ++i) {
                const float du = g[u][i] * slope<TYPE, ACTIVATION>(K.argument(v[u][i], i));
                if (N == 1 && i >= n) continue;
                one[i] += du;                                  // (MOST_PERIODS of them at most)
                two[i] = __builtin_fmaf(du, v[u][i] - K.mean[i], two[i]);
            }
    });
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) two[i] *= P.count ? A.stats[known::group_of(A, P, i) * 2 + 1] : 0.0f;
    __shared__ float2 room[CHUNK][BLOCK];
    int half = 1;
    while (half < P.turns) half *= 2;
    for (half /= 2; half > 0; half /= 2) {
        __syncthreads();
        if (P.turn >= half && P.turn < 2 * half)
#pragma unroll
            for (int i = 0; i < CHUNK; ++i) room[i][threadIdx.x] = make_float2(one[i], two[i]);
        __syncthreads();
        if (P.turn < half && P.turn + half < P.turns)
#pragma unroll
            for (int i = 0; i < CHUNK; ++i) {
                const float2 o = room[i][threadIdx.x + half * D.positions];
                one[i] += o.x, two[i] += o.y;
            }
    }
    if (P.turn == 0 && P.position < D.positions) {
        float2 *const to = (float2 *)A.parts + ((P.item * D.strips + P.strip) * D.positions + P.position) * CHUNK;
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) to[i] = make_float2(one[i], two[i]);
    }
}

// A group, a block each: its channels' sums over the item, to channel_sums [items][channels][2], and the means over the group of du weight and du weight h.
__global__ __launch_bounds__(WIDE) void k_group_coefficients(group_args A, double *channel_sums, float *coefficients)
{
    const dealing &D = A.deal;
    __shared__ double room[2][WIDE];
    const int64_t unit = A.first + blockIdx.x, item = unit / D.groups, slots = (int64_t)D.positions * CHUNK;
    const int group = (int)(unit % D.groups);
    const float2 *const from = (const float2 *)A.parts + item * D.strips * slots;
    const int wide = D.size < WIDE ? D.size : WIDE, high = WIDE / wide, col = threadIdx.x % wide, row = threadIdx.x / wide;
    double one = 0.0, two = 0.0;
    for (int c0 = 0; c0 < D.size; c0 += wide) {
        const int c = c0 + col, channel = group * D.size + c;
        double a = 0.0, b = 0.0;
        if (c < D.size && row < high)
            for (int r = 0; r < D.rows; ++r)
#pragma unroll 4
                for (int s = row; s < D.strips; s += high) {
                    const float2 v = from[s * slots + r * D.channels + channel];
                    a += v.x, b += v.y;
                }
        __syncthreads();
        room[0][threadIdx.x] = a, room[1][threadIdx.x] = b;
        __syncthreads();
        int top = 1;                           // rows of threads, two by two
        while (top < high) top *= 2;
        for (int half = top / 2; half > 0; half /= 2) {
            if (row < half && row + half < high) {
                room[0][threadIdx.x] += room[0][threadIdx.x + half * wide];
                room[1][threadIdx.x] += room[1][threadIdx.x + half * wide];
            }
            __syncthreads();
        }
        if (row == 0 && c < D.size) {
            a = room[0][threadIdx.x], b = room[1][threadIdx.x];
            double *const to = channel_sums + (item * D.channels + channel) * 2;
            to[0] = a, to[1] = b;
            const double w = A.weight ? value_at(A.weight, A.weight_type, channel) : 1.0f;
            one += w * a, two += w * b;
        }
    }
    const double m = (double)D.voxels * D.size;
    __syncthreads();
    one = block_sum(row == 0 ? one : 0.0, room[0]);
    two = block_sum(row == 0 ? two : 0.0, room[0]);
    if (threadIdx.x == 0) coefficients[unit * 2] = (float)(one / m), coefficients[unit * 2 + 1] = (float)(two / m);
}

// grad_weight, grad_bias: the channels' sums over the items, after those `before` them (null: none); to `after` as they are where more items follow.
template <int WTYPE>
__global__ __launch_bounds__(BLOCK) void k_group_weights(const double *channel_sums, int64_t items, int channels, const double *before, double *after, void *grad_weight, void *grad_bias)
{
    using raw = typename element<WTYPE>::raw;
    const int c = blockIdx.x * BLOCK + threadIdx.x;
    if (c >= channels) return;
    double one = before ? before[c * 2] : 0.0, two = before ? before[c * 2 + 1] : 0.0;
#pragma unroll 4
    for (int64_t n = 0; n < items; ++n) one += channel_sums[(n * channels + c) * 2], two += channel_sums[(n * channels + c) * 2 + 1];
    if (after) {
        after[c * 2] = one, after[c * 2 + 1] = two;
        return;
    }
    if (grad_bias) ((raw *)grad_bias)[c] = element<WTYPE>::from_float((float)one);
    if (grad_weight) ((raw *)grad_weight)[c] = element<WTYPE>::from_float((float)two);
}

template <int TYPE, bool FULL, int ACTIVATION> __global__ __launch_bounds__(BLOCK, 4) void k_group_grad(group_args A)
{
    const dealing &D = A.deal;
    const part P(D, true);
    using raw = typename element<TYPE>::raw;
    const raw *const x = (const raw *)A.x.data + P.item * A.x.item + P.position * CHUNK, *const grad = (const raw *)A.grad.data + P.item * A.grad.item + P.position * CHUNK;
    raw *const to = (raw *)A.out + P.item * D.voxels * D.channels + P.position * CHUNK;
    const int64_t step = P.step(D, A.x.row), grad_step = P.step(D, A.grad.row), out = P.step(D, D.channels);
    const known K(A, P);
    // rstd (du weight - first - h second) = du by - one - (x - mean) two
    float one[CHUNK], two[CHUNK];
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) {
        const int64_t g = P.count ? known::group_of(A, P, i) : 0;
        const float rstd = A.stats[g * 2 + 1];
        one[i] = A.coefficients[g * 2] * rstd, two[i] = A.coefficients[g * 2 + 1] * rstd * rstd;
    }
    over_periods<AT_ONCE<TYPE>>(D, P, [&](auto at_once, int64_t p, int n) {
        constexpr int N = decltype(at_once)::value;
        eight_of<TYPE> v[N], g[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            v[u].template load<FULL && N != 1>(x + (p + u * P.turns) * step, n);
            g[u].template load<FULL && N != 1>(grad + (p + u * P.turns) * grad_step, n);
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            float o[CHUNK];
#pragma unroll
            for (int i = 0; i < CHUNK; ++i)
                o[i] = g[u][i] * slope<TYPE, ACTIVATION>(K.argument(v[u][i], i)) * K.by[i] - one[i] - (v[u][i] - K.mean[i]) * two[i];
            store8<TYPE>(to, (p + u * P.turns) * out, FULL && N != 1 ? CHUNK : n, o, A.past);
        }
    });
}

// ---- host side ----

int64_t divisor(int64_t a, int64_t b) { return b ? divisor(b, a % b) : a; }

// Periods of a thread at most, since its sums are floats; it has that many of an item of 2^30 values dealt out to 1024 blocks, and larger items have more blocks.
constexpr int64_t MOST_PERIODS = 512;

// flat: rows of both arrays have no gaps.
dealing dealing_of(int64_t items, int64_t voxels, int64_t channels, int64_t groups, bool flat)
{
    dealing D;
    const int64_t common = divisor(channels, CHUNK);
    D.voxels = voxels;
    D.channels = (int32_t)channels, D.groups = (int32_t)groups, D.size = (int32_t)(channels / groups);
    D.rows = flat ? (int32_t)(CHUNK / common) : 1;
    D.positions = (int32_t)(D.rows > 1 ? channels / common : (channels + CHUNK - 1) / CHUNK);
    D.periods = (voxels + D.rows - 1) / D.rows;
    D.segments = (D.positions + BLOCK - 1) / BLOCK;
    const int64_t turns = D.positions < BLOCK ? BLOCK / D.positions : 1;
    // enough blocks for the chip, and no fewer than a few pieces of each thread
    int64_t strips = 1024 / (items * D.segments > 0 ? items * D.segments : 1);
    const int64_t most = D.periods / (turns * 2 * PIECE);
    strips = strips < most ? strips : most;
    const int64_t least = (D.periods + turns * MOST_PERIODS - 1) / (turns * MOST_PERIODS);
    strips = strips < least ? least : strips;
    strips = strips < 1 ? 1 : strips;
    D.length = (D.periods + strips - 1) / strips;
    D.length = (D.length + turns - 1) / turns * turns;
    if (D.length < 1) D.length = 1;
    D.strips = (int32_t)((D.periods + D.length - 1) / D.length);
    if (D.strips < 1) D.strips = 1;
    return D;
}

const char *bad_group(int64_t items, int64_t voxels, int64_t channels, int64_t groups)
{
    if (items < 0 || voxels < 0 || channels < 1) return "sizes must not be negative, and there are channels";
    if (groups < 1 || channels % groups) return "channels must be a multiple of the groups";
    if (channels > MOST_COLS || voxels > MOST_VALUES / channels || items > MOST_VALUES / channels / (voxels ? voxels : 1) || items > ((int64_t)1 << 31) / channels)
        return "more than 2^20 channels, 2^42 values or 2^31 channels of items";
    return nullptr;
}

const char *bad_distances(int64_t item, int64_t row, int64_t items, int64_t voxels, int64_t channels)
{
    if (item < 0 || item > ((int64_t)1 << 58) / (items + 1)) return "the distance of items is negative or reaches beyond what addresses hold";
    return bad_stride(row, voxels, channels);
}

constexpr int64_t AT_ONCE_FORWARD = (int64_t)1 << 26, AT_ONCE_BACKWARD = (int64_t)1 << 25;

// Items that are read for their sums and again before the next: `values` of x, or one.  The workspace is theirs alone, since the stream orders what works on them before
// what works on the next.  An item has no fewer slots than channels however few its voxels are, so those at once have no more than an eighth of all values, or 2^20; and values are cut
// regardless of rows where an item has at least eight periods of them: with a voxel of 63 channels to an item a period would be eight times what there is.
// Channels' sums are added up after `held` items, a multiple of `at_once`.
struct plan {
    dealing deal;
    int64_t at_once, held;

    // flat: rows of both arrays have no gaps.
    plan(int64_t items, int64_t voxels, int64_t channels, int64_t groups, bool flat, int64_t values)
    {
        const int64_t common = divisor(channels, CHUNK), rows = CHUNK / common, all = items * voxels * channels;
        flat = flat && voxels >= 8 * rows;
        const int64_t slots = flat ? channels * rows : (channels + CHUNK - 1) / CHUNK * CHUNK, room = all / 8 > (int64_t)1 << 20 ? all / 8 : (int64_t)1 << 20;
        const auto at_most = [](int64_t a, int64_t b) { return a < b ? a : b; };
        at_once = at_most(values / (voxels * channels > 0 ? voxels * channels : 1), room / slots);
        at_once = at_most(at_most(at_once < 1 ? 1 : at_once, (int64_t)1 << 20), items);
        const int64_t times = at_once ? room / 2 / (at_once * channels) : 1;
        held = at_most(at_once * (times < 1 ? 1 : times), items);
        deal = dealing_of(at_once, voxels, channels, groups, flat);
    }
    int64_t parts() const { return at_once * deal.strips * deal.positions * CHUNK; }
};

int64_t sixteens(int64_t bytes) { return (bytes + 15) / 16 * 16; }

// Bytes of the parts, of `each` a slot, and of the channels' sums, for the dealing that has more of them.
struct room {
    int64_t parts = 0, coefficients = 0, sums = 0;
    room(int64_t items, int64_t voxels, int64_t channels, int64_t groups, int64_t values, int64_t each)
    {
        for (const bool flat : {false, true}) {
            const plan L(items, voxels, channels, groups, flat, values);
            const auto at_least = [](int64_t &a, int64_t b) { a = a > b ? a : b; };
            at_least(parts, sixteens(L.parts() * each));
            at_least(coefficients, sixteens(L.at_once * groups * 8));
            at_least(sums, L.held * channels * 16);
        }
    }
};

// Where item `item` of an array begins.
const void *item_of(const void *p, int32_t type, int64_t item, int64_t distance) { return (const char *)p + item * distance * (type == LEAP_F32 ? 4 : 2); }

bool is_small(int64_t items, int64_t voxels, int64_t channels, int64_t groups)
{
    const int64_t size = channels / groups;
    return size % CHUNK == 0 && voxels <= SMALL_GROUP / size && items <= SMALL / channels / voxels;
}

// Outputs of more values than this go past the caches, which x is to stay in.
constexpr int64_t PAST_VALUES = (int64_t)1 << 25;

// f(whether all threads have eight values but at an item's end)
template <class F> int by_full(const dealing &D, F &&f)
{
    return D.rows > 1 || D.channels % CHUNK == 0 ? f(std::true_type{}) : f(std::false_type{});
}

template <class F> int by_activation(int32_t activation, F &&f)
{
    if (activation == LEAP_SILU) return f(std::integral_constant<int, LEAP_SILU>{});
    if (activation == LEAP_RELU) return f(std::integral_constant<int, LEAP_RELU>{});
    return f(std::integral_constant<int, LEAP_LINEAR>{});
}

const char *bad_kinds(int32_t type, int32_t weight_type, int32_t activation)
{
    if (!known_type(type) || !known_type(weight_type)) return "unknown element type";
    if (weight_type != type && weight_type != LEAP_F32) return "the weight must be float32 or of x's type";
    return activation == LEAP_LINEAR || activation == LEAP_RELU || activation == LEAP_SILU ? nullptr : "unknown activation";
}

}  // namespace

extern "C" int64_t leap_group_norm_work(int64_t items, int64_t voxels, int64_t channels, int64_t groups)
{
    if (bad_group(items, voxels, channels, groups) || !items || !voxels || is_small(items, voxels, channels, groups)) return 0;
    const room R(items, voxels, channels, groups, AT_ONCE_FORWARD, sizeof(moments));
    return R.parts + R.coefficients;
}

extern "C" int leap_group_norm(const void *d_x, int32_t type, int64_t x_item, int64_t x_row, const void *d_weight, const void *d_bias, int32_t weight_type, int64_t items,
                               int64_t voxels, int64_t channels, int64_t groups, float eps, int32_t activation, void *d_y, float *d_stats, void *d_work,
                               void *hip_stream)
{
    if (const char *why = bad_group(items, voxels, channels, groups)) return refuse(why);
    if (const char *why = bad_kinds(type, weight_type, activation)) return refuse(why);
    if (const char *why = bad_distances(x_item, x_row, items, voxels, channels)) return refuse(why);
    if (!(eps >= 0.0f)) return refuse("eps must not be negative");
    if (!items || !voxels) return LEAP_OK;
    if (!d_x || !d_y) return refuse("null data pointer");
    const hipStream_t st = stream_of(hip_stream);
    if (is_small(items, voxels, channels, groups)) {
        group_args A{};
        A.deal = dealing_of(items, voxels, channels, groups, false);
        A.x = {d_x, x_item, x_row};
        A.weight = d_weight, A.bias = d_bias, A.weight_type = weight_type, A.eps = eps, A.out = d_y, A.stats = d_stats;
        return by_type(type, [&](auto t) {
            return by_activation(activation, [&](auto a) {
                return over_blocks(items * groups, [&](int64_t first, unsigned n) {
                    A.first = first;
                    hipLaunchKernelGGL((k_group_small<decltype(t)::value, decltype(a)::value>), dim3(n), dim3(BLOCK), 0, st, A);
                });
            });
        });
    }
    if (unaligned(d_work)) return refuse(NO_WORK);
    const plan L(items, voxels, channels, groups, x_row == channels, AT_ONCE_FORWARD);
    const room R(items, voxels, channels, groups, AT_ONCE_FORWARD, sizeof(moments));
    group_args A{};
    A.deal = L.deal;
    A.x = {d_x, x_item, x_row};
    A.weight = d_weight, A.bias = d_bias, A.weight_type = weight_type, A.eps = eps;
    A.parts = (float *)d_work, A.past = voxels * channels * items > PAST_VALUES;
    const int64_t each = (int64_t)A.deal.strips * A.deal.segments;
    if (L.at_once * each >= (int64_t)1 << 24) return refuse("more than 2^24 blocks of items");
    return by_type(type, [&](auto t) {
        return by_activation(activation, [&](auto a) {
            return by_full(A.deal, [&](auto full) -> int {
                constexpr int T = decltype(t)::value;
                for (int64_t item = 0; item < items; item += L.at_once) {
                    const int64_t now = items - item < L.at_once ? items - item : L.at_once;
                    A.x.data = item_of(d_x, type, item, x_item), A.out = (void *)item_of(d_y, type, item, voxels * channels);
                    A.stats = d_stats ? d_stats + item * groups * 2 : (float *)((char *)d_work + R.parts);
                    hipLaunchKernelGGL((k_group_moments<T, decltype(full)::value>), dim3((unsigned)(now * each)), dim3(BLOCK), 0, st, A);
                    int rc = launched();
                    if (rc == LEAP_OK)
                        rc = over_blocks(now * groups, [&](int64_t first, unsigned n) {
                            A.first = first;
                            hipLaunchKernelGGL(k_group_stats, dim3(n), dim3(WIDE), 0, st, A);
                        });
                    if (rc != LEAP_OK) return rc;
                    hipLaunchKernelGGL((k_group_apply<T, decltype(full)::value, decltype(a)::value>), dim3((unsigned)(now * each)), dim3(BLOCK), 0, st, A);
                    if ((rc = launched()) != LEAP_OK) return rc;
                }
                return LEAP_OK;
            });
        });
    });
}

extern "C" int64_t leap_group_norm_backward_work(int64_t items, int64_t voxels, int64_t channels, int64_t groups)
{
    if (bad_group(items, voxels, channels, groups)) return 0;
    if (!items || !voxels) return 16;
    const room R(items, voxels, channels, groups, AT_ONCE_BACKWARD, 8);
    return R.parts + R.sums + channels * 16 + R.coefficients;
}

extern "C" int leap_group_norm_backward(const void *d_grad, int64_t grad_item, int64_t grad_row, const void *d_x, int32_t type, int64_t x_item, int64_t x_row,
                                        const void *d_weight, const void *d_bias, int32_t weight_type, const float *d_stats, int64_t items, int64_t voxels,
                                        int64_t channels, int64_t groups, int32_t activation, void *d_grad_x, void *d_grad_weight, void *d_grad_bias, void *d_work,
                                        void *hip_stream)
{
    if (const char *why = bad_group(items, voxels, channels, groups)) return refuse(why);
    if (const char *why = bad_kinds(type, weight_type, activation)) return refuse(why);
    if (const char *why = bad_distances(x_item, x_row, items, voxels, channels)) return refuse(why);
    if (const char *why = bad_distances(grad_item, grad_row, items, voxels, channels)) return refuse(why);
    const bool some = items && voxels;
    if (some && (!d_grad || !d_x || !d_stats)) return refuse("null data pointer");
    if (unaligned(d_work)) return refuse(NO_WORK);
    const hipStream_t st = stream_of(hip_stream);
    const plan L(items, voxels, channels, groups, x_row == channels && grad_row == channels, AT_ONCE_BACKWARD);
    const room R(items, voxels, channels, groups, AT_ONCE_BACKWARD, 8);
    group_args A{};
    A.deal = L.deal;
    A.x = {d_x, x_item, x_row}, A.grad = {d_grad, grad_item, grad_row};
    A.weight = d_weight, A.bias = d_bias, A.weight_type = weight_type;
    A.parts = (float *)d_work, A.past = voxels * channels * items > PAST_VALUES;
    double *const channel_sums = (double *)((char *)d_work + R.parts), *const running = channel_sums + R.sums / 8;
    float *const coefficients = (float *)(running + channels * 2);
    A.coefficients = coefficients;
    const int64_t each = (int64_t)A.deal.strips * A.deal.segments;
    if (L.at_once * each >= (int64_t)1 << 24) return refuse("more than 2^24 blocks of items");
    // The sums of the items from `from` to `to`, which channel_sums holds, on the weight's gradient and the bias'.
    const auto weights = [&](int64_t from, int64_t to) {
        if (!d_grad_weight && !d_grad_bias) return (int)LEAP_OK;
        return by_type(weight_type, [&](auto w) {
            hipLaunchKernelGGL((k_group_weights<decltype(w)::value>), dim3((unsigned)((channels + BLOCK - 1) / BLOCK)), dim3(BLOCK), 0, st, channel_sums, to - from, (int)channels,
                               from ? running : nullptr, some && to < items ? running : nullptr, d_grad_weight, d_grad_bias);
            return launched();
        });
    };
    if (!some) return weights(0, 0);
    return by_type(type, [&](auto t) {
        return by_activation(activation, [&](auto a) {
            return by_full(A.deal, [&](auto full) -> int {
                constexpr int T = decltype(t)::value, ACT = decltype(a)::value;
                constexpr bool FULL = decltype(full)::value;
                int64_t held = 0;                          // the first item that channel_sums holds
                for (int64_t item = 0; item < items; item += L.at_once) {
                    const int64_t now = items - item < L.at_once ? items - item : L.at_once;
                    A.x.data = item_of(d_x, type, item, x_item), A.grad.data = item_of(d_grad, type, item, grad_item);
                    A.stats = (float *)d_stats + item * groups * 2;
                    hipLaunchKernelGGL((k_group_sums<T, FULL, ACT>), dim3((unsigned)(now * each)), dim3(BLOCK), 0, st, A);
                    int status = launched();
                    if (status == LEAP_OK)
                        status = over_blocks(now * groups, [&](int64_t first, unsigned n) {
                            A.first = first;
                            hipLaunchKernelGGL(k_group_coefficients, dim3(n), dim3(WIDE), 0, st, A, channel_sums + (item - held) * channels * 2, coefficients);
                        });
                    if (status == LEAP_OK && (item + now - held >= L.held || item + now == items)) {
                        status = weights(held, item + now);
                        held = item + now;
                    }
                    if (status != LEAP_OK) return status;
                    if (!d_grad_x) continue;
                    A.out = (void *)item_of(d_grad_x, type, item, voxels * channels);
                    hipLaunchKernelGGL((k_group_grad<T, FULL, ACT>), dim3((unsigned)(now * each)), dim3(BLOCK), 0, st, A);
                    if ((status = launched()) != LEAP_OK) return status;
                }
                return LEAP_OK;
            });
        });
    });
}
