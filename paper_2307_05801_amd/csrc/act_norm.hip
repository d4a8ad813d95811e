// Root-mean-square norm with the residual's addition, its output and what its backward pass reads packed in 8 bits.
//
// Forward, a row: s = x + r (rounded to the type), rstd = (sum s^2 / cols + eps)^-1/2, normed = packed s rstd w, kept =
// packed s.  Backward, with h = kept rstd and d = grad w: grad_x = grad_sum + rstd (d - h sum(d h) / cols), grad_weight =
// sum over rows of grad h.  Both read and write each array once: a row stays in the registers of LANES lanes, eight values a
// chunk and up to MOST_CHUNKS chunks a lane.  Memory bounds them: 262144 x 512 bfloat16 forward in 185 us (5.9 TB/s), backward in 168 (5.7).
// Rows of more than 2048 columns are read twice forward and three times backward, a block to a row, which needs no registers for them: 65536 x 4096
// forward in 473 us, backward in 907 (4.6 and 2.1 TB/s of what one pass would move), 584 without the weight's gradient.
#include "act_common.h"

namespace {

using namespace act;

constexpr int BLOCK = 256;
constexpr int WAVE = 64;

// Sum over the LANES neighbouring lanes of a row, LANES a power of two up to a wave, in every one of them.
template <int LANES> __device__ inline float row_sum(float v)
{
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) v += __shfl_xor(v, d);
    return v;
}

// The same over a block, for rows that take one; every thread calls it.
__device__ inline float block_sum(float v, float *room)
{
    v = row_sum<WAVE>(v);
    __syncthreads();
    if (threadIdx.x % WAVE == 0) room[threadIdx.x / WAVE] = v;
    __syncthreads();
    float sum = 0.0f;
    for (int i = 0; i < BLOCK / WAVE; ++i) sum += room[i];
    return sum;
}

struct norm_args {
    const void *x, *residual, *weight;
    int64_t x_stride, residual_stride, rows, cols, groups;
    float eps, inverse_cols;
    void *sum;
    uint8_t *normed_codes, *normed_scales, *kept_codes, *kept_scales;
    float *rstd;
    bool past;                   // outputs past the caches
    int64_t first;               // block of this launch
};

// s of one chunk: x + residual, as the type holds it
template <int TYPE, bool ADD> __device__ inline void sum_chunk(const norm_args &A, int64_t row, int64_t col, int n, float (&s)[CHUNK])
{
    load8<TYPE>(A.x, row * A.x_stride + col, n, s);
    if constexpr (ADD) {
        float r[CHUNK];
        load8<TYPE>(A.residual, row * A.residual_stride + col, n, r);
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) s[i] = element<TYPE>::to_float(element<TYPE>::from_float(s[i] + r[i]));
    }
}

template <int TYPE, int WTYPE>
__device__ inline void norm_chunk(const norm_args &A, int64_t row, int64_t col, int n, const float (&s)[CHUNK], float rstd)
{
    if (A.sum && n > 0) store8<TYPE>(A.sum, row * A.cols + col, n, s, A.past);
    if (A.kept_codes) pack_chunk(s, n, A.kept_codes, A.kept_scales, row, A.cols, A.groups, col, A.past);
    float w[CHUNK], v[CHUNK];
    load8<WTYPE>(A.weight, col, n, w);
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) v[i] = s[i] * rstd * w[i];
    pack_chunk(v, n, A.normed_codes, A.normed_scales, row, A.cols, A.groups, col, A.past);
}

// Rows of up to LANES * CHUNKS chunks, BLOCK / LANES of them in a block.
template <int TYPE, int WTYPE, bool ADD, int LANES, int CHUNKS>
__global__ __launch_bounds__(BLOCK) void k_norm(norm_args A)
{
    const int lane = threadIdx.x % LANES;
    const int64_t row = (A.first + blockIdx.x) * (BLOCK / LANES) + threadIdx.x / LANES;
    const bool there = row < A.rows;
    float s[CHUNKS][CHUNK], square = 0.0f;
    int n[CHUNKS];
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        const int64_t left = A.cols - (int64_t)(k * LANES + lane) * CHUNK;
        n[k] = !there || left <= 0 ? 0 : left < CHUNK ? (int)left : CHUNK;
        sum_chunk<TYPE, ADD>(A, row, (int64_t)(k * LANES + lane) * CHUNK, n[k], s[k]);
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) square += s[k][i] * s[k][i];
    }
    const float rstd = rsqrtf(row_sum<LANES>(square) * A.inverse_cols + A.eps);
    if (A.rstd && lane == 0 && there) A.rstd[row] = rstd;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) norm_chunk<TYPE, WTYPE>(A, row, (int64_t)(k * LANES + lane) * CHUNK, n[k], s[k], rstd);
}

// Rows of any length, a block each; x and the residual are read twice.
template <int TYPE, int WTYPE, bool ADD> __global__ __launch_bounds__(BLOCK) void k_norm_long(norm_args A)
{
    __shared__ float room[BLOCK / WAVE];
    const int64_t row = A.first + blockIdx.x, most = A.groups * GROUP;
    float square = 0.0f, s[CHUNK];
    for (int64_t col = threadIdx.x * CHUNK; col < A.cols; col += BLOCK * CHUNK) {
        sum_chunk<TYPE, ADD>(A, row, col, (int)(A.cols - col < CHUNK ? A.cols - col : CHUNK), s);
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) square += s[i] * s[i];
    }
    const float rstd = rsqrtf(block_sum(square, room) * A.inverse_cols + A.eps);
    if (A.rstd && threadIdx.x == 0) A.rstd[row] = rstd;
    for (int64_t col = threadIdx.x * CHUNK; col < most; col += BLOCK * CHUNK) {          // whole groups: whole quads of lanes
        const int64_t left = A.cols - col;
        const int n = left <= 0 ? 0 : left < CHUNK ? (int)left : CHUNK;
        sum_chunk<TYPE, ADD>(A, row, col, n, s);
        norm_chunk<TYPE, WTYPE>(A, row, col, n, s, rstd);
    }
}

struct grad_args {
    const void *grad, *grad_sum, *weight;
    int64_t grad_stride, grad_sum_stride, rows, cols, groups;
    float inverse_cols;
    const uint8_t *kept_codes, *kept_scales;
    const float *rstd;
    void *grad_x;
    float *part;                 // [blocks][cols]: each block's sum of grad h, or null
    bool past;
    int64_t first;               // block of this launch, of those that take a row each
};

// How many of a chunk's values a row has, from what is left of it.
__device__ inline int there(int64_t left) { return left <= 0 ? 0 : left < CHUNK ? (int)left : CHUNK; }

// What is kept of one chunk; h is rstd times that
__device__ inline void unit_chunk(const grad_args &A, int64_t row, int64_t col, int n, float (&h)[CHUNK])
{
    const uint2 c = load_codes(A.kept_codes + row * A.cols + col, n);
    decode8(c, scale_value(n > 0 ? A.kept_scales[row * A.groups + col / GROUP] : 0u), h);
}

template <int TYPE>
__device__ inline void grad_chunk(const grad_args &A, int64_t row, int64_t col, int n, const float (&d)[CHUNK], const float (&h)[CHUNK],
                                  const float (&gs)[CHUNK], float rstd, float mean)
{
    if (n <= 0) return;
    float o[CHUNK];
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) o[i] = gs[i] + rstd * (d[i] - h[i] * mean);
    store8<TYPE>(A.grad_x, row * A.cols + col, n, o, A.past);
}

// Blocks walk over the rows, AHEAD of them at a time so that loads of a few rows are under way at once; a lane sums grad h of
// its own columns in registers, the block's rows of lanes join in shared memory at the end.
template <int TYPE, int GTYPE, int WTYPE, int LANES, int CHUNKS>
__global__ __launch_bounds__(BLOCK) void k_norm_grad(grad_args A)
{
    constexpr int ROWS = BLOCK / LANES, AHEAD = CHUNKS == 1 ? 2 : 1;
    __shared__ float room[ROWS > 1 ? BLOCK * CHUNK : 1];
    const int lane = threadIdx.x % LANES;
    float w[CHUNKS][CHUNK], dw[CHUNKS][CHUNK] = {};
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        const int64_t left = A.cols - (int64_t)(k * LANES + lane) * CHUNK;
        load8<WTYPE>(A.weight, (int64_t)(k * LANES + lane) * CHUNK, left <= 0 ? 0 : left < CHUNK ? (int)left : CHUNK, w[k]);
    }
    for (int64_t row0 = (int64_t)blockIdx.x * (ROWS * AHEAD); row0 < A.rows; row0 += (int64_t)gridDim.x * (ROWS * AHEAD)) {
        float d[AHEAD][CHUNKS][CHUNK], h[AHEAD][CHUNKS][CHUNK], gs[AHEAD][CHUNKS][CHUNK], rstd[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int64_t row = row0 + a * ROWS + threadIdx.x / LANES;
            rstd[a] = row < A.rows ? A.rstd[row] : 0.0f;
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                const int64_t col = (int64_t)(k * LANES + lane) * CHUNK;
                const int n = row < A.rows ? there(A.cols - col) : 0;
                load8<GTYPE>(A.grad, row * A.grad_stride + col, n, d[a][k]);
                unit_chunk(A, row, col, n, h[a][k]);
                load8<TYPE>(A.grad_sum, row * A.grad_sum_stride + col, A.grad_sum ? n : 0, gs[a][k]);
            }
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int64_t row = row0 + a * ROWS + threadIdx.x / LANES;
            float dot = 0.0f;
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                const bool here = row < A.rows && there(A.cols - (int64_t)(k * LANES + lane) * CHUNK) > 0;
#pragma unroll
                for (int i = 0; i < CHUNK; ++i) {
                    h[a][k][i] *= rstd[a];
                    if (here) dw[k][i] += d[a][k][i] * h[a][k][i];
                    d[a][k][i] *= w[k][i];
                    dot += d[a][k][i] * h[a][k][i];
                }
            }
            const float mean = row_sum<LANES>(dot) * A.inverse_cols;
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                const int64_t col = (int64_t)(k * LANES + lane) * CHUNK;
                grad_chunk<TYPE>(A, row, col, row < A.rows ? there(A.cols - col) : 0, d[a][k], h[a][k], gs[a][k], rstd[a], mean);
            }
        }
    }
    if (!A.part) return;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        const int64_t col = (int64_t)(k * LANES + lane) * CHUNK, left = A.cols - col;
        if constexpr (ROWS > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < CHUNK; ++i) room[i * BLOCK + threadIdx.x] = dw[k][i];
            __syncthreads();
            if (threadIdx.x < LANES) {
#pragma unroll
                for (int i = 0; i < CHUNK; ++i) {
                    float sum = 0.0f;
                    for (int r = 0; r < ROWS; ++r) sum += room[i * BLOCK + r * LANES + lane];
                    dw[k][i] = sum;
                }
            }
        }
        if (threadIdx.x < LANES && left > 0) store8<LEAP_F32>(A.part, blockIdx.x * A.cols + col, left < CHUNK ? (int)left : CHUNK, dw[k]);
    }
}

// Rows of any length, a block each.
template <int TYPE, int GTYPE, int WTYPE> __global__ __launch_bounds__(BLOCK) void k_norm_grad_long(grad_args A)
{
    __shared__ float room[BLOCK / WAVE];
    const int64_t row = A.first + blockIdx.x;
    const float rstd = A.rstd[row];
    float d[CHUNK], h[CHUNK], w[CHUNK], dot = 0.0f;
    for (int64_t col = threadIdx.x * CHUNK; col < A.cols; col += BLOCK * CHUNK) {
        const int n = (int)(A.cols - col < CHUNK ? A.cols - col : CHUNK);
        load8<GTYPE>(A.grad, row * A.grad_stride + col, n, d);
        load8<WTYPE>(A.weight, col, n, w);
        unit_chunk(A, row, col, n, h);
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) dot += d[i] * w[i] * (h[i] * rstd);
    }
    const float mean = block_sum(dot, room) * A.inverse_cols;
    for (int64_t col = threadIdx.x * CHUNK; col < A.cols; col += BLOCK * CHUNK) {
        const int n = (int)(A.cols - col < CHUNK ? A.cols - col : CHUNK);
        load8<GTYPE>(A.grad, row * A.grad_stride + col, n, d);
        load8<WTYPE>(A.weight, col, n, w);
        unit_chunk(A, row, col, n, h);
        float gs[CHUNK];
        load8<TYPE>(A.grad_sum, row * A.grad_sum_stride + col, A.grad_sum ? n : 0, gs);
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) d[i] *= w[i], h[i] *= rstd;
        grad_chunk<TYPE>(A, row, col, n, d, h, gs, rstd, mean);
    }
}

// Its grad h sums: a thread's eight columns over the rows of its part.
template <int GTYPE> __global__ __launch_bounds__(BLOCK) void k_norm_grad_weight_long(grad_args A)
{
    const int64_t col = ((int64_t)blockIdx.x * BLOCK + threadIdx.x) * CHUNK, left = A.cols - col;
    if (left <= 0) return;
    const int n = left < CHUNK ? (int)left : CHUNK;
    float dw[CHUNK] = {};
    for (int64_t row = blockIdx.y; row < A.rows; row += gridDim.y) {
        float g[CHUNK], h[CHUNK];
        load8<GTYPE>(A.grad, row * A.grad_stride + col, n, g);
        unit_chunk(A, row, col, n, h);
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) dw[i] += g[i] * (h[i] * A.rstd[row]);
    }
    store8<LEAP_F32>(A.part, blockIdx.y * A.cols + col, n, dw);
}

// grad_weight <- the sum of the parts: 16 columns a block, 64 threads to a column, each of which adds every 64th part.
template <int WTYPE> __global__ __launch_bounds__(1024) void k_join(const float *__restrict__ part, int64_t parts, int64_t cols, void *__restrict__ out)
{
    constexpr int COLS = 16, AT_ONCE = 64;
    __shared__ float room[AT_ONCE][COLS];
    const int c = threadIdx.x % COLS, r = threadIdx.x / COLS;
    const int64_t col = (int64_t)blockIdx.x * COLS + c;
    float sum = 0.0f;
    if (col < cols) {
#pragma unroll 8
        for (int64_t p = r; p < parts; p += AT_ONCE) sum += part[p * cols + col];
    }
    room[r][c] = sum;
    __syncthreads();
    for (int half = AT_ONCE / 2; half > 0; half /= 2) {
        if (r < half) room[r][c] += room[r + half][c];
        __syncthreads();
    }
    if (r == 0 && col < cols) ((typename element<WTYPE>::raw *)out)[col] = element<WTYPE>::from_float(room[0][c]);
}

constexpr int MOST_CHUNKS = 4;                                       // chunks a lane holds
constexpr int64_t LONG = (int64_t)WAVE * MOST_CHUNKS * CHUNK;        // columns from which a row takes a block

// f(lanes, chunks a lane) as constants: the fewest lanes (8 and up) that hold the row in one chunk each, then more chunks.
template <class F> int by_length(int64_t cols, F &&f)
{
    using std::integral_constant;
    const int64_t chunks = (cols + CHUNK - 1) / CHUNK;
    if (chunks <= 8) return f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    if (chunks <= 16) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    if (chunks <= 32) return f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    if (chunks <= 64) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    if (chunks <= 128) return f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    return f(integral_constant<int, 64>{}, integral_constant<int, MOST_CHUNKS>{});
}

// Blocks that walk over the rows in the backward pass: a few for each of the 256 compute units.
int64_t grad_blocks(int64_t rows, int64_t cols)
{
    if (cols > LONG) return rows < 256 ? (rows > 0 ? rows : 1) : 256;
    const int64_t lanes = cols <= 64 ? 8 : cols <= 128 ? 16 : cols <= 256 ? 32 : 64, at_once = BLOCK / lanes * (cols <= 512 ? 2 : 1), all = (rows + at_once - 1) / at_once;
    const int64_t most = cols <= 512 ? 1024 : 2048;                   // (262144 x 512: 180 us, 185 with 2048; 131072 x 1024: 217, 257 with 1024)
    return all < 1 ? 1 : all < most ? all : most;
}

template <class F> int by_weight(int32_t type, int32_t weight_type, F &&f)
{
    return by_type(type, [&](auto t) {
        if (weight_type == LEAP_F32) return f(t, std::integral_constant<int, LEAP_F32>{});
        return f(t, t);
    });
}

const char *bad_weight(int32_t type, int32_t weight_type)
{
    if (!known_type(type) || !known_type(weight_type)) return "unknown element type";
    return weight_type == LEAP_F32 || weight_type == type ? nullptr : "the weight must be float32 or of the rows' type";
}

}  // namespace

extern "C" int leap_rms_norm8(const void *d_x, int64_t x_stride, const void *d_residual, int64_t residual_stride, int32_t type, const void *d_weight,
                              int32_t weight_type, int64_t rows, int64_t cols, float eps, void *d_sum, uint8_t *d_normed_codes,
                              uint8_t *d_normed_scales, uint8_t *d_kept_codes, uint8_t *d_kept_scales, float *d_rstd, void *hip_stream)
{
    if (const char *why = bad_weight(type, weight_type)) return refuse(why);
    if (const char *why = bad_sizes(rows, cols)) return refuse(why);
    if (const char *why = bad_stride(x_stride, rows, cols)) return refuse(why);
    if (const char *why = d_residual ? bad_stride(residual_stride, rows, cols) : nullptr) return refuse(why);
    if (!(eps >= 0.0f)) return refuse("eps must not be negative");
    if (!rows) return LEAP_OK;
    if (!d_x || !d_weight || !d_normed_codes || !d_normed_scales) return refuse("null data pointer");
    if (!d_kept_codes != !d_kept_scales) return refuse("kept codes and scales: both or neither");
    if (rows > 0x7fffffff) return refuse("more than 2^31 rows");
    norm_args A{d_x, d_residual, d_weight, x_stride, residual_stride, rows, cols, groups_of(cols), eps, 1.0f / (float)cols,
                      d_sum, d_normed_codes, d_normed_scales, d_kept_codes, d_kept_scales, d_rstd, rows * cols * 2 > PAST_CACHES, 0};
    return by_weight(type, weight_type, [&](auto t, auto w) {
        constexpr int T = decltype(t)::value, W = decltype(w)::value;
        const hipStream_t st = stream_of(hip_stream);
        if (cols > LONG)
            return over_blocks(rows, [&](int64_t first, unsigned blocks) {
                A.first = first;
                if (d_residual) hipLaunchKernelGGL((k_norm_long<T, W, true>), dim3(blocks), dim3(BLOCK), 0, st, A);
                else hipLaunchKernelGGL((k_norm_long<T, W, false>), dim3(blocks), dim3(BLOCK), 0, st, A);
            });
        return by_length(cols, [&](auto l, auto c) {
            constexpr int L = decltype(l)::value, C = decltype(c)::value;
            return over_blocks((rows + BLOCK / L - 1) / (BLOCK / L), [&](int64_t first, unsigned blocks) {
                A.first = first;
                if (d_residual) hipLaunchKernelGGL((k_norm<T, W, true, L, C>), dim3(blocks), dim3(BLOCK), 0, st, A);
                else hipLaunchKernelGGL((k_norm<T, W, false, L, C>), dim3(blocks), dim3(BLOCK), 0, st, A);
            });
        });
    });
}

extern "C" int64_t leap_rms_norm8_work(int64_t rows, int64_t cols)
{
    return bad_sizes(rows, cols) ? 0 : grad_blocks(rows, cols) * cols;
}

extern "C" int leap_rms_norm8_backward(const void *d_grad, int32_t grad_type, int64_t grad_stride, const void *d_grad_sum, int64_t grad_sum_stride,
                                       int32_t type, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, const float *d_rstd,
                                       const void *d_weight, int32_t weight_type, int64_t rows, int64_t cols, void *d_grad_x,
                                       void *d_grad_weight, float *d_work, void *hip_stream)
{
    if (const char *why = bad_weight(type, weight_type)) return refuse(why);
    if (grad_type != type && grad_type != LEAP_F32) return refuse("the gradient must be float32 or of the rows' type");
    if (const char *why = bad_sizes(rows, cols)) return refuse(why);
    if (const char *why = bad_stride(grad_stride, rows, cols)) return refuse(why);
    if (const char *why = d_grad_sum ? bad_stride(grad_sum_stride, rows, cols) : nullptr) return refuse(why);
    if (rows > 0x7fffffff) return refuse("more than 2^31 rows");
    if (rows && (!d_grad || !d_kept_codes || !d_kept_scales || !d_rstd || !d_weight || !d_grad_x)) return refuse("null data pointer");
    if (d_grad_weight && !d_work) return refuse("the weight's gradient needs the workspace");
    grad_args A{d_grad, d_grad_sum, d_weight, grad_stride, grad_sum_stride, rows, cols, groups_of(cols), 1.0f / (float)cols,
                      d_kept_codes, d_kept_scales, d_rstd, d_grad_x, d_grad_weight ? d_work : nullptr, rows * cols * 2 > PAST_CACHES, 0};
    const hipStream_t st = stream_of(hip_stream);
    const int64_t parts = rows ? grad_blocks(rows, cols) : 0;
    int rc = LEAP_OK;
    if (rows)
        rc = by_weight(type, weight_type, [&](auto t, auto w) {
            constexpr int T = decltype(t)::value, W = decltype(w)::value;
            const auto run = [&](auto g) {
                constexpr int G = decltype(g)::value;
                if (cols > LONG) {
                    const int status = over_blocks(rows, [&](int64_t first, unsigned blocks) {
                        A.first = first;
                        hipLaunchKernelGGL((k_norm_grad_long<T, G, W>), dim3(blocks), dim3(BLOCK), 0, st, A);
                    });
                    if (status != LEAP_OK) return status;
                    if (A.part) {
                        const unsigned across = (unsigned)((cols + BLOCK * CHUNK - 1) / (BLOCK * CHUNK));
                        hipLaunchKernelGGL((k_norm_grad_weight_long<G>), dim3(across, (unsigned)parts), dim3(BLOCK), 0, st, A);
                    }
                    return launched();
                }
                return by_length(cols, [&](auto l, auto c) {
                    constexpr int L = decltype(l)::value, C = decltype(c)::value;
                    hipLaunchKernelGGL((k_norm_grad<T, G, W, L, C>), dim3((unsigned)parts), dim3(BLOCK), 0, st, A);
                    return launched();
                });
            };
            return grad_type == type ? run(t) : run(std::integral_constant<int, LEAP_F32>{});
        });
    if (rc != LEAP_OK || !d_grad_weight) return rc;
    return by_type(weight_type, [&](auto w) {
        hipLaunchKernelGGL((k_join<decltype(w)::value>), dim3((unsigned)((cols + 15) / 16)), dim3(1024), 0, st, d_work, parts, cols, d_grad_weight);
        return launched();
    });
}
