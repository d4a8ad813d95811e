// Products with rows held in 8 bits, and the gated product: leap_linear8 and its kin.
//
// All of them are D[j][i] = sum over k of P(i, k) Q(j, k) for two operands that are rows of bfloat16 or of packed values, read
// along k or across it.  A packed value is exact in bfloat16, so tiles of both go to shared memory as bfloat16 and through the
// matrix instructions, which sum in 32 bits.
#include "act_common.h"

namespace {

using namespace act;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int BLOCK = 256;
constexpr int TILE = 128, DEPTH = 32;      // a block's share of D is TILE x TILE, DEPTH values of k at a time
constexpr int PITCH = DEPTH + 8;           // of a tile's rows in shared memory: neighbouring rows in other banks

enum { ALONG, ACROSS };                    // an operand's values of one k-run are neighbours; or those of one k

// An operand: `rows` rows of `depth` values of k.  ALONG: memory rows are the operand's rows; ACROSS: they are k.
struct operand {
    const uint8_t *data;         // bfloat16 values, or codes
    const uint8_t *scales;       // null: bfloat16
    int64_t stride, groups;      // between memory rows: elements, scale bytes
    int64_t rows, depth;
};

// Eight values from (row, col) of the memory on, n of them there, as bfloat16.
template <bool PACKED> __device__ inline bf16x8 fetch8(const operand &O, int64_t row, int64_t col, int n)
{
    float v[CHUNK] = {};
    if (n > 0) {
        if constexpr (PACKED) decode8(load_codes(O.data + row * O.stride + col, n), scale_value(O.scales[row * O.groups + col / GROUP]), v);
        else load8<LEAP_BF16>(O.data, row * O.stride + col, n, v);
    }
    bf16x8 b;
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) b[i] = (__bf16)v[i];
    return b;
}

__device__ inline int clip8(int64_t left) { return left <= 0 ? 0 : left < CHUNK ? (int)left : CHUNK; }

// tile[r][k] <- O(row0 + r, k0 + k), zeros beyond its ends
template <int HOW, bool PACKED> __device__ inline void fill(const operand &O, int64_t row0, int64_t k0, __bf16 (*tile)[PITCH])
{
    for (int c = threadIdx.x; c < TILE * DEPTH / CHUNK; c += BLOCK) {
        if constexpr (HOW == ALONG) {
            const int r = c / (DEPTH / CHUNK), k = c % (DEPTH / CHUNK) * CHUNK;
            const bf16x8 b = fetch8<PACKED>(O, row0 + r, k0 + k, row0 + r < O.rows ? clip8(O.depth - k0 - k) : 0);
            *(bf16x8 *)&tile[r][k] = b;
        } else {
            const int k = c / (TILE / CHUNK), r = c % (TILE / CHUNK) * CHUNK;
            const bf16x8 b = fetch8<PACKED>(O, k0 + k, row0 + r, k0 + k < O.depth ? clip8(O.rows - row0 - r) : 0);
#pragma unroll
            for (int i = 0; i < CHUNK; ++i) tile[r + i][k] = b[i];
        }
    }
}

// out[j][i] of OTYPE, its rows `stride` apart
template <int PHOW, bool PPACKED, int QHOW, bool QPACKED, int OTYPE>
__global__ __launch_bounds__(BLOCK) void k_product(operand P, operand Q, void *__restrict__ out, int64_t stride)
{
    __shared__ __attribute__((aligned(16))) __bf16 p[TILE][PITCH], q[TILE][PITCH];
    const int64_t i0 = (int64_t)blockIdx.x * TILE, j0 = (int64_t)blockIdx.y * TILE;
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, wi = wave % 2 * 64, wj = wave / 2 * 64;
    f32x16 acc[2][2] = {};
    for (int64_t k0 = 0; k0 < P.depth; k0 += DEPTH) {
        __syncthreads();
        fill<PHOW, PPACKED>(P, i0, k0, p);
        fill<QHOW, QPACKED>(Q, j0, k0, q);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < DEPTH; k += 16) {
            bf16x8 a[2], b[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                a[t] = *(const bf16x8 *)&p[wi + t * 32 + lane % 32][k + lane / 32 * 8];
                b[t] = *(const bf16x8 *)&q[wj + t * 32 + lane % 32][k + lane / 32 * 8];
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int t = 0; t < 2; ++t) acc[s][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[s], b[t], acc[s][t], 0, 0, 0);
        }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int64_t i = i0 + wi + s * 32 + r / 4 * 8 + lane / 32 * 4 + r % 4, j = j0 + wj + t * 32 + lane % 32;
                if (i < P.rows && j < Q.rows) ((typename element<OTYPE>::raw *)out)[j * stride + i] = element<OTYPE>::from_float(acc[s][t][r]);
            }
}

operand plain(const void *p, int64_t stride, int64_t rows, int64_t depth) { return {(const uint8_t *)p, nullptr, stride, 0, rows, depth}; }
operand packed(const uint8_t *codes, const uint8_t *scales, int64_t cols, int64_t rows, int64_t depth)
{
    return {codes, scales, cols, groups_of(cols), rows, depth};
}

template <int PHOW, bool PPACKED, int QHOW, bool QPACKED, int OTYPE>
int product(const operand &P, const operand &Q, void *out, int64_t stride, hipStream_t st)
{
    const int64_t across = (P.rows + TILE - 1) / TILE;
    for (int64_t j0 = 0; j0 < Q.rows; j0 += (int64_t)65535 * TILE) {       // a launch's second dimension ends at 65535
        operand part = Q;
        part.rows = Q.rows - j0 < (int64_t)65535 * TILE ? Q.rows - j0 : (int64_t)65535 * TILE;
        part.data += QHOW == ALONG ? j0 * Q.stride * (QPACKED ? 1 : 2) : j0 * (QPACKED ? 1 : 2);
        if (QPACKED) part.scales += QHOW == ALONG ? j0 * Q.groups : j0 / GROUP;
        hipLaunchKernelGGL((k_product<PHOW, PPACKED, QHOW, QPACKED, OTYPE>), dim3((unsigned)across, (unsigned)((part.rows + TILE - 1) / TILE)),
                           dim3(BLOCK), 0, st, P, part, (char *)out + j0 * stride * (OTYPE == LEAP_F32 ? 4 : 2), stride);
        const int rc = launched();
        if (rc != LEAP_OK) return rc;
    }
    return LEAP_OK;
}

// ---- the gate ----

// gated, kept <- u = (g, p), [rows][2 * out] float; one chunk of `out` a lane
__global__ __launch_bounds__(BLOCK) void k_gate(const float *__restrict__ u, int64_t rows, int64_t out, uint8_t *__restrict__ gated_codes,
                                                uint8_t *__restrict__ gated_scales, uint8_t *__restrict__ kept_codes, uint8_t *__restrict__ kept_scales)
{
    const int64_t groups = groups_of(out), per_row = groups * (GROUP / CHUNK), c = (int64_t)blockIdx.x * BLOCK + threadIdx.x;
    const int64_t row = c / per_row, col = (c - row * per_row) * CHUNK;
    const int n = row < rows ? clip8(out - col) : 0;
    float g[CHUNK], p[CHUNK], a[CHUNK];
    load8<LEAP_F32>(u, row * 2 * out + col, n, g);
    load8<LEAP_F32>(u, row * 2 * out + out + col, n, p);
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) a[i] = g[i] * sigmoid(g[i]) * p[i];
    pack_chunk(a, n, gated_codes, gated_scales, row, out, groups, col);
    if (kept_codes) {
        pack_chunk(g, n, kept_codes, kept_scales, 2 * row, out, groups, col);
        pack_chunk(p, n, kept_codes, kept_scales, 2 * row + 1, out, groups, col);
    }
}

template <int TYPE>
__global__ __launch_bounds__(BLOCK) void k_gate_grad(const void *__restrict__ da, int64_t stride, const uint8_t *__restrict__ kept_codes,
                                                     const uint8_t *__restrict__ kept_scales, int64_t rows, int64_t out, void *__restrict__ du)
{
    const int64_t groups = groups_of(out), per_row = groups * (GROUP / CHUNK), c = (int64_t)blockIdx.x * BLOCK + threadIdx.x;
    const int64_t row = c / per_row, col = (c - row * per_row) * CHUNK;
    const int n = row < rows ? clip8(out - col) : 0;
    if (n <= 0) return;
    float d[CHUNK], g[CHUNK], p[CHUNK], dg[CHUNK], dp[CHUNK];
    load8<TYPE>(da, row * stride + col, n, d);
    decode8(load_codes(kept_codes + 2 * row * out + col, n), scale_value(kept_scales[2 * row * groups + col / GROUP]), g);
    decode8(load_codes(kept_codes + (2 * row + 1) * out + col, n), scale_value(kept_scales[(2 * row + 1) * groups + col / GROUP]), p);
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) {
        const float s = sigmoid(g[i]);
        dg[i] = d[i] * p[i] * s * (1.0f + g[i] * (1.0f - s));
        dp[i] = d[i] * g[i] * s;
    }
    store8<LEAP_BF16>(du, row * 2 * out + col, n, dg);
    store8<LEAP_BF16>(du, row * 2 * out + out + col, n, dp);
}

// Blocks of the gate's kernels; 0: more than a launch holds.
unsigned gate_blocks(int64_t rows, int64_t out)
{
    const int64_t blocks = (rows * groups_of(out) * (GROUP / CHUNK) + BLOCK - 1) / BLOCK;
    return blocks <= 0x7fffffff ? (unsigned)blocks : 0u;
}

const char *bad_product(int64_t rows, int64_t cols, int64_t w_stride, int64_t out)
{
    if (const char *why = bad_sizes(rows, cols)) return why;
    if (const char *why = bad_sizes(rows, out)) return why;
    return bad_stride(w_stride, out, cols);
}

}  // namespace

extern "C" int leap_linear8(const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride,
                            int64_t out, void *d_y, void *hip_stream)
{
    if (const char *why = bad_product(rows, cols, w_stride, out)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_codes || !d_scales || !d_weight || !d_y) return refuse("null data pointer");
    return product<ALONG, false, ALONG, true, LEAP_BF16>(plain(d_weight, w_stride, out, cols), packed(d_codes, d_scales, cols, rows, cols), d_y, out,
                                                         stream_of(hip_stream));
}

extern "C" int64_t leap_linear8_work(int64_t rows, int64_t cols, int64_t out)
{
    (void)rows, (void)cols, (void)out;
    return 0;
}

extern "C" int leap_linear8_backward(const void *d_dy, int64_t dy_stride, const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols,
                                     const void *d_weight, int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight,
                                     void *d_work, void *hip_stream)
{
    if (const char *why = bad_product(rows, cols, w_stride, out)) return refuse(why);
    if (const char *why = bad_stride(dy_stride, rows, out)) return refuse(why);
    if (grad_x_type != LEAP_BF16 && grad_x_type != LEAP_F32) return refuse("grad_x is bfloat16 or float32");
    if (rows && (!d_dy || !d_codes || !d_scales || !d_weight)) return refuse("null data pointer");
    if (!d_work && leap_linear8_work(rows, cols, out)) return refuse("null workspace");
    const hipStream_t st = stream_of(hip_stream);
    int rc = LEAP_OK;
    if (d_grad_x && rows) {
        const operand W = plain(d_weight, w_stride, cols, out), G = plain(d_dy, dy_stride, rows, out);
        rc = grad_x_type == LEAP_F32 ? product<ACROSS, false, ALONG, false, LEAP_F32>(W, G, d_grad_x, cols, st)
                                     : product<ACROSS, false, ALONG, false, LEAP_BF16>(W, G, d_grad_x, cols, st);
    }
    if (rc != LEAP_OK || !d_grad_weight) return rc;
    return product<ACROSS, true, ACROSS, false, LEAP_BF16>(packed(d_codes, d_scales, cols, cols, rows), plain(d_dy, dy_stride, out, rows), d_grad_weight,
                                                           cols, st);
}

extern "C" int64_t leap_gated_linear8_work(int64_t rows, int64_t cols, int64_t out)
{
    return bad_product(rows, cols, cols, out) ? 0 : rows * 2 * out * (int64_t)sizeof(float);
}

extern "C" int leap_gated_linear8(const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride,
                                  int64_t out, uint8_t *d_gated_codes, uint8_t *d_gated_scales, uint8_t *d_kept_codes, uint8_t *d_kept_scales,
                                  void *d_work, void *hip_stream)
{
    if (out > MOST_COLS / 2) return refuse("more than 2^19 gated columns");
    if (const char *why = bad_product(rows, cols, w_stride, 2 * out)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_codes || !d_scales || !d_weight || !d_gated_codes || !d_gated_scales || !d_work) return refuse("null data pointer");
    if (!d_kept_codes != !d_kept_scales) return refuse("kept codes and scales: both or neither");
    const unsigned blocks = gate_blocks(rows, out);
    if (!blocks) return refuse("more values than one launch covers");
    const hipStream_t st = stream_of(hip_stream);
    const int rc = product<ALONG, false, ALONG, true, LEAP_F32>(plain(d_weight, w_stride, 2 * out, cols), packed(d_codes, d_scales, cols, rows, cols),
                                                                d_work, 2 * out, st);
    if (rc != LEAP_OK) return rc;
    hipLaunchKernelGGL(k_gate, dim3(blocks), dim3(BLOCK), 0, st, (const float *)d_work, rows, out, d_gated_codes, d_gated_scales, d_kept_codes, d_kept_scales);
    return launched();
}

namespace {

template <int TYPE> int gate_backward(const void *da, int64_t stride, const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t out, void *du, hipStream_t st)
{
    const unsigned blocks = gate_blocks(rows, out);
    if (!blocks) return refuse("more values than one launch covers");
    hipLaunchKernelGGL((k_gate_grad<TYPE>), dim3(blocks), dim3(BLOCK), 0, st, da, stride, codes, scales, rows, out, du);
    return launched();
}

}  // namespace

extern "C" int leap_gate8_backward(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows,
                                   int64_t out, void *d_du, void *hip_stream)
{
    if (out > MOST_COLS / 2) return refuse("more than 2^19 gated columns");
    if (const char *why = bad_sizes(rows, out)) return refuse(why);
    if (const char *why = bad_stride(da_stride, rows, out)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_da || !d_kept_codes || !d_kept_scales || !d_du) return refuse("null data pointer");
    return gate_backward<LEAP_BF16>(d_da, da_stride, d_kept_codes, d_kept_scales, rows, out, d_du, stream_of(hip_stream));
}

extern "C" int64_t leap_linear_gate8_work(int64_t rows, int64_t out, int64_t next)
{
    return bad_product(rows, next, next, out) ? 0 : rows * out * (int64_t)sizeof(float);
}

extern "C" int leap_linear_gate8_backward(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next,
                                          const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows, int64_t out, void *d_du,
                                          void *d_work, void *hip_stream)
{
    if (out > MOST_COLS / 2) return refuse("more than 2^19 gated columns");
    if (const char *why = bad_product(rows, out, w_stride, next)) return refuse(why);
    if (const char *why = bad_stride(dy_stride, rows, next)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_dy || !d_weight || !d_kept_codes || !d_kept_scales || !d_du || !d_work) return refuse("null data pointer");
    const hipStream_t st = stream_of(hip_stream);
    const int rc = product<ACROSS, false, ALONG, false, LEAP_F32>(plain(d_weight, w_stride, out, next), plain(d_dy, dy_stride, rows, next), d_work, out, st);
    if (rc != LEAP_OK) return rc;
    return gate_backward<LEAP_F32>(d_work, out, d_kept_codes, d_kept_scales, rows, out, d_du, st);
}
