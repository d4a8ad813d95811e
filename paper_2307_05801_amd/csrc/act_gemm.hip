// Products with rows held in 8 bits, and the gated product: leap_linear8 and its kin (act_product.h has the kernel).
//
// Its fetches want memory rows that begin at multiples of 16 bytes.  Operands that do not (odd sizes, odd strides) are
// first laid out anew in the workspace, a pass over them that costs a few percent of the product.
#include "act_product.h"

namespace {

using namespace act;

constexpr int BLOCK = 256;

// ---- operands laid out for the product ----

// An array whose rows, `bytes` long, are copied to rows of `pitch` bytes (a multiple of 16) with zeros at their ends.
struct copied_rows {
    const uint8_t *from;
    uint8_t *to;
    int64_t stride, rows, bytes, pitch;
    divider pieces;              // of 16 bytes, of a row
    uint32_t blocks;             // that copy it
};

struct copies {
    copied_rows of[3];
};

__global__ __launch_bounds__(BLOCK) void k_lay_out(copies C)
{
    uint32_t block = blockIdx.x;
    int c = 0;
    while (c < 2 && block >= C.of[c].blocks) block -= C.of[c++].blocks;
    const copied_rows &A = C.of[c];
    // a block's first piece may lie beyond 32 bits, what it holds of rows may not
    const int64_t first = (int64_t)block * BLOCK, row0 = first / A.pieces.by;
    const uint32_t q = (uint32_t)(first - row0 * A.pieces.by) + threadIdx.x, in = A.pieces(q);
    const int64_t row = row0 + in, at = (int64_t)(q - in * A.pieces.by) * 16;
    if (row >= A.rows) return;
    uint8_t piece[16] = {};
    if (A.bytes - at >= 16) {
        __builtin_memcpy(piece, A.from + row * A.stride + at, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 15; ++i)
            if (at + i < A.bytes) piece[i] = A.from[row * A.stride + at + i];
    }
    __builtin_memcpy(A.to + row * A.pitch + at, piece, 16);
}

int64_t cut(int64_t n, int64_t by) { return (n + by - 1) / by; }
int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// Memory rows as the product takes them: as they are, or a copy of them in the workspace.  Rows further apart than this are copied too, so
// that a tile's rows lie within 31-bit offsets, and rows that overlap (one for all), so that what lies beyond the last reads as zeros.
constexpr int64_t FAR_APART = (int64_t)1 << 22;                          // bytes; 2^20 columns, the most, are half of it

struct laid {
    const uint8_t *data;
    int64_t stride, rows, bytes, pitch;              // in bytes
    bool copied;
    // padded: its rows are followed by zeros up to a multiple of 16 bytes
    laid(const void *p, int64_t stride_, int64_t rows_, int64_t cols, int size, bool padded = false)
        : data((const uint8_t *)p), stride(stride_ * size), rows(rows_), bytes(cols * size), pitch(up16(cols * size))
    {
        copied = rows > 0 && (stride % 16 != 0 || (bytes % 16 != 0 && !padded) || (uintptr_t)p % 16 != 0 || stride < bytes || stride > FAR_APART);
    }
    int64_t room() const { return copied ? rows * pitch : 0; }

    operand wide(int64_t i, int64_t k) const { return {data, nullptr, stride / 2, 0, i, k}; }
    operand codes(const uint8_t *scales, int64_t cols, int64_t i, int64_t k) const { return {data, scales, stride, groups_of(cols), i, k}; }
};

// The copies of up to three arrays, into `room` one after the other, which moves on.
int lay_out(uint8_t *&room, hipStream_t st, laid *a, laid *b = nullptr, laid *c = nullptr)
{
    copies C = {{{nullptr, nullptr, 0, 0, 0, 16, divider(1), 0}, {nullptr, nullptr, 0, 0, 0, 16, divider(1), 0}, {nullptr, nullptr, 0, 0, 0, 16, divider(1), 0}}};
    int64_t blocks = 0;
    int n = 0;
    for (laid *x : {a, b, c}) {
        if (!x || !x->copied) continue;
        const int64_t mine = cut(x->rows * (x->pitch / 16), BLOCK);
        blocks += mine;
        if (blocks > 0x7fffffff) return refuse("more values to lay out than one launch covers");
        C.of[n++] = {x->data, room, x->stride, x->rows, x->bytes, x->pitch, divider((uint32_t)(x->pitch / 16)), (uint32_t)mine};
        x->data = room, x->stride = x->pitch, x->copied = false;
        room += x->rows * x->pitch;
    }
    if (!n) return LEAP_OK;
    hipLaunchKernelGGL(k_lay_out, dim3((unsigned)blocks), dim3(BLOCK), 0, st, C);
    return launched();
}

// ---- launches ----

// Tiles of 256 x 256, eight waves and a block a compute unit; or of 128 x 128, four waves and two blocks, at 0.8 of the rate (262144 x
// 512 -> 2 * 1024, gated: 844 and 1056 us) but with less left over where tiles are few.  In units of the time of a large tile, 256 units
// taking tiles at once:
bool large_tiles(int64_t i, int64_t j)
{
    return (double)cut(cut(i, 256) * cut(j, 256), 256) <= 0.62 * (double)cut(cut(i, 128) * cut(j, 128), 512);
}

template <int PKIND, int QKIND, int TO, int TI, int TJ, int WI, int WJ, int GROUPS, int DEPTH>
int launch(const operand &P, const operand &Q, const result &R, int64_t depth_part, hipStream_t st)
{
    const int64_t across = TO == TO_GATED ? cut(R.columns, TI / 2) : cut(P.rows, TI), along = cut(Q.rows, TJ), parts = depth_part ? cut(P.depth, depth_part) : 1;
    if (across * along * parts > 0x7fffffff) return refuse("more rows and columns than one launch covers");
    // as many blocks as the 256 compute units hold at once, by shared memory and registers
    constexpr int RESIDENT = WI * WJ * GROUPS > 4 ? 1 : 2;
    const int64_t blocks = !stays<TO>() || GROUPS > 1 || across * along * parts < 256 * RESIDENT ? across * along * parts : 256 * RESIDENT;
    hipLaunchKernelGGL((k_product<PKIND, QKIND, TO, TI, TJ, WI, WJ, GROUPS, DEPTH>), dim3((unsigned)blocks), dim3(WI * WJ * GROUPS * 64), 0, st, P, Q, R, (uint32_t)across,
                       (uint32_t)along, (uint32_t)parts, depth_part ? depth_part : P.depth);
    return launched();
}

template <int PKIND, int QKIND, int TO> int product(const operand &P, const operand &Q, const result &R, int64_t depth_part, bool large, hipStream_t st)
{
    // the gate's gradient moves more than it multiplies: small tiles always (262144 x 512 -> 2 * 512: 300 us, large ones 369)
    if constexpr (TO != TO_GATE_GRAD)
        if (large) return launch<PKIND, QKIND, TO, 256, 256, 2, 4, 1, 2>(P, Q, R, depth_part, st);
    // At most as many tiles as units: two groups of waves share one, and half as many rows a tile while that makes no second round of
    // them (4096 x 2048 -> 512: 17 us in 256 tiles of 64 rows, 29 in 128 of 128 and two buffers).
    if constexpr (PKIND != CODES_ACROSS) {
        const int64_t across = cut(TO == TO_GATED ? 2 * R.columns : P.rows, 128);
        if (across * cut(Q.rows, 64) <= 256) return launch<PKIND, QKIND, TO, 128, 64, 2, 2, 2, 3>(P, Q, R, depth_part, st);
        if (across * cut(Q.rows, 128) <= 256) return launch<PKIND, QKIND, TO, 128, 128, 2, 2, 2, QKIND == CODES_ALONG ? 3 : 2>(P, Q, R, depth_part, st);
    }
    return launch<PKIND, QKIND, TO, 128, 128, 2, 2, 1, 2>(P, Q, R, depth_part, st);
}

template <int PKIND, int QKIND, int TO> int product(const operand &P, const operand &Q, const result &R, hipStream_t st)
{
    return product<PKIND, QKIND, TO>(P, Q, R, 0, large_tiles(P.rows, Q.rows), st);
}

// grad_weight: few tiles, many rows to sum over.  The rows are cut into parts, as many as give every compute unit a tile,
// of at least 512 rows; each part's sum goes to the workspace in 32 bits, and a kernel adds them in order.
struct weight_plan {
    bool large;
    int64_t parts, depth_part;
    weight_plan(int64_t rows, int64_t cols, int64_t out)
    {
        const int64_t tiles = cut(cols, 256) * cut(out, 256), small = cut(cols, 128) * cut(out, 128);
        // a small tile takes 0.31 of a large one's time; what of a tile lies beyond the edges is work for nothing
        large = tiles * cut(rows, 1024) >= 256 && (double)tiles <= 0.31 * (double)small;
        const int64_t t = large ? tiles : small, want = (large ? 256 : 512) / t;
        parts = want < 1 ? 1 : want;
        if (parts > cut(rows, 512)) parts = cut(rows, 512);
        if (parts < 1) parts = 1;
        depth_part = cut(cut(rows, parts), 64) * 64;
        if (depth_part < 64) depth_part = 64;
        parts = rows ? cut(rows, depth_part) : 1;
    }
    int64_t room(int64_t cols, int64_t out) const { return parts > 1 ? up16(parts * cols * out * (int64_t)sizeof(float)) : 0; }
};

// to <- the sum of the parts, in a fixed order: 16 threads to four values each, which add every 16th part, 64 values a block.
constexpr int ADDED = 64;

template <int TYPE> __global__ __launch_bounds__(BLOCK) void k_add_parts(const float *__restrict__ from, int64_t parts, int64_t n, void *__restrict__ to)
{
    constexpr int WAYS = BLOCK / (ADDED / 4);
    __shared__ float room[WAYS][ADDED];
    const int way = threadIdx.x / (ADDED / 4), in = threadIdx.x % (ADDED / 4) * 4;
    const int64_t at = (int64_t)blockIdx.x * ADDED + in;
    const int left = n - at < 4 ? (int)(n - at) : 4;
    float sum[4] = {};
    if (left == 4) {
#pragma unroll 4
        for (int64_t p = way; p < parts; p += WAYS) {
            float f[4];
            __builtin_memcpy(f, from + p * n + at, 16);
#pragma unroll
            for (int x = 0; x < 4; ++x) sum[x] += f[x];
        }
    } else {
        for (int64_t p = way; p < parts; p += WAYS)
            for (int x = 0; x < left; ++x) sum[x] += from[p * n + at + x];
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) room[way][in + x] = sum[x];
    __syncthreads();
    if (threadIdx.x < ADDED && (int64_t)blockIdx.x * ADDED + threadIdx.x < n) {
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < WAYS; ++w) total += room[w][threadIdx.x];
        ((typename element<TYPE>::raw *)to)[(int64_t)blockIdx.x * ADDED + threadIdx.x] = element<TYPE>::from_float(total);
    }
}

// y and grad_x of few rows and columns, with many values of k to sum over: the same, in parts of k, 256 at least.  128 values of k take a
// tile of 128 x 64 0.8 us, another launch 3 us, and the parts' sums the more the more tiles there are: from 1024 values on, and
// 64 for each tile (1 x 2048 -> 512: 7.0 us, 14.8 in one; 512 x 2048 -> 512, 32 tiles: 12.4 and 16.2; 1024 x 1024 -> 512, 64 tiles: 13.6 and 10.2).
struct depth_plan {
    int64_t parts, depth_part;
    depth_plan(int64_t i, int64_t j, int64_t depth)
    {
        const int64_t tiles = cut(i, 128) * cut(j, 64);
        parts = 1, depth_part = depth;
        if (tiles < 1 || tiles * 64 > depth || depth < 1024) return;
        parts = 256 / tiles < depth / 256 ? 256 / tiles : depth / 256;
        if (parts < 1) parts = 1;
        depth_part = cut(cut(depth, parts), 128) * 128;
        parts = cut(depth, depth_part);
    }
    int64_t room(int64_t i, int64_t j) const { return parts > 1 ? up16(parts * i * j * (int64_t)sizeof(float)) : 0; }
};

template <int PKIND, int QKIND> int product_in_parts(const operand &P, const operand &Q, void *out, int32_t type, const depth_plan &plan, uint8_t *room, hipStream_t st)
{
    result R{};
    R.out = room, R.stride = P.rows, R.part = P.rows * Q.rows;
    const int rc = launch<PKIND, QKIND, TO_FULL, 128, 64, 2, 2, 2, 3>(P, Q, R, plan.depth_part, st);
    if (rc != LEAP_OK) return rc;
    const dim3 adders((unsigned)cut(R.part, ADDED));
    if (type == LEAP_F32) hipLaunchKernelGGL((k_add_parts<LEAP_F32>), adders, dim3(BLOCK), 0, st, (const float *)room, plan.parts, R.part, out);
    else hipLaunchKernelGGL((k_add_parts<LEAP_BF16>), adders, dim3(BLOCK), 0, st, (const float *)room, plan.parts, R.part, out);
    return launched();
}

// ---- the gate by itself ----

// du, rows of du_stride, <- da and what is kept, and zeros between its rows; one chunk of `out` a lane
__global__ __launch_bounds__(BLOCK) void k_gate_grad(const void *__restrict__ da, int64_t stride, const uint8_t *__restrict__ kept_codes,
                                                     const uint8_t *__restrict__ kept_scales, int64_t rows, int64_t out, void *__restrict__ du,
                                                     int64_t du_stride)
{
    const int64_t groups = groups_of(out), per_row = groups * (GROUP / CHUNK), c = (int64_t)blockIdx.x * BLOCK + threadIdx.x;
    const int64_t row = c / per_row, col = (c - row * per_row) * CHUNK;
    const int n = row < rows ? (out - col < CHUNK ? (int)(out - col) : CHUNK) : 0;
    if (n <= 0) return;
    float d[CHUNK], g[CHUNK], p[CHUNK], dg[CHUNK], dp[CHUNK];
    load8<LEAP_BF16>(da, row * stride + col, n, d);
    decode8(load_codes(kept_codes + 2 * row * out + col, n), scale_value(kept_scales[2 * row * groups + col / GROUP]), g);
    decode8(load_codes(kept_codes + (2 * row + 1) * out + col, n), scale_value(kept_scales[(2 * row + 1) * groups + col / GROUP]), p);
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) {
        const float s = sigmoid(g[i]);
        dg[i] = d[i] * p[i] * s * (1.0f + g[i] * (1.0f - s));
        dp[i] = d[i] * g[i] * s;
    }
    store8<LEAP_BF16>(du, row * du_stride + col, n, dg, rows * out * 4 > READ_NEXT);
    store8<LEAP_BF16>(du, row * du_stride + out + col, n, dp, rows * out * 4 > READ_NEXT);
    if (col + n == out)
        for (int64_t i = 2 * out; i < du_stride; ++i) ((uint16_t *)du)[row * du_stride + i] = 0;
}

// Zeros between rows, behind the `cols` values of each.
__global__ __launch_bounds__(BLOCK) void k_pad_rows(uint16_t *__restrict__ to, int64_t stride, int64_t rows, int64_t cols)
{
    const int64_t row = (int64_t)blockIdx.x * BLOCK + threadIdx.x;
    if (row >= rows) return;
    for (int64_t i = cols; i < stride; ++i) to[row * stride + i] = 0;
}

const char *bad_product(int64_t rows, int64_t cols, int64_t w_stride, int64_t out)
{
    if (const char *why = bad_sizes(rows, cols)) return why;
    if (const char *why = bad_sizes(rows, out)) return why;
    return bad_stride(w_stride, out, cols);
}

constexpr const char *GATED_LIMIT = "more than 2^19 gated columns";

}  // namespace

extern "C" int64_t leap_linear8_work(const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out)
{
    if (bad_product(rows, cols, w_stride, out)) return 0;
    return depth_plan(out, rows, cols).room(out, rows) + laid(d_codes, cols, rows, cols, 1).room() + laid(d_weight, w_stride, out, cols, 2).room();
}

extern "C" int leap_linear8(const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride,
                            int64_t out, void *d_y, void *d_work, void *hip_stream)
{
    if (const char *why = bad_product(rows, cols, w_stride, out)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_codes || !d_scales || !d_weight || !d_y) return refuse("null data pointer");
    if (!d_work && leap_linear8_work(d_codes, rows, cols, d_weight, w_stride, out)) return refuse("null workspace");
    const hipStream_t st = stream_of(hip_stream);
    uint8_t *room = (uint8_t *)d_work;
    laid W(d_weight, w_stride, out, cols, 2), X(d_codes, cols, rows, cols, 1);
    const int rc = lay_out(room, st, &W, &X);
    if (rc != LEAP_OK) return rc;
    const depth_plan plan(out, rows, cols);
    if (plan.parts > 1)
        return product_in_parts<WIDE_ALONG, CODES_ALONG>(W.wide(out, cols), X.codes(d_scales, cols, rows, cols), d_y, LEAP_BF16, plan, room, st);
    result R{};
    R.out = d_y, R.stride = out;
    return product<WIDE_ALONG, CODES_ALONG, TO_WIDE>(W.wide(out, cols), X.codes(d_scales, cols, rows, cols), R, st);
}

int64_t act::linear8_backward_work(const void *d_dy, int64_t dy_stride, bool padded, const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight,
                                   int64_t w_stride, int64_t out)
{
    if (bad_product(rows, cols, w_stride, out) || bad_stride(dy_stride, rows, out)) return 0;
    return weight_plan(rows, cols, out).room(cols, out) + depth_plan(cols, rows, out).room(cols, rows) + laid(d_dy, dy_stride, rows, out, 2, padded).room() + laid(d_codes, cols, rows, cols, 1).room() +
           laid(d_weight, w_stride, out, cols, 2).room();
}

int act::linear8_backward(const void *d_dy, int64_t dy_stride, bool padded, const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols,
                          const void *d_weight, int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight, void *d_work,
                          void *hip_stream)
{
    if (const char *why = bad_product(rows, cols, w_stride, out)) return refuse(why);
    if (const char *why = bad_stride(dy_stride, rows, out)) return refuse(why);
    if (grad_x_type != LEAP_BF16 && grad_x_type != LEAP_F32) return refuse("grad_x is bfloat16 or float32");
    if (rows && (!d_dy || !d_codes || !d_scales || !d_weight)) return refuse("null data pointer");
    if (!d_work && act::linear8_backward_work(d_dy, dy_stride, padded, d_codes, rows, cols, d_weight, w_stride, out)) return refuse("null workspace");
    const hipStream_t st = stream_of(hip_stream);
    uint8_t *room = (uint8_t *)d_work;
    laid G(d_dy, dy_stride, rows, out, 2, padded), W(d_weight, w_stride, out, cols, 2), X(d_codes, cols, rows, cols, 1);
    int rc = lay_out(room, st, &G, d_grad_x && rows ? &W : nullptr, d_grad_weight ? &X : nullptr);
    if (rc == LEAP_OK && d_grad_x && rows) {
        result R{};
        R.out = d_grad_x, R.stride = cols;
        const operand P = W.wide(cols, out), Q = G.wide(rows, out);
        const depth_plan plan(cols, rows, out);
        if (plan.parts > 1) {
            rc = product_in_parts<WIDE_ACROSS, WIDE_ALONG>(P, Q, d_grad_x, grad_x_type, plan, room, st);
            room += plan.room(cols, rows);
        } else
            rc = grad_x_type == LEAP_F32 ? product<WIDE_ACROSS, WIDE_ALONG, TO_FULL>(P, Q, R, st) : product<WIDE_ACROSS, WIDE_ALONG, TO_WIDE>(P, Q, R, st);
    }
    if (rc != LEAP_OK || !d_grad_weight) return rc;
    const int64_t added = cut(cols * out, ADDED);
    if (added > 0x7fffffff) return refuse("a weight of more than 2^37 values");
    const dim3 adders((unsigned)added);
    if (!rows) {                                     // a sum of nothing
        hipLaunchKernelGGL((k_add_parts<LEAP_BF16>), adders, dim3(BLOCK), 0, st, (const float *)nullptr, (int64_t)0, cols * out, d_grad_weight);
        return launched();
    }
    const weight_plan plan(rows, cols, out);
    const operand P = X.codes(d_scales, cols, cols, rows), Q = G.wide(out, rows);
    result R{};
    R.stride = cols, R.part = cols * out;
    if (plan.parts == 1) {
        R.out = d_grad_weight;
        return product<CODES_ACROSS, WIDE_ACROSS, TO_WIDE>(P, Q, R, 0, plan.large, st);
    }
    R.out = room;
    rc = product<CODES_ACROSS, WIDE_ACROSS, TO_FULL>(P, Q, R, plan.depth_part, plan.large, st);
    if (rc != LEAP_OK) return rc;
    hipLaunchKernelGGL((k_add_parts<LEAP_BF16>), adders, dim3(BLOCK), 0, st, (const float *)room, plan.parts, cols * out, d_grad_weight);
    return launched();
}

extern "C" int64_t leap_linear8_backward_work(const void *d_dy, int64_t dy_stride, const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight,
                                              int64_t w_stride, int64_t out)
{
    return act::linear8_backward_work(d_dy, dy_stride, false, d_codes, rows, cols, d_weight, w_stride, out);
}

extern "C" int leap_linear8_backward(const void *d_dy, int64_t dy_stride, const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols,
                                     const void *d_weight, int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight,
                                     void *d_work, void *hip_stream)
{
    return act::linear8_backward(d_dy, dy_stride, false, d_codes, d_scales, rows, cols, d_weight, w_stride, out, d_grad_x, grad_x_type, d_grad_weight, d_work,
                                 hip_stream);
}

extern "C" int leap_gated_linear8(const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride,
                                  int64_t out, uint8_t *d_gated_codes, uint8_t *d_gated_scales, uint8_t *d_kept_codes, uint8_t *d_kept_scales,
                                  void *d_work, void *hip_stream)
{
    if (out > MOST_COLS / 2) return refuse(GATED_LIMIT);
    if (const char *why = bad_product(rows, cols, w_stride, 2 * out)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_codes || !d_scales || !d_weight || !d_gated_codes || !d_gated_scales) return refuse("null data pointer");
    if (!d_kept_codes != !d_kept_scales) return refuse("kept codes and scales: both or neither");
    if (!d_work && leap_linear8_work(d_codes, rows, cols, d_weight, w_stride, 2 * out)) return refuse("null workspace");
    const hipStream_t st = stream_of(hip_stream);
    uint8_t *room = (uint8_t *)d_work;
    laid W(d_weight, w_stride, 2 * out, cols, 2), X(d_codes, cols, rows, cols, 1);
    const int rc = lay_out(room, st, &W, &X);
    if (rc != LEAP_OK) return rc;
    result R{};
    R.columns = out, R.gated_codes = d_gated_codes, R.gated_scales = d_gated_scales, R.kept_codes = d_kept_codes, R.kept_scales = d_kept_scales;
    return product<WIDE_ALONG, CODES_ALONG, TO_GATED>(W.wide(2 * out, cols), X.codes(d_scales, cols, rows, cols), R, st);
}

namespace {

int gate_backward(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows, int64_t out, void *d_du,
                  int64_t du_stride, void *hip_stream)
{
    if (out > MOST_COLS / 2) return refuse(GATED_LIMIT);
    if (const char *why = bad_sizes(rows, out)) return refuse(why);
    if (const char *why = bad_stride(da_stride, rows, out)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_da || !d_kept_codes || !d_kept_scales || !d_du) return refuse("null data pointer");
    const int64_t blocks = cut(rows * groups_of(out) * (GROUP / CHUNK), BLOCK);
    if (blocks > 0x7fffffff) return refuse("more values than one launch covers");
    hipLaunchKernelGGL(k_gate_grad, dim3((unsigned)blocks), dim3(BLOCK), 0, stream_of(hip_stream), d_da, da_stride, d_kept_codes, d_kept_scales, rows, out, d_du,
                       du_stride);
    return launched();
}

}  // namespace

extern "C" int leap_gate8_backward(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows,
                                   int64_t out, void *d_du, void *hip_stream)
{
    return gate_backward(d_da, da_stride, d_kept_codes, d_kept_scales, rows, out, d_du, 2 * out, hip_stream);
}

extern "C" int64_t leap_gated_linear8_backward_work(const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out)
{
    if (out > MOST_COLS / 2 || out < 1 || bad_product(rows, cols, w_stride, 2 * out)) return 0;
    return rows * padded_row(2 * out) * 2 + act::linear8_backward_work((const void *)16, padded_row(2 * out), true, d_codes, rows, cols, d_weight, w_stride, 2 * out);
}

extern "C" int leap_gated_linear8_backward(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales,
                                           const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight,
                                           int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight, void *d_work,
                                           void *hip_stream)
{
    if (out > MOST_COLS / 2) return refuse(GATED_LIMIT);
    if (const char *why = bad_product(rows, cols, w_stride, 2 * out)) return refuse(why);
    if (const char *why = bad_stride(da_stride, rows, out)) return refuse(why);
    if (grad_x_type != LEAP_BF16 && grad_x_type != LEAP_F32) return refuse("grad_x is bfloat16 or float32");
    if (rows && (!d_codes || !d_scales || !d_weight)) return refuse("null data pointer");
    if (rows && (!d_work || (uintptr_t)d_work % 16 != 0)) return refuse("the workspace needs memory from a multiple of 16 bytes on");
    if (!d_grad_x && !d_grad_weight) return LEAP_OK;
    const int64_t stride = padded_row(2 * out);
    const int rc = gate_backward(d_da, da_stride, d_kept_codes, d_kept_scales, rows, out, d_work, stride, hip_stream);
    if (rc != LEAP_OK) return rc;
    return act::linear8_backward(d_work, stride, true, d_codes, d_scales, rows, cols, d_weight, w_stride, 2 * out, d_grad_x, grad_x_type, d_grad_weight,
                                 rows ? (uint8_t *)d_work + rows * stride * 2 : nullptr, hip_stream);
}

extern "C" int64_t leap_linear_gate8_work(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next, int64_t rows, int64_t out)
{
    if (bad_product(rows, out, w_stride, next) || bad_stride(dy_stride, rows, next)) return 0;
    return laid(d_dy, dy_stride, rows, next, 2).room() + laid(d_weight, w_stride, next, out, 2).room();
}

int act::linear_gate8_backward(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next, const uint8_t *d_kept_codes,
                               const uint8_t *d_kept_scales, int64_t rows, int64_t out, void *d_du, int64_t du_stride, void *d_work, void *hip_stream)
{
    if (out > MOST_COLS / 2) return refuse(GATED_LIMIT);
    if (const char *why = bad_product(rows, out, w_stride, next)) return refuse(why);
    if (const char *why = bad_stride(dy_stride, rows, next)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_dy || !d_weight || !d_kept_codes || !d_kept_scales || !d_du) return refuse("null data pointer");
    if (!d_work && leap_linear_gate8_work(d_dy, dy_stride, d_weight, w_stride, next, rows, out)) return refuse("null workspace");
    const hipStream_t st = stream_of(hip_stream);
    uint8_t *room = (uint8_t *)d_work;
    laid W(d_weight, w_stride, next, out, 2), G(d_dy, dy_stride, rows, next, 2);
    const int rc = lay_out(room, st, &W, &G);
    if (rc != LEAP_OK) return rc;
    if (du_stride > 2 * out) hipLaunchKernelGGL(k_pad_rows, dim3((unsigned)cut(rows, BLOCK)), dim3(BLOCK), 0, st, (uint16_t *)d_du, du_stride, rows, 2 * out);
    result R{};
    R.out = d_du, R.stride = du_stride, R.columns = out, R.kept_codes = (uint8_t *)d_kept_codes, R.kept_scales = (uint8_t *)d_kept_scales;
    return product<WIDE_ACROSS, WIDE_ALONG, TO_GATE_GRAD>(W.wide(out, next), G.wide(rows, next), R, st);
}

extern "C" int leap_linear_gate8_backward(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next,
                                          const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows, int64_t out, void *d_du,
                                          void *d_work, void *hip_stream)
{
    return act::linear_gate8_backward(d_dy, dy_stride, d_weight, w_stride, next, d_kept_codes, d_kept_scales, rows, out, d_du, 2 * out, d_work, hip_stream);
}
