// Products with rows held in 8 bits, and the gated product: leap_linear8 and its kin (act_product.h has the kernel).
//
// Its fetches want memory rows that begin at multiples of 16 bytes.  Operands that do not (odd sizes, odd strides) are
// first laid out anew in the workspace, a pass over them that costs a few percent of the product.
#include "act_product.h"

namespace {

using namespace act;

constexpr int BLOCK = 256;

// ---- operands laid out for the product ----

// An array whose rows, `bytes` long, are copied to rows of `pitch` bytes (a multiple of 16) with zeros at their ends; `rows` of them are
// written, those beyond the `there` that it has as zeros.
struct copied_rows {
    const uint8_t *from;
    uint8_t *to;
    int64_t stride, there, rows, bytes, pitch;
    divider pieces;              // of 16 bytes, of a row
    uint32_t blocks;             // that copy it
};

struct copies {
    copied_rows of[3];
};

__global__ __launch_bounds__(BLOCK) void k_lay_out(copies C, uint32_t first_block)
{
    uint32_t block = first_block + blockIdx.x;
    int c = 0;
    while (c < 2 && block >= C.of[c].blocks) block -= C.of[c++].blocks;
    const copied_rows &A = C.of[c];
    // a block's first piece may lie beyond 32 bits, what it holds of rows may not
    const int64_t first = (int64_t)block * BLOCK, row0 = first / A.pieces.by;
    const uint32_t q = (uint32_t)(first - row0 * A.pieces.by) + threadIdx.x, in = A.pieces(q);
    const int64_t row = row0 + in, at = (int64_t)(q - in * A.pieces.by) * 16;
    if (row >= A.rows) return;
    uint8_t piece[16] = {};
    const int64_t left = row < A.there ? A.bytes - at : 0;
    if (left >= 16) {
        __builtin_memcpy(piece, A.from + row * A.stride + at, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 15; ++i)
            if (i < left) piece[i] = A.from[row * A.stride + at + i];
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
    int64_t rows_to;                                 // of a copy: zeros behind the rows there are
    bool copied;
    laid(const void *p, int64_t stride_, int64_t rows_, int64_t cols, int size)
        : data((const uint8_t *)p), stride(stride_ * size), rows(rows_), bytes(cols * size), pitch(up16(cols * size)), rows_to(rows_)
    {
        copied = rows > 0 && (stride % 16 != 0 || bytes % 16 != 0 || (uintptr_t)p % 16 != 0 || stride < bytes || stride > FAR_APART);
    }
    int64_t room() const { return copied ? rows_to * pitch : 0; }

    operand wide(int64_t i, int64_t k) const { return {data, nullptr, stride / 2, 0, i, k}; }
    operand codes(const uint8_t *scales, int64_t cols, int64_t i, int64_t k) const { return {data, scales, stride, groups_of(cols), i, k}; }
};

// The copies of up to three arrays, into `room` one after the other, which moves on.
int lay_out(uint8_t *&room, hipStream_t st, laid *a, laid *b = nullptr, laid *c = nullptr)
{
    copies C = {{{nullptr, nullptr, 0, 0, 0, 0, 16, divider(1), 0}, {nullptr, nullptr, 0, 0, 0, 0, 16, divider(1), 0}, {nullptr, nullptr, 0, 0, 0, 0, 16, divider(1), 0}}};
    int64_t blocks = 0;
    int n = 0;
    for (laid *x : {a, b, c}) {
        if (!x || !x->copied) continue;
        const int64_t mine = cut(x->rows_to * (x->pitch / 16), BLOCK);
        blocks += mine;
        if (blocks > 0x7fffffff) return refuse("more values to lay out than 31 bits count blocks for");
        C.of[n++] = {x->data, room, x->stride, x->rows, x->rows_to, x->bytes, x->pitch, divider((uint32_t)(x->pitch / 16)), (uint32_t)mine};
        x->data = room, x->stride = x->pitch, x->copied = false;
        room += x->rows_to * x->pitch;
    }
    return over_blocks(blocks, [&](int64_t first, unsigned some) { hipLaunchKernelGGL(k_lay_out, dim3(some), dim3(BLOCK), 0, st, C, (uint32_t)first); });
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
    if constexpr (!gate_grad<TO>())
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
    // n: values of a part
    int64_t room(int64_t n, bool always) const { return parts > 1 || always ? up16(parts * n * (int64_t)sizeof(float)) : 0; }
};

// to <- the sum of the parts, n values every `apart`, in a fixed order: 16 threads to four values each, which add every 16th part, 64 values a block.
constexpr int ADDED = 64;

template <int TYPE> __global__ __launch_bounds__(BLOCK) void k_add_parts(const float *__restrict__ from, int64_t parts, int64_t apart, int64_t n, void *__restrict__ to,
                                                                             int64_t first_block)
{
    constexpr int WAYS = BLOCK / (ADDED / 4);
    __shared__ float room[WAYS][ADDED];
    const int way = threadIdx.x / (ADDED / 4), in = threadIdx.x % (ADDED / 4) * 4;
    const int64_t begin = (first_block + blockIdx.x) * ADDED, at = begin + in;
    const int left = n - at < 4 ? (int)(n - at) : 4;
    float sum[4] = {};
    if (left == 4) {
#pragma unroll 4
        for (int64_t p = way; p < parts; p += WAYS) {
            float f[4];
            __builtin_memcpy(f, from + p * apart + at, 16);
#pragma unroll
            for (int x = 0; x < 4; ++x) sum[x] += f[x];
        }
    } else {
        for (int64_t p = way; p < parts; p += WAYS)
            for (int x = 0; x < left; ++x) sum[x] += from[p * apart + at + x];
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) room[way][in + x] = sum[x];
    __syncthreads();
    if (threadIdx.x < ADDED && begin + threadIdx.x < n) {
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < WAYS; ++w) total += room[w][threadIdx.x];
        ((typename element<TYPE>::raw *)to)[begin + threadIdx.x] = element<TYPE>::from_float(total);
    }
}

int add_parts(const float *from, int64_t parts, int64_t apart, int64_t n, void *to, int32_t type, hipStream_t st)
{
    return over_blocks(cut(n, ADDED), [&](int64_t first, unsigned blocks) {
        if (type == LEAP_F32) hipLaunchKernelGGL((k_add_parts<LEAP_F32>), dim3(blocks), dim3(BLOCK), 0, st, from, parts, apart, n, to, first);
        else hipLaunchKernelGGL((k_add_parts<LEAP_BF16>), dim3(blocks), dim3(BLOCK), 0, st, from, parts, apart, n, to, first);
    });
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
    return add_parts((const float *)room, plan.parts, R.part, R.part, out, type, st);
}

// ---- the gate by itself ----

// Zeros behind the values of a row of du, of both of its parts.
__device__ inline void pad_row(uint16_t *row, int64_t values, const du_layout &L)
{
    const int64_t end = L.low ? L.low : L.stride;
    for (int64_t i = values; i < end; ++i) row[i] = 0;
    if (L.low)
        for (int64_t i = L.low + values; i < L.stride; ++i) row[i] = 0;
}

// du <- da and what is kept, and zeros between its rows; one chunk of `out` a lane
__global__ __launch_bounds__(BLOCK) void k_gate_grad(const void *__restrict__ da, int64_t stride, const uint8_t *__restrict__ kept_codes,
                                                     const uint8_t *__restrict__ kept_scales, int64_t rows, int64_t out, void *__restrict__ du,
                                                     du_layout L, int64_t first_block)
{
    const int64_t groups = groups_of(out), per_row = groups * (GROUP / CHUNK), c = (first_block + blockIdx.x) * BLOCK + threadIdx.x;
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
    const bool past = L.bytes(rows) > READ_NEXT;
    store8<LEAP_BF16>(du, row * L.stride + col, n, dg, past);
    store8<LEAP_BF16>(du, row * L.stride + out + col, n, dp, past);
    if (L.low) {
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) dg[i] = rest_of_bf16(dg[i]), dp[i] = rest_of_bf16(dp[i]);
        store8<LEAP_BF16>(du, row * L.stride + L.low + col, n, dg, past);
        store8<LEAP_BF16>(du, row * L.stride + L.low + out + col, n, dp, past);
    }
    if (col + n == out) pad_row((uint16_t *)du + row * L.stride, 2 * out, L);
}

// The same zeros by themselves, a row a thread.
__global__ __launch_bounds__(BLOCK) void k_pad_rows(uint16_t *__restrict__ du, int64_t rows, int64_t values, du_layout L, int64_t first_block)
{
    const int64_t row = (first_block + blockIdx.x) * BLOCK + threadIdx.x;
    if (row < rows) pad_row(du + row * L.stride, values, L);
}

const char *bad_product(int64_t rows, int64_t cols, int64_t w_stride, int64_t out)
{
    if (const char *why = bad_sizes(rows, cols)) return why;
    if (const char *why = bad_sizes(rows, out)) return why;
    return bad_stride(w_stride, out, cols);
}

constexpr const char *NO_FINE = "a fine gradient needs memory from a multiple of 16 bytes on";
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
    if (unaligned(d_work) && leap_linear8_work(d_codes, rows, cols, d_weight, w_stride, out)) return refuse(NO_WORK);
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

namespace {

// The gradients of v W^T from G, which is dy; or, with low, dy and what its rounding leaves, `low` values further on: then grad_x multiplies rows
// twice as long with the weight twice, one below the other, and grad_weight adds the two halves of twice as many rows.
int64_t backward_work(const laid &G, int64_t low, const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out)
{
    if (!rows) return 0;                             // of nothing: nothing is laid out
    const int64_t deep = low + out;
    laid W(d_weight, w_stride, out, cols, 2);
    const int64_t weight = low ? (low + out) * W.pitch : W.room();
    return weight_plan(rows, cols, deep).room(cols * (low ? 2 * low : out), low != 0) + depth_plan(cols, rows, deep).room(cols, rows) + G.room() +
           laid(d_codes, cols, rows, cols, 1).room() + weight;
}

int backward(laid G, int64_t low, const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride,
             int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight, void *d_work, void *hip_stream)
{
    if (grad_x_type != LEAP_BF16 && grad_x_type != LEAP_F32) return refuse("grad_x is bfloat16 or float32");
    if (rows && (!G.data || !d_codes || !d_scales || !d_weight)) return refuse("null data pointer");
    if (unaligned(d_work) && backward_work(G, low, d_codes, rows, cols, d_weight, w_stride, out)) return refuse(NO_WORK);
    const hipStream_t st = stream_of(hip_stream);
    uint8_t *room = (uint8_t *)d_work;
    const int64_t deep = low + out;
    laid W(d_weight, w_stride, out, cols, 2), again = W, X(d_codes, cols, rows, cols, 1);
    if (low) W.copied = again.copied = true, W.rows_to = low;
    laid *const w = d_grad_x && rows ? &W : nullptr;
    int rc = lay_out(room, st, low ? w : &G, low && w ? &again : w, d_grad_weight ? &X : nullptr);
    if (rc == LEAP_OK && d_grad_x && rows) {
        result R{};
        R.out = d_grad_x, R.stride = cols;
        const operand P = W.wide(cols, deep), Q = G.wide(rows, deep);
        const depth_plan plan(cols, rows, deep);
        if (plan.parts > 1) {
            rc = product_in_parts<WIDE_ACROSS, WIDE_ALONG>(P, Q, d_grad_x, grad_x_type, plan, room, st);
            room += plan.room(cols, rows);
        } else
            rc = grad_x_type == LEAP_F32 ? product<WIDE_ACROSS, WIDE_ALONG, TO_FULL>(P, Q, R, st) : product<WIDE_ACROSS, WIDE_ALONG, TO_WIDE>(P, Q, R, st);
    }
    if (rc != LEAP_OK || !d_grad_weight) return rc;
    if (!rows) return add_parts(nullptr, 0, 0, cols * out, d_grad_weight, LEAP_BF16, st);        // a sum of nothing
    const weight_plan plan(rows, cols, deep);
    const operand P = X.codes(d_scales, cols, cols, rows), Q = G.wide(deep, rows);
    result R{};
    R.stride = cols, R.part = cols * (low ? 2 * low : out);
    if (plan.parts == 1 && !low) {
        R.out = d_grad_weight;
        return product<CODES_ACROSS, WIDE_ACROSS, TO_WIDE>(P, Q, R, 0, plan.large, st);
    }
    R.out = room;
    rc = product<CODES_ACROSS, WIDE_ACROSS, TO_FULL>(P, Q, R, plan.depth_part, plan.large, st);
    if (rc != LEAP_OK) return rc;
    return add_parts((const float *)room, low ? 2 * plan.parts : plan.parts, low ? low * cols : R.part, cols * out, d_grad_weight, LEAP_BF16, st);
}

// du's rows end at a multiple of 16 bytes: they are never copied.
laid du_rows(const void *d_du, const du_layout &L, int64_t rows) { return laid(d_du, L.stride, rows, L.stride, 2); }

}  // namespace

int64_t act::du_backward_work(const du_layout &L, const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out)
{
    if (bad_product(rows, cols, w_stride, out)) return 0;
    return backward_work(du_rows((const void *)16 /* aligned, as it will be */, L, rows), L.low, d_codes, rows, cols, d_weight, w_stride, out);
}

int act::du_backward(const void *d_du, const du_layout &L, const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight,
                     int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight, void *d_work, void *hip_stream)
{
    if (const char *why = bad_product(rows, cols, w_stride, out)) return refuse(why);
    return backward(du_rows(d_du, L, rows), L.low, d_codes, d_scales, rows, cols, d_weight, w_stride, out, d_grad_x, grad_x_type, d_grad_weight, d_work, hip_stream);
}

extern "C" int64_t leap_linear8_backward_work(const void *d_dy, int64_t dy_stride, const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight,
                                              int64_t w_stride, int64_t out)
{
    if (bad_product(rows, cols, w_stride, out) || bad_stride(dy_stride, rows, out)) return 0;
    return backward_work(laid(d_dy, dy_stride, rows, out, 2), 0, d_codes, rows, cols, d_weight, w_stride, out);
}

extern "C" int leap_linear8_backward(const void *d_dy, int64_t dy_stride, const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols,
                                     const void *d_weight, int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight,
                                     void *d_work, void *hip_stream)
{
    if (const char *why = bad_product(rows, cols, w_stride, out)) return refuse(why);
    if (const char *why = bad_stride(dy_stride, rows, out)) return refuse(why);
    return backward(laid(d_dy, dy_stride, rows, out, 2), 0, d_codes, d_scales, rows, cols, d_weight, w_stride, out, d_grad_x, grad_x_type, d_grad_weight, d_work,
                    hip_stream);
}

extern "C" int64_t leap_linear8_backward_fine_work(const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out)
{
    return act::du_backward_work({padded_row(out), 2 * padded_row(out)}, d_codes, rows, cols, d_weight, w_stride, out);
}

extern "C" int leap_linear8_backward_fine(const void *d_dy, const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight,
                                          int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight, void *d_work,
                                          void *hip_stream)
{
    if (rows && unaligned(d_dy)) return refuse(NO_FINE);
    return act::du_backward(d_dy, {padded_row(out), 2 * padded_row(out)}, d_codes, d_scales, rows, cols, d_weight, w_stride, out, d_grad_x, grad_x_type,
                            d_grad_weight, d_work, hip_stream);
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
    if (unaligned(d_work) && leap_linear8_work(d_codes, rows, cols, d_weight, w_stride, 2 * out)) return refuse(NO_WORK);
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
                  const du_layout &L, void *hip_stream)
{
    if (out > MOST_COLS / 2) return refuse(GATED_LIMIT);
    if (const char *why = bad_sizes(rows, out)) return refuse(why);
    if (const char *why = bad_stride(da_stride, rows, out)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_da || !d_kept_codes || !d_kept_scales || !d_du) return refuse("null data pointer");
    return over_blocks(cut(rows * groups_of(out) * (GROUP / CHUNK), BLOCK), [&](int64_t first, unsigned blocks) {
        hipLaunchKernelGGL(k_gate_grad, dim3(blocks), dim3(BLOCK), 0, stream_of(hip_stream), d_da, da_stride, d_kept_codes, d_kept_scales, rows, out, d_du, L, first);
    });
}

}  // namespace

extern "C" int leap_gate8_backward(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows,
                                   int64_t out, void *d_du, void *hip_stream)
{
    return gate_backward(d_da, da_stride, d_kept_codes, d_kept_scales, rows, out, d_du, du_layout{0, 2 * out}, hip_stream);
}

extern "C" int leap_gate8_backward_fine(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows,
                                        int64_t out, void *d_du, void *hip_stream)
{
    if (rows && unaligned(d_du)) return refuse(NO_FINE);
    return gate_backward(d_da, da_stride, d_kept_codes, d_kept_scales, rows, out, d_du, padded_layout(out, true), hip_stream);
}

namespace {

int64_t gated_backward_work(bool fine, const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out)
{
    if (out > MOST_COLS / 2 || out < 1 || bad_product(rows, cols, w_stride, 2 * out)) return 0;
    const du_layout L = padded_layout(out, fine);
    return L.bytes(rows) + act::du_backward_work(L, d_codes, rows, cols, d_weight, w_stride, 2 * out);
}

int gated_backward(bool fine, const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, const uint8_t *d_codes,
                   const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out, void *d_grad_x,
                   int32_t grad_x_type, void *d_grad_weight, void *d_work, void *hip_stream)
{
    if (out > MOST_COLS / 2) return refuse(GATED_LIMIT);
    if (const char *why = bad_product(rows, cols, w_stride, 2 * out)) return refuse(why);
    if (const char *why = bad_stride(da_stride, rows, out)) return refuse(why);
    if (grad_x_type != LEAP_BF16 && grad_x_type != LEAP_F32) return refuse("grad_x is bfloat16 or float32");
    if (rows && (!d_codes || !d_scales || !d_weight)) return refuse("null data pointer");
    if (rows && unaligned(d_work)) return refuse(NO_WORK);
    if (!d_grad_x && !d_grad_weight) return LEAP_OK;
    // The matrix units take bfloat16.  A fine du is two of those, and its products take twice as long (262144 x 512 -> 2 * 1024 forward and backward:
    // 3.47 ms, 2.25); the results are 0.0017 of their norm off, their own rounding to bfloat16.  With du rounded, which a caller may ask for, 0.0024.
    const du_layout L = padded_layout(out, fine);
    const int rc = gate_backward(d_da, da_stride, d_kept_codes, d_kept_scales, rows, out, d_work, L, hip_stream);
    if (rc != LEAP_OK) return rc;
    return act::du_backward(d_work, L, d_codes, d_scales, rows, cols, d_weight, w_stride, 2 * out, d_grad_x, grad_x_type, d_grad_weight,
                            rows ? (uint8_t *)d_work + L.bytes(rows) : nullptr, hip_stream);
}

}  // namespace

extern "C" int64_t leap_gated_linear8_backward_work(const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out)
{
    return gated_backward_work(false, d_codes, rows, cols, d_weight, w_stride, out);
}

extern "C" int leap_gated_linear8_backward(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales,
                                           const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight,
                                           int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight, void *d_work,
                                           void *hip_stream)
{
    return gated_backward(false, d_da, da_stride, d_kept_codes, d_kept_scales, d_codes, d_scales, rows, cols, d_weight, w_stride, out, d_grad_x, grad_x_type,
                          d_grad_weight, d_work, hip_stream);
}

extern "C" int64_t leap_gated_linear8_backward_fine_work(const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out)
{
    return gated_backward_work(true, d_codes, rows, cols, d_weight, w_stride, out);
}

extern "C" int leap_gated_linear8_backward_fine(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales,
                                                const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight,
                                                int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight, void *d_work,
                                                void *hip_stream)
{
    return gated_backward(true, d_da, da_stride, d_kept_codes, d_kept_scales, d_codes, d_scales, rows, cols, d_weight, w_stride, out, d_grad_x, grad_x_type,
                          d_grad_weight, d_work, hip_stream);
}

extern "C" int64_t leap_linear_gate8_work(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next, int64_t rows, int64_t out)
{
    if (bad_product(rows, out, w_stride, next) || bad_stride(dy_stride, rows, next)) return 0;
    return laid(d_dy, dy_stride, rows, next, 2).room() + laid(d_weight, w_stride, next, out, 2).room();
}

int act::linear_gate8_backward(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next, const uint8_t *d_kept_codes,
                               const uint8_t *d_kept_scales, int64_t rows, int64_t out, void *d_du, const du_layout &L, void *d_work, void *hip_stream)
{
    if (out > MOST_COLS / 2) return refuse(GATED_LIMIT);
    if (const char *why = bad_product(rows, out, w_stride, next)) return refuse(why);
    if (const char *why = bad_stride(dy_stride, rows, next)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_dy || !d_weight || !d_kept_codes || !d_kept_scales || !d_du) return refuse("null data pointer");
    if (unaligned(d_work) && leap_linear_gate8_work(d_dy, dy_stride, d_weight, w_stride, next, rows, out)) return refuse(NO_WORK);
    const hipStream_t st = stream_of(hip_stream);
    uint8_t *room = (uint8_t *)d_work;
    laid W(d_weight, w_stride, next, out, 2), G(d_dy, dy_stride, rows, next, 2);
    int rc = lay_out(room, st, &W, &G);
    if (rc == LEAP_OK && 2 * out % 8 != 0 && L.stride > 2 * out)
        rc = over_blocks(cut(rows, BLOCK), [&](int64_t first, unsigned blocks) {
            hipLaunchKernelGGL(k_pad_rows, dim3(blocks), dim3(BLOCK), 0, st, (uint16_t *)d_du, rows, 2 * out, L, first);
        });
    // a block a tile here: as many rows at once as a launch has blocks for
    const int64_t at_once = MOST_BLOCKS / cut(out, 128) * 128;
    for (int64_t row0 = 0; rc == LEAP_OK && row0 < rows; row0 += at_once) {
        const int64_t n = rows - row0 < at_once ? rows - row0 : at_once;
        operand Q = G.wide(n, next);
        Q.data += row0 * G.stride;
        result R{};
        R.out = (uint8_t *)d_du + L.bytes(row0), R.stride = L.stride, R.low = L.low, R.columns = out;
        R.kept_codes = (uint8_t *)d_kept_codes + row0 * 2 * out, R.kept_scales = (uint8_t *)d_kept_scales + row0 * 2 * groups_of(out);
        rc = L.low ? product<WIDE_ACROSS, WIDE_ALONG, TO_GATE_GRAD_FINE>(W.wide(out, next), Q, R, st)
                   : product<WIDE_ACROSS, WIDE_ALONG, TO_GATE_GRAD>(W.wide(out, next), Q, R, st);
    }
    return rc;
}

extern "C" int leap_linear_gate8_backward(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next,
                                          const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows, int64_t out, void *d_du,
                                          void *d_work, void *hip_stream)
{
    return act::linear_gate8_backward(d_dy, dy_stride, d_weight, w_stride, next, d_kept_codes, d_kept_scales, rows, out, d_du, du_layout{0, 2 * out}, d_work, hip_stream);
}

extern "C" int leap_linear_gate8_backward_fine(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next,
                                               const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows, int64_t out, void *d_du,
                                               void *d_work, void *hip_stream)
{
    if (rows && unaligned(d_du)) return refuse(NO_FINE);
    return act::linear_gate8_backward(d_dy, dy_stride, d_weight, w_stride, next, d_kept_codes, d_kept_scales, rows, out, d_du, padded_layout(out, true), d_work, hip_stream);
}
