// What the operators on activations in 8 bits share: the format's arithmetic, vector access without alignment, launch helpers.
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>

#include <stdint.h>

#include <string>
#include <type_traits>

#include "../../include/leap.h"
#include "../../include/leap_activations.h"

void leap_set_error(const std::string &msg);
int leap_hip_fail(hipError_t e, const char *what);

namespace act {

constexpr int GROUP = 32;              // values that share a scale
constexpr int CHUNK = 8;               // values a lane handles at once; four neighbouring lanes hold a group
constexpr int64_t MOST_VALUES = (int64_t)1 << 42, MOST_COLS = (int64_t)1 << 20;

inline __host__ __device__ int64_t groups_of(int64_t cols) { return (cols + GROUP - 1) / GROUP; }

// ---- element types ----

template <int TYPE> struct element;
template <> struct element<LEAP_F32> {
    using raw = float;
    static __device__ float to_float(raw v) { return v; }
    static constexpr float LARGEST = 0x1.fffffep127f;
    static __device__ raw from_float(float v) { return v; }
};
template <> struct element<LEAP_BF16> {
    using raw = uint16_t;
    static __device__ float to_float(raw v) { return __uint_as_float((uint32_t)v << 16); }
    static constexpr float LARGEST = 0x1.fep127f;
    static __device__ raw from_float(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
};
template <> struct element<LEAP_F16> {
    using raw = uint16_t;
    static __device__ float to_float(raw v) { return (float)__builtin_bit_cast(_Float16, v); }
    static constexpr float LARGEST = 65504.0f;
    static __device__ raw from_float(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};

// Eight values of a row from `p` on, of which `n` are there (the others read as zeros).  Any alignment: the loads are
// as wide as the type's eight values, which the hardware splits where an address asks for it.
template <int TYPE> __device__ inline void load8(const void *base, int64_t at, int n, float (&v)[CHUNK])
{
    using raw = typename element<TYPE>::raw;
    const raw *p = (const raw *)base + at;
    raw r[CHUNK] = {};
    if (n >= CHUNK) {
        __builtin_memcpy(r, p, sizeof r);
    } else {
#pragma unroll
        for (int i = 0; i < CHUNK - 1; ++i)
            if (i < n) r[i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) v[i] = element<TYPE>::to_float(r[i]);
}

// Outputs of more than this go past the caches: little of them is left there when they are read, and they push out what is (2^27
// bfloat16 values unpacked: 57 us, 68 through the caches; packed 61 and 70).
// What the next kernel reads pays from further on, the 256 MB cache in mind (du of 18414 x 2058 and of 16384 x 2048, in bfloat16, through the caches: a
// gated step 213 us, 220 past them, a block's 273 and 284).
constexpr int64_t PAST_CACHES = (int64_t)64 << 20, READ_NEXT = (int64_t)192 << 20;

typedef uint32_t words4 __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t words2 __attribute__((ext_vector_type(2), aligned(1)));

// BYTES (8, 16 or 32) to any address.
template <int BYTES> __device__ inline void store_bytes(void *to, const void *from, bool past)
{
    if (past) {
        asm volatile("");            // between two of these the compiler does not make one plain store of both branches
        if constexpr (BYTES == 8) {
            words2 w;
            __builtin_memcpy(&w, from, 8);
            __builtin_nontemporal_store(w, (words2 *)to);
        } else {
#pragma unroll
            for (int i = 0; i < BYTES; i += 16) {
                words4 w;
                __builtin_memcpy(&w, (const char *)from + i, 16);
                __builtin_nontemporal_store(w, (words4 *)((char *)to + i));
            }
        }
        asm volatile("");
    } else {
        __builtin_memcpy(to, from, BYTES);
    }
}

template <int TYPE> __device__ inline void store8(void *base, int64_t at, int n, const float (&v)[CHUNK], bool past = false)
{
    using raw = typename element<TYPE>::raw;
    raw *p = (raw *)base + at;
    raw r[CHUNK];
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) r[i] = element<TYPE>::from_float(v[i]);
    if (n >= CHUNK) {
        store_bytes<sizeof r>(p, r, past);
    } else {
#pragma unroll
        for (int i = 0; i < CHUNK - 1; ++i)
            if (i < n) p[i] = r[i];
    }
}

// ---- the format ----

// Magnitude of v as an integer that orders like it; 0 for infinities and NaN, which do not take part in the scale.
__device__ inline uint32_t finite_magnitude(float v)
{
    const uint32_t bits = __float_as_uint(v) & 0x7fffffffu;
    return bits < 0x7f800000u ? bits : 0u;
}

// The scale byte of a group: e + 127 for the smallest e >= -127 with amax <= 448 * 2^e.  448 = 1.75 * 2^8: a mantissa of
// at most 0x600000 keeps its exponent, a larger one carries into the next.
__device__ inline uint32_t scale_byte(uint32_t amax_bits)
{
    const int e = (int)((amax_bits + 0x1fffffu) >> 23) - 8;
    return e > 0 ? (uint32_t)e : 0u;
}

__device__ inline float scale_value(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }   // 2^(byte - 127)
__device__ inline float scale_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }            // byte <= 247

// Codes of eight values; the conversion rounds to nearest, ties to even, and makes NaN of what is not finite.
__device__ inline uint2 encode8(const float (&v)[CHUNK], float inverse)
{
    uint32_t lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inverse, v[1] * inverse, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inverse, v[3] * inverse, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inverse, v[5] * inverse, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inverse, v[7] * inverse, hi, true);
    return make_uint2(lo, hi);
}

__device__ inline void decode8(uint2 codes, float scale, float (&v)[CHUNK])
{
    auto a = __builtin_amdgcn_cvt_pk_f32_fp8(codes.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(codes.x, true);
    auto c = __builtin_amdgcn_cvt_pk_f32_fp8(codes.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8(codes.y, true);
    v[0] = a[0] * scale, v[1] = a[1] * scale, v[2] = b[0] * scale, v[3] = b[1] * scale;
    v[4] = c[0] * scale, v[5] = c[1] * scale, v[6] = d[0] * scale, v[7] = d[1] * scale;
}

__device__ inline uint2 load_codes(const uint8_t *p, int n)
{
    uint2 c = make_uint2(0, 0);
    if (n >= CHUNK) {
        __builtin_memcpy(&c, p, CHUNK);
    } else {
        uint8_t b[CHUNK] = {};
#pragma unroll
        for (int i = 0; i < CHUNK - 1; ++i)
            if (i < n) b[i] = p[i];
        __builtin_memcpy(&c, b, CHUNK);
    }
    return c;
}

__device__ inline void store_codes(uint8_t *p, int n, uint2 c, bool past)
{
    if (n >= CHUNK) {
        store_bytes<CHUNK>(p, &c, past);
    } else {
        uint8_t b[CHUNK];
        __builtin_memcpy(b, &c, CHUNK);
#pragma unroll
        for (int i = 0; i < CHUNK - 1; ++i)
            if (i < n) p[i] = b[i];
    }
}

// Packs the eight values of this lane, n of them there; its three neighbours of a quad hold the rest of the group.  All four
// lanes of a quad call it together.
__device__ inline void pack_chunk(const float (&v)[CHUNK], int n, uint8_t *codes, uint8_t *scales, int64_t row, int64_t cols, int64_t groups, int64_t col,
                                  bool past)
{
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) {
        const uint32_t m = finite_magnitude(v[i]);
        amax = m > amax ? m : amax;
    }
    // the largest of the quad: lanes (1, 0, 3, 2), then (2, 3, 0, 1)
    uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0xb1, 0xf, 0xf, false);
    amax = other > amax ? other : amax;
    other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0x4e, 0xf, 0xf, false);
    amax = other > amax ? other : amax;
    const uint32_t byte = scale_byte(amax);
    if (n > 0) {
        store_codes(codes + row * cols + col, n, encode8(v, scale_inverse(byte)), past);
        if (col % GROUP == 0) scales[row * groups + col / GROUP] = (uint8_t)byte;
    }
}

// What rounding v to bfloat16 leaves of it; nothing of what becomes an infinity or NaN.
__device__ inline float rest_of_bf16(float v)
{
    const float rest = v - (float)(__bf16)v;
    return finite_magnitude(rest) ? rest : 0.0f;
}

// 1 / (1 + exp(-g)), off by 2 units of 2^-24 of its value where g >= 0 and by up to 3 + |g| below (6 at -4, 10 at -8, 31 at -30, 66 at -87; exact
// exponential and reciprocal assumed): the product with the constant rounds, and exp(-g) is the square of exp(-g / 2).  Taking
// along what the product's rounding leaves would hold it at 5 throughout, in ten instructions instead of six; the results go to codes of 2^-4, to
// bfloat16, or to two of those, 2^-17.  A square, because an exponent that carries an offset would lose what the offset's size rounds away.  Its 2^-32nd part does not
// overflow before the result is zero, and the reciprocal of that, which the hardware forms within a unit but not as a subnormal number, is
// brought back by a product.
__device__ inline float sigmoid(float g)
{
    const float root = __builtin_amdgcn_exp2f(g * -0.72134752f);
    return __builtin_amdgcn_rcpf(__builtin_fmaf(root * 0x1p-32f, root, 0x1p-32f)) * 0x1p-32f;
}

// ---- division of 32-bit numbers by one that a launch knows ----

struct divider {
    uint32_t by, mul, shift;
    explicit divider(uint32_t d) : by(d)
    {
        shift = 0;
        while (shift < 32 && ((uint64_t)1 << shift) < d) ++shift;
        mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - d)) / d + 1);
    }
    // n < 2^31
    __device__ uint32_t operator()(uint32_t n) const { return (uint32_t)(((uint64_t)__umulhi(n, mul) + n) >> shift); }
};

// ---- host side ----

inline hipStream_t stream_of(void *s) { return (hipStream_t)s; }

inline int launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LEAP_OK : leap_hip_fail(e, "kernel launch");
}

// launch(first, blocks) over `all` blocks in as many launches as it takes: one has fewer than 2^32 threads (2^30 rows of 8 channels are 2^33).
constexpr int64_t MOST_BLOCKS = (int64_t)1 << 21;
template <class F> inline int over_blocks(int64_t all, F &&launch)
{
    for (int64_t first = 0; first < all; first += MOST_BLOCKS) {
        launch(first, (unsigned)(all - first < MOST_BLOCKS ? all - first : MOST_BLOCKS));
        const int rc = launched();
        if (rc != LEAP_OK) return rc;
    }
    return LEAP_OK;
}

inline int refuse(const char *why)
{
    try {
        leap_set_error(why);
    } catch (...) {          // no memory for the message: the status says enough
    }
    return LEAP_INVALID_ARG;
}

inline bool known_type(int32_t t) { return t == LEAP_F32 || t == LEAP_BF16 || t == LEAP_F16; }

// Sizes of an array; null if they are fine.
inline const char *bad_sizes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 1) return "rows must not be negative, columns must be positive";
    if (cols > MOST_COLS || rows > MOST_VALUES / cols) return "more than 2^20 columns or 2^42 values";
    return nullptr;
}

// Rows `stride` elements apart (0: every row is the same memory); null if fine.
inline const char *bad_stride(int64_t stride, int64_t rows, int64_t cols)
{
    if (stride < 0 || stride > MOST_VALUES || (rows > 1 && stride > 0 && stride < cols)) return "rows overlap or their stride is negative";
    if (rows > 1 && stride > ((int64_t)1 << 60) / rows) return "rows reach beyond what addresses hold";
    return nullptr;
}

// A workspace is memory from a multiple of 16 bytes on.
inline bool unaligned(const void *p) { return !p || (uintptr_t)p % 16 != 0; }
constexpr const char *NO_WORK = "the workspace needs memory from a multiple of 16 bytes on";

// f(the type as a constant) for a type known at run time.
template <class F> inline int by_type(int32_t type, F &&f)
{
    switch (type) {
    case LEAP_F32: return f(std::integral_constant<int, LEAP_F32>{});
    case LEAP_BF16: return f(std::integral_constant<int, LEAP_BF16>{});
    default: return f(std::integral_constant<int, LEAP_F16>{});
    }
}

// ---- products that other operators are made of (act_gemm.hip) ----

// Values from one row to the next where rows of bfloat16 are followed by zeros up to a multiple of 16 bytes: such rows are not laid out anew.
inline int64_t padded_row(int64_t cols) { return (cols + 7) / 8 * 8; }

// How du [rows][2 * out] lies: in bfloat16, rows `stride` apart with zeros between them; or, fine, as two such arrays side by side.
struct du_layout {
    int64_t low, stride;               // values from one of du to its rest (0: none); from row to row
    __host__ __device__ int64_t bytes(int64_t rows) const { return rows * stride * 2; }
};
inline du_layout padded_layout(int64_t out, bool fine) { return {fine ? padded_row(2 * out) : 0, padded_row(2 * out) * (fine ? 2 : 1)}; }

// leap_linear8_backward of a du that lies like that, and leap_linear_gate8_backward to one; `out`: of the weight's rows, twice the gate's.
int64_t du_backward_work(const du_layout &L, const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out);
int du_backward(const void *d_du, const du_layout &L, const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight,
                int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight, void *d_work, void *hip_stream);
int linear_gate8_backward(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next, const uint8_t *d_kept_codes,
                          const uint8_t *d_kept_scales, int64_t rows, int64_t out, void *d_du, const du_layout &L, void *d_work, void *hip_stream);

}  // namespace act
