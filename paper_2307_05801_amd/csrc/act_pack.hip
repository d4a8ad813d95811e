// Packing to 8 bits and back: leap_pack8, leap_unpack8.
//
// A lane holds eight neighbouring values, four lanes a group, so the group's largest magnitude is two exchanges within a
// quad of lanes and every load and store is eight values wide.  Memory bounds both: 2^30 bfloat16 values packed in 550 us and unpacked in
// 500 (5.9 and 6.5 TB/s, 4.7 for a plain copy through the caches).
#include "act_common.h"

namespace {

using namespace act;

constexpr int BLOCK = 256;

// A launch covers rows row0 .. row0 + part, `per_row` chunks each (whole groups: the last may reach past the row).
struct rows_part {
    int64_t row0, cols, groups;
    uint32_t chunks;             // in this launch
    divider per_row;
    bool past;                   // outputs past the caches
};

template <int TYPE, int EACH>
__global__ __launch_bounds__(BLOCK) void k_pack(const void *__restrict__ x, int64_t stride, rows_part P, uint8_t *__restrict__ codes,
                                                uint8_t *__restrict__ scales)
{
    float v[EACH][CHUNK];
    int64_t row[EACH], col[EACH];
    int n[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const uint32_t q = (blockIdx.x * EACH + k) * (uint32_t)BLOCK + threadIdx.x;
        const uint32_t r = P.per_row(q);
        row[k] = P.row0 + r;
        col[k] = (int64_t)(q - r * P.per_row.by) * CHUNK;
        n[k] = q < P.chunks ? (int)(P.cols - col[k] < CHUNK ? P.cols - col[k] : CHUNK) : 0;
        load8<TYPE>(x, row[k] * stride + col[k], n[k], v[k]);
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k) pack_chunk(v[k], n[k], codes, scales, row[k], P.cols, P.groups, col[k], P.past);
}

// A lane writes 16 bytes, so that neighbouring lanes write whole lines: eight values of 16 bits, four of 32.  finite: infinities, which nothing but
// the type's range makes (those packed are NaN), become its largest number.
template <int TYPE, int EACH>
__global__ __launch_bounds__(BLOCK) void k_unpack(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, rows_part P,
                                                  void *__restrict__ out, bool finite)
{
    constexpr int N = 16 / sizeof(typename element<TYPE>::raw);
    uint32_t c[EACH][2] = {};
    uint32_t byte[EACH];
    int64_t at[EACH];
    int n[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const uint32_t q = (blockIdx.x * EACH + k) * (uint32_t)BLOCK + threadIdx.x;
        const uint32_t r = P.per_row(q);
        const int64_t col = (int64_t)(q - r * P.per_row.by) * N;
        at[k] = (P.row0 + r) * P.cols + col;
        n[k] = q < P.chunks ? (int)(P.cols - col < N ? P.cols - col : N) : 0;
        byte[k] = 0;
        if (n[k] > 0) {
            byte[k] = scales[(P.row0 + r) * P.groups + col / GROUP];
            if (n[k] == N) {
                __builtin_memcpy(c[k], codes + at[k], N);
            } else {
                uint8_t b[N] = {};
#pragma unroll
                for (int i = 0; i < N - 1; ++i)
                    if (i < n[k]) b[i] = codes[at[k] + i];
                __builtin_memcpy(c[k], b, N);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        float v[CHUNK];
        decode8(make_uint2(c[k][0], c[k][1]), scale_value(byte[k]), v);
        if (finite) {
            constexpr float LARGEST = element<TYPE>::LARGEST;
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = v[i] > LARGEST ? LARGEST : v[i] < -LARGEST ? -LARGEST : v[i];
        }
        typename element<TYPE>::raw *to = (typename element<TYPE>::raw *)out + at[k], raw[N];
#pragma unroll
        for (int i = 0; i < N; ++i) raw[i] = element<TYPE>::from_float(v[i]);
        if (n[k] == N) {
            store_bytes<16>(to, raw, P.past);
        } else {
#pragma unroll
            for (int i = 0; i < N - 1; ++i)
                if (i < n[k]) to[i] = raw[i];
        }
    }
}

// launch(part, blocks) over as many rows at a time as 31-bit chunk numbers hold.
template <int EACH, int N, class F> int over_rows(int64_t rows, int64_t cols, int size, F &&launch)
{
    const int64_t per_row = groups_of(cols) * (GROUP / N), most = ((int64_t)1 << 30) / per_row;
    for (int64_t row0 = 0; row0 < rows; row0 += most) {
        const int64_t part = rows - row0 < most ? rows - row0 : most;
        const rows_part P{row0, cols, groups_of(cols), (uint32_t)(part * per_row), divider((uint32_t)per_row), rows * cols * size > PAST_CACHES};
        launch(P, (P.chunks + BLOCK * EACH - 1) / (BLOCK * EACH));
        const int rc = launched();
        if (rc != LEAP_OK) return rc;
    }
    return LEAP_OK;
}

}  // namespace

extern "C" int leap_pack8(const void *d_x, int32_t type, int64_t stride, int64_t rows, int64_t cols, uint8_t *d_codes, uint8_t *d_scales,
                          void *hip_stream)
{
    if (!known_type(type)) return refuse("unknown element type");
    if (const char *why = bad_sizes(rows, cols)) return refuse(why);
    if (const char *why = bad_stride(stride, rows, cols)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_x || !d_codes || !d_scales) return refuse("null data pointer");
    return by_type(type, [&](auto t) {
        constexpr int EACH = 2;
        return over_rows<EACH, CHUNK>(rows, cols, 1, [&](const rows_part &P, uint32_t blocks) {
            hipLaunchKernelGGL((k_pack<decltype(t)::value, EACH>), dim3(blocks), dim3(BLOCK), 0, stream_of(hip_stream), d_x, stride, P, d_codes, d_scales);
        });
    });
}

namespace {

int unpack(const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, void *d_out, int32_t type, bool finite, void *hip_stream)
{
    if (!known_type(type)) return refuse("unknown element type");
    if (const char *why = bad_sizes(rows, cols)) return refuse(why);
    if (!rows) return LEAP_OK;
    if (!d_out || !d_codes || !d_scales) return refuse("null data pointer");
    return by_type(type, [&](auto t) {
        constexpr int EACH = 2, N = 16 / sizeof(typename element<decltype(t)::value>::raw);
        return over_rows<EACH, N>(rows, cols, 16 / N, [&](const rows_part &P, uint32_t blocks) {
            hipLaunchKernelGGL((k_unpack<decltype(t)::value, EACH>), dim3(blocks), dim3(BLOCK), 0, stream_of(hip_stream), d_codes, d_scales, P, d_out, finite);
        });
    });
}

}  // namespace

extern "C" int leap_unpack8(const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, void *d_out, int32_t type,
                            void *hip_stream)
{
    return unpack(d_codes, d_scales, rows, cols, d_out, type, false, hip_stream);
}

extern "C" int leap_unpack8_finite(const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, void *d_out, int32_t type,
                                   void *hip_stream)
{
    return unpack(d_codes, d_scales, rows, cols, d_out, type, true, hip_stream);
}
