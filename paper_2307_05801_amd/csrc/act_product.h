// The tiled product behind leap_linear8 and its kin: D[j][i] = sum over k of P(i, k) Q(j, k).
//
// A block owns TI x TJ of D and walks over k in steps of 64; a step's tiles of P and Q are fetched into shared memory (mostly
// straight from memory, past the registers) while the step before is multiplied: two buffers, one barrier a step.  i runs along a lane's
// registers and j across lanes, so a lane ends with runs of neighbouring i: what a row of an output, and a group of 32 that
// shares a scale, is made of.
//
// Which k a lane's eight values stand for is free as long as P and Q agree: of each 32, lane half h takes 16 h .. 16 h + 15
// in two turns of eight, so that 16 codes are one shared-memory read.
#pragma once

#include "act_common.h"

namespace act {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(3))) uint8_t lds_byte;

constexpr int STEP = 64;                   // values of k a step
constexpr uint32_t NOWHERE = 0x80000000u;  // an offset beyond every buffer: reads as zeros

// How an operand lies in memory: rows of bfloat16 along k; rows of k; codes along k; rows of k of codes.
enum { WIDE_ALONG, WIDE_ACROSS, CODES_ALONG, CODES_ACROSS };

// `rows` rows (i or j) of `depth` values of k.  Memory rows are `stride` elements apart; every one begins at a multiple of 16
// bytes and has memory up to one, zeros beyond its end.
struct operand {
    const uint8_t *data, *scales;
    int64_t stride, groups;                // groups: scale bytes of a memory row
    int64_t rows, depth;
};

// The first `bytes` from `base` on: reads beyond them give zeros.
__device__ inline u32x4 buffer(const uint8_t *base, int64_t bytes)
{
    const uint64_t at = (uint64_t)base;
    const auto uniform = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };        // it is; the compiler has to see it
    return u32x4{uniform((uint32_t)at), uniform((uint32_t)(at >> 32) & 0xffffu),
                 uniform(bytes <= 0 ? 0u : bytes < 0x7ffffff0 ? (uint32_t)bytes : 0x7ffffff0u), 0x00020000u};
}

// n in whole pieces of 16 bytes: a fetch that ends inside a word reads nothing of it.
__device__ inline int64_t whole(int64_t n, int piece) { return (n + piece - 1) / piece * piece; }

// Starts a fetch of 16 bytes a lane, from `offset` of the buffer to 16 * lane beyond `to`.  In assembly, because the compiler would
// wait for the fetch before the next read of any shared memory; it has no result but shared memory, and arrive() waits for it.  (m0
// is reserved: nothing the compiler makes of these kernels uses it.)
__device__ inline void fetch16(const u32x4 &from, uint32_t offset, lds_byte *to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"((uint32_t)(uintptr_t)to), "v"(offset), "s"(from) : "memory");
}

// A tile of T rows of an operand in shared memory, by KIND.  ALONG: T rows of 128 (codes: 64) bytes, their 16-byte pieces
// in an order that spreads 16 neighbouring rows over all banks; ACROSS: 64 rows of 2 T bytes, pieces likewise spread for the
// transposing read, which takes four of them at once.
template <int KIND, int T, int THREADS> struct tile {
    static constexpr int BYTES = KIND == CODES_ALONG ? T * STEP : T * STEP * 2;
    static constexpr int WAVES = THREADS / 64, PIECES = BYTES / 1024, EACH = PIECES / WAVES;       // 1 KiB pieces: a wave's fetch
    static_assert(PIECES % WAVES == 0, "a tile is fetched by all waves alike");

    // Starts the fetch of k0 .. k0 + 63 of rows row(0) .. ; row maps a multiple of 8 in the tile to the operand's row.
    template <class ROW> static __device__ inline void fetch(const operand &O, int64_t k0, int wave, int lane, lds_byte *to, ROW &&row)
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int piece = e * WAVES + wave;
            if constexpr (KIND == WIDE_ALONG) {
                const int64_t r = row(piece * 8), left = ((O.rows - 1 - r) * O.stride + whole(O.depth, 8) - k0) * 2;
                const int chunk = (lane % 8) ^ (lane / 16) ^ (piece % 2 * 4);
                const uint32_t offset = k0 + chunk * 8 < O.depth ? (uint32_t)(lane / 8) * (uint32_t)O.stride * 2 + chunk * 16 : NOWHERE;
                fetch16(buffer(O.data + (r * O.stride + k0) * 2, r < O.rows ? left : 0), offset, to + piece * 1024);
            } else if constexpr (KIND == CODES_ALONG) {
                const int64_t r = row(piece * 16), left = (O.rows - 1 - r) * O.stride + whole(O.depth, 16) - k0;
                const int chunk = (lane % 4) ^ (lane / 16);
                const uint32_t offset = k0 + chunk * 16 < O.depth ? (uint32_t)(lane / 4) * (uint32_t)O.stride + chunk * 16 : NOWHERE;
                fetch16(buffer(O.data + r * O.stride + k0, r < O.rows ? left : 0), offset, to + piece * 1024);
            } else if constexpr (KIND == WIDE_ACROSS) {
                constexpr int DEEP = 512 / T;                                                       // rows of k in a piece
                const int64_t k = k0 + piece * DEEP, r = row(0), left = ((O.depth - 1 - k) * O.stride + whole(O.rows, 8) - r) * 2;
                const int in = lane / (T / 8), chunk = (lane % (T / 8)) ^ ((piece * DEEP + in) % 4 * 4);
                fetch16(buffer(O.data + (k * O.stride + r) * 2, k < O.depth ? left : 0), (uint32_t)in * (uint32_t)O.stride * 2 + chunk * 16, to + piece * 1024);
            }
        }
    }

    // The eight values of turn s of 32-run `run` of the tile's rows first .. first + 31.
    static __device__ inline bf16x8 read(const lds_byte *from, int first, int run, int s, int lane)
    {
        const int half = lane / 32;
        if constexpr (KIND == WIDE_ALONG) {
            const int r = first + lane % 32, chunk = (run * 4 + half * 2 + s) ^ (r / 2 % 8);
            return *(const __attribute__((address_space(3))) bf16x8 *)(from + r * 128 + chunk * 16);
        } else {
            const int k = run * 32 + half * 16 + s * 8 + lane % 16 / 4, col = first + lane / 16 % 2 * 16 + lane % 4 * 4;
            const lds_byte *at = from + k * (T * 2) + ((col / 8) ^ (k % 4 * 4)) * 16 + col % 8 * 2;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at);
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + 4 * T * 2));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }

    // Both turns from codes along k, with their scale.
    static __device__ inline void read_codes(const lds_byte *from, int first, int run, int lane, uint32_t byte, bf16x8 (&v)[2])
    {
        const int r = first + lane % 32, chunk = (run * 2 + lane / 32) ^ (r / 4 % 4);
        const u32x4 c = *(const __attribute__((address_space(3))) u32x4 *)(from + r * 64 + chunk * 16);
        const float scale = __uint_as_float(byte << 23);
#pragma unroll
        for (int s = 0; s < 2; ++s) v[s] = widen(c[2 * s], c[2 * s + 1], scale);
    }

    // Eight codes as bfloat16; `scale` counts by its exponent alone.
    static __device__ inline bf16x8 widen(uint32_t lo, uint32_t hi, float scale)
    {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
        return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
};

// Codes across k on their way through the registers: widened between fetch and store.
template <int T, int THREADS> struct staged_codes {
    static constexpr int EACH = T * STEP / 16 / THREADS;
    u32x4 codes[EACH];
    uint32_t byte[EACH];

    __device__ inline void fetch(const operand &O, int64_t k0, int64_t row0)
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int q = e * THREADS + threadIdx.x, k = q / (T / 16);
            const int64_t r = row0 + q % (T / 16) * 16;
            codes[e] = u32x4{0, 0, 0, 0};
            byte[e] = 0;
            if (k0 + k < O.depth && r < O.rows) {
                codes[e] = *(const u32x4 *)(O.data + (k0 + k) * O.stride + r);
                byte[e] = O.scales[(k0 + k) * O.groups + r / GROUP];
            }
        }
    }

    __device__ inline void store(lds_byte *to) const
    {
        using as = tile<WIDE_ACROSS, T, THREADS>;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int q = e * THREADS + threadIdx.x, k = q / (T / 16), chunk = (q % (T / 16) * 2) ^ (k % 4 * 4);
            const float scale = __uint_as_float(byte[e] << 23);
            lds_byte *at = to + k * (T * 2) + chunk * 16;
            *(__attribute__((address_space(3))) bf16x8 *)at = as::widen(codes[e][0], codes[e][1], scale);
            *(__attribute__((address_space(3))) bf16x8 *)(at + 16) = as::widen(codes[e][2], codes[e][3], scale);
        }
    }
};

// Exchanges between lane halves so that the runs of four a lane holds of 32 neighbouring i (8 q + 4 half + 0 .. 3, q = 0 .. 3)
// become 16 neighbours: half 0 gets 0 .. 15, half 1 16 .. 31.  W words a run.
template <int W> __device__ inline void join_runs(uint32_t (&run)[4][W])
{
#pragma unroll
    for (int w = 0; w < W; ++w) {
        // the upper half of the first changes places with the lower half of the second
        const auto a = __builtin_amdgcn_permlane32_swap(run[0][w], run[2][w], false, false);
        const auto b = __builtin_amdgcn_permlane32_swap(run[1][w], run[3][w], false, false);
        run[0][w] = a[0], run[1][w] = a[1], run[2][w] = b[0], run[3][w] = b[1];
    }
}

// And back, a word a run.
__device__ inline void split_runs(uint32_t (&run)[4])
{
    const auto a = __builtin_amdgcn_permlane32_swap(run[0], run[1], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(run[2], run[3], false, false);
    run[0] = a[0], run[2] = a[1], run[1] = b[0], run[3] = b[1];
}

__device__ inline uint32_t two_bf16(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); }

// 16 neighbours of a row, `n` of them inside it, as bfloat16; v as the matrix instruction leaves it.
__device__ inline void store_wide(uint16_t *row, int64_t i, int64_t n, int half, const f32x16 &v)
{
    uint32_t w[4][2];
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q][0] = two_bf16(v[4 * q], v[4 * q + 1]), w[q][1] = two_bf16(v[4 * q + 2], v[4 * q + 3]);
    join_runs(w);
    uint16_t *at = row + i + half * 16;
    n -= half * 16;
    if (n >= 16) {
        __builtin_memcpy(at, w, 32);
    } else {
        uint16_t e[16];
        __builtin_memcpy(e, w, 32);
#pragma unroll
        for (int x = 0; x < 15; ++x)
            if (x < n) at[x] = e[x];
    }
}

__device__ inline void store_full(float *row, int64_t i, int64_t n, int half, const f32x16 &v)
{
    float *at = row + i + half * 4;
    n -= half * 4;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (n >= 8 * q + 4) {
            const float f[4] = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
            __builtin_memcpy(at + 8 * q, f, 16);
        } else {
#pragma unroll
            for (int x = 0; x < 3; ++x)
                if (8 * q + x < n) at[8 * q + x] = v[4 * q + x];
        }
    }
}

// The group of 32 that two lanes hold of a row, packed; n of its values are inside the row.
__device__ inline void pack_group(uint8_t *codes, uint8_t *scale, int64_t n, int half, const f32x16 &v)
{
    uint32_t amax = 0;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const uint32_t m = 8 * (r / 4) + 4 * half + r % 4 < n ? finite_magnitude(v[r]) : 0u;
        amax = m > amax ? m : amax;
    }
    const auto other = __builtin_amdgcn_permlane32_swap(amax, amax, false, false);
    amax = other[0] > other[1] ? other[0] : other[1];
    const uint32_t byte = scale_byte(amax);
    const float inverse = scale_inverse(byte);
    uint32_t w[4][1];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * q] * inverse, v[4 * q + 1] * inverse, 0, false);
        w[q][0] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * q + 2] * inverse, v[4 * q + 3] * inverse, lo, true);
    }
    join_runs(w);
    if (n <= 0) return;
    if (half == 0) *scale = (uint8_t)byte;
    uint8_t *at = codes + half * 16;
    n -= half * 16;
    if (n >= 16) {
        __builtin_memcpy(at, w, 16);
    } else {
        uint8_t b[16];
        __builtin_memcpy(b, w, 16);
#pragma unroll
        for (int x = 0; x < 15; ++x)
            if (x < n) at[x] = b[x];
    }
}

// The values of a packed group as the matrix instruction would leave them.
__device__ inline f32x16 unpack_group(const uint8_t *codes, uint32_t byte, int64_t n, int half)
{
    uint32_t w[4] = {};
    const uint8_t *at = codes + half * 16;
    n -= half * 16;
    if (n >= 16) {
        __builtin_memcpy(w, at, 16);
    } else {
        uint8_t b[16] = {};
#pragma unroll
        for (int x = 0; x < 15; ++x)
            if (x < n) b[x] = at[x];
        __builtin_memcpy(w, b, 16);
    }
    split_runs(w);
    const float scale = scale_value(byte);
    f32x16 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w[q], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w[q], true);
        v[4 * q] = a[0] * scale, v[4 * q + 1] = a[1] * scale, v[4 * q + 2] = b[0] * scale, v[4 * q + 3] = b[1] * scale;
    }
    return v;
}

// What becomes of D: rows of bfloat16; of float (of its part of k, `part` floats apart); gate and the other half packed, and
// their gated product; the gradient of those two from D and what is kept of them.
enum { TO_WIDE, TO_FULL, TO_GATED, TO_GATE_GRAD };

struct result {
    void *out;
    int64_t stride, part;
    int64_t columns;                       // gated: of `out`
    uint8_t *gated_codes, *gated_scales, *kept_codes, *kept_scales;
};

// WI x WJ waves share TI x TJ of D.  Blocks: `across` tiles of i, `along` of j, parts of `depth_part` values of k.
template <int PKIND, int QKIND, int TO, int TI, int TJ, int WI, int WJ>
__global__ __launch_bounds__(WI * WJ * 64) void k_product(operand P, operand Q, result R, uint32_t across, uint32_t along, int64_t depth_part)
{
    constexpr int THREADS = WI * WJ * 64, FI = TI / WI / 32, FJ = TJ / WJ / 32;
    constexpr int PWIDE = PKIND == CODES_ACROSS ? WIDE_ACROSS : PKIND;
    using ptile = tile<PWIDE, TI, THREADS>;
    using qtile = tile<QKIND, TJ, THREADS>;
    __shared__ __attribute__((aligned(1024))) uint8_t room[2][ptile::BYTES + qtile::BYTES];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    const int wi = wave % WI, wj = wave / WI;

    // neighbouring tiles to one of the eight dies, so that what they share comes from its cache: blocks go round the dies
    const uint32_t all = gridDim.x, die = blockIdx.x % 8, nth = blockIdx.x / 8, share = all / 8, more = all % 8;
    const uint32_t at = die * share + (die < more ? die : more) + nth;
    const uint32_t part = at / (across * along), in = at % (across * along);
    const int64_t i0 = (int64_t)(in % across) * (TO == TO_GATED ? TI / 2 : TI), j0 = (int64_t)(in / across) * TJ;
    const int64_t first = part * depth_part, last = first + depth_part < P.depth ? first + depth_part : P.depth;
    P.depth = Q.depth = last;

    const auto prow = [&](int r) -> int64_t {
        if constexpr (TO != TO_GATED) return i0 + r;
        // a wave's fragments: its columns of the gate, then the same ones of the other half; beyond the end there are no rows
        constexpr int SPAN = TI / WI;
        const int64_t col = i0 + r / SPAN * (SPAN / 2) + r % (SPAN / 2);
        return col >= R.columns ? P.rows : r % SPAN < SPAN / 2 ? col : R.columns + col;
    };
    const auto qrow = [&](int r) -> int64_t { return j0 + r; };

    lds_byte *const lds = (lds_byte *)&room[0][0];
    const auto ptile_at = [&](int b) { return lds + b * (ptile::BYTES + qtile::BYTES); };
    const auto qtile_at = [&](int b) { return lds + b * (ptile::BYTES + qtile::BYTES) + ptile::BYTES; };

    f32x16 acc[FI][FJ] = {};
    staged_codes<TI, THREADS> through;
    uint32_t byte[FJ][2], byte_next[FJ][2];
    const auto start = [&](int64_t k0, int b) {
        if constexpr (PKIND == CODES_ACROSS) through.fetch(P, k0, i0);
        else ptile::fetch(P, k0, wave, lane, ptile_at(b), prow);
        if constexpr (QKIND == CODES_ALONG) {
#pragma unroll
            for (int t = 0; t < FJ; ++t)
#pragma unroll
                for (int run = 0; run < 2; ++run) {
                    int64_t r = j0 + (wj * FJ + t) * 32 + lane % 32, g = k0 / GROUP + run;
                    r = r < Q.rows ? r : Q.rows - 1;
                    g = g < Q.groups ? g : Q.groups - 1;                        // its codes are zeros
                    byte_next[t][run] = Q.scales[r * Q.groups + g];
                }
        }
        qtile::fetch(Q, k0, wave, lane, qtile_at(b), qrow);
    };
    const auto arrive = [&](int b) {
        if constexpr (PKIND == CODES_ACROSS) through.store(ptile_at(b));
        if constexpr (QKIND == CODES_ALONG) {
#pragma unroll
            for (int t = 0; t < FJ; ++t) byte[t][0] = byte_next[t][0], byte[t][1] = byte_next[t][1];
        }
        __builtin_amdgcn_s_waitcnt(0x0070);          // vmcnt(0) lgkmcnt(0): what this wave fetched and stored has arrived
        __syncthreads();
    };

    if (first < last) {
        start(first, 0);
        arrive(0);
    }
    int b = 0;
    for (int64_t k0 = first; k0 < last; k0 += STEP, b ^= 1) {
        const bool more_k = k0 + STEP < last;
        if (more_k) start(k0 + STEP, b ^ 1);
#pragma unroll
        for (int run = 0; run < 2; ++run) {
            bf16x8 q[FJ][2];
#pragma unroll
            for (int t = 0; t < FJ; ++t) {
                const int r = (wj * FJ + t) * 32;
                if constexpr (QKIND == CODES_ALONG) {
                    qtile::read_codes(qtile_at(b), r, run, lane, byte[t][run], q[t]);
                } else {
                    q[t][0] = qtile::read(qtile_at(b), r, run, 0, lane);
                    q[t][1] = qtile::read(qtile_at(b), r, run, 1, lane);
                }
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                bf16x8 p[FI];
#pragma unroll
                for (int f = 0; f < FI; ++f) p[f] = ptile::read(ptile_at(b), (wi * FI + f) * 32, run, s, lane);
#pragma unroll
                for (int f = 0; f < FI; ++f)
#pragma unroll
                    for (int t = 0; t < FJ; ++t) acc[f][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p[f], q[t][s], acc[f][t], 0, 0, 0);
            }
        }
        if (more_k) arrive(b ^ 1);
    }

#pragma unroll
    for (int t = 0; t < FJ; ++t) {
        const int64_t j = j0 + (wj * FJ + t) * 32 + lane % 32;
        const bool there = j < Q.rows;
        if constexpr (TO == TO_WIDE || TO == TO_FULL) {
#pragma unroll
            for (int f = 0; f < FI; ++f) {
                const int64_t i = i0 + (wi * FI + f) * 32, n = there ? P.rows - i : 0;
                if constexpr (TO == TO_WIDE) store_wide((uint16_t *)R.out + j * R.stride, i, n, half, acc[f][t]);
                else store_full((float *)R.out + part * R.part + j * R.stride, i, n, half, acc[f][t]);
            }
        } else {
            const int64_t groups = groups_of(R.columns);
#pragma unroll
            for (int f = 0; f < (TO == TO_GATED ? FI / 2 : FI); ++f) {
                const int64_t i = i0 + (TO == TO_GATED ? wi * (FI / 2) + f : wi * FI + f) * 32, n = there ? R.columns - i : 0;
                if constexpr (TO == TO_GATED) {
                    const f32x16 g = acc[f][t], p = acc[f + FI / 2][t];
                    f32x16 a;
#pragma unroll
                    for (int x = 0; x < 16; ++x) a[x] = g[x] * sigmoid(g[x]) * p[x];
                    pack_group(R.gated_codes + j * R.columns + i, R.gated_scales + j * groups + i / GROUP, n, half, a);
                    if (R.kept_codes) {
                        pack_group(R.kept_codes + 2 * j * R.columns + i, R.kept_scales + 2 * j * groups + i / GROUP, n, half, g);
                        pack_group(R.kept_codes + (2 * j + 1) * R.columns + i, R.kept_scales + (2 * j + 1) * groups + i / GROUP, n, half, p);
                    }
                } else {
                    const uint32_t gb = n > 0 ? R.kept_scales[2 * j * groups + i / GROUP] : 0u, pb = n > 0 ? R.kept_scales[(2 * j + 1) * groups + i / GROUP] : 0u;
                    const f32x16 g = unpack_group(R.kept_codes + 2 * j * R.columns + i, gb, n, half);
                    const f32x16 p = unpack_group(R.kept_codes + (2 * j + 1) * R.columns + i, pb, n, half), d = acc[f][t];
                    f32x16 dg, dp;
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        const float s = sigmoid(g[x]);
                        dg[x] = d[x] * p[x] * s * (1.0f + g[x] * (1.0f - s));
                        dp[x] = d[x] * g[x] * s;
                    }
                    uint16_t *row = (uint16_t *)R.out + j * 2 * R.columns;
                    store_wide(row, i, n, half, dg);
                    store_wide(row + R.columns, i, n, half, dp);
                }
            }
        }
    }
}

}  // namespace act
