// 4-bit weights with a scale (and an optional zero point) per group of neighbours along K: quantisation,
// dequantisation, and the skinny projection of up to EESD_MAX_ROWS token rows (sm_100a).
//
//   value(r, k) = (c(r, k) - z(r, k / g)) * s(r, k / g),   c = 0..15, z = 0..15 (8 without zero points)
//   out[m][r]   = sum_G s(r, G) * sum_{k in G} (c(r, k) - z(r, G)) * A[m][k]
//
// Storage: codes are kept in the register order of the matrix instruction that consumes them (m16n8k16: 16 weight
// rows, 16 columns).  A tile is 16 rows x 64 columns = 512 bytes, lane l's 16 bytes together (four k16 steps), so a warp's
// load of a tile is one contiguous 16-byte-per-lane read that needs no shared memory and no shuffles; tiles of a row
// block follow one another along K.  Scales (and zero points) are group-major, [group][rows padded to 16].
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <atomic>

#include "../../include/eesd.h"
#include "common.cuh"
#include "kernels.cuh"

namespace eesd {
namespace w4 {

namespace cg = cooperative_groups;

// Element (r, k) of a tile: lane (r % 8) * 4 + (k % 8) / 2, word k / 16, bits 4 * (r / 8 + 2 * (k / 8 % 2) + 4 * (k % 2)) of it.
// The pair (k, k + 1) of a fragment register sits 16 bits apart and the word's four registers 4 bits apart, so one AND
// takes a register's pair out of the word.

// ------------------------------------------------------------------------------------ quantisation
// float64 -> nearest bf16 (ties to even) without double rounding: towards zero in fp32, the lost part kept in the last bit
__device__ __forceinline__ float round_scale(double x, int scale_dtype) {
    if (scale_dtype == EESD_F32) return __double2float_rn(x);
    float f = __double2float_rz(x);
    if ((double)f != x) f = __uint_as_float(__float_as_uint(f) | 1u);
    return __bfloat162float(__float2bfloat16_rn(f));
}

// nearest integer (ties to even) to the exact quotient x / s, clamped to [lo, hi].  The rounded quotient can only be off by
// one, and only when x / s is within rounding of a half: the exact remainder (one fused multiply-add) settles it.
__device__ __forceinline__ int nearest_quotient(float x, float s, int lo, int hi) {
    float q = rintf(__fdiv_rn(x, s));
    q = fminf(fmaxf(q, (float)lo - 1.f), (float)hi + 1.f);   // (also ends a NaN or an infinite quotient; |q| <= 16, so the remainder is exact where it matters)
    const float rem = __fmaf_rn(-q, s, x), twice = rem + rem;
    if (twice > s || (twice == s && ((int)q & 1))) q += 1.f;
    else if (-twice > s || (-twice == s && ((int)q & 1))) q -= 1.f;
    return (int)fminf(fmaxf(q, (float)lo), (float)hi);
}

template <typename WT> __device__ __forceinline__ void load16(const WT *row, int k, int K, bool vec, float *v) {
    constexpr int N = Vec16<WT>::N;
    if (vec && k + 16 <= K) {
#pragma unroll
        for (int i = 0; i < 16; i += N) Vec16<WT>::load(row + k + i, v + i);
    } else {
#pragma unroll
        for (int i = 0; i < 16; i++) v[i] = k + i < K ? to_f(row[k + i]) : 0.f;
    }
}

// One warp: 16 rows x 128 columns (two tiles).  A unit is rows (g, g + 8) x one k16 step: its 32 codes are exactly four
// words of the tile.  Lane l takes step l % 8 of rows l / 8 and l / 8 + 4 (mod 8), so eight neighbouring lanes read 128 contiguous columns of a
// row, and a group's statistics are a butterfly over 2, 4 or 8 of them.
template <typename WT>
__global__ void __launch_bounds__(256) quantize_kernel(const WT *W, size_t ldw, int R, int K, int group, int scale_dtype, bool zp,
                                                       uint32_t *codes, void *scales, uint8_t *zeros, int KT, int R16, bool vec) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, step = lane & 7;
    const int pairs = (KT + 1) / 2;
    const size_t job = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (job >= (size_t)(R16 / 16) * pairs) return;
    const int rb = (int)(job / pairs), kp = (int)(job % pairs);
    const int k = kp * 128 + step * 16;
    const int lanes = group / 16;   // lanes that share a group
#pragma unroll
    for (int half = 0; half < 2; half++) {
        const int g8 = (lane >> 3) + 4 * half;
        float s[2];
        int z[2], c[2][16];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int r = rb * 16 + g8 + 8 * h;
            float v[16];
            if (r < R) {
                load16(W + (size_t)r * ldw, k, K, vec, v);
            } else {
#pragma unroll
                for (int i = 0; i < 16; i++) v[i] = 0.f;
            }
            float lo = 0.f, hi = 0.f;
            bool bad = false;
#pragma unroll
            for (int i = 0; i < 16; i++) { lo = fminf(lo, v[i]); hi = fmaxf(hi, v[i]); bad |= !(fabsf(v[i]) <= 3.402823466e38f); }
            for (int o = 1; o < lanes; o <<= 1) {
                lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
                hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
                bad |= (bool)__shfl_xor_sync(0xffffffffu, (int)bad, o);
            }
            s[h] = zp ? round_scale(((double)hi - (double)lo) / 15.0, scale_dtype) : round_scale((double)fmaxf(hi, -lo) / 7.0, scale_dtype);
            if (bad) s[h] = __uint_as_float(0x7fc00000u);   // a NaN or infinity among the weights: the whole group reads back as NaN
            const bool some = s[h] > 0.f && !bad;
            z[h] = zp ? (some ? nearest_quotient(-lo, s[h], 0, 15) : 0) : 8;
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int lowest = -z[h];
                // padding columns (and an all-zero group) hold the zero point's code: they stand for 0
                c[h][i] = some && k + i < K ? (zp ? min(max(nearest_quotient(v[i], s[h], -15, 15), lowest), 15 - z[h]) : nearest_quotient(v[i], s[h], -8, 7)) + z[h] : z[h];
            }
            if (step % lanes == 0 && k < K) {
                const size_t at = (size_t)(k / group) * R16 + r;
                if (scale_dtype == EESD_F32) ((float *)scales)[at] = s[h];
                else ((__nv_bfloat16 *)scales)[at] = __float2bfloat16_rn(s[h]);
                if (zp) zeros[at] = (uint8_t)z[h];
            }
        }
        const int kt = kp * 2 + (step >> 2);
        if (kt < KT) {
#pragma unroll
            for (int t = 0; t < 4; t++) {   // fragment columns 2t, 2t + 1 and 2t + 8, 2t + 9
                uint32_t w = 0;
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int q = 0; q < 2; q++)
#pragma unroll
                        for (int e = 0; e < 2; e++) w |= (uint32_t)c[h][q * 8 + 2 * t + e] << (4 * (h + 2 * q + 4 * e));
                codes[(((size_t)rb * KT + kt) * 32 + g8 * 4 + t) * 4 + (step & 3)] = w;
            }
        }
    }
}

template <typename OT>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint32_t *codes, const void *scales, const uint8_t *zeros, int R, int K, int group,
                                                         int scale_dtype, OT *out, size_t ldo, int KT, int R16, bool vec) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, step = lane & 7;
    const int pairs = (KT + 1) / 2;
    const size_t job = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (job >= (size_t)(R16 / 16) * pairs) return;
    const int rb = (int)(job / pairs), kp = (int)(job % pairs);
    const int k = kp * 128 + step * 16, kt = kp * 2 + (step >> 2);
    if (k >= K) return;
#pragma unroll
    for (int half = 0; half < 2; half++) {
        const int g8 = (lane >> 3) + 4 * half;
        uint32_t w[4];
#pragma unroll
        for (int t = 0; t < 4; t++) w[t] = __ldg(&codes[(((size_t)rb * KT + kt) * 32 + g8 * 4 + t) * 4 + (step & 3)]);
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int r = rb * 16 + g8 + 8 * h;
            if (r >= R) continue;
            const size_t at = (size_t)(k / group) * R16 + r;
            const float s = scale_dtype == EESD_F32 ? ((const float *)scales)[at] : to_f(((const __nv_bfloat16 *)scales)[at]);
            const int z = zeros ? zeros[at] : 8;
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; i++) v[i] = __fmul_rn((float)((int)((w[(i & 7) >> 1] >> (4 * (h + 2 * (i >> 3) + 4 * (i & 1)))) & 15u) - z), s);
            OT *o = out + (size_t)r * ldo + k;
            if (vec && k + 16 <= K) {
                if constexpr (sizeof(OT) == 4) {
#pragma unroll
                    for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4 *>(o + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                } else {
                    uint32_t p[8];
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        p[i] = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v[2 * i])) | ((uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v[2 * i + 1])) << 16);
                    *reinterpret_cast<uint4 *>(o) = make_uint4(p[0], p[1], p[2], p[3]);
                    *reinterpret_cast<uint4 *>(o + 8) = make_uint4(p[4], p[5], p[6], p[7]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (k + i < K) o[i] = from_f<OT>(v[i]);
            }
        }
    }
}

// places codes given one per byte, row-major, and [R][G] scales / zero points into the stored order
__global__ void __launch_bounds__(256) pack_kernel(const uint8_t *src, int R, int K, const void *sc, const uint8_t *zs, int scale_dtype, int group,
                                                   uint32_t *codes, void *scales, uint8_t *zeros, int KT, int R16, int G) {
    pdl_wait();
    pdl_trigger();
    const size_t words = (size_t)(R16 / 16) * KT * 128, n = (size_t)gridDim.x * blockDim.x;
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < words; i += n) {
        const int j = (int)(i & 3), lane = (int)((i >> 2) & 31);
        const size_t tile = i >> 7;
        const int rb = (int)(tile / KT), kt = (int)(tile % KT);
        uint32_t w = 0;
#pragma unroll
        for (int b = 0; b < 8; b++) {
            const int h = b & 1, q = (b >> 1) & 1, e = b >> 2;
            const int r = rb * 16 + (lane >> 2) + 8 * h, k = kt * 64 + j * 16 + (lane & 3) * 2 + 8 * q + e;
            uint32_t c = 8;
            if (r < R && k < K) c = src[(size_t)r * K + k] & 15u;
            else if (zs) c = r < R ? zs[(size_t)r * G + min(k, K - 1) / group] & 15u : 0u;   // padding stands for 0
            w |= c << (4 * b);
        }
        codes[i] = w;
    }
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < (size_t)G * R16; i += n) {
        const int r = (int)(i % R16), g = (int)(i / R16);
        const size_t at = (size_t)r * G + g;
        if (scale_dtype == EESD_F32) ((float *)scales)[i] = r < R ? ((const float *)sc)[at] : 0.f;
        else ((__nv_bfloat16 *)scales)[i] = r < R ? ((const __nv_bfloat16 *)sc)[at] : __float2bfloat16_rn(0.f);
        if (zs) zeros[i] = r < R ? zs[at] & 15u : 0;
    }
}

// ------------------------------------------------------------------------------------ projection
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t h2_sub(uint32_t a, uint32_t b) {
    __half2 r = __hsub2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
    return *reinterpret_cast<uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t h2_fma(uint32_t a, uint32_t b, uint32_t c) {
    __half2 r = __hfma2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b), *reinterpret_cast<__half2 *>(&c));
    return *reinterpret_cast<uint32_t *>(&r);
}
__device__ __forceinline__ uint4 ld_stream(const uint4 *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

struct ProjArgs {
    const uint4 *codes;
    const void *scales;
    const uint8_t *zeros;
    const void *A;
    float *out;
    size_t lda, ldo;
    int R, R16, K, KT, M, a_dtype, scale_dtype, vec;
};

constexpr int kWarps = 8;

// NT n-tiles of 8 columns; an fp32 row takes two columns (two fp16 terms), a bf16 row one.  RB row blocks of 16 per warp.
// KC: tiles (64 columns of the matrix) whose activations are staged at a time.
template <int NT, int RB> struct Shape {
    static constexpr int rows = kWarps * RB * 16;
    static constexpr int U = RB == 1 ? 4 : 2;         // tiles a warp loads ahead
    static constexpr int KC = NT == 1 ? 16 : 8;
    static constexpr int act_words = KC * 4 * NT * 64;
    static constexpr int red_ld = rows + 4;
    __host__ __device__ static constexpr size_t act_bytes() {
        const size_t act = (size_t)act_words * 4, red = (size_t)(NT == 1 ? 8 : EESD_MAX_ROWS) * red_ld * 4;
        return act > red ? act : red;
    }
};

__device__ __forceinline__ float4 load_a4(const ProjArgs &p, int m, int k) {
    float v[4];
    if (p.a_dtype == EESD_F32) {
        const float *a = (const float *)p.A + (size_t)m * p.lda + k;
        if (p.vec && k + 4 <= p.K) return *reinterpret_cast<const float4 *>(a);
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = k + i < p.K ? a[i] : 0.f;
    } else {
        const __nv_bfloat16 *a = (const __nv_bfloat16 *)p.A + (size_t)m * p.lda + k;
        if (p.vec && k + 4 <= p.K) {
            const uint2 w = *reinterpret_cast<const uint2 *>(a);
            return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
        }
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = k + i < p.K ? to_f(a[i]) : 0.f;
    }
    return make_float4(v[0], v[1], v[2], v[3]);
}

// The activations enter as fp16 after a power-of-two scale per token row that puts the largest staged magnitude into
// [2^14, 2^15): an fp32 row as two terms (22 bits; what is below 2^-39 of the row's largest is lost), a bf16 row as one (exact
// down to 2^-29 of it).  Fields are the biased exponents of that scale; they only ever fall, so sums already taken are brought
// along by an exact multiplication.
__device__ __forceinline__ int scale_field(uint32_t max_bits) {
    if (max_bits >= 0x7f800000u) return 127;            // an infinity or NaN: the row's results are not finite anyway
    const int f = 268 - (int)(max_bits >> 23);          // 2^(14 - exponent)
    return f < 253 ? f : 253;
}

template <int NT, int RB, int G, bool ZP>
__global__ void __launch_bounds__(kWarps * 32) project_kernel(const ProjArgs p) {
    using S = Shape<NT, RB>;
    constexpr int U = S::U, KC = S::KC, ROWS = S::rows;
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t *act = reinterpret_cast<uint32_t *>(smem);   // activations as B fragments [tile][step pair][n-tile][lane][4]; afterwards the partial results
    float *sS = reinterpret_cast<float *>(smem + S::act_bytes());   // scales of the staged groups, [group][row]
    constexpr int kGrp = KC * 64 / G + 1;
    uint8_t *sZ = reinterpret_cast<uint8_t *>(sS + kGrp * ROWS);
    __shared__ uint32_t s_max[2][EESD_MAX_ROWS];
    __shared__ int s_field[2][EESD_MAX_ROWS];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t = lane & 3;
    const int splits = (int)gridDim.y, split = (int)blockIdx.y;
    const int kt0 = (int)((long long)p.KT * split / splits), n = (int)((long long)p.KT * (split + 1) / splits) - kt0;
    const int row0 = blockIdx.x * ROWS;
    const bool two = p.a_dtype == EESD_F32;
    const int n_tok = two ? NT * 4 : NT * 8;             // token rows the n-tiles can hold

    if (tid < EESD_MAX_ROWS) { s_max[0][tid] = 0; s_field[1][tid] = 253; }
    pdl_wait();
    pdl_trigger();

    const uint4 *src[RB];
    bool live[RB];
#pragma unroll
    for (int rb = 0; rb < RB; rb++) {
        const int blk = row0 / 16 + warp * RB + rb;
        live[rb] = blk * 16 < p.R16;
        src[rb] = p.codes + ((size_t)(live[rb] ? blk : 0) * p.KT + kt0) * 32 + lane;
    }
    uint4 cur[U][RB], nxt[U][RB];
    auto fetch = [&](uint4 (&w)[U][RB], int base) {
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int rb = 0; rb < RB; rb++)
                w[u][rb] = base + u < n && live[rb] ? ld_stream(src[rb] + (size_t)(base + u) * 32) : make_uint4(0, 0, 0, 0);
    };
    fetch(cur, 0);

    float acc[RB][NT][4], gacc[RB][NT][4];
#pragma unroll
    for (int rb = 0; rb < RB; rb++)
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 4; i++) acc[rb][nt][i] = gacc[rb][nt][i] = 0.f;

    int g0 = 0;   // first staged group
    auto stage = [&](int c0) {
        const int ph = (c0 / KC) & 1;
        const int k0 = (kt0 + c0) * 64, nk = min(KC, n - c0) * 64, pieces = (nk + 127) / 128;
        __syncthreads();   // the previous stage is used up; s_max[ph] is zero
        for (int it = warp; it < p.M * pieces; it += kWarps) {
            const int m = it % p.M, k = it / p.M * 128 + lane * 4;
            uint32_t mx = 0;
            if (k < nk) {
                const float4 v = load_a4(p, m, k0 + k);
                mx = max(max(__float_as_uint(v.x) & 0x7fffffffu, __float_as_uint(v.y) & 0x7fffffffu),
                         max(__float_as_uint(v.z) & 0x7fffffffu, __float_as_uint(v.w) & 0x7fffffffu));
            }
            mx = __reduce_max_sync(0xffffffffu, mx);
            if (lane == 0) atomicMax(&s_max[ph][m], mx);
        }
        g0 = k0 / G;
        const int ng = (k0 + nk - 1) / G - g0 + 1, groups = (p.K + G - 1) / G;   // (a group past the end only meets zero activations: scale 0)
        for (int i = tid; i < ng * ROWS; i += kWarps * 32) {
            const int gr = i / ROWS, r = row0 + i % ROWS;
            const size_t at = (size_t)(g0 + gr) * p.R16 + r;
            const bool in = r < p.R16 && g0 + gr < groups;
            sS[i] = in ? (p.scale_dtype == EESD_F32 ? __ldg((const float *)p.scales + at) : to_f(__ldg((const __nv_bfloat16 *)p.scales + at))) : 0.f;
            if (ZP) sZ[i] = in ? __ldg(p.zeros + at) : 0;
        }
        __syncthreads();
        for (int it = warp; it < p.M * pieces; it += kWarps) {
            const int m = it % p.M, k = it / p.M * 128 + lane * 4;
            const int field = min(s_field[ph ^ 1][m], scale_field(s_max[ph][m]));
            if (k < nk) {
                const float4 v = load_a4(p, m, k0 + k);
                const float sc = __int_as_float(field << 23);
                const float x[4] = {v.x * sc, v.y * sc, v.z * sc, v.w * sc};
                __half hi[4], lo[4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    hi[i] = __float2half_rn(x[i]);
                    lo[i] = __float2half_rn(x[i] - __half2float(hi[i]));
                }
                const int j = (k & 63) >> 4, q = (k >> 3) & 1, tt = (k & 7) >> 1;
                auto put = [&](int col, const __half *h) {
                    uint32_t *d = act + ((((k >> 6) * 2 + (j >> 1)) * NT + (col >> 3)) * 32 + (col & 7) * 4 + tt) * 4 + (j & 1) * 2 + q;
                    __half2 a = __halves2half2(h[0], h[1]), b = __halves2half2(h[2], h[3]);
                    d[0] = *reinterpret_cast<uint32_t *>(&a);
                    d[4] = *reinterpret_cast<uint32_t *>(&b);
                };
                put(m, hi);
                if (two) put(m + n_tok, lo);
            }
        }
        if (c0) {   // bring the sums along to the new scale
            float f[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const int m = (nt * 8 + 2 * t + e) % n_tok;
                    const int old = s_field[ph ^ 1][m], d = min(old, scale_field(s_max[ph][m])) - old;
                    f[nt][e] = m >= p.M || d == 0 ? 1.f : d < -126 ? 0.f : __int_as_float((127 + d) << 23);
                }
#pragma unroll
            for (int rb = 0; rb < RB; rb++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int i = 0; i < 4; i++) acc[rb][nt][i] *= f[nt][i & 1];
        }
        if (tid < EESD_MAX_ROWS) {
            s_field[ph][tid] = min(s_field[ph ^ 1][tid], scale_field(s_max[ph][tid]));
            s_max[ph ^ 1][tid] = 0;
        }
        __syncthreads();
    };

    auto fold = [&](int gr) {   // group sums times the group's scales into the totals
#pragma unroll
        for (int rb = 0; rb < RB; rb++) {
            const float *s = sS + gr * ROWS + (warp * RB + rb) * 16 + g8;
            const float s0 = s[0], s1 = s[8];
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                acc[rb][nt][0] = fmaf(gacc[rb][nt][0], s0, acc[rb][nt][0]);
                acc[rb][nt][1] = fmaf(gacc[rb][nt][1], s0, acc[rb][nt][1]);
                acc[rb][nt][2] = fmaf(gacc[rb][nt][2], s1, acc[rb][nt][2]);
                acc[rb][nt][3] = fmaf(gacc[rb][nt][3], s1, acc[rb][nt][3]);
                gacc[rb][nt][0] = gacc[rb][nt][1] = gacc[rb][nt][2] = gacc[rb][nt][3] = 0.f;
            }
        }
    };

    for (int base = 0; base < n; base += U) {
        fetch(nxt, base + U);
        if (base % KC == 0) stage(base);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int c = base + u;
            if (c < n) {
                const int k0 = (kt0 + c) * 64;
                const uint4 *bp = reinterpret_cast<const uint4 *>(act) + (size_t)(c % KC) * 2 * NT * 32 + lane;
                uint32_t z0[RB], z1[RB];
#pragma unroll
                for (int jp = 0; jp < 2; jp++) {
                    const int gr = (k0 + jp * 32) / G - g0;
                    if (jp == 0 || G == 32) {
#pragma unroll
                        for (int rb = 0; rb < RB; rb++) {
                            // 1024 + z and -(64 + z) as fp16 pairs, by their bit patterns
                            if (ZP) {
                                const uint8_t *z = sZ + gr * ROWS + (warp * RB + rb) * 16 + g8;
                                z0[rb] = 0x64006400u + (uint32_t)z[0] * 0x00010001u;
                                z1[rb] = 0xD400D400u + (uint32_t)z[8] * 0x00100010u;
                            } else {
                                z0[rb] = 0x64086408u;
                                z1[rb] = 0xD480D480u;
                            }
                        }
                    }
                    uint4 b[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) b[nt] = bp[(jp * NT + nt) * 32];
#pragma unroll
                    for (int jj = 0; jj < 2; jj++) {
#pragma unroll
                        for (int rb = 0; rb < RB; rb++) {
                            const uint4 v = cur[u][rb];
                            const uint32_t w = jp == 0 ? (jj == 0 ? v.x : v.y) : (jj == 0 ? v.z : v.w), w8 = w >> 8;
                            uint32_t a[4];
                            a[0] = h2_sub((w & 0x000f000fu) | 0x64006400u, z0[rb]);               // 1024 + c - (1024 + z)
                            a[1] = h2_fma((w & 0x00f000f0u) | 0x64006400u, 0x2c002c00u, z1[rb]);   // (1024 + 16 c) / 16 - (64 + z)
                            a[2] = h2_sub((w8 & 0x000f000fu) | 0x64006400u, z0[rb]);
                            a[3] = h2_fma((w8 & 0x00f000f0u) | 0x64006400u, 0x2c002c00u, z1[rb]);
#pragma unroll
                            for (int nt = 0; nt < NT; nt++) mma_16816(gacc[rb][nt], a, jj == 0 ? b[nt].x : b[nt].z, jj == 0 ? b[nt].y : b[nt].w);
                        }
                    }
                    if (G == 32) fold(gr);
                    else if (jp == 1 && (G == 64 || ((kt0 + c) & 1) || c == n - 1 || c % KC == KC - 1)) fold(gr);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int rb = 0; rb < RB; rb++) cur[u][rb] = nxt[u][rb];
    }

    // partial results [token][row] into shared memory: the two terms joined, the power of two taken out
    const int last = n > 0 ? ((n - 1) / KC) & 1 : 1;
    __syncthreads();
    float *red = reinterpret_cast<float *>(act);
#pragma unroll
    for (int rb = 0; rb < RB; rb++) {
        const int r = (warp * RB + rb) * 16 + g8;
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                float v = acc[rb][nt][i];
                const int col = nt * 8 + 2 * t + (i & 1);
                if (two) {
                    if constexpr (NT == 1) v += __shfl_xor_sync(0xffffffffu, v, 2);   // columns c and c + 4
                    else if (nt < NT / 2) v += acc[rb][nt + NT / 2][i];
                }
                if (col < n_tok && col < p.M) red[col * S::red_ld + r + (i >> 1) * 8] = v * __int_as_float((254 - s_field[last][col]) << 23);
            }
    }
    const int total = p.M * ROWS;
    if (splits == 1) {
        __syncthreads();
        for (int i = tid; i < total; i += kWarps * 32) {
            const int m = i / ROWS, r = i % ROWS;
            if (row0 + r < p.R) p.out[(size_t)m * p.ldo + row0 + r] = red[m * S::red_ld + r];
        }
        return;
    }
    // the slices of K are one cluster: every block adds its share of the rows over all of them, in slice order
    cg::cluster_group cl = cg::this_cluster();
    cl.sync();
    for (int i = split * kWarps * 32 + tid; i < total; i += splits * kWarps * 32) {
        const int m = i / ROWS, r = i % ROWS;
        float v = 0.f;
        for (int s = 0; s < splits; s++) v += cl.map_shared_rank(red, s)[m * S::red_ld + r];
        if (row0 + r < p.R) p.out[(size_t)m * p.ldo + row0 + r] = v;
    }
    cl.sync();   // nobody leaves while its partial results are still being read
}

template <int NT, int RB, int G, bool ZP>
cudaError_t launch_project(cudaStream_t s, const ProjArgs &p, int splits) {
    using S = Shape<NT, RB>;
    const size_t n_grp = (size_t)S::KC * 64 / G + 1;
    const size_t smem = S::act_bytes() + n_grp * S::rows * 4 + (ZP ? n_grp * S::rows : 0);
    auto kernel = project_kernel<NT, RB, G, ZP>;
    if (smem > 40 * 1024) {   // more than a kernel gets unasked: once per device
        static std::atomic<uint64_t> done{0};
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev > 63 || !(done.load(std::memory_order_acquire) >> dev & 1)) {
            e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e != cudaSuccess) return e;
            if (dev <= 63) done.fetch_or(1ull << dev, std::memory_order_release);
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((p.R16 + S::rows - 1) / S::rows, splits);
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int na = 0;
    if (splits > 1) {
        attr[na].id = cudaLaunchAttributeClusterDimension;
        attr[na].val.clusterDim.x = 1;
        attr[na].val.clusterDim.y = splits;
        attr[na].val.clusterDim.z = 1;
        na++;
    }
    if (pdl_enabled()) {
        attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[na].val.programmaticStreamSerializationAllowed = 1;
        na++;
    }
    cfg.attrs = attr;
    cfg.numAttrs = na;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <int NT, int RB>
cudaError_t launch_group(cudaStream_t s, const ProjArgs &p, int group, int splits) {
    const bool zp = p.zeros != nullptr;
    switch (group) {
        case 32: return zp ? launch_project<NT, RB, 32, true>(s, p, splits) : launch_project<NT, RB, 32, false>(s, p, splits);
        case 64: return zp ? launch_project<NT, RB, 64, true>(s, p, splits) : launch_project<NT, RB, 64, false>(s, p, splits);
        default: return zp ? launch_project<NT, RB, 128, true>(s, p, splits) : launch_project<NT, RB, 128, false>(s, p, splits);
    }
}

// slices of K: as many as keep about four blocks per multiprocessor, at most 8 (a cluster) and at least two tiles each
inline int pick_splits(int row_tiles, int KT) {
    int s = 1;
    while (s < 8 && row_tiles * s * 2 <= 4 * 148 && KT >= 4 * s) s *= 2;
    return s;
}

}  // namespace w4

namespace {
inline size_t up(size_t v, size_t a) { return (v + a - 1) / a * a; }

int w4_check(const eesd_w4 *m) {
    if (!m || m->R < 1 || m->K < 1 || m->R > (1 << 28) || m->K > (1 << 28)) return EESD_ERR_BADARG;
    if (m->group != 32 && m->group != 64 && m->group != 128) return EESD_ERR_UNSUPPORTED;
    if (m->scale_dtype != EESD_F32 && m->scale_dtype != EESD_BF16) return EESD_ERR_BADARG;
    if (m->zero_point != 0 && m->zero_point != 1) return EESD_ERR_BADARG;
    return EESD_OK;
}
int w4_open(const eesd_w4 *m, const void *packed, size_t bytes, eesd_w4_layout *l) {
    const int st = eesd_w4_layout_of(m, l);
    if (st) return st;
    if (!packed || ((uintptr_t)packed & 15)) return EESD_ERR_BADARG;
    if (bytes < l->total_bytes) return EESD_ERR_NOMEM;
    return EESD_OK;
}
// warps' jobs of the quantisation kernels, eight to a block
bool w4_grid(const eesd_w4_layout &l, unsigned int *blocks) {
    const size_t jobs = (size_t)l.row_blocks * ((l.k_tiles + 1) / 2), b = (jobs + 7) / 8;
    if (b > 0x7fffffffu) return false;
    *blocks = (unsigned int)b;
    return true;
}
}  // namespace
}  // namespace eesd

using namespace eesd;

extern "C" {

int eesd_w4_layout_of(const eesd_w4 *m, eesd_w4_layout *out) {
    const int st = w4_check(m);
    if (st) return st;
    if (!out) return EESD_ERR_BADARG;
    out->row_blocks = (m->R + 15) / 16;
    out->k_tiles = (m->K + 63) / 64;
    out->groups = (m->K + m->group - 1) / m->group;
    const size_t r16 = (size_t)out->row_blocks * 16;
    out->codes = 0;
    out->scales = up((size_t)out->row_blocks * out->k_tiles * 512, 256);
    out->zeros = up(out->scales + r16 * out->groups * (m->scale_dtype == EESD_F32 ? 4 : 2), 256);
    out->total_bytes = up(out->zeros + (m->zero_point ? r16 * out->groups : 0), 256);
    return EESD_OK;
}

int eesd_w4_quantize(void *cuda_stream, const eesd_w4 *m, int w_dtype, const void *W, int64_t ldw, void *packed, size_t packed_bytes) {
    eesd_w4_layout l;
    const int st = w4_open(m, packed, packed_bytes, &l);
    if (st) return st;
    if (!W || (w_dtype != EESD_F32 && w_dtype != EESD_BF16) || ldw < m->K) return EESD_ERR_BADARG;
    unsigned int blocks;
    if (!w4_grid(l, &blocks)) return EESD_ERR_UNSUPPORTED;
    const size_t es = w_dtype == EESD_F32 ? 4 : 2;
    if ((uintptr_t)W % es) return EESD_ERR_BADARG;
    const bool vec = ((uintptr_t)W & 15) == 0 && (size_t)ldw * es % 16 == 0;
    char *p = (char *)packed;
    uint8_t *z = m->zero_point ? (uint8_t *)(p + l.zeros) : nullptr;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (w_dtype == EESD_F32)
        launch_k(w4::quantize_kernel<float>, dim3(blocks), dim3(256), 0, s, pdl_enabled(), (const float *)W, (size_t)ldw, m->R, m->K, m->group, m->scale_dtype,
                 m->zero_point != 0, (uint32_t *)p, (void *)(p + l.scales), z, l.k_tiles, l.row_blocks * 16, vec);
    else
        launch_k(w4::quantize_kernel<__nv_bfloat16>, dim3(blocks), dim3(256), 0, s, pdl_enabled(), (const __nv_bfloat16 *)W, (size_t)ldw, m->R, m->K, m->group,
                 m->scale_dtype, m->zero_point != 0, (uint32_t *)p, (void *)(p + l.scales), z, l.k_tiles, l.row_blocks * 16, vec);
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

int eesd_w4_dequantize(void *cuda_stream, const eesd_w4 *m, const void *packed, size_t packed_bytes, int out_dtype, void *out, int64_t ldo) {
    eesd_w4_layout l;
    const int st = w4_open(m, packed, packed_bytes, &l);
    if (st) return st;
    if (!out || (out_dtype != EESD_F32 && out_dtype != EESD_BF16) || ldo < m->K) return EESD_ERR_BADARG;
    unsigned int blocks;
    if (!w4_grid(l, &blocks)) return EESD_ERR_UNSUPPORTED;
    const size_t es = out_dtype == EESD_F32 ? 4 : 2;
    if ((uintptr_t)out % es) return EESD_ERR_BADARG;
    const bool vec = ((uintptr_t)out & 15) == 0 && (size_t)ldo * es % 16 == 0;
    const char *p = (const char *)packed;
    const uint8_t *z = m->zero_point ? (const uint8_t *)(p + l.zeros) : nullptr;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (out_dtype == EESD_F32)
        launch_k(w4::dequantize_kernel<float>, dim3(blocks), dim3(256), 0, s, pdl_enabled(), (const uint32_t *)p, (const void *)(p + l.scales), z, m->R, m->K,
                 m->group, m->scale_dtype, (float *)out, (size_t)ldo, l.k_tiles, l.row_blocks * 16, vec);
    else
        launch_k(w4::dequantize_kernel<__nv_bfloat16>, dim3(blocks), dim3(256), 0, s, pdl_enabled(), (const uint32_t *)p, (const void *)(p + l.scales), z, m->R,
                 m->K, m->group, m->scale_dtype, (__nv_bfloat16 *)out, (size_t)ldo, l.k_tiles, l.row_blocks * 16, vec);
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

int eesd_w4_pack(void *cuda_stream, const eesd_w4 *m, const uint8_t *codes, const void *scales, const uint8_t *zeros, void *packed, size_t packed_bytes) {
    eesd_w4_layout l;
    const int st = w4_open(m, packed, packed_bytes, &l);
    if (st) return st;
    if (!codes || !scales || (zeros != nullptr) != (m->zero_point != 0)) return EESD_ERR_BADARG;
    if ((uintptr_t)scales % (m->scale_dtype == EESD_F32 ? 4 : 2)) return EESD_ERR_BADARG;
    char *p = (char *)packed;
    const size_t words = (size_t)l.row_blocks * l.k_tiles * 128, want = (words + 255) / 256;
    const unsigned int blocks = (unsigned int)(want < 148 * 64 ? want : 148 * 64);
    launch_k(w4::pack_kernel, dim3(blocks), dim3(256), 0, (cudaStream_t)cuda_stream, pdl_enabled(), codes, m->R, m->K, scales, zeros, m->scale_dtype, m->group,
             (uint32_t *)p, (void *)(p + l.scales), m->zero_point ? (uint8_t *)(p + l.zeros) : (uint8_t *)nullptr, l.k_tiles, l.row_blocks * 16, l.groups);
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

int eesd_w4_project_rows(void *cuda_stream, const eesd_w4 *m, const void *packed, size_t packed_bytes, int a_dtype, const void *A, int64_t lda,
                         float *out, int64_t ldo, int M) {
    eesd_w4_layout l;
    const int st = w4_open(m, packed, packed_bytes, &l);
    if (st) return st;
    if (!A || !out || M < 1 || M > EESD_MAX_ROWS || lda < m->K || ldo < m->R) return EESD_ERR_BADARG;
    if (a_dtype != EESD_F32 && a_dtype != EESD_BF16) return EESD_ERR_BADARG;
    const size_t es = a_dtype == EESD_F32 ? 4 : 2;
    if ((uintptr_t)A % es || ((uintptr_t)out & 3)) return EESD_ERR_BADARG;
    const char *b = (const char *)packed;
    w4::ProjArgs p;
    p.codes = (const uint4 *)(b + l.codes);
    p.scales = b + l.scales;
    p.zeros = m->zero_point ? (const uint8_t *)(b + l.zeros) : nullptr;
    p.A = A;
    p.out = out;
    p.lda = (size_t)lda;
    p.ldo = (size_t)ldo;
    p.R = m->R;
    p.R16 = l.row_blocks * 16;
    p.K = m->K;
    p.KT = l.k_tiles;
    p.M = M;
    p.a_dtype = a_dtype;
    p.scale_dtype = m->scale_dtype;
    p.vec = ((uintptr_t)A % (4 * es)) == 0 && lda % 4 == 0;
    const int cols = a_dtype == EESD_F32 ? 2 * M : M;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    cudaError_t e;
    if (cols <= 8) e = w4::launch_group<1, 1>(s, p, m->group, w4::pick_splits((p.R16 + 127) / 128, p.KT));
    else if (cols <= 16) e = w4::launch_group<2, 1>(s, p, m->group, w4::pick_splits((p.R16 + 127) / 128, p.KT));
    else e = w4::launch_group<4, 2>(s, p, m->group, w4::pick_splits((p.R16 + 255) / 256, p.KT));
    if (e != cudaSuccess) return EESD_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

}  // extern "C"
