// 4-bit weights with a scale (and an optional zero point) per group of neighbours along K: quantisation,
// dequantisation, and the skinny projection of up to EESD_MAX_ROWS token rows (sm_100a).
//
//   value(r, k) = (c(r, k) - z(r, k / g)) * s(r, k / g),   c = 0..15, z = 0..15 (8 without zero points)
//   out[m][r]   = sum_G s(r, G) * sum_{k in G} (c(r, k) - z(r, G)) * A[m][k]
//
// Storage: blocks of 16 rows x 128 columns, the blocks of a row block one after the other along K, so that a warp streams
// contiguous memory.  A block holds its codes near the register order of the matrix instruction that consumes them (m16n8k16 on fp16: 16
// weight rows, 16 columns; two tiles of 64 columns, lane l's 16 bytes of a tile together), then its groups' scales, then their zero
// points, both [row % 8][row / 8][group]: what a lane needs of them lies together.  Element (r, k) of a tile: lane (r % 8) * 4 + (k %
// 16) / 4, word k / 16, bits 8 * (k % 4) + 4 * (r / 8) of it: a word is a lane's share of one instruction's 16 x 16 codes, the low
// nibbles of row r % 8, the high ones of row r % 8 + 8.
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <atomic>

#include "../../include/eesd.h"
#include "common.cuh"
#include "kernels.cuh"

namespace eesd {
namespace w4 {

namespace cg = cooperative_groups;

struct Geom {   // where things are in a block
    int group, scale_dtype, zp, R, K, KB, block_bytes, off_zeros;
};

__device__ __forceinline__ int scale_slot(int r, int g, int per_row) { return ((r & 7) * 2 + ((r >> 3) & 1)) * per_row + g; }   // per_row: 128 / group
__device__ __forceinline__ float load_scale(const unsigned char *blk, const Geom &q, int slot) {
    return q.scale_dtype == EESD_F32 ? reinterpret_cast<const float *>(blk + 1024)[slot] : to_f(reinterpret_cast<const __nv_bfloat16 *>(blk + 1024)[slot]);
}
__device__ __forceinline__ void store_scale(unsigned char *blk, const Geom &q, int slot, float s) {
    if (q.scale_dtype == EESD_F32) reinterpret_cast<float *>(blk + 1024)[slot] = s;
    else reinterpret_cast<__nv_bfloat16 *>(blk + 1024)[slot] = __float2bfloat16_rn(s);
}

// ------------------------------------------------------------------------------------ quantisation
// The quotient's nearest value of the scale's type (ties to even).  For bf16 it is rounded once: towards zero in fp32 with what is lost
// kept in the last bit, then to nearest.
__device__ __forceinline__ float round_scale(float x, float by, int scale_dtype) {
    if (scale_dtype == EESD_F32) return __fdiv_rn(x, by);
    float f = __fdiv_rz(x, by);
    if (__fmaf_rn(-f, by, x) != 0.f) f = __uint_as_float(__float_as_uint(f) | 1u);
    return __bfloat162float(__float2bfloat16_rn(f));
}
// (hi - lo) / 15 with hi >= 0 >= lo, likewise.  The difference may take more than the 53 bits of a double and its quotient more again: both
// remainders are exact, and they tell the side where the rounded quotient lies on the border between two scales (the true one lies on
// the same side of a border as the rounded one, or that is the border itself, since rounding keeps order and a border times 15 is a double).
__device__ __forceinline__ float round_range(float hi, float lo, int scale_dtype) {
    const double a = fmax((double)hi, -(double)lo), b = fmin((double)hi, -(double)lo);
    const double sum = a + b, lost = b - (sum - a);
    const double q = sum / 15.0, rest = fma(-q, 15.0, sum) + lost;
    const uint32_t step = scale_dtype == EESD_F32 ? 1u : 0x10000u;
    const uint32_t below = __float_as_uint(__double2float_rz(q)) & ~(step - 1u);   // the scale at or below q
    const double at = __uint_as_float(below), next = __uint_as_float(below + step);
    double side = q - (at + next) * 0.5;
    if (side == 0.0) side = rest;
    return __uint_as_float(side > 0.0 || (side == 0.0 && (below & step)) ? below + step : below);
}

// nearest integer (ties to even) to the exact quotient x / s.  The rounded quotient can only be off by one, and only when x / s
// is within rounding of a half: the exact remainder (one fused multiply-add) settles it.
__device__ __forceinline__ float nearest_quotient(float x, float s) {
    float q = rintf(__fdiv_rn(x, s));
    q = fminf(fmaxf(q, -17.f), 17.f);
    const float rem = __fmaf_rn(-q, s, x), twice = rem + rem;
    if (twice > s || (twice == s && ((int)q & 1))) q += 1.f;
    else if (-twice > s || (-twice == s && ((int)q & 1))) q -= 1.f;
    return q;
}

// Both kernels give a warp one block, a lane the same four neighbouring columns of all its 16 rows (lane l: columns 4 l .. 4 l + 3), so
// that a row is one contiguous access; the lane's codes of rows g and g + 8 are one word of the block: word (l / 4) % 4 of
// fragment lane 4 g + l % 4 in tile l / 16.
__device__ __forceinline__ int word_at(int lane, int g) { return (lane >> 4) * 512 + (g * 4 + (lane & 3)) * 16 + ((lane >> 2) & 3) * 4; }

// four neighbouring weights as they come from memory
template <typename WT> struct Four;
template <> struct Four<float> {
    float4 v;
    __device__ __forceinline__ void load(const float *p) { v = __ldcs(reinterpret_cast<const float4 *>(p)); }
    __device__ __forceinline__ void set(float4 x) { v = x; }
    __device__ __forceinline__ float4 get() const { return v; }
};
template <> struct Four<__nv_bfloat16> {
    uint2 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = __ldcs(reinterpret_cast<const uint2 *>(p)); }
    __device__ __forceinline__ void set(float4 x) {   // (exact: the values are bf16)
        v.x = __float_as_uint(x.x) >> 16 | (__float_as_uint(x.y) & 0xffff0000u);
        v.y = __float_as_uint(x.z) >> 16 | (__float_as_uint(x.w) & 0xffff0000u);
    }
    __device__ __forceinline__ float4 get() const {
        return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
    }
};
template <typename WT> __device__ __forceinline__ float4 load4(const WT *p, int left) {   // the first `left` of four, the others 0
    return make_float4(left > 0 ? to_f(p[0]) : 0.f, left > 1 ? to_f(p[1]) : 0.f, left > 2 ? to_f(p[2]) : 0.f, left > 3 ? to_f(p[3]) : 0.f);
}
__device__ __forceinline__ float min_nan(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// The extreme of each of 16 rows over a group's 8, 16 or 32 lanes, the rows halved among the lanes at each exchange: afterwards a lane
// holds row first_row(lane) and, for 8 lanes, the eighth after it (lane bit 3 tells the two apart otherwise). 
// fp32: 15 exchanges, not 80; bf16: rows g and g + 8 share a register, 8 exchanges for 16 lanes.
__device__ __forceinline__ int first_row(int lane) { return (lane & 1) * 4 + (lane & 2) + (lane >> 2 & 1); }
enum Extreme { kMost, kLeast, kMagnitude };
template <Extreme E> __device__ __forceinline__ uint32_t extreme2(uint32_t a, uint32_t b) {   // of bf16 pairs; NaN wins; the sign of a magnitude means nothing
    uint32_t r;
    if (E == kMost) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else if (E == kLeast) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <Extreme E> __device__ __forceinline__ float extreme(float a, float b) {
    return E == kMost ? max_nan(a, b) : E == kLeast ? min_nan(a, b) : max_nan(fabsf(a), fabsf(b));
}
template <int G, Extreme E> __device__ __forceinline__ void row_extremes(const Four<__nv_bfloat16> (&v)[16], int lane, float (&out)[2]) {
    uint32_t m[8];
#pragma unroll
    for (int g = 0; g < 8; g++) {
        const uint32_t a = extreme2<E>(v[g].v.x, v[g].v.y), b = extreme2<E>(v[g + 8].v.x, v[g + 8].v.y);
        m[g] = extreme2<E>(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
    }
#pragma unroll
    for (int b = 0; b < 3; b++) {
        const bool up = lane >> b & 1;
#pragma unroll
        for (int i = 0; i < 4 >> b; i++) {
            const uint32_t send = up ? m[i] : m[i + (4 >> b)], keep = up ? m[i + (4 >> b)] : m[i];
            m[i] = extreme2<E>(keep, __shfl_xor_sync(0xffffffffu, send, 1 << b));
        }
    }
    if (G >= 64) m[0] = extreme2<E>(m[0], __shfl_xor_sync(0xffffffffu, m[0], 8));
    if (G == 128) m[0] = extreme2<E>(m[0], __shfl_xor_sync(0xffffffffu, m[0], 16));
    out[0] = __uint_as_float(m[0] << 16);
    out[1] = __uint_as_float(m[0] & 0xffff0000u);
    if (G >= 64 && (lane & 8)) out[0] = out[1];
    if (E == kMagnitude) out[0] = fabsf(out[0]), out[1] = fabsf(out[1]);
}
template <int G, Extreme E> __device__ __forceinline__ void row_extremes(const Four<float> (&v)[16], int lane, float (&out)[2]) {
    float m[16];
#pragma unroll
    for (int r = 0; r < 16; r++) m[r] = extreme<E>(extreme<E>(v[r].v.x, v[r].v.y), extreme<E>(v[r].v.z, v[r].v.w));
#pragma unroll
    for (int b = 0; b < 3; b++) {
        const bool up = lane >> b & 1;
#pragma unroll
        for (int h = 0; h < 16; h += 8)
#pragma unroll
            for (int i = 0; i < 4 >> b; i++) {
                const float send = up ? m[h + i] : m[h + i + (4 >> b)], keep = up ? m[h + i + (4 >> b)] : m[h + i];
                m[h + i] = extreme<E>(keep, __shfl_xor_sync(0xffffffffu, send, 1 << b));
            }
    }
    out[0] = m[0];
    out[1] = m[8];
    if (G >= 64) {
        const bool up = lane & 8;
        const float send = up ? out[0] : out[1], keep = up ? out[1] : out[0];
        out[0] = extreme<E>(keep, __shfl_xor_sync(0xffffffffu, send, 8));
    }
    if (G == 128) out[0] = extreme<E>(out[0], __shfl_xor_sync(0xffffffffu, out[0], 16));
}

// Reads a weight once, writes half a byte.  The product with 1 / s, rounded to an integer, is the quotient's nearest or its neighbour
// across a half: the exact remainder (one fused multiply-add) tells, and a row where some remainder reaches half a scale is put
// right (common only as ties: bf16 weights over bf16 scales, 3 us of the 37).  Scales below 2^-100, whose reciprocal would not
// do, are left to nearest_quotient at the end.
// Measured, 5120 x 13824: fp32 weights 45 to 56 us (floor 48.5: bound by memory, with zero points by issue), bf16 weights 34 to 52 us
// (floor 27: bound by issue, 14 instructions for a lane's weight, 3.1 of 4 a cycle with 4 blocks a multiprocessor, although most of these kernels
// spill a few registers then; 3 blocks 40 us, 4 blocks 37, with groups of 128 and bf16 scales).  Columns 16 to a lane (one lane a scale, no exchange) reads in
// pieces of 32 bytes and took 167 to 184 us.
template <typename WT, int G, bool ZP>
__global__ void __launch_bounds__(256, sizeof(WT) == 2 ? 4 : 2) quantize_kernel(const WT *W, size_t ldw, unsigned char *packed, const Geom q, size_t jobs, bool vec) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const size_t job = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (job >= jobs) return;
    const int rb = (int)(job / q.KB), k = (int)(job % q.KB) * 128 + lane * 4;
    unsigned char *blk = packed + job * q.block_bytes;
    const WT *src = W + (size_t)rb * 16 * ldw + k;
    const bool whole = vec && k + 4 <= q.K;
    const int last = q.R - 1 - rb * 16;   // (rows that do not exist: the last one's address, zeros)
    Four<WT> v[16];
    if (whole && last >= 15) {   // (decided once, so that all 16 loads are in flight together)
        const WT *at = src;
#pragma unroll
        for (int r = 0; r < 16; r++, at += ldw) v[r].load(at);
    } else {
#pragma unroll
        for (int r = 0; r < 16; r++) v[r].set(load4(src + (size_t)min(r, last) * ldw, r <= last ? q.K - k : 0));
    }
    // what a row's codes take: {s, 1 / s, 1.5 * 2^23 + z, -}, worked out by one lane a row and group
    constexpr int NG = 128 / G, N = G == 32 ? 2 : 1;
    __shared__ float4 table[8][NG][17];
    float4 (*rows)[17] = table[threadIdx.x >> 5];
    float hi[2], lo[2] = {0.f, 0.f};
    if (ZP) {
        row_extremes<G, kMost>(v, lane, hi);
        row_extremes<G, kLeast>(v, lane, lo);
    } else {
        row_extremes<G, kMagnitude>(v, lane, hi);
    }
    bool left = false;   // rows left to the end
#pragma unroll
    for (int i = 0; i < N; i++) {
        if (ZP) {
            hi[i] = max_nan(hi[i], 0.f);
            lo[i] = min_nan(lo[i], 0.f);
        }
        float s = ZP ? round_range(hi[i], lo[i], q.scale_dtype) : round_scale(hi[i], 7.f, q.scale_dtype);
        // a NaN or infinity among the weights: the whole group reads back as NaN
        if (!(hi[i] <= 3.402823466e38f) || (ZP && !(lo[i] >= -3.402823466e38f))) s = __uint_as_float(0x7fc00000u);
        const bool fine = s >= 0x1p-100f;
        const int z = ZP ? (s > 0.f ? (int)fminf(nearest_quotient(-lo[i], s), 15.f) : 0) : 8, r = first_row(lane) + (N == 2 ? 8 * i : lane & 8), g = lane / (G / 4);
        left = left || (s > 0.f && !fine);
        if (G != 128 || lane < 16) {
            rows[g][r] = make_float4(s == 0.f ? 1.f : s, fine ? __frcp_rn(s) : 0.f, 12582912.f + (float)z, 0.f);
            const int slot = scale_slot(r, g, NG);
            store_scale(blk, q, slot, s);
            if (ZP) blk[q.off_zeros + slot] = (unsigned char)z;
        }
    }
    __syncwarp();
    const float4 *mine = rows[lane / (G / 4)];
    constexpr int kTogether = sizeof(WT) == 4 ? 2 : 1;   // rows that one branch decides for (bf16, whose ties are common, 2: 43 us instead of 40)
#pragma unroll
    for (int g = 0; g < 8; g++) {
        uint32_t c[2];
#pragma unroll
        for (int h0 = 0; h0 < 2; h0 += kTogether) {
            float y[kTogether][4], rem[kTogether][4], sr[kTogether], zf[kTogether];
            bool off = false;
#pragma unroll
            for (int h = 0; h < kTogether; h++) {
                const int r = g + 8 * (h0 + h);
                float ir;
                zf[h] = 12582920.f;
                if (ZP) {
                    const float4 e = mine[r];
                    sr[h] = e.x, ir = e.y, zf[h] = e.z;
                } else {
                    const float2 e = *reinterpret_cast<const float2 *>(&mine[r]);
                    sr[h] = e.x, ir = e.y;
                }
                const float4 x4 = v[r].get();
                const float x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    y[h][j] = __fmaf_rn(x[j], ir, zf[h]);   // 1.5 * 2^23 + the code
                    rem[h][j] = __fmaf_rn(zf[h] - y[h][j], sr[h], x[j]);
                }
                const float most = fmaxf(fmaxf(fabsf(rem[h][0]), fabsf(rem[h][1])), fmaxf(fabsf(rem[h][2]), fabsf(rem[h][3])));
                off |= most + most >= sr[h];
            }
            if (off) {
#pragma unroll
                for (int h = 0; h < kTogether; h++)
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const float twice = fabsf(rem[h][j] + rem[h][j]);
                        if (twice > sr[h] || (twice == sr[h] && ((__float_as_int(y[h][j]) ^ __float_as_int(zf[h])) & 1))) y[h][j] += copysignf(1.f, rem[h][j]);
                    }
            }
#pragma unroll
            for (int h = 0; h < kTogether; h++) {
                uint32_t &q4 = c[h0 + h];
                q4 = __byte_perm(__byte_perm(__float_as_uint(y[h][0]), __float_as_uint(y[h][1]), 0x0040), __byte_perm(__float_as_uint(y[h][2]), __float_as_uint(y[h][3]), 0x0040), 0x5410);
                if (ZP) q4 -= q4 >> 4 & 0x01010101u;   // 16 becomes 15
            }
        }
        *reinterpret_cast<uint32_t *>(blk + word_at(lane, g)) = (c[0] & 0x0f0f0f0fu) | (c[1] << 4 & 0xf0f0f0f0u);
    }
    if (!__any_sync(0xffffffffu, left)) return;
    for (int r = 0; r < 16; r++) {
        const float sr = mine[r].x;
        if (!(sr < 0x1p-100f)) continue;
        const float4 x4 = load4(src + (size_t)r * ldw, q.K - k);   // (a row that does not exist is never here: its scale is 0)
        const float x[4] = {x4.x, x4.y, x4.z, x4.w}, zr = mine[r].z - 12582912.f;
        uint32_t c = 0;
#pragma unroll
        for (int j = 0; j < 4; j++) c |= (uint32_t)(int)(fminf(fmaxf(nearest_quotient(x[j], sr), ZP ? -zr : -8.f), ZP ? 15.f - zr : 7.f) + zr) << (8 * j);
        uint32_t *w = reinterpret_cast<uint32_t *>(blk + word_at(lane, r & 7));
        const int sh = r & 8 ? 4 : 0;
        *w = (*w & ~(0x0f0f0f0fu << sh)) | c << sh;
    }
}

// Reads half a byte a weight, writes it whole: bound by memory.  Measured, 5120 x 13824 to fp32: 52 to 55 us (floor 48.5); 1025 x 1000: 3.4.
template <typename OT, int G>
__global__ void __launch_bounds__(256) dequantize_kernel(const unsigned char *packed, OT *out, size_t ldo, const Geom q, size_t jobs, bool vec) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const size_t job = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (job >= jobs) return;
    const int rb = (int)(job / q.KB), k = (int)(job % q.KB) * 128 + lane * 4;
    const unsigned char *blk = packed + job * q.block_bytes;
    if (k >= q.K) return;
    uint32_t w[8];
#pragma unroll
    for (int g = 0; g < 8; g++) w[g] = __ldcs(reinterpret_cast<const uint32_t *>(blk + word_at(lane, g)));
#pragma unroll
    for (int r = 0; r < 16; r++) {
        if (rb * 16 + r >= q.R) continue;
        const int slot = scale_slot(r, lane / (G / 4), 128 / G);
        const float s = load_scale(blk, q, slot), z = 8388608.f + (q.zp ? (float)blk[q.off_zeros + slot] : 8.f);
        const uint32_t c = w[r & 7] >> (r & 8 ? 4 : 0) & 0x0f0f0f0fu;
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; j++) v[j] = __fmul_rn(__uint_as_float(__byte_perm(c, 0x4b000000u, 0x7650 + j)) - z, s);   // 2^23 + c - (2^23 + z)
        OT *o = out + (size_t)(rb * 16 + r) * ldo + k;
        if (vec && k + 4 <= q.K) {
            if constexpr (sizeof(OT) == 4) {
                *reinterpret_cast<float4 *>(o) = make_float4(v[0], v[1], v[2], v[3]);
            } else {
                const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
                *reinterpret_cast<uint2 *>(o) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (k + j < q.K) o[j] = from_f<OT>(v[j]);
        }
    }
}

template <typename WT>
void launch_quantize(cudaStream_t s, unsigned int blocks, const WT *W, size_t ldw, unsigned char *packed, const Geom &q, size_t jobs, bool vec) {
    auto k = q.zp ? (q.group == 32 ? quantize_kernel<WT, 32, true> : q.group == 64 ? quantize_kernel<WT, 64, true> : quantize_kernel<WT, 128, true>)
                  : (q.group == 32 ? quantize_kernel<WT, 32, false> : q.group == 64 ? quantize_kernel<WT, 64, false> : quantize_kernel<WT, 128, false>);
    launch_k(k, dim3(blocks), dim3(256), 0, s, pdl_enabled(), W, ldw, packed, q, jobs, vec);
}
template <typename OT>
void launch_dequantize(cudaStream_t s, unsigned int blocks, const unsigned char *packed, OT *out, size_t ldo, const Geom &q, size_t jobs, bool vec) {
    auto k = q.group == 32 ? dequantize_kernel<OT, 32> : q.group == 64 ? dequantize_kernel<OT, 64> : dequantize_kernel<OT, 128>;
    launch_k(k, dim3(blocks), dim3(256), 0, s, pdl_enabled(), packed, out, ldo, q, jobs, vec);
}

// places codes given one per byte, row-major, and [R][G] scales / zero points into blocks (one warp: one block)
__global__ void __launch_bounds__(256) pack_kernel(const uint8_t *src, const void *sc, const uint8_t *zs, unsigned char *packed, const Geom q, size_t jobs) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const size_t job = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (job >= jobs) return;
    const int rb = (int)(job / q.KB), k0 = (int)(job % q.KB) * 128, G = (q.K + q.group - 1) / q.group;
    unsigned char *blk = packed + job * q.block_bytes;
#pragma unroll 1
    for (int i = 0; i < 8; i++) {
        const int tile = i >> 2, j = i & 3;
        uint32_t w = 0;
#pragma unroll
        for (int b = 0; b < 8; b++) {
            const int r = rb * 16 + (lane >> 2) + 8 * (b & 1), k = k0 + tile * 64 + j * 16 + (lane & 3) * 4 + (b >> 1);
            uint32_t c = 8;   // padding stands for 0
            if (r < q.R && k < q.K) c = src[(size_t)r * q.K + k] & 15u;
            else if (zs) c = r < q.R ? zs[(size_t)r * G + min(k / q.group, G - 1)] & 15u : 0u;
            w |= c << (4 * b);
        }
        *reinterpret_cast<uint32_t *>(blk + tile * 512 + lane * 16 + j * 4) = w;
    }
    const int n = 128 / q.group;
    for (int i = lane; i < n * 16; i += 32) {
        const int r = rb * 16 + (i & 15), g = k0 / q.group + (i >> 4), slot = scale_slot(i & 15, i >> 4, n);
        const bool in = r < q.R && g < G;
        const size_t at = (size_t)r * G + g;
        store_scale(blk, q, slot, !in ? 0.f : q.scale_dtype == EESD_F32 ? ((const float *)sc)[at] : to_f(((const __nv_bfloat16 *)sc)[at]));
        // (a padded group's codes are those of the last real one: so is its zero point)
        if (zs) blk[q.off_zeros + slot] = r < q.R ? zs[(size_t)r * G + min(g, G - 1)] & 15u : 0;
    }
}

// the reverse; what is null is left out
__global__ void __launch_bounds__(256) unpack_kernel(const unsigned char *packed, uint8_t *dst, void *sc, uint8_t *zs, const Geom q, size_t jobs) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const size_t job = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (job >= jobs) return;
    const int rb = (int)(job / q.KB), k0 = (int)(job % q.KB) * 128, G = (q.K + q.group - 1) / q.group;
    const unsigned char *blk = packed + job * q.block_bytes;
    if (dst) {
        const int k = k0 + lane * 4;
#pragma unroll
        for (int g = 0; g < 8; g++) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(blk + word_at(lane, g));
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int r = rb * 16 + g + 8 * h;
                const uint32_t c = w >> (4 * h) & 0x0f0f0f0fu;
                uint8_t *o = dst + (size_t)r * q.K + k;
                if (r < q.R && k + 4 <= q.K && ((uintptr_t)o & 3) == 0) *reinterpret_cast<uint32_t *>(o) = c;
                else if (r < q.R)
                    for (int j = 0; j < 4 && k + j < q.K; j++) o[j] = (uint8_t)(c >> (8 * j));
            }
        }
    }
    const int n = 128 / q.group;
    for (int i = lane; i < n * 16; i += 32) {
        const int r = rb * 16 + i / n, g = k0 / q.group + i % n, slot = scale_slot(i / n, i % n, n);
        if (r >= q.R || g >= G) continue;
        const size_t at = (size_t)r * G + g;
        if (sc) {
            if (q.scale_dtype == EESD_F32) ((float *)sc)[at] = reinterpret_cast<const float *>(blk + 1024)[slot];
            else ((__nv_bfloat16 *)sc)[at] = reinterpret_cast<const __nv_bfloat16 *>(blk + 1024)[slot];
        }
        if (zs) zs[at] = blk[q.off_zeros + slot];
    }
}

// ------------------------------------------------------------------------------------ projection
// A block of threads (one per multiprocessor, kWarps warps) owns a run of row blocks and a slice of K; the slices of a
// run are one cluster.  Its (row block, 128 columns) units are cut evenly among its warps, chunk by chunk of the columns whose
// activations fit with 16 rows, so the load is even to a unit whatever the shape and however few chunks are staged at a time; a
// warp's first and last row block may be shared with its neighbours and are added up at the end.  Weights go straight into registers,
// kAhead units ahead.  Where a warp's units lie is written down once for a stage (`segs`): worked out between the units, with the ring of loads
// unrolled, it cost 8 to 15 % (instructions seldom run, each copy fetched anew).
//
// The products are fp16 with fp32 sums: a code enters as 32 (c - z), exactly (the nibble set into the mantissa of 1024, or of 1024 + 16 c
// for a high one, and one fused multiply-add that takes the zero point off), an activation as two fp16 terms of 11 bits, hi and 2048 lo,
// after a power of two for each token row and 128 columns has put the largest magnitude there into [2^14, 2^15).  Each term is a column of
// the matrix instruction, so the two have sums of their own, joined at the end of a group; each activation keeps its own
// exponent, so a large one takes nothing from its neighbours: an activation of at least 2^-27 of the largest is off by 2^-23 of itself,
// a smaller one by 2^-50 of the largest, and one whose code stands for 0 adds nothing.  fp32 begins with the sums: hi terms of like size add
// up exactly (11 bits and a code's 4), the tensor core cuts off below 2^-23 of the running sum, the scale of a group comes after.
// Signed 8-bit digits of fixed-point numbers (integer products, exact sums, a third of the expanding operations) were faster at 16 rows but held an
// activation to 2^-23 or 2^-31 of the largest of its 128 columns, whatever its own size.
//
// Measured (a graph of calls, matrices that pass the L2 cache in turn; floor: bytes at the measured copy rate):
//   15360 x 5120, groups of 128:               M = 1 13.3 us, 4 14.6, 8 17.1, 16 23.4 (floor 6.2)
//   27648 x 5120, groups of 64, zero points:   M = 1 20.3, 4 21.3, 8 25.5, 16 38.6 (floor 11.7)
//   8192 x 28672, groups of 128, zero points:  M = 1 30.5 (4.0 TB/s), 4 32.9, 8 40.6, 16 63.5 (floor 18.6)
constexpr int kWarps = 16;
// Units a warp's loads run ahead.  Few rows need the bytes in flight (8192 x 28672, M = 1: 2, 3, 4, 5 units 32.2, 30.7, 30.4, 30.1 us; 5 are slower on short
// matrices); with more the products leave time, and the registers are worth more (27648 x 5120, M = 8: 1, 2, 3 units 26.2, 25.4, 25.6; 15360 x
// 5120, M = 16: 1, 2, 3 units 23.4, 23.8, 24.5).
template <int TOK> constexpr int kAhead = TOK == 16 ? 1 : TOK == 8 ? 2 : 4;
constexpr int kMaxRun = 32;     // row blocks of a run
constexpr int kSmem = 227 * 1024;
// A kernel is for up to TOK token rows (1, 2, 4, 8, 16): tiles of the matrix instruction, and columns of a tile that are kept (term j of a
// tile's row i is its column 2 i + j, so a lane's two results of a weight row are one token row's; 1 and 2 rows fill the tile by repetition)
__host__ __device__ constexpr int tiles(int TOK) { return TOK <= 4 ? 1 : TOK / 4; }
__host__ __device__ constexpr int columns(int TOK) { return TOK <= 4 ? 2 * TOK : 8; }
// Staged activations of 128 columns: fragments [step pair][tile][column][lane % 4][4 words], then the rows' unscales.
__host__ __device__ constexpr int frag_size(int TOK) { return 256 * tiles(TOK) * columns(TOK); }
__host__ __device__ constexpr int act_bytes(int TOK) { return frag_size(TOK) + (TOK < 2 ? 16 : TOK * 8); }

struct ProjArgs {
    const unsigned char *packed;
    const void *A;
    const unsigned char *frag;   // staged form of A (stage_kernel); null: every block of threads stages for itself
    float *out;
    size_t lda, ldo;
    int R, K, KB, RB, M, a_dtype, vec, chunk, stage;   // KB, RB: blocks along K, row blocks; chunk: blocks along K of a chunk; stage: chunks staged at a time
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

// A warp turns 128 columns of token row m (lane: columns 4 * lane .. + 3) into two fp16 terms each at dst.  The scale 2^f puts the largest
// magnitude into [2^14, 2^15), so that no sum overflows and 28 binary orders below it are normal numbers; f stops at 126 (2^-f stays normal).
// A group's sum is unscaled by 2^-f, of which at most 2^20 before it meets its scale (the sum is below 2^31, so nothing overflows there that stays
// in range as a result) and the rest, 1 or more, after.
template <int TOK>
__device__ __forceinline__ void stage_piece(unsigned char *dst, float4 v, int m) {
    const int lane = threadIdx.x & 31;
    const uint32_t mx = __reduce_max_sync(0xffffffffu, max(max(__float_as_uint(v.x) & 0x7fffffffu, __float_as_uint(v.y) & 0x7fffffffu),
                                                           max(__float_as_uint(v.z) & 0x7fffffffu, __float_as_uint(v.w) & 0x7fffffffu)));
    const bool bad = mx >= 0x7f800000u;   // a NaN or infinity: the row's results are NaN
    const int f = min(14 + 127 - (int)(mx >> 23), 126);
    const float sc = __int_as_float((127 + f) << 23);
    const float x[4] = {v.x, v.y, v.z, v.w};
    __half hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float y = bad ? 0.f : x[i] * sc;
        hi[i] = __float2half_rn(y);
        lo[i] = __float2half_rn((y - __half2float(hi[i])) * 2048.f);
    }
    // operand words: columns 0 and 2, columns 1 and 3 of the lane's four (the order that codes expand in)
    auto two = [](__half a, __half b) { return (uint32_t)__half_as_ushort(a) | (uint32_t)__half_as_ushort(b) << 16; };
    const int step = lane >> 2, t = lane & 3;
    uint2 *act = reinterpret_cast<uint2 *>(dst) + (((step >> 1) * tiles(TOK) + (m >> 2)) * columns(TOK) * 4 + (m & 3) * 8 + t) * 2 + (step & 1);
    act[0] = make_uint2(two(hi[0], hi[2]), two(hi[1], hi[3]));
    act[8] = make_uint2(two(lo[0], lo[2]), two(lo[1], lo[3]));
    if (lane == 0) {   // (codes enter 32-fold)
        const int f1 = max(f, -25);
        const float u1 = (bad ? __uint_as_float(0x7fc00000u) : __int_as_float((127 - f1) << 23)) * 0.03125f;
        reinterpret_cast<float2 *>(dst + frag_size(TOK))[m] = make_float2(u1, __int_as_float((127 + f1 - f) << 23));
    }
}

// the same for a whole matrix, into global memory (many token rows: staging once costs less than once per block of threads)
template <int TOK>
__global__ void __launch_bounds__(256) stage_kernel(const ProjArgs p, unsigned char *frag) {
    pdl_wait();      // everything before this launch is complete once the trigger fires: the projection may read the matrix before its own wait
    pdl_trigger();
    const int lane = threadIdx.x & 31, job = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (job >= p.KB * p.M) return;
    const int m = job / p.KB, kb = job % p.KB;
    stage_piece<TOK>(frag + (size_t)kb * act_bytes(TOK), load_a4(p, m, kb * 128 + lane * 4), m);
}

// 32 (c - z) of two codes as fp16: the nibbles of x that MASK names, set into the mantissa of 1024, times 2 or 32 and less the zero point's
// part, exactly (with mask and 1024 both known the compiler would take two operations for the first)
template <uint32_t MASK> __device__ __forceinline__ uint32_t expand(uint32_t x, uint32_t ones, uint32_t less) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(x), "n"(MASK), "r"(ones));   // (a & b) | c
    asm("fma.rn.f16x2 %0, %0, %1, %2;" : "+r"(r) : "r"(MASK == 0x000f000fu ? 0x50005000u : 0x40004000u), "r"(less));
    return r;
}
// fp16 products onto c
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float (&c)[4]) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ void copy16(uint32_t dst, const unsigned char *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// N bytes (2 to 32) of a matrix that is read once
template <int N> struct Bytes { uint32_t v[(N + 3) / 4]; };
template <int N> __device__ __forceinline__ void load_once(Bytes<N> &d, const unsigned char *p) {
    if constexpr (N == 2) asm volatile("{.reg .b16 t; ld.global.L1::no_allocate.b16 t, [%1]; cvt.u32.u16 %0, t;}" : "=r"(d.v[0]) : "l"(p));
    if constexpr (N == 4) asm volatile("ld.global.L1::no_allocate.b32 %0, [%1];" : "=r"(d.v[0]) : "l"(p));
    if constexpr (N == 8) asm volatile("ld.global.L1::no_allocate.v2.b32 {%0,%1}, [%2];" : "=r"(d.v[0]), "=r"(d.v[1]) : "l"(p));
    if constexpr (N >= 16)
#pragma unroll
        for (int i = 0; i < N / 16; i++)
            asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(d.v[4 * i]), "=r"(d.v[4 * i + 1]), "=r"(d.v[4 * i + 2]), "=r"(d.v[4 * i + 3]) : "l"(p + 16 * i));
}

// shared memory: activations of `stage` chunks | the warps' segments of them | partial results of shared row blocks | results
__host__ __device__ constexpr int segments(int stage) { return 2 * stage + kMaxRun / kWarps + 1; }   // a warp's: two shared row blocks by chunks, whole ones, the end
struct Smem { int segs, slots, outs, total; };
__host__ __device__ inline Smem carve(int TOK, int M, int stage, int chunk, int run) {
    Smem s;
    s.segs = stage * chunk * act_bytes(TOK);
    s.slots = s.segs + kWarps * segments(stage) * 16;
    s.outs = s.slots + kWarps * 2 * M * 64;
    s.total = s.outs + run * M * 64;
    return s;
}

// first unit of warp w
__device__ __forceinline__ int unit_of(int units, int w) { return (int)(((long long)units * w) / kWarps); }

template <int TOK, int G, bool ZP, bool F32S>
__global__ void __launch_bounds__(kWarps * 32, 1) project_kernel(const ProjArgs p) {
    constexpr int NG = 128 / G, kScaleBytes = 2 * NG * (F32S ? 4 : 2), kZeros = 1024 + 8 * kScaleBytes, kRecord = kZeros + (ZP ? NG * 16 : 0), U = kAhead<TOK>;
    constexpr int kAct = act_bytes(TOK), NT = tiles(TOK), COLS = columns(TOK);
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t = lane & 3;
    const int splits = (int)gridDim.y, split = (int)blockIdx.y, runs = (int)gridDim.x;
    const int rb0 = (int)((long long)p.RB * blockIdx.x / runs), run = (int)((long long)p.RB * (blockIdx.x + 1) / runs) - rb0;
    const int kb0 = (int)((long long)p.KB * split / splits), kbn = (int)((long long)p.KB * (split + 1) / splits) - kb0;
    const Smem sm = carve(TOK, p.M, p.stage, p.chunk, 0);
    unsigned char *act = smem;
    float *slots = reinterpret_cast<float *>(smem + sm.slots), *outs = reinterpret_cast<float *>(smem + sm.outs);

    if (!p.frag) pdl_wait();   // (with staged activations the launch before this one is their kernel, and the matrix is complete already)
    pdl_trigger();

    // The warp's row blocks: a part of `head`, if it begins inside of it, the whole ones from `first` on, a part of `last`.  Their units go one
    // after the other, those of a shared row block chunk by chunk (the warp's share is the same part of every chunk).
    const int head = run * warp / kWarps, first = (run * warp + kWarps - 1) / kWarps, last = run * (warp + 1) / kWarps;
    const bool shares_last = run * (warp + 1) % kWarps != 0 && last >= first;
    int4 *segs = reinterpret_cast<int4 *>(smem + sm.segs) + warp * segments(p.stage);
    for (int i = tid * 4; i < kWarps * 2 * p.M * 16; i += kWarps * 128) *reinterpret_cast<float4 *>(slots + i) = make_float4(0.f, 0.f, 0.f, 0.f);
    const int chunks = (kbn + p.chunk - 1) / p.chunk;
    for (int c0 = 0; c0 < chunks; c0 += p.stage) {
        const int c1 = min(c0 + p.stage, chunks), k0 = c0 * p.chunk, staged = min(kbn, c1 * p.chunk) - k0;
        // Segments: runs of units in storage order, {first, from the first staged of row block 0; its block of 128 columns; units; where in
        // shared memory the row block's sums go on: in the results where the warp has all of it, else in the warp's slot for its first or last row block}
        {
            const int nc = c1 - c0, nh = first != head ? nc : 0, nw = max(last - first, 0), total = nh + nw + (shares_last ? nc : 0);
            int n = 0;
            for (int j0 = 0; j0 < total; j0 += 32) {
                const int j = j0 + lane, rb = j < nh ? head : min(first + j - nh, last);
                const bool whole = j >= nh && j < nh + nw;
                const int c = j < nh ? j : j - nh - nw;   // (of a shared one)
                int k = 0, units = staged;
                if (!whole) {
                    const int cn = min(p.chunk, kbn - (c0 + c) * p.chunk), lo = max(unit_of(run * cn, warp) - rb * cn, 0);
                    units = min(unit_of(run * cn, warp + 1) - rb * cn, cn) - lo;
                    k = c * p.chunk + lo;
                }
                const bool any = j < total && units > 0;
                const uint32_t those = __ballot_sync(0xffffffffu, any);
                if (any) segs[n + __popc(those & ((1u << lane) - 1))] = make_int4(rb * p.KB + k, k, units, (whole ? sm.outs / 4 + rb * p.M * 16 : sm.slots / 4 + (warp * 2 + (rb != head)) * p.M * 16));
                n += __popc(those);
            }
            if (lane == 0) segs[n] = make_int4(0, 0, 0, 0);
            __syncwarp();
        }
        struct Unit {
            Bytes<16> w[2];
            Bytes<kScaleBytes> s;
            Bytes<2 * NG> z;
        } ring[U];
        // loads ahead
        const unsigned char *base = p.packed + ((size_t)rb0 * p.KB + kb0 + k0) * kRecord, *src;
        const int4 *fnext = segs;
        int fleft;
        auto follow = [&]() {
            const int4 e = *fnext++;
            src = base + (size_t)e.x * kRecord;
            fleft = e.z;
        };
        follow();
        auto fetch = [&](Unit &r) {
            if (fleft > 0) {
                load_once(r.w[0], src + lane * 16);
                load_once(r.w[1], src + 512 + lane * 16);
                load_once(r.s, src + 1024 + g8 * kScaleBytes);
                if (ZP) load_once(r.z, src + kZeros + g8 * 2 * NG);
            }
            src += kRecord;
            if (--fleft == 0) follow();   // (after the last segment it goes on below 0)
        };
#pragma unroll
        for (int s = 0; s < U; s++) fetch(ring[s]);

        if (c0) __syncthreads();   // the activations staged before are used up
        if (p.frag) {
            if (!c0) pdl_wait();
            const unsigned char *from = p.frag + (size_t)(kb0 + k0) * kAct;
            const uint32_t at = (uint32_t)__cvta_generic_to_shared(act);
            for (int i = tid * 16; i < staged * kAct; i += kWarps * 512) copy16(at + i, from + i);
            asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
        } else {
            constexpr int kBatch = 4;
            for (int it0 = warp; it0 < p.M * staged; it0 += kWarps * kBatch) {
                float4 v[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; i++) {
                    const int it = it0 + i * kWarps, m = it / staged, k = (kb0 + k0 + it - m * staged) * 128 + lane * 4;
                    v[i] = it < p.M * staged ? load_a4(p, m, k) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
#pragma unroll
                for (int i = 0; i < kBatch; i++) {
                    const int it = it0 + i * kWarps, m = it / staged;
                    if (it < p.M * staged) stage_piece<TOK>(act + (it - m * staged) * kAct, v[i], m);
                }
            }
        }
        __syncthreads();

        float acc[NT][2];   // token row 4 n + t, weight rows g8 and g8 + 8
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
        uint32_t ones;
        asm volatile("mov.b32 %0, 0x64006400;" : "=r"(ones));
        float *sums = reinterpret_cast<float *>(smem) + t * 16 + g8;
        auto resume = [&](int d) {
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int i = 0; i < 2; i++) acc[n][i] = c0 && n * 4 + t < p.M ? sums[d + n * 64 + i * 8] : 0.f;
        };
        const int4 *next = segs;
        int4 e = *next;
        resume(e.w);
        int left = e.z;
        const unsigned char *bp = act + e.y * kAct;
        while (left) {
#pragma unroll
            for (int slot = 0; slot < U; slot++) {
                if (!left) break;
                Unit &r = ring[slot];
                float g[NT][4];
                float2 un[NT];
#pragma unroll
                for (int n = 0; n < NT; n++) un[n] = reinterpret_cast<const float2 *>(bp + frag_size(TOK))[n * 4 + t % (TOK < 4 ? TOK : 4)];
#pragma unroll
                for (int jp = 0; jp < 4; jp++) {   // 32 columns: two steps
                    uint4 b[NT];
#pragma unroll
                    for (int n = 0; n < NT; n++) b[n] = *reinterpret_cast<const uint4 *>(bp + (jp * NT + n) * COLS * 64 + (COLS == 8 ? lane : lane % (4 * COLS)) * 16);
                    const int gr = jp * 32 / G;
                    uint32_t less0 = 0xf800f800u + 8u * 0x00010001u, less1 = 0xe800e800u + 8u * 0x00100010u;   // -32 (1024 + z), -2 (1024 + 16 z)
                    if (ZP) {   // bytes gr and NG + gr
                        less0 = 0xf800f800u + (r.z.v[gr / 4] >> (8 * (gr % 4)) & 0xffu) * 0x00010001u;
                        less1 = 0xe800e800u + (r.z.v[(NG + gr) / 4] >> (8 * ((NG + gr) % 4)) & 0xffu) * 0x00100010u;
                    }
#pragma unroll
                    for (int jj = 0; jj < 2; jj++) {
                        const uint32_t x = r.w[jp >> 1].v[(jp & 1) * 2 + jj], x8 = x >> 8;
                        const uint32_t a[4] = {expand<0x000f000fu>(x, ones, less0), expand<0x00f000f0u>(x, ones, less1),
                                               expand<0x000f000fu>(x8, ones, less0), expand<0x00f000f0u>(x8, ones, less1)};
                        const bool first = (jp * 32 + jj * 16) % G == 0;
#pragma unroll
                        for (int n = 0; n < NT; n++) {
                            if (first) mma(g[n], a, jj == 0 ? b[n].x : b[n].z, jj == 0 ? b[n].y : b[n].w, zero);
                            else mma(g[n], a, jj == 0 ? b[n].x : b[n].z, jj == 0 ? b[n].y : b[n].w, g[n]);
                        }
                    }
                    if ((jp * 32 + 32) % G != 0) continue;
                    // the group is complete: the two terms' sums joined, unscaled, times the scale
                    float s0, s1;
                    if (F32S) {
                        s0 = __uint_as_float(r.s.v[gr]);
                        s1 = __uint_as_float(r.s.v[NG + gr]);
                    } else {   // halfwords gr and NG + gr
                        const uint32_t sa = r.s.v[gr / 2], sb = r.s.v[(NG + gr) / 2];
                        s0 = __uint_as_float(gr & 1 ? sa & 0xffff0000u : sa << 16);
                        s1 = __uint_as_float((NG + gr) & 1 ? sb & 0xffff0000u : sb << 16);
                    }
#pragma unroll
                    for (int n = 0; n < NT; n++) {
                        const float h0 = fmaf(g[n][1], 0x1p-11f, g[n][0]) * un[n].x, h1 = fmaf(g[n][3], 0x1p-11f, g[n][2]) * un[n].x;
                        acc[n][0] = fmaf(h0 * s0, un[n].y, acc[n][0]);
                        acc[n][1] = fmaf(h1 * s1, un[n].y, acc[n][1]);
                    }
                }
                fetch(r);
                bp += kAct;
                if (--left == 0) {
                    const int d = next->w;
                    e = *++next;
                    left = e.z;
                    bp = act + e.y * kAct;
                    if (e.w != d) {   // (0 at the end)
#pragma unroll
                        for (int n = 0; n < NT; n++)
#pragma unroll
                            for (int i = 0; i < 2; i++)
                                if (n * 4 + t < p.M) sums[d + n * 64 + i * 8] = acc[n][i];
                        resume(e.w);
                    }
                }
            }
        }
    }
    __syncthreads();
    // shared row blocks: the warps' parts in order
    for (int i = warp; i < run; i += kWarps) {
        int x = kWarps * i / run;                            // the last warp that begins at or before the row block
        if (kWarps * (i + 1) <= run * (x + 1)) continue;     // it has the whole: already in the results
        float v[EESD_MAX_ROWS / 2];
#pragma unroll
        for (int j = 0; j < EESD_MAX_ROWS / 2; j++) v[j] = 0.f;
        for (; x < kWarps && run * x < kWarps * (i + 1); x++) {
            const float *part = slots + (x * 2 + (i != run * x / kWarps)) * p.M * 16 + lane;
#pragma unroll
            for (int j = 0; j < EESD_MAX_ROWS / 2; j++)
                if (j * 32 + lane < p.M * 16) v[j] += part[j * 32];
        }
#pragma unroll
        for (int j = 0; j < EESD_MAX_ROWS / 2; j++)
            if (j * 32 + lane < p.M * 16) outs[i * p.M * 16 + j * 32 + lane] = v[j];
    }

    // the slices of K are one cluster: every block adds up its share of the row blocks over all of them, in slice order
    if (splits > 1) cg::this_cluster().sync();
    else __syncthreads();
    for (int i = split + warp * splits; i < run; i += kWarps * splits)
        for (int e = lane; e < p.M * 16; e += 32) {
            const int m = e >> 4, r = (rb0 + i) * 16 + (e & 15);
            float v = 0.f;
            if (splits > 1) {
                for (int s = 0; s < splits; s++) v += cg::this_cluster().map_shared_rank(outs, s)[i * p.M * 16 + e];
            } else {
                v = outs[i * p.M * 16 + e];
            }
            if (r < p.R) p.out[(size_t)m * p.ldo + r] = v;
        }
    if (splits > 1) cg::this_cluster().sync();   // nobody leaves while its results are still being read
}

// How a matrix is cut: `splits` slices of K (a cluster of 1, 2, 4 or 8 blocks), `runs` runs of row blocks (of at most `run`), chunks of `chunk`
// blocks of 128 columns.  The order of every addition follows from it, so it looks at the matrix alone: a token row has the same
// result however many rows go with it.  A chunk is what fits with 16 rows; fewer rows stage several at a time.  Forced to 1, 2, 4 or 8 slices, 12
// matrices from 1024 x 4096 to 128256 x 8192 with 1, 4 and 16 rows ran at most 5 % faster than with the choice made here (most of them
// none), and up to twice slower.
struct Cut { int splits, runs, run, chunk; };

inline int chunks_staged(int TOK, int M, const Cut &c, int KB) {
    const int slice = (KB + c.splits - 1) / c.splits, chunks = (slice + c.chunk - 1) / c.chunk;
    int most = 1;
    while (most < chunks && carve(TOK, M, most + 1, c.chunk, c.run).total <= kSmem) most++;
    const int stages = (chunks + most - 1) / most;
    return (chunks + stages - 1) / stages;
}

// The cost estimates the time of 1 row and of 16 rows together, about in microseconds: a unit of 16 x 128 codes a warp (0.5 and 1), staging 16
// rows by block and by chunk, joining a cluster.
inline Cut pick_cut(int RB, int KB) {
    Cut best = {};
    double cost = 1e300;
    for (int s = 1; s <= 8; s *= 2) {
        if (s > KB) break;
        const int clusters = s <= 2 ? 148 / s : s == 4 ? 33 : 15;   // that are resident together (what the occupancy query answers on a B200)
        const int waves = (RB + clusters * kMaxRun - 1) / (clusters * kMaxRun);
        const int runs = RB < clusters * waves ? RB : clusters * waves;
        const int run = (RB + runs - 1) / runs, slice = (KB + s - 1) / s;
        int chunk = (kSmem - carve(16, 16, 1, 0, run).total) / act_bytes(16);
        const int n_chunks = (slice + chunk - 1) / chunk;
        chunk = (slice + n_chunks - 1) / n_chunks;
        const double c = waves * (1.5 * run * slice / kWarps + 0.07 * slice + 0.6 * n_chunks + (s > 1 ? 0.8 + 0.09 * run : 0.0));
        if (c < cost) {
            cost = c;
            best = {s, runs, run, chunk};
        }
    }
    return best;
}

// Staged activations: bytes of scratch, and whether a launch of its own stages them there.  That launch costs about 0.9 us, staging in every block 0.3 us for
// 16 pieces of 128 columns: in the blocks and by a launch 1024 x 256 with 16 rows (32 pieces a block) 5.5 and 6.0 us, 15360 x 5120 with 2 rows
// (40) 13.7 and 14.3, with 4 rows (80) 15.1 and 14.6, 1024 x 1024 with 16 rows 8.0 and 6.5.
inline int tokens(int M) { return M <= 2 ? M : M <= 4 ? 4 : M <= 8 ? 8 : 16; }
inline size_t frag_bytes(int M, int KB) { return M * KB <= 32 ? 0 : (size_t)KB * act_bytes(tokens(M)); }
inline bool stage_first(int M, int slice) { return M * slice > 48; }   // (never where there is no scratch)

template <int TOK, int G, bool ZP, bool F32S>
cudaError_t launch_project(cudaStream_t s, ProjArgs p, unsigned char *scratch) {
    auto kernel = project_kernel<TOK, G, ZP, F32S>;
    {   // more shared memory than a kernel gets unasked: once per device
        static std::atomic<uint64_t> done{0};
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev > 63 || !(done.load(std::memory_order_acquire) >> dev & 1)) {
            e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
            if (e != cudaSuccess) return e;
            if (dev <= 63) done.fetch_or(1ull << dev, std::memory_order_release);
        }
    }
    const Cut cut = pick_cut(p.RB, p.KB);
    p.chunk = cut.chunk;
    p.stage = chunks_staged(TOK, p.M, cut, p.KB);
    p.frag = nullptr;
    if (stage_first(p.M, (p.KB + cut.splits - 1) / cut.splits)) {
        launch_k(stage_kernel<TOK>, dim3((p.KB * p.M + 7) / 8), dim3(256), 0, s, pdl_enabled(), p, scratch);
        p.frag = scratch;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(cut.runs, cut.splits);
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = carve(TOK, p.M, p.stage, p.chunk, cut.run).total;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int na = 0;
    if (cut.splits > 1) {
        attr[na].id = cudaLaunchAttributeClusterDimension;
        attr[na].val.clusterDim.x = 1;
        attr[na].val.clusterDim.y = cut.splits;
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

template <int TOK, int G>
cudaError_t launch_kind(cudaStream_t s, const ProjArgs &p, bool zp, bool f32s, unsigned char *scratch) {
    if (zp) return f32s ? launch_project<TOK, G, true, true>(s, p, scratch) : launch_project<TOK, G, true, false>(s, p, scratch);
    return f32s ? launch_project<TOK, G, false, true>(s, p, scratch) : launch_project<TOK, G, false, false>(s, p, scratch);
}
template <int TOK>
cudaError_t launch_group(cudaStream_t s, const ProjArgs &p, int group, bool zp, bool f32s, unsigned char *scratch) {
    return group == 32 ? launch_kind<TOK, 32>(s, p, zp, f32s, scratch)
           : group == 64 ? launch_kind<TOK, 64>(s, p, zp, f32s, scratch)
                         : launch_kind<TOK, 128>(s, p, zp, f32s, scratch);
}

}  // namespace w4

namespace {
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
w4::Geom w4_geom(const eesd_w4 *m, const eesd_w4_layout &l) {
    w4::Geom q;
    q.group = m->group;
    q.scale_dtype = m->scale_dtype;
    q.zp = m->zero_point;
    q.R = m->R;
    q.K = m->K;
    q.KB = l.k_blocks;
    q.block_bytes = (int)l.block_bytes;
    q.off_zeros = (int)l.zeros;
    return q;
}
// blocks of storage, one warp each, eight to a thread block
bool w4_grid(const eesd_w4_layout &l, size_t *jobs, unsigned int *blocks) {
    *jobs = (size_t)l.row_blocks * l.k_blocks;
    const size_t b = (*jobs + 7) / 8;
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
    out->k_blocks = (m->K + 127) / 128;
    out->groups = (m->K + m->group - 1) / m->group;
    const size_t n = 128 / m->group * 16;
    out->scales = 1024;
    out->zeros = out->scales + n * (m->scale_dtype == EESD_F32 ? 4 : 2);
    out->block_bytes = out->zeros + (m->zero_point ? n : 0);
    out->total_bytes = (size_t)out->row_blocks * out->k_blocks * out->block_bytes;
    return EESD_OK;
}

int eesd_w4_quantize(void *cuda_stream, const eesd_w4 *m, int w_dtype, const void *W, int64_t ldw, void *packed, size_t packed_bytes) {
    eesd_w4_layout l;
    const int st = w4_open(m, packed, packed_bytes, &l);
    if (st) return st;
    if (!W || (w_dtype != EESD_F32 && w_dtype != EESD_BF16) || ldw < m->K) return EESD_ERR_BADARG;
    size_t jobs;
    unsigned int blocks;
    if (!w4_grid(l, &jobs, &blocks)) return EESD_ERR_UNSUPPORTED;
    const size_t es = w_dtype == EESD_F32 ? 4 : 2;
    if ((uintptr_t)W % es) return EESD_ERR_BADARG;
    const bool vec = ((uintptr_t)W % (4 * es)) == 0 && ldw % 4 == 0;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    const w4::Geom q = w4_geom(m, l);
    if (w_dtype == EESD_F32) w4::launch_quantize(s, blocks, (const float *)W, (size_t)ldw, (unsigned char *)packed, q, jobs, vec);
    else w4::launch_quantize(s, blocks, (const __nv_bfloat16 *)W, (size_t)ldw, (unsigned char *)packed, q, jobs, vec);
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

int eesd_w4_dequantize(void *cuda_stream, const eesd_w4 *m, const void *packed, size_t packed_bytes, int out_dtype, void *out, int64_t ldo) {
    eesd_w4_layout l;
    const int st = w4_open(m, packed, packed_bytes, &l);
    if (st) return st;
    if (!out || (out_dtype != EESD_F32 && out_dtype != EESD_BF16) || ldo < m->K) return EESD_ERR_BADARG;
    size_t jobs;
    unsigned int blocks;
    if (!w4_grid(l, &jobs, &blocks)) return EESD_ERR_UNSUPPORTED;
    const size_t es = out_dtype == EESD_F32 ? 4 : 2;
    if ((uintptr_t)out % es) return EESD_ERR_BADARG;
    const bool vec = ((uintptr_t)out % (4 * es)) == 0 && ldo % 4 == 0;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    const w4::Geom q = w4_geom(m, l);
    if (out_dtype == EESD_F32) w4::launch_dequantize(s, blocks, (const unsigned char *)packed, (float *)out, (size_t)ldo, q, jobs, vec);
    else w4::launch_dequantize(s, blocks, (const unsigned char *)packed, (__nv_bfloat16 *)out, (size_t)ldo, q, jobs, vec);
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

int eesd_w4_pack(void *cuda_stream, const eesd_w4 *m, const uint8_t *codes, const void *scales, const uint8_t *zeros, void *packed, size_t packed_bytes) {
    eesd_w4_layout l;
    const int st = w4_open(m, packed, packed_bytes, &l);
    if (st) return st;
    if (!codes || !scales || (zeros != nullptr) != (m->zero_point != 0)) return EESD_ERR_BADARG;
    if ((uintptr_t)scales % (m->scale_dtype == EESD_F32 ? 4 : 2)) return EESD_ERR_BADARG;
    size_t jobs;
    unsigned int blocks;
    if (!w4_grid(l, &jobs, &blocks)) return EESD_ERR_UNSUPPORTED;
    launch_k(w4::pack_kernel, dim3(blocks), dim3(256), 0, (cudaStream_t)cuda_stream, pdl_enabled(), codes, scales, zeros, (unsigned char *)packed, w4_geom(m, l), jobs);
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

int eesd_w4_unpack(void *cuda_stream, const eesd_w4 *m, const void *packed, size_t packed_bytes, uint8_t *codes, void *scales, uint8_t *zeros) {
    eesd_w4_layout l;
    const int st = w4_open(m, packed, packed_bytes, &l);
    if (st) return st;
    if ((!codes && !scales && !zeros) || (zeros && !m->zero_point)) return EESD_ERR_BADARG;
    if ((uintptr_t)scales % (m->scale_dtype == EESD_F32 ? 4 : 2)) return EESD_ERR_BADARG;
    size_t jobs;
    unsigned int blocks;
    if (!w4_grid(l, &jobs, &blocks)) return EESD_ERR_UNSUPPORTED;
    launch_k(w4::unpack_kernel, dim3(blocks), dim3(256), 0, (cudaStream_t)cuda_stream, pdl_enabled(), (const unsigned char *)packed, codes, scales, zeros, w4_geom(m, l), jobs);
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

size_t eesd_w4_project_scratch_bytes(const eesd_w4 *m, int M) {
    if (w4_check(m) || M < 1 || M > EESD_MAX_ROWS) return 0;
    return w4::frag_bytes(M, (m->K + 127) / 128);
}

int eesd_w4_project_rows(void *cuda_stream, const eesd_w4 *m, const void *packed, size_t packed_bytes, int a_dtype, const void *A, int64_t lda,
                         float *out, int64_t ldo, int M, void *scratch, size_t scratch_bytes) {
    eesd_w4_layout l;
    const int st = w4_open(m, packed, packed_bytes, &l);
    if (st) return st;
    if (!A || !out || M < 1 || M > EESD_MAX_ROWS || lda < m->K || ldo < m->R) return EESD_ERR_BADARG;
    if (a_dtype != EESD_F32 && a_dtype != EESD_BF16) return EESD_ERR_BADARG;
    const size_t es = a_dtype == EESD_F32 ? 4 : 2;
    if ((uintptr_t)A % es || ((uintptr_t)out & 3)) return EESD_ERR_BADARG;
    if (const size_t need = w4::frag_bytes(M, l.k_blocks)) {
        if (!scratch || ((uintptr_t)scratch & 15)) return EESD_ERR_BADARG;
        if (scratch_bytes < need) return EESD_ERR_NOMEM;
    }
    w4::ProjArgs p = {};
    p.packed = (const unsigned char *)packed;
    p.A = A;
    p.out = out;
    p.lda = (size_t)lda;
    p.ldo = (size_t)ldo;
    p.R = m->R;
    p.K = m->K;
    p.KB = l.k_blocks;
    p.RB = l.row_blocks;
    p.M = M;
    p.a_dtype = a_dtype;
    p.vec = ((uintptr_t)A % (4 * es)) == 0 && lda % 4 == 0;
    const int tok = w4::tokens(M);
    const bool zp = m->zero_point != 0, f32s = m->scale_dtype == EESD_F32;
    unsigned char *sc = (unsigned char *)scratch;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    const cudaError_t e = tok == 1   ? w4::launch_group<1>(s, p, m->group, zp, f32s, sc)
                          : tok == 2 ? w4::launch_group<2>(s, p, m->group, zp, f32s, sc)
                          : tok == 4 ? w4::launch_group<4>(s, p, m->group, zp, f32s, sc)
                          : tok == 8 ? w4::launch_group<8>(s, p, m->group, zp, f32s, sc)
                                     : w4::launch_group<16>(s, p, m->group, zp, f32s, sc);
    if (e != cudaSuccess) return EESD_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

}  // extern "C"
