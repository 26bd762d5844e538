// Attention of up to 16 rows a sequence over the 4-bit key / value cache (sm_100a).
//
//   x_p = scale * sum_G s_pG (q_G . (c - z)_pG),   out = sum_p (e_p s_pG) (c - z)_pG / sum_p e_p,   e_p = exp(x_p - max x)
//
// The integers c - z are exact in fp16, so the scales stay outside the matrix products: a key's scales multiply the groups' scores,
// a value's the softmax numerator.  One pass over the codes with a running maximum.
//
// A warp takes tiles of 16 tokens.  Scores are S^T[token][column] = K Q^T (m16n8k16, columns = (row, head) pairs that share the key head),
// outputs O^T[dimension][column] = V^T P^T, with keys and values as the 16-row operand straight from their codes in registers and
// one 8 x 8 transposition (movmatrix) between the score's accumulators and the numerators' operand.  Tiles come through a ring of asynchronous
// copies that belongs to the warp; the warps of a block meet once, at a segment's end.
//
// A segment is what one key head of one sequence has to do for up to 8 NT columns.  Two ways to share the machine:
//   clusters  the blocks of a cluster share a segment and join their parts through each other's shared memory (one launch)
//   runs      the tiles of all segments stand in a row and are dealt out evenly, whatever the sequences' lengths; a second kernel joins what was cut
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <atomic>
#include <type_traits>

#include "kernels.cuh"
#include "kv4.cuh"

namespace eesd {
namespace kv4 {

namespace cg = cooperative_groups;

constexpr int kWarps = 8, kAttnThreads = kWarps * 32;
constexpr int kStages = 4;   // tiles of a warp's ring
constexpr int kUnit = kWarps;
constexpr int kMaxGrid = 296;
constexpr int grid_of(int nt) { return nt == 1 ? kMaxGrid : kMaxGrid / 2; }   // blocks that fit the machine's 148 multiprocessors at once
constexpr int kRise = 4;     // a running maximum is let fall behind by this much (powers of two)
constexpr float kLowest = -3.402823466e38f;

struct AttnArgs {
    Cache c;
    const int32_t *n_ctx, *n_rows, *positions, *visible;
    const float *rope;
    int n_rope;
    const void *q;
    int64_t qs[3];
    void *out;
    float scale2;        // scale * log2(e)
    int B, rows, heads;  // heads: query heads of a key head
    int blocks;          // column blocks of a key head
    int share;           // blocks of a cluster (runs: 0)
    float *part;         // runs: [2 * grid][columns][D + 4]: outputs, maximum, sum
};

__device__ __forceinline__ int rows_of(const AttnArgs &a, int b) { return a.n_rows ? min(max(a.n_rows[b], 0), a.rows) : a.rows; }
// tiles that hold what some row of the sequence may see, at least 1
__device__ __forceinline__ int tiles_of(const AttnArgs &a, int b) {
    if (a.n_rows && a.n_rows[b] <= 0) return 1;
    return (int)max((int64_t)1, min((int64_t)a.c.max_pages << a.c.shift, ((int64_t)a.n_ctx[b] + 15) / 16));
}

// ---------------------------------------------------------------------------------- runs
// A cut inside a segment lies at a multiple of kUnit tiles (one a warp), and at an end where fewer than that would be left.
__device__ __forceinline__ int64_t cut_at(int64_t off, int64_t n) {
    if (off <= 0) return 0;
    if (off >= n) return n;
    const int64_t c = (off + kUnit / 2) / kUnit * kUnit;
    return c + kUnit > n ? n : c;
}
struct Plan {
    int64_t before[EESD_KV4_MAX_BATCH + 1];   // tiles of the sequences before (of one key head and column block)
};
__device__ __forceinline__ void make_plan(const AttnArgs &a, Plan &p) {
    if (threadIdx.x < 32) {
        int64_t sum = 0;
        for (int b0 = 0; b0 < a.B; b0 += 32) {
            const int b = b0 + threadIdx.x;
            int64_t v = b < a.B ? tiles_of(a, b) : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
                if ((int)threadIdx.x >= o) v += u;
            }
            if (b < a.B) p.before[b + 1] = sum + v;
            sum += __shfl_sync(0xffffffffu, v, 31);
        }
        if (threadIdx.x == 0) p.before[0] = 0;
    }
    __syncthreads();
}
struct Place {
    int b, seg;    // sequence; key head * blocks + column block
    int off, n;    // tile in the segment, of n
};
__device__ __forceinline__ Place find(const AttnArgs &a, const Plan &p, int64_t pos) {
    const int64_t per = (int64_t)a.c.Hkv * a.blocks;
    int lo = 0, hi = a.B;   // before[lo] * per <= pos < before[hi] * per
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.before[mid] * per <= pos) lo = mid; else hi = mid;
    }
    Place r;
    r.b = lo;
    r.n = (int)(p.before[lo + 1] - p.before[lo]);
    const int64_t in = pos - p.before[lo] * per;
    r.seg = (int)(in / r.n);
    r.off = (int)(in - (int64_t)r.seg * r.n);
    return r;
}
// where block i's run begins
__device__ __forceinline__ int64_t run_start(const AttnArgs &a, const Plan &p, int64_t i, int64_t grid) {
    const int64_t total = p.before[a.B] * a.c.Hkv * a.blocks, raw = total * i / grid;
    if (raw >= total) return total;
    const Place f = find(a, p, raw);
    return raw - f.off + cut_at(f.off, f.n);
}

// ---------------------------------------------------------------------------------- pieces
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // 2^e, -126..127
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// what rounding to fp16 left of the two
__device__ __forceinline__ uint32_t pack_rest(float lo, float hi, uint32_t taken) {
    const float2 t = __half22float2(*reinterpret_cast<const __half2 *>(&taken));
    return pack(lo - t.x, hi - t.y);
}
__device__ __forceinline__ uint32_t transpose(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// c - z of two codes, exactly: the low nibbles of x's bytes 0 and 2 set into the mantissa of 1024, or the high ones into that of 64, less what the zero
// point makes of it.  (The two bases in registers: with mask and base both known the compiler would take two operations for one.)
struct Pair { uint32_t low, high; };
__device__ __forceinline__ uint32_t low(uint32_t x, const Pair &base, const Pair &zero) {
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xea;\n\tadd.rn.f16x2 %0, %0, %3;" : "=&r"(r) : "r"(x), "r"(base.low), "r"(zero.low));
    return r;
}
__device__ __forceinline__ uint32_t high(uint32_t x, const Pair &base, const Pair &zero) {
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x00f000f0, %2, 0xea;\n\tadd.rn.f16x2 %0, %0, %3;" : "=&r"(r) : "r"(x), "r"(base.high), "r"(zero.high));
    return r;
}
// -(1024 + z) and -(64 + z) of two zero points: byte 0 of z twice, or bytes 0 and 1 (below 16)
template <bool SAME> __device__ __forceinline__ Pair zeros(uint32_t z) {
    constexpr uint32_t pick = SAME ? 0x4040u : 0x4140u;
    return Pair{__byte_perm(z, 0xe4u, pick), __byte_perm(z << 4, 0xd4u, pick)};
}
__device__ __forceinline__ void copy16(uint32_t dst, const unsigned char *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void end_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

template <typename T> __device__ __forceinline__ void store4(T *p, float4 v) {
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(p) = v;
    } else {
        const __nv_bfloat162 x = __floats2bfloat162_rn(v.x, v.y), y = __floats2bfloat162_rn(v.z, v.w);
        *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&x), *reinterpret_cast<const uint32_t *>(&y));
    }
}
__device__ __forceinline__ void add4(float4 &y, float f, float4 v) {
    y.x = fmaf(f, v.x, y.x), y.y = fmaf(f, v.y, y.y), y.z = fmaf(f, v.z, y.z), y.w = fmaf(f, v.w, y.w);
}
// the row and head of a column; the result's place
template <int D, typename T> __device__ __forceinline__ void store_out(const AttnArgs &a, int b, int h, int rho, int d, int n, float4 y, float total) {
    const int m = rho / a.heads;
    const float r = m < n && total != 0.f ? 1.f / total : 0.f;
    T *out = (T *)a.out + ((((size_t)b * a.rows + m) * a.c.Hkv + h) * a.heads + rho % a.heads) * D + d;
    store4(out, r == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(y.x * r, y.y * r, y.z * r, y.w * r));
}

template <int D, int G, int NT> struct Shared {
    static constexpr int C = 8 * NT;
    union {
        unsigned char ring[kWarps][kStages][Tile<D, G>::BYTES];
        float o[kWarps][C][D + 4];   // the warps' outputs
    };
    struct {
        uint32_t hi[NT][D / 32][32][4], lo[NT][D / 32][32][4];   // in operand order
    } q;
    float2 ml[kWarps][C];   // the warps' maxima and sums
    float most[C][2];       // largest finite query of a column (of its halves)
    float alpha[C];         // what a unit of its scores is worth
    float2 ml_all[C];       // the block's
    float y[C][D];
    Plan plan;              // (runs alone; last)
};

template <int D, int G, int NT, bool F32> __global__ void __launch_bounds__(kAttnThreads, NT == 1 ? 2 : 1) attend_kernel(const AttnArgs a) {
    using L = Tile<D, G>;
    constexpr int J = D / 32, W = D / 64, C = 8 * NT, HALF = D / 2;
    using T = std::conditional_t<F32, float, __nv_bfloat16>;
    extern __shared__ __align__(16) unsigned char raw[];
    Shared<D, G, NT> &sh = *reinterpret_cast<Shared<D, G, NT> *>(raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    Pair base;
    asm volatile("mov.b32 %0, 0x64006400;" : "=r"(base.low));
    asm volatile("mov.b32 %0, 0x54005400;" : "=r"(base.high));
    pdl_trigger();
    pdl_wait();
    int64_t pos = 0, end = 1;
    if (!a.share) {
        make_plan(a, sh.plan);
        pos = run_start(a, sh.plan, blockIdx.x, gridDim.x);
        end = run_start(a, sh.plan, blockIdx.x + 1, gridDim.x);
    }
    while (pos < end) {
        Place f;
        int tile1, first, step = kWarps;
        if (a.share) {
            const int seg = blockIdx.x / a.share, per = a.c.Hkv * a.blocks;
            f.b = seg / per;
            f.seg = seg % per;
            f.off = 0;
            f.n = tile1 = tiles_of(a, f.b);
            first = blockIdx.x % a.share * kWarps + warp;
            step *= a.share;
        } else {
            f = find(a, sh.plan, pos);
            tile1 = (int)min((int64_t)f.n, f.off + end - pos);
            first = f.off + warp;
        }
        const int b = f.b, h = f.seg / a.blocks, pair0 = f.seg % a.blocks * C;
        const int n = rows_of(a, b), old = (int)max((int64_t)a.n_ctx[b] - n, (int64_t)-64);   // positions before the new rows

        // ---- the ring: stage i % kStages holds the warp's tile first + i * step
        const uint32_t ring = (uint32_t)__cvta_generic_to_shared(sh.ring[warp][0]);
        const int32_t *table = a.c.table + b * a.c.table_stride;
        uint32_t there = 0;   // bit s: stage s holds a tile
        auto page_of = [&](int tile) { return tile < tile1 ? table[tile >> a.c.shift] : -1; };
        auto fetch = [&](int stage, int tile, int page) {
            there &= ~(1u << stage);
            if ((unsigned)page < (unsigned)a.c.n_pages) {
                const unsigned char *src = a.c.pool + ((((size_t)page * a.c.Hkv + h) << a.c.shift) + (tile & ((1 << a.c.shift) - 1))) * L::BYTES + lane * 16;
                const uint32_t dst = ring + stage * L::BYTES + lane * 16;
#pragma unroll
                for (int i = 0; i < L::BYTES / 512; i++) copy16(dst + i * 512, src + i * 512);
                if (lane < L::BYTES % 512 / 16) copy16(dst + L::BYTES / 512 * 512, src + L::BYTES / 512 * 512);
                there |= 1u << stage;
            }
            end_copies();
        };
        int next_page;
        {
            int pages[kStages];
#pragma unroll
            for (int i = 0; i < kStages; i++) pages[i] = page_of(first + i * step);
#pragma unroll
            for (int i = 0; i < kStages - 1; i++) fetch(i, first + i * step, pages[i]);
            next_page = pages[kStages - 1];
        }

        // ---- queries: turned, scaled by a power of two that takes the largest below 2^15, split into fp16 terms
        constexpr int QI = (C * HALF + kAttnThreads - 1) / kAttnThreads;
        static_assert(C * HALF % 32 == 0 && HALF % 32 == 0, "a warp's values belong to one column");
        float2 qv[QI];
#pragma unroll
        for (int i = 0; i < QI; i++) {
            const int idx = tid + i * kAttnThreads, c = idx / HALF, e = idx % HALF, rho = pair0 + c, m = rho / a.heads;
            qv[i] = make_float2(0.f, 0.f);
            float most = 0.f;
            if (c < C && m < n) {
                const T *src = (const T *)a.q + b * a.qs[0] + m * a.qs[1] + (int64_t)(h * a.heads + rho % a.heads) * a.qs[2] + 2 * e;
                qv[i] = make_float2(to_f(src[0]), to_f(src[1]));
                if (a.rope) {
                    const int at = a.positions ? a.positions[(int64_t)b * a.rows + m] : old + m;
                    qv[i] = turn(qv[i].x, qv[i].y, reinterpret_cast<const float2 *>(a.rope)[(int64_t)min(max(at, 0), a.n_rope - 1) * HALF + e]);
                }
                const float u = fabsf(qv[i].x), v = fabsf(qv[i].y);   // (what is not finite does not count)
                if (u <= -kLowest) most = fmaxf(most, u);
                if (v <= -kLowest) most = fmaxf(most, v);
            }
            most = warp_max(most);
            if (c < C && lane == 0) sh.most[c][e / 32] = most;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < QI; i++) {
            const int idx = tid + i * kAttnThreads, c = idx / HALF, d = idx % HALF * 2;
            if (c < C) {
                const float most = HALF == 64 ? fmaxf(sh.most[c][0], sh.most[c][1]) : sh.most[c][0];
                const int ex = max((int)(__float_as_uint(most) >> 23) - 127, -110);   // floor(log2), not below -110
                const float up = __uint_as_float((uint32_t)(127 + 14 - ex) << 23);
                if (d == 0) sh.alpha[c] = a.scale2 * __uint_as_float((uint32_t)(127 + ex - 14) << 23);
                // operand order: word p of lane 4 (c % 8) + t holds dimensions 32 j + 8 t + p and + 4 of it
                const int j = d / 32, tt = d % 32 / 8, p = d % 4, half = d % 8 / 4;
                const float x = qv[i].x * up, y = qv[i].y * up;
                const __half hx = __float2half_rn(x), hy = __float2half_rn(y);
                __half *hi = reinterpret_cast<__half *>(sh.q.hi[c / 8][j][c % 8 * 4 + tt]) + half;
                hi[2 * p] = hx;
                hi[2 * p + 2] = hy;
                if (F32) {
                    __half *lo = reinterpret_cast<__half *>(sh.q.lo[c / 8][j][c % 8 * 4 + tt]) + half;
                    lo[2 * p] = __float2half_rn(x - __half2float(hx));
                    lo[2 * p + 2] = __float2half_rn(y - __half2float(hy));
                }
            }
        }
        __syncthreads();

        // ---- what the lane's columns (2 t, 2 t + 1 of each eight) see
        int limit[NT][2];
        uint32_t bits[NT][2];
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const int m = (pair0 + i * 8 + 2 * t + k) / a.heads;
                limit[i][k] = m < n ? (a.visible ? old : old + m + 1) : INT_MIN;
                bits[i][k] = a.visible && m < n ? (uint32_t)a.visible[(int64_t)b * a.rows + m] & (0xffffu >> (16 - n)) : 0u;
            }

        float o[D / 16][NT][4], mx[NT][2], sum[NT][2], alpha[NT][2];
        // A numerator enters the product as e * scale * unit, with a power of two for each column that puts the largest so far near 2^8: e <=
        // 2^kRise then keeps them below fp16's range, and what is dropped is below 2^-33 of the largest.  units: the largest of the lane's
        float unit[NT][2], weight[NT][2], units = 0x1p120f;
#pragma unroll
        for (int i = 0; i < NT; i++) {
#pragma unroll
            for (int k = 0; k < 2; k++) mx[i][k] = kLowest, sum[i][k] = 0.f, unit[i][k] = units, weight[i][k] = 0.f, alpha[i][k] = sh.alpha[i * 8 + 2 * t + k];
#pragma unroll
            for (int r = 0; r < D / 16; r++)
#pragma unroll
                for (int k = 0; k < 4; k++) o[r][i][k] = 0.f;
        }

        int stage = 0;
        for (int tile = first; tile < tile1; tile += step, stage = (stage + 1) % kStages) {
            wait_copies<kStages - 2>();
            __syncwarp();   // (every lane's copies; and the stage before this one has been read)
            fetch((stage + kStages - 1) % kStages, tile + (kStages - 1) * step, next_page);
            next_page = page_of(tile + kStages * step);
            if (!(there >> stage & 1)) continue;
            const unsigned char *src = sh.ring[warp][stage];
            // ---- scores
            float x[NT][4], vs[G][2];
#pragma unroll
            for (int i = 0; i < NT; i++)
#pragma unroll
                for (int k = 0; k < 4; k++) x[i][k] = 0.f;
            uint32_t kw[2][J];
#pragma unroll
            for (int r = 0; r < 2; r++) {
                if constexpr (J == 4) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(src + (g + 8 * r) * (D / 2) + t * 16);
                    kw[r][0] = v.x, kw[r][1] = v.y, kw[r][2] = v.z, kw[r][3] = v.w;
                } else {
                    const uint2 v = *reinterpret_cast<const uint2 *>(src + (g + 8 * r) * (D / 2) + t * 8);
                    kw[r][0] = v.x, kw[r][1] = v.y;
                }
            }
#pragma unroll
            for (int gi = 0; gi < G; gi++) {
                float ks[2];
                Pair z[2];
#pragma unroll
                for (int r = 0; r < 2; r++) {
                    const uint32_t word = reinterpret_cast<const uint32_t *>(src + L::SCALES)[gi * 16 + g + 8 * r];
                    ks[r] = __uint_as_float(word << 16);
                    vs[gi][r] = __uint_as_float(word & 0xffff0000u);
                    z[r] = zeros<true>(src[L::KZ + gi * 16 + g + 8 * r]);
                }
                float acc[NT][4];
#pragma unroll
                for (int i = 0; i < NT; i++)
#pragma unroll
                    for (int k = 0; k < 4; k++) acc[i][k] = 0.f;
#pragma unroll
                for (int j = gi * J / G; j < (gi + 1) * J / G; j++) {
                    uint32_t e[2][4];   // [row][dimensions p, p + 4 of the word]
#pragma unroll
                    for (int r = 0; r < 2; r++) {
                        e[r][0] = low(kw[r][j], base, z[r]);
                        e[r][1] = high(kw[r][j], base, z[r]);
                        e[r][2] = low(kw[r][j] >> 8, base, z[r]);
                        e[r][3] = high(kw[r][j] >> 8, base, z[r]);
                    }
                    const uint32_t a0[4] = {e[0][0], e[1][0], e[0][1], e[1][1]}, a1[4] = {e[0][2], e[1][2], e[0][3], e[1][3]};
#pragma unroll
                    for (int i = 0; i < NT; i++) {
                        const uint4 q = *reinterpret_cast<const uint4 *>(sh.q.hi[i][j][lane]);
                        mma(acc[i], a0, q.x, q.y);
                        mma(acc[i], a1, q.z, q.w);
                        if (F32) {
                            const uint4 l = *reinterpret_cast<const uint4 *>(sh.q.lo[i][j][lane]);
                            mma(acc[i], a0, l.x, l.y);
                            mma(acc[i], a1, l.z, l.w);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < NT; i++)
#pragma unroll
                    for (int k = 0; k < 4; k++) x[i][k] = gi ? fmaf(acc[i][k], ks[k >> 1], x[i][k]) : acc[i][k] * ks[k >> 1];
            }
#pragma unroll
            for (int i = 0; i < NT; i++)
#pragma unroll
                for (int k = 0; k < 4; k++) x[i][k] *= alpha[i][k & 1];
            // ---- masks
            uint32_t hidden = 0;   // bit 4 i + k
            const bool masked = old - tile * 16 < 16;
            if (masked) {
#pragma unroll
                for (int i = 0; i < NT; i++)
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const int p = tile * 16 + g + 8 * (k >> 1);
                        const uint32_t j = (uint32_t)p - (uint32_t)old;   // (past the old ones: which of the new)
                        const bool seen = p < limit[i][k & 1] || (j < 16u && bits[i][k & 1] >> j & 1);
                        if (!seen) hidden |= 1u << (4 * i + k), x[i][k] = -INFINITY;
                    }
            }
            // ---- a new maximum, or a new unit, where some score (or scale) is far above the last: seldom
            float vmost = 0.f;
#pragma unroll
            for (int gi = 0; gi < G; gi++) vmost = fmaxf(vmost, fmaxf(vs[gi][0], vs[gi][1]));
            bool rise = masked || vmost * units > 65000.f / (1 << kRise);
#pragma unroll
            for (int i = 0; i < NT; i++)
#pragma unroll
                for (int k = 0; k < 4; k++) rise |= x[i][k] > mx[i][k & 1] + (float)kRise;
            if (__any_sync(0xffffffffu, rise)) {
                float v[2] = {vs[0][0], vs[0][1]};   // the tokens' largest scales
#pragma unroll
                for (int gi = 1; gi < G; gi++) v[0] = fmaxf(v[0], vs[gi][0]), v[1] = fmaxf(v[1], vs[gi][1]);
                units = 0.f;
#pragma unroll
                for (int i = 0; i < NT; i++)
#pragma unroll
                    for (int k = 0; k < 2; k++) {
                        float top = fmaxf(x[i][k], x[i][k + 2]);
#pragma unroll
                        for (int s = 4; s < 32; s <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
                        top = fmaxf(top, mx[i][k]);
                        // (what a column does not see changes neither its maximum nor its unit)
                        float most = fmaxf(hidden >> (4 * i + k) & 1 ? 0.f : ex2(x[i][k] - top) * v[0], hidden >> (4 * i + k + 2) & 1 ? 0.f : ex2(x[i][k + 2] - top) * v[1]);
#pragma unroll
                        for (int s = 4; s < 32; s <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
                        float shift = mx[i][k] - top;
                        const float f1 = ex2(shift);
                        mx[i][k] = top;
                        sum[i][k] *= f1;
                        weight[i][k] = fmaxf(weight[i][k] * f1, most);
                        if (weight[i][k] > 0.f && weight[i][k] <= -kLowest) {
                            const int next = 8 + 127 - max((int)(__float_as_uint(weight[i][k]) >> 23), 15), last = (int)(__float_as_uint(unit[i][k]) >> 23) - 127;
                            shift += (float)(next - last);
                            unit[i][k] = power(next);
                        }
                        units = fmaxf(units, unit[i][k]);
                        const float f = ex2(shift);
#pragma unroll
                        for (int r = 0; r < D / 16; r++) o[r][i][k] *= f, o[r][i][k + 2] *= f;
                    }
            }
            // ---- numerators
#pragma unroll
            for (int i = 0; i < NT; i++)
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    x[i][k] = ex2(x[i][k] - mx[i][k & 1]);
                    sum[i][k & 1] += x[i][k];
                }
            // ---- outputs
            uint32_t vw[W][4];
#pragma unroll
            for (int w = 0; w < W; w++) {
                const uint4 v = *reinterpret_cast<const uint4 *>(src + L::V + w * 512 + lane * 16);
                vw[w][0] = v.x, vw[w][1] = v.y, vw[w][2] = v.z, vw[w][3] = v.w;
            }
#pragma unroll
            for (int gi = 0; gi < G; gi++) {
                uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
                for (int i = 0; i < NT; i++) {
                    float y[4];
#pragma unroll
                    for (int k = 0; k < 4; k++) y[k] = x[i][k] * (vs[gi][k >> 1] * unit[i][k & 1]);
                    if (masked) {   // (0 times a scale that is not finite)
#pragma unroll
                        for (int k = 0; k < 4; k++)
                            if (hidden >> (4 * i + k) & 1) y[k] = 0.f;
                    }
                    ph[i][0] = pack(y[0], y[1]);
                    ph[i][1] = pack(y[2], y[3]);
                    if (F32) {
                        pl[i][0] = transpose(pack_rest(y[0], y[1], ph[i][0]));
                        pl[i][1] = transpose(pack_rest(y[2], y[3], ph[i][1]));
                    }
                    ph[i][0] = transpose(ph[i][0]);
                    ph[i][1] = transpose(ph[i][1]);
                }
                Pair z[2];   // of tokens 2 t, 2 t + 1 and those 8 after them
#pragma unroll
                for (int r = 0; r < 2; r++) z[r] = zeros<false>(*reinterpret_cast<const uint16_t *>(src + L::VZ + gi * 16 + 8 * r + 2 * t));
#pragma unroll
                for (int r16 = gi * (D / 16) / G; r16 < (gi + 1) * (D / 16) / G; r16++) {
                    const int w = r16 / 4, q = r16 % 4;   // nibbles 2 q, 2 q + 1 of the words
                    uint32_t av[4];
#pragma unroll
                    for (int r = 0; r < 2; r++) {
                        uint32_t y = __byte_perm(vw[w][2 * r], vw[w][2 * r + 1], q < 2 ? 0x5410 : 0x7632);
                        if (q & 1) y >>= 8;
                        av[2 * r] = low(y, base, z[r]);
                        av[2 * r + 1] = high(y, base, z[r]);
                    }
#pragma unroll
                    for (int i = 0; i < NT; i++) {
                        mma(o[r16][i], av, ph[i][0], ph[i][1]);
                        if (F32) mma(o[r16][i], av, pl[i][0], pl[i][1]);
                    }
                }
            }
        }
        wait_copies<0>();

        // ---- the warps' results meet
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
            for (int k = 0; k < 2; k++)
#pragma unroll
                for (int s = 4; s < 32; s <<= 1) sum[i][k] += __shfl_xor_sync(0xffffffffu, sum[i][k], s);
        __syncthreads();   // (the tiles and the queries have been read)
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const int c = i * 8 + 2 * t + k;
                const float worth = 1.f / unit[i][k];
                if (g == 0) sh.ml[warp][c] = make_float2(mx[i][k], sum[i][k]);
#pragma unroll
                for (int r = 0; r < D / 16; r++) sh.o[warp][c][16 * r + g] = o[r][i][k] * worth, sh.o[warp][c][16 * r + 8 + g] = o[r][i][k + 2] * worth;
            }
        __syncthreads();
        const bool all = a.share ? a.share == 1 : f.off == 0 && tile1 == f.n;
        float *part = a.part + (size_t)(2 * blockIdx.x + (f.off == 0)) * C * (D + 4);
        for (int idx = tid; idx < C * (D / 4); idx += kAttnThreads) {
            const int c = idx / (D / 4), d = idx % (D / 4) * 4, rho = pair0 + c;
            if (rho >= a.rows * a.heads) break;
            float top = kLowest, total = 0.f;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; w++) top = fmaxf(top, sh.ml[w][c].x);
#pragma unroll
            for (int w = 0; w < kWarps; w++) {
                const float2 ml = sh.ml[w][c];
                const float f1 = ex2(ml.x - top);
                total = fmaf(f1, ml.y, total);
                add4(y, f1, *reinterpret_cast<const float4 *>(&sh.o[w][c][d]));
            }
            if (all) {
                store_out<D, T>(a, b, h, rho, d, n, y, total);
            } else if (a.share) {
                *reinterpret_cast<float4 *>(&sh.y[c][d]) = y;
                if (d == 0) sh.ml_all[c] = make_float2(top, total);
            } else {
                *reinterpret_cast<float4 *>(part + c * (D + 4) + d) = y;
                if (d == 0) *reinterpret_cast<float2 *>(part + c * (D + 4) + D) = make_float2(top, total);
            }
        }
        if (a.share > 1) {
            cg::cluster_group cluster = cg::this_cluster();
            cluster.sync();
            for (int idx = blockIdx.x % a.share * kAttnThreads + tid; idx < C * (D / 4); idx += a.share * kAttnThreads) {
                const int c = idx / (D / 4), d = idx % (D / 4) * 4, rho = pair0 + c;
                if (rho >= a.rows * a.heads) break;
                float top = kLowest, total = 0.f;
                float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int r = 0; r < a.share; r++) top = fmaxf(top, cluster.map_shared_rank(&sh.ml_all[c], r)->x);
                for (int r = 0; r < a.share; r++) {
                    const float2 ml = *cluster.map_shared_rank(&sh.ml_all[c], r);
                    const float f1 = ex2(ml.x - top);
                    total = fmaf(f1, ml.y, total);
                    add4(y, f1, *reinterpret_cast<const float4 *>(cluster.map_shared_rank(&sh.y[c][d], r)));
                }
                store_out<D, T>(a, b, h, rho, d, n, y, total);
            }
            cluster.sync();   // (the others read this block's memory)
        }
        if (a.share) return;
        __syncthreads();
        pos += tile1 - f.off;
    }
}

// One block: a column of a segment that several blocks shared; their parts are added in the order of the tiles.
template <int D, int NT, bool F32> __global__ void __launch_bounds__(kAttnThreads) join_kernel(const AttnArgs a, int grid) {
    constexpr int C = 8 * NT, LANES = D / 4, GROUPS = kAttnThreads / LANES;
    using T = std::conditional_t<F32, float, __nv_bfloat16>;
    __shared__ Plan plan;
    __shared__ float2 ml[kMaxGrid + 1];
    __shared__ float4 ys[GROUPS][LANES];
    __shared__ float tops[kWarps], sums[kWarps];
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = a.c.Hkv * a.blocks, b = blockIdx.x / per, seg = blockIdx.x % per, c = blockIdx.y, rho = seg % a.blocks * C + c;
    if (rho >= a.rows * a.heads) return;
    make_plan(a, plan);
    const int64_t len = plan.before[b + 1] - plan.before[b], start = plan.before[b] * per + seg * len, total = plan.before[a.B] * per;
    if (len < 2 * kUnit) return;   // (never cut)
    auto cut = [&](int64_t i) { return cut_at(total * i / grid - start, len); };
    // runs i0 .. i0 + count - 1 may hold a part of it
    const int i0 = (int)(start * grid / total), count = (int)min((int64_t)grid - 1, (start + len - 1) * grid / total + 1) - i0 + 1;
    int parts = 0;
    float top = kLowest;
    for (int k0 = 0; k0 < count; k0 += kAttnThreads) {
        const int k = k0 + tid;
        const int64_t from = k < count ? cut(i0 + k) : 0, to = k < count ? cut(i0 + k + 1) : 0;
        parts += __syncthreads_count(from < to);
        if (k < count) {
            ml[k].x = kLowest, ml[k].y = 0.f;
            if (from < to) ml[k] = *reinterpret_cast<const float2 *>(a.part + ((size_t)(2 * (i0 + k) + (from == 0)) * C + c) * (D + 4) + D);
            top = fmaxf(top, ml[k].x);
        }
    }
    if (parts < 2) return;
    top = warp_max(top);
    if (lane == 0) tops[warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; w++) top = fmaxf(top, tops[w]);
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    const int d = tid % LANES * 4;
#pragma unroll 8
    for (int k = tid / LANES; k < count; k += GROUPS) {
        const int64_t from = cut(i0 + k);
        if (from < cut(i0 + k + 1)) add4(y, ex2(ml[k].x - top), __ldcg(reinterpret_cast<const float4 *>(a.part + ((size_t)(2 * (i0 + k) + (from == 0)) * C + c) * (D + 4) + d)));
    }
    ys[tid / LANES][tid % LANES] = y;
    float sum = 0.f;
    for (int k = tid; k < count; k += kAttnThreads) sum = fmaf(ex2(ml[k].x - top), ml[k].y, sum);
    sum = warp_sum(sum);
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    if (tid < LANES) {
        sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; w++) sum += sums[w];
#pragma unroll
        for (int k = 1; k < GROUPS; k++) add4(y, 1.f, ys[k][tid]);
        store_out<D, T>(a, b, seg / a.blocks, rho, d, rows_of(a, b), y, sum);
    }
}

// ---------------------------------------------------------------------------------- launches
// How a call is shared out: column tiles a block takes at once, blocks of a cluster (0: runs)
struct Way { int nt, share; };
Way way_of(const eesd_kv4 *c, const eesd_kv4_rows *r, int n_heads) {
    const int64_t columns = (int64_t)(n_heads / c->n_kv_heads) * r->rows, tiles = (int64_t)r->max_pages * (c->page_tokens / 16);
    Way w;
    w.nt = columns <= 8 ? 1 : 2;
    const int64_t segments = (int64_t)r->B * c->n_kv_heads * ((columns + 8 * w.nt - 1) / (8 * w.nt));
    w.share = 1;
    while (w.share < 8 && segments * w.share * 2 <= grid_of(w.nt) && w.share * kWarps < tiles) w.share *= 2;
    if (segments * tiles > 64LL * grid_of(w.nt) || tiles > 64LL * w.share * 4) w.share = 0;
    return w;
}

template <int D, int G, int NT, bool F32> cudaError_t launch(cudaStream_t s, const AttnArgs &a, int64_t segments) {
    constexpr int kSmem = sizeof(Shared<D, G, NT>);
    auto kernel = attend_kernel<D, G, NT, F32>;
    {
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
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.share ? (unsigned int)(segments * a.share) : grid_of(NT));
    cfg.blockDim = dim3(kAttnThreads);
    cfg.dynamicSmemBytes = a.share ? kSmem - sizeof(Plan) : kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int na = 0;
    if (a.share > 1) {
        attr[na].id = cudaLaunchAttributeClusterDimension;
        attr[na].val.clusterDim.x = a.share;
        attr[na].val.clusterDim.y = 1;
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
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
    if (e != cudaSuccess) return e;
    if (!a.share) launch_k(join_kernel<D, NT, F32>, dim3((unsigned int)segments, 8 * NT), dim3(kAttnThreads), 0, s, pdl_enabled(), a, grid_of(NT));
    return cudaGetLastError();
}
template <int D, int G> cudaError_t launch_type(cudaStream_t s, const AttnArgs &a, bool f32, int nt, int64_t segments) {
    if (nt == 1) return f32 ? launch<D, G, 1, true>(s, a, segments) : launch<D, G, 1, false>(s, a, segments);
    return f32 ? launch<D, G, 2, true>(s, a, segments) : launch<D, G, 2, false>(s, a, segments);
}

}  // namespace kv4
}  // namespace eesd

using namespace eesd;

extern "C" {

size_t eesd_kv4_attend_scratch_bytes(const eesd_kv4 *c, const eesd_kv4_rows *r, int n_heads, int dtype) {
    eesd_kv4_layout l;
    if (eesd_kv4_layout_of(c, &l) || !r || r->max_pages < 1 || r->rows < 1 || r->rows > EESD_MAX_ROWS) return 0;
    if (n_heads < 1 || n_heads % c->n_kv_heads || (dtype != EESD_F32 && dtype != EESD_BF16) || r->B < 1) return 0;
    const kv4::Way w = kv4::way_of(c, r, n_heads);
    return w.share ? 0 : (size_t)2 * kv4::grid_of(w.nt) * 8 * w.nt * (c->head_dim + 4) * 4;
}

int eesd_kv4_attend(void *cuda_stream, const eesd_kv4 *c, const void *pool, size_t pool_bytes, const eesd_kv4_rows *r, int dtype, const eesd_kv4_tensor *q,
                    int n_heads, float scale, const int32_t *visible, void *out, void *scratch, size_t scratch_bytes) {
    kv4::AttnArgs a = {};
    eesd_kv4_layout l;
    int st = kv4_open(c, pool, pool_bytes, r, &a.c, &l);
    if (st) return st;
    if (!r->at || (dtype != EESD_F32 && dtype != EESD_BF16) || r->rows > EESD_MAX_ROWS || n_heads < 1 || n_heads % c->n_kv_heads) return EESD_ERR_BADARG;
    if ((st = kv4_rows_check(q, dtype))) return st;
    if (!out || ((uintptr_t)out & 15) || ((uintptr_t)visible & 3) || !(scale > 0.f) || !(scale <= 3.402823466e38f)) return EESD_ERR_BADARG;
    if (const size_t need = eesd_kv4_attend_scratch_bytes(c, r, n_heads, dtype)) {
        if (!scratch || ((uintptr_t)scratch & 15)) return EESD_ERR_BADARG;
        if (scratch_bytes < need) return EESD_ERR_NOMEM;
    }
    a.n_ctx = r->at;
    a.n_rows = r->n_rows;
    a.positions = r->positions;
    a.visible = visible;
    a.rope = r->rope;
    a.n_rope = r->n_rope;
    a.q = q->data;
    a.qs[0] = q->stride_b, a.qs[1] = q->stride_row, a.qs[2] = q->stride_head;
    a.out = out;
    a.scale2 = scale * 1.4426950408889634f;
    a.B = r->B;
    a.rows = r->rows;
    a.heads = n_heads / c->n_kv_heads;
    const kv4::Way w = kv4::way_of(c, r, n_heads);
    a.blocks = (int)(((int64_t)a.heads * r->rows + 8 * w.nt - 1) / (8 * w.nt));
    a.share = w.share;
    a.part = (float *)scratch;
    const int64_t segments = (int64_t)r->B * c->n_kv_heads * a.blocks;
    if (segments * (w.share ? w.share : 1) > 0x7fffffffLL) return EESD_ERR_UNSUPPORTED;
    const bool f32 = dtype == EESD_F32;
    const int G = c->head_dim / c->group;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    const cudaError_t e = c->head_dim == 64 ? (G == 1 ? kv4::launch_type<64, 1>(s, a, f32, w.nt, segments) : kv4::launch_type<64, 2>(s, a, f32, w.nt, segments))
                          : G == 1          ? kv4::launch_type<128, 1>(s, a, f32, w.nt, segments)
                          : G == 2          ? kv4::launch_type<128, 2>(s, a, f32, w.nt, segments)
                                            : kv4::launch_type<128, 4>(s, a, f32, w.nt, segments);
    return e == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

}  // extern "C"
