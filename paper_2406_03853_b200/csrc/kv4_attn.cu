// Attention of up to 16 rows a sequence over the 4-bit key / value cache (sm_100a).
//
//   x_p = scale * sum_G s_pG (q_G . (c - z)_pG),   out = sum_p (e_p s_pG) (c - z)_pG / sum_p e_p,   e_p = exp(x_p - max x)
//
// Codes less zero points are small whole numbers, so the scales stay outside the matrix products: a key's scales multiply the groups' scores, a
// value's the softmax numerator. One pass over the codes with a running maximum.
//
// A warp takes tiles of 16 tokens for 8 columns (pairs of a row and a head that share the key head) or 16. Both products have the tile as their
// 16-row operand, straight from its codes in registers:
//   scores   S^T[token][column] = K Q^T (m16n8k16, fp16): queries of two fp16 terms under a power of two that puts a row and head's largest at 2^14, so that
//            each keeps 22 bits of its own down to 2^-18 of the largest; codes less their zero points, exactly. (As whole numbers of 16 or 24 bits by bytes,
//            which takes fewer operations a code and 8 of the 32 sequences' 66 us below less, one loud channel would cost all others their bits)
//   outputs  O^T[dimension][column] = V^T P^T (m16n8k16, fp16): numerators of two fp16 terms (22 bits, for bf16 rows too: with one, pairs of positions
//            that cancel would leave errors of 2^-12 of either) by codes set into an fp16 mantissa; an 8 x 8 transposition (movmatrix) stands between a
//            score's accumulators and the numerators' operand
// Sums are held in 32 bits. Tiles come through a ring of asynchronous copies that belongs to the warp; the warps of a block meet once, at a segment's
// end.
//
// A segment is what one key head of one sequence has to do for 8 NT columns. Two ways to share the machine (way_of):
//   clusters  the blocks of a cluster share a segment and push their parts into the shared memory of the block that joins them (one launch)
//   runs      the tiles of all segments stand in a row and are dealt out evenly, whatever the sequences' lengths; a second kernel joins what was cut.
//             Two tiles a step of a warp (TT), which hide each other's latency: the 130001 tokens below 217 us, one tile a step 228 (and none of the
//             spills, 152 to 232 bytes a thread with heads of 128, that two take at 128 registers)
//
// What bounds it (70B shape, 64 heads on 8 of 128; B200): 32 sequences of up to 8192 tokens, one row, bf16: 66 us, 180 MB, 0.42 of the copy rate;
// 130001 tokens, 5 rows, fp32: 217 us, 21 GFLOP. A warp's unit of 16 tokens by 8 columns is 413 instructions (two groups a head: 439), 32 of them matrix
// instructions, at four warps a scheduler: 57 to 64 % of the issue slots, 43 to 47 % of the ALU pipe. Short calls (one sequence of 1056 tokens, 5 rows, 13B
// shape: 8.4 us) are launch, four dependent reads and the joining.
#include <cooperative_groups.h>
#include <cuda_fp16.h>
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "kernels.cuh"
#include "kv4.cuh"

namespace eesd {
namespace kv4 {

namespace cg = cooperative_groups;

constexpr int kWarps = 8, kAttnThreads = kWarps * 32;
constexpr int kMaxShare = 16;     // blocks of a cluster
constexpr int kUnit = 2 * kWarps;   // runs: tiles between the places where a segment may be cut
constexpr int kMaxGrid = 296;
__host__ __device__ constexpr int grid_of(int nt) { return nt == 1 ? kMaxGrid : kMaxGrid / 2; }   // blocks that fit the machine's 148 multiprocessors at once
constexpr int kRise = 8;     // a running maximum is let fall behind by this much (powers of two)
constexpr float kLowest = -3.402823466e38f;

struct AttnArgs {
    Cache c;
    const int32_t *n_ctx, *n_rows, *positions, *visible;
    const float *rope;
    int n_rope;
    const void *q;
    int64_t qs[3];
    void *out;
    float scale2;        // scale * log2(e), as scale2 * 2^scale_exp, 0.5 <= scale2 < 1
    int scale_exp;
    int B, rows, heads;  // heads: query heads of a key head
    int blocks;          // column blocks of a key head
    int share;           // blocks of a cluster (runs: 0)
    bool wide;           // runs: the call may have 2^31 tiles
    bool pairs;          // pairs of queries are aligned
    int4 *head;          // runs: of each block, the sequence and segment that it began and left to the next ones (-1: none), and what it did of the one
                         // that it found begun: 0 nothing, 1 some, 2 its end
    float *part;         // runs: [2 * grid][columns][D + 4]: outputs, maximum, sum; of what a block found begun, and of what it left
};

__device__ __forceinline__ int rows_of(const AttnArgs &a, int b) { return a.n_rows ? min(max(a.n_rows[b], 0), a.rows) : a.rows; }
// tiles that hold what some of n rows of a sequence of ctx tokens may see, at least 1
__device__ __forceinline__ int tiles_of(const AttnArgs &a, int ctx, int n) {
    return n ? (int)max((int64_t)1, min((int64_t)a.c.max_pages << a.c.shift, ((int64_t)ctx + 15) / 16)) : 1;
}

// ---------------------------------------------------------------------------------- runs
// A cut inside a segment lies at a multiple of kUnit tiles, and at an end where fewer than that would be left.
__device__ __forceinline__ int cut_at(int off, int n) {   // 0 <= off < n <= 2^27
    if (off == 0) return 0;
    const int c = (off + kUnit / 2) / kUnit * kUnit;
    return c + kUnit > n ? n : c;
}
struct Place {
    int b, seg;    // sequence; key head * blocks + column block
    int off, n;    // tile in the segment, of n
};
struct Plan {
    int ctx[EESD_KV4_MAX_BATCH];   // tokens and rows of each sequence
    uint8_t rows[EESD_KV4_MAX_BATCH];
    Place begin;                   // where the block's run begins
    int64_t count;                 // how many tiles it takes
    __device__ __forceinline__ int tiles(const AttnArgs &a, int b) const { return tiles_of(a, ctx[b], rows[b]); }
};
// The run of block `block` of GRID, worked out by the first warp.  T: what holds all tiles of the call.
template <int GRID, typename T> __device__ __forceinline__ void find_run(const AttnArgs &a, Plan &p, int block) {
    {
        const int lane = threadIdx.x;
        const T per = (T)a.c.Hkv * a.blocks;
        T total = 0;
        for (int b = lane; b < a.B; b += 32) {
            p.ctx[b] = a.n_ctx[b];
            p.rows[b] = (uint8_t)rows_of(a, b);
            total += p.tiles(a, b);
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        total *= per;
        __syncwarp();
        // lane 0 .. 31: the sequences 32 i + lane; the one whose tiles hold a run's end says where
        Place f = {a.B, 0, 0, 1};
        T at[2] = {total, total};
        T before = 0;   // tiles of one head and column block up to the chunk
        for (int b0 = 0; b0 < a.B; b0 += 32) {
            const int n = b0 + lane < a.B ? p.tiles(a, b0 + lane) : 0;
            T sum = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const T u = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += u;
            }
#pragma unroll
            for (int end = 0; end < 2; end++) {
                const T raw = (T)((uint64_t)total * (uint64_t)(block + end) / GRID), in = raw - (before + sum - n) * per;   // tiles past the start of the lane's sequence
                const bool here = n > 0 && in >= 0 && in < n * per;
                const uint32_t who = __ballot_sync(0xffffffffu, here);
                if (!who) continue;
                T start = 0;
                if (here) {
                    int seg = sizeof(T) == 8 && (uint64_t)in >> 32 ? (int)(in / n) : (int)((uint32_t)in / (uint32_t)n);
                    const int off = (int)(in - (T)seg * n);
                    int cut = (int)cut_at(off, n);
                    start = raw - off + cut;
                    int b = b0 + lane;
                    if (cut == n) {   // (the next segment's first)
                        cut = 0;
                        if (++seg == per) seg = 0, b++;
                    }
                    f = Place{b, seg, cut, b < a.B ? p.tiles(a, b) : 1};
                    if (end == 0) p.begin = f;
                }
                at[end] = __shfl_sync(0xffffffffu, start, __ffs(who) - 1);
            }
            before += __shfl_sync(0xffffffffu, sum, 31);
        }
        if (lane == 0) p.count = at[1] - at[0];
    }
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
// -(1024 + z) and -(64 + z) twice, of a zero point below 16
__device__ __forceinline__ Pair zero_twice(uint32_t z) { return Pair{__byte_perm(z, 0xe4u, 0x4040), __byte_perm(z << 4, 0xd4u, 0x4040)}; }
// the same of two zero points, bytes 0 and 1 of z
__device__ __forceinline__ Pair zeros(uint32_t z) { return Pair{__byte_perm(z, 0xe4u, 0x4140), __byte_perm(z << 4, 0xd4u, 0x4140)}; }
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

template <int D, int G, int NT, int TT> struct Shared {
    static constexpr int C = 8 * NT, STAGES = TT == 1 ? 4 : 2;   // STAGES: steps of a warp's ring
    union {
        unsigned char ring[kWarps][STAGES][TT * Tile<D, G>::BYTES];
        float o[kWarps][C][D + 4];   // the warps' outputs
    };
    uint32_t q[NT][D / 32][2][32][4]; // the queries' terms, in operand order
    float2 ml[kWarps][C];   // the warps' maxima and sums
    float2 alpha[C];        // what a unit of its scores is worth, as two factors
    // clusters: the blocks' parts of the results that this block joins: [block][its share], and their maxima and sums
    float4 in_y[C * D / 4 + kMaxShare];
    float2 in_ml[kMaxShare][C];
    Plan plan;              // (runs alone; last)
};

template <int D, int G, int NT, int TT, bool RUNS, bool F32> __global__ void __launch_bounds__(kAttnThreads, NT == 1 ? 2 : 1) attend_kernel(const AttnArgs a) {
    using L = Tile<D, G>;
    constexpr int J = D / 32, W = D / 64, C = 8 * NT, HALF = D / 2, kStages = Shared<D, G, NT, TT>::STAGES;
    using T = std::conditional_t<F32, float, __nv_bfloat16>;
    extern __shared__ __align__(16) unsigned char raw[];
    using S = Shared<D, G, NT, TT>;
    S &sh = *reinterpret_cast<S *>(raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    Pair base;
    asm volatile("mov.b32 %0, 0x64006400;" : "=r"(base.low));
    asm volatile("mov.b32 %0, 0x54005400;" : "=r"(base.high));
    if (!RUNS && a.share > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // (waited for before another block's memory is written)
    pdl_trigger();
    pdl_wait();
    Place f;
    int64_t left = 1;   // runs: tiles to do
    if constexpr (RUNS) {
        if (tid < 32) {
            if (a.wide) find_run<grid_of(NT), int64_t>(a, sh.plan, blockIdx.x);
            else find_run<grid_of(NT), int>(a, sh.plan, blockIdx.x);
        }
        __syncthreads();
        f = sh.plan.begin;
        left = sh.plan.count;
        if (tid == 0) a.head[blockIdx.x] = make_int4(-1, 0, 0, 0);
    } else {
        const int seg = blockIdx.x / a.share, per = a.c.Hkv * a.blocks;
        f.b = seg / per;
        f.seg = seg % per;
        f.off = 0;
        f.n = tiles_of(a, a.n_ctx[f.b], rows_of(a, f.b));
    }
    // What a segment begins with: its rows, the pages of the first tiles, its queries and their angles.  Asked for before the last segment's parts meet.
    constexpr int QK = HALF / 32;   // pairs of a lane in a column; a warp has the columns warp + 8 i
    static_assert(kWarps == 8 && C == 8 * NT && HALF % 32 == 0, "");
    const int step = TT * kWarps * (RUNS ? 1 : a.share);
    struct Pages { int v[TT]; };
    using Two = std::conditional_t<F32, float2, uint32_t>;
    struct Start {
        int b, h, pair0, n, old, tile1, first;
        Pages pages[kStages];
        Two q[NT][QK];   // as they lie in memory (what would use them waits for them)
        float2 turn[NT][QK];
    };
    auto pages_of = [&](const int32_t *table, int tile, int tile1) {
        Pages p;
#pragma unroll
        for (int i = 0; i < TT; i++) p.v[i] = tile + i < tile1 ? table[(tile + i) >> a.c.shift] : -1;
        return p;
    };
    auto read_ahead = [&](Start &s) {
        s.b = f.b, s.h = f.seg / a.blocks, s.pair0 = f.seg % a.blocks * C;
        s.tile1 = RUNS ? (int)min((int64_t)f.n, f.off + left) : f.n;
        s.first = f.off + (RUNS ? warp : blockIdx.x % a.share * kWarps + warp) * TT;
        s.n = RUNS ? sh.plan.rows[f.b] : rows_of(a, f.b);
        s.old = (int)max((int64_t)(RUNS ? sh.plan.ctx[f.b] : a.n_ctx[f.b]) - s.n, (int64_t)-64);   // positions before the new rows
        const int32_t *table = a.c.table + s.b * a.c.table_stride;
#pragma unroll
        for (int i = 0; i < kStages; i++) s.pages[i] = pages_of(table, s.first + i * step, s.tile1);
#pragma unroll
        for (int i = 0; i < NT; i++) {
            const int rho = s.pair0 + warp + 8 * i, m = rho / a.heads;
            const bool there = m < s.n;
            const T *src = (const T *)a.q + s.b * a.qs[0] + m * a.qs[1] + (int64_t)(s.h * a.heads + rho - m * a.heads) * a.qs[2] + 2 * lane;
            const float2 *cs = nullptr;
            if (there && a.rope) {
                const int at = a.positions ? a.positions[(int64_t)s.b * a.rows + m] : s.old + m;
                cs = reinterpret_cast<const float2 *>(a.rope) + (int64_t)min(max(at, 0), a.n_rope - 1) * HALF + lane;
            }
#pragma unroll
            for (int k = 0; k < QK; k++) {
                if (!there) s.q[i][k] = Two{};
                else if (a.pairs) s.q[i][k] = *reinterpret_cast<const Two *>(src + 64 * k);
                else if constexpr (F32) s.q[i][k] = make_float2(src[64 * k], src[64 * k + 1]);
                else s.q[i][k] = (uint32_t)__bfloat16_as_ushort(src[64 * k]) | (uint32_t)__bfloat16_as_ushort(src[64 * k + 1]) << 16;
                s.turn[i][k] = cs ? cs[32 * k] : make_float2(1.f, 0.f);
            }
        }
    };
    Start now;
    if (left > 0) read_ahead(now);
    while (left > 0) {
        const int b = now.b, h = now.h, pair0 = now.pair0, n = now.n, old = now.old, tile1 = now.tile1, first = now.first;

        // ---- the ring: stage i % kStages holds the warp's TT tiles from first + i * step on
        const uint32_t ring = (uint32_t)__cvta_generic_to_shared(sh.ring[warp][0]);
        const int32_t *table = a.c.table + b * a.c.table_stride;
        uint32_t there = 0;   // bit TT s + i: tile i of stage s exists
        auto fetch = [&](int stage, int tile, const Pages &pages) {
#pragma unroll
            for (int i = 0; i < TT; i++) {
                there &= ~(1u << (TT * stage + i));
                if ((unsigned)pages.v[i] < (unsigned)a.c.n_pages) {
                    const unsigned char *src =
                        a.c.pool + ((((size_t)pages.v[i] * a.c.Hkv + h) << a.c.shift) + ((tile + i) & ((1 << a.c.shift) - 1))) * L::BYTES + lane * 16;
                    const uint32_t dst = ring + (stage * TT + i) * L::BYTES + lane * 16;
#pragma unroll
                    for (int j = 0; j < L::BYTES / 512; j++) copy16(dst + j * 512, src + j * 512);
                    if (lane < L::BYTES % 512 / 16) copy16(dst + L::BYTES / 512 * 512, src + L::BYTES / 512 * 512);
                    there |= 1u << (TT * stage + i);
                }
            }
            end_copies();
        };
#pragma unroll
        for (int i = 0; i < kStages - 1; i++) fetch(i, first + i * step, now.pages[i]);
        Pages next_pages = now.pages[kStages - 1];

        // ---- queries: turned, and as two fp16 terms under a power of two of their column
#pragma unroll
        for (int i = 0; i < NT; i++) {
            const int c = warp + 8 * i;
            float2 qv[QK];
            float most = 0.f;
            bool bad = false;
#pragma unroll
            for (int k = 0; k < QK; k++) {
                // ((1, 0) would turn what is not finite)
                if constexpr (F32) qv[k] = now.q[i][k];
                else qv[k] = make_float2(__uint_as_float(now.q[i][k] << 16), __uint_as_float(now.q[i][k] & 0xffff0000u));
                if (a.rope) qv[k] = turn(qv[k].x, qv[k].y, now.turn[i][k]);
                const float u = fabsf(qv[k].x), v = fabsf(qv[k].y);
                if (!(u <= -kLowest) || !(v <= -kLowest)) bad = true, qv[k] = make_float2(0.f, 0.f);   // (the column is NaN)
                else most = fmaxf(most, fmaxf(u, v));
            }
            most = warp_max(most);
            bad = __any_sync(0xffffffffu, bad);
            // The largest comes to 2^14 .. 2^15 (subnormal ones to less), in two factors since one may pass fp32's range.  A score is (sum * first) * a key's scale * second, first
            // being kept from where sums (below 2^26) by the largest or the least scales would leave fp32's range; it takes all but at the ends
            const int ex = most == 0.f ? 0 : max((int)(__float_as_uint(most) >> 23) - 127, -126), up = 14 - ex;
            const float up0 = power(up >> 1), up1 = power(up - (up >> 1));
            const int worth = a.scale_exp - up, first = min(max(worth, -60), 40), rest = min(max(worth - first, -126), 127);
            if (lane == 0) sh.alpha[c] = make_float2(bad ? __uint_as_float(0x7fc00000u) : a.scale2 * power(first), power(rest));
#pragma unroll
            for (int k = 0; k < QK; k++) {
                // word w of lane 4 (c % 8) + t holds dimensions 32 j + 8 t + w and + 4; the lane has dimensions 64 k + 2 lane and + 1
                const float x = qv[k].x * up0 * up1, y = qv[k].y * up0 * up1;
                const uint32_t h = pack(x, y), l = pack_rest(x, y, h);
                const int j = 2 * k + lane / 16, slot = warp * 4 + lane % 16 / 4, word = lane % 2 * 2, half = lane % 4 / 2;
                uint16_t *qh = reinterpret_cast<uint16_t *>(sh.q[i][j][0][slot]) + 2 * word + half, *ql = reinterpret_cast<uint16_t *>(sh.q[i][j][1][slot]) + 2 * word + half;
                qh[0] = (uint16_t)h, qh[2] = (uint16_t)(h >> 16);
                ql[0] = (uint16_t)l, ql[2] = (uint16_t)(l >> 16);
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
        bool apart = false;   // some column's second factor is not 1
        // A numerator enters the product as e * scale * unit, with a power of two for each column that puts the largest so far near 2^4: e <=
        // 2^kRise then keeps them below fp16's range, and what is dropped is below 2^-29 of the largest.  units: the largest of the lane's
        float unit[NT][2], weight[NT][2], units = 0x1p120f;
#pragma unroll
        for (int i = 0; i < NT; i++) {
#pragma unroll
            for (int k = 0; k < 2; k++) {
                mx[i][k] = kLowest, sum[i][k] = 0.f, unit[i][k] = units, weight[i][k] = 0.f;
                const float2 worth = sh.alpha[i * 8 + 2 * t + k];
                alpha[i][k] = worth.x;
                apart |= worth.y != 1.f;
            }
#pragma unroll
            for (int r = 0; r < D / 16; r++)
#pragma unroll
                for (int k = 0; k < 4; k++) o[r][i][k] = 0.f;
        }

        apart = __any_sync(0xffffffffu, apart);
        int stage = 0;
        for (int tile = first; tile < tile1; tile += step, stage = (stage + 1) % kStages) {
            wait_copies<kStages - 2>();
            __syncwarp();   // (every lane's copies; and the stage before this one has been read)
            fetch((stage + kStages - 1) % kStages, tile + (kStages - 1) * step, next_pages);
            next_pages = pages_of(table, tile + kStages * step, tile1);
            const uint32_t here = there >> (TT * stage) & ((1u << TT) - 1);
            if (!here) continue;
            const unsigned char *src = sh.ring[warp][stage];
            // ---- scores
            float x[TT][NT][4], vs[TT][G][2];
            uint32_t kw[TT][2][J];
#pragma unroll
            for (int u = 0; u < TT; u++)
#pragma unroll
                for (int r = 0; r < 2; r++) {
                    const unsigned char *at = src + u * L::BYTES + (g + 8 * r) * (D / 2) + t * (D / 8);
                    if constexpr (J == 4) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(at);
                        kw[u][r][0] = v.x, kw[u][r][1] = v.y, kw[u][r][2] = v.z, kw[u][r][3] = v.w;
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2 *>(at);
                        kw[u][r][0] = v.x, kw[u][r][1] = v.y;
                    }
                }
#pragma unroll
            for (int gi = 0; gi < G; gi++) {
                float acc[TT][NT][4];
                float ks[TT][2];
                Pair z[TT][2];
#pragma unroll
                for (int u = 0; u < TT; u++) {
#pragma unroll
                    for (int r = 0; r < 2; r++) {
                        const uint32_t word = reinterpret_cast<const uint32_t *>(src + u * L::BYTES + L::SCALES)[gi * 16 + g + 8 * r];
                        ks[u][r] = __uint_as_float(word << 16);
                        vs[u][gi][r] = __uint_as_float(word & 0xffff0000u);
                        z[u][r] = zero_twice(src[u * L::BYTES + L::KZ + gi * 16 + g + 8 * r]);
                    }
#pragma unroll
                    for (int i = 0; i < NT; i++)
#pragma unroll
                        for (int k = 0; k < 4; k++) acc[u][i][k] = 0.f;
                }
#pragma unroll
                for (int j = gi * J / G; j < (gi + 1) * J / G; j++) {
#pragma unroll
                    for (int u = 0; u < TT; u++) {
                        const uint32_t w0 = kw[u][0][j], w1 = kw[u][1][j], x0 = w0 >> 8, x1 = w1 >> 8;
                        const uint32_t c0[4] = {low(w0, base, z[u][0]), low(w1, base, z[u][1]), high(w0, base, z[u][0]), high(w1, base, z[u][1])};
                        const uint32_t c1[4] = {low(x0, base, z[u][0]), low(x1, base, z[u][1]), high(x0, base, z[u][0]), high(x1, base, z[u][1])};
#pragma unroll
                        for (int i = 0; i < NT; i++) {
                            const uint4 qh = *reinterpret_cast<const uint4 *>(sh.q[i][j][0][lane]), ql = *reinterpret_cast<const uint4 *>(sh.q[i][j][1][lane]);
                            mma(acc[u][i], c0, ql.x, ql.y);
                            mma(acc[u][i], c1, ql.z, ql.w);
                            mma(acc[u][i], c0, qh.x, qh.y);
                            mma(acc[u][i], c1, qh.z, qh.w);
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < TT; u++)
#pragma unroll
                    for (int i = 0; i < NT; i++)
#pragma unroll
                        for (int k = 0; k < 4; k++) {
                            const float v = acc[u][i][k] * alpha[i][k & 1];
                            x[u][i][k] = gi ? fmaf(v, ks[u][k >> 1], x[u][i][k]) : v * ks[u][k >> 1];
                        }
            }
            if (apart) {
#pragma unroll
                for (int u = 0; u < TT; u++)
#pragma unroll
                    for (int i = 0; i < NT; i++)
#pragma unroll
                        for (int k = 0; k < 4; k++) x[u][i][k] *= sh.alpha[i * 8 + 2 * t + (k & 1)].y;
            }
            // ---- masks
            uint32_t hidden = 0;   // bit 4 (u NT + i) + k
            const bool masked = old - tile * 16 < 16 * TT || here != (1u << TT) - 1;
            if (masked) {
#pragma unroll
                for (int u = 0; u < TT; u++)
#pragma unroll
                    for (int i = 0; i < NT; i++)
#pragma unroll
                        for (int k = 0; k < 4; k++) {
                            const int p = (tile + u) * 16 + g + 8 * (k >> 1);
                            const uint32_t j = (uint32_t)p - (uint32_t)old;   // (past the old ones: which of the new)
                            const bool seen = (here >> u & 1) && (p < limit[i][k & 1] || (j < 16u && bits[i][k & 1] >> j & 1));
                            if (!seen) hidden |= 1u << (4 * (u * NT + i) + k), x[u][i][k] = -INFINITY;
                        }
            }
            // ---- a new maximum, or a new unit, where some score (or scale) is far above the last: seldom
            float v[TT][2], vmost = 0.f;   // the tokens' largest scales
#pragma unroll
            for (int u = 0; u < TT; u++)
#pragma unroll
                for (int r = 0; r < 2; r++) {
                    v[u][r] = vs[u][0][r];
#pragma unroll
                    for (int gi = 1; gi < G; gi++) v[u][r] = fmaxf(v[u][r], vs[u][gi][r]);
                    vmost = fmaxf(vmost, v[u][r]);
                }
            bool rise = masked || vmost * units > 65000.f / (1 << kRise);
#pragma unroll
            for (int i = 0; i < NT; i++)
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    float top = fmaxf(x[0][i][k], x[0][i][k + 2]);
#pragma unroll
                    for (int u = 1; u < TT; u++) top = fmaxf(top, fmaxf(x[u][i][k], x[u][i][k + 2]));
                    rise |= top > mx[i][k] + (float)kRise;
                }
            if (__any_sync(0xffffffffu, rise)) {
                units = 0.f;
#pragma unroll
                for (int i = 0; i < NT; i++)
#pragma unroll
                    for (int k = 0; k < 2; k++) {
                        float top = mx[i][k], most = 0.f;
#pragma unroll
                        for (int u = 0; u < TT; u++) top = fmaxf(top, fmaxf(x[u][i][k], x[u][i][k + 2]));
#pragma unroll
                        for (int s = 4; s < 32; s <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
                        // (what a column does not see changes neither its maximum nor its unit)
#pragma unroll
                        for (int u = 0; u < TT; u++)
#pragma unroll
                            for (int r = 0; r < 2; r++)
                                if (!(hidden >> (4 * (u * NT + i) + k + 2 * r) & 1)) most = fmaxf(most, ex2(x[u][i][k + 2 * r] - top) * v[u][r]);
#pragma unroll
                        for (int s = 4; s < 32; s <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
                        float shift = mx[i][k] - top;
                        const float f1 = ex2(shift);
                        mx[i][k] = top;
                        sum[i][k] *= f1;
                        weight[i][k] = fmaxf(weight[i][k] * f1, most);
                        if (weight[i][k] > 0.f && weight[i][k] <= -kLowest) {
                            const int next = 4 + 127 - max((int)(__float_as_uint(weight[i][k]) >> 23), 11), last = (int)(__float_as_uint(unit[i][k]) >> 23) - 127;
                            shift += (float)(next - last);
                            unit[i][k] = power(next);
                        }
                        units = fmaxf(units, unit[i][k]);
                        const float f0 = ex2(shift);
#pragma unroll
                        for (int r = 0; r < D / 16; r++) o[r][i][k] *= f0, o[r][i][k + 2] *= f0;
                    }
            }
            // ---- numerators
#pragma unroll
            for (int u = 0; u < TT; u++)
#pragma unroll
                for (int i = 0; i < NT; i++)
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        x[u][i][k] = ex2(x[u][i][k] - mx[i][k & 1]);
                        sum[i][k & 1] += x[u][i][k];
                    }
            // ---- outputs
#pragma unroll
            for (int u = 0; u < TT; u++) {
                const unsigned char *at = src + u * L::BYTES;
                uint32_t vw[W][4];
#pragma unroll
                for (int w = 0; w < W; w++) {
                    const uint4 q = *reinterpret_cast<const uint4 *>(at + L::V + w * 512 + lane * 16);
                    vw[w][0] = q.x, vw[w][1] = q.y, vw[w][2] = q.z, vw[w][3] = q.w;
                }
#pragma unroll
                for (int gi = 0; gi < G; gi++) {
                    uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
                    for (int i = 0; i < NT; i++) {
                        float y[4];
#pragma unroll
                        for (int k = 0; k < 4; k++) y[k] = x[u][i][k] * (vs[u][gi][k >> 1] * unit[i][k & 1]);
                        if (masked) {   // (0 times a scale that is not finite)
#pragma unroll
                            for (int k = 0; k < 4; k++)
                                if (hidden >> (4 * (u * NT + i) + k) & 1) y[k] = 0.f;
                        }
                        ph[i][0] = pack(y[0], y[1]);
                        ph[i][1] = pack(y[2], y[3]);
                        pl[i][0] = transpose(pack_rest(y[0], y[1], ph[i][0]));
                        pl[i][1] = transpose(pack_rest(y[2], y[3], ph[i][1]));
                        ph[i][0] = transpose(ph[i][0]);
                        ph[i][1] = transpose(ph[i][1]);
                    }
                    // zero points of tokens 2 t, 2 t + 1 and those 8 after them.  Codes enter less their zero points: beside sums of 64 + c and of 64 + z, taken off
                    // one another at the end, what the codes stand for would lose bits to sums ten times as large and more
                    Pair z[2];
#pragma unroll
                    for (int r = 0; r < 2; r++) z[r] = zeros(*reinterpret_cast<const uint16_t *>(at + L::VZ + gi * 16 + 8 * r + 2 * t));
#pragma unroll
                    for (int r16 = gi * (D / 16) / G; r16 < (gi + 1) * (D / 16) / G; r16++) {
                        const int w = r16 / 4, q = r16 % 4;   // nibbles 2 q, 2 q + 1 of the words
                        uint32_t av[4];
#pragma unroll
                        for (int r = 0; r < 2; r++) {
                            const uint32_t y = __byte_perm(vw[w][2 * r], vw[w][2 * r + 1], q < 2 ? 0x5410 : 0x7632);
                            av[2 * r] = low(q & 1 ? y >> 8 : y, base, z[r]);
                            av[2 * r + 1] = high(q & 1 ? y >> 8 : y, base, z[r]);
                        }
#pragma unroll
                        for (int i = 0; i < NT; i++) {
                            mma(o[r16][i], av, ph[i][0], ph[i][1]);
                            mma(o[r16][i], av, pl[i][0], pl[i][1]);
                        }
                    }
                }
            }
        }
        wait_copies<0>();
        const bool all = RUNS ? f.off == 0 && tile1 == f.n : a.share == 1;
        const int off = f.off, seg = f.seg;
        if (RUNS) {
            if (tid == 0 && !all) {
                if (off) a.head[blockIdx.x].z = tile1 == f.n ? 2 : 1;
                else a.head[blockIdx.x].x = b, a.head[blockIdx.x].y = seg;
            }
        }

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
        if (RUNS) {
            left -= tile1 - off;
            f.off = 0;
            if (++f.seg == a.c.Hkv * a.blocks) f.seg = 0, f.b++;
            if (left > 0) {
                f.n = sh.plan.tiles(a, f.b);
                read_ahead(now);   // (while the parts meet)
            }
        }
        __syncthreads();
        float *part = a.part + (size_t)(2 * blockIdx.x + (off == 0)) * C * (D + 4);
        const int rank = RUNS ? 0 : blockIdx.x % a.share, chunk = RUNS ? 1 : (C * (D / 4) + a.share - 1) / a.share;   // results that a block of a cluster joins
        if (!RUNS && a.share > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
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
            } else if (!RUNS) {
                cg::cluster_group cluster = cg::this_cluster();
                const int to = idx / chunk, at = idx - to * chunk;
                *cluster.map_shared_rank(&sh.in_y[rank * chunk + at], to) = y;
                if (d == 0 || at == 0) *cluster.map_shared_rank(&sh.in_ml[rank][c], to) = make_float2(top, total);
            } else {
                *reinterpret_cast<float4 *>(part + c * (D + 4) + d) = y;
                if (d == 0) *reinterpret_cast<float2 *>(part + c * (D + 4) + D) = make_float2(top, total);
            }
        }
        if (!RUNS && a.share > 1) {
            cg::this_cluster().sync();   // (the last touch of another block's memory lies before it)
            const int idx = rank * chunk + tid, c = idx / (D / 4), d = idx % (D / 4) * 4, rho = pair0 + c;
            if (tid < chunk && idx < C * (D / 4) && rho < a.rows * a.heads) {
                float top = kLowest, total = 0.f;
                float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int r = 0; r < a.share; r++) top = fmaxf(top, sh.in_ml[r][c].x);
                for (int r = 0; r < a.share; r++) {
                    const float f1 = ex2(sh.in_ml[r][c].x - top);
                    total = fmaf(f1, sh.in_ml[r][c].y, total);
                    add4(y, f1, sh.in_y[r * chunk + tid]);
                }
                store_out<D, T>(a, b, h, rho, d, n, y, total);
            }
        }
        if (!RUNS) return;
        __syncthreads();
    }
}

// One block: the segment that block blockIdx.x of the runs began and left; the parts are added in the order of the tiles.  A thread has four dimensions of a
// column; with a grid of as many blocks high as there are columns, a block has one column and its threads share the parts (few segments of
// many parts).
template <int D, int NT, bool F32> __global__ void __launch_bounds__(kAttnThreads) join_kernel(const AttnArgs a) {
    constexpr int C = 8 * NT, LANES = D / 4, GROUPS = kAttnThreads / LANES, GRID = grid_of(NT);
    using T = std::conditional_t<F32, float, __nv_bfloat16>;
    __shared__ int slot[GRID + 1];
    __shared__ int parts_of;
    __shared__ float4 ys[GROUPS][LANES];
    __shared__ float2 mls[GROUPS];
    const int tid = threadIdx.x, lane = tid & 31;
    pdl_wait();
    pdl_trigger();
    const int4 head = a.head[blockIdx.x];
    if (tid < 32) {
        int parts = 1;
        if (lane == 0) slot[0] = 2 * blockIdx.x + 1;
        for (int i0 = blockIdx.x + 1; i0 < GRID; i0 += 32) {
            const int does = i0 + lane < GRID ? a.head[i0 + lane].z : 0;
            if (head.x < 0) break;
            const uint32_t ends = __ballot_sync(0xffffffffu, does == 2), upto = ends ? (ends & -ends) * 2 - 1 : 0xffffffffu;
            const uint32_t some = __ballot_sync(0xffffffffu, does != 0) & upto;
            if (some >> lane & 1) slot[parts + __popc(some & ((1u << lane) - 1))] = 2 * (i0 + lane);
            parts += __popc(some);
            if (ends) break;
        }
        if (lane == 0) parts_of = parts;
    }
    if (head.x < 0) return;
    __syncthreads();
    const int parts = parts_of, b = head.x, seg = head.y, pair0 = seg % a.blocks * C;
    const bool apart = gridDim.y > 1;
    const int from = apart ? tid / LANES : 0, by = apart ? GROUPS : 1;
    for (int idx = apart ? blockIdx.y * LANES + tid % LANES : tid; idx < C * LANES; idx += apart ? C * LANES : kAttnThreads) {
        const int c = idx / LANES, d = idx % LANES * 4, rho = pair0 + c;
        if (rho >= a.rows * a.heads) break;
        float top = kLowest, sum = 0.f;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](float2 ml, float4 part) {
            const float last = top;
            top = fmaxf(top, ml.x);
            const float keep = ex2(last - top), f = ex2(ml.x - top);
            sum = fmaf(f, ml.y, sum * keep);
            y = make_float4(y.x * keep, y.y * keep, y.z * keep, y.w * keep);
            add4(y, f, part);
        };
#pragma unroll 4
        for (int k = from; k < parts; k += by) {
            const float *p = a.part + ((size_t)slot[k] * C + c) * (D + 4);
            add(*reinterpret_cast<const float2 *>(p + D), *reinterpret_cast<const float4 *>(p + d));
        }
        if (apart) {
            ys[tid / LANES][tid % LANES] = y;
            if (tid % LANES == 0) mls[tid / LANES] = make_float2(top, sum);
            __syncthreads();
            if (tid >= LANES) break;
            for (int k = 1; k < GROUPS; k++) add(mls[k], ys[k][tid]);
        }
        store_out<D, T>(a, b, seg / a.blocks, rho, d, rows_of(a, b), y, sum);
    }
}

// ---------------------------------------------------------------------------------- launches
// Whether the call's columns, segments and tiles stay in the kernels' integers (a run's ends are tiles times blocks in 64 bits).
bool countable(const eesd_kv4 *c, const eesd_kv4_rows *r, int n_heads) {
    const double columns = (double)r->rows * n_heads, tiles = (double)r->max_pages * (c->page_tokens / 16);
    return columns <= 0x1p30 && tiles * columns * r->B <= 0x1p50;
}

// How a call is shared out: column tiles a block takes at once, blocks of a cluster (0: runs). A unit: a tile for 8 columns.
//   clusters  as many blocks of a cluster as fit at once, less what leaves the rounds of tiles as they are. A round of a block's warps takes 1.2 us
//             (64 dimensions: half of it), and the second kernel of the runs, with what it reads, 6 us, and a segment's start and end in a run 2.4:
//             clusters where those are more than the rounds beyond an even share (several sequences: three quarters of it, their lengths differ). 70B
//             shape, one row, 4097 tokens: 9.8 us, by runs 14.1; 16384: 17.1 and 17.0; 32768: 29 and 23; 4 x 8192 tokens: 18 and 25; 13B shape, 13 rows,
//             4000 tokens: 23 and 27; 32 x 300 tokens of the 70B shape: 8.6 and 11.8. (Near the border it errs: 2 rows on 4 x 8192 31, by runs 35)
//   runs      two column tiles at once where there are many units and no tile stays empty: codes are read and expanded once for both (a tile takes a
//             multiprocessor 160 ns instead of 2 x 99), but with one block a multiprocessor what comes before and after takes 2 us more. 16
//             rows x 8 heads on 32768 tokens: 143 instead of 176 us; 2 rows on 4 x 8192: 34 and 35
struct Way { int nt, share; };
// clusters of so many blocks that the machine holds at once, two blocks a multiprocessor (cudaOccupancyMaxActiveClusters)
constexpr int kFit[kMaxShare + 1] = {0, 296, 148, 93, 71, 56, 45, 37, 33, 30, 26, 21, 21, 17, 14, 14, 14};
Way way_of(const eesd_kv4 *c, const eesd_kv4_rows *r, int n_heads) {
    const int64_t columns = (int64_t)(n_heads / c->n_kv_heads) * r->rows, tiles = (int64_t)r->max_pages * (c->page_tokens / 16), blocks = (columns + 7) / 8;
    const int64_t segments = (int64_t)r->B * c->n_kv_heads * blocks, units = segments * tiles;
    int most = kMaxShare;
    while (most > 1 && kFit[most] < segments) most--;
    const int64_t rounds = (tiles + kWarps * most - 1) / (kWarps * most);
    const int64_t even = units / (kWarps * grid_of(1)) * (r->B > 1 ? 3 : 4) / 4;
    const int64_t turns = (segments + grid_of(1) - 1) / grid_of(1);   // of segments, past what fits at once
    if (turns * rounds <= even + 640 / c->head_dim + 2 * segments / grid_of(1)) return Way{1, (int)((tiles + kWarps * rounds - 1) / (kWarps * rounds))};
    return Way{blocks % 2 == 0 && units > 256 * grid_of(1) ? 2 : 1, 0};
}

// Whether a launch holds the clusters' blocks.
bool launchable(const eesd_kv4 *c, const eesd_kv4_rows *r, int n_heads, const Way &w) {
    const int64_t blocks = ((int64_t)(n_heads / c->n_kv_heads) * r->rows + 7) / 8;
    return (double)r->B * c->n_kv_heads * blocks * w.share <= 2147483647.0;
}

size_t scratch_of(const eesd_kv4 *c, const Way &w) { return w.share ? 0 : (size_t)grid_of(w.nt) * (16 + 2 * 8 * w.nt * (c->head_dim + 4) * 4); }

template <int D, int G, int NT, int TT, bool RUNS, bool F32> cudaError_t launch(cudaStream_t s, const AttnArgs &a, int64_t segments) {
    constexpr int kSmem = sizeof(Shared<D, G, NT, TT>) - (RUNS ? 0 : sizeof(Plan));
    auto kernel = attend_kernel<D, G, NT, TT, RUNS, F32>;
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev > 63 || !(done.load(std::memory_order_acquire) >> dev & 1)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e == cudaSuccess && !RUNS) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        if (dev <= 63) done.fetch_or(1ull << dev, std::memory_order_release);
    }
    if (RUNS) {
        launch_k(kernel, dim3(grid_of(NT)), dim3(kAttnThreads), kSmem, s, pdl_enabled(), a);
        launch_k(join_kernel<D, NT, F32>, dim3(grid_of(NT), segments * 16 < grid_of(NT) ? 8 * NT : 1), dim3(kAttnThreads), 0, s, pdl_enabled(), a);
        return cudaGetLastError();
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned int)(segments * a.share));
    cfg.blockDim = dim3(kAttnThreads);
    cfg.dynamicSmemBytes = kSmem;
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
    return cudaLaunchKernelEx(&cfg, kernel, a);
}
template <int D, int G, bool F32> cudaError_t launch_kind(cudaStream_t s, const AttnArgs &a, int nt, int64_t segments) {
    if (a.share) return launch<D, G, 1, 1, false, F32>(s, a, segments);
    return nt == 1 ? launch<D, G, 1, 2, true, F32>(s, a, segments) : launch<D, G, 2, 2, true, F32>(s, a, segments);
}
template <int D, int G> cudaError_t launch_type(cudaStream_t s, const AttnArgs &a, bool f32, int nt, int64_t segments) {
    return f32 ? launch_kind<D, G, true>(s, a, nt, segments) : launch_kind<D, G, false>(s, a, nt, segments);
}

}  // namespace kv4
}  // namespace eesd

using namespace eesd;

extern "C" {

size_t eesd_kv4_attend_scratch_bytes(const eesd_kv4 *c, const eesd_kv4_rows *r, int n_heads) {
    eesd_kv4_layout l;
    if (eesd_kv4_layout_of(c, &l) || !r || r->B < 1 || r->max_pages < 1 || r->rows < 1 || r->rows > EESD_MAX_ROWS) return 0;
    if (n_heads < 1 || n_heads % c->n_kv_heads || !kv4::countable(c, r, n_heads)) return 0;
    return kv4::scratch_of(c, kv4::way_of(c, r, n_heads));
}

int eesd_kv4_attend(void *cuda_stream, const eesd_kv4 *c, const void *pool, size_t pool_bytes, const eesd_kv4_attention *call) {
    if (!call) return EESD_ERR_BADARG;
    const eesd_kv4_rows *r = &call->rows;
    const int dtype = call->dtype, n_heads = call->n_heads;
    kv4::AttnArgs a = {};
    eesd_kv4_layout l;
    int st = kv4_open(c, pool, pool_bytes, r, &a.c, &l);
    if (st) return st;
    if (!r->at || (dtype != EESD_F32 && dtype != EESD_BF16) || r->rows > EESD_MAX_ROWS || n_heads < 1 || n_heads % c->n_kv_heads) return EESD_ERR_BADARG;
    if ((st = kv4_rows_check(&call->q, dtype))) return st;
    if (!call->out || ((uintptr_t)call->out & 15) || ((uintptr_t)call->visible & 3) || !(call->scale > 0.f) || !(call->scale <= 3.402823466e38f)) return EESD_ERR_BADARG;
    if (!kv4::countable(c, r, n_heads)) return EESD_ERR_UNSUPPORTED;
    const kv4::Way w = kv4::way_of(c, r, n_heads);
    if (!kv4::launchable(c, r, n_heads, w)) return EESD_ERR_UNSUPPORTED;
    if (const size_t need = kv4::scratch_of(c, w)) {
        if (!call->scratch || ((uintptr_t)call->scratch & 15)) return EESD_ERR_BADARG;
        if (call->scratch_bytes < need) return EESD_ERR_NOMEM;
    }
    a.n_ctx = r->at;
    a.n_rows = r->n_rows;
    a.positions = r->positions;
    a.visible = call->visible;
    a.rope = r->rope;
    a.n_rope = r->n_rope;
    a.q = call->q.data;
    a.qs[0] = call->q.stride_b, a.qs[1] = call->q.stride_row, a.qs[2] = call->q.stride_head;
    a.out = call->out;
    a.scale2 = (float)frexp((double)call->scale * 1.4426950408889634, &a.scale_exp);
    a.B = r->B;
    a.rows = r->rows;
    a.heads = n_heads / c->n_kv_heads;
    a.blocks = (int)(((int64_t)a.heads * r->rows + 8 * w.nt - 1) / (8 * w.nt));
    a.share = w.share;
    a.wide = (double)r->max_pages * (c->page_tokens / 16) * r->B * c->n_kv_heads * a.blocks >= 2147483648.0;
    const uintptr_t es = dtype == EESD_F32 ? 4 : 2;
    a.pairs = (uintptr_t)call->q.data % (2 * es) == 0 && ((call->q.stride_b | call->q.stride_row | call->q.stride_head) & 1) == 0;
    a.head = (int4 *)call->scratch;
    a.part = (float *)(a.head + kv4::grid_of(w.nt));
    const int64_t segments = (int64_t)r->B * c->n_kv_heads * a.blocks;
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
