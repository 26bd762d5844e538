// Key / value cache in 4 bits: rows quantised as they are written, and read back (sm_100a).
//
//   group of a head's values w:  s = bf16((hi - lo) / 15), z = rn(-lo / s), c = rn(w / s) + z;  value = (c - z) s
//
// Storage: tiles of 16 tokens of one head (Tile), laid out so that a lane of attention's matrix instructions finds its share of a tile in 8- or 16-byte
// pieces: keys as the rows of 16 tokens x 32 dimensions (bytes), values as the rows of 16 dimensions x 16 tokens (fp16).
#include "kernels.cuh"
#include "kv4.cuh"
#include "quant4.cuh"

namespace eesd {
namespace kv4 {

constexpr int kThreads = 256;

struct Rows {
    const int32_t *at, *n_rows;
    int rows, tiles;   // tiles: those that a sequence's rows may touch
};

// bf16((hi + down) / 15) of hi, down >= 0, to nearest, ties to even: round_range without 64 bits.  The product with 1 / 15 gives the scale or its
// neighbour; the exact sum (its rounding error beside it) against 15 times the borders, which are fp32 numbers, tells.  Sums whose borders
// might not be are left to round_range.
__device__ __forceinline__ float range_scale(float hi, float down) {
    const float sum = __fadd_rn(hi, down);
    if (!(sum >= 0x1p-90f && sum <= 0x1p120f)) return round_range(hi, -down, EESD_BF16);
    const float part = __fsub_rn(sum, hi), lost = __fadd_rn(__fsub_rn(hi, __fsub_rn(sum, part)), __fsub_rn(down, part));
    const uint32_t bits = __float_as_uint(__fmul_rn(sum, 1.f / 15.f)), near = bits + 0x7fffu + (bits >> 16 & 1) & 0xffff0000u;
    auto side = [&](uint32_t border) {   // > 0: the sum lies above 15 times the border
        const float d = __fsub_rn(sum, __fmul_rn(15.f, __uint_as_float(border)));
        return d != 0.f ? d : lost;
    };
    const float above = side(near + 0x8000u), below = side(near - 0x8000u);
    const bool odd = near & 0x10000u;
    if (above > 0.f || (above == 0.f && odd)) return __uint_as_float(near + 0x10000u);
    if (below < 0.f || (below == 0.f && odd)) return __uint_as_float(near - 0x10000u);
    return __uint_as_float(near);
}
__device__ __forceinline__ float reciprocal(float x) {   // within 2 units in the last place
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// N neighbouring values of a row
template <int N, typename T> __device__ __forceinline__ void load(const T *p, bool vec, float (&x)[N]) {
    if (vec) {
        if constexpr (sizeof(T) == 4 && N == 4) {
            const float4 v = __ldcs(reinterpret_cast<const float4 *>(p));
            x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
        } else if constexpr (sizeof(T) == 4) {
            const float2 v = __ldcs(reinterpret_cast<const float2 *>(p));
            x[0] = v.x, x[1] = v.y;
        } else {
            uint32_t w[N / 2];
            if constexpr (N == 4) {
                const uint2 v = __ldcs(reinterpret_cast<const uint2 *>(p));
                w[0] = v.x, w[1] = v.y;
            } else {
                w[0] = __ldcs(reinterpret_cast<const uint32_t *>(p));
            }
#pragma unroll
            for (int i = 0; i < N / 2; i++) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = to_f(p[i]);
    }
}

struct AppendArgs {
    Cache c;
    Rows r;
    const void *k, *v;
    int64_t ks[3], vs[3];
    const float *rope;
    const int32_t *positions;
    int n_rope;
    bool vec;
};

// One block: a tile of 16 tokens of one head, as far as the call's rows fill it; one warp the keys and values of two tokens (four tasks), N = D / 32
// neighbours a lane.  The tasks' extremes are found together, the tasks halved among the lanes at each exchange, so that a group's scale is worked
// out once, beside the others' (a task by itself, every lane its scale: 57 us instead of 28 for 5100 rows of 8 heads of 128, bf16).  Codes by the reciprocal,
// settled by the remainder (as in w4.cu).  They meet in shared memory and go out as the tile's bytes, whole where the tile is.
// 32 MB in 27 us: the issue slots bound it (80 % used, 250 instructions a row's keys or values), not memory (4.9 us).  Six blocks a multiprocessor
// (left to itself five, 1.5 us more; eight the same).
template <int D, int G, typename T> __global__ void __launch_bounds__(kThreads, 6) append_kernel(const AppendArgs a) {
    constexpr int N = D / 32, GL = 32 / G;   // GL: lanes of a group
    using L = Tile<D, G>;
    __shared__ __align__(16) unsigned char tile[L::BYTES];
    __shared__ float4 table[kThreads / 32][4][G];   // {s, 1 / s, 1.5 * 2^23 + z, s / 2: the remainder that is looked at} of each task and group
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned int blk = blockIdx.x;
    const int h = blk % a.c.Hkv;
    blk /= a.c.Hkv;
    const int x = blk % a.r.tiles, b = blk / a.r.tiles;
    const int64_t start = a.r.at[b], ti = (start >> 4) + x;   // (>> rounds down)
    const int n = a.r.n_rows ? min(max(a.r.n_rows[b], 0), a.r.rows) : a.r.rows;
    const int64_t first = start - ti * 16, past = first + n;   // the rows' places in the tile
    const int lo = first > 0 ? (int)first : 0, hi = past < 16 ? (int)past : 16;
    if (ti < 0 || lo >= hi) return;
    unsigned char *dst = tile_at(a.c, b, h, ti, L::BYTES);
    if (!dst) return;
    constexpr float M = 12582912.f;   // 1.5 * 2^23
    constexpr uint32_t MB = 0x4b400000u;
    const int tok0 = lo + 2 * warp, left = hi - tok0;   // the warp's tokens: min(left, 2)
    if (left > 0) {
        float w[4][N];   // tasks: keys, keys, values, values
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int m = (int)(tok0 + (i & 1 && left > 1) - first);   // (a token that is not there: the first again)
            const int64_t *st = i < 2 ? a.ks : a.vs;
            load<N>((const T *)(i < 2 ? a.k : a.v) + b * st[0] + m * st[1] + h * st[2] + lane * N, a.vec, w[i]);
        }
        if (a.rope) {
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const int tok = tok0 + (i && left > 1);
                const int64_t pos = a.positions ? (int64_t)a.positions[(int64_t)b * a.r.rows + (tok - first)] : ti * 16 + tok;
                const int64_t row = min(max(pos, (int64_t)0), (int64_t)(a.n_rope - 1));
                const float2 *cs = reinterpret_cast<const float2 *>(a.rope) + row * (D / 2) + lane * (N / 2);
#pragma unroll
                for (int j = 0; j < N / 2; j++) {
                    const float2 y = turn(w[i][2 * j], w[i][2 * j + 1], cs[j]);
                    w[i][2 * j] = y.x, w[i][2 * j + 1] = y.y;
                }
            }
        }
        // extremes: e[task] the largest, e[4 + task] the least turned over; afterwards the lane has that of task (lane >> 1 & 1) * 2 + (lane >> 2 & 1), the largest
        // where its bit 0 is not set
        float e[8];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            e[i] = e[4 + i] = 0.f;
#pragma unroll
            for (int j = 0; j < N; j++) e[i] = max_nan(e[i], w[i][j]), e[4 + i] = max_nan(e[4 + i], -w[i][j]);
        }
#pragma unroll
        for (int s = 0; s < 3; s++) {
            const bool up = lane >> s & 1;
#pragma unroll
            for (int i = 0; i < 4 >> s; i++) {
                const float send = up ? e[i] : e[i + (4 >> s)], keep = up ? e[i + (4 >> s)] : e[i];
                e[i] = max_nan(keep, __shfl_xor_sync(0xffffffffu, send, 1 << s));
            }
        }
#pragma unroll
        for (int o = 8; o < GL; o <<= 1) e[0] = max_nan(e[0], __shfl_xor_sync(0xffffffffu, e[0], o));
        {
            const float other = __shfl_xor_sync(0xffffffffu, e[0], 1);
            const float most = lane & 1 ? other : e[0], least = lane & 1 ? e[0] : other;   // (least: turned over)
            float s = range_scale(most, least);
            if (!(most <= 3.402823466e38f) || !(least <= 3.402823466e38f)) s = __uint_as_float(0x7fc00000u);
            const bool plain = s > 0.f, fine = s >= 0x1p-90f;   // plain: neither 0 nor NaN
            const float inv = fine ? reciprocal(s) : 0.f;
            float z = 0.f;
            if (fine) {
                float q = __fmaf_rn(least, inv, M);
                const float rem = __fmaf_rn(M - q, s, least);
                const bool odd = __float_as_int(q) & 1;
                if (rem > 0.5f * s || (rem == 0.5f * s && odd)) q += 1.f;
                else if (-rem > 0.5f * s || (-rem == 0.5f * s && odd)) q -= 1.f;
                z = fminf(q - M, 15.f);
            } else if (plain) {
                z = fminf(nearest_quotient(least, s), 15.f);
            }
            const int task = (lane >> 1 & 1) * 2 + (lane >> 2 & 1), gi = lane / GL;
            if (lane % GL < 8 && !(lane & 1)) {
                table[warp][task][gi] = make_float4(plain ? s : 1.f, inv, M + z, fine ? 0.5f * s : plain ? 0.f : 3.402823466e38f);
                const int tok = tok0 + (task & 1), is_v = task >> 1;
                if ((task & 1) < left) {
                    reinterpret_cast<uint16_t *>(tile + L::SCALES)[(gi * 16 + tok) * 2 + is_v] = __bfloat16_as_ushort(__float2bfloat16_rn(s));
                    tile[(is_v ? L::VZ : L::KZ) + gi * 16 + tok] = (unsigned char)z;
                }
            }
        }
        __syncwarp();
        const int d = lane * N, shift = 4 * (d % 64 / 8);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float4 t = table[warp][i][lane / GL];
            float y[N], rem[N], most = 0.f;
#pragma unroll
            for (int j = 0; j < N; j++) {
                y[j] = __fmaf_rn(w[i][j], t.y, t.z);   // 1.5 * 2^23 + the code
                rem[j] = __fmaf_rn(t.z - y[j], t.x, w[i][j]);
                most = fmaxf(most, fabsf(rem[j]));
            }
            if (most >= t.w) {   // a quotient at (or beside) a half: to the nearer, or the even one; or a scale whose reciprocal will not do (t.w 0)
#pragma unroll
                for (int j = 0; j < N; j++) {
                    const bool odd = (__float_as_int(y[j]) ^ __float_as_int(t.z)) & 1;
                    if (rem[j] > t.w || (rem[j] == t.w && odd)) y[j] += 1.f;
                    else if (-rem[j] > t.w || (-rem[j] == t.w && odd)) y[j] -= 1.f;
                    if (t.w == 0.f) y[j] = t.z + nearest_quotient(w[i][j], t.x);
                }
            }
            uint32_t c[N];   // MB + the code (what is not finite: 0)
#pragma unroll
            for (int j = 0; j < N; j++) c[j] = __float_as_uint(fminf(fmaxf(y[j], M), M + 15.f));
            const int tok = tok0 + (i & 1);
            if (i < 2) {
                const int at = tok * (D / 2) + d % 32 / 8 * (D / 8) + d / 32 * 4 + d % 8 / 2;
                if constexpr (N == 4) {
                    const uint32_t v = c[0] + c[1] * 16u + c[2] * 256u + c[3] * 4096u - MB * 4369u;
                    if ((i & 1) < left) *reinterpret_cast<uint16_t *>(tile + at) = (uint16_t)v;
                } else {
                    if ((i & 1) < left) tile[at] = (unsigned char)(c[0] + c[1] * 16u - MB * 17u);
                }
            } else {
                // a word takes one nibble of each of 8 lanes: N words, halved among the lanes at each exchange
                const int t2 = tok % 8 / 2, he = tok / 8 * 2 + tok % 2;
                int word;
                uint32_t v;
#pragma unroll
                for (int j = 0; j < N; j++) c[j] = (c[j] - MB) << shift;
                if constexpr (N == 4) {
                    const bool up1 = lane & 2, up2 = lane & 4;
                    uint32_t k0 = up1 ? c[2] : c[0], k1 = up1 ? c[3] : c[1];
                    k0 |= __shfl_xor_sync(0xffffffffu, up1 ? c[0] : c[2], 2);
                    k1 |= __shfl_xor_sync(0xffffffffu, up1 ? c[1] : c[3], 2);
                    v = (up2 ? k1 : k0) | __shfl_xor_sync(0xffffffffu, up2 ? k0 : k1, 4);
                    v |= __shfl_xor_sync(0xffffffffu, v, 8);
                    word = up1 * 2 + up2;
                } else {
                    const bool up = lane & 4;
                    v = (up ? c[1] : c[0]) | __shfl_xor_sync(0xffffffffu, up ? c[0] : c[1], 4);
                    v |= __shfl_xor_sync(0xffffffffu, v, 8);
                    v |= __shfl_xor_sync(0xffffffffu, v, 16);
                    word = up;
                }
                if ((N == 4 ? !(lane & 8) : !(lane & 24)) && (i & 1) < left) reinterpret_cast<uint32_t *>(tile + L::V)[((d / 64 * 8 + d % 8 + word) * 4 + t2) * 4 + he] = v;
            }
        }
    }
    __syncthreads();
    if (hi - lo == 16) {
        for (int i = threadIdx.x; i < L::BYTES / 16; i += kThreads) reinterpret_cast<uint4 *>(dst)[i] = reinterpret_cast<const uint4 *>(tile)[i];
        return;
    }
    for (int i = threadIdx.x; i < L::KZ / 4; i += kThreads) {
        const int at = i * 4;
        const int tok = at < L::V ? at / (D / 2) : at < L::SCALES ? (i & 2) * 4 + (i >> 2 & 3) * 2 + (i & 1) : i - L::SCALES / 4 & 15;
        if (tok >= lo && tok < hi) reinterpret_cast<uint32_t *>(dst)[i] = reinterpret_cast<const uint32_t *>(tile)[i];
    }
    for (int i = L::KZ + threadIdx.x; i < L::BYTES; i += kThreads)
        if ((i & 15) >= lo && (i & 15) < hi) dst[i] = tile[i];
}

struct ReadArgs {
    Cache c;
    Rows r;
    const int32_t *n_ctx;
    void *k, *v;
};

// Where 16-byte piece i of a tile stands in shared memory when a lane takes N neighbouring dimensions: the values' pieces that a warp reads together are 32 apart (dimensions
// 64 apart; N = 4: also 16), in the same banks, unless the higher bits of their number change the lowest.
template <int D, int N> __device__ __forceinline__ int piece(int i) { return i >= D / 2 && i < D ? i ^ (i - D / 2) >> (N == 8 ? 5 : 4) : i; }

// One block: kTiles neighbouring tiles of a head, brought into shared memory.  A lane takes N neighbouring values of a token's keys and of its values: 16 bytes of
// what is written.  2 x 16385 tokens of 8 heads of 128 as bf16: 32 us, 174 MB, 0.83 of the copy rate (a token a warp, N = D / 32, was 110 instructions a token and
// head, and 46 us).
template <int D, int G, int kTiles, typename T> __global__ void __launch_bounds__(kThreads) read_kernel(const ReadArgs a) {
    constexpr int N = 16 / sizeof(T), LT = D / N, TW = 32 / LT;   // lanes of a token, tokens of a warp
    using L = Tile<D, G>;
    __shared__ __align__(16) unsigned char tiles[kTiles][L::BYTES];
    __shared__ int ends[kTiles];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned int blk = blockIdx.x;
    const int h = blk % a.c.Hkv;
    blk /= a.c.Hkv;
    const int groups = (a.r.tiles + kTiles - 1) / kTiles, x = blk % groups * kTiles, b = blk / groups;
    const int64_t start = a.r.at ? a.r.at[b] : 0, ti = (start >> 4) + x, first = start - ti * 16, past = first + a.r.rows;   // (of the block's first tile)
    const int lo = first > 0 ? (int)first : 0, hi = past < 16 * kTiles ? (int)past : 16 * kTiles;
    if (lo >= hi) return;
    // a warp brings a tile (kTiles <= 8); one tile is brought by all
    const int64_t left = a.n_ctx ? (int64_t)a.n_ctx[b] - ti * 16 : 16 * kTiles;
    if (kTiles == 1 || warp < kTiles) {
        const int j = kTiles == 1 ? 0 : warp, by = kTiles == 1 ? kThreads : 32;
        const unsigned char *src = ti + j < 0 || left <= max(lo, 16 * j) || 16 * j >= hi ? nullptr : tile_at(a.c, b, h, ti + j, L::BYTES);
        if (src)
#pragma unroll 5
            for (int i = kTiles == 1 ? (int)threadIdx.x : lane; i < L::BYTES / 16; i += by)
                reinterpret_cast<uint4 *>(tiles[j])[piece<D, N>(i)] = __ldcs(reinterpret_cast<const uint4 *>(src) + i);
        if (kTiles == 1 ? threadIdx.x == 0 : lane == 0) ends[j] = src ? (int)min((int64_t)16, left - 16 * j) : 0;   // tokens that are there
    }
    __syncthreads();
    const int d = lane % LT * N, gi = d / (D / G), i = d % 64 / 8;   // i: the nibble of the values' words
    const size_t row = (size_t)a.c.Hkv * D;
    const size_t at = ((size_t)((int64_t)b * a.r.rows - first) * a.c.Hkv + h) * D + d;   // of token 0
    const int k_at = d % 32 / 8 * (D / 8) + d / 32 * 4, k_shift = 4 * (d % 8), v_at = d / 64 * 32 + d % 8 * 4, v_shift = 4 * (i & 1);
    const uint32_t v_bytes = 0x0400u + i / 2 * 0x0101u;   // byte i / 2 of two words, in the halves' low bytes
#pragma unroll 1   // (2: 36 us)
    for (int place = warp * TW + lane / LT; place < 16 * kTiles; place += TW * kThreads / 32) {
        if (place < lo || place >= hi) continue;
        const int j = place >> 4, tok = place & 15;
        const unsigned char *tile = tiles[j];
        uint4 ko = make_uint4(0, 0, 0, 0), vo = ko;   // 0 in either type
        if (tok < ends[j]) {
            const uint32_t scales = *reinterpret_cast<const uint32_t *>(tile + L::SCALES + (gi * 16 + tok) * 4);
            const uint32_t c = *reinterpret_cast<const uint32_t *>(tile + tok * (D / 2) + k_at) >> (N == 8 ? 0 : k_shift);
            // words of the lane's dimensions, 64 bytes apart
            const uint32_t *vc = reinterpret_cast<const uint32_t *>(tile + piece<D, N>(L::V / 16 + v_at + tok % 8 / 2) * 16) + tok / 8 * 2 + tok % 2;
            uint32_t v2[N / 2];   // their codes, in the lowest bits of the halves
#pragma unroll
            for (int n = 0; n < N / 2; n++) v2[n] = __byte_perm(vc[32 * n], vc[32 * n + 16], v_bytes) >> v_shift;
            if constexpr (sizeof(T) == 2) {
                // two codes at a time: 128 + c (the nibble set into the mantissa of bf16's 128) - (128 + z), times s, rounded once
                const uint32_t zk = tile[L::KZ + gi * 16 + tok] * 0x10001u | 0x43004300u, zv = tile[L::VZ + gi * 16 + tok] * 0x10001u | 0x43004300u;
                const uint32_t sk = __byte_perm(scales, 0, 0x1010), sv = __byte_perm(scales, 0, 0x3232);
                auto pair = [](uint32_t two, uint32_t z, uint32_t s) {
                    uint32_t r = two & 0x000f000fu | 0x43004300u;
                    asm("sub.rn.bf16x2 %0, %0, %1;\n\tmul.rn.bf16x2 %0, %0, %2;" : "+r"(r) : "r"(z), "r"(s));
                    return r;
                };
                const uint32_t c0 = c & 0xffffu, c1 = c >> 16;
                ko = make_uint4(pair(c0 | c0 << 12, zk, sk), pair(c0 >> 8 | c0 << 4, zk, sk), pair(c1 | c1 << 12, zk, sk), pair(c1 >> 8 | c1 << 4, zk, sk));
                vo = make_uint4(pair(v2[0], zv, sv), pair(v2[1], zv, sv), pair(v2[2], zv, sv), pair(v2[3], zv, sv));
            } else {
                const float sk = __uint_as_float(scales << 16), sv = __uint_as_float(scales & 0xffff0000u);
                const float zk = __uint_as_float(0x4b000000u | tile[L::KZ + gi * 16 + tok]), zv = __uint_as_float(0x4b000000u | tile[L::VZ + gi * 16 + tok]);
                // 2^23 + c (the code's nibble set into the mantissa) - (2^23 + z), times s
                auto value = [](uint32_t word, float z, float s) { return __float_as_uint(__fmul_rn(__uint_as_float((word & 15u) | 0x4b000000u) - z, s)); };
                ko = make_uint4(value(c, zk, sk), value(c >> 4, zk, sk), value(c >> 8, zk, sk), value(c >> 12, zk, sk));
                vo = make_uint4(value(v2[0], zv, sv), value(v2[0] >> 16, zv, sv), value(v2[1], zv, sv), value(v2[1] >> 16, zv, sv));
            }
        }
        const size_t to = at + place * row;
        if (a.k) __stcs(reinterpret_cast<uint4 *>((T *)a.k + to), ko);
        if (a.v) __stcs(reinterpret_cast<uint4 *>((T *)a.v + to), vo);
    }
}

template <typename T> void (*pick_append(int D, int G))(AppendArgs) {
    if (D == 64) return G == 1 ? append_kernel<64, 1, T> : append_kernel<64, 2, T>;
    return G == 1 ? append_kernel<128, 1, T> : G == 2 ? append_kernel<128, 2, T> : append_kernel<128, 4, T>;
}
template <int TILES, typename T> void (*pick_read(int D, int G))(ReadArgs) {
    if (D == 64) return G == 1 ? read_kernel<64, 1, TILES, T> : read_kernel<64, 2, TILES, T>;
    return G == 1 ? read_kernel<128, 1, TILES, T> : G == 2 ? read_kernel<128, 2, TILES, T> : read_kernel<128, 4, TILES, T>;
}

}  // namespace kv4

int kv4_open(const eesd_kv4 *c, const void *pool, size_t pool_bytes, const eesd_kv4_rows *r, kv4::Cache *out, eesd_kv4_layout *l) {
    const int st = eesd_kv4_layout_of(c, l);
    if (st) return st;
    if (!pool || ((uintptr_t)pool & 15) || !r || !r->page_table || r->max_pages < 1 || r->table_stride < r->max_pages || r->B < 1 || r->rows < 1) return EESD_ERR_BADARG;
    const void *const words[] = {r->page_table, r->at, r->n_rows, r->positions};
    for (const void *p : words)
        if ((uintptr_t)p & 3) return EESD_ERR_BADARG;
    if (r->rope && (((uintptr_t)r->rope & 7) || r->n_rope < 1)) return EESD_ERR_BADARG;
    if (pool_bytes < l->total_bytes) return EESD_ERR_NOMEM;
    if (r->B > EESD_KV4_MAX_BATCH) return EESD_ERR_UNSUPPORTED;
    out->pool = (unsigned char *)pool;
    out->table = r->page_table;
    out->table_stride = r->table_stride;
    out->n_pages = c->n_pages;
    out->max_pages = r->max_pages;
    out->Hkv = c->n_kv_heads;
    out->shift = c->page_tokens == 16 ? 0 : c->page_tokens == 32 ? 1 : c->page_tokens == 64 ? 2 : 3;
    return EESD_OK;
}

int kv4_rows_check(const eesd_kv4_tensor *t, int dtype) {
    if (!t || !t->data || t->stride_b < 0 || t->stride_row < 0 || t->stride_head < 0) return EESD_ERR_BADARG;
    return (uintptr_t)t->data % (dtype == EESD_F32 ? 4 : 2) ? EESD_ERR_BADARG : EESD_OK;
}

}  // namespace eesd

using namespace eesd;

namespace {
// blocks for the tiles that `rows` positions may touch, wherever they begin
bool kv4_grid(const eesd_kv4_rows *r, int Hkv, kv4::Rows *out, unsigned int *blocks) {
    out->at = r->at;
    out->n_rows = r->n_rows;
    out->rows = r->rows;
    out->tiles = (int)(((int64_t)r->rows + 14) / 16 + 1);
    const double n = (double)out->tiles * Hkv * r->B;
    if (n > 2147483647.0) return false;
    *blocks = (unsigned int)n;
    return true;
}
bool whole(const eesd_kv4_tensor *t, int n, size_t bytes) {
    return (uintptr_t)t->data % (n * bytes) == 0 && t->stride_b % n == 0 && t->stride_row % n == 0 && t->stride_head % n == 0;
}
}  // namespace

extern "C" {

int eesd_kv4_layout_of(const eesd_kv4 *c, eesd_kv4_layout *out) {
    if (!c || !out || c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535) return EESD_ERR_BADARG;
    if (c->head_dim != 64 && c->head_dim != 128) return EESD_ERR_UNSUPPORTED;
    if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return EESD_ERR_UNSUPPORTED;
    if ((c->group != 32 && c->group != 64 && c->group != 128) || c->group > c->head_dim) return EESD_ERR_UNSUPPORTED;
    const size_t D = (size_t)c->head_dim, G = D / (size_t)c->group;
    out->v_codes = 8 * D;
    out->scales = 16 * D;
    out->k_zeros = out->scales + 64 * G;
    out->v_zeros = out->k_zeros + 16 * G;
    out->tile_bytes = out->v_zeros + 16 * G;
    out->page_bytes = out->tile_bytes * (size_t)(c->page_tokens / 16) * (size_t)c->n_kv_heads;
    out->total_bytes = out->page_bytes * (size_t)c->n_pages;
    return EESD_OK;
}

int eesd_kv4_append(void *cuda_stream, const eesd_kv4 *c, void *pool, size_t pool_bytes, const eesd_kv4_rows *r, int dtype, const eesd_kv4_tensor *k,
                    const eesd_kv4_tensor *v) {
    kv4::AppendArgs a = {};
    eesd_kv4_layout l;
    int st = kv4_open(c, pool, pool_bytes, r, &a.c, &l);
    if (st) return st;
    if (!r->at || (dtype != EESD_F32 && dtype != EESD_BF16)) return EESD_ERR_BADARG;
    if ((st = kv4_rows_check(k, dtype)) || (st = kv4_rows_check(v, dtype))) return st;
    unsigned int blocks;
    if (!kv4_grid(r, c->n_kv_heads, &a.r, &blocks)) return EESD_ERR_UNSUPPORTED;
    a.k = k->data;
    a.v = v->data;
    a.ks[0] = k->stride_b, a.ks[1] = k->stride_row, a.ks[2] = k->stride_head;
    a.vs[0] = v->stride_b, a.vs[1] = v->stride_row, a.vs[2] = v->stride_head;
    a.rope = r->rope;
    a.positions = r->positions;
    a.n_rope = r->n_rope;
    const size_t es = dtype == EESD_F32 ? 4 : 2;
    a.vec = whole(k, c->head_dim / 32, es) && whole(v, c->head_dim / 32, es);
    const int G = c->head_dim / c->group;
    launch_k(dtype == EESD_F32 ? kv4::pick_append<float>(c->head_dim, G) : kv4::pick_append<__nv_bfloat16>(c->head_dim, G), dim3(blocks), dim3(kv4::kThreads), 0,
             (cudaStream_t)cuda_stream, pdl_enabled(), a);
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

int eesd_kv4_read(void *cuda_stream, const eesd_kv4 *c, const void *pool, size_t pool_bytes, const eesd_kv4_rows *r, const int32_t *n_ctx, int out_dtype, void *k,
                  void *v) {
    kv4::ReadArgs a = {};
    eesd_kv4_layout l;
    const int st = kv4_open(c, pool, pool_bytes, r, &a.c, &l);
    if (st) return st;
    if ((!k && !v) || ((uintptr_t)k & 15) || ((uintptr_t)v & 15) || ((uintptr_t)n_ctx & 3) || (out_dtype != EESD_F32 && out_dtype != EESD_BF16)) return EESD_ERR_BADARG;
    unsigned int blocks;
    if (!kv4_grid(r, c->n_kv_heads, &a.r, &blocks)) return EESD_ERR_UNSUPPORTED;
    a.n_ctx = n_ctx;
    a.k = k;
    a.v = v;
    const int G = c->head_dim / c->group;
    // eight tiles a block (its start costs as much as a tile) where that leaves every multiprocessor eight blocks: 2 x 16385 tokens of 8 heads as bf16 32 us, by single
    // tiles 43; 4 x 2047 as fp32, which would be 516 blocks, takes 3 us longer by eights
    const bool eight = blocks >= 8u * 8u * 148u;
    if (eight) blocks = (unsigned int)((a.r.tiles + 7) / 8 * (int64_t)c->n_kv_heads * r->B);
    auto kernel = out_dtype == EESD_F32 ? (eight ? kv4::pick_read<8, float>(c->head_dim, G) : kv4::pick_read<1, float>(c->head_dim, G))
                                        : (eight ? kv4::pick_read<8, __nv_bfloat16>(c->head_dim, G) : kv4::pick_read<1, __nv_bfloat16>(c->head_dim, G));
    launch_k(kernel, dim3(blocks), dim3(kv4::kThreads), 0, (cudaStream_t)cuda_stream, pdl_enabled(), a);
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}

}  // extern "C"
