// Logit rules: penalties for repeated tokens, biases and grammar masks on the logit rows of a decode or verification
// round (sm_100a).  For entry v of row i of sequence b, with n the times v was generated (history past the prompt, and the
// drafts x_1..x_i that precede the row) and `seen` telling that it was generated or is in the prompt:
//   l1 = seen ? (l > 0 ? l / repetition : l * repetition) : l
//   l2 = l1 - (n > 0 ? frequency * n + presence : 0)
//   out = allowed(v) ? l2 + bias(v) : -inf
// every operation rounded to fp32 by itself.  A quotient is the product with the rounded reciprocal, corrected once by its remainder (P.
// Markstein's method of 1990): compared with the rounded quotient for all 2^46 pairs of significands on a B200, none differs.  Where x or the
// penalty is not within 2^-60 .. 2^60, so that a step might leave the normal numbers, it is divided instead (4 columns in one branch, seldom
// taken; dividing everywhere: 76 us instead of 69 with all rules, 66 instead of 57 with penalties alone).
//
// Memory bound: 8 bytes per entry and one mask bit.  A block owns a run of the vocabulary for one sequence, counts the
// sequence's tokens that fall into it in shared memory (integer atomics: the result does not depend on their order),
// takes the counts and biases of its threads' columns into registers and then walks the rows, so that counting is paid once
// per sequence and not once per row; a draft adds to the count of the one thread that owns its column.
//
// Measured (a graph of calls over inputs that pass the L2 cache in turn; floor: bytes at the measured copy rate):
//   64 sequences x 17 rows x 32000: mask alone 51 us, penalties alone 57, all rules 69 (floor 43)
//   64 x 1 x 128256, all rules: 28.1 (floor 10.2: every block counts 2048 tokens for 4096 columns of one row)
//   16 x 5 x 50257, biases and mask: 12.3 (floor 5.0);  8 x 2 x 32000, all rules: 4.7;  1 x 1 x 32000, penalties: 3.1 (latency)
// With everything on, the one round of blocks counts first (about 7 us of dependent reads) and then streams, with two items a
// thread in flight in 64 registers; a ring of 3 spills (77 us), 3 blocks a multiprocessor make two rounds (107), and a ring of 4 in shared memory
// takes the L1 cache that masks and drafts are read through (80).
#include "../../include/eesd.h"
#include "common.cuh"
#include "kernels.cuh"

namespace eesd {
namespace rules {

constexpr int kThreads = 256;
constexpr int kSpan = kThreads * 4;         // columns a block handles at a time: four per thread
constexpr uint32_t kPrompt = 0x80000000u;   // the token is in the prompt (the other bits count the generated ones)

struct Args {
    eesd_logit_rules r;
    const float *in;
    float *out;
    size_t ld_in, ld_out;
    int rows, V, spans, spans_per_block, chunks, row_split, rows_per_block;
};

// what a block of threads works on
struct Block {
    uint32_t *count;         // per column: times generated, and kPrompt
    int *bias_at;            // 1 + place of the column's bias in the list; 0: none
    const int32_t *drafted;  // drafts from the block's first row on
    int b, col0, rows;
    size_t first;            // its first row
};

// Spans sub0 .. sub1 - 1 of the block's columns, all its rows, for one thread: `cols` of its four columns exist (WHOLE: all).
// VEC: they are neighbours, one 16-byte access a row; otherwise they lie kThreads apart.
template <bool VEC, bool WHOLE, bool PEN, bool BIAS, bool MASK> __device__ __forceinline__ void run(const Args &a, const Block &w, int sub0, int sub1, int cols) {
    constexpr int kAhead = PEN ? 2 : 4, step = VEC ? 1 : kThreads;
    const eesd_logit_rules &r = a.r;
    const int mine = (VEC ? 4 : 1) * (int)threadIdx.x, rows = w.rows, at0 = sub0 * kSpan + mine;
    const int items = (sub1 - sub0) * rows;
    if (WHOLE) cols = 4;
    const float rep = PEN && r.repetition ? __ldg(r.repetition + w.b) : 1.f, inv = __frcp_rn(rep);
    const bool near_one = rep >= 0x1p-60f && rep <= 0x1p60f;   // (else the reciprocal would not do)
    const float freq = PEN && r.frequency ? __ldg(r.frequency + w.b) : 0.f, pres = PEN && r.presence ? __ldg(r.presence + w.b) : 0.f;

    // a ring of (span, row) items, loads kAhead items ahead
    float l[kAhead][4];
    uint32_t m[kAhead][VEC ? 1 : 4];   // the mask's words as they come (a shift here would wait for the load)
    const float *src = a.in + w.first * a.ld_in + w.col0 + at0;
    const uint32_t *msrc = MASK ? (const uint32_t *)r.mask + w.first * (size_t)r.mask_stride + ((w.col0 + at0) >> 5) : nullptr;
    int fetched = 0, frow = 0;
    auto fetch = [&](int k) {
        if (fetched == items) return;
        if (VEC && WHOLE) {
            const float4 v = __ldcs(reinterpret_cast<const float4 *>(src));
            l[k][0] = v.x; l[k][1] = v.y; l[k][2] = v.z; l[k][3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) l[k][i] = i < cols ? __ldcs(src + i * step) : 0.f;
        }
        if (MASK) {
#pragma unroll
            for (int i = 0; i < (VEC ? 1 : 4); i++)
                if (i < cols) m[k][i] = __ldg(msrc + i * (step / 32));
            msrc += r.mask_stride;
        }
        src += a.ld_in;
        fetched++;
        if (++frow == rows) {   // on to the next span
            frow = 0;
            src += kSpan - (ptrdiff_t)rows * (ptrdiff_t)a.ld_in;
            if (MASK) msrc += kSpan / 32 - (ptrdiff_t)rows * (ptrdiff_t)r.mask_stride;
        }
    };
#pragma unroll
    for (int k = 0; k < kAhead; k++) fetch(k);

    // of the current span's columns: the repetition penalty (1: not seen), its reciprocal, what the other penalties take off, the bias
    float by[4], un[4], less[4], more[4];
    bool special = false;   // any but 1, 1, 0, 0
    auto state = [&](int i, int at) {
        bool any = false;
        if (PEN) {
            const uint32_t c = w.count[at], n = c & ~kPrompt;
            by[i] = c ? rep : 1.f;
            un[i] = c ? inv : 1.f;
            less[i] = n ? __fadd_rn(__fmul_rn(freq, (float)n), pres) : 0.f;
            any = c != 0;
        }
        if (BIAS) {
            const int j = w.bias_at[at];
            more[i] = j ? __ldg(r.bias_values + j - 1) : 0.f;
            any |= j != 0;
        }
        return any;
    };
    float *dst = a.out + w.first * a.ld_out + w.col0 + at0;
    int row = 0, at = at0;
    for (int done = 0; done < items;) {
#pragma unroll
        for (int k = 0; k < kAhead; k++) {
            if (done == items) break;
            if ((PEN || BIAS) && row == 0) {
                special = false;
#pragma unroll
                for (int i = 0; i < 4; i++) special |= state(i, at + i * step);
            } else if (PEN && w.drafted) {   // the draft that precedes this row
                const int off = __ldg(w.drafted + row - 1) - w.col0 - at;
                if (VEC ? (unsigned int)off < 4u : (unsigned int)off < (unsigned int)kSpan && off % kThreads == 0) {
                    ++w.count[at + off];   // (its column is this thread's own)
                    special = true;
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (i * step == off) state(i, at + off);
                }
            }
            if ((PEN || BIAS) && special) {
                if (PEN) {
                    float q[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        q[i] = l[k][i] * un[i];
                        q[i] = fmaf(fmaf(-q[i], by[i], l[k][i]), un[i], q[i]);
                    }
                    const float most = fmaxf(fmaxf(fabsf(l[k][0]), fabsf(l[k][1])), fmaxf(fabsf(l[k][2]), fabsf(l[k][3])));
                    const float least = fminf(fminf(fabsf(l[k][0]), fabsf(l[k][1])), fminf(fabsf(l[k][2]), fabsf(l[k][3])));
                    if (!(near_one && most <= 0x1p60f && least >= 0x1p-60f)) {
#pragma unroll
                        for (int i = 0; i < 4; i++) q[i] = __fdiv_rn(l[k][i], by[i]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; i++) l[k][i] = __fsub_rn(l[k][i] > 0.f ? q[i] : __fmul_rn(l[k][i], by[i]), less[i]);
                }
                if (BIAS) {
#pragma unroll
                    for (int i = 0; i < 4; i++) l[k][i] = __fadd_rn(l[k][i], more[i]);
                }
            }
            if (MASK) {
#pragma unroll
                for (int i = 0; i < 4; i++)   // (bit col % 32 of word col / 32; kThreads is a multiple of 32)
                    if (!(m[k][VEC ? 0 : i] >> ((mine & 31) + (VEC ? i : 0)) & 1u)) l[k][i] = -INFINITY;
            }
            if (VEC && WHOLE) {
                *reinterpret_cast<float4 *>(dst) = make_float4(l[k][0], l[k][1], l[k][2], l[k][3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (i < cols) dst[i * step] = l[k][i];
            }
            dst += a.ld_out;
            done++;
            if (++row == rows) {
                row = 0;
                at += kSpan;
                dst += kSpan - (ptrdiff_t)rows * (ptrdiff_t)a.ld_out;
            }
            fetch(k);
        }
    }
}

// VEC: rows are 16-byte aligned (the vocabulary's last 1 to 3 columns are accessed one by one)
template <bool VEC, bool PEN, bool BIAS, bool MASK>
__global__ void __launch_bounds__(kThreads, 4) process_kernel(const Args a) {
    extern __shared__ uint32_t smem[];
    const eesd_logit_rules &r = a.r;
    const int ncol = a.spans_per_block * kSpan, tid = threadIdx.x;
    Block w;
    w.count = smem;
    w.bias_at = (int *)(smem + (PEN ? ncol : 0));
    int job = blockIdx.x;
    w.col0 = job % a.chunks * ncol;
    job /= a.chunks;
    const int row_lo = job % a.row_split * a.rows_per_block;
    w.b = job / a.row_split;
    w.rows = min(a.rows, row_lo + a.rows_per_block) - row_lo;
    w.first = (size_t)w.b * a.rows + row_lo;
    w.drafted = r.drafted ? r.drafted + (size_t)w.b * r.drafted_stride + row_lo : nullptr;

    pdl_wait();
    pdl_trigger();
    // On their way while the sequence's tokens are counted: the block's first rows (to the L2 cache), the lengths, the first tokens (by
    // the length of the list, so that they need not wait for the sequence's).
    {
        const float *src = a.in + w.first * a.ld_in + w.col0 + tid * 4;
        if (w.col0 + tid * 4 < a.V && (tid & 7) == 0)   // (32 columns: 128 bytes)
            for (int i = 0; i < min(w.rows, 4); i++) asm volatile("prefetch.global.L2 [%0];" ::"l"(src + (size_t)i * a.ld_in));
    }
    const int32_t *h = PEN && r.history ? r.history + (size_t)w.b * r.history_stride : nullptr;
    const int len = h ? r.history_len : 0;
    constexpr int kTokens = 8;
    int tok[kTokens];
    auto tokens = [&](int base) {
#pragma unroll
        for (int u = 0; u < kTokens; u++) {
            const int i = base + u * kThreads + tid;
            tok[u] = i < len ? __ldg(h + i) : -1;
        }
    };
    tokens(0);
    int n = len, np = 0, lo = 0, hi = 0;
    if (h && r.n_history) n = __ldg(r.n_history + w.b);
    if (h && r.n_prompt) np = __ldg(r.n_prompt + w.b);
    if (BIAS) {
        lo = __ldg(r.bias_start + w.b);
        hi = __ldg(r.bias_start + w.b + 1);
    }
    for (int i = tid; i < ((PEN ? ncol : 0) + (BIAS ? ncol : 0)) / 4; i += kThreads) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
    n = min(max(n, 0), len);
    np = min(max(np, 0), n);
    lo = min(max(lo, 0), r.n_bias);
    hi = min(max(hi, lo), r.n_bias);
    __syncthreads();
    auto column = [&](int t) -> unsigned int { return t < 0 ? 0xffffffffu : (unsigned int)t - (unsigned int)w.col0; };
    for (int base = 0; base < n; base += kThreads * kTokens) {
        if (base) tokens(base);
#pragma unroll
        for (int u = 0; u < kTokens; u++) {
            const int i = base + u * kThreads + tid;
            const unsigned int at = column(tok[u]);
            if (i < n && at < (unsigned int)ncol) {
                if (i < np) atomicOr(&w.count[at], kPrompt);
                else atomicAdd(&w.count[at], 1u);
            }
        }
    }
    if (PEN && w.drafted && tid < row_lo) {   // drafts before the block's first row
        const unsigned int at = column(__ldg(w.drafted - row_lo + tid));
        if (at < (unsigned int)ncol) atomicAdd(&w.count[at], 1u);
    }
    for (int i = lo + tid; i < hi; i += kThreads) {
        const unsigned int at = column(__ldg(r.bias_ids + i));
        if (at < (unsigned int)ncol) atomicMax(&w.bias_at[at], i + 1);   // an id given twice: its last value
    }
    __syncthreads();
    // from here on a count is touched by the one thread that owns its column only
    const int subs = min(a.spans_per_block, (a.V - w.col0 + kSpan - 1) / kSpan);
    const int left = a.V - w.col0 - (subs - 1) * kSpan - (VEC ? tid * 4 : tid);   // columns of the last span from the thread's first on
    const int cols = VEC ? min(4, left) : min(4, (left + kThreads - 1) / kThreads);
    const int whole = cols == 4 ? subs : subs - 1;
    if (whole) run<VEC, true, PEN, BIAS, MASK>(a, w, 0, whole, 4);
    if (whole < subs && cols > 0) run<VEC, false, PEN, BIAS, MASK>(a, w, whole, subs, cols);
}

// one kernel for each set of rules: what a call does not use costs it no registers
template <bool VEC> void (*pick(bool pen, bool bias, bool mask))(Args) {
    if (pen) return bias ? (mask ? process_kernel<VEC, true, true, true> : process_kernel<VEC, true, true, false>)
                         : (mask ? process_kernel<VEC, true, false, true> : process_kernel<VEC, true, false, false>);
    return bias ? (mask ? process_kernel<VEC, false, true, true> : process_kernel<VEC, false, true, false>)
                : (mask ? process_kernel<VEC, false, false, true> : process_kernel<VEC, false, false, false>);
}

}  // namespace rules
}  // namespace eesd

using namespace eesd;

extern "C" int eesd_process_logits(void *cuda_stream, const float *logits, int64_t ld_logits, float *out, int64_t ld_out, int B, int rows, int V,
                                   const eesd_logit_rules *r) {
    if (!logits || !out || !r || B < 1 || rows < 1 || rows > EESD_MAX_RULE_ROWS || V < 1 || ld_logits < V || ld_out < V) return EESD_ERR_BADARG;
    const void *const words[] = {logits, out, r->history, r->n_history, r->n_prompt, r->drafted, r->repetition, r->frequency, r->presence, r->bias_start, r->bias_ids, r->bias_values, r->mask};
    for (const void *p : words)
        if ((uintptr_t)p & 3) return EESD_ERR_BADARG;
    if (r->history && (r->history_len < 0 || r->history_stride < r->history_len)) return EESD_ERR_BADARG;
    if (r->drafted && r->drafted_stride < rows - 1) return EESD_ERR_BADARG;
    if (r->n_bias < 0 || (r->n_bias > 0 && (!r->bias_start || !r->bias_ids || !r->bias_values))) return EESD_ERR_BADARG;
    if (r->mask && r->mask_stride < ((int64_t)V + 31) / 32) return EESD_ERR_BADARG;
    // (the kernel's 32-bit indices pass an end by less than a block's columns, or its threads' tokens)
    if (V > EESD_MAX_RULE_LENGTH || (r->history && r->history_len > EESD_MAX_RULE_LENGTH) || r->n_bias > EESD_MAX_RULE_LENGTH) return EESD_ERR_UNSUPPORTED;
    const long long n_rows = (long long)B * rows;
    if (n_rows > 0x7fffffffLL) return EESD_ERR_UNSUPPORTED;
    // in place means exactly in place; any other overlap would read rows that are already processed
    const bool same = logits == out && ld_logits == ld_out;
    const uintptr_t i0 = (uintptr_t)logits, i1 = i0 + ((size_t)(n_rows - 1) * ld_logits + V) * 4;
    const uintptr_t o0 = (uintptr_t)out, o1 = o0 + ((size_t)(n_rows - 1) * ld_out + V) * 4;
    if (!same && i0 < o1 && o0 < i1) return EESD_ERR_BADARG;

    rules::Args a;
    a.r = *r;
    if (rows < 2) a.r.drafted = nullptr;
    if (a.r.history_len == 0) a.r.history = nullptr;
    if (!a.r.repetition && !a.r.frequency && !a.r.presence) a.r.history = a.r.drafted = nullptr;   // nothing looks at the counts
    a.in = logits;
    a.out = out;
    a.ld_in = (size_t)ld_logits;
    a.ld_out = (size_t)ld_out;
    a.rows = rows;
    a.V = V;
    a.spans = (V + rules::kSpan - 1) / rules::kSpan;
    a.spans_per_block = 1;
    a.row_split = 1;
    // Few sequences split their rows among blocks until the machine is full (8 x 17 x 32000: 15.3 us, 17.2 without); many take
    // several spans a block, so that a sequence's tokens are counted by fewer blocks (64 x 1 x 128256: 1, 2, 4 spans 51, 34, 28 us), as long as
    // they fill most of the machine.  On either side of the border, 1, 2, 4 spans: 12 x 5 x 50257 10.0, 11.3, 16.9; 15 x 5 x 50257 12.3, 12.2, 17.5; 17 x 5
    // x 50257 12.9, 12.6, 18.1; 24 x 5 x 32000 14.4, 13.6, 19.1; 26 x 5 x 32000 14.8, 13.7, 19.3; 49 x 4 x 32000 19.9, 20.6, 19.3; 51 x 4 x 32000 20.4,
    // 20.9, 19.5.
    while (a.row_split * 2 <= rows && (long long)B * a.spans * a.row_split < 4 * 148) a.row_split *= 2;
    if (a.row_split == 1)
        while (a.spans_per_block < 4 && (long long)B * a.spans / (a.spans_per_block * 2) >= 400) a.spans_per_block *= 2;
    a.rows_per_block = (rows + a.row_split - 1) / a.row_split;
    a.row_split = (rows + a.rows_per_block - 1) / a.rows_per_block;
    a.chunks = (a.spans + a.spans_per_block - 1) / a.spans_per_block;
    const long long blocks = (long long)a.chunks * a.row_split * B;
    if (blocks > 0x7fffffffLL) return EESD_ERR_UNSUPPORTED;
    const size_t ncol = (size_t)a.spans_per_block * rules::kSpan;
    const size_t smem = ncol * 4 * ((a.r.history || a.r.drafted ? 1 : 0) + (a.r.n_bias ? 1 : 0));
    const bool vec = ld_logits % 4 == 0 && ld_out % 4 == 0 && (((uintptr_t)logits | (uintptr_t)out) & 15) == 0;
    const bool pen = a.r.history || a.r.drafted, bias = a.r.n_bias != 0, mask = a.r.mask != nullptr;
    auto kernel = vec ? rules::pick<true>(pen, bias, mask) : rules::pick<false>(pen, bias, mask);
    launch_k(kernel, dim3((unsigned int)blocks), dim3(rules::kThreads), smem, (cudaStream_t)cuda_stream, pdl_enabled(), a);
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}
