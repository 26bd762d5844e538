// Logit rules: penalties for repeated tokens, biases and grammar masks on the logit rows of a decode or verification
// round (sm_100a).  For entry v of row i of sequence b, with n the times v was generated (history past the prompt, and the
// drafts x_1..x_i that precede the row) and `seen` telling that it was generated or is in the prompt:
//   l1 = seen ? (l > 0 ? l / repetition : l * repetition) : l
//   l2 = l1 - (frequency * n + (n > 0 ? presence : 0))
//   l3 = l2 + bias(v)
//   out = allowed(v) ? l3 : -inf
// every operation rounded to fp32 by itself.
//
// Memory bound: 8 bytes per entry and one mask bit.  A block owns a run of the vocabulary for one sequence, counts the
// sequence's tokens that fall into it in shared memory (integer atomics: the result does not depend on their order),
// takes the counts and biases of its threads' columns into registers and then walks the rows, so that counting is paid once
// per sequence and not once per row; a draft adds to the count of the one thread that owns its column.
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

__device__ __forceinline__ float apply(float l, uint32_t c, float rep, float freq, float pres) {
    if (c) l = l > 0.f ? __fdiv_rn(l, rep) : __fmul_rn(l, rep);
    const uint32_t n = c & ~kPrompt;
    if (n) l = __fsub_rn(l, __fadd_rn(__fmul_rn(freq, (float)n), pres));
    return l;
}

// VEC: rows are 16-byte aligned and V % 4 == 0: a thread's four columns are neighbours, one 16-byte access a row.  Otherwise they
// lie kThreads apart, 4-byte accesses.
template <bool VEC>
__global__ void __launch_bounds__(kThreads) process_kernel(const Args a) {
    extern __shared__ uint32_t smem[];
    const eesd_logit_rules &r = a.r;
    const int ncol = a.spans_per_block * kSpan;
    uint32_t *count = smem;
    int *bias_at = (int *)(smem + (r.history || r.drafted ? ncol : 0));   // 1 + place of the column's bias in the list; 0: none
    const int tid = threadIdx.x;
    int job = blockIdx.x;
    const int chunk = job % a.chunks;
    job /= a.chunks;
    const int rs = job % a.row_split, b = job / a.row_split;
    const int col0 = chunk * ncol, row_lo = rs * a.rows_per_block, row_hi = min(a.rows, row_lo + a.rows_per_block);
    const bool counting = r.history || r.drafted;
    const int32_t *drafted = r.drafted ? r.drafted + (size_t)b * r.drafted_stride : nullptr;

    if (counting)
        for (int i = tid; i < ncol; i += kThreads) count[i] = 0;
    if (r.n_bias)
        for (int i = tid; i < ncol; i += kThreads) bias_at[i] = 0;
    pdl_wait();
    pdl_trigger();
    __syncthreads();
    if (r.history) {
        const int32_t *h = r.history + (size_t)b * r.history_stride;
        const int n = r.n_history ? min(max(__ldg(r.n_history + b), 0), r.history_len) : r.history_len;
        const int np = r.n_prompt ? min(max(__ldg(r.n_prompt + b), 0), n) : 0;
        for (int base = 0; base < n; base += kThreads * 4) {
            int tok[4];
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const int i = base + u * kThreads + tid;
                tok[u] = i < n ? __ldg(h + i) : -1;
            }
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const unsigned int at = (unsigned int)tok[u] - (unsigned int)col0;
                if (tok[u] >= 0 && at < (unsigned int)ncol) {
                    if (base + u * kThreads + tid < np) atomicOr(&count[at], kPrompt);
                    else atomicAdd(&count[at], 1u);
                }
            }
        }
    }
    if (drafted && tid < row_lo) {   // drafts before the block's first row
        const int tok = __ldg(drafted + tid);
        const unsigned int at = (unsigned int)tok - (unsigned int)col0;
        if (tok >= 0 && at < (unsigned int)ncol) atomicAdd(&count[at], 1u);
    }
    if (r.n_bias) {
        const int lo = min(max(__ldg(r.bias_start + b), 0), r.n_bias), hi = min(max(__ldg(r.bias_start + b + 1), lo), r.n_bias);
        for (int i = lo + tid; i < hi; i += kThreads) {
            const int tok = __ldg(r.bias_ids + i);
            const unsigned int at = (unsigned int)tok - (unsigned int)col0;
            if (tok >= 0 && at < (unsigned int)ncol) atomicMax(&bias_at[at], i + 1);   // an id given twice: its last value
        }
    }
    __syncthreads();

    const float rep = r.repetition ? __ldg(r.repetition + b) : 1.f;
    const float freq = r.frequency ? __ldg(r.frequency + b) : 0.f, pres = r.presence ? __ldg(r.presence + b) : 0.f;
    const size_t first = (size_t)b * a.rows;
    for (int sub = 0; sub < a.spans_per_block; sub++) {
        const int c0 = col0 + sub * kSpan;
        if (c0 >= a.V) break;
        const int col = VEC ? c0 + tid * 4 : c0 + tid;
        constexpr int step = VEC ? 1 : kThreads;
        uint32_t cnt[4];
        float bias[4];
        bool any_bias = false;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int at = col + i * step - col0;
            cnt[i] = counting ? count[at] : 0;
            const int j = r.n_bias ? bias_at[at] : 0;
            bias[i] = j ? __ldg(r.bias_values + j - 1) : 0.f;
            any_bias |= j != 0;
        }
        if (col >= a.V) continue;
        constexpr int kBatch = 4;   // rows in flight
        for (int i0 = row_lo; i0 < row_hi; i0 += kBatch) {
            float l[kBatch][4];
            uint32_t m[kBatch][VEC ? 1 : 4];
#pragma unroll
            for (int k = 0; k < kBatch; k++) {
                if (i0 + k >= row_hi) break;
                const float *src = a.in + (first + i0 + k) * a.ld_in + col;
                if (VEC) {
                    const float4 v = __ldcs(reinterpret_cast<const float4 *>(src));
                    l[k][0] = v.x; l[k][1] = v.y; l[k][2] = v.z; l[k][3] = v.w;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; i++) l[k][i] = col + i * step < a.V ? __ldcs(src + i * step) : 0.f;
                }
                if (r.mask) {
                    const uint32_t *w = (const uint32_t *)r.mask + (first + i0 + k) * (size_t)r.mask_stride;
                    if (VEC) {
                        m[k][0] = __ldg(w + (col >> 5)) >> (col & 31);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            const int c = col + i * step;
                            m[k][VEC ? 0 : i] = c < a.V ? __ldg(w + (c >> 5)) >> (c & 31) : 0;
                        }
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < kBatch; k++) {
                const int row = i0 + k;
                if (row >= row_hi) break;
                if (drafted && row > row_lo) {   // the draft that precedes this row
                    const int tok = __ldg(drafted + row - 1);
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (tok == col + i * step) cnt[i]++;
                }
                if (cnt[0] | cnt[1] | cnt[2] | cnt[3]) {
#pragma unroll
                    for (int i = 0; i < 4; i++) l[k][i] = apply(l[k][i], cnt[i], rep, freq, pres);
                }
                if (any_bias) {
#pragma unroll
                    for (int i = 0; i < 4; i++) l[k][i] = __fadd_rn(l[k][i], bias[i]);
                }
                if (r.mask) {
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (!(VEC ? m[k][0] >> i & 1u : m[k][VEC ? 0 : i] & 1u)) l[k][i] = -INFINITY;
                }
                float *dst = a.out + (first + row) * a.ld_out + col;
                if (VEC) {
                    *reinterpret_cast<float4 *>(dst) = make_float4(l[k][0], l[k][1], l[k][2], l[k][3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (col + i * step < a.V) dst[i * step] = l[k][i];
                }
            }
        }
    }
}

}  // namespace rules
}  // namespace eesd

using namespace eesd;

extern "C" int eesd_process_logits(void *cuda_stream, const float *logits, int64_t ld_logits, float *out, int64_t ld_out, int B, int rows, int V,
                                   const eesd_logit_rules *r) {
    if (!logits || !out || !r || B < 1 || rows < 1 || rows > EESD_MAX_RULE_ROWS || V < 1 || ld_logits < V || ld_out < V) return EESD_ERR_BADARG;
    if (((uintptr_t)logits | (uintptr_t)out) & 3) return EESD_ERR_BADARG;
    if (r->history && (r->history_len < 0 || r->history_stride < r->history_len)) return EESD_ERR_BADARG;
    if (r->drafted && r->drafted_stride < rows - 1) return EESD_ERR_BADARG;
    if (r->n_bias < 0 || (r->n_bias > 0 && (!r->bias_start || !r->bias_ids || !r->bias_values))) return EESD_ERR_BADARG;
    if (r->mask && r->mask_stride < ((int64_t)V + 31) / 32) return EESD_ERR_BADARG;
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
    // Enough blocks to fill the machine several times: few sequences split their rows, many take several spans a block so
    // that a sequence's tokens are counted over by fewer blocks.
    const long long fill = 148 * 8;
    while (a.row_split * 2 <= rows && (long long)B * a.spans * a.row_split < fill) a.row_split *= 2;
    if (a.r.history) while (a.spans_per_block < 4 && (long long)B * a.spans / (a.spans_per_block * 2) >= 2 * fill) a.spans_per_block *= 2;
    a.rows_per_block = (rows + a.row_split - 1) / a.row_split;
    a.row_split = (rows + a.rows_per_block - 1) / a.rows_per_block;
    a.chunks = (a.spans + a.spans_per_block - 1) / a.spans_per_block;
    const long long blocks = (long long)a.chunks * a.row_split * B;
    if (blocks > 0x7fffffffLL) return EESD_ERR_UNSUPPORTED;
    const size_t ncol = (size_t)a.spans_per_block * rules::kSpan;
    const size_t smem = ncol * 4 * ((a.r.history || a.r.drafted ? 1 : 0) + (a.r.n_bias ? 1 : 0));
    const bool vec = V % 4 == 0 && ld_logits % 4 == 0 && ld_out % 4 == 0 && (((uintptr_t)logits | (uintptr_t)out) & 15) == 0;
    launch_k(vec ? rules::process_kernel<true> : rules::process_kernel<false>, dim3((unsigned int)blocks), dim3(rules::kThreads), smem, (cudaStream_t)cuda_stream,
             pdl_enabled(), a);
    return cudaGetLastError() == cudaSuccess ? EESD_OK : EESD_ERR_CUDA;
}
