// Instantiations and launch of the attention over packed sequences.
#include "operators.h"
#include "seq_attention.h"

namespace vpe {
namespace {

// A wave per row and head.
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_rows_kernel(const vpe_attention_args p) {
    const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int h = (int)(task % p.heads);
    const int64_t r = task / p.heads;
    const int i = (int)(r % p.max_q);
    if (r / p.max_q >= p.sequences) return;
    const Seq sq = sequence(p, (int)(r / p.max_q));
    if (i < sq.nq) attention_row<T, D>(p, sq, i, h, threadIdx.x & 63);
}

}  // namespace

SeqAttnPlan plan_seq_attention(const vpe_attention_args& a) {
    const int64_t tasks = (int64_t)a.sequences * a.max_q * a.heads;
    return SeqAttnPlan{0, (int)((tasks + 3) / 4 < 0x7fffffff ? (tasks + 3) / 4 : -1), 0, 1, a.max_k, 0};
}

hipError_t launch_seq_attention(const vpe_attention_args& a, const SeqAttnPlan& plan, hipStream_t s) {
    typedef void (*Kernel)(const vpe_attention_args);
    const Kernel k = a.dtype == VPE_BF16 ? (a.head_dim == 64 ? &attention_rows_kernel<bf16, 64> : &attention_rows_kernel<bf16, 128>)
                                         : (a.head_dim == 64 ? &attention_rows_kernel<float, 64> : &attention_rows_kernel<float, 128>);
    hipLaunchKernelGGL(k, dim3(plan.blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace vpe
