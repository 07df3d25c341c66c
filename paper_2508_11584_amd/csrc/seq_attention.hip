// Instantiations, plan and launch of the attention over packed sequences.
#include <algorithm>

#include "operators.h"
#include "seq_attention.h"

namespace vpe {
namespace {

SeqShape shape_of(const vpe_attention_args& a, const SeqAttnPlan& plan) {
    // (plain scores stay raw until the exponential: a factor that is not positive would turn their order round, a tiny one make 0 x infinity of
    // hidden ones; LINE multiplies first, and without slopes takes nothing off)
    const bool cap = a.cap > 0.0f;
    const int dist = a.q_coords ? DIST_GRID : a.slopes || (!cap && !(a.scale > 1e-30f)) ? DIST_LINE : DIST_NONE;
    return a.dtype == VPE_BF16 ? seq_shape_bf16(cap, dist, a.head_dim, plan.rows) : seq_shape_f32(cap, dist, a.head_dim, plan.rows);
}

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

SeqAttnPlan plan_seq_attention(const vpe_attention_args& a) {
    const int G = a.heads / a.kv_heads;
    SeqAttnPlan plan{};
    const int64_t most = (int64_t)a.max_q * G;                    // rows of a sequence and key head
    auto with_rows = [&](int rows) {
        const int64_t direct = up(most, rows), all = (int64_t)a.q_rows * G / rows + a.sequences;
        plan.rows = rows;
        plan.packed = direct * a.sequences > all;
        plan.sets = a.kv_heads * (int64_t)(plan.packed ? 1 : a.sequences);
        return plan.packed ? all : direct;
    };
    // us, workgroups of 128 rows (four waves of 32) / 64 (two, by two that share the keys) / 32 (four that share the keys), by workgroups of 128:
    //     72  ViT-S 476x630         26 / 23 / 15       176  ViT-L 518x518             33 / 24 / 25      2112  ViT-g 518x518 x 8           126 / 155 / 211
    //    132  ViT-B 518x518         30 / 23 / 24       264  ViT-B 518x518 x 2         31 / 28 / 37       256  8192 causal, 16 heads of 128  285 / 338 / 615
    //    132  the same, a grid      36 / 31 / 32       352  ViT-L 518x518 x 2         32 / 30 / 41       410  five views on a grid         58 / 56 / 62
    //    132  the same, fp32        66 / 75 / 88       192  3000 fp32, 8 heads of 128 184 / 175 / 304
    // Few rows: one launch is as long as its longest workgroup, so the keys are shared by more waves; many: reading the tiles counts, and a
    // workgroup's rows share them.  fp32 waves split every operand that they read: keys shared by four waves of 32 rows are split four times as often.
    int64_t blocks = with_rows(most <= 32 ? 32 : 128);
    if (most > 32 && blocks * plan.sets < 256) blocks = with_rows(a.dtype == VPE_F32 || blocks * plan.sets >= 96 ? 64 : 32);
    // Parts of at least 256 keys until two workgroups for every CU are there
    const int64_t base = blocks * plan.sets;
    plan.splits = base < 256 ? (int)std::max<int64_t>(1, std::min<int64_t>({512 / base, up(a.max_k, 256), 64})) : 1;
    plan.per_split = (int)up(up(a.max_k, plan.splits), 128) * 128;
    plan.per_split = std::max(plan.per_split, 128);
    plan.splits = (int)std::max<int64_t>(1, up(a.max_k, plan.per_split));
    plan.sets *= plan.splits;
    plan.chunk = (int)std::max<int64_t>(1, std::min<int64_t>({16, blocks, blocks * plan.sets / 64}));
    const int64_t grid = up(up(blocks, plan.chunk) * plan.sets, 8) * 8 * plan.chunk;
    plan.blocks = blocks <= 0x7fffffff && grid <= 0x7fffffff ? (int)blocks : -1;
    plan.grid = (uint32_t)grid;
    const uint64_t part = (uint64_t)plan.splits * a.q_rows * a.heads;
    plan.workspace = plan.splits > 1 ? part * 4 * (a.head_dim + 2) : 0;
    return plan;
}

hipError_t launch_seq_attention(const vpe_attention_args& a, const SeqAttnPlan& plan, hipStream_t s) {
    const SeqShape k = shape_of(a, plan);
    SeqAttnGrid grid{plan.blocks, plan.packed, plan.splits, plan.per_split, plan.chunk, nullptr, nullptr};
    if (plan.splits > 1) {
        grid.part_o = reinterpret_cast<float*>(a.workspace);
        grid.part_ml = grid.part_o + (uint64_t)plan.splits * a.q_rows * a.heads * a.head_dim;
    }
    if (k.lds > 64 * 1024) {
        const hipError_t rc = hipFuncSetAttribute(reinterpret_cast<const void*>(k.kernel), hipFuncAttributeMaxDynamicSharedMemorySize, k.lds);
        if (rc != hipSuccess) return rc;
    }
    hipLaunchKernelGGL(k.kernel, dim3(plan.grid), dim3(k.threads), k.lds, s, a, grid);
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess || plan.splits == 1) return rc;
    const SeqKernel join = a.dtype == VPE_BF16 ? (a.head_dim == 64 ? &seq_attention_join_kernel<bf16, 64> : &seq_attention_join_kernel<bf16, 128>)
                                            : (a.head_dim == 64 ? &seq_attention_join_kernel<float, 64> : &seq_attention_join_kernel<float, 128>);
    hipLaunchKernelGGL(join, dim3((uint32_t)up((int64_t)a.q_rows * a.heads, 4)), dim3(256), 0, s, a, grid);
    return hipGetLastError();
}

}  // namespace vpe
