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
    //     72  ViT-S 476x630         27 / 22 / 16       176  ViT-L 518x518             27 / 24 / 27      2112  ViT-g 518x518 x 8           133 / 160 / 218
    //    132  ViT-B 518x518         26 / 23 / 25       264  ViT-B 518x518 x 2         32 / 29 / 39       256  8192 causal, 16 heads of 128  301 / 357 / 708
    //    132  the same, a grid      46 / 32 / 33       352  ViT-L 518x518 x 2         32 / 31 / 42       410  five views on a grid         60 / 57 / 63
    //    132  the same, fp32        69 / 74 / 91       192  3000 fp32, 8 heads of 128 194 / 184 / 312
    // Few rows: one launch is as long as its longest workgroup, so the keys are shared by more waves; many: reading the tiles counts, and a
    // workgroup's rows share them.  fp32 waves split every operand that they read: keys shared by four waves of 32 rows are split four times as often.
    int64_t blocks = with_rows(most <= 32 ? 32 : 128);
    if (most > 32 && blocks * plan.sets < 256) blocks = with_rows(a.dtype == VPE_F32 || blocks * plan.sets >= 96 ? 64 : 32);
    // Parts of the keys where row blocks are few, joined by a second launch.  One launch, for few keys: us on the card / on the host for one and for
    // two, 6 heads of 64: 257 keys 6.8 / 13.2 and 9.0 / 16.0, 700 8.6 / 13.2 and 9.4 / 16.1, 1370 11.5 / 13.1 and 10.0 / 16.1, 2740 18.0 / 13.1 and
    // 11.3 / 16.0; 32 of 128: 700 12.4 / 12.6 and 11.9 / 15.5, 1370 17.8 / 12.7 and 12.9 / 15.3; 12 of 64 in fp32: 257 11.7 / 12.4 and 12.5 / 15.0,
    // 700 18.5 / 12.9 and 13.1 / 15.7.
    const bool wide = a.dtype == VPE_F32, one = (int64_t)a.max_k * a.head_dim <= (wide ? 24 : 96) << 10;
    // Workgroups for every CU and no more (a token, 8 key heads of 128, 16384 keys: 12 parts 25.6 us, 32 29.3, 64 42; 16 heads of 64, 12000
    // keys: 12 19.9, 32 24.8), of 512 keys and up (32 heads of 128, 2740 keys: 18.4, of 256 24.5); fp32, bound by its products, shares 256 keys
    // and up (a token, 8 heads of 128, 16384 keys: 12 parts 97 us, 32 53, 64 66), with more rows among two workgroups for a CU, which fit then
    // (ViT-S 476x630: one part 63 us, three 45).  Many sequences are taken to be of many lengths: then up to four for a CU, of 3200 keys and up,
    // even things out (24 sequences up to 16384, 8 key heads of 128: one part 214 us, 3 154, 5 138, 7 151).  Their number is odd: sets go round the
    // 8 XCDs, and with 2, 4 or 8 parts an XCD has the first parts, which all sequences have, or the last ones always (the same, 4 parts: 165; 48
    // sequences up to 14200: 2 parts 313, 3 266, 4 331, 5 263).
    const int64_t base = blocks * plan.sets;
    int64_t parts = std::min<int64_t>({(wide && most > 32 ? 512 : 256) / base, up(a.max_k, wide ? 256 : 512), wide ? 63 : 15});
    if (a.sequences > 1) {
        parts = std::max(parts, std::min<int64_t>(1024 / base, a.max_k / 3200));
        if (parts % 2 == 0 && parts) parts = parts == 2 ? 3 : parts - 1;
    }
    plan.splits = one ? 1 : (int)std::max<int64_t>(1, parts);
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
