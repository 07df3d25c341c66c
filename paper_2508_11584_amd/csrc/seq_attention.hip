// Instantiations, plan and launch of the attention over packed sequences.
#include <algorithm>
#include <cstdlib>

#include "operators.h"
#include "seq_attention.h"

namespace vpe {
namespace {

typedef void (*Kernel)(const vpe_attention_args, const SeqAttnGrid);
// What a launch needs to know of a shape: rows of a workgroup, threads, LDS, keys that it takes at a time.
struct Shape { Kernel kernel; int rows, threads, lds, keys; };

template <typename T, int D, int KT, int QW, int KW, int MODE, int OCC>
Shape shape() { return {&seq_attention_kernel<T, D, KT, QW, KW, MODE, OCC>, 32 * QW, 64 * QW * KW, seq_lds_bytes<T, D, KT, QW, KW, MODE>(), KT * KW}; }

template <int MODE>
Shape shape_of(int dtype, int head_dim, int rows) {
    // (with coordinates 64 keys of fp32 at a time take a register too many)
    constexpr int F64 = MODE == SCORES_GRID ? 32 : 64;
    if (dtype == VPE_BF16) {
        if (head_dim == 64) return rows == 128 ? shape<bf16, 64, 64, 4, 1, MODE, 3>() : shape<bf16, 64, 32, 1, 4, MODE, 2>();
        return rows == 128 ? shape<bf16, 128, 64, 4, 1, MODE, 2>() : shape<bf16, 128, 32, 1, 4, MODE, 1>();
    }
    if (head_dim == 64) return rows == 128 ? shape<float, 64, F64, 4, 1, MODE, 2>() : shape<float, 64, 32, 1, 4, MODE, 1>();
    return rows == 128 ? shape<float, 128, 32, 4, 1, MODE, 1>() : shape<float, 128, 32, 1, 2, MODE, 1>();
}
Shape shape_of(const vpe_attention_args& a, const SeqAttnPlan& plan) {
    // (a factor that is not positive turns maxima of raw scores round, a tiny one could make 0 x infinity of masked ones: LINE multiplies first)
    if (a.q_coords) return shape_of<SCORES_GRID>(a.dtype, a.head_dim, plan.rows);
    if (a.cap > 0.0f || a.slopes || !(a.scale > 1e-30f)) return shape_of<SCORES_LINE>(a.dtype, a.head_dim, plan.rows);
    return shape_of<SCORES_PLAIN>(a.dtype, a.head_dim, plan.rows);
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
    int64_t blocks = most > 32 ? with_rows(128) : 0;
    const int th = getenv("SA_TH") ? atoi(getenv("SA_TH")) : 384, tg = getenv("SA_TG") ? atoi(getenv("SA_TG")) : 512;
    if (most <= 32 || blocks * plan.sets < (getenv("SA_W") ? atoi(getenv("SA_W")) : 384)) blocks = with_rows(32);
    const int64_t base = blocks * plan.sets;
    plan.splits = 1;
    const int keys = 256;
    if (base < th) plan.splits = (int)std::min<int64_t>({tg / base, up(a.max_k, keys), 64});
    if (plan.splits < 1) plan.splits = 1;
    plan.per_split = (int)up(up(a.max_k, plan.splits), 128) * 128;
    if (plan.per_split < 128) plan.per_split = 128;
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
    const Shape k = shape_of(a, plan);
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
    const Kernel join = a.dtype == VPE_BF16 ? (a.head_dim == 64 ? &seq_attention_join_kernel<bf16, 64> : &seq_attention_join_kernel<bf16, 128>)
                                            : (a.head_dim == 64 ? &seq_attention_join_kernel<float, 64> : &seq_attention_join_kernel<float, 128>);
    hipLaunchKernelGGL(join, dim3((uint32_t)up((int64_t)a.q_rows * a.heads, 4)), dim3(256), 0, s, a, grid);
    return hipGetLastError();
}

}  // namespace vpe
