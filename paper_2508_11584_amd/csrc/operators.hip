// C entry points of the operators on packed rows: what a call may ask for is checked here, before anything is enqueued.
#include <cmath>
#include <cstdio>

#include "operators.h"

using namespace vpe;

namespace {

// One refusal: the message and the code.  (No std::string: nothing here may throw through the C boundary.)
#define REFUSE(...)                                                \
    do {                                                           \
        char buf__[256];                                           \
        snprintf(buf__, sizeof buf__, __VA_ARGS__);                \
        return call_error(VPE_EINVAL, buf__);                      \
    } while (0)

bool aligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

int launched(hipError_t rc, const char* what) {
    if (rc == hipSuccess) return VPE_OK;
    char buf[256];
    snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(rc));
    return call_error(VPE_EHIP, buf);
}

int check_sizes(const vpe_attention_args* a) {
    if (!a) REFUSE("args is null");
    if (a->dtype != VPE_F32 && a->dtype != VPE_BF16) REFUSE("unknown dtype");
    if (a->head_dim != 64 && a->head_dim != 128) REFUSE("head_dim is %d: 64 or 128 required", a->head_dim);
    if (a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads || a->heads > 4096) REFUSE("heads must be a multiple of kv_heads, at most 4096");
    if (a->sequences > (1 << 24)) REFUSE("more than 2^24 sequences");
    if (a->sequences < 0 || a->max_q < 0 || a->max_k < 0 || a->q_rows < 0 || a->k_rows < 0) REFUSE("sizes must not be negative");
    // (row places are 32-bit sums of two lengths; a workspace row count stays below 2^31)
    if (a->q_rows > (1 << 30) || a->k_rows > (1 << 30) || a->max_q > (1 << 30) || a->max_k > (1 << 30)) REFUSE("more than 2^30 rows");
    return VPE_OK;
}

bool nothing_to_do(const vpe_attention_args& a) { return a.sequences == 0 || a.max_q == 0 || a.q_rows == 0; }

int check_sizes(const vpe_adapter_linear_args* a) {
    if (!a) REFUSE("args is null");
    if (a->dtype != VPE_F32 && a->dtype != VPE_BF16) REFUSE("unknown dtype");
    if (a->rows < 0 || a->out_features < 1) REFUSE("rows must not be negative, out_features positive");
    if (a->in_features < 64 || a->in_features % 64) REFUSE("in_features is %d: a multiple of 64 required", a->in_features);
    if (a->adapters < 0) REFUSE("adapters must not be negative");
    if (a->adapters > 0 && (a->rank < 8 || a->rank % 8 || a->rank > 128)) REFUSE("rank is %d: a multiple of 8 up to 128 required", a->rank);
    if (a->rows > (1 << 30) || a->out_features > (1 << 23) || a->in_features > (1 << 20)) REFUSE("sizes too large");
    return VPE_OK;
}

int check_workspace(const void* ptr, uint64_t bytes, uint64_t need) {
    if (need && (!ptr || bytes < need)) REFUSE("workspace has %llu bytes, %llu needed", (unsigned long long)(ptr ? bytes : 0), (unsigned long long)need);
    if (need && !aligned(ptr, 256)) REFUSE("workspace is not 256-byte aligned");
    return VPE_OK;
}

}  // namespace

extern "C" {

int vpe_attention_workspace_bytes(const vpe_attention_args* args, uint64_t* bytes) {
    const int rc = check_sizes(args);
    if (rc) return rc;
    if (!bytes) REFUSE("bytes is null");
    *bytes = nothing_to_do(*args) ? 0 : plan_seq_attention(*args).workspace;
    return VPE_OK;
}

int vpe_attention(const vpe_attention_args* args, void* stream) {
    int rc = check_sizes(args);
    if (rc) return rc;
    const vpe_attention_args& a = *args;
    if (!std::isfinite(a.scale) || !std::isfinite(a.cap) || a.cap < 0.0f) REFUSE("scale must be finite, cap finite and not negative");
    if (a.causal != 0 && a.causal != 1) REFUSE("causal must be 0 or 1");
    if (a.q_row < 0 || a.q_head < 0 || a.k_row < 0 || a.k_head < 0 || a.v_row < 0 || a.v_head < 0) REFUSE("strides must not be negative");
    if (a.out_row < a.head_dim || a.out_head < a.head_dim) REFUSE("out's strides must be at least head_dim");
    const int per16 = a.dtype == VPE_BF16 ? 8 : 4;
    for (int64_t v : {a.q_row, a.q_head, a.k_row, a.k_head, a.v_row, a.v_head, a.out_row, a.out_head})
        if (v % per16) REFUSE("strides must be multiples of 16 bytes");
    if (a.k_row > (1 << 23) || a.v_row > (1 << 23)) REFUSE("row strides of k and v above 2^23 elements");      // (a tile's offsets are 32-bit)
    if (nothing_to_do(a)) return VPE_OK;
    if (!a.q || !a.out || !a.q_offsets || !a.k_offsets) REFUSE("null pointer");
    if (a.k_rows > 0 && a.max_k > 0 && (!a.k || !a.v)) REFUSE("k or v is null");
    for (const void* p : {a.q, a.k, a.v, (const void*)a.out})
        if (!aligned(p, 16)) REFUSE("q, k, v and out must be 16-byte aligned");
    for (const void* p : {(const void*)a.q_offsets, (const void*)a.k_offsets, (const void*)a.k_lengths, (const void*)a.prefix, (const void*)a.slopes, (const void*)a.lse})
        if (!aligned(p, 4)) REFUSE("arrays must be aligned to their elements");
    if (!a.q_coords != !a.k_coords || (a.q_coords && !a.slopes)) REFUSE("q_coords and k_coords go together, with slopes");
    if (!aligned(a.q_coords, 8) || !aligned(a.k_coords, 8)) REFUSE("coordinates must be 8-byte aligned");
    const SeqAttnPlan plan = plan_seq_attention(a);
    if (plan.blocks < 0) REFUSE("too many rows for one call");
    rc = check_workspace(a.workspace, a.workspace_bytes, plan.workspace);
    if (rc) return rc;
    return launched(launch_seq_attention(a, plan, (hipStream_t)stream), "attention launch");
}

int vpe_block_norm(const vpe_block_norm_args* args, void* stream) {
    if (!args) REFUSE("args is null");
    const vpe_block_norm_args& a = *args;
    if (a.dtype != VPE_F32 && a.dtype != VPE_BF16) REFUSE("unknown dtype");
    if (a.rows < 0 || a.requests < 0) REFUSE("sizes must not be negative");
    if (a.dim < 1 || a.dim > 8192) REFUSE("dim is %d: 1 to 8192 required", a.dim);
    for (int kind : {a.post, a.pre})
        if (kind != VPE_NORM_NONE && kind != VPE_NORM_LAYER && kind != VPE_NORM_RMS) REFUSE("unknown norm");
    if (!(a.eps > 0.0f) || !std::isfinite(a.eps) || !std::isfinite(a.residual_scale)) REFUSE("eps must be positive and finite, residual_scale finite");
    if (a.rows == 0) return VPE_OK;
    if (!a.x || !a.out) REFUSE("x or out is null");
    if (a.x_row < a.dim || a.out_row < a.dim || (a.branch && a.branch_row < a.dim) || (a.normed && a.normed_row < a.dim)) REFUSE("row strides must be at least dim");
    if (a.x == a.out && a.x_row != a.out_row) REFUSE("out may be x with the same row stride only");
    const uintptr_t esz = a.dtype == VPE_BF16 ? 2 : 4;
    for (const void* p : {(const void*)a.x, (const void*)a.out, (const void*)a.post_gain, (const void*)a.post_bias, (const void*)a.pre_gain, (const void*)a.pre_bias,
                          (const void*)a.layer_scale, (const void*)a.gate, (const void*)a.scale, (const void*)a.shift, (const void*)a.request})
        if (!aligned(p, 4)) REFUSE("arrays must be aligned to their elements");
    if (!aligned(a.branch, esz) || !aligned(a.normed, esz)) REFUSE("arrays must be aligned to their elements");
    return launched(launch_block_norm(a, (hipStream_t)stream), "block norm launch");
}

int vpe_adapter_linear_workspace_bytes(const vpe_adapter_linear_args* args, uint64_t* bytes) {
    const int rc = check_sizes(args);
    if (rc) return rc;
    if (!bytes) REFUSE("bytes is null");
    *bytes = args->rows ? adapter_linear_workspace(*args) : 0;
    return VPE_OK;
}

int vpe_adapter_linear(const vpe_adapter_linear_args* args, void* stream) {
    int rc = check_sizes(args);
    if (rc) return rc;
    const vpe_adapter_linear_args& a = *args;
    if (a.out_f32 != 0 && a.out_f32 != 1) REFUSE("out_f32 must be 0 or 1");
    if (a.rows == 0) return VPE_OK;
    if (!a.x || !a.weight || !a.out) REFUSE("null pointer");
    if (a.x_row < a.in_features || a.x_row % (a.dtype == VPE_BF16 ? 8 : 4)) REFUSE("x's row stride must be at least in_features and a multiple of 16 bytes");
    if (a.rows > 1 && a.x_row > (1 << 20)) REFUSE("x's row stride above 2^20 elements");       // (a tile's offsets are 32-bit)
    if (a.out_row < a.out_features) REFUSE("out's row stride must be at least out_features");
    if (!aligned(a.x, 16) || !aligned(a.weight, 16)) REFUSE("x and weight must be 16-byte aligned");
    if (!aligned(a.out, a.out_f32 || a.dtype == VPE_F32 ? 4 : 2) || !aligned(a.bias, 4)) REFUSE("arrays must be aligned to their elements");
    if (a.adapters > 0 && a.adapter) {
        if (!a.a || !a.b) REFUSE("a or b is null");
        if (!aligned(a.a, 16) || !aligned(a.b, 16)) REFUSE("a and b must be 16-byte aligned");
        if (!aligned(a.adapter, 4) || !aligned(a.scale, 4)) REFUSE("arrays must be aligned to their elements");
    }
    rc = check_workspace(a.workspace, a.workspace_bytes, adapter_linear_workspace(a));
    if (rc) return rc;
    return launched(launch_adapter_linear(a, (hipStream_t)stream), "adapter projection launch");
}

}  // extern "C"
