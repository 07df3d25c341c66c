// Attention over packed sequences with capped scores, distances and prefix masks (vpe_attention).
//
//   s_ij = scale q_i.k_j;  cap > 0: s = cap tanh(s / cap);  s -= slope_h dist(i, j)
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(s_ij - m_i) over the keys j that row i sees,  lse_i = m_i + log sum_j p_ij
#pragma once
#include "common.h"
#include "vpe.h"

namespace vpe {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Sequence s: its rows, cut to the rows that there are (offsets are read from device memory and may hold anything).
struct Seq { int q0, nq, k0, nk, prefix; };
__device__ __forceinline__ int between(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ int seq_rows(const vpe_attention_args& p, int s, int& q0) {
    q0 = between(p.q_offsets[s], 0, p.q_rows);
    const int n = between(p.q_offsets[s + 1], q0, p.q_rows) - q0;
    return n < p.max_q ? n : p.max_q;
}
__device__ __forceinline__ Seq sequence(const vpe_attention_args& p, int s) {
    Seq r;
    r.nq = seq_rows(p, s, r.q0);
    r.k0 = between(p.k_offsets[s], 0, p.k_rows);
    const int n = p.k_lengths ? between(p.k_lengths[s], 0, p.k_rows - r.k0) : between(p.k_offsets[s + 1], r.k0, p.k_rows) - r.k0;
    r.nk = n < p.max_k ? n : p.max_k;
    r.prefix = p.prefix ? p.prefix[s] : 0;
    return r;
}

// Row i of sequence `sq`, head h, by one wave in plain fp32: 64 keys at a time, a lane has a key's score and then one or two
// columns of the result.  Keys that the row does not see are never read: nothing they hold can reach the result.
template <typename T, int D>
__device__ __forceinline__ void attention_row(const vpe_attention_args& p, const Seq& sq, int i, int h, int lane) {
    constexpr int CE = Elem<T>::CE, ND = D / 64;
    const int kh = h / (p.heads / p.kv_heads), place = i + sq.nk - sq.nq;
    const int64_t row = sq.q0 + i;
    const T* q = reinterpret_cast<const T*>(p.q) + row * p.q_row + h * p.q_head;
    const T* k = reinterpret_cast<const T*>(p.k) + (int64_t)sq.k0 * p.k_row + kh * p.k_head;
    const T* v = reinterpret_cast<const T*>(p.v) + (int64_t)sq.k0 * p.v_row + kh * p.v_head;
    const float slope = p.slopes ? p.slopes[h] : 0.0f;
    f32x2 at = {0.0f, 0.0f};
    if (p.q_coords) at = *reinterpret_cast<const f32x2*>(p.q_coords + 2 * row);
    float qv[ND], acc[ND], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int n = 0; n < ND; ++n) { qv[n] = to_f32(q[64 * n + lane]); acc[n] = 0.0f; }
    for (int j0 = 0; j0 < sq.nk; j0 += 64) {
        const int j = j0 + lane;
        const bool seen = j < sq.nk && (!p.causal || j <= place || j < sq.prefix);
        const uint64_t any = __ballot(seen);
        if (!any) continue;
        float s = 0.0f;
        const T* kr = k + (int64_t)(seen ? j : j0 + __builtin_ctzll(any)) * p.k_row;
#pragma unroll
        for (int n = 0; n < ND; ++n)
#pragma unroll 2
            for (int d = 0; d < 64; d += CE) {
                const u32x4 raw = *reinterpret_cast<const u32x4*>(kr + 64 * n + d);
                T e[CE];
                __builtin_memcpy(e, &raw, 16);
#pragma unroll
                for (int c = 0; c < CE; ++c) s = fmaf(__int_as_float(__builtin_amdgcn_readlane(__float_as_int(qv[n]), d + c)), to_f32(e[c]), s);
            }
        s *= p.scale;
        if (p.cap > 0.0f) s = p.cap * tanhf(s / p.cap);
        if (p.q_coords) {
            const f32x2 to = *reinterpret_cast<const f32x2*>(p.k_coords + 2 * (int64_t)(sq.k0 + (seen ? j : j0)));
            const float dy = at[0] - to[0], dx = at[1] - to[1];
            s -= slope * sqrtf(dy * dy + dx * dx);
        } else if (p.slopes) {
            s -= slope * fabsf((float)(place - j));
        }
        s = seen ? s * LOG2E : -INFINITY;
        float mx = s;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
        if (__any(s != s)) l = NAN;                               // (a maximum passes a NaN by)
        const float top = fmaxf(m, mx);
        if (top == -INFINITY) continue;
        const float e = __builtin_amdgcn_exp2f(s - top), alpha = __builtin_amdgcn_exp2f(m - top);
        l = l * alpha + wave_sum(e);
        m = top;
#pragma unroll
        for (int n = 0; n < ND; ++n) acc[n] *= alpha;
        for (uint64_t left = any; left; left &= left - 1) {
            const int jj = __builtin_ctzll(left);
            const float pj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(e), jj));
            const T* vr = v + (int64_t)(j0 + jj) * p.v_row;
#pragma unroll
            for (int n = 0; n < ND; ++n) acc[n] = fmaf(pj, to_f32(vr[64 * n + lane]), acc[n]);
        }
    }
    T* out = reinterpret_cast<T*>(p.out) + row * p.out_row + h * p.out_head;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int n = 0; n < ND; ++n) out[64 * n + lane] = from_f32<T>(l == 0.0f ? 0.0f : acc[n] * inv);
    if (p.lse && lane == 0) p.lse[row * p.heads + h] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
}

}  // namespace vpe
