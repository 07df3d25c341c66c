// What stands between two blocks, in one pass over the rows (vpe_block_norm):
//   y = post(branch) layer_scale gate_r,   out = residual_scale x + y,   normed = pre(out) (1 + scale_r) + shift_r
// post and pre: (v - mean) / sqrt(var + eps) gain + bias, the same without the mean, or v itself.
//
// Bound by HBM: a row is read once (x fp32, branch) and written once (out fp32, normed) and stays in registers between the two
// reductions; vectors of the width and the request's gates come from the caches.
#include "common.h"
#include "operators.h"

namespace vpe {
namespace {

// Four columns of a row at any alignment of the type (the hardware takes wide accesses at element alignment); of the pack that holds a
// row's end the `left` columns that exist, zero behind them.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x4_any __attribute__((ext_vector_type(4), aligned(2)));
template <typename T> struct Pack;
template <> struct Pack<float> { typedef f32x4_any type; };
template <> struct Pack<bf16> { typedef bf16x4_any type; };

template <bool TAIL, typename T>
__device__ __forceinline__ void load4(const T* src, int left, float* v) {
    if (!TAIL || left >= 4) {
        const typename Pack<T>::type e = *reinterpret_cast<const typename Pack<T>::type*>(src);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to_f32((T)e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < left ? to_f32(src[i]) : 0.0f;
    }
}
template <bool TAIL, typename T>
__device__ __forceinline__ void store4(T* dst, int left, const float* v) {
    if (!TAIL || left >= 4) {
        typename Pack<T>::type e;
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = from_f32<T>(v[i]);
        *reinterpret_cast<typename Pack<T>::type*>(dst) = e;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) dst[i] = from_f32<T>(v[i]);
    }
}

constexpr int PASSES = 8;        // packs of a row that a lane holds at most

// A row by WPR waves.  TAIL: the width is no multiple of four.
template <typename T, int WPR, bool TAIL>
__global__ __launch_bounds__(256) void block_norm_kernel(const vpe_block_norm_args p) {
    constexpr int STEP = 256 * WPR;
    __shared__ float part[8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = WPR == 4 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
    if (row >= p.rows) return;                                       // (whole rows: WPR waves leave together)
    const int c0 = (WPR == 4 ? threadIdx.x : lane) * 4, D = p.dim;
    int turn = 0;
    auto row_sum = [&](float v) {
        v = wave_sum(v);
        if constexpr (WPR == 4) {
            // (two sets of places in turn: the next sum is written while a slow wave still reads this one)
            if (lane == 0) part[4 * turn + wave] = v;
            __syncthreads();
            v = (part[4 * turn] + part[4 * turn + 1]) + (part[4 * turn + 2] + part[4 * turn + 3]);
            turn ^= 1;
        }
        return v;
    };
    float x[PASSES][4], y[PASSES][4];
    // f(pass, first column, columns from there to the row's end) for every pack that the lane has of the row
    auto packs = [&](auto&& f) {
#pragma unroll
        for (int n = 0; n < PASSES; ++n) {
            const int c = c0 + n * STEP;
            if (n * STEP < D && c < D) f(n, c, D - c);
        }
    };
#pragma unroll
    for (int n = 0; n < PASSES; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[n][i] = y[n][i] = 0.0f;
    const bool has_branch = p.branch != nullptr;
    packs([&](int n, int c, int left) {
        if (has_branch) load4<TAIL>(reinterpret_cast<const T*>(p.branch) + row * p.branch_row + c, left, y[n]);
        load4<TAIL>(p.x + row * p.x_row + c, left, x[n]);
    });
    const int req = p.request ? p.request[row] : 0;
    const bool mine = req >= 0 && req < p.requests;
    const float* gate = mine && p.gate ? p.gate + (int64_t)req * D : nullptr;
    const float* scale = mine && p.scale ? p.scale + (int64_t)req * D : nullptr;
    const float* shift = mine && p.shift ? p.shift + (int64_t)req * D : nullptr;
    auto multiply = [&](float* v, const float* by, int c, int left, float plus) {
        if (!by) return;
        float g[4];
        load4<TAIL>(by + c, left, g);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= plus + g[i];
    };
    auto add = [&](float* v, const float* what, int c, int left) {
        if (!what) return;
        float g[4];
        load4<TAIL>(what + c, left, g);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += g[i];
    };
    // (columns past the row's end are zero in the first sum and stay out of the centred squares)
    auto normalise = [&](float (&v)[PASSES][4], int kind, const float* gain, const float* bias) {
        float mean = 0.0f, sum = 0.0f;
        if (kind == VPE_NORM_LAYER) {
#pragma unroll
            for (int n = 0; n < PASSES; ++n) sum += (v[n][0] + v[n][1]) + (v[n][2] + v[n][3]);
            mean = row_sum(sum) / D;
        }
        sum = 0.0f;
        packs([&](int n, int, int left) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float d = v[n][i] - mean;
                if (!TAIL || i < left) sum += d * d;
            }
        });
        const float rstd = 1.0f / sqrtf(row_sum(sum) / D + p.eps);
        packs([&](int n, int c, int left) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[n][i] = (v[n][i] - mean) * rstd;
            multiply(v[n], gain, c, left, 0.0f);
            add(v[n], bias, c, left);
        });
    };
    if (has_branch && p.post != VPE_NORM_NONE) normalise(y, p.post, p.post_gain, p.post_bias);
    packs([&](int n, int c, int left) {
        multiply(y[n], p.layer_scale, c, left, 0.0f);
        multiply(y[n], gate, c, left, 0.0f);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[n][i] = p.residual_scale * x[n][i] + y[n][i];
        store4<TAIL>(p.out + row * p.out_row + c, left, x[n]);
    });
    if (!p.normed) return;
    if (TAIL) packs([&](int n, int, int left) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[n][i] = i < left ? x[n][i] : 0.0f;
    });
    if (p.pre != VPE_NORM_NONE) normalise(x, p.pre, p.pre_gain, p.pre_bias);
    packs([&](int n, int c, int left) {
        multiply(x[n], scale, c, left, 1.0f);
        add(x[n], shift, c, left);
        store4<TAIL>(reinterpret_cast<T*>(p.normed) + row * p.normed_row + c, left, x[n]);
    });
}

template <typename T>
hipError_t launch(const vpe_block_norm_args& a, hipStream_t s) {
    const bool wide = a.dim > 256 * PASSES, tail = a.dim % 4 != 0;
    typedef void (*Kernel)(const vpe_block_norm_args);
    const Kernel k = wide ? (tail ? &block_norm_kernel<T, 4, true> : &block_norm_kernel<T, 4, false>) : (tail ? &block_norm_kernel<T, 1, true> : &block_norm_kernel<T, 1, false>);
    hipLaunchKernelGGL(k, dim3(wide ? a.rows : cdiv(a.rows, 4)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_block_norm(const vpe_block_norm_args& a, hipStream_t s) { return a.dtype == VPE_BF16 ? launch<bf16>(a, s) : launch<float>(a, s); }

}  // namespace vpe
