// A projection that all rows share and the low-rank adapter of each row beside it (vpe_adapter_linear):
//   y_r = x_r W^T + bias + t_r B_a^T,   t_r = scale_a x_r A_a^T,   a = adapter[r]
#include "common.h"
#include "operators.h"

namespace vpe {
namespace {

// t: a wave per row and rank index.
template <typename T>
__global__ __launch_bounds__(256) void adapter_down_kernel(const vpe_adapter_linear_args p, float* __restrict__ t) {
    const int lane = threadIdx.x & 63;
    const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), row = task / p.rank;
    const int j = (int)(task % p.rank);
    if (row >= p.rows) return;
    const int a = p.adapter[row];
    if (a < 0 || a >= p.adapters) return;                     // (its t is not looked at)
    const T* x = reinterpret_cast<const T*>(p.x) + row * p.x_row;
    const T* w = reinterpret_cast<const T*>(p.a) + ((int64_t)a * p.rank + j) * p.in_features;
    float sum = 0.0f;
    for (int k = lane; k < p.in_features; k += 64) sum = fmaf(to_f32(x[k]), to_f32(w[k]), sum);
    sum = wave_sum(sum);
    if (lane == 0) t[row * p.rank + j] = p.scale ? sum * p.scale[a] : sum;
}

template <typename T>
__global__ __launch_bounds__(256) void adapter_out_kernel(const vpe_adapter_linear_args p, const float* __restrict__ t) {
    const int col = blockIdx.y * 256 + threadIdx.x;
    const int64_t row = blockIdx.x;
    if (col >= p.out_features) return;
    const T* x = reinterpret_cast<const T*>(p.x) + row * p.x_row;
    const T* w = reinterpret_cast<const T*>(p.weight) + (int64_t)col * p.in_features;
    float sum = 0.0f;
    for (int k = 0; k < p.in_features; ++k) sum = fmaf(to_f32(x[k]), to_f32(w[k]), sum);
    if (p.bias) sum += p.bias[col];
    const int a = p.adapters > 0 && p.adapter ? p.adapter[row] : -1;
    if (a >= 0 && a < p.adapters) {
        const T* b = reinterpret_cast<const T*>(p.b) + ((int64_t)a * p.out_features + col) * p.rank;
        for (int k = 0; k < p.rank; ++k) sum = fmaf(t[row * p.rank + k], to_f32(b[k]), sum);
    }
    if (p.out_f32) reinterpret_cast<float*>(p.out)[row * p.out_row + col] = sum;
    else reinterpret_cast<T*>(p.out)[row * p.out_row + col] = from_f32<T>(sum);
}

template <typename T>
hipError_t launch(const vpe_adapter_linear_args& a, hipStream_t s) {
    float* t = reinterpret_cast<float*>(a.workspace);
    if (a.adapters > 0 && a.adapter) {
        hipLaunchKernelGGL(adapter_down_kernel<T>, dim3((uint32_t)(((int64_t)a.rows * a.rank + 3) / 4)), dim3(256), 0, s, a, t);
        const hipError_t rc = hipGetLastError();
        if (rc != hipSuccess) return rc;
    }
    hipLaunchKernelGGL(adapter_out_kernel<T>, dim3(a.rows, cdiv(a.out_features, 256)), dim3(256), 0, s, a, t);
    return hipGetLastError();
}

}  // namespace

uint64_t adapter_linear_workspace(const vpe_adapter_linear_args& a) { return a.adapters > 0 ? (uint64_t)a.rows * a.rank * 4 : 0; }

hipError_t launch_adapter_linear(const vpe_adapter_linear_args& a, hipStream_t s) { return a.dtype == VPE_BF16 ? launch<bf16>(a, s) : launch<float>(a, s); }

}  // namespace vpe
