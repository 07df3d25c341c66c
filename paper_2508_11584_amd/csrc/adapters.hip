// A projection that all rows share and the low-rank adapter of each row beside it (vpe_adapter_linear):
//   y_r = x_r W^T + bias + t_r B_a^T,   t_r = scale_a x_r A_a^T,   a = adapter[r]
//
// Two launches: the rows' low-rank values t, which need all of x_r, then the projection with t B_a^T on its accumulators.  t goes through the
// workspace: fp32, or for the matrix instructions of bf16 calls as an upper and a lower bf16 term (together 16 bits of the value: what the
// second product loses of the adapter's share is 2^-17 of it, less than a 128th of the result's own rounding).
#include <mutex>

#include "kernels.h"
#include "operators.h"
#include "wave_sum.h"

namespace vpe {
namespace {

int rank16(const vpe_adapter_linear_args& a) { return (a.rank + 15) / 16 * 16; }
// Rows up to which the projection goes to skinny_kernel, which reads the weight once with workgroups of 16 columns; beyond, x, read by every
// one of them, is most of what they load, and the tiled GEMM shares it among 64 columns.  us, skinny / tiled, bf16 and fp32, rank 16, 1536 x
// 4608 and 4096 x 4096: 17 rows 14.2 / 14.1, 26 / 45; 32 rows 16.0 / 14.1, 24.5 / 30.6; 48 rows 20.2 / 13.0, 34 / 29 and 23.1 / 22.8, 42.7 / 49.7;
// 64 rows 25 / 11.6, 43 / 26.4 and 27 / 22, 59 / 48.
template <typename T> constexpr int skinny_rows() { return sizeof(T) == 2 ? 16 : 32; }
// Rows up to which a wave makes one low-rank value (us a call, such waves / those of 4 x 8 values: 512 rows of 1536 20.7 / 25.7, 1000 33 / 37.5,
// 4000 86 / 78, of mixed adapters 112 / 110; 10992 rows, rank 32 275 / 218).
constexpr int ONE_VALUE_ROWS = 1024;
constexpr int WAVES = 8;            // of a workgroup that shares a width

template <typename T> __device__ __forceinline__ void unpack(const u32x4& raw, float* v) {
    T e[Elem<T>::CE];
    __builtin_memcpy(e, &raw, 16);
#pragma unroll
    for (int i = 0; i < Elem<T>::CE; ++i) v[i] = to_f32(e[i]);
}

// One low-rank value into the workspace: fp32 [rows][ld], or T = bf16 and `terms`: the two terms, `half` columns apart.
template <typename T, bool TERMS>
__device__ __forceinline__ void leave(void* t, int64_t row, int ld, int j, int half, float v) {
    if constexpr (TERMS && sizeof(T) == 2) {
        bf16* dst = reinterpret_cast<bf16*>(t) + row * ld + j;
        const bf16 upper = (bf16)v;
        dst[0] = upper;
        // (of an infinite value the rest is NaN: its upper term says all)
        dst[half] = v - (float)upper == v - (float)upper ? (bf16)(v - (float)upper) : (bf16)0.0f;
    } else {
        reinterpret_cast<float*>(t)[row * ld + j] = v;
    }
}

// Sum of eight (four) products of 16 bytes of two rows, added to `sum` in fp32.
template <typename T> __device__ __forceinline__ float dot16(const u32x4& a, const u32x4& b, float sum) {
    if constexpr (sizeof(T) == 2) {
        // (two exact products and their sum an instruction: no conversions)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = a[i], v = b[i];                // (a cast of the element itself takes the first)
            sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, u), __builtin_bit_cast(bf16x2, v), sum, false);
        }
    } else {
        const f32x4 u = __builtin_bit_cast(f32x4, a), v = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = fmaf(u[i], v[i], sum);
    }
    return sum;
}

// t: a wave has R rows and J rank indices, 16 bytes of each a lane at a time, once for every adapter among its rows.  One of each for few rows:
// as many waves as there are values, and an adapter is read for the rows that have it; four rows and eight indices for many: twelve
// loads make thirty-two values where one of each makes one of two.
template <typename T, bool TERMS, int R, int J>
__global__ __launch_bounds__(256) void adapter_down_kernel(const vpe_adapter_linear_args p, void* t, int r16) {
    constexpr int CE = Elem<T>::CE;
    const int lane = threadIdx.x & 63, ld = TERMS && sizeof(T) == 2 ? 2 * r16 : r16, per_row = r16 / J;
    const int64_t task = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row0 = task / per_row * R;
    const int j0 = (int)(task % per_row) * J;
    if (row0 >= p.rows) return;
    const T* x[R];
    int id[R];
#pragma unroll
    for (int n = 0; n < R; ++n) {
        const int64_t r = row0 + n < p.rows ? row0 + n : p.rows - 1;
        x[n] = reinterpret_cast<const T*>(p.x) + r * p.x_row;
        id[n] = row0 + n < p.rows ? __builtin_amdgcn_readfirstlane(p.adapter[r]) : -1;
    }
#pragma unroll
    for (int first = 0; first < R; ++first) {
        const int a = id[first];
        if (a < 0 || a >= p.adapters) continue;               // (its t is not looked at)
        bool done = false;
#pragma unroll
        for (int n = 0; n < first; ++n) done = done || id[n] == a;
        if (done) continue;
        const T* w[J];
#pragma unroll
        for (int j = 0; j < J; ++j) w[j] = reinterpret_cast<const T*>(p.a) + ((int64_t)a * p.rank + (j0 + j < p.rank ? j0 + j : p.rank - 1)) * p.in_features;
        float sum[R][J];
#pragma unroll
        for (int n = 0; n < R; ++n)
#pragma unroll
            for (int j = 0; j < J; ++j) sum[n][j] = 0.0f;
        for (int k = lane * CE; k < p.in_features; k += 64 * CE) {
            u32x4 xv[R], wv[J];
#pragma unroll
            for (int n = 0; n < R; ++n) xv[n] = ld_global_16(x[n] + k);
#pragma unroll
            for (int j = 0; j < J; ++j) wv[j] = ld_global_16(w[j] + k);
#pragma unroll
            for (int n = 0; n < R; ++n)
#pragma unroll
                for (int j = 0; j < J; ++j) sum[n][j] = dot16<T>(xv[n], wv[j], sum[n][j]);
        }
        const float scale = p.scale ? p.scale[a] : 1.0f;
#pragma unroll
        for (int n = 0; n < R; ++n) {
            if (id[n] != a) continue;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const float v = wave_total(sum[n][j]);
                if (lane == 0) leave<T, TERMS>(t, row0 + n, ld, j0 + j, r16, j0 + j < p.rank ? v * scale : 0.0f);
            }
        }
    }
}

// The projection of up to 16 RB rows: bound by reading the weight once.  A workgroup has 16 output columns, its eight waves share the
// width, and every wave's weight loads (16 bytes a lane, 16 columns x 64 bytes an instruction) go straight to registers, four or eight on
// their way.
// The waves' sums meet in LDS; a thread then has one column of a row, adds the row's adapter in fp32 and stores.
template <typename T, int RB>
__global__ __launch_bounds__(512, 4) void skinny_kernel(const vpe_adapter_linear_args p, const float* __restrict__ t, int r16) {
    constexpr int STEP = sizeof(T) == 2 ? 32 : 16;            // width of an instruction group (four lanes of 16 bytes)
    __shared__ __attribute__((aligned(16))) float part[WAVES][RB * 256];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col0 = blockIdx.x * 16, n = lane & 15, q = lane >> 4;
    const int col = col0 + n < p.out_features ? col0 + n : p.out_features - 1;
    const T* w = reinterpret_cast<const T*>(p.weight) + (int64_t)col * p.in_features + q * Elem<T>::CE;
    const T* x[RB];
    f32x4 acc[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = 16 * b + n < p.rows ? 16 * b + n : p.rows - 1;
        x[b] = reinterpret_cast<const T*>(p.x) + (int64_t)r * p.x_row + q * Elem<T>::CE;
        acc[b] = f32x4{0, 0, 0, 0};
    }
    // (in_features is a multiple of 64: whole steps; waves take them in turn, AHEAD of them asked for before the first is used)
    constexpr int AHEAD = RB == 1 ? 8 : 4;
    u32x4 wv[AHEAD], xv[AHEAD][RB];
    auto ask = [&](int k) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int at = k + u * WAVES * STEP < p.in_features ? k + u * WAVES * STEP : k;
            wv[u] = ld_global_16(w + at);
#pragma unroll
            for (int b = 0; b < RB; ++b) xv[u][b] = ld_global_16(x[b] + at);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    const int k0 = wave * STEP;
    if (k0 < p.in_features) ask(k0);
    // the adapters' share of the values that this thread will store, bias included: its loads come behind the weight's first ones, not behind
    // the product
    constexpr int OUT = (RB * 256 + 64 * WAVES - 1) / (64 * WAVES);
    float extra[OUT];
#pragma unroll
    for (int n = 0; n < OUT; ++n) {
        const int o = tid + n * 64 * WAVES, row = o >> 4, c = col0 + (o & 15);
        extra[n] = 0.0f;
        if (o >= RB * 256 || row >= p.rows || c >= p.out_features) continue;
        const int a = p.adapter ? p.adapter[row] : -1;
        if (p.bias) extra[n] = p.bias[c];
        if (a < 0 || a >= p.adapters) continue;
        const T* up = reinterpret_cast<const T*>(p.b) + ((int64_t)a * p.out_features + c) * p.rank;
        const float* low = t + (int64_t)row * r16;
        float sum = 0.0f;
#pragma unroll 2
        for (int j = 0; j < p.rank; j += 8) {
            float b[8];
            unpack<T>(ld_global_16(up + j), b);
            if (sizeof(T) == 4) unpack<T>(ld_global_16(up + j + 4), b + 4);
            const f32x4 l0 = *reinterpret_cast<const f32x4*>(low + j), l1 = *reinterpret_cast<const f32x4*>(low + j + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fmaf(l0[e], b[e], sum);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fmaf(l1[e], b[4 + e], sum);
        }
        extra[n] += sum;
    }
    for (int k = k0; k < p.in_features; k += AHEAD * WAVES * STEP) {
        if (k != k0) ask(k);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (k + u * WAVES * STEP >= p.in_features) break;
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                if constexpr (sizeof(T) == 2) {
                    acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wv[u]), __builtin_bit_cast(bf16x8, xv[u][b]), acc[b], 0, 0, 0);
                } else {
                    const f32x4 fa = __builtin_bit_cast(f32x4, wv[u]), fc = __builtin_bit_cast(f32x4, xv[u][b]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[e], fc[e], acc[b], 0, 0, 0);
                }
            }
        }
    }
    // (lane: row n of a block, columns 4 q .. 4 q + 3)
#pragma unroll
    for (int b = 0; b < RB; ++b) *reinterpret_cast<f32x4*>(&part[wave][(b * 16 + n) * 16 + 4 * q]) = acc[b];
    __syncthreads();
#pragma unroll
    for (int n2 = 0; n2 < OUT; ++n2) {
        const int o = tid + n2 * 64 * WAVES, row = o >> 4, c = col0 + (o & 15);
        if (o >= RB * 256 || row >= p.rows || c >= p.out_features) continue;
        float y = 0.0f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) y += part[k][o];
        y += extra[n2];
        if (p.out_f32) reinterpret_cast<float*>(p.out)[row * p.out_row + c] = y;
        else reinterpret_cast<T*>(p.out)[row * p.out_row + c] = from_f32<T>(y);
    }
}

template <typename T>
hipError_t launch(const vpe_adapter_linear_args& args, hipStream_t s) {
    vpe_adapter_linear_args a = args;
    if (a.adapters == 0 || !a.adapter) { a.adapters = 0; a.adapter = nullptr; }
    const int r16 = rank16(a);
    const bool skinny = a.rows <= skinny_rows<T>();
    if (a.adapter) {
        auto waves = [&](int rows, int indices) { return dim3((uint32_t)(((int64_t)cdiv(a.rows, rows) * (r16 / indices) + 3) / 4)); };
        if (skinny) hipLaunchKernelGGL((adapter_down_kernel<T, false, 1, 1>), waves(1, 1), dim3(256), 0, s, a, a.workspace, r16);
        else if (a.rows <= ONE_VALUE_ROWS) hipLaunchKernelGGL((adapter_down_kernel<T, true, 1, 1>), waves(1, 1), dim3(256), 0, s, a, a.workspace, r16);
        else hipLaunchKernelGGL((adapter_down_kernel<T, true, 4, 8>), waves(4, 8), dim3(256), 0, s, a, a.workspace, r16);
        const hipError_t rc = hipGetLastError();
        if (rc != hipSuccess) return rc;
    }
    if (skinny) {
        const dim3 grid(cdiv(a.out_features, 16)), block(64 * WAVES);
        const float* t = reinterpret_cast<const float*>(a.workspace);
        if (sizeof(T) == 2 || a.rows <= 16) hipLaunchKernelGGL((skinny_kernel<T, 1>), grid, block, 0, s, a, t, r16);
        else hipLaunchKernelGGL((skinny_kernel<T, sizeof(T) == 2 ? 1 : 2>), grid, block, 0, s, a, t, r16);
        return hipGetLastError();
    }
    GemmArgs m{};
    m.A = a.x; m.lda = a.x_row; m.W = a.weight; m.bias = a.bias; m.M = a.rows; m.N = a.out_features; m.K = a.in_features;
    m.a_rpi = m.o_rpi = a.rows;
    m.epi = EPI_ADAPT; m.act = ACT_NONE; m.out = a.out; m.out_f32 = a.out_f32; m.ldo = a.out_row;
    m.adapter = a.adapter; m.adapters = a.adapters; m.rank = a.rank; m.up = a.b; m.low = a.workspace; m.low_ld = sizeof(T) == 2 ? 2 * r16 : r16;
    if (!a.adapter) m.adapters = 0;
    return launch_gemm(sizeof(T) == 2, m, A_PLAIN, s);
}

// LDS opt-in of the GEMM's tilings, once for every device (as when an engine is created there).
hipError_t configure_once() {
    static std::mutex mutex;
    static bool done[64] = {};
    int device = 0;
    hipError_t rc = hipGetDevice(&device);
    if (rc != hipSuccess) return rc;
    if (device < 0 || device >= 64) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(mutex);
    if (done[device]) return hipSuccess;
    for (hipError_t (*f)() : {configure_gemm, configure_gemm_bf16, configure_gemm_f32}) {
        rc = f();
        if (rc != hipSuccess) return rc;
    }
    done[device] = true;
    return hipSuccess;
}

}  // namespace

// bf16 keeps two bf16 terms where fp32 keeps a value: the same bytes either way.
uint64_t adapter_linear_workspace(const vpe_adapter_linear_args& a) { return a.adapters > 0 ? (uint64_t)a.rows * rank16(a) * 4 : 0; }

hipError_t launch_adapter_linear(const vpe_adapter_linear_args& a, hipStream_t s) {
    const hipError_t rc = configure_once();
    if (rc != hipSuccess) return rc;
    return a.dtype == VPE_BF16 ? launch<bf16>(a, s) : launch<float>(a, s);
}

}  // namespace vpe
