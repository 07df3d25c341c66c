// A projection that all rows share and the low-rank adapter of each row beside it (vpe_adapter_linear):
//   y_r = x_r W^T + bias + t_r B_a^T,   t_r = scale_a x_r A_a^T,   a = adapter[r]
//
// Two launches: the rows' low-rank values t, which need all of x_r, then the projection with t B_a^T on its accumulators.  t goes through the
// workspace: fp32, or for the matrix instructions of bf16 calls as an upper and a lower bf16 term (together 16 bits of the value: what the
// second product loses of the adapter's share is 2^-17 of it, less than a 128th of the result's own rounding).
#include <mutex>

#include "kernels.h"
#include "operators.h"

namespace vpe {
namespace {

int rank16(const vpe_adapter_linear_args& a) { return (a.rank + 15) / 16 * 16; }
// Rows up to which the projection is bound by its weight and read by many workgroups (skinny_kernel); more go to the tiled GEMM.
constexpr int SKINNY_ROWS = 64;

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

// t of few rows: a wave per row and rank index, 16 bytes a lane.  Whatever adapters the rows have, each adapter row is read once per row.
template <typename T, bool TERMS>
__global__ __launch_bounds__(256) void adapter_rows_kernel(const vpe_adapter_linear_args p, void* t, int r16) {
    const int lane = threadIdx.x & 63;
    const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), row = task / r16;
    const int j = (int)(task - row * r16);
    if (row >= p.rows) return;
    const int a = p.adapter[row], ld = TERMS && sizeof(T) == 2 ? 2 * r16 : r16;
    if (a < 0 || a >= p.adapters) return;                     // (its t is not looked at)
    float sum = 0.0f;
    if (j < p.rank) {
        constexpr int CE = Elem<T>::CE;
        const T* x = reinterpret_cast<const T*>(p.x) + row * p.x_row;
        const T* w = reinterpret_cast<const T*>(p.a) + ((int64_t)a * p.rank + j) * p.in_features;
        for (int k = lane * CE; k < p.in_features; k += 64 * CE) {
            float u[CE], v[CE];
            unpack<T>(ld_global_16(x + k), u);
            unpack<T>(ld_global_16(w + k), v);
#pragma unroll
            for (int i = 0; i < CE; ++i) sum = fmaf(u[i], v[i], sum);
        }
        sum = wave_sum(sum);
        if (p.scale) sum *= p.scale[a];
    }
    if (lane == 0) leave<T, TERMS>(t, row, ld, j, r16, sum);
}

// t of many rows: 32 rows a workgroup, their width shared by eight waves, 32 rank indices at a time, once for every adapter among the rows.
// Bound by reading x where rows of an adapter lie together.
template <typename T>
__global__ __launch_bounds__(512) void adapter_tiles_kernel(const vpe_adapter_linear_args p, void* t, int r16) {
    __shared__ __attribute__((aligned(16))) float part[8][32 * 32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 5, li = lane & 31, ld = sizeof(T) == 2 ? 2 * r16 : r16;
    const int row0 = blockIdx.x * 32, r = row0 + li < p.rows ? row0 + li : p.rows - 1;
    const int id = p.adapter[r], per = cdiv(p.in_features / 16, 8), k0 = wave * per * 16, k1 = k0 + per * 16 < p.in_features ? k0 + per * 16 : p.in_features;
    const T* x = reinterpret_cast<const T*>(p.x) + (int64_t)r * p.x_row + 8 * g;
    for (uint64_t todo = __ballot(id >= 0 && id < p.adapters); todo;) {
        const int a = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
        const uint64_t rows = __ballot(id == a);
        todo &= ~rows;
        const float scale = p.scale ? p.scale[a] : 1.0f;
        for (int j0 = 0; j0 < r16; j0 += 32) {
            const int j = j0 + li < p.rank ? j0 + li : p.rank - 1;
            const T* w = reinterpret_cast<const T*>(p.a) + ((int64_t)a * p.rank + j) * p.in_features + 8 * g;
            f32x16 c;
#pragma unroll
            for (int v = 0; v < 16; ++v) c[v] = 0.0f;
#pragma unroll 4
            for (int k = k0; k < k1; k += 16) {
                if constexpr (sizeof(T) == 2) {
                    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(w + k), *reinterpret_cast<const bf16x8*>(x + k), c, 0, 0, 0);
                } else {
                    const f32x4 w0 = *reinterpret_cast<const f32x4*>(w + k), w1 = *reinterpret_cast<const f32x4*>(w + k + 4);
                    const f32x4 x0 = *reinterpret_cast<const f32x4*>(x + k), x1 = *reinterpret_cast<const f32x4*>(x + k + 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(w0[e], x0[e], c, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(w1[e], x1[e], c, 0, 0, 0);
                }
            }
            // (lane: row li, rank indices 8 (v / 4) + 4 g + v % 4)
#pragma unroll
            for (int n = 0; n < 4; ++n) *reinterpret_cast<f32x4*>(&part[wave][((2 * n + g) * 32 + li) * 4]) = f32x4{c[4 * n], c[4 * n + 1], c[4 * n + 2], c[4 * n + 3]};
            __syncthreads();
            // two values a thread: rows by lane, so that the sums are read without bank conflicts
            const int row = (tid >> 1) & 31, q = tid >> 6, e0 = (tid & 1) * 2;
            float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
            for (int w8 = 0; w8 < 8; ++w8) {
                const float* at = &part[w8][(q * 32 + row) * 4 + e0];
                s0 += at[0];
                s1 += at[1];
            }
            const int jj = j0 + 4 * q + e0;
            if (((rows >> row) & 1) && row0 + row < p.rows && jj < r16) {
                leave<T, true>(t, row0 + row, ld, jj, r16, jj < p.rank ? s0 * scale : 0.0f);
                leave<T, true>(t, row0 + row, ld, jj + 1, r16, jj + 1 < p.rank ? s1 * scale : 0.0f);
            }
            __syncthreads();
        }
    }
}

// The projection of up to 16 RB rows: bound by reading the weight once.  A workgroup has 16 output columns, its eight waves share the
// width, and every wave's weight loads (16 bytes a lane, 16 columns x 64 bytes an instruction) go straight to registers, several on their way.
// The waves' sums meet in LDS; a thread then has one column of a row, adds the row's adapter in fp32 and stores.
template <typename T, int RB>
__global__ __launch_bounds__(512) void skinny_kernel(const vpe_adapter_linear_args p, const float* __restrict__ t, int r16) {
    constexpr int STEP = sizeof(T) == 2 ? 32 : 16;            // width of an instruction group (four lanes of 16 bytes)
    __shared__ __attribute__((aligned(16))) float part[8][RB * 256];
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
    // (in_features is a multiple of 64: whole steps; waves take them in turn)
#pragma unroll 4
    for (int k = wave * STEP; k < p.in_features; k += 8 * STEP) {
        const u32x4 a = ld_global_16(w + k);
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const u32x4 c = ld_global_16(x[b] + k);
            if constexpr (sizeof(T) == 2) {
                acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, c), acc[b], 0, 0, 0);
            } else {
                const f32x4 fa = __builtin_bit_cast(f32x4, a), fc = __builtin_bit_cast(f32x4, c);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[e], fc[e], acc[b], 0, 0, 0);
            }
        }
    }
    // (lane: row n of a block, columns 4 q .. 4 q + 3)
#pragma unroll
    for (int b = 0; b < RB; ++b) *reinterpret_cast<f32x4*>(&part[wave][(b * 16 + n) * 16 + 4 * q]) = acc[b];
    __syncthreads();
    for (int o = tid; o < RB * 256; o += 512) {
        const int row = o >> 4, c = col0 + (o & 15);
        if (row >= p.rows || c >= p.out_features) continue;
        float y = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) y += part[k][o];
        const int a = p.adapter ? p.adapter[row] : -1;
        if (a >= 0 && a < p.adapters) {
            const T* up = reinterpret_cast<const T*>(p.b) + ((int64_t)a * p.out_features + c) * p.rank;
            const float* low = t + (int64_t)row * r16;
            for (int j = 0; j < p.rank; j += 8) {
                float b[8];
                unpack<T>(ld_global_16(up + j), b);
                if (sizeof(T) == 4) unpack<T>(ld_global_16(up + j + 4), b + 4);
                const f32x4 l0 = *reinterpret_cast<const f32x4*>(low + j), l1 = *reinterpret_cast<const f32x4*>(low + j + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) y = fmaf(l0[e], b[e], y);
#pragma unroll
                for (int e = 0; e < 4; ++e) y = fmaf(l1[e], b[4 + e], y);
            }
        }
        if (p.bias) y += p.bias[c];
        if (p.out_f32) reinterpret_cast<float*>(p.out)[row * p.out_row + c] = y;
        else reinterpret_cast<T*>(p.out)[row * p.out_row + c] = from_f32<T>(y);
    }
}

template <typename T>
hipError_t launch(const vpe_adapter_linear_args& args, hipStream_t s) {
    vpe_adapter_linear_args a = args;
    if (a.adapters == 0 || !a.adapter) { a.adapters = 0; a.adapter = nullptr; }
    const int r16 = rank16(a);
    const bool skinny = a.rows <= SKINNY_ROWS;
    if (a.adapter) {
        const dim3 tasks((uint32_t)(((int64_t)a.rows * r16 + 3) / 4));
        if (skinny) hipLaunchKernelGGL((adapter_rows_kernel<T, false>), tasks, dim3(256), 0, s, a, a.workspace, r16);
        else if (a.rows <= 256) hipLaunchKernelGGL((adapter_rows_kernel<T, true>), tasks, dim3(256), 0, s, a, a.workspace, r16);
        else hipLaunchKernelGGL(adapter_tiles_kernel<T>, dim3(cdiv(a.rows, 32)), dim3(512), 0, s, a, a.workspace, r16);
        const hipError_t rc = hipGetLastError();
        if (rc != hipSuccess) return rc;
    }
    if (skinny) {
        const dim3 grid(cdiv(a.out_features, 16)), block(512);
        const float* t = reinterpret_cast<const float*>(a.workspace);
        switch (cdiv(a.rows, 16)) {
            case 1: hipLaunchKernelGGL((skinny_kernel<T, 1>), grid, block, 0, s, a, t, r16); break;
            case 2: hipLaunchKernelGGL((skinny_kernel<T, 2>), grid, block, 0, s, a, t, r16); break;
            case 3: hipLaunchKernelGGL((skinny_kernel<T, 3>), grid, block, 0, s, a, t, r16); break;
            default: hipLaunchKernelGGL((skinny_kernel<T, 4>), grid, block, 0, s, a, t, r16); break;
        }
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
