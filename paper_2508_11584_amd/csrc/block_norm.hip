// What stands between two blocks, in one pass over the rows (vpe_block_norm):
//   y = post(branch) layer_scale gate_r,   out = residual_scale x + y,   normed = pre(out) (1 + scale_r) + shift_r
// post and pre: (v - mean) / sqrt(var + eps) gain + bias, the same without the mean, or v itself.
//
// Bound by HBM: a row is read once (x fp32, branch) and written once (out fp32, normed) and stays in registers between the reductions.
// The vectors of the width -- two gains, two biases, LayerScale, the request's gate, scale and shift -- are 32 bytes a column where the row
// itself is 12 of a bf16 call: read for every row they were most of the traffic (10992 rows of 1536: 67 us, folded 53).  A
// wave folds them into four (y = z A + B in front of the sum, z C + E behind it), keeps those in registers and takes several rows with them.
#include "common.h"
#include "operators.h"
#include "wave_sum.h"

namespace vpe {
namespace {

// Four columns of a row at any alignment of the type (the hardware takes wide accesses at element alignment).  The pack that holds the end of a
// row, `left` < 4 columns, is read as the row's last four and put right where it is used (settle): a branch of its own for it would wait for
// the row's other loads, and a row that is asked for early would be waited for at once.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x4_any __attribute__((ext_vector_type(4), aligned(2)));
template <typename T> struct Pack;
template <> struct Pack<float> { typedef f32x4_any type; };
template <> struct Pack<bf16> { typedef bf16x4_any type; };

template <bool TAIL, typename T>
__device__ __forceinline__ typename Pack<T>::type load_raw(const T* src, int left, int width) {
    if (TAIL && width < 4) {
        typename Pack<T>::type e = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) e[i] = src[i];
        return e;
    }
    return *reinterpret_cast<const typename Pack<T>::type*>(TAIL && left < 4 ? src - (4 - left) : src);
}
template <bool TAIL, typename T>
__device__ __forceinline__ void settle(typename Pack<T>::type e, int left, int width, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_f32((T)e[i]);
    if (TAIL && width >= 4 && left < 4) {
        const float a = v[1], b = v[2], c = v[3];              // the last `left` of the four, zeros behind them
        v[0] = left == 3 ? a : left == 2 ? b : c;
        v[1] = left == 3 ? b : left == 2 ? c : 0.0f;
        v[2] = left == 3 ? c : 0.0f;
        v[3] = 0.0f;
    }
}
template <bool TAIL, typename T>
__device__ __forceinline__ void load4(const T* src, int left, int width, float* v) { settle<TAIL, T>(load_raw<TAIL>(src, left, width), left, width, v); }
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

// A workgroup of WPR waves takes `rows_each` consecutive rows, one after the other; a lane has NP packs of four columns.  TAIL: the width is no
// multiple of four.
template <typename T, int WPR, int NP, bool TAIL>
__global__ __launch_bounds__(64 * WPR) void block_norm_kernel(const vpe_block_norm_args p, int rows_each) {
    constexpr int STEP = 256 * WPR;
    __shared__ float part[2 * WPR];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)blockIdx.x * rows_each, last = first + rows_each < p.rows ? first + rows_each : p.rows;
    const int c0 = threadIdx.x * 4, D = p.dim;
    int turn = 0;
    auto row_sum = [&](float v) {
        v = wave_total(v);
        if constexpr (WPR > 1) {
            // (two sets of places in turn: the next sum is written while a slow wave still reads this one)
            if (lane == 0) part[WPR * turn + wave] = v;
            __syncthreads();
            v = 0.0f;
#pragma unroll
            for (int w = 0; w < WPR; ++w) v += part[WPR * turn + w];
            turn ^= 1;
        }
        return v;
    };
    // f(pack, first column, columns from there to the row's end) for every pack that the lane has of a row
    auto packs = [&](auto&& f) {
        int width = D;
        if (TAIL) asm volatile("" : "+s"(width));             // (comparisons kept from one use to the next have no scalar registers)
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            const int c = c0 + n * STEP;
            if (c < width) f(n, c, width - c);
        }
    };
    const bool has_branch = p.branch != nullptr;
    float A[NP][4], B[NP][4], C[NP][4], E[NP][4];
    auto fold = [&](int req) {
        const bool mine = req >= 0 && req < p.requests;
        const int64_t at = (int64_t)req * D;
        auto column = [&](const float* v, int c, int left, float* into) {
            if (v) load4<TAIL>(v + c, left, D, into);
        };
        packs([&](int n, int c, int left) {
            float g[4] = {1, 1, 1, 1}, b[4] = {0, 0, 0, 0}, f[4] = {1, 1, 1, 1}, t[4] = {1, 1, 1, 1};
            if (has_branch) {
                if (p.post != VPE_NORM_NONE) { column(p.post_gain, c, left, g); column(p.post_bias, c, left, b); }
                column(p.layer_scale, c, left, f);
                if (mine && p.gate) column(p.gate + at, c, left, t);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) { A[n][i] = g[i] * (f[i] * t[i]); B[n][i] = b[i] * (f[i] * t[i]); }
            float g2[4] = {1, 1, 1, 1}, b2[4] = {0, 0, 0, 0}, m[4] = {0, 0, 0, 0}, a[4] = {0, 0, 0, 0};
            if (p.normed) {
                if (p.pre != VPE_NORM_NONE) { column(p.pre_gain, c, left, g2); column(p.pre_bias, c, left, b2); }
                if (mine && p.scale) column(p.scale + at, c, left, m);
                if (mine && p.shift) column(p.shift + at, c, left, a);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) { C[n][i] = g2[i] * (1.0f + m[i]); E[n][i] = fmaf(b2[i], 1.0f + m[i], a[i]); }
        });
    };
    // (columns past the row's end are zero in the first sum and stay out of the centred squares)
    auto standardise = [&](float (&v)[NP][4], int kind) {
        float mean = 0.0f, sum = 0.0f;
        if (kind == VPE_NORM_LAYER) {
#pragma unroll
            for (int n = 0; n < NP; ++n) sum += (v[n][0] + v[n][1]) + (v[n][2] + v[n][3]);
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
#pragma unroll
        for (int n = 0; n < NP; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[n][i] = (v[n][i] - mean) * rstd;
    };
    // a row's values as they come, asked for while the row before it is worked on (10992 rows of 1536, bf16: 53 us without, 41 with)
    typename Pack<T>::type next_y[NP];
    f32x4_any next_x[NP];
    int next_req = 0;
    auto ask = [&](int64_t row) {
        packs([&](int n, int c, int left) {
            if (has_branch) next_y[n] = load_raw<TAIL>(reinterpret_cast<const T*>(p.branch) + row * p.branch_row + c, left, D);
            next_x[n] = load_raw<TAIL>(p.x + row * p.x_row + c, left, D);
        });
        if (p.request) next_req = p.request[row];
    };
#pragma unroll
    for (int n = 0; n < NP; ++n) { next_y[n] = typename Pack<T>::type{0, 0, 0, 0}; next_x[n] = f32x4_any{0, 0, 0, 0}; }
    int have = 0;
    bool any = false;
    if (first < last) ask(first);
    for (int64_t row = first; row < last; ++row) {
        float x[NP][4], y[NP][4];
#pragma unroll
        for (int n = 0; n < NP; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[n][i] = y[n][i] = 0.0f;
        packs([&](int n, int, int left) {
            settle<TAIL, float>(next_x[n], left, D, x[n]);
            settle<TAIL, T>(next_y[n], left, D, y[n]);
        });
        const int req = __builtin_amdgcn_readfirstlane(next_req);
        if (row + 1 < last) ask(row + 1);
        if (!any || req != have) {
            fold(req);
            have = req;
            any = true;
        }
        if (has_branch && p.post != VPE_NORM_NONE) standardise(y, p.post);
        packs([&](int n, int c, int left) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[n][i] = fmaf(p.residual_scale, x[n][i], fmaf(y[n][i], A[n][i], B[n][i]));
            store4<TAIL>(p.out + row * p.out_row + c, left, x[n]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (TAIL && i >= left) x[n][i] = 0.0f;
        });
        if (!p.normed) continue;
        if (p.pre != VPE_NORM_NONE) standardise(x, p.pre);
        packs([&](int n, int c, int left) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[n][i] = fmaf(x[n][i], C[n][i], E[n][i]);
            store4<TAIL>(reinterpret_cast<T*>(p.normed) + row * p.normed_row + c, left, x[n]);
        });
    }
}

typedef void (*Kernel)(const vpe_block_norm_args, int);
template <typename T, bool TAIL, int WPR>
Kernel packs_of(int np) {
    return np <= 1 ? &block_norm_kernel<T, WPR, 1, TAIL> : np <= 2 ? &block_norm_kernel<T, WPR, 2, TAIL> : np <= 3 ? &block_norm_kernel<T, WPR, 3, TAIL> : &block_norm_kernel<T, WPR, 4, TAIL>;
}
template <typename T, bool TAIL>
Kernel kernel_for(int wpr, int np) {
    return wpr == 1 ? packs_of<T, TAIL, 1>(np) : wpr == 2 ? packs_of<T, TAIL, 2>(np) : wpr == 4 ? packs_of<T, TAIL, 4>(np) : packs_of<T, TAIL, 8>(np);
}

template <typename T>
hipError_t launch(const vpe_block_norm_args& a, hipStream_t s) {
    // As many waves a row as leave a lane four packs at most (three reductions across waves cost more than a pack: 10992 rows of 1536 with 2 / 4 /
    // 8 waves 38 / 44 / 70 us, 10992 of 1024 with 1 / 2 / 4 25 / 26 / 35), two where the width is no multiple of four (their registers: 2741
    // rows of 777 with 1 / 2 waves 12.6 / 11.1), and up to eight where the rows are too few to fill the chip.  2048 waves are what it holds
    // of them with a row asked for ahead (2048 / 4096 / 8192: 1536 38.0 / 41.0 / 39.2 us, 4096 rows of 4096 36.3 / 36.9 / 46.3).
    const bool tail = a.dim % 4 != 0;
    int wpr = 1;
    while (wpr < 8 && a.dim > (tail ? 512 : 1024) * wpr) wpr *= 2;
    while (wpr < 8 && a.dim > 256 * wpr && (int64_t)a.rows * wpr < 1024) wpr *= 2;
    const int np = cdiv(a.dim, 256 * wpr);
    const Kernel k = tail ? kernel_for<T, true>(wpr, np) : kernel_for<T, false>(wpr, np);
    const int each = cdiv(a.rows, 2048 / wpr);
    hipLaunchKernelGGL(k, dim3(cdiv(a.rows, each)), dim3(64 * wpr), 0, s, a, each);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_block_norm(const vpe_block_norm_args& a, hipStream_t s) { return a.dtype == VPE_BF16 ? launch<bf16>(a, s) : launch<float>(a, s); }

}  // namespace vpe
