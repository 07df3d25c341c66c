// Attention over packed sequences with capped scores, distances and prefix masks (vpe_attention).
//
//   s_ij = scale q_i.k_j;  cap > 0: s = cap tanh(s / cap);  s -= slope_h dist(i, j)
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(s_ij - m_i) over the keys j that row i sees,  lse_i = m_i + log sum_j p_ij
#pragma once
#include "attention.h"
#include "common.h"
#include "gemm_dma.h"
#include "split3.h"
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

// What a call's launches share beyond its arguments.
struct SeqAttnGrid {
    int blocks, packed, splits, per_split, chunk;
    float *part_o, *part_ml;     // splits > 1: [split][q_rows][heads][D] sums against the part's reference, [split][q_rows][heads][2] (reference, sum)
};

// A kernel's argument at `offset`, read from its argument segment where this stands.
template <typename A>
__device__ __forceinline__ A kernel_args(int offset) {
    auto base = (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(base));
    A a;
    __builtin_memcpy(&a, (const char*)(base + offset), sizeof a);
    return a;
}

// Keys that the row at `place` sees: 0 .. limit - 1.  (Causal rows see what is before them and the prefix: one range.)
__device__ __forceinline__ int key_limit(const vpe_attention_args& p, const Seq& sq, int place) {
    if (!p.causal) return sq.nk;
    const int n = place + 1 > sq.prefix ? place + 1 : sq.prefix;
    return n < 0 ? 0 : n < sq.nk ? n : sq.nk;
}

// Leaves columns c .. c + N - 1 of a row: the result, or with several parts of the keys the part's sum.
template <int N, typename T>
__device__ __forceinline__ void store_columns(T* dst, const float* v) {
    T e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = from_f32<T>(v[i]);
    typedef uint32_t Raw __attribute__((ext_vector_type(N * sizeof(T) / 4)));
    Raw raw;
    __builtin_memcpy(&raw, e, sizeof raw);
    *reinterpret_cast<Raw*>(dst) = raw;
}
__device__ __forceinline__ int64_t part_row(const vpe_attention_args& p, int64_t row, int h, int split) { return ((int64_t)split * p.q_rows + row) * p.heads + h; }
template <typename T>
__device__ __forceinline__ void store_stats(const vpe_attention_args& p, const SeqAttnGrid& g, int64_t row, int h, int split, float m, float l) {
    if (g.splits > 1) *reinterpret_cast<f32x2*>(g.part_ml + 2 * part_row(p, row, h, split)) = f32x2{m, l};
    else if (p.lse) p.lse[row * p.heads + h] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
}

// Row i of sequence `sq`, head h, over the keys j_begin .. j_end - 1, by one wave in plain fp32: 64 keys at a time, a lane has a key's
// score and then one or two columns of the result.  Keys that the row does not see are never read, so nothing they hold can reach the
// result, and infinite or NaN scores and values come out as the definition has them: the tiled kernel hands the rows over here whose sums
// are not finite.  (A call of nothing but such rows takes 80-160 times as long as one of none: ViT-B 518x518 2.7 ms.)
template <typename T, int D>
__device__ __forceinline__ void attention_row(const vpe_attention_args& p, const SeqAttnGrid& g, const Seq& sq, int i, int h, int j_begin, int j_end, int split, int lane) {
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
    const int limit = key_limit(p, sq, place), end = limit < j_end ? limit : j_end;
    for (int j0 = j_begin; j0 < end; j0 += 64) {
        const int j = j0 + lane < end ? j0 + lane : end - 1, n_here = end - j0 < 64 ? end - j0 : 64;
        float s = 0.0f;
        const T* kr = k + (int64_t)j * p.k_row;
#pragma unroll
        for (int n = 0; n < ND; ++n)
#pragma unroll 1
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
            const f32x2 to = *reinterpret_cast<const f32x2*>(p.k_coords + 2 * (int64_t)(sq.k0 + j));
            const float dy = at[0] - to[0], dx = at[1] - to[1];
            s -= slope * sqrtf(dy * dy + dx * dx);
        } else if (p.slopes) {
            s -= slope * fabsf((float)(place - j));
        }
        s = lane < n_here ? s * LOG2E : -INFINITY;
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
        for (int jj = 0; jj < n_here; ++jj) {
            const float pj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(e), jj));
            const T* vr = v + (int64_t)(j0 + jj) * p.v_row;
#pragma unroll
            for (int n = 0; n < ND; ++n) acc[n] = fmaf(pj, to_f32(vr[64 * n + lane]), acc[n]);
        }
    }
    const float inv = g.splits > 1 ? 1.0f : 1.0f / l;
#pragma unroll
    for (int n = 0; n < ND; ++n) {
        const float r = l == 0.0f ? 0.0f : acc[n] * inv;
        if (g.splits > 1) g.part_o[part_row(p, row, h, split) * D + 64 * n + lane] = r;
        else reinterpret_cast<T*>(p.out)[row * p.out_row + h * p.out_head + 64 * n + lane] = from_f32<T>(r);
    }
    if (lane == 0) store_stats<T>(p, g, row, h, split, m, l);
}

// --- matrix pieces: 32 x 32 blocks, 16 k elements a step; a lane (li = lane % 32, h = lane / 32) gives row li's eight elements
// 8 h .. 8 h + 7 of a step, and holds of a result column li rows 8 (v / 4) + 4 h + v % 4, v = 0 .. 15.
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char LdsByte;

template <typename T, int D> struct SeqMma;

template <int D> struct SeqMma<bf16, D> {
    typedef bf16x8 Frag;
    static constexpr int ROWB = 2 * D;                // bytes of a tile row; 16-byte chunks are exchanged by the row:
    // 16 consecutive rows reading one chunk of the keys fall on different banks;
    static __device__ __forceinline__ int k_swz(int r) { return D == 64 ? (r >> 1) & 7 : r & 15; }
    // four consecutive rows reading the same 64 bytes of the values do (the transposing read below)
    static __device__ __forceinline__ int v_swz(int r) { return D == 64 ? ((r >> 1) & 1) << 2 : (r & 3) << 2; }
    static __device__ __forceinline__ Frag load(const bf16* src) { return *reinterpret_cast<const bf16x8*>(src); }
    static __device__ __forceinline__ Frag k_frag(const char* tile, int row, int ks, int g) {
        return *reinterpret_cast<const bf16x8*>(tile + row * ROWB + (((2 * ks + g) ^ k_swz(row)) << 4));
    }
    // Values as the second product's first operand: of columns 32 d + li the keys 16 st + 4 g .. + 3 and 16 st + 8 + 4 g .. + 3 (where a score
    // block's column has its probabilities).  ds_read_b64_tr_b16 gives lane i of 16 column i of the four rows whose 32 bytes those lanes
    // address.  Eight reads and the wait for them are one block of assembly: for the builtin the compiler waits for all loads into the LDS
    // that are under way, the next tile's.  A block holds STEPS steps of 16 keys, from step `st` on.
    static constexpr int STEPS = D == 64 ? 2 : 1;
    struct Values { uint32_t at[D / 32]; };              // LDS address of the lane's read of tile row 0, by column block
    static __device__ __forceinline__ Values values(const char* tile, int lane) {
        const int t = lane & 15, row = 4 * (lane >> 5) + (t >> 2);
        Values v;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
            const int chunk = 4 * d + 2 * ((lane >> 4) & 1) + ((t >> 1) & 1);
            v.at[d] = (uint32_t)(uintptr_t)(LdsByte*)tile + row * ROWB + ((chunk ^ v_swz(row)) << 4) + (t & 1) * 8;      // (rows 8 apart have the same exchange)
        }
        return v;
    }
    template <int ST>
    static __device__ __forceinline__ void v_frags(const Values& a, Frag (&f)[STEPS][D / 32]) {
        constexpr int Z = 16 * ST * ROWB;
        u32x2 r[8];
        if constexpr (D == 64) {
            asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%c10\n\tds_read_b64_tr_b16 %1, %8 offset:%c11\n\t"
                         "ds_read_b64_tr_b16 %2, %9 offset:%c10\n\tds_read_b64_tr_b16 %3, %9 offset:%c11\n\t"
                         "ds_read_b64_tr_b16 %4, %8 offset:%c12\n\tds_read_b64_tr_b16 %5, %8 offset:%c13\n\t"
                         "ds_read_b64_tr_b16 %6, %9 offset:%c12\n\tds_read_b64_tr_b16 %7, %9 offset:%c13\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
                         : "v"(a.at[0]), "v"(a.at[1]), "n"(Z), "n"(Z + 8 * ROWB), "n"(Z + 16 * ROWB), "n"(Z + 24 * ROWB)
                         : "memory");
        } else {
            asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%c12\n\tds_read_b64_tr_b16 %1, %8 offset:%c13\n\t"
                         "ds_read_b64_tr_b16 %2, %9 offset:%c12\n\tds_read_b64_tr_b16 %3, %9 offset:%c13\n\t"
                         "ds_read_b64_tr_b16 %4, %10 offset:%c12\n\tds_read_b64_tr_b16 %5, %10 offset:%c13\n\t"
                         "ds_read_b64_tr_b16 %6, %11 offset:%c12\n\tds_read_b64_tr_b16 %7, %11 offset:%c13\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
                         : "v"(a.at[0]), "v"(a.at[1]), "v"(a.at[2]), "v"(a.at[3]), "n"(Z), "n"(Z + 8 * ROWB)
                         : "memory");
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) f[n / (D / 32)][n % (D / 32)] = __builtin_bit_cast(bf16x8, u32x4{r[2 * n][0], r[2 * n][1], r[2 * n + 1][0], r[2 * n + 1][1]});
    }
    static __device__ __forceinline__ Frag probs(const float* e) {
        bf16x8 b;
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = (bf16)e[i];
        return b;
    }
    static __device__ __forceinline__ f32x16 mma(const Frag& a, const Frag& b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

// fp32: three bf16 terms per operand (split3.h), six products.
template <int D> struct SeqMma<float, D> {
    typedef Split3 Frag;
    static constexpr int ROWB = 4 * D;
    // (the values are read element by element, two keys four rows apart at once: they fall on different halves of the banks)
    static __device__ __forceinline__ int k_swz(int r) { return (r & 3) | (r & 4) << 1 | (r & 8) >> 1; }
    static __device__ __forceinline__ int v_swz(int r) { return k_swz(r); }
    static __device__ __forceinline__ Frag load(const float* src) { return split3(*reinterpret_cast<const f32x4*>(src), *reinterpret_cast<const f32x4*>(src + 4)); }
    static __device__ __forceinline__ Frag k_frag(const char* tile, int row, int ks, int g) {
        const char* at = tile + row * ROWB;
        const int c = 4 * ks + 2 * g, sw = k_swz(row);
        return split3(*reinterpret_cast<const f32x4*>(at + ((c ^ sw) << 4)), *reinterpret_cast<const f32x4*>(at + (((c + 1) ^ sw) << 4)));
    }
    static constexpr int STEPS = 1;
    struct Values { const char* tile; int lane; };
    static __device__ __forceinline__ Values values(const char* tile, int lane) { return {tile, lane}; }
    template <int ST>
    static __device__ __forceinline__ void v_frags(const Values& a, Frag (&f)[1][D / 32]) {
        const int li = a.lane & 31, g = a.lane >> 5;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
            f32x4 e[2];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = 16 * ST + 8 * n + 4 * g + i;
                    e[n][i] = *reinterpret_cast<const float*>(a.tile + row * ROWB + (((8 * d + (li >> 2)) ^ v_swz(row)) << 4) + (li & 3) * 4);
                }
            f[0][d] = split3(e[0], e[1]);
        }
    }
    static __device__ __forceinline__ Frag probs(const float* e) { return split3(f32x4{e[0], e[1], e[2], e[3]}, f32x4{e[4], e[5], e[6], e[7]}); }
    static __device__ __forceinline__ f32x16 mma(const Frag& a, const Frag& b, f32x16 c) {
#pragma unroll
        for (int t = 0; t < 6; ++t) c = split_mma(t, a, b, c);
        return c;
    }
};

// What lowers a score between the two products besides a cap: nothing, distances in a line, distances between coordinates.
enum { DIST_NONE = 0, DIST_LINE = 1, DIST_GRID = 2 };

template <typename T, int D, int KT, int KW, int DIST>
constexpr int seq_stage_bytes() { return KW * (2 * KT * SeqMma<T, D>::ROWB + (DIST == DIST_GRID ? KT * 8 : 0)); }
template <typename T, int D, int KT, int QW, int KW, int DIST>
constexpr int seq_lds_bytes() {
    const int stages = 2 * seq_stage_bytes<T, D, KT, KW, DIST>(), merge = KW > 1 ? QW * KW * (32 * (D + 2) * 4 + 4) : 0;
    return stages > merge ? stages : merge;
}

// A workgroup takes 32 QW consecutive rows of a sequence and key head and the keys of one part; a row is a query and one of the G =
// heads / kv_heads query heads that read the key head (row r: query r / G, head r % G), so those share every tile.  Wave (qw, kw) of QW x KW has 32
// of the rows and every KW-th tile; a row's KW results meet in LDS and are added in a fixed order.
// A wave computes scores transposed, S^T = K Q^T: a lane holds half of one row's scores, reductions over the keys stay in the lane but for one
// exchange, and the probabilities are the second product's operand, O^T = V^T P^T, as they lie.
// An instantiation per kind of score (with all of them behind run-time branches a tile of slopes alone took twice a plain one's time: ViT-B 518x518 32
// us, so 28).
template <typename T, int D, int KT, int QW, int KW, bool CAP, int DIST, int OCC>
__global__ __launch_bounds__(64 * QW * KW, OCC) void seq_attention_kernel(const vpe_attention_args p, const SeqAttnGrid grid) {
    using M = SeqMma<T, D>;
    typedef typename M::Frag Frag;
    constexpr bool PLAIN = !CAP && DIST == DIST_NONE;
    constexpr int NW = QW * KW, ROWB = M::ROWB, TILE = KT * ROWB, OWN = 2 * TILE + (DIST == DIST_GRID ? KT * 8 : 0), STAGE = KW * OWN;
    constexpr int NB = KT / 32, DB = D / 32, KS = D / 16, CE = Elem<T>::CE;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int qw = wave % QW, kw = wave / QW, g = lane >> 5, li = lane & 31;
    const int G = p.heads / p.kv_heads;

    // --- which rows.  Runs of `chunk` row blocks that read the same keys (one sequence, key head and part) go to one XCD (consecutive workgroups
    // to the eight in turn); a run further on every such set has moved to the next XCD, so that long and short sequences spread; and the
    // longest row blocks of causal calls come first.
    const int n_sets = p.kv_heads * grid.splits * (grid.packed ? 1 : p.sequences);
    int t = blockIdx.x >> 3;
    const int within = t % grid.chunk;
    t = t / grid.chunk * 8 + (blockIdx.x & 7);
    const int run = t / n_sets, set = (t + run) % n_sets, split = set % grid.splits, group = set / grid.splits;
    int blk = run * grid.chunk + within, s = 0, kh;
    if (blk >= grid.blocks) return;                      // (the grid is whole runs for eight XCDs)
    if (grid.packed) {
        kh = group;
        // the sequence that has row block `blk` of all: 64 sequences at a time, a lane counts one's blocks
        int before = 0;
        for (int s0 = 0;; s0 += 64) {
            if (s0 >= p.sequences) return;
            int n = 0, q0;
            if (s0 + lane < p.sequences) n = (int)(((int64_t)seq_rows(p, s0 + lane, q0) * G + 32 * QW - 1) / (32 * QW));
            int sum = n;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int less = __shfl_up(sum, o);
                if (lane >= o) sum += less;
            }
            const uint64_t past = __ballot(before + sum > blk);
            if (past) {
                const int at = __builtin_ctzll(past);
                s = s0 + at;
                blk -= before + __shfl(sum - n, at);
                break;
            }
            before += __shfl(sum, 63);
        }
        s = __builtin_amdgcn_readfirstlane(s);
        blk = __builtin_amdgcn_readfirstlane(blk);
        if (blk < 0) return;                             // (offsets that make no sense: their counts may have wrapped)
    } else {
        kh = group % p.kv_heads;
        s = group / p.kv_heads;
    }
    const Seq sq = sequence(p, s);
    const int64_t rows = (int64_t)sq.nq * G;
    if (p.causal) {                                      // (blocks that the sequence does not have stay where they are)
        const int mine = (int)((rows + 32 * QW - 1) / (32 * QW));
        if (blk < mine) blk = mine - 1 - blk;
    }
    const int64_t r0 = (int64_t)blk * 32 * QW;
    if (r0 >= rows) return;
    const int64_t r = r0 + qw * 32 + li;
    const bool real = r < rows;
    const int i = (int)((real ? r : rows - 1) / G), h = kh * G + (int)((real ? r : rows - 1) - (int64_t)i * G);
    const int place = i + sq.nk - sq.nq, limit = real ? key_limit(p, sq, place) : 0;
    const int64_t row = sq.q0 + i;

    // keys of this part that any row of the workgroup sees: the last row's (limits do not fall)
    const int64_t r_last = r0 + 32 * QW < rows ? r0 + 32 * QW - 1 : rows - 1;
    const int wg_limit = key_limit(p, sq, (int)(r_last / G) + sq.nk - sq.nq);
    const int j_begin = split * grid.per_split, j_stop = j_begin + grid.per_split;           // (plan: fits 32 bits)
    const int j_end = wg_limit < j_stop ? wg_limit : j_stop;
    const int tiles = j_end > j_begin ? (j_end - j_begin + KT - 1) / KT : 0;
    // the wave's own range of limits: tiles below the smallest need no mask, tiles past the largest no work
    int lim_min = real ? limit : 0x7fffffff, lim_max = limit;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int a = __shfl_xor(lim_min, o), b = __shfl_xor(lim_max, o);
        lim_min = a < lim_min ? a : lim_min;
        lim_max = b > lim_max ? b : lim_max;
    }
    lim_min = __builtin_amdgcn_readfirstlane(lim_min);
    lim_max = __builtin_amdgcn_readfirstlane(lim_max);

    // --- loader: an instruction of a wave fills 1 KB, lane l the 16-byte chunk l of it; the lane fetches the chunk that belongs there.  QW > 1: call
    // `t` loads the KW tiles of an iteration, each by all waves; else tile t, by the wave that takes it.
    constexpr int CPR = ROWB / 16, RPI = 64 / CPR, LW = QW > 1 ? NW : 1, NI = TILE / 1024 / LW;
    static_assert(TILE % (1024 * LW) == 0, "whole instructions");
    const int lw = QW > 1 ? wave : 0;
    const T* kbase = reinterpret_cast<const T*>(p.k) + (int64_t)sq.k0 * p.k_row + kh * p.k_head;
    const T* vbase = reinterpret_cast<const T*>(p.v) + (int64_t)sq.k0 * p.v_row + kh * p.v_head;
    auto dma_tile = [&](char* own, int t) {              // keys j0 .. j0 + KT - 1, those from j_end on as the last of them
        const int j0 = j_begin + t * KT, last = j_end - 1 - j0;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const char* base = reinterpret_cast<const char*>((which ? vbase : kbase) + (int64_t)j0 * (which ? p.v_row : p.k_row));
            const uint32_t pitch = (uint32_t)(which ? p.v_row : p.k_row) * (uint32_t)sizeof(T);
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const int tr = (lw + LW * n) * RPI + lane / CPR, chunk = (lane % CPR) ^ (which ? M::v_swz(tr) : M::k_swz(tr));
                const int kr = tr < last ? tr : last;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base + (uint64_t)((uint32_t)kr * pitch + chunk * 16)),
                                                 (__attribute__((address_space(3))) void*)(own + which * TILE + (lw + LW * n) * 1024), 16, 0, 0);
            }
        }
        if constexpr (DIST == DIST_GRID) {
            if (lw == 0) {
#pragma unroll
                for (int n = 0; n < KT / 32; ++n) {      // 64 floats = 32 pairs an instruction
                    const int tr = 32 * n + (lane >> 1), kr = tr < last ? tr : last;
                    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p.k_coords + 2 * (int64_t)(sq.k0 + j0 + kr) + (lane & 1)),
                                                     (__attribute__((address_space(3))) void*)(own + 2 * TILE + n * 256), 4, 0, 0);
                }
            }
        }
    };
    auto dma = [&](char* stage, int t) {
        if constexpr (QW == 1) {
            dma_tile(stage + kw * OWN, t);
        } else {
#pragma unroll
            for (int j = 0; j < KW; ++j)
                if (t * KW + j < tiles) dma_tile(stage + j * OWN, t * KW + j);       // (of the last iteration the tiles that there are)
        }
    };

    Frag q[KS];
    {
        const T* src = reinterpret_cast<const T*>(p.q) + row * p.q_row + h * p.q_head + 8 * g;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[ks] = M::load(src + 16 * ks);
    }
    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[d][v] = 0.0f;
    // m: the reference that exponentials are taken against, in log2 units; `started` when the row has met a key
    float m = 0.0f, l = 0.0f;
    bool started = false;
    const float scale2 = p.scale * LOG2E, cap2 = p.cap * LOG2E;
    const float slope2 = DIST != DIST_NONE && p.slopes ? p.slopes[h] * LOG2E : 0.0f;
    f32x2 at = {0.0f, 0.0f};
    if constexpr (DIST == DIST_GRID) at = *reinterpret_cast<const f32x2*>(p.q_coords + 2 * row);
    // c tanh(y / c) = y (1 - x / 3 + 2 x^2 / 15 - 17 x^3 / 315 + 62 x^4 / 2835 - ...), x = (y / c)^2, for scores within c / 4 (what follows is 9e-9 of
    // the value there; bf16 stops a term earlier, at 3e-7), elsewhere c - 2 c / (1 + e^(2 y / c)), whose difference loses what is near zero
    const float kk = CAP ? 1.0f / (cap2 * cap2) : 0.0f;
    const bool series = p.cap >= 1e-3f && p.cap <= 1e15f;
    const float c1 = -1.0f / 3.0f * kk, c2 = 2.0f / 15.0f * kk * kk, c3 = -17.0f / 315.0f * kk * kk * kk, c4 = 62.0f / 2835.0f * kk * kk * (kk * kk);
    auto near_zero = [&](float y) {
        const float x = y * y;
        return fmaf(fmaf(fmaf(sizeof(T) == 4 ? fmaf(c4, x, c3) : c3, x, c2), x, c1), x, 1.0f);
    };
    const float tanh_f = CAP ? 2.0f * LOG2E / cap2 * scale2 : 0.0f, near_limit = 0.25f * cap2 / fabsf(scale2);
    // (of a raw score, less `ref`)
    auto capped = [&](float s, float ref) { return fmaf(-2.0f * cap2, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s * tanh_f)), cap2 - ref); };
    auto capped_near = [&](float s, float ref) {
        const float y = s * scale2;
        return fmaf(y, near_zero(y), -ref);
    };

    auto tile_scores = [&](f32x16 (&sc)[NB], const char* tile) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) sc[b][v] = 0.0f;
        // Fragments are read two steps ahead of their products; left to itself the compiler reads each just before it is wanted, with a wait of
        // 130 clocks
        constexpr int SETS = sizeof(T) == 2 ? 3 : 1;
        Frag k[SETS][NB];
        auto read = [&](int ks) {
#pragma unroll
            for (int b = 0; b < NB; ++b) k[ks % SETS][b] = M::k_frag(tile, 32 * b + li, ks, g);
        };
        if constexpr (SETS == 3) { read(0); read(1); }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (SETS == 1) read(ks);
            else if (ks + 2 < KS) read(ks + 2);
            if (SETS == 3) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int b = 0; b < NB; ++b) sc[b] = M::mma(k[ks % SETS][b], q[ks], sc[b]);
            if (SETS == 3) __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Is every score of the tile near zero, as caps go?
    auto all_near = [&](const f32x16 (&sc)[NB]) {
        float top = 0.0f;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) top = fmaxf(top, fabsf(sc[b][v]));
        return series && !__any(top > near_limit);
    };
    // Makes raw scores exponents: in log2 units, capped, lowered by distance, less the reference.
    auto shape = [&](f32x16 (&sc)[NB], const char* tile, int j0) {
        if constexpr (!CAP) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[b][v] = fmaf(sc[b][v], scale2, -m);
        } else if (all_near(sc)) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[b][v] = capped_near(sc[b][v], m);
        } else {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float s = sc[b][v];
                    sc[b][v] = sizeof(T) == 4 && series && fabsf(s) < near_limit ? capped_near(s, m) : capped(s, m);
                }
        }
        if constexpr (DIST == DIST_GRID) {
            const char* c = tile + 2 * TILE + 32 * g;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int n = 0; n < 8; ++n) {             // two keys
                    const f32x4 to = *reinterpret_cast<const f32x4*>(c + b * 256 + (n >> 1) * 64 + (n & 1) * 16);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float dy = at[0] - to[2 * e], dx = at[1] - to[2 * e + 1];
                        sc[b][2 * n + e] = fmaf(-slope2, __builtin_amdgcn_sqrtf(fmaf(dy, dy, dx * dx)), sc[b][2 * n + e]);
                    }
                }
        } else if constexpr (DIST == DIST_LINE) {
            const float d0 = (float)(place - j0 - 4 * g);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[b][v] = fmaf(-slope2, fabsf(d0 - (float)(32 * b + 8 * (v >> 2) + (v & 3))), sc[b][v]);
        }
    };
    // (plain scores stay raw: their factor and the reference are part of the exponentials' argument)
    auto exponent = [&](float s) { return PLAIN ? fmaf(s, scale2, -m) : s; };
    // Takes the reference up by `by` (rows of which it is 0 stay).
    auto rescale = [&](float by, float alpha) {
        m += by;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[d][v] *= alpha;
    };
    // The largest probability that a lane has seen since the reference moved.  The reference is a row's maximum over its first tile; from then on
    // nobody looks for a maximum before the exponentials, and when a probability has passed 2^30 it moves ahead of the next tile: up to there
    // fp32 sums and bf16 probabilities are as precise as at 1, and a jump that overflows within one tile (2^97 times a row's largest so far)
    // leaves sums that are not finite, which attention_row computes.  (Searching the maximum of every tile first took a lone wave 400 clocks of
    // 2100 a tile, all latency: an exchange, a vote and a branch.)
    constexpr float MOVE = 1073741824.0f;
    float highest = 0.0f;
    bool all_started = false;
    // Steep scores may pass that within a tile, and attention_row takes a hundred times as long: then the tile's exponents are looked at first.  Scores
    // are taken to be steep by what a wave sees: distances whose slope may add 48 from its tile to its next (of coordinates nothing is known), 100
    // between two scores of its first tile, or a probability of 2^60.  (16 tokens of caches up to 7600, slopes up to 0.7: 782 us, 53 so; ViT-B 518x518, scores
    // of 30 and of 60 nats a standard deviation: 190 and 836, 29 so.  Costs 3 % where it is not needed: on a grid 31.8, 32.8 so.)
    bool steep = DIST == DIST_GRID || (DIST == DIST_LINE && __any(fabsf(slope2) * (KW * KT) > 48.0f));
    auto hold = [&](f32x16 (&sc)[NB]) {
        float top = sc[0][0];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) top = fmaxf(top, sc[b][v]);
        top = exponent(top);
        if (!__any(top > 64.0f)) return;
        top = halves_max(top);
        const float by = top > 30.0f && top < INFINITY ? top : 0.0f;
        rescale(by, __builtin_amdgcn_exp2f(-by));
        if constexpr (!PLAIN) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[b][v] -= by;
        }
    };
    auto begin_rows = [&](f32x16 (&sc)[NB]) {
        float rel = sc[0][0], low = INFINITY;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                rel = fmaxf(rel, sc[b][v]);
                low = sc[b][v] > -INFINITY && sc[b][v] < low ? sc[b][v] : low;
            }
        rel = exponent(halves_max(rel));
        steep = steep || __any(rel - exponent(low) > 100.0f);
        const bool first = !started && rel > -INFINITY;
        const float by = first ? rel : 0.0f;
        m += by;                                          // (the row's sums are zero)
        if constexpr (!PLAIN) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[b][v] -= by;
        }
        started = started | first;
        all_started = __all(started | !real);
    };
    auto move_reference = [&] {
        const float top = halves_max(highest);
        const bool grow = top > MOVE;
        steep = steep || __any(top > 1.15e18f);
        const float by = grow ? __builtin_amdgcn_logf(top) : 0.0f;
        rescale(by, grow ? __builtin_amdgcn_exp2f(-by) : 1.0f);
        highest = 0.0f;
    };
    // Probabilities of the tile, their sums and the products with the values: STEPS steps of 16 keys a block.  The first block's fragments are read
    // by the caller, ahead of the work on the scores, where there are registers for them (EARLY).
    constexpr int BLOCKS = KT / 16 / M::STEPS;
    constexpr bool EARLY = sizeof(T) == 2 && D == 64;
    auto finish = [&](f32x16 (&sc)[NB], const typename M::Values& values, Frag (&f0)[M::STEPS][DB]) {
        __builtin_amdgcn_s_setprio(2);
        auto block = [&](auto N) {
            constexpr int first = decltype(N)::value * M::STEPS;
            Frag later[M::STEPS][DB];
            constexpr bool here = decltype(N)::value > 0 || !EARLY;
            if constexpr (here) M::template v_frags<first>(values, later);
#pragma unroll
            for (int k = 0; k < M::STEPS; ++k) {
                float e[8];
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    e[n] = __builtin_amdgcn_exp2f(exponent(sc[(first + k) >> 1][8 * ((first + k) & 1) + n]));
                    l += e[n];
                }
#pragma unroll
                for (int n = 0; n < 8; n += 2) highest = fmaxf(fmaxf(highest, e[n]), e[n + 1]);
                const Frag b = M::probs(e);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    if constexpr (here) o[d] = M::mma(later[k][d], b, o[d]);
                    else o[d] = M::mma(f0[k][d], b, o[d]);
                }
            }
        };
        block(std::integral_constant<int, 0>{});
        if constexpr (BLOCKS > 1) block(std::integral_constant<int, 1>{});
        if constexpr (BLOCKS > 2) block(std::integral_constant<int, 2>{});
        if constexpr (BLOCKS > 3) block(std::integral_constant<int, 3>{});
        __builtin_amdgcn_s_setprio(0);
    };
    // Tile t, with `loads` (the next tile's) issued while the first products run: the CU's one address unit takes 16 clocks for each of them, and a
    // wave that waits for it issues nothing else.
    auto compute = [&](const char* stage, int t, auto&& loads) {
        const char* tile = stage + kw * OWN;
        const int j0 = j_begin + t * KT;
        if (j0 >= lim_max) { loads(); return; }           // (the wave's rows see nothing of it)
        const bool masked = j0 + KT > lim_min || j0 + KT > j_end;
        f32x16 sc[NB];
        __builtin_amdgcn_s_setprio(1);                    // (of a SIMD's waves the one with products to issue goes first)
        tile_scores(sc, tile);
        loads();
        __builtin_amdgcn_s_setprio(0);
        const auto values = M::values(tile + TILE, lane);
        Frag f0[M::STEPS][DB];
        if constexpr (EARLY) M::template v_frags<0>(values, f0);
        if (__any(highest > MOVE)) move_reference();
        if constexpr (!PLAIN) shape(sc, tile, j0);
        if (masked) {
            const int left = (limit < j_end ? limit : j_end) - j0 - 4 * g;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (32 * b + 8 * (v >> 2) + (v & 3) >= left) sc[b][v] = -INFINITY;
        }
        if (!all_started) begin_rows(sc);
        if (steep) hold(sc);
        finish(sc, values, f0);
    };

    if constexpr (QW > 1) {
        // all waves load all tiles of an iteration (KW of them), and wait for each other
        const int turns = (tiles + KW - 1) / KW;
        if (turns > 0) dma(smem, 0);
        __builtin_amdgcn_s_waitcnt(0x0F70);               // vmcnt(0): the loads into LDS have landed
        __syncthreads();
        for (int it = 0; it < turns; ++it) {
            auto loads = [&] { if (it + 1 < turns) dma(smem + ((it + 1) & 1) * STAGE, it + 1); };
            if (KW == 1 || it * KW + kw < tiles) compute(smem + (it & 1) * STAGE, it * KW + kw, loads);
            else loads();
            __builtin_amdgcn_s_waitcnt(0x0F70);
            __syncthreads();
        }
    } else {
        // a wave's tiles are its own: it waits for its loads and for nobody
        if (kw < tiles) dma(smem, kw);
        int buf = 0;
        for (int t = kw; t < tiles; t += KW, buf ^= 1) {
            if (t + KW < tiles) {
                dma(smem + (buf ^ 1) * STAGE, t + KW);
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_waitcnt(vmcnt_imm(2 * NI + (DIST == DIST_GRID ? KT / 32 : 0)));
            } else {
                __builtin_amdgcn_s_waitcnt(0x0F70);
            }
            asm volatile("" ::: "memory");
            compute(smem + buf * STAGE, t, [] {});
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(vmcnt_imm(63) & ~0x0F00);      // (its reads are done: the next loads may land there)
        }
        __syncthreads();
    }
    if (!started) m = -1e30f;
    l = halves_sum(l);

    // --- results.  A row is handed to attention_row if a sum of it is not finite, or nothing if it sees keys.  (The arguments are read once
    // more from the kernel's own segment: what only this part needs holds no scalar registers through the loop.)
    auto leave = [&](const vpe_attention_args& p, const SeqAttnGrid& grid) {
    const int seen_end = limit < j_stop ? limit : j_stop;
    if constexpr (KW == 1) {
        float odd = l * 0.0f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) odd = fmaf(o[d][v], 0.0f, odd);
        const bool bad = real && (odd != odd || (l == 0.0f && seen_end > j_begin));
        uint64_t redo = __ballot(bad);
        redo = (redo | redo >> 32) & 0xffffffffu;
        const bool store = real && !((redo >> li) & 1);
        const float f = grid.splits > 1 || l == 0.0f ? 1.0f : 1.0f / l;
        if (store) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const float v[4] = {o[d][4 * n] * f, o[d][4 * n + 1] * f, o[d][4 * n + 2] * f, o[d][4 * n + 3] * f};
                    const int c = 32 * d + 8 * n + 4 * g;
                    if (grid.splits > 1) store_columns<4>(grid.part_o + part_row(p, row, h, split) * D + c, v);
                    else store_columns<4>(reinterpret_cast<T*>(p.out) + row * p.out_row + h * p.out_head + c, v);
                }
            if (g == 0) store_stats<T>(p, grid, row, h, split, m, l);
        }
        for (; redo; redo &= redo - 1) {
            const int64_t rr = r0 + qw * 32 + __builtin_ctzll(redo);
            const int ii = (int)(rr / G);
            attention_row<T, D>(p, grid, sq, ii, kh * G + (int)(rr - (int64_t)ii * G), j_begin, j_stop, split, lane);
        }
    } else {
        // every wave leaves its sums, (c, row) 16 bytes apart by row, and its (m, l); then a thread of a row's KW waves adds four columns
        constexpr int RED = 32 * D;                       // floats of a wave's sums
        float* sums = reinterpret_cast<float*>(smem);
        float* ml = sums + NW * RED;
        __syncthreads();
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int n = 0; n < 4; ++n)
                *reinterpret_cast<f32x4*>(sums + wave * RED + ((8 * d + 2 * n + g) * 32 + li) * 4) = f32x4{o[d][4 * n], o[d][4 * n + 1], o[d][4 * n + 2], o[d][4 * n + 3]};
        if (g == 0) *reinterpret_cast<f32x2*>(ml + (wave * 32 + li) * 2) = f32x2{m, l};
        __syncthreads();
        float w[KW], top = -1e30f, total = 0.0f;
#pragma unroll
        for (int k = 0; k < KW; ++k) top = fmaxf(top, ml[((k * QW + qw) * 32 + li) * 2]);
#pragma unroll
        for (int k = 0; k < KW; ++k) {
            w[k] = __builtin_amdgcn_exp2f(ml[((k * QW + qw) * 32 + li) * 2] - top);
            total += w[k] * ml[((k * QW + qw) * 32 + li) * 2 + 1];
        }
        const float f = grid.splits > 1 || total == 0.0f ? 1.0f : 1.0f / total;
        float odd = total * 0.0f;
        constexpr int PER = D / 4 / (2 * KW);             // column groups of a thread
        f32x4 out[PER];
#pragma unroll
        for (int n = 0; n < PER; ++n) {
            const int c = (2 * kw + g) + 2 * KW * n;
            out[n] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(sums + (k * QW + qw) * RED + (c * 32 + li) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) out[n][e] = fmaf(w[k], v[e], out[n][e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) odd = fmaf(out[n][e], 0.0f, odd);
        }
        // a row that is bad for one of its waves is for all: they tell each other before anybody stores
        uint32_t* flags = reinterpret_cast<uint32_t*>(ml + NW * 64);
        uint64_t mine = __ballot(real && (odd != odd || (total == 0.0f && seen_end > j_begin)));
        if (lane == 0) flags[wave] = (uint32_t)(mine | mine >> 32);
        __syncthreads();
        uint32_t redo = 0;
#pragma unroll
        for (int k = 0; k < KW; ++k) redo |= flags[k * QW + qw];
        if (real && !((redo >> li) & 1)) {
#pragma unroll
            for (int n = 0; n < PER; ++n) {
                const int c = ((2 * kw + g) + 2 * KW * n) * 4;
                const float v[4] = {out[n][0] * f, out[n][1] * f, out[n][2] * f, out[n][3] * f};
                if (grid.splits > 1) store_columns<4>(grid.part_o + part_row(p, row, h, split) * D + c, v);
                else store_columns<4>(reinterpret_cast<T*>(p.out) + row * p.out_row + h * p.out_head + c, v);
            }
            if (kw == 0 && g == 0) store_stats<T>(p, grid, row, h, split, top, total);
        }
        int n = 0;
        for (uint32_t left = __builtin_amdgcn_readfirstlane(redo); left; left &= left - 1, ++n) {
            if (n % KW != kw) continue;
            const int64_t rr = r0 + qw * 32 + __builtin_ctz(left);
            const int ii = (int)(rr / G);
            attention_row<T, D>(p, grid, sq, ii, kh * G + (int)(rr - (int64_t)ii * G), j_begin, j_stop, split, lane);
        }
    }
    };
    leave(kernel_args<vpe_attention_args>(0), kernel_args<SeqAttnGrid>(sizeof(vpe_attention_args)));
}

// The parts of the keys put together: a wave per row and head.
template <typename T, int D>
__global__ __launch_bounds__(256) void seq_attention_join_kernel(const vpe_attention_args p, const SeqAttnGrid grid) {
    const int lane = threadIdx.x & 63;
    const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), n_rows = (int64_t)p.q_rows * p.heads;
    if (task >= n_rows) return;
    const int64_t row = task / p.heads;
    const int h = (int)(task - row * p.heads);
    // rows of no sequence have no parts: the wave looks the row up, 64 sequences at a time
    bool found = false;
    for (int s0 = 0; s0 < p.sequences && !found; s0 += 64) {
        bool in = false;
        if (s0 + lane < p.sequences) {
            int q0;
            const int n = seq_rows(p, s0 + lane, q0);
            in = row >= q0 && row < q0 + n;
        }
        found = __any(in);
    }
    if (!found) return;
    // a lane has a part's reference and sum (up to 64 parts), then one or two columns of all parts, several loads on their way
    constexpr int ND = D / 64;
    f32x2 ml = {-INFINITY, 0.0f};
    if (lane < grid.splits) ml = *reinterpret_cast<const f32x2*>(grid.part_ml + 2 * part_row(p, row, h, lane));
    float m = ml[1] == 0.0f ? -INFINITY : ml[0];          // (no keys of the row in this part)
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float w = ml[1] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(ml[0] - m);
    const float l = wave_sum(ml[1] == 0.0f ? 0.0f : ml[1] * w);
    float acc[ND];
#pragma unroll
    for (int n = 0; n < ND; ++n) acc[n] = 0.0f;
    const float* part = grid.part_o + part_row(p, row, h, 0) * D + lane;
    const int64_t step = n_rows * D;
#pragma unroll 8
    for (int k = 0; k < grid.splits; ++k) {
        const float by = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), k));
#pragma unroll
        for (int n = 0; n < ND; ++n) {
            const float v = part[k * step + 64 * n];
            acc[n] += by == 0.0f ? 0.0f : by * v;
        }
    }
#pragma unroll
    for (int n = 0; n < ND; ++n)
        reinterpret_cast<T*>(p.out)[row * p.out_row + h * p.out_head + 64 * n + lane] = from_f32<T>(l == 0.0f ? 0.0f : acc[n] / l);
    if (p.lse && lane == 0) p.lse[row * p.heads + h] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
}

// What a launch needs to know of an instantiation.
typedef void (*SeqKernel)(const vpe_attention_args, const SeqAttnGrid);
struct SeqShape { SeqKernel kernel; int threads, lds; };
template <typename T, int D, int KT, int QW, int KW, bool CAP, int DIST, int OCC>
SeqShape seq_shape() { return {&seq_attention_kernel<T, D, KT, QW, KW, CAP, DIST, OCC>, 64 * QW * KW, seq_lds_bytes<T, D, KT, QW, KW, DIST>()}; }
// The instantiation for a kind of score, a head's width and a workgroup's rows (a translation unit per type).
SeqShape seq_shape_bf16(bool cap, int dist, int head_dim, int rows);
SeqShape seq_shape_f32(bool cap, int dist, int head_dim, int rows);

}  // namespace vpe
