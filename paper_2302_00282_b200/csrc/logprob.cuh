// Answers from rows of scores: log-probabilities of given labels, entropy, and the k best entries with theirs.
//
//   m = max x,  S = sum e^(x - m),  T = sum (x - m) e^(x - m)
//   log p_i = x_i - m - ln S,   entropy = ln S - T / S,   best: by value, equal values by index
//
// Bound by HBM at long rows (one read, next to nothing written).  One pass: a thread keeps its running maximum with S and T relative to
// it (rescaled when the maximum grows, which happens some ln n times), and the chunk that its maximum came from.
// The k best come almost free from what the pass leaves: G maxima of threads, in 64 groups (32: lanes of a warp).  The k-th largest
// group maximum is a lower bound of the k-th best entry, since k groups have an entry at or above it; so only threads whose own maximum
// reaches it look at their chunks again (from L1 or L2), and put the entries that reach it, some k of them, into a list in
// shared memory, where an entry's place is the number of entries before it.  A list that overflows (many equal or sorted scores in one
// thread's chunks) is replaced by k rounds of a maximum below the last one.
// Entries are ordered by (value, index), which no two share: results do not depend on the order in which threads reach the list.
//
// Rows: up to 2048 entries a warp, up to 8192 128 threads, above 512 threads.  Few long rows are cut over several CTAs (up to 16 a
// row); each leaves (m, S, T) and its k best in the workspace, the last to arrive joins them in ascending order.
#pragma once

#include "rows.cuh"

namespace xk {

constexpr int kLpMaxTop = 32;
constexpr int kLpMaxParts = 16;

struct LogprobParams {
    const void *x;
    const int *labels;
    float *lp, *entropy, *top_lp;          // null: not wanted
    int *top_id;
    unsigned int *status;
    long long rows;
    int V, L, k;
    int parts, part_chunks;                // CTAs per row; 16-byte chunks each of them takes
    float *part_mst;                       // [row][part][4]
    unsigned long long *part_key;          // [row][part][k]
    unsigned int *arrived;                 // [row]
};

typedef unsigned long long LpKey;          // (value in ascending bit order, ~index); 0: none

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Bits in ascending order of the values; the two zeros are one value.  -inf (never an answer) and NaN are 0.
__device__ __forceinline__ uint32_t lp_order(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return v > -INFINITY ? b ^ ((uint32_t)((int)b >> 31) | 0x80000000u) : 0u;
}
__device__ __forceinline__ float lp_value(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }

struct LpSum { float m, s, t; };
// Sums relative to m, brought to the maximum `to` (0 where that is -inf).  An empty side has s = t = 0 and adds nothing.
__device__ __forceinline__ LpSum lp_rebase(const LpSum &a, float to) {
    const float d = fmaxf((a.m > -INFINITY ? a.m : 0.0f) - to, -1e4f), f = ex2(d * 1.44269504f);
    return a.m > -INFINITY || a.s != 0.0f ? LpSum{to, a.s * f, fmaf(a.s, d, a.t) * f} : LpSum{to, 0.0f, 0.0f};
}

template <int G> struct LpShape {
    static constexpr int threads = G == 32 ? 256 : G;
    static constexpr int rows = threads / G;
    static constexpr int groups = G == 32 ? 32 : 64;
    static constexpr int cap = G == 32 ? 256 : 512;
    static constexpr int warps = G / 32;
};
template <int G>
struct LpShared {
    LpKey list[LpShape<G>::cap];
    LpKey best[kLpMaxTop];
    LpKey key[G == 32 ? 1 : G];
    LpKey group[G == 32 ? 1 : 64];
    LpKey floor;
    LpSum sum[LpShape<G>::warps];
    float mx[LpShape<G>::warps];
    LpKey mk[LpShape<G>::warps];
    int n, last;
};
template <int G> __device__ __forceinline__ void lp_sync() { if (G == 32) __syncwarp(); else __syncthreads(); }

// A row's chunks as aligned 16-byte pieces: chunk j holds entries [j * E - lead, ...) of the row; pieces that reach over
// the row's ends are read entry by entry.
template <bool kIn32>
struct LpRow {
    static constexpr int E = kIn32 ? 4 : 8;
    const char *base;              // of chunk 0
    int lead, V, chunks;
    __device__ __forceinline__ void init(const void *x, long long row, int n) {
        const char *p = static_cast<const char *>(x) + row * n * (16 / E);
        lead = (int)((uintptr_t)p & 15u) / (16 / E);
        base = p - lead * (16 / E);
        V = n; chunks = (n + lead + E - 1) / E;
    }
    __device__ __forceinline__ bool whole(int j) const { return j * E >= lead && (j + 1) * E <= V + lead; }
    __device__ __forceinline__ void edge(int j, float *v) const {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int e = j * E + i - lead;
            v[i] = e < 0 || e >= V ? -INFINITY
                 : kIn32 ? reinterpret_cast<const float *>(base)[j * E + i] : __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(base)[j * E + i]);
        }
    }
    __device__ __forceinline__ static void unpack(const uint4 &u, float *v) {
        if (kIn32) { v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w); return; }
        const f8 f = unpack8(u);
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = f.v[i];
    }
    __device__ __forceinline__ void load(int j, float *v) const {
        if (whole(j)) unpack(*reinterpret_cast<const uint4 *>(base + (size_t)j * 16), v);
        else edge(j, v);
    }
    __device__ __forceinline__ float entry(int e) const {
        return kIn32 ? reinterpret_cast<const float *>(base)[e + lead] : __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(base)[e + lead]);
    }
};

// Results of a row from its sums and its best entries in order.
template <int G, bool kIn32>
__device__ __forceinline__ void lp_finish(const LogprobParams &p, const LpRow<kIn32> &x, long long row, int t, const LpSum &a, const LpKey *best) {
    const bool empty = !(a.m > -INFINITY) && a.s == 0.0f;
    const float m = empty ? 0.0f : a.m, ls = empty ? 0.0f : logf(a.s);
    for (int l = t; p.lp && l < p.L; l += G) {
        const int lab = p.labels[row * p.L + l];
        float r = 0.0f;
        if (lab >= 0 && lab < p.V) r = (x.entry(lab) - m) - ls;
        else if (lab != -1) {
            r = __uint_as_float(0x7fc00000u);
            atomicCAS(p.status, 0u, kStatusBounds);
        }
        p.lp[row * p.L + l] = r;
    }
    if (p.entropy && t == 0) p.entropy[row] = empty ? 0.0f : ls - a.t / a.s;
    for (int i = t; i < p.k; i += G) {
        const LpKey key = best[i];
        if (p.top_id) p.top_id[row * p.k + i] = key ? (int)~(uint32_t)key : -1;
        if (p.top_lp) p.top_lp[row * p.k + i] = key ? (lp_value((uint32_t)(key >> 32)) - m) - ls : a.s == a.s ? -INFINITY : a.s;
    }
}

// Places of the n listed keys; the first k go to best (which holds zeros).
template <int G>
__device__ __forceinline__ void lp_rank(const LpKey *list, int n, int k, LpKey *best, int t) {
    for (int c = t; c < n; c += G) {
        const LpKey mine = list[c];
        int before = 0;
        for (int o = 0; o < n; ++o) before += list[o] > mine;
        if (before < k && mine) best[before] = mine;
    }
}

template <int G, bool kIn32>
__global__ void __launch_bounds__(LpShape<G>::threads)
logprob_kernel(const LogprobParams p) {
    typedef LpShape<G> Shape;
    constexpr int E = LpRow<kIn32>::E, U = 4;
    constexpr float log2e = 1.44269504f;
    __shared__ LpShared<G> shared[Shape::rows];
    LpShared<G> &sh = shared[threadIdx.x / G];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x % G;
    const int part = G == 512 ? (int)(blockIdx.x % p.parts) : 0;
    const long long row = G == 512 ? (long long)(blockIdx.x / p.parts) : (long long)blockIdx.x * Shape::rows + threadIdx.x / G;
    if (row >= p.rows) return;
    LpRow<kIn32> x;
    x.init(p.x, row, p.V);
    const int c0 = G == 512 ? part * p.part_chunks : 0, c1 = G == 512 ? min(x.chunks, c0 + p.part_chunks) : x.chunks;

    LpSum a{-INFINITY, 0.0f, 0.0f};
    float ms = 0.0f;                       // a.m, 0 while that is -inf
    int jb = 0;
    auto take = [&](const float *v, int j) {
        float cm = v[0];
#pragma unroll
        for (int i = 1; i < E; ++i) cm = fmaxf(cm, v[i]);
        if (cm > a.m) {
            if (a.s != 0.0f) a = lp_rebase(a, cm);
            a.m = ms = cm; jb = j;
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float d = v[i] - ms, e = ex2(d * log2e);
            a.s += e;
            a.t = fmaf(fmaxf(d, -200.0f), e, a.t);        // (e is 0 there; -inf * 0 would not be)
        }
    };
    int j = c0 + t;
    if (t == 0 && j < c1 && !x.whole(j)) { float v[E]; x.edge(j, v); take(v, j); j += G; }      // (only a row's first chunk and its last)
    const int whole1 = c1 == x.chunks && !x.whole(c1 - 1) ? c1 - 1 : c1;
    for (; j + (U - 1) * G < whole1; j += U * G) {
        uint4 u[U];
#pragma unroll
        for (int i = 0; i < U; ++i) u[i] = *reinterpret_cast<const uint4 *>(x.base + (size_t)(j + i * G) * 16);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            float v[E];
            x.unpack(u[i], v);
            take(v, j + i * G);
        }
    }
    for (; j < c1; j += G) { float v[E]; x.load(j, v); take(v, j); }

    // ---- sums of the group
    const int lane = t & 31, warp = t >> 5;
    const LpKey mine = (LpKey)lp_order(a.m) << 32 | (uint32_t)~jb;
    const LpKey key = lp_order(a.m) ? mine : 0ull;
    float m = a.m;
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
    if (G > 32) {
        if (lane == 0) sh.mx[warp] = m;
        sh.key[t] = key;
        __syncthreads();
        m = sh.mx[0];
#pragma unroll
        for (int w = 1; w < Shape::warps; ++w) m = fmaxf(m, sh.mx[w]);
    }
    a = lp_rebase(a, m > -INFINITY ? m : 0.0f);
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) { a.s += __shfl_xor_sync(0xffffffffu, a.s, s); a.t += __shfl_xor_sync(0xffffffffu, a.t, s); }
    if (G > 32) {
        if (lane == 0) sh.sum[warp] = a;
        if (t < 64) {
            LpKey g = sh.key[t];
#pragma unroll
            for (int i = 64; i < G; i += 64) g = max(g, sh.key[t + i]);
            sh.group[t] = g;
        }
    }
    if (t < kLpMaxTop) sh.best[t] = 0ull;
    if (t == 0) { sh.n = 0; sh.floor = 0ull; }
    lp_sync<G>();
    if (G > 32) {
        a = sh.sum[0];
#pragma unroll
        for (int w = 1; w < Shape::warps; ++w) { a.s += sh.sum[w].s; a.t += sh.sum[w].t; }
    }
    a.m = m;

    if (p.k) {
        // ---- the k-th largest group maximum
        if (G == 32) {
            int before = 0;
#pragma unroll
            for (int o = 0; o < 32; ++o) before += __shfl_sync(0xffffffffu, key, o) > key;
            if (before == p.k - 1) sh.floor = key;
        } else if (t < 64) {
            const LpKey g = sh.group[t];
            int before = 0;
#pragma unroll 8
            for (int o = 0; o < 64; ++o) before += sh.group[o] > g;
            if (before == p.k - 1) sh.floor = g;
        }
        lp_sync<G>();
        const uint32_t fv = (uint32_t)(sh.floor >> 32), fj = ~(uint32_t)sh.floor;       // (no floor: every entry above -inf counts)
        // ---- entries that reach it
        if (key && key >= sh.floor)
            for (int j = c0 + t; j < c1; j += G) {
                float v[E];
                x.load(j, v);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const uint32_t o = lp_order(v[i]);
                    if (o > fv || (o == fv && o && (uint32_t)j <= fj)) {
                        const int at = atomicAdd(&sh.n, 1);
                        if (at < Shape::cap) sh.list[at] = (LpKey)o << 32 | (uint32_t)~(j * E + i - x.lead);
                    }
                }
            }
        lp_sync<G>();
        if (sh.n <= Shape::cap) lp_rank<G>(sh.list, sh.n, p.k, sh.best, t);
        else {
            LpKey last = ~0ull;
            for (int r = 0; r < p.k; ++r) {
                LpKey b = 0ull;
                if (key)
                    for (int j = c0 + t; j < c1; j += G) {
                        float v[E];
                        x.load(j, v);
#pragma unroll
                        for (int i = 0; i < E; ++i) {
                            const uint32_t o = lp_order(v[i]);
                            const LpKey q = o ? (LpKey)o << 32 | (uint32_t)~(j * E + i - x.lead) : 0ull;
                            if (q < last) b = max(b, q);
                        }
                    }
#pragma unroll
                for (int s = 16; s >= 1; s >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, s));
                if (G > 32) {
                    if (lane == 0) sh.mk[warp] = b;
                    __syncthreads();
                    b = sh.mk[0];
#pragma unroll
                    for (int w = 1; w < Shape::warps; ++w) b = max(b, sh.mk[w]);
                    __syncthreads();
                }
                if (t == 0) sh.best[r] = b;
                last = b;
                if (!b) break;
            }
        }
        lp_sync<G>();
    }
    if (G != 512 || p.parts == 1) {
        lp_finish<G, kIn32>(p, x, row, t, a, sh.best);
        return;
    }
    // ---- a row of several CTAs: leave the part, the last to arrive joins them
    const long long slot = row * p.parts + part;
    if (t == 0) *reinterpret_cast<float4 *>(p.part_mst + slot * 4) = make_float4(a.m, a.s, a.t, 0.0f);
    if (t < p.k) p.part_key[slot * p.k + t] = sh.best[t];
    __threadfence();
    __syncthreads();
    if (t == 0) {
        sh.last = atomicAdd(p.arrived + row, 1u) == (unsigned)p.parts - 1;
        if (sh.last) p.arrived[row] = 0u;
    }
    __syncthreads();
    if (!sh.last) return;
    __threadfence();
    LpSum all{-INFINITY, 0.0f, 0.0f};
    for (int q = 0; q < p.parts; ++q) all.m = fmaxf(all.m, __ldcg(p.part_mst + (row * p.parts + q) * 4));
    const float to = all.m > -INFINITY ? all.m : 0.0f;
    for (int q = 0; q < p.parts; ++q) {
        const float4 f = __ldcg(reinterpret_cast<const float4 *>(p.part_mst + (row * p.parts + q) * 4));
        const LpSum b = lp_rebase(LpSum{f.x, f.y, f.z}, to);
        all.s += b.s; all.t += b.t;
    }
    const int n = p.parts * p.k;
    for (int i = t; i < n; i += G) sh.list[i] = __ldcg(p.part_key + row * n + i);
    if (t < kLpMaxTop) sh.best[t] = 0ull;
    __syncthreads();
    lp_rank<G>(sh.list, n, p.k, sh.best, t);
    __syncthreads();
    lp_finish<G, kIn32>(p, x, row, t, all, sh.best);
}

}  // namespace xk
