// Answers from rows of scores: log-probabilities of given labels, entropy, and the k best entries with theirs.
//
//   m = max x,  S = sum e^(x - m),  T = sum (x - m) e^(x - m)
//   log p_i = x_i - m - ln S,   entropy = ln S - T / S,   best: by value, equal values by index
//
// One pass over a row in 16-byte chunks, four a thread and step, which are on their way to shared memory a step ahead (each thread reads what it
// asked for itself: no barrier).  A thread keeps its maximum with the step that it came from, and S and T relative to a reference that
// follows the maximum only when that is more than 20 above it (terms up to e^20 are as good as terms up to 1; a running maximum as reference would
// be rescaled in every step by one lane of a warp or another).  An entry costs one instruction of the special function unit (16 a
// cycle and SM) and some five others, two entries per instruction where the fp32 pipe has packed forms.
// The k best come almost free from what the pass leaves, G maxima of threads: of 32 groups of threads the k-th largest maximum is a lower
// bound of the k-th best entry, since k groups have an entry at or above it; so only chunks of threads whose own maximum reaches
// it are looked at again (from L1 or L2, by all threads), and entries that reach it, some k of them, go into a list in shared memory, where an
// entry's place is the number of entries before it.  A list that overflows (many sorted scores) is replaced by k rounds of a
// maximum below the last one.
// Entries are ordered by (value, index), which no two share: results do not depend on the order in which threads reach the list.
//
// A row is a warp's, 128 threads' or 256 threads' (what a row costs beside its entries, 400 instructions a warp and as many again with the best entries, is the
// less the fewer warps share it; so the rule is the fewest that keep the SMs busy), and few long rows are cut over several CTAs (up to 16 a row): each leaves (m, S, T) and its
// k best in the workspace, the last to arrive joins them.
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
    unsigned int *bad_label;               // set where a label is outside its row
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

// The sums of a warp's lanes joined, relative to the largest m (each has the result).
__device__ __forceinline__ LpSum lp_join(LpSum a) {
    float m = a.m;
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
    a = lp_rebase(a, m > -INFINITY ? m : 0.0f);
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) { a.s += __shfl_xor_sync(0xffffffffu, a.s, s); a.t += __shfl_xor_sync(0xffffffffu, a.t, s); }
    a.m = m;
    return a;
}

__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// Adds 2^d and d 2^d, d = x log2(e) - c, of U chunks.
template <bool kIn32, int U, bool kMasked>
__device__ __forceinline__ void lp_add(const uint4 *u, f32x2 l2, f32x2 nc2, f32x2 &s, f32x2 &t) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t w[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
        for (int c = 0; c < (kIn32 ? 2 : 4); ++c) {
            const float lo = kIn32 ? __uint_as_float(w[2 * c % 4]) : __uint_as_float(w[c] << 16);
            const float hi = kIn32 ? __uint_as_float(w[(2 * c + 1) % 4]) : __uint_as_float(w[c] & 0xffff0000u);
            f32x2 d = fma2(pair2(lo, hi), l2, nc2);
            float da, db;
            split2(d, da, db);
            if (kMasked) { da = max_nan(da, -300.0f); db = max_nan(db, -300.0f); d = pair2(da, db); }
            const f32x2 e = pair2(ex2(da), ex2(db));
            s = add2(s, e);
            t = fma2(d, e, t);
        }
    }
}

template <int G> struct LpShape {
    static constexpr int threads = G == 32 ? 128 : G;
    static constexpr int resident = 1024 / threads;     // CTAs per SM that the registers are for
    static constexpr int rows = threads / G;
    static constexpr int cap = G == 32 ? 256 : 512;
    static constexpr int warps = G / 32;
    static constexpr int ahead = 1;                        // steps under way beside the one at hand
};
template <int G>
struct LpShared {
    __align__(16) uint32_t value[32];          // (read 16 bytes at a time)
    LpKey list[LpShape<G>::cap];
    LpKey best[kLpMaxTop];
    LpKey key[G == 32 ? 1 : G];
    uint32_t floor;
    int floor_at;
    LpSum sum[LpShape<G>::warps];
    float mx[LpShape<G>::warps];
    LpKey mk[LpShape<G>::warps];
    unsigned short who[G];         // threads whose chunks are looked at again
    int n, nwho, last;
};
static_assert(sizeof(LpShared<32>) % 16 == 0 && sizeof(LpShared<128>) % 16 == 0 && sizeof(LpShared<256>) % 16 == 0, "value must stay aligned in an array");
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
    // The bits of a chunk at a row's end or behind it, -inf for what is not the row's.
    __device__ __forceinline__ uint4 cut(int j, int end) const {
        constexpr uint32_t none = kIn32 ? 0xff800000u : 0xff80ff80u;
        uint4 u = make_uint4(none, none, none, none);
        if (j < end) {
            float v[E];
            edge(j, v);
            u = kIn32 ? make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]))
                      : make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4 % E], v[5 % E]), pack2(v[6 % E], v[7 % E]));
        }
        return u;
    }
    __device__ __forceinline__ float entry(int e) const {
        return kIn32 ? reinterpret_cast<const float *>(base)[e + lead] : __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(base)[e + lead]);
    }
};

// Results of a row from its sums and its best entries in order.  lab0, x0: the thread's first label and its score.
template <int G, bool kIn32>
__device__ __forceinline__ void lp_finish(const LogprobParams &p, const LpRow<kIn32> &x, long long row, int t, const LpSum &a, const LpKey *best, int lab0, float x0) {
    if (t >= 32) return;
    const bool empty = !(a.m > -INFINITY) && a.s == 0.0f;
    const float m = empty ? 0.0f : a.m, ls = empty ? 0.0f : logf(a.s);
    for (int l = t; p.lp && l < p.L; l += 32) {
        const int lab = l == t ? lab0 : p.labels[row * p.L + l];
        float r = 0.0f;
        if (lab >= 0 && lab < p.V) r = ((l == t ? x0 : x.entry(lab)) - m) - ls;
        else if (lab != -1) {
            r = __uint_as_float(0x7fc00000u);
            *p.bad_label = 1u;
        }
        p.lp[row * p.L + l] = r;
    }
    if (p.entropy && t == 0) p.entropy[row] = empty ? 0.0f : ls - a.t / a.s;
    if (t < p.k) {
        const int i = t;
        const LpKey key = best[i];
        if (p.top_id) p.top_id[row * p.k + i] = key ? (int)~(uint32_t)key : -1;
        if (p.top_lp) p.top_lp[row * p.k + i] = key ? (lp_value((uint32_t)(key >> 32)) - m) - ls : a.s == a.s ? -INFINITY : a.s;
    }
}

// Places of the n listed keys; the first k go to best (which holds zeros).  Four lanes compare a key with a quarter of the others each.
template <int G>
__device__ __forceinline__ void lp_rank(const LpKey *list, int n, int k, LpKey *best, int t) {
    for (int c0 = 0; c0 < n; c0 += G / 4) {
        const int c = c0 + (t >> 2);
        const LpKey mine = c < n ? list[c] : 0ull;
        int before = 0;
#pragma unroll 4
        for (int o = t & 3; o < n; o += 4) before += list[o] > mine;
        before += __shfl_xor_sync(0xffffffffu, before, 1);
        before += __shfl_xor_sync(0xffffffffu, before, 2);
        if ((t & 3) == 0 && before < k && mine) best[before] = mine;
    }
}

template <int G, bool kIn32>
__global__ void __launch_bounds__(LpShape<G>::threads, LpShape<G>::resident)
logprob_kernel(const LogprobParams p) {
    typedef LpShape<G> Shape;
    constexpr int E = LpRow<kIn32>::E, U = 4;
    constexpr float log2e = 1.44269504f;
    __shared__ LpShared<G> shared[Shape::rows];
    __shared__ uint4 ring[Shape::ahead + 1][U][Shape::threads];
    LpShared<G> &sh = shared[threadIdx.x / G];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x % G;
    const int part = G == 256 ? (int)(blockIdx.x % p.parts) : 0;
    const long long row = G == 256 ? (long long)(blockIdx.x / p.parts) : (long long)blockIdx.x * Shape::rows + threadIdx.x / G;
    if (row >= p.rows) return;
    LpRow<kIn32> x;
    x.init(p.x, row, p.V);
    const int c0 = G == 256 ? part * p.part_chunks : 0, c1 = G == 256 ? min(x.chunks, c0 + p.part_chunks) : x.chunks;
    int lab0 = -1;
    if (p.lp && t < p.L && t < 32) lab0 = p.labels[row * p.L + t];

    // The sums are kept in powers of two: with c = ms log2(e) rounded, a term is 2^(x log2(e) - c), one fused multiply-add and one
    // instruction; what c is off by is known (a fused multiply-add gives it) and taken back at the end.
    float m = -INFINITY, ms = 0.0f, above = -INFINITY;      // the thread's maximum, the sums' reference and what makes that follow
    int jb = 0;                                             // first chunk of the step with the maximum
    f32x2 s2 = 0ull, t2 = 0ull, nc2 = 0ull;                 // sums of terms, of terms times exponents; -c
    const f32x2 l2 = pair2(log2e, log2e);
    bool masked = false;
    // 16 or 32 entries: their maximum first, then two by two
    auto take = [&](const uint4 *u, int j, bool cut) {
        float gm;
        if (kIn32) {
            gm = -INFINITY;
#pragma unroll
            for (int i = 0; i < U; ++i)
                gm = fmaxf(fmaxf(fmaxf(__uint_as_float(u[i].x), __uint_as_float(u[i].y)), fmaxf(__uint_as_float(u[i].z), __uint_as_float(u[i].w))), gm);
        } else {
            uint32_t w = 0xff80ff80u;
#pragma unroll
            for (int i = 0; i < U; ++i) w = max_bf16x2(max_bf16x2(max_bf16x2(u[i].x, u[i].y), max_bf16x2(u[i].z, u[i].w)), w);
            gm = fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
        }
        jb = gm > m ? j : jb;
        m = fmaxf(m, gm);
        if (gm > above) {
            const float c = gm * log2e;
            if (above > -INFINITY) {       // (before the first finite entry the sums are 0, or NaN)
                float old, same;
                split2(nc2, old, same);
                const float d = fmaxf(-old - c, -1e4f), f = ex2(d);
                const f32x2 f2 = pair2(f, f);
                t2 = mul2(fma2(s2, pair2(d, d), t2), f2); s2 = mul2(s2, f2);
            }
            ms = gm; above = gm + 20.0f;
            nc2 = pair2(-c, -c);
        }
        if (!(fabsf(ms) < 1e37f)) {        // (such a reference leaves the range when multiplied: differences first)
#pragma unroll
            for (int i = 0; i < U; ++i) {      // (unrolled: a run-time index would put the entries into local memory in every step)
                float v[E], s = 0.0f, q = 0.0f;
                x.unpack(u[i], v);
#pragma unroll
                for (int c = 0; c < E; ++c) {
                    const float d = (v[c] - ms) * log2e, e = ex2(d);
                    s += e;
                    q = fmaf(fmaxf(d, -300.0f), e, q);
                }
                s2 = add2(s2, pair2(s, 0.0f)); t2 = add2(t2, pair2(q, 0.0f));
            }
        }
        const bool near = fabsf(ms) < 1e37f;
        // Masked entries (-inf, or so low that the exponent leaves the range) have the term 0, and -inf * 0 is NaN.  A warp that meets one adds
        // the step again with no exponent below -300, and goes on so (a fifth more instructions);
        // steps with places behind the row's end (cut) are added that way.
        if (!masked && !cut) {
            f32x2 sn = s2, tn = t2;
            lp_add<kIn32, U, false>(u, l2, nc2, sn, tn);
            float ta, tb;
            split2(tn, ta, tb);
            masked = __any_sync(0xffffffffu, near && !(ta + tb == ta + tb));
            if (!masked && near) { s2 = sn; t2 = tn; }
        }
        if (masked || cut) {
            f32x2 sn = s2, tn = t2;
            lp_add<kIn32, U, true>(u, l2, nc2, sn, tn);
            if (near) { s2 = sn; t2 = tn; }
        }
    };
    const int w0 = x.whole(0) ? 0 : 1, w1 = x.whole(x.chunks - 1) ? c1 : min(c1, x.chunks - 1);
    // step n of the thread: chunks c0 + t + (n U + i) G, i = 0 .. U - 1
    constexpr int D = Shape::ahead + 1;
    const uint32_t slot0 = smem_u32(&ring[0][0][threadIdx.x]);
    constexpr uint32_t per_chunk = Shape::threads * 16, per_step = U * per_chunk;
    auto whole_step = [&](int j) { return j >= w0 && j + (U - 1) * G < w1; };
    auto ask = [&](int j, uint32_t slot) {
        if (whole_step(j)) {
#pragma unroll
            for (int i = 0; i < U; ++i) cp_async16(slot + i * per_chunk, x.base + (size_t)(uint32_t)j * 16 + i * G * 16, 16u);
        } else {
#pragma unroll
            for (int i = 0; i < U; ++i)
                if (j + i * G >= w0 && j + i * G < w1) cp_async16(slot + i * per_chunk, x.base + (size_t)(uint32_t)(j + i * G) * 16, 16u);
        }
        cp_async_commit();
    };
    uint32_t put = slot0, get = slot0;
#pragma unroll
    for (int n = 0; n < D - 1; ++n) { ask(c0 + t + n * U * G, put); put += per_step; }
    const int steps = max(0, (c1 - c0 - (t & ~31) + U * G - 1) / (U * G));      // of the warp
#pragma unroll 1
    for (int n = 0, j = c0 + t; n < steps; ++n, j += U * G) {
        if (n + D - 1 < steps) ask(j + (D - 1) * U * G, put);
        else cp_async_commit();
        put = put == slot0 + (D - 1) * per_step ? slot0 : put + per_step;
        cp_async_wait<D - 1>();
        uint4 u[U];
        const bool cut = __any_sync(0xffffffffu, !whole_step(j));
        if (!cut) {
#pragma unroll
            for (int i = 0; i < U; ++i) u[i] = ld_shared16(get + i * per_chunk);
        } else {
#pragma unroll
            for (int i = 0; i < U; ++i) u[i] = j + i * G >= w0 && j + i * G < w1 ? ld_shared16(get + i * per_chunk) : x.cut(j + i * G, c1);
        }
        get = get == slot0 + (D - 1) * per_step ? slot0 : get + per_step;
        take(u, j, cut);
    }
    float x0 = 0.0f;
    if (lab0 >= 0 && lab0 < p.V) x0 = x.entry(lab0);

    // ---- sums of the group
    const int lane = t & 31, warp = t >> 5;
    LpSum a;
    {
        float sa, sb, ta, tb;
        split2(s2, sa, sb); split2(t2, ta, tb);
        // back to natural exponents relative to ms itself
        const float c = ms * log2e, off = fabsf(ms) < 1e37f ? fmaf(ms, log2e, -c) : 0.0f, f = ex2(-off);
        a.m = m > -INFINITY ? ms : m; a.s = (sa + sb) * f; a.t = fmaf(-off, sa + sb, ta + tb) * f * 0.693147181f;
    }
    const LpKey key = lp_order(m) ? (LpKey)lp_order(m) << 32 | (uint32_t)~jb : 0ull;
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
    if (t < kLpMaxTop) sh.best[t] = 0ull;
    if (t == 0) { sh.n = 0; sh.nwho = 0; }
    if (G > 32) {
        if (lane == 0) sh.mx[warp] = m;
        sh.key[t] = key;
        __syncthreads();
        m = sh.mx[0];
#pragma unroll
        for (int w = 1; w < Shape::warps; ++w) m = fmaxf(m, sh.mx[w]);
    }
    // ---- the k-th largest maximum of 32 groups of threads (0: fewer have one)
    if (p.k && warp == 0) {
        LpKey g = key;
        if (G > 32) {
#pragma unroll
            for (int i = 32; i < G; i += 32) g = max(g, sh.key[lane + i]);
        }
        // A lane's place is the number of larger values (k rounds of a warp-wide maximum take 20 cycles of the SM each).  Equal values count
        // up to the last step that one of their lanes has it from.
        const uint32_t o = (uint32_t)(g >> 32);
        sh.value[lane] = o;
        __syncwarp();
        int before = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint4 q = *reinterpret_cast<const uint4 *>(&sh.value[4 * i]);
            before += (q.x > o) + (q.y > o) + (q.z > o) + (q.w > o);
        }
        const uint32_t f = __reduce_min_sync(0xffffffffu, before < p.k ? o : 0xffffffffu);
        const uint32_t at = __reduce_max_sync(0xffffffffu, o == f ? ~(uint32_t)g : 0u);
        if (lane == 0) { sh.floor = f; sh.floor_at = (int)at; }
    }
    a = lp_rebase(a, m > -INFINITY ? m : 0.0f);
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) { a.s += __shfl_xor_sync(0xffffffffu, a.s, s); a.t += __shfl_xor_sync(0xffffffffu, a.t, s); }
    if (G > 32 && lane == 0) sh.sum[warp] = a;
    lp_sync<G>();
    if (G > 32) {
        a = sh.sum[0];
#pragma unroll
        for (int w = 1; w < Shape::warps; ++w) { a.s += sh.sum[w].s; a.t += sh.sum[w].t; }
    }
    a.m = m;

    if (p.k) {
        // ---- entries that reach it, among the chunks of the threads whose maximum does
        const uint32_t fo = sh.floor;
        const float fv = fo ? lp_value(fo) : -INFINITY;            // (no floor: every entry above -inf counts)
        // Entries equal to the floor count up to the last chunk of that step: k groups have theirs no later, nor do the maxima of the threads that
        // hold such entries come later.
        const int fj = fo ? sh.floor_at + (U - 1) * G : -1;
        const uint32_t ko = (uint32_t)(key >> 32);
        const uint32_t reach = __ballot_sync(0xffffffffu, ko > fo || (ko == fo && ko && jb <= fj));
        if (reach) {
            int at = 0;
            if (G > 32 && lane == 0) at = atomicAdd(&sh.nwho, __popc(reach));
            if (G > 32) at = __shfl_sync(0xffffffffu, at, 0);
            else if (lane == 0) sh.nwho = __popc(reach);
            if (reach >> lane & 1u) sh.who[at + __popc(reach & ((1u << lane) - 1u))] = (unsigned short)t;
        }
        lp_sync<G>();
        // (a row of few steps is still in shared memory)
        const bool kept = (c1 - c0 + U * G - 1) / (U * G) <= D;
        const int lg = 32 - __clz(max((c1 - c0 + G - 1) / G - 1, 0)), items = sh.nwho << lg;      // chunks of a thread, up to a power of two
        for (int it = t; it < items; it += G) {
            const int w = sh.who[it >> lg], n = it & ((1 << lg) - 1), j = c0 + w + n * G;
            if (j >= c1) continue;
            float v[E];
            if (kept && j >= w0 && j < w1) x.unpack(ld_shared16(slot0 + (uint32_t)(w - t) * 16 + (uint32_t)n * per_chunk), v);
            else x.load(j, v);
            const float fe = j <= fj ? fv : __uint_as_float(0x7fc00000u);
            uint32_t hit = 0;
#pragma unroll
            for (int i = 0; i < E; ++i) hit |= v[i] > fv || v[i] == fe ? 1u << i : 0u;
            for (; hit; hit &= hit - 1) {
                const int i = __ffs(hit) - 1, at = atomicAdd(&sh.n, 1);
                float h = v[0];
#pragma unroll
                for (int c = 1; c < E; ++c) h = i == c ? v[c] : h;
                if (at < Shape::cap) sh.list[at] = (LpKey)lp_order(h) << 32 | (uint32_t)~(j * E + i - x.lead);
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
    if (G != 256 || p.parts == 1) {
        lp_finish<G, kIn32>(p, x, row, t, a, sh.best, lab0, x0);
        return;
    }
    // ---- a row of several CTAs: leave the part, the last to arrive joins them
    const long long slot = row * p.parts + part;
    if (t == 0) *reinterpret_cast<float4 *>(p.part_mst + slot * 4) = make_float4(a.m, a.s, a.t, 0.0f);
    if (t < p.k) p.part_key[slot * p.k + t] = sh.best[t];
    __syncthreads();
    if (t == 0) {
        // (releases what the barrier has put before it, and acquires what the other CTAs released)
        unsigned before;
        asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(p.arrived + row) : "memory");
        sh.last = before == (unsigned)p.parts - 1;
        if (sh.last) p.arrived[row] = 0u;
    }
    __syncthreads();
    if (!sh.last) return;
    const int n = p.parts * p.k;
    LpSum all{-INFINITY, 0.0f, 0.0f};
    if (t < p.parts) {
        const float4 f = __ldcg(reinterpret_cast<const float4 *>(p.part_mst + (row * p.parts + t) * 4));
        all = LpSum{f.x, f.y, f.z};
    }
    for (int i = t; i < n; i += G) sh.list[i] = __ldcg(p.part_key + row * n + i);
    if (t < kLpMaxTop) sh.best[t] = 0ull;
    if (t == 0) sh.n = 0;
    if (warp == 0) all = lp_join(all);
    __syncthreads();
    const LpKey *from = sh.list;
    int listed = n;
    if (p.k && p.k <= p.parts) {
        // The k-th best of the parts' first entries is a lower bound again, which only those k parts' entries reach: k * k at most.
        // (Parts without an entry have 0 there, which no other is below; then fewer than k parts have any.)  Ranking all entries instead: 7.1 against
        // 6.5 us for the 8 best of one row of 131072 in 16 parts.
        static_assert(G != 256 || kLpMaxParts * kLpMaxParts <= G, "the entries that reach the bound must fit");
        if (warp == 0) {
            const LpKey head = lane < p.parts ? sh.list[lane * p.k] : 0ull;
            int before = 0;
#pragma unroll
            for (int q = 0; q < kLpMaxParts; ++q) before += __shfl_sync(0xffffffffu, head, q) > head;
            const uint32_t at = __ballot_sync(0xffffffffu, head && before == p.k - 1);
            if (at ? lane == __ffs(at) - 1 : lane == 0) sh.mk[0] = at ? head : 0ull;
        }
        __syncthreads();
        const LpKey bound = sh.mk[0];
        for (int i = t; i < n; i += G) {
            const LpKey q = sh.list[i];
            if (q && q >= bound) sh.key[atomicAdd(&sh.n, 1)] = q;
        }
        __syncthreads();
        from = sh.key; listed = sh.n;
    }
    lp_rank<G>(from, listed, p.k, sh.best, t);
    __syncthreads();
    lp_finish<G, kIn32>(p, x, row, t, all, sh.best, lab0, x0);
}

}  // namespace xk
