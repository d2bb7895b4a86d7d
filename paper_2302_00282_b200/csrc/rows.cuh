// Row operators on the CUDA cores: layer normalisation over the channels of a row, and the rounding of a row to 8-bit integers
// with a scale of its own (what the 8-bit product reads).  A row is the channels of one pixel of an NHWC tensor.
//
//   norm       mu = mean(x), v = mean((x - mu)^2), y = (x - mu) / sqrt(v + eps) * gamma + beta
//   to 8 bits  a = max |x|, q = round(127 x / a) (halves to even), scale = a / 127;  a = 0: q = 0
//
// Both are bound by HBM: the row is read once, kept in registers in its own type and written once.  A group of G threads owns a row, each thread V
// chunks of 8 channels (one 16-byte access of bf16, two of fp32); the loads of a whole row are under way at once, and groups that are at different
// points of their rows keep memory busy.  Mean and squared deviations are two reductions over the registers, not the
// difference of two sums over memory, which would lose the digits of a variance that is small against the mean; the second one also sums
// the deviations d, whose mean is the rounding of the first mean: (d - mean d) is exact to the last digits of d also for rows far from
// zero.  The reductions of a group of several warps go through shared memory; gamma and beta come through L1, the row past it.
// Rows that are not whole chunks (row_odd_kernel) are read and written channel by channel, a group's threads side by side.
// The sums of a row have one order for each length, type and alignment, in every kernel here: that of columns of chunks (row_sum).  So a row's result
// does not depend on the number of rows, and it is the same bit for bit where the link hands its 8-bit values to the product.
#pragma once

#include "gemm_tc.cuh"

namespace xk {

enum { RO_BF16 = 0, RO_F32 = 1, RO_Q8 = 2 };      // how a row leaves

struct RowParams {
    const void *x;
    const float *gamma, *beta;     // beta may be null
    void *y;                       // rows of `pitch` elements
    float *scale;                  // RO_Q8: one per row
    long long rows;
    int C, pitch;
    float eps;
    unsigned int *status;
    int launch_id;
};

// Two fp32 values that one instruction works on.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair2(float a, float b) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void split2(f32x2 v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) { f32x2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ uint4 ld_stream16(const void *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ float bf16_bits(uint32_t lo16) { return __uint_as_float(lo16 << 16); }
__device__ __forceinline__ float ld_scalar(const float *p) { return *p; }
__device__ __forceinline__ float ld_scalar(const __nv_bfloat16 *p) { return __bfloat162float(*p); }

// What multiplies a row to bring it to [-127, 127], and the row's scale, from the bits of its largest magnitude.  Rows whose
// magnitudes are so small that 127 / a overflows are lifted by 2^100 first (exact).  A row with an infinity or a NaN (bits of
// 0x7f800000 and above: the maximum is taken of the bits, so that a NaN wins it) gets the scale NaN, which reaches all its products.
struct RowScale { float lift, r, a, scale; };
__device__ __forceinline__ RowScale row_scale(uint32_t bits) {
    RowScale s;
    const float a = __uint_as_float(bits);
    s.lift = bits < 0x0d800000u ? 1.2676506e30f : 1.0f;      // below 2^-100
    s.a = a * s.lift;
    s.r = bits == 0u || bits >= 0x7f800000u ? 0.0f : __fdiv_rn(127.0f, s.a);
    s.scale = bits >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __fdiv_rn(a, 127.0f);
    return s;
}
// round(127 x / a), halves to even, in the low byte.  The product x * r is off by two roundings (1.2e-7 of it).  For bf16 values the exact
// quotient of two 8-bit significands is either half-way between integers or at least 1.5e-5 of itself away from that (all
// pairs tried), so rounding the product to 19 bits first (grid 1.9e-6) puts every half-way quotient back on its place.  For
// fp32 values the few that come near the middle are divided in 64 bits.
template <bool kIn32>
__device__ __forceinline__ uint32_t row_quant(float x, const RowScale &s) {
    const float t = (x * s.lift) * s.r;
    if (!kIn32) {
        const float u = __uint_as_float((__float_as_uint(t) + 16u) & 0xffffffe0u);
        return __float_as_uint(__fadd_rn(u, 12582912.0f)) & 0xffu;
    }
    const float v = __fadd_rn(t, 12582912.0f);
    const float off = fabsf(t - __fadd_rn(v, -12582912.0f));
    if (off > 0.4999f && off < 0.5001f) return (uint32_t)__double2int_rn(127.0 * (double)(x * s.lift) / (double)s.a) & 0xffu;
    return __float_as_uint(v) & 0xffu;
}

// Reductions over a group of G threads: within a warp by exchanges, across warps through `red`.
template <int G, class F>
__device__ __forceinline__ uint32_t row_reduce(uint32_t v, uint32_t *red, F f) {
#pragma unroll
    for (int s = (G < 32 ? G : 32) / 2; s >= 1; s >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, s));
    if (G > 32) {
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < G / 32; ++w) v = f(v, red[w]);
    }
    return v;
}
// Sums over a row's G * A columns of chunks: a thread has A of them, column a G + t in v[a].  The order is that of G * A threads with one column each:
// a tree over 32 columns, then their sums one after the other.
// The tree over 32 lanes for one value, or for two: lanes that are 16 apart hand each other the one that they do not go on with, so two trees take as
// many exchanges as one; lanes 0 to 15 have the first value's sum then, the others the second's.
template <int A>
__device__ __forceinline__ float row_trees(const float *v) {
    static_assert(A == 1 || A == 2, "");
    const bool up = A == 2 && (threadIdx.x & 16);
    const float mine = up ? v[A - 1] : v[0], other = A == 1 || up ? v[0] : v[A - 1];
    float x = mine + __shfl_xor_sync(0xffffffffu, other, 16);
#pragma unroll
    for (int s = 8; s >= 1; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
    return x;
}
// The sums of a warp's columns (G <= 32).
template <int G, int A>
__device__ __forceinline__ float row_columns(const float *v) {
    static_assert(G <= 32 && (A == 1 || G * A == 32), "the columns of a row are one tree");
    float x = v[0];
    if (A == 2) x += v[A - 1];
#pragma unroll
    for (int s = G / 2; s >= 1; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
    return x;
}
// ... of several warps', left in shared memory, and their sum.
template <int G, int A>
__device__ __forceinline__ void row_leave(const float *v, uint32_t *red) {
    const float x = row_trees<A>(v);
    const int lane = threadIdx.x & 31;
    if (lane % (32 / A) == 0) red[lane / (32 / A) * (G / 32) + (threadIdx.x >> 5)] = __float_as_uint(x);
}
template <int N>
__device__ __forceinline__ float row_left(const uint32_t *red) {
    float r = __uint_as_float(red[0]);
#pragma unroll
    for (int w = 1; w < N; ++w) r += __uint_as_float(red[w]);
    return r;
}
template <int G, int A>
__device__ __forceinline__ float row_sum(const float *v, uint32_t *red) {
    if constexpr (G <= 32) return row_columns<G, A>(v);
    else {
        row_leave<G, A>(v, red);
        __syncthreads();
        return row_left<G / 32 * A>(red);
    }
}
template <int G>
__device__ __forceinline__ float row_sum(float v, uint32_t *red) { return row_sum<G, 1>(&v, red); }
// ... of two values, behind one barrier.
template <int G, int A>
__device__ __forceinline__ float2 row_sum2(const float *x, const float *y, uint32_t *rx, uint32_t *ry) {
    if constexpr (G <= 32) return make_float2(row_columns<G, A>(x), row_columns<G, A>(y));
    else {
        row_leave<G, A>(x, rx); row_leave<G, A>(y, ry);
        __syncthreads();
        return make_float2(row_left<G / 32 * A>(rx), row_left<G / 32 * A>(ry));
    }
}
template <int G>
__device__ __forceinline__ float2 row_sum2(float a, float b, uint32_t *ra, uint32_t *rb) { return row_sum2<G, 1>(&a, &b, ra, rb); }
template <int G>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t *red) {
    return row_reduce<G>(v, red, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

// Threads of a CTA and rows it takes: several rows per group of short rows, so that enough bytes are under way.
template <int G, int V> struct RowShape {
    static constexpr int threads = G <= 32 ? 128 : G;
    static constexpr int per_group = G <= 32 && V < 4 ? 4 / V : 1;
    static constexpr int rows = threads / G * per_group;
};

// Eight channels as four pairs.
template <bool kIn32>
__device__ __forceinline__ void row_pairs(const uint4 *u, f32x2 *e) {
    if (kIn32) {
        e[0] = pair2(__uint_as_float(u[0].x), __uint_as_float(u[0].y)); e[1] = pair2(__uint_as_float(u[0].z), __uint_as_float(u[0].w));
        e[2] = pair2(__uint_as_float(u[1].x), __uint_as_float(u[1].y)); e[3] = pair2(__uint_as_float(u[1].z), __uint_as_float(u[1].w));
    } else {
        const uint32_t w[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = pair2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
}
__device__ __forceinline__ uint32_t pack2(f32x2 v) { float a, b; split2(v, a, b); return pack2(a, b); }

// Eight normalised channels: two words of fp32 or one of bf16.
template <bool kIn32, int kOut>
__device__ __forceinline__ void row_norm8(const uint4 *u, uint4 *o, const f32x2 *ga, const f32x2 *be, f32x2 nmu, f32x2 rs, f32x2 noff) {
    f32x2 e[4];
    row_pairs<kIn32>(u, e);
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = fma2(fma2(add2(e[i], nmu), rs, noff), ga[i], be[i]);
    if (kOut == RO_F32) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) split2(e[i], f[2 * i], f[2 * i + 1]);
        o[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        o[1] = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
    } else o[0] = make_uint4(pack2(e[0]), pack2(e[1]), pack2(e[2]), pack2(e[3]));
}
template <int kOut>
__device__ __forceinline__ void row_store8(const RowParams &p, long long row, int c, const uint4 *o) {
    if (kOut == RO_F32) {
        uint4 *d = reinterpret_cast<uint4 *>(static_cast<float *>(p.y) + row * p.pitch + c);
        d[0] = o[0]; d[1] = o[1];
    } else *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.y) + row * p.pitch + c) = o[0];
}
// Largest magnitude so far, in the order of the bits (two of bf16 at a time).
template <bool kWide>
__device__ __forceinline__ void row_peak8(const uint4 *u, uint32_t &peak) {
    if (kWide) {
#pragma unroll
        for (int w = 0; w < 2; ++w) peak = max(max(max(peak, u[w].x & 0x7fffffffu), max(u[w].y & 0x7fffffffu, u[w].z & 0x7fffffffu)), u[w].w & 0x7fffffffu);
    } else peak = __vmaxu2(__vmaxu2(__vmaxu2(peak, u[0].x & 0x7fff7fffu), __vmaxu2(u[0].y & 0x7fff7fffu, u[0].z & 0x7fff7fffu)), u[0].w & 0x7fff7fffu);
}
// Four values' low bytes in a word.
__device__ __forceinline__ uint32_t row_bytes4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
template <bool kWide>
__device__ __forceinline__ void row_quant8(const RowParams &p, long long row, int c, const uint4 *u, const RowScale &sc) {
    f32x2 e[4];
    row_pairs<kWide>(u, e);
    uint32_t q[8];
    if (!kWide && sc.lift != 1.0f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = mul2(e[i], pair2(sc.lift, sc.lift));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        if (kWide) {
            split2(e[i], a, b);
            q[2 * i] = row_quant<true>(a, sc); q[2 * i + 1] = row_quant<true>(b, sc);
        } else {      // (row_quant<false> for two)
            split2(mul2(e[i], pair2(sc.r, sc.r)), a, b);
            a = __uint_as_float((__float_as_uint(a) + 16u) & 0xffffffe0u); b = __uint_as_float((__float_as_uint(b) + 16u) & 0xffffffe0u);
            split2(add2(pair2(a, b), pair2(12582912.0f, 12582912.0f)), a, b);
            q[2 * i] = __float_as_uint(a); q[2 * i + 1] = __float_as_uint(b);
        }
    }
    *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(p.y) + row * p.pitch + c) = make_uint2(row_bytes4(q[0], q[1], q[2], q[3]), row_bytes4(q[4], q[5], q[6], q[7]));
}

// Rows of whole chunks (channels a multiple of 8).  A: columns whose sums a thread keeps apart (row_sum), chunk v being of column v % A.  (Linked norms with
// two columns of four chunks are held to the registers of seven CTAs of 128 threads: 8192 rows of 512 fp32 13.6 us for 11.9 without that.)
template <int G, int V, int A, bool kIn32, int kOut, bool kNorm>
__global__ void __launch_bounds__(RowShape<G, V>::threads, kNorm && kOut == RO_Q8 && V == 4 && A == 2 ? 896 / RowShape<G, V>::threads : 0)
row_kernel(const RowParams p) {
    typedef RowShape<G, V> Shape;
    constexpr int R = Shape::per_group, W = kIn32 ? 2 : 1;          // rows of a group; 16-byte words of a chunk
    __shared__ uint32_t red[4][32];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x % G;
    const long long row0 = (long long)blockIdx.x * Shape::rows + threadIdx.x / G;
    uint4 u[R][V][W];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const long long row = row0 + (long long)r * (Shape::threads / G);
        const char *base = static_cast<const char *>(p.x) + (row * p.C + t * 8) * (kIn32 ? 4 : 2);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int w = 0; w < W; ++w)
                u[r][v][w] = row < p.rows && (v * G + t) * 8 < p.C ? ld_stream16(base + v * G * 16 * W + w * 16) : make_uint4(0, 0, 0, 0);
    }
    f32x2 nmu[R], rs[R], noff[R];          // -mean, 1 / deviation, -(mean of the deviations) / deviation
    if (kNorm) {
        const float inv = 1.0f / (float)p.C;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x2 s0[A] = {}, s1[A] = {};                              // (zeros outside the row)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                f32x2 e[4];
                row_pairs<kIn32>(u[r][v], e);
                s0[v % A] = add2(s0[v % A], add2(e[0], e[1])); s1[v % A] = add2(s1[v % A], add2(e[2], e[3]));
            }
            float sum[A];
#pragma unroll
            for (int a = 0; a < A; ++a) {
                float x, y;
                split2(add2(s0[a], s1[a]), x, y);
                sum[a] = x + y;
            }
            const float mu = __fdiv_rn(row_sum<G, A>(sum, red[0]), (float)p.C);
            nmu[r] = pair2(-mu, -mu);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x2 s0[A] = {}, s1[A] = {}, q0[A] = {}, q1[A] = {};
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if ((v * G + t) * 8 >= p.C) continue;
                const int a = v % A;
                f32x2 e[4];
                row_pairs<kIn32>(u[r][v], e);
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = add2(e[i], nmu[r]);
                q0[a] = add2(q0[a], add2(e[0], e[1])); q1[a] = add2(q1[a], add2(e[2], e[3]));
                s0[a] = fma2(e[0], e[0], s0[a]); s1[a] = fma2(e[1], e[1], s1[a]); s0[a] = fma2(e[2], e[2], s0[a]); s1[a] = fma2(e[3], e[3], s1[a]);
            }
            float squares[A], rest[A];
#pragma unroll
            for (int a = 0; a < A; ++a) {
                float x, y, z, w;
                split2(add2(s0[a], s1[a]), x, y); split2(add2(q0[a], q1[a]), z, w);
                squares[a] = x + y; rest[a] = z + w;
            }
            const float2 f = row_sum2<G, A>(squares, rest, red[1], red[2]);
            const float off = f.y * inv, rstd = rsqrtf(fmaxf(fmaf(f.x, inv, -off * off), 0.0f) + p.eps);
            rs[r] = pair2(rstd, rstd); noff[r] = pair2(-off * rstd, -off * rstd);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const long long row = row0 + (long long)r * (Shape::threads / G);
        if (kNorm) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = (v * G + t) * 8;
                if (c >= p.C) continue;
                // (a row that is rounded to 8 bits is rounded to bf16 first, as it would be between two kernels)
                const uint4 *gp = reinterpret_cast<const uint4 *>(p.gamma + c), *bp = reinterpret_cast<const uint4 *>(p.beta + c);
                const uint4 g[2] = {__ldg(gp), __ldg(gp + 1)}, b[2] = {__ldg(bp), __ldg(bp + 1)};
                f32x2 ga[4], be[4];
                row_pairs<true>(g, ga); row_pairs<true>(b, be);
                uint4 o[2];
                row_norm8<kIn32, kOut>(u[r][v], o, ga, be, nmu[r], rs[r], noff[r]);
                if (kOut == RO_Q8) u[r][v][0] = o[0];
                else if (row < p.rows) row_store8<kOut>(p, row, c, o);
            }
        }
        if (kOut == RO_Q8) {
            constexpr bool wide = kIn32 && !kNorm;
            uint32_t peak = 0u;
#pragma unroll
            for (int v = 0; v < V; ++v) row_peak8<wide>(u[r][v], peak);
            const RowScale sc = row_scale(row_max<G>(wide ? peak : max(peak << 16, peak & 0xffff0000u), red[3]));
            if (row >= p.rows) continue;
            if (t == 0) p.scale[row] = sc.scale;
#pragma unroll
            for (int v = 0; v < V; ++v)                                // (filled up to the pitch with zeros: u = 0 there)
                if ((v * G + t) * 8 < p.pitch) row_quant8<wide>(p, row, (v * G + t) * 8, u[r][v], sc);
        }
    }
}

// Layer norm of many rows of whole chunks: groups of G threads that stay and walk over rows.  A thread keeps gamma and beta of its 8 V channels in
// registers (read per row they are 64 bytes of L1 traffic for 16 of the row); the copy engine brings rows to shared memory, two per
// group.  A row's slot is free for the next one as soon as the threads have it in registers, behind the first reduction, so loads are on their
// way all the time.
template <int G, int V, bool kIn32> struct StreamShape {
    static constexpr int cta = G == 32 ? 128 : G;          // (larger groups are CTAs of their own: they meet at CTA barriers)
    static constexpr int groups = G == 32 ? 4 : 1;
    static constexpr int slots = 2;
    static constexpr int resident = cta >= 512 ? 1 : 512 / cta;
};
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
template <int G, int V, bool kIn32, int kOut>
__global__ void __launch_bounds__(StreamShape<G, V, kIn32>::cta, StreamShape<G, V, kIn32>::resident)
row_stream_kernel(const RowParams p) {
    typedef StreamShape<G, V, kIn32> Shape;
    constexpr int W = kIn32 ? 2 : 1, S = Shape::slots;
    extern __shared__ __align__(128) uint8_t row_slots[];
    __shared__ uint32_t red[4][32];
    __shared__ __align__(8) unsigned long long full[Shape::groups][S];
    pdl_launch_dependents();
    const int t = threadIdx.x % G, grp = threadIdx.x / G;
    const uint32_t bytes = (uint32_t)p.C * (kIn32 ? 4u : 2u), slots = smem_u32(row_slots) + (uint32_t)grp * S * bytes, bars = smem_u32(full[grp]);
    if (t < S) mbar_init(bars + 8u * t, 1u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    f32x2 ga[V][4], be[V][4];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = (v * G + t) * 8;
        uint4 g[2], b[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            g[w] = c < p.C ? __ldg(reinterpret_cast<const uint4 *>(p.gamma + c) + w) : make_uint4(0, 0, 0, 0);
            b[w] = c < p.C ? __ldg(reinterpret_cast<const uint4 *>(p.beta + c) + w) : make_uint4(0, 0, 0, 0);
        }
        row_pairs<true>(g, ga[v]); row_pairs<true>(b, be[v]);
    }
    __syncthreads();
    pdl_wait();
    const long long step = (long long)gridDim.x * Shape::groups;
    auto ask = [&](long long row, int s) {
        if (t == 0 && row < p.rows) {
            mbar_arrive_expect_tx(bars + 8u * s, bytes);
            bulk_load(slots + (uint32_t)s * bytes, static_cast<const char *>(p.x) + row * (long long)bytes, bytes, bars + 8u * s);
        }
    };
    const long long row0 = (long long)blockIdx.x * Shape::groups + grp;
#pragma unroll
    for (int s = 0; s < S; ++s) ask(row0 + s * step, s);
    bool dead = false;                     // (a wait ran out: the rows that are left are walked over without waiting, so that every barrier is met)
    int s = 0;
    uint32_t ph = 0u;
    const float inv = 1.0f / (float)p.C;
#pragma unroll 1
    for (long long row = row0; row < p.rows; row += step) {
        if (!dead && !mbar_wait(bars + 8u * s, ph)) {
            dead = true;
            atomicCAS(p.status, 0u, kStatusTimeout | (3u << 8) | (((unsigned)p.launch_id & 0xfffu) << 12));
        }
        __syncwarp();
        uint4 u[V][W];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int w = 0; w < W; ++w)
                u[v][w] = (v * G + t) * 8 < p.C ? ld_shared16(slots + (uint32_t)s * bytes + (uint32_t)((v * G + t) * W + w) * 16u) : make_uint4(0, 0, 0, 0);
        f32x2 s0 = 0ull, s1 = 0ull, q0 = 0ull, q1 = 0ull;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            f32x2 e[4];
            row_pairs<kIn32>(u[v], e);
            s0 = add2(s0, add2(e[0], e[1])); s1 = add2(s1, add2(e[2], e[3]));
        }
        float a, b, c, d;
        split2(add2(s0, s1), a, b);
        const float mu = __fdiv_rn(row_sum<G>(a + b, red[0]), (float)p.C);
        ask(row + S * step, s);
        if (++s == S) { s = 0; ph ^= 1u; }
        const f32x2 nmu = pair2(-mu, -mu);
        s0 = s1 = 0ull;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if ((v * G + t) * 8 >= p.C) continue;
            f32x2 e[4];
            row_pairs<kIn32>(u[v], e);
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = add2(e[i], nmu);
            q0 = add2(q0, add2(e[0], e[1])); q1 = add2(q1, add2(e[2], e[3]));
            s0 = fma2(e[0], e[0], s0); s1 = fma2(e[1], e[1], s1); s0 = fma2(e[2], e[2], s0); s1 = fma2(e[3], e[3], s1);
        }
        split2(add2(s0, s1), a, b); split2(add2(q0, q1), c, d);
        const float2 f = row_sum2<G>(a + b, c + d, red[1], red[2]);
        const float off = f.y * inv, rstd = rsqrtf(fmaxf(fmaf(f.x, inv, -off * off), 0.0f) + p.eps);
        const f32x2 rs = pair2(rstd, rstd), noff = pair2(-off * rstd, -off * rstd);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c0 = (v * G + t) * 8;
            if (c0 >= p.C) continue;
            uint4 o[2];
            row_norm8<kIn32, kOut>(u[v], o, ga[v], be[v], nmu, rs, noff);
            row_store8<kOut>(p, row, c0, o);
        }
    }
    if (dead) for (int i = 0; i < 64; ++i) __nanosleep(1000);      // (time for copies under way)
}

// Any rows, one a group: a thread's channels are G apart, so that sums have the order of row_stream_odd_kernel.  Rows that are only rounded to 8 bits
// have no sums; there a thread takes four channels together, a word of the result.  (Linked norms are held to the registers of so many CTAs: 8192 rows of 4095
// 80 us with the 106 registers that they would take, 60 with 80.)
template <int G, int V, bool kIn32, int kOut, bool kNorm>
__global__ void __launch_bounds__(G <= 32 ? 128 : G, kOut == RO_Q8 && kNorm ? (G <= 32 ? (V == 2 ? 8 : 5) : V == 2 ? 10 : G == 512 ? 2 : 768 / G) : 0)
row_odd_kernel(const RowParams p) {
    constexpr int per_cta = G <= 32 ? 128 / G : 1;
    constexpr bool words = kOut == RO_Q8 && !kNorm;
    __shared__ uint32_t red[4][32];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x % G;
    const long long row = (long long)blockIdx.x * per_cta + threadIdx.x / G;
    const bool live = row < p.rows;
    auto col = [&](int i) { return words ? ((i >> 2) * G + t) * 4 + (i & 3) : i * G + t; };
    float x[8 * V];
#pragma unroll
    for (int i = 0; i < 8 * V; ++i)
        x[i] = !(live && col(i) < p.C) ? 0.0f : kIn32 ? ld_scalar(static_cast<const float *>(p.x) + row * p.C + col(i))
                                                      : ld_scalar(static_cast<const __nv_bfloat16 *>(p.x) + row * p.C + col(i));
    if (kNorm) {
        const float inv = 1.0f / (float)p.C;
        float s = 0.0f, e = 0.0f;
#pragma unroll
        for (int i = 0; i < 8 * V; ++i) s += x[i];                      // (zeros outside the row)
        const float mu = __fdiv_rn(row_sum<G>(s, red[0]), (float)p.C);
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8 * V; ++i) {
            x[i] = col(i) < p.C ? x[i] - mu : 0.0f;
            e += x[i];
            s = fmaf(x[i], x[i], s);
        }
        const float2 f = row_sum2<G>(s, e, red[1], red[2]);
        const float off = f.y * inv, rstd = rsqrtf(fmaxf(fmaf(f.x, inv, -off * off), 0.0f) + p.eps);
#pragma unroll
        for (int i = 0; i < 8 * V; ++i) {
            const int c = col(i);
            if (c >= p.C) continue;
            x[i] = fmaf(fmaf(x[i], rstd, -off * rstd), __ldg(p.gamma + c), __ldg(p.beta + c));
            // (a row that is rounded to 8 bits is rounded to bf16 first, as it would be between two kernels)
            if (kOut == RO_Q8) x[i] = __bfloat162float(__float2bfloat16_rn(x[i]));
        }
    }
    if (kOut == RO_Q8) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8 * V; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
        const RowScale sc = row_scale(row_max<G>(m, red[3]));
        if (words && !live) return;
        if (live && t == 0) p.scale[row] = sc.scale;
        // channels G apart: four threads with four channels each exchange halves, then bytes, and each has four channels that lie together
        const bool up2 = t & 2, up1 = t & 1;
#pragma unroll
        for (int i = 0; i < 8 * V; i += 4) {
            uint32_t q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) q[k] = row_quant<kIn32 && !kNorm>(x[i + k], sc);
            uint32_t w = row_bytes4(q[0], q[1], q[2], q[3]);
            int at = col(i);
            if (!words) {
                const uint32_t far2 = __shfl_xor_sync(0xffffffffu, w, 2);
                w = up2 ? __byte_perm(far2, w, 0x7632) : __byte_perm(w, far2, 0x5410);
                const uint32_t far1 = __shfl_xor_sync(0xffffffffu, w, 1);
                w = up1 ? __byte_perm(far1, w, 0x7351) : __byte_perm(w, far1, 0x6240);
                at = (i + (t & 3)) * G + (t & ~3);
                if (!live) continue;
            }
            // (rows are filled up to the pitch, a multiple of 128, with zeros: x = 0 there)
            if (at < p.pitch) *reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(p.y) + row * p.pitch + at) = w;
        }
        return;
    }
    if (!live) return;
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) {
        const int c = col(i);
        if (c >= p.C) continue;
        if (kOut == RO_F32) static_cast<float *>(p.y)[row * p.pitch + c] = x[i];
        else static_cast<__nv_bfloat16 *>(p.y)[row * p.pitch + c] = __float2bfloat16_rn(x[i]);
    }
}

// Layer norm of many rows of any length, as row_stream_kernel: a thread's channels are G apart, so that gamma and beta stay in registers whatever the
// rows' alignment; the copy engine brings the 16-byte pieces that a row meets, its neighbours' ends with them, but nothing behind the tensor (the
// last row's end is read from where it is).
template <int G, int V, int A, bool kIn32, int kOut>
__global__ void __launch_bounds__(G, 512 / G)
row_stream_odd_kernel(const RowParams p) {
    constexpr int S = 2, ES = kIn32 ? 4 : 2, N = 8 * V;
    extern __shared__ __align__(128) uint8_t row_slots[];
    __shared__ uint32_t red[3][32];
    __shared__ __align__(8) unsigned long long full[S];
    pdl_launch_dependents();
    const int t = threadIdx.x;
    const uint32_t slot = ((uint32_t)p.C * ES + 15u & ~15u) + 16u, slots = smem_u32(row_slots), bars = smem_u32(full);
    if (t < S) mbar_init(bars + 8u * t, 1u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    float ga[N], be[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = i * G + t;
        ga[i] = c < p.C ? __ldg(p.gamma + c) : 0.0f; be[i] = c < p.C ? __ldg(p.beta + c) : 0.0f;
    }
    __syncthreads();
    pdl_wait();
    auto ask = [&](long long row, int s) {
        if (t != 0 || row >= p.rows) return;
        const unsigned long long from = row * (unsigned long long)(p.C * ES), to = from + (unsigned)(p.C * ES);
        const unsigned long long a = from & ~15ull, b = row + 1 < p.rows ? (to + 15) & ~15ull : to & ~15ull;
        const uint32_t bytes = b > a ? (uint32_t)(b - a) : 0u;
        mbar_arrive_expect_tx(bars + 8u * s, bytes);
        if (bytes) bulk_load(slots + (uint32_t)s * slot, static_cast<const char *>(p.x) + a, bytes, bars + 8u * s);
    };
#pragma unroll
    for (int s = 0; s < S; ++s) ask(blockIdx.x + (long long)s * gridDim.x, s);
    bool dead = false;                     // (a wait ran out: the rows that are left are walked over without waiting, so that every barrier is met)
    int s = 0;
    uint32_t ph = 0u;
    const float inv = 1.0f / (float)p.C;
#pragma unroll 1
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
        if (!dead && !mbar_wait(bars + 8u * s, ph)) {
            dead = true;
            atomicCAS(p.status, 0u, kStatusTimeout | (3u << 8) | (((unsigned)p.launch_id & 0xfffu) << 12));
        }
        const unsigned long long from = row * (unsigned long long)(p.C * ES);
        const uint32_t lead = (uint32_t)(from & 15ull);
        // channels that came by copy
        const int came = row + 1 < p.rows ? p.C : (int)(((from + (unsigned)(p.C * ES)) & ~15ull) > from ? (((from + (unsigned)(p.C * ES)) & ~15ull) - from) / ES : 0);
        const uint8_t *at = row_slots + (size_t)s * slot + lead;
        float x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * G + t;
            if (kIn32) x[i] = c < came ? reinterpret_cast<const float *>(at)[c] : 0.0f;
            else x[i] = c < came ? __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(at)[c]) : 0.0f;
        }
        if (came < p.C) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = i * G + t;
                if (c >= came && c < p.C) x[i] = kIn32 ? ld_scalar(static_cast<const float *>(p.x) + row * p.C + c) : ld_scalar(static_cast<const __nv_bfloat16 *>(p.x) + row * p.C + c);
            }
        }
        float a[A] = {}, e[A] = {};          // (sums of columns, as row_kernel has them)
#pragma unroll
        for (int i = 0; i < N; ++i) a[i % A] += x[i];
        const float mu = __fdiv_rn(row_sum<G, A>(a, red[0]), (float)p.C);
        ask(row + (long long)S * gridDim.x, s);
        if (++s == S) { s = 0; ph ^= 1u; }
#pragma unroll
        for (int i = 0; i < A; ++i) a[i] = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = i * G + t < p.C ? x[i] - mu : 0.0f;
            e[i % A] += x[i];
            a[i % A] = fmaf(x[i], x[i], a[i % A]);
        }
        const float2 f = row_sum2<G, A>(a, e, red[1], red[2]);
        const float off = f.y * inv, rstd = rsqrtf(fmaxf(fmaf(f.x, inv, -off * off), 0.0f) + p.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * G + t;
            if (c >= p.C) continue;
            const float y = fmaf(fmaf(x[i], rstd, -off * rstd), ga[i], be[i]);
            if (kOut == RO_F32) static_cast<float *>(p.y)[row * p.pitch + c] = y;
            else static_cast<__nv_bfloat16 *>(p.y)[row * p.pitch + c] = __float2bfloat16_rn(y);
        }
    }
    if (dead) for (int i = 0; i < 64; ++i) __nanosleep(1000);      // (time for copies under way)
}

// Rows that no group holds in registers (more than 16384 channels): a CTA walks over its row once per pass, from L2 after the first.
template <bool kIn32, int kOut, bool kNorm>
__global__ void __launch_bounds__(512)
row_long_kernel(const RowParams p) {
    __shared__ uint32_t red[4][32];
    pdl_launch_dependents();
    pdl_wait();
    const long long row = blockIdx.x;
    auto at = [&](int c) {
        return kIn32 ? ld_scalar(static_cast<const float *>(p.x) + row * p.C + c) : ld_scalar(static_cast<const __nv_bfloat16 *>(p.x) + row * p.C + c);
    };
    float mu = 0.0f, off = 0.0f, rstd = 1.0f;
    if (kNorm) {
        const float inv = 1.0f / (float)p.C;
        float s = 0.0f, e = 0.0f;
#pragma unroll 8
        for (int c = threadIdx.x; c < p.C; c += 512) s += at(c);
        mu = __fdiv_rn(row_sum<512>(s, red[0]), (float)p.C);
        s = 0.0f;
#pragma unroll 8
        for (int c = threadIdx.x; c < p.C; c += 512) { const float d = at(c) - mu; s = fmaf(d, d, s); e += d; }
        const float2 f = row_sum2<512>(s, e, red[1], red[2]);
        off = f.y * inv;
        rstd = rsqrtf(fmaxf(fmaf(f.x, inv, -off * off), 0.0f) + p.eps);
    }
    auto value = [&](int c) {
        const float x = at(c);
        if (!kNorm) return x;
        const float y = fmaf(((x - mu) - off) * rstd, __ldg(p.gamma + c), __ldg(p.beta + c));
        return kOut == RO_Q8 ? __bfloat162float(__float2bfloat16_rn(y)) : y;
    };
    if (kOut == RO_Q8) {
        uint32_t m = 0;
#pragma unroll 8
        for (int c = threadIdx.x; c < p.C; c += 512) m = max(m, __float_as_uint(value(c)) & 0x7fffffffu);
        const RowScale sc = row_scale(row_max<512>(m, red[3]));
        if (threadIdx.x == 0) p.scale[row] = sc.scale;
        for (int c = threadIdx.x; c < p.pitch; c += 512)
            (static_cast<uint8_t *>(p.y) + row * p.pitch)[c] = c < p.C ? (uint8_t)row_quant<kIn32 && !kNorm>(value(c), sc) : (uint8_t)0;
    } else {
        for (int c = threadIdx.x; c < p.C; c += 512) {
            if (kOut == RO_F32) static_cast<float *>(p.y)[row * p.pitch + c] = value(c);
            else static_cast<__nv_bfloat16 *>(p.y)[row * p.pitch + c] = __float2bfloat16_rn(value(c));
        }
    }
}

}  // namespace xk
