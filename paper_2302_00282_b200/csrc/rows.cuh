// Row operators on the CUDA cores: layer normalisation over the channels of a row, and the rounding of a row to 8-bit integers
// with a scale of its own (what the 8-bit product reads).  A row is the channels of one pixel of an NHWC tensor.
//
//   norm       mu = mean(x), v = mean((x - mu)^2), y = (x - mu) / sqrt(v + eps) * gamma + beta
//   to 8 bits  a = max |x|, q = round(127 x / a) (halves to even), scale = a / 127;  a = 0: q = 0
//
// Both are bound by HBM: the row is read once, kept in registers as fp32 and written once.  A group of G threads owns a row, each
// thread V chunks of 8 consecutive channels (one 16-byte access of bf16, two of fp32); G and V are the smallest that hold the row, so
// that short rows share a warp and no thread idles.  Mean and squared deviations are two reductions over the registers, not the
// difference of two sums over memory, which would lose the digits of a variance that is small against the mean; the second one also sums
// the deviations d, whose mean is the rounding of the first mean: (d - mean d) is exact to the last digits of d also for rows far from zero.
// The reductions of a
// group of several warps go through shared memory; gamma and beta come through L1, the row past it.
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
};

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
template <int G>
__device__ __forceinline__ float row_sum(float v, uint32_t *red) {
    return __uint_as_float(row_reduce<G>(__float_as_uint(v), red, [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
template <int G>
__device__ __forceinline__ float2 row_sum2(float a, float b, uint32_t *ra, uint32_t *rb) {
#pragma unroll
    for (int s = (G < 32 ? G : 32) / 2; s >= 1; s >>= 1) { a += __shfl_xor_sync(0xffffffffu, a, s); b += __shfl_xor_sync(0xffffffffu, b, s); }
    if (G > 32) {
        if ((threadIdx.x & 31) == 0) { ra[threadIdx.x >> 5] = __float_as_uint(a); rb[threadIdx.x >> 5] = __float_as_uint(b); }
        __syncthreads();
        a = __uint_as_float(ra[0]); b = __uint_as_float(rb[0]);
#pragma unroll
        for (int w = 1; w < G / 32; ++w) { a += __uint_as_float(ra[w]); b += __uint_as_float(rb[w]); }
    }
    return make_float2(a, b);
}
template <int G>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t *red) {
    return row_reduce<G>(v, red, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

// Threads of a CTA and rows it takes.  Short rows: 256 threads, and several rows per group so that enough bytes are under way.
template <int G, int V> struct RowShape {
    static constexpr int threads = G <= 32 ? 256 : G;
    static constexpr int per_group = G <= 32 ? (V >= 4 ? 1 : 4 / V) : 1;
    static constexpr int rows = threads / G * per_group;
};

// kVec: rows are whole chunks and 16-byte aligned; else a thread's channels are G apart and loaded one by one.
template <int G, int V, bool kIn32, int kOut, bool kNorm, bool kVec>
__global__ void __launch_bounds__(RowShape<G, V>::threads)
row_kernel(const RowParams p) {
    constexpr int R = RowShape<G, V>::per_group;
    __shared__ uint32_t red[4][32];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x % G, grp = threadIdx.x / G;
    const long long row0 = (long long)blockIdx.x * RowShape<G, V>::rows + grp;
    float x[R][V][8];
    auto col = [&](int v, int i) { return kVec ? (v * G + t) * 8 + i : (v * 8 + i) * G + t; };
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const long long row = row0 + (long long)r * (RowShape<G, V>::threads / G);
        const bool live = row < p.rows;
        const long long base = row * p.C;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (kVec) {
                const bool in = live && col(v, 0) < p.C;
                if (kIn32) {
                    const float *q = static_cast<const float *>(p.x) + base + col(v, 0);
                    const uint4 z = make_uint4(0, 0, 0, 0), a = in ? ld_stream16(q) : z, b = in ? ld_stream16(q + 4) : z;
                    x[r][v][0] = __uint_as_float(a.x); x[r][v][1] = __uint_as_float(a.y); x[r][v][2] = __uint_as_float(a.z); x[r][v][3] = __uint_as_float(a.w);
                    x[r][v][4] = __uint_as_float(b.x); x[r][v][5] = __uint_as_float(b.y); x[r][v][6] = __uint_as_float(b.z); x[r][v][7] = __uint_as_float(b.w);
                } else {
                    const f8 u = unpack8(in ? ld_stream16(static_cast<const __nv_bfloat16 *>(p.x) + base + col(v, 0)) : make_uint4(0, 0, 0, 0));
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[r][v][i] = u.v[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = col(v, i);
                    x[r][v][i] = !(live && c < p.C) ? 0.0f : kIn32 ? ld_scalar(static_cast<const float *>(p.x) + base + c)
                                                                   : ld_scalar(static_cast<const __nv_bfloat16 *>(p.x) + base + c);
                }
            }
        }
    }
    if (kNorm) {
        const float inv = 1.0f / (float)p.C;
        float mu[R], rstd[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float s = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) s += x[r][v][i];          // (zero outside the row)
            mu[r] = __fdiv_rn(row_sum<G>(s, red[0]), (float)p.C);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float s = 0.0f, e = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = col(v, i) < p.C ? x[r][v][i] - mu[r] : 0.0f;
                    x[r][v][i] = d;
                    e += d;
                    s = fmaf(d, d, s);
                }
            const float2 f = row_sum2<G>(s, e, red[1], red[2]);
            mu[r] = f.y * inv;                               // (of the deviations, from here on)
            rstd[r] = rsqrtf(fmaxf(fmaf(f.x, inv, -mu[r] * mu[r]), 0.0f) + p.eps);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float ga[8], be[8];
            if (kVec) {
                const bool in = col(v, 0) < p.C;
                const float4 z = make_float4(0, 0, 0, 0);
                const float4 *gp = reinterpret_cast<const float4 *>(p.gamma + col(v, 0)), *bp = reinterpret_cast<const float4 *>(p.beta + col(v, 0));
                const float4 g0 = in ? __ldg(gp) : z, g1 = in ? __ldg(gp + 1) : z, b0 = in ? __ldg(bp) : z, b1 = in ? __ldg(bp + 1) : z;
                ga[0] = g0.x; ga[1] = g0.y; ga[2] = g0.z; ga[3] = g0.w; ga[4] = g1.x; ga[5] = g1.y; ga[6] = g1.z; ga[7] = g1.w;
                be[0] = b0.x; be[1] = b0.y; be[2] = b0.z; be[3] = b0.w; be[4] = b1.x; be[5] = b1.y; be[6] = b1.z; be[7] = b1.w;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = col(v, i);
                    ga[i] = c < p.C ? __ldg(p.gamma + c) : 0.0f; be[i] = c < p.C ? __ldg(p.beta + c) : 0.0f;
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float y = fmaf((x[r][v][i] - mu[r]) * rstd[r], ga[i], be[i]);
                    // (a row that is rounded to 8 bits is rounded to bf16 first, as it would be between two kernels)
                    if (kOut == RO_Q8) y = col(v, i) < p.C ? __bfloat162float(__float2bfloat16_rn(y)) : 0.0f;
                    x[r][v][i] = y;
                }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const long long row = row0 + (long long)r * (RowShape<G, V>::threads / G);
        const bool live = row < p.rows;
        const long long base = row * p.pitch;
        RowScale sc;
        if (kOut == RO_Q8) {
            uint32_t m = 0;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[r][v][i]) & 0x7fffffffu);
            sc = row_scale(row_max<G>(m, red[3]));
            if (live && t == 0) p.scale[row] = sc.scale;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (kOut == RO_Q8) {
                uint32_t q[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) q[i] = row_quant<kIn32 && !kNorm>(x[r][v][i], sc);
                // (the row is filled up to its pitch with zeros: x = 0 there)
                if (kVec) {
                    if (live && col(v, 0) < p.pitch)
                        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(p.y) + base + col(v, 0)) =
                            make_uint2(q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24, q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (live && col(v, i) < p.pitch) (static_cast<uint8_t *>(p.y) + base)[col(v, i)] = (uint8_t)q[i];
                }
            } else if (kVec) {
                if (live && col(v, 0) < p.C) {
                    if (kOut == RO_F32) {
                        float4 *d = reinterpret_cast<float4 *>(static_cast<float *>(p.y) + base + col(v, 0));
                        d[0] = make_float4(x[r][v][0], x[r][v][1], x[r][v][2], x[r][v][3]);
                        d[1] = make_float4(x[r][v][4], x[r][v][5], x[r][v][6], x[r][v][7]);
                    } else {
                        f8 o;
#pragma unroll
                        for (int i = 0; i < 8; ++i) o.v[i] = x[r][v][i];
                        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.y) + base + col(v, 0)) = pack8(o);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (live && col(v, i) < p.C) {
                        if (kOut == RO_F32) static_cast<float *>(p.y)[base + col(v, i)] = x[r][v][i];
                        else static_cast<__nv_bfloat16 *>(p.y)[base + col(v, i)] = __float2bfloat16_rn(x[r][v][i]);
                    }
            }
        }
    }
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
