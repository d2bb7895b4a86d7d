// Matrix product in 8-bit integers: y[m][n] = act(sx[m] * sw[n] * sum_k q[m][k] w[n][k] + b[n]), q and w int8, the sum exact in int32
// (at most 131072 products), one scale per row of the activation (found by row_kernel) and per output channel.  The sum is converted to fp32
// and the product of the scales is applied there (the sum times one scale alone could leave the range of fp32): three roundings of 2^-24,
// then one to the result's type.
//
// q8_tc_kernel (more than 16 rows): tcgen05.mma kind::i8 (32 products deep per instruction, twice the rate of bf16), both operands K-major
// by the copy engine in blocks of 128 bytes, 128-byte swizzle, as the bf16 kernels have them.  Roles as in conv_tc_kernel: warp 0 activation, warp
// 1 products, warp 2 weights (constants: they arrive while the predecessor drains), warp 3 tensor memory, warps 4-11 epilogue of tile i
// beside the products of tile i + 1.
//   one CTA   tiles of 128 rows x 32..256 channels, for products whose larger tiles would leave SMs idle
//   a pair    two CTAs of a cluster share a tile of 256 x 256 (cta_group::2): each brings its 128 rows of both operands, so a block of 128 deep
//             takes 32 KB per SM for 512 cycles of the tensor pipe instead of 48 KB (L2 gives an SM some 75 bytes a cycle)
// Results leave through 32-row boxes in shared memory by bulk tensor stores (4096 x 1024 x 16384: 69 us, 3 more where the threads store 16-byte pieces of
// rows); rows that are not whole 16-byte pieces leave element by element (16383 channels: 123).
//
// q8_small_kernel (up to 16 rows): a pass over the weights, bound by their bytes.  A CTA owns 16 channels, its 8 warps share the
// depth; mma.sync takes the channels as its 16 rows and the activation's rows as its 8 columns (tcgen05 has no shape that reads
// weights from registers).  The weights (512 bytes of depth a warp and channel, and while those are used the next) are asked for before the predecessor is waited
// for.  Each CTA stays for several sets of channels where there are many; it finds the rows' scales and
// rounds the rows to shared memory by itself: no second launch, but work that every CTA repeats, so the rule is 16384 values in all (4096 x 4096: 4
// rows 7.4 us here and 10.5 there; 16 rows 19 and 10.5).
#pragma once

#include "conv_tc.cuh"
#include "rows.cuh"

namespace xk {

constexpr int kQ8Threads = 384, kQ8EpiWarps = 8, kQ8MaxStages = 8;
// Registers as for more threads (128 instead of 168): a CTA then fits beside those of the row kernel that it follows, and sets itself up while they work.
constexpr int kQ8RegThreads = 512;

struct Q8Params {
    const float *xs;               // scale per row
    const float *ws, *bias;        // per channel
    void *y;
    unsigned int *status;
    int M, N, kblocks;             // rows, channels, blocks of 128 deep
    int tile_n, m_tiles, n_tiles, stages, stage_bytes, tmem_cols;
    int per_stage;                 // blocks of a stage: 2 where a tile is narrow
    uint32_t a_bytes;              // a box of the activation (its rows x 128)
    int act, out_f32, vec;         // vec: rows of the result are whole 16-byte pieces
    int wide;                      // boxes of 64 channels of bf16 (else 32): 128 bytes a row either way where it counts
    int off_stage, off_par, off_bar;
    uint32_t idesc;
    int launch_id;
};

__device__ __forceinline__ float q8_act(float v, int act) {      // (a NaN stays one)
    if (act >= 1) v = v < 0.0f ? 0.0f : v;
    if (act == 2) v = v > 6.0f ? 6.0f : v;
    return v;
}

template <int kPair>
__device__ __forceinline__ void q8_load(uint32_t dst, const CUtensorMap *tm, int x, int y, uint32_t bar) {
    if (kPair == 2)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
            ::"r"(dst), "l"(tm), "r"(bar & 0xfeffffffu), "r"(x), "r"(y) : "memory");      // (the barrier of the pair's first CTA)
    else tma_load_2d(dst, tm, x, y, bar);
}
// Arrival at a barrier of every CTA of the tile when the products issued so far are done.
template <int kPair>
__device__ __forceinline__ void q8_commit(uint32_t bar) {
    if (kPair == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((unsigned short)3) : "memory");
    else umma_commit(bar);
}
// The products of a stage (four of 32 deep per block of 128, `two` blocks or one), their commit to the barrier that frees it, and the
// state of the next stage's barrier: asked for first, looked at last (see umma_block).  Descriptors' lower halves in 16-byte units; a_next, b_next:
// distance of the second block's operands.
#define XENOS_Q8_STAGE(GROUP, COMMIT)                                                                                                          \
    asm volatile(                                                                                                                              \
        "{\n\t.reg .pred p, q, w;\n\t.reg .b64 da, db;\n\t.reg .b32 x, y;\n\t"                                                                  \
        "mbarrier.test_wait.parity.shared::cta.b64 q, [%11], %12;\n\t"                                                                         \
        "setp.ne.b32 p, %8, 0;\n\tsetp.ne.b32 w, %9, 0;\n\t"                                                                                   \
        "mov.b64 da, {%3, %2};\n\tmov.b64 db, {%4, %2};\n\ttcgen05.mma." GROUP ".kind::i8 [%1], da, db, %7, p;\n\tsetp.eq.u32 p, 0, 0;\n\t"   \
        "add.u32 x, %3, 2;\n\tadd.u32 y, %4, 2;\n\tmov.b64 da, {x, %2};\n\tmov.b64 db, {y, %2};\n\ttcgen05.mma." GROUP ".kind::i8 [%1], da, db, %7, p;\n\t" \
        "add.u32 x, %3, 4;\n\tadd.u32 y, %4, 4;\n\tmov.b64 da, {x, %2};\n\tmov.b64 db, {y, %2};\n\ttcgen05.mma." GROUP ".kind::i8 [%1], da, db, %7, p;\n\t" \
        "add.u32 x, %3, 6;\n\tadd.u32 y, %4, 6;\n\tmov.b64 da, {x, %2};\n\tmov.b64 db, {y, %2};\n\ttcgen05.mma." GROUP ".kind::i8 [%1], da, db, %7, p;\n\t" \
        "add.u32 x, %3, %5;\n\tadd.u32 y, %4, %6;\n\tmov.b64 da, {x, %2};\n\tmov.b64 db, {y, %2};\n\t@w tcgen05.mma." GROUP ".kind::i8 [%1], da, db, %7, p;\n\t" \
        "add.u32 x, x, 2;\n\tadd.u32 y, y, 2;\n\tmov.b64 da, {x, %2};\n\tmov.b64 db, {y, %2};\n\t@w tcgen05.mma." GROUP ".kind::i8 [%1], da, db, %7, p;\n\t" \
        "add.u32 x, x, 2;\n\tadd.u32 y, y, 2;\n\tmov.b64 da, {x, %2};\n\tmov.b64 db, {y, %2};\n\t@w tcgen05.mma." GROUP ".kind::i8 [%1], da, db, %7, p;\n\t" \
        "add.u32 x, x, 2;\n\tadd.u32 y, y, 2;\n\tmov.b64 da, {x, %2};\n\tmov.b64 db, {y, %2};\n\t@w tcgen05.mma." GROUP ".kind::i8 [%1], da, db, %7, p;\n\t" \
        COMMIT "selp.u32 %0, 1, 0, q;\n\t}"                                                                                                    \
        : "=r"(ready)                                                                                                                          \
        : "r"(d), "r"(hi), "r"(a), "r"(b), "r"(a_next), "r"(b_next), "r"(idesc), "r"(acc), "r"(two), "r"(freed), "r"(next), "r"(next_ph), "h"((unsigned short)3) \
        : "memory")
template <int kPair>
__device__ __forceinline__ uint32_t q8_stage(uint32_t d, uint32_t a, uint32_t b, uint32_t a_next, uint32_t b_next, uint32_t idesc, uint32_t acc, uint32_t two,
                                             uint32_t freed, uint32_t next, uint32_t next_ph) {
    constexpr uint32_t hi = 64u | (1u << 14) | (2u << 29);      // 128-byte swizzle, 1024-byte groups
    uint32_t ready;
    if (kPair == 2)
        XENOS_Q8_STAGE("cta_group::2", "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%10], %13;\n\t");
    else
        XENOS_Q8_STAGE("cta_group::1", "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%10];\n\t");
    return ready;
}
#undef XENOS_Q8_STAGE
// One arrival at the barrier with this offset in the tile's first CTA.
template <int kPair>
__device__ __forceinline__ void q8_arrive_first(uint32_t bar) {
    if (kPair == 2) {
        uint32_t far;
        asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(far) : "r"(bar));
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(far) : "memory");
    } else mbar_arrive(bar);
}

// Tiles in bands of 8 row tiles, row tiles fastest: CTAs at work at the same time share rows and channels through L2.
struct Q8Tile { int mt, nt; };
__device__ __forceinline__ Q8Tile q8_tile(const Q8Params &g, int ti) {
    const int band = 8 * g.n_tiles, b = ti / band, rem = ti - b * band, h = min(8, g.m_tiles - 8 * b);
    Q8Tile t;
    t.nt = rem / h; t.mt = 8 * b + rem - t.nt * h;
    return t;
}

template <int kPair>
__global__ void __launch_bounds__(kQ8RegThreads, 1)
q8_tc_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmO, const __grid_constant__ Q8Params g) {
    extern __shared__ uint8_t smem_raw[];
    pdl_launch_dependents();
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t sbase = (raw + 1023u) & ~1023u;
    uint8_t *sm = smem_raw + (sbase - raw);
    const uint32_t bar = sbase + g.off_bar;
    auto full_bar = [&](int s) { return bar + 8u * s; };                          // 2 arrivals and the bytes
    auto empty_bar = [&](int s) { return bar + 8u * (kQ8MaxStages + s); };
    auto accf_bar = [&](int b) { return bar + 8u * (2 * kQ8MaxStages + b); };
    auto acce_bar = [&](int b) { return bar + 8u * (2 * kQ8MaxStages + 2 + b); }; // of the tile's first CTA
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(sm + g.off_bar + 8 * (2 * kQ8MaxStages + 4));
    volatile int *gave_up = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = kPair == 2 ? (int)(blockIdx.x & 1) : 0;
    if (warp == 0) {
        if (lane < 2 * kQ8MaxStages + 4)
            mbar_init(bar + 8u * lane, lane < kQ8MaxStages ? 2u : lane < 2 * kQ8MaxStages + 2 ? 1u : (uint32_t)(kPair * kQ8EpiWarps));
        if (lane == 0) *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmA) : "memory");
        if (lane == 1) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmB) : "memory");
    }
    if (warp == 3) {
        if (kPair == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)g.tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)g.tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (kPair == 2) cluster_sync();              // the other CTA's barriers exist
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const int total = g.m_tiles * g.n_tiles, step = (int)gridDim.x / kPair, first = (int)blockIdx.x / kPair;
    bool ok = true;
    const unsigned word = kStatusTimeout | (((unsigned)g.launch_id & 0xfffu) << 12);

    if (warp == 0 || warp == 2) {
        // ---- operands: 128 rows of the activation, tile_n channels of the weights (a pair: 128 each) ----
        if (elect_one()) {
            const bool act = warp == 0;
            const int boxes = !act && kPair == 1 && g.tile_n == 256 ? 2 : 1, per = in_reg(g.per_stage);
            const uint32_t box = act ? g.a_bytes : (uint32_t)min(g.tile_n, 128) * 128u;
            const uint32_t bytes = box * boxes * kPair, step_k = act ? 16384u : (uint32_t)g.tile_n * 128u;      // what a block delivers; where the next one goes
            const uint32_t off = act ? 0u : 16384u * per;
            const CUtensorMap *tm = act ? &tmA : &tmB;
            const int kblocks = in_reg(g.kblocks), stages = in_reg(g.stages);
            if (act) pdl_wait();
            int s = 0, n = 0;
            uint32_t ph = 1u;
#pragma unroll 1
            for (int ti = first; ti < total && ok; ti += step) {
                const Q8Tile t = q8_tile(g, ti);
                const int row = act ? (t.mt * kPair + rank) * 128 : t.nt * g.tile_n + rank * 128;
#pragma unroll 1
                for (int kb = 0; kb < kblocks; kb += per) {
                    if (n >= stages && !mbar_wait(empty_bar(s), ph)) { ok = false; break; }
                    const uint32_t dst = sbase + (uint32_t)s * g.stage_bytes + off;
                    const bool two = per == 2 && kb + 1 < kblocks;
                    if (rank == 0) mbar_arrive_expect_tx(full_bar(s), two ? 2 * bytes : bytes);
                    q8_load<kPair>(dst, tm, kb * 128, row, full_bar(s));
                    if (boxes == 2) q8_load<kPair>(dst + 16384u, tm, kb * 128, row + 128, full_bar(s));
                    if (two) q8_load<kPair>(dst + step_k, tm, kb * 128 + 128, row, full_bar(s));
                    ++n;
                    if (++s == stages) { s = 0; ph ^= 1u; }
                }
            }
            // every slot has been read: no signal is on its way to this CTA's barriers any more
            if (act && n < stages) { s = 0; ph = 0u; }
            for (int i = min(n, stages); act && ok && i > 0; --i) {
                ok = mbar_wait(empty_bar(s), ph);
                if (++s == stages) { s = 0; ph ^= 1u; }
            }
            if (!ok) { *gave_up = 1; atomicCAS(g.status, 0u, word | (1u << 8)); }
        }
    } else if (warp == 1 && rank == 0) {
        // ---- products ----
        if (elect_one()) {
            const int kblocks = in_reg(g.kblocks), stages = in_reg(g.stages), per = in_reg(g.per_stage);
            const uint32_t idesc = in_reg(g.idesc), stage16 = in_reg((uint32_t)g.stage_bytes >> 4), first16 = 0x10000u | (sbase >> 4);
            const uint32_t b_off = 1024u * per, b_next = in_reg((uint32_t)g.tile_n * 8u);
            int s = 0, i = 0;
            uint32_t ph = 0u, ready = 0u, a16 = first16;
#pragma unroll 1
            for (int ti = first; ti < total && ok; ti += step, ++i) {
                const int b = i & 1;
                if (i > 1 && !mbar_wait(acce_bar(b), ((i >> 1) & 1) ^ 1u)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d = tmem_base + (uint32_t)(b * g.tile_n);
#pragma unroll 1
                for (int kb = 0; kb < kblocks; kb += per) {
                    if (!ready && !mbar_wait(full_bar(s), ph)) { ok = false; break; }
                    const uint32_t freed = empty_bar(s), now = a16;
                    const bool wrap = s + 1 == stages;
                    s = wrap ? 0 : s + 1;
                    a16 = wrap ? first16 : a16 + stage16;
                    ph ^= wrap ? 1u : 0u;
                    ready = q8_stage<kPair>(d, now, now + b_off, 1024u, b_next, idesc, kb, per == 2 && kb + 1 < kblocks, freed, full_bar(s), ph);
                }
                if (ok) q8_commit<kPair>(accf_bar(b));
            }
            if (!ok) { *gave_up = 1; atomicCAS(g.status, 0u, word | (2u << 8)); }
        }
    } else if (warp >= 4) {
        // ---- epilogue ----
        pdl_wait();
        const int e = warp - 4, quarter = warp & 3, half = e >> 2;
        const uint32_t t_warp = tmem_base + ((uint32_t)(quarter * 32) << 16);
        uint8_t *box = sm + g.off_stage + e * 4096;
        // the warp's s-th chunk of 32 columns: two warps of a quarter take turns, two chunks at a time where a box holds those
        const bool wide = g.wide;
        auto chunk = [&](int s) { return wide ? 4 * (s >> 1) + 2 * half + (s & 1) : half + 2 * s; };
        float *pars = reinterpret_cast<float *>(sm + g.off_par + e * 1024);
        const int chunks = g.tile_n / 32;
        int i = 0;
#pragma unroll 1
        for (int ti = first; ti < total && ok; ti += step, ++i) {
            const Q8Tile t = q8_tile(g, ti);
            const int b = i & 1, m0 = (t.mt * kPair + rank) * 128 + quarter * 32;
            const float sx = m0 + lane < g.M ? g.xs[m0 + lane] : 0.0f;
            // scales and biases of the warp's chunks, on their way while the tile is multiplied
            float wv[4], bv[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int x = t.nt * g.tile_n + chunk(c) * 32 + lane;
                const bool in = chunk(c) < chunks && x < g.N;
                wv[c] = in ? __ldg(g.ws + x) : 0.0f; bv[c] = in ? __ldg(g.bias + x) : 0.0f;
            }
            __syncwarp();                                        // (those of the tile before have been read)
#pragma unroll
            for (int c = 0; c < 4; ++c) { pars[c * 64 + lane] = wv[c]; pars[c * 64 + 32 + lane] = bv[c]; }
            if (!mbar_wait(accf_bar(b), (i >> 1) & 1)) { ok = false; break; }
            tc_fence_after();
#pragma unroll 1
            for (int s = 0; chunk(s) < chunks; ++s) {
                const int j = chunk(s), x0 = t.nt * g.tile_n + j * 32, x = x0 + lane;
                const bool upper = wide && (s & 1);              // the right half of a box
                const float *par = pars + s * 64;
                float v[32];
                tmem_ld32(t_warp + b * g.tile_n + j * 32, v);
                if (g.vec && !upper && elect_one()) bulk_wait_read<0>();      // the store that last left the box has read it
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                    const float4 w = *reinterpret_cast<const float4 *>(par + c), bb = *reinterpret_cast<const float4 *>(par + 32 + c);
                    v[c] = fmaf((float)__float_as_int(v[c]), sx * w.x, bb.x);
                    v[c + 1] = fmaf((float)__float_as_int(v[c + 1]), sx * w.y, bb.y);
                    v[c + 2] = fmaf((float)__float_as_int(v[c + 2]), sx * w.z, bb.z);
                    v[c + 3] = fmaf((float)__float_as_int(v[c + 3]), sx * w.w, bb.w);
                }
                if (g.act) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) v[c] = q8_act(v[c], g.act);
                }
                if (g.out_f32) {
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        *reinterpret_cast<float4 *>(box + lane * 128 + ((c ^ (lane & 7)) << 4)) = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
                } else {
                    const uint32_t row = wide ? lane * 128 : lane * 64, c0 = upper ? 4u : 0u, turn = wide ? lane & 7 : (lane >> 1) & 3;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        *reinterpret_cast<uint4 *>(box + row + (((c0 + c) ^ turn) << 4)) =
                            make_uint4(pack2(v[8 * c], v[8 * c + 1]), pack2(v[8 * c + 2], v[8 * c + 3]), pack2(v[8 * c + 4], v[8 * c + 5]), pack2(v[8 * c + 6], v[8 * c + 7]));
                }
                if (wide && !upper) continue;
                if (g.vec) {
                    fence_proxy_async();
                    __syncwarp();
                    // (what reaches behind the last row or channel is not stored)
                    if (elect_one()) { tma_store_2d(&tmO, smem_u32(box), upper ? x0 - 32 : x0, m0); bulk_commit(); }
                    __syncwarp();
                    continue;
                }
                __syncwarp();
                if (x < g.N) {
#pragma unroll 8
                    for (int r = 0; r < 32; ++r) {
                        if (m0 + r >= g.M) continue;
                        if (g.out_f32)
                            static_cast<float *>(g.y)[(size_t)(m0 + r) * g.N + x] = *reinterpret_cast<const float *>(box + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4);
                        else
                            static_cast<__nv_bfloat16 *>(g.y)[(size_t)(m0 + r) * g.N + x] =
                                *reinterpret_cast<const __nv_bfloat16 *>(box + r * 64 + (((lane >> 3) ^ ((r >> 1) & 3)) << 4) + (lane & 7) * 2);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) q8_arrive_first<kPair>(acce_bar(b));
        }
        if (elect_one()) bulk_wait_read<0>();
        __syncwarp();
        if (!ok && lane == 0) { *gave_up = 1; atomicCAS(g.status, 0u, word | (5u << 8)); }
    }
    tc_fence_before();
    __syncthreads();
    // (after a give-up: time for the copies and products under way)
    if (*gave_up) for (int i = 0; i < 64; ++i) __nanosleep(1000);
    if (kPair == 2) cluster_sync();
    if (warp == 3) {
        tc_fence_after();
        if (kPair == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)g.tmem_cols) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)g.tmem_cols) : "memory");
    }
}

// ---- few rows --------------------------------------------------------------------------------------------------------------
struct Q8SmallParams {
    const void *x;
    const uint8_t *w;              // [N][pitch]
    const float *ws, *bias;
    void *y;
    int M, N, K, pitch;
    int act, out_f32, vec;         // vec: rows of x are whole 16-byte pieces
};
__device__ __forceinline__ void mma_s8(int *c, const uint32_t *a, const uint32_t *b) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
// Eight consecutive values of a row from k on (zeros behind the row).
template <bool kIn32>
__device__ __forceinline__ void q8_values(const Q8SmallParams &g, int m, int k, float *v) {
    if (g.vec && k + 8 <= g.K) {
        if (kIn32) {
            const float4 *q = reinterpret_cast<const float4 *>(static_cast<const float *>(g.x) + (size_t)m * g.K + k);
            const float4 a = q[0], b = q[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const f8 f = unpack8(*reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(g.x) + (size_t)m * g.K + k));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = f.v[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = k + i >= g.K ? 0.0f : kIn32 ? static_cast<const float *>(g.x)[(size_t)m * g.K + k + i]
                                               : __bfloat162float(static_cast<const __nv_bfloat16 *>(g.x)[(size_t)m * g.K + k + i]);
    }
}

// kN: rows of the activation in eights.  Shared memory: the rows rounded to 8 bits, pitch + 64 bytes apart (the lanes of a fragment's load then meet
// all banks).
template <int kN, bool kIn32>
__global__ void __launch_bounds__(256, 2)
q8_small_kernel(const Q8SmallParams g) {
    constexpr int U = 8;
    extern __shared__ __align__(16) uint8_t q8_rows[];
    __shared__ uint32_t peak[8 * kN];
    __shared__ int sums[8][8 * kN][17];
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = lane >> 2, q = lane & 3;
    const int ld = g.pitch + 64, sets = (g.N + 15) / 16;
    // a step is 64 bytes of depth: the lane's 16 bytes of two channels are the operand of two products, in an order of the depth that both
    // operands share
    const int steps = g.pitch / 64;
    uint4 a[U], b[U];
    // step s of a set of channels (none behind the last)
    auto fetch = [&](int u, int set, int s) {
        if (s >= steps || set >= sets) return;
        const uint8_t *w = g.w + (size_t)s * 64 + q * 16;
        a[u] = ld_stream16(w + (size_t)min(set * 16 + grp, g.N - 1) * g.pitch); b[u] = ld_stream16(w + (size_t)min(set * 16 + 8 + grp, g.N - 1) * g.pitch);
    };
#pragma unroll
    for (int u = 0; u < U; ++u) fetch(u, blockIdx.x, warp + 8 * u);
    if (threadIdx.x < 8 * kN) peak[threadIdx.x] = 0u;
    __syncthreads();
    pdl_wait();
    // ---- the rows' largest magnitudes, then their values: 256, 128, 64 or 32 threads a row (whole warps)
    const int lg = g.M <= 1 ? 8 : g.M <= 2 ? 7 : g.M <= 4 ? 6 : 5, tr = threadIdx.x & ((1 << lg) - 1);
    for (int m = threadIdx.x >> lg; m < g.M; m += 256 >> lg) {
        uint32_t mx = 0;
#pragma unroll 4
        for (int k = tr * 8; k < g.K; k += 8 << lg) {
            float v[8];
            q8_values<kIn32>(g, m, k, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) mx = max(mx, __float_as_uint(v[i]) & 0x7fffffffu);
        }
        mx = __reduce_max_sync(0xffffffffu, mx);
        if (lane == 0) atomicMax(&peak[m], mx);
    }
    __syncthreads();
    for (int m = threadIdx.x >> lg; m < g.M; m += 256 >> lg) {
        const RowScale sc = row_scale(peak[m]);
#pragma unroll 2
        for (int k = tr * 8; k < g.pitch; k += 8 << lg) {
            float v[8];
            q8_values<kIn32>(g, m, k, v);
            uint32_t x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = row_quant<kIn32>(v[i], sc);
            *reinterpret_cast<uint2 *>(q8_rows + (size_t)m * ld + k) = make_uint2(row_bytes4(x[0], x[1], x[2], x[3]), row_bytes4(x[4], x[5], x[6], x[7]));
        }
    }
    __syncthreads();
    uint32_t at[kN];                       // (columns behind the last row repeat it; nobody reads their sums)
#pragma unroll
    for (int n = 0; n < kN; ++n) at[n] = smem_u32(q8_rows) + (uint32_t)(min(n * 8 + grp, g.M - 1) * ld + q * 16);
#pragma unroll 1
    for (int set = blockIdx.x; set < sets; set += gridDim.x) {
        int acc[kN][4];
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[n][i] = 0;
#pragma unroll 1
        for (int s0 = warp; s0 < steps; s0 += 8 * U) {
            const bool last = s0 + 8 * U >= steps;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int s = s0 + 8 * u;
                if (s < steps) {
#pragma unroll
                    for (int n = 0; n < kN; ++n) {
                        const uint4 xv = ld_shared16(at[n] + (uint32_t)s * 64u);
                        const uint32_t x[4] = {xv.x, xv.y, xv.z, xv.w};
                        const uint32_t a0[4] = {a[u].x, b[u].x, a[u].y, b[u].y}, a1[4] = {a[u].z, b[u].z, a[u].w, b[u].w};
                        mma_s8(acc[n], a0, x);
                        mma_s8(acc[n], a1, x + 2);
                    }
                }
                if (last) fetch(u, set + gridDim.x, warp + 8 * u);
                else fetch(u, set, s + 8 * U);
            }
        }
        // ---- the warps' sums
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            sums[warp][n * 8 + 2 * q][grp] = acc[n][0]; sums[warp][n * 8 + 2 * q + 1][grp] = acc[n][1];
            sums[warp][n * 8 + 2 * q][grp + 8] = acc[n][2]; sums[warp][n * 8 + 2 * q + 1][grp + 8] = acc[n][3];
        }
        __syncthreads();
        if (threadIdx.x < 128 * kN) {
            const int m = threadIdx.x >> 4, c = threadIdx.x & 15, n = set * 16 + c;
            if (m < g.M && n < g.N) {
                int s = 0;
#pragma unroll
                for (int w = 0; w < 8; ++w) s += sums[w][m][c];
                const float r = q8_act(fmaf((float)s, row_scale(peak[m]).scale * __ldg(g.ws + n), __ldg(g.bias + n)), g.act);
                if (g.out_f32) static_cast<float *>(g.y)[(size_t)m * g.N + n] = r;
                else static_cast<__nv_bfloat16 *>(g.y)[(size_t)m * g.N + n] = __float2bfloat16_rn(r);
            }
        }
        __syncthreads();
    }
}

}  // namespace xk
