// Matrix products with an epilogue, on TMA + tcgen05 (include/linfusion_layers.h): the forward product x w, and the two of the
// backward pass, du w^T and x^T du.  All three are D[M, N] = A[M, K] B[K, N] with each operand contiguous along K or along its
// other axis, which the matrix instructions take either way: one kernel, no transposed copies.
//
// A tile is 256 x BN and belongs to a pair of CTAs on two SMs (cta_group::2: each holds 128 rows of A and of D and half of B, so a
// value of B is read from shared memory once for two SMs), or 128 x BN and one CTA.  Roles in a CTA: a TMA warp, an MMA warp (one
// thread, in the first CTA of a pair), and a group of four epilogue warps for every 64 columns of a tile; the accumulator is
// double-buffered in tensor memory, so a tile's epilogue runs under the next tile's products.  An epilogue has about 20 issue slots a value
// (K = 640); with gelu and the pre-activation in 8 bits it takes 24: its arithmetic runs on pairs of fp32 values, an instruction for two.
//
// Every SM is busy for the same time whatever the number of tiles: as many tiles as make whole rounds of the machine are dealt out whole,
// the K axes of the others are laid end to end and cut into equal runs, one for each pair.  A run that ends inside a tile
// leaves its fp32 sums in the workspace; the pair whose run has the tile's end adds them in the order of K (a fixed order)
// before its epilogue.  A pair does that unfinished tile first, then the tiles that it completes, then the whole ones (under whose
// products the joining disappears), and waits only for pairs before it, which were scheduled no later: waits are short, and
// bounded.
//
// What bounds it: an SM takes in about 64 bytes a cycle, 256 rows of 128 bytes a chunk in 512 cycles, which is also what the matrix
// instructions of a 256 x 256 tile take.  Narrower tiles load nearly as much for half the products; they serve where there
// are few tiles.  Measured (M x K x N, bf16; in brackets cuBLAS, the product alone): 32768 x 640 x 2560 88 us (1220 TFLOP/s; 86), with gelu 96 to
// 100, with gelu and the pre-activation in 8 bits 128 to 131 and in 16 bits 119; 8192 x 1280 x 5120 77 us (1390 TFLOP/s; 80); 8192 x 1280 x
// 1280 26 us (22); 2048 x 1280 x 1280 11.7 us (6.8); 128 x 1280 x 1280 5.9 us (3.8).  Of a small call's time 3 us are the launch, the first
// loads and the last tile's way out.
#pragma once

#include "block_kernels.cuh"
#include "column_sums.cuh"
#include "handover.h"
#include "pack8.cuh"
#include "sigmoid.cuh"

namespace lf {

static __device__ unsigned int linear_expired_waits;

constexpr int kLinKc = 64;           // K of a stage: 128 bytes of a row
constexpr int kLinRows = 128;        // rows of A and D in a CTA
constexpr int kLinColumns = 64;      // columns of D of an epilogue group: 128 bytes of a row
constexpr int kLinStaging = kLinRows * 128;

enum : int { kUNone = 0, kUFull = 1, kUPacked = 2 };

template <int CG, int BN>
struct LinCfg {
    static constexpr int A_BYTES = kLinRows * 128;
    static constexpr int B_BYTES = BN / CG * 128;
    static_assert(BN / CG == 64 || BN / CG == 128, "one or two blocks of 64 of B in a CTA");
    static constexpr int STAGE = A_BYTES + B_BYTES;
    static constexpr int GROUPS = BN / kLinColumns;
    static constexpr int STAGES = (224 * 1024 - GROUPS * kLinStaging) / STAGE > 8 ? 8 : (224 * 1024 - GROUPS * kLinStaging) / STAGE;
    static constexpr int TMEM_COLS = 2 * BN;
    static constexpr int EPILOGUE_WARPS = 4 * GROUPS, TMA_WARP = EPILOGUE_WARPS, MMA_WARP = TMA_WARP + 1;
    static constexpr int THREADS = 32 * (EPILOGUE_WARPS + 2);
    static constexpr int BIAS = BN * 4;  // the tile's bias in fp32
    static constexpr int SMEM = STAGES * STAGE + GROUPS * kLinStaging + BIAS + 1024 + 512;
    static_assert(SMEM <= 227 * 1024 && 16 * STAGES + 8 * (4 + GROUPS) + 4 <= 512, "shared memory of a CTA; barriers");
};

struct LinParams {
    int M, N, chunks;            // chunks of K
    int tiles_n, whole;          // tiles side by side; tiles that are dealt out whole
    int tiles;
    int a_mn, b_mn;              // an operand's contiguous axis is M / N, not K
    int act, u_mode, has_residual;
    const char* bias;            // 16-bit [N] or null
    signed char* codes;          // u in 8 bits; codes_map: through map_u (rows of whole 16-byte pieces)
    unsigned char* scales;
    int scale_groups, codes_map;
    int a_rows;                  // rows of A's boxes where K is contiguous: fewer than 128 where there are fewer
    float4* partials;            // [CTA][column / 4][row]
    Handover* flags;             // [CTA][group]: `mark` while the CTA's sums wait to be fetched, anything else before, 0 after
    Handover mark;               // another for every call; replays of a captured one find their flags taken down again
};

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void lin_cluster_sync()
{
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// A shared-memory address of this CTA as that of the same place in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t lin_map(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
template <int CG>
__device__ __forceinline__ void lin_load(uint32_t dst, const void* tmap, int x, int y, uint32_t bar)
{
    if constexpr (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(tmap), "r"(x), "r"(y), "r"(bar)
            : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                     "l"(tmap), "r"(x), "r"(y), "r"(bar)
                     : "memory");
}
__device__ __forceinline__ void lin_store(const void* tmap, uint32_t src, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(tmap), "r"(x), "r"(y), "r"(src) : "memory");
}
template <int CG>
__device__ __forceinline__ void lin_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (CG == 2)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
            "r"(idesc), "r"(accumulate)
            : "memory");
    else
        umma_ss(d, a, b, idesc, accumulate);
}
// One arrival on the barrier at this place in every CTA of the pair, once the MMAs issued so far are complete.
template <int CG>
__device__ __forceinline__ void lin_commit(uint32_t bar)
{
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                     "h"(static_cast<uint16_t>(3))
                     : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void lin_tmem_alloc(uint32_t* slot, uint32_t cols)
{
    if constexpr (CG == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        tmem_alloc(slot, cols);
    }
}
template <int CG>
__device__ __forceinline__ void lin_tmem_dealloc(uint32_t addr, uint32_t cols)
{
    if constexpr (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
    else tmem_dealloc(addr, cols);
}
__device__ __forceinline__ bool lin_wait(uint32_t bar, uint32_t parity)
{
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = global_timer_ns();
    do {
        if (mbar_try_wait(bar, parity)) return true;
    } while (global_timer_ns() - t0 < kMaxBarrierWaitNs);
    return false;
}
__device__ __forceinline__ void lin_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void lin_arrive(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ bool lin_all(int id, int threads, bool ok)
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.and.pred p, %2, %3, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r)
        : "r"(ok ? 1u : 0u), "r"(id), "r"(threads)
        : "memory");
    return r != 0u;
}
// True in one lane of a converged warp.  A branch on this, unlike one on the lane's number, tells the compiler that one thread is behind
// it: the TMA loop took 420 cycles a chunk with `lane == 0`, and set the pace of everything.
__device__ __forceinline__ bool lin_elect()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0u;
}
// A flag in global memory; what this thread's block has written before, and what is read after, goes with the exchange.
struct LinFlag {
    Handover* at;
    __device__ __forceinline__ Handover operator()(Handover v) const
    {
        Handover was;
        asm volatile("atom.acq_rel.gpu.global.exch.b64 %0, [%1], %2;" : "=l"(was) : "l"(at), "l"(v) : "memory");
        return was;
    }
};
__device__ __forceinline__ void lin_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// How many blocks of 64 of an operand's `most` rows (or columns) begin inside, where `left` are left.
__device__ __forceinline__ int lin_blocks(int left, int most) { return left <= 0 ? 0 : left >= most ? most / 64 : (left + 63) / 64; }

// ------------------------------------------------------------------------------------------ the tiles of a pair
struct LinItem {
    int tile, k0, k1;     // chunks [k0, k1) of its K axis
    bool partial;         // sums to the workspace, not to the epilogue
    int helpers;          // pairs [helpers, own) have left sums of this tile; own: none have
};
struct LinSchedule {
    int pair, pairs, chunks, whole;
    int units, u0, u1;   // of the tiles that are cut: all (fewer than 2^31), and this pair's run
    int at;              // next whole tile; -1: the unfinished tile first
    int u;               // next unit of the tiles that this pair completes

    __device__ __forceinline__ LinSchedule(const LinParams& p, int pair_, int pairs_) : pair(pair_), pairs(pairs_), chunks(p.chunks), whole(p.whole)
    {
        units = (p.tiles - whole) * chunks;
        u0 = start(pair);
        u1 = start(pair + 1);
        at = units != 0 ? -1 : pair;
        u = u0;
    }
    __device__ __forceinline__ int start(int pair_) const { return static_cast<int>(static_cast<long long>(units) * pair_ / pairs); }
    __device__ __forceinline__ bool next(LinItem* it)
    {
        it->helpers = pair;
        if (at < 0) {
            at = pair;
            const int tile = u1 / chunks, first = tile * chunks;
            if (u1 > first && u1 > u0) {
                it->tile = whole + tile;
                it->k0 = (u0 > first ? u0 : first) - first;
                it->k1 = u1 - first;
                it->partial = true;
                return true;
            }
        }
        it->partial = false;
        it->k1 = chunks;
        if (u < u1) {
            const int tile = u / chunks, first = tile * chunks;
            if (first + chunks <= u1) {
                it->tile = whole + tile;
                it->k0 = u - first;
                if (it->k0 != 0) {  // the first pair whose run passes the tile's first unit
                    int q = static_cast<int>(static_cast<long long>(first) * pairs / units);
                    while (start(q + 1) <= first) ++q;
                    it->helpers = q;
                }
                u = first + chunks;
                return true;
            }
            u = u1;
        }
        if (at >= whole) return false;
        it->tile = at;
        it->k0 = 0;
        at += pairs;
        return true;
    }
};

// ------------------------------------------------------------------------------------------ activations
constexpr float kLinTanhScale = 0.7978845608f, kLinTanhCube = 0.044715f;
// ACT: linfusion_act_t.
template <int ACT>
__device__ __forceinline__ float lin_act(float u)
{
    if (ACT == 1) return u < 0.0f ? 0.0f : u;  // a NaN stays one
    if (ACT == 2) return u * sigmoid1(u);
    if (ACT == 4) return u * sigmoid1(2.0f * kLinTanhScale * fmaf(kLinTanhCube * u * u, u, u));
    return u;
}
// |u|, at most 30 (where Phi(-a) is zero); a NaN stays one.
__device__ __forceinline__ f32x2 lin_magnitude(float2 u)
{
    float a, b;
    asm("min.NaN.f32 %0, %1, 0f41F00000;" : "=f"(a) : "f"(fabsf(u.x)));
    asm("min.NaN.f32 %0, %1, 0f41F00000;" : "=f"(b) : "f"(fabsf(u.y)));
    return pack2(a, b);
}
// The normal distribution's tail as a product, Phi(-a) = bell * ratio for 0 <= a <= 30, bell = exp(-a^2 / 2): for a negative u the tail is all
// there is of gelu, so its error has to be one of itself.  The ratio, exp(a^2 / 2) erfc(a / sqrt 2) / 2, falls slowly from 1/2 like 1 / a; it is
// a polynomial of degree seven in 1 / (1 + 0.35 a), least squares of the relative error on 0 .. 14 with weights moved towards the largest
// error (Lawson), off by at most 3.1e-7 of itself.  In fp32 the tail is good to 8e-7 of itself up to a = 3, 3e-6 up to 6 and 9e-6 up to
// 13, where it reaches the end of the format (the exponent's rounding).  One reciprocal and one exponential a value.
__device__ __forceinline__ f32x2 lin_normal_ratio(f32x2 a, f32x2* bell)
{
    const float2 e = unpack2(mul2(mul2(a, a), both(-0.5f * kLog2e)));
    const f32x2 t = rcp2(fma2(a, both(0.35f), both(1.0f)));
    *bell = pack2(ex2_approx(e.x), ex2_approx(e.y));
    f32x2 s = fma2(t, both(0.0489425994f), both(-0.202119902f));
    s = fma2(t, s, both(0.240641817f));
    s = fma2(t, s, both(-0.0170242917f));
    s = fma2(t, s, both(0.155961901f));
    s = fma2(t, s, both(0.133354992f));
    s = fma2(t, s, both(0.140270352f));
    return fma2(t, s, both(-2.73163387e-05f));
}

// Two values held to -128 .. 128; a NaN stays one.
__device__ __forceinline__ f32x2 lin_within(float2 u)
{
    float a, b;
    asm("{\n\t.reg .f32 t;\n\tmax.NaN.f32 t, %1, 0fC3000000;\n\tmin.NaN.f32 %0, t, 0f43000000;\n\t}" : "=f"(a) : "f"(u.x));
    asm("{\n\t.reg .f32 t;\n\tmax.NaN.f32 t, %1, 0fC3000000;\n\tmin.NaN.f32 %0, t, 0f43000000;\n\t}" : "=f"(b) : "f"(u.y));
    return pack2(a, b);
}

// The activation's slope, two values at a time.  Where sigmoids are 0 or 1 in fp32 (from 128 on all of them), a factor that would pass fp32, or an
// infinity (a pre-activation beyond fp16), must not meet the zero beside it.
template <int ACT>
__device__ __forceinline__ f32x2 lin_act_slope(f32x2 v)
{
    const float2 u = unpack2(v);
    if constexpr (ACT == 1) return pack2(u.x > 0.0f ? 1.0f : u.x <= 0.0f ? 0.0f : u.x, u.y > 0.0f ? 1.0f : u.y <= 0.0f ? 0.0f : u.y);
    if constexpr (ACT == 2) {
        const f32x2 s = sigmoid2(v);
        return mul2(s, fma2(lin_within(u), fma2(s, both(-1.0f), both(1.0f)), both(1.0f)));
    }
    if constexpr (ACT == 3) {
        // Phi(u) + u phi(u), which is w(|u|) = Phi(-|u|) - |u| phi(u) for a negative u and 1 - w for a positive one; both terms have the bell as a
        // factor, so w keeps its digits.  Infinities give the limits, a NaN stays one.
        const f32x2 a = lin_magnitude(u);
        f32x2 bell;
        const f32x2 ratio = lin_normal_ratio(a, &bell), w = mul2(bell, fma2(a, both(-0.3989422804f), ratio));
        const auto minus_sign = [](float x) { return __uint_as_float((~__float_as_uint(x) & 0x80000000u) | 0x3f800000u); };
        const f32x2 s = pack2(minus_sign(u.x), minus_sign(u.y));
        return fma2(s, w, fma2(s, both(-0.5f), both(0.5f)));
    }
    if constexpr (ACT == 4) {
        const f32x2 c = lin_within(u), uu = mul2(c, c), s = sigmoid2(mul2(c, fma2(uu, both(2.0f * kLinTanhScale * kLinTanhCube), both(2.0f * kLinTanhScale))));
        const f32x2 w = fma2(uu, both(6.0f * kLinTanhScale * kLinTanhCube), both(2.0f * kLinTanhScale));
        return fma2(mul2(mul2(c, s), fma2(s, both(-1.0f), both(1.0f))), w, s);
    }
    return both(1.0f);
}
// The activation of 32 values in place, two at a time.
template <int ACT>
__device__ __forceinline__ void lin_act_all(f32x2 (&v)[16])
{
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float2 u = unpack2(v[i]);
        if constexpr (ACT == 3) {
            // u Phi(u) = max(u, 0) - |u| Phi(-|u|); a NaN stays one in |u|
            const f32x2 a = lin_magnitude(u);
            f32x2 bell;
            const f32x2 ratio = lin_normal_ratio(a, &bell);
            v[i] = fma2(mul2(a, both(-1.0f)), mul2(bell, ratio), pack2(fmaxf(u.x, 0.0f), fmaxf(u.y, 0.0f)));
        } else {
            v[i] = pack2(lin_act<ACT>(u.x), lin_act<ACT>(u.y));
        }
    }
}

// ------------------------------------------------------------------------------------------ the product
template <int KIND, int CG, int BN>
__global__ void __launch_bounds__(LinCfg<CG, BN>::THREADS, 1)
linear_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_y,
              const __grid_constant__ CUtensorMap map_r, const __grid_constant__ CUtensorMap map_u, const __grid_constant__ LinParams p)
{
    using C = LinCfg<CG, BN>;
    extern __shared__ unsigned char smem_raw[];
    // the same place in both CTAs of a pair: descriptors and commits address both by one offset
    const uint32_t raw = smem_u32(smem_raw), stages = (raw + 1023u) & ~1023u, staging = stages + C::STAGES * C::STAGE;
    const uint32_t bias_at = staging + C::GROUPS * kLinStaging, bars = bias_at + C::BIAS;
    const uint32_t full = bars, empty = full + 8 * C::STAGES, acc_full = empty + 8 * C::STAGES, acc_empty = acc_full + 16, res_full = acc_empty + 16;
    uint32_t* slot = reinterpret_cast<uint32_t*>(smem_raw + (res_full + 32 - raw));

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (warp == C::TMA_WARP && lane == 0) {
        prefetch_tmap(&map_a);
        prefetch_tmap(&map_b);
        prefetch_tmap(&map_y);
    }
    const int rank = CG == 2 ? static_cast<int>(cluster_rank()) : 0;
    const int pair = blockIdx.x / CG, pairs = gridDim.x / CG;
    if (tid == 0) {
        const auto init = [](uint32_t bar, uint32_t n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory"); };
        for (int s = 0; s < C::STAGES; ++s) {
            init(full + 8 * s, 1);
            init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            init(acc_full + 8 * b, 1);
            init(acc_empty + 8 * b, CG * C::EPILOGUE_WARPS);
        }
        for (int b = 0; b < C::GROUPS; ++b) init(res_full + 8 * b, 1);
        mbar_fence_init();
    }
    if (warp == 0) lin_tmem_alloc<CG>(slot, C::TMEM_COLS);
    tc_fence_before_sync();
    if (CG == 2) lin_cluster_sync();
    else __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *slot;
    LinSchedule todo(p, pair, pairs);
    pdl_launch_dependents();
    pdl_wait();
    LinItem it;

    if (warp == C::TMA_WARP) {
        if (lin_elect()) {
            const uint32_t lead = CG == 2 ? lin_map(full, 0) : full;
            int s = 0;
            uint32_t phase = 0;
            long long issued = 0;
            bool ok = true;
            while (ok && todo.next(&it)) {
                const int m0 = (it.tile / p.tiles_n) * (CG * kLinRows) + rank * kLinRows, n0 = (it.tile % p.tiles_n) * BN + rank * (BN / CG);
                // blocks of 64 rows or columns that lie outside are not loaded: nothing of what they would give is kept
                const int a_blocks = p.a_mn ? lin_blocks(p.M - m0, kLinRows) : 0, b_blocks = p.b_mn ? lin_blocks(p.N - n0, BN / CG) : 0;
                uint32_t bytes = 0;  // of the pair
                if (rank == 0)
#pragma unroll
                    for (int c = 0; c < CG; ++c)
                        bytes += (p.a_mn ? lin_blocks(p.M - m0 - c * kLinRows, kLinRows) * 8192 : p.a_rows * 128) +
                                 (p.b_mn ? lin_blocks(p.N - n0 - c * (BN / CG), BN / CG) * 8192 : C::B_BYTES);
                for (int k = it.k0; k < it.k1; ++k) {
                    ok = lin_wait(empty + 8 * s, phase ^ 1u);
                    if (!ok) break;
                    // all bytes of the pair are counted on the first CTA's barrier
                    if (rank == 0) lin_expect(full + 8 * s, bytes);
                    const uint32_t a = stages + s * C::STAGE, b = a + C::A_BYTES, bar = lead + 8 * s;
                    if (!p.a_mn) lin_load<CG>(a, &map_a, k * kLinKc, m0, bar);
                    if (a_blocks > 0) lin_load<CG>(a, &map_a, m0, k * kLinKc, bar);
                    if (a_blocks > 1) lin_load<CG>(a + 8192, &map_a, m0 + 64, k * kLinKc, bar);
                    if (!p.b_mn) lin_load<CG>(b, &map_b, k * kLinKc, n0, bar);
                    if (b_blocks > 0) lin_load<CG>(b, &map_b, n0, k * kLinKc, bar);
                    if (BN / CG > 64 && b_blocks > 1) lin_load<CG>(b + 8192, &map_b, n0 + 64, k * kLinKc, bar);
                    ++issued;
                    if (++s == C::STAGES) {
                        s = 0;
                        phase ^= 1u;
                    }
                }
            }
            // The tensor core arrives on `empty` for the last chunks too, in both CTAs of a pair, and nothing else waits for that: as if every stage
            // were filled once more, so that no arrival comes to the shared memory of a CTA that has left.
            for (int i = 0; ok && i < C::STAGES; ++i) {
                ok = lin_wait(empty + 8 * s, phase ^ 1u);
                if (++s == C::STAGES) {
                    s = 0;
                    phase ^= 1u;
                }
            }
            if (!ok) {
                atomicAdd(&linear_expired_waits, 1u);
                // what is still in flight lands before the pair leaves (the first CTA's barriers count both CTAs' bytes)
                if (rank == 0)
                    for (long long i = issued > C::STAGES ? issued - C::STAGES : 0; i < issued; ++i)
                        if (!lin_wait(full + 8 * static_cast<uint32_t>(i % C::STAGES), static_cast<uint32_t>(i / C::STAGES) & 1u)) break;
            }
        }
    } else if (warp == C::MMA_WARP) {
        if (rank == 0 && lin_elect()) {
            const uint32_t idesc = umma_idesc_f32acc(kind_dtype(KIND), CG * kLinRows, BN, (p.a_mn ? kUmmaAMnMajor : 0u) | (p.b_mn ? kUmmaBMnMajor : 0u));
            const uint64_t a0 = p.a_mn ? umma_desc_mnmajor_sw128(stages, 8192, 1024) : umma_desc_kmajor_sw128(stages);
            const uint64_t b0 = p.b_mn ? umma_desc_mnmajor_sw128(stages + C::A_BYTES, 8192, 1024) : umma_desc_kmajor_sw128(stages + C::A_BYTES);
            const uint64_t a_step = p.a_mn ? 128 : 2, b_step = p.b_mn ? 128 : 2;  // 16 values of K, in 16-byte units
            int s = 0, n = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (; ok && todo.next(&it); ++n) {
                const int buf = n & 1;
                ok = n < 2 || lin_wait(acc_empty + 8 * buf, ((n >> 1) - 1) & 1);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t d = tmem + buf * BN;
                for (int k = it.k0; k < it.k1; ++k) {
                    ok = lin_wait(full + 8 * s, phase);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint64_t a = a0 + static_cast<uint64_t>(s * (C::STAGE >> 4)), b = b0 + static_cast<uint64_t>(s * (C::STAGE >> 4));
                    lin_mma<CG>(d, a, b, idesc, k > it.k0 ? 1u : 0u);
#pragma unroll
                    for (int i = 1; i < kLinKc / 16; ++i) lin_mma<CG>(d, a + i * a_step, b + i * b_step, idesc, 1u);
                    lin_commit<CG>(empty + 8 * s);
                    if (++s == C::STAGES) {
                        s = 0;
                        phase ^= 1u;
                    }
                }
                if (ok) lin_commit<CG>(acc_full + 8 * buf);
            }
            if (!ok) atomicAdd(&linear_expired_waits, 1u);
        }
    } else {
        const int group = warp >> 2, row = (warp & 3) * 32 + lane, in_group = tid & 127;
        const bool chief = in_group == 0;
        const uint32_t buffer = staging + group * kLinStaging, res_bar = res_full + 8 * group;
        const uint32_t acc = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + group * kLinColumns;
        const uint32_t acc_free = CG == 2 ? lin_map(acc_empty, 0) : acc_empty;
        uint32_t res_phase = 0u;
        // Once a wait has expired none is begun any more but that for the residual on its way into the buffer, and every barrier is met,
        // so that all of the CTA's threads come to the end.
        bool good = true;
        for (int n = 0; todo.next(&it); ++n) {
            const int buf = n & 1;
            const int m0 = (it.tile / p.tiles_n) * (CG * kLinRows) + rank * kLinRows, col0 = (it.tile % p.tiles_n) * BN + group * kLinColumns;
            const bool residual = p.has_residual && !it.partial, inside = m0 < p.M && col0 < p.N;
            const uint32_t bias = bias_at + group * kLinColumns * 4;
            // the buffer has to be free; the residual comes into it while the products run
            if (chief) {
                tma_store_wait_read();
                if (residual) {
                    lin_expect(res_bar, kLinStaging);
                    lin_load<1>(buffer, &map_r, col0, m0, res_bar);
                }
            }
            if (in_group < kLinColumns) {
                const int col = col0 + in_group;
                float b = 0.0f;
                if (p.bias != nullptr && col < p.N) {
                    unsigned short w;  // a plain load: what was there when this kernel began may have been written over since
                    asm volatile("ld.global.u16 %0, [%1];" : "=h"(w) : "l"(p.bias + 2ll * col) : "memory");
                    b = pair_lo<KIND>(w);
                }
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(bias + 4 * in_group), "f"(b) : "memory");
            }
            good = good && lin_wait(acc_full + 8 * buf, (n >> 1) & 1);
            if (it.helpers < pair && chief)
                for (int q = it.helpers; q < pair; ++q) {
                    Handover* flag = p.flags + (q * CG + rank) * C::GROUPS + group;
                    if (good) {
                        const unsigned long long t0 = global_timer_ns();
                        Handover there;
                        do {
                            asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(there) : "l"(flag) : "memory");
                            good = there == p.mark;
                        } while (!good && global_timer_ns() - t0 < kMaxBarrierWaitNs);
                    }
                    if (good) *flag = 0ull;  // this group alone looks at it
                    else handover_leave(LinFlag{flag}, p.mark);
                }
            if (residual) {  // waited for in any case: its copy has been issued
                const bool there = lin_wait(res_bar, res_phase);
                good = good && there;
                res_phase ^= 1u;
            }
            __syncwarp();
            good = lin_all(1 + group, 128, good);
            tc_fence_after_sync();

            // 32 columns of u: the accumulator, what other pairs have left of the tile, and the bias
            constexpr long long slot_size = static_cast<long long>(BN / 4) * kLinRows;
            const long long block = static_cast<long long>(group * (kLinColumns / 4)) * kLinRows + row;
            const auto sums = [&](int half, f32x2 (&v)[16]) {
                uint32_t d[32];
                __syncwarp();
                tmem_load_32cols(acc + buf * BN + 32 * half, d);
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = pack2(__uint_as_float(d[2 * j]), __uint_as_float(d[2 * j + 1]));
                for (int q = it.helpers; q < pair; ++q) {
                    const float4* from = p.partials + (q * CG + rank) * slot_size + block + half * 8 * kLinRows;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float4 f;
                        asm volatile("ld.global.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "l"(from + j * kLinRows) : "memory");
                        v[2 * j] = add2(v[2 * j], pack2(f.x, f.y));
                        v[2 * j + 1] = add2(v[2 * j + 1], pack2(f.z, f.w));
                    }
                }
                if (p.bias != nullptr && !it.partial)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float4 f;
                        asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "r"(bias + 128 * half + 16 * j));
                        v[2 * j] = add2(v[2 * j], pack2(f.x, f.y));
                        v[2 * j + 1] = add2(v[2 * j + 1], pack2(f.z, f.w));
                    }
            };
            const auto release = [&] {  // the accumulator has been read
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) lin_arrive(acc_free + 8 * buf);
            };
            // eight values of this row in 16 bits into the staging buffer
            const auto stage = [&](int piece, const f32x2* v) {
                const float2 a = unpack2(v[0]), b = unpack2(v[1]), c = unpack2(v[2]), e = unpack2(v[3]);
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(buffer + row * 128 + ((piece ^ (row & 7)) << 4)), "r"(pack_pair<KIND>(a.x, a.y)),
                             "r"(pack_pair<KIND>(b.x, b.y)), "r"(pack_pair<KIND>(c.x, c.y)), "r"(pack_pair<KIND>(e.x, e.y))
                             : "memory");
            };
            const auto leave = [&](const void* map) {  // the buffer to its place in memory
                fence_proxy_async_smem();
                __syncwarp();
                lin_sync(1 + group, 128);
                if (chief) {
                    if (inside) lin_store(map, buffer, col0, m0);
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
            };

            if (it.partial) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    f32x2 v[16];
                    sums(half, v);
                    float4* to = p.partials + (pair * CG + rank) * slot_size + block + half * 8 * kLinRows;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float2 a = unpack2(v[2 * j]), b = unpack2(v[2 * j + 1]);
                        to[j * kLinRows] = make_float4(a.x, a.y, b.x, b.y);
                    }
                }
                release();
                __threadfence();
                __syncwarp();
                lin_sync(1 + group, 128);
                if (chief) handover_raise(LinFlag{p.flags + (pair * CG + rank) * C::GROUPS + group}, p.mark);
                continue;
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x2 v[16];
                sums(half, v);
                switch (p.act) {
                    case 1: lin_act_all<1>(v); break;
                    case 2: lin_act_all<2>(v); break;
                    case 3: lin_act_all<3>(v); break;
                    case 4: lin_act_all<4>(v); break;
                    default: break;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (residual) {
                        uint4 w;
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(buffer + row * 128 + (((4 * half + j) ^ (row & 7)) << 4)) : "memory");
                        v[4 * j] = add2(v[4 * j], pack2(pair_lo<KIND>(w.x), pair_hi<KIND>(w.x)));
                        v[4 * j + 1] = add2(v[4 * j + 1], pack2(pair_lo<KIND>(w.y), pair_hi<KIND>(w.y)));
                        v[4 * j + 2] = add2(v[4 * j + 2], pack2(pair_lo<KIND>(w.z), pair_hi<KIND>(w.z)));
                        v[4 * j + 3] = add2(v[4 * j + 3], pack2(pair_lo<KIND>(w.w), pair_hi<KIND>(w.w)));
                    }
                    stage(4 * half + j, v + 4 * j);
                }
            }
            if (p.u_mode == kUNone) release();
            leave(&map_y);
            if (p.u_mode == kUNone) continue;
            // u takes the same way, once y has left the buffer
            if (chief) tma_store_wait_read();
            __syncwarp();
            lin_sync(1 + group, 128);
            int scales[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x2 v[16];
                sums(half, v);
                if (p.u_mode == kUFull) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) stage(4 * half + j, v + 4 * j);
                    continue;
                }
                // 32 columns are a group of the 8-bit format; columns behind the last are sums of zeros, without a bias
                uint32_t w[8];
                const bool plain = all_finite(v);
                const float most = largest(v, plain);
                scales[half] = pack8_scale<KIND>(most);
                pack8_codes(v, most, pack8_inverse_step(scales[half]), plain, w);
                if (p.codes_map) {  // rows of 64 bytes in the 64-byte swizzle
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(buffer + row * 64 + (((2 * half + j) ^ ((row >> 1) & 3)) << 4)), "r"(w[4 * j]),
                                     "r"(w[4 * j + 1]), "r"(w[4 * j + 2]), "r"(w[4 * j + 3])
                                     : "memory");
                } else if (m0 + row < p.M) {
                    const int col = col0 + 32 * half;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (col + 8 * j < p.N)
                            *reinterpret_cast<uint2*>(p.codes + static_cast<long long>(m0 + row) * p.N + col + 8 * j) = make_uint2(w[2 * j], w[2 * j + 1]);
                }
            }
            release();
            __syncwarp();
            if (p.u_mode == kUFull || p.codes_map) leave(&map_u);
            else lin_sync(1 + group, 128);  // everybody has read the bias
            if (p.u_mode == kUPacked && m0 + row < p.M) {
                unsigned char* to = p.scales + static_cast<long long>(m0 + row) * p.scale_groups + col0 / 32;
                if (col0 + 32 < p.N && (reinterpret_cast<uintptr_t>(to) & 1) == 0) {
                    *reinterpret_cast<unsigned short*>(to) = static_cast<unsigned short>(scales[0] | (scales[1] << 8));
                } else {
                    if (col0 < p.N) to[0] = static_cast<unsigned char>(scales[0]);
                    if (col0 + 32 < p.N) to[1] = static_cast<unsigned char>(scales[1]);
                }
            }
        }
        if (!good && lane == 0) atomicAdd(&linear_expired_waits, 1u);
        if (chief) tma_store_wait_read();  // what has been read gets to memory by itself
    }
    // nobody leaves while the other CTA may still arrive on its barriers or read its shared memory
    __syncwarp();
    tc_fence_before_sync();
    if (CG == 2) lin_cluster_sync();
    else __syncthreads();
    tc_fence_after_sync();
    if (warp == 0) lin_tmem_dealloc<CG>(tmem, C::TMEM_COLS);
}

// ------------------------------------------------------------------------------------------ before the backward products
// du = dy act'(u), rounded once to the 16 bits that the products take, and its sums over the rows from the unrounded values.
// A block takes 256 columns, a thread eight of them; eight rows at a time, four times unrolled; blocks that all run at once (600 of them in
// two rounds took 118 us where 440 take 99).  Six bytes a value, five where u is a checkpoint, two where there is no activation (the sums
// alone).  32768 x 2560 with gelu and the sums' joining: 94 to 97 us, 119 to 123 from a checkpoint (77 and 64 at the copy rate); its 20 to 27
// instructions a value keep the issue slots (56 %) busier than DRAM (39 %).  From a checkpoint 8 to 36 bytes a thread are spilled.
constexpr int kDuThreads = 256, kDuColumns = 256, kDuUnroll = 4;
struct DuParams {
    const char *dy, *u;
    const unsigned char* scales;  // of u in 8 bits
    char* du;
    float* sums;                  // [block row][width] or null
    long long dy_row, u_row;      // bytes
    int M, N, width, rows_per_block, scale_groups;
};
template <int KIND, int ACT, bool PACKED>
__global__ void __launch_bounds__(kDuThreads, 3) linear_du_kernel(const __grid_constant__ DuParams p)
{
    __shared__ float joined[kDuThreads / 32][kDuColumns];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * kDuColumns + 8 * lane;
    const bool live = col < p.N;
    const long long first = static_cast<long long>(blockIdx.y) * p.rows_per_block;
    const long long end = first + p.rows_per_block < p.M ? first + p.rows_per_block : p.M;
    f32x2 sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = both(0.0f);
    pdl_wait();
    pdl_launch_dependents();
    if (live)
        for (long long r0 = first + warp; r0 < end; r0 += kDuUnroll * (kDuThreads / 32)) {
            uint4 dy[kDuUnroll], u[kDuUnroll];
            int scale[kDuUnroll];
#pragma unroll
            for (int k = 0; k < kDuUnroll; ++k) {
                const long long r = r0 + k * (kDuThreads / 32);
                if (r < end) {
                    dy[k] = load16(p.dy + r * p.dy_row + 2ll * col);
                    if constexpr (ACT != 0 && PACKED) {
                        const uint2 c = *reinterpret_cast<const uint2*>(p.u + r * p.u_row + col);
                        u[k].x = c.x;
                        u[k].y = c.y;
                        scale[k] = p.scales[r * p.scale_groups + col / 32];
                    } else if constexpr (ACT != 0) {
                        u[k] = load16(p.u + r * p.u_row + 2ll * col);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < kDuUnroll; ++k) {
                const long long r = r0 + k * (kDuThreads / 32);
                if (r < end) {
                    f32x2 g[4], v[4];
                    g[0] = pack2(pair_lo<KIND>(dy[k].x), pair_hi<KIND>(dy[k].x));
                    g[1] = pack2(pair_lo<KIND>(dy[k].y), pair_hi<KIND>(dy[k].y));
                    g[2] = pack2(pair_lo<KIND>(dy[k].z), pair_hi<KIND>(dy[k].z));
                    g[3] = pack2(pair_lo<KIND>(dy[k].w), pair_hi<KIND>(dy[k].w));
                    if constexpr (ACT != 0) {
                        if constexpr (PACKED) {
                            unpack8_codes4(u[k].x, pack8_step(scale[k]), v);
                            unpack8_codes4(u[k].y, pack8_step(scale[k]), v + 2);
                        } else {
                            v[0] = pack2(pair_lo<KIND>(u[k].x), pair_hi<KIND>(u[k].x));
                            v[1] = pack2(pair_lo<KIND>(u[k].y), pair_hi<KIND>(u[k].y));
                            v[2] = pack2(pair_lo<KIND>(u[k].z), pair_hi<KIND>(u[k].z));
                            v[3] = pack2(pair_lo<KIND>(u[k].w), pair_hi<KIND>(u[k].w));
                        }
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            g[i] = mul2(g[i], lin_act_slope<ACT>(v[i]));
                            const float2 a = unpack2(g[i]);
                            w[i] = pack_pair<KIND>(a.x, a.y);
                        }
                        // read again by the two products that follow: no streaming store
                        *reinterpret_cast<uint4*>(p.du + 2ll * (r * p.N + col)) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] = add2(sum[i], g[i]);
                }
            }
        }
    if (p.sums == nullptr) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float2*>(&joined[warp][8 * lane + 2 * i]) = unpack2(sum[i]);
    __syncthreads();
    const int c = blockIdx.x * kDuColumns + threadIdx.x;
    if (c < p.width) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kDuThreads / 32; ++w) s += joined[w][threadIdx.x];
        p.sums[static_cast<long long>(blockIdx.y) * p.width + c] = s;
    }
}

}  // namespace lf
