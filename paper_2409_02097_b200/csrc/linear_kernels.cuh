// Matrix products with an epilogue, on TMA + tcgen05 (include/linfusion_layers.h): the forward product x w, and the two of the
// backward pass, du w^T and x^T du.  All three are D[M, N] = A[M, K] B[K, N] with each operand contiguous along K or along its
// other axis, which the matrix instructions take either way: one kernel, no transposed copies.
//
// A tile is 256 x BN and belongs to a pair of CTAs on two SMs (cta_group::2: each holds 128 rows of A and of D and half of B, so a
// value of B is read from shared memory once for two SMs), or 128 x BN and one CTA.  Roles in a CTA: a TMA warp, an MMA warp (one
// thread, in the first CTA of a pair), and two groups of four epilogue warps that share a tile's columns; the accumulator is
// double-buffered in tensor memory, so a tile's epilogue runs under the next tile's products.
//
// Every SM is busy for the same time whatever the number of tiles: as many tiles as make whole rounds of the machine are dealt out whole,
// the K axes of the others are laid end to end and cut into equal runs, one for each pair.  A run that ends inside a tile
// leaves its fp32 sums in the workspace; the pair whose run has the tile's end adds them in the order of K (a fixed order)
// before its epilogue.  A pair does that unfinished tile first and the tiles that it completes last, and waits only for pairs
// before it, which were scheduled no later: waits are short, and bounded.
#pragma once

#include "block_kernels.cuh"
#include "column_sums.cuh"
#include "pack8.cuh"

namespace lf {

static __device__ unsigned int linear_expired_waits;

constexpr int kLinKc = 64;           // K of a stage: 128 bytes of a row
constexpr int kLinRows = 128;        // rows of A and D in a CTA
constexpr int kLinEpilogueWarps = 8;
constexpr int kLinTmaWarp = kLinEpilogueWarps, kLinMmaWarp = kLinTmaWarp + 1;
constexpr int kLinThreads = 32 * (kLinEpilogueWarps + 2);
constexpr int kLinChunk = 64;        // columns of D that are staged at a time: 128 bytes of a row
constexpr int kLinStaging = kLinRows * 128;

enum : int { kUNone = 0, kUFull = 1, kUPacked = 2 };

template <int CG, int BN>
struct LinCfg {
    static constexpr int A_BYTES = kLinRows * 128;
    static constexpr int B_BYTES = BN / CG * 128;
    static constexpr int STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = (224 * 1024 - 4 * kLinStaging) / STAGE > 8 ? 8 : (224 * 1024 - 4 * kLinStaging) / STAGE;
    static constexpr int TMEM_COLS = 2 * BN;
    static constexpr int SMEM = STAGES * STAGE + 4 * kLinStaging + 1024 + 512;
};

struct LinParams {
    int M, N, chunks;            // chunks of K
    int tiles_n, whole;          // tiles side by side; tiles that are dealt out whole
    int tiles;
    int a_mn, b_mn;              // an operand's contiguous axis is M / N, not K
    int act, u_mode, has_residual;
    const char* bias;            // 16-bit [N] or null
    signed char* codes;          // u in 8 bits
    unsigned char* scales;
    int scale_groups;
    float4* partials;            // [CTA][column / 4][row]
    uint32_t* flags;             // [CTA], zero when the kernel starts
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
__device__ __forceinline__ void lin_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// ------------------------------------------------------------------------------------------ the tiles of a pair
struct LinItem {
    int tile, k0, k1;     // chunks [k0, k1) of its K axis
    bool partial;         // sums to the workspace, not to the epilogue
    int helpers;          // pairs [helpers, own) have left sums of this tile; own: none have
};
struct LinSchedule {
    int pair, pairs, chunks, whole, tiles;
    long long units, u0, u1;   // of the tiles that are cut: all, and this pair's run
    int at;                    // next whole tile; -1: the unfinished tile first
    long long u;               // next unit of the tiles that this pair completes

    __device__ __forceinline__ LinSchedule(const LinParams& p, int pair_, int pairs_)
        : pair(pair_), pairs(pairs_), chunks(p.chunks), whole(p.whole), tiles(p.tiles)
    {
        units = static_cast<long long>(tiles - whole) * chunks;
        u0 = units * pair / pairs;
        u1 = units * (pair + 1) / pairs;
        at = -1;
        u = u0;
    }
    __device__ __forceinline__ bool next(LinItem* it)
    {
        if (at < 0) {
            at = pair;
            const long long tile = u1 / chunks, first = tile * chunks;
            if (u1 > first && u1 > u0) {
                it->tile = whole + static_cast<int>(tile);
                it->k0 = static_cast<int>((u0 > first ? u0 : first) - first);
                it->k1 = static_cast<int>(u1 - first);
                it->partial = true;
                it->helpers = pair;
                return true;
            }
        }
        if (at < whole) {
            it->tile = at;
            it->k0 = 0;
            it->k1 = chunks;
            it->partial = false;
            it->helpers = pair;
            at += pairs;
            return true;
        }
        const long long tile = u / chunks, last = (tile + 1) * chunks;
        if (u >= u1 || last > u1) return false;
        it->tile = whole + static_cast<int>(tile);
        it->k0 = static_cast<int>(u - tile * chunks);
        it->k1 = chunks;
        it->partial = false;
        it->helpers = pair;
        if (it->k0 != 0) {
            // the first pair whose run passes the tile's first unit
            const long long first = tile * chunks;
            long long q = first * pairs / units;
            while (units * (q + 1) / pairs <= first) ++q;
            it->helpers = static_cast<int>(q);
        }
        u = last;
        return true;
    }
};

// ------------------------------------------------------------------------------------------ activations
__device__ __forceinline__ float lin_rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLinLog2e = 1.4426950408889634f;
__device__ __forceinline__ float lin_sigmoid(float x) { return lin_rcp(1.0f + ex2_approx(-kLinLog2e * x)); }
// Phi(-|u|), the tail of the normal distribution, and its density without 1 / sqrt(2 pi): formula 7.1.26 of Abramowitz and Stegun, Handbook
// of Mathematical Functions, for erfc(|u| / sqrt 2); off by at most 7.5e-8, below what fp32 keeps of the other branch.
__device__ __forceinline__ float lin_normal_tail(float u, float* bell)
{
    const float a = fabsf(u), t = lin_rcp(fmaf(0.3275911f * 0.70710678f, a, 1.0f));
    *bell = ex2_approx(-0.5f * kLinLog2e * u * u);
    float s = fmaf(1.061405429f, t, -1.453152027f);
    s = fmaf(s, t, 1.421413741f);
    s = fmaf(s, t, -0.284496736f);
    s = fmaf(s, t, 0.254829592f);
    return 0.5f * s * t * *bell;
}
constexpr float kLinTanhScale = 0.7978845608f, kLinTanhCube = 0.044715f;
// ACT: linfusion_act_t.
template <int ACT>
__device__ __forceinline__ float lin_act(float u)
{
    if (ACT == 1) return u < 0.0f ? 0.0f : u;  // a NaN stays one
    if (ACT == 2) return u * lin_sigmoid(u);
    if (ACT == 3) {
        float bell;
        const float tail = lin_normal_tail(u, &bell);
        return u * (u < 0.0f ? tail : 1.0f - tail);
    }
    if (ACT == 4) return u * lin_sigmoid(2.0f * kLinTanhScale * fmaf(kLinTanhCube * u * u, u, u));
    return u;
}
template <int ACT>
__device__ __forceinline__ float lin_act_slope(float u)
{
    if (ACT == 1) return u > 0.0f ? 1.0f : u <= 0.0f ? 0.0f : u;
    if (ACT == 2) {
        const float s = lin_sigmoid(u);
        return s * fmaf(u, 1.0f - s, 1.0f);
    }
    if (ACT == 3) {
        float bell;
        const float tail = lin_normal_tail(u, &bell);
        return fmaf(0.3989422804f * u, bell, u < 0.0f ? tail : 1.0f - tail);
    }
    if (ACT == 4) {
        const float s = lin_sigmoid(2.0f * kLinTanhScale * fmaf(kLinTanhCube * u * u, u, u));
        return fmaf(u * s * (1.0f - s), 2.0f * kLinTanhScale * fmaf(3.0f * kLinTanhCube * u, u, 1.0f), s);
    }
    return 1.0f;
}
template <int ACT>
__device__ __forceinline__ void lin_act_all(float (&v)[32])
{
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = lin_act<ACT>(v[i]);
}

// ------------------------------------------------------------------------------------------ the product
template <int KIND, int CG, int BN>
__global__ void __launch_bounds__(kLinThreads, 1)
linear_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_y,
              const __grid_constant__ CUtensorMap map_r, const __grid_constant__ CUtensorMap map_u, const __grid_constant__ LinParams p)
{
    using C = LinCfg<CG, BN>;
    extern __shared__ unsigned char smem_raw[];
    // the same place in both CTAs of a pair: descriptors and commits address both by one offset
    const uint32_t raw = smem_u32(smem_raw), stages = (raw + 1023u) & ~1023u, staging = stages + C::STAGES * C::STAGE;
    const uint32_t bars = staging + 4 * kLinStaging;
    const uint32_t full = bars, empty = full + 8 * C::STAGES, acc_full = empty + 8 * C::STAGES, acc_empty = acc_full + 16, res_full = acc_empty + 16;
    uint32_t* slot = reinterpret_cast<uint32_t*>(smem_raw + (res_full + 32 - raw));

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
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
            init(acc_empty + 8 * b, CG * kLinEpilogueWarps);
        }
        for (int b = 0; b < 4; ++b) init(res_full + 8 * b, 1);
        mbar_fence_init();
    }
    if (warp == 0) lin_tmem_alloc<CG>(slot, C::TMEM_COLS);
    tc_fence_before_sync();
    if (CG == 2) lin_cluster_sync();
    else __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *slot;
    LinSchedule todo(p, pair, pairs);
    LinItem it;

    if (warp == kLinTmaWarp) {
        if (lane == 0) {
            prefetch_tmap(&map_a);
            prefetch_tmap(&map_b);
            const uint32_t lead = CG == 2 ? lin_map(full, 0) : full;
            int s = 0;
            uint32_t phase = 0;
            long long issued = 0;
            bool ok = true;
            while (ok && todo.next(&it)) {
                const int m0 = (it.tile / p.tiles_n) * (CG * kLinRows) + rank * kLinRows, n0 = (it.tile % p.tiles_n) * BN + rank * (BN / CG);
                for (int k = it.k0; k < it.k1; ++k) {
                    ok = lin_wait(empty + 8 * s, phase ^ 1u);
                    if (!ok) break;
                    // all bytes of the pair are counted on the first CTA's barrier
                    if (rank == 0) lin_expect(full + 8 * s, CG * C::STAGE);
                    const uint32_t a = stages + s * C::STAGE, b = a + C::A_BYTES, bar = lead + 8 * s;
                    if (p.a_mn) {
#pragma unroll
                        for (int i = 0; i < kLinRows / 64; ++i) lin_load<CG>(a + i * 8192, &map_a, m0 + 64 * i, k * kLinKc, bar);
                    } else {
                        lin_load<CG>(a, &map_a, k * kLinKc, m0, bar);
                    }
                    if (p.b_mn) {
#pragma unroll
                        for (int i = 0; i < BN / CG / 64; ++i) lin_load<CG>(b + i * 8192, &map_b, n0 + 64 * i, k * kLinKc, bar);
                    } else {
                        lin_load<CG>(b, &map_b, k * kLinKc, n0, bar);
                    }
                    ++issued;
                    if (++s == C::STAGES) {
                        s = 0;
                        phase ^= 1u;
                    }
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
    } else if (warp == kLinMmaWarp) {
        if (lane == 0 && rank == 0) {
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
                    const uint64_t at = static_cast<uint64_t>(s * (C::STAGE >> 4));
#pragma unroll
                    for (int i = 0; i < kLinKc / 16; ++i)
                        lin_mma<CG>(d, a0 + at + i * a_step, b0 + at + i * b_step, idesc, k > it.k0 || i > 0 ? 1u : 0u);
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
        const int group = warp >> 2, row = (warp & 3) * 32 + lane;
        const bool chief = (tid & 127) == 0;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t stage0 = staging + group * 2 * kLinStaging, res0 = res_full + 16 * group;
        const uint32_t acc_free = CG == 2 ? lin_map(acc_empty, 0) : acc_empty;
        constexpr int kChunks = BN / kLinChunk;   // of a tile, taken in turn by the groups
        const bool one_buffer = p.u_mode == kUFull;  // the other is for u
        uint32_t res_phase[2] = {0u, 0u};
        int turn = 0;     // the buffer of the next chunk
        // Once a wait has expired none is begun any more, but every barrier is met, so that all of the CTA's threads come to the end.
        bool good = true;
        for (int n = 0; todo.next(&it); ++n) {
            const int buf = n & 1;
            const int m0 = (it.tile / p.tiles_n) * (CG * kLinRows) + rank * kLinRows, n0 = (it.tile % p.tiles_n) * BN;
            const bool residual = p.has_residual && !it.partial;
            // the residual comes into the buffers that y will leave from, while the products run
            if (residual && chief) {
                tma_store_wait_read();
                for (int i = 0; i < (one_buffer ? 1 : 2); ++i) {
                    const int c = group + 2 * i, b = one_buffer ? 0 : turn ^ i;
                    if (c < kChunks) {
                        lin_expect(res0 + 8 * b, kLinStaging);
                        lin_load<1>(stage0 + b * kLinStaging, &map_r, n0 + c * kLinChunk, m0, res0 + 8 * b);
                    }
                }
            }
            good = good && lin_wait(acc_full + 8 * buf, (n >> 1) & 1);
            if (good && it.helpers < pair && tid == 0)
                for (int q = it.helpers; q < pair && good; ++q) {
                    const uint32_t* flag = p.flags + q * CG + rank;
                    const unsigned long long t0 = global_timer_ns();
                    uint32_t there;
                    do {
                        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(there) : "l"(flag) : "memory");
                        good = there != 0u;
                    } while (!good && global_timer_ns() - t0 < kMaxBarrierWaitNs);
                }
            __syncwarp();
            good = lin_all(1, 32 * kLinEpilogueWarps, good);
            tc_fence_after_sync();
            for (int c = group; c < kChunks; c += 2, turn ^= 1) {
                const int b = one_buffer ? 0 : turn;
                const int col0 = n0 + c * kLinChunk;
                const uint32_t mine = stage0 + b * kLinStaging + row * 128;
                if (!it.partial) {
                    // the buffer is free, or holds the residual
                    if (residual) {
                        if (one_buffer && c != group && chief) {
                            tma_store_wait_read();
                            lin_expect(res0, kLinStaging);
                            lin_load<1>(stage0, &map_r, col0, m0, res0);
                        }
                        good = good && lin_wait(res0 + 8 * b, res_phase[b]);
                        res_phase[b] ^= 1u;
                    } else if (chief) {
                        if (one_buffer) tma_store_wait_read();
                        else asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                    }
                    __syncwarp();
                    lin_sync(2 + group, 128);
                }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t d[32];
                    float v[32];
                    __syncwarp();
                    tmem_load_32cols(tmem + lanes + buf * BN + c * kLinChunk + 32 * half, d);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(d[j]);
                    const long long block = static_cast<long long>((c * 2 + half) * 8) * kLinRows + row;
                    constexpr long long slot_size = static_cast<long long>(BN / 4) * kLinRows;
                    for (int q = it.helpers; q < pair; ++q) {
                        const float4* from = p.partials + (q * CG + rank) * slot_size + block;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            float4 f;
                            asm volatile("ld.global.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "l"(from + j * kLinRows) : "memory");
                            v[4 * j] += f.x;
                            v[4 * j + 1] += f.y;
                            v[4 * j + 2] += f.z;
                            v[4 * j + 3] += f.w;
                        }
                    }
                    if (it.partial) {
                        float4* to = p.partials + (pair * CG + rank) * slot_size + block;
#pragma unroll
                        for (int j = 0; j < 8; ++j) to[j * kLinRows] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                        continue;
                    }
                    const int col = col0 + 32 * half;
                    if (p.bias != nullptr)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (col + 8 * j < p.N) {
                                const uint4 w = __ldg(reinterpret_cast<const uint4*>(p.bias + 2ll * (col + 8 * j)));
                                v[8 * j] += pair_lo<KIND>(w.x); v[8 * j + 1] += pair_hi<KIND>(w.x);
                                v[8 * j + 2] += pair_lo<KIND>(w.y); v[8 * j + 3] += pair_hi<KIND>(w.y);
                                v[8 * j + 4] += pair_lo<KIND>(w.z); v[8 * j + 5] += pair_hi<KIND>(w.z);
                                v[8 * j + 6] += pair_lo<KIND>(w.w); v[8 * j + 7] += pair_hi<KIND>(w.w);
                            }
                    if (p.u_mode == kUFull) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(mine + kLinStaging + (((4 * half + j) ^ (row & 7)) << 4)),
                                         "r"(pack_pair<KIND>(v[8 * j], v[8 * j + 1])), "r"(pack_pair<KIND>(v[8 * j + 2], v[8 * j + 3])),
                                         "r"(pack_pair<KIND>(v[8 * j + 4], v[8 * j + 5])), "r"(pack_pair<KIND>(v[8 * j + 6], v[8 * j + 7]))
                                         : "memory");
                    } else if (p.u_mode == kUPacked && m0 + row < p.M && col < p.N) {
                        // 32 columns are a group of the 8-bit format; columns behind the last are zero but for no bias: sums of zeros
                        float most = 0.0f;
#pragma unroll
                        for (int j = 0; j < 32; ++j) most = fmaxf(most, finite_abs(v[j]));
                        const int scale = pack8_scale<KIND>(most);
                        const float inverse = pack8_inverse_step(scale);
                        const long long at = static_cast<long long>(m0 + row) * p.N + col;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (col + 8 * j < p.N)
                                *reinterpret_cast<uint2*>(p.codes + at + 8 * j) = make_uint2(pack8_codes4(v + 8 * j, inverse), pack8_codes4(v + 8 * j + 4, inverse));
                        p.scales[static_cast<long long>(m0 + row) * p.scale_groups + col / 32] = static_cast<unsigned char>(scale);
                    }
                    switch (p.act) {
                        case 1: lin_act_all<1>(v); break;
                        case 2: lin_act_all<2>(v); break;
                        case 3: lin_act_all<3>(v); break;
                        case 4: lin_act_all<4>(v); break;
                        default: break;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t at = mine + (((4 * half + j) ^ (row & 7)) << 4);
                        if (residual) {
                            uint4 w;
                            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(at) : "memory");
                            v[8 * j] += pair_lo<KIND>(w.x); v[8 * j + 1] += pair_hi<KIND>(w.x);
                            v[8 * j + 2] += pair_lo<KIND>(w.y); v[8 * j + 3] += pair_hi<KIND>(w.y);
                            v[8 * j + 4] += pair_lo<KIND>(w.z); v[8 * j + 5] += pair_hi<KIND>(w.z);
                            v[8 * j + 6] += pair_lo<KIND>(w.w); v[8 * j + 7] += pair_hi<KIND>(w.w);
                        }
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(pack_pair<KIND>(v[8 * j], v[8 * j + 1])),
                                     "r"(pack_pair<KIND>(v[8 * j + 2], v[8 * j + 3])), "r"(pack_pair<KIND>(v[8 * j + 4], v[8 * j + 5])),
                                     "r"(pack_pair<KIND>(v[8 * j + 6], v[8 * j + 7]))
                                     : "memory");
                    }
                }
                if (it.partial) continue;
                fence_proxy_async_smem();
                __syncwarp();
                lin_sync(2 + group, 128);
                if (chief) {
                    if (m0 < p.M && col0 < p.N) {
                        lin_store(&map_y, stage0 + b * kLinStaging, col0, m0);
                        if (p.u_mode == kUFull) lin_store(&map_u, stage0 + kLinStaging, col0, m0);
                    }
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
            }
            // the accumulator has been read
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) lin_arrive(acc_free + 8 * buf);
            if (it.partial) {
                __threadfence();
                __syncwarp();
                lin_sync(1, 32 * kLinEpilogueWarps);
                if (tid == 0) asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(p.flags + pair * CG + rank), "r"(1u) : "memory");
            }
        }
        if (!good && lane == 0) atomicAdd(&linear_expired_waits, 1u);
        if (chief) tma_store_wait_all();
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
// A block takes 256 columns, a thread eight of them; eight rows at a time, four times unrolled.  Bound by DRAM: six bytes a value, five
// where u is a checkpoint, two where there is no activation (the sums alone).
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
__global__ void __launch_bounds__(kDuThreads) linear_du_kernel(const __grid_constant__ DuParams p)
{
    __shared__ float joined[kDuThreads / 32][kDuColumns];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * kDuColumns + 8 * lane;
    const bool live = col < p.N;
    const long long first = static_cast<long long>(blockIdx.y) * p.rows_per_block;
    const long long end = first + p.rows_per_block < p.M ? first + p.rows_per_block : p.M;
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
    if (live)
        for (long long r0 = first + warp; r0 < end; r0 += kDuUnroll * (kDuThreads / 32)) {
            uint4 dy[kDuUnroll], u[kDuUnroll];
            int scale[kDuUnroll];
#pragma unroll
            for (int k = 0; k < kDuUnroll; ++k) {
                const long long r = r0 + k * (kDuThreads / 32);
                if (r < end) {
                    dy[k] = load16(p.dy + r * p.dy_row + 2ll * col);
                    if (ACT != 0 && PACKED) {
                        const uint2 c = *reinterpret_cast<const uint2*>(p.u + r * p.u_row + col);
                        u[k].x = c.x;
                        u[k].y = c.y;
                        scale[k] = p.scales[r * p.scale_groups + col / 32];
                    } else if (ACT != 0) {
                        u[k] = load16(p.u + r * p.u_row + 2ll * col);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < kDuUnroll; ++k) {
                const long long r = r0 + k * (kDuThreads / 32);
                if (r < end) {
                    F8 g = unpack8<KIND>(dy[k]);
                    if (ACT != 0) {
                        F8 v;
                        if (PACKED) {
                            unpack8_codes4(u[k].x, pack8_step(scale[k]), v.v);
                            unpack8_codes4(u[k].y, pack8_step(scale[k]), v.v + 4);
                        } else {
                            v = unpack8<KIND>(u[k]);
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) g.v[i] *= lin_act_slope<ACT>(v.v[i]);
                        // read again by the two products that follow: no streaming store
                        *reinterpret_cast<uint4*>(p.du + 2ll * (r * p.N + col)) = pack8<KIND>(g);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i] += g.v[i];
                }
            }
        }
    if (p.sums == nullptr) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) joined[warp][8 * lane + i] = sum[i];
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
