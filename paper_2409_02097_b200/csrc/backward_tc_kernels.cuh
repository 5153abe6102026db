// Backward pass of the normalized linear attention on TMA + tcgen05, for widths up to 64 (the formulas and the head /
// tail operands are those of backward_kernels.cuh).  Channels past d (d = 32, 40) lie outside the tensor maps: loads
// fill them with zeros, stores do not write them.
//
//   backward_tc_state_kernel  Q, dY -> dQ and partial dS | dz  (GRAD), or K, V -> partial S | z
//   backward_tc_reduce_kernel sums a slab's partials in CTA order
//   backward_tc_kv_kernel     K, V -> dK, dV
//
// Work is cut into 128-token tiles numbered slab-major; CTA g of G (one per SM) owns tiles [g W/G, (g+1) W/G), so
// every CTA streams the same amount and at most a few slabs' operands and accumulators change hands inside a run.  The split is
// a function of the shape and the SM count alone: fixed summation order, no atomics.
//
// A tile is one MMA tile: thread r of a warpgroup owns token r.  It reads its row from the swizzled stage, applies phi, and
// needs nothing from other threads but the products' rows in tensor memory (its own lane): no shuffles for den, f . t or c.
// Two warpgroups take turns at the tiles, a warp loads by TMA into a ring of five tiles (32 KB each), a warp issues the
// MMAs, a warp sends gradients out:
//
//   state:  T[128 x 64]  = dY R^T             (hi, then lo: 8 steps of K = 16, dY straight from the stage)
//           D[128 x 64] += [F_hi | F_lo]^T dY (F = w phi(q); head and tail are the two halves of M = 128: 8 steps)
//   kv:     T[128 x 64]  = V dS^T  (8 steps)   and   T'[128 x 64] = F dS = F_hi dS_hi + F_hi dS_lo + F_lo dS_hi (12)
//
// Gradients are written over Q (K, V) in the stage and leave by TMA.  D is added to the fp32 partial
// in global memory every 32 tiles (the tensor core truncates its running sums: chains stay short, and two accumulators
// take turns).  Each thread keeps the dz of its tokens in 64 columns of its own tensor-memory lane for a slab's run (in
// registers, beside phi of the row, it made the kernel spill), and the lanes are summed at the end.
//
// Per tile an SM moves 48 KB (state) or 64 KB (kv) of DRAM traffic, about 2100 or 2800 clocks at the measured copy rate; the
// MMAs take about 800 or 1000 clocks, the threads' arithmetic about 900 issue slots of each scheduler.
#pragma once

#include <type_traits>

#include "backward_kernels.cuh"
#include "common.cuh"
#include "packed_math.cuh"

namespace lf {

constexpr int kTcTile = 128, kTcTileBytes = kTcTile * 128;  // one tensor's tile: 16 KB
struct BackwardTc {
    // Two warpgroups, a thread has a token's whole row.  (Four in the state kernel, two threads a row: 562 us where this takes
    // 517, at 40 slabs x 131072: the threads' chains are shorter, but half of each crosses a shuffle or shared memory.)
    static constexpr int KV_WARPS = 8, KV_THREADS = 32 * (KV_WARPS + 3);
    static constexpr int STATE_WARPS = 8, STATE_THREADS = 32 * (STATE_WARPS + 3);
    static constexpr int STAGE_BYTES = 2 * kTcTileBytes;
    static constexpr int F_BYTES = 2 * kTcTileBytes;         // head, tail
    static constexpr int STATE_F = 1, STATE_STAGES = 5, KV_F = 1, KV_STAGES = 5;
    static constexpr int S_BYTES = 2 * 64 * 128;             // 64 rows of 64 channels: head, tail
    static constexpr int T_BUFFERS = 4, SEGMENT_TILES = 32;
    static constexpr int TMEM_COLS = 512;                    // T: 4 x 64, D: 2 x 64, dz: 2 x 64 (kv: 4 x 128)
    static constexpr int LEAD = 2;                           // tiles by which the first product runs ahead of the second
    static constexpr int STATE_SMEM = STATE_STAGES * STAGE_BYTES + STATE_F * F_BYTES + S_BYTES + 1024 /*align*/ + 2048 /*z, scales, mu, barriers*/;
    static constexpr int KV_SMEM = KV_STAGES * STAGE_BYTES + KV_F * F_BYTES + S_BYTES + 1024 /*align*/ + 1024 /*z, barriers*/;
    static constexpr int PARTIAL_FLOATS = 128 * 64 + 8 * 64; // D (head rows, tail rows), then dz of each consumer warp
};
static_assert(BackwardTc::STATE_SMEM <= 227 * 1024 && BackwardTc::KV_SMEM <= 227 * 1024, "shared memory");

__host__ __device__ __forceinline__ long long tc_first_tile(long long g, long long W, long long G) { return g * W / G; }

// How often kernels of the backward pass gave up on a wait on this device since the library was loaded: what is left of it when
// a call's workspace, with the status word in it, has gone.
static __device__ unsigned int backward_expired_waits;
__device__ __forceinline__ void tc_expired(uint32_t* status)
{
    atomicExch(status, kStatusWaitExpired);
    atomicAdd(&backward_expired_waits, 1u);
}
__device__ __forceinline__ uint64_t policy_evict_normal()
{
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
    return p;
}
template <int WARPS>
__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void sts16(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w)
{
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void sts8(uint32_t a, uint32_t x, uint32_t y)
{
    asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(a), "r"(x), "r"(y) : "memory");
}
// Byte offset of 16-byte piece j of row r in a tile of 128-byte rows with the 128-byte swizzle.
__device__ __forceinline__ uint32_t swizzled(int r, int j) { return r * 128 + ((j ^ (r & 7)) << 4); }

// 16 columns of two places of the lane's row of tensor memory, one wait; and 16 columns back (tmem_store_wait before they
// are read again).
__device__ __forceinline__ void tmem_load_2x16cols(uint32_t a, uint32_t (&x)[16], uint32_t b, uint32_t (&y)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%32];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%33];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]),
          "=r"(x[10]), "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15]), "=r"(y[0]), "=r"(y[1]), "=r"(y[2]),
          "=r"(y[3]), "=r"(y[4]), "=r"(y[5]), "=r"(y[6]), "=r"(y[7]), "=r"(y[8]), "=r"(y[9]), "=r"(y[10]), "=r"(y[11]),
          "=r"(y[12]), "=r"(y[13]), "=r"(y[14]), "=r"(y[15])
        : "r"(a), "r"(b)
        : "memory");
}
__device__ __forceinline__ void tmem_store_16cols(uint32_t a, const uint32_t (&x)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(a),
        "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]),
        "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15])
        : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// phi of 8 PIECES packed values of a row, from 16-byte piece `first` on.
template <int KIND, int PIECES>
__device__ __forceinline__ void phi_row(uint32_t tile, int r, int first, float (&f)[8 * PIECES])
{
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const uint4 x = lds16(tile + swizzled(r, first + j));
        const uint32_t p[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[8 * j + 2 * i] = phi_or_nan<KIND>(pair_lo<KIND>(p[i]));
            f[8 * j + 2 * i + 1] = phi_or_nan<KIND>(pair_hi<KIND>(p[i]));
        }
    }
}
// phi' from phi: above zero phi > 1 and the slope is 1, below the slope is phi itself.
template <int KIND>
__device__ __forceinline__ float slope_of(float f) { return kind_phi(KIND) == kPhiIdentity ? 1.0f : min_nan(f, 1.0f); }

// mu . g of a token's row in ATOMS tiles of dY.  A call: in the loop over tiles, which hardly ever takes it, its registers made the
// compiler spill the row of phi (1046 against 999 us at 40 slabs x 131072 x 64).
template <int KIND, int ATOMS>
__device__ __noinline__ float row_mean_dot(uint32_t tile, int r, const float* mu)
{
    float sum = 0.0f;
#pragma unroll 1
    for (int j = 0; j < 8 * ATOMS; ++j) sum = mean_dot<KIND>(lds16(tile + (j / 8) * kTcTileBytes + swizzled(r, j & 7)), mu + 8 * j, sum);
    return sum;
}

// Largest of three values over the consumers; `scratch`: three floats of shared memory for each warp.
template <int WARPS>
__device__ __forceinline__ float3 consumer_max(float3 v, float* scratch, int warp, int lane)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.x = fmaxf(v.x, __shfl_xor_sync(0xffffffffu, v.x, o));
        v.y = fmaxf(v.y, __shfl_xor_sync(0xffffffffu, v.y, o));
        v.z = fmaxf(v.z, __shfl_xor_sync(0xffffffffu, v.z, o));
    }
    if (lane == 0) scratch[3 * warp] = v.x, scratch[3 * warp + 1] = v.y, scratch[3 * warp + 2] = v.z;
    consumer_sync<WARPS>();
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
        v.x = fmaxf(v.x, scratch[3 * i]);
        v.y = fmaxf(v.y, scratch[3 * i + 1]);
        v.z = fmaxf(v.z, scratch[3 * i + 2]);
    }
    return v;
}

// The consumers lay S (dS) of a slab out as KROWS K-major rows (features) of VW channels in atoms of 64, head, then tail, and z (dz) as
// KROWS floats; zeros where the widths end.  CENTRED: R = S - z mu^T in place of S where eps is not negative, with mu as VW floats; its
// sums pass through the operand's place.  Returns with the scales of fp16 operands: of S (R), and, CENTRED, of each feature's
// w f in scale_w.  A thread has four columns of every ROWS-th row, in registers from one read of S to the operand.
template <int KIND, int WARPS, int KROWS, int VW, bool CENTRED>
__device__ __forceinline__ void tc_load_state(const float* S, int dk, int dv, unsigned char* operand, float* z, float* mu, float* scale_w,
                                              float* scratch, int tid, float eps, float* scale_s)
{
    constexpr int PER_ROW = VW / 4, ROWS = 32 * WARPS / PER_ROW, STEPS = KROWS / ROWS, HALF = VW / 64 * KROWS * 128;
    static_assert(KROWS <= 32 * WARPS && ROWS * (VW + 1) * 4 <= 2 * HALF, "one thread for each feature; the sums of mu take the operand's place");
    const int warp = tid / 32, lane = tid & 31, slice = tid / PER_ROW, col = 4 * (tid % PER_ROW);
    float x[STEPS][4];
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
        const int row = n * ROWS + slice;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (row < dk && col < dv) v = *reinterpret_cast<const float4*>(S + row * dv + col);
        x[n][0] = v.x, x[n][1] = v.y, x[n][2] = v.z, x[n][3] = v.w;
    }
    const float zv = tid < dk ? S[dk * dv + tid] : 0.0f;
    if (tid < KROWS) z[tid] = zv;
    if (CENTRED && eps >= 0.0f) {
        float* sums = reinterpret_cast<float*>(operand);  // [ROWS][VW], then [ROWS] of z . z
        consumer_sync<WARPS>();
        float s[4] = {}, zz = 0.0f;
#pragma unroll
        for (int n = 0; n < STEPS; ++n) {
            const float zr = z[n * ROWS + slice];
            zz = fmaf(zr, zr, zz);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = fmaf(zr, x[n][i], s[i]);
        }
        *reinterpret_cast<float4*>(sums + slice * VW + col) = make_float4(s[0], s[1], s[2], s[3]);
        if (col == 0) sums[ROWS * VW + slice] = zz;
        consumer_sync<WARPS>();
        if (tid < VW) {
            float sum = 0.0f, squares = 0.0f;
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                sum += sums[i * VW + tid];
                squares += sums[ROWS * VW + i];
            }
            mu[tid] = mean_of(sum, squares);
        }
        consumer_sync<WARPS>();
#pragma unroll
        for (int n = 0; n < STEPS; ++n) {
            const float zr = -z[n * ROWS + slice];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[n][i] = fmaf(zr, mu[col + i], x[n][i]);
        }
    }
    *scale_s = 1.0f;
    if (kind_dtype(KIND) == kDtypeFp16) {
        float big = 0.0f;
#pragma unroll
        for (int n = 0; n < STEPS; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) big = fmaxf(big, fabsf(x[n][i]));
        const float3 m = consumer_max<WARPS>(make_float3(big, zv, tid >= dk ? 0.0f : zv > 0.0f ? 1.0f / zv : 3.0e38f), scratch, warp, lane);
        *scale_s = pow2_scale(m.x, 12);
        if (CENTRED && tid < KROWS)
            scale_w[tid] = eps < 0.0f ? 1.0f : kind_phi(KIND) == kPhiIdentity ? slab_scale(m.y, m.z, eps) : feature_scale(zv, eps);
    }
    const uint32_t to = smem_u32(operand) + (col / 64) * (KROWS * 128) + (col & 4) * 2;
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
        uint32_t hi[2], lo[2];
        split_pair<KIND>(x[n][0] * *scale_s, x[n][1] * *scale_s, &hi[0], &lo[0]);
        split_pair<KIND>(x[n][2] * *scale_s, x[n][3] * *scale_s, &hi[1], &lo[1]);
        const uint32_t at = to + swizzled(n * ROWS + slice, (col & 63) / 8);
        sts8(at, hi[0], hi[1]);
        sts8(at + HALF, lo[0], lo[1]);
    }
}

// The walk over a CTA's run that every role makes alike: units are the stretches of one slab.
struct TcRun {
    long long u0;
    int n, tiles_per_slab;
    __device__ __forceinline__ int slab(int it) const { return static_cast<int>((u0 + it) / tiles_per_slab); }
    // first tile of the run behind the unit that tile `it` belongs to
    __device__ __forceinline__ int unit_end(int it) const
    {
        const long long e = (static_cast<long long>(slab(it)) + 1) * tiles_per_slab - u0;
        return e < n ? static_cast<int>(e) : n;
    }
};

// The producer: tiles of two tensors into the ring.
template <int STAGES>
__device__ __forceinline__ void tc_produce(const CUtensorMap* a, const CUtensorMap* b, unsigned char* ring, uint64_t* full,
                                           uint64_t* empty, const TcRun& run, int H, uint64_t policy, uint32_t* status)
{
    int issued = 0;
    for (int it = 0; it < run.n; ++it) {
        const int s = it % STAGES;
        if (it >= STAGES && !mbar_wait(&empty[s], ((it / STAGES) & 1) ^ 1)) {
            tc_expired(status);
            break;
        }
        const int slab = run.slab(it), row = static_cast<int>((run.u0 + it) % run.tiles_per_slab) * kTcTile;
        unsigned char* dst = ring + s * BackwardTc::STAGE_BYTES;
        mbar_expect_tx(&full[s], BackwardTc::STAGE_BYTES);
        tma_load_4d(dst, a, 0, row, slab % H, slab / H, &full[s], policy);
        tma_load_4d(dst + kTcTileBytes, b, 0, row, slab % H, slab / H, &full[s], policy);
        ++issued;
    }
    // no copy may land in shared memory after the CTA has gone
    for (int it = issued > STAGES ? issued - STAGES : 0; it < issued; ++it)
        if (!mbar_wait(&full[it % STAGES], (it / STAGES) & 1)) {
            tc_expired(status);
            return;
        }
}

// The storing warp's thread: tiles of gradients leave the ring in order; a stage is handed back as soon as its store has
// been read (the consumers come back to it only a tile later: too late for the loads to keep DRAM busy).
template <int STAGES, int TENSORS>
__device__ __forceinline__ void tc_store(const CUtensorMap* a, const CUtensorMap* b, unsigned char* ring, uint64_t* written, uint64_t* empty,
                                         const TcRun& run, int H, uint32_t* status)
{
    const uint64_t policy = policy_evict_first();
    for (int it = 0; it < run.n; ++it) {
        const int s = it % STAGES;
        if (!mbar_wait(&written[s], (it / STAGES) & 1)) {
            tc_expired(status);
            break;
        }
        const int slab = run.slab(it), row = static_cast<int>((run.u0 + it) % run.tiles_per_slab) * kTcTile;
        unsigned char* src = ring + s * BackwardTc::STAGE_BYTES;
        tma_store_4d(a, src, 0, row, slab % H, slab / H, policy);
        if (TENSORS == 2) tma_store_4d(b, src + kTcTileBytes, 0, row, slab % H, slab / H, policy);
        tma_store_wait_read();
        mbar_arrive(&empty[s]);
    }
    tma_store_wait_all();
}

// Waits on a barrier that nothing completes, as the kernels below wait, and reports it as they do.
static __global__ void backward_wait_selftest_kernel(uint32_t* __restrict__ status)
{
    __shared__ uint64_t bar;
    if (threadIdx.x == 0) {
        mbar_init(&bar, 1);
        mbar_fence_init();
        if (!mbar_wait(&bar, 0)) tc_expired(status);
    }
}

template <int KIND, bool GRAD>
__global__ void __launch_bounds__(BackwardTc::STATE_THREADS, 1)
backward_tc_state_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_g,
                         const __grid_constant__ CUtensorMap tmap_dq, const float* __restrict__ state, float* __restrict__ partials,
                         uint32_t* __restrict__ status, int N, int dk, int dv, int tiles_per_slab, long long W, int spans, int H,
                         BackwardScales sc, int clear_status)
{
    using C = BackwardTc;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char* F = smem + C::STATE_STAGES * C::STAGE_BYTES;
    unsigned char* So = F + C::STATE_F * C::F_BYTES;
    float* z = reinterpret_cast<float*>(So + C::S_BYTES);
    float* scale_w = z + 64;  // [64] fp16: of each feature's w f
    float* mu = scale_w + 64; // [64]
    float* scratch = mu + 64;
    uint64_t* full = reinterpret_cast<uint64_t*>(scratch + 32);
    uint64_t* empty = full + C::STATE_STAGES;
    uint64_t* t_full = empty + C::STATE_STAGES;      // [T_BUFFERS]
    uint64_t* f_full = t_full + C::T_BUFFERS;  // F of a tile is written
    // [2] ... and has been read (commit), odd and even tiles apart: with one barrier the pair that waits for the tile before
    // its own could find the phase it wants two behind, which a parity cannot tell from one not yet reached
    uint64_t* f_free = f_full + 1;
    uint64_t* s_ready = f_free + 2;            // a slab's operand is in place (8 warps)
    uint64_t* d_done = s_ready + 1;            // [2] an accumulator is complete (commit)
    uint64_t* d_free = d_done + 2;             // [2] ... and has been read (8 warps)
    uint64_t* written = d_free + 2;            // [STATE_STAGES] dQ is in place of Q
    uint64_t* drained = written + C::STATE_STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    TcRun run;
    run.u0 = tc_first_tile(blockIdx.x, W, gridDim.x);
    run.n = static_cast<int>(tc_first_tile(blockIdx.x + 1ll, W, gridDim.x) - run.u0);
    run.tiles_per_slab = tiles_per_slab;
    if (tid == 0) {
        for (int s = 0; s < C::STATE_STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], GRAD ? 2 : 1);  // the second product's commit; with dQ, its store
            mbar_init(&written[s], 4);
        }
        for (int b = 0; b < C::T_BUFFERS; ++b) mbar_init(&t_full[b], 1);
        mbar_init(f_full, 4);
        mbar_init(&f_free[0], 1), mbar_init(&f_free[1], 1);
        mbar_init(s_ready, C::STATE_WARPS);
        for (int b = 0; b < 2; ++b) mbar_init(&d_done[b], 1), mbar_init(&d_free[b], C::STATE_WARPS);
        mbar_init(drained, 1);
        mbar_fence_init();
    }
    if (warp == 0) tmem_alloc(tmem_slot, C::TMEM_COLS);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot, tmem_d = tmem + C::T_BUFFERS * 64;
    if (warp == C::STATE_WARPS && lane == 0) {
        prefetch_tmap(&tmap_q);
        prefetch_tmap(&tmap_g);
    }
    pdl_launch_dependents();
    pdl_wait();
    if (clear_status != 0 && blockIdx.x == 0 && tid == 0) *status = kStatusOk;

    if (warp == C::STATE_WARPS) {
        // Q and dY are not read again; K and V are, by the kernel after next.
        if (lane == 0)
            tc_produce<C::STATE_STAGES>(&tmap_q, &tmap_g, smem, full, empty, run, H, GRAD ? policy_evict_first() : policy_evict_normal(), status);
    } else if (warp == C::STATE_WARPS + 2) {
        if (GRAD && lane == 0) tc_store<C::STATE_STAGES, 1>(&tmap_dq, nullptr, smem, written, empty, run, H, status);
    } else if (warp == C::STATE_WARPS + 1) {
        if (lane == 0) {
            const uint32_t idesc_t = umma_idesc_f32acc(kind_dtype(KIND), 128, 64);
            const uint32_t idesc_d = umma_idesc_f32acc(kind_dtype(KIND), 128, 64, kUmmaAMnMajor | kUmmaBMnMajor);
            const uint32_t f_addr = smem_u32(F), s_addr = smem_u32(So);
            bool ok = true;
            int j = 0, seg = 0, in_seg = 0, unit = 0;  // j: next tile of the second product
            auto second = [&]() {  // D += [F_hi | F_lo]^T dY of tile j
                if (in_seg == 0 && seg >= 2) ok = ok && mbar_wait(&d_free[seg & 1], ((seg >> 1) & 1) ^ 1);
                ok = ok && mbar_wait(f_full, j & 1);
                if (ok) {
                    tc_fence_after_sync();
                    const uint32_t g_addr = smem_u32(smem + (j % C::STATE_STAGES) * C::STAGE_BYTES + kTcTileBytes);
#pragma unroll
                    for (int k = 0; k < kTcTile / 16; ++k)
                        umma_ss(tmem_d + (seg & 1) * 64, umma_desc_mnmajor_sw128(f_addr + k * 2048, kTcTileBytes, 1024),
                                umma_desc_mnmajor_sw128(g_addr + k * 2048, 0, 1024), idesc_d, in_seg == 0 && k == 0 ? 0u : 1u);
                    umma_commit(&f_free[j & 1]);
                    umma_commit(&empty[j % C::STATE_STAGES]);
                }
                ++in_seg;
                if (in_seg == C::SEGMENT_TILES || j + 1 == run.unit_end(j)) {
                    if (ok) umma_commit(&d_done[seg & 1]);
                    ++seg;
                    in_seg = 0;
                }
                ++j;
            };
            for (int it = 0; it < run.n && ok; ++it) {
                if (GRAD) {
                    if (it == 0 || run.slab(it) != run.slab(it - 1)) {
                        // the operand changes once the consumers are through with the slab before
                        while (j < it && ok) second();
                        ok = ok && mbar_wait(s_ready, unit & 1);
                        ++unit;
                    }
                    ok = ok && mbar_wait(&full[it % C::STATE_STAGES], (it / C::STATE_STAGES) & 1);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint32_t g_addr = smem_u32(smem + (it % C::STATE_STAGES) * C::STAGE_BYTES + kTcTileBytes);
                    const uint32_t t_at = tmem + (it % C::T_BUFFERS) * 64;
                    // the buffer's last tile is it - 4, whose F the loop below has waited for: its T has been read
#pragma unroll
                    for (int h = 1; h >= 0; --h)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            umma_ss(t_at, umma_desc_kmajor_sw128(g_addr) + 2 * k, umma_desc_kmajor_sw128(s_addr + h * 64 * 128) + 2 * k,
                                    idesc_t, h == 1 && k == 0 ? 0u : 1u);
                    umma_commit(&t_full[it % C::T_BUFFERS]);
                    if (it - j >= C::LEAD) second();
                } else {
                    second();
                }
            }
            while (j < run.n && ok) second();
            if (!ok) tc_expired(status);
            umma_commit(drained);  // tensor memory may be freed only behind the last MMA
            if (!mbar_wait(drained, 0)) tc_expired(status);
        }
    } else {
        // ---------------- consumers ----------------
        const int group = warp / 4, r = tid & 127;
        const uint32_t t_lane = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t f_at = smem_u32(F), dz_at = tmem_d + 128 + group * 64 + t_lane;
        bool ok = true;  // alike in a warp; a warp that gave up still goes through every barrier of the consumers
        auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, parity)); };
        int seg0 = 0, span = 0;  // segments before this unit
        for (int a = 0; a < run.n;) {
            const int slab = run.slab(a), b = run.unit_end(a);
            float scale_s = 1.0f;
            float* partial = partials + (static_cast<size_t>(blockIdx.x) * spans + span) * C::PARTIAL_FLOATS;
            if (GRAD) {
                const float* S = state + static_cast<size_t>(slab) * grad_state_floats(dk, dv);
                consumer_sync<C::STATE_WARPS>();  // everybody is through with the slab before
                tc_load_state<KIND, C::STATE_WARPS, 64, 64, true>(S, dk, dv, So, z, mu, scale_w, scratch, tid, sc.eps, &scale_s);
                fence_proxy_async_smem();
                consumer_sync<C::STATE_WARPS>();  // z is there
                if (lane == 0) mbar_arrive(s_ready);
            }
            constexpr bool SCALED = GRAD && kind_dtype(KIND) == kDtypeFp16;
            const float unscale_t = 1.0f / scale_s, unscale_w = SCALED ? 1.0f / scale_w[r & 63] : 1.0f;
            if (ok) {
                uint32_t nothing[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) nothing[i] = 0u;
#pragma unroll
                for (int h = 0; h < 4; ++h) tmem_store_16cols(dz_at + 16 * h, nothing);
                tmem_store_wait();
            }
            int flushed = 0;  // segments of this unit that have gone to the partial
            const int segs = (b - a + C::SEGMENT_TILES - 1) / C::SEGMENT_TILES;
            // this warp's 32 lanes x its group's 32 columns; behind the unit's last tile also dS mu, whose code in the loop over
            // tiles made the compiler spill
            auto flush_until = [&](int want, auto behind) {
                constexpr bool WITH_MU = GRAD && decltype(behind)::value;
                for (; flushed < want; ++flushed) {
                    const int sg = seg0 + flushed;
                    wait(&d_done[sg & 1], (sg >> 1) & 1);
                    if (ok) {
                        tc_fence_after_sync();
                        float* to = partial + r * 64 + group * 32;
                        float with_mu = 0.0f;  // the row's columns times mu
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t d[16];
                            tmem_load_16cols(tmem_d + (sg & 1) * 64 + group * 32 + h * 16 + t_lane, d);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float4 v = make_float4(__uint_as_float(d[4 * i]) * unscale_w, __uint_as_float(d[4 * i + 1]) * unscale_w,
                                                       __uint_as_float(d[4 * i + 2]) * unscale_w, __uint_as_float(d[4 * i + 3]) * unscale_w);
                                float4* at = reinterpret_cast<float4*>(to) + h * 4 + i;
                                if (flushed > 0) {
                                    const float4 o = *at;
                                    v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
                                }
                                *at = v;
                                if (WITH_MU) {
                                    const float4 m = *reinterpret_cast<const float4*>(mu + group * 32 + h * 16 + 4 * i);
                                    with_mu = fmaf(v.x, m.x, fmaf(v.y, m.y, fmaf(v.z, m.z, fmaf(v.w, m.w, with_mu))));
                                }
                            }
                        }
                        // F's place is free: the last product that read it is complete
                        if (WITH_MU && flushed + 1 == segs) reinterpret_cast<float*>(F)[group * 128 + r] = with_mu;
                        tc_fence_before_sync();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&d_free[sg & 1]);
                }
            };
            for (int it = a; it < b; ++it) {
                if ((it & 1) != group) continue;
                flush_until((it - a) / C::SEGMENT_TILES, std::false_type());
                const int s = it % C::STATE_STAGES;
                unsigned char* stage = smem + s * C::STAGE_BYTES;
                const uint32_t q_at = smem_u32(stage);
                const bool in = static_cast<int>((run.u0 + it) % tiles_per_slab) * kTcTile + r < N;
                wait(&full[s], (it / C::STATE_STAGES) & 1);
                float f[64];
                float w = in ? 1.0f : 0.0f, c = 0.0f;
                const uint32_t t_at = tmem + (it % C::T_BUFFERS) * 64 + t_lane;
                if (ok) phi_row<KIND, 8>(q_at, r, 0, f);
                if (GRAD) {
                    wait(&t_full[it % C::T_BUFFERS], (it / C::T_BUFFERS) & 1);
                    if (ok) {
                        tc_fence_after_sync();
                        if (sc.eps >= 0.0f) {
                            f32x2 den = both(0.0f), ft = both(0.0f);
#pragma unroll
                            for (int h = 0; h < 4; ++h) {
                                uint32_t t[16];
                                tmem_load_16cols(t_at + 16 * h, t);
#pragma unroll
                                for (int i = 0; i < 16; i += 2) {
                                    const f32x2 fp = pack2(f[16 * h + i], f[16 * h + i + 1]);
                                    den = fma2(fp, *reinterpret_cast<const f32x2*>(z + 16 * h + i), den);
                                    ft = fma2(fp, pack2(__uint_as_float(t[i]), __uint_as_float(t[i + 1])), ft);
                                }
                            }
                            w = in ? 1.0f / (sum2(den) + sc.eps) : 0.0f;
                            c = in ? sum2(ft) * w : 0.0f;  // scaled as S is
                            if (__any_sync(0xffffffffu, w * sc.eps >= kEpsCounts)) {
                                const float mg = row_mean_dot<KIND, 1>(q_at + kTcTileBytes, r, mu);
                                c = fmaf(-sc.eps * scale_s * w, mg, c);
                            }
                        }
                    }
                }
                const f32x2 ws = both(w);
                auto write_f = [&](int j) {  // piece j of the row of F, head and tail
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        f32x2 x = mul2(pack2(f[8 * j + 2 * i], f[8 * j + 2 * i + 1]), ws);
                        if (SCALED) x = mul2(x, *reinterpret_cast<const f32x2*>(scale_w + 8 * j + 2 * i));
                        const float2 wf = unpack2(x);
                        split_pair<KIND>(wf.x, wf.y, &hi[i], &lo[i]);
                    }
                    sts16(f_at + swizzled(r, j), hi[0], hi[1], hi[2], hi[3]);
                    sts16(f_at + kTcTileBytes + swizzled(r, j), lo[0], lo[1], lo[2], lo[3]);
                };
                // F belongs to one tile at a time, from its first store to the end of the product that reads it.  Writing it in
                // the pass that writes dQ was the faster with dQ (517 against 537 us), after dz the faster without (304 against 327).
                if (GRAD && it > 0) wait(&f_free[(it - 1) & 1], ((it - 1) >> 1) & 1);
                if (ok) {
                    const f32x2 mc = both(-c), wu = both(w * unscale_t), cz = both(GRAD ? -c * unscale_t * w : w);
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        uint32_t t[16], dz[16];
                        if (GRAD) tmem_load_2x16cols(t_at + 16 * h, t, dz_at + 16 * h, dz);
                        else tmem_load_16cols(dz_at + 16 * h, dz);
                        uint32_t d[8];
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const int ch = 16 * h + i;
                            const f32x2 fp = pack2(f[ch], f[ch + 1]);
                            const float2 sum = unpack2(fma2(fp, cz, pack2(__uint_as_float(dz[i]), __uint_as_float(dz[i + 1]))));
                            dz[i] = __float_as_uint(sum.x);
                            dz[i + 1] = __float_as_uint(sum.y);
                            if (GRAD) {
                                const f32x2 tp = pack2(__uint_as_float(t[i]), __uint_as_float(t[i + 1]));
                                const f32x2 x = mul2(fma2(*reinterpret_cast<const f32x2*>(z + ch), mc, tp), wu);
                                const float2 o = unpack2(mul2(x, pack2(slope_of<KIND>(f[ch]), slope_of<KIND>(f[ch + 1]))));
                                d[i / 2] = pack_pair<KIND>(o.x, o.y);
                            }
                        }
                        tmem_store_16cols(dz_at + 16 * h, dz);
                        if (GRAD) {
                            sts16(q_at + swizzled(r, 2 * h), d[0], d[1], d[2], d[3]);
                            sts16(q_at + swizzled(r, 2 * h + 1), d[4], d[5], d[6], d[7]);
                            write_f(2 * h);
                            write_f(2 * h + 1);
                        }
                    }
                    tmem_store_wait();
                }
                if (!GRAD) {
                    if (it > 0) wait(&f_free[(it - 1) & 1], ((it - 1) >> 1) & 1);
                    if (ok) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) write_f(j);
                    }
                }
                tc_fence_before_sync();
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(f_full);
                    if (GRAD) mbar_arrive(&written[s]);
                }
            }
            flush_until(segs, std::true_type());
            seg0 += segs;
            if (GRAD) consumer_sync<C::STATE_WARPS>();  // dS mu of all rows is there
            // dz of the thread's tokens -> sums over the warp: 64 values are halved with the lanes, two are left in each
            if (ok) {
                float v[64];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    uint32_t x[16];
                    tmem_load_16cols(dz_at + 16 * h, x);
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[16 * h + i] = __uint_as_float(x[i]);
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const bool hi = (lane & o) != 0;
#pragma unroll
                    for (int i = 0; i < 2 * o; ++i) {
                        const float keep = hi ? v[i + 2 * o] : v[i], send = hi ? v[i] : v[i + 2 * o];
                        v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                    }
                }
                // o = 16 kept values 32 * (lane bit 4) .., o = 8 then 16 * (bit 3) .., down to 2 * (bit 0)
                if (GRAD && sc.eps >= 0.0f && warp == 0) {  // dz lacks -dS mu so far: heads and tails, either half of the columns
                    const float2* m = reinterpret_cast<const float2*>(F) + lane;
                    v[0] -= (m[0].x + m[32].x) + (m[64].x + m[96].x);
                    v[1] -= (m[0].y + m[32].y) + (m[64].y + m[96].y);
                }
                *reinterpret_cast<float2*>(partial + 128 * 64 + warp * 64 + 2 * lane) = make_float2(v[0], v[1]);
            }
            ++span;
            a = b;
        }
        if (!ok && lane == 0) tc_expired(status);
    }
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, C::TMEM_COLS);
}

// Sum of a slab's partials over the CTAs that worked on it, in a fixed order: out[slab] = S | z (dS | dz).  A partial holds, for each
// 64-feature atom, 64 rows of heads and 64 of tails, vw floats each, and then 64 floats of z from each of the eight warps,
// the warps of an atom next to one another.
template <int SLICES>
static __global__ void __launch_bounds__(kReduceThreads)
backward_tc_reduce_kernel(const float* __restrict__ partials, float* __restrict__ out, int dk, int dv, int tiles_per_slab, long long W,
                          int G, int spans, int vw, int atoms)
{
    constexpr int AT_ONCE = kReduceThreads, OUT = kReduceThreads / SLICES;
    __shared__ long long where[AT_ONCE];  // of a contributing CTA's partial; -1: none
    __shared__ float4 scratch[kReduceThreads];
    const int slab = blockIdx.y, slice = threadIdx.x / OUT, i = 4 * (blockIdx.x * OUT + threadIdx.x % OUT);
    const int floats = grad_state_floats(dk, dv);
    const long long first = static_cast<long long>(slab) * tiles_per_slab, last = first + tiles_per_slab;
    // the CTA that holds the slab's first tile: the largest g with g W / G <= first
    const int g0 = static_cast<int>(((first + 1) * G - 1) / W), g1 = static_cast<int>((last * G - 1) / W);
    const bool of_z = i >= dk * dv;
    const int row = of_z ? i - dk * dv : i / dv, col = of_z ? 0 : i - row * dv, a = row >> 6, ar = row & 63;
    const long long partial_floats = static_cast<long long>(atoms) * 128 * vw + 512;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    auto at4 = [](const float* p) { return *reinterpret_cast<const float4*>(p); };
    bool waited = false;
    pdl_launch_dependents();
    for (int at = g0; at <= g1; at += AT_ONCE) {
        const int n = min(AT_ONCE, g1 + 1 - at);
        __syncthreads();
        if (threadIdx.x < n) {
            const int g = at + threadIdx.x;
            const long long u0 = tc_first_tile(g, W, G), u1 = tc_first_tile(g + 1, W, G);
            where[threadIdx.x] = u1 > u0 && u1 > first && u0 < last
                                     ? (static_cast<long long>(g) * spans + (slab - static_cast<int>(u0 / tiles_per_slab))) * partial_floats
                                     : -1;
        }
        if (!waited) pdl_wait();  // the table needs nothing of the kernel before
        waited = true;
        __syncthreads();
        if (i < floats) {
#pragma unroll 4
            for (int k = slice; k < n; k += SLICES) {
                if (where[k] < 0) continue;
                const float* p = partials + where[k];
                if (!of_z) {
                    sum = add4(sum, add4(at4(p + (a * 128 + ar) * vw + col), at4(p + (a * 128 + 64 + ar) * vw + col)));
                } else {
                    const float* z = p + atoms * 128 * vw + ar;
                    for (int w = a * 8 / atoms; w < (a + 1) * 8 / atoms; w += 4)
                        sum = add4(sum, add4(add4(at4(z + w * 64), at4(z + (w + 1) * 64)), add4(at4(z + (w + 2) * 64), at4(z + (w + 3) * 64))));
                }
            }
        }
    }
    sum = reduce_slices<SLICES>(sum, scratch);
    if (slice == 0 && i < floats) *reinterpret_cast<float4*>(out + static_cast<size_t>(slab) * floats + i) = sum;
}

template <int KIND>
__global__ void __launch_bounds__(BackwardTc::KV_THREADS, 1)
backward_tc_kv_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                      const __grid_constant__ CUtensorMap tmap_dk, const __grid_constant__ CUtensorMap tmap_dv,
                      const float* __restrict__ grad_state, uint32_t* __restrict__ status, int N, int dk, int dv, int tiles_per_slab,
                      long long W, int H, BackwardScales sc, int clear_status)
{
    using C = BackwardTc;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char* F = smem + C::KV_STAGES * C::STAGE_BYTES;
    unsigned char* So = F + C::F_BYTES;
    float* z = reinterpret_cast<float*>(So + C::S_BYTES);
    float* scratch = z + 64;
    uint64_t* full = reinterpret_cast<uint64_t*>(scratch + 32);
    uint64_t* empty = full + C::KV_STAGES;
    uint64_t* t_full = empty + C::KV_STAGES;      // [T_BUFFERS] both products of a tile are complete (commit)
    uint64_t* t_free = t_full + C::T_BUFFERS;  // [T_BUFFERS] ... and have been read (4 warps)
    uint64_t* f_full = t_free + C::T_BUFFERS;
    // [2] for odd and even tiles: with one barrier the group that waits for the tile before its own could find the phase it
    // wants two behind, which a parity cannot tell from one not yet reached
    uint64_t* f_free = f_full + 1;
    uint64_t* s_ready = f_free + 2;
    uint64_t* written = s_ready + 1;  // [KV_STAGES] dK and dV are in place of K and V (4 warps)
    uint64_t* drained = written + C::KV_STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    TcRun run;
    run.u0 = tc_first_tile(blockIdx.x, W, gridDim.x);
    run.n = static_cast<int>(tc_first_tile(blockIdx.x + 1ll, W, gridDim.x) - run.u0);
    run.tiles_per_slab = tiles_per_slab;
    if (tid == 0) {
        for (int s = 0; s < C::KV_STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);  // the tile's stores
            mbar_init(&written[s], 4);
        }
        for (int b = 0; b < C::T_BUFFERS; ++b) mbar_init(&t_full[b], 1), mbar_init(&t_free[b], 4);
        mbar_init(f_full, 4);
        mbar_init(&f_free[0], 1), mbar_init(&f_free[1], 1);
        mbar_init(s_ready, C::KV_WARPS);
        mbar_init(drained, 1);
        mbar_fence_init();
    }
    if (warp == 0) tmem_alloc(tmem_slot, C::TMEM_COLS);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    if (warp == C::KV_WARPS && lane == 0) {
        prefetch_tmap(&tmap_k);
        prefetch_tmap(&tmap_v);
    }
    pdl_launch_dependents();
    pdl_wait();
    if (clear_status != 0 && blockIdx.x == 0 && tid == 0) *status = kStatusOk;

    if (warp == C::KV_WARPS) {
        if (lane == 0) tc_produce<C::KV_STAGES>(&tmap_k, &tmap_v, smem, full, empty, run, H, policy_evict_first(), status);
    } else if (warp == C::KV_WARPS + 2) {
        if (lane == 0) tc_store<C::KV_STAGES, 2>(&tmap_dk, &tmap_dv, smem, written, empty, run, H, status);
    } else if (warp == C::KV_WARPS + 1) {
        if (lane == 0) {
            const uint32_t idesc_k = umma_idesc_f32acc(kind_dtype(KIND), 128, 64);
            const uint32_t idesc_v = umma_idesc_f32acc(kind_dtype(KIND), 128, 64, kUmmaBMnMajor);
            const uint32_t f_addr = smem_u32(F), s_addr = smem_u32(So);
            bool ok = true;
            int unit = 0, j = 0;
            auto second = [&]() {  // T' = F dS of tile j
                ok = ok && mbar_wait(f_full, j & 1);
                if (ok) {
                    tc_fence_after_sync();
                    const uint32_t t_at = tmem + (j % C::T_BUFFERS) * 128 + 64;
#pragma unroll
                    for (int p = 0; p < 3; ++p)  // hi lo, lo hi, hi hi: the small terms first
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            umma_ss(t_at, umma_desc_kmajor_sw128(f_addr + (p == 1 ? kTcTileBytes : 0)) + 2 * k,
                                    umma_desc_mnmajor_sw128(s_addr + (p == 0 ? 64 * 128 : 0) + k * 2048, 0, 1024), idesc_v,
                                    p == 0 && k == 0 ? 0u : 1u);
                    umma_commit(&f_free[j & 1]);
                    umma_commit(&t_full[j % C::T_BUFFERS]);
                }
                ++j;
            };
            for (int it = 0; it < run.n && ok; ++it) {
                if (it == 0 || run.slab(it) != run.slab(it - 1)) {
                    while (j < it && ok) second();
                    ok = ok && mbar_wait(s_ready, unit & 1);
                    ++unit;
                }
                if (it >= C::T_BUFFERS) ok = ok && mbar_wait(&t_free[it % C::T_BUFFERS], ((it / C::T_BUFFERS) & 1) ^ 1);
                ok = ok && mbar_wait(&full[it % C::KV_STAGES], (it / C::KV_STAGES) & 1);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t v_addr = smem_u32(smem + (it % C::KV_STAGES) * C::STAGE_BYTES + kTcTileBytes);
#pragma unroll
                for (int h = 1; h >= 0; --h)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        umma_ss(tmem + (it % C::T_BUFFERS) * 128, umma_desc_kmajor_sw128(v_addr) + 2 * k,
                                umma_desc_kmajor_sw128(s_addr + h * 64 * 128) + 2 * k, idesc_k, h == 1 && k == 0 ? 0u : 1u);
                if (it - j >= 1) second();
            }
            while (j < run.n && ok) second();
            if (!ok) tc_expired(status);
            umma_commit(drained);
            if (!mbar_wait(drained, 0)) tc_expired(status);
        }
    } else {
        const int group = warp / 4, r = tid & 127;
        const uint32_t t_lane = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t f_at = smem_u32(F);
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, parity)); };
        for (int a = 0; a < run.n;) {
            const int slab = run.slab(a), b = run.unit_end(a);
            float scale_s;
            consumer_sync<C::KV_WARPS>();
            tc_load_state<KIND, C::KV_WARPS, 64, 64, false>(grad_state + static_cast<size_t>(slab) * grad_state_floats(dk, dv), dk, dv, So, z,
                                                            nullptr, nullptr, scratch, tid, -1.0f, &scale_s);
            fence_proxy_async_smem();
            consumer_sync<C::KV_WARPS>();
            if (lane == 0) mbar_arrive(s_ready);
            const f32x2 unscale = both(1.0f / scale_s);
            for (int it = a; it < b; ++it) {
                if ((it & 1) != group) continue;
                const int s = it % C::KV_STAGES;
                unsigned char* stage = smem + s * C::STAGE_BYTES;
                const uint32_t k_at = smem_u32(stage), v_at = k_at + kTcTileBytes;
                wait(&full[s], (it / C::KV_STAGES) & 1);
                float f[64];
                if (ok) phi_row<KIND, 8>(k_at, r, 0, f);
                if (it > 0) wait(&f_free[(it - 1) & 1], ((it - 1) >> 1) & 1);
                if (ok) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        uint32_t hi[4], lo[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) split_pair<KIND>(f[8 * j + 2 * i], f[8 * j + 2 * i + 1], &hi[i], &lo[i]);
                        sts16(f_at + swizzled(r, j), hi[0], hi[1], hi[2], hi[3]);
                        sts16(f_at + kTcTileBytes + swizzled(r, j), lo[0], lo[1], lo[2], lo[3]);
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(f_full);
                wait(&t_full[it % C::T_BUFFERS], (it / C::T_BUFFERS) & 1);
                if (ok) {
                    tc_fence_after_sync();
                    const uint32_t t_at = tmem + (it % C::T_BUFFERS) * 128 + t_lane;
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        uint32_t t[16], y[16], d[8], e[8];
                        tmem_load_16cols(t_at + 16 * h, t);
                        tmem_load_16cols(t_at + 64 + 16 * h, y);
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const int ch = 16 * h + i;
                            const f32x2 x = fma2(pack2(__uint_as_float(t[i]), __uint_as_float(t[i + 1])), unscale,
                                                 *reinterpret_cast<const f32x2*>(z + ch));
                            const float2 o = unpack2(mul2(x, pack2(slope_of<KIND>(f[ch]), slope_of<KIND>(f[ch + 1]))));
                            const float2 u = unpack2(mul2(pack2(__uint_as_float(y[i]), __uint_as_float(y[i + 1])), unscale));
                            d[i / 2] = pack_pair<KIND>(o.x, o.y);
                            e[i / 2] = pack_pair<KIND>(u.x, u.y);
                        }
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            sts16(k_at + swizzled(r, 2 * h + p), d[4 * p], d[4 * p + 1], d[4 * p + 2], d[4 * p + 3]);
                            sts16(v_at + swizzled(r, 2 * h + p), e[4 * p], e[4 * p + 1], e[4 * p + 2], e[4 * p + 3]);
                        }
                    }
                }
                tc_fence_before_sync();
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&t_free[it % C::T_BUFFERS]);
                    mbar_arrive(&written[s]);
                }
            }
            a = b;
        }
        if (!ok && lane == 0) tc_expired(status);
    }
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, C::TMEM_COLS);
}

}  // namespace lf
