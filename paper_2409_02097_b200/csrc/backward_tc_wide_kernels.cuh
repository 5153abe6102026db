// The tcgen05 backward pass for feature widths of two 64-channel atoms (d' = 80 and 128, values up to 128 wide): the same
// products, operands and split of the tiles as backward_tc_kernels.cuh, cut differently for shared memory.
//
// One tile is in work at a time, by both warpgroups: thread r of warpgroup a has the 64 features of atom a of token r, so
// den and f . t are sums of two threads, exchanged through shared memory.  The state's operand takes 64 KB, a stage
// (both tensors) 64 KB, and there are two; F's head is written over Q (K) in the stage, its tail into a buffer of its own,
// and the gradients wait in registers until the product that reads F is done, then take F's place and leave by TMA while the
// next tile is under way.
//
//   state:  T[128 x 128] = dY R^T      (16 MMAs of N = 128 for head and tail at dv = 128)
//           D_a[128 x dv] += [F_hi,a | F_lo,a]^T dY for each atom a (8 MMAs each)
//   kv:     T[128 x 128] = V dS^T,  T'[128 x dv] = F_hi dS_hi + F_hi dS_lo + F_lo dS_hi  (24 MMAs)
//
// Per tile of dv = 128: 96 KB (state) or 128 KB (kv) of DRAM traffic, 4200 and 5600 clocks at the measured copy rate; MMAs
// about 2000 and 2600 clocks.  Feature atoms past d' are zeros of the tensor maps: they cost MMA time and no traffic.
#pragma once

#include "backward_tc_kernels.cuh"

namespace lf {

template <int VA>  // 64-channel atoms of the values
struct BackwardTcWide {
    static constexpr int WARPS = 8, PRODUCER_WARP = 8, MMA_WARP = 9, STORE_WARP = 10, THREADS = 32 * 11;
    static constexpr int STAGES = VA == 2 ? 2 : 3, STAGE_BYTES = (2 + VA) * kTcTileBytes;
    static constexpr int FLO_BYTES = 2 * kTcTileBytes, S_HALF = VA * kTcTileBytes, S_BYTES = 2 * S_HALF;
    static constexpr int VW = 64 * VA, SEGMENT_TILES = 32;
    static constexpr int T_COL = 0, D_COL = 128, DZ_COL = 384;      // state: T, two D of VW columns, dz of each atom
    static constexpr int SMEM = STAGES * STAGE_BYTES + FLO_BYTES + S_BYTES + 1024 /*align*/ + 2048 /*z, scales, mu, barriers*/;
    static constexpr int PARTIAL_FLOATS = 2 * 128 * VW + WARPS * 64;
};
static_assert(BackwardTcWide<2>::SMEM <= 227 * 1024 && BackwardTcWide<1>::SMEM <= 227 * 1024, "shared memory");

// The producer and the storing warp: like tc_produce / tc_store with the tensors' atoms one by one.
template <int VA>
__device__ __forceinline__ void wide_produce(const CUtensorMap* a, const CUtensorMap* b, unsigned char* ring, uint64_t* full,
                                             uint64_t* empty, const TcRun& run, int H, uint64_t policy, uint32_t* status)
{
    using C = BackwardTcWide<VA>;
    int issued = 0;
    for (int it = 0; it < run.n; ++it) {
        const int s = it % C::STAGES;
        if (it >= C::STAGES && !mbar_wait(&empty[s], ((it / C::STAGES) & 1) ^ 1)) {
            tc_expired(status);
            break;
        }
        const int slab = run.slab(it), row = static_cast<int>((run.u0 + it) % run.tiles_per_slab) * kTcTile;
        unsigned char* dst = ring + s * C::STAGE_BYTES;
        mbar_expect_tx(&full[s], C::STAGE_BYTES);
        for (int x = 0; x < 2; ++x) tma_load_4d(dst + x * kTcTileBytes, a, 64 * x, row, slab % H, slab / H, &full[s], policy);
        for (int x = 0; x < VA; ++x) tma_load_4d(dst + (2 + x) * kTcTileBytes, b, 64 * x, row, slab % H, slab / H, &full[s], policy);
        ++issued;
    }
    for (int it = issued > C::STAGES ? issued - C::STAGES : 0; it < issued; ++it)
        if (!mbar_wait(&full[it % C::STAGES], (it / C::STAGES) & 1)) {
            tc_expired(status);
            return;
        }
}
template <int VA, bool BOTH>
__device__ __forceinline__ void wide_store(const CUtensorMap* a, const CUtensorMap* b, unsigned char* ring, uint64_t* written,
                                           uint64_t* empty, const TcRun& run, int H, uint32_t* status)
{
    using C = BackwardTcWide<VA>;
    const uint64_t policy = policy_evict_first();
    for (int it = 0; it < run.n; ++it) {
        const int s = it % C::STAGES;
        if (!mbar_wait(&written[s], (it / C::STAGES) & 1)) {
            tc_expired(status);
            break;
        }
        const int slab = run.slab(it), row = static_cast<int>((run.u0 + it) % run.tiles_per_slab) * kTcTile;
        unsigned char* src = ring + s * C::STAGE_BYTES;
        for (int x = 0; x < 2; ++x) tma_store_4d(a, src + x * kTcTileBytes, 64 * x, row, slab % H, slab / H, policy);
        if (BOTH)
            for (int x = 0; x < VA; ++x) tma_store_4d(b, src + (2 + x) * kTcTileBytes, 64 * x, row, slab % H, slab / H, policy);
        tma_store_wait_read();
        mbar_arrive(&empty[s]);
    }
    tma_store_wait_all();
}

template <int KIND, int VA, bool GRAD>
__global__ void __launch_bounds__(BackwardTcWide<VA>::THREADS, 1)
backward_tc_wide_state_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_g,
                              const __grid_constant__ CUtensorMap tmap_dq, const float* __restrict__ state, float* __restrict__ partials,
                              uint32_t* __restrict__ status, int N, int dk, int dv, int tiles_per_slab, long long W, int spans, int H,
                              BackwardScales sc, int clear_status)
{
    using C = BackwardTcWide<VA>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char* Flo = smem + C::STAGES * C::STAGE_BYTES;
    unsigned char* So = Flo + C::FLO_BYTES;
    float* z = reinterpret_cast<float*>(So + C::S_BYTES);
    float* scale_w = z + 128;  // [128] fp16: of each feature's w f
    float* mu = scale_w + 128; // [VW]
    float* scratch = mu + 128;
    uint64_t* full = reinterpret_cast<uint64_t*>(scratch + 32);
    uint64_t* empty = full + C::STAGES;
    uint64_t* written = empty + C::STAGES;
    uint64_t* t_full = written + C::STAGES;  // T of a tile is complete (commit)
    uint64_t* f_full = t_full + 1;           // F of a tile is written (8 warps)
    uint64_t* f_free = f_full + 1;           // ... and has been read (commit)
    uint64_t* s_ready = f_free + 1;
    uint64_t* d_done = s_ready + 1;
    uint64_t* d_free = d_done + 1;
    uint64_t* drained = d_free + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    TcRun run;
    run.u0 = tc_first_tile(blockIdx.x, W, gridDim.x);
    run.n = static_cast<int>(tc_first_tile(blockIdx.x + 1ll, W, gridDim.x) - run.u0);
    run.tiles_per_slab = tiles_per_slab;
    if (tid == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], GRAD ? 2 : 1);  // the second product's commit; with dQ, its store
            mbar_init(&written[s], C::WARPS);
        }
        mbar_init(t_full, 1);
        mbar_init(f_full, C::WARPS);
        mbar_init(f_free, 1);
        mbar_init(s_ready, C::WARPS);
        mbar_init(d_done, 1);
        mbar_init(d_free, C::WARPS);
        mbar_init(drained, 1);
        mbar_fence_init();
    }
    if (warp == 0) tmem_alloc(tmem_slot, 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    if (warp == C::PRODUCER_WARP && lane == 0) {
        prefetch_tmap(&tmap_q);
        prefetch_tmap(&tmap_g);
    }
    pdl_launch_dependents();
    pdl_wait();
    if (clear_status != 0 && blockIdx.x == 0 && tid == 0) *status = kStatusOk;

    if (warp == C::PRODUCER_WARP) {
        if (lane == 0)
            wide_produce<VA>(&tmap_q, &tmap_g, smem, full, empty, run, H, GRAD ? policy_evict_first() : policy_evict_normal(), status);
    } else if (warp == C::STORE_WARP) {
        if (GRAD && lane == 0) wide_store<VA, false>(&tmap_dq, nullptr, smem, written, empty, run, H, status);
    } else if (warp == C::MMA_WARP) {
        if (lane == 0) {
            const uint32_t idesc_t = umma_idesc_f32acc(kind_dtype(KIND), 128, 128);
            const uint32_t idesc_d = umma_idesc_f32acc(kind_dtype(KIND), 128, C::VW, kUmmaAMnMajor | kUmmaBMnMajor);
            const uint32_t flo = smem_u32(Flo), s_addr = smem_u32(So);
            bool ok = true;
            int seg = 0, in_seg = 0, unit = 0;
            for (int it = 0; it < run.n && ok; ++it) {
                const uint32_t q_addr = smem_u32(smem + (it % C::STAGES) * C::STAGE_BYTES), g_addr = q_addr + 2 * kTcTileBytes;
                if (GRAD) {
                    if (it == 0 || run.slab(it) != run.slab(it - 1)) {
                        ok = ok && mbar_wait(s_ready, unit & 1);
                        ++unit;
                    }
                    ok = ok && mbar_wait(&full[it % C::STAGES], (it / C::STAGES) & 1);
                    if (!ok) break;
                    tc_fence_after_sync();
                    // T has been read: the tile before is through f_full below
#pragma unroll
                    for (int h = 1; h >= 0; --h)
#pragma unroll
                        for (int k = 0; k < 4 * VA; ++k)
                            umma_ss(tmem + C::T_COL, umma_desc_kmajor_sw128(g_addr + (k / 4) * kTcTileBytes) + 2 * (k & 3),
                                    umma_desc_kmajor_sw128(s_addr + h * C::S_HALF + (k / 4) * kTcTileBytes) + 2 * (k & 3), idesc_t,
                                    h == 1 && k == 0 ? 0u : 1u);
                    umma_commit(t_full);
                }
                if (in_seg == 0 && seg >= 1) ok = ok && mbar_wait(d_free, (seg & 1) ^ 1);
                ok = ok && mbar_wait(f_full, it & 1);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    const uint32_t hi = q_addr + a * kTcTileBytes, lo = flo + a * kTcTileBytes;
#pragma unroll
                    for (int k = 0; k < kTcTile / 16; ++k)  // rows 0 .. 63 of A: the head; 64 .. 127: the tail, lo - hi bytes on
                        umma_ss(tmem + C::D_COL + a * C::VW, umma_desc_mnmajor_sw128(hi + k * 2048, lo - hi, 1024),
                                umma_desc_mnmajor_sw128(g_addr + k * 2048, kTcTileBytes, 1024), idesc_d, in_seg == 0 && k == 0 ? 0u : 1u);
                }
                umma_commit(f_free);
                umma_commit(&empty[it % C::STAGES]);
                ++in_seg;
                if (in_seg == C::SEGMENT_TILES || it + 1 == run.unit_end(it)) {
                    umma_commit(d_done);
                    ++seg;
                    in_seg = 0;
                }
            }
            if (!ok) tc_expired(status);
            umma_commit(drained);
            if (!mbar_wait(drained, 0)) tc_expired(status);
        }
    } else {
        const int a = warp / 4, quarter = warp & 3, r = tid & 127;  // a: the thread's feature atom
        const uint32_t t_lane = static_cast<uint32_t>(quarter * 32) << 16;
        const uint32_t flo_at = smem_u32(Flo) + a * kTcTileBytes, dz_at = tmem + C::DZ_COL + a * 64 + t_lane;
        const uint32_t t_at = tmem + C::T_COL + a * 64 + t_lane;
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, parity)); };
        uint32_t d[32];    // dQ of the tile before, packed, until the product has read F
        int pending = -1;  // its index
        auto finish = [&]() {
            if (pending < 0) return;
            wait(f_free, pending & 1);
            if (GRAD) {
                const uint32_t at = smem_u32(smem + (pending % C::STAGES) * C::STAGE_BYTES) + a * kTcTileBytes;
                if (ok) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) sts16(at + swizzled(r, j), d[4 * j], d[4 * j + 1], d[4 * j + 2], d[4 * j + 3]);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&written[pending % C::STAGES]);
            }
            pending = -1;
        };
        int seg0 = 0, span = 0;
        for (int first = 0; first < run.n;) {
            const int slab = run.slab(first), last = run.unit_end(first);
            float scale_s = 1.0f;
            float* partial = partials + (static_cast<size_t>(blockIdx.x) * spans + span) * C::PARTIAL_FLOATS;
            if (GRAD) {
                const float* S = state + static_cast<size_t>(slab) * grad_state_floats(dk, dv);
                consumer_sync<C::WARPS>();
                tc_load_state<KIND, C::WARPS, 128, C::VW, true>(S, dk, dv, So, z, mu, scale_w, scratch, tid, sc.eps, &scale_s);
                fence_proxy_async_smem();
                consumer_sync<C::WARPS>();
                if (lane == 0) mbar_arrive(s_ready);
            }
            constexpr bool SCALED = GRAD && kind_dtype(KIND) == kDtypeFp16;
            const float unscale_t = 1.0f / scale_s, unscale_w = SCALED ? 1.0f / scale_w[a * 64 + (r & 63)] : 1.0f;
            if (ok) {
                uint32_t nothing[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) nothing[i] = 0u;
#pragma unroll
                for (int h = 0; h < 4; ++h) tmem_store_16cols(dz_at + 16 * h, nothing);
                tmem_store_wait();
            }
            int flushed = 0;
            const int segs = (last - first + C::SEGMENT_TILES - 1) / C::SEGMENT_TILES;
            auto flush_until = [&](int want, auto behind) {  // this warp's 32 rows of its atom's accumulator
                constexpr bool WITH_MU = GRAD && decltype(behind)::value;
                for (; flushed < want; ++flushed) {
                    wait(d_done, (seg0 + flushed) & 1);
                    if (ok) {
                        tc_fence_after_sync();
                        float* to = partial + (a * 128 + r) * C::VW;
                        float with_mu = 0.0f;  // the row times mu
#pragma unroll
                        for (int h = 0; h < C::VW / 16; ++h) {
                            uint32_t x[16];
                            tmem_load_16cols(tmem + C::D_COL + a * C::VW + 16 * h + t_lane, x);
                            float4* at = reinterpret_cast<float4*>(to + 16 * h);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float4 v = make_float4(__uint_as_float(x[4 * i]) * unscale_w, __uint_as_float(x[4 * i + 1]) * unscale_w,
                                                       __uint_as_float(x[4 * i + 2]) * unscale_w, __uint_as_float(x[4 * i + 3]) * unscale_w);
                                if (flushed > 0) {
                                    const float4 o = at[i];
                                    v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
                                }
                                at[i] = v;
                                if (WITH_MU) {
                                    const float4 m = *reinterpret_cast<const float4*>(mu + 16 * h + 4 * i);
                                    with_mu = fmaf(v.x, m.x, fmaf(v.y, m.y, fmaf(v.z, m.z, fmaf(v.w, m.w, with_mu))));
                                }
                            }
                        }
                        // the tail's place is free: the last product that read it is complete
                        if (WITH_MU && flushed + 1 == segs) reinterpret_cast<float*>(Flo)[a * 128 + r] = with_mu;
                        tc_fence_before_sync();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(d_free);
                }
            };
            for (int it = first; it < last; ++it) {
                const int s = it % C::STAGES;
                const uint32_t q_at = smem_u32(smem + s * C::STAGE_BYTES) + a * kTcTileBytes;
                const bool in = static_cast<int>((run.u0 + it) % tiles_per_slab) * kTcTile + r < N;
                wait(&full[s], (it / C::STAGES) & 1);
                float f[64];
                float w = in ? 1.0f : 0.0f, c = 0.0f;
                if (ok) phi_row<KIND, 8>(q_at, r, 0, f);
                finish();
                flush_until((it - first) / C::SEGMENT_TILES, std::false_type());
                if (GRAD) {
                    wait(t_full, it & 1);
                    tc_fence_after_sync();
                    if (sc.eps >= 0.0f) {
                        f32x2 den = both(0.0f), ft = both(0.0f);
                        if (ok) {
#pragma unroll
                            for (int h = 0; h < 4; ++h) {
                                uint32_t t[16];
                                tmem_load_16cols(t_at + 16 * h, t);
#pragma unroll
                                for (int i = 0; i < 16; i += 2) {
                                    const f32x2 fp = pack2(f[16 * h + i], f[16 * h + i + 1]);
                                    den = fma2(fp, *reinterpret_cast<const f32x2*>(z + a * 64 + 16 * h + i), den);
                                    ft = fma2(fp, pack2(__uint_as_float(t[i]), __uint_as_float(t[i + 1])), ft);
                                }
                            }
                        }
                        // The other atom's thread of the token takes these through the tail's buffer, which nothing reads now.
                        float2* mine = reinterpret_cast<float2*>(Flo) + a * 128 + r;
                        const float2* other = reinterpret_cast<const float2*>(Flo) + (1 - a) * 128 + r;
                        const float my_den = sum2(den), my_ft = sum2(ft);
                        *mine = make_float2(my_den, my_ft);
                        consumer_sync<C::WARPS>();
                        const float2 o = *other;
                        consumer_sync<C::WARPS>();  // before the tail is written there
                        // the same order on both sides
                        const float d0 = a == 0 ? my_den : o.x, d1 = a == 0 ? o.x : my_den, f0 = a == 0 ? my_ft : o.y, f1 = a == 0 ? o.y : my_ft;
                        w = in ? 1.0f / (d0 + d1 + sc.eps) : 0.0f;
                        c = in ? (f0 + f1) * w : 0.0f;  // scaled as S is
                        if (__any_sync(0xffffffffu, w * sc.eps >= kEpsCounts)) {
                            const float mg = row_mean_dot<KIND, VA>(smem_u32(smem + s * C::STAGE_BYTES) + 2 * kTcTileBytes, r, mu);
                            c = fmaf(-sc.eps * scale_s * w, mg, c);
                        }
                    }
                }
                if (ok) {
                    const f32x2 mc = both(-c), wu = both(w * unscale_t), cz = both(GRAD ? -c * unscale_t * w : w), ws = both(w);
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        uint32_t t[16], dz[16];
                        if (GRAD) tmem_load_2x16cols(t_at + 16 * h, t, dz_at + 16 * h, dz);
                        else tmem_load_16cols(dz_at + 16 * h, dz);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            uint32_t hi[4], lo[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int k = 8 * e + 2 * i, ch = 16 * h + k;
                                const f32x2 fp = pack2(f[ch], f[ch + 1]);
                                const float2 sum = unpack2(fma2(fp, cz, pack2(__uint_as_float(dz[k]), __uint_as_float(dz[k + 1]))));
                                dz[k] = __float_as_uint(sum.x);
                                dz[k + 1] = __float_as_uint(sum.y);
                                f32x2 wfp = mul2(fp, ws);
                                if (SCALED) wfp = mul2(wfp, *reinterpret_cast<const f32x2*>(scale_w + a * 64 + ch));
                                const float2 wf = unpack2(wfp);
                                split_pair<KIND>(wf.x, wf.y, &hi[i], &lo[i]);
                                if (GRAD) {
                                    const f32x2 tp = pack2(__uint_as_float(t[k]), __uint_as_float(t[k + 1]));
                                    const f32x2 x = mul2(fma2(*reinterpret_cast<const f32x2*>(z + a * 64 + ch), mc, tp), wu);
                                    const float2 o = unpack2(mul2(x, pack2(slope_of<KIND>(f[ch]), slope_of<KIND>(f[ch + 1]))));
                                    d[ch / 2] = pack_pair<KIND>(o.x, o.y);
                                }
                            }
                            sts16(q_at + swizzled(r, 2 * h + e), hi[0], hi[1], hi[2], hi[3]);
                            sts16(flo_at + swizzled(r, 2 * h + e), lo[0], lo[1], lo[2], lo[3]);
                        }
                        tmem_store_16cols(dz_at + 16 * h, dz);
                    }
                    tmem_store_wait();
                }
                tc_fence_before_sync();
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(f_full);
                pending = it;
            }
            finish();
            flush_until(segs, std::true_type());
            seg0 += segs;
            if (GRAD) consumer_sync<C::WARPS>();  // dS mu of all rows is there
            if (ok) {  // dz of the thread's tokens -> sums over the warp, as in the narrow kernel
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
                if (GRAD && sc.eps >= 0.0f && quarter == 0) {  // dz lacks -dS mu so far: heads and tails
                    const float2* m = reinterpret_cast<const float2*>(Flo) + a * 64 + lane;
                    v[0] -= m[0].x + m[32].x;
                    v[1] -= m[0].y + m[32].y;
                }
                *reinterpret_cast<float2*>(partial + 2 * 128 * C::VW + warp * 64 + 2 * lane) = make_float2(v[0], v[1]);
            }
            ++span;
            first = last;
        }
        if (!ok && lane == 0) tc_expired(status);
    }
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

template <int KIND, int VA>
__global__ void __launch_bounds__(BackwardTcWide<VA>::THREADS, 1)
backward_tc_wide_kv_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                           const __grid_constant__ CUtensorMap tmap_dk, const __grid_constant__ CUtensorMap tmap_dv,
                           const float* __restrict__ grad_state, uint32_t* __restrict__ status, int N, int dk, int dv, int tiles_per_slab,
                           long long W, int H, BackwardScales sc, int clear_status)
{
    using C = BackwardTcWide<VA>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char* Flo = smem + C::STAGES * C::STAGE_BYTES;
    unsigned char* So = Flo + C::FLO_BYTES;
    float* z = reinterpret_cast<float*>(So + C::S_BYTES);
    float* scratch = z + 128;
    uint64_t* full = reinterpret_cast<uint64_t*>(scratch + 32);
    uint64_t* empty = full + C::STAGES;
    uint64_t* written = empty + C::STAGES;
    uint64_t* t_full = written + C::STAGES;  // [2] both products of a tile are complete (commit): F has been read too
    uint64_t* t_free = t_full + 2;           // [2] ... and have been read (8 warps)
    uint64_t* f_full = t_free + 2;
    uint64_t* s_ready = f_full + 1;
    uint64_t* drained = s_ready + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    TcRun run;
    run.u0 = tc_first_tile(blockIdx.x, W, gridDim.x);
    run.n = static_cast<int>(tc_first_tile(blockIdx.x + 1ll, W, gridDim.x) - run.u0);
    run.tiles_per_slab = tiles_per_slab;
    if (tid == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);  // the tile's stores
            mbar_init(&written[s], C::WARPS);
        }
        for (int b = 0; b < 2; ++b) mbar_init(&t_full[b], 1), mbar_init(&t_free[b], C::WARPS);
        mbar_init(f_full, C::WARPS);
        mbar_init(s_ready, C::WARPS);
        mbar_init(drained, 1);
        mbar_fence_init();
    }
    if (warp == 0) tmem_alloc(tmem_slot, 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    if (warp == C::PRODUCER_WARP && lane == 0) {
        prefetch_tmap(&tmap_k);
        prefetch_tmap(&tmap_v);
    }
    pdl_launch_dependents();
    pdl_wait();
    if (clear_status != 0 && blockIdx.x == 0 && tid == 0) *status = kStatusOk;

    if (warp == C::PRODUCER_WARP) {
        if (lane == 0) wide_produce<VA>(&tmap_k, &tmap_v, smem, full, empty, run, H, policy_evict_first(), status);
    } else if (warp == C::STORE_WARP) {
        if (lane == 0) wide_store<VA, true>(&tmap_dk, &tmap_dv, smem, written, empty, run, H, status);
    } else if (warp == C::MMA_WARP) {
        if (lane == 0) {
            const uint32_t idesc_k = umma_idesc_f32acc(kind_dtype(KIND), 128, 128);
            const uint32_t idesc_v = umma_idesc_f32acc(kind_dtype(KIND), 128, C::VW, kUmmaBMnMajor);
            const uint32_t flo = smem_u32(Flo), s_addr = smem_u32(So);
            bool ok = true;
            int unit = 0;
            for (int it = 0; it < run.n && ok; ++it) {
                const uint32_t k_addr = smem_u32(smem + (it % C::STAGES) * C::STAGE_BYTES), v_addr = k_addr + 2 * kTcTileBytes;
                const uint32_t t_at = tmem + (it & 1) * 256;
                if (it == 0 || run.slab(it) != run.slab(it - 1)) {
                    ok = ok && mbar_wait(s_ready, unit & 1);
                    ++unit;
                }
                if (it >= 2) ok = ok && mbar_wait(&t_free[it & 1], ((it >> 1) & 1) ^ 1);
                ok = ok && mbar_wait(&full[it % C::STAGES], (it / C::STAGES) & 1);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll
                for (int h = 1; h >= 0; --h)
#pragma unroll
                    for (int k = 0; k < 4 * VA; ++k)
                        umma_ss(t_at, umma_desc_kmajor_sw128(v_addr + (k / 4) * kTcTileBytes) + 2 * (k & 3),
                                umma_desc_kmajor_sw128(s_addr + h * C::S_HALF + (k / 4) * kTcTileBytes) + 2 * (k & 3), idesc_k,
                                h == 1 && k == 0 ? 0u : 1u);
                ok = ok && mbar_wait(f_full, it & 1);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll
                for (int p = 0; p < 3; ++p)  // hi lo, lo hi, hi hi: the small terms first
#pragma unroll
                    for (int k = 0; k < 8; ++k)  // 16 features a step: four of each atom of F, rows 16 k of dS
                        umma_ss(t_at + 128, umma_desc_kmajor_sw128((p == 1 ? flo : k_addr) + (k / 4) * kTcTileBytes) + 2 * (k & 3),
                                umma_desc_mnmajor_sw128(s_addr + (p == 0 ? C::S_HALF : 0) + k * 2048, kTcTileBytes, 1024), idesc_v,
                                p == 0 && k == 0 ? 0u : 1u);
                umma_commit(&t_full[it & 1]);
            }
            if (!ok) tc_expired(status);
            umma_commit(drained);
            if (!mbar_wait(drained, 0)) tc_expired(status);
        }
    } else {
        const int a = warp / 4, quarter = warp & 3, r = tid & 127;
        const uint32_t t_lane = static_cast<uint32_t>(quarter * 32) << 16;
        const uint32_t flo_at = smem_u32(Flo) + a * kTcTileBytes;
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, parity)); };
        for (int first = 0; first < run.n;) {
            const int slab = run.slab(first), last = run.unit_end(first);
            float scale_s;
            consumer_sync<C::WARPS>();
            tc_load_state<KIND, C::WARPS, 128, C::VW, false>(grad_state + static_cast<size_t>(slab) * grad_state_floats(dk, dv), dk, dv, So, z,
                                                             nullptr, nullptr, scratch, tid, -1.0f, &scale_s);
            fence_proxy_async_smem();
            consumer_sync<C::WARPS>();
            if (lane == 0) mbar_arrive(s_ready);
            const f32x2 unscale = both(1.0f / scale_s);
            for (int it = first; it < last; ++it) {
                const int s = it % C::STAGES;
                const uint32_t k_at = smem_u32(smem + s * C::STAGE_BYTES) + a * kTcTileBytes;
                wait(&full[s], (it / C::STAGES) & 1);
                float f[64];
                if (ok) {
                    phi_row<KIND, 8>(k_at, r, 0, f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        uint32_t hi[4], lo[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) split_pair<KIND>(f[8 * j + 2 * i], f[8 * j + 2 * i + 1], &hi[i], &lo[i]);
                        sts16(k_at + swizzled(r, j), hi[0], hi[1], hi[2], hi[3]);
                        sts16(flo_at + swizzled(r, j), lo[0], lo[1], lo[2], lo[3]);  // the tile before was through t_full
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(f_full);
                wait(&t_full[it & 1], (it >> 1) & 1);
                if (ok) {
                    tc_fence_after_sync();
                    const uint32_t t_at = tmem + (it & 1) * 256 + a * 64 + t_lane;
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        uint32_t t[16], d[8];
                        tmem_load_16cols(t_at + 16 * h, t);
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const int ch = 16 * h + i;
                            const f32x2 x = fma2(pack2(__uint_as_float(t[i]), __uint_as_float(t[i + 1])), unscale,
                                                 *reinterpret_cast<const f32x2*>(z + a * 64 + ch));
                            const float2 o = unpack2(mul2(x, pack2(slope_of<KIND>(f[ch]), slope_of<KIND>(f[ch + 1]))));
                            d[i / 2] = pack_pair<KIND>(o.x, o.y);
                        }
                        sts16(k_at + swizzled(r, 2 * h), d[0], d[1], d[2], d[3]);
                        sts16(k_at + swizzled(r, 2 * h + 1), d[4], d[5], d[6], d[7]);
                    }
                    // dV: an atom for each warpgroup, or half an atom
                    constexpr int PIECES = 4 * VA;
                    const int col0 = a * 8 * PIECES;
                    const uint32_t v_at = smem_u32(smem + s * C::STAGE_BYTES) + (2 + col0 / 64) * kTcTileBytes;
#pragma unroll
                    for (int h = 0; h < PIECES / 2; ++h) {
                        uint32_t y[16], e[8];
                        tmem_load_16cols(tmem + (it & 1) * 256 + 128 + col0 + 16 * h + t_lane, y);
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const float2 u = unpack2(mul2(pack2(__uint_as_float(y[i]), __uint_as_float(y[i + 1])), unscale));
                            e[i / 2] = pack_pair<KIND>(u.x, u.y);
                        }
                        const int j = (col0 & 63) / 8 + 2 * h;
                        sts16(v_at + swizzled(r, j), e[0], e[1], e[2], e[3]);
                        sts16(v_at + swizzled(r, j + 1), e[4], e[5], e[6], e[7]);
                    }
                }
                tc_fence_before_sync();
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&t_free[it & 1]);
                    mbar_arrive(&written[s]);
                }
            }
            first = last;
        }
        if (!ok && lane == 0) tc_expired(status);
    }
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

}  // namespace lf
