// The gated linear recurrence of include/linfusion_layers.h, forward and backward.
//
// Mathematics.  h_t = h_(t-1) + e_t (v_t - h_(t-1)) is the map h -> A h + H with A = 1 - e, H = e v, and maps compose:
// (A1, H1) then (A2, H2) is (A1 A2, A2 H1 + H2).  So is the gradient's way back, G -> (1 - e)(dh + G).  The update is kept in the form
// h + e (v - h) with e formed without cancellation: near e = 0 (long memories) 1 - e has lost e's digits, and a product of
// thousands of such factors would show it.
//
// Three launches.  recurrence_maps_kernel forms the map of every tile of 64 tokens (in a backward pass without kept states those of the
// states and of the gradient at once), recurrence_scan_kernel goes through the tiles of each channel (a run of them a thread, then the
// runs' maps, then the run again with what enters it) and leaves what enters each tile, which is also what a forward pass keeps;
// recurrence_kernel and recurrence_backward_kernel then do every tile by itself.  Sums and products have a fixed order, nothing waits for
// another block.  The price is that inputs are read twice: 14 bytes a value instead of 8 forward, 18 instead of 14 backward (the maps need
// decay and dh alone; the states are kept), but the second time from L2 where they fit.  The one-pass form, in which a tile waits for the
// maps of the tiles before it while its own inputs stay in registers, was built first and was slower: 363 against 265 us forward for
// 131072 x 640, 49 against 42 for 2 x 4096 x 1280, and 145 against 108 backward for 2 x 16384 x 640; its blocks spent two thirds of
// their time waiting or at barriers, and registers allow but two on an SM.
//
// What bounds it now: latency.  Neither DRAM (15 to 40 % of its rate) nor the issue slots (48 to 59 %) are full; the registers allow 16 to 24
// warps an SM, and each block loads, waits and meets three to five barriers once.  A value takes 32 instructions in the maps, 37 in the
// forward pass and 77 in the backward pass (93 from checkpoints), of which the arithmetic proper is half; it runs on pairs of fp32 values.
// The maps of the states alone spill 196 bytes a thread (80 registers, 24 warps an SM), those of both kinds from checkpoints
// 112 and 312, the gated backward pass 24.
#pragma once

#include "column_sums.cuh"
#include "pack8.cuh"
#include "sigmoid.cuh"

namespace lf {

constexpr int kRecSlab = 64;    // channels of a tile: rows of 128 bytes
constexpr int kRecEvery = 64;   // tokens of a tile, and from one kept state to the next
constexpr int kRecShort = 8;    // tokens up to which a thread goes through the sequence alone

struct RecInput {
    const char* p;                // 16-bit values, or codes
    const unsigned char* scales;  // of codes, else null
    long long batch, row;         // bytes
};
struct RecOutput {
    char* p;
    long long batch, row;
};
struct RecParams {
    RecInput x, decay, gate, dh;
    RecOutput h;                  // forward
    RecOutput dx, ddecay, dgate;  // backward
    const float *rate, *h0, *dlast;
    const float* states;          // [B][tiles][C]: what enters each tile (null: one tile, h0 does)
    const float* grads;           // [B][tiles][C]: the gradient that enters each tile from behind (null: one tile, dlast does)
    float2 *maps, *grad_maps;     // [B][tiles][width]
    float *last, *dh0, *rate_partials, *keep;  // keep: where the state that enters the only tile is left
    int B, N, C, slabs, tiles, stacks, width, scale_groups, reverse;  // width: channels in whole slabs; stacks: see RecPlace
};

// The sigmoid in a form from which 1 - sigmoid comes without a difference: k = exp(-x), the sigmoid 1 / (1 + k), the rest of it k / (1 + k).
// k is held to 2^127, where the sigmoid is 0 (and so is the product: what it multiplies is 0 there).  A NaN stays one.
constexpr float kRecClosed = 1.7014118346046923e38f;
__device__ __forceinline__ f32x2 rec_odds(f32x2 x)
{
    const float2 k = unpack2(exp_minus2(x));
    float a, b;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(k.x), "f"(kRecClosed));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(b) : "f"(k.y), "f"(kRecClosed));
    return pack2(a, b);
}
__device__ __forceinline__ f32x2 rec_open(f32x2 k) { return rcp2(add2(k, both(1.0f))); }
// 1 - exp(-L) for 0 <= L <= 1, where it is L times a polynomial of degree six: least-squares fit of (1 - exp(-L)) / L at 4000
// Chebyshev nodes with the reciprocal of its value as the weight, off by at most 2.6e-9 of itself, 1.8e-8 with the coefficients rounded to
// fp32 and 1.4e-7 evaluated in it.  No cancellation, and none of the special function unit's time, of which the sigmoids take most.
__device__ __forceinline__ f32x2 rec_one_minus_exp_unit(f32x2 L)
{
    f32x2 s = fma2(L, both(0.00012827072f), both(-0.0012983276f));
    s = fma2(L, s, both(0.008272708f));
    s = fma2(L, s, both(-0.04164537f));
    s = fma2(L, s, both(0.16666305f));
    s = fma2(L, s, both(-0.49999976f));
    s = fma2(L, s, both(1.0f));
    return mul2(L, s);
}
// The same for any L >= 0: above 1 from the exponential.
__device__ __forceinline__ f32x2 rec_one_minus_exp(f32x2 L)
{
    const float2 a = unpack2(L), b = unpack2(rec_one_minus_exp_unit(L)), c = unpack2(fma2(exp_minus2(L), both(-1.0f), both(1.0f)));
    return pack2(a.x <= 1.0f ? b.x : c.x, a.y <= 1.0f ? b.y : c.y);
}
// exp(-L), with all its digits whether it is next to 1 or to 0.
__device__ __forceinline__ f32x2 rec_keep(f32x2 L)
{
    const float2 a = unpack2(L), b = unpack2(fma2(rec_one_minus_exp_unit(L), both(-1.0f), both(1.0f))), c = unpack2(exp_minus2(L));
    return pack2(a.x < 0.25f ? b.x : c.x, a.y < 0.25f ? b.y : c.y);
}
// e = 1 - exp(-L) and exp(-L) in one number: e up to L = 0.7, beyond it -exp(-L) (with its sign, also where it is zero).
__device__ __forceinline__ f32x2 rec_both(f32x2 L)
{
    const float2 a = unpack2(L), e = unpack2(rec_one_minus_exp(L)), k = unpack2(exp_minus2(L));
    return pack2(a.x > 0.7f ? -k.x : e.x, a.y > 0.7f ? -k.y : e.y);
}
__device__ __forceinline__ f32x2 rec_both_e(f32x2 w)
{
    const float2 a = unpack2(w);
    return pack2(__float_as_int(a.x) < 0 ? 1.0f + a.x : a.x, __float_as_int(a.y) < 0 ? 1.0f + a.y : a.y);
}
__device__ __forceinline__ f32x2 rec_both_keep(f32x2 w)
{
    const float2 a = unpack2(w);
    return pack2(__float_as_int(a.x) < 0 ? -a.x : 1.0f - a.x, __float_as_int(a.y) < 0 ? -a.y : 1.0f - a.y);
}
template <bool WIDE>
__device__ __forceinline__ f32x2 rec_decay(f32x2 L) { return WIDE ? rec_one_minus_exp(L) : rec_one_minus_exp_unit(L); }
// Whether a lane's rates pass 1 (or are NaN), for the whole warp; all warps of a block have the same channels.
template <int P>
__device__ __forceinline__ bool rec_wide(const f32x2 (&rate)[P])
{
    bool unit = true;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const float2 r = unpack2(rate[i]);
        unit = unit && r.x <= 1.0f && r.y <= 1.0f;
    }
    return !__all_sync(0xffffffffu, unit);
}
template <bool B>
struct RecBool {
    static constexpr bool value = B;
};
__device__ __forceinline__ float rec_least(float least, f32x2 s)
{
    const float2 f = unpack2(s);
    return fminf(least, fminf(f.x, f.y));
}
// v where the token counts, 0 where its sigmoid(decay) is 0: padding, whatever v holds.
__device__ __forceinline__ f32x2 rec_unless_padding(f32x2 s, f32x2 v)
{
    const float2 a = unpack2(s), b = unpack2(v);
    return pack2(a.x == 0.0f ? 0.0f : b.x, a.y == 0.0f ? 0.0f : b.y);
}

// ------------------------------------------------------------------------------------------ a thread's share of a tile
// Four channels a thread, so sixteen lanes make a row; R tokens a thread: four, so that a tile is eight warps of two segments each, or
// eight and four warps, where the registers allow it (what a thread does once, some 200 instructions, weighs half as much).
constexpr int kRecV = 4, kRecP = kRecV / 2, kRecR = 4, kRecMapsR = 8, kRecForwardR = 8;
constexpr int kRecLanes = kRecSlab / kRecV, kRecSegs = 32 / kRecLanes;
__host__ __device__ constexpr int rec_warps(int R) { return kRecEvery / (kRecSegs * R); }
constexpr int kRecWarps = rec_warps(kRecR), kRecThreads = 32 * kRecWarps, kRecMapsThreads = 32 * rec_warps(kRecMapsR),
              kRecForwardThreads = 32 * rec_warps(kRecForwardR);
static_assert(kRecWarps * kRecSegs * kRecR == kRecEvery, "a tile");

// Blocks: slabs along x, so that neighbours read the same rows; tiles along y, and where there are more than kRecTilesY, on along z.
constexpr int kRecTilesY = 32768;
template <int R>
struct RecPlace {
    int b, tile, slab, lane, warp, cl, ch, pos0, left;  // cl: channel in the slab; left: tokens from pos0 on (none behind the last channel)
    __device__ __forceinline__ explicit RecPlace(const RecParams& p)
    {
        slab = blockIdx.x;
        tile = blockIdx.y;
        b = blockIdx.z;
        if (p.stacks > 1) {
            b = static_cast<int>(blockIdx.z) / p.stacks;
            tile += (static_cast<int>(blockIdx.z) - b * p.stacks) * kRecTilesY;
        }
        lane = threadIdx.x & 31;
        warp = threadIdx.x >> 5;
        cl = (lane % kRecLanes) * kRecV;
        ch = slab * kRecSlab + cl;
        pos0 = tile * kRecEvery + (warp * kRecSegs + lane / kRecLanes) * R;
        left = ch < p.C && tile < p.tiles ? p.N - pos0 : 0;
    }
};
// A thread's tokens in a tensor: the first one's address, and the way to the next.
struct RecRun {
    char* p;
    long long step;
    template <int R>
    __device__ __forceinline__ RecRun(const char* base, long long batch, long long row, const RecParams& q, const RecPlace<R>& at, long long channel_bytes)
    {
        step = q.reverse ? -row : row;
        p = const_cast<char*>(base) + at.b * batch + (q.reverse ? q.N - 1 - at.pos0 : at.pos0) * row + channel_bytes;
    }
    __device__ __forceinline__ char* at(int r) const { return p + r * step; }
};
// A thread's tokens of an input as they are read: two words each, or a word of codes.  In packed ones the eight lanes of a scale load
// one of their R tokens' scales each, and hand it on when it is needed.
template <int R, bool PACKED>
struct RecRaw {
    uint32_t w[R][PACKED ? 1 : 2];
    int scale;
};
template <int R, bool PACKED>
__device__ __forceinline__ void rec_read(RecRaw<R, PACKED>& raw, const RecInput& in, const RecParams& p, const RecPlace<R>& at)
{
    const RecRun run(in.p, in.batch, in.row, p, at, PACKED ? at.ch : 2ll * at.ch);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        raw.w[r][0] = 0u;
        if (!PACKED) raw.w[r][PACKED ? 0 : 1] = 0u;
        if (r < at.left) {
            // plain loads: an output may lie over this input, each element written by the thread that has read it
            if constexpr (PACKED) asm volatile("ld.global.u32 %0, [%1];" : "=r"(raw.w[r][0]) : "l"(run.at(r)) : "memory");
            else asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(raw.w[r][0]), "=r"(raw.w[r][1]) : "l"(run.at(r)) : "memory");
        }
    }
    if constexpr (PACKED) {
        const int pos = at.pos0 + (at.lane & 7), tok = p.reverse ? p.N - 1 - pos : pos;
        raw.scale = 127;
        if ((at.lane & 7) < R && at.tile < p.tiles && at.ch / 32 < p.scale_groups && pos < p.N)  // a lane past the last channel loads for its group too
            raw.scale = in.scales[(static_cast<long long>(at.b) * p.N + tok) * p.scale_groups + at.ch / 32];
    }
}
// DECAY: what was not finite reads as -infinity, a padded token.
template <int KIND, bool DECAY = false, int R, bool PACKED>
__device__ __forceinline__ void rec_values(const RecRaw<R, PACKED>& raw, int r, int lane, f32x2 (&v)[kRecP])
{
    if constexpr (PACKED) {
        unpack8_codes4(raw.w[r][0], pack8_step(__shfl_sync(0xffffffffu, raw.scale, (lane & 24) | r)), v, DECAY ? 0xff800000u : 0x7fffffffu);
    } else {
#pragma unroll
        for (int i = 0; i < kRecP; ++i) v[i] = pack2(pair_lo<KIND>(raw.w[r][i % (PACKED ? 1 : 2)]), pair_hi<KIND>(raw.w[r][i % (PACKED ? 1 : 2)]));
    }
}
template <int KIND, int V>
__device__ __forceinline__ void rec_store(char* at, const f32x2* v)
{
    uint32_t w[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const float2 a = unpack2(v[i]);
        w[i] = pack_pair<KIND>(a.x, a.y);
    }
    if constexpr (V == 4) asm volatile("st.global.cs.v2.u32 [%0], {%1,%2};" ::"l"(at), "r"(w[0]), "r"(w[1]) : "memory");
    else asm volatile("st.global.cs.u32 [%0], %1;" ::"l"(at), "r"(w[0]) : "memory");
}
template <int V>
__device__ __forceinline__ void rec_load_floats(f32x2* v, const float* p)  // 4 V bytes on a boundary of eight
{
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const float2 t = *reinterpret_cast<const float2*>(p + 2 * i);
        v[i] = pack2(t.x, t.y);
    }
}
// Rates; a negative one counts as NaN, an infinite one as fp32's largest, so that a token that counts for nothing (rate * 0) still does.
template <int V>
__device__ __forceinline__ void rec_load_rates(f32x2* v, const float* p)
{
    rec_load_floats<V>(v, p);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const float2 t = unpack2(v[i]);
        const float nan = __uint_as_float(0x7fffffffu), most = __uint_as_float(0x7f7fffffu);
        v[i] = pack2(t.x >= 0.0f ? fminf(fabsf(t.x), most) : nan, t.y >= 0.0f ? fminf(fabsf(t.y), most) : nan);
    }
}
template <int V>
__device__ __forceinline__ void rec_store_floats(float* p, const f32x2* v)
{
#pragma unroll
    for (int i = 0; i < V / 2; ++i) *reinterpret_cast<float2*>(p + 2 * i) = unpack2(v[i]);
}


// Inclusive scan of maps over the token segments of a warp (lanes LANES apart), forward or backward in the tokens; then the
// map of what lies before the own segment.
template <int V, int LANES, bool UP>
__device__ __forceinline__ void rec_warp_scan(f32x2 (&A)[V / 2], f32x2 (&H)[V / 2], f32x2 (&Ax)[V / 2], f32x2 (&Hx)[V / 2], int lane)
{
    const int seg = lane / LANES;
    constexpr int segs = 32 / LANES;
    const auto from = [&](f32x2 x, int off) { return UP ? __shfl_up_sync(0xffffffffu, x, off) : __shfl_down_sync(0xffffffffu, x, off); };
#pragma unroll
    for (int off = 1; off < segs; off *= 2) {
        const bool in = UP ? seg >= off : seg + off < segs;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const f32x2 a = from(A[i], off * LANES), h = from(H[i], off * LANES);
            if (in) {
                H[i] = fma2(A[i], h, H[i]);
                A[i] = mul2(A[i], a);
            }
        }
    }
    const bool first = UP ? seg == 0 : seg == segs - 1;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const f32x2 a = from(A[i], LANES), h = from(H[i], LANES);
        Ax[i] = first ? both(1.0f) : a;
        Hx[i] = first ? both(0.0f) : h;
    }
}
// Per channel, the map before each warp of a tile in the place of the warp's, and the tile's.  One thread a channel.
template <bool UP, int WARPS>
__device__ __forceinline__ float2 rec_join(float2 (&totals)[WARPS][kRecSlab], int c)
{
    float2 own = make_float2(1.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
        const int w = UP ? i : WARPS - 1 - i;
        const float2 m = totals[w][c];
        totals[w][c] = own;
        own = make_float2(own.x * m.x, fmaf(m.x, own.y, m.y));
    }
    return own;
}
__device__ __forceinline__ void rec_put(float2* to, const f32x2* A, const f32x2* H)
{
#pragma unroll
    for (int i = 0; i < kRecP; ++i) {
        const float2 a = unpack2(A[i]), h = unpack2(H[i]);
        *reinterpret_cast<float4*>(to + 2 * i) = make_float4(a.x, h.x, a.y, h.y);
    }
}
// What enters the thread's segment, from what enters the tile: through the warps before, then the segments before.
__device__ __forceinline__ void rec_arrive(f32x2 (&h)[kRecP], const float2* before_warp, const float* enters, const f32x2* Ax, const f32x2* Hx)
{
#pragma unroll
    for (int i = 0; i < kRecP; ++i) {
        const float4 m = *reinterpret_cast<const float4*>(before_warp + 2 * i);
        const float2 s = *reinterpret_cast<const float2*>(enters + 2 * i);
        h[i] = fma2(Ax[i], pack2(fmaf(m.x, s.x, m.y), fmaf(m.z, s.y, m.w)), Hx[i]);
    }
}
__device__ __forceinline__ f32x2 rec_minus(f32x2 a, f32x2 b) { return fma2(b, both(-1.0f), a); }

// ------------------------------------------------------------------------------------------ maps of the tiles
// Of the state (from x, decay and gate), of the gradient (from decay and dh, backward in the tokens), or both at once.
enum : int { kRecMapState = 1, kRecMapGrad = 2, kRecMapBoth = 3 };

// The map of a tile from those of its threads' segments: those of a warp, then the warps'.  UP: in the order of the tokens.
template <bool UP, int WARPS>
__device__ __forceinline__ void rec_tile_map(f32x2 (&A)[kRecP], f32x2 (&H)[kRecP], float2 (&totals)[WARPS][kRecSlab], int lane, int warp, int cl)
{
#pragma unroll
    for (int i = 0; i < kRecP; ++i)
#pragma unroll
        for (int off = 1; off < kRecSegs; off *= 2) {
            const f32x2 a = __shfl_xor_sync(0xffffffffu, A[i], off * kRecLanes), h = __shfl_xor_sync(0xffffffffu, H[i], off * kRecLanes);
            const bool second = ((lane / kRecLanes) & off) != 0;
            H[i] = second == UP ? fma2(A[i], h, H[i]) : fma2(a, H[i], h);
            A[i] = mul2(A[i], a);
        }
    if (lane < kRecLanes) rec_put(&totals[warp][cl], A, H);
}

template <int KIND, bool GATE, bool PACKED, int WHAT>
__global__ void __launch_bounds__(kRecMapsThreads, WHAT == kRecMapBoth ? 4 : 6) recurrence_maps_kernel(const __grid_constant__ RecParams p)
{
    constexpr int R = kRecMapsR, WARPS = rec_warps(R);
    constexpr bool STATE = (WHAT & kRecMapState) != 0, GRAD = (WHAT & kRecMapGrad) != 0;
    __shared__ __align__(16) float2 totals[2][WARPS][kRecSlab];
    __shared__ __align__(16) float decays[WARPS][kRecSlab];
    const RecPlace<R> at(p);
    pdl_wait();
    pdl_launch_dependents();
    RecRaw<R, PACKED> d, x, g;
    RecRaw<R, false> y;
    rec_read(d, p.decay, p, at);
    if constexpr (GRAD) rec_read(y, p.dh, p, at);
    if constexpr (STATE) rec_read(x, p.x, p, at);
    if constexpr (STATE && GATE) rec_read(g, p.gate, p, at);
    f32x2 rate[kRecP], A[kRecP], H[kRecP], G[kRecP];
#pragma unroll
    for (int i = 0; i < kRecP; ++i) rate[i] = both(0.0f);
    if (at.ch < p.C) rec_load_rates<kRecV>(rate, p.rate + at.ch);
    const bool ragged = (at.tile + 1) * kRecEvery > p.N;
    float least = 1.0f;
    // PADDED: with regard to tokens whose other inputs must not count
    const auto pass = [&](auto wide, auto padded) {
        constexpr bool kWide = decltype(wide)::value;
        // 1 - exp(-L), or exp(-L) where WIDE: for the gradient, whose tokens come the other way.  (The sums of L are formed in one order
        // whatever is asked for, so that a pass with kept states gives the bits of one without.)
        [[maybe_unused]] f32x2 kept[R][kRecP];
#pragma unroll
        for (int i = 0; i < kRecP; ++i) A[i] = H[i] = G[i] = both(0.0f);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            [[maybe_unused]] f32x2 s[kRecP], v[kRecP], q[kRecP];
            rec_values<KIND, true>(d, r, at.lane, s);
            if constexpr (STATE) rec_values<KIND>(x, r, at.lane, v);
            if constexpr (STATE && GATE) rec_values<KIND>(g, r, at.lane, q);
#pragma unroll
            for (int i = 0; i < kRecP; ++i) {
                s[i] = sigmoid2(s[i]);
                if (ragged && r >= at.left) s[i] = both(0.0f);
                const f32x2 L = mul2(rate[i], s[i]), e = rec_decay<kWide>(L);
                A[i] = add2(A[i], L);
                if constexpr (STATE) {
                    least = rec_least(least, s[i]);
                    if constexpr (GATE) v[i] = mul2(v[i], sigmoid2(q[i]));
                    if constexpr (decltype(padded)::value) v[i] = rec_unless_padding(s[i], v[i]);
                    H[i] = fma2(e, rec_minus(v[i], H[i]), H[i]);
                }
                if constexpr (GRAD) kept[r][i] = kWide ? rec_keep(L) : e;
            }
        }
        if constexpr (GRAD) {
#pragma unroll
            for (int r = R - 1; r >= 0; --r) {
                f32x2 t[kRecP];
                rec_values<KIND>(y, r, at.lane, t);
#pragma unroll
                for (int i = 0; i < kRecP; ++i) {
                    const f32x2 sum = add2(t[i], G[i]);
                    G[i] = kWide ? mul2(kept[r][i], sum) : rec_minus(sum, mul2(kept[r][i], sum));
                }
            }
        }
    };
    if (rec_wide(rate)) {
        pass(RecBool<true>(), RecBool<true>());
    } else {
        pass(RecBool<false>(), RecBool<false>());
        if (STATE && __any_sync(0xffffffffu, least == 0.0f)) pass(RecBool<false>(), RecBool<true>());
    }
    // The tile's decay is exp(-L) of the sum over all its tokens, rounded once: a product of its sixteen segments' would be off by some units in the
    // last place of one, which is a good part of 1 - A where memories are long, and shows in the rates' gradients.
    f32x2 B[kRecP];
#pragma unroll
    for (int i = 0; i < kRecP; ++i) {
        f32x2 L = A[i];
#pragma unroll
        for (int off = kRecLanes; off < 32; off *= 2) L = add2(L, __shfl_xor_sync(0xffffffffu, L, off));
        if (at.lane < kRecLanes) *reinterpret_cast<float2*>(&decays[at.warp][at.cl + 2 * i]) = unpack2(L);
        A[i] = B[i] = rec_keep(A[i]);
    }
    if constexpr (STATE) rec_tile_map<true>(A, H, totals[0], at.lane, at.warp, at.cl);
    if constexpr (GRAD) rec_tile_map<false>(B, G, totals[1], at.lane, at.warp, at.cl);
    __syncthreads();
    const int c = threadIdx.x % kRecSlab, which = threadIdx.x / kRecSlab;
    const long long to = (static_cast<long long>(at.b) * p.tiles + at.tile) * p.width + at.slab * kRecSlab + c;
    if (at.tile >= p.tiles) return;
    float L = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) L += decays[w][c];
    const float decay = unpack2(rec_keep(both(L))).x;
    if (STATE && which == 0) p.maps[to] = make_float2(decay, rec_join<true>(totals[0], c).y);
    if (GRAD && which == 1) p.grad_maps[to] = make_float2(decay, rec_join<false>(totals[1], c).y);
}

// ------------------------------------------------------------------------------------------ from tile to tile
// What enters each tile of a channel, in the order of the tiles or (backward) from the last to the first.  A block takes 16 channels, a
// thread a run of tiles: its map, the runs' maps by doubling, then the run again.  Two such jobs may share a launch (blocks along y).
constexpr int kRecScanChannels = 16, kRecScanRuns = 64;
struct RecScan {
    const float2* maps;
    const float* first;  // what enters the first one, or null
    float* enters;
    int backward;
};
static __global__ void __launch_bounds__(kRecScanChannels* kRecScanRuns) recurrence_scan_kernel(const __grid_constant__ RecScan one, const __grid_constant__ RecScan two,
                                                                                               int tiles, int width, int C)
{
    __shared__ float2 both_runs[2][kRecScanRuns][kRecScanChannels];
    const int c = threadIdx.x % kRecScanChannels, run = threadIdx.x / kRecScanChannels, ch = static_cast<int>(blockIdx.x % (width / kRecScanChannels)) * kRecScanChannels + c,
              b = static_cast<int>(blockIdx.x / (width / kRecScanChannels));
    const RecScan& job = blockIdx.y == 0 ? one : two;
    const float2* const maps = job.maps;
    const float* const first = job.first;
    float* const enters = job.enters;
    pdl_wait();
    pdl_launch_dependents();
    const int length = (tiles + kRecScanRuns - 1) / kRecScanRuns, k0 = run * length, k1 = min(tiles, k0 + length);
    const auto tile = [&](int k) { return static_cast<long long>(b) * tiles + (job.backward ? tiles - 1 - k : k); };
    constexpr int U = 8;
    float2 m[U], own = make_float2(1.0f, 0.0f);
    for (int k = k0; k < k1; k += U) {
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (k + j < k1) m[j] = maps[tile(k + j) * width + ch];
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (k + j < k1) own = make_float2(own.x * m[j].x, fmaf(m[j].x, own.y, m[j].y));
    }
    // the runs' maps, each with all before it, by doubling
    int side = 0;
#pragma unroll
    for (int n = 1; n < kRecScanRuns; n *= 2, side ^= 1) {
        both_runs[side][run][c] = own;
        __syncthreads();
        const float2 before = both_runs[side][run >= n ? run - n : run][c];
        if (run >= n) own = make_float2(before.x * own.x, fmaf(own.x, before.y, own.y));
    }
    float2 (&runs)[kRecScanRuns][kRecScanChannels] = both_runs[side];
    runs[run][c] = own;
    __syncthreads();
    if (ch >= C) return;
    float s = first != nullptr ? first[static_cast<long long>(b) * C + ch] : 0.0f;
    if (run > 0) s = fmaf(runs[run - 1][c].x, s, runs[run - 1][c].y);
    for (int k = k0; k < k1; k += U) {
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (k + j < k1) m[j] = maps[tile(k + j) * width + ch];
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (k + j < k1) {
                enters[tile(k + j) * C + ch] = s;
                s = fmaf(m[j].x, s, m[j].y);
            }
    }
}

// ------------------------------------------------------------------------------------------ forward
template <int KIND, bool GATE>
__global__ void __launch_bounds__(kRecForwardThreads, 4) recurrence_kernel(const __grid_constant__ RecParams p)
{
    constexpr int R = kRecForwardR, WARPS = rec_warps(R);
    __shared__ __align__(16) float2 totals[WARPS][kRecSlab];
    __shared__ __align__(16) float enters[kRecSlab];
    const RecPlace<R> at(p);
    // With more than one tile the kernels before, which have waited for what was before them, write none of the inputs.
    if (p.tiles == 1) pdl_wait();
    RecRaw<R, false> x, d, g;
    rec_read(d, p.decay, p, at);
    rec_read(x, p.x, p, at);
    if constexpr (GATE) rec_read(g, p.gate, p, at);
    f32x2 rate[kRecP], e[R][kRecP], v[R][kRecP], A[kRecP], H[kRecP], Ax[kRecP], Hx[kRecP];
#pragma unroll
    for (int i = 0; i < kRecP; ++i) rate[i] = A[i] = H[i] = both(0.0f);
    if (at.ch < p.C) rec_load_rates<kRecV>(rate, p.rate + at.ch);
    const bool ragged = (at.tile + 1) * kRecEvery > p.N;
    float least = 1.0f;
    const auto gates = [&](auto wide) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            [[maybe_unused]] f32x2 s[kRecP], q[kRecP];
            rec_values<KIND, true>(d, r, at.lane, s);
            rec_values<KIND>(x, r, at.lane, v[r]);
            if constexpr (GATE) rec_values<KIND>(g, r, at.lane, q);
#pragma unroll
            for (int i = 0; i < kRecP; ++i) {
                s[i] = sigmoid2(s[i]);
                if (ragged && r >= at.left) s[i] = both(0.0f);
                const f32x2 L = mul2(rate[i], s[i]);
                A[i] = add2(A[i], L);
                e[r][i] = rec_decay<decltype(wide)::value>(L);
                least = rec_least(least, s[i]);
                if constexpr (GATE) v[r][i] = mul2(v[r][i], sigmoid2(q[i]));
            }
        }
    };
    if (rec_wide(rate)) gates(RecBool<true>());
    else gates(RecBool<false>());
    if (least == 0.0f) {  // what a padded token holds must not count; read again (nothing has been written yet): e may be zero by the rate alone
        rec_read(d, p.decay, p, at);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x2 s[kRecP];
            rec_values<KIND, true>(d, r, at.lane, s);
#pragma unroll
            for (int i = 0; i < kRecP; ++i) v[r][i] = rec_unless_padding(sigmoid2(s[i]), v[r][i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kRecP; ++i) {
#pragma unroll
        for (int r = 0; r < R; ++r) H[i] = fma2(e[r][i], rec_minus(v[r][i], H[i]), H[i]);
        A[i] = rec_keep(A[i]);
    }
    rec_warp_scan<kRecV, kRecLanes, true>(A, H, Ax, Hx, at.lane);
    if (at.lane / kRecLanes == kRecSegs - 1) rec_put(&totals[at.warp][at.cl], A, H);
    if (p.tiles > 1) pdl_wait();
    if (threadIdx.x >= kRecForwardThreads - kRecSlab) {
        const int c = threadIdx.x - (kRecForwardThreads - kRecSlab), ch = at.slab * kRecSlab + c;
        float s = 0.0f;
        if (ch < p.C && at.tile < p.tiles && p.states != nullptr) s = p.states[(static_cast<long long>(at.b) * p.tiles + at.tile) * p.C + ch];
        else if (ch < p.C && p.h0 != nullptr) s = p.h0[static_cast<long long>(at.b) * p.C + ch];
        if (ch < p.C && p.keep != nullptr) p.keep[static_cast<long long>(at.b) * p.C + ch] = s;
        enters[c] = s;
    }
    __syncthreads();
    if (threadIdx.x < kRecSlab) rec_join<true>(totals, threadIdx.x);
    __syncthreads();
    f32x2 h[kRecP];
    rec_arrive(h, &totals[at.warp][at.cl], &enters[at.cl], Ax, Hx);
    if (at.ch >= p.C || at.tile >= p.tiles) return;
    const RecRun run(p.h.p, p.h.batch, p.h.row, p, at, 2ll * at.ch);
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int i = 0; i < kRecP; ++i) h[i] = fma2(e[r][i], rec_minus(v[r][i], h[i]), h[i]);
        if (r < at.left) rec_store<KIND, kRecV>(run.at(r), h);
    }
    // tokens behind the end have left the state as it was
    if (p.last != nullptr && at.tile == p.tiles - 1 && at.warp == WARPS - 1 && at.lane / kRecLanes == kRecSegs - 1)
        rec_store_floats<kRecV>(p.last + static_cast<long long>(at.b) * p.C + at.ch, h);
}

// A few tokens (one, when a sequence is continued token by token): a thread takes two channels through all of them.  Latency.
constexpr int kRecShortThreads = 128;
template <int KIND, bool GATE>
__global__ void __launch_bounds__(kRecShortThreads) recurrence_short_kernel(const __grid_constant__ RecParams p)
{
    const long long i = static_cast<long long>(blockIdx.x) * kRecShortThreads + threadIdx.x;
    const int pairs = p.C / 2, b = static_cast<int>(i / pairs), ch = 2 * static_cast<int>(i - static_cast<long long>(b) * pairs);
    pdl_wait();
    if (b >= p.B) return;
    f32x2 rate, h = both(0.0f);
    rec_load_rates<2>(&rate, p.rate + ch);
    if (p.h0 != nullptr) rec_load_floats<2>(&h, p.h0 + static_cast<long long>(b) * p.C + ch);
    if (p.keep != nullptr) rec_store_floats<2>(p.keep + static_cast<long long>(b) * p.C + ch, &h);
    uint32_t x[kRecShort], d[kRecShort], g[kRecShort];
#pragma unroll
    for (int r = 0; r < kRecShort; ++r)
        if (r < p.N) {
            const int tok = p.reverse ? p.N - 1 - r : r;
            x[r] = *reinterpret_cast<const uint32_t*>(p.x.p + b * p.x.batch + tok * p.x.row + 2ll * ch);
            d[r] = *reinterpret_cast<const uint32_t*>(p.decay.p + b * p.decay.batch + tok * p.decay.row + 2ll * ch);
            if (GATE) g[r] = *reinterpret_cast<const uint32_t*>(p.gate.p + b * p.gate.batch + tok * p.gate.row + 2ll * ch);
        }
#pragma unroll
    for (int r = 0; r < kRecShort; ++r)
        if (r < p.N) {
            const int tok = p.reverse ? p.N - 1 - r : r;
            f32x2 v = pack2(pair_lo<KIND>(x[r]), pair_hi<KIND>(x[r]));
            if (GATE) v = mul2(v, sigmoid2(pack2(pair_lo<KIND>(g[r]), pair_hi<KIND>(g[r]))));
            const f32x2 s = sigmoid2(pack2(pair_lo<KIND>(d[r]), pair_hi<KIND>(d[r])));
            h = fma2(rec_one_minus_exp(mul2(rate, s)), fma2(h, both(-1.0f), rec_unless_padding(s, v)), h);
            rec_store<KIND, 2>(p.h.p + b * p.h.batch + tok * p.h.row + 2ll * ch, &h);
        }
    if (p.last != nullptr) rec_store_floats<2>(p.last + static_cast<long long>(b) * p.C + ch, &h);
}

// ------------------------------------------------------------------------------------------ backward
// The states inside the tile from the one that enters it, then the gradients from the last token to the first.
template <int KIND, bool GATE, bool PACKED>
__global__ void __launch_bounds__(kRecThreads, 2) recurrence_backward_kernel(const __grid_constant__ RecParams p)
{
    __shared__ __align__(16) float2 totals[2][kRecWarps][kRecSlab];
    __shared__ __align__(16) float enters[2][kRecSlab];
    const RecPlace<kRecR> at(p);
    if (p.tiles == 1) pdl_wait();
    RecRaw<kRecR, PACKED> x, d, g;
    RecRaw<kRecR, false> dh;
    rec_read(d, p.decay, p, at);
    rec_read(x, p.x, p, at);
    if constexpr (GATE) rec_read(g, p.gate, p, at);
    rec_read(dh, p.dh, p, at);
    f32x2 rate[kRecP];
#pragma unroll
    for (int i = 0; i < kRecP; ++i) rate[i] = both(0.0f);
    if (at.ch < p.C) rec_load_rates<kRecV>(rate, p.rate + at.ch);

    // exp(-decay) and exp(-gate), from which the sigmoids s and q come (again, below: both they and 1 - s, 1 - q are needed, which have no digits left
    // in the other where a gate is saturated), e, v = q x; a padded token's s, q, e and v are zero
    f32x2 odds_s[kRecR][kRecP], e[kRecR][kRecP], odds_q[kRecR][kRecP], v[kRecR][kRecP], A[kRecP], H[kRecP], G[kRecP];
#pragma unroll
    for (int i = 0; i < kRecP; ++i) A[i] = H[i] = G[i] = both(0.0f);
    const bool ragged = (at.tile + 1) * kRecEvery > p.N;
    float least = 1.0f;
    const auto gates = [&](auto wide) {
#pragma unroll
        for (int r = 0; r < kRecR; ++r) {
            [[maybe_unused]] f32x2 decay[kRecP], gate[kRecP];
            rec_values<KIND, true>(d, r, at.lane, decay);
            rec_values<KIND>(x, r, at.lane, v[r]);
            if constexpr (GATE) rec_values<KIND>(g, r, at.lane, gate);
#pragma unroll
            for (int i = 0; i < kRecP; ++i) {
                odds_s[r][i] = rec_odds(decay[i]);
                if (ragged && r >= at.left) odds_s[r][i] = both(kRecClosed);
                const f32x2 s = rec_open(odds_s[r][i]), L = mul2(rate[i], s);
                A[i] = add2(A[i], L);
                e[r][i] = decltype(wide)::value ? rec_both(L) : rec_decay<false>(L);
                least = rec_least(least, s);
                if constexpr (GATE) {
                    odds_q[r][i] = rec_odds(gate[i]);
                    v[r][i] = mul2(v[r][i], rec_open(odds_q[r][i]));
                }
            }
        }
    };
    const bool wide = rec_wide(rate);
    if (wide) gates(RecBool<true>());
    else gates(RecBool<false>());
    if (least == 0.0f)  // what a padded token holds must not count
#pragma unroll
        for (int r = 0; r < kRecR; ++r)
#pragma unroll
            for (int i = 0; i < kRecP; ++i) {
                const f32x2 s = rec_open(odds_s[r][i]);
                if constexpr (GATE) {
                    const float2 a = unpack2(s), b = unpack2(odds_q[r][i]);
                    odds_q[r][i] = pack2(a.x == 0.0f ? kRecClosed : b.x, a.y == 0.0f ? kRecClosed : b.y);
                }
                v[r][i] = rec_unless_padding(s, v[r][i]);
            }
    const auto sums = [&](auto w) {
        constexpr bool kWide = decltype(w)::value;
#pragma unroll
        for (int r = 0; r < kRecR; ++r)
#pragma unroll
            for (int i = 0; i < kRecP; ++i) H[i] = fma2(kWide ? rec_both_e(e[r][i]) : e[r][i], rec_minus(v[r][i], H[i]), H[i]);
#pragma unroll
        for (int r = kRecR - 1; r >= 0; --r) {
            f32x2 y[kRecP];
            rec_values<KIND>(dh, r, at.lane, y);
#pragma unroll
            for (int i = 0; i < kRecP; ++i) {
                const f32x2 sum = add2(y[i], G[i]);
                G[i] = kWide ? mul2(rec_both_keep(e[r][i]), sum) : rec_minus(sum, mul2(e[r][i], sum));
            }
        }
    };
    if (wide) sums(RecBool<true>());
    else sums(RecBool<false>());
    f32x2 Ar[kRecP], Axr[kRecP], Gx[kRecP], Ax[kRecP], Hx[kRecP];
#pragma unroll
    for (int i = 0; i < kRecP; ++i) Ar[i] = A[i] = rec_keep(A[i]);
    rec_warp_scan<kRecV, kRecLanes, true>(A, H, Ax, Hx, at.lane);
    rec_warp_scan<kRecV, kRecLanes, false>(Ar, G, Axr, Gx, at.lane);
    if (at.lane / kRecLanes == kRecSegs - 1) rec_put(&totals[0][at.warp][at.cl], A, H);
    if (at.lane / kRecLanes == 0) rec_put(&totals[1][at.warp][at.cl], Ar, G);
    if (p.tiles > 1) pdl_wait();
    if (threadIdx.x >= kRecThreads - 2 * kRecSlab) {
        const int i = threadIdx.x - (kRecThreads - 2 * kRecSlab), which = i / kRecSlab, c = i % kRecSlab, ch = at.slab * kRecSlab + c;
        const float *many = which == 0 ? p.states : p.grads, *one = which == 0 ? p.h0 : p.dlast;
        float t = 0.0f;
        if (ch < p.C && at.tile < p.tiles && many != nullptr) t = many[(static_cast<long long>(at.b) * p.tiles + at.tile) * p.C + ch];
        else if (ch < p.C && one != nullptr) t = one[static_cast<long long>(at.b) * p.C + ch];
        enters[which][c] = t;
    }
    __syncthreads();
    if (threadIdx.x < kRecSlab) rec_join<true>(totals[0], threadIdx.x);
    else if (threadIdx.x < 2 * kRecSlab) rec_join<false>(totals[1], threadIdx.x - kRecSlab);
    __syncthreads();
    f32x2 h[kRecP], drate[kRecP];
    rec_arrive(h, &totals[0][at.warp][at.cl], &enters[0][at.cl], Ax, Hx);
    rec_arrive(G, &totals[1][at.warp][at.cl], &enters[1][at.cl], Axr, Gx);
    // v - h_(t-1); then from the last token to the first
    f32x2 step[kRecR][kRecP];
    const RecRun run_x(p.dx.p, p.dx.batch, p.dx.row, p, at, 2ll * at.ch), run_d(p.ddecay.p, p.ddecay.batch, p.ddecay.row, p, at, 2ll * at.ch),
        run_g(p.dgate.p, p.dgate.batch, p.dgate.row, p, at, 2ll * at.ch);
    const auto gradients = [&](auto w) {
        constexpr bool kWide = decltype(w)::value;
#pragma unroll
        for (int r = 0; r < kRecR; ++r)
#pragma unroll
            for (int i = 0; i < kRecP; ++i) {
                step[r][i] = rec_minus(v[r][i], h[i]);
                h[i] = fma2(kWide ? rec_both_e(e[r][i]) : e[r][i], step[r][i], h[i]);
                drate[i] = both(0.0f);
            }
#pragma unroll
        for (int r = kRecR - 1; r >= 0; --r) {
            [[maybe_unused]] f32x2 y[kRecP], ox[kRecP], od[kRecP], og[kRecP];
            rec_values<KIND>(dh, r, at.lane, y);
#pragma unroll
            for (int i = 0; i < kRecP; ++i) {
                const f32x2 sum = add2(y[i], G[i]), dv = mul2(kWide ? rec_both_e(e[r][i]) : e[r][i], sum);
                G[i] = kWide ? mul2(rec_both_keep(e[r][i]), sum) : rec_minus(sum, dv);
                const f32x2 s = rec_open(odds_s[r][i]), dL = mul2(mul2(G[i], step[r][i]), s);  // dL sigmoid(decay)
                drate[i] = add2(drate[i], dL);
                od[i] = mul2(mul2(dL, rate[i]), mul2(odds_s[r][i], s));
                if constexpr (GATE) {
                    const f32x2 q = rec_open(odds_q[r][i]);
                    ox[i] = mul2(dv, q);
                    og[i] = mul2(mul2(dv, v[r][i]), mul2(odds_q[r][i], q));
                } else {
                    ox[i] = dv;
                }
            }
            if (r < at.left) {
                rec_store<KIND, kRecV>(run_x.at(r), ox);
                rec_store<KIND, kRecV>(run_d.at(r), od);
                if constexpr (GATE) rec_store<KIND, kRecV>(run_g.at(r), og);
            }
        }
    };
    if (wide) gradients(RecBool<true>());
    else gradients(RecBool<false>());
    if (at.ch < p.C && p.dh0 != nullptr && at.tile == 0 && at.warp == 0 && at.lane < kRecLanes)
        rec_store_floats<kRecV>(p.dh0 + static_cast<long long>(at.b) * p.C + at.ch, G);
    if (p.rate_partials != nullptr) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kRecP; ++i)
#pragma unroll
            for (int off = kRecLanes; off < 32; off *= 2) drate[i] = add2(drate[i], __shfl_xor_sync(0xffffffffu, drate[i], off));
        if (at.lane < kRecLanes) rec_put(&totals[0][at.warp][at.cl], drate, drate);
        __syncthreads();
        if (threadIdx.x < kRecSlab && at.tile < p.tiles) {
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kRecWarps; ++w) sum += totals[0][w][threadIdx.x].x;
            p.rate_partials[(static_cast<long long>(at.b) * p.tiles + at.tile) * p.width + at.slab * kRecSlab + threadIdx.x] = sum;
        }
    }
}

}  // namespace lf
