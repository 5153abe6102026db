// Kernels of include/linfusion_block.h: rotary positions with several axes, and the norms before and
// after a block with gate, modulation and residual.  All are bound by DRAM: each input is read once and
// each output written once, in 16-byte pieces; nothing is kept between calls.
#pragma once

#include "common.cuh"
#include "packed_math.cuh"

namespace lf {

// 16 bytes = eight channels of the 16-bit storage type <-> eight floats.
struct F8 {
    float v[8];
};
template <int KIND>
__device__ __forceinline__ F8 unpack8(const uint4& p)
{
    F8 f;
    f.v[0] = pair_lo<KIND>(p.x); f.v[1] = pair_hi<KIND>(p.x);
    f.v[2] = pair_lo<KIND>(p.y); f.v[3] = pair_hi<KIND>(p.y);
    f.v[4] = pair_lo<KIND>(p.z); f.v[5] = pair_hi<KIND>(p.z);
    f.v[6] = pair_lo<KIND>(p.w); f.v[7] = pair_hi<KIND>(p.w);
    return f;
}
template <int KIND>
__device__ __forceinline__ uint4 pack8(const F8& f)
{
    return make_uint4(pack_pair<KIND>(f.v[0], f.v[1]), pack_pair<KIND>(f.v[2], f.v[3]),
                      pack_pair<KIND>(f.v[4], f.v[5]), pack_pair<KIND>(f.v[6], f.v[7]));
}
// Plain (coherent) loads: outputs may lie over inputs, each element written by the thread that read it.
__device__ __forceinline__ uint4 load16(const void* p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void store16(void* p, const uint4& v)
{
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// ---------------------------------------------------------------------------------------------
// Rotary positions.  A thread owns one token and the same eight channels (interleaved) or eight pairs
// (halves) in every head of its head group, so the sines and cosines are formed once and used for all
// heads of Q and K; the loop over heads moves 16 (32) bytes each way per step, unrolled so that
// kRopeUnroll loads are in flight.
//
// The angle of a far position loses its fraction of a turn in fp32 (position 10^4 x frequency 1: 10^-3
// radians).  The frequency is therefore held in turns per position as hi + lo floats (48 bits); with
// p = pos * hi rounded and e = fma(pos, hi, -p) its exact error, p - rint(p) is exact, and
// r = (p - rint(p)) + (e + pos * lo) is the fraction of a turn to 2^-25 for angles below 2^24 radians; beyond, to 2^-48 or so of
// the turns (the 48 bits, and the last sum, whose second term then passes a turn).
// ---------------------------------------------------------------------------------------------
constexpr int kRopeMaxPairs = 128;
constexpr int kRopeThreads = 256;
struct RopeTensor {
    const char* in;
    char* out;
    int heads;
    long long in_b, in_t, in_h, out_b, out_t, out_h;  // bytes
};
struct RopeParams {
    RopeTensor t[2];
    const float* pos;
    long long pos_b;
    int N, d, P, n_axes;
    int items;           // threads of a token
    int pair_items;      // halves: those that rotate; the others copy
    int heads_per_group;
    float sign;
    float f_hi[kRopeMaxPairs], f_lo[kRopeMaxPairs];
    unsigned char axis[kRopeMaxPairs];
};

// Sine and cosine of r turns: the nearest quarter turn q is taken off exactly, the rest is at most 1/8 turn (pi / 4), where
// the Taylor series to x^9 and x^10 are off by 2e-9 and 1e-10; then q swaps and signs them.  About thirty instructions,
// fewer than sincospif takes with its own reduction (18.8 against 19.2 us for B = 3, N = 2531, 16 heads of 80, while each value
// was computed once for eight heads).
__device__ __forceinline__ void rope_sincos(float pos, float hi, float lo, float sign, float* s, float* c)
{
    const float p = pos * hi;
    const float e = fmaf(pos, hi, -p);
    const float r = (p - rintf(p)) + fmaf(pos, lo, e);
    const float q = rintf(4.0f * r);
    const float x = 6.2831853071795865f * fmaf(-0.25f, q, r), x2 = x * x;
    float u = fmaf(x2, 1.0f / 362880.0f, -1.0f / 5040.0f);
    u = fmaf(x2, u, 1.0f / 120.0f);
    u = fmaf(x2, u, -1.0f / 6.0f);
    u = fmaf(x2 * x, u, x);
    float v = fmaf(x2, -1.0f / 3628800.0f, 1.0f / 40320.0f);
    v = fmaf(x2, v, -1.0f / 720.0f);
    v = fmaf(x2, v, 1.0f / 24.0f);
    v = fmaf(x2, v, -0.5f);
    v = fmaf(x2, v, 1.0f);
    const int k = static_cast<int>(q);
    const float a = k & 1 ? v : u, b = k & 1 ? u : v;
    *s = (k & 2 ? -a : a) * sign;
    *c = (k + 1) & 2 ? -b : b;
}

constexpr int kRopeUnroll = 4;

// Eight channels in pieces of W, each at its own address.
template <int W>
__device__ __forceinline__ uint4 gather_pieces(const char* const (&p)[8 / W], long long ahead)
{
    uint32_t r[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8 / W; ++i) {
        if (W == 4) asm volatile("ld.global.v2.u32 {%0,%1}, [%2];" : "=r"(r[2 * i % 4]), "=r"(r[(2 * i + 1) % 4]) : "l"(p[i] + ahead) : "memory");
        if (W == 2) asm volatile("ld.global.u32 %0, [%1];" : "=r"(r[i % 4]) : "l"(p[i] + ahead) : "memory");
        if (W == 1) {
            unsigned short h;
            asm volatile("ld.global.u16 %0, [%1];" : "=h"(h) : "l"(p[i] + ahead) : "memory");
            r[i / 2] |= static_cast<uint32_t>(h) << (16 * (i & 1));
        }
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// PAIRS:
//   kRopeInterleaved   a thread turns the four pairs of its eight channels
//   kRopeHalves        P is a multiple of 8: a thread turns eight pairs, both sides in whole 16-byte pieces
//   W = 4, 2, 1        P is a multiple of W only: a thread makes one 16-byte piece of the output, whatever roles its
//                      channels have, from its own channels and their partners, P further or P back, which it gathers in pieces
//                      of W elements (they lie in lines that its neighbours fetch).  Stores stay whole; no warp splits into
//                      first, second and copied channels, which cost 27 us where this takes 16.5 (B = 3, N = 2531, 16 heads of 80,
//                      P = 30).  In place, the block's threads load before any of them stores: it holds whole rows.
constexpr int kRopeInterleaved = 16, kRopeHalves = 8;

template <int KIND, int PAIRS>
__global__ void __launch_bounds__(kRopeThreads, 4) rope_kernel(const __grid_constant__ RopeParams p)
{
    // The frequencies are indexed per thread: from shared memory, where lanes with different pairs do not take turns.
    __shared__ float s_hi[kRopeMaxPairs], s_lo[kRopeMaxPairs];
    __shared__ unsigned char s_axis[kRopeMaxPairs];
    for (int i = threadIdx.x; i < p.P; i += blockDim.x) {
        s_hi[i] = p.f_hi[i];
        s_lo[i] = p.f_lo[i];
        s_axis[i] = p.axis[i];
    }
    __syncthreads();
    constexpr bool GATHER = PAIRS < kRopeHalves;
    const unsigned int idx = blockIdx.x * blockDim.x + threadIdx.x;
    unsigned int n = idx / p.items;
    const int item = static_cast<int>(idx - n * p.items);
    const bool in_range = n < static_cast<unsigned int>(p.N);
    if (!GATHER && !in_range) return;
    if (!in_range) n = p.N - 1;  // takes part in the barriers only
    const int b = blockIdx.z;

    constexpr int NP = PAIRS == kRopeInterleaved ? 4 : 8;
    float sn[NP], cs[NP];
    const bool rotates = PAIRS != kRopeHalves || item < p.pair_items;
    constexpr int W = GATHER ? PAIRS : 1;
    int partner[8 / W];        // byte offsets in the row
    unsigned int copied = 0u;  // channels that pass
    if (rotates) {
        const float* pos = p.pos + static_cast<long long>(b) * p.pos_b + static_cast<long long>(n) * p.n_axes;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            int pair = item * NP + i;
            float sign = p.sign;
            if (GATHER) {
                if (pair >= 2 * p.P) copied |= 1u << i;
                // (u, w) -> (u cos - w sin, w cos + u sin): a first channel takes its partner times -sin
                if (pair < p.P) sign = -sign;
                if (i % W == 0) partner[i / W] = 2 * (pair < p.P ? pair + p.P : pair < 2 * p.P ? pair - p.P : pair);
                if (pair >= p.P) pair = pair < 2 * p.P ? pair - p.P : p.P;
            }
            sn[i] = 0.0f;
            cs[i] = 1.0f;
            if (pair < p.P) rope_sincos(pos[s_axis[pair]], s_hi[pair], s_lo[pair], sign, &sn[i], &cs[i]);
        }
    }
    const int first = blockIdx.y * p.heads_per_group;
    const int last = min(first + p.heads_per_group, p.t[0].heads + p.t[1].heads);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const RopeTensor& t = p.t[w];
        const int h0 = max(first - (w == 0 ? 0 : p.t[0].heads), 0);
        const int h1 = min(last - (w == 0 ? 0 : p.t[0].heads), t.heads);
        const char* in = t.in + b * t.in_b + n * t.in_t;
        char* out = t.out + b * t.out_b + n * t.out_t + 16 * item;
        if (GATHER) {
            constexpr int AT_ONCE = 2;  // heads; four took 128 registers and half of the occupancy
            const char* own = in + h0 * t.in_h + 16 * item;
            const char* of[8 / W];
#pragma unroll
            for (int i = 0; i < 8 / W; ++i) of[i] = in + h0 * t.in_h + partner[i];
            out += h0 * t.out_h;
            for (int h = h0; h < h1; h += AT_ONCE) {
                const bool two = h + 1 < h1;
                uint4 x[AT_ONCE], y[AT_ONCE];
                asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0].x), "=r"(x[0].y), "=r"(x[0].z), "=r"(x[0].w) : "l"(own) : "memory");
                y[0] = gather_pieces<W>(of, 0);
                if (two) {
                    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];"
                                 : "=r"(x[1].x), "=r"(x[1].y), "=r"(x[1].z), "=r"(x[1].w) : "l"(own + t.in_h) : "memory");
                    y[1] = gather_pieces<W>(of, t.in_h);
                }
                if (t.in == t.out) __syncthreads();
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j)
                    if ((j == 0 || two) && in_range) {
                        const F8 f = unpack8<KIND>(x[j]), g = unpack8<KIND>(y[j]);
                        F8 r;
#pragma unroll
                        for (int i = 0; i < 8; ++i) r.v[i] = fmaf(f.v[i], cs[i % NP], g.v[i] * sn[i % NP]);
                        if (copied != 0u) {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if ((copied >> i) & 1u) r.v[i] = f.v[i];
                        }
                        store16(out + j * t.out_h, pack8<KIND>(r));
                    }
                if (t.in == t.out) __syncthreads();
                own += 2 * t.in_h;
#pragma unroll
                for (int i = 0; i < 8 / W; ++i) of[i] += 2 * t.in_h;
                out += 2 * t.out_h;
            }
        } else if (PAIRS == kRopeInterleaved) {
            in += 16 * item;
            for (int h = h0; h < h1; h += kRopeUnroll) {
                uint4 x[kRopeUnroll];
#pragma unroll
                for (int j = 0; j < kRopeUnroll; ++j)
                    if (h + j < h1) x[j] = load16(in + (h + j) * t.in_h);
#pragma unroll
                for (int j = 0; j < kRopeUnroll; ++j)
                    if (h + j < h1) {
                        const F8 f = unpack8<KIND>(x[j]);
                        F8 r;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const bool turns = item * 4 + i < p.P;
                            r.v[2 * i] = turns ? f.v[2 * i] * cs[i] - f.v[2 * i + 1] * sn[i] : f.v[2 * i];
                            r.v[2 * i + 1] = turns ? f.v[2 * i] * sn[i] + f.v[2 * i + 1] * cs[i] : f.v[2 * i + 1];
                        }
                        store16(out + (h + j) * t.out_h, pack8<KIND>(r));
                    }
            }
        } else if (rotates) {
            const long long second = 2ll * p.P;
            in += 16 * item;
            for (int h = h0; h < h1; h += kRopeUnroll / 2) {
                uint4 x[kRopeUnroll / 2], y[kRopeUnroll / 2];
#pragma unroll
                for (int j = 0; j < kRopeUnroll / 2; ++j)
                    if (h + j < h1) {
                        x[j] = load16(in + (h + j) * t.in_h);
                        y[j] = load16(in + (h + j) * t.in_h + second);
                    }
#pragma unroll
                for (int j = 0; j < kRopeUnroll / 2; ++j)
                    if (h + j < h1) {
                        const F8 f = unpack8<KIND>(x[j]), g = unpack8<KIND>(y[j]);
                        F8 r, q;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            r.v[i] = f.v[i] * cs[i % NP] - g.v[i] * sn[i % NP];
                            q.v[i] = f.v[i] * sn[i % NP] + g.v[i] * cs[i % NP];
                        }
                        store16(out + (h + j) * t.out_h, pack8<KIND>(r));
                        store16(out + (h + j) * t.out_h + second, pack8<KIND>(q));
                    }
            }
        } else {  // channels behind the rotated ones: item counts eight-channel pieces from 2P on
            const long long at = 4ll * p.P - 16ll * p.pair_items;
            for (int h = h0; h < h1; ++h)
                store16(out + h * t.out_h + at, load16(in + h * t.in_h + at + 16 * item));
        }
    }
}

// ---------------------------------------------------------------------------------------------
// The norms around a block.  A group of W = ceil(C / (256 V)) warps works on whole rows, one at a time; each thread keeps
// to the same 8 V channels of every row, so its gate, scale, shift, weights and column sums stay in registers (V is 1 or 2).  Rows are fetched three (two) ahead into the thread's own slots of shared memory (16-byte
// asynchronous copies that only the thread itself waits for), so DRAM latency is hidden without registers.
//
// A row's mean and variance: each warp takes its sum by shuffles, then the sum of squares about its own mean, and the
// warps' (sum, squares) pairs are joined exactly:  M2 = sum_w [M2_w + n_w (mean_w - mean)^2].  Nothing cancels in them,
// whatever the row's mean; the normed value is then x rstd - mean rstd in one fma, off by the rounding of its last term (2^-24 of
// mean / deviation).  Two quantities (the two norms of a row, or two sums) travel together, one in each half of the
// warp: halving the values while the lanes are halved costs five shuffles instead of ten.
//
// What bounds them: DRAM at large C x rows, 4.9 TB/s forward and 4.3 TB/s backward of the 6.5 of a copy (68.6 and 117 us at 2 x 16384 x
// 1280, both norms with gate and modulation); behind it the latency of a row's exchanges, some 3000 clocks from its first sum to its
// last store, and the issue slots (365 instructions per row and warp in the backward pass of both norms; 560 before packed fp32x2
// arithmetic, which halves the multiply-adds).  More rows in flight would take registers: 96 of them for a fourth block
// spilled (177 us where 128 take 117).
// ---------------------------------------------------------------------------------------------
constexpr int kNormNone = 0, kNormLayer = 1, kNormRms = 2;
constexpr int kNormMaxWarps = 16;  // of a group: a half warp holds one value of each
constexpr int kNormMaxThreads = 32 * kNormMaxWarps;  // which leaves a thread 128 registers: three blocks of five warps on an SM
// Most threads of a block whose groups have one warp (J = 0) or more.
__host__ __device__ constexpr int norm_threads(int V, int J) { return V > 1 && J == 0 ? 128 : kNormMaxThreads; }
__host__ __device__ constexpr int norm_stages(int V) { return V == 1 ? 4 : 3; }

struct Rows {
    char* p;
    long long b, r;  // bytes
};
struct Channels {
    const char* p;
    long long b;
};
struct NormParams {
    Rows x, a, y, n;         // forward: x, a -> y, n.   backward: x holds y
    Rows dy, dn, dx, da;     // backward
    Channels gate, scale, shift;
    const char *pre_w, *pre_b, *post_w, *post_b;
    int N, C;
    int warps;               // of a group
    int chunks;              // groups of a batch entry
    int groups;              // all
    float eps, rs, inv_c;
    float inv_last, last;    // channels of a group's last warp, and 1 / them
    float* partials;         // backward: [sums][group][C]
    int want;                // backward: bit k set where column sum k is wanted
};

// Eight channels as four pairs.
struct P8 {
    f32x2 v[4];
};
template <int KIND>
__device__ __forceinline__ P8 unpack_pairs(const uint4& p)
{
    P8 f;
    f.v[0] = pack2(pair_lo<KIND>(p.x), pair_hi<KIND>(p.x));
    f.v[1] = pack2(pair_lo<KIND>(p.y), pair_hi<KIND>(p.y));
    f.v[2] = pack2(pair_lo<KIND>(p.z), pair_hi<KIND>(p.z));
    f.v[3] = pack2(pair_lo<KIND>(p.w), pair_hi<KIND>(p.w));
    return f;
}
template <int KIND>
__device__ __forceinline__ uint4 pack_pairs(const P8& f)
{
    const float2 a = unpack2(f.v[0]), b = unpack2(f.v[1]), c = unpack2(f.v[2]), d = unpack2(f.v[3]);
    return make_uint4(pack_pair<KIND>(a.x, a.y), pack_pair<KIND>(b.x, b.y), pack_pair<KIND>(c.x, c.y), pack_pair<KIND>(d.x, d.y));
}
template <int KIND>
__device__ __forceinline__ P8 load_vector(const char* p, int c, bool active, float absent)
{
    P8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = both(active ? absent : 0.0f);
    if (p != nullptr && active) f = unpack_pairs<KIND>(load16(p + 2 * c));
    return f;
}

__device__ __forceinline__ void group_sync(int group_in_cta, int warps)
{
    if (warps > 1) asm volatile("bar.sync %0, %1;" ::"r"(group_in_cta + 1), "r"(warps * 32) : "memory");
}
// Sums over the warp of two values: lanes 0 - 15 end with the first's, 16 - 31 with the second's.
__device__ __forceinline__ float fold(float a, float b, int lane)
{
    const bool second = lane >= 16;
    float k = second ? b : a;
    k += __shfl_xor_sync(0xffffffffu, second ? a : b, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) k += __shfl_xor_sync(0xffffffffu, k, o);
    return k;
}
__device__ __forceinline__ float from_first(float v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ float from_second(float v) { return __shfl_sync(0xffffffffu, v, 16); }

// What a thread is in its group, and the group's exchange of one pair of numbers per warp and half.  The two buffers
// take turns: a buffer is written again only behind the barrier of the exchange in between, which every warp
// reaches after it has read.  J: steps that join the warps' values, 2^J >= W (0: the group is one warp).
template <int J>
struct Group {
    float2* buf;  // [2][32]
    int turn, warp, lane, g;
    __device__ __forceinline__ float2 swap(float2 mine, const NormParams& p)
    {
        float2* b = buf + turn;
        turn ^= 32;
        if ((lane & 15) == 0) b[lane + warp] = mine;
        group_sync(g, p.warps);
        return (lane & 15) < p.warps ? b[lane] : make_float2(0.0f, 0.0f);
    }
    __device__ __forceinline__ float join(float v) const
    {
#pragma unroll
        for (int o = 1 << J >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
};
struct Stats {
    float mean, rstd;
};

// Mean (0 for RMS) and 1 / sqrt(var + eps) of one row of `a` and one of `b`, each of its norm (kNormNone: not wanted).
// Lanes without channels hold zeros, and take a mean of zero when deviations are formed.
template <int NA, int NB, int V, int J>
__device__ __forceinline__ void two_stats(const P8 (&a)[V], const P8 (&b)[V], const bool (&active)[V], const NormParams& p,
                                          Group<J>& g, Stats* sa, Stats* sb)
{
    float m = 0.0f, sum = 0.0f;
    if (NA == kNormLayer || NB == kNormLayer) {
        f32x2 ta = both(0.0f), tb = both(0.0f);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (NA == kNormLayer) ta = i + v == 0 ? a[v].v[i] : add2(ta, a[v].v[i]);
                if (NB == kNormLayer) tb = i + v == 0 ? b[v].v[i] : add2(tb, b[v].v[i]);
            }
        sum = fold(NA == kNormLayer ? sum2(ta) : 0.0f, NB == kNormLayer ? sum2(tb) : 0.0f, g.lane);
        m = sum * (J == 0 ? p.inv_c : g.warp == p.warps - 1 ? p.inv_last : 1.0f / (256 * V));
    }
    const float ma = NA == kNormLayer ? -from_first(m) : 0.0f, mb = NB == kNormLayer ? -from_second(m) : 0.0f;
    f32x2 qa = both(0.0f), qb = both(0.0f);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const f32x2 va = both(active[v] ? ma : 0.0f), vb = both(active[v] ? mb : 0.0f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (NA != kNormNone) {
                const f32x2 d = NA == kNormLayer ? add2(a[v].v[i], va) : a[v].v[i];
                qa = i + v == 0 ? mul2(d, d) : fma2(d, d, qa);
            }
            if (NB != kNormNone) {
                const f32x2 d = NB == kNormLayer ? add2(b[v].v[i], vb) : b[v].v[i];
                qb = i + v == 0 ? mul2(d, d) : fma2(d, d, qb);
            }
        }
    }
    float sq = fold(NA != kNormNone ? sum2(qa) : 0.0f, NB != kNormNone ? sum2(qb) : 0.0f, g.lane);
    if (J > 0) {
        const float2 o = g.swap(make_float2(sum, sq), p);
        sq = o.y;
        if (NA == kNormLayer || NB == kNormLayer) {
            // a half whose norm is RMS has sums of zero: its mean stays zero and nothing is added
            m = g.join(o.x) * p.inv_c;
            const int w = g.lane & 15;
            const bool full = w < p.warps - 1;
            const float d = o.x * (full ? 1.0f / (256 * V) : p.inv_last) - m;
            if (w < p.warps) sq = fmaf((full ? 256.0f * V : p.last) * d, d, sq);
        }
        sq = g.join(sq);
    }
    const float rs = rsqrtf(fmaf(sq, p.inv_c, p.eps));
    if (NA != kNormNone) sa->mean = NA == kNormLayer ? from_first(m) : 0.0f, sa->rstd = from_first(rs);
    if (NB != kNormNone) sb->mean = NB == kNormLayer ? from_second(m) : 0.0f, sb->rstd = from_second(rs);
}

// Means over the row of two values.
template <int J>
__device__ __forceinline__ float2 two_means(f32x2 u, f32x2 w, const NormParams& p, Group<J>& g)
{
    float v = fold(sum2(u), sum2(w), g.lane);
    if (J > 0) v = g.join(g.swap(make_float2(v, 0.0f), p).x);
    v *= p.inv_c;
    return make_float2(from_first(v), from_second(v));
}

// Which rows of which batch entry a group works on: contiguous runs of near-equal length.
struct GroupRows {
    int b, begin, end;
};
__device__ __forceinline__ GroupRows group_rows(const NormParams& p, int group)
{
    GroupRows r;
    r.b = group / p.chunks;
    const long long c = group - r.b * p.chunks;
    r.begin = static_cast<int>(c * p.N / p.chunks);
    r.end = static_cast<int>((c + 1) * p.N / p.chunks);
    return r;
}

__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// The thread's slots of S streams x V vectors x STAGES rows: [stage][warp][stream][vector][lane], so that a slot is the
// stage's address plus a constant.  Slots of lanes without channels, and of streams that are absent, hold zeros.
template <int S, int V>
struct RowRing {
    static constexpr int STAGES = norm_stages(V), SLOT = 512;
    uint32_t first, pitch, read_at, fill_at;
    __device__ __forceinline__ void begin(uint32_t base)
    {
        pitch = blockDim.x * (16 * S * V);
        first = base + (threadIdx.x / 32) * (S * V * SLOT) + (threadIdx.x & 31) * 16;
        read_at = fill_at = first;
        for (int i = 0; i < STAGES; ++i)
#pragma unroll
            for (int s = 0; s < S * V; ++s)
                asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(first + i * pitch + s * SLOT), "r"(0u) : "memory");
    }
    __device__ __forceinline__ uint32_t next(uint32_t at) const
    {
        const uint32_t n = at + pitch;
        return n == first + STAGES * pitch ? first : n;
    }
    __device__ __forceinline__ void fill(int s, int v, const char* src) const
    {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(fill_at + (s * V + v) * SLOT), "l"(src) : "memory");
    }
    __device__ __forceinline__ uint4 read(int s, int v) const
    {
        uint4 r;
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(read_at + (s * V + v) * SLOT) : "memory");
        return r;
    }
};
__host__ __device__ constexpr int norm_smem_bytes(int streams, int V, int threads, int groups) { return groups * 64 * 8 + norm_stages(V) * streams * V * threads * 16; }

// Rows handed from one to the next by their stride.
struct Walk {
    char* p;
    long long r;
    __device__ __forceinline__ Walk(const Rows& t, const GroupRows& rows, int c)
        : p(t.p == nullptr ? nullptr : t.p + rows.b * t.b + rows.begin * t.r + 2 * c), r(t.r) {}
    __device__ __forceinline__ void step() { p += r; }
};

template <int KIND, int POST, int PRE, bool A, int V, int J>
__global__ void __launch_bounds__(norm_threads(V, J)) block_norm_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ __align__(16) unsigned char norm_smem[];
    constexpr int S = A ? 2 : 1;
    const int per_cta = J == 0 ? blockDim.x / 32 : blockDim.x / (32 * p.warps), g = J == 0 ? threadIdx.x / 32 : threadIdx.x / (32 * p.warps);
    const int group = blockIdx.x * per_cta + g;
    if (group >= p.groups) return;
    Group<J> me = {reinterpret_cast<float2*>(norm_smem) + g * 64, 0, static_cast<int>(threadIdx.x / 32) - g * (J == 0 ? 1 : p.warps),
                   static_cast<int>(threadIdx.x & 31), g};
    RowRing<S, V> ring;
    ring.begin(smem_u32(norm_smem) + per_cta * 64 * 8);
    // vector v of the thread: channels 256 (V warp + v) + 8 lane ..
    const int c0 = 256 * V * me.warp + 8 * me.lane;
    bool active[V];
#pragma unroll
    for (int v = 0; v < V; ++v) active[v] = c0 + 256 * v < p.C;
    const GroupRows rows = group_rows(p, group);

    Walk x(p.x, rows, c0), a(p.a, rows, c0), y(p.y, rows, c0), n(p.n, rows, c0);
    int to_fetch = rows.end - rows.begin;
    auto fetch = [&]() {
        if (to_fetch > 0) {
            --to_fetch;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (active[v]) {
                    ring.fill(0, v, x.p + 512 * v);
                    if (A) ring.fill(S - 1, v, a.p + 512 * v);
                }
            ring.fill_at = ring.next(ring.fill_at);
            x.step();
            if (A) a.step();
        }
        copies_commit();
    };
#pragma unroll
    for (int i = 0; i < norm_stages(V) - 1; ++i) fetch();

    // y = rs x + (h Ap + Bp);  n = h An + Bn
    P8 Ap[V], Bp[V], An[V], Bn[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = c0 + 256 * v;
        if (A) {
            const P8 gate = load_vector<KIND>(p.gate.p == nullptr ? nullptr : p.gate.p + rows.b * p.gate.b, c, active[v], 1.0f);
            Ap[v] = load_vector<KIND>(p.post_w, c, active[v], 1.0f);
            Bp[v] = load_vector<KIND>(p.post_b, c, active[v], 0.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) Ap[v].v[i] = mul2(Ap[v].v[i], gate.v[i]), Bp[v].v[i] = mul2(Bp[v].v[i], gate.v[i]);
        }
        if (PRE != kNormNone) {
            const P8 scale = load_vector<KIND>(p.scale.p == nullptr ? nullptr : p.scale.p + rows.b * p.scale.b, c, active[v], 0.0f);
            const P8 shift = load_vector<KIND>(p.shift.p == nullptr ? nullptr : p.shift.p + rows.b * p.shift.b, c, active[v], 0.0f);
            An[v] = load_vector<KIND>(p.pre_w, c, active[v], 1.0f);
            Bn[v] = load_vector<KIND>(p.pre_b, c, active[v], 0.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x2 s = add2(scale.v[i], both(1.0f));
                An[v].v[i] = mul2(An[v].v[i], s);
                Bn[v].v[i] = fma2(Bn[v].v[i], s, shift.v[i]);
            }
        }
    }
    const f32x2 rs = both(p.rs);
    for (int left = rows.end - rows.begin; left > 0; --left) {
        copies_wait<norm_stages(V) - 2>();
        P8 s[V], h[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            s[v] = unpack_pairs<KIND>(ring.read(0, v));
            if (A) h[v] = unpack_pairs<KIND>(ring.read(S - 1, v));
        }
        ring.read_at = ring.next(ring.read_at);
        fetch();  // into the slots of the row before, which has been read
        Stats st = {0.0f, 1.0f};
        if (A) {
            if (POST != kNormNone) two_stats<POST, kNormNone, V, J>(h, h, active, p, me, &st, nullptr);
            const f32x2 r = both(st.rstd), m = both(-st.mean * st.rstd);
#pragma unroll
            for (int v = 0; v < V; ++v) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x2 e = POST == kNormNone ? h[v].v[i] : POST == kNormRms ? mul2(h[v].v[i], r) : fma2(h[v].v[i], r, m);
                    s[v].v[i] = fma2(rs, s[v].v[i], fma2(e, Ap[v].v[i], Bp[v].v[i]));
                }
                const uint4 stored = pack_pairs<KIND>(s[v]);
                if (active[v]) store16(y.p + 512 * v, stored);
                if (PRE != kNormNone) s[v] = unpack_pairs<KIND>(stored);  // the norm below is that of the stored stream
            }
            y.step();
        }
        if (PRE != kNormNone) {
            two_stats<PRE, kNormNone, V, J>(s, s, active, p, me, &st, nullptr);
            const f32x2 r = both(st.rstd), m = both(-st.mean * st.rstd);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                P8 o;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    o.v[i] = fma2(PRE == kNormRms ? mul2(s[v].v[i], r) : fma2(s[v].v[i], r, m), An[v].v[i], Bn[v].v[i]);
                if (active[v]) store16(n.p + 512 * v, pack_pairs<KIND>(o));
            }
            n.step();
        }
    }
}

// Backward.  With h = Pre(y), e = Post(a), g = dn * (1 + scale) * pre_weight and u the gradient of y:
//     u  = dy + rstd_y (g - mean(g) - h mean(g h))          (no mean(g) for the RMS norm)
//     dx = rs u,   w = u * gate * post_weight,   da = rstd_a (w - mean(w) - e mean(w e))
// and every vector's gradient follows from four column sums over a batch entry's rows:
//     [0] sum dn   [1] sum dn h   [2] sum u e   [3] sum u
// which the group keeps in registers over its rows and leaves as partials for block_norm_grads_kernel.
template <int KIND, int POST, int PRE, bool A, int V, int J>
__global__ void __launch_bounds__(norm_threads(V, J)) block_norm_backward_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ __align__(16) unsigned char norm_smem[];
    constexpr int S = (PRE != kNormNone ? 2 : 0) + (A ? 2 : 1);
    constexpr int kY = 0, kDn = 1, kDy = PRE != kNormNone ? 2 : 0, kA = S - 1;
    const int per_cta = J == 0 ? blockDim.x / 32 : blockDim.x / (32 * p.warps), g = J == 0 ? threadIdx.x / 32 : threadIdx.x / (32 * p.warps);
    const int group = blockIdx.x * per_cta + g;
    if (group >= p.groups) return;
    Group<J> me = {reinterpret_cast<float2*>(norm_smem) + g * 64, 0, static_cast<int>(threadIdx.x / 32) - g * (J == 0 ? 1 : p.warps),
                   static_cast<int>(threadIdx.x & 31), g};
    RowRing<S, V> ring;
    ring.begin(smem_u32(norm_smem) + per_cta * 64 * 8);
    const int c0 = 256 * V * me.warp + 8 * me.lane;
    bool active[V];
#pragma unroll
    for (int v = 0; v < V; ++v) active[v] = c0 + 256 * v < p.C;
    const GroupRows rows = group_rows(p, group);
    const bool has_dy = p.dy.p != nullptr;
    Walk y(p.x, rows, c0), a(p.a, rows, c0), dy(p.dy, rows, c0), dnw(p.dn, rows, c0), dx(p.dx, rows, c0), da(p.da, rows, c0);
    int to_fetch = rows.end - rows.begin;
    auto fetch = [&]() {
        if (to_fetch > 0) {
            --to_fetch;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (active[v]) {
                    if (PRE != kNormNone) ring.fill(kY, v, y.p + 512 * v);
                    if (PRE != kNormNone) ring.fill(kDn, v, dnw.p + 512 * v);
                    if (has_dy) ring.fill(kDy, v, dy.p + 512 * v);
                    if (A) ring.fill(kA, v, a.p + 512 * v);
                }
            ring.fill_at = ring.next(ring.fill_at);
            if (PRE != kNormNone) y.step(), dnw.step();
            if (has_dy) dy.step();
            if (A) a.step();
        }
        copies_commit();
    };
#pragma unroll
    for (int i = 0; i < norm_stages(V) - 1; ++i) fetch();

    P8 Ap[V], An[V], sum[4][V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = c0 + 256 * v;
        if (A) {
            const P8 gate = load_vector<KIND>(p.gate.p == nullptr ? nullptr : p.gate.p + rows.b * p.gate.b, c, active[v], 1.0f);
            Ap[v] = load_vector<KIND>(p.post_w, c, active[v], 1.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) Ap[v].v[i] = mul2(Ap[v].v[i], gate.v[i]);
        }
        if (PRE != kNormNone) {
            const P8 scale = load_vector<KIND>(p.scale.p == nullptr ? nullptr : p.scale.p + rows.b * p.scale.b, c, active[v], 0.0f);
            An[v] = load_vector<KIND>(p.pre_w, c, active[v], 1.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) An[v].v[i] = mul2(An[v].v[i], add2(scale.v[i], both(1.0f)));
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[k][v].v[i] = both(0.0f);
    }
    const f32x2 rs = both(p.rs), zero = both(0.0f);
    for (int left = rows.end - rows.begin; left > 0; --left) {
        copies_wait<norm_stages(V) - 2>();
        P8 h[V], dn[V], u[V], e[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (PRE != kNormNone) h[v] = unpack_pairs<KIND>(ring.read(kY, v));
            if (A) e[v] = unpack_pairs<KIND>(ring.read(kA, v));
        }
        Stats sy = {0.0f, 1.0f}, sa = {0.0f, 1.0f};
        if (PRE != kNormNone || (A && POST != kNormNone)) two_stats<PRE, A ? POST : kNormNone, V, J>(h, e, active, p, me, &sy, &sa);
        if (PRE != kNormNone) {
            const f32x2 r = both(sy.rstd);
            f32x2 m1 = zero, m2 = zero;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const f32x2 m = both(active[v] ? -sy.mean * sy.rstd : 0.0f);
                dn[v] = unpack_pairs<KIND>(ring.read(kDn, v));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    h[v].v[i] = PRE == kNormRms ? mul2(h[v].v[i], r) : fma2(h[v].v[i], r, m);
                    sum[0][v].v[i] = add2(sum[0][v].v[i], dn[v].v[i]);
                    sum[1][v].v[i] = fma2(dn[v].v[i], h[v].v[i], sum[1][v].v[i]);
                    dn[v].v[i] = mul2(dn[v].v[i], An[v].v[i]);
                    if (PRE == kNormLayer) m1 = i + v == 0 ? dn[v].v[i] : add2(m1, dn[v].v[i]);
                    m2 = i + v == 0 ? mul2(dn[v].v[i], h[v].v[i]) : fma2(dn[v].v[i], h[v].v[i], m2);
                }
            }
            const float2 b = two_means<J>(m1, m2, p, me);
            const f32x2 b1 = both(-sy.rstd * b.x), b2 = both(-sy.rstd * b.y);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                u[v] = unpack_pairs<KIND>(ring.read(kDy, v));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x2 k = PRE == kNormLayer ? fma2(h[v].v[i], b2, b1) : mul2(h[v].v[i], b2);
                    u[v].v[i] = add2(u[v].v[i], fma2(r, dn[v].v[i], k));
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) u[v] = unpack_pairs<KIND>(ring.read(kDy, v));
        }
        ring.read_at = ring.next(ring.read_at);
        fetch();  // into the slots of the row before
#pragma unroll
        for (int v = 0; v < V; ++v) {
            P8 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o.v[i] = mul2(rs, u[v].v[i]);
            if (active[v]) store16(dx.p + 512 * v, pack_pairs<KIND>(o));
        }
        dx.step();
        if (A) {
            const f32x2 r = both(sa.rstd);
            f32x2 m1 = zero, m2 = zero;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const f32x2 m = both(-sa.mean * sa.rstd);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (POST != kNormNone) e[v].v[i] = POST == kNormRms ? mul2(e[v].v[i], r) : fma2(e[v].v[i], r, m);
                    sum[2][v].v[i] = fma2(u[v].v[i], e[v].v[i], sum[2][v].v[i]);
                    sum[3][v].v[i] = add2(sum[3][v].v[i], u[v].v[i]);
                    u[v].v[i] = mul2(u[v].v[i], Ap[v].v[i]);  // zero where the lane has no channels
                    if (POST == kNormLayer) m1 = i + v == 0 ? u[v].v[i] : add2(m1, u[v].v[i]);
                    if (POST != kNormNone) m2 = i + v == 0 ? mul2(u[v].v[i], e[v].v[i]) : fma2(u[v].v[i], e[v].v[i], m2);
                }
            }
            f32x2 b1 = zero, b2 = zero;
            if (POST != kNormNone) {
                const float2 b = two_means<J>(m1, m2, p, me);
                b1 = both(-sa.rstd * b.x);
                b2 = both(-sa.rstd * b.y);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (POST != kNormNone) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        u[v].v[i] = fma2(r, u[v].v[i], POST == kNormLayer ? fma2(e[v].v[i], b2, b1) : mul2(e[v].v[i], b2));
                }
                if (active[v]) store16(da.p + 512 * v, pack_pairs<KIND>(u[v]));
            }
            da.step();
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if ((p.want >> k) & 1)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (active[v]) {
                    float4* to = reinterpret_cast<float4*>(p.partials + (static_cast<size_t>(k) * p.groups + group) * p.C + c0 + 256 * v);
                    const float2 q0 = unpack2(sum[k][v].v[0]), q1 = unpack2(sum[k][v].v[1]), q2 = unpack2(sum[k][v].v[2]),
                                 q3 = unpack2(sum[k][v].v[3]);
                    to[0] = make_float4(q0.x, q0.y, q1.x, q1.y);
                    to[1] = make_float4(q2.x, q2.y, q3.x, q3.y);
                }
    pdl_launch_dependents();
}

// Second stage: the column sums in a fixed order, and from them the vectors' gradients.  grid.y = 0 sums over all batch
// entries (gradients of weights, biases and shared vectors), grid.y = 1 + b over entry b (vectors of its own).  A block takes
// eight channels (one 32-byte sector of each partial: enough blocks for the narrow rows too): two threads of four channels,
// 128 slices of the groups; a slice adds its groups in order, the slices are added in a fixed tree.
struct NormGradParams {
    const float* partials;
    int B, C, chunks, groups, want;
    Channels gate, scale;
    const char *pre_w, *pre_b, *post_w, *post_b;
    int gate_per_batch, scale_per_batch, shift_per_batch;
    float *d_gate, *d_scale, *d_shift, *d_pre_w, *d_pre_b, *d_post_w, *d_post_b;
};
constexpr int kNormGradThreads = 256, kNormGradChannels = 8;

template <int KIND>
__device__ __forceinline__ float channel(const char* p, int c, float absent)
{
    if (p == nullptr) return absent;
    const uint32_t h = *reinterpret_cast<const unsigned short*>(p + 2 * c);
    return pair_lo<KIND>(h);
}

template <int KIND>
__global__ void __launch_bounds__(kNormGradThreads) block_norm_grads_kernel(const __grid_constant__ NormGradParams p)
{
    constexpr int WARPS = kNormGradThreads / 32, SLICES = kNormGradThreads / 2, CH = kNormGradChannels;
    __shared__ float s[8][WARPS][CH];
    const int column = threadIdx.x & 1, slice = threadIdx.x / 2, warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const int c = blockIdx.x * CH + column * 4;
    const bool all = blockIdx.y == 0;
    const int first = all ? 0 : (blockIdx.y - 1) * p.chunks, last = all ? p.groups : first + p.chunks;
    // [0 .. 3]: the column sums; [4 .. 7], over all entries: weighted by 1 + scale (dn, dn h) and by the gate (u e, u)
    float acc[8][4] = {};
    pdl_wait();
    {
        const bool weighted = all && (p.scale.p != nullptr || p.gate.p != nullptr);
        for (int i = first + slice; i < last; i += SLICES) {
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                v[k] = ((p.want >> k) & 1) ? *reinterpret_cast<const float4*>(p.partials + (static_cast<size_t>(k) * p.groups + i) * p.C + c)
                                           : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            float sc[4] = {1.0f, 1.0f, 1.0f, 1.0f}, gt[4] = {1.0f, 1.0f, 1.0f, 1.0f};
            if (weighted) {
                const int b = i / p.chunks;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    sc[j] = 1.0f + channel<KIND>(p.scale.p == nullptr ? nullptr : p.scale.p + b * p.scale.b, c + j, 0.0f);
                    gt[j] = channel<KIND>(p.gate.p == nullptr ? nullptr : p.gate.p + b * p.gate.b, c + j, 1.0f);
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float x[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    acc[k][j] += x[j];
                    acc[k + 4][j] = fmaf(k < 2 ? sc[j] : gt[j], x[j], acc[k + 4][j]);
                }
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int o = 2; o < 32; o <<= 1) acc[k][j] += __shfl_xor_sync(0xffffffffu, acc[k][j], o);
            if (lane < 2) s[k][warp][column * 4 + j] = acc[k][j];
        }
    __syncthreads();
    if (threadIdx.x < 8 * CH) {
        const int k = threadIdx.x / CH, j = threadIdx.x % CH;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) v += s[k][w][j];
        s[k][0][j] = v;
    }
    __syncthreads();
    const int ch = blockIdx.x * CH + threadIdx.x;
    if (threadIdx.x >= CH) return;
    const float dn = s[0][0][lane], dnh = s[1][0][lane], ue = s[2][0][lane], u = s[3][0][lane];
    const float d_scale = channel<KIND>(p.pre_w, ch, 1.0f) * dnh + channel<KIND>(p.pre_b, ch, 0.0f) * dn;
    const float d_gate = channel<KIND>(p.post_w, ch, 1.0f) * ue + channel<KIND>(p.post_b, ch, 0.0f) * u;
    const size_t at = (all ? 0 : static_cast<size_t>(blockIdx.y - 1) * p.C) + ch;
    if (p.d_shift != nullptr && all != (p.shift_per_batch != 0)) p.d_shift[at] = dn;
    if (p.d_scale != nullptr && all != (p.scale_per_batch != 0)) p.d_scale[at] = d_scale;
    if (p.d_gate != nullptr && all != (p.gate_per_batch != 0)) p.d_gate[at] = d_gate;
    if (!all) return;
    if (p.d_pre_b != nullptr) p.d_pre_b[ch] = s[4][0][lane];
    if (p.d_pre_w != nullptr) p.d_pre_w[ch] = s[5][0][lane];
    if (p.d_post_w != nullptr) p.d_post_w[ch] = s[6][0][lane];
    if (p.d_post_b != nullptr) p.d_post_b[ch] = s[7][0][lane];
}

}  // namespace lf
