// Kernels of include/linfusion_block.h: rotary positions with several axes, and the norms before and
// after a block with gate, modulation and residual.  All are bound by DRAM: each input is read once and
// each output written once, in 16-byte pieces; nothing is kept between calls.
#pragma once

#include "common.cuh"

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
// r = (p - rint(p)) + (e + pos * lo) is the fraction of a turn to 2^-25.
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

__device__ __forceinline__ void rope_sincos(float pos, float hi, float lo, float sign, float* s, float* c)
{
    const float p = pos * hi;
    const float e = fmaf(pos, hi, -p);
    const float r = (p - rintf(p)) + fmaf(pos, lo, e);
    sincospif(2.0f * r, s, c);
    *s *= sign;
}

// Eight 16-bit values at an address that is aligned to W elements only: pieces of W, those that begin before
// element `end` (counted from the address).
template <int W>
__device__ __forceinline__ uint4 load_pieces(const char* p, int end)
{
    if (W == 8) return load16(p);
    uint32_t r[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; i += W) {
        if (i >= end) break;
        if (W == 4) asm volatile("ld.global.v2.u32 {%0,%1}, [%2];" : "=r"(r[i / 2]), "=r"(r[i / 2 + 1]) : "l"(p + 2 * i) : "memory");
        if (W == 2) asm volatile("ld.global.u32 %0, [%1];" : "=r"(r[i / 2]) : "l"(p + 2 * i) : "memory");
        if (W == 1) {
            unsigned short h;
            asm volatile("ld.global.u16 %0, [%1];" : "=h"(h) : "l"(p + 2 * i) : "memory");
            r[i / 2] |= static_cast<uint32_t>(h) << (16 * (i & 1));
        }
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}
template <int W>
__device__ __forceinline__ void store_pieces(char* p, const uint4& v, int end)
{
    if (W == 8) {
        store16(p, v);
        return;
    }
    const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; i += W) {
        if (i >= end) break;
        if (W == 4) asm volatile("st.global.v2.u32 [%0], {%1,%2};" ::"l"(p + 2 * i), "r"(r[i / 2]), "r"(r[i / 2 + 1]) : "memory");
        if (W == 2) asm volatile("st.global.u32 [%0], %1;" ::"l"(p + 2 * i), "r"(r[i / 2]) : "memory");
        if (W == 1)
            asm volatile("st.global.u16 [%0], %1;" ::"l"(p + 2 * i), "h"(static_cast<unsigned short>(r[i / 2] >> (16 * (i & 1)))) : "memory");
    }
}

constexpr int kRopeUnroll = 4;

// W: alignment in elements of channel P, where the second halves of the pairs begin (8 where P is a multiple of
// 8: whole 16-byte pieces); INTERLEAVED needs none.  Pieces of 4, 2 or 1 keep the same sectors in use and
// cost load and store instructions only.
template <int KIND, bool INTERLEAVED, int W>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeParams p)
{
    // The frequencies are indexed per thread: from shared memory, where lanes with different pairs do not take turns.
    __shared__ float s_hi[kRopeMaxPairs], s_lo[kRopeMaxPairs];
    __shared__ unsigned char s_axis[kRopeMaxPairs];
    if (threadIdx.x < kRopeMaxPairs) {
        s_hi[threadIdx.x] = p.f_hi[threadIdx.x];
        s_lo[threadIdx.x] = p.f_lo[threadIdx.x];
        s_axis[threadIdx.x] = p.axis[threadIdx.x];
    }
    __syncthreads();
    const unsigned int idx = blockIdx.x * kRopeThreads + threadIdx.x;
    const unsigned int n = idx / p.items;
    const int item = static_cast<int>(idx - n * p.items);
    if (n >= static_cast<unsigned int>(p.N)) return;
    const int b = blockIdx.z;

    constexpr int NP = INTERLEAVED ? 4 : 8;
    float sn[NP], cs[NP];
    const bool rotates = INTERLEAVED || item < p.pair_items;
    if (rotates) {
        const float* pos = p.pos + static_cast<long long>(b) * p.pos_b + static_cast<long long>(n) * p.n_axes;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int pair = item * NP + i;
            sn[i] = 0.0f;
            cs[i] = 1.0f;
            if (pair < p.P) rope_sincos(pos[s_axis[pair]], s_hi[pair], s_lo[pair], p.sign, &sn[i], &cs[i]);
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
        char* out = t.out + b * t.out_b + n * t.out_t;
        if (INTERLEAVED) {
            in += 16 * item;
            out += 16 * item;
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
                            r.v[2 * i] = f.v[2 * i] * cs[i] - f.v[2 * i + 1] * sn[i];
                            r.v[2 * i + 1] = f.v[2 * i] * sn[i] + f.v[2 * i + 1] * cs[i];
                        }
                        store16(out + (h + j) * t.out_h, pack8<KIND>(r));
                    }
            }
        } else if (rotates) {
            const int end = p.P - 8 * item;  // pairs left from this item's first on
            const long long second = 2ll * p.P;
            in += 16 * item;
            out += 16 * item;
            for (int h = h0; h < h1; h += kRopeUnroll / 2) {
                uint4 x[kRopeUnroll / 2], y[kRopeUnroll / 2];
#pragma unroll
                for (int j = 0; j < kRopeUnroll / 2; ++j)
                    if (h + j < h1) {
                        const char* at = in + (h + j) * t.in_h;
                        x[j] = (W == 8 || end >= 8) ? load16(at) : load_pieces<W>(at, end);
                        y[j] = load_pieces<W>(at + second, end);
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
                        char* to = out + (h + j) * t.out_h;
                        if (W == 8 || end >= 8) store16(to, pack8<KIND>(r));
                        else store_pieces<W>(to, pack8<KIND>(r), end);
                        store_pieces<W>(to + second, pack8<KIND>(q), end);
                    }
            }
        } else {  // channels behind the rotated ones
            const int at = 2 * p.P + 8 * (item - p.pair_items);
            for (int h = h0; h < h1; ++h)
                store_pieces<W>(out + h * t.out_h + 2 * at, load_pieces<W>(in + h * t.in_h + 2 * at, p.d - at), p.d - at);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// The norms around a block.  A group of W = ceil(C / 256) warps works on whole rows, each thread on the same
// eight channels of every row (its gate, scale, shift, weights and column sums stay in registers), kRows rows
// at a time so that their loads are in flight together and one barrier serves them all.  A row's mean and
// variance: each warp takes its sum by shuffles, then the sum of squares about its own mean, and the warps'
// (sum, squares) pairs are joined exactly:  M2 = sum_w [M2_w + n_w (mean_w - mean)^2].  Nothing cancels, whatever
// the row's mean.
// ---------------------------------------------------------------------------------------------
constexpr int kNormNone = 0, kNormLayer = 1, kNormRms = 2;
constexpr int kNormMaxWarps = 32;

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
    float* partials;         // backward: [sums][group][C]
    int want;                // backward: bit k set where column sum k is wanted
};

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ void group_sync(int group_in_cta, int warps)
{
    if (warps > 1) asm volatile("bar.sync %0, %1;" ::"r"(group_in_cta + 1), "r"(warps * 32) : "memory");
}
template <int KIND>
__device__ __forceinline__ F8 load_vector(const char* p, int c, bool active, float absent)
{
    F8 f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = absent;
    if (p != nullptr && active) f = unpack8<KIND>(load16(p + 2 * c));
    return f;
}

// Exchange of one pair of sums per row between the warps of a group.  The two buffers take turns: a buffer is
// written again only behind the barrier of the exchange in between, which every warp reaches after it has read.
template <int R>
struct GroupExchange {
    float2* buf;  // [2][R][kNormMaxWarps] of this group
    int turn;
    __device__ __forceinline__ float2* next()
    {
        float2* b = buf + turn * R * kNormMaxWarps;
        turn ^= 1;
        return b;
    }
};

// mean (0 for RMS) and 1 / sqrt(var + eps) of R rows at once; NORM: kNormLayer or kNormRms.
template <int NORM, int R>
__device__ __forceinline__ void row_stats(const F8 (&v)[R], bool active, const NormParams& p, int warp, int lane, int g,
                                          GroupExchange<R>& ex, float (&mean)[R], float (&rstd)[R])
{
    // channels of this warp: 256, fewer in the last one
    const float cnt = static_cast<float>(min(256, p.C - warp * 256));
    float sum[R], sq[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float s = 0.0f;
        if (NORM == kNormLayer) {
            if (active) {
#pragma unroll
                for (int i = 0; i < 8; ++i) s += v[r].v[i];
            }
            s = warp_sum(s);
        }
        sum[r] = s;
        const float m = NORM == kNormLayer ? s / cnt : 0.0f;
        float q = 0.0f;
        if (active) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = v[r].v[i] - m;
                q = fmaf(d, d, q);
            }
        }
        sq[r] = warp_sum(q);
    }
    if (p.warps > 1) {
        float2* b = ex.next();
        if (lane == 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) b[r * kNormMaxWarps + warp] = make_float2(sum[r], sq[r]);
        }
        group_sync(g, p.warps);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float s = 0.0f, q = 0.0f;
            if (NORM == kNormLayer) {
                for (int w = 0; w < p.warps; ++w) s += b[r * kNormMaxWarps + w].x;
            }
            const float m = s * p.inv_c;
            for (int w = 0; w < p.warps; ++w) {
                const float2 o = b[r * kNormMaxWarps + w];
                q += o.y;
                if (NORM == kNormLayer) {
                    const float n = static_cast<float>(min(256, p.C - w * 256));
                    const float d = o.x / n - m;
                    q = fmaf(n * d, d, q);
                }
            }
            mean[r] = m;
            rstd[r] = rsqrtf(q * p.inv_c + p.eps);
        }
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean[r] = sum[r] * p.inv_c;
            rstd[r] = rsqrtf(sq[r] * p.inv_c + p.eps);
        }
    }
}

// Sums over the row of two values per row.
template <int R>
__device__ __forceinline__ void row_sums(float (&u)[R], float (&w)[R], const NormParams& p, int warp, int lane, int g,
                                         GroupExchange<R>& ex)
{
#pragma unroll
    for (int r = 0; r < R; ++r) {
        u[r] = warp_sum(u[r]);
        w[r] = warp_sum(w[r]);
    }
    if (p.warps <= 1) return;
    float2* b = ex.next();
    if (lane == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) b[r * kNormMaxWarps + warp] = make_float2(u[r], w[r]);
    }
    group_sync(g, p.warps);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        u[r] = w[r] = 0.0f;
        for (int i = 0; i < p.warps; ++i) {
            const float2 o = b[r * kNormMaxWarps + i];
            u[r] += o.x;
            w[r] += o.y;
        }
    }
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

template <int KIND, int POST, int PRE, bool A, int R, int T>
__global__ void __launch_bounds__(T) block_norm_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ float2 norm_smem[];
    const int g = threadIdx.x / (32 * p.warps);
    const int group = blockIdx.x * (blockDim.x / (32 * p.warps)) + g;
    if (group >= p.groups) return;
    const int t = threadIdx.x - g * 32 * p.warps, warp = t / 32, lane = t & 31, c = 8 * t;
    const bool active = c < p.C;
    const GroupRows rows = group_rows(p, group);
    GroupExchange<R> ex = {norm_smem + g * 2 * R * kNormMaxWarps, 0};

    // y = rs x + (h Ap + Bp);  n = h An + Bn
    F8 Ap, Bp, An, Bn;
    if (A) {
        const F8 gate = load_vector<KIND>(p.gate.p == nullptr ? nullptr : p.gate.p + rows.b * p.gate.b, c, active, 1.0f);
        Ap = load_vector<KIND>(p.post_w, c, active, 1.0f);
        Bp = load_vector<KIND>(p.post_b, c, active, 0.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) Ap.v[i] *= gate.v[i], Bp.v[i] *= gate.v[i];
    }
    if (PRE != kNormNone) {
        const F8 scale = load_vector<KIND>(p.scale.p == nullptr ? nullptr : p.scale.p + rows.b * p.scale.b, c, active, 0.0f);
        const F8 shift = load_vector<KIND>(p.shift.p == nullptr ? nullptr : p.shift.p + rows.b * p.shift.b, c, active, 0.0f);
        An = load_vector<KIND>(p.pre_w, c, active, 1.0f);
        Bn = load_vector<KIND>(p.pre_b, c, active, 0.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            An.v[i] *= 1.0f + scale.v[i];
            Bn.v[i] = fmaf(Bn.v[i], 1.0f + scale.v[i], shift.v[i]);
        }
    }
    const char* x0 = p.x.p + rows.b * p.x.b + 2 * c;
    const char* a0 = A ? p.a.p + rows.b * p.a.b + 2 * c : nullptr;
    char* y0 = A ? p.y.p + rows.b * p.y.b + 2 * c : nullptr;
    char* n0 = PRE != kNormNone ? p.n.p + rows.b * p.n.b + 2 * c : nullptr;
    for (int i0 = rows.begin; i0 < rows.end; i0 += R) {
        uint4 xr[R], ar[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            xr[r] = ar[r] = make_uint4(0u, 0u, 0u, 0u);
            if (active && i0 + r < rows.end) {
                xr[r] = load16(x0 + (i0 + r) * p.x.r);
                if (A) ar[r] = load16(a0 + (i0 + r) * p.a.r);
            }
        }
        F8 y[R];
#pragma unroll
        for (int r = 0; r < R; ++r) y[r] = unpack8<KIND>(xr[r]);
        float mean[R], rstd[R];
        if (A) {
            F8 h[R];
#pragma unroll
            for (int r = 0; r < R; ++r) h[r] = unpack8<KIND>(ar[r]);
            if (POST != kNormNone) {
                row_stats<POST == kNormNone ? kNormRms : POST, R>(h, active, p, warp, lane, g, ex, mean, rstd);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[r].v[i] = (h[r].v[i] - mean[r]) * rstd[r];
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[r].v[i] = fmaf(p.rs, y[r].v[i], fmaf(h[r].v[i], Ap.v[i], Bp.v[i]));
                const uint4 stored = pack8<KIND>(y[r]);
                if (active && i0 + r < rows.end) store16(y0 + (i0 + r) * p.y.r, stored);
                y[r] = unpack8<KIND>(stored);  // the norm below is that of the stored stream
            }
        }
        if (PRE != kNormNone) {
            row_stats<PRE == kNormNone ? kNormRms : PRE, R>(y, active, p, warp, lane, g, ex, mean, rstd);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                F8 o;
#pragma unroll
                for (int i = 0; i < 8; ++i) o.v[i] = fmaf((y[r].v[i] - mean[r]) * rstd[r], An.v[i], Bn.v[i]);
                if (active && i0 + r < rows.end) store16(n0 + (i0 + r) * p.n.r, pack8<KIND>(o));
            }
        }
    }
}

// Backward.  With h = Pre(y), e = Post(a), g = dn * (1 + scale) * pre_weight and u the gradient of y:
//     u  = dy + rstd_y (g - mean(g) - h mean(g h))          (no mean(g) for the RMS norm)
//     dx = rs u,   w = u * gate * post_weight,   da = rstd_a (w - mean(w) - e mean(w e))
// and every vector's gradient follows from four column sums over a batch entry's rows:
//     [0] sum dn   [1] sum dn h   [2] sum u e   [3] sum u
// which the group keeps in registers over its rows and leaves as partials for block_norm_grads_kernel.
template <int KIND, int POST, int PRE, bool A, int R, int T>
__global__ void __launch_bounds__(T) block_norm_backward_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ float2 norm_smem[];
    const int g = threadIdx.x / (32 * p.warps);
    const int group = blockIdx.x * (blockDim.x / (32 * p.warps)) + g;
    if (group >= p.groups) return;
    const int t = threadIdx.x - g * 32 * p.warps, warp = t / 32, lane = t & 31, c = 8 * t;
    const bool active = c < p.C;
    const GroupRows rows = group_rows(p, group);
    GroupExchange<R> ex = {norm_smem + g * 2 * R * kNormMaxWarps, 0};

    F8 Ap, An;
    if (A) {
        const F8 gate = load_vector<KIND>(p.gate.p == nullptr ? nullptr : p.gate.p + rows.b * p.gate.b, c, active, 1.0f);
        Ap = load_vector<KIND>(p.post_w, c, active, 1.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) Ap.v[i] *= gate.v[i];
    }
    if (PRE != kNormNone) {
        const F8 scale = load_vector<KIND>(p.scale.p == nullptr ? nullptr : p.scale.p + rows.b * p.scale.b, c, active, 0.0f);
        An = load_vector<KIND>(p.pre_w, c, active, 1.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) An.v[i] *= 1.0f + scale.v[i];
    }
    F8 sum[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[k].v[i] = 0.0f;

    const bool has_dy = p.dy.p != nullptr;
    const char* y0 = PRE != kNormNone ? p.x.p + rows.b * p.x.b + 2 * c : nullptr;
    const char* a0 = A ? p.a.p + rows.b * p.a.b + 2 * c : nullptr;
    const char* dy0 = has_dy ? p.dy.p + rows.b * p.dy.b + 2 * c : nullptr;
    const char* dn0 = PRE != kNormNone ? p.dn.p + rows.b * p.dn.b + 2 * c : nullptr;
    char* dx0 = p.dx.p + rows.b * p.dx.b + 2 * c;
    char* da0 = A ? p.da.p + rows.b * p.da.b + 2 * c : nullptr;
    for (int i0 = rows.begin; i0 < rows.end; i0 += R) {
        uint4 yr[R], ar[R], ur[R], gr[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            yr[r] = ar[r] = ur[r] = gr[r] = make_uint4(0u, 0u, 0u, 0u);
            if (active && i0 + r < rows.end) {
                if (PRE != kNormNone) yr[r] = load16(y0 + (i0 + r) * p.x.r);
                if (PRE != kNormNone) gr[r] = load16(dn0 + (i0 + r) * p.dn.r);
                if (has_dy) ur[r] = load16(dy0 + (i0 + r) * p.dy.r);
                if (A) ar[r] = load16(a0 + (i0 + r) * p.a.r);
            }
        }
        F8 u[R];
#pragma unroll
        for (int r = 0; r < R; ++r) u[r] = unpack8<KIND>(ur[r]);
        float mean[R], rstd[R], m1[R], m2[R];
        if (PRE != kNormNone) {
            F8 h[R];
#pragma unroll
            for (int r = 0; r < R; ++r) h[r] = unpack8<KIND>(yr[r]);
            row_stats<PRE == kNormNone ? kNormRms : PRE, R>(h, active, p, warp, lane, g, ex, mean, rstd);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const F8 dn = unpack8<KIND>(gr[r]);
                m1[r] = m2[r] = 0.0f;
                if (active && i0 + r < rows.end) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        h[r].v[i] = (h[r].v[i] - mean[r]) * rstd[r];
                        sum[0].v[i] += dn.v[i];
                        sum[1].v[i] = fmaf(dn.v[i], h[r].v[i], sum[1].v[i]);
                        const float w = dn.v[i] * An.v[i];
                        m1[r] += w;
                        m2[r] = fmaf(w, h[r].v[i], m2[r]);
                    }
                }
            }
            row_sums<R>(m1, m2, p, warp, lane, g, ex);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const F8 dn = unpack8<KIND>(gr[r]);
                const float b1 = PRE == kNormLayer ? m1[r] * p.inv_c : 0.0f, b2 = m2[r] * p.inv_c;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    u[r].v[i] = fmaf(rstd[r], dn.v[i] * An.v[i] - b1 - h[r].v[i] * b2, u[r].v[i]);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (active && i0 + r < rows.end) {
                F8 o;
#pragma unroll
                for (int i = 0; i < 8; ++i) o.v[i] = p.rs * u[r].v[i];
                store16(dx0 + (i0 + r) * p.dx.r, pack8<KIND>(o));
            }
        if (A) {
            F8 e[R];
#pragma unroll
            for (int r = 0; r < R; ++r) e[r] = unpack8<KIND>(ar[r]);
            if (POST != kNormNone) row_stats<POST == kNormNone ? kNormRms : POST, R>(e, active, p, warp, lane, g, ex, mean, rstd);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                m1[r] = m2[r] = 0.0f;
                if (active && i0 + r < rows.end) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (POST != kNormNone) e[r].v[i] = (e[r].v[i] - mean[r]) * rstd[r];
                        sum[2].v[i] = fmaf(u[r].v[i], e[r].v[i], sum[2].v[i]);
                        sum[3].v[i] += u[r].v[i];
                        u[r].v[i] *= Ap.v[i];
                        m1[r] += u[r].v[i];
                        m2[r] = fmaf(u[r].v[i], e[r].v[i], m2[r]);
                    }
                }
            }
            if (POST != kNormNone) row_sums<R>(m1, m2, p, warp, lane, g, ex);
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (active && i0 + r < rows.end) {
                    if (POST != kNormNone) {
                        const float b1 = POST == kNormLayer ? m1[r] * p.inv_c : 0.0f, b2 = m2[r] * p.inv_c;
#pragma unroll
                        for (int i = 0; i < 8; ++i) u[r].v[i] = rstd[r] * (u[r].v[i] - b1 - e[r].v[i] * b2);
                    }
                    store16(da0 + (i0 + r) * p.da.r, pack8<KIND>(u[r]));
                }
        }
    }
    if (active) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if ((p.want >> k) & 1) {
                float4* to = reinterpret_cast<float4*>(p.partials + (static_cast<size_t>(k) * p.groups + group) * p.C + c);
                to[0] = make_float4(sum[k].v[0], sum[k].v[1], sum[k].v[2], sum[k].v[3]);
                to[1] = make_float4(sum[k].v[4], sum[k].v[5], sum[k].v[6], sum[k].v[7]);
            }
    }
    pdl_launch_dependents();
}

// Second stage: the column sums of each batch entry in a fixed order, and from them the vectors' gradients.
struct NormGradParams {
    const float* partials;
    int B, C, chunks, groups, want;
    Channels gate, scale;
    const char *pre_w, *pre_b, *post_w, *post_b;
    int gate_per_batch, scale_per_batch, shift_per_batch;
    float *d_gate, *d_scale, *d_shift, *d_pre_w, *d_pre_b, *d_post_w, *d_post_b;
};
constexpr int kNormGradSlices = 32;

template <int KIND>
__device__ __forceinline__ float channel(const char* p, int c, float absent)
{
    if (p == nullptr) return absent;
    const uint32_t h = *reinterpret_cast<const unsigned short*>(p + 2 * c);
    return pair_lo<KIND>(h);
}

// 32 channels x 32 slices of the groups; the slices are joined through shared memory.
template <int KIND>
__global__ void __launch_bounds__(32 * kNormGradSlices) block_norm_grads_kernel(const __grid_constant__ NormGradParams p)
{
    __shared__ float s[4][kNormGradSlices][33];
    const int lane = threadIdx.x & 31, slice = threadIdx.x / 32, c = blockIdx.x * 32 + lane;
    pdl_wait();
    float all[7] = {};  // over the batch: shift, scale, pre_b, pre_w, gate, post_w, post_b (slice 0)
    for (int b = 0; b < p.B; ++b) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float v = 0.0f;
            if (((p.want >> k) & 1) && c < p.C)
                for (int i = slice; i < p.chunks; i += kNormGradSlices)
                    v += p.partials[(static_cast<size_t>(k) * p.groups + static_cast<size_t>(b) * p.chunks + i) * p.C + c];
            s[k][slice][lane] = v;
        }
        __syncthreads();
        // warp k joins column sum k: lane l over the slices of channel c
        if (slice < 4) {
            float v = 0.0f;
            for (int i = 0; i < kNormGradSlices; ++i) v += s[slice][i][lane];
            s[slice][0][lane] = v;
        }
        __syncthreads();
        if (slice == 0 && c < p.C) {
            const float dn = s[0][0][lane], dnh = s[1][0][lane], ue = s[2][0][lane], u = s[3][0][lane];
            const size_t at = static_cast<size_t>(b) * p.C + c;
            const float w = channel<KIND>(p.pre_w, c, 1.0f), wb = channel<KIND>(p.pre_b, c, 0.0f);
            const float sc = 1.0f + channel<KIND>(p.scale.p == nullptr ? nullptr : p.scale.p + b * p.scale.b, c, 0.0f);
            const float d_scale = w * dnh + wb * dn;
            const float gate = channel<KIND>(p.gate.p == nullptr ? nullptr : p.gate.p + b * p.gate.b, c, 1.0f);
            const float d_gate = channel<KIND>(p.post_w, c, 1.0f) * ue + channel<KIND>(p.post_b, c, 0.0f) * u;
            if (p.d_shift != nullptr && p.shift_per_batch) p.d_shift[at] = dn;
            if (p.d_scale != nullptr && p.scale_per_batch) p.d_scale[at] = d_scale;
            if (p.d_gate != nullptr && p.gate_per_batch) p.d_gate[at] = d_gate;
            all[0] += dn;
            all[1] += d_scale;
            all[2] += sc * dn;
            all[3] += sc * dnh;
            all[4] += d_gate;
            all[5] += gate * ue;
            all[6] += gate * u;
        }
        __syncthreads();
    }
    if (slice != 0 || c >= p.C) return;
    if (p.d_shift != nullptr && !p.shift_per_batch) p.d_shift[c] = all[0];
    if (p.d_scale != nullptr && !p.scale_per_batch) p.d_scale[c] = all[1];
    if (p.d_pre_b != nullptr) p.d_pre_b[c] = all[2];
    if (p.d_pre_w != nullptr) p.d_pre_w[c] = all[3];
    if (p.d_gate != nullptr && !p.gate_per_batch) p.d_gate[c] = all[4];
    if (p.d_post_w != nullptr) p.d_post_w[c] = all[5];
    if (p.d_post_b != nullptr) p.d_post_b[c] = all[6];
}

}  // namespace lf
