// The gated linear recurrence of include/linfusion_layers.h, forward and backward.
//
// Mathematics.  h_t = h_(t-1) + e_t (v_t - h_(t-1)) is the map h -> A h + H with A = 1 - e, H = e v, and maps compose:
// (A1, H1) then (A2, H2) is (A1 A2, A2 H1 + H2).  A tile of tokens is read once, into registers; each thread forms the map of its
// few tokens, threads and warps are joined by a scan, and tiles by the state that enters them, which a tile gets from those
// before it while its own data stays where it is.  The update is kept in the form h + e (v - h) with e formed without
// cancellation: near e = 0 (long memories) 1 - e has lost e's digits, and a product of thousands of such factors would show it.
//
// Between tiles.  Every tile publishes its map at once.  Tiles come in groups of kGroup; the last of a group also publishes the
// state behind it.  A tile composes the maps of those before it in its group and applies them to the last group's state:
// always the same products in the same order, so results do not depend on which tile was how far (a look-back that takes the
// first state it finds would).  Tiles are dealt out by a counter in the order of the scan, so whatever a tile waits for
// belongs to a tile that runs already.  Waits are bounded.
//
// Bound by DRAM: forward 8 bytes a value with a gate (three inputs, h), backward 14, or 11.1 from checkpoints.
#pragma once

#include "column_sums.cuh"
#include "pack8.cuh"

namespace lf {

constexpr int kRecSlab = 64;    // channels of a tile: rows of 128 bytes
constexpr int kRecEvery = 64;   // tokens from one kept state to the next
constexpr int kRecGroup = 16;   // tiles whose maps a tile composes at most, but one
constexpr int kRecShort = 8;    // tokens up to which a thread goes through the sequence alone

static __device__ unsigned int recurrence_expired_waits;

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
    const float *rate, *h0, *state_in, *dlast;
    float *last, *state_out, *dh0, *rate_partials;
    unsigned int* ticket;         // these three are zero when the kernel starts; not used with one tile
    ulonglong2* maps;             // [tile][channel]: a word for A and one for H, each with a flag above its 32 bits
    unsigned long long* states;   // [group][channel]: the state behind the group, in the same way
    int B, N, C, slabs, tiles, groups, scale_groups, n_states, reverse;
};

// Where lanes sit in a tile: V channels a thread, so kRecSlab / V lanes make a row of tokens, R tokens a thread.
template <int V, int R, int WARPS>
struct RecShape {
    static constexpr int kLanes = kRecSlab / V;      // lanes across the channels
    static constexpr int kSegs = 32 / kLanes;        // token segments in a warp
    static constexpr int kTokens = WARPS * kSegs * R;
    static constexpr int kThreads = 32 * WARPS;
};

__device__ __forceinline__ float rec_rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float rec_sigmoid(float x) { return rec_rcp(1.0f + ex2_approx(-kLog2e * x)); }
// 1 - exp(-L).  Below 1/4 by its series (the next term is below 2^-24 of the sum), above from the exponential.
__device__ __forceinline__ float rec_one_minus_exp(float L)
{
    float s = fmaf(L, -1.0f / 720, 1.0f / 120);
    s = fmaf(L, s, -1.0f / 24);
    s = fmaf(L, s, 1.0f / 6);
    s = fmaf(L, s, -0.5f);
    s = fmaf(L * L, s, L);
    const float direct = 1.0f - ex2_approx(-kLog2e * L);
    return fabsf(L) < 0.25f ? s : direct;
}

// V values of one token: 2 V bytes, or V bytes and the byte of their group's scale.
template <int KIND, int V, bool PACKED>
struct RecRaw {
    uint32_t w[PACKED ? V / 4 : V / 2];
    int scale;
    __device__ __forceinline__ void load(const RecInput& in, long long at, long long scale_at)
    {
        constexpr int words = PACKED ? V / 4 : V / 2;
        const char* q = in.p + at;
        if (words == 4) asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1 % words]), "=r"(w[2 % words]), "=r"(w[3 % words]) : "l"(q) : "memory");
        else if (words == 2) asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1 % words]) : "l"(q) : "memory");
        else asm volatile("ld.global.u32 %0, [%1];" : "=r"(w[0]) : "l"(q) : "memory");
        if (PACKED) scale = in.scales[scale_at];
    }
    // What stands in for a token behind the end: `pair` in every pair of a 16-bit input, zeros in a packed one.
    __device__ __forceinline__ void fill(uint32_t pair)
    {
#pragma unroll
        for (int i = 0; i < (PACKED ? V / 4 : V / 2); ++i) w[i] = PACKED ? 0u : pair;
        scale = 127;
    }
    __device__ __forceinline__ void values(float* v) const
    {
        if constexpr (PACKED) {
#pragma unroll
            for (int i = 0; i < V / 4; ++i) unpack8_codes4(w[i], pack8_step(scale), v + 4 * i);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                v[2 * i] = pair_lo<KIND>(w[i]);
                v[2 * i + 1] = pair_hi<KIND>(w[i]);
            }
        }
    }
};
template <int KIND, int V>
__device__ __forceinline__ void rec_store(char* at, const float* v)
{
    uint32_t w[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) w[i] = pack_pair<KIND>(v[2 * i], v[2 * i + 1]);
    if constexpr (V == 8) asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    else if constexpr (V == 4) asm volatile("st.global.cs.v2.u32 [%0], {%1,%2};" ::"l"(at), "r"(w[0]), "r"(w[1]) : "memory");
    else asm volatile("st.global.cs.u32 [%0], %1;" ::"l"(at), "r"(w[0]) : "memory");
}
template <int V>
__device__ __forceinline__ void rec_load_floats(float* v, const float* p)  // 4 V bytes on a boundary of that
{
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const float2 t = *reinterpret_cast<const float2*>(p + 2 * i);
        v[2 * i] = t.x;
        v[2 * i + 1] = t.y;
    }
}
template <int V>
__device__ __forceinline__ void rec_store_floats(float* p, const float* v)
{
#pragma unroll
    for (int i = 0; i < V / 2; ++i) *reinterpret_cast<float2*>(p + 2 * i) = make_float2(v[2 * i], v[2 * i + 1]);
}

// ------------------------------------------------------------------------------------------ between tiles
__device__ __forceinline__ unsigned long long rec_word(float x) { return (1ull << 32) | __float_as_uint(x); }
__device__ __forceinline__ void rec_publish(ulonglong2* p, float A, float H)
{
    asm volatile("st.relaxed.gpu.global.v2.b64 [%0], {%1, %2};" ::"l"(p), "l"(rec_word(A)), "l"(rec_word(H)) : "memory");
}
__device__ __forceinline__ void rec_publish(unsigned long long* p, float s)
{
    asm volatile("st.relaxed.gpu.global.b64 [%0], %1;" ::"l"(p), "l"(rec_word(s)) : "memory");
}
__device__ __forceinline__ ulonglong2 rec_peek(const ulonglong2* p)
{
    ulonglong2 v;
    asm volatile("ld.relaxed.gpu.global.v2.b64 {%0, %1}, [%2];" : "=l"(v.x), "=l"(v.y) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ unsigned long long rec_peek(const unsigned long long* p)
{
    unsigned long long v;
    asm volatile("ld.relaxed.gpu.global.b64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ bool rec_there(ulonglong2 v) { return (v.x >> 32) != 0ull && (v.y >> 32) != 0ull; }
__device__ __forceinline__ bool rec_there(unsigned long long v) { return (v >> 32) != 0ull; }
// `v`, read from p before, again until it is there or the time is up.  A value that never came counts as NaN.
template <typename W>
__device__ __forceinline__ W rec_await(const W* p, W v, W never)
{
    if (rec_there(v)) return v;
    const unsigned long long t0 = global_timer_ns();
    do {
        v = rec_peek(p);
        if (rec_there(v)) return v;
    } while (global_timer_ns() - t0 < kMaxBarrierWaitNs);
    atomicAdd(&recurrence_expired_waits, 1u);
    return never;
}
__device__ __forceinline__ float rec_low(unsigned long long w) { return __uint_as_float(static_cast<uint32_t>(w)); }

// The state that enters tile k (in the order of the pass) of a slab.  All threads call it; those of channel tid % 64 share the
// maps before it, four threads of up to four each.  `own` is this tile's map, `first` what enters tile 0 (both looked at in the
// first 64 threads, and `first` in tile 0 alone: it publishes the state behind it as a map that forgets what enters.  So nobody reads h0
// after tile 0 has, and the last state may be written over it).  Returns the state to the first 64 threads.  part: 4 x 64 maps in
// shared memory.
template <int THREADS>
__device__ __forceinline__ float rec_enter(const RecParams& p, long long slab_index, int k, float2 own, float first, float2 (*part)[kRecSlab])
{
    static_assert(THREADS == 256 && kRecGroup == 16, "four threads a channel, four maps each");
    const int ch = threadIdx.x & (kRecSlab - 1), quarter = threadIdx.x / kRecSlab;
    const int g = k / kRecGroup, in_group = k - g * kRecGroup;
    ulonglong2* maps = p.maps + slab_index * p.tiles * kRecSlab + ch;
    unsigned long long* states = p.states + slab_index * p.groups * kRecSlab + ch;
    if (quarter == 0) {
        if (k == 0) own = make_float2(0.0f, fmaf(own.x, first, own.y));
        rec_publish(maps + static_cast<long long>(k) * kRecSlab, own.x, own.y);
    }
    float A = 1.0f, H = 0.0f;
    const int j0 = 4 * quarter, n = min(4, in_group - j0);
    if (n > 0) {
        const ulonglong2* q = maps + static_cast<long long>(g * kRecGroup + j0) * kRecSlab;
        ulonglong2 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) v[j] = rec_peek(q + j * kRecSlab);
        const unsigned long long nan = (1ull << 32) | 0x7fffffffull;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) {
                const ulonglong2 w = rec_await(q + j * kRecSlab, v[j], make_ulonglong2(nan, nan));
                H = fmaf(rec_low(w.x), H, rec_low(w.y));
                A *= rec_low(w.x);
            }
    }
    part[quarter][ch] = make_float2(A, H);
    __syncthreads();
    float s = 0.0f;
    if (quarter == 0) {
        s = first;
        if (g > 0) {
            const unsigned long long* q = states + static_cast<long long>(g - 1) * kRecSlab;
            s = rec_low(rec_await(q, rec_peek(q), (1ull << 32) | 0x7fffffffull));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 m = part[i][ch];
            s = fmaf(m.x, s, m.y);
        }
        if (in_group == kRecGroup - 1) rec_publish(states + static_cast<long long>(g) * kRecSlab, fmaf(own.x, s, own.y));
    }
    return s;
}

// The tile that this block takes.
struct RecTile {
    int b, slab, k;           // k: its place in the order of the pass
    long long slab_index;     // b * slabs + slab
};
__device__ __forceinline__ RecTile rec_take(const RecParams& p, unsigned int* box)
{
    unsigned int t = blockIdx.x;
    if (p.tiles > 1) {
        if (threadIdx.x == 0) *box = atomicAdd(p.ticket, 1u);
        __syncthreads();
        t = *box;
    }
    const unsigned int all = static_cast<unsigned int>(p.B) * p.slabs;
    RecTile o;
    o.k = static_cast<int>(t / all);
    const unsigned int i = t - static_cast<unsigned int>(o.k) * all;
    o.b = static_cast<int>(i / p.slabs);
    o.slab = static_cast<int>(i - static_cast<unsigned int>(o.b) * p.slabs);
    o.slab_index = i;
    return o;
}

// Inclusive scan of maps over the token segments of a warp (lanes kLanes apart), forward or backward in the tokens; then the
// map of what lies before the own segment.
template <int V, int LANES, bool UP>
__device__ __forceinline__ void rec_warp_scan(float (&A)[V], float (&H)[V], float (&Ax)[V], float (&Hx)[V], int lane)
{
    const int seg = lane / LANES;
    constexpr int segs = 32 / LANES;
#pragma unroll
    for (int off = 1; off < segs; off *= 2) {
        const bool in = UP ? seg >= off : seg + off < segs;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float a = UP ? __shfl_up_sync(0xffffffffu, A[i], off * LANES) : __shfl_down_sync(0xffffffffu, A[i], off * LANES);
            const float h = UP ? __shfl_up_sync(0xffffffffu, H[i], off * LANES) : __shfl_down_sync(0xffffffffu, H[i], off * LANES);
            if (in) {
                H[i] = fmaf(A[i], h, H[i]);
                A[i] *= a;
            }
        }
    }
    const bool first = UP ? seg == 0 : seg == segs - 1;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        Ax[i] = UP ? __shfl_up_sync(0xffffffffu, A[i], LANES) : __shfl_down_sync(0xffffffffu, A[i], LANES);
        Hx[i] = UP ? __shfl_up_sync(0xffffffffu, H[i], LANES) : __shfl_down_sync(0xffffffffu, H[i], LANES);
        if (first) {
            Ax[i] = 1.0f;
            Hx[i] = 0.0f;
        }
    }
}

// Pairs that stand for tokens behind the end: -infinity as a decay, zeros otherwise.
template <int KIND>
__device__ __forceinline__ constexpr uint32_t rec_minus_infinity() { return kind_dtype(KIND) == kDtypeFp16 ? 0xFC00FC00u : 0xFF80FF80u; }

// ------------------------------------------------------------------------------------------ forward
// 128 tokens x 64 channels a block.  STORE: writes h and what else is asked for; without it only the kept states (the first half of a
// backward pass that was given none).
template <int KIND, bool GATE, bool PACKED, bool STORE>
__global__ void __launch_bounds__(256, 2) recurrence_kernel(const __grid_constant__ RecParams p)
{
    constexpr int V = 8, R = 4, WARPS = 8;
    using S = RecShape<V, R, WARPS>;
    __shared__ unsigned int box;
    __shared__ float2 totals[WARPS][kRecSlab];
    __shared__ float2 part[4][kRecSlab];
    __shared__ float enters[kRecSlab];

    const RecTile t = rec_take(p, &box);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int seg = warp * S::kSegs + lane / S::kLanes, ch = t.slab * kRecSlab + (lane % S::kLanes) * V;
    const bool live = ch < p.C;
    const int pos0 = t.k * S::kTokens + seg * R;

    RecRaw<KIND, V, PACKED> x[R], d[R], g[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int pos = pos0 + r, tok = p.reverse ? p.N - 1 - pos : pos;
        if (live && pos < p.N) {
            const long long width = PACKED ? ch : 2ll * ch, scale_at = (static_cast<long long>(t.b) * p.N + tok) * p.scale_groups + ch / 32;
            x[r].load(p.x, t.b * p.x.batch + tok * p.x.row + width, scale_at);
            d[r].load(p.decay, t.b * p.decay.batch + tok * p.decay.row + width, scale_at);
            if (GATE) g[r].load(p.gate, t.b * p.gate.batch + tok * p.gate.row + width, scale_at);
        } else {
            x[r].fill(0u);
            d[r].fill(rec_minus_infinity<KIND>());
            if (GATE) g[r].fill(0u);
        }
    }
    float rate[V];
    if (live) rec_load_floats<V>(rate, p.rate + ch);
    else
#pragma unroll
        for (int i = 0; i < V; ++i) rate[i] = 0.0f;

    float e[R][V], v[R][V], A[V], H[V], Ax[V], Hx[V];
#pragma unroll
    for (int i = 0; i < V; ++i) A[i] = H[i] = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float f[V];
        d[r].values(f);
        x[r].values(v[r]);
        const bool behind = PACKED && pos0 + r >= p.N;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float s = behind ? 0.0f : rec_sigmoid(f[i]), L = rate[i] * s;
            A[i] += L;
            e[r][i] = rec_one_minus_exp(L);
            if (s == 0.0f) v[r][i] = 0.0f;  // padding: whatever it holds
            f[i] = s;
        }
        if (GATE) {
            float q[V];
            g[r].values(q);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (f[i] != 0.0f) v[r][i] *= rec_sigmoid(q[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) H[i] = fmaf(e[r][i], v[r][i] - H[i], H[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) A[i] = ex2_approx(-kLog2e * A[i]);

    rec_warp_scan<V, S::kLanes, true>(A, H, Ax, Hx, lane);
    if (lane / S::kLanes == S::kSegs - 1)
#pragma unroll
        for (int i = 0; i < V; ++i) totals[warp][(lane % S::kLanes) * V + i] = make_float2(A[i], H[i]);
    __syncthreads();
    // per channel: the map before each warp, and the tile's
    float2 own = make_float2(1.0f, 0.0f);
    float first = 0.0f;
    if (tid < kRecSlab) {
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float2 m = totals[w][tid];
            totals[w][tid] = own;
            own = make_float2(own.x * m.x, fmaf(m.x, own.y, m.y));
        }
        const int c = t.slab * kRecSlab + tid;
        if (p.h0 != nullptr && c < p.C && t.k == 0) first = p.h0[static_cast<long long>(t.b) * p.C + c];
    }
    if (p.tiles > 1) first = rec_enter<S::kThreads>(p, t.slab_index, t.k, own, first, part);
    if (tid < kRecSlab) enters[tid] = first;
    __syncthreads();

    float h[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (lane % S::kLanes) * V + i;
        const float2 m = totals[warp][c];
        h[i] = fmaf(Ax[i], fmaf(m.x, enters[c], m.y), Hx[i]);
    }
    if (!live) return;
    if (p.state_out != nullptr && pos0 % kRecEvery == 0 && pos0 < p.N)
        rec_store_floats<V>(p.state_out + (static_cast<long long>(t.b) * p.n_states + pos0 / kRecEvery) * p.C + ch, h);
    if constexpr (STORE) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int pos = pos0 + r, tok = p.reverse ? p.N - 1 - pos : pos;
#pragma unroll
            for (int i = 0; i < V; ++i) h[i] = fmaf(e[r][i], v[r][i] - h[i], h[i]);
            if (pos < p.N) rec_store<KIND, V>(p.h.p + t.b * p.h.batch + tok * p.h.row + 2ll * ch, h);
        }
        // tokens behind the end have left the state as it was
        if (p.last != nullptr && t.k == p.tiles - 1 && seg == WARPS * S::kSegs - 1)
            rec_store_floats<V>(p.last + static_cast<long long>(t.b) * p.C + ch, h);
    }
}

// A few tokens (one, when a sequence is continued token by token): a thread takes two channels through all of them.  Latency.
constexpr int kRecShortThreads = 128;
template <int KIND, bool GATE>
__global__ void __launch_bounds__(kRecShortThreads) recurrence_short_kernel(const __grid_constant__ RecParams p)
{
    const long long i = static_cast<long long>(blockIdx.x) * kRecShortThreads + threadIdx.x;
    const int pairs = p.C / 2, b = static_cast<int>(i / pairs), ch = 2 * static_cast<int>(i - static_cast<long long>(b) * pairs);
    if (b >= p.B) return;
    float rate[2], h[2] = {0.0f, 0.0f};
    rec_load_floats<2>(rate, p.rate + ch);
    if (p.h0 != nullptr) rec_load_floats<2>(h, p.h0 + static_cast<long long>(b) * p.C + ch);
    if (p.state_out != nullptr) rec_store_floats<2>(p.state_out + static_cast<long long>(b) * p.C + ch, h);
    RecRaw<KIND, 2, false> x[kRecShort], d[kRecShort], g[kRecShort];
#pragma unroll
    for (int r = 0; r < kRecShort; ++r)
        if (r < p.N) {
            const int tok = p.reverse ? p.N - 1 - r : r;
            x[r].load(p.x, b * p.x.batch + tok * p.x.row + 2ll * ch, 0);
            d[r].load(p.decay, b * p.decay.batch + tok * p.decay.row + 2ll * ch, 0);
            if (GATE) g[r].load(p.gate, b * p.gate.batch + tok * p.gate.row + 2ll * ch, 0);
        }
#pragma unroll
    for (int r = 0; r < kRecShort; ++r)
        if (r < p.N) {
            const int tok = p.reverse ? p.N - 1 - r : r;
            float v[2], f[2], q[2] = {0.0f, 0.0f};
            x[r].values(v);
            d[r].values(f);
            if (GATE) g[r].values(q);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float s = rec_sigmoid(f[k]), e = rec_one_minus_exp(rate[k] * s);
                if (GATE) v[k] *= rec_sigmoid(q[k]);
                if (s == 0.0f) v[k] = 0.0f;
                h[k] = fmaf(e, v[k] - h[k], h[k]);
            }
            rec_store<KIND, 2>(p.h.p + b * p.h.batch + tok * p.h.row + 2ll * ch, h);
        }
    if (p.last != nullptr) rec_store_floats<2>(p.last + static_cast<long long>(b) * p.C + ch, h);
}

// ------------------------------------------------------------------------------------------ backward
// 64 tokens x 64 channels a block, tiles from the last to the first.  The states inside the tile come from the kept one, the gradient
// G from the tiles behind; G's map over a token is G -> (1 - e)(dh + G), so its A is the forward pass' own.
template <int KIND, bool GATE, bool PACKED>
__global__ void __launch_bounds__(256, 2) recurrence_backward_kernel(const __grid_constant__ RecParams p)
{
    constexpr int V = 4, R = 4, WARPS = 8;
    using S = RecShape<V, R, WARPS>;
    static_assert(S::kTokens == kRecEvery, "a kept state for each tile");
    __shared__ unsigned int box;
    __shared__ float2 totals[2][WARPS][kRecSlab];
    __shared__ float2 part[4][kRecSlab];
    __shared__ float enters[2][kRecSlab];

    const RecTile t = rec_take(p, &box);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int seg = warp * S::kSegs + lane / S::kLanes, cl = (lane % S::kLanes) * V, ch = t.slab * kRecSlab + cl;
    const bool live = ch < p.C;
    const int tile = p.tiles - 1 - t.k, pos0 = tile * S::kTokens + seg * R;

    RecRaw<KIND, V, PACKED> x[R], d[R], g[R];
    RecRaw<KIND, V, false> dh[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int pos = pos0 + r, tok = p.reverse ? p.N - 1 - pos : pos;
        if (live && pos < p.N) {
            const long long width = PACKED ? ch : 2ll * ch, scale_at = (static_cast<long long>(t.b) * p.N + tok) * p.scale_groups + ch / 32;
            x[r].load(p.x, t.b * p.x.batch + tok * p.x.row + width, scale_at);
            d[r].load(p.decay, t.b * p.decay.batch + tok * p.decay.row + width, scale_at);
            if (GATE) g[r].load(p.gate, t.b * p.gate.batch + tok * p.gate.row + width, scale_at);
            dh[r].load(p.dh, t.b * p.dh.batch + tok * p.dh.row + 2ll * ch, 0);
        } else {
            x[r].fill(0u);
            d[r].fill(rec_minus_infinity<KIND>());
            if (GATE) g[r].fill(0u);
            dh[r].fill(0u);
        }
    }
    float rate[V];
#pragma unroll
    for (int i = 0; i < V; ++i) rate[i] = 0.0f;
    if (live) rec_load_floats<V>(rate, p.rate + ch);

    // s = sigmoid(decay), q = sigmoid(gate), e, v = q x; a padded token's are zero
    float s[R][V], e[R][V], q[R][V], v[R][V], A[V], H[V], G[V];
#pragma unroll
    for (int i = 0; i < V; ++i) A[i] = H[i] = G[i] = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool behind = PACKED && pos0 + r >= p.N;
        d[r].values(s[r]);
        x[r].values(v[r]);
        if (GATE) g[r].values(q[r]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s[r][i] = behind ? 0.0f : rec_sigmoid(s[r][i]);
            const float L = rate[i] * s[r][i];
            A[i] += L;
            e[r][i] = rec_one_minus_exp(L);
            if (GATE) {
                q[r][i] = rec_sigmoid(q[r][i]);
                v[r][i] *= q[r][i];
            }
            if (s[r][i] == 0.0f) v[r][i] = q[r][i] = 0.0f;
            H[i] = fmaf(e[r][i], v[r][i] - H[i], H[i]);
        }
    }
#pragma unroll
    for (int r = R - 1; r >= 0; --r) {
        float y[V];
        dh[r].values(y);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float sum = y[i] + G[i];
            G[i] = fmaf(-e[r][i], sum, sum);
        }
    }
    float Ar[V], Axr[V], Gx[V], Ax[V], Hx[V];
#pragma unroll
    for (int i = 0; i < V; ++i) Ar[i] = A[i] = ex2_approx(-kLog2e * A[i]);
    rec_warp_scan<V, S::kLanes, true>(A, H, Ax, Hx, lane);
    rec_warp_scan<V, S::kLanes, false>(Ar, G, Axr, Gx, lane);
    if (lane / S::kLanes == S::kSegs - 1)
#pragma unroll
        for (int i = 0; i < V; ++i) totals[0][warp][cl + i] = make_float2(A[i], H[i]);
    if (lane / S::kLanes == 0)
#pragma unroll
        for (int i = 0; i < V; ++i) totals[1][warp][cl + i] = make_float2(Ar[i], G[i]);
    __syncthreads();
    float2 own = make_float2(1.0f, 0.0f);
    float first = 0.0f;
    if (tid < kRecSlab) {  // the gradient, from the last warp to the first
#pragma unroll
        for (int w = WARPS - 1; w >= 0; --w) {
            const float2 m = totals[1][w][tid];
            totals[1][w][tid] = own;
            own = make_float2(own.x * m.x, fmaf(m.x, own.y, m.y));
        }
        const int c = t.slab * kRecSlab + tid;
        if (p.dlast != nullptr && c < p.C && t.k == 0) first = p.dlast[static_cast<long long>(t.b) * p.C + c];
    } else if (tid < 2 * kRecSlab) {  // the state
        const int cs = tid - kRecSlab, c = t.slab * kRecSlab + cs;
        float h = c < p.C ? p.state_in[(static_cast<long long>(t.b) * p.n_states + tile) * p.C + c] : 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float2 m = totals[0][w][cs];
            totals[0][w][cs].x = h;  // what enters the warp
            h = fmaf(m.x, h, m.y);
        }
    }
    if (p.tiles > 1) first = rec_enter<S::kThreads>(p, t.slab_index, t.k, own, first, part);
    if (tid < kRecSlab) enters[0][tid] = first;
    __syncthreads();

    float h[V], drate[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 m = totals[1][warp][cl + i];
        G[i] = fmaf(Axr[i], fmaf(m.x, enters[0][cl + i], m.y), Gx[i]);
        h[i] = fmaf(Ax[i], totals[0][warp][cl + i].x, Hx[i]);
        drate[i] = 0.0f;
    }
    // v - h_(t-1), in v's place; then from the last token to the first
    float step[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            step[r][i] = v[r][i] - h[i];
            h[i] = fmaf(e[r][i], step[r][i], h[i]);
        }
#pragma unroll
    for (int r = R - 1; r >= 0; --r) {
        const int pos = pos0 + r, tok = p.reverse ? p.N - 1 - pos : pos;
        float y[V], ox[V], od[V], og[V];
        dh[r].values(y);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float sum = y[i] + G[i], dv = e[r][i] * sum;
            G[i] = sum - dv;
            const float dL = G[i] * step[r][i] * s[r][i];  // dL sigmoid(decay)
            drate[i] += dL;
            od[i] = dL * rate[i] * (1.0f - s[r][i]);
            ox[i] = GATE ? dv * q[r][i] : dv;
            if (GATE) og[i] = dv * v[r][i] * (1.0f - q[r][i]);
        }
        if (live && pos < p.N) {
            rec_store<KIND, V>(p.dx.p + t.b * p.dx.batch + tok * p.dx.row + 2ll * ch, ox);
            rec_store<KIND, V>(p.ddecay.p + t.b * p.ddecay.batch + tok * p.ddecay.row + 2ll * ch, od);
            if (GATE) rec_store<KIND, V>(p.dgate.p + t.b * p.dgate.batch + tok * p.dgate.row + 2ll * ch, og);
        }
    }
    if (live && p.dh0 != nullptr && tile == 0 && seg == 0) rec_store_floats<V>(p.dh0 + static_cast<long long>(t.b) * p.C + ch, G);
    if (p.rate_partials != nullptr) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
            for (int off = S::kLanes; off < 32; off *= 2) drate[i] += __shfl_xor_sync(0xffffffffu, drate[i], off);
            if (lane < S::kLanes) totals[0][warp][cl + i].x = drate[i];
        }
        __syncthreads();
        if (tid < kRecSlab) {
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) sum += totals[0][w][tid].x;
            p.rate_partials[(static_cast<long long>(t.b) * p.tiles + tile) * (p.slabs * kRecSlab) + t.slab * kRecSlab + tid] = sum;
        }
    }
}

}  // namespace lf
