// Backward pass of the normalized linear attention (include/linfusion_attn.h), for every supported pair of widths.
//
// With f = phi(q_i), g = dY_i, the state S | z of the forward pass and den = f . z + eps:
//
//     t = S g        w = 1 / den        c = w (f . t)  (= Y_i . g, so Y is not needed)
//     dq_i = phi'(q_i) * w (t - c z)
//     dS  += (w f)^T g        dz -= (w f) c
//
// and then, with f = phi(k_j):
//
//     dk_j = phi'(k_j) * (dS v_j + dz)        dv_j = dS^T f
//
// (without the normalizer: w = 1, c = 0, dz = 0).  phi'(x) = min(1, exp(x)) for elu + 1, 1 for the identity.  So the
// backward pass is two streams over the tokens, as the forward is: Q, dY -> dQ with the state gradient dS | dz summed
// on the way, then K, V -> dK, dV.  Nothing of size N x N, and nothing of size N but the gradients, is written.
//
// Precision.  t - c z is a difference: with values that have a mean, S is that mean times z plus a remainder about
// sqrt(N) times smaller, and only the remainder is left.  So the mean leaves before the products: with any fixed mu and
// R = S - z mu^T, and c' = w (f . R g - eps mu . g),
//
//     t - c z = R g - c' z        c = c' + mu . g        dz = - sum (w f) c' - dS mu
//
// mu = S^T z / (z . z) leaves the smallest R.  (The term with eps is formed only for tokens where w eps is 2^-24 or more: below,
// it is less than what the rounding of S to fp32 leaves.)  Every operand of the tensor-core products that is not an input
// tensor (R, w f, dS, phi(k)) is carried as a head and a tail of the storage type, x = hi + lo with |x - hi - lo| <= 2^-17 |x|
// (bf16) or 2^-23 (fp16): two products in place of one (three for dS^T f).  The results are then off by little more
// than the one rounding of the 16-bit outputs.
#pragma once

#include "common.cuh"
#include "packed_math.cuh"

namespace lf {

// Layout of S | z and of dS | dz per slab: dk x dv row-major, then dk.
__host__ __device__ constexpr int grad_state_floats(int dk, int dv) { return dk * dv + dk; }

__device__ __forceinline__ void stmatrix_x4_trans(uint32_t addr, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3)
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r0), "r"(r1), "r"(r2),
                 "r"(r3)
                 : "memory");
}
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, bool valid)
{
    const uint32_t bytes = valid ? 16u : 0u;  // 0: the destination is filled with zeros, the source not read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

// The smaller of two values, NaN where one is NaN (fminf drops it, and with it phi of a NaN would be 1).
__device__ __forceinline__ float min_nan(float a, float b)
{
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// phi and its slope of one value; both NaN for a NaN.
template <int KIND>
__device__ __forceinline__ void phi_and_slope(float x, float* f, float* slope)
{
    if (kind_phi(KIND) == kPhiIdentity) {
        *f = x;
        *slope = 1.0f;
        return;
    }
    const float e = ex2_approx(min_nan(x, 0.0f) * 1.4426950408889634f);
    *f = fmaxf(x, 0.0f) + e;
    *slope = e;
}
template <int KIND>
__device__ __forceinline__ float phi_or_nan(float x)
{
    float f, slope;
    phi_and_slope<KIND>(x, &f, &slope);
    return f;
}

// A pair of values as head and tail in the storage type.
template <int KIND>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t* hi, uint32_t* lo)
{
    *hi = pack_pair<KIND>(a, b);
    const float2 rest = unpack2(fma2(pack2(pair_lo<KIND>(*hi), pair_hi<KIND>(*hi)), both(-1.0f), pack2(a, b)));
    *lo = pack_pair<KIND>(rest.x, rest.y);
}

template <int DK, int DV>
struct BackwardCfg {
    static constexpr int KP = (DK + 15) / 16 * 16, VP = (DV + 15) / 16 * 16;  // widths padded to the products' step
    static constexpr int WQ = KP / 16;                                       // warps: 16 features each
    static constexpr int WKV = (KP > VP ? KP : VP) / 16;                     // ... or 16 channels of dV
    // Tokens at a time, fewer where more CTAs then fit on an SM beside the state: 79 us with 16 against 96 with 32 at 16 slabs x
    // 2048 x 128, 72 with 32 against 80 with 64 at 16 x 4096 x 80; 160 channels leave room for one CTA either way.
    static constexpr int TILE = KP + VP <= 128 ? 64 : KP + VP <= 160 ? 32 : KP + VP <= 256 ? 16 : 32;
    // A row takes an odd number of 16-byte units: eight rows of a matrix fragment fall into different banks.
    static constexpr int PITCHK = ((KP / 8) | 1) * 16, PITCHV = ((VP / 8) | 1) * 16;
    static constexpr int STAGE = TILE * (PITCHK + PITCHV);
    static constexpr int S_HALF = KP * PITCHV;  // the state's head, or its tail
    static constexpr int SMEM_STATE = 2 * STAGE;
    static constexpr int SMEM_Q = 2 * STAGE + 2 * S_HALF + KP * 4 + WQ * TILE * 8 + TILE * 8 + WQ * 16 * TILE * 4 + VP * 4;
    static constexpr int SMEM_KV = 2 * STAGE + 2 * S_HALF + KP * 4 + 2 * TILE * PITCHK;  // head and tail of phi(k)
};

struct BackwardScales {
    float eps;        // negative: without the normalizer
    int scaled;       // fp16 operands: scale R, w f and dS by powers of two of their own sizes
};

// Power of two 2^-e with 2^e <= x < 2^(e+1), times 2^up; 1 for zero, infinite or NaN x.
__device__ __forceinline__ float pow2_scale(float x, int up)
{
    if (!(x > 0.0f) || isinf(x)) return 1.0f;
    int e = static_cast<int>((__float_as_uint(x) >> 23) & 0xffu) - 127;
    e = min(max(up - e, -120), 120);
    return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}

// fp16: the power of two by which w f of feature a is multiplied to become an operand.  Features of elu + 1 are not negative, so
// w f_a = f_a / (f . z + eps) is at most 1 / z_a, and at most 2^16 / eps: each feature's own bound goes to 2^12, whatever the
// others' sizes (one scale for all let a token whose weight is on a feature of small z overflow; so did z = 0, keys that
// are all masked).
__device__ __forceinline__ float feature_scale(float z, float eps) { return pow2_scale(1.0f / fmaxf(z, eps * 1.52587890625e-5f), 12); }
// ... for features of either sign (phi(x) = x): one scale for the slab, from its largest z and its largest 1 / z (3e38 for a z that is
// not positive and so says nothing).
__device__ __forceinline__ float slab_scale(float z_max, float z_inv, float eps)
{
    return fmaxf(pow2_scale(z_inv, 12), 1.0f / pow2_scale(fmaxf(z_max, eps), 4));
}

// Copy tile `row0` .. of a slab into shared memory, rows past N as zeros.
template <int D, int PITCH, int TILE, int THREADS>
__device__ __forceinline__ void load_tile(unsigned char* dst, const __nv_bfloat16* base, int row_stride, int row0, int N)
{
    constexpr int VECS = D / 8;
    for (int i = threadIdx.x; i < TILE * VECS; i += THREADS) {
        const int r = i / VECS, v = i - r * VECS;
        const bool in = row0 + r < N;
        const __nv_bfloat16* src = base + static_cast<long long>(in ? row0 + r : 0) * row_stride + v * 8;
        cp_async_16(smem_u32(dst + r * PITCH + v * 16), src, in);
    }
}
template <int D, int PITCH, int TILE, int THREADS>
__device__ __forceinline__ void store_tile(const unsigned char* src, __nv_bfloat16* base, int row_stride, int row0, int N)
{
    constexpr int VECS = D / 8;
    for (int i = threadIdx.x; i < TILE * VECS; i += THREADS) {
        const int r = i / VECS, v = i - r * VECS;
        if (row0 + r < N)
            *reinterpret_cast<uint4*>(base + static_cast<long long>(row0 + r) * row_stride + v * 8) =
                *reinterpret_cast<const uint4*>(src + r * PITCH + v * 16);
    }
}
template <int D, int PITCH, int TILE, int THREADS>
__device__ __forceinline__ void clear_padding(unsigned char* dst)
{
    constexpr int P = (D + 15) / 16 * 16;
    if (P > D)
        for (int r = threadIdx.x; r < TILE; r += THREADS)
            for (int v = D / 8; v < P / 8; ++v) *reinterpret_cast<uint4*>(dst + r * PITCH + v * 16) = make_uint4(0u, 0u, 0u, 0u);
}

// The largest |x| over the block's threads; `scratch`: 33 floats.
__device__ __forceinline__ float block_max(float v, float* scratch, int warps)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x / 32] = v;
    __syncthreads();
    for (int i = 0; i < warps; ++i) v = fmaxf(v, scratch[i]);
    __syncthreads();
    return v;
}

// The term of c' with eps counts from this w eps on.
constexpr float kEpsCounts = 5.9604645e-8f;  // 2^-24

// A column of mu = S^T z / (z . z) from the two sums; zero where it is not finite (no keys at all, sums beyond fp32): any mu is right.
__device__ __forceinline__ float mean_of(float sum, float squares)
{
    const float m = sum / squares;
    return fabsf(m) < 3.0e38f ? m : 0.0f;
}
// mu . g of eight channels from one 16-byte piece of a row of dY.
template <int KIND>
__device__ __forceinline__ float mean_dot(const uint4& g, const float* mu, float sum)
{
    const uint32_t p[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = fmaf(pair_lo<KIND>(p[i]), mu[2 * i], fmaf(pair_hi<KIND>(p[i]), mu[2 * i + 1], sum));
    return sum;
}

// The block lays S (dS) out in shared memory as rows of features, head and tail, zeros where the widths end, and z (dz)
// as floats; CENTRED: R = S - z mu^T in place of S where eps is not negative, and mu as VP floats, zeros behind DV.  SCALED: by the
// power of two that takes the largest value to 2^12, which is returned.  Each thread has one 16-byte piece of every ROWS-th row
// (all loads in flight together: one by one, ten of them were a third of a call of one tile), kept in registers through the
// sums of mu, which pass through the rows' place.
template <int KIND, int DK, int DV, int THREADS, bool CENTRED>
__device__ __forceinline__ float load_state(const float* S, float eps, bool scaled, unsigned char* hi_rows, float* z, float* mu,
                                            float* scratch)
{
    using C = BackwardCfg<DK, DV>;
    constexpr int PER_ROW = C::VP / 8, ROWS = THREADS / PER_ROW, STEPS = (C::KP + ROWS - 1) / ROWS;
    static_assert(ROWS * (C::VP + 1) * 4 <= 2 * C::S_HALF && C::VP <= THREADS, "the sums of mu take the rows' place");
    const int slice = threadIdx.x / PER_ROW, piece = threadIdx.x - slice * PER_ROW;
    float x[STEPS][8];
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
        const int row = n * ROWS + slice;
        float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f), b = a;
        if (slice < ROWS && row < DK && piece < DV / 8) {
            const float4* p = reinterpret_cast<const float4*>(S + row * DV + 8 * piece);
            a = p[0];
            b = p[1];
        }
        x[n][0] = a.x, x[n][1] = a.y, x[n][2] = a.z, x[n][3] = a.w, x[n][4] = b.x, x[n][5] = b.y, x[n][6] = b.z, x[n][7] = b.w;
    }
    for (int i = threadIdx.x; i < C::KP; i += THREADS) z[i] = i < DK ? S[DK * DV + i] : 0.0f;
    if (CENTRED) {
        float* sums = reinterpret_cast<float*>(hi_rows);  // [ROWS][VP], then [ROWS] of z . z
        __syncthreads();
        if (slice < ROWS && eps >= 0.0f) {
            float s[8] = {}, zz = 0.0f;
#pragma unroll
            for (int n = 0; n < STEPS; ++n) {
                const int row = n * ROWS + slice;
                const float zr = row < C::KP ? z[row] : 0.0f;
                zz = fmaf(zr, zr, zz);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] = fmaf(zr, x[n][i], s[i]);
            }
            float4* to = reinterpret_cast<float4*>(sums + slice * C::VP + 8 * piece);
            to[0] = make_float4(s[0], s[1], s[2], s[3]);
            to[1] = make_float4(s[4], s[5], s[6], s[7]);
            if (piece == 0) sums[ROWS * C::VP + slice] = zz;
        }
        __syncthreads();
        if (threadIdx.x < C::VP) {
            float s = 0.0f, zz = 0.0f;
            if (eps >= 0.0f) {
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    s += sums[i * C::VP + threadIdx.x];
                    zz += sums[ROWS * C::VP + i];
                }
            }
            mu[threadIdx.x] = eps >= 0.0f ? mean_of(s, zz) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < STEPS; ++n) {
            const int row = n * ROWS + slice;
            const float zr = slice < ROWS && row < C::KP ? -z[row] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[n][i] = fmaf(zr, mu[8 * piece + i], x[n][i]);
        }
    }
    float scale = 1.0f;
    if (scaled) {
        float big = 0.0f;
#pragma unroll
        for (int n = 0; n < STEPS; ++n)
#pragma unroll
            for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(x[n][i]));
        scale = pow2_scale(block_max(big, scratch, THREADS / 32), 12);
    }
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
        const int row = n * ROWS + slice;
        if (slice >= ROWS || row >= C::KP) continue;
        uint4 hi, lo;
        split_pair<KIND>(x[n][0] * scale, x[n][1] * scale, &hi.x, &lo.x);
        split_pair<KIND>(x[n][2] * scale, x[n][3] * scale, &hi.y, &lo.y);
        split_pair<KIND>(x[n][4] * scale, x[n][5] * scale, &hi.z, &lo.z);
        split_pair<KIND>(x[n][6] * scale, x[n][7] * scale, &hi.w, &lo.w);
        unsigned char* at = hi_rows + row * C::PITCHV + 16 * piece;
        *reinterpret_cast<uint4*>(at) = hi;
        *reinterpret_cast<uint4*>(at + C::S_HALF) = lo;
    }
    return scale;
}
// A fragment of 16 features (rows m0 ..) x 16 channels (k0 ..) of those rows; and of its transpose: 16 channels (m0 ..) x 16
// features (k0 ..).
__device__ __forceinline__ void state_a(const unsigned char* rows, int pitch, int m0, int k0, int lane, uint32_t (&r)[4])
{
    ldmatrix_x4(smem_u32(rows + (m0 + (lane & 15)) * pitch + (k0 + (lane >> 4) * 8) * 2), r[0], r[1], r[2], r[3]);
}
__device__ __forceinline__ void state_a_transposed(const unsigned char* rows, int pitch, int m0, int k0, int lane, uint32_t (&r)[4])
{
    const int row = k0 + (lane & 7) + ((lane >> 4) & 1) * 8, col = m0 + ((lane >> 3) & 1) * 8;
    ldmatrix_x4_trans(smem_u32(rows + row * pitch + col * 2), r[0], r[1], r[2], r[3]);
}

// B fragments of two groups of eight tokens, contraction over channels k0 .. k0 + 15 of rows [token][channel].
__device__ __forceinline__ void tokens_b(const unsigned char* tile, int pitch, int n0, int k0, int lane, uint32_t (&b)[4])
{
    const int row = n0 + (lane & 7) + ((lane >> 4) & 1) * 8, col = k0 + ((lane >> 3) & 1) * 8;
    ldmatrix_x4(smem_u32(tile + row * pitch + col * 2), b[0], b[1], b[2], b[3]);
}
// B fragments of two groups of eight channels, contraction over tokens k0 .. k0 + 15.
__device__ __forceinline__ void channels_b(const unsigned char* tile, int pitch, int k0, int n0, int lane, uint32_t (&b)[4])
{
    const int row = k0 + (lane & 7) + ((lane >> 3) & 1) * 8, col = n0 + ((lane >> 4) & 1) * 8;
    ldmatrix_x4_trans(smem_u32(tile + row * pitch + col * 2), b[0], b[1], b[2], b[3]);
}
// Where the transposed 16 x 16 block (features m0 .., tokens n0 ..) of rows [token][feature] lies for ldmatrix /
// stmatrix .trans: registers 0, 1: the first eight tokens, rows lane/4 and lane/4 + 8; 2, 3: the next eight.
__device__ __forceinline__ uint32_t transposed_at(const unsigned char* tile, int pitch, int n0, int m0, int lane)
{
    const int row = n0 + (lane & 7) + ((lane >> 4) & 1) * 8, col = m0 + ((lane >> 3) & 1) * 8;
    return smem_u32(tile + row * pitch + col * 2);
}

// ---------------------------------------------------------------------------------------------
// First stream.  GRAD: Q, dY -> dQ, partial dS | dz.  Without GRAD: K, V -> partial S | z (the state itself, for a
// backward pass that was given none).  grid (chunks, slabs); a CTA works through its chunk's tiles.  A warp owns
// 16 features, whose rows of dS stay in its registers:
//     t^T [16 x TILE] = S [16 x dv] dY^T         and        dS [16 x dv] += (w f)^T [16 x TILE] dY
// The accumulators of the first have the layout of the second's left operand: phi, the quotient and the
// difference are done where the numbers lie, and only the two sums per token (den and f . t) cross warps, between two
// passes over the tile's groups of 16 tokens.  S stays in shared memory and the loops over groups and k steps stay loops:
// unrolled, with S in registers, the code was some 90 KB, which a call of one tile per CTA spent its time fetching.
// ---------------------------------------------------------------------------------------------
template <int DK, int DV, int KIND, bool GRAD>
__global__ void __launch_bounds__(32 * BackwardCfg<DK, DV>::WQ)
backward_state_kernel(const __nv_bfloat16* __restrict__ q, const __nv_bfloat16* __restrict__ dy, const float* __restrict__ state,
                      __nv_bfloat16* __restrict__ dq, float* __restrict__ partials, int N, int chunks, SlabLayout Lk,
                      SlabLayout Lv, BackwardScales sc, uint32_t* __restrict__ clear_status)
{
    using C = BackwardCfg<DK, DV>;
    constexpr int TILE = C::TILE, THREADS = 32 * C::WQ;
    extern __shared__ __align__(16) unsigned char smem[];
    unsigned char* s_rows = smem + 2 * C::STAGE;
    float* z = reinterpret_cast<float*>(s_rows + 2 * C::S_HALF);
    float2* sums = reinterpret_cast<float2*>(z + C::KP);        // [WQ][TILE]: den and f . t of a warp's features
    float2* wc = sums + C::WQ * TILE;                           // [TILE]: w and c
    float4* kept = reinterpret_cast<float4*>(wc + TILE);        // t, as the threads hold it: [WQ][TILE / 8][lane]
    float* mu = reinterpret_cast<float*>(kept + C::WQ * TILE * 4);  // [VP]
    __shared__ float scratch[33];
    const int slab = blockIdx.y, chunk = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x & 31, m0 = warp * 16;
    const int tiles = (N + TILE - 1) / TILE;
    const int t_begin = static_cast<int>(static_cast<long long>(chunk) * tiles / chunks);
    const int t_end = static_cast<int>(static_cast<long long>(chunk + 1) * tiles / chunks);
    q += slab_base(Lk, slab);
    dy += slab_base(Lv, slab);
    if (GRAD) dq += slab_base(Lk, slab);

    for (int s = 0; s < 2; ++s) {
        clear_padding<DK, C::PITCHK, TILE, THREADS>(smem + s * C::STAGE);
        clear_padding<DV, C::PITCHV, TILE, THREADS>(smem + s * C::STAGE + TILE * C::PITCHK);
    }
    pdl_launch_dependents();
    pdl_wait();
    if (clear_status != nullptr && blockIdx.x + blockIdx.y + threadIdx.x == 0) *clear_status = kStatusOk;
    auto fetch = [&](int t) {
        unsigned char* st = smem + (t & 1) * C::STAGE;
        load_tile<DK, C::PITCHK, TILE, THREADS>(st, q, Lk.row_stride, t * TILE, N);
        load_tile<DV, C::PITCHV, TILE, THREADS>(st + TILE * C::PITCHK, dy, Lv.row_stride, t * TILE, N);
        cp_async_commit();
    };
    if (t_begin < t_end) fetch(t_begin);

    float scale_s = 1.0f, unscale_t = 1.0f, scale_w[2] = {1.0f, 1.0f};  // of the thread's two features
    if (GRAD) {
        const float* S = state + static_cast<size_t>(slab) * grad_state_floats(DK, DV);
        // fp16: R and w f by powers of two that keep head and tail inside the format.
        scale_s = load_state<KIND, DK, DV, THREADS, true>(S, sc.eps, sc.scaled != 0, s_rows, z, mu, scratch);
        unscale_t = 1.0f / scale_s;
        if (sc.scaled) {
            if (sc.eps >= 0.0f && kind_phi(KIND) == kPhiIdentity) {
                float z_max = 0.0f, z_inv = 0.0f;
                for (int i = threadIdx.x; i < DK; i += THREADS) {
                    const float v = S[DK * DV + i];
                    z_max = fmaxf(z_max, v);
                    z_inv = fmaxf(z_inv, v > 0.0f ? 1.0f / v : 3.0e38f);
                }
                z_max = block_max(z_max, scratch, C::WQ);
                z_inv = block_max(z_inv, scratch, C::WQ);
                scale_w[0] = scale_w[1] = slab_scale(z_max, z_inv, sc.eps);
            } else if (sc.eps >= 0.0f) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int row = m0 + lane / 4 + 8 * r;
                    scale_w[r] = feature_scale(row < DK ? S[DK * DV + row] : 0.0f, sc.eps);
                }
            }
        }
    }
    float acc[C::VP / 8][4];
#pragma unroll
    for (int n = 0; n < C::VP / 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
    float dz[2] = {0.0f, 0.0f};

    for (int t = t_begin; t < t_end; ++t) {
        cp_async_wait_all();
        __syncthreads();  // the tile has landed (and S is in place), and everybody is done with the other stage
        if (t + 1 < t_end) fetch(t + 1);
        unsigned char* tq = smem + (t & 1) * C::STAGE;
        unsigned char* tg = tq + TILE * C::PITCHK;
        float zr[2] = {0.0f, 0.0f};
        if (GRAD) {
            zr[0] = z[m0 + lane / 4];
            zr[1] = z[m0 + lane / 4 + 8];
#pragma unroll 1
            for (int j = 0; j < TILE / 8; j += 2) {  // 16 tokens
                float tt[2][4] = {};
#pragma unroll 2
                for (int s = 0; s < C::VP / 16; ++s) {
                    uint32_t hi[4], lo[4], b[4];
                    state_a(s_rows, C::PITCHV, m0, s * 16, lane, hi);
                    state_a(s_rows + C::S_HALF, C::PITCHV, m0, s * 16, lane, lo);
                    tokens_b(tg, C::PITCHV, j * 8, s * 16, lane, b);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        mma_16816<KIND>(tt[h], lo[0], lo[1], lo[2], lo[3], b[2 * h], b[2 * h + 1]);
                        mma_16816<KIND>(tt[h], hi[0], hi[1], hi[2], hi[3], b[2 * h], b[2 * h + 1]);
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    kept[(warp * (TILE / 8) + j + h) * 32 + lane] = make_float4(tt[h][0], tt[h][1], tt[h][2], tt[h][3]);
                if (sc.eps >= 0.0f) {
                    uint32_t x[4];
                    ldmatrix_x4_trans(transposed_at(tq, C::PITCHK, j * 8, m0, lane), x[0], x[1], x[2], x[3]);
                    float part[8];  // den and f . t of the thread's four tokens
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float den = 0.0f, ft = 0.0f;
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                const float f = phi_or_nan<KIND>(e == 0 ? pair_lo<KIND>(x[2 * h + r]) : pair_hi<KIND>(x[2 * h + r]));
                                den = fmaf(f, zr[r], den);
                                ft = fmaf(f, tt[h][2 * r + e], ft);
                            }
                            part[4 * h + 2 * e] = den;
                            part[4 * h + 2 * e + 1] = ft;
                        }
                    // over the eight lanes of a column: the eight numbers are halved with the lanes, one is left in each
#pragma unroll
                    for (int o = 16, n = 4; o >= 4; o >>= 1, n >>= 1) {
                        const bool up = (lane & o) != 0;
#pragma unroll
                        for (int i = 0; i < n; ++i) {
                            const float keep = up ? part[i + n] : part[i], send = up ? part[i] : part[i + n];
                            part[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                        }
                    }
                    // lane bits 4, 3, 2: group of eight tokens, odd token, f . t
                    const int tok = (j + (lane >> 4)) * 8 + 2 * (lane & 3) + ((lane >> 3) & 1);
                    reinterpret_cast<float*>(sums + warp * TILE + tok)[(lane >> 2) & 1] = part[0];
                }
            }
            if (sc.eps >= 0.0f) {
                __syncthreads();
                for (int i = threadIdx.x; i < TILE; i += THREADS) {
                    float den = 0.0f, ft = 0.0f;
#pragma unroll
                    for (int k = 0; k < C::WQ; ++k) {
                        const float2 o = sums[k * TILE + i];
                        den += o.x;
                        ft += o.y;
                    }
                    const bool in = t * TILE + i < N;
                    const float w = in ? 1.0f / (den + sc.eps) : 0.0f;
                    if (w * sc.eps >= kEpsCounts) {
                        float mg = 0.0f;
#pragma unroll 1
                        for (int j = 0; j < DV / 8; ++j)
                            mg = mean_dot<KIND>(*reinterpret_cast<const uint4*>(tg + i * C::PITCHV + 16 * j), mu + 8 * j, mg);
                        ft = fmaf(-sc.eps * scale_s, mg, ft);
                    }
                    wc[i] = make_float2(w, in ? ft * w : 0.0f);  // c scaled as S is
                }
                __syncthreads();
            }
        }
#pragma unroll 1
        for (int j = 0; j < TILE / 8; j += 2) {
            uint32_t x[4], a_hi[4], a_lo[4], out[4];
            const uint32_t at = transposed_at(tq, C::PITCHK, j * 8, m0, lane);
            ldmatrix_x4_trans(at, x[0], x[1], x[2], x[3]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float4 tt = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (GRAD) tt = kept[(warp * (TILE / 8) + j + h) * 32 + lane];
                const float tv[4] = {tt.x, tt.y, tt.z, tt.w};
                float wf[2][2], d[2][2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int tok = (j + h) * 8 + 2 * (lane & 3) + e;
                    float w = t * TILE + tok < N ? 1.0f : 0.0f, c = 0.0f;
                    if (GRAD && sc.eps >= 0.0f) {
                        const float2 o = wc[tok];
                        w = o.x;
                        c = o.y;
                    }
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float v = e == 0 ? pair_lo<KIND>(x[2 * h + r]) : pair_hi<KIND>(x[2 * h + r]);
                        float f, slope;
                        phi_and_slope<KIND>(v, &f, &slope);
                        wf[r][e] = w * f;
                        if (GRAD) {
                            d[r][e] = slope * (w * ((tv[2 * r + e] - c * zr[r]) * unscale_t));
                            dz[r] = fmaf(-wf[r][e], c * unscale_t, dz[r]);
                        } else {
                            dz[r] += wf[r][e];
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    split_pair<KIND>(wf[r][0] * scale_w[r], wf[r][1] * scale_w[r], &a_hi[2 * h + r], &a_lo[2 * h + r]);
                    if (GRAD) out[2 * h + r] = pack_pair<KIND>(d[r][0], d[r][1]);
                }
            }
            if (GRAD) stmatrix_x4_trans(at, out[0], out[1], out[2], out[3]);
#pragma unroll
            for (int n = 0; n < C::VP / 16; ++n) {
                uint32_t b[4];
                channels_b(tg, C::PITCHV, j * 8, n * 16, lane, b);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    mma_16816<KIND>(acc[2 * n + h], a_lo[0], a_lo[1], a_lo[2], a_lo[3], b[2 * h], b[2 * h + 1]);
                    mma_16816<KIND>(acc[2 * n + h], a_hi[0], a_hi[1], a_hi[2], a_hi[3], b[2 * h], b[2 * h + 1]);
                }
            }
        }
        if (GRAD) {
            __syncthreads();  // dQ of all features is in place of Q
            store_tile<DK, C::PITCHK, TILE, THREADS>(tq, dq, Lk.row_stride, t * TILE, N);
        }
    }
    float* out = partials + (static_cast<size_t>(slab) * chunks + chunk) * grad_state_floats(DK, DV);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = m0 + lane / 4 + 8 * r;
        const float unscale_w = 1.0f / scale_w[r];
#pragma unroll
        for (int n = 0; n < C::VP / 8; ++n) {
            const int col = n * 8 + 2 * (lane & 3);
            if (GRAD && sc.eps >= 0.0f) dz[r] = fmaf(-unscale_w, fmaf(acc[n][2 * r], mu[col], acc[n][2 * r + 1] * mu[col + 1]), dz[r]);
            if (row < DK && col < DV)
                *reinterpret_cast<float2*>(out + row * DV + col) = make_float2(acc[n][2 * r] * unscale_w, acc[n][2 * r + 1] * unscale_w);
        }
        dz[r] += __shfl_xor_sync(0xffffffffu, dz[r], 1);
        dz[r] += __shfl_xor_sync(0xffffffffu, dz[r], 2);
        if ((lane & 3) == 0 && row < DK) out[DK * DV + row] = dz[r];
    }
}

// Sum of a slab's partials.  A block of 256 has 256 / SLICES numbers of the state; SLICES threads for each take every
// SLICES-th chunk in order and are added in order.  Eight where a slab has many chunks (one thread for up to 444 of them took
// 23 us), one where it has a few (eight made 66000 blocks of 128 slabs x 128 x 128: 307 against 94 us in all).
constexpr int kReduceThreads = 256;
__host__ __device__ constexpr int reduce_slices_for(int chunks) { return chunks <= 3 ? 1 : chunks <= 6 ? 4 : 8; }
__device__ __forceinline__ float4 add4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
template <int SLICES>
__device__ __forceinline__ float4 reduce_slices(float4 sum, float4* scratch)
{
    if (SLICES == 1) return sum;
    constexpr int OUT = kReduceThreads / SLICES;
    scratch[threadIdx.x] = sum;
    __syncthreads();
    sum = scratch[threadIdx.x % OUT];
#pragma unroll
    for (int i = 1; i < SLICES; ++i) sum = add4(sum, scratch[i * OUT + threadIdx.x % OUT]);
    return sum;
}
// Blocks that write `floats` sums (a multiple of 8), four to a thread.
__host__ __device__ constexpr int reduce_blocks(int floats, int slices) { return (floats / 4 + kReduceThreads / slices - 1) / (kReduceThreads / slices); }
template <int SLICES>
static __global__ void __launch_bounds__(kReduceThreads)
backward_reduce_kernel(const float* __restrict__ partials, float* __restrict__ out, int floats, int chunks)
{
    constexpr int OUT = kReduceThreads / SLICES;
    __shared__ float4 scratch[kReduceThreads];
    const int slice = threadIdx.x / OUT, i = 4 * (blockIdx.x * OUT + threadIdx.x % OUT);
    pdl_launch_dependents();
    pdl_wait();
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (i < floats) {
        const float* p = partials + static_cast<size_t>(blockIdx.y) * chunks * floats + i;
#pragma unroll 4
        for (int c = slice; c < chunks; c += SLICES) s = add4(s, *reinterpret_cast<const float4*>(p + static_cast<size_t>(c) * floats));
    }
    s = reduce_slices<SLICES>(s, scratch);
    if (slice == 0 && i < floats) *reinterpret_cast<float4*>(out + static_cast<size_t>(blockIdx.y) * floats + i) = s;
}

// ---------------------------------------------------------------------------------------------
// Second stream: K, V -> dK, dV with dS | dz at hand.  A warp owns 16 features of dK and 16 channels of dV:
//     dK^T [16 x TILE] = dS [16 x dv] V^T + dz          dV^T [16 x TILE] = dS^T [16 x dk] phi(K)^T
// phi(K) crosses warps through shared memory as head and tail.
// ---------------------------------------------------------------------------------------------
template <int DK, int DV, int KIND>
__global__ void __launch_bounds__(32 * BackwardCfg<DK, DV>::WKV)
backward_kv_kernel(const __nv_bfloat16* __restrict__ k, const __nv_bfloat16* __restrict__ v, const float* __restrict__ grad_state,
                   __nv_bfloat16* __restrict__ dk, __nv_bfloat16* __restrict__ dv, int N, int chunks, SlabLayout Lk,
                   SlabLayout Lv, BackwardScales sc, uint32_t* __restrict__ clear_status)
{
    using C = BackwardCfg<DK, DV>;
    constexpr int TILE = C::TILE, THREADS = 32 * C::WKV;
    extern __shared__ __align__(16) unsigned char smem[];
    unsigned char* s_rows = smem + 2 * C::STAGE;
    unsigned char* f_hi = s_rows + 2 * C::S_HALF;
    unsigned char* f_lo = f_hi + TILE * C::PITCHK;
    float* z = reinterpret_cast<float*>(f_lo + TILE * C::PITCHK);
    __shared__ float scratch[33];
    const int slab = blockIdx.y, chunk = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x & 31, m0 = warp * 16;
    const int tiles = (N + TILE - 1) / TILE;
    const int t_begin = static_cast<int>(static_cast<long long>(chunk) * tiles / chunks);
    const int t_end = static_cast<int>(static_cast<long long>(chunk + 1) * tiles / chunks);
    k += slab_base(Lk, slab);
    dk += slab_base(Lk, slab);
    v += slab_base(Lv, slab);
    dv += slab_base(Lv, slab);
    for (int s = 0; s < 2; ++s) {
        clear_padding<DK, C::PITCHK, TILE, THREADS>(smem + s * C::STAGE);
        clear_padding<DV, C::PITCHV, TILE, THREADS>(smem + s * C::STAGE + TILE * C::PITCHK);
    }
    pdl_launch_dependents();
    pdl_wait();
    if (clear_status != nullptr && blockIdx.x + blockIdx.y + threadIdx.x == 0) *clear_status = kStatusOk;
    auto fetch = [&](int t) {
        unsigned char* st = smem + (t & 1) * C::STAGE;
        load_tile<DK, C::PITCHK, TILE, THREADS>(st, k, Lk.row_stride, t * TILE, N);
        load_tile<DV, C::PITCHV, TILE, THREADS>(st + TILE * C::PITCHK, v, Lv.row_stride, t * TILE, N);
        cp_async_commit();
    };
    if (t_begin < t_end) fetch(t_begin);

    const float* S = grad_state + static_cast<size_t>(slab) * grad_state_floats(DK, DV);
    const float unscale = 1.0f / load_state<KIND, DK, DV, THREADS, false>(S, -1.0f, sc.scaled != 0, s_rows, z, nullptr, scratch);

    for (int t = t_begin; t < t_end; ++t) {
        cp_async_wait_all();
        __syncthreads();
        if (t + 1 < t_end) fetch(t + 1);
        unsigned char* tk = smem + (t & 1) * C::STAGE;
        unsigned char* tv = tk + TILE * C::PITCHK;
        if (m0 < C::KP) {
            const float dz[2] = {z[m0 + lane / 4], z[m0 + lane / 4 + 8]};
#pragma unroll 1
            for (int j = 0; j < TILE / 8; j += 2) {
                float acc[2][4] = {};
#pragma unroll 2
                for (int s = 0; s < C::VP / 16; ++s) {
                    uint32_t a_hi[4], a_lo[4], b[4];
                    state_a(s_rows, C::PITCHV, m0, s * 16, lane, a_hi);
                    state_a(s_rows + C::S_HALF, C::PITCHV, m0, s * 16, lane, a_lo);
                    tokens_b(tv, C::PITCHV, j * 8, s * 16, lane, b);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        mma_16816<KIND>(acc[h], a_lo[0], a_lo[1], a_lo[2], a_lo[3], b[2 * h], b[2 * h + 1]);
                        mma_16816<KIND>(acc[h], a_hi[0], a_hi[1], a_hi[2], a_hi[3], b[2 * h], b[2 * h + 1]);
                    }
                }
                uint32_t x[4], hi[4], lo[4], out[4];
                const uint32_t at = transposed_at(tk, C::PITCHK, j * 8, m0, lane);
                ldmatrix_x4_trans(at, x[0], x[1], x[2], x[3]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {  // i = 2 * (group of eight tokens) + (row of the fragment)
                    const int r = i & 1;
                    float f0, f1, s0, s1;
                    phi_and_slope<KIND>(pair_lo<KIND>(x[i]), &f0, &s0);
                    phi_and_slope<KIND>(pair_hi<KIND>(x[i]), &f1, &s1);
                    split_pair<KIND>(f0, f1, &hi[i], &lo[i]);
                    out[i] = pack_pair<KIND>(s0 * fmaf(acc[i / 2][2 * r], unscale, dz[r]),
                                             s1 * fmaf(acc[i / 2][2 * r + 1], unscale, dz[r]));
                }
                stmatrix_x4_trans(transposed_at(f_hi, C::PITCHK, j * 8, m0, lane), hi[0], hi[1], hi[2], hi[3]);
                stmatrix_x4_trans(transposed_at(f_lo, C::PITCHK, j * 8, m0, lane), lo[0], lo[1], lo[2], lo[3]);
                stmatrix_x4_trans(at, out[0], out[1], out[2], out[3]);
            }
        }
        __syncthreads();  // phi(K) and dK are in place; V has been read
        if (m0 < C::VP) {
#pragma unroll 1
            for (int j = 0; j < TILE / 8; j += 2) {
                float acc[2][4] = {};
#pragma unroll 2
                for (int s = 0; s < C::KP / 16; ++s) {
                    uint32_t a_hi[4], a_lo[4], b[4], bl[4];
                    state_a_transposed(s_rows, C::PITCHV, m0, s * 16, lane, a_hi);
                    state_a_transposed(s_rows + C::S_HALF, C::PITCHV, m0, s * 16, lane, a_lo);
                    tokens_b(f_hi, C::PITCHK, j * 8, s * 16, lane, b);
                    tokens_b(f_lo, C::PITCHK, j * 8, s * 16, lane, bl);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        mma_16816<KIND>(acc[h], a_lo[0], a_lo[1], a_lo[2], a_lo[3], b[2 * h], b[2 * h + 1]);
                        mma_16816<KIND>(acc[h], a_hi[0], a_hi[1], a_hi[2], a_hi[3], bl[2 * h], bl[2 * h + 1]);
                        mma_16816<KIND>(acc[h], a_hi[0], a_hi[1], a_hi[2], a_hi[3], b[2 * h], b[2 * h + 1]);
                    }
                }
                uint32_t out[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    out[i] = pack_pair<KIND>(acc[i / 2][2 * (i & 1)] * unscale, acc[i / 2][2 * (i & 1) + 1] * unscale);
                stmatrix_x4_trans(transposed_at(tv, C::PITCHV, j * 8, m0, lane), out[0], out[1], out[2], out[3]);
            }
        }
        __syncthreads();
        store_tile<DK, C::PITCHK, TILE, THREADS>(tk, dk, Lk.row_stride, t * TILE, N);
        store_tile<DV, C::PITCHV, TILE, THREADS>(tv, dv, Lv.row_stride, t * TILE, N);
    }
}

}  // namespace lf
