// Host side of the backward pass declared in include/linfusion_attn.h: argument checks, the fixed split of
// the tokens, workspace layout and launches.
#include "../../include/linfusion_attn.h"

#include "backward_kernels.cuh"
#include "backward_tc_kernels.cuh"
#include "backward_tc_wide_kernels.cuh"
#include "host_util.h"

using namespace lf;

namespace {

int feature_width(const linfusion_attn_desc_t& d) { return d.d_qk > 0 ? d.d_qk : d.d; }

int kernel_kind(const linfusion_attn_desc_t& d)
{
    return make_kind(d.phi == LINFUSION_PHI_IDENTITY ? kPhiIdentity : kPhiEluPlusOne,
                     (d.flags & LINFUSION_DTYPE_FP16) != 0u ? kDtypeFp16 : kDtypeBf16);
}

SlabLayout slab_layout(const linfusion_attn_desc_t& d, int width)
{
    SlabLayout L;
    L.H = d.H;
    if ((d.flags & LINFUSION_LAYOUT_TOKEN_MAJOR) != 0u) {
        L.batch_stride = static_cast<long long>(d.N) * d.H * width;
        L.head_stride = width;
        L.row_stride = d.H * width;
    } else {
        L.batch_stride = static_cast<long long>(d.H) * d.N * width;
        L.head_stride = static_cast<long long>(d.N) * width;
        L.row_stride = width;
    }
    return L;
}

constexpr int kPlanSms = 148;  // a B200's, where no count is given

// What follows from (descriptor, SM count) alone.
struct BackwardPlan {
    int slabs, dk, dv, floats;  // floats of S | z of a slab
    int chunks_q, chunks_kv;    // CTAs per slab of the two streams
    int tc;                     // the tcgen05 kernels' cut: 0 (none for these widths), 1 (40 or 64 channels), 2 (features up to 128)
    bool tc_state, tc_q, tc_kv; // the streams that they take
    size_t tc_partial;          // ... floats of a partial
    int tiles_per_slab, ctas, spans;  // ... their tiles of a slab, CTAs, and slabs that a CTA meets at most
    long long tiles;
    size_t partials_off, state_off, grad_off, total;  // behind a status word
};

// CTAs per slab of the warp-level kernels: the fewest whose longest run of tiles ends first, with as many CTAs at a time
// as shared memory admits and a tile's time for laying out the state.  (Filling the SMs regardless of where tiles and waves
// end cost 41 us where this takes 31 at 20 slabs x 1024 x 64, 57 where this takes 40 at 128 x 256 x 64.)
template <int DK, int DV>
void plan_chunks(const linfusion_attn_desc_t& d, int sm_count, BackwardPlan* p)
{
    using C = BackwardCfg<DK, DV>;
    constexpr int kSmem = C::SMEM_Q > C::SMEM_KV ? C::SMEM_Q : C::SMEM_KV, kPerSm = 228 * 1024 / (kSmem + 1024);
    const long long tiles = (d.N + C::TILE - 1) / C::TILE, at_once = static_cast<long long>(kPerSm) * sm_count;
    long long best = 0;
    p->chunks_q = p->chunks_kv = 1;
    for (long long c = 1; c <= tiles && (c == 1 || p->slabs * (c - 1) < at_once); ++c) {
        const long long longest = (tiles + c - 1) / c, cost = (p->slabs * c + at_once - 1) / at_once * (longest + 1);
        if (c == 1 || cost < best) {
            best = cost;
            p->chunks_q = p->chunks_kv = static_cast<int>(c);
        }
    }
}

#define LF_DISPATCH_WIDTHS(dk, dv, CALL)  \
    switch ((dk) * 1000 + (dv)) {         \
        case 32032: CALL(32, 32); break;   \
        case 40040: CALL(40, 40); break;   \
        case 64064: CALL(64, 64); break;   \
        case 80080: CALL(80, 80); break;   \
        case 128128: CALL(128, 128); break; \
        case 160160: CALL(160, 160); break; \
        case 128064: CALL(128, 64); break; \
        case 80040: CALL(80, 40); break;   \
        case 32064: CALL(32, 64); break;   \
        default: break;                    \
    }

// Which streams the tcgen05 kernels take (us, tcgen05 / warp-level, slabs x N x widths; a replayed graph of the stream alone):
//   state   15 / 16 at 20 x 4096 x 64, 13 / 10 at 20 x 2048 x 64, 67 / 149 at 16 x 65536 x 64; 58 / 67 at 16 x 16384 x 128,
//           41 / 39 at 16 x 8192 x 128; 79 / 84 at 16 x 32768 x 80, 50 / 46 at 16 x 16384 x 80
//   q       14.4 / 17.2 at 20 x 2048 x 64, 12.6 / 11.8 at 20 x 1024 x 64, 113 / 214 at 16 x 65536 x 64; 65 / 84 at 16 x 8192 x 128,
//           44 / 49 at 16 x 4096 x 128; 76 / 79 at 16 x 16384 x 80/40, but 161 / 160 at 16 x 32768 x 80, whose 80 are padded to 128 twice
//   kv      12.6 / 19.6 at 20 x 4096 x 64, 6.3 / 7.4 at 128 x 64 x 64; 12.9 / 14.9 at 16 x 1024 x 128, 12.3 / 9.3 at 16 x 512 x 128
// Widths of 32, padded to 64: 123 / 105, 211 / 168, 181 / 146 at 32 x 65536.  Short slabs: where a CTA changes its state every
// tile, state and q take 73 / 15 and 69 / 40 at 1024 x 128 x 64, 245 / 44 and 199 / 112 at 1024 x 128 x 128, kv still 27 / 40 and
// 82 / 113, but 25 / 21 at 1024 x 16 x 64.
void plan_tc(const linfusion_attn_desc_t& d, int sm_count, BackwardPlan* p)
{
    p->tiles_per_slab = (d.N + kTcTile - 1) / kTcTile;
    p->tiles = static_cast<long long>(p->slabs) * p->tiles_per_slab;
    p->tc = p->dk <= 32 && p->dv <= 32 ? 0 : p->dk <= 64 && p->dv <= 64 ? 1 : p->dk <= 128 && p->dv <= 128 ? 2 : 0;
    p->tc_state = p->tc_q = p->tc_kv = false;
    const double work = static_cast<double>(p->slabs) * d.N * p->dk * p->dv / sm_count, tiles = static_cast<double>(p->tiles) / sm_count;
    if (p->tc == 1) {
        p->tc_state = p->tiles_per_slab >= 16 && work >= 2.2e6;
        p->tc_q = p->tiles_per_slab >= 4 && work >= 1e6;
        p->tc_kv = d.N >= 64;
    } else if (p->tc == 2) {
        const bool padded = p->dk < 128;
        p->tc_state = p->tiles_per_slab >= 16 && tiles >= (p->dv <= 64 ? 4.0 : padded ? 16.0 : 8.0);
        p->tc_q = p->tiles_per_slab >= 8 && tiles >= (padded ? 12.0 : 3.0) && !(padded && p->dv > 64);
        p->tc_kv = d.N >= 64 && tiles >= 0.75;
    }
    p->tc_partial = p->tc == 1 ? BackwardTc::PARTIAL_FLOATS : p->dv > 64 ? BackwardTcWide<2>::PARTIAL_FLOATS : BackwardTcWide<1>::PARTIAL_FLOATS;
    if (!(p->tc_state || p->tc_q || p->tc_kv)) return;
    p->ctas = static_cast<int>(p->tiles < sm_count ? p->tiles : sm_count);
    // The same number of CTAs on every slab where that lengthens the longest run by three tiles at most: a CTA that meets a
    // second slab fetches another state and hands back another partial, some 4 us (44 / 38 us at 20 slabs x 4096 x 64; 193 / 216 at
    // 40 x 16384 x 64, whose 128 tiles on three CTAs each would leave 28 SMs without any).
    const int each = sm_count / p->slabs;
    if (each > 0 && each * p->slabs <= p->ctas &&
        (p->tiles_per_slab + each - 1) / each <= (p->tiles + p->ctas - 1) / p->ctas + 3)
        p->ctas = each * p->slabs;
    // a run of L tiles meets at most this many slabs
    const long long L = (p->tiles + p->ctas - 1) / p->ctas;
    p->spans = static_cast<int>((L + p->tiles_per_slab - 2) / p->tiles_per_slab) + 1;
}

linfusion_status_t make_backward_plan(const linfusion_attn_desc_t* desc, int sm_count, BackwardPlan* p)
{
    if (desc == nullptr) return LINFUSION_ERR_INVALID_ARG;
    // The checks of create(); the forward variant plays no part here.
    if ((desc->flags & LINFUSION_VARIANT_MASK) > LINFUSION_VARIANT_FUSED) return LINFUSION_ERR_UNSUPPORTED;
    linfusion_attn_desc_t d = *desc;
    d.flags = (d.flags & ~LINFUSION_VARIANT_MASK) | LINFUSION_VARIANT_SPLIT;
    size_t unused = 0;
    const linfusion_status_t st = linfusion_attn_workspace_bytes(&d, sm_count, &unused);
    if (st != LINFUSION_OK) return st;
    if (sm_count <= 0) sm_count = kPlanSms;
    p->slabs = d.B * d.H;
    p->dk = feature_width(d);
    p->dv = d.d;
    p->floats = grad_state_floats(p->dk, p->dv);
#define LF_CALL(DK, DV) plan_chunks<DK, DV>(d, sm_count, p)
    LF_DISPATCH_WIDTHS(p->dk, p->dv, LF_CALL)
#undef LF_CALL
    plan_tc(d, sm_count, p);
    const size_t slab_state = static_cast<size_t>(p->slabs) * p->floats * sizeof(float), state = align_up_256(slab_state);
    p->state_off = 256;
    p->grad_off = p->state_off + state;
    p->partials_off = p->grad_off + state;
    const size_t warp_level = slab_state * static_cast<size_t>(p->chunks_q);
    const size_t tc = p->tc_state || p->tc_q ? static_cast<size_t>(p->ctas) * p->spans * p->tc_partial * sizeof(float) : 0;
    p->total = p->partials_off + align_up_256(p->tc_state && p->tc_q || tc > warp_level ? tc : warp_level);
    return LINFUSION_OK;
}

template <int DK, int DV, int KIND, bool GRAD>
cudaError_t launch_state(const linfusion_attn_desc_t& d, const BackwardPlan& p, const void* q, const void* dy, const float* state,
                         void* dq, float* partials, float* out, uint32_t* clear, cudaStream_t s)
{
    using C = BackwardCfg<DK, DV>;
    static std::atomic<uint64_t> done{0};
    cudaError_t e = allow_smem(backward_state_kernel<DK, DV, KIND, GRAD>, GRAD ? C::SMEM_Q : C::SMEM_STATE, d.device, &done);
    if (e != cudaSuccess) return e;
    BackwardScales sc;
    sc.eps = (d.flags & LINFUSION_FLAG_UNNORMALIZED) != 0u ? kEpsUnnormalized : d.eps;
    sc.scaled = kind_dtype(KIND) == kDtypeFp16 ? 1 : 0;
    e = launch_pdl(backward_state_kernel<DK, DV, KIND, GRAD>, dim3(p.chunks_q, p.slabs), dim3(32 * C::WQ),
                   GRAD ? C::SMEM_Q : C::SMEM_STATE, s,
                   static_cast<const __nv_bfloat16*>(q), static_cast<const __nv_bfloat16*>(dy), state,
                   static_cast<__nv_bfloat16*>(dq), p.chunks_q == 1 ? out : partials, d.N, p.chunks_q, slab_layout(d, DK),
                   slab_layout(d, DV), sc, clear);
    if (e != cudaSuccess || p.chunks_q == 1) return e;
#define LF_REDUCE(S)                                                                                                               \
    launch_pdl(backward_reduce_kernel<S>, dim3(reduce_blocks(p.floats, S), p.slabs), dim3(kReduceThreads), 0, \
               s, partials, out, p.floats, p.chunks_q)
    const int slices = reduce_slices_for(p.chunks_q);
    return slices == 1 ? LF_REDUCE(1) : slices == 4 ? LF_REDUCE(4) : LF_REDUCE(8);
#undef LF_REDUCE
}

template <int DK, int DV, int KIND>
cudaError_t launch_kv(const linfusion_attn_desc_t& d, const BackwardPlan& p, const void* k, const void* v, const float* grad_state,
                      void* dk, void* dv, uint32_t* clear, cudaStream_t s)
{
    using C = BackwardCfg<DK, DV>;
    static std::atomic<uint64_t> done{0};
    cudaError_t e = allow_smem(backward_kv_kernel<DK, DV, KIND>, C::SMEM_KV, d.device, &done);
    if (e != cudaSuccess) return e;
    BackwardScales sc;
    sc.eps = d.eps;
    sc.scaled = kind_dtype(KIND) == kDtypeFp16 ? 1 : 0;
    return launch_pdl(backward_kv_kernel<DK, DV, KIND>, dim3(p.chunks_kv, p.slabs), dim3(32 * C::WKV), C::SMEM_KV, s,
                      static_cast<const __nv_bfloat16*>(k), static_cast<const __nv_bfloat16*>(v), grad_state,
                      static_cast<__nv_bfloat16*>(dk), static_cast<__nv_bfloat16*>(dv), d.N, p.chunks_kv, slab_layout(d, DK),
                      slab_layout(d, DV), sc, clear);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// A dense tensor of `width` channels as (channel, token, head, batch) -> boxes of 64 channels x a tile's tokens of one
// slab in the 128-byte swizzle.  What lies past the width or past N is read as zero and not written.
bool encode_map(CUtensorMap* map, const void* base, const linfusion_attn_desc_t& d, int width)
{
    static std::atomic<EncodeTiledFn> known{nullptr};
    EncodeTiledFn fn = known.load(std::memory_order_acquire);
    if (fn == nullptr) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return false;
        fn = reinterpret_cast<EncodeTiledFn>(p);
        known.store(fn, std::memory_order_release);
    }
    const SlabLayout L = slab_layout(d, width);
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(width), static_cast<cuuint64_t>(d.N), static_cast<cuuint64_t>(d.H),
                                static_cast<cuuint64_t>(d.B)};
    const cuuint64_t strides[3] = {static_cast<cuuint64_t>(L.row_stride) * 2, static_cast<cuuint64_t>(L.head_stride) * 2,
                                   static_cast<cuuint64_t>(L.batch_stride) * 2};
    const cuuint32_t box[4] = {64u, kTcTile, 1u, 1u}, step[4] = {1u, 1u, 1u, 1u};
    // Rows of a slab that follow one another: 256 bytes per miss.  Rows between other heads' rows: what the box needs.
    const CUtensorMapL2promotion promo = (d.flags & LINFUSION_LAYOUT_TOKEN_MAJOR) != 0u ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B
                                                                                        : CU_TENSOR_MAP_L2_PROMOTION_L2_256B;
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, step,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, promo, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The kernel of one of the three cuts: widths up to 64, or two feature atoms with one or two value atoms.
template <typename K, typename... Args>
cudaError_t launch_tc(K* kernel, int smem, int threads, std::atomic<uint64_t>* done, const linfusion_attn_desc_t& d, const BackwardPlan& p,
                      cudaStream_t s, Args... args)
{
    const cudaError_t e = allow_smem(kernel, smem, d.device, done);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3(p.ctas), dim3(threads), smem, s, args...);
}

template <int KIND, bool GRAD>
cudaError_t launch_tc_state(const linfusion_attn_desc_t& d, const BackwardPlan& p, const void* q, const void* dy, const float* state,
                            void* dq, float* partials, float* out, uint32_t* status, bool clear, cudaStream_t s)
{
    static std::atomic<uint64_t> done[3];
    CUtensorMap mq, mg, mdq;
    if (!encode_map(&mq, q, d, p.dk) || !encode_map(&mg, dy, d, p.dv) || !encode_map(&mdq, GRAD ? dq : q, d, p.dk))
        return cudaErrorInvalidValue;
    BackwardScales sc;
    sc.eps = (d.flags & LINFUSION_FLAG_UNNORMALIZED) != 0u ? kEpsUnnormalized : d.eps;
    sc.scaled = kind_dtype(KIND) == kDtypeFp16 ? 1 : 0;
    const int first = clear ? 1 : 0;
#define LF_STATE(KERNEL, SMEM, THREADS, I)                                                                                             \
    launch_tc(KERNEL, SMEM, THREADS, &done[I], d, p, s, mq, mg, mdq, state, partials, status, d.N, p.dk, p.dv, p.tiles_per_slab, p.tiles, \
              p.spans, d.H, sc, first)
    const cudaError_t e =
        p.tc == 1     ? LF_STATE((backward_tc_state_kernel<KIND, GRAD>), BackwardTc::STATE_SMEM, BackwardTc::STATE_THREADS, 0)
        : p.dv <= 64 ? LF_STATE((backward_tc_wide_state_kernel<KIND, 1, GRAD>), BackwardTcWide<1>::SMEM, BackwardTcWide<1>::THREADS, 1)
                     : LF_STATE((backward_tc_wide_state_kernel<KIND, 2, GRAD>), BackwardTcWide<2>::SMEM, BackwardTcWide<2>::THREADS, 2);
#undef LF_STATE
    if (e != cudaSuccess) return e;
#define LF_REDUCE(S)                                                                                                                  \
    launch_pdl(backward_tc_reduce_kernel<S>, dim3(reduce_blocks(p.floats, S), p.slabs), dim3(kReduceThreads), 0, \
               s, partials, out, p.dk, p.dv, p.tiles_per_slab, p.tiles, p.ctas, p.spans, p.dv <= 64 ? 64 : 128, p.tc)
    const int slices = reduce_slices_for(p.ctas / p.slabs + 1);
    return slices == 1 ? LF_REDUCE(1) : slices == 4 ? LF_REDUCE(4) : LF_REDUCE(8);
#undef LF_REDUCE
}

template <int KIND>
cudaError_t launch_tc_kv(const linfusion_attn_desc_t& d, const BackwardPlan& p, const void* k, const void* v, const float* grad_state,
                         void* dk, void* dv, uint32_t* status, bool clear, cudaStream_t s)
{
    static std::atomic<uint64_t> done[3];
    CUtensorMap mk, mv, mdk, mdv;
    if (!encode_map(&mk, k, d, p.dk) || !encode_map(&mv, v, d, p.dv) || !encode_map(&mdk, dk, d, p.dk) || !encode_map(&mdv, dv, d, p.dv))
        return cudaErrorInvalidValue;
    BackwardScales sc;
    sc.eps = d.eps;
    sc.scaled = kind_dtype(KIND) == kDtypeFp16 ? 1 : 0;
    const int first = clear ? 1 : 0;
#define LF_KV(KERNEL, SMEM, THREADS, I)                                                                                                   \
    launch_tc(KERNEL, SMEM, THREADS, &done[I], d, p, s, mk, mv, mdk, mdv, grad_state, status, d.N, p.dk, p.dv, p.tiles_per_slab, p.tiles, d.H, \
              sc, first)
    return p.tc == 1     ? LF_KV((backward_tc_kv_kernel<KIND>), BackwardTc::KV_SMEM, BackwardTc::KV_THREADS, 0)
           : p.dv <= 64 ? LF_KV((backward_tc_wide_kv_kernel<KIND, 1>), BackwardTcWide<1>::SMEM, BackwardTcWide<1>::THREADS, 1)
                        : LF_KV((backward_tc_wide_kv_kernel<KIND, 2>), BackwardTcWide<2>::SMEM, BackwardTcWide<2>::THREADS, 2);
#undef LF_KV
}

#define LF_DISPATCH_KINDS(kind, CALL) \
    switch (kind) {                   \
        case 0: CALL(0); break;       \
        case 1: CALL(1); break;       \
        case 2: CALL(2); break;       \
        case 3: CALL(3); break;       \
        default: break;               \
    }

// grad: Q, dY -> dQ and dS | dz.  Otherwise K, V -> S | z.  `first`: of the call's kernels (it clears the status word).
template <bool GRAD>
cudaError_t run_state(const linfusion_attn_desc_t& d, const BackwardPlan& p, const void* q, const void* dy, const float* state,
                      void* dq, unsigned char* ws, float* out, bool first, cudaStream_t s)
{
    cudaError_t e = cudaErrorInvalidValue;
    uint32_t* status = reinterpret_cast<uint32_t*>(ws);
    float* partials = reinterpret_cast<float*>(ws + p.partials_off);
    if (GRAD ? p.tc_q : p.tc_state) {
#define LF_KIND(KV) e = launch_tc_state<KV, GRAD>(d, p, q, dy, state, dq, partials, out, status, first, s)
        LF_DISPATCH_KINDS(kernel_kind(d), LF_KIND)
#undef LF_KIND
        return e;
    }
#define LF_KIND(KV) e = launch_state<kDK, kDV, KV, GRAD>(d, p, q, dy, state, dq, partials, out, first ? status : nullptr, s)
#define LF_CALL(DKV, DVV)                          \
    {                                              \
        constexpr int kDK = DKV, kDV = DVV;        \
        LF_DISPATCH_KINDS(kernel_kind(d), LF_KIND) \
    }
    LF_DISPATCH_WIDTHS(p.dk, p.dv, LF_CALL)
#undef LF_CALL
#undef LF_KIND
    return e;
}

cudaError_t run_kv(const linfusion_attn_desc_t& d, const BackwardPlan& p, const void* k, const void* v, const float* grad_state,
                   void* dk, void* dv, unsigned char* ws, bool first, cudaStream_t s)
{
    cudaError_t e = cudaErrorInvalidValue;
    uint32_t* status = reinterpret_cast<uint32_t*>(ws);
    if (p.tc_kv) {
#define LF_KIND(KV) e = launch_tc_kv<KV>(d, p, k, v, grad_state, dk, dv, status, first, s)
        LF_DISPATCH_KINDS(kernel_kind(d), LF_KIND)
#undef LF_KIND
        return e;
    }
#define LF_KIND(KV) e = launch_kv<kDK, kDV, KV>(d, p, k, v, grad_state, dk, dv, first ? status : nullptr, s)
#define LF_CALL(DKV, DVV)                          \
    {                                              \
        constexpr int kDK = DKV, kDV = DVV;        \
        LF_DISPATCH_KINDS(kernel_kind(d), LF_KIND) \
    }
    LF_DISPATCH_WIDTHS(p.dk, p.dv, LF_CALL)
#undef LF_CALL
#undef LF_KIND
    return e;
}

struct Span {
    const void* p;
    size_t bytes;
    bool output;
};

// Every pointer set and aligned; no output overlaps an input or another output.
bool spans_ok(const Span* spans, int n)
{
    for (int i = 0; i < n; ++i)
        if (spans[i].p == nullptr || !is_aligned(spans[i].p, 16)) return false;
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if ((spans[i].output || spans[j].output) && overlaps(spans[i].p, spans[i].bytes, spans[j].p, spans[j].bytes))
                return false;
    return true;
}

struct Call {
    BackwardPlan plan;
    size_t bytes_qk, bytes_vy, bytes_state;
    linfusion_status_t st;
};

// The plan for the descriptor's device and the checks every entry point makes first.
Call begin(const linfusion_attn_desc_t* desc, const void* workspace, size_t workspace_bytes)
{
    Call c = {};
    c.st = make_backward_plan(desc, 0, &c.plan);
    if (c.st != LINFUSION_OK) return c;
    if (workspace == nullptr || !is_aligned(workspace, 256)) {
        c.st = LINFUSION_ERR_INVALID_ARG;
        return c;
    }
    const int sms = device_sm_count(desc->device);
    if (sms == -2) c.st = LINFUSION_ERR_UNSUPPORTED;
    if (sms == -1) c.st = LINFUSION_ERR_CUDA;
    if (sms < 0) return c;
    if (sms != kPlanSms) c.st = make_backward_plan(desc, sms, &c.plan);
    if (c.st != LINFUSION_OK) return c;
    if (workspace_bytes < c.plan.total) c.st = LINFUSION_ERR_ALLOC;
    const size_t rows = static_cast<size_t>(c.plan.slabs) * desc->N;
    c.bytes_qk = rows * c.plan.dk * 2;
    c.bytes_vy = rows * c.plan.dv * 2;
    c.bytes_state = static_cast<size_t>(c.plan.slabs) * c.plan.floats * 4;
    return c;
}

linfusion_status_t end(cudaError_t e)
{
    if (e == cudaSuccess) return LINFUSION_OK;
    cudaGetLastError();
    return LINFUSION_ERR_CUDA;
}

}  // namespace

extern "C" {

linfusion_status_t linfusion_attn_backward_status(const linfusion_attn_desc_t* desc, const void* workspace, void* cuda_stream)
{
    BackwardPlan p;
    const linfusion_status_t st = make_backward_plan(desc, 0, &p);
    if (st != LINFUSION_OK) return st;
    if (workspace == nullptr || !is_aligned(workspace, 256)) return LINFUSION_ERR_INVALID_ARG;
    CurrentDevice guard(desc->device);
    if (!guard.ok) return LINFUSION_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    uint32_t word = 0;
    if (cudaMemcpyAsync(&word, workspace, sizeof(word), cudaMemcpyDeviceToHost, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
        cudaGetLastError();
        return LINFUSION_ERR_CUDA;
    }
    return word == kStatusOk ? LINFUSION_OK : LINFUSION_ERR_TIMEOUT;
}

linfusion_status_t linfusion_attn_backward_expired(int32_t device, uint32_t* count, void* cuda_stream)
{
    if (count == nullptr || device < 0) return LINFUSION_ERR_INVALID_ARG;
    const int sms = device_sm_count(device);
    if (sms < 0) return sms == -2 ? LINFUSION_ERR_UNSUPPORTED : LINFUSION_ERR_CUDA;
    CurrentDevice guard(device);
    if (!guard.ok) return LINFUSION_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    unsigned int n = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(&n, backward_expired_waits, sizeof(n), 0, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e == cudaSuccess) *count = n;
    return end(e);
}

linfusion_status_t linfusion_attn_selftest_backward_wait(const linfusion_attn_desc_t* desc, void* workspace, void* cuda_stream)
{
    BackwardPlan p;
    const linfusion_status_t st = make_backward_plan(desc, 0, &p);
    if (st != LINFUSION_OK) return st;
    if (workspace == nullptr || !is_aligned(workspace, 256)) return LINFUSION_ERR_INVALID_ARG;
    const int sms = device_sm_count(desc->device);
    if (sms < 0) return sms == -2 ? LINFUSION_ERR_UNSUPPORTED : LINFUSION_ERR_CUDA;
    CurrentDevice guard(desc->device);
    if (!guard.ok) return LINFUSION_ERR_CUDA;
    backward_wait_selftest_kernel<<<1, 32, 0, static_cast<cudaStream_t>(cuda_stream)>>>(static_cast<uint32_t*>(workspace));
    return end(cudaGetLastError());
}

linfusion_status_t linfusion_attn_backward_workspace_bytes(const linfusion_attn_desc_t* desc, int sm_count, size_t* bytes)
{
    if (bytes == nullptr) return LINFUSION_ERR_INVALID_ARG;
    BackwardPlan p;
    const linfusion_status_t st = make_backward_plan(desc, sm_count, &p);
    if (st != LINFUSION_OK) return st;
    *bytes = p.total;
    return LINFUSION_OK;
}

linfusion_status_t linfusion_attn_save_state(linfusion_attn_t* h, float* state, void* cuda_stream)
{
    if (h == nullptr || state == nullptr || !is_aligned(state, 16)) return LINFUSION_ERR_INVALID_ARG;
    float* from = nullptr;
    size_t floats = 0;
    const linfusion_status_t st = linfusion_attn_state_buffer(h, &from, &floats);
    if (st != LINFUSION_OK) return st;
    if (overlaps(from, floats * 4, state, floats * 4)) return LINFUSION_ERR_INVALID_ARG;
    cudaPointerAttributes where;
    if (cudaPointerGetAttributes(&where, from) != cudaSuccess) {
        cudaGetLastError();
        return LINFUSION_ERR_CUDA;
    }
    CurrentDevice guard(where.device);
    if (!guard.ok) return LINFUSION_ERR_CUDA;
    return end(cudaMemcpyAsync(state, from, floats * 4, cudaMemcpyDeviceToDevice, static_cast<cudaStream_t>(cuda_stream)));
}

linfusion_status_t linfusion_attn_backward(const linfusion_attn_desc_t* desc, const void* q, const void* k, const void* v,
                                           const void* dy, const float* state, void* dq, void* dk, void* dv, void* workspace,
                                           size_t workspace_bytes, void* cuda_stream)
{
    const Call c = begin(desc, workspace, workspace_bytes);
    if (c.st != LINFUSION_OK) return c.st;
    const Span spans[] = {{q, c.bytes_qk, false}, {k, c.bytes_qk, false}, {v, c.bytes_vy, false}, {dy, c.bytes_vy, false},
                          {dq, c.bytes_qk, true}, {dk, c.bytes_qk, true}, {dv, c.bytes_vy, true},
                          {workspace, c.plan.total, true}, {state, c.bytes_state, false}};
    if (!spans_ok(spans, state != nullptr ? 9 : 8)) return LINFUSION_ERR_INVALID_ARG;
    CurrentDevice guard(desc->device);
    if (!guard.ok) return LINFUSION_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    float* own_state = reinterpret_cast<float*>(ws + c.plan.state_off);
    float* grad = reinterpret_cast<float*>(ws + c.plan.grad_off);
    cudaError_t e = cudaSuccess;
    if (state == nullptr) e = run_state<false>(*desc, c.plan, k, v, nullptr, nullptr, ws, own_state, true, s);
    if (e == cudaSuccess)
        e = run_state<true>(*desc, c.plan, q, dy, state != nullptr ? state : own_state, dq, ws, grad, state != nullptr, s);
    if (e == cudaSuccess) e = run_kv(*desc, c.plan, k, v, grad, dk, dv, ws, false, s);
    return end(e);
}

linfusion_status_t linfusion_attn_backward_state(const linfusion_attn_desc_t* desc, const void* k, const void* v, float* state,
                                                 void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    const Call c = begin(desc, workspace, workspace_bytes);
    if (c.st != LINFUSION_OK) return c.st;
    const Span spans[] = {{k, c.bytes_qk, false}, {v, c.bytes_vy, false}, {state, c.bytes_state, true}, {workspace, c.plan.total, true}};
    if (!spans_ok(spans, 4)) return LINFUSION_ERR_INVALID_ARG;
    CurrentDevice guard(desc->device);
    if (!guard.ok) return LINFUSION_ERR_CUDA;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    return end(run_state<false>(*desc, c.plan, k, v, nullptr, nullptr, ws, state, true, static_cast<cudaStream_t>(cuda_stream)));
}

linfusion_status_t linfusion_attn_backward_q(const linfusion_attn_desc_t* desc, const void* q, const void* dy, const float* state,
                                             void* dq, float* grad_state, void* workspace, size_t workspace_bytes,
                                             void* cuda_stream)
{
    const Call c = begin(desc, workspace, workspace_bytes);
    if (c.st != LINFUSION_OK) return c.st;
    const Span spans[] = {{q, c.bytes_qk, false}, {dy, c.bytes_vy, false}, {state, c.bytes_state, false},
                          {dq, c.bytes_qk, true}, {grad_state, c.bytes_state, true}, {workspace, c.plan.total, true}};
    if (!spans_ok(spans, 6)) return LINFUSION_ERR_INVALID_ARG;
    CurrentDevice guard(desc->device);
    if (!guard.ok) return LINFUSION_ERR_CUDA;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    return end(run_state<true>(*desc, c.plan, q, dy, state, dq, ws, grad_state, true, static_cast<cudaStream_t>(cuda_stream)));
}

linfusion_status_t linfusion_attn_backward_kv(const linfusion_attn_desc_t* desc, const void* k, const void* v,
                                              const float* grad_state, void* dk, void* dv, void* workspace,
                                              size_t workspace_bytes, void* cuda_stream)
{
    const Call c = begin(desc, workspace, workspace_bytes);
    if (c.st != LINFUSION_OK) return c.st;
    const Span spans[] = {{k, c.bytes_qk, false}, {v, c.bytes_vy, false}, {grad_state, c.bytes_state, false},
                          {dk, c.bytes_qk, true}, {dv, c.bytes_vy, true}, {workspace, c.plan.total, true}};
    if (!spans_ok(spans, 6)) return LINFUSION_ERR_INVALID_ARG;
    CurrentDevice guard(desc->device);
    if (!guard.ok) return LINFUSION_ERR_CUDA;
    return end(run_kv(*desc, c.plan, k, v, grad_state, dk, dv, static_cast<unsigned char*>(workspace), true,
                      static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
