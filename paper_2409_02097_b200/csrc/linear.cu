// Host side of the matrix products of include/linfusion_layers.h: argument checks, the choice of tiles, tensor maps and launches.
#include <cuda.h>

#include "../../include/linfusion_layers.h"

#include "host_checks.h"
#include "linear_kernels.cuh"

using namespace lf;

namespace {

constexpr int kBf = make_kind(kPhiIdentity, kDtypeBf16), kHf = make_kind(kPhiIdentity, kDtypeFp16);

// ------------------------------------------------------------------------------------------ plans
// How a product D[M, N] = A[M, K] B[K, N] is laid over the machine.
struct Product {
    int cg, bn;                   // CTAs that share a tile, and its columns
    int tiles_n, tiles, chunks;
    int pairs, whole;             // groups of cg CTAs; tiles dealt out whole
    size_t partials, flags;       // bytes of workspace
};

// Estimated cycles.  A chunk (64 of K) of a tile takes what its matrix instructions or its operands' way into shared memory take; a
// round of tiles comes with a gap of its own, and joining cut tiles with the way of their sums through memory.  From the times of
// twenty sizes with each of the four shapes, whole and cut (us): 8192 x 5120 x 1280 (M x K x N) 86 whole and 76 cut with 256 x 256
// tiles, 82 and 79 with 256 x 128, 95 with 128 x 128; 8192 x 1280 x 1280 30, 32, 28, 32, 31; 1024 x 1280 x 1280 11.5, 18.7, 8.1,
// 12.1, 7.7 and 9.9 with 128 x 64; 128 x 1280 x 1280 11, 17, 7.3, 12, 7.2, 6.3; 640 x 32768 x 2560 152, 107, 104, 101, 133, 222.
struct Shape {
    int cg, bn, chunk, join;
};
constexpr Shape kShapes[] = {{2, 256, 560, 13000}, {2, 128, 350, 9000}, {1, 128, 370, 9000}, {1, 64, 330, 8000}};
constexpr int kRoundGap = 900;

Product plan_product(int M, int N, int K, int sms)
{
    Product best = {};
    double least = 1e300;
    for (const Shape& s : kShapes) {
        Product p = {};
        p.cg = s.cg;
        p.bn = s.bn;
        const int rows = s.cg * kLinRows;
        p.tiles_n = (N + s.bn - 1) / s.bn;
        const long long tiles = static_cast<long long>((M + rows - 1) / rows) * p.tiles_n;
        if (tiles > INT32_MAX / 2) continue;
        p.tiles = static_cast<int>(tiles);
        p.chunks = (K + kLinKc - 1) / kLinKc;
        const int most = sms / s.cg > 0 ? sms / s.cg : 1;
        // all tiles whole
        const long long rounds = (tiles + most - 1) / most;
        double cost = static_cast<double>(rounds) * (p.chunks * s.chunk + kRoundGap);
        p.pairs = static_cast<int>(tiles < most ? tiles : most);
        p.whole = p.tiles;
        // or the last rounds cut: at least four chunks for each pair, and at least one round (where there is one) goes with the rest
        const long long full = tiles / most > 1 ? (tiles / most - 1) * most : 0, units = (tiles - full) * p.chunks;
        const long long pairs = units / 4 < most ? (units / 4 > 0 ? units / 4 : 1) : most;
        if (tiles % most != 0 && pairs > 1 && (full == 0 || pairs == most) && units <= INT32_MAX / 2) {
            const double per = static_cast<double>((units + pairs - 1) / pairs), helpers = p.chunks / (per < p.chunks ? per : p.chunks);
            const double cut = static_cast<double>(full / most) * (p.chunks * s.chunk + kRoundGap) + per * s.chunk + kRoundGap + s.join + helpers * s.bn * 8;
            if (cut < cost) {
                cost = cut;
                p.pairs = static_cast<int>(pairs);
                p.whole = static_cast<int>(full);
            }
        }
        if (p.whole < p.tiles) {
            p.partials = static_cast<size_t>(p.pairs) * p.cg * (p.bn / 4) * kLinRows * sizeof(float4);
            p.flags = align_up_256(static_cast<size_t>(p.pairs) * p.cg * (p.bn / kLinColumns) * sizeof(Handover));
        }
        if (cost < least) {
            least = cost;
            best = p;
        }
    }
    return best;
}

// The sums over du's columns: blocks of rows, as many as run at once (three on an SM).
struct Sums {
    int width, columns, blocks, rows;
};
Sums plan_sums(int M, int N, int sms)
{
    Sums s;
    s.width = (N + kSumChannels - 1) / kSumChannels * kSumChannels;
    s.columns = (N + kDuColumns - 1) / kDuColumns;
    int blocks = 3 * sms / s.columns > 0 ? 3 * sms / s.columns : 1;
    const int step = kDuUnroll * kDuThreads / 32, most = (M + step - 1) / step;
    if (blocks > most) blocks = most;
    if (blocks > 65535) blocks = 65535;
    s.rows = (M + blocks - 1) / blocks;
    s.blocks = (M + s.rows - 1) / s.rows;
    return s;
}

// The parts of a call's workspace.
struct Workspace {
    Product forward, dx, dw;
    Sums sums;
    size_t flags_dw, partials, du, x, column_sums, bytes;
};
Workspace plan_forward(const linfusion_linear_desc_t& d, int sms)
{
    Workspace w = {};
    w.forward = plan_product(d.M, d.N, d.K, sms);
    w.partials = w.forward.flags;
    w.bytes = w.partials + w.forward.partials;
    return w;
}
Workspace plan_backward(const linfusion_linear_desc_t& d, bool x_packed, int sms)
{
    Workspace w = {};
    w.dx = plan_product(d.M, d.K, d.N, sms);
    w.dw = d.w_transposed ? plan_product(d.N, d.K, d.M, sms) : plan_product(d.K, d.N, d.M, sms);
    w.sums = plan_sums(d.M, d.N, sms);
    w.flags_dw = w.dx.flags;
    w.partials = w.flags_dw + w.dw.flags;
    w.du = w.partials + std::max(w.dx.partials, w.dw.partials);  // one product after the other
    w.x = w.du + (d.act != LINFUSION_ACT_NONE ? align_up_256(static_cast<size_t>(d.M) * d.N * 2) : 0);
    w.column_sums = w.x + (x_packed ? align_up_256(static_cast<size_t>(d.M) * d.K * 2) : 0);
    w.bytes = w.column_sums + align_up_256(static_cast<size_t>(w.sums.blocks) * w.sums.width * sizeof(float));
    return w;
}

// ------------------------------------------------------------------------------------------ checks
linfusion_status_t check(const linfusion_linear_desc_t* d)
{
    if (d == nullptr || d->M <= 0 || d->K <= 0 || d->N <= 0 || (d->w_transposed & ~1) != 0) return LINFUSION_ERR_INVALID_ARG;
    if (d->K % 8 != 0 || d->N % 8 != 0 || (d->flags & ~LINFUSION_DTYPE_FP16) != 0u) return LINFUSION_ERR_UNSUPPORTED;
    if (d->act < LINFUSION_ACT_NONE || d->act > LINFUSION_ACT_GELU_TANH) return LINFUSION_ERR_UNSUPPORTED;
    // coordinates, with a tile past the end, are 32 bits
    for (const int32_t n : {d->M, d->K, d->N})
        if (n > INT32_MAX - 1024) return LINFUSION_ERR_UNSUPPORTED;
    return LINFUSION_OK;
}
// A matrix of `rows` x `cols`, whose rows lie apart; tensor maps hold strides below 2^40 bytes.
bool matrix_ok(const linfusion_matrix_t* m, int64_t rows, int64_t cols)
{
    if (m == nullptr || m->p == nullptr || !is_aligned(m->p, 16)) return false;
    return rows == 1 || (m->row >= cols && good_stride(rows, m->row) && m->row < (int64_t(1) << 38));
}
// The stride of a single row says nothing.
int64_t row_of(const linfusion_matrix_t& m, int64_t rows, int64_t cols) { return rows == 1 ? cols : m.row; }
Extent extent_of(const linfusion_matrix_t& m, int64_t rows, int64_t cols)
{
    return {static_cast<const char*>(m.p), static_cast<size_t>((rows - 1) * row_of(m, rows, cols) + cols) * 2};
}
Extent bytes_of(const void* p, size_t n) { return {static_cast<const char*>(p), n}; }
int scale_groups(int C) { return (C + LINFUSION_PACK8_GROUP - 1) / LINFUSION_PACK8_GROUP; }
bool packed_given(const linfusion_packed8_t& p) { return p.codes != nullptr; }

// Ranges of a call: none of the first `n_out` meets another of them or one behind.
bool ranges_apart(const Extent* e, int n_out, int n)
{
    for (int o = 0; o < n_out; ++o)
        for (int i = o + 1; i < n; ++i)
            if (meet(e[o], e[i])) return false;
    return true;
}

// ------------------------------------------------------------------------------------------ launches
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Boxes of 64 values x `box_rows` of a matrix of 16-bit values in the 128-byte swizzle, or of bytes in that of 64 bytes.  What lies
// outside is read as zero and not written.
bool encode(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t row, int box_rows, bool bytes = false)
{
    static std::atomic<EncodeTiledFn> known{nullptr};
    EncodeTiledFn fn = known.load(std::memory_order_acquire);
    if (fn == nullptr) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return false;
        fn = reinterpret_cast<EncodeTiledFn>(p);
        known.store(fn, std::memory_order_release);
    }
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(row) * (bytes ? 1 : 2)};
    const cuuint32_t box[2] = {64u, static_cast<cuuint32_t>(box_rows)}, step[2] = {1u, 1u};
    return fn(map, bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, step,
              CU_TENSOR_MAP_INTERLEAVE_NONE, bytes ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// An operand: `mn` rows or columns of D by K values, contiguous along K or along mn.
struct Operand {
    const void* p;
    int64_t row;
    bool mn_contiguous;
};
bool encode_operand(CUtensorMap* map, const Operand& o, int64_t mn, int64_t K, int per_cta)
{
    return o.mn_contiguous ? encode(map, o.p, K, mn, o.row, kLinKc) : encode(map, o.p, mn, K, o.row, per_cta);
}

// What an epilogue does besides storing y.
struct Epilogue {
    int act = LINFUSION_ACT_NONE;
    const void* bias = nullptr;
    const linfusion_matrix_t* residual = nullptr;
    const linfusion_matrix_t* u = nullptr;
    const linfusion_packed8_t* u_packed = nullptr;
};

template <int KIND, int CG, int BN>
cudaError_t launch(const CUtensorMap (&maps)[5], const LinParams& p, int pairs, int device, cudaStream_t s)
{
    static std::atomic<uint64_t> done{0};
    using C = LinCfg<CG, BN>;
    const cudaError_t e = allow_smem(linear_kernel<KIND, CG, BN>, C::SMEM, device, &done);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(pairs * CG);
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CG;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, linear_kernel<KIND, CG, BN>, maps[0], maps[1], maps[2], maps[3], maps[4], p);
}

// A mark for the flags of one call: a different one each time, odd, and unlikely to be what memory holds by chance.
Handover next_mark()
{
    static std::atomic<unsigned long long> calls{0x9E3779B97F4A7C15ull};
    return calls.fetch_add(0xD1342543DE82EF95ull, std::memory_order_relaxed) | 1ull;
}

// D[M, N] = A B with its epilogue.
linfusion_status_t product(const Product& plan, int M, int N, int K, const Operand& a, const Operand& b, const linfusion_matrix_t& y,
                           const Epilogue& ep, bool half, void* flags, void* partials, int device, cudaStream_t s)
{
    CUtensorMap maps[5];
    const int a_rows = M >= kLinRows ? kLinRows : (M + 7) / 8 * 8;
    bool ok = encode_operand(&maps[0], a, M, K, a_rows) && encode_operand(&maps[1], b, N, K, plan.bn / plan.cg) &&
              encode(&maps[2], y.p, M, N, row_of(y, M, N), kLinRows);
    maps[3] = maps[4] = maps[2];
    if (ok && ep.residual != nullptr) ok = encode(&maps[3], ep.residual->p, M, N, row_of(*ep.residual, M, N), kLinRows);
    if (ok && ep.u != nullptr) ok = encode(&maps[4], ep.u->p, M, N, row_of(*ep.u, M, N), kLinRows);
    const bool codes_map = ep.u_packed != nullptr && N % 16 == 0;
    if (ok && codes_map) ok = encode(&maps[4], ep.u_packed->codes, M, N, N, kLinRows, true);
    if (!ok) return LINFUSION_ERR_CUDA;
    LinParams p = {};
    p.M = M;
    p.N = N;
    p.chunks = plan.chunks;
    p.tiles_n = plan.tiles_n;
    p.whole = plan.whole;
    p.tiles = plan.tiles;
    p.a_mn = a.mn_contiguous;
    p.b_mn = b.mn_contiguous;
    p.act = ep.act;
    p.u_mode = ep.u != nullptr ? kUFull : ep.u_packed != nullptr ? kUPacked : kUNone;
    p.has_residual = ep.residual != nullptr;
    p.bias = static_cast<const char*>(ep.bias);
    if (ep.u_packed != nullptr) {
        p.codes = static_cast<signed char*>(ep.u_packed->codes);
        p.scales = static_cast<unsigned char*>(ep.u_packed->scales);
        p.scale_groups = scale_groups(N);
        p.codes_map = codes_map;
    }
    p.a_rows = a_rows;
    p.partials = static_cast<float4*>(partials);
    p.flags = static_cast<Handover*>(flags);
    p.mark = next_mark();
    cudaError_t e = cudaErrorInvalidValue;
#define LF_PRODUCT(CG, BN) \
    if (plan.cg == CG && plan.bn == BN) e = half ? launch<kHf, CG, BN>(maps, p, plan.pairs, device, s) : launch<kBf, CG, BN>(maps, p, plan.pairs, device, s)
    LF_PRODUCT(2, 256);
    LF_PRODUCT(2, 128);
    LF_PRODUCT(1, 128);
    LF_PRODUCT(1, 64);
#undef LF_PRODUCT
    return end(e);
}

template <int KIND, bool PACKED>
cudaError_t launch_du(const DuParams& p, int act, dim3 grid, cudaStream_t s)
{
    const dim3 block(kDuThreads);
    switch (act) {
        case LINFUSION_ACT_RELU: return launch_pdl(linear_du_kernel<KIND, 1, PACKED>, grid, block, 0, s, p);
        case LINFUSION_ACT_SILU: return launch_pdl(linear_du_kernel<KIND, 2, PACKED>, grid, block, 0, s, p);
        case LINFUSION_ACT_GELU: return launch_pdl(linear_du_kernel<KIND, 3, PACKED>, grid, block, 0, s, p);
        case LINFUSION_ACT_GELU_TANH: return launch_pdl(linear_du_kernel<KIND, 4, PACKED>, grid, block, 0, s, p);
        default: return launch_pdl(linear_du_kernel<KIND, 0, false>, grid, block, 0, s, p);
    }
}

linfusion_status_t workspace_ok(const void* workspace, size_t given, size_t need)
{
    if (need == 0) return LINFUSION_OK;
    if (workspace == nullptr || !is_aligned(workspace, 256)) return LINFUSION_ERR_INVALID_ARG;
    return given < need ? LINFUSION_ERR_ALLOC : LINFUSION_OK;
}

}  // namespace

extern "C" {

linfusion_status_t linfusion_linear_workspace_bytes(const linfusion_linear_desc_t* desc, int32_t backward, int32_t sm_count, size_t* bytes)
{
    if (bytes == nullptr || backward < 0 || backward > 2) return LINFUSION_ERR_INVALID_ARG;
    const linfusion_status_t st = check(desc);
    if (st != LINFUSION_OK) return st;
    const int sms = sm_count > 0 ? sm_count : 148;
    *bytes = (backward == 0 ? plan_forward(*desc, sms) : plan_backward(*desc, backward == 2, sms)).bytes;
    return LINFUSION_OK;
}

linfusion_status_t linfusion_linear(const linfusion_linear_desc_t* desc, const linfusion_matrix_t* x, const linfusion_matrix_t* w,
                                    const void* bias, const linfusion_matrix_t* residual, const linfusion_matrix_t* y,
                                    const linfusion_matrix_t* u, const linfusion_packed8_t* u_packed, void* workspace,
                                    size_t workspace_bytes, void* cuda_stream)
{
    linfusion_status_t st = check(desc);
    if (st != LINFUSION_OK) return st;
    const linfusion_linear_desc_t& d = *desc;
    const int64_t w_rows = d.w_transposed ? d.N : d.K, w_cols = d.w_transposed ? d.K : d.N;
    if (residual != nullptr && residual->p == nullptr) residual = nullptr;
    if (u != nullptr && u->p == nullptr) u = nullptr;
    if (u_packed != nullptr && !packed_given(*u_packed)) u_packed = nullptr;
    if (!matrix_ok(x, d.M, d.K) || !matrix_ok(w, w_rows, w_cols) || !matrix_ok(y, d.M, d.N)) return LINFUSION_ERR_INVALID_ARG;
    if (bias != nullptr && !is_aligned(bias, 16)) return LINFUSION_ERR_INVALID_ARG;
    if (residual != nullptr && !matrix_ok(residual, d.M, d.N)) return LINFUSION_ERR_INVALID_ARG;
    if (u != nullptr && (u_packed != nullptr || !matrix_ok(u, d.M, d.N))) return LINFUSION_ERR_INVALID_ARG;
    if (u_packed != nullptr && (!is_aligned(u_packed->codes, 16) || u_packed->scales == nullptr)) return LINFUSION_ERR_INVALID_ARG;
    const Here at = here();
    // refusals come before the want of a device
    const Workspace plan = plan_forward(d, at.st == LINFUSION_OK ? at.sms : 148);
    st = workspace_ok(workspace, workspace_bytes, plan.bytes);
    if (st != LINFUSION_OK) return st;
    Extent e[9];
    int n = 0;
    const Extent ey = extent_of(*y, d.M, d.N);
    e[n++] = ey;
    if (u != nullptr) e[n++] = extent_of(*u, d.M, d.N);
    if (u_packed != nullptr) {
        e[n++] = bytes_of(u_packed->codes, static_cast<size_t>(d.M) * d.N);
        e[n++] = bytes_of(u_packed->scales, static_cast<size_t>(d.M) * scale_groups(d.N));
    }
    if (plan.bytes != 0) e[n++] = bytes_of(workspace, plan.bytes);
    const int outs = n;
    e[n++] = extent_of(*x, d.M, d.K);
    e[n++] = extent_of(*w, w_rows, w_cols);
    if (bias != nullptr) e[n++] = bytes_of(bias, static_cast<size_t>(d.N) * 2);
    if (residual != nullptr) {
        const Extent er = extent_of(*residual, d.M, d.N);
        const bool over = residual->p == y->p && row_of(*residual, d.M, d.N) == row_of(*y, d.M, d.N);
        if (!over && meet(ey, er)) return LINFUSION_ERR_INVALID_ARG;
        for (int o = 1; o < outs; ++o)
            if (meet(e[o], er)) return LINFUSION_ERR_INVALID_ARG;
    }
    if (!ranges_apart(e, outs, n)) return LINFUSION_ERR_INVALID_ARG;
    if (at.st != LINFUSION_OK) return at.st;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(workspace);
    Epilogue ep;
    ep.act = d.act;
    ep.bias = bias;
    ep.residual = residual;
    ep.u = u;
    ep.u_packed = u_packed;
    return product(plan.forward, d.M, d.N, d.K, {x->p, row_of(*x, d.M, d.K), false}, {w->p, row_of(*w, w_rows, w_cols), d.w_transposed == 0}, *y, ep,
                   (d.flags & LINFUSION_DTYPE_FP16) != 0u, ws, ws + plan.partials, at.device, s);
}

linfusion_status_t linfusion_linear_backward(const linfusion_linear_desc_t* desc, const linfusion_matrix_t* dy,
                                             const linfusion_linear_saved_t* saved, const linfusion_matrix_t* w,
                                             const linfusion_matrix_t* dx, const linfusion_matrix_t* dw, float* dbias,
                                             void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    linfusion_status_t st = check(desc);
    if (st != LINFUSION_OK) return st;
    const linfusion_linear_desc_t& d = *desc;
    const linfusion_linear_saved_t none = {};
    if (saved == nullptr) saved = &none;
    if (dx != nullptr && dx->p == nullptr) dx = nullptr;
    if (dw != nullptr && dw->p == nullptr) dw = nullptr;
    if (dx == nullptr && dw == nullptr && dbias == nullptr) return LINFUSION_ERR_INVALID_ARG;
    const int64_t w_rows = d.w_transposed ? d.N : d.K, w_cols = d.w_transposed ? d.K : d.N;
    const bool act = d.act != LINFUSION_ACT_NONE, x_packed = dw != nullptr && packed_given(saved->x_packed),
               u_packed = act && packed_given(saved->u_packed);
    if (!matrix_ok(dy, d.M, d.N)) return LINFUSION_ERR_INVALID_ARG;
    if (dx != nullptr && (!matrix_ok(dx, d.M, d.K) || !matrix_ok(w, w_rows, w_cols))) return LINFUSION_ERR_INVALID_ARG;
    if (dw != nullptr && !matrix_ok(dw, w_rows, w_cols)) return LINFUSION_ERR_INVALID_ARG;
    if (dw != nullptr && !x_packed && !matrix_ok(&saved->x, d.M, d.K)) return LINFUSION_ERR_INVALID_ARG;
    if (act && !u_packed && !matrix_ok(&saved->u, d.M, d.N)) return LINFUSION_ERR_INVALID_ARG;
    if (x_packed && (!is_aligned(saved->x_packed.codes, 16) || saved->x_packed.scales == nullptr || saved->x.p != nullptr)) return LINFUSION_ERR_INVALID_ARG;
    if (u_packed && (!is_aligned(saved->u_packed.codes, 16) || saved->u_packed.scales == nullptr || saved->u.p != nullptr)) return LINFUSION_ERR_INVALID_ARG;
    if (dbias != nullptr && !is_aligned(dbias, 16)) return LINFUSION_ERR_INVALID_ARG;
    const Here at = here();
    const Workspace plan = plan_backward(d, x_packed, at.st == LINFUSION_OK ? at.sms : 148);
    st = workspace_ok(workspace, workspace_bytes, plan.bytes);
    if (st != LINFUSION_OK) return st;
    Extent e[12];
    int n = 0;
    if (dx != nullptr) e[n++] = extent_of(*dx, d.M, d.K);
    if (dw != nullptr) e[n++] = extent_of(*dw, w_rows, w_cols);
    if (dbias != nullptr) e[n++] = bytes_of(dbias, static_cast<size_t>(d.N) * 4);
    e[n++] = bytes_of(workspace, plan.bytes);
    const int outs = n;
    e[n++] = extent_of(*dy, d.M, d.N);
    if (dx != nullptr) e[n++] = extent_of(*w, w_rows, w_cols);
    if (x_packed) {
        e[n++] = bytes_of(saved->x_packed.codes, static_cast<size_t>(d.M) * d.K);
        e[n++] = bytes_of(saved->x_packed.scales, static_cast<size_t>(d.M) * scale_groups(d.K));
    } else if (dw != nullptr) {
        e[n++] = extent_of(saved->x, d.M, d.K);
    }
    if (u_packed) {
        e[n++] = bytes_of(saved->u_packed.codes, static_cast<size_t>(d.M) * d.N);
        e[n++] = bytes_of(saved->u_packed.scales, static_cast<size_t>(d.M) * scale_groups(d.N));
    } else if (act) {
        e[n++] = extent_of(saved->u, d.M, d.N);
    }
    if (!ranges_apart(e, outs, n)) return LINFUSION_ERR_INVALID_ARG;
    if (at.st != LINFUSION_OK) return at.st;

    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(workspace);
    const bool half = (d.flags & LINFUSION_DTYPE_FP16) != 0u;
    linfusion_matrix_t du = *dy;
    if (act || dbias != nullptr) {
        DuParams p = {};
        p.dy = static_cast<const char*>(dy->p);
        p.dy_row = row_of(*dy, d.M, d.N) * 2;
        if (u_packed) {
            p.u = static_cast<const char*>(saved->u_packed.codes);
            p.scales = static_cast<const unsigned char*>(saved->u_packed.scales);
            p.u_row = d.N;
        } else if (act) {
            p.u = static_cast<const char*>(saved->u.p);
            p.u_row = row_of(saved->u, d.M, d.N) * 2;
        }
        p.du = ws + plan.du;
        p.sums = dbias != nullptr ? reinterpret_cast<float*>(ws + plan.column_sums) : nullptr;
        p.M = d.M;
        p.N = d.N;
        p.width = plan.sums.width;
        p.rows_per_block = plan.sums.rows;
        p.scale_groups = scale_groups(d.N);
        const dim3 grid(plan.sums.columns, plan.sums.blocks);
        cudaError_t err;
        if (half) err = u_packed ? launch_du<kHf, true>(p, d.act, grid, s) : launch_du<kHf, false>(p, d.act, grid, s);
        else err = u_packed ? launch_du<kBf, true>(p, d.act, grid, s) : launch_du<kBf, false>(p, d.act, grid, s);
        if (err == cudaSuccess && dbias != nullptr)
            err = launch_pdl(column_sums_kernel, dim3(plan.sums.width / kSumChannels), dim3(kSumThreads), 0, s, p.sums, dbias, plan.sums.blocks,
                             plan.sums.width, d.N);
        if (err != cudaSuccess) return end(err);
        if (act) du = {ws + plan.du, d.N};
    }
    const int64_t du_row = row_of(du, d.M, d.N);
    if (dx != nullptr) {
        st = product(plan.dx, d.M, d.K, d.N, {du.p, du_row, false}, {w->p, row_of(*w, w_rows, w_cols), d.w_transposed != 0}, *dx, {}, half, ws,
                     ws + plan.partials, at.device, s);
        if (st != LINFUSION_OK) return st;
    }
    if (dw != nullptr) {
        linfusion_matrix_t xm = saved->x;
        if (x_packed) {
            const linfusion_pack8_desc_t pd = {1, d.M, d.K, d.flags};
            const linfusion_rows_t rows = {ws + plan.x, 0, d.K};
            st = linfusion_unpack8(&pd, &saved->x_packed, &rows, s);
            if (st != LINFUSION_OK) return st;
            xm = {ws + plan.x, d.K};
        }
        const Operand xo = {xm.p, row_of(xm, d.M, d.K), true}, duo = {du.p, du_row, true};
        if (d.w_transposed) st = product(plan.dw, d.N, d.K, d.M, duo, xo, *dw, {}, half, ws + plan.flags_dw, ws + plan.partials, at.device, s);
        else st = product(plan.dw, d.K, d.N, d.M, xo, duo, *dw, {}, half, ws + plan.flags_dw, ws + plan.partials, at.device, s);
    }
    return st;
}

linfusion_status_t linfusion_layers_expired(int32_t device, uint32_t* count, void* cuda_stream)
{
    if (count == nullptr || device < 0) return LINFUSION_ERR_INVALID_ARG;
    const int sms = device_sm_count(device);
    if (sms < 0) return sms == -2 ? LINFUSION_ERR_UNSUPPORTED : LINFUSION_ERR_CUDA;
    CurrentDevice guard(device);
    if (!guard.ok) return LINFUSION_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    unsigned int n = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(&n, linear_expired_waits, sizeof(n), 0, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e == cudaSuccess) *count = n;
    return end(e);
}

}  // extern "C"
