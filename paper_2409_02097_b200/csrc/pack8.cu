// 16-bit tensors into 8 bits and back: kernels and host side of linfusion_pack8 and linfusion_unpack8.
#include "pack8.cuh"

#include "../../include/linfusion_layers.h"
#include "block_kernels.cuh"
#include "host_checks.h"

using namespace lf;

namespace {

// A thread takes eight channels (16 bytes there, 8 here) and the four threads of a group share its maximum.  Bound by DRAM: 3.03
// bytes a value.  A thread goes through pieces a grid apart, four of them in flight; only the first one's row is found by a division, and
// the batch is one long column of rows wherever its stride says so.  61441 x 648: 28 us there, 25 us back (18.4 each at the copy rate).
constexpr int kThreads = 256, kPieces = 4;

struct Pack8Params {
    const char* x;
    char* codes;
    unsigned char* scales;
    long long batch, row;          // of x, bytes
    int B, N, C, groups;           // groups of 32 in a row
    long long total;               // pieces of eight channels, four to each group, over all rows
};

// The pieces of a thread, one after the other.
struct Pieces {
    long long row;   // of the dense tensor
    int piece, per_row, step_piece;
    long long step_row;
    bool flat;       // B == 1
    __device__ __forceinline__ explicit Pieces(const Pack8Params& p)
    {
        per_row = 4 * p.groups;
        const long long first = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x, step = static_cast<long long>(gridDim.x) * kThreads;
        row = first / per_row;
        piece = static_cast<int>(first - row * per_row);
        step_row = step / per_row;
        step_piece = static_cast<int>(step - step_row * per_row);
        flat = p.B == 1;
    }
    __device__ __forceinline__ void next()
    {
        row += step_row;
        piece += step_piece;
        if (piece >= per_row) {
            piece -= per_row;
            ++row;
        }
    }
    __device__ __forceinline__ long long at(const Pack8Params& p) const
    {
        if (flat) return row * p.row + 16ll * piece;
        const unsigned int r = static_cast<unsigned int>(row);  // rows are fewer than 2^31
        return static_cast<long long>(r / p.N) * p.batch + static_cast<long long>(r % p.N) * p.row + 16ll * piece;
    }
};

template <int KIND>
__global__ void __launch_bounds__(kThreads) pack8_kernel(const __grid_constant__ Pack8Params p)
{
    const long long rows = static_cast<long long>(p.B) * p.N;
    Pieces q(p);
    pdl_wait();
    pdl_launch_dependents();
    while (__any_sync(0xffffffffu, q.row < rows)) {
        uint4 raw[kPieces];
        long long row[kPieces];
        int piece[kPieces];
#pragma unroll
        for (int k = 0; k < kPieces; ++k, q.next()) {
            row[k] = q.row;
            piece[k] = q.piece;
            raw[k] = make_uint4(0u, 0u, 0u, 0u);
            if (q.row < rows && 8 * q.piece < p.C) raw[k] = load16(p.x + q.at(p));
        }
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            f32x2 f[4];
            f[0] = pack2(pair_lo<KIND>(raw[k].x), pair_hi<KIND>(raw[k].x));
            f[1] = pack2(pair_lo<KIND>(raw[k].y), pair_hi<KIND>(raw[k].y));
            f[2] = pack2(pair_lo<KIND>(raw[k].z), pair_hi<KIND>(raw[k].z));
            f[3] = pack2(pair_lo<KIND>(raw[k].w), pair_hi<KIND>(raw[k].w));
            const bool plain = all_finite(f);
            float most = largest(f, plain);
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const int scale = pack8_scale<KIND>(most);
            if (row[k] < rows && 8 * piece[k] < p.C) {
                uint32_t w[2];
                pack8_codes(f, most, pack8_inverse_step(scale), plain, w);
                *reinterpret_cast<uint2*>(p.codes + row[k] * p.C + 8ll * piece[k]) = make_uint2(w[0], w[1]);
                if ((piece[k] & 3) == 0) p.scales[row[k] * p.groups + (piece[k] >> 2)] = static_cast<unsigned char>(scale);
            }
        }
    }
}

template <int KIND>
__global__ void __launch_bounds__(kThreads) unpack8_kernel(const __grid_constant__ Pack8Params p)
{
    const long long rows = static_cast<long long>(p.B) * p.N;
    Pieces q(p);
    pdl_wait();
    pdl_launch_dependents();
    while (q.row < rows) {
        uint2 codes[kPieces];
        int scale[kPieces];
        long long at[kPieces];
#pragma unroll
        for (int k = 0; k < kPieces; ++k, q.next()) {
            at[k] = -1;
            if (q.row < rows && 8 * q.piece < p.C) {
                at[k] = q.at(p);
                codes[k] = *reinterpret_cast<const uint2*>(p.codes + q.row * p.C + 8ll * q.piece);
                scale[k] = p.scales[q.row * p.groups + (q.piece >> 2)];
            }
        }
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
            if (at[k] >= 0) {
                f32x2 f[4];
                unpack8_codes4(codes[k].x, pack8_step(scale[k]), f);
                unpack8_codes4(codes[k].y, pack8_step(scale[k]), f + 2);
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 a = unpack2(f[i]);
                    w[i] = pack_pair<KIND>(a.x, a.y);
                }
                store16(const_cast<char*>(p.x) + at[k], make_uint4(w[0], w[1], w[2], w[3]));
            }
    }
}

linfusion_status_t run(const linfusion_pack8_desc_t* d, const linfusion_rows_t* x, const linfusion_packed8_t* packed, bool pack, void* stream)
{
    if (d == nullptr || x == nullptr || packed == nullptr) return LINFUSION_ERR_INVALID_ARG;
    if (d->B <= 0 || d->N <= 0 || d->C <= 0 || d->C % 8 != 0) return LINFUSION_ERR_INVALID_ARG;
    if ((d->flags & ~LINFUSION_DTYPE_FP16) != 0u) return LINFUSION_ERR_UNSUPPORTED;
    const int groups = d->C / 32 + (d->C % 32 != 0 ? 1 : 0);
    const int64_t rows = static_cast<int64_t>(d->B) * d->N;
    if (rows > INT32_MAX || rows * groups > INT32_MAX) return LINFUSION_ERR_UNSUPPORTED;
    if (x->p == nullptr || !is_aligned(x->p, 16) || !good_stride(d->B, x->batch) || !good_stride(d->N, x->row)) return LINFUSION_ERR_INVALID_ARG;
    if (packed->codes == nullptr || packed->scales == nullptr || !is_aligned(packed->codes, 16)) return LINFUSION_ERR_INVALID_ARG;
    if (!pack && !rows_disjoint({{d->B, x->batch}, {d->N, x->row}}, d->C)) return LINFUSION_ERR_INVALID_ARG;
    const Extent ex = extent(x->p, d->B, x->batch, d->N, x->row, 1, 0, d->C);
    const Extent ec = {static_cast<const char*>(packed->codes), static_cast<size_t>(rows) * d->C};
    const Extent es = {static_cast<const char*>(packed->scales), static_cast<size_t>(rows) * groups};
    if (meet(ex, ec) || meet(ex, es) || meet(ec, es)) return LINFUSION_ERR_INVALID_ARG;
    const Here at = here();
    if (at.st != LINFUSION_OK) return at.st;
    Pack8Params p = {static_cast<const char*>(x->p), static_cast<char*>(packed->codes), static_cast<unsigned char*>(packed->scales),
                     x->batch * 2, x->row * 2, d->B, d->N, d->C, groups, rows * groups * 4};
    if (d->B > 1 && d->N == 1) p.row = p.batch;
    if (d->N == 1 || d->B == 1 || x->batch == d->N * x->row) {  // one column of rows
        p.B = 1;
        p.N = static_cast<int>(rows);
    }
    // as many blocks as run at once, fewer where there is less to do
    const long long most = (p.total + kThreads - 1) / kThreads;
    const unsigned int grid = static_cast<unsigned int>(std::min<long long>(most, 8ll * at.sms));
    const bool half = (d->flags & LINFUSION_DTYPE_FP16) != 0u;
    constexpr int bf = make_kind(kPhiIdentity, kDtypeBf16), hf = make_kind(kPhiIdentity, kDtypeFp16);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (pack) e = half ? launch_pdl(pack8_kernel<hf>, dim3(grid), dim3(kThreads), 0, s, p) : launch_pdl(pack8_kernel<bf>, dim3(grid), dim3(kThreads), 0, s, p);
    else e = half ? launch_pdl(unpack8_kernel<hf>, dim3(grid), dim3(kThreads), 0, s, p) : launch_pdl(unpack8_kernel<bf>, dim3(grid), dim3(kThreads), 0, s, p);
    return end(e);
}

}  // namespace

extern "C" {

linfusion_status_t linfusion_pack8(const linfusion_pack8_desc_t* desc, const linfusion_rows_t* x, const linfusion_packed8_t* packed,
                                   void* cuda_stream)
{
    return run(desc, x, packed, true, cuda_stream);
}

linfusion_status_t linfusion_unpack8(const linfusion_pack8_desc_t* desc, const linfusion_packed8_t* packed, const linfusion_rows_t* x,
                                     void* cuda_stream)
{
    return run(desc, x, packed, false, cuda_stream);
}

}  // extern "C"
