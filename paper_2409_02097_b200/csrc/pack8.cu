// 16-bit tensors into 8 bits and back: kernels and host side of linfusion_pack8 and linfusion_unpack8.
#include "pack8.cuh"

#include "../../include/linfusion_layers.h"
#include "block_kernels.cuh"
#include "host_checks.h"

using namespace lf;

namespace {

// A thread takes eight channels (16 bytes there, 8 here) and the four threads of a group share its maximum.  Bound by DRAM: 3.03
// bytes a value.  Two pieces a thread, half a grid apart, are in flight together.
constexpr int kThreads = 256, kPieces = 2;

struct Pack8Params {
    const char* x;
    char* codes;
    unsigned char* scales;
    long long batch, row;          // of x, bytes
    int N, C, groups;              // groups of 32 in a row
    long long total;               // pieces of eight channels, four to each group, over all rows
};

struct Piece {
    long long row;   // of the dense tensor
    long long at;    // of x, bytes
    int piece;       // in the row
    bool live;
};
__device__ __forceinline__ Piece piece_of(const Pack8Params& p, long long i)
{
    Piece o;
    const int per_row = 4 * p.groups;
    // the totals of all but giant tensors fit 32 bits, where a division is much cheaper
    if (p.total <= 0x7fffffffll) {
        const unsigned int r = static_cast<unsigned int>(i) / per_row;
        o.row = r;
        o.piece = static_cast<int>(static_cast<unsigned int>(i) - r * per_row);
        o.at = static_cast<long long>(r / p.N) * p.batch + static_cast<long long>(r % p.N) * p.row;
    } else {
        o.row = i / per_row;
        o.piece = static_cast<int>(i - o.row * per_row);
        o.at = o.row / p.N * p.batch + o.row % p.N * p.row;
    }
    o.at += 16ll * o.piece;
    o.live = i < p.total && 8 * o.piece < p.C;
    return o;
}

template <int KIND>
__global__ void __launch_bounds__(kThreads) pack8_kernel(Pack8Params p)
{
    const long long step = static_cast<long long>(gridDim.x) * kThreads, first = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    Piece q[kPieces];
    uint4 raw[kPieces];
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        q[k] = piece_of(p, first + k * step);
        raw[k] = q[k].live ? load16(p.x + q[k].at) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        const F8 f = unpack8<KIND>(raw[k]);
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, finite_abs(f.v[i]));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int scale = pack8_scale<KIND>(most);
        if (q[k].live) {
            const float inverse = pack8_inverse_step(scale);
            const uint2 c = make_uint2(pack8_codes4(f.v, inverse), pack8_codes4(f.v + 4, inverse));
            *reinterpret_cast<uint2*>(p.codes + q[k].row * p.C + 8ll * q[k].piece) = c;
            if ((q[k].piece & 3) == 0) p.scales[q[k].row * p.groups + (q[k].piece >> 2)] = static_cast<unsigned char>(scale);
        }
    }
}

template <int KIND>
__global__ void __launch_bounds__(kThreads) unpack8_kernel(Pack8Params p)
{
    const long long step = static_cast<long long>(gridDim.x) * kThreads, first = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    Piece q[kPieces];
    uint2 codes[kPieces];
    int scale[kPieces];
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        q[k] = piece_of(p, first + k * step);
        if (q[k].live) {
            codes[k] = *reinterpret_cast<const uint2*>(p.codes + q[k].row * p.C + 8ll * q[k].piece);
            scale[k] = p.scales[q[k].row * p.groups + (q[k].piece >> 2)];
        }
    }
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
        if (q[k].live) {
            F8 f;
            unpack8_codes4(codes[k].x, pack8_step(scale[k]), f.v);
            unpack8_codes4(codes[k].y, pack8_step(scale[k]), f.v + 4);
            store16(const_cast<char*>(p.x) + q[k].at, pack8<KIND>(f));
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
                     x->batch * 2, x->row * 2, d->N, d->C, groups, rows * groups * 4};
    const unsigned int grid = static_cast<unsigned int>((p.total + kThreads * kPieces - 1) / (kThreads * kPieces));
    const bool half = (d->flags & LINFUSION_DTYPE_FP16) != 0u;
    constexpr int bf = make_kind(kPhiIdentity, kDtypeBf16), hf = make_kind(kPhiIdentity, kDtypeFp16);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (pack) {
        if (half) pack8_kernel<hf><<<grid, kThreads, 0, s>>>(p);
        else pack8_kernel<bf><<<grid, kThreads, 0, s>>>(p);
    } else {
        if (half) unpack8_kernel<hf><<<grid, kThreads, 0, s>>>(p);
        else unpack8_kernel<bf><<<grid, kThreads, 0, s>>>(p);
    }
    return end(cudaGetLastError());
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
