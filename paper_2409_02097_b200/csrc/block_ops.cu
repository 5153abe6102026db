// Host side of include/linfusion_block.h: argument checks and launches of the rotary positions and of the norms
// around a block.
#include "../../include/linfusion_block.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "block_kernels.cuh"
#include "host_util.h"

using namespace lf;

namespace {

// The current device and its SM count.
struct Here {
    int device, sms;
    linfusion_status_t st;
};
Here here()
{
    Here h = {0, 0, LINFUSION_OK};
    if (cudaGetDevice(&h.device) != cudaSuccess) {
        cudaGetLastError();
        h.st = LINFUSION_ERR_CUDA;
        return h;
    }
    h.sms = device_sm_count(h.device);
    if (h.sms == -2) h.st = LINFUSION_ERR_UNSUPPORTED;
    else if (h.sms < 0) h.st = LINFUSION_ERR_CUDA;
    return h;
}

linfusion_status_t end(cudaError_t e)
{
    if (e == cudaSuccess) return LINFUSION_OK;
    cudaGetLastError();
    return LINFUSION_ERR_CUDA;
}

// An axis of n rows, s elements apart: whole 16-byte pieces, and within 2^46 elements, so that sums of such reaches are exact.
// The stride of an axis of one row says nothing.
bool good_stride(int64_t n, int64_t s) { return n <= 1 || (s >= 0 && s % 8 == 0 && s <= (int64_t(1) << 46) / (n - 1)); }

// The bytes from the first to behind the last element that strides reach, as a half-open range.
struct Extent {
    const char* p;
    size_t bytes;
};
Extent extent(const void* p, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t row)
{
    const int64_t last = (n0 - 1) * s0 + (n1 - 1) * s1 + (n2 - 1) * s2 + row;
    return {static_cast<const char*>(p), static_cast<size_t>(last) * 2};
}
bool meet(const Extent& a, const Extent& b) { return overlaps(a.p, a.bytes, b.p, b.bytes); }

// Rows of `row` elements over axes of length n and stride s: no two of them share an element when, taken from the
// smallest stride to the largest, each stride steps over everything below it.  Axes of length one do not count.
struct Axis {
    int64_t n, s;
};
bool rows_disjoint(std::initializer_list<Axis> axes, int64_t row)
{
    Axis a[4];
    int count = 0;
    for (const Axis& x : axes)
        if (x.n > 1) a[count++] = x;
    std::sort(a, a + count, [](const Axis& x, const Axis& y) { return x.s < y.s; });
    int64_t reach = row;
    for (int i = 0; i < count; ++i) {
        if (a[i].s < reach) return false;
        reach += (a[i].n - 1) * a[i].s;
    }
    return true;
}

// ------------------------------------------------------------------------------------------ rope
linfusion_status_t check_rope(const linfusion_rope_desc_t* d, int* pairs)
{
    if (d == nullptr) return LINFUSION_ERR_INVALID_ARG;
    if (d->B <= 0 || d->N <= 0 || d->d <= 0 || d->d % 8 != 0) return LINFUSION_ERR_INVALID_ARG;
    if (d->n_axes < 1 || d->n_axes > LINFUSION_ROPE_MAX_AXES) return LINFUSION_ERR_INVALID_ARG;
    if (!std::isfinite(d->theta) || d->theta <= 0.0) return LINFUSION_ERR_INVALID_ARG;
    if ((d->interleaved & ~1) != 0 || (d->backward & ~1) != 0) return LINFUSION_ERR_INVALID_ARG;
    if (d->d > LINFUSION_ROPE_MAX_WIDTH || d->B > 65535) return LINFUSION_ERR_UNSUPPORTED;
    if ((d->flags & ~LINFUSION_DTYPE_FP16) != 0u) return LINFUSION_ERR_UNSUPPORTED;
    int64_t sum = 0;
    for (int a = 0; a < d->n_axes; ++a) {
        if (d->pairs[a] < 0) return LINFUSION_ERR_INVALID_ARG;
        sum += d->pairs[a];
    }
    if (sum < 1 || 2 * sum > d->d) return LINFUSION_ERR_INVALID_ARG;
    // theta^(-j / n) of the last pair of an axis is its largest where theta is below 1
    for (int a = 0; a < d->n_axes; ++a)
        if (d->pairs[a] > 0 && !(std::pow(d->theta, -static_cast<double>(d->pairs[a] - 1) / d->pairs[a]) <= 1e30)) return LINFUSION_ERR_INVALID_ARG;
    *pairs = static_cast<int>(sum);
    return LINFUSION_OK;
}

linfusion_status_t check_rope_tensor(const linfusion_rope_desc_t& d, const linfusion_rope_tensor_t& t)
{
    if (t.in == nullptr || t.out == nullptr || !is_aligned(t.in, 16) || !is_aligned(t.out, 16)) return LINFUSION_ERR_INVALID_ARG;
    if (!good_stride(d.B, t.in_batch) || !good_stride(d.N, t.in_token) || !good_stride(t.heads, t.in_head) ||
        !good_stride(d.B, t.out_batch) || !good_stride(d.N, t.out_token) || !good_stride(t.heads, t.out_head))
        return LINFUSION_ERR_INVALID_ARG;
    // no two output rows on top of one another
    if (!rows_disjoint({{d.B, t.out_batch}, {d.N, t.out_token}, {t.heads, t.out_head}}, d.d)) return LINFUSION_ERR_INVALID_ARG;
    const Extent in = extent(t.in, d.B, t.in_batch, d.N, t.in_token, t.heads, t.in_head, d.d);
    const Extent out = extent(t.out, d.B, t.out_batch, d.N, t.out_token, t.heads, t.out_head, d.d);
    const bool in_place = t.in == t.out && (d.B == 1 || t.in_batch == t.out_batch) && (d.N == 1 || t.in_token == t.out_token) &&
                          (t.heads == 1 || t.in_head == t.out_head);
    return in_place || !meet(in, out) ? LINFUSION_OK : LINFUSION_ERR_INVALID_ARG;
}

struct RopeView {
    const char* p;
    int64_t heads, batch, token, head;
};
RopeView rope_view(const linfusion_rope_tensor_t& t, bool out)
{
    return out ? RopeView{static_cast<const char*>(t.out), t.heads, t.out_batch, t.out_token, t.out_head}
               : RopeView{static_cast<const char*>(t.in), t.heads, t.in_batch, t.in_token, t.in_head};
}
// Two views share no element: they lie apart, or they are interlaced views of one tensor with the same strides (Q and K
// side by side in each token, or one behind the other in each batch entry).  What neither test can tell is refused.
bool views_apart(const linfusion_rope_desc_t& d, RopeView a, RopeView b)
{
    const Extent ea = extent(a.p, d.B, a.batch, d.N, a.token, a.heads, a.head, d.d);
    const Extent eb = extent(b.p, d.B, b.batch, d.N, b.token, b.heads, b.head, d.d);
    if (!meet(ea, eb)) return true;
    if ((d.B > 1 && a.batch != b.batch) || (d.N > 1 && a.token != b.token)) return false;
    if (b.p < a.p) std::swap(a, b);
    const int64_t bytes = b.p - a.p;
    if (bytes % 16 != 0) return false;
    const int64_t apart = bytes / 2, heads_a = (a.heads - 1) * a.head + d.d, heads_b = (b.heads - 1) * b.head + d.d;
    if (apart >= heads_a && rows_disjoint({{d.B, a.batch}, {d.N, a.token}}, apart + heads_b)) return true;
    if (a.heads > 1 && b.heads > 1 && a.head != b.head) return false;
    const RopeView& more = a.heads >= b.heads ? a : b;
    return rows_disjoint({{d.B, a.batch}, {d.N, a.token}, {more.heads, more.head}, {2, apart}}, d.d);
}

template <int KIND>
cudaError_t launch_rope(const RopeParams& p, int pairs, dim3 grid, int threads, cudaStream_t s)
{
    switch (pairs) {
        case kRopeInterleaved: rope_kernel<KIND, kRopeInterleaved><<<grid, threads, 0, s>>>(p); break;
        case kRopeHalves: rope_kernel<KIND, kRopeHalves><<<grid, threads, 0, s>>>(p); break;
        case 4: rope_kernel<KIND, 4><<<grid, threads, 0, s>>>(p); break;
        case 2: rope_kernel<KIND, 2><<<grid, threads, 0, s>>>(p); break;
        default: rope_kernel<KIND, 1><<<grid, threads, 0, s>>>(p); break;
    }
    return cudaGetLastError();
}

// ------------------------------------------------------------------------------------------ norms
linfusion_status_t check_norm(const linfusion_block_norm_desc_t* d)
{
    if (d == nullptr) return LINFUSION_ERR_INVALID_ARG;
    if (d->B <= 0 || d->N <= 0 || d->C <= 0) return LINFUSION_ERR_INVALID_ARG;
    if (!std::isfinite(d->eps) || d->eps < 0.0f || !std::isfinite(d->residual_scale)) return LINFUSION_ERR_INVALID_ARG;
    if (d->C % 8 != 0 || d->C > LINFUSION_BLOCK_NORM_MAX_C || d->B > 65534) return LINFUSION_ERR_UNSUPPORTED;
    if ((d->flags & ~LINFUSION_DTYPE_FP16) != 0u) return LINFUSION_ERR_UNSUPPORTED;
    for (const int32_t n : {d->pre, d->post})
        if (n < LINFUSION_NORM_NONE || n > LINFUSION_NORM_RMS) return LINFUSION_ERR_UNSUPPORTED;
    return LINFUSION_OK;
}

bool rows_given(const linfusion_rows_t* r) { return r != nullptr && r->p != nullptr; }
bool rows_ok(const linfusion_block_norm_desc_t& d, const linfusion_rows_t* r)
{
    return rows_given(r) && is_aligned(r->p, 16) && good_stride(d.B, r->batch) && good_stride(d.N, r->row);
}
Rows to_rows(const linfusion_rows_t* r)
{
    Rows o = {nullptr, 0, 0};
    if (rows_given(r)) o = {static_cast<char*>(r->p), r->batch * 2, r->row * 2};
    return o;
}
bool channels_ok(int B, const linfusion_channels_t& c) { return c.p == nullptr || (is_aligned(c.p, 16) && good_stride(B, c.batch)); }
Channels to_channels(const linfusion_channels_t& c) { return {static_cast<const char*>(c.p), c.batch * 2}; }

// What the forward and the backward pass ask of the vectors.
bool vectors_ok(const linfusion_block_norm_desc_t& d, const linfusion_block_norm_vectors_t& v, bool branch)
{
    if (!channels_ok(d.B, v.gate) || !channels_ok(d.B, v.scale) || !channels_ok(d.B, v.shift)) return false;
    for (const void* p : {v.pre_weight, v.pre_bias, v.post_weight, v.post_bias})
        if (p != nullptr && !is_aligned(p, 16)) return false;
    if ((v.scale.p == nullptr) != (v.shift.p == nullptr)) return false;
    if (d.pre == LINFUSION_NORM_NONE && (v.scale.p != nullptr || v.pre_weight != nullptr || v.pre_bias != nullptr)) return false;
    if (d.post == LINFUSION_NORM_NONE && (v.post_weight != nullptr || v.post_bias != nullptr)) return false;
    if (!branch && (d.post != LINFUSION_NORM_NONE || v.gate.p != nullptr)) return false;
    return branch || d.pre != LINFUSION_NORM_NONE;
}

Extent rows_extent(const linfusion_block_norm_desc_t& d, const linfusion_rows_t* r)
{
    return extent(r->p, d.B, r->batch, d.N, r->row, 1, 0, d.C);
}
bool out_ok(const linfusion_block_norm_desc_t& d, const linfusion_rows_t* r)
{
    return rows_ok(d, r) && rows_disjoint({{d.B, r->batch}, {d.N, r->row}}, d.C);
}
// `out` shares no memory with `in`, or lies exactly over it and may.
bool apart(const linfusion_block_norm_desc_t& d, const linfusion_rows_t* out, const linfusion_rows_t* in, bool may_lie_over)
{
    if (!rows_given(in) || !meet(rows_extent(d, out), rows_extent(d, in))) return true;
    return may_lie_over && out->p == in->p && (d.B == 1 || out->batch == in->batch) && (d.N == 1 || out->row == in->row);
}
// `out` shares no memory with a vector.
bool apart(const linfusion_block_norm_desc_t& d, const linfusion_rows_t* out, const linfusion_block_norm_vectors_t& v)
{
    const Extent o = rows_extent(d, out);
    for (const linfusion_channels_t& c : {v.gate, v.scale, v.shift})
        if (c.p != nullptr && meet(o, extent(c.p, d.B, c.batch, 1, 0, 1, 0, d.C))) return false;
    for (const void* p : {v.pre_weight, v.pre_bias, v.post_weight, v.post_bias})
        if (p != nullptr && meet(o, extent(p, 1, 0, 1, 0, 1, 0, d.C))) return false;
    return true;
}

// The vectors' gradients and the workspace (where `workspace_bytes` of one is used) share no memory with each other, with a tensor
// of the call or with a vector.
bool sums_apart(const linfusion_block_norm_desc_t& d, const linfusion_block_norm_vectors_t& v, const linfusion_block_norm_grads_t& g,
                std::initializer_list<const linfusion_rows_t*> tensors, const void* workspace, size_t workspace_bytes)
{
    const size_t shared = static_cast<size_t>(d.C) * 4, each = shared * d.B;
    const auto bytes = [&](const linfusion_channels_t& c, uint32_t bit) { return c.batch != 0 || (g.per_entry & bit) != 0u ? each : shared; };
    const Extent sums[8] = {{reinterpret_cast<const char*>(g.gate), bytes(v.gate, LINFUSION_PER_ENTRY_GATE)},
                            {reinterpret_cast<const char*>(g.scale), bytes(v.scale, LINFUSION_PER_ENTRY_SCALE)},
                            {reinterpret_cast<const char*>(g.shift), bytes(v.shift, LINFUSION_PER_ENTRY_SHIFT)},
                            {reinterpret_cast<const char*>(g.pre_weight), shared},
                            {reinterpret_cast<const char*>(g.pre_bias), shared},
                            {reinterpret_cast<const char*>(g.post_weight), shared},
                            {reinterpret_cast<const char*>(g.post_bias), shared},
                            {workspace_bytes != 0 ? static_cast<const char*>(workspace) : nullptr, workspace_bytes}};
    for (int i = 0; i < 8; ++i) {
        if (sums[i].p == nullptr) continue;
        for (int j = 0; j < i; ++j)
            if (sums[j].p != nullptr && meet(sums[i], sums[j])) return false;
        for (const linfusion_rows_t* t : tensors)
            if (rows_given(t) && meet(sums[i], rows_extent(d, t))) return false;
        for (const linfusion_channels_t& c : {v.gate, v.scale, v.shift})
            if (c.p != nullptr && meet(sums[i], extent(c.p, d.B, c.batch, 1, 0, 1, 0, d.C))) return false;
        for (const void* p : {v.pre_weight, v.pre_bias, v.post_weight, v.post_bias})
            if (p != nullptr && meet(sums[i], extent(p, 1, 0, 1, 0, 1, 0, d.C))) return false;
    }
    return true;
}

// How rows are dealt out: groups of `warps` warps, each thread with `vectors` pieces of eight channels, `per_cta` groups in
// a block, `chunks` groups for each batch entry.
struct NormPlan {
    int vectors, warps, per_cta, chunks, groups, ctas;
};
// Sixteen channels a thread in the forward pass wherever eight do not leave a row to one warp: half the warps to exchange a
// row's sums, more rows in flight (us, sixteen / eight: 21 / 26 at 3 x 8192 x 320, 25 / 30 at 2 x 8192 x 640, 29 / 34 at 2 x 8192 x
// 1024, 28 / 34 at 2 x 4096 x 2048; 68.6 / 69.1 at 2 x 16384 x 1280, 23 / 22 at 2 x 4096 x 1280, where the third warp is half empty).
// The backward pass keeps four column sums of each channel and has no registers for that (162 / 117 at 2 x 16384 x 1280, 53 / 53
// at 2 x 8192 x 1024), but where sixteen channels leave a row to one warp (43 / 50 at 2 x 16384 x 320, 20 / 21 at 2 x 4099 x 320;
// 7.2 / 6.4 at 2 x 64 x 320).  Above 4096 channels eight would not do.
NormPlan norm_plan(const linfusion_block_norm_desc_t& d, int sms, bool backward)
{
    NormPlan p;
    p.vectors = d.C <= 256 ? 1 : !backward ? 2 : d.C > 256 * kNormMaxWarps || d.C <= 512 ? 2 : 1;
    p.warps = (d.C + 256 * p.vectors - 1) / (256 * p.vectors);
    p.per_cta = p.warps >= 4 ? 1 : 4 / p.warps;
    // As many groups as run at once, so that none waits for another to end; fewer where there are fewer rows.  At 128
    // registers a thread an SM holds sixteen warps (but four blocks of three); at the 212 of two vectors in one warp, eight.
    const int block = p.warps * p.per_cta, per_sm = backward && p.vectors == 2 && p.warps == 1 ? 2 : block == 3 ? 4 : 16 / block;
    const long long target = static_cast<long long>(sms) * per_sm * p.per_cta;
    long long chunks = target / d.B;
    if (chunks > d.N) chunks = d.N;
    if (chunks < 1) chunks = 1;
    p.chunks = static_cast<int>(chunks);
    p.groups = p.chunks * d.B;
    p.ctas = (p.groups + p.per_cta - 1) / p.per_cta;
    return p;
}

void fill(NormParams* p, const linfusion_block_norm_desc_t& d, const linfusion_block_norm_vectors_t& v, const NormPlan& plan, bool branch)
{
    p->gate = to_channels(v.gate);
    p->scale = to_channels(v.scale);
    p->shift = to_channels(v.shift);
    p->pre_w = static_cast<const char*>(v.pre_weight);
    p->pre_b = static_cast<const char*>(v.pre_bias);
    p->post_w = static_cast<const char*>(v.post_weight);
    p->post_b = static_cast<const char*>(v.post_bias);
    p->N = d.N;
    p->C = d.C;
    p->warps = plan.warps;
    p->chunks = plan.chunks;
    p->groups = plan.groups;
    p->eps = d.eps;
    p->rs = branch ? d.residual_scale : 1.0f;  // without a branch y is x itself
    p->inv_c = 1.0f / static_cast<float>(d.C);
    p->last = static_cast<float>(d.C - 256 * plan.vectors * (plan.warps - 1));
    p->inv_last = 1.0f / p->last;
}

template <int KIND, int POST, int PRE, bool A, int V, int J, bool BACKWARD>
cudaError_t launch_norm_one(const NormParams& p, const NormPlan& plan, int device, cudaStream_t s)
{
    static std::atomic<uint64_t> done{0};
    const int threads = 32 * plan.warps * plan.per_cta;
    const int streams = BACKWARD ? (PRE != kNormNone ? 2 : 0) + (A ? 2 : 1) : (A ? 2 : 1);
    const size_t smem = norm_smem_bytes(streams, V, threads, plan.per_cta), most = norm_smem_bytes(streams, V, norm_threads(V, J), 4);
    cudaError_t e;
    if constexpr (BACKWARD) {
        e = allow_smem(block_norm_backward_kernel<KIND, POST, PRE, A, V, J>, most, device, &done);
        if (e == cudaSuccess) block_norm_backward_kernel<KIND, POST, PRE, A, V, J><<<plan.ctas, threads, smem, s>>>(p);
    } else {
        e = allow_smem(block_norm_kernel<KIND, POST, PRE, A, V, J>, most, device, &done);
        if (e == cudaSuccess) block_norm_kernel<KIND, POST, PRE, A, V, J><<<plan.ctas, threads, smem, s>>>(p);
    }
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <int KIND, int V, int J, bool BACKWARD>
cudaError_t launch_norm(const NormParams& p, const NormPlan& plan, int post, int pre, bool branch, int device, cudaStream_t s)
{
#define LF_NORM(POST, PRE, A) return launch_norm_one<KIND, POST, PRE, A, V, J, BACKWARD>(p, plan, device, s)
    if (!branch) {
        if (pre == LINFUSION_NORM_LAYER) LF_NORM(kNormNone, kNormLayer, false);
        LF_NORM(kNormNone, kNormRms, false);
    }
    switch (post * 3 + pre) {
        case 0: LF_NORM(kNormNone, kNormNone, true);
        case 1: LF_NORM(kNormNone, kNormLayer, true);
        case 2: LF_NORM(kNormNone, kNormRms, true);
        case 3: LF_NORM(kNormLayer, kNormNone, true);
        case 4: LF_NORM(kNormLayer, kNormLayer, true);
        case 5: LF_NORM(kNormLayer, kNormRms, true);
        case 6: LF_NORM(kNormRms, kNormNone, true);
        case 7: LF_NORM(kNormRms, kNormLayer, true);
        default: LF_NORM(kNormRms, kNormRms, true);
    }
#undef LF_NORM
}

template <bool BACKWARD>
cudaError_t launch_norm_kind(const linfusion_block_norm_desc_t& d, const NormParams& p, const NormPlan& plan, bool branch, int device,
                             cudaStream_t s)
{
    const bool half = (d.flags & LINFUSION_DTYPE_FP16) != 0u;
    constexpr int bf = make_kind(kPhiIdentity, kDtypeBf16), hf = make_kind(kPhiIdentity, kDtypeFp16);
#define LF_SIZED(V, J)                                                                            \
    return half ? launch_norm<hf, V, J, BACKWARD>(p, plan, d.post, d.pre, branch, device, s)       \
                : launch_norm<bf, V, J, BACKWARD>(p, plan, d.post, d.pre, branch, device, s)
    if (plan.vectors == 1 && plan.warps == 1) LF_SIZED(1, 0);
    if (plan.warps == 1) LF_SIZED(2, 0);
    if (plan.vectors == 2 && plan.warps > 8) LF_SIZED(2, 4);
    if constexpr (BACKWARD) {
        if (plan.warps > 8) LF_SIZED(1, 4);
        LF_SIZED(1, 3);
    } else {
        LF_SIZED(2, 3);
    }
#undef LF_SIZED
}

}  // namespace

extern "C" {

linfusion_status_t linfusion_rope(const linfusion_rope_desc_t* desc, const linfusion_rope_tensor_t* q,
                                  const linfusion_rope_tensor_t* k, const float* positions, int64_t pos_batch_stride,
                                  void* cuda_stream)
{
    int P = 0;
    linfusion_status_t st = check_rope(desc, &P);
    if (st != LINFUSION_OK) return st;
    const linfusion_rope_tensor_t* given[2] = {q != nullptr && q->heads != 0 ? q : nullptr,
                                               k != nullptr && k->heads != 0 ? k : nullptr};
    if (given[0] == nullptr && given[1] == nullptr) return LINFUSION_ERR_INVALID_ARG;
    if (positions == nullptr || !is_aligned(positions, 4) || pos_batch_stride < 0 || pos_batch_stride >= (int64_t(1) << 40)) return LINFUSION_ERR_INVALID_ARG;
    const Extent pos = {reinterpret_cast<const char*>(positions),
                        4 * (static_cast<size_t>(desc->B - 1) * pos_batch_stride + static_cast<size_t>(desc->N) * desc->n_axes)};
    for (const linfusion_rope_tensor_t* t : given)
        if (t != nullptr) {
            if (t->heads < 0) return LINFUSION_ERR_INVALID_ARG;
            st = check_rope_tensor(*desc, *t);
            if (st != LINFUSION_OK) return st;
            if (meet(pos, extent(t->out, desc->B, t->out_batch, desc->N, t->out_token, t->heads, t->out_head, desc->d)))
                return LINFUSION_ERR_INVALID_ARG;
        }
    if (given[0] != nullptr && given[1] != nullptr) {
        if (static_cast<int64_t>(given[0]->heads) + given[1]->heads > INT32_MAX) return LINFUSION_ERR_UNSUPPORTED;
        const linfusion_rope_tensor_t &a = *given[0], &b = *given[1];
        const RopeView ai = rope_view(a, false), ao = rope_view(a, true), bi = rope_view(b, false), bo = rope_view(b, true);
        if (!views_apart(*desc, ao, bo) || !views_apart(*desc, ao, bi) || !views_apart(*desc, bo, ai)) return LINFUSION_ERR_INVALID_ARG;
    }
    const Here at = here();
    if (at.st != LINFUSION_OK) return at.st;

    RopeParams p = {};
    int heads = 0;
    for (int w = 0; w < 2; ++w) {
        if (given[w] == nullptr) continue;
        const linfusion_rope_tensor_t& t = *given[w];
        p.t[w] = {static_cast<const char*>(t.in), static_cast<char*>(t.out), t.heads, t.in_batch * 2, t.in_token * 2,
                  t.in_head * 2, t.out_batch * 2, t.out_token * 2, t.out_head * 2};
        heads += t.heads;
    }
    p.pos = positions;
    p.pos_b = pos_batch_stride;
    p.N = desc->N;
    p.d = desc->d;
    p.P = P;
    p.n_axes = desc->n_axes;
    p.sign = desc->backward ? -1.0f : 1.0f;
    const int pairs = desc->interleaved != 0 ? kRopeInterleaved : P % 8 == 0 ? kRopeHalves : P % 4 == 0 ? 4 : P % 2 == 0 ? 2 : 1;
    p.pair_items = P / 8;                                                                         // halves only
    p.items = pairs == kRopeHalves ? p.pair_items + (desc->d - 2 * P) / 8 : desc->d / 8;
    for (int a = 0, i = 0; a < desc->n_axes; ++a)
        for (int j = 0; j < desc->pairs[a]; ++j, ++i) {
            const double turns = std::pow(desc->theta, -static_cast<double>(j) / desc->pairs[a]) / 6.283185307179586476925;
            p.axis[i] = static_cast<unsigned char>(a);
            p.f_hi[i] = static_cast<float>(turns);
            p.f_lo[i] = static_cast<float>(turns - static_cast<double>(p.f_hi[i]));
        }
    // Head groups: a block goes through its group's heads and forms its sines and cosines once, at the price of about three
    // heads.  What counts is how many rounds of blocks the machine goes through (four blocks on an SM) times what one does.
    const long long threads = static_cast<long long>(desc->N) * p.items;
    // (where partners are gathered a block holds whole rows)
    const int block = pairs < kRopeHalves ? kRopeThreads / p.items * p.items : kRopeThreads;
    const long long blocks = (threads + block - 1) / block;
    if (threads + kRopeThreads > 0xffffffffll) return LINFUSION_ERR_UNSUPPORTED;
    p.heads_per_group = heads;
    double best = 1e300;
    for (int g = 1; g <= heads && g <= 64; ++g) {
        const int per_group = (heads + g - 1) / g;
        const long long all = blocks * desc->B * ((heads + per_group - 1) / per_group), rounds = (all + 4 * at.sms - 1) / (4 * at.sms);
        const double cost = static_cast<double>(rounds) * (3 + per_group);
        if (cost < best) best = cost, p.heads_per_group = per_group;
    }
    const long long grid_y = (heads + p.heads_per_group - 1) / p.heads_per_group;
    if (grid_y > 65535) return LINFUSION_ERR_UNSUPPORTED;
    const dim3 grid(static_cast<unsigned int>(blocks), static_cast<unsigned int>(grid_y), desc->B);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return end((desc->flags & LINFUSION_DTYPE_FP16) != 0u
                   ? launch_rope<make_kind(kPhiIdentity, kDtypeFp16)>(p, pairs, grid, block, s)
                   : launch_rope<make_kind(kPhiIdentity, kDtypeBf16)>(p, pairs, grid, block, s));
}

linfusion_status_t linfusion_block_norm(const linfusion_block_norm_desc_t* desc, const linfusion_rows_t* x,
                                        const linfusion_rows_t* a, const linfusion_block_norm_vectors_t* v,
                                        const linfusion_rows_t* y, const linfusion_rows_t* n, void* cuda_stream)
{
    linfusion_status_t st = check_norm(desc);
    if (st != LINFUSION_OK) return st;
    const linfusion_block_norm_vectors_t none = {};
    if (v == nullptr) v = &none;
    const bool branch = rows_given(a), pre = desc->pre != LINFUSION_NORM_NONE;
    if (!vectors_ok(*desc, *v, branch) || !rows_ok(*desc, x) || (branch && !rows_ok(*desc, a))) return LINFUSION_ERR_INVALID_ARG;
    if (rows_given(y) != branch || rows_given(n) != pre) return LINFUSION_ERR_INVALID_ARG;
    if (branch && (!out_ok(*desc, y) || !apart(*desc, y, x, true) || !apart(*desc, y, a, true) || !apart(*desc, y, *v)))
        return LINFUSION_ERR_INVALID_ARG;
    if (pre && (!out_ok(*desc, n) || !apart(*desc, n, x, false) || !apart(*desc, n, a, false) || !apart(*desc, n, y, false) ||
                !apart(*desc, n, *v)))
        return LINFUSION_ERR_INVALID_ARG;
    const Here at = here();
    if (at.st != LINFUSION_OK) return at.st;
    const NormPlan plan = norm_plan(*desc, at.sms, false);
    NormParams p = {};
    fill(&p, *desc, *v, plan, branch);
    p.x = to_rows(x);
    p.a = to_rows(a);
    p.y = to_rows(y);
    p.n = to_rows(n);
    return end(launch_norm_kind<false>(*desc, p, plan, branch, at.device, static_cast<cudaStream_t>(cuda_stream)));
}

linfusion_status_t linfusion_block_norm_workspace_bytes(const linfusion_block_norm_desc_t* desc, int32_t sm_count, size_t* bytes)
{
    if (bytes == nullptr) return LINFUSION_ERR_INVALID_ARG;
    const linfusion_status_t st = check_norm(desc);
    if (st != LINFUSION_OK) return st;
    const NormPlan plan = norm_plan(*desc, sm_count > 0 ? sm_count : 148, true);
    *bytes = align_up_256(static_cast<size_t>(4) * plan.groups * desc->C * sizeof(float));
    return LINFUSION_OK;
}

linfusion_status_t linfusion_block_norm_backward(const linfusion_block_norm_desc_t* desc, const linfusion_rows_t* y,
                                                 const linfusion_rows_t* a, const linfusion_block_norm_vectors_t* v,
                                                 const linfusion_rows_t* dy, const linfusion_rows_t* dn,
                                                 const linfusion_rows_t* dx, const linfusion_rows_t* da,
                                                 const linfusion_block_norm_grads_t* grads, void* workspace,
                                                 size_t workspace_bytes, void* cuda_stream)
{
    linfusion_status_t st = check_norm(desc);
    if (st != LINFUSION_OK) return st;
    const linfusion_block_norm_vectors_t none = {};
    const linfusion_block_norm_grads_t no_grads = {};
    if (v == nullptr) v = &none;
    if (grads == nullptr) grads = &no_grads;
    const bool branch = rows_given(a), pre = desc->pre != LINFUSION_NORM_NONE;
    if (!vectors_ok(*desc, *v, branch) || (branch && !rows_ok(*desc, a))) return LINFUSION_ERR_INVALID_ARG;
    if (pre && (!rows_ok(*desc, y) || !rows_ok(*desc, dn))) return LINFUSION_ERR_INVALID_ARG;
    if (!pre && (rows_given(dn) || !rows_ok(*desc, dy))) return LINFUSION_ERR_INVALID_ARG;
    if (rows_given(dy) && !rows_ok(*desc, dy)) return LINFUSION_ERR_INVALID_ARG;
    if (!out_ok(*desc, dx) || rows_given(da) != branch || (branch && !out_ok(*desc, da))) return LINFUSION_ERR_INVALID_ARG;
    const linfusion_rows_t* y_read = pre ? y : nullptr;
    if (!apart(*desc, dx, y_read, false) || !apart(*desc, dx, a, false) || !apart(*desc, dx, dy, true) ||
        !apart(*desc, dx, dn, false) || !apart(*desc, dx, *v))
        return LINFUSION_ERR_INVALID_ARG;
    if (branch && (!apart(*desc, da, y_read, false) || !apart(*desc, da, a, true) || !apart(*desc, da, dy, false) ||
                   !apart(*desc, da, dn, false) || !apart(*desc, da, dx, false) || !apart(*desc, da, *v)))
        return LINFUSION_ERR_INVALID_ARG;
    if ((grads->per_entry & ~(LINFUSION_PER_ENTRY_GATE | LINFUSION_PER_ENTRY_SCALE | LINFUSION_PER_ENTRY_SHIFT)) != 0u)
        return LINFUSION_ERR_INVALID_ARG;
    // a gradient of a vector that is not there
    if ((grads->gate != nullptr && v->gate.p == nullptr) || (grads->scale != nullptr && v->scale.p == nullptr) ||
        (grads->shift != nullptr && v->shift.p == nullptr) || (grads->pre_weight != nullptr && v->pre_weight == nullptr) ||
        (grads->pre_bias != nullptr && v->pre_bias == nullptr) || (grads->post_weight != nullptr && v->post_weight == nullptr) ||
        (grads->post_bias != nullptr && v->post_bias == nullptr))
        return LINFUSION_ERR_INVALID_ARG;
    for (const float* g : {grads->gate, grads->scale, grads->shift, grads->pre_weight, grads->pre_bias, grads->post_weight,
                           grads->post_bias})
        if (g != nullptr && !is_aligned(g, 4)) return LINFUSION_ERR_INVALID_ARG;
    int want = 0;
    if (grads->shift || grads->scale || grads->pre_bias) want |= 1;  // a bias' share of the scale's gradient needs sum dn
    if (grads->scale || grads->pre_weight) want |= 2;
    if (grads->gate || grads->post_weight) want |= 4;
    if (grads->post_bias || (grads->gate && v->post_bias)) want |= 8;

    if (want != 0 && (workspace == nullptr || !is_aligned(workspace, 256))) return LINFUSION_ERR_INVALID_ARG;
    // The check of the workspace's range: what the call uses of it on the device, or, before that is known, on a B200.
    const auto needs = [&](const NormPlan& plan) {
        return want == 0 ? 0 : align_up_256(static_cast<size_t>(4) * plan.groups * desc->C * sizeof(float));
    };
    const auto clear = [&](size_t bytes) {
        return sums_apart(*desc, *v, *grads, {y_read, a, dy, dn, dx, da}, workspace, std::min(bytes, workspace_bytes));
    };
    constexpr int kSms = 148;
    if (!clear(needs(norm_plan(*desc, kSms, true)))) return LINFUSION_ERR_INVALID_ARG;
    const Here at = here();
    if (at.st != LINFUSION_OK) return at.st;
    const NormPlan plan = norm_plan(*desc, at.sms, true);
    if (want != 0 && workspace_bytes < needs(plan)) return LINFUSION_ERR_ALLOC;
    if (at.sms != kSms && !clear(needs(plan))) return LINFUSION_ERR_INVALID_ARG;
    NormParams p = {};
    fill(&p, *desc, *v, plan, branch);
    p.x = to_rows(y);
    p.a = to_rows(a);
    p.dy = to_rows(dy);
    p.dn = to_rows(dn);
    p.dx = to_rows(dx);
    p.da = to_rows(da);
    p.partials = static_cast<float*>(workspace);
    p.want = want;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e = launch_norm_kind<true>(*desc, p, plan, branch, at.device, s);
    if (e != cudaSuccess || want == 0) return end(e);

    NormGradParams g = {};
    g.partials = p.partials;
    g.B = desc->B;
    g.C = desc->C;
    g.chunks = plan.chunks;
    g.groups = plan.groups;
    g.want = want;
    g.gate = p.gate;
    g.scale = p.scale;
    g.pre_w = p.pre_w;
    g.pre_b = p.pre_b;
    g.post_w = p.post_w;
    g.post_b = p.post_b;
    g.gate_per_batch = v->gate.batch != 0 || (grads->per_entry & LINFUSION_PER_ENTRY_GATE) != 0u;
    g.scale_per_batch = v->scale.batch != 0 || (grads->per_entry & LINFUSION_PER_ENTRY_SCALE) != 0u;
    g.shift_per_batch = v->shift.batch != 0 || (grads->per_entry & LINFUSION_PER_ENTRY_SHIFT) != 0u;
    g.d_gate = grads->gate;
    g.d_scale = grads->scale;
    g.d_shift = grads->shift;
    g.d_pre_w = grads->pre_weight;
    g.d_pre_b = grads->pre_bias;
    g.d_post_w = grads->post_weight;
    g.d_post_b = grads->post_bias;
    const bool own = (g.d_gate != nullptr && g.gate_per_batch) || (g.d_scale != nullptr && g.scale_per_batch) ||
                     (g.d_shift != nullptr && g.shift_per_batch);
    const dim3 grid(desc->C / kNormGradChannels, own ? 1 + desc->B : 1), block(kNormGradThreads);
    e = (desc->flags & LINFUSION_DTYPE_FP16) != 0u
            ? launch_pdl(block_norm_grads_kernel<make_kind(kPhiIdentity, kDtypeFp16)>, grid, block, 0, s, g)
            : launch_pdl(block_norm_grads_kernel<make_kind(kPhiIdentity, kDtypeBf16)>, grid, block, 0, s, g);
    return end(e);
}

}  // extern "C"
