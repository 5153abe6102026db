// Host side of the gated linear recurrence of include/linfusion_layers.h: argument checks, workspace and launches.
#include "../../include/linfusion_layers.h"

#include "host_checks.h"
#include "recurrence_kernels.cuh"

using namespace lf;

namespace {

linfusion_status_t check(const linfusion_recurrence_desc_t* d)
{
    if (d == nullptr || d->B <= 0 || d->N <= 0 || d->C <= 0 || d->C % 8 != 0 || (d->reverse & ~1) != 0) return LINFUSION_ERR_INVALID_ARG;
    if ((d->flags & ~LINFUSION_DTYPE_FP16) != 0u) return LINFUSION_ERR_UNSUPPORTED;
    // positions, tiles and rows are counted in 32 bits
    if (d->N > INT32_MAX - kRecEvery || d->C > INT32_MAX - kRecSlab) return LINFUSION_ERR_UNSUPPORTED;
    const int64_t tiles = (d->N + kRecEvery - 1) / kRecEvery, slabs = (d->C + kRecSlab - 1) / kRecSlab;
    // and the grid is slabs x 32768 tiles x the rest
    if (d->B * ((tiles + kRecTilesY - 1) / kRecTilesY) > 65535) return LINFUSION_ERR_UNSUPPORTED;
    return d->B * tiles <= INT32_MAX / slabs ? LINFUSION_OK : LINFUSION_ERR_UNSUPPORTED;
}

// The tiles of a call, and where the parts of its workspace are.
struct Plan {
    int slabs, tiles, width;
    size_t maps, grad_maps, enters, kept, rate, bytes;
};
// `backward`: with the rates' sums; `kept`: room for the states that a backward pass recomputes.
Plan make_plan(const linfusion_recurrence_desc_t& d, bool backward, bool kept)
{
    Plan p = {};
    p.slabs = (d.C + kRecSlab - 1) / kRecSlab;
    p.tiles = (d.N + kRecEvery - 1) / kRecEvery;
    p.width = p.slabs * kRecSlab;
    const size_t rows = static_cast<size_t>(d.B) * p.tiles;
    const bool many = p.tiles > 1;
    // maps of the state, and of the gradient behind them where both are formed; else in their place
    const size_t maps = many ? align_up_256(rows * p.width * sizeof(float2)) : 0;
    p.grad_maps = backward && kept ? maps : 0;
    p.enters = p.grad_maps + maps;
    p.kept = p.enters + (many ? align_up_256(rows * d.C * sizeof(float)) : 0);
    p.rate = p.kept + (many && kept ? align_up_256(rows * d.C * sizeof(float)) : 0);
    p.bytes = p.rate + (backward ? align_up_256(rows * p.width * sizeof(float)) : 0);
    return p;
}

bool is_packed(const linfusion_recurrence_input_t* in) { return in->packed.codes != nullptr; }
bool given(const linfusion_recurrence_input_t* in) { return in != nullptr && (in->rows.p != nullptr || in->packed.codes != nullptr); }
bool rows_ok(const linfusion_recurrence_desc_t& d, const linfusion_rows_t& r)
{
    return r.p != nullptr && is_aligned(r.p, 16) && good_stride(d.B, r.batch) && good_stride(d.N, r.row);
}
bool input_ok(const linfusion_recurrence_desc_t& d, const linfusion_recurrence_input_t* in, bool packed)
{
    if (!given(in) || is_packed(in) != packed) return false;
    return packed ? is_aligned(in->packed.codes, 16) && in->packed.scales != nullptr : rows_ok(d, in->rows);
}
int scale_groups(const linfusion_recurrence_desc_t& d) { return (d.C + LINFUSION_PACK8_GROUP - 1) / LINFUSION_PACK8_GROUP; }

// A tensor of the call: rows with strides, or a dense range.
struct View {
    Extent e;
    bool strided;
    linfusion_rows_t r;
};
View view(const linfusion_recurrence_desc_t& d, const linfusion_rows_t& r) { return {extent(r.p, d.B, r.batch, d.N, r.row, 1, 0, d.C), true, r}; }
View view(const void* p, size_t bytes) { return {{static_cast<const char*>(p), bytes}, false, {}}; }
void add_input(const linfusion_recurrence_desc_t& d, const linfusion_recurrence_input_t* in, View* v, int* n)
{
    if (!given(in)) return;
    if (is_packed(in)) {
        const size_t rows = static_cast<size_t>(d.B) * d.N;
        v[(*n)++] = view(in->packed.codes, rows * d.C);
        v[(*n)++] = view(in->packed.scales, rows * scale_groups(d));
    } else {
        v[(*n)++] = view(d, in->rows);
    }
}
// No byte of `a` is one of `b`: their ranges lie apart, or they are windows side by side of rows with the same strides.
bool apart(const linfusion_recurrence_desc_t& d, const View& a, const View& b)
{
    if (!meet(a.e, b.e)) return true;
    if (!a.strided || !b.strided || (d.B > 1 && a.r.batch != b.r.batch) || (d.N > 1 && a.r.row != b.r.row)) return false;
    const int64_t bytes = a.e.p < b.e.p ? b.e.p - a.e.p : a.e.p - b.e.p;
    if (bytes % 2 != 0 || bytes / 2 < d.C) return false;
    return rows_disjoint({{d.B, a.r.batch}, {d.N, a.r.row}}, bytes / 2 + d.C);
}
// `a` lies exactly over `b`.
bool over(const linfusion_recurrence_desc_t& d, const View& a, const View& b)
{
    return a.strided && b.strided && a.e.p == b.e.p && (d.B == 1 || a.r.batch == b.r.batch) && (d.N == 1 || a.r.row == b.r.row);
}
bool output_ok(const linfusion_recurrence_desc_t& d, const linfusion_rows_t& r)
{
    return rows_ok(d, r) && rows_disjoint({{d.B, r.batch}, {d.N, r.row}}, d.C);
}

RecInput to_input(const linfusion_recurrence_desc_t& d, const linfusion_recurrence_input_t* in)
{
    if (!given(in)) return {};
    if (is_packed(in))
        return {static_cast<const char*>(in->packed.codes), static_cast<const unsigned char*>(in->packed.scales),
                static_cast<long long>(d.N) * d.C, d.C};
    return {static_cast<const char*>(in->rows.p), nullptr, in->rows.batch * 2, in->rows.row * 2};
}
RecOutput to_output(const linfusion_rows_t& r) { return {static_cast<char*>(r.p), r.batch * 2, r.row * 2}; }

RecParams base(const linfusion_recurrence_desc_t& d, const Plan& plan, const linfusion_recurrence_input_t* x,
               const linfusion_recurrence_input_t* decay, const linfusion_recurrence_input_t* gate, const float* rate, const float* h0, void* workspace)
{
    RecParams p = {};
    p.x = to_input(d, x);
    p.decay = to_input(d, decay);
    p.gate = to_input(d, gate);
    p.rate = rate;
    p.h0 = h0;
    p.maps = reinterpret_cast<float2*>(static_cast<char*>(workspace) + plan.maps);
    p.B = d.B;
    p.N = d.N;
    p.C = d.C;
    p.slabs = plan.slabs;
    p.tiles = plan.tiles;
    p.stacks = (plan.tiles + kRecTilesY - 1) / kRecTilesY;
    p.width = plan.width;
    p.scale_groups = scale_groups(d);
    p.reverse = d.reverse;
    return p;
}

constexpr int kBf = make_kind(kPhiIdentity, kDtypeBf16), kHf = make_kind(kPhiIdentity, kDtypeFp16);

dim3 blocks(const RecParams& p) { return dim3(p.slabs, p.stacks > 1 ? kRecTilesY : p.tiles, p.B * p.stacks); }

template <int KIND, int WHAT>
cudaError_t launch_maps(const RecParams& p, bool gated, bool packed, cudaStream_t s)
{
    constexpr bool state = (WHAT & kRecMapState) != 0;  // the gradient's maps need no gate
    const dim3 grid = blocks(p), block(kRecMapsThreads);
    constexpr bool may = WHAT != kRecMapState;          // be packed: the forward pass reads 16 bits
    if (state && gated)
        return may && packed ? launch_pdl(recurrence_maps_kernel<KIND, state, may, WHAT>, grid, block, 0, s, p)
                             : launch_pdl(recurrence_maps_kernel<KIND, state, false, WHAT>, grid, block, 0, s, p);
    return may && packed ? launch_pdl(recurrence_maps_kernel<KIND, false, may, WHAT>, grid, block, 0, s, p)
                         : launch_pdl(recurrence_maps_kernel<KIND, false, false, WHAT>, grid, block, 0, s, p);
}
// What enters each tile: the maps, then the way from tile to tile, of the state, the gradient or both.
template <int WHAT>
cudaError_t launch_enters(const linfusion_recurrence_desc_t& d, const RecParams& p, bool gated, bool packed, float* states, float* grads, cudaStream_t s)
{
    const bool half = (d.flags & LINFUSION_DTYPE_FP16) != 0u;
    const cudaError_t e = half ? launch_maps<kHf, WHAT>(p, gated, packed, s) : launch_maps<kBf, WHAT>(p, gated, packed, s);
    if (e != cudaSuccess) return e;
    const RecScan state = {p.maps, p.h0, states, 0}, grad = {p.grad_maps, p.dlast, grads, 1};
    const dim3 grid(static_cast<unsigned int>(p.width / kRecScanChannels) * p.B, WHAT == kRecMapBoth ? 2 : 1), block(kRecScanChannels * kRecScanRuns);
    return launch_pdl(recurrence_scan_kernel, grid, block, 0, s, WHAT == kRecMapGrad ? grad : state, grad, p.tiles, p.width, p.C);
}
template <int KIND>
cudaError_t launch_backward(const RecParams& p, bool gated, bool packed, cudaStream_t s)
{
    const dim3 grid = blocks(p), block(kRecThreads);
    if (gated)
        return packed ? launch_pdl(recurrence_backward_kernel<KIND, true, true>, grid, block, 0, s, p)
                      : launch_pdl(recurrence_backward_kernel<KIND, true, false>, grid, block, 0, s, p);
    return packed ? launch_pdl(recurrence_backward_kernel<KIND, false, true>, grid, block, 0, s, p)
                  : launch_pdl(recurrence_backward_kernel<KIND, false, false>, grid, block, 0, s, p);
}

bool floats_ok(const float* p) { return p == nullptr || is_aligned(p, 16); }

}  // namespace

extern "C" {

linfusion_status_t linfusion_recurrence_workspace_bytes(const linfusion_recurrence_desc_t* desc, int32_t backward, size_t* bytes)
{
    if (bytes == nullptr || backward < 0 || backward > 2) return LINFUSION_ERR_INVALID_ARG;
    const linfusion_status_t st = check(desc);
    if (st != LINFUSION_OK) return st;
    if (backward == 0) {
        *bytes = make_plan(*desc, false, false).bytes;
    } else {
        *bytes = make_plan(*desc, true, backward == 2).bytes;
    }
    return LINFUSION_OK;
}

linfusion_status_t linfusion_recurrence(const linfusion_recurrence_desc_t* desc, const linfusion_recurrence_input_t* x,
                                        const linfusion_recurrence_input_t* decay, const linfusion_recurrence_input_t* gate,
                                        const float* rate, const float* h0, const linfusion_rows_t* h, float* last, float* state,
                                        void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    const linfusion_status_t st = check(desc);
    if (st != LINFUSION_OK) return st;
    const linfusion_recurrence_desc_t& d = *desc;
    const bool gated = given(gate);
    for (const linfusion_recurrence_input_t* in : {x, decay, gate})
        if (given(in) && is_packed(in)) return LINFUSION_ERR_UNSUPPORTED;
    if (!input_ok(d, x, false) || !input_ok(d, decay, false) || (gated && !input_ok(d, gate, false))) return LINFUSION_ERR_INVALID_ARG;
    if (rate == nullptr || !floats_ok(rate) || !floats_ok(h0) || !floats_ok(last) || !floats_ok(state)) return LINFUSION_ERR_INVALID_ARG;
    if (h == nullptr || !output_ok(d, *h)) return LINFUSION_ERR_INVALID_ARG;
    const bool brief = d.N <= kRecShort;
    const Plan plan = make_plan(d, false, false);
    const size_t need = plan.bytes;
    const size_t ends = static_cast<size_t>(d.B) * d.C * 4, kept = ends * plan.tiles;
    View in[8], out[3];
    int ni = 0, no = 0;
    for (const linfusion_recurrence_input_t* i : {x, decay, gate}) add_input(d, i, in, &ni);
    const View vh = view(d, *h);
    for (int i = 0; i < ni; ++i)
        if (!over(d, vh, in[i]) && !apart(d, vh, in[i])) return LINFUSION_ERR_INVALID_ARG;
    in[ni++] = view(rate, static_cast<size_t>(d.C) * 4);
    if (h0 != nullptr) in[ni++] = view(h0, ends);
    out[no++] = vh;
    if (last != nullptr) out[no++] = view(last, ends);
    if (state != nullptr) out[no++] = view(state, kept);
    for (int o = 0; o < no; ++o) {
        for (int j = 0; j < o; ++j)
            if (!apart(d, out[o], out[j])) return LINFUSION_ERR_INVALID_ARG;
        for (int i = 0; i < ni; ++i) {
            if (o == 0 && in[i].strided) continue;  // looked at above
            if (out[o].e.p == reinterpret_cast<const char*>(last) && last == h0 && in[i].e.p == reinterpret_cast<const char*>(h0)) continue;
            if (!apart(d, out[o], in[i])) return LINFUSION_ERR_INVALID_ARG;
        }
    }
    if (need != 0) {
        if (workspace == nullptr || !is_aligned(workspace, 256)) return LINFUSION_ERR_INVALID_ARG;
        if (workspace_bytes < need) return LINFUSION_ERR_ALLOC;
        const View w = view(workspace, need);
        for (int i = 0; i < ni; ++i)
            if (!apart(d, w, in[i])) return LINFUSION_ERR_INVALID_ARG;
        for (int o = 0; o < no; ++o)
            if (!apart(d, w, out[o])) return LINFUSION_ERR_INVALID_ARG;
    }
    const Here at = here();
    if (at.st != LINFUSION_OK) return at.st;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    RecParams p = base(d, plan, x, decay, gate, rate, h0, workspace);
    p.h = to_output(*h);
    p.last = last;
    if (plan.tiles == 1) p.keep = state;
    if (brief) {
        const long long threads = static_cast<long long>(d.B) * (d.C / 2), grid = (threads + kRecShortThreads - 1) / kRecShortThreads;
        if (grid > INT32_MAX) return LINFUSION_ERR_UNSUPPORTED;
        const unsigned int g = static_cast<unsigned int>(grid);
        const bool half = (d.flags & LINFUSION_DTYPE_FP16) != 0u;
        const dim3 block(kRecShortThreads);
        if (half) return end(gated ? launch_pdl(recurrence_short_kernel<kHf, true>, dim3(g), block, 0, s, p) : launch_pdl(recurrence_short_kernel<kHf, false>, dim3(g), block, 0, s, p));
        return end(gated ? launch_pdl(recurrence_short_kernel<kBf, true>, dim3(g), block, 0, s, p) : launch_pdl(recurrence_short_kernel<kBf, false>, dim3(g), block, 0, s, p));
    }
    cudaError_t e = cudaSuccess;
    if (plan.tiles > 1) {
        float* enters = state != nullptr ? state : reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.enters);
        e = launch_enters<kRecMapState>(d, p, gated, false, enters, nullptr, s);
        if (e != cudaSuccess) return end(e);
        p.states = enters;
    }
    const dim3 grid = blocks(p), block(kRecForwardThreads);
    if ((d.flags & LINFUSION_DTYPE_FP16) != 0u)
        e = gated ? launch_pdl(recurrence_kernel<kHf, true>, grid, block, 0, s, p) : launch_pdl(recurrence_kernel<kHf, false>, grid, block, 0, s, p);
    else
        e = gated ? launch_pdl(recurrence_kernel<kBf, true>, grid, block, 0, s, p) : launch_pdl(recurrence_kernel<kBf, false>, grid, block, 0, s, p);
    return end(e);
}

linfusion_status_t linfusion_recurrence_backward(const linfusion_recurrence_desc_t* desc, const linfusion_recurrence_input_t* x,
                                                 const linfusion_recurrence_input_t* decay, const linfusion_recurrence_input_t* gate,
                                                 const float* rate, const float* h0, const float* state, const linfusion_rows_t* dh,
                                                 const float* dlast, const linfusion_recurrence_grads_t* grads, void* workspace,
                                                 size_t workspace_bytes, void* cuda_stream)
{
    const linfusion_status_t st = check(desc);
    if (st != LINFUSION_OK) return st;
    const linfusion_recurrence_desc_t& d = *desc;
    if (!given(x) || grads == nullptr || dh == nullptr) return LINFUSION_ERR_INVALID_ARG;
    const bool gated = given(gate), packed = is_packed(x);
    if (!input_ok(d, x, packed) || !input_ok(d, decay, packed) || (gated && !input_ok(d, gate, packed))) return LINFUSION_ERR_INVALID_ARG;
    if (rate == nullptr || !rows_ok(d, *dh)) return LINFUSION_ERR_INVALID_ARG;
    for (const float* f : {rate, h0, state, dlast, static_cast<const float*>(grads->rate), static_cast<const float*>(grads->h0)})
        if (!floats_ok(f)) return LINFUSION_ERR_INVALID_ARG;
    if (!output_ok(d, grads->x) || !output_ok(d, grads->decay)) return LINFUSION_ERR_INVALID_ARG;
    if ((grads->gate.p != nullptr) != gated || (gated && !output_ok(d, grads->gate))) return LINFUSION_ERR_INVALID_ARG;

    const Plan plan = make_plan(d, true, state == nullptr);
    const size_t ends = static_cast<size_t>(d.B) * d.C * 4, kept = ends * plan.tiles;
    View in[12], out[6];
    int ni = 0, no = 0;
    for (const linfusion_recurrence_input_t* i : {x, decay, gate}) add_input(d, i, in, &ni);
    in[ni++] = view(d, *dh);
    in[ni++] = view(rate, static_cast<size_t>(d.C) * 4);
    if (h0 != nullptr) in[ni++] = view(h0, ends);
    if (state != nullptr) in[ni++] = view(state, kept);
    if (dlast != nullptr) in[ni++] = view(dlast, ends);
    out[no++] = view(d, grads->x);
    out[no++] = view(d, grads->decay);
    if (gated) out[no++] = view(d, grads->gate);
    if (grads->rate != nullptr) out[no++] = view(grads->rate, static_cast<size_t>(d.C) * 4);
    if (grads->h0 != nullptr) out[no++] = view(grads->h0, ends);
    if (workspace == nullptr || !is_aligned(workspace, 256)) return LINFUSION_ERR_INVALID_ARG;
    if (workspace_bytes < plan.bytes) return LINFUSION_ERR_ALLOC;
    out[no++] = view(workspace, plan.bytes);
    for (int o = 0; o < no; ++o) {
        for (int j = 0; j < o; ++j)
            if (!apart(d, out[o], out[j])) return LINFUSION_ERR_INVALID_ARG;
        for (int i = 0; i < ni; ++i)
            if (!over(d, out[o], in[i]) && !apart(d, out[o], in[i])) return LINFUSION_ERR_INVALID_ARG;
    }
    const Here at = here();
    if (at.st != LINFUSION_OK) return at.st;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(workspace);
    cudaError_t e = cudaSuccess;
    RecParams p = base(d, plan, x, decay, gate, rate, h0, workspace);
    p.dh = {static_cast<const char*>(dh->p), nullptr, dh->batch * 2, dh->row * 2};
    p.dlast = dlast;
    p.dx = to_output(grads->x);
    p.ddecay = to_output(grads->decay);
    if (gated) p.dgate = to_output(grads->gate);
    p.dh0 = grads->h0;
    p.rate_partials = grads->rate != nullptr ? reinterpret_cast<float*>(ws + plan.rate) : nullptr;
    p.states = state;
    if (plan.tiles > 1) {
        float* enters = reinterpret_cast<float*>(ws + plan.enters);
        p.grad_maps = reinterpret_cast<float2*>(ws + plan.grad_maps);
        if (state == nullptr) {
            float* kept_states = reinterpret_cast<float*>(ws + plan.kept);
            e = launch_enters<kRecMapBoth>(d, p, gated, packed, kept_states, enters, s);
            p.states = kept_states;
        } else {
            e = launch_enters<kRecMapGrad>(d, p, gated, packed, nullptr, enters, s);
        }
        if (e != cudaSuccess) return end(e);
        p.grads = enters;
    }
    const bool half = (d.flags & LINFUSION_DTYPE_FP16) != 0u;
    e = half ? launch_backward<kHf>(p, gated, packed, s) : launch_backward<kBf>(p, gated, packed, s);
    if (e == cudaSuccess && grads->rate != nullptr) {
        e = launch_pdl(column_sums_kernel, dim3(plan.width / kSumChannels), dim3(kSumThreads), 0, s, p.rate_partials, grads->rate,
                       static_cast<long long>(d.B) * plan.tiles, plan.width, d.C);
    }
    return end(e);
}

}  // extern "C"
