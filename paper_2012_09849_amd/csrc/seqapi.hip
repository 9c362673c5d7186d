// C ABI of the sequence memory: argument checks, the context, and sums of partial results (see include/hts.h).
#include <initializer_list>
#include <new>

#include "internal.hpp"
#include "seq.hpp"
#include "spans.hpp"

using namespace hts;

// a launch that no grid is large enough for is a shape's fault
#define LAUNCH_TRY(x) do { const hipError_t l_ = (x); if (l_ == hipErrorInvalidConfiguration) return HTS_ESHAPE; HIP_TRY(l_); } while (0)
#define HIP_TRY(x) do { const hipError_t e_ = (x); if (e_ != hipSuccess) { note_hip_error(e_); return HTS_EHIP; } } while (0)

namespace hts {
namespace {
__global__ __launch_bounds__(1024) void sum_partials_kernel(const float *part, const int64_t parts, const int64_t width, const SumTarget a, const SumTarget b, const SumTarget d)
{
    __shared__ float sums[16][64];
    sum_partials<16>(sums, blockIdx.x, part, parts, width, a, b, d);
}
}  // namespace

hipError_t launch_sum_partials(hts_seq_ctx &c, const float *part, int64_t parts, int64_t width, SumTarget a, SumTarget b, SumTarget d)
{
    hipLaunchKernelGGL(sum_partials_kernel, dim3((uint32_t)ceil_div(width, 64)), dim3(1024), 0, c.stream, part, parts, width, a, b, d);
    return hipGetLastError();
}
}  // namespace hts

static bool bad_precision(int32_t p) { return p != HTS_PRECISION_FP32 && p != HTS_PRECISION_BF16; }
constexpr int32_t MOST_STEPS = 1 << 30;       // the kernels count steps in 32 bits, and go beyond the last one by up to a few chunks
static int size_of(int32_t precision) { return precision == HTS_PRECISION_BF16 ? 2 : 4; }
static bool misaligned(const void *p, int size) { return (uintptr_t)p % size != 0; }

// Rows of an array: `output` rows must not overlap.  A single row's distance says nothing: it becomes one that suits every kernel.
static int32_t check_rows(hts_rows &r, int64_t rows, int64_t cols, int size, bool output)
{
    if (!r.p || misaligned(r.p, size) || r.ld < 0) return HTS_EINVAL;
    if (rows == 1) r.ld = round_up(cols, 16);
    if (r.ld > (1ll << 40)) return HTS_ESHAPE;
    return output && rows > 1 && r.ld < cols ? HTS_EINVAL : HTS_OK;
}
static int32_t check_steps(hts_steps &s, int64_t T, int64_t N, int64_t cols, int size, bool output)
{
    if (!s.p || misaligned(s.p, size) || s.st < 0 || s.sn < 0) return HTS_EINVAL;
    if (T == 1) s.st = 0;
    if (N == 1) s.sn = 0;
    // (a few steps' distance is counted in 32 bits)
    if (s.st > (1ll << 24) || s.sn > (1ll << 40)) return HTS_ESHAPE;
    if (!output) return HTS_OK;
    const bool by_step = (N == 1 || s.sn >= cols) && (T == 1 || s.st >= (N == 1 ? cols : s.sn * (N - 1) + cols));
    const bool by_sequence = (T == 1 || s.st >= cols) && (N == 1 || s.sn >= (T == 1 ? cols : s.st * (T - 1) + cols));
    return by_step || by_sequence ? HTS_OK : HTS_EINVAL;
}
#define CHECK(x) do { const int32_t rc_ = (x); if (rc_ != HTS_OK) return rc_; } while (0)
// What a call writes shares nothing with the other arrays, but for `place`, whose rows it may take (p 0: none)
static int32_t check_apart(const Span &out, std::initializer_list<Span> others, const Span &place)
{
    for (const Span &o : others) if (meet(out, o)) return HTS_EINVAL;
    return meet(out, place) && !same(out, place) ? HTS_EINVAL : HTS_OK;
}
static int32_t check_workspace(const hts_seq_ctx *ctx, int64_t need) { return need > ctx->bytes ? HTS_ESHAPE : HTS_OK; }

extern "C" int32_t hts_seq_create(int64_t workspace_bytes, void *hip_stream, hts_seq_ctx **out)
{
    if (!out || workspace_bytes < 0) return HTS_EINVAL;
    hts_seq_ctx *c = new (std::nothrow) hts_seq_ctx();
    if (!c) return HTS_ENOMEM;
    c->stream = (hipStream_t)hip_stream; c->cus = stream_cus(c->stream);
    c->ws = nullptr; c->bytes = workspace_bytes;
    if (workspace_bytes > 0) {
        const hipError_t e = hipMalloc((void **)&c->ws, (size_t)workspace_bytes);
        if (e != hipSuccess) { delete c; note_hip_error(e); return HTS_ENOMEM; }
    }
    *out = c;
    return HTS_OK;
}

extern "C" int32_t hts_seq_destroy(hts_seq_ctx *ctx)
{
    if (!ctx) return HTS_EINVAL;
    const hipError_t e = ctx->ws ? hipFree(ctx->ws) : hipSuccess;
    delete ctx;
    HIP_TRY(e);
    return HTS_OK;
}

// ---- matrix product -----------------------------------------------------------------------------------------------
static int32_t check_linear(const hts_linear_desc *d)
{
    if (!d) return HTS_EINVAL;
    if (d->M <= 0 || d->N <= 0 || d->K <= 0 || d->act < HTS_ACT_NONE || d->act > HTS_ACT_GELU) return HTS_EINVAL;
    if (bad_precision(d->precision) || d->M > (1 << 24) || d->N > (1 << 24) || d->K > (1 << 24)) return HTS_ESHAPE;
    return HTS_OK;
}

extern "C" int64_t hts_linear_workspace(const hts_linear_desc *d)
{
    CHECK(check_linear(d));
    return linear_workspace(d->precision, d->act, d->M, d->N, d->K);
}

extern "C" int32_t hts_linear(hts_seq_ctx *ctx, const hts_linear_desc *d, hts_rows x, hts_rows w, const float *bias, hts_rows residual,
                              hts_rows y, hts_rows pre)
{
    if (!ctx) return HTS_EINVAL;
    CHECK(check_linear(d));
    const int s = size_of(d->precision);
    CHECK(check_rows(x, d->M, d->K, s, false)); CHECK(check_rows(w, d->N, d->K, s, false)); CHECK(check_rows(y, d->M, d->N, s, true));
    if (residual.p) CHECK(check_rows(residual, d->M, d->N, s, false));
    if (pre.p) CHECK(check_rows(pre, d->M, d->N, s, true));
    if (misaligned(bias, 4)) return HTS_EINVAL;
    const Span xs = span(x.p, x.ld, d->M, d->K, s), ws = span(w.p, w.ld, d->N, d->K, s), bs = span(bias, 0, 1, d->N, 4), rs = span(residual.p, residual.ld, d->M, d->N, s);
    const Span ys = span(y.p, y.ld, d->M, d->N, s), ps = span(pre.p, pre.ld, d->M, d->N, s);
    CHECK(check_apart(ys, {xs, ws, bs, ps}, rs)); CHECK(check_apart(ps, {xs, ws, bs, rs}, Span{}));
    LinearOp op = {};
    op.M = d->M; op.N = d->N; op.K = d->K; op.act = d->act;
    op.x = x; op.w = w; op.bias = bias; op.residual = residual; op.y = y; op.pre = pre;
    LAUNCH_TRY(launch_linear(*ctx, d->precision, op));
    return HTS_OK;
}

extern "C" int32_t hts_linear_backward(hts_seq_ctx *ctx, const hts_linear_desc *d, hts_rows x, hts_rows w, hts_rows pre, hts_rows dy,
                                       hts_rows add, hts_rows dx, float *dw, float *db)
{
    if (!ctx) return HTS_EINVAL;
    CHECK(check_linear(d));
    if (!dx.p && !dw && !db) return HTS_EINVAL;
    const int s = size_of(d->precision);
    CHECK(check_rows(dy, d->M, d->N, s, false));
    if (dw) CHECK(check_rows(x, d->M, d->K, s, false));
    if (d->act != HTS_ACT_NONE) CHECK(check_rows(pre, d->M, d->N, s, false));
    if (dx.p) {
        CHECK(check_rows(dx, d->M, d->K, s, true)); CHECK(check_rows(w, d->N, d->K, s, false));
        if (add.p) CHECK(check_rows(add, d->M, d->K, s, false));
    }
    if (misaligned(dw, 4) || misaligned(db, 4)) return HTS_EINVAL;
    CHECK(check_workspace(ctx, linear_workspace(d->precision, d->act, d->M, d->N, d->K)));
    // what is read: x for dw, w and add for dx, pre for an activation
    const Span xs = span(dw ? x.p : nullptr, x.ld, d->M, d->K, s), ws = span(dx.p ? w.p : nullptr, w.ld, d->N, d->K, s), as = span(dx.p ? add.p : nullptr, add.ld, d->M, d->K, s);
    const Span ps = span(d->act != HTS_ACT_NONE ? pre.p : nullptr, pre.ld, d->M, d->N, s), gs = span(dy.p, dy.ld, d->M, d->N, s);
    const Span dxs = span(dx.p, dx.ld, d->M, d->K, s), dws = span(dw, 0, 1, (int64_t)d->N * d->K, 4), dbs = span(db, 0, 1, d->N, 4);
    CHECK(check_apart(dxs, {xs, ws, ps, gs, dws, dbs}, as)); CHECK(check_apart(dws, {xs, ws, as, ps, gs, dbs}, Span{})); CHECK(check_apart(dbs, {xs, ws, as, ps, gs}, Span{}));
    LinearOp op = {};
    op.M = d->M; op.N = d->N; op.K = d->K; op.act = d->act;
    op.x = x; op.w = w; op.pre = pre; op.dy = dy; op.add = add; op.dx = dx; op.dw = dw; op.db = db;
    LAUNCH_TRY(launch_linear_backward(*ctx, d->precision, op));
    return HTS_OK;
}

// ---- short convolution --------------------------------------------------------------------------------------------
static int32_t check_conv(const hts_short_conv_desc *d)
{
    if (!d) return HTS_EINVAL;
    if (d->T <= 0 || d->N <= 0 || d->D <= 0 || (d->act != HTS_ACT_NONE && d->act != HTS_ACT_SILU)) return HTS_EINVAL;
    if (bad_precision(d->precision) || d->T > MOST_STEPS || d->W < 2 || d->W > 4 || d->D > (1 << 20) || d->N > (1 << 24)) return HTS_ESHAPE;
    // (tasks of 8 steps of a sequence, 64 channels each or more, are counted in 32 bits)
    return ceil_div(d->T, 8) * d->N * ceil_div(d->D, 64) > (1ll << 31) ? HTS_ESHAPE : HTS_OK;
}

extern "C" int64_t hts_short_conv_workspace(const hts_short_conv_desc *d)
{
    CHECK(check_conv(d));
    return conv_workspace(d->T, d->N, d->D, d->W);
}

static int32_t check_conv_arrays(const hts_short_conv_desc *d, hts_steps &x, const float *w, const float *bias, const int32_t *lengths, const float *state_in)
{
    CHECK(check_steps(x, d->T, d->N, d->D, size_of(d->precision), false));
    return !w || misaligned(w, 4) || misaligned(bias, 4) || misaligned(lengths, 4) || misaligned(state_in, 4) ? HTS_EINVAL : HTS_OK;
}

extern "C" int32_t hts_short_conv(hts_seq_ctx *ctx, const hts_short_conv_desc *d, hts_steps x, const float *w, const float *bias,
                                  const uint8_t *starts, const int32_t *lengths, const float *state_in, hts_steps y, float *state_out)
{
    if (!ctx) return HTS_EINVAL;
    CHECK(check_conv(d));
    CHECK(check_conv_arrays(d, x, w, bias, lengths, state_in));
    CHECK(check_steps(y, d->T, d->N, d->D, size_of(d->precision), true));
    if (misaligned(state_out, 4)) return HTS_EINVAL;
    ConvOp op = {};
    op.T = d->T; op.N = d->N; op.D = d->D; op.W = d->W; op.act = d->act;
    op.x = x; op.y = y; op.w = w; op.bias = bias; op.starts = starts; op.lengths = lengths; op.state_in = state_in; op.state_out = state_out;
    LAUNCH_TRY(launch_conv(*ctx, d->precision, op));
    return HTS_OK;
}

extern "C" int32_t hts_short_conv_backward(hts_seq_ctx *ctx, const hts_short_conv_desc *d, hts_steps x, const float *w, const float *bias,
                                           const uint8_t *starts, const int32_t *lengths, const float *state_in, hts_steps dy,
                                           const float *dstate_out, hts_steps dx, float *dw, float *db, float *dstate_in)
{
    if (!ctx) return HTS_EINVAL;
    CHECK(check_conv(d));
    CHECK(check_conv_arrays(d, x, w, bias, lengths, state_in));
    const int s = size_of(d->precision);
    CHECK(check_steps(dy, d->T, d->N, d->D, s, false)); CHECK(check_steps(dx, d->T, d->N, d->D, s, true));
    if (!dw || misaligned(dw, 4) || misaligned(db, 4) || misaligned(dstate_out, 4) || misaligned(dstate_in, 4)) return HTS_EINVAL;
    if (dstate_in && dstate_in == dstate_out) return HTS_EINVAL;
    CHECK(check_workspace(ctx, conv_workspace(d->T, d->N, d->D, d->W)));
    ConvOp op = {};
    op.T = d->T; op.N = d->N; op.D = d->D; op.W = d->W; op.act = d->act;
    op.x = x; op.dy = dy; op.dx = dx; op.w = w; op.bias = bias; op.starts = starts; op.lengths = lengths; op.state_in = state_in;
    op.dstate_out = dstate_out; op.dw = dw; op.db = db; op.dstate_in = dstate_in;
    LAUNCH_TRY(launch_conv_backward(*ctx, d->precision, op));
    return HTS_OK;
}

// ---- selective scan -----------------------------------------------------------------------------------------------
static int32_t check_scan(const hts_scan_desc *d)
{
    if (!d) return HTS_EINVAL;
    if (d->T <= 0 || d->N <= 0 || d->D <= 0 || d->S <= 0 || d->G <= 0 || (d->softplus != 0 && d->softplus != 1)) return HTS_EINVAL;
    if (bad_precision(d->precision) || d->T > MOST_STEPS || d->S > 64 || d->D % d->G != 0 || d->D > (1 << 20) || d->N > (1 << 24)) return HTS_ESHAPE;
    // (a wavefront for 16 channels of a group and 16 steps at least; they are counted in 32 bits)
    return ceil_div(d->T, 16) * d->N * (ceil_div(d->D / d->G, 16) * d->G) > (1ll << 30) ? HTS_ESHAPE : HTS_OK;
}

extern "C" int64_t hts_selective_scan_workspace(const hts_scan_desc *d)
{
    CHECK(check_scan(d));
    const int64_t forward = scan_workspace(*d, false), backward = scan_workspace(*d, true);
    return forward > backward ? forward : backward;
}
extern "C" int64_t hts_selective_scan_states(const hts_scan_desc *d)
{
    CHECK(check_scan(d));
    return scan_states(*d);
}

static int32_t check_scan_arrays(const hts_scan_desc *d, const hts_scan_inputs *given, hts_scan_inputs *in)
{
    if (!given) return HTS_EINVAL;
    *in = *given;
    const int s = size_of(d->precision);
    const int64_t pair = (int64_t)d->G * d->S;
    CHECK(check_steps(in->x, d->T, d->N, d->D, s, false)); CHECK(check_steps(in->dt, d->T, d->N, d->D, s, false));
    CHECK(check_steps(in->B, d->T, d->N, pair, s, false)); CHECK(check_steps(in->C, d->T, d->N, pair, s, false));
    if (in->z.p) CHECK(check_steps(in->z, d->T, d->N, d->D, s, false));
    return !in->A || misaligned(in->A, 4) || misaligned(in->skip, 4) || misaligned(in->dt_bias, 4) || misaligned(in->lengths, 4) || misaligned(in->h_in, 4) ? HTS_EINVAL : HTS_OK;
}

extern "C" int32_t hts_selective_scan(hts_seq_ctx *ctx, const hts_scan_desc *d, const hts_scan_inputs *in, hts_steps y, float *h_out, float *states)
{
    if (!ctx) return HTS_EINVAL;
    CHECK(check_scan(d));
    ScanOp op = {};
    op.d = *d;
    CHECK(check_scan_arrays(d, in, &op.in));
    CHECK(check_steps(y, d->T, d->N, d->D, size_of(d->precision), true));
    if (misaligned(h_out, 4) || misaligned(states, 16)) return HTS_EINVAL;
    CHECK(check_workspace(ctx, scan_workspace(*d, false)));
    op.y = y; op.h_out = h_out; op.states_out = states;
    LAUNCH_TRY(launch_scan(*ctx, op));
    return HTS_OK;
}

extern "C" int32_t hts_selective_scan_backward(hts_seq_ctx *ctx, const hts_scan_desc *d, const hts_scan_inputs *in, hts_steps dy,
                                               const float *dh_out, const float *states, const hts_scan_grads *grads)
{
    if (!ctx || !grads || !states) return HTS_EINVAL;
    CHECK(check_scan(d));
    ScanOp op = {};
    op.d = *d;
    CHECK(check_scan_arrays(d, in, &op.in));
    hts_scan_grads *g = &op.g;
    *g = *grads;
    const int s = size_of(d->precision);
    const int64_t pair = (int64_t)d->G * d->S;
    CHECK(check_steps(dy, d->T, d->N, d->D, s, false));
    CHECK(check_steps(g->dx, d->T, d->N, d->D, s, true)); CHECK(check_steps(g->ddt, d->T, d->N, d->D, s, true));
    CHECK(check_steps(g->dB, d->T, d->N, pair, s, true)); CHECK(check_steps(g->dC, d->T, d->N, pair, s, true));
    if ((g->dz.p != nullptr) != (op.in.z.p != nullptr)) return HTS_EINVAL;
    if (g->dz.p) CHECK(check_steps(g->dz, d->T, d->N, d->D, s, true));
    if (!g->dA || misaligned(g->dA, 4) || misaligned(g->dskip, 4) || misaligned(g->ddt_bias, 4) || misaligned(g->dh_in, 4)) return HTS_EINVAL;
    if (misaligned(states, 16) || misaligned(dh_out, 4) || (dh_out && g->dh_in == dh_out)) return HTS_EINVAL;
    CHECK(check_workspace(ctx, scan_workspace(*d, true)));
    op.dy = dy; op.dh_out = dh_out; op.states = states;
    LAUNCH_TRY(launch_scan_backward(*ctx, op));
    return HTS_OK;
}

// ---- layer norm ---------------------------------------------------------------------------------------------------
static int32_t check_norm(const hts_layer_norm_desc *d)
{
    if (!d) return HTS_EINVAL;
    if (d->M <= 0 || d->F <= 0 || !(d->eps >= 0.0f && d->eps <= 3.402823466e38f)) return HTS_EINVAL;
    return bad_precision(d->precision) || d->M > (1 << 24) || d->F > 16384 ? HTS_ESHAPE : HTS_OK;
}

extern "C" int64_t hts_layer_norm_workspace(const hts_layer_norm_desc *d)
{
    CHECK(check_norm(d));
    return norm_workspace(d->M, d->F);
}

extern "C" int32_t hts_layer_norm(hts_seq_ctx *ctx, const hts_layer_norm_desc *d, hts_rows x, const float *w, const float *b, hts_rows y)
{
    if (!ctx) return HTS_EINVAL;
    CHECK(check_norm(d));
    const int s = size_of(d->precision);
    CHECK(check_rows(x, d->M, d->F, s, false)); CHECK(check_rows(y, d->M, d->F, s, true));
    if (misaligned(w, 4) || misaligned(b, 4)) return HTS_EINVAL;
    CHECK(check_apart(span(y.p, y.ld, d->M, d->F, s), {span(w, 0, 1, d->F, 4), span(b, 0, 1, d->F, 4)}, span(x.p, x.ld, d->M, d->F, s)));
    NormOp op = {};
    op.M = d->M; op.F = d->F; op.eps = d->eps; op.x = x; op.y = y; op.w = w; op.b = b;
    LAUNCH_TRY(launch_norm(*ctx, d->precision, op));
    return HTS_OK;
}

extern "C" int32_t hts_layer_norm_backward(hts_seq_ctx *ctx, const hts_layer_norm_desc *d, hts_rows x, const float *w, hts_rows dy, hts_rows add,
                                           hts_rows dx, float *dw, float *db)
{
    if (!ctx) return HTS_EINVAL;
    CHECK(check_norm(d));
    if (!dx.p && !dw && !db) return HTS_EINVAL;
    const int s = size_of(d->precision);
    CHECK(check_rows(x, d->M, d->F, s, false)); CHECK(check_rows(dy, d->M, d->F, s, false));
    if (dx.p) {
        CHECK(check_rows(dx, d->M, d->F, s, true));
        if (add.p) CHECK(check_rows(add, d->M, d->F, s, false));
    } else add.p = nullptr;
    if (misaligned(w, 4) || misaligned(dw, 4) || misaligned(db, 4)) return HTS_EINVAL;
    const Span xs = span(x.p, x.ld, d->M, d->F, s), gs = span(dy.p, dy.ld, d->M, d->F, s), as = span(add.p, add.ld, d->M, d->F, s), ws = span(w, 0, 1, d->F, 4);
    const Span dxs = span(dx.p, dx.ld, d->M, d->F, s), dws = span(dw, 0, 1, d->F, 4), dbs = span(db, 0, 1, d->F, 4);
    // a row's gradient takes its place in any of what it comes from, which may be one another
    for (const Span &place : {xs, gs, as}) if (meet(dxs, place) && !same(dxs, place)) return HTS_EINVAL;
    CHECK(check_apart(dxs, {ws, dws, dbs}, Span{})); CHECK(check_apart(dws, {xs, gs, as, ws, dbs}, Span{})); CHECK(check_apart(dbs, {xs, gs, as, ws}, Span{}));
    if (dw || db) CHECK(check_workspace(ctx, norm_workspace(d->M, d->F)));
    NormOp op = {};
    op.M = d->M; op.F = d->F; op.eps = d->eps; op.x = x; op.w = w; op.dy = dy; op.add = add; op.dx = dx; op.dw = dw; op.db = db;
    LAUNCH_TRY(launch_norm_backward(*ctx, d->precision, op));
    return HTS_OK;
}

// ---- gated delta rule ---------------------------------------------------------------------------------------------
static int32_t check_delta(const hts_delta_rule_desc *d)
{
    if (!d) return HTS_EINVAL;
    if (d->T <= 0 || d->N <= 0 || d->H <= 0 || d->G <= 0 || d->K <= 0 || d->V <= 0 || (d->normalize != 0 && d->normalize != 1) || (d->softplus != 0 && d->softplus != 1) ||
        !(d->scale >= -3.402823466e38f && d->scale <= 3.402823466e38f)) return HTS_EINVAL;
    if (bad_precision(d->precision) || d->T > MOST_STEPS || d->N > (1 << 24) || d->H > (1 << 16) || d->H % d->G != 0 || d->K > 128 || d->V > (1 << 16)) return HTS_ESHAPE;
    // (workgroups for a chunk of 64 steps of a head, and for 32 values of a head, are counted in 31 bits)
    const int64_t heads = (int64_t)d->N * d->H, most = (1ll << 31) - 1;
    return heads > most || ceil_div(d->T, 64) > most / heads || ceil_div(d->V, 32) > most / heads ? HTS_ESHAPE : HTS_OK;
}

extern "C" int64_t hts_delta_rule_workspace(const hts_delta_rule_desc *d)
{
    CHECK(check_delta(d));
    const int64_t forward = delta_workspace(*d, false), backward = delta_workspace(*d, true);
    return forward > backward ? forward : backward;
}
extern "C" int64_t hts_delta_rule_states(const hts_delta_rule_desc *d)
{
    CHECK(check_delta(d));
    return delta_states(*d);
}

static int32_t check_delta_arrays(const hts_delta_rule_desc *d, const hts_delta_rule_inputs *given, hts_delta_rule_inputs *in)
{
    if (!given) return HTS_EINVAL;
    *in = *given;
    const int s = size_of(d->precision);
    const int64_t keys = (int64_t)d->G * d->K, values = (int64_t)d->H * d->V;
    CHECK(check_steps(in->q, d->T, d->N, keys, s, false)); CHECK(check_steps(in->k, d->T, d->N, keys, s, false)); CHECK(check_steps(in->v, d->T, d->N, values, s, false));
    CHECK(check_steps(in->a, d->T, d->N, d->H, s, false)); CHECK(check_steps(in->b, d->T, d->N, d->H, s, false));
    return !in->A || misaligned(in->A, 4) || misaligned(in->a_bias, 4) || misaligned(in->lengths, 4) || misaligned(in->h_in, 4) ? HTS_EINVAL : HTS_OK;
}
// Where a call's arrays lie: what it reads, then what it writes, which shares memory with nothing else
struct DeltaAreas {
    const hts_delta_rule_desc &d;
    Area of[24];
    int read = 0, count = 0;
    void steps(const hts_steps &s, int64_t cols) { of[count++] = area(s.p, s.st, s.sn, d.T, d.N, cols, size_of(d.precision)); }
    void dense(const void *p, int64_t n, int size) { of[count++] = area(p, n, size); }
    int64_t keys() const { return (int64_t)d.G * d.K; }
    int64_t values() const { return (int64_t)d.H * d.V; }
    int64_t held() const { return (int64_t)d.N * d.H * d.K * d.V; }
    // h_in: not where an output takes its place
    void inputs(const hts_delta_rule_inputs &in, bool h_in)
    {
        steps(in.q, keys()); steps(in.k, keys()); steps(in.v, values()); steps(in.a, d.H); steps(in.b, d.H);
        dense(in.A, d.H, 4); dense(in.a_bias, d.H, 4); dense(in.starts, (int64_t)d.T * d.N, 1); dense(in.lengths, d.N, 4);
        if (h_in) dense(in.h_in, held(), 4);
    }
    bool apart() const
    {
        for (int i = read; i < count; ++i) for (int k = 0; k < i; ++k) if (meet(of[i], of[k])) return false;
        return true;
    }
};

extern "C" int32_t hts_delta_rule(hts_seq_ctx *ctx, const hts_delta_rule_desc *d, const hts_delta_rule_inputs *in, hts_steps y, float *h_out, float *states)
{
    if (!ctx) return HTS_EINVAL;
    CHECK(check_delta(d));
    DeltaOp op = {};
    op.d = *d;
    CHECK(check_delta_arrays(d, in, &op.in));
    CHECK(check_steps(y, d->T, d->N, (int64_t)d->H * d->V, size_of(d->precision), true));
    if (misaligned(h_out, 4) || misaligned(states, 16)) return HTS_EINVAL;
    DeltaAreas all{*d};
    all.inputs(op.in, h_out != op.in.h_in);
    all.read = all.count;
    all.steps(y, all.values()); all.dense(h_out, all.held(), 4); all.dense(states, delta_states(*d), 4);
    if (!all.apart()) return HTS_EINVAL;
    CHECK(check_workspace(ctx, delta_workspace(*d, false)));
    op.y = y; op.h_out = h_out; op.states = states;
    LAUNCH_TRY(launch_delta(*ctx, op));
    return HTS_OK;
}

extern "C" int32_t hts_delta_rule_backward(hts_seq_ctx *ctx, const hts_delta_rule_desc *d, const hts_delta_rule_inputs *in, hts_steps dy,
                                           const float *dh_out, const float *states, const hts_delta_rule_grads *grads)
{
    if (!ctx || !grads || !states) return HTS_EINVAL;
    CHECK(check_delta(d));
    DeltaOp op = {};
    op.d = *d;
    CHECK(check_delta_arrays(d, in, &op.in));
    hts_delta_rule_grads *g = &op.g;
    *g = *grads;
    const int s = size_of(d->precision);
    const int64_t keys = (int64_t)d->G * d->K, values = (int64_t)d->H * d->V;
    CHECK(check_steps(dy, d->T, d->N, values, s, false));
    CHECK(check_steps(g->dq, d->T, d->N, keys, s, true)); CHECK(check_steps(g->dk, d->T, d->N, keys, s, true)); CHECK(check_steps(g->dv, d->T, d->N, values, s, true));
    CHECK(check_steps(g->da, d->T, d->N, d->H, s, true)); CHECK(check_steps(g->db, d->T, d->N, d->H, s, true));
    if (!g->dA || misaligned(g->dA, 4) || misaligned(g->da_bias, 4) || misaligned(g->dh_in, 4) || misaligned(states, 16) || misaligned(dh_out, 4)) return HTS_EINVAL;
    DeltaAreas all{*d};
    all.inputs(op.in, true);
    all.steps(dy, values); all.dense(dh_out, all.held(), 4); all.dense(states, delta_states(*d), 4);
    all.read = all.count;
    all.steps(g->dq, keys); all.steps(g->dk, keys); all.steps(g->dv, values); all.steps(g->da, d->H); all.steps(g->db, d->H);
    all.dense(g->dA, d->H, 4); all.dense(g->da_bias, d->H, 4); all.dense(g->dh_in, all.held(), 4);
    if (!all.apart()) return HTS_EINVAL;
    CHECK(check_workspace(ctx, delta_workspace(*d, true)));
    op.dy = dy; op.dh_out = dh_out; op.states = const_cast<float *>(states);
    LAUNCH_TRY(launch_delta_backward(*ctx, op));
    return HTS_OK;
}
