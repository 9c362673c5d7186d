// Short causal convolution along time, a filter of W taps for each channel, and its gradients (see include/hts.h).
//
// Bound by memory: x is read and y written once (backward: x and dy read, dx written), W products an entry.  A lane owns 16 bytes (backward 8) of
// neighbouring channels, or one channel where strides or addresses forbid it, for TC steps; the W - 1 inputs before them are read again,
// from the L2.  What an episode's first step cuts off is a number per step, `vis`: how many earlier inputs the step sees.
#include "seq.hpp"

namespace hts {
namespace {

constexpr int TC = 16;               // steps of a task
constexpr int ROWS = 4;              // wavefronts of a workgroup, each with tasks of its own

// steps visible before step t (at most W - 1): those of its episode and, where no episode begins in between, the state's
template <int W> __device__ __forceinline__ int visible(const uint8_t *starts, int t, int n, int N)
{
    int vis = W - 1;
    if (starts)
#pragma unroll
        for (int i = W - 2; i >= 0; --i)
            if (t - i >= 0 && starts[(int64_t)(t - i) * N + n]) vis = i;
    return vis;
}
__device__ __forceinline__ int length_of(const int32_t *lengths, int n, int T) { return lengths ? max(0, min(T, lengths[n])) : T; }

template <typename T, int V> struct Row {
    float e[V];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = 0.0f;
    }
    __device__ __forceinline__ void load(const T *p) { take(load_v<T, V>(p)); }
    __device__ __forceinline__ void take(const Loaded<T, V> &r)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = to_f32(r.e[i]);
    }
    __device__ __forceinline__ void load32(const float *p)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = p[i];
    }
    __device__ __forceinline__ void store(T *p) const
    {
        Loaded<T, V> r;
#pragma unroll
        for (int i = 0; i < V; ++i) r.e[i] = from_f32<T>(e[i]);
        store_v<T, V>(p, r);
    }
};

template <typename T, int V, int W, int ACT>
__global__ __launch_bounds__(64 * ROWS) void conv_kernel(const ConvOp p, const int dv_blocks, const int chunks)
{
    const int lane = threadIdx.x & 63, row = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t at = blockIdx.x / dv_blocks * (int64_t)ROWS + row;
    const int d = ((int)(blockIdx.x % dv_blocks) * 64 + lane) * V;
    if (at >= (int64_t)p.N * chunks) return;
    const int n = (int)(at / chunks), chunk = (int)(at % chunks), t0 = chunk * TC, len = length_of(p.lengths, n, p.T);
    if (d >= p.D) return;
    const T *x = (const T *)p.x.p + n * p.x.sn + d;
    T *y = (T *)p.y.p + n * p.y.sn + d;
    float w[W][V], bias[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        bias[i] = p.bias ? p.bias[d + i] : 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) w[j][i] = p.w[(int64_t)(d + i) * W + j];
    }
    Row<T, V> win[W];                            // win[j]: input t - W + 1 + j
    Loaded<T, V> in[TC];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int i = t0 - (W - 1) + j;
        if (i >= 0 && i < len) win[j].load(x + i * p.x.st);
        else if (i < 0 && p.state_in) win[j].load32(p.state_in + ((int64_t)n * (W - 1) + i + W - 1) * p.D + d);
        else win[j].zero();
    }
#pragma unroll
    for (int k = 0; k < TC; ++k)
        if (t0 + k < len) in[k] = load_v<T, V>(x + (t0 + k) * p.x.st);
    if (p.state_out && chunk == 0) {
        // by the lane that holds state_in already, which may be the same array
        const int vis = visible<W>(p.starts, len - 1, n, p.N);
        Row<T, V> out[W - 1];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int i = len - (W - 1) + j;
            out[j].zero();
            if (len - 1 - i <= vis) {
                if (i >= 0) out[j].load(x + i * p.x.st);
                else
#pragma unroll
                    for (int k = 0; k < W - 1; ++k) if (k == i + W - 1) out[j] = win[k];
            }
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) p.state_out[((int64_t)n * (W - 1) + j) * p.D + d + i] = out[j].e[i];
    }
    int vis = visible<W>(p.starts, t0 - 1, n, p.N);
#pragma unroll
    for (int k = 0; k < TC; ++k) {
        const int t = t0 + k;
        if (t >= p.T) break;
        Row<T, V> out;
        out.zero();
        if (t < len) {
            vis = p.starts && p.starts[(int64_t)t * p.N + n] ? 0 : min(vis + 1, W - 1);
            win[W - 1].take(in[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) out.e[i] = bias[i];
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (W - 1 - j <= vis)
#pragma unroll
                    for (int i = 0; i < V; ++i) out.e[i] = __builtin_fmaf(w[j][i], win[j].e[i], out.e[i]);
#pragma unroll
            for (int i = 0; i < V; ++i) out.e[i] = act_f<ACT>(out.e[i]);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
        }
        out.store(y + t * p.y.st);
    }
}

// A wavefront's tasks are (sequence, TC steps).  Step t's pre-activation is formed again from x; g_t = dy_t act'(v_t) reaches the inputs
// t - q, q <= vis(t), whose sums wait in `pend`.  An input's last share comes W - 1 steps later, so a task goes on that far (those
// steps' g belongs to the next task's filter gradient).  Filter gradients of a workgroup's tasks are added in registers, then over its
// wavefronts in a fixed order, and leave as one partial sum a workgroup.
template <typename T, int V, int W, int ACT>
__global__ __launch_bounds__(64 * ROWS) void conv_backward_kernel(const ConvOp p, const int dv_blocks, const int chunks, const int groups, float *part)
{
    const int lane = threadIdx.x & 63, row = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = blockIdx.x / dv_blocks;
    const int d = ((int)(blockIdx.x % dv_blocks) * 64 + lane) * V;
    const bool on = d < p.D;
    float w[W][V], bias[V], dw[W][V], db[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        bias[i] = on && p.bias ? p.bias[d + i] : 0.0f;
        db[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) { w[j][i] = on ? p.w[(int64_t)(d + i) * W + j] : 0.0f; dw[j][i] = 0.0f; }
    }
    const int64_t tasks = (int64_t)p.N * chunks;
    if (on)
    for (int64_t at = group * (int64_t)ROWS + row; at < tasks; at += (int64_t)groups * ROWS) {
        const int n = (int)(at / chunks), t0 = (int)(at % chunks) * TC, len = length_of(p.lengths, n, p.T), t1 = min(t0 + TC, p.T);
        const T *x = (const T *)p.x.p + n * p.x.sn + d, *dy = (const T *)p.dy.p + n * p.dy.sn + d;
        T *dx = (T *)p.dx.p + n * p.dx.sn + d;
        const float *dso = p.dstate_out ? p.dstate_out + (int64_t)n * (W - 1) * p.D + d : nullptr;
        const int vis_end = visible<W>(p.starts, len - 1, n, p.N);
        Row<T, V> win[W], pend[W];
        Loaded<T, V> xi[TC + W - 1], gi[TC + W - 1];
#pragma unroll
        for (int j = 0; j < W; ++j) pend[j].zero();
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int i = t0 - (W - 1) + j;
            if (i >= 0 && i < len) win[j].load(x + i * p.x.st);
            else if (i < 0 && p.state_in) win[j].load32(p.state_in + ((int64_t)n * (W - 1) + i + W - 1) * p.D + d);
            else win[j].zero();
        }
#pragma unroll
        for (int k = 0; k < TC + W - 1; ++k)
            if (t0 + k < len) { xi[k] = load_v<T, V>(x + (t0 + k) * p.x.st); gi[k] = load_v<T, V>(dy + (t0 + k) * p.dy.st); }
        int vis = visible<W>(p.starts, t0 - 1, n, p.N);
#pragma unroll
        for (int k = 0; k < TC + W - 1; ++k) {
            const int t = t0 + k;
            if (t < len) {
                vis = p.starts && p.starts[(int64_t)t * p.N + n] ? 0 : min(vis + 1, W - 1);
                win[W - 1].take(xi[k]);
                float v[V], g[V];
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = bias[i];
#pragma unroll
                for (int j = 0; j < W; ++j)
                    if (W - 1 - j <= vis)
#pragma unroll
                        for (int i = 0; i < V; ++i) v[i] = __builtin_fmaf(w[j][i], win[j].e[i], v[i]);
#pragma unroll
                for (int i = 0; i < V; ++i) g[i] = to_f32(gi[k].e[i]) * act_slope<ACT>(v[i]);
#pragma unroll
                for (int j = 0; j < W; ++j)
                    if (W - 1 - j <= vis)
#pragma unroll
                        for (int i = 0; i < V; ++i) pend[W - 1 - j].e[i] = __builtin_fmaf(w[j][i], g[i], pend[W - 1 - j].e[i]);
                if (k < TC) {
#pragma unroll
                    for (int i = 0; i < V; ++i) db[i] += g[i];
#pragma unroll
                    for (int j = 0; j < W; ++j)
                        if (W - 1 - j <= vis)
#pragma unroll
                            for (int i = 0; i < V; ++i) dw[j][i] = __builtin_fmaf(win[j].e[i], g[i], dw[j][i]);
                }
#pragma unroll
                for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
            }
            // input i has all its shares
            const int i = t - (W - 1);
            if (i < len && dso && i >= len - (W - 1) && len - 1 - i <= vis_end)
#pragma unroll
                for (int e = 0; e < V; ++e) pend[W - 1].e[e] += dso[(int64_t)(i - (len - (W - 1))) * p.D + e];
            if (i >= t0 && i < t1) pend[W - 1].store(dx + i * p.dx.st);
            else if (i < 0 && p.dstate_in)
#pragma unroll
                for (int e = 0; e < V; ++e) p.dstate_in[((int64_t)n * (W - 1) + i + W - 1) * p.D + d + e] = pend[W - 1].e[e];
#pragma unroll
            for (int j = W - 1; j > 0; --j) pend[j] = pend[j - 1];
            pend[0].zero();
        }
    }
    // [D][W] filters, then [D] biases, a partial sum a workgroup
    __shared__ float sums[ROWS][(W + 1) * V][64];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        sums[row][W * V + i][lane] = db[i];
#pragma unroll
        for (int j = 0; j < W; ++j) sums[row][j * V + i][lane] = dw[j][i];
    }
    __syncthreads();
    float *out = part + (int64_t)group * p.D * (W + 1);
    for (int k = row; k < (W + 1) * V; k += ROWS) {
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) s += sums[r][k][lane];
        const int j = k / V, c = d + k % V;
        if (on) out[j < W ? (int64_t)c * W + j : (int64_t)p.D * W + c] = s;
    }
}

template <typename T> bool wide(const hts_steps &s, int V) { return ((uintptr_t)s.p % (sizeof(T) * V)) == 0 && s.st % V == 0 && s.sn % V == 0; }

constexpr int MAX_GROUPS = 512;      // partial sums of the filter gradients
int groups_of(int64_t T, int64_t N) { const int64_t g = ceil_div(N * ceil_div(T, TC), ROWS); return (int)(g < MAX_GROUPS ? g : MAX_GROUPS); }

template <bool BACKWARD, typename T, int V, int W, int ACT> hipError_t run(hts_seq_ctx &c, const ConvOp &op)
{
    const int dv = (int)ceil_div(ceil_div(op.D, V), 64), chunks = (int)ceil_div(op.T, TC);
    if constexpr (!BACKWARD) {
        hipLaunchKernelGGL((conv_kernel<T, V, W, ACT>), dim3((uint32_t)(ceil_div((int64_t)op.N * chunks, ROWS) * dv)), dim3(64 * ROWS), 0, c.stream, op, dv, chunks);
        return hipGetLastError();
    } else {
        const int groups = groups_of(op.T, op.N);
        hipLaunchKernelGGL((conv_backward_kernel<T, V, W, ACT>), dim3((uint32_t)(groups * dv)), dim3(64 * ROWS), 0, c.stream, op, dv, chunks, groups, (float *)c.ws);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        return launch_sum_partials(c, (const float *)c.ws, groups, (int64_t)op.D * (W + 1), SumTarget{op.dw, (int64_t)op.D * W}, SumTarget{op.db, (int64_t)op.D}, SumTarget{nullptr, 0});
    }
}
template <bool BACKWARD, typename T, int V> hipError_t by_width(hts_seq_ctx &c, const ConvOp &op)
{
    const bool silu = op.act == HTS_ACT_SILU;
    switch (op.W) {
    case 2: return silu ? run<BACKWARD, T, V, 2, HTS_ACT_SILU>(c, op) : run<BACKWARD, T, V, 2, HTS_ACT_NONE>(c, op);
    case 3: return silu ? run<BACKWARD, T, V, 3, HTS_ACT_SILU>(c, op) : run<BACKWARD, T, V, 3, HTS_ACT_NONE>(c, op);
    default: return silu ? run<BACKWARD, T, V, 4, HTS_ACT_SILU>(c, op) : run<BACKWARD, T, V, 4, HTS_ACT_NONE>(c, op);
    }
}
template <typename T> hipError_t by_layout(hts_seq_ctx &c, const ConvOp &op, bool backward)
{
    // 16 bytes a lane; backward 8, since a lane keeps the inputs and output gradients of a whole task in registers
    constexpr int V = 16 / sizeof(T), VB = 8 / sizeof(T);
    if (backward) return op.D % VB == 0 && wide<T>(op.x, VB) && wide<T>(op.dy, VB) && wide<T>(op.dx, VB) ? by_width<true, T, VB>(c, op) : by_width<true, T, 1>(c, op);
    return op.D % V == 0 && wide<T>(op.x, V) && wide<T>(op.y, V) ? by_width<false, T, V>(c, op) : by_width<false, T, 1>(c, op);
}

}  // namespace

int64_t conv_workspace(int64_t T, int64_t N, int64_t D, int W) { return 4 * groups_of(T, N) * D * (W + 1); }
hipError_t launch_conv(hts_seq_ctx &c, int precision, const ConvOp &op) { return precision == HTS_PRECISION_BF16 ? by_layout<bf16_t>(c, op, false) : by_layout<float>(c, op, false); }
hipError_t launch_conv_backward(hts_seq_ctx &c, int precision, const ConvOp &op) { return precision == HTS_PRECISION_BF16 ? by_layout<bf16_t>(c, op, true) : by_layout<float>(c, op, true); }

}  // namespace hts
