// Short causal convolution along time, a filter of W taps for each channel, and its gradients (see include/hts.h).
//
// Bound by memory: x is read and y written once (backward: x and dy read, dx written), W products an entry.  A lane owns two
// neighbouring channels, or one where strides or addresses forbid it, for TC steps (512 x 16 x 1024 in bfloat16: forward 8.6 us, four channels a lane 9.8,
// eight 11.0 to 12.4: more wavefronts overlap reading, arithmetic and writing); all of a task's rows are requested before the first is used,
// the W - 1 inputs before them once more, from the L2.  Where an episode begins is a mask of steps, gathered by one load and a ballot (a load for each
// step, waited for, took 18 us at eight channels a lane, the mask 15).
#include "seq.hpp"

namespace hts {
namespace {

// steps of a task; a single step (an actor's) is a task of its own.  Backward a lane keeps a task's inputs and output gradients in registers
constexpr int FORWARD = 8, BACKWARD = 8;
constexpr int ROWS = 4;              // wavefronts of a workgroup, each with tasks of its own

__device__ __forceinline__ int length_of(const int32_t *lengths, int n, int T) { return lengths ? max(0, min(T, lengths[n])) : T; }
// bit k: step first + k begins an episode (steps that there are, below `len`)
__device__ __forceinline__ uint32_t begins(const uint8_t *starts, int first, int count, int len, int n, int N, int lane)
{
    const int t = first + lane;
    const bool there = starts && lane < count && t >= 0 && t < len;
    const uint32_t flag = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(reach((const char *)starts + n + (int64_t)first * N), there ? (int)(lane * (uint32_t)N) : (int)NOWHERE, 0, 0);
    return (uint32_t)__ballot(flag != 0);
}
// earlier inputs that the step of bit k sees, at most W - 1: those of its episode and, where none begins in between, the state's
template <int W> __device__ __forceinline__ int seen(uint32_t mask, int k)
{
    int vis = W - 1;
#pragma unroll
    for (int i = W - 2; i >= 0; --i)
        if (k - i >= 0 && (mask >> (k - i) & 1)) vis = i;
    return vis;
}

// A task's rows of an array, from step t0 - (W - 1) on: a lane's V channels in row k
template <typename T, int V> struct Track {
    __amdgpu_buffer_rsrc_t rows;
    uint32_t step, lane;
    __device__ __forceinline__ void open(const hts_steps &a, int n, int first, int d, int D)
    {
        rows = reach((const char *)a.p + (n * a.sn + first * a.st) * (int64_t)sizeof(T));
        step = (uint32_t)(a.st * (int64_t)sizeof(T));
        lane = d < D ? (uint32_t)d * (uint32_t)sizeof(T) : NOWHERE;
    }
    __device__ __forceinline__ void load(Raw<T, V, (V > 1)> &v, int k, bool there) const { v.load(rows, there ? lane : NOWHERE, 1, (uint32_t)k * step); }
    __device__ __forceinline__ void store(const float (&v)[V], int k, bool there) const { put_raw<T, V, (V > 1)>(rows, there ? lane : NOWHERE, 1, v, (uint32_t)k * step); }
};
// N neighbouring floats of a lane, at any address
template <int N> __device__ __forceinline__ void read32(float (&v)[N], __amdgpu_buffer_rsrc_t src, uint32_t lane)
{
    constexpr int FOURS = N / 4 * 4, TWOS = N / 2 * 2;
#pragma unroll
    for (int i = 0; i < FOURS; i += 4) {
        Raw<float, 4, true> r;
        r.load(src, lane, 1, 4 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i + e] = r[e];
    }
    if constexpr (TWOS > FOURS) {
        Raw<float, 2, true> r;
        r.load(src, lane, 1, 4 * FOURS);
        v[FOURS] = r[0]; v[FOURS + 1] = r[1];
    }
    if constexpr (N > TWOS) {
        Raw<float, 1, true> r;
        r.load(src, lane, 1, 4 * TWOS);
        v[TWOS] = r[0];
    }
}
// row j of sequence n's state: a lane's V channels
template <int V> __device__ __forceinline__ void read_state(float (&v)[V], const float *p, int64_t row, int d, int D)
{
    read32(v, reach((const char *)(p + row * D)), d < D ? (uint32_t)d * 4u : NOWHERE);
}
template <int V> __device__ __forceinline__ void clear(float (&v)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.0f;
}
template <typename T, int V, bool WIDE> __device__ __forceinline__ void take(float (&v)[V], const Raw<T, V, WIDE> &r)
{
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = r[i];
}
template <int V> __device__ __forceinline__ void copy(float (&v)[V], const float (&w)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = w[i];
}
template <int W, int V> struct Filter {
    float w[W][V], bias[V];
    __device__ __forceinline__ void load(const ConvOp &p, int d)
    {
        float all[V * W];
        read32(all, reach((const char *)p.w), d < p.D ? (uint32_t)(d * W) * 4u : NOWHERE);
        read32(bias, reach((const char *)p.bias), p.bias && d < p.D ? (uint32_t)d * 4u : NOWHERE);
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][i] = all[i * W + j];
    }
    // the pre-activation of the step whose inputs are in `win`, of which it sees the last 1 + vis (-1: none).  CUT: perhaps not all
    template <bool CUT> __device__ __forceinline__ void apply(float (&v)[V], const float (&win)[W][V], int vis) const
    {
        copy(v, bias);
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float more = __builtin_fmaf(w[j][i], win[j][i], v[i]);
                v[i] = !CUT || W - 1 - j <= vis ? more : v[i];
            }
    }
};

template <typename T, int V, int W, int ACT, int TC>
__global__ __launch_bounds__(64 * ROWS) void conv_kernel(const ConvOp p, const int dv_blocks, const int chunks)
{
    const int lane = threadIdx.x & 63, row = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t at = blockIdx.x / dv_blocks * ROWS + row;                 // (the number of tasks has 31 bits)
    const int d = ((int)(blockIdx.x % dv_blocks) * 64 + lane) * V;
    if (at >= (uint32_t)p.N * chunks) return;
    const int n = at / chunks, t0 = at % chunks * TC, len = length_of(p.lengths, n, p.T), first = t0 - (W - 1);
    const bool on = d < p.D;
    Track<T, V> xa, ya;
    xa.open(p.x, n, first, d, p.D);
    ya.open(p.y, n, t0, d, p.D);
    Raw<T, V, (V > 1)> in[TC + W - 1];
#pragma unroll
    for (int k = 0; k < TC + W - 1; ++k) xa.load(in[k], k, first + k >= 0 && first + k < len);
    const uint32_t mask = begins(p.starts, first, TC + W - 1, len, n, p.N, lane);
    Filter<W, V> f;
    f.load(p, d);
    float win[W][V];                             // win[j]: input t - W + 1 + j
#pragma unroll
    for (int j = 0; j < W - 1; ++j) take(win[j], in[j]);
    // (the mask of the sequence's end by all lanes)
    const int vis_end = t0 == 0 && p.state_out ? seen<W>(begins(p.starts, len - (W - 1), W - 1, len, n, p.N, lane), W - 2) : 0;
    if (t0 == 0 && on) {
        if (p.state_in)
#pragma unroll
            for (int j = 0; j < W - 1; ++j) read_state(win[j], p.state_in, (int64_t)n * (W - 1) + j, d, p.D);
        if (p.state_out) {
            // by the lane that holds state_in already, which may be the same array
            Track<T, V> tail;
            tail.open(p.x, n, len - (W - 1), d, p.D);
            float out[W - 1][V];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                const int i = len - (W - 1) + j;
                Raw<T, V, (V > 1)> r;
                tail.load(r, j, i >= 0);
                take(out[j], r);
#pragma unroll
                for (int k = 0; k < W - 1; ++k) if (k == i + W - 1) copy(out[j], win[k]);
                if (W - 2 - j > vis_end) clear(out[j]);
            }
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) p.state_out[((int64_t)n * (W - 1) + j) * p.D + d + i] = out[j][i];
        }
    }
    auto pass = [&](auto cut) {
        constexpr bool CUT = decltype(cut)::value;
#pragma unroll
        for (int k = 0; k < TC; ++k) {
            const int t = t0 + k;
            __builtin_amdgcn_sched_barrier(0);           // a step after the other: mixed, they need more registers than there are
            take(win[W - 1], in[k + W - 1]);
            float v[V];
            f.template apply<CUT>(v, win, CUT ? seen<W>(mask, k + W - 1) : 0);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = t < len ? act_f<ACT>(v[i]) : 0.0f;
            ya.store(v, k, t < p.T);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) copy(win[j], win[j + 1]);
        }
    };
    if (mask) pass(std::true_type()); else pass(std::false_type());
}

// A wavefront's tasks are (sequence, TC steps).  Step t's pre-activation is formed again from x; g_t = dy_t act'(v_t) reaches the inputs
// t - q, q <= seen(t), whose sums wait in `pend`.  An input's last share comes W - 1 steps later, so a task goes on that far (those
// steps' g belongs to the next task's filter gradient).  A step beyond the sequence's end sees nothing and gives nothing, whatever is in the state.  Filter gradients of a workgroup's tasks are added in registers, then over its
// wavefronts in a fixed order, and leave as one partial sum a workgroup.
template <typename T, int V, int W, int ACT>
__global__ __launch_bounds__(64 * ROWS, 4) void conv_backward_kernel(const ConvOp p, const int dv_blocks, const int chunks, const int groups, float *part)
{
    constexpr int TC = BACKWARD, IN = TC + 2 * (W - 1), OUT = TC + W - 1;
    const int lane = threadIdx.x & 63, row = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = blockIdx.x / dv_blocks;
    const int d = ((int)(blockIdx.x % dv_blocks) * 64 + lane) * V;
    const bool on = d < p.D;
    Filter<W, V> f;
    f.load(p, d);
    float dw[W][V], db[V];
    clear(db);
#pragma unroll
    for (int j = 0; j < W; ++j) clear(dw[j]);
    const uint32_t tasks = (uint32_t)p.N * chunks;
    for (uint32_t at = group * ROWS + row; at < tasks; at += groups * ROWS) {
        const int n = at / chunks, t0 = at % chunks * TC, len = length_of(p.lengths, n, p.T), first = t0 - (W - 1);
        Track<T, V> xa, ga, dxa;
        xa.open(p.x, n, first, d, p.D); ga.open(p.dy, n, t0, d, p.D); dxa.open(p.dx, n, t0, d, p.D);
        if (t0 > 0 && len <= first) {                // nothing reaches these steps
            float none[V];
            clear(none);
#pragma unroll
            for (int k = 0; k < TC; ++k) dxa.store(none, k, t0 + k < p.T);
            continue;
        }
        Raw<T, V, (V > 1)> xi[IN], gi[OUT];
#pragma unroll
        for (int k = 0; k < IN; ++k) xa.load(xi[k], k, first + k >= 0 && first + k < len);
#pragma unroll
        for (int k = 0; k < OUT; ++k) ga.load(gi[k], k, t0 + k < len);
        Raw<T, V, (V > 1)> tail[W - 1];
        if (t0 + OUT > len)
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                const int i = len - (W - 1) + j;
                xa.load(tail[j], i - first, i >= max(first, 0));
            }
        const uint32_t mask = begins(p.starts, first, IN, len, n, p.N, lane);
        float win[W][V], pend[W][V], last[W - 1][V];
#pragma unroll
        for (int j = 0; j < W; ++j) clear(pend[j]);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) take(win[j], xi[j]);
        if (t0 == 0 && p.state_in && on)
#pragma unroll
            for (int j = 0; j < W - 1; ++j) read_state(win[j], p.state_in, (int64_t)n * (W - 1) + j, d, p.D);
        // what dstate_out gives to the last W - 1 inputs
        const bool ends = p.dstate_out && len < t0 + TC + W - 1 && len >= first;
        if (ends) {
            const int vis = seen<W>(begins(p.starts, len - (W - 1), W - 1, len, n, p.N, lane), W - 2);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                clear(last[j]);
                if (on && W - 2 - j <= vis) read_state(last[j], p.dstate_out, (int64_t)n * (W - 1) + j, d, p.D);
            }
        }
        // CUT: perhaps the step does not see all of its window.  ENDS: perhaps there is no such step
        auto one = [&](auto cut, auto ends_here, const int k, const Raw<T, V, (V > 1)> &xk, const Raw<T, V, (V > 1)> &gk) {
            constexpr bool CUT = decltype(cut)::value, ENDS = decltype(ends_here)::value;
            const int t = t0 + k, vis = ENDS && t >= len ? -1 : CUT ? seen<W>(mask, k + W - 1) : 0;
            __builtin_amdgcn_sched_barrier(0);
            take(win[W - 1], xk);
            float v[V], g[V];
            f.template apply<CUT>(v, win, vis);
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] = ENDS && t >= len ? 0.0f : gk[i] * act_slope<ACT>(v[i]);       // (0 where there is no step)
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const bool sees = !CUT || W - 1 - j <= vis;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float given = __builtin_fmaf(f.w[j][i], g[i], pend[W - 1 - j][i]);
                    pend[W - 1 - j][i] = sees ? given : pend[W - 1 - j][i];
                    if (k < TC) {
                        const float more = __builtin_fmaf(win[j][i], g[i], dw[j][i]);
                        dw[j][i] = sees ? more : dw[j][i];
                    }
                }
            }
            if (k < TC)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    db[i] += g[i];
                    // (here and now: left to the compiler, a task's filter gradients wait for its end, with all their factors)
                    asm volatile("" : "+v"(db[i]));
#pragma unroll
                    for (int j = 0; j < W; ++j) asm volatile("" : "+v"(dw[j][i]));
                }
#pragma unroll
            for (int j = 0; j < W - 1; ++j) copy(win[j], win[j + 1]);
            // input i has all its shares
            const int i = t - (W - 1);
            if (ends)
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
                    if (i == len - (W - 1) + j)
#pragma unroll
                        for (int e = 0; e < V; ++e) pend[W - 1][e] += last[j][e];
            if (k >= W - 1) dxa.store(pend[W - 1], k - (W - 1), i < p.T);
            else if (t0 == 0 && p.dstate_in && on)
#pragma unroll
                for (int e = 0; e < V; ++e) p.dstate_in[((int64_t)n * (W - 1) + k) * p.D + d + e] = pend[W - 1][e];
#pragma unroll
            for (int j = W - 1; j > 0; --j) copy(pend[j], pend[j - 1]);
            clear(pend[0]);
        };
        // Beyond the sequence's end products with 0 give nothing, as long as everything is finite; where it is not, the task selects, a step after the other
        // (512 x 16 x 1024 in bfloat16: 18.3 us, selecting in every sequence's last task 19.4; asking nothing 17.4)
        float zero = 0.0f;                           // NaN where what the steps beyond the end would see, or the filter, is not finite
        if (t0 + OUT > len) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                zero = __builtin_fmaf(f.bias[i], 0.0f, zero);
#pragma unroll
                for (int j = 0; j < W; ++j) zero = __builtin_fmaf(f.w[j][i], 0.0f, zero);
#pragma unroll
                for (int j = 0; j < W - 1; ++j) zero = __builtin_fmaf(tail[j][i], 0.0f, zero);
                if (t0 == 0)
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) zero = __builtin_fmaf(win[j][i], 0.0f, zero);
            }
        }
        if (__ballot(zero != zero)) {
#pragma unroll 1
            for (int k = 0; k < OUT; ++k) {
                Raw<T, V, (V > 1)> xk, gk;
                xa.load(xk, k + W - 1, t0 + k < len);
                ga.load(gk, k, t0 + k < len);
                one(std::true_type(), std::true_type(), k, xk, gk);
            }
        } else if (mask)
#pragma unroll
            for (int k = 0; k < OUT; ++k) one(std::true_type(), std::false_type(), k, xi[k + W - 1], gi[k]);
        else
#pragma unroll
            for (int k = 0; k < OUT; ++k) one(std::false_type(), std::false_type(), k, xi[k + W - 1], gi[k]);
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

// workgroups over the tasks, each with a partial sum of the filter gradients: about four a compute unit (512 x 16 x 1024 in bfloat16: 18.2 us; 17.0 before tasks at a
// sequence's end looked at what they have, and with twice as many workgroups 19.2 then)
int groups_of(int64_t T, int64_t N, int64_t dv)
{
    const int64_t g = ceil_div(N * ceil_div(T, BACKWARD), ROWS), most = ceil_div(1024, dv);
    return (int)(g < most ? g : most);
}

template <bool BACKWARD_CALL, typename T, int V, int W, int ACT> hipError_t run(hts_seq_ctx &c, const ConvOp &op)
{
    const int dv = (int)ceil_div(ceil_div(op.D, V), 64);
    if constexpr (!BACKWARD_CALL) {
        const int chunks = (int)ceil_div(op.T, FORWARD);
        const int64_t workgroups = ceil_div((int64_t)op.N * chunks, ROWS) * dv;
        if (!launchable(workgroups, 64 * ROWS)) return hipErrorInvalidConfiguration;
        const dim3 grid((uint32_t)workgroups), block(64 * ROWS);
        if (op.T == 1) hipLaunchKernelGGL((conv_kernel<T, V, W, ACT, 1>), grid, block, 0, c.stream, op, dv, chunks);
        else hipLaunchKernelGGL((conv_kernel<T, V, W, ACT, FORWARD>), grid, block, 0, c.stream, op, dv, chunks);
        return hipGetLastError();
    } else {
        const int chunks = (int)ceil_div(op.T, BACKWARD);
        const int groups = groups_of(op.T, op.N, dv);
        hipLaunchKernelGGL((conv_backward_kernel<T, V, W, ACT>), dim3((uint32_t)(groups * dv)), dim3(64 * ROWS), 0, c.stream, op, dv, chunks, groups, (float *)c.ws);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        return launch_sum_partials(c, (const float *)c.ws, groups, (int64_t)op.D * (W + 1), SumTarget{op.dw, (int64_t)op.D * W}, SumTarget{op.db, (int64_t)op.D}, SumTarget{nullptr, 0});
    }
}
template <bool BACKWARD_CALL, typename T, int V> hipError_t by_width(hts_seq_ctx &c, const ConvOp &op)
{
    const bool silu = op.act == HTS_ACT_SILU;
    switch (op.W) {
    case 2: return silu ? run<BACKWARD_CALL, T, V, 2, HTS_ACT_SILU>(c, op) : run<BACKWARD_CALL, T, V, 2, HTS_ACT_NONE>(c, op);
    case 3: return silu ? run<BACKWARD_CALL, T, V, 3, HTS_ACT_SILU>(c, op) : run<BACKWARD_CALL, T, V, 3, HTS_ACT_NONE>(c, op);
    default: return silu ? run<BACKWARD_CALL, T, V, 4, HTS_ACT_SILU>(c, op) : run<BACKWARD_CALL, T, V, 4, HTS_ACT_NONE>(c, op);
    }
}
template <typename T> hipError_t by_layout(hts_seq_ctx &c, const ConvOp &op, bool backward)
{
    constexpr int V = 2;
    if (backward) return op.D % V == 0 && wide<T>(op.x, V) && wide<T>(op.dy, V) && wide<T>(op.dx, V) ? by_width<true, T, V>(c, op) : by_width<true, T, 1>(c, op);
    return op.D % V == 0 && wide<T>(op.x, V) && wide<T>(op.y, V) ? by_width<false, T, V>(c, op) : by_width<false, T, 1>(c, op);
}

}  // namespace

// (a channel a lane takes no more groups than two)
int64_t conv_workspace(int64_t T, int64_t N, int64_t D, int W) { return 4 * groups_of(T, N, ceil_div(ceil_div(D, 2), 64)) * D * (W + 1); }
hipError_t launch_conv(hts_seq_ctx &c, int precision, const ConvOp &op) { return precision == HTS_PRECISION_BF16 ? by_layout<bf16_t>(c, op, false) : by_layout<float>(c, op, false); }
hipError_t launch_conv_backward(hts_seq_ctx &c, int precision, const ConvOp &op) { return precision == HTS_PRECISION_BF16 ? by_layout<bf16_t>(c, op, true) : by_layout<float>(c, op, true); }

}  // namespace hts
