// Selective state space scan and its gradients (see include/hts.h).
//
// h_t = a_t h_{t-1} + delta_t x_t B_t with a_t = exp(delta_t A) for every channel d and state s: time is serial, channels and states are not.
// Four neighbouring lanes (a quad) hold a channel's states, SL of them a lane, in registers; a wavefront holds 16 channels of one sequence.
// Steps come in fours: lane p of a quad loads and prepares step 4 j + p (softplus, gate), the quad's other lanes get what they need of it by
// lane broadcasts, and the sums over the states are dealt out again to the lane that owns the step.  B and C, the same for all channels of a
// group, are kept for L steps in LDS as binary32.  The work is vector instructions: exp2 (two issue slots) and four others for a state and step.
//
// Steps that are none (beyond a sequence's length) have delta = x = B = C = 0: a = 1, h stays.
#include "seq.hpp"

namespace hts {
namespace {

template <int SL> struct Shape {
    static constexpr int L = SL <= 4 ? 16 : SL == 8 ? 8 : 4;      // steps of a chunk; the backward pass keeps a chunk's states in registers
    static constexpr int NB = L / 4, SP = 4 * SL, PAIR = 2 * SP;
};
constexpr int chunk_steps(int S) { return S <= 16 ? 16 : S <= 32 ? 8 : 4; }
constexpr int padded(int S) { return S <= 8 ? 8 : S <= 16 ? 16 : S <= 32 ? 32 : 64; }

__device__ __forceinline__ float quad_from(float v, int q)
{
    const int x = __float_as_int(v);
    switch (q) {
    case 0: return __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0x00, 0xf, 0xf, true));
    case 1: return __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0x55, 0xf, 0xf, true));
    case 2: return __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0xAA, 0xf, 0xf, true));
    default: return __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0xFF, 0xf, 0xf, true));
    }
}
__device__ __forceinline__ float quad_xor1(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xf, 0xf, true)); }
__device__ __forceinline__ float quad_xor2(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xf, 0xf, true)); }
template <int CTRL> __device__ __forceinline__ float row_move(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true)); }
// lane p of a quad gets the quad's sum of v[p]
__device__ __forceinline__ float quad_deal(const float (&v)[4], int p)
{
    const bool odd = p & 1, high = p & 2;
    const float a = (odd ? v[1] : v[0]) + quad_xor1(odd ? v[0] : v[1]), b = (odd ? v[3] : v[2]) + quad_xor1(odd ? v[2] : v[3]);
    return (high ? b : a) + quad_xor2(high ? a : b);
}
__device__ __forceinline__ float quad_sum(float v) { v += quad_xor1(v); return v + quad_xor2(v); }

// order for the compiler between a wavefront's LDS writes and its other lanes' reads (the hardware keeps a wavefront's LDS accesses in order)
__device__ __forceinline__ void wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

struct Places { int per_group, waves; };          // channels of a group, wavefronts (16 channels) of a group

template <typename T> __device__ __forceinline__ float wide_of(T v) { return to_f32(v); }
__device__ __forceinline__ int length_of(const int32_t *lengths, int n, int T) { return lengths ? max(0, min(T, lengths[n])) : T; }
// bit k: step t0 + k begins an episode
template <int L> __device__ __forceinline__ uint32_t starts_of(const uint8_t *starts, int t0, int len, int n, int N, int lane)
{
    if (!starts) return 0;
    const int t = t0 + (lane & (L - 1));
    const bool s = t < len && starts[(int64_t)t * N + n] != 0;
    return (uint32_t)__ballot(s) & ((1u << L) - 1);
}

// What a lane loads of a chunk: steps t0 + 4 j + p of its channel.  `full`: all of the chunk's steps exist.
template <typename T, int NB> struct Strip {
    T v[NB];
    __device__ __forceinline__ void load(const T *q, int64_t st, int t, int len)
    {
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            if (t + 4 * j < len) v[j] = q[(int64_t)(t + 4 * j) * st];
            else v[j] = from_f32<T>(0.0f);
        }
    }
};

// B and C of a chunk: the value with number i = (step, B or C, state) of L * 2 SP
template <typename T, int SL, int THREADS> struct PairLoad {
    static constexpr int PAIR = Shape<SL>::PAIR, SP = Shape<SL>::SP, L = Shape<SL>::L, NL = (L * PAIR + THREADS - 1) / THREADS;
    T v[NL];
    __device__ __forceinline__ void load(const hts_scan_inputs &in, int64_t S, int g, int n, int t0, int len, int tid)
    {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int k = i * THREADS + tid, t = t0 + k / PAIR, r = k % PAIR, s = r % SP;
            const hts_steps &a = r < SP ? in.B : in.C;
            v[i] = from_f32<T>(0.0f);
            if (k < L * PAIR && t < len && s < S) v[i] = ((const T *)a.p)[t * a.st + n * a.sn + g * S + s];
        }
    }
    __device__ __forceinline__ void put(float *lds, int tid) const
    {
#pragma unroll
        for (int i = 0; i < NL; ++i) if (i * THREADS + tid < L * PAIR) lds[i * THREADS + tid] = to_f32(v[i]);
    }
};

template <int SL> __device__ __forceinline__ void read_states(float (&v)[SL], const float *p)
{
#pragma unroll
    for (int s = 0; s < SL; ++s) v[s] = p[s];
}

constexpr int FWD_WAVES = 4;

template <typename T, int SL>
__global__ __launch_bounds__(64 * FWD_WAVES) void scan_kernel(const ScanOp p, const Places at)
{
    typedef Shape<SL> H;
    constexpr int L = H::L, NB = H::NB, SP = H::SP;
    __shared__ __attribute__((aligned(16))) float pairs[FWD_WAVES][L * H::PAIR];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per = at.waves * p.d.G;                                   // wavefronts of a sequence
    const int64_t task = (int64_t)blockIdx.x * FWD_WAVES + wave;
    if (task >= (int64_t)per * p.d.N) return;
    const int n = (int)(task / per), g = (int)(task % per) / at.waves, c = (int)(task % at.waves) * 16 + (lane >> 2), q = lane & 3;
    const bool on = c < at.per_group;
    const int d = g * at.per_group + min(c, at.per_group - 1), len = length_of(p.in.lengths, n, p.d.T), S = p.d.S;
    const T *x = (const T *)p.in.x.p + n * p.in.x.sn + d, *dt = (const T *)p.in.dt.p + n * p.in.dt.sn + d, *z = (const T *)p.in.z.p + (p.in.z.p ? n * p.in.z.sn + d : 0);
    T *y = (T *)p.y.p + n * p.y.sn + d;
    const float skip = p.in.skip ? p.in.skip[d] : 0.0f, bias = p.in.dt_bias ? p.in.dt_bias[d] : 0.0f;
    float A[SL], h[SL];
#pragma unroll
    for (int s = 0; s < SL; ++s) {
        const int k = q * SL + s;
        A[s] = k < S ? p.in.A[(int64_t)d * S + k] * LOG2E : 0.0f;
        h[s] = k < S && p.in.h_in ? p.in.h_in[((int64_t)n * p.d.D + d) * S + k] : 0.0f;
    }
    Strip<T, NB> xs, ds, zs;
    PairLoad<T, SL, 64> bc;
    uint32_t begins;
    auto fetch = [&](int t0) {
        xs.load(x, p.in.x.st, t0 + q, len);
        ds.load(dt, p.in.dt.st, t0 + q, len);
        if (p.in.z.p) zs.load(z, p.in.z.st, t0 + q, len);
        bc.load(p.in, S, g, n, t0, len, lane);
        begins = starts_of<L>(p.in.starts, t0, len, n, p.d.N, lane);
    };
    fetch(0);
    float *lds = pairs[wave];
    for (int t0 = 0, chunk = 0; t0 < p.d.T; t0 += L, ++chunk) {
        float xv[NB], size[NB], moved[NB], gate[NB];
        wave_order();
        bc.put(lds, lane);
        wave_order();
        const uint32_t fresh = begins;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int t = t0 + 4 * j + q;
            xv[j] = to_f32(xs.v[j]);
            float v = to_f32(ds.v[j]) + bias, slope;
            size[j] = v;
            if (p.d.softplus) softplus_f(v, size[j], slope);
            if (t >= len) size[j] = 0.0f;
            moved[j] = size[j] * xv[j];
            gate[j] = t >= len ? 0.0f : p.in.z.p ? act_f<HTS_ACT_SILU>(to_f32(zs.v[j])) : 1.0f;
        }
        if (t0 + L < p.d.T) fetch(t0 + L);
        if (p.states_out && on) {
            float *out = p.states_out + (((int64_t)chunk * p.d.N + n) * p.d.D + d) * SP + q * SL;
#pragma unroll
            for (int s = 0; s < SL; ++s) out[s] = h[s];
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            float sums[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = 4 * j + i;
                const float de = quad_from(size[j], i), dx = quad_from(moved[j], i);
                float B[SL], C[SL];
                read_states<SL>(B, lds + k * H::PAIR + q * SL);
                read_states<SL>(C, lds + k * H::PAIR + SP + q * SL);
                if (fresh >> k & 1)
#pragma unroll
                    for (int s = 0; s < SL; ++s) h[s] = 0.0f;
                float sum = 0.0f;
#pragma unroll
                for (int s = 0; s < SL; ++s) {
                    h[s] = __builtin_fmaf(__builtin_amdgcn_exp2f(de * A[s]), h[s], dx * B[s]);
                    sum = __builtin_fmaf(h[s], C[s], sum);
                }
                sums[i] = sum;
            }
            const float sum = quad_deal(sums, q);
            const int t = t0 + 4 * j + q;
            // (a gate of 0 and a sum that is not finite beyond the sequence's end, or for a gate of -infinity, give 0)
            if (on && t < p.d.T) y[(int64_t)t * p.y.st] = from_f32<T>(t < len ? __builtin_fmaf(skip, xv[j], sum) * gate[j] : 0.0f);
        }
    }
    if (p.h_out && on)
#pragma unroll
        for (int s = 0; s < SL; ++s)
            if (q * SL + s < S) p.h_out[((int64_t)n * p.d.D + d) * S + q * SL + s] = h[s];
}

// Sums over the 16 channels of a wavefront (lane bits 2 .. 5) of NV = 4 K values: after two exchanges of halves a lane has the sums over bits 4
// and 5 of K values, those of v[(2 bit5 + bit4) K ...], and two rotations add bits 2 and 3.
template <int K> __device__ __forceinline__ void channel_sums(float (&out)[K], const float (&v)[4 * K])
{
    float a[2 * K];
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 2 * K]), false, false);
        a[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[i]), __float_as_uint(a[i + K]), false, false);
        float s = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        s += row_move<0x128>(s);
        out[i] = s + row_move<0x124>(s);
    }
}

constexpr int BWD_WAVES = 4;

// The chunks in reverse.  A chunk's states are formed again from the state before it (kept by the forward pass) and stay in registers with the
// factors a; then, from the last step on, with r_t = dy_t silu(z_t):
//   g_t = r_t C_t + a_{t+1} g_{t+1},  dB = sum_d g delta x,  dC = sum_d r h,  d(delta) = sum_s g a h_{t-1} A + x sum_s g B,  dA = sum_t g a h_{t-1} delta
// dB and dC of a workgroup's channels are added in LDS in a fixed order and leave as a partial sum a workgroup; dA, dskip and ddt_bias stay in
// registers for the whole sequence.  At an episode's first step the products with a are 0, also where the other factor is not finite.
template <typename T, int SL>
__global__ __launch_bounds__(64 * BWD_WAVES) void scan_backward_kernel(const ScanOp p, const Places at, const int blocks, float *pair_part, float *param_part)
{
    typedef Shape<SL> H;
    constexpr int L = H::L, NB = H::NB, SP = H::SP, PAIR = H::PAIR, THREADS = 64 * BWD_WAVES;
    __shared__ __attribute__((aligned(16))) float pairs[2][L * PAIR];
    __shared__ __attribute__((aligned(16))) float sums[2][BWD_WAVES][L * PAIR];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane & 3;
    const int block = blockIdx.x % blocks, g = blockIdx.x / blocks % p.d.G, n = blockIdx.x / blocks / p.d.G;
    const int c = (block * BWD_WAVES + wave) * 16 + (lane >> 2);
    const bool on = c < at.per_group;
    const int D = p.d.D, S = p.d.S, TT = p.d.T, d = g * at.per_group + min(c, at.per_group - 1), len = length_of(p.in.lengths, n, TT);
    const T *x = (const T *)p.in.x.p + n * p.in.x.sn + d, *dt = (const T *)p.in.dt.p + n * p.in.dt.sn + d, *dy = (const T *)p.dy.p + n * p.dy.sn + d;
    const T *z = (const T *)p.in.z.p + (p.in.z.p ? n * p.in.z.sn + d : 0);
    const float skip = p.in.skip ? p.in.skip[d] : 0.0f, bias = p.in.dt_bias ? p.in.dt_bias[d] : 0.0f;
    float A[SL], ag[SL], dA[SL], dskip = 0.0f, dbias = 0.0f;
#pragma unroll
    for (int s = 0; s < SL; ++s) {
        const int k = q * SL + s;
        A[s] = k < S ? p.in.A[(int64_t)d * S + k] * LOG2E : 0.0f;
        ag[s] = on && k < S && p.dh_out ? p.dh_out[((int64_t)n * D + d) * S + k] : 0.0f;
        dA[s] = 0.0f;
    }
    Strip<T, NB> xs, ds, zs, gs;
    PairLoad<T, SL, THREADS> bc;
    float h0[SL];
    uint32_t begins;
    auto fetch = [&](int chunk) {
        const int t0 = chunk * L;
        xs.load(x, p.in.x.st, t0 + q, len);
        ds.load(dt, p.in.dt.st, t0 + q, len);
        gs.load(dy, p.dy.st, t0 + q, len);
        if (p.in.z.p) zs.load(z, p.in.z.st, t0 + q, len);
        bc.load(p.in, S, g, n, t0, len, tid);
        read_states<SL>(h0, p.states + (((int64_t)chunk * p.d.N + n) * D + d) * SP + q * SL);
        begins = starts_of<L>(p.in.starts, t0, len, n, p.d.N, lane);
    };
    auto leave = [&](int chunk, int buf) {        // the workgroup's sums of a chunk
        for (int i = tid; i < L * PAIR; i += THREADS) {
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < BWD_WAVES; ++w) s += sums[buf][w][i];
            const int t = chunk * L + i / PAIR;
            if (t < TT) pair_part[((((int64_t)block * TT + t) * p.d.N + n) * p.d.G + g) * PAIR + i % PAIR] = s;
        }
    };
    const int chunks = (TT + L - 1) / L;
    fetch(chunks - 1);
    for (int chunk = chunks - 1, buf = 0; chunk >= 0; --chunk, buf ^= 1) {
        const int t0 = chunk * L;
        bc.put(pairs[buf], tid);
        float xv[NB], size[NB], moved[NB], slope[NB], r[NB], zf[NB], hb[SL];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const bool live = t0 + 4 * j + q < len;
            xv[j] = on ? to_f32(xs.v[j]) : 0.0f;
            const float v = to_f32(ds.v[j]) + bias;
            size[j] = v; slope[j] = 1.0f;
            if (p.d.softplus) softplus_f(v, size[j], slope[j]);
            if (!live) size[j] = slope[j] = 0.0f;
            moved[j] = size[j] * xv[j];
            const float dyv = on ? to_f32(gs.v[j]) : 0.0f, zv = p.in.z.p ? to_f32(zs.v[j]) : 0.0f;
            r[j] = p.in.z.p ? dyv * act_f<HTS_ACT_SILU>(zv) : dyv;
            zf[j] = dyv * act_slope<HTS_ACT_SILU>(zv);
        }
#pragma unroll
        for (int s = 0; s < SL; ++s) hb[s] = h0[s];
        const uint32_t fresh = begins;
        __syncthreads();
        if (chunk > 0) fetch(chunk - 1);
        if (chunk < chunks - 1) leave(chunk + 1, buf ^ 1);
        const float *lds = pairs[buf];
        // twice: chunks in which no episode begins, most of them, select nothing
        auto pass = [&](auto has) {
            constexpr bool FRESH = decltype(has)::value;
            float a[L][SL], h[L][SL], raw[NB];
    #pragma unroll
            for (int j = 0; j < NB; ++j) {
                float part[4];
    #pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = 4 * j + i;
                    const float de = quad_from(size[j], i), dx = quad_from(moved[j], i);
                    float B[SL], C[SL], sum = 0.0f;
                    read_states<SL>(B, lds + k * PAIR + q * SL);
                    read_states<SL>(C, lds + k * PAIR + SP + q * SL);
                    const bool begin = FRESH && (fresh >> k & 1);
    #pragma unroll
                    for (int s = 0; s < SL; ++s) {
                        a[k][s] = __builtin_amdgcn_exp2f(de * A[s]);
                        h[k][s] = __builtin_fmaf(dx, B[s], (begin ? 0.0f : a[k][s] * (k ? h[k ? k - 1 : 0][s] : hb[s])));
                        sum = __builtin_fmaf(h[k][s], C[s], sum);
                    }
                    part[i] = sum;
                }
                raw[j] = quad_deal(part, q);
            }
    #pragma unroll
            for (int j = NB - 1; j >= 0; --j) {
                float gB[4], dd[4], val[8 * SL];
    #pragma unroll
                for (int i = 3; i >= 0; --i) {
                    const int k = 4 * j + i;
                    const float de = quad_from(size[j], i), dx = quad_from(moved[j], i), rk = quad_from(r[j], i);
                    float B[SL], C[SL];
                    read_states<SL>(B, lds + k * PAIR + q * SL);
                    read_states<SL>(C, lds + k * PAIR + SP + q * SL);
                    const bool begin = FRESH && (fresh >> k & 1);
                    gB[i] = dd[i] = 0.0f;
    #pragma unroll
                    for (int s = 0; s < SL; ++s) {
                        const float gk = __builtin_fmaf(rk, C[s], ag[s]);
                        val[2 * SL * i + s] = gk * dx;
                        val[2 * SL * i + SL + s] = rk * h[k][s];
                        gB[i] = __builtin_fmaf(gk, B[s], gB[i]);
                        const float ga = gk * (begin ? 0.0f : a[k][s] * (k ? h[k ? k - 1 : 0][s] : hb[s]));
                        dd[i] = __builtin_fmaf(ga, A[s], dd[i]);
                        dA[s] = __builtin_fmaf(ga, de, dA[s]);
                        ag[s] = begin ? 0.0f : a[k][s] * gk;
                    }
                }
                float out[2 * SL];
                channel_sums<2 * SL>(out, val);
                // lanes of channel 0 of each row: step 4 j + 2 bit5 + bit4, states q SL ...
                if ((lane & 12) == 0) {
                    float *to = sums[buf][wave] + (4 * j + 2 * (lane >> 5) + (lane >> 4 & 1)) * PAIR + q * SL;
    #pragma unroll
                    for (int s = 0; s < SL; ++s) { to[s] = out[s]; to[SP + s] = out[SL + s]; }
                }
                const float sB = quad_deal(gB, q), sd = quad_deal(dd, q) * (1.0f / LOG2E);
                const int t = t0 + 4 * j + q;
                const float ddt = __builtin_fmaf(sB, xv[j], sd) * slope[j], dx = __builtin_fmaf(sB, size[j], r[j] * skip);
                dbias += ddt; dskip = __builtin_fmaf(r[j], xv[j], dskip);
                if (on && t < TT) {
                    const bool live = t < len;
                    ((T *)p.g.dx.p)[t * p.g.dx.st + n * p.g.dx.sn + d] = from_f32<T>(live ? dx : 0.0f);
                    ((T *)p.g.ddt.p)[t * p.g.ddt.st + n * p.g.ddt.sn + d] = from_f32<T>(live ? ddt : 0.0f);
                    if (p.g.dz.p) ((T *)p.g.dz.p)[t * p.g.dz.st + n * p.g.dz.sn + d] = from_f32<T>(live ? zf[j] * __builtin_fmaf(skip, xv[j], raw[j]) : 0.0f);
                }
            }
        };
        if (fresh) pass(std::true_type()); else pass(std::false_type());
    }
    __syncthreads();
    leave(0, (chunks - 1) & 1);
    dskip = quad_sum(dskip); dbias = quad_sum(dbias);
    if (!on) return;
    float *out = param_part + (int64_t)n * D * (S + 2);
#pragma unroll
    for (int s = 0; s < SL; ++s)
        if (q * SL + s < S) {
            out[(int64_t)d * S + q * SL + s] = dA[s];
            if (p.g.dh_in) p.g.dh_in[((int64_t)n * D + d) * S + q * SL + s] = ag[s];
        }
    if (q == 0) { out[(int64_t)D * S + d] = dskip; out[(int64_t)D * (S + 1) + d] = dbias; }
}

// dB and dC from the workgroups' sums
template <typename T>
__global__ __launch_bounds__(256) void pair_sum_kernel(const ScanOp p, const int blocks, const int SP, const float *part)
{
    const int64_t width = (int64_t)p.d.T * p.d.N * p.d.G * 2 * SP, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= width) return;
    float s = 0.0f;
    for (int b = 0; b < blocks; ++b) s += part[b * width + i];
    const int r = (int)(i % (2 * SP)), k = r % SP;
    const int64_t at = i / (2 * SP), g = at % p.d.G, n = at / p.d.G % p.d.N, t = at / p.d.G / p.d.N;
    if (k >= p.d.S) return;
    const hts_steps &to = r < SP ? p.g.dB : p.g.dC;
    ((T *)to.p)[t * to.st + n * to.sn + g * p.d.S + k] = from_f32<T>(s);
}

Places places(const hts_scan_desc &d) { const int per = d.D / d.G; return Places{per, (int)ceil_div(per, 16)}; }
int blocks_of(const hts_scan_desc &d) { return (int)ceil_div(places(d).waves, BWD_WAVES); }
int64_t pair_floats(const hts_scan_desc &d) { return round_up((int64_t)blocks_of(d) * d.T * d.N * d.G * 2 * padded(d.S), 64); }
int64_t param_floats(const hts_scan_desc &d) { return (int64_t)d.N * d.D * (d.S + 2); }

template <typename T, int SL> hipError_t run(hts_seq_ctx &c, const ScanOp &op, bool backward)
{
    const Places at = places(op.d);
    if (!backward) {
        const int64_t waves = (int64_t)at.waves * op.d.G * op.d.N;
        hipLaunchKernelGGL((scan_kernel<T, SL>), dim3((uint32_t)ceil_div(waves, FWD_WAVES)), dim3(64 * FWD_WAVES), 0, c.stream, op, at);
        return hipGetLastError();
    }
    const int blocks = blocks_of(op.d);
    float *pairs = (float *)c.ws, *params = pairs + pair_floats(op.d);
    hipLaunchKernelGGL((scan_backward_kernel<T, SL>), dim3((uint32_t)((int64_t)blocks * op.d.G * op.d.N)), dim3(64 * BWD_WAVES), 0, c.stream, op, at, blocks, pairs, params);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t width = (int64_t)op.d.T * op.d.N * op.d.G * Shape<SL>::PAIR;
    hipLaunchKernelGGL((pair_sum_kernel<T>), dim3((uint32_t)ceil_div(width, 256)), dim3(256), 0, c.stream, op, blocks, Shape<SL>::SP, pairs);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int64_t D = op.d.D;
    return launch_sum_partials(c, params, op.d.N, D * (op.d.S + 2), SumTarget{op.g.dA, D * op.d.S}, SumTarget{op.g.dskip, D}, SumTarget{op.g.ddt_bias, D});
}
template <typename T> hipError_t by_states(hts_seq_ctx &c, const ScanOp &op, bool backward)
{
    switch (padded(op.d.S)) {
    case 8: return run<T, 2>(c, op, backward);
    case 16: return run<T, 4>(c, op, backward);
    case 32: return run<T, 8>(c, op, backward);
    default: return run<T, 16>(c, op, backward);
    }
}

}  // namespace

int64_t scan_states(const hts_scan_desc &d) { return ceil_div(d.T, chunk_steps(d.S)) * d.N * d.D * padded(d.S); }
int64_t scan_workspace(const hts_scan_desc &d) { return 4 * (pair_floats(d) + param_floats(d)); }
hipError_t launch_scan(hts_seq_ctx &c, const ScanOp &op) { return op.d.precision == HTS_PRECISION_BF16 ? by_states<bf16_t>(c, op, false) : by_states<float>(c, op, false); }
hipError_t launch_scan_backward(hts_seq_ctx &c, const ScanOp &op) { return op.d.precision == HTS_PRECISION_BF16 ? by_states<bf16_t>(c, op, true) : by_states<float>(c, op, true); }

}  // namespace hts
