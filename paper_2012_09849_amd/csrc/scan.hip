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
// Loads and stores through buffer descriptors: a base that all lanes share (the chunk's), 32 bits of a lane and 32 bits that all lanes share from it.
// A lane that has nothing to load or store gets an offset beyond the descriptor's 2 GB: it reads zero and writes nothing, without a branch.
// (the largest sum of both is below 2^32: the unit does not see a carry)
constexpr uint32_t REACH = 1u << 31, NOWHERE = REACH;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t reach(const char *base) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, REACH, 0x00020000); }
// (the bits in a register of its own: two 16-bit values packed into one would have to be waited for where they are loaded)
template <typename T> __device__ __forceinline__ uint32_t take(__amdgpu_buffer_rsrc_t src, uint32_t lane, uint32_t all)
{
    if constexpr (sizeof(T) == 2) return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(src, (int)lane, (int)all, 0);
    else return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(src, (int)lane, (int)all, 0);
}
template <typename T> __device__ __forceinline__ float value_of(uint32_t bits) { return __uint_as_float(sizeof(T) == 2 ? bits << 16 : bits); }
template <typename T> __device__ __forceinline__ void give(__amdgpu_buffer_rsrc_t dst, uint32_t lane, uint32_t all, float v)
{
    const T r = from_f32<T>(v);
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, r), dst, (int)lane, (int)all, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, r), dst, (int)lane, (int)all, 0);
}

// An array's chunk: the base goes from chunk to chunk, so that a chunk's addresses are a few scalar additions
struct Walk {
    const char *base;
    int64_t chunk;                     // bytes to the next chunk
    uint32_t step;                     // bytes from step to step, at most 2^26
    __device__ __forceinline__ void open(const void *p, int64_t offset, int64_t step_, int t0, int L)
    {
        base = (const char *)p + offset + t0 * step_;
        chunk = L * step_; step = (uint32_t)step_;
    }
    __device__ __forceinline__ void forth() { base += chunk; }
    __device__ __forceinline__ void back() { base -= chunk; }
};
// Where a wavefront's 16 channels of a sequence are; the lanes of step q are q steps further
template <typename T> struct Track : Walk {
    uint32_t lane;
    __device__ __forceinline__ void open(const hts_steps &a, int n, int first, int channel, int q, int t0, int L)
    {
        Walk::open(a.p, (n * a.sn + first) * (int64_t)sizeof(T), a.st * (int64_t)sizeof(T), t0, L);
        lane = a.p ? (uint32_t)q * step + (uint32_t)(channel - first) * (uint32_t)sizeof(T) : NOWHERE;
    }
    // the lane's channel in steps 4 j + q of the chunk at t0, and the next chunk's turn.  Without a branch, here and below: values that were loaded on
    // different paths would be waited for where the paths meet
    template <int NB> __device__ __forceinline__ void load(uint32_t (&v)[NB], int t0, int q, int len) const
    {
        const __amdgpu_buffer_rsrc_t src = reach(base);
#pragma unroll
        for (int j = 0; j < NB; ++j) v[j] = take<T>(src, t0 + 4 * j + q < len ? lane : NOWHERE, 4 * j * step);
    }
    template <int NB> __device__ __forceinline__ void store(const float (&v)[NB], int t0, int q, int T_, bool on) const
    {
        const __amdgpu_buffer_rsrc_t dst = reach(base);
#pragma unroll
        for (int j = 0; j < NB; ++j) give<T>(dst, on && t0 + 4 * j + q < T_ ? lane : NOWHERE, 4 * j * step, v[j]);
    }
};
// B or C of a chunk, THREADS lanes: value number i THREADS + tid is (step, state)
template <typename T, int SL, int THREADS> struct Half : Walk {
    static constexpr int SP = Shape<SL>::SP, L = Shape<SL>::L, NL = (L * SP + THREADS - 1) / THREADS, STEPS = THREADS / SP;
    static_assert(THREADS % SP == 0, "lanes");
    uint32_t lane;
    int first;                         // the lane's step of a load
    __device__ __forceinline__ void open(const hts_steps &a, int n, int g, int S, int tid, int t0)
    {
        const int k = tid % SP;
        Walk::open(a.p, (n * a.sn + (int64_t)g * S) * (int64_t)sizeof(T), a.st * (int64_t)sizeof(T), t0, L);
        first = tid / SP;
        lane = k < S && first < L ? (uint32_t)first * step + k * (uint32_t)sizeof(T) : NOWHERE;
    }
    __device__ __forceinline__ void load(uint32_t (&v)[NL], int t0, int len) const
    {
        const __amdgpu_buffer_rsrc_t src = reach(base);
#pragma unroll
        for (int i = 0; i < NL; ++i) v[i] = take<T>(src, t0 + i * STEPS + first < len ? lane : NOWHERE, i * STEPS * step);
    }
    __device__ __forceinline__ void put(const uint32_t (&v)[NL], float *lds, int tid) const
    {
#pragma unroll
        for (int i = 0; i < NL; ++i)
            if (L * SP >= THREADS || first < L) lds[(i * STEPS + first) * (2 * SP) + tid % SP] = value_of<T>(v[i]);
    }
};
// which of a chunk's steps begin an episode: a lane loads a step's flag, `mask` collects them (bit k: step t0 + k), as late as it is needed
template <int L> struct Begins : Walk {
    uint32_t lane;
    __device__ __forceinline__ void open(const uint8_t *p, int n, int N, int tid, int t0)
    {
        Walk::open(p, n, N, t0, L);
        lane = p ? (uint32_t)(tid & (L - 1)) * step : NOWHERE;
    }
    __device__ __forceinline__ void load(uint32_t &v, int t0, int len, int tid) const
    {
        v = (uint32_t)(uint8_t)__builtin_amdgcn_raw_buffer_load_b8(reach(base), t0 + (tid & (L - 1)) < len ? (int)lane : (int)NOWHERE, 0, 0);
    }
    static __device__ __forceinline__ uint32_t mask(uint32_t v) { return (uint32_t)__ballot(v != 0) & ((1u << L) - 1); }
};
// the states that a training pass keeps: SL floats of a lane, the same place in every chunk
template <int SL> struct Kept : Walk {
    uint32_t lane;
    __device__ __forceinline__ void open(const float *p, int64_t N, int n, int D, int first, int channel, int q, int chunk)
    {
        Walk::open(p, ((int64_t)n * D + first) * Shape<SL>::SP * 4, N * D * Shape<SL>::SP * 4, chunk, 1);
        lane = (uint32_t)((channel - first) * Shape<SL>::SP + q * SL) * 4u;
    }
    __device__ __forceinline__ float *at() const { return (float *)(const_cast<char *>(base) + lane); }
    // zeros where there is no such chunk
    __device__ __forceinline__ void load(float (&v)[SL], bool some) const
    {
        const __amdgpu_buffer_rsrc_t src = reach(base);
        const int from = some ? (int)lane : (int)NOWHERE;
        if constexpr (SL == 2) {
            const auto r = __builtin_amdgcn_raw_buffer_load_b64(src, from, 0, 0);
            v[0] = __uint_as_float(r[0]); v[1] = __uint_as_float(r[1]);
        } else
#pragma unroll
            for (int i = 0; i < SL / 4; ++i) {
                const auto r = __builtin_amdgcn_raw_buffer_load_b128(src, from, 16 * i, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * i + e] = __uint_as_float(r[e]);
            }
    }
};

template <int SL> __device__ __forceinline__ void read_states(float (&v)[SL], const float *p)
{
#pragma unroll
    for (int s = 0; s < SL; ++s) v[s] = p[s];
}

// B and C of the steps to come, read from LDS two steps ahead
template <int SL, bool BOTH> struct Ahead {
    static constexpr int DEPTH = 2, RING = DEPTH + 1, PAIR = Shape<SL>::PAIR, SP = Shape<SL>::SP;
    const float *lds;
    float b[RING][SL], c[RING][SL];
    __device__ __forceinline__ explicit Ahead(const float *at) : lds(at) {}
    __device__ __forceinline__ void read(int t)
    {
        read_states<SL>(b[t % RING], lds + t * PAIR);
        if (BOTH) read_states<SL>(c[t % RING], lds + t * PAIR + SP);
    }
    // before step t of L, in the order of `way`
    __device__ __forceinline__ void next(int t, int L, int way)
    {
        if (t == (way > 0 ? 0 : L - 1))
#pragma unroll
            for (int k = 0; k < DEPTH; ++k) read(t + way * k);
        if (t + way * DEPTH >= 0 && t + way * DEPTH < L) read(t + way * DEPTH);
    }
    __device__ __forceinline__ const float *B(int t) const { return b[t % RING]; }
    __device__ __forceinline__ const float *C(int t) const { return c[t % RING]; }
};

// A long sequence of few channels is cut into segments that are worked on at the same time: a first pass leaves each segment's last state, begun
// from nothing (the first one from h_in), and its sum of step sizes; exp(sum A) is then what the state before the segment counts at its end.  The
// second pass begins every segment from the states that these give, in order, so the result does not depend on who comes first.
struct Segments {
    int count, steps;                  // steps: whole chunks
    float *state, *sum;                // [count - 1][N][D][SP], [count - 1][N][D]: a sum is NaN where an episode begins in the segment and nothing before it counts
    float *h_in;                       // [N][D][SP]: h_in once more, since h_out may be h_in
};
template <int SL> __device__ __forceinline__ int64_t state_at(int64_t row, int d, int D, int q) { return (row * D + d) * Shape<SL>::SP + q * SL; }
// the state before segment k; NaN: a real sum that is NaN gives NaN states in the segment's last one too
template <int SL> __device__ __forceinline__ void state_before(float (&h)[SL], const Segments &seg, int k, int n, int N, int d, int D, int q, const float (&A)[SL])
{
    read_states<SL>(h, k == 0 ? seg.h_in + state_at<SL>(n, d, D, q) : seg.state + state_at<SL>(n, d, D, q));
#pragma unroll 4
    for (int i = 1; i < k; ++i) {
        const float sum = seg.sum[((int64_t)i * N + n) * D + d];
        float own[SL];
        read_states<SL>(own, seg.state + state_at<SL>((int64_t)i * N + n, d, D, q));
#pragma unroll
        for (int s = 0; s < SL; ++s) h[s] = sum != sum ? own[s] : __builtin_fmaf(__builtin_amdgcn_exp2f(sum * A[s]), h[s], own[s]);
    }
}

constexpr int FWD_WAVES = 4;

// STATES: the first pass over segments, which needs neither C nor the gate and writes no output
template <typename T, int SL, bool STATES>
__global__ __launch_bounds__(64 * FWD_WAVES) void scan_kernel(const ScanOp p, const Places at, const Segments seg)
{
    typedef Shape<SL> H;
    constexpr int L = H::L, NB = H::NB, SP = H::SP;
    __shared__ __attribute__((aligned(16))) float pairs[FWD_WAVES][L * H::PAIR];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), D = p.d.D, S = p.d.S, N = p.d.N;
    const int per = at.waves * p.d.G;                                   // wavefronts of a sequence's segment
    const uint32_t task = blockIdx.x * FWD_WAVES + wave, row = task / per, in_row = task % per;        // (their number has 31 bits)
    if (row >= (uint32_t)(N * (seg.count - STATES))) return;
    const int k = row / N, n = row % N, g = in_row / at.waves, c = in_row % at.waves * 16, q = lane & 3;
    const bool on = c + (lane >> 2) < at.per_group;
    const int d0 = g * at.per_group + c, d = g * at.per_group + min(c + (lane >> 2), at.per_group - 1), len = length_of(p.in.lengths, n, p.d.T);
    const int first = k * seg.steps, end = min(p.d.T, first + seg.steps);
    Track<T> xa, da, za, ya;
    Kept<SL> kept;
    xa.open(p.in.x, n, d0, d, q, first, L); da.open(p.in.dt, n, d0, d, q, first, L);
    if (!STATES) { za.open(p.in.z, n, d0, d, q, first, L); ya.open(p.y, n, d0, d, q, first, L); kept.open(p.states_out, N, n, D, d0, d, q, first / L); }
    const float skip = p.in.skip ? p.in.skip[d] : 0.0f, bias = p.in.dt_bias ? p.in.dt_bias[d] : 0.0f;
    float A[SL], h[SL], sum = 0.0f;
    bool cut = false;
#pragma unroll
    for (int s = 0; s < SL; ++s) {
        const int i = q * SL + s;
        A[s] = i < S ? p.in.A[(int64_t)d * S + i] * LOG2E : 0.0f;
        h[s] = i < S && p.in.h_in && (STATES ? k == 0 : seg.count == 1) ? p.in.h_in[((int64_t)n * D + d) * S + i] : 0.0f;
        if (STATES && k == 0 && on) seg.h_in[state_at<SL>(n, d, D, q) + s] = h[s];
    }
    if (!STATES && seg.count > 1) state_before<SL>(h, seg, k, n, N, d, D, q, A);
    Half<T, SL, 64> bs, cs;
    Begins<L> begins;
    bs.open(p.in.B, n, g, S, lane, first);
    if (!STATES) cs.open(p.in.C, n, g, S, lane, first);
    begins.open(p.in.starts, n, N, lane, first);
    struct Loads { uint32_t x[NB], dt[NB], z[NB], b[Half<T, SL, 64>::NL], c[Half<T, SL, 64>::NL], begins; } in;          // what is on its way for the next chunk
    // (beyond the segment's end nothing is loaded.)  Fenced off: were the loads moved before the last use of what they replace, they would need registers
    // of their own, and copies from these at the loop's end, which wait for them
    auto fetch = [&](int t0) {
        __builtin_amdgcn_sched_barrier(0);
        const int live = min(len, end);
        begins.load(in.begins, t0, live, lane);
        xa.load(in.x, t0, q, live);
        da.load(in.dt, t0, q, live);
        bs.load(in.b, t0, live);
        xa.forth(); da.forth(); bs.forth(); begins.forth();
        if (!STATES) {
            za.load(in.z, t0, q, live);
            cs.load(in.c, t0, live);
            za.forth(); cs.forth();
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    float *lds = pairs[wave];
    fetch(first);
    for (int t0 = first; t0 < end; t0 += L) {
        float xv[NB], size[NB], moved[NB], gate[NB];
        wave_order();
        bs.put(in.b, lds, lane);
        if (!STATES) cs.put(in.c, lds + SP, lane);
        wave_order();
        const uint32_t fresh = Begins<L>::mask(in.begins);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const bool live = t0 + 4 * j + q < len;
            xv[j] = value_of<T>(in.x[j]);
            const float v = value_of<T>(in.dt[j]) + bias;
            float soft, slope;
            softplus_f(v, soft, slope);
            size[j] = live ? p.d.softplus ? soft : v : 0.0f;
            moved[j] = size[j] * xv[j];
            const float open = act_f<HTS_ACT_SILU>(value_of<T>(in.z[j]));
            gate[j] = p.in.z.p ? open : 1.0f;
            sum += size[j];
        }
        if (STATES) cut |= fresh != 0;
        fetch(t0 + L);
        if (!STATES && p.states_out && on) {
            float *out = kept.at();
#pragma unroll
            for (int s = 0; s < SL; ++s) out[s] = h[s];
        }
        float ys[NB];
        // twice: chunks in which no episode begins, most of them, reset nothing
        auto pass = [&](auto has) {
            Ahead<SL, !STATES> ahead(lds + q * SL);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                float sums[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 4 * j + i;
                    const float de = quad_from(size[j], i), dx = quad_from(moved[j], i);
                    ahead.next(t, L, +1);
                    if (decltype(has)::value && (fresh >> t & 1))
#pragma unroll
                        for (int s = 0; s < SL; ++s) h[s] = 0.0f;
                    float y = 0.0f;
#pragma unroll
                    for (int s = 0; s < SL; ++s) {
                        h[s] = __builtin_fmaf(__builtin_amdgcn_exp2f(de * A[s]), h[s], dx * ahead.B(t)[s]);
                        if (!STATES) y = __builtin_fmaf(h[s], ahead.C(t)[s], y);
                    }
                    sums[i] = y;
                }
                if (STATES) continue;
                const float y = __builtin_fmaf(skip, xv[j], quad_deal(sums, q)) * gate[j];      // (by all lanes of the quad, those of no step too)
                ys[j] = t0 + 4 * j + q < len ? y : 0.0f;
            }
        };
        if (fresh) pass(std::true_type()); else pass(std::false_type());
        if (!STATES) { ya.store(ys, t0, q, p.d.T, on); ya.forth(); kept.forth(); }
    }
    if (!on) return;
    if (STATES) {
        float *out = seg.state + state_at<SL>((int64_t)k * N + n, d, D, q);
#pragma unroll
        for (int s = 0; s < SL; ++s) out[s] = h[s];
        sum = quad_sum(sum);
        if (q == 0) seg.sum[((int64_t)k * N + n) * D + d] = cut ? __builtin_nanf("") : sum;
    } else if (p.h_out && k == seg.count - 1)
#pragma unroll
        for (int s = 0; s < SL; ++s)
            if (q * SL + s < S) p.h_out[((int64_t)n * D + d) * S + q * SL + s] = h[s];
}

// A single step (an actor's, a server's): nothing to share between steps, so B and C come straight to the lanes that hold their states.
template <typename T, int SL>
__global__ __launch_bounds__(256) void step_kernel(const ScanOp p)
{
    constexpr int SP = Shape<SL>::SP;
    const int D = p.d.D, S = p.d.S, q = threadIdx.x & 3;
    const int64_t row = (int64_t)blockIdx.x * 64 + (threadIdx.x >> 2);
    if (row >= (int64_t)p.d.N * D) return;                              // a quad leaves together
    const int n = (int)(row / D), d = (int)(row % D), g = d / (D / p.d.G);
    const bool live = !p.in.lengths || p.in.lengths[n] > 0, fresh = live && p.in.starts && p.in.starts[n];
    float A[SL], B[SL], C[SL], h[SL];
#pragma unroll
    for (int s = 0; s < SL; ++s) {
        const int i = q * SL + s;
        A[s] = B[s] = C[s] = h[s] = 0.0f;
        if (i < S) {
            A[s] = p.in.A[(int64_t)d * S + i] * LOG2E;
            if (p.in.h_in) h[s] = p.in.h_in[row * S + i];
            if (live) { B[s] = to_f32(((const T *)p.in.B.p)[n * p.in.B.sn + (int64_t)g * S + i]); C[s] = to_f32(((const T *)p.in.C.p)[n * p.in.C.sn + (int64_t)g * S + i]); }
        }
    }
    if (p.states_out)
#pragma unroll
        for (int s = 0; s < SL; ++s) p.states_out[row * SP + q * SL + s] = h[s];
    float y = 0.0f;
    if (live) {
        const float x = to_f32(((const T *)p.in.x.p)[n * p.in.x.sn + d]), v = to_f32(((const T *)p.in.dt.p)[n * p.in.dt.sn + d]) + (p.in.dt_bias ? p.in.dt_bias[d] : 0.0f);
        const float z = p.in.z.p ? to_f32(((const T *)p.in.z.p)[n * p.in.z.sn + d]) : 0.0f;
        float size = v, slope;
        if (p.d.softplus) softplus_f(v, size, slope);
        const float dx = size * x;
#pragma unroll
        for (int s = 0; s < SL; ++s) {
            h[s] = __builtin_fmaf(__builtin_amdgcn_exp2f(size * A[s]), fresh ? 0.0f : h[s], dx * B[s]);
            y = __builtin_fmaf(h[s], C[s], y);
        }
        y = __builtin_fmaf(p.in.skip ? p.in.skip[d] : 0.0f, x, quad_sum(y)) * (p.in.z.p ? act_f<HTS_ACT_SILU>(z) : 1.0f);
    }
    if (p.h_out)
#pragma unroll
        for (int s = 0; s < SL; ++s) if (q * SL + s < S) p.h_out[row * S + q * SL + s] = h[s];
    if (q == 0) ((T *)p.y.p)[n * p.y.sn + d] = from_f32<T>(y);
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
    Track<T> xa, da, za, ga, dxa, dda, dza;
    const int d0 = g * at.per_group + min((block * BWD_WAVES + wave) * 16, at.per_group - 1);
    const int chunks = (TT + L - 1) / L, last = (chunks - 1) * L;
    xa.open(p.in.x, n, d0, d, q, last, L); da.open(p.in.dt, n, d0, d, q, last, L); za.open(p.in.z, n, d0, d, q, last, L); ga.open(p.dy, n, d0, d, q, last, L);
    dxa.open(p.g.dx, n, d0, d, q, last, L); dda.open(p.g.ddt, n, d0, d, q, last, L); dza.open(p.g.dz, n, d0, d, q, last, L);
    Kept<SL> kept;
    kept.open(p.states, p.d.N, n, D, d0, d, q, chunks - 1);
    const float skip = p.in.skip ? p.in.skip[d] : 0.0f, bias = p.in.dt_bias ? p.in.dt_bias[d] : 0.0f;
    float A[SL], ag[SL], dA[SL], dskip = 0.0f, dbias = 0.0f;
#pragma unroll
    for (int s = 0; s < SL; ++s) {
        const int k = q * SL + s;
        A[s] = k < S ? p.in.A[(int64_t)d * S + k] * LOG2E : 0.0f;
        ag[s] = on && k < S && p.dh_out ? p.dh_out[((int64_t)n * D + d) * S + k] : 0.0f;
        dA[s] = 0.0f;
    }
    uint32_t xs[NB], ds[NB], zs[NB], gs[NB];
    Half<T, SL, THREADS> bs, cs;
    bs.open(p.in.B, n, g, S, tid, last);
    cs.open(p.in.C, n, g, S, tid, last);
    float h0[SL];
    uint32_t bv[Half<T, SL, THREADS>::NL], cv[Half<T, SL, THREADS>::NL];
    Begins<L> begins;
    begins.open(p.in.starts, n, p.d.N, lane, last);
    uint32_t flag;
    auto fetch = [&](int chunk) {          // (there is nothing to load before the first chunk)
        __builtin_amdgcn_sched_barrier(0);
        const int t0 = chunk * L, live = chunk >= 0 ? len : t0;
        begins.load(flag, t0, live, lane);
        xa.load(xs, t0, q, live);
        da.load(ds, t0, q, live);
        ga.load(gs, t0, q, live);
        za.load(zs, t0, q, live);
        bs.load(bv, t0, live);
        cs.load(cv, t0, live);
        kept.load(h0, chunk >= 0);
        xa.back(); da.back(); za.back(); ga.back(); bs.back(); cs.back(); begins.back(); kept.back();
        __builtin_amdgcn_sched_barrier(0);
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
    fetch(chunks - 1);
    for (int chunk = chunks - 1, buf = 0; chunk >= 0; --chunk, buf ^= 1) {
        const int t0 = chunk * L;
        bs.put(bv, pairs[buf], tid);
        cs.put(cv, pairs[buf] + SP, tid);
        float xv[NB], size[NB], moved[NB], slope[NB], r[NB], zf[NB], hb[SL];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const bool live = t0 + 4 * j + q < len;
            xv[j] = on ? value_of<T>(xs[j]) : 0.0f;
            const float v = value_of<T>(ds[j]) + bias;
            float soft, rise;
            softplus_f(v, soft, rise);
            size[j] = live ? p.d.softplus ? soft : v : 0.0f;
            slope[j] = live ? p.d.softplus ? rise : 1.0f : 0.0f;
            moved[j] = size[j] * xv[j];
            const float dyv = on ? value_of<T>(gs[j]) : 0.0f, zv = value_of<T>(zs[j]);
            const float open = act_f<HTS_ACT_SILU>(zv);
            r[j] = dyv * (p.in.z.p ? open : 1.0f);
            zf[j] = dyv * act_slope<HTS_ACT_SILU>(zv);
        }
#pragma unroll
        for (int s = 0; s < SL; ++s) hb[s] = h0[s];
        const uint32_t fresh = Begins<L>::mask(flag);
        __syncthreads();
        fetch(chunk - 1);
        if (chunk < chunks - 1) leave(chunk + 1, buf ^ 1);
        const float *lds = pairs[buf];
        // twice: chunks in which no episode begins, most of them, select nothing
        auto pass = [&](auto has) {
            constexpr bool FRESH = decltype(has)::value;
            float a[L][SL], h[L][SL], raw[NB];
            {
                Ahead<SL, true> ahead(lds + q * SL);
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    float part[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int k = 4 * j + i;
                        const float de = quad_from(size[j], i), dx = quad_from(moved[j], i);
                        ahead.next(k, L, +1);
                        const bool begin = FRESH && (fresh >> k & 1);
                        float sum = 0.0f;
#pragma unroll
                        for (int s = 0; s < SL; ++s) {
                            a[k][s] = __builtin_amdgcn_exp2f(de * A[s]);
                            h[k][s] = __builtin_fmaf(dx, ahead.B(k)[s], begin ? 0.0f : a[k][s] * (k ? h[k ? k - 1 : 0][s] : hb[s]));
                            sum = __builtin_fmaf(h[k][s], ahead.C(k)[s], sum);
                        }
                        part[i] = sum;
                    }
                    raw[j] = quad_deal(part, q);
                }
            }
            float outx[NB], outd[NB], outz[NB];
            Ahead<SL, true> ahead(lds + q * SL);
#pragma unroll
            for (int j = NB - 1; j >= 0; --j) {
                float gB[4], dd[4], val[8 * SL];
#pragma unroll
                for (int i = 3; i >= 0; --i) {
                    const int k = 4 * j + i;
                    const float de = quad_from(size[j], i), dx = quad_from(moved[j], i), rk = quad_from(r[j], i);
                    ahead.next(k, L, -1);
                    const bool begin = FRESH && (fresh >> k & 1);
                    gB[i] = dd[i] = 0.0f;
#pragma unroll
                    for (int s = 0; s < SL; ++s) {
                        const float gk = __builtin_fmaf(rk, ahead.C(k)[s], ag[s]);
                        val[2 * SL * i + s] = gk * dx;
                        val[2 * SL * i + SL + s] = rk * h[k][s];
                        gB[i] = __builtin_fmaf(gk, ahead.B(k)[s], gB[i]);
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
                const bool live = t0 + 4 * j + q < len;
                const float ddt = __builtin_fmaf(sB, xv[j], sd) * slope[j];
                dbias += ddt; dskip = __builtin_fmaf(r[j], xv[j], dskip);
                outx[j] = live ? __builtin_fmaf(sB, size[j], r[j] * skip) : 0.0f;
                outd[j] = live ? ddt : 0.0f;
                outz[j] = live ? zf[j] * __builtin_fmaf(skip, xv[j], raw[j]) : 0.0f;
            }
            dxa.store(outx, t0, q, TT, on);
            dda.store(outd, t0, q, TT, on);
            if (p.g.dz.p) dza.store(outz, t0, q, TT, on);
            dxa.back(); dda.back(); dza.back();
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

// Segments of a sequence: where its wavefronts leave most units idle, as many as give two to a SIMD, of 64 steps at least.  The first pass costs
// four fifths of the second.
constexpr int MOST_SEGMENTS = 64;
int segments_of(const hts_scan_desc &d, int cus)
{
    const int64_t waves = (int64_t)places(d).waves * d.G * d.N, units = 4ll * cus;
    if (2 * waves > units) return 1;
    int64_t count = 2 * units / waves;
    if (count > d.T / 64) count = d.T / 64;
    if (count > MOST_SEGMENTS) count = MOST_SEGMENTS;
    if (count < 3) return 1;           // two passes over halves gain nothing
    return (int)ceil_div(d.T, round_up(ceil_div(d.T, count), chunk_steps(d.S)));
}
int64_t segment_floats(const hts_scan_desc &d, int count) { return count > 1 ? (int64_t)d.N * d.D * (padded(d.S) * (int64_t)count + (count - 1)) : 0; }

template <typename T, int SL> hipError_t run(hts_seq_ctx &c, const ScanOp &op, bool backward)
{
    const Places at = places(op.d);
    if (!backward) {
        if (op.d.T == 1) {
            hipLaunchKernelGGL((step_kernel<T, SL>), dim3((uint32_t)ceil_div((int64_t)op.d.N * op.d.D, 64)), dim3(256), 0, c.stream, op);
            return hipGetLastError();
        }
        Segments seg = {};
        seg.count = segments_of(op.d, c.cus < 256 ? c.cus : 256);
        seg.steps = (int)round_up(ceil_div(op.d.T, seg.count), Shape<SL>::L);
        const int64_t states = (int64_t)op.d.N * op.d.D * Shape<SL>::SP, waves = (int64_t)at.waves * op.d.G * op.d.N;
        if (seg.count > 1) {
            seg.h_in = (float *)c.ws;
            seg.state = seg.h_in + states;
            seg.sum = seg.state + (seg.count - 1) * states;
            hipLaunchKernelGGL((scan_kernel<T, SL, true>), dim3((uint32_t)ceil_div(waves * (seg.count - 1), FWD_WAVES)), dim3(64 * FWD_WAVES), 0, c.stream, op, at, seg);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL((scan_kernel<T, SL, false>), dim3((uint32_t)ceil_div(waves * seg.count, FWD_WAVES)), dim3(64 * FWD_WAVES), 0, c.stream, op, at, seg);
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
int64_t scan_workspace(const hts_scan_desc &d, bool backward)
{
    // (on fewer compute units there are fewer segments)
    if (!backward) return 4 * segment_floats(d, segments_of(d, 256));
    return 4 * (pair_floats(d) + param_floats(d));
}
hipError_t launch_scan(hts_seq_ctx &c, const ScanOp &op) { return op.d.precision == HTS_PRECISION_BF16 ? by_states<bf16_t>(c, op, false) : by_states<float>(c, op, false); }
hipError_t launch_scan_backward(hts_seq_ctx &c, const ScanOp &op) { return op.d.precision == HTS_PRECISION_BF16 ? by_states<bf16_t>(c, op, true) : by_states<float>(c, op, true); }

}  // namespace hts
