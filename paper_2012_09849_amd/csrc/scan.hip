// Selective state space scan and its gradients (see include/hts.h).
//
// h_t = a_t h_{t-1} + delta_t x_t B_t with a_t = exp(delta_t A) for every channel d and state s: time is serial, channels and states are not.
// Four neighbouring lanes (a quad) hold a channel's states, SL of them a lane, in registers; a wavefront holds 16 channels of one sequence, L steps
// (a chunk) at a time.  What belongs to a step and channel (softplus, gate, the outputs) is another lane's work: memory is read and written with a lane
// for NB neighbouring channels of a step, so that a chunk is one instruction an array, and step sizes, inputs and sums over the states pass between the
// two orders through LDS, which also holds B and C, the same for all channels of a group, as binary32.  The work is vector instructions: exp2 (two issue
// slots) and four others for a state and step.
// What bounds it: issue.  512 x 16 x 1024 channels of 16 states in bfloat16, forward 68 us: a wavefront a SIMD that issues in 72 % of its cycles, 555 vector instructions
// for 16 steps, 384 slots of them the states'; a prompt of 8192 steps 33 + 56 us, two wavefronts a SIMD, whose vector instructions take 89 % of the cycles; backward 27
// (a wavefront a SIMD, 71 %) + 124 (two, 97 %).  Twice as many segments (four wavefronts a SIMD) left the prompt at 32 + 61 where these took 33 + 53.
//
// States beyond S and channels beyond the last are zeros all through; where infinities come, whose products with those would be NaN, a chunk selects.
// Steps that are none (beyond a sequence's length) do nothing, whatever the state: 0 times an infinite one would be NaN.  Chunks of them are passed over.
#include <algorithm>

#include "seq.hpp"

namespace hts {
namespace {

// L: steps of a chunk.  The backward pass keeps a chunk's states and factors in registers, 2 L SL of them: half as many steps for 16 states, which leaves
// two wavefronts a SIMD
template <int SL_, int L_> struct Shape { static constexpr int SL = SL_, L = L_, NB = L / 4, SP = 4 * SL, PAIR = 2 * SP; };
template <int SL> using Forth = Shape<SL, SL <= 4 ? 16 : SL == 8 ? 8 : 4>;
template <int SL> using Back = Shape<SL, SL <= 2 ? 16 : SL <= 8 ? 8 : 4>;
constexpr int back_steps(int S) { return S <= 8 ? 16 : S <= 32 ? 8 : 4; }
constexpr int padded(int S) { return S <= 8 ? 8 : S <= 16 ? 16 : S <= 32 ? 32 : 64; }

__device__ __forceinline__ float quad_xor1(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xf, 0xf, true)); }
__device__ __forceinline__ float quad_xor2(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xf, 0xf, true)); }
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

// A chunk's steps, by what is in it: most chunks have no episode that begins, no end of the sequence and no infinities, and ask nothing; a sequence ends once.  EACH: a
// copy for episodes' beginnings alone, otherwise one for all (the gradients' main kernel, whose registers are full: 256 x 16 x 1024 channels of 32 states, both passes, 317 us,
// with three copies 331; the other kernels three: 512 x 16 of 16 states 206 us, with two 210)
template <bool EACH, class Pass> __device__ __forceinline__ void by_kind(const Pass &pass, bool fresh, bool odd)
{
    if (odd || (!EACH && fresh)) pass(std::integral_constant<int, 2>());
    else if (EACH && fresh) pass(std::integral_constant<int, 1>());
    else pass(std::integral_constant<int, 0>());
}

// how many of a lane's states exist, counted anew where it is asked for (kept, the comparisons with it would take scalar registers all through)
template <int SL> __device__ __forceinline__ int states_of(int S, int q, bool on)
{
    int n = on ? S - q * SL : 0;
    asm volatile("" : "+v"(n));
    return n;
}
// zero, or NaN from the first value on that is not finite
__device__ __forceinline__ void look(float &zero, float v) { zero = __builtin_fmaf(v, 0.0f, zero); }

struct Places { int per_group, waves; };          // channels of a group, wavefronts (16 channels) of a group

__device__ __forceinline__ int length_of(const int32_t *lengths, int n, int T) { return lengths ? max(0, min(T, lengths[n])) : T; }
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

// The order of memory: lane = (step of the chunk, V neighbouring ones of the wavefront's 16 channels)
template <class H> struct Cell {
    static constexpr int V = H::NB, PER = 16 / V;
    int step, channel, count;          // count: of the V channels that exist
    __device__ __forceinline__ void open(int lane, int channels)
    {
        step = lane / PER; channel = lane % PER * V;
        count = max(0, min(V, channels - channel));
    }
};
template <typename T, class H, bool WIDE> struct Track : Walk {
    static constexpr int V = H::NB;
    uint32_t lane;
    __device__ __forceinline__ void open(const hts_steps &a, int n, int first, const Cell<H> &c, int t0)
    {
        Walk::open(a.p, (n * a.sn + first) * (int64_t)sizeof(T), a.st * (int64_t)sizeof(T), t0, H::L);
        lane = a.p && c.count > 0 ? (uint32_t)c.step * step + (uint32_t)c.channel * (uint32_t)sizeof(T) : NOWHERE;
    }
    __device__ __forceinline__ void load(Raw<T, V, WIDE> &v, bool live, const Cell<H> &c) const { v.load(reach(base), live ? lane : NOWHERE, live ? c.count : 0); }
    __device__ __forceinline__ void store(const float (&v)[V], bool some, const Cell<H> &c) const { put_raw<T, V, WIDE>(reach(base), some ? lane : NOWHERE, some ? c.count : 0, v); }
};
// B or C of a chunk: 4 neighbouring states of a step a lane
template <typename T, class H, bool WIDE> struct Half : Walk {
    static constexpr int SP = H::SP, L = H::L;
    static_assert(L * SP <= 256, "lanes");
    uint32_t lane;
    int at, count, row;                // its step, how many of the 4 states exist, its place in LDS
    __device__ __forceinline__ void open(const hts_steps &a, int n, int g, int S, int tid, int t0)
    {
        const int s = tid * 4 % SP;
        Walk::open(a.p, (n * a.sn + (int64_t)g * S) * (int64_t)sizeof(T), a.st * (int64_t)sizeof(T), t0, L);
        at = tid * 4 / SP;
        count = at < L ? max(0, min(4, S - s)) : 0;
        lane = count > 0 ? (uint32_t)at * step + (uint32_t)s * (uint32_t)sizeof(T) : NOWHERE;
        row = at * H::PAIR + s;
    }
    __device__ __forceinline__ void load(Raw<T, 4, WIDE> &v, int t0, int len) const { v.load(reach(base), t0 + at < len ? lane : NOWHERE, t0 + at < len ? count : 0); }
    __device__ __forceinline__ void put(const Raw<T, 4, WIDE> &v, float *lds) const
    {
        if (L * SP < 256 && at >= L) return;
        *reinterpret_cast<f32x4 *>(lds + row) = f32x4{v[0], v[1], v[2], v[3]};
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
// Between the two orders: [16 channels][L steps] of binary32, a row a multiple of 16 bytes long that spreads the channels over the banks
template <class H> struct Swap {
    static constexpr int V = H::NB, L = H::L, PITCH = L + 4, SIZE = 16 * PITCH;
    static __device__ __forceinline__ void put(float *lds, const Cell<H> &c, const float (&v)[V])
    {
#pragma unroll
        for (int e = 0; e < V; ++e) lds[(c.channel + e) * PITCH + c.step] = v[e];
    }
    static __device__ __forceinline__ void get(float (&v)[V], const float *lds, const Cell<H> &c)
    {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = lds[(c.channel + e) * PITCH + c.step];
    }
    // steps 4 j .. 4 j + 3 of a quad's channel
    static __device__ __forceinline__ f32x4 four(const float *lds, int channel, int j) { return *reinterpret_cast<const f32x4 *>(lds + channel * PITCH + 4 * j); }
};
// the states that a training pass keeps: SL floats of a lane, the same place in every chunk
template <int SL> struct Kept : Walk {
    uint32_t lane;
    __device__ __forceinline__ void open(const float *p, int64_t N, int n, int D, int first, int channel, int q, int chunk)
    {
        Walk::open(p, ((int64_t)n * D + first) * 4 * SL * 4, N * D * 4 * SL * 4, chunk, 1);
        lane = (uint32_t)((channel - first) * 4 * SL + q * SL) * 4u;
    }
    __device__ __forceinline__ void store(const float (&v)[SL], bool some) const
    {
        typedef uint32_t u2 __attribute__((ext_vector_type(2)));
        typedef uint32_t u4 __attribute__((ext_vector_type(4)));
        const __amdgpu_buffer_rsrc_t dst = reach(base);
        const int to = some ? (int)lane : (int)NOWHERE;
        auto w = [&](int i) { return __float_as_uint(v[i]); };
        if constexpr (SL == 2) __builtin_amdgcn_raw_buffer_store_b64(u2{w(0), w(1)}, dst, to, 0, 0);
        else
#pragma unroll
            for (int i = 0; i < SL; i += 4) __builtin_amdgcn_raw_buffer_store_b128(u4{w(i), w(i + 1), w(i + 2), w(i + 3)}, dst, to, 4 * i, 0);
    }
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
template <class H, bool BOTH> struct Ahead {
    static constexpr int DEPTH = 2, RING = DEPTH + 1, PAIR = H::PAIR, SP = H::SP, SL = H::SL, L = H::L;
    const float *lds;
    float b[RING][SL], c[RING][SL];
    __device__ __forceinline__ explicit Ahead(const float *at) : lds(at) {}
    __device__ __forceinline__ void read(int t)
    {
        read_states<SL>(b[t % RING], lds + t * PAIR);
        if (BOTH) read_states<SL>(c[t % RING], lds + t * PAIR + SP);
    }
    // before step t, in the order of `way`
    __device__ __forceinline__ void next(int t, int way)
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
// second pass begins every segment from the states that these give, in order, so the result does not depend on who comes first.  Backward the same with
// the gradient of the state, from the last segment to the first.
struct Segments {
    int count, steps;                  // steps: whole chunks
    float *state, *sum;                // [segment][N][D][SP], [segment][N][D]: a sum is NaN where an episode begins in the segment and nothing before it counts
    float *h_in;                       // forward: [N][D][SP]: h_in once more, since h_out may be h_in
};
template <int SL> __device__ __forceinline__ int64_t state_at(int64_t row, int d, int D, int q) { return (row * D + d) * 4 * SL + q * SL; }
// h over what the segments from `first` to before `last` (in steps of `way`) do to it.  (A real sum that is NaN gives NaN states of its own too; one of 0, of
// a segment without steps, leaves h whatever A.)
template <int SL> __device__ __forceinline__ void over_segments(float (&h)[SL], const Segments &seg, int first, int last, int way, int n, int N, int d, int D, int q, const float (&A)[SL])
{
#pragma unroll 4
    for (int i = first; i != last; i += way) {
        const float sum = seg.sum[((int64_t)i * N + n) * D + d];
        // exp(sum A) in two factors, since it may be beyond binary32's range where the state times it is not.  Finite, for the sake of states of 0 (those beyond S, too), and
        // not 0 for infinite ones, which no finite step size takes away
        const float least = sum == 0.0f ? 1.0f : __builtin_fabsf(sum) < __builtin_inff() ? 0x1p-126f : 0.0f;
        float own[SL];
        read_states<SL>(own, seg.state + state_at<SL>((int64_t)i * N + n, d, D, q));
#pragma unroll
        for (int s = 0; s < SL; ++s) {
            const float half = fminf(fmaxf(__builtin_amdgcn_exp2f(0.5f * sum * A[s]), least), 0x1.fffffep+127f);
            h[s] = sum != sum ? own[s] : __builtin_fmaf(h[s] * half, half, own[s]);
        }
    }
}

constexpr int FWD_WAVES = 4;

// STATES: the first pass over segments, which needs neither C nor the gate and writes no output.  ABSENT: there are states beyond S
template <typename T, int SL, bool WIDE, bool ABSENT, bool STATES>
__global__ __launch_bounds__(64 * FWD_WAVES) void scan_kernel(const ScanOp p, const Places at, const Segments seg)
{
    typedef Forth<SL> H;
    typedef Swap<H> X;
    constexpr int L = H::L, NB = H::NB, SP = H::SP, KEEP = Back<SL>::L;
    __shared__ __attribute__((aligned(16))) float shared[FWD_WAVES][L * H::PAIR + 3 * X::SIZE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), D = p.d.D, S = p.d.S, N = p.d.N;
    const int per = at.waves * p.d.G;                                   // wavefronts of a sequence's segment
    const uint32_t task = blockIdx.x * FWD_WAVES + wave, row = task / per, in_row = task % per;        // (their number has 31 bits)
    if (row >= (uint32_t)(N * (seg.count - STATES))) return;
    const int k = row / N, n = row % N, g = in_row / at.waves, c = in_row % at.waves * 16, q = lane & 3, own = lane >> 2;
    const int d0 = g * at.per_group + c, d = d0 + own, len = length_of(p.in.lengths, n, p.d.T);
    const bool on = c + own < at.per_group;
    const int first = k * seg.steps, end = min(p.d.T, first + seg.steps), live = min(len, end);
    Cell<H> cell;
    cell.open(lane, at.per_group - c);
    Track<T, H, WIDE> xa, da, za, ya;
    Kept<SL> kept;
    xa.open(p.in.x, n, d0, cell, first); da.open(p.in.dt, n, d0, cell, first);
    if (!STATES) { za.open(p.in.z, n, d0, cell, first); ya.open(p.y, n, d0, cell, first); kept.open(p.states_out, N, n, D, d0, d, q, first / KEEP); }
    float skip[NB], bias[NB], sum[NB];
#pragma unroll
    for (int e = 0; e < NB; ++e) {
        const bool some = e < cell.count;
        skip[e] = some && p.in.skip ? p.in.skip[d0 + cell.channel + e] : 0.0f;
        bias[e] = some && p.in.dt_bias ? p.in.dt_bias[d0 + cell.channel + e] : 0.0f;
        sum[e] = 0.0f;
    }
    float A[SL], h[SL];
    bool cut = false;
#pragma unroll
    for (int s = 0; s < SL; ++s) {
        const int i = q * SL + s;
        A[s] = on && i < S ? p.in.A[(int64_t)d * S + i] * LOG2E : 0.0f;
        h[s] = on && i < S && p.in.h_in && (STATES ? k == 0 : seg.count == 1) ? p.in.h_in[((int64_t)n * D + d) * S + i] : 0.0f;
        if (STATES && k == 0 && on) seg.h_in[state_at<SL>(n, d, D, q) + s] = h[s];
    }
    if (!STATES && seg.count > 1 && on) {
        read_states<SL>(h, k == 0 ? seg.h_in + state_at<SL>(n, d, D, q) : seg.state + state_at<SL>(n, d, D, q));
        over_segments<SL>(h, seg, 1, max(k, 1), 1, n, N, d, D, q, A);
    }
    Half<T, H, WIDE> bs, cs;
    Begins<L> begins;
    bs.open(p.in.B, n, g, S, lane, first);
    if (!STATES) cs.open(p.in.C, n, g, S, lane, first);
    begins.open(p.in.starts, n, N, lane, first);
    struct { Raw<T, NB, WIDE> x, dt, z; Raw<T, 4, WIDE> b, c; uint32_t begins; } in;          // what is on its way for the next chunk
    // (beyond the segment's end nothing is loaded.)  Fenced off: were the loads moved before the last use of what they replace, they would need registers
    // of their own, and copies from these at the loop's end, which wait for them
    auto fetch = [&](int t0) {
        __builtin_amdgcn_sched_barrier(0);
        const bool some = t0 + cell.step < live;
        begins.load(in.begins, t0, live, lane);
        xa.load(in.x, some, cell);
        da.load(in.dt, some, cell);
        bs.load(in.b, t0, live);
        xa.forth(); da.forth(); bs.forth(); begins.forth();
        if (!STATES) {
            za.load(in.z, some, cell);
            cs.load(in.c, t0, live);
            za.forth(); cs.forth();
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    float *pairs = shared[wave], *sizes = pairs + L * H::PAIR, *moves = sizes + X::SIZE, *outs = moves + X::SIZE;
    fetch(first);
    int t0 = first;
    for (; t0 < live; t0 += L) {
        const bool some = t0 + cell.step < live;
        float xv[NB], size[NB], moved[NB], gate[NB], zero = 0.0f;
        wave_order();
        bs.put(in.b, pairs);
        if (!STATES) cs.put(in.c, pairs + SP);
        const uint32_t fresh = Begins<L>::mask(in.begins);
#pragma unroll
        for (int e = 0; e < NB; ++e) {
            xv[e] = in.x[e];
            const float v = in.dt[e] + bias[e];
            float soft, slope;
            softplus_f(v, soft, slope);
            size[e] = some ? p.d.softplus ? soft : v : 0.0f;
            moved[e] = size[e] * xv[e];
            if (ABSENT) look(zero, moved[e]);
            const float open = STATES ? 1.0f : act_f<HTS_ACT_SILU>(in.z[e]);
            gate[e] = p.in.z.p ? open : 1.0f;
            sum[e] += size[e];
        }
        X::put(sizes, cell, size);
        X::put(moves, cell, moved);
        if (STATES) cut |= fresh != 0;
        wave_order();
        fetch(t0 + L);
        const bool keep = !STATES && p.states_out;
        const int steps = live - t0;                                    // that there are, of the chunk's
        auto pass = [&](auto kind) {
            constexpr bool FRESH = decltype(kind)::value > 0, ODD = decltype(kind)::value > 1;
            const int exist = ABSENT && ODD ? states_of<SL>(S, q, on) : SL;
            Ahead<H, !STATES> ahead(pairs + q * SL);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const f32x4 de = X::four(sizes, own, j), dx = X::four(moves, own, j);
                float sums[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 4 * j + i;
                    ahead.next(t, +1);
                    if (t % KEEP == 0 && keep) { kept.store(h, on && t0 + t < p.d.T); kept.forth(); }
                    if (FRESH && (fresh >> t & 1))
#pragma unroll
                        for (int s = 0; s < SL; ++s) h[s] = 0.0f;
                    float y = 0.0f;
#pragma unroll
                    for (int s = 0; s < SL; ++s) {
                        const bool none = ODD && (t >= steps || s >= exist);
                        const float next = __builtin_fmaf(__builtin_amdgcn_exp2f(de[i] * A[s]), h[s], dx[i] * ahead.B(t)[s]);
                        h[s] = none ? h[s] : next;
                        if (!STATES) y = __builtin_fmaf(h[s], ahead.C(t)[s], y);
                    }
                    sums[i] = y;
                }
                if (!STATES) outs[own * X::PITCH + 4 * j + q] = quad_deal(sums, q);
            }
        };
        by_kind<true>(pass, fresh, steps < L || (ABSENT && __ballot(zero != zero)));
        if (!STATES) {
            wave_order();
            float y[NB];
            X::get(y, outs, cell);
            // (beyond the sequence's end 0 whatever the state)
#pragma unroll
            for (int e = 0; e < NB; ++e) y[e] = some ? __builtin_fmaf(skip[e], xv[e], y[e]) * gate[e] : 0.0f;
            ya.store(y, t0 + cell.step < p.d.T, cell);
            ya.forth();
        }
    }
    if (!STATES)                                                        // chunks without steps
        for (; t0 < end; t0 += L) {
            float y[NB];
#pragma unroll
            for (int e = 0; e < NB; ++e) y[e] = 0.0f;
            ya.store(y, t0 + cell.step < p.d.T, cell);
            ya.forth();
            if (p.states_out)
#pragma unroll
                for (int t = 0; t < L; t += KEEP) { kept.store(h, on && t0 + t < p.d.T); kept.forth(); }
        }
    if (STATES) {
        if (on) {
            float *out = seg.state + state_at<SL>((int64_t)k * N + n, d, D, q);
#pragma unroll
            for (int s = 0; s < SL; ++s) out[s] = h[s];
        }
        // over the chunk's steps, which are other lanes
#pragma unroll
        for (int e = 0; e < NB; ++e) {
#pragma unroll
            for (int m = Cell<H>::PER; m < 64; m *= 2) sum[e] += __shfl_xor(sum[e], m);
            if (cell.step == 0 && e < cell.count) seg.sum[((int64_t)k * N + n) * D + d0 + cell.channel + e] = cut ? __builtin_nanf("") : sum[e];
        }
    } else if (on && p.h_out && k == seg.count - 1)
#pragma unroll
        for (int s = 0; s < SL; ++s)
            if (q * SL + s < S) p.h_out[((int64_t)n * D + d) * S + q * SL + s] = h[s];
}

// A single step (an actor's, a server's): nothing to share between steps, so B and C come straight to the lanes that hold their states.
template <typename T, int SL>
__global__ __launch_bounds__(256) void step_kernel(const ScanOp p)
{
    constexpr int SP = 4 * SL;
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
            if (q * SL + s >= S) continue;
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

// Sums over the 16 channels of a wavefront (lane bits 2 .. 5) of NV values; each step halves the values that a lane keeps.  Within a row of 16 lanes an
// addition takes its neighbour's value along and writes half the row's banks only, so two of them halve a pair of values: 1 issue slot a value, where an
// exchange between rows takes 1.5.  A lane ends with the sums of v[(8 bit3 + 4 bit2 + 2 bit4 + bit5) NV / 16 ...].
// (written out, since the compiler selects with instructions of its own; an instruction that takes a neighbour's value has to be two slots after the one
// that wrote it, and the exchange that follows one after)
#define HTS_FOLD(NAME, LOW, HIGH, LOWBANKS, HIGHBANKS)                                                                                                     \
    __device__ __forceinline__ void NAME(float &a, float &b, float a0, float a1, float b0, float b1)                                                      \
    {                                                                                                                                                     \
        asm("s_nop 1\n\t"                                                                                                                                 \
            "v_add_f32_dpp %0, %2, %2 " LOW " row_mask:0xf bank_mask:" LOWBANKS "\n\t"                                                                    \
            "v_add_f32_dpp %1, %4, %4 " LOW " row_mask:0xf bank_mask:" LOWBANKS "\n\t"                                                                    \
            "v_add_f32_dpp %0, %3, %3 " HIGH " row_mask:0xf bank_mask:" HIGHBANKS "\n\t"                                                                  \
            "v_add_f32_dpp %1, %5, %5 " HIGH " row_mask:0xf bank_mask:" HIGHBANKS "\n\t"                                                                  \
            "s_nop 1"                                                                                                                                     \
            : "=&v"(a), "=&v"(b) : "v"(a0), "v"(a1), "v"(b0), "v"(b1));                                                                                   \
    }
HTS_FOLD(fold_bit3, "row_ror:8", "row_ror:8", "0x3", "0xc")
HTS_FOLD(fold_bit2, "row_shl:4", "row_shr:4", "0x5", "0xa")
#undef HTS_FOLD
template <int NV> __device__ __forceinline__ void channel_sums(float (&out)[NV / 16], const float (&v)[NV])
{
    float a[NV / 2], b[NV / 4], c[NV / 8];
#pragma unroll
    for (int i = 0; i < NV / 2; i += 2) fold_bit3(a[i], a[i + 1], v[i], v[i + NV / 2], v[i + 1], v[i + 1 + NV / 2]);
#pragma unroll
    for (int i = 0; i < NV / 4; i += 2) fold_bit2(b[i], b[i + 1], a[i], a[i + NV / 4], a[i + 1], a[i + 1 + NV / 4]);
#pragma unroll
    for (int i = 0; i < NV / 8; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(b[i]), __float_as_uint(b[i + NV / 8]), false, false);
        c[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
#pragma unroll
    for (int i = 0; i < NV / 16; ++i) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(c[i]), __float_as_uint(c[i + NV / 16]), false, false);
        out[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
}

constexpr int BWD_WAVES = 4;

// The chunks in reverse.  A chunk's states are formed again from the state before it (kept by the forward pass) and stay in registers with the
// factors a; then, from the last step on, with r_t = dy_t silu(z_t):
//   g_t = r_t C_t + a_{t+1} g_{t+1},  dB = sum_d g delta x,  dC = sum_d r h,  d(delta) = sum_s g a h_{t-1} A + x sum_s g B,  dA = sum_t g a h_{t-1} delta
// dB and dC of a workgroup's channels are added in LDS in a fixed order and leave as a partial sum a workgroup; dA, dskip and ddt_bias stay in
// registers for the whole sequence.  At an episode's first step the products with a are 0, also where the other factor is not finite.
// ABSENT: there are states beyond S or channels beyond a group's last
template <typename T, int SL, bool WIDE, bool ABSENT>
__global__ __launch_bounds__(64 * BWD_WAVES, 2) void scan_backward_kernel(const ScanOp p, const Places at, const Segments seg, const int blocks, float *pair_part, float *param_part)
{
    typedef Back<SL> H;
    typedef Swap<H> X;
    constexpr int L = H::L, NB = H::NB, SP = H::SP, PAIR = H::PAIR, THREADS = 64 * BWD_WAVES;
    __shared__ __attribute__((aligned(16))) float pairs[2][L * PAIR];
    __shared__ __attribute__((aligned(16))) float sums[2][BWD_WAVES][L * PAIR];
    __shared__ __attribute__((aligned(16))) float swaps[BWD_WAVES][6 * X::SIZE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane & 3, own = lane >> 2;
    const int block = blockIdx.x % blocks, g = blockIdx.x / blocks % p.d.G, nk = blockIdx.x / blocks / p.d.G, n = nk % p.d.N, k = nk / p.d.N;
    const int c = (block * BWD_WAVES + wave) * 16, D = p.d.D, S = p.d.S, TT = p.d.T, len = length_of(p.in.lengths, n, TT);
    const bool on = c + own < at.per_group;
    const int d0 = g * at.per_group + c, d = d0 + own;
    // the segment's chunks; beyond `top` they have no steps
    const int lowest = k * seg.steps / L, highest = (min(TT, (k + 1) * seg.steps) + L - 1) / L - 1, top = min(highest, len > lowest * L ? (len - 1) / L : lowest - 1), last = top * L;
    Cell<H> cell;
    cell.open(lane, at.per_group - c);
    Track<T, H, WIDE> xa, da, za, ga, dxa, dda, dza;
    xa.open(p.in.x, n, d0, cell, last); da.open(p.in.dt, n, d0, cell, last); za.open(p.in.z, n, d0, cell, last); ga.open(p.dy, n, d0, cell, last);
    dxa.open(p.g.dx, n, d0, cell, highest * L); dda.open(p.g.ddt, n, d0, cell, highest * L); dza.open(p.g.dz, n, d0, cell, highest * L);
    Kept<SL> kept;
    kept.open(p.states, p.d.N, n, D, d0, d, q, top);
    float skip[NB], bias[NB], dskip[NB], dbias[NB];
#pragma unroll
    for (int e = 0; e < NB; ++e) {
        const bool some = e < cell.count;
        skip[e] = some && p.in.skip ? p.in.skip[d0 + cell.channel + e] : 0.0f;
        bias[e] = some && p.in.dt_bias ? p.in.dt_bias[d0 + cell.channel + e] : 0.0f;
        dskip[e] = dbias[e] = 0.0f;
    }
    float A[SL], ag[SL], dA[SL];
#pragma unroll
    for (int s = 0; s < SL; ++s) {
        const int i = q * SL + s;
        A[s] = on && i < S ? p.in.A[(int64_t)d * S + i] * LOG2E : 0.0f;
        ag[s] = on && i < S && p.dh_out && k == seg.count - 1 ? p.dh_out[((int64_t)n * D + d) * S + i] : 0.0f;
        dA[s] = 0.0f;
    }
    if (on && k < seg.count - 1) {
        read_states<SL>(ag, seg.state + state_at<SL>((int64_t)(seg.count - 1) * p.d.N + n, d, D, q));
        over_segments<SL>(ag, seg, seg.count - 2, k, -1, n, p.d.N, d, D, q, A);
    }
    // the workgroup's first wavefront brings B, its second C
    Half<T, H, WIDE> ps;
    ps.open(wave == 1 ? p.in.C : p.in.B, n, g, S, lane, last);
    if (wave > 1) ps.lane = NOWHERE, ps.count = 0;
    Begins<L> begins;
    begins.open(p.in.starts, n, p.d.N, lane, last);
    struct { Raw<T, NB, WIDE> x, dt, z, dy; Raw<T, 4, WIDE> pair; uint32_t begins; float h[SL]; } in;
    auto fetch = [&](int chunk) {          // (there is nothing to load before the segment's first chunk)
        __builtin_amdgcn_sched_barrier(0);
        const int t0 = chunk * L, live = chunk >= lowest ? len : t0;
        const bool some = t0 + cell.step < live;
        begins.load(in.begins, t0, live, lane);
        xa.load(in.x, some, cell);
        da.load(in.dt, some, cell);
        ga.load(in.dy, some, cell);
        za.load(in.z, some, cell);
        ps.load(in.pair, t0, live);
        kept.load(in.h, on && chunk >= lowest);
        xa.back(); da.back(); za.back(); ga.back(); ps.back(); begins.back(); kept.back();
        __builtin_amdgcn_sched_barrier(0);
    };
    // the workgroup's sums of a chunk: a thread has two neighbouring ones of a step
    static_assert(L * PAIR <= 2 * THREADS, "sums");
    const int mine = 2 * tid / PAIR;
    float *leaves = pair_part + ((((int64_t)block * TT + mine) * p.d.N + n) * p.d.G + g) * PAIR + 2 * tid % PAIR;
    const int64_t row = (int64_t)p.d.N * p.d.G * PAIR;
    auto leave = [&](int chunk, int buf) {
        if (mine >= L || chunk * L + mine >= TT) return;
        float a = 0.0f, b = 0.0f;
#pragma unroll
        for (int w = 0; w < BWD_WAVES; ++w) { a += sums[buf][w][2 * tid]; b += sums[buf][w][2 * tid + 1]; }
        float *to = leaves + chunk * (L * row);
        to[0] = a; to[1] = b;
    };
    float *sizes = swaps[wave], *moves = sizes + X::SIZE, *rs = moves + X::SIZE, *raws = rs + X::SIZE, *sBs = raws + X::SIZE, *sds = sBs + X::SIZE;
    const int share = (2 * (lane >> 3 & 1) + (lane >> 2 & 1)) * PAIR + (lane >> 4 & 1) * SP + q * SL + (lane >> 5) * (SL / 2);
    for (int chunk = highest; chunk > top; --chunk) {
        float none[NB];
#pragma unroll
        for (int e = 0; e < NB; ++e) none[e] = 0.0f;
        const bool there = chunk * L + cell.step < TT;
        dxa.store(none, there, cell);
        dda.store(none, there, cell);
        dza.store(none, there, cell);
        dxa.back(); dda.back(); dza.back();
        if (mine < L && chunk * L + mine < TT) {
            float *to = leaves + chunk * (L * row);
            to[0] = to[1] = 0.0f;
        }
    }
    fetch(top);
    for (int chunk = top, buf = 0; chunk >= lowest; --chunk, buf ^= 1) {
        const int t0 = chunk * L;
        const bool some = t0 + cell.step < len;
        if (wave < 2) ps.put(in.pair, pairs[buf] + wave * SP);
        float zero = 0.0f;
        float xv[NB], size[NB], slope[NB], r[NB], zf[NB], hb[SL];
        {
            float moved[NB];
#pragma unroll
            for (int e = 0; e < NB; ++e) {
                xv[e] = in.x[e];
                const float v = in.dt[e] + bias[e];
                float soft, rise;
                softplus_f(v, soft, rise);
                size[e] = some ? p.d.softplus ? soft : v : 0.0f;
                slope[e] = some ? p.d.softplus ? rise : 1.0f : 0.0f;
                moved[e] = size[e] * xv[e];
                const float dy = in.dy[e], z = in.z[e], open = act_f<HTS_ACT_SILU>(z);
                r[e] = dy * (p.in.z.p ? open : 1.0f);
                if (ABSENT) {
                    look(zero, moved[e]);
                    look(zero, r[e]);
                }
                zf[e] = dy * act_slope<HTS_ACT_SILU>(z);
            }
            X::put(sizes, cell, size);
            X::put(moves, cell, moved);
            X::put(rs, cell, r);
        }
#pragma unroll
        for (int s = 0; s < SL; ++s) hb[s] = in.h[s];
        const uint32_t fresh = Begins<L>::mask(in.begins);
        lds_barrier();
        fetch(chunk - 1);
        if (chunk < top) leave(chunk + 1, buf ^ 1);
        const float *lds = pairs[buf];
        // states beyond S meet what is their channel's, absent channels B and C, which are every channel's
        if (ABSENT && c + 16 > at.per_group)
#pragma unroll
            for (int i = 0; i < L * PAIR; i += 64) look(zero, lds[i + lane]);
        const int steps = len - t0;                                     // that there are, of the chunk's
        auto pass = [&](auto kind) {
            constexpr bool FRESH = decltype(kind)::value > 0, ODD = decltype(kind)::value > 1;
            const int exist = ABSENT && ODD ? states_of<SL>(S, q, on) : SL;
            // (fences between four steps and the next: mixed, they take more registers than two wavefronts a SIMD have; 145 -> 123 us with the shares of dA)
            float a[L][SL], h[L][SL];
            {
                Ahead<H, true> ahead(lds + q * SL);
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    __builtin_amdgcn_sched_barrier(0);
                    const f32x4 de = X::four(sizes, own, j), dx = X::four(moves, own, j);
                    float part[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = 4 * j + i;
                        ahead.next(t, +1);
                        const bool begin = FRESH && (fresh >> t & 1);
                        float sum = 0.0f;
#pragma unroll
                        for (int s = 0; s < SL; ++s) {
                            a[t][s] = __builtin_amdgcn_exp2f(de[i] * A[s]);
                            h[t][s] = __builtin_fmaf(a[t][s], begin ? 0.0f : t ? h[t ? t - 1 : 0][s] : hb[s], dx[i] * ahead.B(t)[s]);
                            if (ODD && s >= exist) h[t][s] = 0.0f;
                            sum = __builtin_fmaf(h[t][s], ahead.C(t)[s], sum);
                        }
                        part[i] = sum;
                    }
                    raws[own * X::PITCH + 4 * j + q] = quad_deal(part, q);
                }
            }
            Ahead<H, true> ahead(lds + q * SL);
#pragma unroll
            for (int j = NB - 1; j >= 0; --j) {
                __builtin_amdgcn_sched_barrier(0);
                const f32x4 de = X::four(sizes, own, j), dx = X::four(moves, own, j), rk = X::four(rs, own, j);
                float gB[4], dd[4], val[8 * SL];
#pragma unroll
                for (int i = 3; i >= 0; --i) {
                    const int t = 4 * j + i;
                    ahead.next(t, -1);
                    const bool begin = FRESH && (fresh >> t & 1);
                    gB[i] = dd[i] = 0.0f;
#pragma unroll
                    for (int s = 0; s < SL; ++s) {
                        // (of h only the steps before are read)
                        const bool no = ODD && s >= exist, none = no || (ODD && t >= steps);
                        const float gk = __builtin_fmaf(rk[i], ahead.C(t)[s], ag[s]);
                        val[2 * SL * i + s] = none ? 0.0f : gk * dx[i];
                        val[2 * SL * i + SL + s] = none ? 0.0f : rk[i] * h[t][s];
                        gB[i] = no ? gB[i] : __builtin_fmaf(gk, ahead.B(t)[s], gB[i]);
                        const float back = begin ? 0.0f : a[t][s] * gk, ga = begin || none ? 0.0f : back * (t ? h[t ? t - 1 : 0][s] : hb[s]);
                        ag[s] = none ? ag[s] : back;
                        dd[i] = no ? dd[i] : __builtin_fmaf(ga, A[s], dd[i]);
                        dA[s] = no ? dA[s] : __builtin_fmaf(ga, de[i], dA[s]);
                        asm volatile("" : "+v"(dA[s]));          // (here and now: left to the compiler, a chunk's shares wait for its end, with all their factors)
                    }
                }
                // a lane's sums: step 4 j + 2 bit3 + bit2, B or C by bit 4, half of its quad's states by bit 5
                float out[SL / 2];
                channel_sums<8 * SL>(out, val);
                float *to = sums[buf][wave] + 4 * j * PAIR + share;
#pragma unroll
                for (int s = 0; s < SL / 2; ++s) to[s] = out[s];
                sBs[own * X::PITCH + 4 * j + q] = quad_deal(gB, q);
                sds[own * X::PITCH + 4 * j + q] = quad_deal(dd, q);
            }
        };
        by_kind<false>(pass, fresh, steps < L || (ABSENT && __ballot(zero != zero)));
        wave_order();
        float raw[NB], sB[NB], sd[NB], dx[NB], ddt[NB], dz[NB];
        X::get(raw, raws, cell);
        X::get(sB, sBs, cell);
        X::get(sd, sds, cell);
#pragma unroll
        for (int e = 0; e < NB; ++e) {
            ddt[e] = __builtin_fmaf(sB[e], xv[e], sd[e] * (1.0f / LOG2E)) * slope[e];
            dx[e] = some ? __builtin_fmaf(sB[e], size[e], r[e] * skip[e]) : 0.0f;
            dz[e] = some ? zf[e] * __builtin_fmaf(skip[e], xv[e], raw[e]) : 0.0f;
            ddt[e] = some ? ddt[e] : 0.0f;
            dbias[e] += ddt[e];
            dskip[e] = __builtin_fmaf(r[e], xv[e], dskip[e]);
        }
        const bool there = t0 + cell.step < TT;
        dxa.store(dx, there, cell);
        dda.store(ddt, there, cell);
        dza.store(dz, there, cell);
        dxa.back(); dda.back(); dza.back();
        wave_order();
    }
    lds_barrier();
    if (top >= lowest) leave(lowest, (top - lowest) & 1);
    float *out = param_part + (int64_t)nk * D * (S + 2);
    if (on)
#pragma unroll
        for (int s = 0; s < SL; ++s)
            if (q * SL + s < S) {
                out[(int64_t)d * S + q * SL + s] = dA[s];
                if (p.g.dh_in && k == 0) p.g.dh_in[((int64_t)n * D + d) * S + q * SL + s] = ag[s];
            }
    // over the chunk's steps, which are other lanes
#pragma unroll
    for (int e = 0; e < NB; ++e) {
#pragma unroll
        for (int m = Cell<H>::PER; m < 64; m *= 2) { dskip[e] += __shfl_xor(dskip[e], m); dbias[e] += __shfl_xor(dbias[e], m); }
        if (cell.step == 0 && e < cell.count) { out[(int64_t)D * S + d0 + cell.channel + e] = dskip[e]; out[(int64_t)D * (S + 1) + d0 + cell.channel + e] = dbias[e]; }
    }
}

// The first pass over segments, from the last to the second: the gradient that a segment's own outputs (and, the last one, dh_out) give to the state
// before it
template <typename T, int SL, bool WIDE, bool ABSENT>
__global__ __launch_bounds__(64 * FWD_WAVES) void scan_adjoint_kernel(const ScanOp p, const Places at, const Segments seg)
{
    typedef Forth<SL> H;
    typedef Swap<H> X;
    constexpr int L = H::L, NB = H::NB, SP = H::SP;
    __shared__ __attribute__((aligned(16))) float shared[FWD_WAVES][L * H::PAIR + 2 * X::SIZE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), D = p.d.D, S = p.d.S, N = p.d.N;
    const int per = at.waves * p.d.G;
    const uint32_t task = blockIdx.x * FWD_WAVES + wave, row = task / per, in_row = task % per;
    if (row >= (uint32_t)(N * (seg.count - 1))) return;
    const int k = row / N + 1, n = row % N, g = in_row / at.waves, c = in_row % at.waves * 16, q = lane & 3, own = lane >> 2;
    const int d0 = g * at.per_group + c, d = d0 + own, len = length_of(p.in.lengths, n, p.d.T);
    const bool on = c + own < at.per_group;
    const int first = k * seg.steps, last = len > first ? (min(len, first + seg.steps) + L - 1) / L * L - L : first - L;          // the last chunk with steps
    Cell<H> cell;
    cell.open(lane, at.per_group - c);
    Track<T, H, WIDE> da, za, ga;
    da.open(p.in.dt, n, d0, cell, last); za.open(p.in.z, n, d0, cell, last); ga.open(p.dy, n, d0, cell, last);
    float bias[NB], sum[NB];
#pragma unroll
    for (int e = 0; e < NB; ++e) {
        bias[e] = e < cell.count && p.in.dt_bias ? p.in.dt_bias[d0 + cell.channel + e] : 0.0f;
        sum[e] = 0.0f;
    }
    float A[SL], ag[SL];
    bool cut = false;
#pragma unroll
    for (int s = 0; s < SL; ++s) {
        const int i = q * SL + s;
        A[s] = on && i < S ? p.in.A[(int64_t)d * S + i] * LOG2E : 0.0f;
        ag[s] = on && i < S && p.dh_out && k == seg.count - 1 ? p.dh_out[((int64_t)n * D + d) * S + i] : 0.0f;
    }
    Half<T, H, WIDE> cs;
    Begins<L> begins;
    cs.open(p.in.C, n, g, S, lane, last);
    begins.open(p.in.starts, n, N, lane, last);
    struct { Raw<T, NB, WIDE> dt, z, dy; Raw<T, 4, WIDE> c; uint32_t begins; } in;
    auto fetch = [&](int t0) {
        __builtin_amdgcn_sched_barrier(0);
        const int live = t0 >= first ? len : t0;
        const bool some = t0 + cell.step < live;
        begins.load(in.begins, t0, live, lane);
        da.load(in.dt, some, cell);
        za.load(in.z, some, cell);
        ga.load(in.dy, some, cell);
        cs.load(in.c, t0, live);
        da.back(); za.back(); ga.back(); cs.back(); begins.back();
        __builtin_amdgcn_sched_barrier(0);
    };
    float *pairs = shared[wave], *sizes = pairs + L * H::PAIR, *rs = sizes + X::SIZE;
    fetch(last);
    for (int t0 = last; t0 >= first; t0 -= L) {
        const bool some = t0 + cell.step < len;
        float size[NB], r[NB], zero = 0.0f;
        wave_order();
        cs.put(in.c, pairs);
        const uint32_t fresh = Begins<L>::mask(in.begins);
#pragma unroll
        for (int e = 0; e < NB; ++e) {
            const float v = in.dt[e] + bias[e], open = act_f<HTS_ACT_SILU>(in.z[e]);
            float soft, slope;
            softplus_f(v, soft, slope);
            size[e] = some ? p.d.softplus ? soft : v : 0.0f;
            r[e] = in.dy[e] * (p.in.z.p ? open : 1.0f);
            if (ABSENT) {
                look(zero, r[e]);
                look(zero, size[e]);
            }
            sum[e] += size[e];
        }
        X::put(sizes, cell, size);
        X::put(rs, cell, r);
        cut |= fresh != 0;
        wave_order();
        fetch(t0 - L);
        const int steps = len - t0;
        auto pass = [&](auto kind) {
            constexpr bool FRESH = decltype(kind)::value > 0, ODD = decltype(kind)::value > 1;
            const int exist = ABSENT && ODD ? states_of<SL>(S, q, on) : SL;
            Ahead<H, false> ahead(pairs + q * SL);
#pragma unroll
            for (int j = NB - 1; j >= 0; --j) {
                const f32x4 de = X::four(sizes, own, j), rk = X::four(rs, own, j);
#pragma unroll
                for (int i = 3; i >= 0; --i) {
                    const int t = 4 * j + i;
                    ahead.next(t, -1);
                    const bool begin = FRESH && (fresh >> t & 1);
#pragma unroll
                    for (int s = 0; s < SL; ++s) {
                        const bool none = ODD && (t >= steps || s >= exist);
                        const float gk = __builtin_fmaf(rk[i], ahead.B(t)[s], ag[s]), back = begin ? 0.0f : __builtin_amdgcn_exp2f(de[i] * A[s]) * gk;
                        ag[s] = none ? ag[s] : back;
                    }
                }
            }
        };
        by_kind<true>(pass, fresh, steps < L || (ABSENT && __ballot(zero != zero)));
    }
    if (on) {
        float *out = seg.state + state_at<SL>((int64_t)k * N + n, d, D, q);
#pragma unroll
        for (int s = 0; s < SL; ++s) out[s] = ag[s];
    }
#pragma unroll
    for (int e = 0; e < NB; ++e) {
#pragma unroll
        for (int m = Cell<H>::PER; m < 64; m *= 2) sum[e] += __shfl_xor(sum[e], m);
        if (cell.step == 0 && e < cell.count) seg.sum[((int64_t)k * N + n) * D + d0 + cell.channel + e] = cut ? __builtin_nanf("") : sum[e];
    }
}

// dB and dC from the workgroups' sums, and, by the workgroups after those, dA, dskip and ddt_bias from the sequences' (one launch: 2 us less than two)
template <typename T>
__global__ __launch_bounds__(256) void sums_kernel(const ScanOp p, const int blocks, const int SP, const float *part, const int64_t pair_groups, const float *params, const int64_t rows)
{
    if (blockIdx.x >= pair_groups) {
        __shared__ float sums[4][64];
        const int64_t D = p.d.D, S = p.d.S;
        sum_partials<4>(sums, blockIdx.x - pair_groups, params, rows, D * (S + 2), SumTarget{p.g.dA, D * S}, SumTarget{p.g.dskip, D}, SumTarget{p.g.ddt_bias, D});
        return;
    }
    const int64_t width = (int64_t)p.d.T * p.d.N * p.d.G * 2 * SP, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= width) return;
    float s = 0.0f;
#pragma unroll 8
    for (int b = 0; b < blocks; ++b) s += part[b * width + i];
    const int r = (int)(i % (2 * SP)), k = r % SP;
    const int64_t at = i / (2 * SP), g = at % p.d.G, n = at / p.d.G % p.d.N, t = at / p.d.G / p.d.N;
    if (k >= p.d.S) return;
    const hts_steps &to = r < SP ? p.g.dB : p.g.dC;
    ((T *)to.p)[t * to.st + n * to.sn + g * p.d.S + k] = from_f32<T>(s);
}

Places places(const hts_scan_desc &d) { const int per = d.D / d.G; return Places{per, (int)ceil_div(per, 16)}; }
int blocks_of(const hts_scan_desc &d) { return (int)ceil_div(places(d).waves, BWD_WAVES); }

// Segments of a sequence: where its wavefronts leave units idle, as many as give two to a SIMD, of 32 steps or so at least, in whole chunks of either direction.
// Forward the first pass costs two thirds of the second and a launch, so that up to three segments gain nothing; backward a fifth, and a lone wavefront
// waits for itself a third of its time.  129 steps of 5 sequences of 330 channels in binary32, five segments (segments of 64 steps at least: one and
// two): forward 18.9 us, backward 30.9 (before these kernels looked for infinities 19.7 and 28.2, with one and two segments 25.0 and 46.2).  (On fewer compute units than 256 there are fewer segments: the workspace is for those.)
constexpr int MOST_SEGMENTS = 64, LEAST_STEPS = 24;        // (before they are made whole chunks)
int segments_of(const hts_scan_desc &d, int cus, bool backward)
{
    const int64_t waves = (int64_t)places(d).waves * d.G * d.N, units = 4ll * (cus < 256 ? cus : 256);
    int64_t count = 2 * units / waves;
    if (count > d.T / LEAST_STEPS) count = d.T / LEAST_STEPS;
    if (count > MOST_SEGMENTS) count = MOST_SEGMENTS;
    if (count < (!backward ? 4 : d.T < 128 ? 3 : 2)) return 1;
    return (int)ceil_div(d.T, round_up(ceil_div(d.T, count), 16));
}
Segments segments(const hts_scan_desc &d, int cus, bool backward)
{
    Segments seg = {};
    seg.count = segments_of(d, cus, backward);
    seg.steps = (int)round_up(ceil_div(d.T, seg.count), 16);
    return seg;
}
struct Layout { int64_t h_in, state, sum, pairs, params, total; };      // floats
Layout layout(const hts_scan_desc &d, const Segments &seg, bool backward)
{
    const int64_t held = (int64_t)d.N * d.D * padded(d.S), some = seg.count > 1;
    Layout l;
    l.h_in = 0;
    l.state = l.h_in + (backward ? 0 : some * held);
    l.sum = l.state + some * held * seg.count;
    l.pairs = l.sum + some * round_up((int64_t)seg.count * d.N * d.D, 64);
    l.params = l.pairs + (backward ? round_up((int64_t)blocks_of(d) * d.T * d.N * d.G * 2 * padded(d.S), 64) : 0);
    l.total = l.params + (backward ? (int64_t)seg.count * d.N * d.D * (d.S + 2) : 0);
    return l;
}

// whether rows of these channels can be read four entries at a time
template <typename T> bool wide(const hts_steps &s, int64_t N, int64_t cols) { return !s.p || ((uintptr_t)s.p % (4 * sizeof(T)) == 0 && s.st % 4 == 0 && (N == 1 || s.sn % 4 == 0) && cols % 4 == 0); }
template <typename T> bool wide(const ScanOp &op, bool backward)
{
    const hts_scan_desc &d = op.d;
    bool w = wide<T>(op.in.B, d.N, d.S) && wide<T>(op.in.C, d.N, d.S);
    for (const hts_steps *s : {&op.in.x, &op.in.dt, &op.in.z}) w = w && wide<T>(*s, d.N, d.D / d.G);
    if (!backward) return w && wide<T>(op.y, d.N, d.D / d.G);
    for (const hts_steps *s : {&op.dy, &op.g.dx, &op.g.ddt, &op.g.dz}) w = w && wide<T>(*s, d.N, d.D / d.G);
    return w;
}

#define LAUNCH(KERNEL, GRID, THREADS, ...)                                                                                                                 \
    do {                                                                                                                                                  \
        hipLaunchKernelGGL(KERNEL, dim3((uint32_t)(GRID)), dim3(THREADS), 0, c.stream, __VA_ARGS__);                                                       \
        const hipError_t e_ = hipGetLastError();                                                                                                          \
        if (e_ != hipSuccess) return e_;                                                                                                                  \
    } while (0)

template <typename T, int SL, bool WIDE, bool ABSENT> hipError_t scan(hts_seq_ctx &c, const ScanOp &op)
{
    const Places at = places(op.d);
    Segments seg = segments(op.d, c.cus, false);
    const Layout l = layout(op.d, seg, false);
    const int64_t waves = (int64_t)at.waves * op.d.G * op.d.N;
    seg.h_in = (float *)c.ws + l.h_in; seg.state = (float *)c.ws + l.state; seg.sum = (float *)c.ws + l.sum;
    if (!launchable(ceil_div(waves * seg.count, FWD_WAVES), 64 * FWD_WAVES)) return hipErrorInvalidConfiguration;
    if (seg.count > 1) LAUNCH((scan_kernel<T, SL, WIDE, ABSENT, true>), ceil_div(waves * (seg.count - 1), FWD_WAVES), 64 * FWD_WAVES, op, at, seg);
    LAUNCH((scan_kernel<T, SL, WIDE, ABSENT, false>), ceil_div(waves * seg.count, FWD_WAVES), 64 * FWD_WAVES, op, at, seg);
    return hipSuccess;
}

template <typename T, int SL, bool WIDE, bool ABSENT> hipError_t scan_backward(hts_seq_ctx &c, const ScanOp &op)
{
    const Places at = places(op.d);
    Segments seg = segments(op.d, c.cus, true);
    const Layout l = layout(op.d, seg, true);
    const int64_t waves = (int64_t)at.waves * op.d.G * op.d.N, width = (int64_t)op.d.T * op.d.N * op.d.G * 8 * SL, D = op.d.D;
    const int blocks = blocks_of(op.d);
    float *pairs = (float *)c.ws + l.pairs, *params = (float *)c.ws + l.params;
    seg.state = (float *)c.ws + l.state; seg.sum = (float *)c.ws + l.sum;
    const int64_t pair_groups = ceil_div(width, 256), sum_groups = pair_groups + ceil_div(D * (op.d.S + 2), 64), workgroups = (int64_t)blocks * op.d.G * op.d.N * seg.count;
    if (!launchable(workgroups, 64 * BWD_WAVES) || !launchable(sum_groups, 256)) return hipErrorInvalidConfiguration;
    if (seg.count > 1) LAUNCH((scan_adjoint_kernel<T, SL, WIDE, ABSENT>), ceil_div(waves * (seg.count - 1), FWD_WAVES), 64 * FWD_WAVES, op, at, seg);
    LAUNCH((scan_backward_kernel<T, SL, WIDE, ABSENT>), workgroups, 64 * BWD_WAVES, op, at, seg, blocks, pairs, params);
    LAUNCH((sums_kernel<T>), sum_groups, 256, op, blocks, 4 * SL, pairs, pair_groups, params, (int64_t)op.d.N * seg.count);
    return hipSuccess;
}

template <typename T, int SL> hipError_t run(hts_seq_ctx &c, const ScanOp &op, bool backward)
{
    // kernels that look for infinities where there are states or channels that do not exist: others have no use for it (512 x 16 both ways 206 us, looking 214; of
    // more than 32 states there are these alone)
    const bool states = SL == 16 || op.d.S < 4 * SL, absent = states || places(op.d).per_group % (16 * BWD_WAVES) != 0;
    if (backward) {
        if (absent) return wide<T>(op, true) ? scan_backward<T, SL, true, true>(c, op) : scan_backward<T, SL, false, true>(c, op);
        return wide<T>(op, true) ? scan_backward<T, SL, true, SL == 16>(c, op) : scan_backward<T, SL, false, SL == 16>(c, op);
    }
    if (op.d.T > 1) {
        if (states) return wide<T>(op, false) ? scan<T, SL, true, true>(c, op) : scan<T, SL, false, true>(c, op);
        return wide<T>(op, false) ? scan<T, SL, true, SL == 16>(c, op) : scan<T, SL, false, SL == 16>(c, op);
    }
    if (!launchable(ceil_div((int64_t)op.d.N * op.d.D, 64), 256)) return hipErrorInvalidConfiguration;
    LAUNCH((step_kernel<T, SL>), ceil_div((int64_t)op.d.N * op.d.D, 64), 256, op);
    return hipSuccess;
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

int64_t scan_states(const hts_scan_desc &d) { return ceil_div(d.T, back_steps(d.S)) * d.N * d.D * padded(d.S); }
// Enough for every shape of no more steps and sequences: fewer sequences are cut into more segments, at most two wavefronts a SIMD in all
int64_t scan_workspace(const hts_scan_desc &d, bool backward)
{
    const int64_t most = std::min<int64_t>(std::min<int64_t>(d.T / LEAST_STEPS, MOST_SEGMENTS) * d.N, 2048 / ((int64_t)places(d).waves * d.G)), rows = std::max<int64_t>(d.N, most);
    const int64_t held = (int64_t)d.D * padded(d.S), cut = most > 1 ? (most + (backward ? 0 : std::min<int64_t>(d.N, most))) * held + round_up(most * d.D, 64) : 0;
    return 4 * (cut + (backward ? round_up((int64_t)blocks_of(d) * d.T * d.N * d.G * 2 * padded(d.S), 64) + rows * d.D * (d.S + 2) : 0));
}
hipError_t launch_scan(hts_seq_ctx &c, const ScanOp &op) { return op.d.precision == HTS_PRECISION_BF16 ? by_states<bf16_t>(c, op, false) : by_states<float>(c, op, false); }
hipError_t launch_scan_backward(hts_seq_ctx &c, const ScanOp &op) { return op.d.precision == HTS_PRECISION_BF16 ? by_states<bf16_t>(c, op, true) : by_states<float>(c, op, true); }

}  // namespace hts
