// The gated delta rule and its gradients (see include/hts.h).
//
// Step by step, with al = exp(delta A), be = 1 / (1 + exp(-b)), k and q of length one (or as they are):
//   z = v - al S^T k,  S <- al S + be k z^T,  y = scale S^T q.
// Up to 64 steps of a chunk at a time, S the state before it, G[i][j] = the product of the decays of steps j + 1 .. i (0 where an episode begins among them),
// kept[i] that of steps 0 .. i, left[j] that of steps j + 1 .. to the end, M = (k_i . k_j) G[i][j] below the diagonal:
//   Z = (I + M diag(be))^-1 (V - kept K S),  U = be Z,  Y = scale (kept Q S + (Q K^T G) U),  S' = kept[end] S + K^T (left U).
// The gradients, dS' being the state's at the chunk's end, W the inverse above:
//   dU = (Q K^T G)^T dY + left K dS',  dV = W^T (be dU),  dS = kept[end] dS' + Q^T (kept dY) - K^T (kept dV)
//   dQ = kept dY S^T + (dY U^T G) K,  dK = left U dS'^T - kept dV S^T + (dY U^T G)^T Q - X K - X^T K,  X = dV U^T G below the diagonal
//   db = (1 - be) Z . dV,  and the logarithm of a step's decay has what passes it: all that goes from before it (earlier steps, S) to it and what is after.
//
// Three kinds of kernels: what needs the chunk's own steps only (prep: every chunk at a time), what goes from chunk to chunk (forward, reverse: 32 of the values'
// entries of a head at a time, whose states never meet), and the gradients that sum over the values (grads: every chunk at a time again).
// (The chunked form is the published one of Yang, Wang, Zhang, Shen and Kim, "Parallelizing Linear Transformers with the Delta Rule over Sequence Length", 2024, the decays those of
// Yang, Kautz and Hatamizadeh, "Gated Delta Networks", 2024; the derivations here are from the rule above.)
#include "delta.hpp"

namespace hts {
namespace {

constexpr int TILE = 32;                  // the values' entries of a workgroup
constexpr int ROOM = 256;                 // workgroups that segments are made for, and the most of them
__host__ __device__ __forceinline__ int keys_padded(int K) { return K <= 32 ? 32 : K <= 64 ? 64 : 128; }

// sums over as many neighbouring lanes as a row of eights has
template <int LANES> __device__ __forceinline__ float add_row(float x)
{
    x = add_moved<0x4E>(add_moved<0xB1>(x));
    if constexpr (LANES >= 8) x = add_moved<0x141>(x);
    if constexpr (LANES >= 16) x = add_moved<0x140>(x);
    return x;
}

__device__ __forceinline__ float sizes_of(const f32x4 &x) { return (__builtin_fabsf(x[0]) + __builtin_fabsf(x[1])) + (__builtin_fabsf(x[2]) + __builtin_fabsf(x[3])); }
struct Decay { float delta, slope, exponent; };       // exponent: of 2
__device__ __forceinline__ Decay decay_of(float x, float bias, float A, int softplus)
{
    Decay r;
    x += bias;
    r.delta = x; r.slope = 1.0f;
    if (softplus) softplus_f(x, r.delta, r.slope);
    r.exponent = r.delta * A;
    return r;
}
// below this (in exponents of 2) nothing of binary32 is left: the step forgets
constexpr double FORGETS = -150.0;
constexpr double LOG2E_64 = 1.4426950408889634074;

// tiles of 16 x 16 steps on and below the diagonal
constexpr int PAIRS = 10;
__device__ __forceinline__ int pair_of(int back, int seen) { return back * (back + 1) / 2 + seen; }

// ---- what needs the chunk's steps only --------------------------------------------------------------------------------
// A workgroup for a chunk of a head.  What leaves is in the order that the kernels after it take it in (fragments in lane order, read in whole lines).  Bound by the latency of its
// dependent phases (gates, lengths, products, substitution in blocks of 16, two levels of products), with three workgroups a unit to overlap them: 1024 chunks of 128 keys in bf16
// 38 us, 18 MB read and 63 MB written (101 MB for the backward call); 90 chunks of 37 in binary32 17.
template <typename T, int KP> struct PrepLds {
    static constexpr int PITCH = Num<T>::exact_pitch(KP), LINE = 65;
    static constexpr int FAR = 0, EPISODE = FAR + 8 * CHUNK, STRENGTH = EPISODE + 4 * CHUNK, Q = STRENGTH + 4 * CHUNK, K = Q + 4 * CHUNK, BAD = K + 4 * CHUNK;
    static constexpr int BELOW = BAD + 64, KEYS = BELOW + 4 * CHUNK * LINE, QUERIES = KEYS + CHUNK * PITCH, INVERSE = KEYS, HALF = INVERSE + 4 * CHUNK * LINE;  // (the keys have left by then)
    static constexpr int BYTES = KEYS + (2 * CHUNK * PITCH > 4 * (CHUNK * LINE + 32 * 33) ? 2 * CHUNK * PITCH : 4 * (CHUNK * LINE + 32 * 33));
};

// C (16x16) = sum over n of A[row][k] B[k][col], binary32 from LDS
__device__ __forceinline__ f32x4 tile_product(const float *a, int lda, const float *b, int ldb, int n, int col, int quad)
{
    f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < n; k += 4) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[col * lda + k + quad], b[(k + quad) * ldb + col], c, 0, 0, 0);
    return c;
}

template <typename T, int KP, bool BACK> __global__ __launch_bounds__(256) void prep_kernel(const DeltaArgs a)
{
    typedef PrepLds<T, KP> L;
    typedef Num<T> N_;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const hts_delta_rule_desc &d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quad = lane >> 4;
    const int64_t unit = blockIdx.x;
    const int h = (int)(unit % d.H), n = (int)(unit / d.H % d.N), c = (int)(unit / d.H / d.N), t0 = c * CHUNK, len = length_of(a, n);
    if (t0 >= len) return;
    const int K = d.K, group = h / (d.H / d.G);
    double *far = (double *)(lds + L::FAR);
    int *episode = (int *)(lds + L::EPISODE);
    float *strength = (float *)(lds + L::STRENGTH), *q_unit = (float *)(lds + L::Q), *k_unit = (float *)(lds + L::K);
    uint32_t *bad = (uint32_t *)(lds + L::BAD);                     // [2] keys, and rows of the matrix; [2] queries
    float *below = (float *)(lds + L::BELOW), *inverse = (float *)(lds + L::INVERSE), *half = (float *)(lds + L::HALF);
    Gates &gates = a.gates[unit];

    uint64_t gates_bad = 0, resets = 0;
    if (wave == 0) {
        const int t = t0 + lane;
        const bool live = t < len;
        float be = 0.0f, rest = 0.0f;
        double e = 0.0;
        bool reset = false, wrong = false;
        if (live) {
            const Decay dc = decay_of(to_f32(step_of<T>(a.in.a, t, n)[h]), a.in.a_bias ? a.in.a_bias[h] : 0.0f, a.in.A[h], d.softplus);
            const float b = to_f32(step_of<T>(a.in.b, t, n)[h]);
            be = sigmoid_f(b);
            if constexpr (BACK) rest = sigmoid_f(-b);
            e = (double)dc.exponent * LOG2E_64;
            const bool start = a.in.starts && a.in.starts[(int64_t)t * d.N + n];          // (has no decay, whatever its input)
            wrong = !finite(be) || (!start && !(e < MOST_EXPONENT));
            reset = start || (e < FORGETS && !wrong);          // (a step that is wrong is marked, also for the ones before it, which its state's gradient goes to)
            if (wrong) be = 0.0f;
            if (reset || wrong) e = 0.0;
        }
        resets = __ballot(reset);
        gates_bad = __ballot(wrong);
        const uint64_t upto = resets & (~0ull >> (63 - lane));
        const int ep = __popcll(upto), last = __popcll(resets), first = upto ? 63 - __clzll(upto) : 0;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double x = __shfl_up(e, o, 64);
            if (lane >= o) e += x;
        }
        const double end = __shfl(e, 63, 64);
        far[lane] = e; episode[lane] = ep; strength[lane] = be;
        gates.far[lane] = e; gates.strength[lane] = be; gates.episode[lane] = ep; gates.first[lane] = first;
        if constexpr (BACK) gates.rest[lane] = rest;
        gates.keep[lane] = ep == 0 ? exp2_wide(e) : -1.0f;
        gates.left[lane] = ep == last ? exp2_wide(end - e) : -1.0f;
    }
    // rows of keys and queries, zeros for those that are not finite, and their lengths: a thread has 8 entries of a row at a time
    char *keys = lds + L::KEYS, *queries = lds + L::QUERIES;
    constexpr int EIGHTS = KP / 8, TIMES = CHUNK * EIGHTS / 256, ROWS = 256 / EIGHTS;
    T kx[TIMES][8], qx[TIMES][8];
    const int my_at = 8 * (tid % EIGHTS);
#pragma unroll
    for (int i = 0; i < TIMES; ++i) {
        const int t = t0 + i * ROWS + tid / EIGHTS;
        row8(kx[i], t < len ? step_of<T>(a.in.k, t, n) + (int64_t)group * K : nullptr, my_at, K);
        row8(qx[i], t < len ? step_of<T>(a.in.q, t, n) + (int64_t)group * K : nullptr, my_at, K);
    }
    if (tid < 16) bad[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TIMES; ++i) {
        const int row = i * ROWS + tid / EIGHTS;
        float ks = 0.0f, qs = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            ks = __builtin_fmaf(to_f32(kx[i][e]), to_f32(kx[i][e]), ks);
            qs = __builtin_fmaf(to_f32(qx[i][e]), to_f32(qx[i][e]), qs);
        }
        ks = add_row<EIGHTS>(ks); qs = add_row<EIGHTS>(qs);
        const bool k_wrong = !finite(ks), q_wrong = !finite(qs);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (k_wrong) kx[i][e] = from_f32<T>(0.0f);
            if (q_wrong) qx[i][e] = from_f32<T>(0.0f);
        }
        put_exact<T>(keys + row * L::PITCH + my_at / 8 * N_::EXACT, 16, make_exact<T>(kx[i]));
        put_exact<T>(queries + row * L::PITCH + my_at / 8 * N_::EXACT, 16, make_exact<T>(qx[i]));
        if (my_at == 0) {
            k_unit[row] = gates.k_unit[row] = d.normalize && !k_wrong ? 1.0f / __builtin_sqrtf(ks + 1e-6f) : 1.0f;
            q_unit[row] = gates.q_unit[row] = q_wrong ? __builtin_nanf("") : d.normalize ? 1.0f / __builtin_sqrtf(qs + 1e-6f) : 1.0f;
            if (k_wrong) atomicOr(&bad[row >> 5], 1u << (row & 31));
            if (q_wrong) atomicOr(&bad[2 + (row >> 5)], 1u << (row & 31));
        }
    }
    __syncthreads();

    // M diag(be) below the diagonal; Q K^T G
    {
        // A wavefront takes three of the ten tiles on and below the diagonal and of the two above it that fragments reach over.  i looks back at m: results are handed on along the
        // steps that are looked at (forward) or that look back (back).
        for (int tile = wave; tile < PAIRS + 2; tile += 4) {
            const int it = tile < 4 ? 3 : tile < 7 ? 2 : tile < 9 ? 1 : tile < 11 ? 0 : 2, jt = tile < 4 ? tile : tile < 7 ? tile - 4 : tile < 9 ? tile - 7 : tile == 9 ? 0 : tile == 10 ? 1 : 3;
            f32x4 kk = {0.0f, 0.0f, 0.0f, 0.0f}, qk = {0.0f, 0.0f, 0.0f, 0.0f};
            if (jt <= it)
#pragma unroll
                for (int s = 0; s < KP / 32; ++s) {
                    const int at = (4 * s + quad) * N_::EXACT;
                    const Exact<T> ki = get_exact<T>(keys + (16 * it + col) * L::PITCH + at, 16), kj = get_exact<T>(keys + (16 * jt + col) * L::PITCH + at, 16);
                    const Exact<T> qi = get_exact<T>(queries + (16 * it + col) * L::PITCH + at, 16);
                    if constexpr (BACK) { mma(kk, ki, kj); mma(qk, qi, kj); }
                    else { mma(kk, kj, ki); mma(qk, kj, qi); }
                }
            float p[4];
            Four<float> by_q, by_k;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = BACK ? 16 * it + 4 * quad + r : 16 * it + col, m = BACK ? 16 * jt + col : 16 * jt + 4 * quad + r;
                const bool sees = m <= i && episode[m] == episode[i];
                float x = 0.0f;
                p[r] = 0.0f;
                by_q.e[r] = qk[r] * (q_unit[i] * d.scale * k_unit[m]);
                by_k.e[r] = kk[r] * (k_unit[i] * k_unit[m]);
                if (sees) {
                    const float decay = exp2_wide(far[i] - far[m]);
                    p[r] = by_q.e[r] * decay;
                    if (m < i) x = by_k.e[r] * decay * strength[m];
                    if (!finite(x)) { atomicOr(&bad[i >> 5], 1u << (i & 31)); x = 0.0f; }
                }
                if (jt <= it) below[i * L::LINE + m] = x;
            }
            if constexpr (BACK)
                if (jt <= it) {
                    float *to = a.pairs + (unit * 2 * PAIRS + pair_of(it, jt)) * 256;
                    store_at(to, lane * 16, by_q);
                    store_at(to + PAIRS * 256, lane * 16, by_k);
                }
            // fragments of 16 rows and 32 entries: rows are the steps that look back (forward), those that are looked at (back)
            const int row = BACK ? 16 * jt + col : 16 * it + col, at = BACK ? 16 * it + 4 * quad : 16 * jt + 4 * quad;
            char *f = a.read + (unit * 8 + (row >> 4) * 2 + (at >> 5)) * N_::WIDE_FRAGMENT + ((at & 31) >> 3) * 256 + (row & 15) * 16;
            put_wide4<T>(f, 1024, (at >> 2) & 1, p);
        }
    }
    if (a.rows)
        for (int p = tid; p < CHUNK * KP / 8; p += 256) {
            const int row = p / (KP / 8), at = p % (KP / 8);
            T *to = (T *)a.rows + unit * 2 * CHUNK * KP + row * KP + 8 * at;
            const Exact<T> kx = get_exact<T>(keys + row * L::PITCH + at * N_::EXACT, 16), qx = get_exact<T>(queries + row * L::PITCH + at * N_::EXACT, 16);
            __builtin_memcpy(to, &kx, sizeof kx);
            __builtin_memcpy(to + CHUNK * KP, &qx, sizeof qx);
        }
    // keys (and queries) with the steps along a row
    for (int f = wave; f < KP / 16 * 2; f += 4) {
        const int row = 16 * (f >> 1) + col, at = 32 * (f & 1) + 8 * quad;
        T x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = *(const T *)(keys + (at + i) * L::PITCH + row * sizeof(T));
        put_exact<T>(a.keys + (unit * (KP / 8) + f) * N_::EXACT_FRAGMENT + lane * 16, 1024, make_exact<T>(x));
        if constexpr (BACK) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = *(const T *)(queries + (at + i) * L::PITCH + row * sizeof(T));
            put_exact<T>(a.queries + (unit * (KP / 8) + f) * N_::EXACT_FRAGMENT + lane * 16, 1024, make_exact<T>(x));
        }
    }
    __syncthreads();
    // the inverse: blocks of 16 on the diagonal by substitution, a column a lane; then those of 32 and the whole, W10 = -W11 M10 W00.  A step whose row leaves binary32 (by keys that lengthen
    // the state) is one that is not finite, and leaves nothing in the products: 0 times it would be NaN of other episodes
    const auto keep_finite = [&](float &x, int step) {
        if (finite(x)) return;
        atomicOr(&bad[step >> 5], 1u << (step & 31));
        x = 0.0f;
    };
    const auto keep_finite4 = [&](f32x4 &x, int step) {
        if (!finite(sizes_of(x)))
            for (int r = 0; r < 4; ++r) {
                float v = x[r];
                keep_finite(v, step + r);
                x[r] = v;
            }
    };
    if (lane < 16) {
        const float *m = below + 16 * wave * (L::LINE + 1);
        float x[16], sizes = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            x[r] = r == lane ? 1.0f : 0.0f;
#pragma unroll
            for (int k = 0; k < r; ++k) x[r] = __builtin_fmaf(-m[r * L::LINE + k], x[k], x[r]);
            sizes += __builtin_fabsf(x[r]);
        }
        if (!finite(sizes))                                    // again, row by row
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[r] = r == lane ? 1.0f : 0.0f;
#pragma unroll
                for (int k = 0; k < r; ++k) x[r] = __builtin_fmaf(-m[r * L::LINE + k], x[k], x[r]);
                keep_finite(x[r], 16 * wave + r);
            }
#pragma unroll
        for (int r = 0; r < 16; ++r) inverse[(16 * wave + r) * L::LINE + 16 * wave + lane] = x[r];
    }
    // zeros above the diagonal's blocks
#pragma unroll
    for (int jt = 1; jt < 4; ++jt)
        if (jt > wave)
#pragma unroll
            for (int r = 0; r < 4; ++r) inverse[(16 * wave + 4 * quad + r) * L::LINE + 16 * jt + col] = 0.0f;
    __syncthreads();
    const int block = 32 * wave;              // wavefronts 0, 1: block rows 16 .. 31 and 48 .. 63
    f32x4 x;
    if (wave < 2) {
        x = tile_product(below + (block + 16) * L::LINE + block, L::LINE, inverse + block * (L::LINE + 1), L::LINE, 16, col, quad);
        keep_finite4(x, block + 16 + 4 * quad);
#pragma unroll
        for (int r = 0; r < 4; ++r) half[(16 * wave + 4 * quad + r) * 33 + col] = x[r];
    }
    __syncthreads();
    if (wave < 2) {
        x = tile_product(inverse + (block + 16) * (L::LINE + 1), L::LINE, half + 16 * wave * 33, 33, 16, col, quad);
        keep_finite4(x, block + 16 + 4 * quad);
#pragma unroll
        for (int r = 0; r < 4; ++r) inverse[(block + 16 + 4 * quad + r) * L::LINE + block + col] = -x[r];
    }
    __syncthreads();
    const int tr = 16 * (wave >> 1), tc = 16 * (wave & 1);
    x = tile_product(below + (32 + tr) * L::LINE, L::LINE, inverse + tc, L::LINE, 32, col, quad);
    keep_finite4(x, 32 + tr + 4 * quad);
#pragma unroll
    for (int r = 0; r < 4; ++r) half[(tr + 4 * quad + r) * 33 + tc + col] = x[r];
    __syncthreads();
    x = tile_product(inverse + (32 + tr) * L::LINE + 32, L::LINE, half + tc, 33, 32, col, quad);
    keep_finite4(x, 32 + tr + 4 * quad);
#pragma unroll
    for (int r = 0; r < 4; ++r) inverse[(32 + tr + 4 * quad + r) * L::LINE + tc + col] = -x[r];
    __syncthreads();
    for (int p = tid; p < CHUNK * CHUNK / 4; p += 256) {
        const int row = p >> 4, at = 4 * (p & 15);
        float v[4];
        const int64_t f = (unit * 8 + (row >> 4) * 2 + (at >> 5)) * N_::WIDE_FRAGMENT + ((at & 31) >> 3) * 256 + (row & 15) * 16;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = BACK ? inverse[(at + i) * L::LINE + row] : inverse[row * L::LINE + at + i];
        put_wide4<T>((BACK ? a.inverse_t : a.inverse) + f, 1024, (at >> 2) & 1, v);
    }
    if (tid == 0) {
        gates.bad_k = gates_bad | bad[0] | (uint64_t)bad[1] << 32;
        gates.bad_q = bad[2] | (uint64_t)bad[3] << 32;
        gates.resets = resets;
    }
}

// ---- from chunk to chunk ------------------------------------------------------------------------------------------------
// Columns of values that are not finite: what they were at which step.  They are taken out of the products, which would spread them, and put back where the rule has them.
struct Marks {
    uint32_t any, most[3];                // the chunk (+ 1) that has some; the largest of the state's entries after a chunk, of three in turn (see lift_of)
    uint32_t steps[TILE][2];
    __device__ __forceinline__ uint64_t of(int column) const { return (uint64_t)steps[column][0] | (uint64_t)steps[column][1] << 32; }
};
__device__ __forceinline__ void mark(Marks &m, int column, int step, int chunk)
{
    atomicOr(&m.steps[column][step >> 5], 1u << (step & 31));
    m.any = chunk + 1;
}
__device__ __forceinline__ uint64_t steps_between(int from, int to) { return (~0ull >> (63 - to)) & (~0ull << from); }

// What a segment makes of ones on the diagonal may leave binary32 where no state does: growing steps make more of them than there is, also of a state of nothing, and strong decays less,
// which later steps may bring back.  So it is held as numbers between 2^-40 and 2^-10 at each chunk's beginning (a chunk may lengthen by 2^127) and a power of two, which joins them when
// they have met the state.  Powers of two round nothing.  (A prompt of 8192, 8 heads of 128 x 128, bf16, in turn: 209 us, without 208; lifted in every chunk 214.)
__device__ __forceinline__ int lift_of(uint32_t most)
{
    const int e = (int)(most >> 23);
    return e == 0 || e == 255 || (e >= 127 - 40 && e <= 127 - 10) ? 0 : 127 - e - 20;
}
// ... the part of the power that the numbers take before they meet the state: up to 2^60, so that a small state's products are not the smallest numbers, and no less than there is
__device__ __forceinline__ int early_part(int power) { return power < 0 ? 0 : power < 60 ? power : 60; }

template <typename T> __device__ __forceinline__ void store4(T *p, const float (&v)[4], int count)
{
    T x[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = from_f32<T>(v[r]);
    if (count >= 4) __builtin_memcpy(p, x, sizeof x);
    else
#pragma unroll
        for (int r = 0; r < 4; ++r) if (r < count) p[r] = x[r];
}

// A head's tiles on one die (workgroups go to the dies in turn), whose L2 then has the chunks' fragments for all of them
constexpr int DIES = 8;
struct Part { int tile, h, n; };
__device__ __forceinline__ Part part_of(const DeltaArgs &a, int tiles)
{
    const uint32_t die = blockIdx.x % DIES, i = blockIdx.x / DIES, head = i / tiles * DIES + die;
    return Part{(int)(i % tiles), (int)(head % a.d.H), (int)(head / a.d.H)};
}
inline int64_t parts(const DeltaArgs &a, int tiles) { return round_up((int64_t)a.d.N * a.d.H, DIES) * tiles; }

template <typename T, int KP> struct RunLds {
    typedef Num<T> N_;
    static constexpr int STATE_PITCH = N_::pitch(KP), ROW_PITCH = N_::pitch(CHUNK), EXACT_PITCH = N_::exact_pitch(CHUNK);
    static constexpr int STATE = 0, ONE = STATE + TILE * STATE_PITCH, TWO = ONE + TILE * ROW_PITCH, THREE = TWO + TILE * ROW_PITCH, MARKS = THREE + TILE * ROW_PITCH;
    static constexpr int FOUR = MARKS + (int)sizeof(Marks), BYTES = FOUR, BACK_BYTES = FOUR + TILE * EXACT_PITCH;
};
// tiles of 16 keys' entries of a wavefront
template <int KP> constexpr int key_tiles() { return KP / 64 > 0 ? KP / 64 : 1; }

// A workgroup for 32 of a head's values (a column of the state meets no other one), its state in registers; rows of LDS hand on what another wavefront takes.  A chunk is a chain of four
// phases (left over, Z, outputs and state), and a prompt or storage a chain of chunks: bound by latency, with two workgroups a unit.  512 x 16 steps, 8 heads of 128 x 128, bf16: 76 us,
// 3 us a chunk of the chain where memory is near, the rest the states for the backward call (126 MB written).  The matrix units work for 12 us of it, the vector units for 18.  129 x 5 in binary32 19.
//
// ENDS: a segment's part of the states after it, of its own steps and, in tiles behind the values', of the state before it: that of a one for each key, and no values
template <typename T, int KP, bool ENDS> __global__ __launch_bounds__(256, 2) void forward_kernel(const DeltaArgs a)
{
    typedef RunLds<T, KP> L;
    typedef Num<T> N_;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const hts_delta_rule_desc &d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quad = lane >> 4;
    const Part at = part_of(a, a.tiles + (ENDS ? KP / TILE : 0));
    if (at.n >= d.N) return;
    const bool ones = ENDS && at.tile >= a.tiles;
    const int tile = ones ? at.tile - a.tiles : at.tile, h = at.h, n = at.n, segment = blockIdx.y;
    const int K = d.K, V = d.V, v0 = tile * TILE, group = h / (d.H / d.G), len = length_of(a, n);
    const int begin = segment * a.per_segment, all_chunks = (len + CHUNK - 1) / CHUNK, used = begin + a.per_segment < all_chunks ? begin + a.per_segment : all_chunks;
    if (begin >= used && segment > 0) return;
    const int64_t place = ((int64_t)segment * d.N + n) * d.H + h;
    constexpr int MT = key_tiles<KP>();
    const bool has_keys = wave * MT * 16 < KP;
    char *state = lds + L::STATE, *left_over = lds + L::ONE, *writes = lds + L::TWO, *late = lds + L::THREE;
    Marks &marks = *(Marks *)(lds + L::MARKS);
    if (tid < TILE) marks.steps[tid][0] = marks.steps[tid][1] = 0;
    if (tid == TILE) marks.any = 0;
    if (ENDS && tid < 3) marks.most[tid] = tid == 2 ? __float_as_uint(1.0f) : 0u;

    f32x4 S[MT][2];
    const int64_t held = ((int64_t)n * d.H + h) * K * V;
    const auto each_state = [&](auto f) {
        if (!has_keys) return;
        const int row4 = again(4 * quad), column = again(col);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int k = 16 * (wave * MT + m) + row4 + r, v = v0 + 16 * nt + column;
                    S[m][nt][r] = f(S[m][nt][r], k < K && v < V, (int64_t)k * V + v);
                }
    };
    const auto lift_state = [&](int by) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[m][nt][r] = __builtin_ldexpf(S[m][nt][r], by);
    };
    int power = 0, turn = 2;                                   // turn: which of the three holds what is largest now
    const auto share_state = [&]() {
        if (!has_keys) return;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                const float x[4] = {S[m][nt][0], S[m][nt][1], S[m][nt][2], S[m][nt][3]};
                put_wide4<T>(state + (16 * nt + col) * L::STATE_PITCH + (2 * (wave * MT + m) + (quad >> 1)) * N_::WIDE, 16, quad & 1, x);
            }
    };
    const int VP = a.VP;
    if constexpr (ENDS) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[m][nt][r] = ones && 16 * (wave * MT + m) + 4 * quad + r == v0 + 16 * nt + col ? 1.0f : 0.0f;
    } else if (a.segments > 1) {                             // (the first one's too: the last one may be writing h_out into h_in's place by now)
        if (has_keys)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) S[m][nt][r] = a.begins[(place * KP + 16 * (wave * MT + m) + 4 * quad + r) * VP + v0 + 16 * nt + col];
    } else each_state([&](float, bool there, int64_t at) { return there && a.in.h_in ? a.in.h_in[held + at] : 0.0f; });
    share_state();
    const uint32_t state_at = row_at<float>(16 * wave * MT + 4 * quad, VP, col), z_at = row_at<float>(16 * wave + 4 * quad, VP, col);

    // A chunk's operands are requested when the chunk's before it have been used, and arrive while it is worked on (the barriers wait for LDS only)
    const int row = 16 * wave + 4 * quad, i = 16 * wave + col;     // of 4 steps, one after the other; of a step
    Exact<T> kf[KP / 32], qf[KP / 32], tf[MT][2];
    Wide<T> wf[2], pf[2];
    T val[2][4] = {};
    float keep[4], k_unit[4], strength[4], left[4], keep_i = 0.0f, q_unit_i = 0.0f, all = 0.0f;
    uint64_t bad_k = 0;
    const auto unit_of = [&](int c) { return ((int64_t)c * d.N + n) * d.H + h; };
    // rows behind the end: the last one again, whose products go nowhere; keys' entries behind K, where the state has zeros: the first ones
    const auto load_rows = [&](int c) {
        const int t = c * CHUNK + i < len ? i : len - 1 - c * CHUNK;
        const T *k = a.rows ? (const T *)a.rows + unit_of(c) * 2 * CHUNK * KP : step_of<T>(a.in.k, c * CHUNK, n) + (int64_t)group * K;
        const T *q = a.rows ? k + CHUNK * KP : step_of<T>(a.in.q, c * CHUNK, n) + (int64_t)group * K;
        const uint32_t k_at = row_at<T>(t, a.rows ? KP : a.in.k.st, 0), q_at = row_at<T>(t, a.rows ? KP : a.in.q.st, 0);
#pragma unroll
        for (int s = 0; s < KP / 32; ++s) {
            const uint32_t at = (K < KP && 32 * s + 8 * quad >= K ? 0 : 32 * s + 8 * quad) * (uint32_t)sizeof(T);
            kf[s] = load_at<Exact<T>>(k, k_at + at);
            if constexpr (!ENDS) qf[s] = load_at<Exact<T>>(q, q_at + at);
        }
    };
    const auto load_values = [&](int c) {
        if (ones) return;                                      // (zeros)
        const T *v = step_of<T>(a.in.v, c * CHUNK, n) + (int64_t)h * V;
        const int last = len - 1 - c * CHUNK;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t at = row_at<T>(row + r < last ? row + r : last, a.in.v.st, 0);
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                const int column = v0 + 16 * nt + col;
                val[nt][r] = load_at<T>(v, at + (column < V ? column : V - 1) * (uint32_t)sizeof(T));
            }
        }
    };
    const auto load_gates = [&](int c) {
        const Gates &g = a.gates[unit_of(c)];
        __builtin_memcpy(keep, g.keep + row, 16); __builtin_memcpy(k_unit, g.k_unit + row, 16);
        __builtin_memcpy(strength, g.strength + row, 16); __builtin_memcpy(left, g.left + row, 16);
        keep_i = g.keep[i]; q_unit_i = g.q_unit[i]; all = g.keep[CHUNK - 1]; bad_k = g.bad_k;
    };
    const auto load_pair = [&](Wide<T> (&f)[2], const char *base, int c) {      // (the second one of rows 0 .. 31 is zeros)
#pragma unroll
        for (int s = 0; s < 2; ++s)
            if (s == 0 || wave >= 2) f[s] = get_wide<T>(base + (unit_of(c) * 8 + wave * 2 + s) * N_::WIDE_FRAGMENT + lane * 16, 1024);
    };
    const auto load_keys = [&](int c) {
        if (!has_keys) return;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int s = 0; s < 2; ++s) tf[m][s] = get_exact<T>(a.keys + (unit_of(c) * (KP / 8) + (wave * MT + m) * 2 + s) * N_::EXACT_FRAGMENT + lane * 16, 1024);
    };
    if (begin < used) { load_rows(begin); load_gates(begin); load_values(begin); }
    lds_barrier();
    for (int c = begin; c < used; ++c) {
        const int64_t unit = unit_of(c);
        const int t0 = c * CHUNK;
        const bool more = c + 1 < used;
        load_pair(wf, a.inverse, c);
        const uint32_t largest = ENDS ? marks.most[turn] : 0u;
        if (!ENDS && a.states && has_keys) {
            float *to = a.states + unit * KP * VP + v0;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) store_at(to + (16 * m + r) * (int64_t)VP + 16 * nt, state_at, S[m][nt][r]);
        }
        // what the state has for the keys, and for the queries
        f32x4 ks[2] = {}, qs[2] = {};
#pragma unroll
        for (int s = 0; s < KP / 32; ++s) {
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                const Wide<T> sf = get_wide<T>(state + (16 * nt + col) * L::STATE_PITCH + (4 * s + quad) * N_::WIDE, 16);
                mma(ks[nt], kf[s], sf);
                if constexpr (!ENDS) mma(qs[nt], sf, qf[s]);
            }
            __builtin_amdgcn_sched_barrier(0);                 // (operands of every s at once are more than there are registers)
        }
        if constexpr (!ENDS) load_pair(pf, a.read, c);
        if (more) load_rows(c + 1);
        int lift = 0;
        if (ENDS && ones) {
            lift = __builtin_amdgcn_readfirstlane(lift_of(largest));
            power -= lift;
            turn = turn == 2 ? 0 : turn + 1;
            if (lift != 0) {                                   // (the rows in LDS are still as they were: their products take the same)
                lift_state(lift);
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) ks[nt][r] = __builtin_ldexpf(ks[nt][r], lift);
            }
        }
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            float e[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool live = t0 + row + r < len && (ones || v0 + 16 * nt + col < V);
                e[r] = to_f32(val[nt][r]);
                if (keep[r] >= 0.0f) e[r] -= keep[r] * k_unit[r] * ks[nt][r];
                if (!live) e[r] = 0.0f;
                else if (!finite(e[r]) || (bad_k >> (row + r) & 1)) { e[r] = 0.0f; mark(marks, 16 * nt + col, row + r, c); }
            }
            put_wide4<T>(left_over + (16 * nt + col) * L::ROW_PITCH + (row >> 3) * N_::WIDE, 16, quad & 1, e);
        }
        if (more) load_values(c + 1);
        lds_barrier();
        // Z, and what it writes
        f32x4 z[2] = {};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (s == 1 && wave < 2) continue;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) mma(z[nt], wf[s], get_wide<T>(left_over + (16 * nt + col) * L::ROW_PITCH + (4 * s + quad) * N_::WIDE, 16));
        }
        load_keys(c);
        if (!finite(sizes_of(z[0]) + sizes_of(z[1])))          // (the state leaves binary32 at such a step)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (!finite(z[nt][r])) { z[nt][r] = 0.0f; mark(marks, again(16 * nt + col), again(row) + r, c); }
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            float u[4], l[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                u[r] = strength[r] * z[nt][r];
                l[r] = left[r] >= 0.0f ? left[r] * k_unit[r] * u[r] : 0.0f;
            }
            if constexpr (!ENDS) put_wide4<T>(writes + (16 * nt + col) * L::ROW_PITCH + (row >> 3) * N_::WIDE, 16, quad & 1, u);
            put_wide4<T>(late + (16 * nt + col) * L::ROW_PITCH + (row >> 3) * N_::WIDE, 16, quad & 1, l);
            if (!ENDS && a.z) {
                float *to = a.z + unit * CHUNK * VP + v0 + 16 * nt;
#pragma unroll
                for (int r = 0; r < 4; ++r) store_at(to + r * (int64_t)VP, z_at, z[nt][r]);
            }
        }
        lds_barrier();
        const bool some = marks.any == (uint32_t)c + 1;
        // outputs, the values along a row
        if constexpr (!ENDS) {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int r = 0; r < 4; ++r) qs[nt][r] = keep_i >= 0.0f ? keep_i * q_unit_i * d.scale * qs[nt][r] : 0.0f;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (s == 1 && wave < 2) continue;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) mma(qs[nt], get_wide<T>(writes + (16 * nt + col) * L::ROW_PITCH + (4 * s + quad) * N_::WIDE, 16), pf[s]);
        }
        if (t0 + i < len) {
            const uint64_t seen = some ? steps_between(a.gates[unit].first[i], i) : 0;
            T *y = step_of<T>(a.y, t0, n) + (int64_t)h * V + v0;
            const uint32_t y_at = row_at<T>(i, a.y.st, 4 * quad);
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                Four<T> o;
#pragma unroll
                for (int r = 0; r < 4; ++r) o.e[r] = from_f32<T>(some && (marks.of(16 * nt + 4 * quad + r) & seen) ? __builtin_nanf("") : qs[nt][r]);
                const int count = V - (v0 + 16 * nt + 4 * quad);
                if (count >= 4) store_at(y + 16 * nt, y_at, o);
                else
#pragma unroll
                    for (int r = 0; r < 4; ++r) if (r < count) store_at(y + 16 * nt + r, y_at, o.e[r]);
            }
        }
        }
        // the state at the end
        if (has_keys) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[m][nt][r] = all >= 0.0f ? all * S[m][nt][r] : 0.0f;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                Wide<T> l[2];
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) l[nt] = get_wide<T>(late + (16 * nt + col) * L::ROW_PITCH + (4 * s + quad) * N_::WIDE, 16);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) mma(S[m][nt], tf[m][s], l[nt]);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (some) {
                const uint64_t last = steps_between(a.gates[unit].first[CHUNK - 1], CHUNK - 1);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
                        if (marks.of(16 * nt + col) & last)
#pragma unroll
                            for (int r = 0; r < 4; ++r) S[m][nt][r] = __builtin_nanf("");
            }
            if (ENDS && ones) {
                float most = 0.0f;
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int r = 0; r < 4; ++r) most = fmaxf(most, __builtin_fabsf(S[m][nt][r]));
                most = most16(most);
                if (col == 0) atomicMax(&marks.most[turn], __float_as_uint(most));       // (sizes are in their bits' order)
            }
            share_state();
        }
        if (more) load_gates(c + 1);
        lds_barrier();
        if (ENDS && ones && tid == 0) marks.most[turn == 2 ? 0 : turn + 1] = 0;      // (read in the chunk before this one, and written in the next one, two barriers on)
        if (some) {
            if (!ENDS && a.z)
                for (int p = again(0); p < 8; ++p) {               // (a lane's own, after what it has written there)
                    const int step = row + (p & 3), column = 16 * (p >> 2) + col;
                    if (t0 + step < len && (marks.of(column) & steps_between(a.gates[unit].first[step], step))) a.z[(unit * CHUNK + step) * VP + v0 + column] = __builtin_nanf("");
                }
            lds_barrier();
            if (tid < TILE) marks.steps[tid][0] = marks.steps[tid][1] = 0;
            lds_barrier();
        }
    }
    if constexpr (ENDS) {
        const int width = VP + KP, first = ones ? VP + v0 : v0;
        if (ones) {
            const int lift = lift_of(marks.most[turn]), early = early_part(power - lift);
            lift_state(lift + early);
            if (tid == 0) a.powers[place * (KP / TILE) + tile] = power - lift - early;
        }
        if (has_keys)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) a.ends[(place * KP + 16 * (wave * MT + m) + 4 * quad + r) * width + first + 16 * nt + col] = S[m][nt][r];
        return;
    }
    if (a.h_out && used == all_chunks) each_state([&](float s, bool there, int64_t at) { if (there) a.h_out[held + at] = s; return s; });
    if (segment > 0) return;
    for (int64_t p = tid; p < (int64_t)(d.T - len) * TILE; p += 256) {
        const int v = v0 + (int)(p % TILE);
        if (v < V) step_of<T>(a.y, len + p / TILE, n)[(int64_t)h * V + v] = from_f32<T>(0.0f);
    }
}

// The states that the segments begin with: from one to the next, what its steps make of the state before it and what they add.  A segment in which an episode begins leaves
// nothing of it (not 0 times it, which would be NaN of what is not finite).  A step's latency is all that counts: a wavefront for 16 of the keys' entries (with two such parts
// each a prompt of 8192 and 8 heads of 128 keys took 31 us, and 35 with operands requested where they are used; now 25, with the powers of two 27, seven steps).
template <typename T, int KP> __global__ __launch_bounds__(4 * KP) void begin_kernel(const DeltaArgs a)
{
    typedef RunLds<T, KP> L;
    typedef Num<T> N_;
    __shared__ __attribute__((aligned(16))) char state[TILE * L::STATE_PITCH];
    __shared__ int forgets[ROOM];
    const hts_delta_rule_desc &d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quad = lane >> 4;
    const Part at = part_of(a, a.tiles);
    if (at.n >= d.N) return;
    const int h = at.h, n = at.n, v0 = at.tile * TILE, VP = a.VP, width = VP + KP, chunks = (length_of(a, n) + CHUNK - 1) / CHUNK, row = 16 * wave + 4 * quad;
    f32x4 S[2] = {};
    if (a.in.h_in)
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int k = row + r, v = v0 + 16 * nt + col;
                if (k < d.K && v < d.V) S[nt][r] = a.in.h_in[(((int64_t)n * d.H + h) * d.K + k) * d.V + v];
            }
    const auto place_of = [&](int s) { return (((int64_t)s * d.N + n) * d.H + h) * KP; };
    const auto put_begin = [&](int s) {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int r = 0; r < 4; ++r) a.begins[(place_of(s) + row + r) * VP + v0 + 16 * nt + col] = S[nt][r];
    };
    put_begin(0);
    // a segment's operands arrive while the one before it is worked on
    static_assert(TILE == 32, "a tile's power is that of 32 of the entries that a product sums over");
    float next_move[KP / 32][8], next_own[2][4];
    int next_power[KP / 32];
    const auto more = [&](int s) { return s + 1 < a.segments && (s + 1) * a.per_segment < chunks; };
    const auto load = [&](int s) {
        const float *from = a.ends + (place_of(s) + 16 * wave) * width;
#pragma unroll
        for (int k = 0; k < KP / 32; ++k) {
            __builtin_memcpy(next_move[k], __builtin_assume_aligned(from + (int64_t)col * width + VP + 32 * k + 8 * quad, 16), 32);
            next_power[k] = a.powers[place_of(s) / KP * (KP / TILE) + k];
        }
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int r = 0; r < 4; ++r) next_own[nt][r] = from[(int64_t)(4 * quad + r) * width + v0 + 16 * nt + col];
    };
    if (more(0)) load(0);
    for (int i = tid; i < ROOM; i += 4 * KP) forgets[i] = 0;
    lds_barrier();
    for (int c = tid; c < chunks; c += 4 * KP)
        if (a.gates[((int64_t)c * d.N + n) * d.H + h].keep[CHUNK - 1] < 0.0f) forgets[c / a.per_segment] = 1;
    for (int s = 0; more(s); ++s) {
        float move[KP / 32][8];
        int power[KP / 32];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            const float x[4] = {S[nt][0], S[nt][1], S[nt][2], S[nt][3]};
            put_wide4<T>(state + (16 * nt + col) * L::STATE_PITCH + (2 * wave + (quad >> 1)) * N_::WIDE, 16, quad & 1, x);
#pragma unroll
            for (int r = 0; r < 4; ++r) S[nt][r] = next_own[nt][r];
        }
        __builtin_memcpy(move, next_move, sizeof move);
#pragma unroll
        for (int k = 0; k < KP / 32; ++k) power[k] = __builtin_amdgcn_readfirstlane(next_power[k]);
        if (more(s + 1)) load(s + 1);
        lds_barrier();
        if (!forgets[s])
#pragma unroll
            for (int k = 0; k < KP / 32; ++k) {
                const Wide<T> moved = make_wide<T>(move[k]);
                if (power[k] == 0)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) mma(S[nt], moved, get_wide<T>(state + (16 * nt + col) * L::STATE_PITCH + (4 * k + quad) * N_::WIDE, 16));
                else
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) {
                        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
                        mma(x, moved, get_wide<T>(state + (16 * nt + col) * L::STATE_PITCH + (4 * k + quad) * N_::WIDE, 16));
#pragma unroll
                        for (int r = 0; r < 4; ++r) S[nt][r] += __builtin_ldexpf(x[r], power[k]);
                    }
            }
        put_begin(s + 1);
        lds_barrier();
    }
}

// A few steps: the state in registers, 64 of the values' entries a workgroup, 4 to a thread, every 16th of the keys'.  One sum over the keys a step: of the state before it
// with the key and with the query, y = scale (al q . S + (q . k) be z).  A step reads and writes the state once: 32 rows of 8 heads of 128 x 128 11.7 us, 33.5 MB (2.9 TB/s; all of it is on its
// way at once, in and then out).  Five steps of 16 rows of 4 heads of 64 x 64 10.5: a reduction
// and a barrier a step (14.6 with each step's gates and lengths made in it, of which the exponentials are most).
// Calls of so many steps or fewer go step by step: 16 steps of 32 x 8 heads of 128 x 128 in bf16 31 us, in a chunk 40; of 1 x 8 heads 26 and 26; of 16 x 4 heads of 64 x 64 in binary32
// 23 and 24.  (24 steps of the smaller ones would cost more than a chunk.)
constexpr int MOST_STEPS = 16;
constexpr int STEP_TILE = 64, STEP_ROWS = 8;
template <typename T> __global__ __launch_bounds__(256) void step_kernel(const DeltaArgs a)
{
    const hts_delta_rule_desc &d = a.d;
    // what the steps have by themselves is made for all of them before the first one: keys and queries, [16 m + r] at 8 r + m; what a step takes of each
    struct Step { float decay, strength, k_unit, q_unit, along; int reset; };
    __shared__ __attribute__((aligned(16))) float kq[MOST_STEPS][2][128], sums[2][4][2][STEP_TILE];
    __shared__ Step steps[MOST_STEPS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, four = tid & 15, rg = tid >> 4;
    const int tile = blockIdx.x % a.tiles, h = blockIdx.x / a.tiles % d.H, n = blockIdx.x / a.tiles / d.H;
    const int K = d.K, V = d.V, v0 = tile * STEP_TILE + 4 * four, group = h / (d.H / d.G), len = length_of(a, n), count = V - v0;
    const int64_t held = ((int64_t)n * d.H + h) * K * V;
    // a wavefront for every fourth step's key and query, lanes of the last one for the gates; the state arrives meanwhile
    T k_in[MOST_STEPS / 4][2], q_in[MOST_STEPS / 4][2], a_in = from_f32<T>(0.0f), b_in = a_in, v_in[4];
    uint8_t start = 0;
#pragma unroll
    for (int i = 0; i < MOST_STEPS / 4; ++i) {
        const int t = 4 * i + wave;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const bool there = t < len && lane + 64 * e < K;
            k_in[i][e] = there ? step_of<T>(a.in.k, t, n)[(int64_t)group * K + lane + 64 * e] : from_f32<T>(0.0f);
            q_in[i][e] = there ? step_of<T>(a.in.q, t, n)[(int64_t)group * K + lane + 64 * e] : from_f32<T>(0.0f);
        }
    }
    const bool gated = wave == 3 && lane < len;
    if (gated) {
        a_in = step_of<T>(a.in.a, lane, n)[h];
        b_in = step_of<T>(a.in.b, lane, n)[h];
        if (a.in.starts) start = a.in.starts[(int64_t)lane * d.N + n];
    }
    const auto load_values = [&](int t) {
        const T *v = step_of<T>(a.in.v, t, n) + (int64_t)h * V + v0;
        if (count >= 4) __builtin_memcpy(v_in, v, sizeof v_in);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) v_in[i] = i < count ? v[i] : from_f32<T>(0.0f);
    };
    if (len > 0) load_values(0);
    float S[STEP_ROWS][4];
#pragma unroll
    for (int m = 0; m < STEP_ROWS; ++m) {
        const int k = rg + 16 * m;
        const float *p = a.in.h_in + held + (int64_t)k * V + v0;
#pragma unroll
        for (int i = 0; i < 4; ++i) S[m][i] = 0.0f;
        if (a.in.h_in && k < K) {
            if (count >= 4) __builtin_memcpy(S[m], p, 16);
            else
#pragma unroll
                for (int i = 0; i < 4; ++i) if (i < count) S[m][i] = p[i];
        }
    }
#pragma unroll
    for (int i = 0; i < MOST_STEPS / 4; ++i) {
        const int t = 4 * i + wave;
        if (t >= len) break;
        float k_square = 0.0f, q_square = 0.0f, both = 0.0f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float kv = to_f32(k_in[i][e]), qv = to_f32(q_in[i][e]);
            const int at = 8 * (lane & 15) + (lane >> 4) + 4 * e;
            kq[t][0][at] = kv; kq[t][1][at] = qv;
            k_square = __builtin_fmaf(kv, kv, k_square); q_square = __builtin_fmaf(qv, qv, q_square); both = __builtin_fmaf(qv, kv, both);
        }
        k_square = wave_add(k_square); q_square = wave_add(q_square); both = wave_add(both);
        // (a key or query whose square is not finite is none, also where its entries are)
        const float k_unit = !finite(k_square) ? __builtin_nanf("") : d.normalize ? 1.0f / __builtin_sqrtf(k_square + 1e-6f) : 1.0f;
        const float q_unit = d.scale * (!finite(q_square) ? __builtin_nanf("") : d.normalize ? 1.0f / __builtin_sqrtf(q_square + 1e-6f) : 1.0f);
        if (lane == 0) { steps[t].k_unit = k_unit; steps[t].q_unit = q_unit; steps[t].along = both * k_unit; }
    }
    if (gated) {
        const Decay dc = decay_of(to_f32(a_in), a.in.a_bias ? a.in.a_bias[h] : 0.0f, a.in.A[h], d.softplus);
        const double e = (double)dc.exponent * LOG2E_64;
        const bool reset = start || e < FORGETS;
        steps[lane].reset = reset;
        steps[lane].decay = reset ? 0.0f : e < MOST_EXPONENT ? exp2_wide(e) : __builtin_nanf("");
        steps[lane].strength = sigmoid_f(to_f32(b_in));
    }
    const auto put_state = [&](float *to, int keys, int values) {
#pragma unroll
        for (int m = 0; m < STEP_ROWS; ++m) {
            const int k = rg + 16 * m;
            if (k < keys) store4(to + (int64_t)k * values + v0, S[m], values - v0);
        }
    };
    const int64_t unit = (int64_t)n * d.H + h;
    const float none[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (a.states && len > 0) {
        put_state(a.states + unit * keys_padded(K) * a.VP, keys_padded(K), a.VP);
        for (int t = len + rg; t < CHUNK; t += 16) store4(a.z + (unit * CHUNK + t) * a.VP + v0, none, a.VP - v0);
    }
    lds_barrier();
    for (int t = 0; t < len; ++t) {
        const Step step = steps[t];
        float val[4], kv[STEP_ROWS], qv[STEP_ROWS];
#pragma unroll
        for (int i = 0; i < 4; ++i) val[i] = to_f32(v_in[i]);
        if (t + 1 < len) load_values(t + 1);
        __builtin_memcpy(kv, __builtin_assume_aligned(&kq[t][0][8 * rg], 16), sizeof kv);
        __builtin_memcpy(qv, __builtin_assume_aligned(&kq[t][1][8 * rg], 16), sizeof qv);
        if (step.reset)
#pragma unroll
            for (int m = 0; m < STEP_ROWS; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) S[m][i] = 0.0f;
        float has[2][4] = {};
#pragma unroll
        for (int m = 0; m < STEP_ROWS; ++m)
            if (rg + 16 * m < K)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    has[0][i] = __builtin_fmaf(kv[m], S[m][i], has[0][i]);
                    has[1][i] = __builtin_fmaf(qv[m], S[m][i], has[1][i]);
                }
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                has[w][i] += __shfl_xor(has[w][i], 16, 64);
                has[w][i] += __shfl_xor(has[w][i], 32, 64);
            }
        float (&all)[4][2][STEP_TILE] = sums[t & 1];             // (whoever reads those of the step before has not passed this step's barrier)
        if ((rg & 3) == 0)
#pragma unroll
            for (int w = 0; w < 2; ++w) __builtin_memcpy(&all[wave][w][4 * four], has[w], 16);
        lds_barrier();
        float u[4], y[4], z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float ks = (all[0][0][4 * four + i] + all[1][0][4 * four + i]) + (all[2][0][4 * four + i] + all[3][0][4 * four + i]);
            const float qs = (all[0][1][4 * four + i] + all[1][1][4 * four + i]) + (all[2][1][4 * four + i] + all[3][1][4 * four + i]);
            z[i] = step.reset ? val[i] : val[i] - step.decay * step.k_unit * ks;
            u[i] = step.strength * z[i];
            y[i] = step.q_unit * (step.reset ? step.along * u[i] : __builtin_fmaf(step.decay, qs, step.along * u[i]));
        }
#pragma unroll
        for (int m = 0; m < STEP_ROWS; ++m) {
            const float by = kv[m] * step.k_unit;
#pragma unroll
            for (int i = 0; i < 4; ++i) S[m][i] = step.reset ? by * u[i] : __builtin_fmaf(step.decay, S[m][i], by * u[i]);
        }
        if (rg == 0) {
            store4(step_of<T>(a.y, t, n) + (int64_t)h * V + v0, y, count);
            if (a.z) store4(a.z + (unit * CHUNK + t) * a.VP + v0, z, a.VP - v0);
        }
    }
    if (a.h_out) put_state(a.h_out + held, K, V);
    if (rg == 0)
        for (int t = len; t < d.T; ++t) store4(step_of<T>(a.y, t, n) + (int64_t)h * V + v0, none, count);
}

__device__ __forceinline__ float sign_of(int chunk, int n) { return (chunk + n) & 1 ? -1.0f : 1.0f; }

// The state's gradient from chunk to chunk, from the last one.
//
// What a matrix instruction drops of its products goes towards minus infinity.  Gradients have either sign, but keys, queries, values and states may be mostly positive, and then
// the sums of the decays' gradients over thousands of steps add up what was dropped (da_bias 4.6e-6 of its values off, 512 x 16 steps).  So every second chunk has all gradients
// with the other sign, here and in the sums after it.
// The same shape as the forward kernel's, with one phase more: 512 x 16 steps, 8 heads of 128 x 128, bf16 104 us, 129 x 5 in binary32 21.
template <typename T, int KP> __global__ __launch_bounds__(256, 2) void reverse_kernel(const DeltaArgs a)
{
    typedef RunLds<T, KP> L;
    typedef Num<T> N_;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const hts_delta_rule_desc &d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quad = lane >> 4;
    const Part at = part_of(a, a.tiles);
    if (at.n >= d.N) return;
    const int tile = at.tile, h = at.h, n = at.n;
    const int K = d.K, V = d.V, v0 = tile * TILE, group = h / (d.H / d.G), len = length_of(a, n);
    constexpr int MT = key_tiles<KP>();
    const bool has_keys = wave * MT * 16 < KP;
    // the output's gradient (Exact); that of what is written, times its strength; minus that of the values, kept; the output's, kept
    char *state = lds + L::STATE, *given = lds + L::FOUR, *sent = lds + L::ONE, *kept = lds + L::TWO, *asked = lds + L::THREE;
    Marks &marks = *(Marks *)(lds + L::MARKS);
    if (tid < TILE) marks.steps[tid][0] = marks.steps[tid][1] = 0;
    if (tid == TILE) marks.any = 0;

    f32x4 S[MT][2];
    const int64_t held = ((int64_t)n * d.H + h) * K * V;
    const auto each_state = [&](auto f) {
        if (!has_keys) return;
        const int row4 = again(4 * quad), column = again(col);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int k = 16 * (wave * MT + m) + row4 + r, v = v0 + 16 * nt + column;
                    S[m][nt][r] = f(S[m][nt][r], k < K && v < V, (int64_t)k * V + v);
                }
    };
    each_state([&](float, bool there, int64_t at) { return there && a.dh_out ? a.dh_out[held + at] : 0.0f; });

    const int used = (len + CHUNK - 1) / CHUNK, row = 16 * wave + 4 * quad, i = 16 * wave + col;
    const int VP = a.VP;
    const uint32_t state_at = row_at<float>(16 * wave * MT + 4 * quad, VP, col), dv_at = row_at<float>(row, VP, col);
    const int my_v = tid & 31, my_i = 8 * (tid >> 5);                  // 8 steps of one of the values' entries
    Exact<T> kf[KP / 32], tf[MT][2], gf[MT][2];
    Wide<T> wf[2], pf[2];
    T given_y[8];
    float asked_by[8], keep[4], k_unit[4], strength[4], left[4], all = 0.0f;
    uint64_t bad_k = 0, bad_q = 0;
    const auto unit_of = [&](int c) { return ((int64_t)c * d.N + n) * d.H + h; };
    const auto load_outputs = [&](int c) {
        const Gates &g = a.gates[unit_of(c)];
        float q_unit[8];
        __builtin_memcpy(asked_by, g.keep + my_i, 32); __builtin_memcpy(q_unit, g.q_unit + my_i, 32);
        bad_q = g.bad_q;
        const T *y = step_of<T>(a.dy, c * CHUNK, n) + (int64_t)h * V;
        const int last = len - 1 - c * CHUNK;
        const uint32_t column = (v0 + my_v < V ? v0 + my_v : V - 1) * (uint32_t)sizeof(T);
#pragma unroll
        for (int x = 0; x < 8; ++x) given_y[x] = load_at<T>(y, row_at<T>(my_i + x < last ? my_i + x : last, a.dy.st, 0) + column);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            asked_by[x] = asked_by[x] >= 0.0f && !(bad_q >> (my_i + x) & 1) ? asked_by[x] * q_unit[x] * d.scale : 0.0f;
        }
    };
    const auto load_rows = [&](int c) {                                // (as in the forward kernel)
        const int t = c * CHUNK + i < len ? i : len - 1 - c * CHUNK;
        const T *k = a.rows ? (const T *)a.rows + unit_of(c) * 2 * CHUNK * KP : step_of<T>(a.in.k, c * CHUNK, n) + (int64_t)group * K;
        const uint32_t k_at = row_at<T>(t, a.rows ? KP : a.in.k.st, 0);
#pragma unroll
        for (int s = 0; s < KP / 32; ++s) kf[s] = load_at<Exact<T>>(k, k_at + (K < KP && 32 * s + 8 * quad >= K ? 0 : 32 * s + 8 * quad) * (uint32_t)sizeof(T));
    };
    const auto load_gates = [&](int c) {
        const Gates &g = a.gates[unit_of(c)];
        __builtin_memcpy(keep, g.keep + row, 16); __builtin_memcpy(k_unit, g.k_unit + row, 16);
        __builtin_memcpy(strength, g.strength + row, 16); __builtin_memcpy(left, g.left + row, 16);
        all = g.keep[CHUNK - 1]; bad_k = g.bad_k;
    };
    const auto load_pair = [&](Wide<T> (&f)[2], const char *base, int c) {      // (the first one of rows 32 .. 63 is zeros)
#pragma unroll
        for (int s = 0; s < 2; ++s)
            if (s == 1 || wave < 2) f[s] = get_wide<T>(base + (unit_of(c) * 8 + wave * 2 + s) * N_::WIDE_FRAGMENT + lane * 16, 1024);
    };
    const auto load_keys = [&](int c) {
        if (!has_keys) return;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int64_t f = (unit_of(c) * (KP / 8) + (wave * MT + m) * 2 + s) * N_::EXACT_FRAGMENT + lane * 16;
                tf[m][s] = get_exact<T>(a.keys + f, 1024); gf[m][s] = get_exact<T>(a.queries + f, 1024);
            }
    };
    if (used > 0) { const int c = used - 1; load_outputs(c); load_rows(c); load_gates(c); }
    float held_sign = 1.0f;
    for (int c = used - 1; c >= 0; --c) {
        const int64_t unit = unit_of(c);
        const int t0 = c * CHUNK;
        const bool more = c > 0;
        load_pair(pf, a.read, c);
        const float sign = sign_of(c, n);
        if (sign != held_sign)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) S[m][nt] = -S[m][nt];
        held_sign = sign;
        if (has_keys) {
            float *to = a.late + unit * KP * VP + v0;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) store_at(to + (16 * m + r) * (int64_t)VP + 16 * nt, state_at, sign * S[m][nt][r]);
        }
        lds_barrier();                                         // (the arrays of the chunk after this one have been read)
        if (has_keys)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
                    const float x[4] = {S[m][nt][0], S[m][nt][1], S[m][nt][2], S[m][nt][3]};
                    put_wide4<T>(state + (16 * nt + col) * L::STATE_PITCH + (2 * (wave * MT + m) + (quad >> 1)) * N_::WIDE, 16, quad & 1, x);
                }
        {
            T x[8];
            float w[2][4];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool live = t0 + my_i + e < len && v0 + my_v < V;
                x[e] = from_f32<T>(live ? sign * to_f32(given_y[e]) : 0.0f);
                if (!finite(to_f32(x[e])) || (bad_q >> (my_i + e) & 1)) {
                    x[e] = from_f32<T>(0.0f);
                    if (live) mark(marks, my_v, my_i + e, c);
                }
                w[e >> 2][e & 3] = asked_by[e] * to_f32(x[e]);
            }
            put_exact<T>(given + my_v * L::EXACT_PITCH + (my_i >> 3) * N_::EXACT, 16, make_exact<T>(x));
            put_wide4<T>(asked + my_v * L::ROW_PITCH + (my_i >> 3) * N_::WIDE, 16, 0, w[0]);
            put_wide4<T>(asked + my_v * L::ROW_PITCH + (my_i >> 3) * N_::WIDE, 16, 1, w[1]);
        }
        if (more) load_outputs(c - 1);
        lds_barrier();
        // dU: by the outputs of this chunk, by the state at its end
        f32x4 du[2] = {}, ks[2] = {};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (s == 0 && wave >= 2) continue;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) mma(du[nt], pf[s], get_exact<T>(given + (16 * nt + col) * L::EXACT_PITCH + (4 * s + quad) * N_::EXACT, 16));
        }
        load_pair(wf, a.inverse_t, c);
#pragma unroll
        for (int s = 0; s < KP / 32; ++s) {
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) mma(ks[nt], kf[s], get_wide<T>(state + (16 * nt + col) * L::STATE_PITCH + (4 * s + quad) * N_::WIDE, 16));
            __builtin_amdgcn_sched_barrier(0);
        }
        if (more) load_rows(c - 1);
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            float x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = du[nt][r];
                if (left[r] >= 0.0f) x[r] += left[r] * k_unit[r] * ks[nt][r];
                x[r] = t0 + row + r < len ? x[r] * strength[r] : 0.0f;
                if (!finite(x[r]) || (bad_k >> (row + r) & 1)) { x[r] = 0.0f; if (v0 + 16 * nt + col < V) mark(marks, 16 * nt + col, row + r, c); }
            }
            put_wide4<T>(sent + (16 * nt + col) * L::ROW_PITCH + (row >> 3) * N_::WIDE, 16, quad & 1, x);
        }
        lds_barrier();
        const bool some = marks.any == (uint32_t)c + 1;
        f32x4 dv[2] = {};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (s == 0 && wave >= 2) continue;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) mma(dv[nt], wf[s], get_wide<T>(sent + (16 * nt + col) * L::ROW_PITCH + (4 * s + quad) * N_::WIDE, 16));
        }
        load_keys(c);
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            float x[4], *to = a.write + unit * CHUNK * VP + v0 + 16 * nt;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = keep[r] >= 0.0f ? -(keep[r] * k_unit[r] * dv[nt][r]) : 0.0f;
                // a step's gradient has what the later ones of its episode have
                bool wrong = false;
                if (some && t0 + row + r < len) {
                    const uint64_t later = row + r == 63 ? 0 : a.gates[unit].resets & (~0ull << (row + r + 1));
                    wrong = marks.of(16 * nt + col) & steps_between(row + r, later ? __builtin_ctzll(later) - 1 : 63);
                }
                store_at(to + r * (int64_t)VP, dv_at, wrong ? __builtin_nanf("") : sign * dv[nt][r]);
            }
            put_wide4<T>(kept + (16 * nt + col) * L::ROW_PITCH + (row >> 3) * N_::WIDE, 16, quad & 1, x);
        }
        const float all_of = all;
        if (more) load_gates(c - 1);
        lds_barrier();
        if (has_keys) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[m][nt][r] = all_of >= 0.0f ? all_of * S[m][nt][r] : 0.0f;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                Wide<T> w[2], y[2];
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
                    w[nt] = get_wide<T>(kept + (16 * nt + col) * L::ROW_PITCH + (4 * s + quad) * N_::WIDE, 16);
                    y[nt] = get_wide<T>(asked + (16 * nt + col) * L::ROW_PITCH + (4 * s + quad) * N_::WIDE, 16);
                }
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) { mma(S[m][nt], tf[m][s], w[nt]); mma(S[m][nt], gf[m][s], y[nt]); }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (some) {
                const uint64_t resets = a.gates[unit].resets, before = resets ? (resets & 1 ? 0 : steps_between(0, __builtin_ctzll(resets) - 1)) : ~0ull;
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
                        if (marks.of(16 * nt + col) & before)
#pragma unroll
                            for (int r = 0; r < 4; ++r) S[m][nt][r] = __builtin_nanf("");
            }
        }
        if (some) {
            lds_barrier();
            if (tid < TILE) marks.steps[tid][0] = marks.steps[tid][1] = 0;
        }
    }
    if (a.g.dh_in) each_state([&](float s, bool there, int64_t at) { if (there) a.g.dh_in[held + at] = held_sign * s; return s; });
}

// ---- gradients that sum over the values -----------------------------------------------------------------------------------
// Eight wavefronts.  Products with the states: a wavefront has 16 of the keys' entries and up to four tiles of 16 steps, so a state's entry is read and cut into parts by
// one wavefront (two or four where keys are short), straight from memory.  A tile's rows are steps 32 (t / 2) + 8 (row / 4) + 4 (t % 2) + row % 4, so that the 8 steps of a
// lane's two tiles are those of a fragment of the keys: their values are there for sums along them.
template <typename T, int KP> struct GradLds {
    typedef Num<T> N_;
    static constexpr int PITCH = N_::pitch(TILE), Y_PITCH = N_::exact_pitch(TILE), LINE = 68;
    // a tile's 16 rows are fours of every eight: with 64 bytes more between sixteens they begin in 16 places of four banks, without in 8
    static __device__ __forceinline__ int row_of(int row, int pitch) { return row * pitch + (row >> 4) * 64; }
    static constexpr int MORE = CHUNK / 16 * 64;
    static constexpr int WRITES = 0, VALUES = WRITES + CHUNK * PITCH + MORE, GIVEN = VALUES + CHUNK * PITCH + MORE, STAGE = GIVEN + CHUNK * Y_PITCH + MORE;      // two of these, in turn
    // after the values: a matrix of 64 x 64, what passes from step to step; at last the rows that leave
    static constexpr int MATRIX = 0, MATRIX_PITCH = N_::pitch(CHUNK), PASSING = MATRIX + CHUNK * MATRIX_PITCH + MORE, AFTER = PASSING + 4 * CHUNK * LINE;
    static constexpr int OUT_PITCH = KP * (int)sizeof(T) + 16, OUT = 2 * CHUNK * OUT_PITCH;
    static constexpr int AREA = (2 * STAGE > AFTER ? 2 * STAGE : AFTER) > OUT ? (2 * STAGE > AFTER ? 2 * STAGE : AFTER) : OUT;
    static constexpr int ROWS = AREA, SUMS = ROWS + 4 * 2 * 8 * CHUNK, GATES = SUMS + 4 * (5 * CHUNK + 8), BYTES = GATES + (int)sizeof(Gates);
};

template <typename T> __device__ __forceinline__ void row4(T (&x)[4], const T *row, int at, int K)
{
    if (row && at + 4 <= K) __builtin_memcpy(x, row + at, sizeof x);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = row && at + i < K ? row[at + i] : from_f32<T>(0.0f);
}
__device__ __forceinline__ float entry(const Exact<float> &x, int i) { return x.e[i]; }
__device__ __forceinline__ float entry(const Exact<bf16_t> &x, int i) { return (float)x.v[i]; }

// the entry of the fragments that row 4 q + r of a lane's tile t is
template <typename T> __device__ __forceinline__ float entry(const Exact<T> (&f)[2], int t, int r) { return t & 1 ? (t & 2 ? entry(f[1], 4 + r) : entry(f[0], 4 + r)) : t & 2 ? entry(f[1], r) : entry(f[0], r); }

// One workgroup a unit, by its registers: 1024 chunks of 128 x 128 in bf16 149 us, four one after the other on a unit.  193 MB come and go (38 us at a copy's rate) and the matrix units work
// for 19 us; two wavefronts a SIMD do not hide more of each other's waiting.  90 chunks of 37 x 53 in binary32 22.
//
// A workgroup for a chunk of a head.  SHARED: other heads have the same queries and keys, whose gradients leave in binary32, to be added up.
//
// The gradient of the logarithm of a step's decay is the sum of what passes the step: C[i][j], the part of the gradient that goes through G[i][j], of all pairs j < step <= i, and of the
// state before the chunk and its end.  (Those are also a difference of sums, q . dq - v . dv of the steps from it on, in which what does not pass it cancels, and with
// strong decays all digits: 1.7e-4 of dA's values against 64 bits, 512 x 16 steps of 8 heads.)
template <typename T, int KP, bool SHARED> __global__ __launch_bounds__(512) void grads_kernel(const DeltaArgs a)
{
    typedef GradLds<T, KP> L;
    typedef Num<T> N_;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int KT = KP / 16, IT = KT / 2;
    const hts_delta_rule_desc &d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quad = lane >> 4;
    const int64_t unit = blockIdx.x;
    const int h = (int)(unit % d.H), n = (int)(unit / d.H % d.N), c = (int)(unit / d.H / d.N), group = h / (d.H / d.G), t0 = c * CHUNK, len = length_of(a, n);
    const int K = d.K, V = d.V, steps = d.T - t0 < CHUNK ? d.T - t0 : CHUNK;
    float *part = a.part + ((int64_t)c * d.N + n) * 2 * d.H;
    if (t0 >= len) {
        for (int i = wave; i < steps; i += 8) {
            if constexpr (!SHARED)
                for (int k = lane; k < K; k += 64) step_of<T>(a.g.dq, t0 + i, n)[(int64_t)group * K + k] = step_of<T>(a.g.dk, t0 + i, n)[(int64_t)group * K + k] = from_f32<T>(0.0f);
            for (int v = lane; v < V; v += 64) step_of<T>(a.g.dv, t0 + i, n)[(int64_t)h * V + v] = from_f32<T>(0.0f);
            if (lane == 0) step_of<T>(a.g.da, t0 + i, n)[h] = step_of<T>(a.g.db, t0 + i, n)[h] = from_f32<T>(0.0f);
        }
        if (tid == 0) part[h] = part[d.H + h] = 0.0f;
        return;
    }
    // with the states: keys 16 kt .. and tiles first_tile ..; of the steps among themselves: rows 16 ti .., by the outputs' gradients (wavefronts 0 .. 3) or by the values' (4 .. 7)
    const int kt = wave % KT, first_tile = wave / KT * IT, ti = wave & 3;
    const bool by_values = wave >= 4;
    const float sign = sign_of(c, n);
    const auto tile_row = [](int t, int m) { return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3); };
    char *matrix = lds + L::MATRIX;
    float *passing = (float *)(lds + L::PASSING), *rows = (float *)(lds + L::ROWS);       // rows: [2][KT][64] sums along the keys
    float *sums = (float *)(lds + L::SUMS);                                               // [64]: z . dv; 4 x what passes; [8]: <dS', S>
    Exact<T> kf[2], qf[2];
    const int my_row = tid >> 3, my_part = tid & 7;
    const bool my_live = t0 + my_row < len;
    static_assert(sizeof(Gates) % 16 == 0, "whole pieces");
    if (tid < (int)sizeof(Gates) / 16) *(u32x4 *)(lds + L::GATES + 16 * tid) = ((const u32x4 *)(a.gates + unit))[tid];       // read by every part from here on
    const Gates &gates = *(const Gates *)(lds + L::GATES);
    f32x4 by_step[4] = {};                                   // rows 16 ti .. with columns 16 jt ..
    f32x4 q_state[IT] = {}, k_late[IT] = {}, k_state[IT] = {};
    float z_dv = 0.0f, end = 0.0f;
    const float my_strength = a.gates[unit].strength[my_row];
    float z[4], g[4], s8[8], l8[8], next_s[8], next_l[8];
    T y[4];
    const bool whole = t0 + CHUNK <= len;
    const uint32_t my_at = row_at<float>(my_row, a.VP, 4 * my_part), my_y = row_at<T>(my_row, a.dy.st, 4 * my_part), my_dv = row_at<T>(my_row, a.g.dv.st, 4 * my_part);
    const uint32_t state_at = row_at<float>(16 * kt + col, a.VP, 8 * quad);
    const auto load = [&](int v0) {
        __builtin_memcpy(z, (const char *)(a.z + unit * CHUNK * a.VP + v0) + my_at, 16);
        __builtin_memcpy(g, (const char *)(a.write + unit * CHUNK * a.VP + v0) + my_at, 16);
        if (whole && v0 + TILE <= V) __builtin_memcpy(y, (const char *)(step_of<T>(a.dy, t0, n) + (int64_t)h * V + v0) + my_y, sizeof y);
        else row4(y, my_live ? step_of<T>(a.dy, t0 + my_row, n) + (int64_t)h * V : nullptr, v0 + 4 * my_part, V);
    };
    const auto load_states = [&](int v0) {
        __builtin_memcpy(next_s, (const char *)(a.states + unit * KP * a.VP + v0) + state_at, 32);
        __builtin_memcpy(next_l, (const char *)(a.late + unit * KP * a.VP + v0) + state_at, 32);
    };
    const auto fragment = [&](const char *base, int s) { return get_exact<T>(base + (unit * (KP / 8) + kt * 2 + s) * N_::EXACT_FRAGMENT + lane * 16, 1024); };
    f32x4 pass[4] = {};
    // the states, most of what is read, come two tiles ahead, the rest one (there are no registers for more, nor, meanwhile, for what the products after the loop take)
    load_states(0);
    __builtin_memcpy(s8, next_s, 32); __builtin_memcpy(l8, next_l, 32);
    load(0);
    if (TILE < V) load_states(TILE);
    for (int v0 = 0, turn = 0; v0 < V; v0 += TILE, turn ^= 1) {
        char *writes = lds + turn * L::STAGE + L::WRITES, *values = lds + turn * L::STAGE + L::VALUES, *given = lds + turn * L::STAGE + L::GIVEN;
        {
            const int p = L::row_of(my_row, L::PITCH) + (my_part >> 1) * N_::WIDE;
            float u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { z_dv = __builtin_fmaf(z[i], g[i], z_dv); u[i] = sign * my_strength * z[i]; }
            put_wide4<T>(writes + p, 16, my_part & 1, u);
            put_wide4<T>(values + p, 16, my_part & 1, g);
            __builtin_memcpy(given + L::row_of(my_row, L::Y_PITCH) + 4 * my_part * sizeof(T), y, sizeof y);
            if (whole && v0 + TILE <= V) {
                Four<T> o;
#pragma unroll
                for (int i = 0; i < 4; ++i) o.e[i] = from_f32<T>(g[i]);
                store_at(step_of<T>(a.g.dv, t0, n) + (int64_t)h * V + v0, my_dv, o);
            } else if (my_row < steps) {
                const int v = v0 + 4 * my_part;
                store4(step_of<T>(a.g.dv, t0 + my_row, n) + (int64_t)h * V + v, g, V - v);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) { end = __builtin_fmaf(s8[i], l8[i], end); s8[i] *= sign; }
        const Wide<T> sf = make_wide<T>(s8), lf = make_wide<T>(l8);
        __builtin_memcpy(s8, next_s, 32); __builtin_memcpy(l8, next_l, 32);
        if (v0 + TILE < V) load(v0 + TILE);
        if (v0 + 2 * TILE < V) load_states(v0 + 2 * TILE);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < IT; ++t) {
            const int row = tile_row(first_tile + t, col);
            mma(q_state[t], get_exact<T>(given + L::row_of(row, L::Y_PITCH) + quad * N_::EXACT, 16), sf);
            mma(k_state[t], get_wide<T>(values + L::row_of(row, L::PITCH) + quad * N_::WIDE, 16), sf);
            mma(k_late[t], get_wide<T>(writes + L::row_of(row, L::PITCH) + quad * N_::WIDE, 16), lf);
        }
        const Exact<T> yf = get_exact<T>(given + L::row_of(16 * ti + col, L::Y_PITCH) + quad * N_::EXACT, 16);
        const Wide<T> gf = get_wide<T>(values + L::row_of(16 * ti + col, L::PITCH) + quad * N_::WIDE, 16);
#pragma unroll
        for (int jt = 0; jt < 4; ++jt)
            if (jt <= ti) {
                const Wide<T> u = get_wide<T>(writes + L::row_of(16 * jt + col, L::PITCH) + quad * N_::WIDE, 16);
                if (by_values) mma(by_step[jt], gf, u);
                else mma(by_step[jt], yf, u);
            }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) { kf[s] = fragment(a.keys, s); qf[s] = fragment(a.queries, s); }
#pragma unroll
    for (int jt = 0; jt < 4; ++jt)
        if (jt <= ti) pass[jt] = load_at<f32x4>(a.pairs + ((unit * 2 + by_values) * PAIRS + pair_of(ti, jt)) * 256, lane * 16);
    // sums along the keys of what goes through the state before the chunk, and through the one at its end
#pragma unroll
    for (int t = 0; t < IT; ++t) {
        const int tt = first_tile + t, step = tile_row(tt, 4 * quad);
        float keep[4], left[4], q_unit[4], k_unit[4];
        __builtin_memcpy(keep, gates.keep + step, 16); __builtin_memcpy(left, gates.left + step, 16);
        __builtin_memcpy(q_unit, gates.q_unit + step, 16); __builtin_memcpy(k_unit, gates.k_unit + step, 16);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float kv = entry(kf, tt, r) * k_unit[r];
            const float qv = entry(qf, tt, r) * (q_unit[r] * d.scale);
            float from_state = 0.0f, from_late = 0.0f;
            if (keep[r] >= 0.0f) {
                q_state[t][r] *= sign * keep[r];
                k_state[t][r] *= sign * keep[r];
                from_state = __builtin_fmaf(qv, q_state[t][r], -kv * k_state[t][r]);
            } else q_state[t][r] = k_state[t][r] = 0.0f;
            if (left[r] >= 0.0f) {
                k_late[t][r] *= sign * left[r];
                from_late = kv * k_late[t][r];
            } else k_late[t][r] = 0.0f;
            k_late[t][r] -= k_state[t][r];
            from_state = add16(from_state); from_late = add16(from_late);
            if (col == 0) { rows[kt * CHUNK + step + r] = from_state; rows[(KT + kt) * CHUNK + step + r] = from_late; }
        }
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) z_dv += __shfl_xor(z_dv, o, 64);
    if (my_part == 0) sums[my_row] = z_dv;
    end = wave_add(first_tile == 0 ? end : 0.0f);
    if (lane == 0) sums[5 * CHUNK + wave] = end;
    // the steps among themselves, each pair's decay on it
    const int row = 16 * ti + 4 * quad, i_seen = 16 * ti + col;
    {
        double far_i[4];
        int ep_i[4];
        __builtin_memcpy(far_i, gates.far + row, 32); __builtin_memcpy(ep_i, gates.episode + row, 16);
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) {
            if (jt > ti) continue;
            const int j = 16 * jt + col;
            const double far_j = gates.far[j];
            const int ep_j = gates.episode[j];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = row + r;
                const bool sees = (by_values ? j < i : j <= i) && ep_j == ep_i[r];
                const float x = sees ? by_step[jt][r] * exp2_wide(far_i[r] - far_j) : 0.0f;
                by_step[jt][r] = by_values ? -sign * x : sign * x;
                pass[jt][r] = sees && j < i ? by_step[jt][r] * pass[jt][r] : 0.0f;
            }
        }
    }
    const uint64_t bad_q = gates.bad_q, bad_k = gates.bad_k;
    const auto product = [&](f32x4 (&out)[IT], const Exact<T> (&f)[2]) {
#pragma unroll
        for (int t = 0; t < IT; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) mma(out[t], get_wide<T>(matrix + L::row_of(tile_row(first_tile + t, col), L::MATRIX_PITCH) + (4 * s + quad) * N_::WIDE, 16), f[s]);
    };
    const auto put_matrix = [&](int r, int at, const float (&x)[4]) { put_wide4<T>(matrix + L::row_of(r, L::MATRIX_PITCH) + (at >> 3) * N_::WIDE, 16, (at >> 2) & 1, x); };
    const auto put_one = [&](int r, int at, float x) { put_wide1<T>(matrix + L::row_of(r, L::MATRIX_PITCH) + (at >> 3) * N_::WIDE, 16, at & 7, x); };
    const float none[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    __syncthreads();
    // dQ: rows are the steps that look back
    if (!by_values) {
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) {
            if (jt > ti) { put_matrix(i_seen, 16 * jt + 4 * quad, none); continue; }
            const float unit_j = gates.k_unit[16 * jt + col];
#pragma unroll
            for (int r = 0; r < 4; ++r) put_one(row + r, 16 * jt + col, by_step[jt][r] * unit_j);
        }
    } else {
#pragma unroll
        for (int jt = 0; jt < 4; ++jt)
#pragma unroll
            for (int r = 0; r < 4; ++r) passing[(row + r) * L::LINE + 16 * jt + col] = jt <= ti ? pass[jt][r] : 0.0f;
    }
    __syncthreads();
    product(q_state, kf);
    __syncthreads();
    // dK by the queries: rows are the steps that are looked at
    if (!by_values) {
        float unit_i[4];
        __builtin_memcpy(unit_i, gates.q_unit + row, 16);
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) {
            float x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = jt <= ti && !(bad_q >> (row + r) & 1) ? by_step[jt][r] * (unit_i[r] * d.scale) : 0.0f;
                if (jt <= ti) passing[(row + r) * L::LINE + 16 * jt + col] += pass[jt][r];
            }
            put_matrix(16 * jt + col, row, x);
        }
    }
    __syncthreads();
    product(k_late, qf);
    __syncthreads();
    // dK by the keys, on both sides: X + X^T
    if (by_values) {
        float unit_i[4];
        __builtin_memcpy(unit_i, gates.k_unit + row, 16);
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) {
            if (jt > ti) continue;
            const int j = 16 * jt + col;
            const float unit_j = gates.k_unit[j];
            float x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = by_step[jt][r] * unit_i[r];
                if (jt < ti || j < row + r) put_one(row + r, j, by_step[jt][r] * unit_j);
                if (jt == ti && j < row + r) put_one(j, row + r, x[r]);
                if (jt == ti && j == row + r) put_one(j, j, 0.0f);
            }
            if (jt < ti) put_matrix(j, row, x);
        }
    } else {
        // what passes, along each row up to a column: 16 columns a thread, and those of the threads before it
        const int r = tid >> 2, p = tid & 3;
        float *line = passing + r * L::LINE + 16 * p, x = 0.0f, below[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) { below[j] = x; x += line[j]; }
        float before = 0.0f;
#pragma unroll
        for (int o = 0; o < 3; ++o) {
            const float other = __shfl(x, (lane & ~3) + o, 64);
            if (o < p) before += other;
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) line[j] = before + below[j];
    }
    __syncthreads();
    product(k_late, kf);
    if (wave < 4) {
        // ... and down a column from its row on
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = 16 * wave + i;
            if (at >= lane) x += passing[at * L::LINE + lane];
        }
        sums[(1 + wave) * CHUNK + lane] = x;
    }
    __syncthreads();
    if (wave == 0) {
        // the gates
        const int t = t0 + lane;
        const bool live = t < len;
        float after = 0.0f, earlier = 0.0f;                  // of the state before the chunk: this step's and later ones; at its end: earlier ones
#pragma unroll
        for (int k = 0; k < KT; ++k) { after += rows[k * CHUNK + lane]; earlier += rows[(KT + k) * CHUNK + lane]; }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const float x = __shfl_down(after, o, 64), w = __shfl_up(earlier, o, 64);
            if (lane + o < 64) after += x;
            if (lane >= o) earlier += w;
        }
        earlier = __shfl_up(earlier, 1, 64);
        float grad = after + (lane > 0 ? earlier : 0.0f) + ((sums[CHUNK + lane] + sums[2 * CHUNK + lane]) + (sums[3 * CHUNK + lane] + sums[4 * CHUNK + lane]));
        const float all = gates.keep[CHUNK - 1];
        if (all >= 0.0f) {
            float held = 0.0f;
#pragma unroll
            for (int w = 0; w < 8; ++w) held += sums[5 * CHUNK + w];
            grad += all * held;
        }
        float da = 0.0f, dA = 0.0f;
        if (live) {
            const Decay dc = decay_of(to_f32(step_of<T>(a.in.a, t, n)[h]), a.in.a_bias ? a.in.a_bias[h] : 0.0f, a.in.A[h], d.softplus);
            if (!(gates.resets >> lane & 1)) { da = grad * a.in.A[h] * dc.slope; dA = grad * dc.delta; }
            if (bad_k >> lane & 1) da = dA = __builtin_nanf("");
            step_of<T>(a.g.da, t, n)[h] = from_f32<T>(da);
            step_of<T>(a.g.db, t, n)[h] = from_f32<T>(gates.rest[lane] * sums[lane]);
        } else if (t < d.T) step_of<T>(a.g.da, t, n)[h] = step_of<T>(a.g.db, t, n)[h] = from_f32<T>(0.0f);
        dA = wave_add(dA); da = wave_add(da);
        if (lane == 0) { part[h] = dA; part[d.H + h] = da; }
    }
    __syncthreads();                                         // (the sums have been read, and the matrix)
    if constexpr (SHARED) {
#pragma unroll
        for (int t = 0; t < IT; ++t) {
            const int step = tile_row(first_tile + t, 4 * quad), k = 16 * kt + col;
            if (k < K)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    a.heads[((2 * unit + 0) * CHUNK + step + r) * K + k] = q_state[t][r];
                    a.heads[((2 * unit + 1) * CHUNK + step + r) * K + k] = k_late[t][r];
                }
        }
        return;
    }
    // back through the lengths, and out
    if (d.normalize) {
#pragma unroll
        for (int t = 0; t < IT; ++t) {
            const int tt = first_tile + t, step = tile_row(tt, 4 * quad);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float q_dq = add16(entry(qf, tt, r) * q_state[t][r]);
                const float k_dk = add16(entry(kf, tt, r) * k_late[t][r]);
                if (col == 0) { rows[kt * CHUNK + step + r] = q_dq; rows[(KT + kt) * CHUNK + step + r] = k_dk; }
            }
        }
        __syncthreads();
        if (tid < 2 * CHUNK) {
            float x = 0.0f;
#pragma unroll
            for (int k = 0; k < KT; ++k) x += rows[(tid / CHUNK * KT + k) * CHUNK + tid % CHUNK];
            sums[tid] = x;
        }
        __syncthreads();
    }
    char *out_q = lds, *out_k = lds + CHUNK * L::OUT_PITCH;
#pragma unroll
    for (int t = 0; t < IT; ++t) {
        const int tt = first_tile + t, step = tile_row(tt, 4 * quad);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float x = d.scale * q_state[t][r], w = k_late[t][r];
            if (d.normalize) {
                const float q_unit = gates.q_unit[step + r], k_unit = gates.k_unit[step + r];
                const float q_dq = sums[step + r], k_dk = sums[CHUNK + step + r];
                const float qv = entry(qf, tt, r), kv = entry(kf, tt, r);
                x = q_unit * (x - q_unit * qv * (q_unit * d.scale * q_dq));
                w = k_unit * (w - k_unit * kv * (k_unit * k_dk));
                if (bad_k >> (step + r) & 1) w = __builtin_nanf("");
            }
            *(T *)(out_q + (step + r) * L::OUT_PITCH + (16 * kt + col) * sizeof(T)) = from_f32<T>(x);
            *(T *)(out_k + (step + r) * L::OUT_PITCH + (16 * kt + col) * sizeof(T)) = from_f32<T>(w);
        }
    }
    __syncthreads();
    constexpr int PIECE = 16 / (int)sizeof(T), PIECES = KP / PIECE;
    for (int p = tid; p < 2 * CHUNK * PIECES; p += 512) {
        const int which = p / (CHUNK * PIECES), i = p / PIECES % CHUNK, at = p % PIECES * PIECE, count = K - at;
        if (i >= steps || count <= 0) continue;
        T *to = step_of<T>(which ? a.g.dk : a.g.dq, t0 + i, n) + (int64_t)group * K + at, x[PIECE];
        __builtin_memcpy(x, __builtin_assume_aligned((which ? out_k : out_q) + i * L::OUT_PITCH + at * sizeof(T), 16), 16);
        if (t0 + i >= len)
#pragma unroll
            for (int e = 0; e < PIECE; ++e) x[e] = from_f32<T>(0.0f);
        if (count >= PIECE) __builtin_memcpy(to, x, 16);
        else
#pragma unroll
            for (int e = 0; e < PIECE; ++e) if (e < count) to[e] = x[e];
    }
}

// Queries and keys of several heads: their gradients added up, back through the lengths, and out.  A wavefront for a step of a group.
// (129 x 5 steps, 3 groups of 2 heads: 4.6 us, a launch.)
template <typename T> __global__ __launch_bounds__(256) void join_kernel(const DeltaArgs a)
{
    const hts_delta_rule_desc &d = a.d;
    const int lane = threadIdx.x & 63, i = (int)(blockIdx.x % (CHUNK / 4)) * 4 + (threadIdx.x >> 6), per = d.H / d.G, K = d.K;
    const int64_t of = blockIdx.x / (CHUNK / 4);
    const int group = (int)(of % d.G), n = (int)(of / d.G % d.N), c = (int)(of / d.G / d.N), t = c * CHUNK + i;
    if (t >= d.T) return;
    const bool live = t < length_of(a, n);
    const int64_t unit = ((int64_t)c * d.N + n) * d.H + group * per;
    float q[2] = {}, k[2] = {}, dq[2] = {}, dk[2] = {}, q_dq = 0.0f, k_dk = 0.0f;
    if (live) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int at = lane + 64 * e;
            if (at >= K) continue;
            q[e] = to_f32(step_of<T>(a.in.q, t, n)[(int64_t)group * K + at]);
            k[e] = to_f32(step_of<T>(a.in.k, t, n)[(int64_t)group * K + at]);
            for (int h = 0; h < per; ++h) {
                dq[e] += a.heads[((2 * (unit + h) + 0) * CHUNK + i) * K + at];
                dk[e] += a.heads[((2 * (unit + h) + 1) * CHUNK + i) * K + at];
            }
            q_dq = __builtin_fmaf(q[e], dq[e], q_dq);
            k_dk = __builtin_fmaf(k[e], dk[e], k_dk);
        }
        if (d.normalize) {
            const float q_unit = a.gates[unit].q_unit[i], k_unit = a.gates[unit].k_unit[i];
            q_dq = wave_add(q_dq); k_dk = wave_add(k_dk);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                dq[e] = q_unit * (d.scale * dq[e] - q_unit * q[e] * (q_unit * d.scale * q_dq));
                dk[e] = k_unit * (dk[e] - k_unit * k[e] * (k_unit * k_dk));
            }
        } else { dq[0] *= d.scale; dq[1] *= d.scale; }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int at = lane + 64 * e;
        if (at >= K) continue;
        step_of<T>(a.g.dq, t, n)[(int64_t)group * K + at] = from_f32<T>(dq[e]);
        step_of<T>(a.g.dk, t, n)[(int64_t)group * K + at] = from_f32<T>(dk[e]);
    }
}

// ---- launches ---------------------------------------------------------------------------------------------------------------
// (more LDS than 64 KB has to be asked for)
template <class F> hipError_t launch(F kernel, int64_t groups, int lds, hipStream_t stream, const DeltaArgs &a, int threads = 256, int segments = 1)
{
    if (!launchable(groups, threads)) return hipErrorInvalidConfiguration;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((uint32_t)groups, (uint32_t)segments), dim3(threads), (uint32_t)lds, stream, a);
    return hipGetLastError();
}
template <typename F> hipError_t by_keys(int K, F f)
{
    if (K <= 32) return f(std::integral_constant<int, 32>{});
    if (K <= 64) return f(std::integral_constant<int, 64>{});
    return f(std::integral_constant<int, 128>{});
}


// Segments: as many as a device of 256 units has room for beside each other, of 4 chunks or more, where there are three of them at least (with two the passes over the segments'
// ends cost what they save).  The same on every device and range of units: results do not depend on where they are computed.
struct Segments { int count, chunks; };
Segments segments_of(const hts_delta_rule_desc &d)
{
    const int64_t chunks = ceil_div(d.T, CHUNK), groups = (int64_t)d.N * d.H * ceil_div(d.V, TILE);
    int64_t count = ROOM / groups;
    if (count > chunks / 4) count = chunks / 4;
    if (count < 3) return Segments{1, (int)chunks};
    const int64_t each = ceil_div(chunks, count);
    return Segments{(int)ceil_div(chunks, each), (int)each};
}
// ... their arrays, for the most that any number of sequences has
int64_t most_places(const hts_delta_rule_desc &d)
{
    if (ceil_div(d.T, CHUNK) < 12) return 0;
    return ROOM / ceil_div(d.V, TILE);
}

struct Layout { int64_t ends, begins, powers, inverse, read, keys, queries, pairs, rows, gates, late, write, part, heads, total; };
Layout layout(const hts_delta_rule_desc &d, bool back)
{
    const int64_t units = ceil_div(d.T, CHUNK) * d.N * d.H, wide = d.precision == HTS_PRECISION_BF16 ? Num<bf16_t>::WIDE_FRAGMENT : Num<float>::WIDE_FRAGMENT, exact = d.precision == HTS_PRECISION_BF16 ? Num<bf16_t>::EXACT_FRAGMENT : Num<float>::EXACT_FRAGMENT;
    Layout l;
    const int64_t KP = keys_padded(d.K), VP = round_up(d.V, TILE), places = back ? 0 : most_places(d);
    l.ends = 0;
    l.begins = l.ends + 4 * places * KP * (VP + KP);
    l.powers = l.begins + 4 * places * KP * VP;
    l.inverse = l.powers + round_up(4 * places * (KP / TILE), 256);
    l.read = l.inverse + units * 8 * wide;
    l.keys = l.read + units * 8 * wide;
    l.queries = l.keys + units * (keys_padded(d.K) / 8) * exact;
    l.pairs = l.queries + (back ? units * (keys_padded(d.K) / 8) * exact : 0);
    l.rows = l.pairs + (back ? units * 2 * PAIRS * 1024 : 0);
    l.gates = l.rows + (d.K % 8 ? units * 2 * (keys_padded(d.K) / 8) * exact : 0);
    l.late = l.gates + round_up(units * (int64_t)sizeof(Gates), 256);
    l.write = l.late + (back ? units * keys_padded(d.K) * round_up(d.V, TILE) * 4 : 0);
    l.part = l.write + (back ? units * CHUNK * round_up(d.V, TILE) * 4 : 0);
    l.heads = l.part + (back ? round_up(ceil_div(d.T, CHUNK) * d.N * 2 * d.H * 4, 256) : 0);
    l.total = l.heads + (back && d.H > d.G ? units * 2 * CHUNK * d.K * 4 : 0);
    return l;
}
DeltaArgs arguments(hts_seq_ctx &c, const DeltaOp &op, bool back)
{
    const Layout l = layout(op.d, back);
    DeltaArgs a = {};
    a.d = op.d; a.in = op.in; a.y = op.y; a.dy = op.dy; a.h_out = op.h_out; a.states = op.states; a.dh_out = op.dh_out; a.g = op.g;
    a.chunks = (int)ceil_div(op.d.T, CHUNK);
    const Segments seg = segments_of(op.d);
    a.segments = back ? 1 : seg.count; a.per_segment = back ? a.chunks : seg.chunks;
    a.ends = (float *)(c.ws + l.ends); a.begins = (float *)(c.ws + l.begins); a.powers = (int32_t *)(c.ws + l.powers);
    a.tiles = (int)ceil_div(op.d.V, TILE); a.VP = a.tiles * TILE;
    if (op.states) a.z = op.states + delta_state_floats(op.d);
    a.inverse = a.inverse_t = c.ws + l.inverse; a.read = c.ws + l.read; a.keys = c.ws + l.keys; a.queries = c.ws + l.queries; a.gates = (Gates *)(c.ws + l.gates); a.pairs = (float *)(c.ws + l.pairs); a.rows = op.d.K % 8 ? c.ws + l.rows : nullptr;
    a.late = (float *)(c.ws + l.late); a.write = (float *)(c.ws + l.write); a.part = (float *)(c.ws + l.part); a.heads = (float *)(c.ws + l.heads);
    return a;
}
// whether every launch of a call is within what the runtime takes: none is made otherwise
bool fits(const DeltaArgs &a, bool back)
{
    const int64_t units = (int64_t)a.chunks * a.d.N * a.d.H;
    if (!launchable(units, back ? 512 : 256) || !launchable(parts(a, a.tiles), 256)) return false;
    return !back || a.d.H == a.d.G || launchable((int64_t)a.chunks * a.d.N * a.d.G * (CHUNK / 4), 256);
}
template <typename T> hipError_t forward(hts_seq_ctx &c, const DeltaOp &op)
{
    const hts_delta_rule_desc &d = op.d;
    DeltaArgs a = arguments(c, op, false);
    if (d.T <= MOST_STEPS) {
        a.tiles = (int)ceil_div(d.V, STEP_TILE);
        return launch(step_kernel<T>, (int64_t)d.N * d.H * a.tiles, 0, c.stream, a);
    }
    if (!fits(a, false)) return hipErrorInvalidConfiguration;
    return by_keys(d.K, [&](auto kp) {
        constexpr int KP = decltype(kp)::value;
        hipError_t e = launch(prep_kernel<T, KP, false>, (int64_t)a.chunks * d.N * d.H, PrepLds<T, KP>::BYTES, c.stream, a);
        if (e == hipSuccess && a.segments > 1) {
            e = launch(forward_kernel<T, KP, true>, parts(a, a.tiles + KP / TILE), RunLds<T, KP>::BYTES, c.stream, a, 256, a.segments - 1);
            if (e == hipSuccess) e = launch(begin_kernel<T, KP>, parts(a, a.tiles), 0, c.stream, a, 4 * KP);
        }
        return e != hipSuccess ? e : launch(forward_kernel<T, KP, false>, parts(a, a.tiles), RunLds<T, KP>::BYTES, c.stream, a, 256, a.segments);
    });
}
template <typename T> hipError_t backward(hts_seq_ctx &c, const DeltaOp &op)
{
    const hts_delta_rule_desc &d = op.d;
    const DeltaArgs a = arguments(c, op, true);
    if (!fits(a, true)) return hipErrorInvalidConfiguration;
    const hipError_t e = by_keys(d.K, [&](auto kp) {
        constexpr int KP = decltype(kp)::value;
        hipError_t e = launch(prep_kernel<T, KP, true>, (int64_t)a.chunks * d.N * d.H, PrepLds<T, KP>::BYTES, c.stream, a);
        if (e == hipSuccess) e = launch(reverse_kernel<T, KP>, parts(a, a.tiles), RunLds<T, KP>::BACK_BYTES, c.stream, a);
        if (e == hipSuccess) e = launch(d.H > d.G ? grads_kernel<T, KP, true> : grads_kernel<T, KP, false>, (int64_t)a.chunks * d.N * d.H, GradLds<T, KP>::BYTES, c.stream, a, 512);
        if (e == hipSuccess && d.H > d.G) e = launch(join_kernel<T>, (int64_t)a.chunks * d.N * d.G * (CHUNK / 4), 0, c.stream, a);
        return e;
    });
    if (e != hipSuccess) return e;
    return launch_sum_partials(c, a.part, (int64_t)a.chunks * d.N, 2 * (int64_t)d.H, SumTarget{op.g.dA, d.H}, SumTarget{op.g.da_bias, d.H}, SumTarget{nullptr, 0});
}
}  // namespace

int64_t delta_workspace(const hts_delta_rule_desc &d, bool back) { return !back && d.T <= MOST_STEPS ? 0 : layout(d, back).total; }
int64_t delta_state_floats(const hts_delta_rule_desc &d) { return ceil_div(d.T, CHUNK) * d.N * d.H * keys_padded(d.K) * round_up(d.V, TILE); }
int64_t delta_states(const hts_delta_rule_desc &d) { return delta_state_floats(d) + ceil_div(d.T, CHUNK) * CHUNK * d.N * d.H * round_up(d.V, TILE); }

hipError_t launch_delta(hts_seq_ctx &c, const DeltaOp &op) { return op.d.precision == HTS_PRECISION_BF16 ? forward<bf16_t>(c, op) : forward<float>(c, op); }
hipError_t launch_delta_backward(hts_seq_ctx &c, const DeltaOp &op) { return op.d.precision == HTS_PRECISION_BF16 ? backward<bf16_t>(c, op) : backward<float>(c, op); }

}  // namespace hts
