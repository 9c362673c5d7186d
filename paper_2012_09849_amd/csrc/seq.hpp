// Sequence memory: declarations and device helpers shared by linear.hip, shortconv.hip, scan.hip and seqapi.hip (not part of the C ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/hts.h"
#include "gemm.hpp"

struct hts_seq_ctx {
    hipStream_t stream;
    int cus;                  // compute units that the stream's kernels run on
    char *ws;
    int64_t bytes;
};

namespace hts {

int stream_cus(hipStream_t stream);       // api.hip

struct LinearOp {
    int M, N, K, act;
    hts_rows x, w, residual, y, pre, dy, add, dx;
    const float *bias;
    float *dw, *db;
};
struct ConvOp {
    int T, N, D, W, act;
    hts_steps x, y, dy, dx;
    const float *w, *bias, *state_in, *dstate_out;
    float *state_out, *dw, *db, *dstate_in;
    const uint8_t *starts;
    const int32_t *lengths;
};
struct ScanOp {
    hts_scan_desc d;
    hts_scan_inputs in;
    hts_steps y, dy;
    float *h_out, *states_out;
    const float *dh_out, *states;
    hts_scan_grads g;
};

int64_t linear_workspace(int precision, int act, int64_t M, int64_t N, int64_t K);      // of the backward call; the forward call needs none
int64_t conv_workspace(int64_t T, int64_t N, int64_t D, int W);
int64_t scan_workspace(const hts_scan_desc &d, bool backward);
int64_t scan_states(const hts_scan_desc &d);
hipError_t launch_linear(hts_seq_ctx &c, int precision, const LinearOp &op);
hipError_t launch_linear_backward(hts_seq_ctx &c, int precision, const LinearOp &op);
hipError_t launch_conv(hts_seq_ctx &c, int precision, const ConvOp &op);
hipError_t launch_conv_backward(hts_seq_ctx &c, int precision, const ConvOp &op);
hipError_t launch_scan(hts_seq_ctx &c, const ScanOp &op);
hipError_t launch_scan_backward(hts_seq_ctx &c, const ScanOp &op);

// out = sum over p of part[p][0 .. width), in a fixed order; consecutive entries go to up to three arrays (p NULL: not wanted)
struct SumTarget { float *p; int64_t n; };
hipError_t launch_sum_partials(hts_seq_ctx &c, const float *part, int64_t parts, int64_t width, SumTarget a, SumTarget b, SumTarget d);
// the same by a workgroup of ROWS wavefronts for 64 neighbouring entries: a wavefront takes every ROWS-th partial sum, 4 of them at a time
template <int ROWS> __device__ __forceinline__ void sum_partials(float (&sums)[ROWS][64], const int64_t block, const float *part, const int64_t parts, const int64_t width, const SumTarget &a, const SumTarget &b, const SumTarget &d)
{
    const int lane = threadIdx.x & 63, row = threadIdx.x >> 6;
    int64_t i = block * 64 + lane;
    float s = 0.0f;
    if (i < width) {
        float q[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        int64_t k = row;
        for (; k + 3 * ROWS < parts; k += 4 * ROWS)
#pragma unroll
            for (int u = 0; u < 4; ++u) q[u] += part[(k + ROWS * u) * width + i];
        for (int u = 0; k < parts; k += ROWS, ++u) q[u & 3] += part[k * width + i];
        s = (q[0] + q[1]) + (q[2] + q[3]);
    }
    sums[row][lane] = s;
    __syncthreads();
    if (row || i >= width) return;
    s = 0.0f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) s += sums[r][lane];
    if (i < a.n) { if (a.p) a.p[i] = s; }
    else if ((i -= a.n) < b.n) { if (b.p) b.p[i] = s; }
    else if ((i -= b.n) < d.n) { if (d.p) d.p[i] = s; }
}

// whether a launch of that many workgroups is within what the runtime takes (the grid's threads have 32 bits); hipErrorInvalidConfiguration says that a shape is not
inline bool launchable(int64_t groups, int threads) { return groups * threads < (1ll << 32); }

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

constexpr float LOG2E = 1.44269504088896341f;

// exp, 1 / (1 + exp(-v)): one rounding of the exponent and the matrix unit's neighbours' 1 ulp exp2 and reciprocal; exact limits at both ends
__device__ __forceinline__ float exp_f(float v) { return __builtin_amdgcn_exp2f(v * LOG2E); }
__device__ __forceinline__ float sigmoid_f(float v) { return __builtin_amdgcn_rcpf(1.0f + exp_f(-v)); }
// log(1 + e), 0 <= e <= 1, to a few ulp where 1 + e would lose e's bits: 2 artanh(e / (2 + e)), |argument| <= 1/3, eight terms of its series
__device__ __forceinline__ float log1p_f(float e)
{
    const float w = e * __builtin_amdgcn_rcpf(2.0f + e), q = w * w;
    float p = 1.0f / 17.0f;
    p = __builtin_fmaf(p, q, 1.0f / 15.0f); p = __builtin_fmaf(p, q, 1.0f / 13.0f); p = __builtin_fmaf(p, q, 1.0f / 11.0f);
    p = __builtin_fmaf(p, q, 1.0f / 9.0f); p = __builtin_fmaf(p, q, 1.0f / 7.0f); p = __builtin_fmaf(p, q, 1.0f / 5.0f);
    p = __builtin_fmaf(p, q, 1.0f / 3.0f);
    return __builtin_fmaf(2.0f * w, q * p, 2.0f * w);
}
// softplus and its slope, the logistic function, from one exponential; NaN stays NaN
__device__ __forceinline__ void softplus_f(float v, float &value, float &slope)
{
    const float e = exp_f(-__builtin_fabsf(v)), r = __builtin_amdgcn_rcpf(1.0f + e);
    value = (v > 0.0f ? v : 0.0f) + log1p_f(e);
    slope = v >= 0.0f ? r : e * r;
}

// (the factors are held within finite bounds, so that infinities give the limits, 0 or 1 times themselves, without a branch; NaN comes through the others)
template <int ACT> __device__ __forceinline__ float act_f(float v)
{
    if constexpr (ACT == HTS_ACT_RELU) return v < 0.0f ? 0.0f : v;
    if constexpr (ACT == HTS_ACT_SILU) return fmaxf(v, -1e4f) * sigmoid_f(v);
    if constexpr (ACT == HTS_ACT_GELU) return 0.5f * fmaxf(v, -1e4f) * (1.0f + erff(v * 0.70710678118654752f));
    return v;
}
template <int ACT> __device__ __forceinline__ float act_slope(float v)
{
    const float w = fminf(fmaxf(v, -1e4f), 1e4f);
    if constexpr (ACT == HTS_ACT_RELU) return v > 0.0f ? 1.0f : 0.0f;
    if constexpr (ACT == HTS_ACT_SILU) {
        const float s = sigmoid_f(v);
        return s * __builtin_fmaf(w, 1.0f - s, 1.0f);
    }
    if constexpr (ACT == HTS_ACT_GELU) return 0.5f * (1.0f + erff(v * 0.70710678118654752f)) + w * 0.39894228040143268f * exp_f(-0.5f * v * v);
    return 1.0f;
}
// V entries from memory, or one at a time where their address is no multiple of their size
template <typename T, int V> struct Loaded { T e[V]; };
template <typename T, int V> __device__ __forceinline__ Loaded<T, V> load_v(const T *p)
{
    Loaded<T, V> r;
    __builtin_memcpy(&r, __builtin_assume_aligned(p, sizeof(T) * V), sizeof r);
    return r;
}
template <typename T, int V> __device__ __forceinline__ void store_v(T *p, const Loaded<T, V> &v) { __builtin_memcpy(__builtin_assume_aligned(p, sizeof(T) * V), &v, sizeof v); }

// Loads and stores through buffer descriptors: a base that all lanes share and 32 bits of a lane (and 32 that all lanes share) from it.  A lane that has nothing to
// load or store gets an offset beyond the descriptor's 2 GB: it reads zero and writes nothing, without a branch (values that were loaded on different
// paths would be waited for where the paths meet).
constexpr uint32_t REACH = 1u << 31, NOWHERE = REACH;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t reach(const char *base) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, REACH, 0x00020000); }

// V neighbouring entries of a lane: one access where addresses and counts allow it (WIDE), otherwise an entry at a time, `count` of them
template <typename T, int V, bool WIDE> struct Raw {
    static constexpr int WORDS = WIDE ? (V * (int)sizeof(T) + 3) / 4 : V;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t src, uint32_t lane, int count, uint32_t all = 0)
    {
        if constexpr (WIDE && WORDS == 4) {
            const auto r = __builtin_amdgcn_raw_buffer_load_b128(src, (int)lane, (int)all, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = r[i];
        } else if constexpr (WIDE && WORDS == 2) {
            const auto r = __builtin_amdgcn_raw_buffer_load_b64(src, (int)lane, (int)all, 0);
            w[0] = r[0]; w[1] = r[1];
        } else if constexpr (WIDE && V * sizeof(T) == 4) w[0] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(src, (int)lane, (int)all, 0);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int at = i < count ? (int)(lane + i * (uint32_t)sizeof(T)) : (int)NOWHERE;
                if constexpr (sizeof(T) == 2) w[i] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(src, at, (int)all, 0);
                else w[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(src, at, (int)all, 0);
            }
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else if constexpr (!WIDE || V == 1) return __uint_as_float(w[i] << 16);
        else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
};
template <typename T> __device__ __forceinline__ uint32_t bits_of(float v)
{
    if constexpr (sizeof(T) == 2) return __builtin_bit_cast(uint16_t, from_f32<T>(v));
    else return __float_as_uint(v);
}
template <typename T, int V, bool WIDE> __device__ __forceinline__ void put_raw(__amdgpu_buffer_rsrc_t dst, uint32_t lane, int count, const float (&v)[V], uint32_t all = 0)
{
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    if constexpr (WIDE && V * sizeof(T) >= 4) {
        constexpr int WORDS = V * (int)sizeof(T) / 4;
        uint32_t w[WORDS];
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = sizeof(T) == 4 ? bits_of<T>(v[i]) : bits_of<T>(v[V > 1 ? 2 * i : 0]) | bits_of<T>(v[V > 1 ? 2 * i + 1 : 0]) << 16;
        if constexpr (WORDS == 1) __builtin_amdgcn_raw_buffer_store_b32(w[0], dst, (int)lane, (int)all, 0);
        else if constexpr (WORDS == 2) __builtin_amdgcn_raw_buffer_store_b64(u2{w[0], w[1]}, dst, (int)lane, (int)all, 0);
        else __builtin_amdgcn_raw_buffer_store_b128(u4{w[0], w[1], w[2], w[3]}, dst, (int)lane, (int)all, 0);
    } else
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int at = i < count ? (int)(lane + i * (uint32_t)sizeof(T)) : (int)NOWHERE;
            if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)bits_of<T>(v[i]), dst, at, (int)all, 0);
            else __builtin_amdgcn_raw_buffer_store_b32(bits_of<T>(v[i]), dst, at, (int)all, 0);
        }
}

}  // namespace hts
