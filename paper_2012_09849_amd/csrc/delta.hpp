// Gated delta rule: operands of the matrix instructions, arguments and layouts that delta.hip's kernels share (not part of the C ABI).
//
// Every product is of 16x16x32 blocks, C[m][n] += sum over 32 k of A[m][k] B[n][k]: lane 16 q + r has row r of A and of B, k = 8 q .. 8 q + 7, and of C
// rows 4 q .. 4 q + 3 of column r.  With A and B exchanged it has C transposed, so that a result can be handed on along either of its indices.
//   Exact: entries of the operands' type, as they are in memory.
//   Wide: binary32 numbers.  For bfloat16 operands each is the sum of three bfloat16 numbers (8 bits cut off, the next 8, the last 8: nothing is rounded, and none
//   of the parts leaves bfloat16's range), and a product takes the six pairs of parts that count in binary32, three where the other side is Exact: 6 x 16 cycles of
//   the matrix units, where binary32 instructions take 256.
#pragma once
#include "seq.hpp"

namespace hts {

constexpr int CHUNK = 64;                   // steps that are worked on at a time: a wavefront's lanes for their gates, four tiles of 16

template <typename T> struct Exact;
template <typename T> struct Wide;
template <> struct Exact<float> { float e[8]; };
template <> struct Wide<float> { float e[8]; };
template <> struct Exact<bf16_t> { bf16x8 v; };
template <> struct Wide<bf16_t> { bf16x8 p[3]; };
// 8 neighbouring entries of a row lie together, in planes of 16 bytes
template <typename T> struct Num {
    static constexpr int WIDE_PLANES = sizeof(T) == 4 ? 2 : 3, EXACT_PLANES = sizeof(T) / 2, WIDE = 16 * WIDE_PLANES, EXACT = 16 * EXACT_PLANES;
    static constexpr int WIDE_FRAGMENT = 1024 * WIDE_PLANES, EXACT_FRAGMENT = 1024 * EXACT_PLANES;      // 16 rows of 32 entries in lane order, plane by plane
    static constexpr int pitch(int entries) { return entries / 8 * WIDE + 16; }                          // of rows in LDS: neighbours begin in other banks
    static constexpr int exact_pitch(int entries) { return entries / 8 * EXACT + 16; }
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void mma1(f32x4 &c, const bf16x8 &a, const bf16x8 &b) { c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
template <class A, class B> __device__ __forceinline__ void mma_f32(f32x4 &c, const A &a, const B &b)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.e[i], b.e[i], c, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x4 &c, const Exact<float> &a, const Exact<float> &b) { mma_f32(c, a, b); }
__device__ __forceinline__ void mma(f32x4 &c, const Exact<float> &a, const Wide<float> &b) { mma_f32(c, a, b); }
__device__ __forceinline__ void mma(f32x4 &c, const Wide<float> &a, const Exact<float> &b) { mma_f32(c, a, b); }
__device__ __forceinline__ void mma(f32x4 &c, const Wide<float> &a, const Wide<float> &b) { mma_f32(c, a, b); }
__device__ __forceinline__ void mma(f32x4 &c, const Exact<bf16_t> &a, const Exact<bf16_t> &b) { mma1(c, a.v, b.v); }
// Smallest parts first.  (The instruction drops what lies below C's last digits towards minus infinity, by a few guard digits: 1.4% of a last digit on average where
// products are 2^-15 of C, measured.  Where sums over thousands of steps would add that up, every second chunk has the other sign.)
__device__ __forceinline__ void mma(f32x4 &c, const Exact<bf16_t> &a, const Wide<bf16_t> &b)
{
    mma1(c, a.v, b.p[2]); mma1(c, a.v, b.p[1]); mma1(c, a.v, b.p[0]);
}
__device__ __forceinline__ void mma(f32x4 &c, const Wide<bf16_t> &a, const Exact<bf16_t> &b)
{
    mma1(c, a.p[2], b.v); mma1(c, a.p[1], b.v); mma1(c, a.p[0], b.v);
}
__device__ __forceinline__ void mma(f32x4 &c, const Wide<bf16_t> &a, const Wide<bf16_t> &b)
{
    mma1(c, a.p[2], b.p[0]); mma1(c, a.p[1], b.p[1]); mma1(c, a.p[0], b.p[2]);
    mma1(c, a.p[1], b.p[0]); mma1(c, a.p[0], b.p[1]);
    mma1(c, a.p[0], b.p[0]);
}

template <typename T> __device__ __forceinline__ Exact<T> get_exact(const char *p, int plane)
{
    Exact<T> r;
    if constexpr (sizeof(T) == 4) {
        __builtin_memcpy(r.e, __builtin_assume_aligned(p, 16), 16);
        __builtin_memcpy(r.e + 4, __builtin_assume_aligned(p + plane, 16), 16);
    } else __builtin_memcpy(&r.v, __builtin_assume_aligned(p, 16), 16);
    return r;
}
template <typename T> __device__ __forceinline__ void put_exact(char *p, int plane, const Exact<T> &x)
{
    if constexpr (sizeof(T) == 4) {
        __builtin_memcpy(__builtin_assume_aligned(p, 16), x.e, 16);
        __builtin_memcpy(__builtin_assume_aligned(p + plane, 16), x.e + 4, 16);
    } else __builtin_memcpy(__builtin_assume_aligned(p, 16), &x.v, 16);
}
template <typename T> __device__ __forceinline__ Wide<T> get_wide(const char *p, int plane)
{
    Wide<T> r;
    if constexpr (sizeof(T) == 4) {
        __builtin_memcpy(r.e, __builtin_assume_aligned(p, 16), 16);
        __builtin_memcpy(r.e + 4, __builtin_assume_aligned(p + plane, 16), 16);
    } else
#pragma unroll
        for (int i = 0; i < 3; ++i) __builtin_memcpy(&r.p[i], __builtin_assume_aligned(p + i * plane, 16), 16);
    return r;
}
// two numbers' upper halves
__device__ __forceinline__ uint32_t uppers(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
__device__ __forceinline__ float cut8(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
// 4 neighbouring numbers into the first or second half of 8
template <typename T> __device__ __forceinline__ void put_wide4(char *p, int plane, int half, const float (&x)[4])
{
    if constexpr (sizeof(T) == 4) __builtin_memcpy(__builtin_assume_aligned(p + half * plane, 16), x, 16);
    else {
        float r[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const u32x2 w = {uppers(r[0], r[1]), uppers(r[2], r[3])};
            __builtin_memcpy(__builtin_assume_aligned(p + i * plane + 8 * half, 8), &w, 8);
#pragma unroll
            for (int k = 0; k < 4; ++k) r[k] -= cut8(r[k]);
        }
    }
}
// one number, the i-th of 8
template <typename T> __device__ __forceinline__ void put_wide1(char *p, int plane, int i, float x)
{
    if constexpr (sizeof(T) == 4) *(float *)(p + (i >> 2) * plane + 4 * (i & 3)) = x;
    else {
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            *(uint16_t *)(p + k * plane + 2 * i) = (uint16_t)(__float_as_uint(x) >> 16);
            x -= cut8(x);
        }
    }
}
template <typename T> __device__ __forceinline__ Wide<T> make_wide(const float (&x)[8])
{
    Wide<T> r;
    if constexpr (sizeof(T) == 4) __builtin_memcpy(r.e, x, 32);
    else {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = x[k];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const u32x4 w = {uppers(v[0], v[1]), uppers(v[2], v[3]), uppers(v[4], v[5]), uppers(v[6], v[7])};
            __builtin_memcpy(&r.p[i], &w, 16);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] -= cut8(v[k]);
        }
    }
    return r;
}
template <typename T> __device__ __forceinline__ Exact<T> make_exact(const T (&x)[8])
{
    Exact<T> r;
    __builtin_memcpy(&r, x, sizeof r);
    return r;
}
// entries at .. at + 7 of a row of K in memory (NULL: zeros), zeros behind its end
template <typename T> __device__ __forceinline__ void row8(T (&x)[8], const T *row, int at, int K)
{
    if (row && at + 8 <= K) __builtin_memcpy(x, row + at, sizeof x);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = row && at + i < K ? row[at + i] : from_f32<T>(0.0f);
}
template <typename T> __device__ __forceinline__ Exact<T> exact_row(const T *row, int at, int K)
{
    T x[8];
    row8(x, row, at, K);
    return make_exact<T>(x);
}

// An address as a base that all lanes share and 32 bits of a lane, which an access takes as they are: no arithmetic in vector registers.  (Steps are at most 2^24 entries
// apart, so a chunk's lie within 4 GB of its first one.)
template <typename P> __device__ __forceinline__ P load_at(const void *base, uint32_t at)
{
    P r;
    __builtin_memcpy(&r, (const char *)base + at, sizeof r);
    return r;
}
template <typename P> __device__ __forceinline__ void store_at(void *base, uint32_t at, const P &x) { __builtin_memcpy((char *)base + at, &x, sizeof x); }
template <typename T> __device__ __forceinline__ uint32_t row_at(int64_t row, int64_t distance, int entry) { return (uint32_t)((row * distance + entry) * (int64_t)sizeof(T)); }
template <typename P> struct Four { P e[4]; };
// the same value, which the compiler takes for another: addresses of paths that are hardly ever taken are formed on them, not kept in registers for them
__device__ __forceinline__ int again(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) <= 3.402823466e38f; }
// 2^x for exponents that are sums of up to 64 steps' (each below MOST_EXPONENT in size, or forgets): what is left after the whole part is taken off has binary32's precision
constexpr double MOST_EXPONENT = 4096.0;
__device__ __forceinline__ float exp2_wide(double x)
{
    const double whole = __builtin_rint(x);
    return __builtin_ldexpf(__builtin_amdgcn_exp2f((float)(x - whole)), (int)whole);
}

// What a chunk's steps share with the kernels after the first one.  keep, left: what remains of the state before the chunk at a step, of a step at the chunk's end;
// -1: nothing, an episode began in between (a factor of 0 would make NaN of what is not finite).
struct Gates {
    double far[CHUNK];                    // sums of the decays' exponents (base 2) from the chunk's beginning
    float rest[CHUNK];                    // 1 - strength, by itself: of a strength next to one the difference has no digits left (for the backward call)
    float keep[CHUNK], left[CHUNK], strength[CHUNK], q_unit[CHUNK], k_unit[CHUNK];
    int32_t episode[CHUNK], first[CHUNK]; // episodes that began in the chunk up to a step; the first step of its own
    uint64_t bad_k, bad_q, resets;        // steps whose key or gates, whose query, are not finite; steps that see nothing of what was before
    int32_t pad[2];
};

struct DeltaArgs {
    hts_delta_rule_desc d;
    hts_delta_rule_inputs in;
    hts_steps y, dy;
    float *h_out, *states, *z;                    // states [chunk][N][H][KP][VP]; z [chunk][N][H][64][VP]: v minus what the state had for the key
    const float *dh_out;
    hts_delta_rule_grads g;
    int chunks, tiles, VP;                        // tiles of the values; V in whole tiles (KP: K in whole fragments; zeros in what K, V and a sequence's end leave over)
    char *inverse, *inverse_t, *read, *keys, *queries;     // fragments of each chunk, sequence and head
    float *pairs;                                 // [unit][20][64 lanes][4]: products of queries or keys that look back with keys, all of length one (and scaled), tiles on and below the diagonal
    char *rows;                                   // K no multiple of 8: keys [unit][64][KP], then queries, that rows are read from in eights
    Gates *gates;
    // long sequences of few heads, in segments of so many chunks that are worked on at the same time: what each makes of nothing and of a state of ones on the diagonal,
    // [segment][N][H][KP][VP + KP], and the states that they begin with, [segment][N][H][KP][VP]
    int segments, per_segment;
    float *ends, *begins;
    int32_t *powers;                              // of two, that products with the ends of ones are to be multiplied by: [segment][N][H][KP / 32]
    float *late, *write, *part, *heads;           // gradients of the states at the chunks' ends; of the values; sums of the decays' parameters; of shared queries and keys
};
__device__ __forceinline__ int length_of(const DeltaArgs &a, int n)
{
    const int T = a.d.T;
    if (!a.in.lengths) return T;
    const int l = a.in.lengths[n];
    return l < 0 ? 0 : l < T ? l : T;
}
template <typename T> __device__ __forceinline__ T *step_of(const hts_steps &s, int64_t t, int64_t n) { return (T *)s.p + t * s.st + n * s.sn; }

}  // namespace hts
