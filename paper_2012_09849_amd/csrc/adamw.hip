// AdamW over many tensors at once (see include/hts.h).
//
//   g <- g min(1, c / (|g| + 1e-6));  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2;  p <- p (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by bytes: every entry's numbers are read once and written once, by one launch for all tensors (and one before it for the norm, where it is asked for).
// 41 M entries with states in 8 bits: a call among others 196 us, under a trace 31 for the norm (82 MB; its wavefronts wait for 80% of their cycles) and 175 to 191 for the update, which untraced
// leaves about 165 for 653 MB (4.0 TB/s): issue of vector instructions, 99 million of a wavefront's, 161 us at 2.4 GHz, those of the random bits and the rounding first of all; 1.7 M in 32 bits, which stay in the cache between updates, 4.2 and 11.7; 49 thousand 2.7 and 4.9.
//
// A workgroup takes 2048 entries of one tensor, which a table of the plan names; a wavefront 256 of them at a time, 4 neighbours a lane.  Without contraction of
// products and sums (a build flag of this file) the arithmetic is that of its terms one by one, so states in 8 bits have the same bits wherever these rules are followed.
#include <algorithm>
#include <cmath>
#include <new>

#include "gemm.hpp"
#include "internal.hpp"

struct hts_adamw {
    hipStream_t stream;
    char *device;             // one allocation: the norm's partial sums, the tensors, the pieces
    int32_t count;            // tensors
    int64_t pieces;           // workgroups
};

namespace hts {
namespace {

constexpr int PIECE = 2048, GROUP = 256, NORM_GROUPS = 1024;       // entries of a workgroup; that share a scale; partial sums of the norm

struct Tensor {
    float *p;
    const void *g;
    void *m, *v;
    float *m_scale, *v_scale;
    bf16_t *copy;
    int64_t n;
    float decay, lr_scale;
    int32_t half_grads, eight;
};
struct Piece { int32_t tensor, part; };

struct StepArgs {
    const Tensor *tensors;
    const Piece *pieces;
    double *norm;
    float *grad_norm;
    int64_t count;
    uint64_t seed, step;
    float b1, b2, rest1, rest2, lr, correct1, root, eps, clip;
    bool normed;
};

template <int N> __device__ __forceinline__ void take(float (&x)[N], const float *p, int count)
{
    if (count >= N) __builtin_memcpy(x, p, sizeof x);
    else
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = i < count ? p[i] : 0.0f;
}
__device__ __forceinline__ void take_grads(float (&x)[4], const Tensor &t, int64_t at, int count)
{
    if (!t.half_grads) return take(x, (const float *)t.g + at, count);
    const bf16_t *p = (const bf16_t *)t.g + at;
    bf16_t h[4];
    if (count >= 4) __builtin_memcpy(h, p, sizeof h);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = i < count ? p[i] : (bf16_t)0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)h[i];
}

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
}
// the sum of a workgroup's values by every thread, wavefront by wavefront
template <int THREADS> __device__ __forceinline__ double group_sum(double x, double *shared)
{
    x = wave_sum(x);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) s += shared[w];
    return s;
}

// Sums of squares, in 64 bits: the factor on the gradients is then the same however the sum is formed.  A workgroup takes two pieces at a time, 8 neighbours a thread of each
__global__ __launch_bounds__(256) void norm_kernel(const StepArgs a)
{
    __shared__ double shared[4];
    double s = 0.0;
    for (int64_t i = blockIdx.x; i < a.count; i += 2 * NORM_GROUPS) {
        float g[2][2][4] = {};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (i + k * NORM_GROUPS >= a.count) continue;
            const Piece piece = a.pieces[i + k * NORM_GROUPS];
            const Tensor t = a.tensors[piece.tensor];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int64_t at = (int64_t)piece.part * PIECE + 8 * (int)threadIdx.x + 4 * e, left = t.n - at;
                take_grads(g[k][e], t, at, left > 4 ? 4 : left > 0 ? (int)left : 0);
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += (double)g[k][e >> 2][e & 3] * (double)g[k][e >> 2][e & 3];
    }
    s = group_sum<256>(s, shared);
    if (threadIdx.x == 0) a.norm[blockIdx.x] = s;
}

// Philox4x32-10 (Salmon et al., SC'11)
__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        // (both halves of a product by one instruction)
        const uint64_t p0 = (uint64_t)0xD2511F53u * c[0], p1 = (uint64_t)0xCD9E8D57u * c[2];
        c[0] = (uint32_t)(p1 >> 32) ^ c[1] ^ k0; c[1] = (uint32_t)p1; c[2] = (uint32_t)(p0 >> 32) ^ c[3] ^ k1; c[3] = (uint32_t)p0;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
}
__device__ __forceinline__ int exponent(float x) { return (int)(__float_as_uint(x) >> 23 & 255) - 127; }
__device__ __forceinline__ float power_of_2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int o = 32; o >= 16; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
    // over 16 neighbouring lanes: pairs, fours, eights (mirrored), sixteen
#define MOVED(control) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), control, 0xf, 0xf, true)))
    MOVED(0xB1); MOVED(0x4E); MOVED(0x141); MOVED(0x140);
#undef MOVED
    return x;
}
__device__ __forceinline__ float size_of_finite(float x)
{
    const float s = __builtin_fabsf(x);
    return s <= 3.402823466e38f ? s : 0.0f;
}
// e4m3 of x / scale, below 256: the digits after the third are dropped after a random part of the last one is added.  POSITIVE: what is above zero stays above.
template <bool POSITIVE> __device__ __forceinline__ uint32_t held(float x, float by, uint32_t part)
{
    const float y = x * by, s = __builtin_fabsf(y);
    // from 2^-6 on the exponent's digits go on above the number's: the random part is added to the 20 that are dropped, and a carry is the next power of two
    const int normal = (int)((__float_as_uint(s) + (part << 4)) >> 20) - (120 << 3);
    const int small = (int)__builtin_floorf(s * 512.0f + (float)part * (1.0f / 65536.0f));
    int code = s >= 0.015625f ? normal : small;
    if (POSITIVE && code == 0 && s > 0.0f) code = 1;
    if (!(__builtin_fabsf(x) <= 3.402823466e38f)) return 0x7f;       // NaN
    return (uint32_t)code | (y < 0.0f ? 0x80u : 0u);
}
__device__ __forceinline__ void given(float (&x)[4], const uint8_t *p, int count, float scale)
{
    uint32_t w = 0;
    if (count >= 4) __builtin_memcpy(&w, p, 4);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) if (i < count) w |= (uint32_t)p[i] << (8 * i);
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0) * scale; x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * scale;
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * scale; x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * scale;
}
template <typename P> __device__ __forceinline__ void put(P *to, const P (&x)[4], int count)
{
    if (count >= 4) __builtin_memcpy(to, x, sizeof x);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) if (i < count) to[i] = x[i];
}

__global__ __launch_bounds__(256) void step_kernel(const StepArgs a)
{
    constexpr int TIMES = PIECE / 1024;
    __shared__ double shared[4];
    const Piece piece = a.pieces[blockIdx.x];
    const Tensor t = a.tensors[piece.tensor];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)piece.part * PIECE + wave * GROUP + 4 * lane;
    float p[TIMES][4], g[TIMES][4], m[TIMES][4], v[TIMES][4];
    int count[TIMES];
#pragma unroll
    for (int k = 0; k < TIMES; ++k) {
        const int64_t at = first + 1024 * k, left = t.n - at;
        count[k] = left > 4 ? 4 : left > 0 ? (int)left : 0;
        take(p[k], t.p + at, count[k]);
        take_grads(g[k], t, at, count[k]);
        if (t.eight) {
            const bool any = first + 1024 * k - 4 * lane < t.n;
            given(m[k], (const uint8_t *)t.m + at, count[k], any ? t.m_scale[at / GROUP] : 0.0f);
            given(v[k], (const uint8_t *)t.v + at, count[k], any ? t.v_scale[at / GROUP] : 0.0f);
        } else {
            take(m[k], (const float *)t.m + at, count[k]);
            take(v[k], (const float *)t.v + at, count[k]);
        }
    }
    float by = 1.0f;
    if (a.normed) {
        double part = 0.0;
#pragma unroll
        for (int k = 0; k < NORM_GROUPS / 256; ++k) part += a.norm[256 * k + threadIdx.x];
        const float norm = (float)__builtin_sqrt(group_sum<256>(part, shared));
        if (a.clip > 0.0f) {
            by = a.clip / (norm + 1e-6f);
            by = by >= 1.0f ? 1.0f : by;            // (NaN stays)
        }
        if (a.grad_norm && blockIdx.x == 0 && threadIdx.x == 0) *a.grad_norm = norm;
    }
    const float lr = a.lr * t.lr_scale, size = a.correct1 * t.lr_scale, keep = 1.0f - lr * t.decay;
#pragma unroll
    for (int k = 0; k < TIMES; ++k) {
        const int64_t at = first + 1024 * k;
        float r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = g[k][i] * by;
            if (t.eight) v[k][i] *= v[k][i];
            m[k][i] = m[k][i] * a.b1 + x * a.rest1;
            v[k][i] = v[k][i] * a.b2 + x * a.rest2 * x;
            r[i] = __builtin_sqrtf(v[k][i]);
            p[k][i] = p[k][i] * keep - size * (m[k][i] / (r[i] * a.root + a.eps));
        }
        put(t.p + at, p[k], count[k]);
        if (t.copy) {
            const bf16_t h[4] = {(bf16_t)p[k][0], (bf16_t)p[k][1], (bf16_t)p[k][2], (bf16_t)p[k][3]};
            put(t.copy + at, h, count[k]);
        }
        if (!t.eight) {
            put((float *)t.m + at, m[k], count[k]);
            put((float *)t.v + at, v[k], count[k]);
            continue;
        }
        float most_m = 0.0f, most_r = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count[k]) { most_m = fmaxf(most_m, size_of_finite(m[k][i])); most_r = fmaxf(most_r, size_of_finite(r[i])); }
        int em = exponent(wave_max(most_m)) - 7, er = exponent(wave_max(most_r)) - 7;
        if (em < -126) em = -126;
        if (er < -126) er = -126;
        uint32_t w[4] = {(uint32_t)(at >> 2), (uint32_t)piece.tensor, (uint32_t)a.step, (uint32_t)(a.step >> 32)};
        philox(w, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
        uint8_t hm[4], hr[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            hm[i] = (uint8_t)held<false>(m[k][i], power_of_2(-em), w[i] & 0xffffu);
            hr[i] = (uint8_t)held<true>(r[i], power_of_2(-er), w[i] >> 16);
        }
        put((uint8_t *)t.m + at, hm, count[k]);
        put((uint8_t *)t.v + at, hr, count[k]);
        if (lane == 0 && count[k] > 0) { t.m_scale[at / GROUP] = power_of_2(em); t.v_scale[at / GROUP] = power_of_2(er); }
    }
}

struct Stretch { uint64_t from, to; bool written; };
}  // namespace
}  // namespace hts

using namespace hts;

#define HIP_TRY(x) do { const hipError_t e_ = (x); if (e_ != hipSuccess) { note_hip_error(e_); return HTS_EHIP; } } while (0)

static bool off(const void *p, int size) { return (uintptr_t)p % size != 0; }

// Checks a plan's tensors, and that no two arrays of which one is written share memory.
static int32_t check_tensors(const hts_adamw_tensor *tensors, int32_t count, int64_t *pieces)
{
    if (!tensors || count <= 0) return HTS_EINVAL;
    if (count > (1 << 20)) return HTS_ESHAPE;
    *pieces = 0;
    for (int32_t i = 0; i < count; ++i) {
        const hts_adamw_tensor &t = tensors[i];
        if (!t.p || !t.g || !t.m || !t.v || t.n <= 0 || (t.bits != 8 && t.bits != 32)) return HTS_EINVAL;
        if (t.grad_precision != HTS_PRECISION_FP32 && t.grad_precision != HTS_PRECISION_BF16) return HTS_ESHAPE;
        if (off(t.p, 4) || off(t.g, t.grad_precision == HTS_PRECISION_BF16 ? 2 : 4) || off(t.copy, 2)) return HTS_EINVAL;
        if (t.bits == 8 ? !t.m_scale || !t.v_scale || off(t.m_scale, 4) || off(t.v_scale, 4) : off(t.m, 4) || off(t.v, 4)) return HTS_EINVAL;
        if (!(t.weight_decay >= 0.0f && t.weight_decay <= 3.4e38f) || !(t.lr_scale >= 0.0f && t.lr_scale <= 3.4e38f)) return HTS_EINVAL;
        if (t.n > (1ll << 34)) return HTS_ESHAPE;
        *pieces += (t.n + PIECE - 1) / PIECE;
    }
    if (*pieces > (1 << 24) - 1) return HTS_ESHAPE;              // (2^32 threads are a grid's most)
    Stretch *all = new (std::nothrow) Stretch[7 * (int64_t)count];
    if (!all) return HTS_ENOMEM;
    int64_t n = 0;
    const auto add = [&](const void *p, int64_t bytes, bool written) { if (p) all[n++] = Stretch{(uint64_t)(uintptr_t)p, (uint64_t)(uintptr_t)p + (uint64_t)bytes, written}; };
    for (int32_t i = 0; i < count; ++i) {
        const hts_adamw_tensor &t = tensors[i];
        const int64_t scales = 4 * ((t.n + GROUP - 1) / GROUP);
        add(t.p, 4 * t.n, true); add(t.g, (t.grad_precision == HTS_PRECISION_BF16 ? 2 : 4) * t.n, false); add(t.copy, 2 * t.n, true);
        add(t.m, t.bits / 8 * t.n, true); add(t.v, t.bits / 8 * t.n, true);
        if (t.bits == 8) { add(t.m_scale, scales, true); add(t.v_scale, scales, true); }
    }
    std::sort(all, all + n, [](const Stretch &x, const Stretch &y) { return x.from < y.from; });
    uint64_t end = 0, written_end = 0;
    bool apart = true;
    for (int64_t i = 0; i < n; ++i) {
        if (all[i].from < (all[i].written ? end : written_end)) apart = false;
        end = std::max(end, all[i].to);
        if (all[i].written) written_end = std::max(written_end, all[i].to);
    }
    delete[] all;
    return apart ? HTS_OK : HTS_EINVAL;
}

static int64_t tensors_bytes(int32_t count) { return (int64_t)sizeof(Tensor) * count; }

extern "C" int32_t hts_adamw_create(const hts_adamw_tensor *tensors, int32_t count, void *hip_stream, hts_adamw **out)
{
    if (!out) return HTS_EINVAL;
    int64_t pieces = 0;
    const int32_t rc = check_tensors(tensors, count, &pieces);
    if (rc != HTS_OK) return rc;
    const int64_t bytes = 8 * NORM_GROUPS + tensors_bytes(count) + (int64_t)sizeof(Piece) * pieces;
    char *host = new (std::nothrow) char[bytes];
    hts_adamw *o = new (std::nothrow) hts_adamw();
    if (!host || !o) { delete[] host; delete o; return HTS_ENOMEM; }
    std::fill(host, host + 8 * NORM_GROUPS, 0);
    Tensor *ts = (Tensor *)(host + 8 * NORM_GROUPS);
    Piece *ps = (Piece *)(host + 8 * NORM_GROUPS + tensors_bytes(count));
    int64_t k = 0;
    for (int32_t i = 0; i < count; ++i) {
        const hts_adamw_tensor &t = tensors[i];
        ts[i] = Tensor{t.p, t.g, t.m, t.v, t.m_scale, t.v_scale, (bf16_t *)t.copy, t.n, t.weight_decay, t.lr_scale, t.grad_precision == HTS_PRECISION_BF16, t.bits == 8};
        for (int64_t part = 0; part * PIECE < t.n; ++part) ps[k++] = Piece{i, (int32_t)part};
    }
    o->stream = (hipStream_t)hip_stream; o->count = count; o->pieces = pieces; o->device = nullptr;
    hipError_t e = hipMalloc((void **)&o->device, (size_t)bytes);
    const bool memory = e != hipSuccess;
    if (!memory) e = hipMemcpy(o->device, host, (size_t)bytes, hipMemcpyHostToDevice);
    delete[] host;
    if (e != hipSuccess) {
        if (!memory) (void)hipFree(o->device);
        delete o;
        note_hip_error(e);
        return memory ? HTS_ENOMEM : HTS_EHIP;
    }
    *out = o;
    return HTS_OK;
}

extern "C" int32_t hts_adamw_destroy(hts_adamw *opt)
{
    if (!opt) return HTS_EINVAL;
    const hipError_t e = hipFree(opt->device);
    delete opt;
    HIP_TRY(e);
    return HTS_OK;
}

extern "C" int32_t hts_adamw_step(hts_adamw *opt, const hts_adamw_hparams *hp, int64_t *step, float *grad_norm_or_null)
{
    if (!opt || !hp || !step || *step < 0 || *step >= (1ll << 62) || off(grad_norm_or_null, 4)) return HTS_EINVAL;
    const auto share = [](float x) { return x >= 0.0f && x < 1.0f; };
    if (!share(hp->beta1) || !share(hp->beta2) || !(hp->lr >= 0.0f && hp->lr <= 3.4e38f) || !(hp->eps >= 0.0f && hp->eps <= 3.4e38f) || !(hp->max_grad_norm <= 3.4e38f)) return HTS_EINVAL;
    const int64_t t = *step + 1;
    StepArgs a = {};
    a.norm = (double *)opt->device;
    a.tensors = (const Tensor *)(opt->device + 8 * NORM_GROUPS);
    a.pieces = (const Piece *)(opt->device + 8 * NORM_GROUPS + tensors_bytes(opt->count));
    a.count = opt->pieces; a.grad_norm = grad_norm_or_null;
    a.seed = hp->seed; a.step = (uint64_t)t;
    a.b1 = hp->beta1; a.b2 = hp->beta2; a.rest1 = (float)(1.0 - (double)hp->beta1); a.rest2 = (float)(1.0 - (double)hp->beta2);
    a.lr = hp->lr;
    a.correct1 = (float)((double)hp->lr / (1.0 - std::pow((double)hp->beta1, (double)t)));
    a.root = (float)(1.0 / std::sqrt(1.0 - std::pow((double)hp->beta2, (double)t)));
    a.eps = hp->eps; a.clip = hp->max_grad_norm;
    a.normed = hp->max_grad_norm > 0.0f || grad_norm_or_null;
    if (a.normed) {
        hipLaunchKernelGGL(norm_kernel, dim3(NORM_GROUPS), dim3(256), 0, opt->stream, a);
        HIP_TRY(hipGetLastError());
    }
    hipLaunchKernelGGL(step_kernel, dim3((uint32_t)opt->pieces), dim3(256), 0, opt->stream, a);
    HIP_TRY(hipGetLastError());
    *step = t;
    return HTS_OK;
}
