// Layer norm of rows and its gradients (see include/hts.h).
//
//   y = (x - mean) r w + b,  r = 1 / sqrt(var + eps);   with h = (x - mean) r, g = dy w:  dx = r (g - mean(g) - h mean(g h)) + add,  dw = sum dy h,  db = sum dy
//
// Bound by bytes: a row is read once, into the registers of a wavefront (up to 1024 entries), of four or of sixteen, its variance is the mean square of what is left
// after the mean is taken off, so that nothing cancels, and it is written once.  (Rows whose squares leave binary32 are read again.)  The backward call keeps nothing of the forward call: the mean and r of a row
// that is in registers cost two reductions and no bytes.
#include "seq.hpp"

namespace hts {
namespace {

struct NormArgs {
    const void *x, *dy, *add;
    void *y, *dx;
    int64_t x_ld, dy_ld, add_ld, y_ld, dx_ld;
    const float *w, *b;
    float *part;              // [workgroups][2 F]: dw, db
    float eps;
    int M, F;
    bool sums;                // dw or db is wanted
};

// What a thread holds of a row: PER times V neighbouring entries, 16 bytes, of which `count` exist.  16-byte accesses at any address: the hardware takes them.  As words, so that a
// load is not waited for where it is taken apart into entries.
template <typename T> struct Piece {
    static constexpr int V = 16 / (int)sizeof(T), IN_WORD = 4 / (int)sizeof(T);
    uint32_t w[4];
    __device__ __forceinline__ void load(const T *p, int count)
    {
        if (count >= V) __builtin_memcpy(w, p, 16);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = 0;
#pragma unroll
                for (int k = 0; k < IN_WORD; ++k) if (i * IN_WORD + k < count) w[i] |= bits_of<T>(to_f32(p[i * IN_WORD + k])) << (16 * k);
            }
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (IN_WORD == 1) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
};
template <typename T> __device__ __forceinline__ void store(T *p, const float (&v)[16 / sizeof(T)], int count)
{
    constexpr int V = 16 / (int)sizeof(T);
    T e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = from_f32<T>(v[i]);
    if (count >= V) __builtin_memcpy(p, e, 16);
    else
#pragma unroll
        for (int i = 0; i < V; ++i) if (i < count) p[i] = e[i];
}
template <int V> __device__ __forceinline__ void load_params(float (&v)[V], const float *p, int count, float none)
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = none;
    } else if (count >= V) __builtin_memcpy(v, p, sizeof v);
    else
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = i < count ? p[i] : 0.0f;
}

// The sums of N values over the ROW threads of a row, by all of them, in the same order.  `turn`: the array that the next sums take, of two (whoever is still reading the other one
// has not passed the barrier of this one).
constexpr int SUMS = 16 * 2;
template <int ROW, int N> __device__ __forceinline__ void row_sums(float (&v)[N], float *shared, int &turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_add(v[i]);
    if constexpr (ROW > 64) {
        constexpr int W = ROW / 64;
        float *to = shared + turn * SUMS;
        turn ^= 1;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) to[wave * N + i] = v[i];
        lds_barrier();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.0f;
#pragma unroll
            for (int k = 0; k < W; ++k) v[i] += to[(wave / W * W + k) * N + i];
        }
    }
}

// ... and the largest of a row's values (0 or more)
template <int ROW> __device__ __forceinline__ float row_most(float v, float *shared, int &turn)
{
    v = most16(v);
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    v = fmaxf(v, __shfl_xor(v, 32, 64));
    if constexpr (ROW > 64) {
        constexpr int W = ROW / 64;
        float *to = shared + turn * SUMS;
        turn ^= 1;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) to[wave] = v;
        lds_barrier();
#pragma unroll
        for (int k = 0; k < W; ++k) v = fmaxf(v, to[wave / W * W + k]);
    }
    return v;
}

// (x 2^by - mean) of a row that is in registers (0 where there is no entry), and the sum of its squares
template <typename T, int ROW, int PER, bool SCALED> __device__ __forceinline__ float deviations(const Piece<T> (&x)[PER], float (&h)[PER][Piece<T>::V], const int by, const int first, const int F, float *shared, int &turn)
{
    constexpr int V = Piece<T>::V;
    float s[1] = {0.0f};
#pragma unroll
    for (int p = 0; p < PER; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            h[p][i] = x[p][i];
            if constexpr (SCALED) h[p][i] = __builtin_ldexpf(h[p][i], by);
            s[0] += h[p][i];
        }
    row_sums<ROW>(s, shared, turn);
    const float mean = s[0] / (float)F;
    s[0] = 0.0f;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int count = F - first - p * ROW * V;
        if (count >= V)
#pragma unroll
            for (int i = 0; i < V; ++i) h[p][i] -= mean;
        else
#pragma unroll
            for (int i = 0; i < V; ++i) h[p][i] = i < count ? h[p][i] - mean : 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) s[0] = __builtin_fmaf(h[p][i], h[p][i], s[0]);
    }
    row_sums<ROW>(s, shared, turn);
    return s[0];
}

// A row whose squares leave binary32, or are so small that they have no digits left (without eps), is worked on again with its largest entry between 1 and 2
__device__ __forceinline__ bool ordinary(float sum, int F, float eps)
{
    const float v = sum / (float)F + eps;
    return v >= 0x1p-100f && v <= 3.402823466e38f;
}
__device__ __forceinline__ float inverse_root(float sum, int F, float eps) { return 1.0f / __builtin_sqrtf(sum / (float)F + eps); }
// h as such deviations, of a row that is read again; what makes them of length one, and the power of two in them.  Rows that are ordinary come out as they were (in a workgroup whose rows meet
// at barriers).
struct Roots { float of_h; int power; };
template <typename T, int ROW, int PER> __device__ __forceinline__ Roots again_scaled(const T *from, const bool there, float (&h)[PER][Piece<T>::V], const bool as_it_is, const int first, const int F, const float eps, float *shared,
                                                                                     int &turn)
{
    Piece<T> x[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int at = first + p * ROW * Piece<T>::V;
        x[p].load(from + at, there ? F - at : 0);
    }
    float most = 0.0f;
#pragma unroll
    for (int p = 0; p < PER; ++p)
#pragma unroll
        for (int i = 0; i < Piece<T>::V; ++i) most = fmaxf(most, __builtin_fabsf(x[p][i]));
    most = fmaxf(row_most<ROW>(most, shared, turn), __builtin_sqrtf(eps));
    const int e = (int)(__float_as_uint(most) >> 23), by = as_it_is || e == 255 ? 0 : 127 - e;         // (the smallest numbers: by 2^127)
    const float r = inverse_root(deviations<T, ROW, PER, true>(x, h, by, first, F, shared, turn), F, __builtin_ldexpf(eps, 2 * by));
    return Roots{r, by};
}

// Rows in turn, by four workgroups a unit: 8192 x 512 in bf16 6.0 to 6.4 us (2.6 to 2.8 TB/s of 16.8 MB; the launch, a row's arrival and two reductions are most of it), 16 rows 2.6.
template <int ROW> constexpr int threads() { return ROW > 256 ? ROW : 256; }
template <typename T, int ROW, int PER> __global__ __launch_bounds__(threads<ROW>()) void norm_kernel(const NormArgs a)
{
    constexpr int V = Piece<T>::V, ROWS = threads<ROW>() / ROW;
    __shared__ float shared[2 * SUMS];
    const int in_row = threadIdx.x % ROW, first = in_row * V;
    const int64_t rows = (int64_t)gridDim.x * ROWS, begin = (int64_t)blockIdx.x * ROWS + threadIdx.x / ROW;
    int turn = 0;
    float w[PER][V], b[PER][V];
    Piece<T> x[PER], next[PER];
    const auto load = [&](Piece<T> (&to)[PER], int64_t row) {
#pragma unroll
        for (int p = 0; p < PER; ++p) to[p].load((const T *)a.x + row * a.x_ld + first + p * ROW * V, a.F - first - p * ROW * V);
    };
    if (begin < a.M) load(x, begin);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int at = first + p * ROW * V;
        load_params<V>(w[p], a.w ? a.w + at : nullptr, a.F - at, 1.0f);
        load_params<V>(b[p], a.b ? a.b + at : nullptr, a.F - at, 0.0f);
    }
    for (int64_t row = begin; row < a.M; row += rows) {
        if (row + rows < a.M) load(next, row + rows);          // on its way while this one is worked on
        float h[PER][V];
        const float sum = deviations<T, ROW, PER, false>(x, h, 0, first, a.F, shared, turn);
        float r = inverse_root(sum, a.F, a.eps);
        if (!ordinary(sum, a.F, a.eps)) r = again_scaled<T, ROW, PER>((const T *)a.x + row * a.x_ld, true, h, false, first, a.F, a.eps, shared, turn).of_h;      // (a workgroup's threads have one row here, or no barriers)
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = __builtin_fmaf(h[p][i] * r, w[p][i], b[p][i]);
            store((T *)a.y + row * a.y_ld + first + p * ROW * V, y, a.F - first - p * ROW * V);
            x[p] = next[p];
        }
    }
}

// Registers hold the sums of dw and db of all rows that a thread sees, and rows come while others are worked on: 8192 x 2048 in bf16 with a residual's gradient, 134 MB, 36.2 us
// (3.7 TB/s: wavefronts wait for 56% of their cycles, for rows and at the three reductions of each, and the vector units work for 18 us), 1021 x 777 in binary32 6.8 (128 workgroups of eight rows on 256
// units), and 3 to 5 for the workgroups' sums (the call 39 us).
// Rows that a workgroup works on at a time: eight of a wavefront each, two of four, one of sixteen; and all of its threads go round together
template <int ROW> constexpr int back_threads() { return ROW > 256 ? ROW : 512; }

// workgroups of a backward call, whose sums are added up afterwards, at the most: two a unit, one of sixteen wavefronts
template <int ROW> constexpr int back_most() { return ROW > 256 ? 256 : 512; }

template <typename T, int ROW, int PER> __global__ __launch_bounds__(back_threads<ROW>()) void norm_backward_kernel(const NormArgs a)
{
    constexpr int V = Piece<T>::V, ROWS = back_threads<ROW>() / ROW, COLS = ROW * PER * V;
    // Rows that are to be worked on again, a bit for each of the workgroup's: after the others, so that the loop has nothing of it
    constexpr int MOST_ROWS = (1 << 24) / back_most<ROW>();
    __shared__ uint32_t seldom[MOST_ROWS / 32], some;
    __shared__ float shared[(ROWS > 1 ? ROWS * COLS : 0) + 2 * SUMS];
    float *sums = shared + (ROWS > 1 ? ROWS * COLS : 0);
    constexpr bool AHEAD = ROW <= 256;           // the next row's entries are requested before this one's are worked on (sixteen wavefronts have no registers for them)
    const int in_row = threadIdx.x % ROW, first = in_row * V, mine = threadIdx.x / ROW;
    const int64_t rows = (int64_t)gridDim.x * ROWS;
    int turn = 0;
    float w[PER][V], dw[PER][V], db[PER][V];
    Piece<T> x[PER], dy[PER], add[PER], next_x[PER] = {}, next_dy[PER] = {}, next_add[PER] = {};
    const auto load = [&](Piece<T> (&to)[PER], const void *from, int64_t ld, int64_t row) {
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int at = first + p * ROW * V;
            to[p].load((const T *)from + row * ld + at, row < a.M ? a.F - at : 0);
        }
    };
    const bool adds = a.dx && a.add;
    const auto along_row = [&](float (&h)[PER][V], const Piece<T> (&dy)[PER], float (&s)[2], float own, bool take) {
#pragma unroll
        for (int p = 0; p < PER; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = dy[p][i], g = d * w[p][i];
                h[p][i] *= own;
                if (take) {
                    dw[p][i] = __builtin_fmaf(d, h[p][i], dw[p][i]);          // (of rows behind the last one: zeros)
                    db[p][i] += d;
                }
                s[0] += g;
                s[1] = __builtin_fmaf(g, h[p][i], s[1]);
            }
    };
    const auto give = [&](const float (&h)[PER][V], const Piece<T> (&dy)[PER], const Piece<T> (&add)[PER], const float (&s)[2], float r, auto finish, int64_t to) {
        const float mean = s[0] / (float)a.F, along = s[1] / (float)a.F;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                o[i] = finish(r * __builtin_fmaf(-h[p][i], along, dy[p][i] * w[p][i] - mean));
                if (a.add) o[i] += add[p][i];
            }
            store((T *)a.dx + to * a.dx_ld + first + p * ROW * V, o, a.F - first - p * ROW * V);
        }
    };
    for (int i = threadIdx.x; i < MOST_ROWS / 32 && i * 32ll * gridDim.x < a.M; i += back_threads<ROW>()) seldom[i] = 0;
    if (threadIdx.x == 0) some = 0;
    __syncthreads();
    int64_t row = (int64_t)blockIdx.x * ROWS;
    int at_row = mine;                                       // of the workgroup's
    load(x, a.x, a.x_ld, row + mine);
    load(dy, a.dy, a.dy_ld, row + mine);
    if (adds) load(add, a.add, a.add_ld, row + mine);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int at = first + p * ROW * V;
        load_params<V>(w[p], a.w ? a.w + at : nullptr, a.F - at, 1.0f);
#pragma unroll
        for (int i = 0; i < V; ++i) dw[p][i] = db[p][i] = 0.0f;
    }
    for (; row < a.M; row += rows, at_row += ROWS) {
        const int64_t to = row + mine;
        if (AHEAD && row + rows < a.M) {
            load(next_x, a.x, a.x_ld, to + rows);
            load(next_dy, a.dy, a.dy_ld, to + rows);
            if (adds) load(next_add, a.add, a.add_ld, to + rows);
        }
        float h[PER][V];
        const float sum = deviations<T, ROW, PER, false>(x, h, 0, first, a.F, sums, turn);
        float r = inverse_root(sum, a.F, a.eps);
        const bool rare = to < a.M && !ordinary(sum, a.F, a.eps);          // (of rows behind the last one r is that of zeros, which eps = 0 makes infinite)
        float s[2] = {0.0f, 0.0f};
        if (rare) {
            if (in_row == 0) { atomicOr(&seldom[at_row >> 5], 1u << (at_row & 31)); some = 1; }
        } else along_row(h, dy, s, to < a.M ? r : 0.0f, true);
        if (a.dx) {
            row_sums<ROW>(s, sums, turn);
            if (to < a.M && !rare) give(h, dy, add, s, r, [](float x) { return x; }, to);
        }
#pragma unroll
        for (int p = 0; p < PER; ++p) { x[p] = next_x[p]; dy[p] = next_dy[p]; add[p] = next_add[p]; }
        if (!AHEAD && row + rows < a.M) {
            load(x, a.x, a.x_ld, to + rows);
            load(dy, a.dy, a.dy_ld, to + rows);
            if (adds) load(add, a.add, a.add_ld, to + rows);
        }
    }
    __syncthreads();
    if (some)
        for (row = (int64_t)blockIdx.x * ROWS, at_row = 0; row < a.M; row += rows, at_row += ROWS) {
            const uint32_t which = seldom[at_row >> 5] >> (at_row & 31) & ((1u << ROWS) - 1);
            if (!which) continue;
            const bool rare = which >> mine & 1;             // (the others' threads meet these at barriers)
            const int64_t to = row + mine;
            load(dy, a.dy, a.dy_ld, to);
            if (adds) load(add, a.add, a.add_ld, to);
            float h[PER][V], s[2] = {0.0f, 0.0f};
            const Roots roots = again_scaled<T, ROW, PER>((const T *)a.x + to * a.x_ld, to < a.M, h, !rare, first, a.F, a.eps, sums, turn);
            along_row(h, dy, s, roots.of_h, rare);
            if (!a.dx) continue;
            row_sums<ROW>(s, sums, turn);
            if (rare) give(h, dy, add, s, roots.of_h, [&](float x) { return __builtin_ldexpf(x, roots.power); }, to);
        }
    if (!a.sums) return;
    // a workgroup's sums: its rows in order
    float *part = a.part + (int64_t)blockIdx.x * 2 * a.F;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (ROWS > 1) {
            __syncthreads();
#pragma unroll
            for (int p = 0; p < PER; ++p)
#pragma unroll
                for (int i = 0; i < V; ++i) shared[mine * COLS + first + p * ROW * V + i] = which ? db[p][i] : dw[p][i];
            __syncthreads();
            for (int c = threadIdx.x; c < a.F; c += back_threads<ROW>()) {
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < ROWS; ++k) s += shared[k * COLS + c];
                part[which * a.F + c] = s;
            }
        } else {
#pragma unroll
            for (int p = 0; p < PER; ++p)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = first + p * ROW * V + i;
                    if (c < a.F) part[which * a.F + c] = which ? db[p][i] : dw[p][i];
                }
        }
    }
}

// Threads of a row, and entries that each holds: 8 or 16 of a wavefront's, of four or of sixteen wavefronts'.  (32 of a wavefront's left one or two of them to a SIMD: gradients of
// 8192 x 2048 in bf16, operands partly in the cache, 38 us, with four wavefronts a row 30.)
template <int V, typename F> hipError_t by_width(int width, F f)
{
    const auto with = [&](auto row, auto entries) { return f(std::integral_constant<int, decltype(row)::value>{}, std::integral_constant<int, decltype(entries)::value / V>{}); };
    typedef std::integral_constant<int, 64> wave;
    typedef std::integral_constant<int, 256> four;
    typedef std::integral_constant<int, 1024> sixteen;
    const std::integral_constant<int, 8> eight;
    const std::integral_constant<int, 16> more;
    if (width <= 512) return with(wave{}, eight);
    if (width <= 1024) return with(wave{}, more);
    if (width <= 2048) return with(four{}, eight);
    if (width <= 4096) return with(four{}, more);
    if (width <= 8192) return with(sixteen{}, eight);
    return with(sixteen{}, more);
}

int back_parts(int64_t M, int64_t F)
{
    const int64_t rows = F <= 1024 ? 8 : F <= 4096 ? 2 : 1, most = F <= 4096 ? back_most<64>() : back_most<1024>(), groups = ceil_div(M, rows);
    return (int)(groups < most ? groups : most);
}

template <typename T> hipError_t norm(hts_seq_ctx &c, const NormArgs &a)
{
    return by_width<Piece<T>::V>(a.F, [&](auto row, auto per) {
        constexpr int ROW = decltype(row)::value, PER = decltype(per)::value, ROWS = threads<ROW>() / ROW;
        const int64_t groups = ceil_div(a.M, ROWS), most = (int64_t)c.cus * (ROW > 256 ? 2 : 4);
        hipLaunchKernelGGL((norm_kernel<T, ROW, PER>), dim3((uint32_t)(groups < most ? groups : most)), dim3(threads<ROW>()), 0, c.stream, a);
        return hipGetLastError();
    });
}
template <typename T> hipError_t norm_backward(hts_seq_ctx &c, const NormArgs &a, float *dw, float *db)
{
    const int parts = back_parts(a.M, a.F);
    const hipError_t e = by_width<Piece<T>::V>(a.F, [&](auto row, auto per) {
        constexpr int ROW = decltype(row)::value, PER = decltype(per)::value;
        hipLaunchKernelGGL((norm_backward_kernel<T, ROW, PER>), dim3((uint32_t)parts), dim3(back_threads<ROW>()), 0, c.stream, a);
        return hipGetLastError();
    });
    if (e != hipSuccess || !a.sums) return e;
    return launch_sum_partials(c, a.part, parts, 2 * (int64_t)a.F, SumTarget{dw, a.F}, SumTarget{db, a.F}, SumTarget{nullptr, 0});
}
}  // namespace

int64_t norm_workspace(int64_t M, int64_t F) { return 8 * back_parts(M, F) * F; }

hipError_t launch_norm(hts_seq_ctx &c, int precision, const NormOp &op)
{
    NormArgs a = {};
    a.x = op.x.p; a.x_ld = op.x.ld; a.y = op.y.p; a.y_ld = op.y.ld; a.w = op.w; a.b = op.b; a.eps = op.eps; a.M = op.M; a.F = op.F;
    return precision == HTS_PRECISION_BF16 ? norm<bf16_t>(c, a) : norm<float>(c, a);
}
hipError_t launch_norm_backward(hts_seq_ctx &c, int precision, const NormOp &op)
{
    NormArgs a = {};
    a.x = op.x.p; a.x_ld = op.x.ld; a.dy = op.dy.p; a.dy_ld = op.dy.ld; a.add = op.add.p; a.add_ld = op.add.ld; a.dx = op.dx.p; a.dx_ld = op.dx.ld;
    a.w = op.w; a.eps = op.eps; a.M = op.M; a.F = op.F; a.sums = op.dw || op.db; a.part = (float *)c.ws;
    return precision == HTS_PRECISION_BF16 ? norm_backward<bf16_t>(c, a, op.dw, op.db) : norm_backward<float>(c, a, op.dw, op.db);
}

}  // namespace hts
