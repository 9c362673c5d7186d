// Matrix products of the sequence memory: y = act(x W^T + b) + r and its gradients (see include/hts.h), on tiles of 32x32 matrix instructions.
//
// All three products are C[i][j] = sum_k A(i,k) B(j,k) with a kernel for each layout of the operands: along k in memory (x and W of the forward
// product, dz of dx) or across (W of dx, both operands of dw).  An operand tile is copied to LDS as it lies in memory, 16 bytes at a time; one along k
// is read by rows, one across by the transposing LDS read in bfloat16 (four neighbouring k of a column a lane) and word by word in binary32.
//   bfloat16: v_mfma_f32_32x32x16_bf16, k-tiles of 64;  binary32: v_mfma_f32_32x32x2_f32, k-tiles of 32.
// The operands go to the instruction in exchanged order, so a lane holds a row of C and four neighbouring columns of it.
#include "seq.hpp"

namespace hts {
namespace {

struct Product {
    const void *a, *b, *a_low;     // a_low: the same operand's low part; the reduction goes over it, with the same b, after a
    int64_t lda, ldb;
    int M, N, K;                   // C is M x N, reduction over K
    int klen;                      // reduction of a slice (of both parts of A together), whole k-tiles
    int act;
    const float *bias;
    const void *res;
    void *y, *pre;
    int64_t ldr, ldy, ldp;
    float *part;                   // slices > 1: [slice][M][N]
};

template <typename T> struct Kind { static constexpr int V = 16 / sizeof(T), BK = 128 / sizeof(T); };       // entries of 16 bytes, k-tile

// where the 16 bytes with number s (along the row) of row r of an operand tile are, for operands along k: rows of 128 bytes, the slots exchanged so
// that the rows of an operand read fall into different banks
__device__ __forceinline__ int along_at(int r, int s) { return r * 128 + 16 * (s ^ ((r >> 1) & 7)); }
// ... and for operands across: rows are k, B the tile's width.  bfloat16: 32-byte pieces exchanged by k, so that the four rows of a transposing read
// fall into different banks; binary32: halves of 128 bytes by k's bit 2, which the two halves of a wavefront differ in
template <typename T, int B> __device__ __forceinline__ int across_at(int k, int s)
{
    if constexpr (sizeof(T) == 2) {
        const int f = B >= 128 ? ((k & 3) << 1 | (k >> 2 & 1)) : (k >> 1 & 1) << 1;
        return k * (B * 2) + ((s ^ f << 1) << 4);
    } else return k * (B * 4) + ((s ^ (k >> 2 & 1) << 3) << 4);
}

struct Piece { uint32_t w[4]; };
template <typename T> __device__ __forceinline__ Piece load_piece(const T *p, int64_t count)
{
    constexpr int V = Kind<T>::V;
    Piece r = {{0, 0, 0, 0}};
    if (count >= V) __builtin_memcpy(&r, p, 16);
    else if (count > 0) {
        T e[V];
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = i < count ? p[i] : from_f32<T>(0.0f);
        __builtin_memcpy(&r, e, 16);
    }
    return r;
}

// One operand's tile: B entries of C's edge from `first`, k-tile at k0
template <typename T, bool ACROSS, int B, int THREADS> struct Staged {
    static constexpr int V = Kind<T>::V, BK = Kind<T>::BK, PIECES = B * BK / V / THREADS, SLOTS = ACROSS ? B / V : BK / V;
    static_assert(PIECES * THREADS * V == B * BK, "tile");
    Piece v[PIECES];
    __device__ __forceinline__ void load(const T *p, int64_t ld, int first, int edge, int k0, int K, int tid)
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int r = (i * THREADS + tid) / SLOTS, s = (i * THREADS + tid) % SLOTS;
            const int row = (ACROSS ? k0 : first) + r, rows = ACROSS ? K : edge, col = (ACROSS ? first : k0) + s * V, cols = ACROSS ? edge : K;
            v[i] = load_piece(p + row * ld + col, row < rows ? cols - col : 0);
        }
    }
    __device__ __forceinline__ void put(char *lds, int tid) const
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int r = (i * THREADS + tid) / SLOTS, s = (i * THREADS + tid) % SLOTS;
            *reinterpret_cast<Piece *>(lds + (ACROSS ? across_at<T, B>(r, s) : along_at(r, s))) = v[i];
        }
    }
};

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 *lds_quad;

// operands of a k-tile's kk-th part (16 k in bfloat16, 8 in binary32) for 32 entries from `at`
template <typename T, bool ACROSS, int B> __device__ __forceinline__ Vec<T, Kind<T>::V> operand(const char *lds, int at, int kk, int lane)
{
    if constexpr (!ACROSS) return *reinterpret_cast<const Vec<T, Kind<T>::V> *>(lds + along_at(at + (lane & 31), 2 * kk + (lane >> 5)));
    else if constexpr (sizeof(T) == 2) {
        const int k = kk * 16 + (lane >> 5) * 8 + (lane >> 2 & 3), col = at + (lane & 16) + (lane & 3) * 4;
        const char *q0 = lds + across_at<T, B>(k, col >> 3) + (col & 7) * 2, *q1 = lds + across_at<T, B>(k + 4, col >> 3) + (col & 7) * 2;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad)(uintptr_t)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)q0);
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad)(uintptr_t)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)q1);
        const short both[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        Vec<T, 8> r;
        __builtin_memcpy(&r, both, 16);
        return r;
    } else {
        Vec<T, 4> r;
        const int col = at + (lane & 31);
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = *reinterpret_cast<const float *>(lds + across_at<T, B>(kk * 8 + (lane >> 5) * 4 + i, col >> 2) + (col & 3) * 4);
        return r;
    }
}
template <typename T> __device__ __forceinline__ f32x16 multiply(const Vec<T, Kind<T>::V> &a, const Vec<T, Kind<T>::V> &b, f32x16 c)
{
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, c, 0, 0, 0);
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(b[i], a[i], c, 0, 0, 0);
        return c;
    }
}

// C's entry (m, n), v = sum
template <typename T, typename OUT> __device__ __forceinline__ void finish(const Product &p, int64_t m, int64_t n, float v)
{
    if (p.bias) v += p.bias[n];
    if (p.pre) ((T *)p.pre)[m * p.ldp + n] = from_f32<T>(v);
    v = act_of(p.act, v);
    if (p.res) v += to_f32(((const T *)p.res)[m * p.ldr + n]);
    ((OUT *)p.y)[m * p.ldy + n] = from_f32<OUT>(v);
}

template <typename T, typename OUT, bool AX, bool BX, int BM, int BN>
__global__ __launch_bounds__(256) void product_kernel(const Product p, const int tiles_n)
{
    constexpr int THREADS = 256, BK = Kind<T>::BK, TM = BM / 64, TN = BN / 64;
    __shared__ __attribute__((aligned(1024))) char tile[(BM + BN) * 128];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave & 1, wn = wave >> 1;
    const int m0 = (int)(blockIdx.x / tiles_n) * BM, n0 = (int)(blockIdx.x % tiles_n) * BN, z = blockIdx.y;
    const int half = (p.K + BK - 1) / BK, total = p.a_low ? 2 * half : half, first = z * (p.klen / BK), last = min(total, first + p.klen / BK);
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    Staged<T, AX, BM, THREADS> as;
    Staged<T, BX, BN, THREADS> bs;
    auto fetch = [&](int t) {
        const int k0 = (t >= half ? t - half : t) * BK;
        as.load((const T *)(t >= half ? p.a_low : p.a), p.lda, m0, p.M, k0, p.K, tid);
        bs.load((const T *)p.b, p.ldb, n0, p.N, k0, p.K, tid);
    };
    if (first < last) fetch(first);
    for (int t = first; t < last; ++t) {
        __syncthreads();
        as.put(tile, tid);
        bs.put(tile + BM * 128, tid);
        __syncthreads();
        if (t + 1 < last) fetch(t + 1);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            Vec<T, Kind<T>::V> a[TM], b[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) a[i] = operand<T, AX, BM>(tile, (wm * TM + i) * 32, kk, lane);
#pragma unroll
            for (int j = 0; j < TN; ++j) b[j] = operand<T, BX, BN>(tile + BM * 128, (wn * TN + j) * 32, kk, lane);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = multiply<T>(a[i], b[j], acc[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int m = m0 + (wm * TM + i) * 32 + (lane & 31), n = n0 + (wn * TN + j) * 32 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
                if (m < p.M && n < p.N) {
                    if (p.part) p.part[((int64_t)z * p.M + m) * p.N + n] = acc[i][j][e];
                    else finish<T, OUT>(p, m, n, acc[i][j][e]);
                }
            }
}

// g = dy act'(pre) in two parts (binary32: one), and sums of g over a share of the rows for db.  A lane has a column.
constexpr int COLUMN_ROWS = 64;
template <typename T>
__global__ __launch_bounds__(256) void slope_kernel(const LinearOp p, const int groups, T *high, T *low, float *part)
{
    __shared__ float sums[4][64];
    const int lane = threadIdx.x & 63, row = threadIdx.x >> 6, blocks = (p.N + 63) / 64;
    const int n = (int)(blockIdx.x % blocks) * 64 + lane, group = blockIdx.x / blocks;
    float s = 0.0f;
    if (n < p.N)
        for (int64_t m = group * 4 + row; m < p.M; m += groups * 4) {
            float g = to_f32(((const T *)p.dy.p)[m * p.dy.ld + n]);
            if (p.act != HTS_ACT_NONE) {
                g *= slope_of(p.act, to_f32(((const T *)p.pre.p)[m * p.pre.ld + n]));
                const T h = from_f32<T>(g);
                high[m * p.N + n] = h;
                if (low) low[m * p.N + n] = from_f32<T>(g - to_f32(h));
            }
            s += g;
        }
    sums[row][lane] = s;
    __syncthreads();
    if (row == 0 && n < p.N && part) part[(int64_t)group * p.N + n] = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
}

int column_groups(int64_t M) { const int64_t g = ceil_div(M, COLUMN_ROWS); return (int)(g < 128 ? g : 128); }
// dw's reduction over the rows is cut where C has too few tiles for the compute units
int slices_of(int64_t rows, int64_t N, int64_t K, int bk)
{
    const int64_t tiles = ceil_div(N, 128) * ceil_div(K, 128), most = ceil_div(rows, 4 * bk);
    int64_t z = 512 / tiles;
    if (z > 16) z = 16;
    if (z > most) z = most;
    return (int)(z < 1 ? 1 : z);
}

template <typename T, typename OUT, bool AX, bool BX> hipError_t product(hts_seq_ctx &c, Product p, int slices)
{
    constexpr int BK = Kind<T>::BK;
    const int64_t total = ceil_div(p.K, BK) * (p.a_low ? 2 : 1);
    p.klen = (int)(ceil_div(total, slices) * BK);
    slices = (int)ceil_div(total * BK, p.klen);
    const int tn = (int)ceil_div(p.N, 128);
    hipLaunchKernelGGL((product_kernel<T, OUT, AX, BX, 128, 128>), dim3((uint32_t)(ceil_div(p.M, 128) * tn), slices), dim3(256), 0, c.stream, p, tn);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.part) e = launch_sum_partials(c, p.part, slices, (int64_t)p.M * p.N, SumTarget{(float *)p.y, (int64_t)p.M * p.N}, SumTarget{nullptr, 0}, SumTarget{nullptr, 0});
    return e;
}

struct Layout { int64_t high, low, columns, dw, total; };       // bytes
Layout layout(int size, int act, int64_t M, int64_t N, int64_t K)
{
    Layout l;
    l.high = 0;
    l.low = l.high + (act == HTS_ACT_NONE ? 0 : round_up(M * N * size, 256));
    l.columns = l.low + (act == HTS_ACT_NONE || size == 4 ? 0 : round_up(M * N * size, 256));
    l.dw = l.columns + round_up(4 * column_groups(M) * N, 256);
    const int z = slices_of(M, N, K, 128 / size);
    l.total = l.dw + (z > 1 ? 4 * z * N * K : 0);
    return l;
}

template <typename T> hipError_t forward(hts_seq_ctx &c, const LinearOp &op)
{
    Product p = {};
    p.a = op.x.p; p.lda = op.x.ld; p.b = op.w.p; p.ldb = op.w.ld; p.M = op.M; p.N = op.N; p.K = op.K;
    p.act = op.act; p.bias = op.bias; p.res = op.residual.p; p.ldr = op.residual.ld; p.y = op.y.p; p.ldy = op.y.ld; p.pre = op.pre.p; p.ldp = op.pre.ld;
    return product<T, T, false, false>(c, p, 1);
}

template <typename T> hipError_t backward(hts_seq_ctx &c, const LinearOp &op)
{
    const Layout at = layout(sizeof(T), op.act, op.M, op.N, op.K);
    const bool act = op.act != HTS_ACT_NONE;
    T *high = act ? (T *)(c.ws + at.high) : nullptr, *low = act && sizeof(T) == 2 ? (T *)(c.ws + at.low) : nullptr;
    float *columns = (float *)(c.ws + at.columns);
    hipError_t e = hipSuccess;
    if (act || op.db) {
        const int groups = column_groups(op.M);
        hipLaunchKernelGGL((slope_kernel<T>), dim3((uint32_t)(groups * ceil_div(op.N, 64))), dim3(256), 0, c.stream, op, groups, high, low, op.db ? columns : nullptr);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (op.db && (e = launch_sum_partials(c, columns, groups, op.N, SumTarget{op.db, op.N}, SumTarget{nullptr, 0}, SumTarget{nullptr, 0})) != hipSuccess) return e;
    }
    Product g = {};
    g.a = act ? high : op.dy.p; g.lda = act ? op.N : op.dy.ld;
    if (op.dx.p) {
        Product p = g;
        p.b = op.w.p; p.ldb = op.w.ld; p.M = op.M; p.N = op.K; p.K = op.N;
        p.res = op.add.p; p.ldr = op.add.ld; p.y = op.dx.p; p.ldy = op.dx.ld;
        if ((e = product<T, T, false, true>(c, p, 1)) != hipSuccess) return e;
    }
    if (op.dw) {
        Product p = g;
        const int z = slices_of(op.M, op.N, op.K, Kind<T>::BK);
        p.a_low = low; p.b = op.x.p; p.ldb = op.x.ld; p.M = op.N; p.N = op.K; p.K = op.M; p.y = op.dw; p.ldy = op.K;
        p.part = z > 1 ? (float *)(c.ws + at.dw) : nullptr;
        e = product<T, float, true, true>(c, p, z);
    }
    return e;
}

}  // namespace

int64_t linear_workspace(int precision, int act, int64_t M, int64_t N, int64_t K) { return layout(precision == HTS_PRECISION_BF16 ? 2 : 4, act, M, N, K).total; }
hipError_t launch_linear(hts_seq_ctx &c, int precision, const LinearOp &op) { return precision == HTS_PRECISION_BF16 ? forward<bf16_t>(c, op) : forward<float>(c, op); }
hipError_t launch_linear_backward(hts_seq_ctx &c, int precision, const LinearOp &op) { return precision == HTS_PRECISION_BF16 ? backward<bf16_t>(c, op) : backward<float>(c, op); }

}  // namespace hts
