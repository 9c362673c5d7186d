// Matrix products of the sequence memory: y = act(x W^T + b) + r and its gradients (see include/hts.h), on tiles of 32x32 matrix instructions.
//
// All three products are C[i][j] = sum_k A(i,k) B(j,k) with a kernel for each layout of the operands: along k in memory (x and W of the forward
// product, dz of dx) or across (W of dx, both operands of dw).  An operand tile is copied to LDS as it lies in memory, 16 bytes at a time; one along k
// is read by rows, one across by the transposing LDS read in bfloat16 (four neighbouring k of a column a lane) and word by word in binary32.
//   bfloat16: v_mfma_f32_32x32x16_bf16, k-tiles of 64;  binary32: v_mfma_f32_32x32x2_f32, k-tiles of 32.
// The operands go to the instruction in exchanged order, so a lane holds a row of C and four neighbouring columns of it; the sums go through LDS
// once more, so that rows leave as whole lines, with bias, activation and residual on the way.
// Rows that are whole numbers of 16 bytes, at addresses that are, are copied straight into LDS (buffer_load ... lds), a k-tile ahead; others
// through registers, entry by entry where a row ends.
// An activation's gradient in bfloat16 is the sum of three matrices, which a reduction goes over one after the other: 8192 x 2048 x 512 with silu, dx 69 us, dw 87, forming
// them 32 (in a trace; the call 170).
// What bounds it: 8192 x 2048 from 512 in bfloat16 with silu and its pre-activation, 32.2 us: 67 MB of outputs (13.5 us at the rate of a large copy), and
// 268 MB of operands from L2 to LDS at 15 TB/s or so, which two workgroups a compute unit overlap in part; matrix units are busy for a fifth.  The gradient of x there,
// without an activation, 25 us, of W 29 + 5.4, at the same rate from the L2.  Binary32 gradients of 1024 x 1024 x 512, 39 us: a wavefront alone on its SIMD, whose matrix
// instructions (a third of its cycles), LDS reads and scalar instructions follow one another.
#include "dmagemm.hpp"
#include "linear_plan.hpp"
#include "seq.hpp"

namespace hts {
namespace {

struct Product {
    const void *a, *b;
    int64_t part_stride;           // A may be the sum of `parts` matrices that far apart (entries): the reduction goes over each in turn, with the same b
    int parts;
    int64_t lda, ldb;
    int M, N, K;                   // C is M x N, reduction over K
    int klen;                      // reduction of a slice (of all parts of A together), whole k-tiles
    int act;
    const float *bias;
    const void *res;
    void *y, *pre;
    int64_t ldr, ldy, ldp;
    float *rows;                   // receives A's own sums over the reduction (db), NULL: not wanted.  y NULL: nothing else is wanted
    float *part;                   // slices > 1: a slice's C, where y is wanted, and at rows_at its `rows`
    int64_t rows_at, stride;       // entries; stride from slice to slice, a multiple of 4
    int slices;
};

template <typename T> struct Kind { static constexpr int V = 16 / sizeof(T), BK = 128 / sizeof(T); };       // entries of 16 bytes, k-tile

// where the 16 bytes with number s (along the row) of row r of an operand tile are, for operands along k: rows of 128 bytes, the slots exchanged so
// that the rows of an operand read fall into different banks
__host__ __device__ __forceinline__ int along_slot(int r, int s) { return s ^ ((r >> 1) & 7); }
// ... and for operands across: rows are k, B the tile's width.  bfloat16: 32-byte pieces exchanged by k, so that the four rows of a transposing read
// fall into different banks (of 32 entries four rows are all of them); binary32: 128-byte halves by k's bit 2, in which the halves of a wavefront differ
template <typename T, int B> __host__ __device__ __forceinline__ int across_slot(int k, int s)
{
    if constexpr (sizeof(T) == 2) return s ^ (B >= 128 ? (k & 3) << 2 | (k >> 2 & 1) << 1 : B >= 64 ? (k >> 1 & 1) << 2 : 0);
    else return B >= 64 ? s ^ (k >> 2 & 1) << 3 : s;
}
template <typename T, bool ACROSS, int B> __device__ __forceinline__ int piece_at(int r, int s) { return ACROSS ? r * (B * (int)sizeof(T)) + 16 * across_slot<T, B>(r, s) : r * 128 + 16 * along_slot(r, s); }

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
            *reinterpret_cast<Piece *>(lds + piece_at<T, ACROSS, B>(r, s)) = v[i];
        }
    }
};

// 16 bytes a lane, memory -> LDS: lane l's land at lds + 16 l (one address for the wavefront).  Written out, since the compiler waits for every copy that it knows to
// be on its way before a transposing LDS read, those of the k-tile after included; the kernel's own waits count them.  The compiler keeps no distances to
// what is inside: m0 is written one wait state ahead, and a scalar that a vector instruction writes has to be five ahead, which none is
// (tests/test_linear_copy_wait_states.py reads it from the built library).  (Rows of 8192, 512 x 2048: the
// gradient of x 38.7 -> 30.3 us).
typedef uint32_t Source __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void copy16(Source src, uint32_t lane, uint32_t all, const char *lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 : : "s"((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)lds), "v"(lane), "s"(src), "s"(all) : "memory", "m0");
}

// The same tile copied straight into LDS by WAVES wavefronts: 1 KB an instruction, k-tile after k-tile.  The exchange of slots is in the lanes' addresses; a
// piece that is not there gets an address beyond the matrix, which reads as zero.  From k-tile to k-tile a few scalar additions (with the addresses formed
// anew, 63 scalar instructions a k-tile: the gradient of x above 30.3 -> 27.0 us).
template <typename T, bool ACROSS, int B, int WAVES> struct Copied {
    static constexpr int V = Kind<T>::V, BK = Kind<T>::BK, COPIES = B / 8 / WAVES, SLOTS = ACROSS ? B / V : BK / V;
    static constexpr uint32_t BEYOND = 0xfffffff0u;
    static_assert(COPIES * 8 * WAVES == B, "tile");
    uint32_t at[COPIES];           // bytes from the tile's first row (along) or from the k-tile's (across)
    const char *start, *now;       // across: row 0 of the part, the k-tile's first row
    int64_t step, all, left;       // across: bytes from k-tile to k-tile, of a part, from the k-tile's first row on
    int64_t part;                  // bytes to the next part
    int k0, K;
    __device__ __forceinline__ void open(const T *p, int64_t ld, int first, int edge, int K_, int64_t part_stride, int part0, int k_first, int wave, int lane)
    {
        K = K_; k0 = k_first;
        part = part_stride * (int64_t)sizeof(T);
        step = BK * ld * (int64_t)sizeof(T);
        start = (const char *)p + part0 * part + (ACROSS ? 0 : first * ld * (int64_t)sizeof(T));
        all = ACROSS ? ((K - 1) * ld + edge) * (int64_t)sizeof(T) : ((edge - 1 - first) * ld + K) * (int64_t)sizeof(T);
        now = start + (ACROSS ? k0 / BK * step : 0);
        left = all - (ACROSS ? k0 / BK * step : 0);
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int piece = (wave * COPIES + i) * 64 + lane, r = piece / SLOTS, phys = piece % SLOTS;
            const int s = ACROSS ? across_slot<T, B>(r, phys) : along_slot(r, phys);
            at[i] = (uint32_t)((r * ld + (ACROSS ? first : 0) + s * V) * (int64_t)sizeof(T));
            if (ACROSS ? first + s * V >= edge : first + r >= edge) at[i] = BEYOND;
        }
    }
    __device__ __forceinline__ void copy(char *lds, int wave, int lane)
    {
        const uint64_t from = (uint64_t)(uintptr_t)now;
        const Source src = {(uint32_t)from, (uint32_t)(from >> 32), (uint32_t)(left < (int64_t)BEYOND ? left : (int64_t)BEYOND), 0x00020000u};
        const uint32_t off = ACROSS ? 0 : k0 * (int)sizeof(T);
        char *to = lds + wave * COPIES * 1024;
        if (ACROSS || k0 + BK <= K)
#pragma unroll
            for (int i = 0; i < COPIES; ++i) copy16(src, at[i], off, to + i * 1024);
        else                       // the row ends in this k-tile
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                const int piece = (wave * COPIES + i) * 64 + lane, s = along_slot(piece / SLOTS, piece % SLOTS);
                copy16(src, k0 + s * V < K ? at[i] : BEYOND, off, to + i * 1024);
            }
        k0 += BK;
        if constexpr (ACROSS) {
            if (k0 < K) { now += step; left -= step; }
            else { k0 = 0; start += part; now = start; left = all; }
        } else if (k0 >= K) { k0 = 0; now += part; }
    }
};

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 *lds_quad;

template <typename T> using Eight = Vec<T, 8>;

// operands of a k-tile's kk-th part (16 k in bfloat16, 8 in binary32) for 32 entries from `at`
template <typename T, bool ACROSS, int B> __device__ __forceinline__ Vec<T, Kind<T>::V> operand(const char *lds, int at, int kk, int lane)
{
    if constexpr (!ACROSS) return *reinterpret_cast<const Vec<T, Kind<T>::V> *>(lds + piece_at<T, false, B>(at + (lane & 31), 2 * kk + (lane >> 5)));
    else if constexpr (sizeof(T) == 2) {
        const int k = kk * 16 + (lane >> 5) * 8 + (lane >> 2 & 3), col = at + (lane & 16) + (lane & 3) * 4;
        const char *q0 = lds + piece_at<T, true, B>(k, col >> 3) + (col & 7) * 2, *q1 = lds + piece_at<T, true, B>(k + 4, col >> 3) + (col & 7) * 2;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad)(uintptr_t)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)q0);
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad)(uintptr_t)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)q1);
        return __builtin_bit_cast(Eight<T>, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        Vec<T, 4> r;
        const int col = at + (lane & 31);
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = *reinterpret_cast<const float *>(lds + piece_at<T, true, B>(kk * 8 + (lane >> 5) * 4 + i, col >> 2) + (col & 3) * 4);
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

// 8 neighbouring entries of a row, in 16-byte accesses at any address (entry by entry where rows were not whole words, 8192 x 1999 outputs and
// pre-activations took 86 us, now 60)
typedef uint32_t AnyWord __attribute__((ext_vector_type(4), aligned(2)));
template <typename T> __device__ __forceinline__ void get8(float (&v)[8], const T *p, int count)
{
    if (count >= 8) {
        Vec<T, 8> r;
        __builtin_memcpy(&r, p, sizeof r);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32(r[i]);
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? to_f32(p[i]) : 0.0f;
}
template <typename T> __device__ __forceinline__ void put8(T *p, const float (&v)[8], int count)
{
    if (count >= 8) {
        Vec<T, 8> r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = from_f32<T>(v[i]);
        // (past the L2's lines: 8192 x 2048 outputs and pre-activations 40 -> 33 us, since the operands stay there)
        AnyWord w[sizeof r / 16];
        __builtin_memcpy(w, &r, sizeof r);
#pragma unroll
        for (int i = 0; i < (int)(sizeof r / 16); ++i) __builtin_nontemporal_store(w[i], reinterpret_cast<AnyWord *>(p) + i);
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < count) p[i] = from_f32<T>(v[i]);
}
template <int ACT> __device__ __forceinline__ void activate(float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_f<ACT>(v[i]);
}
// C's entries (m, n ..), v their sums
template <typename T, typename OUT> __device__ __forceinline__ void finish(const Product &p, int m, int n, float (&v)[8], const float (&bias)[8])
{
    const int count = p.N - n;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += bias[i];
    if (p.pre) put8((T *)p.pre + m * p.ldp + n, v, count);
    if (p.act == HTS_ACT_RELU) activate<HTS_ACT_RELU>(v);
    else if (p.act == HTS_ACT_SILU) activate<HTS_ACT_SILU>(v);
    else if (p.act == HTS_ACT_GELU) activate<HTS_ACT_GELU>(v);
    if (p.res) {
        float r[8];
        get8(r, (const T *)p.res + m * p.ldr + n, count);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    put8((OUT *)p.y + m * p.ldy + n, v, count);
}

// Workgroups go to the eight dies in turn; a die gets neighbouring tiles, of a slice of the reduction and of a band of C, so that its L2 holds their operands.
__device__ __forceinline__ bool place(int tiles, int &tile)
{
    const int share = (tiles + 7) / 8;
    tile = (int)(blockIdx.x % 8) * share + (int)(blockIdx.x / 8);
    return blockIdx.x / 8 < share && tile < tiles;
}

// A workgroup: WM x WN x KS wavefronts.  A wavefront has BM / WM x BN / WN of the tile and every KS-th part of a k-tile.  DMA: copies straight into
// LDS, NS stages, one barrier a k-tile; otherwise two stages through registers.
template <int BM_, int BN_, int WM_, int WN_, int KS_, int NS_> struct Tiling { static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KS = KS_, NS = NS_, WAVES = WM_ * WN_ * KS_; };

template <typename T, typename OUT, bool AX, bool BX, class C, bool DMA>
__global__ __launch_bounds__(C::WAVES * 64, 2) void product_kernel(const Product p, const int tiles_n, const int tiles)
{
    constexpr int WAVES = C::WAVES, THREADS = WAVES * 64, BM = C::BM, BN = C::BN, BK = Kind<T>::BK, TM = BM / C::WM / 32, TN = BN / C::WN / 32, KS = C::KS, NS = DMA ? C::NS : 2;
    constexpr int STAGE = (BM + BN) * 128, SUMS = KS * BM * BN * 4;
    static_assert(TM * C::WM * 32 == BM && TN * C::WN * 32 == BN && 4 % KS == 0, "tiling");
    __shared__ __attribute__((aligned(1024))) char tile[NS * STAGE > SUMS ? NS * STAGE : SUMS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % C::WM, wn = wave / C::WM % C::WN, ks = wave / (C::WM * C::WN);
    int which;
    if (!place(tiles, which)) return;                  // the whole workgroup leaves
    const int per_slice = p.slices > 1 ? tiles / p.slices : tiles, z = which / per_slice, in_slice = which % per_slice;
    const int m0 = in_slice / tiles_n * BM, n0 = in_slice % tiles_n * BN;
    const int each = (p.K + BK - 1) / BK, total = p.parts * each, first = z * (p.klen / BK), nt = min(total, first + p.klen / BK) - first;
    // db: from the operands of A that the wavefronts of C's first column tile have anyway.  bfloat16: times a matrix of ones (by additions they would take twice as
    // long to unpack); binary32: added (dw of
    // 1024 x 512 from 1024 rows 23.0 us with a matrix of ones, whose wavefronts had twice the others' products, now 17.2)
    constexpr bool ROW_SUMS = AX && BX, BY_ONES = sizeof(T) == 2;
    const bool row_sums = ROW_SUMS && p.rows && n0 == 0 && wn == 0;
    f32x16 acc[TM][TN], sum[ROW_SUMS && BY_ONES ? TM : 1];
    float added[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) added[i] = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j][e] = 0.0f;
#pragma unroll
        for (int i = 0; i < (ROW_SUMS && BY_ONES ? TM : 1); ++i) sum[i][e] = 0.0f;
    }
    // all of a k-tile's reads are issued before its products
    auto compute = [&](const char *stage) {
        Vec<T, Kind<T>::V> a[4 / KS][TM], b[4 / KS][TN];
#pragma unroll
        for (int k = 0; k < 4 / KS; ++k) {
#pragma unroll
            for (int i = 0; i < TM; ++i) a[k][i] = operand<T, AX, BM>(stage, (wm * TM + i) * 32, k * KS + ks, lane);
#pragma unroll
            for (int j = 0; j < TN; ++j) b[k][j] = operand<T, BX, BN>(stage + BM * 128, (wn * TN + j) * 32, k * KS + ks, lane);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < 4 / KS; ++k)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = multiply<T>(a[k][i], b[k][j], acc[i][j]);
        if constexpr (ROW_SUMS) if (row_sums) {
            Vec<T, Kind<T>::V> ones;
#pragma unroll
            for (int e = 0; e < Kind<T>::V; ++e) ones[e] = from_f32<T>(1.0f);
#pragma unroll
            for (int k = 0; k < 4 / KS; ++k)
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    if constexpr (BY_ONES) sum[i] = multiply<T>(a[k][i], ones, sum[i]);
                    else added[i] += (a[k][i][0] + a[k][i][1]) + (a[k][i][2] + a[k][i][3]);
                }
        }
    };
    if constexpr (DMA) {
        Copied<T, AX, BM, WAVES> as;
        Copied<T, BX, BN, WAVES> bs;
        const int part0 = p.parts > 1 ? first / each : 0, k_first = (first - part0 * each) * BK;
        as.open((const T *)p.a, p.lda, m0, p.M, p.K, p.part_stride, part0, k_first, wave, lane);
        bs.open((const T *)p.b, p.ldb, n0, p.N, p.K, 0, 0, k_first, wave, lane);
        auto fetch = [&](int s) {
            as.copy(tile + s * STAGE, wave, lane);
            bs.copy(tile + s * STAGE + BM * 128, wave, lane);
        };
#pragma unroll
        for (int s = 0; s < NS - 1; ++s) if (s < nt) fetch(s);
        auto step = [&](int t, auto u) {
            constexpr int S = decltype(u)::value;
            // this wavefront's copies of k-tile t have landed (later ones' may be on their way) and its reads of k-tile t - 1 are done
            wait_tiles<NS - 2, Copied<T, AX, BM, WAVES>::COPIES + Copied<T, BX, BN, WAVES>::COPIES>(nt - 1 - t);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();              // everybody's
            asm volatile("" ::: "memory");
            if (t + NS - 1 < nt) fetch((S + NS - 1) % NS);
            compute(tile + S * STAGE);
        };
        for (int t = 0; t < nt; t += NS) dma_steps(step, t, nt, std::make_integer_sequence<int, NS>{});
    } else {
        Staged<T, AX, BM, THREADS> as;
        Staged<T, BX, BN, THREADS> bs;
        auto fetch = [&](int t) {
            const int part = p.parts > 1 ? (first + t) / each : 0, k0 = (first + t - part * each) * BK;
            as.load((const T *)p.a + part * p.part_stride, p.lda, m0, p.M, k0, p.K, tid);
            bs.load((const T *)p.b, p.ldb, n0, p.N, k0, p.K, tid);
        };
        auto put = [&](int s) { as.put(tile + s * STAGE, tid); bs.put(tile + s * STAGE + BM * 128, tid); };
        if (nt > 0) { fetch(0); put(0); }
        __syncthreads();
        for (int t = 0; t < nt; ++t) {
            if (t + 1 < nt) fetch(t + 1);
            compute(tile + (t & 1) * STAGE);
            if (t + 1 < nt) put((t + 1) & 1);
            __syncthreads();
        }
    }
    // the sums to LDS, 16 bytes at a time, slots exchanged by row; then a thread finishes 8 neighbouring entries
    float *sums = reinterpret_cast<float *>(tile);
    auto at = [](int k, int r, int slot) { return ((k * BM + r) * (BN / 4) + (slot ^ (r & 7))) * 4; };
    __syncthreads();
    if constexpr (ROW_SUMS) {
        if (p.rows && n0 == 0) {
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                float v = added[i];
                if constexpr (BY_ONES) v = sum[i][0];
                else v += __shfl_xor(v, 32);           // a lane has half of a row's k
                if (wn == 0 && lane < 32) sums[ks * BM + (wm * TM + i) * 32 + lane] = v;
            }
            __syncthreads();
            for (int r = tid; r < BM && m0 + r < p.M; r += THREADS) {
                float v = 0.0f;
#pragma unroll
                for (int s = 0; s < KS; ++s) v += sums[s * BM + r];
                (p.slices > 1 ? p.part + z * p.stride + p.rows_at : p.rows)[m0 + r] = v;
            }
            if (!p.y) return;
            __syncthreads();
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e];
                *reinterpret_cast<f32x4 *>(sums + at(ks, (wm * TM + i) * 32 + (lane & 31), (wn * TN + j) * 8 + 2 * q + (lane >> 5))) = v;
            }
    __syncthreads();
    // a thread's entries are in the same columns of its rows
    constexpr int ROW = BN / 8, ROWS = THREADS / ROW;
    const int c = tid % ROW, n = n0 + 8 * c;
    if (n >= p.N) return;
    float bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = p.bias && n + e < p.N ? p.bias[n + e] : 0.0f;
#pragma unroll 2
    for (int r = tid / ROW; r < BM; r += ROWS) {
        const int m = m0 + r;
        if (m >= p.M) break;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.0f;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 w = *reinterpret_cast<const f32x4 *>(sums + at(s, r, 2 * c + h));
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * h + e] += w[e];
            }
        if (p.slices > 1) put8(p.part + z * p.stride + (int64_t)m * p.N + n, v, p.N - n);
        else finish<T, OUT>(p, m, n, v, bias);
    }
}

// g = dy act'(pre), in bfloat16 as the sum of three numbers, 24 bits together: V neighbouring entries a thread
template <typename T, int V, int ACT>
__global__ __launch_bounds__(256) void slope_kernel(const LinearOp p, T *out, const int64_t part)
{
    const int across = p.N / V;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, m = i / across;
    if (m >= p.M) return;
    const int n = (int)(i - m * across) * V;
    const Loaded<T, V> dy = load_v<T, V>((const T *)p.dy.p + m * p.dy.ld + n), pre = load_v<T, V>((const T *)p.pre.p + m * p.pre.ld + n);
    constexpr int PARTS = sizeof(T) == 2 ? 3 : 1;
    float g[V];
#pragma unroll
    for (int e = 0; e < V; ++e) g[e] = to_f32(dy.e[e]) * act_slope<ACT>(to_f32(pre.e[e]));
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
        Loaded<T, V> h;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            // (what is left of a number that is not finite would be NaN, and of one that bfloat16 rounds to infinity infinite)
            const bool finite = __builtin_isfinite(g[e]);
            h.e[e] = from_f32<T>(PARTS > 1 && finite ? fminf(fmaxf(g[e], -0x1.fep+127f), 0x1.fep+127f) : g[e]);
            g[e] = finite ? g[e] - to_f32(h.e[e]) : 0.0f;
        }
        store_v<T, V>(out + k * part + m * p.N + n, h);
    }
}

// dw and db from the slices' sums: 4 neighbouring entries a thread, the slices in order
__global__ __launch_bounds__(256) void slices_kernel(const float *part, const int slices, const int64_t stride, float *dw, const int64_t n, float *db, const int rows)
{
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= stride) return;
    f32x4 s = *reinterpret_cast<const f32x4 *>(part + i);
#pragma unroll 8
    for (int k = 1; k < slices; ++k) s += *reinterpret_cast<const f32x4 *>(part + k * stride + i);
    if (dw && i + 4 <= n && ((uintptr_t)dw & 15) == 0) *reinterpret_cast<f32x4 *>(dw + i) = s;
    else
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (i + e < n) { if (dw) dw[i + e] = s[e]; }
            else if (db && i + e - n < rows) db[i + e - n] = s[e];
        }
}

template <typename T> bool words(const void *p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld * (int64_t)sizeof(T) % 16 == 0; }
// whether an operand's rows (`cols` entries) can be copied straight into LDS: whole 16-byte words, and a tile's rows within 32 bits.  Across, rows beyond
// the reduction's end have to be beyond the matrix, which they are not where its rows overlap or are one.
template <typename T, bool ACROSS> bool copies(const void *p, int64_t ld, int64_t cols)
{
    return words<T>(p, ld) && cols % Kind<T>::V == 0 && ld < (1ll << 31) / (128 * (int64_t)sizeof(T)) && (!ACROSS || ld >= cols);
}

template <typename T, typename OUT, bool AX, bool BX, class C> hipError_t product_on(hts_seq_ctx &c, Product p)
{
    const int64_t tn = ceil_div(p.N, C::BN), tiles = ceil_div(p.M, C::BM) * tn * p.slices;
    const bool dma = copies<T, AX>(p.a, p.lda, AX ? p.M : p.K) && copies<T, BX>(p.b, p.ldb, BX ? p.N : p.K) && p.part_stride % Kind<T>::V == 0;
    if (tiles > INT32_MAX - 8 || !launchable(ceil_div(tiles, 8) * 8, C::WAVES * 64)) return hipErrorInvalidConfiguration;
    const dim3 grid((uint32_t)(ceil_div(tiles, 8) * 8)), block(C::WAVES * 64);
    if (dma) hipLaunchKernelGGL((product_kernel<T, OUT, AX, BX, C, true>), grid, block, 0, c.stream, p, (int)tn, (int)tiles);
    else hipLaunchKernelGGL((product_kernel<T, OUT, AX, BX, C, false>), grid, block, 0, c.stream, p, (int)tn, (int)tiles);
    return hipGetLastError();
}

// columns: C's, by which the tiles are chosen
template <typename T, typename OUT, bool AX, bool BX> hipError_t product(hts_seq_ctx &c, Product p, const Slices &slices, int columns)
{
    p.klen = slices.klen; p.slices = slices.count; p.rows_at = slices.rows; p.stride = slices.stride;
    auto tiles = [&](int m, int n) { return ceil_div(p.M, m) * ceil_div(columns, n) * p.slices; };
    // The largest tiles that still give most compute units one: operands come from the L2 at a rate of its own, and the smaller the tiles the more of them.
    // Two workgroups of four wavefronts a unit from 400 tiles on (8192 x 2048 from 512: 33.5 us, eight wavefronts 45, 64 x 64 tiles 55), eight wavefronts on three stages
    // below (8192 x 512 from 2048 and its other gradient: 66.9, four wavefronts and four stages 76.6, 64 x 64 tiles 74.3).
    hipError_t e;
    if (tiles(128, 128) >= 400) e = product_on<T, OUT, AX, BX, Tiling<128, 128, 2, 2, 1, 2>>(c, p);
    else if (tiles(128, 128) >= 192) e = product_on<T, OUT, AX, BX, Tiling<128, 128, 2, 2, 2, 3>>(c, p);
    else if (tiles(64, 64) >= 192) e = product_on<T, OUT, AX, BX, Tiling<64, 64, 2, 2, 1, sizeof(T) == 2 ? 2 : 3>>(c, p);
    else if (tiles(64, 32) >= 192) e = product_on<T, OUT, AX, BX, Tiling<64, 32, 2, 1, 2, 3>>(c, p);
    else e = product_on<T, OUT, AX, BX, Tiling<32, 32, 1, 1, 4, 4>>(c, p);
    if (e != hipSuccess || p.slices == 1) return e;
    hipLaunchKernelGGL(slices_kernel, dim3((uint32_t)ceil_div(p.stride, 1024)), dim3(256), 0, c.stream, p.part, p.slices, p.stride, (float *)p.y, p.rows_at, p.rows, p.M);
    return hipGetLastError();
}

template <typename T> hipError_t forward(hts_seq_ctx &c, const LinearOp &op)
{
    Product p = {};
    p.parts = 1;
    p.a = op.x.p; p.lda = op.x.ld; p.b = op.w.p; p.ldb = op.w.ld; p.M = op.M; p.N = op.N; p.K = op.K;
    p.act = op.act; p.bias = op.bias; p.res = op.residual.p; p.ldr = op.residual.ld; p.y = op.y.p; p.ldy = op.y.ld; p.pre = op.pre.p; p.ldp = op.pre.ld;
    return product<T, T, false, false>(c, p, cut(p.M, p.N, p.K, Kind<T>::BK, 1, 1, true), p.N);
}

template <typename T, int V> hipError_t slopes(hts_seq_ctx &c, const LinearOp &op, T *out, int64_t part)
{
    const int64_t workgroups = ceil_div((int64_t)op.M * (op.N / V), 256);
    if (!launchable(workgroups, 256)) return hipErrorInvalidConfiguration;
    const dim3 grid((uint32_t)workgroups), block(256);
    if (op.act == HTS_ACT_RELU) hipLaunchKernelGGL((slope_kernel<T, V, HTS_ACT_RELU>), grid, block, 0, c.stream, op, out, part);
    else if (op.act == HTS_ACT_SILU) hipLaunchKernelGGL((slope_kernel<T, V, HTS_ACT_SILU>), grid, block, 0, c.stream, op, out, part);
    else hipLaunchKernelGGL((slope_kernel<T, V, HTS_ACT_GELU>), grid, block, 0, c.stream, op, out, part);
    return hipGetLastError();
}

template <typename T> hipError_t backward(hts_seq_ctx &c, const LinearOp &op)
{
    const LinearLayout at = linear_layout(sizeof(T), op.act, op.M, op.N, op.K);
    const bool act = op.act != HTS_ACT_NONE;
    T *slope = (T *)(c.ws + at.slope);
    constexpr int V = Kind<T>::V;
    hipError_t e = hipSuccess;
    if (act) {
        const bool wide = op.N % V == 0 && words<T>(op.dy.p, op.dy.ld) && words<T>(op.pre.p, op.pre.ld);
        if ((e = wide ? slopes<T, V>(c, op, slope, at.stride) : slopes<T, 1>(c, op, slope, at.stride)) != hipSuccess) return e;
    }
    Product g = {};
    g.parts = 1;
    g.a = act ? slope : op.dy.p; g.lda = act ? op.N : op.dy.ld;
    if (op.dx.p) {
        Product p = g;
        p.b = op.w.p; p.ldb = op.w.ld; p.M = op.M; p.N = op.K; p.K = op.N;
        p.res = op.add.p; p.ldr = op.add.ld; p.y = op.dx.p; p.ldy = op.dx.ld;
        p.parts = parts_of(sizeof(T), op.act); p.part_stride = at.stride;
        if ((e = product<T, T, false, true>(c, p, cut(p.M, p.N, p.K, Kind<T>::BK, p.parts, 1, true), p.N)) != hipSuccess) return e;
    }
    if (op.dw || op.db) {
        Product p = g;
        const Slices slices = weight_slices(sizeof(T), op.act, op.M, op.N, op.K, op.dw != nullptr);
        p.parts = parts_of(sizeof(T), op.act); p.part_stride = at.stride; p.b = op.x.p; p.ldb = op.x.ld; p.M = op.N; p.N = weight_columns(sizeof(T), op.dw != nullptr, op.N, op.K); p.K = op.M; p.y = op.dw; p.ldy = op.K; p.rows = op.db;
        // without dw: one column tile, of any operand with as many rows (x may not be there), whose products go nowhere; the same slices and tiles, hence the same bits
        if (!op.dw) { p.b = g.a; p.ldb = g.lda; }
        p.part = slices.count > 1 ? (float *)(c.ws + at.part) : nullptr;
        e = product<T, float, true, true>(c, p, slices, op.K);
    }
    return e;
}

}  // namespace

int64_t linear_workspace(int precision, int act, int64_t M, int64_t N, int64_t K) { return linear_layout(precision == HTS_PRECISION_BF16 ? 2 : 4, act, M, N, K).total; }
hipError_t launch_linear(hts_seq_ctx &c, int precision, const LinearOp &op) { return precision == HTS_PRECISION_BF16 ? forward<bf16_t>(c, op) : forward<float>(c, op); }
hipError_t launch_linear_backward(hts_seq_ctx &c, int precision, const LinearOp &op) { return precision == HTS_PRECISION_BF16 ? backward<bf16_t>(c, op) : backward<float>(c, op); }

}  // namespace hts
