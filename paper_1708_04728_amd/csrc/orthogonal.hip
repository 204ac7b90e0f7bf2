// Orthogonalised matrices by Newton-Schulz products, and the descent step on them (dr_orthogonalise, dr_muon_step).
//
//   X = U / (|U|_F + eps), on the transpose where U has more rows than columns: X has m rows and n >= m columns.
//   `steps` times:  A = X X^T,   Q = a I + b A + c A A,   X = Q X
//
// The polynomial moves every singular value of X towards one and leaves the singular vectors, so that X ends near U V^T of U = U S V^T.  It multiplies
// small singular values by a = 3.4 in every step, and with them what roundings of X leave there: 64 to 512 rows of a filter's gradient end 1e-2 off with X, A and Q
// in bf16, 2e-5 with two bf16 pieces of each value (16 bits), 2e-6 to 3e-5 in fp32.  So matrices are held as bf16 pieces whose sum is the value, three for fp32 (all
// of its bits) and two for bf16 results, and multiplied on the bf16 matrix cores: six and three products of pieces for each product (f32_pieces.h).
//
// A and A A are symmetric: only blocks on and below the diagonal are computed, and stored on both sides.
//
// Layout.  All three products are of rows with rows (A = X X^T; A A = A A^T; Q X = Q (X^T)^T, with X kept in both orders).  An operand is stored as the matrix
// instruction reads it: blocks of 32 rows x 16 k, a KiB for each piece, lane l's 16 bytes (row l % 32, k from 8 (l / 32) on) at 16 l; blocks of a row of blocks follow each
// other, the pieces of a block too.  So an operand of the matrix instruction is one contiguous KiB, wherever it is read from.  Rows and columns are padded with zeros to 32.
//
// A call works on a list of matrices of any sizes: each of its launches runs one product of all of them.  What a launch needs to know of them travels as its argument
// (a table in memory costs every launch two loads one after the other before the first operand, 2 us of 6).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dr_internal.h"
#include "f32_pieces.h"

namespace dr {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int BLOCK = 1024;                  // bytes of a block of 32 rows x 16 k of one piece
constexpr int PITCH = 36;                    // floats of a row of 32 in LDS
constexpr int SQUARES = 1024;                // most workgroups (and partial sums of squares) of a matrix
enum { GRAM = 0, POLY = 1, APPLY = 2, PRODUCTS = 3 };

// The matrices of a launch; arrays by what is looked up together.  A list is worked on JOBS at a time.
constexpr int JOBS = 64;
struct Jobs {
    int first[JOBS];                         // first workgroup; INT_MAX behind the last matrix
    unsigned operands[JOBS];                 // its operands' place in the workspace, in KiB
    int mb[JOBS], nb[JOBS];                  // blocks of 32 of the short and of the long side
    int rows[JOBS], cols[JOBS];
    int squares[JOBS];                       // its first partial sum of squares
    const void* g[JOBS];
    float* momentum[JOBS];                   // (descent step only)
    void* o[JOBS];                           // the result, or the weights
    float scale[JOBS];                       // descent step: lr sqrt(max(1, rows / cols))
};

struct Call {
    double* squares;
    unsigned char* ws;
    int count;
    float a, b, c, eps;
    float mu, keep;                          // descent step: momentum; 1 - lr decay
};

// A matrix of a launch as its kernels see it
struct Mat {
    int k, mb, nb, rows, cols;
    bool tall;                               // rows > cols: X is the transpose
};
__device__ __forceinline__ Mat find_matrix(const Jobs& j, int count, int id)
{
    int k = 0;
    if (count > 1) {
#pragma unroll
        for (int i = 1; i < JOBS; ++i) k += j.first[i] <= id ? 1 : 0;
    }
    k = __builtin_amdgcn_readfirstlane(k);
    return Mat{k, j.mb[k], j.nb[k], j.rows[k], j.cols[k], j.rows[k] > j.cols[k]};
}

// Operands of a matrix: X, X^T twice (a product reads one and writes the other), A, Q
template <int P>
struct Operands {
    unsigned char *x, *xt0, *xt1, *a, *q;
    __device__ __forceinline__ Operands(const Call& c, const Jobs& j, const Mat& m)
    {
        const size_t wide = (size_t)m.mb * m.nb * (2 * P * BLOCK), square = (size_t)m.mb * m.mb * (2 * P * BLOCK);
        x = c.ws + (size_t)j.operands[m.k] * 1024;
        xt0 = x + wide;
        xt1 = xt0 + wide;
        a = xt1 + wide;
        q = a + square;
    }
};
__device__ __forceinline__ size_t block_at(int P, int rb, int kblocks32, int kb32) { return ((size_t)rb * kblocks32 + kb32) * (2 * P * BLOCK); }

// partial sums of squares of a matrix: workgroups of 256 threads, 16 elements each and more
__host__ __device__ inline int squares_of(int rows, int cols)
{
    const size_t n = ((size_t)rows * cols + 4095) / 4096;
    return (int)(n < SQUARES ? n : SQUARES);
}

__device__ __forceinline__ double sum256(double v, double* red)
{
    red[threadIdx.x] = v;
    __syncthreads();
    for (int d = 128; d >= 1; d >>= 1) {
        if ((int)threadIdx.x < d) red[threadIdx.x] += red[threadIdx.x + d];
        __syncthreads();
    }
    return red[0];
}

// Momentum (descent step), and the sums of the squares of U's elements, in double: a square of 1e20 or 1e-30 is no fp32 number
template <typename T, bool MUON>
__global__ __launch_bounds__(256) void squares_kernel(const Call c, const Jobs j)
{
    __shared__ double red[256];
    const Mat m = find_matrix(j, c.count, blockIdx.x);
    const T* const g = (const T*)j.g[m.k];
    float* const mom = j.momentum[m.k];
    const int me = (int)blockIdx.x - j.first[m.k];
    const size_t total = (size_t)m.rows * m.cols, step = (size_t)squares_of(m.rows, m.cols) * 256;
    double s = 0.0;
    for (size_t i = (size_t)me * 256 + threadIdx.x; i < total; i += step * 8) {
        float u[8], v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u[e] = i + e * step < total ? Store<T>::ld(g + i + e * step) : 0.f;
            if constexpr (MUON) v[e] = i + e * step < total ? mom[i + e * step] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (MUON) {
                v[e] = c.mu * v[e] + u[e];
                if (i + e * step < total) mom[i + e * step] = v[e];
                u[e] += c.mu * v[e];
            }
            s += (double)u[e] * (double)u[e];
        }
    }
    s = sum256(s, red);
    if (threadIdx.x == 0) c.squares[j.squares[m.k] + me] = s;
}

// Eight values as P bf16 pieces
template <int P>
__device__ __forceinline__ void cut8(const float (&v)[8], u32x4 (&p)[P])
{
    if constexpr (P == 3) split8(v, p[0], p[1], p[2]);
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned h = pack_bf16x2(v[2 * i], v[2 * i + 1]);
            p[0][i] = h;
            p[1][i] = pack_bf16x2(v[2 * i] - __uint_as_float(h << 16), v[2 * i + 1] - __uint_as_float(h & 0xFFFF0000u));
        }
    }
}

template <int P>
__device__ __forceinline__ void join8(const u32x4 (&p)[P], float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = v[2 * i + 1] = 0.f;
#pragma unroll
        for (int e = P - 1; e >= 0; --e) {
            v[2 * i] += __uint_as_float(p[e][i] << 16);
            v[2 * i + 1] += __uint_as_float(p[e][i] & 0xFFFF0000u);
        }
    }
}

// Half of a 32 x 32 block that is in LDS, k from 16 kb on, as this lane's 16 bytes of an operand block: rows = the tile's rows (COLUMNS: its columns)
template <bool COLUMNS>
__device__ __forceinline__ void operand8(const float* tile, int kb, float (&v)[8])
{
    const int lane = threadIdx.x & 63, l32 = lane & 31, k0 = kb * 16 + (lane >> 5) * 8;
    if constexpr (COLUMNS) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[(k0 + e) * PITCH + l32];
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 t = *reinterpret_cast<const f32x4*>(tile + l32 * PITCH + k0 + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * h + e] = t[e];
        }
    }
}
template <int P>
__device__ __forceinline__ void put8(const float (&v)[8], unsigned char* block, int kb)
{
    u32x4 p[P];
    cut8<P>(v, p);
#pragma unroll
    for (int e = 0; e < P; ++e) *reinterpret_cast<u32x4*>(block + (kb * P + e) * BLOCK + (threadIdx.x & 63) * 16) = p[e];
}

// X = U / (|U| + eps) in both orders, cut into pieces: a wave per 32 x 32 block
template <typename T, int P, bool MUON>
__global__ __launch_bounds__(256) void cut_kernel(const Call c, const Jobs j)
{
    __shared__ __attribute__((aligned(16))) float tiles[4][32 * PITCH];
    __shared__ double red[256];
    const Mat m = find_matrix(j, c.count, blockIdx.x);
    const Operands<P> op(c, j, m);
    const T* const g = (const T*)j.g[m.k];
    const float* const mom = j.momentum[m.k];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int b = ((int)blockIdx.x - j.first[m.k]) * 4 + wave;
    const bool on = b < m.mb * m.nb;
    const int bi = on ? b / m.nb : 0, bj = on ? b - bi * m.nb : 0;
    float* const tile = tiles[wave];
    // lanes along the matrix's own columns; the tile's rows are X's
    const int r0 = (m.tall ? bj : bi) * 32, col = (m.tall ? bi : bj) * 32 + l32;
    float u[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = r0 + 2 * r + half;
        const size_t i = (size_t)row * m.cols + col;
        u[r] = 0.f;
        if (on && row < m.rows && col < m.cols) {
            u[r] = Store<T>::ld(g + i);
            if constexpr (MUON) u[r] += c.mu * mom[i];
        }
    }
    double s = 0.0;
    for (int i = threadIdx.x; i < squares_of(m.rows, m.cols); i += 256) s += c.squares[j.squares[m.k] + i];
    const double inv = 1.0 / (sqrt(sum256(s, red)) + (double)c.eps);
#pragma unroll
    for (int r = 0; r < 16; ++r) tile[m.tall ? l32 * PITCH + 2 * r + half : (2 * r + half) * PITCH + l32] = (float)((double)u[r] * inv);
    __syncthreads();
    if (!on) return;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
        float v[8];
        operand8<false>(tile, kb, v);
        put8<P>(v, op.x + block_at(P, bi, m.nb, bj), kb);
        operand8<true>(tile, kb, v);
        put8<P>(v, op.xt0 + block_at(P, bj, m.mb, bi), kb);
    }
}

// What becomes of a 32 x 32 block (bi, bj) of a product, which is in LDS: task t = 0 .. 3 stores a half of it in one of the two orders
template <int P, int WHAT>
__device__ __forceinline__ void finish_task(const Call& c, const Mat& m, const Operands<P>& op, const float* tile, int bi, int bj, int turn, int t)
{
    const int kb = t & 1;
    const bool flip = t >= 2;
    float v[8];
    if (WHAT != APPLY && flip && bi == bj) return;
    if (flip) operand8<true>(tile, kb, v);
    else operand8<false>(tile, kb, v);
    const int rb = flip ? bj : bi, cb = flip ? bi : bj;
    if constexpr (WHAT == APPLY) put8<P>(v, flip ? (turn ? op.xt0 : op.xt1) + block_at(P, rb, m.mb, cb) : op.x + block_at(P, rb, m.nb, cb), kb);
    else if constexpr (WHAT == GRAM) put8<P>(v, op.a + block_at(P, rb, m.mb, cb), kb);
    else {
        const int lane = threadIdx.x & 63, diagonal = cb * 32 + kb * 16 + (lane >> 5) * 8 - rb * 32 - (lane & 31);      // column of element 0 minus row
        const unsigned char* const a = op.a + block_at(P, rb, m.mb, cb) + kb * P * BLOCK + lane * 16;
        u32x4 p[P];
        float w[8];
#pragma unroll
        for (int e = 0; e < P; ++e) p[e] = *reinterpret_cast<const u32x4*>(a + e * BLOCK);
        join8<P>(p, w);
        // (also on the diagonal of the rows that pad X: what they multiply is zero)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c.b * w[e] + c.c * v[e] + (diagonal + e == 0 ? c.a : 0.f);
        put8<P>(v, op.q + block_at(P, rb, m.mb, cb), kb);
    }
}
// ... of the last product: the result, or the weights; rows r0, r0 + step, ... of the matrix' own 32 x 32 block
template <typename T, bool MUON>
__device__ __forceinline__ void finish_result(const Call& c, const Jobs& j, const Mat& m, const float* tile, int bi, int bj, int r0, int step)
{
    const int l32 = threadIdx.x & 31;
#pragma unroll 4
    for (int r = r0; r < 32; r += step) {
        const int row = (m.tall ? bj : bi) * 32 + r, col = (m.tall ? bi : bj) * 32 + l32;
        if (row >= m.rows || col >= m.cols) continue;
        const float v = tile[m.tall ? l32 * PITCH + r : r * PITCH + l32];
        const size_t i = (size_t)row * m.cols + col;
        if constexpr (MUON) {
            float* const w = (float*)j.o[m.k];
            w[i] = c.keep * w[i] - j.scale[m.k] * v;
        } else Store<T>::st((T*)j.o[m.k] + i, v);
    }
}

// Tile number t of a matrix -> its first blocks; tiles of T x T blocks
template <int WHAT, int T>
__device__ __forceinline__ void tile_blocks(const Mat& m, int t, int& bi, int& bj)
{
    if constexpr (WHAT == APPLY) {
        const int tn = (m.nb + T - 1) / T, i = t / tn;
        bi = i * T;
        bj = (t - i * tn) * T;
    } else {                                 // on and below the diagonal, row by row
        int i = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
        while ((i + 1) * (i + 2) / 2 <= t) ++i;
        while (i * (i + 1) / 2 > t) --i;
        bi = i * T;
        bj = (t - i * (i + 1) / 2) * T;
    }
}

template <int P>
__device__ __forceinline__ void multiply(const u32x4 (&a)[P], const u32x4 (&b)[P], f32x16& large, f32x16& small)
{
    large = mfma(a[0], b[0], large);
    small = mfma(a[0], b[1], small);
    small = mfma(a[1], b[0], small);
    if constexpr (P == 3) {
        small = mfma(a[1], b[1], small);
        small = mfma(a[0], b[2], small);
        small = mfma(a[2], b[0], small);
    }
}

// A product of small matrices: W waves share a tile of T x T blocks, every wave a W-th of the contraction.  Operands go straight to registers, AHEAD k-blocks of them
// while as many are multiplied: what such a product waits for is its first operands.
template <typename E, int P, int WHAT, int T, int W, bool MUON>
__global__ __launch_bounds__(W * 64) void product_kernel(const Call c, const Jobs j, int turn, int last)
{
    constexpr int AHEAD = T == 1 ? 4 : 2;
    __shared__ __attribute__((aligned(16))) float sums[W][T * T][32 * PITCH];
    const Mat m = find_matrix(j, c.count, blockIdx.x);
    const Operands<P> op(c, j, m);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    int bi, bj;
    tile_blocks<WHAT, T>(m, (int)blockIdx.x - j.first[m.k], bi, bj);
    const unsigned char* const left = WHAT == GRAM ? op.x : WHAT == POLY ? op.a : op.q;
    const unsigned char* const right = WHAT == GRAM ? op.x : WHAT == POLY ? op.a : turn ? op.xt1 : op.xt0;
    const int kblocks = 2 * (WHAT == GRAM ? m.nb : m.mb), lrows = m.mb, rrows = WHAT == APPLY ? m.nb : m.mb;
    const unsigned char *lp[T], *rp[T];
#pragma unroll
    for (int i = 0; i < T; ++i) {            // (a block beyond the last is the last again, and is not stored)
        lp[i] = left + (size_t)min(bi + i, lrows - 1) * kblocks * P * BLOCK + lane * 16;
        rp[i] = right + (size_t)min(bj + i, rrows - 1) * kblocks * P * BLOCK + lane * 16;
    }
    f32x16 large[T][T], small[T][T];
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int k = 0; k < T; ++k)
#pragma unroll
            for (int v = 0; v < 16; ++v) large[i][k][v] = small[i][k][v] = 0.f;
    u32x4 a[2][AHEAD][T][P], b[2][AHEAD][T][P];
    auto fetch = [&](int kb0, auto set) __attribute__((always_inline)) {
        constexpr int S = decltype(set)::value;
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            const size_t at = (size_t)min(kb0 + n * W, kblocks - 1) * P * BLOCK;
#pragma unroll
            for (int i = 0; i < T; ++i)
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    a[S][n][i][e] = *reinterpret_cast<const u32x4*>(lp[i] + at + e * BLOCK);
                    b[S][n][i][e] = *reinterpret_cast<const u32x4*>(rp[i] + at + e * BLOCK);
                }
        }
    };
    auto products = [&](int kb0, auto set) __attribute__((always_inline)) {
        constexpr int S = decltype(set)::value;
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            if (kb0 + n * W >= kblocks) break;
#pragma unroll
            for (int i = 0; i < T; ++i)
#pragma unroll
                for (int k = 0; k < T; ++k) multiply<P>(a[S][n][i], b[S][n][k], large[i][k], small[i][k]);
        }
    };
    using std::integral_constant;
    fetch(wave, integral_constant<int, 0>{});
    for (int kb = wave; kb < kblocks; kb += 2 * AHEAD * W) {
        if (kb + AHEAD * W < kblocks) fetch(kb + AHEAD * W, integral_constant<int, 1>{});
        products(kb, integral_constant<int, 0>{});
        if (kb + 2 * AHEAD * W < kblocks) fetch(kb + 2 * AHEAD * W, integral_constant<int, 0>{});
        products(kb + AHEAD * W, integral_constant<int, 1>{});
    }
    // register v holds row 8 (v / 4) + 4 half + v % 4 of column lane % 32
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int k = 0; k < T; ++k)
#pragma unroll
            for (int v = 0; v < 16; ++v) sums[wave][i * T + k][(8 * (v >> 2) + 4 * half + (v & 3)) * PITCH + l32] = large[i][k][v] + small[i][k][v];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < (T * T * 1024 + W * 64 - 1) / (W * 64); ++n) {
        const int i = n * W * 64 + threadIdx.x, blk = i >> 10, at = ((i >> 5) & 31) * PITCH + (i & 31);
        if (T * T * 1024 % (W * 64) != 0 && i >= T * T * 1024) break;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) s += sums[w][blk][at];
        sums[0][blk][at] = s;
    }
    __syncthreads();
    if (WHAT == APPLY && last) {
        for (int blk = 0; blk < T * T; ++blk) {
            const int i = bi + blk / T, k = bj + blk % T;
            if (i < lrows && k < rrows) finish_result<E, MUON>(c, j, m, sums[0][blk], i, k, wave * 2 + half, 2 * W);
        }
        return;
    }
    for (int t = wave; t < T * T * 4; t += W) {
        const int blk = t >> 2, i = bi + blk / T, k = bj + blk % T;
        if (i < lrows && k < rrows && (WHAT == APPLY || i >= k)) finish_task<P, WHAT>(c, m, op, sums[0][blk], i, k, turn, t & 3);
    }
}

// ---- the plan of a call: made in the same way to size the workspace and to run
struct Plan { size_t operands, total; };      // in the workspace; squares come first

int tiles_of(int what, int mb, int nb, int T)
{
    const int tm = (mb + T - 1) / T, tn = (nb + T - 1) / T;
    return what == APPLY ? tm * tn : tm * (tm + 1) / 2;
}
size_t operand_bytes(int rows, int cols, int P)
{
    const size_t mb = (std::min(rows, cols) + 31) / 32, nb = (std::max(rows, cols) + 31) / 32;
    return (3 * mb * nb + 2 * mb * mb) * 2 * P * BLOCK;
}

template <class Shape>
Plan make_plan(int count, int P, Shape shape)
{
    size_t squares = 0, at = 0;
    for (int i = 0; i < count; ++i) {
        int rows, cols;
        shape(i, rows, cols);
        squares += squares_of(rows, cols);
        at += operand_bytes(rows, cols, P);
    }
    Plan p;
    p.operands = align_up(squares * sizeof(double), 1024);
    p.total = p.operands + at;
    return p;
}

// count entries of j, for launches whose matrix i has `units(mb, nb, rows, cols)` workgroups
template <class Units>
unsigned number(Jobs& j, int count, Units units)
{
    unsigned at = 0;
    for (int i = 0; i < JOBS; ++i) {
        j.first[i] = i < count ? (int)at : 0x7FFFFFFF;
        if (i < count) at += units(j.mb[i], j.nb[i], j.rows[i], j.cols[i]);
    }
    return at;
}

template <typename E, int P, bool MUON>
int run(Call c, Jobs& j, int count, int steps, hipStream_t st)
{
    c.count = count;
    const unsigned squares = number(j, count, [](int, int, int r, int co) { return squares_of(r, co); });
    if (squares == 0) return DR_OK;
    hipLaunchKernelGGL((squares_kernel<E, MUON>), dim3(squares), dim3(256), 0, st, c, j);
    const unsigned cuts = number(j, count, [](int mb, int nb, int, int) { return (mb * nb + 3) / 4; });
    hipLaunchKernelGGL((cut_kernel<E, P, MUON>), dim3(cuts), dim3(256), 0, st, c, j);
    auto product = [&](auto what, int turn, int last) {
        constexpr int WHAT = decltype(what)::value;
        constexpr bool END = WHAT == APPLY && MUON;      // (the other products are the same for every result)
        typedef std::conditional_t<WHAT == APPLY, E, float> R;
        const unsigned fine = number(j, count, [](int mb, int nb, int, int) { return tiles_of(WHAT, mb, nb, 1); });
        if (fine <= 2u * device_cus()) hipLaunchKernelGGL((product_kernel<R, P, WHAT, 1, 8, END>), dim3(fine), dim3(512), 0, st, c, j, turn, last);
        else {
            const unsigned units = number(j, count, [](int mb, int nb, int, int) { return tiles_of(WHAT, mb, nb, 2); });
            hipLaunchKernelGGL((product_kernel<R, P, WHAT, 2, 4, END>), dim3(units), dim3(256), 0, st, c, j, turn, last);
        }
    };
    for (int s = 0; s < steps; ++s) {
        const int last = s + 1 == steps;
        product(std::integral_constant<int, GRAM>{}, s & 1, last);
        product(std::integral_constant<int, POLY>{}, s & 1, last);
        product(std::integral_constant<int, APPLY>{}, s & 1, last);
    }
    return check_launch("orthogonalise");
}

// The list, JOBS matrices that are not empty at a time.  fill(i, rows, cols, j, k): matrix i's shape and, with j, its entry k
template <typename E, int P, bool MUON, class Fill>
int run_list(const Plan& p, Call c, int count, int steps, hipStream_t st, Fill fill)
{
    Jobs j;
    int n = 0, squares = 0;
    size_t at = p.operands;
    for (int i = 0; i < count; ++i) {
        int rows, cols;
        fill(i, rows, cols, j, n);
        if (rows && cols) {
            j.rows[n] = rows; j.cols[n] = cols;
            j.mb[n] = (std::min(rows, cols) + 31) / 32;
            j.nb[n] = (std::max(rows, cols) + 31) / 32;
            j.operands[n] = (unsigned)(at / 1024);
            j.squares[n] = squares;
            at += operand_bytes(rows, cols, P);
            squares += squares_of(rows, cols);
            ++n;
        }
        if (n == JOBS || (i + 1 == count && n)) {
            if (const int rc = run<E, P, MUON>(c, j, n, steps, st)) return rc;
            n = 0;
        }
    }
    return DR_OK;
}

Call make_call(const dr_newton_schulz& ns, void* ws)
{
    Call c{};
    c.ws = (unsigned char*)ws;
    c.squares = (double*)ws;
    c.a = ns.a; c.b = ns.b; c.c = ns.c; c.eps = ns.eps;
    return c;
}

}  // namespace

size_t orthogonalise_workspace_bytes(int count, const dr_matrix* ms, int dtype)
{
    return make_plan(count, dtype == DR_F32 ? 3 : 2, [&](int i, int& r, int& c) { r = ms[i].rows; c = ms[i].cols; }).total;
}

int launch_orthogonalise(int count, const dr_matrix* ms, int dtype, const void* const* g, void* const* o, const dr_newton_schulz& ns, void* ws, hipStream_t st)
{
    const Plan p = make_plan(count, dtype == DR_F32 ? 3 : 2, [&](int i, int& r, int& c) { r = ms[i].rows; c = ms[i].cols; });
    const Call c = make_call(ns, ws);
    TraceScope trace("orthogonalise", nullptr, count, st);
    auto fill = [&](int i, int& r, int& cols, Jobs& j, int k) {
        r = ms[i].rows; cols = ms[i].cols;
        j.g[k] = g[i];
        j.momentum[k] = nullptr;
        j.o[k] = o[i];
        j.scale[k] = 0.f;
    };
    return dtype == DR_F32 ? run_list<float, 3, false>(p, c, count, ns.steps, st, fill) : run_list<uint16_t, 2, false>(p, c, count, ns.steps, st, fill);
}

size_t muon_step_workspace_bytes(int count, const dr_muon_param* ps)
{
    return make_plan(count, 3, [&](int i, int& r, int& c) { r = ps[i].rows; c = ps[i].cols; }).total;
}

int launch_muon_step(int count, const dr_muon_param* ps, const dr_muon& opt, void* ws, hipStream_t st)
{
    const Plan p = make_plan(count, 3, [&](int i, int& r, int& c) { r = ps[i].rows; c = ps[i].cols; });
    Call c = make_call(opt.ns, ws);
    c.mu = opt.momentum;
    c.keep = (float)(1.0 - (double)opt.lr * opt.weight_decay);
    TraceScope trace("muon_step", nullptr, count, st);
    return run_list<float, 3, true>(p, c, count, opt.ns.steps, st, [&](int i, int& r, int& cols, Jobs& j, int k) {
        r = ps[i].rows; cols = ps[i].cols;
        j.g[k] = ps[i].dw;
        j.momentum[k] = ps[i].momentum;
        j.o[k] = ps[i].w;
        j.scale[k] = (float)((double)opt.lr * sqrt(std::max(1.0, (double)r / std::max(cols, 1))));
    });
}

}  // namespace dr
