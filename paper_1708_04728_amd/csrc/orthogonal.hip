// Orthogonalised matrices by Newton-Schulz products, and the descent step on them (dr_orthogonalise, dr_muon_step).
//
//   X = U / (|U|_F + eps), on the transpose where U has more rows than columns: X has m rows and n >= m columns.
//   `steps` times:  A = X X^T,   Q = a I + b A + c A A,   X = Q X
//
// The polynomial moves every singular value of X towards one and leaves the singular vectors, so that X ends near U V^T of U = U S V^T.  It multiplies
// small singular values by a = 3.4 in every step, and with them what roundings of X leave there: 64 to 512 rows of a filter's gradient end 1e-2 off with X, A and Q
// in bf16, and 1e-6 to 1e-5 in fp32.  So matrices are held as two fp16 pieces whose sum is the value to 2^-23 (11 bits each, the lower one with a sign of its own), at
// scales that keep them in fp16's range, and multiplied on the matrix cores: three products of pieces, with sums in fp32, for each product; the fourth, of the lower
// pieces, is 2^-24 of it.  They end where fp32 ends (4096 x 4096: 3.5e-6 off, in fp32 4.3e-6) in 0.6 of the time of three bf16 pieces, whose six products hold all of fp32's bits
// and all of its range: polynomials whose values could pass fp16's take those (f32_pieces.h), and so do callers who ask for all bits.  Results in bf16 go the same way: 16 bits would do, and two fp16 pieces cost no more.
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
#include <utility>

#include "dr_internal.h"
#include "f32_pieces.h"
#include "orthogonal_plan.h"

namespace dr {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int BLOCK = NS_BLOCK;
constexpr int PITCH = 36;                    // floats of a row of 32 in LDS

// Powers of two that operands are held multiplied by: fp16 has 11 bits from 2^-14 on, so that two pieces of X's have 22 bits from 2^-17 on, and A's and Q's from 2^-15 on.
// (bf16 reaches as far as fp32.)  A sum of products becomes the operand A, Q or X, or the result, multiplied by what is below.
template <int P> constexpr float X_SCALE = P == 2 ? NS_X_SCALE : 1.f;
template <int P> constexpr float A_SCALE = P == 2 ? NS_A_SCALE : 1.f;
template <int P> constexpr float FROM_GRAM = A_SCALE<P> / (X_SCALE<P> * X_SCALE<P>);
template <int P> constexpr float FROM_APPLY = 1.f / A_SCALE<P>;
template <int P> constexpr float TO_RESULT = 1.f / X_SCALE<P>;

// The matrices of a launch; arrays by what is looked up together.  A list is worked on JOBS at a time.  (N: room for as many.  A launch reads its arguments from memory, one after
// the other where an index is among them: a single matrix has kernels whose arguments are its own.)
constexpr int JOBS = NS_JOBS;
template <int N>
struct Jobs {
    int first[N];                         // first workgroup of the launch's k-th matrix; INT_MAX behind the last
    int which[N];                         // the launch's k-th matrix
    unsigned operands[N];                 // its operands' place in the workspace, in KiB
    int mb[N], nb[N];                  // blocks of 32 of the short and of the long side
    int rows[N], cols[N];
    int squares[N];                       // its first partial sum of squares
    const void* g[N];
    float* momentum[N];                   // (descent step only)
    void* o[N];                           // the result, or the weights
    float scale[N];                       // descent step: lr sqrt(max(1, rows / cols))
};

struct Call {
    double* squares;
    int* shifts;                             // of the matrices (pieces of fp16): X is held multiplied by 2^held_at(shift, growth, spare, step)
    int growth;
    float spare;
    float* partial;                          // sums of workgroups that share a tile
    unsigned char* ws;
    float a, b, c, eps;                      // a times, c by the scale of A and Q: Q's scale times (a I + b A + c A A) of A's sums
    float mu, keep;                          // descent step: momentum; 1 - lr decay
};

// A matrix of a launch as its kernels see it
struct Mat {
    int k, first, mb, nb, rows, cols;        // first: its first workgroup
    bool tall;                               // rows > cols: X is the transpose
};
template <int N>
__device__ __forceinline__ Mat find_matrix(const Jobs<N>& j, int id)
{
    if constexpr (N == 1) return Mat{0, 0, j.mb[0], j.nb[0], j.rows[0], j.cols[0], j.rows[0] > j.cols[0]};
    int k = 0;
#pragma unroll
    for (int i = 1; i < N; ++i) k += j.first[i] <= id ? 1 : 0;
    k = __builtin_amdgcn_readfirstlane(k);
    const int i = j.which[k];
    return Mat{i, j.first[k], j.mb[i], j.nb[i], j.rows[i], j.cols[i], j.rows[i] > j.cols[i]};
}

// What a product of step `step` makes of its sums
template <int P>
struct Scales {
    float gram, b, c, apply;
    int down;                                // the result, times 2^-down
    __device__ __forceinline__ Scales(const Call& call, int shift, int step)
    {
        const int now = P == 2 ? held_at(shift, call.growth, call.spare, step) : 0, next = P == 2 ? held_at(shift, call.growth, call.spare, step + 1) : 0;
        gram = FROM_GRAM<P>;
        b = P == 2 ? ldexpf(call.b, -2 * now) : call.b;
        c = P == 2 ? ldexpf(call.c, -4 * now) : call.c;
        apply = P == 2 ? ldexpf(FROM_APPLY<P>, next - now) : 1.f;
        down = now;
    }
    __device__ __forceinline__ float result_of(float v) const { return P == 2 ? ldexpf(v * (FROM_APPLY<P> * TO_RESULT<P>), -down) : v; }
};
// (0 where |U| + eps is: a matrix of zeros stays zero with eps = 0 too)
__device__ __forceinline__ double one_over(double v) { return v == 0.0 ? 0.0 : 1.0 / v; }
// 2^shift times a norm of `norm` after the division is from 1/2 to 1
__device__ __forceinline__ int shift_of(double norm)
{
    int exponent = 0;
    if (norm > 0.0 && norm < 0.5) frexp(norm, &exponent);
    return -exponent;
}

// Operands of a matrix: X, X^T twice (a product reads one and writes the other), A, Q
template <int P>
struct Operands {
    unsigned char *x, *xt0, *xt1, *a, *q;
    template <int N>
    __device__ __forceinline__ Operands(const Call& c, const Jobs<N>& j, const Mat& m)
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

// The sum over 256 threads, added in the same order in every run
__device__ __forceinline__ double sum256(double v, double* red)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// Momentum (descent step), and the sums of the squares of U's elements, in double: a square of 1e20 or 1e-30 is no fp32 number.  HBM bounds it: the step's 7.0 million
// parameters of GoogLeNet 15.6 us, 5.4 TB/s; small ones a launch of 3 to 6 us.  (2048 elements a workgroup for 4096: 0.5 to 1 % of a single matrix' time less, 0.7 % of that list's more.)
template <typename T, bool MUON, int N>
__global__ __launch_bounds__(256) void squares_kernel(const Call c, const Jobs<N> j)
{
    __shared__ double red[4];
    const Mat m = find_matrix(j, blockIdx.x);
    const T* const g = (const T*)j.g[m.k];
    float* const mom = j.momentum[m.k];
    const int me = (int)blockIdx.x - m.first;
    const size_t total = (size_t)m.rows * m.cols, step = (size_t)squares_of(m.rows, m.cols) * 256;
    double s = 0.0;
    for (size_t i = (size_t)me * 256 + threadIdx.x; i < total; i += step * 8) {
        float u[8], v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const size_t n = i + e * step < total ? i + e * step : total - 1;      // (a load under a condition waits for the one before it)
            u[e] = Store<T>::ld(g + n);
            if constexpr (MUON) v[e] = mom[n];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (i + e * step >= total) break;
            if constexpr (MUON) {
                v[e] = c.mu * v[e] + u[e];
                mom[i + e * step] = v[e];
                u[e] += c.mu * v[e];
            }
            s += (double)u[e] * (double)u[e];
        }
    }
    s = sum256(s, red);
    if (threadIdx.x == 0) c.squares[j.squares[m.k] + me] = s;
}

// Eight values as P pieces: two of fp16, three of bf16
template <int P>
__device__ __forceinline__ void cut8(const float (&v)[8], u32x4 (&p)[P])
{
    if constexpr (P == 3) split8(v, p[0], p[1], p[2]);
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 x = {v[2 * i], v[2 * i + 1]};
            const f16x2 high = __builtin_convertvector(x, f16x2);
            const f32x2 back = __builtin_convertvector(high, f32x2), rest = {x[0] - back[0], x[1] - back[1]};
            p[0][i] = __builtin_bit_cast(unsigned, high);
            p[1][i] = __builtin_bit_cast(unsigned, __builtin_convertvector(rest, f16x2));
        }
    }
}

template <int P>
__device__ __forceinline__ float value_of(unsigned pair, int n)      // of the n-th piece of a pair
{
    if constexpr (P == 3) return __uint_as_float(n ? pair & 0xFFFF0000u : pair << 16);
    else return (float)__builtin_bit_cast(f16x2, pair)[n];
}
template <int P>
__device__ __forceinline__ void join8(const u32x4 (&p)[P], float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = 0.f;
#pragma unroll
        for (int e = P - 1; e >= 0; --e) v[i] += value_of<P>(p[e][i >> 1], i & 1);
    }
}

template <int P>
__device__ __forceinline__ f32x16 mfma_of(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (P == 3) return mfma(a, b, c);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
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

// X = U / (|U| + eps) in both orders, cut into pieces: a wave per 32 x 32 block, through LDS, so that both are stored as whole KiB.  HBM bounds it: GoogLeNet's parameters
// 112 MB in 21.6 us, 5.2 TB/s; small ones a launch of 5 us.
template <typename T, int P, bool MUON, int N>
__global__ __launch_bounds__(256) void cut_kernel(const Call c, const Jobs<N> j)
{
    __shared__ __attribute__((aligned(16))) float tiles[4][32 * PITCH];
    __shared__ double red[4];
    const Mat m = find_matrix(j, blockIdx.x);
    const Operands<P> op(c, j, m);
    const T* const g = (const T*)j.g[m.k];
    const float* const mom = j.momentum[m.k];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int b = ((int)blockIdx.x - m.first) * 4 + wave;
    const bool on = b < m.mb * m.nb;
    const int bi = on ? b / m.nb : 0, bj = on ? b - bi * m.nb : 0;
    float* const tile = tiles[wave];
    // lanes along the matrix's own columns; the tile's rows are X's
    const int r0 = (m.tall ? bj : bi) * 32, col = (m.tall ? bi : bj) * 32 + l32;
    float u[16], v[16];
    auto at = [&](int r) __attribute__((always_inline)) { return (size_t)min(r0 + 2 * r + half, m.rows - 1) * m.cols + min(col, m.cols - 1); };
#pragma unroll
    for (int r = 0; r < 16; ++r) u[r] = Store<T>::ld(g + at(r));
    if constexpr (MUON) {
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = mom[at(r)];
    }
    double s = 0.0;
    for (int i = threadIdx.x; i < squares_of(m.rows, m.cols); i += 256) s += c.squares[j.squares[m.k] + i];
    const double norm = sqrt(sum256(s, red)), inv = one_over(norm + (double)c.eps);
    double scale = inv;
    if constexpr (P == 2) {
        const int shift = shift_of(norm * inv);
        scale = ldexp(inv * X_SCALE<P>, shift);
        if ((int)blockIdx.x == m.first && threadIdx.x == 0) c.shifts[m.k] = shift;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        if constexpr (MUON) u[r] += c.mu * v[r];
        const bool in = r0 + 2 * r + half < m.rows && col < m.cols;
        tile[m.tall ? l32 * PITCH + 2 * r + half : (2 * r + half) * PITCH + l32] = in ? (float)((double)u[r] * scale) : 0.f;
    }
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
__device__ __forceinline__ void finish_task(const Call& c, const Mat& m, const Operands<P>& op, const float* tile, int bi, int bj, const Scales<P>& by, int turn, int t)
{
    const int kb = t & 1;
    const bool flip = t >= 2;
    float v[8];
    if (WHAT != APPLY && flip && bi == bj) return;
    if (flip) operand8<true>(tile, kb, v);
    else operand8<false>(tile, kb, v);
    if (P == 2 && WHAT != POLY) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= WHAT == GRAM ? by.gram : by.apply;
    }
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
        for (int e = 0; e < 8; ++e) v[e] = by.b * w[e] + by.c * v[e] + (diagonal + e == 0 ? c.a : 0.f);
        put8<P>(v, op.q + block_at(P, rb, m.mb, cb), kb);
    }
}
// ... of the last product: the result, or the weights; rows r0, r0 + step, ... of the matrix' own 32 x 32 block
template <typename T, int P, bool MUON, int N>
__device__ __forceinline__ void finish_result(const Call& c, const Jobs<N>& j, const Mat& m, const float* tile, int bi, int bj, const Scales<P>& by, int r0, int step)
{
    const int l32 = threadIdx.x & 31, row0 = (m.tall ? bj : bi) * 32, col = (m.tall ? bi : bj) * 32 + l32;
    for (int r8 = r0; r8 < 32; r8 += 8 * step) {         // (eight weights at a time: loads behind stores would wait for each other)
        float old[8];
        if constexpr (MUON) {
#pragma unroll
            for (int e = 0; e < 8; ++e) old[e] = ((const float*)j.o[m.k])[(size_t)min(row0 + r8 + e * step, m.rows - 1) * m.cols + min(col, m.cols - 1)];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int r = r8 + e * step;
            if (r >= 32 || row0 + r >= m.rows || col >= m.cols) continue;
            const float v = by.result_of(tile[m.tall ? l32 * PITCH + r : r * PITCH + l32]);
            const size_t i = (size_t)(row0 + r) * m.cols + col;
            if constexpr (MUON) ((float*)j.o[m.k])[i] = c.keep * old[e] - j.scale[m.k] * v;
            else Store<T>::st((T*)j.o[m.k] + i, v);
        }
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
    large = mfma_of<P>(a[0], b[0], large);
    small = mfma_of<P>(a[0], b[1], small);
    small = mfma_of<P>(a[1], b[0], small);
    if constexpr (P == 3) {
        small = mfma_of<P>(a[1], b[1], small);
        small = mfma_of<P>(a[0], b[2], small);
        small = mfma_of<P>(a[2], b[0], small);
    }
}

// A product of small matrices: W waves share a tile of T x T blocks, every wave a W-th of the contraction.  Operands go straight to registers, some k-blocks of them
// while as many are multiplied: what such a product waits for is its first operands.  splits > 1: as many workgroups share a tile, and leave sums for sum_kernel.
// 4 to 5 us for matrices of one round of short contractions; Q X of 1201 x 500 10, GoogLeNet's list 27 for A and 20 for Q, by what a compute unit reads from L2 (64 bytes a cycle).
// 32 x 32 tiles: four k-blocks a wave ahead.  64 x 64: eight waves with one (four waves with two: five steps of 1201 x 500 127 us for 124, of 1024 x 1024 208 for 201, a step
// of GoogLeNet's filters 487 for 475; 1024 x 4096 444 for 451).
template <typename E, int P, int WHAT, int T, int W, bool MUON, int N>
__global__ __launch_bounds__(W * 64) void product_kernel(const Call c, const Jobs<N> j, int nth, int last, int splits)
{
    constexpr int KEEP = AHEAD[T == 1 ? FINE : DIRECT];
    static_assert(W == WAVES[T == 1 ? FINE : DIRECT], "the plan's waves");
    __shared__ __attribute__((aligned(16))) float sums[W][T * T][32 * PITCH];
    const int unit = splits > 1 ? (int)blockIdx.x / splits : (int)blockIdx.x, part = (int)blockIdx.x - unit * splits;
    const Mat m = find_matrix(j, unit);
    const Operands<P> op(c, j, m);
    const int turn = nth & 1;
    const Scales<P> by(c, P == 2 ? c.shifts[m.k] : 0, nth);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    int bi, bj;
    tile_blocks<WHAT, T>(m, unit - m.first, bi, bj);
    const unsigned char* const left = WHAT == GRAM ? op.x : WHAT == POLY ? op.a : op.q;
    const unsigned char* const right = WHAT == GRAM ? op.x : WHAT == POLY ? op.a : turn ? op.xt1 : op.xt0;
    const int kblocks = 2 * (WHAT == GRAM ? m.nb : m.mb), lrows = m.mb, rrows = WHAT == APPLY ? m.nb : m.mb;
    const int step = W * splits, mine = wave + part * W;      // this wave's k-blocks: mine, mine + step, ...
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
    u32x4 a[2][KEEP][T][P], b[2][KEEP][T][P];
    auto fetch = [&](int kb0, auto set) __attribute__((always_inline)) {
        constexpr int S = decltype(set)::value;
#pragma unroll
        for (int n = 0; n < KEEP; ++n) {
            const size_t at = (size_t)min(kb0 + n * step, kblocks - 1) * P * BLOCK;
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
        for (int n = 0; n < KEEP; ++n) {
            if (kb0 + n * step >= kblocks) break;
#pragma unroll
            for (int i = 0; i < T; ++i)
#pragma unroll
                for (int k = 0; k < T; ++k) multiply<P>(a[S][n][i], b[S][n][k], large[i][k], small[i][k]);
        }
    };
    using std::integral_constant;
    fetch(mine, integral_constant<int, 0>{});
    for (int kb = mine; kb < kblocks; kb += 2 * KEEP * step) {
        if (kb + KEEP * step < kblocks) fetch(kb + KEEP * step, integral_constant<int, 1>{});
        products(kb, integral_constant<int, 0>{});
        if (kb + 2 * KEEP * step < kblocks) fetch(kb + 2 * KEEP * step, integral_constant<int, 0>{});
        products(kb + KEEP * step, integral_constant<int, 1>{});
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
        if (splits > 1) c.partial[(size_t)blockIdx.x * (T * T * 1024) + i] = s;
        else sums[0][blk][at] = s;
    }
    if (splits > 1) return;
    __syncthreads();
    if (WHAT == APPLY && last) {
        for (int blk = 0; blk < T * T; ++blk) {
            const int i = bi + blk / T, k = bj + blk % T;
            if (i < lrows && k < rrows) finish_result<E, P, MUON, N>(c, j, m, sums[0][blk], i, k, by, wave * 2 + half, 2 * W);
        }
        return;
    }
    for (int t = wave; t < T * T * 4; t += W) {
        const int blk = t >> 2, i = bi + blk / T, k = bj + blk % T;
        if (i < lrows && k < rrows && (WHAT == APPLY || i >= k)) finish_task<P, WHAT>(c, m, op, sums[0][blk], i, k, by, turn, t & 3);
    }
}

__device__ __forceinline__ void lds_barrier()        // orders LDS traffic only
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ void wave_lds()           // orders a wave's LDS traffic between its lanes
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// Q and Q X in one launch, for matrices of few rows: a workgroup makes one block of X, and for it the blocks of Q of its rows, a wave each, which stay in LDS.  A's rows that
// all of these share come through LDS (each wave loading them for itself, 192 x 576 takes 92 us for 87 with three pieces, 71 for 69 with two: a compute unit reads 64 bytes a cycle from beyond it), the other
// factor straight to registers, KEEP k-blocks of it while as many are multiplied.  Waits in a row bound it: loads, the products of a wave, a barrier, products, a barrier.
template <typename E, int P, bool MUON, int N>
__global__ __launch_bounds__(512) void poly_apply_kernel(const Call c, const Jobs<N> j, int nth, int last)
{
    constexpr int W = 8, KEEP = 4;
    static_assert(NS_JOINED_ROWS <= W, "a wave for each block of Q");
    __shared__ __attribute__((aligned(16))) float sums[W][32 * PITCH];
    __shared__ __attribute__((aligned(16))) unsigned char q[2 * NS_JOINED_ROWS * P * BLOCK], arows[2 * NS_JOINED_ROWS * P * BLOCK];
    const Mat m = find_matrix(j, blockIdx.x);
    const Operands<P> op(c, j, m);
    const int turn = nth & 1;
    const Scales<P> by(c, P == 2 ? c.shifts[m.k] : 0, nth);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5, kblocks = 2 * m.mb;
    int bi, bj;
    tile_blocks<APPLY, 1>(m, (int)blockIdx.x - m.first, bi, bj);
    const unsigned char* const rows = op.a + (size_t)bi * kblocks * P * BLOCK + lane * 16;
    const unsigned char* const others = op.a + (size_t)min(wave, m.mb - 1) * kblocks * P * BLOCK + lane * 16;
    const unsigned char* const right = (turn ? op.xt1 : op.xt0) + (size_t)bj * kblocks * P * BLOCK + lane * 16;
    auto load = [](const unsigned char* from, int kb, u32x4 (&to)[P]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < P; ++e) to[e] = *reinterpret_cast<const u32x4*>(from + (kb * P + e) * BLOCK);
    };
    f32x16 large, small;
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int v = 0; v < 16; ++v) large[v] = small[v] = 0.f;
    };
    auto leave = [&]() __attribute__((always_inline)) {      // register v holds row 8 (v / 4) + 4 half + v % 4 of column lane % 32
#pragma unroll
        for (int v = 0; v < 16; ++v) sums[wave][(8 * (v >> 2) + 4 * half + (v & 3)) * PITCH + l32] = large[v] + small[v];
    };
    u32x4 mine[2][P], b[2][KEEP][P], x[2][P];      // k-blocks wave and wave + 8 of A's rows; A's rows that give this wave's block of Q; k-blocks wave and wave + 8 of X
    auto fetch = [&](int kb0, auto set) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < KEEP; ++n) load(others, min(kb0 + n, kblocks - 1), b[decltype(set)::value][n]);
    };
    using std::integral_constant;
#pragma unroll
    for (int n = 0; n < 2; ++n) load(rows, min(wave + n * W, kblocks - 1), mine[n]);
    fetch(0, integral_constant<int, 0>{});
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < P; ++e)
            if (wave + n * W < kblocks) *reinterpret_cast<u32x4*>(arows + ((wave + n * W) * P + e) * BLOCK + lane * 16) = mine[n][e];
    lds_barrier();
    if (wave < m.mb) {
        clear();
        auto products = [&](int kb0, auto set) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < KEEP; ++n) {
                if (kb0 + n >= kblocks) break;
                u32x4 a[P];
                load(arows + lane * 16, kb0 + n, a);
                multiply<P>(a, b[decltype(set)::value][n], large, small);
            }
        };
        for (int kb = 0; kb < kblocks; kb += 2 * KEEP) {
            if (kb + KEEP < kblocks) fetch(kb + KEEP, integral_constant<int, 1>{});
            products(kb, integral_constant<int, 0>{});
            if (kb + 2 * KEEP < kblocks) fetch(kb + 2 * KEEP, integral_constant<int, 0>{});
            products(kb + KEEP, integral_constant<int, 1>{});
        }
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) load(right, min(wave + n * W, kblocks - 1), x[n]);
    if (wave < m.mb) {
        leave();
        wave_lds();
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            float v[8], w[8];
            const int diagonal = wave * 32 + n * 16 + half * 8 - bi * 32 - l32;
            u32x4 own[P];
            load(arows + lane * 16, 2 * wave + n, own);
            operand8<false>(sums[wave], n, v);
            join8<P>(own, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = by.b * w[e] + by.c * v[e] + (diagonal + e == 0 ? c.a : 0.f);
            put8<P>(v, q + 2 * wave * P * BLOCK, n);
        }
    }
    __syncthreads();
    clear();
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int kb = wave + n * W;
        if (kb >= kblocks) break;
        u32x4 a[P];
#pragma unroll
        for (int e = 0; e < P; ++e) a[e] = *reinterpret_cast<const u32x4*>(q + (kb * P + e) * BLOCK + lane * 16);
        multiply<P>(a, x[n], large, small);
    }
    leave();
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int i = n * 512 + threadIdx.x, at = (i >> 5) * PITCH + (i & 31);
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) s += sums[w][at];
        sums[0][at] = s;
    }
    __syncthreads();
    if (last) finish_result<E, P, MUON, N>(c, j, m, sums[0], bi, bj, by, wave * 2 + half, 2 * W);
    else if (wave < 4) finish_task<P, APPLY>(c, m, op, sums[0], bi, bj, by, turn, wave);
}

// Adds the sums that the workgroups of a tile of A have left, in their order: a launch more, 4 us, for contractions that would keep few compute units busy for longer
template <int P, int T, int N>
__global__ __launch_bounds__(256) void sum_kernel(const Call c, const Jobs<N> j, int nth, int splits)
{
    __shared__ __attribute__((aligned(16))) float tile[32 * PITCH];
    const int unit = (int)blockIdx.x / (T * T), blk = (int)blockIdx.x - unit * (T * T);
    const Mat m = find_matrix(j, unit);
    const Operands<P> op(c, j, m);
    const Scales<P> by(c, P == 2 ? c.shifts[m.k] : 0, nth);
    int bi, bj;
    tile_blocks<GRAM, T>(m, unit - m.first, bi, bj);
    bi += blk / T;
    bj += blk % T;
    if (bi >= m.mb || bj >= m.mb || bi < bj) return;
    const float* const from = c.partial + ((size_t)unit * splits * (T * T) + blk) * 1024;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < splits; ++k)
#pragma unroll
        for (int n = 0; n < 4; ++n) s[n] += from[(size_t)k * (T * T * 1024) + n * 256 + threadIdx.x];
#pragma unroll
    for (int n = 0; n < 4; ++n) tile[(n * 8 + (threadIdx.x >> 5)) * PITCH + (threadIdx.x & 31)] = s[n];
    __syncthreads();
    finish_task<P, GRAM>(c, m, op, tile, bi, bj, by, nth & 1, threadIdx.x >> 6);
}

// f(0), ..., f(N - 1), as constants
template <class F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void each(F f) { each_of(f, std::make_integer_sequence<int, N>{}); }

// A product of larger matrices: WM x WN waves share a tile, TM x TN blocks of 32 x 32 each.  A stage is one k-block (16 k) of the tile's operands in LDS; of three stages
// one is multiplied, one is complete, one is written, from registers that were loaded DEPTH iterations before, with a barrier an iteration.  A wave keeps one k-block of
// its operands in registers.  The products of pieces come in an order in which every piece of the next k-block is read between the last product that needs the present one
// and the first that needs it; reads, writes and loads are issued one by one between matrix instructions, which cover them: one wave per SIMD keeps its unit busy.
// APART: sums of products with lower pieces on their own, where registers allow it; elsewhere a sum is rounded three (six) times a k-block instead of once, by 2^-24 of it each time.
// The matrix cores' power seems to bound it: 4096 x 4096 on two pieces takes 193 us for A and 206 for Q (1.1 PFLOP/s of products in 192 x 192 tiles) and 327 for Q X (1.26 in
// 256 x 256), three pieces 310, 325 and 540; of a matrix of zeros five steps take 2.41 ms for 3.73, on three pieces 4.35 for 6.22.
template <int P, int BM, int BN> constexpr int tile_lds() { return 3 * (BM + BN) * P * BLOCK; }
template <typename E, int P, int WHAT, int WM, int WN, int TM, int TN, int DEPTH, bool APART, bool MUON, int N>
__global__ __launch_bounds__(WM * WN * 64) void tile_kernel(const Call c, const Jobs<N> j, int nth, int last)
{
    constexpr int W = WM * WN, BM = WM * TM, BN = WN * TN, STAGE = (BM + BN) * P * BLOCK, LOADS = (BM + BN) * P / W;
    static_assert((BM + BN) * P % W == 0 && BM == BN && (DEPTH == 1 || DEPTH == 2) && tile_lds<P, BM, BN>() >= W * 32 * PITCH * 4, "a tile's operands");
    __shared__ __attribute__((aligned(16))) unsigned char lds[tile_lds<P, BM, BN>()];
    // workgroup b runs on die b & 7: of one matrix a die takes a contiguous range of tiles, which share operands (of a list, whose long contractions come first, that
    // would give one die the most work)
    const int die = blockIdx.x & 7, share = (int)gridDim.x >> 3, odd = gridDim.x & 7;
    const int id = N > 1 ? (int)blockIdx.x : die * share + min(die, odd) + (int)(blockIdx.x >> 3);
    const Mat m = find_matrix(j, id);
    const Operands<P> op(c, j, m);
    const int turn = nth & 1;
    const Scales<P> by(c, P == 2 ? c.shifts[m.k] : 0, nth);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int wm = wave / WN, wn = wave % WN;
    int bi, bj;
    tile_blocks<WHAT, BM>(m, id - m.first, bi, bj);
    const unsigned char* const left = WHAT == GRAM ? op.x : WHAT == POLY ? op.a : op.q;
    const unsigned char* const right = WHAT == GRAM ? op.x : WHAT == POLY ? op.a : turn ? op.xt1 : op.xt0;
    const int kblocks = 2 * (WHAT == GRAM ? m.nb : m.mb), lrows = m.mb, rrows = WHAT == APPLY ? m.nb : m.mb;

    // load n of a wave: KiB wave + n W of the stage: piece % P of row of blocks / P
    const unsigned char* from[LOADS];
#pragma unroll
    for (int n = 0; n < LOADS; ++n) {
        const int q = wave + n * W, row = q / P, piece = q % P;
        from[n] = (row < BM ? left + (size_t)min(bi + row, lrows - 1) * kblocks * P * BLOCK : right + (size_t)min(bj + row - BM, rrows - 1) * kblocks * P * BLOCK) + piece * BLOCK;
    }
    u32x4 in[DEPTH][LOADS];
    auto fetch = [&](auto set, int n) __attribute__((always_inline)) {
        in[decltype(set)::value][n] = *reinterpret_cast<const u32x4*>(from[n] + lane * 16);
        from[n] += P * BLOCK;
    };
    auto put = [&](auto set, int stage, int n) __attribute__((always_inline)) {
        *reinterpret_cast<u32x4*>(lds + stage + (wave + n * W) * BLOCK + lane * 16) = in[decltype(set)::value][n];
    };
    u32x4 a[TM][P], b[TN][P];
    const unsigned char* const mine_a = lds + wm * TM * P * BLOCK + lane * 16;
    const unsigned char* const mine_b = lds + (BM + wn * TN) * P * BLOCK + lane * 16;
    auto read_a = [&](int stage, int i, int e) __attribute__((always_inline)) { a[i][e] = *reinterpret_cast<const u32x4*>(mine_a + stage + (i * P + e) * BLOCK); };
    auto read_b = [&](int stage, int i, int e) __attribute__((always_inline)) { b[i][e] = *reinterpret_cast<const u32x4*>(mine_b + stage + (i * P + e) * BLOCK); };
    f32x16 acc[TM][TN], small[APART ? TM : 1][APART ? TN : 1];      // APART: the small products in sums of their own
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int k = 0; k < TN; ++k)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                acc[i][k][v] = 0.f;
                if constexpr (APART) small[i][k][v] = 0.f;
            }

    using std::integral_constant;
    typedef integral_constant<int, 0> First;
    typedef integral_constant<int, DEPTH - 1> Second;
#pragma unroll
    for (int k = 0; k < 2; ++k) {            // (k-blocks come in pairs)
#pragma unroll
        for (int n = 0; n < LOADS; ++n) fetch(First{}, n);
#pragma unroll
        for (int n = 0; n < LOADS; ++n) put(First{}, k * STAGE, n);
    }
    if (kblocks > 2) {
#pragma unroll
        for (int n = 0; n < LOADS; ++n) fetch(First{}, n);
        if constexpr (DEPTH == 2) {
#pragma unroll
            for (int n = 0; n < LOADS; ++n) fetch(Second{}, n);
        }
    }
    lds_barrier();
    // (pieces of the first k-block that are not read where it is multiplied)
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < P - 1; ++e) read_a(0, i, e);
#pragma unroll
    for (int k = 0; k < TN; ++k)
#pragma unroll
        for (int e = 1; e < P; ++e) read_b(0, k, e);

    int here = 0, next = STAGE, write = 2 * STAGE;       // the stages of k-blocks kb, kb + 1 and kb + 2
    auto iteration = [&](auto set, bool putting, bool fetching) __attribute__((always_inline)) {
        constexpr int G = TM * TN, PAIRS = P == 3 ? 6 : 3;
        // products of pieces: first the one that needs neither b's first piece nor a's last, which are read meanwhile
        constexpr int X[6] = {0, 0, 0, 1, 1, 2}, Y[6] = {2, 1, 0, 1, 0, 0};
        constexpr int X2[3] = {0, 0, 1}, Y2[3] = {1, 0, 0};
        each<PAIRS * G>([&](auto slot) __attribute__((always_inline)) {
            constexpr int t = decltype(slot)::value, g = t / G, i = t % G / TN, k = t % TN, x = P == 3 ? X[g] : X2[g % 3], y = P == 3 ? Y[g] : Y2[g % 3];
            if constexpr (APART && x + y != 0) small[i][k] = mfma_of<P>(a[i][x], b[k][y], small[i][k]);
            else acc[i][k] = mfma_of<P>(a[i][x], b[k][y], acc[i][k]);
            __builtin_amdgcn_sched_barrier(0);
            // this k-block's pieces that come last
            if constexpr (t < TN) read_b(here, t, 0);
            else if constexpr (t < TN + TM) read_a(here, t - TN, P - 1);
            // the next one's
            constexpr int u = t - g * G;
            if constexpr (P == 3 && g == 1 && u < TN) read_b(next, u, 2);
            if constexpr (P == 3 && g == 3 && u < TM) read_a(next, u, 0);
            if constexpr (P == 3 && g == 4 && u < TN) read_b(next, u, 1);
            if constexpr (P == 3 && g == 5 && u < TM) read_a(next, u, 1);
            if constexpr (P == 2 && g == 1 && u < TN) read_b(next, u, 1);
            if constexpr (P == 2 && g == 2 && u < TM) read_a(next, u, 0);
            // the one behind, and the loads of the one DEPTH behind that
            constexpr int FROM = G / 2, SPAN = (P == 3 ? 3 : 2) * G - FROM;
#pragma unroll
            for (int n = 0; n < LOADS; ++n) {
                if (putting && t == FROM + n * SPAN / LOADS) put(set, write, n);
                if (fetching && t == FROM + n * SPAN / LOADS + 1) fetch(set, n);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        lds_barrier();
        const int done = here;
        here = next;
        next = write;
        write = done;
    };
    int kb = 0;
    for (; kb + 2 + DEPTH < kblocks; kb += DEPTH) {
        iteration(First{}, true, true);
        if constexpr (DEPTH == 2) iteration(Second{}, true, true);
    }
    // the last k-blocks: nothing more to load, then nothing more to write
    for (; kb + 2 < kblocks; kb += DEPTH) {
        iteration(First{}, true, false);
        if constexpr (DEPTH == 2) iteration(Second{}, true, false);
    }
    iteration(First{}, false, false);
    iteration(First{}, false, false);
    // block by block through LDS, each wave in its own part
    float* const tile = reinterpret_cast<float*>(lds) + wave * 32 * PITCH;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int k = 0; k < TN; ++k) {
            const int ri = bi + wm * TM + i, rk = bj + wn * TN + k;
            if (ri >= lrows || rk >= rrows || (WHAT != APPLY && ri < rk)) continue;
            // register v holds row 8 (v / 4) + 4 half + v % 4 of column lane % 32
#pragma unroll
            for (int v = 0; v < 16; ++v) tile[(8 * (v >> 2) + 4 * half + (v & 3)) * PITCH + l32] = APART ? acc[i][k][v] + small[APART ? i : 0][APART ? k : 0][v] : acc[i][k][v];
            wave_lds();
            if (WHAT == APPLY && last) finish_result<E, P, MUON, N>(c, j, m, tile, ri, rk, by, half, 2);
            else {
#pragma unroll 1
                for (int t = 0; t < 4; ++t) finish_task<P, WHAT>(c, m, op, tile, ri, rk, by, turn, t);
            }
            wave_lds();
        }
}

// ---- matrices small enough for one workgroup's LDS: the whole iteration there, X in fp32, cut into pieces where it is multiplied, A and Q in pieces, as operands.
// 64 rows and 352 columns, or 32 and 896: eight waves.  Nothing but the matrix is read or written, and a step is four barriers instead of two or three launches.  Vector
// instructions bound it, most of them the cutting: with A and Q in fp32 too, cut by every wave that multiplies them, a step on 64 x 64 took 5.8 us, 1650 of them on its path.
// All of five steps, fp32 or bf16: 16 x 16 15 us, 64 x 64 25, 64 x 147 34 (5.2 a step), 64 x 352 55, 32 x 800 41; three pieces 17, 29, 40, 64 and 47.  (Four waves for A's block below the
// diagonal, where both operands are cut, and two for each on it cost registers and gain nothing: with three pieces 64 x 147 42 us for 41, 64 x 352 65 for 66.)
constexpr int WHOLE_BYTES = 163840 - 256;

template <typename E, int P, bool MUON, int N>
__global__ __launch_bounds__(512) void whole_kernel(const Call c, const Jobs<N> j, int steps)
{
    __shared__ __attribute__((aligned(16))) unsigned char lds[WHOLE_BYTES];
    __shared__ double red[8];
    const int k = blockIdx.x, mb = j.mb[k], nb = j.nb[k], rows = j.rows[k], cols = j.cols[k];
    const bool tall = rows > cols;
    // X; A as operand, 2 mb k-blocks for each 32 rows; Q likewise; sums of A's blocks on and below the diagonal that single waves have made, in the place of Q and behind it
    const int XP = nb * 32 + 4;
    float* const X = (float*)lds;
    unsigned char* const A = lds + mb * 32 * XP * 4;
    unsigned char* const Q = A + 2 * mb * mb * P * BLOCK;
    float* const sums = (float*)Q;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;

    // elements i = tid, tid + 512, ... of the matrix, AT_ONCE at a time: f(the first's number, their places in X)
    constexpr int AT_ONCE = 16;
    const int total = rows * cols, step_r = 512 / cols, step_c = 512 - step_r * cols;
    const int row_at = tall ? 1 : XP, col_at = tall ? XP : 1, step_at = step_r * row_at + step_c * col_at, wrap_at = row_at - cols * col_at;
    auto elements = [&](auto f) __attribute__((always_inline)) {
        int col = tid % cols, place = tid / cols * row_at + col * col_at;
        for (int i = tid; i < total; i += AT_ONCE * 512) {
            int at[AT_ONCE];
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) {
                at[e] = place;
                col += step_c;
                place += step_at;
                if (col >= cols) { col -= cols; place += wrap_at; }
            }
            f(i, at);
        }
    };
    const int pieces = mb * 8 * XP;          // of 16 bytes of X
    for (int i = tid; i < pieces; i += 512) reinterpret_cast<f32x4*>(X)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    __syncthreads();
    double s = 0.0;
    elements([&](int i, const int (&at)[AT_ONCE]) {
        float u[AT_ONCE], v[AT_ONCE];
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) {
            const int n = min(i + e * 512, total - 1);
            u[e] = Store<E>::ld((const E*)j.g[k] + n);
            if constexpr (MUON) v[e] = j.momentum[k][n];
        }
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) {
            if (i + e * 512 >= total) break;
            if constexpr (MUON) {
                v[e] = c.mu * v[e] + u[e];
                j.momentum[k][i + e * 512] = v[e];
                u[e] += c.mu * v[e];
            }
            X[at[e]] = u[e];
            s += (double)u[e] * (double)u[e];
        }
    });
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    if (lane == 0) red[wave] = s;
    __syncthreads();
    const double norm = sqrt(((red[0] + red[1]) + (red[2] + red[3])) + ((red[4] + red[5]) + (red[6] + red[7]))), inv = one_over(norm + (double)c.eps);
    const int shift = P == 2 ? shift_of(norm * inv) : 0;
    // (inv as factor 2^exponent: inv itself may be no fp32 number, and a product in double is four times the work)
    int exponent;
    const float factor = (float)frexp(inv * X_SCALE<P>, &exponent);
    exponent += shift;
    for (int i = tid; i < pieces; i += 4 * 512) {          // (four at once: a pass that waits for every read takes 5 us of 32 x 800)
        f32x4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = reinterpret_cast<const f32x4*>(X)[min(i + e * 512, pieces - 1)];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (i + e * 512 >= pieces) break;
#pragma unroll
            for (int n = 0; n < 4; ++n) v[e][n] = ldexpf(v[e][n], exponent) * factor;
            reinterpret_cast<f32x4*>(X)[i + e * 512] = v[e];
        }
    }
    __syncthreads();

    // eight values along a row of X, cut; down a column
    auto along = [&](int row, int k0, u32x4 (&p)[P]) __attribute__((always_inline)) {
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 t = *reinterpret_cast<const f32x4*>(X + row * XP + k0 + half * 8 + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * h + e] = t[e];
        }
        cut8<P>(v, p);
    };
    auto down = [&](int col, int k0, u32x4 (&p)[P]) __attribute__((always_inline)) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = X[(k0 + half * 8 + e) * XP + col];
        cut8<P>(v, p);
    };
    auto read = [&](const unsigned char* M, int rb, int kb, u32x4 (&p)[P]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < P; ++e) p[e] = *reinterpret_cast<const u32x4*>(M + ((rb * 2 * mb + kb) * P + e) * BLOCK + lane * 16);
    };
    auto zero = [](f32x16& a, f32x16& b) __attribute__((always_inline)) {
#pragma unroll
        for (int v = 0; v < 16; ++v) a[v] = b[v] = 0.f;
    };
    // register v holds row 8 (v / 4) + 4 half + v % 4 of column lane % 32
    auto row_of = [&](int v) __attribute__((always_inline)) { return 8 * (v >> 2) + 4 * half + (v & 3); };
    auto iterate = [&](auto blocks) __attribute__((always_inline)) {
        constexpr int MB = decltype(blocks)::value, SPLITS = MB == 1 ? 8 : 2;      // waves that share a block of A
        f32x16 large[2], small[2];
        auto multiply2 = [&](int which, const u32x4 (&a)[P], const u32x4 (&b)[P]) __attribute__((always_inline)) { multiply<P>(a, b, large[which], small[which]); };
        auto sum = [&](int v) __attribute__((always_inline)) { return (large[0][v] + large[1][v]) + (small[0][v] + small[1][v]); };
        for (int step = 0; step < steps; ++step) {
            const Scales<P> by(c, shift, step);
            // A = X X^T
            if (MB == 1 || wave < 6) {
                const int blk = MB == 1 ? 0 : wave >> 1, split = MB == 1 ? wave : wave & 1, bi = blk ? 1 : 0, bj = blk == 2 ? 1 : 0;
                zero(large[0], small[0]);
                zero(large[1], small[1]);
                // (two k-blocks at a time, in sums of their own: what a product waits for is the one before it)
                for (int kb = split; kb < 2 * nb; kb += 2 * SPLITS) {
                    u32x4 a[2][P], b[2][P];
                    const bool two = kb + SPLITS < 2 * nb;
#pragma unroll
                    for (int h = 0; h < 2; ++h) along(bi * 32 + l32, (h && two ? kb + SPLITS : kb) * 16, a[h]);
                    if (bi == bj) {
                        multiply2(0, a[0], a[0]);
                        if (two) multiply2(1, a[1], a[1]);
                    } else {
#pragma unroll
                        for (int h = 0; h < 2; ++h) along(bj * 32 + l32, (h && two ? kb + SPLITS : kb) * 16, b[h]);
                        multiply2(0, a[0], b[0]);
                        if (two) multiply2(1, a[1], b[1]);
                    }
                }
                float* const to = sums + (blk * SPLITS + split) * 32 * PITCH;
#pragma unroll
                for (int v = 0; v < 16; ++v) to[row_of(v) * PITCH + l32] = sum(v);
            }
            __syncthreads();
            // ... as operand: a wave per k-block of 32 rows
            if (wave < 2 * MB * MB) {
                const int rb = wave / (2 * MB), kb = wave % (2 * MB), cb = kb >> 1, blk = rb + cb, k0 = (kb & 1) * 16 + half * 8;
                const float* const from = sums + blk * SPLITS * 32 * PITCH;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll
                for (int w = 0; w < SPLITS; ++w) {
                    if (rb < cb) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += from[w * 32 * PITCH + (k0 + e) * PITCH + l32];
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += from[w * 32 * PITCH + l32 * PITCH + k0 + e];
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= by.gram;
                u32x4 p[P];
                cut8<P>(v, p);
#pragma unroll
                for (int e = 0; e < P; ++e) *reinterpret_cast<u32x4*>(A + (wave * P + e) * BLOCK + lane * 16) = p[e];
            }
            __syncthreads();
            // Q = a I + b A + c A A, which is symmetric: element (row, column) is stored as (column, row), four of a lane's one after the other
            if (wave < MB * MB) {
                const int bi = wave / MB, bj = wave % MB;
                zero(large[0], small[0]);
                zero(large[1], small[1]);
#pragma unroll
                for (int kb = 0; kb < 2 * MB; ++kb) {
                    u32x4 a[P], b[P];
                    read(A, bi, kb, a);
                    read(A, bj, kb, b);
                    multiply2(kb & 1, a, b);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {             // rows 16 h .. 16 h + 15 of the block: a k-block
                    float v[8];
                    u32x2 p[2][P];
                    const int block = ((bj * 2 * MB + bi * 2 + h) * P) * BLOCK + l32 * 16 + half * 8;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
#pragma unroll
                        for (int e = 0; e < P; ++e) p[q][e] = *reinterpret_cast<const u32x2*>(A + block + q * 512 + e * BLOCK);
                    }
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int n = (2 * h + q) * 4 + r;
                            float w = 0.f;
#pragma unroll
                            for (int e = P - 1; e >= 0; --e) w += value_of<P>(p[q][e][r >> 1], r & 1);
                            v[q * 4 + r] = by.b * w + by.c * sum(n) + (bi == bj && row_of(n) == l32 ? c.a : 0.f);
                        }
                    u32x4 t[P];
                    cut8<P>(v, t);
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int e = 0; e < P; ++e) *reinterpret_cast<u32x2*>(Q + block + q * 512 + e * BLOCK) = u32x2{t[e][2 * q], t[e][2 * q + 1]};
                }
            }
            __syncthreads();
            // X = Q X: a wave has whole columns, which it replaces
            for (int bj = wave; bj < nb; bj += 8) {
                f32x16 big[MB], little[MB];
#pragma unroll
                for (int i = 0; i < MB; ++i) zero(big[i], little[i]);
#pragma unroll
                for (int kb = 0; kb < 2 * MB; ++kb) {
                    u32x4 b[P];
                    down(bj * 32 + l32, kb * 16, b);
#pragma unroll
                    for (int i = 0; i < MB; ++i) {
                        u32x4 q[P];
                        read(Q, i, kb, q);
                        multiply<P>(q, b, big[i], little[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int v = 0; v < 16; ++v) X[(i * 32 + row_of(v)) * XP + bj * 32 + l32] = (big[i][v] + little[i][v]) * by.apply;
            }
            __syncthreads();
        }
    };
    if (mb == 1) iterate(std::integral_constant<int, 1>{});
    else iterate(std::integral_constant<int, 2>{});
    const int held = held_at(shift, c.growth, c.spare, steps);
    auto result_of = [&](float v) __attribute__((always_inline)) { return P == 2 ? ldexpf(v * TO_RESULT<P>, -held) : v; };
    elements([&](int i, const int (&at)[AT_ONCE]) {
        float w[AT_ONCE];
        if constexpr (MUON) {
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) w[e] = ((const float*)j.o[k])[min(i + e * 512, total - 1)];
        }
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) {
            if (i + e * 512 >= total) break;
            if constexpr (MUON) ((float*)j.o[k])[i + e * 512] = c.keep * w[e] - j.scale[k] * result_of(X[at[e]]);
            else Store<E>::st((E*)j.o[k] + i + e * 512, result_of(X[at[e]]));
        }
    });
}

// ---- a call
template <class Shape>
size_t workspace_bytes(int count, Shape shape)
{
    size_t most = 0;
    Group g;
    g.start();
    for (int i = 0; i < count; ++i) {
        int rows, cols;
        shape(i, rows, cols);
        if (rows && cols) g.add(rows, cols);
        if (g.count == JOBS || (i + 1 == count && g.count)) {
            for (int pieces = 2; pieces <= 3; ++pieces) most = std::max(most, g.bytes(pieces, device_cus()));      // (whatever the polynomial)
            g.start();
        }
    }
    return most;
}

// The order of a launch's matrices: those with the largest length(mb, nb) first, so that what is started last is short
struct Order { int which[JOBS]; };
template <int N, class Length>
Order order_by(const Jobs<N>& j, int count, Length length)
{
    Order o;
    for (int i = 0; i < count; ++i) {
        int at = i;
        for (; at > 0 && length(j.mb[o.which[at - 1]], j.nb[o.which[at - 1]]) < length(j.mb[i], j.nb[i]); --at) o.which[at] = o.which[at - 1];
        o.which[at] = i;
    }
    return o;
}

// the first workgroups of j's matrices, for launches whose matrix has `units(mb, nb, rows, cols)` of them; their number
template <int N, class Units>
unsigned number(Jobs<N>& j, int count, const Order& order, Units units)
{
    unsigned at = 0;
    for (int k = 0; k < N; ++k) {
        j.first[k] = 0x7FFFFFFF;
        if (k >= count) continue;
        const int i = order.which[k];
        j.which[k] = i;
        j.first[k] = (int)at;
        at += units(j.mb[i], j.nb[i], j.rows[i], j.cols[i]);
    }
    return at;
}

template <typename E, int P, bool MUON, int N>
int run_group(const Group& group, Call c, Jobs<N>& j, int steps, void* ws, hipStream_t st)
{
    if (group.whole) {
        hipLaunchKernelGGL((whole_kernel<E, P, MUON, N>), dim3(group.count), dim3(512), 0, st, c, j, steps);
        return check_launch("orthogonalise");
    }
    c.squares = (double*)ws;
    c.shifts = (int*)((unsigned char*)ws + group.squares);
    c.ws = (unsigned char*)ws + group.squares_bytes();
    c.partial = (float*)(c.ws + group.operands_bytes(P));
    size_t operands = 0;
    int squares_at = 0;
    for (int i = 0; i < group.count; ++i) {
        j.operands[i] = (unsigned)(operands / 1024);
        j.squares[i] = squares_at;
        operands += operand_bytes(j.mb[i], j.nb[i], P);
        squares_at += squares_of(j.rows[i], j.cols[i]);
    }
    const Order orders[PRODUCTS] = {order_by(j, group.count, [](int, int nb) { return nb; }), order_by(j, group.count, [](int mb, int) { return mb; }),
                                    order_by(j, group.count, [](int mb, int) { return mb; })};
    const unsigned squares = number(j, group.count, orders[GRAM], [](int, int, int r, int co) { return squares_of(r, co); });
    hipLaunchKernelGGL((squares_kernel<E, MUON, N>), dim3(squares), dim3(256), 0, st, c, j);
    const unsigned cuts = number(j, group.count, orders[GRAM], [](int mb, int nb, int, int) { return (mb * nb + 3) / 4; });
    hipLaunchKernelGGL((cut_kernel<E, P, MUON, N>), dim3(cuts), dim3(256), 0, st, c, j);
    using std::integral_constant;
    auto product = [&](auto what, int nth, int last) {
        constexpr int WHAT = decltype(what)::value;
        constexpr bool END = WHAT == APPLY && MUON;      // (the other products are the same for every result)
        typedef std::conditional_t<WHAT == APPLY, E, float> R;
        const Choice choice = choose(P, WHAT, group.work[WHAT], device_cus());
        const unsigned tiles = number(j, group.count, orders[WHAT], [&](int mb, int nb, int, int) { return tiles_of(WHAT, mb, nb, SIDE[choice.kernel]); });
        auto direct = [&](auto side, auto waves) {
            constexpr int T = decltype(side)::value, W = decltype(waves)::value;
            hipLaunchKernelGGL((product_kernel<R, P, WHAT, T, W, END, N>), dim3(tiles * choice.splits), dim3(W * 64), 0, st, c, j, nth, last, choice.splits);
            if constexpr (WHAT == GRAM) {
                if (choice.splits > 1) hipLaunchKernelGGL((sum_kernel<P, T, N>), dim3(tiles * T * T), dim3(256), 0, st, c, j, nth, choice.splits);
            }
        };
        auto tile = [&](auto side, auto depth, auto apart) {
            constexpr int T = decltype(side)::value;
            hipLaunchKernelGGL((tile_kernel<R, P, WHAT, 2, 2, T / 2, T / 2, decltype(depth)::value, decltype(apart)::value, END, N>), dim3(tiles), dim3(256), 0, st, c, j, nth, last);
        };
        if (choice.kernel == FINE) direct(integral_constant<int, 1>{}, integral_constant<int, 8>{});
        else if (choice.kernel == DIRECT) direct(integral_constant<int, 2>{}, integral_constant<int, 8>{});
        else if (choice.kernel == TILE4) tile(integral_constant<int, 4>{}, integral_constant<int, 2>{}, std::bool_constant<P == 3>{});
        else if (choice.kernel == TILE6) tile(integral_constant<int, 6>{}, integral_constant<int, 2>{}, std::false_type{});
        else tile(integral_constant<int, 8>{}, integral_constant<int, P == 3 ? 1 : 2>{}, std::false_type{});      // (registers: three pieces two deep 658 us for 590)
    };
    for (int s = 0; s < steps; ++s) {
        const int last = s + 1 == steps;
        product(integral_constant<int, GRAM>{}, s, last);
        if (group.joined(device_cus())) {
            const unsigned tiles = number(j, group.count, orders[APPLY], [](int mb, int nb, int, int) { return mb * nb; });
            hipLaunchKernelGGL((poly_apply_kernel<E, P, MUON, N>), dim3(tiles), dim3(512), 0, st, c, j, s, last);
            continue;
        }
        product(integral_constant<int, POLY>{}, s, last);
        product(integral_constant<int, APPLY>{}, s, last);
    }
    return check_launch("orthogonalise");
}

// fill(i, rows, cols, j, k): matrix i's shape, and entry k of j but for its shape and places
template <typename E, int P, bool MUON, int N, class Fill>
int run_jobs(Call c, int count, int steps, void* ws, hipStream_t st, Fill fill)
{
    Jobs<N> j;
    Group g;
    g.start();
    for (int i = 0; i < count; ++i) {
        int rows, cols;
        fill(i, rows, cols, j, g.count);
        if (rows && cols) {
            j.rows[g.count] = rows; j.cols[g.count] = cols;
            j.mb[g.count] = (std::min(rows, cols) + 31) / 32;
            j.nb[g.count] = (std::max(rows, cols) + 31) / 32;
            g.add(rows, cols);
        }
        if (g.count == N || (i + 1 == count && g.count)) {
            if (const int rc = run_group<E, P, MUON>(g, c, j, steps, ws, st)) return rc;
            g.start();
        }
    }
    return DR_OK;
}
template <typename E, bool MUON, class Fill>
int run_list(Call c, int count, const dr_newton_schulz& ns, void* ws, hipStream_t st, Fill fill)
{
    c.b = ns.b; c.eps = ns.eps;
    auto run = [&](auto pieces) {
        constexpr int P = decltype(pieces)::value;
        c.a = ns.a * A_SCALE<P>; c.c = ns.c / A_SCALE<P>;
        return count == 1 ? run_jobs<E, P, MUON, 1>(c, count, ns.steps, ws, st, fill) : run_jobs<E, P, MUON, JOBS>(c, count, ns.steps, ws, st, fill);
    };
    return !ns.all_bits && stays_small(ns.steps, ns.a, ns.b, ns.c, &c.growth, &c.spare) ? run(std::integral_constant<int, 2>{}) : run(std::integral_constant<int, 3>{});
}

}  // namespace

size_t orthogonalise_workspace_bytes(int count, const dr_matrix* ms)
{
    return workspace_bytes(count, [&](int i, int& r, int& c) { r = ms[i].rows; c = ms[i].cols; });
}

int launch_orthogonalise(int count, const dr_matrix* ms, int dtype, const void* const* g, void* const* o, const dr_newton_schulz& ns, void* ws, hipStream_t st)
{
    TraceScope trace("orthogonalise", nullptr, count, st);
    auto fill = [&](int i, int& r, int& cols, auto& j, int k) {
        r = ms[i].rows; cols = ms[i].cols;
        j.g[k] = g[i];
        j.momentum[k] = nullptr;
        j.o[k] = o[i];
        j.scale[k] = 0.f;
    };
    return dtype == DR_F32 ? run_list<float, false>(Call{}, count, ns, ws, st, fill) : run_list<uint16_t, false>(Call{}, count, ns, ws, st, fill);
}

size_t muon_step_workspace_bytes(int count, const dr_muon_param* ps)
{
    return workspace_bytes(count, [&](int i, int& r, int& c) { r = ps[i].rows; c = ps[i].cols; });
}

int launch_muon_step(int count, const dr_muon_param* ps, const dr_muon& opt, void* ws, hipStream_t st)
{
    Call c{};
    c.mu = opt.momentum;
    c.keep = (float)(1.0 - (double)opt.lr * opt.weight_decay);
    TraceScope trace("muon_step", nullptr, count, st);
    return run_list<float, true>(c, count, opt.ns, ws, st, [&](int i, int& r, int& cols, auto& j, int k) {
        r = ps[i].rows; cols = ps[i].cols;
        j.g[k] = ps[i].dw;
        j.momentum[k] = ps[i].momentum;
        j.o[k] = ps[i].w;
        j.scale[k] = (float)((double)opt.lr * sqrt(std::max(1.0, (double)r / std::max(cols, 1))));
    });
}

}  // namespace dr
