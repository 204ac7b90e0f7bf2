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
// A call works on a list of matrices of any sizes: each of its launches runs one product of all of them.
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
constexpr int SQUARES = 256;                 // most workgroups (and partial sums of squares) of a matrix
enum { GRAM = 0, POLY = 1, APPLY = 2, PRODUCTS = 3 };

// One matrix of a call.  In the workspace, for the kernels to read.
struct Mat {
    const void* g;                           // rows x cols
    float* momentum;                         // (descent step only)
    float* w;
    void* o;                                 // (orthogonalise only)
    long long x, xt[2], a, q;                // offsets of the operands in the workspace
    int rows, cols, mb, nb;                  // mb, nb: blocks of 32 of the short and of the long side
    int tall;                                // rows > cols: X is the transpose
    float scale;                             // descent step: lr sqrt(max(1, rows / cols))
    int squares_first, squares;              // partial sums of squares: first, how many
    int cut_first;                           // first group of four 32 x 32 blocks of the cutting kernel
    int unit_first[PRODUCTS], splits[PRODUCTS];     // first workgroup; workgroups that share a tile's contraction
};

constexpr int TABLE_CHUNK = 16;
struct Table { Mat m[TABLE_CHUNK]; };

struct Call {
    const Mat* mats;
    double* squares;
    unsigned char* ws;
    float* partial;
    int count;
    float a, b, c, eps;
    float mu, keep;                          // descent step: momentum; 1 - lr decay
};

__global__ __launch_bounds__(64) void table_kernel(const Table t, Mat* mats, int first, int count)
{
    const int i = threadIdx.x;
    if (i < count) mats[first + i] = t.m[i];
}

// The matrix that workgroup `id` works on: the last whose first workgroup is not behind it.  The table in steps of 64, a matrix per lane.
template <class F>
__device__ __forceinline__ int find_matrix(int count, int id, F first)
{
    int at = -1;
    for (int i = 0; i < count; i += 64) {
        const int k = i + (threadIdx.x & 63);
        const unsigned long long in = __ballot(k < count && first(k) <= id);
        at += __popcll(in);
        if (in != ~0ull) break;
    }
    return __builtin_amdgcn_readfirstlane(at);
}

template <typename T, bool MUON>
__device__ __forceinline__ float update_of(const Mat& m, const Call& c, size_t i)
{
    const float g = Store<T>::ld((const T*)m.g + i);
    return MUON ? g + c.mu * m.momentum[i] : g;
}

// Momentum (descent step), and the sums of the squares of U's elements, in double: a square of 1e20 or 1e-30 is no fp32 number
template <typename T, bool MUON>
__global__ __launch_bounds__(256) void squares_kernel(const Call c)
{
    __shared__ double red[256];
    const int id = blockIdx.x, k = find_matrix(c.count, id, [&](int i) { return c.mats[i].squares_first; });
    const Mat& m = c.mats[k];
    const size_t total = (size_t)m.rows * m.cols;
    double s = 0.0;
    for (size_t i = (size_t)(id - m.squares_first) * 256 + threadIdx.x; i < total; i += (size_t)m.squares * 256) {
        float u = Store<T>::ld((const T*)m.g + i);
        if constexpr (MUON) {
            const float v = c.mu * m.momentum[i] + u;
            m.momentum[i] = v;
            u += c.mu * v;
        }
        s += (double)u * (double)u;
    }
    red[threadIdx.x] = s;
    __syncthreads();
    for (int d = 128; d >= 1; d >>= 1) {
        if ((int)threadIdx.x < d) red[threadIdx.x] += red[threadIdx.x + d];
        __syncthreads();
    }
    if (threadIdx.x == 0) c.squares[id] = red[0];
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

// A wave's 32 x 32 values in LDS, as an operand's two blocks: rows = the tile's rows (COLUMNS: its columns).  f(v, at): v as they are stored, at: byte offset of the
// lane's 16 bytes of the first piece.
template <int P, bool COLUMNS, class F>
__device__ __forceinline__ void emit(const float* tile, unsigned char* dst, F f)
{
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
        float v[8];
        const int k0 = kb * 16 + half * 8;
        if constexpr (COLUMNS) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = tile[(k0 + e) * PITCH + l32];
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const f32x4 t = *reinterpret_cast<const f32x4*>(tile + l32 * PITCH + k0 + 4 * j);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * j + e] = t[e];
            }
        }
        const int at = kb * P * BLOCK + lane * 16;
        f(v, at, k0);
        u32x4 p[P];
        cut8<P>(v, p);
#pragma unroll
        for (int e = 0; e < P; ++e) *reinterpret_cast<u32x4*>(dst + at + e * BLOCK) = p[e];
    }
}

__device__ __forceinline__ long long block_at(int P, int rb, int kblocks32, int kb32) { return ((long long)rb * kblocks32 + kb32) * (2 * P * BLOCK); }

// X = U / (|U| + eps) in both orders, cut into pieces: a wave per 32 x 32 block
template <typename T, int P, bool MUON>
__global__ __launch_bounds__(256) void cut_kernel(const Call c)
{
    __shared__ __attribute__((aligned(16))) float tiles[4][32 * PITCH];
    __shared__ double red[256];
    const int id = blockIdx.x, k = find_matrix(c.count, id, [&](int i) { return c.mats[i].cut_first; });
    const Mat& m = c.mats[k];
    red[threadIdx.x] = (int)threadIdx.x < m.squares ? c.squares[m.squares_first + threadIdx.x] : 0.0;
    __syncthreads();
    for (int d = 128; d >= 1; d >>= 1) {
        if ((int)threadIdx.x < d) red[threadIdx.x] += red[threadIdx.x + d];
        __syncthreads();
    }
    const double inv = 1.0 / (sqrt(red[0]) + (double)c.eps);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int b = (id - m.cut_first) * 4 + wave;
    if (b >= m.mb * m.nb) return;
    const int bi = b / m.nb, bj = b - bi * m.nb;
    float* const tile = tiles[wave];
    // lanes along the matrix's own columns; the tile's rows are X's
    const int r0 = (m.tall ? bj : bi) * 32, c0 = (m.tall ? bi : bj) * 32;
#pragma unroll 4
    for (int r = half; r < 32; r += 2) {
        const int row = r0 + r, col = c0 + l32;
        const float u = row < m.rows && col < m.cols ? (float)((double)update_of<T, MUON>(m, c, (size_t)row * m.cols + col) * inv) : 0.f;
        tile[m.tall ? l32 * PITCH + r : r * PITCH + l32] = u;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    auto keep = [](float (&)[8], int, int) {};
    emit<P, false>(tile, c.ws + m.x + block_at(P, bi, m.nb, bj), keep);
    emit<P, true>(tile, c.ws + m.xt[0] + block_at(P, bj, m.mb, bi), keep);
}

// What becomes of a 32 x 32 block (bi, bj) of a product, which the wave has in LDS
template <typename T, int P, int WHAT, bool MUON>
__device__ __forceinline__ void finish_block(const Call& c, const Mat& m, const float* tile, int bi, int bj, int turn, bool last)
{
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    if constexpr (WHAT == APPLY) {
        if (last) {
#pragma unroll 4
            for (int r = half; r < 32; r += 2) {
                const int row = (m.tall ? bj : bi) * 32 + r, col = (m.tall ? bi : bj) * 32 + l32;
                if (row >= m.rows || col >= m.cols) continue;
                const float v = tile[m.tall ? l32 * PITCH + r : r * PITCH + l32];
                const size_t i = (size_t)row * m.cols + col;
                if constexpr (MUON) m.w[i] = c.keep * m.w[i] - m.scale * v;
                else Store<T>::st((T*)m.o + i, v);
            }
            return;
        }
        auto keep = [](float (&)[8], int, int) {};
        emit<P, false>(tile, c.ws + m.x + block_at(P, bi, m.nb, bj), keep);
        emit<P, true>(tile, c.ws + m.xt[turn ^ 1] + block_at(P, bj, m.mb, bi), keep);
    } else {
        const long long here = block_at(P, bi, m.mb, bj), there = block_at(P, bj, m.mb, bi);
        if constexpr (WHAT == GRAM) {
            auto keep = [](float (&)[8], int, int) {};
            emit<P, false>(tile, c.ws + m.a + here, keep);
            if (bi != bj) emit<P, true>(tile, c.ws + m.a + there, keep);
        } else {
            const int short_side = m.tall ? m.cols : m.rows;
            auto poly = [&](const unsigned char* a, int row0, int col0) {
                return [=](float (&v)[8], int at, int k0) {
                    u32x4 p[P];
                    float t[8];
#pragma unroll
                    for (int e = 0; e < P; ++e) p[e] = *reinterpret_cast<const u32x4*>(a + at + e * BLOCK);
                    join8<P>(p, t);
                    const int row = row0 + l32, col = col0 + k0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = c.b * t[e] + c.c * v[e] + (row == col + e && row < short_side ? c.a : 0.f);
                };
            };
            emit<P, false>(tile, c.ws + m.q + here, poly(c.ws + m.a + here, bi * 32, bj * 32));
            if (bi != bj) emit<P, true>(tile, c.ws + m.q + there, poly(c.ws + m.a + there, bj * 32, bi * 32));
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
    large = mfma(a[0], b[0], large);
    small = mfma(a[0], b[1], small);
    small = mfma(a[1], b[0], small);
    if constexpr (P == 3) {
        small = mfma(a[1], b[1], small);
        small = mfma(a[0], b[2], small);
        small = mfma(a[2], b[0], small);
    }
}

template <int WHAT>
__device__ __forceinline__ void operands(const Call& c, const Mat& m, int turn, const unsigned char*& left, const unsigned char*& right, int& kblocks, int& left_rows, int& right_rows)
{
    left = c.ws + (WHAT == GRAM ? m.x : WHAT == POLY ? m.a : m.q);
    right = c.ws + (WHAT == GRAM ? m.x : WHAT == POLY ? m.a : m.xt[turn]);
    kblocks = 2 * (WHAT == GRAM ? m.nb : m.mb);
    left_rows = m.mb;
    right_rows = WHAT == APPLY ? m.nb : m.mb;
}

// A product of small matrices: a workgroup of four waves per tile of T x T blocks, every wave a quarter of the contraction, operands straight to registers
template <typename E, int P, int WHAT, int T, bool MUON>
__global__ __launch_bounds__(256) void product_kernel(const Call c, int turn, int last)
{
    __shared__ __attribute__((aligned(16))) float sums[4][T * T][32 * PITCH];
    const int id = blockIdx.x, k = find_matrix(c.count, id, [&](int i) { return c.mats[i].unit_first[WHAT]; });
    const Mat& m = c.mats[k];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    int bi, bj;
    tile_blocks<WHAT, T>(m, id - m.unit_first[WHAT], bi, bj);
    const unsigned char *left, *right;
    int kblocks, lrows, rrows;
    operands<WHAT>(c, m, turn, left, right, kblocks, lrows, rrows);
    const unsigned char *lp[T], *rp[T];
#pragma unroll
    for (int i = 0; i < T; ++i) {            // (a block beyond the last is the last again, and is not stored)
        lp[i] = left + (long long)min(bi + i, lrows - 1) * kblocks * P * BLOCK + lane * 16;
        rp[i] = right + (long long)min(bj + i, rrows - 1) * kblocks * P * BLOCK + lane * 16;
    }
    f32x16 large[T][T], small[T][T];
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) large[i][j][v] = small[i][j][v] = 0.f;
    for (int kb = wave; kb < kblocks; kb += 4) {
        u32x4 a[T][P], b[T][P];
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int e = 0; e < P; ++e) {
                a[i][e] = *reinterpret_cast<const u32x4*>(lp[i] + ((long long)kb * P + e) * BLOCK);
                b[i][e] = *reinterpret_cast<const u32x4*>(rp[i] + ((long long)kb * P + e) * BLOCK);
            }
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int j = 0; j < T; ++j) multiply<P>(a[i], b[j], large[i][j], small[i][j]);
    }
    // register v holds row 8 (v / 4) + 4 half + v % 4 of column lane % 32
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) sums[wave][i * T + j][(8 * (v >> 2) + 4 * half + (v & 3)) * PITCH + l32] = large[i][j][v] + small[i][j][v];
    __syncthreads();
    for (int i = threadIdx.x; i < T * T * 32 * 32; i += 256) {
        const int blk = i >> 10, at = ((i >> 5) & 31) * PITCH + (i & 31);
        sums[0][blk][at] = (sums[0][blk][at] + sums[1][blk][at]) + (sums[2][blk][at] + sums[3][blk][at]);
    }
    __syncthreads();
    for (int blk = wave; blk < T * T; blk += 4) {
        const int i = bi + blk / T, j = bj + blk % T;
        if (i < lrows && j < rrows && (WHAT == APPLY || i >= j)) finish_block<E, P, WHAT, MUON>(c, m, sums[0][blk], i, j, turn, last != 0);
    }
}

// ---- the plan of a call: made in the same way to size the workspace and to run
struct Plan {
    size_t table, squares, operands, total;      // offsets in the workspace, and its size
    int squares_units, cut_units, units[PRODUCTS];
};

template <int T>
int tiles_of(int what, int mb, int nb)
{
    const int tm = (mb + T - 1) / T, tn = (nb + T - 1) / T;
    return what == APPLY ? tm * tn : tm * (tm + 1) / 2;
}

constexpr int TILE = 2;

// Fills one matrix' entry and moves the plan's counters behind it
void place(int rows, int cols, int P, Plan& p, size_t& at, Mat& m)
{
    m.rows = rows; m.cols = cols;
    m.tall = rows > cols;
    const int s = std::min(rows, cols), l = std::max(rows, cols);
    m.mb = (s + 31) / 32;
    m.nb = (l + 31) / 32;
    const size_t wide = (size_t)m.mb * m.nb * 2 * P * BLOCK, square = (size_t)m.mb * m.mb * 2 * P * BLOCK;
    auto take = [&](size_t bytes) { const size_t o = at; at += bytes; return (long long)o; };
    m.x = take(wide);
    m.xt[0] = take(wide);
    m.xt[1] = take(wide);
    m.a = take(square);
    m.q = take(square);
    m.squares_first = p.squares_units;
    m.squares = (int)std::min<size_t>(SQUARES, ((size_t)rows * cols + 4095) / 4096);
    p.squares_units += m.squares;
    m.cut_first = p.cut_units;
    p.cut_units += (m.mb * m.nb + 3) / 4;
    for (int w = 0; w < PRODUCTS; ++w) {
        m.unit_first[w] = p.units[w];
        m.splits[w] = 1;
        p.units[w] += tiles_of<TILE>(w, m.mb, m.nb);
    }
}

template <class Shape>
Plan make_plan(int count, int P, Shape shape)
{
    Plan p{};
    size_t at = 0;
    Mat m{};
    for (int i = 0; i < count; ++i) {
        int rows, cols;
        shape(i, rows, cols);
        place(rows, cols, P, p, at, m);
    }
    p.table = 0;
    p.squares = align_up((size_t)count * sizeof(Mat), 256);
    p.operands = align_up(p.squares + (size_t)p.squares_units * sizeof(double), 256);
    p.total = p.operands + at;
    return p;
}

template <typename E, int P, bool MUON>
int run(const Plan& p, const Call& c, int steps, hipStream_t st)
{
    hipLaunchKernelGGL((squares_kernel<E, MUON>), dim3(p.squares_units), dim3(256), 0, st, c);
    hipLaunchKernelGGL((cut_kernel<E, P, MUON>), dim3(p.cut_units), dim3(256), 0, st, c);
    for (int s = 0; s < steps; ++s) {
        const int last = s + 1 == steps;
        hipLaunchKernelGGL((product_kernel<E, P, GRAM, TILE, MUON>), dim3(p.units[GRAM]), dim3(256), 0, st, c, s & 1, last);
        hipLaunchKernelGGL((product_kernel<E, P, POLY, TILE, MUON>), dim3(p.units[POLY]), dim3(256), 0, st, c, s & 1, last);
        hipLaunchKernelGGL((product_kernel<E, P, APPLY, TILE, MUON>), dim3(p.units[APPLY]), dim3(256), 0, st, c, s & 1, last);
    }
    return check_launch("orthogonalise");
}

// Writes the table of matrices to the workspace: its entries travel as arguments of small launches, so that a recorded call holds them
template <class Fill>
void write_table(int count, int P, Mat* table, size_t operands, hipStream_t st, Fill fill)
{
    Plan p{};
    size_t at = operands;
    Table t;
    for (int i = 0; i < count; ++i) {
        Mat& m = t.m[i % TABLE_CHUNK];
        m = Mat{};
        int rows, cols;
        fill(i, rows, cols, m);
        place(rows, cols, P, p, at, m);
        const int n = i % TABLE_CHUNK + 1;
        if (n == TABLE_CHUNK || i + 1 == count) hipLaunchKernelGGL(table_kernel, dim3(1), dim3(64), 0, st, t, table, i + 1 - n, n);
    }
}

Call make_call(const Plan& p, int count, const dr_newton_schulz& ns, void* ws)
{
    Call c{};
    c.ws = (unsigned char*)ws;
    c.mats = (const Mat*)(c.ws + p.table);
    c.squares = (double*)(c.ws + p.squares);
    c.count = count;
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
    const int P = dtype == DR_F32 ? 3 : 2;
    const Plan p = make_plan(count, P, [&](int i, int& r, int& c) { r = ms[i].rows; c = ms[i].cols; });
    if (p.cut_units == 0) return DR_OK;
    const Call c = make_call(p, count, ns, ws);
    TraceScope trace("orthogonalise", nullptr, count, st);
    write_table(count, P, (Mat*)c.mats, p.operands, st, [&](int i, int& r, int& cols, Mat& m) {
        r = ms[i].rows; cols = ms[i].cols;
        m.g = g[i];
        m.o = o[i];
    });
    return dtype == DR_F32 ? run<float, 3, false>(p, c, ns.steps, st) : run<uint16_t, 2, false>(p, c, ns.steps, st);
}

size_t muon_step_workspace_bytes(int count, const dr_muon_param* ps)
{
    return make_plan(count, 3, [&](int i, int& r, int& c) { r = ps[i].rows; c = ps[i].cols; }).total;
}

int launch_muon_step(int count, const dr_muon_param* ps, const dr_muon& opt, void* ws, hipStream_t st)
{
    const Plan p = make_plan(count, 3, [&](int i, int& r, int& c) { r = ps[i].rows; c = ps[i].cols; });
    if (p.cut_units == 0) return DR_OK;
    Call c = make_call(p, count, opt.ns, ws);
    c.mu = opt.momentum;
    c.keep = (float)(1.0 - (double)opt.lr * opt.weight_decay);
    TraceScope trace("muon_step", nullptr, count, st);
    write_table(count, 3, (Mat*)c.mats, p.operands, st, [&](int i, int& r, int& cols, Mat& m) {
        r = ps[i].rows; cols = ps[i].cols;
        m.g = ps[i].dw;
        m.momentum = ps[i].momentum;
        m.w = ps[i].w;
        m.scale = (float)((double)opt.lr * sqrt(std::max(1.0, (double)r / cols)));
    });
    return run<float, 3, true>(p, c, opt.ns.steps, st);
}

}  // namespace dr
