// Low-rank adapters of many requests beside one shared projection (dr_adapter_fwd) and their gradient (dr_adapter_bwd).  Rows are the pixels of channels-last images, and
// every image names its adapter a:
//
//   forward    t = s_a A_a drop(x),  y = W x + b + B_a t
//   gradient   u = s_a B_a^T dy,  dx = W^T dy + drop'(A_a^T u),  dA_a = sum u drop(x)^T,  dB_a = sum dy t^T  over the rows of adapter a
//
// Both are a narrow product (t, u: rows x rank), a wide one whose contraction runs over the projection and then over the rank, and for the gradient two sums over the rows
// of each adapter.  Rows are visited in the order of their adapters, so that few tiles hold rows of several; such a tile takes its adapters one after the other.
// t and u are held in fp32 and enter bf16 products as three pieces each, all their bits: an output in which the projection and the adapter nearly cancel shows them.
//
// 8192 rows of 4096 channels to 4096 in bf16, eight adapters of rank 16, dropout: forward 267 us, gradient 346.  Their kernels under the profiler, shortest and average of 20:
// order 7.5 and 8.4, narrow 26 and 32, wide 234 and 264 (1.17 and 1.04 PFLOP/s; the library's product alone takes 217); order and copies 18 and 19, narrow 17 and 19, sums 62 and 70 with
// 6 for their join, wide 249 and 275.
#include <algorithm>
#include <type_traits>

#include "dr_internal.h"
#include "philox.h"
#include "rows8.h"

namespace dr {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight 16-bit elements, of which those without a bit become zero (their bits times 0 or 1)
__device__ __forceinline__ void keep_halves(u32x4& v, unsigned bits)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned two = bits >> (2 * i) & 3, word = v[i], times = (two | two << 15) & 0x00010001u;      // (a cast of v[i] itself would read v[0])
        const u16x2 kept = __builtin_bit_cast(u16x2, word) * __builtin_bit_cast(u16x2, times);
        v[i] = __builtin_bit_cast(unsigned, kept);
    }
}

// Eight elements of a row.  load(row, k, K) reads elements k .. k + 7 of a row of K >= 8, or its last eight where it ends before, which settle() then moves to their places, with zeros behind
// them: loads without a condition between them stay in flight together.  load_any() is for rows of any length.
template <typename T> struct Operand;
template <> struct Operand<uint16_t> {
    u32x4 v;
    __device__ __forceinline__ void load(const uint16_t* row, int k, int K) { v = *reinterpret_cast<const u32x4_any*>(row + min(k, K - 8)); }
    __device__ __forceinline__ void settle(int k, int K)
    {
        const int s = max(0, min(k - (K - 8), 8));
        uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
        if (s >= 4) { lo = hi; hi = 0; }
        const int bits = 16 * (s & 3);
        lo = lo >> bits | (bits ? hi << (64 - bits) : 0);
        hi >>= bits;
        if (s == 8) lo = 0;
        v = u32x4{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
    }
    __device__ __forceinline__ void load_any(const uint16_t* row, int k, int K)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (k + 2 * i < K ? row[k + 2 * i] : 0u) | (k + 2 * i + 1 < K ? (unsigned)row[k + 2 * i + 1] << 16 : 0u);
    }
    __device__ __forceinline__ void clear() { v = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ void keep(unsigned bits) { keep_halves(v, bits); }
    __device__ __forceinline__ void values(float (&e)[8]) const { unpack8(v, e); }
};
template <> struct Operand<float> {
    f32x4 v[2];
    __device__ __forceinline__ void load(const float* row, int k, int K)
    {
        const float* p = row + min(k, K - 8);
        v[0] = *reinterpret_cast<const f32x4_any*>(p);
        v[1] = *reinterpret_cast<const f32x4_any*>(p + 4);
    }
    __device__ __forceinline__ void settle(int k, int K)
    {
        const int s = max(0, min(k - (K - 8), 8));
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1)
            if (s & d) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = i + d < 8 ? v[(i + d) >> 2 & 1][(i + d) & 3] : 0.f;
            }
    }
    __device__ __forceinline__ void load_any(const float* row, int k, int K)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = k + i < K ? row[k + i] : 0.f;
    }
    __device__ __forceinline__ void clear() { v[0] = v[1] = f32x4{0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ void keep(unsigned bits)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j >> 2][j & 3] = bits >> j & 1 ? v[j >> 2][j & 3] : 0.f;
    }
    __device__ __forceinline__ void values(float (&e)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = v[i >> 2][i & 3];
    }
};
// Which of the eight elements from `first` on dropout keeps, a bit each
__device__ __forceinline__ unsigned kept8_from(const Drop& d, uint64_t place, uint64_t first)
{
    const unsigned bits = kept8(d, place, first >> 3);
    return first & 7 ? ((bits | kept8(d, place, (first >> 3) + 1) << 8) >> (first & 7)) & 0xFFu : bits;
}

// Which row is at a position, and its adapter.  Positions walk the images in `order` (NULL: as they come).
struct Rows {
    int count, hw;               // rows; pixels of an image
    int adapters, rank;
    const int* ids;              // of every image (NULL: none has an adapter)
    const int* order;
    const int* starts;           // adapter a's images are order[starts[a]] .. order[starts[a + 1] - 1] (read by the sums over rows)
    const float* scales;
    __device__ __forceinline__ int row(int p, int* id) const
    {
        const int slot = p / hw, img = order ? order[slot] : slot, a = ids ? ids[img] : -1;
        *id = (unsigned)a < (unsigned)adapters ? a : -1;
        return img * hw + (p - slot * hw);
    }
};

// ---- what the products start from: the order of the images by adapter, and transposed copies ------------------------------------------------------
// Order: workgroup a writes the images of adapter a (the last one those without) in the order in which they come: first how many belong before them, then which they
// are.  A wave takes a quarter of the ids, four of a lane at a time.
// Copies: src[batch][R][C] -> dst[batch][C][R], 64 x 64 elements a workgroup.  Of W, A and B for the gradient, whose products run over the other dimension: 18 us of 346 at
// 4096 x 4096 in bf16, most of it W's 64 MB; one launch with the order, where four took 53.
struct Copy { const void* src; void* dst; int R, C, tiles_r, tiles_c, first, last; };      // workgroups first .. last - 1
struct Prepare {
    const int* ids;
    int n, adapters, orders;     // orders: workgroups of the order (0: none)
    int *order, *starts;
    Copy copy[3];
};
__device__ __forceinline__ void put_in_order(const Prepare& p, int a, int* red)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int share = ((p.n + 1023) / 1024) * 256, lo = min(wave * share, p.n), hi = min(lo + share, p.n);
    constexpr int AHEAD = 8;     // runs of 256 ids whose loads are in flight together
    auto load = [&](int i0, int (&key)[AHEAD][4]) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) key[u][j] = p.ids[min(i0 + u * 256 + lane * 4 + j, p.n - 1)];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) key[u][j] = i0 + u * 256 + lane * 4 + j < hi ? min((unsigned)key[u][j], (unsigned)p.adapters) : 0x7FFFFFFF;
    };
    int before = 0, own = 0;
    for (int i0 = lo; i0 < hi; i0 += AHEAD * 256) {
        int key[AHEAD][4];
        load(i0, key);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                before += key[u][j] < a;
                own += key[u][j] == a;
            }
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        before += __shfl_xor(before, d, 64);
        own += __shfl_xor(own, d, 64);
    }
    if (lane == 0) {
        red[wave] = before;
        red[4 + wave] = own;
    }
    __syncthreads();
    const int base = red[0] + red[1] + red[2] + red[3];
    if (threadIdx.x == 0) {
        p.starts[a] = base;
        if (a == p.adapters) p.starts[a + 1] = p.n;
    }
    int at = base;
    for (int w = 0; w < wave; ++w) at += red[4 + w];
    if (red[4 + wave] == 0) return;
    const unsigned long long below = (1ull << lane) - 1;
    for (int i0 = lo; i0 < hi; i0 += AHEAD * 256) {
        int key[AHEAD][4];
        load(i0, key);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            int mine = at;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned long long set = __ballot(key[u][j] == a);
                mine += __popcll(set & below);
                at += __popcll(set);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (key[u][j] == a) p.order[mine++] = i0 + u * 256 + lane * 4 + j;
        }
    }
}
template <typename T>
__global__ __launch_bounds__(256) void prepare_kernel(const Prepare p)
{
    constexpr int E = 16 / sizeof(T);
    constexpr int PITCH = 64 + 4 / (int)sizeof(T);           // an odd number of words: a column is in as many banks as it has rows
    __shared__ __attribute__((aligned(16))) T tile[64][PITCH];
    __shared__ int red[8];
    const int block = blockIdx.x;
    if (block < p.orders) return put_in_order(p, block, red);
    const int which = block < p.copy[0].last ? 0 : block < p.copy[1].last ? 1 : 2;
    auto of = [&](auto field) { return which == 0 ? p.copy[0].*field : which == 1 ? p.copy[1].*field : p.copy[2].*field; };
    const Copy c = {of(&Copy::src), of(&Copy::dst), of(&Copy::R), of(&Copy::C), of(&Copy::tiles_r), of(&Copy::tiles_c), of(&Copy::first), 0};
    const int i = block - c.first, per = c.tiles_r * c.tiles_c, b = i / per, j = i - b * per, r0 = j / c.tiles_c * 64, c0 = (j - j / c.tiles_c * c.tiles_c) * 64;
    const T* src = (const T*)c.src + (size_t)b * c.R * c.C;
    T* dst = (T*)c.dst + (size_t)b * c.R * c.C;
    if (r0 + 64 <= c.R && c0 + 64 <= c.C) {
#pragma unroll
        for (int k = 0; k < 16 / E; ++k) {
            const int e = threadIdx.x + k * 256, r = e / (64 / E), o = e % (64 / E) * E;
            const u32x4 v = *reinterpret_cast<const u32x4_any*>(src + (size_t)(r0 + r) * c.C + c0 + o);
#pragma unroll
            for (int u = 0; u < 4; ++u) reinterpret_cast<unsigned*>(&tile[r][o])[u] = v[u];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16 / E; ++k) {
            const int e = threadIdx.x + k * 256, r = e / (64 / E), o = e % (64 / E) * E;
            T v[E];
#pragma unroll
            for (int u = 0; u < E; ++u) v[u] = tile[o + u][r];
            u32x4 w;
            __builtin_memcpy(&w, v, 16);
            *reinterpret_cast<u32x4_any*>(dst + (size_t)(c0 + r) * c.R + r0 + o) = w;
        }
        return;
    }
    for (int e = threadIdx.x; e < 4096; e += 256)
        if (r0 + e / 64 < c.R && c0 + e % 64 < c.C) tile[e / 64][e % 64] = src[(size_t)(r0 + e / 64) * c.C + c0 + e % 64];
    __syncthreads();
    for (int e = threadIdx.x; e < 4096; e += 256)
        if (c0 + e / 64 < c.C && r0 + e % 64 < c.R) dst[(size_t)(c0 + e / 64) * c.R + r0 + e % 64] = tile[e % 64][e / 64];
}

// A number's upper 16 bits, a bf16 of its first 8 significant ones; `e` is left with the rest (none of an infinity).  Cut, not rounded: three pieces hold all 24 bits, none is
// infinite unless the number is, and all have its sign.
__device__ __forceinline__ uint16_t cut(float& e)
{
    const unsigned bits = __float_as_uint(e);
    const float upper = __uint_as_float(bits & 0xFFFF0000u);
    e = e == upper ? 0.f : e - upper;
    return (uint16_t)(bits >> 16);
}
__device__ __forceinline__ u32x4 cut8(float (&e)[8])
{
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned low = cut(e[2 * i]);
        v[i] = low | (unsigned)cut(e[2 * i + 1]) << 16;
    }
    return v;
}
// What the lower pieces are multiplied by: infinities (and NaN) as bf16's largest number of their sign.  The upper piece alone meets them: a lower one may be zero, and zero times an
// infinity would make a NaN of what is infinite.  (As signed numbers the positive ones beyond 0x7F7F, as unsigned ones those beyond 0xFF7F.)
__device__ __forceinline__ u32x4 finite8(u32x4 v)
{
    typedef short i16x2 __attribute__((ext_vector_type(2)));
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned word = v[i];
        const i16x2 above = __builtin_elementwise_min(__builtin_bit_cast(i16x2, word), i16x2{0x7F7F, 0x7F7F});
        const u16x2 both = __builtin_elementwise_min(__builtin_bit_cast(u16x2, above), u16x2{0xFF7F, 0xFF7F});
        v[i] = __builtin_bit_cast(unsigned, both);
    }
    return v;
}

// 16 bytes of a row, of which `n` elements exist (zeros behind them)
__device__ __forceinline__ u32x4 piece(const char* p) { return *reinterpret_cast<const u32x4_any*>(p); }
template <typename T>
__device__ __forceinline__ u32x4 piece(const char* p, int n)
{
    constexpr int E = 16 / sizeof(T);
    if (n >= E) return piece(p);
    u32x4 v = {0, 0, 0, 0};
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) v[i >> 1] |= (unsigned)reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i & 1));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) v[i] = reinterpret_cast<const unsigned*>(p)[i];
    }
    return v;
}

// ---- products of few rows or few ranks: a wave by itself ----------------------------------------------------------------------------------------
// Rows of two matrices, A blocks of 16 of the one and B of the other, 128 bytes of a row at a time: loads in which eight lanes take a row's 128 bytes (lanes that take a row
// each, as the matrix instructions want them, are served one row a cycle: four times as long), D slices of them in flight in registers, through the wave's own LDS,
// in the order piece ^ (row / 2 & 7) (sixteen rows' pieces then lie in all 64 banks), to the operands.  Waves of a workgroup share the contraction: wave w takes slices w, w + NW, ...
struct Piece { u32x4 v; };
// What the wave's lanes have written to its own LDS is what they read behind this (the wave's LDS accesses run in order: nothing to wait for)
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
template <typename T> __device__ __forceinline__ void load_piece(Piece& e, const T* row, int k, int K)      // the row's last ones where it ends before (K >= 16 bytes)
{
    constexpr int E = 16 / sizeof(T);
    e.v = *reinterpret_cast<const u32x4_any*>(row + min(k, K - E));
}
template <typename T> __device__ __forceinline__ void load_piece_any(Piece& e, const T* row, int k, int K) { e.v = piece<T>((const char*)(row + k), K - k); }
// ... then moved to their places, zeros behind them
template <typename T> __device__ __forceinline__ void settle_piece(Piece& e, int k, int K)
{
    constexpr int E = 16 / sizeof(T);
    const int s = max(0, min(k - (K - E), E)) * (int)sizeof(T);
    uint64_t lo = (uint64_t)e.v[1] << 32 | e.v[0], hi = (uint64_t)e.v[3] << 32 | e.v[2];
    if (s >= 8) { lo = hi; hi = 0; }
    const int bits = 8 * (s & 7);
    lo = lo >> bits | (bits ? hi << (64 - bits) : 0);
    hi >>= bits;
    if (s == 16) lo = 0;
    e.v = u32x4{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
}
// Which elements of the piece that starts at element `first` dropout keeps: sets the others to zero (what is kept is scaled where the sums are, exactly)
__device__ __forceinline__ void mask_piece(const Drop& d, uint64_t place, uint64_t first, Piece& e, uint16_t)
{
    const unsigned bits = kept8_from(d, place, first);
    keep_halves(e.v, bits);
}
__device__ __forceinline__ void mask_piece(const Drop& d, uint64_t place, uint64_t first, Piece& e, float)
{
    unsigned bits = kept8(d, place, first >> 3);
    if ((first & 7) > 4) bits |= kept8(d, place, (first >> 3) + 1) << 8;
    bits >>= first & 7;
#pragma unroll
    for (int i = 0; i < 4; ++i) e.v[i] = bits >> i & 1 ? e.v[i] : 0u;
}
template <typename T> __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (sizeof(T) == 2) return mfma(a, b, c);
    else {
        const f32x4 p = __builtin_bit_cast(f32x4, a), q = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(p[i], q[i], c, 0, 0, 0);
        return c;
    }
}

// ra(i), rb(i): row of the first and of the second matrix that lane / 8 loads for rows 8 i .. 8 i + 7 of its blocks.  lds: (A + B) x 2 KiB of the wave's own.
template <typename T, int A, int B, int D, int NW, bool DROP, class RA, class RB_>
__device__ __forceinline__ void wave_product(const T* a, RA ra, const T* b, RB_ rb, int K, int wave, unsigned char* lds, const Drop& drop, uint64_t place, f32x4 (&acc)[A][B])
{
    constexpr int E = 16 / sizeof(T), SLICE = 8 * E, N = 2 * (A + B);
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, r8 = lane >> 3, c = lane & 7, slices = (K + SLICE - 1) / SLICE;
    const T* from[N];
#pragma unroll
    for (int i = 0; i < N; ++i) from[i] = i < 2 * A ? a + (size_t)ra(i) * K : b + (size_t)rb(i - 2 * A) * K;
    const bool tiny = K < E;
    Piece held[D][N];
    auto load = [&](int s, Piece (&h)[N]) {
        const int k = s * SLICE + c * E;
        if (!tiny) {
#pragma unroll
            for (int i = 0; i < N; ++i) load_piece(h[i], from[i], k, K);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) load_piece_any(h[i], from[i], k, K);
        }
    };
    auto put = [&](int s, Piece (&h)[N]) {
        const int k = s * SLICE + c * E;
        if ((s + 1) * SLICE > K && !tiny) {
#pragma unroll
            for (int i = 0; i < N; ++i) settle_piece<T>(h[i], k, K);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (DROP && i >= 2 * A) mask_piece(drop, place, (uint64_t)((size_t)rb(i - 2 * A) * K + k), h[i], T());
            *reinterpret_cast<u32x4*>(lds + (i * 8 + r8) * 128 + ((c ^ (r8 >> 1) ^ (i & 1) << 2) << 4)) = h[i].v;
        }
    };
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (wave + d * NW < slices) load(wave + d * NW, held[d]);
    for (int s0 = wave; s0 < slices; s0 += NW * D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int s = s0 + d * NW;
            if (s >= slices) break;
            put(s, held[d]);
            wave_fence();
            if (s + D * NW < slices) load(s + D * NW, held[d]);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                u32x4 x[B];
#pragma unroll
                for (int j = 0; j < B; ++j) x[j] = *reinterpret_cast<const u32x4*>(lds + (A * 16 + j * 16 + l16) * 128 + (((t * 4 + g) ^ (l16 >> 1)) << 4));
#pragma unroll
                for (int i = 0; i < A; ++i) {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(lds + (i * 16 + l16) * 128 + (((t * 4 + g) ^ (l16 >> 1)) << 4));
#pragma unroll
                    for (int j = 0; j < B; ++j) acc[i][j] = mfma16<T>(w, x[j], acc[i][j]);
                }
            }
            wave_fence();
        }
    }
}

// ---- a narrow product: out[row][r] = s_a sum_k v[row][k] M_a[r][k] -----------------------------------------------------------------------------
// A workgroup takes 16 rows and the adapters among them, every gridDim.y-th from its own on (the i-th adapter is that of the i-th row whose adapter no row before has); its NW
// waves share the contraction and add up in LDS.  Bound by memory (8192 rows of 4096 in bf16: 17-19 us, 3.5-3.9 TB/s of v, and M_a again from L2 for every 16 rows), with dropout by
// the vector instructions that draw the mask (26-32 us; 33 at its shortest where registers leave a compute unit one workgroup); 64 rows with an adapter each 7-8 us.
template <typename T, int RB, int NW, int D, bool DROP>
__global__ __launch_bounds__(NW * 64, RB == 1 && sizeof(T) == 2 ? 4 : 1) void narrow_kernel(const Rows q, const T* __restrict__ v, int K, const T* __restrict__ m, const Drop drop, float* __restrict__ out)
{
    __shared__ __attribute__((aligned(128))) unsigned char lds[NW][(RB + 1) * 2048];
    __shared__ float red[NW][RB * 16][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
    const int p = blockIdx.x * 16 + l16;
    int id = -2, row = -1;
    if (p < q.count) row = q.row(p, &id);
    bool again = id < 0;
#pragma unroll
    for (int i = 0; i < 15; ++i) again |= i < l16 && __builtin_amdgcn_readlane(id, i) == id;
    unsigned firsts = (unsigned)__ballot(!again) & 0xFFFFu;
    if (blockIdx.y == 0 && id == -1)
        for (int r = wave * 4 + g; r < q.rank; r += NW * 4) out[(size_t)row * q.rank + r] = 0.f;
    const uint64_t place = DROP ? drop_place(drop) : 0;
    for (int turn = 0; firsts; firsts &= firsts - 1, ++turn) {
        if (turn % gridDim.y != blockIdx.y) continue;
        const int first = __builtin_ctz(firsts), a = __builtin_amdgcn_readlane(id, first);
        // (what comes of rows of other adapters is not stored: they read this adapter's first row)
        const int mine = id == a ? row : __builtin_amdgcn_readlane(row, first), low = __shfl(mine, lane >> 3, 64), high = __shfl(mine, 8 + (lane >> 3), 64);
        f32x4 acc[RB][1] = {};
        auto ra = [&](int i) { return min(i * 8 + (lane >> 3), q.rank - 1); };
        auto rb = [&](int i) { return i ? high : low; };
        const T* ma = m + (size_t)a * q.rank * K;
        wave_product<T, RB, 1, D, NW, DROP>(ma, ra, v, rb, K, wave, lds[wave], drop, place, acc);
        __syncthreads();
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) red[wave][b * 16 + g * 4 + i][l16] = acc[b][0][i];
        __syncthreads();
        const float scale = (q.scales ? q.scales[a] : 1.f) * (DROP ? drop.scale : 1.f);
        // 16 lanes hold the rows, the others of the workgroup the ranks
        if (id == a)
            for (int r = wave * 4 + g; r < q.rank; r += NW * 4) {
                float s = red[0][r][l16];
#pragma unroll
                for (int w = 1; w < NW; ++w) s += red[w][r][l16];
                out[(size_t)row * q.rank + r] = s * scale;
            }
    }
}

// ---- the wide product: y[row][o] = sum_k W[o][k] x[row][k] + bias[o] + drop'(sum_r B_a[o][r] t[row][r]) ---------------------------------------------
// A workgroup of WM x WN waves owns TM = 32 MB WM outputs of TN = 32 NB WN rows, a wave MB x NB blocks of 32 x 32.  PB pieces of 16 bytes of every row of W and x are a
// stage, of which LDS holds NS: one that is multiplied and others on their way, by loads that write LDS (DMA: rows of whole, aligned 16-byte pieces), or one by way of
// registers.  A row's pieces lie in the order piece ^ (row PB / 16): the same piece of sixteen rows is then in all 64 banks.
// 8192 x 4096 x 4096 bf16 234 us with adapters, the shortest of 20 launches as are the figures behind it (1.17 PFLOP/s, 1.04 on average; before registers stopped spilling 241 without adapters; stages of 64 bytes four deep 253, bank conflicts and 8-byte stores from registers 272, by way of registers
// 315); a step of 4096 in the contraction costs what 1.29 PFLOP/s cost, the rest (35 us in two rounds of tiles) is first loads, adapters and stores.  Four waves of 128 x 128
// would read a third less from LDS, but the compiler then moves accumulators between register files (933 us).  2000 rows 66 us, 512 28, 128 19; fp32 8192 x 1024 x 1024
// 131 us (131 TFLOP/s of 157 that the fp32 instruction has; 145 where accumulators in registers of their own leave a compute unit one workgroup).
// A mask drawn here (no da, or c_in no multiple of 8) is drawn again for every adapter and step of rank of a wave, and the tile of 256 x 256 then spills about 100 registers: with dropout the
// gradient to x alone takes 321 us, 260 without; 8192 rows to 4100 channels 515.
template <typename T> struct Wide {
    Rows q;
    const T *x, *w, *b;
    const float *bias, *t;
    int K, N;
    Drop drop;
    const uint8_t* bits;         // drop's mask, if the sums over rows have left it, or NULL
    T* y;
    int tiles_n, tiles;          // tiles of rows; all tiles
};

typedef float f32x16 __attribute__((ext_vector_type(16)));
// one 16-byte piece of each operand: a lane of half h = lane / 32 holds piece 2 s + h
template <typename T> __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c);
template <> __device__ __forceinline__ f32x16 mfma32<uint16_t>(u32x4 a, u32x4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 mfma32<float>(u32x4 a, u32x4 b, f32x16 c)
{
    const f32x4 p = __builtin_bit_cast(f32x4, a), q = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(p[i], q[i], c, 0, 0, 0);
    return c;
}

// The tiles that the 8 dies' workgroups (dealt out in turn) see are neighbours: die d takes the d-th run of the list, which goes down runs of 8 tiles of rows.
__device__ __forceinline__ void tile_of(int block, int tiles, int tiles_n, int* m, int* n)
{
    const int die = block & 7, per = tiles >> 3, odd = tiles & 7, i = die * per + min(die, odd) + (block >> 3);
    const int tiles_m = tiles / tiles_n, run = i / (8 * tiles_m), wide = min(8, tiles_n - run * 8), j = i - run * 8 * tiles_m;
    *m = j / wide;
    *n = run * 8 + (j - *m * wide);
}

// 16 bytes per lane from `base` + voff + soff to LDS: lane l's at `lds` + 16 l.  Zeros where voff lies outside the buffer.  The compiler does not see the write: the
// caller waits for it (wait_loads) in front of the barrier behind which it is read.
__device__ __forceinline__ void load_lds16(const u32x4& rsrc, const unsigned char* lds, unsigned voff, unsigned soff)
{
#if defined(__HIP_DEVICE_COMPILE__)
    unsigned m0;                 // (put back: the compiler may hold something in it)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"((unsigned)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)lds), "v"(voff), "s"(rsrc), "s"(soff) : "memory");
#endif
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }      // but the last N
// the workgroup's barrier alone, without the waits of a fence (a wave's own LDS reads have been consumed before it)
__device__ __forceinline__ void meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// A tensor as a buffer of raw bytes; NOWHERE is an offset outside of it
constexpr unsigned NOWHERE = 0xFFFFFFF0u;
__device__ __forceinline__ u32x4 buffer_of(const void* p, size_t bytes)
{
    const uint64_t a = (uint64_t)p;
    return u32x4{(unsigned)__builtin_amdgcn_readfirstlane((unsigned)a), (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(a >> 32) & 0xFFFFu),
                 (unsigned)__builtin_amdgcn_readfirstlane((unsigned)bytes), 0x00020000u};
}

enum { NO_MASK = 0, MASK_DRAWN = 1, MASK_BITS = 2 };
template <typename T, int WM, int WN, int MB, int NB, int PB, int NS, bool DMA, int DROP>
__global__ __launch_bounds__(WM * WN * 64, 2) void tiled_kernel(const Wide<T> p)
{
    constexpr int TM = 32 * MB * WM, TN = 32 * NB * WN, THREADS = WM * WN * 64, PIECES = (TM + TN) * PB / THREADS, E = 16 / sizeof(T), STAGE_K = PB * E;
    constexpr int PITCH = PB * 16, WITH = 16 / PB;        // bytes of a row; rows to all 64 banks
    __shared__ __attribute__((aligned(128))) unsigned char lds[NS][(TM + TN) * PITCH];
    __shared__ int row_of[TN], id_of[TN];
    __shared__ __attribute__((aligned(16))) float bias_of[TM];
    const Rows& q = p.q;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, h = lane >> 5, wm = wave % WM, wn = wave / WM;
    int tm, tn;
    tile_of(blockIdx.x, p.tiles, p.tiles_n, &tm, &tn);
    const int o0 = tm * TM, p0 = tn * TN;
    for (int i = threadIdx.x; i < TN; i += THREADS) {
        int id = -2, row = -1;
        if (p0 + i < q.count) row = q.row(p0 + i, &id);
        row_of[i] = row;
        id_of[i] = id;
    }
    for (int i = threadIdx.x; i < TM; i += THREADS) bias_of[i] = p.bias ? p.bias[min(o0 + i, p.N - 1)] : 0.f;
    __syncthreads();

    // this thread's pieces of a stage: row and piece are the same in every stage.  Rows that do not exist repeat one that does: what comes of them is not stored
    std::conditional_t<DMA, unsigned, size_t> from[PIECES];
    int at[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int e = threadIdx.x + i * THREADS, r = e / PB, c = e % PB;
        const int row = r < TM ? min(o0 + r, p.N - 1) : max(row_of[r - TM], 0);
        // (DMA: the lane's place in LDS is given, and it fetches the piece that belongs there)
        from[i] = (decltype(from[i] + 0))((size_t)row * p.K * sizeof(T)) + (DMA ? c ^ (r / WITH & (PB - 1)) : c) * 16;
        at[i] = r * PITCH + ((c ^ (r / WITH & (PB - 1))) << 4);
    }
    const int stages = (p.K + STAGE_K - 1) / STAGE_K, whole = p.K / STAGE_K;
    u32x4 held[PIECES];
    auto fetch = [&](int s) {
        const char *w = (const char*)p.w + (size_t)s * PITCH, *x = (const char*)p.x + (size_t)s * PITCH;
        if (s < whole) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) held[i] = piece((i < PIECES * TM / (TM + TN) ? w : x) + from[i]);
        } else {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) held[i] = piece<T>((i < PIECES * TM / (TM + TN) ? w : x) + from[i], p.K - s * STAGE_K - (int)((threadIdx.x + i * THREADS) % PB) * E);
        }
    };
    auto put = [&](unsigned char* to) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) *reinterpret_cast<u32x4*>(to + at[i]) = held[i];
    };
    [[maybe_unused]] const u32x4 rw = buffer_of(p.w, (size_t)p.N * p.K * sizeof(T)), rx = buffer_of(p.x, (size_t)q.count * p.K * sizeof(T));
    auto stream = [&](int s, unsigned char* to) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            unsigned voff = from[i];
            if (s >= whole) {                // (the last stage, if it is no whole one)
                const int e = threadIdx.x + i * THREADS;
                if (s * PITCH + ((e ^ (e / PB / WITH)) & (PB - 1)) * 16 >= p.K * (int)sizeof(T)) voff = NOWHERE;
            }
            load_lds16(i < PIECES * TM / (TM + TN) ? rw : rx, to + (wave + i * (THREADS / 64)) * 1024, voff, s * PITCH);
        }
    };
    f32x16 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float from_bias = bias_of[(wm * MB + i) * 32 + (e >> 2) * 8 + h * 4 + (e & 3)];
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j][e] = from_bias;
        }
    const int rd_m = (wm * MB * 32 + l32) * PITCH, rd_n = (TM + wn * NB * 32 + l32) * PITCH;
    // operands two steps deep: those of step k + 1 are read while step k is multiplied, the next stage's first ones behind the barrier and in front of the last step
    u32x4 a[2][MB], b[2][NB];
    auto read = [&](const unsigned char* buf, int k, int to) {
        const int c = ((2 * k + h) ^ (l32 / WITH & (PB - 1))) << 4;
#pragma unroll
        for (int i = 0; i < MB; ++i) a[to][i] = *reinterpret_cast<const u32x4*>(buf + rd_m + i * 32 * PITCH + c);
#pragma unroll
        for (int j = 0; j < NB; ++j) b[to][j] = *reinterpret_cast<const u32x4*>(buf + rd_n + j * 32 * PITCH + c);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = mfma32<T>(a[from][i], b[from][j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    if constexpr (DMA) {
#pragma unroll
        for (int s = 0; s < NS; ++s)
            if (s < stages) stream(s, lds[s]);
        wait_loads<0>();
        meet();
    } else {
        fetch(0);
        put(lds[0]);
        __syncthreads();
        if (stages > 1) fetch(1);
    }
    read(lds[0], 0, 0);
    for (int s = 0; s < stages; ++s) {
        unsigned char *const here = lds[s % NS], *const next = lds[(s + 1) % NS];
#pragma unroll
        for (int k = 0; k < PB / 2 - 1; ++k) {
            read(here, k + 1, (k + 1) & 1);
            multiply(k & 1);
        }
        if constexpr (DMA) {
            __builtin_amdgcn_s_waitcnt(0xC07F);            // lgkmcnt(0): nothing of this stage is still to be read
            if (s + NS - 1 < stages) wait_loads<(NS - 2) * PIECES>();    // the next stage has landed, those behind it may be on their way
            else wait_loads<0>();
            meet();
            if (s + NS < stages) stream(s + NS, here);
        } else {
            if (s + 1 < stages) put(next);
            __syncthreads();
            if (s + 2 < stages) fetch(s + 2);
        }
        if (s + 1 < stages) read(next, 0, 0);
        multiply(1);
    }

    // the adapters of this wave's rows, one after the other
    int row[NB], id[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        row[j] = row_of[(wn * NB + j) * 32 + l32];
        id[j] = id_of[(wn * NB + j) * 32 + l32];
    }
    const int ow = o0 + wm * MB * 32;
    const uint64_t place = DROP == MASK_DRAWN ? drop_place(p.drop) : 0;
    const float scale = DROP ? p.drop.scale : 1.f;
    [[maybe_unused]] unsigned kept_bits[MB][NB];
    if constexpr (DROP == MASK_BITS) {
        typedef unsigned int u32_any __attribute__((aligned(1)));
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
                kept_bits[i][j] = *reinterpret_cast<const u32_any*>(p.bits + (((size_t)max(row[j], 0) * p.N + min(ow + i * 32, p.N - 1)) >> 3));
    }
    for (int a = -1;;) {
        int next = 0x7FFFFFFF;
#pragma unroll
        for (int j = 0; j < NB; ++j) next = id[j] > a ? min(next, id[j]) : next;
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) next = min(next, __shfl_xor(next, d, 64));
        next = __builtin_amdgcn_readfirstlane(next);
        if (next == 0x7FFFFFFF) break;
        a = next;
        constexpr int STEP = 2 * E;
        for (int r0 = 0; r0 < q.rank; r0 += STEP) {
            // (what comes of rows of other adapters is not taken, so their t need not be left out)
            const int r = r0 + h * E;
            const bool all = r0 + STEP <= q.rank;
            u32x4 high[NB], middle[NB], low[NB], factor[MB];
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const char* at = (const char*)(p.b + ((size_t)a * p.N + min(ow + i * 32 + l32, p.N - 1)) * q.rank + r);
                factor[i] = all ? piece(at) : piece<T>(at, q.rank - r);
            }
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const float* at = p.t + (size_t)max(row[j], 0) * q.rank + r;
                if constexpr (sizeof(T) == 2) {
                    float e[8];
                    if (all) load8(at, e);
                    else load8(at, q.rank - r, 0.f, e);
                    high[j] = cut8(e);
                    middle[j] = cut8(e);
                    low[j] = cut8(e);
                } else high[j] = all ? piece((const char*)at) : piece<T>((const char*)at, q.rank - r);
            }
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const u32x4 v = factor[i], vf = sizeof(T) == 2 ? finite8(v) : v;
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    // this lane's row of the block: outputs 16 h .. 16 h + 15, the others from the lane that holds the same row
                    unsigned keep = 0xFFFFFFFFu;
                    if constexpr (DROP == MASK_BITS) keep = kept_bits[i][j] >> (h * 4);
                    if constexpr (DROP == MASK_DRAWN) {
                        const unsigned own = kept16(p.drop, place, (size_t)max(row[j], 0) * p.N + min(ow + i * 32, p.N - 1) + h * 16), other = __shfl_xor(own, 32, 64);
                        keep = (h ? own << 16 | other : other << 16 | own) >> (h * 4);
                    }
                    f32x16 part = {};          // of its own: rows of other adapters must not meet this one's numbers, not even times zero
                    part = mfma32<T>(v, high[j], part);
                    if constexpr (sizeof(T) == 2) {
                        part = mfma32<T>(vf, middle[j], part);
                        part = mfma32<T>(vf, low[j], part);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const bool mine = id[j] == a && (keep >> ((e >> 2) * 8 + (e & 3)) & 1);
                        acc[i][j][e] += mine ? part[e] * scale : 0.f;
                    }
                }
            }
        }
    }
    // 32 rows at a time through the wave's own part of LDS, so that a store writes a row's outputs together (16 bytes of 32 rows each would take L2 a request apiece)
    constexpr int ROW = MB * 32 * sizeof(T), IN_ROW = ROW / 16, SPREAD = ROW < 256 ? 256 / ROW : 1;
    static_assert(WM * WN * 32 * ROW <= (int)sizeof(lds), "a wave's rows");
    unsigned char* const mine = &lds[0][0] + wave * 32 * ROW;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NB; ++j) {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float v[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] = acc[i][j][e * 4 + c];
                const int in = (i * 32 + e * 8 + h * 4) * (int)sizeof(T);
                store4(reinterpret_cast<T*>(mine + l32 * ROW + (((in >> 4) ^ (l32 / SPREAD & (IN_ROW - 1))) << 4) + (in & 15)), v);
            }
        wave_fence();
#pragma unroll
        for (int k = 0; k < 32 * IN_ROW / 64; ++k) {
            const int e = lane + k * 64, r = e / IN_ROW, c = e % IN_ROW, o = ow + c * E, to_row = row_of[(wn * NB + j) * 32 + r];
            const u32x4 v = *reinterpret_cast<const u32x4*>(mine + r * ROW + ((c ^ (r / SPREAD & (IN_ROW - 1))) << 4));
            if (to_row < 0) continue;
            T* to = p.y + (size_t)to_row * p.N + o;
            if (o + E <= p.N) *reinterpret_cast<u32x4_any*>(to) = v;
            else {
                T part[E];
                __builtin_memcpy(part, &v, 16);
#pragma unroll
                for (int u = 0; u < E; ++u)
                    if (o + u < p.N) to[u] = part[u];
            }
        }
        wave_fence();
    }
}

// ---- the wide product of few rows ---------------------------------------------------------------------------------------------------------------
// A workgroup owns 16 outputs of up to 64 rows (NB blocks of 16) and its eight waves share the contraction, so that W is read by as many compute units as there are blocks
// of 16 outputs.  The sums of the waves are added in LDS, where a lane adds the adapter's part of its output by itself: rank products.
// 64 rows of 4096 to 4096 in bf16: 13 us, 33.5 MB of W at 2.6 TB/s beside x again for each block (134 MB from L2); tiles of 64 x 64 take 27 there.
template <typename T, int NB, int D>
__global__ __launch_bounds__(512) void few_kernel(const Wide<T> p)
{
    constexpr int NW = 8;
    __shared__ __attribute__((aligned(128))) unsigned char lds[NW][(NB + 1) * 2048];
    __shared__ int row_of[NB * 16], id_of[NB * 16];
    __shared__ __attribute__((aligned(16))) float red[NW][NB * 16][20];
    const Rows& q = p.q;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4, p0 = blockIdx.x % p.tiles_n * (NB * 16), o0 = blockIdx.x / p.tiles_n * 16;
    if (threadIdx.x < NB * 16) {
        int id = -2, row = -1;
        if (p0 + (int)threadIdx.x < q.count) row = q.row(p0 + threadIdx.x, &id);
        row_of[threadIdx.x] = row;
        id_of[threadIdx.x] = id;
    }
    __syncthreads();
    // this lane's outputs and the first sixteen of their rows of B_a, which are on their way while the projection is multiplied
    constexpr int PER = (NB * 256 + 511) / 512;
    Operand<T> early[PER][2];
    int n[PER], a[PER];
    const int o = o0 + (threadIdx.x & 15);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        n[i] = (threadIdx.x >> 4) + i * 32;
        a[i] = n[i] < NB * 16 ? id_of[n[i]] : -2;
        if (a[i] < 0) continue;
        const T* b = p.b + ((size_t)a[i] * p.N + min(o, p.N - 1)) * q.rank;
        if (q.rank >= 8) {
            early[i][0].load(b, 0, q.rank);
            early[i][1].load(b, 8, q.rank);
        } else early[i][0].load_any(b, 0, q.rank);
    }
    f32x4 acc[1][NB] = {};
    wave_product<T, 1, NB, D, NW, false>(p.w, [&](int i) { return min(o0 + i * 8 + (lane >> 3), p.N - 1); }, p.x, [&](int i) { return max(row_of[i * 8 + (lane >> 3)], 0); }, p.K,
                                         wave, lds[wave], p.drop, 0, acc);
#pragma unroll
    for (int j = 0; j < NB; ++j) *reinterpret_cast<f32x4*>(&red[wave][j * 16 + l16][g * 4]) = acc[0][j];
    float part[PER] = {};
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (a[i] < 0) continue;
        const T* b = p.b + ((size_t)a[i] * p.N + min(o, p.N - 1)) * q.rank;
        const float* t = p.t + (size_t)row_of[n[i]] * q.rank;
        for (int r = 0; r < q.rank; r += 8) {
            Operand<T> v = early[i][0];
            Operand<float> f;
            if (q.rank >= 8) {
                if (r == 8) v = early[i][1];
                if (r > 8) v.load(b, r, q.rank);
                f.load(t, r, q.rank);
                if (r + 8 > q.rank) {
                    v.settle(r, q.rank);
                    f.settle(r, q.rank);
                }
            } else f.load_any(t, r, q.rank);
            float e[8], d[8];
            v.values(e);
            f.values(d);
#pragma unroll
            for (int c = 0; c < 8; ++c) part[i] = __builtin_fmaf(e[c], d[c], part[i]);
        }
    }
    __syncthreads();
    const uint64_t place = p.drop.border ? drop_place(p.drop) : 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (a[i] < -1 || o >= p.N) continue;
        const size_t at = (size_t)row_of[n[i]] * p.N + o;
        if (p.drop.border && a[i] >= 0) part[i] = kept8(p.drop, place, at >> 3) >> (at & 7) & 1 ? part[i] * p.drop.scale : 0.f;
        float sum = red[0][n[i]][threadIdx.x & 15];
#pragma unroll
        for (int w = 1; w < NW; ++w) sum += red[w][n[i]][threadIdx.x & 15];
        Store<T>::st(p.y + at, sum + (p.bias ? p.bias[o] : 0.f) + part[i]);
    }
}

// ---- sums over the rows of an adapter: out[a][r][c] (or [a][c][r]) = sum f[row][r] drop(v[row][c]) ---------------------------------------------------
// A workgroup takes `length` positions, 512 bytes of columns (a quarter of them a wave) and up to 64 of the rank, and the adapters among those positions one after the
// other: a segment each.  Both operands are contracted over rows, so they go through LDS, 32 rows at a time: bf16 is read from there transposed, f cut into three pieces
// (all its bits: the sums are fp32).  A segment that is all of its adapter is the result; others are partial sums, that of chunk k and adapter a in slot k + a (one of the
// two grows from a segment to the next), added in their order after.
// 8192 rows of 4096 + 4096 columns in bf16, rank 16: 62-70 us for 134 MB, bound by the vector instructions that draw x's mask (58 and 44 without it, before lower pieces met infinities as numbers) and move both operands through LDS.
struct Sum {
    const void* v;
    const float* f;
    int C, ranks_last;           // ranks_last: out[a][c][r]
    Drop drop;                   // (of the first part)
    uint8_t* bits;               // which elements of v's rows were kept, a bit each, for the wide product (C % 8 == 0), or NULL
    float *out, *partial;        // partial: [slot][rank][C] in the order of out
};
struct Sums {                    // of x and of dy, in one launch
    Sum part[2];
    int length, blocks;          // blocks of columns of the first part
};
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
// Of a block of 4 rows x 16 columns of 16 bits, whose lane i of 16 names the address of four elements (row i / 4, columns 4 (i % 4) ..): column i's four rows
__device__ __forceinline__ u32x2 read_transposed(const unsigned char* p)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
#else
    return u32x2{};
#endif
}

template <typename T, int RB>
__global__ __launch_bounds__(256, RB == 1 ? 4 : 1) void sums_kernel(const Rows q, const Sums both)
{
    constexpr bool BF = sizeof(T) == 2;
    constexpr int UNITS = 512 / (8 * sizeof(T)), PER = 32 * UNITS / 256, CB = 512 / sizeof(T) / 64, FB = 32 * RB * 16, F_PER = FB / 256, WINDOW = 256;
    __shared__ __attribute__((aligned(128))) unsigned char xt[2][32 * 512];
    __shared__ __attribute__((aligned(128))) unsigned char ft[2][FB * (BF ? 6 : 4)];          // bf16: upper pieces, then middle and lower ones
    __shared__ int rows_of[WINDOW];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
    const bool second = (int)blockIdx.x >= both.blocks;
    auto of = [&](auto field) { return second ? both.part[1].*field : both.part[0].*field; };
    Sum s;
    s.C = of(&Sum::C); s.ranks_last = of(&Sum::ranks_last); s.bits = of(&Sum::bits); s.out = of(&Sum::out); s.partial = of(&Sum::partial);
    const T* const __restrict__ v = (const T*)of(&Sum::v);
    const float* const __restrict__ f = of(&Sum::f);
    Drop drop = both.part[0].drop;           // (dy is not dropped)
    if (second) drop.border = 0;
    const int c0 = (blockIdx.x - ((int)blockIdx.x >= both.blocks ? both.blocks : 0)) * (512 / (int)sizeof(T)), chunk = blockIdx.y, p0 = chunk * both.length;
    const int p1 = min(p0 + both.length, q.count), r0 = blockIdx.z * 64;
    const uint64_t place = drop.border ? drop_place(drop) : 0;
    const float scale = drop.border ? drop.scale : 1.f;
    // 32-byte pieces of a row lie in the order piece ^ turn(row), so that the rows that one read takes do not meet in a bank
    auto turn = [](int row) { return ((row & 3) | ((row >> 1) & 4)) << (BF ? 0 : 1); };
    Operand<T> held[PER];
    unsigned kept[PER];
    float heldf[F_PER];
    auto fetch = [&](int st) {               // (masks are drawn while the loads are on their way)
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = threadIdx.x + i * 256, row = rows_of[st * 32 + e / UNITS], c = c0 + (e % UNITS) * 8;
            const T* from = v + (size_t)max(row, 0) * s.C;
            if (s.C >= 8) held[i].load(from, c, s.C);
            else held[i].load_any(from, c, s.C);
        }
#pragma unroll
        for (int i = 0; i < F_PER; ++i) {
            const int at = threadIdx.x + i * 256, row = rows_of[st * 32 + at / (RB * 16)], r = r0 + at % (RB * 16);
            const float e = f[(size_t)max(row, 0) * q.rank + min(r, q.rank - 1)];
            heldf[i] = row >= 0 && r < q.rank ? e : 0.f;
        }
        if (drop.border) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = threadIdx.x + i * 256, row = rows_of[st * 32 + e / UNITS], c = c0 + (e % UNITS) * 8;
                kept[i] = kept8_from(drop, place, (uint64_t)((size_t)max(row, 0) * s.C + c));
                if (s.bits && r0 == 0 && row >= 0 && c < s.C) s.bits[((size_t)row * s.C + c) >> 3] = (uint8_t)kept[i];
            }
        }
    };
    auto put = [&](int st, int to) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = threadIdx.x + i * 256, r = e / UNITS, u = e % UNITS;
            if (s.C >= 8 && c0 + 512 / (int)sizeof(T) > s.C) held[i].settle(c0 + u * 8, s.C);
            if (rows_of[st * 32 + r] < 0) held[i].clear();
            if (drop.border) held[i].keep(kept[i]);
            unsigned char* at = xt[to] + r * 512;
            if constexpr (BF) *reinterpret_cast<u32x4*>(at + ((u >> 1) ^ turn(r)) * 32 + (u & 1) * 16) = held[i].v;
            else {
                *reinterpret_cast<f32x4*>(at + (u ^ turn(r)) * 32) = held[i].v[0];
                *reinterpret_cast<f32x4*>(at + (u ^ turn(r)) * 32 + 16) = held[i].v[1];
            }
        }
#pragma unroll
        for (int i = 0; i < F_PER; ++i) {
            const int e = threadIdx.x + i * 256;
            if constexpr (BF) {
                float rest = heldf[i];
#pragma unroll
                for (int third = 0; third < 3; ++third) reinterpret_cast<uint16_t*>(ft[to])[third * FB + e] = cut(rest);
            } else reinterpret_cast<float*>(ft[to])[e] = heldf[i];
        }
    };
    for (int p = p0; p < p1;) {
        int a;
        q.row(p, &a);
        if (a < 0) break;
        const long long begin = (long long)q.starts[a] * q.hw, finish = (long long)q.starts[a + 1] * q.hw;
        const int end = (int)min((long long)p1, finish);
        f32x4 acc[RB][CB] = {};
        for (int base = p; base < end; base += WINDOW) {
            const int n = min(WINDOW, end - base), steps = (n + 31) / 32;
            __syncthreads();
            int id;
            rows_of[threadIdx.x] = (int)threadIdx.x < n ? q.row(base + threadIdx.x, &id) : -1;
            __syncthreads();
            fetch(0);
            put(0, 0);
            __syncthreads();
            for (int st = 0; st < steps; ++st) {
                if (st + 1 < steps) fetch(st + 1);
                const unsigned char *x = xt[st & 1], *fs = ft[st & 1];
                if constexpr (BF) {
                    const int row = 8 * g + (l16 >> 2), fx = (l16 >> 2) | ((g & 1) << 2);
                    u32x4 b[CB];
#pragma unroll
                    for (int j = 0; j < CB; ++j) {
                        const unsigned char* at = x + row * 512 + (((wave * CB + j) ^ fx) << 5) + (l16 & 3) * 8;
                        const u32x2 lo = read_transposed(at), hi = read_transposed(at + 4 * 512);
                        b[j] = u32x4{lo[0], lo[1], hi[0], hi[1]};
                    }
#pragma unroll
                    for (int third = 0; third < 3; ++third) {
                        if (third == 1) {
#pragma unroll
                            for (int j = 0; j < CB; ++j) b[j] = finite8(b[j]);
                        }
#pragma unroll
                        for (int i = 0; i < RB; ++i) {
                            const unsigned char* at = fs + third * FB * 2 + row * (RB * 32) + i * 32 + (l16 & 3) * 8;
                            const u32x2 lo = read_transposed(at), hi = read_transposed(at + 4 * RB * 32);
                            const u32x4 w = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
                            for (int j = 0; j < CB; ++j) acc[i][j] = mfma(w, b[j], acc[i][j]);
                        }
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int row = 4 * k + g, fx = (g | ((k << 1) & 4)) << 1;
                        float b[CB];
#pragma unroll
                        for (int j = 0; j < CB; ++j) b[j] = *reinterpret_cast<const float*>(x + row * 512 + ((((wave * CB + j) * 2 + (l16 >> 3)) ^ fx) << 5) + (l16 & 7) * 4);
#pragma unroll
                        for (int i = 0; i < RB; ++i) {
                            const float w = reinterpret_cast<const float*>(fs)[row * (RB * 16) + i * 16 + l16];
#pragma unroll
                            for (int j = 0; j < CB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w, b[j], acc[i][j], 0, 0, 0);
                        }
                    }
                }
                if (st + 1 < steps) put(st + 1, (st + 1) & 1);
                __syncthreads();
            }
        }
        const bool all = begin == p && finish == end;
        float* out = all ? s.out + (size_t)a * q.rank * s.C : s.partial + (size_t)(chunk + a) * q.rank * s.C;
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int j = 0; j < CB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = r0 + i * 16 + g * 4 + e, c = c0 + (wave * CB + j) * 16 + l16;
                    if (r < q.rank && c < s.C) out[s.ranks_last ? (size_t)c * q.rank + r : (size_t)r * s.C + c] = acc[i][j][e] * scale;
                }
        p = end;
    }
}
// Adapters whose rows lie in several chunks, and zeros for those without rows: `groups` workgroups for each adapter of each part
__global__ __launch_bounds__(256) void join_kernel(const Rows q, const Sums both, int groups)
{
    const Sum& s = both.part[blockIdx.y];
    if (!s.out) return;
    const int a = blockIdx.x / groups, group = blockIdx.x - a * groups;
    const long long begin = (long long)q.starts[a] * q.hw, end = (long long)q.starts[a + 1] * q.hw;
    const int first = (int)(begin / both.length), last = (int)((end - 1) / both.length);
    if (end > begin && first == last) return;
    const size_t count = (size_t)q.rank * s.C;
    for (size_t i = (group * 256u + threadIdx.x) * 4; i < count; i += groups * 1024u) {
        float sum[4] = {};
        const int n = (int)min(count - i, (size_t)4);
        if (end > begin && n == 4) {
#pragma unroll 8
            for (int k = first; k <= last; ++k) {
                const f32x4 v = *reinterpret_cast<const f32x4_any*>(s.partial + (size_t)(k + a) * count + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += v[e];
            }
        } else if (end > begin)
            for (int k = first; k <= last; ++k)
                for (int e = 0; e < n; ++e) sum[e] += s.partial[(size_t)(k + a) * count + i + e];
        if (n == 4) store4(s.out + a * count + i, sum);
        else
            for (int e = 0; e < n; ++e) s.out[a * count + i + e] = sum[e];
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------------------------------
template <typename T>
void narrow(const Rows& q, const void* v, int K, const void* m, const Drop& drop, float* out, hipStream_t st)
{
    if (!q.count) return;
    const int tiles = (q.count + 15) / 16;
    auto launch = [&](auto kernel, int waves, int slots) { hipLaunchKernelGGL(kernel, dim3(tiles, slots), dim3(waves * 64), 0, st, q, (const T*)v, K, (const T*)m, drop, out); };
    // few rows: each of a tile's adapters in a workgroup of its own, while there are compute units (maps of five adapters, 232 tiles: 6.3 us with 2, 8.5 with 5)
    const int slots = tiles < 256 ? std::max(1, std::min({16, q.adapters, (255 + tiles) / tiles})) : 1;
    auto run = [&](auto masked) {
        constexpr bool DROP = decltype(masked)::value;
        if (q.rank <= 16) launch(narrow_kernel<T, 1, 8, 4, DROP>, 8, slots);
        else if (q.rank <= 32) launch(narrow_kernel<T, 2, 8, 3, DROP>, 8, slots);
        else if (q.rank <= 64) launch(narrow_kernel<T, 4, 8, 2, DROP>, 8, slots);
        else launch(narrow_kernel<T, 8, 4, 1, DROP>, 4, slots);
    };
    drop.border ? run(std::true_type()) : run(std::false_type());
}

template <typename T>
void wide(const Rows& q, const void* x, int K, const void* w, const float* bias, const float* t, const void* b, int N, const Drop& drop, const uint8_t* bits,
          void* y, hipStream_t st)
{
    if (!q.count) return;
    Wide<T> p;
    p.bits = bits;
    p.q = q; p.x = (const T*)x; p.w = (const T*)w; p.b = (const T*)b; p.bias = bias; p.t = t; p.K = K; p.N = N; p.drop = drop; p.y = (T*)y;
    auto tiles = [&](int tm, int tn) {
        p.tiles_n = (q.count + tn - 1) / tn;
        p.tiles = p.tiles_n * ((N + tm - 1) / tm);
        return p.tiles;
    };
    const int cus = device_cus();
    // fewer tiles of 64 x 64 than half the compute units: blocks of 16 outputs (128 rows of 1024 to 1000 in fp32 25 -> 13 us; 64 rows of 4096 to 4096 in bf16 27 -> 13;
    // 128 rows of 4096 to 4096, 128 tiles, 21 in tiles and 2 x 13 so)
    if (tiles(64, 64) < cus / 2) {
        if (q.count <= 16) { tiles(16, 16); hipLaunchKernelGGL((few_kernel<T, 1, 4>), dim3(p.tiles), dim3(512), 0, st, p); }
        else if (q.count <= 32) { tiles(16, 32); hipLaunchKernelGGL((few_kernel<T, 2, 3>), dim3(p.tiles), dim3(512), 0, st, p); }
        else { tiles(16, 64); hipLaunchKernelGGL((few_kernel<T, 4, 2>), dim3(p.tiles), dim3(512), 0, st, p); }
        return;
    }
    const bool dma = aligned16(x) && aligned16(w) && K * sizeof(T) % 16 == 0 && (size_t)std::max(q.count, N) * K * sizeof(T) <= NOWHERE && (size_t)K * sizeof(T) < 0x7FFFFF00u;
    auto run = [&](auto dma, auto masked) {
        constexpr bool DMA = decltype(dma)::value;
        constexpr int DROP = decltype(masked)::value;
        if (tiles(256, 256) >= cus) hipLaunchKernelGGL((tiled_kernel<T, 2, 4, 4, 2, 8, 2, DMA, DROP>), dim3(p.tiles), dim3(512), 0, st, p);
        else if (tiles(128, 128) >= cus) hipLaunchKernelGGL((tiled_kernel<T, 2, 2, 2, 2, 8, 2, DMA, DROP>), dim3(p.tiles), dim3(256), 0, st, p);
        else if (tiles(64, 64)) hipLaunchKernelGGL((tiled_kernel<T, 2, 2, 1, 1, 8, 4, DMA, DROP>), dim3(p.tiles), dim3(256), 0, st, p);
    };
    auto run_masked = [&](auto masked) { dma ? run(std::true_type(), masked) : run(std::false_type(), masked); };
    if (!drop.border) run_masked(std::integral_constant<int, NO_MASK>());
    else if (bits) run_masked(std::integral_constant<int, MASK_BITS>());
    else run_masked(std::integral_constant<int, MASK_DRAWN>());
}

constexpr int columns_of(int dtype) { return 512 / (dtype == DR_BF16 ? 2 : 4); }
// The sums over rows: positions come in chunks, at most as many as give each compute unit four workgroups (512, as there are two blocks of columns or more), of 32 positions
// and more.  A chunk's length is a whole number of 32, so a few rows more can make fewer chunks: scratch is for the most that any batch up to this one has.
int most_chunks(const AdapterShape& p)
{
    const int per = columns_of(p.dtype), blocks = (p.in + per - 1) / per + (p.out + per - 1) / per;
    return std::max(1, 1024 / blocks);
}
int length_of(const AdapterShape& p)
{
    const int rows = p.images * p.hw, chunks = most_chunks(p);
    return (int)align_up(std::max((rows + chunks - 1) / chunks, 1), 32);
}
size_t slots_of(const AdapterShape& p)
{
    const int rows = p.images * p.hw;
    return (size_t)std::min(most_chunks(p), (rows + 31) / 32) + p.adapters;
}

template <typename T>
void sum_rows(const Rows& q, const Sums& s, hipStream_t st)
{
    constexpr int COLUMNS = 512 / sizeof(T);
    auto blocks = [&](int i) { return s.part[i].out ? (s.part[i].C + COLUMNS - 1) / COLUMNS : 0; };
    const dim3 grid(blocks(0) + blocks(1), (q.count + s.length - 1) / s.length, (q.rank + 63) / 64);
    if (q.count) {
        if (q.rank <= 16) hipLaunchKernelGGL((sums_kernel<T, 1>), grid, dim3(256), 0, st, q, s);
        else if (q.rank <= 32) hipLaunchKernelGGL((sums_kernel<T, 2>), grid, dim3(256), 0, st, q, s);
        else hipLaunchKernelGGL((sums_kernel<T, 4>), grid, dim3(256), 0, st, q, s);
    }
    const int groups = (int)std::min<size_t>(64, ((size_t)q.rank * std::max(s.part[0].C, s.part[1].C) + 1023) / 1024);
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)(q.adapters * groups), 2), dim3(256), 0, st, q, s, groups);
}

struct Scratch {                 // places in the workspace
    size_t order, starts, inner, wt, at, bt, partial[2], bits, bytes;
};
Scratch scratch_of(const AdapterShape& p, bool backward)
{
    Scratch s = {};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += align_up(bytes, 256); return here; };
    const size_t el = elem_size(p.dtype), factors = (size_t)p.adapters * p.rank, rows = (size_t)p.images * p.hw;
    s.order = take((size_t)p.images * 4);
    s.starts = take(((size_t)p.adapters + 2) * 4);
    s.inner = take(rows * p.rank * 4);
    if (backward) {
        s.wt = take((size_t)p.in * p.out * el);
        s.at = take(factors * p.in * el);
        s.bt = take(factors * p.out * el);
        s.partial[0] = take((size_t)p.rank * slots_of(p) * p.in * 4);
        s.partial[1] = take((size_t)p.rank * slots_of(p) * p.out * 4);
        s.bits = take(p.in % 8 == 0 ? rows * p.in / 8 + 64 : 0);         // (words that begin in the last row's bytes)
    }
    s.bytes = at;
    return s;
}

Rows rows_of(const AdapterShape& p, const AdapterArgs& g, char* ws, const Scratch& s, bool sorted)
{
    Rows q;
    q.count = p.images * p.hw; q.hw = p.hw; q.adapters = p.adapters; q.rank = p.rank;
    q.ids = p.adapters ? g.ids : nullptr; q.scales = g.scales;
    q.order = sorted ? (const int*)(ws + s.order) : nullptr;
    q.starts = (const int*)(ws + s.starts);
    return q;
}

Prepare ordering(const AdapterShape& p, const AdapterArgs& g, char* ws, const Scratch& s)
{
    Prepare r = {};
    r.ids = g.ids; r.n = p.images; r.adapters = p.adapters; r.orders = p.adapters + 1;
    r.order = (int*)(ws + s.order); r.starts = (int*)(ws + s.starts);
    for (Copy& c : r.copy) c.first = c.last = r.orders;
    return r;
}
template <typename T>
void prepare(const Prepare& r, hipStream_t st)
{
    if (r.copy[2].last) hipLaunchKernelGGL((prepare_kernel<T>), dim3(r.copy[2].last), dim3(256), 0, st, r);
}

template <typename T>
void forward(const AdapterShape& p, const AdapterArgs& g, const void* x, void* y, float* inner, const Drop& drop, char* ws, hipStream_t st)
{
    const Scratch s = scratch_of(p, false);
    // few images, or images as long as a tile: as they come (a tile then holds few adapters, and the order's launch is 4-8 us)
    const bool sorted = p.images > 64 && p.hw < 64 && p.adapters > 1;
    if (sorted) prepare<T>(ordering(p, g, ws, s), st);
    const Rows q = rows_of(p, g, ws, s, sorted);
    float* t = inner ? inner : (float*)(ws + s.inner);
    if (p.adapters || inner) narrow<T>(q, x, p.in, g.a, drop, t, st);
    wide<T>(q, x, p.in, g.w, g.bias, t, g.b, p.out, make_drop(0.f, 0, 0, nullptr), nullptr, y, st);
}

template <typename T>
void backward(const AdapterShape& p, const AdapterArgs& g, const void* dy, const void* x, const float* inner, void* dx, float* da, float* db, const Drop& drop, char* ws,
              hipStream_t st)
{
    const Scratch s = scratch_of(p, true);
    const Drop none = make_drop(0.f, 0, 0, nullptr);
    Prepare r = ordering(p, g, ws, s);
    if (!p.adapters) r.orders = 0;
    int copies = 0, first = r.orders;
    for (Copy& c : r.copy) c.first = c.last = first;
    auto copy = [&](const void* src, size_t dst, int batch, int R, int C) {
        Copy& c = r.copy[copies++];
        c.src = src; c.dst = ws + dst; c.R = R; c.C = C;
        c.tiles_r = (R + 63) / 64; c.tiles_c = (C + 63) / 64;
        c.first = first;
        for (int i = copies - 1; i < 3; ++i) r.copy[i].last = first + batch * c.tiles_r * c.tiles_c;
        first = c.last;
    };
    if (p.images) {
        if (p.adapters && (dx || da)) copy(g.b, s.bt, p.adapters, p.out, p.rank);
        if (dx) copy(g.w, s.wt, 1, p.out, p.in);
        if (p.adapters && dx) copy(g.a, s.at, p.adapters, p.rank, p.in);
    }
    prepare<T>(r, st);
    const Rows q = rows_of(p, g, ws, s, p.adapters > 0);
    float* u = (float*)(ws + s.inner);
    if (p.adapters && (dx || da)) narrow<T>(q, dy, p.out, ws + s.bt, none, u, st);
    uint8_t* bits = drop.border && p.adapters && da && dx && p.in % 8 == 0 ? (uint8_t*)(ws + s.bits) : nullptr;
    if (p.adapters && (da || db)) {
        Sums both = {};
        both.part[0] = Sum{x, u, p.in, 0, drop, bits, da, (float*)(ws + s.partial[0])};
        both.part[1] = Sum{dy, inner, p.out, 1, none, nullptr, db, (float*)(ws + s.partial[1])};
        both.length = length_of(p);
        both.blocks = da ? (p.in + columns_of(p.dtype) - 1) / columns_of(p.dtype) : 0;
        sum_rows<T>(q, both, st);
    }
    if (dx) wide<T>(q, dy, p.out, ws + s.wt, nullptr, u, ws + s.at, p.in, drop, bits, dx, st);
}

long long product_bytes(const AdapterShape& p, bool backward)
{
    const size_t rows = (size_t)p.images * p.hw;
    return (long long)((rows * (p.in * (backward ? 2 : 1) + p.out) + (size_t)p.in * p.out + (size_t)p.adapters * p.rank * (p.in + p.out)) * elem_size(p.dtype));
}

}  // namespace

size_t adapter_workspace_bytes(const AdapterShape& p, bool backward) { return scratch_of(p, backward).bytes; }

int launch_adapter_fwd(const AdapterShape& p, const AdapterArgs& g, const void* x, void* y, float* inner, const Drop& drop, void* ws, hipStream_t st)
{
    TraceScope trace("adapter", nullptr, (long long)p.images * p.hw, st, product_bytes(p, false));
    if (p.dtype == DR_BF16) forward<uint16_t>(p, g, x, y, inner, drop, (char*)ws, st);
    else forward<float>(p, g, x, y, inner, drop, (char*)ws, st);
    return check_launch("adapter");
}

int launch_adapter_bwd(const AdapterShape& p, const AdapterArgs& g, const void* dy, const void* x, const float* inner, void* dx, float* da, float* db, const Drop& drop,
                       void* ws, hipStream_t st)
{
    TraceScope trace("adapter_bwd", nullptr, (long long)p.images * p.hw, st, product_bytes(p, true));
    if (p.dtype == DR_BF16) backward<uint16_t>(p, g, dy, x, inner, dx, da, db, drop, (char*)ws, st);
    else backward<float>(p, g, dy, x, inner, dx, da, db, drop, (char*)ws, st);
    return check_launch("adapter_bwd");
}

}  // namespace dr
