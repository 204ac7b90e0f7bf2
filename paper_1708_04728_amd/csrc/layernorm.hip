// Layer normalisation over the channels of every pixel, and its gradient (dr_layernorm_fwd, dr_layernorm_bwd).
//
//   forward    y = gamma (x - mean) rstd + beta [, max(., 0)],  mean = sum_c x / C,  rstd = 1 / sqrt(sum_c (x - mean)^2 / C + eps)
//   gradient   with g = dy gamma and z = (x - mean) rstd:
//              dx = rstd (g - sum_c g / C - z sum_c (g z) / C),  dgamma_c = sum over pixels of dy z,  dbeta_c = sum over pixels of dy
//
// The variance is the mean square of differences from the mean, not a difference of squares: a pixel's values may lie far from zero.  Squares are added divided by a
// power of two near C, so that their sum is no infinity where the variance is a number.
#include <algorithm>
#include <type_traits>

#include "dr_internal.h"
#include "dr_store.h"

namespace dr {
namespace {

// Element (pixel, c) of a tensor: base(pixel) + c * step
struct Pixels {
    size_t count;          // pixels
    int C, HW;
    bool planes;           // NCHW
    __device__ __forceinline__ size_t base(size_t p) const
    {
        if (!planes) return p * C;
        const size_t img = p / HW;
        return img * C * HW + (p - img * HW);
    }
    __device__ __forceinline__ size_t step() const { return planes ? (size_t)HW : 1; }
};

// 2^-k <= 1 / C
__device__ __forceinline__ float square_scale(int C) { return __uint_as_float((unsigned)(127 - (C > 1 ? 32 - __clz(C - 1) : 0)) << 23); }

// sum over the 256 threads of a workgroup, the same value in every thread
__device__ __forceinline__ float block_sum(float v, float* red)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// ---- any tensor: a workgroup per pixel, its channels read once for each sum
template <typename T>
__global__ __launch_bounds__(256) void norm_any_kernel(const Pixels px, const T* x, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                       float eps, int relu, T* y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    __shared__ float red[4];
    const size_t step = px.step();
    const float down = square_scale(px.C);
    for (size_t p = blockIdx.x; p < px.count; p += gridDim.x) {
        const size_t at = px.base(p);
        float s = 0.f;
        for (int c = threadIdx.x; c < px.C; c += 256) s += Store<T>::ld(x + at + c * step);
        const float mean = block_sum(s, red) / (float)px.C;
        s = 0.f;
        for (int c = threadIdx.x; c < px.C; c += 256) {
            const float d = Store<T>::ld(x + at + c * step) - mean;
            s = __builtin_fmaf(d * down, d, s);
        }
        const float rstd = 1.f / sqrtf(block_sum(s, red) / ((float)px.C * down) + eps);
        for (int c = threadIdx.x; c < px.C; c += 256) {
            float v = (Store<T>::ld(x + at + c * step) - mean) * rstd;
            v = v * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f);
            Store<T>::st(y + at + c * step, relu ? fmaxf(v, 0.f) : v);
        }
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[p] = mean;
            if (rstd_out) rstd_out[p] = rstd;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void norm_grad_any_kernel(const Pixels px, const T* dy, const T* x, const float* __restrict__ gamma,
                                                            const float* __restrict__ mean, const float* __restrict__ rstd, T* dx)
{
    __shared__ float red[4];
    const size_t step = px.step();
    for (size_t p = blockIdx.x; p < px.count; p += gridDim.x) {
        const size_t at = px.base(p);
        const float mu = mean[p], r = rstd[p];
        float s = 0.f, t = 0.f;
        for (int c = threadIdx.x; c < px.C; c += 256) {
            const float g = Store<T>::ld(dy + at + c * step) * (gamma ? gamma[c] : 1.f);
            s += g;
            t += g * ((Store<T>::ld(x + at + c * step) - mu) * r);
        }
        s = block_sum(s, red) / (float)px.C;
        t = block_sum(t, red) / (float)px.C;
        for (int c = threadIdx.x; c < px.C; c += 256) {
            const float g = Store<T>::ld(dy + at + c * step) * (gamma ? gamma[c] : 1.f), z = (Store<T>::ld(x + at + c * step) - mu) * r;
            Store<T>::st(dx + at + c * step, r * (g - s - z * t));
        }
    }
}

// Partial sums of the vectors' gradients: workgroup (i, j) adds the pixels of range j for channels 64 i .. 64 i + 63, partial[j][2][C]
template <typename T>
__global__ __launch_bounds__(256) void norm_vectors_any_kernel(const Pixels px, const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ mean,
                                                               const float* __restrict__ rstd, float* __restrict__ partial)
{
    __shared__ float red[2][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    const size_t lo = px.count * blockIdx.y / gridDim.y, hi = px.count * (blockIdx.y + 1) / gridDim.y;
    float dg = 0.f, db = 0.f;
    if (c < px.C)
        for (size_t p = lo + wave; p < hi; p += 4) {
            const size_t at = px.base(p) + c * px.step();
            const float d = Store<T>::ld(dy + at);
            db += d;
            dg += d * ((Store<T>::ld(x + at) - mean[p]) * rstd[p]);
        }
    red[0][wave][lane] = dg;
    red[1][wave][lane] = db;
    __syncthreads();
    if (wave < 2 && c < px.C) {
        const float (*r)[64] = red[wave];
        partial[((size_t)blockIdx.y * 2 + wave) * px.C + c] = (r[0][lane] + r[1][lane]) + (r[2][lane] + r[3][lane]);
    }
}

// dgamma and dbeta from the partial sums of `ranges` ranges of pixels, in a fixed order, in double
__global__ __launch_bounds__(256) void norm_vectors_sum_kernel(const float* __restrict__ partial, int ranges, int C, float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ double red[16][16];
    const int col = blockIdx.x * 16 + (threadIdx.x & 15), row = threadIdx.x >> 4;
    double s = 0.0;
    if (col < 2 * C) {
#pragma unroll 4
        for (int r = row; r < ranges; r += 16) s += (double)partial[(size_t)r * 2 * C + col];
    }
    red[row][threadIdx.x & 15] = s;
    __syncthreads();
    if (threadIdx.x < 16 && col < 2 * C) {
        s = 0.0;
        for (int r = 0; r < 16; ++r) s += red[r][threadIdx.x];
        if (col < C) { if (dgamma) dgamma[col] = (float)s; }
        else if (dbeta) dbeta[col - C] = (float)s;
    }
}

// ---- sums over lanes
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) { return v + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true)); }

// over groups of G lanes (a power of two), the same value in every lane of a group
template <int G>
__device__ __forceinline__ float lanes_sum(float v)
{
    if constexpr (G >= 2) v = add_dpp<0xB1>(v);         // lanes 1 0 3 2
    if constexpr (G >= 4) v = add_dpp<0x4E>(v);         // lanes 2 3 0 1
    if constexpr (G >= 8) v = add_dpp<0x141>(v);        // eight, mirrored
    if constexpr (G >= 16) v = add_dpp<0x140>(v);       // sixteen, mirrored
    if constexpr (G >= 32) {
        const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(t[0]) + __uint_as_float(t[1]);
    }
    if constexpr (G >= 64) {
        const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(t[0]) + __uint_as_float(t[1]);
    }
    return v;
}

// ---- channels last, 16-byte aligned rows of a multiple of 16 bytes: a row in the registers of G lanes, NV vectors of 16 bytes each.  G > 64: G / 64 waves.
// The workgroup's THREADS / G groups walk the rows together.
template <typename T>
__device__ __forceinline__ void unpack(const uint4& r, float* v)
{
    if constexpr (sizeof(T) == 4) {
        v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
    } else {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

// sums of N values over a group of G lanes; red: LDS of THREADS / 64 x N floats, two of them used in turn
template <int G, int THREADS, int N>
__device__ __forceinline__ void group_sums(float (&v)[N], float (*red)[THREADS / 64][N], int& turn)
{
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = lanes_sum<(G < 64 ? G : 64)>(v[n]);
    if constexpr (G > 64) {
        const int wave = threadIdx.x >> 6, first = wave / (G / 64) * (G / 64);
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n) red[turn][wave][n] = v[n];
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v[n] = 0.f;
#pragma unroll
            for (int w = 0; w < G / 64; ++w) v[n] += red[turn][first + w][n];
        }
        turn ^= 1;
    }
}

template <int VN>
__device__ __forceinline__ void load_vector(const float* p, int at, float other, float* v)
{
#pragma unroll
    for (int e = 0; e < VN; ++e) v[e] = p ? p[at + e] : other;
}

template <typename T, int G, int NV, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_rows_kernel(size_t rows, int C, const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, float eps,
                                                            int relu, T* y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    constexpr int VN = Store<T>::VN, GROUPS = THREADS / G;
    __shared__ float red[2][THREADS / 64][1];
    int turn = 0;
    const int lane = threadIdx.x % G, group = threadIdx.x / G, nvec = C / VN;
    const float down = square_scale(C);
    uint4 next[NV];
    auto fetch = [&](size_t row) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (lane + j * G < nvec && row < rows) next[j] = reinterpret_cast<const uint4*>(x + row * C)[lane + j * G];
    };
    size_t row = (size_t)blockIdx.x * GROUPS + group;
    const size_t stride = (size_t)gridDim.x * GROUPS;
#pragma unroll
    for (int j = 0; j < NV; ++j) next[j] = uint4{0, 0, 0, 0};
    fetch(row);
    float g[NV][VN], b[NV][VN];
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (lane + j * G < nvec) {
            load_vector<VN>(gamma, (lane + j * G) * VN, 1.f, g[j]);
            load_vector<VN>(beta, (lane + j * G) * VN, 0.f, b[j]);
        }
    for (size_t first = (size_t)blockIdx.x * GROUPS; first < rows; first += stride, row += stride) {      // (the same rounds for all lanes)
        float v[NV][VN], s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            unpack<T>(next[j], v[j]);                  // (zero beyond the row)
#pragma unroll
            for (int e = 0; e < VN; ++e) s[0] += v[j][e];
        }
        fetch(row + stride);
        group_sums<G, THREADS, 1>(s, red, turn);
        const float mean = s[0] / (float)C;
        s[0] = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (lane + j * G < nvec) {
#pragma unroll
                for (int e = 0; e < VN; ++e) {
                    v[j][e] -= mean;
                    s[0] = __builtin_fmaf(v[j][e] * down, v[j][e], s[0]);
                }
            }
        group_sums<G, THREADS, 1>(s, red, turn);
        const float rstd = 1.f / sqrtf(s[0] / ((float)C * down) + eps);
        if (row < rows) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (lane + j * G < nvec) {
#pragma unroll
                    for (int e = 0; e < VN; ++e) {
                        const float t = v[j][e] * rstd * g[j][e] + b[j][e];
                        v[j][e] = relu ? fmaxf(t, 0.f) : t;
                    }
                    Store<T>::stv(y + row * C + (size_t)(lane + j * G) * VN, v[j]);
                }
            if (lane == 0) {
                if (mean_out) mean_out[row] = mean;
                if (rstd_out) rstd_out[row] = rstd;
            }
        }
    }
}

// ... and the gradient: every lane adds its columns of dgamma and dbeta over the workgroup's rows; partial[workgroup][2][C]
template <typename T, int G, int NV, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_grad_rows_kernel(size_t rows, int C, const T* dy, const T* x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                                                 const float* __restrict__ rstd, T* dx, float* __restrict__ partial)
{
    constexpr int VN = Store<T>::VN, GROUPS = THREADS / G, IN_WAVE = G < 64 ? 64 / G : 1, TURNS = GROUPS / IN_WAVE;
    __shared__ float red[2][THREADS / 64][2];
    extern __shared__ float columns[];                 // [2][C]
    int turn = 0;
    const int lane = threadIdx.x % G, group = threadIdx.x / G, nvec = C / VN;
    uint4 nx[NV], nd[NV];
    float n_mean = 0.f, n_rstd = 0.f;
    auto fetch = [&](size_t row) __attribute__((always_inline)) {
        if (row >= rows) return;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (lane + j * G < nvec) {
                nd[j] = reinterpret_cast<const uint4*>(dy + row * C)[lane + j * G];
                nx[j] = reinterpret_cast<const uint4*>(x + row * C)[lane + j * G];
            }
        n_mean = mean[row];
        n_rstd = rstd[row];
    };
    size_t row = (size_t)blockIdx.x * GROUPS + group;
    const size_t stride = (size_t)gridDim.x * GROUPS;
#pragma unroll
    for (int j = 0; j < NV; ++j) nx[j] = nd[j] = uint4{0, 0, 0, 0};
    fetch(row);
    float g[NV][VN], dg[NV][VN], db[NV][VN];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int e = 0; e < VN; ++e) dg[j][e] = db[j][e] = g[j][e] = 0.f;
        if (lane + j * G < nvec) load_vector<VN>(gamma, (lane + j * G) * VN, 1.f, g[j]);
    }
    for (size_t first = (size_t)blockIdx.x * GROUPS; first < rows; first += stride, row += stride) {
        float z[NV][VN], d[NV][VN], s[2] = {0.f, 0.f};
        const float mu = n_mean, r = n_rstd;
        const bool on = row < rows;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            unpack<T>(nx[j], z[j]);
            unpack<T>(nd[j], d[j]);
            if (on && lane + j * G < nvec) {
#pragma unroll
                for (int e = 0; e < VN; ++e) {
                    z[j][e] = (z[j][e] - mu) * r;
                    const float u = d[j][e] * g[j][e];
                    s[0] += u;
                    s[1] += u * z[j][e];
                    db[j][e] += d[j][e];
                    dg[j][e] += d[j][e] * z[j][e];
                }
            }
        }
        fetch(row + stride);
        group_sums<G, THREADS, 2>(s, red, turn);
        const float s0 = s[0] / (float)C, s1 = s[1] / (float)C;
        if (dx && on) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (lane + j * G < nvec) {
#pragma unroll
                    for (int e = 0; e < VN; ++e) d[j][e] = r * (d[j][e] * g[j][e] - s0 - z[j][e] * s1);
                    Store<T>::stv(dx + row * C + (size_t)(lane + j * G) * VN, d[j]);
                }
        }
    }
    if (!partial) return;
    // the groups of a wave, then the waves in turn
#pragma unroll
    for (int k = G; k < 64; k *= 2)
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                dg[j][e] += __shfl_xor(dg[j][e], k, 64);
                db[j][e] += __shfl_xor(db[j][e], k, 64);
            }
    for (int t = 0; t < TURNS; ++t) {
        if (group / IN_WAVE == t && group % IN_WAVE == 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (lane + j * G < nvec) {
#pragma unroll
                    for (int e = 0; e < VN; ++e) {
                        const int c = (lane + j * G) * VN + e;
                        columns[c] = t ? columns[c] + dg[j][e] : dg[j][e];
                        columns[C + c] = t ? columns[C + c] + db[j][e] : db[j][e];
                    }
                }
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < 2 * C; i += THREADS) partial[(size_t)blockIdx.x * 2 * C + i] = columns[i];
}

// ---- channels last, any row length and alignment: runs of whole rows go through LDS, fetched and written in aligned 16-byte pieces
// A run's first byte lies (address % 16) into LDS, so that every piece is 16 bytes of memory and of LDS.
template <typename T>
__device__ __forceinline__ int run_in(const T* base, size_t total, size_t at, int count, unsigned char* lds)
{
    const uintptr_t lo = (uintptr_t)base, hi = lo + total * sizeof(T), from = lo + at * sizeof(T), first = from & ~(uintptr_t)15;
    const int shift = (int)(from - first), pieces = (shift + count * (int)sizeof(T) + 15) >> 4;
    for (int i = threadIdx.x; i < pieces; i += 256) {
        const uintptr_t p = first + (uintptr_t)i * 16;
        if (p >= lo && p + 16 <= hi) reinterpret_cast<uint4*>(lds)[i] = *reinterpret_cast<const uint4*>(p);
        else {
#pragma unroll
            for (int e = 0; e < (int)(16 / sizeof(T)); ++e) {
                const uintptr_t q = p + e * sizeof(T);
                if (q >= lo && q < hi) reinterpret_cast<T*>(lds)[i * (16 / sizeof(T)) + e] = *reinterpret_cast<const T*>(q);
            }
        }
    }
    return shift / (int)sizeof(T);
}
template <typename T>
__device__ __forceinline__ void run_out(T* base, size_t at, int count, const unsigned char* lds)      // lds: laid out as for this address
{
    const uintptr_t from = (uintptr_t)(base + at), to = from + (size_t)count * sizeof(T), first = from & ~(uintptr_t)15;
    const int pieces = (int)((to - first + 15) >> 4);
    for (int i = threadIdx.x; i < pieces; i += 256) {
        const uintptr_t p = first + (uintptr_t)i * 16;
        if (p >= from && p + 16 <= to) *reinterpret_cast<uint4*>(p) = reinterpret_cast<const uint4*>(lds)[i];
        else {
#pragma unroll
            for (int e = 0; e < (int)(16 / sizeof(T)); ++e) {
                const uintptr_t q = p + e * sizeof(T);
                if (q >= from && q < to) *reinterpret_cast<T*>(q) = reinterpret_cast<const T*>(lds)[i * (16 / sizeof(T)) + e];
            }
        }
    }
}

constexpr int RUN_BYTES = 16384;         // most bytes of a run (of each tensor)
template <typename T> constexpr int run_bytes() { return RUN_BYTES + 32; }

template <typename T, int G>
__global__ __launch_bounds__(256) void norm_runs_kernel(size_t rows, int C, int run, const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, float eps,
                                                        int relu, T* y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    __shared__ __attribute__((aligned(16))) unsigned char in[run_bytes<T>()], out[run_bytes<T>()];
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    const float down = square_scale(C);
    const size_t runs = (rows + run - 1) / run;
    for (size_t k = blockIdx.x; k < runs; k += gridDim.x) {
        const size_t row0 = k * run;
        const int here = (int)(rows - row0 < (size_t)run ? rows - row0 : (size_t)run);
        const int shift = run_in<T>(x, rows * C, row0 * C, here * C, in);
        const int out_shift = (int)(((uintptr_t)(y + row0 * C) & 15) / sizeof(T));
        __syncthreads();
        for (int r = group; r < here; r += 256 / G) {
            const T* v = reinterpret_cast<const T*>(in) + shift + r * C;
            T* o = reinterpret_cast<T*>(out) + out_shift + r * C;
            float s = 0.f;
            for (int c = lane; c < C; c += G) s += Store<T>::ld(v + c);
            const float mean = lanes_sum<G>(s) / (float)C;
            s = 0.f;
            for (int c = lane; c < C; c += G) {
                const float d = Store<T>::ld(v + c) - mean;
                s = __builtin_fmaf(d * down, d, s);
            }
            const float rstd = 1.f / sqrtf(lanes_sum<G>(s) / ((float)C * down) + eps);
            for (int c = lane; c < C; c += G) {
                const float t = (Store<T>::ld(v + c) - mean) * rstd * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f);
                Store<T>::st(o + c, relu ? fmaxf(t, 0.f) : t);
            }
            if (lane == 0) {
                if (mean_out) mean_out[row0 + r] = mean;
                if (rstd_out) rstd_out[row0 + r] = rstd;
            }
        }
        __syncthreads();
        run_out<T>(y, row0 * C, here * C, out);
        // (the next run's rows are written behind the barrier that follows its fetch)
    }
}

// ... and the gradient: the sums row by row, then column by column (thread t: columns t, t + 256, ...) what needs both
constexpr int RUN_COLUMNS = 8;           // most columns of a thread
template <typename T, int G, int NC>
__global__ __launch_bounds__(256) void norm_grad_runs_kernel(size_t rows, int C, int run, const T* dy, const T* x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, T* dx, float* __restrict__ partial)
{
    __shared__ __attribute__((aligned(16))) unsigned char in_d[run_bytes<T>()], in_x[run_bytes<T>()], out[run_bytes<T>()];
    __shared__ float4 of_row[512];       // mean, rstd, sum g / C, sum g z / C
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    const size_t runs = (rows + run - 1) / run;
    float g[NC], dg[NC], db[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c = threadIdx.x + j * 256;
        g[j] = gamma && c < C ? gamma[c] : 1.f;
        dg[j] = db[j] = 0.f;
    }
    for (size_t k = blockIdx.x; k < runs; k += gridDim.x) {
        const size_t row0 = k * run;
        const int here = (int)(rows - row0 < (size_t)run ? rows - row0 : (size_t)run);
        const int sd = run_in<T>(dy, rows * C, row0 * C, here * C, in_d), sx = run_in<T>(x, rows * C, row0 * C, here * C, in_x);
        const int so = dx ? (int)(((uintptr_t)(dx + row0 * C) & 15) / sizeof(T)) : 0;
        __syncthreads();
        for (int r = group; r < here; r += 256 / G) {
            const T *vd = reinterpret_cast<const T*>(in_d) + sd + r * C, *vx = reinterpret_cast<const T*>(in_x) + sx + r * C;
            const float mu = mean[row0 + r], rs = rstd[row0 + r];
            float s = 0.f, t = 0.f;
            for (int c = lane; c < C; c += G) {
                const float u = Store<T>::ld(vd + c) * (gamma ? gamma[c] : 1.f);
                s += u;
                t += u * ((Store<T>::ld(vx + c) - mu) * rs);
            }
            s = lanes_sum<G>(s) / (float)C;
            t = lanes_sum<G>(t) / (float)C;
            if (lane == 0) of_row[r] = make_float4(mu, rs, s, t);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int c = threadIdx.x + j * 256;
            if (c >= C) break;
            const T *vd = reinterpret_cast<const T*>(in_d) + sd + c, *vx = reinterpret_cast<const T*>(in_x) + sx + c;
            T* o = reinterpret_cast<T*>(out) + so + c;
            for (int r = 0; r < here; ++r) {
                const float4 q = of_row[r];
                const float d = Store<T>::ld(vd + r * C), z = (Store<T>::ld(vx + r * C) - q.x) * q.y;
                db[j] += d;
                dg[j] += d * z;
                if (dx) Store<T>::st(o + r * C, q.y * (d * g[j] - q.z - z * q.w));
            }
        }
        __syncthreads();
        if (dx) run_out<T>(dx, row0 * C, here * C, out);
    }
    if (!partial) return;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c = threadIdx.x + j * 256;
        if (c >= C) break;
        partial[(size_t)blockIdx.x * 2 * C + c] = dg[j];
        partial[(size_t)blockIdx.x * 2 * C + C + c] = db[j];
    }
}

// ---- channel planes: a lane per pixel, 64 pixels a workgroup (of any images), wave w of W takes channels w, w + W, ..., NC of them at most, in registers
template <typename T, int NC, int W>
__global__ __launch_bounds__(W * 64) void norm_planes_kernel(const Pixels px, const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, float eps, int relu,
                                                             T* y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    __shared__ float red[2][W][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), C = px.C;
    const float down = square_scale(C);
    const size_t pixel = (size_t)blockIdx.x * 64 + lane;
    const bool on = pixel < px.count;
    const size_t at = px.base(on ? pixel : px.count - 1), step = px.step();
    float v[NC], s = 0.f;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c = wave + j * W;
        v[j] = c < C ? Store<T>::ld(x + at + c * step) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < NC; ++j) s += v[j];
    auto sum = [&](float mine, int turn) __attribute__((always_inline)) {
        red[turn][wave][lane] = mine;
        __syncthreads();
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) t += red[turn][w][lane];
        return t;
    };
    const float mean = sum(s, 0) / (float)C;
    s = 0.f;
#pragma unroll
    for (int j = 0; j < NC; ++j)
        if (wave + j * W < C) {
            v[j] -= mean;
            s = __builtin_fmaf(v[j] * down, v[j], s);
        }
    const float rstd = 1.f / sqrtf(sum(s, 1) / ((float)C * down) + eps);
    if (!on) return;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c = wave + j * W;
        if (c < C) {
            const float t = v[j] * rstd * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f);
            Store<T>::st(y + at + c * step, relu ? fmaxf(t, 0.f) : t);
        }
    }
    if (wave == 0) {
        if (mean_out) mean_out[pixel] = mean;
        if (rstd_out) rstd_out[pixel] = rstd;
    }
}

// Sums over the 64 lanes of N values each, N a power of two from 4 to 32: every lane gets the sum of value lane * N / 64.  A step hands half of a lane's values to the
// lane it meets and takes the others' in return: about two instructions a value in all, in the place of twelve.
template <int N, int M, int D, int CTRL>
__device__ __forceinline__ void transpose_step(float (&v)[N])      // M values left; lanes meet across bit D
{
    auto met = [](float f) __attribute__((always_inline)) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, f), CTRL, 0xF, 0xF, true)); };
    if constexpr (M > 1) {
        const bool high = (threadIdx.x & D) != 0;
#pragma unroll
        for (int i = 0; i < M / 2; ++i) {
            const float keep = high ? v[i + M / 2] : v[i], give = high ? v[i] : v[i + M / 2];
            v[i] = keep + met(give);
        }
    } else v[0] += met(v[0]);
}
template <int N>
__device__ __forceinline__ float transpose_sum(float (&v)[N])
{
    static_assert(N >= 4 && N <= 32, "values of a lane");
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + N / 2]), false, false);
        v[i] = __uint_as_float(t[0]) + __uint_as_float(t[1]);
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + N / 4]), false, false);
        v[i] = __uint_as_float(t[0]) + __uint_as_float(t[1]);
    }
    constexpr int A = N / 4, B = A > 1 ? A / 2 : 1, C = B > 1 ? B / 2 : 1, D = C > 1 ? C / 2 : 1;
    transpose_step<N, A, 8, 0x128>(v);      // lane +- 8 of sixteen
    transpose_step<N, B, 4, 0x141>(v);      // 7 - lane of eight (a lane's later partners have met the others of the eight)
    transpose_step<N, C, 2, 0x4E>(v);
    transpose_step<N, D, 1, 0xB1>(v);
    return v[0];
}

// The gradient on planes: a workgroup walks groups of 64 pixels; the sums over a group's pixels by transpose_sum, so that a lane holds the running sums of one channel
template <typename T, int NC, int W>
__global__ __launch_bounds__(W * 64) void norm_grad_planes_kernel(const Pixels px, const T* dy, const T* x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                                                  const float* __restrict__ rstd, T* dx, float* __restrict__ partial)
{
    __shared__ float red[2][2][W][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), C = px.C;
    const size_t step = px.step(), groups = (px.count + 63) / 64;
    float dg = 0.f, db = 0.f;
    int turn = 0;
    for (size_t k = blockIdx.x; k < groups; k += gridDim.x, turn ^= 1) {
        const size_t pixel = k * 64 + lane;
        const bool on = pixel < px.count;
        const size_t q = on ? pixel : px.count - 1, at = px.base(q);
        const float mu = mean[q], r = rstd[q];
        float z[NC], d[NC], s = 0.f, t = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int c = wave + j * W;
            d[j] = c < C ? Store<T>::ld(dy + at + c * step) : 0.f;
            z[j] = c < C ? Store<T>::ld(x + at + c * step) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int c = wave + j * W;
            z[j] = c < C ? (z[j] - mu) * r : 0.f;
            const float u = d[j] * (gamma && c < C ? gamma[c] : 1.f);
            s += u;
            t += u * z[j];
        }
        red[turn][0][wave][lane] = s;
        red[turn][1][wave][lane] = t;
        __syncthreads();
        s = t = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            s += red[turn][0][w][lane];
            t += red[turn][1][w][lane];
        }
        s /= (float)C;
        t /= (float)C;
        if (dx && on) {
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const int c = wave + j * W;
                if (c < C) Store<T>::st(dx + at + c * step, r * (d[j] * (gamma ? gamma[c] : 1.f) - s - z[j] * t));
            }
        }
        if (partial) {
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                d[j] = on ? d[j] : 0.f;
                z[j] = on ? d[j] * z[j] : 0.f;
            }
            dg += transpose_sum<NC>(z);
            db += transpose_sum<NC>(d);
        }
    }
    const int c = wave + lane * NC / 64 * W;
    if (partial && lane % (64 / NC) == 0 && c < C) {
        partial[(size_t)blockIdx.x * 2 * C + c] = dg;
        partial[(size_t)blockIdx.x * 2 * C + C + c] = db;
    }
}

// ... of more channels than registers hold: read again for each use (from the caches), CHUNK channels a wave at a time
constexpr int LONG_W = 16, CHUNK = 16;
template <typename T>
__global__ __launch_bounds__(LONG_W * 64) void norm_long_planes_kernel(const Pixels px, const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, float eps,
                                                                       int relu, T* y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    __shared__ float red[2][LONG_W][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), C = px.C;
    const float down = square_scale(C);
    const size_t pixel = (size_t)blockIdx.x * 64 + lane;
    const bool on = pixel < px.count;
    const size_t at = px.base(on ? pixel : px.count - 1), step = px.step();
    auto sum = [&](float mine, int turn) __attribute__((always_inline)) {
        red[turn][wave][lane] = mine;
        __syncthreads();
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < LONG_W; ++w) t += red[turn][w][lane];
        return t;
    };
    auto each = [&](auto f) __attribute__((always_inline)) {
        for (int c0 = wave; c0 < C; c0 += LONG_W * CHUNK) {
            float v[CHUNK];
#pragma unroll
            for (int j = 0; j < CHUNK; ++j) v[j] = c0 + j * LONG_W < C ? Store<T>::ld(x + at + (c0 + j * LONG_W) * step) : 0.f;
#pragma unroll
            for (int j = 0; j < CHUNK; ++j)
                if (c0 + j * LONG_W < C) f(c0 + j * LONG_W, v[j]);
        }
    };
    float s = 0.f;
    each([&](int, float v) { s += v; });
    const float mean = sum(s, 0) / (float)C;
    s = 0.f;
    each([&](int, float v) {
        const float d = v - mean;
        s = __builtin_fmaf(d * down, d, s);
    });
    const float rstd = 1.f / sqrtf(sum(s, 1) / ((float)C * down) + eps);
    each([&](int c, float v) {
        const float t = (v - mean) * rstd * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f);
        if (on) Store<T>::st(y + at + c * step, relu ? fmaxf(t, 0.f) : t);
    });
    if (on && wave == 0) {
        if (mean_out) mean_out[pixel] = mean;
        if (rstd_out) rstd_out[pixel] = rstd;
    }
}

template <typename T>
__global__ __launch_bounds__(LONG_W * 64) void norm_grad_long_planes_kernel(const Pixels px, const T* dy, const T* x, const float* __restrict__ gamma,
                                                                            const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, float* __restrict__ partial)
{
    __shared__ float red[2][2][LONG_W][64];
    extern __shared__ float columns[];       // [2][C]: running sums, each touched by one lane
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), C = px.C;
    const size_t step = px.step(), groups = (px.count + 63) / 64;
    for (int i = threadIdx.x; i < 2 * C; i += LONG_W * 64) columns[i] = 0.f;
    __syncthreads();
    int turn = 0;
    for (size_t k = blockIdx.x; k < groups; k += gridDim.x, turn ^= 1) {
        const size_t pixel = k * 64 + lane;
        const bool on = pixel < px.count;
        const size_t q = on ? pixel : px.count - 1, at = px.base(q);
        const float mu = mean[q], r = rstd[q];
        auto each = [&](auto f) __attribute__((always_inline)) {
            for (int c0 = wave; c0 < C; c0 += LONG_W * CHUNK) {
                float d[CHUNK], z[CHUNK];
#pragma unroll
                for (int j = 0; j < CHUNK; ++j) {
                    const int c = c0 + j * LONG_W;
                    d[j] = c < C ? Store<T>::ld(dy + at + c * step) : 0.f;
                    z[j] = c < C ? Store<T>::ld(x + at + c * step) : mu;
                }
#pragma unroll
                for (int j = 0; j < CHUNK; ++j) z[j] = (z[j] - mu) * r;
                f(c0, d, z);
            }
        };
        float s = 0.f, t = 0.f;
        each([&](int c0, float (&d)[CHUNK], float (&z)[CHUNK]) {
#pragma unroll
            for (int j = 0; j < CHUNK; ++j) {
                const int c = c0 + j * LONG_W;
                const float u = d[j] * (gamma && c < C ? gamma[c] : 1.f);
                s += u;
                t += u * z[j];
            }
        });
        red[turn][0][wave][lane] = s;
        red[turn][1][wave][lane] = t;
        __syncthreads();
        s = t = 0.f;
#pragma unroll
        for (int w = 0; w < LONG_W; ++w) {
            s += red[turn][0][w][lane];
            t += red[turn][1][w][lane];
        }
        s /= (float)C;
        t /= (float)C;
        each([&](int c0, float (&d)[CHUNK], float (&z)[CHUNK]) {
#pragma unroll
            for (int j = 0; j < CHUNK; ++j) {
                const int c = c0 + j * LONG_W;
                if (dx && on && c < C) Store<T>::st(dx + at + c * step, r * (d[j] * (gamma ? gamma[c] : 1.f) - s - z[j] * t));
                d[j] = on ? d[j] : 0.f;
                z[j] = on ? d[j] * z[j] : 0.f;
            }
            if (partial) {
                const float dg = transpose_sum<CHUNK>(z), db = transpose_sum<CHUNK>(d);
                const int c = c0 + lane * CHUNK / 64 * LONG_W;
                if (lane % (64 / CHUNK) == 0 && c < C) {
                    columns[c] += dg;
                    columns[C + c] += db;
                }
            }
        });
    }
    if (!partial) return;
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * C; i += LONG_W * 64) partial[(size_t)blockIdx.x * 2 * C + i] = columns[i];
}

// ---- which kernel
template <int V> using IC = std::integral_constant<int, V>;

Pixels pixels_of(const dr_tensor& d)
{
    const size_t count = (size_t)d.n * d.h * d.w;
    const int HW = count ? d.h * d.w : 0;
    return Pixels{count, d.c, HW, d.layout == DR_NCHW && HW > 1};
}

// most workgroups that add the vectors' gradients, and so partial sums in the workspace
int norm_ranges(const dr_tensor& d)
{
    const size_t pixels = (size_t)d.n * d.h * d.w;
    return (int)std::min<size_t>(d.c > 1024 ? 256 : 512, std::max<size_t>(1, pixels / 4));
}

// f(G, NV) for rows of nvec vectors: the fewest lanes that hold a row in at most `most` vectors each; more of them while the rows are too few to give every compute unit
// a wave
template <class F>
void with_lanes(int nvec, int most, size_t rows, F f)
{
    int G = 4;
    while (G < 64 && (nvec > most * G || (nvec > G && rows * G < 64 * (size_t)device_cus()))) G *= 2;
    const int nv = (nvec + G - 1) / G;
    auto with_nv = [&](auto g) {
        if (nv <= 1) f(g, IC<1>{});
        else if (nv == 2) f(g, IC<2>{});
        else if (nv == 3) f(g, IC<3>{});
        else f(g, IC<4>{});
    };
    if (G == 4) with_nv(IC<4>{});
    else if (G == 8) with_nv(IC<8>{});
    else if (G == 16) with_nv(IC<16>{});
    else if (G == 32) with_nv(IC<32>{});
    else with_nv(IC<64>{});
}

// f(NC, W): channels of a wave, waves
template <class F>
void with_planes(int C, F f)
{
    if (C <= 16) f(IC<4>{}, IC<4>{});
    else if (C <= 64) f(IC<8>{}, IC<8>{});
    else if (C <= 128) f(IC<16>{}, IC<8>{});
    else if (C <= 256) f(IC<32>{}, IC<8>{});
    else f(IC<32>{}, IC<16>{});
}
constexpr int PLANES_MOST = 512, COLUMNS_MOST = 8192;      // channels: in registers; sums in LDS (64 KB)

template <class F>
void with_run_lanes(int C, F f)
{
    if (C <= 64) f(IC<8>{});
    else if (C <= 160) f(IC<16>{});
    else f(IC<64>{});
}

// rows of a run: as many as fit, but a run for every other compute unit at least; in eights, so that only the first and the last run of a tensor have pieces of their own
int rows_of_run(size_t rows, int C, int size)
{
    int r = (int)std::min<size_t>(std::min(512, RUN_BYTES / (C * size)), std::max<size_t>(1, rows / (2 * device_cus())));
    if (r >= 8) r &= ~7;
    return r;
}

template <typename T>
int norm_fwd(const dr_tensor& d, const T* x, const float* gamma, const float* beta, float eps, int relu, T* y, float* mean, float* rstd, hipStream_t st)
{
    constexpr int VN = Store<T>::VN;
    const Pixels px = pixels_of(d);
    const int C = d.c, nvec = C / VN;
    const bool vectors = C % VN == 0 && aligned16(x) && aligned16(y);
    TraceScope trace("layernorm", nullptr, (long long)tensor_elems(d), st, 2ll * tensor_bytes(d));
    auto rows = [&](auto g, auto nv, auto threads) {
        constexpr int G = decltype(g)::value, NV = decltype(nv)::value, TH = decltype(threads)::value;
        const unsigned grid = blocks_for(px.count, TH / G, (size_t)device_cus() * (2048 / TH));
        hipLaunchKernelGGL((norm_rows_kernel<T, G, NV, TH>), dim3(grid), dim3(TH), 0, st, px.count, C, x, gamma, beta, eps, relu, y, mean, rstd);
    };
    if (px.planes) {
        const unsigned grid = (unsigned)((px.count + 63) / 64);
        if (C <= PLANES_MOST)
            with_planes(C, [&](auto nc, auto w) {
                constexpr int NC = decltype(nc)::value, W = decltype(w)::value;
                hipLaunchKernelGGL((norm_planes_kernel<T, NC, W>), dim3(grid), dim3(W * 64), 0, st, px, x, gamma, beta, eps, relu, y, mean, rstd);
            });
        else hipLaunchKernelGGL((norm_long_planes_kernel<T>), dim3(grid), dim3(LONG_W * 64), 0, st, px, x, gamma, beta, eps, relu, y, mean, rstd);
    } else if (vectors && nvec <= 4 * 64) {
        with_lanes(nvec, 4, px.count, [&](auto g, auto nv) { rows(g, nv, IC<256>{}); });
    } else if (vectors && nvec <= 4 * 256) {
        if (nvec <= 2 * 256) rows(IC<256>{}, IC<2>{}, IC<256>{});
        else rows(IC<256>{}, IC<4>{}, IC<256>{});
    } else if (vectors && nvec <= 4 * 1024) {
        if (nvec <= 2 * 1024) rows(IC<1024>{}, IC<2>{}, IC<1024>{});
        else rows(IC<1024>{}, IC<4>{}, IC<1024>{});
    } else if (C * (int)sizeof(T) <= RUN_BYTES && C <= RUN_BYTES) {
        const int run = rows_of_run(px.count, C, sizeof(T));
        with_run_lanes(C, [&](auto g) {
            constexpr int G = decltype(g)::value;
            hipLaunchKernelGGL((norm_runs_kernel<T, G>), dim3(blocks_for(px.count, run, (size_t)device_cus() * 4)), dim3(256), 0, st, px.count, C, run, x, gamma, beta, eps, relu, y,
                               mean, rstd);
        });
    } else
        hipLaunchKernelGGL((norm_any_kernel<T>), dim3(blocks_for(px.count, 1, 16384)), dim3(256), 0, st, px, x, gamma, beta, eps, relu, y, mean, rstd);
    return check_launch("layernorm_fwd");
}

template <typename T>
int norm_bwd(const dr_tensor& d, const T* dy, const T* x, const float* gamma, const float* mean, const float* rstd, T* dx, float* dgamma, float* dbeta, float* ws,
             hipStream_t st)
{
    constexpr int VN = Store<T>::VN;
    const Pixels px = pixels_of(d);
    const int C = d.c, nvec = C / VN, most = norm_ranges(d);
    float* const partial = dgamma || dbeta ? ws : nullptr;
    const bool vectors = C % VN == 0 && aligned16(x) && aligned16(dy) && (!dx || aligned16(dx));
    TraceScope trace("layernorm_bwd", nullptr, (long long)tensor_elems(d), st, 3ll * tensor_bytes(d));
    int ranges = 0;                                      // partial sums made; 0: by no kernel yet
    if (px.count) {
        auto rows = [&](auto g, auto nv, auto threads) {
            constexpr int G = decltype(g)::value, NV = decltype(nv)::value, TH = decltype(threads)::value;
            ranges = (int)blocks_for(px.count, TH / G, std::min(most, device_cus() * (TH > 256 ? 1 : 2)));
            hipLaunchKernelGGL((norm_grad_rows_kernel<T, G, NV, TH>), dim3(ranges), dim3(TH), 2 * C * sizeof(float), st, px.count, C, dy, x, gamma, mean, rstd, dx, partial);
        };
        if (px.planes && C <= COLUMNS_MOST) {
            ranges = (int)blocks_for(px.count, 64, most);
            if (C <= PLANES_MOST)
                with_planes(C, [&](auto nc, auto w) {
                    constexpr int NC = decltype(nc)::value, W = decltype(w)::value;
                    hipLaunchKernelGGL((norm_grad_planes_kernel<T, NC, W>), dim3(ranges), dim3(W * 64), 0, st, px, dy, x, gamma, mean, rstd, dx, partial);
                });
            else hipLaunchKernelGGL((norm_grad_long_planes_kernel<T>), dim3(ranges), dim3(LONG_W * 64), 2 * C * sizeof(float), st, px, dy, x, gamma, mean, rstd, dx, partial);
        } else if (!px.planes && vectors && nvec <= 2 * 64) {
            with_lanes(nvec, VN == 4 ? 4 : 3, px.count, [&](auto g, auto nv) { rows(g, nv, IC<256>{}); });
        } else if (!px.planes && vectors && nvec <= 2 * 256) {
            rows(IC<256>{}, IC<2>{}, IC<512>{});
        } else if (!px.planes && vectors && nvec <= 2 * 1024 && C <= COLUMNS_MOST) {
            rows(IC<1024>{}, IC<2>{}, IC<1024>{});
        } else if (!px.planes && C <= 256 * RUN_COLUMNS && C * (int)sizeof(T) <= RUN_BYTES) {
            const int run = rows_of_run(px.count, C, sizeof(T));
            ranges = (int)blocks_for(px.count, run, most);
            with_run_lanes(C, [&](auto g) {
                constexpr int G = decltype(g)::value;
                auto launch = [&](auto nc) {
                    hipLaunchKernelGGL((norm_grad_runs_kernel<T, G, decltype(nc)::value>), dim3(ranges), dim3(256), 0, st, px.count, C, run, dy, x, gamma, mean, rstd, dx, partial);
                };
                if constexpr (G < 64) launch(IC<1>{});
                else if (C <= 256) launch(IC<1>{});
                else if (C <= 512) launch(IC<2>{});
                else if (C <= 1024) launch(IC<4>{});
                else launch(IC<RUN_COLUMNS>{});
            });
        }
    }
    if (ranges == 0) {
        ranges = most;
        if (partial) hipLaunchKernelGGL((norm_vectors_any_kernel<T>), dim3((C + 63) / 64, ranges), dim3(256), 0, st, px, dy, x, mean, rstd, ws);
        if (dx && px.count) hipLaunchKernelGGL((norm_grad_any_kernel<T>), dim3(blocks_for(px.count, 1, 16384)), dim3(256), 0, st, px, dy, x, gamma, mean, rstd, dx);
    }
    if (partial) hipLaunchKernelGGL(norm_vectors_sum_kernel, dim3((2 * C + 15) / 16), dim3(256), 0, st, ws, ranges, C, dgamma, dbeta);
    return check_launch("layernorm_bwd");
}

}  // namespace

int launch_layernorm_fwd(const dr_tensor& d, const void* x, const float* gamma, const float* beta, float eps, int relu, void* y, float* mean, float* rstd, hipStream_t st)
{
    if (d.dtype == DR_F32) return norm_fwd<float>(d, (const float*)x, gamma, beta, eps, relu, (float*)y, mean, rstd, st);
    return norm_fwd<uint16_t>(d, (const uint16_t*)x, gamma, beta, eps, relu, (uint16_t*)y, mean, rstd, st);
}

size_t layernorm_bwd_workspace_bytes(const dr_tensor& d) { return (size_t)norm_ranges(d) * 2 * d.c * sizeof(float); }

int launch_layernorm_bwd(const dr_tensor& d, const void* dy, const void* x, const float* gamma, const float* mean, const float* rstd, void* dx, float* dgamma, float* dbeta,
                         void* ws, hipStream_t st)
{
    if (d.dtype == DR_F32) return norm_bwd<float>(d, (const float*)dy, (const float*)x, gamma, mean, rstd, (float*)dx, dgamma, dbeta, (float*)ws, st);
    return norm_bwd<uint16_t>(d, (const uint16_t*)dy, (const uint16_t*)x, gamma, mean, rstd, (uint16_t*)dx, dgamma, dbeta, (float*)ws, st);
}

}  // namespace dr
