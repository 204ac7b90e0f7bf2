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

// ---- any tensor: a workgroup per pixel, its channels read once for each sum.  For rows beyond 4096 vectors of 16 bytes (1024 x 32768 fp32 132 us, 2.0 TB/s), and planes so large that 32
// bits do not address 64 pixels of an image (8192 channels of 301 x 300 fp32 48 ms: 4 bytes of every 64 that it fetches)
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

// dgamma and dbeta from the partial sums of `ranges` ranges of pixels, in a fixed order, in double: 4 us, a launch
__global__ __launch_bounds__(1024) void norm_vectors_sum_kernel(const float* __restrict__ partial, int ranges, int C, float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ double red[64][17];
    const int lane = threadIdx.x & 15, col = blockIdx.x * 16 + lane, row = threadIdx.x >> 4;
    double s = 0.0;
    if (col < 2 * C) {
#pragma unroll 8
        for (int r = row; r < ranges; r += 64) s += (double)partial[(size_t)r * 2 * C + col];
    }
    red[row][lane] = s;
    __syncthreads();
    if (row < 4) {
        s = 0.0;
#pragma unroll
        for (int r = 0; r < 16; ++r) s += red[row * 16 + r][lane];
    }
    __syncthreads();
    if (row < 4) red[row][lane] = s;
    __syncthreads();
    if (row == 0 && col < 2 * C) {
        const float v = (float)((red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]));
        if (col < C) { if (dgamma) dgamma[col] = v; }
        else if (dbeta) dbeta[col - C] = v;
    }
}

// ---- sums over lanes
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true)); }
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) { return v + dpp<CTRL>(v); }

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

// ---- channels last, rows of 16 bytes and more: a row in the registers of G lanes, NV vectors of 16 bytes each.  G > 64: G / 64 waves.  The workgroup's THREADS / G
// groups walk the rows together.  Rows may start anywhere: 16-byte loads and stores need no alignment.  RAGGED: where 16 bytes do not divide a row, its last vector ends where
// the row ends and holds some elements of the one before it again, which count once and are stored twice, with the same value.
__device__ __forceinline__ uint4 load16(const void* p)
{
    uint4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
template <typename T>
__device__ __forceinline__ void store16(T* p, const float* v)
{
    uint4 t;
    if constexpr (sizeof(T) == 4) t = uint4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    else t = uint4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    __builtin_memcpy(p, &t, 16);
}

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

// Where vector k of a row of C elements starts, and how many of its elements the vector before it holds too
template <int VN, bool RAGGED>
struct Place {
    int first, skip;
    __device__ __forceinline__ Place(int k, int C) : first(k * VN), skip(0)
    {
        if (RAGGED && first + VN > C) {
            skip = first + VN - C;
            first = C - VN;
        }
    }
};

// HBM bounds it: each element once.  192 channels of 56 x 56 x 128 bf16 56 us, 5.5 TB/s (part of it stays in the memory-side cache), fp32 119, 5.2; 333 of 56 x 56 x 64 fp32, whose rows start
// anywhere, 111, 4.8; rows of 8192 fp32 5.9.  Small maps take a launch: 7.2 us of 14.7 MB.
template <typename T, int G, int NV, int THREADS, bool RAGGED>
__global__ __launch_bounds__(THREADS) void norm_rows_kernel(size_t rows, int C, const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, float eps,
                                                            int relu, T* y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    constexpr int VN = Store<T>::VN, GROUPS = THREADS / G;
    __shared__ float red[2][THREADS / 64][1];
    int turn = 0;
    const int lane = threadIdx.x % G, group = threadIdx.x / G, nvec = (C + VN - 1) / VN;
    const float down = square_scale(C);
    uint4 next[NV];
    auto at = [&](int j) __attribute__((always_inline)) { return Place<VN, RAGGED>(lane + j * G, C); };
    auto fetch = [&](size_t row) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (lane + j * G < nvec && row < rows) next[j] = load16(x + row * C + at(j).first);
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
            load_vector<VN>(gamma, at(j).first, 1.f, g[j]);
            load_vector<VN>(beta, at(j).first, 0.f, b[j]);
        }
    for (size_t first = (size_t)blockIdx.x * GROUPS; first < rows; first += stride, row += stride) {      // (the same rounds for all lanes)
        float v[NV][VN], s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            unpack<T>(next[j], v[j]);                  // (zero beyond the row)
#pragma unroll
            for (int e = 0; e < VN; ++e) s[0] += !RAGGED || e >= at(j).skip ? v[j][e] : 0.f;
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
                    s[0] = __builtin_fmaf(!RAGGED || e >= at(j).skip ? v[j][e] * down : 0.f, v[j][e], s[0]);
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
                    store16<T>(y + row * C + at(j).first, v[j]);
                }
            if (lane == 0) {
                if (mean_out) mean_out[row] = mean;
                if (rstd_out) rstd_out[row] = rstd;
            }
        }
    }
}

// ... and the gradient: every lane adds its columns of dgamma and dbeta over the workgroup's rows; partial[workgroup][2][C].  192 channels of 56 x 56 x 128 bf16 95 us with the sum behind it,
// 4.9 TB/s; rows of 4096 bf16 46, 4.4; 14.9 MB 11.5, 6.3 in this launch (9.6 where the waves added their columns to one array in turn)
template <typename T, int G, int NV, int THREADS, bool RAGGED>
__global__ __launch_bounds__(THREADS) void norm_grad_rows_kernel(size_t rows, int C, const T* dy, const T* x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                                                 const float* __restrict__ rstd, T* dx, float* __restrict__ partial)
{
    constexpr int VN = Store<T>::VN, GROUPS = THREADS / G, IN_WAVE = G < 64 ? 64 / G : 1, TURNS = GROUPS / IN_WAVE;
    __shared__ float red[2][THREADS / 64][2];
    extern __shared__ float columns[];                 // [TURNS][2][C]
    int turn = 0;
    const int lane = threadIdx.x % G, group = threadIdx.x / G, nvec = (C + VN - 1) / VN;
    uint4 nx[NV], nd[NV];
    float n_mean = 0.f, n_rstd = 0.f;
    auto at = [&](int j) __attribute__((always_inline)) { return Place<VN, RAGGED>(lane + j * G, C); };
    auto fetch = [&](size_t row) __attribute__((always_inline)) {
        if (row >= rows) return;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (lane + j * G < nvec) {
                nd[j] = load16(dy + row * C + at(j).first);
                nx[j] = load16(x + row * C + at(j).first);
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
        if (lane + j * G < nvec) load_vector<VN>(gamma, at(j).first, 1.f, g[j]);
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
                    const float once = !RAGGED || e >= at(j).skip ? d[j][e] : 0.f, u = once * g[j][e];
                    s[0] += u;
                    s[1] += u * z[j][e];
                    db[j][e] += once;
                    dg[j][e] += once * z[j][e];
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
                    store16<T>(dx + row * C + at(j).first, d[j]);
                }
        }
    }
    if (!partial) return;
    // the groups of a wave, each wave's sums (those of the waves that share a row) on their own in LDS, then all of a column's
#pragma unroll
    for (int k = G; k < 64; k *= 2)
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                dg[j][e] += __shfl_xor(dg[j][e], k, 64);
                db[j][e] += __shfl_xor(db[j][e], k, 64);
            }
    if (group % IN_WAVE == 0) {
        float* const mine = columns + (size_t)(group / IN_WAVE) * 2 * C;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (lane + j * G < nvec) {
#pragma unroll
                for (int e = 0; e < VN; ++e) {
                    if (RAGGED && e < at(j).skip) continue;
                    mine[at(j).first + e] = dg[j][e];
                    mine[C + at(j).first + e] = db[j][e];
                }
            }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * C; i += THREADS) {
        float s = columns[i];
#pragma unroll
        for (int t = 1; t < TURNS; ++t) s += columns[t * 2 * C + i];
        partial[(size_t)blockIdx.x * 2 * C + i] = s;
    }
}

// ---- channels last, rows shorter than 16 bytes: a lane has a whole row.  3 channels of 16.8 million pixels fp32 132 us, 3.1 TB/s (the gradient 188, 3.2); 7 of 8.4 million
// in bf16 137 (159): element by element, bound by instructions
constexpr int NARROW = 8;
template <typename T>
__global__ __launch_bounds__(256) void norm_narrow_kernel(size_t rows, int C, const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, float eps, int relu, T* y,
                                                          float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    const float down = square_scale(C);
    for (size_t row = (size_t)blockIdx.x * 256 + threadIdx.x; row < rows; row += (size_t)gridDim.x * 256) {
        float v[NARROW], s = 0.f;
#pragma unroll
        for (int c = 0; c < NARROW; ++c) {
            v[c] = c < C ? Store<T>::ld(x + row * C + c) : 0.f;
            s += v[c];
        }
        const float mean = s / (float)C;
        s = 0.f;
#pragma unroll
        for (int c = 0; c < NARROW; ++c)
            if (c < C) {
                v[c] -= mean;
                s = __builtin_fmaf(v[c] * down, v[c], s);
            }
        const float rstd = 1.f / sqrtf(s / ((float)C * down) + eps);
#pragma unroll
        for (int c = 0; c < NARROW; ++c)
            if (c < C) {
                const float t = v[c] * rstd * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f);
                Store<T>::st(y + row * C + c, relu ? fmaxf(t, 0.f) : t);
            }
        if (mean_out) mean_out[row] = mean;
        if (rstd_out) rstd_out[row] = rstd;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void norm_grad_narrow_kernel(size_t rows, int C, const T* dy, const T* x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                                               const float* __restrict__ rstd, T* dx, float* __restrict__ partial)
{
    __shared__ float red[4][2 * NARROW];
    float dg[NARROW], db[NARROW];
#pragma unroll
    for (int c = 0; c < NARROW; ++c) dg[c] = db[c] = 0.f;
    for (size_t row = (size_t)blockIdx.x * 256 + threadIdx.x; row < rows; row += (size_t)gridDim.x * 256) {
        const float mu = mean[row], r = rstd[row];
        float d[NARROW], z[NARROW], s = 0.f, t = 0.f;
#pragma unroll
        for (int c = 0; c < NARROW; ++c) {
            d[c] = c < C ? Store<T>::ld(dy + row * C + c) : 0.f;
            z[c] = c < C ? (Store<T>::ld(x + row * C + c) - mu) * r : 0.f;
            db[c] += d[c];
            dg[c] += d[c] * z[c];
            const float u = d[c] * (gamma && c < C ? gamma[c] : 1.f);
            s += u;
            t += u * z[c];
        }
        s /= (float)C;
        t /= (float)C;
        if (dx) {
#pragma unroll
            for (int c = 0; c < NARROW; ++c)
                if (c < C) Store<T>::st(dx + row * C + c, r * (d[c] * (gamma ? gamma[c] : 1.f) - s - z[c] * t));
        }
    }
    if (!partial) return;
#pragma unroll
    for (int c = 0; c < NARROW; ++c) {
        dg[c] = lanes_sum<64>(dg[c]);
        db[c] = lanes_sum<64>(db[c]);
        if ((threadIdx.x & 63) == 0) {
            red[threadIdx.x >> 6][c] = dg[c];
            red[threadIdx.x >> 6][NARROW + c] = db[c];
        }
    }
    __syncthreads();
    if (threadIdx.x < 2 * NARROW) {
        const int c = threadIdx.x % NARROW, which = threadIdx.x / NARROW;
        if (c < C) partial[(size_t)blockIdx.x * 2 * C + which * C + c] = (red[0][threadIdx.x] + red[1][threadIdx.x]) + (red[2][threadIdx.x] + red[3][threadIdx.x]);
    }
}

// ---- channel planes: LP pixels of any images a workgroup, a lane for each in 64 / LP channels at a time; its waves (16 at most) share the channels, NC of them at most in a
// lane's registers.  An element's address is a plane's, the same for the wave, and the lane's 32-bit distance from it: with 64-bit addresses of their own the loads wait for
// arithmetic (the gradient of 192 channels on 28 x 28 x 32 pixels fp32 22.8 us for 17.2).  HBM bounds them:
// 192 channels of 56 x 56 x 64 fp32 62 us, 5.0 TB/s, the gradient 105, 4.4; bf16, whose planes are 128 bytes of 64 pixels, 3.3 and 3.8; 28 x 28 x 32 fp32 11.3 and 19.4, a round of workgroups.
constexpr int PLANES_WAVES = 16;
template <typename T, int LP>
struct Planes {
    static constexpr int SUB = 64 / LP;
    size_t step, at;         // elements from channel to channel; of the first pixel's image
    size_t pixel;
    unsigned off0, off;      // bytes from `at` to this lane's pixel in channel 0, and in its own of the SUB channels
    int sub, C;
    bool on;
    __device__ __forceinline__ Planes(const Pixels& px, size_t group)
    {
        const size_t first = group * LP, img0 = first / px.HW;
        const unsigned in0 = (unsigned)(first - img0 * px.HW), lane = threadIdx.x % LP;      // (in0: wave-uniform)
        pixel = first + lane;
        on = pixel < px.count;
        if (!on) pixel = px.count - 1;
        const unsigned p = in0 + (unsigned)(pixel - first), img = p / (unsigned)px.HW;
        step = px.HW;
        at = img0 * px.C * px.HW;
        C = px.C;
        sub = (threadIdx.x & 63) / LP;
        off0 = (img * (unsigned)px.C * px.HW + (p - img * px.HW)) * (unsigned)sizeof(T);
        off = off0 + sub * (unsigned)px.HW * (unsigned)sizeof(T);
    }
    // channel c0 + sub, c0 the same for the wave.  Of a channel that does not exist: another's value.
    __device__ __forceinline__ float ld(const T* base, int c0) const
    {
        c0 = min(c0, C - 1);
        const unsigned o = SUB == 1 || c0 + sub < C ? off : off0;
        return Store<T>::ld(reinterpret_cast<const T*>(reinterpret_cast<const char*>(base + at + c0 * step) + o));
    }
    __device__ __forceinline__ void st(T* base, int c0, float v) const
    {
        if (on && c0 + sub < C) Store<T>::st(reinterpret_cast<T*>(reinterpret_cast<char*>(base + at + c0 * step) + off), v);
    }
};
// the distances above fit 32 bits
bool planes_near(const Pixels& px, int size) { return (double)(64 / px.HW + 2) * px.C * px.HW * size + 4.0 * px.HW * size < 4294967296.0; }

// sums over a pixel's channels: its lanes' in all waves of the workgroup
template <int LP, int N>
__device__ __forceinline__ void pixel_sums(float (&v)[N], float (*red)[PLANES_WAVES][64])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, W = blockDim.x >> 6;
#pragma unroll
    for (int n = 0; n < N; ++n) red[n][wave][lane] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        float t = 0.f;
        for (int w = 0; w < W; ++w)
#pragma unroll
            for (int u = 0; u < 64 / LP; ++u) t += red[n][w][u * LP + lane % LP];
        v[n] = t;
    }
}

template <typename T, int LP, int NC>
__global__ __launch_bounds__(PLANES_WAVES * 64) void norm_planes_kernel(const Pixels px, const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, float eps,
                                                                        int relu, T* y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    constexpr int SUB = 64 / LP;
    __shared__ float red[2][PLANES_WAVES][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), step = (blockDim.x >> 6) * SUB, C = px.C;
    const float down = square_scale(C);
    const Planes<T, LP> p(px, blockIdx.x);
    float v[NC], s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NC; ++j) v[j] = p.ld(x, wave * SUB + j * step);
#pragma unroll
    for (int j = 0; j < NC; ++j) s[0] += wave * SUB + p.sub + j * step < C ? v[j] : 0.f;
    pixel_sums<LP>(s, red);
    const float mean = s[0] / (float)C;
    s[0] = 0.f;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        v[j] -= mean;
        s[0] = __builtin_fmaf(wave * SUB + p.sub + j * step < C ? v[j] * down : 0.f, v[j], s[0]);
    }
    pixel_sums<LP>(s, red + 1);
    const float rstd = 1.f / sqrtf(s[0] / ((float)C * down) + eps);
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c0 = wave * SUB + j * step, c = min(c0 + p.sub, C - 1);
        const float t = v[j] * rstd * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f);
        p.st(y, c0, relu ? fmaxf(t, 0.f) : t);
    }
    if (threadIdx.x < LP && p.on) {
        if (mean_out) mean_out[p.pixel] = mean;
        if (rstd_out) rstd_out[p.pixel] = rstd;
    }
}

// Sums over groups of LP lanes of N <= LP values each, both powers of two: every lane gets the sum of value (lane % LP) N / LP.  A step hands half of a lane's values to the
// lane it meets and takes the others' in return: about two instructions a value in all, in the place of twelve.
template <int N, int M, int D>
__device__ __forceinline__ void transpose_step(float (&v)[N])      // M values left; lanes meet across bit D
{
    if constexpr (D >= 16) {
        auto sum = [](float a, float b) __attribute__((always_inline)) {      // lanes without bit D: a of both lanes; with it: b
            if constexpr (D == 32) {
                const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
                return __uint_as_float(t[0]) + __uint_as_float(t[1]);
            } else {
                const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
                return __uint_as_float(t[0]) + __uint_as_float(t[1]);
            }
        };
        if constexpr (M > 1) {
#pragma unroll
            for (int i = 0; i < M / 2; ++i) v[i] = sum(v[i], v[i + M / 2]);
        } else v[0] = sum(v[0], v[0]);
    } else {
        // lane +- 8 of sixteen; 7 - lane of eight (a lane's later partners have met the others of the eight); lane ^ 2; lane ^ 1
        constexpr int CTRL = D == 8 ? 0x128 : D == 4 ? 0x141 : D == 2 ? 0x4E : 0xB1;
        if constexpr (M > 1) {
            const bool high = (threadIdx.x & D) != 0;
#pragma unroll
            for (int i = 0; i < M / 2; ++i) {
                const float keep = high ? v[i + M / 2] : v[i], give = high ? v[i] : v[i + M / 2];
                v[i] = keep + dpp<CTRL>(give);
            }
        } else v[0] += dpp<CTRL>(v[0]);
    }
    if constexpr (D > 1) transpose_step<N, (M > 1 ? M / 2 : 1), D / 2>(v);
}
template <int LP, int N>
__device__ __forceinline__ float transpose_sum(float (&v)[N])
{
    static_assert(N <= LP, "a value for a lane at most");
    transpose_step<N, N, LP / 2>(v);
    return v[0];
}
// The gradient on planes: a workgroup walks groups of LP pixels; the sums over a group's pixels by transpose_sum, so that a lane holds the running sums of a channel
template <typename T, int LP, int NC>
__global__ __launch_bounds__(PLANES_WAVES * 64) void norm_grad_planes_kernel(const Pixels px, const T* dy, const T* x, const float* __restrict__ gamma,
                                                                             const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, float* __restrict__ partial)
{
    constexpr int SUB = 64 / LP;
    __shared__ float red[2][2][PLANES_WAVES][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), step = (blockDim.x >> 6) * SUB, C = px.C;
    const size_t groups = (px.count + LP - 1) / LP;
    float dg = 0.f, db = 0.f;
    int turn = 0;
    for (size_t k = blockIdx.x; k < groups; k += gridDim.x, turn ^= 1) {
        const Planes<T, LP> p(px, k);
        float z[NC], d[NC], s[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            d[j] = p.ld(dy, wave * SUB + j * step);
            z[j] = p.ld(x, wave * SUB + j * step);
        }
        const float mu = mean[p.pixel], r = rstd[p.pixel];
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int c = wave * SUB + p.sub + j * step;
            d[j] = c < C ? d[j] : 0.f;
            z[j] = c < C ? (z[j] - mu) * r : 0.f;
            const float u = d[j] * (gamma ? gamma[min(c, C - 1)] : 1.f);
            s[0] += u;
            s[1] += u * z[j];
        }
        pixel_sums<LP>(s, red[turn]);
        s[0] /= (float)C;
        s[1] /= (float)C;
        if (dx) {
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const int c0 = wave * SUB + j * step;
                p.st(dx, c0, r * (d[j] * (gamma ? gamma[min(c0 + p.sub, C - 1)] : 1.f) - s[0] - z[j] * s[1]));
            }
        }
        if (partial) {
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                d[j] = p.on ? d[j] : 0.f;
                z[j] = p.on ? d[j] * z[j] : 0.f;
            }
            dg += transpose_sum<LP>(z);
            db += transpose_sum<LP>(d);
        }
    }
    const int lane = threadIdx.x % LP, c = wave * SUB + (int)(threadIdx.x & 63) / LP + lane * NC / LP * step;
    if (partial && lane % (LP / NC) == 0 && c < C) {
        partial[(size_t)blockIdx.x * 2 * C + c] = dg;
        partial[(size_t)blockIdx.x * 2 * C + C + c] = db;
    }
}

// ... of more channels than registers hold: read again for each use (from the caches), CHUNK channels of a lane at a time, by 16 waves: 2048 of 28 x 28 x 32 fp32
// 183 us, 3.3 TB/s of three passes, the gradient 232, 4.4 of five
constexpr int CHUNK = 16;
template <typename T, int LP>
__global__ __launch_bounds__(PLANES_WAVES * 64) void norm_long_planes_kernel(const Pixels px, const T* x, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                                             float eps, int relu, T* y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    constexpr int SUB = 64 / LP, LONG_STEP = PLANES_WAVES * SUB;
    __shared__ float red[2][PLANES_WAVES][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), C = px.C;
    const float down = square_scale(C);
    const Planes<T, LP> p(px, blockIdx.x);
    auto chunks = [&](auto f) __attribute__((always_inline)) {
        for (int c0 = wave * SUB; c0 < C; c0 += LONG_STEP * CHUNK) {
            float v[CHUNK];
#pragma unroll
            for (int j = 0; j < CHUNK; ++j) v[j] = p.ld(x, c0 + j * LONG_STEP);
#pragma unroll
            for (int j = 0; j < CHUNK; ++j) f(c0 + j * LONG_STEP, v[j]);
        }
    };
    float s[1] = {0.f};
    chunks([&](int c0, float v) { s[0] += c0 + p.sub < C ? v : 0.f; });
    pixel_sums<LP>(s, red);
    const float mean = s[0] / (float)C;
    s[0] = 0.f;
    chunks([&](int c0, float v) {
        const float d = v - mean;
        s[0] = __builtin_fmaf(c0 + p.sub < C ? d * down : 0.f, d, s[0]);
    });
    pixel_sums<LP>(s, red + 1);
    const float rstd = 1.f / sqrtf(s[0] / ((float)C * down) + eps);
    chunks([&](int c0, float v) {
        const int c = min(c0 + p.sub, C - 1);
        const float t = (v - mean) * rstd * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f);
        p.st(y, c0, relu ? fmaxf(t, 0.f) : t);
    });
    if (threadIdx.x < LP && p.on) {
        if (mean_out) mean_out[p.pixel] = mean;
        if (rstd_out) rstd_out[p.pixel] = rstd;
    }
}

template <typename T, int LP>
__global__ __launch_bounds__(PLANES_WAVES * 64) void norm_grad_long_planes_kernel(const Pixels px, const T* dy, const T* x, const float* __restrict__ gamma,
                                                                                  const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, float* __restrict__ partial)
{
    constexpr int SUB = 64 / LP, LONG_STEP = PLANES_WAVES * SUB;
    __shared__ float red[2][2][PLANES_WAVES][64];
    extern __shared__ float columns[];       // [2][C]: running sums, each touched by one lane
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), C = px.C;
    const size_t groups = (px.count + LP - 1) / LP;
    for (int i = threadIdx.x; i < 2 * C; i += PLANES_WAVES * 64) columns[i] = 0.f;
    __syncthreads();
    int turn = 0;
    for (size_t k = blockIdx.x; k < groups; k += gridDim.x, turn ^= 1) {
        const Planes<T, LP> p(px, k);
        const float mu = mean[p.pixel], r = rstd[p.pixel];
        auto chunks = [&](auto f) __attribute__((always_inline)) {
            for (int c0 = wave * SUB; c0 < C; c0 += LONG_STEP * CHUNK) {
                float d[CHUNK], z[CHUNK];
#pragma unroll
                for (int j = 0; j < CHUNK; ++j) {
                    d[j] = p.ld(dy, c0 + j * LONG_STEP);
                    z[j] = p.ld(x, c0 + j * LONG_STEP);
                }
#pragma unroll
                for (int j = 0; j < CHUNK; ++j) {
                    const bool in = c0 + p.sub + j * LONG_STEP < C;
                    d[j] = in ? d[j] : 0.f;
                    z[j] = in ? (z[j] - mu) * r : 0.f;
                }
                f(c0, d, z);
            }
        };
        float s[2] = {0.f, 0.f};
        chunks([&](int c0, float (&d)[CHUNK], float (&z)[CHUNK]) {
#pragma unroll
            for (int j = 0; j < CHUNK; ++j) {
                const float u = d[j] * (gamma ? gamma[min(c0 + p.sub + j * LONG_STEP, C - 1)] : 1.f);
                s[0] += u;
                s[1] += u * z[j];
            }
        });
        pixel_sums<LP>(s, red[turn]);
        s[0] /= (float)C;
        s[1] /= (float)C;
        chunks([&](int c0, float (&d)[CHUNK], float (&z)[CHUNK]) {
#pragma unroll
            for (int j = 0; j < CHUNK; ++j) {
                const int c = c0 + j * LONG_STEP;
                if (dx) p.st(dx, c, r * (d[j] * (gamma ? gamma[min(c + p.sub, C - 1)] : 1.f) - s[0] - z[j] * s[1]));
                d[j] = p.on ? d[j] : 0.f;
                z[j] = p.on ? d[j] * z[j] : 0.f;
            }
            if (partial) {
                const float dg = transpose_sum<LP>(z), db = transpose_sum<LP>(d);
                const int c = c0 + p.sub + (int)(threadIdx.x % LP) * CHUNK / LP * LONG_STEP;
                if (threadIdx.x % (LP / CHUNK) == 0 && c < C) {
                    columns[c] += dg;
                    columns[C + c] += db;
                }
            }
        });
    }
    if (!partial) return;
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * C; i += PLANES_WAVES * 64) partial[(size_t)blockIdx.x * 2 * C + i] = columns[i];
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
    return (int)std::min<size_t>(d.c <= 256 ? 1024 : d.c <= 1024 ? 512 : 256, std::max<size_t>(1, pixels / 4));
}
// workgroups for `groups` groups of pixels, `most` at most: every one has the same number of them, or one less
int even_blocks(size_t groups, int most)
{
    const size_t each = (groups + most - 1) / most;
    return (int)((groups + each - 1) / each);
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

// f(LP, NC): pixels of a workgroup, channels of a lane; NC = 0: more channels than registers hold (`most` of a lane).  64 pixels, a whole 256 bytes of a plane, but where they
// make fewer workgroups than half of the compute units: 16 (832 channels of 7 x 7 x 128 fp32 33.5 us with 64, 22.8 with 16; 192 of 28 x 28 x 32 11.2 and 14.2 with 32),
// and where 16 have up to `once` channels in registers which 64 have not (forward: 832 channels of 14 x 14 x 128 90.8 us read twice, 81.1 once; 1024 of 28 x 28 x 64 183 and 137;
// the gradient 109 and 133, 212 and 224; 2048 of 28 x 28 x 32, 32 channels of a lane, forward 183 and 189).
template <class F>
void with_planes(const Pixels& px, int most, int once, F f)
{
    auto with_nc = [&](auto lp) {
        constexpr int LP = decltype(lp)::value, GROUPS = PLANES_WAVES * (64 / LP);      // lanes of a pixel at most
        if (px.C <= 8 * GROUPS / 2) f(lp, IC<8>{});
        else if (px.C <= 16 * GROUPS) f(lp, IC<16>{});
        else if (px.C <= most * GROUPS) f(lp, IC<32>{});
        else f(lp, IC<0>{});
    };
    if (px.count >= 32 * (size_t)device_cus() && (px.C <= most * PLANES_WAVES || px.C > once)) with_nc(IC<64>{});
    else with_nc(IC<16>{});
}
constexpr int COLUMNS_MOST = 8192;      // channels whose sums fit LDS (64 KB)

template <typename T>
int norm_fwd(const dr_tensor& d, const T* x, const float* gamma, const float* beta, float eps, int relu, T* y, float* mean, float* rstd, hipStream_t st)
{
    constexpr int VN = Store<T>::VN;
    const Pixels px = pixels_of(d);
    const int C = d.c, nvec = (C + VN - 1) / VN;
    TraceScope trace("layernorm", nullptr, (long long)tensor_elems(d), st, 2ll * tensor_bytes(d));
    auto rows = [&](auto g, auto nv, auto threads) {
        constexpr int G = decltype(g)::value, NV = decltype(nv)::value, TH = decltype(threads)::value;
        const unsigned grid = blocks_for(px.count, TH / G, (size_t)device_cus() * (2048 / TH));
        if (C % VN == 0) hipLaunchKernelGGL((norm_rows_kernel<T, G, NV, TH, false>), dim3(grid), dim3(TH), 0, st, px.count, C, x, gamma, beta, eps, relu, y, mean, rstd);
        else hipLaunchKernelGGL((norm_rows_kernel<T, G, NV, TH, true>), dim3(grid), dim3(TH), 0, st, px.count, C, x, gamma, beta, eps, relu, y, mean, rstd);
    };
    if (px.planes && planes_near(px, sizeof(T))) {
        with_planes(px, 32, 16 * 4 * PLANES_WAVES, [&](auto lp, auto nc) {
            constexpr int LP = decltype(lp)::value, NC = decltype(nc)::value, EACH = NC * (64 / LP);
            const dim3 grid((unsigned)((px.count + LP - 1) / LP));
            if constexpr (NC == 0) hipLaunchKernelGGL((norm_long_planes_kernel<T, LP>), grid, dim3(PLANES_WAVES * 64), 0, st, px, x, gamma, beta, eps, relu, y, mean, rstd);
            else hipLaunchKernelGGL((norm_planes_kernel<T, LP, NC>), grid, dim3((C + EACH - 1) / EACH * 64), 0, st, px, x, gamma, beta, eps, relu, y, mean, rstd);
        });
    } else if (px.planes)
        hipLaunchKernelGGL((norm_any_kernel<T>), dim3(blocks_for(px.count, 1, 16384)), dim3(256), 0, st, px, x, gamma, beta, eps, relu, y, mean, rstd);
    else if (C < VN)
        hipLaunchKernelGGL((norm_narrow_kernel<T>), dim3(blocks_for(px.count, 256, 4096)), dim3(256), 0, st, px.count, C, x, gamma, beta, eps, relu, y, mean, rstd);
    else if (nvec <= 4 * 64) with_lanes(nvec, 4, px.count, [&](auto g, auto nv) { rows(g, nv, IC<256>{}); });
    else if (nvec <= 2 * 256) rows(IC<256>{}, IC<2>{}, IC<256>{});
    else if (nvec <= 4 * 256) rows(IC<256>{}, IC<4>{}, IC<256>{});
    else if (nvec <= 2 * 1024) rows(IC<1024>{}, IC<2>{}, IC<1024>{});
    else if (nvec <= 4 * 1024) rows(IC<1024>{}, IC<4>{}, IC<1024>{});
    else
        hipLaunchKernelGGL((norm_any_kernel<T>), dim3(blocks_for(px.count, 1, 16384)), dim3(256), 0, st, px, x, gamma, beta, eps, relu, y, mean, rstd);
    return check_launch("layernorm_fwd");
}

template <typename T>
int norm_bwd(const dr_tensor& d, const T* dy, const T* x, const float* gamma, const float* mean, const float* rstd, T* dx, float* dgamma, float* dbeta, float* ws,
             hipStream_t st)
{
    constexpr int VN = Store<T>::VN;
    const Pixels px = pixels_of(d);
    const int C = d.c, nvec = (C + VN - 1) / VN, most = norm_ranges(d);
    float* const partial = dgamma || dbeta ? ws : nullptr;
    TraceScope trace("layernorm_bwd", nullptr, (long long)tensor_elems(d), st, 3ll * tensor_bytes(d));
    int ranges = 0;                                      // partial sums made; 0: by no kernel yet
    if (px.count) {
        auto rows = [&](auto g, auto nv, auto threads) {
            constexpr int G = decltype(g)::value, NV = decltype(nv)::value, TH = decltype(threads)::value;
            ranges = (int)blocks_for(px.count, TH / G, std::min(most, device_cus() * (TH > 256 ? 1 : 2)));
            const size_t columns = (size_t)(G < 64 ? TH / 64 : TH / G) * 2 * C * sizeof(float);      // (64 KB at most)
            if (C % VN == 0) hipLaunchKernelGGL((norm_grad_rows_kernel<T, G, NV, TH, false>), dim3(ranges), dim3(TH), columns, st, px.count, C, dy, x, gamma, mean, rstd, dx, partial);
            else hipLaunchKernelGGL((norm_grad_rows_kernel<T, G, NV, TH, true>), dim3(ranges), dim3(TH), columns, st, px.count, C, dy, x, gamma, mean, rstd, dx, partial);
        };
        if (px.planes) {
            if (planes_near(px, sizeof(T)) && C <= COLUMNS_MOST)
                with_planes(px, px.count >= 32 * (size_t)device_cus() ? 32 : 16, 0, [&](auto lp, auto nc) {
                    constexpr int LP = decltype(lp)::value, NC = decltype(nc)::value, EACH = NC * (64 / LP);
                    ranges = even_blocks((px.count + LP - 1) / LP, most);
                    if constexpr (NC == 0)
                        hipLaunchKernelGGL((norm_grad_long_planes_kernel<T, LP>), dim3(ranges), dim3(PLANES_WAVES * 64), 2 * C * sizeof(float), st, px, dy, x, gamma, mean, rstd, dx, partial);
                    else if constexpr (NC <= 16 || LP == 64)
                        hipLaunchKernelGGL((norm_grad_planes_kernel<T, LP, NC>), dim3(ranges), dim3((C + EACH - 1) / EACH * 64), 0, st, px, dy, x, gamma, mean, rstd, dx, partial);
                });
        } else if (C < VN) {
            ranges = (int)blocks_for(px.count, 256, most);
            hipLaunchKernelGGL((norm_grad_narrow_kernel<T>), dim3(ranges), dim3(256), 0, st, px.count, C, dy, x, gamma, mean, rstd, dx, partial);
        } else if (nvec <= 2 * 64) with_lanes(nvec, VN == 4 ? 4 : 3, px.count, [&](auto g, auto nv) { rows(g, nv, IC<256>{}); });
        else if (nvec <= 2 * 256) rows(IC<256>{}, IC<2>{}, IC<512>{});
        else if (nvec <= 2 * 1024 && C <= COLUMNS_MOST) rows(IC<1024>{}, IC<2>{}, IC<1024>{});
    }
    if (ranges == 0) {
        ranges = most;
        if (partial) hipLaunchKernelGGL((norm_vectors_any_kernel<T>), dim3((C + 63) / 64, ranges), dim3(256), 0, st, px, dy, x, mean, rstd, ws);
        if (dx && px.count) hipLaunchKernelGGL((norm_grad_any_kernel<T>), dim3(blocks_for(px.count, 1, 16384)), dim3(256), 0, st, px, dy, x, gamma, mean, rstd, dx);
    }
    if (partial) hipLaunchKernelGGL(norm_vectors_sum_kernel, dim3((2 * C + 15) / 16), dim3(1024), 0, st, ws, ranges, C, dgamma, dbeta);
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
