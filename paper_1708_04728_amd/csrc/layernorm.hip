// Layer normalisation over the channels of every pixel, and its gradient (dr_layernorm_fwd, dr_layernorm_bwd).
//
//   forward    y = gamma (x - mean) rstd + beta [, max(., 0)],  mean = sum_c x / C,  rstd = 1 / sqrt(sum_c (x - mean)^2 / C + eps)
//   gradient   with g = dy gamma and z = (x - mean) rstd:
//              dx = rstd (g - sum_c g / C - z sum_c (g z) / C),  dgamma_c = sum over pixels of dy z,  dbeta_c = sum over pixels of dy
//
// The variance is the mean square of differences from the mean, not a difference of squares: a pixel's values may lie far from zero.  Squares are added divided by a
// power of two near C, so that their sum is no infinity where the variance is a number.
#include <algorithm>

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

Pixels pixels_of(const dr_tensor& d)
{
    const size_t count = (size_t)d.n * d.h * d.w;
    const int HW = count ? d.h * d.w : 0;
    return Pixels{count, d.c, HW, d.layout == DR_NCHW && HW > 1};
}

// ranges of pixels that the vectors' gradients are added over
int norm_ranges(const dr_tensor& d)
{
    const size_t pixels = (size_t)d.n * d.h * d.w;
    return (int)std::min<size_t>(256, std::max<size_t>(1, pixels / 16));
}

template <typename T>
int norm_fwd(const dr_tensor& d, const T* x, const float* gamma, const float* beta, float eps, int relu, T* y, float* mean, float* rstd, hipStream_t st)
{
    const Pixels px = pixels_of(d);
    TraceScope trace("layernorm", nullptr, (long long)tensor_elems(d), st, 2ll * tensor_bytes(d));
    hipLaunchKernelGGL((norm_any_kernel<T>), dim3(blocks_for(px.count, 1, 16384)), dim3(256), 0, st, px, x, gamma, beta, eps, relu, y, mean, rstd);
    return check_launch("layernorm_fwd");
}

template <typename T>
int norm_bwd(const dr_tensor& d, const T* dy, const T* x, const float* gamma, const float* mean, const float* rstd, T* dx, float* dgamma, float* dbeta, float* ws,
             hipStream_t st)
{
    const Pixels px = pixels_of(d);
    const int ranges = norm_ranges(d);
    TraceScope trace("layernorm_bwd", nullptr, (long long)tensor_elems(d), st, 3ll * tensor_bytes(d));
    if (dgamma || dbeta) {
        hipLaunchKernelGGL((norm_vectors_any_kernel<T>), dim3((d.c + 63) / 64, ranges), dim3(256), 0, st, px, dy, x, mean, rstd, ws);
        hipLaunchKernelGGL(norm_vectors_sum_kernel, dim3((2 * d.c + 15) / 16), dim3(256), 0, st, ws, ranges, d.c, dgamma, dbeta);
    }
    if (dx && px.count) hipLaunchKernelGGL((norm_grad_any_kernel<T>), dim3(blocks_for(px.count, 1, 16384)), dim3(256), 0, st, px, dy, x, gamma, mean, rstd, dx);
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
