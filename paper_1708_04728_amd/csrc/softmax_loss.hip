// Softmax loss of rows of class logits and its gradient (dr_softmax_loss_grad): with the label t of a row of C logits z and smoothing e,
//
//   l = log sum exp z - (1 - e) z_t - e / C sum z,   dz = g (exp(z - log sum exp z) - (1 - e) [j = t] - e / C),   g = 1 or 1 / (rows with a label)
//
// A row is read once: its lanes hold it in registers from the maximum to the gradient.  Sums are in fp32 over a lane's elements, then over lanes in a fixed order; the
// loss of all rows is added in double.  Bound by memory where rows are many (8192 x 32768 bf16 223 us, 4.8 TB/s; 353 with loads behind conditions, 276 with exponentials of
// eight instructions, 294 with 512 lanes of 64 elements, whose registers spill), by launches where they are few (128 x 1000: 4.5 + 2.5 us), by the one workgroup that counts labels and the one that adds losses where
// they are many and short (2^20 x 16: 876 us).
#include <algorithm>

#include "dr_internal.h"
#include "rows8.h"

namespace dr {
namespace {

constexpr int COUNT_ROWS = 2048;         // most labels that every workgroup counts for itself

// exp(d) for d <= 0: 2^p with p = d log2 e, whose rounding and that of log2 e put it off by up to 1.3 |d| 2^-24 of itself.  fp32 gradients show that (70 x 2^-24 at d = -80), so in fp32 what
// is lost, d - p ln 2, is put back: off by (3 + |d| / 20) 2^-24.  bf16 ones are rounded at 2^-8, and the sum, of which exp(d_j) is the share p_j, is off by
// 1.3 sum p_j |d_j| 2^-24 <= 1.3 ln C 2^-24 (sum p_j |d_j| is the entropy less ln of the sum), 14 x 2^-24 at 65536 classes, where its additions may round away up to 90: three
// instructions more cost 8192 x 32768 classes 13 us of 229 there, and nothing in fp32.
// -inf gives 0, a NaN stays one; below 2^-126 zero, where the instruction ends: a sum, which is 1 at least, does not see it, and a gradient that small is 0.
template <typename T>
__device__ __forceinline__ float exp_of(float d)
{
    const float p = d * 1.44269502162933349609375f, e = __builtin_amdgcn_exp2f(p);
    if (sizeof(T) == 2) return e;
    const float lost = fminf(__builtin_fmaf(p, -0.693147182464599609375f, d), 1.f);      // (of -inf not a number, taken for 1: 0 stays 0)
    return __builtin_fmaf(e, lost, e);
}

template <int THREADS, class F>
__device__ __forceinline__ float reduce(float v, float* red, F f)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v = f(v, __shfl_xor(v, d, 64));
    if (THREADS == 64) return v;
    constexpr int W = THREADS / 64;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < W; ++w) v = f(v, red[w]);
    return v;
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }

// rows with a label, counted by all `threads` of a workgroup; the same in every thread
__device__ __forceinline__ int count_labels(const int* __restrict__ labels, int rows, int C, int threads, int* red)
{
    int n = 0;
    for (int i = threadIdx.x; i < rows; i += threads) n += (unsigned)labels[i] < (unsigned)C;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) n += __shfl_xor(n, d, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < threads / 64; ++w) n += red[w];
    __syncthreads();
    return n;
}

__global__ __launch_bounds__(1024) void count_kernel(const int* __restrict__ labels, int rows, int C, int* __restrict__ counted)
{
    __shared__ int red[16];
    const int n = count_labels(labels, rows, C, 1024, red);
    if (threadIdx.x == 0) *counted = n;
}

struct Loss {
    int rows, C;
    const int* labels;
    float smoothing;
    int mean;
    const int* counted;          // rows with a label, or NULL: every workgroup counts them
    float share;                 // a power of two of at most 1 / (2 C): so much of a row's numbers adds up to no more than the largest of them
    float* row_loss;
};

// what one row's gradient and loss need beside its exponentials
struct RowSums { float top, sum, shifted; };       // max z, sum exp(z - top), sum (z - top) share

__device__ __forceinline__ float row_loss_of(const Loss& q, const RowSums& s, float z_t)
{
    const float about = q.smoothing != 0.f ? q.smoothing * s.shifted / ((float)q.C * q.share) : 0.f;
    // (halves: their difference is a number wherever both are)
    const float label = q.smoothing != 1.f ? 2.f * ((1.f - q.smoothing) * (0.5f * z_t - 0.5f * s.top)) : 0.f;
    return logf(s.sum) - label - about;
}

// PER lanes a row, NV blocks of eight elements a lane; workgroups of max(PER, 256) threads walk the rows
template <typename T, int PER, int NV>
__global__ __launch_bounds__(PER < 256 ? 256 : PER, 4) void loss_kernel(const Loss q, const T* z, T* dz)
{
    constexpr int THREADS = PER < 256 ? 256 : PER, TEAMS = THREADS / PER;
    __shared__ float red[16];
    __shared__ int redi[16];
    const int lane = threadIdx.x & (PER - 1), team = threadIdx.x / PER;
    float g = 1.f;
    if (q.mean && dz) {
        const int n = q.counted ? *q.counted : count_labels(q.labels, q.rows, q.C, THREADS, redi);
        g = n > 0 ? 1.f / (float)n : 0.f;
    }
    for (int row = blockIdx.x * TEAMS + team; row < q.rows; row += gridDim.x * TEAMS) {       // (whole waves agree; with TEAMS > 1 nothing below synchronises)
        const T* zr = z + (size_t)row * q.C;
        const int label = q.labels[row];
        const bool has = (unsigned)label < (unsigned)q.C;
        // A lane's eight places, the row's last eight where it ends before them: those of them that another lane has too (the first `twice`) are left out of the sums, and
        // written by both with the same bits.  Loads without a condition between them stay in flight together.
        auto start = [&](int i) { return min((i * PER + lane) * 8, q.C - 8); };
        auto twice = [&](int i) { return min((i * PER + lane) * 8 - start(i), 8); };
        auto ragged = [&](int i) { return (i + 1) * PER * 8 > q.C; };
        if (!has) {
            if (lane == 0) q.row_loss[row] = 0.f;
            if (dz) {
                const float zero[8] = {};
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if ((i * PER + lane) * 8 < q.C) store8(dz + (size_t)row * q.C + start(i), zero);
            }
            continue;
        }
        float v[NV][8];
        const float z_t = Store<T>::ld(zr + label);
#pragma unroll
        for (int i = 0; i < NV; ++i) load8(zr + start(i), v[i]);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, v[i][j]);
        RowSums s;
        s.top = top = reduce<PER>(top, red, larger);
        float sum = 0.f, shifted = 0.f;
        if (q.smoothing != 0.f) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) shifted += !ragged(i) || j >= twice(i) ? __builtin_fmaf(v[i][j], q.share, -top * q.share) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = exp_of<T>(v[i][j] - top);
            if (ragged(i)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += j >= twice(i) ? v[i][j] : 0.f;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += v[i][j];
            }
        }
        s.sum = reduce<PER>(sum, red, add);
        s.shifted = q.smoothing != 0.f ? reduce<PER>(shifted, red, add) : 0.f;
        if (lane == 0) q.row_loss[row] = row_loss_of(q, s, z_t);
        if (dz) {
            const float scale = g / s.sum, less = g * (q.smoothing / (float)q.C), at_label = g * (1.f - q.smoothing);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = start(i);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = __builtin_fmaf(v[i][j], scale, -less);
                if ((unsigned)(label - c) < 8u) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[i][j] -= c + j == label ? at_label : 0.f;
                }
                if ((i * PER + lane) * 8 < q.C) store8(dz + (size_t)row * q.C + c, v[i]);
            }
        }
    }
}

// Fewer than eight classes: a lane a row
template <typename T>
__global__ __launch_bounds__(256) void loss_short_kernel(const Loss q, const T* z, T* dz)
{
    __shared__ int redi[16];
    float g = 1.f;
    if (q.mean && dz) {
        const int n = q.counted ? *q.counted : count_labels(q.labels, q.rows, q.C, 256, redi);
        g = n > 0 ? 1.f / (float)n : 0.f;
    }
    for (int row = blockIdx.x * 256 + threadIdx.x; row < q.rows; row += gridDim.x * 256) {
        const int label = q.labels[row];
        const bool has = (unsigned)label < (unsigned)q.C;
        float v[8];
        load8(z + (size_t)row * q.C, q.C, -INFINITY, v);
        RowSums s = {-INFINITY, 0.f, 0.f};
        float z_t = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s.top = fmaxf(s.top, v[j]);
            z_t = j == label ? v[j] : z_t;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j < q.C) s.shifted += __builtin_fmaf(v[j], q.share, -s.top * q.share);
            v[j] = j < q.C ? exp_of<T>(v[j] - s.top) : 0.f;
            s.sum += v[j];
        }
        q.row_loss[row] = has ? row_loss_of(q, s, z_t) : 0.f;
        if (!dz) continue;
        const float scale = g / s.sum, less = g * (q.smoothing / (float)q.C), at_label = g * (1.f - q.smoothing);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = has ? v[j] * scale - (j == label ? less + at_label : less) : 0.f;
        store8(dz + (size_t)row * q.C, q.C, v);
    }
}

// Rows too long for registers: read twice, the maximum and the sum running together the first time
template <typename T>
__global__ __launch_bounds__(1024) void loss_long_kernel(const Loss q, const T* z, T* dz)
{
    __shared__ float red[16];
    __shared__ int redi[16];
    float g = 1.f;
    if (q.mean && dz) {
        const int n = q.counted ? *q.counted : count_labels(q.labels, q.rows, q.C, 1024, redi);
        g = n > 0 ? 1.f / (float)n : 0.f;
    }
    for (int row = blockIdx.x; row < q.rows; row += gridDim.x) {
        const T* zr = z + (size_t)row * q.C;
        const int label = q.labels[row];
        const bool has = (unsigned)label < (unsigned)q.C;
        RowSums s;
        if (has) {
            const float z_t = Store<T>::ld(zr + label);
            float top = -INFINITY, sum = 0.f, shifted = 0.f;
            for (int c = threadIdx.x * 8; c < q.C; c += 8192) {
                float v[8], most = top;
                load8(zr + c, q.C - c, -INFINITY, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, v[j]);
                const float from = most == -INFINITY ? 0.f : most;       // nothing but -inf so far: exp(-inf - 0) = 0
                sum *= exp_of<T>(top - from);
                if (q.smoothing != 0.f) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) shifted += c + j < q.C ? v[j] * q.share : 0.f;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += exp_of<T>(v[j] - from);
                top = most;
            }
            s.top = reduce<1024>(top, red, larger);
            s.sum = reduce<1024>(top == -INFINITY ? (s.top == -INFINITY ? NAN : sum) : sum * exp_of<T>(top - s.top), red, add);
            s.shifted = q.smoothing != 0.f ? reduce<1024>(shifted, red, add) - (float)q.C * q.share * s.top : 0.f;
            if (threadIdx.x == 0) q.row_loss[row] = row_loss_of(q, s, z_t);
            __syncthreads();                                                    // (dz may be z: the label's logit has been read)
        } else if (threadIdx.x == 0) q.row_loss[row] = 0.f;
        if (!dz) continue;
        const float scale = g / s.sum, less = g * (q.smoothing / (float)q.C), at_label = g * (1.f - q.smoothing);
        for (int c = threadIdx.x * 8; c < q.C; c += 8192) {
            float v[8] = {};
            if (has) {
                load8(zr + c, q.C - c, -INFINITY, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = exp_of<T>(v[j] - s.top) * scale - (c + j == label ? less + at_label : less);
            }
            store8(dz + (size_t)row * q.C + c, q.C - c, v);
        }
    }
}

__global__ __launch_bounds__(1024) void loss_sum_kernel(const Loss q, float* __restrict__ loss)
{
    __shared__ double red[16];
    __shared__ int redi[16];
    const int n = !q.mean ? 1 : q.counted ? *q.counted : count_labels(q.labels, q.rows, q.C, 1024, redi);
    double s = 0;
    for (int i = threadIdx.x; i < q.rows; i += 1024) s += (double)q.row_loss[i];
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0;
        for (int w = 0; w < 16; ++w) s += red[w];
        *loss = n > 0 ? (float)(s / n) : 0.f;
    }
}

template <typename T, int PER, int NV>
void launch_rows(const Loss& q, const void* z, void* dz, hipStream_t st)
{
    constexpr int THREADS = PER < 256 ? 256 : PER, TEAMS = THREADS / PER;
    const int groups = (q.rows + TEAMS - 1) / TEAMS;
    hipLaunchKernelGGL((loss_kernel<T, PER, NV>), dim3(std::min(groups, 8192)), dim3(THREADS), 0, st, q, (const T*)z, (T*)dz);
}

// The fewest lanes that hold a row in at most 32 elements each; in 64 above 32768 classes, where 1024 lanes are all there are and some registers spill (2048 x 50001 bf16 178 us, fp32 208; read
// twice, 2048 x 65537 bf16 162)
template <typename T>
void launch(const Loss& q, const void* z, void* dz, hipStream_t st)
{
    if (q.C < 8) hipLaunchKernelGGL((loss_short_kernel<T>), dim3(std::min((q.rows + 255) / 256, 4096)), dim3(256), 0, st, q, (const T*)z, (T*)dz);
    else if (q.C <= 512) launch_rows<T, 64, 1>(q, z, dz, st);
    else if (q.C <= 1024) launch_rows<T, 64, 2>(q, z, dz, st);
    else if (q.C <= 2048) launch_rows<T, 256, 1>(q, z, dz, st);
    else if (q.C <= 4096) launch_rows<T, 256, 2>(q, z, dz, st);
    else if (q.C <= 8192) launch_rows<T, 256, 4>(q, z, dz, st);
    else if (q.C <= 16384) launch_rows<T, 512, 4>(q, z, dz, st);
    else if (q.C <= 32768) launch_rows<T, 1024, 4>(q, z, dz, st);
    else if (q.C <= 65536) launch_rows<T, 1024, 8>(q, z, dz, st);
    else hipLaunchKernelGGL((loss_long_kernel<T>), dim3(std::min(q.rows, 4096)), dim3(1024), 0, st, q, (const T*)z, (T*)dz);
}

}  // namespace

size_t softmax_loss_workspace_bytes(int rows) { return 256 + align_up((size_t)rows * 4, 256); }

int launch_softmax_loss_grad(int dtype, int rows, int classes, const void* z, const int* labels, float smoothing, int mean, void* dz, float* loss, float* row_loss,
                             void* ws, hipStream_t st)
{
    TraceScope trace("softmax_loss", nullptr, (long long)rows * classes, st, (long long)rows * classes * (long long)elem_size(dtype) * (dz ? 2 : 1));
    Loss q;
    q.share = 0.5f;
    for (unsigned c = 1; c < (unsigned)classes; c *= 2) q.share *= 0.5f;
    q.rows = rows; q.C = classes; q.labels = labels; q.smoothing = smoothing; q.mean = mean;
    q.row_loss = row_loss ? row_loss : (float*)((char*)ws + 256);
    q.counted = nullptr;
    if (mean && rows > COUNT_ROWS) {
        hipLaunchKernelGGL(count_kernel, dim3(1), dim3(1024), 0, st, labels, rows, classes, (int*)ws);
        q.counted = (const int*)ws;
    }
    if (rows) {
        if (dtype == DR_BF16) launch<uint16_t>(q, z, dz, st);
        else launch<float>(q, z, dz, st);
    }
    if (loss) hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(1024), 0, st, q, loss);
    return check_launch("softmax_loss");
}

}  // namespace dr
