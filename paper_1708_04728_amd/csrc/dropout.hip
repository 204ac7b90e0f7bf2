// Dropout (dr_dropout_fwd): y = x 65536 / (65536 - T) where the element's draw is T or more, else 0; T = round(65536 p).
//
// The draws are 16 bits of Philox4x32-10 for the element's place in memory, so the mask is nowhere stored: the gradient is the same call on dy, and the adapters'
// kernels make it while they read x.
#include "dr_internal.h"
#include "philox.h"
#include "rows8.h"

namespace dr {
namespace {

// A lane takes blocks of eight elements, U of them 256 apart, all loaded before the first is used.  Bound by memory: 128 x 192 x 56 x 56 in bf16 58 us, 5.3 TB/s; a block's
// ten rounds of two 32 x 32-bit products are ~560 cycles of a wave for 512 elements, half of what memory takes for them.
template <typename T, int U>
__global__ __launch_bounds__(256) void dropout_kernel(const Drop drop, const T* x, T* y, unsigned count)
{
    const uint64_t place = drop_place(drop);
    const unsigned first = blockIdx.x * (256u * U) + threadIdx.x;
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned at = (first + u * 256u) * 8u;
        if (at < count) load8(x + at, (int)min(count - at, 8u), 0.f, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned block = first + u * 256u, at = block * 8u;
        if (at >= count) continue;
        drop8(drop, place, block, v[u]);
        store8(y + at, (int)min(count - at, 8u), v[u]);
    }
}

template <typename T>
void launch(const Drop& drop, const void* x, void* y, unsigned count, hipStream_t st)
{
    const unsigned blocks = (count + 7) / 8;
    if (blocks > 4u * 256 * 1024) hipLaunchKernelGGL((dropout_kernel<T, 4>), dim3((blocks + 1023) / 1024), dim3(256), 0, st, drop, (const T*)x, (T*)y, count);
    else hipLaunchKernelGGL((dropout_kernel<T, 1>), dim3((blocks + 255) / 256), dim3(256), 0, st, drop, (const T*)x, (T*)y, count);
}

}  // namespace

int launch_dropout(int dtype, const void* x, const Drop& drop, void* y, size_t count, hipStream_t st)
{
    if (count == 0) return DR_OK;
    TraceScope trace("dropout", nullptr, (long long)count, st, (long long)(2 * count * elem_size(dtype)));
    if (dtype == DR_BF16) launch<uint16_t>(drop, x, y, (unsigned)count, st);
    else launch<float>(drop, x, y, (unsigned)count, st);
    return check_launch("dropout");
}

}  // namespace dr
