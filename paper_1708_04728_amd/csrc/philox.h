// The random numbers of dropout: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, 2011), a function of a key and a counter, so
// that a mask is made again wherever it is needed and never stored.  Plain C++, so that the same lines run in the kernels and in a test on the host.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define DR_ANY __host__ __device__ __forceinline__
#else
#define DR_ANY inline
#endif

namespace dr {

// 128 bits for counter (block, place) under the key `seed`
DR_ANY void philox(uint64_t seed, uint64_t block, uint64_t place, uint32_t (&r)[4])
{
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
    uint32_t a = (uint32_t)block, b = (uint32_t)(block >> 32), c = (uint32_t)place, d = (uint32_t)(place >> 32);
#if defined(__HIPCC__)
#pragma unroll
#endif
    for (int i = 0; i < 10; ++i) {
        const uint64_t p = (uint64_t)0xD2511F53u * a, q = (uint64_t)0xCD9E8D57u * c;
        a = (uint32_t)(q >> 32) ^ b ^ k0;
        b = (uint32_t)q;
        c = (uint32_t)(p >> 32) ^ d ^ k1;
        d = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    r[0] = a; r[1] = b; r[2] = c; r[3] = d;
}

// An element is dropped where its 16 bits are below the border, with probability border / 65536: p to within 2^-17.  Sixteen bits rather than 32, because a block of
// ten rounds (about 140 instruction slots of a lane, 80 of them in 32-bit products) then serves eight elements: four would make a bf16 tensor's dropout wait for it.
constexpr int DROP_BITS = 65536;
inline unsigned drop_border(float p) { return (unsigned)((double)p * DROP_BITS + 0.5); }
inline float drop_scale(unsigned border) { return border >= DROP_BITS ? 0.f : (float)((double)DROP_BITS / (DROP_BITS - (int)border)); }

// What kernels take of a dr_dropout
struct Drop {
    uint64_t seed, offset;
    const uint64_t* step;        // device; NULL: 0
    unsigned border;             // 0: nothing is dropped
    float scale;                 // of what is kept
};
inline Drop make_drop(float p, uint64_t seed, uint64_t offset, const uint64_t* step)
{
    Drop d;
    d.seed = seed; d.offset = offset; d.step = step;
    d.border = drop_border(p);
    d.scale = drop_scale(d.border);
    return d;
}

// Draw of element j (0..7) of a block
DR_ANY unsigned drop_draw(const uint32_t (&r)[4], int j) { return j & 1 ? r[j >> 1] >> 16 : r[j >> 1] & 0xFFFFu; }

#if defined(__HIPCC__)
__device__ __forceinline__ uint64_t drop_place(const Drop& d) { return d.offset + (d.step ? *d.step : 0); }

// Which of a block's elements are kept: 1 or 0 in the half of a word that held the element's draw (border >= 1)
__device__ __forceinline__ void kept_halves(const Drop& d, uint64_t place, uint64_t block, uint32_t (&m)[4])
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    uint32_t r[4];
    philox(d.seed, block, place, r);
    const unsigned short last = (unsigned short)(d.border - 1);          // the last draw that is dropped
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u16x2 beyond = __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, r[i]), u16x2{last, last});
        m[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(beyond, u16x2{1, 1}));
    }
}
// ... bit j for element 8 block + j
__device__ __forceinline__ unsigned kept8(const Drop& d, uint64_t place, uint64_t block)
{
    uint32_t m[4];
    kept_halves(d, place, block, m);
    const unsigned t = m[0] | m[1] << 2 | m[2] << 4 | m[3] << 6;         // even elements in bits 0, 2, .., odd ones in 16, 18, ..
    return (t | t >> 15) & 0xFFu;
}
// ... of sixteen from any `first` on
__device__ __forceinline__ unsigned kept16(const Drop& d, uint64_t place, uint64_t first)
{
    const int shift = (int)(first & 7), blocks = shift ? 3 : 2;
    unsigned bits = 0;
#pragma unroll 1
    for (int i = 0; i < blocks; ++i) bits |= kept8(d, place, (first >> 3) + i) << (8 * i);
    return (bits >> shift) & 0xFFFFu;
}

// Dropout of the eight elements of a block (v[j] is element 8 block + j)
__device__ __forceinline__ void drop8(const Drop& d, uint64_t place, uint64_t block, float (&v)[8])
{
    uint32_t r[4];
    philox(d.seed, block, place, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = drop_draw(r, j) >= d.border ? v[j] * d.scale : 0.f;
}
#endif

}  // namespace dr
