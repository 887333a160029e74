// The format of matrices in 8 bits with a power of two for each 128 entries of a row, and reading and writing
// eight entries of a matrix of any type.
#pragma once

#include <cstdint>

#include "ecq_common.cuh"
#include "ecq_elem.cuh"

namespace ecq {

// The format.  A block is 128 consecutive entries of a row.  Its scale 2^e is the smallest power of two
// with max|x| <= L 2^e, L the type's largest value (e4m3: 448 = 1.75 2^8, e5m2: 57344 = 1.75 2^15), not
// below 2^-127; it is held as the byte e + 127, and 255 says that the block had a NaN or Inf.  Entries
// are x 2^-e rounded to nearest even: scaling by a power of two loses nothing, so there is one rounding
// (e4m3: 2^-4 of the entry, for entries from 2^-6 2^e on), a second storing along the other axis changes
// nothing but entries below that, and restored values are exact in 16 bits.
//
// Scale bytes lie as the tensor cores take them: 512 bytes for 128 rows and four blocks.
__host__ __device__ __forceinline__ uint64_t act8_scale_at(uint32_t row, uint32_t block, uint32_t groups) {
    return ((uint64_t)(row >> 7) * groups + (block >> 2)) * 512u + (row & 31u) * 16u + ((row >> 5) & 3u) * 4u + (block & 3u);
}

// A matrix of a call: bytes from row to row, and for 8 bits its scales in groups of four blocks.
struct Act8Mat {
    unsigned char* data;
    uint64_t stride;
    uint8_t* scales;
    uint32_t groups;
    int dtype;                           // 0 .. 2 plain, 3 e4m3, 4 e5m2
    int wide;                            // rows begin on 16-byte boundaries
};

// Scale byte of a block by the bit pattern of its largest magnitude; what entries are multiplied by.
__device__ __forceinline__ uint32_t act8_byte(uint32_t amax, int dtype) {
    if (amax >= 0x7F800000u) return 255u;
    const int b = (int)(amax >> 23) - (dtype == 3 ? 8 : 15) + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return b > 0 ? (uint32_t)b : 0u;
}
__device__ __forceinline__ float act8_down(uint32_t byte) {
    return byte == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float((254u - byte) << 23);
}
__device__ __forceinline__ float act8_up(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte ? byte << 23 : 0x00400000u);
}

__device__ __forceinline__ uint32_t act8_pair(float lo, float hi, int dtype) {
    uint16_t r;
    if (dtype == 3) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t act8_quad(const float* x, float by, int dtype) {
    float a, b, c, d;
    const uint64_t by2 = pack2(by, by);
    unpack2(mul2(pack2(x[0], x[1]), by2), a, b);
    unpack2(mul2(pack2(x[2], x[3]), by2), c, d);
    return act8_pair(a, b, dtype) | act8_pair(c, d, dtype) << 16;
}
__device__ __forceinline__ void act8_unpair(uint32_t two, int dtype, float by, float* x) {
    uint32_t h;
    if (dtype == 3) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    else asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    unpack2(mul2(pack2(f.x, f.y), pack2(by, by)), x[0], x[1]);
}

__device__ __forceinline__ uint32_t act8_largest(const float* x, uint32_t m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    return m;
}
// Of the 16 lanes that have a block.
__device__ __forceinline__ uint32_t act8_block_max(uint32_t m) {
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) m = max(m, __shfl_xor_sync(~0u, m, o));
    return m;
}

// Eight consecutive entries of a row as they lie in memory.
template <typename T> struct Raw8 { uint4 w[sizeof(T) / 2]; };
template <> struct Raw8<uint8_t> { uint2 w; uint32_t byte; };

// `n` of them are inside the matrix; the others are zeros.
template <typename T>
__device__ __forceinline__ void get8(const Act8Mat& m, uint32_t row, uint32_t col, uint32_t n, Raw8<T>& r) {
    const unsigned char* p = m.data + row * m.stride + (uint64_t)col * sizeof(T);
    if (n == 8 && m.wide) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = *(reinterpret_cast<const uint4*>(p) + i);
        return;
    }
    T e[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) e[i] = i < n ? reinterpret_cast<const T*>(p)[i] : T(0.f);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = *(reinterpret_cast<const uint4*>(e) + i);
}
template <>
__device__ __forceinline__ void get8<uint8_t>(const Act8Mat& m, uint32_t row, uint32_t col, uint32_t n, Raw8<uint8_t>& r) {
    const unsigned char* p = m.data + row * m.stride + col;
    r.byte = n ? m.scales[act8_scale_at(row, col >> 7, m.groups)] : 127u;
    if (n == 8) {
        r.w = *reinterpret_cast<const uint2*>(p);
        return;
    }
    r.w = make_uint2(0, 0);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        if (i < n) (i < 4 ? r.w.x : r.w.y) |= (uint32_t)p[i] << (8 * (i & 3));
}

template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T>& r, int, float* x) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) Elem<T>::widen(r.w[i], x + i * Elem<T>::kPer16);
}
template <>
__device__ __forceinline__ void widen8<uint8_t>(const Raw8<uint8_t>& r, int dtype, float* x) {
    const float by = act8_up(r.byte);
    act8_unpair(r.w.x, dtype, by, x);
    act8_unpair(r.w.x >> 16, dtype, by, x + 2);
    act8_unpair(r.w.y, dtype, by, x + 4);
    act8_unpair(r.w.y >> 16, dtype, by, x + 6);
}

template <typename T>
__device__ __forceinline__ void put8(const Act8Mat& m, uint32_t row, uint32_t col, uint32_t n, const float* x) {
    unsigned char* p = m.data + row * m.stride + (uint64_t)col * sizeof(T);
    if (n == 8 && m.wide) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            *(reinterpret_cast<uint4*>(p) + i) = Elem<T>::narrow(x + i * Elem<T>::kPer16);
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        if (i < n) Elem<T>::store(reinterpret_cast<T*>(p) + i, x[i]);
}

// Eight entries and, from the first lane of a block, its scale, by the block's largest magnitude.
__device__ __forceinline__ void put8_coded(const Act8Mat& m, uint32_t row, uint32_t col, uint32_t n, const float* x,
                                           uint32_t block_max) {
    if (!n) return;
    const uint32_t byte = act8_byte(block_max, m.dtype);
    const float by = act8_down(byte);
    unsigned char* p = m.data + row * m.stride + col;
    const uint2 w = make_uint2(act8_quad(x, by, m.dtype), act8_quad(x + 4, by, m.dtype));
    if (n == 8) {
        *reinterpret_cast<uint2*>(p) = w;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < n) p[i] = (unsigned char)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
    if ((col & 127u) == 0) m.scales[act8_scale_at(row, col >> 7, m.groups)] = (uint8_t)byte;
}

__device__ __forceinline__ uint32_t inside(uint32_t col, uint32_t cols) { return col >= cols ? 0u : min(8u, cols - col); }

}  // namespace ecq
