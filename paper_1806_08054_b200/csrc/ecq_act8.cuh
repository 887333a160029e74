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
    unsigned char *data, *end;           // first byte, and behind the last
    uint64_t stride;
    uint8_t* scales;
    uint32_t groups;
    int dtype;                           // 0 .. 2 plain, 3 e4m3, 4 e5m2
    int wide;                            // rows begin on 16-byte boundaries
};

// The scale byte is found from the bit pattern of a magnitude: adding 2^21 - 1 carries into the exponent
// exactly where the mantissa is above 1.75, the limit of both types.  It grows with the magnitude, so the
// largest byte of a block's parts is the block's.  NaN and Inf give 255.
__device__ __forceinline__ uint32_t act8_byte(uint32_t amax, int dtype) {
    const int b = (int)((amax + 0x1FFFFFu) >> 23) - (dtype == 3 ? 8 : 15);
    return amax >= 0x7F800000u ? 255u : (uint32_t)max(b, 0);
}
// What entries are multiplied by, to and from 8 bits.
__device__ __forceinline__ float act8_down(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : (254u - byte) << 23);
}
__device__ __forceinline__ float act8_up(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte ? byte << 23 : 0x00400000u);
}

// Larger of magnitudes; NaN wins.
__device__ __forceinline__ float top3(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t act8_largest(const float* x) {
    return __float_as_uint(top3(top3(top3(x[0], x[1], x[2]), x[3], x[4]), top3(x[5], x[6], x[7]), 0.f));
}

__device__ __forceinline__ uint16_t act8_e4m3(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint16_t act8_e5m2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// N entries times `by` in 8 bits, four a word.  (Branches on the type lie around as much as possible: a
// conversion that is predicated on it is issued all the same.)
template <int N>
__device__ __forceinline__ void act8_code(const float* x, float by, int dtype, uint32_t* w) {
    float y[N];
    const uint64_t by2 = pack2(by, by);
#pragma unroll
    for (int i = 0; i < N; i += 2) unpack2(mul2(pack2(x[i], x[i + 1]), by2), y[i], y[i + 1]);
    if (dtype == 3) {
#pragma unroll
        for (int i = 0; i < N; i += 4) w[i / 4] = act8_e4m3(y[i], y[i + 1]) | (uint32_t)act8_e4m3(y[i + 2], y[i + 3]) << 16;
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) w[i / 4] = act8_e5m2(y[i], y[i + 1]) | (uint32_t)act8_e5m2(y[i + 2], y[i + 3]) << 16;
    }
}
// And back: unscaled, and times `by`.
__device__ __forceinline__ void act8_decode8(uint2 q, int dtype, float* x) {
    const uint32_t two[4] = {q.x & 0xFFFFu, q.x >> 16, q.y & 0xFFFFu, q.y >> 16};
    uint32_t h[4];
    if (dtype == 3) {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h[i]) : "h"((uint16_t)two[i]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h[i]) : "h"((uint16_t)two[i]));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void act8_decode8(uint2 q, int dtype, float by, float* x) {
    act8_decode8(q, dtype, x);
    const uint64_t by2 = pack2(by, by);
#pragma unroll
    for (int i = 0; i < 8; i += 2) unpack2(mul2(pack2(x[i], x[i + 1]), by2), x[i], x[i + 1]);
}

// Eight consecutive entries of a row as they lie in memory (of 8 bits with their block's scale byte).  FULL:
// all eight are inside the matrix and its rows begin on 16-byte boundaries; otherwise `n` of them are
// and the others are zeros.
template <typename T> struct Raw8 { uint4 w[sizeof(T) / 2]; };
template <> struct Raw8<uint8_t> { uint2 w; uint32_t byte; };

// Words w[by] .. w[by + N - 1], by < 4, without indexing.
template <int N, int M>
__device__ __forceinline__ void from_word(const uint32_t (&w)[M], uint32_t by, uint32_t (&to)[N]) {
    static_assert(M >= N + 3, "");
    uint32_t x[N + 2];
#pragma unroll
    for (int i = 0; i < N + 2; ++i) x[i] = by & 1u ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < N; ++i) to[i] = by & 2u ? x[i + 2] : x[i];
}

// Rows that begin anywhere: the 16-byte pieces that the eight lie in, moved by where they begin.  Pieces that are
// not in the matrix's memory as a whole are not read; the entries are then read one by one.
template <bool FULL, typename T>
__device__ __forceinline__ void get8(const Act8Mat& m, const unsigned char* p, const uint8_t*, uint32_t n, Raw8<T>& r) {
    constexpr int kVecs = (int)sizeof(T) / 2;                        // of 16 bytes
    if (FULL || (n == 8 && m.wide)) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) r.w[i] = *(reinterpret_cast<const uint4*>(p) + i);
        return;
    }
    const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15u;
    const unsigned char* base = p - off;
    if (n == 8 && base >= m.data && base + 16 * (kVecs + 1) <= m.end) {
        uint32_t w[4 * kVecs + 4];
#pragma unroll
        for (int i = 0; i <= kVecs; ++i) {
            const uint4 v = *(reinterpret_cast<const uint4*>(base) + i);
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
        if (sizeof(T) == 4) {
            uint32_t x[4 * kVecs];
            from_word(w, off >> 2, x);
#pragma unroll
            for (int i = 0; i < kVecs; ++i) r.w[i] = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
        } else {
            uint32_t x[5], z[4];
            // the ninth word is needed for nothing but the shift's form
            const uint32_t more[8] = {w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]};
            from_word(more, off >> 2, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = __funnelshift_r(x[i], x[i + 1], 8 * (off & 2u));
            r.w[0] = make_uint4(z[0], z[1], z[2], z[3]);
        }
        return;
    }
    T e[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) e[i] = i < n ? reinterpret_cast<const T*>(p)[i] : T(0.f);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) r.w[i] = *(reinterpret_cast<const uint4*>(e) + i);
}
template <bool FULL>
__device__ __forceinline__ void get8(const Act8Mat&, const unsigned char* p, const uint8_t* scale, uint32_t n, Raw8<uint8_t>& r) {
    if (FULL || n == 8) {
        r.w = *reinterpret_cast<const uint2*>(p);
        r.byte = *scale;
        return;
    }
    r.w = make_uint2(0, 0);
    r.byte = n ? *scale : 127u;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        if (i < n) (i < 4 ? r.w.x : r.w.y) |= (uint32_t)p[i] << (8 * (i & 3));
}

template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T>& r, int, float* x) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) Elem<T>::widen(r.w[i], x + i * Elem<T>::kPer16);
}
__device__ __forceinline__ void widen8(const Raw8<uint8_t>& r, int dtype, float* x) { act8_decode8(r.w, dtype, act8_up(r.byte), x); }

// Writes them; LANES lanes (the whole warp takes part) have consecutive eights of a row.  Where rows begin anywhere a lane
// writes the 16-byte pieces that begin in its eight, with the next lane's first entries; what is left at
// both ends of the lanes' part goes out one by one.
template <bool FULL, int LANES, typename T>
__device__ __forceinline__ void put8(const Act8Mat& m, unsigned char* p, uint32_t n, const float* x) {
    constexpr int kVecs = (int)sizeof(T) / 2;
    if (FULL || m.wide) {
        if (FULL || n == 8) {
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
                *(reinterpret_cast<uint4*>(p) + i) = Elem<T>::narrow(x + i * Elem<T>::kPer16);
            return;
        }
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < n) Elem<T>::store(reinterpret_cast<T*>(p) + i, x[i]);
        return;
    }
    uint32_t w[4 * kVecs + 4];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const uint4 v = Elem<T>::narrow(x + i * Elem<T>::kPer16);
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
    }
    const uint32_t lane = threadIdx.x & (LANES - 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[4 * kVecs + i] = __shfl_down_sync(~0u, w[i], 1, LANES);
    const uint32_t after = __shfl_down_sync(~0u, n, 1, LANES);
    // bytes, and entries, to the first piece
    const uint32_t off = (16u - ((uint32_t)reinterpret_cast<uintptr_t>(p) & 15u)) & 15u, h = off / (uint32_t)sizeof(T);
    const bool whole = n == 8 && (h == 0 || (lane + 1 < LANES && after >= h));
    const bool before = __shfl_up_sync(~0u, (int)whole, 1, LANES) && lane > 0;
    if (whole) {
        uint4* to = reinterpret_cast<uint4*>(p + off);
        if (sizeof(T) == 4) {
            uint32_t z[4 * kVecs];
            from_word(w, off >> 2, z);
#pragma unroll
            for (int i = 0; i < kVecs; ++i) to[i] = make_uint4(z[4 * i], z[4 * i + 1], z[4 * i + 2], z[4 * i + 3]);
        } else {
            uint32_t y[5], z[4];
            const uint32_t more[8] = {w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]};
            from_word(more, off >> 2, y);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = __funnelshift_r(y[i], y[i + 1], 8 * (off & 2u));
            to[0] = make_uint4(z[0], z[1], z[2], z[3]);
        }
    }
    if ((h && !before && n) || (!whole && n))
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < n && (i < h ? !before : !whole)) Elem<T>::store(reinterpret_cast<T*>(p) + i, x[i]);
}

// Eight entries in 8 bits by their block's scale byte, and from the first of the block's lanes the byte.
template <bool FULL>
__device__ __forceinline__ void put8_coded(unsigned char* p, uint8_t* scale, uint32_t n, bool first, int dtype, uint32_t byte,
                                           const float* x) {
    uint32_t w[2];
    act8_code<8>(x, act8_down(byte), dtype, w);
    if (FULL || n == 8) {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < n) p[i] = (unsigned char)(w[i >> 2] >> (8 * (i & 3)));
    }
    if (first && (FULL || n)) *scale = (uint8_t)byte;
}

__device__ __forceinline__ uint32_t inside(uint32_t col, uint32_t cols) { return col >= cols ? 0u : min(8u, cols - col); }

// The 16 lanes that have a block agree on its scale byte: two blocks' bytes in the halves of a word.
__device__ __forceinline__ uint32_t act8_agree(uint32_t two) {
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) two = __vmaxu2(two, __shfl_xor_sync(~0u, two, o));
    return two;
}

}  // namespace ecq
