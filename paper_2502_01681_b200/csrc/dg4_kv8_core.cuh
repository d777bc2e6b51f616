// One row of the 8-bit K | V table, as the kernels that write, read and attend over it see it.
//
// A row of d = 128 is 16 pieces of 8 elements, one per lane; piece p holds its 8 K codes and its 8 V codes side by
// side, so that one 16-byte load brings a lane both.  Behind the 256 code bytes stand 16 pairs of scale exponents
// (K, V), one pair per head (unused pairs are zero): 288 bytes, nine 32-byte sectors.
//
// A code is an e4m3 number c; the value it stands for is c * 2^(b - 127) with b the exponent byte of its head.  The
// scale of a head's slice of a row is the smallest power of two, no smaller than 2^-127, that brings its largest
// magnitude to at most 448 (the largest e4m3 number).  A power of two costs nothing in precision against max / 448:
// e4m3 is a floating format, its relative step does not depend on where in its range a value falls; and it makes
// the scaling exact, so the only rounding of a value is the one to 3 mantissa bits.
// A slice that holds an infinity or a NaN gets b = 255 and codes 0x7f (NaN): all of it reads back as NaN.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "dg4_attn_core.cuh"

namespace kv8 {

constexpr int kCodeBytes = 256;
constexpr int kLanes = 16;                    // lanes per row
constexpr int kEl = 8;                        // elements of K (and of V) per lane

// 8 consecutive elements of a bf16 or fp32 row
template <bool BF16>
__device__ __forceinline__ void store8(void* row, int sub, const float* f) {
    if (BF16) {
        attn::st_piece_stream((char*)row + sub * 16, attn::Elem<true>::pack(f));
    } else {
        attn::st_piece_stream((char*)row + sub * 32, attn::Elem<false>::pack(f));
        attn::st_piece_stream((char*)row + sub * 32 + 16, attn::Elem<false>::pack(f + 4));
    }
}

// exponent byte of a slice whose largest magnitude has the bit pattern `top`: with top = m * 2^e, 1 <= m < 2, the
// smallest k with m * 2^e <= 1.75 * 2^8 * 2^k is e - 8, or e - 7 if m > 1.75
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    if (top >= 0x7f800000u) return 255u;
    const int b = (int)((top + 0x1fffffu) >> 23) - 8;
    return (uint32_t)(b > 0 ? b : 0);
}
// 2^(b - 127) of the K byte (low) and of the V byte (high) of a head's pair.  2^-127 (b = 0) is subnormal in fp32 and
// has the pattern 0x00400000, below that of every b > 0, so a maximum puts it in; 255 gives an infinity, which the NaN
// codes that go with it turn into NaN.
__device__ __forceinline__ float scale_k(uint32_t pair) { return __uint_as_float(max((pair << 23) & 0x7f800000u, 0x00400000u)); }
__device__ __forceinline__ float scale_v(uint32_t pair) { return __uint_as_float(max((pair << 15) & 0x7f800000u, 0x00400000u)); }
// The same times 2, which is a normal number for b = 0 too (and -0 for 255: NaN with the NaN codes all the same): a
// mask and a multiply-add
__device__ __forceinline__ float twice_scale_k(uint32_t pair) { return __uint_as_float((pair & 0xffu) * 0x00800000u + 0x00800000u); }
__device__ __forceinline__ float twice_scale_v(uint32_t pair) { return __uint_as_float((pair & 0xff00u) * 0x00008000u + 0x00800000u); }
// log2 of the V scale: the byte stands in the mantissa of 2^23 + 256 b
__device__ __forceinline__ float log2_scale_v(uint32_t pair) { return fmaf(__uint_as_float(0x4b000000u | (pair & 0xff00u)), 0.00390625f, -32895.f); }

// 8 values -> 8 codes.  The slice's scale is 2^(b - 127), so the factor 2^(127 - b) has the exponent field 254 - b;
// b <= 247 for a finite slice, so the factor is a normal number and the product is exact (or far below e4m3's range).
__device__ __forceinline__ void encode8(const float* f, uint32_t b, uint32_t* out) {
    if (b == 255u) {
        out[0] = out[1] = 0x7f7f7f7fu;
        return;
    }
    const float inv = __uint_as_float((254u - b) << 23);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint16_t lo, hi;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(f[4 * i + 1] * inv), "f"(f[4 * i] * inv));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(f[4 * i + 3] * inv), "f"(f[4 * i + 2] * inv));
        out[i] = (uint32_t)lo | ((uint32_t)hi << 16);
    }
}

// 4 codes -> 2 pairs of fp16 (every e4m3 number is an fp16 number), or 4 floats.  (The conversion takes the low half of a
// register only.  Bringing the high half down by a wide multiplication, off the conversions' pipe, was slower: 261
// against 244 us for the attention over 1.01M two-hop cones.)
__device__ __forceinline__ void decode4_half(uint32_t w, uint32_t* h) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(h[0]), "=r"(h[1]) : "r"(w));
}
__device__ __forceinline__ void decode4(uint32_t w, float* f) {
    uint32_t h[2];
    decode4_half(w, h);
    const float2 x = __half22float2(*reinterpret_cast<__half2*>(&h[0]));
    const float2 y = __half22float2(*reinterpret_cast<__half2*>(&h[1]));
    f[0] = x.x; f[1] = x.y; f[2] = y.x; f[3] = y.y;
}

__device__ __forceinline__ uint32_t ld_pair(const void* p) {          // a head's pair of exponent bytes
    uint16_t r;
    asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(r) : "l"(p));
    return r;
}

}  // namespace kv8
