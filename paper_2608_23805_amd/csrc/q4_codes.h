// q4_codes.h -- 4-bit codes (two's complement, element e of a word at bits 4e) as
// MFMA operands, and their fp16 scales: the int4 experts (experts_q4.hip) and
// the projection with 4-bit weights (linear_q4.hip).
#pragma once

#include "common.h"

namespace msi {

// 8 nibbles (element e at bits 4e..4e+3, two's complement q) -> 8 exact bf16
// values 136 + q: the bits 0x4300 | u are the bf16 128 + u, u = q + 8 = the
// nibble with its top bit flipped.  Byte permutes place the nibbles (even
// elements from the low halves of the bytes, odd ones from the high halves)
// under the 0x43 bytes: nine operations per 8 values.
__device__ __forceinline__ bf16x8 unpack_q4_136(uint32_t w)
{
    const uint32_t e = (w ^ 0x08080808u) & 0x0F0F0F0Fu;           // u of elements 0, 2, 4, 6
    const uint32_t o = ((w >> 4) ^ 0x08080808u) & 0x0F0F0F0Fu;    // u of elements 1, 3, 5, 7
    const uint32_t lo = __builtin_amdgcn_perm(o, e, 0x05010400u);  // bytes u0 u1 u2 u3
    const uint32_t hi = __builtin_amdgcn_perm(o, e, 0x07030602u);  // bytes u4 u5 u6 u7
    u32x4 r;
    r[0] = __builtin_amdgcn_perm(0x43434343u, lo, 0x04010400u);
    r[1] = __builtin_amdgcn_perm(0x43434343u, lo, 0x04030402u);
    r[2] = __builtin_amdgcn_perm(0x43434343u, hi, 0x04010400u);
    r[3] = __builtin_amdgcn_perm(0x43434343u, hi, 0x04030402u);
    return __builtin_bit_cast(bf16x8, r);
}

// 8 nibbles (element e at bits 4e..4e+3, two's complement q) -> 8 exact bf16
// values q / 16: the 4-bit integer conversion reads the low nibble of a byte
// and returns q / 16 in binary32, whose top half holds it; thirteen operations
// per 8 values.
__device__ __forceinline__ bf16x8 unpack_q4_16th(uint32_t w)
{
    uint32_t o = w >> 4;
    asm("" : "+v"(o));          // (one shift; the conversions then pick their byte of it)
    u32x4 r;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const float fe = __builtin_amdgcn_cvt_off_f32_i4(int((w >> (8 * h)) & 0xFFu));   // element 2h
        const float fo = __builtin_amdgcn_cvt_off_f32_i4(int((o >> (8 * h)) & 0xFFu));   // element 2h + 1
        r[h] = __builtin_amdgcn_perm(__float_as_uint(fo), __float_as_uint(fe), 0x07060302u);
    }
    return __builtin_bit_cast(bf16x8, r);
}

__device__ __forceinline__ float half_to_float(uint16_t h) { return float(__builtin_bit_cast(_Float16, h)); }

}  // namespace msi
