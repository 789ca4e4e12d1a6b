// kv_device.h -- device helpers of the cache's kernels.
#pragma once

#include "common.h"
#include "kv_common.h"

namespace msi {

__device__ __forceinline__ KvSeq kv_seq(const KvSeqs &s, int i, bool cached)
{
    const int row0 = s.cu ? __builtin_amdgcn_readfirstlane(s.cu[i]) : 0;
    const int row1 = s.cu ? __builtin_amdgcn_readfirstlane(s.cu[i + 1]) : 0;
    const int len = __builtin_amdgcn_readfirstlane(s.lens[i]);
    return kv_check_seq(row0, row1, len, s.n_rows, s.max_rows, s.max_len, cached);
}

__device__ __forceinline__ void kv_raise(uint32_t *status, uint32_t bits)
{
    if (status && bits)
        atomicOr(status, bits);
}

__device__ __forceinline__ void unpack_bf16x8(const u32x4 &w, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// Four codes of a word as floats.
template <int FMT>
__device__ __forceinline__ f32x4 kv_unpack4(uint32_t w)
{
    if constexpr (FMT == KV_INT8) {
        return f32x4{float(int8_t(w & 0xFF)), float(int8_t((w >> 8) & 0xFF)), float(int8_t((w >> 16) & 0xFF)),
                     float(int8_t(w >> 24))};
    } else {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), false);
        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), true);
        return f32x4{lo[0], lo[1], hi[0], hi[1]};
    }
}

// Four finite floats, already divided by their scale, as codes: clamped to the
// largest code, rounded to nearest, ties to even (at most half a step of the
// format: 2^-4 of the value for e4m3, half the scale for int8).
template <int FMT>
__device__ __forceinline__ uint32_t kv_pack4(float a, float b, float c, float d)
{
    constexpr float Q = FMT == KV_INT8 ? 127.0f : 448.0f;
    a = fminf(fmaxf(a, -Q), Q), b = fminf(fmaxf(b, -Q), Q), c = fminf(fmaxf(c, -Q), Q), d = fminf(fmaxf(d, -Q), Q);
    if constexpr (FMT == KV_INT8) {
        return uint32_t(uint8_t(int(rintf(a)))) | uint32_t(uint8_t(int(rintf(b)))) << 8 |
               uint32_t(uint8_t(int(rintf(c)))) << 16 | uint32_t(uint8_t(int(rintf(d)))) << 24;
    } else {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
    }
}

// Largest of one value per thread of a 256-thread workgroup, the same in every
// thread.  `part`: 4 words.  A caller that reuses `part` puts a barrier first.
__device__ __forceinline__ float block_max256(float v, float *part)
{
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}

}  // namespace msi
