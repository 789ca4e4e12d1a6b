// linear_epilogue.h -- what the projections (linear.hip, linear_q4.hip) have in
// common: their activations, the way of their rows to memory and the order of
// their tiles.
#pragma once

#include "gemm_ring.h"
#include "kernels.h"

namespace msi {

// SiLU and the tanh form share z / (1 + e^-u) (u = z, or twice the tanh's
// argument), with expf and a true division.  GELU is max(z, 0) - |z| Phi(-|z|),
// Phi(-x) = e^(-x^2 / 2) t P(t) with t = 1 / (1 + 0.35 x): P, of degree 8, is a
// minimax fit of our own to the relative error (4.3e-8 over 0 <= x <= 14 with
// its coefficients in fp32), so the negative tail is as good as the rest.  What
// rounding adds stays under (z^2 + 4) 2^-22 of the value (z^2 2^-24 of it is
// what a z rounded to fp32 leaves); over normal arguments 3.6e-8 of the root mean
// square, 0.5 z (1 + erff) 3.8e-8.
template <int ACT>
__device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == LINEAR_SILU) {
        return silu(z);
    } else if constexpr (ACT == LINEAR_GELU_TANH) {
        return z / (1.0f + expf(-1.5957691216057308f * (z + 0.044715f * z * z * z)));
    } else if constexpr (ACT == LINEAR_GELU) {
        constexpr float P[9] = {0.13962140679359436f, 0.13986186683177948f, 0.11983285844326019f, 0.10550802946090698f,
                                -0.02310989610850811f, 0.15917424857616425f, -0.2557143270969391f, 0.1439717411994934f,
                                -0.029145939275622368f};
        const float x = fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(0.35f, x, 1.0f));
        float p = P[8];
#pragma unroll
        for (int i = 7; i >= 0; --i)
            p = fmaf(p, t, P[i]);
        const float q = p * t * __builtin_amdgcn_exp2f(-0.72134752044448170f * (z * z));
        return fmaf(-fminf(x, 3.0e38f), q, fmaxf(z, 0.0f));
    } else {
        return z;
    }
}

// Rows may start at any element: with an odd N, or a stride that is no multiple of four, a lane's four features are
// still one access, aligned only to their type (1000 x 5001 outputs of K 1000, bf16: 24.2 us; one by one 27.1).
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;
typedef __attribute__((ext_vector_type(2), aligned(2))) uint32_t bf16x4_any;

// Residual of features n .. n + 3 of row m.
__device__ __forceinline__ f32x4 residual4(const LinearArgs &A, int64_t m, int n)
{
    if (A.res_f32)
        return *reinterpret_cast<const f32x4_any *>(A.res_f32 + m * A.res_stride + n);
    const bf16x4_any r = *reinterpret_cast<const bf16x4_any *>(A.res_bf16 + m * A.res_stride + n);
    return f32x4{__uint_as_float(r[0] << 16), __uint_as_float(r[0] & 0xFFFF0000u), __uint_as_float(r[1] << 16),
                 __uint_as_float(r[1] & 0xFFFF0000u)};
}

// Features n .. n + 3 of row m leave: act(v + bias) + residual; bias: their
// four (zero past N).  `res`: their residual, where all four are inside.  PAST:
// stored past the caches, where the tiles make more than the L2s could hold for
// whoever reads them next (4096 x 8192 bf16 of K 2048 with GELU 144.1 -> 136.6
// us, fp32 of K 1024 143.3 -> 135.4; 64 rows of 8192 and the product that reads
// them would go from 27.6 to 28.9).
template <int ACT, bool PAST>
__device__ __forceinline__ void store4(const LinearArgs &A, int64_t m, int n, f32x4 v, const f32x4 &bias, const f32x4 &res)
{
    v += bias;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = activate<ACT>(v[i]);
    if (n + 4 <= A.N) {
        v += res;
        auto store = [](auto *p, auto w) {
            if constexpr (PAST)
                __builtin_nontemporal_store(w, p);
            else
                *p = w;
        };
        if (A.out_f32)
            store(reinterpret_cast<f32x4_any *>(A.out_f32 + m * A.out_stride + n), static_cast<f32x4_any>(v));
        else
            store(reinterpret_cast<bf16x4_any *>(A.out_bf16 + m * A.out_stride + n),
                  bf16x4_any{pack_bf16x2_hw(v[0], v[1]), pack_bf16x2_hw(v[2], v[3])});
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (n + i < A.N) {
            float z = v[i];
            if (A.res_f32)
                z += A.res_f32[m * A.res_stride + n + i];
            else if (A.res_bf16)
                z += bf16_to_f32(A.res_bf16[m * A.res_stride + n + i]);
            if (A.out_f32)
                A.out_f32[m * A.out_stride + n + i] = z;
            else
                A.out_bf16[m * A.out_stride + n + i] = f32_to_bf16(z);
        }
}

__device__ __forceinline__ f32x4 bias4(const LinearArgs &A, int n)
{
    f32x4 b{0.f, 0.f, 0.f, 0.f};
    if (A.bias)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            b[i] = n + i < A.N ? A.bias[n + i] : 0.0f;
    return b;
}

// A wavefront's block of 16 MB rows x 16 NB features leaves through LDS of its
// own (`mine`, 16 rows at a time), so that rows are written in runs of 16 NB
// features and the epilogue's code is small.  The residual comes the same way:
// read 16 rows ahead, so that a group's reads are in flight while the one before
// is stored (2048 x 6144 of K 1024, fp32 residual and output: 71.5 -> 52.6 us).  Lane (row,
// group) of an MFMA block holds four consecutive features of one row.
template <int NB>
constexpr int STORE_LDS = 2 * 16 * (16 * NB + 4);      // words of a wavefront

template <int ACT, bool PAST, int NB, int MB>
__device__ __forceinline__ void store_block(const LinearArgs &A, float *mine, const f32x4 (&acc)[NB][MB], int m0, int rows,
                                            int n0)
{
    constexpr int W = 16 * NB, LD = W + 4, LPR = W / 4, RPI = 64 / LPR;   // lanes of a row, rows of a pass
    constexpr int IT = 16 / RPI;
    const int lane = threadIdx.x & 63;
    const int n = n0 + 4 * (lane % LPR), r0 = lane / LPR;
    const f32x4 bias = bias4(A, n);
    const bool residual = A.res_f32 || A.res_bf16;
    float *const there = mine + 16 * LD;
    f32x4 res[IT];
    auto fetch = [&](int q) {
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            const int m = 16 * q + r0 + k * RPI;
            if (m < rows && n + 4 <= A.N)
                res[k] = residual4(A, int64_t(m0) + m, n);
        }
    };
    if (residual)
        fetch(0);
#pragma unroll
    for (int q = 0; q < MB; ++q) {
#pragma unroll
        for (int a = 0; a < NB; ++a)
            *reinterpret_cast<f32x4 *>(mine + (lane & 15) * LD + 16 * a + 4 * (lane >> 4)) = acc[a][q];
        if (residual) {
#pragma unroll
            for (int k = 0; k < IT; ++k)
                *reinterpret_cast<f32x4 *>(there + (r0 + k * RPI) * LD + 4 * (lane % LPR)) = res[k];
            if (q + 1 < MB)
                fetch(q + 1);
        }
        // (a wavefront's LDS operations are in order; the fences keep the compiler from moving them)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
#pragma unroll 2
        for (int r = r0; r < 16; r += RPI) {
            const int m = 16 * q + r, at = r * LD + 4 * (lane % LPR);
            if (m < rows && n < A.N)
                store4<ACT, PAST>(A, int64_t(m0) + m, n, *reinterpret_cast<const f32x4 *>(mine + at), bias,
                            residual ? *reinterpret_cast<const f32x4 *>(there + at) : f32x4{0.f, 0.f, 0.f, 0.f});
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

// Tile t of a launch as (row tile, feature tile): bands of 8 row tiles, down
// the band before the next feature tile, so that the tiles one XCD works on
// together (xcd_swizzle gives it a contiguous range) share rows on both sides.
__device__ __forceinline__ int2 tile_at(int t, int ntm, int ntn)
{
    const int band = t / (8 * ntn), in = t - band * 8 * ntn;
    const int height = min(8, ntm - 8 * band);
    return make_int2(8 * band + in % height, in / height);
}

}  // namespace msi
