// linear.hip -- projection y = act(x W^T + b) + r, gfx950: x [M, K] and
// W [N, K] bf16 with the reduction axis contiguous, b fp32, r and y bf16 or
// fp32.  Sums, bias, activation and the residual's addition are fp32; y is
// rounded once (to nearest, at most 2^-9 relative, when it is bf16).
#include "gemm_ring.h"
#include "kernels.h"

namespace msi {

namespace {

// exact: expf and a true division, erff, tanhf
template <int ACT>
__device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == LINEAR_SILU)
        return silu(z);
    else if constexpr (ACT == LINEAR_GELU)
        return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    else if constexpr (ACT == LINEAR_GELU_TANH)
        return 0.5f * z * (1.0f + tanhf(0.79788456080286536f * (z + 0.044715f * z * z * z)));
    else
        return z;
}

// Four consecutive features n .. n + 3 of row m leave together.
template <int ACT>
__device__ __forceinline__ void store4(const LinearArgs &A, int64_t m, int n, f32x4 v)
{
    if (n >= A.N)
        return;
    if (A.vec4) {
        if (A.bias)
            v += *reinterpret_cast<const f32x4 *>(A.bias + n);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = activate<ACT>(v[i]);
        if (A.res_f32) {
            v += *reinterpret_cast<const f32x4 *>(A.res_f32 + m * A.res_stride + n);
        } else if (A.res_bf16) {
            const uint2 r = *reinterpret_cast<const uint2 *>(A.res_bf16 + m * A.res_stride + n);
            v += f32x4{__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xFFFF0000u), __uint_as_float(r.y << 16),
                       __uint_as_float(r.y & 0xFFFF0000u)};
        }
        if (A.out_f32)
            *reinterpret_cast<f32x4 *>(A.out_f32 + m * A.out_stride + n) = v;
        else
            *reinterpret_cast<uint2 *>(A.out_bf16 + m * A.out_stride + n) =
                make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < A.N) {
            float z = activate<ACT>(A.bias ? v[i] + A.bias[n + i] : v[i]);
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

// ---------------------------------------------------------------- few rows
//
// Up to 16 MT rows: bound by streaming W.  A workgroup of eight wavefronts
// owns 16 features; each wavefront an eighth of K (in whole 64-element
// pieces), so that a CU has many loads in flight however few features there
// are; the eight sums meet in LDS in a fixed order.
constexpr int FEW_WAVES = 8;

template <int ACT, int MT>
__global__ void __launch_bounds__(64 * FEW_WAVES) linear_few_kernel(LinearArgs A)
{
    __shared__ float sums[FEW_WAVES][MT][16][20];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int col = lane & 15, j = lane >> 4;
    const int n0 = int(blockIdx.x) * 16;
    const int K = A.K, pieces = (K + 63) / 64, per = (pieces + FEW_WAVES - 1) / FEW_WAVES;
    const int p0 = wave * per, p1 = min(p0 + per, pieces);
    const uint16_t *wr = A.w + int64_t(min(n0 + col, A.N - 1)) * K + 8 * j;
    const uint16_t *xr[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
        xr[t] = A.x + int64_t(min(16 * t + col, A.M - 1)) * A.x_stride + 8 * j;
    f32x4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
        acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const u32x4 zero{0, 0, 0, 0};
    auto piece = [&](int p, u32x4 (&w)[2], u32x4 (&x)[MT][2]) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int k = 64 * p + 32 * c;
            const bool in = k + 8 * j < K;           // K is a multiple of 8
            w[c] = in ? load_stream16(wr + k) : zero;
#pragma unroll
            for (int t = 0; t < MT; ++t)
                x[t][c] = in ? *reinterpret_cast<const u32x4 *>(xr[t] + k) : zero;
        }
    };
    auto mma = [&](const u32x4 (&w)[2], const u32x4 (&x)[MT][2]) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int t = 0; t < MT; ++t)
                acc[t] = mfma16(as_bf16x8(w[c]), as_bf16x8(x[t][c]), acc[t]);
    };
    constexpr int U = MT == 1 ? 4 : 2;               // pieces in flight
    int p = p0;
    for (; p + U <= p1; p += U) {
        u32x4 w[U][2], x[U][MT][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
            piece(p + u, w[u], x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            mma(w[u], x[u]);
    }
    for (; p < p1; ++p) {
        u32x4 w[2], x[MT][2];
        piece(p, w, x);
        mma(w, x);
    }
    // lane (col, j) holds features 4 j .. 4 j + 3 of row col
#pragma unroll
    for (int t = 0; t < MT; ++t)
        *reinterpret_cast<f32x4 *>(&sums[wave][t][col][4 * j]) = acc[t];
    __syncthreads();
    if (wave < MT) {
        f32x4 v = *reinterpret_cast<const f32x4 *>(&sums[0][wave][col][4 * j]);
#pragma unroll
        for (int u = 1; u < FEW_WAVES; ++u)
            v += *reinterpret_cast<const f32x4 *>(&sums[u][wave][col][4 * j]);
        const int m = 16 * wave + col;
        if (m < A.M)
            store4<ACT>(A, m, n0 + 4 * j, v);
    }
}

// ---------------------------------------------------------------- tiles
//
// BM rows x TN features a workgroup; K in stages of 64 elements copied
// straight into one of NBUF LDS buffers, NBUF - 1 in flight; WR x WC
// wavefronts of 16 x 16 x 32 MFMAs with the weights as the A operand, so a lane
// ends with four consecutive features of a row.  Slot s of stage row r holds
// 16-byte chunk s ^ ((r / 2) % 8), which spreads a fragment read over the banks.
template <int BM_, int TN_, int WR_, int WC_, int NBUF_, int WPC_>
struct LinearShape {
    static constexpr int BM = BM_, TN = TN_, WR = WR_, WC = WC_, NBUF = NBUF_, WPC = WPC_;
    static constexpr int WAVES = WR * WC, THREADS = 64 * WAVES;
    static constexpr int BK = 64, ROWB = BK * 2;
    static constexpr int STAGE = (BM + TN) * ROWB;
    static constexpr int MB = BM / WR / 16, NB = TN / WC / 16;
    static constexpr int LA = BM / 8 / WAVES, LB = TN / 8 / WAVES, LPS = LA + LB;
    static constexpr size_t LDS = size_t(NBUF) * STAGE;
    static_assert(BM % (8 * WAVES) == 0 && TN % (8 * WAVES) == 0 && LDS * WPC <= 160 * 1024, "");
};
using Tile64 = LinearShape<64, 64, 2, 2, 4, 2>;
using Tile128 = LinearShape<128, 128, 2, 2, 2, 2>;
using Tile256 = LinearShape<256, 256, 4, 2, 2, 1>;

template <int ACT, class S>
__global__ void __launch_bounds__(S::THREADS, S::WPC * S::WAVES / 4) linear_tile_kernel(LinearArgs A)
{
    constexpr int BM = S::BM, TN = S::TN, NBUF = S::NBUF, WAVES = S::WAVES, ROWB = S::ROWB, STAGE = S::STAGE, MB = S::MB,
                  NB = S::NB, LA = S::LA, LB = S::LB, LPS = S::LPS;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds8[];
    const int ntn = (A.N + TN - 1) / TN;
    const int t = xcd_swizzle(int(blockIdx.x), int(gridDim.x));
    const int m0 = (t / ntn) * BM, n0 = (t % ntn) * TN;
    const int K = A.K;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int rl = lane >> 3, sl = lane & 7;
    const int vm = min(BM, A.M - m0), vn = min(TN, A.N - n0);
    // offsets from the tile's first rows (under 2^31: the caller's strides are bounded)
    uint32_t aoff[LA], boff[LB];
    int last = 0;                                 // bit i: A copy i of the last stage lies past K; bit 16 + i: B copy i
    const int nstage = (K + 63) / 64, tail = K - 64 * (nstage - 1);
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int r = 8 * (WAVES * i + wave) + rl, ch = sl ^ ((r >> 1) & 7);
        aoff[i] = uint32_t(min(r, vm - 1)) * uint32_t(A.x_stride * 2) + uint32_t(ch << 4);
        last |= int(8 * ch >= tail) << i;
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int r = 8 * (WAVES * i + wave) + rl, ch = sl ^ ((r >> 1) & 7);
        boff[i] = uint32_t(min(r, vn - 1)) * uint32_t(K * 2) + uint32_t(ch << 4);
        last |= int(8 * ch >= tail) << (16 + i);
    }
    const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(A.x + int64_t(m0) * A.x_stride), 0, 0x7fffffff, ring::RSRC_FLAGS);
    const __amdgpu_buffer_rsrc_t br = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(A.w + int64_t(n0) * K), 0,
                                                                        0x7fffffff, ring::RSRC_FLAGS);
    auto issue = [&](int stage, int buf) {
        uint8_t *b = lds8 + buf * STAGE;
        // an offset past the buffer's end reads nothing and leaves zeros in LDS
        const bool edge = stage == nstage - 1 && tail < 64;
#pragma unroll
        for (int i = 0; i < LB; ++i)
            dma16_lds(br, b + BM * ROWB + (WAVES * i + wave) * 1024,
                      edge && (last >> (16 + i) & 1) ? 0x80000000u : boff[i] + uint32_t(stage * ROWB), 0);
#pragma unroll
        for (int i = 0; i < LA; ++i)
            dma16_lds(ar, b + (WAVES * i + wave) * 1024,
                      edge && (last >> i & 1) ? 0x80000000u : aoff[i] + uint32_t(stage * ROWB), 0);
    };
    const int r16 = lane & 15, g = lane >> 4;
    const int wm = wave / S::WC, wn = wave % S::WC;
    f32x4 acc[NB][MB];
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
        for (int q = 0; q < MB; ++q)
            acc[a][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto compute = [&](int buf) {
        const uint8_t *b = lds8 + buf * STAGE;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const uint32_t fo = uint32_t(r16 * ROWB + (((4 * kb + g) ^ ((r16 >> 1) & 7)) << 4));
            u32x4 fw[NB], fx[MB];
#pragma unroll
            for (int a = 0; a < NB; ++a)
                fw[a] = *reinterpret_cast<const u32x4 *>(b + (BM + (wn * NB + a) * 16) * ROWB + fo);
#pragma unroll
            for (int q = 0; q < MB; ++q)
                fx[q] = *reinterpret_cast<const u32x4 *>(b + (wm * MB + q) * 16 * ROWB + fo);
#pragma unroll
            for (int q = 0; q < MB; ++q)
#pragma unroll
                for (int a = 0; a < NB; ++a)
                    acc[a][q] = mfma16(as_bf16x8(fw[a]), as_bf16x8(fx[q]), acc[a][q]);
        }
    };
    constexpr int AHEAD = NBUF - 1;
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
        if (j < nstage)
            issue(j, j);
    int cur = 0, nxt = AHEAD;
    for (int s = 0; s < nstage; ++s) {
        // stage s has landed; the buffer of stage s + AHEAD was last read at s - 1
        if (s + AHEAD <= nstage)
            __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(LPS * (AHEAD - 1)));
        else
            __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(0));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + AHEAD < nstage)
            issue(s + AHEAD, nxt);
        compute(cur);
        cur = cur == NBUF - 1 ? 0 : cur + 1;
        nxt = nxt == NBUF - 1 ? 0 : nxt + 1;
    }
#pragma unroll
    for (int q = 0; q < MB; ++q) {
        const int row = (wm * MB + q) * 16 + r16;
        if (row < vm)
#pragma unroll
            for (int a = 0; a < NB; ++a)
                store4<ACT>(A, m0 + row, n0 + (wn * NB + a) * 16 + 4 * g, acc[a][q]);
    }
}

template <int ACT, class S>
hipError_t launch_tile(const LinearArgs &A, hipStream_t st)
{
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(linear_tile_kernel<ACT, S>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, int(S::LDS));
    if (e != hipSuccess)
        return e;
    const int64_t tiles = int64_t((A.M + S::BM - 1) / S::BM) * ((A.N + S::TN - 1) / S::TN);
    launch_k(linear_tile_kernel<ACT, S>, unsigned(tiles), S::THREADS, S::LDS, st, A);
    return hipGetLastError();
}

template <int ACT>
hipError_t launch_act(const LinearArgs &A, hipStream_t st)
{
    if (A.M <= 32) {
        const unsigned grid = unsigned((A.N + 15) / 16);
        if (A.M <= 16)
            launch_k(linear_few_kernel<ACT, 1>, grid, 64 * FEW_WAVES, 0, st, A);
        else
            launch_k(linear_few_kernel<ACT, 2>, grid, 64 * FEW_WAVES, 0, st, A);
        return hipGetLastError();
    }
    auto tiles = [&](int64_t b) { return (A.M + b - 1) / b * ((A.N + b - 1) / b); };
    if (tiles(256) >= 256)
        return launch_tile<ACT, Tile256>(A, st);
    if (tiles(128) >= 256)
        return launch_tile<ACT, Tile128>(A, st);
    return launch_tile<ACT, Tile64>(A, st);
}

}  // namespace

hipError_t launch_linear(const LinearArgs &A, int act, hipStream_t st)
{
    switch (act) {
    case LINEAR_SILU: return launch_act<LINEAR_SILU>(A, st);
    case LINEAR_GELU: return launch_act<LINEAR_GELU>(A, st);
    case LINEAR_GELU_TANH: return launch_act<LINEAR_GELU_TANH>(A, st);
    default: return launch_act<LINEAR_NONE>(A, st);
    }
}

}  // namespace msi
