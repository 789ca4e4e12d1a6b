// linear.hip -- projection y = act(x W^T + b) + r, gfx950: x [M, K] and
// W [N, K] bf16 with the reduction axis contiguous, b fp32, r and y bf16 or
// fp32.  Sums, bias, activation and the residual's addition are fp32; y is
// rounded once (to nearest, at most 2^-8 relative, when it is bf16).
#include "gemm_ring.h"
#include "kernels.h"

namespace msi {

namespace {

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

// ---------------------------------------------------------------- tiles
//
// BM rows x TN features a workgroup; K in stages of 64 KG elements copied
// straight into one of NBUF LDS buffers, NBUF - 1 in flight.  KG groups of WR x
// WC wavefronts each multiply their own 64 elements of a stage (16 x 16 x 32
// MFMAs with the weights as the A operand, so a lane ends with four
// consecutive features of a row) and their sums meet in LDS in a fixed order.
// Without the groups a stage's barrier, copies, fragment reads and few MFMAs
// follow each other with nothing beside them.  Slot s of stage row r holds
// 16-byte chunk s ^ ((r / 2) % 8), which spreads a fragment read over the banks.
template <int BM_, int TN_, int WR_, int WC_, int KG_, int NBUF_, int WPC_>
struct LinearShape {
    static constexpr int BM = BM_, TN = TN_, WR = WR_, WC = WC_, KG = KG_, NBUF = NBUF_, WPC = WPC_;
    static constexpr int WAVES = WR * WC * KG, THREADS = 64 * WAVES;
    static constexpr int ROWB = 128, SLICE = (BM + TN) * ROWB, STAGE = KG * SLICE;
    static constexpr int MB = BM / WR / 16, NB = TN / WC / 16;
    static constexpr int LA = KG * BM / 8 / WAVES, LB = KG * TN / 8 / WAVES, LPS = LA + LB;
    static constexpr int OUT = WR * WC * STORE_LDS<NB> * 4, SUMS = OUT + (KG - 1) * BM * TN * 4;   // LDS of the epilogue
    static constexpr size_t LDS = NBUF * STAGE > SUMS ? NBUF * STAGE : SUMS;
    static_assert(KG * BM % (8 * WAVES) == 0 && KG * TN % (8 * WAVES) == 0 && LDS * WPC <= 160 * 1024, "");
    static_assert(LA <= 16 && LB <= 16 && LPS * (NBUF - 2) < 64, "");
};

template <int ACT, class S>
__global__ void __launch_bounds__(S::THREADS, S::WPC * S::WAVES / 4) linear_tile_kernel(LinearArgs A)
{
    constexpr int BM = S::BM, TN = S::TN, NBUF = S::NBUF, WAVES = S::WAVES, ROWB = S::ROWB, STAGE = S::STAGE, MB = S::MB,
                  NB = S::NB, LA = S::LA, LB = S::LB, LPS = S::LPS, KG = S::KG;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds8[];
    const int2 at = tile_at(xcd_swizzle(int(blockIdx.x), int(gridDim.x)), (A.M + BM - 1) / BM, (A.N + TN - 1) / TN);
    const int m0 = at.x * BM, n0 = at.y * TN;
    const int K = A.K;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int rl = lane >> 3, sl = lane & 7;
    const int vm = min(BM, A.M - m0), vn = min(TN, A.N - n0);
    // offsets from the tile's first rows (under 2^31: the caller's strides are bounded); copy c of the workgroup
    // brings 8 rows of slice c / (BM / 8)
    uint32_t aoff[LA], boff[LB];
    int last = 0;                                 // bit i: A copy i of the last stage lies past K; bit 16 + i: B copy i
    const int nstage = (K + 64 * KG - 1) / (64 * KG), tail = K - 64 * KG * (nstage - 1);
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int c = WAVES * i + wave, r = 8 * (c % (BM / 8)) + rl, ch = 8 * (c / (BM / 8)) + (sl ^ ((r >> 1) & 7));
        aoff[i] = uint32_t(min(r, vm - 1)) * uint32_t(A.x_stride * 2) + uint32_t(ch << 4);
        last |= int(8 * ch >= tail) << i;
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int c = WAVES * i + wave, r = 8 * (c % (TN / 8)) + rl, ch = 8 * (c / (TN / 8)) + (sl ^ ((r >> 1) & 7));
        boff[i] = uint32_t(min(r, vn - 1)) * uint32_t(K * 2) + uint32_t(ch << 4);
        last |= int(8 * ch >= tail) << (16 + i);
    }
    const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(A.x + int64_t(m0) * A.x_stride), 0, 0x7fffffff, ring::RSRC_FLAGS);
    const __amdgpu_buffer_rsrc_t br = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(A.w + int64_t(n0) * K), 0,
                                                                        0x7fffffff, ring::RSRC_FLAGS);
    // a stage: the slices' A rows (KG BM of them), then their B rows
    auto issue = [&](int stage, int buf) {
        uint8_t *b = lds8 + buf * STAGE;
        // an offset past the buffer's end reads nothing and leaves zeros in LDS
        const bool edge = stage == nstage - 1 && tail < 64 * KG;
        const uint32_t kb = uint32_t(stage * (KG * ROWB));
#pragma unroll
        for (int i = 0; i < LB; ++i)
            dma16_lds(br, b + KG * BM * ROWB + (WAVES * i + wave) * 1024,
                      edge && (last >> (16 + i) & 1) ? 0x80000000u : boff[i] + kb, 0);
#pragma unroll
        for (int i = 0; i < LA; ++i)
            dma16_lds(ar, b + (WAVES * i + wave) * 1024, edge && (last >> i & 1) ? 0x80000000u : aoff[i] + kb, 0);
    };
    const int r16 = lane & 15, g = lane >> 4;
    const int grp = wave / (S::WR * S::WC), wi = wave % (S::WR * S::WC);
    const int wm = wi / S::WC, wn = wi % S::WC;
    f32x4 acc[NB][MB];
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
        for (int q = 0; q < MB; ++q)
            acc[a][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto compute = [&](int buf) {
        const uint8_t *xa = lds8 + buf * STAGE + (grp * BM + wm * MB * 16) * ROWB;
        const uint8_t *wb = lds8 + buf * STAGE + (KG * BM + grp * TN + wn * NB * 16) * ROWB;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const uint32_t fo = uint32_t(r16 * ROWB + (((4 * kb + g) ^ ((r16 >> 1) & 7)) << 4));
            u32x4 fw[NB], fx[MB];
#pragma unroll
            for (int a = 0; a < NB; ++a)
                fw[a] = *reinterpret_cast<const u32x4 *>(wb + a * 16 * ROWB + fo);
#pragma unroll
            for (int q = 0; q < MB; ++q)
                fx[q] = *reinterpret_cast<const u32x4 *>(xa + q * 16 * ROWB + fo);
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
        // stage s has landed; the buffer of stage s + AHEAD was last read at s - 1, by reads that are waited for as well
        // (LGKM_DONE: no LDS operation of this wavefront in flight)
        constexpr int LGKM_DONE = ~(0xF << 8);
        if (s + AHEAD <= nstage)
            __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(LPS * (AHEAD - 1)) & LGKM_DONE);
        else
            __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(0) & LGKM_DONE);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + AHEAD < nstage)
            issue(s + AHEAD, nxt);
        compute(cur);
        cur = cur == NBUF - 1 ? 0 : cur + 1;
        nxt = nxt == NBUF - 1 ? 0 : nxt + 1;
    }
    __syncthreads();                              // every fragment has been read: LDS changes its use
    if constexpr (KG > 1) {
        // groups 1 .. leave their sums, lane by lane; group 0 adds them in order
        f32x4 *sums = reinterpret_cast<f32x4 *>(lds8 + S::OUT);
        constexpr int PER = S::WR * S::WC * MB * NB * 64;
        if (grp > 0) {
#pragma unroll
            for (int a = 0; a < NB; ++a)
#pragma unroll
                for (int q = 0; q < MB; ++q)
                    sums[(grp - 1) * PER + ((wi * NB + a) * MB + q) * 64 + lane] = acc[a][q];
        }
        __syncthreads();
        if (grp > 0)
            return;
        for (int o = 0; o < KG - 1; ++o)
#pragma unroll
            for (int a = 0; a < NB; ++a)
#pragma unroll
                for (int q = 0; q < MB; ++q)
                    acc[a][q] += sums[o * PER + ((wi * NB + a) * MB + q) * 64 + lane];
    }
    store_block<ACT, false, NB, MB>(A, reinterpret_cast<float *>(lds8) + wi * STORE_LDS<NB>, acc, m0 + wm * MB * 16,
                             vm - wm * MB * 16, n0 + wn * NB * 16);
}

// ---------------------------------------------------------------- 256 x 256 tiles
//
// Many tiles: bound by the matrix cores.  Eight wavefronts as 4 (rows) x 2
// (features), each 64 rows x 128 features; K in stages of 64 elements through
// two LDS buffers, rows of 128 bytes with the tiles' slots.  A stage is two
// halves of 32 elements: the fragments of the next half are read between the
// MFMAs of this one, so by the middle of a stage all of its fragments are in
// registers and, after the one barrier, its buffer takes the stage after next.
// 4096 rows, K 2048, N 8192, call after call: 111 us, 1240 TFLOP/s (with GELU 124, SiLU 130, GELU by tanh
// 133; the library's product alone 95).  About 10 us a tile are its start and its
// rows' way out, which nothing overlaps.  (At lower clocks, 125 us: stages of 32
// elements in rows of 64 bytes, whose reads meet on banks: 133.6 us; four
// wavefronts of 128 x 128: 187; without reads between the MFMAs: 132.)
template <int ACT>
__global__ void __launch_bounds__(512, 2) linear_wide_kernel(LinearArgs A)
{
    constexpr int T = 256, ROWB = 128, STAGE = 2 * T * ROWB, OUT = 8 * STORE_LDS<8> * 4;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE > OUT ? 2 * STAGE : OUT];
    const int2 at = tile_at(xcd_swizzle(int(blockIdx.x), int(gridDim.x)), (A.M + T - 1) / T, (A.N + T - 1) / T);
    const int m0 = at.x * T, n0 = at.y * T;
    const int K = A.K;
    const int vm = min(T, A.M - m0), vn = min(T, A.N - n0);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    // copy i of this wavefront covers rows 8 (8 i + wave) + lane / 8; lane % 8 is the 16-byte slot it fills
    const int ch = (lane & 7) ^ (lane >> 4 & 3) ^ ((wave & 1) << 2);
    uint32_t aoff[4], boff[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * (8 * i + wave) + (lane >> 3);
        aoff[i] = uint32_t(min(r, vm - 1)) * uint32_t(A.x_stride * 2) + uint32_t(ch << 4);
        boff[i] = uint32_t(min(r, vn - 1)) * uint32_t(K * 2) + uint32_t(ch << 4);
    }
    const int nstage = (K + 63) / 64;
    const bool past = 64 * (nstage - 1) + 8 * ch >= K;      // this lane's chunk of the last stage lies past K
    const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(A.x + int64_t(m0) * A.x_stride), 0, 0x7fffffff, ring::RSRC_FLAGS);
    const __amdgpu_buffer_rsrc_t br = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(A.w + int64_t(n0) * K), 0,
                                                                        0x7fffffff, ring::RSRC_FLAGS);
    auto issue = [&](int stage) {
        if (stage >= nstage)
            return;
        uint8_t *buf = lds + (stage & 1) * STAGE;
        // offsets past the buffers' ends read nothing and leave zeros
        const uint32_t none = stage == nstage - 1 && past ? 0x80000000u : 0u, kb = uint32_t(stage * ROWB);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            dma16_lds(br, buf + T * ROWB + (8 * i + wave) * 1024, (boff[i] + kb) | none, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            dma16_lds(ar, buf + (8 * i + wave) * 1024, (aoff[i] + kb) | none, 0);
    };
    auto landed = [&]() {
        __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(0));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wavefront's reads are done with
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    const int wm = wave >> 1, wn = wave & 1, r16 = lane & 15;
    uint32_t fofs[2];                                       // of the halves
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
        fofs[kb] = uint32_t(r16 * ROWB + (((4 * kb + (lane >> 4)) ^ ((r16 >> 1) & 7)) << 4));
    f32x4 acc[8][4];                                        // [feature block][row block]
#pragma unroll
    for (int a = 0; a < 8; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 fw[2][8], fx[4];
    auto read_w = [&](int stage, int kb, int a) {
        return *reinterpret_cast<const u32x4 *>(lds + (stage & 1) * STAGE + T * ROWB + (wn * 128 + a * 16) * ROWB + fofs[kb]);
    };
    auto read_x = [&](int stage, int kb, int b) {
        return *reinterpret_cast<const u32x4 *>(lds + (stage & 1) * STAGE + (wm * 64 + b * 16) * ROWB + fofs[kb]);
    };
    issue(0);
    landed();
    issue(1);
#pragma unroll
    for (int a = 0; a < 8; ++a)
        fw[0][a] = read_w(0, 0, a);
#pragma unroll
    for (int b = 0; b < 4; ++b)
        fx[b] = read_x(0, 0, b);
    // MFMAs of the half whose fragments are in fw[H], fx; the fragments of half 1 - H (of `stage`) are read
    auto half = [&](int stage, auto h) {
        constexpr int H = decltype(h)::value;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
#pragma unroll
            for (int a = 0; a < 8; ++a)
                acc[a][b] = mfma16(as_bf16x8(fw[H][a]), as_bf16x8(fx[b]), acc[a][b]);
#pragma unroll
            for (int q = 0; q < 2; ++q)
                fw[H ^ 1][b * 2 + q] = read_w(stage, H ^ 1, b * 2 + q);
            fx[b] = read_x(stage, H ^ 1, b);
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
    };
    for (int s = 0; s < nstage; ++s) {
        half(s, std::integral_constant<int, 0>{});
        landed();                                           // stage s + 1
        issue(s + 2);
        half(s + 1, std::integral_constant<int, 1>{});      // (after the last stage its fragments are never used)
    }
    __syncthreads();                                        // every fragment has been read: LDS changes its use
    store_block<ACT, true, 8, 4>(A, reinterpret_cast<float *>(lds) + wave * STORE_LDS<8>, acc, m0 + wm * 64, vm - wm * 64,
                           n0 + wn * 128);
}

template <int ACT, class S>
hipError_t launch_tile(const LinearArgs &A, hipStream_t st)
{
    static std::atomic<uint64_t> done{0};
    const hipError_t e = allow_lds_once(reinterpret_cast<const void *>(linear_tile_kernel<ACT, S>), S::LDS, done);
    if (e != hipSuccess)
        return e;
    const int64_t tiles = int64_t((A.M + S::BM - 1) / S::BM) * ((A.N + S::TN - 1) / S::TN);
    launch_k(linear_tile_kernel<ACT, S>, unsigned(tiles), S::THREADS, S::LDS, st, A);
    return hipGetLastError();
}

template <int ACT>
hipError_t launch_act(const LinearArgs &A, hipStream_t st)
{
    const LinearTile t = linear_tile(A.M, A.N);
    if (t.rows == 32)
        return t.features == 32 ? launch_tile<ACT, LinearShape<32, 32, 2, 2, 2, 4, 2>>(A, st)
                                : launch_tile<ACT, LinearShape<32, 64, 1, 2, 4, 3, 1>>(A, st);
    if (t.rows == 64)
        return t.features == 64 ? launch_tile<ACT, LinearShape<64, 64, 2, 2, 2, 4, 1>>(A, st)
                                : launch_tile<ACT, LinearShape<64, 128, 2, 2, 2, 3, 1>>(A, st);
    if (t.rows == 128)
        return t.per_cu == 1 ? launch_tile<ACT, LinearShape<128, 128, 4, 4, 1, 3, 1>>(A, st)
                             : launch_tile<ACT, LinearShape<128, 128, 4, 2, 1, 2, 2>>(A, st);
    const int64_t tiles = int64_t((A.M + 255) / 256) * ((A.N + 255) / 256);
    launch_k(linear_wide_kernel<ACT>, unsigned(tiles), 512, 0, st, A);
    return hipGetLastError();
}

}  // namespace

// The smallest tiles that give one to every CU at most, since one wave of
// workgroups lasts as long as a tile does: a stage of 64 K elements takes a CU
// 0.10 us with tiles of 32 x 32, 0.11 with 32 x 64, 0.19 with 64 x 64, 0.24 with 64 x 128, 0.42
// with 128 x 128.  [us; 16 rows, K 2048, N 5120: 7.0 / 7.7 / 9.9 / 13.9 / 17.7; 256, 4096, 2048: 14.8 / 12.7 / 16.7
// / 23.4 / 31.9; 509, 4096, 2048: 26.3 / 22.9 / 18.0 / 23.9 / 31.5; 1000, 1000, 3000: 27.7 / 30.9 / 20.0 / 20.9 / 14.1.]
// Past that, 128 x 128 tiles two to a CU, about 1.0 us a pair and stage, or
// 256 x 256 ones, about 1.85 us with a tile's start and end, whichever fills its
// rounds better [2500 rows, K 2048, N 2500: 34.6 and 50.5; 1500, 3000, 5000: 63.4
// and 78.3; 2048, 4096, 2048: 41.7 and 41.9; 4096, 2048, 4096: 73.4 and 63.0;
// 4096, 1024, 8192: 80 and 70].
LinearTile linear_tile(int64_t M, int64_t N)
{
    constexpr int64_t CUS = 256;
    auto tiles = [&](int64_t m, int64_t n) { return (M + m - 1) / m * ((N + n - 1) / n); };
    for (const LinearTile t : {LinearTile{32, 32, 2}, LinearTile{32, 64, 1}, LinearTile{64, 64, 1}, LinearTile{64, 128, 1},
                               LinearTile{128, 128, 1}})
        if (tiles(t.rows, t.features) <= CUS)
            return t;
    const int64_t t128 = tiles(128, 128), t256 = tiles(256, 256);
    if (37 * ((t256 + CUS - 1) / CUS) > 20 * ((t128 + 2 * CUS - 1) / (2 * CUS)))
        return LinearTile{128, 128, 2};
    return LinearTile{256, 256, 1};
}

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
