// linear_q4.hip -- projection y = act(x W^T + b) + r with 4-bit weights, gfx950:
// W[n, k] = scale[n, k / g] q[n, k], q = -8 .. 7 (two's complement, element 2j in
// the low nibble of byte j), one fp16 scale for each g = 32, 64 or 128 weights
// of a row; x, b, r and y as in linear.hip.
//
// Codes enter the MFMA as the exact bf16 q / 16, a group's products are summed
// in fp32 and scaled in fp32, so nothing is rounded to fewer than 32 bits before
// y (a weight itself, 11 + 4 significant bits, would not fit bf16), and an
// infinite x gives what it gives in the formula (an offset of the codes would
// make it NaN).
#include "gemm_ring.h"
#include "kernels.h"
#include "linear_epilogue.h"
#include "q4_codes.h"

namespace msi {

namespace {

// ---------------------------------------------------------------- few rows
//
// Up to 16 MB rows: bound by the weights' bytes, small calls by the launch and one
// chain of loads.  A workgroup owns 16 R features; its eight wavefronts take
// chunks of 256 elements of K in turn and their sums meet in LDS in wavefront
// order.  Rows of x are the MFMA's A operand, weights the B operand: both are read
// along their rows (a load covers 8 rows x 128 bytes of weights, 4 rows x 256 or 8 x
// 128 of x) and rearranged in the wavefront's own LDS part; what lies there for rows
// past M ends in results past M.  (Fragments of x straight from memory, every lane from
// another row than its neighbour, cost four times the L1's cycles: 16 rows, K 4096,
// N 2048 7.9 us for 5.9.)  A lane's outputs are four rows of one feature, so it
// applies that feature's scales.  Weights from HBM, one row: 2048 x 5120 5.0 us,
// 4096 x 8199 8.9 us (1.9 TB/s), 8192 x 8192 11.5 us (3.0 TB/s), whose wavefronts
// wait for 60 % of their cycles and issue in 20 %: the chunks' chains.
constexpr int ROWS_WAVES = 8, CHUNK = 8;      // blocks of 32 elements in a chunk

typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t u32x4_any;
typedef __attribute__((ext_vector_type(2), aligned(2))) uint32_t u32x2_any;
typedef __attribute__((aligned(2))) uint32_t u32_any;

// N fp16 scales (pairs in words) from p on, in one access at any alignment.
template <int N>
__device__ __forceinline__ void read_scales(uint32_t (&w)[N / 2], const uint16_t *p)
{
    if constexpr (N == 8) {
        const u32x4_any v = *reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = v[i];
    } else if constexpr (N == 4) {
        const u32x2_any v = *reinterpret_cast<const u32x2_any *>(p);
        w[0] = v[0], w[1] = v[1];
    } else {
        w[0] = *reinterpret_cast<const u32_any *>(p);
    }
}

// The same with the scales from `count` on zero (count < N).
template <int N>
__device__ __forceinline__ void read_scales_tail(uint32_t (&w)[N / 2], const uint16_t *p, int count)
{
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const uint32_t lo = 2 * i < count ? p[2 * i] : 0u, hi = 2 * i + 1 < count ? p[2 * i + 1] : 0u;
        w[i] = lo | hi << 16;
    }
}

__device__ __forceinline__ float activate_any(int act, float z)
{
    switch (act) {
    case LINEAR_SILU: return activate<LINEAR_SILU>(z);
    case LINEAR_GELU: return activate<LINEAR_GELU>(z);
    case LINEAR_GELU_TANH: return activate<LINEAR_GELU_TANH>(z);
    default: return z;
    }
}

// One output: act(z + bias) + residual.
__device__ __forceinline__ void store1(const LinearArgs &A, int act, int64_t m, int n, float z)
{
    z = activate_any(act, A.bias ? z + A.bias[n] : z);
    if (A.res_f32)
        z += A.res_f32[m * A.res_stride + n];
    else if (A.res_bf16)
        z += bf16_to_f32(A.res_bf16[m * A.res_stride + n]);
    if (A.out_f32)
        A.out_f32[m * A.out_stride + n] = z;
    else
        A.out_bf16[m * A.out_stride + n] = f32_to_bf16(z);
}

template <int R, int MB, int GB>
__global__ void __launch_bounds__(64 * ROWS_WAVES, R * MB == 1 ? 4 : 2) q4_rows_kernel(LinearQ4Args Q, int act)
{
    constexpr int RS = 16 * CHUNK + 16;                    // LDS bytes of a row of a chunk, padded against bank conflicts
    constexpr int NG = CHUNK / GB;                         // groups of a chunk
    constexpr int XB = 4 / MB, XS = 64 * XB + 16;          // blocks of x in LDS at a time, bytes of such a row
    constexpr int XL = 4 * XB, XR = 64 / XL;               // lanes of a row of a load of x, rows
    constexpr int STAGE = R * 16 * RS + MB * 16 * XS, SUMS = R * MB * 1024;
    __shared__ __attribute__((aligned(16))) uint8_t lds[ROWS_WAVES * (STAGE > SUMS ? STAGE : SUMS)];
    const LinearArgs &A = Q.l;
    const int n0 = int(blockIdx.x) * 16 * R;
    const int K = A.K, nblk = K / 32, nchunk = (nblk + CHUNK - 1) / CHUNK, ng = nblk / GB;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    uint8_t *const mine = lds + wave * STAGE, *const xs = mine + R * 16 * RS;

    // weights: load k of feature block m brings rows 8 k + lane / 8, the lane's 16 bytes are block lane % 8 of the chunk
    const uint8_t *wp[R][2];
    const uint16_t *sp[R];
#pragma unroll
    for (int m = 0; m < R; ++m) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            wp[m][k] = Q.codes + int64_t(min(n0 + 16 * m + 8 * k + (lane >> 3), A.N - 1)) * (K / 2) + 16 * (lane & 7);
        sp[m] = Q.scales + int64_t(min(n0 + 16 * m + r16, A.N - 1)) * ng;
    }
    const uint16_t *xp[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        xp[j] = A.x + int64_t(min(XR * j + lane / XL, A.M - 1)) * A.x_stride + 8 * (lane % XL);

    u32x4 w[R][2];
    uint32_t sc[R][NG / 2];
    auto load_weights = [&](int c) {
        const int back = 16 * max(CHUNK * c + (lane & 7) - (nblk - 1), 0);   // (blocks past the end: the last one again)
#pragma unroll
        for (int m = 0; m < R; ++m)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                w[m][k] = load_stream16(wp[m][k] + (16 * CHUNK * c - back));
#pragma unroll
        for (int m = 0; m < R; ++m) {
            if (CHUNK * (c + 1) <= nblk)
                read_scales<NG>(sc[m], sp[m] + NG * c);
            else
                read_scales_tail<NG>(sc[m], sp[m] + NG * c, ng - NG * c);
        }
    };
    f32x4 acc[MB][R];
#pragma unroll
    for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int m = 0; m < R; ++m)
            acc[a][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (wave < nchunk)
        load_weights(wave);
    for (int c = wave; c < nchunk; c += ROWS_WAVES) {
        u32x4 x[CHUNK / XB][4];
        const int left = nblk - CHUNK * c;                 // blocks from here on
#pragma unroll
        for (int h = 0; h < CHUNK / XB; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (XR * j < A.M)                          // (nothing times whatever is there: past K is zero)
                    x[h][j] = left >= CHUNK || XB * h + lane % XL / 4 < left
                                  ? *reinterpret_cast<const u32x4 *>(xp[j] + 32 * (CHUNK * c + XB * h))
                                  : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int m = 0; m < R; ++m)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                *reinterpret_cast<u32x4 *>(mine + (16 * m + 8 * k + (lane >> 3)) * RS + 16 * (lane & 7)) = w[m][k];
        uint32_t now[R][NG / 2];
#pragma unroll
        for (int m = 0; m < R; ++m)
#pragma unroll
            for (int i = 0; i < NG / 2; ++i)
                now[m][i] = sc[m][i];
        if (c + ROWS_WAVES < nchunk)
            load_weights(c + ROWS_WAVES);
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            f32x4 part[MB][R];
#pragma unroll
            for (int a = 0; a < MB; ++a)
#pragma unroll
                for (int m = 0; m < R; ++m)
                    part[a][m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < GB; ++b) {
                const int u = j * GB + b;
                if (u % XB == 0) {                         // (a wavefront's LDS operations are in order; the fences keep
                    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");   // the compiler from moving them)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (XR * i < A.M)
                            *reinterpret_cast<u32x4 *>(xs + (XR * i + lane / XL) * XS + 16 * (lane % XL)) = x[u / XB][i];
                    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                }
                bf16x8 xf[MB];
#pragma unroll
                for (int a = 0; a < MB; ++a)
                    xf[a] = as_bf16x8(*reinterpret_cast<const u32x4 *>(xs + (16 * a + r16) * XS + u % XB * 64 + 16 * g));
#pragma unroll
                for (int m = 0; m < R; ++m) {
                    const bf16x8 wf = unpack_q4_16th(*reinterpret_cast<const uint32_t *>(mine + (16 * m + r16) * RS + 16 * u + 4 * g));
#pragma unroll
                    for (int a = 0; a < MB; ++a)
                        part[a][m] = mfma16(xf[a], wf, part[a][m]);
                }
            }
#pragma unroll
            for (int m = 0; m < R; ++m) {
                const float s = half_to_float(uint16_t(now[m][j >> 1] >> (16 * (j & 1))));
#pragma unroll
                for (int a = 0; a < MB; ++a)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        acc[a][m][k] = fmaf(s, part[a][m][k], acc[a][m][k]);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    __syncthreads();                                       // the rows' place becomes the sums'
    f32x4 *const sums = reinterpret_cast<f32x4 *>(lds);
#pragma unroll
    for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int m = 0; m < R; ++m)
            sums[((wave * MB + a) * R + m) * 64 + lane] = acc[a][m];
    __syncthreads();
    if (wave < MB * R) {
        f32x4 z = sums[wave * 64 + lane];
#pragma unroll
        for (int o = 1; o < ROWS_WAVES; ++o)
            z += sums[(o * MB * R + wave) * 64 + lane];
        const int n = n0 + 16 * (wave % R) + r16, m = 16 * (wave / R) + 4 * g;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (m + k < A.M && n < A.N)
                store1(A, act, m + k, n, 16.0f * z[k]);
    }
}

// ---------------------------------------------------------------- tiles
//
// BM rows x TN features a workgroup; K in stages of 64 KG elements copied
// straight into one of NBUF LDS buffers, NBUF - 1 in flight.  KG groups of WR x
// WC wavefronts each multiply their own 64 elements of a stage, and their sums
// meet in LDS in a fixed order.  Rows of x: 16-byte chunk c of a slice of stage
// row r in slot c ^ ((r / 2) % 8); codes: chunk c (of 2 KG) of feature r in slot
// c ^ (r KG / 8 % (2 KG)): both spread a fragment read over the banks.  Weights
// are the A operand, so a lane ends with four consecutive features of a row.  The
// scales of two to eight stages are brought to LDS at a time (a panel), by group,
// so that a lane reads its four features' at once.
//
// Up to a few hundred rows a stage is one chain of LDS reads, conversion, MFMAs
// and scaling with little beside it, 0.6 to 1 us.  In large calls a block's
// conversion, MFMAs and scaling follow one another as well, in two wavefronts a
// SIMD, and overlap little: the vector unit is busy for 50 % of the time, the matrix
// cores for 27 % (2000 x 8192 of K 2048 85 us, 790 TFLOP/s).
template <int BM_, int TN_, int WR_, int WC_, int KG_, int NBUF_, int WPC_>
struct Q4Shape {
    static constexpr int BM = BM_, TN = TN_, WR = WR_, WC = WC_, KG = KG_, NBUF = NBUF_, WPC = WPC_;
    static constexpr int WAVES = WR * WC * KG, THREADS = 64 * WAVES;
    static constexpr int ROWB = 128, QROWB = 32 * KG, CPR = 2 * KG, PANEL = KG > 2 ? 16 / KG : 8;   // bytes, code chunks of a row; stages of a panel
    static constexpr int MB = BM / WR / 16, NB = TN / WC / 16;
    static constexpr int A_BYTES = KG * BM * ROWB, STAGE = A_BYTES + TN * QROWB;
    static constexpr int LA = KG * BM / 8 / WAVES, QC = KG * TN / 32, LQ = (QC + WAVES - 1) / WAVES, LPS = LA + LQ;
    template <int GB>
    static constexpr int SCALES = PANEL * 2 * KG / GB * TN * 2;                    // bytes of a panel
    static constexpr int OUT = WR * WC * STORE_LDS<NB> * 4, SUMS = OUT + (KG - 1) * BM * TN * 4;   // of the epilogue
    template <int GB>
    static constexpr size_t LDS = NBUF * STAGE + 2 * SCALES<GB> > SUMS ? NBUF * STAGE + 2 * SCALES<GB> : SUMS;
    static_assert(KG * BM % (8 * WAVES) == 0 && KG * TN % 32 == 0 && LDS<1> * WPC <= 160 * 1024, "");
    static_assert(LA <= 16 && LQ <= 8 && LPS * (NBUF - 2) < 64, "");
};

template <int ACT, class S, int GB>
__global__ void __launch_bounds__(S::THREADS, S::WPC * S::WAVES / 4) q4_tile_kernel(LinearQ4Args Q)
{
    constexpr int BM = S::BM, TN = S::TN, KG = S::KG, NBUF = S::NBUF, WAVES = S::WAVES, MB = S::MB, NB = S::NB, STAGE = S::STAGE,
                  ROWB = S::ROWB, QROWB = S::QROWB, CPR = S::CPR, A_BYTES = S::A_BYTES, LA = S::LA, LQ = S::LQ;
    constexpr int NGP = S::PANEL * 2 * KG / GB, SPT = (TN * NGP + S::THREADS - 1) / S::THREADS;   // groups of a panel, scales of a thread
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds8[];
    uint16_t *const panels = reinterpret_cast<uint16_t *>(lds8 + NBUF * STAGE);
    const LinearArgs &A = Q.l;
    const int2 at = tile_at(xcd_swizzle(int(blockIdx.x), int(gridDim.x)), (A.M + BM - 1) / BM, (A.N + TN - 1) / TN);
    const int m0 = at.x * BM, n0 = at.y * TN;
    const int K = A.K, ng = K / (32 * GB), nstage = (K + 64 * KG - 1) / (64 * KG), tail = K - 64 * KG * (nstage - 1);
    const int vm = min(BM, A.M - m0), vn = min(TN, A.N - n0);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = wave / (S::WR * S::WC), wi = wave % (S::WR * S::WC), wm = wi / S::WC, wn = wi % S::WC;
    const int r16 = lane & 15, g = lane >> 4;
    // offsets from the tile's first rows (under 2^31: strides are bounded); rows past the end repeat the last one
    uint32_t aoff[LA], qoff[LQ];
    int last = 0;                             // bit i: A copy i, bit 16 + i: code copy i of the last stage lies past K
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int c = WAVES * i + wave, r = 8 * (c % (BM / 8)) + (lane >> 3), slice = c / (BM / 8), ch = (lane & 7) ^ ((r >> 1) & 7);
        aoff[i] = uint32_t(min(r, vm - 1)) * uint32_t(A.x_stride * 2) + uint32_t(slice * ROWB + (ch << 4));
        last |= int(64 * slice + 8 * ch >= tail) << i;
    }
#pragma unroll
    for (int i = 0; i < LQ; ++i) {
        const int c = 64 * ((WAVES * i + wave) % S::QC) + lane, r = c / CPR, ch = (c % CPR) ^ (r * KG / 8 % CPR);
        qoff[i] = uint32_t(min(r, vn - 1)) * uint32_t(K / 2) + uint32_t(16 * ch);
        last |= int(32 * ch >= tail) << (16 + i);
    }
    const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(A.x + int64_t(m0) * A.x_stride), 0, 0x7fffffff, ring::RSRC_FLAGS);
    const __amdgpu_buffer_rsrc_t qr = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t *>(Q.codes + int64_t(n0) * (K / 2)), 0, 0x7fffffff, ring::RSRC_FLAGS);
    auto issue = [&](int stage, int buf) {
        uint8_t *st = lds8 + buf * STAGE;
        const bool edge = tail < 64 * KG && stage == nstage - 1;   // an offset past the buffer's end leaves zeros
#pragma unroll
        for (int i = 0; i < LQ; ++i)
            dma16_lds(qr, st + A_BYTES + (WAVES * i + wave) % S::QC * 1024,   // (with fewer copies than wavefronts: some twice)
                      edge && (last >> (16 + i) & 1) ? 0x80000000u : qoff[i] + uint32_t(stage * QROWB), 0);
#pragma unroll
        for (int i = 0; i < LA; ++i)
            dma16_lds(ar, st + (WAVES * i + wave) * 1024,
                      edge && (last >> i & 1) ? 0x80000000u : aoff[i] + uint32_t(stage * (KG * ROWB)), 0);
    };
    // scales: neighbouring threads take a feature's groups in turn, through registers
    uint16_t sw[SPT];
    auto load_panel = [&](int p) {
#pragma unroll
        for (int k = 0; k < SPT; ++k) {
            const int e = tid + k * S::THREADS, r = e / NGP, j = p * NGP + e % NGP;
            sw[k] = e < TN * NGP && j < ng ? Q.scales[int64_t(n0 + min(r, vn - 1)) * ng + j] : uint16_t(0);
        }
    };
    auto keep_panel = [&](int p) {
#pragma unroll
        for (int k = 0; k < SPT; ++k) {
            const int e = tid + k * S::THREADS;
            if (e < TN * NGP)
                panels[(p & 1) * (NGP * TN) + e % NGP * TN + e / NGP] = sw[k];
        }
    };

    f32x4 acc[NB][MB];
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
        for (int b = 0; b < MB; ++b)
            acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto compute = [&](int stage, int buf) {
        const uint8_t *xa = lds8 + buf * STAGE + (grp * BM + wm * MB * 16) * ROWB, *qb = lds8 + buf * STAGE + A_BYTES;
        const uint16_t *scales = panels + (stage / S::PANEL & 1) * (NGP * TN) + wn * NB * 16 + 4 * g;
        const int j0 = 2 * (stage % S::PANEL * KG + grp) / GB;   // the slice's first group in the panel
        bf16x8 af[2][MB];
        uint32_t cw[2][NB];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int c = (wn * NB + nb) * 16 + r16;
                cw[kb][nb] = *reinterpret_cast<const uint32_t *>(qb + c * QROWB + (((2 * grp + kb) ^ (c * KG / 8 % CPR)) << 4) + 4 * g);
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
                af[kb][mb] = as_bf16x8(*reinterpret_cast<const u32x4 *>(xa + (mb * 16 + r16) * ROWB + (((4 * kb + g) ^ ((r16 >> 1) & 7)) << 4)));
        }
        auto scaled = [&](int nb, int j, const f32x4 (&part)[MB]) {
            const uint2 s = *reinterpret_cast<const uint2 *>(scales + j * TN + nb * 16);
            const float f[4] = {half_to_float(uint16_t(s.x)), half_to_float(uint16_t(s.x >> 16)), half_to_float(uint16_t(s.y)),
                                half_to_float(uint16_t(s.y >> 16))};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
                    acc[nb][mb][i] = fmaf(f[i], part[mb][i], acc[nb][mb][i]);
        };
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            f32x4 part[MB];
            const bf16x8 w0 = unpack_q4_16th(cw[0][nb]), w1 = unpack_q4_16th(cw[1][nb]);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
                part[mb] = mfma16(w0, af[0][mb], f32x4{0.f, 0.f, 0.f, 0.f});
            if constexpr (GB == 1) {
                scaled(nb, j0, part);
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
                    part[mb] = mfma16(w1, af[1][mb], f32x4{0.f, 0.f, 0.f, 0.f});
                scaled(nb, j0 + 1, part);
            } else {
                // (a group of 128 in two parts: the sum over its second half then starts from zero, too)
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
                    part[mb] = mfma16(w1, af[1][mb], part[mb]);
                scaled(nb, j0, part);
            }
        }
    };

    constexpr int AHEAD = NBUF - 1;
    load_panel(0);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
        if (j < nstage)
            issue(j, j);
    keep_panel(0);
    int cur = 0, nxt = AHEAD;
    auto step = [&](int s) {
        // stage s has landed; the buffer of stage s + AHEAD was last read at s - 1, by reads that are waited for as well
        // (LGKM_DONE: no LDS operation of this wavefront in flight)
        constexpr int LGKM_DONE = ~(0xF << 8);
        if (s + AHEAD <= nstage)
            __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(S::LPS * (AHEAD - 1)) & LGKM_DONE);
        else
            __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(0) & LGKM_DONE);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + AHEAD < nstage)
            issue(s + AHEAD, nxt);
        compute(s, cur);
        cur = cur == NBUF - 1 ? 0 : cur + 1;
        nxt = nxt == NBUF - 1 ? 0 : nxt + 1;
    };
    // the next panel is read at this one's start and kept at its middle: its place was last read a panel ago.  (Loops of
    // their own: where a stage may or may not have read a panel, the compiler waits for every copy in every stage.)
    for (int s = 0, p = 1; s < nstage; ++p) {
        const int end = min(p * S::PANEL, nstage), middle = min(end, s + S::PANEL / 2);
        const bool more = end < nstage;
        if (more)
            load_panel(p);
        for (; s < middle; ++s)
            step(s);
        if (more)
            keep_panel(p);
        for (; s < end; ++s)
            step(s);
    }
    __syncthreads();                                        // every fragment has been read: LDS changes its use
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
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
        for (int b = 0; b < MB; ++b)
            acc[a][b] *= 16.0f;                             // the codes were sixteenths
    store_block<ACT, false, NB, MB>(A, reinterpret_cast<float *>(lds8) + wi * STORE_LDS<NB>, acc, m0 + wm * MB * 16,
                                    vm - wm * MB * 16, n0 + wn * NB * 16);
}

template <int R, int MB>
hipError_t launch_rows(const LinearQ4Args &A, int act, hipStream_t st)
{
    const unsigned grid = unsigned((A.l.N + 16 * R - 1) / (16 * R));
    if (A.group == 32)
        launch_k(q4_rows_kernel<R, MB, 1>, grid, 64 * ROWS_WAVES, 0, st, A, act);
    else if (A.group == 64)
        launch_k(q4_rows_kernel<R, MB, 2>, grid, 64 * ROWS_WAVES, 0, st, A, act);
    else
        launch_k(q4_rows_kernel<R, MB, 4>, grid, 64 * ROWS_WAVES, 0, st, A, act);
    return hipGetLastError();
}

template <int ACT, class S>
hipError_t launch_tile(const LinearQ4Args &A, hipStream_t st)
{
    const int64_t tiles = int64_t((A.l.M + S::BM - 1) / S::BM) * ((A.l.N + S::TN - 1) / S::TN);
    auto go = [&](auto gb) {
        constexpr int GB = decltype(gb)::value;
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_lds_once(reinterpret_cast<const void *>(q4_tile_kernel<ACT, S, GB>), S::template LDS<GB>, done);
        if (e != hipSuccess)
            return e;
        launch_k(q4_tile_kernel<ACT, S, GB>, unsigned(tiles), S::THREADS, S::template LDS<GB>, st, A);
        return hipGetLastError();
    };
    if (A.group == 32)
        return go(std::integral_constant<int, 1>{});
    return A.group == 64 ? go(std::integral_constant<int, 2>{}) : go(std::integral_constant<int, 4>{});
}

template <int ACT>
hipError_t launch_act(const LinearQ4Args &A, const LinearTile &t, hipStream_t st)
{
    if (t.rows == 16)
        return launch_tile<ACT, Q4Shape<16, 32, 1, 2, 8, 2, 1>>(A, st);
    if (t.rows == 32)
        return t.features == 32 ? launch_tile<ACT, Q4Shape<32, 32, 1, 2, 8, 2, 1>>(A, st)
                                : launch_tile<ACT, Q4Shape<32, 64, 1, 4, 4, 2, 1>>(A, st);
    if (t.rows == 64 && t.features == 32)
        return launch_tile<ACT, Q4Shape<64, 32, 1, 2, 8, 2, 1>>(A, st);
    if (t.rows == 64 && t.features == 64)
        return launch_tile<ACT, Q4Shape<64, 64, 1, 4, 4, 2, 1>>(A, st);
    if (t.rows == 128)
        return t.per_cu == 1 ? launch_tile<ACT, Q4Shape<128, 128, 1, 8, 2, 2, 1>>(A, st)
                             : launch_tile<ACT, Q4Shape<128, 128, 1, 4, 1, 2, 2>>(A, st);
    return t.per_cu == 1 ? launch_tile<ACT, Q4Shape<64, 128, 1, 8, 2, 2, 1>>(A, st)
                         : launch_tile<ACT, Q4Shape<64, 128, 1, 4, 1, 3, 3>>(A, st);
}

}  // namespace

// Up to 16 rows: no tiles (rows and features of a workgroup), 32 features where
// 16 make more than 256 workgroups and there are more than 8 rows, whose x is read
// by half as many [us, 16 and 32 features: 1 row, K 8192, N 8192 11.5 and 12.4; 8
// rows, 4096, 8199 10.0 and 10.5; 16 rows, 4096, 2048 5.8 and 7.5; 4096, 5120 9.0 and
// 7.8; 8192, 8192 16.1 and 14.0].  Up to 32 rows likewise, while that makes no more than
// 256 workgroups [20, 8192, 2048 11.3 for 16.9 in tiles; 24, 4096, 2048 7.3 for 8.5; 32,
// 4096, 5120 9.9 for 11.7; 32, 2048, 16384 13.7 for 11.1].  Past 2^22 features tiles take
// over for few rows, too: up to there a long K is better off without them, a short one with
// them [1 row, N 2^22 and 64 more, K 2048 1376 and 1495, K 256 921 and 333; 16 rows 1261
// and 1534, 1013 and 362; 131072, K 4096 78, 3.7 TB/s].  Above, the smallest
// tiles that give one to every CU at most, since one wave of workgroups lasts as
// long as a tile does, and that is the latency of its stages.  [16 x 32, 32 x 32,
// 32 x 64, 64 x 64, 64 x 128, 128 x 128: 61 rows, K 4096, N 2048 8.8 / 10.3 / 14.3 /
// 17.6 / 27.2 / 40.3; 61, 4096, 8199 30.0 / 31.2 / 23.7 / 21.6 / 32.1 / 42.9; 128,
// 2048, 5120 19.2 / 19.9 / 16.3 / 13.6 / 21.3 / 32.9; 256, 2048, 8192 55 / 52 / 27.1 /
// 25.2 / 18.7 / 26.3; 509, 2048, 8192 104 / 102 / 51 / 49 / 34.7 / 28.4; weights from
// HBM.]  Their wavefronts, 16 a CU, have all of the tile's rows, so that a weight is
// converted once (64 x 64, each converted twice and a third buffer: 24.5 for 21.6).
// Long K takes 64 x 32, stages of 512 elements, for 32 x 64 where as many tiles do
// [61, 4096, 8192 17.2 and 19.2; 128, 4096, 4096 17.0 and 18.8; 61, 8192, 8192 28.3
// and 32.1; 61, 2048, 8192 12.9 and 12.6; 128, 2048, 4096 11.7 and 11.0].
// Past that, tiles of 128 x 128, two to a CU (wavefronts of 128 x 32, which convert
// a weight for eight row blocks), or of 64 x 128, three to a CU, whose rounds last
// about three quarters as long, whichever fills its rounds better [1000, 2048, 8192 43.8
// and 50.0; 2000, 2048, 8192 84.8 and 97.5; 2000, 2048, 5120 66.5 and 62.9; 4096, 4096, 4096
// 160 and 179].
LinearTile linear_q4_tile(int64_t M, int64_t N, int64_t K)
{
    constexpr int64_t CUS = 256;
    auto tiles = [&](int64_t m, int64_t n) { return (M + m - 1) / m * ((N + n - 1) / n); };
    if (M <= 16 && N <= 1 << 22)
        return LinearTile{0, tiles(16, 16) > CUS && M > 8 ? 32 : 16, 1};
    if (M <= 32 && tiles(32, 32) <= CUS)
        return LinearTile{0, tiles(32, 16) > CUS ? 32 : 16, 1};
    for (const LinearTile t : {LinearTile{16, 32, 1}, LinearTile{32, 32, 1}, LinearTile{32, 64, 1}, LinearTile{64, 64, 1},
                               LinearTile{64, 128, 1}, LinearTile{128, 128, 1}})
        if (tiles(t.rows, t.features) <= CUS)
            return t.rows == 32 && t.features == 64 && K >= 4096 && tiles(64, 32) <= tiles(32, 64) ? LinearTile{64, 32, 1} : t;
    const int64_t big = (tiles(128, 128) + 2 * CUS - 1) / (2 * CUS), small = (tiles(64, 128) + 3 * CUS - 1) / (3 * CUS);
    return 4 * big <= 3 * small ? LinearTile{128, 128, 2} : LinearTile{64, 128, 3};
}

hipError_t launch_linear_q4(const LinearQ4Args &A, int act, hipStream_t st)
{
    const LinearTile t = linear_q4_tile(A.l.M, A.l.N, A.l.K);
    if (t.rows == 0) {
        if (A.l.M <= 16)
            return t.features == 16 ? launch_rows<1, 1>(A, act, st) : launch_rows<2, 1>(A, act, st);
        return t.features == 16 ? launch_rows<1, 2>(A, act, st) : launch_rows<2, 2>(A, act, st);
    }
    switch (act) {
    case LINEAR_SILU: return launch_act<LINEAR_SILU>(A, t, st);
    case LINEAR_GELU: return launch_act<LINEAR_GELU>(A, t, st);
    case LINEAR_GELU_TANH: return launch_act<LINEAR_GELU_TANH>(A, t, st);
    default: return launch_act<LINEAR_NONE>(A, t, st);
    }
}

}  // namespace msi
