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
// Up to 64 rows: bound by the weights' bytes, small calls by the launch and one
// chain of loads.  A workgroup owns 16 R features and 16 MT rows; its eight
// wavefronts take chunks of 256 elements of K in turn and their sums meet in
// LDS in wavefront order.  Rows of x are the MFMA's A operand, read straight
// from memory (rows past M repeat the last one), weights the B operand, read
// along their rows (a load covers 8 rows x 128 bytes) and rearranged in the
// wavefront's own LDS part.  A lane's outputs are four rows of one feature, so
// it applies that feature's scales.
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

template <int MT, int R, int GB>
__global__ void __launch_bounds__(64 * ROWS_WAVES, MT == 1 && R == 1 ? 4 : 2) q4_rows_kernel(LinearQ4Args Q, int act)
{
    constexpr int RS = 16 * CHUNK + 16;                    // LDS bytes of a row of a chunk, padded against bank conflicts
    constexpr int NG = CHUNK / GB;                         // groups of a chunk
    constexpr int STAGE = R * 16 * RS, SUMS = MT * R * 1024;
    __shared__ __attribute__((aligned(16))) uint8_t lds[ROWS_WAVES * (STAGE > SUMS ? STAGE : SUMS)];
    const LinearArgs &A = Q.l;
    const int n0 = int(blockIdx.x) * 16 * R, m0 = int(blockIdx.y) * 16 * MT;
    const int K = A.K, nblk = K / 32, nchunk = (nblk + CHUNK - 1) / CHUNK, ng = nblk / GB;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    uint8_t *const mine = lds + wave * STAGE;

    // weights: load k of feature block m brings rows 8 k + lane / 8, the lane's 16 bytes are block lane % 8 of the chunk
    const uint8_t *wp[R][2];
    const uint16_t *sp[R];
    const uint16_t *xp[MT];
#pragma unroll
    for (int m = 0; m < R; ++m) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            wp[m][k] = Q.codes + int64_t(min(n0 + 16 * m + 8 * k + (lane >> 3), A.N - 1)) * (K / 2) + 16 * (lane & 7);
        sp[m] = Q.scales + int64_t(min(n0 + 16 * m + r16, A.N - 1)) * ng;
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
        xp[t] = A.x + int64_t(min(m0 + 16 * t + r16, A.M - 1)) * A.x_stride + 8 * g;

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
    f32x4 acc[MT][R];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int m = 0; m < R; ++m)
            acc[t][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (wave < nchunk)
        load_weights(wave);
    for (int c = wave; c < nchunk; c += ROWS_WAVES) {
        u32x4 x[MT][CHUNK];
        const int left = nblk - CHUNK * c;                 // blocks from here on
        if (left >= CHUNK) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int u = 0; u < CHUNK; ++u)
                    x[t][u] = *reinterpret_cast<const u32x4 *>(xp[t] + 32 * (CHUNK * c + u));
        } else {                                           // (nothing times whatever is there: the rest is zero)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int u = 0; u < CHUNK; ++u)
                    x[t][u] = u < left ? *reinterpret_cast<const u32x4 *>(xp[t] + 32 * (CHUNK * c + u)) : u32x4{0, 0, 0, 0};
        }
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
        // (a wavefront's LDS operations are in order; the fences keep the compiler from moving them)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        if (c + ROWS_WAVES < nchunk)
            load_weights(c + ROWS_WAVES);
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            f32x4 part[MT][R];
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int m = 0; m < R; ++m)
                    part[t][m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < GB; ++b) {
                const int u = j * GB + b;
#pragma unroll
                for (int m = 0; m < R; ++m) {
                    const bf16x8 wf = unpack_q4_16th(*reinterpret_cast<const uint32_t *>(mine + (16 * m + r16) * RS + 16 * u + 4 * g));
#pragma unroll
                    for (int t = 0; t < MT; ++t)
                        part[t][m] = mfma16(as_bf16x8(x[t][u]), wf, part[t][m]);
                }
            }
#pragma unroll
            for (int m = 0; m < R; ++m) {
                const float s = half_to_float(uint16_t(now[m][j >> 1] >> (16 * (j & 1))));
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        acc[t][m][k] = fmaf(s, part[t][m][k], acc[t][m][k]);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    __syncthreads();                                       // the rows' place becomes the sums'
    f32x4 *const sums = reinterpret_cast<f32x4 *>(lds);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int m = 0; m < R; ++m)
            sums[(wave * MT * R + t * R + m) * 64 + lane] = acc[t][m];
    __syncthreads();
    for (int i = wave; i < MT * R; i += ROWS_WAVES) {
        f32x4 z = sums[i * 64 + lane];
#pragma unroll
        for (int o = 1; o < ROWS_WAVES; ++o)
            z += sums[(o * MT * R + i) * 64 + lane];
        const int n = n0 + 16 * (i % R) + r16, m = m0 + 16 * (i / R) + 4 * g;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (m + k < A.M && n < A.N)
                store1(A, act, m + k, n, 16.0f * z[k]);
    }
}

// ---------------------------------------------------------------- tiles
//
// BM rows x TN features a workgroup, K in stages of 64 elements copied straight
// into one of two LDS buffers: rows of x as eight 16-byte chunks, chunk c of row
// r in slot c ^ ((r / 2) % 8), codes as two, chunk c of feature r in slot
// c ^ ((r / 8) % 2), which spreads a fragment read over the banks.  Weights are
// the A operand, so a lane ends with four consecutive features of a row.  The
// scales of 512 elements are brought to LDS at a time, by group, so that a lane
// reads its four features' at once.
template <int BM_, int TN_, int WR_, int WC_, int WPC_>
struct Q4Shape {
    static constexpr int BM = BM_, TN = TN_, WR = WR_, WC = WC_, WPC = WPC_;
    static constexpr int WAVES = WR * WC, THREADS = 64 * WAVES;
    static constexpr int ROWB = 128, QROWB = 32, PANEL = 8;                  // stages of a panel of scales
    static constexpr int MB = BM / WR / 16, NB = TN / WC / 16;
    static constexpr int A_BYTES = BM * ROWB, STAGE = A_BYTES + TN * QROWB;
    static constexpr int LA = BM / 8 / WAVES, LQ = TN / 32 / WAVES;
    static constexpr int PIECES = THREADS / TN;                             // threads of a feature's scales
    template <int GB>
    static constexpr int SCALES = PANEL * 2 / GB * TN * 2;                  // bytes of a panel
    static constexpr int OUT = WAVES * STORE_LDS<NB> * 4;
    template <int GB>
    static constexpr size_t LDS = size_t(2 * STAGE + 2 * SCALES<GB>) > OUT ? size_t(2 * STAGE + 2 * SCALES<GB>) : OUT;
    static_assert(BM % (8 * WAVES) == 0 && TN % (32 * WAVES) == 0 && THREADS % TN == 0 && LDS<1> * WPC <= 160 * 1024, "");
};

template <int ACT, class S, int GB>
__global__ void __launch_bounds__(S::THREADS, S::WPC * S::WAVES / 4) q4_tile_kernel(LinearQ4Args Q)
{
    constexpr int BM = S::BM, TN = S::TN, WAVES = S::WAVES, MB = S::MB, NB = S::NB, STAGE = S::STAGE, ROWB = S::ROWB,
                  QROWB = S::QROWB, A_BYTES = S::A_BYTES;
    constexpr int NGP = S::PANEL * 2 / GB, PER = NGP / S::PIECES;            // groups of a panel, scales of a thread
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds8[];
    uint16_t *const panels = reinterpret_cast<uint16_t *>(lds8 + 2 * STAGE);
    const LinearArgs &A = Q.l;
    const int2 at = tile_at(xcd_swizzle(int(blockIdx.x), int(gridDim.x)), (A.M + BM - 1) / BM, (A.N + TN - 1) / TN);
    const int m0 = at.x * BM, n0 = at.y * TN;
    const int K = A.K, ng = K / (32 * GB), nstage = (K + 63) / 64;
    const int vm = min(BM, A.M - m0), vn = min(TN, A.N - n0);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / S::WC, wn = wave % S::WC, r16 = lane & 15, g = lane >> 4;
    // offsets from the tile's first rows (under 2^31: strides are bounded); rows past the end repeat the last one
    uint32_t aoff[S::LA], qoff[S::LQ];
    int last = 0;                             // bit i: A copy i, bit 16 + i: code copy i of the last stage lies past K
    const bool half = K % 64 != 0;
#pragma unroll
    for (int i = 0; i < S::LA; ++i) {
        const int r = 8 * (WAVES * i + wave) + (lane >> 3), ch = (lane & 7) ^ ((r >> 1) & 7);
        aoff[i] = uint32_t(min(r, vm - 1)) * uint32_t(A.x_stride * 2) + uint32_t(ch << 4);
        last |= int(ch >= 4) << i;
    }
#pragma unroll
    for (int i = 0; i < S::LQ; ++i) {
        const int c = 32 * (WAVES * i + wave) + (lane >> 1), ch = (lane & 1) ^ ((c >> 3) & 1);
        qoff[i] = uint32_t(min(c, vn - 1)) * uint32_t(K / 2) + uint32_t(16 * ch);
        last |= ch << (16 + i);
    }
    const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(A.x + int64_t(m0) * A.x_stride), 0, 0x7fffffff, ring::RSRC_FLAGS);
    const __amdgpu_buffer_rsrc_t qr = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t *>(Q.codes + int64_t(n0) * (K / 2)), 0, 0x7fffffff, ring::RSRC_FLAGS);
    auto issue = [&](int stage, int buf) {
        uint8_t *st = lds8 + buf * STAGE;
        const bool edge = half && stage == nstage - 1;     // an offset past the buffer's end leaves zeros
#pragma unroll
        for (int i = 0; i < S::LQ; ++i)
            dma16_lds(qr, st + A_BYTES + (WAVES * i + wave) * 1024,
                      edge && (last >> (16 + i) & 1) ? 0x80000000u : qoff[i] + uint32_t(stage * QROWB), 0);
#pragma unroll
        for (int i = 0; i < S::LA; ++i)
            dma16_lds(ar, st + (WAVES * i + wave) * 1024,
                      edge && (last >> i & 1) ? 0x80000000u : aoff[i] + uint32_t(stage * ROWB), 0);
    };
    // scales: PER groups of one feature a thread, through registers
    const int srow = tid / S::PIECES, sfirst = tid % S::PIECES * PER;
    const uint16_t *sp = Q.scales + int64_t(n0 + min(srow, vn - 1)) * ng + sfirst;
    uint32_t sw[PER / 2];
    auto load_panel = [&](int p) {
        const int have = ng - p * NGP - sfirst;
        if (have >= PER)
            read_scales<PER>(sw, sp + p * NGP);
        else
            read_scales_tail<PER>(sw, sp + p * NGP, have);
    };
    auto keep_panel = [&](int p) {
        uint16_t *to = panels + (p & 1) * (NGP * TN) + sfirst * TN + srow;
#pragma unroll
        for (int j = 0; j < PER; ++j)
            to[j * TN] = uint16_t(sw[j >> 1] >> (16 * (j & 1)));
    };

    f32x4 acc[NB][MB];
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
        for (int b = 0; b < MB; ++b)
            acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto compute = [&](int stage) {
        const uint8_t *st = lds8 + (stage & 1) * STAGE;
        const uint16_t *scales = panels + (stage / S::PANEL & 1) * (NGP * TN);
        const int j0 = (2 * stage / GB) % NGP;             // the stage's first group
        bf16x8 af[2][MB];
        uint32_t cw[2][NB];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int c = (wn * NB + nb) * 16 + r16;
                cw[kb][nb] = *reinterpret_cast<const uint32_t *>(st + A_BYTES + c * QROWB + 16 * (kb ^ ((c >> 3) & 1)) + 4 * g);
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                const int r = (wm * MB + mb) * 16 + r16;
                af[kb][mb] = as_bf16x8(*reinterpret_cast<const u32x4 *>(st + r * ROWB + (((4 * kb + g) ^ ((r >> 1) & 7)) << 4)));
            }
        }
        auto scaled = [&](int nb, int j, const f32x4 (&part)[MB]) {
            const uint2 s = *reinterpret_cast<const uint2 *>(scales + j * TN + (wn * NB + nb) * 16 + 4 * g);
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

    load_panel(0);
    issue(0, 0);
    keep_panel(0);
    for (int s = 0; s < nstage; ++s) {
        __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(0));          // this stage landed ...
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (and this wavefront's LDS operations are done with)
        __builtin_amdgcn_s_barrier();                       // ... for every wavefront; the other buffer was last read
        asm volatile("" ::: "memory");                      //     one stage ago
        if (s + 1 < nstage)
            issue(s + 1, (s + 1) & 1);
        // the next panel is read at this one's start and kept at its middle: its place was last read a panel ago
        const int p = s / S::PANEL + 1;
        if (s % S::PANEL == 0 && p * S::PANEL < nstage)
            load_panel(p);
        compute(s);
        if (s % S::PANEL == S::PANEL / 2 && p * S::PANEL < nstage)
            keep_panel(p);
    }
    __syncthreads();                                        // every fragment has been read: LDS changes its use
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
        for (int b = 0; b < MB; ++b)
            acc[a][b] *= 16.0f;                             // the codes were sixteenths
    store_block<ACT, false, NB, MB>(A, reinterpret_cast<float *>(lds8) + wave * STORE_LDS<NB>, acc, m0 + wm * MB * 16,
                                    vm - wm * MB * 16, n0 + wn * NB * 16);
}

template <int MT, int R>
hipError_t launch_rows(const LinearQ4Args &A, int act, hipStream_t st)
{
    const dim3 grid((A.l.N + 16 * R - 1) / (16 * R), (A.l.M + 16 * MT - 1) / (16 * MT));
    if (A.group == 32)
        launch_k(q4_rows_kernel<MT, R, 1>, grid, 64 * ROWS_WAVES, 0, st, A, act);
    else if (A.group == 64)
        launch_k(q4_rows_kernel<MT, R, 2>, grid, 64 * ROWS_WAVES, 0, st, A, act);
    else
        launch_k(q4_rows_kernel<MT, R, 4>, grid, 64 * ROWS_WAVES, 0, st, A, act);
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

}  // namespace

hipError_t launch_linear_q4(const LinearQ4Args &A, int act, hipStream_t st)
{
    if (A.l.M <= 64) {
        if (A.l.M <= 16)
            return launch_rows<1, 1>(A, act, st);
        return A.l.M <= 32 ? launch_rows<2, 2>(A, act, st) : launch_rows<4, 2>(A, act, st);
    }
    using Tile = Q4Shape<128, 128, 2, 2, 2>;
    switch (act) {
    case LINEAR_SILU: return launch_tile<LINEAR_SILU, Tile>(A, st);
    case LINEAR_GELU: return launch_tile<LINEAR_GELU, Tile>(A, st);
    case LINEAR_GELU_TANH: return launch_tile<LINEAR_GELU_TANH, Tile>(A, st);
    default: return launch_tile<LINEAR_NONE, Tile>(A, st);
    }
}

}  // namespace msi
