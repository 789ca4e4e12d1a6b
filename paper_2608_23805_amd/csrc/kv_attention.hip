// kv_attention.hip -- attention over the paged 8-bit cache, gfx950.
//
// For a query row of sequence i at position len - n + r of its tokens, head a
// of the G query heads that share cache head h:
//     s_t = scale * q . k_t      over the tokens t <= len - n + r,
//     p = softmax(s),  out = sum_t p_t v_t,
// and, where the tokens' weights are kept, mass_t = decay * mass_t + the sum of
// p_t over the last mass_rows rows and the G heads.
//
// Rows of one cache head are packed (row, head of the group) so that every byte
// of the cache that a workgroup reads serves all of them.  One pass over the
// cache with a running maximum and sum per row.  Products are transposed:
// S^T = K Q^T and O^T = V^T P^T, so that the scores of a query row stay in one
// lane column, and the token order of an MFMA's reduction is the one in which
// the scores already lie, so P never moves between lanes.  Codes become bf16
// exactly; the block's K scale multiplies the fp32 scores and its V scale the
// probabilities.  Probabilities are rounded to bf16 for the second product,
// the only operand type of its matrix instruction that holds V's codes and that
// range: at most 2^-8 relative each, as the output's own rounding, and about as
// much again in sum where few tokens carry a row (root mean square against 64
// bits: prompt chunks 2.4e-3, single tokens 1.7e-3, of which the output's own
// rounding is 1.7e-3); their sum, the maxima, the scores and all accumulators
// are fp32.
#include <algorithm>

#include "gemm_ring.h"
#include "kernels.h"
#include "kv_device.h"

namespace msi {

namespace {

// Eight codes as bf16 (exact).
template <int FMT>
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t a, uint32_t b)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t w = i ? b : a;
        if constexpr (FMT == KV_INT8) {
            const f32x4 f = kv_unpack4<FMT>(w);
            typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
            r[2 * i] = __builtin_bit_cast(uint32_t, bf16x2_t{static_cast<__bf16>(f[0]), static_cast<__bf16>(f[1])});
            r[2 * i + 1] = __builtin_bit_cast(uint32_t, bf16x2_t{static_cast<__bf16>(f[2]), static_cast<__bf16>(f[3])});
        } else {
            r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
            r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
        }
    }
    return __builtin_bit_cast(bf16x8, r);
}

// 4 x 4 bytes transposed: byte d of word t becomes byte t of word d.
__device__ __forceinline__ void transpose4(const uint32_t (&in)[4], uint32_t (&out)[4])
{
    const uint32_t a = __builtin_amdgcn_perm(in[1], in[0], 0x05010400u);   // t0d0 t1d0 t0d1 t1d1
    const uint32_t b = __builtin_amdgcn_perm(in[1], in[0], 0x07030602u);   // t0d2 t1d2 t0d3 t1d3
    const uint32_t c = __builtin_amdgcn_perm(in[3], in[2], 0x05010400u);
    const uint32_t d = __builtin_amdgcn_perm(in[3], in[2], 0x07030602u);
    out[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

template <typename Op>
__device__ __forceinline__ float across16(float v, Op op)      // over the lanes l % 16 equal
{
    const auto s16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(s16[0]), __uint_as_float(s16[1]));
    const auto s32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(s32[0]), __uint_as_float(s32[1]));
}

__device__ __forceinline__ float vmax(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float vsum(float a, float b) { return a + b; }

// log2 of the sum of a row's powers; a row that sees nothing has none: +infinity makes its probabilities zero.
__device__ __forceinline__ float log_sum(float m, float l) { return l == 0.0f ? INFINITY : m + log2f(l); }

// Rows are numbered row * G + head of the group within a sequence and cache head.
__device__ __forceinline__ int row_limit(const KvSeq &q, int token_row) { return q.len - q.n + token_row + 1; }

// The append takes every finite value, so V reaches the largest bf16 (scales up
// to 2^122), and outputs are sums over up to 2^29 tokens of probabilities (up to
// 2^7 with many rows) before they are divided: units' outputs are kept in units
// of 2^40, which leaves those sums under 2^127.
constexpr float V_LOG = 40.0f, V_DOWN = 0x1p-40f, V_UP = 0x1p40f;

// ---------------------------------------------------------------- units
//
// The caches of a call are cut into units of about equally many blocks, sized
// on the device from the actual lengths, however ragged the batch is and
// however loose the host's bounds are. Units
// are numbered along the sequences, so the workgroups that have work come
// first, and every wavefront finds its unit by a scan of the lengths (64
// sequences a step; a few loads for a usual batch).  Where the host already
// knows that cutting would gain nothing (A.direct), unit i is sequence i whole.
__device__ __forceinline__ int blocks_of(const KvSeqs &s, int i)      // per lane
{
    if (i >= s.S)
        return 0;
    const KvSeq q = kv_check_seq(s.cu[i], s.cu[i + 1], s.lens[i], s.n_rows, s.max_rows, s.max_len, s.all_rows);
    return q.n ? (q.len + KV_BLOCK - 1) / KV_BLOCK : 0;
}

struct Unit {
    int seq, split, n, first;        // the split-th of the n units of sequence seq, which start at number `first`
};

// Blocks of a unit for `work` blocks in all (times heads and row tiles): one
// workgroup per CU as long as each has at most 16 blocks, four a wavefront;
// then units of 16, which hide their start and their partial results' way
// through memory, until there are 2048 of them (131072 tokens of one sequence, 2 heads
// of 256: 36 us with 16 blocks, 46 with 4; 48 sequences of up to 16384, 8 heads of 128:
// 246, 233, 223 and 219 us with 256, 512, 1024 and 2048 workgroups).
// Sequences of up to 8 blocks are not cut (4 to 16 sequences of 500 tokens: 9.3 and 10.1 us,
// 11.6 and 13.5 cut; of 1000 tokens with heads of 256 17.0, 14.1 cut).
constexpr int DIRECT_BLOCKS = 8, LEAST_BLOCKS = 4, ENOUGH_BLOCKS = 16, FILL_WORKGROUPS = 256, MOST_WORKGROUPS = 2048;

__device__ __forceinline__ int unit_chunk(int64_t work)
{
    const int64_t fill = (work + FILL_WORKGROUPS - 1) / FILL_WORKGROUPS;
    if (fill <= ENOUGH_BLOCKS)
        return max(int(fill), LEAST_BLOCKS);
    return int(max(int64_t(ENOUGH_BLOCKS), (work + MOST_WORKGROUPS - 1) / MOST_WORKGROUPS));
}

// The unit numbered `at` (seq = -1: there are not so many).
__device__ __forceinline__ Unit find_unit(const AttentionLaunch &A, int at)
{
    if (A.direct)
        return Unit{at, 0, 1, at};
    const int lane = threadIdx.x & 63;
    const int mine = blocks_of(A.s, lane);
    int total = mine;
    for (int base = 64; base < A.s.S; base += 64)
        total += blocks_of(A.s, base + lane);
    total = __builtin_amdgcn_readlane(wave_scan_incl(total), 63);
    const int chunk = unit_chunk(int64_t(total) * A.per);
    int before = 0;
    for (int base = 0; base < A.s.S; base += 64) {
        const int b = base ? blocks_of(A.s, base + lane) : mine;
        const int n = (b + chunk - 1) / chunk, incl = wave_scan_incl(n);
        const uint64_t hit = __ballot(at < before + incl);
        if (hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            const int nl = __builtin_amdgcn_readlane(n, l), first = before + __builtin_amdgcn_readlane(incl, l) - nl;
            return Unit{base + l, at - first, nl, first};
        }
        before += __builtin_amdgcn_readlane(incl, 63);
    }
    return Unit{-1, 0, 0, 0};
}

// Blocks [first, second) of a unit of a sequence of `blocks`.
__device__ __forceinline__ int2 unit_blocks(const Unit &u, int blocks)
{
    return make_int2(int(int64_t(blocks) * u.split / u.n), int(int64_t(blocks) * (u.split + 1) / u.n));
}

// Index of a packed row's partial result.
__device__ __forceinline__ int64_t part_index(const AttentionLaunch &A, int unit, int h, int r)
{
    return (int64_t(unit) * A.c.H + h) * A.part_rows + r;
}

// First score of a block: by page where the pool is smaller than the batch's tables.
__device__ __forceinline__ int64_t score_index(const AttentionLaunch &A, int i, int blk, int page, int h, int row)
{
    const int64_t at = A.score_blocks ? int64_t(i) * A.score_blocks + blk : int64_t(page);
    return ((at * A.c.H + h) * A.part_rows + row) * KV_BLOCK;
}

// ---------------------------------------------------------------- other rows
//
// Rows that no sequence answers for: those between and behind the sequences'
// rows and those of a sequence whose numbers break a bound.  Workgroups behind
// the grid's units take 64 rows at a time, mark which of them some sequence
// brings (offsets that fall could overlap, so every sequence is looked at) and
// clear the others.  They run beside the units (a block's step of 16 single tokens 38.5 us with and without them, 42
// with a launch of their own).  Calls without them take kernels without their code, which costs those 0.5 to 2 %.
constexpr int REST_ROWS = 64, MOST_REST = 128;

__host__ __device__ __forceinline__ int rest_groups(const KvSeqs &s)
{
    return s.all_rows ? min((s.n_rows + REST_ROWS - 1) / REST_ROWS, MOST_REST) : 0;
}

// Rows 64 group .., 64 (group + groups) .. and so on; `words`: 8 words of LDS.
__device__ __forceinline__ void clear_rest(const KvSeqs &s, uint16_t *__restrict__ out, int64_t stride, int width, int group,
                                           int groups, uint32_t *words)
{
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    for (int64_t first = int64_t(group) * REST_ROWS; first < s.n_rows; first += int64_t(groups) * REST_ROWS) {
        const int r0 = int(first), n = min(REST_ROWS, s.n_rows - r0);
        uint64_t rows = 0;
        for (int i = threadIdx.x; i < s.S; i += 256) {
            const KvSeq q = kv_check_seq(s.cu[i], s.cu[i + 1], s.lens[i], s.n_rows, s.max_rows, s.max_len, true);
            const int lo = max(q.row0 - r0, 0), hi = min(q.row0 - r0 + q.n, n);
            if (q.n > 0 && lo < hi)
                rows |= (~uint64_t(0) >> (64 - (hi - lo))) << lo;
        }
        auto either = [](float a, float b) { return __uint_as_float(__float_as_uint(a) | __float_as_uint(b)); };
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float w = wave_reduce(__uint_as_float(uint32_t(rows >> 32 * k)), either);
            if ((threadIdx.x & 63) == 0)
                words[2 * wave + k] = __float_as_uint(w);
        }
        __syncthreads();
        uint32_t brought[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
            brought[k] = __builtin_amdgcn_readfirstlane(words[k] | words[2 + k] | words[4 + k] | words[6 + k]);
        for (int r = 0; r < n; ++r)
            if (!(brought[r >> 5] >> (r & 31) & 1))
                for (int c = threadIdx.x; c < width / 8; c += 256)
                    *reinterpret_cast<u32x4 *>(out + (first + r) * stride + 8 * c) = u32x4{0, 0, 0, 0};
        __syncthreads();
    }
}

__global__ void __launch_bounds__(256) kv_rest_kernel(KvSeqs s, uint16_t *out, int64_t stride, int width)
{
    __shared__ uint32_t words[8];
    clear_rest(s, out, stride, width, int(blockIdx.x), int(gridDim.x), words);
}

// ---------------------------------------------------------------- few rows
//
// Up to 16 RT packed rows (single tokens, drafted tokens): bound by reading the
// cache.  No LDS on the way: the wavefront's loads are the MFMA operands.  A
// workgroup of four wavefronts takes a unit's blocks, the wavefronts every
// fourth one; their results meet in LDS, and those of a sequence's units in
// the finish kernel.  Single tokens of 48 sequences of up to 16384, 8 heads of
// 128: 167 us, 5.1 TB/s of codes (a large copy moves 4.65); 189 us where the
// scores are stored for the weights.  A small call is bound by the chain of
// lengths, pages, codes: 5 us.  (Steps of 32 tokens with heads of 128: the same;
// held to three wavefronts a SIMD: 282 us, spilled registers; loads past the
// caches: slower.  Two row tiles of 256 by one wavefront a SIMD, with 62 us for 16
// sequences of up to 8192, are as fast as one tile each by half of the wavefronts.)
//
// K: lane (i, j) = (lane % 16, lane / 16) reads 16 bytes 16 j of each 64-byte
// piece of token 16 g + i; the elements of a reduction step of 32 are in the
// order 64 (c / 2) + 16 j + 8 (c % 2) + 0..7, and the queries are read in the same.
// V: lane (i, j) reads D / 16 bytes from i D / 16 of the eight tokens
// 32 u + 4 j + 0..3 and 32 u + 16 + 4 j + 0..3, whose scores it holds, and
// transposes them in registers to eight tokens of each of its D / 16 elements.
template <int FMT, int D, int RT>
struct FewRows {
    static constexpr int TOK = D * RT >= 256 ? 32 : KV_BLOCK;    // tokens of a step: what fits the registers
    static constexpr int STEPS = KV_BLOCK / TOK;            // steps of a block
    static constexpr int GT = TOK / 16;                     // groups of 16 tokens
    static constexpr int KL = D / 64;                       // 16-byte loads of a K row per lane
    static constexpr int W = D / 16;                        // V bytes per lane and token
    static constexpr int VW = W / 4;                        // words
    static constexpr int OS = D + 4;                        // LDS row stride of the outputs (words)

    struct Codes {
        u32x4 k[GT][KL];
        uint32_t v[GT / 2][8][VW];
    };

    static __device__ __forceinline__ void load_k(u32x4 (&k)[GT][KL], const uint8_t *block, int step)
    {
        const int lane = threadIdx.x & 63;
        const uint8_t *p = block + (step * TOK + (lane & 15)) * D + 16 * (lane >> 4);
#pragma unroll
        for (int g = 0; g < GT; ++g)
#pragma unroll
            for (int l = 0; l < KL; ++l)
                k[g][l] = *reinterpret_cast<const u32x4 *>(p + 16 * g * D + 64 * l);
    }

    static __device__ __forceinline__ void load_v(uint32_t (&v)[GT / 2][8][VW], const uint8_t *block, int step)
    {
        const int lane = threadIdx.x & 63;
        const uint8_t *p = block + KV_BLOCK * D + (step * TOK + 4 * (lane >> 4)) * D + (lane & 15) * W;
#pragma unroll
        for (int u = 0; u < GT / 2; ++u)
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const uint8_t *a = p + (32 * u + (t < 4 ? t : 12 + t)) * D;
                typedef __attribute__((ext_vector_type(VW))) uint32_t vec;
                const vec w = *reinterpret_cast<const vec *>(a);
                if constexpr (VW == 1) {
                    v[u][t][0] = w[0];
                } else {
#pragma unroll
                    for (int x = 0; x < VW; ++x)
                        v[u][t][x] = w[x];
                }
            }
    }
};

template <int FMT, int D, int RT, bool ALL>
__global__ void __launch_bounds__(256, D * RT >= 512 ? 1 : 2) kv_few_rows_kernel(AttentionLaunch A)
{
    using F = FewRows<FMT, D, RT>;
    constexpr int TOK = F::TOK, GT = F::GT, W = F::W, VW = F::VW, OS = F::OS;
    __shared__ __attribute__((aligned(16))) float olds[4][16][OS];
    __shared__ float ml[4][RT][16][2];
    __shared__ float lsum[16 * RT];
    constexpr bool QLDS = D == 256 && RT == 2;               // two tiles of long queries do not fit the registers
    __shared__ bf16x8 qlds[QLDS ? RT * (D / 32) * 64 : 1];

    if constexpr (ALL)
        if (int(blockIdx.x) >= A.main) {
            clear_rest(A.s, A.out, A.out_stride, A.c.H * A.G * D, int(blockIdx.x) - A.main, int(gridDim.x) - A.main,
                       reinterpret_cast<uint32_t *>(lsum));
            return;
        }
    const Unit unit = find_unit(A, int(blockIdx.x) / A.per);
    if (unit.seq < 0)
        return;
    const int i = unit.seq, sub = int(blockIdx.x) % A.per, h = sub % A.c.H, tile = sub / A.c.H;
    const KvSeq q = kv_seq(A.s, i, A.s.all_rows);
    if (!q.ok && sub == 0 && threadIdx.x == 0)
        kv_raise(A.status, KV_BAD_LENGTH);
    if (A.plan && unit.split == 0 && sub == 0 && threadIdx.x == 0)
        A.plan[i] = make_int2(unit.first, unit.n);
    const int rows = q.n * A.G, r0 = tile * 16 * RT;
    const int2 range = unit_blocks(unit, (q.len + KV_BLOCK - 1) / KV_BLOCK);
    const int b0 = range.x, b1 = range.y;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, j = lane >> 4;
    // the weights of a sequence that is not cut: its only workgroup has the rows' sums and reads its scores back (by
    // the finish kernel: 4 sequences of 200 tokens 11.4 us for 8.5, 1024 of 2000 tokens 560 for 542)
    auto weigh = [&]() {
        for (int b = b0 + wave; b < b1; b += 4) {
            const int page = A.s.table[int64_t(i) * A.s.max_blocks + b];
            if (!kv_page_ok(page, A.c.n_pages) || b * KV_BLOCK + lane >= q.len)
                continue;
            const float *src = A.scores + score_index(A, i, b, page, h, 0) + lane;
            float *dst = A.c.mass + (int64_t(page) * A.c.H + h) * KV_BLOCK + lane;
            const float was = A.decay != 0.0f ? *dst : 0.0f;
            float w = 0.0f;
#pragma unroll 4
            for (int r = max(q.n - A.mass_rows, 0) * A.G; r < rows; ++r)
                w += __builtin_amdgcn_exp2f(src[r * KV_BLOCK] - lsum[r]);
            *dst = A.decay != 0.0f ? fmaf(A.decay, was, w) : w;
        }
    };
    const bool weighs = A.direct && A.scores;
    if (r0 >= rows) {
        if (weighs)
            weigh();                                           // (no rows: the weights decay)
        return;
    }

    // pages of this wavefront's next 64 blocks, one a lane (-1: bad)
    auto page_list = [&](int k) {
        const int b = b0 + wave + 4 * (k + lane);
        int page = -1;
        if (b < b1) {
            page = A.s.table[int64_t(i) * A.s.max_blocks + b];
            if (!kv_page_ok(page, A.c.n_pages)) {
                kv_raise(A.status, KV_BAD_PAGE);
                page = -1;
            }
        }
        return page;
    };
    int pages = page_list(0);

    bf16x8 qf[QLDS ? 1 : RT][QLDS ? 1 : D / 32];
    int limit[RT];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int r = r0 + 16 * x + col, rc = min(r, rows - 1);
        const int tr = rc / A.G, hd = rc - tr * A.G;
        limit[x] = r < rows ? row_limit(q, tr) : 0;
        const uint16_t *src = A.q + (int64_t(q.row0) + tr) * A.q_stride + (h * A.G + hd) * D;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            const bf16x8 v = *reinterpret_cast<const bf16x8 *>(src + 64 * (c / 2) + 16 * j + 8 * (c % 2));
            if constexpr (QLDS) {
                if (wave == 0)
                    qlds[(x * (D / 32) + c) * 64 + lane] = v;
            } else {
                qf[x][c] = v;
            }
        }
    }
    if constexpr (QLDS)
        __syncthreads();
    auto query = [&](int x, int c) {
        if constexpr (QLDS)
            return qlds[(x * (D / 32) + c) * 64 + lane];
        else
            return qf[x][c];
    };

    f32x4 acc[RT][W];
    float m[RT], l[RT];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        m[x] = -INFINITY;
        l[x] = 0.0f;
#pragma unroll
        for (int c = 0; c < W; ++c)
            acc[x][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const int nb = b1 - b0 > wave ? (b1 - b0 - wave + 3) / 4 : 0;      // blocks of this wavefront
    const int steps = nb * F::STEPS;
    auto block_at = [&](int page) { return A.c.data + kv_offset(max(page, 0), h, A.c.H, D); };
    auto scales_at = [&](int page) {
        return *reinterpret_cast<const float2 *>(A.c.scales + (int64_t(max(page, 0)) * A.c.H + h) * 2);
    };
    typename F::Codes cur;
    float2 sc{1.0f, 1.0f};
    int page = __builtin_amdgcn_readlane(pages, 0);
    if (steps > 0) {
        sc = scales_at(page);
        F::load_k(cur.k, block_at(page), 0);
        F::load_v(cur.v, block_at(page), 0);
    }
    for (int s = 0; s < steps; ++s) {
        const int blk = b0 + wave + 4 * (s / F::STEPS);
        const bool here = page >= 0;
        const int t0 = blk * KV_BLOCK + (s % F::STEPS) * TOK;
        const int s1 = min(s + 1, steps - 1), k1 = s1 / F::STEPS;
        if (k1 % 64 == 0 && k1 != s / F::STEPS)
            pages = page_list(k1);
        const int page1 = __builtin_amdgcn_readlane(pages, k1 % 64);
        const uint8_t *next = block_at(page1);
        const float2 sc_next = scales_at(page1);

        // ---- scores of TOK tokens (rows of S^T) and 16 RT rows (columns)
        f32x4 sv[RT][GT];
#pragma unroll
        for (int g = 0; g < GT; ++g) {
#pragma unroll
            for (int x = 0; x < RT; ++x)
                sv[x][g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                const bf16x8 kf = codes_bf16<FMT>(cur.k[g][c / 2][2 * (c % 2)], cur.k[g][c / 2][2 * (c % 2) + 1]);
#pragma unroll
                for (int x = 0; x < RT; ++x)
                    sv[x][g] = mfma16(kf, query(x, c), sv[x][g]);
            }
        }
        F::load_k(cur.k, next, s1 % F::STEPS);                 // (the last step reads its own block again)

        const float ks = (here ? sc.x : 0.0f) * A.scale_log2, vs = here ? sc.y * V_DOWN : 0.0f;
        const bool tail = !here || t0 + TOK > q.len;
        if (tail) {                                            // bytes past the last token may be anything
#pragma unroll
            for (int u = 0; u < GT / 2; ++u)
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const int tok = t0 + 32 * u + 4 * j + (t < 4 ? t : 12 + t);
#pragma unroll
                    for (int w = 0; w < VW; ++w)
                        cur.v[u][t][w] = here && tok < q.len ? cur.v[u][t][w] : 0u;
                }
        }
        bf16x8 pf[RT][GT / 2];
#pragma unroll
        for (int x = 0; x < RT; ++x) {
            float top = -INFINITY;
            // every row sees the whole step unless the step reaches past the first row's limit
            const bool masked = !here || t0 + TOK > q.len - q.n + 1 || r0 + 16 * (x + 1) > rows;
#pragma unroll
            for (int g = 0; g < GT; ++g)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float z = sv[x][g][r] * ks;
                    if (masked)
                        z = here && t0 + 16 * g + 4 * j + r < limit[x] ? z : -INFINITY;
                    sv[x][g][r] = z;
                    top = fmaxf(top, z);
                }
            if (A.scores && r0 + 16 * x + col < rows) {
                float *dst = A.scores + score_index(A, i, blk, page, h, r0 + 16 * x + col) + (s % F::STEPS) * TOK + 4 * j;
                if (here || A.score_blocks)
#pragma unroll
                    for (int g = 0; g < GT; ++g)
                        *reinterpret_cast<f32x4 *>(dst + 16 * g) = sv[x][g];
            }
            top = across16(top, vmax);
            const float m1 = fmaxf(m[x], top);
            const float ref = m1 == -INFINITY ? 0.0f : m1;
            if (__any(m1 != m[x])) {
                const float a = __builtin_amdgcn_exp2f(m[x] - ref);
                l[x] *= a;
#pragma unroll
                for (int c = 0; c < W; ++c)
                    acc[x][c] *= a;
                m[x] = m1;
            }
            float sum = 0.0f;
#pragma unroll
            for (int g = 0; g < GT; ++g)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float p = __builtin_amdgcn_exp2f(sv[x][g][r] - ref);
                    sum += p;
                    sv[x][g][r] = p * vs;
                }
            l[x] += sum;
#pragma unroll
            for (int u = 0; u < GT / 2; ++u)
                pf[x][u] = __builtin_bit_cast(
                    bf16x8, u32x4{pack_bf16x2_hw(sv[x][2 * u][0], sv[x][2 * u][1]), pack_bf16x2_hw(sv[x][2 * u][2], sv[x][2 * u][3]),
                                  pack_bf16x2_hw(sv[x][2 * u + 1][0], sv[x][2 * u + 1][1]),
                                  pack_bf16x2_hw(sv[x][2 * u + 1][2], sv[x][2 * u + 1][3])});
        }
        // ---- O^T: lane (i, j) holds elements i D / 16 + c of the eight tokens
#pragma unroll
        for (int u = 0; u < GT / 2; ++u)
#pragma unroll
            for (int w = 0; w < VW; ++w) {
                uint32_t lo[4], hi[4];
                const uint32_t a[4] = {cur.v[u][0][w], cur.v[u][1][w], cur.v[u][2][w], cur.v[u][3][w]};
                const uint32_t b[4] = {cur.v[u][4][w], cur.v[u][5][w], cur.v[u][6][w], cur.v[u][7][w]};
                transpose4(a, lo);
                transpose4(b, hi);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bf16x8 vf = codes_bf16<FMT>(lo[e], hi[e]);
#pragma unroll
                    for (int x = 0; x < RT; ++x)
                        acc[x][4 * w + e] = mfma16(vf, pf[x][u], acc[x][4 * w + e]);
                }
            }
        F::load_v(cur.v, next, s1 % F::STEPS);
        sc = sc_next;
        page = page1;
    }

    // ---- the four wavefronts' results: lane (col, j) holds elements (4 j + r) W + c of row col
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const float lx = across16(l[x], vsum);
        if (j == 0) {
            ml[wave][x][col][0] = m[x];
            ml[wave][x][col][1] = lx;
        }
    }
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        if (x)
            __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < W; c += 4)
                *reinterpret_cast<f32x4 *>(&olds[wave][col][(4 * j + r) * W + c]) =
                    f32x4{acc[x][c][r], acc[x][c + 1][r], acc[x][c + 2][r], acc[x][c + 3][r]};
        __syncthreads();
        // thread: row tid / 16, elements tid % 16 * 4 + 64 k
        const int row = tid >> 4, r = r0 + 16 * x + row;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            mx = fmaxf(mx, ml[w][x][row][0]);
        const float ref = mx == -INFINITY ? 0.0f : mx;
        float a[4], sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            a[w] = __builtin_amdgcn_exp2f(ml[w][x][row][0] - ref);
            sum += a[w] * ml[w][x][row][1];
        }
        if ((tid & 15) == 0)
            lsum[16 * x + row] = log_sum(mx, sum);
        if (r < rows) {
            const int tr = r / A.G, hd = r - tr * A.G;
            const int64_t part = part_index(A, unit.first + unit.split, h, r);
            if ((tid & 15) == 0 && !A.direct) {
                A.part_ml[2 * part] = mx;
                A.part_ml[2 * part + 1] = sum;
            }
            const float inv = sum == 0.0f ? 0.0f : V_UP / sum;
#pragma unroll
            for (int k = 0; k < D / 64; ++k) {
                const int e = (tid & 15) * 4 + 64 * k;
                f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    o += a[w] * *reinterpret_cast<const f32x4 *>(&olds[w][row][e]);
                if (A.direct) {
                    uint16_t *dst = A.out + (int64_t(q.row0) + tr) * A.out_stride + (h * A.G + hd) * D + e;
                    *reinterpret_cast<uint2 *>(dst) =
                        make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
                } else {
                    *reinterpret_cast<f32x4 *>(A.part_o + part * D + e) = o;
                }
            }
        }
    }
    if (weighs) {
        __syncthreads();                                       // (the scores that the four wavefronts stored, and lsum)
        weigh();
    }
}

// ---------------------------------------------------------------- many rows
//
// Bound by the matrix cores and the vector unit beside them.  A workgroup of
// four wavefronts owns 128 packed rows, 32 a wavefront, and walks the cache a
// block of 64 tokens at a time.  The blocks' codes are copied as they are into
// a ring of three LDS buffers (half the LDS traffic of bf16 tiles, which would
// bound 32-row wavefronts) and become bf16 on their way from LDS to
// v_mfma_f32_32x32x16_bf16.  With D = 256 the 32 rows' outputs alone take 128
// registers, so the queries lie in LDS as well, in the order of their fragments; that keeps
// everything in the vector registers, where the rescaling needs the outputs (in
// the accumulation registers every block would move all of them there and back:
// 753 us for 640).  4096 rows on top of 4096 tokens, two sequences, 16 query heads
// of 256: 890 us, 926 TFLOP/s; 32 of 128: 795 us, 1038 TFLOP/s (int8 codes, whose
// conversion takes the vector unit twice as long: about 790).  The conversions
// bound it: with heads of 256 and eight wavefronts of 16 rows, two a SIMD, every
// wavefront converts the whole block, 928 us for 890.
//
// LDS: 16-byte chunk c of token row t (K rows, then V rows) sits at slot
// c ^ many_swz(t) of its row: the 16-byte reads of eight consecutive K rows and the
// transposing reads of the eight V rows of a lane group fall on distinct banks.
// K: lane (i, hf) = (lane % 32, lane / 32) reads chunk 2 p + hf of token i: the
// reduction order of MFMA 2 p + e is d = 16 (2 p + hf) + 8 e + 0..7, and the
// queries are read in the same.  V: ds_read_b64_tr_b8 hands lane b + 8 x of a
// 16-lane group byte b of the eight bytes that lanes x, x + 2, .. x + 14 point
// at, so the lanes point at the eight tokens whose scores they hold and come
// back with eight tokens of one element.
template <int D>
struct ManyRows {
    static constexpr int ROWS = 128, NBUF = 3;
    static constexpr int BLOCK = 2 * KV_BLOCK * D;        // bytes of a block's codes
    static constexpr int COPIES = BLOCK / 4096;           // copy instructions of a wavefront and block
    static constexpr int CPR = D / 16;                    // chunks of a row
    static constexpr bool QLDS = D == 256;
    static constexpr int QBYTES = QLDS ? ROWS * D * 2 : 0;
    static constexpr size_t LDS = size_t(NBUF) * BLOCK + QBYTES;
    static_assert(LDS <= 160 * 1024, "");
};

template <int D>
__device__ __forceinline__ int many_swz(int t)
{
    return ((t & 3) | ((t >> 1) & 4) | ((t << 1) & 8)) & (D / 16 - 1);
}

// Copies of one block into LDS: copy i of a wavefront covers 16-byte slots 64 (4 i + wave) .., whole groups of
// 16 rows apart, so a lane's offset within the block is one number for all of them.  Rows past `valid` (none
// of the block with valid = 0) become zeros: an offset past the buffer's end reads nothing.
template <int D>
struct CopyLane {
    uint32_t offset;
    int row;

    __device__ __forceinline__ CopyLane()
    {
        const int at = int(threadIdx.x), c = at % ManyRows<D>::CPR;
        row = at / ManyRows<D>::CPR;
        offset = uint32_t(row * D + ((c ^ many_swz<D>(row)) << 4));
    }

    __device__ __forceinline__ void copy(uint8_t *lds, const uint8_t *block, int valid) const
    {
        using M = ManyRows<D>;
        const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
        const __amdgpu_buffer_rsrc_t r =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(block), 0, M::BLOCK, ring::RSRC_FLAGS);
#pragma unroll
        for (int i = 0; i < M::COPIES; ++i)
            dma16_lds(r, lds + (i * 4 + wave) * 1024,
                      row < valid - (i * 4096 / D & (KV_BLOCK - 1)) ? offset : 0x80000000u, i * 4096);
    }
};

__device__ __forceinline__ float across32(float v, float (*op)(float, float))
{
    const auto s32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(s32[0]), __uint_as_float(s32[1]));
}

// Fragment c of the queries of 32 rows from r0 on (lane's row r0 + lane % 32); their sign takes a negative scale's.
template <int D>
__device__ __forceinline__ void load_q32(bf16x8 (&qf)[D / 16], const AttentionLaunch &A, const KvSeq &q, int h, int r0,
                                         int rows)
{
    const int lane = threadIdx.x & 63;
    const int rc = min(r0 + (lane & 31), rows - 1), tr = rc / A.G, hd = rc - tr * A.G;
    const uint16_t *src = A.q + (int64_t(q.row0) + tr) * A.q_stride + (h * A.G + hd) * D + 16 * (lane >> 5);
    const uint32_t flip = A.scale_log2 < 0.0f ? 0x80008000u : 0u;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(src + 32 * (c / 2) + 8 * (c % 2));
        qf[c] = as_bf16x8(v ^ u32x4{flip, flip, flip, flip});
    }
}

// S^T of 64 tokens and 32 rows: sv[b][v] is token 32 b + 8 (v / 4) + 4 hf + v % 4 of the lane's row.
// query(c): fragment c.
template <int FMT, int D, typename Query>
__device__ __forceinline__ void scores32(f32x16 (&sv)[2], const uint8_t *__restrict__ lds, Query query)
{
    const int lane = threadIdx.x & 63;
    const int t = lane & 31, swz = many_swz<D>(t), hf = lane >> 5;   // (many_swz(t + 32) is the same)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v)
            sv[b][v] = 0.0f;
#pragma unroll
    for (int p = 0; p < D / 32; ++p) {
        const bf16x8 q0 = query(2 * p), q1 = query(2 * p + 1);
        u32x4 w[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
            w[b] = *reinterpret_cast<const u32x4 *>(lds + (32 * b + t) * D + (((2 * p + hf) ^ swz) << 4));
#pragma unroll
        for (int b = 0; b < 2; ++b)
            sv[b] = mfma32(codes_bf16<FMT>(w[b][0], w[b][1]), q0, sv[b]);
#pragma unroll
        for (int b = 0; b < 2; ++b)
            sv[b] = mfma32(codes_bf16<FMT>(w[b][2], w[b][3]), q1, sv[b]);
    }
}

typedef __attribute__((ext_vector_type(2))) int i32x2;
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// Eight tokens of one element for every lane, see above; `at`: the lane's own eight bytes.
__device__ __forceinline__ i32x2 read_tr8(const uint8_t *at)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)at);
#else
    (void)at;
    return i32x2{0, 0};
#endif
}

// Copies of a later block into `later`, then the scores of the block at `tile`.  The
// LDS parts are restricted parameters, here and below, or the compiler would have reads of one
// buffer wait for every copy in flight into another.
template <int FMT, int D, typename Query>
__device__ __forceinline__ void copy_and_score(f32x16 (&sv)[2], const uint8_t *__restrict__ tile, Query query,
                                               uint8_t *__restrict__ later, const CopyLane<D> &cl, const uint8_t *block,
                                               int valid)
{
    cl.copy(later, block, valid);
    scores32<FMT, D>(sv, tile, query);
}

// O^T += V^T P^T of the block at `tile`.
template <int FMT, int D>
__device__ __forceinline__ void times_v(f32x16 (&acc)[D / 32], const bf16x8 (&pf)[4], const uint8_t *__restrict__ tile,
                                        const uint32_t (&chunk)[D / 32])
{
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            const i32x2 w = read_tr8(tile + 16 * u * D + chunk[c]);
            acc[c] = mfma32(codes_bf16<FMT>(uint32_t(w[0]), uint32_t(w[1])), pf[u], acc[c]);
        }
}

constexpr float NO_SCALE = 0x1p-126f;       // a scale of 0 counts as this (its logarithm is finite)
// The exponent of a probability takes its block's V scale, and the rows' sums come from the same powers.  Up to V scales of
// 2^60 that fits binary32 as it is.  From the first list of blocks with a larger one on, a wavefront goes over to units of
// 2^40; blocks whose scale is under 2^-24 (vanishing V, zeros among them) then have their share of the rows' sums computed
// by itself, since tokens below 2^-22 of the largest would be lost with scales of 2^-64.  Two sequences of 2041 and 3815
// rows, heads of 256: 670 us, 667 without.
constexpr float LARGE_V_LOG = 60.0f, LOW_V_LOG = -24.0f;

// Running maximum and sum of a block's powers by themselves.
__device__ __forceinline__ void add_low(const f32x16 (&sv)[2], float ks, float &m, float &l)
{
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int v = 0; v < 16; ++v)
            top = fmaxf(top, sv[x][v]);
    const float m1 = fmaxf(m, across32(top, vmax) * ks), ref = m1 == -INFINITY ? 0.0f : m1;
    l *= __builtin_amdgcn_exp2f(m - ref);
    m = m1;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int v = 0; v < 16; ++v)
            l += __builtin_amdgcn_exp2f(fmaf(sv[x][v], ks, -ref));
}

template <int FMT, int D, bool ALL>
__global__ void __launch_bounds__(256, 2) kv_many_rows_kernel(AttentionLaunch A)
{
    using M = ManyRows<D>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds8[];
    if constexpr (ALL)
        if (int(blockIdx.x) >= A.main) {
            clear_rest(A.s, A.out, A.out_stride, A.c.H * A.G * D, int(blockIdx.x) - A.main, int(gridDim.x) - A.main,
                       reinterpret_cast<uint32_t *>(lds8));
            return;
        }
    const Unit unit = find_unit(A, int(blockIdx.x) / A.per);
    if (unit.seq < 0)
        return;
    // the last row tiles, which see the most tokens, start first
    const int i = unit.seq, sub = A.per - 1 - int(blockIdx.x) % A.per, h = sub % A.c.H, r0 = sub / A.c.H * M::ROWS;
    const KvSeq q = kv_seq(A.s, i, A.s.all_rows);
    if (!q.ok && sub == 0 && threadIdx.x == 0)
        kv_raise(A.status, KV_BAD_LENGTH);
    if (A.plan && unit.split == 0 && sub == 0 && threadIdx.x == 0)
        A.plan[i] = make_int2(unit.first, unit.n);
    const int rows = q.n * A.G;
    if (r0 >= rows)
        return;
    // blocks up to the last row's limit
    const int last = min(r0 + M::ROWS, rows) - 1;
    const int most = max(row_limit(q, last / A.G), 0);
    const int2 range = unit_blocks(unit, (q.len + KV_BLOCK - 1) / KV_BLOCK);
    const int b0 = range.x, b1 = min(range.y, (most + KV_BLOCK - 1) / KV_BLOCK);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hf = lane >> 5;
    const int w0 = r0 + 32 * wave;                          // this wavefront's rows
    const bool idle = w0 >= rows;
    const int r = w0 + col;
    const int limit = r < rows ? row_limit(q, r / A.G) : 0;
    const int least = idle ? 0 : row_limit(q, w0 / A.G);    // the first row's limit: blocks below it need no mask
    const int wave_most = idle ? 0 : row_limit(q, min(w0 + 31, rows - 1) / A.G);

    bf16x8 qf[D / 16];
    load_q32<D>(qf, A, q, h, w0, rows);
    bf16x8 *const ql = reinterpret_cast<bf16x8 *>(lds8 + M::NBUF * M::BLOCK) + wave * (D / 16) * 64 + lane;
    if constexpr (M::QLDS)                                  // (each lane reads what it wrote)
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            ql[c * 64] = qf[c];
    auto query = [&](int c) {
        if constexpr (M::QLDS)
            return ql[c * 64];
        else
            return qf[c];
    };
    f32x16 acc[D / 32];
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int v = 0; v < 16; ++v)
            acc[c][v] = 0.0f;
    float m = -INFINITY, l = 0.0f;                          // m: reference of the exponents, a whole number
    float m_low = -INFINITY, l_low = 0.0f;                  // maximum and sum of the low blocks

    // page (-1: bad), K factor and log2 of the V scale in the present units of the 64 blocks from `list_at` on, one a lane;
    // `lows`: those of low blocks
    int list_at = b0 - 64, pages = -1;
    float kscale = 0.0f, vlog = 0.0f, v_units = 0.0f;
    uint64_t lows = 0;
    const float factor = fabsf(A.scale_log2);
    auto make_list = [&](int b) {
        list_at = b;
        pages = -1;
        kscale = 1e-37f, vlog = 0.0f;
        if (b + lane < b1) {
            pages = A.s.table[int64_t(i) * A.s.max_blocks + b + lane];
            if (!kv_page_ok(pages, A.c.n_pages)) {
                kv_raise(A.status, KV_BAD_PAGE);
                pages = -1;
            } else {
                const float2 sc = *reinterpret_cast<const float2 *>(A.c.scales + (int64_t(pages) * A.c.H + h) * 2);
                kscale = fmaxf(sc.x * factor, 1e-37f);       // (not 0: times -infinity that would be NaN)
                vlog = log2f(fmaxf(sc.y, NO_SCALE));         // whole for powers of two
            }
        }
        if (v_units == 0.0f && __any(vlog > LARGE_V_LOG)) {
            v_units = V_LOG;
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
                acc[c] *= V_DOWN;
        }
        lows = __ballot(v_units != 0.0f && vlog < LOW_V_LOG);
        vlog -= v_units;
    };
    int next_pages = -1, next_at = b0;                      // pages of the copies, which run ahead of the list
    auto copy_list = [&](int b) {
        next_at = b;
        next_pages = -1;
        if (b + lane < b1) {
            next_pages = A.s.table[int64_t(i) * A.s.max_blocks + b + lane];
            if (!kv_page_ok(next_pages, A.c.n_pages))
                next_pages = -1;
        }
    };
    copy_list(b0);
    const CopyLane<D> cl;
    auto block_at = [&](int b) {
        if (b - next_at == 64)
            copy_list(b);
        return A.c.data + kv_offset(max(__builtin_amdgcn_readlane(next_pages, b - next_at), 0), h, A.c.H, D);
    };
    auto valid_at = [&](int b) {                            // (blocks past the end copy zeros: the waits count on them)
        return __builtin_amdgcn_readlane(next_pages, b - next_at) >= 0 ? q.len - b * KV_BLOCK : 0;
    };
    auto issue = [&](int b) {
        const uint8_t *block = block_at(b);
        cl.copy(lds8 + (b - b0) % M::NBUF * M::BLOCK, block, valid_at(b));
    };
    auto arrive = [&](auto waitn) {
        __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(decltype(waitn)::value));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wavefront's reads are done with
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    issue(b0);
    issue(b0 + 1);
    // this lane's bytes of V: token row 64 + 16 u + tv, elements 32 c + 16 (lane / 16 % 2) + 8 (lane % 2) ..
    const int tl = (lane & 15) >> 1, tv = (tl < 4 ? tl : 4 + tl) + 4 * hf;
    const int vswz = many_swz<D>(tv);                       // (the same for tv + 16 u)
    const int vc = (lane >> 4) & 1;
    uint32_t vchunk[D / 32];
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
        vchunk[c] = uint32_t(((2 * c + vc) ^ vswz) << 4);
    const uint32_t vrow = uint32_t((KV_BLOCK + tv) * D + 8 * (lane & 1));

    for (int b = b0; b < b1; ++b) {
        // block b has landed (b + 1 is in flight); the buffer of block b - 1 is free
        arrive(std::integral_constant<int, M::COPIES>{});
        if (b - list_at == 64)
            make_list(b);
        const int t0 = b * KV_BLOCK;
        const uint8_t *block = block_at(b + 2);
        const int valid = valid_at(b + 2);
        const uint8_t *const tile = lds8 + (b - b0) % M::NBUF * M::BLOCK;
        uint8_t *const later = lds8 + (b + 2 - b0) % M::NBUF * M::BLOCK;
        if (t0 >= wave_most) {                              // (as is every later block)
            cl.copy(later, block, valid);
            continue;
        }
        f32x16 sv[2];
        copy_and_score<FMT, D>(sv, tile, query, later, cl, block, valid);
        const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(kscale), b - list_at));
        const float vl = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vlog), b - list_at));
        const bool here = __builtin_amdgcn_readlane(pages, b - list_at) >= 0;
        const bool low = lows >> (b - list_at) & 1;
        if (low || !here || t0 + KV_BLOCK > least) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    sv[x][v] = here && t0 + 32 * x + 8 * (v >> 2) + 4 * hf + (v & 3) < limit ? sv[x][v] : -INFINITY;
            if (low)                                        // (in a branch of its own, further down: 689 to 722 us for 667)
                add_low(sv, ks, m_low, l_low);
        }
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                top = fmaxf(top, sv[x][v]);
        top = across32(top, vmax) * ks;
        // the reference follows the maximum once it is 2^6 ahead: any reference gives the same quotients
        if (__any(top > m + 6.0f)) {
            const float m1 = ceilf(fmaxf(m, top));
            const float a = m1 == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m1);
            l *= a;
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
                acc[c] *= a;
            m = m1;
        }
        const float shift = m == -INFINITY ? 0.0f : vl - m;  // whole (V scales are powers of two), so no rounding
        bf16x8 pf[4];
        float sum = 0.0f;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                sv[x][v] = __builtin_amdgcn_exp2f(fmaf(sv[x][v], ks, shift));    // probability times V scale
                sum += sv[x][v];
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
                pf[2 * x + u] = __builtin_bit_cast(
                    bf16x8, u32x4{pack_bf16x2_hw(sv[x][8 * u], sv[x][8 * u + 1]), pack_bf16x2_hw(sv[x][8 * u + 2], sv[x][8 * u + 3]),
                                  pack_bf16x2_hw(sv[x][8 * u + 4], sv[x][8 * u + 5]), pack_bf16x2_hw(sv[x][8 * u + 6], sv[x][8 * u + 7])});
        }
        l = fmaf(sum, low ? 0.0f : __builtin_amdgcn_exp2f(-vl), l);
        times_v<FMT, D>(acc, pf, tile + vrow, vchunk);
    }
    __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(0));              // copies in flight write this workgroup's LDS

    // ---- lane (col, hf) holds elements 32 c + 8 (v / 4) + 4 hf + v % 4 of its row
    l = across32(l, vsum);
    if (m_low != -INFINITY)                                 // (m followed these scores too: it is at most 2^6 behind)
        l += across32(l_low, vsum) * __builtin_amdgcn_exp2f(m_low - m);
    if (r >= rows)
        return;
    const int tr = r / A.G, hd = r - tr * A.G;
    const float inv = l == 0.0f ? 0.0f : (v_units != 0.0f ? V_UP : 1.0f) / l, down = v_units != 0.0f ? 1.0f : V_DOWN;
    if (A.direct) {
        uint16_t *dst = A.out + (int64_t(q.row0) + tr) * A.out_stride + (h * A.G + hd) * D + 4 * hf;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int v = 0; v < 16; v += 4)
                *reinterpret_cast<uint2 *>(dst + 32 * c + 2 * v) =
                    make_uint2(pack_bf16x2_hw(acc[c][v] * inv, acc[c][v + 1] * inv),
                               pack_bf16x2_hw(acc[c][v + 2] * inv, acc[c][v + 3] * inv));
        if (A.lse && hf == 0)
            A.lse[(int64_t(q.row0) + tr) * (A.c.H * A.G) + h * A.G + hd] = l == 0.0f ? INFINITY : m + log2f(l);
    } else {
        const int64_t part = part_index(A, unit.first + unit.split, h, r);
        if (hf == 0) {
            A.part_ml[2 * part] = l == 0.0f ? -INFINITY : m;
            A.part_ml[2 * part + 1] = l;
        }
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int v = 0; v < 16; v += 4)
                *reinterpret_cast<f32x4 *>(A.part_o + part * D + 32 * c + 2 * v + 4 * hf) =
                    f32x4{acc[c][v] * down, acc[c][v + 1] * down, acc[c][v + 2] * down, acc[c][v + 3] * down};
    }
}

// ---------------------------------------------------------------- finish
//
// Two (maximum, sum) pairs of a row as one.
__device__ __forceinline__ void join_pair(float &m, float &l, float m1, float l1)
{
    const float top = fmaxf(m, m1), ref = top == -INFINITY ? 0.0f : top;
    l = __builtin_amdgcn_exp2f(m - ref) * l + __builtin_amdgcn_exp2f(m1 - ref) * l1;
    m = top;
}

constexpr int MASS_BLOCKS = 16;              // blocks of a workgroup
constexpr int PIECE = 64;                    // elements of a workgroup that joins many units of one row
constexpr int WIDE_ROWS = 512;               // (row, head, sequence) triples from which rows stand side by side

// Workgroups [0, join) of a (head, sequence) join the units' results: with few
// rows, 64 elements of one packed row each, four a lane, the rest of the lanes
// over the units; with many (`wide`), whole rows side by side, four elements a
// lane, which walks the units (one sequence of 1000 tokens, 8 heads of 128, 100 rows
// with 8 heads each: 29.6 -> 21.7 us in all; 16 rows 18.1 -> 16.9).  Then, where the
// few-rows kernel left scores of cut sequences, one workgroup per MASS_BLOCKS
// blocks: lane = token, a wavefront's four blocks side by side.  Bound by
// latency for usual batches, so loads depend on as few others as possible: 4.4
// us for one sequence's 128 units, 20 us for the weights of 48 sequences of up
// to 16384 tokens (80 MB of scores and weights).
__global__ void __launch_bounds__(256) kv_finish_kernel(AttentionLaunch A, int join, bool wide)
{
    __shared__ __attribute__((aligned(16))) float part[1024];
    __shared__ float ml[2][8][32];
    const int i = blockIdx.z, h = blockIdx.y;
    const KvSeq q = kv_seq(A.s, i, A.s.all_rows);
    const int2 units = A.plan[i];
    const int rows = q.n * A.G, blocks = (q.len + KV_BLOCK - 1) / KV_BLOCK;
    const int first = __builtin_amdgcn_readfirstlane(units.x);
    const int n = blocks == 0 ? 0 : __builtin_amdgcn_readfirstlane(units.y);     // (no unit wrote the plan)
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    if (!q.ok && blockIdx.x == 0 && h == 0 && tid == 0)
        kv_raise(A.status, KV_BAD_LENGTH);           // (such a sequence has no units)
    if (int(blockIdx.x) < join && wide) {
        const int lanes = A.c.D / 4, r = int(blockIdx.x) * (256 / lanes) + tid / lanes, e = 4 * (tid % lanes);
        if (r >= rows)
            return;
        float m = -INFINITY, l = 0.0f;
        f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int u = 0; u < n; ++u) {
            const int64_t p = part_index(A, first + u, h, r);
            const float2 x = *reinterpret_cast<const float2 *>(A.part_ml + 2 * p);
            const f32x4 v = *reinterpret_cast<const f32x4 *>(A.part_o + p * A.c.D + e);
            const float top = fmaxf(m, x.x), ref = top == -INFINITY ? 0.0f : top;
            const float a = __builtin_amdgcn_exp2f(m - ref), b = __builtin_amdgcn_exp2f(x.x - ref);
            l = a * l + b * x.y;
            o = a * o + b * v;
            m = top;
        }
        const int tr = r / A.G, hd = r - tr * A.G;
        o *= l == 0.0f ? 0.0f : V_UP / l;
        *reinterpret_cast<uint2 *>(A.out + (int64_t(q.row0) + tr) * A.out_stride + (h * A.G + hd) * A.c.D + e) =
            make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
        if (A.lse && e == 0)
            A.lse[(int64_t(q.row0) + tr) * (A.c.H * A.G) + h * A.G + hd] = log_sum(m, l);
        return;
    }
    if (int(blockIdx.x) < join) {
        constexpr int LANES = PIECE / 4, GROUPS = 256 / LANES;
        const int pieces = A.c.D / PIECE, r = int(blockIdx.x) / pieces, e0 = PIECE * (int(blockIdx.x) % pieces);
        if (r >= rows)
            return;
        float m = -INFINITY, l = 0.0f;
        for (int s = lane; s < n; s += 64) {
            const float2 x = *reinterpret_cast<const float2 *>(A.part_ml + 2 * part_index(A, first + s, h, r));
            join_pair(m, l, x.x, x.y);
        }
        const float top = wave_max(m), ref = top == -INFINITY ? 0.0f : top;
        l = wave_sum(l * __builtin_amdgcn_exp2f(m - ref));
        const int g = tid / LANES, e = 4 * (tid % LANES);
        f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int s = g; s < n; s += GROUPS) {
            const int64_t p = part_index(A, first + s, h, r);
            o += __builtin_amdgcn_exp2f(A.part_ml[2 * p] - ref) * *reinterpret_cast<const f32x4 *>(A.part_o + p * A.c.D + e0 + e);
        }
        *reinterpret_cast<f32x4 *>(part + g * PIECE + e) = o;
        __syncthreads();
        const int tr = r / A.G, hd = r - tr * A.G;
        if (tid < PIECE) {
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < GROUPS; ++k)
                sum += part[k * PIECE + tid];
            A.out[(int64_t(q.row0) + tr) * A.out_stride + (h * A.G + hd) * A.c.D + e0 + tid] =
                f32_to_bf16(l == 0.0f ? 0.0f : sum / l * V_UP);
        }
        if (A.lse && tid == 0 && e0 == 0)
            A.lse[(int64_t(q.row0) + tr) * (A.c.H * A.G) + h * A.G + hd] = log_sum(top, l);
        return;
    }
    const int b0 = (int(blockIdx.x) - join) * MASS_BLOCKS;
    if (b0 >= blocks)
        return;
    const int from = max(q.n - A.mass_rows, 0) * A.G;
    constexpr int PER = MASS_BLOCKS / 4;
    int page[PER];
    float was[PER], w[PER];
    const float *src[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int b = b0 + wave + 4 * k;
        page[k] = b < blocks ? A.s.table[int64_t(i) * A.s.max_blocks + b] : -1;
        if (!kv_page_ok(page[k], A.c.n_pages))
            page[k] = -1;
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int b = b0 + wave + 4 * k;
        src[k] = A.scores + score_index(A, i, page[k] < 0 ? 0 : b, max(page[k], 0), h, 0) + lane;
        was[k] = w[k] = 0.0f;
        if (A.decay != 0.0f && page[k] >= 0 && b * KV_BLOCK + lane < q.len)
            was[k] = A.c.mass[(int64_t(page[k]) * A.c.H + h) * KV_BLOCK + lane];
    }
    // the rows' log-sums: eight threads a row (at most 32 rows) over the units, then joined in order
    {
        const int r = tid & 31, g = tid >> 5;
        float m = -INFINITY, l = 0.0f;
        if (r < rows)
            for (int u = g; u < n; u += 8) {
                const float2 x = *reinterpret_cast<const float2 *>(A.part_ml + 2 * part_index(A, first + u, h, r));
                join_pair(m, l, x.x, x.y);
            }
        ml[0][g][r] = m;
        ml[1][g][r] = l;
        __syncthreads();
        if (tid < 32) {
            for (int k = 1; k < 8; ++k)
                join_pair(m, l, ml[0][k][tid], ml[1][k][tid]);
            part[tid] = log_sum(m, l);
        }
    }
    __syncthreads();
#pragma unroll 4
    for (int r = from; r < rows; ++r) {
        const float z = part[r];
#pragma unroll
        for (int k = 0; k < PER; ++k)
            w[k] += __builtin_amdgcn_exp2f(src[k][r * KV_BLOCK] - z);
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int b = b0 + wave + 4 * k;
        if (page[k] >= 0 && b * KV_BLOCK + lane < q.len)
            A.c.mass[(int64_t(page[k]) * A.c.H + h) * KV_BLOCK + lane] =
                A.decay != 0.0f ? fmaf(A.decay, was[k], w[k]) : w[k];
    }
}

// For many rows the scores are computed again from K.  A wavefront keeps a
// block's K in registers (as bf16, with D = 256 as codes) and walks groups of
// 32 rows; the next group's queries are on their way during this one's products
// and exponentials (with D = 256 they would not fit the registers beside K: 438
// us with them, 375 without).  All of 2048 rows of two sequences of 4096 tokens, 8 query heads a head: 2
// heads of 256 384 us, 4 heads of 128 229.  Bound by latency with heads of 256, where
// a wavefront waits for its queries for 66 % of its time (one a SIMD; the vector
// unit issues 20 % of it, the matrix cores work 10 %); with 128 it waits 33 %, and
// another 36 % for its turn beside the second wavefront of its SIMD.  With `share` = 4 the four
// wavefronts of a workgroup have a block each and meet the same queries at about
// the same time (in L1); with 1 they share one block and take every fourth
// group, for calls with few blocks.
template <int FMT, int D>
__global__ void __launch_bounds__(256, 2) kv_mass_rows_kernel(AttentionLaunch A, int share)
{
    __shared__ float part[4][KV_BLOCK];
    constexpr bool RAW = D == 256;
    const int i = blockIdx.z, h = blockIdx.y;
    const KvSeq q = kv_seq(A.s, i, A.s.all_rows);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int b = int(blockIdx.x) * share + wave % share, group = wave / share, groups = 4 / share;
    if (int(blockIdx.x) * share * KV_BLOCK >= q.len)
        return;
    const int col = lane & 31, hf = lane >> 5;
    int page = b * KV_BLOCK < q.len ? A.s.table[int64_t(i) * A.s.max_blocks + b] : -1;
    page = __builtin_amdgcn_readfirstlane(kv_page_ok(page, A.c.n_pages) ? page : -1);
    const int rows = page < 0 ? 0 : q.n * A.G;
    // rows below `from` do not count, or do not see the block
    const int from = max(max(q.n - A.mass_rows, 0), b * KV_BLOCK - (q.len - q.n)) * A.G;
    f32x16 w[2];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int v = 0; v < 16; ++v)
            w[x][v] = 0.0f;
    int r0 = from + 32 * group;
    if (r0 < rows) {
        u32x4 codes[RAW ? 2 : 1][RAW ? D / 32 : 1];
        bf16x8 kf[RAW ? 1 : 2][RAW ? 1 : D / 16];
        const uint8_t *block = A.c.data + kv_offset(page, h, A.c.H, D) + col * D + 16 * hf;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int p = 0; p < D / 32; ++p) {
                const u32x4 c = *reinterpret_cast<const u32x4 *>(block + 32 * x * D + 32 * p);
                if constexpr (RAW) {
                    codes[x][p] = c;
                } else {
                    kf[x][2 * p] = codes_bf16<FMT>(c[0], c[1]);
                    kf[x][2 * p + 1] = codes_bf16<FMT>(c[2], c[3]);
                }
            }
        const float ks = A.c.scales[(int64_t(page) * A.c.H + h) * 2] * fabsf(A.scale_log2);
        auto log_sum_of = [&](int first) {
            const int rc = min(first + col, rows - 1), tr = rc / A.G;
            return A.lse[(int64_t(q.row0) + tr) * (A.c.H * A.G) + h * A.G + rc - tr * A.G];
        };
        bf16x8 qf[D / 16];
        load_q32<D>(qf, A, q, h, r0, rows);
        float z = log_sum_of(r0);
        for (; r0 < rows; r0 += 32 * groups) {
            f32x16 sv[2];
            if constexpr (RAW)
                load_q32<D>(qf, A, q, h, r0, rows);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    sv[x][v] = 0.0f;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    if constexpr (RAW)
                        sv[x] = mfma32(codes_bf16<FMT>(codes[x][c / 2][2 * (c % 2)], codes[x][c / 2][2 * (c % 2) + 1]), qf[c],
                                       sv[x]);
                    else
                        sv[x] = mfma32(kf[x][c], qf[c], sv[x]);
                }
            }
            const float z0 = z;
            const int next = min(r0 + 32 * groups, rows - 1);
            if constexpr (!RAW)
                load_q32<D>(qf, A, q, h, next, rows);
            z = log_sum_of(next);
            const int r = r0 + col, limit = r < rows ? row_limit(q, r / A.G) : 0;
            // (a row past the last one, or one that does not see the whole block)
            if (r0 + 32 > rows || row_limit(q, r0 / A.G) < (b + 1) * KV_BLOCK) {
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const float e = __builtin_amdgcn_exp2f(fmaf(sv[x][v], ks, -z0));
                        w[x][v] += b * KV_BLOCK + 32 * x + 8 * (v >> 2) + 4 * hf + (v & 3) < limit ? e : 0.0f;
                    }
            } else {
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        w[x][v] += __builtin_amdgcn_exp2f(fmaf(sv[x][v], ks, -z0));
            }
        }
    }
    // over the 32 columns: four steps within 16 lanes, then the other 16
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            float a = w[x][v];
            a += __uint_as_float(dpp_move<dpp::QUAD_1032>(__float_as_uint(a)));
            a += __uint_as_float(dpp_move<dpp::QUAD_2301>(__float_as_uint(a)));
            a += __uint_as_float(dpp_move<dpp::ROW_HALF_MIRROR>(__float_as_uint(a)));
            a += __uint_as_float(dpp_move<dpp::ROW_MIRROR>(__float_as_uint(a)));
            const auto s16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(a), false, false);
            a = __uint_as_float(s16[0]) + __uint_as_float(s16[1]);
            if (col == 0)
                part[wave][32 * x + 8 * (v >> 2) + 4 * hf + (v & 3)] = a;
        }
    __syncthreads();
    if (group == 0 && page >= 0 && b * KV_BLOCK + lane < q.len) {
        float sum = part[wave][lane];
        for (int g = 1; g < groups; ++g)
            sum += part[wave + g * share][lane];
        float *dst = A.c.mass + (int64_t(page) * A.c.H + h) * KV_BLOCK + lane;
        *dst = A.decay != 0.0f ? fmaf(A.decay, *dst, sum) : sum;
    }
}

template <typename F>
void with_shape(int fmt, int D, F f)
{
    auto by_d = [&](auto fm) {
        if (D == 64)
            f(fm, std::integral_constant<int, 64>{});
        else if (D == 128)
            f(fm, std::integral_constant<int, 128>{});
        else
            f(fm, std::integral_constant<int, 256>{});
    };
    if (fmt == KV_INT8)
        by_d(std::integral_constant<int, KV_INT8>{});
    else
        by_d(std::integral_constant<int, KV_E4M3>{});
}

size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

}  // namespace

// How a call is cut, by its host-side bounds alone: the same cut sizes the
// workspace and launches the kernels.
AttentionCut attention_cut(int S, int H, int G, int D, int n_pages, int max_rows, int max_len, bool mass)
{
    AttentionCut c{};
    const int64_t rows = int64_t(max_rows) * G;
    const int blocks = (max_len + KV_BLOCK - 1) / KV_BLOCK;
    c.few = rows <= 32;
    c.tile_rows = c.few ? (rows <= 16 ? 16 : 32) : 128;
    c.per = int((rows + c.tile_rows - 1) / c.tile_rows) * H;
    c.direct = blocks <= DIRECT_BLOCKS || int64_t(S) * c.per >= (c.few ? 8192 : 256);
    // sum of ceil(blocks_i / chunk) <= total / chunk + S, and total * per <= chunk * MOST_WORKGROUPS
    c.units = c.direct ? S : int(std::min<int64_t>(int64_t(S) * ((blocks + LEAST_BLOCKS - 1) / LEAST_BLOCKS),
                                                   MOST_WORKGROUPS / c.per + S));
    size_t off = c.direct ? 0 : up256(size_t(S) * sizeof(int2));     // the plan comes first
    c.part_ml = off;
    off += !c.direct ? up256(size_t(c.units) * H * rows * 2 * sizeof(float)) : 0;
    c.part_o = off;
    off += !c.direct ? up256(size_t(c.units) * H * rows * D * sizeof(float)) : 0;
    c.scores = off;
    c.score_blocks = int64_t(S) * blocks <= n_pages ? blocks : 0;
    if (mass && c.few)
        off += up256(size_t(c.score_blocks ? int64_t(S) * blocks : n_pages) * H * rows * KV_BLOCK * sizeof(float));
    c.bytes = off;                              // (the log-sums of many rows follow: they go by n_rows)
    return c;
}

hipError_t launch_kv_rest(const KvSeqs &s, uint16_t *out, int64_t out_stride, int width, hipStream_t st)
{
    launch_k(kv_rest_kernel, unsigned(rest_groups(s)), 256, 0, st, s, out, out_stride, width);
    return hipGetLastError();
}

hipError_t launch_kv_attention(AttentionLaunch A, int fmt, const AttentionCut &c, hipStream_t st)
{
    const int H = A.c.H, S = A.s.S;
    const int rows = A.s.max_rows * A.G;
    A.main = c.units * c.per;
    const unsigned grid = unsigned(A.main + rest_groups(A.s));
    hipError_t e = hipSuccess;
    auto launch = [&](auto f, auto d, auto all) {
        constexpr int FMT = decltype(f)::value, D = decltype(d)::value;
        constexpr bool ALL = decltype(all)::value;
        if (!c.few) {
            static std::atomic<uint64_t> done{0};
            e = allow_lds_once(reinterpret_cast<const void *>(kv_many_rows_kernel<FMT, D, ALL>), ManyRows<D>::LDS, done);
            if (e == hipSuccess)
                launch_k(kv_many_rows_kernel<FMT, D, ALL>, grid, 256, ManyRows<D>::LDS, st, A);
        } else if (c.tile_rows == 16)
            launch_k(kv_few_rows_kernel<FMT, D, 1, ALL>, grid, 256, 0, st, A);
        else
            launch_k(kv_few_rows_kernel<FMT, D, 2, ALL>, grid, 256, 0, st, A);
    };
    with_shape(fmt, A.c.D, [&](auto f, auto d) {
        if (A.s.all_rows)
            launch(f, d, std::true_type{});
        else
            launch(f, d, std::false_type{});
    });
    if (e == hipSuccess)
        e = hipGetLastError();
    const int blocks = (A.s.max_len + KV_BLOCK - 1) / KV_BLOCK;
    const bool wide = int64_t(rows) * H * S >= WIDE_ROWS;
    const int side = 1024 / A.c.D;                          // rows side by side
    const int join = c.direct ? 0 : wide ? (rows + side - 1) / side : rows * (A.c.D / PIECE);
    const int groups = A.mass_rows && c.few && !c.direct ? (blocks + MASS_BLOCKS - 1) / MASS_BLOCKS : 0;
    if (e == hipSuccess && join + groups) {
        launch_k(kv_finish_kernel, dim3(join + groups, H, S), 256, 0, st, A, join, wide);
        e = hipGetLastError();
    }
    if (e == hipSuccess && A.mass_rows && !c.few && blocks) {
        const int share = int64_t(blocks) * H * S >= 4 * 256 ? 4 : 1;
        with_shape(fmt, A.c.D, [&](auto f, auto d) {
            launch_k(kv_mass_rows_kernel<decltype(f)::value, decltype(d)::value>, dim3((blocks + share - 1) / share, H, S),
                     256, 0, st, A, share);
        });
        e = hipGetLastError();
    }
    return e;
}

}  // namespace msi
