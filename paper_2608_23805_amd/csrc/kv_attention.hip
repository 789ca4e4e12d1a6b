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
#include <type_traits>

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

// Rows 64 group .., 64 (group + groups) .. and so on; seq(i): sequence i; `words`: 8 words of LDS.
template <typename Seq>
__device__ __forceinline__ void clear_rest(const KvSeqs &s, Seq seq, uint16_t *__restrict__ out, int64_t stride, int width,
                                           int group, int groups, uint32_t *words)
{
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    for (int64_t first = int64_t(group) * REST_ROWS; first < s.n_rows; first += int64_t(groups) * REST_ROWS) {
        const int r0 = int(first), n = min(REST_ROWS, s.n_rows - r0);
        uint64_t rows = 0;
        for (int i = threadIdx.x; i < s.S; i += 256) {
            const KvSeq q = seq(i);
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

__device__ __forceinline__ void clear_rest(const KvSeqs &s, uint16_t *__restrict__ out, int64_t stride, int width, int group,
                                           int groups, uint32_t *words)
{
    auto seq = [&](int i) {
        return kv_check_seq(s.cu[i], s.cu[i + 1], s.lens[i], s.n_rows, s.max_rows, s.max_len, true);
    };
    clear_rest(s, seq, out, stride, width, group, groups, words);
}

__global__ void __launch_bounds__(256) kv_rest_kernel(KvSeqs s, uint16_t *out, int64_t stride, int width)
{
    __shared__ uint32_t words[8];
    clear_rest(s, out, stride, width, int(blockIdx.x), int(gridDim.x), words);
}

// ---------------------------------------------------------------- forms
//
// What a kernel of units is compiled for: PLAIN; ALL, which clears other rows;
// SHARED, whose units come from a list of owners (see below) and always leave
// partial results.
enum Form : int { PLAIN, ALL, SHARED };

template <int FORM>
using LaunchOf = std::conditional_t<FORM == SHARED, SharedLaunch, AttentionLaunch>;

// ---------------------------------------------------------------- shared pages
//
// Batches whose sequences hold the same first pages.  The rows of a group are
// neighbours, so on its shared pages the group is one sequence whose rows see
// every token: those pages are read once for all of them.  Every sequence's
// rows meet its other pages as usual, and a row's result is joined from the
// units of both.  The owners of units are the groups, then the sequences.  Where
// a group's numbers break a bound, or its pages reach past a sequence's first
// row, or offsets of groups fall, the pages count as each sequence's own: what
// comes out is the same.  A group's pages are read through the table of the first
// sequence that stands behind them; where none does, nobody reads them.
//
// With up to 64 groups and 64 sequences, one a lane, every wavefront of the first
// launch lays the owners out by itself (its first workgroup leaves them for the
// kernels behind it); larger batches take a launch of one workgroup (4 answers
// from a prompt of 192 tokens: 22.6 us with it, 12.8 without; 64 rows of 32768 shared
// tokens: 105.7 and 94).
constexpr int PLAN_THREADS = 1024;
constexpr int NO_SEQ = 0x7fffffff;

// Group with the sequences [a, z) and `blocks` shared blocks, whose rows are [row0, row1); ok: its offsets are in order.
__device__ __forceinline__ KvOwner group_owner(const SharedLaunch &A, int a, int z, int blocks, int row0, int row1, bool &ok)
{
    KvOwner o{};
    o.group = -1;
    o.all = 1;
    if (!ok || a == z)
        return o;
    ok = blocks >= 0 && blocks <= A.g.max_blocks && row0 >= 0 && row1 >= row0 && row1 <= A.s.n_rows && row1 - row0 <= A.g.max_rows;
    if (ok && blocks <= A.g.usable) {                       // (more blocks than any sequence has: their table entries are nobody's)
        o.row0 = row0, o.n = row1 - row0, o.seq = NO_SEQ;       // (its sequences say who is the first)
        o.len = blocks * KV_BLOCK, o.blocks = blocks;
        o.tiles = tiles_of(o.n, A.G, A.cut.tile_p);
    }
    return o;
}

// Sequence i, which may belong to group g (-1: to none) with the rows [row0, row0 + n) and `blocks` shared blocks.
__device__ __forceinline__ KvOwner seq_owner(const SharedLaunch &A, const KvSeq &q, int i, int g, int row0, int n, int blocks)
{
    KvOwner o{};
    o.row0 = q.row0, o.n = q.n, o.len = q.len, o.seq = i;
    o.group = -1;
    if (q.n && g >= 0 && blocks && q.len - q.n >= blocks * KV_BLOCK && q.row0 >= row0 && q.row0 + q.n <= row0 + n)
        o.group = g, o.b0 = blocks;
    if (q.n) {
        o.blocks = (q.len + KV_BLOCK - 1) / KV_BLOCK - o.b0;
        o.tiles = tiles_of(q.n, A.G, A.cut.tile_s);
    }
    return o;
}

// Blocks of a 128-row unit for up to 64 owners, one a lane (blocks, row tiles):
// the card holds `fill` workgroups at once, and rounds of them last as long as
// a unit and what a workgroup costs besides (about four blocks).  Lane l tries the
// largest owner in l + 1 pieces.
__device__ __forceinline__ int balanced_chunk(int blocks, int tiles, int H, int owners, int fill, int least)
{
    const int lane = threadIdx.x & 63;
    const int most = int(wave_max(float(tiles ? blocks : 0)));
    const int c = max(int(unsigned(most + lane) / unsigned(lane + 1)), least);
    int64_t n = 0;
    for (int o = 0; o < owners; ++o)
        n += int64_t(unsigned(__builtin_amdgcn_readlane(blocks, o) + c - 1) / unsigned(c)) * __builtin_amdgcn_readlane(tiles, o);
    const float cost = float((n * H + fill - 1) >> log2_of(fill)) * float(c + 4);
    const float best = -wave_max(-cost);
    return __builtin_amdgcn_readlane(c, __ffsll((unsigned long long)__ballot(cost == best)) - 1);
}

// Owners of a small batch: group and sequence `lane`, and the first item of each.
struct WavePlan {
    KvOwner g, s;
    int first_g, first_s, items_g, items;    // first items; items of all groups, of all owners
};

__device__ __forceinline__ WavePlan plan_wave(const SharedLaunch &A, uint32_t &status)
{
    const int lane = threadIdx.x & 63, H = A.c.H, G = A.G;
    const SharedCut &cut = A.cut;
    WavePlan p;
    int a = 0, z = 0, b = 0, c0 = 0, c1 = 0, len = 0;
    if (lane < A.g.n)
        a = A.g.cu[lane], z = A.g.cu[lane + 1], b = A.g.blocks[lane];
    if (lane < A.s.S)
        c0 = A.s.cu[lane], c1 = A.s.cu[lane + 1], len = A.s.lens[lane];
    bool ok = a >= 0 && a <= z && z <= A.s.S;
    status = 0;
    const bool none = __ballot(!ok) != 0;                   // (offsets out of order: groups could overlap)
    const int row0 = __shfl(c0, a & 63), row1 = __shfl(c1, (z - 1) & 63);
    if (lane < A.g.n && !none) {
        p.g = group_owner(A, a, z, b, row0, row1, ok);
    } else {
        p.g = KvOwner{};
        p.g.group = -1, p.g.all = 1;
    }
    if (!ok || none)
        status = KV_BAD_LENGTH;
    KvSeq q{0, 0, 0, true};
    if (lane < A.s.S)
        q = kv_check_seq(c0, c1, len, A.s.n_rows, A.s.max_rows, A.s.max_len, A.s.all_rows);
    if (!q.ok)
        status = KV_BAD_LENGTH;
    int mine = -1, g_row0 = 0, g_n = 0, g_blocks = 0;
    for (int g = 0; g < A.g.n && !none; ++g) {
        const bool in = lane >= __builtin_amdgcn_readlane(a, g) && lane < __builtin_amdgcn_readlane(z, g);
        mine = in ? g : mine;
        g_row0 = in ? __builtin_amdgcn_readlane(p.g.row0, g) : g_row0;
        g_n = in ? __builtin_amdgcn_readlane(p.g.n, g) : g_n;
        g_blocks = in ? __builtin_amdgcn_readlane(p.g.blocks, g) : g_blocks;
    }
    p.s = seq_owner(A, q, lane, mine, g_row0, g_n, g_blocks);
    // the first sequence from `a` on that shares pages, if it is one of the group's
    const uint64_t behind = __ballot(p.s.group >= 0) >> (a & 63);
    if (p.g.seq == NO_SEQ) {
        p.g.seq = behind ? a + __ffsll((unsigned long long)behind) - 1 : z;
        if (p.g.seq >= z)
            p.g.n = p.g.blocks = p.g.tiles = 0;
    }
    // (small batches' sums are under 2^30)
    const int work_p = __builtin_amdgcn_readlane(wave_scan_incl(p.g.blocks * p.g.tiles * H), 63);
    const int work_s = __builtin_amdgcn_readlane(wave_scan_incl(p.s.blocks * p.s.tiles * H), 63);
    const int total_p = cut.both ? work_p + work_s : work_p, total_s = cut.both ? work_p + work_s : work_s;
    int chunk_p = shared_chunk(total_p, cut.few_p, cut.most_p), chunk_s = shared_chunk(total_s, cut.few_s, cut.most_s);
    const int fill = A.c.D == 256 ? 256 : 512;
    if (!cut.few_p && cut.items_p)
        chunk_p = balanced_chunk(p.g.blocks, p.g.tiles, H, A.g.n, fill, chunk_p);
    if (!cut.few_s)
        chunk_s = balanced_chunk(p.s.blocks, p.s.tiles, H, A.s.S, fill, chunk_s);
    auto place = [&](KvOwner &o, int chunk, int64_t before, int most, int &first, int &items, int &rows) {
        o.units = o.n ? int(unsigned(o.blocks + chunk - 1) / unsigned(chunk)) : 0;
        const int64_t n = int64_t(o.units) * o.tiles, r = int64_t(o.units) * o.n * G * H;
        // (more than the bounds: only offsets of rows that fall bring that; held down, sums stay in 32 bits)
        const int n1 = int(min(n, int64_t(most) + 1)), r1 = int(min(r, cut.parts + 1));
        const int ni = wave_scan_incl(n1), ri = wave_scan_incl(r1);
        items = __builtin_amdgcn_readlane(ni, 63), rows = __builtin_amdgcn_readlane(ri, 63);
        first = ni - n1;
        o.part = before + ri - r1;
        if (n && (ni > most || before + ri > cut.parts)) {
            o.n = o.units = 0;
            status = KV_BAD_LENGTH;
        }
    };
    int rows_g, rows_s, items_s;
    place(p.g, chunk_p, 0, cut.items_p, p.first_g, p.items_g, rows_g);
    // (of one launch for both, the sequences have what the groups leave, left-out ones among them)
    place(p.s, chunk_s, rows_g, cut.both ? max(cut.items_p + cut.items_s - p.items_g, 0) : cut.items_s, p.first_s, items_s, rows_s);
    p.first_s += p.items_g;
    p.items = p.items_g + items_s;
    if (__ballot(p.g.blocks && p.g.tiles && p.g.units == 0)) {     // a group was left out: so are its sequences
        const int whole = __shfl(p.g.units, max(p.s.group, 0));
        if (p.s.group >= 0 && whole == 0)
            p.s.n = p.s.units = 0;
    }
    return p;
}

// One workgroup's share of a SHARED launch: a row tile and head of a unit.
struct SharedItem {
    KvSeq q;                                 // the owner's rows and tokens
    int seq, h, tile, b0, b1;                // table, head, row tile, blocks
    int64_t part;                            // partial result of its packed row 0
    bool all, ok;
};

// The last of n ascending numbers that is at most `at` (the first is): 64 ways at a time.
__device__ __forceinline__ int last_at_most(const int32_t *first, int n, int at)
{
    const int lane = threadIdx.x & 63;
    int base = 0;
    while (n > 1) {
        const int run = (n + 63) >> 6, i = lane * run;
        const int hit = __popcll(__ballot(i < n && first[base + min(i, n - 1)] <= at)) - 1;
        base += hit * run;
        n = min(run, n - hit * run);
    }
    return base;
}

__device__ __forceinline__ SharedItem find_item(const SharedLaunch &A)
{
    SharedItem it{};
    const int n = A.g.n + A.s.S, H = A.c.H;
    it.h = int(blockIdx.x) % H;
    int at = int(blockIdx.x) / H, start;
    KvOwner w;
    if (A.cut.small && A.list != 1) {
        uint32_t status;
        const WavePlan p = plan_wave(A, status);
        if (blockIdx.x == 0 && threadIdx.x < 64) {          // for the kernels behind this one
            const int lane = threadIdx.x;
            kv_raise(A.status, status);
            if (lane < A.g.n) {
                A.owners[lane] = p.g;
                A.first[lane] = p.first_g;
            }
            if (lane < A.s.S) {
                A.owners[A.g.n + lane] = p.s;
                A.first[A.g.n + lane] = p.first_s;
            }
            if (lane == 0)
                A.first[n] = p.items;
        }
        const bool shared = at < p.items_g;
        if (at >= (A.list == 0 ? p.items_g : p.items))
            return it;
        // (owners without items have their neighbour's first one: the last lane that starts at or before `at`)
        const int l = 63 - __clzll((unsigned long long)__ballot(shared ? p.first_g <= at && (threadIdx.x & 63) < A.g.n
                                                                       : p.first_s <= at && (threadIdx.x & 63) < A.s.S));
        auto field = [&](int g, int s) { return __builtin_amdgcn_readlane(shared ? g : s, l); };
        w.row0 = field(p.g.row0, p.s.row0), w.n = field(p.g.n, p.s.n), w.len = field(p.g.len, p.s.len);
        w.seq = field(p.g.seq, p.s.seq), w.b0 = field(p.g.b0, p.s.b0), w.blocks = field(p.g.blocks, p.s.blocks);
        w.units = field(p.g.units, p.s.units), w.tiles = field(p.g.tiles, p.s.tiles), w.all = field(p.g.all, p.s.all);
        w.part = field(int(p.g.part), int(p.s.part));       // (under SMALL_PARTS)
        start = field(p.first_g, p.first_s);
    } else {
        at += A.list == 1 ? A.first[A.g.n] : 0;
        if (at >= A.first[A.list == 0 ? A.g.n : n])
            return it;
        const int o = __builtin_amdgcn_readfirstlane(last_at_most(A.first, n, at));
        w = A.owners[o];
        start = A.first[o];
    }
    const unsigned local = at - start, tiles = max(w.tiles, 1), units = max(w.units, 1);
    const int unit = int(local / tiles);
    it.ok = w.units > 0;
    it.q = KvSeq{w.row0, w.n, w.len, true};
    it.seq = w.seq;
    it.tile = int(local - unsigned(unit) * tiles);
    const int each = int(unsigned(w.blocks) / units), more = w.blocks - each * int(units);   // the first units have one more
    it.b0 = w.b0 + unit * each + min(unit, more);
    it.b1 = it.b0 + each + (unit < more);
    it.part = w.part + (int64_t(unit) * H + it.h) * (int64_t(w.n) * A.G);
    it.all = w.all != 0;
    return it;
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

template <int FMT, int D, int RT, int FORM>
__global__ void __launch_bounds__(256, D * RT >= 512 ? 1 : 2) kv_few_rows_kernel(LaunchOf<FORM> A)
{
    using F = FewRows<FMT, D, RT>;
    constexpr int TOK = F::TOK, GT = F::GT, W = F::W, VW = F::VW, OS = F::OS;
    __shared__ __attribute__((aligned(16))) float olds[4][16][OS];
    __shared__ float ml[4][RT][16][2];
    __shared__ float lsum[16 * RT];
    constexpr bool QLDS = D == 256 && RT == 2;               // two tiles of long queries do not fit the registers
    __shared__ bf16x8 qlds[QLDS ? RT * (D / 32) * 64 : 1];

    if constexpr (FORM == ALL)
        if (int(blockIdx.x) >= A.main) {
            clear_rest(A.s, A.out, A.out_stride, A.c.H * A.G * D, int(blockIdx.x) - A.main, int(gridDim.x) - A.main,
                       reinterpret_cast<uint32_t *>(lsum));
            return;
        }
    int i, h, tile, b0, b1;
    KvSeq q;
    [[maybe_unused]] Unit unit{};
    [[maybe_unused]] SharedItem item{};
    if constexpr (FORM == SHARED) {
        item = find_item(A);
        if (!item.ok)
            return;
        i = item.seq, h = item.h, tile = item.tile, q = item.q, b0 = item.b0, b1 = item.b1;
    } else {
        unit = find_unit(A, int(blockIdx.x) / A.per);
        if (unit.seq < 0)
            return;
        const int sub = int(blockIdx.x) % A.per;
        i = unit.seq, h = sub % A.c.H, tile = sub / A.c.H;
        q = kv_seq(A.s, i, A.s.all_rows);
        if (!q.ok && sub == 0 && threadIdx.x == 0)
            kv_raise(A.status, KV_BAD_LENGTH);
        if (A.plan && unit.split == 0 && sub == 0 && threadIdx.x == 0)
            A.plan[i] = make_int2(unit.first, unit.n);
        const int2 range = unit_blocks(unit, (q.len + KV_BLOCK - 1) / KV_BLOCK);
        b0 = range.x, b1 = range.y;
    }
    const bool sees_all = FORM == SHARED && item.all;          // (shared pages come before every row)
    const int rows = q.n * A.G, r0 = tile * 16 * RT;
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
    const bool weighs = FORM != SHARED && A.direct && A.scores;
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
        limit[x] = r >= rows ? 0 : sees_all ? q.len : row_limit(q, tr);
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
            const bool masked = !here || t0 + TOK > (sees_all ? q.len : q.len - q.n + 1) || r0 + 16 * (x + 1) > rows;
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
            if (FORM != SHARED && A.scores && r0 + 16 * x + col < rows) {
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
            const int64_t part = FORM == SHARED ? item.part + r : part_index(A, unit.first + unit.split, h, r);
            const bool direct = FORM != SHARED && A.direct;
            if ((tid & 15) == 0 && !direct) {
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
                if (direct) {
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
// a ring of two or three LDS buffers (half the LDS traffic of bf16 tiles, which would
// bound 32-row wavefronts) and become bf16 on their way from LDS to
// v_mfma_f32_32x32x16_bf16.  With D = 256 the 32 rows' outputs alone take 128
// registers, so the queries lie in LDS as well, in the order of their fragments; that keeps
// everything in the vector registers, where the rescaling needs the outputs (in
// the accumulation registers every block would move all of them there and back:
// 753 us for 640).  4096 rows on top of 4096 tokens, two sequences, 16 query heads
// of 256: 890 us, 926 TFLOP/s; 32 of 128: 795 us, 1038 TFLOP/s.  Neither unit is
// full: a block's conversions, products and exponentials follow one another in a
// wavefront, and one (heads of 256) or two a SIMD overlap little of them (2048 rows
// of 8 sequences on 16384 shared tokens, heads of 128: vector unit 52 % of the time,
// matrix cores 34 %; 240 rows, heads of 256: 26 and 18).  More wavefronts convert
// more: with heads of 256 and eight of 16 rows, two a SIMD, every wavefront converts
// the whole block, 928 us for 890.
//
// int8 codes take the vector unit twice as long as e4m3 to convert.  The four
// wavefronts convert a quarter of a block each and leave it in LDS as the fragments
// in bf16 that all of them then read; with heads of 256 LDS has room for those of V
// (two sequences of 4096 tokens: the last 2048 rows, 32 query heads of 128 237 us for
// 263, of 64 148 for 185; the last 1024 rows, 16 of 256 198 for 220.  64 rows of 32768
// shared tokens 88 for 95).  For e4m3 those reads take longer than the conversions
// (8 questions of 256 rows on 16384 shared tokens 414 us for 391, two sequences of
// 2041 and 3815 rows with heads of 256 700 for 663).
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
    static constexpr int ROWS = 128;
    static constexpr int BLOCK = 2 * KV_BLOCK * D;        // bytes of a block's codes
    static constexpr int COPIES = BLOCK / 4096;           // copy instructions of a wavefront and block
    static constexpr int CPR = D / 16;                    // chunks of a row
    static constexpr bool QLDS = D == 256;
    static constexpr int QBYTES = QLDS ? ROWS * D * 2 : 0;
};

// What a workgroup converts once (K, V: each wavefront a quarter of a block), and its LDS: codes, queries, fragments.
template <int FMT, int D>
struct ManyForm {
    static constexpr bool K = FMT == KV_INT8 && D <= 128, V = FMT == KV_INT8;
    static constexpr int NBUF = V && !K ? 2 : 3, AHEAD = NBUF - 1;
    static constexpr int QUERIES = NBUF * ManyRows<D>::BLOCK, FRAGS = QUERIES + ManyRows<D>::QBYTES;
    static constexpr size_t LDS = FRAGS + (int(K) + int(V)) * ManyRows<D>::BLOCK;
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

// Copies of a later block into `later`, and this wavefront's quarter of the block at `tile` as bf16 fragments: K's (if they
// are shared) 4 p + 2 e + b as scores32 reads them, then V's (D / 32) u + c as times_v does, 1024 bytes each, lane by lane.
template <int FMT, int D>
__device__ __forceinline__ void copy_and_convert(bf16x8 *__restrict__ frags, const uint8_t *__restrict__ tile,
                                                 uint8_t *__restrict__ later, const CopyLane<D> &cl, const uint8_t *block, int valid,
                                                 int wave, uint32_t vrow, uint32_t vswz)
{
    cl.copy(later, block, valid);
    const int lane = threadIdx.x & 63;
    const int t = lane & 31, swz = many_swz<D>(t), hf = lane >> 5, vc = (lane >> 4) & 1;
    constexpr bool K = ManyForm<FMT, D>::K;
#pragma unroll
    for (int i = 0; i < (K ? D / 64 : 0); ++i) {             // (row block b, chunk pair p: both halves e of its chunk)
        const int at = wave * (D / 64) + i, p = at >> 1, b = at & 1;
        const u32x4 w = *reinterpret_cast<const u32x4 *>(tile + (32 * b + t) * D + (((2 * p + hf) ^ swz) << 4));
        frags[(4 * p + b) * 64 + lane] = codes_bf16<FMT>(w[0], w[1]);
        frags[(4 * p + 2 + b) * 64 + lane] = codes_bf16<FMT>(w[2], w[3]);
    }
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {                       // V's token rows 16 wave ..
        const i32x2 w = read_tr8(tile + vrow + 16 * wave * D + (((2 * c + vc) ^ vswz) << 4));
        frags[((K ? D / 8 : 0) + wave * (D / 32) + c) * 64 + lane] = codes_bf16<FMT>(uint32_t(w[0]), uint32_t(w[1]));
    }
}

template <int D, typename Query>
__device__ __forceinline__ void score_frags(f32x16 (&sv)[2], const bf16x8 *__restrict__ frags, Query query)
{
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v)
            sv[b][v] = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int b = 0; b < 2; ++b)
            sv[b] = mfma32(frags[(2 * c + b) * 64], query(c), sv[b]);
}

template <int D>
__device__ __forceinline__ void frags_times_v(f32x16 (&acc)[D / 32], const bf16x8 (&pf)[4], const bf16x8 *__restrict__ frags)
{
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
            acc[c] = mfma32(frags[(u * (D / 32) + c) * 64], pf[u], acc[c]);
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

template <int FMT, int D, int FORM>
__global__ void __launch_bounds__(256, 2) kv_many_rows_kernel(LaunchOf<FORM> A)
{
    using M = ManyRows<D>;
    using F = ManyForm<FMT, D>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds8[];
    if constexpr (FORM == ALL)
        if (int(blockIdx.x) >= A.main) {
            clear_rest(A.s, A.out, A.out_stride, A.c.H * A.G * D, int(blockIdx.x) - A.main, int(gridDim.x) - A.main,
                       reinterpret_cast<uint32_t *>(lds8));
            return;
        }
    int i, h, r0;
    int2 range;
    KvSeq q;
    [[maybe_unused]] Unit unit{};
    [[maybe_unused]] SharedItem item{};
    if constexpr (FORM == SHARED) {
        item = find_item(A);
        if (!item.ok)
            return;
        i = item.seq, h = item.h, r0 = item.tile * M::ROWS, q = item.q, range = make_int2(item.b0, item.b1);
    } else {
        unit = find_unit(A, int(blockIdx.x) / A.per);
        if (unit.seq < 0)
            return;
        // the last row tiles, which see the most tokens, start first
        const int sub = A.per - 1 - int(blockIdx.x) % A.per;
        i = unit.seq, h = sub % A.c.H, r0 = sub / A.c.H * M::ROWS;
        q = kv_seq(A.s, i, A.s.all_rows);
        if (!q.ok && sub == 0 && threadIdx.x == 0)
            kv_raise(A.status, KV_BAD_LENGTH);
        if (A.plan && unit.split == 0 && sub == 0 && threadIdx.x == 0)
            A.plan[i] = make_int2(unit.first, unit.n);
        range = unit_blocks(unit, (q.len + KV_BLOCK - 1) / KV_BLOCK);
    }
    const bool sees_all = FORM == SHARED && item.all;       // (shared pages come before every row)
    const int rows = q.n * A.G;
    if (r0 >= rows)
        return;
    auto limit_of = [&](int row) { return sees_all ? q.len : row_limit(q, row); };
    // blocks up to the last row's limit
    const int last = min(r0 + M::ROWS, rows) - 1;
    const int most = max(limit_of(last / A.G), 0);
    const int b0 = range.x, b1 = min(range.y, (most + KV_BLOCK - 1) / KV_BLOCK);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hf = lane >> 5;
    const int w0 = r0 + 32 * wave;                          // this wavefront's rows
    const bool idle = w0 >= rows;
    const int r = w0 + col;
    const int limit = r < rows ? limit_of(r / A.G) : 0;
    const int least = idle ? 0 : limit_of(w0 / A.G);        // the first row's limit: blocks below it need no mask
    const int wave_most = idle ? 0 : limit_of(min(w0 + 31, rows - 1) / A.G);

    bf16x8 qf[D / 16];
    bf16x8 *const ql = reinterpret_cast<bf16x8 *>(lds8 + F::QUERIES) + wave * (D / 16) * 64 + lane;
    load_q32<D>(qf, A, q, h, w0, rows);
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
    int next_pages = -1, next_at = b0;                      // pages of the copies, which run ahead of the list
    int list_at = b0 - 64, pages = -1;
    float kscale = 0.0f, vlog = 0.0f, v_units = 0.0f;
    uint64_t lows = 0;
    const float factor = fabsf(A.scale_log2);
    auto fetch_list = [&](int b) {                           // (the copies' list has come to the same blocks)
        float2 sc{0.0f, 1.0f};
        if (b + lane < b1) {
            if (next_pages < 0)
                kv_raise(A.status, KV_BAD_PAGE);
            else
                sc = *reinterpret_cast<const float2 *>(A.c.scales + (int64_t(next_pages) * A.c.H + h) * 2);
        }
        return sc;
    };
    auto make_list = [&](int b, float2 sc) {
        list_at = b;
        pages = next_pages;
        kscale = fmaxf(sc.x * factor, 1e-37f);               // (not 0: times -infinity that would be NaN)
        vlog = log2f(fmaxf(sc.y, NO_SCALE));                 // whole for powers of two
        if (v_units == 0.0f && __any(vlog > LARGE_V_LOG)) {
            v_units = V_LOG;
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
                acc[c] *= V_DOWN;
        }
        lows = __ballot(v_units != 0.0f && vlog < LOW_V_LOG);
        vlog -= v_units;
    };
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
        cl.copy(lds8 + (b - b0) % F::NBUF * M::BLOCK, block, valid_at(b));
    };
    auto arrive = [&](auto waitn) {
        __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(decltype(waitn)::value));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wavefront's reads are done with
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    issue(b0);
    if constexpr (F::AHEAD > 1)
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
    bf16x8 *const frags = reinterpret_cast<bf16x8 *>(lds8 + F::FRAGS);

    for (int b = b0; b < b1; ++b) {
        // block b has landed (b + 1 is in flight); the buffer of block b - 1 is free
        arrive(std::integral_constant<int, M::COPIES * (F::AHEAD - 1)>{});
        if (b - list_at == 64)
            make_list(b, fetch_list(b));
        const int t0 = b * KV_BLOCK;
        const uint8_t *block = block_at(b + F::AHEAD);
        const int valid = valid_at(b + F::AHEAD);
        const uint8_t *const tile = lds8 + (b - b0) % F::NBUF * M::BLOCK;
        uint8_t *const later = lds8 + (b + F::AHEAD - b0) % F::NBUF * M::BLOCK;
        f32x16 sv[2];
        if constexpr (F::V) {
            copy_and_convert<FMT, D>(frags, tile, later, cl, block, valid, wave, vrow, uint32_t(vswz));
            if constexpr (!F::K)
                if (t0 < wave_most)
                    scores32<FMT, D>(sv, tile, query);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();                   // the block is there in bf16
            asm volatile("" ::: "memory");
            if (t0 >= wave_most)                            // (as is every later block)
                continue;
            if constexpr (F::K)
                score_frags<D>(sv, frags + lane, query);
        } else {
            if (t0 >= wave_most) {
                cl.copy(later, block, valid);
                continue;
            }
            copy_and_score<FMT, D>(sv, tile, query, later, cl, block, valid);
        }
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
        if constexpr (F::V)
            frags_times_v<D>(acc, pf, frags + (F::K ? D / 8 * 64 : 0) + lane);
        else
            times_v<FMT, D>(acc, pf, tile + vrow, vchunk);
    }
    __builtin_amdgcn_s_waitcnt(VMCNT_WAIT(0));              // copies in flight write this workgroup's LDS

    // ---- lane (col, hf) holds elements 32 c + 8 (v / 4) + 4 hf + v % 4 of its row
    l = across32(l, vsum);
    if (m_low != -INFINITY)                                 // (m followed these scores too: it is at most 2^6 behind)
        l += across32(l_low, vsum) * __builtin_amdgcn_exp2f(m_low - m);
    const float inv = l == 0.0f ? 0.0f : (v_units != 0.0f ? V_UP : 1.0f) / l, down = v_units != 0.0f ? 1.0f : V_DOWN;
    if (FORM != SHARED && A.direct) {
        if (r >= rows)
            return;
        const int tr = r / A.G, hd = r - tr * A.G;
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
        const int64_t part = FORM == SHARED ? item.part : part_index(A, unit.first + unit.split, h, 0);
        if (hf == 0 && r < rows) {
            A.part_ml[2 * (part + r)] = l == 0.0f ? -INFINITY : m;
            A.part_ml[2 * (part + r) + 1] = l;
        }
        // 32 elements of the wavefront's 32 rows at a time through LDS of its own, so that a store covers whole lines of
        // eight rows (lane by lane, 16 bytes of a row each, the way out of 128 rows of 256 takes 4.4 us)
        __syncthreads();                                    // (the blocks' buffers are no longer read)
        constexpr int LD = 36;
        float *const mine = reinterpret_cast<float *>(lds8) + wave * 32 * LD;
        const int r8 = lane >> 3, e8 = 4 * (lane & 7);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
#pragma unroll
            for (int v = 0; v < 16; v += 4)
                *reinterpret_cast<f32x4 *>(mine + col * LD + 2 * v + 4 * hf) =
                    f32x4{acc[c][v] * down, acc[c][v + 1] * down, acc[c][v + 2] * down, acc[c][v + 3] * down};
            // (a wavefront's LDS operations are in order; the fences keep the compiler from moving them)
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (w0 + 8 * k + r8 < rows)
                    *reinterpret_cast<f32x4 *>(A.part_o + (part + w0 + 8 * k + r8) * D + 32 * c + e8) =
                        *reinterpret_cast<const f32x4 *>(mine + (8 * k + r8) * LD + e8);
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
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

// The owners of larger batches: one workgroup lays them out, checks their numbers and cuts them.
__device__ __forceinline__ int64_t group_scan64(int64_t v, int64_t *part, int64_t &total)
{
    // inclusive sum over the workgroup's threads, and the total; `part`: a word a wavefront
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t x = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t u = __shfl_up(x, d);
        x += lane >= d ? u : 0;
    }
    if (lane == 63)
        part[wave] = x;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll 1
    for (int w = 0; w < PLAN_THREADS / 64; ++w) {
        before += w < wave ? part[w] : 0;
        total += part[w];
    }
    __syncthreads();
    return x + before;
}

__global__ void __launch_bounds__(PLAN_THREADS) kv_shared_plan_kernel(SharedLaunch A)
{
    __shared__ int64_t part[PLAN_THREADS / 64];
    __shared__ int falling, dropped, chunk;
    const int tid = threadIdx.x, H = A.c.H, G = A.G, N = A.g.n + A.s.S;
    const SharedCut &cut = A.cut;
    uint32_t status = 0;
    if (tid == 0)
        falling = dropped = 0;
    __syncthreads();
    // ---- the groups
    for (int g = tid; g < A.g.n; g += PLAN_THREADS) {
        const int a = A.g.cu[g], z = A.g.cu[g + 1];
        bool ok = a >= 0 && a <= z && z <= A.s.S;
        if (!ok)
            falling = 1;                                    // (offsets out of order: groups could overlap)
        const int row0 = ok ? A.s.cu[a] : 0, row1 = ok ? A.s.cu[z] : 0;
        const KvOwner o = group_owner(A, a, z, A.g.blocks[g], row0, row1, ok);
        if (!ok)
            status |= KV_BAD_LENGTH;
        A.owners[g] = o;
    }
    __syncthreads();                                        // (the sequences' threads read the groups)
    const bool none = falling != 0;
    // ---- the sequences
    int64_t work_s = 0;
    for (int i = tid; i < A.s.S; i += PLAN_THREADS) {
        const KvSeq q = kv_check_seq(A.s.cu[i], A.s.cu[i + 1], A.s.lens[i], A.s.n_rows, A.s.max_rows, A.s.max_len, A.s.all_rows);
        if (!q.ok)
            status |= KV_BAD_LENGTH;
        int lo = 0, hi = none ? 0 : A.g.n;                  // the group: the last that starts at or before i
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            (A.g.cu[mid] <= i ? lo : hi) = mid;
        }
        const bool in = hi > 0 && A.g.cu[lo] <= i && i < A.g.cu[lo + 1];
        const KvOwner *w = A.owners + (in ? lo : 0);
        const KvOwner o = in ? seq_owner(A, q, i, lo, w->row0, w->n, w->blocks) : seq_owner(A, q, i, -1, 0, 0, 0);
        work_s += int64_t(o.blocks) * o.tiles * H;
        A.owners[A.g.n + i] = o;
        const int left = __shfl_up(o.group, 1);             // (of a run of lanes, the first alone)
        if (o.group >= 0 && ((tid & 63) == 0 || left != o.group))
            __hip_atomic_fetch_min(&A.owners[o.group].seq, i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    __syncthreads();
    int64_t work_p = 0;
    for (int g = tid; g < A.g.n; g += PLAN_THREADS) {
        const int seq = __hip_atomic_load(&A.owners[g].seq, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        KvOwner o = A.owners[g];
        o.seq = seq;
        if (none || seq == NO_SEQ)
            o.n = o.blocks = o.tiles = 0;
        A.owners[g] = o;
        work_p += int64_t(o.blocks) * o.tiles * H;
    }
    int64_t total_p, total_s;
    group_scan64(work_p, part, total_p);
    group_scan64(work_s, part, total_s);
    if (cut.both)
        total_p = total_s = total_p + total_s;
    int chunk_p = shared_chunk(total_p, cut.few_p, cut.most_p);
    const int chunk_s = shared_chunk(total_s, cut.few_s, cut.most_s);
    if (!cut.few_p && A.g.n <= 64) {                        // (written before the sums' barriers)
        if (tid < 64) {
            const KvOwner *w = A.owners + min(tid, max(A.g.n - 1, 0));
            const int c = balanced_chunk(tid < A.g.n ? w->blocks : 0, tid < A.g.n ? w->tiles : 0, H, A.g.n, A.c.D == 256 ? 256 : 512, chunk_p);
            if (tid == 0)
                chunk = c;
        }
        __syncthreads();
        chunk_p = chunk;
    }
    // ---- units, items, places of the partial results
    int64_t items = 0, parts = 0, items_p = 0;
    for (int base = 0; base < N; base += PLAN_THREADS) {
        const int e = base + tid;
        const bool shared = e < A.g.n;
        KvOwner o{};
        if (e < N)
            o = A.owners[e];
        const int c = shared ? chunk_p : chunk_s;
        o.units = o.n ? (o.blocks + c - 1) / c : 0;
        const int64_t mine = int64_t(o.units) * o.tiles, rows = int64_t(o.units) * o.n * G * H;
        int64_t all_items, all_rows, group_items;
        const int64_t i1 = items + group_scan64(mine, part, all_items), p1 = parts + group_scan64(rows, part, all_rows);
        group_scan64(shared ? mine : 0, part, group_items); // of this step's groups
        items_p += group_items;
        if (e < N) {
            // (owners past the bounds: only offsets of rows that fall can bring them there)
            const int64_t most = shared ? cut.items_p : cut.both ? int64_t(cut.items_p) + cut.items_s : cut.items_s;
            if (mine && (p1 > cut.parts || i1 - (shared || cut.both ? 0 : items_p) > most)) {
                o.units = 0, o.n = 0;
                status |= KV_BAD_LENGTH;
                if (shared)
                    dropped = 1;
            }
            o.part = p1 - rows;
            A.owners[e] = o;
            A.first[e] = int(min(i1 - mine, int64_t(0x7fffffff)));
        }
        items += all_items, parts += all_rows;
    }
    kv_raise(A.status, status);
    if (tid == 0)
        A.first[N] = int(min(items, int64_t(0x7fffffff)));
    __syncthreads();
    if (dropped)                                            // sequences without their group are left out, too
        for (int i = tid; i < A.s.S; i += PLAN_THREADS) {
            KvOwner *o = A.owners + A.g.n + i;
            if (o->group >= 0 && A.owners[o->group].units == 0)
                o->n = o->units = 0;
        }
}

// Joins a row's partial results: `lanes` = D / 4 threads a (row, head), four
// elements each; `ways` such sets share a row's units, four sets or more side by
// side in a workgroup otherwise.  Units of the group first, then the sequence's
// own, always in the same order.  Behind the first `mine` workgroups of every
// sequence, those that clear rows (MSI_KV_ALL_ROWS).
__global__ void __launch_bounds__(256) kv_shared_finish_kernel(SharedLaunch A, int ways, int mine)
{
    __shared__ __attribute__((aligned(16))) float sums[1024];
    __shared__ float ml[2][16];
    __shared__ uint32_t words[8];
    const int D = A.c.D, H = A.c.H, G = A.G, Hq = H * G;
    if (int(blockIdx.x) >= mine) {
        auto seq = [&](int i) {
            const KvOwner o = A.owners[A.g.n + i];
            return KvSeq{o.row0, o.n, o.len, true};
        };
        const int each = int(gridDim.x) - mine;
        clear_rest(A.s, seq, A.out, A.out_stride, Hq * D, int(blockIdx.z) * each + int(blockIdx.x) - mine, each * A.s.S, words);
        return;
    }
    const KvOwner o = A.owners[A.g.n + int(blockIdx.z)];
    const int lanes = D / 4, sets = 256 / lanes, set = threadIdx.x / lanes, e = 4 * (threadIdx.x % lanes);
    const int per = sets / ways;                            // (row, head) pairs of a workgroup
    const int64_t at = int64_t(blockIdx.x) * per + set / ways;
    const int way = set % ways;
    if (int64_t(blockIdx.x) * per >= int64_t(o.n) * Hq)
        return;
    const bool in = at < int64_t(o.n) * Hq;
    const int tr = in ? int(at / Hq) : 0, a = in ? int(at % Hq) : 0, h = a / G, hd = a - h * G;
    float m = -INFINITY, l = 0.0f;
    f32x4 v{0.f, 0.f, 0.f, 0.f};
    auto join = [&](const KvOwner &w, int row, int u0) {
        const int64_t rows = int64_t(w.n) * G;
        const int64_t p0 = w.part + h * rows + int64_t(row) * G + hd;
#pragma unroll 4
        for (int u = u0; u < w.units; u += ways) {
            const int64_t p = p0 + u * (H * rows);
            const float2 x = *reinterpret_cast<const float2 *>(A.part_ml + 2 * p);
            const f32x4 y = *reinterpret_cast<const f32x4 *>(A.part_o + p * D + e);
            const float top = fmaxf(m, x.x), ref = top == -INFINITY ? 0.0f : top;
            const float f = __builtin_amdgcn_exp2f(m - ref), b = __builtin_amdgcn_exp2f(x.x - ref);
            l = f * l + b * x.y;
            v = f * v + b * y;
            m = top;
        }
    };
    int shift = 0;
    if (o.group >= 0) {
        const KvOwner w = A.owners[o.group];
        join(w, o.row0 - w.row0 + tr, way);
        shift = w.units % ways;
    }
    join(o, tr, (way + ways - shift) % ways);               // (the sets go on in turn)
    if (ways > 1) {                                         // the sets' results, in order
        if (e == 0) {
            ml[0][set] = m;
            ml[1][set] = l;
        }
        *reinterpret_cast<f32x4 *>(sums + set * D + e) = v;
        __syncthreads();
        if (way)
            return;
        for (int k = 1; k < ways; ++k) {
            const float m1 = ml[0][set + k], l1 = ml[1][set + k];
            const f32x4 y = *reinterpret_cast<const f32x4 *>(sums + (set + k) * D + e);
            const float top = fmaxf(m, m1), ref = top == -INFINITY ? 0.0f : top;
            const float f = __builtin_amdgcn_exp2f(m - ref), b = __builtin_amdgcn_exp2f(m1 - ref);
            l = f * l + b * l1;
            v = f * v + b * y;
            m = top;
        }
    }
    if (!in)
        return;
    v *= l == 0.0f ? 0.0f : V_UP / l;
    *reinterpret_cast<uint2 *>(A.out + (int64_t(o.row0) + tr) * A.out_stride + a * D + e) =
        make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
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

// The kernel of units for tiles of 16, 32 or 128 packed rows.
template <int FMT, int D, int FORM>
hipError_t launch_units(const LaunchOf<FORM> &A, int tile_rows, unsigned grid, hipStream_t st)
{
    if (tile_rows == 128) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_lds_once(reinterpret_cast<const void *>(kv_many_rows_kernel<FMT, D, FORM>), ManyForm<FMT, D>::LDS, done);
        if (e != hipSuccess)
            return e;
        launch_k(kv_many_rows_kernel<FMT, D, FORM>, grid, 256, ManyForm<FMT, D>::LDS, st, A);
    } else if (tile_rows == 16) {
        launch_k(kv_few_rows_kernel<FMT, D, 1, FORM>, grid, 256, 0, st, A);
    } else {
        launch_k(kv_few_rows_kernel<FMT, D, 2, FORM>, grid, 256, 0, st, A);
    }
    return hipGetLastError();
}

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
    with_shape(fmt, A.c.D, [&](auto f, auto d) {
        constexpr int FMT = decltype(f)::value, D = decltype(d)::value;
        if (A.s.all_rows)
            e = launch_units<FMT, D, ALL>(A, c.tile_rows, grid, st);
        else
            e = launch_units<FMT, D, PLAIN>(A, c.tile_rows, grid, st);
    });
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

hipError_t launch_kv_attention_shared(SharedLaunch A, int fmt, hipStream_t st)
{
    const SharedCut &c = A.cut;
    const int H = A.c.H, Hq = H * A.G;
    hipError_t e = hipSuccess;
    if (!c.small) {
        launch_k(kv_shared_plan_kernel, 1, PLAN_THREADS, 0, st, A);
        e = hipGetLastError();
    }
    auto units = [&](int list, int tile_rows, int64_t items) {
        A.list = list;
        if (e == hipSuccess && items)
            with_shape(fmt, A.c.D, [&](auto f, auto d) {
                e = launch_units<decltype(f)::value, decltype(d)::value, SHARED>(A, tile_rows, unsigned(items * H), st);
            });
    };
    const int64_t least = c.small ? 1 : 0;                  // (the first launch leaves the owners)
    if (c.both) {
        units(2, c.tile_p, std::max(least, int64_t(c.items_p) + c.items_s));
    } else {
        units(0, c.tile_p, std::max(least, int64_t(c.items_p)));
        units(1, c.tile_s, c.items_s);
    }
    if (e != hipSuccess)
        return e;
    // few (row, head) pairs: each shared by all sets of a workgroup, since a row may have many units
    const int sets = 1024 / A.c.D;
    const int ways = int64_t(A.s.n_rows) * Hq <= 8192 ? sets : 1;
    const int64_t pairs = int64_t(A.s.max_rows) * Hq, per = sets / ways;
    const int mine = int((pairs + per - 1) / per), rest = A.s.all_rows ? (rest_groups(A.s) + A.s.S - 1) / A.s.S : 0;
    launch_k(kv_shared_finish_kernel, dim3(unsigned(mine + rest), 1, unsigned(A.s.S)), 256, 0, st, A, ways, mine);
    return hipGetLastError();
}

}  // namespace msi
