// kv_cache.hip -- writing, reading and cutting back the paged 8-bit cache of
// keys and values, gfx950.
//
// A page holds 64 tokens of every head; (page, head) is K codes [64, D], then
// V codes [64, D], with one fp32 scale each: value = scale * code.  All three
// operators move each byte once and are bound by HBM (long calls) or by the
// launch (single tokens).
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "kv_device.h"

namespace msi {

namespace {

// Thread t of 256 owns the D / 8 chunks of 8 elements of a row in turn: chunk
// t % (D / 8) of rows t / (D / 8) + i * ROWS.  16 bytes of bf16, 8 of codes.
template <int D>
struct RowChunks {
    static constexpr int CPR = D / 8;             // chunks of a row
    static constexpr int ROWS = 256 / CPR;        // rows of one pass of the workgroup
    static constexpr int N = KV_BLOCK / ROWS;     // passes over a block
};

__device__ __forceinline__ void unpack_bf16x8(const u32x4 &w, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// ---------------------------------------------------------------- append
//
// One workgroup per (block, K or V, head, sequence) that receives rows.  Its new
// rows stay in registers between the two passes (largest magnitude, then
// codes); old rows of the block are touched only if its scale grows.  One token
// of 64 sequences 5.1 us (launch and the chain of lengths, pages, scale);
// prompts of 8 sequences, 14108 tokens of 8 heads of 128, 20 us, 87 MB at 4.4 TB/s
// (K and V by one workgroup: 5.7 and 21 us).
template <int FMT, int D>
__global__ void __launch_bounds__(256) kv_append_kernel(KvCache c, KvSeqs s, const uint16_t *__restrict__ k,
                                                        const uint16_t *__restrict__ v, int64_t k_stride,
                                                        int64_t v_stride, uint32_t *status)
{
    using R = RowChunks<D>;
    __shared__ float part[4];
    const int h = blockIdx.y >> 1, j = blockIdx.y & 1, i = blockIdx.z;
    const KvSeq q = kv_seq(s, i, true);
    if (!q.ok && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0)
        kv_raise(status, KV_BAD_LENGTH);
    const int start = q.len - q.n;                       // position of the first new row
    const int blk = start / KV_BLOCK + int(blockIdx.x);
    if (q.n == 0 || blk * KV_BLOCK >= q.len)
        return;
    const int lo = max(start - blk * KV_BLOCK, 0), hi = min(q.len - blk * KV_BLOCK, KV_BLOCK);   // new rows of the block
    const int chunk = threadIdx.x % R::CPR, r0 = threadIdx.x / R::CPR;
    const int64_t src0 = int64_t(q.row0) + (blk * KV_BLOCK - start);       // call's row of the block's row 0
    const uint16_t *src = (j ? v + src0 * v_stride : k + src0 * k_stride) + h * D + chunk * 8;
    const int64_t stride = j ? v_stride : k_stride;
    u32x4 x[R::N];
#pragma unroll
    for (int p = 0; p < R::N; ++p) {
        const int r = r0 + p * R::ROWS;
        x[p] = r >= lo && r < hi ? load_stream16(src + r * stride) : u32x4{0, 0, 0, 0};
    }
    const int page = __builtin_amdgcn_readfirstlane(s.table[int64_t(i) * s.max_blocks + blk]);
    if (!kv_page_ok(page, c.n_pages)) {
        if (threadIdx.x == 0)
            kv_raise(status, KV_BAD_PAGE);
        return;
    }
    float *sc = c.scales + (int64_t(page) * c.H + h) * 2 + j;
    const float was = lo ? *sc : 0.0f;                   // (read before the barrier below, written after)
    uint32_t flags = 0, m = 0;                           // largest finite magnitude: bf16 bits order as integers
#pragma unroll
    for (int p = 0; p < R::N; ++p)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t a = x[p][w] & 0x7FFFu, b = (x[p][w] >> 16) & 0x7FFFu;
            if (a >= 0x7F80u || b >= 0x7F80u)
                flags = KV_NONFINITE;
            m = max(m, max(a >= 0x7F80u ? 0u : a, b >= 0x7F80u ? 0u : b));
        }
    kv_raise(status, flags);
    const float top = block_max256(__uint_as_float(m << 16), part);
    const float need = __uint_as_float(kv_scale_bits(__float_as_uint(top), FMT));
    const float scale = fmaxf(need, was), inv = 1.0f / scale;
    uint8_t *dst = c.data + kv_offset(page, h, c.H, D) + j * (KV_BLOCK * D);
    if (lo && scale != was) {                            // the old rows move to the larger scale
        for (int r = r0; r < lo; r += R::ROWS) {
            uint2 *o = reinterpret_cast<uint2 *>(dst + r * D + chunk * 8);
            const uint2 w = *o;
            const f32x4 a = kv_unpack4<FMT>(w.x), b = kv_unpack4<FMT>(w.y);
            // (both products are exact unless a caller's own scale is no power of two)
            const f32x4 y = a * was * inv, z = b * was * inv;
            *o = make_uint2(kv_pack4<FMT>(y[0], y[1], y[2], y[3]), kv_pack4<FMT>(z[0], z[1], z[2], z[3]));
        }
    }
#pragma unroll
    for (int p = 0; p < R::N; ++p) {
        const int r = r0 + p * R::ROWS;
        if (r >= lo && r < hi) {
            float f[8];
            unpack_bf16x8(x[p], f);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                f[e] = f[e] != f[e] ? 0.0f : f[e] * inv;          // NaN is stored as zero, infinities as the largest code
            *reinterpret_cast<uint2 *>(dst + r * D + chunk * 8) =
                make_uint2(kv_pack4<FMT>(f[0], f[1], f[2], f[3]), kv_pack4<FMT>(f[4], f[5], f[6], f[7]));
        }
    }
    if (threadIdx.x == 0)
        *sc = scale;
    if (j == 0 && c.mass && int(threadIdx.x) >= lo && int(threadIdx.x) < hi)
        c.mass[(int64_t(page) * c.H + h) * KV_BLOCK + threadIdx.x] = 0.0f;
}

// ---------------------------------------------------------------- read
//
// The mirror of append: row r of a sequence is its token len - n + r.  Values
// leave as bf16: exact for scales that are powers of two, as append writes
// them (a code has at most 8 significant bits), rounded to nearest otherwise.
// The rows pass the caches by: a call's outputs are many times an L2 (the open
// blocks of 64 sequences 8.2 us, 10.4 without and with K and V by one workgroup;
// 16384 tokens of 2 heads of 256, 50 MB, 10.2 and 15.1 us).  (Codes are read again soon; past the caches append and the
// copies of an eviction take 8% more.)
template <int FMT, int D>
__global__ void __launch_bounds__(256) kv_read_kernel(KvCache c, KvSeqs s, uint16_t *__restrict__ k,
                                                      uint16_t *__restrict__ v, int64_t k_stride, int64_t v_stride,
                                                      uint32_t *status)
{
    using R = RowChunks<D>;
    const int h = blockIdx.y >> 1, j = blockIdx.y & 1, i = blockIdx.z;
    const KvSeq q = kv_seq(s, i, true);
    if (!q.ok && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0)
        kv_raise(status, KV_BAD_LENGTH);
    const int start = q.len - q.n;
    const int blk = start / KV_BLOCK + int(blockIdx.x);
    if (q.n == 0 || blk * KV_BLOCK >= q.len)
        return;
    const int page = __builtin_amdgcn_readfirstlane(s.table[int64_t(i) * s.max_blocks + blk]);
    const bool ok = kv_page_ok(page, c.n_pages);
    if (!ok && threadIdx.x == 0)
        kv_raise(status, KV_BAD_PAGE);
    const int lo = max(start - blk * KV_BLOCK, 0), hi = min(q.len - blk * KV_BLOCK, KV_BLOCK);
    const int chunk = threadIdx.x % R::CPR, r0 = threadIdx.x / R::CPR;
    const int64_t dst0 = int64_t(q.row0) + (blk * KV_BLOCK - start);
    uint16_t *dst = (j ? v + dst0 * v_stride : k + dst0 * k_stride) + h * D + chunk * 8;
    const int64_t stride = j ? v_stride : k_stride;
    const uint8_t *base = c.data + kv_offset(ok ? page : 0, h, c.H, D) + j * (KV_BLOCK * D) + chunk * 8;
    const float scale = ok ? c.scales[(int64_t(page) * c.H + h) * 2 + j] : 0.0f;
    uint2 w[R::N];
#pragma unroll
    for (int p = 0; p < R::N; ++p) {
        const int r = r0 + p * R::ROWS;
        w[p] = make_uint2(0, 0);                           // a bad page reads as zeros
        if (ok && r >= lo && r < hi)
            w[p] = *reinterpret_cast<const uint2 *>(base + r * D);
    }
#pragma unroll
    for (int p = 0; p < R::N; ++p) {
        const int r = r0 + p * R::ROWS;
        if (r >= lo && r < hi) {
            const f32x4 a = kv_unpack4<FMT>(w[p].x) * scale, b = kv_unpack4<FMT>(w[p].y) * scale;
            __builtin_nontemporal_store(u32x4{pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]),
                                              pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3])},
                                        reinterpret_cast<u32x4 *>(dst + r * stride));
        }
    }
}

// ---------------------------------------------------------------- evict
//
// Selection, one 1024-thread workgroup per (head, sequence): token t of the
// chunk sits in round t / 1024 of thread t % 1024, so a wavefront's round is 64
// consecutive tokens and reads one page's weights (256 bytes).  Every token has
// a 32-bit key that orders as its weight does; protected tokens have the
// largest key of all.  The key of the last kept token is found by three rounds
// of histograms over 11, 11 and 10 bits; equal keys are kept from the lowest
// index on, by a prefix count in index order.  Sequences of up to
// 1024 * ROUNDS tokens keep their keys in registers through all passes; longer
// ones read them again in chunks of that size.  Where there are fewer (head,
// sequence) pairs than CUs, several workgroups find the same key and each writes
// a share of the indices.  A CU's instructions bound it: 16384 of 65536 tokens
// take 36 us (weights 8, histograms 16, counts and indices 12; 43 us by one
// workgroup), 2048 of 16384 for 16 sequences of 8 heads 16 us.  Four copies of
// each bin halve the collisions of weights that are alike.  (Keys in LDS with
// rolled loops: 70 and 20 us; indices gathered in LDS first: 3 us more.)
constexpr int SELECT_THREADS = 1024, SELECT_WAVES = SELECT_THREADS / 64, BINS = 2048, COPIES = 4;

// Keys: larger weights have larger ones, -0 is +0; NaN and the tokens of a bad
// page are below every number, places past the last token below everything,
// and protected tokens above (+infinity is 0xFF800000, -infinity 0x007FFFFF).
constexpr uint32_t KEY_NONE = 0u, KEY_NAN = 1u, KEY_PROTECTED = 0xFFFFFFFEu;
__device__ __forceinline__ uint32_t mass_key(float m)
{
    const uint32_t u = __float_as_uint(m + 0.0f);          // (-0 + 0 is +0)
    return m != m ? KEY_NAN : u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}

// base plus the set bits of `mask` below this lane
__device__ __forceinline__ int lanes_below(uint64_t mask, int base)
{
    return int(__builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), uint32_t(base))));
}

template <int ROUNDS>
__global__ void __launch_bounds__(SELECT_THREADS) kv_select_kernel(KvCache c, KvSeqs s, int32_t *__restrict__ keep,
                                                                   int32_t *__restrict__ new_lens, int budget, int sinks,
                                                                   int recent, uint32_t *status)
{
    constexpr int CHUNK = SELECT_THREADS * ROUNDS, GROUP = 4;
    __shared__ __attribute__((aligned(16))) int hist[BINS * COPIES];
    __shared__ int counts[2][ROUNDS * SELECT_WAVES];
    __shared__ int part[2][SELECT_WAVES];
    __shared__ int found[2];
    const int h = blockIdx.x, i = blockIdx.y, share = blockIdx.z, shares = gridDim.z;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const KvSeq q = kv_seq(s, i, false);
    if (!q.ok) {                                           // left out: its new length and indices stay as they were
        if (tid == 0)
            kv_raise(status, KV_BAD_LENGTH);
        return;
    }
    const int len = q.len, kept = min(len, budget);
    int32_t *out = keep + (int64_t(i) * c.H + h) * budget;
    if (h == 0 && share == 0 && tid == 0)
        new_lens[i] = kept;
    for (int t = kept + share * SELECT_THREADS + tid; t < budget; t += shares * SELECT_THREADS)
        out[t] = -1;
    if (len <= budget) {
        for (int t = share * SELECT_THREADS + tid; t < len; t += shares * SELECT_THREADS)
            out[t] = t;
        return;
    }
    const int32_t *table = s.table + int64_t(i) * s.max_blocks;
    const int chunks = (len + CHUNK - 1) / CHUNK;
    static_assert(ROUNDS <= 64, "one page a lane");
    uint32_t key[ROUNDS];
    bool bad = false;
    auto load = [&](int base) {
        // the page of round l in lane l, then all the weights at once
        const int tl = base + lane * SELECT_THREADS + wave * 64;
        int page = -1;
        if (lane < ROUNDS && tl < len) {
            page = table[tl / KV_BLOCK];
            if (!kv_page_ok(page, c.n_pages)) {
                page = -1;
                bad = true;
            }
        }
        // byte offset of the page's weights, in two halves
        const uint64_t at = (uint64_t(max(page, 0)) * c.H + h) * (KV_BLOCK * sizeof(float));
        const int bad_pages = __ballot(page < 0 && lane < ROUNDS && tl < len) != 0;
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const uint32_t lo = __builtin_amdgcn_readlane(uint32_t(at), r), hi = __builtin_amdgcn_readlane(uint32_t(at >> 32), r);
            const uint8_t *w = reinterpret_cast<const uint8_t *>(c.mass) + (uint64_t(hi) << 32 | lo);
            key[r] = *reinterpret_cast<const uint32_t *>(w + 4u * uint32_t(lane));
        }
        const uint32_t free = uint32_t(len - recent - sinks);              // (sinks + recent <= budget < len)
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int t = base + r * SELECT_THREADS + tid;
            uint32_t k = mass_key(__uint_as_float(key[r]));
            if (bad_pages && __builtin_amdgcn_readlane(page, r) < 0)
                k = KEY_NAN;
            k = uint32_t(t - sinks) >= free ? KEY_PROTECTED : k;           // below sinks the difference wraps
            key[r] = t >= len ? KEY_NONE : k;
        }
    };

    // ---- the key of the last kept token, and how many equal ones are kept (len > budget: it is above KEY_NONE)
    uint32_t prefix = 0, mask = 0;
    int rest = budget;
    if (chunks == 1)
        load(0);
    {
        constexpr int SHIFT[3] = {21, 10, 0}, WIDTH[3] = {11, 11, 10};
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = SHIFT[pass];
            const uint32_t digits = (1u << WIDTH[pass]) - 1;
            for (int b = tid; b < BINS; b += SELECT_THREADS)
                *reinterpret_cast<int4 *>(hist + b * COPIES) = make_int4(0, 0, 0, 0);
            __syncthreads();
            for (int ch = 0; ch < chunks; ++ch) {
                if (chunks > 1)
                    load(ch * CHUNK);
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r)
                    if (((key[r] ^ prefix) & mask) == 0) {
                        const uint32_t d = (key[r] >> shift) & digits, d0 = __builtin_amdgcn_readfirstlane(d);
                        const uint64_t same = __ballot(d == d0), all = __ballot(true);
                        // one addition where every counted lane agrees (all weights zero, or equal)
                        if (same != all)
                            atomicAdd(&hist[d * COPIES + lane % COPIES], 1);
                        else if (lane == __ffsll((unsigned long long)all) - 1)
                            atomicAdd(&hist[d * COPIES], __popcll(all));
                    }
            }
            __syncthreads();
            // thread t owns bins b, b - 1 counted from the top: find the bin where the running count reaches `rest`
            const int b = BINS - 1 - 2 * tid;
            const int4 h1 = *reinterpret_cast<const int4 *>(hist + b * COPIES);
            const int4 h0 = *reinterpret_cast<const int4 *>(hist + (b - 1) * COPIES);
            const int n1 = h1.x + h1.y + h1.z + h1.w, n0 = h0.x + h0.y + h0.z + h0.w;
            const int incl = wave_scan_incl(n1 + n0);
            if (lane == 63)
                part[0][wave] = incl;
            __syncthreads();
            int before = incl - (n1 + n0);
            for (int w = 0; w < wave; ++w)
                before += part[0][w];
            if (before < rest && before + n1 + n0 >= rest) {
                const bool second = before + n1 < rest;
                found[0] = second ? b - 1 : b;
                found[1] = rest - before - (second ? n1 : 0);
            }
            __syncthreads();
            prefix |= uint32_t(found[0]) << shift;
            mask |= digits << shift;
            rest = found[1];                               // of the keys with this prefix, so many are kept
            __syncthreads();
        }
    }

    // ---- kept tokens in ascending order: counts of those kept for sure and of the equal ones by (round,
    // wavefront), their prefixes in index order; of the equal ones before a token, at most `rest` are kept
    constexpr int CELLS = ROUNDS * SELECT_WAVES;
    static_assert(CELLS <= SELECT_THREADS, "one prefix per thread");
    int done[2] = {0, 0};                                  // sure and equal tokens of earlier chunks
    for (int ch = 0; ch < chunks; ++ch) {
        if (chunks > 1)
            load(ch * CHUNK);
        int mine[2] = {0, 0};                              // this wavefront's counts of round l in lane l
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int ns = __popcll(__ballot(key[r] > prefix)), ne = __popcll(__ballot(key[r] == prefix));
            mine[0] = lane == r ? ns : mine[0];
            mine[1] = lane == r ? ne : mine[1];
        }
        if (lane < ROUNDS) {
            counts[0][lane * SELECT_WAVES + wave] = mine[0];
            counts[1][lane * SELECT_WAVES + wave] = mine[1];
        }
        __syncthreads();
        int v[2], incl[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            v[j] = tid < CELLS ? counts[j][tid] : 0;
            incl[j] = wave_scan_incl(v[j]);
            if (lane == 63)
                part[j][wave] = incl[j];
        }
        __syncthreads();
        int total[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            int before = done[j] + incl[j] - v[j];
            total[j] = 0;
            for (int w = 0; w < SELECT_WAVES; ++w) {
                before += w < wave ? part[j][w] : 0;
                total[j] += part[j][w];
            }
            if (tid < CELLS)
                counts[j][tid] = before;
        }
        __syncthreads();
        if (lane < ROUNDS) {
            mine[0] = counts[0][lane * SELECT_WAVES + wave];
            mine[1] = counts[1][lane * SELECT_WAVES + wave];
        }
#pragma unroll
        for (int g = 0; g < ROUNDS; g += GROUP)            // this workgroup's share of the rounds
            if (g / GROUP % shares == share)
#pragma unroll
                for (int r = g; r < g + GROUP; ++r) {
                    const int ne = lanes_below(__ballot(key[r] == prefix), __builtin_amdgcn_readlane(mine[1], r));
                    const int ns = lanes_below(__ballot(key[r] > prefix), __builtin_amdgcn_readlane(mine[0], r));
                    if (key[r] + uint32_t(ne < rest) > prefix)         // (no key is 2^32 - 1)
                        *reinterpret_cast<int32_t *>(reinterpret_cast<uint8_t *>(out) + 4u * uint32_t(ns + min(ne, rest))) =
                            ch * CHUNK + r * SELECT_THREADS + tid;
                }
        done[0] += total[0];
        done[1] += total[1];
        __syncthreads();
    }
    if (bad)
        kv_raise(status, KV_BAD_PAGE);
}

// The kept tokens, copied to their new pages: one workgroup per (new block,
// head, sequence) gathers 64 rows of K and V and codes them again under the
// block's own scale, as an append of their values to an empty page would.
// 16 x 2048 tokens of 8 heads of 128: 28 us, 134 MB at 4.8 TB/s.
template <int FMT, int D>
__global__ void __launch_bounds__(256) kv_compact_kernel(KvCache c, KvSeqs s, const int32_t *__restrict__ dst_table,
                                                         int dst_blocks, const int32_t *__restrict__ keep, int budget,
                                                         uint32_t *status)
{
    using R = RowChunks<D>;
    __shared__ float part[8];
    __shared__ int row_page[KV_BLOCK], row_slot[KV_BLOCK];
    const int b = blockIdx.x, h = blockIdx.y, i = blockIdx.z;
    const KvSeq q = kv_seq(s, i, false);
    const int n = min(KV_BLOCK, min(q.len, budget) - b * KV_BLOCK);
    if (n <= 0)
        return;
    const int to = __builtin_amdgcn_readfirstlane(dst_table[int64_t(i) * dst_blocks + b]);
    if (!kv_page_ok(to, c.n_pages)) {
        if (threadIdx.x == 0)
            kv_raise(status, KV_BAD_PAGE);
        return;
    }
    if (threadIdx.x < KV_BLOCK) {
        int page = -1, slot = 0;
        if (int(threadIdx.x) < n) {
            const int t = keep[(int64_t(i) * c.H + h) * budget + b * KV_BLOCK + threadIdx.x];
            page = s.table[int64_t(i) * s.max_blocks + t / KV_BLOCK];
            slot = t % KV_BLOCK;
            if (!kv_page_ok(page, c.n_pages)) {
                kv_raise(status, KV_BAD_PAGE);         // (selection skips the pages of a sequence within its budget)
                page = -1;
            }
        }
        row_page[threadIdx.x] = page;
        row_slot[threadIdx.x] = slot;
        if (int(threadIdx.x) < n)
            c.mass[(int64_t(to) * c.H + h) * KV_BLOCK + threadIdx.x] =
                page < 0 ? 0.0f : c.mass[(int64_t(page) * c.H + h) * KV_BLOCK + slot];
    }
    __syncthreads();
    const int chunk = threadIdx.x % R::CPR, r0 = threadIdx.x / R::CPR;
    uint2 w[2][R::N];
    float sc[2][R::N];
#pragma unroll
    for (int p = 0; p < R::N; ++p) {
        const int r = r0 + p * R::ROWS;
        const int page = row_page[r];
        const int64_t at = kv_offset(max(page, 0), h, c.H, D) + row_slot[r] * D + chunk * 8;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            w[j][p] = make_uint2(0, 0);
            sc[j][p] = 0.0f;
            if (page >= 0) {
                w[j][p] = *reinterpret_cast<const uint2 *>(c.data + at + j * (KV_BLOCK * D));
                sc[j][p] = c.scales[(int64_t(page) * c.H + h) * 2 + j];
            }
        }
    }
    float top[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        float m = 0.0f;
#pragma unroll
        for (int p = 0; p < R::N; ++p) {
            const f32x4 a = kv_unpack4<FMT>(w[j][p].x) * sc[j][p], d = kv_unpack4<FMT>(w[j][p].y) * sc[j][p];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                m = fmaxf(m, fmaxf(fabsf(a[e]), fabsf(d[e])));
        }
        top[j] = block_max256(m, part + 4 * j);
    }
    uint8_t *base = c.data + kv_offset(to, h, c.H, D);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float scale = __uint_as_float(kv_scale_bits(__float_as_uint(top[j]), FMT)), inv = 1.0f / scale;
#pragma unroll
        for (int p = 0; p < R::N; ++p) {
            const int r = r0 + p * R::ROWS;
            if (r < n) {
                const f32x4 a = kv_unpack4<FMT>(w[j][p].x) * sc[j][p] * inv, d = kv_unpack4<FMT>(w[j][p].y) * sc[j][p] * inv;
                *reinterpret_cast<uint2 *>(base + j * (KV_BLOCK * D) + r * D + chunk * 8) =
                    make_uint2(kv_pack4<FMT>(a[0], a[1], a[2], a[3]), kv_pack4<FMT>(d[0], d[1], d[2], d[3]));
            }
        }
        if (threadIdx.x == 0)
            c.scales[(int64_t(to) * c.H + h) * 2 + j] = scale;
    }
}

// Calls f with the format and head size as constants.
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

}  // namespace

hipError_t launch_kv_append(const KvCache &c, int fmt, const KvSeqs &s, const uint16_t *k, const uint16_t *v,
                            int64_t k_stride, int64_t v_stride, uint32_t *status, hipStream_t st)
{
    // n rows from any position touch at most (n + 126) / 64 blocks
    const dim3 grid((s.max_rows + 126) / KV_BLOCK, 2 * c.H, s.S);
    with_shape(fmt, c.D, [&](auto f, auto d) {
        launch_k(kv_append_kernel<decltype(f)::value, decltype(d)::value>, grid, 256, 0, st, c, s, k, v, k_stride,
                 v_stride, status);
    });
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvCache &c, int fmt, const KvSeqs &s, uint16_t *k, uint16_t *v, int64_t k_stride,
                          int64_t v_stride, uint32_t *status, hipStream_t st)
{
    const dim3 grid((s.max_rows + 126) / KV_BLOCK, 2 * c.H, s.S);
    with_shape(fmt, c.D, [&](auto f, auto d) {
        launch_k(kv_read_kernel<decltype(f)::value, decltype(d)::value>, grid, 256, 0, st, c, s, k, v, k_stride,
                 v_stride, status);
    });
    return hipGetLastError();
}

hipError_t launch_kv_evict(const KvCache &c, int fmt, const KvSeqs &s, const int32_t *dst_table, int dst_blocks,
                           int32_t *new_lens, int32_t *keep, int budget, int sinks, int recent, uint32_t *status,
                           hipStream_t st)
{
    const int rounds = s.max_len <= 4 * SELECT_THREADS ? 4 : s.max_len <= 16 * SELECT_THREADS ? 16 : 64;
    const dim3 grid(c.H, s.S, std::max(1, std::min(rounds / 4, 256 / (c.H * s.S))));
    if (s.max_len <= 4 * SELECT_THREADS)
        launch_k(kv_select_kernel<4>, grid, SELECT_THREADS, 0, st, c, s, keep, new_lens, budget, sinks, recent, status);
    else if (s.max_len <= 16 * SELECT_THREADS)
        launch_k(kv_select_kernel<16>, grid, SELECT_THREADS, 0, st, c, s, keep, new_lens, budget, sinks, recent, status);
    else
        launch_k(kv_select_kernel<64>, grid, SELECT_THREADS, 0, st, c, s, keep, new_lens, budget, sinks, recent, status);
    hipError_t e = hipGetLastError();
    const int blocks = (std::min(budget, s.max_len) + KV_BLOCK - 1) / KV_BLOCK;
    if (e != hipSuccess || blocks == 0)
        return e;
    with_shape(fmt, c.D, [&](auto f, auto d) {
        launch_k(kv_compact_kernel<decltype(f)::value, decltype(d)::value>, dim3(blocks, c.H, s.S), 256, 0, st, c, s,
                 dst_table, dst_blocks, static_cast<const int32_t *>(keep), budget, status);
    });
    return hipGetLastError();
}

}  // namespace msi
