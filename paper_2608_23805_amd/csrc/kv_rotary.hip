// kv_rotary.hip -- append to the paged 8-bit cache with queries and keys rotated
// by their positions on the way, gfx950.
//
// The pair i of the first `rot` elements of a head, (i, i + rot / 2) or (2 i,
// 2 i + 1), turns by the angle position[axis[i]] * freq[i]:
//     (a, b) -> (a cos - b sin, b cos + a sin),
// in fp32 from bf16, rounded once to bf16 (at most 2^-8 relative): queries leave
// like that, keys are coded from there as msi_kv_append codes them, so that a
// cache holds the same bytes whether its keys were rotated here or before.
//
// Every byte moves once.  Prompts are bound by HBM: 14108 tokens, 32 query heads
// and 8 of 128, 68 us, 4.7 TB/s (85 us with loads past the caches and one
// workgroup for 16 heads); single tokens by the launch and the chain of lengths,
// positions or pages, and scales: 64 of them 7.8 us.
//
// Angles are fixed-point turns: freq is the frequency's fraction of a turn in
// units of 2^-64, so the low 64 bits of position * freq are the angle with its
// whole turns already gone, off by at most 2^-34 turns at any 32-bit position
// (in fp32 a position of 2^20 would leave 2^-5 radians), and cutting what is left
// of a quarter turn to 32 bits costs another 2^-34.
#include <algorithm>
#include <type_traits>

#include "gemm_ring.h"
#include "kernels.h"
#include "kv_device.h"

namespace msi {

namespace {

// Sine and cosine of an angle of `turn` 2^-64 turns (two's complement).  The
// nearest quarter turn comes off exactly; what is left, 62 bits, is cut to units of
// 2^-34 turns, and |x| <= pi / 4 goes through the Taylor polynomials up to x^9 and
// x^10 (their next terms are under 2^-28), each rounded operation 2^-24 of its value.
__device__ __forceinline__ void turn_sincos(uint64_t turn, float &s, float &c)
{
    const uint32_t hi = uint32_t(turn >> 32), k = (hi + 0x20000000u) >> 30;            // quarter turns
    const uint32_t rest = (hi - (k << 30)) << 2 | uint32_t(turn) >> 30;
    const float x = float(int32_t(rest)) * 0x1.921fb6p-32f;            // 2 pi 2^-34
    const float z = x * x;
    float ps = 2.7557319224e-6f, pc = -2.7557319224e-7f;               // 1 / 9!, -1 / 10!
    ps = fmaf(ps, z, -1.9841269841e-4f), pc = fmaf(pc, z, 2.4801587302e-5f);
    ps = fmaf(ps, z, 8.3333333333e-3f), pc = fmaf(pc, z, -1.3888888889e-3f);
    ps = fmaf(ps, z, -1.6666666667e-1f), pc = fmaf(pc, z, 4.1666666667e-2f);
    pc = fmaf(pc, z, -0.5f);
    const float sx = fmaf(ps * z, x, x), cx = fmaf(pc, z, 1.0f);
    const float a = k & 1 ? cx : sx, b = k & 1 ? sx : cx;
    s = k & 2 ? -a : a;
    c = (k + 1) & 2 ? -b : b;
}

// position * freq without whole turns.
__device__ __forceinline__ uint64_t turns(int32_t position, uint64_t freq) { return uint64_t(int64_t(position)) * freq; }

// The 16 elements that a thread owns of a head's row: slot s is chunks s and
// s + rot / 16 of 8 elements (pairs of halves), or chunks 2 s and 2 s + 1; slots
// from rot / 16 on do not rotate and are two chunks side by side either way.
template <bool INTERLEAVED>
__device__ __forceinline__ int2 slot_chunks(int s, int rot)
{
    return INTERLEAVED || s >= rot / 16 ? make_int2(2 * s, 2 * s + 1) : make_int2(s, s + rot / 16);
}

// Sines and cosines of slot s's eight pairs for one row.
struct Angles {
    float s[8], c[8];
};

struct Frequencies {
    uint64_t f[8];
    int axis[8];
};

__device__ __forceinline__ Frequencies load_frequencies(const RotaryAppend &A, int s)
{
    Frequencies q;
    uint64_t axes = 0;
    if (A.axis)
        axes = *reinterpret_cast<const uint64_t *>(A.axis + 8 * s);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        q.f[e] = A.freq[8 * s + e];
        q.axis[e] = min(int(axes >> (8 * e) & 0xFF), A.n_axes - 1);
    }
    return q;
}

// The positions of a row.
struct Position {
    int32_t p[4];
};

__device__ __forceinline__ Position load_position(const RotaryAppend &A, int64_t row)
{
    Position r;
#pragma unroll
    for (int x = 0; x < 4; ++x)
        r.p[x] = x == 0 || x < A.n_axes ? A.positions[x * A.position_stride + row] : 0;
    return r;
}

__device__ __forceinline__ Angles angles_of(const Frequencies &q, const Position &r)
{
    Angles a;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int x = q.axis[e];
        const int32_t at = x == 0 ? r.p[0] : x == 1 ? r.p[1] : x == 2 ? r.p[2] : r.p[3];
        turn_sincos(turns(at, q.f[e]), a.s[e], a.c[e]);
    }
    return a;
}

template <bool INTERLEAVED>
__device__ __forceinline__ void rotate(u32x4 (&x)[2], const Angles &t)
{
    float a[8], b[8];
    unpack_bf16x8(x[0], a);
    unpack_bf16x8(x[1], b);
    float u[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        // pair e: its two elements
        const float p = INTERLEAVED ? (e < 4 ? a[2 * e] : b[2 * e - 8]) : a[e];
        const float q = INTERLEAVED ? (e < 4 ? a[2 * e + 1] : b[2 * e - 7]) : b[e];
        u[e] = fmaf(p, t.c[e], -(q * t.s[e]));
        v[e] = fmaf(q, t.c[e], p * t.s[e]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (INTERLEAVED) {
            x[0][i] = pack_bf16x2_hw(u[i], v[i]);
            x[1][i] = pack_bf16x2_hw(u[i + 4], v[i + 4]);
        } else {
            x[0][i] = pack_bf16x2_hw(u[2 * i], u[2 * i + 1]);
            x[1][i] = pack_bf16x2_hw(v[2 * i], v[2 * i + 1]);
        }
    }
}

// The queries of up to q_rows rows of a sequence and q_heads heads: threads over
// (slot, row, head), a row's angles computed once for all of a thread's heads,
// while the first heads are on their way.
template <int D, bool INTERLEAVED>
__device__ __forceinline__ void rotate_queries(const RotaryAppend &A, const KvSeq &q, int tile, int part)
{
    constexpr int SLOTS = D / 16, BATCH = 4;
    const int subs = A.q_tiles, first = tile * KV_BLOCK + part % subs * A.q_rows, group = part / subs;
    const int s = threadIdx.x % SLOTS, t = threadIdx.x / SLOTS, step = 256 / (SLOTS * A.q_rows);
    const int r = first + t % A.q_rows, h0 = group * A.q_heads + t / A.q_rows, h1 = min((group + 1) * A.q_heads, A.n_q_heads);
    const bool turn = s < A.rot / 16;
    if (r >= min(q.n, (tile + 1) * KV_BLOCK) || h0 >= h1 || (!turn && A.q == A.q_out))    // (in place: nothing to move)
        return;
    const int2 ch = slot_chunks<INTERLEAVED>(s, A.rot);
    const int64_t row = int64_t(q.row0) + r;
    const uint16_t *src = A.q + row * A.q_stride;
    uint16_t *dst = A.q_out + row * A.q_out_stride;
    u32x4 x[BATCH][2];
    auto load = [&](int h) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int hb = min(h + b * step, h1 - 1) * D;
            x[b][0] = *reinterpret_cast<const u32x4 *>(src + hb + 8 * ch.x);
            x[b][1] = *reinterpret_cast<const u32x4 *>(src + hb + 8 * ch.y);
        }
    };
    Angles a;
    if (turn) {
        const Position p = load_position(A, row);
        const Frequencies f = load_frequencies(A, s);
        load(h0);
        a = angles_of(f, p);
    } else {
        load(h0);
    }
    for (int h = h0;;) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            if (h + b * step >= h1)
                break;
            if (turn)
                rotate<INTERLEAVED>(x[b], a);
            uint16_t *to = dst + (h + b * step) * D;
            *reinterpret_cast<u32x4 *>(to + 8 * ch.x) = x[b][0];
            *reinterpret_cast<u32x4 *>(to + 8 * ch.y) = x[b][1];
        }
        h += BATCH * step;
        if (h >= h1)
            return;
        load(h);
    }
}

// Grid: (tiles of 64 rows, 2 H workgroups of keys and values then those of the
// queries' heads, sequences).  A workgroup of keys or values owns a block, head
// and K or V as msi_kv_append's do: its new rows stay in registers between the
// rotation, the largest magnitude and the codes; old rows of the block are
// touched only if its scale grows.
template <int FMT, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(256) kv_append_rotary_kernel(RotaryAppend A)
{
    constexpr int SLOTS = D / 16, ROWS = 256 / SLOTS, N = KV_BLOCK / ROWS;
    __shared__ float part[4];
    const KvCache &c = A.c;
    const int i = blockIdx.z;
    const KvSeq q = kv_seq(A.s, i, true);
    if (!q.ok && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0)
        kv_raise(A.status, KV_BAD_LENGTH);
    if (q.n == 0)
        return;
    if (int(blockIdx.y) >= 2 * c.H) {
        if (int(blockIdx.x) * KV_BLOCK < q.n)
            rotate_queries<D, INTERLEAVED>(A, q, int(blockIdx.x), int(blockIdx.y) - 2 * c.H);
        return;
    }
    const int h = blockIdx.y >> 1, j = blockIdx.y & 1;
    const int start = q.len - q.n;                         // position in the cache of the first new row
    const int blk = start / KV_BLOCK + int(blockIdx.x);
    if (blk * KV_BLOCK >= q.len)
        return;
    const int lo = max(start - blk * KV_BLOCK, 0), hi = min(q.len - blk * KV_BLOCK, KV_BLOCK);   // new rows of the block
    const int s = threadIdx.x % SLOTS, r0 = threadIdx.x / SLOTS;
    const bool turn = j == 0 && s < A.rot / 16;
    const int2 ch = j ? make_int2(2 * s, 2 * s + 1) : slot_chunks<INTERLEAVED>(s, A.rot);
    const int64_t src0 = int64_t(q.row0) + (blk * KV_BLOCK - start);       // call's row of the block's row 0
    const int64_t stride = j ? A.v_stride : A.k_stride;
    const uint16_t *src = (j ? A.v : A.k) + src0 * stride + h * D;
    // everything that does not depend on the page is on its way before it
    Frequencies f;
    Position pos[N];
    if (turn) {
        f = load_frequencies(A, s);
#pragma unroll
        for (int p = 0; p < N; ++p)
            pos[p] = load_position(A, src0 + min(max(r0 + p * ROWS, lo), hi - 1));
    }
    u32x4 x[N][2];
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const int r = r0 + p * ROWS;
        const bool in = r >= lo && r < hi;
        x[p][0] = in ? *reinterpret_cast<const u32x4 *>(src + r * stride + 8 * ch.x) : u32x4{0, 0, 0, 0};
        x[p][1] = in ? *reinterpret_cast<const u32x4 *>(src + r * stride + 8 * ch.y) : u32x4{0, 0, 0, 0};
    }
    const int page = __builtin_amdgcn_readfirstlane(A.s.table[int64_t(i) * A.s.max_blocks + blk]);
    if (!kv_page_ok(page, c.n_pages)) {
        if (threadIdx.x == 0)
            kv_raise(A.status, KV_BAD_PAGE);
        return;
    }
    float *sc = c.scales + (int64_t(page) * c.H + h) * 2 + j;
    const float was = lo ? *sc : 0.0f;                     // (read before the barrier below, written after)
    if (turn)
#pragma unroll
        for (int p = 0; p < N; ++p) {
            const int r = r0 + p * ROWS;
            if (r >= lo && r < hi)
                rotate<INTERLEAVED>(x[p], angles_of(f, pos[p]));
        }
    uint32_t flags = 0, m = 0;                             // largest finite magnitude: bf16 bits order as integers
#pragma unroll
    for (int p = 0; p < N; ++p)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t a = x[p][y][w] & 0x7FFFu, b = (x[p][y][w] >> 16) & 0x7FFFu;
                if (a >= 0x7F80u || b >= 0x7F80u)
                    flags = KV_NONFINITE;
                m = max(m, max(a >= 0x7F80u ? 0u : a, b >= 0x7F80u ? 0u : b));
            }
    kv_raise(A.status, flags);
    const float top = block_max256(__uint_as_float(m << 16), part);
    const float need = __uint_as_float(kv_scale_bits(__float_as_uint(top), FMT));
    const float scale = fmaxf(need, was), inv = 1.0f / scale;
    uint8_t *dst = c.data + kv_offset(page, h, c.H, D) + j * (KV_BLOCK * D);
    const int chunk[2] = {ch.x, ch.y};
    if (lo && scale != was) {                              // the old rows move to the larger scale
        for (int r = r0; r < lo; r += ROWS)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                uint2 *o = reinterpret_cast<uint2 *>(dst + r * D + 8 * chunk[y]);
                const uint2 w = *o;
                // (both products are exact unless a caller's own scale is no power of two)
                const f32x4 a = kv_unpack4<FMT>(w.x) * was * inv, b = kv_unpack4<FMT>(w.y) * was * inv;
                *o = make_uint2(kv_pack4<FMT>(a[0], a[1], a[2], a[3]), kv_pack4<FMT>(b[0], b[1], b[2], b[3]));
            }
    }
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const int r = r0 + p * ROWS;
        if (r >= lo && r < hi)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                float f[8];
                unpack_bf16x8(x[p][y], f);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    f[e] = f[e] != f[e] ? 0.0f : f[e] * inv;           // NaN is stored as zero, infinities as the largest code
                *reinterpret_cast<uint2 *>(dst + r * D + 8 * chunk[y]) =
                    make_uint2(kv_pack4<FMT>(f[0], f[1], f[2], f[3]), kv_pack4<FMT>(f[4], f[5], f[6], f[7]));
            }
    }
    if (threadIdx.x == 0)
        *sc = scale;
    if (j == 0 && c.mass && int(threadIdx.x) >= lo && int(threadIdx.x) < hi)
        c.mass[(int64_t(page) * c.H + h) * KV_BLOCK + threadIdx.x] = 0.0f;
}

}  // namespace

hipError_t launch_kv_append_rotary(RotaryAppend A, int fmt, bool interleaved, hipStream_t st)
{
    const int slots = A.c.D / 16;
    // rows of a workgroup: all that there may be, up to what leaves a thread a slot of one head
    A.q_rows = 1;
    while (A.q_rows < A.s.max_rows && A.q_rows * slots < 256 && A.q_rows < KV_BLOCK)
        A.q_rows *= 2;
    const int tiles = (A.s.max_rows + KV_BLOCK - 1) / KV_BLOCK;
    A.q_tiles = std::min(KV_BLOCK, A.s.max_rows + A.q_rows - 1) / A.q_rows;
    // heads of a workgroup: the side-by-side ones, then as many as still leave some thousand workgroups: more share a row's
    // angles, fewer have their loads in flight together (prompts of 14108 tokens, 32 heads, with the read of what was
    // appended: 136 us with 1 or 2, 85 with 4, 90 with 8, 105 with 16)
    const int side = 256 / (slots * A.q_rows);
    A.q_heads = std::max(side, int(std::min<int64_t>(A.n_q_heads, int64_t(A.n_q_heads) * tiles * A.q_tiles * A.s.S / 8192)));
    const int parts = A.q ? (A.n_q_heads + A.q_heads - 1) / A.q_heads * A.q_tiles : 0;
    const dim3 grid(std::min((A.s.max_rows + 2 * KV_BLOCK - 2) / KV_BLOCK, (A.s.max_len + KV_BLOCK - 1) / KV_BLOCK),
                    2 * A.c.H + parts, A.s.S);
    auto by_d = [&](auto f, auto i) {
        constexpr int FMT = decltype(f)::value;
        constexpr bool I = decltype(i)::value;
        if (A.c.D == 64)
            launch_k(kv_append_rotary_kernel<FMT, 64, I>, grid, 256, 0, st, A);
        else if (A.c.D == 128)
            launch_k(kv_append_rotary_kernel<FMT, 128, I>, grid, 256, 0, st, A);
        else
            launch_k(kv_append_rotary_kernel<FMT, 256, I>, grid, 256, 0, st, A);
    };
    auto by_style = [&](auto f) {
        if (interleaved)
            by_d(f, std::true_type{});
        else
            by_d(f, std::false_type{});
    };
    if (fmt == KV_INT8)
        by_style(std::integral_constant<int, KV_INT8>{});
    else
        by_style(std::integral_constant<int, KV_E4M3>{});
    return hipGetLastError();
}

}  // namespace msi
