// kv_common.h -- the paged 8-bit cache of keys and values: what its kernels
// and the host agree on.  Plain C++ apart from the qualifiers, so that the
// bounds checks and the scale rule are tested on the host.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define MSI_HD __host__ __device__ __forceinline__
#else
#define MSI_HD inline
#endif

namespace msi {

constexpr int KV_BLOCK = 64;                // tokens of a page
constexpr int KV_E4M3 = 0, KV_INT8 = 1;

// bits of the status word
constexpr uint32_t KV_BAD_PAGE = 1u;        // a page index outside the pool
constexpr uint32_t KV_NONFINITE = 2u;       // an appended key or value is infinite or NaN
constexpr uint32_t KV_BAD_LENGTH = 4u;      // a length or row range outside its bounds

struct KvCache {
    uint8_t *data;                          // [n_pages, H, 2, 64, D] codes
    float *scales;                          // [n_pages, H, 2]
    float *mass;                            // [n_pages, H, 64], or null
    int n_pages, H, D;
};

struct KvSeqs {
    const int32_t *table;                   // [S, max_blocks]
    const int32_t *lens;                    // [S]
    const int32_t *cu;                      // [S + 1]
    int S, max_blocks, n_rows, max_rows, max_len;
    bool all_rows;                          // attention: a sequence has no more rows than tokens, other rows become zeros
};

// One sequence of a call: its rows [row0, row0 + n), its tokens [0, len).
struct KvSeq {
    int row0, n, len;
    bool ok;
};

// The sequence if its numbers keep every access inside the caller's arrays,
// ok = false otherwise.  cached: every row is one of the sequence's tokens.
MSI_HD KvSeq kv_check_seq(int row0, int row1, int len, int n_rows, int max_rows, int max_len, bool cached)
{
    KvSeq s{row0, 0, len, true};
    s.ok = len >= 0 && len <= max_len && row0 >= 0 && row0 <= n_rows && row1 >= row0 && row1 <= n_rows;
    if (s.ok) {
        s.n = row1 - row0;                   // (of values in [0, n_rows]: no overflow)
        s.ok = s.n <= max_rows && (!cached || s.n <= len);
    }
    if (!s.ok)
        s.n = s.len = 0;
    return s;
}

MSI_HD bool kv_page_ok(int page, int n_pages) { return page >= 0 && page < n_pages; }

// First byte of the codes of a page and head; K first, then V (64 D bytes each).
MSI_HD int64_t kv_offset(int64_t page, int head, int H, int D) { return (page * H + head) * (2 * KV_BLOCK) * int64_t(D); }

// Scale of a block whose largest magnitude has the bits `amax` (finite): the
// least power of two s >= 2^-64 with amax <= s Q, Q = 448 = 1.75 2^8 (e4m3) or
// 127 = 1.984375 2^6 (int8).  With a power of two, x / s is exact, and a block
// whose scale grows moves its e4m3 codes without a second rounding.
MSI_HD uint32_t kv_scale_bits(uint32_t amax, int fmt)
{
    const int e = int(amax >> 23);           // biased; 0 for zero and subnormals
    const uint32_t m = amax & 0x7FFFFFu;
    const int k = fmt == KV_INT8 ? e - 6 + (m > 0x7E0000u) : e - 8 + (m > 0x600000u);
    return uint32_t(k > 127 - 64 ? k : 127 - 64) << 23;
}

}  // namespace msi
