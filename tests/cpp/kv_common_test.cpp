// Bounds checks and the scale rule of the paged cache, on the host.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "../../paper_2608_23805_amd/csrc/kv_common.h"

using namespace msi;

static int failures = 0;
#define CHECK(c)                                                     \
    do {                                                             \
        if (!(c)) {                                                  \
            std::printf("line %d: %s\n", __LINE__, #c);              \
            ++failures;                                              \
        }                                                            \
    } while (0)

static float as_float(uint32_t u)
{
    float f;
    std::memcpy(&f, &u, 4);
    return f;
}

int main()
{
    const int big = 0x7fffffff;
    // sequences
    CHECK(kv_check_seq(0, 5, 9, 5, 5, 64, true).ok);
    CHECK(kv_check_seq(3, 3, 0, 5, 5, 64, true).ok);              // no rows, no tokens
    CHECK(!kv_check_seq(0, 6, 9, 5, 9, 64, true).ok);             // rows past the call's
    CHECK(!kv_check_seq(0, 5, 9, 9, 4, 64, true).ok);             // more rows than the bound
    CHECK(!kv_check_seq(4, 3, 9, 9, 4, 64, true).ok);             // falling offsets
    CHECK(!kv_check_seq(-1, 3, 9, 9, 9, 64, true).ok);
    CHECK(!kv_check_seq(-big - 1, big, 9, 9, 9, 64, true).ok);    // (a difference that would overflow)
    CHECK(!kv_check_seq(0, 5, 4, 9, 9, 64, true).ok);             // rows that are not among the tokens
    CHECK(kv_check_seq(0, 5, 4, 9, 9, 64, false).ok);
    CHECK(!kv_check_seq(0, 1, 65, 9, 9, 64, true).ok);
    CHECK(!kv_check_seq(0, 1, -1, 9, 9, 64, true).ok);
    CHECK(!kv_check_seq(0, 1, big, 9, 9, 64, false).ok);
    const KvSeq bad = kv_check_seq(0, big, big, 9, 9, 64, false);
    CHECK(bad.n == 0 && bad.len == 0);
    // pages
    CHECK(kv_page_ok(0, 1) && kv_page_ok(6, 7) && !kv_page_ok(7, 7) && !kv_page_ok(-1, 7) && !kv_page_ok(big, 7));
    CHECK(kv_offset(100000, 7, 8, 256) == (int64_t(100000) * 8 + 7) * 128 * 256);     // past 32 bits
    // scales: the least power of two s >= 2^-64 with x <= s Q, by trying them
    for (int fmt = 0; fmt < 2; ++fmt) {
        const double q = fmt == KV_INT8 ? 127.0 : 448.0;
        for (uint32_t hi = 0; hi < 0x7F80u; ++hi)
            for (int d = -1; d <= 1; ++d) {
                const uint32_t u = (hi << 16) + uint32_t(d);
                if (u >= 0x7F800000u)
                    continue;
                const float x = as_float(u), s = as_float(kv_scale_bits(u, fmt));
                if (!(double(x) <= double(s) * q && (s == 0x1p-64f || double(x) > double(s) / 2 * q))) {
                    std::printf("fmt %d x %a scale %a\n", fmt, x, s);
                    return 1;
                }
                int e;
                CHECK(std::frexp(s, &e) == 0.5f && std::isnormal(s) && std::isnormal(1.0f / s));
            }
    }
    if (failures == 0)
        std::puts("ok");
    return failures != 0;
}
