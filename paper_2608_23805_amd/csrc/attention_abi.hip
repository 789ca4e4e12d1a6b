// attention_abi.hip -- C ABI of the attention block's operators (declared in
// include/msi.h): checks of the arguments, then the launches.
#include <algorithm>
#include <cmath>

#include "../../include/msi.h"
#include "kernels.h"

using namespace msi;

namespace {

msi_status bad(const char *text) { return abi_error(MSI_E_INVALID_ARG, text); }

msi_status launched(hipError_t e) { return e == hipSuccess ? MSI_OK : abi_error(MSI_E_DEVICE, hipGetErrorString(e)); }

bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

constexpr uint64_t MOST_STRIDE = 1u << 21;      // elements: tile offsets stay under 2^31 bytes
constexpr uint32_t MOST = 1u << 29;              // rows, tokens, features: grids of 64 of them stay under 2^32 threads
constexpr uint64_t MOST_OUTPUTS = uint64_t(1) << 36;
constexpr uint32_t MOST_PAGES = 1u << 30;
constexpr uint64_t MOST_GROUPS = 1u << 24;       // workgroups of 256 along a grid's x

// Cache and sequences as the kernels take them; nullptr if the call may go on, else what is wrong.
const char *view_cache(const msi_kv_cache *c, KvCache &out)
{
    if (!c)
        return "null cache";
    if (c->format != MSI_KV_E4M3 && c->format != MSI_KV_INT8)
        return "unknown cache format";
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
        return "head_dim must be 64, 128 or 256";
    if (c->n_heads < 1 || c->n_heads > 256)
        return "n_heads must be 1 .. 256";
    if (c->n_pages < 1 || c->n_pages > MOST_PAGES)
        return "n_pages must be 1 .. 2^30";
    if (!c->data || !c->scales)
        return "null cache array";
    if (!aligned(c->data, 16) || !aligned(c->scales, 16) || !aligned(c->mass, 16))
        return "cache arrays must be 16-byte aligned";
    out = KvCache{static_cast<uint8_t *>(c->data), c->scales, c->mass, int(c->n_pages), int(c->n_heads), int(c->head_dim)};
    return nullptr;
}

const char *view_seqs(const msi_kv_seqs *s, bool rows, KvSeqs &out)
{
    if (!s)
        return "null sequences";
    if (s->n_seqs > 65535)
        return "n_seqs must be at most 65535";
    if (s->flags & ~MSI_KV_ALL_ROWS)
        return "unknown flags of the sequences";
    if (s->max_blocks > MOST / MSI_KV_BLOCK || s->max_len > uint64_t(s->max_blocks) * MSI_KV_BLOCK)
        return "max_len must be at most 64 * max_blocks, max_blocks at most 2^23";
    if (s->n_seqs && (!s->lens || (s->max_len && !s->table)))
        return "null sequence array";
    if (rows) {
        if (s->n_rows > MOST || s->max_rows > s->n_rows)
            return "max_rows must be at most n_rows, n_rows at most 2^29";
        if (s->n_seqs && !s->cu_rows)
            return "null cu_rows";
    }
    if (!aligned(s->table, 4) || !aligned(s->lens, 4) || !aligned(s->cu_rows, 4))
        return "sequence arrays must be 4-byte aligned";
    out = KvSeqs{s->table, s->lens, rows ? s->cu_rows : nullptr, int(s->n_seqs), int(s->max_blocks),
                 rows ? int(s->n_rows) : 0, rows ? int(s->max_rows) : 0, int(s->max_len),
                 (s->flags & MSI_KV_ALL_ROWS) != 0};
    return nullptr;
}

bool rows_ok(const void *p, uint64_t stride, uint64_t least)
{
    return p && aligned(p, 16) && stride >= least && stride % 8 == 0 && stride <= MOST_STRIDE;
}

constexpr const char *STATUS_TEXT = "status must be a 4-byte aligned word";

// what append and read have in common; go: there is work
const char *view_rows(const msi_kv_cache *cache, const msi_kv_seqs *seqs, const void *k, const void *v, uint64_t ks,
                      uint64_t vs, const uint32_t *status, KvCache &c, KvSeqs &s, bool &go)
{
    if (!aligned(status, 4))
        return STATUS_TEXT;
    if (const char *e = view_cache(cache, c))
        return e;
    if (const char *e = view_seqs(seqs, true, s))
        return e;
    go = s.S && s.max_rows && s.max_len;
    const uint64_t least = uint64_t(c.H) * c.D;
    if (go && (!rows_ok(k, ks, least) || !rows_ok(v, vs, least)))
        return "k and v need 16-byte aligned rows of n_heads * head_dim, strides a multiple of 8 up to 2^21";
    return nullptr;
}

const char *check_heads(const KvCache &c, const KvSeqs &s, uint32_t n_q_heads)
{
    if (n_q_heads == 0 || n_q_heads % uint32_t(c.H) || n_q_heads > 4096)
        return "n_q_heads must be a multiple of n_heads, at most 4096";
    const uint64_t rows = uint64_t(s.max_rows) * (n_q_heads / c.H);
    if (rows > MOST)
        return "max_rows times the heads of a group must be at most 2^29";
    if ((rows + 127) / 128 * uint64_t(c.H) * uint64_t(s.S) >= MOST_GROUPS - (s.all_rows ? 128 : 0))
        return "n_seqs * n_heads * (max_rows * heads of a group / 128) must be under 2^24 (less 128 with MSI_KV_ALL_ROWS)";
    if (uint64_t(s.S) * ((s.max_len + KV_BLOCK - 1) / KV_BLOCK) > MOST)
        return "n_seqs times the blocks of max_len must be at most 2^29";
    return nullptr;
}

// bytes of the log-sums that follow the cut's workspace
size_t lse_bytes(const AttentionCut &cut, const KvSeqs &s, uint32_t n_q_heads, uint32_t mass_rows)
{
    return mass_rows && !cut.few ? size_t(s.n_rows) * n_q_heads * sizeof(float) : 0;
}

}  // namespace

extern "C" {

msi_status msi_linear(const msi_linear_args *a, void *stream)
{
    if (!a)
        return bad("null arguments");
    if (a->activation > MSI_ACT_GELU_TANH)
        return bad("unknown activation");
    if (a->out_dtype > MSI_BF16 || (a->residual && a->residual_dtype > MSI_BF16))
        return bad("unknown dtype");
    if (a->K < 8 || a->K % 8 || a->K > MOST_STRIDE)
        return bad("K must be a multiple of 8, 8 .. 2^21");
    if (a->M > MOST || a->N > MOST || uint64_t(a->M) * a->N > MOST_OUTPUTS)
        return bad("M and N must be at most 2^29, M * N at most 2^36");
    if (a->M == 0 || a->N == 0)
        return MSI_OK;
    if (!rows_ok(a->x, a->x_stride, a->K))
        return bad("x needs 16-byte aligned rows of K, a stride that is a multiple of 8 up to 2^21");
    if (!a->w || !aligned(a->w, 16))
        return bad("w must be a 16-byte aligned [N, K]");
    const size_t ob = a->out_dtype == MSI_F32 ? 4 : 2, rb = a->residual_dtype == MSI_F32 ? 4 : 2;
    if (!a->out || !aligned(a->out, ob) || a->out_stride < a->N || a->out_stride > MOST)
        return bad("out needs rows of N, aligned to its type, a stride up to 2^29");
    if (a->residual && (!aligned(a->residual, rb) || a->residual_stride < a->N || a->residual_stride > MOST))
        return bad("residual needs rows of N, aligned to its type, a stride up to 2^29");
    if (a->residual == a->out && (a->residual_dtype != a->out_dtype || a->residual_stride != a->out_stride))
        return bad("a residual that is out needs its type and stride");
    if (a->out == a->x || a->out == a->w)
        return bad("out must not be x or w");
    if (!aligned(a->bias, 4))
        return bad("bias must be 4-byte aligned");
    LinearArgs l{};
    l.x = static_cast<const uint16_t *>(a->x);
    l.w = static_cast<const uint16_t *>(a->w);
    l.bias = a->bias;
    if (a->residual) {
        if (a->residual_dtype == MSI_F32)
            l.res_f32 = static_cast<const float *>(a->residual);
        else
            l.res_bf16 = static_cast<const uint16_t *>(a->residual);
    }
    if (a->out_dtype == MSI_F32)
        l.out_f32 = static_cast<float *>(a->out);
    else
        l.out_bf16 = static_cast<uint16_t *>(a->out);
    l.x_stride = int64_t(a->x_stride);
    l.res_stride = int64_t(a->residual_stride);
    l.out_stride = int64_t(a->out_stride);
    l.M = int(a->M);
    l.N = int(a->N);
    l.K = int(a->K);
    return launched(launch_linear(l, int(a->activation), static_cast<hipStream_t>(stream)));
}

msi_status msi_debug_linear_tile(uint32_t M, uint32_t N, uint32_t *rows, uint32_t *features, uint32_t *per_cu)
{
    if (!rows || !features || !per_cu)
        return bad("null output");
    if (M < 1 || N < 1 || M > MOST || N > MOST || uint64_t(M) * N > MOST_OUTPUTS)
        return bad("M and N must be 1 .. 2^29, M * N at most 2^36");
    const LinearTile t = linear_tile(M, N);
    *rows = uint32_t(t.rows);
    *features = uint32_t(t.features);
    *per_cu = uint32_t(t.per_cu);
    return MSI_OK;
}

msi_status msi_kv_append(const msi_kv_cache *cache, const msi_kv_seqs *seqs, const void *k, const void *v,
                         uint64_t k_stride, uint64_t v_stride, uint32_t *status, void *stream)
{
    KvCache c;
    KvSeqs s;
    bool go = false;
    if (const char *e = view_rows(cache, seqs, k, v, k_stride, v_stride, status, c, s, go))
        return bad(e);
    if (!go)
        return MSI_OK;
    return launched(launch_kv_append(c, int(cache->format), s, static_cast<const uint16_t *>(k),
                                     static_cast<const uint16_t *>(v), int64_t(k_stride), int64_t(v_stride), status,
                                     static_cast<hipStream_t>(stream)));
}

msi_status msi_kv_read(const msi_kv_cache *cache, const msi_kv_seqs *seqs, void *k, void *v, uint64_t k_stride,
                       uint64_t v_stride, uint32_t *status, void *stream)
{
    KvCache c;
    KvSeqs s;
    bool go = false;
    if (const char *e = view_rows(cache, seqs, k, v, k_stride, v_stride, status, c, s, go))
        return bad(e);
    if (!go)
        return MSI_OK;
    return launched(launch_kv_read(c, int(cache->format), s, static_cast<uint16_t *>(k), static_cast<uint16_t *>(v),
                                   int64_t(k_stride), int64_t(v_stride), status, static_cast<hipStream_t>(stream)));
}

msi_status msi_kv_attention_workspace(const msi_kv_cache *cache, const msi_kv_seqs *seqs, uint32_t n_q_heads,
                                      uint32_t mass_rows, uint64_t *bytes)
{
    KvCache c;
    KvSeqs s;
    if (!bytes)
        return bad("null bytes");
    if (const char *e = view_cache(cache, c))
        return bad(e);
    if (const char *e = view_seqs(seqs, true, s))
        return bad(e);
    if (const char *e = check_heads(c, s, n_q_heads))
        return bad(e);
    if (mass_rows && !c.mass)
        return bad("mass_rows needs the cache's mass");
    *bytes = 0;
    if (s.S && s.max_rows) {
        const AttentionCut cut = attention_cut(s.S, c.H, int(n_q_heads) / c.H, c.D, c.n_pages, s.max_rows, s.max_len, mass_rows != 0);
        *bytes = cut.bytes + lse_bytes(cut, s, n_q_heads, mass_rows);
    }
    return MSI_OK;
}

msi_status msi_kv_attention(const msi_kv_cache *cache, const msi_kv_seqs *seqs, const msi_kv_attention_args *a,
                            void *stream)
{
    KvCache c;
    KvSeqs s;
    if (!a)
        return bad("null arguments");
    if (const char *e = view_cache(cache, c))
        return bad(e);
    if (const char *e = view_seqs(seqs, true, s))
        return bad(e);
    if (const char *e = check_heads(c, s, a->n_q_heads))
        return bad(e);
    const float scale_log2 = float(double(a->scale) * 1.4426950408889634);
    if (!std::isfinite(scale_log2))
        return bad("scale must be finite, under 2^127");
    if (!aligned(a->status, 4))
        return bad(STATUS_TEXT);
    if (a->mass_rows && !c.mass)
        return bad("mass_rows needs the cache's mass");
    if (a->mass_rows && !(a->mass_decay >= 0.0f && std::isfinite(a->mass_decay)))
        return bad("mass_decay must be finite and not negative");
    const bool go = s.S && s.max_rows, rest = s.all_rows && s.n_rows;
    if (!go && !rest)
        return MSI_OK;
    const uint64_t least = uint64_t(a->n_q_heads) * c.D;
    if (!rows_ok(a->q, a->q_stride, least) || !rows_ok(a->out, a->out_stride, least))
        return bad("q and out need 16-byte aligned rows of n_q_heads * head_dim, strides a multiple of 8 up to 2^21");
    if (a->q == a->out)
        return bad("out must not be q");
    if (!go)
        return launched(launch_kv_rest(s, static_cast<uint16_t *>(a->out), int64_t(a->out_stride), int(least),
                                       static_cast<hipStream_t>(stream)));
    const AttentionCut cut =
        attention_cut(s.S, c.H, int(a->n_q_heads) / c.H, c.D, c.n_pages, s.max_rows, s.max_len, a->mass_rows != 0);
    const size_t lse = lse_bytes(cut, s, a->n_q_heads, a->mass_rows), need = cut.bytes + lse;
    if (need && (!a->workspace || a->workspace_bytes < need))
        return abi_error(MSI_E_NOMEM, "workspace smaller than msi_kv_attention_workspace says");
    if (!aligned(a->workspace, 16))
        return bad("workspace must be 16-byte aligned");
    uint8_t *ws = static_cast<uint8_t *>(a->workspace);
    AttentionLaunch A{};
    A.c = c;
    A.s = s;
    A.q = static_cast<const uint16_t *>(a->q);
    A.out = static_cast<uint16_t *>(a->out);
    A.q_stride = int64_t(a->q_stride);
    A.out_stride = int64_t(a->out_stride);
    A.G = int(a->n_q_heads) / c.H;
    A.scale_log2 = scale_log2;
    A.direct = cut.direct;
    A.per = cut.per;
    A.part_rows = s.max_rows * A.G;
    if (!cut.direct) {
        A.plan = reinterpret_cast<int2 *>(ws);
        A.part_ml = reinterpret_cast<float *>(ws + cut.part_ml);
        A.part_o = reinterpret_cast<float *>(ws + cut.part_o);
    }
    if (a->mass_rows && cut.few)
        A.scores = reinterpret_cast<float *>(ws + cut.scores);
    A.score_blocks = cut.score_blocks;
    if (lse)
        A.lse = reinterpret_cast<float *>(ws + cut.bytes);
    A.mass_rows = int(std::min(a->mass_rows, MOST));
    A.decay = a->mass_decay;
    A.status = a->status;
    return launched(launch_kv_attention(A, int(cache->format), cut, static_cast<hipStream_t>(stream)));
}

msi_status msi_kv_evict(const msi_kv_cache *cache, const msi_kv_seqs *seqs, const msi_kv_evict_args *a, void *stream)
{
    KvCache c;
    KvSeqs s;
    if (!a)
        return bad("null arguments");
    if (const char *e = view_cache(cache, c))
        return bad(e);
    if (const char *e = view_seqs(seqs, false, s))
        return bad(e);
    if (!aligned(a->status, 4))
        return bad(STATUS_TEXT);
    if (!c.mass)
        return bad("eviction needs the cache's mass");
    if (a->budget < 1 || a->budget > MOST || uint64_t(a->sinks) + a->recent > a->budget)
        return bad("budget must be 1 .. 2^29 and at least sinks + recent");
    if (s.S == 0)
        return MSI_OK;
    const uint32_t most = std::min<uint32_t>(a->budget, uint32_t(s.max_len));
    if (a->dst_blocks > MOST / MSI_KV_BLOCK || uint64_t(a->dst_blocks) * MSI_KV_BLOCK < most)
        return bad("dst_table is too short for min(budget, max_len) tokens");
    if (!a->new_lens || !a->keep || (most && !a->dst_table))
        return bad("null output");
    if (a->new_lens == s.lens || a->dst_table == s.table)
        return bad("new_lens and dst_table must not be the call's lens and table");
    if (!aligned(a->new_lens, 4) || !aligned(a->keep, 4) || !aligned(a->dst_table, 4))
        return bad("outputs must be 4-byte aligned");
    return launched(launch_kv_evict(c, int(cache->format), s, a->dst_table, int(a->dst_blocks), a->new_lens, a->keep,
                                    int(a->budget), int(a->sinks), int(a->recent), a->status,
                                    static_cast<hipStream_t>(stream)));
}

}  // extern "C"
