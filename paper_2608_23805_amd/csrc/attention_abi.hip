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

// Groups of a call and how it is cut; nullptr if the call may go on, else what is wrong.
const char *view_groups(const msi_kv_groups *g, const KvCache &c, const KvSeqs &s, uint32_t n_q_heads, KvGroups &out, SharedCut &cut)
{
    if (!g)
        return "null groups";
    if (g->n_groups > 65535)
        return "n_groups must be at most 65535";
    if (g->reserved)
        return "reserved must be 0";
    if (g->n_groups && (!g->cu_seqs || !g->blocks))
        return "null group array";
    if (!aligned(g->cu_seqs, 4) || !aligned(g->blocks, 4))
        return "group arrays must be 4-byte aligned";
    const uint64_t G = n_q_heads / uint32_t(c.H);
    const uint32_t max_rows = std::min(g->max_rows, uint32_t(s.n_rows)), max_blocks = std::min(g->max_blocks, uint32_t(s.max_blocks));
    if (max_rows * G > MOST)
        return "a group's max_rows times the heads of a cache head must be at most 2^29";
    if (uint64_t(s.max_rows) * n_q_heads >= MOST_GROUPS)
        return "max_rows times n_q_heads must be under 2^24";
    out = KvGroups{g->cu_seqs, g->blocks, int(g->n_groups), int(max_rows), int(max_blocks),
                   std::min(int(max_blocks), s.max_len / KV_BLOCK)};
    cut = shared_cut(s, out, c.H, int(G), c.D);
    if ((uint64_t(cut.items_p) + uint64_t(cut.items_s)) * uint64_t(c.H) >= MOST_GROUPS)
        return "the groups' and sequences' row tiles times n_heads must be under 2^24";
    return nullptr;
}

// A projection's arguments as the kernels take them; go: there is work.
const char *view_linear(const msi_linear_args *a, LinearArgs &l, bool &go)
{
    if (!a)
        return "null arguments";
    if (a->activation > MSI_ACT_GELU_TANH)
        return "unknown activation";
    if (a->out_dtype > MSI_BF16 || (a->residual && a->residual_dtype > MSI_BF16))
        return "unknown dtype";
    if (a->K < 8 || a->K % 8 || a->K > MOST_STRIDE)
        return "K must be a multiple of 8, 8 .. 2^21";
    if (a->M > MOST || a->N > MOST || uint64_t(a->M) * a->N > MOST_OUTPUTS)
        return "M and N must be at most 2^29, M * N at most 2^36";
    if (a->M == 0 || a->N == 0)
        return nullptr;
    if (!rows_ok(a->x, a->x_stride, a->K))
        return "x needs 16-byte aligned rows of K, a stride that is a multiple of 8 up to 2^21";
    if (!a->w || !aligned(a->w, 16))
        return "w must be a 16-byte aligned [N, K]";
    const size_t ob = a->out_dtype == MSI_F32 ? 4 : 2, rb = a->residual_dtype == MSI_F32 ? 4 : 2;
    if (!a->out || !aligned(a->out, ob) || a->out_stride < a->N || a->out_stride > MOST)
        return "out needs rows of N, aligned to its type, a stride up to 2^29";
    if (a->residual && (!aligned(a->residual, rb) || a->residual_stride < a->N || a->residual_stride > MOST))
        return "residual needs rows of N, aligned to its type, a stride up to 2^29";
    if (a->residual == a->out && (a->residual_dtype != a->out_dtype || a->residual_stride != a->out_stride))
        return "a residual that is out needs its type and stride";
    if (a->out == a->x || a->out == a->w)
        return "out must not be x or w";
    if (!aligned(a->bias, 4))
        return "bias must be 4-byte aligned";
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
    go = true;
    return nullptr;
}

// What attention calls have in common: their views, and scale, status, q and out; go: there are rows to attend, rest:
// there are rows to clear.
const char *view_attention(const msi_kv_cache *cache, const msi_kv_seqs *seqs, const msi_kv_attention_args *a, AttentionLaunch &A,
                           bool &go, bool &rest)
{
    if (!a)
        return "null arguments";
    if (const char *e = view_cache(cache, A.c))
        return e;
    if (const char *e = view_seqs(seqs, true, A.s))
        return e;
    if (const char *e = check_heads(A.c, A.s, a->n_q_heads))
        return e;
    A.scale_log2 = float(double(a->scale) * 1.4426950408889634);
    if (!std::isfinite(A.scale_log2))
        return "scale must be finite, under 2^127";
    if (!aligned(a->status, 4))
        return STATUS_TEXT;
    if (a->mass_rows && !A.c.mass)
        return "mass_rows needs the cache's mass";
    if (a->mass_rows && !(a->mass_decay >= 0.0f && std::isfinite(a->mass_decay)))
        return "mass_decay must be finite and not negative";
    go = A.s.S && A.s.max_rows;
    rest = A.s.all_rows && A.s.n_rows;
    if (!go && !rest)
        return nullptr;
    const uint64_t least = uint64_t(a->n_q_heads) * A.c.D;
    if (!rows_ok(a->q, a->q_stride, least) || !rows_ok(a->out, a->out_stride, least))
        return "q and out need 16-byte aligned rows of n_q_heads * head_dim, strides a multiple of 8 up to 2^21";
    if (a->q == a->out)
        return "out must not be q";
    A.q = static_cast<const uint16_t *>(a->q);
    A.out = static_cast<uint16_t *>(a->out);
    A.q_stride = int64_t(a->q_stride);
    A.out_stride = int64_t(a->out_stride);
    A.G = int(a->n_q_heads) / A.c.H;
    A.part_rows = A.s.max_rows * A.G;
    A.status = a->status;
    return nullptr;
}

msi_status clear_all(const AttentionLaunch &A, hipStream_t st)
{
    return launched(launch_kv_rest(A.s, A.out, A.out_stride, A.c.H * A.G * A.c.D, st));
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
    LinearArgs l{};
    bool go = false;
    if (const char *e = view_linear(a, l, go))
        return bad(e);
    if (!go)
        return MSI_OK;
    return launched(launch_linear(l, int(a->activation), static_cast<hipStream_t>(stream)));
}

msi_status msi_linear_q4(const msi_linear_q4_args *a, void *stream)
{
    if (!a)
        return bad("null arguments");
    if (a->group != 32 && a->group != 64 && a->group != 128)
        return bad("group must be 32, 64 or 128");
    if (a->linear.K == 0 || a->linear.K % a->group)
        return bad("K must be a multiple of group");
    if (a->reserved)
        return bad("reserved must be 0");
    LinearQ4Args q{};
    bool go = false;
    if (const char *e = view_linear(&a->linear, q.l, go))
        return bad(e);
    if (!go)
        return MSI_OK;
    if (!a->scales || !aligned(a->scales, 2))
        return bad("scales must be a 2-byte aligned [N, K / group]");
    if (a->linear.out == a->scales)
        return bad("out must not be scales");
    q.codes = static_cast<const uint8_t *>(a->linear.w);
    q.scales = static_cast<const uint16_t *>(a->scales);
    q.group = int(a->group);
    return launched(launch_linear_q4(q, int(a->linear.activation), static_cast<hipStream_t>(stream)));
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

msi_status msi_debug_linear_q4_tile(uint32_t M, uint32_t N, uint32_t K, uint32_t *rows, uint32_t *features, uint32_t *per_cu)
{
    if (!rows || !features || !per_cu)
        return bad("null output");
    if (M < 1 || N < 1 || M > MOST || N > MOST || uint64_t(M) * N > MOST_OUTPUTS || K < 32 || K % 32 || K > MOST_STRIDE)
        return bad("M and N must be 1 .. 2^29, M * N at most 2^36, K a multiple of 32, 32 .. 2^21");
    const LinearTile t = linear_q4_tile(M, N, K);
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

msi_status msi_kv_append_rotary(const msi_kv_cache *cache, const msi_kv_seqs *seqs,
                                const msi_kv_append_rotary_args *a, void *stream)
{
    RotaryAppend A{};
    bool go = false;
    if (!a)
        return bad("null arguments");
    if (const char *e = view_rows(cache, seqs, a->k, a->v, a->k_stride, a->v_stride, a->status, A.c, A.s, go))
        return bad(e);
    if (a->rot_dim < 16 || a->rot_dim % 16 || a->rot_dim > uint32_t(A.c.D))
        return bad("rot_dim must be a multiple of 16, 16 .. head_dim");
    if (a->n_axes < 1 || a->n_axes > 4)
        return bad("n_axes must be 1 .. 4");
    if (a->interleaved > 1)
        return bad("interleaved must be 0 or 1");
    if (a->q && (a->n_q_heads < 1 || a->n_q_heads > 4096))
        return bad("n_q_heads must be 1 .. 4096");
    if (!go)
        return MSI_OK;
    if (!a->freq || !aligned(a->freq, 8) || !aligned(a->axis, 8))
        return bad("freq and axis must be 8-byte aligned, freq not null");
    if (!a->positions || !aligned(a->positions, 4) || a->position_stride > (uint64_t(1) << 32) ||
        (a->n_axes > 1 && a->position_stride < uint64_t(A.s.n_rows)))
        return bad("positions must be a 4-byte aligned [n_axes, n_rows], their stride at least n_rows, at most 2^32");
    if (a->q) {
        const uint64_t least = uint64_t(a->n_q_heads) * A.c.D;
        if (!rows_ok(a->q, a->q_stride, least) || !rows_ok(a->q_out, a->q_out_stride, least))
            return bad("q and q_out need 16-byte aligned rows of n_q_heads * head_dim, strides a multiple of 8 up to 2^21");
        if (a->q == a->q_out && a->q_stride != a->q_out_stride)
            return bad("a q_out that is q needs its stride");
        if (a->q_out == a->k || a->q_out == a->v)
            return bad("q_out must not be k or v");
    }
    A.q = static_cast<const uint16_t *>(a->q);
    A.q_out = static_cast<uint16_t *>(a->q_out);
    A.k = static_cast<const uint16_t *>(a->k);
    A.v = static_cast<const uint16_t *>(a->v);
    A.q_stride = int64_t(a->q_stride);
    A.q_out_stride = int64_t(a->q_out_stride);
    A.k_stride = int64_t(a->k_stride);
    A.v_stride = int64_t(a->v_stride);
    A.n_q_heads = int(a->n_q_heads);
    A.rot = int(a->rot_dim);
    A.n_axes = int(a->n_axes);
    A.freq = a->freq;
    A.axis = a->axis;
    A.positions = a->positions;
    A.position_stride = int64_t(a->position_stride);
    A.status = a->status;
    return launched(launch_kv_append_rotary(A, int(cache->format), a->interleaved != 0, static_cast<hipStream_t>(stream)));
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
    AttentionLaunch A{};
    bool go = false, rest = false;
    if (const char *e = view_attention(cache, seqs, a, A, go, rest))
        return bad(e);
    if (!go)
        return rest ? clear_all(A, static_cast<hipStream_t>(stream)) : MSI_OK;
    const AttentionCut cut = attention_cut(A.s.S, A.c.H, A.G, A.c.D, A.c.n_pages, A.s.max_rows, A.s.max_len, a->mass_rows != 0);
    const size_t lse = lse_bytes(cut, A.s, a->n_q_heads, a->mass_rows), need = cut.bytes + lse;
    if (need && (!a->workspace || a->workspace_bytes < need))
        return abi_error(MSI_E_NOMEM, "workspace smaller than msi_kv_attention_workspace says");
    if (!aligned(a->workspace, 16))
        return bad("workspace must be 16-byte aligned");
    uint8_t *ws = static_cast<uint8_t *>(a->workspace);
    A.direct = cut.direct;
    A.per = cut.per;
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
    return launched(launch_kv_attention(A, int(cache->format), cut, static_cast<hipStream_t>(stream)));
}

msi_status msi_kv_attention_shared_workspace(const msi_kv_cache *cache, const msi_kv_seqs *seqs, const msi_kv_groups *groups,
                                             uint32_t n_q_heads, uint64_t *bytes)
{
    KvCache c;
    KvSeqs s;
    KvGroups g;
    SharedCut cut;
    if (!bytes)
        return bad("null bytes");
    if (const char *e = view_cache(cache, c))
        return bad(e);
    if (const char *e = view_seqs(seqs, true, s))
        return bad(e);
    if (const char *e = check_heads(c, s, n_q_heads))
        return bad(e);
    if (const char *e = view_groups(groups, c, s, n_q_heads, g, cut))
        return bad(e);
    *bytes = cut.bytes;
    return MSI_OK;
}

msi_status msi_kv_attention_shared(const msi_kv_cache *cache, const msi_kv_seqs *seqs, const msi_kv_groups *groups,
                                   const msi_kv_attention_args *a, void *stream)
{
    SharedLaunch A{};
    bool go = false, rest = false;
    if (const char *e = view_attention(cache, seqs, a, A, go, rest))
        return bad(e);
    if (const char *e = view_groups(groups, A.c, A.s, a->n_q_heads, A.g, A.cut))
        return bad(e);
    if (a->mass_rows)
        return bad("mass_rows must be 0: a shared page has several sequences' weights");
    if (!go)
        return rest ? clear_all(A, static_cast<hipStream_t>(stream)) : MSI_OK;
    if (!a->workspace || a->workspace_bytes < A.cut.bytes)
        return abi_error(MSI_E_NOMEM, "workspace smaller than msi_kv_attention_shared_workspace says");
    if (!aligned(a->workspace, 16))
        return bad("workspace must be 16-byte aligned");
    uint8_t *ws = static_cast<uint8_t *>(a->workspace);
    A.owners = reinterpret_cast<KvOwner *>(ws);
    A.first = reinterpret_cast<int32_t *>(ws + A.cut.first);
    A.part_ml = reinterpret_cast<float *>(ws + A.cut.part_ml);
    A.part_o = reinterpret_cast<float *>(ws + A.cut.part_o);
    return launched(launch_kv_attention_shared(A, int(cache->format), static_cast<hipStream_t>(stream)));
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
