// Attention over a paged cache (nq_decoder.h): its entry points and how a call is cut.  The kernels are in nq_attn_kernels.h, one source to a type of cache.
#include "nq_attn_kernels.h"

struct nq_attn_s {
    nq::KvDesc kv;
    int q_heads, out_dtype;
    float scale, cap;
};

namespace nq {

// How a call is cut: rows of a tile (16: attn_split_kernel; 64, 128: attn_wide_kernel) and most items of a key head
struct AttnCut {
    int rows, slots, items;
    bool few;                // up to 64 rows of a sequence, on average
};
// rows: of a sequence, on average
static AttnCut cut_rows(const nq_attn_s& a, int64_t rows, int64_t n_seqs, int n_tokens)
{
    AttnCut c;
    const int group = a.q_heads / a.kv.heads;
    // (32 sequences of eight rows: tiles of 16 rows 127 us, of 64 137; one of 16384 rows: of 128 rows 342 us, of 64 440)
    c.few = rows <= 64;
    c.rows = rows <= 16 ? 16 : c.few || padded_dim(a.kv.head_dim) == 256 ? 64 : 128;      // (heads of 256: sums of 128 rows do not fit the registers)
    const int to_cu = padded_dim(a.kv.head_dim) == 256 && c.rows == 16 ? 1 : 2;             // workgroups that a CU's registers hold
    c.slots = std::max(1, to_cu * device_cu_count() / a.kv.heads);
    c.items = (int)(2 * c.slots + (int64_t)n_tokens * group / c.rows + n_seqs);
    return c;
}
static AttnCut cut_attention(const nq_attn_s& a, int n_seqs, int n_tokens)
{
    return cut_rows(a, std::max<int64_t>(1, (int64_t)n_tokens * (a.q_heads / a.kv.heads) / std::max(1, n_seqs)), n_seqs, n_tokens);
}
static size_t part_rows(const nq_attn_s& a, const AttnCut& c) { return (size_t)c.items * a.kv.heads * c.rows; }
// Room for a call and for every call with fewer sequences or tokens, so that one buffer serves whatever batch a program has next: of the cuts that such a call may have the
// largest (64 tokens of 32 sequences leave 16 rows to a tile, 64 of one sequence 128, with eight times the rows to an item).
static size_t workspace_of(const nq_attn_s& a, int n_seqs, int n_tokens)
{
    const int64_t rows = (int64_t)n_tokens * (a.q_heads / a.kv.heads);
    size_t most = 0;
    for (const int least : {0, 17, 65}) {                                   // rows of a sequence, on average, from which tiles are larger
        if (rows < least) break;
        const int64_t seqs = least ? std::min<int64_t>(n_seqs, rows / least) : n_seqs;
        most = std::max(most, part_rows(a, cut_rows(a, std::max(1, least), seqs, n_tokens)));
    }
    return most * (padded_dim(a.kv.head_dim) + 4) * sizeof(float);
}

}  // namespace nq

using namespace nq;

extern "C" int nq_attn_create(nq_attn* out, nq_kv kv, int q_heads, double scale, double cap, int out_dtype)
{
    const char* const who = "nq_attn_create";
    if (!out) return refuse(NQ_E_NULL, who, "out is NULL");
    *out = nullptr;
    if (!kv) return refuse(NQ_E_NULL, who, "NULL cache");
    if (q_heads < 1 || q_heads % kv->d.heads || q_heads > 65535) return refuse(NQ_E_SHAPE, who, "q_heads must be a multiple of the cache's heads, at most 65535");
    if (!std::isfinite(scale) || !std::isfinite(cap) || cap < 0.0) return refuse(NQ_E_INVALID_ARG, who, "scale must be finite, cap finite and >= 0");
    // what the kernels form of them in 32 bits: scale log2(e), cap log2(e), scale / cap
    const double most = 2.3e38, least = 1.2e-38, slope = std::fabs(scale) / cap;
    if (std::fabs(scale) > most) return refuse(NQ_E_INVALID_ARG, who, "scale is beyond fp32");
    if (cap > 0.0 && (cap < least || cap > most || (scale != 0.0 && (slope < least || slope > most))))
        return refuse(NQ_E_INVALID_ARG, who, "cap, or scale / cap, is beyond fp32");
    if (!is_float_type(out_dtype)) return refuse(NQ_E_INVALID_ARG, who, "out_dtype must be NQ_F32, NQ_F16 or NQ_BF16");
    nq_attn a = new (std::nothrow) nq_attn_s{kv->d, q_heads, out_dtype, (float)scale, (float)cap};
    if (!a) return refuse(NQ_E_HIP, who, "out of host memory");
    *out = a;
    return NQ_OK;
}

extern "C" int nq_attn_destroy(nq_attn a)
{
    delete a;
    return NQ_OK;
}

static int check_sizes(const char* who, nq_attn a, int n_seqs, int n_tokens)
{
    if (!a) return refuse(NQ_E_NULL, who, "NULL handle");
    if (n_seqs < 1) return refuse(NQ_E_INVALID_ARG, who, "n_seqs must be >= 1");
    if (n_tokens < 0) return refuse(NQ_E_INVALID_ARG, who, "n_tokens must be >= 0");
    // rows are counted in 32 bits; a launch has fewer than 2^32 threads (and 64 sequences' items, at most one more than all to each, fit 32 bits)
    if ((int64_t)n_tokens * a->q_heads > (INT64_C(1) << 30) || ((int64_t)n_seqs + 4096) * a->kv.heads > (INT64_C(1) << 30) ||
        (int64_t)cut_attention(*a, n_seqs, n_tokens).items * a->kv.heads >= (INT64_C(1) << 24))
        return refuse(NQ_E_SHAPE, who, "too many tokens or sequences for one call");
    return NQ_OK;
}

extern "C" int nq_attn_workspace_bytes(nq_attn a, int n_seqs, int n_tokens, size_t* bytes)
{
    const char* const who = "nq_attn_workspace_bytes";
    if (!bytes) return refuse(NQ_E_NULL, who, "bytes is NULL");
    if (const int rc = check_sizes(who, a, n_seqs, n_tokens)) return rc;
    *bytes = workspace_of(*a, n_seqs, n_tokens);
    return NQ_OK;
}

extern "C" int nq_attn_forward(nq_attn a, const void* q, int64_t q_stride, const int32_t* new_begin, const int32_t* ctx_len, const int32_t* page_table, int64_t table_stride,
                               const uint32_t* tree, int tree_words, int n_seqs, int n_tokens, void* out, int64_t out_stride, float* lse, void* workspace,
                               size_t workspace_bytes, void* stream)
{
    const char* const who = "nq_attn_forward";
    if (const int rc = check_sizes(who, a, n_seqs, n_tokens)) return rc;
    if (n_tokens == 0) return NQ_OK;
    if (!q || !out) return refuse(NQ_E_NULL, who, "q or out is NULL");
    if (!new_begin || !ctx_len || !page_table) return refuse(NQ_E_NULL, who, "new_begin, ctx_len or page_table is NULL");
    if (off_align(q, 2) || off_align(out, type_bytes(a->out_dtype))) return refuse(NQ_E_ALIGN, who, "q and out must have the alignment of their elements");
    if (off_align(new_begin, 4) || off_align(ctx_len, 4) || off_align(page_table, 4) || off_align(tree, 4) || off_align(lse, 4))
        return refuse(NQ_E_ALIGN, who, "arrays must be 4-byte aligned");
    const int64_t width = (int64_t)a->q_heads * a->kv.head_dim;
    if (q_stride < width || out_stride < width) return refuse(NQ_E_SHAPE, who, "stride between tokens below a token's length");
    if (q_stride > (INT64_C(1) << 31) || out_stride > (INT64_C(1) << 31)) return refuse(NQ_E_SHAPE, who, "stride beyond 2^31");
    if (table_stride < 1 || table_stride > INT32_MAX) return refuse(NQ_E_SHAPE, who, "table_stride must be 1 to 2^31 - 1");
    if (tree && tree_words < 1) return refuse(NQ_E_SHAPE, who, "tree_words must be >= 1");
    const AttnCut c = cut_attention(*a, n_seqs, n_tokens);
    if (!workspace) return refuse(NQ_E_NULL, who, "workspace is NULL");
    if (off_align(workspace, 16)) return refuse(NQ_E_ALIGN, who, "workspace must be 16-byte aligned");
    if (workspace_bytes < workspace_of(*a, n_seqs, n_tokens)) return refuse(NQ_E_INVALID_ARG, who, "workspace too small");
    AttnArgs k = {};
    k.kv = a->kv;
    k.q = q;
    k.begin = new_begin;
    k.ctx = ctx_len;
    k.table = page_table;
    k.tree = tree;
    k.out = out;
    k.lse = lse;
    k.part_o = (float*)workspace;
    k.part_ml = k.part_o + part_rows(*a, c) * padded_dim(a->kv.head_dim);
    k.q_stride = q_stride;
    k.out_stride = out_stride;
    k.table_stride = table_stride;
    k.tree_words = tree ? tree_words : 0;
    k.n_seqs = n_seqs;
    k.n_tokens = n_tokens;
    k.q_heads = a->q_heads;
    k.group = a->q_heads / a->kv.heads;
    k.out_dtype = a->out_dtype;
    k.scale = a->scale;
    k.cap = a->cap;
    k.slots = c.slots;
    k.rows = c.rows;
    k.few = c.few;
    k.items = c.items;
    const hipStream_t s = (hipStream_t)stream;
    return a->kv.dtype == NQ_F16 ? attend_f16(k, who, s) : attend_bf16(k, who, s);
}
