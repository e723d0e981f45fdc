// The paged cache of nq_decoder.h: its description, copies of whole pages and the compaction of accepted drafts, both over all layers of
// a model in one launch.  Nothing is computed: both are bound by the bytes they read and write.  64 pages of 16 tokens in 32 layers of a 7B-shaped
// model (1.07 GB read and written) take 205 us, 5.2 TB/s; the accepted paths of eight drafted trees in 80 layers 6.8 us, a launch and a chain of three loads.
#include <algorithm>

#include "nq_decoder_internal.h"

namespace nq {

// layers of one launch: their addresses travel as kernel arguments (2 KiB of the 4 that a launch may have), so that nothing has to be
// copied to the device first
constexpr int kKvLayers = 128;
struct KvLayers {
    uint16_t* k[kKvLayers];
    uint16_t* v[kKvLayers];
};

// A page is one block of memory where its rows (a slot's elements of a head) follow one another in either order; else it is copied row by row.
__global__ __launch_bounds__(256) void copy_pages_kernel(KvLayers layers, KvDesc d, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, bool block, int chunks)
{
    const int pair = blockIdx.x, layer = blockIdx.y, part = blockIdx.z;
    const int64_t from = src[pair], to = dst[pair];
    if (from < 0 || from >= d.n_pages || to < 0 || to >= d.n_pages) return;
    uint16_t* const base = (part & 1) ? layers.v[layer] : layers.k[layer];
    const uint16_t* const a = base + from * d.page_stride;
    uint16_t* const b = base + to * d.page_stride;
    const int per = d.head_dim >> 3, slots = 1 << d.page_shift;
    const int parts = gridDim.z >> 1, step = 256 * parts;
    // four loads of a thread before their stores
    for (int c0 = (part >> 1) * 256 + threadIdx.x; c0 < chunks; c0 += 4 * step) {
        v4u value[4];
        int64_t at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = c0 + i * step;
            if (block) {
                at[i] = (int64_t)c * 8;
            } else {
                const int row = c / per, head = row >> d.page_shift, slot = row & (slots - 1);
                at[i] = head * d.head_stride + slot * d.slot_stride + (c - row * per) * 8;
            }
            if (c < chunks) value[i] = *(gptr_v4u)(a + at[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c0 + i * step < chunks) *(__attribute__((address_space(1))) v4u*)(b + at[i]) = value[i];
    }
}

// One thread per 16 bytes of a slot of a head: it walks its sequence's path from the front, so that a slot is read (as a source, path[j] >= j)
// before the same thread writes it (as the destination of a later j).  Moves are read eight at a time, before their stores.
__global__ __launch_bounds__(256) void compact_kernel(KvLayers layers, KvDesc d, const int32_t* __restrict__ ctx_len, const int32_t* __restrict__ table,
                                                      int64_t table_stride, const int32_t* __restrict__ path, int64_t path_stride, const int32_t* __restrict__ path_len)
{
    const int seq = blockIdx.x, layer = blockIdx.y;
    const int per = d.head_dim >> 3;
    const int c = (blockIdx.z >> 1) * 256 + threadIdx.x;
    if (c >= d.heads * per) return;
    uint16_t* const base = ((blockIdx.z & 1) ? layers.v[layer] : layers.k[layer]) + (c / per) * d.head_stride + (c % per) * 8;
    const int64_t ctx = ctx_len[seq], most = table_stride << d.page_shift;
    const int len = (int)min((int64_t)path_len[seq], path_stride);
    const int32_t* const pages = table + seq * table_stride;
    const int32_t* const way = path + seq * path_stride;
    // where token i of the sequence lies, or -1
    auto place = [&](int64_t i) -> int64_t {
        if (i < 0 || i >= most) return -1;
        const int64_t page = pages[i >> d.page_shift];
        if (page < 0 || page >= d.n_pages) return -1;
        return page * d.page_stride + (i & ((1 << d.page_shift) - 1)) * d.slot_stride;
    };
    for (int j0 = 0; j0 < len; j0 += 8) {
        v4u value[8];
        int64_t to[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            to[i] = -1;
            if (j0 + i >= len) continue;
            const int32_t old = way[j0 + i];
            const int64_t from = old == j0 + i ? -1 : place(ctx + old);           // a move to its own place is none
            to[i] = from < 0 ? -1 : place(ctx + j0 + i);
            if (to[i] >= 0) value[i] = *(gptr_v4u)(base + from);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (to[i] >= 0) *(__attribute__((address_space(1))) v4u*)(base + to[i]) = value[i];
    }
}

// the caches' common description; NULL and differing handles are refused
static int same_caches(const char* who, const nq_kv* kvs, int n, KvDesc* d)
{
    if (!kvs) return refuse(NQ_E_NULL, who, "NULL array of caches");
    if (n < 1) return refuse(NQ_E_INVALID_ARG, who, "n must be >= 1");
    for (int i = 0; i < n; ++i)
        if (!kvs[i]) return refuse(NQ_E_NULL, who, "NULL cache in list");
    *d = kvs[0]->d;
    for (int i = 1; i < n; ++i) {
        const KvDesc& e = kvs[i]->d;
        if (e.page_stride != d->page_stride || e.slot_stride != d->slot_stride || e.head_stride != d->head_stride || e.n_pages != d->n_pages ||
            e.heads != d->heads || e.head_dim != d->head_dim || e.page_shift != d->page_shift || e.dtype != d->dtype)
            return refuse(NQ_E_INVALID_ARG, who, "the caches differ in shape, strides or type");
    }
    return NQ_OK;
}

static KvLayers some_layers(const nq_kv* kvs, int from, int count)
{
    KvLayers l = {};
    for (int i = 0; i < count; ++i) {
        l.k[i] = kvs[from + i]->d.k;
        l.v[i] = kvs[from + i]->d.v;
    }
    return l;
}

}  // namespace nq

using namespace nq;

extern "C" int nq_kv_create(nq_kv* out, void* k, void* v, int dtype, int kv_heads, int head_dim, int page_size, int64_t n_pages, int64_t page_stride,
                            int64_t slot_stride, int64_t head_stride)
{
    const char* const who = "nq_kv_create";
    if (!out) return refuse(NQ_E_NULL, who, "out is NULL");
    *out = nullptr;
    if (!k || !v) return refuse(NQ_E_NULL, who, "k or v is NULL");
    if (dtype != NQ_F16 && dtype != NQ_BF16) return refuse(NQ_E_INVALID_ARG, who, "dtype must be NQ_F16 or NQ_BF16");
    if (kv_heads < 1 || kv_heads > 65535) return refuse(NQ_E_SHAPE, who, "kv_heads must be 1 to 65535");
    if (head_dim < 8 || head_dim > NQ_MAX_HEAD_DIM || head_dim % 8) return refuse(NQ_E_SHAPE, who, "head_dim must be a multiple of 8, 8 to %d", NQ_MAX_HEAD_DIM);
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1))) return refuse(NQ_E_SHAPE, who, "page_size must be a power of two, 16 to 1024");
    if (n_pages < 1 || n_pages > INT32_MAX) return refuse(NQ_E_SHAPE, who, "n_pages must be 1 to 2^31 - 1");
    if (off_align(k, 16) || off_align(v, 16)) return refuse(NQ_E_ALIGN, who, "k and v must be 16-byte aligned");
    if (!page_stride && !slot_stride && !head_stride) {
        slot_stride = head_dim;
        head_stride = slot_stride * page_size;
        page_stride = head_stride * kv_heads;
    }
    // the elements stay apart: ordered by stride, each is at least the extent of the one before it; a dimension of one element has none
    struct { int64_t stride, count; } dim[3] = {{slot_stride, page_size}, {head_stride, kv_heads}, {page_stride, n_pages}};
    std::sort(dim, dim + 3, [](const auto& a, const auto& b) { return a.stride < b.stride; });
    int64_t extent = head_dim;
    for (const auto& e : dim) {
        if (e.stride < 0 || e.stride % 8) return refuse(NQ_E_ALIGN, who, "strides must be multiples of 8 elements");
        if (e.count == 1) continue;
        if (e.stride < extent) return refuse(NQ_E_SHAPE, who, "strides let elements overlap");
        if (e.stride > INT64_MAX / 4 / e.count) return refuse(NQ_E_SHAPE, who, "the cache is too large to be addressed");
        extent = e.stride * e.count;
    }
    const int64_t most = INT64_C(1) << 30;
    if (slot_stride > most || (kv_heads > 1 && head_stride > most) || (page_size - 1) * slot_stride + (kv_heads - 1) * (kv_heads > 1 ? head_stride : 0) + head_dim > most)
        return refuse(NQ_E_SHAPE, who, "a page must span less than 2 GiB");
    nq_kv h = new (std::nothrow) nq_kv_s;
    if (!h) return refuse(NQ_E_HIP, who, "out of host memory");
    int shift = 0;
    while ((1 << shift) < page_size) ++shift;
    h->d = KvDesc{(uint16_t*)k, (uint16_t*)v, page_stride, slot_stride, head_stride, n_pages, kv_heads, head_dim, shift, dtype};
    *out = h;
    return NQ_OK;
}

extern "C" int nq_kv_destroy(nq_kv kv)
{
    delete kv;
    return NQ_OK;
}

extern "C" int nq_kv_copy_pages(const nq_kv* kvs, int n, const int32_t* src, const int32_t* dst, int n_pairs, void* stream)
{
    const char* const who = "nq_kv_copy_pages";
    KvDesc d;
    if (const int rc = same_caches(who, kvs, n, &d)) return rc;
    if (n_pairs < 0) return refuse(NQ_E_INVALID_ARG, who, "n_pairs must be >= 0");
    if (n_pairs == 0) return NQ_OK;
    if (!src || !dst) return refuse(NQ_E_NULL, who, "src or dst is NULL");
    if (off_align(src, 4) || off_align(dst, 4)) return refuse(NQ_E_ALIGN, who, "src and dst must be 4-byte aligned");
    const int slots = 1 << d.page_shift, chunks = d.heads * slots * (d.head_dim / 8);
    const bool by_head = d.slot_stride == d.head_dim && (d.heads == 1 || d.head_stride == (int64_t)slots * d.head_dim);
    const bool by_slot = (d.heads == 1 || d.head_stride == d.head_dim) && d.slot_stride == (int64_t)d.heads * d.head_dim;
    for (int l0 = 0; l0 < n; l0 += kKvLayers) {
        const int count = std::min(kKvLayers, n - l0);
        // 16 KiB to a workgroup, less where there are few pages: up to four workgroups to a CU
        const int64_t units = 2ll * count * n_pairs;
        int parts = (int)std::max<int64_t>(1, std::min<int64_t>((chunks + 255) / 256, (4ll * device_cu_count() + units - 1) / units));
        parts = std::max(parts, std::min(32767, (chunks + 1023) / 1024));
        hipLaunchKernelGGL(copy_pages_kernel, dim3(n_pairs, count, 2 * parts), dim3(256), 0, (hipStream_t)stream, some_layers(kvs, l0, count), d, src, dst, by_head || by_slot,
                           chunks);
        if (const int rc = launched(who)) return rc;
    }
    return NQ_OK;
}

extern "C" int nq_kv_compact(const nq_kv* kvs, int n, const int32_t* ctx_len, const int32_t* page_table, int64_t table_stride, const int32_t* path, int64_t path_stride,
                             const int32_t* path_len, int n_seqs, void* stream)
{
    const char* const who = "nq_kv_compact";
    KvDesc d;
    if (const int rc = same_caches(who, kvs, n, &d)) return rc;
    if (n_seqs < 0) return refuse(NQ_E_INVALID_ARG, who, "n_seqs must be >= 0");
    if (n_seqs == 0) return NQ_OK;
    if (!ctx_len || !page_table || !path || !path_len) return refuse(NQ_E_NULL, who, "NULL array");
    if (off_align(ctx_len, 4) || off_align(page_table, 4) || off_align(path, 4) || off_align(path_len, 4)) return refuse(NQ_E_ALIGN, who, "arrays must be 4-byte aligned");
    if (table_stride < 1 || table_stride > INT32_MAX) return refuse(NQ_E_SHAPE, who, "table_stride must be 1 to 2^31 - 1");
    if (path_stride < 1 || path_stride > INT32_MAX) return refuse(NQ_E_SHAPE, who, "path_stride must be 1 to 2^31 - 1");
    const int groups = (d.heads * (d.head_dim / 8) + 255) / 256;
    for (int l0 = 0; l0 < n; l0 += kKvLayers) {
        const int count = std::min(kKvLayers, n - l0);
        hipLaunchKernelGGL(compact_kernel, dim3(n_seqs, count, 2 * groups), dim3(256), 0, (hipStream_t)stream, some_layers(kvs, l0, count), d, ctx_len, page_table,
                           table_stride, path, path_stride, path_len);
        if (const int rc = launched(who)) return rc;
    }
    return NQ_OK;
}
