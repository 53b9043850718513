// C ABI of the cache that keeps keys and values in 8 bits: places, append, attention.  Argument validation, workspace
// carving, launches.
#include <cstring>

#include "splash_kv8.cuh"
#include "splash_umma.cuh"

namespace splash {

cudaError_t launch_kv_slots(int32_t B, const int32_t *seq_lens, const int32_t *new_lens, const int32_t *free_pages, int64_t num_free,
                            const int32_t *free_begin, int32_t *table, int64_t table_stride, int32_t table_width, int64_t num_slots,
                            int64_t *slot_map, int32_t *positions, int32_t *q_start, int32_t *new_seq_lens, int32_t *counts, int sm_count,
                            cudaStream_t stream);
cudaError_t launch_kv8_append(const splash_kv8_cache &cache, int32_t dtype, int64_t rows, const void *k, int64_t k_row, int64_t k_head, const void *v,
                              int64_t v_row, int64_t v_head, const int64_t *slot_map, int sm_count, cudaStream_t stream);
void kv8_decode_shape(int64_t pairs, int head_dim, int sm_count, int *rows, int *workers);
bool kv8_pool_maps(const splash_kv8_cache &c, CUtensorMap *k_map, CUtensorMap *v_map);
int kv8_chunk_rows();
int kv8_chunk_workers(int sm_count);
cudaError_t launch_kv8_chunk(const kv8::AttnParams &p, const splash_kv8_cache &cache, cudaStream_t stream);
cudaError_t launch_kv8_decode(const kv8::AttnParams &p, int D, int rows, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream);

namespace {

bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int invalid(const char *what) { set_error("%s", what); return SPLASH_INVALID_ARG; }
int unsupported(const char *what) { set_error("%s", what); return SPLASH_UNSUPPORTED; }
int launched(cudaError_t e) {
    if (e == cudaSuccess) return SPLASH_OK;
    set_error("CUDA error: %s", cudaGetErrorString(e));
    return SPLASH_CUDA_ERROR;
}

int check_cache(const splash_kv8_cache *c) {
    if (c == nullptr) return invalid("cache is NULL");
    if (c->struct_size != sizeof(splash_kv8_cache)) {
        set_error("cache.struct_size is %u, this library expects %zu", c->struct_size, sizeof(splash_kv8_cache));
        return SPLASH_INVALID_ARG;
    }
    if (c->head_dim != 64 && c->head_dim != 128) return unsupported("only head_dim 64 and 128 are built");
    if (c->page_size != kPage) return unsupported("only page_size = 64 is built");
    if (c->num_kv_heads < 1 || c->num_kv_heads > 65535) return unsupported("num_kv_heads must be in [1, 65535]");
    if (c->num_pages < 1) return invalid("num_pages must be positive");
    if (!c->k_pool || !c->v_pool || !c->k_scales || !c->v_scales) return invalid("a pointer of the cache is NULL");
    if (!aligned_to(c->k_pool, 16) || !aligned_to(c->v_pool, 16) || !aligned_to(c->k_scales, 4) || !aligned_to(c->v_scales, 4))
        return invalid("misaligned pointer (pools 16 B, scales 4 B)");
    const int64_t rows = 64 * (int64_t)c->head_dim;
    for (const int64_t stride : {c->k_page_stride, c->v_page_stride})
        if (c->num_pages > 1 && (stride < rows || stride % 16)) return invalid("page strides must be multiples of 16 bytes and hold a head's 64 rows");
    for (const int64_t stride : {c->k_head_stride, c->v_head_stride})
        if (c->num_kv_heads > 1 && (stride < rows || stride % 16)) return invalid("head strides must be multiples of 16 bytes and hold a head's 64 rows");
    if (c->num_pages > 1 && (c->k_scale_stride < c->num_kv_heads || c->v_scale_stride < c->num_kv_heads))
        return invalid("scale strides must be at least num_kv_heads");
    return SPLASH_OK;
}

int check_query(const splash_kv8_cache *c, const splash_kv8_query *s) {
    if (s == nullptr) return invalid("query is NULL");
    if (s->struct_size != sizeof(splash_kv8_query)) {
        set_error("query.struct_size is %u, this library expects %zu", s->struct_size, sizeof(splash_kv8_query));
        return SPLASH_INVALID_ARG;
    }
    if (s->num_requests < 0 || s->num_rows < 0 || s->table_width < 0) return invalid("negative size");
    if (s->num_rows > 0x7fffffff) return unsupported("more than 2^31 - 1 query rows");
    if (s->num_heads < 1 || s->num_heads % c->num_kv_heads) return invalid("num_heads must be a multiple of num_kv_heads");
    if (s->num_heads / c->num_kv_heads > 1024) return unsupported("more than 1,024 heads for each key head");
    if (s->max_q_rows < 1) return invalid("max_q_rows must be positive");
    const int64_t rows = s->max_q_rows < s->num_rows ? s->max_q_rows : s->num_rows;
    if (rows * (s->num_heads / c->num_kv_heads) > 0x3fffffff) return unsupported("too many query rows in one request");
    if (s->dtype != SPLASH_DTYPE_BF16 && s->dtype != SPLASH_DTYPE_FP16) return unsupported("q must be bf16 or fp16");
    if (s->out_dtype != s->dtype && s->out_dtype != SPLASH_DTYPE_FP32) return unsupported("out must have the type of q or be fp32");
    const int64_t D = c->head_dim;
    if (s->q_row_stride % 8 || s->q_head_stride % 8 || s->out_row_stride % 8 || s->out_head_stride % 8)
        return invalid("strides of q and out must be multiples of 8 elements");
    if (s->num_heads > 1 && (s->q_head_stride < D || s->out_head_stride < D)) return invalid("head strides of q and out must be at least head_dim");
    if (s->num_rows > 1 && (s->q_row_stride < D || s->out_row_stride < D)) return invalid("row strides of q and out must be at least head_dim");
    if (s->num_rows > 1 && s->lse_row_stride < s->num_heads) return invalid("lse_row_stride < num_heads");
    if (s->num_requests > 1 && s->block_table_stride < s->table_width) return invalid("block_table_stride < table_width");
    if (!(s->softmax_scale == s->softmax_scale)) return invalid("softmax_scale is NaN");
    return SPLASH_OK;
}

// The workspace: status block, records of cut items, partial results of the workers (two each).
struct View { int32_t *status; int4 *cut; float *lse, *out; size_t bytes; };

View carve(void *base, int workers, int rows, int D) {
    uint8_t *const b = static_cast<uint8_t *>(base);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return b + here; };
    View v;
    v.status = reinterpret_cast<int32_t *>(take(64));
    v.cut = reinterpret_cast<int4 *>(take((size_t)workers * 2 * sizeof(int4)));
    v.lse = reinterpret_cast<float *>(take((size_t)2 * workers * rows * 4));
    v.out = reinterpret_cast<float *>(take((size_t)2 * workers * rows * D * 4));
    v.bytes = at;
    return v;
}

// How a call runs: requests of up to this many (row, head) pairs on the decode kernel, the others, if there may be any, on the kernel for chunks.  What the
// two take, in us, for contexts of 4,096 tokens and eight key heads (decode / chunks):
//     heads of 128   64 contexts: 16 pairs 119 / 175, 24 215 / 177, 32 223 / 178     16 contexts: 44 / 62, 64 / 62, 66 / 63     four: 22.5 / 27, 26 / 27.5, 26 / 27.5
//     heads of 64    64 contexts: 24 pairs 101 / 133, 32 135 / 135, 40 179 / 136     16 contexts: 34 / 46, 46 / 46, 54 / 47     four: 23 / 24, 30 / 24, 24 / 24
// 64 pairs of 128 are 411 / 185 with 64 contexts.  So the limits suit few contexts; of many, the chunk kernel has 17 to 32 pairs of 128 and 33 to 40 of 64 done
// sooner.  Pairs alone do not tell the two apart: the work of a block would have to come into it.
int decode_pairs(const splash_kv8_cache *c) { return c->head_dim == 64 ? 40 : 32; }

constexpr int64_t kMaxTokens = 1LL << 30;      // of a context: positions and page ends stay in 32 bits

struct Plan { int rows, workers, chunk_workers; int64_t pairs; bool decode; };

Plan plan_call(const splash_kv8_cache *c, const splash_kv8_query *s, int sms) {
    Plan p;
    p.pairs = (int64_t)s->max_q_rows * (s->num_heads / c->num_kv_heads);
    const int64_t pairs = p.pairs < decode_pairs(c) ? p.pairs : decode_pairs(c);
    kv8_decode_shape(pairs, c->head_dim, sms, &p.rows, &p.workers);
    // no more blocks than the work can cost (with its overhead of five pages)
    const int64_t cost = (pairs + p.rows - 1) / p.rows * c->num_kv_heads * s->num_requests * (s->table_width + 5LL);
    if (cost > 0 && cost < p.workers) p.workers = (int)cost;
    p.chunk_workers = p.pairs > decode_pairs(c) ? kv8_chunk_workers(sms) : 0;
    // How many requests have few rows only the device knows.  If all of the T rows belong to requests, of at most R each, (B R - T) / (R - 1) of them at most have a
    // single one.  Where that is a quarter of them or less (a step of a fixed number of rows, one prompt), the kernel for chunks takes them all: two launches less,
    // 6 us of such a call.  It is a guess: with rows of nobody among the T (a batch padded to B R rows), or rows beyond R, there may be more, and they take the
    // slower kernel, with the same results (64 contexts of 4,096 tokens, eight heads a key head, a row each: 172 us with T = B R = 512 where 125 with T = 64).
    p.decode = p.chunk_workers == 0 || (int64_t)s->num_requests * s->max_q_rows - s->num_rows > (s->max_q_rows - 1LL) * s->num_requests / 4;
    return p;
}

// One region serves both kernels: the second writes only when the first's combine kernel is done.
View carve(void *base, const splash_kv8_cache *c, const Plan &p) {
    View v = carve(base, p.workers, p.rows, c->head_dim);
    const size_t chunk = carve(base, p.chunk_workers, kv8_chunk_rows(), c->head_dim).bytes;
    if (chunk > v.bytes) v.bytes = chunk;
    return v;
}

}  // namespace
}  // namespace splash

using namespace splash;

extern "C" {

int splash_kv_slots(int32_t num_requests, const int32_t *seq_lens, const int32_t *new_lens, const int32_t *free_pages, int64_t num_free,
                    const int32_t *free_begin, int32_t *block_table, int64_t block_table_stride, int32_t table_width, int64_t num_slots,
                    int64_t *slot_map, int32_t *positions, int32_t *q_start, int32_t *new_seq_lens, int32_t *counts, void *stream) {
    begin_call();
    if (num_requests < 0 || num_free < 0 || table_width < 0 || num_slots < 0) return invalid("negative size");
    if (num_requests > SPLASH_KV_SLOTS_MAX_REQUESTS) return unsupported("more than 16,384 requests");
    if (num_free > 0x7fffffff || num_slots > 0x7ffffffe) return unsupported("more than 2^31 - 1 free pages or places");
    if (num_requests > 1 && block_table_stride < table_width) return invalid("block_table_stride < table_width");
    if (!free_begin || !q_start || !counts || (num_free > 0 && !free_pages) || (num_slots > 0 && (!slot_map || !positions)) ||
        (num_requests > 0 && (!seq_lens || !new_lens || !new_seq_lens || (table_width > 0 && !block_table))))
        return invalid("a required pointer is NULL");
    for (const void *p : {(const void *)seq_lens, (const void *)new_lens, (const void *)free_pages, (const void *)free_begin, (const void *)block_table,
                          (const void *)positions, (const void *)q_start, (const void *)new_seq_lens, (const void *)counts})
        if (!aligned_to(p, 4)) return invalid("misaligned pointer (4 B, slot_map 8 B)");
    if (!aligned_to(slot_map, 8)) return invalid("misaligned pointer (4 B, slot_map 8 B)");
    // every block reads the inputs while another may have written its outputs
    const struct { const void *at; int64_t bytes; bool written; } a[] = {
        {seq_lens, 4LL * num_requests, false}, {new_lens, 4LL * num_requests, false}, {free_pages, 4 * num_free, false}, {free_begin, 4, false},
        {block_table, num_requests > 0 ? 4 * ((num_requests - 1) * block_table_stride + table_width) : 0, true}, {slot_map, 8 * num_slots, true},
        {positions, 4 * num_slots, true}, {q_start, 4LL * num_requests + 4, true}, {new_seq_lens, 4LL * num_requests, true}, {counts, 16, true}};
    for (const auto &x : a)
        for (const auto &y : a) {
            const char *const xa = static_cast<const char *>(x.at), *const ya = static_cast<const char *>(y.at);
            if (&x != &y && x.written && x.bytes > 0 && y.bytes > 0 && xa < ya + y.bytes && ya < xa + x.bytes)
                return invalid("an output overlaps another argument");
        }
    int sms = 0;
    const int rc = usable_device(sms);
    if (rc != SPLASH_OK) return rc;
    return launched(launch_kv_slots(num_requests, seq_lens, new_lens, free_pages, num_free, free_begin, block_table, block_table_stride, table_width,
                                    num_slots, slot_map, positions, q_start, new_seq_lens, counts, sms, static_cast<cudaStream_t>(stream)));
}

int splash_kv8_append(const splash_kv8_cache *cache, int32_t dtype, int64_t num_rows, const void *k, int64_t k_row_stride, int64_t k_head_stride,
                      const void *v, int64_t v_row_stride, int64_t v_head_stride, const int64_t *slot_map, void *stream) {
    begin_call();
    int rc = check_cache(cache);
    if (rc != SPLASH_OK) return rc;
    if (dtype != SPLASH_DTYPE_BF16 && dtype != SPLASH_DTYPE_FP16) return unsupported("k and v must be bf16 or fp16");
    if (num_rows < 0) return invalid("num_rows < 0");
    if (num_rows == 0) return SPLASH_OK;
    if (!k || !v || !slot_map) return invalid("a required pointer is NULL");
    if (!aligned_to(k, 16) || !aligned_to(v, 16) || !aligned_to(slot_map, 8)) return invalid("misaligned pointer (k, v 16 B, slot_map 8 B)");
    for (const int64_t stride : {k_row_stride, v_row_stride})
        if (num_rows > 1 && (stride % 8 || stride < cache->head_dim)) return invalid("row strides must be multiples of 8 elements and at least head_dim");
    for (const int64_t stride : {k_head_stride, v_head_stride})
        if (cache->num_kv_heads > 1 && (stride % 8 || stride < cache->head_dim)) return invalid("head strides must be multiples of 8 elements and at least head_dim");
    int sms = 0;
    rc = usable_device(sms);
    if (rc != SPLASH_OK) return rc;
    return launched(launch_kv8_append(*cache, dtype, num_rows, k, k_row_stride, k_head_stride, v, v_row_stride, v_head_stride, slot_map, sms,
                                      static_cast<cudaStream_t>(stream)));
}

size_t splash_kv8_attention_workspace_bytes(const splash_kv8_cache *cache, const splash_kv8_query *query) {
    if (check_cache(cache) != SPLASH_OK || check_query(cache, query) != SPLASH_OK) return 0;
    int sms = 0;
    if (usable_device(sms) != SPLASH_OK) return 0;
    return carve(nullptr, cache, plan_call(cache, query, sms)).bytes;
}

int splash_kv8_attention(const splash_kv8_cache *cache, const splash_kv8_query *query, const void *q, const int32_t *block_table,
                         const int32_t *seq_lens, const int32_t *q_start, const int32_t *kv_begin, const int32_t *kv_end, void *out, float *lse,
                         void *workspace, size_t workspace_bytes, void *stream) {
    begin_call();
    int rc = check_cache(cache);
    if (rc == SPLASH_OK) rc = check_query(cache, query);
    if (rc != SPLASH_OK) return rc;
    if (q_start == nullptr && query->num_rows != query->num_requests) return invalid("without q_start every request has one row: num_rows must be num_requests");
    if (query->num_requests == 0 || query->num_rows == 0) return SPLASH_OK;
    if (!q || !seq_lens || !out || !lse || !workspace || (!block_table && query->table_width > 0)) return invalid("a required pointer is NULL");
    if (!aligned_to(q, 16) || !aligned_to(out, 16) || !aligned_to(lse, 4) || !aligned_to(workspace, 256) || !aligned_to(block_table, 4) ||
        !aligned_to(seq_lens, 4) || !aligned_to(q_start, 4) || !aligned_to(kv_begin, 4) || !aligned_to(kv_end, 4))
        return invalid("misaligned pointer (q, out 16 B, workspace 256 B, the others 4 B)");
    int sms = 0;
    rc = usable_device(sms);
    if (rc != SPLASH_OK) return rc;
    const Plan plan = plan_call(cache, query, sms);
    const View v = carve(workspace, cache, plan);
    if (workspace_bytes < v.bytes) {
        set_error("workspace has %zu bytes, %zu needed", workspace_bytes, v.bytes);
        return SPLASH_INVALID_ARG;
    }
    CUtensorMap k_map, v_map;
    if (plan.decode && !kv8_pool_maps(*cache, &k_map, &v_map)) return SPLASH_CUDA_ERROR;
    kv8::AttnParams p;
    memset(&p, 0, sizeof p);
    p.q = q; p.out = out; p.lse = lse;
    p.table = block_table; p.seq_lens = seq_lens; p.q_start = q_start; p.kv_begin = kv_begin; p.kv_end = kv_end;
    p.k_scales = cache->k_scales; p.v_scales = cache->v_scales;
    p.k_scale_stride = cache->k_scale_stride; p.v_scale_stride = cache->v_scale_stride;
    p.q_row = query->q_row_stride; p.q_head = query->q_head_stride; p.out_row = query->out_row_stride; p.out_head = query->out_head_stride;
    p.lse_row = query->lse_row_stride; p.table_stride = query->block_table_stride; p.max_tokens = 64LL * query->table_width < kMaxTokens ? 64LL * query->table_width : kMaxTokens;
    p.B = query->num_requests; p.T = (int32_t)query->num_rows; p.kv_heads = cache->num_kv_heads; p.group = query->num_heads / cache->num_kv_heads;
    p.num_pages = cache->num_pages; p.max_rows = query->max_q_rows;
    p.q_bf16 = query->dtype == SPLASH_DTYPE_BF16; p.out_f32 = query->out_dtype == SPLASH_DTYPE_FP32;
    p.whole = query->table_width <= kWholeRequestPages;
    p.workers = plan.workers;
    p.min_pairs = 1; p.max_pairs = decode_pairs(cache);
    p.scale_log2 = query->softmax_scale * umma::kLog2e;
    p.status = v.status; p.cut = v.cut; p.part_lse = v.lse; p.part_out = v.out;
    cudaError_t e = plan.decode ? launch_kv8_decode(p, cache->head_dim, plan.rows, k_map, v_map, static_cast<cudaStream_t>(stream)) : cudaSuccess;
    if (e == cudaSuccess && plan.chunk_workers > 0) {
        const View w = carve(workspace, plan.chunk_workers, kv8_chunk_rows(), cache->head_dim);
        p.workers = plan.chunk_workers;
        p.clear_status = !plan.decode;
        p.min_pairs = plan.decode ? decode_pairs(cache) + 1 : 1; p.max_pairs = 0x7fffffff;
        p.cut = w.cut; p.part_lse = w.lse; p.part_out = w.out;
        e = launch_kv8_chunk(p, *cache, static_cast<cudaStream_t>(stream));
    }
    return launched(e);
}

}  // extern "C"
