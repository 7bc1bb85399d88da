// cache_api.cu -- the extern "C" entry points of the paged cache and of the
// token log probabilities (declared in include/rheo.h): argument validation, the
// scratch layout and launches on the caller's stream.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdlib>

#include "cache_kernels.h"
#include "rheo.h"
#include "rheo_device.cuh"
#include "rheo_kernels.h"

namespace rheo {
namespace {

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
int elem_bytes(int dtype) { return dtype == RHEO_BF16 ? 2 : 4; }
bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

int multiprocessors() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1)
        return 1;
    return sms;
}

bool valid(const rheo_cache_config* c) {
    if (!c || (c->dtype != RHEO_F32 && c->dtype != RHEO_BF16)) return false;
    if (c->batch < 1 || c->batch > kMaxCacheBatch || c->tokens < 1 || c->tokens > kMaxCacheTokens) return false;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return false;
    if (c->pages < 1 || (int64_t)c->pages * c->page_size > (int64_t)1 << 40) return false;
    if (c->max_pages < 1 || (int64_t)c->max_pages * c->page_size > (int64_t)1 << 30) return false;
    if ((int64_t)c->batch * c->max_pages > INT32_MAX) return false;
    if (c->head_dim != 64 && c->head_dim != 128) return false;
    if (c->kv_heads < 1 || c->q_heads < c->kv_heads || c->q_heads > 1024 || c->q_heads % c->kv_heads) return false;
    return true;
}

bool valid(const rheo_logprob_config* c) {
    return c && (c->dtype == RHEO_F32 || c->dtype == RHEO_BF16) && c->rows >= 1 && c->rows <= (1 << 20) &&
           c->vocab >= 1 && c->vocab <= kMaxVocab && c->top >= 0 && c->top <= kMaxTop && c->rows_per_temperature >= 1;
}

int page_shift(int page_size) {
    int s = 0;
    while ((1 << s) < page_size) ++s;
    return s;
}

// Whether n values of 4 bytes at p and m at q have none in common.
bool apart(const void* p, int64_t n, const void* q, int64_t m) {
    const uintptr_t x = (uintptr_t)p, y = (uintptr_t)q;
    return x + 4 * (uintptr_t)n <= y || y + 4 * (uintptr_t)m <= x;
}

// A stride of n > 1 places, in elements: whole 16-byte pieces and below 2^38 (a dimension of one has none).
constexpr int64_t kStrideEnd = (int64_t)1 << 38;
bool stride_ok(int64_t s, int64_t n, int es) {
    return n == 1 || (s > -kStrideEnd && s < kStrideEnd && s * es % 16 == 0);
}

bool kv_ok(const rheo_kv* kv, const rheo_cache_config& c) {
    if (!kv || !kv->key || !kv->value || !aligned16(kv->key) || !aligned16(kv->value)) return false;
    const auto fits = [&](int64_t s, int n) { return n == 1 || (s > 0 && stride_ok(s, n, elem_bytes(c.dtype))); };
    return fits(kv->key_page, c.pages) && fits(kv->key_head, c.kv_heads) && fits(kv->key_token, c.page_size) &&
           fits(kv->value_page, c.pages) && fits(kv->value_head, c.kv_heads) && fits(kv->value_token, c.page_size);
}

// Strides [batch][token][head] of queries, keys, values or outputs.
bool rows_ok(const rheo_cache_config& c, int64_t batch, int64_t token, int64_t head, int heads) {
    const int es = elem_bytes(c.dtype);
    return stride_ok(batch, c.batch, es) && stride_ok(token, c.tokens, es) && stride_ok(head, heads, es);
}

// The same of an output, whose rows share no element: from the smallest stride on, each is at least what the
// dimensions before it span.
bool out_rows_ok(const rheo_cache_config& c, int64_t batch, int64_t token, int64_t head, int heads) {
    if (!rows_ok(c, batch, token, head, heads)) return false;
    struct Dim { int64_t stride, n; };
    const auto dim = [](int64_t s, int64_t n) { return Dim{n == 1 ? 0 : std::abs(s), n}; };
    Dim d[3] = {dim(batch, c.batch), dim(token, c.tokens), dim(head, heads)};
    std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
    int64_t span = c.head_dim;
    for (const Dim& x : d) {
        if (x.n == 1) continue;
        if (x.stride < span) return false;
        span += (x.n - 1) * x.stride;
    }
    return true;
}

// What a call has to find at zero comes first and lies at the same places in every
// scratch buffer: the status word, the ticket of the tables and the tickets of the
// log probabilities' rows.  What a call leaves behind (parts, join records) lies
// behind that, so one buffer serves any of the functions at any sizes, in any order.
constexpr size_t kStatusAt = 0, kTicketAt = 256, kRowTicketsAt = 512;
constexpr size_t kPartsAt = (kRowTicketsAt + sizeof(unsigned) * kLogprobCutRows + 255) / 256 * 256;

struct CacheLayout {
    size_t join, part_ml, part_o, total;
};

CacheLayout cache_layout(const rheo_cache_config& c) {
    const int G = c.q_heads / c.kv_heads;
    const size_t ctas = kAttendCtas, rows = attend_part_rows(c.dtype, c.tokens, G);
    CacheLayout L{};
    size_t o = kPartsAt;
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o = up256(o + bytes);
        return at;
    };
    L.join = take(sizeof(int4) * ctas);
    L.part_ml = take(2 * ctas * rows * 2 * sizeof(float));
    L.part_o = take(2 * ctas * rows * c.head_dim * sizeof(float));
    L.total = o;
    return L;
}

// Rows that are not cut leave no parts, so the sizes do not depend on the configuration.
constexpr size_t kLogprobPartAt = kPartsAt;
constexpr size_t kLogprobKeysAt = (kLogprobPartAt + sizeof(float) * 4 * kLogprobParts + 255) / 256 * 256;
constexpr size_t kLogprobBytes = kLogprobKeysAt + sizeof(unsigned long long) * kMaxTop * kLogprobParts;

template <class T> T* at(void* p, size_t off) { return reinterpret_cast<T*>(static_cast<char*>(p) + off); }
int code(cudaError_t e) { return e == cudaSuccess ? RHEO_OK : RHEO_ELAUNCH; }

}  // namespace
}  // namespace rheo

using namespace rheo;

extern "C" int rheo_cache_sizes(const rheo_cache_config* cfg, size_t* scratch_bytes) {
    if (!valid(cfg)) return RHEO_EINVAL;
    if (scratch_bytes) *scratch_bytes = cache_layout(*cfg).total;
    return RHEO_OK;
}

extern "C" int rheo_logprob_sizes(const rheo_logprob_config* cfg, size_t* scratch_bytes) {
    if (!valid(cfg)) return RHEO_EINVAL;
    if (scratch_bytes) *scratch_bytes = kLogprobBytes;
    return RHEO_OK;
}

extern "C" int rheo_scratch_init(void* scratch, size_t bytes, rheo_stream_t stream) {
    if (!scratch || bytes < sizeof(unsigned)) return RHEO_EINVAL;
    return code(cudaMemsetAsync(scratch, 0, bytes, (cudaStream_t)stream));
}

extern "C" int rheo_scratch_status(void* scratch, rheo_stream_t stream, int32_t* status) {
    if (!scratch || !status) return RHEO_EINVAL;
    cudaStream_t s = (cudaStream_t)stream;
    unsigned host = 0;
    if (cudaMemcpyAsync(&host, scratch, sizeof(unsigned), cudaMemcpyDeviceToHost, s) != cudaSuccess) return RHEO_ELAUNCH;
    if (cudaMemsetAsync(scratch, 0, sizeof(unsigned), s) != cudaSuccess) return RHEO_ELAUNCH;
    if (cudaStreamSynchronize(s) != cudaSuccess) return RHEO_ELAUNCH;
    *status = (int32_t)host;
    return RHEO_OK;
}

extern "C" int rheo_cache_reserve(const rheo_cache_config* cfg, const int32_t* ctx_len, const int32_t* new_len,
                                  const int32_t* depth, const rheo_pages* before, const rheo_pages* after,
                                  int64_t* slot, int32_t* position, void* scratch, rheo_stream_t stream) {
    if (!valid(cfg) || !ctx_len || !before || !after || !slot || !position || !scratch) return RHEO_EINVAL;
    const int32_t* x[4] = {before->block_table, before->n_pages, before->free_list, before->n_free};
    const int32_t* y[4] = {after->block_table, after->n_pages, after->free_list, after->n_free};
    int same = 0;
    for (int i = 0; i < 4; ++i) {
        if (!x[i] || !y[i]) return RHEO_EINVAL;
        same += x[i] == y[i];
    }
    if (same != 0 && same != 4) return RHEO_EINVAL;
    ReserveArgs a{};
    a.B = cfg->batch;
    a.T = cfg->tokens;
    a.P = cfg->page_size;
    a.max_pages = cfg->max_pages;
    a.pages = cfg->pages;
    a.in_place = same == 4;
    a.ctx_len = ctx_len;
    a.new_len = new_len;
    a.depth = depth;
    a.before = *before;
    a.after = *after;
    a.slot = slot;
    a.position = position;
    a.status = at<unsigned>(scratch, kStatusAt);
    a.ticket = at<unsigned>(scratch, kTicketAt);
    return code(launch_reserve(a, multiprocessors(), (cudaStream_t)stream));
}

extern "C" int rheo_qk_norm_rope(const rheo_cache_config* cfg, const rheo_qkv* in, const void* q_weight,
                                 const void* k_weight, float eps, const float* cos_sin, int32_t max_position,
                                 int32_t rot, int32_t interleaved, const int64_t* slot, const int32_t* position,
                                 const rheo_kv* kv, void* q_out, int64_t q_out_batch, int64_t q_out_token,
                                 int64_t q_out_head, void* scratch, rheo_stream_t stream) {
    if (!valid(cfg) || !in || !in->q || !in->k || !in->v || !slot || !position || !q_out || !scratch) return RHEO_EINVAL;
    if (!kv_ok(kv, *cfg)) return RHEO_EINVAL;
    if (rot < 0 || rot > cfg->head_dim || rot % 8 != 0 || (rot > 0 && (!cos_sin || max_position < 1))) return RHEO_EINVAL;
    if (!(eps >= 0.0f) || (interleaved != 0 && interleaved != 1)) return RHEO_EINVAL;
    for (const void* p : {in->q, in->k, in->v, q_weight, k_weight, (const void*)cos_sin, (const void*)q_out})
        if (!aligned16(p)) return RHEO_EINVAL;
    if (!rows_ok(*cfg, in->q_batch, in->q_token, in->q_head, cfg->q_heads) ||
        !rows_ok(*cfg, in->k_batch, in->k_token, in->k_head, cfg->kv_heads) ||
        !rows_ok(*cfg, in->v_batch, in->v_token, in->v_head, cfg->kv_heads) ||
        !out_rows_ok(*cfg, q_out_batch, q_out_token, q_out_head, cfg->q_heads))
        return RHEO_EINVAL;
    RopeArgs a{};
    a.B = cfg->batch;
    a.T = cfg->tokens;
    a.Hq = cfg->q_heads;
    a.H = cfg->kv_heads;
    a.rot = rot;
    a.max_position = max_position;
    a.page_shift = page_shift(cfg->page_size);
    a.slots = (int64_t)cfg->pages * cfg->page_size;
    a.in = *in;
    a.q_weight = q_weight;
    a.k_weight = k_weight;
    a.eps = eps;
    a.cos_sin = cos_sin;
    a.slot = slot;
    a.position = position;
    a.kv = *kv;
    a.q_out = q_out;
    a.o_batch = q_out_batch;
    a.o_token = q_out_token;
    a.o_head = q_out_head;
    a.status = at<unsigned>(scratch, kStatusAt);
    return code(launch_rope(a, cfg->dtype == RHEO_BF16 ? 1 : 0, cfg->head_dim, interleaved != 0, multiprocessors(),
                            (cudaStream_t)stream));
}

extern "C" int rheo_tree_attend(const rheo_cache_config* cfg, const rheo_attend_io* io, const rheo_kv* kv,
                                const int32_t* block_table, const int32_t* ctx_len, const int32_t* new_len,
                                const uint8_t* mask, float scale, void* scratch, rheo_stream_t stream) {
    if (!valid(cfg) || !io || !io->q || !io->out || !block_table || !ctx_len || !scratch) return RHEO_EINVAL;
    if (!kv_ok(kv, *cfg) || !aligned16(io->q) || !aligned16(io->out)) return RHEO_EINVAL;
    if (!rows_ok(*cfg, io->q_batch, io->q_token, io->q_head, cfg->q_heads) ||
        !out_rows_ok(*cfg, io->out_batch, io->out_token, io->out_head, cfg->q_heads))
        return RHEO_EINVAL;
    if (!(scale > -INFINITY && scale < INFINITY)) return RHEO_EINVAL;
    const CacheLayout L = cache_layout(*cfg);
    AttendArgs a{};
    a.B = cfg->batch;
    a.T = cfg->tokens;
    a.H = cfg->kv_heads;
    a.G = cfg->q_heads / cfg->kv_heads;
    a.D = cfg->head_dim;
    a.P = cfg->page_size;
    a.page_shift = page_shift(cfg->page_size);
    a.pages = cfg->pages;
    a.max_pages = cfg->max_pages;
    a.ctas = kAttendCtas;
    a.lead = attend_lead(cfg->dtype);
    a.least = attend_least(cfg->dtype);
    a.item_rows = attend_item_rows(cfg->dtype, a.T, a.G);
    a.part_rows = attend_part_rows(cfg->dtype, a.T, a.G);
    a.io = *io;
    a.kv = *kv;
    a.block_table = block_table;
    a.ctx_len = ctx_len;
    a.new_len = new_len;
    a.mask = mask;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.part_o = at<float>(scratch, L.part_o);
    a.part_ml = at<float>(scratch, L.part_ml);
    a.join = at<int4>(scratch, L.join);
    a.status = at<unsigned>(scratch, kStatusAt);
    const cudaError_t e = launch_attend(a, cfg->dtype == RHEO_BF16 ? 1 : 0, (cudaStream_t)stream);
    return e == cudaErrorInvalidValue ? RHEO_EINVAL : code(e);  // a cache that no tensor map describes
}

extern "C" int rheo_cache_commit(const rheo_cache_config* cfg, int32_t layers, const rheo_kv* kv, int64_t key_layer,
                                 int64_t value_layer, const int32_t* block_table, const int32_t* ctx_len,
                                 const int32_t* accepted_len, const int32_t* accepted_nodes, int32_t depth,
                                 int32_t* next_len, void* scratch, rheo_stream_t stream) {
    if (!valid(cfg) || layers < 1 || layers > 4096 || !block_table || !ctx_len || !accepted_len || !accepted_nodes ||
        depth < 1 || depth > 128 || !next_len || !scratch)
        return RHEO_EINVAL;
    // a request's first CTA writes next_len while its others still read these
    const int64_t B = cfg->batch;
    if (!apart(next_len, B, ctx_len, B) || !apart(next_len, B, accepted_len, B) ||
        !apart(next_len, B, accepted_nodes, B * depth) || !apart(next_len, B, block_table, B * cfg->max_pages))
        return RHEO_EINVAL;
    const int es = elem_bytes(cfg->dtype);
    if (!kv_ok(kv, *cfg)) return RHEO_EINVAL;
    for (const int64_t s : {key_layer, value_layer})
        if (!stride_ok(s, 2, es) || (layers > 1 && s <= 0)) return RHEO_EINVAL;
    CommitArgs a{};
    a.B = cfg->batch;
    a.T = cfg->tokens;
    a.H = cfg->kv_heads;
    a.P = cfg->page_size;
    a.pages = cfg->pages;
    a.max_pages = cfg->max_pages;
    a.layers = layers;
    a.depth = depth;
    a.kv_elem_bytes = es;
    a.kv = *kv;
    a.key_layer = key_layer;
    a.value_layer = value_layer;
    a.block_table = block_table;
    a.ctx_len = ctx_len;
    a.accepted_len = accepted_len;
    a.accepted_nodes = accepted_nodes;
    a.next_len = next_len;
    a.status = at<unsigned>(scratch, kStatusAt);
    return code(launch_commit(a, cfg->head_dim * es, (cudaStream_t)stream));
}

extern "C" int rheo_token_logprobs(const rheo_logprob_config* cfg, const void* logits, int64_t row_stride,
                                   int64_t logit_rows, const int32_t* row_index, const int32_t* token,
                                   const float* temperature, const rheo_logprobs* out, void* scratch,
                                   rheo_stream_t stream) {
    if (!valid(cfg) || !logits || row_stride < cfg->vocab || logit_rows < 1 || !token || !out || !out->logprob ||
        !out->rank || !out->entropy || !scratch)
        return RHEO_EINVAL;
    if (cfg->top > 0 && (!out->top_ids || !out->top_logprobs)) return RHEO_EINVAL;
    const int es = elem_bytes(cfg->dtype);
    if ((uintptr_t)logits % es != 0) return RHEO_EINVAL;
    LogprobArgs a{};
    a.R = cfg->rows;
    a.V = cfg->vocab;
    a.k = cfg->top;
    a.per_t = cfg->rows_per_temperature;
    a.segments = logprob_segments(cfg->rows, cfg->vocab, cfg->dtype);
    a.logits = static_cast<const char*>(logits);
    a.row_stride_bytes = row_stride * es;
    a.logit_rows = logit_rows;
    a.row_index = row_index;
    a.token = token;
    a.temperature = temperature;
    a.out = *out;
    a.status = at<unsigned>(scratch, kStatusAt);
    a.ticket = at<unsigned>(scratch, kRowTicketsAt);
    a.part = at<float>(scratch, kLogprobPartAt);
    a.part_key = at<unsigned long long>(scratch, kLogprobKeysAt);
    return code(launch_logprobs(a, cfg->dtype == RHEO_BF16 ? 1 : 0, aligned16(logits) && a.row_stride_bytes % 16 == 0,
                                (cudaStream_t)stream));
}
