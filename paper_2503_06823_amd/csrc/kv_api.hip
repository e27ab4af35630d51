// C ABI of the paged 4-bit cache and of the attention over it: host-side argument checks and dispatch.  The operations are
// documented in include/emoe.h.
#include <math.h>

#include <initializer_list>

#include "kv_cache.h"

namespace emoe {

int validate_kv_desc(const emoe_kv_desc* d) {
    if (d == nullptr) return EMOE_ERR_NULL;
    if (d->page_size < 16 || d->page_size > 256 || (d->page_size & (d->page_size - 1)) != 0) return EMOE_ERR_UNSUPPORTED;
    if (d->head_dim != 64 && d->head_dim != 128) return EMOE_ERR_UNSUPPORTED;
    if (d->pages <= 0 || d->kv_heads <= 0 || d->rows < 0 || d->table_width <= 0) return EMOE_ERR_SHAPE;
    if (d->kv_heads > 256 || d->rows > 65536) return EMOE_ERR_UNSUPPORTED;
    const long long most = (1ll << 31) - 1;
    if ((long long)d->pages * d->page_size > most || (long long)d->table_width * d->page_size > most) return EMOE_ERR_SHAPE;
    return EMOE_OK;
}

int validate_attention(const emoe_kv_desc* d, const emoe_attention_desc* a) {
    int rc = validate_kv_desc(d);
    if (rc != EMOE_OK) return rc;
    if (a == nullptr) return EMOE_ERR_NULL;
    if (a->dtype != EMOE_F32 && a->dtype != EMOE_BF16) return EMOE_ERR_UNSUPPORTED;
    if (a->reserved != 0) return EMOE_ERR_UNSUPPORTED;
    if (a->T < 0 || a->q_heads <= 0 || a->q_heads % d->kv_heads != 0 || a->window < 0 || a->sinks < 0) return EMOE_ERR_SHAPE;
    if (a->max_new < 0 || a->max_new > a->T || (a->T > 0 && a->max_new == 0)) return EMOE_ERR_SHAPE;
    if (a->q_heads / d->kv_heads > 256) return EMOE_ERR_UNSUPPORTED;
    if ((long long)a->T * a->q_heads >= (1ll << 27)) return EMOE_ERR_SHAPE;
    if (!isfinite(a->scale)) return EMOE_ERR_SHAPE;
    const long long row = (long long)a->q_heads * d->head_dim;
    if (a->q_stride < row || a->out_stride < row) return EMOE_ERR_SHAPE;
    if (a->q_stride % 8 != 0 || a->out_stride % 8 != 0) return EMOE_ERR_UNSUPPORTED;
    return EMOE_OK;
}

namespace {
constexpr int64_t kMostElements = 1ll << 33;  // of the rows of one append or read: threads of eight in a launch
bool unaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
// Whether some buffer of `written` is one of `read` (NULL: none).
bool shared(std::initializer_list<const void*> written, std::initializer_list<const void*> read) {
    for (const void* w : written)
        for (const void* r : read)
            if (w != nullptr && w == r) return true;
    return false;
}
int status_of(hipError_t e) { return e == hipSuccess ? EMOE_OK : EMOE_ERR_DEVICE; }
}  // namespace

}  // namespace emoe

using namespace emoe;

extern "C" {

int emoe_kv_cache_bytes(const emoe_kv_desc* desc, size_t* bytes) {
    int rc = validate_kv_desc(desc);
    if (rc != EMOE_OK) return rc;
    if (!bytes) return EMOE_ERR_NULL;
    *bytes = (size_t)desc->pages * desc->kv_heads * (size_t)kv_page(*desc).bytes();
    return EMOE_OK;
}

int emoe_kv_plan(const emoe_kv_desc* desc, int32_t T, const int32_t* len, const int32_t* new_len, int32_t* block_table,
                 const int32_t* free_pages, const int64_t* counters, int32_t* cu_new, int32_t* slot, int32_t* position,
                 int32_t* seq_len, int64_t* counters_out, int32_t* refused, void* stream) {
    int rc = validate_kv_desc(desc);
    if (rc != EMOE_OK) return rc;
    if (T < 0) return EMOE_ERR_SHAPE;
    if (!free_pages || !counters || !cu_new || !counters_out || !refused) return EMOE_ERR_NULL;
    if (desc->rows > 0 && (!len || !new_len || !block_table || !seq_len)) return EMOE_ERR_NULL;
    if (T > 0 && (!slot || !position)) return EMOE_ERR_NULL;
    if (shared({block_table, cu_new, slot, position, seq_len, counters_out, refused}, {len, new_len, free_pages, counters})) return EMOE_ERR_SHAPE;
    return status_of(launch_kv_plan(*desc, T, len, new_len, block_table, free_pages, counters, cu_new, slot, position, seq_len,
                                    counters_out, refused, static_cast<hipStream_t>(stream)));
}

int emoe_kv_release(const emoe_kv_desc* desc, const int32_t* len_before, const int32_t* len, const int32_t* ended, int32_t window,
                    int32_t sinks, const int32_t* block_table, int32_t* free_pages, const int64_t* counters,
                    int64_t* counters_out, void* stream) {
    int rc = validate_kv_desc(desc);
    if (rc != EMOE_OK) return rc;
    if (window < 0 || sinks < 0) return EMOE_ERR_SHAPE;
    if (!free_pages || !counters || !counters_out) return EMOE_ERR_NULL;
    if (desc->rows > 0 && (!len || !block_table || (window > 0 && !len_before))) return EMOE_ERR_NULL;
    if (shared({free_pages, counters_out}, {len_before, len, ended, block_table, counters})) return EMOE_ERR_SHAPE;
    return status_of(launch_kv_release(*desc, len_before, len, ended, window, sinks, block_table, free_pages, counters, counters_out,
                                       static_cast<hipStream_t>(stream)));
}

int emoe_kv_advance(const emoe_kv_desc* desc, const int32_t* seq_len, const int32_t* ended, int32_t* len, void* stream) {
    int rc = validate_kv_desc(desc);
    if (rc != EMOE_OK) return rc;
    if (desc->rows == 0) return EMOE_OK;
    if (!seq_len || !len) return EMOE_ERR_NULL;
    if (shared({len}, {seq_len, ended})) return EMOE_ERR_SHAPE;
    return status_of(launch_kv_advance(*desc, seq_len, ended, len, static_cast<hipStream_t>(stream)));
}

int emoe_kv_append(const emoe_kv_desc* desc, int32_t T, int32_t dtype, const void* k, int64_t k_stride, const void* v,
                   int64_t v_stride, const int32_t* slot, void* cache, void* stream) {
    int rc = validate_kv_desc(desc);
    if (rc != EMOE_OK) return rc;
    if (dtype != EMOE_F32 && dtype != EMOE_BF16) return EMOE_ERR_UNSUPPORTED;
    const int64_t row = (int64_t)desc->kv_heads * desc->head_dim;
    if (T < 0 || k_stride < row || v_stride < row || T * row > kMostElements) return EMOE_ERR_SHAPE;
    if (k_stride % 8 != 0 || v_stride % 8 != 0) return EMOE_ERR_UNSUPPORTED;
    if (T == 0) return EMOE_OK;  // whatever the pointers: an empty buffer may have no address
    if (!k || !v || !slot || !cache) return EMOE_ERR_NULL;
    if (unaligned(k) || unaligned(v) || unaligned(cache)) return EMOE_ERR_UNSUPPORTED;
    return status_of(launch_kv_append(*desc, T, dtype, k, k_stride, v, v_stride, slot, cache, static_cast<hipStream_t>(stream)));
}

int emoe_kv_read(const emoe_kv_desc* desc, int32_t T, int32_t dtype, const void* cache, const int32_t* slot, void* k, void* v,
                 void* stream) {
    int rc = validate_kv_desc(desc);
    if (rc != EMOE_OK) return rc;
    if (dtype != EMOE_F32 && dtype != EMOE_BF16) return EMOE_ERR_UNSUPPORTED;
    if (T < 0 || (int64_t)T * desc->kv_heads * desc->head_dim > kMostElements) return EMOE_ERR_SHAPE;
    if (T == 0) return EMOE_OK;
    if (!k || !v || !slot || !cache) return EMOE_ERR_NULL;
    if (unaligned(k) || unaligned(v) || unaligned(cache)) return EMOE_ERR_UNSUPPORTED;
    return status_of(launch_kv_read(*desc, T, dtype, cache, slot, k, v, static_cast<hipStream_t>(stream)));
}

int emoe_kv_attention_workspace_bytes(const emoe_kv_desc* desc, const emoe_attention_desc* attention, size_t* bytes) {
    int rc = validate_attention(desc, attention);
    if (rc != EMOE_OK) return rc;
    if (!bytes) return EMOE_ERR_NULL;
    *bytes = attention_ws_bytes(*desc, *attention);
    return EMOE_OK;
}

int emoe_kv_attention(const emoe_kv_desc* desc, const emoe_attention_desc* attention, const void* q, const void* cache,
                      const int32_t* block_table, const int32_t* seq_len, const int32_t* cu_new, void* out, void* ws,
                      size_t ws_bytes, void* stream) {
    int rc = validate_attention(desc, attention);
    if (rc != EMOE_OK) return rc;
    if (attention->T == 0 || desc->rows == 0) return EMOE_OK;
    if (!q || !cache || !block_table || !seq_len || !cu_new || !out) return EMOE_ERR_NULL;
    if (unaligned(q) || unaligned(cache) || unaligned(out)) return EMOE_ERR_UNSUPPORTED;
    if (!ws || unaligned(ws) || ws_bytes < attention_ws_bytes(*desc, *attention)) return EMOE_ERR_WORKSPACE;
    AttentionArgs a;
    a.q = q;
    a.cache = static_cast<const uint8_t*>(cache);
    a.table = block_table;
    a.seq_len = seq_len;
    a.cu_new = cu_new;
    a.out = out;
    a.ws = static_cast<uint8_t*>(ws);
    a.q_stride = attention->q_stride;
    a.out_stride = attention->out_stride;
    a.scale_log2 = attention->scale * 1.44269504088896340736f;
    a.T = attention->T;
    a.R = desc->rows;
    a.max_new = attention->max_new;
    a.q_heads = attention->q_heads;
    a.kv_heads = desc->kv_heads;
    a.set_group(attention->q_heads / desc->kv_heads);
    a.width = desc->table_width;
    a.pages = desc->pages;
    a.window = attention->window;
    a.sinks = attention->sinks;
    a.page = kv_page(*desc);
    return status_of(launch_attention(*desc, *attention, a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
