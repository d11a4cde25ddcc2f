// Host runtime of the quantised cache: argument checks, its memory, and the
// launches on the caller's stream. Implements the last part of include/raas.h.
#include <algorithm>
#include <new>
#include <vector>

#include "raas.h"
#include "raas_handle.h"
#include "raas_quant_internal.h"

using namespace raas;

namespace {

// Sequences of a call (every workgroup reads all lengths), KV heads of them all (a
// workgroup of 256 threads each and those of cut ones: a launch has below 2^32 threads;
// 2^15 blocks of each, a 256th of them to a workgroup, are below 2^31), rows of their heads.
constexpr int kMaxBatch = 4096, kMaxUnits = 1 << 23, kMaxCallRows = 1 << 24;

}  // namespace

struct raas_quant_cache {
    raas_quant_config cfg;
    int device;
    bool bf16;
    size_t layer_bytes = 0;
    void *memory = nullptr, *pool = nullptr;
    float *part = nullptr, *ml = nullptr;
    int32_t* arrived = nullptr;
    size_t bytes = 0;
    std::vector<unsigned long long> streamed_at;  // count_streamed after each layer's last attention; 0: none yet
    hipStream_t last_stream = nullptr;
};

namespace {

// The call's layer and table, checked.
raas_status view(const raas_quant_cache* c, int32_t layer, const int32_t* table, int32_t width, int32_t batch,
                 QuantView& L) {
    if (!c) return fail(RAAS_E_INVALID, "cache is NULL");
    if (layer < 0 || layer >= c->cfg.n_layers)
        return fail(RAAS_E_INVALID, "layer %d out of range [0, %d)", layer, c->cfg.n_layers);
    if (batch < 0 || batch > c->cfg.max_batch)
        return fail(RAAS_E_INVALID, "batch must lie in [0, max_batch = %d] (got %d)", c->cfg.max_batch, batch);
    if (width < 1 || width > kMaxTokens / c->cfg.page_size)
        return fail(RAAS_E_INVALID, "table_width must lie in [1, %d] (got %d)", kMaxTokens / c->cfg.page_size, width);
    if (batch > 0 && !table) return fail(RAAS_E_INVALID, "table is NULL");
    L = QuantView{};
    L.pool = (uint8_t*)c->pool + (size_t)layer * c->layer_bytes;
    L.table = table;
    L.batch = batch;
    L.width = width;
    L.n_pages = c->cfg.n_pages;
    L.nkv = c->cfg.n_kv_heads;
    L.G = c->cfg.n_q_heads / c->cfg.n_kv_heads;
    L.D = c->cfg.head_dim;
    L.key_bits = c->cfg.key_bits;
    L.value_bits = c->cfg.value_bits;
    L.page_shift = __builtin_ctz(c->cfg.page_size / kQuantBlock);
    L.cap = width * c->cfg.page_size;
    return RAAS_OK;
}

raas_status copy(raas_quant_cache* c, int32_t layer, const void* k, const void* v, const int32_t* table, int32_t width,
                 const int32_t* start, const int32_t* counts, int32_t batch, int32_t max_tokens, bool write,
                 void* stream) {
    QuantView L;
    const raas_status st = view(c, layer, table, width, batch, L);
    if (st != RAAS_OK) return st;
    if (max_tokens < 0 || max_tokens > kMaxTokens)
        return fail(RAAS_E_INVALID, "max_tokens must lie in [0, %d] (got %d)", kMaxTokens, max_tokens);
    if (batch == 0 || max_tokens == 0) return RAAS_OK;
    if (!k || !v || !start) return fail(RAAS_E_INVALID, "k, v and start must be non-NULL");
    DeviceScope scope(c->device);
    if (scope.error() != hipSuccess) return hip_fail(scope.error(), "hipSetDevice");
    const QuantCopy io{const_cast<void*>(k), const_cast<void*>(v), start, counts, max_tokens};
    const hipError_t e = write ? launch_quant_write(L, c->bf16, io, (hipStream_t)stream)
                               : launch_quant_read(L, c->bf16, io, (hipStream_t)stream);
    if (e != hipSuccess) return hip_fail(e, write ? "write launch" : "read launch");
    c->last_stream = (hipStream_t)stream;
    return RAAS_OK;
}

// The attention of a call. What it reads is counted among the steps' reads: the
// table's pages, or the pool if that is less (lengths are not known here). By what
// was read since the layer's last attention its codes are still in the memory-side
// cache or not; a captured call, whose replays are not seen here, counts the cache's
// other layers, and `prefix_bytes` for each.
raas_status attention(raas_quant_cache* c, int32_t layer, const QuantView& L, QuantAttention& io, double prefix_bytes,
                      hipStream_t s) {
    io.scale_log2 = scale_log2(L.D);
    io.part = c->part;
    io.ml = c->ml;
    io.arrived = c->arrived;
    const double page = (double)(c->layer_bytes / L.n_pages);
    const double own = page * std::min((double)L.n_pages, (double)L.batch * L.width);
    double others = (c->cfg.n_layers - 1.0) * own + c->cfg.n_layers * prefix_bytes;
    if (!capturing(s)) {
        const unsigned long long before = count_streamed(c->device, (unsigned long long)own);
        if (c->streamed_at[layer] != 0) others = (double)(before - c->streamed_at[layer]);
        c->streamed_at[layer] = before + (unsigned long long)own;
    }
    const hipError_t e = launch_quant_attention(L, c->bf16, io, non_temporal(own, others), s);
    if (e != hipSuccess) return hip_fail(e, "attention launch");
    c->last_stream = s;
    return RAAS_OK;
}

}  // namespace

extern "C" {

raas_status raas_create_quant_cache(const raas_quant_config* cfg, void* stream, raas_quant_cache** out) {
    if (!out) return fail(RAAS_E_INVALID, "out is NULL");
    if (!cfg) return fail(RAAS_E_INVALID, "cfg is NULL");
    if (cfg->n_layers < 1) return fail(RAAS_E_INVALID, "n_layers must be >= 1 (got %d)", cfg->n_layers);
    const raas_status st = check_heads(cfg->n_q_heads, cfg->n_kv_heads, cfg->head_dim, cfg->dtype);
    if (st != RAAS_OK) return st;
    const int ps = cfg->page_size;
    if (ps != 32 && ps != 64 && ps != 128 && ps != 256)
        return fail(RAAS_E_INVALID, "page_size must be 32, 64, 128 or 256 (got %d)", ps);
    if (cfg->n_pages < 1) return fail(RAAS_E_INVALID, "n_pages must be >= 1 (got %d)", cfg->n_pages);
    if (cfg->max_batch < 1 || cfg->max_batch > kMaxBatch)
        return fail(RAAS_E_INVALID, "max_batch must lie in [1, %d] (got %d)", kMaxBatch, cfg->max_batch);
    if ((double)cfg->max_batch * cfg->n_kv_heads > kMaxUnits)
        return fail(RAAS_E_INVALID, "max_batch * n_kv_heads must be at most %d (got %d * %d)", kMaxUnits, cfg->max_batch,
                    cfg->n_kv_heads);
    if (cfg->max_queries < 1 || (double)cfg->max_batch * cfg->max_queries * cfg->n_q_heads > kMaxCallRows)
        return fail(RAAS_E_INVALID, "max_queries must be >= 1, and max_batch * max_queries * n_q_heads at most %d (got %d)",
                    kMaxCallRows, cfg->max_queries);
    if ((cfg->key_bits != 4 && cfg->key_bits != 8) || (cfg->value_bits != 4 && cfg->value_bits != 8))
        return fail(RAAS_E_INVALID, "key_bits and value_bits must be 4 or 8 (got %d and %d)", cfg->key_bits,
                    cfg->value_bits);
    const raas_status sb =
        check_bytes(cfg->n_layers, (double)cfg->n_pages * cfg->n_kv_heads, cfg->page_size, cfg->head_dim, true);
    if (sb != RAAS_OK) return sb;
    const raas_status sc = check_creation(stream);
    if (sc != RAAS_OK) return sc;
    raas_quant_cache* c = nullptr;
    try {
        c = new raas_quant_cache();
        c->cfg = *cfg;
        c->streamed_at.assign((size_t)cfg->n_layers, 0);
        c->bf16 = cfg->dtype == RAAS_BF16;
        const hipError_t e = hipGetDevice(&c->device);
        if (e != hipSuccess) {
            delete c;
            return hip_fail(e, "hipGetDevice");
        }
        const size_t blocks = (size_t)cfg->n_pages * cfg->n_kv_heads * (ps / kQuantBlock);
        c->layer_bytes = blocks * quant_record(cfg->head_dim, cfg->key_bits, cfg->value_bits);
        const QuantScratch x =
            quant_scratch(cfg->max_batch, cfg->max_queries, cfg->n_kv_heads, cfg->n_q_heads / cfg->n_kv_heads);
        const std::vector<Req> reqs = {
            {(void**)&c->arrived, x.arrivals * 4, true},
            {(void**)&c->part, x.rows * cfg->head_dim * 4, false},
            {(void**)&c->ml, x.rows * 2 * 4, false},
            {&c->pool, c->layer_bytes * cfg->n_layers, true},  // (a table may name tokens that no call has written)
        };
        raas_status sa = allocate(reqs, &c->memory, c->bytes, (hipStream_t)stream);
        if (sa == RAAS_OK) {  // (the first call may run on another stream)
            const hipError_t w = hipStreamSynchronize((hipStream_t)stream);
            if (w != hipSuccess) sa = hip_fail(w, "hipStreamSynchronize");
        }
        if (sa != RAAS_OK) {
            raas_destroy_quant_cache(c);
            return sa;
        }
    } catch (const std::bad_alloc&) {
        raas_destroy_quant_cache(c);
        return fail(RAAS_E_OOM, "host allocation failed");
    }
    c->last_stream = (hipStream_t)stream;
    *out = c;
    return RAAS_OK;
}

void raas_destroy_quant_cache(raas_quant_cache* c) {
    if (!c) return;
    DeviceScope scope(c->device);
    if (c->memory) {
        (void)hipStreamSynchronize(c->last_stream);
        (void)hipFree(c->memory);
    }
    delete c;
}

size_t raas_quant_cache_bytes(const raas_quant_cache* c) { return c ? c->bytes : 0; }

raas_status raas_quant_write(raas_quant_cache* c, int32_t layer, const void* k, const void* v, const int32_t* table,
                             int32_t table_width, const int32_t* start, const int32_t* counts, int32_t batch,
                             int32_t max_tokens, void* stream) {
    return copy(c, layer, k, v, table, table_width, start, counts, batch, max_tokens, true, stream);
}

raas_status raas_quant_read(raas_quant_cache* c, int32_t layer, void* k, void* v, const int32_t* table,
                            int32_t table_width, const int32_t* start, const int32_t* counts, int32_t batch,
                            int32_t max_tokens, void* stream) {
    return copy(c, layer, k, v, table, table_width, start, counts, batch, max_tokens, false, stream);
}

raas_status raas_quant_attention(raas_quant_cache* c, int32_t layer, const void* q, const int32_t* table,
                                 int32_t table_width, const int32_t* lens, const int32_t* counts, int32_t batch,
                                 int32_t queries, void* out, float* lse, void* stream) {
    QuantView L;
    const raas_status st = view(c, layer, table, table_width, batch, L);
    if (st != RAAS_OK) return st;
    if (queries < 0 || queries > c->cfg.max_queries)
        return fail(RAAS_E_INVALID, "queries must lie in [0, max_queries = %d] (got %d)", c->cfg.max_queries, queries);
    if (batch == 0 || queries == 0) return RAAS_OK;
    if (!q || !lens || !out) return fail(RAAS_E_INVALID, "q, lens and out must be non-NULL");
    DeviceScope scope(c->device);
    if (scope.error() != hipSuccess) return hip_fail(scope.error(), "hipSetDevice");
    QuantAttention io{};
    io.q = q;
    io.out = out;
    io.lse = lse;
    io.len = lens;
    io.count = counts;
    io.queries = queries;
    return attention(c, layer, L, io, 0.0, (hipStream_t)stream);
}

raas_status raas_quant_step(raas_quant_cache* c, int32_t layer, const void* q, const void* k_new, const void* v_new,
                            const int32_t* table, int32_t table_width, const int32_t* lens, int32_t batch, void* out,
                            float* lse, void* k_held, void* v_held, raas_prefix* prefix, void* stream) {
    QuantView L;
    raas_status st = view(c, layer, table, table_width, batch, L);
    if (st != RAAS_OK) return st;
    if (batch == 0) return RAAS_OK;
    if (!q || !k_new || !v_new || !lens || !out)
        return fail(RAAS_E_INVALID, "q, k_new, v_new, lens and out must be non-NULL");
    if (prefix) {
        const raas_quant_config& f = c->cfg;
        st = check_step_prefix(prefix, layer, {f.n_q_heads, f.n_kv_heads, f.head_dim, f.dtype, c->device, batch});
        if (st != RAAS_OK) return st;
    }
    DeviceScope scope(c->device);
    if (scope.error() != hipSuccess) return hip_fail(scope.error(), "hipSetDevice");
    QuantAttention io{};
    io.q = q;
    io.out = out;
    io.lse = lse;
    io.len = lens;
    io.queries = 1;
    io.k_new = k_new;
    io.v_new = v_new;
    io.k_held = k_held;
    io.v_held = v_held;
    double prefix_bytes = 0.0;
    if (prefix) {
        st = step_prefix_parts(prefix, layer, q, batch, io.prefix, prefix_bytes, (hipStream_t)stream);
        if (st != RAAS_OK) return st;
    }
    return attention(c, layer, L, io, prefix_bytes, (hipStream_t)stream);
}

}  // extern "C"
