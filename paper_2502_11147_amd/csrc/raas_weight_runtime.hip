// Host runtime of the weight cache, the shared prefix and the prompt weights:
// argument checks, their memory, and the launches on the caller's stream.
// Implements the second half of include/raas.h.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <vector>

#include "raas.h"
#include "raas_host.h"
#include "raas_weight_internal.h"

using namespace raas;

namespace {

// Tokens that a unit of a cache, a prefix or a prompt may have.
constexpr int kMaxTokens = 1 << 20;
// Query rows of one call over a prefix, and of one KV head's window (the grids' limits).
constexpr int kMaxQueries = 1 << 17, kMaxWindowRows = 1 << 23;

// The handle's device for the length of a call.
class DeviceScope {
  public:
    explicit DeviceScope(int device) {
        if (hipGetDevice(&before_) != hipSuccess) before_ = -1;
        if (before_ != device) error_ = hipSetDevice(device);
        else before_ = -1;
    }
    ~DeviceScope() {
        if (before_ >= 0) (void)hipSetDevice(before_);
    }
    DeviceScope(const DeviceScope&) = delete;
    DeviceScope& operator=(const DeviceScope&) = delete;
    hipError_t error() const { return error_; }

  private:
    int before_ = -1;
    hipError_t error_ = hipSuccess;
};

float scale_log2(int d) { return (float)(1.4426950408889634 / sqrt((double)d)); }
int block_tokens(bool bf16) { return bf16 ? 32 : 16; }
int pad_tokens(int n, bool bf16) { return (n + block_tokens(bf16) - 1) / block_tokens(bf16) * block_tokens(bf16); }

// The layer's shape, as every one of these calls takes it.
raas_status check_heads(int n_q_heads, int n_kv_heads, int head_dim, int dtype) {
    if (n_kv_heads < 1 || n_kv_heads > 65535)
        return fail(RAAS_E_INVALID, "n_kv_heads must lie in [1, 65535] (got %d)", n_kv_heads);
    if (n_q_heads < 1 || n_q_heads % n_kv_heads != 0)
        return fail(RAAS_E_INVALID, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", n_q_heads,
                    n_kv_heads);
    if (n_q_heads / n_kv_heads > 16)
        return fail(RAAS_E_INVALID, "query group n_q_heads/n_kv_heads = %d exceeds 16", n_q_heads / n_kv_heads);
    if (head_dim != 64 && head_dim != 128) return fail(RAAS_E_INVALID, "head_dim must be 64 or 128 (got %d)", head_dim);
    if (dtype != RAAS_F32 && dtype != RAAS_BF16)
        return fail(RAAS_E_INVALID, "dtype must be RAAS_F32 or RAAS_BF16 (got %d)", dtype);
    return RAAS_OK;
}

// Bytes that no device has; sizes below it do not overflow.
constexpr double kNoDevice = 1e17;
raas_status check_bytes(double layers, double units, double tokens, int head_dim, bool bf16) {
    const double bytes = 2.0 * layers * units * tokens * head_dim * (bf16 ? 2 : 4);
    if (bytes > kNoDevice) return fail(RAAS_E_OOM, "keys and values of %.3g bytes fit no device", bytes);
    return RAAS_OK;
}

// A captured creation would clear its records only when the graph runs.
raas_status check_creation(void* stream) {
    if (capturing((hipStream_t)stream))
        return fail(RAAS_E_STATE, "a handle cannot be created on a stream that is being captured");
    return RAAS_OK;
}

// A part of a handle's memory; `clear`: it starts at zero.
struct Req {
    void** ptr;
    size_t bytes;
    bool clear;
};

// One allocation, cut into parts of 256 bytes and up (an allocation takes some
// 30 us); what must start at zero is cleared on the stream. Keys, values and
// scratch need not: no place is looked at before it is written, but for the rest
// of a block, whose logits and values are masked.
raas_status allocate(const std::vector<Req>& reqs, void** base, size_t& total, hipStream_t s) {
    auto padded = [](size_t n) { return (n + 255) & ~(size_t)255; };
    total = 0;
    for (const Req& r : reqs) total += padded(r.bytes);
    hipError_t e = hipMalloc(base, total);
    if (e != hipSuccess) {
        *base = nullptr;
        (void)hipGetLastError();
        return fail(e == hipErrorOutOfMemory ? RAAS_E_OOM : RAAS_E_HIP, "hipMalloc(%zu bytes): %s", total,
                    hipGetErrorString(e));
    }
    char* at = (char*)*base;
    for (const Req& r : reqs) {
        *r.ptr = at;
        at += padded(r.bytes);
        if (!r.clear) continue;
        e = hipMemsetAsync(*r.ptr, 0, r.bytes, s);
        if (e != hipSuccess) return hip_fail(e, "hipMemsetAsync");
    }
    return RAAS_OK;
}

// Lengths of sequences seq0 .. of a launch: lens (NULL: max_len), -1 where the mask leaves one out.
int fill_lens(SeqLens& out, const int32_t* lens, const int32_t* mask, int max_len, int seq0, int nseq) {
    int selected = 0;
    for (int i = 0; i < nseq; ++i) {
        const bool on = !mask || mask[seq0 + i];
        out.len[i] = on ? (lens ? lens[seq0 + i] : max_len) : -1;
        selected += on;
    }
    return selected;
}

}  // namespace

struct raas_weight_cache {
    raas_weight_config cfg;
    int U, G, C, cpad, device;
    bool bf16;
    WeightPlan plan;
    void *memory = nullptr, *K = nullptr, *V = nullptr;
    int32_t *pos = nullptr, *unit = nullptr, *arrived = nullptr;
    unsigned long long* best = nullptr;
    float *w = nullptr, *logits = nullptr, *part = nullptr, *ml = nullptr;
    size_t bytes = 0;
    std::vector<unsigned char> prefilled;
    std::vector<unsigned long long> streamed_at;  // count_streamed after each layer's last step; 0: no step yet
    hipStream_t last_stream = nullptr;
};

struct raas_prefix {
    raas_prefix_config cfg;
    int G, tpad, rows, device;
    bool bf16;
    void *memory = nullptr, *K = nullptr, *V = nullptr;
    int32_t* len = nullptr;  // [layers]
    float *part = nullptr, *ml = nullptr;
    size_t bytes = 0;
    std::vector<int> stored;  // tokens of each layer, -1 before the first store
    hipStream_t last_stream = nullptr;
};

namespace {

WeightView view(const raas_weight_cache* c, int layer) {
    WeightView L{};
    const size_t kv = (size_t)layer * c->U * c->cpad * c->cfg.head_dim * (c->bf16 ? 2 : 4);
    L.K = (char*)c->K + kv;
    L.V = (char*)c->V + kv;
    L.pos = c->pos + (size_t)layer * c->U * c->cpad;
    L.w = c->w + (size_t)layer * c->U * c->cpad;
    L.unit = c->unit + (size_t)layer * c->U * kWeightFields;
    L.logits = c->logits;
    L.part = c->part;
    L.ml = c->ml;
    L.arrived = c->arrived;
    L.best = c->best;
    L.U = c->U;
    L.G = c->G;
    L.D = c->cfg.head_dim;
    L.C = c->C;
    L.cpad = c->cpad;
    L.nkv = c->cfg.n_kv_heads;
    L.recent = c->cfg.recent;
    L.nsplit = c->plan.nsplit;
    L.scale_log2 = scale_log2(L.D);
    return L;
}

raas_status check_layer(const raas_weight_cache* c, int32_t layer) {
    if (!c) return fail(RAAS_E_INVALID, "cache is NULL");
    if (layer < 0 || layer >= c->cfg.n_layers)
        return fail(RAAS_E_INVALID, "layer %d out of range [0, %d)", layer, c->cfg.n_layers);
    return RAAS_OK;
}

raas_status check_layer(const raas_prefix* p, int32_t layer) {
    if (!p) return fail(RAAS_E_INVALID, "prefix is NULL");
    if (layer < 0 || layer >= p->cfg.n_layers)
        return fail(RAAS_E_INVALID, "layer %d out of range [0, %d)", layer, p->cfg.n_layers);
    return RAAS_OK;
}

// Whether a step reads its layer of `own` bytes with non-temporal loads, which
// leave the memory-side cache (256 MB) alone: where too little of the layer is
// still there (us per step, ordinary / non-temporal: 268 MB alone 47.1 / 48.7,
// in turn with two more caches of that size 58.3 / 52.9; 134 MB 38.0 / 41.8 and
// 45.8 / 43.4; 67 MB 21.7 / 22.9 and 21.8 / 23.8; 403 MB alone 84.4 / 70.5; with a
// prefix in front, its attention included: 268 MB and a prefix of 134 MB 100.0 /
// 90.5, 67 MB and 268 MB 85.0 / 79.6).
bool non_temporal(double own, double others) { return others + own * 2.0 / 3.0 > 256e6; }

// Bytes of keys and values that attention over a layer of the prefix reads.
double prefix_bytes(const raas_prefix* p, int32_t layer) {
    return 2.0 * p->cfg.n_kv_heads * pad_tokens(p->stored[layer], p->bf16) * p->cfg.head_dim * (p->bf16 ? 2 : 4);
}

// The prefix's attention of `rows` sequences' queries into its parts.
raas_status prefix_parts(raas_prefix* p, int32_t layer, const void* q, int rows, PrefixView& P, hipStream_t s) {
    const size_t kv = (size_t)layer * p->cfg.n_kv_heads * p->tpad * p->cfg.head_dim * (p->bf16 ? 2 : 4);
    P = PrefixView{};
    P.K = (char*)p->K + kv;
    P.V = (char*)p->V + kv;
    P.len = p->len + layer;
    P.part = p->part;
    P.ml = p->ml;
    P.nkv = p->cfg.n_kv_heads;
    P.G = p->G;
    P.D = p->cfg.head_dim;
    P.tpad = p->tpad;
    P.rows = rows * p->G;
    P.nsplit = plan_prefix(P.nkv, P.rows, p->stored[layer], p->bf16);
    P.scale_log2 = scale_log2(P.D);
    const hipError_t e = launch_prefix_attention(P, p->bf16, q, s);
    if (e != hipSuccess) return hip_fail(e, "prefix attention launch");
    if (!capturing(s)) count_streamed(p->device, (unsigned long long)prefix_bytes(p, layer));
    p->last_stream = s;
    return RAAS_OK;
}

// A launch of the prompt weights: its sequences, its plan, the floats of its scratch.
struct PromptSpace {
    int nseq;
    PromptPlan plan;
    size_t stat, ml, part;
};
PromptSpace prompt_space(int batch, int n_q_heads, int n_kv_heads, int max_len, int window, bool bf16) {
    PromptSpace sp;
    sp.nseq = std::min({batch, kLenSeqs, std::max(1, 65535 / n_kv_heads)});
    const int W = std::min(window, max_len);
    sp.plan = plan_prompt(sp.nseq * n_kv_heads, n_q_heads / n_kv_heads, W, max_len, bf16);
    sp.stat = (size_t)sp.nseq * n_q_heads * W * 2;
    sp.ml = sp.plan.chunks > 1 ? sp.stat * sp.plan.chunks : 0;
    sp.part = sp.plan.row_chunks > 1 ? (size_t)sp.plan.row_chunks * sp.nseq * n_kv_heads * max_len : 0;
    return sp;
}

// The sizes that a call of the prompt weights may have.
raas_status check_prompt(int batch, int n_q_heads, int n_kv_heads, int head_dim, int dtype, int max_len, int window) {
    if (batch < 1) return fail(RAAS_E_INVALID, "batch must be >= 1 (got %d)", batch);
    const raas_status st = check_heads(n_q_heads, n_kv_heads, head_dim, dtype);
    if (st != RAAS_OK) return st;
    if (max_len < 0 || max_len > kMaxTokens)
        return fail(RAAS_E_INVALID, "max_len must lie in [0, %d] (got %d)", kMaxTokens, max_len);
    if (window < 1 || window > std::max(1, max_len))
        return fail(RAAS_E_INVALID, "window must lie in [1, max_len = %d] (got %d)", max_len, window);
    if ((long long)window * (n_q_heads / n_kv_heads) > kMaxWindowRows)
        return fail(RAAS_E_INVALID, "window * n_q_heads / n_kv_heads must be at most %d", kMaxWindowRows);
    return RAAS_OK;
}

}  // namespace

extern "C" {

raas_status raas_create_weight_cache(const raas_weight_config* cfg, void* stream, raas_weight_cache** out) {
    if (!out) return fail(RAAS_E_INVALID, "out is NULL");
    if (!cfg) return fail(RAAS_E_INVALID, "cfg is NULL");
    if (cfg->batch < 1) return fail(RAAS_E_INVALID, "batch must be >= 1 (got %d)", cfg->batch);
    if (cfg->n_layers < 1) return fail(RAAS_E_INVALID, "n_layers must be >= 1 (got %d)", cfg->n_layers);
    const raas_status st = check_heads(cfg->n_q_heads, cfg->n_kv_heads, cfg->head_dim, cfg->dtype);
    if (st != RAAS_OK) return st;
    if (cfg->capacity < 2 || cfg->capacity > kMaxTokens)
        return fail(RAAS_E_INVALID, "capacity must lie in [2, %d] (got %d)", kMaxTokens, cfg->capacity);
    if (cfg->recent < 0 || cfg->recent >= cfg->capacity)
        return fail(RAAS_E_INVALID, "recent must lie in [0, capacity) (got %d)", cfg->recent);
    if ((double)cfg->batch * cfg->n_kv_heads > 1e6) return fail(RAAS_E_INVALID, "batch * n_kv_heads too large");
    const raas_status sb = check_bytes(cfg->n_layers, (double)cfg->batch * cfg->n_kv_heads, cfg->capacity, cfg->head_dim,
                                       cfg->dtype == RAAS_BF16);
    if (sb != RAAS_OK) return sb;
    const raas_status sc = check_creation(stream);
    if (sc != RAAS_OK) return sc;
    raas_weight_cache* c = nullptr;
    try {
        c = new raas_weight_cache();
        c->prefilled.assign((size_t)cfg->n_layers, 0);
        c->streamed_at.assign((size_t)cfg->n_layers, 0);
        c->cfg = *cfg;
        c->bf16 = cfg->dtype == RAAS_BF16;
        c->U = cfg->batch * cfg->n_kv_heads;
        c->G = cfg->n_q_heads / cfg->n_kv_heads;
        c->C = cfg->capacity;
        c->cpad = pad_tokens(cfg->capacity, c->bf16);
        const size_t Ly = (size_t)cfg->n_layers, U = (size_t)c->U, d = (size_t)cfg->head_dim, esz = c->bf16 ? 2 : 4;
        c->plan = plan_weight_step(c->U, c->G, cfg->head_dim, c->C, c->bf16);
        hipError_t e = hipGetDevice(&c->device);
        if (e == hipSuccess) e = weight_allow_lds(c->bf16, cfg->head_dim, c->plan.waves);
        if (e != hipSuccess) {
            delete c;
            return hip_fail(e, "hipFuncSetAttribute");
        }
        const bool split = !c->plan.fused;
        const size_t parts = split ? U * c->plan.nsplit * c->G : 1;
        const std::vector<Req> reqs = {
            {(void**)&c->pos, Ly * U * c->cpad * 4, true},
            {(void**)&c->w, Ly * U * c->cpad * 4, true},
            {(void**)&c->unit, Ly * U * kWeightFields * 4, true},
            {(void**)&c->arrived, U * 4, true},
            {(void**)&c->best, c->plan.finish_parts > 0 ? U * c->plan.finish_parts * 16 : 16, false},
            {(void**)&c->logits, split ? U * c->G * c->cpad * 4 : 4, false},
            {(void**)&c->part, parts * d * 4, false},
            {(void**)&c->ml, parts * 2 * 4, false},
            {&c->K, Ly * U * c->cpad * d * esz, false},
            {&c->V, Ly * U * c->cpad * d * esz, false},
        };
        const raas_status sa = allocate(reqs, &c->memory, c->bytes, (hipStream_t)stream);
        if (sa != RAAS_OK) {
            raas_destroy_weight_cache(c);
            return sa;
        }
    } catch (const std::bad_alloc&) {
        raas_destroy_weight_cache(c);
        return fail(RAAS_E_OOM, "host allocation failed");
    }
    c->last_stream = (hipStream_t)stream;
    *out = c;
    return RAAS_OK;
}

void raas_destroy_weight_cache(raas_weight_cache* c) {
    if (!c) return;
    DeviceScope scope(c->device);
    if (c->memory) {
        (void)hipStreamSynchronize(c->last_stream);
        (void)hipFree(c->memory);
    }
    delete c;
}

size_t raas_weight_cache_bytes(const raas_weight_cache* c) { return c ? c->bytes : 0; }

raas_status raas_weight_prefill(raas_weight_cache* c, int32_t layer, const void* k, const void* v,
                                const float* weights, const int32_t* lens, const int32_t* seq_mask, int32_t max_len,
                                void* stream) {
    raas_status st = check_layer(c, layer);
    if (st != RAAS_OK) return st;
    if (max_len < 0 || max_len > kMaxTokens)
        return fail(RAAS_E_INVALID, "max_len must lie in [0, %d] (got %d)", kMaxTokens, max_len);
    const int B = c->cfg.batch;
    int selected = 0;
    bool any = false;
    for (int b = 0; b < B; ++b) {
        if (seq_mask && !seq_mask[b]) continue;
        const int len = lens ? lens[b] : max_len;
        if (len < 0 || len > max_len)
            return fail(RAAS_E_INVALID, "lens[%d] = %d outside [0, max_len = %d]", b, len, max_len);
        selected += 1;
        any = any || len > 0;
    }
    if (any && (!k || !v)) return fail(RAAS_E_INVALID, "k or v is NULL");
    if (!c->prefilled[layer] && selected != B)
        return fail(RAAS_E_STATE, "the first prefill of layer %d must cover every sequence", layer);
    DeviceScope scope(c->device);
    if (scope.error() != hipSuccess) return hip_fail(scope.error(), "hipSetDevice");
    const WeightView L = view(c, layer);
    hipStream_t s = (hipStream_t)stream;
    for (int b = 0; b < B; b += kLenSeqs) {
        SeqLens sl{};
        const int n = std::min(kLenSeqs, B - b);
        if (fill_lens(sl, lens, seq_mask, max_len, b, n) == 0) continue;
        const hipError_t e = launch_weight_prefill(L, c->bf16, k, v, weights, sl, b, n, max_len, s);
        if (e != hipSuccess) return hip_fail(e, "prefill launch");
    }
    c->prefilled[layer] = 1;
    c->last_stream = s;
    return RAAS_OK;
}

raas_status raas_weight_step(raas_weight_cache* c, int32_t layer, const void* q, const void* k_new, const void* v_new,
                             void* out, int32_t* positions_out, float* weights_out, int32_t* evicted_out,
                             const int32_t* active, raas_prefix* prefix, void* stream) {
    raas_status st = check_layer(c, layer);
    if (st != RAAS_OK) return st;
    if (!q || !k_new || !v_new || !out) return fail(RAAS_E_INVALID, "q, k_new, v_new and out must be non-NULL");
    if (!c->prefilled[layer]) return fail(RAAS_E_STATE, "layer %d has not been prefilled", layer);
    if (prefix) {
        const raas_prefix_config& f = prefix->cfg;
        if (f.n_q_heads != c->cfg.n_q_heads || f.n_kv_heads != c->cfg.n_kv_heads || f.head_dim != c->cfg.head_dim ||
            f.dtype != c->cfg.dtype)
            return fail(RAAS_E_INVALID, "the prefix has other heads or another type than the cache");
        if (prefix->device != c->device) return fail(RAAS_E_INVALID, "the prefix lies on another device");
        if (layer >= f.n_layers) return fail(RAAS_E_INVALID, "the prefix has no layer %d", layer);
        if (prefix->stored[layer] < 0) return fail(RAAS_E_STATE, "layer %d of the prefix has not been stored", layer);
        if (c->cfg.batch > f.max_rows)
            return fail(RAAS_E_INVALID, "batch %d exceeds the prefix's max_rows %d", c->cfg.batch, f.max_rows);
    }
    DeviceScope scope(c->device);
    if (scope.error() != hipSuccess) return hip_fail(scope.error(), "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;
    WeightStepIO io{q, k_new, v_new, out, positions_out, weights_out, evicted_out, active, PrefixParts{}};
    if (prefix) {
        PrefixView P;
        st = prefix_parts(prefix, layer, q, c->cfg.batch, P, s);
        if (st != RAAS_OK) return st;
        io.prefix = PrefixParts{P.part, P.ml, P.nsplit, P.rows};
    }
    // What other layers, caches and pools have read since the layer's last step
    // decides whether it is still in the memory-side cache; a captured step, whose
    // replays are not seen here, counts the cache's other layers, and the prefix
    // as if each of them had one of this length.
    const double own = 2.0 * c->U * c->cpad * c->cfg.head_dim * (c->bf16 ? 2 : 4);
    const bool captured = capturing(s);
    double others = (c->cfg.n_layers - 1.0) * own + (prefix ? c->cfg.n_layers * prefix_bytes(prefix, layer) : 0.0);
    if (!captured) {
        const unsigned long long before = count_streamed(c->device, (unsigned long long)own);
        if (c->streamed_at[layer] != 0) others = (double)(before - c->streamed_at[layer]);
        c->streamed_at[layer] = before + (unsigned long long)own;
    }
    const hipError_t e =
        launch_weight_step(view(c, layer), c->bf16, io, c->plan, non_temporal(own, others), s);
    if (e != hipSuccess) return hip_fail(e, "step launch");
    c->last_stream = s;
    return RAAS_OK;
}

raas_status raas_weight_export_state(raas_weight_cache* c, int32_t layer, int32_t* positions, float* weights,
                                     int32_t* clocks, void* stream) {
    raas_status st = check_layer(c, layer);
    if (st != RAAS_OK) return st;
    if (!positions || !weights || !clocks) return fail(RAAS_E_INVALID, "positions, weights and clocks must be non-NULL");
    DeviceScope scope(c->device);
    if (scope.error() != hipSuccess) return hip_fail(scope.error(), "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;
    const WeightView L = view(c, layer);
    const size_t row = (size_t)c->C * 4, pitch = (size_t)c->cpad * 4;
    std::vector<int32_t> unit;
    try {
        unit.resize((size_t)c->U * kWeightFields);
    } catch (const std::bad_alloc&) {
        return fail(RAAS_E_OOM, "host allocation failed");
    }
    hipError_t e = hipMemcpy2DAsync(positions, row, L.pos, pitch, row, (size_t)c->U, hipMemcpyDeviceToHost, s);
    if (e == hipSuccess)
        e = hipMemcpy2DAsync(weights, row, L.w, pitch, row, (size_t)c->U, hipMemcpyDeviceToHost, s);
    if (e == hipSuccess) e = hipMemcpyAsync(unit.data(), L.unit, unit.size() * 4, hipMemcpyDeviceToHost, s);
    if (e != hipSuccess) return hip_fail(e, "hipMemcpyAsync");
    e = hipStreamSynchronize(s);
    if (e != hipSuccess) return hip_fail(e, "hipStreamSynchronize");
    for (int u = 0; u < c->U; ++u) {
        const int count = unit[(size_t)u * kWeightFields + kCount];
        for (size_t j = (size_t)u * c->C + count; j < (size_t)(u + 1) * c->C; ++j) {
            positions[j] = -1;
            weights[j] = 0.0f;
        }
        clocks[u] = unit[(size_t)u * kWeightFields + kNow];
    }
    return RAAS_OK;
}

raas_status raas_create_prefix(const raas_prefix_config* cfg, void* stream, raas_prefix** out) {
    if (!out) return fail(RAAS_E_INVALID, "out is NULL");
    if (!cfg) return fail(RAAS_E_INVALID, "cfg is NULL");
    if (cfg->n_layers < 1) return fail(RAAS_E_INVALID, "n_layers must be >= 1 (got %d)", cfg->n_layers);
    const raas_status st = check_heads(cfg->n_q_heads, cfg->n_kv_heads, cfg->head_dim, cfg->dtype);
    if (st != RAAS_OK) return st;
    if (cfg->max_tokens < 1 || cfg->max_tokens > kMaxTokens)
        return fail(RAAS_E_INVALID, "max_tokens must lie in [1, %d] (got %d)", kMaxTokens, cfg->max_tokens);
    if (cfg->max_rows < 1 || (double)cfg->max_rows * cfg->n_q_heads > kMaxQueries)
        return fail(RAAS_E_INVALID, "max_rows must be >= 1, and max_rows * n_q_heads at most %d (got %d rows)", kMaxQueries,
                    cfg->max_rows);
    const raas_status sb =
        check_bytes(cfg->n_layers, cfg->n_kv_heads, cfg->max_tokens, cfg->head_dim, cfg->dtype == RAAS_BF16);
    if (sb != RAAS_OK) return sb;
    const raas_status sc = check_creation(stream);
    if (sc != RAAS_OK) return sc;
    raas_prefix* p = nullptr;
    try {
        p = new raas_prefix();
        p->stored.assign((size_t)cfg->n_layers, -1);
        p->cfg = *cfg;
        p->bf16 = cfg->dtype == RAAS_BF16;
        p->G = cfg->n_q_heads / cfg->n_kv_heads;
        p->tpad = pad_tokens(cfg->max_tokens, p->bf16);
        const hipError_t e = hipGetDevice(&p->device);
        if (e != hipSuccess) {
            delete p;
            return hip_fail(e, "hipGetDevice");
        }
        const size_t Ly = (size_t)cfg->n_layers, d = (size_t)cfg->head_dim, esz = p->bf16 ? 2 : 4;
        const size_t parts = prefix_scratch_rows(cfg->n_kv_heads, cfg->max_rows * p->G);
        const std::vector<Req> reqs = {
            {(void**)&p->len, Ly * 4, true},
            {(void**)&p->part, parts * d * 4, false},
            {(void**)&p->ml, parts * 2 * 4, false},
            {&p->K, Ly * cfg->n_kv_heads * p->tpad * d * esz, false},
            {&p->V, Ly * cfg->n_kv_heads * p->tpad * d * esz, false},
        };
        const raas_status sa = allocate(reqs, &p->memory, p->bytes, (hipStream_t)stream);
        if (sa != RAAS_OK) {
            raas_destroy_prefix(p);
            return sa;
        }
    } catch (const std::bad_alloc&) {
        raas_destroy_prefix(p);
        return fail(RAAS_E_OOM, "host allocation failed");
    }
    p->last_stream = (hipStream_t)stream;
    *out = p;
    return RAAS_OK;
}

void raas_destroy_prefix(raas_prefix* p) {
    if (!p) return;
    DeviceScope scope(p->device);
    if (p->memory) {
        (void)hipStreamSynchronize(p->last_stream);
        (void)hipFree(p->memory);
    }
    delete p;
}

size_t raas_prefix_bytes(const raas_prefix* p) { return p ? p->bytes : 0; }

raas_status raas_prefix_store(raas_prefix* p, int32_t layer, const void* k, const void* v, int32_t tokens,
                              void* stream) {
    const raas_status st = check_layer(p, layer);
    if (st != RAAS_OK) return st;
    if (tokens < 0 || tokens > p->cfg.max_tokens)
        return fail(RAAS_E_INVALID, "tokens must lie in [0, max_tokens = %d] (got %d)", p->cfg.max_tokens, tokens);
    if (tokens > 0 && (!k || !v)) return fail(RAAS_E_INVALID, "k or v is NULL");
    DeviceScope scope(p->device);
    if (scope.error() != hipSuccess) return hip_fail(scope.error(), "hipSetDevice");
    const size_t kv = (size_t)layer * p->cfg.n_kv_heads * p->tpad * p->cfg.head_dim * (p->bf16 ? 2 : 4);
    hipStream_t s = (hipStream_t)stream;
    const hipError_t e = launch_prefix_store((char*)p->K + kv, (char*)p->V + kv, p->len + layer, p->cfg.n_kv_heads,
                                             p->cfg.head_dim, p->tpad, p->bf16, k, v, tokens, s);
    if (e != hipSuccess) return hip_fail(e, "prefix store launch");
    p->stored[layer] = tokens;
    p->last_stream = s;
    return RAAS_OK;
}

raas_status raas_prefix_attention(raas_prefix* p, int32_t layer, const void* q, int32_t rows, void* out, float* lse,
                                  void* stream) {
    raas_status st = check_layer(p, layer);
    if (st != RAAS_OK) return st;
    if (rows < 0 || rows > p->cfg.max_rows)
        return fail(RAAS_E_INVALID, "rows must lie in [0, max_rows = %d] (got %d)", p->cfg.max_rows, rows);
    if (p->stored[layer] < 0) return fail(RAAS_E_STATE, "layer %d has not been stored", layer);
    if (rows == 0) return RAAS_OK;
    if (!q || !out) return fail(RAAS_E_INVALID, "q and out must be non-NULL");
    DeviceScope scope(p->device);
    if (scope.error() != hipSuccess) return hip_fail(scope.error(), "hipSetDevice");
    PrefixView P;
    st = prefix_parts(p, layer, q, rows, P, (hipStream_t)stream);
    if (st != RAAS_OK) return st;
    const hipError_t e = launch_prefix_join(P, p->bf16, out, lse, (hipStream_t)stream);
    if (e != hipSuccess) return hip_fail(e, "prefix join launch");
    return RAAS_OK;
}

size_t raas_prompt_weights_workspace(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t max_len,
                                     int32_t window) {
    if (check_prompt(batch, n_q_heads, n_kv_heads, 64, RAAS_F32, max_len, window) != RAAS_OK || max_len == 0) return 0;
    size_t most = 0;  // over both types, which are cut differently
    for (bool bf16 : {false, true}) {
        const PromptSpace sp = prompt_space(batch, n_q_heads, n_kv_heads, max_len, window, bf16);
        most = std::max(most, sp.stat + sp.ml + sp.part);
    }
    return most * sizeof(float);
}

raas_status raas_prompt_weights(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                                const void* q, const void* k, const float* prefix_lse, const int32_t* lens,
                                int32_t max_len, int32_t window, float* weights, void* workspace,
                                size_t workspace_bytes, void* stream) {
    const raas_status st = check_prompt(batch, n_q_heads, n_kv_heads, head_dim, dtype, max_len, window);
    if (st != RAAS_OK) return st;
    for (int b = 0; b < batch && lens; ++b)
        if (lens[b] < 0 || lens[b] > max_len)
            return fail(RAAS_E_INVALID, "lens[%d] = %d outside [0, max_len = %d]", b, lens[b], max_len);
    if (max_len == 0) return RAAS_OK;
    if (!q || !k || !weights) return fail(RAAS_E_INVALID, "q, k and weights must be non-NULL");
    const size_t need = raas_prompt_weights_workspace(batch, n_q_heads, n_kv_heads, max_len, window);
    if (!workspace || workspace_bytes < need)
        return fail(RAAS_E_INVALID, "workspace must hold %zu bytes (got %zu)", need, workspace ? workspace_bytes : 0);
    const PromptSpace sp = prompt_space(batch, n_q_heads, n_kv_heads, max_len, window, dtype == RAAS_BF16);
    PromptView v{};
    static_cast<PromptPlan&>(v) = sp.plan;
    v.q = q;
    v.k = k;
    v.prefix_lse = prefix_lse;
    v.weights = weights;
    v.stat = (float*)workspace;
    v.ml = v.stat + sp.stat;
    v.part = v.ml + sp.ml;
    v.W = window;
    v.P = max_len;
    v.G = n_q_heads / n_kv_heads;
    v.D = head_dim;
    v.nkv = n_kv_heads;
    v.g_magic = v.G > 1 ? (uint32_t)(((1ull << 32) + v.G - 1) / v.G) : 0;
    v.scale_log2 = scale_log2(head_dim);
    for (int b = 0; b < batch; b += sp.nseq) {
        SeqLens sl{};
        v.seq0 = b;
        v.nseq = std::min(sp.nseq, batch - b);
        fill_lens(sl, lens, nullptr, max_len, b, v.nseq);
        const hipError_t e = launch_prompt_weights(v, dtype == RAAS_BF16, sl, (hipStream_t)stream);
        if (e != hipSuccess) return hip_fail(e, "prompt weights launch");
    }
    return RAAS_OK;
}

}  // extern "C"
