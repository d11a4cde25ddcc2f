// What the handles of the weight cache, the shared prefix and the quantised cache
// have in common on the host: their device, their memory, the checks of a
// layer's shape. Not part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>

#include <vector>

#include "raas.h"
#include "raas_host.h"

namespace raas {

// Tokens that a unit of a cache, a prefix or a prompt may have.
constexpr int kMaxTokens = 1 << 20;

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

inline float scale_log2(int d) { return (float)(1.4426950408889634 / sqrt((double)d)); }
inline int block_tokens(bool bf16) { return bf16 ? 32 : 16; }
inline int pad_tokens(int n, bool bf16) { return (n + block_tokens(bf16) - 1) / block_tokens(bf16) * block_tokens(bf16); }

// The layer's shape, as every one of these calls takes it.
inline raas_status check_heads(int n_q_heads, int n_kv_heads, int head_dim, int dtype) {
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
inline raas_status check_bytes(double layers, double units, double tokens, int head_dim, bool bf16) {
    const double bytes = 2.0 * layers * units * tokens * head_dim * (bf16 ? 2 : 4);
    if (bytes > kNoDevice) return fail(RAAS_E_OOM, "keys and values of %.3g bytes fit no device", bytes);
    return RAAS_OK;
}

// A captured creation would clear its records only when the graph runs.
inline raas_status check_creation(void* stream) {
    if (capturing((hipStream_t)stream))
        return fail(RAAS_E_STATE, "a handle cannot be created on a stream that is being captured");
    return RAAS_OK;
}

// Whether a step reads its layer of `own` bytes with non-temporal loads, which
// leave the memory-side cache (256 MB) alone: where too little of the layer is
// still there (us per step, ordinary / non-temporal: 268 MB alone 47.1 / 48.7,
// in turn with two more caches of that size 58.3 / 52.9; 134 MB 38.0 / 41.8 and
// 45.8 / 43.4; 67 MB 21.7 / 22.9 and 21.8 / 23.8; 403 MB alone 84.4 / 70.5; with a
// prefix in front, its attention included: 268 MB and a prefix of 134 MB 100.0 /
// 90.5, 67 MB and 268 MB 85.0 / 79.6).
inline bool non_temporal(double own, double others) { return others + own * 2.0 / 3.0 > 256e6; }

// A part of a handle's memory; `clear`: it starts at zero.
struct Req {
    void** ptr;
    size_t bytes;
    bool clear;
};

// One allocation, cut into parts of 256 bytes and up (an allocation takes some
// 30 us); what must start at zero is cleared on the stream. Scratch, and keys and
// values of a weight cache or a prefix, need not: no place is looked at before it is
// written, but for the rest of a block, whose logits and values are masked.
inline raas_status allocate(const std::vector<Req>& reqs, void** base, size_t& total, hipStream_t s) {
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

}  // namespace raas
