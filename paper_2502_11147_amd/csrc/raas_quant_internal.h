// Internal interface between the host runtime and the kernels of the quantised
// cache. Not part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "raas_weight_internal.h"

namespace raas {

// Tokens of a block, the unit of storage: pages hold whole blocks.
constexpr int kQuantBlock = 32;
// Channels that share a power of two.
constexpr int kQuantGroup = 32;

// Bytes of a block's record: codes of keys and values, exponents of both.
constexpr size_t quant_record(int D, int key_bits, int value_bits) {
    return (size_t)kQuantBlock * (D * (key_bits + value_bits) / 8 + 2 * D / kQuantGroup);
}

// One layer of the cache and the sequences of a call.
struct QuantView {
    uint8_t* pool;         // [n_pages][nkv][blocks of a page] records (raas_quant_blocks.h)
    const int32_t* table;  // [batch][width] page of a sequence's tokens page_size * i ..
    int batch, width, n_pages, nkv, G, D, key_bits, value_bits;
    int page_shift;        // log2 of a page's blocks
    int cap;               // tokens of a table's row: width << page_shift blocks
};

// Tokens start[b] .. start[b] + count[b] - 1 of each sequence, from or to rows 0 .. of k, v.
struct QuantCopy {
    void* k;  // [batch][nkv][stride][D]
    void* v;
    const int32_t* start;
    const int32_t* count;  // NULL: stride
    int stride;
};
hipError_t launch_quant_write(const QuantView& L, bool bf16, const QuantCopy& io, hipStream_t s);
hipError_t launch_quant_read(const QuantView& L, bool bf16, const QuantCopy& io, hipStream_t s);

// Attention of the last count[b] of len[b] tokens' queries. A step (k_new given)
// stores the token at position len[b] first and attends to it too.
struct QuantAttention {
    const void* q;         // [batch][queries][nkv * G][D]
    void* out;             // likewise
    float* lse;            // [batch][queries][nkv * G], or NULL
    const int32_t* len;    // [batch], < 0: the sequence sits out
    const int32_t* count;  // [batch], or NULL: `queries`
    int queries;
    const void* k_new;     // [batch][nkv][D], or NULL: no step
    const void* v_new;
    void* k_held;          // [batch][nkv][D], or NULL: the new token as it is held
    void* v_held;
    PrefixParts prefix;    // n = 0: none (a step's only)
    float scale_log2;
    // scratch: unnormalised outputs, maxima (base 2) and sums of tiles that are
    // split, a slot of a tile's rows per workgroup; arrivals per unit, zero between launches
    float* part;
    float* ml;
    int32_t* arrived;
};

// Most workgroups that a tile of a unit's rows is split over.
constexpr int kMaxQuantParts = 64;
// Scratch of calls of up to `batch` sequences of up to `queries` queries.
struct QuantScratch {
    size_t rows;      // of part and ml
    size_t arrivals;  // of arrived
};
QuantScratch quant_scratch(int batch, int queries, int nkv, int G);
size_t quant_wide_scratch_rows(int batch, int queries, int nkv, int G);
// stream: codes are read with non-temporal loads
hipError_t launch_quant_attention(const QuantView& L, bool bf16, const QuantAttention& io, bool stream, hipStream_t s);
// Its kernels for many rows per unit.
hipError_t launch_quant_wide(const QuantView& L, bool bf16, const QuantAttention& io, hipStream_t s);

}  // namespace raas
