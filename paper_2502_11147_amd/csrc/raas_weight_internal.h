// Internal interface between the host runtime and the kernels of the weight
// cache, the shared prefix and the prompt weights. Not part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "raas.h"

namespace raas {

// Per-unit record of a weight cache:
//  count   tokens held (places 0 .. count-1)
//  clock   absolute position of the next token
//  place   place the next token takes: the first free one, or the lightest token's
//  victim  position of the token that it displaces, or -1
enum WeightField : int { kCount = 0, kNow = 1, kPlace = 2, kVictim = 3 };
constexpr int kWeightFields = 4;

// Sequences whose lengths travel as arguments of one launch.
constexpr int kLenSeqs = 256;
struct SeqLens {
    int32_t len[kLenSeqs];  // -1: not selected
};

// One layer of a weight cache. Unit u = seq * nkv + kv_head.
struct WeightView {
    void* K;       // [U][cpad][D] in blocks (raas_blocks.h)
    void* V;       // [U][cpad][D] likewise
    int32_t* pos;  // [U][cpad] absolute position, -1 when free
    float* w;      // [U][cpad] accumulated weight
    int32_t* unit; // [U][kWeightFields]
    float* logits; // [U][G][cpad] scratch of one step of split units
    float* part;   // [U][nsplit][G][D] unnormalised outputs of the splits, likewise
    float* ml;     // [U][nsplit][G][2] their maxima (base 2) and sums
    int32_t* arrived;  // [U] splits of the unit that have published; zero between launches
    int U, G, D, C, cpad, nkv, recent, nsplit;
    int wfloats;   // LDS floats of the parts' shares
    int finish_parts;  // workgroups per unit of the kernel that ends a step, 0: none
    unsigned long long* best;  // [U][finish_parts][2] key and place of each one's lightest token
    float scale_log2;
};

// Unnormalised attention over a shared prefix, in `n` parts: rows seq * G + g
// of KV head h at index h * rows + row.
struct PrefixParts {
    const float* o;   // [n][nkv * rows][D]
    const float* ml;  // [n][nkv * rows][2]
    int n, rows;
};
constexpr int kMaxPrefixParts = 64;

struct WeightStepIO {
    const void* q;
    const void* k_new;
    const void* v_new;
    void* out;
    int32_t* positions_out;
    float* weights_out;
    int32_t* evicted_out;
    const int32_t* active;
    PrefixParts prefix;  // n = 0: none
};

// Most workgroups that a unit of the step is split over.
constexpr int kMaxStepSplits = 64;
struct WeightPlan {
    int waves;    // wavefronts per workgroup
    int nsplit;   // workgroups per unit
    bool fused;   // one workgroup per unit, which keeps the logits in LDS
    int finish_parts;  // workgroups per unit of the kernel that ends a step, 0: the step kernel does
};
WeightPlan plan_weight_step(int U, int G, int D, int C, bool bf16);
hipError_t weight_allow_lds(bool bf16, int D, int waves);
// Chooses the kept tokens of each selected unit and writes its records, then
// stores their keys and values. Sequences seq0 .. seq0 + nseq - 1.
hipError_t launch_weight_prefill(const WeightView& L, bool bf16, const void* k, const void* v, const float* weights,
                                 const SeqLens& lens, int seq0, int nseq, int max_len, hipStream_t s);
// stream: keys and values are read with non-temporal loads
hipError_t launch_weight_step(const WeightView& L, bool bf16, const WeightStepIO& io, const WeightPlan& plan,
                              bool stream, hipStream_t s);

// One layer of a shared prefix: K, V [nkv][tpad][D] in blocks.
struct PrefixView {
    void* K;
    void* V;
    const int32_t* len;  // device: tokens stored
    float* part;         // [n][nkv * rows][D]
    float* ml;           // [n][nkv * rows][2]
    int nkv, G, D, tpad, rows;  // rows = sequences * G
    int nsplit;
    float scale_log2;
};
// Parts that the attention of `rows` rows per KV head is cut into.
int plan_prefix(int nkv, int rows, int tokens, bool bf16);
// Rows of the parts that attention of up to `rows` rows may write, whatever is
// stored: sizes the scratch.
size_t prefix_scratch_rows(int nkv, int rows);
hipError_t launch_prefix_store(void* K, void* V, int32_t* len, int nkv, int D, int tpad, bool bf16, const void* k,
                               const void* v, int tokens, hipStream_t s);
hipError_t launch_prefix_attention(const PrefixView& P, bool bf16, const void* q, hipStream_t s);
hipError_t launch_prefix_join(const PrefixView& P, bool bf16, void* out, float* lse, hipStream_t s);

// A cache whose step attends to a shared prefix besides, and the refusals that
// follow; then the prefix's attention of the step's queries into its parts, and the bytes
// that it reads.
struct PrefixUser {
    int n_q_heads, n_kv_heads, head_dim, dtype, device, batch;
};
raas_status check_step_prefix(const raas_prefix* p, int32_t layer, const PrefixUser& u);
raas_status step_prefix_parts(raas_prefix* p, int32_t layer, const void* q, int batch, PrefixParts& parts, double& bytes,
                              hipStream_t s);

// Keys and values of units to blocks: row t of unit u comes from row
// pos[u * pad + t] of its source (pos NULL: row t), for t < min(len, C).
struct StoreIn {
    const int32_t* pos;
    int C, pad, nkv, seq0, stride, tokens;  // tokens >= 0: every unit's length; else lens
};

// Weights of prompts (raas_prompt_weights): sequences seq0 .. seq0 + nseq - 1.
struct PromptPlan {
    int chunks, chunk_keys;      // pieces of the keys in the pass that finds the rows' sums
    int row_chunks, chunk_rows;  // pieces of the rows in the pass that adds up their probabilities
};
PromptPlan plan_prompt(int units, int G, int W, int P, bool bf16);
struct PromptView : PromptPlan {
    const void* q;           // [B][W][Hq][D]
    const void* k;           // [B][nkv][P][D]
    const float* prefix_lse; // [B][W][Hq] or NULL
    float* weights;          // [B][nkv][P]
    float* stat;             // [nseq * nkv][W * G][2] scratch: each row's maximum (base 2) and 1 / sum
    float* ml;               // [nseq * nkv][W * G][chunks][2] scratch, if chunks > 1: maxima and sums
    float* part;             // [row_chunks][nseq * nkv][P] scratch, if row_chunks > 1
    int W, P, G, D, nkv, seq0, nseq;
    uint32_t g_magic;        // row / G = umulhi(row, g_magic), G > 1
    float scale_log2;
};
hipError_t launch_prompt_weights(const PromptView& v, bool bf16, const SeqLens& lens, hipStream_t s);

}  // namespace raas
