// gfx950 kernels of the prompt weights: what the queries of a prompt's last
// `window` tokens give each of its tokens,
//   x_ij = q_i . k_j / sqrt(d), j <= i;  lse_i = log sum_j exp(x_ij)
//   w_j = sum_{i >= j} exp(x_ij - lse_i), over the group's heads besides.
// A first kernel finds each query row's maximum and sum, a second one walks
// the rows that see a tile of keys and adds their probabilities up in
// registers: the products are computed twice, but no probability is written
// (a window of the whole prompt has as many as P^2 / 2 per head), and no
// atomic changes the order of a sum.
#include <math.h>

#include <algorithm>

#include "raas_blocks.h"
#include "raas_weight_internal.h"

namespace raas {
namespace {

using namespace blk;

constexpr int kWaves = 4;
constexpr int kKeys = 16;   // keys of a tile
constexpr int kRowTiles = 4, kKeyTiles = 4;  // of 16, per wavefront: rows in the first kernel, keys in the second

__device__ __forceinline__ int seq_rows(const PromptView& v, int len) { return min(len, v.W); }
// row i * G + g is head g of query i
__device__ __forceinline__ int query_of(const PromptView& v, int row) {
    return v.G == 1 ? row : (int)__umulhi((uint32_t)row, v.g_magic);
}
template <typename T, int D>
__device__ __forceinline__ const T* query_row(const PromptView& v, int b, int h, int row) {
    const int i = query_of(v, row);
    return (const T*)v.q + (((size_t)b * v.W + i) * v.nkv * v.G + (size_t)h * v.G + (row - i * v.G)) * D;
}

// Grid: row tiles, key chunks, units.
template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void k_prompt_rows(PromptView v, SeqLens lens) {
    constexpr int VE = kVec<T>, KS = D / (4 * VE);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, a = lane >> 4, col = lane & 15;
    const int unit = blockIdx.z, b = v.seq0 + unit / v.nkv, h = unit % v.nkv, chunk = blockIdx.y;
    const int len = lens.len[unit / v.nkv], nq = seq_rows(v, len), rows = nq * v.G;
    const int r0 = (blockIdx.x * kWaves + w) * 16 * kRowTiles;
    if (r0 >= rows) return;
    u32x4 q[kRowTiles][KS];
    int last[kRowTiles];  // last key that the row sees
    float m[kRowTiles], l[kRowTiles];
#pragma unroll
    for (int t = 0; t < kRowTiles; ++t) {
        const int r = r0 + 16 * t + col, rr = min(r, rows - 1);
        load_row<T, D>(query_row<T, D>(v, b, h, rr), true, a, q[t]);
        last[t] = len - nq + query_of(v, rr);
        m[t] = -INFINITY;
        l[t] = 0.0f;
    }
    const int seen = len - nq + query_of(v, min(r0 + 16 * kRowTiles, rows) - 1) + 1;
    const int hi = min(seen, (chunk + 1) * v.chunk_keys);
    const T* K = (const T*)v.k + ((size_t)b * v.nkv + h) * v.P * D;
    for (int j0 = chunk * v.chunk_keys; j0 < hi; j0 += kKeys) {
        u32x4 k[KS];
        load_row<T, D>(K + (size_t)min(j0 + col, len - 1) * D, true, a, k);
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t) {
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) x = mfma16<T>(k[ks], q[t][ks], x);
            float mb = -INFINITY;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = j0 + 4 * a + r <= last[t] ? x[r] * v.scale_log2 : -INFINITY;
                mb = fmaxf(mb, x[r]);
            }
            const float mn = fmaxf(m[t], mb), ref = mn == -INFINITY ? 0.0f : mn;
            l[t] *= __builtin_amdgcn_exp2f(m[t] - ref);
#pragma unroll
            for (int r = 0; r < 4; ++r) l[t] += __builtin_amdgcn_exp2f(x[r] - ref);
            m[t] = mn;
        }
    }
#pragma unroll
    for (int t = 0; t < kRowTiles; ++t) {
        const float M = max_groups(m[t]), ref = M == -INFINITY ? 0.0f : M;
        const float Z = sum_groups(l[t] * __builtin_amdgcn_exp2f(m[t] - ref));
        const int r = r0 + 16 * t + col;
        if (a == 0 && r < rows) {
            float* to = v.ml + 2 * (((size_t)unit * v.W * v.G + r) * v.chunks + chunk);
            to[0] = M;
            to[1] = Z;
        }
    }
}

// Grid: key tiles of a workgroup, units.
template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void k_prompt_keys(PromptView v, SeqLens lens) {
    constexpr int VE = kVec<T>, KS = D / (4 * VE);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, a = lane >> 4, col = lane & 15;
    const int unit = blockIdx.y, b = v.seq0 + unit / v.nkv, h = unit % v.nkv;
    const int len = lens.len[unit / v.nkv], nq = seq_rows(v, len), rows = nq * v.G;
    const int j0 = (blockIdx.x * kWaves + w) * 16 * kKeyTiles;
    if (j0 >= len) return;
    const T* K = (const T*)v.k + ((size_t)b * v.nkv + h) * v.P * D;
    u32x4 k[kKeyTiles][KS];
    f32x4 sum[kKeyTiles];
#pragma unroll
    for (int t = 0; t < kKeyTiles; ++t) {
        load_row<T, D>(K + (size_t)min(j0 + 16 * t + col, len - 1) * D, true, a, k[t]);
        sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // the first query that sees this tile's first key
    const int first = max(0, j0 - (len - nq)) * v.G;
    for (int r0 = first & ~15; r0 < rows; r0 += 16) {
        const int r = r0 + col, rr = min(r, rows - 1);
        u32x4 q[KS];
        load_row<T, D>(query_row<T, D>(v, b, h, rr), true, a, q);
        const int i = query_of(v, rr);
        const float* ml = v.ml + 2 * ((size_t)unit * v.W * v.G + rr) * v.chunks;
        float M = -INFINITY, Z = 0.0f, pre = -INFINITY;
        if (v.prefix_lse != nullptr)
            pre = v.prefix_lse[((size_t)b * v.W + i) * v.nkv * v.G + (size_t)h * v.G + (rr - i * v.G)] *
                  1.44269504088896340736f;
        M = pre;
        for (int c = 0; c < v.chunks; ++c) M = fmaxf(M, ml[2 * c]);
        if (pre != -INFINITY) Z = __builtin_amdgcn_exp2f(pre - M);
        for (int c = 0; c < v.chunks; ++c) Z += ml[2 * c + 1] * __builtin_amdgcn_exp2f(ml[2 * c] - M);
        const float lse = M + __builtin_amdgcn_logf(Z);
        const int last = r < rows ? len - nq + i : -1;
#pragma unroll
        for (int t = 0; t < kKeyTiles; ++t) {
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) x = mfma16<T>(k[t][ks], q[ks], x);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum[t][e] += j0 + 16 * t + 4 * a + e <= last
                                 ? __builtin_amdgcn_exp2f(x[e] * v.scale_log2 - lse) : 0.0f;
        }
    }
#pragma unroll
    for (int t = 0; t < kKeyTiles; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = sum[t][e];
#pragma unroll
            for (int d = 8; d >= 1; d >>= 1) x += __shfl_xor(x, d);
            const int j = j0 + 16 * t + 4 * a + e;
            if (col == 0 && j < len) v.weights[((size_t)b * v.nkv + h) * v.P + j] = x;
        }
}

template <typename T, int D>
void launch_t(const PromptView& v, const SeqLens& lens, int most, hipStream_t s) {
    const int units = v.nseq * v.nkv, rows = std::min(most, v.W) * v.G;
    const int row_step = kWaves * 16 * kRowTiles, key_step = kWaves * 16 * kKeyTiles;
    hipLaunchKernelGGL((k_prompt_rows<T, D>), dim3((rows + row_step - 1) / row_step, v.chunks, units),
                       dim3(kWaves * 64), 0, s, v, lens);
    hipLaunchKernelGGL((k_prompt_keys<T, D>), dim3((most + key_step - 1) / key_step, units), dim3(kWaves * 64), 0, s,
                       v, lens);
}

}  // namespace

int plan_prompt_chunks(int units, int G, int W, int P) {
    const int row_step = kWaves * 16 * kRowTiles;
    const long long wgs = (long long)units * (((long long)W * G + row_step - 1) / row_step);
    const int want = (int)std::max<long long>(1, std::min<long long>(16, 512 / std::max<long long>(1, wgs)));
    return std::max(1, std::min(want, P / 256));
}

hipError_t launch_prompt_weights(const PromptView& v, bool bf16, const SeqLens& lens, hipStream_t s) {
    int most = 0;
    for (int i = 0; i < v.nseq; ++i) most = std::max(most, lens.len[i]);
    if (most == 0) return hipSuccess;
    if (bf16) v.D == 128 ? launch_t<uint16_t, 128>(v, lens, most, s) : launch_t<uint16_t, 64>(v, lens, most, s);
    else v.D == 128 ? launch_t<float, 128>(v, lens, most, s) : launch_t<float, 64>(v, lens, most, s);
    return hipGetLastError();
}

}  // namespace raas
