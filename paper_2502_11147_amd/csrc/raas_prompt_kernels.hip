// gfx950 kernels of the prompt weights: what the queries of a prompt's last
// `window` tokens give each of its tokens,
//   x_ij = q_i . k_j / sqrt(d), j <= i;  m_i = max_j x_ij
//   w_j = sum_{i >= j} exp(x_ij - m_i) / sum_j' exp(x_ij' - m_i), over the
// group's heads besides. A first kernel finds each query row's maximum and sum,
// a second one walks the rows that see a tile of keys and adds their
// probabilities up in registers: the products are computed twice, but no probability is written
// (a window of the whole prompt has as many as P^2 / 2 per head), and no
// atomic changes the order of a sum.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "raas_blocks.h"
#include "raas_weight_internal.h"

namespace raas {
namespace {

using namespace blk;

constexpr int kWaves = 4;
constexpr int kThreads = 256;  // of the kernels that join and add
constexpr float kNothing = -1e30f;  // the maximum (base 2) of no logits: finite, so that no difference is NaN
constexpr int kStage = 64;  // rows (keys of the first kernel, queries of the second) that a workgroup stages in LDS
// 16-row tiles that a wavefront holds in registers
template <typename T>
constexpr int kHeld = sizeof(T) == 2 ? 4 : 2;

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

// kStage rows on their way to LDS: 16-byte pieces, row-major, a piece's place
// in its row turned by the row's number, so that the 16 rows of an operand's
// read fall on different banks.
template <typename T, int D>
struct Staged {
    static constexpr int HALVES = D * sizeof(T) > 256 ? 1 : 2;  // of LDS, filled in turn: 32 KB in all either way
    static constexpr int NT = kWaves * 64, NCH = D / kVec<T>, PER = kStage * NCH / NT;  // pieces of a row, and of a thread
    u32x4 x[PER];
    template <class Row>
    __device__ __forceinline__ void load(int tid, Row row) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int p = tid + i * NT;
            x[i] = ld16_in<T>(row(p / NCH) + (p % NCH) * kVec<T>);
        }
    }
    // Puts the rows into LDS, where every wavefront may read them afterwards.
    // (With two halves all have read what this one held before: their reads of it
    // came before the last barrier.)
    __device__ __forceinline__ void store(int tid, u32x4* s) const {
        if constexpr (HALVES == 1) lds_barrier();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int p = tid + i * NT, r = p / NCH;
            s[r * NCH + ((p % NCH) ^ (r & (NCH - 1)))] = x[i];
        }
    }
    // operand of the 16 rows of tile t
    __device__ static __forceinline__ void read(const u32x4* s, int t, int a, int col, u32x4 (&o)[D / (4 * kVec<T>)]) {
        const int r = 16 * t + col;
#pragma unroll
        for (int ks = 0; ks < D / (4 * kVec<T>); ++ks) o[ks] = s[r * NCH + ((4 * ks + a) ^ (r & (NCH - 1)))];
    }
};

typedef float f32x2 __attribute__((ext_vector_type(2)));
// Two floats of the workspace, which is aligned to one.
typedef float f32x2_in __attribute__((ext_vector_type(2), aligned(4)));

// What the second kernel needs of row r of a unit, from its maximum and sum over
// the prompt's keys: the maximum and the sum's inverse, those over a prefix
// counted in. They stay apart: a log-sum-exp would round at its own size, which
// far from 0 is much more than a probability's. (The maximum's own rounding cancels
// between numerator and sum.)
__device__ __forceinline__ f32x2_in row_stat(const PromptView& v, int b, int h, int r, float M, float Z) {
    if (v.prefix_lse != nullptr) {
        constexpr float kLog2e = 1.44269504088896340736f, kRest = (float)(1.44269504088896340736 - (double)kLog2e);
        const int i = query_of(v, r);
        const float lse = v.prefix_lse[((size_t)b * v.W + i) * v.nkv * v.G + (size_t)h * v.G + (r - i * v.G)];
        const float pre = lse * kLog2e, m = fmaxf(M, pre);
        // (what the product's rounding left; of an empty prefix, -inf, nothing)
        const float rest = pre == -INFINITY ? 0.0f : __builtin_fmaf(lse, kRest, __builtin_fmaf(lse, kLog2e, -pre));
        Z = Z * __builtin_amdgcn_exp2f(M - m) + __builtin_amdgcn_exp2f(pre - m + rest);
        M = m;
    }
    return f32x2_in{M, 1.0f / Z};
}
// A row's maximum and sum over one chunk: what the second kernel needs if there is no other.
__device__ __forceinline__ void row_done(const PromptView& v, int unit, int b, int h, int r, int chunk, float M,
                                         float Z) {
    const size_t at = (size_t)unit * v.W * v.G + r;
    if (v.chunks == 1) *reinterpret_cast<f32x2_in*>(v.stat + 2 * at) = row_stat(v, b, h, r, M, Z);
    else *reinterpret_cast<f32x2_in*>(v.ml + 2 * (at * v.chunks + chunk)) = f32x2_in{M, Z};
}

// The chunks of a row joined, 16 lanes a row. Grid: rows, units.
constexpr int kJoinRows = kThreads / 16;
__global__ __launch_bounds__(kThreads) void k_prompt_join(PromptView v, SeqLens lens) {
    const int unit = blockIdx.y, len = lens.len[unit / v.nkv], nq = seq_rows(v, len);
    const int row = blockIdx.x * kJoinRows + threadIdx.x / 16, lane = threadIdx.x & 15;
    const int r = min(row, nq * v.G - 1);
    if (r < 0) return;
    const float* ml = v.ml + 2 * ((size_t)unit * v.W * v.G + r) * v.chunks;
    const int chunks = (len - nq + query_of(v, r)) / v.chunk_keys + 1;  // those that hold keys for it
    float M = kNothing, Z = 0.0f;
    for (int c = lane; c < chunks; c += 16) {
        const f32x2_in x = *reinterpret_cast<const f32x2_in*>(ml + 2 * c);
        const float m = fmaxf(M, x[0]);
        Z = Z * __builtin_amdgcn_exp2f(M - m) + x[1] * __builtin_amdgcn_exp2f(x[0] - m);
        M = m;
    }
    const float most = row16_max(M);
    Z = row16_sum(Z * __builtin_amdgcn_exp2f(M - most));
    if (lane == 0 && row < nq * v.G)
        *reinterpret_cast<f32x2_in*>(v.stat + 2 * ((size_t)unit * v.W * v.G + r)) =
            row_stat(v, v.seq0 + unit / v.nkv, unit % v.nkv, r, most, Z);
}

// Maximum (base 2) and sum of every query row over a chunk of keys. Grid:
// units, row tiles (the ones that see the most keys first), key chunks: the
// workgroups that follow each other have equal work, and with eight units each
// XCD's L2 serves one (row tiles first, some shader engines always got the long
// ones: 125 us for 100). KW wavefronts share RT tiles of 16 rows and take a part
// of the staged keys each. Bound by the vector instructions (62 % of the cycles,
// a prompt of 4096 tokens, every query) and the products (35 %), which follow each
// other; LDS moves 28 bytes a cycle. The more rows a wavefront holds, the fewer
// of its reads a product takes.
template <typename T, int D, int RT, int KW>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(2))) void k_prompt_rows(PromptView v,
                                                                                                   SeqLens lens) {
    constexpr int KS = D / (4 * kVec<T>), SUB = kStage / 16 / KW, HALVES = Staged<T, D>::HALVES;
    constexpr int WG_ROWS = 16 * RT * (kWaves / KW);
    __shared__ __align__(16) u32x4 s_k[HALVES][kStage * D / kVec<T>];
    __shared__ float s_m[KW][WG_ROWS], s_l[KW][WG_ROWS];
    const int tid = threadIdx.x, lane = tid & 63, w = wave_of(tid), a = lane >> 4, col = lane & 15;
    const int unit = blockIdx.x, b = v.seq0 + unit / v.nkv, h = unit % v.nkv, chunk = blockIdx.z;
    const int len = lens.len[unit / v.nkv], nq = seq_rows(v, len), rows = nq * v.G;
    const int wg0 = (gridDim.y - 1 - blockIdx.y) * WG_ROWS;
    if (wg0 >= rows) return;
    const int wk = w % KW, rw = w / KW * 16 * RT, r0 = wg0 + rw, lo = chunk * v.chunk_keys;
    // keys that the workgroup's and this wavefront's last row see
    const int seen = len - nq + query_of(v, min(wg0 + WG_ROWS, rows) - 1) + 1, hi = min(seen, lo + v.chunk_keys);
    if (lo >= hi) return;
    const int mine = r0 < rows ? min(hi, len - nq + query_of(v, min(r0 + 16 * RT, rows) - 1) + 1) : 0;
    const int full = len - nq + query_of(v, min(r0, rows - 1));  // last key that every row of the wavefront sees
    u32x4 q[RT][KS];
    float m[RT], l[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        load_row<T, D>(query_row<T, D>(v, b, h, min(r0 + 16 * t + col, rows - 1)), true, a, q[t]);
        m[t] = kNothing;
        l[t] = 0.0f;
    }
    const T* K = (const T*)v.k + ((size_t)b * v.nkv + h) * v.P * D;
    Staged<T, D> next;
    next.load(tid, [&](int r) { return K + (size_t)min(lo + r, len - 1) * D; });
    for (int j0 = lo, buf = 0; j0 < hi; j0 += kStage, buf = (buf + 1) % HALVES) {
        next.store(tid, s_k[buf]);
        lds_barrier();
        if (j0 + kStage < hi) next.load(tid, [&](int r) { return K + (size_t)min(j0 + kStage + r, len - 1) * D; });
        const int jw = j0 + wk * 16 * SUB;
        if (jw >= mine) continue;
        auto stage = [&](auto masked) {
            f32x4 x[RT][SUB];
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int c = 0; c < SUB; ++c) x[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < SUB; ++c) {
                u32x4 k[KS];
                Staged<T, D>::read(s_k[buf], wk * SUB + c, a, col, k);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int t = 0; t < RT; ++t) x[t][c] = mfma16<T>(k[ks], q[t][ks], x[t][c]);
            }
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if constexpr (masked) {
                    const int last = len - nq + query_of(v, min(r0 + 16 * t + col, rows - 1));
#pragma unroll
                    for (int c = 0; c < SUB; ++c)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            x[t][c][e] = jw + 16 * c + 4 * a + e <= last ? x[t][c][e] : -INFINITY;
                }
                float mb = x[t][0][0];
#pragma unroll
                for (int c = 0; c < SUB; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) mb = fmaxf(mb, x[t][c][e]);
                const float mn = fmaxf(m[t], mb * v.scale_log2);
                float add = 0.0f;
#pragma unroll
                for (int c = 0; c < SUB; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        add += __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][c][e], v.scale_log2, -mn));
                l[t] = __builtin_fmaf(l[t], __builtin_amdgcn_exp2f(m[t] - mn), add);
                m[t] = mn;
            }
        };
        // (two bodies: a branch inside would keep products and exponentials apart)
        if (jw + 16 * SUB - 1 > full) stage(std::true_type{});
        else stage(std::false_type{});
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const float M = max_groups(m[t]);
        const float Z = sum_groups(l[t] * __builtin_amdgcn_exp2f(m[t] - M));
        const int r = rw + 16 * t + col;
        if constexpr (KW > 1) {
            if (a == 0) {
                s_m[wk][r] = M;
                s_l[wk][r] = Z;
            }
        } else {
            if (a == 0 && wg0 + r < rows) row_done(v, unit, b, h, wg0 + r, chunk, M, Z);
        }
    }
    if constexpr (KW > 1) {
        lds_barrier();
        if (tid < WG_ROWS && wg0 + tid < rows) {
            float M = kNothing, Z = 0.0f;
#pragma unroll
            for (int i = 0; i < KW; ++i) M = fmaxf(M, s_m[i][tid]);
#pragma unroll
            for (int i = 0; i < KW; ++i) Z += s_l[i][tid] * __builtin_amdgcn_exp2f(s_m[i][tid] - M);
            row_done(v, unit, b, h, wg0 + tid, chunk, M, Z);
        }
    }
}

// Probabilities of a chunk of query rows, summed per key. Grid: units, key
// tiles (the ones that most rows see first), row chunks. A wavefront holds kHeld
// tiles of 16 keys; the rows pass through LDS with their maximum (base 2) and the
// inverse of their sum.
// Bound as the kernel above (52 and 29 %). Three wavefronts per SIMD at head_dim 64, where two
// registers too many would leave two (a whole prompt of 3000 tokens 94.6 us, 97).
template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2))) void k_prompt_keys(
    PromptView v, SeqLens lens) {
    constexpr int KS = D / (4 * kVec<T>), KT = kHeld<T>, SUB = kStage / 16, HALVES = Staged<T, D>::HALVES;
    constexpr int WG_KEYS = kWaves * 16 * KT;
    __shared__ __align__(16) u32x4 s_q[HALVES][kStage * D / kVec<T>];
    __shared__ f32x2 s_stat[HALVES][kStage];
    const int tid = threadIdx.x, lane = tid & 63, w = wave_of(tid), a = lane >> 4, col = lane & 15;
    const int unit = blockIdx.x, b = v.seq0 + unit / v.nkv, h = unit % v.nkv;
    const int len = lens.len[unit / v.nkv], nq = seq_rows(v, len), rows = nq * v.G;
    const int wg0 = blockIdx.y * WG_KEYS, j0 = wg0 + w * 16 * KT;
    if (wg0 >= len) return;
    const T* K = (const T*)v.k + ((size_t)b * v.nkv + h) * v.P * D;
    u32x4 k[KT][KS];
    f32x4 sum[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        load_row<T, D>(K + (size_t)min(j0 + 16 * t + col, len - 1) * D, true, a, k[t]);
        sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // the first rows that see the workgroup's and this wavefront's first key
    const int first = max(0, wg0 - (len - nq)) * v.G, mine = max(0, j0 - (len - nq)) * v.G;
    const int lo = blockIdx.z * v.chunk_rows, hi = min(rows, lo + v.chunk_rows);
    Staged<T, D> next;
    f32x2 stat = {0.f, 0.f};
    auto load = [&](int r0) {
        next.load(tid, [&](int r) { return query_row<T, D>(v, b, h, min(r0 + r, rows - 1)); });
        if (tid >= kStage) return;
        // (rows behind the last weigh nothing)
        stat = f32x2{INFINITY, 0.f};
        if (r0 + tid < rows)
            stat = *reinterpret_cast<const f32x2_in*>(v.stat + 2 * ((size_t)unit * v.W * v.G + r0 + tid));
    };
    const int start = max(lo, first) / kStage * kStage;
    if (start < hi) load(start);
    for (int r0 = start, buf = 0; r0 < hi; r0 += kStage, buf = (buf + 1) % HALVES) {
        next.store(tid, s_q[buf]);
        if (tid < kStage) s_stat[buf][tid] = stat;
        lds_barrier();
        if (r0 + kStage < hi) load(r0 + kStage);
        if (r0 + kStage <= mine || j0 >= len) continue;
        // (two bodies: a branch inside would keep products and exponentials apart)
        auto stage = [&](auto masked) {
#pragma unroll
            for (int c = 0; c < SUB; ++c) {
                u32x4 q[KS];
                Staged<T, D>::read(s_q[buf], c, a, col, q);
                const f32x2 st = s_stat[buf][16 * c + col];
                const int last = masked ? len - nq + query_of(v, r0 + 16 * c + col) : 0;
                f32x4 x[KT];
#pragma unroll
                for (int t = 0; t < KT; ++t) x[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int t = 0; t < KT; ++t) x[t] = mfma16<T>(k[t][ks], q[ks], x[t]);
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = __builtin_fmaf(x[t][e], v.scale_log2, -st[0]);
                        const float p = __builtin_amdgcn_exp2f(masked && j0 + 16 * t + 4 * a + e > last ? -INFINITY : y);
                        sum[t][e] = __builtin_fmaf(p, st[1], sum[t][e]);
                    }
            }
        };
        if (len - nq + query_of(v, r0) < j0 + 16 * KT - 1) stage(std::true_type{});
        else stage(std::false_type{});
    }
    float* to = v.row_chunks == 1 ? v.weights + ((size_t)b * v.nkv + h) * v.P
                                  : v.part + ((size_t)blockIdx.z * v.nseq * v.nkv + unit) * v.P;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = row16_sum(sum[t][e]);
            const int j = j0 + 16 * t + 4 * a + e;
            if (col == 0 && j < len) to[j] = x;
        }
}

// The row chunks' sums, added up. Grid: keys, units.
__global__ __launch_bounds__(kThreads) void k_prompt_sum(PromptView v, SeqLens lens) {
    const int unit = blockIdx.y, j = blockIdx.x * kThreads + threadIdx.x;
    if (j >= lens.len[unit / v.nkv]) return;
    const size_t step = (size_t)v.nseq * v.nkv * v.P;
    const float* from = v.part + (size_t)unit * v.P + j;
    float x = 0.0f;
    for (int c0 = 0; c0 < v.row_chunks; c0 += 8) {  // eight reads on their way together
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = from[min(c0 + k, v.row_chunks - 1) * step];
#pragma unroll
        for (int k = 0; k < 8; ++k) x += c0 + k < v.row_chunks ? y[k] : 0.0f;
    }
    v.weights[((size_t)v.seq0 * v.nkv + unit) * v.P + j] = x;
}

template <typename T, int D>
void launch_t(const PromptView& v, const SeqLens& lens, int most, hipStream_t s) {
    constexpr int H = kHeld<T>;
    const int units = v.nseq * v.nkv, rows = std::min(most, v.W) * v.G, all = v.W * v.G;
    const int chunks = (most + v.chunk_keys - 1) / v.chunk_keys;
    // (the choice goes by the call's sizes, as the plan's does)
    auto by_rows = [&](auto kernel, int step) {
        hipLaunchKernelGGL(kernel, dim3(units, (rows + step - 1) / step, chunks), dim3(kWaves * 64), 0, s, v, lens);
    };
    if (all <= 16) by_rows(k_prompt_rows<T, D, 1, 4>, 16);
    else if (all <= 16 * H) by_rows(k_prompt_rows<T, D, H, 4>, 16 * H);
    else by_rows(k_prompt_rows<T, D, H, 1>, 64 * H);
    if (v.chunks > 1)
        hipLaunchKernelGGL(k_prompt_join, dim3((rows + kJoinRows - 1) / kJoinRows, units), dim3(kThreads), 0, s, v, lens);
    hipLaunchKernelGGL((k_prompt_keys<T, D>), dim3(units, (most + 64 * H - 1) / (64 * H), v.row_chunks),
                       dim3(kWaves * 64), 0, s, v, lens);
    if (v.row_chunks > 1)
        hipLaunchKernelGGL(k_prompt_sum, dim3((most + kThreads - 1) / kThreads, units), dim3(kThreads), 0, s, v, lens);
}

// Workgroups wanted in each of the two kernels: about six per CU, so that the
// causal part's uneven ones even out (a prompt of 4096 tokens, every query: 214 us
// with 700, 197 with 1536, 204 with twice as many, each of which starts with its
// rows or keys once more).
constexpr int kWorkgroups = 1536;

}  // namespace

PromptPlan plan_prompt(int units, int G, int W, int P, bool bf16) {
    const int held = bf16 ? kHeld<uint16_t> : kHeld<float>;
    const long long rows = (long long)W * G;
    // at least 256 keys or rows a piece (us with 512 / 256 / 128, 8 KV heads: 1 prompt
    // of 2000 tokens, window 64 31.6 / 24.9 / 28.1, 4 of 300, every query 33.9 / 26.5 /
    // 29.8, 1 of 16000, window 32 29.2 / 30.4 / 31.0); of fp32, whose products take
    // eight times as long, 64 (with 256 / 128 / 64: 1 of 957, window 35 47.2 / 38.4 /
    // 32.3, 1 of 500, every query 69.8 / 64.7 / 54.1)
    auto pieces = [&](long long n, long long others, long long tile, int& count, int& size) {
        const long long wgs = units * ((others + tile - 1) / tile);
        const long long want = std::max(1LL, std::min<long long>(kWorkgroups / wgs, n / (bf16 ? 256 : 64)));
        size = (int)(((n + want - 1) / want + kStage - 1) / kStage * kStage);
        count = (int)((n + size - 1) / size);
    };
    PromptPlan p;
    pieces(P, rows, rows <= 16 ? 16 : rows <= 16 * held ? 16 * held : 64 * held, p.chunks, p.chunk_keys);
    pieces(rows, P, 64 * held, p.row_chunks, p.chunk_rows);
    return p;
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
