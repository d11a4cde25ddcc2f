// gfx950 kernels of the shared prefix: attention of every sequence's queries
// over one prompt that the batch shares. Per KV head the queries of all
// sequences are the rows of one product, so the prompt is read once whatever
// the batch:
//   x_rj = q_r . k_j / sqrt(d);  out_r = sum_j exp(x_rj) v_j / sum_j exp(x_rj)
//   lse_r = log sum_j exp(x_rj)
// The prompt is cut into parts, whose unnormalised outputs, maxima and sums
// are joined at the end: by k_prefix_join, or by the step that attends to the
// sequence's own tokens besides.
#include <math.h>

#include <algorithm>

#include "raas_blocks.h"
#include "raas_weight_internal.h"

namespace raas {
namespace {

using namespace blk;

constexpr int kWaves = 4;

// One workgroup per (part, KV head, tile of 16 RT rows); its wavefronts take
// the blocks of the part in turn, straight from memory to registers.
template <typename T, int D, int RT>
__global__ __launch_bounds__(kWaves * 64) void k_prefix(PrefixView P, const T* __restrict__ q) {
    constexpr int VE = kVec<T>, BT = kTokens<T>, QT = kTiles<T>, KS = D / (4 * VE), NP = D / 16;
    __shared__ __align__(16) float s_o[kWaves][16][D + 4];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    const int tid = threadIdx.x, lane = tid & 63, w = wave_of(tid), a = lane >> 4, col = lane & 15;
    const int h = blockIdx.y, r0 = blockIdx.x * 16 * RT, part = blockIdx.z;
    const int n = *P.len, nb = (n + BT - 1) / BT, per = (nb + P.nsplit - 1) / P.nsplit;
    const int lo = min(nb, part * per), hi = min(nb, lo + per);
    const T* K = (const T*)P.K + (size_t)h * P.tpad * D;
    const T* V = (const T*)P.V + (size_t)h * P.tpad * D;
    u32x4 qv[RT][KS];
    Softmax<D> s[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = r0 + 16 * t + col, seq = r / P.G;
        load_row<T, D>(q + ((size_t)seq * P.nkv * P.G + h * P.G + (r - seq * P.G)) * D, r < P.rows, a, qv[t]);
        s[t].clear();
    }
    for (int b = lo + w; b < hi; b += kWaves) {
        u32x4 kr[NP], vr[NP];
        const size_t at = (size_t)b * BT * D + lane * VE;
#pragma unroll
        for (int i = 0; i < NP; ++i) kr[i] = ld16(K + at + i * 64 * VE);
#pragma unroll
        for (int i = 0; i < NP; ++i) vr[i] = ld16(V + at + i * 64 * VE);
        const int valid = min(BT, n - b * BT);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            f32x4 x[QT];
            attend<T, D>(kr, vr, qv[t], valid, a, P.scale_log2, s[t], x);
        }
    }
    const size_t row0 = ((size_t)part * P.nkv + h) * P.rows;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const float l = sum_groups(s[t].l);
        if (a == 0) {
            s_m[w][col] = s[t].m;
            s_l[w][col] = l;
        }
#pragma unroll
        for (int ct = 0; ct < NP; ++ct) *reinterpret_cast<f32x4*>(&s_o[w][col][16 * ct + 4 * a]) = s[t].o[ct];
        __syncthreads();
        for (int i = tid; i < 16 * D; i += kWaves * 64) {
            const int rr = i / D, c = i % D, r = r0 + 16 * t + rr;
            float M = -INFINITY, x = 0.0f, z = 0.0f;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) M = fmaxf(M, s_m[k][rr]);
            const float ref = M == -INFINITY ? 0.0f : M;  // a part may hold no token
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                const float e = __builtin_amdgcn_exp2f(s_m[k][rr] - ref);
                x += s_o[k][rr][c] * e;
                z += s_l[k][rr] * e;
            }
            if (r < P.rows) {
                P.part[(row0 + r) * D + c] = x;
                if (c == 0) {
                    P.ml[2 * (row0 + r)] = M;
                    P.ml[2 * (row0 + r) + 1] = z;
                }
            }
        }
        __syncthreads();
    }
}

// Output and log-sum-exp of every row from the parts: one wavefront per row.
// Over an empty prefix the output is 0 and the log-sum-exp -inf.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_prefix_join(PrefixView P, T* __restrict__ out, float* __restrict__ lse) {
    const int rows = P.nkv * P.rows, i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (i >= rows) return;
    const int h = i / P.rows, r = i - h * P.rows, seq = r / P.G;
    const size_t to = (size_t)seq * P.nkv * P.G + h * P.G + (r - seq * P.G);
    float M = -INFINITY, Z = 0.0f, x[D / 64] = {};
    for (int s = 0; s < P.nsplit; ++s) M = fmaxf(M, P.ml[2 * ((size_t)s * rows + i)]);
    if (M != -INFINITY) {
        for (int s = 0; s < P.nsplit; ++s) {
            const float* ml = P.ml + 2 * ((size_t)s * rows + i);
            const float e = __builtin_amdgcn_exp2f(ml[0] - M);
            Z += ml[1] * e;
#pragma unroll
            for (int c = 0; c < D / 64; ++c) x[c] += P.part[((size_t)s * rows + i) * D + 64 * c + lane] * e;
        }
    }
#pragma unroll
    for (int c = 0; c < D / 64; ++c) out[to * D + 64 * c + lane] = from_f<T>(Z > 0.0f ? x[c] / Z : 0.0f);
    if (lse != nullptr && lane == 0)
        lse[to] = Z > 0.0f ? (M + __builtin_amdgcn_logf(Z)) * 0.69314718055994530942f : -INFINITY;
}

template <typename T, int D>
void launch_t(const PrefixView& P, const void* q, hipStream_t s) {
    if (P.rows <= 16)
        hipLaunchKernelGGL((k_prefix<T, D, 1>), dim3(1, P.nkv, P.nsplit), dim3(kWaves * 64), 0, s, P, (const T*)q);
    else
        hipLaunchKernelGGL((k_prefix<T, D, 2>), dim3((P.rows + 31) / 32, P.nkv, P.nsplit), dim3(kWaves * 64), 0, s, P,
                           (const T*)q);
}

template <typename T, int D>
void join_t(const PrefixView& P, void* out, float* lse, hipStream_t s) {
    hipLaunchKernelGGL((k_prefix_join<T, D>), dim3(((unsigned)P.nkv * P.rows + 3) / 4), dim3(256), 0, s, P, (T*)out,
                       lse);
}

// row tiles of a launch, and the rows of one
int row_tile(int rows) { return rows <= 16 ? 16 : 32; }
int row_tiles(int rows) { return (rows + row_tile(rows) - 1) / row_tile(rows); }
constexpr int kWorkgroups = 512;  // wanted at least

}  // namespace

PrefixPlan plan_prefix(int nkv, int rows, int D, int tokens, bool bf16) {
    const int bt = bf16 ? 32 : 16, nb = (tokens + bt - 1) / bt;
    (void)D;
    const int want = std::min(kMaxPrefixParts, std::max(1, kWorkgroups / (nkv * row_tiles(rows))));
    return PrefixPlan{std::max(1, std::min(want, (nb + kWaves - 1) / kWaves))};
}

size_t prefix_scratch_rows(int nkv, int rows, int D, bool bf16) {
    (void)D;
    (void)bf16;
    // parts * tiles stays below this, and a tile has at most 32 rows
    return 32 * (size_t)std::max(kWorkgroups, nkv * row_tiles(rows));
}

hipError_t launch_prefix_attention(const PrefixView& P, bool bf16, const void* q, hipStream_t s) {
    if (bf16) P.D == 128 ? launch_t<uint16_t, 128>(P, q, s) : launch_t<uint16_t, 64>(P, q, s);
    else P.D == 128 ? launch_t<float, 128>(P, q, s) : launch_t<float, 64>(P, q, s);
    return hipGetLastError();
}

hipError_t launch_prefix_join(const PrefixView& P, bool bf16, void* out, float* lse, hipStream_t s) {
    if (bf16) P.D == 128 ? join_t<uint16_t, 128>(P, out, lse, s) : join_t<uint16_t, 64>(P, out, lse, s);
    else P.D == 128 ? join_t<float, 128>(P, out, lse, s) : join_t<float, 64>(P, out, lse, s);
    return hipGetLastError();
}

}  // namespace raas
