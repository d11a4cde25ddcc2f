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

constexpr int kWaves = 8;

// Few rows: one workgroup per (KV head, tile of 16 RT rows, part). Bound by
// memory: its wavefronts take the blocks of the part in turn, straight from
// memory to registers, a block on its way while the one before it is attended
// to, and join in LDS, so that a part is written once.
template <typename T, int D, int RT>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(2))) void k_prefix(
    PrefixView P, const T* __restrict__ q) {
    constexpr int VE = kVec<T>, BT = kTokens<T>, QT = kTiles<T>, KS = D / (4 * VE), NP = D / 16;
    constexpr int CH = 64;  // channels that are joined at a time
    __shared__ __align__(16) float s_o[kWaves][16][CH + 4];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    const int tid = threadIdx.x, lane = tid & 63, w = wave_of(tid), a = lane >> 4, col = lane & 15;
    const int h = blockIdx.x, r0 = blockIdx.y * 16 * RT, part = blockIdx.z;
    const int n = *P.len, nb = (n + BT - 1) / BT, per = (nb + P.nsplit - 1) / P.nsplit;
    const int lo = min(nb, part * per), hi = min(nb, lo + per);
    const T* K = (const T*)P.K + (size_t)h * P.tpad * D;
    const T* V = (const T*)P.V + (size_t)h * P.tpad * D;
    u32x4 qv[RT][KS], k0[NP], v0[NP], k1[NP], v1[NP];
    Softmax<D> s[RT];
    auto load = [&](int b, u32x4 (&kr)[NP], u32x4 (&vr)[NP]) {
        const size_t at = (size_t)min(b, hi - 1) * BT * D + lane * VE;
#pragma unroll
        for (int i = 0; i < NP; ++i) kr[i] = ld16(K + at + i * 64 * VE);
#pragma unroll
        for (int i = 0; i < NP; ++i) vr[i] = ld16(V + at + i * 64 * VE);
    };
    if (lo < hi) load(lo + w, k0, v0);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = r0 + 16 * t + col, seq = r / P.G;
        load_row<T, D>(q + ((size_t)seq * P.nkv * P.G + h * P.G + (r - seq * P.G)) * D, r < P.rows, a, qv[t]);
        s[t].clear();
    }
    auto block = [&](int b, const u32x4 (&kr)[NP], const u32x4 (&vr)[NP]) {
        const int valid = min(BT, n - b * BT);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            f32x4 x[QT];
            attend<T, D>(kr, vr, qv[t], valid, a, P.scale_log2, s[t], x);
        }
    };
    for (int b = lo + w; b < hi;) {
        load(b + kWaves, k1, v1);
        block(b, k0, v0);
        b += kWaves;
        if (b >= hi) break;
        load(b + kWaves, k0, v0);
        block(b, k1, v1);
        b += kWaves;
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
        for (int c0 = 0; c0 < D; c0 += CH) {
#pragma unroll
            for (int ct = 0; ct < CH / 16; ++ct)
                *reinterpret_cast<f32x4*>(&s_o[w][col][16 * ct + 4 * a]) = s[t].o[c0 / 16 + ct];
            __syncthreads();
            for (int i = tid; i < 16 * CH; i += kWaves * 64) {
                const int rr = i / CH, c = i % CH, r = r0 + 16 * t + rr;
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
                    P.part[(row0 + r) * D + c0 + c] = x;
                    if (c == 0 && c0 == 0) *reinterpret_cast<float2*>(P.ml + 2 * (row0 + r)) = make_float2(M, z);
                }
            }
            __syncthreads();
        }
    }
}

// Many rows: one workgroup per (KV head, tile of 128 or 256 rows, part). Its
// wavefronts hold 32 rows each and share the blocks of the part through LDS,
// where one lies ready while two more are on their way in registers; blocks are
// stored in operand order, so both sides of LDS are consecutive. Bound by the
// matrix cores and the exponentials: 48 products (bf16, head_dim 128) of 16 cycles
// a block and wavefront beside about as many cycles of vector work (54 and 52 % of
// the cycles, 128 sequences over 32768 tokens; LDS moves 52 bytes a cycle). 16 of the
// products are those of the probabilities' lower halves (us without / with them,
// 8 KV heads of G = 4: 128 sequences over 32768 tokens 81 / 102, 64 over 8192 26.9
// / 30.4, 32 over 4096 15.2 / 16.2). A wavefront has both in
// flight, as the logits of the next block are formed while this one's
// probabilities are; so a block's keys are staged with the values of the one
// before. Eight wavefronts where there are the rows: two per SIMD in step with
// each other (of two workgroups of four, the older one went first and left the
// other to run on alone: 53 and 79 us of 80).
constexpr int kWideTiles = 2;
template <int NW>
constexpr int kWideRows = NW * 16 * kWideTiles;

// The softmax's reference need not be the maximum: it follows a row's logits
// once they exceed it by this much (base 2), so that the sums stay within
// 2^kSlack of their usual size and most blocks need no maximum over lanes.
constexpr float kSlack = 8.0f;

template <typename T, int D, int NW>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2))) void k_prefix_wide(
    PrefixView P, const T* __restrict__ q) {
    constexpr int VE = kVec<T>, BT = kTokens<T>, QT = kTiles<T>, KS = D / (4 * VE), NP = D / 16, RT = kWideTiles;
    constexpr int PER = 2 * NP / NW;  // 1 KiB pieces of a stage that a wavefront brings
    __shared__ __align__(16) u32x4 s_kv[2][2 * NP * 64];
    const int tid = threadIdx.x, lane = tid & 63, w = wave_of(tid), a = lane >> 4, col = lane & 15;
    const int h = blockIdx.x, r0 = blockIdx.y * kWideRows<NW> + w * 16 * RT, part = blockIdx.z;
    const int n = *P.len, nb = (n + BT - 1) / BT, per = (nb + P.nsplit - 1) / P.nsplit;
    const int lo = min(nb, part * per), hi = min(nb, lo + per);
    const T* K = (const T*)P.K + (size_t)h * P.tpad * D;
    const T* V = (const T*)P.V + (size_t)h * P.tpad * D;
    u32x4 qv[RT][KS], even[PER], odd[PER];
    Softmax<D> s[RT];
    // stage of block b: its keys, and the values of block b - 1 (within lo .. hi - 1 either way)
    auto load = [&](int b, u32x4 (&next)[PER]) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int piece = w * PER + i;  // the first NP are keys
            const T* from = piece < NP ? K + ((size_t)min(b, hi - 1) * BT * D + piece * 64 * VE)
                                       : V + ((size_t)min(max(b - 1, lo), hi - 1) * BT * D + (piece - NP) * 64 * VE);
            next[i] = ld16(from + lane * VE);
        }
    };
    auto store = [&](int buf, const u32x4 (&next)[PER]) {
#pragma unroll
        for (int i = 0; i < PER; ++i) s_kv[buf][(w * PER + i) * 64 + lane] = next[i];
    };
    f32x4 x[RT][QT], xn[RT][QT];
    auto logits = [&](int buf, f32x4 (&y)[RT][QT]) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int c = 0; c < QT; ++c) y[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int c = 0; c < QT; ++c) {
                const u32x4 k = s_kv[buf][(c * KS + ks) * 64 + lane];
#pragma unroll
                for (int t = 0; t < RT; ++t) y[t][c] = mfma16<T>(k, qv[t][ks], y[t][c]);
            }
    };
    if (lo < hi) {
        load(lo, even);
        load(lo + 1, odd);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = r0 + 16 * t + col, seq = r / P.G;
        load_row<T, D>(q + ((size_t)seq * P.nkv * P.G + h * P.G + (r - seq * P.G)) * D, r < P.rows, a, qv[t]);
        s[t].clear();
    }
    // block b, while stage b + 2 (next) goes to LDS and stage b + 4 sets out
    auto block = [&](int b, u32x4 (&next)[PER]) {
        const int buf = (b + 1 - lo) & 1;  // holds the keys of b + 1 and the values of b
        if (n - b * BT < BT) {
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int c = 0; c < QT; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[t][c][e] = VE * a + 4 * c + e < n - b * BT ? x[t][c][e] : -INFINITY;
        }
        float mb[RT];
        bool over = false;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            mb[t] = x[t][0][0];
#pragma unroll
            for (int c = 0; c < QT; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) mb[t] = fmaxf(mb[t], x[t][c][e]);
            mb[t] *= P.scale_log2;
            over = over || mb[t] > s[t].m + kSlack;  // (the first block: m is -inf)
        }
        if (__ballot(over) != 0ull) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const float m = fmaxf(s[t].m, max_groups(mb[t]));
                const float alpha = __builtin_amdgcn_exp2f(s[t].m - m);
                s[t].l *= alpha;
#pragma unroll
                for (int ct = 0; ct < NP; ++ct) s[t].o[ct] *= alpha;
                s[t].m = m;
            }
        }
        logits(buf, xn);  // (past the part's end: the last block's again, unused)
        u32x4 ph[RT], pl[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            float p[VE], l = 0.0f;
#pragma unroll
            for (int c = 0; c < QT; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[4 * c + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][c][e], P.scale_log2, -s[t].m));
                    l += p[4 * c + e];
                }
            s[t].l += l;
            const Probs<T> pv(p);
            ph[t] = pv.hi;
            if constexpr (sizeof(T) == 2) pl[t] = pv.lo;
        }
#pragma unroll
        for (int ct = 0; ct < NP; ++ct) {
            const u32x4 v = s_kv[buf][(NP + ct) * 64 + lane];
#pragma unroll
            for (int t = 0; t < RT; ++t) s[t].o[ct] = mfma16<T>(v, ph[t], s[t].o[ct]);
            if constexpr (sizeof(T) == 2)
#pragma unroll
                for (int t = 0; t < RT; ++t) s[t].o[ct] = mfma16<T>(v, pl[t], s[t].o[ct]);
        }
        store(buf ^ 1, next);
        load(b + 4, next);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int c = 0; c < QT; ++c) x[t][c] = xn[t][c];
        lds_barrier();
    };
    if (lo < hi) {
        store(0, even);
        load(lo + 2, even);
        lds_barrier();
        logits(0, x);
        store(1, odd);
        load(lo + 3, odd);
        lds_barrier();
        for (int b = lo;;) {
            block(b, even);
            if (++b >= hi) break;
            block(b, odd);
            if (++b >= hi) break;
        }
    }
    const size_t row0 = ((size_t)part * P.nkv + h) * P.rows;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = r0 + 16 * t + col;
        const float l = sum_groups(s[t].l);
        if (r >= P.rows) continue;
        if (a == 0) *reinterpret_cast<float2*>(P.ml + 2 * (row0 + r)) = make_float2(s[t].m, l);
#pragma unroll
        for (int ct = 0; ct < NP; ++ct)
            *reinterpret_cast<f32x4*>(P.part + (row0 + r) * D + 16 * ct + 4 * a) = s[t].o[ct];
    }
}

// Output and log-sum-exp of every row from at most PARTS parts: one wavefront per
// row, a lane per part for the maximum and the sum, then 16 bytes per lane of 4
// (D 64) or 2 parts at a time. All of a row's reads are on their way together
// (60 rows in 64 parts, D 64: 17.3 -> 3.1 us). The KV head comes first in the
// grid here as in the kernels above, so that with eight of them the parts are
// read on the XCD that wrote them (1024 rows in 16 parts: 9.2 -> 5.0 us). Over an
// empty prefix the output is 0 and the log-sum-exp -inf.
template <typename T, int D, int PARTS>
__global__ __launch_bounds__(256) void k_prefix_join(PrefixView P, T* __restrict__ out, float* __restrict__ lse) {
    constexpr int LANES = D / 4, AT = 64 / LANES, READS = PARTS / AT;  // lanes of a row, parts at a time
    typedef T T4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    const int h = blockIdx.x, r = blockIdx.y * 4 + wave_of(threadIdx.x), lane = threadIdx.x & 63;
    if (r >= P.rows) return;
    const size_t rows = (size_t)P.nkv * P.rows, i = (size_t)h * P.rows + r;
    const int seq = r / P.G, c = lane % LANES * 4;
    const size_t to = (size_t)seq * P.nkv * P.G + h * P.G + (r - seq * P.G);
    f32x4 y[READS];
#pragma unroll
    for (int s = 0; s < READS; ++s)  // (past the last part: that one again, which weighs 0 there)
        y[s] = *reinterpret_cast<const f32x4*>(P.part + (min(s * AT + lane / LANES, P.nsplit - 1) * rows + i) * D + c);
    float2 ml = make_float2(-INFINITY, 0.0f);
    if (lane < P.nsplit) ml = *reinterpret_cast<const float2*>(P.ml + 2 * (lane * rows + i));
    const float M = wave_max(ml.x);
    const float e = M == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - M);
    const float Z = wave_sum(ml.y * e);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < READS; ++s) x += y[s] * __shfl(e, s * AT + lane / LANES);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (AT == 4) x[k] = sum_groups(x[k]);
        else x[k] += __shfl_xor(x[k], 32);
    }
    if (lane < LANES) {
        T4 o;
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = from_f<T>(Z > 0.0f ? x[k] / Z : 0.0f);
        *reinterpret_cast<T4*>(out + to * D + c) = o;
    }
    if (lse != nullptr && lane == 0)
        lse[to] = Z > 0.0f ? (M + __builtin_amdgcn_logf(Z)) * 0.69314718055994530942f : -INFINITY;
}

// Wavefronts of the kernel for many rows; 0: the one for few, which reads the
// prefix once per 32 rows but needs no step of all wavefronts per block (us, few
// / many, 8 KV heads: 48 rows, 32768 tokens 32.4 / 35.6, 64 rows 32.6 / 35.2 and
// with 4096 tokens 14.9 / 12.2, 128 rows, 4096 tokens 15.4 / 15.6).
// Four where eight would leave half a tile empty (us, 8 / 4 wavefronts: 368 rows
// of 4 KV heads, 8520 tokens, fp32 87.6 / 73.9, bf16 28.0 / 28.0; 8 KV heads, bf16,
// 128 rows, 4096 tokens 17.3 / 15.5, 124 rows, 8520 tokens 23.0 / 21.7, 384 rows,
// 20000 tokens 63.5 / 58.4).
int wide(int rows) { return rows <= 64 ? 0 : (rows + 127) / 128 % 2 == 1 ? 4 : 8; }
// rows of a workgroup's tile, and the tiles
int row_tile(int rows) { return wide(rows) ? wide(rows) * 16 * kWideTiles : rows <= 16 ? 16 : 32; }
int row_tiles(int rows) { return (rows + row_tile(rows) - 1) / row_tile(rows); }

template <typename T, int D>
void launch_t(const PrefixView& P, const void* q, hipStream_t s) {
    auto go = [&](auto kernel, int waves) {
        hipLaunchKernelGGL(kernel, dim3(P.nkv, row_tiles(P.rows), P.nsplit), dim3(waves * 64), 0, s, P, (const T*)q);
    };
    if (wide(P.rows) == 8) go(k_prefix_wide<T, D, 8>, 8);
    else if (wide(P.rows) == 4) go(k_prefix_wide<T, D, 4>, 4);
    else if (P.rows <= 16) go(k_prefix<T, D, 1>, kWaves);
    else go(k_prefix<T, D, 2>, kWaves);
}

template <typename T, int D>
void join_t(const PrefixView& P, void* out, float* lse, hipStream_t s) {
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(P.nkv, (P.rows + 3) / 4), dim3(256), 0, s, P, (T*)out, lse);
    };
    static_assert(kMaxPrefixParts <= 64, "");
    if (P.nsplit <= 8) go(k_prefix_join<T, D, 8>);
    else if (P.nsplit <= 16) go(k_prefix_join<T, D, 16>);
    else if (P.nsplit <= 32) go(k_prefix_join<T, D, 32>);
    else go(k_prefix_join<T, D, 64>);
}

// workgroups that fill the chip
int workgroups(int rows) { return wide(rows) == 4 ? 512 : 256; }

}  // namespace

int plan_prefix(int nkv, int rows, int tokens, bool bf16) {
    const int bt = bf16 ? 32 : 16, nb = (tokens + bt - 1) / bt;
    const int want = std::min(kMaxPrefixParts, std::max(1, workgroups(rows) / (nkv * row_tiles(rows))));
    int parts;
    if (wide(rows)) {
        // A part takes the time of its blocks, one after the other, and writing and
        // joining its rows takes that of a bf16 block per 4096 rows of all heads:
        // the least of nb / parts + parts * rows / 4096 (us with parts of 8 / 4 blocks
        // / by this rule, 8 KV heads of G = 4: 40 sequences over 700 tokens 18.1 / 14.2
        // / 13.4, 64 over 1024 20.3 / 16.7 / 16.7, 32 over 8192 19.5 / 25.0 / 19.6; an
        // fp32 block is half the tokens at eight times the work: 124 rows, 270 tokens
        // 13.8, with parts of 8 / 4 blocks 22.5 / 18.5).
        parts = (int)lround(sqrt((double)nb * (bf16 ? 4096 : 16384) / ((double)nkv * rows)));
    } else {
        // two blocks per wavefront (us with 1 / 2 / 4: 32 rows, 8192 tokens 16.6 / 16.0
        // / 18.4, 16 rows, 4096 tokens 11.8 / 11.2 / 12.1); of fp32, half the tokens at
        // eight times the work, one (40 rows, 2000 tokens: 22.6, with two 25.6)
        const int least = bf16 ? 2 * kWaves : kWaves;
        parts = (nb + least - 1) / least;
    }
    return std::max(1, std::min({want, parts, nb}));
}

size_t prefix_scratch_rows(int nkv, int rows) {
    // parts * KV heads * tiles stay within the first or the second
    auto most = [&](int r) {
        const int x = nkv * row_tiles(r);
        return (size_t)std::min(std::max(workgroups(r), x), kMaxPrefixParts * x) * row_tile(r);
    };
    // (the most rows of either width, and of the few-rows kernels)
    return std::max({most(std::min(rows, 16)), most(std::min(rows, 64)), most(std::min(rows, 128)),
                     most(rows > 128 ? (rows - 1) / 128 * 128 : rows), most(rows)});
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
