// gfx950 kernels of the weight cache: a per-token cache that evicts by
// accumulated attention weight.
//
// A step of a unit with G query heads q_g, held tokens j and the new token in
// place s (the first free place, else that of the token with the least
// (weight, position) among positions < clock - recent):
//   x_gj = q_g . k_j / sqrt(d);  a_gj = exp(x_gj) / sum_j' exp(x_gj')
//   out_g = sum_j a_gj v_j;      w_j += sum_g a_gj
// where the sums of the softmax run over a shared prefix besides, if there is
// one. The weights need the whole softmax's maximum and sum, so the logits of
// the one pass over the keys are kept (in LDS where one workgroup covers a
// unit, else in scratch) until those are known.
#include <math.h>

#include <algorithm>

#include "raas_blocks.h"
#include "raas_weight_internal.h"

namespace raas {
namespace {

using namespace blk;

// Bytes of dynamic LDS that a step workgroup may use (gfx950 has 160 KiB).
constexpr size_t kStepLds = 144 * 1024;

// ---------------------------------------------------------------------------
// The lightest token: least (weight, position), with its place.
struct Lightest {
    unsigned long long key = ~0ull;  // float_key(weight) << 32 | position
    int place = -1;
    __device__ __forceinline__ void take(unsigned long long k, int p) {
        if (k < key) {
            key = k;
            place = p;
        }
    }
    __device__ __forceinline__ void offer(float w, int pos, int p) {
        take((unsigned long long)float_key(w) << 32 | (uint32_t)pos, p);
    }
};

// Over a workgroup of NT threads; the result is valid on thread 0. Positions
// of a unit differ, so no two keys are equal.
template <int NT>
__device__ __forceinline__ Lightest lightest_wg(Lightest b, int tid) {
    __shared__ unsigned long long s_key[NT / 64];
    __shared__ int s_place[NT / 64];
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const unsigned long long k = __shfl_xor(b.key, d);
        const int p = __shfl_xor(b.place, d);
        b.take(k, p);
    }
    if ((tid & 63) == 0) {
        s_key[tid >> 6] = b.key;
        s_place[tid >> 6] = b.place;
    }
    __syncthreads();
    if (tid == 0)
#pragma unroll
        for (int i = 1; i < NT / 64; ++i) b.take(s_key[i], s_place[i]);
    return b;
}

__device__ __forceinline__ void write_unit(const WeightView& L, int u, int count, int now, const Lightest& b) {
    int4 r;
    r.x = count;
    r.y = now;
    r.z = count < L.C ? count : b.place;
    r.w = count < L.C ? -1 : (int)(uint32_t)b.key;
    *reinterpret_cast<int4*>(L.unit + (size_t)u * kWeightFields) = r;
}

// ---------------------------------------------------------------------------
// Prefill, first part: which tokens of a prompt stay, and the records. Every
// token if they fit, else the `recent` newest and the heaviest others, of equal
// ones the later. One workgroup per unit: a radix select over the weights'
// ordered bits (four 8-bit digits, a histogram each) finds the lightest weight
// that stays, an ordered compaction writes the places in the order of positions.
constexpr int kSelectThreads = 1024;

// Exclusive rank of this thread's flag among the workgroup's, and the total;
// s_n: one int per wavefront, free again after the next barrier but one.
__device__ __forceinline__ int rank_wg(bool flag, int tid, int* s_n, int& total) {
    const unsigned long long m = __ballot(flag);
    const int lane = tid & 63, w = tid >> 6;
    if (lane == 0) s_n[w] = __popcll(m);
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kSelectThreads / 64; ++i) {
        const int n = s_n[i];
        before += i < w ? n : 0;
        total += n;
    }
    return before + __popcll(m & ((1ull << lane) - 1ull));
}

__global__ __launch_bounds__(kSelectThreads) void k_weight_select(WeightView L, const float* __restrict__ weights,
                                                                  SeqLens lens, int seq0, int max_len) {
    __shared__ int s_hist[256], s_pick[2], s_a[kSelectThreads / 64], s_b[kSelectThreads / 64];
    const int tid = threadIdx.x, P = lens.len[blockIdx.x / L.nkv];
    if (P < 0) return;  // not selected
    const int u = seq0 * L.nkv + blockIdx.x, C = L.C;
    const float* wu = weights + (size_t)u * max_len;
    int32_t* pos = L.pos + (size_t)u * C;
    float* w = L.w + (size_t)u * C;
    // (+ 0 turns -0 into 0, which would otherwise rank below it)
    auto weight = [&](int j) { return weights != nullptr ? wu[j] + 0.0f : 0.0f; };
    const int first = max(P - L.recent, 0);  // tokens before it may go
    Lightest best;
    if (P <= C) {
        for (int j = tid; j < C; j += kSelectThreads) {
            const float x = j < P ? weight(j) : 0.0f;
            pos[j] = j < P ? j : -1;
            w[j] = x;
            if (j < first) best.offer(x, j, j);
        }
    } else {
        uint32_t cut = 0;          // digits found so far
        int want = C - L.recent;   // rank from the top among the keys that match them
        int equal = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) s_hist[tid] = 0;
            __syncthreads();
            const uint32_t high = shift == 24 ? 0u : ~0u << (shift + 8);
            for (int j = tid; j < first; j += kSelectThreads) {
                const uint32_t key = float_key(weight(j));
                if ((key & high) == cut) atomicAdd(&s_hist[(key >> shift) & 255u], 1);
            }
            __syncthreads();
            if (tid == 0) {
                int b = 255, left = want;
                while (b > 0 && s_hist[b] < left) left -= s_hist[b--];
                s_pick[0] = b;
                s_pick[1] = left;
            }
            __syncthreads();
            cut |= (uint32_t)s_pick[0] << shift;
            want = s_pick[1];
            equal = s_hist[s_pick[0]];
            __syncthreads();
        }
        const int skip = equal - want;  // the oldest of the tokens at the cut go
        int kept = 0, ties = 0;
        for (int j0 = 0; j0 < P; j0 += kSelectThreads) {
            const int j = j0 + tid;
            const float x = j < P ? weight(j) : 0.0f;
            const uint32_t key = float_key(x);
            const bool tie = j < first && key == cut;
            int nt, nk;
            const int rt = ties + rank_wg(tie, tid, s_a, nt);
            const bool keep = j < P && (j >= first || key > cut || (tie && rt >= skip));
            const int at = kept + rank_wg(keep, tid, s_b, nk);
            if (keep) {
                pos[at] = j;
                w[at] = x;
                if (j < first) best.offer(x, j, at);
            }
            ties += nt;
            kept += nk;
            __syncthreads();
        }
    }
    best = lightest_wg<kSelectThreads>(best, tid);
    if (tid == 0) write_unit(L, u, min(P, C), P, best);
}

// ---------------------------------------------------------------------------
// Prefill, second part, and the store of a shared prefix: one workgroup per
// unit and block. Values turn through LDS; keys are read as their pieces lie.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_store(T* __restrict__ K, T* __restrict__ V, const T* __restrict__ k,
                                               const T* __restrict__ v, StoreIn in, SeqLens lens) {
    constexpr int VE = kVec<T>, BT = kTokens<T>, KS = D / (4 * VE), RP = D / VE;
    __shared__ __align__(16) T s_v[BT][D + VE];
    const int unit = blockIdx.x, tid = threadIdx.x;
    const int P = in.tokens >= 0 ? in.tokens : lens.len[unit / in.nkv];
    const int n = min(P, in.C), u = in.seq0 * in.nkv + unit;  // (a sequence that is not selected has length -1)
    const T* ku = k + (size_t)u * in.stride * D;
    const T* vu = v + (size_t)u * in.stride * D;
    const u32x4 zero = {0u, 0u, 0u, 0u};
    for (int b = blockIdx.y; b * BT < n; b += gridDim.y) {
        const int t0 = b * BT, valid = min(BT, n - t0);
        auto row = [&](int t) { return (size_t)(in.pos != nullptr ? in.pos[(size_t)u * in.C + t0 + t] : t0 + t) * D; };
        T* Kb = K + ((size_t)u * in.pad + t0) * D;
        T* Vb = V + ((size_t)u * in.pad + t0) * D;
        for (int p = tid; p < BT * RP; p += 256) {
            const int t = p / RP, c = p % RP;
            st16(&s_v[t][VE * c], t < valid ? ld16_in<T>(vu + row(t) + VE * c) : zero);
        }
        for (int p = tid; p < BT * RP; p += 256) {
            const int i = p & 15, a = (p >> 4) & 3, ks = (p >> 6) % KS, q = (p >> 6) / KS;
            const int t = VE * (i >> 2) + 4 * q + (i & 3);
            st16(Kb + VE * p, t < valid ? ld16_in<T>(ku + row(t) + 4 * VE * ks + VE * a) : zero);
        }
        __syncthreads();
        for (int p = tid; p < BT * RP; p += 256) {
            const int i = p & 15, a = (p >> 4) & 3, ct = p >> 6;
            u32x4 x = zero;
#pragma unroll
            for (int e = 0; e < VE; ++e) set_elem<T>(x, e, s_v[VE * a + e][16 * ct + i]);
            st16(Vb + VE * p, x);
        }
        __syncthreads();
    }
}

__global__ void k_set_int(int32_t* p, int32_t v) { *p = v; }

// ---------------------------------------------------------------------------
// The end of a step: from the maxima and sums (ml) and unnormalised outputs (o)
// of `nsrc` disjoint parts of the held tokens, and those of the prefix, the
// output; from the logits the weights; the new token's position; the lightest
// token. One workgroup of NT threads.
template <typename T, int D, int NT, class Ml, class O>
__device__ __forceinline__ void finish_step(const WeightView& L, const WeightStepIO& io, int u, const int4& rec,
                                            const float* logits, int lstride, int nsrc, Ml ml, O o) {
    __shared__ float s_m[16], s_rz[16];
    const int tid = threadIdx.x, G = L.G, C = L.C;
    const PrefixParts& pp = io.prefix;
    const size_t rows = (size_t)L.nkv * pp.rows, row0 = (size_t)(u % L.nkv) * pp.rows + (size_t)(u / L.nkv) * G;
    if (tid < G) {
        float M = -INFINITY, Z = 0.0f;
        for (int s = 0; s < nsrc; ++s) M = fmaxf(M, ml(s, tid).x);
        for (int s = 0; s < pp.n; ++s) M = fmaxf(M, pp.ml[2 * (s * rows + row0 + tid)]);
        for (int s = 0; s < nsrc; ++s) Z += ml(s, tid).y * __builtin_amdgcn_exp2f(ml(s, tid).x - M);
        for (int s = 0; s < pp.n; ++s) {
            const float* x = pp.ml + 2 * (s * rows + row0 + tid);
            Z += x[1] * __builtin_amdgcn_exp2f(x[0] - M);
        }
        s_m[tid] = M;
        s_rz[tid] = 1.0f / Z;
    }
    __syncthreads();
    for (int i = tid; i < G * D; i += NT) {
        const int g = i / D, c = i % D;
        const float M = s_m[g];
        float x = 0.0f;
        for (int s = 0; s < nsrc; ++s) x += o(s, g, c) * __builtin_amdgcn_exp2f(ml(s, g).x - M);
        for (int s = 0; s < pp.n; ++s)
            x += pp.o[(s * rows + row0 + g) * D + c] *
                 __builtin_amdgcn_exp2f(pp.ml[2 * (s * rows + row0 + g)] - M);
        ((T*)io.out)[((size_t)u * G + g) * D + c] = from_f<T>(x * s_rz[g]);
    }
    const int now = rec.y, place = rec.z, n = min(rec.x + 1, C), before = now + 1 - L.recent;
    int32_t* pos = L.pos + (size_t)u * C;
    float* w = L.w + (size_t)u * C;
    Lightest best;
    for (int j = tid; j < n; j += NT) {
        float a = 0.0f;
        for (int g = 0; g < G; ++g)
            a += __builtin_amdgcn_exp2f(logits[(size_t)g * lstride + j] - s_m[g]) * s_rz[g];
        const int p = j == place ? now : pos[j];
        const float x = (j == place ? 0.0f : w[j]) + a;
        if (j == place) pos[j] = now;
        w[j] = x;
        if (io.positions_out) io.positions_out[(size_t)u * C + j] = p;
        if (io.weights_out) io.weights_out[(size_t)u * C + j] = x;
        if (p < before) best.offer(x, p, j);
    }
    for (int j = n + tid; j < C; j += NT) {
        if (io.positions_out) io.positions_out[(size_t)u * C + j] = -1;
        if (io.weights_out) io.weights_out[(size_t)u * C + j] = 0.0f;
    }
    if (n == C) best = lightest_wg<NT>(best, tid);
    if (tid == 0) {
        if (io.evicted_out) io.evicted_out[u] = rec.w;
        write_unit(L, u, n, now + 1, best);
    }
}

// ---------------------------------------------------------------------------
// The step: one workgroup of NW wavefronts per (unit, split). A wavefront takes
// every NW-th block of its split, so the order of every sum is fixed; a block
// is read while the one before it is attended to. The new token's row is
// replaced in registers by the wavefront that holds its block, which stores it.
template <typename T, int D, int NW, bool FUSED>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_weight_step(WeightView L,
                                                                                                 WeightStepIO io) {
    constexpr int VE = kVec<T>, BT = kTokens<T>, QT = kTiles<T>, KS = D / (4 * VE), NP = D / 16;
    extern __shared__ __align__(16) float smem[];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, a = lane >> 4, col = lane & 15;
    const int u = blockIdx.x / L.nsplit, split = blockIdx.x - u * L.nsplit;
    if (io.active != nullptr && io.active[u / L.nkv] == 0) return;  // the sequence sits this step out
    const int G = L.G;
    float* s_ml = smem;                    // [NW][16][2]
    float* s_o = s_ml + NW * 32;           // [NW][G][D + 4]
    float* s_x = s_o + NW * G * (D + 4);   // [G][cpad], fused only
    const int4 rec = *reinterpret_cast<const int4*>(L.unit + (size_t)u * kWeightFields);
    const int n = min(rec.x + 1, L.C), nb = (n + BT - 1) / BT, per = (nb + L.nsplit - 1) / L.nsplit;
    const int lo = min(nb, split * per), hi = min(nb, lo + per);
    const int tail = rec.z / BT;  // the block that the new token goes to
    T* Ku = (T*)L.K + (size_t)u * L.cpad * D;
    T* Vu = (T*)L.V + (size_t)u * L.cpad * D;
    const T* kn = (const T*)io.k_new + (size_t)u * D;
    const T* vn = (const T*)io.v_new + (size_t)u * D;
    float* xs = FUSED ? s_x : L.logits + (size_t)u * G * L.cpad;

    u32x4 q[KS];
    load_row<T, D>((const T*)io.q + ((size_t)u * G + col) * D, col < G, a, q);
    Softmax<D> s;
    s.clear();

    auto load = [&](int b, u32x4 (&kr)[NP], u32x4 (&vr)[NP]) {
        const size_t at = (size_t)min(b, nb - 1) * BT * D + lane * VE;
#pragma unroll
        for (int i = 0; i < NP; ++i) kr[i] = ld16(Ku + at + i * 64 * VE);
#pragma unroll
        for (int i = 0; i < NP; ++i) vr[i] = ld16(Vu + at + i * 64 * VE);
    };
    auto block = [&](int b, u32x4 (&kr)[NP], u32x4 (&vr)[NP]) {
        if (b == tail) {
            const int t = rec.z - b * BT, e = t % VE;
            const size_t at = (size_t)b * BT * D + lane * VE;
            if (col == 4 * (t / VE) + t % 4) {
#pragma unroll
                for (int qq = 0; qq < QT; ++qq)
                    if (qq == e / 4)
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            kr[qq * KS + ks] = ld16_in<T>(kn + 4 * VE * ks + VE * a);
                            st16(Ku + at + (qq * KS + ks) * 64 * VE, kr[qq * KS + ks]);
                        }
            }
            if (a == t / VE) {
#pragma unroll
                for (int ct = 0; ct < NP; ++ct) {
                    const T x = vn[16 * ct + col];
#pragma unroll
                    for (int ee = 0; ee < VE; ++ee)
                        if (ee == e) set_elem<T>(vr[ct], ee, x);
                    st16(Vu + at + ct * 64 * VE, vr[ct]);
                }
            }
        }
        const int valid = min(BT, n - b * BT);
        if (valid < BT) {  // places that hold no token weigh 0 whatever is stored there
#pragma unroll
            for (int ct = 0; ct < NP; ++ct) zero_from<T>(vr[ct], valid - VE * a);
        }
        f32x4 x[QT];
        attend<T, D>(kr, vr, q, valid, a, L.scale_log2, s, x);
        if (col < G)
#pragma unroll
            for (int t = 0; t < QT; ++t)
                *reinterpret_cast<f32x4*>(xs + (size_t)col * L.cpad + b * BT + VE * a + 4 * t) = x[t];
    };

    if (lo + w < hi) {
        u32x4 k0[NP], v0[NP], k1[NP], v1[NP];
        int b = lo + w;
        load(b, k0, v0);
        while (true) {
            load(b + NW, k1, v1);
            block(b, k0, v0);
            b += NW;
            if (b >= hi) break;
            load(b + NW, k0, v0);
            block(b, k1, v1);
            b += NW;
            if (b >= hi) break;
        }
    }
    s.l = sum_groups(s.l);
    if (col < G) {
        if (a == 0) {
            s_ml[2 * (w * 16 + col)] = s.m;
            s_ml[2 * (w * 16 + col) + 1] = s.l;
        }
#pragma unroll
        for (int ct = 0; ct < NP; ++ct)
            *reinterpret_cast<f32x4*>(s_o + (size_t)(w * G + col) * (D + 4) + 16 * ct + 4 * a) = s.o[ct];
    }
    __syncthreads();
    auto ml = [&](int i, int g) { return make_float2(s_ml[2 * (i * 16 + g)], s_ml[2 * (i * 16 + g) + 1]); };
    auto o = [&](int i, int g, int c) { return s_o[(size_t)(i * G + g) * (D + 4) + c]; };
    if constexpr (FUSED) {
        finish_step<T, D, NW * 64>(L, io, u, rec, s_x, L.cpad, NW, ml, o);
    } else {
        const size_t part = (size_t)u * L.nsplit + split;
        for (int i = tid; i < G * D; i += NW * 64) {
            const int g = i / D, c = i % D;
            float M = -INFINITY, x = 0.0f, z = 0.0f;
#pragma unroll
            for (int k = 0; k < NW; ++k) M = fmaxf(M, ml(k, g).x);
            const float ref = M == -INFINITY ? 0.0f : M;  // a split may hold no token
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                const float e = __builtin_amdgcn_exp2f(ml(k, g).x - ref);
                x += o(k, g, c) * e;
                z += ml(k, g).y * e;
            }
            L.part[(part * G + g) * D + c] = x;
            if (c == 0) {
                L.ml[2 * (part * G + g)] = M;
                L.ml[2 * (part * G + g) + 1] = z;
            }
        }
    }
}

// The end of a step whose units are split: one workgroup per unit.
constexpr int kFinishThreads = 1024;
template <typename T, int D>
__global__ __launch_bounds__(kFinishThreads) void k_weight_finish(WeightView L, WeightStepIO io) {
    const int u = blockIdx.x, G = L.G;
    if (io.active != nullptr && io.active[u / L.nkv] == 0) return;
    const int4 rec = *reinterpret_cast<const int4*>(L.unit + (size_t)u * kWeightFields);
    const float* mlp = L.ml + (size_t)u * L.nsplit * G * 2;
    const float* part = L.part + (size_t)u * L.nsplit * G * D;
    auto ml = [&](int i, int g) { return make_float2(mlp[2 * (i * G + g)], mlp[2 * (i * G + g) + 1]); };
    auto o = [&](int i, int g, int c) { return part[(size_t)(i * G + g) * D + c]; };
    finish_step<T, D, kFinishThreads>(L, io, u, rec, L.logits + (size_t)u * G * L.cpad, L.cpad, L.nsplit, ml, o);
}

size_t step_lds(int G, int D, int cpad, int nw, bool fused) {
    return sizeof(float) * ((size_t)nw * 32 + (size_t)nw * G * (D + 4) + (fused ? (size_t)G * cpad : 0));
}

template <typename T, int D>
hipError_t launch_step_t(const WeightView& L, const WeightStepIO& io, const WeightPlan& p, hipStream_t s) {
    const dim3 grid((unsigned)L.U * p.nsplit), wg(p.waves * 64);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, wg, p.lds, s, L, io); };
    if (p.waves == 8) p.fused ? go(k_weight_step<T, D, 8, true>) : go(k_weight_step<T, D, 8, false>);
    else p.fused ? go(k_weight_step<T, D, 4, true>) : go(k_weight_step<T, D, 4, false>);
    if (!p.fused)
        hipLaunchKernelGGL((k_weight_finish<T, D>), dim3(L.U), dim3(kFinishThreads), 0, s, L, io);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t allow_t() {
    hipError_t e = hipSuccess;
    for (const void* f : {(const void*)k_weight_step<T, D, 8, true>, (const void*)k_weight_step<T, D, 8, false>,
                          (const void*)k_weight_step<T, D, 4, true>, (const void*)k_weight_step<T, D, 4, false>}) {
        const hipError_t r = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kStepLds);
        if (r != hipSuccess) e = r;
    }
    return e;
}

template <typename T, int D>
void launch_store_t(void* K, void* V, const void* k, const void* v, const StoreIn& in, const SeqLens& lens, int units,
                    int most, hipStream_t s) {
    const int nblk = (most + kTokens<T> - 1) / kTokens<T>;
    if (nblk > 0)
        hipLaunchKernelGGL((k_store<T, D>), dim3(units, std::min(nblk, 65535)), dim3(256), 0, s, (T*)K, (T*)V,
                           (const T*)k, (const T*)v, in, lens);
}

void launch_store(int D, bool bf16, void* K, void* V, const void* k, const void* v, const StoreIn& in,
                  const SeqLens& lens, int units, int most, hipStream_t s) {
    auto go = [&](auto f) { f(K, V, k, v, in, lens, units, most, s); };
    if (bf16) D == 128 ? go(launch_store_t<uint16_t, 128>) : go(launch_store_t<uint16_t, 64>);
    else D == 128 ? go(launch_store_t<float, 128>) : go(launch_store_t<float, 64>);
}

}  // namespace

WeightPlan plan_weight_step(int U, int G, int D, int C, bool bf16) {
    const int bt = bf16 ? 32 : 16, nb = (C + bt - 1) / bt, cpad = nb * bt;
    WeightPlan p{};
    p.waves = 8;
    if (step_lds(G, D, cpad, 8, false) > kStepLds / 2) p.waves = 4;
    const int want = std::min(std::max(512 / U, 1), std::max(1, nb / p.waves));
    p.fused = want == 1 && step_lds(G, D, cpad, p.waves, true) <= kStepLds;
    p.nsplit = p.fused ? 1 : std::max(want, 1);
    p.lds = step_lds(G, D, cpad, p.waves, p.fused);
    return p;
}

hipError_t weight_allow_lds(bool bf16, int D) {
    if (bf16) return D == 128 ? allow_t<uint16_t, 128>() : allow_t<uint16_t, 64>();
    return D == 128 ? allow_t<float, 128>() : allow_t<float, 64>();
}

hipError_t launch_weight_prefill(const WeightView& L, bool bf16, const void* k, const void* v, const float* weights,
                                 const SeqLens& lens, int seq0, int nseq, int max_len, hipStream_t s) {
    hipLaunchKernelGGL(k_weight_select, dim3((unsigned)nseq * L.nkv), dim3(kSelectThreads), 0, s, L, weights, lens,
                       seq0, max_len);
    int most = 0;
    for (int i = 0; i < nseq; ++i) most = std::max(most, std::min(lens.len[i], L.C));
    StoreIn in{L.pos, L.C, L.cpad, L.nkv, seq0, max_len, -1};
    launch_store(L.D, bf16, L.K, L.V, k, v, in, lens, nseq * L.nkv, most, s);
    return hipGetLastError();
}

hipError_t launch_weight_step(const WeightView& L, bool bf16, const WeightStepIO& io, const WeightPlan& p,
                              hipStream_t s) {
    if (bf16) return L.D == 128 ? launch_step_t<uint16_t, 128>(L, io, p, s) : launch_step_t<uint16_t, 64>(L, io, p, s);
    return L.D == 128 ? launch_step_t<float, 128>(L, io, p, s) : launch_step_t<float, 64>(L, io, p, s);
}

hipError_t launch_prefix_store(void* K, void* V, int32_t* len, int nkv, int D, int tpad, bool bf16, const void* k,
                               const void* v, int tokens, hipStream_t s) {
    SeqLens none{};
    StoreIn in{nullptr, tokens, tpad, nkv, 0, tokens, tokens};
    launch_store(D, bf16, K, V, k, v, in, none, nkv, tokens, s);
    hipLaunchKernelGGL(k_set_int, dim3(1), dim3(1), 0, s, len, tokens);
    return hipGetLastError();
}

}  // namespace raas
