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
#include <type_traits>

#include "raas_blocks.h"
#include "raas_weight_internal.h"

namespace raas {
namespace {

using namespace blk;

// Bytes of dynamic LDS that a step workgroup may use (gfx950 has 160 KiB).
constexpr size_t kStepLds = 156 * 1024;

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
// of a unit differ, so no two keys are equal (but those of no token).
template <int NT>
__device__ __forceinline__ Lightest lightest_wg(Lightest b, int tid) {
    __shared__ unsigned long long s_key[NT / 64];
    __shared__ int s_place[NT / 64];
    const unsigned long long least = wave_min(b.key);
    if (b.key == least && (b.place >= 0 || (tid & 63) == 0)) {
        s_key[tid >> 6] = least;
        s_place[tid >> 6] = b.place;
    }
    lds_barrier();
    if (tid == 0)
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) b.take(s_key[i], s_place[i]);
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
    __shared__ int s_hist[256], s_pick[3], s_a[kSelectThreads / 64], s_b[kSelectThreads / 64];
    const int tid = threadIdx.x, P = lens.len[blockIdx.x / L.nkv];
    if (P < 0) return;  // not selected
    const int u = seq0 * L.nkv + blockIdx.x, C = L.C;
    const float* wu = weights + (size_t)u * max_len;
    int32_t* pos = L.pos + (size_t)u * L.cpad;
    float* w = L.w + (size_t)u * L.cpad;
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
            if (tid < 64) {  // lane l: bins 255 - 4 l and the three below, from the top
                int n[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += n[i] = s_hist[255 - 4 * tid - i];
                int upto = sum;  // keys in this lane's bins and all above
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int y = __shfl_up(upto, d);
                    if (tid >= d) upto += y;
                }
                int left = want - (upto - sum);  // rank from the top within this lane's bins
                if (left > 0 && left <= sum) {
                    int i = 0, held = n[0];
#pragma unroll
                    for (int k = 1; k < 4; ++k)
                        if (i == k - 1 && left > held) {
                            left -= held;
                            i = k;
                            held = n[k];
                        }
                    s_pick[0] = 255 - 4 * tid - i;
                    s_pick[1] = left;
                    s_pick[2] = held;
                }
            }
            __syncthreads();
            cut |= (uint32_t)s_pick[0] << shift;
            want = s_pick[1];
            equal = s_pick[2];
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
        auto row = [&](int t) { return (size_t)(in.pos != nullptr ? in.pos[(size_t)u * in.pad + t0 + t] : t0 + t) * D; };
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
// Hand-over between workgroups of one launch. The XCDs' L2s are not coherent
// with each other, so what crosses is written through and read past them (agent
// scope); once a wavefront's stores are acknowledged every XCD reads them.
template <typename T>
__device__ __forceinline__ void publish(T* p, T v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ __forceinline__ T published(const T* p) {
    return __hip_atomic_load(const_cast<T*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void publish4(float* p, f32x4 v) {  // p: 16-byte aligned
    unsigned long long* q = reinterpret_cast<unsigned long long*>(p);
    publish(q, (unsigned long long)__float_as_uint(v[1]) << 32 | __float_as_uint(v[0]));
    publish(q + 1, (unsigned long long)__float_as_uint(v[3]) << 32 | __float_as_uint(v[2]));
}
__device__ __forceinline__ f32x4 published4(const float* p) {
    const unsigned long long* q = reinterpret_cast<const unsigned long long*>(p);
    const unsigned long long x = published(q), y = published(q + 1);
    return f32x4{__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32)), __uint_as_float((uint32_t)y),
                 __uint_as_float((uint32_t)(y >> 32))};
}
// True on the last of `total` workgroups to call it for this counter, once all
// that they published is readable; the counter is zero again afterwards. No
// workgroup waits for another.
__device__ __forceinline__ bool arrive_last(int32_t* counter, int total) {
    __shared__ int s_last;
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (threadIdx.x == 0) {
        const int before = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before == total - 1) publish(counter, 0);
        s_last = before == total - 1;
    }
    __syncthreads();
    return s_last != 0;
}

// ---------------------------------------------------------------------------
// The end of a step: from the maxima and sums (ml) and unnormalised outputs (o)
// of `nsrc` disjoint parts of the held tokens, and those of the prefix, the
// output (if j_lo is 0); from the logits (x4: those of four tokens) the weights
// of places j_lo .. j_hi - 1; the new token's position; the lightest token among
// those places (thread 0's result). One workgroup of NW wavefronts; s_w: [nsrc +
// prefix parts][G] floats of LDS. A wavefront per head finds the maximum and the
// sum, a lane per part; a thread takes four tokens at a time.
typedef int32_t i32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// Positions and weights of four tokens.
struct Records {
    i32x4 p = {0, 0, 0, 0};
    f32x4 w = {0.f, 0.f, 0.f, 0.f};
    template <bool STREAM>
    __device__ __forceinline__ void load(const WeightView& L, int u, int j, int n) {
        if (j >= n) return;
        const i32x4* from = reinterpret_cast<const i32x4*>(L.pos + (size_t)u * L.cpad + j);
        const f32x4* wfrom = reinterpret_cast<const f32x4*>(L.w + (size_t)u * L.cpad + j);
        p = STREAM ? __builtin_nontemporal_load(from) : *from;
        w = STREAM ? __builtin_nontemporal_load(wfrom) : *wfrom;
    }
};

// `now`: the records of this thread's first tokens, j_lo + 4 tid + i STEP on, which the
// caller has had on their way for a while. (All of a group's reads come before
// its first write: a wait for a read that follows a write waits for the write.)
constexpr int kRecords = 4;
template <int NW, bool STREAM>
__device__ __forceinline__ void load_records(const WeightView& L, int u, int j, int n, Records (&now)[kRecords]) {
#pragma unroll
    for (int i = 0; i < kRecords; ++i) now[i].load<STREAM>(L, u, j + i * NW * 256, n);
}

// x += the first n parts' values by their shares, N of them on their way together
// (past the last part: that one again, without weight).
template <int N, class Value, class Share>
__device__ __forceinline__ void add_parts(float& x, int n, Value value, Share share) {
    for (int s0 = 0; s0 < n; s0 += N) {
        float y[N];
#pragma unroll
        for (int k = 0; k < N; ++k) y[k] = value(min(s0 + k, n - 1));
#pragma unroll
        for (int k = 0; k < N; ++k) x = __builtin_fmaf(y[k], s0 + k < n ? share(s0 + k) : 0.0f, x);
    }
}

// The outputs are written past the caches, and the records read and written so
// where the layer does not stay in them (STREAM): as lines leave an L2 by
// themselves, writes come between the other units' reads (128 sequences of 8 KV
// heads, 8192 tokens: 804 us; the outputs past the caches 752, the weights too
// 746, the records' reads too 729).
template <typename T, int D, int NW, bool STREAM, class Ml, class O, class X4>
__device__ __forceinline__ Lightest finish_step(const WeightView& L, const WeightStepIO& io, int u, const int4& rec,
                                                int tid, int j_lo, int j_hi, Records (&now)[kRecords], int nsrc,
                                                float* s_w, Ml ml, O o, X4 x4) {
    constexpr int NT = NW * 64, STEP = NT * 4;
    __shared__ float s_m[16], s_rz[16];
    const int lane = tid & 63, w = wave_of(tid), G = L.G, C = L.C;
    const PrefixParts& pp = io.prefix;
    const size_t rows = (size_t)L.nkv * pp.rows, row0 = (size_t)(u % L.nkv) * pp.rows + (size_t)(u / L.nkv) * G;
    const int clock = rec.y, place = rec.z, n = min(rec.x + 1, C), before = clock + 1 - L.recent;
    int32_t* pos = L.pos + (size_t)u * L.cpad;
    float* wt = L.w + (size_t)u * L.cpad;
    const int parts = nsrc + pp.n;
    for (int g = w; g < G; g += NW) {
        auto part_ml = [&](int s) {
            if (s < nsrc) return ml(s, g);
            const float* x = pp.ml + 2 * ((size_t)(s - nsrc) * rows + row0 + g);
            return make_float2(x[0], x[1]);
        };
        float M = -INFINITY, Z = 0.0f;
        const float2 first = lane < parts ? part_ml(lane) : make_float2(-INFINITY, 0.0f);
        M = first.x;
        for (int s = lane + 64; s < parts; s += 64) M = fmaxf(M, part_ml(s).x);
        M = wave_max(M);
        Z = first.y * __builtin_amdgcn_exp2f(first.x - M);
        for (int s = lane + 64; s < parts; s += 64) {
            const float2 y = part_ml(s);
            Z += y.y * __builtin_amdgcn_exp2f(y.x - M);
        }
        Z = wave_sum(Z);
        const float rz = 1.0f / Z;
        if (lane < parts) s_w[lane * G + g] = __builtin_amdgcn_exp2f(first.x - M) * rz;
        for (int s = lane + 64; s < parts; s += 64) s_w[s * G + g] = __builtin_amdgcn_exp2f(part_ml(s).x - M) * rz;
        if (lane == 0) {
            s_m[g] = M;
            s_rz[g] = rz;
        }
    }
    lds_barrier();
    for (int i = tid; i < (j_lo == 0 ? G * D : 0); i += NT) {
        const int g = i / D, c = i % D;
        float x = 0.0f;
        add_parts<8>(x, nsrc, [&](int s) { return o(s, g, c); }, [&](int s) { return s_w[s * G + g]; });
        add_parts<8>(
            x, pp.n, [&](int s) { return pp.o[(s * rows + row0 + g) * D + c]; },
            [&](int s) { return s_w[(nsrc + s) * G + g]; });
        ((T*)io.out)[((size_t)u * G + g) * D + c] = from_f<T>(x);
    }
    Lightest best;
    const int end = min(j_hi, io.positions_out != nullptr || io.weights_out != nullptr ? C : n);
    for (int j0 = j_lo + 4 * tid; j0 < end; j0 += kRecords * STEP) {
        if (j0 > j_lo + 4 * tid) load_records<NW, STREAM>(L, u, j0, n, now);
#pragma unroll
        for (int i = 0; i < kRecords; ++i) {
            const int j = j0 + i * STEP;
            if (j >= end) break;
            f32x4 a = {0.f, 0.f, 0.f, 0.f};
            if (j < n) {
#pragma unroll 4
                for (int g = 0; g < G; ++g) {
                    const f32x4 x = x4(g, j);
                    const float M = s_m[g], rz = s_rz[g];
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[e] = __builtin_fmaf(__builtin_amdgcn_exp2f(x[e] - M), rz, a[e]);
                }
            }
            i32x4& p4 = now[i].p;
            f32x4& w4 = now[i].w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool fresh = j + e == place, held = j + e < n;
                p4[e] = fresh ? clock : held ? p4[e] : -1;
                w4[e] = held ? (fresh ? 0.0f : w4[e]) + a[e] : 0.0f;
                if (held && p4[e] < before) best.offer(w4[e], p4[e], j + e);
            }
            if (j < n) {
                if constexpr (STREAM) __builtin_nontemporal_store(w4, reinterpret_cast<f32x4*>(wt + j));
                else *reinterpret_cast<f32x4*>(wt + j) = w4;
                if (place >= j && place < j + 4) pos[place] = clock;
            }
            if (j + 4 <= C) {
                if (io.positions_out)
                    __builtin_nontemporal_store(p4, reinterpret_cast<i32x4_at4*>(io.positions_out + (size_t)u * C + j));
                if (io.weights_out)
                    __builtin_nontemporal_store(w4, reinterpret_cast<f32x4_at4*>(io.weights_out + (size_t)u * C + j));
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (j + e < C) {
                        if (io.positions_out) io.positions_out[(size_t)u * C + j + e] = p4[e];
                        if (io.weights_out) io.weights_out[(size_t)u * C + j + e] = w4[e];
                    }
            }
        }
    }
    return n == C ? lightest_wg<NT>(best, tid) : best;
}

// The record after a step whose lightest token is `best`; one thread.
__device__ __forceinline__ void step_done(const WeightView& L, const WeightStepIO& io, int u, const int4& rec,
                                          const Lightest& best) {
    if (io.evicted_out) io.evicted_out[u] = rec.w;
    write_unit(L, u, min(rec.x + 1, L.C), rec.y + 1, best);
}

// ---------------------------------------------------------------------------
// The step. Split s of a unit takes every nsplit-th block, a wavefront every
// NW-th of those, so the order of every sum is fixed and the work is even
// however many tokens are held; a block is read while the one before it is
// attended to. The new token's row is replaced in registers by the wavefront
// that holds its block, which stores it. Bound by memory: 32 KB per wavefront
// are on their way or in use.
// FUSED: one workgroup covers a unit and keeps the logits in LDS. Else one per
// (unit, split), and the last of a unit's to end finishes the step from what all
// of them published, or (finish_parts) a kernel of several workgroups per unit
// does. STREAM: non-temporal loads.
template <typename T, int D, int NW, bool FUSED, bool STREAM>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_weight_step(WeightView L,
                                                                                                 WeightStepIO io) {
    constexpr int VE = kVec<T>, BT = kTokens<T>, QT = kTiles<T>, KS = D / (4 * VE), NP = D / 16;
    extern __shared__ __align__(16) float smem[];
    const int tid = threadIdx.x, lane = tid & 63, w = wave_of(tid), a = lane >> 4, col = lane & 15;
    const int G = L.G, nsplit = FUSED ? 1 : L.nsplit, last_block = L.cpad / BT - 1, step = NW * nsplit;
    float* s_ml = smem;                    // [NW][16][2]
    float* s_w = s_ml + NW * 32;           // [parts][G], 16-byte multiple
    float* s_o = s_w + L.wfloats;          // [NW][G][D + 4]
    float* s_x = s_o + NW * G * (D + 4);   // [G][cpad], fused only
    const int u = FUSED ? blockIdx.x : blockIdx.x / nsplit, split = FUSED ? 0 : blockIdx.x - u * nsplit;
    if (io.active != nullptr && io.active[u / L.nkv] == 0) return;  // the sequence sits this step out

    u32x4 k0[NP], v0[NP], k1[NP], v1[NP], q[KS];
    auto load = [&](int b, u32x4 (&kr)[NP], u32x4 (&vr)[NP]) {
        const size_t at = ((size_t)u * L.cpad + (size_t)min(b, last_block) * BT) * D + lane * VE;
        const T *Kb = (const T*)L.K + at, *Vb = (const T*)L.V + at;
#pragma unroll
        for (int i = 0; i < NP; ++i) kr[i] = STREAM ? ld16_nt(Kb + i * 64 * VE) : ld16(Kb + i * 64 * VE);
#pragma unroll
        for (int i = 0; i < NP; ++i) vr[i] = STREAM ? ld16_nt(Vb + i * 64 * VE) : ld16(Vb + i * 64 * VE);
    };
    // (the first block's place does not depend on the record, which arrives meanwhile)
    load(split + nsplit * w, k0, v0);
    const int4 rec = *reinterpret_cast<const int4*>(L.unit + (size_t)u * kWeightFields);
    load_row<T, D>((const T*)io.q + ((size_t)u * G + col) * D, col < G, a, q);
    const int n = min(rec.x + 1, L.C), nb = (n + BT - 1) / BT;
    const int tail = rec.z / BT;  // the block that the new token goes to
    float* xs = FUSED ? s_x : L.logits + (size_t)u * G * L.cpad;
    Softmax<D> s;
    s.clear();
    auto block = [&](int b, u32x4 (&kr)[NP], u32x4 (&vr)[NP]) {
        if (b == tail) {
            const T* kn = (const T*)io.k_new + (size_t)u * D;
            const T* vn = (const T*)io.v_new + (size_t)u * D;
            const int t = rec.z - b * BT, e = t % VE;
            const size_t at = ((size_t)u * L.cpad + (size_t)b * BT) * D + lane * VE;
            if (col == 4 * (t / VE) + t % 4) {
#pragma unroll
                for (int qq = 0; qq < QT; ++qq)
                    if (qq == e / 4)
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            kr[qq * KS + ks] = ld16_in<T>(kn + 4 * VE * ks + VE * a);
                            st16((T*)L.K + at + (qq * KS + ks) * 64 * VE, kr[qq * KS + ks]);
                        }
            }
            if (a == t / VE) {
#pragma unroll
                for (int ct = 0; ct < NP; ++ct) {
                    const T x = vn[16 * ct + col];
#pragma unroll
                    for (int ee = 0; ee < VE; ++ee)
                        if (ee == e) set_elem<T>(vr[ct], ee, x);
                    st16((T*)L.V + at + ct * 64 * VE, vr[ct]);
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
            for (int t = 0; t < QT; ++t) {
                float* to = xs + (size_t)col * L.cpad + b * BT + VE * a + 4 * t;
                if constexpr (FUSED) *reinterpret_cast<f32x4*>(to) = x[t];
                else publish4(to, x[t]);
            }
    };
    for (int b = split + nsplit * w; b < nb;) {
        load(b + step, k1, v1);
        block(b, k0, v0);
        b += step;
        if (b >= nb) break;
        load(b + step, k0, v0);
        block(b, k1, v1);
        b += step;
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
    Records first[kRecords];
    if constexpr (FUSED) load_records<NW, STREAM>(L, u, 4 * tid, n, first);
    lds_barrier();
    auto ml = [&](int i, int g) { return make_float2(s_ml[2 * (i * 16 + g)], s_ml[2 * (i * 16 + g) + 1]); };
    auto o = [&](int i, int g, int c) { return s_o[(size_t)(i * G + g) * (D + 4) + c]; };
    if constexpr (FUSED) {
        auto x4 = [&](int g, int j) { return *reinterpret_cast<const f32x4*>(s_x + (size_t)g * L.cpad + j); };
        const Lightest best = finish_step<T, D, NW, STREAM>(L, io, u, rec, tid, 0, L.C, first, NW, s_w, ml, o, x4);
        if (tid == 0) step_done(L, io, u, rec, best);
    } else {
        float* mlp = L.ml + (size_t)u * nsplit * G * 2;
        float* part = L.part + (size_t)u * nsplit * G * D;
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
            publish(part + (size_t)(split * G + g) * D + c, x);
            if (c == 0) {
                publish(mlp + 2 * (split * G + g), M);
                publish(mlp + 2 * (split * G + g) + 1, z);
            }
        }
        if (L.finish_parts > 0 || !arrive_last(L.arrived + u, nsplit)) return;
        load_records<NW, STREAM>(L, u, 4 * tid, n, first);
        auto gml = [&](int i, int g) {
            return make_float2(published(mlp + 2 * (i * G + g)), published(mlp + 2 * (i * G + g) + 1));
        };
        auto go = [&](int i, int g, int c) { return published(part + (size_t)(i * G + g) * D + c); };
        auto x4 = [&](int g, int j) { return published4(xs + (size_t)g * L.cpad + j); };
        const Lightest best = finish_step<T, D, NW, STREAM>(L, io, u, rec, tid, 0, L.C, first, nsplit, s_w, gml, go, x4);
        if (tid == 0) step_done(L, io, u, rec, best);
    }
}

// The end of a step of split units with many tokens: finish_parts workgroups per
// unit, which take a range of its places each; the last to end picks the
// lightest token. (One CU reads what the splits left at some 20 GB/s.)
constexpr int kFinishWaves = 8;
constexpr int kFinishPlaces = 2048;  // of a workgroup: four a thread
template <typename T, int D>
__global__ __launch_bounds__(kFinishWaves * 64) void k_weight_finish(WeightView L, WeightStepIO io) {
    __shared__ float s_w[(kMaxStepSplits + kMaxPrefixParts) * 16];
    const int tid = threadIdx.x, parts = L.finish_parts, u = blockIdx.x / parts, part = blockIdx.x - u * parts;
    if (io.active != nullptr && io.active[u / L.nkv] == 0) return;
    const int G = L.G, nsplit = L.nsplit, j_lo = part * kFinishPlaces;
    const int4 rec = *reinterpret_cast<const int4*>(L.unit + (size_t)u * kWeightFields);
    const float* mlp = L.ml + (size_t)u * nsplit * G * 2;
    const float* po = L.part + (size_t)u * nsplit * G * D;
    const float* xs = L.logits + (size_t)u * G * L.cpad;
    Records first[kRecords];
    load_records<kFinishWaves, false>(L, u, j_lo + 4 * tid, min(min(rec.x + 1, L.C), j_lo + kFinishPlaces), first);
    auto ml = [&](int i, int g) { return *reinterpret_cast<const float2*>(mlp + 2 * (i * G + g)); };
    auto o = [&](int i, int g, int c) { return po[(size_t)(i * G + g) * D + c]; };
    auto x4 = [&](int g, int j) { return *reinterpret_cast<const f32x4*>(xs + (size_t)g * L.cpad + j); };
    const Lightest mine = finish_step<T, D, kFinishWaves, false>(L, io, u, rec, tid, j_lo, min(L.C, j_lo + kFinishPlaces), first,
                                                          nsplit, s_w, ml, o, x4);
    unsigned long long* best = L.best + 2 * ((size_t)u * parts);
    if (tid == 0) {
        publish(best + 2 * part, mine.key);
        publish(best + 2 * part + 1, (unsigned long long)(long long)mine.place);
    }
    if (!arrive_last(L.arrived + u, parts)) return;
    Lightest b;
    for (int i = tid; i < parts; i += kFinishWaves * 64) b.take(published(best + 2 * i), (int)published(best + 2 * i + 1));
    b = lightest_wg<kFinishWaves * 64>(b, tid);
    if (tid == 0) step_done(L, io, u, rec, b);
}

// Floats of the parts' shares: those of the workgroup's wavefronts or splits, and of the prefix.
int share_floats(int G, int parts) { return (G * parts + 3) / 4 * 4; }

// A split unit's step ends in a kernel of its own beyond this many bytes (us, in
// the step kernel / of its own, 8 KV heads of G = 4: 2 sequences of 6000 tokens
// 22.4 / 22.5, 4 of 8201 44.4 / 42.4, 1 of 16384 34.8 / 27.5; 4 of 3000 20.0 /
// 22.2).
constexpr double kFinishBytes = 220e3;

// What the splits of a unit are chosen by, in us: a workgroup takes a fixed time
// and its blocks one after the other, each as long as its latency where few
// workgroups run and as long as its bytes where all do; the end of a unit that is
// not covered by one workgroup takes more, and more with every head (C 1024 in 4
// splits against none, 8 units: G 1 11.6 / 11.7, 4 12.3 / 12.0, 7 14.2 / 12.4; in 3,
// C 900, G 16 17.8 / 13.6).
constexpr double kFixed = 5.0, kSplitEnd = 2.3, kSplitEndHead = 0.4;
// a block alone, and its bytes' time with 256 workgroups (16 KB at head_dim 128)
double block_alone(int D, bool bf16) { return bf16 ? (D == 128 ? 0.12 : 0.08) : (D == 128 ? 0.32 : 0.15); }
double block_full(int D) { return D == 128 ? 0.62 : 0.31; }

size_t step_lds(int G, int D, int cpad, int nw, bool fused, int parts) {
    return sizeof(float) * ((size_t)nw * 32 + share_floats(G, parts) + (size_t)nw * G * (D + 4) +
                            (fused ? (size_t)G * cpad : 0));
}

template <typename T, int D, int NW>
hipError_t launch_step_t(const WeightView& L, const WeightStepIO& io, const WeightPlan& p, bool stream, size_t lds,
                         hipStream_t s) {
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)L.U * p.nsplit), dim3(NW * 64), lds, s, L, io);
        if (p.finish_parts > 0)
            hipLaunchKernelGGL((k_weight_finish<T, D>), dim3((unsigned)L.U * p.finish_parts), dim3(kFinishWaves * 64), 0,
                               s, L, io);
        return hipGetLastError();
    };
    if (stream) return p.fused ? go(k_weight_step<T, D, NW, true, true>) : go(k_weight_step<T, D, NW, false, true>);
    return p.fused ? go(k_weight_step<T, D, NW, true, false>) : go(k_weight_step<T, D, NW, false, false>);
}

template <typename T, int D, int NW>
hipError_t allow_t() {
    hipError_t e = hipSuccess;
    for (const void* f : {(const void*)k_weight_step<T, D, NW, true, false>, (const void*)k_weight_step<T, D, NW, true, true>,
                          (const void*)k_weight_step<T, D, NW, false, false>,
                          (const void*)k_weight_step<T, D, NW, false, true>}) {
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
    auto fits = [&](int nw, int per_cu) {
        return per_cu * (step_lds(G, D, cpad, nw, true, nw + kMaxPrefixParts) + 1024) <= kStepLds;
    };
    p.waves = 8;
    // more units than CUs: two workgroups of 4 wavefronts per CU, so that one
    // unit's finish overlaps another's reads (us, 8 / 4 wavefronts, 8 KV heads: 40
    // sequences of 3000 tokens 118.4 / 104.6, 64 of 1024 57.2 / 52.6, 100 of 512
    // 64.8 / 52.0, 128 of 2048 199.5 / 197.5)
    if (U > 256 && fits(4, 2)) p.waves = 4;
    // Splits: the number that ends soonest when `per` workgroups run at a time
    // (us, one workgroup a unit / split, 8 KV heads of G = 4: 1 sequence of 1024
    // tokens 12.0 / 12.3, of 2048 16.0 / 12.7, 4 of 2048 18.9 / 15.6, 16 of 1024 17.3 /
    // 21.0, 16 of 2048 26.8 / 32.6, 19 of 4963 72.1 / 92.5, 82 of 2760 174 / 210; 4 KV
    // heads of G = 7, 32 of 3201 39.0 / 55.0).
    const int per = p.waves == 8 ? 256 : 512;
    int want = 1;
    double best = 0.0;
    // (a layer beyond the memory-side cache: its blocks take longer to come)
    const double alone = block_alone(D, bf16) + (2.0 * U * cpad * D * (bf16 ? 2 : 4) > 256e6 ? 0.08 : 0.0);
    for (int ns = 1; ns <= kMaxStepSplits && (ns == 1 || nb >= ns * p.waves); ++ns) {
        const double end = ns == 1 && fits(p.waves, 1) ? 0.0 : kSplitEnd + kSplitEndHead * G;
        auto round = [&](long long workgroups) {
            const double full = block_full(D) * workgroups / 256;
            return (nb + ns - 1) / ns * std::max(alone + 0.58 * full, full) + kFixed + end;
        };
        const long long all = (long long)U * ns, rest = all % per;
        const double cost = all / per * round(per) + (rest > 0 ? round(rest) : 0.0);
        if (ns == 1 || cost < best) {
            best = cost;
            want = ns;
        }
    }
    p.fused = want == 1 && fits(p.waves, 1);
    p.nsplit = want;
    // (bytes that the end of a unit's step reads and writes)
    p.finish_parts = !p.fused && (double)C * (4 * G + 20) > kFinishBytes ? (C + kFinishPlaces - 1) / kFinishPlaces : 0;
    return p;
}

hipError_t weight_allow_lds(bool bf16, int D, int waves) {
    auto go = [&](auto w) {
        constexpr int NW = decltype(w)::value;
        if (bf16) return D == 128 ? allow_t<uint16_t, 128, NW>() : allow_t<uint16_t, 64, NW>();
        return D == 128 ? allow_t<float, 128, NW>() : allow_t<float, 64, NW>();
    };
    return waves == 8 ? go(std::integral_constant<int, 8>{}) : go(std::integral_constant<int, 4>{});
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

hipError_t launch_weight_step(const WeightView& view, bool bf16, const WeightStepIO& io, const WeightPlan& p,
                              bool stream, hipStream_t s) {
    WeightView L = view;
    const int parts = (p.fused ? p.waves : p.nsplit) + io.prefix.n;
    L.wfloats = share_floats(L.G, parts);
    L.finish_parts = p.finish_parts;
    const size_t lds = step_lds(L.G, L.D, L.cpad, p.waves, p.fused, parts);
    auto go = [&](auto w) {
        constexpr int NW = decltype(w)::value;
        if (bf16)
            return L.D == 128 ? launch_step_t<uint16_t, 128, NW>(L, io, p, stream, lds, s)
                              : launch_step_t<uint16_t, 64, NW>(L, io, p, stream, lds, s);
        return L.D == 128 ? launch_step_t<float, 128, NW>(L, io, p, stream, lds, s)
                          : launch_step_t<float, 64, NW>(L, io, p, stream, lds, s);
    };
    return p.waves == 8 ? go(std::integral_constant<int, 8>{}) : go(std::integral_constant<int, 4>{});
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
