// What the kernels of the weight cache, the shared prefix, the prompt weights and
// the quantised cache have in common: the layout of a block of tokens in memory,
// the products on the matrix cores, the hand-over between workgroups.
//
// A block is the tokens of 64 16-byte reads per 16 channels of values: 32
// tokens in bf16, 16 in fp32. Keys and values are stored in the order in which
// the lanes of v_mfma_f32_16x16x32_bf16 and v_mfma_f32_16x16x4_f32 take their
// operands, so that every 16-byte-per-lane read of a wavefront is 1 KiB of
// consecutive bytes. With VE elements in 16 bytes, and lane = 16 a + i:
//   keys    piece (tile q < VE/4, step ks < D/(4 VE)): token VE (i/4) + 4 q +
//           i%4, channels 4 VE ks + VE a .. + VE;
//   values  piece (tile ct < D/16): channel 16 ct + i, tokens VE a .. + VE.
// The product of keys (rows) and queries (columns) then leaves lane (a, i)
// with the logits of tokens VE a .. + VE of query i, which is the operand that
// the product with the values takes: no data moves between lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace raas {
namespace blk {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// 16 bytes of a caller's tensor, which is aligned to its element type only
typedef uint32_t u32x4_in __attribute__((ext_vector_type(4), aligned(2)));

template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);  // elements of 16 bytes
template <typename T>
constexpr int kTokens = 4 * kVec<T>;  // tokens of a block
template <typename T>
constexpr int kTiles = kVec<T> / 4;  // 16-token tiles of a block

// Workgroup barrier that waits for this wavefront's LDS traffic only: loads
// already issued to global memory stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0); vmcnt and expcnt left at their maxima
    __builtin_amdgcn_s_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// This wavefront's number in its workgroup, as a scalar.
__device__ __forceinline__ int wave_of(int tid) { return __builtin_amdgcn_readfirstlane(tid >> 6); }

__device__ __forceinline__ u32x4 ld16(const void* p) { return *reinterpret_cast<const u32x4*>(p); }
__device__ __forceinline__ u32x4 ld16_nt(const void* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
}
template <typename T>
__device__ __forceinline__ u32x4 ld16_in(const T* p) {
    if constexpr (sizeof(T) == 2) return *reinterpret_cast<const u32x4_in*>(p);
    typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
    return *reinterpret_cast<const u32x4_at4*>(p);
}
__device__ __forceinline__ void st16(void* p, u32x4 x) { *reinterpret_cast<u32x4*>(p) = x; }

__device__ __forceinline__ uint16_t f2bf(float f) {  // to nearest, ties to even
    return __builtin_bit_cast(uint16_t, (__bf16)f);
}
template <typename T>
__device__ __forceinline__ T from_f(float x) {
    if constexpr (sizeof(T) == 2) return f2bf(x);
    else return x;
}

// element e of a 16-byte vector of T replaced by x
template <typename T>
__device__ __forceinline__ void set_elem(u32x4& v, int e, T x) {
    if constexpr (sizeof(T) == 2) {
        const uint32_t sh = (e & 1) * 16, old = v[e >> 1];
        v[e >> 1] = (old & ~(0xFFFFu << sh)) | ((uint32_t)x << sh);
    } else {
        v[e] = __float_as_uint(x);
    }
}

// Elements `valid` .. of a 16-byte vector of T set to zero (none if valid >= VE).
template <typename T>
__device__ __forceinline__ void zero_from(u32x4& v, int valid) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) {
            const uint32_t lo = 2 * i < valid ? 0xFFFFu : 0u, hi = 2 * i + 1 < valid ? 0xFFFF0000u : 0u;
            v[i] &= lo | hi;
        } else {
            v[i] = i < valid ? v[i] : 0u;
        }
    }
}

// max and sum over lanes i, i ^ 16, i ^ 32 and i ^ 48, the same on each: a
// permlane swap of a value with itself leaves both halves side by side
__device__ __forceinline__ float max_groups(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = fmaxf(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
    const unsigned v = __builtin_bit_cast(unsigned, x);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)b[0]), __builtin_bit_cast(float, (unsigned)b[1]));
}
__device__ __forceinline__ float sum_groups(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = __builtin_bit_cast(float, (unsigned)a[0]) + __builtin_bit_cast(float, (unsigned)a[1]);
    const unsigned v = __builtin_bit_cast(unsigned, x);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return __builtin_bit_cast(float, (unsigned)b[0]) + __builtin_bit_cast(float, (unsigned)b[1]);
}

// Moves within 16 lanes that stay in the vector unit: 0xB1 and 0x4E swap
// neighbours and pairs, 0x141 and 0x140 mirror eight and sixteen lanes (whose
// halves hold equal values by then).
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false);
}
template <int CTRL>
__device__ __forceinline__ float dpp_f(float x) { return __uint_as_float(dpp<CTRL>(__float_as_uint(x))); }
// max and sum over lanes 16 a .. 16 a + 15, the same on each
__device__ __forceinline__ float row16_max(float x) {
    x = fmaxf(x, dpp_f<0xB1>(x));
    x = fmaxf(x, dpp_f<0x4E>(x));
    x = fmaxf(x, dpp_f<0x141>(x));
    return fmaxf(x, dpp_f<0x140>(x));
}
__device__ __forceinline__ float row16_sum(float x) {
    x += dpp_f<0xB1>(x);
    x += dpp_f<0x4E>(x);
    x += dpp_f<0x141>(x);
    return x + dpp_f<0x140>(x);
}
// and over a wavefront
__device__ __forceinline__ float wave_max(float x) { return max_groups(row16_max(x)); }
__device__ __forceinline__ float wave_sum(float x) { return sum_groups(row16_sum(x)); }
// min of 64-bit values over a wavefront, the same on each lane
__device__ __forceinline__ unsigned long long wave_min(unsigned long long x) {
    auto with = [&](uint32_t lo, uint32_t hi) {
        const unsigned long long y = (unsigned long long)hi << 32 | lo;
        x = y < x ? y : x;
    };
    with(dpp<0xB1>((uint32_t)x), dpp<0xB1>((uint32_t)(x >> 32)));
    with(dpp<0x4E>((uint32_t)x), dpp<0x4E>((uint32_t)(x >> 32)));
    with(dpp<0x141>((uint32_t)x), dpp<0x141>((uint32_t)(x >> 32)));
    with(dpp<0x140>((uint32_t)x), dpp<0x140>((uint32_t)(x >> 32)));
    auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
    auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(x >> 32), (uint32_t)(x >> 32), false, false);
    with(lo[0], hi[0]);
    with(lo[1], hi[1]);
    lo = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
    hi = __builtin_amdgcn_permlane32_swap((uint32_t)(x >> 32), (uint32_t)(x >> 32), false, false);
    with(lo[0], hi[0]);
    with(lo[1], hi[1]);
    return x;
}

// c += A B for one 16-byte vector of either operand per lane: 4 VE channels.
template <typename T>
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, f32x4 c) {
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    } else {  // step m takes channel m of each lane's four
#pragma unroll
        for (int m = 0; m < 4; ++m)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[m]), __uint_as_float(b[m]), c, 0, 0, 0);
        return c;
    }
}

// This lane's pieces of a query row (row-major, element-aligned), or zeros.
template <typename T, int D>
__device__ __forceinline__ void load_row(const T* row, bool real, int a, u32x4 (&q)[D / (4 * kVec<T>)]) {
#pragma unroll
    for (int ks = 0; ks < D / (4 * kVec<T>); ++ks)
        q[ks] = real ? ld16_in<T>(row + 4 * kVec<T> * ks + kVec<T> * a) : u32x4{0u, 0u, 0u, 0u};
}

// VE probabilities as the operand that multiplies values. Beside bf16 values the
// matrix cores take bf16 only, so each is the sum of two there: its upper 16 bits
// and what they leave, rounded to bf16, which is off by at most 2^-15 of it. (One
// bf16 alone is off by 2^-8: where values of either sign cancel, its errors do so
// no better than the values, and the outputs were off by 0.0020 to 0.0025 of their
// size where their own rounding is 0.0017. The second product is free where
// reading bounds a kernel, the step and the prefix of few rows; k_prefix_wide has
// what it costs there.)
template <typename T>
struct Probs {
    u32x4 hi, lo;  // (lo: bf16 only)
    __device__ __forceinline__ explicit Probs(const float (&p)[kVec<T>]) {
        if constexpr (sizeof(T) == 2) {
            bf16x8 rest;
#pragma unroll
            for (int j = 0; j < 8; ++j) rest[j] = (__bf16)(p[j] - __uint_as_float(__float_as_uint(p[j]) & 0xFFFF0000u));
#pragma unroll
            for (int j = 0; j < 4; ++j)
                hi[j] = __float_as_uint(p[2 * j]) >> 16 | (__float_as_uint(p[2 * j + 1]) & 0xFFFF0000u);
            lo = __builtin_bit_cast(u32x4, rest);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) hi[j] = __float_as_uint(p[j]);
        }
    }
};

// Running softmax of one query column: maximum (base 2), this lane's share of
// the sum, and the accumulated values' rows 16 ct + 4 a + r.
template <int D>
struct Softmax {
    float m = -INFINITY, l = 0.0f;
    f32x4 o[D / 16];
    __device__ void clear() {
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) o[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
};

// One block of `valid` (1 .. tokens of a block) tokens against a tile of 16
// queries: x[q][r] receives the logits (base 2) of token VE a + 4 q + r, -inf
// from `valid` on. Sums are kept in fp32.
template <typename T, int D>
__device__ __forceinline__ void attend(const u32x4 (&kr)[D / 16], const u32x4 (&vr)[D / 16],
                                       const u32x4 (&q)[D / (4 * kVec<T>)], int valid, int a, float scale_log2,
                                       Softmax<D>& s, f32x4 (&x)[kTiles<T>]) {
    constexpr int KS = D / (4 * kVec<T>), QT = kTiles<T>, VE = kVec<T>;
#pragma unroll
    for (int t = 0; t < QT; ++t) x[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int t = 0; t < QT; ++t) x[t] = mfma16<T>(kr[t * KS + ks], q[ks], x[t]);
    float mb = -INFINITY;
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            x[t][r] = VE * a + 4 * t + r < valid ? x[t][r] * scale_log2 : -INFINITY;
            mb = fmaxf(mb, x[t][r]);
        }
    mb = max_groups(mb);
    const float m = fmaxf(s.m, mb);
    if (__ballot(m > s.m) != 0ull) {
        const float alpha = __builtin_amdgcn_exp2f(s.m - m);
        s.l *= alpha;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) s.o[ct] *= alpha;
        s.m = m;
    }
    float p[VE];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            p[4 * t + r] = __builtin_amdgcn_exp2f(x[t][r] - s.m);
            s.l += p[4 * t + r];
        }
    const Probs<T> pv(p);
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) s.o[ct] = mfma16<T>(vr[ct], pv.hi, s.o[ct]);
    if constexpr (sizeof(T) == 2)
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) s.o[ct] = mfma16<T>(vr[ct], pv.lo, s.o[ct]);
}

// Order-preserving unsigned key of a float (NaN above +inf).
__device__ __forceinline__ uint32_t float_key(float x) {
    const uint32_t b = __float_as_uint(x);
    return (b >> 31) ? ~b : b | 0x80000000u;
}

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

}  // namespace blk
}  // namespace raas
