// How the quantised cache holds a block of 32 tokens of a KV head, and the way
// from values to codes and back on gfx950's conversions.
//
// Number format: a group of 32 channels of one token shares a power of two X,
// held as a biased exponent byte e (X = 2^(e - 127)); a value is a code times X,
// 4 bits e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) or 8 bits e4m3
// (up to 448). X is the least power of two with max |x| < 7 X (464 X): the
// largest code plus half its step, so that no value is off by more than half the
// step of the highest binade. In the maximum's bits that is a carry: adding
// 2^23 minus the mantissa of 1.75 (1.8125) moves into the next binade exactly the
// maxima that reach it. Products with powers of two are exact, so codes do not
// depend on how they are computed. e lies in 16 .. 252 (246): below, codes times X
// would leave the normal range of bf16, above, its largest. A group of zeros has
// e = 120, one that holds an infinity or NaN e = 255, which reads as NaN.
//
// Layout: codes lie in the order in which the lanes of v_mfma_f32_16x16x32_bf16
// take their operands once they are converted, so a wavefront reads 1 KiB of
// consecutive bytes per 16-byte load. The products sum over channels (keys) and
// tokens (values), and the order within a sum is free: lane (a, i) = 16 a + i has
// D / 4 consecutive channels of a key, which share an exponent, and of 8 tokens
// the same D / 16 consecutive channels of the values. One record:
//   key codes    piece p of lane l at 1024 p + 16 l; a lane's bytes in order:
//                tile q < 2, channels D/4 a .. of token 8 (i/4) + 4 q + i % 4
//   value codes  likewise: the lower half of channels D/16 i .. of tokens 8 a + j,
//                j < 8, then the upper half
//   exponents    of keys: [group][i][q] bytes; of values: [a][group][j]
#pragma once

#include <type_traits>

#include "raas_blocks.h"
#include "raas_quant_internal.h"

namespace raas {
namespace qnt {

using namespace blk;

template <int N>
using Int = std::integral_constant<int, N>;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

template <int D, int KB, int VB>
struct Format {
    static constexpr int KS = D / 32;            // products over a key's channels
    static constexpr int KC = D / 4;             // channels of a lane's key
    static constexpr int VC = D / 16;            // channels of a lane's values
    static constexpr int NG = D / kQuantGroup;   // groups of a token
    static constexpr int KD = KC * KB / 32;      // dwords of a lane's key (one tile)
    static constexpr int VBYTES = VC * VB / 8;   // bytes of a lane's values (one token)
    static constexpr int VHALF = VBYTES / 2;     // of half of them
    static constexpr int NKP = 2 * KD / 4;       // 16-byte pieces of a lane's keys
    static constexpr int NVP = 8 * VBYTES / 16;  // and of its values
    static constexpr int VALUES = NKP * 1024;    // offsets in a record
    static constexpr int KEXP = VALUES + NVP * 1024;
    static constexpr int VEXP = KEXP + 32 * NG;
    static constexpr int BYTES = VEXP + 32 * NG;
    static_assert(BYTES == (int)quant_record(D, KB, VB), "");
    // group of a lane's key, of its values, and lanes that share the latter
    static __device__ __forceinline__ int kgroup(int a) { return a * KC / kQuantGroup; }
    static __device__ __forceinline__ int vgroup(int i) { return i * VC / kQuantGroup; }
    static constexpr int VSHARE = kQuantGroup / VC;
};

// Exponent byte of a group of zeros.
constexpr uint32_t kZeroExponent = 120;

// The scale operand of a conversion, whose exponent alone counts (its sign and
// mantissa may be anything): of an exponent byte, and of byte j of four.
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e << 23); }
__device__ __forceinline__ uint32_t scale_bits(uint32_t four, int j) {
    return j == 0 ? four << 23 : j == 1 ? four << 15 : j == 2 ? four << 7 : four >> 1;
}

// The bytes of 255 among four exponents, NaN: their uppermost bits; of eight: bit j of byte j.
__device__ __forceinline__ uint32_t nan_bits(uint32_t e) { return ((e & 0x7F7F7F7Fu) + 0x01010101u) & e & 0x80808080u; }
__device__ __forceinline__ bool any_nan(u32x2 e) { return (nan_bits(e[0]) | nan_bits(e[1])) != 0u; }
__device__ __forceinline__ uint32_t nan_mask(u32x2 e) {
    // (bits 0, 8, 16, 24 to 24 .. 27; the other products meet neither these nor each other)
    return ((nan_bits(e[0]) >> 7) * 0x01020408u >> 24 & 15u) | ((nan_bits(e[1]) >> 7) * 0x01020408u >> 20 & 240u);
}

// Two codes, from byte `at` of a dword (a constant once loops are unrolled), as bf16 or (HALF) fp16.
template <int BITS, bool HALF>
__device__ __forceinline__ uint32_t two_values(uint32_t x, int at, float scale) {
    auto cast = [](auto y) { return __builtin_bit_cast(uint32_t, y); };
    if constexpr (BITS == 8) {
        if constexpr (HALF)
            return at ? cast(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, scale, true))
                      : cast(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, scale, false));
        else
            return at ? cast(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true))
                      : cast(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false));
    } else if constexpr (HALF) {
        return at == 0   ? cast(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, scale, 0))
               : at == 1 ? cast(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, scale, 1))
               : at == 2 ? cast(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, scale, 2))
                         : cast(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, scale, 3));
    } else {
        return at == 0   ? cast(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0))
               : at == 1 ? cast(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1))
               : at == 2 ? cast(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2))
                         : cast(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3));
    }
}
// Eight codes, in BITS / 4 dwords, as an operand of bf16.
template <int BITS>
__device__ __forceinline__ u32x4 eight_keys(const uint32_t* x, float scale) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = two_values<BITS, false>(x[BITS == 8 ? i >> 1 : 0], BITS == 8 ? 2 * (i & 1) : i, scale);
    return r;
}

template <bool NT>
__device__ __forceinline__ u32x4 load16(const uint8_t* p) {
    return NT ? ld16_nt(p) : ld16(p);
}

// A lane's keys of a block as they lie in memory.
template <int D, int KB, int VB>
struct Keys {
    using F = Format<D, KB, VB>;
    u32x4 k[F::NKP];
    uint32_t ke;  // exponents of the two tiles' keys
    template <bool NT>
    __device__ __forceinline__ void load(const uint8_t* rec, int lane) {
#pragma unroll
        for (int p = 0; p < F::NKP; ++p) k[p] = load16<NT>(rec + 1024 * p + 16 * lane);
        ke = *reinterpret_cast<const uint16_t*>(rec + F::KEXP + (F::kgroup(lane >> 4) * 16 + (lane & 15)) * 2);
    }
    __device__ __forceinline__ float key_scale(int q) const { return __uint_as_float(scale_bits(ke, q)); }
    // Channels 8 ks .. 8 ks + 7 of this lane's key of tile q, as bf16.
    __device__ __forceinline__ u32x4 key(int q, int ks, float scale) const {
        const int at = (q * F::KS + ks) * (KB / 4);
        const uint32_t x[2] = {k[at >> 2][at & 3], k[(at + KB / 8) >> 2][(at + KB / 8) & 3]};
        return eight_keys<KB>(x, scale);
    }
};

// A lane's values of a block as they lie in memory.
template <int D, int KB, int VB>
struct Values {
    using F = Format<D, KB, VB>;
    u32x4 v[F::NVP];
    u32x2 ve;  // exponents of the eight tokens
    template <bool NT>
    __device__ __forceinline__ void load(const uint8_t* rec, int lane) {
#pragma unroll
        for (int p = 0; p < F::NVP; ++p) v[p] = load16<NT>(rec + F::VALUES + 1024 * p + 16 * lane);
        ve = *reinterpret_cast<const u32x2*>(rec + F::VEXP + ((lane >> 4) * F::NG + F::vgroup(lane & 15)) * 8);
    }
    // Tokens `valid` .. of the block become 0, whatever is stored there.
    __device__ __forceinline__ void zero_values_from(int valid, int a) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (8 * a + j >= valid) {
                set_value(j, u32x2{0u, 0u});
                set_exponent(j, kZeroExponent);
            }
    }
    __device__ __forceinline__ void set_exponent(int j, uint32_t e) {
        const int sh = 8 * (j & 3);
        ve[j >> 2] = (ve[j >> 2] & ~(255u << sh)) | e << sh;
    }
    // Token j's codes of this lane's values (VBYTES of them).
    __device__ __forceinline__ void set_value(int j, u32x2 c) {
        if constexpr (F::VHALF == 4) {
            v[j >> 2][j & 3] = c[0];
            v[2 + (j >> 2)][j & 3] = c[1];
        } else {
            constexpr int BITS = 8 * F::VHALF, PER = 32 / BITS;  // tokens of a dword
            constexpr uint32_t ONES = (1u << BITS) - 1u;
            const int sh = BITS * (j % PER);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = h * (8 / PER) + j / PER;
                v[at >> 2][at & 3] = (v[at >> 2][at & 3] & ~(ONES << sh)) | (c[0] >> (BITS * h) & ONES) << sh;
            }
        }
    }
    __device__ __forceinline__ float value_scale(int j) const {
        return __uint_as_float(scale_bits(ve[j >> 2], j & 3));
    }
    // Channels 2 M and 2 M + 1 of this lane's values of token j, as bf16.
    template <int M>
    __device__ __forceinline__ uint32_t value2(int j, float scale) const {
        constexpr int IN_HALF = F::VC / 4;  // pairs of channels of a half
        const int at = (M / IN_HALF) * 8 * F::VHALF + j * F::VHALF + M % IN_HALF * (VB / 4);
        return two_values<VB, false>(v[at >> 4][at >> 2 & 3], at & 3, scale);
    }
    // All of this lane's values of token j.
    __device__ __forceinline__ void value_row(int j, uint32_t (&x)[F::VC / 2]) const {
        const float scale = value_scale(j);
        x[0] = value2<0>(j, scale);
        x[1] = value2<1>(j, scale);
        if constexpr (F::VC == 8) {
            x[2] = value2<2>(j, scale);
            x[3] = value2<3>(j, scale);
        }
    }
    // Channels 2 M and 2 M + 1 of all eight tokens: two operands of the product
    // with probabilities (values come in pairs of channels of one token, operands
    // in pairs of tokens of one channel).
    template <int M>
    __device__ __forceinline__ void values(const float (&scale)[8], u32x4& even, u32x4& odd) const {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t x = value2<M>(2 * p, scale[2 * p]), y = value2<M>(2 * p + 1, scale[2 * p + 1]);
            even[p] = __builtin_amdgcn_perm(y, x, 0x05040100u);
            odd[p] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        }
    }
};

// A lane's part of a block. NT: codes are read with non-temporal loads.
template <int D, int KB, int VB>
struct Block : Keys<D, KB, VB>, Values<D, KB, VB> {
    using F = Format<D, KB, VB>;
    template <bool NT = false>
    __device__ __forceinline__ void load(const uint8_t* rec, int lane) {
        Keys<D, KB, VB>::template load<NT>(rec, lane);
        Values<D, KB, VB>::template load<NT>(rec, lane);
    }
};

// Exponent byte of a group whose largest magnitude is `most`. (One of zeros may have any: that
// of numbers near 1 keeps their tokens with the others in the kernel for many rows.)
template <int BITS>
__device__ __forceinline__ uint32_t exponent_of(float most) {
    const uint32_t b = __float_as_uint(most);
    if (b >= 0x7F800000u) return 255u;
    const int e = (int)((b + (BITS == 4 ? 0x200000u : 0x180000u)) >> 23) - (BITS == 4 ? 2 : 8);
    return (uint32_t)min(max(e, b == 0u ? (int)kZeroExponent : 16), BITS == 4 ? 252 : 246);
}

// N (a multiple of 4) values to N * BITS / 8 bytes of codes, in dwords (the upper
// half of the last is 0 where they fill half of it).
template <int BITS, int N>
__device__ __forceinline__ void encode(const float (&x)[N], uint32_t e, uint32_t (&code)[(N * BITS + 31) / 32]) {
    const float scale = scale_of(e);
#pragma unroll
    for (int i = 0; i < (N * BITS + 31) / 32; ++i) code[i] = 0;
    if constexpr (BITS == 4) {  // rounds to nearest, ties to even, and saturates
#pragma unroll
        for (int i = 0; i < N / 4; i += 2) {
            uint32_t c = 0;
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4 * i], x[4 * i + 1], scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4 * i + 2], x[4 * i + 3], scale, 1);
            if (4 * i + 7 < N) {
                c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[(4 * i + 4) % N], x[(4 * i + 5) % N], scale, 2);
                c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[(4 * i + 6) % N], x[(4 * i + 7) % N], scale, 3);
            }
            code[i / 2] = c;
        }
    } else {  // (does not saturate by itself)
        const float most = 448.0f * scale;
        auto cut = [&](float y) { return __builtin_amdgcn_fmed3f(y, -most, most); };
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            s16x2 c = {0, 0};
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, cut(x[4 * i]), cut(x[4 * i + 1]), scale, false);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, cut(x[4 * i + 2]), cut(x[4 * i + 3]), scale, true);
            code[i] = __builtin_bit_cast(uint32_t, c);
        }
    }
}

// N consecutive elements of a caller's tensor (element-aligned) as floats.
template <typename T, int N>
__device__ __forceinline__ void load_floats(const T* p, float (&x)[N]) {
    if constexpr (sizeof(T) == 2 && N == 4) {
        typedef uint32_t u32x2_in __attribute__((ext_vector_type(2), aligned(2)));
        const u32x2 r = *reinterpret_cast<const u32x2_in*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(i & 1 ? r[i >> 1] & 0xFFFF0000u : r[i >> 1] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < N / kVec<T>; ++i) {
            const u32x4 r = ld16_in<T>(p + i * kVec<T>);
#pragma unroll
            for (int j = 0; j < kVec<T>; ++j) {
                if constexpr (sizeof(T) == 2)
                    x[i * 8 + j] = __uint_as_float(j & 1 ? r[j >> 1] & 0xFFFF0000u : r[j >> 1] << 16);
                else
                    x[i * 4 + j] = __uint_as_float(r[j]);
            }
        }
    }
}

template <int N>
__device__ __forceinline__ float most_of(const float (&x)[N]) {
    // (the largest magnitude's bits: a NaN's are above those of every number)
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    return __uint_as_float(m);
}
// the larger of two magnitudes, by their bits as above
__device__ __forceinline__ float larger(float x, float y) {
    return __uint_as_float(max(__float_as_uint(x), __float_as_uint(y)));
}

// A key row's channels of this lane: codes and the exponent of their group. All
// four lanes a of a key call it together.
template <typename T, int D, int BITS>
__device__ __forceinline__ uint32_t encode_key(const T* row, int a, uint32_t (&code)[D / 4 * BITS / 32]) {
    float x[D / 4];
    load_floats<T, D / 4>(row + a * (D / 4), x);
    float most = most_of(x);
    if constexpr (D == 64) most = larger(most, __shfl_xor(most, 16));
    const uint32_t e = exponent_of<BITS>(most);
    encode<BITS, D / 4>(x, e, code);
    return e;
}
// A value row's channels of this lane, likewise with its 16 lanes i.
template <typename T, int D, int BITS>
__device__ __forceinline__ uint32_t encode_value(const T* row, int i, u32x2& code) {
    float x[D / 16];
    load_floats<T, D / 16>(row + i * (D / 16), x);
    float most = most_of(x);
    most = larger(most, dpp_f<0xB1>(most));
    most = larger(most, dpp_f<0x4E>(most));
    if constexpr (D == 64) most = larger(most, dpp_f<0x141>(most));
    const uint32_t e = exponent_of<BITS>(most);
    uint32_t c[(D / 16 * BITS + 31) / 32];
    encode<BITS, D / 16>(x, e, c);
    code[0] = c[0];
    code[1] = (D / 16 * BITS) > 32 ? c[(D / 16 * BITS > 32)] : 0u;
    return e;
}

// Token j's codes of a lane's values to its place in a record.
template <int D, int KB, int VB>
__device__ __forceinline__ void store_value(uint8_t* rec, int lane, int j, const u32x2& code) {
    using F = Format<D, KB, VB>;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = (8 * h + j) * F::VHALF;
        uint8_t* to = rec + F::VALUES + 1024 * (at / 16) + 16 * lane + at % 16;
        if constexpr (F::VHALF == 4) *reinterpret_cast<uint32_t*>(to) = code[h];
        else if constexpr (F::VHALF == 2) *reinterpret_cast<uint16_t*>(to) = (uint16_t)(code[0] >> (16 * h));
        else *to = (uint8_t)(code[0] >> (8 * h));
    }
}

// N bf16 values, in dwords, to a caller's tensor of T.
template <typename T, int N>
__device__ __forceinline__ void store_values(T* p, const uint32_t (&x)[N / 2]) {
    if constexpr (sizeof(T) == 2) {
        if constexpr (N == 4) {
            typedef uint32_t u32x2_in __attribute__((ext_vector_type(2), aligned(2)));
            *reinterpret_cast<u32x2_in*>(p) = u32x2{x[0], x[1]};
        } else {
#pragma unroll
            for (int i = 0; i < N / 8; ++i)
                *reinterpret_cast<u32x4_in*>(p + 8 * i) = u32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
        }
    } else {
        typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int i = 0; i < N / 4; ++i)
            *reinterpret_cast<u32x4_at4*>(p + 4 * i) =
                u32x4{x[2 * i] << 16, x[2 * i] & 0xFFFF0000u, x[2 * i + 1] << 16, x[2 * i + 1] & 0xFFFF0000u};
    }
}

// The page's record of block `blk` of KV head h, from its number in the pool.
template <class F>
__device__ __forceinline__ uint8_t* record(const QuantView& L, int page, int blk, int h) {
    const size_t at = (((size_t)page * L.nkv + h) << L.page_shift) + (blk & ((1 << L.page_shift) - 1));
    return L.pool + at * F::BYTES;
}

// Calls go with the types of the cache: go(element, head_dim, key bits, value bits).
template <class Go>
hipError_t with_types(const QuantView& L, bool bf16, Go go) {
    auto bits = [&](auto t, auto d) {
        if (L.key_bits == 8) return L.value_bits == 8 ? go(t, d, Int<8>(), Int<8>()) : go(t, d, Int<8>(), Int<4>());
        return L.value_bits == 8 ? go(t, d, Int<4>(), Int<8>()) : go(t, d, Int<4>(), Int<4>());
    };
    auto dim = [&](auto t) { return L.D == 128 ? bits(t, Int<128>()) : bits(t, Int<64>()); };
    return bf16 ? dim(uint16_t()) : dim(float());
}

}  // namespace qnt
}  // namespace raas
