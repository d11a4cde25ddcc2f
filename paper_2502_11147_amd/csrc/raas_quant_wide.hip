// gfx950 kernels of attention over the quantised cache for many rows per unit
// (pieces of prompts): the sums of raas_quant_attention.hip, 32 rows per wavefront.
#include <algorithm>

#include "raas_quant_attention.h"

namespace raas {
namespace {

using namespace qnt;

// A wavefront is a workgroup: it takes a tile of 32 rows through the blocks of its
// part, straight from memory to registers, converts them there and shares nothing.
// (Through LDS, where eight wavefronts converted each block once for all of them,
// 512 rows of four long prompts took 579 us against 632 then, but a prompt of 4096
// tokens 179 against 168, 256 tokens behind 1000 41 against 35: reading it back, and
// a barrier for every two blocks, took most of what it saved.)
// Bound by vector instructions (active 74 % of the cycles) and products (41 %), which
// two wavefronts per SIMD hardly overlap: 512 rows of four prompts of 16384 tokens
// take 600 us, 896 TFLOP/s. A third wavefront, for which the query is read from LDS
// anew and a block lies in registers only once, made it 699. The next block's logits
// formed beside this one's exponentials changed nothing (604; in fp32 85 us against 75
// for 512 rows behind 2000 tokens).
constexpr int kWideRows = 32;
constexpr Cut kWideCut = {1024, 8, 8};

// Beside a bf16 cache's values, probabilities are rounded to fp16 (half a step,
// 2^-11 of themselves, an eighth of what the rounding of a bf16 output may be; in
// bf16 it takes two products, and twice the vector work, to be as near). Values are
// then fp16 too: codes times X / 2^(kUnit - 127), exact while X's exponent byte lies
// in kLeast .. kLeast + kSpan - 1: the least step of a code is 2^-20 there,
// the largest value 7168 (four bits: 24576). A wavefront that meets another exponent starts over
// with bf16 and two products: 512 rows of four prompts of 16384 tokens in 8 bits 772 us for
// 627 where the first token is such a one, 1218 where the last is. Probabilities are taken relative to 2^-kRaise of
// the row's maximum at the time, so they lie below 2^(kRaise + kSlack) and keep all
// digits down to 2^-14: 2^-21 of the largest or less; below, they are off by 2^-25.
// That holds for references within kFar of 0, where fp32 has steps of 2^-4: rounding and
// the lag it causes add one step. From 2^23 on a step is 1, and 2^(kRaise + kSlack + 1) is
// past fp16's largest number: a wavefront that meets a row beyond kFar starts over with
// bf16 too.
template <int VB>
struct Half {
    static constexpr int kUnit = VB == 4 ? 127 : 120, kLeast = VB == 4 ? 108 : 109, kSpan = VB == 4 ? 32 : 16;
    // Whether one of these exponents lies outside (a byte below kLeast borrows from the
    // next one, but is outside itself).
    static __device__ __forceinline__ uint32_t beyond(uint32_t e) {
        return (e - 0x01010101u * kLeast) & (0x01010101u * (256u - kSpan));
    }
    // Four exponents inside, of X / 2^(kUnit - 127).
    static __device__ __forceinline__ uint32_t scaled(uint32_t e) { return e + 0x01010101u * (127 - kUnit); }
    static __device__ __forceinline__ bool outside(u32x2 e) { return (beyond(e[0]) | beyond(e[1])) != 0u; }
};
static_assert(kZeroExponent >= Half<8>::kLeast && kZeroExponent < Half<8>::kLeast + Half<8>::kSpan &&
                  kZeroExponent >= Half<4>::kLeast && kZeroExponent < Half<4>::kLeast + Half<4>::kSpan, "");
constexpr float kRaise = 7.0f, kFar = 0x1p20f;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <bool HALF>
__device__ __forceinline__ f32x16 mfma32(const u32x4& a, const u32x4& b, f32x16 c) {
    if constexpr (HALF)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                      0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                       0, 0);
}

// A block in the order of v_mfma_f32_32x32x16's operands (two products of 16x16x32
// keep the vector unit waiting for 25 cycles of their 32, one of these for 15): lane
// (h, i) = 32 h + i has row i of the first operand, elements 8 h .. of 16, and of the
// result rows 8 (r / 4) + 4 h + r % 4 of column i. Row 16 s + 8 g + 4 h + j of the
// logits is token 16 s + 8 h + 4 g + j (g, h < 2, j < 4): a lane's results r = 8 s ..
// 8 s + 7 are then tokens 16 s + 8 h .. + 7, which are stored together.
//   keys    token of row i, channels D/2 h ..: the stored lanes a = 2 h and 2 h + 1
//   values  channels D/32 i .., tokens 16 s + 8 h ..: a half of the stored lane
//           a = 2 s + h, i / 2
template <int D, int KB, int VB>
struct WideBlock {
    using F = Format<D, KB, VB>;
    static constexpr int VD = 2 * F::VHALF;  // dwords of eight tokens' values
    uint32_t k[2][F::KD], v[2][VD], ke[2];
    u32x2 ve[2];
    // Offsets of this lane's parts in a record.
    struct Places {
        uint32_t k[2], ke[2], v[2], ve[2];
        __device__ __forceinline__ explicit Places(int lane) {
            const int h = lane >> 5, i = lane & 31;
            const int t = (i & 16) | (i & 4) << 1 | (i & 8) >> 1 | (i & 3);  // token of row i
            const int q = t >> 2 & 1, ki = 4 * (t >> 3) + (t & 3);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int a = 2 * h + x, at = 4 * F::KD * q;
                k[x] = 1024 * (at / 16) + 16 * (16 * a + ki) + at % 16;
                ke[x] = F::KEXP + (F::kgroup(a) * 16 + ki) * 2 + q;
                const int va = 2 * x + h, vat = 8 * F::VHALF * (i & 1);
                v[x] = F::VALUES + 1024 * (vat / 16) + 16 * (16 * va + (i >> 1)) + vat % 16;
                ve[x] = F::VEXP + (va * F::NG + F::vgroup(i >> 1)) * 8;
            }
        }
    };
    // From a record's address in scalar registers (a buffer of its bytes, unstructured), so
    // that a load's own address costs no vector instruction.
    __device__ __forceinline__ void load(const uint8_t* rec, const Places& at) {
        const auto from = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(rec), 0, F::BYTES, 0x00020000);
        auto dwords = [&](uint32_t at, auto& x) {
            constexpr int N = sizeof(x) / 4;
            if constexpr (N == 2) {
                const u32x2 y = __builtin_amdgcn_raw_buffer_load_b64(from, at, 0, 0);
                x[0] = y[0];
                x[1] = y[1];
            } else {
#pragma unroll
                for (int n = 0; n < N; n += 4) {
                    const u32x4 y = __builtin_amdgcn_raw_buffer_load_b128(from, at, 256 * n, 0);  // the next 1 KiB
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[n + e] = y[e];
                }
            }
        };
#pragma unroll
        for (int x = 0; x < 2; ++x) dwords(at.k[x], k[x]);
#pragma unroll
        for (int x = 0; x < 2; ++x) dwords(at.v[x], v[x]);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            ke[x] = __builtin_amdgcn_raw_buffer_load_b8(from, at.ke[x], 0, 0);
            ve[x] = __builtin_amdgcn_raw_buffer_load_b64(from, at.ve[x], 0, 0);
        }
    }
    // Token 16 x + 8 h + j's value becomes 0.
    __device__ __forceinline__ void clear(int x, int j) {
        constexpr int PER = 4 / F::VHALF;  // tokens of a dword
        v[x][j / PER] &= PER == 1 ? 0u : ~((0xFFFFFFFFu >> (32 - 32 / PER)) << (32 / PER * (j % PER)));
        ve[x][j >> 2] = (ve[x][j >> 2] & ~(255u << (8 * (j & 3)))) | kZeroExponent << (8 * (j & 3));
    }
    // Those of tokens `valid` .. of the block, whatever is stored there.
    __device__ __forceinline__ void zero_values_from(int valid, int h) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (16 * x + 8 * h + j >= valid) clear(x, j);
    }
    // As hand_out_nan: a lane's outputs o are those of one row and of 8 consecutive
    // places of r for each group of channels (head_dim 128: of 4).
    __device__ __forceinline__ void hand_out_nan(int lim, f32x16 (&o)[D / 32]) {
        constexpr int EACH = 32 / F::NG;  // lanes i of a group; half as many r
        const uint32_t own = nan_mask(ve[0]) | nan_mask(ve[1]) << 8;  // tokens 8 h .., 16 + 8 h ..
#pragma unroll
        for (int g = 0; g < F::NG; ++g) {
            const uint32_t x = __builtin_amdgcn_readlane(own, EACH * g), y = __builtin_amdgcn_readlane(own, 32 + EACH * g);
            const uint32_t all = (x & 255u) | (y & 255u) << 8 | (x & 0xFF00u) << 8 | (y & 0xFF00u) << 16;
            const bool hit = lim > 0 && (all << (32 - min(lim, 32))) != 0u;
#pragma unroll
            for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
                for (int r = EACH / 2 * g; r < EACH / 2 * (g + 1); ++r) o[ct][r] = hit ? NAN : o[ct][r];
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (own >> (8 * x + j) & 1u) clear(x, j);
    }
    // Channels 8 n .. + 7 of this lane's key, as bf16.
    __device__ __forceinline__ u32x4 key(int n) const {
        constexpr int PER = F::KC / 8;
        return eight_keys<KB>(&k[n / PER][n % PER * (KB / 4)], scale_of(ke[n / PER]));
    }
    // Two operands of the product with probabilities: channels 2 m and 2 m + 1 of the lane's tokens 16 s ..
    template <bool HALF>
    __device__ __forceinline__ void values(int s, int m, const float (&scale)[8], u32x4& even, u32x4& odd) const {
        auto two = [&](int j) {
            const int at = j * F::VHALF + m * (VB / 4);
            return two_values<VB, HALF>(v[s][at >> 2], at & 3, scale[j]);
        };
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t x = two(2 * p), y = two(2 * p + 1);
            even[p] = __builtin_amdgcn_perm(y, x, 0x05040100u);
            odd[p] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        }
    }
};

// A wavefront's rows and blocks.
struct Part {
    int first, end, least;  // rows of the unit; tokens that the first one sees
    int lo, hi;             // blocks
};
// What it has of them: reference and this lane's share of the sum of row `first` + i,
// and unnormalised outputs of channels D/32 (8 (r / 4) + 4 h + r % 4) + ct.
template <int D>
struct Rows {
    float m, l;
    f32x16 o[D / 32];
};

// Attention of a part into s, from the start. HALF: probabilities and values in fp16;
// false if a block has an exponent outside, or a row's logits lie far out.
template <typename T, int D, int KB, int VB, bool HALF>
__device__ __forceinline__ bool attend_part(const QuantView& L, const QuantAttention& io, const Work& w, const Part& pt,
                                            int lane, Rows<D>& s) {
    using F = Format<D, KB, VB>;
    using Wide = WideBlock<D, KB, VB>;
    constexpr int NQ = kQueryPieces<T>, NP = HALF ? 1 : kProbPieces<T>, CT = D / 32;
    const int32_t* table = L.table + (size_t)w.b * L.width;
    const int lo = pt.lo, h = lane >> 5, row = pt.first + (lane & 31);
    const bool real = row < pt.end;
    const typename Wide::Places at(lane);
    int hi = pt.hi;
    bool inside = true;
    // (looked at after the loop: leaving it where a reference moves took 0.7 % longer)
    float far = 0.0f;  // how far from 0 the references were
    // channels D/2 h + 8 n .. of the query; an fp32 one's third pieces, for which there is no register left, in LDS
    u32x4 q[D / 16][NQ < 3 ? NQ : 2];
    __shared__ u32x4 third[NQ < 3 ? 1 : D / 16][64];
    {
        const T* from = (const T*)io.q + row_at(L, io, w, row) * D + D / 2 * h;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
            if constexpr (sizeof(T) == 2) {
                q[n][0] = real ? ld16_in<T>(from + 8 * n) : u32x4{0u, 0u, 0u, 0u};
            } else {
                float x[8] = {};
                if (real) load_floats<T, 8>(from + 8 * n, x);
                const Pieces<3> p(x);
#pragma unroll
                for (int k = 0; k < 2; ++k) q[n][k] = p.p[k];
                third[n][lane] = p.p[2];
            }
        }
    }
    const int lim = real ? w.tokens - w.rows / L.G + 1 + row / L.G : 0;  // tokens that the row sees
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    s.m = kLowest;
    s.l = 0.0f;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) s.o[ct] = zero;
    int win = -1;  // pages of 64 blocks in the lanes
    // the block's page, -1: none; the block (of no page: any, unused)
    auto fetch = [&](int b, Wide& blk) {
        if (((b - lo) & 63) == 0) win = b + lane < hi ? table[(b + lane) >> L.page_shift] : -1;
        const int page = __builtin_amdgcn_readlane(win, (b - lo) & 63);
        const bool good = page >= 0 && page < L.n_pages;
        blk.load(record<F>(L, good ? page : 0, b, w.h), at);
        return good;
    };
    auto attend = [&](int b, bool good, Wide& blk) {
        const int t0 = b * kQuantBlock;
        const bool masked = t0 + kQuantBlock > pt.least;
        if (masked) blk.zero_values_from(w.tokens - t0, h);
        if constexpr (HALF) {
            if (good && __ballot(Half<VB>::outside(blk.ve[0]) || Half<VB>::outside(blk.ve[1])) != 0ull) {
                good = inside = false;
                hi = b;  // the end
            }
        }
        if (!good) return;
        if constexpr (!HALF) {  // (fp16: NaN are outside)
            if (masked && __ballot(any_nan(blk.ve[0]) || any_nan(blk.ve[1])) != 0ull) blk.hand_out_nan(lim - t0, s.o);
        }
        f32x16 x = zero;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
            const u32x4 k = blk.key(n);
#pragma unroll
            for (int c = 0; c < NQ; ++c) x = mfma32<false>(k, c < 2 ? q[n][c] : third[n][lane], x);
        }
        if (masked) {
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = t0 + 16 * (r >> 3) + 8 * h + (r & 7) < lim ? x[r] : -INFINITY;
        }
        float most = x[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) most = fmaxf(most, x[r]);
        most = __builtin_fmaf(most, io.scale_log2, HALF ? -kRaise : 0.0f);
        if (__ballot(most > s.m + kSlack) != 0ull) {
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(most), __float_as_uint(most), false, false);
            const float m = fmaxf(s.m, fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])));
            const float alpha = __builtin_amdgcn_exp2f(s.m - m);
            s.l *= alpha;
            s.m = m;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s.o[ct] *= alpha;
            if constexpr (HALF) {
                far = fmaxf(far, m > kLowest ? fabsf(m) : 0.0f);  // (kLowest: a row that has seen no token)
            }
        }
        u32x4 p[2][NP];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[8 * g + j], io.scale_log2, -s.m));
            s.l += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
            if constexpr (HALF) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    p[g][0][j] =
                        __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{y[2 * j], y[2 * j + 1]}), f16x2));
            } else {
                const Pieces<NP> pieces(y);
#pragma unroll
                for (int n = 0; n < NP; ++n) p[g][n] = pieces.p[n];
            }
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            float scale[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                scale[j] = __uint_as_float(
                    scale_bits(HALF ? Half<VB>::scaled(blk.ve[g][j >> 2]) : blk.ve[g][j >> 2], j & 3));
#pragma unroll
            for (int m = 0; m < CT / 2; ++m) {
                u32x4 even, odd;
                blk.template values<HALF>(g, m, scale, even, odd);
#pragma unroll
                for (int n = 0; n < NP; ++n) {
                    s.o[2 * m] = mfma32<HALF>(even, p[g][n], s.o[2 * m]);
                    s.o[2 * m + 1] = mfma32<HALF>(odd, p[g][n], s.o[2 * m + 1]);
                }
            }
        }
    };
    if (lo < hi) {
        Wide b0, b1;
        bool good0 = fetch(lo, b0);
        for (int b = lo; b < hi; b += 2) {
            const bool good1 = fetch(b + 1, b1);
            attend(b, good0, b0);
            if (b + 1 >= hi) break;
            good0 = fetch(b + 2, b0);
            attend(b + 1, good1, b1);
        }
    }
    return inside && __ballot(far > kFar) == 0ull;
}

template <typename T, int D, int KB, int VB>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_quant_wide(QuantView L,
                                                                                           QuantAttention io) {
    constexpr int CT = D / 32;
    const int lane = threadIdx.x, h = lane >> 5;
    Work w;
    if (!find_work<kWideRows>(L, io, kWideCut, lane, blockIdx.x, w)) return;
    // a row sees the tokens up to its own: query i of `count` lies at tokens - count + i
    auto limit = [&](int row) { return w.tokens - w.rows / L.G + 1 + row / L.G; };
    const int first = w.tile * kWideRows, end = min(first + kWideRows, w.rows);
    const int nb = blocks_of(max(0, limit(end - 1))), per = (nb + w.parts - 1) / w.parts, lo = min(nb, w.part * per);
    const Part pt = {first, end, limit(first), lo, min(nb, lo + per)};
    Rows<D> s;
    float unit = 1.0f;
    if constexpr (sizeof(T) == 2) {
        unit = scale_of(Half<VB>::kUnit);
        if (!attend_part<T, D, KB, VB, true>(L, io, w, pt, lane, s)) {
            unit = 1.0f;
            attend_part<T, D, KB, VB, false>(L, io, w, pt, lane, s);
        }
    } else {
        attend_part<T, D, KB, VB, false>(L, io, w, pt, lane, s);
    }
    const float l = s.l + __shfl_xor(s.l, 32);
    const int row = first + (lane & 31);
    if (row >= end) return;
    if (w.parts > 1) {
        const size_t at = (size_t)(w.slot + w.part) * kWideRows + row - first;
        if (h == 0) *reinterpret_cast<float2*>(io.ml + 2 * at) = make_float2(s.m, l);
#pragma unroll
        for (int r = 0; r < 16; r += 4 / CT) {  // 16 bytes of consecutive channels
            f32x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = s.o[e % CT][r + e / CT] * unit;
            *reinterpret_cast<f32x4*>(io.part + at * D + CT * (8 * (r / 4) + 4 * h + r % 4)) = y;
        }
        return;
    }
    const size_t at = row_at(L, io, w, row);
    const float rl = l == 0.0f ? 0.0f : unit / l;
    if (io.lse != nullptr && h == 0) io.lse[at] = natural_log(s.m, l);
    typedef T Tv __attribute__((ext_vector_type(8), aligned(sizeof(T))));
#pragma unroll
    for (int r = 0; r < 16; r += 8 / CT) {
        Tv y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = from_f<T>(s.o[e % CT][r + e / CT] * rl);
        *reinterpret_cast<Tv*>((T*)io.out + at * D + CT * (8 * (r / 4) + 4 * h + r % 4)) = y;
    }
}

// Outputs and log-sum-exps of the rows of split tiles from their parts: a wavefront
// per row, a lane per part for the shares, then 16 bytes per lane of 4 (head_dim 64)
// or 2 parts at a time, eight reads on their way together. The split rows of all
// sequences are dealt out to the wavefronts in turn.
constexpr int kJoinWorkgroups = 1024;
template <typename T, int D>
__global__ __launch_bounds__(256) void k_quant_join(QuantView L, QuantAttention io) {
    constexpr int LANES = D / 4, AT = 64 / LANES, TR = kWideRows;
    typedef T T4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    const int lane = threadIdx.x & 63, step = (int)gridDim.x * 4;
    for_split_rows<TR>(L, io, kWideCut, lane, (int)blockIdx.x * 4 + wave_of(threadIdx.x), step, [&](const Work& w, int row) {
        const size_t at = (size_t)(w.slot + (w.h * w.tiles + w.tile) * w.parts) * TR + row - w.tile * TR;
        float2 ml = make_float2(kLowest, 0.0f);
        static_assert(kMaxQuantParts <= 64, "");
        if (lane < w.parts) ml = *reinterpret_cast<const float2*>(io.ml + 2 * (at + (size_t)lane * TR));
        const float M = wave_max(ml.x), e = __builtin_amdgcn_exp2f(ml.x - M), Z = wave_sum(ml.y * e);
        const float share = Z == 0.0f ? 0.0f : e / Z;
        const int c = lane % LANES * 4;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        for (int p0 = 0; p0 < w.parts; p0 += 8 * AT) {
            f32x4 y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                y[k] = *reinterpret_cast<const f32x4*>(
                    io.part + (at + (size_t)min(p0 + k * AT + lane / LANES, w.parts - 1) * TR) * D + c);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int p = p0 + k * AT + lane / LANES;
                const float e = __shfl(share, p & 63);  // (of every lane: not within the choice)
                x += y[k] * (p < w.parts ? e : 0.0f);
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (AT == 4) x[k] = sum_groups(x[k]);
            else x[k] += __shfl_xor(x[k], 32);
        }
        const size_t to = row_at(L, io, w, row);
        if (lane < LANES) {
            T4 o;
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = from_f<T>(x[k]);
            *reinterpret_cast<T4*>((T*)io.out + to * D + c) = o;
        }
        if (io.lse != nullptr && lane == 0) io.lse[to] = natural_log(M, Z);
    });
}

template <typename T, int D, int KB, int VB>
hipError_t launch(const QuantView& L, const QuantAttention& io, hipStream_t s) {
    const size_t grid = most_workgroups(kWideCut, kWideRows, L.batch, io.queries, L.nkv, L.G);
    hipLaunchKernelGGL((k_quant_wide<T, D, KB, VB>), dim3((unsigned)grid), dim3(64), 0, s, L, io);
    if (L.cap / kQuantBlock > kWideCut.whole) {  // (else no tile is cut)
        const size_t rows = (size_t)L.batch * L.nkv * io.queries * L.G;
        hipLaunchKernelGGL((k_quant_join<T, D>), dim3((unsigned)std::min((rows + 3) / 4, (size_t)kJoinWorkgroups)),
                           dim3(256), 0, s, L, io);
    }
    return hipGetLastError();
}

}  // namespace

size_t quant_wide_scratch_rows(int batch, int queries, int nkv, int G) {
    const size_t tiles = (size_t)batch * nkv * ((queries * G + kWideRows - 1) / kWideRows);
    return std::min((size_t)2 * kWideCut.target, tiles * kMaxQuantParts) * kWideRows;
}

hipError_t launch_quant_wide(const QuantView& L, bool bf16, const QuantAttention& io, hipStream_t s) {
    return with_types(L, bf16, [&](auto t, auto d, auto kb, auto vb) {
        return launch<decltype(t), d(), kb(), vb()>(L, io, s);
    });
}

}  // namespace raas
