// gfx950 kernels of attention over the quantised cache for many rows per unit
// (pieces of prompts): the sums of raas_quant_attention.hip, 16 RT rows per
// wavefront.
#include <algorithm>

#include "raas_quant_attention.h"

namespace raas {
namespace {

using namespace qnt;

// A wavefront is a workgroup: it takes a tile of 16 RT rows through the blocks of
// its part, straight from memory to registers, converts them there and shares
// nothing. (Through LDS, where eight wavefronts converted each block once for all of
// them, 512 rows of four long prompts took 579 us against 632, but a prompt of 4096
// tokens 179 against 168, 256 tokens behind 1000 41 against 35: reading it back, and
// a barrier for every two blocks, took most of what it saved.)
template <typename T>
constexpr int kRowTiles = sizeof(T) == 2 ? 2 : 1;
template <typename T>
constexpr int kWideRows = 16 * kRowTiles<T>;
constexpr Cut kWideCut = {1024, 8, 8};

// Beside a bf16 cache's values, probabilities are rounded to fp16 (half a step,
// 2^-11 of themselves, an eighth of what the rounding of a bf16 output may be; in
// bf16 it takes two products, and twice the vector work, to be as near). Values are
// then fp16 too: codes times X / 2^(kUnit - 127), exact while X's exponent byte lies
// in kLeast .. kLeast + kSpan - 1: the least step of a code is 2^-20 (2^-21) there,
// the largest value 7168 (12288). A wavefront that meets another exponent starts over
// with attend_block, two products. Probabilities are taken relative to 2^-kRaise of
// the row's maximum at the time, so they lie below 2^(kRaise + kSlack) and keep all
// digits down to 2^-14: 2^-21 of the largest or less; below, they are off by 2^-25.
template <int VB>
struct Half {
    static constexpr int kUnit = VB == 4 ? 128 : 120, kLeast = VB == 4 ? 108 : 109, kSpan = VB == 4 ? 32 : 16;
    // Whether one of these exponents lies outside (a byte below kLeast borrows from the
    // next one, but is outside itself).
    static __device__ __forceinline__ uint32_t beyond(uint32_t e) {
        return (e - 0x01010101u * kLeast) & (0x01010101u * (256u - kSpan));
    }
    static __device__ __forceinline__ bool outside(u32x2 e) { return (beyond(e[0]) | beyond(e[1])) != 0u; }
};
constexpr float kRaise = 7.0f;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mfma_half(const u32x4& a, const u32x4& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// One block against RT tiles of rows, as attend_block, with probabilities and values
// in fp16.
template <int D, int KB, int VB, int RT>
__device__ __forceinline__ void attend_half(const Block<D, KB, VB>& blk, const u32x4 (&q)[RT][D / 32][1], bool masked,
                                            const int (&lim)[RT], int a, float scale_log2, Softmax<D> (&s)[RT]) {
    f32x4 x[RT][2];
    block_logits<uint16_t, D, KB, VB, RT>(blk, q, masked, lim, a, x);
    follow<D, RT>(x, scale_log2, kRaise, s);
    u32x4 p[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float y[8], sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            y[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][j >> 2][j & 3], scale_log2, -s[t].m));
            sum += y[j];
        }
        s[t].l += sum;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            p[t][j] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{y[2 * j], y[2 * j + 1]}), f16x2));
    }
    float scale[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) scale[j] = blk.value_scale(j, 127 - Half<VB>::kUnit);
    auto two = [&](auto m) {
        constexpr int M = decltype(m)::value;
        u32x4 even, odd;
        blk.template values<M, true>(scale, even, odd);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            s[t].o[2 * M] = mfma_half(even, p[t], s[t].o[2 * M]);
            s[t].o[2 * M + 1] = mfma_half(odd, p[t], s[t].o[2 * M + 1]);
        }
    };
    two(Int<0>());
    two(Int<1>());
    if constexpr (D == 128) {
        two(Int<2>());
        two(Int<3>());
    }
}

// A wavefront's rows and blocks.
struct Part {
    int first, end, least;  // rows of the unit; tokens that the first one sees
    int lo, hi;             // blocks
};

// Attention of a part into s, from the start. HALF: as attend_half, false if a block
// has an exponent outside.
template <typename T, int D, int KB, int VB, bool HALF>
__device__ __forceinline__ bool attend_part(const QuantView& L, const QuantAttention& io, const Work& w, const Part& pt,
                                            int lane, Softmax<D> (&s)[kRowTiles<T>]) {
    using F = Format<D, KB, VB>;
    constexpr int RT = kRowTiles<T>;
    const int32_t* table = L.table + (size_t)w.b * L.width;
    const int lo = pt.lo, a = lane >> 4, col = lane & 15;
    int hi = pt.hi;
    bool inside = true;
    int lim[RT];
    u32x4 q[RT][F::KS][kQueryPieces<T>];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int row = pt.first + 16 * t + col;
        load_query<T, D>((const T*)io.q + row_at(L, io, w, row) * D, row < pt.end, a, q[t]);
        lim[t] = row < pt.end ? w.tokens - w.rows / L.G + 1 + row / L.G : 0;
        s[t].clear();
        s[t].m = kLowest;
    }
    int win = -1;  // pages of 64 blocks in the lanes
    // the block's page, -1: none; the block (of no page: any, unused)
    auto fetch = [&](int b, Block<D, KB, VB>& blk) {
        if (((b - lo) & 63) == 0) win = b + lane < hi ? table[(b + lane) >> L.page_shift] : -1;
        const int page = __builtin_amdgcn_readlane(win, (b - lo) & 63);
        const bool good = page >= 0 && page < L.n_pages;
        blk.load(record<F>(L, good ? page : 0, b, w.h), lane);
        return good;
    };
    auto attend = [&](int b, bool good, Block<D, KB, VB>& blk) {
        const int t0 = b * kQuantBlock;
        const bool masked = t0 + kQuantBlock > pt.least;
        if (masked) blk.zero_values_from(w.tokens - t0, a);
        if constexpr (HALF) {
            if (good && __ballot(Half<VB>::outside(blk.ve)) != 0ull) {
                good = inside = false;
                hi = b;  // the end
            }
        }
        if (!good) return;
        int l[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) l[t] = lim[t] - t0;
        if constexpr (HALF) attend_half<D, KB, VB, RT>(blk, q, masked, l, a, io.scale_log2, s);
        else attend_block<T, D, KB, VB, RT>(blk, q, masked, l, a, io.scale_log2, s);
    };
    if (lo < hi) {
        Block<D, KB, VB> b0, b1;
        bool good0 = fetch(lo, b0);
        for (int b = lo; b < hi; b += 2) {
            const bool good1 = fetch(b + 1, b1);
            attend(b, good0, b0);
            if (b + 1 >= hi) break;
            good0 = fetch(b + 2, b0);
            attend(b + 1, good1, b1);
        }
    }
    return inside;
}

template <typename T, int D, int KB, int VB>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_quant_wide(QuantView L,
                                                                                           QuantAttention io) {
    using F = Format<D, KB, VB>;
    constexpr int RT = kRowTiles<T>, TR = kWideRows<T>;
    const int lane = threadIdx.x, a = lane >> 4, col = lane & 15;
    Work w;
    if (!find_work<TR>(L, io, kWideCut, lane, blockIdx.x, w)) return;
    // a row sees the tokens up to its own: query i of `count` lies at tokens - count + i
    auto limit = [&](int row) { return w.tokens - w.rows / L.G + 1 + row / L.G; };
    const int first = w.tile * TR, end = min(first + TR, w.rows);
    const int nb = blocks_of(max(0, limit(end - 1))), per = (nb + w.parts - 1) / w.parts, lo = min(nb, w.part * per);
    const Part pt = {first, end, limit(first), lo, min(nb, lo + per)};
    Softmax<D> s[RT];
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
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int row = first + 16 * t + col;
        const float l = sum_groups(s[t].l);
        if (row >= end) continue;
        if (w.parts > 1) {
            const size_t at = (size_t)(w.slot + w.part) * TR + row - first;
            if (a == 0) *reinterpret_cast<float2*>(io.ml + 2 * at) = make_float2(s[t].m, l);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int ct = 0; ct < F::VC; ct += 4)
                    *reinterpret_cast<f32x4*>(io.part + at * D + (4 * a + r) * F::VC + ct) =
                        f32x4{s[t].o[ct][r], s[t].o[ct + 1][r], s[t].o[ct + 2][r], s[t].o[ct + 3][r]} * unit;
            continue;
        }
        const size_t at = row_at(L, io, w, row);
        const float rl = l == 0.0f ? 0.0f : unit / l;
        if (io.lse != nullptr && a == 0) io.lse[at] = natural_log(s[t].m, l);
        typedef T Tv __attribute__((ext_vector_type(F::VC), aligned(sizeof(T))));
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            Tv y;
#pragma unroll
            for (int ct = 0; ct < F::VC; ++ct) y[ct] = from_f<T>(s[t].o[ct][r] * rl);
            *reinterpret_cast<Tv*>((T*)io.out + at * D + (4 * a + r) * F::VC) = y;
        }
    }
}

// Outputs and log-sum-exps of the rows of split tiles from their parts: a wavefront
// per row, a lane per part for the shares, then 16 bytes per lane of 4 (head_dim 64)
// or 2 parts at a time, eight reads on their way together. The split rows of all
// sequences are dealt out to the wavefronts in turn.
constexpr int kJoinWorkgroups = 1024;
template <typename T, int D>
__global__ __launch_bounds__(256) void k_quant_join(QuantView L, QuantAttention io) {
    constexpr int LANES = D / 4, AT = 64 / LANES, TR = kWideRows<T>;
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
    const size_t grid = most_workgroups(kWideCut, kWideRows<T>, L.batch, io.queries, L.nkv, L.G);
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
    size_t rows = 0;
    for (int tile : {kWideRows<uint16_t>, kWideRows<float>}) {
        const size_t tiles = (size_t)batch * nkv * ((queries * G + tile - 1) / tile);
        rows = std::max(rows, std::min((size_t)2 * kWideCut.target, tiles * kMaxQuantParts) * tile);
    }
    return rows;
}

hipError_t launch_quant_wide(const QuantView& L, bool bf16, const QuantAttention& io, hipStream_t s) {
    return with_types(L, bf16, [&](auto t, auto d, auto kb, auto vb) {
        return launch<decltype(t), d(), kb(), vb()>(L, io, s);
    });
}

}  // namespace raas
