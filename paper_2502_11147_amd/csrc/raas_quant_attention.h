// What the kernels of attention over the quantised cache have in common: operands
// of the products, and which rows and blocks a workgroup takes.
#pragma once

#include "raas_quant_blocks.h"

namespace raas {
namespace qnt {

// ---------------------------------------------------------------------------
// Eight fp32 numbers as the sum of N operands of the bf16 products. Each takes
// the upper 16 bits of what is left, so three leave nothing of an fp32 number; the
// second of two is rounded to bf16, which leaves at most 2^-15 of the number: less
// than 2^-7 after the first, of which rounding is off by half a step, 2^-8. (One
// bf16 alone would be off by 2^-8, as much as the rounding of a bf16 output.)
template <int N>
struct Pieces {
    u32x4 p[N];
    __device__ __forceinline__ explicit Pieces(const float (&x)[8]) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[j];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (N == 2 && n == 1) {
                bf16x8 r;
#pragma unroll
                for (int j = 0; j < 8; ++j) r[j] = (__bf16)y[j];
                p[n] = __builtin_bit_cast(u32x4, r);
                break;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)  // the upper halves of two side by side
                p[n][j] = __builtin_amdgcn_perm(__float_as_uint(y[2 * j + 1]), __float_as_uint(y[2 * j]), 0x07060302u);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] -= __uint_as_float(__float_as_uint(y[j]) & 0xFFFF0000u);
        }
    }
};
// operands that a query, and a probability, of a cache of T is made of
template <typename T>
constexpr int kQueryPieces = sizeof(T) == 2 ? 1 : 3;
template <typename T>
constexpr int kProbPieces = sizeof(T) == 2 ? 2 : 3;

__device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, f32x4 c) { return mfma16<uint16_t>(a, b, c); }

// This lane's channels D/4 a + 8 ks .. of a query row.
template <typename T, int D>
__device__ __forceinline__ void load_query(const T* row, bool real, int a,
                                           u32x4 (&q)[D / 32][kQueryPieces<T>]) {
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
        const T* at = row + a * (D / 4) + 8 * ks;
        if constexpr (sizeof(T) == 2) {
            q[ks][0] = real ? ld16_in<T>(at) : u32x4{0u, 0u, 0u, 0u};
        } else {
            float x[8] = {};
            if (real) load_floats<T, 8>(at, x);
            const Pieces<3> p(x);
#pragma unroll
            for (int n = 0; n < 3; ++n) q[ks][n] = p.p[n];
        }
    }
}

// ---------------------------------------------------------------------------
// Which rows and blocks a workgroup takes. The rows of a unit (queries of its
// sequence times G heads) are cut into tiles, a tile's tokens into parts of about
// equally many blocks over the whole batch, so that ragged sequences load the
// chip evenly: every workgroup finds its own from the lengths, which the host does
// not know. Parts are cut so that about `target` workgroups come out, but of at
// least `least` blocks, of 8 where there would be more than 16 of them, and at most
// kMaxQuantParts per tile; a tile of up to `whole` blocks is not cut.
struct Cut {
    int target, least, whole;
};
struct Work {
    int b, h, tile, tiles, part, parts;
    int slot;    // of the tile's first part in the scratch, if parts > 1
    int tokens;  // held by the sequence, a step's new one among them
    int fresh;   // place of a step's new token, -1: none
    int rows;    // of the unit
};

__device__ __forceinline__ int blocks_of(int tokens) { return (tokens + kQuantBlock - 1) / kQuantBlock; }
// A sequence's tokens before the call and its rows per unit; rows 0: it sits out.
__device__ __forceinline__ void sizes_of(const QuantView& L, const QuantAttention& io, int b, int& held, int& rows) {
    held = rows = 0;
    if (b >= L.batch) return;
    const int len = io.len[b], count = io.count != nullptr ? min(io.count[b], io.queries) : io.queries;
    if (len < 0 || count <= 0) return;
    held = min(len, L.cap);
    rows = count * L.G;
}
// Blocks that the call attends to (a step's new token counts if it finds a place).
__device__ __forceinline__ int blocks_of(const QuantView& L, const QuantAttention& io, int held) {
    return blocks_of(held + (io.k_new != nullptr && held < L.cap ? 1 : 0));
}

// Sum over this lane and those before it: within rows of 16 lanes by 1, 2, 4 and 8
// places, then the last lane of a row, and of the lower half, onto those behind.
__device__ __forceinline__ int scan_sum(int x) {
    auto add = [&](auto ctrl, auto rows) {
        x += __builtin_amdgcn_update_dpp(0, x, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
    };
    add(Int<0x111>(), Int<0xF>());
    add(Int<0x112>(), Int<0xF>());
    add(Int<0x114>(), Int<0xF>());
    add(Int<0x118>(), Int<0xF>());
    add(Int<0x142>(), Int<0xA>());
    add(Int<0x143>(), Int<0xC>());
    return x;
}

// Blocks of a part, by which each workgroup cuts the sequences.
template <int ROWS>
__device__ __forceinline__ int chunk_of(const QuantView& L, const QuantAttention& io, const Cut& cut, int lane) {
    float cost = 0.0f;
    for (int b = lane; b < L.batch; b += 64) {
        int held, rows;
        sizes_of(L, io, b, held, rows);
        cost += (float)blocks_of(L, io, held) * ((rows + ROWS - 1) / ROWS);
    }
    return (int)ceilf(wave_sum(cost) * L.nkv / cut.target);
}
__device__ __forceinline__ int parts_of(int blocks, int chunk, const Cut& cut) {
    const int each = max(chunk, blocks > 16 * cut.least ? 8 : cut.least);
    return blocks <= cut.whole ? 1 : min(kMaxQuantParts, (blocks + each - 1) / each);
}

// The work of workgroup `wg`, or false where there is less than the grid allows for.
template <int ROWS>
__device__ __forceinline__ bool find_work(const QuantView& L, const QuantAttention& io, const Cut& cut, int lane, int wg,
                                          Work& w) {
    auto tiles_of = [](int rows) { return (rows + ROWS - 1) / ROWS; };
    const int chunk = chunk_of<ROWS>(L, io, cut, lane);
    int before = 0, slots = 0;
    for (int b0 = 0; b0 < L.batch; b0 += 64) {
        int t0, r0;
        sizes_of(L, io, b0 + lane, t0, r0);
        const int parts = parts_of(blocks_of(L, io, t0), chunk, cut), n = L.nkv * tiles_of(r0) * parts, own = parts > 1 ? n : 0;
        const int upto = scan_sum(n), split = scan_sum(own);
        const unsigned long long m = __ballot(wg < before + upto);
        if (m == 0ull) {
            before += __builtin_amdgcn_readlane(upto, 63);
            slots += __builtin_amdgcn_readlane(split, 63);
            continue;
        }
        const int at = __ffsll(m) - 1;
        auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
        w.b = b0 + at;
        const int held = of(t0);
        w.fresh = io.k_new != nullptr && held < L.cap ? held : -1;
        w.tokens = held + (w.fresh >= 0 ? 1 : 0);
        w.rows = of(r0);
        w.parts = of(parts);
        w.tiles = tiles_of(w.rows);
        // KV heads innermost, so that with eight of them the tiles and parts of one
        // meet on an XCD; the tiles that see the most tokens first
        const int idx = wg - (before + of(upto) - of(n)), rest = idx / L.nkv;
        w.h = idx - rest * L.nkv;
        const int turn = rest / w.parts;
        w.part = rest - turn * w.parts;
        w.tile = w.tiles - 1 - turn;
        // a tile's parts lie side by side
        w.slot = slots + of(split) - of(own) + (w.h * w.tiles + w.tile) * w.parts;
        return true;
    }
    return false;
}

// go(work, row) for the rows i, i + step, ... among all rows of split sequences.
template <int ROWS, class Go>
__device__ __forceinline__ void for_split_rows(const QuantView& L, const QuantAttention& io, const Cut& cut, int lane,
                                               int i, int step, Go go) {
    const int chunk = chunk_of<ROWS>(L, io, cut, lane);
    int before = 0, slots = 0;
    for (int b0 = 0; b0 < L.batch; b0 += 64) {
        int t0, r0;
        sizes_of(L, io, b0 + lane, t0, r0);
        const int parts = parts_of(blocks_of(L, io, t0), chunk, cut), tiles = (r0 + ROWS - 1) / ROWS;
        const int n = parts > 1 ? L.nkv * r0 : 0, own = parts > 1 ? L.nkv * tiles * parts : 0;
        const int upto = scan_sum(n), split = scan_sum(own), all = before + __builtin_amdgcn_readlane(upto, 63);
        for (; i < all; i += step) {
            const int at = __ffsll(__ballot(i < before + upto)) - 1;
            auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
            Work w;
            w.b = b0 + at;
            w.rows = of(r0);
            w.parts = of(parts);
            w.tiles = of(tiles);
            const int idx = i - (before + of(upto) - of(n)), row = idx / L.nkv;
            w.h = idx - row * L.nkv;
            w.tile = row / ROWS;
            w.slot = slots + of(split) - of(own);
            go(w, row);
        }
        before = all;
        slots += __builtin_amdgcn_readlane(split, 63);
    }
}

// The softmax's reference need not be the maximum: it follows a row's logits once
// they exceed it by this much (base 2), so that the sums stay within 2^kSlack of
// their usual size and most blocks need no maximum over lanes. It starts at a
// finite number far below every logit: the difference to a masked logit is then
// -inf, never NaN.
constexpr float kSlack = 8.0f, kLowest = -1e30f;

// Logits (unscaled) of a block's keys and 16 rows. (v_mfma_scale_f32_16x16x128_f8f6f4
// takes keys of 4 bits as they are stored, beside a query as two e4m3 numbers, and saves
// the 36 conversions of a block; but its sums are off by up to 1.3e-5 of the products'
// magnitudes, a hundred times what these are: a log-sum-exp was off by 3e-4.) The row of
// this lane's column sees tokens below lim of the block; `masked`: some row does not see all.
template <typename T, int D, int KB, int VB>
__device__ __forceinline__ void block_logits(const Block<D, KB, VB>& blk, const u32x4 (&q)[D / 32][kQueryPieces<T>],
                                             bool masked, int lim, int a, f32x4 (&x)[2]) {
    x[0] = x[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const float scale = blk.key_scale(c);
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) {
            const u32x4 k = blk.key(c, ks, scale);
#pragma unroll
            for (int n = 0; n < kQueryPieces<T>; ++n) x[c] = mfma(k, q[ks][n], x[c]);
        }
    }
    if (masked) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[c][e] = 8 * a + 4 * c + e < lim ? x[c][e] : -INFINITY;
    }
}

// Lets the rows' references follow their logits.
template <int D>
__device__ __forceinline__ void follow(const f32x4 (&x)[2], float scale_log2, Softmax<D>& s) {
    float mb = x[0][0];
#pragma unroll
    for (int j = 1; j < 8; ++j) mb = fmaxf(mb, x[j >> 2][j & 3]);
    mb *= scale_log2;
    if (__ballot(mb > s.m + kSlack) == 0ull) return;
    const float m = fmaxf(s.m, max_groups(mb));
    const float alpha = __builtin_amdgcn_exp2f(s.m - m);
    s.l *= alpha;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) s.o[ct] *= alpha;
    s.m = m;
}

// A block some of whose tokens not every row sees, with NaN among its values: a product
// would give it to all rows, a masked probability being 0. The NaN go to the outputs of
// the rows that see them (tokens below lim) and become numbers in the block.
template <int D, int KB, int VB>
__device__ __forceinline__ void hand_out_nan(Block<D, KB, VB>& blk, int lim, int a, Softmax<D>& s) {
    using F = Format<D, KB, VB>;
    const uint32_t own = nan_mask(blk.ve);
    // tokens with NaN in this lane's outputs, channels D/4 a .., which lie in one group
    uint32_t all = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) all |= (uint32_t)__shfl((int)own, 16 * b + F::kgroup(a) * F::VSHARE) << (8 * b);
    const bool hit = lim > 0 && (all << (32 - min(lim, 32))) != 0u;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct)
        if (hit) s.o[ct] = f32x4{NAN, NAN, NAN, NAN};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (own >> j & 1u) {
            if constexpr (VB == 8) blk.set_value(j, u32x2{0u, 0u});  // (4 bits have no NaN of their own)
            blk.set_exponent(j, kZeroExponent);
        }
}

// One block against 16 rows.
template <typename T, int D, int KB, int VB>
__device__ __forceinline__ void attend_block(const Block<D, KB, VB>& blk, const u32x4 (&q)[D / 32][kQueryPieces<T>],
                                             bool masked, int lim, int a, float scale_log2, Softmax<D>& s) {
    constexpr int NP = kProbPieces<T>;
    f32x4 x[2];
    block_logits<T, D, KB, VB>(blk, q, masked, lim, a, x);
    follow<D>(x, scale_log2, s);
    float y[8], l = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        y[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j >> 2][j & 3], scale_log2, -s.m));
        l += y[j];
    }
    s.l += l;
    const Pieces<NP> p(y);
    float vs[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) vs[j] = blk.value_scale(j);
    auto two = [&](auto m) {
        constexpr int M = decltype(m)::value;
        u32x4 even, odd;
        blk.template values<M>(vs, even, odd);
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            s.o[2 * M] = mfma(even, p.p[n], s.o[2 * M]);
            s.o[2 * M + 1] = mfma(odd, p.p[n], s.o[2 * M + 1]);
        }
    };
    two(Int<0>());
    two(Int<1>());
    if constexpr (D == 128) {
        two(Int<2>());
        two(Int<3>());
    }
}

// Natural logarithm of sum 2^m; -inf of none.
__device__ __forceinline__ float natural_log(float m, float sum) {
    return sum == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

// A row's place in out and lse.
__device__ __forceinline__ size_t row_at(const QuantView& L, const QuantAttention& io, const Work& w, int row) {
    const int i = row / L.G, g = row - i * L.G;
    return ((size_t)w.b * io.queries + i) * L.nkv * L.G + w.h * L.G + g;
}

// Workgroups that calls of up to these sizes may need.
inline size_t most_workgroups(const Cut& cut, int row_tile, int batch, int queries, int nkv, int G) {
    return (size_t)cut.target + (size_t)batch * nkv * ((queries * G + row_tile - 1) / row_tile);
}

}  // namespace qnt
}  // namespace raas
