// gfx950 kernels of attention over the quantised cache. For a query row r (head g
// of group h, query i of its sequence) that sees tokens j < n_r:
//   x_rj = q_r . k_j / sqrt(d);  out_r = sum_j exp(x_rj) v_j / sum_j exp(x_rj)
//   lse_r = log sum_j exp(x_rj)
// Codes become bf16 in registers (exactly: at most four significant bits times a
// power of two) and the products run on the matrix cores with fp32 sums.
// Probabilities are fp32 and enter as the sum of two bf16; queries of an fp32
// cache, and its probabilities, as that of three, which is exact.
#include <math.h>

#include <algorithm>

#include "raas_quant_blocks.h"

namespace raas {
namespace {

using namespace qnt;

// ---------------------------------------------------------------------------
// Eight fp32 numbers as the sum of N operands of the bf16 products. Each takes
// the upper 16 bits of what is left, so three leave nothing of an fp32 number; the
// second of two is rounded to bf16, which leaves at most 2^-15 of the number: less
// than 2^-7 after the first, of which rounding is off by half a step, 2^-8. (One
// bf16 alone would be off by 2^-8, as much as the rounding of a bf16 output.)
template <int N>
struct Pieces {
    u32x4 p[N];
    __device__ __forceinline__ Pieces() {}
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
// least `least` blocks, and at most kMaxQuantParts per tile.
struct Cut {
    int target, least;
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

// The workgroup's work, or false where there is less than the grid allows for.
template <int ROWS>
__device__ __forceinline__ bool find_work(const QuantView& L, const QuantAttention& io, const Cut& cut, int lane, int wg,
                                          Work& w) {
    auto tiles_of = [](int rows) { return (rows + ROWS - 1) / ROWS; };
    int t0 = 0, r0 = 0;
    float cost = 0.0f;
    for (int b = lane; b < L.batch; b += 64) {
        sizes_of(L, io, b, t0, r0);
        cost += (float)blocks_of(L, io, t0) * tiles_of(r0);
    }
    if (L.batch <= 64) sizes_of(L, io, lane, t0, r0);
    cost = wave_sum(cost) * L.nkv;
    const int chunk = max(cut.least, (int)ceilf(cost / cut.target));
    auto parts_of = [&](int blocks) {
        return max(1, min(kMaxQuantParts, (blocks + chunk - 1) / chunk));
    };
    int before = 0, slots = 0;
    for (int b0 = 0; b0 < L.batch; b0 += 64) {
        if (L.batch > 64) sizes_of(L, io, b0 + lane, t0, r0);
        const int parts = parts_of(blocks_of(L, io, t0)), n = r0 > 0 ? L.nkv * tiles_of(r0) * parts : 0;
        int upto = n, split = parts > 1 ? n : 0;
        const int own = split;
        upto = scan_sum(upto);
        split = scan_sum(split);
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
        // a tile's parts side by side
        w.slot = slots + of(split) - of(own) + (w.h * w.tiles + w.tile) * w.parts;
        return true;
    }
    return false;
}

// Workgroups that calls of up to these sizes may need.
size_t most_workgroups(const Cut& cut, int row_tile, int batch, int queries, int nkv, int G) {
    return (size_t)cut.target + (size_t)batch * nkv * ((queries * G + row_tile - 1) / row_tile);
}

// ---------------------------------------------------------------------------
// The end of a tile: outputs and log-sum-exps of its rows 0 .. rows - 1 from
// `nsrc` disjoint parts of the tokens (ml: reference and sum, o: unnormalised
// outputs) and those of the prefix. A wavefront per row, a lane per part finds the
// shares; then a thread per output element. s_w: [nsrc + prefix parts][16].
constexpr int kFinishSources = kMaxQuantParts + kMaxPrefixParts;
template <typename T, int D, int NW, class Ml, class O>
__device__ __forceinline__ void finish_rows(const QuantView& L, const QuantAttention& io, const Work& w, int row0,
                                            int rows, int tid, int nsrc, float (*s_w)[16], Ml ml, O o) {
    const int lane = tid & 63;
    const PrefixParts& pp = io.prefix;
    const size_t prows = (size_t)L.nkv * pp.rows, prow = (size_t)w.h * pp.rows + (size_t)w.b * L.G;
    const int parts = nsrc + pp.n;
    auto to = [&](int row) {  // the row's place in out and lse
        const int i = (row0 + row) / L.G, g = row0 + row - i * L.G;
        return ((size_t)w.b * io.queries + i) * L.nkv * L.G + w.h * L.G + g;
    };
    for (int row = wave_of(tid); row < rows; row += NW) {
        auto part_ml = [&](int s) {
            if (s < nsrc) return ml(s, row);
            const float* x = pp.ml + 2 * ((size_t)(s - nsrc) * prows + prow + row);
            return make_float2(x[0], x[1]);
        };
        const float2 none = make_float2(-INFINITY, 0.0f);
        const float2 x = lane < parts ? part_ml(lane) : none, y = lane + 64 < parts ? part_ml(lane + 64) : none;
        const float M = fmaxf(wave_max(fmaxf(x.x, y.x)), -1e30f);
        const float ex = __builtin_amdgcn_exp2f(x.x - M), ey = __builtin_amdgcn_exp2f(y.x - M);
        const float Z = wave_sum(x.y * ex + y.y * ey), rz = Z > 0.0f ? 1.0f / Z : 0.0f;
        if (lane < parts) s_w[lane][row] = ex * rz;
        if (lane + 64 < parts) s_w[lane + 64][row] = ey * rz;
        if (io.lse != nullptr && lane == 0)
            io.lse[to(row)] = Z > 0.0f ? (M + __builtin_amdgcn_logf(Z)) * 0.69314718055994530942f : -INFINITY;
    }
    __syncthreads();
    for (int e = tid; e < rows * D; e += NW * 64) {
        const int row = e / D, c = e % D;
        float x = 0.0f;
        for (int s0 = 0; s0 < nsrc; s0 += 8) {  // eight on their way together
            float y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = o(min(s0 + k, nsrc - 1), row, c);
#pragma unroll
            for (int k = 0; k < 8; ++k) x = __builtin_fmaf(y[k], s0 + k < nsrc ? s_w[s0 + k][row] : 0.0f, x);
        }
        for (int s0 = 0; s0 < pp.n; s0 += 8) {
            float y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = pp.o[(min(s0 + k, pp.n - 1) * prows + prow + row) * D + c];
#pragma unroll
            for (int k = 0; k < 8; ++k) x = __builtin_fmaf(y[k], s0 + k < pp.n ? s_w[nsrc + s0 + k][row] : 0.0f, x);
        }
        ((T*)io.out)[to(row) * D + c] = from_f<T>(x);
    }
    __syncthreads();
}

// The softmax's reference need not be the maximum: it follows a row's logits once
// they exceed it by this much (base 2), so that the sums stay within 2^kSlack of
// their usual size and most blocks need no maximum over lanes. It starts at a
// finite number far below every logit: the difference to a masked logit is then
// -inf, never NaN.
constexpr float kSlack = 8.0f, kLowest = -1e30f;

// One block against RT tiles of 16 rows. A row of this lane's column sees tokens
// below lim[t] of the block; `masked`: some row does not see all of them.
template <typename T, int D, int KB, int VB, int RT>
__device__ __forceinline__ void attend_block(const Block<D, KB, VB>& blk, const u32x4 (&q)[RT][D / 32][kQueryPieces<T>],
                                             bool masked, const int (&lim)[RT], int a, float scale_log2,
                                             Softmax<D> (&s)[RT]) {
    constexpr int KS = D / 32, NQ = kQueryPieces<T>, NP = kProbPieces<T>;
    f32x4 x[RT][2];
#pragma unroll
    for (int t = 0; t < RT; ++t) x[t][0] = x[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const float scale = blk.key_scale(c);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const u32x4 k = blk.key(c, ks, scale);
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int n = 0; n < NQ; ++n) x[t][c] = mfma(k, q[t][ks][n], x[t][c]);
        }
    }
    if (masked) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[t][c][e] = 8 * a + 4 * c + e < lim[t] ? x[t][c][e] : -INFINITY;
    }
    float mb[RT];
    bool over = false;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        mb[t] = x[t][0][0];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) mb[t] = fmaxf(mb[t], x[t][c][e]);
        mb[t] *= scale_log2;
        over = over || mb[t] > s[t].m + kSlack;
    }
    if (__ballot(over) != 0ull) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const float m = fmaxf(s[t].m, max_groups(mb[t]));
            const float alpha = __builtin_amdgcn_exp2f(s[t].m - m);
            s[t].l *= alpha;
#pragma unroll
            for (int ct = 0; ct < D / 16; ++ct) s[t].o[ct] *= alpha;
            s[t].m = m;
        }
    }
    Pieces<NP> p[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float y[8], l = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            y[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][j >> 2][j & 3], scale_log2, -s[t].m));
            l += y[j];
        }
        s[t].l += l;
        p[t] = Pieces<NP>(y);
    }
    float vs[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) vs[j] = blk.value_scale(j);
    auto two = [&](auto m) {
        constexpr int M = decltype(m)::value;
        u32x4 even, odd;
        blk.template values<M>(vs, even, odd);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int n = 0; n < NP; ++n) {
                s[t].o[2 * M] = mfma(even, p[t].p[n], s[t].o[2 * M]);
                s[t].o[2 * M + 1] = mfma(odd, p[t].p[n], s[t].o[2 * M + 1]);
            }
    };
    two(Int<0>());
    two(Int<1>());
    if constexpr (D == 128) {
        two(Int<2>());
        two(Int<3>());
    }
}

// A step's new token, quantised into the lanes that hold its place in the tail
// block (token t of it), and stored; k_held, v_held receive what is held.
template <typename T, int D, int KB, int VB>
__device__ __forceinline__ void take_token(const QuantAttention& io, Block<D, KB, VB>& blk, uint8_t* rec, int t,
                                           size_t unit, int lane) {
    using F = Format<D, KB, VB>;
    const int a = lane >> 4, i = lane & 15, q = t >> 2 & 1, j = t & 7;
    if (i == 4 * (t >> 3) + (t & 3)) {
        uint32_t code[F::KD];
        const uint32_t e = encode_key<T, D, KB>((const T*)io.k_new + unit * D, a, code);
        blk.ke = q ? (blk.ke & 0x00FFu) | e << 8 : (blk.ke & 0xFF00u) | e;
        rec[F::KEXP + (F::kgroup(a) * 16 + i) * 2 + q] = (uint8_t)e;  // (lanes of one group write the same)
#pragma unroll
        for (int qq = 0; qq < 2; ++qq)
            if (qq == q) {
#pragma unroll
                for (int x = 0; x < F::KD; ++x) {
                    const int at = qq * F::KD + x;
                    blk.k[at / 4][at % 4] = code[x];
                    *reinterpret_cast<uint32_t*>(rec + 1024 * (at / 4) + 16 * lane + 4 * (at % 4)) = code[x];
                }
                if (io.k_held != nullptr) {
                    uint32_t y[F::KC / 2];
#pragma unroll
                    for (int ks = 0; ks < F::KS; ++ks) {
                        const u32x4 z = blk.key(qq, ks, scale_of(e));
#pragma unroll
                        for (int k = 0; k < 4; ++k) y[4 * ks + k] = z[k];
                    }
                    store_values<T, F::KC>((T*)io.k_held + unit * D + a * F::KC, y);
                }
            }
    }
    if (a == t >> 3) {
        u32x2 code;
        const uint32_t e = encode_value<T, D, VB>((const T*)io.v_new + unit * D, i, code);
#pragma unroll
        for (int jj = 0; jj < 8; ++jj)
            if (jj == j) {
                blk.set_value(jj, code);
                blk.set_exponent(jj, e);
                store_value<D, KB, VB>(rec, lane, jj, code);
                rec[F::VEXP + (a * F::NG + F::vgroup(i)) * 8 + jj] = (uint8_t)e;
                if (io.v_held != nullptr) {
                    uint32_t y[F::VC / 2];
                    blk.value_row(jj, y);
                    store_values<T, F::VC>((T*)io.v_held + unit * D + i * F::VC, y);
                }
            }
    }
}

// ---------------------------------------------------------------------------
// Few rows per unit: a workgroup's wavefronts take the blocks of its part in
// turn, a block on its way while the one before it is attended to, join in LDS,
// and write the outputs, or publish the part: the last of a tile's parts to end
// joins them all. Pages of a wavefront's next 64 blocks lie in its lanes.
constexpr int kStreamWaves = 4;
template <typename T, int RT>
constexpr int kStreamPerSimd = sizeof(T) == 4 ? 1 : RT == 1 ? 3 : 2;
constexpr Cut kStreamCut = {768, 2 * kStreamWaves};

template <typename T, int D, int KB, int VB, int RT>
__global__ __launch_bounds__(kStreamWaves * 64) __attribute__((amdgpu_waves_per_eu(kStreamPerSimd<T, RT>))) void k_quant_stream(QuantView L, QuantAttention io) {
    using F = Format<D, KB, VB>;
    constexpr int NW = kStreamWaves, TR = 16 * RT;
    __shared__ __align__(16) float s_o[NW][16][D + 4];
    __shared__ float s_m[NW][16], s_l[NW][16], s_w[kFinishSources][16];
    const int tid = threadIdx.x, lane = tid & 63, wv = wave_of(tid), a = lane >> 4, col = lane & 15;
    Work w;
    if (!find_work<TR>(L, io, kStreamCut, lane, blockIdx.x, w)) return;
    const int rows = min(TR, w.rows - w.tile * TR), count = w.rows / L.G;
    // a row sees the tokens up to its own: query i of `count` lies at tokens - count + i
    auto limit = [&](int row) { return w.tokens - count + 1 + row / L.G; };
    int lim[RT];
    u32x4 q[RT][F::KS][kQueryPieces<T>];
    Softmax<D> s[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int row = w.tile * TR + 16 * t + col, i = row / L.G, g = row - i * L.G;
        const bool real = 16 * t + col < rows;
        const size_t at = ((size_t)w.b * io.queries + i) * L.nkv * L.G + w.h * L.G + g;
        load_query<T, D>((const T*)io.q + at * D, real, a, q[t]);
        lim[t] = real ? limit(row) : 0;
        s[t].clear();
        s[t].m = kLowest;
    }
    const int first = w.tile * TR, most = max(0, limit(first + rows - 1)), least = limit(first);
    const int nb = blocks_of(most), per = (nb + w.parts - 1) / w.parts;
    const int lo = min(nb, w.part * per), hi = min(nb, lo + per);
    const int32_t* table = L.table + (size_t)w.b * L.width;
    int win = -1;  // page of this wavefront's block number (turn & ~63) + lane
    auto window = [&](int turn) {
        const int b = lo + wv + (turn + lane) * NW;
        win = b < hi ? table[b >> L.page_shift] : -1;
    };
    // This wavefront's blocks. The sequence's last one, if it is here, comes last, and
    // only it takes a new token or ends with places that hold none.
    const int turns = lo + wv < hi ? (hi - lo - wv + NW - 1) / NW : 0;
    Block<D, KB, VB> b0, b1;
    // page of the turn's block, -1: none; the block (of no page: any, unused)
    auto fetch = [&](int turn, Block<D, KB, VB>& blk) {
        if ((turn & 63) == 0) window(turn);
        int page = __builtin_amdgcn_readlane(win, turn & 63);
        page = page >= 0 && page < L.n_pages ? page : -1;
        blk.load(record<F>(L, max(page, 0), lo + wv + turn * NW, w.h), lane);
        return page;
    };
    auto attend = [&](int b, Block<D, KB, VB>& blk) {
        const int t0 = b * kQuantBlock;
        int l[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) l[t] = lim[t] - t0;
        attend_block<T, D, KB, VB, RT>(blk, q, t0 + kQuantBlock > least, l, a, io.scale_log2, s);
    };
    if (turns > 0) {
        int p0 = fetch(0, b0), turn = 0;
        while (turn + 1 < turns) {
            const int p1 = fetch(turn + 1, b1);
            if (p0 >= 0) attend(lo + wv + turn * NW, b0);
            if (++turn + 1 >= turns) {
                b0 = b1;
                p0 = p1;
                break;
            }
            p0 = fetch(turn + 1, b0);
            if (p1 >= 0) attend(lo + wv + turn * NW, b1);
            ++turn;
        }
        if (p0 >= 0) {
            const int b = lo + wv + turn * NW, t0 = b * kQuantBlock;
            if (w.fresh >= t0 && w.fresh < t0 + kQuantBlock)
                take_token<T, D, KB, VB>(io, b0, record<F>(L, p0, b, w.h), w.fresh - t0, (size_t)w.b * L.nkv + w.h, lane);
            if (t0 + kQuantBlock > w.tokens) b0.zero_values_from(w.tokens - t0, a);
            attend(b, b0);
        }
    }
    const bool split = w.parts > 1;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int here = min(16, rows - 16 * t);
        if (here <= 0) break;
        const float l = sum_groups(s[t].l);
        if (a == 0) {
            s_m[wv][col] = s[t].m;
            s_l[wv][col] = l;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float* to = &s_o[wv][col][(4 * a + r) * F::VC];
#pragma unroll
            for (int ct = 0; ct < F::VC; ct += 4)
                *reinterpret_cast<f32x4*>(to + ct) =
                    f32x4{s[t].o[ct][r], s[t].o[ct + 1][r], s[t].o[ct + 2][r], s[t].o[ct + 3][r]};
        }
        __syncthreads();
        auto ml = [&](int k, int row) { return make_float2(s_m[k][row], s_l[k][row]); };
        if (!split) {
            finish_rows<T, D, NW>(L, io, w, first + 16 * t, here, tid, NW, s_w, ml,
                                  [&](int k, int row, int c) { return s_o[k][row][c]; });
            continue;
        }
        const size_t slot = (size_t)(w.slot + w.part) * TR + 16 * t;
        for (int e = tid; e < here * D; e += NW * 64) {
            const int row = e / D, c = e % D;
            float M = kLowest, x = 0.0f, z = 0.0f;
#pragma unroll
            for (int k = 0; k < NW; ++k) M = fmaxf(M, s_m[k][row]);
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                const float share = __builtin_amdgcn_exp2f(s_m[k][row] - M);
                x = __builtin_fmaf(s_o[k][row][c], share, x);
                z = __builtin_fmaf(s_l[k][row], share, z);
            }
            publish(io.part + (slot + row) * D + c, x);
            if (c == 0) {
                publish(io.ml + 2 * (slot + row), M);
                publish(io.ml + 2 * (slot + row) + 1, z);
            }
        }
        __syncthreads();
    }
    if (!split) return;
    const int tiles = (io.queries * L.G + TR - 1) / TR;  // (of the call: the counters' layout)
    if (!arrive_last(io.arrived + ((size_t)w.b * L.nkv + w.h) * tiles + w.tile, w.parts)) return;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int here = min(16, rows - 16 * t);
        if (here <= 0) break;
        auto at = [&](int k, int row) { return (size_t)(w.slot + k) * TR + 16 * t + row; };
        finish_rows<T, D, NW>(
            L, io, w, first + 16 * t, here, tid, w.parts, s_w,
            [&](int k, int row) {
                return make_float2(published(io.ml + 2 * at(k, row)), published(io.ml + 2 * at(k, row) + 1));
            },
            [&](int k, int row, int c) { return published(io.part + at(k, row) * D + c); });
    }
}

template <typename T, int D, int KB, int VB>
hipError_t launch(const QuantView& L, const QuantAttention& io, hipStream_t s) {
    const int rows = io.queries * L.G;
    auto go = [&](auto kernel, int tile) {
        const size_t grid = most_workgroups(kStreamCut, tile, L.batch, io.queries, L.nkv, L.G);
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kStreamWaves * 64), 0, s, L, io);
    };
    if (rows <= 16) go(k_quant_stream<T, D, KB, VB, 1>, 16);
    else go(k_quant_stream<T, D, KB, VB, 2>, 32);
    return hipGetLastError();
}

}  // namespace

QuantScratch quant_scratch(int batch, int queries, int nkv, int G) {
    // Every split tile has at least two parts of `chunk` blocks but for the last, and
    // all blocks together are at most target * chunk: at most 2 target slots.
    auto tiles = [&](int r) { return (size_t)batch * nkv * ((queries * G + r - 1) / r); };
    QuantScratch x{};
    for (int r : {16, 32}) {
        x.rows = std::max(x.rows, std::min((size_t)2 * kStreamCut.target, tiles(r) * kMaxQuantParts) * r);
        x.arrivals = std::max(x.arrivals, tiles(r));
    }
    return x;
}

hipError_t launch_quant_attention(const QuantView& L, bool bf16, const QuantAttention& io, hipStream_t s) {
    return with_types(L, bf16, [&](auto t, auto d, auto kb, auto vb) {
        return launch<decltype(t), d(), kb(), vb()>(L, io, s);
    });
}

}  // namespace raas
