// gfx950 kernels of attention over the quantised cache. For a query row r (head g
// of group h, query i of its sequence) that sees tokens j < n_r:
//   x_rj = q_r . k_j / sqrt(d);  out_r = sum_j exp(x_rj) v_j / sum_j exp(x_rj)
//   lse_r = log sum_j exp(x_rj)
// Codes become bf16 in registers (exactly: at most four significant bits times a
// power of two) and the products run on the matrix cores with fp32 sums.
// Probabilities are fp32 and enter as the sum of two bf16; queries of an fp32
// cache, and its probabilities, as that of three, which is exact. Here units of few
// rows; raas_quant_wide.hip takes more.
#include <math.h>

#include <algorithm>

#include "raas_quant_attention.h"

namespace raas {
namespace {

using namespace qnt;

// ---------------------------------------------------------------------------
// The end of a tile: outputs and log-sum-exps of its rows 0 .. rows - 1 from
// `nsrc` disjoint parts of the tokens (ml: reference and sum, o: unnormalised
// outputs) and those of the prefix. A wavefront per row, a lane per part finds the
// shares; then a thread per four channels. s_w: [nsrc + prefix parts][16].
constexpr int kFinishSources = kMaxQuantParts + kMaxPrefixParts;
template <typename T, int D, int NW, class Ml, class O>
__device__ __forceinline__ void finish_rows(const QuantView& L, const QuantAttention& io, const Work& w, int row0,
                                            int rows, int tid, int nsrc, float (*s_w)[16], Ml ml, O o) {
    const int lane = tid & 63;
    const PrefixParts& pp = io.prefix;
    const size_t prows = (size_t)L.nkv * pp.rows, prow = (size_t)w.h * pp.rows + (size_t)w.b * L.G;
    const int parts = nsrc + pp.n;
    auto to = [&](int row) { return row_at(L, io, w, row0 + row); };
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
        const float Z = wave_sum(x.y * ex + y.y * ey), rz = Z == 0.0f ? 0.0f : 1.0f / Z;
        if (lane < parts) s_w[lane][row] = ex * rz;
        if (lane + 64 < parts) s_w[lane + 64][row] = ey * rz;
        if (io.lse != nullptr && lane == 0)
            io.lse[to(row)] = natural_log(M, Z);
    }
    __syncthreads();
    typedef T T4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    for (int e = tid; e < rows * (D / 4); e += NW * 64) {
        const int row = e / (D / 4), c = e % (D / 4) * 4;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        // up to 16 reads on their way together; those of the last turn past the end are the last part's again
        auto add = [&](int n, int w0, auto value) {
            auto turn = [&](auto ahead, int s0) {
                constexpr int AHEAD = decltype(ahead)::value;
                f32x4 y[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) y[k] = value(min(s0 + k, n - 1));
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) x += y[k] * (s0 + k < n ? s_w[w0 + s0 + k][row] : 0.0f);
            };
            for (int s0 = 0; s0 < n; s0 += 16) {
                if (n - s0 > 8) turn(Int<16>(), s0);
                else if (n - s0 > 4) turn(Int<8>(), s0);
                else turn(Int<4>(), s0);
            }
        };
        add(nsrc, 0, [&](int k) { return o(k, row, c); });
        add(pp.n, nsrc, [&](int k) { return *reinterpret_cast<const f32x4*>(pp.o + (k * prows + prow + row) * D + c); });
        T4 y;
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = from_f<T>(x[k]);
        *reinterpret_cast<T4*>((T*)io.out + to(row) * D + c) = y;
    }
    __syncthreads();
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
// Up to 16 rows per unit: a workgroup's wavefronts take the blocks of its part in
// turn, a block on its way while the one before it is attended to, join in LDS,
// and write the outputs, or publish the part: the last of a unit's parts to end
// joins them all. Pages of a wavefront's next 64 blocks lie in its lanes. Bound by
// memory, 4.25 or 8.25 bits a value (128 sequences of 8192 tokens in 4 bits 6.3 TB/s);
// small calls by the chain of lengths, table, block, join (6 us, 8 with parts).
constexpr int kStreamWaves = 4, kStreamRows = 16;
// Blocks of a wavefront on their way or in use, and wavefronts per SIMD. A layer
// that streams from memory in 4 bits (128 sequences of 8192 tokens) takes 221 us
// with two and three, 198 with non-temporal loads, 181 with four and two besides;
// caches that stay near are no faster so (49 and 52 us, 64 sequences of 4096), nor
// are 8 bits (91 and 92), whose blocks are twice as large.
template <typename T, int KB, int VB, bool STREAM>
constexpr int kStreamBlocks = STREAM && KB + VB == 8 && sizeof(T) == 2 ? 4 : 2;
template <typename T, int KB, int VB, bool STREAM>
constexpr int kStreamPerSimd = sizeof(T) == 4 ? 1 : kStreamBlocks<T, KB, VB, STREAM> == 4 ? 2 : 3;
// Not more than two either: with three, for which its registers would do, it takes 200 us.
// (head_dim 64: 200 with four, 226 with two.)
template <typename T, int D, int KB, int VB, bool STREAM>
constexpr int kStreamMost = kStreamBlocks<T, KB, VB, STREAM> == 4 && D == 128 ? 2 : 8;
// Parts: of 8 KV heads with 30000 tokens in 64, 43 and 32 parts 17.9, 17.0 and 15.2 us:
// publishing a part and joining it costs more than a workgroup's share of an even
// load, once every compute unit has one. One sequence of 1000 tokens takes 8.2, 8.8
// and 9.9 us in parts of 4, 8 and 16 blocks, of 4000 tokens 10.8 and 8.9 of 4 and 8
// (a join has 16 parts on their way together). Publishing at all costs as much as
// five turns: one sequence of 300 tokens takes 7.2 us in one part, 8.6 in two, of
// 600 tokens 8.4 and 8.9.
constexpr Cut kStreamCut = {256, 4, 20};

template <typename T, int D, int KB, int VB, bool STREAM>
__global__ __launch_bounds__(kStreamWaves * 64)
__attribute__((amdgpu_waves_per_eu(kStreamPerSimd<T, KB, VB, STREAM>, kStreamMost<T, D, KB, VB, STREAM>)))
void k_quant_stream(QuantView L, QuantAttention io) {
    using F = Format<D, KB, VB>;
    constexpr int NW = kStreamWaves, NB = kStreamBlocks<T, KB, VB, STREAM>;
    __shared__ __align__(16) float s_o[NW][16][D + 4];
    __shared__ float s_m[NW][16], s_l[NW][16], s_w[kFinishSources][16];
    const int tid = threadIdx.x, lane = tid & 63, wv = wave_of(tid), a = lane >> 4, col = lane & 15;
    Work w;
    if (!find_work<kStreamRows>(L, io, kStreamCut, lane, blockIdx.x, w)) return;
    const int first = w.tile * kStreamRows, rows = min(kStreamRows, w.rows - first), count = w.rows / L.G;
    // a row sees the tokens up to its own: query i of `count` lies at tokens - count + i
    auto limit = [&](int row) { return w.tokens - count + 1 + row / L.G; };
    u32x4 q[F::KS][kQueryPieces<T>];
    load_query<T, D>((const T*)io.q + row_at(L, io, w, first + col) * D, col < rows, a, q);
    const int lim = col < rows ? limit(first + col) : 0;
    Softmax<D> s;
    s.clear();
    s.m = kLowest;
    const int most = max(0, limit(first + rows - 1)), least = limit(first);
    const int nb = blocks_of(most), per = (nb + w.parts - 1) / w.parts;
    const int lo = min(nb, w.part * per), hi = min(nb, lo + per);
    const int32_t* table = L.table + (size_t)w.b * L.width;
    int win = -1;  // page of this wavefront's block number (turn & ~63) + lane
    // (The compiler waits for the window, and so for all blocks before, where it is used. A
    // wait where it is loaded instead changes nothing, but for few long sequences, which
    // then take more: three of 60001 tokens 36.7 us for 35.2, with four blocks ahead 40.4.)
    auto window = [&](int turn) {
        const int b = lo + wv + (turn + lane) * NW;
        win = b < hi ? table[b >> L.page_shift] : -1;
    };
    // This wavefront's blocks. The sequence's last one, if it is here, comes last, and
    // only it takes a new token or ends with places that hold none.
    const int turns = lo + wv < hi ? (hi - lo - wv + NW - 1) / NW : 0;
    Block<D, KB, VB> ring[NB];
    int page[NB];
    // the block, and its page, -1: none (then the block is any, unused)
    auto fetch = [&](int turn, auto i) {
        constexpr int I = decltype(i)::value;
        if ((turn & 63) == 0) window(turn);
        page[I] = __builtin_amdgcn_readlane(win, turn & 63);
        page[I] = page[I] >= 0 && page[I] < L.n_pages ? page[I] : -1;
        ring[I].template load<STREAM>(record<F>(L, max(page[I], 0), lo + wv + turn * NW, w.h), lane);
    };
    // A row's limit lies within 16 tokens of the end, that is in the last two blocks, which
    // different wavefronts take, each as its last.
    static_assert(kStreamRows <= kQuantBlock && NW >= 2, "");
    auto attend = [&](int b, Block<D, KB, VB>& blk, bool masked) {
        attend_block<T, D, KB, VB>(blk, q, masked, lim - b * kQuantBlock, a, io.scale_log2, s);
    };
    if (turns > 0) {
        fetch(0, Int<0>());
        if constexpr (NB > 2) fetch(1, Int<1>());
        if constexpr (NB > 3) fetch(2, Int<2>());
        // one turn at place I of the ring; false: it is the last one's, which is left there
        int turn = 0;
        auto pass = [&](auto i) {
            constexpr int I = decltype(i)::value, LAST = (I + NB - 1) % NB;
            if (turn + 1 >= turns) {
                if constexpr (I > 0) {
                    ring[0] = ring[I];
                    page[0] = page[I];
                }
                return false;
            }
            fetch(turn + NB - 1, Int<LAST>());
            if (page[I] >= 0) attend(lo + wv + turn * NW, ring[I], false);
            ++turn;
            return true;
        };
        for (;;) {
            if (!pass(Int<0>()) || !pass(Int<1>())) break;
            if constexpr (NB > 2)
                if (!pass(Int<2>())) break;
            if constexpr (NB > 3)
                if (!pass(Int<3>())) break;
        }
        if (page[0] >= 0) {
            Block<D, KB, VB>& blk = ring[0];
            const int b = lo + wv + turn * NW, t0 = b * kQuantBlock;
            if (w.fresh >= t0 && w.fresh < t0 + kQuantBlock)
                take_token<T, D, KB, VB>(io, blk, record<F>(L, page[0], b, w.h), w.fresh - t0, (size_t)w.b * L.nkv + w.h,
                                         lane);
            if (t0 + kQuantBlock > w.tokens) blk.zero_values_from(w.tokens - t0, a);
            const bool masked = t0 + kQuantBlock > least;
            if (masked && __ballot(any_nan(blk.ve)) != 0ull) hand_out_nan<D, KB, VB>(blk, lim - t0, a, s);
            attend(b, blk, masked);
        }
    }
    const float sum = sum_groups(s.l);
    if (a == 0) {
        s_m[wv][col] = s.m;
        s_l[wv][col] = sum;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int ct = 0; ct < F::VC; ct += 4)
            *reinterpret_cast<f32x4*>(&s_o[wv][col][(4 * a + r) * F::VC + ct]) =
                f32x4{s.o[ct][r], s.o[ct + 1][r], s.o[ct + 2][r], s.o[ct + 3][r]};
    __syncthreads();
    auto o = [&](int k, int row, int c) { return *reinterpret_cast<const f32x4*>(&s_o[k][row][c]); };
    if (w.parts == 1) {
        finish_rows<T, D, NW>(
            L, io, w, first, rows, tid, NW, s_w, [&](int k, int row) { return make_float2(s_m[k][row], s_l[k][row]); }, o);
        return;
    }
    const size_t slot = (size_t)(w.slot + w.part) * kStreamRows;
    for (int e = tid; e < rows * (D / 4); e += NW * 64) {
        const int row = e / (D / 4), c = e % (D / 4) * 4;
        float M = kLowest, z = 0.0f;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NW; ++k) M = fmaxf(M, s_m[k][row]);
#pragma unroll
        for (int k = 0; k < NW; ++k) {
            const float share = __builtin_amdgcn_exp2f(s_m[k][row] - M);
            x += o(k, row, c) * share;
            z = __builtin_fmaf(s_l[k][row], share, z);
        }
        publish4(io.part + (slot + row) * D + c, x);
        if (c == 0) {
            publish(io.ml + 2 * (slot + row), M);
            publish(io.ml + 2 * (slot + row) + 1, z);
        }
    }
    if (!arrive_last(io.arrived + (size_t)w.b * L.nkv + w.h, w.parts)) return;  // (a unit's rows are one tile)
    auto at = [&](int k, int row) { return (size_t)(w.slot + k) * kStreamRows + row; };
    finish_rows<T, D, NW>(
        L, io, w, first, rows, tid, w.parts, s_w,
        [&](int k, int row) {
            return make_float2(published(io.ml + 2 * at(k, row)), published(io.ml + 2 * at(k, row) + 1));
        },
        [&](int k, int row, int c) { return published4(io.part + at(k, row) * D + c); });
}

template <typename T, int D, int KB, int VB>
hipError_t launch(const QuantView& L, const QuantAttention& io, bool stream, hipStream_t s) {
    const size_t grid = most_workgroups(kStreamCut, kStreamRows, L.batch, io.queries, L.nkv, L.G);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kStreamWaves * 64), 0, s, L, io);
    };
    if (stream) go(k_quant_stream<T, D, KB, VB, true>);
    else go(k_quant_stream<T, D, KB, VB, false>);
    return hipGetLastError();
}

}  // namespace

QuantScratch quant_scratch(int batch, int queries, int nkv, int G) {
    // Every split tile has at least two parts of `chunk` blocks but for the last, and
    // all blocks together are at most target * chunk: at most 2 target slots.
    // (A unit's rows are one tile here.)
    const size_t units = (size_t)batch * nkv;
    const size_t rows = std::min((size_t)2 * kStreamCut.target, units * kMaxQuantParts) * kStreamRows;
    const size_t wide = queries * G > kStreamRows ? quant_wide_scratch_rows(batch, queries, nkv, G) : 0;
    return {std::max(rows, wide), units};
}

hipError_t launch_quant_attention(const QuantView& L, bool bf16, const QuantAttention& io, bool stream, hipStream_t s) {
    if (io.queries * L.G > kStreamRows) return launch_quant_wide(L, bf16, io, s);
    return with_types(L, bf16, [&](auto t, auto d, auto kb, auto vb) {
        return launch<decltype(t), d(), kb(), vb()>(L, io, stream, s);
    });
}

}  // namespace raas
