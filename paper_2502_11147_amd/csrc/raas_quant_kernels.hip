// gfx950 kernels that quantise keys and values into the pages of the quantised
// cache as they are written, and read them back. A wavefront takes a block of 32
// tokens: its lanes hold the channels and tokens of the stored order
// (raas_quant_blocks.h), so a key's group is one lane's (two lanes' at head_dim 64)
// and a value's four or eight neighbours', and codes are stored 16 bytes per lane.
// Bound by memory: 4 D bytes of bf16 values per token and KV head against D (4 +
// 4 bits) / 8 + D / 16 of the cache.
#include "raas_quant_blocks.h"

namespace raas {
namespace {

using namespace qnt;

constexpr int kWaves = 4;

// The block of a wavefront: its number in the sequence, the call's rows of it.
struct Span {
    int blk, lo, hi;  // tokens lo .. hi - 1 of the block; row of token t: t + shift
    int shift, page;
    __device__ __forceinline__ bool find(const QuantView& L, const QuantCopy& io, int b, int nth) {
        const int start = io.start[b], count = min(io.count != nullptr ? io.count[b] : io.stride, io.stride);
        if (start < 0 || start >= L.cap || count <= 0) return false;
        const int end = min(start + count, L.cap);  // (both below 2^21)
        blk = start / kQuantBlock + nth;
        const int t0 = blk * kQuantBlock;
        lo = max(start - t0, 0);
        hi = min(end - t0, kQuantBlock);
        shift = t0 - start;
        if (lo >= hi) return false;
        page = L.table[(size_t)b * L.width + (blk >> L.page_shift)];
        return page >= 0 && page < L.n_pages;
    }
};

template <typename T, int D, int KB, int VB>
__global__ __launch_bounds__(kWaves * 64) void k_quant_write(QuantView L, QuantCopy io) {
    using F = Format<D, KB, VB>;
    const int lane = threadIdx.x & 63, a = lane >> 4, i = lane & 15, h = blockIdx.y, b = blockIdx.z;
    Span s;
    if (!s.find(L, io, b, blockIdx.x * kWaves + wave_of(threadIdx.x))) return;
    uint8_t* rec = record<F>(L, s.page, s.blk, h);
    const size_t row0 = ((size_t)b * L.nkv + h) * io.stride;
    auto in = [&](int t) { return t >= s.lo && t < s.hi; };
    // (tokens outside the span: the nearest one's row, whose codes are not stored)
    auto row = [&](const void* x, int t) {
        return (const T*)x + (row0 + (min(max(t, s.lo), s.hi - 1) + s.shift)) * D;
    };
    uint32_t kc[2][F::KD], ke[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) ke[q] = encode_key<T, D, KB>(row(io.k, 8 * (i >> 2) + 4 * q + (i & 3)), a, kc[q]);
    u32x2 vc[8];
    uint32_t ve[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) ve[j] = encode_value<T, D, VB>(row(io.v, 8 * a + j), i, vc[j]);
    const bool whole = s.lo == 0 && s.hi == kQuantBlock, exps = i % F::VSHARE == 0;
    uint8_t* kexp = rec + F::KEXP + (F::kgroup(a) * 16 + i) * 2;
    uint8_t* vexp = rec + F::VEXP + (a * F::NG + F::vgroup(i)) * 8;
    const bool kexps = F::KC >= kQuantGroup || (a & 1) == 0;
    if (whole) {
        Block<D, KB, VB> o;
#pragma unroll
        for (int p = 0; p < F::NKP; ++p)
#pragma unroll
            for (int e = 0; e < 4; ++e) o.k[p][e] = kc[(4 * p + e) / F::KD][(4 * p + e) % F::KD];
#pragma unroll
        for (int j = 0; j < 8; ++j) o.set_value(j, vc[j]);
#pragma unroll
        for (int p = 0; p < F::NKP; ++p) st16(rec + 1024 * p + 16 * lane, o.k[p]);
#pragma unroll
        for (int p = 0; p < F::NVP; ++p) st16(rec + F::VALUES + 1024 * p + 16 * lane, o.v[p]);
        if (kexps) *reinterpret_cast<uint16_t*>(kexp) = (uint16_t)(ke[0] | ke[1] << 8);
        if (exps)
            *reinterpret_cast<u32x2*>(vexp) = u32x2{ve[0] | ve[1] << 8 | ve[2] << 16 | ve[3] << 24,
                                                    ve[4] | ve[5] << 8 | ve[6] << 16 | ve[7] << 24};
        return;
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (!in(8 * (i >> 2) + 4 * q + (i & 3))) continue;
#pragma unroll
        for (int x = 0; x < F::KD; ++x) {
            const int at = q * F::KD + x;
            *reinterpret_cast<uint32_t*>(rec + 1024 * (at / 4) + 16 * lane + 4 * (at % 4)) = kc[q][x];
        }
        if (kexps) kexp[q] = (uint8_t)ke[q];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (!in(8 * a + j)) continue;
        store_value<D, KB, VB>(rec, lane, j, vc[j]);
        if (exps) vexp[j] = (uint8_t)ve[j];
    }
}

template <typename T, int D, int KB, int VB>
__global__ __launch_bounds__(kWaves * 64) void k_quant_read(QuantView L, QuantCopy io) {
    using F = Format<D, KB, VB>;
    const int lane = threadIdx.x & 63, a = lane >> 4, i = lane & 15, h = blockIdx.y, b = blockIdx.z;
    Span s;
    if (!s.find(L, io, b, blockIdx.x * kWaves + wave_of(threadIdx.x))) return;
    Block<D, KB, VB> o;
    o.template load<true>(record<F>(L, s.page, s.blk, h), lane);
    const size_t row0 = ((size_t)b * L.nkv + h) * io.stride;
    auto in = [&](int t) { return t >= s.lo && t < s.hi; };
    auto row = [&](void* x, int t) { return (T*)x + (row0 + (t + s.shift)) * D; };
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int t = 8 * (i >> 2) + 4 * q + (i & 3);
        if (!in(t)) continue;
        uint32_t x[F::KC / 2];
#pragma unroll
        for (int ks = 0; ks < F::KS; ++ks) {
            const u32x4 y = o.key(q, ks, o.key_scale(q));
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * ks + e] = y[e];
        }
        store_values<T, F::KC>(row(io.k, t) + a * F::KC, x);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (!in(8 * a + j)) continue;
        uint32_t x[F::VC / 2];
        o.value_row(j, x);
        store_values<T, F::VC>(row(io.v, 8 * a + j) + i * F::VC, x);
    }
}

hipError_t copy(const QuantView& L, bool bf16, const QuantCopy& io, bool write, hipStream_t s) {
    return with_types(L, bf16, [&](auto t, auto d, auto kb, auto vb) {
        using T = decltype(t);
        // (a span that starts inside a block touches one more)
        const int blocks = (io.stride + kQuantBlock - 1) / kQuantBlock + 1;
        const dim3 grid((blocks + kWaves - 1) / kWaves, L.nkv, L.batch);
        if (write) hipLaunchKernelGGL((k_quant_write<T, d(), kb(), vb()>), grid, dim3(kWaves * 64), 0, s, L, io);
        else hipLaunchKernelGGL((k_quant_read<T, d(), kb(), vb()>), grid, dim3(kWaves * 64), 0, s, L, io);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_quant_write(const QuantView& L, bool bf16, const QuantCopy& io, hipStream_t s) {
    return copy(L, bf16, io, true, s);
}

hipError_t launch_quant_read(const QuantView& L, bool bf16, const QuantCopy& io, hipStream_t s) {
    return copy(L, bf16, io, false, s);
}

}  // namespace raas
