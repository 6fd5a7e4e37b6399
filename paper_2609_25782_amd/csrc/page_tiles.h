// One page's K and V tiles of one KV head in a wave's registers, and the product of its
// keys with a group's queries (gfx950, wave64): shared by the kernels that attend with one
// new token per session.
#pragma once

#include "device_common.h"
#include "kernels.h"

#include <math.h>

namespace hck {
namespace {

constexpr int kRsrcWord3 = 0x00020000;  // raw buffer, 32-bit data format (gfx9 family)

// Cache-policy bits of the K/V page loads: 2 = nontemporal (streaming).  Every
// K/V byte is read exactly once per call, so keeping it out of the caches'
// normal replacement leaves them to page ids, queries and partials.
#ifndef HCK_DECODE_LOAD_AUX
#define HCK_DECODE_LOAD_AUX 2
#endif

template <int D, bool BF16>
struct Shape {
    static constexpr int kElt = BF16 ? 2 : 4;
    static constexpr int kTile = kPageTokens * D * kElt;  // bytes of a K or V tile
    static constexpr int kKLoads = kTile / 1024;          // 16-byte K loads per lane
    static constexpr int kChunks = D / 16;                // 16-dim output chunks
};

template <bool BF16>
struct VSlice;
template <>
struct VSlice<true> {
    typedef u32x2 type;  // 4 bf16 tokens of one dim
};
template <>
struct VSlice<false> {
    typedef u32x4 type;  // 4 f32 tokens of one dim
};

template <int D, bool BF16>
struct PageRegs {
    u32x4 k[Shape<D, BF16>::kKLoads];
    typename VSlice<BF16>::type v[Shape<D, BF16>::kChunks];
};

__device__ __forceinline__ float wave_max_4(float x) {
    // max over lanes l, l^16, l^32, l^48 (the four token quarters of one head)
    x = fmaxf(x, __shfl_xor(x, 16));
    x = fmaxf(x, __shfl_xor(x, 32));
    return x;
}

__device__ __forceinline__ float wave_sum_4(float x) {
    x += __shfl_xor(x, 16);
    x += __shfl_xor(x, 32);
    return x;
}

// Where a piece's pages live, already offset to its layer and KV head: hot
// pages, and for tiered entries the cold pool and this layer's staging slots.
struct PageSrc {
    const char* hot = nullptr;
    const char* cold = nullptr;
    const char* stage = nullptr;
    int64_t hot_stride = 0, cold_stride = 0, slice_bytes = 0;
    unsigned num_hot = 0, num_cold = 0, num_stage = 0;
};

// A (page, KV head)'s two tiles.  Page ids are wave-uniform, so the tier choice
// is scalar.  An id outside its pool (or a negative entry) reads nothing: the
// buffer resource gets no records and the row is marked bad (NaN).
struct PageAddr {
    const char* base;
    bool ok;
};

template <bool TIERED>
__device__ __forceinline__ PageAddr page_addr(const PageSrc& ps, int pid, unsigned head_off) {
    const char* lh_base = ps.hot;
    int64_t stride = ps.hot_stride;
    unsigned n = ps.num_hot;
    unsigned id = static_cast<unsigned>(pid);
    if constexpr (TIERED) {
        const unsigned tag = id >> 29;  // 0 hot, 1 staged, 2 cold, otherwise invalid
        id &= static_cast<unsigned>(kPageIdMask);
        if (tag == 1) {
            lh_base = ps.stage;
            stride = ps.slice_bytes;
            n = ps.num_stage;
        } else if (tag == 2) {
            lh_base = ps.cold;
            stride = ps.cold_stride;
            n = ps.num_cold;
        } else if (tag != 0) {
            n = 0;
        }
    }
    const bool ok = id < n;
    return PageAddr{lh_base + static_cast<int64_t>(ok ? id : 0) * stride + head_off, ok};
}

template <int D, bool BF16>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t page_rsrc(const PageAddr& p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p.base), static_cast<short>(0),
                                             p.ok ? 2 * Shape<D, BF16>::kTile : 0, kRsrcWord3);
}

// Offsets past the instruction's 12 bits go into the scalar offset: one VGPR of
// offsets for all K loads and one for all V loads.
template <int D, bool BF16>
__device__ __forceinline__ void load_page_k(PageRegs<D, BF16>& r, __amdgpu_buffer_rsrc_t rs, unsigned koff) {
#pragma unroll
    for (int i = 0; i < Shape<D, BF16>::kKLoads; ++i)
        r.k[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, koff + 1024u * (i % 4), 4096 * (i / 4), HCK_DECODE_LOAD_AUX);
}

template <int D, bool BF16>
__device__ __forceinline__ void load_page_v(PageRegs<D, BF16>& r, __amdgpu_buffer_rsrc_t rs, unsigned voff) {
    using S = Shape<D, BF16>;
#pragma unroll
    for (int c = 0; c < S::kChunks; ++c) {
        if constexpr (BF16)
            r.v[c] = __builtin_amdgcn_raw_buffer_load_b64(rs, voff + 512u * c, S::kTile, HCK_DECODE_LOAD_AUX);
        else
            r.v[c] = __builtin_amdgcn_raw_buffer_load_b128(rs, voff + 1024u * (c % 4), S::kTile + 4096 * (c / 4),
                                                           HCK_DECODE_LOAD_AUX);
    }
}

// S^T tile of one page: lane l gets scores of head l % 16 for tokens 4 (l / 16) + r.
// Two accumulators halve the dependent MFMA chain; their sum is added once.
template <int D, bool BF16>
__device__ __forceinline__ f32x4 page_scores(const PageRegs<D, BF16>& r,
                                             const u32x4 (&q)[Shape<D, BF16>::kKLoads]) {
    using S = Shape<D, BF16>;
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < S::kKLoads; ++i) {
        f32x4& acc = (i & 1) ? s1 : s0;
        if constexpr (BF16) {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r.k[i]),
                                                          __builtin_bit_cast(bf16x8, q[i]), acc, 0,
                                                          0, 0);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(r.k[i][j]),
                                                           __uint_as_float(q[i][j]), acc, 0, 0, 0);
        }
    }
    return s0 + s1;
}

// Zero the V slice entries of tokens >= valid (this lane holds tokens 4 qg + j).
template <int D, bool BF16>
__device__ __forceinline__ void mask_v(PageRegs<D, BF16>& r, int valid, int qg) {
    using S = Shape<D, BF16>;
    const int t0 = 4 * qg;
    if constexpr (BF16) {
        const unsigned m0 = (t0 + 0 < valid ? 0x0000FFFFu : 0u) | (t0 + 1 < valid ? 0xFFFF0000u : 0u);
        const unsigned m1 = (t0 + 2 < valid ? 0x0000FFFFu : 0u) | (t0 + 3 < valid ? 0xFFFF0000u : 0u);
#pragma unroll
        for (int c = 0; c < S::kChunks; ++c) {
            r.v[c][0] &= m0;
            r.v[c][1] &= m1;
        }
    } else {
#pragma unroll
        for (int c = 0; c < S::kChunks; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (t0 + j >= valid) r.v[c][j] = 0u;
    }
}

// Partial result (m2, l2, o2) joined to the running one.
__device__ __forceinline__ void lse_merge(float& M, float& den, f32x4& acc, float m2, float l2,
                                          const f32x4& o2) {
    const float Mn = fmaxf(M, m2);
    const float c1 = (M == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(M - Mn);
    const float c2 = (m2 == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(m2 - Mn);
    acc = acc * c1 + o2 * c2;
    den = den * c1 + l2 * c2;
    M = Mn;
}

}  // namespace
}  // namespace hck
