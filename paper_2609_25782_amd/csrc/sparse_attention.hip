// Decode attention over the pages that a cheap score picks, for gfx950: bounds of each
// page's keys, the choice of pages by those bounds, and the attention over the chosen ones.
//
// Mathematics.  For a page, a KV head and a dim d let lo_d and hi_d be the smallest and the
// largest key value over the page's tokens.  Then for any query q and any token t of it
//     q . k_t = sum_d q_d k_td <= sum_d max(q_d, 0) hi_d + min(q_d, 0) lo_d =: u,
// so pages with a small u hold no token that matters to q.  lo and hi are kept as whole
// numbers of 8 bits times a power of two of the page and head (floor and ceil: the bounds
// stay bounds), q is rounded to whole numbers times a power of two of its own, and u becomes
// a product of 8-bit matrices: [min(q, 0) | max(q, 0)] . [lo | hi], exact in 32 bits (at most
// 128 * 127^2 < 2^21 in magnitude), and so is its product with the two powers of two in
// float32.  Which pages are picked therefore does not depend on the order of any sum.
//
// Records.  A page's record of one layer is [KV head][lo: D bytes, hi: D bytes], then 16
// bytes of which byte h is the power of head h (7 bits) and whether its bounds are newer than those
// of the page's cold copy (the top bit): 1/31 of the page's K and V in bfloat16.
//
// What bounds them (bf16, 32 query and 4 KV heads of 128 dims, a layer of 32 sessions of 8K-32K
// tokens on shuffled pages, unless said; the card reads 7.0 TB/s):
//   bounds     693 MB of keys in 143 us (4.85 TB/s).  Without its stores 100 us (6.6 TB/s): 44 MB
//              written as records of 1 KB all over the buffer cost as much as 200 MB read, with
//              pages in order a fifth less.  What did not help: nontemporal or write-through
//              stores, records of whole lines, sixteen results held and written together
//              (140 us).  One new token of 8 sessions in 48 layers 5.9 us, a chain of loads
//              (length, page id, keys).
//   read back  173 MB of float32 values in 36 us, 6.0 TB/s of reads and writes.
//   scores     44 MB of records in 12 us, of them 2.4 until the first records are asked for; 1.15
//              times the records' bytes are fetched (they are no whole lines).
//   choice     5.2 us, latencies: of its keys, and of two or three rounds of bins at three
//              barriers each.  Bit by bit (up to 32 rounds) it took 13.4.
//   attention  135 MB in 23 us and 4 us for the join; 64 sessions of 512 pages a head (1.08 GB) 161 us,
//              6.7 TB/s.  8 sessions of 2K tokens, 32 pages a head: 5.7 us and the join: of a
//              block's 5 us the length, the list and the page ids take 1.7, the first page 2.5.

#include "device_common.h"
#include "kernels.h"
#include "page_tiles.h"

#include <float.h>
#include <math.h>

#include <algorithm>
#include <cmath>

namespace hck {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// A value that all lanes share, in a scalar register: loads of it go through the vector path, and
// what depends on it would count as different from lane to lane.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

constexpr int kPowerLimit = 50;  // |e| at most: products of two powers and a sum stay normal numbers

// 2^e for |e| < 127.
__device__ __forceinline__ float two_to(int e) { return __uint_as_float(static_cast<unsigned>(e + 127) << 23); }

// The least e of [-50, 50] with top <= 127 * 2^e (-7 for 0; 50 for what no e suits).
__device__ __forceinline__ int power_for(float top) {
    int e = __builtin_amdgcn_frexp_expf(fminf(top, FLT_MAX)) - 7;
    e = e < -kPowerLimit ? -kPowerLimit : e > kPowerLimit ? kPowerLimit : e;
    if (top * two_to(-e) > 127.f && e < kPowerLimit) ++e;
    return e;
}

// The power in a record's byte: its low 7 bits, signed.
__device__ __forceinline__ int power_of(char byte) {
    const int e = (static_cast<int>(byte) << 25) >> 25;
    return e < -kPowerLimit ? -kPowerLimit : e > kPowerLimit ? kPowerLimit : e;
}

// A value that is no number counts as the infinity of its sign.
__device__ __forceinline__ float no_nan(float x) { return x != x ? copysignf(INFINITY, x) : x; }

__device__ __forceinline__ float clamp_127(float x) { return fminf(fmaxf(x, -127.f), 127.f); }

// The page that a table entry names: its number among the records (hot pages, then cold
// ones), or -1 where it names no page of either pool.
__device__ __forceinline__ int page_index(int entry, int num_hot, int num_cold) {
    const unsigned u = static_cast<unsigned>(entry);
    const unsigned id = u & static_cast<unsigned>(kPageIdMask), tag = u >> 29;
    if (tag == 0 && id < static_cast<unsigned>(num_hot)) return static_cast<int>(id);
    if (tag == 2 && id < static_cast<unsigned>(num_cold)) return num_hot + static_cast<int>(id);
    return -1;
}

template <int CTRL>
__device__ __forceinline__ int dpp(int x) {
    return __builtin_amdgcn_update_dpp(x, x, CTRL, 0xF, 0xF, false);
}
// Lane i's value from lane i ^ 1, i ^ 2, 7 - i of its 8 and 15 - i of its 16.
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppMirror8 = 0x141, kDppMirror16 = 0x140;

// Maximum of non-negative floats over the wave, in every lane.
__device__ __forceinline__ float wave_max(float x) {
    int v = __float_as_int(x);  // ordered like the floats
    v = max(v, dpp<kDppXor1>(v));
    v = max(v, dpp<kDppXor2>(v));
    v = max(v, dpp<kDppMirror8>(v));
    v = max(v, dpp<kDppMirror16>(v));
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x142, 0xA, 0xF, false));  // row_bcast:15 into rows 1 and 3
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x143, 0xC, 0xF, false));  // row_bcast:31 into rows 2 and 3
    return __int_as_float(__builtin_amdgcn_readlane(v, 63));
}

// How the waves of a block share (page, KV head) pairs: `heads` waves stand side by side on the
// heads of a page, which HBM serves faster than as many unrelated pages, `slices` such groups
// on different pages.
struct WaveSplit {
    int heads, slices;
};
__host__ __device__ __forceinline__ WaveSplit wave_split(int num_kv_heads) {
    const int h = num_kv_heads % 4 == 0 ? 4 : num_kv_heads % 2 == 0 ? 2 : 1;
    return WaveSplit{h, kBlockWaves / h};
}

// ---------------------------------------------------------------------------
// Bounds of pages.

// The lowest and the highest of sign-and-magnitude values from their bits, halves (bfloat16) or
// whole words: among values without a sign bit integers order them, among those with one backwards.
// So the highest is the greatest signed integer where that is not negative, else the least unsigned
// one; the lowest is the greatest unsigned integer where that has a sign bit, else the least.  Three
// instructions a word of keys.
template <bool BF16>
struct Extremes {
    typedef short s16x2_t __attribute__((ext_vector_type(2)));
    typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
    unsigned smax, umin, umax;
    __device__ __forceinline__ explicit Extremes(unsigned w) : smax(w), umin(w), umax(w) {}
    __device__ __forceinline__ void take(unsigned s, unsigned n, unsigned x) {
        if constexpr (BF16) {
            smax = __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(s16x2_t, smax),
                                                                          __builtin_bit_cast(s16x2_t, s)));
            umin = __builtin_bit_cast(unsigned, __builtin_elementwise_min(__builtin_bit_cast(u16x2_t, umin),
                                                                          __builtin_bit_cast(u16x2_t, n)));
            umax = __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, umax),
                                                                          __builtin_bit_cast(u16x2_t, x)));
        } else {
            smax = static_cast<unsigned>(max(static_cast<int>(smax), static_cast<int>(s)));
            umin = min(umin, n);
            umax = max(umax, x);
        }
    }
    __device__ __forceinline__ void take(unsigned w) { take(w, w, w); }
    // All ones in every half (word) of x with a sign bit.
    __device__ __forceinline__ static unsigned signs(unsigned x) {
        if constexpr (BF16)
            return __builtin_bit_cast(unsigned, static_cast<s16x2_t>(__builtin_bit_cast(s16x2_t, x) >> 15));
        else
            return static_cast<unsigned>(static_cast<int>(x) >> 31);
    }
    __device__ __forceinline__ unsigned highest() const {
        const unsigned m = signs(smax);
        return (smax & ~m) | (umin & m);
    }
    __device__ __forceinline__ unsigned lowest() const {
        const unsigned m = signs(umax);
        return (umax & m) | (umin & ~m);
    }
};

// Blocks of a bounds call, over rows and layers.  Few rows with few new pages each want few
// blocks that find nothing to do, many long rows want many: of one token of 8 sessions in 48 layers,
// turns of 64-1,024 tokens of 8 sessions, and all pages of 32 sessions (each with reading back)
// 2,048 blocks take 8.1, 9.7 and 180 us, 4,096 8.8, 8.6 and 178, 16,384 12.7, 11.4 and 172.
constexpr int64_t kBoundsBlocks = 4096;

// One wave takes a (page, KV head) at a time: the K tile is loaded in its own order, whole lines a
// load, and goes through LDS, from where lane l reads word l of every token (and word l + 64 where a
// token has 128; where it has 32 the lower lanes read tokens 0 .. 7 and the upper ones the rest).  A
// group of 16 tokens' 16 bytes takes 272 bytes there: neither side meets a bank twice.  Loaded
// straight into the lanes that reduce them, every line was fetched two to four times: 655 MB of
// keys 158 us, now 131, in float32 226, now 121.
template <int D, bool BF16>
__global__ __launch_bounds__(kBlockThreads) void bounds_update_kernel(const BoundsUpdateArgs a) {
    constexpr int kElt = BF16 ? 2 : 4;
    constexpr int kTile = kPageTokens * D * kElt;
    constexpr int kLoads = kTile / (16 * kWave);
    constexpr int kWords = D * kElt / 4;                        // 4-byte words of a token: 32, 64 or 128
    constexpr int kRows = kWords > kWave ? kWords / kWave : 1;  // that a lane reduces
    constexpr int kHalves = kWords < kWave ? kWave / kWords : 1;
    constexpr int kTokens = kPageTokens / kHalves;
    constexpr int kDims = 4 / kElt;                             // dims of a word
    constexpr int kPitch = 16 * kPageTokens + 16;
    const int b = blockIdx.y;
    const int layer = a.layer + static_cast<int>(blockIdx.z);
    const int len = uniform(a.lens[b]);
    if (len <= 0 || len > kPageTokens * a.pt_stride) return;
    int first = a.starts ? uniform(a.starts[b]) : 0;
    first = first < 0 ? 0 : first;
    if (first >= len) return;
    const int p0 = first / kPageTokens, p1 = (len - 1) / kPageTokens + 1;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = uniform(threadIdx.x / kWave);
    const WaveSplit ws = wave_split(a.num_kv_heads);
    const int32_t* row = a.table + static_cast<int64_t>(b) * a.pt_stride;
    const int step = ws.slices * static_cast<int>(gridDim.x);
    struct Unit {
        int at, head;   // the page among the records (-1: none), its KV head
        int last;       // its last token's slot, which stands in for those behind it
    };
    __shared__ __align__(16) char s_tile[kBlockWaves][kWords / 4 * kPitch];
    char* const mem = s_tile[wave];
    const int word = lane % kWords, half = kHalves > 1 ? lane / kWords : 0;
    const char* const mine = mem + word / 4 * kPitch + word % 4 * 4 + half * kTokens * 16;
    auto reduce = [&](const Unit& u, const u32x4 (&tile)[kLoads]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            *reinterpret_cast<u32x4*>(mem + (4 * i + lane / 16) * kPitch + lane % 16 * 16) = tile[i];
        __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        unsigned lo[kRows], hi[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            auto at = [&](int t) { return *reinterpret_cast<const unsigned*>(mine + r * 16 * kPitch + 16 * t); };
            unsigned w[kTokens];
            if (u.last == kPageTokens - 1) {
#pragma unroll
                for (int t = 0; t < kTokens; ++t) w[t] = at(t);
            } else {   // the last token once more in the place of those behind it
#pragma unroll
                for (int t = 0; t < kTokens; ++t) w[t] = at(min(half * kTokens + t, u.last) - half * kTokens);
            }
            Extremes<BF16> x(w[0]);
#pragma unroll
            for (int t = 1; t < kTokens; ++t) x.take(w[t]);
            if constexpr (kHalves == 2)
                x.take(static_cast<unsigned>(__shfl_xor(static_cast<int>(x.smax), 32)),
                       static_cast<unsigned>(__shfl_xor(static_cast<int>(x.umin), 32)),
                       static_cast<unsigned>(__shfl_xor(static_cast<int>(x.umax), 32)));
            lo[r] = x.lowest();
            hi[r] = x.highest();
        }
        __asm__ volatile("" ::: "memory");   // the next tile is written after these reads
        float l[kRows][kDims], h[kRows][kDims];
        float top = 0.f;
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int d = 0; d < kDims; ++d) {
                l[r][d] = no_nan(__uint_as_float(BF16 ? (d ? lo[r] & 0xFFFF0000u : lo[r] << 16) : lo[r]));
                h[r][d] = no_nan(__uint_as_float(BF16 ? (d ? hi[r] & 0xFFFF0000u : hi[r] << 16) : hi[r]));
                top = fmaxf(top, fmaxf(fabsf(l[r][d]), fabsf(h[r][d])));
            }
        const int e = power_for(wave_max(top));
        const float down = two_to(-e);
        // Loads and stores stand under no condition (a pair that is none has resources without
        // records): the compiler then knows how many of either are in flight and waits for the
        // next pair's loads alone.
        const __amdgpu_buffer_rsrc_t rec = __builtin_amdgcn_make_buffer_rsrc(
            a.bounds + layer * a.layer_stride + static_cast<int64_t>(u.at < 0 ? 0 : u.at) * a.record,
            static_cast<short>(0), u.at < 0 ? 0 : a.record, kRsrcWord3);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            unsigned ql = 0, qh = 0;
#pragma unroll
            for (int d = 0; d < kDims; ++d) {
                ql |= (static_cast<unsigned>(static_cast<int>(clamp_127(floorf(l[r][d] * down)))) & 0xFFu) << (8 * d);
                qh |= (static_cast<unsigned>(static_cast<int>(clamp_127(ceilf(h[r][d] * down)))) & 0xFFu) << (8 * d);
            }
            const int out = u.head * 2 * D + (r * kWave + word) * kDims;   // (both halves write the same)
            if constexpr (kDims == 2) {
                __builtin_amdgcn_raw_buffer_store_b16(static_cast<unsigned short>(ql), rec, out, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b16(static_cast<unsigned short>(qh), rec, out + D, 0, 0);
            } else {
                __builtin_amdgcn_raw_buffer_store_b8(static_cast<unsigned char>(ql), rec, out, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b8(static_cast<unsigned char>(qh), rec, out + D, 0, 0);
            }
        }
        __builtin_amdgcn_raw_buffer_store_b8(static_cast<unsigned char>((e & 0x7F) | 0x80), rec,
                                             a.num_kv_heads * 2 * D + u.head, 0, 0);
    };
    // A wave's pages are every step-th from its first on, 64 of them at a time: lane j holds the
    // j-th's place.  Its (page, head) pairs follow each other with the next one's keys in flight
    // while one's are reduced.
    for (int base = p0 + ws.slices * static_cast<int>(blockIdx.x) + wave / ws.heads; base < p1; base += kWave * step) {
        const int64_t place = base + static_cast<int64_t>(step) * lane;
        const int places = place < p1 ? page_index(row[place], a.num_hot, a.num_cold) : -1;
        const int pages = min((p1 - base - 1) / step + 1, kWave);
        int at_page = 0, at_head = wave % ws.heads;   // the pair fetched next
        auto fetch = [&](Unit& u, u32x4 (&w)[kLoads]) __attribute__((always_inline)) {
            u.at = at_page < pages ? __builtin_amdgcn_readlane(places, at_page) : -1;
            u.head = at_head;
            const int id = u.at < 0 ? 0 : u.at;
            const bool cold = id >= a.num_hot;
            const PoolGeom& pool = cold ? a.cold : a.hot;
            // every step issues one tile's loads, past the end from a resource without records
            const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                slice_at(pool, cold ? id - a.num_hot : id, layer) + u.head * 2 * kTile, static_cast<short>(0),
                u.at < 0 ? 0 : kTile, kRsrcWord3);
            u.last = u.at < 0 ? 0 : min(len - (base + at_page * step) * kPageTokens, kPageTokens) - 1;
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                w[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, 16 * lane + 1024 * (i % 4), 4096 * (i / 4), 2);
            at_head += ws.heads;
            if (at_head >= a.num_kv_heads) {
                at_head = wave % ws.heads;
                ++at_page;
            }
        };
        const int pairs = pages * ((a.num_kv_heads - 1) / ws.heads + 1);   // (heads come in whole groups)
        Unit u0, u1;
        u32x4 w0[kLoads], w1[kLoads];
        fetch(u0, w0);
        for (int k = 0; k < pairs; k += 2) {
            fetch(u1, w1);
            reduce(u0, w0);
            if (k + 1 >= pairs) break;
            fetch(u0, w0);
            reduce(u1, w1);
        }
    }
}

// Records as values: out [layers][n][KV heads][lo, hi][D] float32, NaN where an entry names no page.
__global__ __launch_bounds__(kBlockThreads) void bounds_read_kernel(const BoundsReadArgs a) {
    const int per = a.num_kv_heads * 2 * a.head_dim / 4;  // 4-byte words of a record's values
    const int side = per < kBlockThreads ? kBlockThreads / per : 1;   // pages of a block and turn
    const int layer = a.layer + static_cast<int>(blockIdx.y);
    const int slot = per < kBlockThreads ? static_cast<int>(threadIdx.x) / per : 0;
    const int first = static_cast<int>(threadIdx.x) - slot * per;
    if (slot >= side) return;
    f32x4* out = reinterpret_cast<f32x4*>(a.out) + static_cast<int64_t>(blockIdx.y) * a.n * per;
    for (int64_t p = static_cast<int64_t>(blockIdx.x) * side + slot; p < a.n;
         p += static_cast<int64_t>(gridDim.x) * side) {
        const int at = page_index(a.pages[p], a.num_hot, a.num_cold);
        const char* rec = a.bounds + layer * a.layer_stride + static_cast<int64_t>(at < 0 ? 0 : at) * a.record;
        for (int word = first; word < per; word += kBlockThreads) {
            const unsigned w = reinterpret_cast<const unsigned*>(rec)[word];
            const float unit = at < 0 ? __builtin_nanf("") : two_to(power_of(rec[4 * per + word * 2 / a.head_dim]));
            f32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = static_cast<float>(static_cast<signed char>(w >> (8 * j))) * unit;
            __builtin_nontemporal_store(v, out + p * per + word);
        }
    }
}

// Records that follow pages: entry e's from page e.src of one pool to page e.dst of the other.  With
// kRenewed a head's bounds and power are written only where they were set since the two records were
// alike: of sessions that share a cold page, one whose bounds are old does not undo another's.  An
// eviction of 8 sessions of 20,000 tokens in 48 layers whose pages all have valid cold copies takes 26 us
// of the GPU without bounds, 171 with none of them renewed, 334 with all (1 GB read and written).
template <typename Entries>
__device__ __forceinline__ void copy_records(const PoolGeom& src, const PoolGeom& dst, const Entries& entries, int32_t n,
                                             int heads, int head_words, RecordCopy how) {
    const int layer = static_cast<int>(blockIdx.y);
    const int words = heads * head_words + 1;
    const int64_t total = static_cast<int64_t>(n) * words;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBlockThreads + threadIdx.x; i < total;
         i += static_cast<int64_t>(gridDim.x) * kBlockThreads) {
        const int k = static_cast<int>(i / words);
        const int word = static_cast<int>(i - static_cast<int64_t>(k) * words);
        const CopyEntry e = entries[k];
        if (e.src < 0) continue;
        const char* from = slice_at(src, e.src, layer);
        char* to = slice_at(dst, e.dst, layer);
        const char* powers = from + 16 * (words - 1);
        if (how == RecordCopy::kRenewed) {
            if (word == words - 1) {
                for (int h = 0; h < heads; ++h)
                    if (powers[h] & 0x80) to[16 * word + h] = static_cast<char>(powers[h] & 0x7F);
                continue;
            }
            if (!(powers[word / head_words] & 0x80)) continue;
        }
        u32x4 w = reinterpret_cast<const u32x4*>(from)[word];
        if (word == words - 1 && how == RecordCopy::kTier) w &= 0x7F7F7F7Fu;   // the two are alike now
        reinterpret_cast<u32x4*>(to)[word] = w;
    }
}

__global__ __launch_bounds__(kBlockThreads) void bounds_copy_kernel(const PoolGeom src, const PoolGeom dst,
                                                                    const CopyEntry* __restrict__ entries, int32_t n,
                                                                    int heads, int head_words, RecordCopy how) {
    copy_records(src, dst, entries, n, heads, head_words, how);
}

// The same for a list in the kernel arguments.
struct RecordList {
    CopyEntry e[kCopyInline];
    __device__ const CopyEntry& operator[](int i) const { return e[i]; }
};
__global__ __launch_bounds__(kBlockThreads) void bounds_copy_inline_kernel(const PoolGeom src, const PoolGeom dst,
                                                                           int32_t n, int heads, int head_words,
                                                                           RecordCopy how, const RecordList list) {
    copy_records(src, dst, list, n, heads, head_words, how);
}

// ---------------------------------------------------------------------------
// Scores of pages.

// Tables of up to this many pages a row take scores and choice in one kernel, a block per list: one
// kernel fewer, but a list's records are read by one CU and without the other heads'.  4 rows
// of 57 pages 4.2 us, in two kernels 7.2; 1, 16, 64 and 256 rows of 512 pages 7.2, 9.0, 13.5 and 41,
// in two 9.5, 10.4, 14.3 and 45.  With two turns a wave, 16 and 64 rows of 1,024 pages 13.7 and
// 23.4 us, in two kernels 11.8 and 20.1.
constexpr int kShortThreads = 512;

constexpr unsigned kKeyBad = 0xFFFFFFFEu;  // above every score: a page that no pool holds

// Scores in an order that unsigned comparisons follow; none maps to 0.
__device__ __forceinline__ unsigned score_key(float s) {
    const unsigned u = __float_as_uint(s);
    return u ^ (u & 0x80000000u ? 0xFFFFFFFFu : 0x80000000u);
}

// One wave's queries of a KV head as the rows of the product: lane l holds head l % 16 of the
// group, 16 dims of every 64 from 16 (l / 16) on.
template <int D>
struct QueryRows {
    i32x4 neg[D / 64], pos[D / 64];
    float unit[4];   // 2^e of heads 4 (l / 16) + r, 0 past the group
};

// Their bits as they lie in memory.
template <int D, bool BF16>
struct QueryBits {
    static constexpr int kElt = BF16 ? 2 : 4;
    u32x4 w[D / 64][kElt];   // 16 dims are kElt words of 16 bytes
};

template <int D, bool BF16>
__device__ __forceinline__ void load_query_bits(QueryBits<D, BF16>& q, const SelectArgs& a, int b, int g, int lane) {
    constexpr int kElt = BF16 ? 2 : 4;
    const int h = lane & 15, part = lane >> 4;
    const char* src = static_cast<const char*>(a.q) + ((static_cast<int64_t>(b) * a.num_q_heads + g * a.group +
                                                        (h < a.group ? h : 0)) * D + 16 * part) * kElt;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int i = 0; i < kElt; ++i) q.w[c][i] = *reinterpret_cast<const u32x4*>(src + 64 * c * kElt + 16 * i);
}

template <int D, bool BF16>
__device__ __forceinline__ void round_queries(QueryRows<D>& q, const QueryBits<D, BF16>& bits, int group, int lane) {
    const int part = lane >> 4;
    const bool in = (lane & 15) < group;
    // unpacked twice, not held: their registers are the records' in the meantime
    auto value = [&](const QueryBits<D, BF16>& x, int c, int j) {
        if constexpr (BF16) {
            const unsigned w = x.w[c][j / 8][(j % 8) / 2];
            return no_nan(__uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16));
        } else {
            return no_nan(__uint_as_float(x.w[c][j / 4][j % 4]));
        }
    };
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) top = fmaxf(top, fabsf(value(bits, c, j)));
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const int e = power_for(top);
    const float down = two_to(-e);
    QueryBits<D, BF16> again = bits;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int i = 0; i < QueryBits<D, BF16>::kElt; ++i) __asm__("" : "+v"(again.w[c][i]));
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            unsigned n = 0, p = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int x = static_cast<int>(clamp_127(rintf(value(again, c, 4 * j + k) * down)));
                n |= (static_cast<unsigned>(min(x, 0)) & 0xFFu) << (8 * k);
                p |= (static_cast<unsigned>(max(x, 0)) & 0xFFu) << (8 * k);
            }
            q.neg[c][j] = static_cast<int>(n);
            q.pos[c][j] = static_cast<int>(p);
        }
    const float unit = in ? two_to(e) : 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) q.unit[r] = __shfl(unit, 4 * part + r);
}

// The keys of 64 pages' scores for KV head g: lane l's page has entry `at` among the records (-1: no
// page, whose key is above all scores).  `meanwhile` runs while the records come.
template <int D, typename F>
__device__ __forceinline__ unsigned score_pages(const QueryRows<D>& q, const char* bounds, const SelectArgs& a, int g,
                                                int at, int lane, F&& meanwhile) {
    const int part = lane >> 4, rec = at < 0 ? 0 : at;
    const char e = bounds[static_cast<int64_t>(rec) * a.record + a.num_kv_heads * 2 * D + g];
    u32x4 w[4][2 * D / 64];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const char* p = bounds + static_cast<int64_t>(__shfl(rec, 16 * t + (lane & 15))) * a.record + g * 2 * D + 16 * part;
#pragma unroll
        for (int c = 0; c < 2 * D / 64; ++c) w[t][c] = *reinterpret_cast<const u32x4*>(p + 64 * c);
    }
    meanwhile();
    float best = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        i32x4 s = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            s = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.neg[c], __builtin_bit_cast(i32x4, w[t][c]), s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.pos[c], __builtin_bit_cast(i32x4, w[t][c + D / 64]), s, 0, 0, 0);
        }
        float x = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (q.unit[r] != 0.f) x = fmaxf(x, static_cast<float>(s[r]) * q.unit[r]);
        x = fmaxf(x, __shfl_xor(x, 16));
        x = fmaxf(x, __shfl_xor(x, 32));
        best = part == t ? x : best;
    }
    return at < 0 ? kKeyBad : score_key(best * two_to(power_of(e)));
}

// Keys of all pages of the rows that have more pages than are picked.  A block takes chunks of 64
// pages of a row, its waves a KV head each where the heads come in twos or fours: the records of
// a page are then read side by side.
template <int D, bool BF16>
__global__ __launch_bounds__(kBlockThreads, BF16 ? 4 : 3) void page_scores_kernel(const SelectArgs a) {
    const int b = blockIdx.y;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = uniform(threadIdx.x / kWave);
    const WaveSplit ws = wave_split(a.num_kv_heads);
    const int step = kWave * ws.slices * static_cast<int>(gridDim.x);
    const int begin = kWave * (ws.slices * static_cast<int>(blockIdx.x) + wave / ws.heads);
    const int32_t* row = a.table + static_cast<int64_t>(b) * a.pt_stride;
    // the first page ids do not wait for the length
    int entry = begin + lane < a.pt_stride ? row[begin + lane] : -1;
    const int len = uniform(a.lens[b]);
    if (len <= 0 || len > kPageTokens * a.pt_stride) return;
    const int n = (len - 1) / kPageTokens + 1;
    if (n <= a.width || begin >= n) return;
    const char* bounds = a.bounds + a.layer * a.layer_stride;
    for (int g = wave % ws.heads; g < a.num_kv_heads; g += ws.heads) {
        QueryBits<D, BF16> bits;
        load_query_bits<D, BF16>(bits, a, b, g, lane);
        QueryRows<D> q;
        unsigned* keys = a.keys + (static_cast<int64_t>(b) * a.num_kv_heads + g) * a.pt_stride;
        for (int p0 = begin; p0 < n; p0 += step) {
            if (p0 != begin || g != wave % ws.heads) entry = p0 + lane < n ? row[p0 + lane] : -1;
            const int at = p0 + lane < n ? page_index(entry, a.num_hot, a.num_cold) : -1;
            const unsigned key = score_pages<D>(q, bounds, a, g, at, lane, [&] {
                if (p0 == begin) round_queries<D, BF16>(q, bits, a.group, lane);
            });
            if (p0 + lane < n) keys[p0 + lane] = key;
        }
    }
}

// ---------------------------------------------------------------------------
// The choice.

__device__ __forceinline__ unsigned wave_max_u32(unsigned x) {
    x = max(x, static_cast<unsigned>(dpp<kDppXor1>(static_cast<int>(x))));
    x = max(x, static_cast<unsigned>(dpp<kDppXor2>(static_cast<int>(x))));
    x = max(x, static_cast<unsigned>(dpp<kDppMirror8>(static_cast<int>(x))));
    x = max(x, static_cast<unsigned>(dpp<kDppMirror16>(static_cast<int>(x))));
    x = max(x, static_cast<unsigned>(__builtin_amdgcn_update_dpp(x, x, 0x142, 0xA, 0xF, false)));
    x = max(x, static_cast<unsigned>(__builtin_amdgcn_update_dpp(x, x, 0x143, 0xC, 0xF, false)));
    return static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(x), 63));
}

// Row b's picks for KV head g of its n > width pages: the first `first`, the last `recent` and the best
// of those between.  The keys' range is cut into bins, the bin that the last place falls into into
// finer ones, and so on until a bin is wanted whole or is one value, whose places go to the lowest
// pages.  Bins stand in descending order of their keys.
template <int THREADS, int KEYS>
__device__ __forceinline__ void pick_pages(const SelectArgs& a, int b, int g, int n, const unsigned* keys) {
    constexpr int kWaves = THREADS / kWave;
    constexpr int kBinBits = THREADS == 1024 ? 12 : 11;
    constexpr int kBins = 1 << kBinBits;
    static_assert(kBins == 4 * THREADS, "four bins a thread");
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int64_t seg = static_cast<int64_t>(b) * a.num_kv_heads + g;
    int32_t* picks = a.picks + seg * a.width;
    __shared__ __align__(16) int s_bins[kBins];
    __shared__ unsigned s_least[kWaves], s_most[kWaves];
    __shared__ int s_sum[kWaves], s_bin, s_above, s_in;
    const int lo = a.first, hi = n - a.recent;
    const int want = a.width - a.first - a.recent;   // at least 0, less than hi - lo
    // keys that are no candidates count as 0, which no candidate's is
    auto key = [&](int i) { return i >= lo && i < hi ? keys[i] : 0u; };
    unsigned held[KEYS > 0 ? KEYS : 1];
    if constexpr (KEYS > 0) {
#pragma unroll
        for (int j = 0; j < KEYS; ++j) held[j] = key(j * THREADS + tid);
    }
    auto each = [&](auto&& f) __attribute__((always_inline)) {
        if constexpr (KEYS > 0) {
#pragma unroll
            for (int j = 0; j < KEYS; ++j)
                if (j * THREADS < n) f(held[j]);
        } else {
            for (int i0 = 0; i0 < n; i0 += THREADS) f(key(i0 + tid));
        }
    };
    reinterpret_cast<i32x4*>(s_bins)[tid] = i32x4{0, 0, 0, 0};
    unsigned cut = 0xFFFFFFFFu;    // keys from here on are picked,
    unsigned tie = 0;              // and of those equal to this one
    int spare = 0;                 // as many
    if (want > 0) {
        unsigned least = 0xFFFFFFFFu, most = 0;
        each([&](unsigned k) {
            least = k != 0 && k < least ? k : least;
            most = k > most ? k : most;
        });
        least = ~wave_max_u32(~least);
        most = wave_max_u32(most);
        if (lane == 0) {
            s_least[wave] = least;
            s_most[wave] = most;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            least = min(least, s_least[w]);
            most = max(most, s_most[w]);
        }
        int left = want;   // places for keys of [least, most]
        while (true) {
            const int bits = 32 - __clz(static_cast<int>((most - least) | 1u));
            const int shift = bits > kBinBits ? bits - kBinBits : 0;
            each([&](unsigned k) {
                if (k >= least && k <= most) atomicAdd(&s_bins[(most - k) >> shift], 1);
            });
            __syncthreads();
            const i32x4 mine = reinterpret_cast<const i32x4*>(s_bins)[tid];
            reinterpret_cast<i32x4*>(s_bins)[tid] = i32x4{0, 0, 0, 0};
            const int sum = mine[0] + mine[1] + mine[2] + mine[3];
            const int upto = wave_scan(sum);
            if (lane == kWave - 1) s_sum[wave] = upto;
            __syncthreads();
            int above = upto - sum;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) above += w < wave ? s_sum[w] : 0;
            if (above < left && left <= above + sum) {   // one thread
                int j = 0;
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (j == i && above + mine[i] < left) {
                        above += mine[i];
                        ++j;
                    }
                s_bin = 4 * tid + j;
                s_above = above;
                s_in = j == 0 ? mine[0] : j == 1 ? mine[1] : j == 2 ? mine[2] : mine[3];
            }
            __syncthreads();
            left -= s_above;
            most -= static_cast<unsigned>(s_bin) << shift;
            const unsigned width = (1u << shift) - 1;
            least = most - least > width ? most - width : least;
            if (s_in == left) {
                cut = least;
                break;
            }
            if (shift == 0) {
                cut = least + 1;
                tie = least;
                spare = left;
                break;
            }
        }
    }
    // In order of the pages: those kept anyway, the keys from the cut on, and the first of the ties.
    auto kinds = [&](int i, unsigned k, bool& more, bool& tied) {
        more = i < n && (i < lo || i >= hi || k >= cut);
        tied = k == tie && k != 0;
    };
    auto put = [&](int i, bool more, bool tied, uint64_t bm, uint64_t bt, int before) {
        const uint64_t below = (1ull << lane) - 1;   // `before`: picks in the low half, ties in the high one
        const int m = (before & 0xFFFF) + __builtin_popcountll(bm & below);
        const int t = (before >> 16) + __builtin_popcountll(bt & below);
        if (more || (tied && t < spare)) picks[m + (t < spare ? t : spare)] = i;
    };
    if constexpr (KEYS > 0) {
        // counts of all (turn, wave) groups of 64 pages, at most 2^14 of each kind
        constexpr int kGroups = KEYS * kWaves;
        __shared__ int s_kinds[kGroups];
        uint64_t bm[KEYS], bt[KEYS];
#pragma unroll
        for (int j = 0; j < KEYS; ++j) {
            bool more, tied;
            kinds(j * THREADS + tid, held[j], more, tied);
            bm[j] = __builtin_amdgcn_ballot_w64(more);
            bt[j] = __builtin_amdgcn_ballot_w64(tied);
            if (lane == 0)
                s_kinds[j * kWaves + wave] = __builtin_popcountll(bm[j]) | __builtin_popcountll(bt[j]) << 16;
        }
        __syncthreads();
        int carry = 0;
        int before[(kGroups + kWave - 1) / kWave];
#pragma unroll
        for (int c = 0; c < kGroups; c += kWave) {
            const int x = c + lane < kGroups ? s_kinds[c + lane] : 0;
            const int upto = wave_scan(x);
            before[c / kWave] = carry + upto - x;
            carry += __builtin_amdgcn_readlane(upto, kWave - 1);
        }
#pragma unroll
        for (int j = 0; j < KEYS; ++j) {
            const int at = j * kWaves + wave;
            const int base = __builtin_amdgcn_readlane(before[j * kWaves / kWave],
                                                       __builtin_amdgcn_readfirstlane(at) % kWave);
            put(j * THREADS + tid, (bm[j] >> lane) & 1, (bt[j] >> lane) & 1, bm[j], bt[j], base);
        }
    } else {
        __shared__ int s_more[kWaves], s_tie[kWaves];
        int base = 0, ties = 0;
        for (int i0 = 0; i0 < n; i0 += THREADS) {
            const int i = i0 + tid;
            bool more, tied;
            kinds(i, key(i), more, tied);
            const uint64_t bm = __builtin_amdgcn_ballot_w64(more), bt = __builtin_amdgcn_ballot_w64(tied);
            if (lane == 0) {
                s_more[wave] = __builtin_popcountll(bm);
                s_tie[wave] = __builtin_popcountll(bt);
            }
            __syncthreads();
            int m = base, t = ties;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                m += w < wave ? s_more[w] : 0;
                t += w < wave ? s_tie[w] : 0;
                base += s_more[w];
                ties += s_tie[w];
            }
            const uint64_t below = (1ull << lane) - 1;
            m += __builtin_popcountll(bm & below);
            t += __builtin_popcountll(bt & below);
            if (more || (tied && t < spare)) picks[m + (t < spare ? t : spare)] = i;
            __syncthreads();
        }
    }
    if (tid == 0) a.counts[seg] = a.width;
}

// Pages of the row, and whether that is more than are picked; else all of them are written here.
template <int THREADS>
__device__ __forceinline__ int row_to_pick(const SelectArgs& a, int b, int g, bool& choose) {
    const int len = uniform(a.lens[b]);
    const int n = len <= 0 || len > kPageTokens * a.pt_stride ? 0 : (len - 1) / kPageTokens + 1;
    choose = n > a.width;
    if (!choose) {
        const int64_t seg = static_cast<int64_t>(b) * a.num_kv_heads + g;
        for (int i = threadIdx.x; i < a.width; i += THREADS) a.picks[seg * a.width + i] = i < n ? i : -1;
        if (threadIdx.x == 0) a.counts[seg] = n;
    }
    return n;
}

// Block (g, b): the choice by the keys that page_scores_kernel wrote.
template <int THREADS, int KEYS>
__global__ __launch_bounds__(THREADS) void page_pick_kernel(const SelectArgs a) {
    const int g = blockIdx.x, b = blockIdx.y;
    bool choose;
    const int n = row_to_pick<THREADS>(a, b, g, choose);
    if (choose)
        pick_pages<THREADS, KEYS>(a, b, g, n, a.keys + (static_cast<int64_t>(b) * a.num_kv_heads + g) * a.pt_stride);
}

// Block (g, b): scores and choice in one, the keys in LDS, for rows of few pages.
template <int D, bool BF16>
__global__ __launch_bounds__(kShortThreads) void page_select_kernel(const SelectArgs a) {
    const int g = blockIdx.x, b = blockIdx.y;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = uniform(threadIdx.x / kWave);
    const int32_t* row = a.table + static_cast<int64_t>(b) * a.pt_stride;
    const int page = wave * kWave + lane;
    const int entry = page < a.pt_stride ? row[page] : -1;   // does not wait for the length
    QueryBits<D, BF16> bits;
    load_query_bits<D, BF16>(bits, a, b, g, lane);
    bool choose;
    const int n = row_to_pick<kShortThreads>(a, b, g, choose);
    if (!choose) return;
    __shared__ unsigned s_keys[kShortThreads];
    QueryRows<D> q;
    round_queries<D, BF16>(q, bits, a.group, lane);
    if (wave * kWave < n) {
        const int at = page < n ? page_index(entry, a.num_hot, a.num_cold) : -1;
        s_keys[page] = score_pages<D>(q, a.bounds + a.layer * a.layer_stride, a, g, at, lane, [] {});
    }
    __syncthreads();
    pick_pages<kShortThreads, 1>(a, b, g, n, s_keys);
}

// ---------------------------------------------------------------------------
// Attention over picked pages.

template <int D, bool BF16>
struct SparseState {
    u32x4 q[Shape<D, BF16>::kKLoads];
    f32x4 o[Shape<D, BF16>::kChunks];
    float m;       // running maximum, -inf before the first page
    float shift;   // what the exponents are taken against: m, or 0 while that is -inf
    float l;
};

// One page with `valid` tokens (1..16): online softmax and weighted V.
template <int D, bool BF16>
__device__ __forceinline__ void sparse_page(SparseState<D, BF16>& st, PageRegs<D, BF16>& pg, int valid,
                                            float scale_log2, int qg) {
    using S = Shape<D, BF16>;
    f32x4 s = page_scores<D, BF16>(pg, st.q);
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] *= scale_log2;
    if (valid < kPageTokens) {
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] = 4 * qg + r < valid ? s[r] : -INFINITY;
        mask_v<D, BF16>(pg, valid, qg);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[r]);
    // The maximum is the same on the four lanes of a head; it is reduced over them, and the
    // sums rescaled, only where some lane sees a score above it.
    if (__builtin_amdgcn_ballot_w64(mx > st.m)) {
        const float m_new = fmaxf(st.m, wave_max_4(mx));
        const float shift = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(st.m - shift);
        st.l *= alpha;
#pragma unroll
        for (int c = 0; c < S::kChunks; ++c) st.o[c] *= alpha;
        st.m = m_new;
        st.shift = shift;
    }
    float p[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(s[r] - st.shift);
    if constexpr (BF16) {
        // Weights rounded to bf16, which the product with V takes (as the decode over all pages does), and
        // the same rounded ones in the sum: a common error of theirs cancels.  Outputs are then off by
        // 0.0018-0.0020 of the values' size against 64 bits, with weights of 32 bits by 0.0016-0.0017:
        // rounding the output is most of either.
        __bf16 pb[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            pb[r] = static_cast<__bf16>(p[r]);
            st.l += static_cast<float>(pb[r]);
        }
        const s16x4 pv = {__builtin_bit_cast(short, pb[0]), __builtin_bit_cast(short, pb[1]),
                          __builtin_bit_cast(short, pb[2]), __builtin_bit_cast(short, pb[3])};
#pragma unroll
        for (int c = 0; c < S::kChunks; ++c)
            st.o[c] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, pg.v[c]), pv, st.o[c], 0, 0, 0);
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) st.l += p[r];
#pragma unroll
        for (int c = 0; c < S::kChunks; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                st.o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(pg.v[c][j]), p[j], st.o[c], 0, 0, 0);
    }
}

// Where a list has tokens but every score was minus infinity its maximum counts as this, so that
// it ends in 0 / 0; a list without tokens keeps minus infinity and ends in zeros.
constexpr float kNoScore = -FLT_MAX;

// Floats of a head's row where a block's waves meet in LDS: rows start in different banks.
template <int D>
constexpr int kJoinPitch = D + 4;

template <int D, bool BF16>
__device__ __forceinline__ void store_result(const SparseArgs& a, int64_t head_row, int quad, float M, float den,
                                             const f32x4& acc, bool invalid) {
    f32x4 v;
    const float nan = __builtin_nanf("");
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = invalid ? nan : M == -INFINITY && !(den != den) ? 0.f : acc[j] / den;
    const int64_t at = head_row * D + 4 * quad;
    if constexpr (BF16) {
        __bf16 w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = static_cast<__bf16>(v[j]);
        *reinterpret_cast<u32x2*>(static_cast<__bf16*>(a.out) + at) = __builtin_bit_cast(u32x2, w);
    } else {
        *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = v;
    }
}

// Block (s, g, b): part s of row b's list for KV head g, shared by the block's waves and joined
// in LDS.  With one part the block writes the output, else a partial result.  A wave holds two
// pages, the one computed and the next: 8 sessions of 32 and 32 of 128 pages a head 8.3 and 27.1
// us a call, with three 8.9 and 28.2, four 9.7 and 28.0; eight waves a block and fewer parts 9.5
// and 27.6, sixteen with one page each 10.2 and 28.8.
template <int D, bool BF16>
__global__ __launch_bounds__(kBlockThreads, BF16 ? 3 : 2) void sparse_split_kernel(const SparseArgs a) {
    using S = Shape<D, BF16>;
    constexpr int R = 2;   // pages held: the one computed and the next
    const int part = blockIdx.x, g = blockIdx.y, b = blockIdx.z;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = uniform(threadIdx.x / kWave);
    const int qg = lane >> 4;
    const int64_t seg = static_cast<int64_t>(b) * a.num_kv_heads + g;
    const int len = uniform(a.lens[b]);
    const bool invalid = len < 0 || len > kPageTokens * a.pt_stride;
    const int n = invalid || len == 0 ? 0 : (len - 1) / kPageTokens + 1;
    int count = a.counts ? uniform(a.counts[seg]) : a.width;
    count = count < 0 || n == 0 ? 0 : count > a.width ? a.width : count;
    // This wave takes entries k, k + stride, ..: which they are does not wait for the count, and
    // the waves of a block read neighbours at a time.
    const int stride = a.parts * kBlockWaves, k = part * kBlockWaves + wave;
    const int entries = count > k ? (count - k - 1) / stride + 1 : 0;
    const int32_t* list = a.picks + seg * a.width;
    const int64_t e_first = k + static_cast<int64_t>(stride) * lane;
    const int p_first = e_first < a.width ? list[e_first] : -1;
    const int32_t* row = a.table + static_cast<int64_t>(b) * a.pt_stride;
    const char* const hot = a.hot + g * 2 * S::kTile;
    const char* const cold = a.cold + g * 2 * S::kTile;
    const int64_t hot_stride = a.hot_stride, cold_stride = a.cold_stride;
    const int num_hot = a.num_hot;
    const unsigned koff = 16u * lane;
    const unsigned voff = BF16 ? (32u * (lane & 15) + 8u * qg) : (64u * (lane & 15) + 16u * qg);

    SparseState<D, BF16> st;
    {
        const __amdgpu_buffer_rsrc_t qr = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<char*>(static_cast<const char*>(a.q) + seg * a.group * (D * S::kElt)), static_cast<short>(0),
            a.group * D * S::kElt, kRsrcWord3);   // head slots past the group read zeros
        const unsigned off = static_cast<unsigned>((lane & 15) * D * S::kElt + 16 * (lane >> 4));
#pragma unroll
        for (int i = 0; i < S::kKLoads; ++i) st.q[i] = __builtin_amdgcn_raw_buffer_load_b128(qr, off + 64u * i, 0, 0);
    }
#pragma unroll
    for (int c = 0; c < S::kChunks; ++c) st.o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    st.m = -INFINITY;
    st.shift = 0.f;
    st.l = 0.f;
    bool bad = false, seen = false;

    for (int base = 0; base < entries; base += kWave) {
        const int cnt = entries - base < kWave ? entries - base : kWave;
        // lane j: the wave's entry base + j, its page and how many tokens of it count (0: not of
        // this row)
        const int p = base == 0 ? p_first : lane < cnt ? list[k + static_cast<int64_t>(stride) * (base + lane)] : -1;
        const bool in = lane < cnt && p >= 0 && p < n;
        const int entry = in ? row[p] : -1;
        const int at = page_index(entry, a.num_hot, a.num_cold);
        const int left = len - p * kPageTokens;
        const int valid = !in ? 0 : left < kPageTokens ? left : kPageTokens;
        if (__builtin_amdgcn_ballot_w64(in && at < 0)) bad = true;
        if (__builtin_amdgcn_ballot_w64(in)) seen = true;
        PageRegs<D, BF16> ring[R];
        auto issue = [&](int r, int j) __attribute__((always_inline)) {
            // every step issues one page's loads, past the end from a resource without records
            const int page = j < cnt ? __builtin_amdgcn_readlane(at, j) : -1;
            const int tokens = j < cnt ? __builtin_amdgcn_readlane(valid, j) : 0;
            PageAddr pa;
            pa.ok = page >= 0 && tokens > 0;
            const int id = pa.ok ? page : 0;
            const char* base = hot;
            int64_t slot = id, pitch = hot_stride;
            if (id >= num_hot) {
                base = cold;
                slot = id - num_hot;
                pitch = cold_stride;
            }
            pa.base = base + slot * pitch;
            const __amdgpu_buffer_rsrc_t rs = page_rsrc<D, BF16>(pa);
            load_page_k<D, BF16>(ring[r], rs, koff);
            load_page_v<D, BF16>(ring[r], rs, voff);
        };
        auto compute = [&](int r, int j) __attribute__((always_inline)) {
            if (j < 0 || j >= cnt) return;
            const int tokens = __builtin_amdgcn_readlane(valid, j);
            if (tokens <= 0) return;
            sparse_page<D, BF16>(st, ring[r], tokens, a.scale_log2, qg);
        };
#pragma unroll
        for (int r = 0; r < R - 1; ++r) issue(r, r);
        for (int j = 0; j < cnt; j += R) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                issue((r + R - 1) % R, j + r + R - 1);
                compute(r, j + r);
            }
        }
    }

    float l = wave_sum_4(st.l);
    if (bad) l = __builtin_nanf("");
    float m = st.m == -INFINITY && seen ? kNoScore : st.m;

    // the waves' results meet in LDS: [wave][head][kJoinPitch], then [wave][max, sum][head]
    extern __shared__ __align__(16) char s_mem[];
    float* s_o = reinterpret_cast<float*>(s_mem);
    float* s_ml = s_o + kBlockWaves * a.group * kJoinPitch<D>;
    const int h = lane & 15;
    if (h < a.group) {
        float* o = s_o + (wave * a.group + h) * kJoinPitch<D> + 4 * qg;
#pragma unroll
        for (int c = 0; c < S::kChunks; ++c) *reinterpret_cast<f32x4*>(o + 16 * c) = st.o[c];
        if (qg == 0) {
            s_ml[wave * 2 * a.group + h] = m;
            s_ml[wave * 2 * a.group + a.group + h] = l;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.group * (D / 4); i += kBlockThreads) {
        const int hh = i / (D / 4), quad = i % (D / 4);
        float M = -INFINITY, den = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kBlockWaves; ++w)
            lse_merge(M, den, acc, s_ml[w * 2 * a.group + hh], s_ml[w * 2 * a.group + a.group + hh],
                      *reinterpret_cast<const f32x4*>(s_o + (w * a.group + hh) * kJoinPitch<D> + 4 * quad));
        if (a.parts == 1) {
            store_result<D, BF16>(a, seg * a.group + hh, quad, M, den, acc, invalid);
        } else {
            const int64_t slot = seg * a.parts + part;
            *reinterpret_cast<f32x4*>(a.part_o + (slot * a.group + hh) * D + 4 * quad) = acc;
            if (quad == 0) {
                a.part_ml[slot * 2 * a.group + hh] = M;
                a.part_ml[slot * 2 * a.group + a.group + hh] = den;
            }
        }
    }
}

// The parts of a list joined: a lane takes one (head, 4 dims), the block's waves every
// kBlockWaves-th part each.
template <int D, bool BF16>
__global__ __launch_bounds__(kBlockThreads) void sparse_merge_kernel(const SparseArgs a) {
    const int g = blockIdx.y, b = blockIdx.z;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = uniform(threadIdx.x / kWave);
    const int items = a.group * (D / 4);
    const int i = blockIdx.x * kWave + lane < items ? blockIdx.x * kWave + lane : items - 1;
    const int h = i / (D / 4), quad = i % (D / 4);
    const int64_t seg = static_cast<int64_t>(b) * a.num_kv_heads + g;
    const int len = uniform(a.lens[b]);
    const bool invalid = len < 0 || len > kPageTokens * a.pt_stride;
    float M = -INFINITY, den = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    constexpr int U = 4;   // parts in flight; past the end the last one again, unused
    for (int p0 = wave; p0 < a.parts; p0 += U * kBlockWaves) {
        float m[U], l[U];
        f32x4 o[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = p0 + u * kBlockWaves < a.parts ? p0 + u * kBlockWaves : a.parts - 1;
            const int64_t slot = seg * a.parts + p;
            m[u] = a.part_ml[slot * 2 * a.group + h];
            l[u] = a.part_ml[slot * 2 * a.group + a.group + h];
            o[u] = *reinterpret_cast<const f32x4*>(a.part_o + (slot * a.group + h) * D + 4 * quad);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p0 + u * kBlockWaves < a.parts) lse_merge(M, den, acc, m[u], l[u], o[u]);
    }
    __shared__ float s_m[kBlockWaves][kWave], s_l[kBlockWaves][kWave];
    __shared__ f32x4 s_o[kBlockWaves][kWave];
    s_m[wave][lane] = M;
    s_l[wave][lane] = den;
    s_o[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < kBlockWaves; ++w) lse_merge(M, den, acc, s_m[w][lane], s_l[w][lane], s_o[w][lane]);
    if (blockIdx.x * kWave + lane < items) store_result<D, BF16>(a, seg * a.group + h, quad, M, den, acc, invalid);
}

template <int D, bool BF16>
hipError_t launch_sparse_for(const SparseArgs& a, hipStream_t s, const LaunchEvents& ev, const LaunchEvents& ev_merge) {
    const size_t lds = static_cast<size_t>(kBlockWaves) * a.group * (kJoinPitch<D> + 2) * sizeof(float);
    void* args[] = {const_cast<SparseArgs*>(&a)};
    const dim3 grid(static_cast<unsigned>(a.parts), static_cast<unsigned>(a.num_kv_heads), static_cast<unsigned>(a.batch));
    hipError_t e = launch_kernel(reinterpret_cast<const void*>(&sparse_split_kernel<D, BF16>), grid, dim3(kBlockThreads),
                                 args, lds, s, ev);
    if (e != hipSuccess || a.parts == 1) return e;
    const unsigned blocks = static_cast<unsigned>((a.group * (D / 4) + kWave - 1) / kWave);
    return launch_kernel(reinterpret_cast<const void*>(&sparse_merge_kernel<D, BF16>),
                         dim3(blocks, static_cast<unsigned>(a.num_kv_heads), static_cast<unsigned>(a.batch)),
                         dim3(kBlockThreads), args, 0, s, ev_merge);
}

}  // namespace

hipError_t launch_bounds_update(const BoundsUpdateArgs& a, int head_dim, int dtype, int32_t num_layers, hipStream_t s,
                                const LaunchEvents& ev) {
    // enough blocks for the GPU however few rows there are, no more than the longest row has units
    const int slices = wave_split(a.num_kv_heads).slices;
    const int64_t rows = static_cast<int64_t>(a.batch) * num_layers;
    int64_t gx = (kBoundsBlocks + rows - 1) / rows;
    gx = std::min<int64_t>(gx, (a.pt_stride + slices - 1) / slices);
    const dim3 grid(static_cast<unsigned>(gx), static_cast<unsigned>(a.batch), static_cast<unsigned>(num_layers));
    const void* k = dtype == kDtypeBf16
                        ? (head_dim == 128 ? reinterpret_cast<const void*>(&bounds_update_kernel<128, true>)
                                           : reinterpret_cast<const void*>(&bounds_update_kernel<64, true>))
                        : (head_dim == 128 ? reinterpret_cast<const void*>(&bounds_update_kernel<128, false>)
                                           : reinterpret_cast<const void*>(&bounds_update_kernel<64, false>));
    void* args[] = {const_cast<BoundsUpdateArgs*>(&a)};
    return launch_kernel(k, grid, dim3(kBlockThreads), args, 0, s, ev);
}

hipError_t launch_bounds_read(const BoundsReadArgs& a, int32_t num_layers, hipStream_t s) {
    if (a.n <= 0) return hipSuccess;
    const int per = a.num_kv_heads * 2 * a.head_dim / 4;
    const int side = per < kBlockThreads ? kBlockThreads / per : 1;
    const int64_t blocks = std::min<int64_t>((static_cast<int64_t>(a.n) + side - 1) / side, 65536);
    hipLaunchKernelGGL(bounds_read_kernel, dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(num_layers)),
                       dim3(kBlockThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_bounds_copy(const PoolGeom& src, const PoolGeom& dst, int32_t num_kv_heads, int32_t head_dim,
                              int32_t layers, const CopyEntry* entries, bool on_host, int32_t n, RecordCopy how,
                              hipStream_t s) {
    if (n <= 0) return hipSuccess;
    if (on_host && n > kCopyInline) return hipErrorInvalidValue;
    const int heads = num_kv_heads, head_words = 2 * head_dim / 16;
    const int64_t words = static_cast<int64_t>(n) * (heads * head_words + 1);
    const int64_t blocks = std::min<int64_t>((words + kBlockThreads - 1) / kBlockThreads, 65536);
    const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(layers));
    if (on_host) {
        RecordList list = {};
        for (int32_t i = 0; i < n; ++i) list.e[i] = entries[i];
        hipLaunchKernelGGL(bounds_copy_inline_kernel, grid, dim3(kBlockThreads), 0, s, src, dst, n, heads, head_words, how,
                           list);
    } else {
        hipLaunchKernelGGL(bounds_copy_kernel, grid, dim3(kBlockThreads), 0, s, src, dst, entries, n, heads, head_words,
                           how);
    }
    return hipGetLastError();
}

bool select_in_one(int64_t pt_stride) { return pt_stride <= kShortThreads; }

hipError_t launch_select_pages(const SelectArgs& a, int head_dim, int dtype, hipStream_t s, const LaunchEvents& ev,
                               const LaunchEvents& ev_pick) {
    void* args[] = {const_cast<SelectArgs*>(&a)};
    if (select_in_one(a.pt_stride)) {
        const void* k = dtype == kDtypeBf16
                            ? (head_dim == 128 ? reinterpret_cast<const void*>(&page_select_kernel<128, true>)
                                               : reinterpret_cast<const void*>(&page_select_kernel<64, true>))
                            : (head_dim == 128 ? reinterpret_cast<const void*>(&page_select_kernel<128, false>)
                                               : reinterpret_cast<const void*>(&page_select_kernel<64, false>));
        return launch_kernel(k, dim3(static_cast<unsigned>(a.num_kv_heads), static_cast<unsigned>(a.batch)),
                             dim3(kShortThreads), args, 0, s, ev_pick);
    }
    if (a.pt_stride > a.width) {   // else no row has pages to choose from
        const int pages = kWave * wave_split(a.num_kv_heads).slices;   // of a block and turn
        // 1,024 blocks are resident at once, so waves go on to further pages with their queries
        // rounded (64 rows of 4,096 pages 68 us a call, with 4,096 blocks 71)
        int64_t gx = (1024 + a.batch - 1) / a.batch;
        gx = std::min<int64_t>(gx, (a.pt_stride + pages - 1) / pages);
        const void* k = dtype == kDtypeBf16
                            ? (head_dim == 128 ? reinterpret_cast<const void*>(&page_scores_kernel<128, true>)
                                               : reinterpret_cast<const void*>(&page_scores_kernel<64, true>))
                            : (head_dim == 128 ? reinterpret_cast<const void*>(&page_scores_kernel<128, false>)
                                               : reinterpret_cast<const void*>(&page_scores_kernel<64, false>));
        const hipError_t e = launch_kernel(k, dim3(static_cast<unsigned>(gx), static_cast<unsigned>(a.batch)),
                                           dim3(kBlockThreads), args, 0, s, ev);
        if (e != hipSuccess) return e;
    }
    const void* k;
    unsigned threads;
    // The keys are held in registers, as many as the table's rows may have; read again in every
    // round, 32 rows of 8K-32K tokens take 19.2 us a call instead of 17.7, 4 of 250K 42 instead of 26.
    if (a.pt_stride <= 4096) {
        k = reinterpret_cast<const void*>(&page_pick_kernel<1024, 4>);
        threads = 1024;
    } else if (a.pt_stride <= 16384) {
        k = reinterpret_cast<const void*>(&page_pick_kernel<1024, 16>);
        threads = 1024;
    } else {
        k = reinterpret_cast<const void*>(&page_pick_kernel<1024, 0>);
        threads = 1024;
    }
    return launch_kernel(k, dim3(static_cast<unsigned>(a.num_kv_heads), static_cast<unsigned>(a.batch)), dim3(threads),
                         args, 0, s, ev_pick);
}

// Parts of a list.  More parts mean fewer pages one after the other in a wave, but a second
// kernel that joins them; past one workgroup a CU they gain nothing (their number is a power of
// two, or the most that gives every CU one).  The time of each choice, in 10 ns and without what
// they share, is taken as
//   - a wave's pages, each 0.15 us and 0.45 more per 4 KiB of K, and all bytes at 6.6 TB/s, joined
//     as the legs of a right angle: the one hides behind the other, but not whole;
//   - with several parts 1.8 us for the second kernel, 0.05 a part and 0.007 a list.
// Of 1, 2, 4, .. 32 parts of 54 calls (1 to 64 rows, 16 to 512 pages a list, 4 and 16 KV heads, bf16 and
// float32) this takes the fastest or one within 5%.  32 lists of 32 pages 8.5 us a call, in one
// part 9.2; 4 of 512 pages 11.3 in 32 parts, in one 77.6, in 64 12.6; 16 of 512 16.9 in 16, 18.7
// in 8; 128 of 64 15.8 in one, 16.9 in two.
int32_t sparse_parts(int cus, int batch, int num_kv_heads, int64_t tile_bytes, int width) {
    const int64_t lists = std::max<int64_t>(static_cast<int64_t>(batch) * num_kv_heads, 1);
    const int64_t most = std::min<int64_t>(std::max<int64_t>(cus / lists, 1), (width + kBlockWaves - 1) / kBlockWaves);
    const double all = static_cast<double>(lists) * width * 2 * tile_bytes / 66000;
    const double page = 15 + 45 * static_cast<double>(tile_bytes) / 4096;
    int64_t best = 1;
    double cost = 0;
    for (int64_t parts = 1; parts <= most; parts = parts < most && 2 * parts > most ? most : 2 * parts) {
        const double wave = page * static_cast<double>((width + parts * kBlockWaves - 1) / (parts * kBlockWaves));
        const double c = std::sqrt(wave * wave + all * all) +
                         (parts > 1 ? 180 + 5 * static_cast<double>(parts) + 0.67 * static_cast<double>(lists) : 0);
        if (parts == 1 || c < cost) {
            best = parts;
            cost = c;
        }
    }
    return static_cast<int32_t>(best);
}

hipError_t launch_sparse_attention(const SparseArgs& a, int head_dim, int dtype, hipStream_t s, const LaunchEvents& ev,
                                   const LaunchEvents& ev_merge) {
    if (dtype == kDtypeBf16)
        return head_dim == 128 ? launch_sparse_for<128, true>(a, s, ev, ev_merge)
                               : launch_sparse_for<64, true>(a, s, ev, ev_merge);
    return head_dim == 128 ? launch_sparse_for<128, false>(a, s, ev, ev_merge)
                           : launch_sparse_for<64, false>(a, s, ev, ev_merge);
}

}  // namespace hck
