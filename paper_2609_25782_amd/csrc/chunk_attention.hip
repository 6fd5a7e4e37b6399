// Attention of several new tokens per session over the paged cache, for gfx950:
// prompt chunks (causal, the chunk's own K and V already in its pages) and trees of
// drafted tokens (each draft sees its session's cached context and the drafts its mask
// names; their K and V come dense and never enter the cache before they are accepted).
//
// Mathematics.  For a query at position p, out = sum_t w_t v_t / sum_t w_t with
// w_t = 2^(c s_t - m), s_t = q . k_t over the tokens it attends to, c = scale log2(e).
// One pass over the keys keeps the running maximum m, sum l and unnormalised output o of
// every query; a new maximum rescales l and o.
//
// Tiles.  The query heads that share a KV head are rows of one product: a tile is `tok`
// tokens x `group` heads of one (row b, KV head g), at most kRows rows, so each K/V
// byte fetched serves all of them.  A wave owns 16 NT rows and computes
//   S^T[t][row] = K[t][:] . Q[row][:]      v_mfma_f32_16x16x32_bf16 (f32: 16x16x4)
//   O^T[d][row] += V^T[d][t] P^T[t][row]   the same instruction
// Lane l of S^T holds row l % 16 and four tokens, so a row's maximum needs two cross-lane
// steps and P goes into the second product without moving: for bf16 the tokens of a pair
// of pages are assigned to the first product's A rows such that lane group l / 16 ends up
// with 8 consecutive tokens, which are the 8 contraction slots it has in the second.
//
// Blocks of kBlock keys move from the pages to LDS by 16-byte direct loads (no
// registers), STAGES - 1 blocks ahead.  A lane of such a load may fetch any 16 bytes
// while its LDS place is fixed, so the order of 16-byte groups in LDS is chosen for the
// fragment reads: every read is over 256 consecutive bytes per 16 lanes (no bank conflicts).
//
// Work split.  Tiles, with the keys they see as their cost, lie end to end in the order
// (b, g, tile); `workers` workgroups take equal ranges, cut at block boundaries inside a
// tile where need be, so prompts of any lengths, causal tiles and long contexts with few
// queries all fill the GPU.  A tile cut between workers leaves partial results
// (o, m, l) in the workspace, which chunk_merge_kernel joins.  Workgroups of one XCD
// take neighbouring ranges: they read the same K/V through the same L2.
//
// Bounds and figures (bf16, d = 128, 8 query heads per KV head, 4 KV heads, unless said).
// Prompt chunks are bound by the products and the weights between them: one prompt of 24,576 tokens takes
// 4.2-4.5 ms = 1.09-1.19 PFLOP/s, where the library's product of two 8192 x 8192 matrices reaches
// 1.19 and of two 16384 x 16384 ones 1.37, both at clocks of about 2 GHz.  Per block
// of 64 keys and 32 rows a wave issues 64 matrix instructions (1024 cycles) and 144 others, of
// them 32 exponentials (960 cycles); the matrix cores are busy 52 % of the time, waves wait for
// their turn to issue 38 % and for data or the others 24 % of theirs.  What was measured and left
// out: half a block's offset between the two waves of a SIMD, by two barriers a block (4.25 ->
// 4.64 ms) or by one that half of the waves pass before their outputs (4.56 -> 4.85 ms, 9.1 -> 10.5
// M cycles: not the clock), the next block's scores between this one's weights (registers spill:
// 6.0 ms), 64 rows per wave (spills as well), wave priorities (no change).  With K and V always in the L2 the
// long prompt would take 8 % less.  Trees of 4-16 drafts over 8K-32K tokens (32 sessions, 1.39
// GB) are bound by the reads: 242 us = 5.75 TB/s, the attention kernel alone 5.9.  Small calls
// are bound by the chain of dependent loads and the two launches: 13.5 us for 2 x 5 drafts in
// float32, 10 of them in this kernel and 2.5-4 in the merge.  No LDS bank conflicts are counted.

#include "chunk_split.h"
#include "device_common.h"
#include "kernels.h"

#include <float.h>
#include <math.h>

#include <atomic>
#include <type_traits>

namespace hck {
namespace {

constexpr int kRsrcWord3 = 0x00020000;  // raw buffer, 32-bit data format (gfx9 family)
constexpr int kXcds = 8;

typedef const __attribute__((address_space(4))) int32_t* const_i32;  // read by scalar loads
__device__ __forceinline__ const_i32 uniform_ptr(const int32_t* p) {
    return (const_i32)(reinterpret_cast<uintptr_t>(p));
}

// Tiles of 128 NT rows: 8 waves of 16 NT rows; one workgroup per CU, two waves per SIMD with 256
// registers each.  Blocks of 64 keys (f32: 32), 32 KiB at a head size of 128, in three stages
// (four measure the same within 3 %).
template <int D, bool BF16, int NT>
struct Cfg {
    static constexpr int kD = D, kWaves = 8, kNT = NT, kPages = BF16 ? 4 : 2, kStages = 3;
    static constexpr bool kBf16 = BF16;
    static constexpr int kElt = BF16 ? 2 : 4;
    static constexpr int kX = 16 / kElt;                  // elements of a 16-byte group
    static constexpr int kTile = kPageTokens * D * kElt;  // bytes of a K or V tile
    static constexpr int kPage = 2 * kTile;               // a page's K and V tiles of one KV head
    static constexpr int kBlock = kPages * kPageTokens;    // keys per block
    static constexpr int kStage = kPages * kPage;         // LDS bytes of a block
    static constexpr int kThreads = kWaves * kWave;
    // Cache policy of the page loads: nontemporal (2) where one tile holds most rows' queries
    // of a KV head, so that its K and V are read once (32 sessions x 4-16 drafts over 8K-32K tokens: 267 -> 241 us);
    // tiles of 256 rows read them again and again.
    static constexpr int kAux = NT == 1 ? 2 : 0;
    static constexpr int kPerSimd = kWaves / 4;           // waves per SIMD the registers are made for
    static constexpr int kWaveRows = 16 * NT;
    static constexpr int kRows = kWaves * kWaveRows;
    static constexpr int kTileLoads = kTile / 1024;       // 1 KiB loads of a tile
    static constexpr int kLoads = kPages * 2 * kTileLoads / kWaves;  // a wave's loads per block
    static constexpr int kQ = D / (4 * kX);               // 16-byte Q fragments of a row per lane
    static constexpr int kC = D / 16;                     // 16-dim output chunks
    static_assert(kLoads >= 1 && kTileLoads % kLoads == 0, "a wave loads one tile or a part of one");
    static_assert(!BF16 || kPages % 2 == 0, "bf16 fragments take pages in pairs");
};

template <class C, bool TREE>
__device__ __forceinline__ Row row_info(const ChunkArgs& a, int b) {
    // (2^30 tokens at most, so that places of keys stay in 32 bits)
    const int64_t most = min(static_cast<int64_t>(kPageTokens) * a.pt_stride, int64_t(1) << 30);
    const int32_t len = uniform_ptr(a.lens)[b];
    int start, n;
    if constexpr (TREE) {
        n = a.draft_lens ? uniform_ptr(a.draft_lens)[b] : a.width;
        n = n < 0 ? 0 : (n > a.width ? a.width : n);
        start = b * a.width;
    } else {
        const int s = uniform_ptr(a.starts)[b], e = uniform_ptr(a.starts)[b + 1];
        const bool in = s >= 0 && e >= s && e <= a.total_q;
        start = in ? s : 0;
        n = in ? e - s : 0;
    }
    const int bad = len < (TREE ? 0 : n) || len > most;
    return make_row<C, TREE>(a.tile_tokens, start, n, bad ? 0 : (TREE ? len : len - n), bad);
}

// What a worker takes: the blocks from `from` up to `to`.  Where `to` lies inside a tile,
// `parts` is the number of workers that share that tile from this one on.
struct Range {
    Place from, to;
    Row row;     // of from.b
    int parts;
};

__device__ __forceinline__ Place uniform_place(const Place& p) {
    return Place{__builtin_amdgcn_readfirstlane(p.b), __builtin_amdgcn_readfirstlane(p.g),
                 __builtin_amdgcn_readfirstlane(p.tile), __builtin_amdgcn_readfirstlane(p.blk)};
}

// Inclusive sum over the lanes of a wave of numbers below 2^52.
__device__ __forceinline__ int64_t wave_scan64(int64_t x) {
    constexpr int kLow = 26;
    const unsigned lo = static_cast<unsigned>(wave_scan(static_cast<int>(x & ((1 << kLow) - 1))));
    const unsigned hi = static_cast<unsigned>(wave_scan(static_cast<int>(x >> kLow)));
    return static_cast<int64_t>(lo) + (static_cast<int64_t>(hi) << kLow);
}
__device__ __forceinline__ int64_t lane_value64(int64_t x, int lane) {
    const unsigned lo = __builtin_amdgcn_readlane(static_cast<int>(x), lane);
    const unsigned hi = __builtin_amdgcn_readlane(static_cast<int>(x >> 32), lane);
    return static_cast<int64_t>(lo) | (static_cast<int64_t>(hi) << 32);
}

// The split into whole parts, a row per lane.  True where the call is cut so; out.parts is then the
// number of parts of the worker's tile, 0 for a worker without one.
template <class C, bool TREE>
__device__ bool whole_parts(const ChunkArgs& a, int k, const Row& r, Range& out) {
    const int heads = a.num_kv_heads;
    const int most = a.workers;
    if (__builtin_amdgcn_ballot_w64(!even_tiles(r))) return false;
    if (__builtin_amdgcn_ballot_w64(static_cast<int64_t>(heads) * r.tiles > most)) return false;
    const int count = heads * r.tiles;       // tiles of the row (rows without queries: none)
    const float cost = tile_cost(r);
    float total = cost * count;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) total += __shfl_xor(total, d);
    const int w = tile_parts<C, TREE>(a.tile_tokens, r, most, total);
    const int mine = count * w;
    const int upto = wave_scan(mine);
    const int all = __builtin_amdgcn_readlane(upto, kWave - 1);
    float longest = cost / w;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) longest = fmaxf(longest, __shfl_xor(longest, d));
    if (all > most || parts_too_long(longest, total, most)) return false;
    out.parts = 0;
    if (k >= all) return true;
    const uint64_t has = __builtin_amdgcn_ballot_w64(mine > 0 && upto - mine <= k);
    const int b = kWave - 1 - __builtin_clzll(has);
    out.row = make_row<C, TREE>(a.tile_tokens, __builtin_amdgcn_readlane(r.start, b), __builtin_amdgcn_readlane(r.n, b),
                                __builtin_amdgcn_readlane(r.ctx, b), __builtin_amdgcn_readlane(r.bad, b));
    out.parts = __builtin_amdgcn_readlane(w, b);
    const int rem = k - (__builtin_amdgcn_readlane(upto, b) - __builtin_amdgcn_readlane(mine, b));
    Place from, to;
    part_place<C, TREE>(a.tile_tokens, out.row, b, rem, out.parts, from, to);
    out.from = uniform_place(from);
    out.to = uniform_place(to);
    return true;
}

// Worker k's range; false where there is none.
template <class C, bool TREE>
__device__ bool worker_range(const ChunkArgs& a, int k, Range& out) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int heads = a.num_kv_heads;
    if (a.batch <= kWave) {
        // a row per lane; every wave finds the range by itself
        Row r = {};
        if (lane < a.batch) r = row_info<C, TREE>(a, lane);
        if (whole_parts<C, TREE>(a, k, r, out)) return out.parts > 0;
        const int64_t keys = heads * r.head_units(0), tiles = static_cast<int64_t>(heads) * r.tiles;
        const int64_t keys_to = wave_scan64(keys), tiles_to = wave_scan64(tiles);
        const Cuts cuts = cuts_of<C>(a.workers, lane_value64(keys_to, kWave - 1), lane_value64(tiles_to, kWave - 1));
        if (k >= cuts.workers) return false;
        const int64_t units = keys + cuts.cost * tiles;
        const int64_t first = keys_to + cuts.cost * tiles_to - units;
        out.parts = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t u = cuts.at(k + j);
            Place p{a.batch, 0, 0, 0};
            if (u < cuts.total) {
                const uint64_t has = __builtin_amdgcn_ballot_w64(units > 0 && first <= u);
                const int b = kWave - 1 - __builtin_clzll(has);
                const Row at = make_row<C, TREE>(a.tile_tokens, __builtin_amdgcn_readlane(r.start, b), __builtin_amdgcn_readlane(r.n, b),
                                                 __builtin_amdgcn_readlane(r.ctx, b), __builtin_amdgcn_readlane(r.bad, b));
                int64_t more;
                p = uniform_place(place_of<C, TREE>(a.tile_tokens, at, b, u - lane_value64(first, b), cuts.cost, more));
                if (j == 0) out.row = at;
                if (j == 1 && p.blk > 0) out.parts = worker_at(cuts, u + more) - k + 1;
            }
            (j == 0 ? out.from : out.to) = p;
        }
        out.parts = __builtin_amdgcn_readfirstlane(out.parts);
        return true;
    }
    // a run of rows per thread; the threads whose runs hold the range's ends walk them
    __shared__ int64_t s_keys[C::kWaves], s_tiles[C::kWaves];
    __shared__ Place s_place[2];
    __shared__ int s_parts;
    const int per = (a.batch + C::kThreads - 1) / C::kThreads;
    const int lo = min(a.batch, tid * per), hi = min(a.batch, lo + per);
    int64_t keys = 0, tiles = 0;
    for (int b = lo; b < hi; ++b) {
        const Row r = row_info<C, TREE>(a, b);
        keys += heads * r.head_units(0);
        tiles += static_cast<int64_t>(heads) * r.tiles;
    }
    const int64_t keys_to = wave_scan64(keys), tiles_to = wave_scan64(tiles);
    if (lane == kWave - 1) {
        s_keys[wave] = keys_to;
        s_tiles[wave] = tiles_to;
    }
    if (tid < 2) s_place[tid] = Place{a.batch, 0, 0, 0};
    if (tid == 0) s_parts = 0;
    __syncthreads();
    int64_t all_keys = 0, all_tiles = 0, keys_before = 0, tiles_before = 0;
    for (int w = 0; w < C::kWaves; ++w) {
        if (w == wave) {
            keys_before = all_keys;
            tiles_before = all_tiles;
        }
        all_keys += s_keys[w];
        all_tiles += s_tiles[w];
    }
    const Cuts cuts = cuts_of<C>(a.workers, all_keys, all_tiles);
    const int64_t sum = keys + cuts.cost * tiles;
    const int64_t first = keys_before + keys_to - keys + cuts.cost * (tiles_before + tiles_to - tiles);
    if (k < cuts.workers) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t u = cuts.at(k + j);
            if (u < first || u >= first + sum) continue;
            int64_t at = first;
            for (int b = lo; b < hi; ++b) {
                const Row r = row_info<C, TREE>(a, b);
                const int64_t units = heads * r.head_units(cuts.cost);
                if (u < at + units) {
                    int64_t more;
                    const Place p = place_of<C, TREE>(a.tile_tokens, r, b, u - at, cuts.cost, more);
                    s_place[j] = p;
                    if (j == 1 && p.blk > 0) s_parts = worker_at(cuts, u + more) - k + 1;
                    break;
                }
                at += units;
            }
        }
    }
    __syncthreads();
    out.from = uniform_place(s_place[0]);
    out.to = uniform_place(s_place[1]);
    out.parts = __builtin_amdgcn_readfirstlane(s_parts);
    if (k >= cuts.workers) return false;
    out.row = row_info<C, TREE>(a, min(out.from.b, a.batch - 1));
    return true;
}

// Page-table entry `pid`: a hot page, a cold page (num_cold is 0 where the pool reads no
// tagged entries), or no page that this call reads.
__device__ __forceinline__ bool is_hot(const ChunkArgs& a, int pid) {
    return static_cast<unsigned>(pid) < static_cast<unsigned>(a.num_hot);
}
__device__ __forceinline__ bool is_cold(const ChunkArgs& a, int pid) {
    return static_cast<unsigned>(pid ^ kPageCold) < static_cast<unsigned>(a.num_cold);
}

template <int AUX>
__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t rs, char* lds, unsigned voff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(lds), 16, voff, 0, 0, AUX);
}

// Waits until at most N of the wave's loads are in flight and its LDS reads are done,
// then for the other waves.
template <int N>
__device__ __forceinline__ void wait_loads_and_sync() {
    static_assert(N <= 63, "vmcnt");
    __asm__ volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// A block's source for one wave: its page ids (context) or drafts.
template <class C>
struct Loader {
    unsigned koff, voff;   // this lane's byte in a tile, first load (an even page's K; V)
    int wave, lane;
    __device__ explicit Loader() {
        lane = threadIdx.x & (kWave - 1);
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int g = lane >> 4, x = lane & 15;
        if constexpr (C::kBf16) {
            // LDS place (dim group 4 i + g, x): x = 8 ab + 4 (t / 8) + t % 4 with ab = (t / 4) % 2
            // (ab flipped in odd pages, so that the two pages of a pair fill all banks)
            const int t = ((x >> 2) & 1) * 8 + (x >> 3) * 4 + (x & 3);
            koff = (g * 16 + t) * 16;
            // LDS place (16-dim chunk, half page, dim): dims of one half page side by side
            voff = C::kTile + ((lane >> 5) * 16 + x) * 32 + (g & 1) * 16;
        } else {
            koff = lane * 16;
            voff = C::kTile + x * 64 + g * 16;
        }
    }
    // This wave's share of a block: one page's K or V tile, or a part of one.
    static constexpr int kShare = C::kTileLoads / C::kLoads;     // waves of a tile
    __device__ __forceinline__ int tile() const { return wave / kShare; }
    __device__ __forceinline__ int page() const { return tile() >> 1; }
    // Its loads of the page that entry `id` names; an id that names none reads zeros.
    __device__ __forceinline__ bool load_page(const ChunkArgs& a, int id, unsigned head_off, char* stage) const {
        const bool hot = is_hot(a, id), cold = is_cold(a, id);
        const char* pool = cold ? a.cold : a.hot;
        const int64_t stride = cold ? a.cold_stride : a.hot_stride;
        const int64_t n = cold ? id ^ kPageCold : (hot ? id : 0);
        const __amdgpu_buffer_rsrc_t rs =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(pool + n * stride + head_off), static_cast<short>(0),
                                              hot || cold ? C::kPage : 0, kRsrcWord3);
        const int t = tile(), first = (wave % kShare) * C::kLoads;
        const unsigned k = C::kBf16 && (page() & 1) ? koff ^ 64 : koff;
        const unsigned off = (t & 1) ? voff : k;
        char* dst = stage + t * C::kTile + first * 1024;
#pragma unroll
        for (int i = 0; i < C::kLoads; ++i) load_lds16<C::kAux>(rs, dst + i * 1024, off + (first + i) * 1024);
        return hot || cold;
    }
    // The K of drafts [key0, key0 + kBlock) of a row, by the same kind of loads; drafts past n read zeros.
    __device__ __forceinline__ void draft_keys(const ChunkArgs& a, int b, int g, int n, int key0, char* stage) const {
        const unsigned row = a.num_kv_heads * D_bytes();
        const char* base = static_cast<const char*>(a.k_new) +
                           (static_cast<int64_t>(b) * a.width * a.num_kv_heads + g) * D_bytes();
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<char*>(base), static_cast<short>(0), n > 0 ? (n - 1) * row + D_bytes() : 0, kRsrcWord3);
        constexpr int kAll = C::kPages * C::kTileLoads;
#pragma unroll
        for (int j = 0; j < (kAll + C::kWaves - 1) / C::kWaves; ++j) {
            const int idx = wave + j * C::kWaves;
            if (idx < kAll) {
                const int page = idx / C::kTileLoads, i = idx % C::kTileLoads;
                const unsigned slot = (C::kBf16 ? koff ^ ((page & 1) * 64) : koff) / 16;  // (g, t)
                const int key = key0 + page * kPageTokens + (slot & 15);
                const unsigned dim_group = 4 * i + (slot >> 4);
                // past the last draft the offset lies past the buffer's records: zeros, nothing is read
                load_lds16<0>(rs, stage + page * C::kPage + i * 1024, key < n ? key * row + dim_group * 16 : 0x7FFFFFF0u);
            }
        }
    }
    // The V of those drafts, transposed through registers.
    __device__ __forceinline__ void draft_values(const ChunkArgs& a, int b, int g, int n, int key0, char* stage) const {
        typedef typename std::conditional<C::kBf16, uint16_t, uint32_t>::type elt;
        constexpr int kQuarters = kPageTokens / C::kX;            // 16-byte groups of a dim in a page
        constexpr int kGroups = C::kPages * C::kD * kQuarters;    // of the block
        const elt* base = static_cast<const elt*>(a.v_new) +
                          (static_cast<int64_t>(b) * a.width * a.num_kv_heads + g) * C::kD;
        const int row = a.num_kv_heads * C::kD;       // (at most 64 drafts: 32-bit offsets do)
        constexpr int kRounds = (kGroups + C::kThreads - 1) / C::kThreads;
#pragma unroll 2
        for (int round = 0; round < kRounds; ++round) {
            const int s = threadIdx.x + round * C::kThreads;
            if (kGroups % C::kThreads && s >= kGroups) break;
            const int page = s / (C::kD * kQuarters), in = s % (C::kD * kQuarters);
            const int c = in / (16 * kQuarters), q = in / 16 % kQuarters, dim = c * 16 + in % 16;
            const int first = key0 + page * kPageTokens + q * C::kX;
            elt e[C::kX];
            // (the last draft in place of those past it, so that the loads go out together)
#pragma unroll
            for (int j = 0; j < C::kX; ++j) e[j] = base[min(first + j, n - 1) * row + dim];
#pragma unroll
            for (int j = 0; j < C::kX; ++j) e[j] = first + j < n ? e[j] : elt(0);
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (C::kBf16) w[j] = e[2 * j] | (static_cast<unsigned>(e[2 * j + 1]) << 16);
                else w[j] = e[j];
            }
            *reinterpret_cast<u32x4*>(stage + page * C::kPage + C::kTile + in * 16) = w;
        }
    }
    static __device__ constexpr unsigned D_bytes() { return C::kD * C::kElt; }
};

template <class C>
struct State {
    u32x4 q[C::kNT][C::kQ];
    f32x4 o[C::kNT][C::kC];
    float m[C::kNT];   // running maximum of the raw scores
    float l[C::kNT];   // this lane's part of the weights' sum
};

// What a block may show a wave's rows (only blocks that need it are masked).
struct Mask {
    int key0;                 // first key of the block
    int len;                  // keys at or past it hold nothing of the row
    unsigned ok;              // bit i: page i of the block exists
    bool draft;
    bool some;                // some row of the wave does not see the block whole
};

__device__ __forceinline__ unsigned nonfinite_code(unsigned h) {
    // 1 for +inf, 2^8 for -inf, 2^16 for NaN, as bf16; 0 for a number.  A sum of up to 64
    // of them tells which were there.
    const unsigned e = h & 0x7FFFu;
    if (e < 0x7F80u) return 0u;
    return e > 0x7F80u ? 0x4780u : ((h & 0x8000u) ? 0x4380u : 0x3F80u);
}
__device__ __forceinline__ float nonfinite_code32(unsigned h) {
    const unsigned e = h & 0x7FFFFFFFu;
    if (e < 0x7F800000u) return 0.f;
    return e > 0x7F800000u ? 65536.f : ((h >> 31) ? 256.f : 1.f);
}
__device__ __forceinline__ float nonfinite_value(float sum) {
    if (sum == 0.f) return 0.f;
    if (sum >= 65536.f) return NAN;
    const float neg = floorf(sum * (1.f / 256.f));
    const float pos = sum - 256.f * neg;
    return neg == 0.f ? INFINITY : (pos == 0.f ? -INFINITY : NAN);
}
__device__ __forceinline__ bool any_nonfinite(const u32x4& v, bool bf16) {
    bool hit = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (bf16) hit |= (v[j] & 0x7F80u) == 0x7F80u || (v[j] & 0x7F800000u) == 0x7F800000u;
        else hit |= (v[j] & 0x7F800000u) == 0x7F800000u;
    }
    return hit;
}

// Fence between a group of LDS reads and a group of matrix instructions: other instructions
// may cross it.  Without fences the compiler puts each read right before its use and the
// wave waits out the LDS latency 32 times per block.
__device__ __forceinline__ void order_fence() { __builtin_amdgcn_sched_barrier(0x0406); }

// Key that this lane's register (t, r) of S^T stands for, from the block's first, and its page.
template <class C>
__device__ __forceinline__ int lane_key(int t, int r) {
    const int g = (threadIdx.x & (kWave - 1)) >> 4;
    return C::kBf16 ? 32 * (t >> 1) + 8 * g + 4 * (t & 1) + r : 16 * t + 4 * g + r;
}
template <class C>
__device__ __forceinline__ int lane_page(int t) {
    const int g = (threadIdx.x & (kWave - 1)) >> 4;
    return C::kBf16 ? 2 * (t >> 1) + (g >> 1) : t;
}

// The lowest `n` of kX bits (n below 0: none, above kX: all).
template <class C>
__device__ __forceinline__ unsigned low_bits(int n) {
    n = n < 0 ? 0 : (n > C::kX ? C::kX : n);
    return (1u << n) - 1u;
}

// Bit 4 t + r: the row attends to that key.  A lane's keys of a contraction step are kX
// consecutive ones, so a step's bits are one run of a limit or of a draft's mask.
template <class C, bool TREE>
__device__ __forceinline__ unsigned seen_keys(const Mask& mk, int lim, uint64_t seen) {
    unsigned bits = 0;
#pragma unroll
    for (int p = 0; p < C::kPages * 4 / C::kX; ++p) {
        const int key = mk.key0 + lane_key<C>(p * C::kX / 4, 0);
        unsigned run = low_bits<C>((TREE && mk.draft ? mk.len : lim) - key);
        if constexpr (TREE)
            if (mk.draft) run &= static_cast<unsigned>(seen >> (key & 63));
        bits |= run << (C::kX * p);
    }
    return bits;
}

// Bits of this lane's V values of step p that belong to the row (the rest is cleared: slots
// past its length and missing pages may hold NaN).
template <class C>
__device__ __forceinline__ u32x4 kept_values(const Mask& mk, int p) {
    unsigned run = low_bits<C>(mk.len - (mk.key0 + lane_key<C>(p * C::kX / 4, 0)));
    if (!((mk.ok >> lane_page<C>(p * C::kX / 4)) & 1u)) run = 0;
    u32x4 keep;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (C::kBf16)
            keep[j] = ((run >> (2 * j)) & 1u) * 0xFFFFu | ((run >> (2 * j + 1)) & 1u) * 0xFFFF0000u;
        else
            keep[j] = 0u - ((run >> j) & 1u);
    }
    return keep;
}

// A block whose V holds infinities or NaN that some row must not see: a weight of 0 times
// such a value would be NaN.  This adds to every row the infinities and NaN of the tokens
// it attends to (a product of the masks with codes of the values); then clear_nonfinite
// takes them out of the block, and compute_block adds the rest.
template <class C, bool TREE>
__device__ __forceinline__ void add_nonfinite(State<C>& st, const char* stage, const Mask& mk, const int (&lim)[C::kNT],
                                              const uint64_t (&seen)[C::kNT]) {
    const int lane = threadIdx.x & (kWave - 1), g = lane >> 4, x = lane & 15;
    const char* vb = C::kBf16 ? stage + (g >> 1) * C::kPage + C::kTile + (g & 1) * 256 + x * 16
                              : stage + C::kTile + lane * 16;
    constexpr int kSteps = C::kBf16 ? C::kPages / 2 : C::kPages;
    unsigned sees[C::kNT];
#pragma unroll
    for (int n = 0; n < C::kNT; ++n) sees[n] = seen_keys<C, TREE>(mk, lim[n], seen[n]);
#pragma unroll
    for (int c = 0; c < C::kC; ++c) {
        f32x4 codes[C::kNT];
#pragma unroll
        for (int n = 0; n < C::kNT; ++n) codes[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < kSteps; ++p) {
            u32x4 v = *reinterpret_cast<const u32x4*>(vb + p * (C::kBf16 ? 2 : 1) * C::kPage + c * 256 * C::kElt);
            v &= kept_values<C>(mk, p);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = C::kBf16 ? nonfinite_code(v[j] & 0xFFFFu) | (nonfinite_code(v[j] >> 16) << 16)
                                : __float_as_uint(nonfinite_code32(v[j]));
#pragma unroll
            for (int n = 0; n < C::kNT; ++n) {
                if constexpr (C::kBf16) {
                    u32x4 one;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int bit = 4 * (2 * p + (j >> 1)) + 2 * (j & 1);
                        one[j] = ((sees[n] >> bit) & 1u ? 0x3F80u : 0u) |
                                 ((sees[n] >> (bit + 1)) & 1u ? 0x3F800000u : 0u);
                    }
                    codes[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, one), codes[n], 0, 0, 0);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        codes[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                            __uint_as_float(v[j]), (sees[n] >> (4 * p + j)) & 1u ? 1.f : 0.f, codes[n], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < C::kNT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) st.o[n][c][r] += nonfinite_value(codes[n][r]);
    }
}

// This thread's share of a block's V: the i-th of its 16-byte groups.
template <class C>
__device__ __forceinline__ u32x4* value_group(char* stage, int i) {
    return reinterpret_cast<u32x4*>(stage + i / (C::kTile / 16) * C::kPage + C::kTile + i % (C::kTile / 16) * 16);
}
template <class C>
__device__ __forceinline__ void clear_nonfinite(char* stage) {
    for (int i = threadIdx.x; i < C::kPages * C::kTile / 16; i += C::kThreads) {
        u32x4 v = *value_group<C>(stage, i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (C::kBf16)
                v[j] &= (nonfinite_code(v[j] & 0xFFFFu) ? 0u : 0xFFFFu) | (nonfinite_code(v[j] >> 16) ? 0u : 0xFFFF0000u);
            else
                v[j] = nonfinite_code32(v[j]) != 0.f ? 0u : v[j];
        }
        *value_group<C>(stage, i) = v;
    }
}

// A rescale factor 2^x <= 1 in two, which multiply o one after the other: where 2^x underflows (the
// instruction gives 0 below 2^-126) they are 2^-126 twice, not 0, so that what o holds of a number vanishes
// (below 2^-123) while an infinity or NaN stays.  (A select per value in place of the second factor: 7 short
// chunks of an odd group 34.7 us, 32.5 so.)
constexpr float kTiny = 0x1p-126f;
struct Factor {
    float f, g;
    __device__ __forceinline__ explicit Factor(float x) : f(fmaxf(__builtin_amdgcn_exp2f(x), kTiny)) {
        g = f == kTiny ? kTiny : 1.f;
    }
};

// One block for one wave.  MASKED blocks hold keys that some row must not see: their
// scores are left out, their weights are 0, and values that are none of the row's are cleared.
template <class C, bool TREE, bool MASKED>
__device__ __forceinline__ void compute_block(State<C>& st, const char* stage, float scale, float slack, const Mask& mk,
                                              const int (&lim)[C::kNT], const uint64_t (&seen)[C::kNT]) {
    const int lane = threadIdx.x & (kWave - 1), g = lane >> 4, x = lane & 15;
    // Fragments of K and then of V, in groups of kG, two groups ahead of the products.
    constexpr int kG = C::kPages * C::kQ >= 8 && C::kD > 64 ? 4 : 2;
    constexpr int kKF = C::kPages * C::kQ;                           // K fragments: (i, page t)
    constexpr int kSteps = C::kBf16 ? C::kPages / 2 : C::kPages;     // contraction steps of the output
    constexpr int kVF = kSteps * C::kC;                              // V fragments: (step p, c)
    static_assert(kKF % kG == 0 && kKF / kG >= 2 && kVF % kG == 0 && kVF / kG >= 2, "groups");
    u32x4 kf[2][kG], vf[2][kG];
    const char *kb, *vb;
    unsigned flip = 0;
    if constexpr (C::kBf16) {
        kb = stage + (x >> 3) * C::kPage + g * 256 + (x & 7) * 16;
        flip = (x >> 3) * 128;
        vb = stage + (g >> 1) * C::kPage + C::kTile + (g & 1) * 256 + x * 16;
    } else {
        kb = stage + lane * 16;
        vb = stage + C::kTile + lane * 16;
    }
    const auto load_k = [&](int group) {
#pragma unroll
        for (int u = 0; u < kG; ++u) {
            const int i = (group * kG + u) / C::kPages, t = (group * kG + u) % C::kPages;
            const char* kt = C::kBf16 ? kb + (t >> 1) * 2 * C::kPage + (((t & 1) * 128) ^ flip) : kb + t * C::kPage;
            kf[group & 1][u] = *reinterpret_cast<const u32x4*>(kt + i * 1024);
        }
    };
    const auto load_v = [&](int group) {
#pragma unroll
        for (int u = 0; u < kG; ++u) {
            const int p = (group * kG + u) / C::kC, c = (group * kG + u) % C::kC;
            vf[group & 1][u] = *reinterpret_cast<const u32x4*>(vb + p * (C::kBf16 ? 2 : 1) * C::kPage + c * 256 * C::kElt);
        }
    };
    f32x4 s[C::kPages][C::kNT];
#pragma unroll
    for (int t = 0; t < C::kPages; ++t)
#pragma unroll
        for (int n = 0; n < C::kNT; ++n) s[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    load_k(0);
    load_k(1);
    order_fence();
#pragma unroll
    for (int group = 0; group < kKF / kG; ++group) {
#pragma unroll
        for (int u = 0; u < kG; ++u) {
            const int i = (group * kG + u) / C::kPages, t = (group * kG + u) % C::kPages;
            const u32x4 k = kf[group & 1][u];
            if constexpr (C::kBf16) {
#pragma unroll
                for (int n = 0; n < C::kNT; ++n)
                    s[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, st.q[n][i]), s[t][n], 0, 0, 0);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int n = 0; n < C::kNT; ++n)
                        s[t][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                            __uint_as_float(k[j]), __uint_as_float(st.q[n][i][j]), s[t][n], 0, 0, 0);
            }
        }
        order_fence();
        if (group + 2 < kKF / kG) load_k(group + 2);
        else load_v(group + 2 - kKF / kG);
        order_fence();
    }
    if (MASKED && mk.some) {
#pragma unroll
        for (int n = 0; n < C::kNT; ++n) {
            const unsigned sees = seen_keys<C, TREE>(mk, lim[n], seen[n]);
#pragma unroll
            for (int t = 0; t < C::kPages; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[t][n][r] = (sees >> (4 * t + r)) & 1u ? s[t][n][r] : -INFINITY;
            if (!TREE && mk.ok != (1u << C::kPages) - 1) {   // tokens of a missing page: NaN to rows that see them
#pragma unroll
                for (int t = 0; t < C::kPages; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!((mk.ok >> lane_page<C>(t)) & 1u) && ((sees >> (4 * t + r)) & 1u)) s[t][n][r] = NAN;
            }
        }
    }
    // Running maximum.  It is raised only where a score exceeds it by more than 2^8 in the
    // weights (`slack` in raw scores): a weight may then be up to 2^8, which float32 sums and
    // bf16 weights hold as well as weights up to 1, and most blocks leave l and o alone.
    bool rise = false;
    float mx[C::kNT];
#pragma unroll
    for (int n = 0; n < C::kNT; ++n) {
        mx[n] = st.m[n];
#pragma unroll
        for (int t = 0; t < C::kPages; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx[n] = fmaxf(mx[n], s[t][n][r]);
        rise |= mx[n] > st.m[n] + slack;
    }
    if (__builtin_amdgcn_ballot_w64(rise)) {
#pragma unroll
        for (int n = 0; n < C::kNT; ++n) {
            float v = fmaxf(mx[n], __shfl_xor(mx[n], 16));
            v = fmaxf(v, __shfl_xor(v, 32));
            // (l and o of a row without a maximum hold 0, or an infinity or NaN that has to stay)
            const Factor w(st.m[n] == -INFINITY ? 0.f : (st.m[n] - v) * scale);
            // A tile's first block finds nothing to rescale, and often no later block does: masked blocks,
            // which come first, look (8 sessions x 8 drafts over 2K tokens 19.3 -> 19.1 us); the loop of the
            // others loses by the branch (8 chunks over 8K-32K tokens 1.39 -> 1.53 ms).
            if (!MASKED || __builtin_amdgcn_ballot_w64(w.f != 1.f)) {
                st.l[n] *= w.f;
#pragma unroll
                for (int c = 0; c < C::kC; ++c) st.o[n][c] = st.o[n][c] * w.f * w.g;
            }
            st.m[n] = v;
        }
    }
    // weights
    u32x4 pb[C::kBf16 ? C::kPages / 2 : 1][C::kNT];
#pragma unroll
    for (int n = 0; n < C::kNT; ++n) {
        const float ms = st.m[n] == -INFINITY ? 0.f : st.m[n] * scale;
#pragma unroll
        for (int t = 0; t < C::kPages; ++t) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][n][r], scale, -ms));   // left out: 0
                s[t][n][r] = w;
                st.l[n] += w;
            }
            if constexpr (C::kBf16) {
                // the weights round to bf16 for the product, as the matrix cores take them;
                // their sum stays in float32
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                    const bf16x2 two = {static_cast<__bf16>(s[t][n][2 * h]), static_cast<__bf16>(s[t][n][2 * h + 1])};
                    pb[t >> 1][n][2 * (t & 1) + h] = __builtin_bit_cast(unsigned, two);
                }
            }
        }
    }
    // output
    u32x4 keep[MASKED ? kSteps : 1];
    if constexpr (MASKED) {
#pragma unroll
        for (int p = 0; p < kSteps; ++p) keep[p] = ~u32x4{0u, 0u, 0u, 0u};
        // (past the last draft there are zeros)
        if (!mk.draft && (mk.key0 + C::kBlock > mk.len || mk.ok != (1u << C::kPages) - 1))
#pragma unroll
            for (int p = 0; p < kSteps; ++p) keep[p] = kept_values<C>(mk, p);
    }
#pragma unroll
    for (int group = 0; group < kVF / kG; ++group) {
#pragma unroll
        for (int u = 0; u < kG; ++u) {
            const int p = (group * kG + u) / C::kC, c = (group * kG + u) % C::kC;
            u32x4 v = vf[group & 1][u];
            if constexpr (MASKED) v &= keep[p];
            if constexpr (C::kBf16) {
#pragma unroll
                for (int n = 0; n < C::kNT; ++n)
                    st.o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, pb[p][n]), st.o[n][c], 0, 0, 0);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int n = 0; n < C::kNT; ++n)
                        st.o[n][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[j]), s[p][n][j], st.o[n][c],
                                                                          0, 0, 0);
            }
        }
        order_fence();
        if (group + 2 < kVF / kG) load_v(group + 2);
        order_fence();
    }
}

__device__ __forceinline__ void store4(const ChunkArgs& a, bool bf16, char* out, const f32x4& v) {
    if (bf16) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        const bf16x4 w = {static_cast<__bf16>(v[0]), static_cast<__bf16>(v[1]), static_cast<__bf16>(v[2]),
                          static_cast<__bf16>(v[3])};
        *reinterpret_cast<u32x2*>(out) = __builtin_bit_cast(u32x2, w);
    } else {
        *reinterpret_cast<f32x4*>(out) = v;
    }
}

template <class C, bool TREE>
__global__ __launch_bounds__(C::kThreads) __attribute__((amdgpu_waves_per_eu(C::kPerSimd, C::kPerSimd))) void chunk_attend_kernel(const ChunkArgs a) {
    extern __shared__ __align__(1024) char s_kv[];
    __shared__ int s_poison;   // 1 + the last block found with infinities or NaN to take out
    __shared__ int s_bad;      // 1: a page that every row of the tile attends to is missing
    const int lane = threadIdx.x & (kWave - 1), gq = lane >> 4, x = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    // neighbouring ranges to one XCD (blocks go to the XCDs in turn)
    int k = blockIdx.x;
    if (gridDim.x % kXcds == 0) k = (k % kXcds) * (gridDim.x / kXcds) + k / kXcds;
    Range range = {};
    const bool work = worker_range<C, TREE>(a, k, range);
    // the range is one for the workgroup: in scalar registers, whichever way it was found
    Place at = uniform_place(range.from);
    const Place end = uniform_place(range.to);
    const int parts = __builtin_amdgcn_readfirstlane(range.parts);
    Row row = make_row<C, TREE>(a.tile_tokens, __builtin_amdgcn_readfirstlane(range.row.start),
                                __builtin_amdgcn_readfirstlane(range.row.n),
                                __builtin_amdgcn_readfirstlane(range.row.ctx),
                                __builtin_amdgcn_readfirstlane(range.row.bad));     // of at.b
    bool recorded = false;   // this worker holds the first part of a cut tile
    const Loader<C> ld;
    const unsigned head_bytes = 2 * C::kTile;
    bool first_piece = true;
    if (work) {
        while (before(at, end)) {
            if (at.b >= a.batch) break;
            if (at.g >= a.num_kv_heads || row.tiles == 0) {   // on to the next row with queries
                int b = at.b + 1;
                while (b < a.batch) {
                    const uint64_t some = __builtin_amdgcn_ballot_w64(
                        b + lane < a.batch && row_info<C, TREE>(a, min(b + lane, a.batch - 1)).tiles > 0);
                    if (some) {
                        b += __builtin_ctzll(some);
                        break;
                    }
                    b += kWave;
                }
                at = Place{b, 0, 0, 0};
                if (b < a.batch) row = row_info<C, TREE>(a, b);
                continue;
            }
            const int nb = tile_blocks<C, TREE>(a.tile_tokens, row, at.tile);
            const int kv_head = at.g;
            const bool to_end = end.b == at.b && end.g == at.g && end.tile == at.tile;
            const int k0 = at.blk, k1 = to_end ? end.blk : nb;
            const int nd = draft_blocks<C, TREE>(row);
            const int keys = tile_keys<C, TREE>(a.tile_tokens, row, at.tile);
            const int tok0 = at.tile * a.tile_tokens;
            const int toks = min(a.tile_tokens, row.n - tok0);
            const unsigned head_off = kv_head * head_bytes;
            const const_i32 pt = uniform_ptr(a.page_table + static_cast<int64_t>(at.b) * a.pt_stride);
            const int last_page = (keys + kPageTokens - 1) / kPageTokens - 1;

            if (!first_piece) wait_loads_and_sync<63>();   // the last piece's reads of the stages are over
            first_piece = false;
            if (threadIdx.x == 0) s_poison = s_bad = 0;
            wait_loads_and_sync<63>();

            // this wave's rows
            State<C> st;
            int lim[C::kNT], tok[C::kNT];
            uint64_t seen[C::kNT];
            bool live[C::kNT];
            int64_t qrow[C::kNT];
            const int w0 = wave * C::kWaveRows;
            const bool wave_live = w0 < toks * a.group;
            const int wtok1 = min(toks - 1, (w0 + C::kWaveRows - 1) / a.group);   // its last token
#pragma unroll
            for (int n = 0; n < C::kNT; ++n) {
                const int r = w0 + n * 16 + x;
                tok[n] = r / a.group;
                live[n] = tok[n] < toks;
                const int t = live[n] ? tok0 + tok[n] : 0;
                const int h = live[n] ? r % a.group : 0;
                qrow[n] = ((static_cast<int64_t>(row.start) + t) * a.num_q_heads + kv_head * a.group + h) * C::kD;
                lim[n] = TREE ? row.ctx : (live[n] ? row.ctx + t + 1 : 0);
                seen[n] = 0;
                if constexpr (TREE)
                    if (live[n]) seen[n] = a.masks[static_cast<int64_t>(at.b) * a.width + t];
                const char* qp = static_cast<const char*>(a.q) + qrow[n] * C::kElt + gq * 16;
#pragma unroll
                for (int i = 0; i < C::kQ; ++i) {
                    u32x4 v = {0u, 0u, 0u, 0u};
                    if (live[n]) v = *reinterpret_cast<const u32x4*>(qp + i * 64);
                    st.q[n][i] = v;
                }
                st.m[n] = -INFINITY;
                st.l[n] = 0.f;
#pragma unroll
                for (int c = 0; c < C::kC; ++c) st.o[n][c] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            // Order of a tile's blocks: the drafts', then the context's from its end down, so that the
            // blocks that need masks come first (they are the ones at the end of what a row sees).
            const int nc = nb - nd;                              // context blocks
            // blocks that some row of the tile does not see whole; those and a tail that is not full;
            // blocks that no row of this wave sees
            int partly, masked, unseen = 0;
            int sure = keys;   // what the wave's first row sees
            if constexpr (TREE) {
                partly = nd;
                masked = nd + (row.ctx % C::kBlock != 0);
            } else {
                partly = masked = nb - (row.ctx + tok0 + 1) / C::kBlock;
                unseen = nb - ((row.ctx + tok0 + wtok1) / C::kBlock + 1);
                sure = row.ctx + tok0 + w0 / a.group + 1;
            }
            if (!wave_live) unseen = nb;
            const auto first_page = [&](int j) { return (nc - 1 - (j - nd)) * C::kPages; };
            // Entry of page i of block j; a page past the row's last holds no key that a row sees: no page.
            const auto page_id = [&](int j, int i) {
                const int p = (j >= nd && j < k1 ? first_page(j) : 0) + i;
                return p <= last_page ? pt[p] : -1;
            };
            int id;                        // of this wave's page of the block that is fetched next
            int first_ids[C::kStages - 1]; // of the first blocks, loaded together
#pragma unroll
            for (int i = 0; i < C::kStages - 1; ++i) first_ids[i] = page_id(k0 + i, ld.page());
            char* into = s_kv;                    // stage of that block
            const auto next_stage = [&](char* p) { return p == s_kv + (C::kStages - 1) * C::kStage ? s_kv : p + C::kStage; };
            const auto next_id = [&](int j) { id = page_id(j, ld.page()); };
            const auto fetch_pages = [&](int j) {   // context block j of [k0, k1)
                // a missing page of a block that every row sees whole is NaN for all of them
                // (tokens past the row's last, in its last block, are no matter)
                if (!ld.load_page(a, id, head_off, into))
                    if (j >= partly && first_page(j) + ld.page() <= last_page) s_bad = 1;
                into = next_stage(into);
            };
            const auto fetch = [&](int j) {         // block j of [k0, k1)
                if (TREE && j < nd) {
                    ld.draft_keys(a, at.b, kv_head, row.n, j * C::kBlock, into);
                    ld.draft_values(a, at.b, kv_head, row.n, j * C::kBlock, into);
                    into = next_stage(into);
                } else {
                    fetch_pages(j);
                }
            };
#pragma unroll
            for (int i = 0; i < C::kStages - 1; ++i)
                if (k0 + i < k1) {
                    id = first_ids[i];
                    fetch(k0 + i);
                }
            next_id(k0 + C::kStages - 1);
            if (a.negate) {
#pragma unroll
                for (int n = 0; n < C::kNT; ++n)
#pragma unroll
                    for (int i = 0; i < C::kQ; ++i) st.q[n][i] ^= C::kBf16 ? 0x80008000u : 0x80000000u;
            }
            int j = k0;
            char* stage = s_kv;
            const auto mask_of = [&](int j) {
                if (TREE && j < nd) return Mask{j * C::kBlock, row.n, ~0u, true, true};
                unsigned ok = 0;
#pragma unroll
                for (int i = 0; i < C::kPages; ++i) {
                    const int e = page_id(j, i);
                    ok |= (TREE || is_hot(a, e) || is_cold(a, e)) ? 1u << i : 0u;   // (trees: s_bad)
                }
                const int key0 = first_page(j) * kPageTokens;
                return Mask{key0, keys, ok, false, key0 + C::kBlock > sure || ok != (1u << C::kPages) - 1};
            };
            // Block j has arrived for every wave (the loads of later blocks may go on: 1 KiB each,
            // kLoads per block and wave).
            const auto arrive = [&]() {
                if ((TREE && j < nd) || k1 - 1 - j < C::kStages - 2)
                    wait_loads_and_sync<0>();
                else
                    wait_loads_and_sync<(C::kStages - 2) * C::kLoads>();
            };
            for (; j < k1 && j < masked; ++j) {
                arrive();
                if (j < partly) {
                    // an infinity or NaN among values that some row must not see?
                    bool hit = false;
                    for (int i = threadIdx.x; i < C::kPages * C::kTile / 16; i += C::kThreads)
                        hit |= any_nonfinite(*value_group<C>(stage, i), C::kBf16);
                    if (__builtin_amdgcn_ballot_w64(hit) && lane == 0) s_poison = j + 1;
                    wait_loads_and_sync<63>();
                    if (s_poison == j + 1) {
                        if (j >= unseen) add_nonfinite<C, TREE>(st, stage, mask_of(j), lim, seen);
                        wait_loads_and_sync<63>();
                        clear_nonfinite<C>(stage);
                        wait_loads_and_sync<63>();
                    }
                }
                if (j + C::kStages - 1 < k1) {
                    fetch(j + C::kStages - 1);
                    next_id(j + C::kStages);
                }
                if (j >= unseen) compute_block<C, TREE, true>(st, stage, a.scale_log2, a.slack, mask_of(j), lim, seen);
                stage = next_stage(stage);
            }
            for (; j < k1; ++j) {
                arrive();
                if (j + C::kStages - 1 < k1) {
                    fetch_pages(j + C::kStages - 1);
                    next_id(j + C::kStages);
                }
                if (wave_live) compute_block<C, TREE, false>(st, stage, a.scale_log2, a.slack, Mask{}, lim, seen);
                stage = next_stage(stage);
            }
            bool bad = row.bad;
            bad |= s_bad != 0;   // set by fetches before the last turn's barrier

            // Whether a row attends to anything at all: to tokens whose scores are all minus infinity the
            // weights are 0 / 0, to nothing the output is zero.
            const auto attends = [&](int n) {
                return !TREE || row.ctx > 0 || (seen[n] & (~0ull >> (64 - row.n))) != 0;
            };
            // the rows' sums over their four lanes
            float l[C::kNT];
#pragma unroll
            for (int n = 0; n < C::kNT; ++n) {
                l[n] = st.l[n] + __shfl_xor(st.l[n], 16);
                l[n] += __shfl_xor(l[n], 32);
                if (bad) l[n] = NAN;
            }
            if (k0 == 0 && k1 == nb) {
#pragma unroll
                for (int n = 0; n < C::kNT; ++n) {
                    const float inv = l[n] == 0.f ? (attends(n) ? NAN : 0.f) : 1.f / l[n];
                    char* out = static_cast<char*>(a.out) + (qrow[n] + 4 * gq) * C::kElt;
                    if (live[n]) {
#pragma unroll
                        for (int c = 0; c < C::kC; ++c) store4(a, C::kBf16, out + c * 16 * C::kElt, st.o[n][c] * inv);
                    }
                }
            } else {
                const int slot = 2 * k + (k0 == 0 ? 1 : 0);
                float* po = a.part_o + static_cast<int64_t>(slot) * C::kRows * C::kD;
                float* pm = a.part_ml + static_cast<int64_t>(slot) * 2 * C::kRows;
#pragma unroll
                for (int n = 0; n < C::kNT; ++n) {
                    if (!live[n]) continue;
                    const int r = w0 + n * 16 + x;
#pragma unroll
                    for (int c = 0; c < C::kC; ++c)
                        *reinterpret_cast<f32x4*>(po + r * C::kD + c * 16 + 4 * gq) = st.o[n][c];
                    if (gq == 0) {
                        // (finite wherever the row attends to anything, in this part or another)
                        pm[r] = attends(n) ? fmaxf(st.m[n] * a.scale_log2, -FLT_MAX) : -INFINITY;
                        pm[C::kRows + r] = l[n];
                    }
                }
                if (k0 == 0) {
                    recorded = true;
                    if (threadIdx.x == 0)
                        a.recs[k] = ChunkRec{parts, toks * a.group,
                                             (static_cast<int64_t>(row.start) + tok0) * a.num_q_heads + kv_head * a.group};
                }
            }
            if (to_end) break;
            at.blk = 0;
            if (++at.tile == row.tiles) {
                at.tile = 0;
                ++at.g;
            }
        }
    }
    if (!recorded && threadIdx.x == 0) a.recs[k] = ChunkRec{0, 0, 0};
}

// Joins the partial results of the tiles cut between workers: with M the largest of the
// parts' maxima, out = sum 2^(m_i - M) o_i / sum 2^(m_i - M) l_i.  A block takes rows of the
// tile whose first part worker k left in slot 2 k + 1; its other parts are in the slots 2 (k + 1),
// 2 (k + 2), ... of the workers after it.  A wave takes kIter rows, kAtOnce parts at a time.
// Most tiles are cut once or twice: then the loads of all of the wave's rows are in flight
// together.  (2 x 5 drafts in float32: 13.6 us; with half as many rows per wave 14.4, the
// blocks without work cost, though 16 sessions with one KV head gain, 70.5 -> 65.4; with twice as many
// 14.4, and 64 rows over 32K tokens 27.3 -> 34.0.)  The record holds all that a row's place needs, so
// that only two loads follow each other.  Where few tiles are cut into equal parts, the k that
// hold a record are multiples of 8 and more, which plain block numbers all send to one XCD:
// the blocks of one k differ in blockIdx.x (4 sessions x 32 drafts over 8K tokens, 16 parts each: the
// call takes 77.9 us with plain numbers, 45.1 so).
template <class C>
struct Merge {
    static constexpr int kLanes = C::kD / 4, kAtOnce = kWave / kLanes;
    static constexpr int kIter = C::kRows / 64;     // rows of a wave
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, den = 0.f;
    __device__ __forceinline__ void join(float m, float l, const f32x4& o) {
        const float t = fmaxf(top, m);
        // (1 for a lane without a part, or parts of a row that attends to nothing: they hold 0)
        const Factor w0(top == -INFINITY ? 0.f : top - t), w1(m == -INFINITY ? 0.f : m - t);
        acc = acc * w0.f * w0.g + o * w1.f * w1.g;
        den = den * w0.f + l * w1.f;
        top = t;
    }
    __device__ __forceinline__ void finish(const ChunkArgs& a, const ChunkRec& rec, int r, int sub, int col) {
#pragma unroll
        for (int d = kLanes; d < kWave; d <<= 1) {
            const float m = __shfl_xor(top, d), l = __shfl_xor(den, d);
            f32x4 o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = __shfl_xor(acc[j], d);
            join(m, l, o);
        }
        if (sub == 0 && r < rec.rows) {
            const int64_t q = rec.first + static_cast<int64_t>(r / a.group) * a.num_q_heads + r % a.group;
            const float inv = den == 0.f ? (top == -INFINITY ? 0.f : NAN) : 1.f / den;
            store4(a, C::kBf16, static_cast<char*>(a.out) + (q * C::kD + col * 4) * C::kElt, acc * inv);
        }
    }
};

template <class C>
__global__ __launch_bounds__(kBlockThreads) void chunk_merge_kernel(const ChunkArgs a) {
    using M = Merge<C>;
    const int k = (blockIdx.x + blockIdx.y) % gridDim.x, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    ChunkRec rec = a.recs[k];
    rec.parts = __builtin_amdgcn_readfirstlane(rec.parts);
    rec.rows = __builtin_amdgcn_readfirstlane(rec.rows);
    const int r0 = blockIdx.y * kBlockWaves + wave, step = gridDim.y * kBlockWaves;
    if (rec.parts == 0 || r0 >= rec.rows) return;
    const int sub = lane / M::kLanes, col = lane % M::kLanes;
    const auto part_of = [&](int p, int r, float& m, float& l, f32x4& o) {
        const int64_t slot = p == 0 ? 2 * k + 1 : 2 * (k + p);
        m = a.part_ml[slot * 2 * C::kRows + r];
        l = a.part_ml[slot * 2 * C::kRows + C::kRows + r];
        o = *reinterpret_cast<const f32x4*>(a.part_o + (slot * C::kRows + r) * C::kD + col * 4);
    };
    constexpr int kFew = 2;     // rounds of kAtOnce parts
    if (rec.parts <= kFew * M::kAtOnce) {
        float m[M::kIter][kFew], l[M::kIter][kFew];
        f32x4 o[M::kIter][kFew];
#pragma unroll
        for (int i = 0; i < M::kIter; ++i)
#pragma unroll
            for (int f = 0; f < kFew; ++f)   // (a row or part past the last: the last)
                part_of(min(sub + f * M::kAtOnce, rec.parts - 1), min(r0 + i * step, rec.rows - 1), m[i][f], l[i][f],
                        o[i][f]);
#pragma unroll
        for (int i = 0; i < M::kIter; ++i) {
            M row;
#pragma unroll
            for (int f = 0; f < kFew; ++f)
                if (sub + f * M::kAtOnce < rec.parts) row.join(m[i][f], l[i][f], o[i][f]);
            row.finish(a, rec, r0 + i * step, sub, col);
        }
        return;
    }
    for (int r = r0; r < rec.rows; r += step) {
        M row;
        constexpr int kMany = 8;
        for (int p0 = sub; p0 < rec.parts; p0 += kMany * M::kAtOnce) {
            float m[kMany], l[kMany];
            f32x4 o[kMany];
#pragma unroll
            for (int f = 0; f < kMany; ++f) part_of(min(p0 + f * M::kAtOnce, rec.parts - 1), r, m[f], l[f], o[f]);
#pragma unroll
            for (int f = 0; f < kMany; ++f)
                if (p0 + f * M::kAtOnce < rec.parts) row.join(m[f], l[f], o[f]);
        }
        row.finish(a, rec, r, sub, col);
    }
}

template <class C, bool TREE>
hipError_t launch_cfg(ChunkArgs a, int workers, hipStream_t s, const LaunchEvents& ev, const LaunchEvents& ev_merge) {
    a.tile_tokens = C::kRows / a.group;
    a.workers = workers;
    chunk_workspace_layout(a, C::kRows, C::kD);
    const size_t lds = static_cast<size_t>(C::kStages) * C::kStage;
    const void* kern = reinterpret_cast<const void*>(&chunk_attend_kernel<C, TREE>);
    // more LDS than a launch gets unasked, asked for once per kernel and device
    static std::atomic<uint64_t> asked{0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = uint64_t(1) << (dev & 63);
    if (dev > 63 || !(asked.load(std::memory_order_relaxed) & bit)) {
        e = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
        if (e != hipSuccess) return e;
        asked.fetch_or(bit, std::memory_order_relaxed);
    }
    void* args[] = {&a};
    e = launch_kernel(kern, dim3(workers), dim3(C::kThreads), args, lds, s, ev);
    if (e != hipSuccess) return e;
    const void* merge = reinterpret_cast<const void*>(&chunk_merge_kernel<C>);
    return launch_kernel(merge, dim3(workers, C::kRows / (kBlockWaves * Merge<C>::kIter)), dim3(kBlockThreads), args, 0,
                         s, ev_merge);
}

template <int D, bool BF16, bool TREE>
hipError_t launch_shape(const ChunkArgs& a, const ChunkPlan& p, hipStream_t s, const LaunchEvents& ev,
                        const LaunchEvents& ev_merge) {
    if (p.rows == 128) return launch_cfg<Cfg<D, BF16, 1>, TREE>(a, p.workers, s, ev, ev_merge);
    return launch_cfg<Cfg<D, BF16, 2>, TREE>(a, p.workers, s, ev, ev_merge);
}

}  // namespace

// Rows of a tile, by the rows that a session brings to a KV head (the average of prompt
// chunks, the most of trees).  256: a wave has 32 rows, and each K and V fragment that it reads
// from LDS serves two products, else the reads bound the call; 128, where a tile of 256 would
// compute rows that are not there or wait for K and V all the same.  16 sessions of 8K-32K
// tokens, 128 rows each: 131 us with tiles of 128 rows, 158 with 256; 136 rows: 231 and 166;
// 256 rows: 247 and 201; 64 sessions of 8 rows: 93 and 111.  64 decode steps of 8 rows and a
// chunk of 4096 rows in one call (71 rows on average): 127 and 158.  Calls whose few tiles do not
// fill the workers would do better with 128 rows, which the rule does not see: 4 x 256 rows over 8K
// tokens 35.6 and 45.1, 7 chunks of 1-701 tokens with 3 heads 28.8 and 32.7.  (Tiles of 64 rows were
// never faster by more than 2 %.)
ChunkPlan chunk_plan(int cus, int64_t rows_per_seq) {
    ChunkPlan p;
    p.rows = rows_per_seq <= 128 ? 128 : 256;
    p.workers = cus;
    return p;
}

hipError_t launch_chunk_attention(const ChunkArgs& a, const ChunkPlan& p, int head_dim, int dtype, bool tree,
                                  hipStream_t s, const LaunchEvents& ev, const LaunchEvents& ev_merge) {
    if (a.batch <= 0) return hipSuccess;
#define HCK_CHUNK(DD, BB) \
    (tree ? launch_shape<DD, BB, true>(a, p, s, ev, ev_merge) : launch_shape<DD, BB, false>(a, p, s, ev, ev_merge))
    if (head_dim == 128) return dtype == kDtypeBf16 ? HCK_CHUNK(128, true) : HCK_CHUNK(128, false);
    return dtype == kDtypeBf16 ? HCK_CHUNK(64, true) : HCK_CHUNK(64, false);
#undef HCK_CHUNK
}

}  // namespace hck
