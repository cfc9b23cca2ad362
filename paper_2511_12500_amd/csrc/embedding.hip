// A rank's share of the lookup of tokens in a vocabulary-parallel table, stored into
// every slot of the heap, and the gradient of the rank's shard of the table.
//
//   rows[t] = scale * table[id_t - first]                for the tokens of the shard;
//   dtable[v] (+)= scale * sum over t with id_t = first + v of drows[t].
//
// The gradient takes the tokens in the order of their ids (equal ones in their own), in
// chunks of as many tokens each: a chunk sums the runs of equal ids that it holds and
// writes them, and the parts of runs that pass a chunk's end are added in their order.
// No sum depends on the order in which workgroups run.
#include "logits_rows.h"
#include "symtile_device.h"

namespace {

using namespace logits;
using symtile::u32x4;

// ---- lookup ---------------------------------------------------------------------------------
constexpr int kTileM = SYMTILE_EMBED_TILE_M, kTileBytes = SYMTILE_EMBED_TILE_BYTES;
constexpr int kLookupThreads = kTileBytes / 16;

// Written through (sc0 sc1) with the streaming hint (nt): the acknowledgement is the same.
constexpr int kStoreThroughStream = symtile::kStoreWriteThrough | symtile::kStoreNonTemporal;

struct LookupParams {
    const int64_t* tokens;
    const void* table;
    const uint64_t* bases;
    uint64_t out_off, flag_off;    // of the rows, and of the rank's counters, in a slot
    size_t ld;
    int64_t first;
    int T, rows, D, world, tiles_n, rank;
    symtile_host::Div by_tiles;
    float scale;
};

// A workgroup takes 16 tokens and 2 KB of their rows: all tokens' loads are out together, and a
// vector goes to every slot from its registers.  Bound by the stores: 8192 tokens of 8192 bf16
// into 8 slots, every eighth the shard's, 151 MB in 33 us, 4.6 TB/s (a fill reaches 6.8, a copy
// 5.0); 64 tokens 5.9 us, the load, the stores' acknowledgement and the counters in turn.
template <int DT>
__global__ void __launch_bounds__(kLookupThreads) embed_kernel(LookupParams p) {
    typedef typename Elem<DT>::type T;
    constexpr int kVec = Elem<DT>::kVec, kCols = kTileBytes / (int)sizeof(T);
    __shared__ int at[kTileM];      // row of the shard; -1: another rank's; -2: zeros
    const int t = threadIdx.x, tile = blockIdx.x;
    const int tm = p.by_tiles(tile), tn = tile - tm * p.tiles_n;
    const int t0 = tm * kTileM, count = min(kTileM, p.T - t0), col = tn * kCols + t * kVec;
    if (t < kTileM) {
        int of = -1;
        if (t < count) {
            const int64_t id = p.tokens[t0 + t];
            const uint64_t local = (uint64_t)id - (uint64_t)p.first;
            of = id < 0 ? (p.rank == 0 ? -2 : -1) : local < (uint64_t)p.rows ? (int)local : -1;
        }
        at[t] = of;
    }
    __syncthreads();
    // the slots' bases, all asked for before the first is needed, and that of the lane's counter
    uint64_t bases[SYMTILE_MAX_WORLD];
#pragma unroll
    for (int s = 0; s < SYMTILE_MAX_WORLD; ++s) bases[s] = p.bases[min(s, p.world - 1)];
    const uint64_t counter_base = p.bases[min(t, p.world - 1)];
    if (col < p.D) {
        u32x4 v[kTileM];
        int of[kTileM];
#pragma unroll
        for (int i = 0; i < kTileM; ++i) {
            of[i] = __builtin_amdgcn_readfirstlane(at[i]);
            v[i] = u32x4{0u, 0u, 0u, 0u};
            if (of[i] >= 0)
                v[i] = symtile::ld16(static_cast<const T*>(p.table) + (size_t)of[i] * p.ld + col);
        }
#pragma unroll
        for (int i = 0; i < kTileM; ++i) {
            float f[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) f[e] = element<DT>(v[i], e) * p.scale;
            v[i] = of[i] == -2 ? u32x4{0u, 0u, 0u, 0u} : pack<DT>(f);
        }
        const uint32_t row_bytes = (uint32_t)(p.D * sizeof(T));
#pragma unroll
        for (int s = 0; s < SYMTILE_MAX_WORLD; ++s) {
            if (s >= p.world) break;
            const symtile::rsrc_t dst = symtile::make_rsrc(
                reinterpret_cast<char*>(bases[s]) + p.out_off + (size_t)t0 * row_bytes,
                (uint32_t)count * row_bytes);
#pragma unroll
            for (int i = 0; i < kTileM; ++i)
                if (of[i] != -1)
                    symtile::buf_st16p<kStoreThroughStream>(v[i], dst, (uint32_t)(col * sizeof(T)),
                                                            i * row_bytes);
        }
    }
    symtile::wg_stores_done();
    if (t < p.world) {
        symtile::release_written_through();
        symtile::flag_signal(reinterpret_cast<uint32_t*>(counter_base + p.flag_off) + tile);
    }
}

// ---- tokens in the order of their ids -------------------------------------------------------
constexpr int kSortBlock = 2048, kSortBits = 11, kSortThreads = 256;
// Tokens that a workgroup places: few where there is a CU for all (64 tokens of 8192 columns
// 8.4 us with 8, 9.1 with 16), more of them share the block's keys where there is not (32768
// tokens of 4096 columns 156 us with 8, 149 with 16, 150 with 32).
constexpr int kFewPart = 8, kSortPart = 16;
constexpr uint32_t kAbsent = 0xFFFFFFFFu;
static_assert(SYMTILE_VOCAB_MAX <= 1 << (32 - kSortBits), "an id and a place in 32 bits");

struct GradParams {
    const int64_t* tokens;
    const void* drows;
    void* dtable;
    size_t ld, ld_table;
    int64_t first;
    int T, D, rows;
    float scale;
    int blocks;
    int chunk, col_blocks;           // positions and columns' parts of a workgroup of the sums
    int clear;                       // workgroups that zero the counters
    uint32_t* counters;              // [chunk][columns' part]
    int n_counters;
    uint32_t* valid;                 // [block] of the block's tokens in the shard
    uint32_t* sorted;                // [block][kSortBlock] id and place, ascending
    int* order;                      // [T] tokens in the order of their ids
    uint32_t* ids;                   // [T] their ids, kAbsent behind the shard's tokens
    float* parts;                    // [chunk][2][columns]
    symtile_host::Div by_cols;
    // of the order by digits
    int tiles, digit_bits;
    uint32_t *hist, *totals;         // [digit][tile] and [digit]
    // a digit's keys and where they go; `keys` NULL: from the tokens
    const uint32_t* keys;
    const int* from;
    uint32_t* keys_to;
    int* to;
    int shift, last;
};

// The row of the shard that a token names; kAbsent for another rank's and padding.
__device__ __forceinline__ uint32_t local_id(const GradParams& p, int64_t token) {
    const uint64_t local = (uint64_t)token - (uint64_t)p.first;
    return token >= 0 && local < (uint64_t)p.rows ? (uint32_t)local : kAbsent;
}

// Every token's rank among its block's: the number of smaller keys.  A workgroup ranks PART
// of its block's keys: each lane one of them against a share of the 2048, which it reads
// from LDS four at a time.  (With a comparison of a wave and a count of its bits each, the
// CU's scalar unit took 16 us for 32768 tokens.)  The other workgroups zero the sums'
// counters meanwhile.  Bound by the comparisons, two instructions a pair: 11 us for 32768 tokens;
// 5.0 for 2048, the ids' way from memory.  (2 to 8 keys a lane, for fewer reads from LDS, took as
// long.)
template <int PART>
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(GradParams p) {
    constexpr int kParts = kSortBlock / PART;
    const int t = threadIdx.x;
    const int other = (int)blockIdx.x - p.blocks * kParts;
    if (other >= 0) {
        for (int i = other * kSortThreads + t; i < p.n_counters; i += p.clear * kSortThreads)
            p.counters[i] = 0u;
        return;
    }
    constexpr int kOwn = kSortBlock / kSortThreads, kShares = kSortThreads / PART;
    __shared__ __attribute__((aligned(16))) uint32_t keys[kSortBlock];
    __shared__ int below[PART];
    __shared__ int valid;
    __shared__ bool last_there;
    const int block = blockIdx.x / kParts, part = blockIdx.x % kParts;
    const int t0 = block * kSortBlock, count = min(kSortBlock, p.T - t0);
    if (part * PART >= count) return;       // (the first part is never empty)
    if (t < PART) below[t] = 0;
    if (t == 0) valid = 0;
    if (t == kSortThreads - 1) last_there = false;
    uint32_t id[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int at = i * kSortThreads + t;
        id[i] = at < count ? local_id(p, p.tokens[t0 + at]) : kAbsent;
        keys[at] = id[i] != kAbsent ? id[i] << kSortBits | (uint32_t)at : kAbsent;
        if (at == kSortBlock - 1 && id[i] != kAbsent) last_there = true;
    }
    __syncthreads();
    int here = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) here += __popcll(__ballot(id[i] != kAbsent));
    if (t % 64 == 0) atomicAdd(&valid, here);
    const uint32_t mine = keys[part * PART + t % PART];
    const u32x4* share = reinterpret_cast<const u32x4*>(keys) + t / PART * (kSortBlock / kShares / 4);
    int n = 0;
#pragma unroll 8
    for (int i = 0; i < kSortBlock / kShares / 4; ++i) {
        const u32x4 k = share[i];
        n += (k[0] < mine) + (k[1] < mine) + (k[2] < mine) + (k[3] < mine);
    }
    atomicAdd(&below[t % PART], n);
    __syncthreads();
    const int at = part * PART + t;
    if (t < PART && at < count) {
        // (the block's last token may have a key like an absent one's, where ids reach 2^21)
        const uint32_t local = mine != kAbsent || (at % kSortBlock == kSortBlock - 1 && last_there)
                                   ? mine >> kSortBits : kAbsent;
        if (p.blocks == 1) {
            if (local != kAbsent) {
                p.order[below[t]] = at;
                p.ids[below[t]] = local;
            }
            if (at >= valid) p.ids[at] = kAbsent;
        } else if (local != kAbsent) {
            p.sorted[(size_t)block * kSortBlock + below[t]] = mine;
        }
    }
    if (part == 0 && t == 0) p.valid[block] = (uint32_t)valid;
}

// The place of every token of a block among all: its place in its own block, and in every
// other one the number of ids below its own, or, in earlier blocks, not above it.  A
// workgroup takes 64 tokens next to each other in their block's order, a wave of it another
// block: one load of every 32nd key bounds where all 64 can lie, and what is left to search
// are a few lines.  Bound by latency: 6.5 us for 32768 tokens (a search over the whole block for
// each of them 10; the lines through LDS 6.6).
constexpr int kMergeThreads = 1024;
__global__ void __launch_bounds__(kMergeThreads) embed_merge_kernel(GradParams p) {
    __shared__ int place[64];
    __shared__ int total;
    const int t = threadIdx.x, lane = t % 64, wave = __builtin_amdgcn_readfirstlane(t / 64);
    const int unit0 = blockIdx.x * 64, block = unit0 / kSortBlock, i = unit0 % kSortBlock + lane;
    const int count = (int)p.valid[block];
    if (t < 64) place[t] = i;
    if (t == 0) total = 0;
    __syncthreads();
    const bool some = i - lane < count;
    // lanes behind the last token search for that one
    const uint32_t key = some ? p.sorted[(size_t)block * kSortBlock + min(i, count - 1)] : 0u;
    const uint32_t id = key >> kSortBits, first = id << kSortBits, last = first | (kSortBlock - 1);
    int n = 0, sum = 0;
    for (int b = wave; b < p.blocks; b += kMergeThreads / 64) {
        const int valid = (int)p.valid[b];
        sum += valid;
        if (b == block || !some) continue;
        const uint32_t* of = p.sorted + (size_t)b * kSortBlock;
        // keys of this id lie from `first` to `last`; the smaller ids' are below the first
        const bool earlier = b < block;
        auto is_below = [&](uint32_t k, uint32_t lo, uint32_t hi) { return earlier ? k <= hi : k < lo; };
        const uint32_t coarse = lane * 32 < valid ? of[lane * 32] : 0u;
        const bool there = lane * 32 < valid;
        const uint32_t f0 = __builtin_amdgcn_readlane(first, 0), f1 = __builtin_amdgcn_readlane(first, 63);
        const int c0 = __popcll(__ballot(there && is_below(coarse, f0, f0 | (kSortBlock - 1))));
        const int c1 = __popcll(__ballot(there && is_below(coarse, f1, f1 | (kSortBlock - 1))));
        int lo = max(0, (c0 - 1) * 32), hi = min(valid, c1 * 32);
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (is_below(of[mid], first, last)) lo = mid + 1;
            else hi = mid;
        }
        n += lo;
    }
    if (n) atomicAdd(&place[lane], n);
    if (lane == 0) atomicAdd(&total, sum);
    __syncthreads();
    if (t < 64) {
        if (i < count) {
            p.order[place[t]] = block * kSortBlock + (int)(key & (kSortBlock - 1));
            p.ids[place[t]] = id;
        }
        if (unit0 + t >= total && unit0 + t < p.T) p.ids[unit0 + t] = kAbsent;
    }
}

// ---- many tokens: their order digit by digit ----------------------------------------------
// From the lowest digit of the ids to the highest, each time in the order so far: the tiles'
// counts of every digit, their sums over the tiles before, and every key to its place.  Other
// ranks' tokens and padding leave with the first digit.  Six launches, or nine from 65537 rows
// on, bound it up to some 100000 tokens (1048576 tokens of 512 columns, with their sums, 316 us).
constexpr int kTile = 2048, kDigitThreads = 256, kDigits = 256, kDigitWaves = kDigitThreads / 64;
constexpr int kPerLane = kTile / kDigitThreads;

// Key i of the tile's wave and lane, kAbsent behind the last; positions go up with i.
__device__ __forceinline__ int tile_place(int i) {
    return (threadIdx.x / 64 * kPerLane + i) * 64 + threadIdx.x % 64;
}
__device__ __forceinline__ uint32_t tile_key(const GradParams& p, int at, int n) {
    if (at >= n) return kAbsent;
    return p.keys ? p.keys[at] : local_id(p, p.tokens[at]);
}
__device__ __forceinline__ int digit_of(const GradParams& p, uint32_t key) {
    return (int)(key >> p.shift & ((1u << p.digit_bits) - 1u));
}

// The other workgroups zero the sums' counters, with the first digit.
__global__ void __launch_bounds__(kDigitThreads) embed_count_kernel(GradParams p) {
    const int t = threadIdx.x, other = (int)blockIdx.x - p.tiles;
    if (other >= 0) {
        for (int i = other * kDigitThreads + t; i < p.n_counters; i += p.clear * kDigitThreads)
            p.counters[i] = 0u;
        return;
    }
    __shared__ uint32_t count[kDigits];
    const int n = p.keys ? (int)p.valid[0] : p.T, tile = blockIdx.x;
    count[t] = 0;
    uint32_t key[kPerLane];
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) key[i] = tile_key(p, tile * kTile + tile_place(i), n);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
        if (key[i] != kAbsent) atomicAdd(&count[digit_of(p, key[i])], 1u);
    __syncthreads();
    p.hist[(size_t)t * p.tiles + tile] = count[t];
}

__device__ __forceinline__ uint32_t sum_below(uint32_t v, uint32_t* lds, uint32_t* total) {
    const int t = threadIdx.x, lane = t % 64;
    uint32_t up = v;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t u = __shfl_up(up, o);
        up += lane >= o ? u : 0u;
    }
    __syncthreads();
    if (lane == 63) lds[t / 64] = up;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kDigitWaves; ++w) {
        before += w < t / 64 ? lds[w] : 0u;
        all += lds[w];
    }
    *total = all;
    return before + up - v;
}

// A workgroup a digit: its tiles' counts become the sums of those before.
__global__ void __launch_bounds__(kDigitThreads) embed_scan_kernel(GradParams p) {
    __shared__ uint32_t lds[kDigitWaves];
    uint32_t* row = p.hist + (size_t)blockIdx.x * p.tiles;
    uint32_t before = 0;
    for (int i0 = 0; i0 < p.tiles; i0 += kDigitThreads) {
        const int i = i0 + threadIdx.x;
        uint32_t total;
        const uint32_t v = i < p.tiles ? row[i] : 0u, sum = sum_below(v, lds, &total);
        if (i < p.tiles) row[i] = before + sum;
        before += total;
    }
    if (threadIdx.x == 0) p.totals[blockIdx.x] = before;
}

// Places: the digits below, the tiles before, the waves before, and in a wave the keys of the
// same digit before, 64 at a time by a comparison of all lanes' bits.
__global__ void __launch_bounds__(kDigitThreads) embed_place_kernel(GradParams p) {
    __shared__ uint32_t lds[kDigitWaves];
    __shared__ volatile uint32_t seen[kDigitWaves][kDigits];
    __shared__ uint32_t first[kDigitWaves][kDigits];
    const int t = threadIdx.x, lane = t % 64, wave = t / 64, tile = blockIdx.x;
    const int n = p.keys ? (int)p.valid[0] : p.T;
    uint32_t key[kPerLane], rank[kPerLane];
    int order[kPerLane];
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        const int at = tile * kTile + tile_place(i);
        key[i] = tile_key(p, at, n);
        order[i] = p.keys && at < n ? p.from[at] : at;
    }
    const uint32_t here = p.hist[(size_t)t * p.tiles + tile];
    uint32_t total;
    const uint32_t below = sum_below(p.totals[t], lds, &total);
#pragma unroll
    for (int w = 0; w < kDigitWaves; ++w) seen[w][t] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        const bool there = key[i] != kAbsent;
        const int d = digit_of(p, key[i]);
        uint64_t same = __ballot(there);
        for (int b = 0; b < p.digit_bits; ++b) {
            const uint64_t set = __ballot(d >> b & 1);
            same &= d >> b & 1 ? set : ~set;
        }
        // (a wave's LDS accesses happen in their order)
        const uint32_t so_far = seen[wave][d];
        rank[i] = so_far + __popcll(same & ((1ull << lane) - 1));
        if (there && lane == __builtin_ctzll(same)) seen[wave][d] = so_far + __popcll(same);
    }
    __syncthreads();
    uint32_t at = below + here;
#pragma unroll
    for (int w = 0; w < kDigitWaves; ++w) {
        first[w][t] = at;
        at += seen[w][t];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        if (key[i] == kAbsent) continue;
        const uint32_t to = first[wave][digit_of(p, key[i])] + rank[i];
        p.keys_to[to] = key[i];
        p.to[to] = order[i];
    }
    if (!p.keys && tile == 0 && t == 0) p.valid[0] = total;
    if (p.last) {
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            const int behind = tile * kTile + tile_place(i);
            if (behind >= (int)total && behind < p.T) p.ids[behind] = kAbsent;
        }
    }
}

// ---- sums ------------------------------------------------------------------------------------
constexpr int kMaxChunk = 128, kSumThreads = 64;

// N values of a row of the table, at most 16 bytes of them together: rows start at
// multiples of that.
template <int DT, int N>
struct TableRow {
    typedef typename Elem<DT>::type T;
    static constexpr int kPart = N * sizeof(T) > 16 ? 16 / (int)sizeof(T) : N;
    typedef T V __attribute__((ext_vector_type(kPart)));
    V held[N / kPart];
    __device__ __forceinline__ void read(const void* table, size_t at) {
        const V* from = reinterpret_cast<const V*>(static_cast<const T*>(table) + at);
#pragma unroll
        for (int i = 0; i < N / kPart; ++i) held[i] = from[i];
    }
    // scale * sum, and what is held where that is added
    template <bool ADD>
    __device__ __forceinline__ void write(void* table, size_t at, const float* sum, float scale) const {
        V* to = reinterpret_cast<V*>(static_cast<T*>(table) + at);
#pragma unroll
        for (int i = 0; i < N / kPart; ++i) {
            V v;
#pragma unroll
            for (int e = 0; e < kPart; ++e) {
                const float f = sum[i * kPart + e];
                v[e] = (T)(ADD ? __builtin_fmaf(f, scale, (float)held[i][e]) : f * scale);
            }
            to[i] = v;
        }
    }
};

// The first position from `lo` on (before `hi`) whose id is not below `id`, or above it; by
// a wave, 64 positions a step.
template <bool ABOVE>
__device__ __forceinline__ int bound(const uint32_t* ids, int lo, int hi, uint32_t id) {
    const int lane = threadIdx.x % 64;
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64, at = lo + lane * step;
        const uint32_t k = at < hi ? ids[at] : kAbsent;
        const int c = __popcll(__ballot(at < hi && (ABOVE ? k <= id : k < id)));
        if (c == 0) break;
        hi = min(hi, lo + c * step);
        lo += (c - 1) * step + 1;
    }
    return lo;
}

// Bound by memory: 32768 tokens of 4096 bf16 added to 28672 fp32 rows 131 us for the 430 MB that
// are fetched and 176 written (the rows that have a token are read and written whole), 4.6 TB/s.
// A workgroup sums the runs of `chunk` positions in its columns.  A run inside the chunk
// goes to the table; of one that passes an end the chunk's part goes to memory, and the
// last of its chunks to arrive adds the parts, in their order.
// The other workgroups zero the rows of the table that no token names, 2 each, where
// nothing is added (2048 tokens, 1024 rows of 4096 columns: 13.1 us, with 8 each 14.3).
constexpr int kFillRows = 2;
template <int TABLE>
__device__ __forceinline__ void fill_rows(const GradParams& p, int r0) {
    const int t = threadIdx.x, n = min(kFillRows, p.rows - r0);
    const int at = bound<false>(p.ids, 0, p.T, (uint32_t)r0);
    const uint32_t id = at + t < p.T ? p.ids[at + t] : kAbsent;
    // lane l < kFillRows: is there a token of row r0 + l?
    bool there = false;
#pragma unroll
    for (int l = 0; l < kFillRows; ++l) {
        const bool any = __ballot(id == (uint32_t)(r0 + l)) != 0;
        there = t == l ? any : there;
    }
    if (__builtin_amdgcn_readlane(id, 63) < (uint32_t)(r0 + n) && t < n && !there) {
        // (the 64 positions end before the rows do)
        int lo = at + 64, hi = p.T;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (p.ids[mid] < (uint32_t)(r0 + t)) lo = mid + 1;
            else hi = mid;
        }
        there = lo < p.T && p.ids[lo] == (uint32_t)(r0 + t);
    }
    const uint64_t absent = __ballot(t < n && !there);
    const int vecs = p.D * (int)sizeof(typename Elem<TABLE>::type) / 16;
    for (int l = 0; l < n; ++l) {
        if (!(absent >> l & 1)) continue;
        u32x4* row = reinterpret_cast<u32x4*>(static_cast<typename Elem<TABLE>::type*>(p.dtable) +
                                              (size_t)(r0 + l) * p.ld_table);
        for (int i = t; i < vecs; i += kSumThreads) row[i] = u32x4{0u, 0u, 0u, 0u};
    }
}

template <int DT, int TABLE, bool ADD>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(GradParams p) {
    typedef typename Elem<DT>::type T;
    constexpr int kVec = Elem<DT>::kVec, kAhead = 8, kPartVecs = kVec / 4;
    typedef TableRow<TABLE, kVec> Row;
    __shared__ uint32_t ids[kMaxChunk + 2];     // of positions begin - 1 .. end
    __shared__ int order[kMaxChunk];
    __shared__ int first_chunk[2], last_chunk[2], arrived[2];
    const int t = threadIdx.x;
    if constexpr (!ADD) {
        if ((int)blockIdx.x >= p.n_counters) {
            fill_rows<TABLE>(p, ((int)blockIdx.x - p.n_counters) * kFillRows);
            return;
        }
    }
    const int chunk = p.by_cols(blockIdx.x), cb = blockIdx.x - chunk * p.col_blocks;
    const int begin = chunk * p.chunk, most = min(p.chunk, p.T - begin);
    for (int i = t; i < most + 2; i += kSumThreads) {
        const int at = begin - 1 + i;
        ids[i] = at >= 0 && at < p.T ? p.ids[at] : kAbsent;
        if (i < most) order[i] = p.order[begin + i];
    }
    // the ids on both sides of the chunk, for runs that pass its ends
    const uint32_t back = begin - 1 - t >= 0 ? p.ids[begin - 1 - t] : kAbsent;
    const uint32_t ahead = begin + most + t < p.T ? p.ids[begin + most + t] : kAbsent;
    __syncthreads();
    int n = most;
    while (n > 0 && ids[n] == kAbsent) --n;      // (few chunks end so)
    if (n == 0) return;
    const int col = (cb * kSumThreads + t) * kVec;
    const bool in = col < p.D;
    float sum[kVec] = {};
    // The chunk's first and last runs, where they pass its ends: they may be the same.
    const bool before = ids[0] == ids[1], after = ids[n + 1] == ids[n];
    const bool whole = before && after && ids[1] == ids[n];
    const symtile::rsrc_t part =
        symtile::make_rsrc(p.parts + (size_t)chunk * 2 * p.D, (uint32_t)p.D * 8);
    bool open = before;                          // the run began before the chunk
    for (int i0 = 0; i0 < n; i0 += kAhead) {
        u32x4 v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            v[i] = in ? symtile::ld16(static_cast<const T*>(p.drows) +
                                      (size_t)__builtin_amdgcn_readfirstlane(order[min(i0 + i, n - 1)]) * p.ld + col)
                      : u32x4{0u, 0u, 0u, 0u};
        // what the table holds where a run ends: asked for with the rows, not after their sum
        Row held[ADD ? kAhead : 1];
        if constexpr (ADD) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int at = min(i0 + i, n - 1);
                if (in && ids[at + 1] != ids[at + 2])
                    held[i].read(p.dtable, (size_t)__builtin_amdgcn_readfirstlane(ids[at + 1]) * p.ld_table + col);
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (i0 + i >= n) break;
            const int at = i0 + i;
#pragma unroll
            for (int e = 0; e < kVec; ++e) sum[e] += element<DT>(v[i], e);
            const uint32_t id = __builtin_amdgcn_readfirstlane(ids[at + 1]);
            const bool same = __builtin_amdgcn_readfirstlane(ids[at + 2]) == id;
            if (at + 1 < n && same) continue;
            if (!open && !same) {
                if (in)
                    held[ADD ? i : 0].template write<ADD>(p.dtable, (size_t)id * p.ld_table + col, sum,
                                                          p.scale);
            } else {
                // part 0: of the run that began before; 1: of the one that goes on.  (The offset of
                // part 1 is no scalar operand: behind a store of 16 bytes that has one the compiler
                // leaves no wait state before the sums' registers are cleared, and the store then
                // wrote the cleared value of some lanes' first word.)
                const uint32_t to = (uint32_t)col * 4 + (open ? 0u : (uint32_t)p.D * 4);
#pragma unroll
                for (int q = 0; q < kPartVecs; ++q) {
                    const u32x4 f = {__float_as_uint(sum[4 * q]), __float_as_uint(sum[4 * q + 1]),
                                     __float_as_uint(sum[4 * q + 2]), __float_as_uint(sum[4 * q + 3])};
                    symtile::buf_st16p<symtile::kStoreWriteThrough>(
                        f, part, in ? to + q * 16 : symtile::kOOB, 0);
                }
            }
            open = false;
#pragma unroll
            for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
        }
    }
    if (!before && !after) return;
    // The runs that pass an end: k = 0 the first one (or the only one), k = 1 the last one.
    symtile::wg_stores_done();
    const uint32_t id0 = __builtin_amdgcn_readfirstlane(ids[1]);
    const uint32_t id1 = __builtin_amdgcn_readfirstlane(ids[n]);
    int from = begin, to = begin + n;
    if (before) {
        const uint64_t other = __ballot(back != id0);
        from = other ? begin - __builtin_ctzll(other) : bound<false>(p.ids, 0, begin - 64, id0);
    }
    if (after) {
        const uint64_t other = __ballot(ahead != id1);
        to = other ? begin + n + __builtin_ctzll(other)
                   : bound<true>(p.ids, begin + n + 64, p.T, id1);
    }
    if (t < 2) {
        const int c0 = t == 0 ? from / p.chunk : chunk, c1 = t == 1 || whole ? (to - 1) / p.chunk : chunk;
        first_chunk[t] = c0;
        last_chunk[t] = c1;
        arrived[t] = 0;
        if (t == 0 ? before : after && !whole) {
            symtile::release_written_through();
            arrived[t] = symtile::atomic_add<__ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT>(
                             p.counters + (size_t)c0 * p.col_blocks + cb, 1u) == (uint32_t)(c1 - c0);
        }
    }
    __syncthreads();
    symtile::acquire_coherent_reads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (!__builtin_amdgcn_readfirstlane(arrived[k]) || !in) continue;
        const int c0 = first_chunk[k], c1 = last_chunk[k];
        const uint32_t id = k == 0 ? ids[1] : ids[n];
        for (int c = c0; c <= c1; c += kAhead) {
            u32x4 v[kAhead][kPartVecs];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const symtile::rsrc_t of = symtile::make_rsrc(
                    p.parts + (size_t)min(c + i, c1) * 2 * p.D, (uint32_t)p.D * 8);
#pragma unroll
                for (int q = 0; q < kPartVecs; ++q)
                    v[i][q] = symtile::buf_ld16p<symtile::kLoadCoherent>(
                        of, c + i <= c1 ? (uint32_t)(col * 4 + q * 16) : symtile::kOOB,
                        c + i == c0 ? (uint32_t)p.D * 4 : 0u);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
#pragma unroll
                for (int e = 0; e < kVec; ++e) sum[e] += __uint_as_float(v[i][e / 4][e % 4]);
        }
        Row row;
        if constexpr (ADD) row.read(p.dtable, (size_t)id * p.ld_table + col);
        row.template write<ADD>(p.dtable, (size_t)id * p.ld_table + col, sum, p.scale);
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
    }
}

// ---- host --------------------------------------------------------------------------------------
int ceil_div(int a, int b) { return (a + b - 1) / b; }
size_t up(size_t n) { return (n + 255) / 256 * 256; }
bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

// How the sums are laid out over workgroups: one wave each, columns by 16 bytes a lane (32768
// tokens of 4096 columns 149 us, four waves 156), and the largest chunks of 8, 32 or 128
// positions that leave 4096 workgroups if all tokens are the shard's, since the parts of runs that
// pass their ends go through memory (16384 tokens of 4096 columns: 8 179 us, 32 157; 131072: 32
// 408, 64 381, 128 369); a chunk's rows are asked for 8 at a time.  The host does not know how many
// tokens are the shard's; the workgroups behind those return at once.  (With chunks by that number,
// which the device knows, a rank of 8 took: 8192 tokens of 8192 columns 26 us for 30, 65536 55 for
// 63, but 32768 35 for 33 and 131072 77 to 81 for 70.)
struct GradPlan {
    int col_blocks, chunk, chunks;
};
GradPlan grad_plan(int T, int D, size_t esize) {
    GradPlan g{};
    g.col_blocks = ceil_div((int)((size_t)D * esize / 16), kSumThreads);
    const size_t positions = (size_t)T * g.col_blocks;
    g.chunk = positions < 4096 * 32 ? 8 : positions < 4096 * kMaxChunk ? 32 : kMaxChunk;
    g.chunks = ceil_div(T, g.chunk);
    return g;
}

// Above it by digits, six launches or more, where counting and merging grow with the square of
// the tokens (of 64 columns, added to 28672 rows, whole calls, us, by digits / by merging: 32768
// 42 / 26, 65536 50 / 50, 131072 52 / 96).
constexpr int kByDigits = 65536;

struct GradWorkspace {
    size_t valid, counters, sorted, order, ids, parts, bytes;
    size_t keys, hist;               // of the order by digits, in place of `sorted`
};
// For rows of any of the types.  Behind the counters that other operators leave at zero for
// each other.
GradWorkspace grad_workspace(int T, int D) {
    GradWorkspace w{};
    const size_t blocks = (size_t)ceil_div(T, kSortBlock);
    size_t counters = 0, chunks = 0;
    for (size_t esize : {2, 4}) {
        const GradPlan g = grad_plan(T, D, esize);
        counters = std::max(counters, (size_t)g.chunks * g.col_blocks);
        chunks = std::max(chunks, (size_t)g.chunks);
    }
    w.valid = (size_t)symtile_host::kWorkspaceCounters * 4;
    w.counters = w.valid + up(blocks * 4);
    w.sorted = w.counters + up(counters * 4);
    w.keys = w.sorted + up((size_t)T * 4);
    w.hist = w.keys + up((size_t)T * 4);
    w.order = T > kByDigits ? w.hist + up((size_t)kDigits * (ceil_div(T, kTile) + 1) * 4)
                            : w.sorted + (blocks > 1 ? blocks * kSortBlock * 4 : 0);
    w.ids = w.order + up((size_t)T * 4);
    w.parts = w.ids + up((size_t)T * 4);
    w.bytes = w.parts + chunks * 2 * D * 4;
    return w;
}

symtile_status check_rows(int T, int D) {
    if (T < 0 || D < 0) return fail(SYMTILE_EINVAL, "negative size");
    if (D % 8) return fail(SYMTILE_EINVAL, "D must be a multiple of 8");
    if (D > (1 << 20)) return fail(SYMTILE_EINVAL, "D exceeds 1048576");
    if (T > (1 << 24)) return fail(SYMTILE_EINVAL, "T exceeds 16777216 tokens");
    if ((size_t)T * D > size_t(1) << 38) return fail(SYMTILE_EINVAL, "T * D exceeds 2^38");
    return SYMTILE_OK;
}
symtile_status check_shard(int64_t first, int rows) {
    if (first < 0) return fail(SYMTILE_EINVAL, "first < 0");
    if (rows < 0 || rows > SYMTILE_VOCAB_MAX)
        return fail(SYMTILE_EINVAL, "rows of the table must be in 0 .. " + std::to_string(SYMTILE_VOCAB_MAX));
    return SYMTILE_OK;
}
symtile_status check_matrix(const char* what, const void* p, size_t* ld, int rows, int cols,
                            size_t esize) {
    if (*ld == 0) *ld = (size_t)cols;
    if (*ld < (size_t)cols) return fail(SYMTILE_EINVAL, std::string(what) + ": row stride smaller than D");
    if (*ld * esize % 16 || misaligned(p, 16))
        return fail(SYMTILE_EINVAL, std::string(what) + ": rows must be 16-byte aligned");
    if (rows && *ld > (SIZE_MAX >> 3) / (size_t)rows)
        return fail(SYMTILE_EINVAL, std::string(what) + " exceeds the address space");
    return SYMTILE_OK;
}

symtile_status launch_grid(const void* kernel, unsigned wgs, unsigned threads, void* params,
                           symtile_stream s, const char* what) {
    void* args[] = {params};
    hipError_t e = hipLaunchKernel(kernel, dim3(wgs), dim3(threads), args, 0,
                                   static_cast<hipStream_t>(s));
    if (e == hipSuccess) e = hipGetLastError();
    return e == hipSuccess ? SYMTILE_OK : symtile_host::hip_fail(e, what);
}

symtile_status order_by_digits(GradParams p, const GradWorkspace& w, char* base, symtile_stream s) {
    int bits = 1;
    while (bits < 32 && (p.rows - 1) >> bits) ++bits;
    const int digits = ceil_div(bits, 8);
    p.digit_bits = ceil_div(bits, digits);
    p.tiles = ceil_div(p.T, kTile);
    p.hist = reinterpret_cast<uint32_t*>(base + w.hist);
    p.totals = p.hist + (size_t)kDigits * p.tiles;
    uint32_t* const keys[2] = {p.ids, reinterpret_cast<uint32_t*>(base + w.keys)};
    int* const order[2] = {p.order, reinterpret_cast<int*>(base + w.sorted)};
    for (int d = 0; d < digits; ++d) {
        const int to = (digits - 1 - d) % 2;         // the last one into ids and order
        p.keys = d ? keys[1 - to] : nullptr;
        p.from = d ? order[1 - to] : nullptr;
        p.keys_to = keys[to];
        p.to = order[to];
        p.shift = d * p.digit_bits;
        p.last = d == digits - 1;
        const unsigned clear = d ? 0u : (unsigned)p.clear;
        symtile_status st = launch_grid(reinterpret_cast<const void*>(&embed_count_kernel),
                                        (unsigned)p.tiles + clear, kDigitThreads, &p, s,
                                        "embed_count_kernel launch");
        if (!st)
            st = launch_grid(reinterpret_cast<const void*>(&embed_scan_kernel), kDigits, kDigitThreads,
                             &p, s, "embed_scan_kernel launch");
        if (!st)
            st = launch_grid(reinterpret_cast<const void*>(&embed_place_kernel), (unsigned)p.tiles,
                             kDigitThreads, &p, s, "embed_place_kernel launch");
        if (st) return st;
    }
    return SYMTILE_OK;
}

const void* sum_kernel_of(int dtype, int table, bool add) {
    auto with = [&](auto d, auto w) -> const void* {
        constexpr int DT = decltype(d)::value, TABLE = decltype(w)::value;
        return add ? reinterpret_cast<const void*>(&embed_sum_kernel<DT, TABLE, true>)
                   : reinterpret_cast<const void*>(&embed_sum_kernel<DT, TABLE, false>);
    };
    auto second = [&](auto d) -> const void* {
        switch (table) {
            case SYMTILE_F16: return with(d, std::integral_constant<int, SYMTILE_F16>{});
            case SYMTILE_BF16: return with(d, std::integral_constant<int, SYMTILE_BF16>{});
            default: return with(d, std::integral_constant<int, SYMTILE_F32>{});
        }
    };
    switch (dtype) {
        case SYMTILE_F16: return second(std::integral_constant<int, SYMTILE_F16>{});
        case SYMTILE_BF16: return second(std::integral_constant<int, SYMTILE_BF16>{});
        default: return second(std::integral_constant<int, SYMTILE_F32>{});
    }
}

}  // namespace

extern "C" symtile_status symtile_embed_all_scatter(
    symtile_heap* h, const int64_t* tokens, int T, const void* table, int rows, int D, size_t ld,
    int dtype, int64_t first, float scale, void* rows_local, uint32_t* arrived_local, int rank,
    int world_size, symtile_stream s) {
    if (!h) return fail(SYMTILE_EINVAL, "heap is NULL");
    const size_t esize = elem_size(dtype);
    if (!esize) return fail(SYMTILE_EINVAL, "unknown dtype");
    if (world_size != h->world) return fail(SYMTILE_EINVAL, "world_size differs from the heap's");
    if (rank < 0 || rank >= world_size) return fail(SYMTILE_EINVAL, "rank out of range");
    if (symtile_status st = check_rows(T, D)) return st;
    if (symtile_status st = check_shard(first, rows)) return st;
    if (!std::isfinite(scale)) return fail(SYMTILE_EINVAL, "scale must be finite");
    if (symtile_status st = check_matrix("table", table, &ld, rows, D, esize)) return st;
    if (T == 0 || D == 0) return SYMTILE_OK;
    if (!tokens || (rows && !table) || !rows_local || !arrived_local)
        return fail(SYMTILE_EINVAL, "NULL pointer");
    if (misaligned(rows_local, 16) || misaligned(arrived_local, 4) || misaligned(tokens, 8))
        return fail(SYMTILE_EINVAL, "rows_local must be 16-byte aligned, tokens 8, counters 4");
    const int tiles_m = ceil_div(T, kTileM);
    const int tiles_n = ceil_div(D, kTileBytes / (int)esize);
    if ((size_t)tiles_m * tiles_n > (size_t(1) << 24))
        return fail(SYMTILE_EINVAL, "more than 16777216 tiles");
    const size_t out_bytes = (size_t)T * D * esize;
    const size_t flag_bytes = (size_t)world_size * tiles_m * tiles_n * 4;
    if (!symtile_host::in_slot(h, rows_local, out_bytes, rank))
        return fail(SYMTILE_EINVAL, "rows_local [T, D] not inside slot of rank");
    if (!symtile_host::in_slot(h, arrived_local, flag_bytes, rank))
        return fail(SYMTILE_EINVAL, "arrived_local not inside slot of rank");
    const uint64_t c0 = reinterpret_cast<uint64_t>(rows_local);
    const uint64_t f0 = reinterpret_cast<uint64_t>(arrived_local);
    if (c0 < f0 + flag_bytes && f0 < c0 + out_bytes)
        return fail(SYMTILE_EINVAL, "arrived_local overlaps rows_local");
    LookupParams p{};
    p.tokens = tokens;
    p.table = table;
    p.bases = h->dev_bases;
    p.out_off = c0 - h->host_bases[rank];
    p.flag_off = f0 - h->host_bases[rank] + (size_t)rank * tiles_m * tiles_n * 4;
    p.ld = ld;
    p.first = first;
    p.T = T;
    p.rows = rows;
    p.D = D;
    p.world = world_size;
    p.tiles_n = tiles_n;
    p.rank = rank;
    p.by_tiles = symtile_host::make_div(tiles_n);
    p.scale = scale;
    int prev = -1;
    if (symtile_status st = symtile_host::set_device(h, &prev)) return st;
    const void* kernel = dtype == SYMTILE_F16    ? reinterpret_cast<const void*>(&embed_kernel<SYMTILE_F16>)
                         : dtype == SYMTILE_BF16 ? reinterpret_cast<const void*>(&embed_kernel<SYMTILE_BF16>)
                                                 : reinterpret_cast<const void*>(&embed_kernel<SYMTILE_F32>);
    const symtile_status st = launch_grid(kernel, (unsigned)(tiles_m * tiles_n), kLookupThreads, &p,
                                          s, "embed_kernel launch");
    if (prev >= 0) (void)hipSetDevice(prev);
    return st;
}

extern "C" symtile_status symtile_embed_workspace_bytes(int device, int T, int D, size_t* bytes) {
    if (!bytes) return fail(SYMTILE_EINVAL, "bytes is NULL");
    *bytes = 0;
    if (symtile_status st = check_rows(T, D)) return st;
    if (symtile_host::cu_count(device) <= 0)
        return fail(SYMTILE_EINVAL, "device " + std::to_string(device) + " out of range");
    if (T && D) *bytes = grad_workspace(T, D).bytes;
    return SYMTILE_OK;
}

extern "C" symtile_status symtile_embed_backward(
    int device, const int64_t* tokens, int T, const void* drows, int D, size_t ld, int dtype,
    int64_t first, int rows, float scale, void* dtable, size_t ld_table, int table_dtype,
    int accumulate, void* workspace, size_t workspace_bytes, symtile_stream s) {
    const size_t esize = elem_size(dtype), table_esize = elem_size(table_dtype);
    if (!esize || !table_esize) return fail(SYMTILE_EINVAL, "unknown dtype");
    if (symtile_status st = check_rows(T, D)) return st;
    if (symtile_status st = check_shard(first, rows)) return st;
    if (!std::isfinite(scale)) return fail(SYMTILE_EINVAL, "scale must be finite");
    if (accumulate != 0 && accumulate != 1) return fail(SYMTILE_EINVAL, "accumulate must be 0 or 1");
    if (symtile_status st = check_matrix("drows", drows, &ld, T, D, esize)) return st;
    if (symtile_status st = check_matrix("dtable", dtable, &ld_table, rows, D, table_esize)) return st;
    if (rows == 0 || D == 0 || (T == 0 && accumulate)) return SYMTILE_OK;
    if (!dtable || (T && (!tokens || !drows))) return fail(SYMTILE_EINVAL, "NULL pointer");
    if (misaligned(tokens, 8)) return fail(SYMTILE_EINVAL, "tokens must be 8-byte aligned");
    const uintptr_t a = reinterpret_cast<uintptr_t>(drows), b = reinterpret_cast<uintptr_t>(dtable);
    if (T && a < b + ((size_t)(rows - 1) * ld_table + D) * table_esize &&
        b < a + ((size_t)(T - 1) * ld + D) * esize)
        return fail(SYMTILE_EINVAL, "dtable overlaps drows");
    const GradWorkspace w = T ? grad_workspace(T, D) : GradWorkspace{};
    if (symtile_status st = check_workspace(workspace, workspace_bytes, w.bytes)) return st;
    GradParams p{};
    p.tokens = tokens;
    p.drows = drows;
    p.dtable = dtable;
    p.ld = ld;
    p.ld_table = ld_table;
    p.first = first;
    p.T = T;
    p.D = D;
    p.rows = rows;
    p.scale = scale;
    p.blocks = ceil_div(T, kSortBlock);
    if (T) {
        const GradPlan g = grad_plan(T, D, esize);
        p.chunk = g.chunk;
        p.col_blocks = g.col_blocks;
        p.by_cols = symtile_host::make_div(g.col_blocks);
        p.n_counters = g.chunks * g.col_blocks;
        p.clear = std::min(64, ceil_div(p.n_counters, kSortThreads));
        char* base = static_cast<char*>(workspace);
        p.valid = reinterpret_cast<uint32_t*>(base + w.valid);
        p.counters = reinterpret_cast<uint32_t*>(base + w.counters);
        p.sorted = reinterpret_cast<uint32_t*>(base + w.sorted);
        p.order = reinterpret_cast<int*>(base + w.order);
        p.ids = reinterpret_cast<uint32_t*>(base + w.ids);
        p.parts = reinterpret_cast<float*>(base + w.parts);
    }
    OnDevice on(device);
    if (on.status) return on.status;
    if (T > kByDigits) {
        if (symtile_status st = order_by_digits(p, w, static_cast<char*>(workspace), s)) return st;
    } else if (T) {
        const int part = p.blocks == 1 ? kFewPart : kSortPart;
        const void* sort = p.blocks == 1
                               ? reinterpret_cast<const void*>(&embed_sort_kernel<kFewPart>)
                               : reinterpret_cast<const void*>(&embed_sort_kernel<kSortPart>);
        if (symtile_status st = launch_grid(sort, (unsigned)(p.blocks * (kSortBlock / part) + p.clear),
                                            kSortThreads, &p, s, "embed_sort_kernel launch"))
            return st;
    }
    if (p.blocks > 1 && T <= kByDigits) {
        if (symtile_status st = launch_grid(reinterpret_cast<const void*>(&embed_merge_kernel),
                                            (unsigned)(p.blocks * (kSortBlock / 64)), kMergeThreads, &p,
                                            s, "embed_merge_kernel launch"))
            return st;
    }
    const unsigned fill = accumulate ? 0u : (unsigned)ceil_div(rows, kFillRows);
    return launch_grid(sum_kernel_of(dtype, table_dtype, accumulate != 0), (unsigned)p.n_counters + fill,
                       kSumThreads, &p, s, "embed_sum_kernel launch");
}
