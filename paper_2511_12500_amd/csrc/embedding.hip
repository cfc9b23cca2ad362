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

// A workgroup takes 16 tokens and 2 KB of their rows.
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
        for (int s = 0; s < p.world; ++s) {
            const symtile::rsrc_t dst = symtile::make_rsrc(
                reinterpret_cast<char*>(p.bases[s]) + p.out_off + (size_t)t0 * row_bytes,
                (uint32_t)count * row_bytes);
#pragma unroll
            for (int i = 0; i < kTileM; ++i)
                if (of[i] != -1)
                    symtile::buf_st16p<symtile::kStoreWriteThrough>(
                        v[i], dst, (uint32_t)(col * sizeof(T)), i * row_bytes);
        }
    }
    symtile::wg_stores_done();
    if (t < p.world) {
        symtile::release_written_through();
        symtile::flag_signal(reinterpret_cast<uint32_t*>(p.bases[t] + p.flag_off) + tile);
    }
}

// ---- tokens in the order of their ids -------------------------------------------------------
constexpr int kSortBlock = 2048, kSortBits = 11, kSortThreads = 256;
constexpr int kSortPart = 32;        // tokens that a workgroup places
constexpr int kSortParts = kSortBlock / kSortPart;
constexpr uint32_t kAbsent = 0xFFFFFFFFu;
static_assert(SYMTILE_VOCAB_MAX <= 1 << (32 - kSortBits), "an id and a place in 32 bits");

struct GradParams {
    const int64_t* tokens;
    const void* drows;
    void* dtable;
    size_t ld, ld_table;
    int64_t first;
    int T, D, rows, accumulate;
    float scale;
    int blocks, col_blocks;
    int fill;                        // workgroups that zero the table
    int* total;                      // tokens of the shard
    uint32_t* valid;                 // [block] of the block
    uint32_t* sorted;                // [block][kSortBlock] id and place, ascending
    int* order;                      // [T] tokens in the order of their ids
    uint32_t* ids;                   // [T] their ids
    float* parts;                    // [chunk][2][columns]
    int columns;
    symtile_host::Div by_cols;
};

// Every token's rank among its block's: the number of smaller keys, each wave comparing
// one key with 8 of its own a lane.  The other workgroups zero the table.
template <int ESIZE>
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(GradParams p) {
    const int t = threadIdx.x;
    if ((int)blockIdx.x >= p.blocks * kSortParts) {
        const int vecs = p.D * ESIZE / 16;
        for (int r = blockIdx.x - p.blocks * kSortParts; r < p.rows; r += p.fill) {
            u32x4* row = reinterpret_cast<u32x4*>(static_cast<char*>(p.dtable) +
                                                  (size_t)r * p.ld_table * ESIZE);
            for (int i = t; i < vecs; i += kSortThreads) row[i] = u32x4{0u, 0u, 0u, 0u};
        }
        return;
    }
    constexpr int kOwn = kSortBlock / kSortThreads;
    __shared__ uint32_t keys[kSortPart];
    __shared__ int below[kSortPart];
    __shared__ int valid;
    const int block = blockIdx.x / kSortParts, part = blockIdx.x % kSortParts;
    const int t0 = block * kSortBlock, count = min(kSortBlock, p.T - t0);
    if (part * kSortPart >= count) return;       // (the first part is never empty)
    if (t < kSortPart) {
        keys[t] = kAbsent;
        below[t] = 0;
    }
    if (t == 0) valid = 0;
    __syncthreads();
    uint32_t own[kOwn];
    int here = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int at = i * kSortThreads + t;
        own[i] = kAbsent;
        if (at < count) {
            const uint64_t local = (uint64_t)p.tokens[t0 + at] - (uint64_t)p.first;
            if (p.tokens[t0 + at] >= 0 && local < (uint64_t)p.rows) {
                own[i] = (uint32_t)local << kSortBits | (uint32_t)at;
                ++here;
                if (at / kSortPart == part) keys[at % kSortPart] = own[i];
            }
        }
    }
    if (part == 0 && here) atomicAdd(&valid, here);
    __syncthreads();
    for (int j = 0; j < kSortPart; ++j) {
        const uint32_t key = __builtin_amdgcn_readfirstlane(keys[j]);
        int n = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) n += __popcll(__ballot(own[i] < key));
        if (t % 64 == 0) atomicAdd(&below[j], n);
    }
    __syncthreads();
    // (an absent token's key may equal a present one's where ids reach 2^21: by its place)
    const int at = part * kSortPart + t;
    if (t < kSortPart && at < count) {
        const uint64_t local = (uint64_t)p.tokens[t0 + at] - (uint64_t)p.first;
        if (p.tokens[t0 + at] >= 0 && local < (uint64_t)p.rows) {
            if (p.blocks == 1) {
                p.order[below[t]] = at;
                p.ids[below[t]] = (uint32_t)local;
            } else {
                p.sorted[(size_t)block * kSortBlock + below[t]] = keys[t];
            }
        }
    }
    if (part == 0 && t == 0) {
        p.valid[block] = (uint32_t)valid;
        if (p.blocks == 1) *p.total = valid;
    }
}

// The place of every token of a block among all: its place in its own block, and in every
// other one the number of ids below its own, or, in earlier blocks, not above it.  16
// lanes a token, a block each.
__global__ void __launch_bounds__(kSortThreads) embed_merge_kernel(GradParams p) {
    const int lane = threadIdx.x % 16;
    const int64_t unit = ((int64_t)blockIdx.x * kSortThreads + threadIdx.x) / 16;
    const int block = (int)(unit / kSortBlock), i = (int)(unit % kSortBlock);
    if (block == 0 && i == 0) {
        int n = 0;
        for (int b = lane; b < p.blocks; b += 16) n += (int)p.valid[b];
#pragma unroll
        for (int o = 8; o; o >>= 1) n += __shfl_xor(n, o);
        if (lane == 0) *p.total = n;
    }
    if (block >= p.blocks || i >= (int)p.valid[block]) return;
    const uint32_t key = p.sorted[(size_t)block * kSortBlock + i], id = key >> kSortBits;
    int place = lane == 0 ? i : 0;
    for (int b = lane; b < p.blocks; b += 16) {
        if (b == block) continue;
        const uint32_t* of = p.sorted + (size_t)b * kSortBlock;
        // keys of this id lie between; those with ids below it are below the first
        const uint32_t first = id << kSortBits, last = first | (kSortBlock - 1);
        int lo = 0, hi = (int)p.valid[b];
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            const uint32_t k = of[mid];
            if (b < block ? k <= last : k < first) lo = mid + 1;
            else hi = mid;
        }
        place += lo;
    }
#pragma unroll
    for (int o = 8; o; o >>= 1) place += __shfl_xor(place, o);
    if (lane == 0) {
        p.order[place] = block * kSortBlock + (int)(key & (kSortBlock - 1));
        p.ids[place] = id;
    }
}

// ---- sums ------------------------------------------------------------------------------------
constexpr int kChunk = 32, kSumThreads = 256;

// n values at p, as the table's type.
template <int DT, int N>
__device__ __forceinline__ void add_row(void* table, size_t at, const float* sum, float scale,
                                        bool accumulate) {
    typedef typename Elem<DT>::type T;
    // (at most 16 bytes of alignment: rows start at multiples of that)
    constexpr int kPart = N * sizeof(T) > 16 ? 16 / (int)sizeof(T) : N;
    typedef T V __attribute__((ext_vector_type(kPart)));
    V* to = reinterpret_cast<V*>(static_cast<T*>(table) + at);
#pragma unroll
    for (int i = 0; i < N / kPart; ++i) {
        const float* f = sum + i * kPart;
        V v = {};
        if (accumulate) v = to[i];
#pragma unroll
        for (int e = 0; e < kPart; ++e)
            v[e] = (T)(accumulate ? __builtin_fmaf(f[e], scale, (float)v[e]) : f[e] * scale);
        to[i] = v;
    }
}

template <int DT, int TABLE>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(GradParams p) {
    typedef typename Elem<DT>::type T;
    constexpr int kVec = Elem<DT>::kVec, kAhead = 8;
    __shared__ uint32_t ids[kChunk + 2];     // of positions begin - 1 .. end
    __shared__ int order[kChunk];
    const int t = threadIdx.x, threads = blockDim.x;
    const int chunk = p.by_cols(blockIdx.x), cb = blockIdx.x - chunk * p.col_blocks;
    const int total = *p.total, begin = chunk * kChunk, end = min(begin + kChunk, total);
    if (begin >= total) return;
    if (t < kChunk + 2) {
        const int at = begin - 1 + t;
        ids[t] = at >= 0 && at < total ? p.ids[at] : kAbsent;
        if (t < kChunk) order[t] = begin + t < end ? p.order[begin + t] : 0;
    }
    __syncthreads();
    const int col = (cb * threads + t) * kVec;
    if (col >= p.D) return;
    const int n = end - begin;
    float sum[kVec] = {};
    bool before = ids[0] == ids[1];          // the run began before the chunk
    for (int i0 = 0; i0 < n; i0 += kAhead) {
        u32x4 v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            v[i] = symtile::ld16(static_cast<const T*>(p.drows) +
                                 (size_t)order[min(i0 + i, n - 1)] * p.ld + col);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (i0 + i >= n) break;
            const int at = i0 + i;
#pragma unroll
            for (int e = 0; e < kVec; ++e) sum[e] += element<DT>(v[i], e);
            const uint32_t id = ids[at + 1];
            if (at + 1 < n && ids[at + 2] == id) continue;
            const bool goes_on = ids[at + 2] == id;
            if (!before && !goes_on) {
                add_row<TABLE, kVec>(p.dtable, (size_t)id * p.ld_table + col, sum, p.scale,
                                     p.accumulate);
            } else {
                float* to = p.parts + ((size_t)chunk * 2 + (before ? 0 : 1)) * p.columns + col;
#pragma unroll
                for (int e = 0; e < kVec; ++e) to[e] = sum[e];
            }
            before = false;
#pragma unroll
            for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
        }
    }
}

// Runs that begin in a chunk and pass its end.
template <int DT, int TABLE>
__global__ void __launch_bounds__(kSumThreads) embed_join_kernel(GradParams p) {
    constexpr int kVec = Elem<DT>::kVec, kAhead = 4;
    __shared__ int last_chunk;
    const int t = threadIdx.x, threads = blockDim.x;
    const int chunk = p.by_cols(blockIdx.x), cb = blockIdx.x - chunk * p.col_blocks;
    const int total = *p.total, begin = chunk * kChunk, end = begin + kChunk;
    if (end >= total) return;
    const uint32_t id = p.ids[end - 1];
    if (p.ids[end] != id || (begin > 0 && p.ids[begin - 1] == id)) return;
    if (t == 0) {
        int lo = end + 1, hi = total;      // the run's end: the first position of another id
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (p.ids[mid] == id) lo = mid + 1;
            else hi = mid;
        }
        last_chunk = (lo - 1) / kChunk;
    }
    __syncthreads();
    const int col = (cb * threads + t) * kVec, last = last_chunk;
    if (col >= p.D) return;
    float sum[kVec];
    const float* from = p.parts + (size_t)chunk * 2 * p.columns + col;
#pragma unroll
    for (int e = 0; e < kVec; ++e) sum[e] = from[p.columns + e];
    for (int c = chunk + 1; c <= last; c += kAhead) {
        float v[kAhead][kVec];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                v[i][e] = p.parts[(size_t)min(c + i, last) * 2 * p.columns + col + e];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (c + i <= last)
#pragma unroll
                for (int e = 0; e < kVec; ++e) sum[e] += v[i][e];
    }
    add_row<TABLE, kVec>(p.dtable, (size_t)id * p.ld_table + col, sum, p.scale, p.accumulate);
}

// ---- host --------------------------------------------------------------------------------------
int ceil_div(int a, int b) { return (a + b - 1) / b; }
size_t up(size_t n) { return (n + 255) / 256 * 256; }
bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

struct GradWorkspace {
    size_t valid, sorted, order, ids, parts, bytes;
};
GradWorkspace grad_workspace(int T, int D) {
    GradWorkspace w{};
    const size_t blocks = (size_t)ceil_div(T, kSortBlock);
    w.valid = 256;                       // the total before it
    w.sorted = w.valid + up(blocks * 4);
    w.order = w.sorted + (blocks > 1 ? blocks * kSortBlock * 4 : 0);
    w.ids = w.order + up((size_t)T * 4);
    w.parts = w.ids + up((size_t)T * 4);
    w.bytes = w.parts + (T > kChunk ? (size_t)ceil_div(T, kChunk) * 2 * D * 4 : 0);
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

template <template <int, int> class K>
const void* by_types(int dtype, int table) {
    auto second = [&](auto d) -> const void* {
        constexpr int DT = decltype(d)::value;
        switch (table) {
            case SYMTILE_F16: return K<DT, SYMTILE_F16>::get();
            case SYMTILE_BF16: return K<DT, SYMTILE_BF16>::get();
            default: return K<DT, SYMTILE_F32>::get();
        }
    };
    switch (dtype) {
        case SYMTILE_F16: return second(std::integral_constant<int, SYMTILE_F16>{});
        case SYMTILE_BF16: return second(std::integral_constant<int, SYMTILE_BF16>{});
        default: return second(std::integral_constant<int, SYMTILE_F32>{});
    }
}
template <int DT, int TABLE>
struct SumKernel {
    static const void* get() { return reinterpret_cast<const void*>(&embed_sum_kernel<DT, TABLE>); }
};
template <int DT, int TABLE>
struct JoinKernel {
    static const void* get() { return reinterpret_cast<const void*>(&embed_join_kernel<DT, TABLE>); }
};

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
    p.accumulate = accumulate;
    p.scale = scale;
    p.blocks = ceil_div(T, kSortBlock);
    p.fill = accumulate ? 0 : std::min(rows, 1024);
    if (T) {
        char* base = static_cast<char*>(workspace);
        p.total = reinterpret_cast<int*>(base);
        p.valid = reinterpret_cast<uint32_t*>(base + w.valid);
        p.sorted = reinterpret_cast<uint32_t*>(base + w.sorted);
        p.order = reinterpret_cast<int*>(base + w.order);
        p.ids = reinterpret_cast<uint32_t*>(base + w.ids);
        p.parts = reinterpret_cast<float*>(base + w.parts);
    }
    p.columns = D;
    OnDevice on(device);
    if (on.status) return on.status;
    const void* sort = table_esize == 4 ? reinterpret_cast<const void*>(&embed_sort_kernel<4>)
                                        : reinterpret_cast<const void*>(&embed_sort_kernel<2>);
    if (symtile_status st = launch_grid(sort, (unsigned)(p.blocks * kSortParts + p.fill), kSortThreads,
                                        &p, s, "embed_sort_kernel launch"))
        return st;
    if (T == 0) return SYMTILE_OK;
    if (p.blocks > 1)
        if (symtile_status st = launch_grid(reinterpret_cast<const void*>(&embed_merge_kernel),
                                            (unsigned)(p.blocks * (kSortBlock * 16 / kSortThreads)),
                                            kSortThreads, &p, s, "embed_merge_kernel launch"))
            return st;
    const int vecs = D * (int)esize / 16;
    const int threads = std::min(kSumThreads, ceil_div(vecs, 64) * 64);
    p.col_blocks = ceil_div(vecs, threads);
    p.by_cols = symtile_host::make_div(p.col_blocks);
    const unsigned wgs = (unsigned)ceil_div(T, kChunk) * (unsigned)p.col_blocks;
    if (symtile_status st = launch_grid(by_types<SumKernel>(dtype, table_dtype), wgs,
                                        (unsigned)threads, &p, s, "embed_sum_kernel launch"))
        return st;
    if (T <= kChunk) return SYMTILE_OK;
    return launch_grid(by_types<JoinKernel>(dtype, table_dtype), wgs, (unsigned)threads, &p, s,
                       "embed_join_kernel launch");
}
