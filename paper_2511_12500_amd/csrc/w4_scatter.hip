// A few tokens' product with a rank's shard of 4-bit weights, stored into every
// slot of the heap (the All-Scatter of Section 4.2.1 behind a matrix-vector
// product).
//
// C[m, n] = sum_k X[m, k] (q[n, k] - zero[n, k / group]) scale[n, k / group].
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <string>

#include "symtile.h"
#include "symtile_device.h"
#include "symtile_internal.h"

namespace {

constexpr int kTileN = SYMTILE_W4_TILE_N;
constexpr int kBlockK = 128;        // weights a lane quartet's loads cover in a column
constexpr int kChunkK = 8192;       // weights of a column whose scales are in LDS

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct W4Params {
    const void* X;
    const uint8_t* q;
    const void* scales;
    const uint8_t* zeros;
    const uint64_t* bases;
    uint64_t c_off, flag_off;   // of the rank's column block and its counters in a slot
    int M, N, K, ldx, groups, world;
    int ldc;                    // elements
    // of the wide kernel: K in `splits` parts of `part_steps` steps each (the last may
    // have fewer), whose sums meet in `partials`
    int splits, part_steps;
    uint32_t* counters;
    float* partials;
};

// Weights as floating point without a conversion: 4 bits in the fraction of a power
// of two are 16 + q (bfloat16) or 64 + q (float16), exactly.  The offset goes out with
// the zero point: sum x (q - z) = sum x (16 + q) + sum x (-(16 + z)), the second sum by
// a matrix instruction too, whose right operand is one number a column and group.
template <bool BF>
struct Nibbles {
    static constexpr uint32_t kBase = BF ? 0x4180u : 0x5400u;
    static constexpr int kAt = BF ? 3 : 4;   // where the 4 bits start
    uint32_t mask, base;

    // The constants in registers (one scalar, one vector): as literals they would
    // keep the and-or from being one instruction.
    __device__ __forceinline__ Nibbles()
        : mask((0xFu << kAt) * 0x10001u), base(kBase * 0x10001u) {
        asm("" : "+s"(mask));
        asm("" : "+v"(base));
    }
    static __device__ __forceinline__ uint32_t shifted(uint32_t w, int left) {
        return left >= 0 ? w << left : w >> -left;
    }
    // The 8 weights of a word in pairs, weights j and j + 4 in dword j, for X in that
    // order: two instructions a pair.
    __device__ __forceinline__ symtile::u32x4 apart(uint32_t w) const {
        symtile::u32x4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = (shifted(w, kAt - 4 * j) & mask) | base;
        return r;
    }
    // Weights 2 j and 2 j + 1 in dword j: the even and the odd ones of the word are
    // moved into place within their bytes, then a byte of each and an and-or a pair.
    __device__ __forceinline__ symtile::u32x4 adjacent(uint32_t w) const {
        const uint32_t even = w << kAt, odd = shifted(w, kAt - 4);
        symtile::u32x4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            r[j] = (__builtin_amdgcn_perm(odd, even, 0x0C040C00u + 0x00010001u * j) & mask) | base;
        return r;
    }
    static __device__ __forceinline__ uint32_t minus_offset(uint32_t zero) {
        return (kBase | 0x8000u | zero << kAt) * 0x10001u;
    }
};

// Eight values in the order of Nibbles::apart: k and k + 4, ...
__device__ __forceinline__ symtile::u32x4 interleave(const symtile::u32x4& x) {
    constexpr uint32_t kLow = 0x05040100u, kHigh = 0x07060302u;
    return symtile::u32x4{__builtin_amdgcn_perm(x[2], x[0], kLow),
                          __builtin_amdgcn_perm(x[2], x[0], kHigh),
                          __builtin_amdgcn_perm(x[3], x[1], kLow),
                          __builtin_amdgcn_perm(x[3], x[1], kHigh)};
}

template <bool BF>
__device__ __forceinline__ f32x4 mfma(symtile::u32x4 a, symtile::u32x4 b, f32x4 c) {
    if constexpr (BF) {
        typedef __bf16 v8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a),
                                                       __builtin_bit_cast(v8, b), c, 0, 0, 0);
    } else {
        typedef _Float16 v8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a),
                                                      __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
}

template <bool BF>
__device__ __forceinline__ float scale_value(uint32_t h) {   // the low half
    if constexpr (BF) return __uint_as_float(h << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)h);
}

// Words of a 4 x 4 transposed between the four quarters of the wave: lane (n, g)
// gets in word j what lane (n, j) had in word g.
__device__ __forceinline__ symtile::u32x4 transpose_quarters(symtile::u32x4 w) {
    const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return symtile::u32x4{c[0], c[1], d[0], d[1]};
}

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef uint8_t u8x8 __attribute__((ext_vector_type(8)));
template <class V>
struct __attribute__((packed, aligned(1))) Unaligned {
    V v;
};

// Scales, and zero points above them, of NT tiles' columns for the groups of CHUNK
// weights from group `group0` on, group by group: a column's are far from the next
// column's in memory and every block needs one of each, so they are read once, along
// the columns.  fetch() asks for them, without a branch, so that loads may follow
// that place() does not wait for; place() puts them into LDS.  Behind the last group
// stand zeros, which meet zeros of X.
template <int GROUP, int NT, int CHUNK, int THREADS>
struct Scales {
    static constexpr int kCols = NT * kTileN, kVec = 8, kGroups = CHUNK / GROUP;
    static constexpr int kVecs = kGroups / kVec;      // 8 groups of a column each
    static constexpr int kMost = (kVecs * kCols + THREADS - 1) / THREADS;
    typedef uint32_t Table[kGroups][kCols];
    u16x8 s[kMost];
    u8x8 z[kMost];

    // Vector i of the thread is the 8 groups from `first` on in column `col`; the
    // last ones of the array come from the 8 before its end (there are 8 columns).
    __device__ __forceinline__ size_t at(const W4Params& p, int n0, int group0, int i, int* col,
                                         int* first) const {
        const int v = threadIdx.x + i * THREADS;
        *col = v / kVecs;
        *first = v % kVecs * kVec;
        const size_t at = (size_t)min(n0 + *col, p.N - 1) * p.groups + group0 + *first;
        const size_t most = (size_t)p.N * p.groups - kVec;
        if (at > most) *first -= (int)(at - most);
        return at > most ? most : at;
    }
    __device__ __forceinline__ void fetch(const W4Params& p, int n0, int group0) {
        // without zero points any bytes of the scales are read in their place
        const uint8_t* zeros = p.zeros ? p.zeros : static_cast<const uint8_t*>(p.scales);
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            int col, first;
            const size_t from = at(p, n0, group0, i, &col, &first);
            s[i] = reinterpret_cast<const Unaligned<u16x8>*>(static_cast<const uint16_t*>(p.scales) +
                                                             from)->v;
            z[i] = reinterpret_cast<const Unaligned<u8x8>*>(zeros + from)->v;
        }
    }
    __device__ __forceinline__ void place(const W4Params& p, int n0, int group0, Table& of) const {
        const int count = p.groups - group0;
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            int col, first;
            at(p, n0, group0, i, &col, &first);
            const int begin = (threadIdx.x + i * THREADS) % kVecs * kVec;
            if (col >= kCols) continue;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const uint32_t zero = p.zeros ? z[i][e] & 15u : 8u;
                if (first + e >= begin && first + e < count) of[first + e][col] = s[i][e] | zero << 16;
                if (begin + e >= count) of[begin + e][col] = 0u;
            }
        }
    }
};

// X of a wave's block in LDS: 256 bytes a row, its 16 vectors of 8 values in an
// order of the row's own (vector v at v ^ (row % 16)), so that a matrix operand's
// load, the same vector of 16 rows, touches every bank once.
template <int MT>
struct StagedX {
    symtile::u32x4 v[16 * MT][16];
};

// What a wave reads X and weights through: buffer resources over X and the tile's
// columns, and each lane's offsets in them.  A block adds the same number to every
// lane's offset, which is the load's scalar operand: no address arithmetic a load.
//
// A lane's piece of a block exists in the blocks before `w_end` (its 32 weights) and
// `x_end` (its 8 values): the others' offsets are set outside of the resource and
// read as zeros, without a branch, so that the loads of several blocks are in
// flight together.  What is behind K is multiplied with zeros of X.
template <int XL>
struct Source {
    symtile::rsrc_t x, w;
    uint32_t at_x[XL], at_w;   // bytes
    int w_end, x_end;

    __device__ __forceinline__ Source(const W4Params& p, int n0) {
        const int lane = threadIdx.x % 64, c = lane % 16, g = lane / 16;
        const int cols = min(kTileN, p.N - n0);
        x = symtile::make_rsrc(p.X, (uint32_t)(((p.M - 1) * p.ldx + p.K) * 2));
        w = symtile::make_rsrc(p.q + (size_t)n0 * (p.K / 2), (uint32_t)(cols * (p.K / 2)));
#pragma unroll
        for (int i = 0; i < XL; ++i)
            at_x[i] = (uint32_t)(min(4 * i + g, p.M - 1) * p.ldx + 8 * c) * 2;
        at_w = (uint32_t)(min(c, cols - 1) * (p.K / 2) + 16 * g);
        w_end = (p.K - 32 * g + kBlockK - 1) / kBlockK;
        x_end = (p.K - 8 * c + kBlockK - 1) / kBlockK;
    }
};

// A block of 128 weights of 16 columns times the rows of X in `staged`, added to
// `total` with the groups' scales: `of_block` points at the first group's in this
// lane's column, `stride` columns before the next group's.  Lane (c = lane % 16,
// g = lane / 16) holds column c's weights 32 g .. 32 g + 31.  With one group a block,
// matrix instruction j takes word j of every lane; with more, the words are transposed
// between the quarters of the wave, so that instruction j has the weights
// 32 j .. 32 j + 31 and a group's are in instructions of their own.  APART: X is in the
// order of Nibbles::apart.
template <bool BF, int MT, int GROUP, bool APART>
__device__ __forceinline__ void multiply_block(f32x4 (&total)[MT], const Nibbles<BF>& q,
                                               const symtile::u32x4& w, const uint32_t* of_block,
                                               int stride, const StagedX<MT>& staged) {
    const int c = threadIdx.x % 16, g = threadIdx.x % 64 / 16;
    const symtile::u32x4 words = GROUP == kBlockK ? w : transpose_quarters(w);
    f32x4 acc[MT];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        symtile::u32x4 xs[MT];
        const int v = GROUP == kBlockK ? 4 * g + j : 4 * j + g;
#pragma unroll
        for (int t = 0; t < MT; ++t) xs[t] = staged.v[16 * t + c][v ^ c];
        const uint32_t of = of_block[j * 32 / GROUP * stride];
        const uint32_t z = Nibbles<BF>::minus_offset(of >> 16);
        const symtile::u32x4 zs = {z, z, z, z};
        const symtile::u32x4 ws = APART ? q.apart(words[j]) : q.adjacent(words[j]);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            f32x4& a = acc[t];
            if (j * 32 % GROUP == 0) a = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            a = mfma<BF>(xs[t], zs, a);
            a = mfma<BF>(xs[t], ws, a);
            if ((j + 1) * 32 % GROUP == 0) {
                const float sc = scale_value<BF>(of & 0xFFFFu);
#pragma unroll
                for (int e = 0; e < 4; ++e) total[t][e] = __builtin_fmaf(sc, a[e], total[t][e]);
            }
        }
    }
}

// Element 4 * lane + i of a tile of sums: column lane % 16, row 4 * (lane / 16) + i.
__device__ __forceinline__ int column_of(int element) { return element / 4 % 16; }
__device__ __forceinline__ int row_of(int element) { return element / 64 * 4 + element % 4; }

template <bool BF>
__device__ __forceinline__ uint16_t rounded(float v) {
    if constexpr (BF) return __builtin_bit_cast(uint16_t, (__bf16)v);
    else return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// The bases of the slots that a wave stores into, asked for where the kernel begins.
template <int WAVES>
__device__ __forceinline__ void slot_bases(const W4Params& p, uint64_t* bases) {
    static_assert(SYMTILE_MAX_WORLD % WAVES == 0 && WAVES <= SYMTILE_MAX_WORLD, "slots by waves");
#pragma unroll
    for (int i = 0; i < SYMTILE_MAX_WORLD / WAVES; ++i)
        bases[i] = p.bases[min((int)threadIdx.x / 64 + i * WAVES, p.world - 1)];
}

// A wave stores rows x 8 `vecs` columns of `out` (row stride `ld` values) into column
// `col` of its slots' blocks and counts them as `tiles` tiles from `tile` on: the
// wave's own stores' acknowledgements are all that its counters have to wait for.
// `bases`: see slot_bases.
template <int WAVES>
__device__ __forceinline__ void store_slots(const W4Params& p, const uint64_t* bases,
                                            const uint16_t* out, int ld, int col, int vecs,
                                            int tile, int tiles) {
    const int lane = threadIdx.x % 64;
#pragma unroll
    for (int i = 0; i < SYMTILE_MAX_WORLD / WAVES; ++i) {
        if ((int)threadIdx.x / 64 + i * WAVES >= p.world) break;
        char* base = reinterpret_cast<char*>(bases[i]);
        const symtile::rsrc_t dst = symtile::make_rsrc(
            base + p.c_off + (size_t)col * 2, (uint32_t)(((size_t)(p.M - 1) * p.ldc + vecs * 8) * 2));
        for (int e = lane; e < p.M * vecs; e += 64) {
            const int m = e / vecs, v = e - m * vecs;
            symtile::buf_st16p<symtile::kStoreWriteThrough>(
                symtile::ld16(out + m * ld + v * 8), dst, (uint32_t)(m * p.ldc + v * 8) * 2, 0);
        }
        symtile::release_written_through();
        if (lane < tiles)
            symtile::flag_signal(reinterpret_cast<uint32_t*>(base + p.flag_off) + tile + lane);
    }
}

// ---- up to 16 rows -----------------------------------------------------------------
// One block of 128 weights of 16 columns in registers, with what it is multiplied by.
// X comes by rows, 256 bytes of four rows a load (XL of them), and takes the matrix
// operands' layout in LDS: loading operands directly reads 64 bytes of 16 rows, whose
// distance is often a power of two, from one cache channel.
template <bool BF, int XL, int GROUP>
struct Block {
    static_assert(XL <= 4, "one tile of 16 rows");
    symtile::u32x4 w;
    symtile::u32x4 x[XL];    // rows 4 i + g, values 8 c .. 8 c + 7

    __device__ __forceinline__ void load(const Source<XL>& s, int block) {
        const int k0 = block * kBlockK;
        w = symtile::buf_ld16p<symtile::kLoadStream>(
            s.w, block < s.w_end ? s.at_w : symtile::kOOB, k0 / 2);
#pragma unroll
        for (int i = 0; i < XL; ++i)
            x[i] = symtile::buf_ld16(s.x, block < s.x_end ? s.at_x[i] : symtile::kOOB, k0 * 2);
    }

    // X in the order of Nibbles::apart: 4 XL instructions a block for 16 fewer on weights.
    __device__ __forceinline__ void multiply(f32x4 (&total)[1], const Nibbles<BF>& q,
                                             const uint32_t* of_block, StagedX<1>& staged) const {
        const int c = threadIdx.x % 16, g = threadIdx.x % 64 / 16;
#pragma unroll
        for (int i = 0; i < XL; ++i)
            staged.v[4 * i + g][c ^ (4 * i + g)] = interleave(x[i]);
        __builtin_amdgcn_wave_barrier();   // the wave reads what its lanes wrote
        multiply_block<BF, 1, GROUP, true>(total, q, w, of_block, kTileN, staged);
        __builtin_amdgcn_wave_barrier();   // the next block's X is written after these reads
    }
};

// One workgroup per 16 columns and up to 4 XL rows; its waves share the blocks of K, in
// pairs, so that a wave reads whole 128-byte lines of its columns.  A wave works on U
// blocks while U to 2 U more are on their way.
//
// Bound by the weights' bytes on a long N (one row through 8192x28672: 33 us, 3.7 TB/s)
// and by latency on a short one (8192x3584: 7.1 us, of which an empty kernel takes 2.9):
// so the loads of the first 2 U blocks are asked for before the scales, whose place in
// LDS is a barrier, and with them the slots' addresses.
template <bool BF, int XL, int GROUP, int U, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 4) w4_kernel(W4Params p) {
    typedef Block<BF, XL, GROUP> B;
    constexpr int kThreads = 64 * WAVES;
    typedef float Partial[256];
    static_assert(sizeof(Partial) <= sizeof(StagedX<1>), "a wave's sums take its X's place");
    __shared__ StagedX<1> staged[WAVES];
    __shared__ __attribute__((aligned(16))) uint16_t out[16][kTileN];
    typedef Scales<GROUP, 1, kChunkK, kThreads> S;
    __shared__ typename S::Table scales;
    const int tile = blockIdx.x, t = threadIdx.x, wave = t / 64, lane = t % 64;
    const int w0 = __builtin_amdgcn_readfirstlane(wave);
    uint64_t bases[SYMTILE_MAX_WORLD / WAVES];
    slot_bases<WAVES>(p, bases);
    f32x4 total[1] = {};
    const Source<XL> src(p, tile * kTileN);
    const Nibbles<BF> nibbles;
    for (int chunk = 0; chunk < p.K; chunk += kChunkK) {
        const int first = chunk / kBlockK;
        const int blocks = (min(p.K, chunk + kChunkK) - chunk + kBlockK - 1) / kBlockK;
        // block u of the wave in the chunk: pairs of blocks, WAVES pairs apart
        auto block_of = [&](int u) { return (u / 2 * WAVES + w0) * 2 + u % 2; };
        B a[U], b[U];
        auto fetch = [&](B (&s)[U], int u0) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = block_of(u0 + u);
                // behind the chunk: a block that does not exist
                s[u].load(src, i < blocks ? first + i : 1 << 20);
            }
        };
        auto use = [&](B (&s)[U], int u0) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = min(block_of(u0 + u), blocks - 1);
                s[u].multiply(total, nibbles, &scales[i * (kBlockK / GROUP)][lane % 16],
                              staged[wave]);
            }
        };
        S s;
        s.fetch(p, tile * kTileN, chunk / GROUP);
        fetch(a, 0);
        fetch(b, U);
        if (chunk) __syncthreads();   // the scales before are used up
        s.place(p, tile * kTileN, chunk / GROUP, scales);
        __syncthreads();
        for (int u = 0; block_of(u) < blocks; u += 2 * U) {
            use(a, u);
            fetch(a, u + 2 * U);
            if (block_of(u + U) >= blocks) break;
            use(b, u + U);
            fetch(b, u + 3 * U);
        }
    }
    // the waves' sums, in the order of the waves
    *reinterpret_cast<f32x4*>(&reinterpret_cast<Partial&>(staged[wave])[4 * lane]) = total[0];
    __syncthreads();
    if (t < 256) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += reinterpret_cast<const Partial&>(staged[w])[t];
        out[row_of(t)][column_of(t)] = rounded<BF>(v);
    }
    __syncthreads();
    store_slots<WAVES>(p, bases, &out[0][0], kTileN, tile * kTileN,
                       p.N - tile * kTileN >= kTileN ? 2 : 1, tile, 1);
}

// ---- up to 64 rows -----------------------------------------------------------------
// A workgroup takes 64 columns: four of its eight waves 16 columns each, the other
// four the same columns' other half of every step of K.  X of a step goes to LDS once
// for all of them.  (Where a workgroup takes 16 columns, every workgroup reads all of
// X: 1 MB for 64 KB of weights with 64 rows of 8192.)  X and weights go straight into
// a ring of stages in LDS, waited for by count, so that later steps' loads stay in
// flight across the barriers; held in registers, the compiler waits for them where
// it moves registers (64 rows through 8192x3584: 19.0 us against 17.9).  Where the
// columns are too few for the GPU, K is split over workgroups; their sums are written
// through to the workspace, and the one that arrives last adds them in the order of K.
//
// 64 rows through 8192x3584 take 17.4 us in the first milliseconds of such calls, 16.2
// after 20 ms: about 8.5 are there whatever K is (the kernel's beginning, the partial
// sums' way through memory, the stores into 8 slots and their acknowledgement); in the K
// loop matrix instructions and LDS reads wait for each other (of the 17.4 us without the
// zero points' matrix instructions 16.0, with a quarter of the reads of X 15.6, without
// both 15.5).  16 rows through 8192x28672: 36 us, 3.5 TB/s of weights.
constexpr int kWideTiles = 4, kWideCols = kWideTiles * kTileN, kWideThreads = 512;
constexpr int kWideGroups = 64;      // groups of a column whose scales are in LDS

// Blocks a step and wave, k of a step, and stages of the ring.
template <int MT>
struct WideStep {
    static constexpr int kBlocks = MT == 2 ? 2 : 1, kK = 2 * kBlocks * kBlockK;
    static constexpr int kStages = MT == 1 ? 3 : 2;
};

// s_waitcnt immediate: at most n vector-memory operations outstanding, no LDS ones
// (gfx9 encoding: vmcnt 3:0 and 15:14, expcnt 6:4, lgkmcnt 11:8).
constexpr int wait_loads(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4); }

template <bool BF, int MT, int GROUP>
__global__ void __launch_bounds__(kWideThreads, MT == 1 ? 4 : 2) w4_wide_kernel(W4Params p) {
    constexpr int CB = WideStep<MT>::kBlocks, kStepK = WideStep<MT>::kK;
    constexpr int kStages = WideStep<MT>::kStages;
    constexpr int XL = CB * MT, kLoads = XL + CB;    // loads of 1 KB a wave and step
    typedef float Partial[kWideTiles][MT][256];
    typedef Scales<GROUP, kWideTiles, kWideGroups * GROUP, kWideThreads> S;
    struct Stage {
        StagedX<MT> x[2 * CB];
        symtile::u32x4 w[kWideThreads / 64][CB][64];
    };
    union Lds {
        Stage ring[kStages];
        struct {
            Partial sums;
            uint16_t out[16 * MT][kWideCols];
        } end;
    };
    __shared__ __attribute__((aligned(16))) Lds lds;
    __shared__ typename S::Table scales;
    const int t = threadIdx.x, lane = t % 64, c = lane % 16, g = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(t / 64), tile = wave % kWideTiles;
    const int half = wave / kWideTiles;
    const int group = blockIdx.x / p.splits, split = blockIdx.x - group * p.splits;
    const int n0 = group * kWideCols, cols = min(kWideCols, p.N - n0);
    const int steps = (p.K + kStepK - 1) / kStepK;
    const int first = split * p.part_steps, end = min(steps, first + p.part_steps);
    const int end_k = min(p.K, end * kStepK);
    uint64_t bases[1];
    slot_bases<kWideThreads / 64>(p, bases);

    const symtile::i32x4_t xr =
        symtile::make_rsrc_words(p.X, (uint32_t)(((p.M - 1) * p.ldx + p.K) * 2));
    const symtile::i32x4_t wr =
        symtile::make_rsrc_words(p.q + (size_t)n0 * (p.K / 2), (uint32_t)(cols * (p.K / 2)));
    // The lane's vector of weights in block i of the wave's half of a step, and of X in
    // the wave's loads: load u fills four rows of one block of LDS, whose place c
    // holds the row's vector c ^ (row % 16).
    const uint32_t at_w = (uint32_t)(min(tile * kTileN + c, cols - 1) * (p.K / 2) + 16 * g) +
                          half * CB * (kBlockK / 2);
    const int k_w = half * CB * kBlockK + 32 * g;
    uint32_t at_x[XL], to_x[XL];
    int k_x[XL];
#pragma unroll
    for (int u = 0; u < XL; ++u) {
        const int load = wave + u * (kWideThreads / 64), block = load / (4 * MT);
        const int row = load % (4 * MT) * 4 + g;
        k_x[u] = block * kBlockK + 8 * (c ^ row % 16);
        at_x[u] = (uint32_t)(min(row, p.M - 1) * p.ldx + k_x[u]) * 2;
        to_x[u] = (uint32_t)(load * 1024);
    }
    const uint32_t lds0 = symtile::lds_addr(&lds);
    const uint32_t to_w = (uint32_t)(offsetof(Stage, w) + wave * CB * 1024);
    // what is behind the part's end is read from outside of the resources: zeros
    auto load = [&](int step, int stage) {
        const int k0 = step * kStepK;
        const uint32_t to = lds0 + stage * (uint32_t)sizeof(Stage);
#pragma unroll
        for (int i = 0; i < CB; ++i)
            symtile::buf_ld16_lds_async(
                wr, to + to_w + i * 1024,
                (at_w + i * (kBlockK / 2)) | ((uint32_t)(end_k - 1 - k0 - k_w - i * kBlockK) & symtile::kOOB),
                k0 / 2);
#pragma unroll
        for (int u = 0; u < XL; ++u)
            symtile::buf_ld16_lds_async(
                xr, to + to_x[u], at_x[u] | ((uint32_t)(end_k - 1 - k0 - k_x[u]) & symtile::kOOB), k0 * 2);
    };
    f32x4 total[MT] = {};
    const Nibbles<BF> nibbles;
    if (first < end) {
        S s;
        s.fetch(p, n0, first * (kStepK / GROUP));
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) load(first + i, i);
        s.place(p, n0, first * (kStepK / GROUP), scales);
        int stage = 0, next = kStages - 1;
        constexpr int kTableSteps = kWideGroups * GROUP / kStepK;   // whose scales are in LDS
        for (int base = first; base < end; base += kTableSteps) {
            if (base != first) {
                s.fetch(p, n0, base * (kStepK / GROUP));
                __syncthreads();   // the scales before are used up
                s.place(p, n0, base * (kStepK / GROUP), scales);
            }
            const int stop = min(end, base + kTableSteps);
            for (int step = base; step < stop; ++step) {
                // this step's loads are there, for all waves; the step's before is used up
                __builtin_amdgcn_s_waitcnt(wait_loads((kStages - 2) * kLoads));
                asm volatile("" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                load(step + kStages - 1, next);
                const Stage& now = lds.ring[stage];
#pragma unroll
                for (int i = 0; i < CB; ++i) {
                    const int block = half * CB + i;
                    const int of = ((step - base) * 2 * CB + block) * (kBlockK / GROUP);
                    multiply_block<BF, MT, GROUP, false>(total, nibbles, now.w[wave][i][lane],
                                                         &scales[of][tile * kTileN + c],
                                                         kWideCols, now.x[block]);
                }
                stage = stage + 1 == kStages ? 0 : stage + 1;
                next = next + 1 == kStages ? 0 : next + 1;
            }
        }
        // the ring's place is the sums' from here on
        __builtin_amdgcn_s_waitcnt(wait_loads(0));
        __syncthreads();
    }
    // the two halves' sums
    if (half == 1) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
            *reinterpret_cast<f32x4*>(&lds.end.sums[tile][i][4 * lane]) = total[i];
    }
    __syncthreads();
    if (half == 0) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
            total[i] += *reinterpret_cast<const f32x4*>(&lds.end.sums[tile][i][4 * lane]);
    }
    if (p.splits > 1) {
        // [column group][split][tile][row tile][4 * lane + i]
        constexpr int kPart = kWideTiles * MT * 256;
        float* mine = p.partials + ((size_t)blockIdx.x * kWideTiles + tile) * MT * 256;
        const symtile::rsrc_t to = symtile::make_rsrc(mine, MT * 1024);
        if (half == 0) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
                symtile::buf_st16p<symtile::kStoreWriteThrough>(
                    __builtin_bit_cast(symtile::u32x4, total[i]), to, (uint32_t)(i * 1024 + lane * 16), 0);
        }
        symtile::wg_stores_done();
        if (t == 0) {
            symtile::release_written_through();
            const uint32_t before = symtile::atomic_add<__ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT>(
                p.counters + group, 1u);
            const bool last = before == (uint32_t)p.splits - 1;
            scales[0][0] = last;   // (the scales are used up)
            if (last)
                __hip_atomic_store(symtile::global_ptr(p.counters + group), 0u, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!scales[0][0]) return;
        symtile::acquire_coherent_reads();
        if (half == 0) {
            const symtile::rsrc_t from = symtile::make_rsrc(
                p.partials + ((size_t)group * p.splits * kWideTiles + tile) * MT * 256,
                (uint32_t)(((p.splits - 1) * kPart + MT * 256) * 4));
#pragma unroll
            for (int i = 0; i < MT; ++i) total[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            // four parts' loads in flight together; parts that are not there are zeros
            for (int s0 = 0; s0 < p.splits; s0 += 4) {
                f32x4 part[4][MT];
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int i = 0; i < MT; ++i)
                        part[s][i] = __builtin_bit_cast(
                            f32x4, symtile::buf_ld16p<symtile::kLoadCoherent>(
                                       from,
                                       s0 + s < p.splits ? (uint32_t)(i * 1024 + lane * 16)
                                                         : symtile::kOOB,
                                       (s0 + s) * kPart * 4));
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int i = 0; i < MT; ++i) total[i] += part[s][i];
            }
        }
    }
    if (half == 0) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                lds.end.out[16 * i + 4 * g + e][tile * kTileN + c] = rounded<BF>(total[i][e]);
    }
    __syncthreads();
    store_slots<kWideThreads / 64>(p, bases, &lds.end.out[0][0], kWideCols, n0, cols / 8,
                                   group * kWideTiles, (cols + kTileN - 1) / kTileN);
}

// ---- host ------------------------------------------------------------------------------
struct Build {
    const void* kernel;
    int waves, tiles;   // waves and tiles of a workgroup
    int step_k;         // of the wide kernel; 0 = the other one
};
template <bool BF, int XL, int GROUP, int U, int WAVES>
Build build_of() {
    return {reinterpret_cast<const void*>(&w4_kernel<BF, XL, GROUP, U, WAVES>), WAVES, 1, 0};
}
template <bool BF, int MT, int GROUP>
Build wide_of() {
    return {reinterpret_cast<const void*>(&w4_wide_kernel<BF, MT, GROUP>), kWideThreads / 64,
            kWideTiles, WideStep<MT>::kK};
}

// Up to 4 rows: one tile a workgroup, of 8 waves while every tile has a CU of its own
// (8192x3584, 224 tiles: 7.1 us against 9.0 with 4), else of 4, so that more
// workgroups overlap their beginnings and ends (8192x28672: 33 against 35 us with 8;
// 8192x5120, 320 tiles: the same).  Up to 16 rows the 8 waves too while every tile has
// a CU (8192x3584: 10.2 us against the wide kernel's 11.7, 4096x1024 5.6 against 9.6),
// not beyond (8192x5120: 17.7 against 12.1).
template <bool BF, int GROUP>
Build build_for(int M, int tiles, int cus) {
    if (M <= 4)
        return tiles > cus ? build_of<BF, 1, GROUP, 2, 4>()
                                : build_of<BF, 1, GROUP, 2, 8>();
    if (M <= 16 && tiles <= cus) return build_of<BF, 4, GROUP, 1, 8>();
    if (M <= 16) return wide_of<BF, 1, GROUP>();
    if (M <= 32) return wide_of<BF, 2, GROUP>();
    return wide_of<BF, 4, GROUP>();
}
template <bool BF>
Build build_for(int M, int group, int tiles, int cus) {
    return group == 128  ? build_for<BF, 128>(M, tiles, cus)
           : group == 64 ? build_for<BF, 64>(M, tiles, cus)
                         : build_for<BF, 32>(M, tiles, cus);
}

int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Parts that K is split into: as many as give every CU one workgroup, of two steps at
// least (a part's way through memory costs 3 us).
int splits_of(int cus, const Build& b, int N, int K) {
    if (!b.step_k) return 1;
    const int groups = ceil_div(N, kWideCols), steps = ceil_div(K, b.step_k);
    if (groups > symtile_host::kWorkspaceCounters) return 1;
    return std::max(1, std::min(cus / groups, steps / 2));
}

// Counters, one per group of columns, then the partial sums.
constexpr size_t kCounterBytes = (size_t)symtile_host::kWorkspaceCounters * 4;

size_t workspace_bytes_of(const Build& b, int splits, int M, int N) {
    if (splits <= 1) return 0;
    const size_t rows = M <= 16 ? 16 : M <= 32 ? 32 : 64;
    return kCounterBytes + (size_t)ceil_div(N, kWideCols) * splits * rows * kWideCols * 4;
}

// What the calls refuse about sizes.
symtile_status check_sizes(int M, int N, int K, int group) {
    using symtile_host::fail;
    if (M < 0 || N < 0 || K < 0) return fail(SYMTILE_EINVAL, "negative size");
    if (M > SYMTILE_W4_TILE_M)
        return fail(SYMTILE_EUNSUPPORTED, "M exceeds " + std::to_string(SYMTILE_W4_TILE_M) + " tokens");
    if (group != 32 && group != 64 && group != 128)
        return fail(SYMTILE_EINVAL, "group must be 32, 64 or 128");
    if (K % 32 || N % 8) return fail(SYMTILE_EINVAL, "K must be a multiple of 32, N_local of 8");
    if ((size_t)K * kWideCols / 2 >= size_t(1) << 31)
        return fail(SYMTILE_EINVAL, "64 columns of weights exceed 2 GiB");
    return SYMTILE_OK;
}

}  // namespace

extern "C" symtile_status symtile_w4_workspace_bytes(int device, int M, int N_local, int K,
                                                     int group, size_t* bytes) {
    if (!bytes) return symtile_host::fail(SYMTILE_EINVAL, "bytes is NULL");
    *bytes = 0;
    if (symtile_status st = check_sizes(M, N_local, K, group)) return st;
    const int cus = symtile_host::cu_count(device);
    if (cus <= 0)
        return symtile_host::fail(SYMTILE_EINVAL, "device " + std::to_string(device) + " out of range");
    if (M == 0 || N_local == 0) return SYMTILE_OK;
    const Build b = build_for<true>(M, group, ceil_div(N_local, kTileN), cus);
    *bytes = workspace_bytes_of(b, splits_of(cus, b, N_local, K), M, N_local);
    return SYMTILE_OK;
}

extern "C" symtile_status symtile_w4_all_scatter(
    symtile_heap* h, const void* X, const uint8_t* q, const void* scales, const uint8_t* zeros,
    void* C_gathered_local, uint32_t* arrived_local, int M, int N_local, int K, int ldx, int group,
    int dtype, int rank, int world_size, void* workspace, size_t workspace_bytes,
    symtile_stream s) {
    using symtile_host::fail;
    if (!h) return fail(SYMTILE_EINVAL, "heap is NULL");
    if (dtype != SYMTILE_F16 && dtype != SYMTILE_BF16)
        return fail(SYMTILE_EUNSUPPORTED, "dtype must be SYMTILE_F16 or SYMTILE_BF16");
    if (world_size != h->world) return fail(SYMTILE_EINVAL, "world_size differs from the heap's");
    if (rank < 0 || rank >= world_size) return fail(SYMTILE_EINVAL, "rank out of range");
    if (symtile_status st = check_sizes(M, N_local, K, group)) return st;
    if (ldx == 0) ldx = K;
    if (ldx % 8 || ldx < K) return fail(SYMTILE_EINVAL, "ldx must be a multiple of 8 and >= K");
    if ((size_t)M * ldx * 2 >= size_t(1) << 31) return fail(SYMTILE_EINVAL, "X exceeds 2 GiB");
    if (M == 0 || N_local == 0) return SYMTILE_OK;
    if (!C_gathered_local || !arrived_local || (K && (!X || !q || !scales)))
        return fail(SYMTILE_EINVAL, "NULL pointer");
    auto misaligned = [](const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; };
    if (misaligned(X, 16) || misaligned(q, 16) || misaligned(C_gathered_local, 16) ||
        misaligned(arrived_local, 4) || misaligned(scales, 2) || misaligned(workspace, 16))
        return fail(SYMTILE_EINVAL,
                    "X, q, C and the workspace must be 16-byte aligned, counters 4, scales 2");
    const int tiles = ceil_div(N_local, kTileN);
    const size_t ldc = (size_t)world_size * N_local;
    const size_t c_bytes = (size_t)M * ldc * 2;
    const size_t flag_bytes = (size_t)world_size * tiles * 4;
    if (c_bytes >= size_t(1) << 31) return fail(SYMTILE_EINVAL, "the gathered output exceeds 2 GiB");
    if (!symtile_host::in_slot(h, C_gathered_local, c_bytes, rank))
        return fail(SYMTILE_EINVAL, "C_gathered_local [M, world*N_local] not inside slot of rank");
    if (!symtile_host::in_slot(h, arrived_local, flag_bytes, rank))
        return fail(SYMTILE_EINVAL, "arrived_local not inside slot of rank");
    const uint64_t c0 = reinterpret_cast<uint64_t>(C_gathered_local);
    const uint64_t f0 = reinterpret_cast<uint64_t>(arrived_local);
    if (c0 < f0 + flag_bytes && f0 < c0 + c_bytes)
        return fail(SYMTILE_EINVAL, "arrived_local overlaps C_gathered_local");
    const int cus = std::max(1, symtile_host::cu_count(h->device));
    const Build build = dtype == SYMTILE_BF16 ? build_for<true>(M, group, tiles, cus)
                                              : build_for<false>(M, group, tiles, cus);
    int splits = workspace ? splits_of(cus, build, N_local, K) : 1;
    const size_t need = workspace_bytes_of(build, splits, M, N_local);
    if (workspace && workspace_bytes < need)
        return fail(SYMTILE_EINVAL, "workspace of " + std::to_string(need) + " bytes needed");

    W4Params p{};
    p.X = X;
    p.q = q;
    p.scales = scales;
    p.zeros = zeros;
    p.bases = h->dev_bases;
    p.c_off = c0 - h->host_bases[rank] + (size_t)rank * N_local * 2;
    p.flag_off = f0 - h->host_bases[rank] + (size_t)rank * tiles * 4;
    p.M = M;
    p.N = N_local;
    p.K = K;
    p.ldx = ldx;
    p.groups = ceil_div(K, group);
    p.world = world_size;
    p.ldc = (int)ldc;
    p.part_steps = build.step_k ? ceil_div(ceil_div(K, build.step_k), splits) : 0;
    if (p.part_steps) splits = ceil_div(ceil_div(K, build.step_k), p.part_steps);   // none empty
    p.splits = splits;
    if (splits > 1) {
        p.counters = static_cast<uint32_t*>(workspace);
        p.partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterBytes);
    }
    int prev = -1;
    if (symtile_status st = symtile_host::set_device(h, &prev)) return st;
    void* args[] = {&p};
    const unsigned wgs = (unsigned)ceil_div(tiles, build.tiles) * (unsigned)splits;
    hipError_t e = hipLaunchKernel(build.kernel, dim3(wgs), dim3(64 * build.waves), args, 0,
                                   static_cast<hipStream_t>(s));
    if (e == hipSuccess) e = hipGetLastError();
    if (prev >= 0) (void)hipSetDevice(prev);
    return e == hipSuccess ? SYMTILE_OK : symtile_host::hip_fail(e, "w4_kernel launch");
}
