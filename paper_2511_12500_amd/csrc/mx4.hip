// Matrices in blocks of 32 values along a row that share a power of two and hold
// 4-bit floating-point elements: quantisation, and the product of two of them stored
// into every slot of the heap (the All-Scatter of Section 4.2.1).
//
// Element codes are sign, two bits of exponent and one of fraction: 0, 1/2, 1, 3/2, 2,
// 3, 4, 6 and their negatives.  A block's byte b stands for 2^(b - 127), 255 for NaN.
//   C[m, n] = sum_blocks 2^(bx + bw - 254) sum_32 x w.
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <string>

#include "logits_rows.h"
#include "symtile.h"
#include "symtile_device.h"
#include "symtile_internal.h"

namespace {

using logits::Elem;
using symtile::u32x4;

constexpr int kBlock = 32;          // values that share a scale
constexpr int kTileM = SYMTILE_MX4_TILE_M, kTileN = SYMTILE_MX4_TILE_N;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// ---- quantisation ---------------------------------------------------------------------
struct QuantiseParams {
    const void* x;
    uint8_t* q;
    uint8_t* scales;
    void* values;
    size_t ld, ld_values;
    int row0, pieces, row_pieces;        // pieces of 8 values, of a row
    symtile_host::Div by_row;
};

// Eight values, 16 or 32 bytes at any multiple of the element size.
template <int DT>
struct Eight {
    static constexpr int kVecs = 8 / Elem<DT>::kVec;
    u32x4 v[kVecs];
    __device__ __forceinline__ void load(const typename Elem<DT>::type* p) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = logits::load16(p + i * Elem<DT>::kVec);
    }
    __device__ __forceinline__ float operator[](int e) const {
        return logits::element<DT>(v[e / Elem<DT>::kVec], e % Elem<DT>::kVec);
    }
};

// A thread takes 8 values, a quad of lanes a block: its largest magnitude's exponent less
// two is the shared one, so the largest element is below 8 times it and those beyond 6
// become 6.  The conversion rounds to nearest even and saturates.  Bound by memory: 28672 x
// 8192 fp32 with values (2.0 GB) 331 to 348 us, 5.8 TB/s, where a large copy reaches 5.0; 4096 x
// 8192 bf16 17 us, 4.9; 64 rows 2.8, a launch.
template <int DT>
__global__ void __launch_bounds__(256) mx4_quantise_kernel(QuantiseParams p) {
    typedef typename Elem<DT>::type T;
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= p.pieces) return;                    // (whole quads: a row holds whole blocks)
    const int r = p.by_row(i);
    const size_t row = (size_t)p.row0 + r;
    const int at = i - r * p.row_pieces;
    Eight<DT> x;
    x.load(static_cast<const T*>(p.x) + row * p.ld + (size_t)at * 8);
    // magnitudes as whole numbers: a NaN is above all others
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    most = max(most, (uint32_t)__builtin_amdgcn_mov_dpp(most, 0xB1, 0xF, 0xF, true));
    most = max(most, (uint32_t)__builtin_amdgcn_mov_dpp(most, 0x4E, 0xF, 0xF, true));
    const uint32_t field = most >> 23;            // the exponent's, 0 below the normal numbers
    const bool finite = field < 255;
    const uint32_t byte = !finite ? 255u : field > 2 ? field - 2 : 0u;
    const float unit = __uint_as_float(byte ? byte << 23 : 0x00400000u);
    uint32_t code = 0;
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0], x[1], unit, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2], x[3], unit, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4], x[5], unit, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6], x[7], unit, 3);
    if (!finite) code = 0;
    const size_t piece = row * p.row_pieces + at;
    reinterpret_cast<uint32_t*>(p.q)[piece] = code;
    if (i % 4 == 0) p.scales[piece / 4] = (uint8_t)byte;
    if (p.values) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t c = code >> (4 * e);
            // 2 + fraction, or the fraction alone, in halves; times 2^(exponent - 1)
            const uint32_t ex = c >> 1 & 3, fr = c & 1;
            const float half = ex ? (float)((2 + fr) << (ex - 1)) : (float)fr;
            const float v = finite ? half * (0.5f * unit) : __builtin_nanf("");
            f[e] = c & 8 ? -v : v;
        }
        T* to = static_cast<T*>(p.values) + row * p.ld_values + (size_t)at * 8;
        if constexpr (DT == SYMTILE_F32) {
            logits::store16(to, logits::pack<DT>(f));
            logits::store16(to + 4, logits::pack<DT>(f + 4));
        } else {
            logits::store16(to, logits::pack<DT>(f));
        }
    }
}

// ---- product ----------------------------------------------------------------------------
struct ProductParams {
    const uint8_t *x, *x_scales, *w, *w_scales;
    const uint64_t* bases;
    uint64_t c_off, flag_off;   // of the rank's column block and its counters in a slot
    int M, N, groups, world;    // groups: blocks of a row
    size_t ldc;                 // elements
    int tiles_n;                // of the counters
    // of the kernel for many rows: its tiles, and how they and their parts are numbered
    int gm, per_xcd, xcd_rest;
    int band;                   // tiles of a band
    symtile_host::Div by_band;
    // K in `splits` parts of `part_stages` stages each (the last may have fewer), whose sums
    // meet in `partials`
    int splits, part_stages;
    symtile_host::Div by_splits;
    uint32_t* counters;
    float* partials;
};

// Tile and part b of the grid.  Workgroups go to the 8 XCDs in turn; each takes tiles next
// to each other, in bands of kBandRows tile rows, so that those that run together share
// rows of both matrices in its L2.  A tile's parts are next to each other too.
constexpr int kXcds = 8, kBandRows = 8;
__device__ __forceinline__ int place_tile(const ProductParams& p, int b, int* tm, int* tn,
                                          int* split) {
    const int xcd = b % kXcds, i = b / kXcds;
    const int unit = xcd * p.per_xcd + min(xcd, p.xcd_rest) + i, id = p.by_splits(unit);
    *split = unit - id * p.splits;
    const int band = p.by_band(id), first = band * kBandRows, in = id - band * p.band;
    const int height = min(kBandRows, p.gm - first);
    const int n = height == kBandRows ? in / kBandRows : in / height;
    *tm = first + in - n * height;
    *tn = n;
    return id;
}

struct __attribute__((packed, aligned(1))) Unaligned16 {
    u32x4 v;
};

// The scales of blocks first .. first + 15 of a row, zeros behind its end (which meet zeros
// of both matrices; a neighbour row's byte there may be a NaN's).
__device__ __forceinline__ u32x4 scales16(const uint8_t* scales, size_t rows, size_t row,
                                          int groups, int first) {
    const size_t at = row * groups + first, total = rows * groups;
    const int valid = groups - first;
    u32x4 r = {0u, 0u, 0u, 0u};
    if (at + 16 <= total) {
        r = reinterpret_cast<const Unaligned16*>(scales + at)->v;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int keep = valid - 4 * j;
            if (keep < 4) r[j] = keep <= 0 ? 0u : r[j] & ((1u << (8 * keep)) - 1u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < valid) r[j / 4] |= (uint32_t)scales[at + j] << (8 * (j % 4));
    }
    return r;
}

// 16 rows of `a` by 16 rows of `b`, 128 values each: lane (c = lane % 16, g = lane / 16)
// holds block g of row c of both, and the scale's byte.
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, f32x4 c, uint32_t sa,
                                        uint32_t sb) {
    const i32x8 va = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const i32x8 vb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, c, 4, 4, 0, (int)sa, 0,
                                                            (int)sb);
}

template <bool BF>
__device__ __forceinline__ uint16_t rounded(float v) {
    if constexpr (BF) return __builtin_bit_cast(uint16_t, (__bf16)v);
    else return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// A workgroup takes 16 columns and up to 64 rows (over 32 only where there is next to nothing to
// sum: K = 0, or a matrix of fewer than 16 scales); its waves share the chunks of 512 values,
// whose 16-byte blocks go from memory to the operands' registers, and add their sums through
// LDS.  Bound by latency: one round of loads, the waves' sums, the stores' acknowledgement and
// the counters follow each other (1 x 8192 x 3584 into 8 slots, 15.7 MB: 6.2 us of which 2.9 are
// an empty kernel's; 16 rows 7.8).
template <bool BF, int MT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) mx4_kernel(ProductParams p) {
    __shared__ float sums[WAVES][MT][256];
    __shared__ __attribute__((aligned(16))) uint16_t out[16 * MT][kTileN];
    const int t = threadIdx.x, lane = t % 64, c = lane % 16, g = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(t / 64);
    const int tn = blockIdx.x, tm = blockIdx.y, n0 = tn * kTileN, m0 = tm * kTileM;
    const int cols = min(kTileN, p.N - n0), rows = min(kTileM, p.M - m0);
    const int row_bytes = p.groups * (kBlock / 2);
    const symtile::rsrc_t ws =
        symtile::make_rsrc(p.w + (size_t)n0 * row_bytes, (uint32_t)(cols * row_bytes));
    const symtile::rsrc_t xs =
        symtile::make_rsrc(p.x + (size_t)m0 * row_bytes, (uint32_t)(rows * row_bytes));
    const int wc = min(c, cols - 1);
    const uint64_t slot_base = p.bases[min(wave, p.world - 1)];
    f32x4 total[MT] = {};
    for (int first = wave * 16; first < p.groups; first += WAVES * 16) {
        const u32x4 sw = scales16(p.w_scales, p.N, n0 + wc, p.groups, first);
        u32x4 sx[MT], w[4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
            sx[i] = scales16(p.x_scales, p.M, m0 + min(16 * i + c, rows - 1), p.groups, first);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int b = 4 * s + g;
            w[s] = symtile::buf_ld16(ws, first + b < p.groups ? (uint32_t)(wc * row_bytes + b * 16)
                                                              : symtile::kOOB, first * 16);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int b = 4 * s + g;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const u32x4 x = symtile::buf_ld16(
                    xs, first + b < p.groups
                            ? (uint32_t)(min(16 * i + c, rows - 1) * row_bytes + b * 16)
                            : symtile::kOOB, first * 16);
                total[i] = mfma16(x, w[s], total[i], sx[i][s] >> (8 * g), sw[s] >> (8 * g));
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) *reinterpret_cast<f32x4*>(&sums[wave][i][4 * lane]) = total[i];
    __syncthreads();
    // element 4 * lane + e: column lane % 16, row 4 * (lane / 16) + e
    for (int e = t; e < MT * 256; e += 64 * WAVES) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += sums[w][e / 256][e % 256];
        out[e / 256 * 16 + e % 256 / 64 * 4 + e % 4][e / 4 % 16] = rounded<BF>(v);
    }
    __syncthreads();
    static_assert(WAVES >= SYMTILE_MAX_WORLD, "a slot a wave");
    if (wave < p.world) {
        char* base = reinterpret_cast<char*>(slot_base);
        const int vecs = cols / 8;
        const symtile::rsrc_t dst = symtile::make_rsrc(
            base + p.c_off + ((size_t)m0 * p.ldc + n0) * 2,
            (uint32_t)(((size_t)(rows - 1) * p.ldc + cols) * 2));
        for (int e = lane; e < rows * vecs; e += 64) {
            const int m = vecs == 2 ? e >> 1 : e, v = vecs == 2 ? e & 1 : 0;
            symtile::buf_st16p<symtile::kStoreWriteThrough>(
                symtile::ld16(&out[m][v * 8]), dst, (uint32_t)(m * p.ldc + v * 8) * 2, 0);
        }
        symtile::release_written_through();
        if (lane == 0)
            symtile::flag_signal(reinterpret_cast<uint32_t*>(base + p.flag_off) +
                                 (size_t)tm * p.tiles_n + tn);
    }
}

// ---- many rows ----------------------------------------------------------------------------
typedef float f32x16 __attribute__((ext_vector_type(16)));

// 32 rows of `a` by 32 rows of `b`, 64 values each: lane (r = lane % 32, g = lane / 32)
// holds a block of row r of both.  Byte S of sa and sb are its scales.
template <int S>
__device__ __forceinline__ f32x16 mfma32(const u32x4& a, const u32x4& b, f32x16 c, uint32_t sa,
                                         uint32_t sb) {
    const i32x8 va = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const i32x8 vb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(va, vb, c, 4, 4, S, (int)sa, S, (int)sb);
}

// s_waitcnt immediate: at most n vector-memory operations outstanding, no LDS ones
// (gfx9 encoding: vmcnt 3:0 and 15:14, expcnt 6:4, lgkmcnt 11:8).
constexpr int wait_loads(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4); }

// Written through (sc0 sc1) with the streaming hint (nt): the acknowledgement is the same,
// and lines that nobody on this GPU reads soon leave the caches first (4096 x 8192 x 3584
// into 8 slots 105.5 us, without the hint 112.9; 28672 columns into one 481, 491).
constexpr int kStoreThroughStream = symtile::kStoreWriteThrough | symtile::kStoreNonTemporal;

// At most N of the wave's loads are out, its LDS accesses done, and so for all waves.
template <int N>
__device__ __forceinline__ void meet() {
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (0 << 8));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A workgroup of 4 waves, 2 x 2, takes TM rows of X by TN of W.  K goes by stages of 256 values,
// 128 bytes a row, loaded straight into one of two buffers in LDS while the other is
// multiplied; row r's 16-byte vector v lies at place v ^ (r / 2 % 8), so that 16 rows' same
// vector touch every bank once.  (Stages of 64 bytes a row and four buffers: 513 us for
// 4096 x 8192 x 28672, since a CU has only so many requests out, of 64 bytes each then.)
// In instruction S of a stage's four lane half g takes block 4 g + S of its rows, so a
// lane's scales of a stage are one word; scales come for two stages (a pair), 16 bytes a
// row, straight into LDS too where rows of scales are whole numbers of 16 aligned bytes
// (ALIGNED: K a multiple of 512), else through registers, one pair ahead (K = 8160 where 8192 takes
// the first time: 64 x K x 3584 into 8 slots 13.2 us and 10.9, 128 x K x 28672 73 and 49, 4096 x K x
// 28672 617 and 495, x 3584 into 8 slots 115 and 104).
//   256 x 256, 2 stages: each 32 x 32 x 64 operand read feeds 4 instructions, and the 256
// accumulators fill the AGPRs of one wave a SIMD.  4096 x 8192 x 28672 in 485 to 495 us, 3.9
// PFLOP/s, with inputs in turn (the first calls after a pause 517; on the same inputs 459); without
// its loads 376 where this took 475.  Power bounds it: matrix units that are busy all the time, from
// registers alone, run at 1.35 to 1.4 GHz on random data (as many instructions at that rate, 5.6
// PFLOP/s, 343 us; 229 at full clock), and here they are busy for half of the cycles.  So hiding
// more did not help: lines asked for into L2 three stages ahead, by the CUs that share them, took
// 474 us where this took 475 (on zeros 361 and 417), one workgroup a CU that goes through tiles with
// the next one's loads ahead of the stores 484 where this took 484, and tiles of 256 x 128, which
// move more, 644.  Into 8 slots, 4096 x 8192 x 3584, 104 us: 59 to the end of K, 235 MB of stores
// behind it, since all tiles run at once.
//   64 x 64, 4 stages, K in parts: 64 x 8192 x 3584 into 8 slots 10.1 to 11 us, 16 MB of weights and
// X read and 7.4 MB written; latency: loads, parts to memory and back, stores.
constexpr int kStageBytes = 128;
template <int TM, int TN, int RING>
struct GemmLds {
    static constexpr int kPairs = RING / 2 + 1;
    struct Stage {
        uint8_t w[TN * kStageBytes], x[TM * kStageBytes];
    };
    union {
        Stage stage[RING];
        uint16_t out[TM * TN];
    };
    u32x4 scales[kPairs][TN + TM];
    int last;
};

template <bool BF, int TM, int TN, int RING, bool ALIGNED>
__global__ void __launch_bounds__(256, sizeof(GemmLds<TM, TN, RING>) > 80 * 1024 ? 1 : 2)
mx4_gemm_kernel(ProductParams p) {
    constexpr bool kSplits = TM * TN == 64 * 64;     // the build whose calls may split K
    typedef GemmLds<TM, TN, RING> Lds;
    __shared__ __attribute__((aligned(16))) Lds lds;
    constexpr int kMT = TM / 64, kNT = TN / 64;           // 32 x 32 tiles of a wave
    constexpr int kRows = TN + TM, kLoads = kRows / 32;   // loads of 8 rows a wave and stage
    constexpr int kScaleLoads = (kRows + 255) / 256;
    const int t = threadIdx.x, lane = t % 64, r = lane % 32, g = lane / 32;
    const int wave = __builtin_amdgcn_readfirstlane(t / 64), wn = wave % 2, wm = wave / 2;
    int tm, tn, split;
    const int tile = place_tile(p, blockIdx.x, &tm, &tn, &split);
    const int m0 = tm * TM, n0 = tn * TN;
    const int rows = min(TM, p.M - m0), cols = min(TN, p.N - n0);
    const int row_bytes = p.groups * (kBlock / 2);
    // the part's stages from `first` on, and the blocks before its end
    const int first = split * p.part_stages;
    const int stages = min((p.groups + 7) / 8 - first, p.part_stages);
    const int end = min(p.groups, (first + stages) * 8);
    const symtile::i32x4_t ws = symtile::make_rsrc_words(p.w + (size_t)n0 * row_bytes,
                                                         (uint32_t)(cols * row_bytes));
    const symtile::i32x4_t xs = symtile::make_rsrc_words(p.x + (size_t)m0 * row_bytes,
                                                         (uint32_t)(rows * row_bytes));
    const uint32_t lds0 = symtile::lds_addr(&lds);
    // A load fills 8 rows, lane l place l % 8 of row l / 8, of the first or second 8 of 16.
    const int vec[2] = {(lane % 8) ^ (lane / 16), (lane % 8) ^ (4 + lane / 16)};
    const uint32_t row_at = (uint32_t)(lane / 8 * row_bytes);
    // Load u of the wave's for stage st of the part into buffer `slot` (behind the part's end:
    // outside of the resources, zeros).
    auto load = [&](int st_, int slot, int u) {
        const int st = first + st_, v = vec[u % 2] * 16;
        const uint32_t from = st * kStageBytes + v < end * 16 ? row_at + v : symtile::kOOB;
        const uint32_t to = lds0 + slot * (uint32_t)sizeof(typename Lds::Stage);
        if (u < TN / 32) {
            const int row = (wave * (TN / 32) + u) * 8;
            symtile::buf_ld16_lds_async(ws, to + row * kStageBytes, from,
                                        (uint32_t)(row * row_bytes + st * kStageBytes));
        } else {
            const int row = (wave * (TM / 32) + u - TN / 32) * 8;
            symtile::buf_ld16_lds_async(xs, to + (TN + row) * kStageBytes, from,
                                        (uint32_t)(row * row_bytes + st * kStageBytes));
        }
    };
    // Scales of two stages (a pair) for the rows of W and X, those of the last ones again for
    // the rows that are not there.
    symtile::i32x4_t scale_rsrc[kScaleLoads];
    uint32_t scale_at[kScaleLoads];
    u32x4 sc[kScaleLoads];
    int shift[kScaleLoads];
    const uint8_t *scales_of[kScaleLoads], *scales_end[kScaleLoads];
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        if constexpr (ALIGNED) {
            const int row = (i * 4 + wave) * 64;      // 64 of one matrix
            const bool of_w = row < TN;
            scale_rsrc[i] = of_w ? symtile::make_rsrc_words(p.w_scales + (size_t)n0 * p.groups,
                                                            (uint32_t)(cols * p.groups))
                                 : symtile::make_rsrc_words(p.x_scales + (size_t)m0 * p.groups,
                                                            (uint32_t)(rows * p.groups));
            scale_at[i] = (uint32_t)(((of_w ? row : row - TN) + lane) * p.groups);
        } else {
            const int row = t + i * 256;
            const bool of_w = row < TN;
            scales_of[i] = of_w ? p.w_scales + (size_t)(n0 + min(row, cols - 1)) * p.groups
                                : p.x_scales + (size_t)(m0 + min(row - TN, rows - 1)) * p.groups;
            scales_end[i] = (of_w ? p.w_scales + (size_t)p.N * p.groups
                                  : p.x_scales + (size_t)p.M * p.groups) - 16;
        }
    }
    // Asks for a pair's scales, into place `to`: into LDS, or 16 bytes a row into registers, the
    // last ones of the array where it ends before; place_scales() moves those into place, zeros
    // behind the part's end (which meet zeros of both matrices; a neighbour row's byte may be a
    // NaN's).
    auto fetch_scales = [&](int pair_, int to) {
        const int pair = first / 2 + pair_;
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) {
            if constexpr (ALIGNED) {
                const int row = (i * 4 + wave) * 64;
                if (row < kRows)
                    symtile::buf_ld16_lds_async(
                        scale_rsrc[i], lds0 + (uint32_t)(offsetof(Lds, scales) + (to * kRows + row) * 16),
                        pair * 16 < end ? scale_at[i] : symtile::kOOB, (uint32_t)(pair * 16));
            } else {
                const uint8_t* from = scales_of[i] + min(pair * 16, p.groups - 1);
                const uint8_t* at = from < scales_end[i] ? from : scales_end[i];
                shift[i] = (int)(from - at) * 8;
                sc[i] = reinterpret_cast<const Unaligned16*>(at)->v;
            }
        }
    };
    auto place_scales = [&](int pair_, int to) {
        if constexpr (!ALIGNED) {
            const int valid = end - (first / 2 + pair_) * 16;
            if (valid < 16) {
#pragma unroll
                for (int i = 0; i < kScaleLoads; ++i) {
                    const uint64_t lo = (uint64_t)sc[i][1] << 32 | sc[i][0];
                    const uint64_t hi = (uint64_t)sc[i][3] << 32 | sc[i][2];
                    const int n = shift[i];
                    const uint64_t l = n == 0 ? lo : n < 64 ? lo >> n | hi << (64 - n) : hi >> (n - 64);
                    const uint64_t h = n < 64 ? hi >> n : 0;
                    sc[i] = u32x4{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int keep = valid - 4 * j;
                        if (keep < 4) sc[i][j] = keep <= 0 ? 0u : sc[i][j] & ((1u << (8 * keep)) - 1u);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kScaleLoads; ++i)
                if (t + i * 256 < kRows) lds.scales[to][t + i * 256] = sc[i];
        }
    };
    f32x16 acc[kNT][kMT] = {};
    // A lane's operands of an instruction, and its scales' bytes of a stage.
    struct Operands {
        u32x4 x[kMT], w[kNT];
    };
    struct Bytes {
        uint32_t w[kNT], x[kMT];
    };
    const int base_w = (wn * (TN / 2) + r) * kStageBytes + (((4 * g) ^ (r / 2 % 8)) * 16);
    const int base_x = (wm * (TM / 2) + r) * kStageBytes + (((4 * g) ^ (r / 2 % 8)) * 16);
    // Read k of the kMT + kNT of instruction S of the stage at `slot`.
    auto read = [&](Operands& o, int slot, int S, int k) {
        const typename Lds::Stage& now = lds.stage[slot];
        if (k < kMT) o.x[k] = symtile::ld16(&now.x[(base_x ^ (S * 16)) + k * 32 * kStageBytes]);
        else o.w[k - kMT] = symtile::ld16(&now.w[(base_w ^ (S * 16)) + (k - kMT) * 32 * kStageBytes]);
    };
    auto read_scale = [&](Bytes& o, int place, int odd, int k) {
        const uint32_t* of = reinterpret_cast<const uint32_t*>(lds.scales[place]) + odd * 2 + g;
        if (k < kMT) o.x[k] = of[(TN + wm * (TM / 2) + k * 32 + r) * 4];
        else o.w[k - kMT] = of[(wn * (TN / 2) + (k - kMT) * 32 + r) * 4];
    };
    // After a stage's third instructions all waves have read it, and the next one is there: its
    // place is the stage's RING further on, whose loads are asked for during the fourth and the
    // next stage's first.
    if (stages > 0) {
        Operands a, b;
        Bytes even, odd;
        int place = 0;               // of the pair's scales
        // The instructions S of stage st on `o`; between them, one or two each, the reads of the
        // next operands (and scales) and half of a stage's loads.  A wave issues in order and is
        // the only one of its SIMD in the largest build: what stands between two matrix
        // instructions for longer than the 32 cycles of the first leaves the unit idle.
        auto multiply = [&](auto s_, auto slot_, int st, const Operands& o, const Bytes& e,
                            Operands& next, Bytes& e_next) {
            constexpr int S = decltype(s_)::value, kSlot = decltype(slot_)::value;
            constexpr int kReads = kMT + kNT, kBytes = S == 3 ? kReads : 0;
            constexpr int kHalf = S == 0 || S == 3 ? kLoads / 2 : 0;
            constexpr int kOthers = kBytes + kReads + kHalf, kTiles = kNT * kMT;
#pragma unroll
            for (int q = 0; q < kTiles; ++q) {
                const int i = q / kMT, j = q % kMT;
                acc[i][j] = mfma32<S>(o.w[i], o.x[j], acc[i][j], e.w[i], e.x[j]);
                asm volatile("" : "+a"(acc[i][j]));
#pragma unroll
                for (int k = q * kOthers / kTiles; k < (q + 1) * kOthers / kTiles; ++k) {
                    if (k < kBytes)
                        read_scale(e_next, place, 1 - kSlot % 2, k);
                    else if (k < kBytes + kReads)
                        read(next, S == 3 ? (kSlot + 1) % RING : kSlot, (S + 1) % 4, k - kBytes);
                    else if (S == 0)
                        load(st + RING - 1, (kSlot + RING - 1) % RING, kHalf + k - kBytes - kReads);
                    else
                        load(st + RING, kSlot, k - kBytes - kReads);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // The place of the scales of the pair `ahead` pairs further on.
        auto place_of = [&](int ahead) {
            const int at = place + ahead;
            return at >= Lds::kPairs ? at - Lds::kPairs : at;
        };
        constexpr int kAhead = ALIGNED ? RING / 2 : 1;      // pairs
        auto stage = [&](auto slot_, int st, const Bytes& e, Bytes& e_next) {
            constexpr int kSlot = decltype(slot_)::value;
            if (kSlot % 2 == 0) fetch_scales((st >> 1) + kAhead, place_of(kAhead));
            multiply(std::integral_constant<int, 0>{}, slot_, st, a, e, b, e_next);
            multiply(std::integral_constant<int, 1>{}, slot_, st, b, e, a, e_next);
            multiply(std::integral_constant<int, 2>{}, slot_, st, a, e, b, e_next);
            if (kSlot % 2 == 1) {
                place_scales((st >> 1) + 1, place_of(1));
                place = place_of(1);
            }
            meet<(RING - 2) * kLoads>();
            multiply(std::integral_constant<int, 3>{}, slot_, st, b, e, a, e_next);
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fetch_scales(i, i);
#pragma unroll
        for (int i = 0; i < RING - 1; ++i)
#pragma unroll
            for (int u = 0; u < kLoads; ++u) load(i, i, u);
#pragma unroll
        for (int u = 0; u < kLoads / 2; ++u) load(RING - 1, RING - 1, u);
        place_scales(0, 0);
        meet<(RING - 2) * kLoads + kLoads / 2>();
#pragma unroll
        for (int k = 0; k < kMT + kNT; ++k) {
            read(a, 0, 0, k);
            read_scale(even, 0, 0, k);
        }
        // (in pairs, or fours; stages behind the part's end are zeros)
        for (int st = 0; st < stages; st += RING) {
            stage(std::integral_constant<int, 0>{}, st, even, odd);
            stage(std::integral_constant<int, 1>{}, st + 1, odd, even);
            if constexpr (RING == 4) {
                stage(std::integral_constant<int, 2>{}, st + 2, even, odd);
                stage(std::integral_constant<int, 3>{}, st + 3, odd, even);
            }
        }
        __builtin_amdgcn_s_waitcnt(wait_loads(0));
    }
    if (kSplits && p.splits > 1) {
        // [tile][split][wave][tile of the wave][quarter][lane]
        constexpr int kPart = TM * TN;
        const uint32_t at = (uint32_t)((wave * kNT * kMT * 4 * 64 + lane) * 16);
        const symtile::rsrc_t to =
            symtile::make_rsrc(p.partials + ((size_t)tile * p.splits + split) * kPart, kPart * 4);
#pragma unroll
        for (int i = 0; i < kNT; ++i)
#pragma unroll
            for (int j = 0; j < kMT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x16& v = acc[i][j];
                    const f32x4 u = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
                    symtile::buf_st16p<symtile::kStoreWriteThrough>(
                        __builtin_bit_cast(u32x4, u), to, at, ((i * kMT + j) * 4 + q) * 1024);
                }
        symtile::wg_stores_done();
        if (t == 0) {
            symtile::release_written_through();
            const uint32_t before = symtile::atomic_add<__ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT>(
                p.counters + tile, 1u);
            lds.last = before == (uint32_t)p.splits - 1;
            if (lds.last)
                __hip_atomic_store(symtile::global_ptr(p.counters + tile), 0u, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!lds.last) return;
        symtile::acquire_coherent_reads();
        const symtile::rsrc_t from = symtile::make_rsrc(p.partials + (size_t)tile * p.splits * kPart,
                                                        (uint32_t)(p.splits * kPart * 4));
#pragma unroll
        for (int i = 0; i < kNT; ++i)
#pragma unroll
            for (int j = 0; j < kMT; ++j) acc[i][j] = f32x16{};
        // the parts in the order of K, several parts' loads in flight together (parts that are
        // not there are zeros)
        constexpr int kTogether = 4;
        for (int s0 = 0; s0 < p.splits; s0 += kTogether) {
            f32x4 u[kTogether][kNT * kMT * 4];
#pragma unroll
            for (int s = 0; s < kTogether; ++s)
#pragma unroll
                for (int q = 0; q < kNT * kMT * 4; ++q)
                    u[s][q] = __builtin_bit_cast(
                        f32x4, symtile::buf_ld16p<symtile::kLoadCoherent>(
                                   from, s0 + s < p.splits ? at : symtile::kOOB,
                                   (uint32_t)((s0 + s) * kPart * 4 + q * 1024)));
#pragma unroll
            for (int s = 0; s < kTogether; ++s)
#pragma unroll
                for (int q = 0; q < kNT * kMT * 4; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[q / 4 / kMT][q / 4 % kMT][q % 4 * 4 + e] += u[s][q][e];
        }
    }
    // The slots' bases, all asked for before the first is needed: for the stores, and for the
    // lane's counter (64x8192x3584 into 8 slots: one after the other in the loops over the slots
    // they took 6 us).
    uint64_t bases[SYMTILE_MAX_WORLD];
#pragma unroll
    for (int s = 0; s < SYMTILE_MAX_WORLD; ++s) bases[s] = p.bases[min(s, p.world - 1)];
    // Rows and columns that a wave stores: 64 rows, whose tiles it counts; of 64 alone a quarter
    // of the rows in their whole width (64x8192x3584 into 8 slots, tiles of 64 x 128: 12.5 us;
    // 64 rows of 32 columns a wave, 64 bytes of a row together, 14.2).
    constexpr bool kShared = TM == 64;
    constexpr int kCols = kShared ? TN : TM * TN / 256, kStoreRows = TM * TN / 4 / kCols;
    constexpr int kTiles16 = kCols / kTileN;
    constexpr int kSlots = 64 / kTiles16;                                // slots that 64 lanes count
    uint64_t counter_base[(SYMTILE_MAX_WORLD + kSlots - 1) / kSlots];
#pragma unroll
    for (int i = 0; i < (SYMTILE_MAX_WORLD + kSlots - 1) / kSlots; ++i)
        counter_base[i] = p.bases[min(i * kSlots + lane / kTiles16, p.world - 1)];
    // The stages' place is the results' from here on, rows of TN: vector v of 8 values of row
    // m at v ^ (m % 32).  A lane has four values in a row of each group of accumulators.
    __syncthreads();
    constexpr int kVecs = TN / 8, kMask = (kVecs < 32 ? kVecs : 32) - 1;
#pragma unroll
    for (int i = 0; i < kNT; ++i)
#pragma unroll
        for (int j = 0; j < kMT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = wn * (TN / 2) + i * 32 + 8 * q + 4 * g, m = wm * (TM / 2) + j * 32 + r;
                uint2 v;
                const f32x16& a = acc[i][j];
                v.x = rounded<BF>(a[4 * q]) | (uint32_t)rounded<BF>(a[4 * q + 1]) << 16;
                v.y = rounded<BF>(a[4 * q + 2]) | (uint32_t)rounded<BF>(a[4 * q + 3]) << 16;
                *reinterpret_cast<uint2*>(
                    &lds.out[m * TN + (((n / 8) ^ (m & kMask)) * 8) + n % 8]) = v;
            }
    __syncthreads();
    constexpr int kAcross = TN / kCols;
    constexpr int kLanes = kCols / 8, kPer = 64 / kLanes, kSteps = kStoreRows / kPer;
    const int sr = wave / kAcross * kStoreRows, sn = wave % kAcross * kCols;
    const int own_rows = min(kStoreRows, rows - sr), own_cols = min(kCols, cols - sn);
    const bool none = own_rows <= 0 || own_cols <= 0;
    if (!kShared && none) return;
    const int row0 = lane / kLanes, v0 = lane % kLanes;
    const uint32_t at = v0 * 8 < own_cols ? (uint32_t)((row0 * p.ldc + v0 * 8) * 2) : symtile::kOOB;
    constexpr int kBatch = kSteps < 8 ? kSteps : 8;
    for (int i0 = 0; i0 < kSteps && !none; i0 += kBatch) {
        u32x4 v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int m = sr + (i0 + i) * kPer + row0;
            v[i] = symtile::ld16(&lds.out[m * TN + (((sn / 8 + v0) ^ (m & kMask)) * 8)]);
        }
#pragma unroll
        for (int s = 0; s < SYMTILE_MAX_WORLD; ++s) {
            if (s >= p.world) break;
            const symtile::rsrc_t dst = symtile::make_rsrc(
                reinterpret_cast<char*>(bases[s]) + p.c_off + ((size_t)(m0 + sr) * p.ldc + n0 + sn) * 2,
                (uint32_t)(((size_t)(own_rows - 1) * p.ldc + own_cols) * 2));
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                symtile::buf_st16p<kStoreThroughStream>(
                    v[i], dst, at, (uint32_t)((i0 + i) * kPer * p.ldc * 2));
        }
    }
    symtile::release_written_through();
    if constexpr (kShared) {
        __syncthreads();
        if (wave) return;
    }
    const int counted = lane % kTiles16;
#pragma unroll
    for (int i = 0; i < (SYMTILE_MAX_WORLD + kSlots - 1) / kSlots; ++i)
        if (i * kSlots + lane / kTiles16 < p.world && counted * kTileN < own_cols)
            symtile::flag_signal(reinterpret_cast<uint32_t*>(counter_base[i] + p.flag_off) +
                                 (size_t)((m0 + sr) / kTileM) * p.tiles_n + (n0 + sn) / kTileN +
                                 counted);
}

// ---- host ------------------------------------------------------------------------------
int ceil_div(int a, int b) { return (a + b - 1) / b; }

using symtile_host::fail;

symtile_status check_sizes(int M, int N, int K) {
    if (M < 0 || N < 0 || K < 0) return fail(SYMTILE_EINVAL, "negative size");
    if (K % kBlock || N % 8) return fail(SYMTILE_EINVAL, "K must be a multiple of 32, N_local of 8");
    if (K > (1 << 22)) return fail(SYMTILE_EINVAL, "K exceeds 4194304");
    if (M > (1 << 21)) return fail(SYMTILE_EINVAL, "M exceeds 2097152");
    return SYMTILE_OK;
}

// A build of the kernel for many rows, and the parts that K is split into; tm = 0: the other
// kernel.
struct GemmBuild {
    int tm, tn, splits;
    const void* kernels[2][2];     // [bfloat16][scales aligned]
};
template <int TM, int TN, int RING>
GemmBuild gemm_of() {
    return {TM, TN, 1,
            {{reinterpret_cast<const void*>(&mx4_gemm_kernel<false, TM, TN, RING, false>),
              reinterpret_cast<const void*>(&mx4_gemm_kernel<false, TM, TN, RING, true>)},
             {reinterpret_cast<const void*>(&mx4_gemm_kernel<true, TM, TN, RING, false>),
              reinterpret_cast<const void*>(&mx4_gemm_kernel<true, TM, TN, RING, true>)}}};
}

GemmBuild gemm_build(int cus, int M, int N, int groups) {
    GemmBuild b{};
    b.splits = 1;
    // Up to 32 rows the other kernel while there is little to do: its tiles read X once each, but
    // K needs no second way through memory.  (M x K x N, us, other kernel / 64 x 64 tiles:
    // 1x8192x3584 6.3 / 9.0, 1x8192x8192 12.5 / 10.5, 1x8192x28672 31 / 20, 16x8192x3584 7.8 / 9.1,
    // 32x4096x4096 6.1 / 7.7, 32x8192x2048 9.2 / 7.9, 16x2048x16384 7.0 / 6.3; over 32 rows, where it
    // gains little at best, never: 48x4096x1024 7.2 / 7.5, 48x1024x8192 5.5 / 4.9, 64x2048x4096 6.0 /
    // 5.8, 64x8192x3584 16.2 / 10.0.)
    const size_t rounds = std::max<size_t>(1, ceil_div(ceil_div(N, kTileN), cus));
    const size_t values = (size_t)ceil_div(M, 16) * groups * kBlock * rounds;
    const bool little = M <= 32 && values <= (rounds == 1 ? 12288 : M <= 16 ? 8192 : 0);
    if (little || (size_t)N * groups < 16 || (size_t)M * groups < 16) return b;   // (scales come by 16)
    // The largest tiles that leave no CU without one, where there are as many (into 8 slots where
    // N is 3584 or 1024; us, tiles of 64 x 64 / 64 x 128 / 128 x 128 / 256 x 256: 64x8192x3584
    // 10.0 / 12.5, 256x8192x3584 13.5 / 15.7 / 20.3 / 60, 1024x4096x1024 10.2 / 13.7 / 17.1 / 37,
    // 128x8192x28672 36 / 32 / 36 / 49, 512x8192x8192 38 / 32 / 30 / 49, 512x8192x28672 115 / 106 / 77 /
    // 67, 2048x8192x3584 72 / 76 / 56 / 70, 2048x8192x8192 130 / 119 / 82 / 70; all on the same
    // weights, which the memory-side cache keeps: from memory 128x8192x28672 takes 48, 512 rows 75).
    auto tiles = [&](int tm, int tn) { return (size_t)ceil_div(M, tm) * ceil_div(N, tn); };
    b = tiles(64, 64) <= (size_t)cus                    ? gemm_of<64, 64, 4>()
        : M <= 128 || tiles(64, 128) <= (size_t)cus     ? gemm_of<64, 128, 4>()
        : 2 * tiles(256, 256) < (size_t)cus             ? gemm_of<128, 128, 2>()
                                                        : gemm_of<256, 256, 2>();
    const size_t n = tiles(b.tm, b.tn);
    // as many parts as give every CU one workgroup, of four pairs of stages at least
    // (64x8192x2048 7.9 us, of two pairs 8.7; 64x4096x1024 7.5, 6.9)
    // (the larger tiles come with more than half as many as there are CUs)
    if (b.tm * b.tn == 64 * 64)
        b.splits = (int)std::max<size_t>(1, std::min<size_t>((size_t)cus / n, ceil_div(groups, 8) / 8));
    return b;
}

// Counters, one per tile, then the partial sums.
constexpr size_t kCounterBytes = (size_t)symtile_host::kWorkspaceCounters * 4;

size_t workspace_bytes_of(const GemmBuild& b, int splits, int M, int N) {
    if (splits <= 1) return 0;
    return kCounterBytes + (size_t)ceil_div(M, b.tm) * ceil_div(N, b.tn) * splits * b.tm * b.tn * 4;
}

bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na && nb && x < y + nb && y < x + na;
}

}  // namespace

extern "C" symtile_status symtile_mx4_quantise(int device, const void* x, int rows, int cols,
                                               size_t ld, int dtype, uint8_t* q, uint8_t* scales,
                                               void* values, size_t ld_values, symtile_stream s) {
    const size_t esize = logits::elem_size(dtype);
    if (!esize) return fail(SYMTILE_EINVAL, "unknown dtype");
    if (rows < 0 || cols < 0 || cols % kBlock)
        return fail(SYMTILE_EINVAL, "rows < 0, or cols not a multiple of 32");
    if (ld == 0) ld = (size_t)cols;
    if (ld_values == 0) ld_values = (size_t)cols;
    if (ld < (size_t)cols || ld_values < (size_t)cols)
        return fail(SYMTILE_EINVAL, "ld or ld_values smaller than cols");
    if (rows && std::max(ld, ld_values) > (SIZE_MAX >> 3) / (size_t)rows)
        return fail(SYMTILE_EINVAL, "the matrix exceeds the address space");
    if (rows == 0 || cols == 0) return SYMTILE_OK;
    if (!x || !q || !scales) return fail(SYMTILE_EINVAL, "NULL pointer");
    if (misaligned(x, esize) || misaligned(values, esize))
        return fail(SYMTILE_EINVAL, "x or values not aligned to their type");
    if (misaligned(q, 16)) return fail(SYMTILE_EINVAL, "q must be 16-byte aligned");
    const size_t n_x = ((size_t)(rows - 1) * ld + cols) * esize;
    const size_t n_v = values ? ((size_t)(rows - 1) * ld_values + cols) * esize : 0;
    const size_t n_q = (size_t)rows * (cols / 2), n_s = (size_t)rows * (cols / kBlock);
    if (values && !(values == x && ld == ld_values) && overlap(x, n_x, values, n_v))
        return fail(SYMTILE_EINVAL, "values overlap x without being it");
    if (overlap(x, n_x, q, n_q) || overlap(x, n_x, scales, n_s) || overlap(q, n_q, scales, n_s) ||
        overlap(values, n_v, q, n_q) || overlap(values, n_v, scales, n_s))
        return fail(SYMTILE_EINVAL, "q or scales overlap another argument");
    logits::OnDevice on(device);
    if (on.status) return on.status;
    QuantiseParams p{};
    p.x = x;
    p.q = q;
    p.scales = scales;
    p.values = values;
    p.ld = ld;
    p.ld_values = ld_values;
    p.row_pieces = cols / 8;
    p.by_row = symtile_host::make_div(p.row_pieces);
    const void* kernel =
        dtype == SYMTILE_F32  ? reinterpret_cast<const void*>(&mx4_quantise_kernel<SYMTILE_F32>)
        : dtype == SYMTILE_F16 ? reinterpret_cast<const void*>(&mx4_quantise_kernel<SYMTILE_F16>)
                               : reinterpret_cast<const void*>(&mx4_quantise_kernel<SYMTILE_BF16>);
    // pieces that fit 31 bits, in whole rows
    const int most = std::max(1, (1 << 30) / p.row_pieces);
    for (int row0 = 0; row0 < rows; row0 += most) {
        p.row0 = row0;
        p.pieces = std::min(most, rows - row0) * p.row_pieces;
        void* args[] = {&p};
        hipError_t e = hipLaunchKernel(kernel, dim3((unsigned)ceil_div(p.pieces, 256)), dim3(256),
                                       args, 0, static_cast<hipStream_t>(s));
        if (e == hipSuccess) e = hipGetLastError();
        if (e != hipSuccess) return symtile_host::hip_fail(e, "mx4_quantise_kernel launch");
        if (rows - row0 <= most) break;
    }
    return SYMTILE_OK;
}

extern "C" symtile_status symtile_mx4_workspace_bytes(int device, int M, int N_local, int K,
                                                      size_t* bytes) {
    if (!bytes) return fail(SYMTILE_EINVAL, "bytes is NULL");
    *bytes = 0;
    if (symtile_status st = check_sizes(M, N_local, K)) return st;
    const int cus = symtile_host::cu_count(device);
    if (cus <= 0)
        return fail(SYMTILE_EINVAL, "device " + std::to_string(device) + " out of range");
    if (M == 0 || N_local == 0) return SYMTILE_OK;
    const GemmBuild build = gemm_build(cus, M, N_local, K / kBlock);
    *bytes = workspace_bytes_of(build, build.splits, M, N_local);
    return SYMTILE_OK;
}

extern "C" symtile_status symtile_mx4_all_scatter(
    symtile_heap* h, const uint8_t* x, const uint8_t* x_scales, const uint8_t* q,
    const uint8_t* scales, void* C_gathered_local, uint32_t* arrived_local, int M, int N_local,
    int K, int dtype, int rank, int world_size, void* workspace, size_t workspace_bytes,
    symtile_stream s) {
    if (!h) return fail(SYMTILE_EINVAL, "heap is NULL");
    if (dtype != SYMTILE_F16 && dtype != SYMTILE_BF16)
        return fail(SYMTILE_EUNSUPPORTED, "dtype must be SYMTILE_F16 or SYMTILE_BF16");
    if (world_size != h->world) return fail(SYMTILE_EINVAL, "world_size differs from the heap's");
    if (rank < 0 || rank >= world_size) return fail(SYMTILE_EINVAL, "rank out of range");
    if (symtile_status st = check_sizes(M, N_local, K)) return st;
    if (M == 0 || N_local == 0) return SYMTILE_OK;
    if (!C_gathered_local || !arrived_local || (K && (!x || !x_scales || !q || !scales)))
        return fail(SYMTILE_EINVAL, "NULL pointer");
    if (misaligned(x, 16) || misaligned(q, 16) || misaligned(C_gathered_local, 16) ||
        misaligned(arrived_local, 4) || misaligned(workspace, 16))
        return fail(SYMTILE_EINVAL,
                    "x, q, C and the workspace must be 16-byte aligned, counters 4");
    const int tiles_m = ceil_div(M, kTileM), tiles_n = ceil_div(N_local, kTileN);
    const size_t ldc = (size_t)world_size * N_local;
    if (ldc > (size_t(1) << 22))
        return fail(SYMTILE_EINVAL, "world_size * N_local exceeds 4194304 columns");
    const size_t c_bytes = (size_t)M * ldc * 2;
    const size_t flag_bytes = (size_t)world_size * tiles_m * tiles_n * 4;
    if (!symtile_host::in_slot(h, C_gathered_local, c_bytes, rank))
        return fail(SYMTILE_EINVAL, "C_gathered_local [M, world*N_local] not inside slot of rank");
    if (!symtile_host::in_slot(h, arrived_local, flag_bytes, rank))
        return fail(SYMTILE_EINVAL, "arrived_local not inside slot of rank");
    if (overlap(C_gathered_local, c_bytes, arrived_local, flag_bytes))
        return fail(SYMTILE_EINVAL, "arrived_local overlaps C_gathered_local");
    const int cus = std::max(1, symtile_host::cu_count(h->device));

    ProductParams p{};
    p.x = x;
    p.x_scales = x_scales;
    p.w = q;
    p.w_scales = scales;
    p.bases = h->dev_bases;
    p.c_off = reinterpret_cast<uint64_t>(C_gathered_local) - h->host_bases[rank] +
              (size_t)rank * N_local * 2;
    p.flag_off = reinterpret_cast<uint64_t>(arrived_local) - h->host_bases[rank] +
                 (size_t)rank * tiles_m * tiles_n * 4;
    p.M = M;
    p.N = N_local;
    p.groups = K / kBlock;
    p.world = world_size;
    p.ldc = ldc;
    p.tiles_n = tiles_n;
    const GemmBuild build = gemm_build(cus, M, N_local, p.groups);
    if (build.tm) {
        p.gm = ceil_div(M, build.tm);
        const int gn = ceil_div(N_local, build.tn);
        const int stages = ceil_div(p.groups, 8);
        int splits = workspace ? build.splits : 1;
        const size_t need = workspace_bytes_of(build, splits, M, N_local);
        if (workspace && workspace_bytes < need)
            return fail(SYMTILE_EINVAL, "workspace of " + std::to_string(need) + " bytes needed");
        p.part_stages = std::max(2, ceil_div(ceil_div(stages, splits), 2) * 2);   // whole pairs
        splits = std::max(1, ceil_div(stages, p.part_stages));                    // none empty
        p.splits = splits;
        p.by_splits = symtile_host::make_div(splits);
        if (splits > 1) {
            p.counters = static_cast<uint32_t*>(workspace);
            p.partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterBytes);
        }
        const size_t units = (size_t)p.gm * gn * splits;
        if (units > (1u << 23)) return fail(SYMTILE_EINVAL, "more than 8388608 tiles");
        p.per_xcd = (int)(units / kXcds);
        p.xcd_rest = (int)(units % kXcds);
        p.band = kBandRows * gn;
        p.by_band = symtile_host::make_div(p.band);
        const bool aligned = p.groups % 16 == 0 && !misaligned(x_scales, 16) && !misaligned(scales, 16);
        int prev = -1;
        if (symtile_status st = symtile_host::set_device(h, &prev)) return st;
        void* args[] = {&p};
        hipError_t e = hipLaunchKernel(build.kernels[dtype == SYMTILE_BF16][aligned],
                                       dim3((unsigned)units), dim3(256), args, 0,
                                       static_cast<hipStream_t>(s));
        if (e == hipSuccess) e = hipGetLastError();
        if (prev >= 0) (void)hipSetDevice(prev);
        return e == hipSuccess ? SYMTILE_OK : symtile_host::hip_fail(e, "mx4_gemm_kernel launch");
    }
    // 16 waves, so that 8192 values are one round of chunks, where every workgroup has a CU and its
    // sums' 16 parts are few
    const int mt = M > 32 ? 2 : M > 16 ? 1 : 0;
    const bool many = mt == 0 && p.groups > 128 && (size_t)tiles_m * tiles_n <= (size_t)cus;
    const void* const kernels[2][4] = {
        {reinterpret_cast<const void*>(&mx4_kernel<false, 1, 8>),
         reinterpret_cast<const void*>(&mx4_kernel<false, 2, 8>),
         reinterpret_cast<const void*>(&mx4_kernel<false, 4, 8>),
         reinterpret_cast<const void*>(&mx4_kernel<false, 1, 16>)},
        {reinterpret_cast<const void*>(&mx4_kernel<true, 1, 8>),
         reinterpret_cast<const void*>(&mx4_kernel<true, 2, 8>),
         reinterpret_cast<const void*>(&mx4_kernel<true, 4, 8>),
         reinterpret_cast<const void*>(&mx4_kernel<true, 1, 16>)}};
    int prev = -1;
    if (symtile_status st = symtile_host::set_device(h, &prev)) return st;
    void* args[] = {&p};
    hipError_t e = hipLaunchKernel(kernels[dtype == SYMTILE_BF16][many ? 3 : mt],
                                   dim3((unsigned)tiles_n, (unsigned)tiles_m),
                                   dim3(many ? 1024 : 512), args, 0, static_cast<hipStream_t>(s));
    if (e == hipSuccess) e = hipGetLastError();
    if (prev >= 0) (void)hipSetDevice(prev);
    return e == hipSuccess ? SYMTILE_OK : symtile_host::hip_fail(e, "mx4_kernel launch");
}
