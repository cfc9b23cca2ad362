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
// become 6.  The conversion rounds to nearest even and saturates.
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
    int tiles_n;
};

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

// A workgroup takes 16 columns and up to 64 rows; its waves share the chunks of 512 values.
constexpr int kWaves = 8;
template <bool BF, int MT>
__global__ void __launch_bounds__(64 * kWaves) mx4_kernel(ProductParams p) {
    __shared__ float sums[kWaves][MT][256];
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
    f32x4 total[MT] = {};
    for (int first = wave * 16; first < p.groups; first += kWaves * 16) {
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
    for (int e = t; e < MT * 256; e += 64 * kWaves) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += sums[w][e / 256][e % 256];
        out[e / 256 * 16 + e % 256 / 64 * 4 + e % 4][e / 4 % 16] = rounded<BF>(v);
    }
    __syncthreads();
    // wave s: slot s
    for (int s = wave; s < p.world; s += kWaves) {
        char* base = reinterpret_cast<char*>(p.bases[s]);
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
    if (symtile_host::cu_count(device) <= 0)
        return fail(SYMTILE_EINVAL, "device " + std::to_string(device) + " out of range");
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
    (void)workspace_bytes;

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
    const int mt = M > 48 ? 4 : M > 32 ? 3 : M > 16 ? 2 : 1;
    const void* const kernels[2][4] = {
        {reinterpret_cast<const void*>(&mx4_kernel<false, 1>),
         reinterpret_cast<const void*>(&mx4_kernel<false, 2>),
         reinterpret_cast<const void*>(&mx4_kernel<false, 3>),
         reinterpret_cast<const void*>(&mx4_kernel<false, 4>)},
        {reinterpret_cast<const void*>(&mx4_kernel<true, 1>),
         reinterpret_cast<const void*>(&mx4_kernel<true, 2>),
         reinterpret_cast<const void*>(&mx4_kernel<true, 3>),
         reinterpret_cast<const void*>(&mx4_kernel<true, 4>)}};
    int prev = -1;
    if (symtile_status st = symtile_host::set_device(h, &prev)) return st;
    void* args[] = {&p};
    hipError_t e = hipLaunchKernel(kernels[dtype == SYMTILE_BF16][mt - 1],
                                   dim3((unsigned)tiles_n, (unsigned)tiles_m), dim3(64 * kWaves),
                                   args, 0, static_cast<hipStream_t>(s));
    if (e == hipSuccess) e = hipGetLastError();
    if (prev >= 0) (void)hipSetDevice(prev);
    return e == hipSuccess ? SYMTILE_OK : symtile_host::hip_fail(e, "mx4_kernel launch");
}
