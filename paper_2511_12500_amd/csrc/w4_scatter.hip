// A few tokens' product with a rank's shard of 4-bit weights, stored into every
// slot of the heap (the All-Scatter of Section 4.2.1 behind a matrix-vector
// product).
//
// C[m, n] = sum_k X[m, k] (q[n, k] - zero[n, k / group]) scale[n, k / group].
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

#include "symtile.h"
#include "symtile_device.h"
#include "symtile_internal.h"

namespace {

constexpr int kThreads = 256;
constexpr int kTileN = SYMTILE_W4_TILE_N;
constexpr int kMaxM = SYMTILE_W4_TILE_M;
constexpr int kPerCol = kThreads / kTileN;   // threads that share a column
constexpr int kRows = 16;                    // rows a pass over the weights serves

struct W4Params {
    const void* X;
    const uint8_t* q;
    const void* scales;
    const uint8_t* zeros;
    const uint64_t* bases;
    uint64_t c_off, flag_off;   // of the rank's column block and its counters in a slot
    int M, N, K, ldx, lg_group, groups, world;
    size_t ldc;                 // elements
};

template <bool BF>
struct T16;
template <>
struct T16<true> { typedef __bf16 type; };
template <>
struct T16<false> { typedef _Float16 type; };

// One workgroup per tile of 16 columns; 16 threads share a column, each takes
// every 16th block of 32 weights.
template <bool BF>
__global__ void __launch_bounds__(kThreads) w4_kernel(W4Params p) {
    typedef typename T16<BF>::type T;
    __shared__ __attribute__((aligned(16))) T out[kMaxM][kTileN];
    const int tile = blockIdx.x;
    const int col = threadIdx.x / kPerCol, part = threadIdx.x % kPerCol;
    const int n = tile * kTileN + col;
    const T* X = static_cast<const T*>(p.X);
    const T* scales = static_cast<const T*>(p.scales);
    for (int m0 = 0; m0 < p.M; m0 += kRows) {
        float acc[kRows] = {};
        if (n < p.N) {
            for (int k0 = part * 32; k0 < p.K; k0 += kPerCol * 32) {
                const symtile::u32x4 w = symtile::ld16(p.q + ((size_t)n * p.K + k0) / 2);
                const size_t g = (size_t)n * p.groups + (k0 >> p.lg_group);
                const float sc = (float)scales[g];
                const float z = p.zeros ? (float)(p.zeros[g] & 15) : 8.0f;
#pragma unroll 1
                for (int i = 0; i < 32; ++i) {
                    const float wv = ((float)((w[i / 8] >> (4 * (i % 8))) & 15u) - z) * sc;
#pragma unroll
                    for (int m = 0; m < kRows; ++m)
                        if (m0 + m < p.M)
                            acc[m] += wv * (float)X[(size_t)(m0 + m) * p.ldx + k0 + i];
                }
            }
        }
#pragma unroll
        for (int m = 0; m < kRows; ++m) {
            float a = acc[m];
#pragma unroll
            for (int d = kPerCol / 2; d; d >>= 1) a += __shfl_xor(a, d);
            if (part == 0 && m0 + m < p.M) out[m0 + m][col] = (T)a;
        }
    }
    __syncthreads();
    // rows of 16 columns are two chunks of 8; N is a multiple of 8
    const int chunks = p.N - tile * kTileN >= kTileN ? 2 : 1;
    for (int i = threadIdx.x; i < p.world * p.M * chunks; i += kThreads) {
        const int c = i % chunks, m = i / chunks % p.M, slot = i / chunks / p.M;
        char* dst = reinterpret_cast<char*>(p.bases[slot]) + p.c_off +
                    ((size_t)m * p.ldc + (size_t)tile * kTileN + c * 8) * 2;
        symtile::st16(dst, symtile::ld16(&out[m][c * 8]), false);
    }
    symtile::wg_stores_done();
    if ((int)threadIdx.x < p.world) {
        uint32_t* flag = reinterpret_cast<uint32_t*>(
            reinterpret_cast<char*>(p.bases[threadIdx.x]) + p.flag_off) + tile;
        symtile::flag_publish(flag);
    }
}

}  // namespace

extern "C" symtile_status symtile_w4_all_scatter(
    symtile_heap* h, const void* X, const uint8_t* q, const void* scales, const uint8_t* zeros,
    void* C_gathered_local, uint32_t* arrived_local, int M, int N_local, int K, int ldx, int group,
    int dtype, int rank, int world_size, symtile_stream s) {
    using symtile_host::fail;
    if (!h) return fail(SYMTILE_EINVAL, "heap is NULL");
    if (dtype != SYMTILE_F16 && dtype != SYMTILE_BF16)
        return fail(SYMTILE_EUNSUPPORTED, "dtype must be SYMTILE_F16 or SYMTILE_BF16");
    if (world_size != h->world) return fail(SYMTILE_EINVAL, "world_size differs from the heap's");
    if (rank < 0 || rank >= world_size) return fail(SYMTILE_EINVAL, "rank out of range");
    if (M < 0 || N_local < 0 || K < 0) return fail(SYMTILE_EINVAL, "negative size");
    if (M > SYMTILE_W4_TILE_M)
        return fail(SYMTILE_EUNSUPPORTED,
                    "M exceeds " + std::to_string(SYMTILE_W4_TILE_M) + " tokens");
    if (group != 32 && group != 64 && group != 128)
        return fail(SYMTILE_EINVAL, "group must be 32, 64 or 128");
    if (ldx == 0) ldx = K;
    if (K % 32 || N_local % 8 || ldx % 8 || ldx < K)
        return fail(SYMTILE_EINVAL, "K must be a multiple of 32, N_local and ldx of 8, ldx >= K");
    if (M == 0 || N_local == 0) return SYMTILE_OK;
    if (!C_gathered_local || !arrived_local || (K && (!X || !q || !scales)))
        return fail(SYMTILE_EINVAL, "NULL pointer");
    auto misaligned = [](const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; };
    if (misaligned(X, 16) || misaligned(q, 16) || misaligned(C_gathered_local, 16) ||
        misaligned(arrived_local, 4) || misaligned(scales, 2))
        return fail(SYMTILE_EINVAL, "X, q and C must be 16-byte aligned, counters 4, scales 2");
    const int tiles = (N_local + SYMTILE_W4_TILE_N - 1) / SYMTILE_W4_TILE_N;
    const size_t ldc = (size_t)world_size * N_local;
    const size_t c_bytes = (size_t)M * ldc * 2;
    const size_t flag_bytes = (size_t)world_size * tiles * 4;
    if (!symtile_host::in_slot(h, C_gathered_local, c_bytes, rank))
        return fail(SYMTILE_EINVAL, "C_gathered_local [M, world*N_local] not inside slot of rank");
    if (!symtile_host::in_slot(h, arrived_local, flag_bytes, rank))
        return fail(SYMTILE_EINVAL, "arrived_local not inside slot of rank");
    const uint64_t c0 = reinterpret_cast<uint64_t>(C_gathered_local);
    const uint64_t f0 = reinterpret_cast<uint64_t>(arrived_local);
    if (c0 < f0 + flag_bytes && f0 < c0 + c_bytes)
        return fail(SYMTILE_EINVAL, "arrived_local overlaps C_gathered_local");

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
    p.lg_group = __builtin_ctz((unsigned)group);
    p.groups = (K + group - 1) / group;
    p.world = world_size;
    p.ldc = ldc;
    int prev = -1;
    if (symtile_status st = symtile_host::set_device(h, &prev)) return st;
    const void* kernel = dtype == SYMTILE_BF16 ? reinterpret_cast<const void*>(&w4_kernel<true>)
                                               : reinterpret_cast<const void*>(&w4_kernel<false>);
    void* args[] = {&p};
    hipError_t e = hipLaunchKernel(kernel, dim3((unsigned)tiles), dim3(kThreads), args, 0,
                                   static_cast<hipStream_t>(s));
    if (e == hipSuccess) e = hipGetLastError();
    if (prev >= 0) (void)hipSetDevice(prev);
    return e == hipSuccess ? SYMTILE_OK : symtile_host::hip_fail(e, "w4_kernel launch");
}
