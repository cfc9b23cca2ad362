// What the operators over rows of logits share (token_logprobs.hip, distill.hip,
// verify_draft.hip); embedding.hip and mx4.hip take the element types and checks.
//
// A workgroup takes one row, or one segment of a row, and holds it in
// registers: NV vectors of 16 bytes a thread.  A row of z = scale * x is used
// through its largest logit m and s = sum_v exp(scale (x_v - m)), logp_v =
// scale (x_v - m) - log s, so both sums and a gradient need the row twice; from
// registers the second time costs no memory traffic, and a row is read once
// and, with a gradient, written once.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <string>
#include <type_traits>

#include "symtile.h"
#include "symtile_device.h"
#include "symtile_internal.h"

namespace logits {

constexpr float kInf = __builtin_inff();
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaxThreads = 1024;
constexpr int kMaxWaves = kMaxThreads / 64;

// ---- element types -----------------------------------------------------------
template <int DT>
struct Elem {   // SYMTILE_F32
    typedef float type;
    static constexpr int kVec = 4;             // elements of 16 bytes
    static constexpr uint32_t kMasked = 0xFF800000u;   // -inf in a 32-bit word
};
template <>
struct Elem<SYMTILE_F16> {
    typedef _Float16 type;
    static constexpr int kVec = 8;
    static constexpr uint32_t kMasked = 0xFC00FC00u;
};
template <>
struct Elem<SYMTILE_BF16> {
    typedef __bf16 type;
    static constexpr int kVec = 8;
    static constexpr uint32_t kMasked = 0xFF80FF80u;
};

// Rows start at any multiple of the element size, so their vectors do too.
struct __attribute__((packed, aligned(2))) Unaligned16 {
    symtile::u32x4 v;
};
__device__ __forceinline__ symtile::u32x4 load16(const void* p) {
    return reinterpret_cast<const Unaligned16*>(p)->v;
}
__device__ __forceinline__ void store16(void* p, symtile::u32x4 v) {
    reinterpret_cast<Unaligned16*>(p)->v = v;
}

// Element e of a vector as fp32 (exact).
template <int DT>
__device__ __forceinline__ float element(const symtile::u32x4& v, int e) {
    if constexpr (DT == SYMTILE_F32) {
        return __uint_as_float(v[e]);
    } else if constexpr (DT == SYMTILE_BF16) {
        return __uint_as_float(e % 2 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16);
    } else {
        typedef _Float16 half2 __attribute__((ext_vector_type(2)));
        return (float)__builtin_bit_cast(half2, (uint32_t)v[e / 2])[e % 2];
    }
}

// A vector of kVec values, each rounded once to the type (nearest even).
template <int DT>
__device__ __forceinline__ symtile::u32x4 pack(const float* f) {
    symtile::u32x4 r;
    if constexpr (DT == SYMTILE_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = __float_as_uint(f[e]);
    } else {
        typedef typename Elem<DT>::type T;
        typedef T pair __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int e = 0; e < 4; ++e)
            r[e] = __builtin_bit_cast(uint32_t, pair{(T)f[2 * e], (T)f[2 * e + 1]});
    }
    return r;
}

// max without the canonicalisation that fmaxf adds for signalling NaNs: the
// inputs come straight from memory, and a NaN of either kind makes the row's
// sums NaN whatever this returns.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// ---- reductions --------------------------------------------------------------
// Over the wave by data-parallel primitives: 1, 2, then the other quad of 8
// and the other 8 of 16 mirrored, then the rows of 16 and the halves swapped.
// Every lane receives the result; the order is fixed.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
template <class F>
__device__ __forceinline__ float quad_reduce(float v, F f) {
    v = f(v, dpp<0xB1>(v));       // quad_perm 1 0 3 2
    return f(v, dpp<0x4E>(v));    // quad_perm 2 3 0 1
}
template <class F>
__device__ __forceinline__ float row_of_quads(float v, F f) {
    v = f(v, dpp<0x141>(v));      // row_half_mirror
    return f(v, dpp<0x140>(v));   // row_mirror
}
template <class F>
__device__ __forceinline__ float wave_of_rows(float v, F f) {
    const uint32_t u = __float_as_uint(v);
    const auto rows = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = f(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
    const uint32_t w = __float_as_uint(v);
    const auto halves = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return f(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
}
template <class F>
__device__ __forceinline__ float row_reduce(float v, F f) {
    return row_of_quads(quad_reduce(v, f), f);
}
template <class F>
__device__ __forceinline__ float wave_reduce(float v, F f) {
    return wave_of_rows(row_reduce(v, f), f);
}
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return max3(a, b, b); }
};
struct Sum {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
__device__ __forceinline__ float wave_max(float v) { return wave_reduce(v, Max()); }
__device__ __forceinline__ float wave_sum(float v) { return wave_reduce(v, Sum()); }

__device__ __forceinline__ uint32_t wave_sum_u32(uint32_t v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// Over the workgroup's `waves` (at most 16) wave results in LDS: every row of 16
// lanes reads and reduces them (one after the other they took a thousand cycles a
// row of logits).
static_assert(kMaxWaves == 16, "a row of lanes holds the waves' results");
template <class F>
__device__ __forceinline__ float over_waves(const float* lds, int waves, float none, F f) {
    const int l = threadIdx.x % 16;
    const float v = lds[l];
    return row_reduce(l < waves ? v : none, f);
}
__device__ __forceinline__ float waves_max(const float* lds, int waves) {
    return over_waves(lds, waves, -kInf, Max());
}
__device__ __forceinline__ float waves_sum(const float* lds, int waves) {
    return over_waves(lds, waves, 0.0f, Sum());
}

// ---- a segment in registers ----------------------------------------------------
// Vector i of thread t is vector i * threads + t of the segment; the elements
// behind its end are -inf.
template <int DT, int NV>
struct Segment {
    static constexpr int kVec = Elem<DT>::kVec;
    symtile::u32x4 v[NV];

    // `len` elements at p (which may be none).
    __device__ __forceinline__ void load(const typename Elem<DT>::type* p, int len, int threads) {
        const int t = threadIdx.x;
        if (len >= NV * threads * kVec) {
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = load16(p + (size_t)(i * threads + t) * kVec);
            return;
        }
        const uint32_t none = Elem<DT>::kMasked;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (i * threads + t) * kVec;
            v[i] = symtile::u32x4{none, none, none, none};
            if (at + kVec <= len) v[i] = load16(p + at);
        }
        const int rem = len % kVec, last = len / kVec;
        if (rem) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i * threads + t == last) v[i] = load_part(p + (size_t)last * kVec, rem);
        }
    }

    // (Parts of vectors are of the elements' own type: other code reads and writes
    // the same elements alone, and through another type the compiler need not keep
    // the order.)
    static __device__ __forceinline__ symtile::u32x4 load_part(const typename Elem<DT>::type* p,
                                                               int n) {
        const uint32_t none = Elem<DT>::kMasked;
        symtile::u32x4 r = {none, none, none, none};
        if constexpr (DT == SYMTILE_F32) {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < n) r[e] = __float_as_uint(p[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < n) {
                    const uint32_t h = __builtin_bit_cast(uint16_t, p[e]);
                    r[e / 2] = e % 2 ? (r[e / 2] & 0xFFFFu) | h << 16
                                     : (r[e / 2] & 0xFFFF0000u) | h;
                }
        }
        return r;
    }

    // A vector of the segment by its first element, from memory again.
    static __device__ __forceinline__ symtile::u32x4 fetch(const typename Elem<DT>::type* p, int len,
                                                           int at) {
        return at + kVec <= len ? load16(p + at) : load_part(p + at, len - at);
    }

    // Vector i of the results at p: whole, or its elements inside `len`.
    static __device__ __forceinline__ void store(typename Elem<DT>::type* p, int len, int at,
                                                 const symtile::u32x4& r) {
        if (at + kVec <= len) {
            store16(p + at, r);
        } else if (at < len) {
            const int n = len - at;
            if constexpr (DT == SYMTILE_F32) {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < n) p[at + e] = __uint_as_float(r[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < n)
                        p[at + e] = __builtin_bit_cast(typename Elem<DT>::type,
                                                       (uint16_t)(r[e / 2] >> (16 * (e % 2))));
            }
        }
    }

    // Before another pass over the registers.  The compiler would otherwise keep
    // the fp32 values of the pass before, twice the registers of 16-bit logits
    // (spills with 16 vectors a thread, and half the waves with 8).
    __device__ __forceinline__ void again() {
#pragma unroll
        for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(v[i]));
    }

    template <class F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < kVec; ++e) f(i, e, element<DT>(v[i], e));
    }

    // The largest element of each vector, and of all.
    __device__ __forceinline__ float thread_max(float (&vec)[NV]) const {
        float m = -kInf;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            vec[i] = -kInf;
#pragma unroll
            for (int e = 0; e < kVec; e += 2)
                vec[i] = max3(vec[i], element<DT>(v[i], e), element<DT>(v[i], e + 1));
            m = max3(m, vec[i], vec[i]);
        }
        return m;
    }
};

// The exponent of a logit in base 2: y = c (x - m) with c = scale * log2(e), as
// one fused multiply-add x * c - o.  o = m * c is rounded, which moves every y by
// the same r = m * c - o (`shift`), to be taken out of what is made of them.  r is
// up to half a unit in o's last place, so from kHugeExponent on, where that is more
// than 1/8 (and 2^r would soon pass the numbers' range: a row that is masked at -1e10),
// and where c is infinite, the difference comes first and r = 0.
constexpr float kHugeExponent = 0x1p22f;
struct Exponent {
    float scale, c, o, m, shift;
    bool huge;
    __host__ __device__ __forceinline__ Exponent(float largest, float scale_) : scale(scale_) {
        m = largest == -kInf ? 0.0f : largest;
        c = scale * kLog2e;
        o = m * c;
        huge = !(fabsf(o) < kHugeExponent);
        shift = huge ? 0.0f : __builtin_fmaf(m, c, -o);
    }
    template <bool HUGE>
    __host__ __device__ __forceinline__ float y(float x) const {
        return HUGE ? (x - m) * scale * kLog2e : __builtin_fmaf(x, c, -o);
    }
};
// Where exp2 has long vanished, and a product with its zero must not be a NaN.
constexpr float kFloorY = -1.0e5f;
__device__ __forceinline__ float exp2_fast(float y) { return __builtin_amdgcn_exp2f(y); }

// ---- the partials of a split row ---------------------------------------------------
// Written through and read coherently (other XCDs' workgroups), published by a
// counter per row: the workgroup that arrives last joins the row.
__device__ __forceinline__ void put(float* p, float v) {
    __hip_atomic_store(symtile::global_ptr(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}
__device__ __forceinline__ void put(uint64_t* p, uint64_t v) {
    __hip_atomic_store(symtile::global_ptr(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}
__device__ __forceinline__ float take(const float* p) {
    return __hip_atomic_load(symtile::global_ptr(const_cast<float*>(p)), __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_SYSTEM);
}
__device__ __forceinline__ uint64_t take(const uint64_t* p) {
    return __hip_atomic_load(symtile::global_ptr(const_cast<uint64_t*>(p)), __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_SYSTEM);
}

// True in the workgroup that finds all others of the row done; its counter is
// back at zero then.  All threads call it after the workgroup's last put().
__device__ __forceinline__ bool arrive_last(uint32_t* counter, int segs, int* lds) {
    symtile::wg_stores_done();
    if (threadIdx.x == 0) {
        symtile::release_written_through();
        const uint32_t before =
            symtile::atomic_add<__ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT>(counter, 1u);
        *lds = before == (uint32_t)segs - 1;
        if (*lds)
            __hip_atomic_store(symtile::global_ptr(counter), 0u, __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    symtile::acquire_coherent_reads();
    return *lds != 0;
}

// ---- host: how rows are laid out over workgroups -------------------------------------
// At most 32 segments a row: a wave joins them, and with SYMTILE_TOP_MAX keys each
// their keys fit LDS; SYMTILE_VOCAB_MAX is what 32 segments of 16384 vectors hold.
constexpr int kMaxSegments = 32;
static_assert(SYMTILE_VOCAB_MAX <= kMaxSegments * 16 * kMaxThreads * 4, "a row fits its segments");

// segs workgroups a row, each of `threads` threads with nv vectors of 16 bytes,
// of seg_len elements (the last may have fewer).
struct Plan {
    int nv, threads, segs, seg_len;
};

inline size_t elem_size(int dtype) {
    return dtype == SYMTILE_F32 ? 4 : dtype == SYMTILE_F16 || dtype == SYMTILE_BF16 ? 2 : 0;
}

// The workgroup for a segment of n vectors.  With more workgroups than CUs 8 vectors
// a thread, enough loads in flight a wave and few waves to meet at barriers (4096x8192
// bf16 distillation: 32.6 us, 36.9 with 4), fewer where that would leave one wave.
// With a CU for each workgroup (`alone`) up to 1024 threads, whose work on a row is
// shorter (one row of 28672 with 20 alternatives: 6.5 us against 6.9).  16 where
// 1024 threads of 8 do not hold it.
inline void shape(int n, bool alone, int* nv, int* threads) {
    *nv = n > 8 * kMaxThreads ? 16
          : alone             ? n > 4096 ? 8 : n > 1024 ? 4 : 2
                              : n > 512 ? 8 : n > 256 ? 4 : 2;
    *threads = std::min(kMaxThreads, std::max(128, (n + *nv * 64 - 1) / (*nv * 64) * 64));
}

// Values alone take rows of more than 4096 vectors (512 threads of 8) in segments,
// several workgroups a CU, so that one's loads go on under another's sums (333x100003
// fp32: 28 us, with segments of 16384 vectors 38).  Segments of at most 2048 vectors: in
// smaller workgroups fewer waves wait at a barrier (2000x50257 fp32 with 20 entries 100
// us, 115 with 4096; 1000x65537 bf16 alone 32, 37).  4096 where more than 32 entries
// make a segment's own selection and the join dear (1024x131072 bf16 with 64 79 us, 89
// with 2048), in rows of more than 16384 vectors (distillation of 200x300000 fp32, loss
// and gradient, 193 us, 229 with 32 segments), and where only those leave every
// workgroup a CU (64x100003 bf16 with 20 11.6 us against 13.7).  With a gradient a row
// that one workgroup holds (16384 vectors) stays whole, since it is read once then.
inline Plan make_plan(int device, int rows, int vocab, int dtype, bool grad, int top) {
    const int vec = dtype == SYMTILE_F32 ? 4 : 8;
    const int n = (vocab + vec - 1) / vec;
    const size_t cus = (size_t)symtile_host::cu_count(device);
    auto workgroups = [&](int most) { return (size_t)rows * ((n + most - 1) / most); };
    int most = 4096;
    if (n > most && n <= 16 * kMaxThreads && top <= 32 &&
        !(workgroups(4096) <= cus && workgroups(2048) > cus))
        most = 2048;
    most = grad && n <= 16 * kMaxThreads ? 16 * kMaxThreads
                                         : std::max(most, (n + kMaxSegments - 1) / kMaxSegments);
    const int segs = (n + most - 1) / most;
    Plan p;
    const int per = (n + segs - 1) / segs;
    p.segs = (n + per - 1) / per;
    p.seg_len = per * vec;
    shape(per, (size_t)rows * p.segs <= cus, &p.nv, &p.threads);
    return p;
}

// Threads that fit 32 bits, and a counter for every split row.
inline int rows_a_launch(const Plan& p) {
    const int most = (int)((size_t(1) << 30) / ((size_t)p.threads * p.segs));
    return p.segs > 1 ? std::min(most, symtile_host::kWorkspaceCounters) : most;
}

// Workspace of a launch's split rows: counters, one per row, then 4 floats per segment,
// then `top` 64-bit keys per segment.
struct Workspace {
    size_t partials, keys, bytes;
};
inline Workspace make_workspace(const Plan& p, int rows, int top) {
    Workspace w{};
    if (p.segs <= 1 || rows == 0) return w;
    const size_t units = (size_t)std::min(rows, rows_a_launch(p)) * p.segs;
    w.partials = (size_t)symtile_host::kWorkspaceCounters * 4;
    w.keys = w.partials + units * 16;
    w.bytes = w.keys + units * (size_t)top * 8;
    return w;
}

// ---- host: checks ----------------------------------------------------------------------
using symtile_host::fail;

inline symtile_status check_sizes(int rows, int vocab, int dtype, int top) {
    if (!elem_size(dtype)) return fail(SYMTILE_EINVAL, "unknown dtype");
    if (rows < 0 || vocab < 1) return fail(SYMTILE_EINVAL, "rows < 0 or vocab < 1");
    if (vocab > SYMTILE_VOCAB_MAX)
        return fail(SYMTILE_EINVAL, "vocab exceeds " + std::to_string(SYMTILE_VOCAB_MAX));
    if (top < 0 || top > SYMTILE_TOP_MAX || top > vocab)
        return fail(SYMTILE_EINVAL, "top must be in 0 .. min(vocab, " +
                                        std::to_string(SYMTILE_TOP_MAX) + ")");
    return SYMTILE_OK;
}

// The logits' address, stride and scale.
inline symtile_status check_logits(const void* logits, int rows, int vocab, size_t* ld, int dtype,
                                   float scale) {
    const size_t esize = elem_size(dtype);
    if (*ld == 0) *ld = (size_t)vocab;
    if (*ld < (size_t)vocab) return fail(SYMTILE_EINVAL, "ld smaller than vocab");
    if (rows && *ld > (SIZE_MAX >> 3) / (size_t)rows)
        return fail(SYMTILE_EINVAL, "logits exceed the address space");
    if (!(scale > 0.0f) || !std::isfinite(scale))
        return fail(SYMTILE_EINVAL, "scale must be positive and finite");
    if (rows && !logits) return fail(SYMTILE_EINVAL, "logits is NULL");
    if (reinterpret_cast<uintptr_t>(logits) % esize)
        return fail(SYMTILE_EINVAL, "logits not aligned to their type");
    return SYMTILE_OK;
}

// The gradient: the logits' own memory, or memory apart from them.
inline symtile_status check_grad(const void* logits, size_t ld, const void* dlogits,
                                 size_t* ld_grad, int rows, int vocab, int dtype) {
    const size_t esize = elem_size(dtype);
    if (*ld_grad == 0) *ld_grad = (size_t)vocab;
    if (*ld_grad < (size_t)vocab) return fail(SYMTILE_EINVAL, "ld_grad smaller than vocab");
    if (rows && *ld_grad > (SIZE_MAX >> 3) / (size_t)rows)
        return fail(SYMTILE_EINVAL, "dlogits exceed the address space");
    if (reinterpret_cast<uintptr_t>(dlogits) % esize)
        return fail(SYMTILE_EINVAL, "dlogits not aligned to their type");
    if (rows && !(dlogits == logits && *ld_grad == ld)) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(logits);
        const uintptr_t b = reinterpret_cast<uintptr_t>(dlogits);
        const size_t na = ((size_t)(rows - 1) * ld + vocab) * esize;
        const size_t nb = ((size_t)(rows - 1) * *ld_grad + vocab) * esize;
        if (a < b + nb && b < a + na)
            return fail(SYMTILE_EINVAL, "dlogits overlaps logits without being them");
    }
    return SYMTILE_OK;
}

inline symtile_status check_workspace(const void* workspace, size_t bytes, size_t need) {
    if (need == 0) return SYMTILE_OK;
    if (!workspace || bytes < need)
        return fail(SYMTILE_EINVAL, "workspace of " + std::to_string(need) + " bytes needed");
    if (reinterpret_cast<uintptr_t>(workspace) % 16)
        return fail(SYMTILE_EINVAL, "workspace must be 16-byte aligned");
    return SYMTILE_OK;
}

// Makes `device` current for the scope of a call.
struct OnDevice {
    int prev = -1;
    symtile_status status = SYMTILE_OK;
    explicit OnDevice(int device) {
        int cur = -1;
        if (hipGetDevice(&cur) == hipSuccess && cur == device) return;
        int n = 0;
        if (hipGetDeviceCount(&n) != hipSuccess || device < 0 || device >= n) {
            (void)hipGetLastError();
            status = fail(SYMTILE_EINVAL, "device " + std::to_string(device) + " out of range");
            return;
        }
        const hipError_t e = hipSetDevice(device);
        if (e != hipSuccess) status = symtile_host::hip_fail(e, "hipSetDevice");
        else prev = cur;
    }
    ~OnDevice() {
        if (prev >= 0) (void)hipSetDevice(prev);
    }
};

// f(type, vectors) with both as compile-time constants.
template <class F>
const void* pick(int dtype, int nv, F f) {
    auto by_nv = [&](auto d) -> const void* {
        switch (nv) {
            case 2: return f(d, std::integral_constant<int, 2>{});
            case 4: return f(d, std::integral_constant<int, 4>{});
            case 8: return f(d, std::integral_constant<int, 8>{});
            default: return f(d, std::integral_constant<int, 16>{});
        }
    };
    switch (dtype) {
        case SYMTILE_F16: return by_nv(std::integral_constant<int, SYMTILE_F16>{});
        case SYMTILE_BF16: return by_nv(std::integral_constant<int, SYMTILE_BF16>{});
        default: return by_nv(std::integral_constant<int, SYMTILE_F32>{});
    }
}

template <class P>
symtile_status launch(const void* kernel, const Plan& plan, int rows, size_t lds, P& params,
                      symtile_stream s, const char* what) {
    void* args[] = {&params};
    hipError_t e = hipLaunchKernel(kernel, dim3((unsigned)rows * (unsigned)plan.segs),
                                   dim3((unsigned)plan.threads), args, lds,
                                   static_cast<hipStream_t>(s));
    if (e == hipSuccess) e = hipGetLastError();
    return e == hipSuccess ? SYMTILE_OK : symtile_host::hip_fail(e, what);
}

}  // namespace logits
