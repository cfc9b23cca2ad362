// What is read off rows of logits: log probabilities of given tokens with
// entropies and top alternatives, the distillation loss against a teacher's top
// entries, and the gradients of both.
//
// A row r of z = scale * x is used through its largest logit m and
// s = sum_v exp(scale * (x_v - m)): logp_v = scale * (x_v - m) - log s.  The
// difference x_v - m is taken first (exact up to one rounding of the
// difference itself), so that logits at the type's lowest value, whose product
// with the scale overflows, keep their differences.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cfloat>
#include <cmath>
#include <string>

#include "symtile.h"
#include "symtile_device.h"
#include "symtile_internal.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kInf = __builtin_inff();
constexpr float kLog2e = 1.4426950408889634f;

template <int DT>
struct Elem;
template <>
struct Elem<SYMTILE_F32> {
    typedef float type;
    static __device__ __forceinline__ float load(float v) { return v; }
    static __device__ __forceinline__ float store(float v) { return v; }
};
template <>
struct Elem<SYMTILE_F16> {
    typedef _Float16 type;
    static __device__ __forceinline__ float load(_Float16 v) { return (float)v; }
    static __device__ __forceinline__ _Float16 store(float v) { return (_Float16)v; }
};
template <>
struct Elem<SYMTILE_BF16> {
    typedef __bf16 type;
    static __device__ __forceinline__ float load(__bf16 v) { return (float)v; }
    static __device__ __forceinline__ __bf16 store(float v) { return (__bf16)v; }
};

struct RowParams {
    const void* x;
    void* dx;
    size_t ld, ld_grad;
    int rows, vocab, top, k;
    int mode, values_dtype;
    float scale;
    const int64_t* targets;
    const int64_t* ids;
    const void* values;
    float *logprob, *entropy, *stats, *loss;
    int64_t* top_ids;
    float* top_logprobs;
    const float *g_logprob, *g_entropy, *g_lse, *row_grad;
};

// ---- reductions over the workgroup; every thread receives the result --------
template <class T, class F>
__device__ __forceinline__ T block_reduce(T v, T* lds, F f) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = f(v, __shfl_xor(v, d));
    __syncthreads();   // the array may still be read from a reduction before
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = f(v, lds[w]);
    return v;
}
__device__ __forceinline__ float block_max(float v, float* lds) {
    return block_reduce(v, lds, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float block_sum(float v, float* lds) {
    return block_reduce(v, lds, [](float a, float b) { return a + b; });
}

// exp(scale * d) with c = scale * log2(e), and d = x - m at most 0.
__device__ __forceinline__ float exp_scaled(float d, float c) { return exp2f(d * c); }

// The order of the top entries as whole numbers: the larger logit first (a NaN
// above all, -0 as +0), then the smaller id.  Never 0 nor ~0.
__device__ __forceinline__ uint64_t top_key(float x, int v) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    const uint32_t o = x != x ? 0xFFFFFFFEu : b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
    return (uint64_t)o << 32 | (0xFFFFFFFFu - (uint32_t)v);
}
__device__ __forceinline__ int key_id(uint64_t key) { return (int)(0xFFFFFFFFu - (uint32_t)key); }

// The gradient of one logit: p (g_lse - g_logprob) - p (logp + H) g_entropy,
// times the scale; the target's own term is added by the caller.
struct LogprobGrad {
    float m, log_s, entropy, a, b;   // a = g_lse - g_logprob, b = g_entropy
    float scale;
    bool empty;
    __device__ __forceinline__ float operator()(float x) const {
        const float logp = fmaxf((x - m) * scale, -FLT_MAX) - log_s;
        const float p = expf(logp);
        return empty ? 0.0f : scale * (p * a - p * (logp + entropy) * b);
    }
};

__device__ __forceinline__ LogprobGrad logprob_grad(const RowParams& p, int r, int64_t target,
                                                    float m, float log_s, float entropy, float* g) {
    LogprobGrad o;
    float gl = p.g_logprob && target >= 0 ? p.g_logprob[r] : 0.0f;
    if (target >= p.vocab) gl = __builtin_nanf("");
    o.empty = m == -kInf && log_s == 0.0f && target < p.vocab;
    o.m = m == -kInf ? 0.0f : m;
    o.log_s = log_s;
    o.entropy = entropy;
    o.a = (p.g_lse ? p.g_lse[r] : 0.0f) - gl;
    o.b = p.g_entropy ? p.g_entropy[r] : 0.0f;
    o.scale = p.scale;
    *g = o.empty ? 0.0f : gl * p.scale;
    return o;
}

template <int DT>
__device__ __forceinline__ void write_logprob_grad(const RowParams& p, int r, int64_t target,
                                                   float m, float log_s, float entropy) {
    typedef typename Elem<DT>::type T;
    float own;
    const LogprobGrad f = logprob_grad(p, r, target, m, log_s, entropy, &own);
    const T* x = static_cast<const T*>(p.x) + (size_t)r * p.ld;
    T* dx = static_cast<T*>(p.dx) + (size_t)r * p.ld_grad;
    for (int v = threadIdx.x; v < p.vocab; v += kThreads) {
        const float d = f(Elem<DT>::load(x[v]));
        dx[v] = Elem<DT>::store(v == target ? d + own : d);
    }
}

// One workgroup a row.
template <int DT>
__global__ void __launch_bounds__(kThreads) logprob_kernel(RowParams p) {
    typedef typename Elem<DT>::type T;
    __shared__ float lds[kWaves];
    __shared__ uint64_t lds64[kWaves];
    const int r = blockIdx.x;
    const T* x = static_cast<const T*>(p.x) + (size_t)r * p.ld;
    float m = -kInf;
    for (int v = threadIdx.x; v < p.vocab; v += kThreads) m = fmaxf(m, Elem<DT>::load(x[v]));
    m = block_max(m, lds);
    const float ms = m == -kInf ? 0.0f : m;
    const float c = p.scale * kLog2e;
    float s = 0.0f, t = 0.0f;
    for (int v = threadIdx.x; v < p.vocab; v += kThreads) {
        const float d = Elem<DT>::load(x[v]) - ms;
        const float e = exp_scaled(d, c);
        s += e;
        t += e * fmaxf(d, -FLT_MAX);
    }
    s = block_sum(s, lds);
    t = block_sum(t, lds);
    const bool empty = m == -kInf && s == 0.0f;
    const float log_s = empty ? 0.0f : logf(s);
    const float entropy = empty ? 0.0f : log_s - p.scale * t / s;
    const int64_t target = p.targets ? p.targets[r] : -1;
    auto logp = [&](float xv) {
        return empty ? -kInf : (xv - ms) * p.scale - log_s;
    };
    if (threadIdx.x == 0) {
        if (p.logprob)
            p.logprob[r] = target < 0           ? 0.0f
                           : target >= p.vocab ? __builtin_nanf("")
                                               : logp(Elem<DT>::load(x[target]));
        if (p.entropy) p.entropy[r] = entropy;
        if (p.stats) {
            p.stats[2 * (size_t)r] = m;
            p.stats[2 * (size_t)r + 1] = log_s;
        }
    }
    uint64_t last = ~0ull;
    for (int j = 0; j < p.top; ++j) {
        uint64_t best = 0;
        for (int v = threadIdx.x; v < p.vocab; v += kThreads) {
            const uint64_t key = top_key(Elem<DT>::load(x[v]), v);
            if (key < last && key > best) best = key;
        }
        last = block_reduce(best, lds64, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
        if (threadIdx.x == 0) {
            const int id = key_id(last);
            p.top_ids[(size_t)r * p.top + j] = id;
            p.top_logprobs[(size_t)r * p.top + j] = logp(Elem<DT>::load(x[id]));
        }
    }
    if (p.dx) {
        __syncthreads();   // the target's and the top logits are read before they are overwritten
        write_logprob_grad<DT>(p, r, target, m, log_s, entropy);
    }
}

template <int DT>
__global__ void __launch_bounds__(kThreads) logprob_backward_kernel(RowParams p) {
    const int r = blockIdx.x;
    write_logprob_grad<DT>(p, r, p.targets ? p.targets[r] : -1, p.stats[2 * (size_t)r],
                           p.stats[2 * (size_t)r + 1], p.entropy[r]);
}

// ---- distillation --------------------------------------------------------------
struct List {
    int64_t id[SYMTILE_TOP_MAX];      // negative: absent
    float x[SYMTILE_TOP_MAX];         // the student's logit
    float q[SYMTILE_TOP_MAX];         // the teacher's probability, then the id's sum at its first entry
    float log_q[SYMTILE_TOP_MAX];
    int first[SYMTILE_TOP_MAX];       // 1 at the first entry of an id
    float red[kWaves];
    int bad, some;
};

__device__ __forceinline__ float teacher_value(const RowParams& p, size_t i) {
    switch (p.values_dtype) {
        case SYMTILE_F16: return (float)static_cast<const _Float16*>(p.values)[i];
        case SYMTILE_BF16: return (float)static_cast<const __bf16*>(p.values)[i];
        default: return static_cast<const float*>(p.values)[i];
    }
}

// Fills the list of row r; returns the sum of q and *q_rest.  Ends with a barrier.
template <int DT>
__device__ __forceinline__ float load_list(const RowParams& p, int r, List& l, float* q_rest) {
    typedef typename Elem<DT>::type T;
    const T* x = static_cast<const T*>(p.x) + (size_t)r * p.ld;
    const int j = threadIdx.x;
    if (j == 0) l.bad = l.some = 0;
    __syncthreads();
    int64_t id = -1;
    float v = -kInf;
    if (j < p.k) {
        id = p.ids[(size_t)r * p.k + j];
        if (id >= p.vocab) l.bad = 1;
        if (id >= 0) l.some = 1;
        l.id[j] = id;
        l.x[j] = id >= 0 && id < p.vocab ? Elem<DT>::load(x[id]) : -kInf;
        if (id >= 0) v = teacher_value(p, (size_t)r * p.k + j);
    }
    float q, log_q;
    if (p.mode == SYMTILE_DISTILL_REST) {
        log_q = v;
        q = id >= 0 ? expf(v) : 0.0f;
    } else {
        const float top = block_max(v, l.red);
        const float d = id >= 0 ? (v - (top == -kInf ? 0.0f : top)) * p.scale : -kInf;
        const float e = expf(d);
        const float sum = block_sum(e, l.red);
        log_q = d - logf(sum);
        q = sum == 0.0f ? 0.0f : e / sum;
    }
    const float sum_q = block_sum(j < p.k ? q : 0.0f, l.red);
    if (j < p.k) {
        l.q[j] = q;
        l.log_q[j] = log_q;
    }
    __syncthreads();
    *q_rest = p.mode == SYMTILE_DISTILL_REST && l.some ? fmaxf(1.0f - sum_q, 0.0f) : 0.0f;
    if (j < p.k) {
        int first = id >= 0;
        for (int i = 0; i < j; ++i)
            if (l.id[i] == id) first = 0;
        l.first[j] = first;
    }
    __syncthreads();
    return sum_q;
}

__device__ __forceinline__ bool listed(const List& l, int k, int v) {
    for (int i = 0; i < k; ++i)
        if (l.id[i] == v) return true;
    return false;
}

// stats: m, log s, and the same two over the tokens outside the list.
template <int DT>
__device__ __forceinline__ void write_distill_grad(const RowParams& p, int r, List& l, float sum_q,
                                                   float q_rest, float m, float log_s,
                                                   float m_rest, float log_rest) {
    typedef typename Elem<DT>::type T;
    const T* x = static_cast<const T*>(p.x) + (size_t)r * p.ld;
    T* dx = static_cast<T*>(p.dx) + (size_t)r * p.ld_grad;
    const float g = p.row_grad[r] * p.scale;
    const bool bad = l.bad;
    const bool empty = !bad && (!l.some || (m == -kInf && log_s == 0.0f));
    const bool has_rest = m_rest != -kInf;
    if (!has_rest) q_rest = 0.0f;
    const float all = sum_q + q_rest;
    const float mr = has_rest ? m_rest : 0.0f;
    const float c = p.scale * kLog2e;
    // d of a token outside the list = exp(scale (x - m_rest)) * coef
    const float coef = bad ? __builtin_nanf("")
                           : g * (all * expf((mr - (m == -kInf ? 0.0f : m)) * p.scale - log_s) -
                                  (q_rest > 0.0f ? q_rest * expf(-log_rest) : 0.0f));
    for (int v = threadIdx.x; v < p.vocab; v += kThreads) {
        const float xv = Elem<DT>::load(x[v]);
        if (listed(l, p.k, v)) continue;
        const float e = has_rest ? exp_scaled(xv - mr, c) : 0.0f;
        dx[v] = Elem<DT>::store(empty ? 0.0f : e * coef);
    }
    const int j = threadIdx.x;
    if (j < p.k && l.first[j] && l.id[j] < p.vocab) {
        float q = 0.0f;
        for (int i = 0; i < p.k; ++i)
            if (l.id[i] == l.id[j]) q += l.q[i];
        const float pj = l.x[j] == -kInf ? 0.0f : expf((l.x[j] - m) * p.scale - log_s);
        const float d = bad ? __builtin_nanf("") : g * (all * pj - q);
        dx[l.id[j]] = Elem<DT>::store(empty ? 0.0f : d);
    }
}

template <int DT>
__global__ void __launch_bounds__(kThreads) distill_kernel(RowParams p) {
    typedef typename Elem<DT>::type T;
    __shared__ List l;
    const int r = blockIdx.x, j = threadIdx.x;
    const T* x = static_cast<const T*>(p.x) + (size_t)r * p.ld;
    float q_rest;
    const float sum_q = load_list<DT>(p, r, l, &q_rest);
    float m_rest = -kInf;
    for (int v = threadIdx.x; v < p.vocab; v += kThreads)
        if (!listed(l, p.k, v)) m_rest = fmaxf(m_rest, Elem<DT>::load(x[v]));
    m_rest = block_max(m_rest, l.red);
    const bool mine = j < p.k && l.first[j];
    const float m = fmaxf(m_rest, block_max(mine ? l.x[j] : -kInf, l.red));
    const float mr = m_rest == -kInf ? 0.0f : m_rest, ms = m == -kInf ? 0.0f : m;
    const float c = p.scale * kLog2e;
    float s_rest = 0.0f;
    for (int v = threadIdx.x; v < p.vocab; v += kThreads)
        if (!listed(l, p.k, v)) s_rest += exp_scaled(Elem<DT>::load(x[v]) - mr, c);
    s_rest = block_sum(s_rest, l.red);
    const float s_list = block_sum(mine ? exp_scaled(l.x[j] - ms, c) : 0.0f, l.red);
    const float s = s_list + (m_rest == -kInf ? s_rest : s_rest * exp_scaled(m_rest - ms, c));
    const bool empty = m == -kInf && s == 0.0f;
    const float log_s = l.bad ? __builtin_nanf("") : empty ? 0.0f : logf(s);
    const float log_rest = m_rest == -kInf && s_rest == 0.0f ? 0.0f : logf(s_rest);
    float term = 0.0f;
    if (j < p.k && l.q[j] != 0.0f) {
        const float logp = l.x[j] == -kInf && s == s ? -kInf : (l.x[j] - ms) * p.scale - log_s;
        term = l.q[j] * (l.log_q[j] - logp);
    }
    float loss = block_sum(term, l.red);
    if (q_rest > 0.0f && m_rest != -kInf)
        loss += q_rest * (logf(q_rest) - ((m_rest - ms) * p.scale + log_rest - log_s));
    if (l.bad) loss = __builtin_nanf("");
    if (threadIdx.x == 0) {
        p.loss[r] = loss;
        if (p.stats) {
            float* o = p.stats + 4 * (size_t)r;
            o[0] = m, o[1] = log_s, o[2] = m_rest, o[3] = log_rest;
        }
    }
    if (p.dx) write_distill_grad<DT>(p, r, l, sum_q, q_rest, m, log_s, m_rest, log_rest);
}

template <int DT>
__global__ void __launch_bounds__(kThreads) distill_backward_kernel(RowParams p) {
    __shared__ List l;
    const int r = blockIdx.x;
    float q_rest;
    const float sum_q = load_list<DT>(p, r, l, &q_rest);
    const float* st = p.stats + 4 * (size_t)r;
    write_distill_grad<DT>(p, r, l, sum_q, q_rest, st[0], st[1], st[2], st[3]);
}

// ---- host ----------------------------------------------------------------------
using symtile_host::fail;

size_t elem_size(int dtype) {
    return dtype == SYMTILE_F32 ? 4 : dtype == SYMTILE_F16 || dtype == SYMTILE_BF16 ? 2 : 0;
}

// What every call checks about the logits and fills in about them.
symtile_status fill_logits(RowParams& p, const void* logits, int rows, int vocab, size_t ld,
                           int dtype, float scale) {
    const size_t esize = elem_size(dtype);
    if (!esize) return fail(SYMTILE_EINVAL, "unknown dtype");
    if (rows < 0 || vocab < 1) return fail(SYMTILE_EINVAL, "rows < 0 or vocab < 1");
    if (ld == 0) ld = (size_t)vocab;
    if (ld < (size_t)vocab) return fail(SYMTILE_EINVAL, "ld smaller than vocab");
    if (rows && ld > (SIZE_MAX >> 3) / (size_t)rows)
        return fail(SYMTILE_EINVAL, "logits exceed the address space");
    if (!(scale > 0.0f) || !std::isfinite(scale))
        return fail(SYMTILE_EINVAL, "scale must be positive and finite");
    if (rows && !logits) return fail(SYMTILE_EINVAL, "logits is NULL");
    if (reinterpret_cast<uintptr_t>(logits) % esize)
        return fail(SYMTILE_EINVAL, "logits not aligned to their type");
    p.x = logits;
    p.rows = rows;
    p.vocab = vocab;
    p.ld = ld;
    p.scale = scale;
    return SYMTILE_OK;
}

// The gradient: the logits' own memory, or memory apart from them.
symtile_status fill_grad(RowParams& p, void* dlogits, size_t ld_grad, int dtype) {
    const size_t esize = elem_size(dtype);
    if (ld_grad == 0) ld_grad = (size_t)p.vocab;
    if (ld_grad < (size_t)p.vocab) return fail(SYMTILE_EINVAL, "ld_grad smaller than vocab");
    if (p.rows && ld_grad > (SIZE_MAX >> 3) / (size_t)p.rows)
        return fail(SYMTILE_EINVAL, "dlogits exceed the address space");
    if (reinterpret_cast<uintptr_t>(dlogits) % esize)
        return fail(SYMTILE_EINVAL, "dlogits not aligned to their type");
    if (p.rows && !(dlogits == p.x && ld_grad == p.ld)) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p.x), b = reinterpret_cast<uintptr_t>(dlogits);
        const size_t na = ((size_t)(p.rows - 1) * p.ld + p.vocab) * esize;
        const size_t nb = ((size_t)(p.rows - 1) * ld_grad + p.vocab) * esize;
        if (a < b + nb && b < a + na)
            return fail(SYMTILE_EINVAL, "dlogits overlaps logits without being them");
    }
    p.dx = dlogits;
    p.ld_grad = ld_grad;
    return SYMTILE_OK;
}

symtile_status check_workspace(const void* workspace, size_t bytes, size_t need) {
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
        if (hipGetDevice(&cur) != hipSuccess || cur != device) {
            int n = 0;
            if (hipGetDeviceCount(&n) != hipSuccess || device < 0 || device >= n) {
                status = fail(SYMTILE_EINVAL, "device " + std::to_string(device) + " out of range");
                return;
            }
            const hipError_t e = hipSetDevice(device);
            if (e != hipSuccess) status = symtile_host::hip_fail(e, "hipSetDevice");
            else prev = cur;
        }
    }
    ~OnDevice() {
        if (prev >= 0) (void)hipSetDevice(prev);
    }
};

template <class F>
const void* by_dtype(int dtype, F f) {
    switch (dtype) {
        case SYMTILE_F16: return f(std::integral_constant<int, SYMTILE_F16>{});
        case SYMTILE_BF16: return f(std::integral_constant<int, SYMTILE_BF16>{});
        default: return f(std::integral_constant<int, SYMTILE_F32>{});
    }
}

symtile_status launch(const void* kernel, RowParams& p, symtile_stream s, const char* what) {
    void* args[] = {&p};
    hipError_t e = hipLaunchKernel(kernel, dim3((unsigned)p.rows), dim3(kThreads), args, 0,
                                   static_cast<hipStream_t>(s));
    if (e == hipSuccess) e = hipGetLastError();
    return e == hipSuccess ? SYMTILE_OK : symtile_host::hip_fail(e, what);
}

symtile_status check_top(int top, int vocab) {
    if (top < 0 || top > SYMTILE_TOP_MAX || top > vocab)
        return fail(SYMTILE_EINVAL, "top must be in 0 .. min(vocab, " +
                                        std::to_string(SYMTILE_TOP_MAX) + ")");
    return SYMTILE_OK;
}

symtile_status fill_list(RowParams& p, const int64_t* ids, const void* values, int values_dtype,
                         int k, int mode) {
    if (k < 1 || k > SYMTILE_TOP_MAX)
        return fail(SYMTILE_EINVAL, "k must be in 1 .. " + std::to_string(SYMTILE_TOP_MAX));
    const size_t vsize = elem_size(values_dtype);
    if (!vsize) return fail(SYMTILE_EINVAL, "unknown values_dtype");
    if (mode != SYMTILE_DISTILL_RENORM && mode != SYMTILE_DISTILL_REST)
        return fail(SYMTILE_EINVAL, "unknown mode");
    if (p.rows && (!ids || !values)) return fail(SYMTILE_EINVAL, "ids or values is NULL");
    if (reinterpret_cast<uintptr_t>(ids) % 8 || reinterpret_cast<uintptr_t>(values) % vsize)
        return fail(SYMTILE_EINVAL, "ids or values not aligned to their type");
    p.ids = ids;
    p.values = values;
    p.values_dtype = values_dtype;
    p.k = k;
    p.mode = mode;
    return SYMTILE_OK;
}

}  // namespace

extern "C" symtile_status symtile_logits_workspace_bytes(int device, int rows, int vocab, int dtype,
                                                         int top, size_t* bytes) {
    if (!bytes) return fail(SYMTILE_EINVAL, "bytes is NULL");
    *bytes = 0;
    if (!elem_size(dtype)) return fail(SYMTILE_EINVAL, "unknown dtype");
    if (rows < 0 || vocab < 1) return fail(SYMTILE_EINVAL, "rows < 0 or vocab < 1");
    (void)device;
    return check_top(top, vocab);
}

extern "C" symtile_status symtile_token_logprobs(
    int device, const void* logits, int rows, int vocab, size_t ld, int dtype, float scale,
    const int64_t* targets, float* logprob, float* entropy, float* stats, int top,
    int64_t* top_ids, float* top_logprobs, const float* grad_logprob, const float* grad_entropy,
    const float* grad_lse, void* dlogits, size_t ld_grad, void* workspace, size_t workspace_bytes,
    symtile_stream s) {
    RowParams p{};
    if (symtile_status st = fill_logits(p, logits, rows, vocab, ld, dtype, scale)) return st;
    if (symtile_status st = check_top(top, vocab)) return st;
    if (rows && ((targets == nullptr) != (logprob == nullptr)))
        return fail(SYMTILE_EINVAL, "targets and logprob come together");
    if (rows && top && (!top_ids || !top_logprobs))
        return fail(SYMTILE_EINVAL, "top needs top_ids and top_logprobs");
    if (dlogits) {
        if (symtile_status st = fill_grad(p, dlogits, ld_grad, dtype)) return st;
        if (rows && (!entropy || !stats))
            return fail(SYMTILE_EINVAL, "dlogits needs entropy and stats");
    } else if (grad_logprob || grad_entropy || grad_lse) {
        return fail(SYMTILE_EINVAL, "gradients without dlogits");
    }
    if (grad_logprob && !targets) return fail(SYMTILE_EINVAL, "grad_logprob without targets");
    size_t need = 0;
    if (symtile_status st = symtile_logits_workspace_bytes(device, rows, vocab, dtype, top, &need))
        return st;
    if (symtile_status st = check_workspace(workspace, workspace_bytes, need)) return st;
    if (rows == 0) return SYMTILE_OK;
    p.targets = targets;
    p.logprob = logprob;
    p.entropy = entropy;
    p.stats = stats;
    p.top = top;
    p.top_ids = top_ids;
    p.top_logprobs = top_logprobs;
    p.g_logprob = grad_logprob;
    p.g_entropy = grad_entropy;
    p.g_lse = grad_lse;
    OnDevice on(device);
    if (on.status) return on.status;
    return launch(by_dtype(dtype, [](auto d) {
        return reinterpret_cast<const void*>(&logprob_kernel<decltype(d)::value>);
    }), p, s, "logprob_kernel launch");
}

extern "C" symtile_status symtile_token_logprobs_backward(
    int device, const void* logits, int rows, int vocab, size_t ld, int dtype, float scale,
    const int64_t* targets, const float* entropy, const float* stats, const float* grad_logprob,
    const float* grad_entropy, const float* grad_lse, void* dlogits, size_t ld_grad,
    symtile_stream s) {
    RowParams p{};
    if (symtile_status st = fill_logits(p, logits, rows, vocab, ld, dtype, scale)) return st;
    if (rows && !dlogits) return fail(SYMTILE_EINVAL, "dlogits is NULL");
    if (symtile_status st = fill_grad(p, dlogits, ld_grad, dtype)) return st;
    if (rows && (!entropy || !stats)) return fail(SYMTILE_EINVAL, "entropy or stats is NULL");
    if (grad_logprob && !targets) return fail(SYMTILE_EINVAL, "grad_logprob without targets");
    if (rows == 0) return SYMTILE_OK;
    p.targets = targets;
    p.entropy = const_cast<float*>(entropy);
    p.stats = const_cast<float*>(stats);
    p.g_logprob = grad_logprob;
    p.g_entropy = grad_entropy;
    p.g_lse = grad_lse;
    OnDevice on(device);
    if (on.status) return on.status;
    return launch(by_dtype(dtype, [](auto d) {
        return reinterpret_cast<const void*>(&logprob_backward_kernel<decltype(d)::value>);
    }), p, s, "logprob_backward_kernel launch");
}

extern "C" symtile_status symtile_distill_topk(int device, const void* logits, int rows, int vocab,
                                               size_t ld, int dtype, float scale,
                                               const int64_t* ids, const void* values,
                                               int values_dtype, int k, int mode, float* loss,
                                               float* stats, const float* row_grad, void* dlogits,
                                               size_t ld_grad, void* workspace,
                                               size_t workspace_bytes, symtile_stream s) {
    RowParams p{};
    if (symtile_status st = fill_logits(p, logits, rows, vocab, ld, dtype, scale)) return st;
    if (symtile_status st = fill_list(p, ids, values, values_dtype, k, mode)) return st;
    if (rows && !loss) return fail(SYMTILE_EINVAL, "loss is NULL");
    if (dlogits) {
        if (symtile_status st = fill_grad(p, dlogits, ld_grad, dtype)) return st;
        if (rows && (!row_grad || !stats))
            return fail(SYMTILE_EINVAL, "dlogits needs row_grad and stats");
    } else if (row_grad) {
        return fail(SYMTILE_EINVAL, "row_grad without dlogits");
    }
    size_t need = 0;
    if (symtile_status st = symtile_logits_workspace_bytes(device, rows, vocab, dtype, 0, &need))
        return st;
    if (symtile_status st = check_workspace(workspace, workspace_bytes, need)) return st;
    if (rows == 0) return SYMTILE_OK;
    p.loss = loss;
    p.stats = stats;
    p.row_grad = row_grad;
    OnDevice on(device);
    if (on.status) return on.status;
    return launch(by_dtype(dtype, [](auto d) {
        return reinterpret_cast<const void*>(&distill_kernel<decltype(d)::value>);
    }), p, s, "distill_kernel launch");
}

extern "C" symtile_status symtile_distill_topk_backward(
    int device, const void* logits, int rows, int vocab, size_t ld, int dtype, float scale,
    const int64_t* ids, const void* values, int values_dtype, int k, int mode, const float* stats,
    const float* row_grad, void* dlogits, size_t ld_grad, symtile_stream s) {
    RowParams p{};
    if (symtile_status st = fill_logits(p, logits, rows, vocab, ld, dtype, scale)) return st;
    if (symtile_status st = fill_list(p, ids, values, values_dtype, k, mode)) return st;
    if (rows && !dlogits) return fail(SYMTILE_EINVAL, "dlogits is NULL");
    if (symtile_status st = fill_grad(p, dlogits, ld_grad, dtype)) return st;
    if (rows && (!stats || !row_grad)) return fail(SYMTILE_EINVAL, "stats or row_grad is NULL");
    if (rows == 0) return SYMTILE_OK;
    p.stats = const_cast<float*>(stats);
    p.row_grad = row_grad;
    OnDevice on(device);
    if (on.status) return on.status;
    return launch(by_dtype(dtype, [](auto d) {
        return reinterpret_cast<const void*>(&distill_backward_kernel<decltype(d)::value>);
    }), p, s, "distill_backward_kernel launch");
}
