// The distillation loss against a teacher's top entries and its gradient, from
// rows of logits.
//
// With the list's tokens apart, a row needs the largest logit m_R and the sum
// s_R = sum exp(scale (x_v - m_R)) over the tokens outside the list, and the
// listed tokens' logits: s = s_R exp(scale (m_R - m)) + sum over the list.  That
// gives log p of the listed tokens and of the rest without a difference of
// nearly equal sums.  The gradient of a token outside the list,
//   scale g (Q p_v - q_R p_v / p_R) = e_v * (scale g (Q exp(..) / s - q_R / s_R)),
// e_v = exp(scale (x_v - m_R)), is its exponential times a constant of the row.
//
// Listed tokens are found through a bit for each token of the segment in LDS, and
// their logits replaced by -inf in registers: they drop out of the sums, and the
// gradient's main pass writes 0 there.  The thread that wrote it overwrites it: every
// thread has a chain of the list's entries in its vectors.
#include "logits_rows.h"
#include "symtile_device.h"

namespace {

using namespace logits;

constexpr int kMaxK = SYMTILE_TOP_MAX;

enum Phase { kValues, kStep, kGrad };   // the loss, both (whole rows), the gradient

struct DistillParams {
    const void* x;
    void* dx;
    const int64_t* ids;
    const void* values;
    float *loss, *stats;
    const float* row_grad;
    uint32_t* counters;
    float* partials;
    size_t ld, ld_grad;
    symtile_host::Div by_segs;
    int row0, vocab, segs, seg_len, k, mode, values_dtype;
    float scale;
};

// The list of a row.  An id that is absent is -1, one outside the vocabulary -2.
struct __attribute__((aligned(16))) List {
    int id[kMaxK];
    float q[kMaxK];
    float x[kMaxK];            // the student's logit
    float q_id[kMaxK];         // sum of q over the entries of the id; -1: not the first of them
    int next[kMaxK];           // the chains
    float m[kMaxWaves], s[kMaxWaves];
    float sum_q, q_rest;
    float coef, all;           // of the gradient
    float g, m_all, log_s;
    int bad, some, repeated, last, zero;
};

__device__ __forceinline__ float teacher_value(const DistillParams& p, size_t i) {
    switch (p.values_dtype) {
        case SYMTILE_F16: return (float)static_cast<const _Float16*>(p.values)[i];
        case SYMTILE_BF16: return (float)static_cast<const __bf16*>(p.values)[i];
        default: return static_cast<const float*>(p.values)[i];
    }
}

// What the first wave knows of the list: lane l holds entries l and l + 64.
struct Entries {
    int id[2];
    float value[2], x[2], q[2], log_q[2], q_id[2];
    bool first[2];      // the first entry of its id
};

// In 64 bits, as the list's exponentials are: the rest's probability is what they
// leave of 1.
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// The teacher's probabilities, by the first wave.  `search`: look for entries that
// name the same id (they count once in the student's sum, together in q).
__device__ __forceinline__ void teacher(const DistillParams& p, Entries& e, List& l, bool search) {
    const int lane = threadIdx.x;
    float sum_q = 0.0f, q_rest = 0.0f;
    const bool some = l.some != 0;
    if (p.mode == SYMTILE_DISTILL_REST) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const double q = e.id[i] != -1 ? exp((double)e.value[i]) : 0.0;
            e.q[i] = (float)q;
            e.log_q[i] = e.value[i];
            sum += q;
        }
        sum = wave_sum64(sum);
        sum_q = (float)sum;
        q_rest = some ? fmaxf((float)(1.0 - sum), 0.0f) : 0.0f;
    } else {
        const float top = wave_max(max3(e.value[0], e.value[1], e.value[1]));
        float d[2], ex[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            d[i] = e.id[i] != -1 ? (e.value[i] - (top == -kInf ? 0.0f : top)) * p.scale : -kInf;
            ex[i] = expf(d[i]);
        }
        const float sum = wave_sum(ex[0] + ex[1]);
        const float log_sum = logf(sum);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            e.q[i] = sum == 0.0f ? 0.0f : ex[i] / sum;
            e.log_q[i] = d[i] - log_sum;
        }
        sum_q = wave_sum(e.q[0] + e.q[1]);
    }
    if (lane == 0) {
        l.sum_q = sum_q;
        l.q_rest = q_rest;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        e.first[i] = e.id[i] >= 0;
        e.q_id[i] = e.q[i];
        l.q[lane + 64 * i] = e.q[i];
    }
    __builtin_amdgcn_wave_barrier();   // the wave reads what its lanes wrote
    if (search) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = lane + 64 * i;
            float sum = 0.0f;
#pragma unroll 4
            for (int o = 0; o < kMaxK; ++o)     // (behind the list stand absent ones)
                if (l.id[o] == e.id[i]) {
                    sum += l.q[o];
                    if (o < j) e.first[i] = false;
                }
            e.q_id[i] = sum;
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) l.q_id[lane + 64 * i] = e.first[i] ? e.q_id[i] : -1.0f;
    __builtin_amdgcn_wave_barrier();
}

// The row's constants of the gradient, by every lane of the first wave.
__device__ __forceinline__ void gradient_constants(const DistillParams& p, int r, List& l, float m,
                                                   float log_s, float m_rest, float log_rest) {
    const float g = p.row_grad[r] * p.scale;
    const bool bad = l.bad != 0;
    const bool zero = !bad && (!l.some || (m == -kInf && log_s == 0.0f));
    const bool has_rest = m_rest != -kInf;
    const float q_rest = has_rest ? l.q_rest : 0.0f;
    const float all = l.sum_q + q_rest;
    float coef = 0.0f;
    if (has_rest)
        coef = g * (all * expf((m_rest - m) * p.scale - log_s) -
                    (q_rest > 0.0f ? q_rest * expf(-log_rest) : 0.0f));
    // without a rest every e_v is 0 or, in a row that is not a number, undefined
    else if (!(log_s == log_s)) coef = __builtin_nanf("");
    if (threadIdx.x == 0) {
        l.coef = zero ? 0.0f : bad ? __builtin_nanf("") : coef;
        l.g = zero ? 0.0f : bad ? __builtin_nanf("") : g;
        l.zero = zero;
        l.all = all;
        l.m_all = m == -kInf ? 0.0f : m;
        l.log_s = log_s;
    }
}

template <int DT, int NV, bool HUGE>
__device__ __forceinline__ float rest_sum(Segment<DT, NV>& d, const Exponent& ex) {
    d.again();
    float s0 = 0.0f, s1 = 0.0f;
    d.each([&](int, int e, float x) {
        const float v = exp2_fast(ex.template y<HUGE>(x));
        if (e % 2) s1 += v;
        else s0 += v;
    });
    return s0 + s1;
}

// READ: whether the registers were read in a pass before.
template <int DT, int NV, bool HUGE, bool READ>
__device__ __forceinline__ void write_rest(Segment<DT, NV>& d,
                                           typename Elem<DT>::type* __restrict__ dx, int len,
                                           float coef, const Exponent& ex) {
    constexpr int kVec = Elem<DT>::kVec;
    const int threads = blockDim.x;
    if constexpr (READ) d.again();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = (i * threads + (int)threadIdx.x) * kVec;
        float f[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            f[e] = exp2_fast(ex.template y<HUGE>(element<DT>(d.v[i], e))) * coef;
        Segment<DT, NV>::store(dx, len, at, pack<DT>(f));
    }
}

// A workgroup per row or segment; its logits come once from memory.  Memory bounds it:
// loss and gradient of 4096 rows of 28672 in bfloat16 94 us (5.0 TB/s), of 1000 rows of
// 50001 in float32 100 us (4.0 TB/s).  Where one workgroup of 1024 threads fills a CU
// (1024 rows of 131072 bfloat16: 135 us, 4.0 TB/s) loading, sums and storing of a row
// follow each other with nothing beside them; in segments the logits would be read
// twice.  64 rows of 8192 take 4.3 us, an empty kernel 2.9.
// The loss alone of rows that are split is bound by the list instead, since every
// segment takes it anew (exponentials, search for repeated ids, the listed logits) ahead
// of a barrier: 1024 rows of 131072 bfloat16 124 us, 1000 of 50257 float32 102 us, where
// token_logprobs takes 53 and 40 for the same logits; whole rows, 4096 of 28672
// bfloat16: 48 us (5.0 TB/s).
template <int DT, int NV, int PHASE>
__global__ void __launch_bounds__(kMaxThreads) distill_kernel(DistillParams p) {
    typedef typename Elem<DT>::type T;
    constexpr int kVec = Elem<DT>::kVec;
    extern __shared__ __attribute__((aligned(16))) uint32_t bits[];
    __shared__ List l;
    const int t = threadIdx.x, threads = blockDim.x, waves = threads / 64;
    const bool first_wave = t < 64;
    const int local = p.by_segs(blockIdx.x), seg = blockIdx.x - local * p.segs;
    const int r = p.row0 + local;
    const int id0 = seg * p.seg_len, len = min(p.seg_len, p.vocab - id0);
    const T* row = static_cast<const T*>(p.x) + (size_t)r * p.ld;
    const int words = (p.seg_len + 31) / 32;
    int* chain = reinterpret_cast<int*>(bits + words);   // a thread's first entry, -1: none
    // the list first: its tokens' logits wait for the ids
    Entries en;
    int64_t wide[2] = {-1, -1};
    if (first_wave) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = t + 64 * i;
            en.value[i] = -kInf;
            if (j < p.k) {
                wide[i] = p.ids[(size_t)r * p.k + j];
                en.value[i] = teacher_value(p, (size_t)r * p.k + j);
            }
        }
    }
    Segment<DT, NV> d;
    d.load(row + id0, len, threads);
    for (int i = t; i < words; i += threads) bits[i] = 0;
    if constexpr (PHASE != kValues) chain[t] = -1;
    __syncthreads();
    if (first_wave) {
        bool bad = false, some = false, repeated = false;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = t + 64 * i;
            en.id[i] = wide[i] < 0 ? -1 : wide[i] >= p.vocab ? -2 : (int)wide[i];
            if (en.id[i] == -1) en.value[i] = -kInf;
            bad |= en.id[i] == -2;
            some |= en.id[i] != -1;
            l.id[j] = en.id[i];
            // read before anything is written: the gradient may overwrite it
            en.x[i] = en.id[i] >= 0 ? (float)row[en.id[i]] : -kInf;
            const unsigned in = (unsigned)(en.id[i] - id0);
            if (en.id[i] >= 0 && in < (unsigned)len) {
                repeated |= atomicOr(&bits[in / 32], 1u << in % 32) >> in % 32 & 1u;
                if constexpr (PHASE != kValues)
                    l.next[j] = atomicExch(&chain[in / kVec % (unsigned)threads], j);
            }
        }
        bad = __any(bad);
        some = __any(some);
        repeated = __any(repeated);
        if (t == 0) {
            l.bad = bad;
            l.some = some;
            l.repeated = repeated;
        }
    }
    __syncthreads();
    if (first_wave) {
        // of a split row's loss all entries count, also those of other segments
        teacher(p, en, l, l.repeated || (PHASE == kValues && p.segs > 1));
        if constexpr (PHASE != kValues) {
            l.x[t] = en.x[0];
            l.x[t + 64] = en.x[1];
        }
    }
    const uint8_t* bytes = reinterpret_cast<const uint8_t*>(bits);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int vec = i * threads + t;
        if (vec * kVec >= len) break;
        const uint32_t here = kVec == 8 ? bytes[vec] : bytes[vec / 2] >> (4 * (vec & 1)) & 15u;
        if (here) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                if (!(here >> e & 1)) continue;
                if constexpr (DT == SYMTILE_F32)
                    d.v[i][e] = Elem<DT>::kMasked;
                else if (e % 2)
                    d.v[i][e / 2] = (d.v[i][e / 2] & 0xFFFFu) | (Elem<DT>::kMasked & 0xFFFF0000u);
                else
                    d.v[i][e / 2] = (d.v[i][e / 2] & 0xFFFF0000u) | (Elem<DT>::kMasked & 0xFFFFu);
            }
        }
    }
    float m_rest;
    if constexpr (PHASE == kGrad) {
        const float* st = p.stats + 4 * (size_t)r;
        m_rest = st[2];
        if (first_wave) gradient_constants(p, r, l, st[0], st[1], m_rest, st[3]);
        __syncthreads();
    } else {
        float vec_max[NV];
        m_rest = wave_max(d.thread_max(vec_max));
        if (t % 64 == 0) l.m[t / 64] = m_rest;
        __syncthreads();
        m_rest = waves_max(l.m, waves);
        const Exponent ex(m_rest, p.scale);
        float s = ex.huge ? rest_sum<DT, NV, true>(d, ex) : rest_sum<DT, NV, false>(d, ex);
        s = wave_sum(s);
        if (t % 64 == 0) l.s[t / 64] = s;
        __syncthreads();
        if (p.segs > 1) {
            const float sum = waves_sum(l.s, waves) * exp2f(-ex.shift);
            if (t == 0) {
                float* o = p.partials + 4 * ((size_t)local * p.segs + seg);
                put(o, m_rest);
                put(o + 1, sum);
            }
            if (!arrive_last(p.counters + local, p.segs, &l.last)) return;
        }
        float ms = 0.0f, m = 0.0f, log_s = 0.0f, log_rest = 0.0f, log_p_rest = 0.0f;
        bool empty = false;
        if (first_wave) {
            float s_rest;
            if (p.segs > 1) {
                const float* o = p.partials + 4 * (size_t)local * p.segs;
                const bool there = t < p.segs;
                const float mine = there ? take(o + 4 * t) : -kInf;
                const float sum = there ? take(o + 4 * t + 1) : 0.0f;
                m_rest = wave_max(mine);
                s_rest = wave_sum(mine == -kInf || mine == m_rest
                                      ? sum
                                      : sum * expf((mine - m_rest) * p.scale));
            } else {
                s_rest = waves_sum(l.s, waves) * exp2f(-ex.shift);
            }
            const float x0 = en.first[0] ? en.x[0] : -kInf, x1 = en.first[1] ? en.x[1] : -kInf;
            m = max3(m_rest, wave_max(max3(x0, x1, x1)), -kInf);
            ms = m == -kInf ? 0.0f : m;
            const float s_list = wave_sum((en.first[0] ? expf((en.x[0] - ms) * p.scale) : 0.0f) +
                                          (en.first[1] ? expf((en.x[1] - ms) * p.scale) : 0.0f));
            const float s_part =
                m_rest == -kInf ? s_rest : s_rest * expf((m_rest - ms) * p.scale);
            const float s_all = s_list + s_part;
            empty = m == -kInf && s_all == 0.0f;
            log_s = l.bad ? __builtin_nanf("") : empty ? 0.0f : logf(s_all);
            log_rest = m_rest == -kInf && s_rest == 0.0f ? 0.0f : logf(s_rest);
            // log p_R from the ratio, unless that vanishes: the logarithms' difference would
            // carry their own roundings into a loss that is small against them
            const float share = s_part / s_all;
            log_p_rest = share > 1e-30f ? logf(share)
                                        : (m_rest - ms) * p.scale + log_rest - log_s;
            if constexpr (PHASE == kStep) gradient_constants(p, r, l, m, log_s, m_rest, log_rest);
        }
        if constexpr (PHASE == kStep) __syncthreads();
        if (first_wave) {   // the loss, while the other waves go on
            float term = 0.0f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (en.q[i] != 0.0f) {
                    const float logp = empty ? -kInf : (en.x[i] - ms) * p.scale - log_s;
                    term += en.q[i] * (en.log_q[i] - logp);
                }
            float loss = wave_sum(term);
            const float q_rest = l.q_rest;
            if (q_rest > 0.0f && m_rest != -kInf)
                loss += q_rest * (logf(q_rest) - log_p_rest);
            if (l.bad) loss = __builtin_nanf("");
            if (t == 0) {
                p.loss[r] = loss;
                if (p.stats) {
                    float* o = p.stats + 4 * (size_t)r;
                    o[0] = m, o[1] = log_s, o[2] = m_rest, o[3] = log_rest;
                }
            }
        }
    }
    if constexpr (PHASE != kValues) {
        T* dx = static_cast<T*>(p.dx) + (size_t)r * p.ld_grad + id0;
        const Exponent ex(m_rest, p.scale);
        const float coef = l.coef * exp2f(-ex.shift);
        if (l.zero) {
            const float none[kVec] = {};
            for (int i = 0; i < NV; ++i)
                Segment<DT, NV>::store(dx, len, (i * threads + t) * kVec, pack<DT>(none));
        } else if (ex.huge) write_rest<DT, NV, true, PHASE == kStep>(d, dx, len, coef, ex);
        else write_rest<DT, NV, false, PHASE == kStep>(d, dx, len, coef, ex);
        for (int j = chain[t]; j >= 0; j = l.next[j]) {
            if (l.q_id[j] < 0.0f) continue;
            const float x = l.x[j];
            const float pj = x == -kInf ? 0.0f : expf((x - l.m_all) * p.scale - l.log_s);
            dx[l.id[j] - id0] = (T)(l.g * (l.all * pj - l.q_id[j]));
        }
    }
}

template <int PHASE>
const void* kernel_of(int dtype, int nv) {
    return pick(dtype, nv, [](auto d, auto n) {
        return reinterpret_cast<const void*>(
            &distill_kernel<decltype(d)::value, decltype(n)::value, PHASE>);
    });
}

// A kernel over rows first .. first + rows - 1, in launches of rows_a_launch().
symtile_status run(DistillParams p, const Plan& plan, int first, int rows, const void* kernel,
                   symtile_stream s, const char* what) {
    p.segs = plan.segs;
    p.seg_len = plan.seg_len;
    p.by_segs = symtile_host::make_div(plan.segs);
    const size_t lds = (size_t)(plan.seg_len + 31) / 32 * 4 + (size_t)plan.threads * 4;
    const int most = rows_a_launch(plan);
    for (int row = 0; row < rows; row += most) {
        p.row0 = first + row;
        if (symtile_status st = launch(kernel, plan, std::min(most, rows - row), lds, p, s, what))
            return st;
    }
    return SYMTILE_OK;
}

symtile_status check_list(const int64_t* ids, const void* values, int values_dtype, int rows, int k,
                          int mode) {
    if (k < 1 || k > SYMTILE_TOP_MAX)
        return fail(SYMTILE_EINVAL, "k must be in 1 .. " + std::to_string(SYMTILE_TOP_MAX));
    const size_t vsize = elem_size(values_dtype);
    if (!vsize) return fail(SYMTILE_EINVAL, "unknown values_dtype");
    if (mode != SYMTILE_DISTILL_RENORM && mode != SYMTILE_DISTILL_REST)
        return fail(SYMTILE_EINVAL, "unknown mode");
    if (rows && (!ids || !values)) return fail(SYMTILE_EINVAL, "ids or values is NULL");
    if (reinterpret_cast<uintptr_t>(ids) % 8 || reinterpret_cast<uintptr_t>(values) % vsize)
        return fail(SYMTILE_EINVAL, "ids or values not aligned to their type");
    return SYMTILE_OK;
}

}  // namespace

extern "C" symtile_status symtile_distill_topk(int device, const void* logits, int rows, int vocab,
                                               size_t ld, int dtype, float scale,
                                               const int64_t* ids, const void* values,
                                               int values_dtype, int k, int mode, float* loss,
                                               float* stats, const float* row_grad, void* dlogits,
                                               size_t ld_grad, void* workspace,
                                               size_t workspace_bytes, symtile_stream s) {
    if (symtile_status st = check_sizes(rows, vocab, dtype, 0)) return st;
    if (symtile_status st = check_logits(logits, rows, vocab, &ld, dtype, scale)) return st;
    if (symtile_status st = check_list(ids, values, values_dtype, rows, k, mode)) return st;
    if (rows && !loss) return fail(SYMTILE_EINVAL, "loss is NULL");
    if (dlogits) {
        if (symtile_status st = check_grad(logits, ld, dlogits, &ld_grad, rows, vocab, dtype))
            return st;
        if (rows && (!row_grad || !stats))
            return fail(SYMTILE_EINVAL, "dlogits needs row_grad and stats");
    } else if (row_grad) {
        return fail(SYMTILE_EINVAL, "row_grad without dlogits");
    }
    const Plan plan = make_plan(device, rows, vocab, dtype, dlogits != nullptr, 0);
    const Workspace ws = make_workspace(plan, rows, 0);
    if (symtile_status st = check_workspace(workspace, workspace_bytes, ws.bytes)) return st;
    if (rows == 0) return SYMTILE_OK;
    DistillParams p{};
    p.x = logits;
    p.dx = dlogits;
    p.ids = ids;
    p.values = values;
    p.loss = loss;
    p.stats = stats;
    p.row_grad = row_grad;
    p.ld = ld;
    p.ld_grad = ld_grad;
    p.vocab = vocab;
    p.k = k;
    p.mode = mode;
    p.values_dtype = values_dtype;
    p.scale = scale;
    if (ws.bytes) {
        p.counters = static_cast<uint32_t*>(workspace);
        p.partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + ws.partials);
    }
    OnDevice on(device);
    if (on.status) return on.status;
    const char* what = "distill_kernel launch";
    if (dlogits && plan.segs == 1)
        return run(p, plan, 0, rows, kernel_of<kStep>(dtype, plan.nv), s, what);
    if (symtile_status st = run(p, plan, 0, rows, kernel_of<kValues>(dtype, plan.nv), s, what))
        return st;
    if (!dlogits) return SYMTILE_OK;
    return run(p, plan, 0, rows, kernel_of<kGrad>(dtype, plan.nv), s, what);
}

extern "C" symtile_status symtile_distill_topk_backward(
    int device, const void* logits, int rows, int vocab, size_t ld, int dtype, float scale,
    const int64_t* ids, const void* values, int values_dtype, int k, int mode, const float* stats,
    const float* row_grad, void* dlogits, size_t ld_grad, symtile_stream s) {
    if (symtile_status st = check_sizes(rows, vocab, dtype, 0)) return st;
    if (symtile_status st = check_logits(logits, rows, vocab, &ld, dtype, scale)) return st;
    if (symtile_status st = check_list(ids, values, values_dtype, rows, k, mode)) return st;
    if (rows && !dlogits) return fail(SYMTILE_EINVAL, "dlogits is NULL");
    if (symtile_status st = check_grad(logits, ld, dlogits, &ld_grad, rows, vocab, dtype)) return st;
    if (rows && (!stats || !row_grad)) return fail(SYMTILE_EINVAL, "stats or row_grad is NULL");
    if (rows == 0) return SYMTILE_OK;
    DistillParams p{};
    p.x = logits;
    p.dx = dlogits;
    p.ids = ids;
    p.values = values;
    p.stats = const_cast<float*>(stats);
    p.row_grad = row_grad;
    p.ld = ld;
    p.ld_grad = ld_grad;
    p.vocab = vocab;
    p.k = k;
    p.mode = mode;
    p.values_dtype = values_dtype;
    p.scale = scale;
    OnDevice on(device);
    if (on.status) return on.status;
    const Plan plan = make_plan(device, rows, vocab, dtype, true, 0);
    return run(p, plan, 0, rows, kernel_of<kGrad>(dtype, plan.nv), s,
               "distill_kernel launch (gradient)");
}
