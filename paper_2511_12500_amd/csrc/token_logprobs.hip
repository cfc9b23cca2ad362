// Log probabilities of given tokens, entropies, the most likely tokens, and
// their gradient, from rows of logits.
//
// With y_v = c (x_v - m) (base 2, logits_rows.h), e_v = 2^y_v, s = sum e_v and
// t = sum e_v y_v over a row:
//   logp_v = ln 2 (y_v - log2 s),   H = ln 2 (log2 s - t / s),
//   d_v = scale (p_v (g_lse - g_lp) - p_v (logp_v + H) g_H) + [v = target] scale g_lp
//       = e_v (A + B y_v) + [v = target] scale g_lp,
// so the gradient of a logit is one more exponential of it and two constants of
// its row.
#include "logits_rows.h"
#include "symtile_device.h"

namespace {

using namespace logits;

typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
constexpr int kCap = 512;           // candidates for the top entries of a segment
constexpr int kCapVecs = 256;       // vectors that hold the candidates in the usual case

enum Phase { kValues, kStep, kGrad };   // the values, both (whole rows), the gradient

struct LogprobParams {
    const void* x;
    void* dx;
    size_t ld, ld_grad;
    const int64_t* targets;
    float *logprob, *entropy, *stats;
    int64_t* top_ids;
    float* top_logprobs;
    const float *g_logprob, *g_entropy, *g_lse;
    uint32_t* counters;
    float* partials;
    uint64_t* keys;
    symtile_host::Div by_segs;
    int row0, vocab, top, segs, seg_len;
    float scale;
};

struct Shared {
    float m[kMaxWaves], s[kMaxWaves], t[kMaxWaves];
    float tau;
    uint32_t count[2][kMaxWaves];
    float x_target;
    int n, vecs, last;
    uint64_t bound;
};

// Dynamic LDS of the top entries: keys, and the vectors that hold the candidates.
// Before there are keys, groups' largest logits stand in their place.  Behind the keys
// zeros fill up a step of all threads that count for one key.
struct TopLds {
    static constexpr int kPad = 32;
    union {
        uint64_t* keys;
        uint32_t* groups;
    };
    symtile::u32x4* vec;
    int* at;               // first element of each
    static size_t bytes(int segs, int top) {
        return (size_t)(std::max(kCap, segs * top) + kPad) * 8 + kCapVecs * 20;
    }
    __device__ __forceinline__ TopLds(void* base, int segs, int top) {
        vec = static_cast<symtile::u32x4*>(base);
        at = reinterpret_cast<int*>(vec + kCapVecs);
        keys = reinterpret_cast<uint64_t*>(at + kCapVecs);
    }
};

// ---- the order of the top entries ------------------------------------------------
// As whole numbers: the larger logit first (a NaN above all, -0 as +0), then the
// smaller id.  0 is below every logit.
__device__ __forceinline__ uint32_t order(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return x != x ? 0xFFFFFFFFu : o;
}
__device__ __forceinline__ float ordered_value(uint32_t o) {
    return __uint_as_float(o == 0xFFFFFFFFu ? 0x7FC00000u
                           : o & 0x80000000u ? o ^ 0x80000000u
                                             : ~o);
}
__device__ __forceinline__ uint64_t top_key(uint32_t o, int id) {
    return (uint64_t)o << 32 | (0xFFFFFFFFu - (uint32_t)id);
}
__device__ __forceinline__ int key_id(uint64_t key) { return (int)(0xFFFFFFFFu - (uint32_t)key); }

// Sum over the workgroup; `step` alternates between the two arrays, so that one
// barrier a call is enough.
__device__ __forceinline__ uint32_t block_count(uint32_t c, Shared& sh, int& step, int waves) {
    c = wave_sum_u32(c);
    uint32_t* a = sh.count[step & 1];
    ++step;
    if (threadIdx.x % 64 == 0) a[threadIdx.x / 64] = c;
    __syncthreads();
    uint32_t n = 0;
    for (int w = 0; w < waves; ++w) n += a[w];
    return n;
}

// Sum over `lanes` (1, 2, 4, 8 or 16) neighbouring lanes that begin at a multiple of them.
__device__ __forceinline__ uint32_t sum_lanes(uint32_t c, int lanes) {
    auto add = [](uint32_t v, float o) { return v + __float_as_uint(o); };
    if (lanes > 1) c = add(c, dpp<0xB1>(__uint_as_float(c)));
    if (lanes > 2) c = add(c, dpp<0x4E>(__uint_as_float(c)));
    if (lanes > 4) c = add(c, dpp<0x141>(__uint_as_float(c)));
    if (lanes > 8) c = add(c, dpp<0x140>(__uint_as_float(c)));
    return c;
}

// n distinct keys in LDS; calls emit(place, key) for the `keep` largest.  The
// place is the number of larger keys, counted by up to 16 neighbouring threads a key,
// two keys a read.  All threads call it after a barrier behind the last key.
template <class F>
__device__ __forceinline__ void rank_keys(uint64_t* keys, int n, int keep, F emit) {
    const int threads = blockDim.x, t = threadIdx.x;
    if (t < TopLds::kPad) keys[n + t] = 0;
    __syncthreads();
    int lg = 0;
    while (lg < 4 && n << (lg + 1) <= threads) ++lg;
    const int lanes = 1 << lg, part = t & (lanes - 1);
    for (int i = t >> lg; i - (t >> lg) < n; i += threads >> lg) {
        const uint64_t mine = i < n ? keys[i] : ~0ull;
        uint32_t c = 0;
        const u64x2* pairs = reinterpret_cast<const u64x2*>(keys) + part;
        // unrolled: one after the other, each would wait for its own read
#pragma unroll 4
        for (int left = n; left > 0; left -= 2 * lanes, pairs += lanes) {
            const u64x2 k = *pairs;
            c += k[0] > mine;
            c += k[1] > mine;
        }
        c = sum_lanes(c, lanes);
        if (part == 0 && i < n && (int)c < keep) emit((int)c, mine);
    }
}

// The bound for the top entries: the `top`-th largest of the largest logits of groups
// of lanes, which as many elements reach as there are groups above it, and hardly
// more.  Groups are rows of 16 lanes, quads, pairs or single lanes, so that there are
// some more than `top` of them.
__device__ __forceinline__ int group_lanes(int top, int waves) {
    return top <= 3 * waves ? 16 : top <= 14 * waves ? 4 : top <= 28 * waves ? 2 : 1;
}
// A group's largest logit in the order of the top entries, to the bits that its index
// leaves: distinct, so that exactly one group is the top-th.
constexpr uint32_t kIndexBits = kMaxThreads - 1;
__device__ __forceinline__ uint32_t group_key(float largest, int index) {
    return (order(largest) & ~kIndexBits) | (uint32_t)index;
}
// The group's lanes count the groups above its own, `mine`, four a read; the group that
// is the top-th sets sh.tau (-inf before).  All threads' work, and two instructions a
// group: the selection is bound by the instructions of all of its steps (4096 rows of
// 28672 bf16: 46 us without top entries, 57 with 20 and 65 with 64 of them).
__device__ __forceinline__ void find_bound(const uint32_t* groups, uint32_t mine, int group, int top,
                                           Shared& sh) {
    const int t = threadIdx.x, quads = (int)blockDim.x / group / 4, part = t % group;
    uint32_t above = 0;
#pragma unroll 4
    for (int i = part; i < quads; i += group) {
        const symtile::u32x4 g = reinterpret_cast<const symtile::u32x4*>(groups)[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) above += g[e] > mine;
    }
    above = sum_lanes(above, group);
    // 0x00800000: the lowest finite number's place
    if (part == 0 && (int)above == top - 1 && mine >= 0x00800000u)
        sh.tau = ordered_value(mine & ~kIndexBits);
}

// The thread's vectors that hold an element which reaches the bound, into LDS
// (sh.vecs is zero before and counts them).  Counted by scalar instructions, with one
// addition to sh.vecs a wave.
template <int DT, int NV>
__device__ __forceinline__ void stage_candidates(const Segment<DT, NV>& d, const float* vec_max,
                                                 float tau, Shared& sh, const TopLds& top) {
    uint64_t hits[NV];
    int all = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        hits[i] = __ballot(vec_max[i] >= tau);
        all += __popcll(hits[i]);
    }
    if (!all) return;
    int base = 0;
    if (threadIdx.x % 64 == 0) base = atomicAdd(&sh.vecs, all);
    base = __builtin_amdgcn_readfirstlane(base);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (!hits[i]) continue;
        const int place = base + (int)__builtin_amdgcn_mbcnt_hi(
                                     (uint32_t)(hits[i] >> 32),
                                     __builtin_amdgcn_mbcnt_lo((uint32_t)hits[i], 0));
        if (vec_max[i] >= tau && place < kCapVecs) {
            top.vec[place] = d.v[i];
            top.at[place] = (i * (int)blockDim.x + (int)threadIdx.x) * Elem<DT>::kVec;
        }
        base += __popcll(hits[i]);
    }
}

// The `keep` largest of the `len` elements at `seg` (keep <= len), as keys with ids
// from `id0` on, to emit(place, key).  All threads call it after a barrier behind
// stage_candidates (if `sane`).
//
// `tau` is at or below the keep-th largest; usually a few more than `keep` elements
// reach it, and those are ranked.  Where
// too many do (ties, a row that is mostly masked, sorted rows, a NaN) the bound
// is the keep-th largest of the threads' largest elements, and if that leaves too
// many the keep-th largest element itself, found bit by bit; what is above the
// bound is taken, and of the elements equal to it those of the lowest ids.  This
// second way reads the segment from memory again: it is rare, and from registers it
// takes code for each element (20 000 instructions with 8 vectors a thread, which a
// single row's call spent 15 us fetching).
template <int DT, int NV, class F>
__device__ __forceinline__ void select_top(const typename Elem<DT>::type* seg, float tau, bool sane,
                                           int keep, int id0, int len, Shared& sh,
                                           const TopLds& top, F emit) {
    typedef Segment<DT, NV> S;
    constexpr int kVec = S::kVec;
    const int threads = blockDim.x, waves = threads / 64, t = threadIdx.x;
    uint64_t* keys = top.keys;
    const int vecs = sane ? sh.vecs : 0;
    if (vecs <= kCapVecs) {
        for (int i = t; i < vecs * kVec; i += threads) {
            const int e = i % kVec;
            const symtile::u32x4 w = top.vec[i / kVec];
            // (element() takes its place as a constant)
            float x = 0.0f;
#pragma unroll
            for (int k = 0; k < kVec; ++k) x = e == k ? element<DT>(w, k) : x;
            if (x >= tau) keys[atomicAdd(&sh.n, 1) % kCap] = top_key(order(x), id0 + top.at[i / kVec] + e);
        }
    }
    __syncthreads();
    int n = sh.n;
    if (!sane || vecs > kCapVecs || n < keep || n > max(4 * keep, 128)) {
        int step = 0;
        __syncthreads();
        // f(element's index, its order) for this thread's elements
        auto each = [&](auto f) {
#pragma unroll 1
            for (int at = t * kVec; at < len; at += threads * kVec) {
                const symtile::u32x4 w = S::fetch(seg, len, at);
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                    if (at + e < len) f(at + e, order(element<DT>(w, e)));
            }
        };
        uint32_t mine = 0;
        each([&](int, uint32_t o) { mine = max(mine, o); });
        uint32_t T = 0;
#pragma unroll 1
        for (int b = 31; b >= 0; --b) {
            const uint32_t trial = T | 1u << b;
            if ((int)block_count(mine >= trial, sh, step, waves) >= keep) T = trial;
        }
        // the number of elements above T; where ranking them would cost more than a pass over the
        // row for each of 32 bits (in cycles), T is raised to the keep-th largest itself
        int gt = 0;
        bool by_bits = false;
        for (int b = -1;;) {
            const uint32_t bound = b < 0 ? T : (T | 1u << b) - 1;
            uint32_t c = 0;
            each([&](int, uint32_t o) { c += o > bound; });
            const int above = (int)block_count(c, sh, step, waves);
            if (b < 0) {
                gt = above;
                if (by_bits || gt <= keep) break;
                const float rank_cost = 10.0f * (float)gt * (float)gt / (float)threads;
                if (gt <= kCap && rank_cost <= 32.0f * (2000.0f + 6.0f * NV * kVec * (float)waves))
                    break;
                by_bits = true;
                T = 0;
                b = 31;
            } else {
                if (above >= keep) T = bound + 1;
                --b;
            }
        }
        if (t == 0) sh.n = 0;
        __syncthreads();
        each([&](int i, uint32_t o) {
            if (o > T) keys[atomicAdd(&sh.n, 1)] = top_key(o, id0 + i);
        });
        // elements equal to T in the order of their ids: vector by vector of all threads
        int taken = gt;
#pragma unroll 1
        for (int first = 0; taken < keep && first < len; first += threads * kVec) {
            const int at = first + t * kVec;
            uint32_t tie = 0;
            if (at < len) {
                const symtile::u32x4 w = S::fetch(seg, len, at);
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                    if (at + e < len && order(element<DT>(w, e)) == T) tie |= 1u << e;
            }
            const uint32_t c = __popc(tie);
            uint32_t before = c;     // inclusive over the wave's lanes
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                const uint32_t u = __shfl_up(before, o);
                if (t % 64 >= o) before += u;
            }
            uint32_t* a = sh.count[step & 1];
            ++step;
            if (t % 64 == 63) a[t / 64] = before;
            __syncthreads();
            uint32_t base = 0, all = 0;
            for (int w = 0; w < waves; ++w) {
                base += w < t / 64 ? a[w] : 0;
                all += a[w];
            }
            int place = taken + (int)(base + before - c);
            for (int e = 0; e < kVec; ++e)
                if (tie >> e & 1) {
                    if (place < keep) keys[place] = top_key(T, id0 + at + e);
                    ++place;
                }
            taken += (int)all;
        }
        n = max(gt, keep);
        __syncthreads();
    }
    rank_keys(keys, n, keep, emit);
}

// What the gradient of a row needs of it.
struct RowGrad {
    float a, b, own;
};
__device__ __forceinline__ RowGrad row_grad(const LogprobParams& p, int r, int64_t target, float m,
                                            float log_s, float entropy, const Exponent& ex) {
    RowGrad o;
    float gl = p.g_logprob && target >= 0 ? p.g_logprob[r] : 0.0f;
    if (target >= p.vocab) gl = __builtin_nanf("");
    const float ge = p.g_entropy ? p.g_entropy[r] : 0.0f;
    const float gs = p.g_lse ? p.g_lse[r] : 0.0f;
    // p = 2^y / s', logp = ln2 (y - log2 s') with s' = s 2^shift, log s' = log s + ln2 shift
    const float log_sy = log_s + kLn2 * ex.shift;
    const float inv = expf(-log_sy) * p.scale;
    o.a = inv * (gs - gl - ge * (entropy - log_sy));
    o.b = -inv * ge * kLn2;
    // a row of -inf alone has no gradient (all its e_v are 0)
    o.own = m == -kInf && log_s == 0.0f ? 0.0f : gl * p.scale;
    return o;
}

// READ: whether the registers were read in a pass before.
template <int DT, int NV, bool HUGE, bool READ>
__device__ __forceinline__ void write_grad(Segment<DT, NV>& d,
                                           typename Elem<DT>::type* __restrict__ dx, int len,
                                           int64_t target, const RowGrad& g, const Exponent& ex) {
    constexpr int kVec = Elem<DT>::kVec;
    const int threads = blockDim.x;
    if constexpr (READ) d.again();
    const int at_target = target >= 0 && target < len ? (int)target : -kVec;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = (i * threads + (int)threadIdx.x) * kVec;
        float f[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const float y = ex.template y<HUGE>(element<DT>(d.v[i], e));
            f[e] = exp2_fast(y) * __builtin_fmaf(g.b, fmaxf(y, kFloorY), g.a);
        }
        if ((unsigned)(at_target - at) < (unsigned)kVec) {
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (at + e == at_target) f[e] += g.own;
        }
        Segment<DT, NV>::store(dx, len, at, pack<DT>(f));
    }
}

template <int DT, int NV, bool HUGE>
__device__ __forceinline__ void sums(Segment<DT, NV>& d, const Exponent& ex, float* s, float* t) {
    d.again();
    float s0 = 0.0f, s1 = 0.0f, t0 = 0.0f, t1 = 0.0f;
    d.each([&](int, int e, float x) {
        const float y = ex.template y<HUGE>(x);
        const float v = exp2_fast(y);
        float& ss = e % 2 ? s1 : s0;
        float& tt = e % 2 ? t1 : t0;
        ss += v;
        tt = __builtin_fmaf(v, fmaxf(y, kFloorY), tt);
    });
    *s = s0 + s1;
    *t = t0 + t1;
}

// m, s and t of a row (t in natural units: sum e scale (x - m)) to its outputs.
struct RowValues {
    float m, log_s, entropy;
    bool empty;
    __device__ __forceinline__ RowValues(float m_, float s, float t) : m(m_) {
        empty = m == -kInf && s == 0.0f;
        log_s = empty ? 0.0f : logf(s);
        entropy = empty ? 0.0f : log_s - t / s;
    }
    __device__ __forceinline__ float logp(float x, float scale) const {
        return empty ? -kInf : (x - (m == -kInf ? 0.0f : m)) * scale - log_s;
    }
};

__device__ __forceinline__ void write_values(const LogprobParams& p, int r, int64_t target,
                                             float x_target, const RowValues& v) {
    if (p.logprob)
        p.logprob[r] = target < 0           ? 0.0f
                       : target >= p.vocab ? __builtin_nanf("")
                                           : v.logp(x_target, p.scale);
    if (p.entropy) p.entropy[r] = v.entropy;
    if (p.stats) {
        p.stats[2 * (size_t)r] = v.m;
        p.stats[2 * (size_t)r + 1] = v.log_s;
    }
}

// Waves a SIMD that the registers have to allow (4: what 1024 threads need).  With top
// entries a workgroup waits at more barriers, and more workgroups beside it cover that
// (4096x28672 bf16 with 20: 63 us at 70 registers, 57 at 60).
constexpr int waves_of(int nv, int phase, bool top) {
    return nv == 8 && phase == kValues && top ? 8 : 4;
}

// A workgroup per row or segment.  Its logits come once from memory, and the passes
// over them (largest, sums, candidates, gradient) take them from registers.  With 4096
// rows of 28672 in bfloat16 memory bounds it: the log probabilities alone 45 us (5.2
// TB/s), with the gradient in the same pass 91 us (5.2 TB/s); the gradient in a call of
// its own reads the logits again (2048x32000 float16, both calls: 80 us).  With top
// entries the selection's instructions and barriers are on top of that, and a split
// row's join (333x100003 float32: 28 us, with 64 entries 47).  A single row takes 6.4 us:
// one load, six barriers, one store, of which an empty kernel takes 2.9.
template <int DT, int NV, int PHASE, bool TOP>
__global__ void __launch_bounds__(kMaxThreads, waves_of(NV, PHASE, TOP)) logprob_kernel(LogprobParams p) {
    typedef typename Elem<DT>::type T;
    extern __shared__ __attribute__((aligned(16))) uint64_t dyn[];
    __shared__ Shared sh;
    const int t = threadIdx.x, threads = blockDim.x, waves = threads / 64;
    const int local = p.by_segs(blockIdx.x), seg = blockIdx.x - local * p.segs;
    const int r = p.row0 + local;
    const int id0 = seg * p.seg_len, len = min(p.seg_len, p.vocab - id0);
    const T* row = static_cast<const T*>(p.x) + (size_t)r * p.ld;
    const int64_t target = p.targets ? p.targets[r] : -1;
    Segment<DT, NV> d;
    d.load(row + id0, len, threads);
    float m, log_s, entropy;
    if constexpr (PHASE == kGrad) {
        m = p.stats[2 * (size_t)r];
        log_s = p.stats[2 * (size_t)r + 1];
        entropy = p.entropy[r];
    } else {
        // read before anything is written: the gradient may overwrite it
        if (t == 0 && target >= 0 && target < p.vocab) {
            if constexpr (DT == SYMTILE_F32) sh.x_target = row[target];
            else sh.x_target = (float)row[target];
        }
        float vec_max[NV];
        const float lane_max = d.thread_max(vec_max);
        const TopLds top(dyn, p.segs, p.top);
        const int group = TOP ? group_lanes(p.top, waves) : 0;
        uint32_t group_best = 0;
        if constexpr (TOP) {
            const float pair = Max()(lane_max, dpp<0xB1>(lane_max));
            const float quad = Max()(pair, dpp<0x4E>(pair)), line = row_of_quads(quad, Max());
            m = wave_of_rows(line, Max());
            group_best = group_key(
                group == 16 ? line : group == 4 ? quad : group == 2 ? pair : lane_max, t / group);
            if (t % group == 0) top.groups[t / group] = group_best;
            if (t == 0) {
                sh.n = sh.vecs = 0;
                sh.tau = -kInf;
            }
        } else {
            m = wave_max(lane_max);
        }
        if (t % 64 == 0) sh.m[t / 64] = m;
        __syncthreads();
        m = waves_max(sh.m, waves);
        if constexpr (TOP) find_bound(top.groups, group_best, group, p.top, sh);
        const Exponent ex(m, p.scale);
        float s, u;
        if (ex.huge) sums<DT, NV, true>(d, ex, &s, &u);
        else sums<DT, NV, false>(d, ex, &s, &u);
        s = wave_sum(s);
        u = wave_sum(u);
        if (t % 64 == 0) {
            sh.s[t / 64] = s;
            sh.t[t / 64] = u;
        }
        __syncthreads();
        float tau = -kInf;
        if constexpr (TOP) {
            tau = sh.tau;
            if (tau > -kInf) stage_candidates(d, vec_max, tau, sh, top);
        }
        const float back = exp2f(-ex.shift);
        s = waves_sum(sh.s, waves) * back;
        u = kLn2 * (waves_sum(sh.t, waves) * back - ex.shift * s);
        if constexpr (TOP) __syncthreads();
        const bool sane = s == s && tau > -kInf;
        if (p.segs == 1) {
            const RowValues v(m, s, u);
            if (t == 0) write_values(p, r, target, sh.x_target, v);
            if constexpr (TOP) {
                select_top<DT, NV>(row + id0, tau, sane, p.top, id0, len, sh, top,
                           [&](int place, uint64_t key) {
                               const size_t o = (size_t)r * p.top + place;
                               p.top_ids[o] = key_id(key);
                               p.top_logprobs[o] =
                                   v.logp(ordered_value((uint32_t)(key >> 32)), p.scale);
                           });
            }
            log_s = v.log_s;
            entropy = v.entropy;
        } else {
            const size_t unit = (size_t)local * p.segs + seg;
            if constexpr (TOP) {
                const int keep = min(p.top, len);
                uint64_t* out = p.keys + unit * p.top;
                select_top<DT, NV>(row + id0, tau, sane, keep, id0, len, sh, top,
                           [&](int place, uint64_t key) { put(out + place, key); });
                for (int i = keep + t; i < p.top; i += threads) put(out + i, 0ull);
                if (t == 0) {      // (read before the barrier in rank_keys)
                    sh.n = 0;
                    sh.bound = ~0ull;
                }
            }
            if (t == 0) {
                float* o = p.partials + 4 * unit;
                put(o, m);
                put(o + 1, s);
                put(o + 2, u);
            }
            if (!arrive_last(p.counters + local, p.segs, &sh.last)) return;
            // the row's values from its segments', by every wave
            const float* o = p.partials + 4 * (size_t)local * p.segs;
            // (all loads asked for together: each is a way to memory and back)
            const uint64_t* in = p.keys + (size_t)local * p.segs * p.top;
            uint64_t first_key = 0, bound = ~0ull;
            if constexpr (TOP) {
                // `top` keys are at or above the lowest of the segments' j-th, j = ceil(top / segs)
                if (t < p.segs * p.top) first_key = take(in + t);
                if (t < p.segs) bound = take(in + (size_t)t * p.top + (p.top + p.segs - 1) / p.segs - 1);
            }
            float ms = -kInf, ss = 0.0f, us = 0.0f;
            const int lane = t % 64;
            if (lane < p.segs) {
                ms = take(o + 4 * lane);
                ss = take(o + 4 * lane + 1);
                us = take(o + 4 * lane + 2);
            }
            m = wave_max(ms);
            const float lower = ms == -kInf || ms == m ? 0.0f : (ms - m) * p.scale;
            const float f = expf(lower);
            s = wave_sum(f * ss);
            u = wave_sum(f * __builtin_fmaf(fmaxf(lower, kFloorY), ss, us));
            const RowValues v(m, s, u);
            if (t == 0) write_values(p, r, target, sh.x_target, v);
            if constexpr (TOP) {
                if (t < p.segs)
                    atomicMin(reinterpret_cast<unsigned long long*>(&sh.bound),
                              (unsigned long long)bound);
                __syncthreads();
                for (int i = t; i < p.segs * p.top; i += threads) {
                    const uint64_t key = i == t ? first_key : take(in + i);
                    if (key != 0 && key >= sh.bound) top.keys[atomicAdd(&sh.n, 1)] = key;
                }
                __syncthreads();
                rank_keys(top.keys, sh.n, p.top, [&](int place, uint64_t key) {
                    const size_t at = (size_t)r * p.top + place;
                    p.top_ids[at] = key_id(key);
                    p.top_logprobs[at] = v.logp(ordered_value((uint32_t)(key >> 32)), p.scale);
                });
            }
            return;
        }
    }
    if constexpr (PHASE != kValues) {
        const Exponent ex(m, p.scale);
        const RowGrad g = row_grad(p, r, target, m, log_s, entropy, ex);
        T* dx = static_cast<T*>(p.dx) + (size_t)r * p.ld_grad + id0;
        const int64_t here = target >= id0 && target < p.vocab ? target - id0 : -1;
        if (ex.huge) write_grad<DT, NV, true, PHASE == kStep>(d, dx, len, here, g, ex);
        else write_grad<DT, NV, false, PHASE == kStep>(d, dx, len, here, g, ex);
    }
}

template <int PHASE, bool TOP>
const void* kernel_of(int dtype, int nv) {
    return pick(dtype, nv, [](auto d, auto n) {
        return reinterpret_cast<const void*>(
            &logprob_kernel<decltype(d)::value, decltype(n)::value, PHASE, TOP>);
    });
}

// A kernel over rows first .. first + rows - 1, in launches of rows_a_launch().
symtile_status run(LogprobParams p, const Plan& plan, int first, int rows, const void* kernel,
                   symtile_stream s, const char* what) {
    p.segs = plan.segs;
    p.seg_len = plan.seg_len;
    p.by_segs = symtile_host::make_div(plan.segs);
    const size_t lds = p.top ? TopLds::bytes(plan.segs, p.top) : 0;
    const int most = rows_a_launch(plan);
    for (int row = 0; row < rows; row += most) {
        p.row0 = first + row;
        if (symtile_status st = launch(kernel, plan, std::min(most, rows - row), lds, p, s, what))
            return st;
    }
    return SYMTILE_OK;
}

}  // namespace

extern "C" symtile_status symtile_logits_workspace_bytes(int device, int rows, int vocab, int dtype,
                                                         int top, size_t* bytes) {
    if (!bytes) return fail(SYMTILE_EINVAL, "bytes is NULL");
    *bytes = 0;
    if (symtile_status st = check_sizes(rows, vocab, dtype, top)) return st;
    if (symtile_host::cu_count(device) <= 0)
        return fail(SYMTILE_EINVAL, "device " + std::to_string(device) + " out of range");
    *bytes = make_workspace(make_plan(device, rows, vocab, dtype, false, top), rows, top).bytes;
    return SYMTILE_OK;
}

extern "C" symtile_status symtile_token_logprobs(
    int device, const void* logits, int rows, int vocab, size_t ld, int dtype, float scale,
    const int64_t* targets, float* logprob, float* entropy, float* stats, int top,
    int64_t* top_ids, float* top_logprobs, const float* grad_logprob, const float* grad_entropy,
    const float* grad_lse, void* dlogits, size_t ld_grad, void* workspace, size_t workspace_bytes,
    symtile_stream s) {
    if (symtile_status st = check_sizes(rows, vocab, dtype, top)) return st;
    if (symtile_status st = check_logits(logits, rows, vocab, &ld, dtype, scale)) return st;
    if (rows && ((targets == nullptr) != (logprob == nullptr)))
        return fail(SYMTILE_EINVAL, "targets and logprob come together");
    if (rows && top && (!top_ids || !top_logprobs))
        return fail(SYMTILE_EINVAL, "top needs top_ids and top_logprobs");
    if (dlogits) {
        if (symtile_status st = check_grad(logits, ld, dlogits, &ld_grad, rows, vocab, dtype))
            return st;
        if (rows && (!entropy || !stats))
            return fail(SYMTILE_EINVAL, "dlogits needs entropy and stats");
    } else if (grad_logprob || grad_entropy || grad_lse) {
        return fail(SYMTILE_EINVAL, "gradients without dlogits");
    }
    if (grad_logprob && !targets) return fail(SYMTILE_EINVAL, "grad_logprob without targets");
    const Plan plan = make_plan(device, rows, vocab, dtype, dlogits != nullptr, top);
    const Workspace ws = make_workspace(plan, rows, top);
    if (symtile_status st = check_workspace(workspace, workspace_bytes, ws.bytes)) return st;
    if (rows == 0) return SYMTILE_OK;
    LogprobParams p{};
    p.x = logits;
    p.dx = dlogits;
    p.ld = ld;
    p.ld_grad = ld_grad;
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
    p.vocab = vocab;
    p.scale = scale;
    if (ws.bytes) {
        char* base = static_cast<char*>(workspace);
        p.counters = reinterpret_cast<uint32_t*>(base);
        p.partials = reinterpret_cast<float*>(base + ws.partials);
        p.keys = reinterpret_cast<uint64_t*>(base + ws.keys);
    }
    OnDevice on(device);
    if (on.status) return on.status;
    if (dlogits && plan.segs == 1)
        return run(p, plan, 0, rows,
                   top ? kernel_of<kStep, true>(dtype, plan.nv)
                       : kernel_of<kStep, false>(dtype, plan.nv),
                   s, "logprob_kernel launch");
    if (symtile_status st = run(p, plan, 0, rows,
                                top ? kernel_of<kValues, true>(dtype, plan.nv)
                                    : kernel_of<kValues, false>(dtype, plan.nv),
                                s, "logprob_kernel launch"))
        return st;
    if (!dlogits) return SYMTILE_OK;
    p.top = 0;
    return run(p, plan, 0, rows, kernel_of<kGrad, false>(dtype, plan.nv), s,
               "logprob_kernel launch (gradient)");
}

extern "C" symtile_status symtile_token_logprobs_backward(
    int device, const void* logits, int rows, int vocab, size_t ld, int dtype, float scale,
    const int64_t* targets, const float* entropy, const float* stats, const float* grad_logprob,
    const float* grad_entropy, const float* grad_lse, void* dlogits, size_t ld_grad,
    symtile_stream s) {
    if (symtile_status st = check_sizes(rows, vocab, dtype, 0)) return st;
    if (symtile_status st = check_logits(logits, rows, vocab, &ld, dtype, scale)) return st;
    if (rows && !dlogits) return fail(SYMTILE_EINVAL, "dlogits is NULL");
    if (symtile_status st = check_grad(logits, ld, dlogits, &ld_grad, rows, vocab, dtype)) return st;
    if (rows && (!entropy || !stats)) return fail(SYMTILE_EINVAL, "entropy or stats is NULL");
    if (grad_logprob && !targets) return fail(SYMTILE_EINVAL, "grad_logprob without targets");
    if (rows == 0) return SYMTILE_OK;
    LogprobParams p{};
    p.x = logits;
    p.dx = dlogits;
    p.ld = ld;
    p.ld_grad = ld_grad;
    p.targets = targets;
    p.entropy = const_cast<float*>(entropy);
    p.stats = const_cast<float*>(stats);
    p.g_logprob = grad_logprob;
    p.g_entropy = grad_entropy;
    p.g_lse = grad_lse;
    p.vocab = vocab;
    p.scale = scale;
    OnDevice on(device);
    if (on.status) return on.status;
    const Plan plan = make_plan(device, rows, vocab, dtype, false, 0);
    return run(p, plan, 0, rows, kernel_of<kGrad, false>(dtype, plan.nv), s,
               "logprob_kernel launch (gradient)");
}
