// Verification of drafted tokens against the target's probabilities, from rows of
// logits and given random numbers.
//
// With p_i and q_i the target's and the draft's probabilities of a sequence's
// position i, its first positions with u_i q_i(d_i) < p_i(d_i) are accepted.  At the
// first other one, a, the token is drawn from w_v = max(0, p_a(v) - q_a(v)) by a race
// of exponential times: the largest w_v / noise_v.  One kernel reads all rows for their
// largest logits and sums; the other one decides (every workgroup of a sequence for
// itself) and reads the rows of position a once more.
#include "logits_rows.h"
#include "symtile_device.h"

namespace {

using namespace logits;
using symtile::u32x4;

enum Mode { kGreedy, kTokens, kDraft };   // drafts without and with their logits

// A segment's part of a row's numbers: the largest logit, the sum of exp(scale (x - m)),
// greedy the lowest id of the largest, and the drafted token's logit (-inf in the other
// segments).
struct __attribute__((aligned(16))) Part {
    float m, s;
    uint32_t best;
    float drafted;
};

struct VerifyParams {
    const void *x, *y;          // target and draft logits
    size_t ldx, ldy, ldn;
    const int64_t* ids;
    const float *uniforms, *noise;
    int64_t *tokens, *accepted;
    float* logprob;
    Part* parts;                // [sequence][row][segment]
    uint32_t* counters;         // one a sequence
    uint64_t* keys;             // [sequence][segment][2]
    symtile_host::Div by_segs, by_rows, by_draw;
    int seq0, k, rows, vocab;   // rows of a sequence: k + 1 target ones, then k draft ones
    int segs, seg_len;          // of the first kernel
    int draw_segs, draw_len;    // of the second
    int join_lanes;             // threads that join a row's parts
    float scale, draft_scale;
};

template <int DT>
__device__ __forceinline__ const typename Elem<DT>::type* row_of(const VerifyParams& p, int seq,
                                                                 int r) {
    typedef typename Elem<DT>::type T;
    const size_t at = (size_t)p.seq0 + seq;
    return r <= p.k ? static_cast<const T*>(p.x) + (at * (p.k + 1) + r) * p.ldx
                    : static_cast<const T*>(p.y) + (at * p.k + (r - p.k - 1)) * p.ldy;
}

// ---- largest logits and sums ---------------------------------------------------------------
// A workgroup holds a row's segment in registers, so logits are read once: the largest first,
// then the sum relative to it.  Bound by the vector units, which are busy for three quarters of
// the cycles (7 instructions an element, the exponential for two), beside the loads: 704 rows of
// 50001 fp16 16 us, 4.4 TB/s; few rows by latency (9 rows of 28672 bf16 in segments 3.3 us).
template <int DT, int NV, bool HUGE>
__device__ __forceinline__ float sum_of(Segment<DT, NV>& d, const Exponent& ex) {
    d.again();
    float s0 = 0.0f, s1 = 0.0f;
    d.each([&](int, int e, float x) {
        (e % 2 ? s1 : s0) += exp2_fast(ex.template y<HUGE>(x));
    });
    return s0 + s1;
}

template <int DT, int NV, bool GREEDY>
__global__ void __launch_bounds__(kMaxThreads) verify_sums_kernel(VerifyParams p) {
    __shared__ float m_of[kMaxWaves], s_of[kMaxWaves];
    __shared__ uint32_t best_of[kMaxWaves];
    const int threads = blockDim.x, waves = threads / 64, t = threadIdx.x;
    const int unit = blockIdx.x, row = p.by_segs(unit), seg = unit - row * p.segs;
    const int seq = p.by_rows(row), r = row - seq * p.rows;
    const int begin = seg * p.seg_len, len = min(p.seg_len, p.vocab - begin);
    const float scale = r <= p.k ? p.scale : p.draft_scale;
    Segment<DT, NV> d;
    const typename Elem<DT>::type* x = row_of<DT>(p, seq, r);
    d.load(x + begin, len, threads);
    const int at = r <= p.k ? r : r - p.k - 1;
    float drafted = -kInf;
    if (at < p.k) {
        const int64_t id = p.ids[((size_t)p.seq0 + seq) * p.k + at];
        if (t == 0 && id >= begin && id < begin + len) drafted = (float)x[id];
    }
    float vec[NV];
    const float mine = wave_max(d.thread_max(vec));
    if (t % 64 == 0) m_of[t / 64] = mine;
    __syncthreads();
    const float m = waves_max(m_of, waves);
    const Exponent ex(m, scale);
    const float sum = wave_sum(ex.huge ? sum_of<DT, NV, true>(d, ex) : sum_of<DT, NV, false>(d, ex));
    uint32_t best = 0xFFFFFFFFu;
    if constexpr (GREEDY) {
        // (few vectors hold the largest)
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (vec[i] == m) {
#pragma unroll
                for (int e = 0; e < Segment<DT, NV>::kVec; ++e) {
                    const uint32_t at = (i * threads + t) * Segment<DT, NV>::kVec + e;
                    if (element<DT>(d.v[i], e) == m && (int)at < len) best = min(best, begin + at);
                }
            }
#pragma unroll
        for (int o = 32; o; o >>= 1) best = min(best, (uint32_t)__shfl_xor(best, o));
        if (t % 64 == 0) best_of[t / 64] = best;
    }
    if (t % 64 == 0) s_of[t / 64] = sum;
    __syncthreads();
    if (t < 64) {
        const float s = waves_sum(s_of, waves) * exp2f(-ex.shift);
        if constexpr (GREEDY)
            for (int w = 0; w < waves; ++w) best = min(best, best_of[w]);
        if (t == 0) p.parts[unit] = Part{m, s, best, drafted};
    }
}

// ---- the decision and the draw ------------------------------------------------------------
// A row's numbers from its parts'; a row without a distribution (a NaN or +inf, or nothing
// above -inf) has s not positive and finite.
struct RowStat {
    float m;
    uint32_t best;
    float inv;         // of the sum as Exponent's own shift has it
    float drafted;
    double s;
    __device__ __forceinline__ bool good() const { return s > 0.0 && s < (double)kInf; }
};

// By `lanes` (a power of two from segs on, at most a wave) threads a row, a part each.
__device__ __forceinline__ RowStat join(Part q, int segs, int lanes, float scale) {
    if ((int)threadIdx.x % lanes >= segs) q = Part{-kInf, 0.0f, 0xFFFFFFFFu, -kInf};
    float m = q.m;
    for (int o = lanes / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    // (a segment at -inf alone has s = 0; beside a NaN sum nothing else matters)
    double s = q.m == -kInf || q.m == m
                   ? (double)q.s : (double)(q.s * exp2f((q.m - m) * scale * kLog2e));
    uint32_t best = q.m == m ? q.best : 0xFFFFFFFFu;
    for (int o = lanes / 2; o; o >>= 1) {
        s += __shfl_xor(s, o);
        best = min(best, (uint32_t)__shfl_xor(best, o));
        q.drafted = fmaxf(q.drafted, __shfl_xor(q.drafted, o));
    }
    return RowStat{m, best, exp2f(-Exponent(m, scale).shift) / (float)s, q.drafted, s};
}

struct Shared {
    RowStat stat[2 * SYMTILE_DRAFT_MAX + 1];
    double log_s[SYMTILE_DRAFT_MAX + 1];
    float score[kMaxWaves], id[kMaxWaves], logit[kMaxWaves];
    int accepted;
    bool drafted;      // position `accepted` has a drafted token, which was not accepted
    bool none;
    int last;
};

// Which positions are accepted; by the workgroup's first wave, lane l with position l's id
// and uniform number.  Lanes l and l + 32 take its p and its q.
template <int MODE>
__device__ __forceinline__ void decide(const VerifyParams& p, int64_t id, float u, Shared& sh) {
    const int lane = threadIdx.x;
    const bool in = lane < p.k;
    bool good = in && id >= 0 && id < p.vocab && sh.stat[lane].good();
    if constexpr (MODE == kGreedy) {
        good = good && (uint32_t)id == sh.stat[lane].best;
    } else {
        static_assert(SYMTILE_DRAFT_MAX <= 32, "two lanes a position");
        const int at = lane % 32;
        const bool draft = MODE == kDraft && lane >= 32;
        double x = 1.0;
        if (at < p.k && (MODE == kDraft || lane < 32)) {
            const RowStat& a = sh.stat[draft ? p.k + 1 + at : at];
            x = a.good() ? exp(((double)a.drafted - a.m) * (double)(draft ? p.draft_scale : p.scale)) / a.s
                         : (double)kInf;
        }
        const double q = __shfl(x, at + 32);
        // (u = 0 and q = inf give a NaN: not accepted)
        good = good && (double)u * q < x;
    }
    const uint64_t mask = __ballot(good), given = __ballot(in && id >= 0);
    if (lane == 0) {
        // a draft ends at its first absent token
        sh.accepted = __builtin_ctzll(~(mask & given));
        sh.drafted = given >> sh.accepted & 1;
    }
}

// The outputs, with the drawn token and its logit; `id` is the thread's drafted one.
__device__ __forceinline__ void finish(const VerifyParams& p, int seq, const Shared& sh, int64_t id,
                                       int64_t token, float x) {
    const int i = threadIdx.x;
    if (i > p.k) return;
    const size_t at = (size_t)p.seq0 + seq;
    const int a = sh.accepted;
    if (i < a) x = sh.stat[i].drafted;
    else id = i == a ? token : -1;
    p.tokens[at * (p.k + 1) + i] = id;
    p.logprob[at * (p.k + 1) + i] =
        id >= 0 ? (float)(((double)x - sh.stat[i].m) * (double)p.scale - sh.log_s[i]) : 0.0f;
    if (i == 0) p.accepted[at] = a;
}

// The exponentials of a row's elements, over their sum: with the exponent's shift in `inv`, or,
// where they are taken of differences, whose shift is 0, without (`huge`: of this row or of the
// other one, since both are taken alike).
struct Weights {
    Exponent ex;
    float inv;
    __device__ __forceinline__ Weights(const RowStat& r, float scale)
        : ex(r.m, scale), inv(r.inv) {}
    __device__ __forceinline__ void of_differences(const RowStat& r) { inv = 1.0f / (float)r.s; }
    template <bool HUGE>
    __device__ __forceinline__ float of(float x) const {
        return exp2_fast(ex.y<HUGE>(x)) * inv;
    }
};

// p - q of two rounded products.
__device__ __forceinline__ float difference(float p, float q) {
#pragma clang fp contract(off)
    return p - q;
}

constexpr int kDrawVecs = 2;      // vectors of a thread in a round
constexpr int kDrawThreads = 512; // at most, so that a thread has 256 registers

// A thread's best of the race so far: ids come in ascending order, so that of equal scores
// the first stays.
template <int DT>
struct Race {
    static constexpr int kVec = Elem<DT>::kVec, kNoise = kVec / 4;
    float score = -1.0f, logit = 0.0f;
    int id = 0;
    u32x4 noise[kDrawVecs][kNoise];

    // No branch, so that what was asked for before can be waited for alone: the last 4 in place
    // of those that pass the end, and anything of the call's where there are no 4.
    __device__ __forceinline__ void ask(const float* of, int len, int at0, const Part* any) {
        const float* from = len >= 4 ? of : reinterpret_cast<const float*>(any);
#pragma unroll
        for (int v = 0; v < kDrawVecs; ++v)
#pragma unroll
            for (int i = 0; i < kNoise; ++i)
                noise[v][i] = load16(from + max(0, min(at_of(at0, v, i), len - 4)));
    }
    static __device__ __forceinline__ int at_of(int at0, int v, int i) {
        return at0 + (v * (int)blockDim.x + (int)threadIdx.x) * kVec + 4 * i;
    }
    // The noise of the vectors that pass the end.
    __device__ __forceinline__ void mend(int v, const float* of, int len, int at0) {
#pragma unroll
        for (int i = 0; i < kNoise; ++i) {
            u32x4& n = noise[v][i];
            const int at = at_of(at0, v, i), by = at + 4 - len;
            if (len < 4) {
                if (at < len) n = Segment<SYMTILE_F32, 1>::fetch(of, len, at);
            } else if (by > 0) {
                if (by & 1) n = u32x4{n[1], n[2], n[3], n[3]};
                if (by & 2) n = u32x4{n[2], n[3], n[3], n[3]};
            }
        }
    }
    // A round's elements; `out`: the id that is none of the candidates (-1: all are).
    template <bool LESS, bool HUGE>
    __device__ __forceinline__ void run(const u32x4 (&x)[kDrawVecs], const u32x4 (&y)[kDrawVecs],
                                        const Weights& wp, const Weights& wq, const float* of,
                                        int len, int at0, int begin, int out) {
        const int threads = blockDim.x;
#pragma unroll
        for (int v = 0; v < kDrawVecs; ++v) {
            const int at = at0 + (v * threads + (int)threadIdx.x) * kVec;
            const int left = len - at, not_this = out - begin - at;
            float w[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                w[e] = wp.template of<HUGE>(element<DT>(x[v], e));
                // (q rounded as p was, not one operation with the difference: of equal
                // distributions nothing may be left)
                if constexpr (LESS) w[e] = difference(w[e], wq.template of<HUGE>(element<DT>(y[v], e)));
            }
            if (left < kVec || (unsigned)not_this < (unsigned)kVec) {
                mend(v, of, len, at0);
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                    if (e >= left || e == not_this) w[e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                // (where the noise is none, a NaN, which is not above the score)
                const float s = w[e] * __builtin_amdgcn_rcpf(__uint_as_float(noise[v][e / 4][e % 4]));
                const bool better = w[e] > 0.0f && s > score;
                score = better ? s : score;
                logit = better ? element<DT>(x[v], e) : logit;
                id = better ? begin + at + e : id;
            }
        }
    }
};

// All of a row's elements from `begin` on, by the workgroup.
template <int DT, bool HUGE>
__device__ __forceinline__ void race_over(Race<DT>& race, const typename Elem<DT>::type* x,
                                          const typename Elem<DT>::type* y, const float* noise,
                                          bool less, const Weights& wp, const Weights& wq, int len,
                                          int begin, int out, bool asked, const Part* any) {
    constexpr int kVec = Elem<DT>::kVec;
    const int threads = blockDim.x, t = threadIdx.x;
    for (int at0 = 0; at0 < len; at0 += threads * kDrawVecs * kVec) {
        u32x4 xv[kDrawVecs], yv[kDrawVecs];
#pragma unroll
        for (int v = 0; v < kDrawVecs; ++v) {
            const int at = at0 + (v * threads + t) * kVec;
            xv[v] = yv[v] = u32x4{0u, 0u, 0u, 0u};
            if (at < len) {
                xv[v] = Segment<DT, 1>::fetch(x, len, at);
                if (less) yv[v] = Segment<DT, 1>::fetch(y, len, at);
            }
        }
        if (at0 || !asked) race.ask(noise, len, at0, any);
        if (less) race.template run<true, HUGE>(xv, yv, wp, wq, noise, len, at0, begin, out);
        else race.template run<false, HUGE>(xv, yv, wp, wq, noise, len, at0, begin, out);
    }
}

// The largest score (-1: none), the lowest id of equal ones, and its logit.
static_assert(SYMTILE_VOCAB_MAX <= 1 << 24, "ids are whole numbers in 32-bit floats");
struct Best {
    float score, id, logit;
    // Of the wave's lanes.
    __device__ __forceinline__ void reduce() {
        const float most = wave_max(score), first = -wave_max(score == most ? -id : -kInf);
        const uint64_t who = __ballot(score == most && id == first);
        logit = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(logit), __builtin_ctzll(who)));
        score = most;
        id = first;
    }
};

// Of the workgroup, in its first wave.
__device__ __forceinline__ Best best_of_all(Best b, Shared& sh) {
    const int t = threadIdx.x;
    b.reduce();
    __syncthreads();
    if (t % 64 == 0) {
        sh.score[t / 64] = b.score;
        sh.id[t / 64] = b.id;
        sh.logit[t / 64] = b.logit;
    }
    __syncthreads();
    if (t < 64) {
        const int w = min(t, (int)blockDim.x / 64 - 1);
        b = Best{sh.score[w], sh.id[w], sh.logit[w]};
        b.reduce();
    }
    return b;
}

// Every workgroup of a sequence joins its rows' parts and decides; each then takes a segment
// of position a's rows, and the last of them to arrive joins the race and writes the outputs.
// Bound by latency: one sequence of 4 drafts over 28672 takes 7.0 to 7.8 us, about a third each for
// the decision, the rows' way from memory and the race, and the segments' join (64 sequences of 5
// over 50001 10.1 us for 24 MB, vector units busy for two fifths of the cycles).
template <int DT, int MODE>
__global__ void __launch_bounds__(kDrawThreads) verify_draw_kernel(VerifyParams p) {
    typedef typename Elem<DT>::type T;
    __shared__ Shared sh;
    const int t = threadIdx.x, threads = blockDim.x, unit = blockIdx.x;
    const int seq = p.by_draw(unit), seg = unit - seq * p.draw_segs;
    const int begin = seg * p.draw_len, len = min(p.draw_len, p.vocab - begin);
    // the drafted tokens, the rows' parts and the noise are all asked for at once
    const int64_t id = t < p.k ? p.ids[((size_t)p.seq0 + seq) * p.k + t] : -1;
    const float* noise = nullptr;
    Race<DT> race;
    const Part* parts = p.parts + (size_t)seq * p.rows * p.segs;
    auto part_of = [&](int r) {
        return parts[min(r, p.rows - 1) * p.segs + min(t % p.join_lanes, p.segs - 1)];
    };
    auto join_row = [&](const Part& part, int r) {
        const RowStat stat = join(part, p.segs, p.join_lanes, r <= p.k ? p.scale : p.draft_scale);
        if (r < p.rows && t % p.join_lanes == 0) sh.stat[r] = stat;
    };
    const int at_once = threads / p.join_lanes;
    const Part part = part_of(t / p.join_lanes);
    float u = 0.0f;
    if constexpr (MODE != kGreedy) {
        const float* uniforms = p.k ? p.uniforms + ((size_t)p.seq0 + seq) * p.k
                                    : reinterpret_cast<const float*>(parts);
        u = uniforms[min(t, max(p.k - 1, 0))];
        noise = p.noise + ((size_t)p.seq0 + seq) * p.ldn + begin;
        race.ask(noise, len, 0, parts);
    }
    join_row(part, t / p.join_lanes);
    for (int r0 = at_once; r0 < p.rows; r0 += at_once)
        join_row(part_of(r0 + t / p.join_lanes), r0 + t / p.join_lanes);
    __syncthreads();
    // (needed at the end, and taken by a wave that would wait)
    auto logs = [&] {
        if (t >= 64 && t - 64 <= p.k) sh.log_s[t - 64] = log(sh.stat[t - 64].s);
    };
    if (t < 64) decide<MODE>(p, id, u, sh);
    else if (MODE == kGreedy) logs();
    __syncthreads();
    const int a = sh.accepted;
    const bool valid = sh.stat[a].good();
    if constexpr (MODE == kGreedy) {
        finish(p, seq, sh, id, valid ? (int64_t)sh.stat[a].best : -1, sh.stat[a].m);
        return;
    }
    if (!valid) {          // (the same for all of the sequence's workgroups)
        if (seg) return;
        logs();
        __syncthreads();
        finish(p, seq, sh, id, -1, 0.0f);
        return;
    }
    // a position with a drafted token, and the draft's own distribution
    const bool less = MODE == kDraft && sh.drafted && sh.stat[p.k + 1 + a].good();
    // the drafted token is none of the candidates, where it is one of the vocabulary
    const int64_t drafted = MODE == kTokens && sh.drafted ? p.ids[((size_t)p.seq0 + seq) * p.k + a] : -1;
    const int out = drafted < p.vocab ? (int)drafted : -1;
    const RowStat &of_p = sh.stat[a], &of_q = less ? sh.stat[p.k + 1 + a] : of_p;
    Weights wp(of_p, p.scale), wq(of_q, less ? p.draft_scale : p.scale);
    const T* x = row_of<DT>(p, seq, a);
    const T* y = less ? row_of<DT>(p, seq, p.k + 1 + a) : x;
    const bool huge = wp.ex.huge || wq.ex.huge;
    if (huge) {
        wp.of_differences(of_p);
        wq.of_differences(of_q);
        race_over<DT, true>(race, x + begin, y + begin, noise, less, wp, wq, len, begin, out, true, parts);
    } else {
        race_over<DT, false>(race, x + begin, y + begin, noise, less, wp, wq, len, begin, out, true, parts);
    }
    Best best = best_of_all(Best{race.score, (float)race.id, race.logit}, sh);
    logs();
    if (p.draw_segs > 1) {
        // (a segment's best and its logit, next to each other)
        uint64_t* mine = p.keys + (size_t)unit * 2;
        if (t == 0) {
            put(mine, (uint64_t)__float_as_uint(best.score) << 32 | __float_as_uint(best.id));
            put(mine + 1, (uint64_t)__float_as_uint(best.logit));
        }
        if (!arrive_last(p.counters + seq, p.draw_segs, &sh.last)) return;
        if (t < 64) {
            const uint64_t* of = p.keys + ((size_t)seq * p.draw_segs + min(t, p.draw_segs - 1)) * 2;
            const uint64_t key = take(of), x = take(of + 1);
            best = Best{__uint_as_float((uint32_t)(key >> 32)), __uint_as_float((uint32_t)key),
                        __uint_as_float((uint32_t)x)};
            best.reduce();
        }
    }
    if (t == 0) sh.none = best.score < 0.0f;
    __syncthreads();
    if (sh.none) {
        // no token has p > q: one is drawn from p, by this workgroup alone
        race.score = -1.0f;
        race_over<DT, true>(race, x, x, noise - begin, false, wp, wp, p.vocab, 0, -1, false, parts);
        best = best_of_all(Best{race.score, (float)race.id, race.logit}, sh);
    }
    if (t < 64) finish(p, seq, sh, id, best.score >= 0.0f ? (int64_t)best.id : -1, best.logit);
}

// ---- host ------------------------------------------------------------------------------------
struct VerifyPlan {
    Plan sums;
    int draw_segs, draw_len, draw_threads, launch;      // sequences of a launch
    size_t parts, keys, bytes;                          // of the workspace
};

VerifyPlan verify_plan(int device, int sequences, int k, int vocab, int dtype) {
    VerifyPlan v{};
    const int rows = 2 * k + 1;
    v.launch = std::max(1, std::min(sequences, symtile_host::kWorkspaceCounters / rows));
    v.sums = make_plan(device, v.launch * rows, vocab, dtype, false, 0);
    const int vec = dtype == SYMTILE_F32 ? 4 : 8, n = (vocab + vec - 1) / vec;
    const int cus = std::max(1, symtile_host::cu_count(device));
    // few rows: in up to 8 segments, while each has a CU (9 rows of 28672 bf16: 3.2 us, whole 4.5)
    const int more = std::min({cus / (v.launch * rows), (n + 511) / 512, 8});
    if (more > v.sums.segs) {
        const int len = (n + more - 1) / more;
        v.sums.segs = (n + len - 1) / len;
        v.sums.seg_len = len * vec;
        shape(len, true, &v.sums.nv, &v.sums.threads);
    }
    // the row of position a by as many workgroups as leave each a CU, of two vectors a thread
    // and 256 threads at least: an element costs a wave some 100 cycles, and the join of several
    // workgroups 2 us
    const int most = 256 * kDrawVecs;
    const int segs = std::max(1, std::min({cus / v.launch, (n + most - 1) / most, 64}));
    const int per = (n + segs - 1) / segs;
    v.draw_segs = (n + per - 1) / per;
    v.draw_len = per * vec;
    v.draw_threads = std::min(kDrawThreads, std::max(128, (per + kDrawVecs * 64 - 1) / (kDrawVecs * 64) * 64));
    v.parts = (size_t)symtile_host::kWorkspaceCounters * 4;
    v.keys = v.parts + (size_t)v.launch * rows * v.sums.segs * sizeof(Part);
    v.bytes = v.keys + (size_t)v.launch * v.draw_segs * 16;
    return v;
}

symtile_status check_verify(int sequences, int k, int vocab, int dtype) {
    if (sequences < 0) return fail(SYMTILE_EINVAL, "sequences < 0");
    if (k < 0 || k > SYMTILE_DRAFT_MAX)
        return fail(SYMTILE_EINVAL, "drafted must be in 0 .. " + std::to_string(SYMTILE_DRAFT_MAX));
    if (sequences > (1 << 24)) return fail(SYMTILE_EINVAL, "sequences exceed 16777216");
    return check_sizes(sequences, vocab, dtype, 0);
}

template <int MODE>
const void* draw_kernel_of(int dtype) {
    switch (dtype) {
        case SYMTILE_F16: return reinterpret_cast<const void*>(&verify_draw_kernel<SYMTILE_F16, MODE>);
        case SYMTILE_BF16: return reinterpret_cast<const void*>(&verify_draw_kernel<SYMTILE_BF16, MODE>);
        default: return reinterpret_cast<const void*>(&verify_draw_kernel<SYMTILE_F32, MODE>);
    }
}

}  // namespace

extern "C" symtile_status symtile_verify_workspace_bytes(int device, int sequences, int drafted,
                                                         int vocab, int dtype, size_t* bytes) {
    if (!bytes) return fail(SYMTILE_EINVAL, "bytes is NULL");
    *bytes = 0;
    if (symtile_status st = check_verify(sequences, drafted, vocab, dtype)) return st;
    if (symtile_host::cu_count(device) <= 0)
        return fail(SYMTILE_EINVAL, "device " + std::to_string(device) + " out of range");
    if (sequences) *bytes = verify_plan(device, sequences, drafted, vocab, dtype).bytes;
    return SYMTILE_OK;
}

extern "C" symtile_status symtile_verify_draft(
    int device, const void* logits, int sequences, int drafted, int vocab, size_t ld, int dtype,
    float scale, const int64_t* ids, const void* draft_logits, size_t ld_draft, float draft_scale,
    const float* uniforms, const float* noise, size_t ld_noise, int64_t* tokens, int64_t* accepted,
    float* logprob, void* workspace, size_t workspace_bytes, symtile_stream s) {
    if (symtile_status st = check_verify(sequences, drafted, vocab, dtype)) return st;
    if ((size_t)sequences * (drafted + 1) > (size_t(1) << 30))
        return fail(SYMTILE_EINVAL, "sequences * (drafted + 1) exceeds 1073741824 rows");
    if (symtile_status st = check_logits(logits, sequences * (drafted + 1), vocab, &ld, dtype, scale))
        return st;
    if (ld_noise == 0) ld_noise = (size_t)vocab;
    if (!noise && (uniforms || draft_logits))
        return fail(SYMTILE_EINVAL, "uniforms and draft_logits come with noise");
    if (draft_logits) {
        if (symtile_status st = check_logits(draft_logits, sequences * drafted, vocab, &ld_draft,
                                             dtype, draft_scale))
            return st;
    }
    if (noise && ld_noise < (size_t)vocab) return fail(SYMTILE_EINVAL, "ld_noise smaller than vocab");
    if (sequences == 0) return SYMTILE_OK;
    if (noise && ld_noise > (SIZE_MAX >> 3) / (size_t)sequences)
        return fail(SYMTILE_EINVAL, "noise exceeds the address space");
    if (noise && drafted && !uniforms) return fail(SYMTILE_EINVAL, "noise comes with uniforms");
    if ((drafted && !ids) || !tokens || !accepted || !logprob)
        return fail(SYMTILE_EINVAL, "NULL pointer");
    auto misaligned = [](const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; };
    if (misaligned(uniforms, 4) || misaligned(noise, 4) || misaligned(logprob, 4))
        return fail(SYMTILE_EINVAL, "uniforms, noise or logprob not aligned to their type");
    if (misaligned(ids, 8) || misaligned(tokens, 8) || misaligned(accepted, 8))
        return fail(SYMTILE_EINVAL, "ids, tokens or accepted not aligned to their type");
    const VerifyPlan plan = verify_plan(device, sequences, drafted, vocab, dtype);
    if (symtile_status st = check_workspace(workspace, workspace_bytes, plan.bytes)) return st;
    const bool draft = draft_logits && drafted;
    VerifyParams p{};
    p.x = logits;
    p.y = draft_logits;
    p.ldx = ld;
    p.ldy = ld_draft;
    p.ldn = ld_noise;
    p.ids = ids;
    p.uniforms = uniforms;
    p.noise = noise;
    p.tokens = tokens;
    p.accepted = accepted;
    p.logprob = logprob;
    char* base = static_cast<char*>(workspace);
    p.counters = reinterpret_cast<uint32_t*>(base);
    p.parts = reinterpret_cast<Part*>(base + plan.parts);
    p.keys = reinterpret_cast<uint64_t*>(base + plan.keys);
    p.k = drafted;
    p.rows = draft ? 2 * drafted + 1 : drafted + 1;
    p.vocab = vocab;
    p.segs = plan.sums.segs;
    p.seg_len = plan.sums.seg_len;
    p.draw_segs = noise ? plan.draw_segs : 1;
    p.draw_len = plan.draw_len;
    p.scale = scale;
    p.draft_scale = draft_scale;
    p.by_segs = symtile_host::make_div(p.segs);
    p.by_rows = symtile_host::make_div(p.rows);
    p.by_draw = symtile_host::make_div(p.draw_segs);
    p.join_lanes = 1;
    while (p.join_lanes < p.segs) p.join_lanes *= 2;
    const void* sums = pick(dtype, plan.sums.nv, [&](auto d, auto nv) -> const void* {
        constexpr int DT = decltype(d)::value, NV = decltype(nv)::value;
        return noise ? reinterpret_cast<const void*>(&verify_sums_kernel<DT, NV, false>)
                     : reinterpret_cast<const void*>(&verify_sums_kernel<DT, NV, true>);
    });
    const void* draw = !noise ? draw_kernel_of<kGreedy>(dtype)
                       : draft ? draw_kernel_of<kDraft>(dtype)
                               : draw_kernel_of<kTokens>(dtype);
    OnDevice on(device);
    if (on.status) return on.status;
    for (int seq0 = 0; seq0 < sequences; seq0 += plan.launch) {
        const int n = std::min(plan.launch, sequences - seq0);
        p.seq0 = seq0;
        if (symtile_status st = launch(sums, plan.sums, n * p.rows, 0, p, s, "verify_sums_kernel launch"))
            return st;
        void* args[] = {&p};
        hipError_t e = hipLaunchKernel(draw, dim3((unsigned)n * (unsigned)p.draw_segs),
                                       dim3(noise ? (unsigned)plan.draw_threads : 256u), args, 0,
                                       static_cast<hipStream_t>(s));
        if (e == hipSuccess) e = hipGetLastError();
        if (e != hipSuccess) return symtile_host::hip_fail(e, "verify_draw_kernel launch");
    }
    return SYMTILE_OK;
}
