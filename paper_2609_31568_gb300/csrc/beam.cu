// beam.cu -- beam search over a paged cache: the best continuations of groups of beams (scale_beam_select), and page
// tables that take the beams' new order (scale_beam_reorder).
#include <cuda_bf16.h>

#include "branch.cuh"
#include "launch.cuh"
#include "ptx_sm103.cuh"
#include "scale_internal.h"

namespace scale {
namespace {

using namespace scale_ptx;

// ---------------------------------------------------------------- the best of a part of a row

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kPer = 32;                       // logits of a thread in a step
constexpr int kStepLogits = kThreads * kPer;   // of a CTA
constexpr int kQuarter = kStepLogits / 4;
constexpr int kList = kQuarter + kMaxBest;     // candidates that a CTA holds
constexpr int kRanked = 128;                   // of them that are ranked without a bound; at most kThreads
template <typename T>
constexpr int kResident = sizeof(T) == 2 ? 4 : 3;  // CTAs of an SM: 64 registers are few beside fp32 logits
constexpr int kMaxCandidates = 4096;           // of a group, for k_beam_pick
constexpr int kMaxParts = 32;                  // of a row
constexpr int kFill = 2 * 152;                 // CTAs that rows of several parts make: two an SM
constexpr float kLog2e = 1.4426950408889634f;

// Candidates are 64-bit keys: the logit's order (0 below all; NaN as -inf; both zeros, and what lies between them and the normal
// numbers, alike, as the kernels' comparisons of logits take them), then the tokens from the highest down, so that of equal
// logits the lower token is the larger key. 0: no candidate.
__device__ __forceinline__ uint32_t order_of(float x)
{
    uint32_t u = __float_as_uint(x);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) u = 0xFF800000u;
    if ((u & 0x7F800000u) == 0u) u = 0u;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order & 0x7FFFFFFFu : ~order); }
__device__ __forceinline__ uint64_t candidate(float x, int token) { return static_cast<uint64_t>(order_of(x)) << 32 | ~static_cast<uint32_t>(token); }

__device__ __forceinline__ uint64_t warp_max(uint64_t x)
{
    const uint32_t hi = static_cast<uint32_t>(x >> 32), top = __reduce_max_sync(0xFFFFFFFFu, hi);
    const uint32_t low = __reduce_max_sync(0xFFFFFFFFu, hi == top ? static_cast<uint32_t>(x) : 0u);
    return static_cast<uint64_t>(top) << 32 | low;
}

struct SelectArgs {
    BeamArgs b;
    int parts, part_steps;  // parts of a row, steps of a part
    float2* sums;           // [rows][parts]: largest logit, sum of exp(logit - that)
    uint64_t* best;         // [rows][parts][n_best] descending
};

struct SelectShared {
    uint64_t list[kList];
    union {
        uint64_t other[kList];           // the list in tighten()
        float4 x[kWarps][kPer / 4][32];  // a warp's logits of a step, where it has candidates among them or the row ends
    };
    uint64_t bound[kWarps], sums[kWarps];
    float tops[kWarps];
    int n, kept;
};

// A key that at least `keep` of the threads' `mine` reach (all different, or 0): the each-th largest of each of the first `warps`
// warps, each = keep / warps rounded up, and the least of those. 0 where a warp has fewer.
__device__ __noinline__ uint64_t bound_of(SelectShared& sh, uint64_t mine, int keep, int warps)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int each = warps > 0 ? (keep + warps - 1) / warps : 0;
    uint64_t bound = 0;
#pragma unroll 1
    for (int i = 0; i < each; ++i) {
        bound = warp_max(mine);
        if (mine == bound) mine = 0;
    }
    if (lane == 0) sh.bound[warp] = bound;
    __syncthreads();
    bound = sh.bound[0];
#pragma unroll 1
    for (int w = 1; w < warps; ++w) bound = sh.bound[w] < bound ? sh.bound[w] : bound;
    return each > 32 ? 0 : bound;
}

// How many of n keys are larger than x.
__device__ __forceinline__ int rank_of(const uint64_t* keys, int n, uint64_t x)
{
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) rank += keys[j] > x;
    return rank;
}

// The best `keep` of the list's n candidates, in descending order at its front; returns how many those are. Of more than kRanked
// those below bound_of() go first; the others, a few more than are kept, are ranked one against the other. Every thread
// calls it, behind a barrier, and leaves through one.
__device__ __noinline__ int tighten(SelectShared& sh, int n, int keep)
{
    const int tid = threadIdx.x;
    if (n <= kRanked) {
        const uint64_t x = tid < n ? sh.list[tid] : 0;
        const int rank = tid < n ? rank_of(sh.list, n, x) : keep;
        __syncthreads();
        if (rank < keep) sh.list[rank] = x;
        n = n < keep ? n : keep;
    } else {
        const int at0 = (tid & 31) * kWarps + (tid >> 5);  // every warp gets its share of a short list
        uint64_t top = 0;
#pragma unroll 1
        for (int at = at0; at < n; at += kThreads) top = sh.list[at] > top ? sh.list[at] : top;
        if (tid == 0) sh.kept = 0;
        const uint64_t bound = bound_of(sh, top, keep, kWarps);
#pragma unroll 1
        for (int at = at0; at < n; at += kThreads) {
            const uint64_t x = sh.list[at];
            if (x >= bound) sh.other[atomicAdd(&sh.kept, 1)] = x;
        }
        __syncthreads();
        const int m = sh.kept;
#pragma unroll 1
        for (int at = tid; at < m; at += kThreads) {
            const uint64_t x = sh.other[at];
            const int rank = rank_of(sh.other, m, x);
            if (rank < keep) sh.list[rank] = x;
        }
        n = m < keep ? m : keep;
    }
    if (tid == 0) sh.n = n;
    __syncthreads();
    return n;
}

// A load that stays where it is written, a step ahead of its use.
__device__ __forceinline__ uint4 load_once(const void* p)
{
    uint4 x;
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p));
    return x;
}

// 16 bytes from `shift` (2 to 14) bytes on of 32.
__device__ __forceinline__ uint4 from_two(const uint4& a, const uint4& b, int shift)
{
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = shift & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = shift & 4 ? w[i + 1] : w[i];
    const int bits = (shift & 3) * 8;
    return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                      __funnelshift_r(w[3], w[4], bits));
}

template <typename T>
__device__ __forceinline__ void unpack(const uint4& w, float* x);
template <>
__device__ __forceinline__ void unpack<float>(const uint4& w, float* x)
{
    x[0] = __uint_as_float(w.x);
    x[1] = __uint_as_float(w.y);
    x[2] = __uint_as_float(w.z);
    x[3] = __uint_as_float(w.w);
}
template <>
__device__ __forceinline__ void unpack<__nv_bfloat16>(const uint4& w, float* x)
{
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
}

template <typename T>
struct Step {
    static constexpr int kLoad = 16 / sizeof(T);  // logits of a load
    static constexpr int kLoads = kPer / kLoad;
    // the i-th logit of the thread whose first is that of token `first`
    static __device__ __forceinline__ int token(int first, int i) { return first + i / kLoad * (kThreads * kLoad) + i % kLoad; }
};

// Candidates of a warp's step whose logits lie in sh.x, of the lanes in `who`: those that reach the bound go into the list, as
// far as it has room; sh.n counts them all. `first`: token of this lane's first logit.
template <typename T>
__device__ __noinline__ void collect(SelectShared& sh, uint32_t who, int first, int vocab, uint64_t bound)
{
    static_assert(kPer == 32, "a lane for each of a thread's logits");
    const int lane = threadIdx.x & 31, i = lane;
    const float* x = reinterpret_cast<const float*>(sh.x[threadIdx.x >> 5][i >> 2]) + (i & 3);
#pragma unroll 1
    for (; who; who &= who - 1) {  // a lane for each of its logits
        const int from = __ffs(who) - 1;
        const int t = Step<T>::token(__shfl_sync(0xFFFFFFFFu, first, from), i);
        const uint64_t c = candidate(x[from * 4], t);
        const uint32_t in = __ballot_sync(0xFFFFFFFFu, t < vocab && c >= bound);
        if (in == 0) continue;
        int at = 0;
        if (lane == 0) at = atomicAdd(&sh.n, __popc(in));
        at = __shfl_sync(0xFFFFFFFFu, at, 0) + __popc(in & ((1u << lane) - 1u));
        if ((in >> lane & 1u) && at < kList) sh.list[at] = c;
    }
}

// A thread's logits of a step that the row ends in, or begins in behind a 16-byte boundary, to sh.x; -inf behind the row.
template <typename T>
__device__ __noinline__ void load_edge(SelectShared& sh, const T* logits, int first, int vocab)
{
    const int lane = threadIdx.x & 31;
    float x[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int t = Step<T>::token(first, i);
        x[i] = t < vocab ? static_cast<float>(logits[t]) : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < kPer; i += 4) sh.x[threadIdx.x >> 5][i >> 2][lane] = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
}

// e^(a - b), off by 2^-22.7 of it at most however far a lies below b (0 beyond 87), for a - b of at most kApart: ex2(fl(a - b) log2 e) is off
// by as much as the roundings of the difference and of the product are, 2^-20 each at 16. What the difference loses is kept
// (Knuth's sum of two), multiples of log 2 go off it (Cody and Waite), and the rest, at most 0.35, has its series. A NaN, or -inf
// from -inf, gives 0.
constexpr float kApart = 4.0f;

__device__ __forceinline__ float exp_of(float a, float b)
{
    const float d = __fadd_rn(a, -b);
    if (!(d >= -87.0f)) return 0.f;
    const float back = __fadd_rn(d, -a);
    const float lost = __fadd_rn(__fadd_rn(a, -__fadd_rn(d, -back)), -__fadd_rn(b, back));
    const float i = rintf(d * kLog2e);
    const float r = fmaf(i, 1.9046543e-9f, fmaf(i, -0.69314718f, d)) + lost;  // log 2 is 0.69314718246 (the fp32 number) - 1.9046543e-9
    float y = fmaf(r, 1.0f / 5040, 1.0f / 720);
    y = fmaf(r, y, 1.0f / 120);
    y = fmaf(r, y, 1.0f / 24);
    y = fmaf(r, y, 1.0f / 6);
    y = fmaf(r, y, 0.5f);
    y = fmaf(r, y, 1.0f);
    y = fmaf(r, y, 1.0f);
    return y * __uint_as_float(static_cast<uint32_t>(127 + static_cast<int>(i)) << 23);
}

// Sums across lanes, warps and parts are of whole multiples of 2^-32, which lose nothing and come to the same in any order. They
// stay below 2^62: 2^24 terms, none above e^kApart of what they are against.
__device__ __forceinline__ uint64_t fixed_of(float x) { return __float2ull_rn(x * 4294967296.0f); }
__device__ __forceinline__ float of_fixed(uint64_t x) { return __ull2float_rn(x) * (1.0f / 4294967296.0f); }

// sum of exp(x - top) of a thread's step with NaN among its logits, which count as -inf
template <typename T>
__device__ __noinline__ float sum_without_nan(const T* logits, int first, int vocab, float top)
{
    float y = 0.f;
#pragma unroll 1
    for (int i = 0; i < kPer; ++i) {
        const int t = Step<T>::token(first, i);
        if (t >= vocab) continue;
        const float x = static_cast<float>(logits[t]);
        if (x > -INFINITY) y += ex2((x - top) * kLog2e);
    }
    return y;
}

// The part's candidates again, where the list ran over: logits that come in ascending order, say. A quarter of a step at a
// time, the list cut and the bound raised before each.
template <typename T>
__device__ __noinline__ int collect_carefully(SelectShared& sh, const T* logits, int vocab, int s0, int s1, int keep)
{
    uint64_t bound = 0;
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0;
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
        const int first = s * kStepLogits + static_cast<int>(threadIdx.x) * Step<T>::kLoad;
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
            __syncthreads();
            int n = sh.n;
            __syncthreads();
            if (n > kMaxBest) {
                n = tighten(sh, n, keep);
                bound = sh.list[keep - 1];  // (n was more than is kept)
                __syncthreads();
            }
            load_edge<T>(sh, logits, first, vocab);
            __syncwarp();
            collect<T>(sh, 0xFFu << 8 * q, first, vocab, bound);
        }
    }
    __syncthreads();
    return sh.n;
}

// Largest logit, sum of exponentials and best candidates of a part of a row of logits, one pass over them.
//
// A step is 8,192 logits, 32 a thread, in 16-byte loads that are made a step ahead. SKEW: rows begin anywhere; behind a
// 16-byte boundary a thread puts its logits together from its load and its neighbour's, so that it has the same tokens
// wherever the row lies: rows of the same logits have the same sum to the bit, and equal scores stay equal. A step's sum is against
// its own largest logit, its thread's against the thread's, with what a step loses carried to the next; those of threads and parts
// meet in whole numbers. It is off by 2^-18 of itself at most (in units of 2^-24: ex2 3, distances in a step 4, its ten sums 9, six of exp_of
// with their products 21, the rest 6), and by 2^-21.3 in the worst of 50,000 rows of many kinds. (Steps against the thread's
// largest logit so far, all joined by ex2: 41.8 us in place of 42.9, but 128,000 logits 11 below one were 2^-20.9 off.) The first step sets the
// bound that a candidate has to reach (bound_of, then the least of the n_best best so far, again after 2, 4, 8 .. steps if as many follow);
// between these warps go on without barriers, and one whose threads all stay at or below the bound, which their largest logits tell,
// needs nothing more. The candidates wait in a list, which is cut at the end. What is rare lies in functions of its own: the loop has to
// stay in the instruction cache (unrolled for 32 logits with the candidates' code in it, 64 x 8 rows of 128,000 took 90 to
// 300 us, by where the code came to lie).
//
// Bound by the loop's latency and the instructions of one wave of CTAs, not by HBM: 64 x 8 rows of 128,000 in bf16 (131 MB), select and pick,
// 42.9 us; 11 x 5 of 100,003 in fp32 (22 MB) 17.0, 4 of 32,000 10.1, of which the pick is about 5.
template <typename T, bool SKEW>
__global__ void __launch_bounds__(kThreads, kResident<T>) k_beam_part(const __grid_constant__ SelectArgs a)
{
    constexpr int kLoad = Step<T>::kLoad, kLoads = Step<T>::kLoads;
    __shared__ SelectShared sh;
    pdl_enter();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
    const int keep = a.b.n_best, vocab = a.b.vocab;
    uint64_t* const out = a.best + static_cast<int64_t>(blockIdx.x) * keep;
    const T* const logits = static_cast<const T*>(a.b.logits) + static_cast<int64_t>(row) * a.b.stride;
    const int skew = SKEW ? static_cast<int>(reinterpret_cast<uintptr_t>(logits) % 16 / sizeof(T)) : 0;
    const float score = a.b.scores[row];
    if (tid == 0) sh.n = 0;
    const int steps = (vocab + kStepLogits - 1) / kStepLogits;
    const int s0 = part * a.part_steps;
    int s1 = s0 + a.part_steps < steps ? s0 + a.part_steps : steps;
    // whether all loads of step s, and the neighbour's behind the last, lie in the row
    auto inside = [&](int s) { return (skew == 0 || s > 0) && (s + 1) * kStepLogits + (skew == 0 ? 0 : kLoad) <= vocab; };
    uint4 next[kLoads];
    auto load = [&](int s) {
        if (s >= s1 || !inside(s)) return;
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            next[u] = load_once(logits + (s * kStepLogits - skew + tid * kLoad + u * kThreads * kLoad));
    };
    load(s0);
    if (!(fabsf(score) < INFINITY)) s1 = s0;  // its candidates are no matter of its logits
    float top = -INFINITY, sum = 0.f, lost = 0.f;
    uint64_t bound = 0;
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
        const int first = s * kStepLogits + tid * kLoad;  // token of this thread's first logit
        float x[kPer];
        if (inside(s)) {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                uint4 w = next[u];
                if (SKEW && skew != 0) {
                    uint4 y = make_uint4(__shfl_down_sync(0xFFFFFFFFu, w.x, 1), __shfl_down_sync(0xFFFFFFFFu, w.y, 1),
                                         __shfl_down_sync(0xFFFFFFFFu, w.z, 1), __shfl_down_sync(0xFFFFFFFFu, w.w, 1));
                    if (lane == 31) y = *reinterpret_cast<const uint4*>(logits + (first - skew + (u * kThreads + 1) * kLoad));
                    w = from_two(w, y, skew * static_cast<int>(sizeof(T)));
                }
                unpack<T>(w, x + u * kLoad);
            }
        } else {
            load_edge<T>(sh, logits, first, vocab);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kPer; i += 4) *reinterpret_cast<float4*>(x + i) = sh.x[warp][i >> 2][lane];
        }
        load(s + 1);
        float m = x[0];
#pragma unroll
        for (int i = 1; i < kPer; ++i) m = fmaxf(m, x[i]);
        // ---- the sum, against the step's own largest logit: what is far below that counts for little among 32
        {
            // the largest goes off first, which costs no bits where it counts; one product with both would leave its rounding
            const float neg = fabsf(m) < INFINITY ? -m : 0.f;
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kPer; i += 2) {
                float d0, d1;
                fadd2(d0, d1, x[i], x[i + 1], neg, neg);
                fmul2(d0, d1, d0, d1, kLog2e, kLog2e);
                fadd2(acc[i & 3], acc[(i & 3) + 1], acc[i & 3], acc[(i & 3) + 1], ex2(d0), ex2(d1));
            }
            float y = (acc[0] + acc[1]) + (acc[2] + acc[3]);
            if (!(y >= 0.f)) y = sum_without_nan<T>(logits, first, vocab, -neg);
            // `top` follows the largest logit by steps of more than kApart, so that no term is multiplied often on its way
            const bool ahead = m - top > kApart;
            const float f = exp_of(ahead ? top : m, ahead ? m : top);
            if (ahead) {
                sum *= f;
                lost *= f;
                top = m;
            } else {
                y *= f;
            }
            y -= lost;
            const float t = sum + y;
            lost = (t - sum) - y;
            sum = t;
        }
        // ---- candidates
        if (s == s0) {
            int at = 0;  // the thread's best: the lowest of its largest
#pragma unroll
            for (int i = kPer - 1; i > 0; --i) at = x[i] == m ? i : at;
            at = x[0] == m ? 0 : at;
            // warps whose threads all have logits
            const int full = (vocab - s * kStepLogits) / (32 * kLoad);
            bound = bound_of(sh, first < vocab ? candidate(m, Step<T>::token(first, at)) : 0, keep, full < kWarps ? full : kWarps);
        }
        // equal logits of later steps have higher tokens; a first step that holds n_best has set the bound
        const float least = bound ? value_of(static_cast<uint32_t>(bound >> 32)) : -INFINITY;
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, first < vocab && (s == s0 || bound == 0 ? !(m < least) : m > least));  // (a NaN counts as -inf)
        if (who) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kPer; i += 4) sh.x[warp][i >> 2][lane] = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
            __syncwarp();
            collect<T>(sh, who, first, vocab, bound);
        }
        const int done = s + 1 - s0;
        if (s1 - s - 1 >= done && (done & (done - 1)) == 0) {
            __syncthreads();
            const int n = sh.n;
            __syncthreads();  // every thread has read it before the list grows on
            if (n > keep && n <= kList) {
                tighten(sh, n, keep);
                bound = sh.list[keep - 1];
                __syncthreads();
            }
        }
    }
    float m = top;
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    if (lane == 0) sh.tops[warp] = m;
    __syncthreads();
    int held = sh.n;
    if (held > kList) held = collect_carefully<T>(sh, logits, vocab, s0, s1, keep);
    __syncthreads();
    held = tighten(sh, held, keep);
    for (int i = tid; i < keep; i += kThreads) out[i] = i < held ? sh.list[i] : 0;
    // ---- the threads' sums
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, sh.tops[w]);
    uint64_t y = fixed_of((sum - lost) * exp_of(top, m));
    for (int o = 16; o > 0; o >>= 1) y += __shfl_xor_sync(0xFFFFFFFFu, y, o);
    if (lane == 0) sh.sums[warp] = y;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kWarps; ++w) y += sh.sums[w];
        a.sums[blockIdx.x] = make_float2(m, of_fixed(y));
    }
}

// ---------------------------------------------------------------- the best of a group

// fp64 in order as unsigned integers, never 0.
__device__ __forceinline__ uint64_t order_of(double x)
{
    uint64_t u = static_cast<uint64_t>(__double_as_longlong(x));
    if (u == 1ull << 63) u = 0;
    return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double score_of(uint64_t order)
{
    return __longlong_as_double(static_cast<long long>(order >> 63 ? order & ~(1ull << 63) : ~order));
}

// The natural logarithm of a sum of 1 or more, whose own accuracy is 2^-18 of it, mostly 2^-22: x = 2^e f with f in [0.75, 1.5), and
// log f = 2 atanh(t), t = (f - 1) / (f + 1), at most 0.2, from its series in 32 bits, off by 2^-24 at most; e log 2 joins it in 64.
// (log() in 64 bits is a chain of 64-bit products, 4,000 cycles here.)
__device__ __forceinline__ double log_of_sum(float x)
{
    const uint32_t u = __float_as_uint(x);
    const int e = static_cast<int>(u - 0x3F400000u) >> 23;
    const float f = __uint_as_float(u - (static_cast<uint32_t>(e) << 23));
    const float t = __fdiv_rn(f - 1.0f, f + 1.0f), q = t * t;
    const float series = fmaf(q, fmaf(q, fmaf(q, fmaf(q, 2.0f / 9.0f, 2.0f / 7.0f), 2.0f / 5.0f), 2.0f / 3.0f), 2.0f);
    return fma(static_cast<double>(e), 0.6931471805599453, static_cast<double>(t * series));
}

// The best of a group, a CTA: the logarithms of its beams' sums, and the scores of all candidates in 64 bits (next to another
// beam's, 32 would decide wrongly). A bound on the score as in bound_of leaves a few more than are kept, which are ranked
// one against the other. All latency: the parts' sums, their logarithm, then the candidates, which come meanwhile.
__global__ void __launch_bounds__(kThreads) k_beam_pick(const __grid_constant__ SelectArgs a)
{
    extern __shared__ uint64_t s_pick[];  // two words for each candidate
    __shared__ double s_lse[kMaxBeams];
    __shared__ uint64_t s_bound[kWarps];
    __shared__ int s_n;
    pdl_enter();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, group = blockIdx.x;
    const int beams = a.b.n_beams, keep = a.b.n_best, per_beam = a.parts * keep, all = beams * per_beam;
    uint64_t* const scores = s_pick;       // of the candidates; then of those that reach the bound
    uint64_t* const ties = s_pick + all;   // which of equal scores come first: beam, logit and token
    const uint64_t* const best = a.best + static_cast<int64_t>(group) * all;
    uint64_t early = tid < all ? best[tid] : 0;  // on its way while the sums are
    if (tid == 0) s_n = 0;
    // a power of two of lanes for each beam's parts
    int width = 1;
    while (width < a.parts) width *= 2;
    for (int i0 = 0; i0 < beams; i0 += kThreads / width) {
        const int i = i0 + tid / width, p = tid & (width - 1);
        const bool in = i < beams;
        const int row = group * beams + i;
        const float2 part = in && p < a.parts ? a.sums[static_cast<int64_t>(row) * a.parts + p] : make_float2(-INFINITY, 0.f);
        float top = part.x;
        for (int o = width / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        uint64_t sum = fixed_of(part.y * exp_of(part.x, top));
        for (int o = width / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        const bool live = in && fabsf(top) < INFINITY && fabsf(a.b.scores[row]) < INFINITY;
        if (in && p == 0) s_lse[i] = live ? static_cast<double>(top) + log_of_sum(of_fixed(sum)) : INFINITY;
    }
    __syncthreads();
    // ---- scores
#pragma unroll 1
    for (int i = tid; i < all; i += kThreads) {
        const int beam = i / per_beam;
        uint64_t key = i == tid ? early : best[i], score = 0;
        if (s_lse[beam] < INFINITY) {
            if (key != 0) score = order_of(static_cast<double>(a.b.scores[group * beams + beam]) + (static_cast<double>(value_of(static_cast<uint32_t>(key >> 32))) - s_lse[beam]));
        } else {  // its tokens in their order
            const int token = i - beam * per_beam;
            const bool any = token < keep && token < a.b.vocab;
            key = any ? candidate(-INFINITY, token) : 0;
            if (any) score = order_of(static_cast<double>(-INFINITY));
        }
        scores[i] = score;
        // equal scores: the lower beam, then the logit, then the lower token
        ties[i] = static_cast<uint64_t>(kMaxBeams - 1 - beam) << 56 | (key >> 32) << 24 | (key & 0xFFFFFFu);
    }
    __syncthreads();
    int n = all;
    if (all > kRanked) {
        // ---- the bound: least of the warps' each-th largest. A warp has every eighth of a list, from another one on in every list,
        // whose best is its first; a lane has a list.
        uint64_t top = 0;
        for (int l = lane; l < beams * a.parts; l += 32) {
            const int first = (warp - l) & (kWarps - 1);
            const uint64_t x = first < keep ? scores[l * keep + first] : 0;
            top = x > top ? x : top;
        }
        const int each = (keep + kWarps - 1) / kWarps;
        uint64_t bound = 0;
#pragma unroll 1
        for (int i = 0; i < each; ++i) {
            bound = warp_max(top);
            const uint32_t who = __ballot_sync(0xFFFFFFFFu, top == bound);
            if (lane == __ffs(who) - 1) top = 0;
        }
        if (lane == 0) s_bound[warp] = bound;
        __syncthreads();
        bound = s_bound[0];
        for (int w = 1; w < kWarps; ++w) bound = s_bound[w] < bound ? s_bound[w] : bound;
        // ---- those that reach it, to the front: a block of the list at a time
#pragma unroll 1
        for (int i0 = 0; i0 < all; i0 += kThreads) {
            const int i = i0 + tid;
            const uint64_t score = i < all ? scores[i] : 0, tie = i < all ? ties[i] : 0;
            __syncthreads();
            if (score != 0 && score >= bound) {
                const int at = atomicAdd(&s_n, 1);
                scores[at] = score;
                ties[at] = tie;
            }
            __syncthreads();
        }
        n = s_n;
    }
#pragma unroll 1
    for (int i = tid; i < n; i += kThreads) {
        const uint64_t score = scores[i], tie = ties[i];
        if (score == 0) continue;
        int rank = 0, equal = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) {
            const uint64_t other = scores[j];
            rank += other > score;
            equal += other == score;
        }
        if (equal > 1) {
#pragma unroll 8
            for (int j = 0; j < n; ++j) rank += static_cast<int>(scores[j] == score) & static_cast<int>(ties[j] > tie);
        }
        if (rank >= keep) continue;
        const int64_t at = static_cast<int64_t>(group) * keep + rank;
        a.b.best_scores[at] = static_cast<float>(score_of(score));
        a.b.best_beams[at] = kMaxBeams - 1 - static_cast<int>(tie >> 56);
        a.b.best_tokens[at] = static_cast<int32_t>(~static_cast<uint32_t>(tie) & 0xFFFFFFu);
    }
}

// ---------------------------------------------------------------- beams in a new order

constexpr int kColumns = 128;  // entries of the page table that a CTA turns over, a thread each

// Beams of a group to the pages of the beams that they go on from. Every CTA works out who keeps whose pages, a lane of
// each warp per beam; a thread reads its column of the group's tables before it writes it, so the new
// tables may lie over the old ones. The CTA that has the column of the page being filled writes the moves.
__global__ void __launch_bounds__(kColumns) k_reorder(const __grid_constant__ ReorderArgs a)
{
    __shared__ int32_t s_old[kMaxBeams][kColumns];
    pdl_enter();
    const int tid = threadIdx.x, lane = tid & 31, n = a.n_beams, group = blockIdx.y;
    const int64_t row0 = static_cast<int64_t>(group) * n;
    // ---- lane i: beam i goes on from p, with the last pages of `donor`
    int p = lane < n ? a.parents[row0 + lane] : -1 - lane;
    if (lane < n && static_cast<uint32_t>(p) >= static_cast<uint32_t>(n)) p = lane;
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, p);
    const int of_parent = __shfl_sync(0xFFFFFFFFu, p, p >= 0 ? p : lane);
    const bool keeps = lane < n && (of_parent == p ? lane == p : lane == __ffs(same) - 1);
    const uint32_t beams = n == 32 ? 0xFFFFFFFFu : (1u << n) - 1u;
    const uint32_t free_ones = beams & ~__reduce_or_sync(0xFFFFFFFFu, lane < n ? 1u << p : 0u);
    const uint32_t others = beams & ~__ballot_sync(0xFFFFFFFFu, keeps);
    int donor = p;
    if (lane < n && !keeps) {
        uint32_t rest = free_ones;
        for (int i = __popc(others & ((1u << lane) - 1u)); i > 0; --i) rest &= rest - 1u;
        donor = __ffs(rest) - 1;
    }
    const int len = a.kv_len[row0] > 0 ? a.kv_len[row0] : 0;
    const int full = len / a.c.page_size, filled = len - full * a.c.page_size;
    // ---- the tables
    const int column = blockIdx.x * kColumns + tid;
    if (column < a.stride)
        for (int i = 0; i < n; ++i) s_old[i][tid] = a.table[(row0 + i) * a.stride + column];
    for (int i = 0; i < n; ++i) {
        const int from = __shfl_sync(0xFFFFFFFFu, p, i), last = __shfl_sync(0xFFFFFFFFu, donor, i);
        if (column < a.stride) a.table_out[(row0 + i) * a.stride + column] = s_old[column < full ? from : last][tid];
    }
    // ---- the moves
    const bool has = full < a.stride;
    if ((has ? full / kColumns : 0) != static_cast<int>(blockIdx.x)) return;
    __syncthreads();
    for (int i = 0; i < n; ++i) {
        const int from = __shfl_sync(0xFFFFFFFFu, p, i), last = __shfl_sync(0xFFFFFFFFu, donor, i);
        const int src = has ? s_old[from][full % kColumns] : -1, dst = has ? s_old[last][full % kColumns] : -1;
        const bool moved = from != last && static_cast<uint32_t>(src) < static_cast<uint32_t>(a.c.num_pages) &&
                           static_cast<uint32_t>(dst) < static_cast<uint32_t>(a.c.num_pages);
        for (int t = tid; t < a.c.page_size; t += kColumns) {
            const int64_t at = (row0 + i) * a.c.page_size + t;
            const bool real = moved && t < filled;
            a.src[at] = real ? src * a.c.page_size + t : -1;
            a.dst[at] = real ? dst * a.c.page_size + t : -1;
        }
    }
}

struct BeamWs {
    size_t sums, best;
    int parts, part_steps;
};

// Parts of a row: so many that the rows give every SM two CTAs. (64 x 8 rows of 128,000, bf16, in one part each 40.9 us, in two 47.7;
// 24 x 8 of 100,000, fp32, in two 21.8, in three 27.3; 11 x 5 of 100,003, fp32, in five 16.7, in thirteen 21.2.)
BeamWs beam_layout(int n_groups, int n_beams, int vocab, int n_best)
{
    BeamWs w{};
    const int64_t rows = static_cast<int64_t>(n_groups) * n_beams;
    const int steps = (vocab + kStepLogits - 1) / kStepLogits;
    int64_t parts = (kFill + rows - 1) / rows;
    const int most = kMaxCandidates / (n_beams * n_best);
    if (parts > most) parts = most;
    if (parts > kMaxParts) parts = kMaxParts;
    if (parts > steps) parts = steps;
    if (parts < 1) parts = 1;
    w.part_steps = static_cast<int>((steps + parts - 1) / parts);
    w.parts = (steps + w.part_steps - 1) / w.part_steps;
    w.sums = 0;
    w.best = align_up(static_cast<size_t>(rows) * w.parts * sizeof(float2), kAlign);
    return w;
}

}  // namespace

// Of every call with no more of any of these: fewer rows have more parts each, but rows times parts stays below rows + kFill, and is
// at most rows times the most parts of one.
size_t beam_ws_bytes(int n_groups, int n_beams, int vocab, int n_best)
{
    const int64_t rows = static_cast<int64_t>(n_groups) * n_beams, steps = (vocab + kStepLogits - 1) / kStepLogits;
    const int64_t each = rows * (steps < kMaxParts ? steps : kMaxParts), all = rows + kFill - 1;
    const size_t lists = static_cast<size_t>(each < all ? each : all);
    return align_up(lists * sizeof(float2), kAlign) + align_up(lists * n_best * sizeof(uint64_t), kAlign);
}

cudaError_t launch_beam_select(const BeamArgs& b, bool fp32, uint8_t* ws, cudaStream_t st)
{
    const BeamWs w = beam_layout(b.n_groups, b.n_beams, b.vocab, b.n_best);
    const SelectArgs a{b, w.parts, w.part_steps, reinterpret_cast<float2*>(ws + w.sums), reinterpret_cast<uint64_t*>(ws + w.best)};
    const dim3 grid(static_cast<unsigned>(b.n_groups * b.n_beams * w.parts));
    const bool skew = reinterpret_cast<uintptr_t>(b.logits) % 16 || b.stride * (fp32 ? 4 : 2) % 16;
    auto* const kern = fp32 ? (skew ? k_beam_part<float, true> : k_beam_part<float, false>)
                            : (skew ? k_beam_part<__nv_bfloat16, true> : k_beam_part<__nv_bfloat16, false>);
    cudaError_t e = launch_after(st, grid, kThreads, 0, 1, kern, a);
    if (e != cudaSuccess) return e;
    const size_t smem = 2 * sizeof(uint64_t) * static_cast<size_t>(b.n_beams) * w.parts * b.n_best;
    if (smem > kPlainSmem) {
        constexpr int kMost = 2 * kMaxCandidates * static_cast<int>(sizeof(uint64_t));
        e = cudaFuncSetAttribute(k_beam_pick, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (e != cudaSuccess) return e;
    }
    return launch_after(st, dim3(b.n_groups), kThreads, smem, 1, k_beam_pick, a);
}

cudaError_t launch_reorder(const ReorderArgs& a, cudaStream_t st)
{
    const dim3 grid((a.stride - 1) / kColumns + 1, a.n_groups);
    return launch_after(st, grid, kColumns, 0, 1, k_reorder, a);
}

}  // namespace scale
