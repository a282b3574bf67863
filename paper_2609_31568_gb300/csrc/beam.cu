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
constexpr int kMine = (kList + kThreads - 1) / kThreads;
constexpr int kResident = 4;                   // CTAs of an SM
constexpr int kMaxCandidates = 4096;           // of a group, for k_beam_pick
constexpr int kMaxParts = 32;                  // of a row
constexpr float kLog2e = 1.4426950408889634f;

// Candidates are 64-bit keys: the logit's order (0 below all; NaN as -inf, both zeros alike), then the tokens from the
// highest down, so that of equal logits the lower token is the larger key. 0: no candidate.
__device__ __forceinline__ uint32_t order_of(float x)
{
    uint32_t u = __float_as_uint(x);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) u = 0xFF800000u;
    if (u == 0x80000000u) u = 0u;
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
    uint64_t bound[kWarps];
    float2 sums[kWarps];
    int n, kept;
};

// A key that at least `keep` of the threads' `mine` reach (each its thread's largest candidate): every warp's largest but
// each - 1, each = keep / warps rounded up, and the least of those. 0 where a warp has fewer.
__device__ __forceinline__ uint64_t bound_of(SelectShared& sh, uint64_t mine, int keep)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int each = (keep + kWarps - 1) / kWarps;
    uint64_t bound = 0;
#pragma unroll 1
    for (int i = 0; i < each; ++i) {
        bound = warp_max(mine);
        if (mine == bound) mine = 0;
    }
    if (lane == 0) sh.bound[warp] = bound;
    __syncthreads();
    bound = sh.bound[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) bound = sh.bound[w] < bound ? sh.bound[w] : bound;
    return bound;
}

// The best `keep` of the list's candidates, in descending order at its front. Those below bound_of() go first; the others,
// a few more than are kept, are ranked one against the other. Every thread calls it, behind a barrier, and leaves
// through one.
__device__ __forceinline__ void tighten(SelectShared& sh, int keep)
{
    const int tid = threadIdx.x, n = sh.n;
    uint64_t mine[kMine], top = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int at = i * kThreads + (tid & 31) * kWarps + (tid >> 5);  // every warp gets its share of a short list
        mine[i] = at < n ? sh.list[at] : 0;
        top = mine[i] > top ? mine[i] : top;
    }
    if (tid == 0) sh.kept = 0;
    const uint64_t bound = bound_of(sh, top, keep);
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (mine[i] != 0 && mine[i] >= bound) sh.list[atomicAdd(&sh.kept, 1)] = mine[i];
    __syncthreads();
    const int m = sh.kept;
    int rank[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int at = i * kThreads + tid;
        rank[i] = keep;
        if (at < m) {
            mine[i] = sh.list[at];
            rank[i] = 0;
            for (int j = 0; j < m; ++j) rank[i] += sh.list[j] > mine[i];
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (rank[i] < keep) sh.list[rank[i]] = mine[i];
    if (tid == 0) sh.n = m < keep ? m : keep;
    __syncthreads();
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

// Largest logit, sum of exponentials and best candidates of a part of a row of logits, one pass over them.
//
// A step is 8,192 logits, 32 a thread, in 16-byte loads. A row may begin anywhere; behind a 16-byte boundary a thread puts its
// logits together from two loads, so that it has the same tokens wherever the row lies: rows of the same logits have the
// same sum to the bit, and equal scores stay equal. The sum is a thread's own against its own largest logit, with what a step's sum loses carried to the
// next. The first step sets the bound that a candidate has to pass (bound_of); from then on a step whose threads all stay
// below it, which their largest logits tell, needs nothing more. The candidates wait in a list, which is cut to
// the n_best largest, and the bound raised to the least of them, when it could run over, and at the end.
template <typename T>
__global__ void __launch_bounds__(kThreads, kResident) k_beam_part(const __grid_constant__ SelectArgs a)
{
    constexpr int kLoad = 16 / sizeof(T);  // logits of a load
    constexpr int kLoads = kPer / kLoad;
    __shared__ SelectShared sh;
    pdl_enter();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
    const int keep = a.b.n_best, vocab = a.b.vocab;
    uint64_t* const out = a.best + static_cast<int64_t>(blockIdx.x) * keep;
    const T* const logits = static_cast<const T*>(a.b.logits) + static_cast<int64_t>(row) * a.b.stride;
    const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(logits) % 16 / sizeof(T));  // of the row behind a 16-byte boundary
    const float score = a.b.scores[row];
    if (!(fabsf(score) < INFINITY)) {  // its candidates are no matter of its logits
        if (tid == 0) a.sums[blockIdx.x] = make_float2(-INFINITY, 0.f);
        return;
    }
    if (tid == 0) sh.n = 0;
    const int steps = (vocab + kStepLogits - 1) / kStepLogits;
    const int s0 = part * a.part_steps, s1 = s0 + a.part_steps < steps ? s0 + a.part_steps : steps;
    float top = -INFINITY, sum = 0.f, lost = 0.f;
    float limit = -INFINITY;  // a candidate's logit is larger
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
        const int first = s * kStepLogits + tid * kLoad;  // token of this thread's first logit
        float x[kPer];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int t = first + u * kThreads * kLoad;
            if (skew == 0 ? t + kLoad <= vocab : t >= skew && t - skew + 2 * kLoad <= vocab) {
                const uint4* from = reinterpret_cast<const uint4*>(logits + (t - skew));
                unpack<T>(skew == 0 ? __ldcs(from) : from_two(from[0], from[1], skew * static_cast<int>(sizeof(T))), x + u * kLoad);
            } else {
#pragma unroll
                for (int e = 0; e < kLoad; ++e) x[u * kLoad + e] = t + e < vocab ? static_cast<float>(logits[t + e]) : -INFINITY;
            }
        }
        auto token = [&](int i) { return first + i / kLoad * (kThreads * kLoad) + i % kLoad; };
        auto valid = [&](int i) { return static_cast<uint32_t>(token(i)) < static_cast<uint32_t>(vocab); };
        float m = x[0];
#pragma unroll
        for (int i = 1; i < kPer; ++i) m = fmaxf(m, x[i]);
        // ---- the sum
        if (m > top) {
            const float f = ex2((top - m) * kLog2e);
            sum *= f;
            lost *= f;
            top = m;
        }
        {
            // the largest goes off first, which costs no bits where it counts; one product with both would leave its rounding
            const float neg = top == -INFINITY ? 0.f : -top;
            float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kPer; i += 2) {
                float d0, d1;
                fadd2(d0, d1, x[i], x[i + 1], neg, neg);
                fmul2(d0, d1, d0, d1, kLog2e, kLog2e);
                fadd2(acc[i & 7], acc[(i & 7) + 1], acc[i & 7], acc[(i & 7) + 1], ex2(d0), ex2(d1));
            }
            float y = ((acc[0] + acc[1]) + (acc[2] + acc[3])) + ((acc[4] + acc[5]) + (acc[6] + acc[7]));
            if (!(y >= 0.f)) {  // a NaN counts as -inf
                y = 0.f;
#pragma unroll
                for (int i = 0; i < kPer; ++i) y += x[i] == x[i] ? ex2((x[i] + neg) * kLog2e) : 0.f;
            }
            y -= lost;
            const float t = sum + y;
            lost = (t - sum) - y;
            sum = t;
        }
        // ---- candidates
        bool all = s > s0;  // of those above the limit
        uint64_t bound = 0;
        if (!all) {
            uint64_t best = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const uint64_t c = valid(i) ? candidate(x[i], token(i)) : 0;
                best = c > best ? c : best;
            }
            bound = bound_of(sh, best, keep);
        }
        // whether logit i is one
        auto fits = [&](int i) { return all ? x[i] > limit : valid(i) && candidate(x[i], token(i)) >= bound; };
        const int hits = __syncthreads_count(all ? m > limit : true);
        if (hits == 0) continue;
        int mine = 0;
        if (!all || m > limit) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) mine += fits(i);
        }
        // room for all of them at once, or a quarter of the step at a time
        int before = sh.n;
        int incl = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += y;
        }
        __syncthreads();
        int at = 0;
        if (lane == 31) at = atomicAdd(&sh.n, incl);
        at = __shfl_sync(0xFFFFFFFFu, at, 31) + incl - mine;
        __syncthreads();
        if (sh.n <= kList) {
            if (mine > 0) {
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (fits(i)) sh.list[at++] = candidate(x[i], token(i));
            }
            __syncthreads();
        } else {
            __syncthreads();  // every thread has seen that there is none
            if (tid == 0) sh.n = before;
            __syncthreads();
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
                const int held = sh.n;
                __syncthreads();  // every thread has read it
                if (held > kMaxBest) {
                    tighten(sh, keep);
                    if (sh.n == keep) {
                        bound = sh.list[keep - 1];
                        all = false;
                    }
                }
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (i / (kPer / 4) == q && fits(i)) sh.list[atomicAdd(&sh.n, 1)] = candidate(x[i], token(i));
                __syncthreads();
            }
            tighten(sh, keep);
            bound = sh.list[keep - 1];  // more than the list holds have come
            all = false;
        }
        if (!all && bound != 0) limit = value_of(static_cast<uint32_t>(bound >> 32));
    }
    __syncthreads();
    tighten(sh, keep);
    for (int i = tid; i < keep; i += kThreads) out[i] = i < sh.n ? sh.list[i] : 0;
    // ---- the threads' sums
    float m = top;
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    float y = top == -INFINITY ? 0.f : (sum - lost) * ex2((top - m) * kLog2e);
    for (int o = 16; o > 0; o >>= 1) y += __shfl_xor_sync(0xFFFFFFFFu, y, o);
    if (lane == 0) sh.sums[warp] = make_float2(m, y);
    __syncthreads();
    if (tid == 0) {
        for (int w = 0; w < kWarps; ++w) m = fmaxf(m, sh.sums[w].x);
        y = 0.f;
        for (int w = 0; w < kWarps; ++w)
            if (sh.sums[w].x > -INFINITY) y += sh.sums[w].y * ex2((sh.sums[w].x - m) * kLog2e);
        a.sums[blockIdx.x] = make_float2(m, y);
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

// The best of a group, a CTA: the logarithms of its beams' sums, the scores of all candidates in 64 bits (next to another
// beam's, 32 would decide wrongly), and one warp that takes the best head of the descending lists n_best times.
constexpr int kPickThreads = 256;

__global__ void __launch_bounds__(kPickThreads) k_beam_pick(const __grid_constant__ SelectArgs a)
{
    extern __shared__ uint64_t s_pick[];
    __shared__ double s_lse[kMaxBeams];
    __shared__ int s_next[kMaxBeams * kMaxParts];
    pdl_enter();
    const int tid = threadIdx.x, lane = tid & 31;
    const int beams = a.b.n_beams, keep = a.b.n_best, lists = beams * a.parts, group = blockIdx.x;
    uint64_t* const scores = s_pick;                  // [lists][keep]
    uint64_t* const keys = s_pick + lists * keep;
    for (int i = tid; i < beams; i += kPickThreads) {
        const int row = group * beams + i;
        const float2* s = a.sums + static_cast<int64_t>(row) * a.parts;
        float top = -INFINITY, sum = 0.f;
        for (int p = 0; p < a.parts; ++p) top = fmaxf(top, s[p].x);
        for (int p = 0; p < a.parts; ++p)
            if (s[p].x > -INFINITY) sum += s[p].y * ex2((s[p].x - top) * kLog2e);
        const bool live = fabsf(top) < INFINITY && fabsf(a.b.scores[row]) < INFINITY;
        s_lse[i] = live ? static_cast<double>(top) + log(static_cast<double>(sum)) : INFINITY;
    }
    for (int i = tid; i < lists; i += kPickThreads) s_next[i] = 0;
    __syncthreads();
    for (int i = tid; i < lists * keep; i += kPickThreads) {
        const int list = i / keep, beam = list / a.parts, row = group * beams + beam;
        uint64_t key = a.best[static_cast<int64_t>(group) * lists * keep + i], score = 0;
        if (s_lse[beam] < INFINITY) {
            if (key != 0)
                score = order_of(static_cast<double>(a.b.scores[row]) + (static_cast<double>(value_of(static_cast<uint32_t>(key >> 32))) - s_lse[beam]));
        } else {  // its tokens in their order
            const int token = i - list * keep;
            const bool any = list == beam * a.parts && token < a.b.vocab;
            key = any ? candidate(-INFINITY, token) : 0;
            if (any) score = order_of(static_cast<double>(-INFINITY));
        }
        scores[i] = score;
        keys[i] = key;
    }
    __syncthreads();
    if (tid >= 32) return;
    // the best head of this lane's lists
    uint64_t score = 0, key = 0;
    int from = 0;
    auto look = [&]() {
        score = key = 0;
        for (int l = lane; l < lists; l += 32) {
            const int n = s_next[l];
            if (n >= keep) continue;
            const uint64_t s = scores[l * keep + n], k = keys[l * keep + n];
            // equal scores: the lower beam, whose lists a lane meets first, unless they are of the same
            if (s > score || (s == score && s != 0 && l / a.parts == from / a.parts && k > key)) {
                score = s;
                key = k;
                from = l;
            }
        }
    };
    look();
    for (int i = 0; i < keep; ++i) {
        const uint64_t best = warp_max(score);
        uint32_t who = __ballot_sync(0xFFFFFFFFu, score == best);
        if (who & (who - 1)) {  // the lowest beam of them, then its largest key
            const bool tied = score == best;
            const uint32_t beam = __reduce_min_sync(0xFFFFFFFFu, tied ? static_cast<uint32_t>(from / a.parts) : 0xFFFFFFFFu);
            const bool in = tied && static_cast<uint32_t>(from / a.parts) == beam;
            const uint64_t largest = warp_max(in ? key : 0);
            who = __ballot_sync(0xFFFFFFFFu, in && key == largest);
        }
        if (lane == __ffs(who) - 1) {
            const int64_t at = static_cast<int64_t>(group) * keep + i;
            a.b.best_scores[at] = static_cast<float>(score_of(score));
            a.b.best_beams[at] = from / a.parts;
            a.b.best_tokens[at] = static_cast<int32_t>(~static_cast<uint32_t>(key));
            ++s_next[from];
            look();
        }
        __syncwarp();
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
    size_t sums, best, end;
    int parts, part_steps;
};

// Parts of a row: so many that the rows fill the SMs.
BeamWs beam_layout(int n_groups, int n_beams, int vocab, int n_best)
{
    BeamWs w{};
    const int64_t rows = static_cast<int64_t>(n_groups) * n_beams;
    const int steps = (vocab + kStepLogits - 1) / kStepLogits;
    int64_t parts = (152 * kResident + rows - 1) / rows;
    const int most = kMaxCandidates / (n_beams * n_best);
    if (parts > most) parts = most;
    if (parts > kMaxParts) parts = kMaxParts;
    if (parts > steps) parts = steps;
    if (parts < 1) parts = 1;
    w.part_steps = static_cast<int>((steps + parts - 1) / parts);
    w.parts = (steps + w.part_steps - 1) / w.part_steps;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align_up(off + bytes, kAlign);
        return at;
    };
    w.sums = take(static_cast<size_t>(rows) * w.parts * sizeof(float2));
    w.best = take(static_cast<size_t>(rows) * w.parts * n_best * sizeof(uint64_t));
    w.end = off;
    return w;
}

}  // namespace

size_t beam_ws_bytes(int n_groups, int n_beams, int vocab, int n_best) { return beam_layout(n_groups, n_beams, vocab, n_best).end; }

cudaError_t launch_beam_select(const BeamArgs& b, bool fp32, uint8_t* ws, cudaStream_t st)
{
    const BeamWs w = beam_layout(b.n_groups, b.n_beams, b.vocab, b.n_best);
    const SelectArgs a{b, w.parts, w.part_steps, reinterpret_cast<float2*>(ws + w.sums), reinterpret_cast<uint64_t*>(ws + w.best)};
    const dim3 grid(static_cast<unsigned>(b.n_groups * b.n_beams * w.parts));
    cudaError_t e = fp32 ? launch_after(st, grid, kThreads, 0, 1, k_beam_part<float>, a)
                         : launch_after(st, grid, kThreads, 0, 1, k_beam_part<__nv_bfloat16>, a);
    if (e != cudaSuccess) return e;
    constexpr int kMost = 2 * kMaxCandidates * static_cast<int>(sizeof(uint64_t));
    e = cudaFuncSetAttribute(k_beam_pick, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e != cudaSuccess) return e;
    const size_t smem = 2 * sizeof(uint64_t) * static_cast<size_t>(b.n_beams) * w.parts * b.n_best;
    return launch_after(st, dim3(b.n_groups), kPickThreads, smem, 1, k_beam_pick, a);
}

cudaError_t launch_reorder(const ReorderArgs& a, cudaStream_t st)
{
    const dim3 grid((a.stride + kColumns - 1) / kColumns, a.n_groups);
    return launch_after(st, grid, kColumns, 0, 1, k_reorder, a);
}

}  // namespace scale
