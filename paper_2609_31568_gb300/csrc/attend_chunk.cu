// attend_chunk.cu -- attention of many new tokens of a sequence over its paged
// cache, on the tensor cores (scale_cache_attend's route for calls whose sequences
// may have more than rows_max rows per KV head).
//
// A query tile is 128 rows (token, query head) of one KV head: 128 / g tokens with
// the g query heads that share its keys, which one TMA box of g heads lays down in
// that order. A CTA holds two tiles of neighbouring tokens, walks the 128-key tiles
// of the sequence that some row of them sees, and is otherwise built as
// k_sparse_attn (attn.cu): a TMA producer, one thread that issues tcgen05.mma, two
// groups of four softmax warps with S, P and O in TMEM. What differs:
//  - a key tile is gathered from pages of any multiple of 16 tokens, in boxes of
//    the largest power of two that divides the page, one lane of the producer's
//    warp per box;
//  - 8-bit keys are multiplied as the codes they are, by Q in two e4m3 parts (twice the
//    products at twice the rate), and their scales join the logits; 8-bit values land as
//    codes and four further warps turn them into bf16 tiles, exactly, scales and all;
//  - k_chunk_plan lays out the work: the query tiles of all sequences, and where those
//    are fewer than the SMs keep busy, each cut along its keys, with (O, reference,
//    sum) of the pieces merged by k_chunk_merge.
// 32 query heads on 8, 4,096 tokens over 64K, bf16: 2,710 us, 1.58 PFLOP/s under the power limit, where k_sparse_attn is
// too (2,535 us on a cool GPU). 8-bit: 3,535 us, bound by shared memory: a key tile takes 4,100 cycles (bf16 2,820), in
// which the operands of the products are 1,540 reads of 128 bytes, the keys' scales 1,020 (four each for 32
// lanes), the turning of V 380 and the copies 260; the MMA pipe has work all the time and is half busy. Scales
// as 16-bit halves put together by a byte permutation are half the reads and 3,855 us: the softmax's chain is next.
// Few query tiles are bound by the plan (7 to 8 us), a CTA's start and end (kPieceTiles tiles) and the
// unevenness of the last wave.
#include <cuda_bf16.h>

#include "attend.cuh"
#include "attn_mma.cuh"
#include "launch.cuh"
#include "tma_host.h"

namespace scale {
namespace {

constexpr int kTile = 128;            // keys of a tile, rows of a query tile
constexpr int kPlanThreads = 512;     // at least 2 kMaxSms
constexpr int kCuts = 3;              // pieces per SM, at most, beyond one per item;
constexpr int kCutsRest = 2;          // of the rest of more items than 2 kMaxSms
constexpr int kPieces = 8;            // pieces of an item that the plan considers
constexpr int kUniform = kPieces + kCuts;  // ways to cut that the plan considers: all alike,
constexpr int kTails = 3, kTailCuts = 4;   // and the last half, quarter or eighth of the work shorter
constexpr int kCandidates = kUniform + kTails * kTailCuts;
static_assert(kCandidates <= 32, "a lane for each");
constexpr int kPieceTiles = 5;        // what a CTA's start and end take, in key tiles
constexpr int kMergeTiles = 4;        // what writing and merging one piece per SM takes

// 8-bit: log2 of the sizes of queries that share a power of two. At most 2^-12 of a row's largest |q| is lost so, 2^-4 of what
// bf16 itself leaves of that value. Rows of sizes up to 2^12 apart, each with its own power, take 1.33 times as long
// (4,096 tokens over 64K: 6,620 us, and 4,990 with one power and the small rows' bits lost); of sizes 1 to 8, which share
// it, 332 and 329 us at 1,024 over 16K (476 where they did not, with a limit of 2^3).
constexpr int kRowsApart = 5;

// A CTA's work. Rows [row0, row0 + ntok) of the row tensors are tokens pos ..; key tiles
// [k0, k1) of those the job's rows see; slot >= 0: partial results there.
struct ChunkJob {
    int b, j, row0, ntok;
    int pos, k0, k1, slot;
};

// Pieces of a query tile that k_chunk_merge puts together.
struct ChunkMerge {
    int j, row0, ntok, slot;
    int pieces, pad[3];
};

struct ChunkPlan {
    int32_t* counts;  // jobs, merges
    ChunkJob* jobs;
    ChunkMerge* merges;
    int max_jobs, max_merges, max_slots;
};

struct ChunkArgs {
    AttendView a;
    CacheView c;
    BatchView b;
    ChunkPlan p;
    int sms;
    int tile_tokens;   // tokens of a query tile
    int box;           // tokens of a TMA box: divides the page and the key tile
    float* part_o;     // [slots][2 tiles or 1][128][128]
    float2* part_ml;   // [slots][2 tiles or 1][128] (reference, sum)
    int part_rows;     // 256 or 128
    int32_t* status;
    uint64_t timeout_ns;
};

// Key tiles that rows at tokens [pos, pos + n) see: those of the sinks, then from
// the window's first. One tile of which nothing is seen for rows before the first token.
struct Tiles {
    int sinks, first, n;
};
__device__ __forceinline__ Tiles tiles_of(const AttendView& a, int pos, int n)
{
    Tiles t;
    const int last = pos + n - 1;
    const int lo = a.n_local >= 0 && pos > a.n_local ? pos - a.n_local : 0;
    t.first = lo / kTile;
    const int sinks = static_cast<int>((static_cast<int64_t>(a.n_sink) + kTile - 1) / kTile);
    t.sinks = sinks < t.first ? sinks : t.first;
    t.n = last < 0 ? 1 : t.sinks + last / kTile + 1 - t.first;
    return t;
}

__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t* s_warp, int64_t* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t incl = x;
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += y;
    }
    __syncthreads();  // the scan before is read
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        int64_t v = lane < kPlanThreads / 32 ? s_warp[lane] : 0;
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xFFFFFFFFu, v, o);
            if (lane >= o) v += y;
        }
        s_warp[lane] = v;
    }
    __syncthreads();
    *total = s_warp[31];
    return incl - x + (warp ? s_warp[warp - 1] : 0);
}

// The list of jobs: one CTA. Items are (sequence, KV head, pair of query tiles), a KV head's pairs from the
// last (the one with most keys) to the first, so that the CTAs running at a time share the keys of few heads.
// No job has more than an even share of all key tiles (64 sequences of 5 tokens, bf16, one at 131072 and the others
// at 1,000: 172 us, and 1,328 with the long one's 8 items whole). Calls of more items than 2 kMaxSms run as many as fill
// the SMs a whole number of times so; how the rest are cut (all of them, in other calls) is one of kCandidates: into
// pieces of at most C tiles, C one of
// longest / 1 .. longest / kPieces and R / SMs .. R / (kCuts SMs), R the rest's key tiles; or only the items that hold
// the last half, quarter or eighth of R, T tiles, into pieces of T / SMs .. T / (kTailCuts SMs), which fill up what the
// jobs before them leave uneven. The one is taken that ends first, by the rounds of the SMs or by what jobs taken in
// order can be late at most, kPieceTiles for each job and the merge of the pieces included. (9 sequences of 1 to 700
// tokens, 200 items, 8-bit: 116 us; 113, and 129 with all cut alike, when the choice was made. 4,096 tokens over 64K: 512
// items, 208 of them cut.)
// The plan takes 7 to 8 us, most of it latency: lengths from memory, scans, the lists' way back.
__global__ void __launch_bounds__(kPlanThreads) k_chunk_plan(const __grid_constant__ ChunkArgs a)
{
    __shared__ int s_before[kMaxSeqs + 1];  // items (of one KV head) of the sequences before
    __shared__ int64_t s_warp[32];
    __shared__ int s_longest, s_long[32], s_tail[32], s_split[32], s_cut;
    __shared__ float s_cut_tail;
    __shared__ unsigned long long s_work;
    pdl_trigger();  // k_chunk's first CTAs set up meanwhile
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31;
    const int per_item = 2 * a.tile_tokens;
    const int per = (a.b.n_seqs + kPlanThreads - 1) / kPlanThreads;
    const int i0 = tid * per < a.b.n_seqs ? tid * per : a.b.n_seqs, i1 = i0 + per < a.b.n_seqs ? i0 + per : a.b.n_seqs;
    int64_t mine = 0;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
        const Seq s = seq_of(a.a, a.b, i);
        s_before[i] = static_cast<int>(mine);
        if (s.rows > 0) mine += static_cast<uint32_t>(s.rows + per_item - 1) / static_cast<uint32_t>(per_item);
    }
    int64_t all;
    const int64_t base = block_scan(mine, s_warp, &all);
    const int64_t items = all * a.c.Hkv;
    if (items > a.p.max_jobs) {  // row_start does not ascend within n_rows
        if (tid == 0) {
            record_status(a.status, SCALE_ERR_DEVICE);
            a.p.counts[0] = a.p.counts[1] = 0;
        }
        return;
    }
#pragma unroll 1
    for (int i = i0; i < i1; ++i) s_before[i] += static_cast<int>(base);
    if (tid == 0) {
        s_before[a.b.n_seqs] = static_cast<int>(all);
        s_work = 0;
        s_longest = 0;
    }
    if (tid < 32) s_long[tid] = s_tail[tid] = s_split[tid] = 0;
    __syncthreads();
    // item x: sequences outermost, then KV heads, then pairs from the last
    auto item = [&](int x, ChunkJob* jb) {
        int lo = 0, hi = a.b.n_seqs;
#pragma unroll 1
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_before[mid] * a.c.Hkv <= x) lo = mid;
            else hi = mid;
        }
        const int n = s_before[lo + 1] - s_before[lo];
        const int rem = x - s_before[lo] * a.c.Hkv;
        const Seq s = seq_of(a.a, a.b, lo);
        jb->b = lo;
        jb->j = static_cast<int>(static_cast<uint32_t>(rem) / static_cast<uint32_t>(n));
        const int first = (n - 1 - (rem - jb->j * n)) * per_item;
        jb->row0 = s.row0 + first;
        jb->ntok = s.rows - first < per_item ? s.rows - first : per_item;
        jb->pos = s.pos0 + first;
        jb->k0 = 0;
        jb->k1 = tiles_of(a.a, jb->pos, jb->ntok).n;
        jb->slot = -1;
    };
    const int whole = items > 2 * kMaxSms ? static_cast<int>(items) / a.sms * a.sms : 0;
    const int rest = static_cast<int>(items) - whole;  // at most 2 kMaxSms: one per thread
    int64_t work = 0;
#pragma unroll 1
    for (int x = tid; x < whole; x += kPlanThreads) {
        ChunkJob jw;
        item(x, &jw);
        work += jw.k1;
    }
    if (whole > 0) {
        for (int o = 16; o > 0; o >>= 1) work += __shfl_xor_sync(0xFFFFFFFFu, work, o);
        if (lane == 0) atomicAdd(&s_work, static_cast<unsigned long long>(work));
    }
    ChunkJob jb{};
    if (tid < rest) item(whole + tid, &jb);
    if ((tid & ~31) < rest) {
        const int top = __reduce_max_sync(0xFFFFFFFFu, jb.k1);
        if (lane == 0) atomicMax(&s_longest, top);
    }
    int64_t rest_work;
    const int64_t work_before = block_scan(jb.k1, s_warp, &rest_work);
    const float R = static_cast<float>(rest_work), per_sm = 1.0f / static_cast<float>(a.sms);
    const float share = fminf((static_cast<float>(s_work) + R) * per_sm, 1e9f);
    const int cut_long = static_cast<int>(share) + 1 < 2 ? 2 : static_cast<int>(share) + 1;
    auto pieces_of = [&](int n, int cut, float inv) {  // ceil(n / cut)
        int q = static_cast<int>(static_cast<float>(n + cut - 1) * inv);
        q += q * cut < n;
        return q - ((q - 1) * cut >= n);
    };
    // lane f: candidate f. Items of which no more than my_tail is left are cut at my_cut, those before at cut_long.
    const float inv_long = 1.0f / static_cast<float>(cut_long);
    const int f2 = lane - kUniform;
    const float my_tail = f2 < 0 ? R : R / static_cast<float>(2 << f2 / kTailCuts);
    const int parts = f2 < 0 ? lane - kPieces + 1 : f2 % kTailCuts + 1;
    int my_cut = lane < kPieces ? (s_longest + lane) / (lane + 1) : static_cast<int>(fminf(my_tail * per_sm / static_cast<float>(parts), 1e9f)) + 1;
    if (my_cut < 2) my_cut = 2;
    const float sfx = static_cast<float>(rest_work - work_before);  // key tiles from this item on
    if ((tid & ~31) < rest) {
        const float inv = 1.0f / static_cast<float>(my_cut);
        const int mine = rest - (tid & ~31) < 32 ? rest - (tid & ~31) : 32;
        int n_long = 0, n_tail = 0, n_cut = 0;
#pragma unroll 4
        for (int i = 0; i < mine; ++i) {  // the warp's items
            const int k1 = __shfl_sync(0xFFFFFFFFu, jb.k1, i);
            const bool tail = __shfl_sync(0xFFFFFFFFu, sfx, i) <= my_tail;
            const int q = pieces_of(k1, tail ? my_cut : cut_long, tail ? inv : inv_long);
            (tail ? n_tail : n_long) += q;
            n_cut += q > 1 ? q : 0;
        }
        if (lane < kCandidates) {
            atomicAdd(&s_long[lane], n_long);
            atomicAdd(&s_tail[lane], n_tail);
            atomicAdd(&s_split[lane], n_cut);
        }
    }
    __syncthreads();
    if (tid < 32) {
        const int n_long = s_long[lane], n = n_long + s_tail[lane];
        auto rounds = [&](int jobs) { return ceilf(static_cast<float>(jobs) * per_sm); };
        float time;
        if (f2 < 0) {
            time = rounds(n) * static_cast<float>(my_cut + kPieceTiles);
        } else {
            const float top = static_cast<float>((s_longest < cut_long ? s_longest : cut_long) + kPieceTiles);
            const float first = fminf(rounds(n_long) * top, (R - my_tail + static_cast<float>(n_long * kPieceTiles)) * per_sm + top);
            time = fmaxf(first, (R + static_cast<float>(n * kPieceTiles)) * per_sm + static_cast<float>(my_cut + kPieceTiles));
        }
        time += static_cast<float>(kMergeTiles * s_split[lane]) * per_sm;
        // candidate kPieces: at most `rest` pieces and one per SM, whatever the lengths
        const bool open = lane < kCandidates && (lane == kPieces || n <= rest + (whole ? kCutsRest : kCuts) * a.sms);
        const uint32_t bits = open ? __float_as_uint(time) : 0xFFFFFFFFu;
        const uint32_t best = __reduce_min_sync(0xFFFFFFFFu, bits);
        if (lane == __ffs(__ballot_sync(0xFFFFFFFFu, bits == best)) - 1) {
            s_cut = my_cut;
            s_cut_tail = my_tail;
        }
    }
    __syncthreads();
    // Jobs, a block of items at a time; at, slot and merge count jobs, partial results and merges so far.
    int at = 0, slot = 0, merge = 0;
#pragma unroll 1
    for (int x0 = 0;; x0 += kPlanThreads) {
        const bool done = x0 >= whole;
        ChunkJob x = jb;
        if (!done) {
            x.k1 = 0;
            if (x0 + tid < whole) item(x0 + tid, &x);
        }
        const int cut = done && sfx <= s_cut_tail ? s_cut : cut_long;
        const int n = x.k1, pieces = n > 0 ? pieces_of(n, cut, 1.0f / static_cast<float>(cut)) : 0;
        // jobs, partial results and merges before this item, one scan of 21 bits each
        int64_t sums;
        const int64_t mask = (1 << 21) - 1;
        const int64_t before = block_scan(pieces > 1 ? pieces | static_cast<int64_t>(pieces) << 21 | 1ll << 42 : pieces, s_warp, &sums);
        const int my_at = at + static_cast<int>(before & mask), my_slot = slot + static_cast<int>((before >> 21) & mask), my_merge = merge + static_cast<int>(before >> 42);
        at += static_cast<int>(sums & mask);
        slot += static_cast<int>((sums >> 21) & mask);
        merge += static_cast<int>(sums >> 42);
        if (at > a.p.max_jobs || slot > a.p.max_slots || merge > a.p.max_merges) {  // as above
            if (tid == 0) {
                record_status(a.status, SCALE_ERR_DEVICE);
                a.p.counts[0] = a.p.counts[1] = 0;
            }
            return;
        }
        const int each = pieces > 1 ? static_cast<int>(static_cast<uint32_t>(n) / static_cast<uint32_t>(pieces)) : n, more = n - each * pieces;
#pragma unroll 1
        for (int i = 0; i < pieces; ++i) {  // the first `more` pieces have one tile more
            const int k0 = each * i + (i < more ? i : more);
            int4* to = reinterpret_cast<int4*>(a.p.jobs + my_at + i);
            to[0] = make_int4(x.b, x.j, x.row0, x.ntok);
            to[1] = make_int4(x.pos, k0, k0 + each + (i < more), pieces > 1 ? my_slot + i : -1);
        }
        if (pieces > 1) a.p.merges[my_merge] = ChunkMerge{x.j, x.row0, x.ntok, my_slot, pieces, {0, 0, 0}};
        if (done) break;
    }
    if (tid == 0) {
        a.p.counts[0] = at;
        a.p.counts[1] = merge;
    }
}

// Dynamic shared memory (offsets from its 1024-aligned base): Q, then K and V in two stages each. 8-bit: Q as its two
// parts, K and V as codes, then V as bf16.
constexpr uint32_t kCodeBytes = kTile * kHeadDim;  // one 128 x 128 tile of codes
constexpr uint32_t kOffQ = 0;
constexpr uint32_t kOffK = kOffQ + 2 * kTileBytes;
__host__ __device__ constexpr uint32_t off_raw(bool e4m3) { return kOffK + 2 * (e4m3 ? kCodeBytes : kTileBytes); }
__host__ __device__ constexpr uint32_t off_v(bool e4m3) { return off_raw(e4m3) + (e4m3 ? 2 * kCodeBytes : 0); }
__host__ __device__ constexpr uint32_t off_shared(bool e4m3) { return off_v(e4m3) + 2 * kTileBytes; }

struct ChunkShared {
    Barriers bars;
    uint32_t tmem_slot;
    volatile int abort_flag;
    // 8-bit only
    uint64_t q_ready;                    // Q is in its parts
    uint64_t raw_full[2], raw_empty[2];  // codes of V: landed; turned
    uint64_t v_full[2];                  // V is bf16
};
// 8-bit: per softmax warp, what the products with each key of its tile are multiplied by
__host__ __device__ constexpr uint32_t off_scales(bool e4m3) { return off_shared(e4m3) + 256; }
__host__ __device__ constexpr uint32_t chunk_smem(bool e4m3) { return off_scales(e4m3) + (e4m3 ? 8 * kTile * 4 : 0); }
static_assert(sizeof(ChunkShared) <= 256 && off_scales(true) % 16 == 0, "scales are read four at a time");
static_assert(chunk_smem(true) <= 227 * 1024 && chunk_smem(false) <= 227 * 1024, "shared memory of a CTA");

// Threads: warps 0-7 softmax, 8 producer, 9 MMA; 8-bit: 12-15 turn V into bf16 (10 and 11 idle,
// for whole groups of four warps in the register split: 2 x 128 x 192 + 2 x 128 x 64 = 512 x 128).
__host__ __device__ constexpr int chunk_threads(bool e4m3) { return e4m3 ? 512 : 320; }

// The lowest n bits, 0 <= n <= 32 or beyond either end.
__device__ __forceinline__ uint32_t ones_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u; }

__device__ __forceinline__ float4 lds_f4(uint32_t addr)
{
    float4 r;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(r.x), "=f"(r.y), "=f"(r.z), "=f"(r.w) : "r"(addr));
    return r;
}

// A CTA's job as its roles see it; T = 0: none.
struct JobView {
    ChunkJob job;
    Tiles tiles;
    int nq, last, lo, T, n_sink;
    // first token of the job's key tile t
    __device__ __forceinline__ int token_of(int t) const
    {
        const int i = job.k0 + t;
        return (i < tiles.sinks ? i : tiles.first + i - tiles.sinks) * kTile;
    }
    // whether no row sees token t
    __device__ __forceinline__ bool unseen(int t) const { return t > last || (t < lo && t >= n_sink); }
    // whether that holds for a token of the tile at t0
    __device__ __forceinline__ bool has_unseen(int t0) const { return t0 + kTile - 1 > last || (t0 < lo && t0 + kTile - 1 >= n_sink); }
};

// Waits for the plan, then reads the job of this CTA.
__device__ __forceinline__ JobView load_job(const ChunkArgs& a)
{
    pdl_enter();
    JobView v;
    const int n_jobs = a.p.counts[0];
    const int4 x = reinterpret_cast<const int4*>(a.p.jobs + blockIdx.x)[0], y = reinterpret_cast<const int4*>(a.p.jobs + blockIdx.x)[1];
    v.job = ChunkJob{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    v.nq = v.job.ntok > a.tile_tokens ? 2 : 1;
    v.last = v.job.pos + v.job.ntok - 1;
    v.lo = a.a.n_local >= 0 && v.job.pos > a.a.n_local ? v.job.pos - a.a.n_local : 0;
    v.n_sink = a.a.n_sink;
    v.tiles = tiles_of(a.a, v.job.pos, v.job.ntok);
    v.T = static_cast<int>(blockIdx.x) < n_jobs ? v.job.k1 - v.job.k0 : 0;
    return v;
}

// S = Q1 K^T + Q2 K^T on codes, and the commit.
__device__ __forceinline__ void mma_codes(ChunkShared& sh, uint32_t tmem, uint64_t qdesc0, uint64_t kdesc, int qt, int st)
{
    constexpr uint64_t kTileStep = kTileBytes >> 4, kCodeStep = kCodeBytes >> 4;
    constexpr uint32_t id = idesc_e4m3_f32(128, 128);
    mma_e4m3_k128(tmem + qt * 256, qdesc0 + qt * kTileStep, kdesc, id, 0u);
    mma_e4m3_k128(tmem + qt * 256, qdesc0 + qt * kTileStep + kCodeStep, kdesc, id, 1u);
    mma_commit(&sh.bars.s_full[qt][st]);
}

// Iteration t > 0 of mma_issue_codes.
__device__ __forceinline__ bool mma_codes_step(ChunkShared& sh, uint32_t tmem, uint64_t qdesc0, uint64_t kdesc0, uint64_t vdesc0,
                                               int nq, int t, uint64_t timeout_ns)
{
    const int st = t & 1;
    Barriers& bars = sh.bars;
    const volatile int* abort_flag = &sh.abort_flag;
    if (!mbar_wait_bounded(&bars.kv_full[st], (t >> 1) & 1, timeout_ns, abort_flag)) return false;
    if (!mbar_wait_bounded(&sh.v_full[st ^ 1], ((t - 1) >> 1) & 1, timeout_ns, abort_flag)) return false;
#pragma unroll 1
    for (int qt = 0; qt < nq; ++qt) {
        if (!mbar_wait_bounded(&bars.p_full[qt], st ^ 1, timeout_ns, abort_flag)) return false;
        tc_fence_after();
        mma_ts_k128<2048>(tmem + qt * 256 + 128, tmem + qt * 256, vdesc0 + (st ^ 1) * (kTileBytes >> 4),
                          idesc_bf16_f32(128, 128, 1), t > 1 ? 1u : 0u);
        mma_codes(sh, tmem, qdesc0, kdesc0 + st * (kCodeBytes >> 4), qt, st);
    }
    return true;
}

// mma_issue_loop (attn_mma.cuh) for 8-bit keys, whose K and V have barriers of their own. Rolled: what all roles run per
// key tile has to stay in the SM's instruction cache. (4,096 tokens over 64K, 8-bit: 3,535 us; 3,730 us with two
// iterations of this loop and four of the values' conversion unrolled, when requests for instructions took 64% of
// what the next level answers, and 16% now.)
__device__ __forceinline__ bool mma_issue_codes(ChunkShared& sh, uint32_t tmem, uint64_t qdesc0, uint64_t kdesc0, uint64_t vdesc0,
                                                int nq, int T, bool skip_last, uint64_t timeout_ns)
{
    Barriers& bars = sh.bars;
    const volatile int* abort_flag = &sh.abort_flag;
    if (!mbar_wait_bounded(&bars.kv_full[0], 0, timeout_ns, abort_flag)) return false;
    tc_fence_after();
#pragma unroll 1
    for (int qt = 0; qt < nq; ++qt) mma_codes(sh, tmem, qdesc0, kdesc0, qt, 0);
#pragma unroll 1
    for (int t = 1; t < T; ++t)
        if (!mma_codes_step(sh, tmem, qdesc0, kdesc0, vdesc0, nq, t, timeout_ns)) return false;
    const int sv = (T - 1) & 1;
    if (!mbar_wait_bounded(&sh.v_full[sv], ((T - 1) >> 1) & 1, timeout_ns, abort_flag)) return false;
#pragma unroll 1
    for (int qt = 0; qt < nq; ++qt) {
        if (!mbar_wait_bounded(&bars.p_full[qt], sv, timeout_ns, abort_flag)) return false;
        tc_fence_after();
        if (nq == 2 && qt == 0 && skip_last) continue;
        mma_ts_k128<2048>(tmem + qt * 256 + 128, tmem + qt * 256, vdesc0 + sv * (kTileBytes >> 4), idesc_bf16_f32(128, 128, 1),
                          T > 1 ? 1u : 0u);
    }
    mma_commit(&bars.o_full);
    return true;
}

template <bool E4M3>
__global__ void __launch_bounds__(chunk_threads(E4M3), 1)
k_chunk(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
        const __grid_constant__ CUtensorMap tv, const __grid_constant__ ChunkArgs a)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    ChunkShared& sh = *reinterpret_cast<ChunkShared*>(smem + off_shared(E4M3));
    Barriers& bars = sh.bars;
    volatile int& abort_flag = sh.abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int tt = a.tile_tokens, g = a.a.g;
    // CTAs of the first wave set up, and run the softmax code once, while the plan is made
    const bool first_wave = static_cast<int>(blockIdx.x) < a.sms;
    if (!first_wave) {
        pdl_enter();
        if (static_cast<int>(blockIdx.x) >= a.p.counts[0]) return;
    }
    if (smem_addr(smem) & 1023u) {  // the swizzle goes by the address
        pdl_enter();
        if (tid == 0) record_status(a.status, SCALE_ERR_DEVICE);
        return;
    }
    if (tid == 0) {
        abort_flag = 0;
        mbar_init(&bars.q_full, 1);
        mbar_init(&sh.q_ready, 128);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars.kv_full[i], 1);
            mbar_init(&bars.s_full[i][0], 1);
            mbar_init(&bars.s_full[i][1], 1);
            mbar_init(&bars.p_full[i], 128);
            mbar_init(&sh.raw_full[i], 1);
            mbar_init(&sh.raw_empty[i], 128);
            mbar_init(&sh.v_full[i], 128);
        }
        mbar_init(&bars.o_full, 1);
        mbar_init(&bars.drain, 1);
        fence_barrier_init();
    }
    if (tid == 256) {
        tma_prefetch_desc(&tq);
        tma_prefetch_desc(&tk);
        tma_prefetch_desc(&tv);
    }
    if (warp == 9) {
        tmem_alloc(&sh.tmem_slot, 512);
        tmem_relinquish();
    }
    // rows of a query tile past its g tt: zeros
    if (g * tt < kTile) {
        const int n = (kTile - g * tt) * 8;  // 16-byte pieces of a half
        for (int i = tid; i < 4 * n; i += chunk_threads(E4M3)) {
            const int part = i / n, x = i - part * n;
            *reinterpret_cast<uint4*>(smem + kOffQ + part * kHalf + g * tt * 128 + x * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem_slot;

    if (warp >= 8) {
        if (E4M3) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        const JobView jv = load_job(a);
        const ChunkJob& job = jv.job;
        const int T = jv.T, nq = jv.nq;
        if (T == 0) {
        } else if (warp == 8) {
            // ------------------------------------------------------------ producer: a lane per box
            constexpr int kHalves = E4M3 ? 1 : 2;
            const int bx = lane / kHalves, hf = lane - bx * kHalves;  // 8 boxes of 16 tokens at most: 16 lanes
            const bool mine = bx < kTile / a.box;
            const int32_t pool_rows = a.c.num_pages * a.c.page_size;
            if (lane == 0) {
                mbar_arrive_expect_tx(&bars.q_full, static_cast<uint32_t>(nq * 2 * g * tt * 128));
                for (int qt = 0; qt < nq; ++qt)
                    for (int h = 0; h < 2; ++h)
                        tma_load_3d(smem + kOffQ + qt * kTileBytes + h * kHalf, &tq, &bars.q_full, h * 64, job.j * g,
                                    job.row0 + qt * tt);
            }
            uint64_t* const s_last = bars.s_full[nq - 1];
            int steps = 0, steps_v = 0;
            auto row_of = [&](int t) {
                const int r = mine ? cache_row(a.c, a.b, job.b, jv.token_of(t) + bx * a.box) : 0;
                return r < 0 ? pool_rows : r;  // past the end: zeros
            };
            int32_t row_k = row_of(0), row_v = 0;  // pool rows of this lane's box in tiles t and t - 1
            // Step t: bf16 loads K(t) and V(t - 1) behind one barrier; 8-bit K(t), and V(t) for the warps that turn it. The stages
            // were last read by products of iteration t - 2, which the commit of its last S covers.
            for (int t = 0; t < T + (E4M3 ? 0 : 1); ++t) {
                const int st = t & 1;
                bool ok = t < 2 || mbar_wait_bounded(&s_last[st], ((t - 2) >> 1) & 1, a.timeout_ns, &abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (ok && E4M3) {
                    if (lane == 0) mbar_arrive_expect_tx(&bars.kv_full[st], kCodeBytes);
                    ++steps;
                    __syncwarp();
                    const uint32_t to = st * kCodeBytes + bx * a.box * kHeadDim;
                    if (mine) tma_load_3d(smem + kOffK + to, &tk, &bars.kv_full[st], 0, job.j, row_k);
                    ok = t < 2 || mbar_wait_bounded(&sh.raw_empty[st], ((t - 2) >> 1) & 1, a.timeout_ns, &abort_flag);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (ok) {
                        if (lane == 0) mbar_arrive_expect_tx(&sh.raw_full[st], kCodeBytes);
                        ++steps_v;
                        __syncwarp();
                        if (mine) tma_load_3d(smem + off_raw(true) + to, &tv, &sh.raw_full[st], 0, job.j, row_k);
                    }
                } else if (ok) {
                    const bool has_k = t < T, has_v = t >= 1;
                    if (lane == 0)
                        mbar_arrive_expect_tx(&bars.kv_full[st], (has_k ? kTileBytes : 0u) + (has_v ? kTileBytes : 0u));
                    ++steps;
                    __syncwarp();
                    const uint32_t to = hf * kHalf + bx * a.box * 128;
                    if (mine && has_v)
                        tma_load_3d(smem + off_v(false) + (st ^ 1) * kTileBytes + to, &tv, &bars.kv_full[st], hf * 64, job.j, row_v);
                    if (mine && has_k)
                        tma_load_3d(smem + kOffK + st * kTileBytes + to, &tk, &bars.kv_full[st], hf * 64, job.j, row_k);
                }
                if (!ok) {
                    if (lane == 0) fail(&abort_flag, a.status);
                    break;
                }
                row_v = row_k;
                if (t + 1 < T) row_k = row_of(t + 1);
            }
            __syncwarp();
            if (abort_flag && lane == 0) {
                // every copy in flight lands before the CTA ends
                mbar_wait_bounded(&bars.q_full, 0, a.timeout_ns, nullptr);
                for (int i = 0; i < 2; ++i) {
                    const int n = (steps + 1 - i) / 2, nv = (steps_v + 1 - i) / 2;  // copies into stage i
                    if (n) mbar_wait_bounded(&bars.kv_full[i], (n - 1) & 1, a.timeout_ns, nullptr);
                    if (E4M3 && nv) mbar_wait_bounded(&sh.raw_full[i], (nv - 1) & 1, a.timeout_ns, nullptr);
                }
            }
        } else if (warp == 9) {
            // ------------------------------------------------------------ MMA issuer
            if (lane == 0) {
                bool ok = mbar_wait_bounded(E4M3 ? &sh.q_ready : &bars.q_full, 0, a.timeout_ns, &abort_flag);
                const uint64_t qdesc0 = sdesc_sw128(smem_addr(smem + kOffQ), 16, 1024);
                const uint64_t kdesc0 = sdesc_sw128(smem_addr(smem + kOffK), 16, 1024);
                const uint64_t vdesc0 = sdesc_sw128(smem_addr(smem + off_v(E4M3)), kHalf, 1024);
                // the last key tile may lie after every row of the first query tile
                const bool skip_last = T > 1 && jv.token_of(T - 1) > job.pos + tt - 1;
                if (ok && E4M3) {
                    ok = mma_issue_codes(sh, tmem, qdesc0, kdesc0, vdesc0, nq, T, skip_last, a.timeout_ns);
                } else if (ok) {
                    const uint32_t id_qk = idesc_bf16_f32(128, 128, 0), id_pv = idesc_bf16_f32(128, 128, 1);
                    ok = nq == 2 ? mma_issue_loop<2>(&bars, tmem, qdesc0, kdesc0, vdesc0, id_qk, id_pv, T, skip_last,
                                                     a.timeout_ns, &abort_flag)
                                 : mma_issue_loop<1>(&bars, tmem, qdesc0, kdesc0, vdesc0, id_qk, id_pv, T, false,
                                                     a.timeout_ns, &abort_flag);
                }
                if (!ok) {
                    fail(&abort_flag, a.status);
                    mma_commit(&bars.drain);
                    mbar_wait_bounded(&bars.drain, 0, a.timeout_ns, nullptr);
                }
            }
        } else if (E4M3 && warp >= 12) {
            // ------------------------------------------------------------ V: codes to bf16
            // Eight lanes take a row, 16 codes each; a warp takes four rows of every 16. The two 16-byte pieces
            // that 16 codes become go to the swizzled place, the lanes of the second half in the other order, so
            // that eight lanes write 128 bytes of different banks. Lane x keeps the scale of the warp's row x, looked
            // up two tiles ahead (the page) and one ahead (the byte).
            const int x = tid - 384, sub = x & 7, r16 = x >> 3;
            const int c0 = 2 * (sub & 3), late = sub >> 2;
            const int my_row = 16 * (lane >> 2) + 4 * (warp - 12) + (lane & 3);
            uint64_t* const s_last = bars.s_full[nq - 1];
            auto place_of = [&](int t) { return t < T ? cache_row(a.c, a.b, job.b, jv.token_of(t) + my_row) : -1; };
            auto byte_of = [&](int place) -> uint32_t {
                if (place < 0) return 127u;
                const int page = place / a.c.page_size;
                return a.c.vs[(static_cast<int64_t>(page) * a.c.Hkv + job.j) * a.c.page_size + place - page * a.c.page_size];
            };
            uint32_t next_scale = byte_of(place_of(0));
            int next_place = place_of(1);
            bool ok = true;
            for (int t = 0; t < T; ++t) {
                const int st = t & 1;
                const uint32_t scale = next_scale;
                next_scale = byte_of(next_place);
                next_place = place_of(t + 2);
                // the bf16 stage was last read by the product with V(t - 2), which S(t - 1) was issued after
                ok = (t < 2 || mbar_wait_bounded(&s_last[st ^ 1], ((t - 1) >> 1) & 1, a.timeout_ns, &abort_flag)) &&
                     mbar_wait_bounded(&sh.raw_full[st], (t >> 1) & 1, a.timeout_ns, &abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                const uint8_t* from = smem + off_raw(true) + st * kCodeBytes + r16 * kHeadDim + sub * 16;
                uint8_t* to = smem + off_v(true) + st * kTileBytes + (sub >> 2) * kHalf + r16 * 128;
                uint8_t* const to0 = to + (((c0 + late) ^ (r16 & 7)) << 4);
                uint8_t* const to1 = to + (((c0 + 1 - late) ^ (r16 & 7)) << 4);
                const int t0 = jv.token_of(t);
                const bool unseen = jv.has_unseen(t0);
#pragma unroll 1  // (the instruction cache: see mma_issue_codes)
                for (int i = 0; i < 8; ++i) {
                    const uint4 w = *reinterpret_cast<const uint4*>(from + i * 16 * kHeadDim);
                    const float f = scale_value(__shfl_sync(0xFFFFFFFFu, scale, 4 * i + (lane >> 3)));
                    const uint2 y0 = e4m3x4_to_bf16(w.x, f), y1 = e4m3x4_to_bf16(w.y, f);
                    const uint2 y2 = e4m3x4_to_bf16(w.z, f), y3 = e4m3x4_to_bf16(w.w, f);
                    uint4 p = make_uint4(y0.x, y0.y, y1.x, y1.y), q = make_uint4(y2.x, y2.y, y3.x, y3.y);
                    if (unseen && jv.unseen(t0 + 16 * i + r16)) p = q = make_uint4(0, 0, 0, 0);
                    *reinterpret_cast<uint4*>(to0 + i * 16 * 128) = late ? q : p;
                    *reinterpret_cast<uint4*>(to1 + i * 16 * 128) = late ? p : q;
                }
                mbar_arrive(&sh.raw_empty[st]);
                fence_proxy_async_smem();
                mbar_arrive(&sh.v_full[st]);
            }
            if (!ok) fail(&abort_flag, a.status);
        }
    } else {
        if (E4M3) asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        // ------------------------------------------------------------ softmax + epilogue
        const int qt = warp >> 2;
        const int quarter = warp & 3;
        const int r = quarter * 32 + lane;
        const uint32_t lane_base = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
        const uint32_t s_addr = lane_base + qt * 256;
        const uint32_t o_addr = s_addr + 128;
        float* const ks = reinterpret_cast<float*>(smem + off_scales(E4M3)) + warp * kTile;
        // p = 2^(s scale - m) of keys [64 h, 64 h + 64) as bf16 pairs; returns their sum
        // (8-bit: a scale for each key, from shared memory)
        // The scales are loaded sixteen keys ahead: read where they are used, 32 waits for shared memory, which the
        // products keep busy, took a tile's softmax from 1,250 to 3,000 cycles.
        const uint32_t ks_at = smem_addr(ks);
        auto load_scales = [&](float4 (&f)[4], int c) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = lds_f4(ks_at + (c + 4 * i) * 4);
        };
        auto exp_half = [&](const float* s, int h, float neg_m, uint32_t (&pk)[32]) {
            float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            float4 f[2][4];
            if (E4M3) load_scales(f[0], h * 64);
#pragma unroll
            for (int b = 0; b < 4; ++b) {  // sixteen keys
                if (E4M3 && b < 3) load_scales(f[(b + 1) & 1], h * 64 + 16 * (b + 1));
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int i = 8 * b + k;
                    const float4 q = f[b & 1][k >> 1];
                    const float f0 = E4M3 ? (k & 1 ? q.z : q.x) : a.a.scale_log2, f1 = E4M3 ? (k & 1 ? q.w : q.y) : a.a.scale_log2;
                    float x0, x1;
                    ffma2(x0, x1, s[h * 64 + 2 * i], s[h * 64 + 2 * i + 1], f0, f1, neg_m, neg_m);
                    x0 = ex2(x0);
                    x1 = ex2(x1);
                    const int jj = (i & 3) * 2;
                    fadd2(acc[jj], acc[jj + 1], acc[jj], acc[jj + 1], x0, x1);
                    pk[i] = pack_bf16x2(x0, x1);
                }
            }
            return ((acc[0] + acc[1]) + (acc[2] + acc[3])) + ((acc[4] + acc[5]) + (acc[6] + acc[7]));
        };
        float m_run = -INFINITY, l_run = 0.f;
        bool ok = true;
        // What the loop keeps of the job: its key tiles from k0 on, those from `sinks` on `past` further; the row's token p,
        // the tile's first, which is also the last that all of the tile's rows see (8-bit: or -1, to mask every tile), and the
        // first from which the window hides nothing of the tile; the CTA's last token
        int T = 0, k0 = 0, sinks = 0, past = 0, p = 0, pos_first = 0, plain_to = 0, open_from = 0, last = 0;
        int seq = 0, kvh = 0;
        auto token_of = [&](int t) { return (k0 + t < sinks ? k0 + t : k0 + t + past) * kTile; };
        // 8-bit: lane x looks up the scales of the keys 4 x .. 4 x + 3 of a tile, its page two tiles ahead, the bytes one
        // ahead. (A warp that did it for both query tiles came late: 600 cycles a tile.)
        int next_place = -1;
        uint32_t next_scales = 0x7F7F7F7Fu;
        float q_scale = 0.f, row_scale = 1.f;  // of the warp's logits, beside its keys' scales; of this row's besides
        auto place_of = [&](int t) { return t < T ? cache_row(a.c, a.b, seq, token_of(t) + 4 * lane) : -1; };
        auto scales_of = [&](int place) -> uint32_t {
            if (place < 0) return 0x7F7F7F7Fu;
            const int page = place / a.c.page_size;
            return *reinterpret_cast<const uint32_t*>(a.c.ks + (static_cast<int64_t>(page) * a.c.Hkv + kvh) * a.c.page_size + place - page * a.c.page_size);
        };
        auto write_scales = [&]() {  // not 0: hidden logits stay -inf
            *reinterpret_cast<float4*>(ks + 4 * lane) = make_float4(fmaxf(scale_value(next_scales & 255u) * q_scale, 1e-37f),
                                                                    fmaxf(scale_value((next_scales >> 8) & 255u) * q_scale, 1e-37f),
                                                                    fmaxf(scale_value((next_scales >> 16) & 255u) * q_scale, 1e-37f),
                                                                    fmaxf(scale_value(next_scales >> 24) * q_scale, 1e-37f));
            __syncwarp();
        };
        // Tile -1 is whatever TMEM and shared memory hold: its softmax brings the code into the instruction cache
        // while the CTA waits for the plan (the first tile of a call took 10,000 to 20,000 cycles for that).
#pragma unroll 1
        for (int t = first_wave ? -1 : 0;; ++t) {
            if (t == 0) {
                const JobView jv = load_job(a);
                T = qt < jv.nq ? jv.T : 0;
                k0 = jv.job.k0;
                sinks = jv.tiles.sinks;
                past = jv.tiles.first - jv.tiles.sinks;
                seq = jv.job.b;
                kvh = jv.job.j;
                last = jv.last;
                pos_first = plain_to = jv.job.pos + qt * tt;
                const int pos_last = qt + 1 == jv.nq ? jv.last : pos_first + tt - 1;
                p = pos_first + r / g;
                p = p < pos_last ? p : pos_last;  // rows past the tile's end see what its last row sees
                open_from = a.a.n_local >= 0 && pos_last > a.a.n_local ? pos_last - a.a.n_local : 0;
                m_run = -INFINITY;
                l_run = 0.f;
                if (E4M3 && T > 0) {
                    next_scales = scales_of(place_of(0));
                    next_place = place_of(1);
                    // Q to two e4m3 parts, Q = Q1 + Q2, by a power of two that brings the largest finite |q| to 2^7 .. 2^8. Q1
                    // takes four of the eight significant bits, Q2 the rest; half of Q2's least step, 2^-10 or 2^-17 of the
                    // largest, is lost at most. The power is one for the warp's rows, which the keys' scales (the warp's)
                    // take along, unless a row is more than 2^kRowsApart below the largest: then each row has its own, and all
                    // tiles take the slow path, which multiplies its logits by it. Not finite becomes NaN.
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(&bars.q_full, 0, a.timeout_ns, &abort_flag));
                    uint8_t* row = smem + kOffQ + qt * kTileBytes + r * 128;
                    uint4 w[16];  // dimensions 8 i .. 8 i + 7
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = *reinterpret_cast<const uint4*>(row + (i >> 3) * kHalf + (((i & 7) ^ (r & 7)) << 4));
                    uint32_t top = 0;
                    if (r < (qt + 1 == jv.nq ? jv.job.ntok - qt * tt : tt) * g) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint32_t x = (v[e] << 16) & 0x7FFFFFFFu, y = v[e] & 0x7FFF0000u;
                                top = max(top, max(x >= 0x7F800000u ? 0u : x, y >= 0x7F800000u ? 0u : y));
                            }
                        }
                    }
                    const int e_row = f16_exponent(top) + 7, e_warp = f16_exponent(__reduce_max_sync(0xFFFFFFFFu, top)) + 7;
                    const bool rows_apart = __any_sync(0xFFFFFFFFu, top != 0 && e_row < e_warp - kRowsApart);
                    const int e = rows_apart ? e_row : e_warp;
                    const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
                    const float up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
                    row_scale = rows_apart ? up : 1.f;
                    if (rows_apart) plain_to = -1;
                    q_scale = rows_apart ? a.a.scale_log2 : a.a.scale_log2 * up;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {  // 16 dimensions: one 16-byte piece of each part
                        const uint32_t v[8] = {w[2 * i].x, w[2 * i].y, w[2 * i].z, w[2 * i].w, w[2 * i + 1].x, w[2 * i + 1].y, w[2 * i + 1].z, w[2 * i + 1].w};
                        uint32_t hi[4], lo[4];
#pragma unroll
                        for (int e4 = 0; e4 < 4; ++e4) {
                            hi[e4] = lo[e4] = 0;
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const float x = __uint_as_float(v[2 * e4 + k] << 16) * down, y = __uint_as_float(v[2 * e4 + k] & 0xFFFF0000u) * down;
                                const uint32_t h = f32_to_e4m3x2(x, y);
                                const float2 back = f16x2_to_f32(e4m3x2_to_f16x2(h));
                                hi[e4] |= h << (16 * k);
                                lo[e4] |= f32_to_e4m3x2(fmaf(x, 0.f, x - back.x), fmaf(y, 0.f, y - back.y)) << (16 * k);  // infinity * 0 = NaN
                            }
                        }
                        uint8_t* at = row + ((i ^ (r & 7)) << 4);
                        *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                        *reinterpret_cast<uint4*>(at + kCodeBytes) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                    }
                    fence_proxy_async_smem();
                    named_barrier(2, 128 * jv.nq);
                    if (qt == 0) mbar_arrive(&sh.q_ready);
                }
            }
            if (t >= T && t >= 0) break;
            if (E4M3) {  // while the products are made
                write_scales();
                next_scales = scales_of(next_place);
                next_place = place_of(t + 2);
            }
            if (t >= 0) {
                const bool got = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(&bars.s_full[qt][t & 1], (t >> 1) & 1, a.timeout_ns, &abort_flag));
                if (!got) {
                    ok = false;
                    break;
                }
            }
            tc_fence_after();
            const int t0 = token_of(t);
            const bool masked = t < 0 || t0 + kTile - 1 > plain_to || (t0 < open_from && t0 + kTile - 1 >= a.a.n_sink);
            const int lim = p - t0 + 1;  // keys t0 + c with c >= lim are in the future
            const int gap = a.a.n_sink - t0, low = a.a.n_local >= 0 && p - t0 > a.a.n_local ? p - t0 - a.a.n_local : 0;
            // Fast: exponentials against the reference as it stands, all of the row at once, unless something is hidden or
            // the sum shows a logit far above the reference (the limits of k_sparse_attn). Slow: the maximum first, and 32
            // columns at a time in loops, so that its instructions leave the fast path's in the cache (4,096 tokens
            // over 64K: 2,730 us with both paths unrolled).
            bool slow = masked || !__all_sync(0xFFFFFFFFu, m_run != -INFINITY);
            float sum = 0.f;
            if (!slow || t < 0) {
                uint32_t sr[128], pk[2][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&sr[c * 32]));
                tmem_ld_wait();
                const float* s = reinterpret_cast<const float*>(sr);
                sum = exp_half(s, 0, -m_run, pk[0]);
                sum += exp_half(s, 1, -m_run, pk[1]);
                slow = slow || __any_sync(0xFFFFFFFFu, !(sum <= kFastSumLimit));
                if (!slow) {
                    tmem_st32(s_addr, pk[0]);
                    tmem_st32(s_addr + 32, pk[1]);
                }
            }
            if (slow) {
                // a bit per column: columns below x of these 32 are ones_below(x - 32 c)
                auto load_32 = [&](uint32_t (&sr)[32], int c) {
                    tmem_ld32(s_addr + c * 32, sr);
                    const uint32_t seen = masked ? ones_below(lim - 32 * c) & ~(ones_below(low - 32 * c) & ~ones_below(gap - 32 * c)) : 0xFFFFFFFFu;
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        if (E4M3) sr[i] = __float_as_uint(__uint_as_float(sr[i]) * row_scale);
                        if (!((seen >> i) & 1u)) sr[i] = 0xFF800000u;
                    }
                };
                float mx = -INFINITY;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t sr[32];
                    load_32(sr, c);
                    const float* s = reinterpret_cast<const float*>(sr);
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 f = E4M3 ? lds_f4(ks_at + (32 * c + i) * 4) : make_float4(1.f, 1.f, 1.f, 1.f);
                        mx = E4M3 ? fmax3(mx, s[i] * f.x, s[i + 1] * f.y) : fmax3(mx, s[i], s[i + 1]);
                        mx = E4M3 ? fmax3(mx, s[i + 2] * f.z, s[i + 3] * f.w) : fmax3(mx, s[i + 2], s[i + 3]);
                    }
                }
                const float m_new = fmaxf(m_run, E4M3 ? mx : mx * a.a.scale_log2);
                const bool raise = m_new > m_run + kRescaleThreshold;
                // the O rescale is warp-collective: taken by the whole warp when any row needs it
                if (__any_sync(0xFFFFFFFFu, raise)) {
                    const float alpha = raise ? ex2(m_run - m_new) : 1.0f;
                    l_run *= alpha;
                    if (t > 0) {
#pragma unroll 1
                        for (int c = 0; c < 8; ++c) {
                            uint32_t v[16];
                            tmem_ld16(o_addr + c * 16, v);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * alpha);
                            tmem_st16(o_addr + c * 16, v);
                        }
                    }
                    if (raise) m_run = m_new;
                }
                const float neg_m = (m_run == -INFINITY) ? 0.f : -m_run;
                sum = 0.f;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t sr[32], pk[16];
                    load_32(sr, c);
                    const float* s = reinterpret_cast<const float*>(sr);
                    float acc0 = 0.f, acc1 = 0.f;
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 f = E4M3 ? lds_f4(ks_at + (32 * c + i) * 4) : make_float4(a.a.scale_log2, a.a.scale_log2, a.a.scale_log2, a.a.scale_log2);
                        float x0, x1, x2, x3;
                        ffma2(x0, x1, s[i], s[i + 1], f.x, f.y, neg_m, neg_m);
                        ffma2(x2, x3, s[i + 2], s[i + 3], f.z, f.w, neg_m, neg_m);
                        x0 = ex2(x0);
                        x1 = ex2(x1);
                        x2 = ex2(x2);
                        x3 = ex2(x3);
                        fadd2(acc0, acc1, acc0, acc1, x0, x1);
                        fadd2(acc0, acc1, acc0, acc1, x2, x3);
                        pk[i / 2] = pack_bf16x2(x0, x1);
                        pk[i / 2 + 1] = pack_bf16x2(x2, x3);
                    }
                    sum += acc0 + acc1;
                    if (t >= 0) tmem_st16(s_addr + 16 * c, pk);  // over columns that are read; in tile -1 the first products may be on their way
                    else sum += __uint_as_float(pk[15]);         // keeps the code
                }
            }
            l_run += sum;
            if (E4M3) __syncwarp();  // the tile's scales are read
            if (t < 0) continue;
            tmem_st_wait();
            if (!E4M3 && qt == 0 && masked) {
                // value rows that no row of the CTA sees: 0 times what lies there may be NaN. The MMA thread waits for this
                // group before either query tile's product with them; the next load into the stage waits for those.
                const bool landed = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(&bars.kv_full[(t + 1) & 1], ((t + 1) >> 1) & 1, a.timeout_ns, &abort_flag));
                if (!landed) {
                    ok = false;
                    break;
                }
                const int tok = t0 + r, lo = a.a.n_local >= 0 && pos_first > a.a.n_local ? pos_first - a.a.n_local : 0;
                if (tok > last || (tok < lo && tok >= a.a.n_sink)) {
                    uint8_t* row = smem + off_v(false) + (t & 1) * kTileBytes + r * 128;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        *reinterpret_cast<uint4*>(row + (i >> 3) * kHalf + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_proxy_async_smem();
            }
            tc_fence_before();
            mbar_arrive(&bars.p_full[qt]);
        }
        if (T > 0) {
            const JobView jv = load_job(a);  // (again: nothing of it is kept through the loop)
            const ChunkJob& job = jv.job;
            bool go = __all_sync(0xFFFFFFFFu, ok && !abort_flag);
            if (go) go = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(&bars.o_full, 0, a.timeout_ns, &abort_flag));
            if (go) {
                tc_fence_after();
                // Every MMA is done and every copy landed, so the tiles in shared memory are free: a warp
                // stages its 32 output rows there and stores whole rows.
                const int rows = (qt + 1 == jv.nq ? job.ntok - qt * tt : tt) * g - quarter * 32;  // of this warp, if more than 0
                if (job.slot < 0) {
                    const float inv_l = l_run > 0.f ? 1.0f / l_run : 0.f;
                    uint32_t v[128];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(o_addr + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&v[c * 32]));
                    tmem_ld_wait();
                    uint8_t* stage = smem + kOffQ + qt * kTileBytes + quarter * 32 * 256;
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            w[i] = pack_bf16x2(__uint_as_float(v[8 * c + 2 * i]) * inv_l, __uint_as_float(v[8 * c + 2 * i + 1]) * inv_l);
                        if (!(l_run > 0.f)) w[0] = w[1] = w[2] = w[3] = l_run == 0.f ? 0u : 0x7FFF7FFFu;  // no keys: 0; NaN stays
                        *reinterpret_cast<uint4*>(stage + lane * 256 + ((c ^ (lane & 15)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    __syncwarp();
                    const int c = lane & 15;
#pragma unroll 4
                    for (int i = 0; i < 16; ++i) {
                        const int x = 2 * i + (lane >> 4), rr = quarter * 32 + x;
                        const uint4 w = *reinterpret_cast<const uint4*>(stage + x * 256 + ((c ^ (x & 15)) << 4));
                        if (x < rows) {
                            const int64_t row = job.row0 + qt * tt + rr / g;
                            auto* out = static_cast<__nv_bfloat16*>(a.a.out) + row * a.a.out_stride + (job.j * g + rr % g) * kHeadDim;
                            reinterpret_cast<uint4*>(out)[c] = w;
                        }
                    }
                    if (a.a.lse && lane < rows)
                        a.a.lse[static_cast<int64_t>(job.row0 + qt * tt + r / g) * a.a.Hq + job.j * g + r % g] =
                            l_run == 0.f ? -INFINITY : (m_run + __log2f(l_run)) * 0.6931471805599453f;
                } else {
                    uint8_t* stage = smem + warp * 32 * 512;  // 128 KB of tiles
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t v[32];
                        tmem_ld32(o_addr + c * 32, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            *reinterpret_cast<uint4*>(stage + lane * 512 + (((c * 8 + i) ^ lane) << 4)) =
                                make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                    }
                    __syncwarp();
                    const int64_t at = static_cast<int64_t>(job.slot) * a.part_rows + qt * kTile + quarter * 32;
                    uint4* dst = reinterpret_cast<uint4*>(a.part_o + at * kHeadDim) + lane;
#pragma unroll 8
                    for (int x = 0; x < 32; ++x)
                        if (x < rows) dst[x * (kHeadDim / 4)] = *reinterpret_cast<const uint4*>(stage + x * 512 + ((lane ^ x) << 4));
                    if (lane < rows) a.part_ml[at + lane] = make_float2(m_run, l_run);
                }
            } else {
                fail(&abort_flag, a.status);
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Pieces of a query tile pair put together: a warp takes four rows, four dimensions a lane, and eight pieces at a time,
// whose references and sums the lanes hold (lane 8 i + p: row i, piece p). Bound by the latency of its loads, which
// depend on nothing but the list: eight rows are on their way at a time. 9 sequences of 1 to 700 new tokens, 8 KV heads,
// 176 pairs in two or three pieces: the call takes 129 us, and 134 with a warp per row that looks the weights up piece by
// piece. A grid of what the SMs hold walks the rows: one CTA for eight of every row that could be cut took 12 us, most of
// it for CTAs without a row.
constexpr int kMergeCtas = 4;  // per SM, of 256 threads

__global__ void __launch_bounds__(256, kMergeCtas) k_chunk_merge(const __grid_constant__ ChunkArgs a)
{
    pdl_enter();
    const int lane = threadIdx.x & 31, per_tile = a.tile_tokens * a.a.g;
    const int total = a.p.counts[1] * (a.part_rows / 4);  // at most 2 kMaxSms pairs of 64
    const int step = gridDim.x * 8;
#pragma unroll 1
    for (int w = blockIdx.x * 8 + (threadIdx.x >> 5); w < total; w += step) {
        const int m = w / (a.part_rows / 4);
        const int r = (w - m * (a.part_rows / 4)) * 4;       // first row of the pair's tiles
        const int4 y0 = reinterpret_cast<const int4*>(a.p.merges + m)[0];  // KV head, first row, tokens, slot
        const int pieces = a.p.merges[m].pieces;
        // live rows: those of the first tile below per_tile, then those of the second
        auto live_row = [&](int rr) { return rr < kTile ? (rr < per_tile ? rr : y0.z * a.a.g) : per_tile + rr - kTile; };
        if (live_row(r) >= y0.z * a.a.g) continue;
        const float* from = a.part_o + (static_cast<int64_t>(y0.w) * a.part_rows + r) * kHeadDim + lane * 4;
        const float2* ml_at = a.part_ml + static_cast<int64_t>(y0.w) * a.part_rows + r + (lane >> 3);
        float top = -INFINITY, sum = 0.f;  // of row lane >> 3, the same in its eight lanes
        float4 acc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int p0 = 0; p0 < pieces; p0 += 8) {
            const int p = p0 + (lane & 7);
            const float2 ml = p < pieces ? __ldcg(ml_at + static_cast<int64_t>(p) * a.part_rows) : make_float2(-INFINITY, 0.f);
            float mx = ml.x;
            for (int o = 4; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o));
            const float now = fmaxf(top, mx), base = now == -INFINITY ? 0.f : now;
            const float old = ex2(top - base);  // 0 for the first eight
            const float f = ex2(ml.x - base);
            float part = ml.y * f;
            for (int o = 4; o > 0; o >>= 1) part += __shfl_xor_sync(0xFFFFFFFFu, part, o);
            sum = fmaf(sum, old, part);
            top = now;
            if (p0 > 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = __shfl_sync(0xFFFFFFFFu, old, 8 * i);
                    acc[i] = make_float4(acc[i].x * x, acc[i].y * x, acc[i].z * x, acc[i].w * x);
                }
            }
            const int n = pieces - p0 < 8 ? pieces - p0 : 8;
#pragma unroll 2
            for (int q = 0; q < n; ++q) {
                const float* row = from + static_cast<int64_t>(p0 + q) * a.part_rows * kHeadDim;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 o = __ldcg(reinterpret_cast<const float4*>(row + i * kHeadDim));
                    const float x = __shfl_sync(0xFFFFFFFFu, f, 8 * i + q);
                    acc[i].x = fmaf(o.x, x, acc[i].x);
                    acc[i].y = fmaf(o.y, x, acc[i].y);
                    acc[i].z = fmaf(o.z, x, acc[i].z);
                    acc[i].w = fmaf(o.w, x, acc[i].w);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float l = __shfl_sync(0xFFFFFFFFu, sum, 8 * i), mx = __shfl_sync(0xFFFFFFFFu, top, 8 * i);
            const int x = live_row(r + i);
            if (x >= y0.z * a.a.g) continue;
            const float inv = l == 0.f ? 0.f : 1.0f / l;
            const int64_t row = y0.y + x / a.a.g;
            const int h = y0.x * a.a.g + x % a.a.g;
            auto* out = static_cast<__nv_bfloat16*>(a.a.out) + row * a.a.out_stride + h * kHeadDim;
            reinterpret_cast<uint2*>(out)[lane] = make_uint2(pack_bf16x2(acc[i].x * inv, acc[i].y * inv), pack_bf16x2(acc[i].z * inv, acc[i].w * inv));
            if (a.a.lse && lane == 0) a.a.lse[row * a.a.Hq + h] = l == 0.f ? -INFINITY : (mx + __log2f(l)) * 0.6931471805599453f;
        }
    }
}

// Workspace regions (byte offsets from the route's part of the workspace).
struct ChunkWs {
    size_t counts, jobs, merges, part_ml, part_o, end;
    int max_jobs, max_merges, max_slots, part_rows;
};

ChunkWs chunk_layout(int g, int Hkv, int n_seqs, int n_rows, int max_rows)
{
    ChunkWs w{};
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align_up(off + bytes, kAlign);
        return at;
    };
    const int tt = kTile / g;
    // every sequence adds one incomplete pair of tiles at most; none has more than max_rows
    int64_t pairs = static_cast<int64_t>(n_rows) / (2 * tt) + n_seqs;
    const int64_t each = (static_cast<int64_t>(max_rows) + 2 * tt - 1) / (2 * tt);
    if (pairs > each * n_seqs) pairs = each * n_seqs;
    const int64_t items = pairs * Hkv;
    // What is cut: all items of a call of few, an item and kCuts pieces per SM; of many, the rest (kCutsRest) and of the others
    // those longer than an SM's share, a job for each SM more at most, which is two pieces. The actual number of items may
    // be below this bound and count as few.
    const int64_t few = items < 2 * kMaxSms ? items : 2 * kMaxSms;
    static_assert(kCuts >= kCutsRest + 1, "jobs of either kind of call");
    const int64_t slots = few + kCuts * kMaxSms;
    w.max_merges = static_cast<int>(few);
    w.max_jobs = static_cast<int>(items + kCuts * kMaxSms);
    w.max_slots = static_cast<int>(slots);
    w.part_rows = max_rows > tt ? 2 * kTile : kTile;
    w.counts = take(2 * sizeof(int32_t));
    w.jobs = take(static_cast<size_t>(w.max_jobs) * sizeof(ChunkJob));
    w.merges = take(static_cast<size_t>(w.max_merges) * sizeof(ChunkMerge));
    w.part_ml = take(static_cast<size_t>(slots) * w.part_rows * sizeof(float2));
    w.part_o = take(static_cast<size_t>(slots) * w.part_rows * kHeadDim * sizeof(float));
    w.end = off;
    return w;
}

template <bool E4M3>
cudaError_t run_chunks(const ChunkArgs& a, cudaStream_t st)
{
    CUtensorMap tq, tk, tv;
    const uint64_t pool = static_cast<uint64_t>(a.c.num_pages) * a.c.page_size;
    bool ok = scale_host::make_rows_map(&tq, a.a.q, kHeadDim, a.a.Hq, a.a.q_stride, a.b.n_rows, a.a.g, a.tile_tokens);
    if (E4M3)
        ok = ok && scale_host::make_byte_rows_map(&tk, a.c.k, kHeadDim, a.c.Hkv, pool, a.box, true) &&
             scale_host::make_byte_rows_map(&tv, a.c.v, kHeadDim, a.c.Hkv, pool, a.box, false);
    else
        ok = ok && scale_host::make_token_major_map(&tk, a.c.k, kHeadDim, a.c.Hkv, pool, 64, a.box) &&
             scale_host::make_token_major_map(&tv, a.c.v, kHeadDim, a.c.Hkv, pool, 64, a.box);
    if (!ok) return cudaErrorInvalidValue;
    cudaError_t e = cudaFuncSetAttribute(k_chunk<E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(chunk_smem(E4M3)));
    if (e == cudaSuccess) e = launch_after(st, dim3(1), kPlanThreads, 0, 1, k_chunk_plan, a);
    if (e == cudaSuccess)
        e = launch_after(st, dim3(a.p.max_jobs), chunk_threads(E4M3), chunk_smem(E4M3), 1, k_chunk<E4M3>, tq, tk, tv, a);
    const int merge_ctas = a.p.max_merges * (a.part_rows / 32), most = a.sms * kMergeCtas;
    if (e == cudaSuccess) e = launch_after(st, dim3(merge_ctas < most ? merge_ctas : most), 256, 0, 1, k_chunk_merge, a);
    return e;
}

}  // namespace

size_t chunk_ws_bytes(int g, int Hkv, int n_seqs, int n_rows, int max_rows)
{
    return chunk_layout(g, Hkv, n_seqs, n_rows, max_rows).end;
}

cudaError_t launch_chunks(const AttendView& a, const CacheView& c, bool e4m3, const BatchView& b, int sms,
                          int32_t* status, uint8_t* ws, uint64_t timeout_ns, cudaStream_t st)
{
    const ChunkWs w = chunk_layout(a.g, c.Hkv, b.n_seqs, b.n_rows, b.max_rows);
    ChunkArgs x{};
    x.a = a;
    x.c = c;
    x.b = b;
    x.p = ChunkPlan{reinterpret_cast<int32_t*>(ws + w.counts), reinterpret_cast<ChunkJob*>(ws + w.jobs),
                    reinterpret_cast<ChunkMerge*>(ws + w.merges), w.max_jobs, w.max_merges, w.max_slots};
    x.sms = sms;
    x.tile_tokens = kTile / a.g;
    x.box = 16;
    while (x.box < kTile && c.page_size % (2 * x.box) == 0) x.box *= 2;
    x.part_o = reinterpret_cast<float*>(ws + w.part_o);
    x.part_ml = reinterpret_cast<float2*>(ws + w.part_ml);
    x.part_rows = w.part_rows;
    x.status = status;
    x.timeout_ns = timeout_ns;
    return e4m3 ? run_chunks<true>(x, st) : run_chunks<false>(x, st);
}

}  // namespace scale
