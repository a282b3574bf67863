// attend.cu -- attention of a batch's new tokens over their sequences in a
// paged cache (scale_cache_attend).
#include <cuda_bf16.h>

#include "attend.cuh"
#include "launch.cuh"
#include "ptx_sm103.cuh"
#include "scale_internal.h"

namespace scale {
namespace {

using namespace scale_ptx;

// ---------------------------------------------------------------- few rows: decode

constexpr int kStep = 16;          // keys of a step; a page holds whole steps
// Steps of a CTA before another one helps: one token at 4K, 4 heads, 8.3 us (8.7, 9.5 with 4 and 9.9 with 32, when it was chosen)
constexpr int kMinSteps = 8;
constexpr float kRaise = 8.0f;     // log2 units by which a logit may pass the reference
constexpr float kLift = 6.0f;      // 8-bit: log2 units that a new reference lies below the largest logit

// Warps of a CTA and stages of a warp's ring. 8-bit rows of few query rows take half the copies and 1.3 times the
// instructions per byte: sixteen warps hide what eight with twice the stages left open (128K tokens 64 us).
__host__ __device__ constexpr int rows_warps(int nt, bool e4m3) { return e4m3 && nt == 1 ? 16 : 8; }
__host__ __device__ constexpr int rows_stages(int nt, bool e4m3) { return e4m3 && nt > 1 ? 6 : 3; }
__host__ __device__ constexpr int rows_step_bytes(bool e4m3) { return e4m3 ? 2 * kStep * kHeadDim + 2 * kStep : 4 * kStep * kHeadDim; }
__host__ __device__ constexpr int rows_warp_bytes(int nt, bool e4m3) { return rows_stages(nt, e4m3) * rows_step_bytes(e4m3); }
__host__ __device__ constexpr int rows_ring_bytes(int nt, bool e4m3) { return rows_warps(nt, e4m3) * rows_warp_bytes(nt, e4m3); }

// Steps of a sequence: those of the sinks, then those from the window's first.
struct Steps {
    int sinks, first, n;
};

__device__ __forceinline__ Steps steps_of(const AttendView& a, const Seq& s)
{
    Steps x;
    const int last = s.pos0 + s.rows - 1;  // below 0: one step that nothing of is seen, whose rows get 0
    x.first = s.lo / kStep;
    const int sinks = static_cast<int>((static_cast<int64_t>(a.n_sink) + kStep - 1) / kStep);
    x.sinks = sinks < x.first ? sinks : x.first;
    x.n = last < 0 ? 1 : x.sinks + last / kStep + 1 - x.first;
    return x;
}

struct RowsArgs {
    AttendView a;
    CacheView c;
    BatchView b;
    int64_t* before;   // [n_seqs + 1] steps (of one KV head) of the sequences before, for k_rows_merge
    float* part_o;     // [2 of each run][rows][128]
    float2* part_ml;   // [2 of each run][rows] (reference, sum)
    int part_rows;
};

// x / n, mostly of 32-bit numbers.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t n)
{
    return (x | n) >> 32 ? x / n : static_cast<uint32_t>(x) / static_cast<uint32_t>(n);
}

// How the steps are shared out: CTA c has the steps [c per_cta, (c + 1) per_cta), its warp w the run of per_warp of them
// from w per_warp on.
struct Runs {
    int64_t work, per_cta, per_warp;
    __device__ __forceinline__ Runs(int64_t n, int ctas, int warps) : work(n)
    {
        per_cta = quotient(n + ctas - 1, ctas);
        per_cta = per_cta < kMinSteps ? kMinSteps : per_cta;
        per_warp = quotient(per_cta + warps - 1, warps);
    }
    __device__ __forceinline__ int64_t cta_end(int64_t c) const { return (c + 1) * per_cta < work ? (c + 1) * per_cta : work; }
    __device__ __forceinline__ int64_t start(int64_t c, int64_t w) const { return c * per_cta + w * per_warp; }
    __device__ __forceinline__ int64_t end(int64_t c, int64_t w) const
    {
        const int64_t x = start(c, w + 1), y = cta_end(c);
        return x < y ? x : y;
    }
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// d += a (16 x 16) b (16 x 8), bf16 or f16
template <bool F16>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// One KV head's item of a sequence, as a warp walks it.
struct Item {
    int b, j;    // sequence, KV head
    int step;    // next step of it
    Seq s;
    Steps x;
};

// Attention of sequences with at most rows_max rows (new tokens times query heads of a KV head).
//
// The work is one list of 16-key steps, sequence by sequence and KV head by KV head, cut into equal runs, one
// per warp, whatever the lengths: a warp walks its run with a ring of its own in shared memory, so nothing in
// the loop waits for another warp and the copies run on across items. What the warps of a CTA have of the same item
// at the ends of their runs is added up there. The rows are the N side of the
// products: S^T = K Q^T with the step's 16 keys as M, O^T += V^T P^T with 16 dimensions as M, so rows are
// padded to 8 and not to 16 and a thread keeps the same two rows in both; P changes sides by a register
// transpose. The reference of a row's exponentials is raised only when a logit passes it by 2^8, so a step
// mostly has no reduction. A run that holds a part of an item leaves (O, reference, sum) to k_rows_merge.
//
// 8-bit rows stay codes up to the registers and become f16 there (exact, one conversion per two values);
// a key's scale multiplies its logit, a value's scale 2^e moves into the exponent, w' = 2^(s + e - m), and the sum
// takes w' 2^-e. Q is brought to f16 by a power of two per row.
//
// P is two bf16 parts (16 bits) beside bf16 values and f16 (11 bits) beside codes, where the reference is set kLift below
// the largest logit: f16 keeps its 11 bits down to 2^-14, so weights do down to 2^-20 of a run's largest, and to 2^-31 of it
// beyond. (w' stays below 2^kRaise either way.) The second product costs nothing that
// was measured, since the tensor pipe stood at 8 %: 48 tokens of 130 to 30,000, 16 of 4 tokens at 8,192 (16 rows) and one at
// 4K take as long with it as with one part of 8 bits.
//
// Keys that no row sees are not read: their places are filled with zeros, so nothing that lies there
// reaches a sum. Bound by HBM: K and V once. With 32 query heads on 8 and 28 on 4: one token at 128K, 8-bit (272 MB), 55 us
// with the merge (60 and 61 on other GPUs), 6.3 TB/s between a start of 6 us (launch, lengths, pages, first rows) and the
// merge of 6 us; 48 tokens of 130 to 30,000, bf16 (560 MB), 92 us, 7 TB/s in the loop; one at 4K 8.3 us, all latency.
template <int NT, bool E4M3>
__global__ void __launch_bounds__(32 * rows_warps(NT, E4M3), 1) k_rows(const __grid_constant__ RowsArgs args)
{
    constexpr int kStages = rows_stages(NT, E4M3), kWarps = rows_warps(NT, E4M3), kRowsThreads = 32 * kWarps;
    constexpr int kRow = E4M3 ? kHeadDim : 2 * kHeadDim;  // bytes of a held row
    constexpr int kTile = kStep * kRow;
    constexpr int kChunks = kRow / 16;
    static_assert(NT * 8 * (kHeadDim * 4 + 8) <= rows_warp_bytes(NT, E4M3), "a run's last piece lies in its ring");
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int64_t s_sum[kWarps];  // then the item that a warp's run ends in
    const AttendView& a = args.a;
    const CacheView& c = args.c;
    const BatchView& bt = args.b;
    int64_t* before = reinterpret_cast<int64_t*>(smem + rows_ring_bytes(NT, E4M3));
    pdl_enter();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int quad = lane & 3, oct = lane >> 2;

    // ---- steps before every sequence: each thread sums its stretch of them
    {
        const int per = (bt.n_seqs + kRowsThreads - 1) / kRowsThreads;
        const int i0 = tid * per, i1 = i0 + per < bt.n_seqs ? i0 + per : bt.n_seqs;
        int64_t sum = 0;
        for (int i = i0; i < i1; ++i) {
            const Seq s = seq_of(a, bt, i);
            before[i] = sum;
            if (s.rows > 0) sum += steps_of(a, s).n;
        }
        int64_t incl = sum;
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += y;
        }
        if (lane == 31) s_sum[warp] = incl;
        __syncthreads();
        int64_t base = incl - sum;
        for (int w = 0; w < warp; ++w) base += s_sum[w];
        for (int i = i0; i < i1; ++i) before[i] += base;
        if (tid == kRowsThreads - 1) before[bt.n_seqs] = base + sum;
        __syncthreads();
        if (blockIdx.x == 0)
            for (int i = tid; i <= bt.n_seqs; i += kRowsThreads) args.before[i] = before[i];
    }
    const Runs runs(before[bt.n_seqs] * c.Hkv, gridDim.x, kWarps);
    const int64_t run = static_cast<int64_t>(blockIdx.x) * kWarps + warp;
    const int64_t x0 = runs.start(blockIdx.x, warp), n = runs.end(blockIdx.x, warp) - x0;  // n <= 0: none
    const uint32_t ring = smem_addr(smem) + warp * rows_warp_bytes(NT, E4M3);
    int64_t open = -1;  // item that the run ends inside of

    if (n > 0) {
    auto enter = [&](Item& it, int b) {  // the first sequence from b on that has steps
        while (before[b + 1] == before[b]) ++b;
        it.b = b;
        it.s = seq_of(a, bt, b);
        it.x = steps_of(a, it.s);
    };
    Item load, use;
    int lp = 0, slot = 0, page = -1;  // where the step to load lies: page of the table, row in it, page of the pool
    auto look_up = [&]() { page = lp < bt.stride ? bt.table[static_cast<int64_t>(load.b) * bt.stride + lp] : -1; };
    {
        int lo = 0, hi = bt.n_seqs;  // the last sequence whose steps start at or before x0
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (before[mid] * c.Hkv <= x0) lo = mid;
            else hi = mid;
        }
        enter(load, lo);
        const int64_t rem = x0 - before[load.b] * c.Hkv;
        load.j = static_cast<int>(quotient(rem, load.x.n));
        load.step = static_cast<int>(rem - static_cast<int64_t>(load.j) * load.x.n);
        use = load;
    }
    // first token of step i of an item
    auto token_of = [&](const Item& it, int i) { return (i < it.x.sinks ? i : it.x.first + i - it.x.sinks) * kStep; };
    auto advance = [&](Item& it) {
        if (++it.step < it.x.n) return;
        it.step = 0;
        if (++it.j < c.Hkv) return;
        it.j = 0;
        if (it.b + 1 < bt.n_seqs && before[it.b + 1] < before[bt.n_seqs]) enter(it, it.b + 1);
    };
    auto find_page = [&]() {
        const int t = token_of(load, load.step);
        lp = static_cast<int>(static_cast<uint32_t>(t) / static_cast<uint32_t>(c.page_size));
        slot = t - lp * c.page_size;
        look_up();
    };
    auto advance_load = [&]() {
        const int it_step = load.step;
        advance(load);
        if (load.step == it_step + 1 && load.step != load.x.sinks) {  // the next 16 keys
            slot += kStep;
            if (slot >= c.page_size) {
                slot = 0;
                ++lp;
                look_up();
            }
        } else {
            find_page();
        }
    };
    constexpr int kRowsAtOnce = 32 / kChunks;  // rows that the warp's 16-byte copies cover
    const int my_row = lane / kChunks, my_chunk = lane % kChunks;
    const int64_t pitch = static_cast<int64_t>(c.Hkv) * kRow;
    auto copy_step = [&](int stage) {
        const int t0 = token_of(load, load.step);
        const int last = load.s.pos0 + load.s.rows - 1;
        const uint32_t dst = ring + stage * rows_step_bytes(E4M3);
        const bool in_pool = static_cast<uint32_t>(page) < static_cast<uint32_t>(c.num_pages);
        const int64_t first = in_pool ? static_cast<int64_t>(page) * c.page_size + slot : 0;
        const int64_t at = (first * c.Hkv + load.j) * kRow + my_row * pitch + my_chunk * 16;
        const uint8_t *k = c.k + at, *v = c.v + at;
        // the keys that some row sees: t <= last and (t >= lo or t < n_sink)
        const bool all = in_pool && t0 + kStep - 1 <= last && (t0 >= load.s.lo || t0 + kStep - 1 < a.n_sink);
#pragma unroll
        for (int i = 0; i < kTile / 512; ++i) {
            const int row = i * kRowsAtOnce + my_row, t = t0 + row;
            const bool real = all || (in_pool && t <= last && (t >= load.s.lo || t < a.n_sink));
            const uint32_t to = dst + row * kRow + ((my_chunk ^ (row & 7)) << 4);
            cp_async16(to, real ? k : c.k, real);
            cp_async16(to + kTile, real ? v : c.v, real);
            k += kRowsAtOnce * pitch;
            v += kRowsAtOnce * pitch;
        }
        if (E4M3 && lane < 2) {  // the step's 16 scales lie in one page
            const int64_t sc = in_pool ? (static_cast<int64_t>(page) * c.Hkv + load.j) * c.page_size + slot : 0;
            cp_async16(dst + 2 * kTile + lane * kStep, (lane ? c.vs : c.ks) + sc, in_pool);
        }
    };

    uint32_t qf[NT][8][2];            // Q^T, 16 dimensions at a time
    float q_scale[NT][2];             // 8-bit: the power of two that Q's row was divided by
    float o[8][NT][4];                // O^T: 16 dimensions at a time
    float m[NT][2], l[NT][2];         // per row: reference (log2 units, a warp's), sum of this lane's keys
    auto load_q = [&]() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = nt * 8 + oct;  // this lane's row of Q
            const bool live = r < use.s.rows * a.g;
            const auto* q = static_cast<const __nv_bfloat16*>(a.q) + static_cast<int64_t>(use.s.row0 + (live ? r / a.g : 0)) * a.q_stride +
                            (use.j * a.g + (live ? r % a.g : 0)) * kHeadDim;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // bf16: dimensions 16 i + 2 quad (+1), and 8 further; 8-bit: four in a row, as the codes come
                if (E4M3) {
                    const uint2 x = *reinterpret_cast<const uint2*>(q + 16 * i + 4 * quad);
                    qf[nt][i][0] = live ? x.x : 0u;
                    qf[nt][i][1] = live ? x.y : 0u;
                } else {
                    qf[nt][i][0] = live ? *reinterpret_cast<const uint32_t*>(q + 16 * i + 2 * quad) : 0u;
                    qf[nt][i][1] = live ? *reinterpret_cast<const uint32_t*>(q + 16 * i + 8 + 2 * quad) : 0u;
                }
            }
        }
    };
    auto begin_item = [&]() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (E4M3) {
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t lo = (qf[nt][i][e] << 16) & 0x7FFFFFFFu, hi = qf[nt][i][e] & 0x7FFF0000u;
                        top = max(top, max(lo >= 0x7F800000u ? 0u : lo, hi >= 0x7F800000u ? 0u : hi));
                    }
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const int ex = f16_exponent(top);
                const float down = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
                const float up = __uint_as_float(static_cast<uint32_t>(127 + ex) << 23);
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        qf[nt][i][e] = pack_f16x2(__uint_as_float(qf[nt][i][e] << 16) * down,
                                                  __uint_as_float(qf[nt][i][e] & 0xFFFF0000u) * down);
                // rows 2 quad, 2 quad + 1 of the tile are held by the lanes 8 quad, 8 quad + 4
                q_scale[nt][0] = __shfl_sync(0xFFFFFFFFu, up, 8 * quad);
                q_scale[nt][1] = __shfl_sync(0xFFFFFFFFu, up, 8 * quad + 4);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][nt][e] = 0.f;
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.f;
        }
    };
    // (O, reference, sum) of the item's steps [from, to): to the output when that is all of them, else to the warp's
    // ring at the run's end, else to the run's place for an item that ended inside it.
    auto end_item = [&](int from, int to, bool at_end) {
        const bool whole = from == 0 && to == use.x.n;
        float* const part = at_end ? reinterpret_cast<float*>(smem + warp * rows_warp_bytes(NT, E4M3))
                                   : args.part_o + 2 * run * args.part_rows * kHeadDim;
        float2* const part_ml = at_end ? reinterpret_cast<float2*>(part + NT * 8 * kHeadDim) : args.part_ml + 2 * run * args.part_rows;
        if (at_end && !whole) {
            cp_async_wait<0>();
            __syncwarp();
            open = static_cast<int64_t>(use.b) * c.Hkv + use.j;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[nt][e];
                sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 4);
                sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 8);
                sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 16);
                const int r = nt * 8 + 2 * quad + e;
                if (r >= use.s.rows * a.g) continue;
                const int64_t row = use.s.row0 + r / a.g;
                const int h = use.j * a.g + r % a.g;
                if (whole) {
                    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
                    auto* out = static_cast<__nv_bfloat16*>(a.out) + row * a.out_stride + h * kHeadDim;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float y0 = o[i][nt][e] * inv, y1 = o[i][nt][2 + e] * inv;
                        if (E4M3) {
                            *reinterpret_cast<uint32_t*>(out + 16 * i + 2 * oct) = pack_bf16x2(y0, y1);
                        } else {
                            out[16 * i + oct] = __float2bfloat16_rn(y0);
                            out[16 * i + 8 + oct] = __float2bfloat16_rn(y1);
                        }
                    }
                    if (a.lse && oct == 0)
                        a.lse[row * a.Hq + h] = sum == 0.f ? -INFINITY : (m[nt][e] + __log2f(sum)) * 0.6931471805599453f;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        part[r * kHeadDim + 16 * i + (E4M3 ? 2 * oct : oct)] = o[i][nt][e];
                        part[r * kHeadDim + 16 * i + (E4M3 ? 2 * oct + 1 : 8 + oct)] = o[i][nt][2 + e];
                    }
                    if (oct == 0) part_ml[r] = make_float2(m[nt][e], sum);
                }
            }
    };

    find_page();
    load_q();  // ahead of the copies
    auto load_next = [&](int64_t i, int stage) {
        if (i < n) {
            copy_step(stage);
            if (i + 1 < n) advance_load();
        }
        cp_async_commit();
    };
#pragma unroll 1
    for (int i = 0; i < kStages - 1; ++i) load_next(i, i);
    begin_item();
    int from = use.step;
    int stage = 0;
#pragma unroll 1
    for (int64_t i = 0; i < n; ++i) {
        cp_async_wait<kStages - 2>();
        __syncwarp();
        // the stage that step i - 1 was in is free: every lane is past its reads
        load_next(i + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
        const uint32_t kt = ring + stage * rows_step_bytes(E4M3), vt = kt + kTile;
        // ---- S^T = K Q^T
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
        if (E4M3) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {  // matrices: keys 0-7 and 8-15 of chunk 2 h, then of chunk 2 h + 1
                uint32_t r[4];
                const int row = lane & 15, ch = 2 * h + (lane >> 4);
                ldsm4(r, kt + row * kRow + ((ch ^ (row & 7)) << 4));
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t f[4] = {e4m3x2_to_f16x2(r[2 * e]), e4m3x2_to_f16x2(r[2 * e + 1]),
                                           e4m3x2_to_f16x2(r[2 * e] >> 16), e4m3x2_to_f16x2(r[2 * e + 1] >> 16)};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma16816<true>(s[nt], f, qf[nt][2 * h + e][0], qf[nt][2 * h + e][1]);
                }
            }
        } else {
#pragma unroll
            for (int h = 0; h < 8; ++h) {  // matrices: keys 0-7, 8-15 of dimensions 16 h .. + 7, then of the next eight
                uint32_t r[4];
                const int row = lane & 15, ch = 2 * h + (lane >> 4);
                ldsm4(r, kt + row * kRow + ((ch ^ (row & 7)) << 4));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma16816<false>(s[nt], r, qf[nt][h][0], qf[nt][h][1]);
            }
        }
        // ---- logits in log2 units: s[nt][2 x + e] is key oct + 8 x, row 2 quad + e
        float ev[2] = {0.f, 0.f}, back[2] = {1.f, 1.f};
        if (E4M3) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                uint32_t ks, vs;
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(ks) : "r"(kt + 2 * kTile + oct + 8 * x));
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(vs) : "r"(kt + 2 * kTile + kStep + oct + 8 * x));
                vs = vs == 0 ? 127u : vs < 253u ? vs : 253u;  // 0: a page outside the pool; the limit: hidden places hold anything
                const float k2 = scale_value(ks) * a.scale_log2;
                ev[x] = static_cast<float>(static_cast<int>(vs) - 127);
                back[x] = __uint_as_float((254u - vs) << 23);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) s[nt][2 * x + e] = fmaf(s[nt][2 * x + e], q_scale[nt][e] * k2, ev[x]);
            }
        } else {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nt][e] *= a.scale_log2;
        }
        const int t0 = token_of(use, use.step);
        const int last = use.s.pos0 + use.s.rows - 1;
        if (t0 + kStep - 1 > use.s.pos0 || (a.n_local >= 0 && last - t0 > a.n_local && t0 + kStep - 1 >= a.n_sink)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int p = use.s.pos0 + (nt * 8 + 2 * quad + e) / a.g;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int t = t0 + oct + 8 * x;
                        if (t > p || (a.n_local >= 0 && p - t > a.n_local && t >= a.n_sink)) s[nt][2 * x + e] = -INFINITY;
                    }
                }
        }
        // ---- references
        bool high = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) high |= fmaxf(s[nt][e], s[nt][2 + e]) > m[nt][e] + kRaise;
        if (__any_sync(0xFFFFFFFFu, high)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = fmaxf(s[nt][e], s[nt][2 + e]);
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
                    top = fmaxf(top - (E4M3 ? kLift : 0.f), m[nt][e]);
                    const float alpha = top == -INFINITY ? 1.f : ex2(m[nt][e] - top);
                    m[nt][e] = top;
                    l[nt][e] *= alpha;
#pragma unroll
                    for (int h = 0; h < 8; ++h) {
                        o[h][nt][e] *= alpha;
                        o[h][nt][2 + e] *= alpha;
                    }
                }
        }
        // ---- weights, and P^T; beside bf16 values in two parts, of which the second is what the first leaves of a weight
        uint32_t pf[NT][2], pf2[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float w[4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float base = m[nt][e] == -INFINITY ? 0.f : m[nt][e];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    w[2 * x + e] = ex2(s[nt][2 * x + e] - base);
                    l[nt][e] = fmaf(w[2 * x + e], back[x], l[nt][e]);
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint32_t p = E4M3 ? pack_f16x2(w[2 * x], w[2 * x + 1]) : pack_bf16x2(w[2 * x], w[2 * x + 1]);
                pf[nt][x] = transpose8x8(p);
                if (!E4M3)
                    pf2[nt][x] = transpose8x8(pack_bf16x2(w[2 * x] - __uint_as_float(p << 16), w[2 * x + 1] - __uint_as_float(p & 0xFFFF0000u)));
            }
        }
        // ---- O^T += V^T P^T
        if (E4M3) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                uint32_t r[4];
                const int row = lane & 15, ch = 2 * h + (lane >> 4);
                ldsm4_t(r, vt + row * kRow + ((ch ^ (row & 7)) << 4));
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // codes of dimensions (2 oct, 2 oct + 1) of two keys to one dimension of two keys
                    const uint32_t y0 = __byte_perm(r[2 * e], 0, 0x3120), y1 = __byte_perm(r[2 * e + 1], 0, 0x3120);
                    const uint32_t f[4] = {e4m3x2_to_f16x2(y0), e4m3x2_to_f16x2(y0 >> 16), e4m3x2_to_f16x2(y1), e4m3x2_to_f16x2(y1 >> 16)};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma16816<true>(o[2 * h + e][nt], f, pf[nt][0], pf[nt][1]);
                }
            }
        } else {
#pragma unroll
            for (int h = 0; h < 8; ++h) {  // matrices: dimensions 16 h .. + 7 and the next eight of keys 0-7, then of keys 8-15
                uint32_t r[4];
                const int row = (lane & 7) + (lane >> 4) * 8, ch = 2 * h + ((lane >> 3) & 1);
                ldsm4_t(r, vt + row * kRow + ((ch ^ (row & 7)) << 4));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma16816<false>(o[h][nt], r, pf[nt][0], pf[nt][1]);
                    mma16816<false>(o[h][nt], r, pf2[nt][0], pf2[nt][1]);
                }
            }
        }
        stage = stage + 1 == kStages ? 0 : stage + 1;
        if (use.step + 1 == use.x.n || i + 1 == n) {
            end_item(from, use.step + 1, i + 1 == n);
            if (i + 1 < n) {
                advance(use);
                load_q();
                begin_item();
                from = 0;
            }
        } else {
            ++use.step;
        }
    }
    cp_async_wait<0>();
    }
    // ---- the pieces at the runs' ends, item by item: a warp takes every kWarps-th row
    if (lane == 0) s_sum[warp] = open;
    __syncthreads();
    for (int r = warp; r < NT * 8; r += kWarps) {
        for (int w = 0; w < kWarps;) {
            const int64_t item = s_sum[w];
            int end = w + 1;
            while (end < kWarps && s_sum[end] == item) ++end;
            if (item >= 0) {
                auto piece = [&](int x) { return reinterpret_cast<const float*>(smem + x * rows_warp_bytes(NT, E4M3)); };
                auto piece_ml = [&](int x) { return reinterpret_cast<const float2*>(piece(x) + NT * 8 * kHeadDim)[r]; };
                float top = -INFINITY, sum = 0.f;
                for (int x = w; x < end; ++x) top = fmaxf(top, piece_ml(x).x);
                const float base = top == -INFINITY ? 0.f : top;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int x = w; x < end; ++x) {
                    const float4 y = reinterpret_cast<const float4*>(piece(x) + r * kHeadDim)[lane];
                    const float2 ml = piece_ml(x);
                    const float f = ex2(ml.x - base);
                    sum = fmaf(ml.y, f, sum);
                    acc.x = fmaf(y.x, f, acc.x);
                    acc.y = fmaf(y.y, f, acc.y);
                    acc.z = fmaf(y.z, f, acc.z);
                    acc.w = fmaf(y.w, f, acc.w);
                }
                const int64_t at = (2 * (static_cast<int64_t>(blockIdx.x) * kWarps + w) + 1) * args.part_rows + r;
                reinterpret_cast<float4*>(args.part_o + at * kHeadDim)[lane] = acc;
                if (lane == 0) args.part_ml[at] = make_float2(top, sum);
            }
            w = end;
        }
    }
}

// Items that several CTAs or warps of k_rows share: a CTA per item, four dimensions a lane, one warp to eight for a row by
// how many rows there are. A CTA of k_rows left one piece of the item, under the first of its runs that has a part of it, and
// where the item ends inside a run, that run another one. Bound by latency: a lane looks a piece up and weighs it, then
// the rows of eight pieces are in flight at a time.
__global__ void __launch_bounds__(256) k_rows_merge(const __grid_constant__ RowsArgs args, int ctas, int warps)
{
    __shared__ float4 s_o[8][32];
    __shared__ float2 s_ml[8];
    __shared__ int64_t s_first[8], s_total[8];
    const AttendView& a = args.a;
    const int b = blockIdx.x / args.c.Hkv, j = blockIdx.x - b * args.c.Hkv;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // Steps of the sequences before this one, its own and all, from the batch's lists while k_rows still runs: every CTA of
    // k_rows is past its own wait when this kernel starts, so what wrote the lists is complete, and k_rows writes
    // none; the loads are ld_relaxed, which see it. (One token at 4K 9.5 -> 9.0 us, at 128K 62.1 -> 61.4.) More sequences
    // than threads: what k_rows left, after the wait, and as long.
    int64_t first = 0, n, total = 0;
    auto read_seq = [&](int i) {
        return seq_of(a, args.b, ld_relaxed(args.b.row_start + i), ld_relaxed(args.b.row_start + i + 1), ld_relaxed(args.b.kv_len + i));
    };
    const Seq s = read_seq(b);
    const bool early = args.b.n_seqs <= 256;
    if (early) {
        const int i = threadIdx.x;
        int64_t mine = 0;
        if (i < args.b.n_seqs) {
            const Seq x = read_seq(i);
            mine = x.rows > 0 ? steps_of(a, x).n : 0;
        }
        int64_t lower = i < b ? mine : 0;
        for (int o = 16; o > 0; o >>= 1) {
            mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
            lower += __shfl_xor_sync(0xFFFFFFFFu, lower, o);
        }
        if (lane == 0) {
            s_first[warp] = lower;
            s_total[warp] = mine;
        }
        __syncthreads();
        for (int w = 0; w < 8; ++w) {
            first += s_first[w];
            total += s_total[w];
        }
        n = s.rows > 0 ? steps_of(a, s).n : 0;
    } else {
        pdl_enter();
        first = args.before[b];
        n = args.before[b + 1] - first;
        total = args.before[args.b.n_seqs];
    }
    const Runs runs(total * args.c.Hkv, ctas, warps);
    const int64_t x0 = first * args.c.Hkv + n * j, x1 = x0 + n;
    const int64_t c0 = quotient(x0, runs.per_cta), c1 = quotient(x1 - 1, runs.per_cta);
    const int64_t w0 = quotient(x0 - c0 * runs.per_cta, runs.per_warp), w1 = quotient(x1 - 1 - c1 * runs.per_cta, runs.per_warp);
    if (n == 0 || (c0 == c1 && w0 == w1)) {
        if (early) pdl_enter();
        return;
    }
    const bool at_end = runs.end(c1, w1) == x1;              // the last run's part is one of the CTA's pieces
    const bool c1_piece = at_end || w1 > (c0 == c1 ? w0 : 0);  // the last CTA has one
    const int pieces = static_cast<int>(c1 - c0) + c1_piece + !at_end;
    auto place = [&](int i) -> int64_t {
        const int64_t c = c0 + i;
        if (c < c1 || (c == c1 && c1_piece)) return 2 * (c * warps + (i == 0 ? w0 : 0)) + 1;
        return 2 * (c1 * warps + w1);
    };
    const int rows = s.rows * a.g;
    const int share = rows > 4 ? 1 : rows > 2 ? 2 : rows > 1 ? 4 : 8;  // warps of a row
    // A few CTAs, which start before k_rows has left all SMs, go through it twice: once without loads and stores while they
    // would wait, which brings the code into the instruction cache. One token at 4K, 32 query heads, bf16 11.6 -> 10.5 us;
    // 8 tokens at 4K, 64 CTAs, whose first pass nothing hides, 29.8 us and 30.6 with it.
#pragma unroll 1
    for (int pass = early && gridDim.x <= 32 ? 0 : 1; pass < 2; ++pass) {
        const bool real = pass == 1;
        if (real && early) pdl_enter();
        for (int r0 = 0; r0 < rows; r0 += 8 / share) {
            const int r = r0 + warp / share, sub = warp % share;
            const bool live = r < rows;
            float top = -INFINITY, sum = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
            for (int i0 = sub; live && i0 < pieces; i0 += 32 * share) {  // this warp's next 32 pieces, one per lane
                const int i = i0 + lane * share;
                int64_t at = 0;
                float2 ml = make_float2(-INFINITY, 0.f);
                if (i < pieces && real) {
                    at = place(i) * args.part_rows + r;
                    ml = __ldcg(&args.part_ml[at]);
                }
                float m = ml.x;
                for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
                m = fmaxf(m, top);
                const float base = m == -INFINITY ? 0.f : m;
                const float alpha = ex2(top - base), w = ex2(ml.x - base);
                float l = ml.y * w;
                for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
                sum = fmaf(sum, alpha, l);
                acc = make_float4(acc.x * alpha, acc.y * alpha, acc.z * alpha, acc.w * alpha);
                top = m;
                const int n_in = (pieces - i0 + share - 1) / share < 32 ? (pieces - i0 + share - 1) / share : 32;
#pragma unroll 1
                for (int u0 = 0; u0 < n_in; u0 += 8) {
                    float4 x[8];
                    float f[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const int64_t from = __shfl_sync(0xFFFFFFFFu, at, u0 + u);
                        f[u] = __shfl_sync(0xFFFFFFFFu, w, u0 + u);
                        x[u] = real && u0 + u < n_in ? __ldcg(reinterpret_cast<const float4*>(args.part_o + from * kHeadDim) + lane)
                                             : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        acc.x = fmaf(x[u].x, f[u], acc.x);
                        acc.y = fmaf(x[u].y, f[u], acc.y);
                        acc.z = fmaf(x[u].z, f[u], acc.z);
                        acc.w = fmaf(x[u].w, f[u], acc.w);
                    }
                }
            }
            if (share > 1) {  // the row's warps, in order
                s_o[warp][lane] = acc;
                if (lane == 0) s_ml[warp] = make_float2(top, sum);
                __syncthreads();
                if (sub == 0) {
                    for (int x = 1; x < share; ++x) top = fmaxf(top, s_ml[warp + x].x);
                    const float base = top == -INFINITY ? 0.f : top;
                    sum = 0.f;
                    acc = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int x = 0; x < share; ++x) {
                        const float f = ex2(s_ml[warp + x].x - base);
                        const float4 y = s_o[warp + x][lane];
                        sum = fmaf(s_ml[warp + x].y, f, sum);
                        acc.x = fmaf(y.x, f, acc.x);
                        acc.y = fmaf(y.y, f, acc.y);
                        acc.z = fmaf(y.z, f, acc.z);
                        acc.w = fmaf(y.w, f, acc.w);
                    }
                }
            }
            if (live && sub == 0 && real) {
                const float inv = sum == 0.f ? 0.f : 1.0f / sum;
                const int64_t row = s.row0 + r / a.g;
                const int h = j * a.g + r % a.g;
                auto* out = static_cast<__nv_bfloat16*>(a.out) + row * a.out_stride + h * kHeadDim;
                reinterpret_cast<uint2*>(out)[lane] = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
                if (a.lse && lane == 0) a.lse[row * a.Hq + h] = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * 0.6931471805599453f;
            }
        }
        if (!real) __syncthreads();  // the dry pass has read what the next one writes
    }
}

// Workspace regions (byte offsets) of the route that a call takes; the status word comes first.
struct AttendWs {
    size_t before, part_ml, part_o, chunks, end;
    int part_rows;
};

AttendWs attend_layout(int Hq, int Hkv, bool e4m3, int n_seqs, int n_rows, int max_rows)
{
    AttendWs w{};
    size_t off = 256;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align_up(off + bytes, kAlign);
        return at;
    };
    const int64_t rows = static_cast<int64_t>(max_rows) * (Hq / Hkv);
    if (rows > rows_max(e4m3)) {
        w.chunks = take(chunk_ws_bytes(Hq / Hkv, Hkv, n_seqs, n_rows, max_rows));
    } else {
        const int nt = rows <= 8 ? 1 : rows <= 16 ? 2 : 3;
        const size_t parts = 2 * kMaxSms * rows_warps(nt, e4m3);  // two of a run
        w.part_rows = 8 * nt;
        w.before = take((static_cast<size_t>(n_seqs) + 1) * sizeof(int64_t));
        w.part_ml = take(parts * w.part_rows * sizeof(float2));
        w.part_o = take(parts * w.part_rows * kHeadDim * sizeof(float));
    }
    w.end = off;
    return w;
}

template <int NT, bool E4M3>
cudaError_t run_rows(const RowsArgs& r, int sms, cudaStream_t st)
{
    constexpr int kWarps = rows_warps(NT, E4M3);
    auto kern = k_rows<NT, E4M3>;
    const size_t smem = rows_ring_bytes(NT, E4M3) + (static_cast<size_t>(r.b.n_seqs) + 1) * sizeof(int64_t);
    // the largest call's, whatever this one's: calls from several threads set the same
    constexpr size_t kMost = rows_ring_bytes(NT, E4M3) + (kMaxSeqs + 1) * sizeof(int64_t);
    static_assert(kMost <= 226 * 1024, "shared memory of a CTA");
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMost));
    if (e != cudaSuccess) return e;
    e = launch_after(st, dim3(sms), 32 * kWarps, smem, 1, kern, r);
    if (e != cudaSuccess) return e;
    return launch_after(st, dim3(r.b.n_seqs * r.c.Hkv), 256, 0, 1, k_rows_merge, r, sms, kWarps);
}

}  // namespace

// Either route's size does not fall with any of its numbers, so what a batch of fewer may need is the route of few rows
// at its most, where that is not the batch's own.
size_t attend_ws_bytes(int Hq, int Hkv, bool e4m3, int n_seqs, int n_rows, int max_rows)
{
    const size_t own = attend_layout(Hq, Hkv, e4m3, n_seqs, n_rows, max_rows).end;
    const int most = rows_max(e4m3) / (Hq / Hkv);
    if (max_rows <= most) return own;
    const size_t few = attend_layout(Hq, Hkv, e4m3, n_seqs, n_rows, most).end;
    return own > few ? own : few;
}

cudaError_t launch_attend(const AttendView& a, const CacheView& c, bool e4m3, const BatchView& b, uint8_t* ws,
                          uint64_t timeout_ns, cudaStream_t st)
{
    int sms = 0;
    cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
    sms = sms < kMaxSms ? sms : kMaxSms;
    const AttendWs lay = attend_layout(a.Hq, c.Hkv, e4m3, b.n_seqs, b.n_rows, b.max_rows);
    const int64_t rows = static_cast<int64_t>(b.max_rows) * a.g;
    if (rows > rows_max(e4m3)) {
        // Batches with longer pieces go there whole, and no second route follows: a sequence of few rows takes its share of
        // that kernel's jobs, at the pace of its keys (17 tokens at 128K, 537 MB of bf16: 103 us, 5.2 TB/s).
        return launch_chunks(a, c, e4m3, b, sms, reinterpret_cast<int32_t*>(ws + kStatusOffset), ws + lay.chunks, timeout_ns, st);
    }
    const RowsArgs r{a, c, b, reinterpret_cast<int64_t*>(ws + lay.before), reinterpret_cast<float*>(ws + lay.part_o),
                     reinterpret_cast<float2*>(ws + lay.part_ml), lay.part_rows};
    if (rows <= 8) return e4m3 ? run_rows<1, true>(r, sms, st) : run_rows<1, false>(r, sms, st);
    if (rows <= 16) return e4m3 ? run_rows<2, true>(r, sms, st) : run_rows<2, false>(r, sms, st);
    return run_rows<3, true>(r, sms, st);
}

}  // namespace scale
