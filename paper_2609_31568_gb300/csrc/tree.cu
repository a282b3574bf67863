// tree.cu -- drafted trees around the model: positions and masks from the nodes' parents (scale_tree_plan), the walk
// down the trees (scale_tree_accept), and rows that move within a cache (scale_cache_move).
#include "branch.cuh"
#include "launch.cuh"
#include "ptx_sm103.cuh"
#include "scale_internal.h"

namespace scale {
namespace {

using namespace scale_ptx;

// Rows of sequence i: n of them from row0 on, the first `nodes` of which are looked at; the token of its node 0.
struct Nodes {
    int row0, n, nodes, base;
};

__device__ __forceinline__ Nodes nodes_of(const BatchView& b, int i)
{
    const int row0 = b.row_start[i], end = b.row_start[i + 1], len = b.kv_len[i];
    Nodes s;
    s.row0 = row0;
    s.n = row0 < 0 || end <= row0 ? 0 : end - row0;
    s.nodes = s.n < b.max_rows ? s.n : b.max_rows;
    if (s.nodes > b.n_rows - row0) s.nodes = b.n_rows - row0 > 0 ? b.n_rows - row0 : 0;
    s.base = (len > 0 ? len : 0) - s.n;
    return s;
}

// Positions and masks, a CTA per sequence, a thread per node. A node's ancestors are doubled: after round k its mask holds
// its next 2^k ancestors, and `up` the one after those (or how the way ends: -1 at a root, -2 at what is no node),
// so a tree of depth d takes log2(d) rounds whatever its shape; then the mask's bits are the depth.
// Bound by latency: the lists, the parents, two barriers for each round and eight words. 3.2 us for 48 trees of 61 nodes, 2.8 for
// one of 16, call after call.
__global__ void __launch_bounds__(kMaxNodes) k_tree_plan(const __grid_constant__ TreeArgs a)
{
    extern __shared__ uint32_t s_mask[];  // [words][threads]
    __shared__ int s_up[2][kMaxNodes];
    pdl_enter();
    const Nodes s = nodes_of(a.b, blockIdx.x);
    const int i = threadIdx.x, n = s.nodes, pitch = blockDim.x;
    if (n == 0) return;
    const int words = (n + 31) / 32;
    int up = -2;
    if (i < n && s.base >= 0) {
        up = a.parents[s.row0 + i];
        if (up < -1 || up >= i) up = -2;
    }
    for (int w = 0; w < words; ++w) s_mask[w * pitch + i] = w == i >> 5 ? 1u << (i & 31) : 0u;
    s_up[0][i] = up;
    int round = 0;
    while (__syncthreads_or(up >= 0)) {
        for (int w0 = 0; w0 < words; w0 += 8) {
            uint32_t x[8];
#pragma unroll
            for (int w = 0; w < 8; ++w) x[w] = up >= 0 && w0 + w < words ? s_mask[(w0 + w) * pitch + up] : 0u;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < 8; ++w)
                if (up >= 0 && w0 + w < words) s_mask[(w0 + w) * pitch + i] |= x[w];
        }
        if (up >= 0) up = s_up[round & 1][up];
        ++round;
        s_up[round & 1][i] = up;
    }
    const bool node = up == -1;
    int depth = -1;
    for (int w = 0; w < words; ++w) depth += __popc(s_mask[w * pitch + i]);
    // The window: ancestor j from the root lies depth - j above the node, at position base + j. (Ancestors are earlier nodes,
    // so they come in the order of their bits.)
    const int far = a.n_local >= 0 && depth > a.n_local ? depth - a.n_local : 0;
    const int kept = a.n_sink > s.base ? a.n_sink - s.base : 0;
    int j = 0;
    for (int w = 0; w < words; ++w) {
        uint32_t m = node ? s_mask[w * pitch + i] : 0u;
        if (far > kept) {
            for (uint32_t rest = m; rest && j < far; rest &= rest - 1, ++j)
                if (j >= kept) m &= ~(rest & (0u - rest));
        }
        s_mask[w * pitch + i] = m;
    }
    if (i < n) a.positions[s.row0 + i] = node ? s.base + depth : -1;
    __syncthreads();
    for (int x = i; x < n * a.words; x += pitch) {
        const int row = x / a.words, w = x - row * a.words;
        a.masks[static_cast<int64_t>(s.row0) * a.words + x] = w < words ? s_mask[w * pitch + row] : 0u;
    }
}

// The walk down a sequence's tree: every node that holds what its parent wants is its parent's child if none lower is, then one
// thread follows the children. Bound by latency: the lists, then tokens and choices, then the path's shared memory. 3.1 us for 48
// trees of 61 nodes, 3.0 for one of 16.
constexpr int kAcceptThreads = 128;

__global__ void __launch_bounds__(kAcceptThreads) k_tree_accept(const __grid_constant__ AcceptArgs a)
{
    __shared__ int s_child[kMaxNodes + 1];  // of the root's root, then of every node
    __shared__ int s_path[kMaxNodes];
    __shared__ int s_count;
    pdl_enter();
    const int b = blockIdx.x, tid = threadIdx.x;
    const Nodes s = nodes_of(a.b, b);
    const int nodes = s.base >= 0 ? s.nodes : 0;
    for (int i = tid; i <= nodes; i += kAcceptThreads) s_child[i] = kMaxNodes;
    const int first = a.first ? a.first[b] : -1;
    __syncthreads();
    for (int i = tid; i < nodes; i += kAcceptThreads) {
        const int p = a.parents[s.row0 + i];
        if (p < -1 || p >= i) continue;
        if (p == -1 ? !a.first || a.tokens[s.row0 + i] == first : a.tokens[s.row0 + i] == a.choices[s.row0 + p])
            atomicMin(&s_child[p + 1], i);
    }
    __syncthreads();
    if (tid == 0) {
        int n = 0;
        for (int at = s_child[0]; at < kMaxNodes; at = s_child[at + 1]) s_path[n++] = at;  // children are later nodes: it ends
        s_count = n;
        a.n_accepted[b] = n;
        a.next[b] = n > 0 ? a.choices[s.row0 + s_path[n - 1]] : first;
        a.new_len[b] = s.n > 0 && s.base >= 0 ? s.base + n : a.b.kv_len[b];
    }
    __syncthreads();
    const int n = s_count;
    for (int i = tid; i < s.nodes; i += kAcceptThreads) {
        int at = -1, src = -1, dst = -1;
        if (i < n) {
            at = s_path[i];
            if (at != i) {
                src = cache_row(a.c, a.b, b, s.base + at);
                dst = cache_row(a.c, a.b, b, s.base + i);
                if (src < 0 || dst < 0) src = dst = -1;
            }
        }
        a.path[s.row0 + i] = at;
        a.src[s.row0 + i] = src;
        a.dst[s.row0 + i] = dst;
    }
    // The moves of the rows that are not looked at belong to the group all the same: whatever their lists held, they are none.
    const int listed = s.n < a.b.n_rows - s.row0 ? s.n : a.b.n_rows - s.row0;
    for (int i = s.nodes + tid; i < listed; i += kAcceptThreads) a.dst[s.row0 + i] = -1;
}

// Moves. A warp has 512 bytes (or the whole row, where that is less) of every row of a group's keys or values in one cache, or
// the scales of either, so that no two warps touch the same bytes and a group's order is a warp's own (groups of equal
// size, whose moves have none, are shared by warps 32 moves at a time). Moves that are none are left out 32 at a time; of the others
// the rows of kAtOnce copies are read before any is written.
//
// Bound by HBM where there is much: 1,435 moves in 128 groups of 64, 8-bit rows of 8 heads in 32 layers (190 MB read and written) 32.5 us,
// 5.8 TB/s; 85 of 2,928 in 48 groups, where a warp walks its group's list for the few that are real, 7.0 us. Three CTAs an SM
// leave registers for kAtOnce rows: with five and six, 50 and 54 us in place of 37 (the reordering with it). By warps that
// walk a whole group of equal size the first takes 35.6 us, and 40 moves in 4 groups 5.0 us in place of 4.5.
constexpr int kMoveWarps = 8;
constexpr int kAtOnce = 8;

struct MoveLayer {
    uint8_t *k, *v, *ks, *vs;
};
struct MoveArgs {
    MovesView m;
    int pool_rows, page_size, Hkv;
    int row_bytes;  // of all heads
    int parts;      // pieces of 512 bytes of a row
    int units;      // parts (and one for scales) of keys and of values
    int blocks;     // of 32 moves of a group whose moves may come in any order; 1 where they may not
    MoveLayer layers[kMoveCaches];
};

__global__ void __launch_bounds__(32 * kMoveWarps, 3) k_move(const __grid_constant__ MoveArgs a)
{
    __shared__ int2 s_moves[kMoveWarps][32];
    pdl_enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int unit = blockIdx.x * kMoveWarps + warp;
    const int block = unit / a.units, group = block / a.blocks;
    if (group >= a.m.n_groups) return;
    const int part = (unit - block * a.units) >> 1;
    const bool values = unit & 1;
    const MoveLayer& layer = a.layers[blockIdx.y];
    int begin, end;
    if (a.m.start) {
        begin = a.m.start[group];
        end = a.m.start[group + 1];
        begin = begin > 0 ? begin : 0;
        end = end < a.m.n_moves ? end : a.m.n_moves;
    } else {
        const int each = a.m.n_moves / a.m.n_groups, first = (block - group * a.blocks) * 32;
        begin = group * each + first;
        end = begin + (each - first < 32 ? each - first : 32);
    }
    int2* const list = s_moves[warp];
    const int left = a.row_bytes - part * 512;
    const int per_row = (left < 512 ? left : 512) / 16;            // lanes of a row's piece
    const int at_once = part < a.parts ? 32 / per_row : 1;         // rows that the lanes cover
    const int sub = part < a.parts ? lane / per_row : 0, chunk = lane - sub * per_row;
    uint8_t* const pages = (values ? layer.v : layer.k) + part * 512 + chunk * 16;
    for (int i0 = begin; i0 < end; i0 += 32) {
        int2 mv = make_int2(-1, -1);
        if (i0 + lane < end) mv = make_int2(a.m.src[i0 + lane], a.m.dst[i0 + lane]);
        const bool real = static_cast<uint32_t>(mv.x) < static_cast<uint32_t>(a.pool_rows) &&
                          static_cast<uint32_t>(mv.y) < static_cast<uint32_t>(a.pool_rows) && mv.x != mv.y;
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, real);
        const int n = __popc(who);
        if (n == 0) continue;
        __syncwarp();  // the list before is read
        if (real) list[__popc(who & ((1u << lane) - 1u))] = mv;
        __syncwarp();
        if (part < a.parts) {
            for (int j0 = 0; j0 < n; j0 += kAtOnce * at_once) {
                uint4 x[kAtOnce];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int j = j0 + u * at_once + sub;
                    if (sub < at_once && j < n) x[u] = *reinterpret_cast<const uint4*>(pages + static_cast<int64_t>(list[j].x) * a.row_bytes);
                }
                __syncwarp();
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int j = j0 + u * at_once + sub;
                    if (sub < at_once && j < n) *reinterpret_cast<uint4*>(pages + static_cast<int64_t>(list[j].y) * a.row_bytes) = x[u];
                }
                __syncwarp();
            }
        } else {  // scales [page][head][place]: a lane per move
            uint8_t* const scales = values ? layer.vs : layer.ks;
            int64_t from = 0, to = 0;
            if (lane < n) {
                const int2 p = list[lane];
                const int sp = p.x / a.page_size, dp = p.y / a.page_size;
                from = static_cast<int64_t>(sp) * a.Hkv * a.page_size + (p.x - sp * a.page_size);
                to = static_cast<int64_t>(dp) * a.Hkv * a.page_size + (p.y - dp * a.page_size);
            }
            for (int h0 = 0; h0 < a.Hkv; h0 += kAtOnce) {
                uint8_t x[kAtOnce];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
                    if (lane < n && h0 + u < a.Hkv) x[u] = scales[from + (h0 + u) * a.page_size];
                __syncwarp();
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
                    if (lane < n && h0 + u < a.Hkv) scales[to + (h0 + u) * a.page_size] = x[u];
                __syncwarp();
            }
        }
    }
}

}  // namespace

cudaError_t launch_tree_plan(const TreeArgs& a, cudaStream_t st)
{
    const int threads = a.b.max_rows <= 32 ? 32 : (a.b.max_rows + 31) / 32 * 32;
    const size_t smem = static_cast<size_t>(threads / 32) * threads * sizeof(uint32_t);
    if (smem > kPlainSmem) {
        // the largest call's, whatever this one's: calls from several threads set the same
        constexpr int kMost = kMaxNodes / 32 * kMaxNodes * static_cast<int>(sizeof(uint32_t));
        const cudaError_t e = cudaFuncSetAttribute(k_tree_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (e != cudaSuccess) return e;
    }
    return launch_after(st, dim3(a.b.n_seqs), threads, smem, 1, k_tree_plan, a);
}

cudaError_t launch_tree_accept(const AcceptArgs& a, cudaStream_t st)
{
    return launch_after(st, dim3(a.b.n_seqs), kAcceptThreads, 0, 1, k_tree_accept, a);
}

cudaError_t launch_moves(const CacheView* caches, int n, bool e4m3, const MovesView& m, cudaStream_t st)
{
    MoveArgs a{};
    a.m = m;
    a.page_size = caches[0].page_size;
    a.Hkv = caches[0].Hkv;
    a.pool_rows = caches[0].num_pages * a.page_size;
    a.row_bytes = a.Hkv * kHeadDim * (e4m3 ? 1 : 2);
    a.parts = (a.row_bytes + 511) / 512;
    a.units = 2 * (a.parts + (e4m3 ? 1 : 0));
    a.blocks = m.start ? 1 : (m.n_moves / m.n_groups + 31) / 32;
    const int64_t warps = static_cast<int64_t>(m.n_groups) * a.blocks * a.units;
    for (int i0 = 0; i0 < n; i0 += kMoveCaches) {
        const int layers = n - i0 < kMoveCaches ? n - i0 : kMoveCaches;
        for (int i = 0; i < layers; ++i) a.layers[i] = MoveLayer{caches[i0 + i].k, caches[i0 + i].v, caches[i0 + i].ks, caches[i0 + i].vs};
        const dim3 grid(static_cast<unsigned>((warps + kMoveWarps - 1) / kMoveWarps), static_cast<unsigned>(layers));
        const cudaError_t e = launch_after(st, grid, 32 * kMoveWarps, 0, 1, k_move, a);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace scale
