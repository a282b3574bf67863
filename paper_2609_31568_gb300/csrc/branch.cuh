// branch.cuh -- several continuations of a sequence over its paged cache, as the kernels see them: drafted
// trees, rows that move, beams.
#pragma once

#include "cache.cuh"

namespace scale {

constexpr int kMaxNodes = 1024;     // rows of a sequence's tree
constexpr int kMaxBeams = 32;       // of a group: a lane each
constexpr int kMaxBest = 64;        // continuations kept of a group
constexpr int kMaxSingles = kMaxSeqs * kMaxNodes;  // groups of one beam: every node of a batch
constexpr int kMaxVocab = 1 << 24;
constexpr int kMaxCaches = 1024;    // of scale_cache_move
constexpr int kMoveCaches = 64;     // of them in a launch
constexpr int kMaxMoves = 1 << 28;  // k_move numbers its warps in 31 bits: 66 at most for 32 moves, or for a group of 33 twice as many
constexpr size_t kPlainSmem = 32 * 1024;  // dynamic shared memory that a kernel has without asking

struct TreeArgs {
    const int32_t* parents;
    int32_t* positions;
    uint32_t* masks;
    int words;
    BatchView b;
    int n_sink, n_local;
};

struct AcceptArgs {
    const int32_t* parents;
    CacheView c;
    BatchView b;
    const int32_t *tokens, *choices, *first;
    int32_t *n_accepted, *path, *next, *new_len, *src, *dst;
};

struct MovesView {
    const int32_t *src, *dst, *start;
    int n_groups, n_moves;
};

struct ReorderArgs {
    CacheView c;
    int n_groups, n_beams;
    const int32_t *parents, *kv_len, *table;
    int stride;
    int32_t *table_out, *src, *dst;
};

struct BeamArgs {
    int n_groups, n_beams, vocab, n_best;
    const void* logits;
    int64_t stride;  // elements
    const float* scores;
    float* best_scores;
    int32_t *best_beams, *best_tokens;
};

cudaError_t launch_tree_plan(const TreeArgs& a, cudaStream_t st);
cudaError_t launch_tree_accept(const AcceptArgs& a, cudaStream_t st);
// `caches`: n of the same shape
cudaError_t launch_moves(const CacheView* caches, int n, bool e4m3, const MovesView& m, cudaStream_t st);
cudaError_t launch_reorder(const ReorderArgs& a, cudaStream_t st);
size_t beam_ws_bytes(int n_groups, int n_beams, int vocab, int n_best);
cudaError_t launch_beam_select(const BeamArgs& a, bool fp32, uint8_t* ws, cudaStream_t st);

}  // namespace scale
