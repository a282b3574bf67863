// branch_api.cu -- the extern "C" boundary of the calls for drafted trees and beams: argument checks, then
// the launches on the caller's stream. (scale_cache_attend_tree stands with scale_cache_attend.)
#include "branch.cuh"
#include "call_checks.h"

namespace scale {
namespace {

// Whether [x, x + xn) and [y, y + yn) share bytes.
bool share(const void* x, size_t xn, const void* y, size_t yn)
{
    const auto x0 = reinterpret_cast<uintptr_t>(x), y0 = reinterpret_cast<uintptr_t>(y);
    return x0 < y0 + yn && y0 < x0 + xn;
}

int check_moves(const scale_moves_t* m)
{
    if (!m || m->n_groups <= 0 || m->n_moves < 0) return SCALE_ERR_INVALID_ARG;
    return m->n_groups > kMaxSeqs || m->n_moves > kMaxMoves ? SCALE_ERR_UNSUPPORTED : SCALE_OK;
}

int check_beam(const scale_beam_t* b)
{
    if (!b || b->n_groups <= 0 || b->n_beams <= 0 || b->vocab <= 0 || b->n_best <= 0 ||
        (b->dtype != SCALE_LOGITS_BF16 && b->dtype != SCALE_LOGITS_FP32))
        return SCALE_ERR_INVALID_ARG;
    if (b->n_best > static_cast<int64_t>(b->n_beams) * b->vocab) return SCALE_ERR_INVALID_ARG;
    if (b->n_beams > kMaxBeams || b->n_best > kMaxBest || b->vocab > kMaxVocab ||
        static_cast<int64_t>(b->n_groups) * b->n_beams > (b->n_beams == 1 ? kMaxSingles : kMaxSeqs))
        return SCALE_ERR_UNSUPPORTED;
    return SCALE_OK;
}

}  // namespace
}  // namespace scale

using namespace scale;

extern "C" {

int scale_tree_plan(const scale_tree_t* tree, const scale_batch_t* batch, int32_t n_sink, int32_t n_local,
                    scale_stream_t stream)
{
    BatchView b;
    int rc = check_batch(batch, &b);
    if (rc) return rc;
    if ((rc = check_tree(tree, b))) return rc;
    if (n_sink < 0) return SCALE_ERR_INVALID_ARG;
    if (b.n_rows == 0 || b.max_rows == 0) return SCALE_OK;
    Pointers p;
    p.need(b.row_start, 4);
    p.need(b.kv_len, 4);
    p.need(tree->parents, 4);
    p.need(tree->positions, 4);
    p.need(tree->masks, 4);
    if (!p.ok) return SCALE_ERR_INVALID_ARG;
    return status_of(launch_tree_plan(TreeArgs{tree->parents, tree->positions, tree->masks, tree->mask_words, b, n_sink, n_local}, stream));
}

int scale_tree_accept(const scale_tree_t* tree, const scale_cache_t* cache, const scale_batch_t* batch,
                      const int32_t* tokens, const int32_t* choices, const int32_t* first, int32_t* n_accepted,
                      int32_t* path, int32_t* next, int32_t* new_len, const scale_moves_t* moves, scale_stream_t stream)
{
    CacheView c;
    BatchView b;
    bool e4m3;
    int rc = check_cache(cache, &c, &e4m3);
    if (rc) return rc;
    if ((rc = check_batch(batch, &b))) return rc;
    if (!tree) return SCALE_ERR_INVALID_ARG;
    if (b.max_rows > kMaxNodes) return SCALE_ERR_UNSUPPORTED;
    if ((rc = check_moves(moves))) return rc;
    if (moves->n_groups != b.n_seqs || moves->n_moves != b.n_rows || moves->start != b.row_start) return SCALE_ERR_INVALID_ARG;
    Pointers p;
    need_batch(&p, b);
    p.need(n_accepted, 4);
    p.need(next, 4);
    p.need(new_len, 4);
    if (first) p.need(first, 4);
    if (b.n_rows > 0) {  // a batch without rows still says what comes next
        p.need(tree->parents, 4);
        p.need(tokens, 4);
        p.need(choices, 4);
        p.need(path, 4);
        p.need(moves->src, 4);
        p.need(moves->dst, 4);
    }
    if (!p.ok) return SCALE_ERR_INVALID_ARG;
    return status_of(launch_tree_accept(AcceptArgs{tree->parents, c, b, tokens, choices, first, n_accepted, path, next, new_len,
                                                   moves->src, moves->dst},
                                        stream));
}

int scale_cache_move(const scale_cache_t* caches, int32_t n_caches, const scale_moves_t* moves, scale_stream_t stream)
{
    if (!caches || n_caches <= 0) return SCALE_ERR_INVALID_ARG;
    if (n_caches > kMaxCaches) return SCALE_ERR_UNSUPPORTED;
    CacheView views[kMaxCaches];
    bool e4m3 = false;
    for (int i = 0; i < n_caches; ++i) {
        const int rc = check_cache(caches + i, &views[i], &e4m3);
        if (rc) return rc;
        if (caches[i].dtype != caches[0].dtype || views[i].Hkv != views[0].Hkv || views[i].page_size != views[0].page_size ||
            views[i].num_pages != views[0].num_pages)
            return SCALE_ERR_INVALID_ARG;
    }
    const int rc = check_moves(moves);
    if (rc) return rc;
    if (!moves->start && moves->n_moves % moves->n_groups) return SCALE_ERR_INVALID_ARG;
    if (moves->n_moves == 0) return SCALE_OK;
    Pointers p;
    // by kind: layers often lie in one allocation for each
    for (int i = 0; i < n_caches; ++i) p.need(views[i].k, 16);
    for (int i = 0; i < n_caches; ++i) p.need(views[i].v, 16);
    for (int i = 0; e4m3 && i < n_caches; ++i) p.need(views[i].ks, 16);
    for (int i = 0; e4m3 && i < n_caches; ++i) p.need(views[i].vs, 16);
    p.need(moves->src, 4);
    p.need(moves->dst, 4);
    if (moves->start) p.need(moves->start, 4);
    if (!p.ok) return SCALE_ERR_INVALID_ARG;
    return status_of(launch_moves(views, n_caches, e4m3, MovesView{moves->src, moves->dst, moves->start, moves->n_groups, moves->n_moves}, stream));
}

int scale_beam_workspace_size(const scale_beam_t* beam, size_t* bytes)
{
    const int rc = check_beam(beam);
    if (rc) return rc;
    if (!bytes) return SCALE_ERR_INVALID_ARG;
    *bytes = beam_ws_bytes(beam->n_groups, beam->n_beams, beam->vocab, beam->n_best);
    return SCALE_OK;
}

int scale_beam_select(const scale_beam_t* beam, const void* logits, int64_t logits_stride, const float* scores,
                      float* best_scores, int32_t* best_beams, int32_t* best_tokens, void* ws, size_t ws_bytes,
                      scale_stream_t stream)
{
    const int rc = check_beam(beam);
    if (rc) return rc;
    if (logits_stride < beam->vocab || logits_stride >= (1ll << 40)) return SCALE_ERR_INVALID_ARG;
    const bool fp32 = beam->dtype == SCALE_LOGITS_FP32;
    Pointers p;
    p.need(logits, fp32 ? 4 : 2);
    p.need(scores, 4);
    p.need(best_scores, 4);
    p.need(best_beams, 4);
    p.need(best_tokens, 4);
    p.need(ws, 256);
    if (!p.ok) return SCALE_ERR_INVALID_ARG;
    if (ws_bytes < beam_ws_bytes(beam->n_groups, beam->n_beams, beam->vocab, beam->n_best)) return SCALE_ERR_WORKSPACE;
    return status_of(launch_beam_select(BeamArgs{beam->n_groups, beam->n_beams, beam->vocab, beam->n_best, logits, logits_stride, scores,
                                                 best_scores, best_beams, best_tokens},
                                        fp32, static_cast<uint8_t*>(ws), stream));
}

int scale_beam_reorder(const scale_cache_t* cache, int32_t n_groups, int32_t n_beams, const int32_t* parents,
                       const int32_t* kv_len, const int32_t* page_table, int32_t table_stride, int32_t* table_out,
                       const scale_moves_t* moves, scale_stream_t stream)
{
    CacheView c;
    bool e4m3;
    int rc = check_cache(cache, &c, &e4m3);
    if (rc) return rc;
    if (n_groups <= 0 || n_beams <= 0 || table_stride <= 0) return SCALE_ERR_INVALID_ARG;
    if (n_beams > kMaxBeams || static_cast<int64_t>(n_groups) * n_beams > kMaxSeqs) return SCALE_ERR_UNSUPPORTED;
    if ((rc = check_moves(moves))) return rc;
    const int64_t beams = static_cast<int64_t>(n_groups) * n_beams;
    if (moves->n_groups != beams || moves->n_moves != beams * c.page_size || moves->start) return SCALE_ERR_INVALID_ARG;
    const size_t bytes = static_cast<size_t>(beams) * table_stride * sizeof(int32_t);
    if (table_out != page_table && share(table_out, bytes, page_table, bytes)) return SCALE_ERR_INVALID_ARG;
    Pointers p;
    p.need(parents, 4);
    p.need(kv_len, 4);
    p.need(page_table, 4);
    p.need(table_out, 4);
    p.need(moves->src, 4);
    p.need(moves->dst, 4);
    if (!p.ok) return SCALE_ERR_INVALID_ARG;
    return status_of(launch_reorder(ReorderArgs{c, n_groups, n_beams, parents, kv_len, page_table, table_stride, table_out, moves->src, moves->dst},
                                    stream));
}

}  // extern "C"
