// cache_api.cu -- the extern "C" boundary of the calls over a batch's paged
// cache: argument checks, then the launches on the caller's stream.
#include <cmath>

#include "cache.cuh"
#include "scale_internal.h"

namespace scale {
namespace {

constexpr int64_t kMaxPoolRows = (1ll << 31) - 256;

// Pointer checks of one call: device (or managed) memory of the current device, aligned.
struct Pointers {
    int dev = -1;
    bool ok = true;
    Pointers() { ok = cudaGetDevice(&dev) == cudaSuccess; }
    void need(const void* p, size_t align)
    {
        if (!ok) return;
        if (!p || reinterpret_cast<uintptr_t>(p) % align) {
            ok = false;
            return;
        }
        cudaPointerAttributes at{};
        if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
            cudaGetLastError();
            ok = false;
            return;
        }
        ok = at.type == cudaMemoryTypeManaged || (at.type == cudaMemoryTypeDevice && at.device == dev);
    }
};

bool stride_ok(int64_t stride, int heads)
{
    return stride >= static_cast<int64_t>(heads) * kHeadDim && stride % 8 == 0 && stride < (1ll << 40);
}

// Whether two row tensors share bytes. Strided tensors that interleave without
// sharing any (slices of one joint row) are told apart by their place in the row.
bool overlap(const void* x, int64_t xs, int xh, const void* y, int64_t ys, int yh, int64_t rows)
{
    const auto x0 = reinterpret_cast<uintptr_t>(x), y0 = reinterpret_cast<uintptr_t>(y);
    const uint64_t xw = static_cast<uint64_t>(xh) * kHeadDim * 2, yw = static_cast<uint64_t>(yh) * kHeadDim * 2;
    const uint64_t xe = x0 + static_cast<uint64_t>(rows - 1) * xs * 2 + xw, ye = y0 + static_cast<uint64_t>(rows - 1) * ys * 2 + yw;
    if (x0 >= ye || y0 >= xe) return false;
    if (xs != ys) return true;
    const uint64_t st = static_cast<uint64_t>(xs) * 2;
    const uint64_t d = (x0 > y0 ? x0 - y0 : y0 - x0) % st;
    // the later one starts d bytes into a row of the earlier one
    const uint64_t first = x0 > y0 ? yw : xw, second = x0 > y0 ? xw : yw;
    return d < first || d + second > st;
}

int check_cache(const scale_cache_t* c, CacheView* v, bool* e4m3)
{
    if (!c || (c->dtype != SCALE_CACHE_BF16 && c->dtype != SCALE_CACHE_E4M3)) return SCALE_ERR_INVALID_ARG;
    if (c->num_kv_heads <= 0 || c->page_size <= 0 || c->num_pages <= 0) return SCALE_ERR_INVALID_ARG;
    if (c->num_kv_heads > 64 || c->page_size % 16 || c->num_pages > kMaxPoolRows ||
        c->num_pages * c->page_size >= kMaxPoolRows)
        return SCALE_ERR_UNSUPPORTED;
    *e4m3 = c->dtype == SCALE_CACHE_E4M3;
    *v = CacheView{static_cast<uint8_t*>(c->k_pages), static_cast<uint8_t*>(c->v_pages), c->k_scales, c->v_scales,
                   c->num_kv_heads, c->page_size, static_cast<int>(c->num_pages)};
    return SCALE_OK;
}

int check_batch(const scale_batch_t* b, BatchView* v)
{
    if (!b || b->n_seqs <= 0 || b->table_stride <= 0 || b->n_rows < 0 || b->max_rows < 0) return SCALE_ERR_INVALID_ARG;
    if (b->n_seqs > kMaxSeqs || b->n_rows >= kMaxPoolRows) return SCALE_ERR_UNSUPPORTED;
    *v = BatchView{b->row_start, b->kv_len, b->page_table, b->n_seqs, b->table_stride, b->n_rows, b->max_rows};
    return SCALE_OK;
}

void need_cache(Pointers* p, const CacheView& c, bool e4m3)
{
    p->need(c.k, 16);
    p->need(c.v, 16);
    if (e4m3) {
        p->need(c.ks, 16);
        p->need(c.vs, 16);
    }
}

void need_batch(Pointers* p, const BatchView& b)
{
    p->need(b.row_start, 4);
    p->need(b.kv_len, 4);
    p->need(b.table, 4);
}

int check_rope(const scale_rope_t* r)
{
    if (!r || r->n_axes < 1 || r->n_axes > 4) return SCALE_ERR_INVALID_ARG;
    for (int i = 0; i < 64; ++i)
        if (r->axis[i] >= r->n_axes) return SCALE_ERR_INVALID_ARG;
    return SCALE_OK;
}

// Heads and strides of a row tensor that is turned from x into y; 0 heads: none. Without rows there need be no tensors.
int check_turned(int heads, int most, const void* x, int64_t xs, const void* y, int64_t ys, int64_t rows)
{
    if (heads < 0 || (rows > 0 && ((heads == 0) != (x == nullptr) || (heads == 0) != (y == nullptr)))) return SCALE_ERR_INVALID_ARG;
    if (heads == 0) return SCALE_OK;
    if (heads > most) return SCALE_ERR_UNSUPPORTED;
    if (!stride_ok(xs, heads) || !stride_ok(ys, heads)) return SCALE_ERR_INVALID_ARG;
    if (rows > 0 && !(x == y && xs == ys) && overlap(x, xs, heads, y, ys, heads, rows)) return SCALE_ERR_INVALID_ARG;
    return SCALE_OK;
}

constexpr int kMaxRopeHeads = 256;

int check_attend(const scale_attend_t* a, const CacheView& c, const BatchView& b)
{
    if (!a || a->num_q_heads <= 0 || a->num_q_heads % c.Hkv || a->n_sink < 0 || !std::isfinite(a->attn_scale) ||
        a->attn_scale < 0.f)
        return SCALE_ERR_INVALID_ARG;
    if (a->num_q_heads / c.Hkv > 32 || static_cast<int64_t>(b.n_rows) * a->num_q_heads >= (1ll << 37))
        return SCALE_ERR_UNSUPPORTED;
    return SCALE_OK;
}

int status_of(cudaError_t e) { return e == cudaSuccess ? SCALE_OK : SCALE_ERR_CUDA; }

}  // namespace
}  // namespace scale

using namespace scale;

extern "C" {

int scale_rope(const scale_rope_t* rope, int32_t n_rows, int32_t num_q_heads, const void* q, int64_t q_stride,
               void* q_out, int64_t q_out_stride, int32_t num_kv_heads, const void* k, int64_t k_stride, void* k_out,
               int64_t k_out_stride, scale_stream_t stream)
{
    int rc = check_rope(rope);
    if (rc) return rc;
    if (n_rows < 0 || num_q_heads <= 0) return SCALE_ERR_INVALID_ARG;
    if (n_rows >= kMaxPoolRows) return SCALE_ERR_UNSUPPORTED;
    if ((rc = check_turned(num_q_heads, kMaxRopeHeads, q, q_stride, q_out, q_out_stride, n_rows))) return rc;
    if ((rc = check_turned(num_kv_heads, 64, k, k_stride, k_out, k_out_stride, n_rows))) return rc;
    if (num_kv_heads && n_rows &&
        (overlap(q_out, q_out_stride, num_q_heads, k, k_stride, num_kv_heads, n_rows) ||
         overlap(q_out, q_out_stride, num_q_heads, k_out, k_out_stride, num_kv_heads, n_rows) ||
         overlap(q, q_stride, num_q_heads, k_out, k_out_stride, num_kv_heads, n_rows)))
        return SCALE_ERR_INVALID_ARG;
    if (n_rows == 0) return SCALE_OK;
    Pointers p;
    p.need(rope->inv_freq, 8);
    p.need(rope->positions, 4);
    p.need(q, 16);
    p.need(q_out, 16);
    if (num_kv_heads) {
        p.need(k, 16);
        p.need(k_out, 16);
    }
    if (!p.ok) return SCALE_ERR_INVALID_ARG;
    return status_of(launch_rope(*rope, n_rows, RowsView{q, q_stride, q_out, q_out_stride, num_q_heads},
                                 RowsView{k, k_stride, k_out, k_out_stride, num_kv_heads}, stream));
}

int scale_cache_append(const scale_cache_t* cache, const scale_batch_t* batch, const void* k, int64_t k_stride,
                       const void* v, int64_t v_stride, const scale_rope_t* rope, int32_t num_q_heads, const void* q,
                       int64_t q_stride, void* q_out, int64_t q_out_stride, scale_stream_t stream)
{
    CacheView c;
    BatchView b;
    bool e4m3;
    int rc = check_cache(cache, &c, &e4m3);
    if (rc) return rc;
    if ((rc = check_batch(batch, &b))) return rc;
    if (rope && (rc = check_rope(rope))) return rc;
    if (!rope && (q || num_q_heads)) return SCALE_ERR_INVALID_ARG;
    if (!stride_ok(k_stride, c.Hkv) || !stride_ok(v_stride, c.Hkv)) return SCALE_ERR_INVALID_ARG;
    if ((rc = check_turned(num_q_heads, kMaxRopeHeads, q, q_stride, q_out, q_out_stride, b.n_rows))) return rc;
    if (num_q_heads && b.n_rows &&
        (overlap(q_out, q_out_stride, num_q_heads, k, k_stride, c.Hkv, b.n_rows) ||
         overlap(q_out, q_out_stride, num_q_heads, v, v_stride, c.Hkv, b.n_rows)))
        return SCALE_ERR_INVALID_ARG;
    if (b.n_rows == 0) return SCALE_OK;
    Pointers p;
    need_cache(&p, c, e4m3);
    need_batch(&p, b);
    p.need(k, 16);
    p.need(v, 16);
    if (rope) {
        p.need(rope->inv_freq, 8);
        p.need(rope->positions, 4);
    }
    if (num_q_heads) {
        p.need(q, 16);
        p.need(q_out, 16);
    }
    if (!p.ok) return SCALE_ERR_INVALID_ARG;
    return status_of(launch_append(c, e4m3, b, rope, RowsView{q, q_stride, q_out, q_out_stride, num_q_heads},
                                   RowsView{k, k_stride, nullptr, 0, c.Hkv}, RowsView{v, v_stride, nullptr, 0, c.Hkv},
                                   stream));
}

int scale_cache_read(const scale_cache_t* cache, const scale_batch_t* batch, void* k_out, int64_t k_out_stride,
                     void* v_out, int64_t v_out_stride, scale_stream_t stream)
{
    CacheView c;
    BatchView b;
    bool e4m3;
    int rc = check_cache(cache, &c, &e4m3);
    if (rc) return rc;
    if ((rc = check_batch(batch, &b))) return rc;
    if (b.n_rows && !k_out && !v_out) return SCALE_ERR_INVALID_ARG;
    if ((k_out && !stride_ok(k_out_stride, c.Hkv)) || (v_out && !stride_ok(v_out_stride, c.Hkv)))
        return SCALE_ERR_INVALID_ARG;
    if (k_out && v_out && b.n_rows && overlap(k_out, k_out_stride, c.Hkv, v_out, v_out_stride, c.Hkv, b.n_rows))
        return SCALE_ERR_INVALID_ARG;
    if (b.n_rows == 0) return SCALE_OK;
    Pointers p;
    need_cache(&p, c, e4m3);
    need_batch(&p, b);
    if (k_out) p.need(k_out, 16);
    if (v_out) p.need(v_out, 16);
    if (!p.ok) return SCALE_ERR_INVALID_ARG;
    return status_of(launch_cache_read(c, e4m3, b, k_out, k_out_stride, v_out, v_out_stride, stream));
}

int scale_cache_attend_workspace_size(const scale_attend_t* attend, const scale_cache_t* cache,
                                      const scale_batch_t* batch, size_t* bytes)
{
    CacheView c;
    BatchView b;
    bool e4m3;
    int rc = check_cache(cache, &c, &e4m3);
    if (rc) return rc;
    if ((rc = check_batch(batch, &b))) return rc;
    if ((rc = check_attend(attend, c, b))) return rc;
    if (!bytes) return SCALE_ERR_INVALID_ARG;
    *bytes = attend_ws_bytes(attend->num_q_heads, c.Hkv, e4m3, b.n_seqs, b.n_rows, b.max_rows);
    return SCALE_OK;
}

int scale_cache_attend(const scale_attend_t* attend, const scale_cache_t* cache, const scale_batch_t* batch,
                       const void* q, int64_t q_stride, void* out, int64_t out_stride, float* lse, void* ws,
                       size_t ws_bytes, scale_stream_t stream)
{
    CacheView c;
    BatchView b;
    bool e4m3;
    int rc = check_cache(cache, &c, &e4m3);
    if (rc) return rc;
    if ((rc = check_batch(batch, &b))) return rc;
    if ((rc = check_attend(attend, c, b))) return rc;
    const int Hq = attend->num_q_heads;
    if (!stride_ok(q_stride, Hq) || !stride_ok(out_stride, Hq)) return SCALE_ERR_INVALID_ARG;
    if (b.n_rows && overlap(q, q_stride, Hq, out, out_stride, Hq, b.n_rows)) return SCALE_ERR_INVALID_ARG;
    if (b.n_rows == 0) return SCALE_OK;
    Pointers p;
    need_cache(&p, c, e4m3);
    need_batch(&p, b);
    p.need(q, 16);
    p.need(out, 16);
    if (lse) p.need(lse, 4);
    p.need(ws, 256);
    if (!p.ok) return SCALE_ERR_INVALID_ARG;
    if (ws_bytes < attend_ws_bytes(Hq, c.Hkv, e4m3, b.n_seqs, b.n_rows, b.max_rows)) return SCALE_ERR_WORKSPACE;
    if (b.max_rows == 0) return SCALE_OK;
    const float scale = attend->attn_scale > 0.f ? attend->attn_scale : 1.0f / std::sqrt(static_cast<float>(kHeadDim));
    const AttendView a{Hq, Hq / c.Hkv, attend->n_sink, attend->n_local, scale * 1.4426950408889634f,
                       q, q_stride, out, out_stride, lse};
    return status_of(launch_attend(a, c, e4m3, b, static_cast<uint8_t*>(ws), wait_timeout_ns(), stream));
}

}  // extern "C"
