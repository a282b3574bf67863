// call_checks.h -- argument checks that the calls over a paged cache share.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>

#include "branch.cuh"
#include "scale_internal.h"

namespace scale {

constexpr int64_t kMaxPoolRows = (1ll << 31) - 256;

// cuPointerGetAttributes, resolved once through the runtime's driver entry point; null where there is none.
inline PFN_cuPointerGetAttributes_v7000 pointer_attributes()
{
    static const PFN_cuPointerGetAttributes_v7000 fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q{};
        const bool ok = cudaGetDriverEntryPointByVersion("cuPointerGetAttributes", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
                        q == cudaDriverEntryPointSuccess;
        if (!ok) cudaGetLastError();
        return ok ? reinterpret_cast<PFN_cuPointerGetAttributes_v7000>(p) : nullptr;
    }();
    return fn;
}

// Pointer checks of one call: device (or managed) memory of the current device, aligned. A pointer into the allocation of the one
// before it is not looked up again: the caches of 32 layers are 128 pointers, 80 ns each.
struct Pointers {
    int dev = -1;
    bool ok = true;
    uintptr_t lo = 0, hi = 0;  // the allocation that was looked up last
    Pointers() { ok = cudaGetDevice(&dev) == cudaSuccess; }
    void need(const void* p, size_t align)
    {
        if (!ok) return;
        if (!p || reinterpret_cast<uintptr_t>(p) % align) {
            ok = false;
            return;
        }
        const uintptr_t x = reinterpret_cast<uintptr_t>(p);
        if (x >= lo && x < hi) return;
        if (const auto look_up = pointer_attributes()) {
            unsigned int type = 0, managed = 0;
            int ordinal = -1;
            void* start = nullptr;
            size_t size = 0;
            CUpointer_attribute which[5] = {CU_POINTER_ATTRIBUTE_MEMORY_TYPE, CU_POINTER_ATTRIBUTE_DEVICE_ORDINAL, CU_POINTER_ATTRIBUTE_IS_MANAGED,
                                            CU_POINTER_ATTRIBUTE_RANGE_START_ADDR, CU_POINTER_ATTRIBUTE_RANGE_SIZE};
            void* to[5] = {&type, &ordinal, &managed, &start, &size};
            ok = look_up(5, which, to, static_cast<CUdeviceptr>(x)) == CUDA_SUCCESS && (managed || (type == CU_MEMORYTYPE_DEVICE && ordinal == dev));
            lo = ok ? reinterpret_cast<uintptr_t>(start) : 0;
            hi = ok ? lo + size : 0;
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

inline bool stride_ok(int64_t stride, int heads)
{
    return stride >= static_cast<int64_t>(heads) * kHeadDim && stride % 8 == 0 && stride < (1ll << 40);
}

// Whether two row tensors share bytes. Strided tensors that interleave without
// sharing any (slices of one joint row) are told apart by their place in the row.
inline bool overlap(const void* x, int64_t xs, int xh, const void* y, int64_t ys, int yh, int64_t rows)
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

inline int check_cache(const scale_cache_t* c, CacheView* v, bool* e4m3)
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

inline int check_batch(const scale_batch_t* b, BatchView* v)
{
    if (!b || b->n_seqs <= 0 || b->table_stride <= 0 || b->n_rows < 0 || b->max_rows < 0) return SCALE_ERR_INVALID_ARG;
    if (b->n_seqs > kMaxSeqs || b->n_rows >= kMaxPoolRows) return SCALE_ERR_UNSUPPORTED;
    *v = BatchView{b->row_start, b->kv_len, b->page_table, b->n_seqs, b->table_stride, b->n_rows, b->max_rows};
    return SCALE_OK;
}

inline void need_cache(Pointers* p, const CacheView& c, bool e4m3)
{
    p->need(c.k, 16);
    p->need(c.v, 16);
    if (e4m3) {
        p->need(c.ks, 16);
        p->need(c.vs, 16);
    }
}

inline void need_batch(Pointers* p, const BatchView& b)
{
    p->need(b.row_start, 4);
    p->need(b.kv_len, 4);
    p->need(b.table, 4);
}

inline int check_tree(const scale_tree_t* t, const BatchView& b)
{
    if (!t || t->mask_words < 0) return SCALE_ERR_INVALID_ARG;
    if (b.max_rows > kMaxNodes || t->mask_words > kMaxNodes / 32) return SCALE_ERR_UNSUPPORTED;
    return static_cast<int64_t>(t->mask_words) * 32 >= b.max_rows ? SCALE_OK : SCALE_ERR_INVALID_ARG;
}

inline int status_of(cudaError_t e) { return e == cudaSuccess ? SCALE_OK : SCALE_ERR_CUDA; }

}  // namespace scale
