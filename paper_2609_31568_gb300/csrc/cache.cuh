// cache.cuh -- the paged cache of a batch as the kernels see it: what a call's
// descriptors become, where a row of a batch lies, and the 8-bit row format.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/scale.h"

namespace scale {

constexpr int kMaxSeqs = 4096;
constexpr int kLowExp = -100;  // least exponent of an 8-bit row's scale: its smallest code is a normal bf16

struct CacheView {
    uint8_t *k, *v;    // pages
    uint8_t *ks, *vs;  // scales (8-bit rows)
    int Hkv, page_size;
    int num_pages;
};

struct BatchView {
    const int32_t* row_start;
    const int32_t* kv_len;
    const int32_t* table;
    int n_seqs, stride, n_rows, max_rows;
};

// Row of the pool of token t of sequence b, or -1: no such token, or a table
// entry outside the pool.
__device__ __forceinline__ int cache_row(const CacheView& c, const BatchView& bt, int b, int t)
{
    if (t < 0) return -1;
    const int lp = static_cast<int>(static_cast<uint32_t>(t) / static_cast<uint32_t>(c.page_size));
    if (lp >= bt.stride) return -1;
    const int page = bt.table[static_cast<int64_t>(b) * bt.stride + lp];
    if (page < 0 || page >= c.num_pages) return -1;
    return page * c.page_size + (t - lp * c.page_size);
}

// Row of the pool of row r of the batch: -1 when its token has no place, -2 when r belongs to no sequence. The
// last sequence that starts at or before r is found by bisection.
__device__ __forceinline__ int place_of_row(const CacheView& c, const BatchView& bt, int r)
{
    int lo = 0, hi = bt.n_seqs;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (bt.row_start[mid] <= r) lo = mid;
        else hi = mid;
    }
    const int end = bt.row_start[lo + 1], len = bt.kv_len[lo];
    if (r < bt.row_start[lo] || r >= end) return -2;
    return cache_row(c, bt, lo, len - (end - r));
}

// Two e4m3 codes (the low 16 bits of x) as f16, exact.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t x)
{
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(x));
    return r;
}

// (lo, hi) of a f16 pair as fp32.
__device__ __forceinline__ float2 f16x2_to_f32(uint32_t x)
{
    float2 r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "r"(x));
    return r;
}

// Two fp32 as e4m3 codes, round to nearest even, `lo` in bits 0-7; beyond the largest code it, NaN stays NaN.
__device__ __forceinline__ uint32_t f32_to_e4m3x2(float lo, float hi)
{
    uint32_t r;
    asm("{\n\t.reg .b16 x;\n\tcvt.rn.satfinite.e4m3x2.f32 x, %1, %2;\n\tcvt.u32.u16 %0, x;\n\t}"
        : "=r"(r)
        : "f"(hi), "f"(lo));
    return r;
}

// 2^(scale - 127) of a scale byte that an append wrote (27..247); 0 and 255, which none writes, give 0 and inf.
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// Four e4m3 codes times a power of two as two bf16 pairs. 4 significant bits and an exponent of the row's
// range: exact.
__device__ __forceinline__ uint2 e4m3x4_to_bf16(uint32_t codes, float scale)
{
    const float2 a = f16x2_to_f32(e4m3x2_to_f16x2(codes)), b = f16x2_to_f32(e4m3x2_to_f16x2(codes >> 16));
    uint2 r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.x) : "f"(a.y * scale), "f"(a.x * scale));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.y) : "f"(b.y * scale), "f"(b.x * scale));
    return r;
}

// ---- launchers ----
struct RowsView {
    const void* in;
    int64_t in_stride;  // elements
    void* out;
    int64_t out_stride;
    int heads;
};
cudaError_t launch_rope(const scale_rope_t& r, int n_rows, const RowsView& q, const RowsView& k, cudaStream_t st);
cudaError_t launch_append(const CacheView& c, bool e4m3, const BatchView& b, const scale_rope_t* r, const RowsView& q,
                          const RowsView& k, const RowsView& v, cudaStream_t st);
cudaError_t launch_cache_read(const CacheView& c, bool e4m3, const BatchView& b, void* k_out, int64_t k_stride,
                              void* v_out, int64_t v_stride, cudaStream_t st);

struct AttendView {
    int Hq, g, n_sink, n_local;
    float scale_log2;
    const void* q;
    int64_t q_stride;
    void* out;
    int64_t out_stride;
    float* lse;
};
size_t attend_ws_bytes(int Hq, int Hkv, bool e4m3, int n_seqs, int n_rows, int max_rows);
cudaError_t launch_attend(const AttendView& a, const CacheView& c, bool e4m3, const BatchView& b, uint8_t* ws,
                          uint64_t timeout_ns, cudaStream_t st);

}  // namespace scale
