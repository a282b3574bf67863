// attend.cu -- attention of a batch's new tokens over their sequences in a
// paged cache (scale_cache_attend).
#include <cuda_bf16.h>

#include "cache.cuh"
#include "launch.cuh"
#include "ptx_sm103.cuh"
#include "scale_internal.h"

namespace scale {
namespace {

using namespace scale_ptx;

// One warp per (row, query head): a key at a time, an online softmax in log2 units.
template <bool E4M3>
__global__ void __launch_bounds__(256) k_attend_warp(const AttendView a, const CacheView c, const BatchView b)
{
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const int64_t task = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    const int row = static_cast<int>(task / a.Hq), h = static_cast<int>(task - static_cast<int64_t>(row) * a.Hq);
    if (row >= b.n_rows) return;
    int p = -1;
    const int seq = seq_of_row(b, row, &p);
    if (seq < 0 || row - b.row_start[seq] >= b.max_rows) return;
    const int j = h / a.g;
    const auto* q = static_cast<const __nv_bfloat16*>(a.q) + row * a.q_stride + h * kHeadDim + 4 * lane;
    float x[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    for (int i = 0; i < 4; ++i) x[i] = __bfloat162float(q[i]);
    const int lo = a.n_local >= 0 && p > a.n_local ? p - a.n_local : 0;
    for (int t = 0; t <= p; ++t) {
        if (t >= a.n_sink && t < lo) t = lo;
        const int place = cache_row(c, b, seq, t);
        float k[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
        if (place >= 0) {
            const int64_t at = (static_cast<int64_t>(place) * c.Hkv + j) * kHeadDim + 4 * lane;
            for (int kv = 0; kv < 2; ++kv) {
                uint2 w;
                if (E4M3) {
                    const int page = place / c.page_size;
                    const uint8_t s = (kv ? c.vs : c.ks)[(static_cast<int64_t>(page) * c.Hkv + j) * c.page_size + place - page * c.page_size];
                    w = e4m3x4_to_bf16(*reinterpret_cast<const uint32_t*>((kv ? c.v : c.k) + at), scale_value(s));
                } else {
                    w = *reinterpret_cast<const uint2*>((kv ? c.v : c.k) + 2 * at);
                }
                float* y = kv ? v : k;
                y[0] = __uint_as_float(w.x << 16);
                y[1] = __uint_as_float(w.x & 0xFFFF0000u);
                y[2] = __uint_as_float(w.y << 16);
                y[3] = __uint_as_float(w.y & 0xFFFF0000u);
            }
        }
        float s = 0.f;
        for (int i = 0; i < 4; ++i) s += x[i] * k[i];
        for (int i = 16; i > 0; i >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, i);
        s *= a.scale_log2;
        const float m_new = fmaxf(m, s);
        const float base = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = ex2(m - base), w = ex2(s - base);
        l = l * alpha + w;
        for (int i = 0; i < 4; ++i) o[i] = o[i] * alpha + w * v[i];
        m = m_new;
    }
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    auto* out = static_cast<__nv_bfloat16*>(a.out) + row * a.out_stride + h * kHeadDim + 4 * lane;
    for (int i = 0; i < 4; ++i) out[i] = __float2bfloat16_rn(o[i] * inv);
    if (a.lse && lane == 0) a.lse[static_cast<int64_t>(row) * a.Hq + h] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace

size_t attend_ws_bytes(int Hq, int Hkv, int n_seqs, int n_rows, int max_rows)
{
    (void)Hq;
    (void)Hkv;
    (void)n_seqs;
    (void)n_rows;
    (void)max_rows;
    return 256;
}

cudaError_t launch_attend(const AttendView& a, const CacheView& c, bool e4m3, const BatchView& b, uint8_t* ws,
                          uint64_t timeout_ns, cudaStream_t st)
{
    (void)ws;
    (void)timeout_ns;
    const int64_t grid = (static_cast<int64_t>(b.n_rows) * a.Hq + 7) / 8;
    if (grid > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
    return launch_after(st, dim3(static_cast<unsigned>(grid)), 256, 0, 1, e4m3 ? k_attend_warp<true> : k_attend_warp<false>, a, c, b);
}

}  // namespace scale
