// cache.cu -- rows into and out of a paged cache: rotary positions (scale_rope),
// the write of new tokens, bf16 or quantised to 8 bits (scale_cache_append), and
// the read of rows as bf16 (scale_cache_read).
#include <cuda_bf16.h>

#include "cache.cuh"
#include "launch.cuh"
#include "ptx_sm103.cuh"
#include "scale_internal.h"

namespace scale {
namespace {

using namespace scale_ptx;

constexpr int kPlaceThreads = 256;
constexpr int kPlaceWarps = kPlaceThreads / 32;
constexpr int kInFlight = 4;  // groups of four heads that a warp loads before it works on the first

// Heads of one tensor of a row: turned or not, into rows or into the cache.
struct Segment {
    const __nv_bfloat16* in;
    int64_t in_stride;
    __nv_bfloat16* out;  // rows (bf16 [rows][out_stride]), or the cache's pages
    int64_t out_stride;
    uint8_t* scales;  // 8-bit pages
    int end;          // one past its last head, counted over the segments
};

struct PlaceArgs {
    Segment q, k, v;  // heads [0, q.end), [q.end, k.end), [k.end, v.end)
    int n_rows;
    int parts;  // warps that share a row's heads
    CacheView c;
    BatchView b;
    const double* inv_freq;
    const int32_t* positions;
    uint8_t axis[64];
};

// f radians as a fraction of a turn, times 2^64, modulo 2^64. In integers: the 53 significant bits of f times
// 2^64 / (2 pi), shifted to their place (64-bit floating point products would take 152 SMs' warps
// longer than the rows of a small call).
__device__ __forceinline__ uint64_t turns_of(double f)
{
    constexpr uint64_t kPerRadian = 2935890503282001226ull;  // 2^64 / (2 pi), rounded
    const uint64_t bits = static_cast<uint64_t>(__double_as_longlong(f));
    const int e = static_cast<int>((bits >> 52) & 0x7FF);
    const uint64_t m = (bits & 0xFFFFFFFFFFFFFull) | (e ? 1ull << 52 : 0ull);
    const uint64_t hi = __umul64hi(m, kPerRadian), lo = m * kPerRadian;
    const int right = 1075 - (e ? e : 1);  // f = m 2^-right
    uint64_t t;
    if (right >= 128) t = 0;
    else if (right >= 64) t = hi >> (right - 64);
    else if (right > 0) t = lo >> right | hi << (64 - right);
    else t = right > -64 ? lo << -right : 0;
    return bits >> 63 ? 0 - t : t;
}

// cos and sin of `turn` / 2^64 of a turn. The turn is split into the nearest quarter and an angle of at
// most an eighth, so the angle in fp32 is off by 2^-25 of an eighth at most.
__device__ __forceinline__ float2 cos_sin_of_turn(uint64_t turn)
{
    const uint32_t t = static_cast<uint32_t>(turn >> 32) + 0x20000000u;
    const int quarter = t >> 30;
    const int rest = static_cast<int>(t & 0x3FFFFFFFu) - 0x20000000;  // 2^-32 turns
    float s, c;
    sincospif(static_cast<float>(rest) * 4.656612873077393e-10f, &s, &c);  // 2^-31: half turns
    if (quarter & 1) {
        const float x = c;
        c = -s;
        s = x;
    }
    return quarter & 2 ? make_float2(-c, -s) : make_float2(c, s);
}

// The k (and v) rows of a batch to their places in the cache and the q rows to q_out, all turned to their
// positions when ORDER is not 0 (1: pairs (i, i + 64), 2: pairs (2 i, 2 i + 1)); without a cache (CACHE
// 0) k goes to rows too. CACHE 1: bf16 pages, 2: e4m3.
//
// A warp takes rows, or a part of the heads of a row when there are few rows: lane j of eight takes the
// dimensions [8 j, 8 j + 8) and [64 + 8 j, ...) of a head, which holds both members of every pair in either
// order, so a head is read and written once in 16-byte pieces and its maximum is three shuffles. The
// warp's lanes share the 64 angles of the row through shared memory; a frequency is kept as a 64-bit
// fraction of a turn, so that position * frequency modulo 1 is one integer product.
// Bound by HBM.
template <int ORDER, int CACHE>
__global__ void __launch_bounds__(kPlaceThreads) k_place(const __grid_constant__ PlaceArgs a)
{
    __shared__ float s_cos[kPlaceWarps][64], s_sin[kPlaceWarps][64];
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sub = lane & 7, quad = lane >> 3;
    const int groups = (a.v.end + 3) / 4;
    uint64_t freq[2] = {0, 0};
    int ax[2] = {0, 0};
    if (ORDER) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            freq[i] = turns_of(a.inv_freq[lane + 32 * i]);
            ax[i] = a.axis[lane + 32 * i];
        }
    }
    const int64_t tasks = static_cast<int64_t>(a.n_rows) * a.parts;
    for (int64_t task = static_cast<int64_t>(blockIdx.x) * kPlaceWarps + warp; task < tasks;
         task += static_cast<int64_t>(gridDim.x) * kPlaceWarps) {
        const int row = static_cast<int>(task / a.parts), part = static_cast<int>(task - static_cast<int64_t>(row) * a.parts);
        int place = -1;  // row of the pool
        if (CACHE) {
            int token = -1;
            const int b = seq_of_row(a.b, row, &token);
            if (b < 0) continue;
            place = cache_row(a.c, a.b, b, token);
        }
        float c[8], s[8];
        if (ORDER) {
            __syncwarp();  // the row before is done with its angles
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int64_t p = a.positions[static_cast<int64_t>(ax[i]) * a.n_rows + row];
                const float2 x = cos_sin_of_turn(static_cast<uint64_t>(p) * freq[i]);
                s_cos[warp][lane + 32 * i] = x.x;
                s_sin[warp][lane + 32 * i] = x.y;
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int pair = ORDER == 1 ? 8 * sub + i : (i < 4 ? 4 * sub + i : 32 + 4 * sub + i - 4);
                c[i] = s_cos[warp][pair];
                s[i] = s_sin[warp][pair];
            }
        }
        const int g0 = static_cast<int>(static_cast<int64_t>(groups) * part / a.parts);
        const int g1 = static_cast<int>(static_cast<int64_t>(groups) * (part + 1) / a.parts);
        for (int g = g0; g < g1; g += kInFlight) {
            uint4 lo[kInFlight], hi[kInFlight];
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
                const int h = 4 * (g + u) + quad;
                lo[u] = hi[u] = make_uint4(0, 0, 0, 0);
                if (g + u < g1 && h < a.v.end) {
                    const Segment& sg = h < a.q.end ? a.q : h < a.k.end ? a.k : a.v;
                    const int hl = h < a.q.end ? h : h < a.k.end ? h - a.q.end : h - a.k.end;
                    const uint4* src = reinterpret_cast<const uint4*>(sg.in + row * sg.in_stride + hl * kHeadDim) + sub;
                    lo[u] = src[0];
                    hi[u] = src[8];
                }
            }
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
                if (g + u >= g1) break;  // the warp's groups end here
                const int h = 4 * (g + u) + quad;
                const bool turned = ORDER && h < a.k.end;
                const uint32_t w[8] = {lo[u].x, lo[u].y, lo[u].z, lo[u].w, hi[u].x, hi[u].y, hi[u].z, hi[u].w};
                float x[16];  // dimensions [8 sub, + 8), then [64 + 8 sub, + 8)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[2 * i] = __uint_as_float(w[i] << 16);
                    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
                }
                if (turned) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int m = ORDER == 1 ? i : 2 * i, n = ORDER == 1 ? 8 + i : 2 * i + 1;
                        const float p = x[m], q = x[n];
                        x[m] = p * c[i] - q * s[i];
                        x[n] = q * c[i] + p * s[i];
                    }
                }
                const bool to_cache = CACHE && h >= a.q.end;
                if (CACHE == 2 && __any_sync(0xFFFFFFFFu, to_cache)) {
                    // the largest finite magnitude of the head, as bits
                    uint32_t top = 0;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t m = __float_as_uint(x[i]) & 0x7FFFFFFFu;
                        top = max(top, m >= 0x7F800000u ? 0u : m);
                    }
#pragma unroll
                    for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                    // top = 1.m * 2^(E - 127) <= 448 * 2^e = 1.75 * 2^(8 + e)
                    int e = static_cast<int>(top >> 23) - 135 + ((top & 0x7FFFFFu) > 0x600000u);
                    e = e < kLowExp ? kLowExp : e;
                    const float inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
                    if (to_cache && h < a.v.end && place >= 0) {
                        const bool is_k = h < a.k.end;
                        const int hl = is_k ? h - a.q.end : h - a.k.end;
                        uint32_t y[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            y[i] = f32_to_e4m3x2(x[4 * i] * inv, x[4 * i + 1] * inv) |
                                   f32_to_e4m3x2(x[4 * i + 2] * inv, x[4 * i + 3] * inv) << 16;
                        uint8_t* dst = (is_k ? a.c.k : a.c.v) + (static_cast<int64_t>(place) * a.c.Hkv + hl) * kHeadDim + 8 * sub;
                        *reinterpret_cast<uint2*>(dst) = make_uint2(y[0], y[1]);
                        *reinterpret_cast<uint2*>(dst + 64) = make_uint2(y[2], y[3]);
                        if (sub == 0) {
                            const int page = place / a.c.page_size;
                            (is_k ? a.c.ks : a.c.vs)[(static_cast<int64_t>(page) * a.c.Hkv + hl) * a.c.page_size +
                                                     (place - page * a.c.page_size)] = static_cast<uint8_t>(e + 127);
                        }
                    }
                }
                if (h < a.v.end && !(CACHE == 2 && to_cache) && !(to_cache && place < 0)) {
                    uint32_t y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
                    const Segment& sg = h < a.q.end ? a.q : h < a.k.end ? a.k : a.v;
                    const int hl = h < a.q.end ? h : h < a.k.end ? h - a.q.end : h - a.k.end;
                    const int64_t at = to_cache ? static_cast<int64_t>(place) * a.c.Hkv * kHeadDim : row * sg.out_stride;
                    uint4* dst = reinterpret_cast<uint4*>(sg.out + at + hl * kHeadDim) + sub;
                    dst[0] = make_uint4(y[0], y[1], y[2], y[3]);
                    dst[8] = make_uint4(y[4], y[5], y[6], y[7]);
                }
            }
        }
    }
}

Segment segment(const RowsView& r, int from)
{
    return Segment{static_cast<const __nv_bfloat16*>(r.in), r.in_stride, static_cast<__nv_bfloat16*>(r.out), r.out_stride,
                   nullptr, from + r.heads};
}

template <int ORDER, int CACHE>
cudaError_t run_place(PlaceArgs& a, cudaStream_t st)
{
    int sms = 0;
    cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
    // Few rows: their heads are shared out, down to one group of four heads a warp.
    const int groups = (a.v.end + 3) / 4;
    const int64_t warps = static_cast<int64_t>(sms) * kPlaceWarps;
    a.parts = static_cast<int>(warps / a.n_rows < 1 ? 1 : warps / a.n_rows < groups ? warps / a.n_rows : groups);
    const int64_t ctas = (static_cast<int64_t>(a.n_rows) * a.parts + kPlaceWarps - 1) / kPlaceWarps;
    const int64_t most = static_cast<int64_t>(sms) * 8;
    return launch_after(st, dim3(static_cast<unsigned>(ctas < most ? ctas : most)), kPlaceThreads, 0, 1, k_place<ORDER, CACHE>, a);
}

// Rows of the batch as bf16: a warp takes a row's keys and values, four heads at a time when they are 8-bit
// (eight lanes of 16 codes each), two when they are bf16. Bound by HBM.
template <bool E4M3>
__global__ void __launch_bounds__(256) k_cache_read(const CacheView c, const BatchView b, __nv_bfloat16* k_out,
                                                    int64_t k_stride, __nv_bfloat16* v_out, int64_t v_stride)
{
    constexpr int kLanes = E4M3 ? 8 : 16;  // of a head
    constexpr int kHeads = 32 / kLanes;
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sub = lane % kLanes;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * 8 + warp; row < b.n_rows; row += static_cast<int64_t>(gridDim.x) * 8) {
        int token = -1;
        const int seq = seq_of_row(b, static_cast<int>(row), &token);
        if (seq < 0) continue;
        const int place = cache_row(c, b, seq, token);
        const int page = place < 0 ? 0 : place / c.page_size, slot = place < 0 ? 0 : place - page * c.page_size;
        const int n = 2 * c.Hkv;  // heads of k, then of v
#pragma unroll 4
        for (int h0 = 0; h0 < n; h0 += kHeads) {
            const int h = h0 + lane / kLanes;
            const bool is_k = h < c.Hkv;
            const int hl = is_k ? h : h - c.Hkv;
            __nv_bfloat16* out = is_k ? k_out : v_out;
            if (h >= n || !out) continue;
            uint4 x = make_uint4(0, 0, 0, 0);
            const int64_t at = (static_cast<int64_t>(place) * c.Hkv + hl) * kLanes + sub;
            if (place >= 0) x = reinterpret_cast<const uint4*>(is_k ? c.k : c.v)[at];
            uint4* dst = reinterpret_cast<uint4*>(out + row * (is_k ? k_stride : v_stride) + hl * kHeadDim);
            if (E4M3) {
                const float s = place < 0 ? 0.f : scale_value((is_k ? c.ks : c.vs)[(static_cast<int64_t>(page) * c.Hkv + hl) * c.page_size + slot]);
                const uint2 y0 = e4m3x4_to_bf16(x.x, s), y1 = e4m3x4_to_bf16(x.y, s);
                const uint2 y2 = e4m3x4_to_bf16(x.z, s), y3 = e4m3x4_to_bf16(x.w, s);
                dst[2 * sub] = make_uint4(y0.x, y0.y, y1.x, y1.y);
                dst[2 * sub + 1] = make_uint4(y2.x, y2.y, y3.x, y3.y);
            } else {
                dst[sub] = x;
            }
        }
    }
}

}  // namespace

cudaError_t launch_rope(const scale_rope_t& r, int n_rows, const RowsView& q, const RowsView& k, cudaStream_t st)
{
    PlaceArgs a{};
    a.q = segment(q, 0);
    a.k = segment(k, a.q.end);
    a.v = Segment{nullptr, 0, nullptr, 0, nullptr, a.k.end};
    a.n_rows = n_rows;
    a.inv_freq = r.inv_freq;
    a.positions = r.positions;
    for (int i = 0; i < 64; ++i) a.axis[i] = r.axis[i];
    return r.adjacent ? run_place<2, 0>(a, st) : run_place<1, 0>(a, st);
}

cudaError_t launch_append(const CacheView& c, bool e4m3, const BatchView& b, const scale_rope_t* r, const RowsView& q,
                          const RowsView& k, const RowsView& v, cudaStream_t st)
{
    PlaceArgs a{};
    a.q = segment(q, 0);
    a.k = segment(k, a.q.end);
    a.v = segment(v, a.k.end);
    a.k.out = reinterpret_cast<__nv_bfloat16*>(c.k);
    a.v.out = reinterpret_cast<__nv_bfloat16*>(c.v);
    a.n_rows = b.n_rows;
    a.c = c;
    a.b = b;
    if (!r) return e4m3 ? run_place<0, 2>(a, st) : run_place<0, 1>(a, st);
    a.inv_freq = r->inv_freq;
    a.positions = r->positions;
    for (int i = 0; i < 64; ++i) a.axis[i] = r->axis[i];
    if (r->adjacent) return e4m3 ? run_place<2, 2>(a, st) : run_place<2, 1>(a, st);
    return e4m3 ? run_place<1, 2>(a, st) : run_place<1, 1>(a, st);
}

cudaError_t launch_cache_read(const CacheView& c, bool e4m3, const BatchView& b, void* k_out, int64_t k_stride,
                              void* v_out, int64_t v_stride, cudaStream_t st)
{
    int sms = 0;
    cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
    const int64_t ctas = (static_cast<int64_t>(b.n_rows) + 7) / 8, most = static_cast<int64_t>(sms) * 8;
    const dim3 grid(static_cast<unsigned>(ctas < most ? ctas : most));
    return launch_after(st, grid, 256, 0, 1, e4m3 ? k_cache_read<true> : k_cache_read<false>, c, b,
                        static_cast<__nv_bfloat16*>(k_out), k_stride, static_cast<__nv_bfloat16*>(v_out), v_stride);
}

}  // namespace scale
