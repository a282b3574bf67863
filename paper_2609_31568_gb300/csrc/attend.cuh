// attend.cuh -- what the two routes of scale_cache_attend share: the rows and
// keys of a sequence, and which route takes it.
#pragma once

#include "cache.cuh"

namespace scale {

// (token, query head) rows of a KV head up to which a call's sequences go to k_rows, whose registers hold no more. 32 query
// heads on 8: one sequence of 2 tokens at 4,096 12 us there and 23 by the tensor cores' route, 16 of 4 at 8,192 96
// and 102. 8-bit: 14 and 26, 72 and 128; 24 rows, 16 of 6 at 8,192 86 and 129, one of 6 at 4,096 25 and 24; 32 rows,
// which spill, 124 and 130, 34 and 25.
__host__ __device__ constexpr int rows_max(bool e4m3) { return e4m3 ? 24 : 16; }
constexpr int kMaxSms = 160;  // SMs that a call uses at most

// Rows and keys of sequence b. Its computed rows are [row0, row0 + rows), tokens
// pos0 .. pos0 + rows - 1; no row sees a key outside [0, n_sink) and [lo, pos0 + rows).
struct Seq {
    int row0, rows;
    int pos0, lo;
};

__device__ __forceinline__ Seq seq_of(const AttendView& a, const BatchView& b, int row0, int end, int len)
{
    Seq s;
    s.row0 = row0;
    const int n = s.row0 < 0 || end <= s.row0 ? 0 : end - s.row0;
    s.rows = n < b.max_rows ? n : b.max_rows;
    if (s.rows > b.n_rows - s.row0) s.rows = b.n_rows - s.row0 > 0 ? b.n_rows - s.row0 : 0;
    s.pos0 = (len > 0 ? len : 0) - n;
    s.lo = a.n_local >= 0 && s.pos0 > a.n_local ? s.pos0 - a.n_local : 0;
    return s;
}

__device__ __forceinline__ Seq seq_of(const AttendView& a, const BatchView& b, int i)
{
    return seq_of(a, b, b.row_start[i], b.row_start[i + 1], b.kv_len[i]);
}

// Exponent of the power of two that brings values of at most `top` (fp32 bits, finite) below 2^15, inside f16;
// it and its negative are exponents of normal fp32 values.
__device__ __forceinline__ int f16_exponent(uint32_t top)
{
    const int e = static_cast<int>(top >> 23) - 127 - 14;
    return e < -100 ? -100 : e;
}

// Calls whose sequences may have more than rows_max rows per KV head: tcgen05, 128 rows at a time.
size_t chunk_ws_bytes(int g, int Hkv, int n_seqs, int n_rows, int max_rows);
cudaError_t launch_chunks(const AttendView& a, const CacheView& c, bool e4m3, const BatchView& b, int sms,
                          int32_t* status, uint8_t* ws, uint64_t timeout_ns, cudaStream_t st);

}  // namespace scale
