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

// Drafted trees: row `row` of the batch, whose sequence's node 0 is its row `row0` and token `pos0`. Bits of the 32 tokens from
// t0 on that it sees: those before pos0, as far as the window goes (not here), and its mask's nodes. None without a
// position, or where the row's own token has no place.
struct TreeRow {
    const uint32_t* mask;
    int words;     // 0: it sees nothing
    int position;  // at least pos0
    int pos0;
};

__device__ __forceinline__ TreeRow tree_row(const TreeView& tree, int row0, int pos0, int row)
{
    TreeRow x;
    const int p = tree.positions[row];
    x.mask = tree.masks + static_cast<int64_t>(row) * tree.words;
    x.words = p < 0 || pos0 + (row - row0) < 0 ? 0 : tree.words;
    x.position = p > pos0 ? p : pos0;
    x.pos0 = pos0;
    return x;
}

// The lowest n bits, 0 <= n <= 32 or beyond either end.
__device__ __forceinline__ uint32_t ones_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u; }

__device__ __forceinline__ uint32_t tree_bits(const TreeRow& x, int t0)
{
    if (x.words == 0) return 0u;
    const int c = t0 - x.pos0, w = c >> 5;  // node of t0, negative before them
    const uint32_t lo = static_cast<uint32_t>(w) < static_cast<uint32_t>(x.words) ? x.mask[w] : 0u;
    const uint32_t hi = static_cast<uint32_t>(w + 1) < static_cast<uint32_t>(x.words) ? x.mask[w + 1] : 0u;
    return __funnelshift_r(lo, hi, c & 31) | ones_below(-c);
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
template <bool TREE>
cudaError_t launch_chunks(const AttendView& a, const TreeView& tree, const CacheView& c, bool e4m3, const BatchView& b, int sms,
                          int32_t* status, uint8_t* ws, uint64_t timeout_ns, cudaStream_t st);

}  // namespace scale
