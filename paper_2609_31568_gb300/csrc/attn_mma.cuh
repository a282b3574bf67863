// attn_mma.cuh -- what the tcgen05 attention kernels share: the barriers of a
// CTA with one or two 128-row query tiles, the loop that issues its products, and
// the limits of its online softmax.
#pragma once

#include "ptx_sm103.cuh"
#include "scale_internal.h"

namespace scale {
namespace {

using namespace scale_ptx;

constexpr uint32_t kTileBytes = 128 * 128 * 2;  // one 128 x 128 bf16 tile
constexpr uint32_t kHalf = kTileBytes / 2;    // one 64-column half (128 rows x 128 B)
constexpr float kRescaleThreshold = 8.0f;     // log2 units
constexpr float kFastSumLimit = 65536.0f;     // 2^16: largest tile sum kept on the fast path

struct Barriers {
    uint64_t q_full;
    uint64_t kv_full[2];    // [t & 1]: K(t) and V(t - 1) landed (step T: V(T - 1) alone)
    uint64_t s_full[2][2];  // [q][t & 1]: S(t) of Q tile q ready (and every earlier MMA of the CTA done)
    uint64_t p_full[2];  // P of Q tile q written (128 arrivals)
    uint64_t o_full;     // last P.V of both tiles done
    uint64_t drain;
};

__device__ __forceinline__ void fail(volatile int* abort_flag, int32_t* status)
{
    *abort_flag = 1;
    record_status(status, SCALE_ERR_TIMEOUT);
}

// One iteration t (t & 1 = ST) of the MMA issue loop of a CTA with NQ (1 or 2)
// query tiles: wait for K(t) and V(t - 1), then per query tile wait for
// P(t - 1), issue O += P(t - 1) V(t - 1) and S = Q K(t)^T, and commit S-ready.
template <int NQ, int ST>
__device__ __forceinline__ bool mma_iteration(Barriers* bars, uint32_t tmem, uint64_t qdesc0, uint64_t kdesc0,
                                              uint64_t vdesc0, uint32_t id_qk, uint32_t id_pv, int t,
                                              uint64_t timeout_ns, const volatile int* abort_flag)
{
    // Descriptors of the two stages differ by kTileBytes >> 4 in the address field.
    constexpr uint64_t kStageStep = kTileBytes >> 4;
    const uint32_t ph = (t >> 1) & 1;
    if (!mbar_test(&bars->kv_full[ST], ph) && !mbar_wait_bounded(&bars->kv_full[ST], ph, timeout_ns, abort_flag))
        return false;
    // TMA data is ordered by the barrier's transaction count; from t = 1
    // the fence after the P wait below precedes every MMA of the iteration.
    if (t == 0) tc_fence_after();
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
        if (t > 0) {
            if (!mbar_wait_bounded(&bars->p_full[qt], ST ^ 1, timeout_ns, abort_flag)) return false;
            tc_fence_after();
            mma_ts_k128<2048>(tmem + qt * 256 + 128, tmem + qt * 256, vdesc0 + (ST ^ 1) * kStageStep, id_pv,
                              t > 1 ? 1u : 0u);
        }
        mma_ss_k128<kHalf>(tmem + qt * 256, qdesc0 + qt * kStageStep, kdesc0 + ST * kStageStep, id_qk, 0u);
        mma_commit(&bars->s_full[qt][ST]);
    }
    return true;
}

// The MMA issue loop, run by one thread: T iterations (two per trip, so the
// stage indices are constants), then the last P.V and the O-ready commit.
// `skip_last`: the last key tile lies in the future of every row of query tile
// 0 (two query blocks of one head), which leaves its P.V out: P is 0, and 0
// times an infinite value row is NaN. This thread is the critical path: NQ is
// a compile-time constant and all state is held in registers. Returns false
// when a wait ran out or the kernel was aborted.
template <int NQ>
__device__ __forceinline__ bool mma_issue_loop(Barriers* bars, uint32_t tmem, uint64_t qdesc0, uint64_t kdesc0,
                                               uint64_t vdesc0, uint32_t id_qk, uint32_t id_pv, int T,
                                               bool skip_last, uint64_t timeout_ns,
                                               const volatile int* abort_flag)
{
    constexpr uint64_t kStageStep = kTileBytes >> 4;
    int t = 0;
    for (; t + 1 < T; t += 2) {
        if (!mma_iteration<NQ, 0>(bars, tmem, qdesc0, kdesc0, vdesc0, id_qk, id_pv, t, timeout_ns, abort_flag) ||
            !mma_iteration<NQ, 1>(bars, tmem, qdesc0, kdesc0, vdesc0, id_qk, id_pv, t + 1, timeout_ns, abort_flag))
            return false;
    }
    if (t < T && !mma_iteration<NQ, 0>(bars, tmem, qdesc0, kdesc0, vdesc0, id_qk, id_pv, t, timeout_ns, abort_flag))
        return false;
    if (!mbar_wait_bounded(&bars->kv_full[T & 1], (T >> 1) & 1, timeout_ns, abort_flag)) return false;
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
        if (!mbar_wait_bounded(&bars->p_full[qt], (T - 1) & 1, timeout_ns, abort_flag)) return false;
        tc_fence_after();
        if (NQ == 2 && qt == 0 && skip_last) continue;
        mma_ts_k128<2048>(tmem + qt * 256 + 128, tmem + qt * 256, vdesc0 + ((T - 1) & 1) * kStageStep, id_pv,
                          T > 1 ? 1u : 0u);
    }
    mma_commit(&bars->o_full);
    return true;
}

}  // namespace
}  // namespace scale
