// How the decode attention kernels cut their work: shared by the bf16 cache's
// (attention_decode.hip) and the 4-bit cache's (attention_decode_kvq.hip).
#pragma once

#include "common.h"
#include "kernels.h"

namespace wide {

constexpr int kSplitThreads = 256;  // threads of a workgroup that lists its units

// Active query heads of (sequence b, KV head hkv): bit i = head hkv*qpk + i.
__device__ __forceinline__ uint32_t active_heads(const AttnDecArgs& a, int b, int hkv) {
  const uint8_t* mrow = a.mask + (int64_t)b * a.ng;
  uint32_t act = 0;
  for (int i = 0; i < a.qpk; ++i)
    if (mrow[(hkv * a.qpk + i) / a.hpg]) act |= 1u << i;
  return act;
}
__device__ __forceinline__ int seq_len(const AttnDecArgs& a, int b) {
  return a.kv_len ? min(a.kv_len[b], a.L) : a.L;
}

// Balanced split.  What a token reads depends on the mask and on its
// sequence's length, both known on the device only, so cutting every
// (sequence, KV head) pair into equal chunks leaves some CUs with several
// times the work of others.  Here every workgroup first lists the pairs' units
// of KU keys (0 for a pair no head of which is active) as a prefix sum in
// LDS; with U units in all, wave i of a.waves (one round of resident waves)
// takes units [i q, (i + 1) q), q = max(ceil(U / waves), KMIN), which may
// cross from one pair into the next.  Each (wave, pair) segment leaves one
// partial result, in slot i + (active pairs before the pair); workgroup 0
// writes every pair's first slot and segment count for the merge.
// bf16 cache, ragged, 32 sequences of up to 8192 keys, half the KV heads active:
// kernel 91 -> 69 us; nothing ragged, all heads active: 201 -> 197.
constexpr uint64_t kUnitBits = (1ull << 40) - 1;  // of a prefix: units; above them: active pairs

// s_pre: B * n_kv + 1 prefixes; s_sum: kSplitThreads / kWave + 1 words, the last one q.
template <int KU, int KMIN>
__device__ __forceinline__ void list_units(const AttnDecArgs& a, uint64_t* s_pre, uint64_t* s_sum) {
  const int tid = threadIdx.x, w = wave_id(), lane = lane_id();
  const int P = a.B * a.n_kv, per = (P + kSplitThreads - 1) / kSplitThreads;
  const int p0 = min(P, tid * per), p1 = min(P, p0 + per);
  uint64_t sum = 0;  // active pairs << 40 | units
  for (int p = p0; p < p1; ++p) {
    const int b = p / a.n_kv, h0 = (p - b * a.n_kv) * a.qpk;
    const uint8_t* mrow = a.mask + (int64_t)b * a.ng;
    const int g0 = h0 / a.hpg, g1 = (h0 + a.qpk - 1) / a.hpg;
    const int len = max(seq_len(a, b), 0);
    uint32_t on = mrow[g0];
    for (int g = g0 + 1; g <= g1; ++g) on |= mrow[g];
    const int n = on ? (len + KU - 1) / KU : 0;
    s_pre[p] = n;
    sum += (uint64_t)(n > 0) << 40 | (uint32_t)n;
  }
  uint64_t x = sum;  // inclusive scan over the wave, then over the waves
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const uint64_t y = __shfl_up((unsigned long long)x, d);
    if (lane >= d) x += y;
  }
  if (lane == kWave - 1) s_sum[w] = x;
  __syncthreads();
  uint64_t run = x - sum, all = 0;
#pragma unroll
  for (int i = 0; i < kSplitThreads / kWave; ++i) {
    if (i < w) run += s_sum[i];
    all += s_sum[i];
  }
  const int units = (int)(all & kUnitBits), q = max((units + a.waves - 1) / a.waves, KMIN);
  for (int p = p0; p < p1; ++p) {
    const int n = (int)s_pre[p], u = (int)(run & kUnitBits), rank = (int)(run >> 40);
    s_pre[p] = run;
    if (blockIdx.x == 0) {
      a.table[2 * p] = u / q + rank;
      a.table[2 * p + 1] = n > 0 ? (u + n - 1) / q - u / q + 1 : 0;
    }
    run += (uint64_t)(n > 0) << 40 | (uint32_t)n;
  }
  if (tid == 0) {
    s_pre[P] = all;
    s_sum[kSplitThreads / kWave] = (uint64_t)q;
  }
  __syncthreads();
}

// The pair of unit u, the last one with at most u units before it: 64
// candidates per step, one per lane.
__device__ __forceinline__ int pair_of_unit(const uint64_t* s_pre, int P, int u) {
  const int lane = lane_id();
  int lo = 0, n = P;
  while (n > 1) {
    const int st = (n + kWave - 1) / kWave, i = lo + lane * st;
    const uint64_t le = __ballot(lane * st < n && (int)(s_pre[min(i, P)] & kUnitBits) <= u);
    const int k = 63 - __builtin_clzll(le);  // (lane 0's candidate always qualifies)
    n = min(st, n - k * st);
    lo += k * st;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

}  // namespace wide
