// What the appends of many rows share, whatever their cache holds: the turned head
// of a row, and a row's query heads.
#pragma once
#include "rope.h"

namespace sidp {

// A row's head in fp32, normed where `gain` is given: 8 dims a lane.
template <int D>
__device__ __forceinline__ void load_head(const uint16_t* src, const uint16_t* gain, float eps, int sub, float (&x)[8]) {
  load8<true>(src + sub * 8, x);
  if (gain) {
    float g[8];
    load8<true>(gain + sub * 8, g);
    const float r = 1.0f / sqrtf(head_sum_sq<D>(x, sub) / (float)D + eps);
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = x[i] * r * g[i];
  }
}

template <int D, bool INTERLEAVED>
__device__ __forceinline__ u32x4_t turned_head(const RopeRowsCall& c, const uint16_t* src, const uint16_t* gain, int sub, const Turn& t) {
  float x[8];
  load_head<D>(src, gain, c.qk_eps, sub, x);
  return turned<INTERLEAVED>(x, t);
}

// The query heads of a row, and the row's errors. ONCE: stores are non-temporal.
template <int D, bool INTERLEAVED, bool ONCE>
__device__ __forceinline__ void query_row(const RopeRowsCall& c, int row) {
  constexpr int kLanes = D / 8, kHeads = 256 / kLanes;
  const int sub = threadIdx.x % kLanes, pos = c.positions[row];
  const bool ok = pos >= 0 && pos < c.max_seq;
  if (threadIdx.x == 0) {
    const int slot = c.slots[row];
    const uint32_t bad = (ok ? 0u : SIDP_DEVERR_POSITION) | (slot >= 0 && slot / kBlockTokens >= c.kv.nblk ? SIDP_DEVERR_BLOCK : 0u);
    if (bad) atomicOr(c.err, bad);
  }
  if (!ok) return;
  Turn t;
  load_turn(c.rope_cos + (int64_t)pos * (D / 2), c.rope_sin + (int64_t)pos * (D / 2), c.rot, INTERLEAVED, threadIdx.x & 63, sub, t);
  const uint16_t* src = c.qkv + (int64_t)row * c.stride;
  uint16_t* out = c.q_out + (int64_t)row * c.hq * D + sub * 8;
#pragma unroll 4
  for (int h = threadIdx.x / kLanes; h < c.hq; h += kHeads) {
    const u32x4_t v = turned_head<D, INTERLEAVED>(c, src + h * D, c.g_q, sub, t);
    if (ONCE) __builtin_nontemporal_store(v, (u32x4_t*)(out + h * D));
    else *(u32x4_t*)(out + h * D) = v;
  }
}

}  // namespace sidp
