// QK-norm, rotary positions and the append to the paged KV cache for many rows
// (prompt chunks, drafted tokens, whole batches) at given positions and slots.
//
// Bound by HBM for prompts: each bf16 is read once and written once. A lane holds
// 8 dims of a head, D / 8 lanes a head, 16 (32 at D = 64) heads a pass; a
// workgroup takes a row's q and k heads, so the row's angles are loaded once and
// stay in registers for all of them.
#include "common.h"
#include "internal.h"
#include "rope.h"

namespace sidp {

namespace {

// The row's block and offset in it; false (and an error bit unless the slot is
// negative) if the row is not to be cached.
__device__ __forceinline__ bool slot_of_row(const RopeRowsCall& c, int slot, int64_t& blk, int& off, uint32_t& bad) {
  if (slot < 0) return false;
  blk = slot / kBlockTokens;
  off = slot % kBlockTokens;
  if (blk >= c.kv.nblk) {
    bad |= SIDP_DEVERR_BLOCK;
    return false;
  }
  blk += (int64_t)c.region * c.kv.nblk;
  return true;
}

template <int D, bool INTERLEAVED>
__global__ void __launch_bounds__(256) k_rope_rows(RopeRowsCall c) {
  constexpr int kLanes = D / 8;
  constexpr int kHeads = 256 / kLanes;
  const int row = blockIdx.x;
  if (c.row_count && row >= *c.row_count) return;
  const int sub = threadIdx.x % kLanes, h_in = threadIdx.x / kLanes, lane = threadIdx.x & 63;
  const int pos = c.positions[row];
  uint32_t bad = 0;
  const bool ok_pos = pos >= 0 && pos < c.max_seq;
  int64_t blk = 0;
  int off = 0;
  const bool ok_slot = slot_of_row(c, c.slots[row], blk, off, bad);
  if (!ok_pos) bad |= SIDP_DEVERR_POSITION;
  if (bad && threadIdx.x == 0 && blockIdx.y == 0) atomicOr(c.err, bad);
  if (!ok_pos) return;
  const int heads = c.hq + 2 * c.hkv;
  const uint16_t* src = c.qkv + (int64_t)row * c.stride;
  Turn t;
  load_turn(c.rope_cos + (int64_t)pos * (D / 2), c.rope_sin + (int64_t)pos * (D / 2), c.rot, INTERLEAVED, lane, sub, t);
  for (int h = blockIdx.y * kHeads + h_in; h < heads; h += gridDim.y * kHeads) {
    float x[8];
    load8<true>(src + h * D + sub * 8, x);
    const bool is_q = h < c.hq, is_k = !is_q && h < c.hq + c.hkv;
    if (!is_q && !is_k) {
      if (ok_slot) {
        uint16_t* vb = c.kv.v + (blk * c.kv.hkv + (h - c.hq - c.hkv)) * (int64_t)(D * kBlockTokens);
#pragma unroll
        for (int i = 0; i < 8; i++) vb[(sub * 8 + i) * kBlockTokens + off] = f2bf(x[i]);
      }
      continue;
    }
    const uint16_t* gn = is_q ? c.g_q : c.g_k;
    if (gn) {
      float g[8];
      load8<true>(gn + sub * 8, g);
      const float r = 1.0f / sqrtf(head_sum_sq<D>(x, sub) / (float)D + c.qk_eps);
#pragma unroll
      for (int i = 0; i < 8; i++) x[i] = x[i] * r * g[i];
    }
    const u32x4_t out = turned<INTERLEAVED>(x, t);
    if (is_q) {
      *(u32x4_t*)(c.q_out + ((int64_t)row * c.hq + h) * D + sub * 8) = out;
    } else if (ok_slot) {
      uint16_t* kb = c.kv.k + (blk * c.kv.hkv + (h - c.hq)) * (int64_t)(D * kBlockTokens);
      *(u32x4_t*)(kb + (sub * kBlockTokens + off) * 8) = out;
    }
  }
}

template <int D>
hipError_t launch_d(const RopeRowsCall& c, hipStream_t s) {
  constexpr int kHeads = 256 / (D / 8);
  const int passes = (c.hq + 2 * c.hkv + kHeads - 1) / kHeads;
  const dim3 grid(c.rows, c.rows >= 8 * c.num_cus ? 1 : passes);
  if (c.interleaved) k_rope_rows<D, true><<<grid, 256, 0, s>>>(c);
  else k_rope_rows<D, false><<<grid, 256, 0, s>>>(c);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_rows(const RopeRowsCall& c, hipStream_t s) {
  if (c.rows <= 0) return hipSuccess;
  return c.kv.d == 128 ? launch_d<128>(c, s) : launch_d<64>(c, s);
}

}  // namespace sidp
