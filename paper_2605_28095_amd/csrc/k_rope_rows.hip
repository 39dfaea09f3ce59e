// QK-norm, rotary positions and the append to the paged KV cache for many rows
// (prompt chunks, drafted tokens, whole batches) at given positions and slots.
//
// Bound by HBM for prompts: each bf16 is read once and written once. A lane holds
// 8 dims of a head, D / 8 lanes a head. One launch, three kinds of workgroup:
//  - query: a row's query heads; its angles are loaded once, for all of them.
//  - key, value: one KV head of a tile of consecutive rows, through LDS. A block
//    keeps its 16 tokens side by side ([d / 8][token][8], [d][token]), so a row by
//    itself writes 16 or 2 bytes of each line, and lines written in parts, from
//    workgroups on different XCDs' L2s, cost HBM a read each. A tile writes whole
//    lines wherever its rows' slots follow each other, whatever they start at.
// 8192 rows of 64 and 8 heads of 128 dims 66 us, 5.1 TB/s (125 with a row's K and V written
// by the row); 256 rows 8 us; 8 rows 3.2 us on the GPU, the launch costs more.
#include "common.h"
#include "internal.h"
#include "rope.h"

namespace sidp {

namespace {

constexpr int kLongTile = 64, kShortTile = 16;
// Calls of at least this many rows take the long tile: a short one cuts more lines, but spreads few rows over more CUs. They also
// store their query rows past the caches, which leaves those to the lines of K and V: 4096 rows 28-30 us (33-36 through the caches),
// 8192 61-66 (65-69), 2048 15.7 (15.9). The attention then reads its queries from memory, and still the two calls behind a source
// just written are no slower together: 8192 rows as 64 chunks 220 us (241), 8 319 (331), one prompt 1074 (1083); 4096 as 16, 4, 1
// 151, 162, 324 (155, 161, 323); 2048 as 8, 2, 1 83, 87, 116 (82, 86, 116). Non-temporal loads as well: 8192 rows 62, but 4096 and
// 2048, whose source the caches hold, 33 and 19.
constexpr int kLongRows = 2048;

template <int D, bool INTERLEAVED>
__device__ __forceinline__ u32x4_t turned_head(const RopeRowsCall& c, const uint16_t* src, const uint16_t* gain, int sub, const Turn& t) {
  float x[8];
  load8<true>(src + sub * 8, x);
  if (gain) {
    float g[8];
    load8<true>(gain + sub * 8, g);
    const float r = 1.0f / sqrtf(head_sum_sq<D>(x, sub) / (float)D + c.qk_eps);
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = x[i] * r * g[i];
  }
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

template <int D, bool INTERLEAVED, int TILE>
__global__ void __launch_bounds__(256) k_rope_rows(RopeRowsCall c, int tiles) {
  constexpr int kLanes = D / 8, kRows = 256 / kLanes;  // rows of a pass
  constexpr int kRow = D + 8;                          // of the tile in LDS, in elements
  __shared__ __attribute__((aligned(16))) uint16_t s_x[TILE * kRow];
  __shared__ int s_slot[TILE];
  __shared__ int s_piece[TILE];
  __shared__ int s_pieces;
  const int rows = c.row_count ? min(c.rows, *c.row_count) : c.rows;
  const int hkv = c.kv.hkv, t = threadIdx.x;
  const int kv_groups = tiles * hkv;
  if ((int)blockIdx.x >= 2 * kv_groups) {
    const int row = blockIdx.x - 2 * kv_groups;
    if (row < rows) query_row<D, INTERLEAVED, TILE == kLongTile>(c, row);
    return;
  }
  // tiles of one head follow each other at a distance of the heads, so that with 8 heads they share an XCD's L2
  const bool value = (int)blockIdx.x >= kv_groups;
  const int at = value ? blockIdx.x - kv_groups : blockIdx.x;
  const int row0 = at / hkv * TILE, head = at % hkv;
  const int n = min(TILE, rows - row0);
  if (n <= 0) return;
  if (t < TILE) {
    int slot = -1;
    if (t < n) {
      const int pos = c.positions[row0 + t];
      slot = c.slots[row0 + t];
      if (pos < 0 || pos >= c.max_seq || slot / kBlockTokens >= c.kv.nblk) slot = -1;
    }
    s_slot[t] = slot;
  }
  const int sub = t % kLanes;
  const uint16_t* src = c.qkv + (int64_t)row0 * c.stride + (c.hq + (value ? hkv : 0) + head) * D;
  // all loads of the tile before the first use
  if (value) {
    u32x4_t x[TILE / kRows > 0 ? TILE / kRows : 1];
#pragma unroll
    for (int i = 0; i < TILE; i += kRows) {
      const int r = i + t / kLanes;
      if (r < n) x[i / kRows] = *(const u32x4_t*)(src + (int64_t)r * c.stride + sub * 8);
    }
#pragma unroll
    for (int i = 0; i < TILE; i += kRows) {
      const int r = i + t / kLanes;
      if (r < n) *(u32x4_t*)(s_x + r * kRow + sub * 8) = x[i / kRows];
    }
  } else {
#pragma unroll
    for (int i = 0; i < TILE; i += kRows) {
      const int r = i + t / kLanes;
      if (r < n) {
        const int pos = min(max(c.positions[row0 + r], 0), c.max_seq - 1);
        Turn turn;
        load_turn(c.rope_cos + (int64_t)pos * (D / 2), c.rope_sin + (int64_t)pos * (D / 2), c.rot, INTERLEAVED, t & 63, sub, turn);
        *(u32x4_t*)(s_x + r * kRow + sub * 8) = turned_head<D, INTERLEAVED>(c, src + (int64_t)r * c.stride, c.g_k, sub, turn);
      }
    }
  }
  __syncthreads();
  const int64_t region = (int64_t)c.region * c.kv.nblk;
  auto block_of = [&](uint16_t* cache, int slot) {
    return cache + ((region + slot / kBlockTokens) * hkv + head) * (int64_t)(D * kBlockTokens);
  };
  if (!value) {
    // a thread a (token, 8 dims) piece, tokens fastest: 16 tokens of a block are 256 bytes
    for (int i = t; i < TILE * kLanes; i += 256) {
      const int r = i / (16 * kLanes) * 16 + i % 16, d8 = i / 16 % kLanes;
      const int slot = s_slot[r];
      if (slot >= 0)
        *(u32x4_t*)(block_of(c.kv.k, slot) + (d8 * kBlockTokens + slot % kBlockTokens) * 8) = *(const u32x4_t*)(s_x + r * kRow + d8 * 8);
    }
    return;
  }
  // Pieces: runs of rows whose slots follow each other within 8 tokens of a block (first row | rows << 16), 16 bytes of each dim
  // where there are 8.
  if (t < 64) {
    const int slot = t < TILE ? s_slot[t] : -1;
    const bool starts = slot >= 0 && (t == 0 || slot % 8 == 0 || s_slot[t - 1] != slot - 1);
    const uint64_t who = __ballot(starts);
    if (starts) {
      int len = 1;
      while (t + len < TILE && (slot + len) % 8 != 0 && s_slot[t + len] == slot + len) len++;
      s_piece[__popcll(who & ((1ull << t) - 1))] = t | len << 16;
    }
    if (t == 0) s_pieces = __popcll(who);
  }
  __syncthreads();
  const int pieces = s_pieces;
  // two pieces, often the halves of a block, at a time: 32 bytes a dim
  for (int i = t; i < (pieces + 1) / 2 * 2 * D; i += 256) {
    const int p = i / (2 * D) * 2 + i % 2, d = i / 2 % D;
    if (p >= pieces) continue;
    const int r = s_piece[p] & 0xffff, len = s_piece[p] >> 16, slot = s_slot[r];
    uint16_t* to = block_of(c.kv.v, slot) + d * kBlockTokens + slot % kBlockTokens;
    const uint16_t* from = s_x + r * kRow + d;
    if (len == 8) {
      u32x4_t v;
#pragma unroll
      for (int k = 0; k < 4; k++) v[k] = from[2 * k * kRow] | (uint32_t)from[(2 * k + 1) * kRow] << 16;
      *(u32x4_t*)to = v;
    } else {
      for (int k = 0; k < len; k++) to[k] = from[k * kRow];
    }
  }
}

int tile_of(int rows) { return rows >= kLongRows ? kLongTile : kShortTile; }
int64_t groups_of(int rows, int hkv) {
  const int tile = tile_of(rows);
  return 2 * (int64_t)((rows + tile - 1) / tile) * hkv + rows;
}

template <int D, bool INTERLEAVED>
hipError_t launch_layout(const RopeRowsCall& c, hipStream_t s) {
  const int tile = tile_of(c.rows), tiles = (c.rows + tile - 1) / tile;
  const unsigned grid = (unsigned)groups_of(c.rows, c.kv.hkv);
  if (tile == kLongTile) k_rope_rows<D, INTERLEAVED, kLongTile><<<grid, 256, 0, s>>>(c, tiles);
  else k_rope_rows<D, INTERLEAVED, kShortTile><<<grid, 256, 0, s>>>(c, tiles);
  return hipGetLastError();
}

}  // namespace

// HIP's launches have fewer than 2^32 threads.
bool rope_rows_fit(int rows, int hkv) { return groups_of(rows, hkv) * 256 < (int64_t)1 << 32; }

hipError_t launch_rope_rows(const RopeRowsCall& c, hipStream_t s) {
  if (c.rows <= 0) return hipSuccess;
  if (c.kv.d == 128) return c.interleaved ? launch_layout<128, true>(c, s) : launch_layout<128, false>(c, s);
  return c.interleaved ? launch_layout<64, true>(c, s) : launch_layout<64, false>(c, s);
}

}  // namespace sidp
