// QK-norm, rotary positions and the append of many rows to the 8-bit KV cache, and
// cached rows read back as bf16. Codes and scales are those of kv8.h; a key is coded
// from its turned dims in fp32, not from their bf16.
//
// The append has the workgroups of the bf16 one: a row's query heads, or one KV head
// of a tile of consecutive rows through LDS, D / 8 lanes a head's token. A block keeps
// [d / 16][16 tokens][16 dims] of K and [d][16 tokens] of V, so that 16 bytes are a
// token's 16 dims, or a dim's 16 tokens, and the scales of a block's K and V are one
// line of 128 bytes. Bound by HBM for prompts (about 8200 rows of 64 and 8 heads of 128: 65 us
// the append, 319 MB at 4.9 TB/s, 16 us the reading back, 51 MB at 3.1), by latency for a token each
// (256 rows with QK-norm 13.5 and 8.5 us, 8 small ones 5 and 4). The bf16 append of 256 rows takes
// 8: here a token by itself goes through the largest of its dims and the list of pieces
// as a prompt's do; which of them makes the difference was not measured. int8 takes the same times, its
// divisions included.
#include "common.h"
#include "internal.h"
#include "kv8.h"
#include "rope_rows.h"

namespace sidp {

namespace {

// Rows of a tile: as in the bf16 append, whose source and queries are the larger part of this one's bytes too.
constexpr int kLongTile = 64, kShortTile = 16;
constexpr int kLongRows = 2048;
int tile_of(int rows) { return rows >= kLongRows ? kLongTile : kShortTile; }

// Runs of rows whose slots follow each other in one block: first row | rows << 16, in s_piece[0 .. count). By the first wave.
template <int TILE>
__device__ __forceinline__ void list_pieces(const int* s_slot, int* s_piece, int* count) {
  const int t = threadIdx.x;
  if (t >= 64) return;
  const int slot = t < TILE ? s_slot[t] : -1;
  const bool starts = slot >= 0 && (t == 0 || slot % kBlockTokens == 0 || s_slot[t - 1] != slot - 1);
  const uint64_t who = __ballot(starts);
  if (starts) {
    int len = 1;
    while (t + len < TILE && (slot + len) % kBlockTokens != 0 && s_slot[t + len] == slot + len) len++;
    s_piece[__popcll(who & ((1ull << t) - 1))] = t | len << 16;
  }
  if (t == 0) *count = __popcll(who);
}

// The largest magnitude's bits of a head's dims, on each of its D / 8 lanes.
template <int D>
__device__ __forceinline__ uint32_t head_most(const float (&x)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
  for (int o = D / 16; o >= 1; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
  return m;
}

template <int D, int TYPE, bool INTERLEAVED, int TILE>
__global__ void __launch_bounds__(256) k_rope_rows8(RopeRows8Call c, int tiles) {
  constexpr int kLanes = D / 8, kRows = 256 / kLanes;  // rows of a pass
  constexpr int kRow = D + 16;                         // bytes of a row in LDS
  __shared__ __attribute__((aligned(16))) uint8_t s_x[TILE * kRow];
  __shared__ float s_scale[TILE];
  __shared__ int s_slot[TILE], s_piece[TILE], s_pieces;
  const int rows = c.row_count ? min(c.rows, *c.row_count) : c.rows;
  const int hkv = c.kv.hkv, t = threadIdx.x;
  const int kv_groups = tiles * hkv;
  if ((int)blockIdx.x >= 2 * kv_groups) {
    const int row = blockIdx.x - 2 * kv_groups;
    if (row < rows) query_row<D, INTERLEAVED, TILE == kLongTile>(c, row);
    return;
  }
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
#pragma unroll
  for (int i = 0; i < TILE; i += kRows) {
    const int r = i + t / kLanes;
    if (r < n) {
      float x[8], y[8];
      if (value) {
        load8<true>(src + (int64_t)r * c.stride + sub * 8, y);
      } else {
        const int pos = min(max(c.positions[row0 + r], 0), c.max_seq - 1);
        Turn turn;
        load_turn(c.rope_cos + (int64_t)pos * (D / 2), c.rope_sin + (int64_t)pos * (D / 2), c.rot, INTERLEAVED, t & 63, sub, turn);
        load_head<D>(src + (int64_t)r * c.stride, c.g_k, c.qk_eps, sub, x);
        turn_dims<INTERLEAVED>(x, turn, y);
      }
      const float scale = kv8_scale<TYPE>(head_most<D>(y));
      *(u32x2_t*)(s_x + r * kRow + sub * 8) =
          u32x2_t{kv8_codes<TYPE>(y[0], y[1], y[2], y[3], scale), kv8_codes<TYPE>(y[4], y[5], y[6], y[7], scale)};
      if (sub == 0) s_scale[r] = scale;
    }
  }
  __syncthreads();
  const int64_t region = (int64_t)c.region * c.kv.nblk;
  auto place_of = [&](int slot) { return (region + slot / kBlockTokens) * hkv + head; };  // the block, of this head
  if (t < n && s_slot[t] >= 0)
    c.kv8.scales[place_of(s_slot[t]) * (2 * kBlockTokens) + (value ? kBlockTokens : 0) + s_slot[t] % kBlockTokens] = s_scale[t];
  if (!value) {
    // a thread a (token, 16 dims) piece, tokens fastest: 16 tokens of a block are 256 bytes
    for (int i = t; i < TILE * (D / 16); i += 256) {
      const int r = i / D * 16 + i % 16, d16 = i / 16 % (D / 16);
      const int slot = s_slot[r];
      if (slot >= 0)
        *(u32x4_t*)(c.kv8.k + place_of(slot) * (int64_t)(D * kBlockTokens) + (d16 * kBlockTokens + slot % kBlockTokens) * 16) =
            *(const u32x4_t*)(s_x + r * kRow + d16 * 16);
    }
    return;
  }
  list_pieces<TILE>(s_slot, s_piece, &s_pieces);
  __syncthreads();
  // a dim's tokens of a piece a thread: whole words where there are any
  for (int i = t; i < s_pieces * D; i += 256) {
    const int r = s_piece[i / D] & 0xffff, len = s_piece[i / D] >> 16, d = i % D, slot = s_slot[r];
    const int lo = slot % kBlockTokens, hi = lo + len;
    uint8_t* to = c.kv8.v + place_of(slot) * (int64_t)(D * kBlockTokens) + d * kBlockTokens;
    const uint8_t* from = s_x + r * kRow + d - lo * kRow;  // of the block's first token
    u32x4_t v;
#pragma unroll
    for (int w = 0; w < 4; w++) {
      uint32_t word = 0;
#pragma unroll
      for (int k = 4 * w; k < 4 * w + 4; k++)
        if (k >= lo && k < hi) word |= (uint32_t)from[k * kRow] << 8 * (k % 4);
      v[w] = word;
    }
    if (len == kBlockTokens) {
      *(u32x4_t*)to = v;
      continue;
    }
#pragma unroll
    for (int w = 0; w < 4; w++) {
      if (4 * w >= lo && 4 * w + 4 <= hi) {
        *(uint32_t*)(to + 4 * w) = v[w];
      } else {
#pragma unroll
        for (int k = 4 * w; k < 4 * w + 4; k++)
          if (k >= lo && k < hi) to[k] = (uint8_t)(v[w] >> 8 * (k % 4));
      }
    }
  }
}

// One KV head's K or V of a tile of rows, back to [row][head][d] in bf16.
template <int D, int TYPE>
__global__ void __launch_bounds__(256) k_kv8_read(Kv8ReadCall c) {
  constexpr int TILE = kShortTile, kRow = D + 16;
  __shared__ __attribute__((aligned(16))) uint8_t s_x[TILE * kRow];
  __shared__ float s_scale[TILE];
  __shared__ int s_slot[TILE], s_piece[TILE], s_pieces;
  const int rows = c.row_count ? min(c.rows, *c.row_count) : c.rows;
  const int hkv = c.kv8.hkv, t = threadIdx.x;
  const bool value = blockIdx.y;
  uint16_t* out = value ? c.v_out : c.k_out;
  const int row0 = blockIdx.x / hkv * TILE, head = blockIdx.x % hkv;
  const int n = min(TILE, rows - row0);
  if (!out || n <= 0) return;
  const int64_t region = (int64_t)c.region * c.kv8.nblk;
  auto place_of = [&](int slot) { return (region + slot / kBlockTokens) * hkv + head; };
  if (t < TILE) {
    int slot = t < n ? c.slots[row0 + t] : -1;
    if (slot >= 0 && slot / kBlockTokens >= c.kv8.nblk) {
      atomicOr(c.err, SIDP_DEVERR_BLOCK);
      slot = -1;
    }
    s_slot[t] = slot;
    if (slot >= 0) s_scale[t] = c.kv8.scales[place_of(slot) * (2 * kBlockTokens) + (value ? kBlockTokens : 0) + slot % kBlockTokens];
  }
  __syncthreads();
  if (value) {
    list_pieces<TILE>(s_slot, s_piece, &s_pieces);
    __syncthreads();
    // a dim's 16 tokens of a piece's block a thread
    for (int i = t; i < s_pieces * D; i += 256) {
      const int r = s_piece[i / D] & 0xffff, len = s_piece[i / D] >> 16, d = i % D, slot = s_slot[r];
      const u32x4_t v = *(const u32x4_t*)(c.kv8.v + place_of(slot) * (int64_t)(D * kBlockTokens) + d * kBlockTokens);
      const int lo = slot % kBlockTokens;
#pragma unroll
      for (int k = 0; k < kBlockTokens; k++)
        if (k >= lo && k < lo + len) s_x[(r + k - lo) * kRow + d] = (uint8_t)(v[k / 4] >> 8 * (k % 4));
    }
    __syncthreads();
  }
  // a row's 16 dims a thread, from LDS or from the cache
  auto put = [&](auto from) {
    for (int i = t; i < TILE * (D / 16); i += 256) {
      const int r = i / (D / 16), d16 = i % (D / 16), slot = s_slot[r];
      if (slot < 0) continue;
      const u32x4_t w = from(r, d16, slot);
      const float scale = s_scale[r];
      u32x4_t o[2];
#pragma unroll
      for (int k = 0; k < 4; k++) {
        float x[4];
        kv8_values<TYPE>(w[k], x);
        o[k / 2][k % 2 * 2] = pack_bf2(x[0] * scale, x[1] * scale);
        o[k / 2][k % 2 * 2 + 1] = pack_bf2(x[2] * scale, x[3] * scale);
      }
      uint16_t* to = out + ((int64_t)(row0 + r) * hkv + head) * D + d16 * 16;
      *(u32x4_t*)to = o[0];
      *(u32x4_t*)(to + 8) = o[1];
    }
  };
  if (value) {
    put([&](int r, int d16, int) { return *(const u32x4_t*)(s_x + r * kRow + d16 * 16); });
  } else {
    put([&](int, int d16, int slot) {
      return *(const u32x4_t*)(c.kv8.k + place_of(slot) * (int64_t)(D * kBlockTokens) + (d16 * kBlockTokens + slot % kBlockTokens) * 16);
    });
  }
}

int64_t groups_of(int rows, int hkv) {
  const int tile = tile_of(rows);
  return 2 * (int64_t)((rows + tile - 1) / tile) * hkv + rows;
}

template <int D, int TYPE, bool INTERLEAVED>
hipError_t launch_append(const RopeRows8Call& c, hipStream_t s) {
  const int tile = tile_of(c.rows), tiles = (c.rows + tile - 1) / tile;
  const unsigned grid = (unsigned)groups_of(c.rows, c.kv.hkv);
  if (tile == kLongTile) k_rope_rows8<D, TYPE, INTERLEAVED, kLongTile><<<grid, 256, 0, s>>>(c, tiles);
  else k_rope_rows8<D, TYPE, INTERLEAVED, kShortTile><<<grid, 256, 0, s>>>(c, tiles);
  return hipGetLastError();
}
template <int D>
hipError_t launch_append_d(const RopeRows8Call& c, hipStream_t s) {
  if (c.kv8.type == kE4m3) return c.interleaved ? launch_append<D, kE4m3, true>(c, s) : launch_append<D, kE4m3, false>(c, s);
  return c.interleaved ? launch_append<D, kInt8, true>(c, s) : launch_append<D, kInt8, false>(c, s);
}
int64_t read_groups(int rows, int hkv) { return (int64_t)((rows + kShortTile - 1) / kShortTile) * hkv; }
template <int D>
hipError_t launch_read_d(const Kv8ReadCall& c, hipStream_t s) {
  const dim3 grid((unsigned)read_groups(c.rows, c.kv8.hkv), 2);
  if (c.kv8.type == kE4m3) k_kv8_read<D, kE4m3><<<grid, 256, 0, s>>>(c);
  else k_kv8_read<D, kInt8><<<grid, 256, 0, s>>>(c);
  return hipGetLastError();
}

}  // namespace

// HIP's launches have fewer than 2^32 threads a dimension: half of them here.
bool kv8_read_fits(int rows, int hkv) { return read_groups(rows, hkv) * 256 <= (int64_t)1 << 31; }

hipError_t launch_rope_rows8(const RopeRows8Call& c, hipStream_t s) {
  if (c.rows <= 0) return hipSuccess;
  return c.kv.d == 128 ? launch_append_d<128>(c, s) : launch_append_d<64>(c, s);
}

hipError_t launch_kv8_read(const Kv8ReadCall& c, hipStream_t s) {
  if (c.rows <= 0) return hipSuccess;
  return c.kv8.d == 128 ? launch_read_d<128>(c, s) : launch_read_d<64>(c, s);
}

}  // namespace sidp
