// Causal grouped-query attention of several new tokens a sequence over the paged
// KV cache: row i of sequence b sees keys 0 .. ctx_b + i.
//
// A tile is the (token, query head) pairs of up to kTileRows rows that share one KV
// head of one sequence; a workgroup takes a tile over a run of 64-token chunks. K
// and V chunks are staged in LDS (double-buffered: the next chunk's loads are in
// flight while this one computes), every wave holds 32 (token, head) pairs as the
// MFMA's columns:
//   S^T[token][pair] = K[token][:] . Q^T[:][pair]   (v_mfma_f32_32x32x16_bf16)
//   O^T[dim][pair]  += V^T[dim][token] . P[token][pair]
// so a pair's scores lie in two lanes and its softmax needs one exchange between
// them. The tokens of S^T's rows are permuted (bits 2 and 3 of a token's place in
// its block change places) so that the eight probabilities a lane needs for the
// second product are the ones it computed. Softmax is online in base-2 units; the
// reference only moves when a score is more than 2^kLazy above it (fp32 sums have
// the room), which leaves the accumulators alone in most chunks.
//
// P is rounded to bf16 for the second product: at most 2^-8 relative and independent from
// key to key, so the sum is off by no more than its own rounding to bf16; the
// sum of P is fp32 and unrounded.
#include "common.h"
#include "internal.h"

namespace sidp {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kChunk = 64;        // tokens staged at a time
constexpr int kChunkBlocks = kChunk / kBlockTokens;
constexpr float kLazy = 8.f;
constexpr int kWaves = 4;

// Items (entry, KV head) the chip holds at once: two workgroups a CU.
constexpr int kSlotsPerCu = 2;
// A launch with fewer items than slots cuts sequences into runs of at least this many chunks.
constexpr int kMinRun = 8;

typedef const __attribute__((address_space(4))) int32_t cint32_t;

struct Entry {
  int b, tile;
  int run;  // first chunk | chunks << 16
  int rec;  // record of a cut tile, -1 for a whole one
};
struct Cut {
  int b, tile, parts, rec;
};

// Workspace: counts, entries, cut tiles, records (o [rows][D], then m and l of each row).
struct Layout {
  int pairs_cap;                     // entries
  int cuts_cap, recs_cap, rec_rows;  // cut tiles, records, rows of a record
  size_t entries, cuts, recs, bytes;
};

__host__ __device__ inline int tile_tokens(int group, int tile_rows) { return tile_rows / group; }

Layout layout_of(int batch, int max_rows, int hq, int hkv, int d, int max_seq, int num_cus, int tile_rows) {
  const int group = hq / hkv, tm = tile_tokens(group, tile_rows), slots = kSlotsPerCu * std::max(1, num_cus);
  Layout l;
  const int tiles = (int)std::min<int64_t>(max_rows, (int64_t)max_rows / tm + std::min(batch, max_rows));
  const int runs = (max_seq + kChunk * kMinRun - 1) / (kChunk * kMinRun);
  l.cuts_cap = std::min(tiles, slots / hkv + 1);
  // a run is at least total / slots chunks: at most slots runs more than tiles
  l.recs_cap = (int)std::min<int64_t>((int64_t)l.cuts_cap * runs, l.cuts_cap + slots / hkv + 1);
  l.pairs_cap = std::max(tiles, l.recs_cap);
  l.rec_rows = std::min(tm, max_rows) * group;
  size_t o = 64;
  auto place = [&](size_t n) {
    const size_t at = o;
    o = (o + n + 255) / 256 * 256;
    return at;
  };
  l.entries = place((size_t)l.pairs_cap * sizeof(Entry));
  l.cuts = place((size_t)l.cuts_cap * sizeof(Cut));
  l.recs = place((size_t)l.recs_cap * hkv * l.rec_rows * (d + 2) * sizeof(float));
  l.bytes = o;
  return l;
}

// Lists the tiles, longest run first, so that the launch ends evenly.
__global__ void __launch_bounds__(1024) k_attn_rows_plan(AttnRowsCall c, Layout lay, int tile_rows) {
  extern __shared__ int32_t s_first[];  // [batch + 1] first tile of each sequence
  __shared__ int s_scan[16], s_longest[16];
  __shared__ long long s_total[16];
  __shared__ int s_hist[256];
  __shared__ int s_cuts, s_recs;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int group = c.hq / c.kv.hkv, tm = tile_tokens(group, tile_rows);
  const int slots = kSlotsPerCu * max(1, c.num_cus);
  char* ws = (char*)c.ws;
  int32_t* counts = (int32_t*)ws;
  Entry* entries = (Entry*)(ws + lay.entries);
  Cut* cuts = (Cut*)(ws + lay.cuts);
  // rows of a sequence; none (and an error) for starts or lengths that the call does not cover
  uint32_t bad = 0;
  auto rows_of = [&](int b) {
    const int r0 = c.row_starts[b], r1 = c.row_starts[b + 1], ctx = c.ctx_lens[b];
    if (r0 < 0 || r1 < r0 || r1 > c.max_rows || ctx < 0 || (int64_t)ctx + (r1 - r0) > (int64_t)c.max_blocks * kBlockTokens ||
        (int64_t)ctx + (r1 - r0) > c.max_seq) {
      bad = SIDP_DEVERR_POSITION;
      return 0;
    }
    return r1 - r0;
  };
  const int per = (c.batch + 1023) / 1024;
  const int b0 = min(t * per, c.batch), b1 = min(b0 + per, c.batch);
  int mine = 0;
  for (int b = b0; b < b1; b++) mine += (rows_of(b) + tm - 1) / tm;
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(incl, o, 64);
    if (lane >= o) incl += v;
  }
  if (lane == 63) s_scan[wave] = incl;
  if (t < 256) s_hist[t] = 0;
  if (t == 0) s_cuts = s_recs = 0;
  __syncthreads();
  int at = incl - mine;
  for (int w = 0; w < wave; w++) at += s_scan[w];
  for (int b = b0; b < b1; b++) {
    s_first[b] = at;
    at += (rows_of(b) + tm - 1) / tm;
  }
  int tiles = 0;
  for (int w = 0; w < 16; w++) tiles += s_scan[w];
  if (t == 0) s_first[c.batch] = tiles;
  if (bad) atomicOr(c.err, bad);
  __syncthreads();
  // tile i: its sequence, place in it and chunks
  auto tile_of = [&](int i, int& b, int& tile) {
    int lo = 0, hi = c.batch;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_first[mid] <= i) lo = mid;
      else hi = mid;
    }
    b = lo;
    tile = i - s_first[lo];
    const int n = c.row_starts[b + 1] - c.row_starts[b];
    return (c.ctx_lens[b] + min(n, (tile + 1) * tm) + kChunk - 1) / kChunk;
  };
  tiles = min(tiles, lay.pairs_cap);  // row starts that overlap could list more
  long long total = 0;
  int longest = 0;
  for (int i = t; i < tiles; i += 1024) {
    int b, tile;
    const int n = tile_of(i, b, tile);
    total += n;
    longest = max(longest, n);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    total += __shfl_xor(total, o, 64);
    longest = max(longest, __shfl_xor(longest, o, 64));
  }
  if (lane == 0) {
    s_total[wave] = total;
    s_longest[wave] = longest;
  }
  __syncthreads();
  total = 0;
  for (int w = 0; w < 16; w++) {
    total += s_total[w];
    longest = max(longest, s_longest[w]);
  }
  // fewer items than slots: runs of an even share, at least kMinRun chunks
  int run = max(longest, 1);
  if ((int64_t)tiles * c.kv.hkv < slots && tiles <= lay.cuts_cap) {
    const int share = (int)((total * c.kv.hkv + slots - 1) / slots);
    run = min(run, max(share, kMinRun));
  }
  auto bucket = [&](int n) { return 255 - (int)((int64_t)n * 255 / run); };
  for (int i = t; i < tiles; i += 1024) {
    int b, tile;
    const int n = tile_of(i, b, tile);
    if (n / run) atomicAdd(&s_hist[bucket(run)], n / run);
    if (n % run) atomicAdd(&s_hist[bucket(n % run)], 1);
  }
  __syncthreads();
  if (t < 64) {
    // exclusive prefix of the 256 buckets, four a lane
    int h[4], sum = 0;
    for (int j = 0; j < 4; j++) {
      h[j] = sum;
      sum += s_hist[4 * t + j];
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(inc, o, 64);
      if (lane >= o) inc += v;
    }
    for (int j = 0; j < 4; j++) s_hist[4 * t + j] = inc - sum + h[j];
    if (t == 63) counts[0] = inc;
  }
  __syncthreads();
  // Within a bucket the order is whatever the atomics give; entries write places of their own, so results do not depend on it.
  for (int i = t; i < tiles; i += 1024) {
    int b, tile;
    const int n = tile_of(i, b, tile);
    const int parts = (n + run - 1) / run;
    int rec = -1;
    if (parts > 1) {
      rec = atomicAdd(&s_recs, parts);
      cuts[atomicAdd(&s_cuts, 1)] = Cut{b, tile, parts, rec};
    }
    for (int p = 0; p < parts; p++) {
      const int len = min(run, n - p * run);
      entries[atomicAdd(&s_hist[bucket(len)], 1)] = Entry{b, tile, p * run | len << 16, parts > 1 ? rec + p : -1};
    }
  }
  __syncthreads();
  if (t == 0) counts[1] = s_cuts;
}

__device__ __forceinline__ uint32_t keep_finite(uint32_t v) {
  const uint32_t lo = (v & 0x7f80u) == 0x7f80u ? 0u : v & 0xffffu;
  const uint32_t hi = (v & 0x7f800000u) == 0x7f800000u ? 0u : v & 0xffff0000u;
  return lo | hi;
}
__device__ __forceinline__ bool any_not_finite(uint32_t v) {
  return (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
}
// bf16 ones where the value is +inf (which 0), -inf (1), NaN (2)
__device__ __forceinline__ uint32_t ones_where(uint32_t v, int which) {
  auto is = [&](uint32_t h) {
    return which == 0 ? h == 0x7f80u : which == 1 ? h == 0xff80u : (h & 0x7fffu) > 0x7f80u;
  };
  return (is(v & 0xffffu) ? 0x3f80u : 0u) | (is(v >> 16) ? 0x3f800000u : 0u);
}

// NR: 32-pair column sets of a wave.
template <int D, int NR>
__global__ void __launch_bounds__(256, NR == 1 ? 2 : 1) k_attn_rows(AttnRowsCall c, Layout lay) {
  constexpr int KK = D / 16, DT = D / 32;
  constexpr int kBlockBytes = kBlockTokens * D * 2;
  constexpr int kHalf = D * 16 + 128;  // V block in LDS: [token / 8][d][token % 8], halves 128 bytes apart in the banks
  constexpr int kVBlock = 2 * kHalf;
  constexpr int kKBytes = kChunkBlocks * kBlockBytes, kBuf = kKBytes + kChunkBlocks * kVBlock;
  constexpr int kPieces = kKBytes / 16 / 256;  // 16-byte pieces of K (and of V) that a thread stages
  constexpr int kPerBlock = kBlockBytes / 16;
  constexpr int kTileRows = 32 * NR * kWaves;
  extern __shared__ __attribute__((aligned(16))) char smem[];  // two buffers
  __shared__ int s_flag[2];

  const int t = threadIdx.x, lane = t & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const char* ws = (const char*)c.ws;
  const int hkv = c.kv.hkv, group = c.hq / hkv, tm = tile_tokens(group, kTileRows);
  const int item = blockIdx.x;
  if (item >= ((cint32_t*)ws)[0] * hkv) return;
  cint32_t* ep = (cint32_t*)(ws + lay.entries) + (item / hkv) * 4;
  const int g = item % hkv;
  const int b = ep[0], tile = ep[1], c0 = ep[2] & 0xffff, c1 = c0 + (ep[2] >> 16), rec = ep[3];
  const int row0 = ((cint32_t*)c.row_starts)[b] + tile * tm;
  const int tokens = min(tm, ((cint32_t*)c.row_starts)[b + 1] - row0);  // of this tile
  const int first_pos = ((cint32_t*)c.ctx_lens)[b] + tile * tm;         // of its first row
  const int kv_end = first_pos + tokens;
  cint32_t* bt = (cint32_t*)(c.block_tables + (int64_t)b * c.max_blocks);
  const int64_t region_blk = (int64_t)c.region * c.kv.nblk;
  const float scale = kLog2e / sqrtf((float)D);
  if (t < 2) s_flag[t] = -1;

  // this lane's pairs, their queries, and the keys they see
  bf16x8_t q[NR][KK];
  int limit[NR];
  int64_t out_row[NR];
#pragma unroll
  for (int n = 0; n < NR; n++) {
    const int pair = (wave * NR + n) * 32 + col;
    const int tok = pair / group, head = pair - tok * group;
    const bool live = tok < tokens;  // pairs past tm * group have tok >= tm
    limit[n] = live ? first_pos + tok + 1 : 0;
    out_row[n] = live ? (int64_t)(row0 + tok) * c.hq + g * group + head : -1;
    const uint16_t* qp = c.q + (live ? out_row[n] : (int64_t)row0 * c.hq + g * group) * D + half * 8;
#pragma unroll
    for (int kk = 0; kk < KK; kk++) q[n][kk] = as_bf16x8(*(const u32x4_t*)(qp + kk * 16));
  }
  // pairs of a wave are in token order: the fewest and the most keys that its pairs see
  const int wave_first = wave * NR * 32 / group;
  const bool wave_live = wave_first < tokens;
  const int wave_least = first_pos + wave_first + 1;
  const int wave_most = first_pos + min(tokens, (wave * NR * 32 + NR * 32 - 1) / group + 1);

  f32x16_t o[NR][DT];
  float m_ref[NR], l[NR];
#pragma unroll
  for (int n = 0; n < NR; n++) {
    m_ref[n] = -INFINITY;
    l[n] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; dt++)
#pragma unroll
      for (int r = 0; r < 16; r++) o[n][dt][r] = 0.f;
  }

  u32x4_t sk[kPieces], sv[kPieces];
  bool bad = false;
  // Loads chunk `ch` into registers; blocks past kv_end are zeros, as is the V of tokens past it (anything may stand there).
  auto load = [&](int ch) {
#pragma unroll
    for (int j = 0; j < kPieces; j++) {
      const int blk_in = kPerBlock >= 256 ? j : __builtin_amdgcn_readfirstlane(j * (256 / kPerBlock) + t / kPerBlock);
      const int piece = kPerBlock >= 256 ? t : t % kPerBlock;
      const int t0 = ch * kChunk + blk_in * kBlockTokens;
      sk[j] = sv[j] = u32x4_t{0, 0, 0, 0};
      if (t0 < kv_end) {
        const int blk = bt[t0 / kBlockTokens];
        if (blk >= 0 && blk < c.kv.nblk) {
          const int64_t off = ((region_blk + blk) * hkv + g) * (int64_t)kBlockBytes + piece * 16;
          sk[j] = *(const u32x4_t*)((const char*)c.kv.k + off);
          sv[j] = *(const u32x4_t*)((const char*)c.kv.v + off);
        } else {
          bad = true;
        }
      }
    }
  };
  // The V checks: only a chunk that the tile's first row does not see whole can hold masked tokens.
  auto store = [&](int ch, int buf) {
    char* kb = smem + buf * kBuf;
    char* vb = kb + kKBytes;
    const bool edge = (ch + 1) * kChunk > first_pos + 1;
#pragma unroll
    for (int j = 0; j < kPieces; j++) {
      const int blk_in = kPerBlock >= 256 ? j : j * (256 / kPerBlock) + t / kPerBlock;
      const int piece = kPerBlock >= 256 ? t : t % kPerBlock;
      if (edge) {
        const int t0 = ch * kChunk + blk_in * kBlockTokens + (piece & 1) * 8;
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 4; i++) {
          if (t0 + 2 * i >= kv_end) sv[j][i] = 0;
          else if (t0 + 2 * i + 1 >= kv_end) sv[j][i] &= 0xffffu;
          odd |= any_not_finite(sv[j][i]);
        }
        if (odd) s_flag[buf] = ch;
      }
      *(u32x4_t*)(kb + blk_in * kBlockBytes + piece * 16) = sk[j];
      *(u32x4_t*)(vb + blk_in * kVBlock + (piece & 1) * kHalf + (piece >> 1) * 16) = sv[j];
    }
  };

  __syncthreads();
  load(c0);
  store(c0, 0);
  __syncthreads();
  // K: the token of S^T's row m is m with bits 2 and 3 exchanged
  const int ktok = (col & 3) | ((col >> 2) & 1) << 3 | ((col >> 3) & 1) << 2;
  const int k_lane = (col >> 4) * kBlockBytes + (half * 16 + ktok) * 16;
  const int v_lane = half * kHalf + col * 16;
  for (int ch = c0; ch < c1; ch++) {
    const int buf = (ch - c0) & 1;
    if (ch + 1 < c1) load(ch + 1);
    const char* kb = smem + buf * kBuf;
    const char* vb = kb + kKBytes;
    const int t0 = ch * kChunk;
    if (wave_live && t0 < wave_most) {
      f32x16_t s[NR][2];
#pragma unroll
      for (int n = 0; n < NR; n++)
#pragma unroll
        for (int tt = 0; tt < 2; tt++)
#pragma unroll
          for (int r = 0; r < 16; r++) s[n][tt][r] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; kk++)
#pragma unroll
        for (int tt = 0; tt < 2; tt++) {
          const bf16x8_t kf = as_bf16x8(*(const u32x4_t*)(kb + tt * 2 * kBlockBytes + kk * 512 + k_lane));
#pragma unroll
          for (int n = 0; n < NR; n++) s[n][tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[n][kk], s[n][tt], 0, 0, 0);
        }
      const bool edge = t0 + kChunk > wave_least;
      bf16x8_t p[NR][4];
      uint32_t seen[NR];  // edge: whether the pair sees the token of each of its 32 scores
#pragma unroll
      for (int n = 0; n < NR; n++) {
        // register r of S^T's tile tt holds token 32 tt + 16 (r / 8) + 8 half + r % 8
        if (edge) {
          seen[n] = 0;
#pragma unroll
          for (int tt = 0; tt < 2; tt++)
#pragma unroll
            for (int r = 0; r < 16; r++) {
              const bool sees = t0 + 32 * tt + 16 * (r / 8) + 8 * half + r % 8 < limit[n];
              seen[n] |= (uint32_t)sees << (16 * tt + r);
              s[n][tt][r] = sees ? s[n][tt][r] : -INFINITY;
            }
        }
        float cm = s[n][0][0];
#pragma unroll
        for (int tt = 0; tt < 2; tt++)
#pragma unroll
          for (int r = 0; r < 16; r++) cm = fmaxf(cm, s[n][tt][r]);
        cm = fmaxf(cm, __shfl_xor(cm, 32, 64)) * scale;
        if (__any(cm > m_ref[n] + kLazy)) {
          const float m_new = fmaxf(m_ref[n], cm);
          const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_ref[n] - m_new);
          m_ref[n] = m_new;
          l[n] *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; dt++)
#pragma unroll
            for (int r = 0; r < 16; r++) o[n][dt][r] *= alpha;
        }
        const float base = m_ref[n] == -INFINITY ? 0.f : -m_ref[n];
        float sum = 0.f;
#pragma unroll
        for (int tt = 0; tt < 2; tt++) {
#pragma unroll
          for (int r = 0; r < 16; r++) {
            const float e = __builtin_amdgcn_exp2f(fmaf(s[n][tt][r], scale, base));
            s[n][tt][r] = e;
            sum += e;
          }
#pragma unroll
          for (int k = 0; k < 2; k++)
            p[n][2 * tt + k] = as_bf16x8(u32x4_t{pack_bf2(s[n][tt][8 * k], s[n][tt][8 * k + 1]), pack_bf2(s[n][tt][8 * k + 2], s[n][tt][8 * k + 3]),
                                                 pack_bf2(s[n][tt][8 * k + 4], s[n][tt][8 * k + 5]), pack_bf2(s[n][tt][8 * k + 6], s[n][tt][8 * k + 7])});
        }
        l[n] += sum;
      }
      if (edge && s_flag[buf] == ch) {
        // Values that are not finite, beside tokens that some pairs do not see: 0 * inf would reach those pairs. The finite
        // ones are multiplied as ever; the others are added where a pair sees them.
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
          for (int dt = 0; dt < DT; dt++) {
            const u32x4_t v = *(const u32x4_t*)(vb + k * kVBlock + v_lane + dt * 512);
            const bf16x8_t vf = as_bf16x8(u32x4_t{keep_finite(v[0]), keep_finite(v[1]), keep_finite(v[2]), keep_finite(v[3])});
#pragma unroll
            for (int n = 0; n < NR; n++) {
              o[n][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p[n][k], o[n][dt], 0, 0, 0);
              uint32_t w[4];
#pragma unroll
              for (int i = 0; i < 4; i++) {
                const uint32_t two = seen[n] >> (8 * k + 2 * i);
                w[i] = (two & 1u ? 0x3f80u : 0u) | (two & 2u ? 0x3f800000u : 0u);
              }
              const bf16x8_t sees = as_bf16x8(u32x4_t{w[0], w[1], w[2], w[3]});
              for (int which = 0; which < 3; which++) {
                const bf16x8_t of = as_bf16x8(u32x4_t{ones_where(v[0], which), ones_where(v[1], which), ones_where(v[2], which), ones_where(v[3], which)});
                f32x16_t cnt;
#pragma unroll
                for (int r = 0; r < 16; r++) cnt[r] = 0.f;
                cnt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(of, sees, cnt, 0, 0, 0);
                const float add = which == 0 ? INFINITY : which == 1 ? -INFINITY : NAN;
#pragma unroll
                for (int r = 0; r < 16; r++)
                  if (cnt[r] > 0.f) o[n][dt][r] += add;
              }
            }
          }
      } else {
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
          for (int dt = 0; dt < DT; dt++) {
            const bf16x8_t vf = as_bf16x8(*(const u32x4_t*)(vb + k * kVBlock + v_lane + dt * 512));
#pragma unroll
            for (int n = 0; n < NR; n++) o[n][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p[n][k], o[n][dt], 0, 0, 0);
          }
      }
    }
    if (ch + 1 < c1) store(ch + 1, buf ^ 1);
    __syncthreads();
  }
  if (bad) atomicOr(c.err, SIDP_DEVERR_BLOCK);

  // Register r of O^T's tile dt is dim 32 dt + 8 (r / 4) + 4 half + r % 4.
#pragma unroll
  for (int n = 0; n < NR; n++) {
    const float sum = l[n] + __shfl_xor(l[n], 32, 64);
    if (out_row[n] < 0) continue;
    if (rec < 0) {
      const float inv = 1.f / sum;
      uint16_t* op = c.out + out_row[n] * D + half * 4;
#pragma unroll
      for (int dt = 0; dt < DT; dt++)
#pragma unroll
        for (int i = 0; i < 4; i++)
          *(u32x2_t*)(op + dt * 32 + i * 8) = u32x2_t{pack_bf2(o[n][dt][4 * i] * inv, o[n][dt][4 * i + 1] * inv),
                                                      pack_bf2(o[n][dt][4 * i + 2] * inv, o[n][dt][4 * i + 3] * inv)};
    } else {
      const int pair = (wave * NR + n) * 32 + col;
      float* r = (float*)((char*)c.ws + lay.recs) + ((int64_t)rec * hkv + g) * lay.rec_rows * (D + 2);
#pragma unroll
      for (int dt = 0; dt < DT; dt++)
#pragma unroll
        for (int i = 0; i < 4; i++)
          *(f32x4_t*)(r + pair * D + dt * 32 + i * 8 + half * 4) =
              f32x4_t{o[n][dt][4 * i], o[n][dt][4 * i + 1], o[n][dt][4 * i + 2], o[n][dt][4 * i + 3]};
      if (half == 0) *(float2*)(r + (int64_t)lay.rec_rows * D + 2 * pair) = make_float2(m_ref[n], sum);
    }
  }
}

// Joins a cut tile's records in run order: one workgroup per (cut tile, KV head), four dims a thread.
template <int D>
__global__ void __launch_bounds__(256) k_attn_rows_join(AttnRowsCall c, Layout lay, int tile_rows) {
  const char* ws = (const char*)c.ws;
  if ((int)blockIdx.x >= ((const int32_t*)ws)[1]) return;
  const Cut cut = ((const Cut*)(ws + lay.cuts))[blockIdx.x];
  const int hkv = c.kv.hkv, g = blockIdx.y, group = c.hq / hkv, tm = tile_tokens(group, tile_rows);
  const int row0 = c.row_starts[cut.b] + cut.tile * tm;
  const int pairs = min(tm, c.row_starts[cut.b + 1] - row0) * group;
  const int64_t step = (int64_t)hkv * lay.rec_rows * (D + 2);
  const float* recs = (const float*)(ws + lay.recs) + ((int64_t)cut.rec * hkv + g) * lay.rec_rows * (D + 2);
  const float* ml = recs + (int64_t)lay.rec_rows * D;
  for (int i = threadIdx.x; i < pairs * (D / 4); i += 256) {
    const int pair = i / (D / 4), d = i % (D / 4) * 4;
    float M = -INFINITY;
    for (int p = 0; p < cut.parts; p++) M = fmaxf(M, ml[p * step + 2 * pair]);
    float L = 0.f;
    f32x4_t O = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < cut.parts; p++) {
      const float m = ml[p * step + 2 * pair];
      const f32x4_t v = *(const f32x4_t*)(recs + p * step + (int64_t)pair * D + d);
      // a run of which the pair sees nothing left zeros
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
      L = fmaf(ml[p * step + 2 * pair + 1], f, L);
      O += v * f;
    }
    const float inv = 1.f / L;
    const int64_t row = (int64_t)(row0 + pair / group) * c.hq + g * group + pair % group;
    *(u32x2_t*)(c.out + row * D + d) = u32x2_t{pack_bf2(O[0] * inv, O[1] * inv), pack_bf2(O[2] * inv, O[3] * inv)};
  }
}

constexpr int kNR = 1;

template <int D>
hipError_t launch_d(const AttnRowsCall& c, hipStream_t s) {
  constexpr int kTileRows = 32 * kNR * kWaves;
  const Layout lay = layout_of(c.batch, c.max_rows, c.hq, c.kv.hkv, D, c.max_seq, c.num_cus, kTileRows);
  k_attn_rows_plan<<<1, 1024, (size_t)(c.batch + 1) * sizeof(int32_t), s>>>(c, lay, kTileRows);
  const size_t lds = 2 * (size_t)(kChunkBlocks * (kBlockTokens * D * 2 + 2 * (D * 16 + 128)));
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)k_attn_rows<D, kNR>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  k_attn_rows<D, kNR><<<(unsigned)((int64_t)lay.pairs_cap * c.kv.hkv), 256, lds, s>>>(c, lay);
  k_attn_rows_join<D><<<dim3(lay.cuts_cap, c.kv.hkv), 256, 0, s>>>(c, lay, kTileRows);
  return hipGetLastError();
}

}  // namespace

size_t attn_rows_ws_bytes(int batch, int max_rows, int hq, int hkv, int d, int max_seq, int num_cus) {
  return layout_of(batch, max_rows, hq, hkv, d, max_seq, num_cus, 32 * kNR * kWaves).bytes;
}

hipError_t launch_attention_rows(const AttnRowsCall& c, hipStream_t s) {
  if (c.max_rows <= 0) return hipSuccess;
  return c.kv.d == 128 ? launch_d<128>(c, s) : launch_d<64>(c, s);
}

}  // namespace sidp
