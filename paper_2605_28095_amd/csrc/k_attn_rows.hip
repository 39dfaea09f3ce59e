// Causal grouped-query attention of several new tokens a sequence over the paged
// KV cache: row i of sequence b sees keys 0 .. ctx_b + i.
//
// A tile is the (token, query head) pairs of up to kTileRows rows that share one KV
// head of one sequence; a workgroup takes a tile over a run of 32-token chunks. K
// and V go straight to LDS, into rings of four chunks each (the next two or three are
// on their way while one is in use), and every wave holds 32 (token, head) pairs as
// the MFMA's columns:
//   S^T[token][pair] = K[token][:] . Q^T[:][pair]   (v_mfma_f32_32x32x16_bf16)
//   O^T[dim][pair]  += V^T[dim][token] . P[token][pair]
// so a pair's scores lie in two lanes and its softmax needs one exchange between
// them. The tokens of S^T's rows are permuted (bits 2 and 3 of a token's place in
// its block change places) so that the eight probabilities a lane needs for the
// second product are the ones it computed. Softmax is online in base-2 units. Its
// reference is a score of the pair, not always the largest: it only moves when a
// chunk's weights sum to more than kMost (fp32 and bf16 have the range), so that
// most chunks need no maximum and leave the accumulators alone. The next chunk's
// scores and the last one's values are on the matrix units while the vector units
// exponentiate this one's.
//
// Bound by the matrix units where rows are many: one prompt of 8192 rows, 64 and 8
// heads of 128 dims, 962-1039 us as the machine's power lets it, 1.06-1.14 PFLOP/s, where
// a library product of two 8192 x 8192 matrices reaches 1.22 (1444 with chunks staged
// through registers, 1183 straight to LDS, 1039 with the turns that every row sees whole
// run without checks, 975 on the same machine now). Eight ragged chunks of prompts
// 301-321 us, 1.01-1.08 PFLOP/s. By HBM where they are few: 16 sequences of 4 rows over
// up to 8191 tokens 69-70 us, of which 57 read the cache at 5.3 TB/s and the plan and the
// join of cut sequences take the rest.
//
// The second product takes P as bf16. In a sequence of one tile (drafted tokens, single
// ones: the calls that HBM bounds) P is cut and what the cut leaves is multiplied as well,
// as in the attention of the decode step, so that P has 16 bits. In longer ones it is rounded:
// the sum of P stays fp32 and unrounded, so a row is off by at most 2^-8 sum p |v| beside
// its own rounding, all of it to one side where scores are equal. Both sides: 16 x 4
// rows over 1-8K 67-68 us rounded, 69 in two parts; 16 rows over 30000 45 and 50; a prompt
// of 8192 rows 985 and 1373, eight chunks 318 and 432. Distance from 64 bits, normal
// keys, values and queries: 0.0022 of the norm rounded, 0.0016 in two parts, which is what
// the result's own rounding makes.
#include <type_traits>

#include "common.h"
#include "internal.h"

namespace sidp {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kChunk = 32;        // tokens staged at a time
constexpr int kRing = 4;          // chunks of K, and of V, in LDS
constexpr int kChunkBlocks = kChunk / kBlockTokens;
constexpr float kMost = 4096.f;
constexpr int kWaves = 4;
constexpr int kTileRows = 32 * kWaves;  // (token, head) pairs of a tile

// Items (entry, KV head) the chip holds at once: two workgroups a CU.
constexpr int kSlotsPerCu = 2;
// A launch with fewer items than slots cuts sequences into runs of at least this many chunks, and a tile into at most this many.
constexpr int kMinRun = 16, kMaxRuns = 32;
// Cutting writes and reads partial outputs, so only where the longest item is this much longer than the runs would be. Whole /
// cut, us a call on the 70B heads, longest item and run in chunks: 16 sequences of 32 rows over 500 cached 17, 16: 28 / 39; of 1 row
// over 1000 32, 16: 32 / 26; of 32 rows over 4000 126, 63: 96 / 98; 1 of 200 rows over 2000 69, 16: 49 / 39; 4 of 100 rows over
// 4000 129, 56: 82 / 80; 1 of 16 rows over 30000 939, 30: 480 / 46.
constexpr float kCutFrom = 1.75f;

typedef const __attribute__((address_space(4))) int32_t cint32_t;

struct Entry {
  int b, tile;
  uint32_t run;  // first chunk | chunks << 16, at most 2^15
  int rec;        // record of a cut tile, -1 for a whole one
};
struct Cut {
  int row0, pairs, parts, rec;
};

// Workspace: counts, entries, cut tiles, records (o [rows][D], then m and l of each row).
struct Layout {
  int tiles_cap, entries_cap;
  int cuts_cap, recs_cap, rec_rows;  // cut tiles, records, pairs of a record
  size_t entries, cuts, recs, bytes;
};

__host__ __device__ inline int tile_tokens(int group) { return kTileRows / group; }
// for one KV head's items
__host__ __device__ inline int slots_of(int num_cus, int hkv) { return kSlotsPerCu * (num_cus < 1 ? 1 : num_cus) / hkv; }

Layout layout_of(int batch, int max_rows, int hq, int hkv, int d, int max_seq, int num_cus) {
  const int group = hq / hkv, tm = tile_tokens(group), slots = slots_of(num_cus, hkv);
  Layout l;
  l.tiles_cap = (int)std::min<int64_t>(max_rows, (int64_t)max_rows / tm + std::min(batch, max_rows));
  l.cuts_cap = std::min(l.tiles_cap, std::max(slots - 1, 0));  // a call with more tiles is not cut
  // a run is at least kMinRun chunks, and the total over slots: at most slots runs more than tiles
  const int runs = (max_seq + kChunk * kMinRun - 1) / (kChunk * kMinRun);
  l.recs_cap = (int)std::min<int64_t>((int64_t)l.cuts_cap * runs, l.cuts_cap + slots);
  l.entries_cap = std::max(l.tiles_cap, l.recs_cap);
  l.rec_rows = std::min(tm, max_rows) * group;
  size_t o = 64;
  auto place = [&](size_t n) {
    const size_t at = o;
    o = (o + n + 255) / 256 * 256;
    return at;
  };
  l.entries = place((size_t)l.entries_cap * sizeof(Entry));
  l.cuts = place((size_t)l.cuts_cap * sizeof(Cut));
  l.recs = place((size_t)l.recs_cap * hkv * l.rec_rows * (d + 2) * sizeof(float));
  l.bytes = o;
  return l;
}

// Lists the items. One workgroup, a chain of latencies in front of the attention:
// lengths are read once, into LDS, and only as many waves work as there are
// sequences or tiles (16 sequences of 4 rows: 6 us; 9 with 16 waves).
//
// At least as many tiles as the chip holds at once: longest first, so that the
// launch ends evenly. Fewer: every tile is cut into even runs of at most `run`
// chunks, the shortest of kTries lengths between an even share of all chunks and one
// that cannot give more runs than fit (a tile's last run may be short: half a run
// a tile lies between the two).
constexpr int kTries = 8;
constexpr int kPlanWaves = 16;
__global__ void __launch_bounds__(64 * kPlanWaves) k_attn_rows_plan(AttnRowsCall c, Layout lay) {
  extern __shared__ int32_t s_lds[];
  int32_t* s_first = s_lds;                // [batch + 1] first tile of each sequence
  int32_t* s_ctx = s_first + c.batch + 1;  // [batch] cached tokens
  int32_t* s_rows = s_ctx + c.batch;       // [batch] rows
  __shared__ int s_scan[kPlanWaves], s_longest[kPlanWaves], s_parts[kPlanWaves];
  __shared__ uint32_t s_total[kPlanWaves];
  __shared__ int s_hist[256];
  __shared__ int s_items[kTries];
  __shared__ int s_base[64 * kPlanWaves];
  __shared__ int s_cuts;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, threads = blockDim.x, waves = threads / 64;
  const int group = c.hq / c.kv.hkv, tm = tile_tokens(group);
  const int slots = slots_of(c.num_cus, c.kv.hkv);
  char* ws = (char*)c.ws;
  int32_t* counts = (int32_t*)ws;
  Entry* entries = (Entry*)(ws + lay.entries);
  if (t < kTries) s_items[t] = 0;
  if (t == 0) s_cuts = 0;
  // a sequence whose starts or lengths the call does not cover has no rows
  bool bad = false;
  for (int b = t; b < c.batch; b += threads) {
    const int r0 = c.row_starts[b], r1 = c.row_starts[b + 1], ctx = c.ctx_lens[b];
    const bool ok = r0 >= 0 && r1 >= r0 && r1 <= c.max_rows && ctx >= 0 &&
                    (int64_t)ctx + (r1 - r0) <= (int64_t)min(c.max_blocks * kBlockTokens, c.max_seq);
    bad |= !ok;
    s_ctx[b] = ctx;
    s_rows[b] = ok ? r1 - r0 : 0;
  }
  if (bad) atomicOr(c.err, SIDP_DEVERR_POSITION);
  __syncthreads();
  // exclusive place of a thread's `mine` among all threads', and the sum
  auto scan = [&](int mine, int* s_sums, int& sum) {
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o, 64);
      if (lane >= o) incl += v;
    }
    if (lane == 63) s_sums[wave] = incl;
    __syncthreads();
    int at = incl - mine;
    sum = 0;
    for (int w = 0; w < waves; w++) {
      if (w < wave) at += s_sums[w];
      sum += s_sums[w];
    }
    return at;
  };
  const int per = (c.batch + threads - 1) / threads;
  const int b0 = min(t * per, c.batch), b1 = min(b0 + per, c.batch);
  int mine = 0, tiles;
  for (int b = b0; b < b1; b++) mine += (s_rows[b] + tm - 1) / tm;
  int at = scan(mine, s_scan, tiles);
  for (int b = b0; b < b1; b++) {
    s_first[b] = at;
    at += (s_rows[b] + tm - 1) / tm;
  }
  if (t == 0) s_first[c.batch] = tiles;
  __syncthreads();
  tiles = min(tiles, lay.tiles_cap);  // row starts that overlap could list more
  auto last_at = [](const int* s, int n, int i) {  // the last of s[0 .. n) that is at most i
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s[mid] <= i) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  // tile i: its sequence, place in it and chunks
  struct Tile {
    int b, place, chunks;
  };
  auto tile_of = [&](int i) {
    const int b = last_at(s_first, c.batch, i), place = i - s_first[b];
    return Tile{b, place, (s_ctx[b] + min(s_rows[b], (place + 1) * tm) + kChunk - 1) / kChunk};
  };
  if (tiles >= slots || tiles > lay.cuts_cap || tiles > threads) {
    // a counting sort by length, in 256 steps of the longest one's
    for (int i = t; i < 256; i += threads) s_hist[i] = 0;
    int longest = 1;
    for (int i = t; i < tiles; i += threads) longest = max(longest, tile_of(i).chunks);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) longest = max(longest, __shfl_xor(longest, o, 64));
    if (lane == 0) s_longest[wave] = longest;
    __syncthreads();
    for (int w = 0; w < waves; w++) longest = max(longest, s_longest[w]);
    auto bucket = [&](int n) { return 255 - n * 255 / longest; };
    for (int i = t; i < tiles; i += threads) atomicAdd(&s_hist[bucket(tile_of(i).chunks)], 1);
    __syncthreads();
    if (t < 64) {
      int h[4], sum = 0;
#pragma unroll
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
#pragma unroll
      for (int j = 0; j < 4; j++) s_hist[4 * t + j] = inc - sum + h[j];
    }
    __syncthreads();
    // Within a step the order is whatever the atomics give; items write places of their own, so results do not depend on it.
    for (int i = t; i < tiles; i += threads) {
      const Tile x = tile_of(i);
      entries[atomicAdd(&s_hist[bucket(x.chunks)], 1)] = Entry{x.b, x.place, (uint32_t)x.chunks << 16, -1};
    }
    if (t == 0) {
      counts[0] = tiles;
      counts[1] = 0;
    }
    return;
  }
  // a tile a thread at most
  const Tile own = t < tiles ? tile_of(t) : Tile{0, 0, 0};
  uint32_t total = own.chunks;
  int longest = own.chunks;
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
  for (int w = 0; w < waves; w++) {
    total += s_total[w];
    longest = max(longest, s_longest[w]);
  }
  int run = max(longest, 1);
  const int least = max(max((int)(total + slots - 1) / slots, kMinRun), (longest + kMaxRuns - 1) / kMaxRuns);
  if (longest >= kCutFrom * least) {
    const int most = max((int)(total + slots - tiles - 1) / (slots - tiles), least);
    auto try_of = [&](int j) { return least + (most - least) * j / (kTries - 1); };
    int n[kTries];
#pragma unroll
    for (int j = 0; j < kTries; j++) n[j] = (own.chunks + try_of(j) - 1) / try_of(j);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1)
#pragma unroll
      for (int j = 0; j < kTries; j++) n[j] += __shfl_xor(n[j], o, 64);
    if (lane == 0)
#pragma unroll
      for (int j = 0; j < kTries; j++) atomicAdd(&s_items[j], n[j]);
    __syncthreads();
    int j = 0;
    while (j < kTries - 1 && s_items[j] > slots) j++;
    run = min(run, try_of(j));
  }
  int runs;
  const int parts = (own.chunks + run - 1) / run, base = scan(parts, s_parts, runs);
  s_base[t] = base;
  if (parts > 1) {
    const int from = own.place * tm, rows = min(tm, s_rows[own.b] - from);
    ((Cut*)(ws + lay.cuts))[atomicAdd(&s_cuts, 1)] = Cut{c.row_starts[own.b] + from, rows * group, parts, base};
  }
  __syncthreads();
  for (int e = t; e < runs; e += threads) {
    const int i = last_at(s_base, tiles, e);
    const Tile x = tile_of(i);
    const int p = e - s_base[i], n = (x.chunks + run - 1) / run;
    const int lo = x.chunks * p / n, hi = x.chunks * (p + 1) / n;
    entries[e] = Entry{x.b, x.place, (uint32_t)lo | (uint32_t)(hi - lo) << 16, n > 1 ? e : -1};
  }
  if (t == 0) {
    counts[0] = runs;
    counts[1] = s_cuts;
  }
}

__device__ __forceinline__ uint32_t keep_finite(uint32_t v) {
  const uint32_t lo = (v & 0x7f80u) == 0x7f80u ? 0u : v & 0xffffu;
  const uint32_t hi = (v & 0x7f800000u) == 0x7f800000u ? 0u : v & 0xffff0000u;
  return lo | hi;
}
__device__ __forceinline__ bool any_not_finite(uint32_t v) {
  return (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
}
// 16 bytes a lane of a block (its address the same for the wave), straight to LDS: lane l's land at dst + 16 l. once: non-temporal,
// nothing is left in the caches. A buffer load: after a global one, which the compiler takes for a flat access, it waits for every
// LDS read instead of the one that is needed (a prompt of 8192 rows: 1013 us, so 975).
template <int BYTES>
__device__ __forceinline__ void load_lds16(const char* block, uint32_t offset, char* dst, bool once) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(block), (short)0, BYTES, 0x00020000);
  const auto to = (__attribute__((address_space(3))) void*)dst;
  if (once) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 16, offset, 0, 0, 2);
  else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 16, offset, 0, 0, 0);
}

// The larger of a lane's value and its counterpart's in the other half of the wave.
__device__ __forceinline__ float max_halves(float v) {
  const u32x2_t r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int D>
__global__ void __launch_bounds__(256, 2) k_attn_rows(AttnRowsCall c, Layout lay) {
  constexpr int KK = D / 16, DT = D / 32;
  constexpr int kBlockBytes = kBlockTokens * D * 2;
  constexpr int kSide = kChunkBlocks * kBlockBytes;  // K or V of a chunk
  constexpr int kBlockWaves = D / 32;                // waves that load a block's K (and V), 16 bytes a lane
  constexpr int kPieces = kChunkBlocks * kBlockWaves / kWaves;
  constexpr int kGroupChunks = 64 / kChunkBlocks;    // chunks whose block ids a wave holds, one a lane
  extern __shared__ __attribute__((aligned(16))) char smem[];  // the rings of K and of V
  __shared__ int s_odd;          // whether an edge chunk held values that are not finite
  __shared__ int s_first[3][D];  // and the first tokens that hold +inf, -inf and NaN, of each dim

  const int t = threadIdx.x, lane = t & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const char* ws = (const char*)c.ws;
  const int hkv = c.kv.hkv, group = c.hq / hkv, tm = tile_tokens(group);
  const int item = blockIdx.x;
  if (item >= ((cint32_t*)ws)[0] * hkv) return;
  cint32_t* ep = (cint32_t*)(ws + lay.entries) + (item / hkv) * 4;
  const int g = item % hkv;
  const int b = ep[0], tile = ep[1], c0 = ep[2] & 0xffff, c1 = c0 + (int)((uint32_t)ep[2] >> 16), rec = ep[3];
  const int seq0 = ((cint32_t*)c.row_starts)[b], seq_rows = ((cint32_t*)c.row_starts)[b + 1] - seq0;
  const int row0 = seq0 + tile * tm;
  const int tokens = min(tm, seq_rows - tile * tm);              // of this tile
  const int first_pos = ((cint32_t*)c.ctx_lens)[b] + tile * tm;  // of its first row
  // A sequence of one tile reads its keys and values once: loads that leave nothing in the caches reach more of HBM's rate (16
  // sequences of 4 rows 69 us, 77 without), but more tiles of a sequence share what one leaves there (8192 rows 1020 us, 1054).
  // Beside such loads there is time for P in two parts.
  const bool one_tile = seq_rows <= tm;
  const int kv_end = first_pos + tokens;
  const int blocks = (kv_end + kBlockTokens - 1) / kBlockTokens;
  const int32_t* bt = c.block_tables + (int64_t)b * c.max_blocks;
  const float scale = kLog2e / sqrtf((float)D);
  if (t == 0) s_odd = 0;
  for (int i = t; i < 3 * D; i += 256) (&s_first[0][0])[i] = 0x7fffffff;

  // this lane's pair, its query, and the keys it sees
  struct Pair {
    int at, tok, head;
  };
  auto pair_of = [&](int thread) {
    const int at = (thread >> 6) * 32 + (thread & 31), tok = at / group;
    return Pair{at, tok, at - tok * group};
  };
  const Pair own = pair_of(t);
  const bool live = own.tok < tokens;  // pairs past tm * group have tok >= tm
  const int limit = live ? first_pos + own.tok + 1 : 0;
  bf16x8_t q[KK];
  {
    const uint16_t* qp = c.q + ((int64_t)(row0 + (live ? own.tok : 0)) * c.hq + g * group + (live ? own.head : 0)) * D + half * 8;
#pragma unroll
    for (int kk = 0; kk < KK; kk++) q[kk] = as_bf16x8(*(const u32x4_t*)(qp + kk * 16));
  }
  // pairs of a wave are in token order: the fewest and the most keys that its pairs see
  const int wave_first = wave * 32 / group;
  const bool wave_live = wave_first < tokens;
  const int wave_least = first_pos + wave_first + 1;
  const int wave_most = wave_live ? first_pos + min(tokens, (wave * 32 + 31) / group + 1) : 0;

  f32x16_t o[DT];
  // A score x weighs 2^(x scale + base). `most`: the largest sum of a chunk's weights that leaves base alone; negative before there
  // is a reference, kMost from then on (and for lanes without a pair).
  float base = 0.f, most = live ? -1.f : kMost, l = 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++) o[dt][r] = 0.f;

  // Places in the cache (in blocks of one KV head) of 32 chunks' blocks, one a
  // lane, and the ids of the 32 behind them (loaded a group ahead: a wait for an id
  // would wait for the chunks in flight too). A block outside the cache is read as
  // block 0, one past the last block as the last.
  bool bad = false;
  auto load_ids = [&](int chunk) { return bt[min(chunk * kChunkBlocks + lane, blocks - 1)]; };
  const int place0 = c.region * c.kv.nblk;
  auto places = [&](int id) {
    const bool ok = id >= 0 && id < c.kv.nblk;
    bad |= !ok;
    return (place0 + (ok ? id : 0)) * hkv + g;
  };
  int at_k = places(load_ids(c0)), ids_next = load_ids(c0 + kGroupChunks), at_v = at_k;  // V is fetched two chunks later
  const int blk_wave = wave / kBlockWaves, in_block = wave % kBlockWaves;
  // K blocks go to LDS as they are; V blocks as [token / 8][d][token % 8], so that 32 dims' pieces are contiguous
  const uint32_t k_src = (in_block * 64 + lane) * 16;
  const uint32_t v_src = (in_block % (kBlockWaves / 2) * 64 + lane) * 32 + in_block / (kBlockWaves / 2) * 16;
  char* const mine = smem + blk_wave * kBlockBytes + in_block * 1024;  // this wave's first piece of a chunk
  auto fetch = [&](int n, int at, const void* cache, uint32_t src, char* to, bool once) {  // n: chunk counted from c0
#pragma unroll
    for (int j = 0; j < kPieces; j++) {
      const int from = j * (kWaves / kBlockWaves);
      const int place = __builtin_amdgcn_readlane(at, n % kGroupChunks * kChunkBlocks + from + blk_wave);
      load_lds16<kBlockBytes>((const char*)cache + (int64_t)place * kBlockBytes, src, to + from * kBlockBytes, once);
    }
  };
  auto fetch_k = [&](int n, int slot, bool once) {
    if (n > 0 && n % kGroupChunks == 0) {
      at_k = places(ids_next);
      ids_next = load_ids(c0 + n + kGroupChunks);
    }
    fetch(n, at_k, c.kv.k, k_src, mine + slot * kSide, once);
  };
  auto fetch_v = [&](int n, int slot, bool once) {
    if (n % kGroupChunks == 0) at_v = at_k;
    fetch(n, at_v, c.kv.v, v_src, mine + (kRing + slot) * kSide, once);
  };
  // Waits for the other waves, with no LDS operation of this one under way: what it read they may load over, what it wrote they
  // may change.
  auto meet = [&] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // Waits until this wave's loads but the last 4 * kPieces have landed (all, with `all`), then for the other waves.
  auto landed = [&](bool all) {
    if (all) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * kPieces) : "memory");
    meet();
  };
  // The V of an edge chunk (one that the tile's first row does not see whole), landed. Tokens past kv_end become zeros (anything
  // may stand there). So do values that are not finite, for 0 * inf would reach the rows that do not see them: they are added to
  // the others at the end, where an inf or a NaN is an inf or a NaN whenever it came.
  auto mend = [&](int ch) {
    if ((ch + 1) * kChunk <= first_pos + 1) return;
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));  // the addresses are made here rather than kept: no register is left for them
    char* vb = smem + (kRing + (ch - c0) % kRing) * kSide;
#pragma unroll 1
    for (int i = t; i < kSide / 16; i += 256) {
      const int t0 = ch * kChunk + i / (2 * D) * kBlockTokens + i / D % 2 * 8;
      u32x4_t v = *(const u32x4_t*)(vb + i * 16);
#pragma unroll
      for (int k = 0; k < 4; k++) {
        if (t0 + 2 * k >= kv_end) v[k] = 0;
        else if (t0 + 2 * k + 1 >= kv_end) v[k] &= 0xffffu;
      }
      if (any_not_finite(v[0]) || any_not_finite(v[1]) || any_not_finite(v[2]) || any_not_finite(v[3])) {
        s_odd = 1;
#pragma unroll 1
        for (int k = 0; k < 8; k++) {
          const uint32_t h = (k & 4 ? (k & 2 ? v[3] : v[2]) : (k & 2 ? v[1] : v[0])) >> 16 * (k & 1) & 0xffffu;
          if ((h & 0x7f80u) == 0x7f80u) atomicMin(&s_first[h == 0x7f80u ? 0 : h == 0xff80u ? 1 : 2][i % D], t0 + k);
        }
#pragma unroll
        for (int k = 0; k < 4; k++) v[k] = keep_finite(v[k]);
      }
      *(u32x4_t*)(vb + i * 16) = v;
    }
    meet();
  };

  // K: the token of S^T's row m is m with bits 2 and 3 exchanged
  const int ktok = (col & 3) | ((col >> 2) & 1) << 3 | ((col >> 3) & 1) << 2;
  const uint32_t k_lane = (col >> 4) * kBlockBytes + (half * 16 + ktok) * 16;
  const uint32_t v_lane = half * (D * 16) + col * 16;
  // Register r: token 16 (r / 8) + 8 half + r % 8 of the chunk.
  auto mask = [&](int ch, f32x16_t& s) {
    if ((ch + 1) * kChunk > wave_least) {
#pragma unroll
      for (int r = 0; r < 16; r++) s[r] = ch * kChunk + 16 * (r / 8) + 8 * half + r % 8 < limit ? s[r] : -INFINITY;
    }
  };
  // Eight weights as bf16: rounded, or cut (p[k]) and what the cut left (p[2 + k]). The second part gets 2^-23 of the weight more,
  // so that it is above zero where the weight is: an infinite value stays one in both products.
  auto to_bf16 = [&](auto parts, const float* e, bf16x8_t (&p)[4], int k) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if (decltype(parts)::value) {
        const uint32_t a = __float_as_uint(e[2 * i]), b = __float_as_uint(e[2 * i + 1]);
        hi[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);  // the upper halves
        lo[i] = pack_bf2(fmaf(e[2 * i], 1.f + 0x1p-23f, -__uint_as_float(a & 0xffff0000u)),
                         fmaf(e[2 * i + 1], 1.f + 0x1p-23f, -__uint_as_float(b & 0xffff0000u)));
      } else {
        hi[i] = pack_bf2(e[2 * i], e[2 * i + 1]);
      }
    }
    p[k] = as_bf16x8(u32x4_t{hi[0], hi[1], hi[2], hi[3]});
    if (decltype(parts)::value) p[2 + k] = as_bf16x8(u32x4_t{lo[0], lo[1], lo[2], lo[3]});
  };
  // Where a pair's weights of a chunk have grown too large for its reference (or it has none): the reference moves to the chunk's
  // largest score, the sums with it, and the weights are made again.
  auto weigh = [&](auto parts, const f32x16_t& s, bf16x8_t (&p)[4], float sum) {
    if (__any(sum > most)) {
      float cm = s[0];
#pragma unroll
      for (int r = 1; r < 16; r++) cm = fmaxf(cm, s[r]);
      cm = max_halves(cm) * scale;
      const float old = most < 0.f ? -INFINITY : -base, now = fmaxf(old, cm);
      if (now > -INFINITY) {
        const float alpha = __builtin_amdgcn_exp2f(old - now);
        base = -now;
        most = kMost;
        l *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; dt++)
#pragma unroll
          for (int r = 0; r < 16; r++) o[dt][r] *= alpha;
      }
      sum = 0.f;
#pragma unroll
      for (int k = 0; k < 2; k++) {
        float e[8];
#pragma unroll
        for (int r = 0; r < 8; r++) {
          e[r] = __builtin_amdgcn_exp2f(fmaf(s[8 * k + r], scale, base));
          sum += e[r];
        }
        to_bf16(parts, e, p, k);
      }
    }
    l += sum;
  };
  auto add = [&](auto parts, bf16x8_t v, const bf16x8_t (&p)[4], int k, f32x16_t& o) {
    o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[k], o, 0, 0, 0);
    if (decltype(parts)::value) o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[2 + k], o, 0, 0, 0);
  };
  auto add_values = [&](auto parts, int slot, const bf16x8_t (&p)[4]) {
    const char* vb = smem + (kRing + slot) * kSide + v_lane;
#pragma unroll
    for (int k = 0; k < 2; k++)
#pragma unroll
      for (int dt = 0; dt < DT; dt++) add(parts, as_bf16x8(*(const u32x4_t*)(vb + k * kBlockBytes + dt * 512)), p, k, o[dt]);
  };
  // Chunk ch's weights on the vector units, while the matrix units add chunk ch - 1's values (not with `first`) and make chunk
  // ch + 1's scores. Products take turns between the two, each with its share of the weights' arithmetic behind it, and fragments
  // are read kAhead products ahead. (Behind the last chunk the scores are of whatever lies there, and nobody's.)
  auto products = [&](auto first, auto parts, int slot, f32x16_t& s, f32x16_t& s_next, bf16x8_t (&p_last)[4], bf16x8_t (&p)[4]) {
    constexpr bool kFirst = decltype(first)::value;
    constexpr int kProducts = KK + (kFirst ? 0 : 2 * DT), kShare = 16 / kProducts, kAhead = 3;
    const char* kb = smem + (slot + 1) % kRing * kSide + k_lane;
    const char* vb = smem + (kRing + (slot + kRing - 1) % kRing) * kSide + v_lane;
    u32x4_t frag[kAhead + 1];
    auto read = [&](int i) {
      const char* from = kFirst ? kb + i * 512 : i % 2 ? kb + i / 2 * 512 : vb + i / 2 / DT * kBlockBytes + i / 2 % DT * 512;
      frag[i % (kAhead + 1)] = *(const u32x4_t*)from;
    };
    float sum = 0.f, e[16];
#pragma unroll
    for (int r = 0; r < 16; r++) s_next[r] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kAhead; i++) read(i);
#pragma unroll
    for (int i = 0; i < kProducts; i++) {
      __builtin_amdgcn_sched_barrier(0);
      if (i + kAhead < kProducts) read(i + kAhead);
      const bf16x8_t f = as_bf16x8(frag[i % (kAhead + 1)]);
      if (kFirst || i % 2) s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, q[kFirst ? i : i / 2], s_next, 0, 0, 0);
      else add(parts, f, p_last, i / 2 / DT, o[i / 2 % DT]);
#pragma unroll
      for (int r = i * kShare; r < (i + 1) * kShare; r++) {
        e[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale, base));
        if (r > 0) sum += e[r - 1];  // a step late: nothing waits for the exponential
        if (r % 8 == 7) to_bf16(parts, e + r - 7, p, r / 8);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    weigh(parts, s, p, sum + e[15]);
  };
  // A turn for chunk c0 + n: at its start V(n - 1) and K(n + 1) have landed, and V(n + 2) and K(n + 4) are fetched into the places
  // of V(n - 2) and K(n), three turns before their use.
  auto turn = [&](auto first, auto single, int n, f32x16_t& s, f32x16_t& s_next, bf16x8_t (&p_last)[4], bf16x8_t (&p)[4]) {
    constexpr bool kFirst = decltype(first)::value, once = decltype(single)::value;
    const int ch = c0 + n, slot = n % kRing;
    if (ch + 2 < c1) fetch_v(n + 2, (n + 2) % kRing, once);
    if (ch + 4 < c1) fetch_k(n + 4, slot, once);
    if (ch * kChunk < wave_most) {
      mask(ch, s);
      products(first, single, slot, s, s_next, p_last, p);
    } else if (!kFirst && (ch - 1) * kChunk < wave_most) {
      add_values(single, (n + kRing - 1) % kRing, p_last);
    }
    landed(ch + 4 >= c1);
    mend(ch);
  };
  // A run of chunks. single: of a sequence of one tile.
  auto chunks = [&](auto single) {
    constexpr bool once = decltype(single)::value;
    f32x16_t sa, sb;
    bf16x8_t pa[4], pb[4];
    const int n_end = c1 - c0;
    fetch_k(0, 0, once);
    if (1 < n_end) fetch_k(1, 1, once);
    fetch_v(0, 0, once);
    if (2 < n_end) fetch_k(2, 2, once);
    if (1 < n_end) fetch_v(1, 1, once);
    if (3 < n_end) fetch_k(3, 3, once);
    landed(4 > n_end);
    if (c0 * kChunk < wave_most) {
      const char* kb = smem + k_lane;
#pragma unroll
      for (int r = 0; r < 16; r++) sa[r] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; kk++)
        sa = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*(const u32x4_t*)(kb + kk * 512)), q[kk], sa, 0, 0, 0);
    }
    meet();  // K(0) is read
    turn(std::true_type{}, single, 0, sa, sb, pb, pa);
    int n = 1;
    {
      // Turns that every row of the tile sees whole and that have chunks to fetch: the same without the questions, four at a time
      // so that their places in the rings are constants.
      auto plain = [&](auto slot, f32x16_t& s, f32x16_t& s_next, bf16x8_t (&p_last)[4], bf16x8_t (&p)[4]) {
        constexpr int kSlot = decltype(slot)::value;
        fetch_v(n + 2, (kSlot + 2) % kRing, once);
        fetch_k(n + 4, kSlot, once);
        if (wave_live) products(std::false_type{}, single, kSlot, s, s_next, p_last, p);
        landed(false);
        n++;
      };
      const int plain_end = min(n_end - 4, (first_pos + 1) / kChunk - c0);
      while (n + 3 < plain_end) {
        plain(std::integral_constant<int, 1>{}, sb, sa, pa, pb);
        plain(std::integral_constant<int, 2>{}, sa, sb, pb, pa);
        plain(std::integral_constant<int, 3>{}, sb, sa, pa, pb);
        plain(std::integral_constant<int, 0>{}, sa, sb, pb, pa);
      }
    }
    for (; n < n_end; n += 2) {
      turn(std::false_type{}, single, n, sb, sa, pa, pb);
      if (n + 1 < n_end) turn(std::false_type{}, single, n + 1, sa, sb, pb, pa);
    }
    if ((c1 - 1) * kChunk < wave_most) {
      if (n_end & 1) add_values(single, (n_end - 1) % kRing, pa);
      else add_values(single, (n_end - 1) % kRing, pb);
    }
  };
  if (one_tile) chunks(std::true_type{});
  else chunks(std::false_type{});
  if (bad) atomicOr(c.err, SIDP_DEVERR_BLOCK);

  // Register r of O^T's tile dt is dim 32 dt + 8 (r / 4) + 4 half + r % 4.
  if (s_odd) {
#pragma unroll
    for (int dt = 0; dt < DT; dt++)
#pragma unroll
      for (int r = 0; r < 16; r++) {
        const int d = 32 * dt + 8 * (r / 4) + 4 * half + r % 4;
        if (s_first[0][d] < limit) o[dt][r] += INFINITY;
        if (s_first[1][d] < limit) o[dt][r] -= INFINITY;
        if (s_first[2][d] < limit) o[dt][r] = NAN;
      }
  }
  const float sum = l + __shfl_xor(l, 32, 64);
  int late = threadIdx.x;
  asm volatile("" : "+v"(late));  // made again here rather than kept
  const Pair out = pair_of(late);
  const int from = (late >> 5 & 1) * 4;  // the lane's first dim
  if (out.tok >= tokens) return;
  const int64_t out_row = (int64_t)(row0 + out.tok) * c.hq + g * group + out.head;
  if (rec < 0) {
    const float inv = 1.f / sum;
    uint16_t* op = c.out + out_row * D + from;
#pragma unroll
    for (int dt = 0; dt < DT; dt++)
#pragma unroll
      for (int i = 0; i < 4; i++)
        *(u32x2_t*)(op + dt * 32 + i * 8) = u32x2_t{pack_bf2(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv),
                                                    pack_bf2(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv)};
  } else {
    float* r = (float*)((char*)c.ws + lay.recs) + ((int64_t)rec * hkv + g) * lay.rec_rows * (D + 2);
#pragma unroll
    for (int dt = 0; dt < DT; dt++)
#pragma unroll
      for (int i = 0; i < 4; i++)
        *(f32x4_t*)(r + out.at * D + dt * 32 + i * 8 + from) =
            f32x4_t{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
    if (from == 0) *(float2*)(r + (int64_t)lay.rec_rows * D + 2 * out.at) = make_float2(most < 0.f ? -INFINITY : -base, sum);
  }
}

// Joins a cut tile's records in run order: four dims a thread, 1024 / D pairs of one (cut tile, KV head) a workgroup, the records
// of kJoin runs in flight at a time.
constexpr int kJoin = 8;
template <int D>
__global__ void __launch_bounds__(256) k_attn_rows_join(AttnRowsCall c, Layout lay) {
  const char* ws = (const char*)c.ws;
  const Cut cut = ((const Cut*)(ws + lay.cuts))[blockIdx.x];  // read beside the count, and of no meaning past it
  if ((int)blockIdx.x >= ((const int32_t*)ws)[1]) return;
  const int hkv = c.kv.hkv, g = blockIdx.y, group = c.hq / hkv;
  const int pair = blockIdx.z * (1024 / D) + threadIdx.x / (D / 4), d = threadIdx.x % (D / 4) * 4;
  if (pair >= cut.pairs) return;
  const int64_t step = (int64_t)hkv * lay.rec_rows * (D + 2);
  const float* rec = (const float*)(ws + lay.recs) + ((int64_t)cut.rec * hkv + g) * lay.rec_rows * (D + 2);
  const float* ml = rec + (int64_t)lay.rec_rows * D + 2 * pair;
  rec += (int64_t)pair * D + d;
  float M = -INFINITY, L = 0.f;
  f32x4_t O = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < cut.parts; p0 += kJoin) {
    float2 r[kJoin];
    f32x4_t v[kJoin];
#pragma unroll
    for (int i = 0; i < kJoin; i++) {
      const int p = min(p0 + i, cut.parts - 1);
      r[i] = *(const float2*)(ml + p * step);
      v[i] = *(const f32x4_t*)(rec + p * step);
    }
    float now = M;
#pragma unroll
    for (int i = 0; i < kJoin; i++) now = fmaxf(now, r[i].x);
    // a run of which the pair sees nothing left zeros and -inf
    const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - now);
    if (p0 > 0) {
      L *= f;
      O *= f;
    }
    M = now;
#pragma unroll
    for (int i = 0; i < kJoin; i++)
      if (p0 + i < cut.parts) {
        const float w = r[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(r[i].x - now);
        L = fmaf(r[i].y, w, L);
        O += v[i] * w;
      }
  }
  const float inv = 1.f / L;
  const int64_t row = (int64_t)(cut.row0 + pair / group) * c.hq + g * group + pair % group;
  *(u32x2_t*)(c.out + row * D + d) = u32x2_t{pack_bf2(O[0] * inv, O[1] * inv), pack_bf2(O[2] * inv, O[3] * inv)};
}

template <int D>
hipError_t launch_d(const AttnRowsCall& c, hipStream_t s) {
  const Layout lay = layout_of(c.batch, c.max_rows, c.hq, c.kv.hkv, D, c.max_seq, c.num_cus);
  const int waves = std::min(kPlanWaves, (std::max(c.batch, lay.tiles_cap) + 63) / 64);
  k_attn_rows_plan<<<1, 64 * waves, (3 * (size_t)c.batch + 1) * sizeof(int32_t), s>>>(c, lay);
  const size_t lds = 2 * kRing * (size_t)kChunk * D * 2;
  if (lds > 32 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)k_attn_rows<D>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  k_attn_rows<D><<<(unsigned)((int64_t)lay.entries_cap * c.kv.hkv), 256, lds, s>>>(c, lay);
  if (lay.cuts_cap > 0 && lay.recs_cap > 1)
    k_attn_rows_join<D><<<dim3(lay.cuts_cap, c.kv.hkv, (lay.rec_rows + 1024 / D - 1) / (1024 / D)), 256, 0, s>>>(c, lay);
  return hipGetLastError();
}

}  // namespace

size_t attn_rows_ws_bytes(int batch, int max_rows, int hq, int hkv, int d, int max_seq, int num_cus) {
  return layout_of(batch, max_rows, hq, hkv, d, max_seq, num_cus).bytes;
}

hipError_t launch_attention_rows(const AttnRowsCall& c, hipStream_t s) {
  if (c.max_rows <= 0) return hipSuccess;
  return c.kv.d == 128 ? launch_d<128>(c, s) : launch_d<64>(c, s);
}

}  // namespace sidp
