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
#include "attn_tile.h"
#include "common.h"
#include "internal.h"

namespace sidp {

namespace {

// Items (entry, KV head) the chip holds at once: two workgroups a CU.
constexpr int kSlotsPerCu = 2;
// A launch with fewer items than slots cuts sequences into runs of at least this many chunks, and a tile into at most this many.
constexpr int kMinRun = 16, kMaxRuns = 32;
// Cutting writes and reads partial outputs, so only where the longest item is this much longer than the runs would be. Whole /
// cut, us a call on the 70B heads, longest item and run in chunks: 16 sequences of 32 rows over 500 cached 17, 16: 28 / 39; of 1 row
// over 1000 32, 16: 32 / 26; of 32 rows over 4000 126, 63: 96 / 98; 1 of 200 rows over 2000 69, 16: 49 / 39; 4 of 100 rows over
// 4000 129, 56: 82 / 80; 1 of 16 rows over 30000 939, 30: 480 / 46.
constexpr float kCutFrom = 1.75f;

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

template <int D>
__global__ void __launch_bounds__(256, 2) k_attn_rows(AttnRowsCall c, Layout lay) {
  const char* ws = (const char*)c.ws;
  const int hkv = c.kv.hkv, group = c.hq / hkv, tm = tile_tokens(group);
  const int item = blockIdx.x;
  if (item >= ((cint32_t*)ws)[0] * hkv) return;
  cint32_t* ep = (cint32_t*)(ws + lay.entries) + (item / hkv) * 4;
  const int g = item % hkv;
  const int b = ep[0], tile = ep[1], c0 = ep[2] & 0xffff, c1 = c0 + (int)((uint32_t)ep[2] >> 16), rec = ep[3];
  const int seq0 = ((cint32_t*)c.row_starts)[b], seq_rows = ((cint32_t*)c.row_starts)[b + 1] - seq0;
  const int tokens = min(tm, seq_rows - tile * tm);
  const int first_pos = ((cint32_t*)c.ctx_lens)[b] + tile * tm;
  const AttnTile<true> x = {b, seq0 + tile * tm, tokens, first_pos, first_pos + tokens, c0, c1, g, seq_rows <= tm};
  attn_tile<D, 0>(c, x, [&](const AttnOut<D>& out) {
    if (rec < 0) {
      out.rows(c.out);
    } else {
      float* r = (float*)((char*)c.ws + lay.recs) + ((int64_t)rec * hkv + g) * lay.rec_rows * (D + 2);
      out.record(r + out.at * D, r + (int64_t)lay.rec_rows * D + 2 * out.at);
    }
  });
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
  const size_t lds = tile_lds<D, 0>();
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
