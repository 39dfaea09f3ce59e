// Causal attention of several new tokens a sequence, as k_attn_rows.hip has it, for
// the calls whose items are not always whole tiles of one sequence: over the 8-bit
// cache, and where groups of sequences share their first blocks.
//
// A group's shared keys are read once for all of its rows: the rows of a group follow
// each other, so they make tiles of 128 / (Hq / Hkv) rows over the shared chunks, every
// row of which sees all of them, and each sequence's own tiles begin behind. With
//   m = max over parts of the parts' references m_i, l = sum l_i 2^(m_i - m)
//   out = sum o_i 2^(m_i - m) / l
// a row's parts (its group's, its sequence's, and the runs that either was cut into) are
// joined. A group of n sequences of one row reads S shared tokens ceil(n G / 128) times
// instead of n, and its products fill the matrices' columns, G being Hq / Hkv.
//
// Only whole chunks of 32 tokens are shared; the rest of the prefix is read by each
// sequence as its own. A group shares where its tiles are at most half of its sequences'
// (parts_plan.h, where the rules of the plan stand with what both their sides measured).
//
// P reaches V with 16 bits in tiles of attn_few.h with up to 16 pairs, and over bf16 in all
// tiles of a sequence or group of one tile; rounded to bf16 in the others. Rounded and in two
// parts there, us a call: 256 rows under 8192 shared bf16 tokens 137 and 162, 64 under 4096 43
// and 47; 8 ragged chunks of e4m3 280 and 367, of int8 299 and 388; 16 sequences of 1-7 rows over
// int8 46 and 48, of 8 rows over 4000 59 and 64. Distance from 64 bits 0.0021 to 0.0023 of the norm,
// 0.0017 with 16 bits, which is what the result's own rounding makes.
//
// Measured with 64 and 8 heads of 128, us with plan and join: over e4m3 64 sequences of a row
// with 1-8K keys 119-131 (625 MB, 5.6 TB/s in the kernel itself), over int8 134-143; 8 ragged
// chunks of 234 to 348 GFLOP, as lengths meet, 280-410 over e4m3 (0.80 to 0.87 PFLOP/s: matrix
// units 40% and vector issue 47%, held by what each waits for of the other), 300-440 over int8;
// 16 sequences of 1-7 rows with 0.5-4K keys 41-46 over int8, 41 over e4m3; 256 sequences of a
// row over 8192 shared keys of bf16 135-147 (566 MB, 8.6 GB if each read them itself), of
// e4m3 146-151, of int8 161; 72 over 6 prefixes of e4m3 50, of int8 51, of which plan and join
// are 17: one workgroup in front of all.
#include "attn_few.h"
#include "attn_tile.h"
#include "common.h"
#include "internal.h"
#include "parts_plan.h"

namespace sidp {

namespace {

// Over codes, tiles of up to this many pairs go by attn_few.h, whose waves spread out what they need by themselves. By it and by
// attn_tile.h, us a call, 16 sequences over 4000 keys, heads of 128: 24 pairs e4m3 41 and 45, int8 43 and 48; 40 pairs 49 and 53, 57
// and 55; 64 pairs 52 and 54, 60 and 57. Heads of 64: 24 pairs 32 and 39, 33 and 42; 64 pairs 41 and 46, 44 and 49. Over 500 keys the
// two are within 2 us. 128 pairs of e4m3 96 and 81. Over bf16, 64 pairs over 2048 shared tokens 29 us by it, 26 by attn_tile.h: only
// 16 pairs go by it.
constexpr int kFewPairs = 64;

__host__ __device__ inline int half_places(int num_cus) { return kSlotsPerCu * (num_cus < 1 ? 1 : num_cus) / 2; }

enum { kOwnKeys = 1, kOneTile = 2 };  // flags: a row sees the keys up to its own; nobody else reads these keys
struct Entry {
  int b, row0, tokens, first_pos, kv_end;
  uint32_t run;  // first chunk | chunks << 16
  int rec;       // the first row's record, -1: the output itself
  int flags;
};
// Rows of a sequence whose parts are joined. A record of part p of row i: rec + p rows + i; of the group's part p: grec + j tm
// gparts + p min(tm, grows - j tm) + w for row goff + i = j tm + w of the group.
struct Cut {
  int row0, rows, parts, rec;
  int grec, gparts, goff, grows;
};

// Workspace: counts, entries, cuts, records (o [row][Hq][D], then m and l [row][Hq][2]).
struct Layout {
  PartsCaps caps;
  size_t entries, cuts, recs, sums, bytes;
};

Layout layout_of(int batch, int max_rows, int hq, int hkv, int d, int num_cus, bool groups) {
  Layout l;
  l.caps = parts_caps(batch, max_rows, tile_tokens(hq / hkv), slots_of(num_cus, hkv), groups);
  size_t o = 64;
  auto place = [&](size_t n) {
    const size_t at = o;
    o = (o + n + 255) / 256 * 256;
    return at;
  };
  l.entries = place((size_t)l.caps.entries * sizeof(Entry));
  l.cuts = place((size_t)l.caps.cuts * sizeof(Cut));
  l.recs = place((size_t)l.caps.recs * hq * d * sizeof(float));
  l.sums = place((size_t)l.caps.recs * hq * 2 * sizeof(float));
  l.bytes = o;
  return l;
}

// Lists the items. One workgroup, a chain of latencies in front of the attention.
//
// Tiles are numbered groups first, then sequences. Fewer than the chip holds at once:
// every tile is cut into even runs of at most `run` chunks, the shortest of kTries
// lengths between an even share of all chunks and one that cannot give more runs than
// fit. Otherwise sequences' tiles stay whole, groups' are cut into runs of an even share
// (256 sequences under 8192 tokens 142 us, 150 with half of one, whose records are twice
// as many; 72 under 6 prefixes 51 and 57), and the longest items come first, so that the launch ends evenly. Tiles of few
// pairs that are short beside a wave's even share are items of a wave each: they are
// listed apart, behind the others.
constexpr int kPlanWaves = 16;
__global__ void __launch_bounds__(64 * kPlanWaves) k_attn_parts_plan(AttnPartsCall c, Layout lay) {
  extern __shared__ int32_t s_lds[];
  __shared__ int s_scan[4][kPlanWaves], s_longest[kPlanWaves];
  __shared__ ChunkSum s_total[kPlanWaves];
  __shared__ int s_hist[256], s_waves[256], s_listed[2];
  __shared__ int s_items[kTries];
  __shared__ int s_cuts, s_bad;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, threads = blockDim.x, waves = threads / 64;
  const int group = c.hq / c.kv.hkv, tm = tile_tokens(group);
  const int slots = slots_of(c.num_cus, c.kv.hkv);
  const int B = c.batch, G = c.groups;
  int32_t* s_first = s_lds;            // [G + B + 1] first tile of each group, then of each sequence
  int32_t* s_ctx = s_first + G + B + 1;  // [B] cached tokens
  int32_t* s_rows = s_ctx + B;         // [B] rows
  int32_t* s_group = s_rows + B;       // [B] its group, if that shares, or -1
  int32_t* s_chunks = s_group + B;     // [G] shared chunks
  int32_t* s_seq = s_chunks + G;       // [G] the first sequence with rows
  int32_t* s_own = s_seq + G;          // [G] its sequences' tiles, and later its first record
  int32_t* s_grows = s_own + G;        // [G] rows
  char* ws = (char*)c.ws;
  int32_t* counts = (int32_t*)ws;
  Entry* entries = (Entry*)(ws + lay.entries);
  Cut* cuts = (Cut*)(ws + lay.cuts);
  if (t < kTries) s_items[t] = 0;
  if (t == 0) s_cuts = s_bad = 0;
  for (int i = t; i < 256; i += threads) s_hist[i] = s_waves[i] = 0;
  __syncthreads();
  // a sequence whose starts or lengths the call does not cover has no rows
  bool bad = false;
  for (int b = t; b < B; b += threads) {
    const int r0 = c.row_starts[b], r1 = c.row_starts[b + 1], ctx = c.ctx_lens[b];
    const bool ok = r0 >= 0 && r1 >= r0 && r1 <= c.max_rows && ctx >= 0 &&
                    (int64_t)ctx + (r1 - r0) <= (int64_t)min(c.max_blocks * kBlockTokens, c.max_seq);
    bad |= !ok;
    s_ctx[b] = ctx;
    s_rows[b] = ok ? r1 - r0 : 0;
    s_group[b] = -1;
  }
  // starts of groups, held where the tiles will be; out of order or range they mean nothing
  for (int i = t; i < G; i += threads) {
    const int g0 = c.group_starts[i], g1 = c.group_starts[i + 1], shared = c.shared_lens[i];
    bad |= g0 < 0 || g1 < g0 || g1 > B || shared < 0;
    s_first[i] = g0;
    s_chunks[i] = shared;
    s_seq[i] = B;
    s_own[i] = 0;
    s_grows[i] = g1;  // for now
  }
  if (bad) {
    atomicOr(c.err, SIDP_DEVERR_POSITION);
    s_bad = 1;
  }
  __syncthreads();
  const bool any_bad = s_bad;  // then nothing is shared: rows of which nothing is known may lie among a group's
  auto last_at = [](const int* s, int n, int i) {  // the last of s[0 .. n) that is at most i
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s[mid] <= i) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  if (G > 0 && !any_bad) {
    for (int b = t; b < B; b += threads) {
      if (s_rows[b] == 0 || b < s_first[0]) continue;
      const int i = last_at(s_first, G, b);
      if (b >= s_grows[i]) continue;
      if (s_ctx[b] < s_chunks[i]) {  // the group's keys are not all this sequence's: every sequence reads its own
        atomicOr(c.err, SIDP_DEVERR_POSITION);
        atomicMin(&s_own[i], -(1 << 30));
      } else {
        s_group[b] = i;
        atomicMin(&s_seq[i], b);
        atomicAdd(&s_own[i], (s_rows[b] + tm - 1) / tm);
      }
    }
    __syncthreads();
    for (int i = t; i < G; i += threads) {
      const int row0 = c.row_starts[s_first[i]], rows = c.row_starts[s_grows[i]] - row0;
      const bool shares = group_shares(s_chunks[i] / kChunk, rows, s_own[i], tm);
      s_chunks[i] = shares ? s_chunks[i] / kChunk : 0;
      s_grows[i] = shares ? rows : 0;
    }
    __syncthreads();
    for (int b = t; b < B; b += threads)
      if (s_group[b] >= 0 && s_chunks[s_group[b]] == 0) s_group[b] = -1;
  } else {
    for (int i = t; i < G; i += threads) s_chunks[i] = s_grows[i] = 0;
  }
  __syncthreads();
  // exclusive place of a thread's `mine` among all threads', and the sum
  auto scan = [&](int mine, int which, int& sum) {
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o, 64);
      if (lane >= o) incl += v;
    }
    if (lane == 63) s_scan[which][wave] = incl;
    __syncthreads();
    int at = incl - mine;
    sum = 0;
    for (int w = 0; w < waves; w++) {
      if (w < wave) at += s_scan[which][w];
      sum += s_scan[which][w];
    }
    return at;
  };
  auto tiles_of = [&](int i) { return ((i < G ? s_grows[i] : s_rows[i - G]) + tm - 1) / tm; };
  int tiles, gtiles;
  {
    const int per = (G + B + threads - 1) / threads, i0 = min(t * per, G + B), i1 = min(i0 + per, G + B);
    int mine = 0, mine_g = 0;
    for (int i = i0; i < i1; i++) {
      mine += tiles_of(i);
      if (i < G) mine_g += tiles_of(i);
    }
    int at = scan(mine, 0, tiles);
    scan(mine_g, 1, gtiles);
    for (int i = i0; i < i1; i++) {
      s_first[i] = at;
      at += tiles_of(i);
    }
    if (t == 0) s_first[G + B] = tiles;
  }
  __syncthreads();
  tiles = min(tiles, lay.caps.tiles + gtiles);  // row starts that overlap could list more
  struct Tile {
    int i, place;     // the group, or G and the sequence; which of its tiles
    int rows, from, chunks;
    bool rec;         // of a group, or of a sequence that shares
  };
  auto tile_of = [&](int n) {
    const int i = last_at(s_first, G + B, n), place = n - s_first[i];
    if (i < G) return Tile{i, place, min(tm, s_grows[i] - place * tm), 0, s_chunks[i], true};
    const int b = i - G, end = min(s_rows[b], (place + 1) * tm), from = s_group[b] >= 0 ? s_chunks[s_group[b]] : 0;
    return Tile{i, place, end - place * tm, from, (s_ctx[b] + end + kChunk - 1) / kChunk - from, s_group[b] >= 0};
  };
  // the tiles of this thread, in order; one, as a rule, which is looked up once
  const int per = (tiles + threads - 1) / threads, n0 = min(t * per, tiles), n1 = min(n0 + per, tiles);
  Tile only = {};
  if (per == 1 && n0 < n1) only = tile_of(n0);
  auto each_tile = [&](auto f) {
    for (int n = n0; n < n1; n++) f(per == 1 ? only : tile_of(n));
  };
  int own_chunks = 0, longest = 1;
  each_tile([&](const Tile& x) {
    own_chunks += x.chunks;  // at most 2^18 / 1024 tiles of 2^15
    longest = max(longest, x.chunks);
  });
  ChunkSum total = own_chunks;
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
  const bool few = tiles < slots && tiles <= threads;
  int run = longest;
  if (few) {
    const int least = least_run(total, slots, longest);
    if (tiles_are_cut(longest, least)) {
      const int safe = safe_run(total, slots, tiles, least);
      auto try_of = [&](int j) { return try_run(j, least, safe); };
      int n[kTries];
#pragma unroll
      for (int j = 0; j < kTries; j++) n[j] = (own_chunks + try_of(j) - 1) / try_of(j);
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
  } else if (gtiles > 0 && slots > 0) {
    run = group_run(total, slots, longest);
  }
  auto parts_of = [&](const Tile& x) { return few || x.i < G ? (x.chunks + run - 1) / run : 1; };
  // places of entries (in order, or by length) and of records
  auto bucket = [&](const Tile& x, int parts) { return 255 - x.chunks / parts * 255 / longest; };
  const int wave_most = wave_item(total, kWaves, slots, longest);
  auto by_wave = [&](const Tile& x) {
    return !few && x.i >= G && x.rows * group <= 16 && (c.kv8.type != 0 || x.rows == 1) && x.chunks <= wave_most;
  };
  int entries_mine = 0, recs_mine = 0, all, recs;
  each_tile([&](const Tile& x) {
    const int parts = parts_of(x);
    entries_mine += parts;
    if (parts > 1 || x.rec) recs_mine += parts * x.rows;
    if (!few) atomicAdd(by_wave(x) ? &s_waves[bucket(x, 1)] : &s_hist[bucket(x, parts)], parts);
  });
  int at = scan(entries_mine, 2, all), rec_at = scan(recs_mine, 3, recs);
  {  // a group's first record
    int r = rec_at;
    each_tile([&](const Tile& x) {
      if (x.i < G && x.place == 0) s_own[x.i] = r;
      const int parts = parts_of(x);
      if (parts > 1 || x.rec) r += parts * x.rows;
    });
  }
  __syncthreads();
  if (!few && t < 128) {  // a wave each
    int* hist = t < 64 ? s_hist : s_waves;
    int h[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; j++) {
      h[j] = sum;
      sum += hist[4 * lane + j];
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(inc, o, 64);
      if (lane >= o) inc += v;
    }
#pragma unroll
    for (int j = 0; j < 4; j++) hist[4 * lane + j] = inc - sum + h[j];
    if (lane == 63) s_listed[t >> 6] = inc;
  }
  __syncthreads();
  const int by_group = few ? all : s_listed[0];  // items of a workgroup
  each_tile([&](const Tile& x) {
    const int parts = parts_of(x);
    const bool shared = x.i < G, rec = parts > 1 || x.rec;
    const int b = shared ? s_seq[x.i] : x.i - G;
    const int row0 = c.row_starts[shared ? c.group_starts[x.i] : b] + x.place * tm;
    const int end = shared ? x.chunks * kChunk : s_ctx[b] + x.place * tm + x.rows;
    const bool alone = (shared ? s_grows[x.i] : s_rows[b]) <= tm;
    // Within a step of length the order is whatever the atomics give; items write places of their own, so results do not depend on it.
    const int e0 = few ? at : by_wave(x) ? by_group + atomicAdd(&s_waves[bucket(x, 1)], 1) : atomicAdd(&s_hist[bucket(x, parts)], parts);
    for (int p = 0; p < parts; p++) {
      const int lo = x.from + x.chunks * p / parts, hi = x.from + x.chunks * (p + 1) / parts;
      entries[e0 + p] = Entry{b, row0, x.rows, shared ? end - 1 : end - x.rows, end, (uint32_t)lo | (uint32_t)(hi - lo) << 16,
                              rec ? rec_at + p * x.rows : -1, (shared ? 0 : kOwnKeys) | (alone ? kOneTile : 0)};
    }
    if (rec && !shared) {
      Cut cut = {row0, x.rows, parts, rec_at, 0, 0, 0, 0};
      const int i = s_group[b];
      if (i >= 0) {
        cut.grec = s_own[i];
        cut.gparts = (s_chunks[i] + run - 1) / run;
        cut.goff = row0 - c.row_starts[c.group_starts[i]];
        cut.grows = s_grows[i];
      }
      cuts[atomicAdd(&s_cuts, 1)] = cut;
    }
    at += parts;
    if (rec) rec_at += parts * x.rows;
  });
  __syncthreads();
  if (t == 0) {
    counts[0] = by_group;
    counts[1] = s_cuts;
    counts[2] = all - by_group;
  }
}

// Workgroups, in the order in which they start: half the chip's places of workgroups' items, then as many of wave items as go beside
// them, and again; the former are products most of all, the latter bytes.
template <int D, int TYPE>
__global__ void __launch_bounds__(256, 2) k_attn_parts(AttnPartsCall c, Layout lay) {
  const char* ws = (const char*)c.ws;
  const int hkv = c.kv.hkv, group = c.hq / hkv;
  const int items = ((cint32_t*)ws)[0] * hkv, wave_items = ((cint32_t*)ws)[2] * hkv, wave_groups = (wave_items + kWaves - 1) / kWaves;
  int item = blockIdx.x, wave_group = -1;
  if (wave_groups > 0) {
    const int half = half_places(c.num_cus), rounds = items / half;
    const int beside = items == 0 ? 0 : (int)(((int64_t)wave_groups * half + items - 1) / items);
    const int round = min(item / (half + beside), rounds), in_round = item - round * (half + beside);
    const int here = round < rounds ? half : items - rounds * half;  // the last round takes what is left of both
    if (in_round < here) item = round * half + in_round;
    else wave_group = round * beside + in_round - here;
  }
  if (wave_group < 0 ? item >= items : wave_group >= wave_groups) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int at = wave_group < 0 ? item : items + wave_group * kWaves + wave;  // among all items, entry by entry
  if (at >= items + wave_items) return;
  cint32_t* ep = (cint32_t*)(ws + lay.entries) + (at / hkv) * 8;
  const int c0 = ep[5] & 0xffff, rec = ep[6], flags = ep[7], g = at % hkv;
  const AttnTile<false> x = {ep[0], ep[1], ep[2], ep[3], ep[4], c0, c0 + (int)((uint32_t)ep[5] >> 16), g,
                             (flags & kOneTile) != 0, flags & kOwnKeys};
  float* const recs = (float*)((char*)c.ws + lay.recs);
  float* const sums = (float*)((char*)c.ws + lay.sums);
  const int pairs = x.tokens * group;
  auto emit = [&](int tok, int head, int dim, f32x4_t o, float sum, float ref) {
    if (rec < 0) {
      const float inv = 1.f / sum;
      *(u32x2_t*)(c.out + ((int64_t)(x.row0 + tok) * c.hq + g * group + head) * D + dim) =
          u32x2_t{pack_bf2(o[0] * inv, o[1] * inv), pack_bf2(o[2] * inv, o[3] * inv)};
    } else {
      const int64_t to = (int64_t)(rec + tok) * c.hq + g * group + head;
      *(f32x4_t*)(recs + to * D + dim) = o;
      if (dim == 0) *(float2*)(sums + to * 2) = make_float2(ref, sum);
    }
  };
  if (pairs <= 16 && (TYPE != 0 || x.tokens == 1 || x.step == 0)) return attn_few<D, TYPE, 1>(c, x, wave_group < 0 ? 1 : 0, emit);
  if constexpr (TYPE != 0) {
    if (pairs <= kFewPairs) return attn_few<D, TYPE, 2>(c, x, pairs <= 32 ? 1 : 2, emit);
  }
  attn_tile<D, TYPE>(c, x, [&](const AttnOut<D>& out) {
    if (rec < 0) {
      out.rows(c.out);
    } else {
      const int64_t to = out.row + (int64_t)(rec - x.row0) * c.hq;  // the same head of the record
      out.record(recs + to * D, sums + to * 2);
    }
  });
}

// Joins rows' parts, the group's first, then the sequence's, in order: four dims a thread, 1024 / D heads of one (cut, KV head) at a
// time, the records of kJoin parts in flight.
constexpr int kJoin = 8;
template <int D>
__global__ void __launch_bounds__(256) k_attn_parts_join(AttnPartsCall c, Layout lay) {
  const char* ws = (const char*)c.ws;
  const Cut cut = ((const Cut*)(ws + lay.cuts))[blockIdx.x];  // read beside the count, and of no meaning past it
  if ((int)blockIdx.x >= ((const int32_t*)ws)[1]) return;
  const int group = c.hq / c.kv.hkv, tm = tile_tokens(group);
  const int d = threadIdx.x % (D / 4) * 4;
  for (int pair = blockIdx.z * (1024 / D) + threadIdx.x / (D / 4); pair < cut.rows * group; pair += gridDim.z * (1024 / D)) {
    const int i = pair / group, head = blockIdx.y * group + pair % group;
    const int j = (cut.goff + i) / tm, w = (cut.goff + i) % tm;
    const int64_t shared = cut.grec + (int64_t)j * tm * cut.gparts + w, step = min(tm, cut.grows - j * tm);
    const int n = cut.gparts + cut.parts;
    auto record = [&](int p) {
      return (p < cut.gparts ? shared + p * step : cut.rec + (int64_t)(p - cut.gparts) * cut.rows + i) * c.hq + head;
    };
    float M = -INFINITY, L = 0.f;
    f32x4_t O = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < n; p0 += kJoin) {
      float2 r[kJoin];
      f32x4_t v[kJoin];
#pragma unroll
      for (int k = 0; k < kJoin; k++) {
        const int64_t at = record(min(p0 + k, n - 1));
        r[k] = *(const float2*)((const float*)(ws + lay.sums) + at * 2);
        v[k] = *(const f32x4_t*)((const float*)(ws + lay.recs) + at * D + d);
      }
      float now = M;
#pragma unroll
      for (int k = 0; k < kJoin; k++) now = fmaxf(now, r[k].x);
      // a run of which the pair sees nothing left zeros and -inf
      const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - now);
      if (p0 > 0) {
        L *= f;
        O *= f;
      }
      M = now;
#pragma unroll
      for (int k = 0; k < kJoin; k++)
        if (p0 + k < n) {
          const float weight = r[k].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(r[k].x - now);
          L = fmaf(r[k].y, weight, L);
          O += v[k] * weight;
        }
    }
    const float inv = 1.f / L;
    *(u32x2_t*)(c.out + ((int64_t)(cut.row0 + i) * c.hq + head) * D + d) =
        u32x2_t{pack_bf2(O[0] * inv, O[1] * inv), pack_bf2(O[2] * inv, O[3] * inv)};
  }
}

// Workgroups: as many as there can be items, and one for each round of them, whose wave items are rounded up.
int64_t grid_of(const Layout& l, int hkv, int num_cus) {
  const int64_t items = (int64_t)l.caps.entries * hkv;
  return items + items / half_places(num_cus) + 2;
}

hipError_t allow_lds(const void* kernel, size_t lds) {
  return lds > 32 * 1024 ? hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) : hipSuccess;
}

template <int D, int TYPE>
hipError_t launch_type(const AttnPartsCall& c, hipStream_t s) {
  const Layout lay = layout_of(c.batch, c.max_rows, c.hq, c.kv.hkv, D, c.num_cus, c.groups > 0);
  const int waves = std::max(2, std::min(kPlanWaves, (std::max(c.batch, lay.caps.tiles + (c.groups > 0 ? lay.caps.tiles / 2 : 0)) + 63) / 64));
  const size_t plan_lds = (4 * (size_t)c.batch + 5 * (size_t)c.groups + 1) * sizeof(int32_t);
  hipError_t e = allow_lds((const void*)k_attn_parts_plan, plan_lds);
  constexpr int lds = std::max(tile_lds<D, TYPE>(), few_lds<D, TYPE ? 2 : 1>());
  if (e == hipSuccess) e = allow_lds((const void*)k_attn_parts<D, TYPE>, lds);
  if (e != hipSuccess) return e;
  k_attn_parts_plan<<<1, 64 * waves, plan_lds, s>>>(c, lay);
  k_attn_parts<D, TYPE><<<(unsigned)grid_of(lay, c.kv.hkv, c.num_cus), 256, lds, s>>>(c, lay);
  // workgroups a cut and KV head: as many as its rows need, or as fill the chip
  const int most = (std::min(tile_tokens(c.hq / c.kv.hkv), c.max_rows) * (c.hq / c.kv.hkv) + 1024 / D - 1) / (1024 / D);
  const int z = std::max<int64_t>(1, std::min<int64_t>(most, 4 * (int64_t)c.num_cus / std::max<int64_t>(1, (int64_t)lay.caps.cuts * c.kv.hkv)));
  if (lay.caps.cuts > 0) k_attn_parts_join<D><<<dim3(lay.caps.cuts, c.kv.hkv, z), 256, 0, s>>>(c, lay);
  return hipGetLastError();
}
template <int D>
hipError_t launch_d(const AttnPartsCall& c, hipStream_t s) {
  return c.kv8.type == kE4m3 ? launch_type<D, kE4m3>(c, s) : c.kv8.type == kInt8 ? launch_type<D, kInt8>(c, s) : launch_type<D, 0>(c, s);
}

}  // namespace

// 0 for more items than one launch covers: HIP's have fewer than 2^32 threads.
size_t attn_parts_ws_bytes(int batch, int max_rows, int hq, int hkv, int d, int num_cus, bool groups) {
  const Layout l = layout_of(batch, max_rows, hq, hkv, d, num_cus, groups);
  return grid_of(l, hkv, num_cus) * 256 < (int64_t)1 << 32 ? l.bytes : 0;
}

hipError_t launch_attention_parts(const AttnPartsCall& c, hipStream_t s) {
  if (c.max_rows <= 0) return hipSuccess;
  return c.kv.d == 128 ? launch_d<128>(c, s) : launch_d<64>(c, s);
}

}  // namespace sidp
