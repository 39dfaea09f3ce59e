// Log probabilities of given tokens, their ranks, the entropy and the K most
// likely tokens of every row of logits.
//
//   lse = m + log sum_i exp(x_i - m),  m = max_i x_i
//   logprob = x_t - lse,  rank = #{i : x_i > x_t},  H = lse - sum_i p_i x_i
//
// One pass: the logits are read once. A workgroup takes a segment of a row, its 4 (or 8)
// waves every 4th (8th) slice of 2048 logits of it, 32 a lane, the next slice's loads in
// flight while one is summed up. Waves do not wait for each other until the segment
// ends. A row's segments (as many as it takes to fill the chip when rows are few, else
// one) are joined in index order by a second launch.
//
// Bound by HBM where rows fill the chip: 2048 rows of 128001 bf16 logits and one
// alternative 95 us, 5.5 TB/s, where a copy reaches 4.9 (230 us with a workgroup to
// every 8192 logits, which waited at five barriers); 256 rows of 151936 fp32 logits and
// 20 alternatives 34 us, 4.6 TB/s. One row 11.5 us, the two launches.
//
// Sums are kept per lane against the lane's largest logit so far: against a smaller
// one the entropy's weighted sum would cancel. Exponents are base 2: with
// a_i = (x_i - m) log2 e, sum 2^a and sum 2^a a give lse and the entropy. The difference
// comes first (one operation more than a fused x_i log2 e - m log2 e): logits at the
// type's lowest value, as masks have them, would overflow in the product.
//
// The K best: the K-th largest of the 256 lanes' running maxima bounds the K-th
// largest logit so far from below, so only logits from that bound on are kept as
// candidates, about 1.1 K of them each time the logits seen double (when the bound is
// renewed). A key is the value's order-preserving bits, then the inverted index, so
// keys are distinct and ties go to the lowest index. Logits at -inf (a mask's) are no
// candidates; a row with fewer others than asked for is filled up from its first tokens.
#include <type_traits>

#include "common.h"
#include "internal.h"

namespace sidp {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kPerLane = 32;
constexpr int kSlice = 64 * kPerLane;  // logits that a wave takes at a time
constexpr int kCandidates = 256;       // of a wave
constexpr float kLeast = -256.f;       // 2^kLeast is 0
constexpr float kLowest = -3.40282347e+38f;  // no finite logit is lower
// Workgroups that fill the chip: a row is cut into segments only while there are fewer rows. 256 rows of 151936 fp32 logits with
// 256: 47 us, 512: 42, 1024: 42, 2048: 49.
constexpr int kGroups = 512;
// Logits of at least this many bytes are loaded past the caches: 524 MB 99.5 us (104.5 through them), 156 MB 40.1 (41.5; 40 both
// where they were in the caches already), but 19 MB from the caches 21.2 (20.7).
constexpr int64_t kOnceBytes = (int64_t)128 << 20;

typedef unsigned long long key_t;

__device__ __forceinline__ key_t make_key(float x, int index) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // -0 becomes +0: equal logits, equal order
  const uint32_t o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return (key_t)o << 32 | (uint32_t)~index;
}
__device__ __forceinline__ int key_index(key_t k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_value(key_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}

__device__ __forceinline__ key_t wave_max_key(key_t v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const key_t w = __shfl_xor(v, o, 64);
    v = w > v ? w : v;
  }
  return v;
}

// How many of keys[0 .. n) (in LDS) are above `mine`, eight reads at a time: one after the other, each would wait for its own.
__device__ __forceinline__ int above(const key_t* keys, int n, key_t mine) {
  int rank = 0, j = 0;
  for (; j + 8 <= n; j += 8) {
    key_t k[8];
#pragma unroll
    for (int u = 0; u < 8; u++) k[u] = keys[j + u];
#pragma unroll
    for (int u = 0; u < 8; u++) rank += k[u] > mine;
  }
  for (; j < n; j++) rank += keys[j] > mine;
  return rank;
}

// The largest of the wave's 64 values (none a NaN), without a trip through LDS.
__device__ __forceinline__ float row_max(float v) {
#define SIDP_ROR(n) \
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), 0x120 + n, 0xf, 0xf, true)))
  SIDP_ROR(8);
  SIDP_ROR(4);
  SIDP_ROR(2);
  SIDP_ROR(1);
#undef SIDP_ROR
  const u32x2_t a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const u32x2_t b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Sums against a reference m: of 2^a and of 2^a a; logits above the target's.
struct Stats {
  float m, l, s;
  int above;
};

// p's sums against reference `m`, which is at least p.m; a part of nothing but -inf has l = s = 0.
__device__ __forceinline__ void rebase(float m, Stats& p) {
  const float d = p.m == -INFINITY ? kLeast : fmaxf((p.m - m) * kLog2e, kLeast);
  const float f = __builtin_amdgcn_exp2f(d);
  p.s = fmaf(p.l, d, p.s) * f;
  p.l *= f;
  p.m = m;
}

// The answers of a row, from its sums and the candidates that hold its `top` best, on one workgroup.
struct Row {
  float m, logl;
  bool none;
  __device__ float logprob(float v) const { return none ? NAN : (v - m) - logl; }
};
template <bool F32>
__device__ __forceinline__ float logit_at(const LogprobCall& c, int64_t row, int i) {
  return F32 ? ((const float*)c.logits)[row * c.stride + i] : bf2f(((const uint16_t*)c.logits)[row * c.stride + i]);
}
template <bool F32, int WAVES>
__device__ __forceinline__ Row answer(const LogprobCall& c, int64_t row, const Stats& st) {
  // no distribution: a NaN or +inf among the logits (l is NaN), or nothing above -inf (l is 0)
  const Row r{st.m, logf(st.l), !(st.l > 0.f) || st.m == INFINITY};
  if (threadIdx.x == 0) {
    const int tgt = c.targets ? c.targets[row] : -1;
    const bool given = tgt >= 0 && tgt < c.vocab;
    if (c.entropy) c.entropy[row] = r.none ? NAN : fmaf(-(st.s / st.l), kLn2, r.logl);
    if (c.logprob) c.logprob[row] = given ? r.logprob(logit_at<F32>(c, row, tgt)) : NAN;
    if (c.rank) c.rank[row] = given && !r.none ? st.above : -1;
  }
  if (r.none)
    for (int i = threadIdx.x; i < c.top; i += 64 * WAVES) {
      c.top_ids[row * c.top + i] = -1;
      c.top_logprobs[row * c.top + i] = NAN;
    }
  return r;
}

// The row's best behind its `kept` finite ones: the lowest tokens at -inf, all among the first `top` (one wave).
template <bool F32>
__device__ __forceinline__ void fill_up(const LogprobCall& c, int64_t row, int kept) {
  if (kept >= c.top || threadIdx.x >= 64) return;
  const int i = threadIdx.x;
  const uint64_t masked = __ballot(i < c.top && logit_at<F32>(c, row, min(i, c.top - 1)) == -INFINITY);
  const int at = kept + __popcll(masked & ((1ull << i) - 1));
  if (masked >> i & 1 && at < c.top) {
    c.top_ids[row * c.top + at] = i;
    c.top_logprobs[row * c.top + at] = -INFINITY;
  }
}

// ONCE: non-temporal loads.
template <bool F32, bool ONCE, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 4) k_logprob(LogprobCall c) {
  constexpr int kVec = F32 ? 4 : 8;         // logits of a 16-byte piece
  constexpr int kPieces = kPerLane / kVec;  // pieces of a lane, 64 apart
  constexpr int kSlicePieces = 64 * kPieces;
  __shared__ key_t s_list[WAVES][kCandidates];
  __shared__ __attribute__((aligned(16))) key_t s_best[WAVES * kCandidates];
  __shared__ Stats s_stats[WAVES];
  __shared__ int s_n[WAVES];
  __shared__ float s_tau[WAVES];
  __shared__ volatile float s_highest[WAVES][64];  // each lane's largest logit
  __shared__ int s_kept;
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int64_t row = blockIdx.x / c.segments;
  const int segment = blockIdx.x % c.segments;
  const int es = F32 ? 4 : 2, top = c.top;
  const uintptr_t base = (uintptr_t)c.logits + (uintptr_t)(row * c.stride) * es;
  const int mis = (int)(base & 15) / es;  // pieces are whole 16-byte lines: the row starts `mis` logits into its first
  const uintptr_t aligned = base & ~(uintptr_t)15;
  const int slices = ((c.vocab + mis + kVec - 1) / kVec + kSlicePieces - 1) / kSlicePieces;
  const int first = (int)((int64_t)slices * segment / c.segments), last = (int)((int64_t)slices * (segment + 1) / c.segments);
  if (t == 0) s_kept = 0;
  s_highest[wave][lane] = -INFINITY;
  __syncthreads();

  float xt = INFINITY;
  if (c.targets) {
    const int tgt = c.targets[row];
    if (tgt >= 0 && tgt < c.vocab) xt = logit_at<F32>(c, row, tgt);
  }

  // Piece j of the lane in a slice; where the row's start or end cuts it, logit by logit, -inf outside.
  auto first_of = [&](int slice, int j) { return (slice * kSlicePieces + j * 64 + lane) * kVec - mis; };
  auto load_piece = [&](int e0) {
    if (e0 >= 0 && e0 + kVec <= c.vocab) return *(const u32x4_t*)(base + (intptr_t)e0 * es);
    u32x4_t raw;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if (F32) {
        const int e = e0 + i;
        raw[i] = e >= 0 && e < c.vocab ? ((const uint32_t*)base)[e] : 0xff800000u;
      } else {
        const int e = e0 + 2 * i;
        const uint32_t lo = e >= 0 && e < c.vocab ? ((const uint16_t*)base)[e] : 0xff80u;
        const uint32_t hi = e + 1 >= 0 && e + 1 < c.vocab ? ((const uint16_t*)base)[e + 1] : 0xff80u;
        raw[i] = lo | hi << 16;
      }
    }
    return raw;
  };
  auto load = [&](int slice, u32x4_t (&raw)[kPieces]) {
    const int p0 = slice * kSlicePieces;
    if (p0 * kVec >= mis && (p0 + kSlicePieces) * kVec - mis <= c.vocab) {
#pragma unroll
      for (int j = 0; j < kPieces; j++) {
        const auto from = (const u32x4_t*)(aligned + (uintptr_t)(p0 + j * 64 + lane) * 16);
        raw[j] = ONCE ? __builtin_nontemporal_load(from) : *from;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kPieces; j++) raw[j] = load_piece(first_of(slice, j));
    }
  };
  auto value = [](const u32x4_t& raw, int i) {
    return __uint_as_float(F32 ? raw[i] : i & 1 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
  };

  Stats st{-INFINITY, 0.f, 0.f, 0};
  float highest = -INFINITY;  // of the lane
  float tau = kLowest;        // logits below it are not among the best; equal ones from token tau_index on neither
  int tau_index = 0x7fffffff;
  int n = 0, done = 0;        // candidates of the wave, slices it has seen
  key_t* const list = s_list[wave];

  u32x4_t raw[kPieces];
  if (first + wave < last) load(first + wave, raw);
  for (int slice = first + wave; slice < last; slice += WAVES) {
    float x[kPerLane], piece_max[kPieces];
#pragma unroll
    for (int i = 0; i < kPerLane; i++) x[i] = value(raw[i / kVec], i % kVec);
    if (slice + WAVES < last) load(slice + WAVES, raw);
#pragma unroll
    for (int j = 0; j < kPieces; j++) {
      piece_max[j] = x[j * kVec];
#pragma unroll
      for (int i = 1; i < kVec; i++) piece_max[j] = fmaxf(piece_max[j], x[j * kVec + i]);
    }
    float most = piece_max[0];
#pragma unroll
    for (int j = 1; j < kPieces; j++) most = fmaxf(most, piece_max[j]);
    if (most > st.m) rebase(most, st);

    // a NaN logit, or inf - inf, makes p and with it l NaN
    const float ref = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
    for (int i = 0; i < kPerLane; i++) {
      const float a = (x[i] - ref) * kLog2e;
      const float p = __builtin_amdgcn_exp2f(a);
      st.l += p;
      st.s = fmaf(p, fmaxf(a, kLeast), st.s);  // 2^-inf (-inf) is 0
    }
    if (__any(most > xt)) {
#pragma unroll
      for (int i = 0; i < kPerLane; i++) st.above += __popcll(__ballot(x[i] > xt));
    }
    if (top == 0) continue;

    highest = fmaxf(highest, most);
    done++;
    if ((done & (done - 1)) == 0) {
      // A bound that at least `top` of the workgroup's lanes' running maxima reach, by bisection between the least and the largest of
      // them (to 2^-8 of their distance: a few candidates more than with the top-th largest itself, for a quarter of its price).
      // Other waves' maxima may be old ones: those hold as well, so nobody waits.
      s_highest[wave][lane] = highest;
      float h[WAVES], least = INFINITY, hi = -INFINITY;
#pragma unroll
      for (int w = 0; w < WAVES; w++) {
        h[w] = s_highest[w][lane];
        hi = fmaxf(hi, h[w]);
        least = fminf(least, h[w] > -INFINITY ? h[w] : INFINITY);
      }
      auto reach = [&](float v) {
        int k = 0;
#pragma unroll
        for (int w = 0; w < WAVES; w++) k += __popcll(__ballot(h[w] >= v));
        return k;
      };
      float bound = -INFINITY;
      if (reach(kLowest) >= top) {
        hi = row_max(hi);
        bound = top == 1 ? hi : -row_max(-least);
        for (int i = 0; top > 1 && i < 8; i++) {
          const float mid = 0.5f * bound + 0.5f * hi;
          if (reach(mid) >= top) bound = mid;
          else hi = mid;
        }
      }
      if (bound > tau) {
        tau = bound;
        tau_index = 0x7fffffff;
      }
    }
    if (!__any(most >= tau)) continue;
    if (tau_index == 0x7fffffff) {  // as nearly always
      int count = 0;  // at most, by pieces; counted one by one only where that is too many
#pragma unroll
      for (int j = 0; j < kPieces; j++) count += kVec * __popcll(__ballot(piece_max[j] >= tau));
      if (n + count > kCandidates) {
        count = 0;
#pragma unroll
        for (int i = 0; i < kPerLane; i++) count += __popcll(__ballot(x[i] >= tau));
      }
      if (n + count <= kCandidates) {
        float bound = tau;
        asm volatile("" : "+v"(bound));  // the comparisons are made again rather than kept
        const int e0 = first_of(slice, 0);
#pragma unroll
        for (int j = 0; j < kPieces; j++)
          if (__any(piece_max[j] >= bound)) {
#pragma unroll
            for (int i = j * kVec; i < (j + 1) * kVec; i++) {
              const bool take = x[i] >= bound;
              const uint64_t who = __ballot(take);
              if (who) {
                if (take) list[n + __popcll(who & ((1ull << lane) - 1))] = make_key(x[i], e0 + j * (64 * kVec) + i % kVec);
                n += __popcll(who);
              }
            }
          }
        continue;
      }
    }
    // A bound with an index, or more candidates than the list holds: the slice again from memory.
    auto takes = [&](float v, int e) { return v > tau || (v == tau && e < tau_index); };
    int count = 0;
#pragma unroll 1
    for (int j = 0; j < kPieces; j++) {
      const int e0 = first_of(slice, j);
      const u32x4_t again = load_piece(e0);
#pragma unroll
      for (int i = 0; i < kVec; i++) count += __popcll(__ballot(takes(value(again, i), e0 + i)));
    }
    if (n + count <= kCandidates) {
#pragma unroll 1
      for (int j = 0; j < kPieces; j++) {
        const int e0 = first_of(slice, j);
        const u32x4_t again = load_piece(e0);
#pragma unroll
        for (int i = 0; i < kVec; i++) {
          const bool take = takes(value(again, i), e0 + i);
          const uint64_t who = __ballot(take);
          if (take) list[n + __popcll(who & ((1ull << lane) - 1))] = make_key(value(again, i), e0 + i);
          n += __popcll(who);
        }
      }
      continue;
    }
    // Many equal logits, or ever larger ones: the best of list and slice, one after the other, become the list, and the last of
    // them the bound.
    key_t prev = ~(key_t)0, kept = 0;
    for (int r = 0; r < top; r++) {
      key_t best = 0;
      for (int i = lane; i < n; i += 64) {
        const key_t k = list[i];
        if (k < prev && k > best) best = k;
      }
#pragma unroll 1
      for (int j = 0; j < kPieces; j++) {
        const int e0 = first_of(slice, j);
        const u32x4_t again = load_piece(e0);
#pragma unroll
        for (int i = 0; i < kVec; i++) {
          const key_t k = takes(value(again, i), e0 + i) ? make_key(value(again, i), e0 + i) : 0;
          if (k < prev && k > best) best = k;
        }
      }
      prev = wave_max_key(best);
      if (lane == r) kept = prev;
    }
    if (lane < top) list[lane] = kept;
    n = top;
    tau = key_value(prev);
    tau_index = key_index(prev);
  }

  // join the lanes, then the waves, in order
  {
    const float m = wave_max(st.m);
    rebase(m, st);
    st.l = wave_sum(st.l);
    st.s = wave_sum(st.s);
    if (lane == 0) {
      s_stats[wave] = st;
      s_n[wave] = n;
      s_tau[wave] = tau;
    }
  }
  __syncthreads();
  Stats all = s_stats[0];
  float m = all.m, bound = s_tau[0];
#pragma unroll
  for (int w = 1; w < WAVES; w++) {
    m = fmaxf(m, s_stats[w].m);
    bound = fmaxf(bound, s_tau[w]);  // every wave's bound holds for all
  }
  rebase(m, all);
#pragma unroll
  for (int w = 1; w < WAVES; w++) {
    Stats p = s_stats[w];
    rebase(m, p);
    all.l += p.l;
    all.s += p.s;
    all.above += p.above;
  }
  const bool whole = c.segments == 1;
  Row r{0.f, 0.f, false};
  if (whole) r = answer<F32, WAVES>(c, row, all);
  else if (t == 0) ((Stats*)c.stats)[blockIdx.x] = all;
  if (top == 0 || r.none) return;
  for (int i = lane; i < s_n[wave]; i += 64)
    if (key_value(list[i]) >= bound) s_best[atomicAdd(&s_kept, 1)] = list[i];
  __syncthreads();
  const int kept = s_kept;
  key_t* keys = (key_t*)c.keys + (int64_t)blockIdx.x * top;
  for (int i = t; i < kept; i += 64 * WAVES) {
    const key_t mine = s_best[i];
    const int rank = above(s_best, kept, mine);
    if (rank >= top) continue;
    if (whole) {
      c.top_ids[row * top + rank] = key_index(mine);
      c.top_logprobs[row * top + rank] = r.logprob(key_value(mine));
    } else {
      keys[rank] = mine;
    }
  }
  if (whole) fill_up<F32>(c, row, kept);
  else
    for (int i = kept + t; i < top; i += 64 * WAVES) keys[i] = 0;  // fewer candidates in the segment than asked for
}

// One workgroup a row. Segments are joined in index order, thread by thread.
template <bool F32>
__global__ void __launch_bounds__(256) k_logprob_join(LogprobCall c) {
  extern __shared__ __attribute__((aligned(16))) key_t s_keys[];  // [segments * top]
  __shared__ Stats s_stats[4];
  __shared__ key_t s_bound[4];
  __shared__ int s_n;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int64_t row = blockIdx.x;
  const Stats* parts = (const Stats*)c.stats + row * c.segments;
  const key_t* keys = (const key_t*)c.keys + row * c.segments * (int64_t)c.top;
  if (t == 0) s_n = 0;
  Stats st{-INFINITY, 0.f, 0.f, 0};
  key_t bound = 0;  // every segment holds `top` keys no smaller than its last one
  for (int i = t; i < c.segments; i += 256) {
    Stats p = parts[i];
    const float m = fmaxf(st.m, p.m);
    rebase(m, st);
    rebase(m, p);
    st.l += p.l;
    st.s += p.s;
    st.above += p.above;
    if (c.top > 0) {
      const key_t k = keys[(int64_t)i * c.top + c.top - 1];
      bound = k > bound ? k : bound;
    }
  }
  {
    const float m = wave_max(st.m);
    rebase(m, st);
    st.l = wave_sum(st.l);
    st.s = wave_sum(st.s);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) st.above += __shfl_xor(st.above, o, 64);
    bound = wave_max_key(bound);
    if (lane == 0) {
      s_stats[wave] = st;
      s_bound[wave] = bound;
    }
  }
  __syncthreads();
  Stats all = s_stats[0];
  float m = all.m;
#pragma unroll
  for (int w = 1; w < 4; w++) m = fmaxf(m, s_stats[w].m);
  rebase(m, all);
#pragma unroll
  for (int w = 1; w < 4; w++) {
    Stats p = s_stats[w];
    rebase(m, p);
    all.l += p.l;
    all.s += p.s;
    all.above += p.above;
  }
#pragma unroll
  for (int w = 0; w < 4; w++) bound = s_bound[w] > bound ? s_bound[w] : bound;
  const Row r = answer<F32, 4>(c, row, all);
  if (c.top == 0 || r.none) return;
  for (int i0 = t; i0 < c.segments * c.top; i0 += 4 * 256) {
    key_t k[4];
#pragma unroll
    for (int u = 0; u < 4; u++) k[u] = i0 + u * 256 < c.segments * c.top ? keys[i0 + u * 256] : 0;
#pragma unroll
    for (int u = 0; u < 4; u++)
      if (k[u] >= bound && k[u]) s_keys[atomicAdd(&s_n, 1)] = k[u];
  }
  __syncthreads();
  const int n = s_n;
  for (int i = t; i < n; i += 256) {
    const key_t mine = s_keys[i];
    const int rank = above(s_keys, n, mine);
    if (rank < c.top) {
      c.top_ids[row * c.top + rank] = key_index(mine);
      c.top_logprobs[row * c.top + rank] = r.logprob(key_value(mine));
    }
  }
  fill_up<F32>(c, row, n);
}

// How a call is cut: one segment a row while rows alone fill the chip, or while workgroups of 8 waves (wide) do nearly, which
// saves the second launch; else enough segments to, of at least a slice for each wave. Wide / two or three segments, us, fp32 of
// 151936 and bf16 of 128001: 256 rows 35.4 / 39.6 and 27.6 / 30.5, 300 49.4 / 48.0 and 35.8 / 35.8, 500 56.6 / 62.5 and 28.1 /
// 31.9 (no alternatives), 180 of 128001 28.8 / 30.0 and 27.3 / 27.6. From 512 rows on 4 waves: 540 rows of bf16 47.9, wide 51.4.
struct Plan {
  bool wide;
  int segments;
};
Plan plan_of(int rows, int vocab) {
  const int most = (vocab + 4 * kSlice - 1) / (4 * kSlice), want = (kGroups + rows - 1) / rows;
  const bool wide = (want == 2 || want == 3) && most > 1;
  return Plan{wide, wide ? 1 : std::min(most, want)};
}

}  // namespace

size_t logprob_ws_bytes(int rows, int vocab, int top) {
  const int segments = plan_of(rows, vocab).segments;
  // the smallest size is asked for as well: a workspace is never empty
  return std::max<size_t>(16, segments == 1 ? 0 : (size_t)rows * segments * (sizeof(Stats) + (size_t)top * sizeof(key_t)));
}

hipError_t launch_logprobs(LogprobCall c, hipStream_t s) {
  if (c.rows <= 0) return hipSuccess;
  const Plan plan = plan_of(c.rows, c.vocab);
  c.segments = plan.segments;
  c.stats = c.ws;
  c.keys = (char*)c.ws + (size_t)c.rows * c.segments * sizeof(Stats);
  const dim3 grid((unsigned)((int64_t)c.rows * c.segments));
  const size_t lds = (size_t)c.segments * c.top * sizeof(key_t);
  const bool once = (int64_t)c.rows * c.vocab * (c.f32 ? 4 : 2) >= kOnceBytes;
  auto launch = [&](auto f32, auto past) {
    constexpr bool F32 = decltype(f32)::value, ONCE = decltype(past)::value;
    if (plan.wide) k_logprob<F32, ONCE, 8><<<grid, 512, 0, s>>>(c);
    else k_logprob<F32, ONCE, 4><<<grid, 256, 0, s>>>(c);
  };
  const std::true_type yes;
  const std::false_type no;
  if (c.f32) once ? launch(yes, yes) : launch(yes, no);
  else once ? launch(no, yes) : launch(no, no);
  if (c.segments > 1) {
    if (c.f32) k_logprob_join<true><<<c.rows, 256, lds, s>>>(c);
    else k_logprob_join<false><<<c.rows, 256, lds, s>>>(c);
  }
  return hipGetLastError();
}

}  // namespace sidp
