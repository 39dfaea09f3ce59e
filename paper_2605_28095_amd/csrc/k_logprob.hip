// Log probabilities of given tokens, their ranks, the entropy and the K most
// likely tokens of every row of logits.
//
//   lse = m + log sum_i exp(x_i - m),  m = max_i x_i
//   logprob = x_t - lse,  rank = #{i : x_i > x_t},  H = lse - sum_i p_i x_i
//
// A row is cut into slices of 8192 logits; a workgroup keeps one in registers
// (32 a thread), so the logits are read once, a single row already fills as many
// CUs as it has slices, and every reduction is within one workgroup. It leaves
// (max, sum, weighted sum, count) and the slice's K best as sorted keys; a second
// launch joins a row's slices in slice order. Exponents are base 2: with a_i =
// (x_i - m) log2 e, sum 2^a and sum 2^a a give lse and the entropy. The difference
// comes first (one operation more than a fused x_i log2 e - m log2 e): logits at
// the type's lowest value, as masks have them, would overflow in the product.
//
// The K best of a slice: the K-th largest of the maxima of 64 groups of 128
// logits bounds the K-th largest logit from below, so only logits from that bound
// on are candidates (about 1.3 K of them), each ranked against the others. A key is
// the value's order-preserving bits, then the inverted index, so keys are distinct
// and ties go to the lowest index.
#include "common.h"
#include "internal.h"

namespace sidp {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kSlice = 8192;       // logits of a workgroup
constexpr int kPerThread = 32;     // of a thread
constexpr int kCandidates = 1024;  // of a slice; past that (thousands of equal logits) one round per rank
constexpr float kLeast = -256.f;   // 2^kLeast is 0

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

// Slice statistics: max, sum of 2^a, sum of 2^a a, logits above the target's.
struct Stats {
  float m, l, s;
  int above;
};

template <bool F32>
__global__ void __launch_bounds__(256) k_logprob_slice(LogprobCall c) {
  constexpr int kVec = F32 ? 4 : 8;             // logits of a 16-byte piece
  constexpr int kPieces = kPerThread / kVec;    // pieces of a thread, 256 apart
  __shared__ float s_max[4], s_group[64], s_tau;
  __shared__ float s_l[4], s_s[4];
  __shared__ int s_above[4];
  __shared__ int s_n;
  __shared__ key_t s_cand[kCandidates];
  __shared__ key_t s_best[4];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int64_t row = blockIdx.x / c.slices;
  const int slice = blockIdx.x % c.slices;
  const int es = F32 ? 4 : 2;
  const uintptr_t base = (uintptr_t)c.logits + (uintptr_t)(row * c.stride) * es;
  const int mis = (int)(base & 15) / es;  // pieces are whole 16-byte lines: the row starts `mis` logits into its first
  const uintptr_t aligned = base & ~(uintptr_t)15;
  const int first = max(0, slice * kSlice - mis);  // the slice's first token

  float x[kPerThread];
#pragma unroll
  for (int j = 0; j < kPieces; j++) {
    const int piece = slice * (kSlice / kVec) + j * 256 + t;
    const int e0 = piece * kVec - mis;
    if (e0 >= 0 && e0 + kVec <= c.vocab) {
      const u32x4_t u = *(const u32x4_t*)(aligned + (uintptr_t)piece * 16);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        if (F32) {
          x[j * kVec + i] = __uint_as_float(u[i]);
        } else {
          x[j * kVec + 2 * i] = bf2f((uint16_t)(u[i] & 0xffffu));
          x[j * kVec + 2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
      }
    } else {  // a piece that the row's start or end cuts
#pragma unroll
      for (int i = 0; i < kVec; i++) {
        const int e = e0 + i;
        float v = -INFINITY;
        if (e >= 0 && e < c.vocab) {
          if (F32) v = ((const float*)base)[e];
          else v = bf2f(((const uint16_t*)base)[e]);
        }
        x[j * kVec + i] = v;
      }
    }
  }
  float xt = INFINITY;
  if (c.targets) {
    const int tgt = c.targets[row];
    if (tgt >= 0 && tgt < c.vocab) xt = F32 ? ((const float*)base)[tgt] : bf2f(((const uint16_t*)base)[tgt]);
  }

  float tm = x[0];
#pragma unroll
  for (int i = 1; i < kPerThread; i++) tm = fmaxf(tm, x[i]);
  // maxima of four threads each, and of the wave
  float gm = fmaxf(tm, __shfl_xor(tm, 1, 64));
  gm = fmaxf(gm, __shfl_xor(gm, 2, 64));
  if ((lane & 3) == 0) s_group[t >> 2] = gm;
  const float wm = wave_max(gm);
  if (lane == 0) s_max[wave] = wm;
  if (t == 0) s_n = 0;
  __syncthreads();
  const float m = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
  const float ref = m == -INFINITY ? 0.f : m;

  if (wave == 0 && c.top > 0) {
    // the largest bound that at least `top` group maxima reach
    const float g = s_group[lane];
    int above = 0;
#pragma unroll
    for (int j = 0; j < 64; j++) above += __shfl(g, j, 64) > g;
    float tau = above < c.top ? g : INFINITY;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) tau = fminf(tau, __shfl_xor(tau, o, 64));
    if (lane == 0) s_tau = tau;
  }

  // a NaN logit, or inf - inf, makes p and with it l NaN
  float l = 0.f, s = 0.f;
  int above = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; i++) {
    const float a = (x[i] - ref) * kLog2e;
    const float p = __builtin_amdgcn_exp2f(a);
    l += p;
    s = fmaf(p, fmaxf(a, kLeast), s);  // 2^-inf (-inf) is 0
    above += __popcll(__ballot(x[i] > xt));
  }
  l = wave_sum(l);
  s = wave_sum(s);
  if (lane == 0) {
    s_l[wave] = l;
    s_s[wave] = s;
    s_above[wave] = above;
  }
  __syncthreads();
  if (t == 0) {
    Stats st;
    st.m = m;
    st.l = ((s_l[0] + s_l[1]) + s_l[2]) + s_l[3];
    st.s = ((s_s[0] + s_s[1]) + s_s[2]) + s_s[3];
    st.above = s_above[0] + s_above[1] + s_above[2] + s_above[3];
    ((Stats*)c.stats)[blockIdx.x] = st;
  }
  if (c.top <= 0) return;

  const float tau = s_tau;
  // Of equal logits only the first `top` count, so of those at -inf (a mask's) only ones among the slice's first `top`.
  auto takes = [&](float v, int e) { return v >= tau && e >= 0 && e < c.vocab && (v > -INFINITY || e - first < c.top); };
  if (tm >= tau) {
#pragma unroll
    for (int i = 0; i < kPerThread; i++) {
      if (x[i] >= tau) {
        const int e = (slice * (kSlice / kVec) + (i / kVec) * 256 + t) * kVec - mis + i % kVec;
        if (takes(x[i], e)) {
          const int at = atomicAdd(&s_n, 1);
          if (at < kCandidates) s_cand[at] = make_key(x[i], e);
        }
      }
    }
  }
  __syncthreads();
  const int n = s_n;
  key_t* out = (key_t*)c.keys + (int64_t)blockIdx.x * c.top;
  if (n <= kCandidates) {
    for (int i = t; i < n; i += 256) {
      const key_t mine = s_cand[i];
      int rank = 0;
      for (int j = 0; j < n; j++) rank += s_cand[j] > mine;
      if (rank < c.top) out[rank] = mine;
    }
    for (int i = n + t; i < c.top; i += 256) out[i] = 0;  // fewer logits in the slice than asked for
  } else {
    key_t prev = ~(key_t)0;
    for (int r = 0; r < c.top; r++) {
      key_t best = 0;
#pragma unroll
      for (int i = 0; i < kPerThread; i++) {
        const int e = (slice * (kSlice / kVec) + (i / kVec) * 256 + t) * kVec - mis + i % kVec;
        const key_t k = takes(x[i], e) ? make_key(x[i], e) : 0;
        if (k < prev && k > best) best = k;
      }
      best = wave_max_key(best);
      if (lane == 0) s_best[wave] = best;
      __syncthreads();
      best = s_best[0];
#pragma unroll
      for (int w = 1; w < 4; w++) best = s_best[w] > best ? s_best[w] : best;
      if (t == 0) out[r] = best;
      prev = best;
      __syncthreads();
    }
  }
}

// One workgroup a row. Slices are joined in index order, thread by thread.
template <bool F32>
__global__ void __launch_bounds__(256) k_logprob_join(LogprobCall c) {
  extern __shared__ __attribute__((aligned(16))) key_t s_keys[];  // [slices * top]
  __shared__ float s_m[4], s_l[4], s_s[4];
  __shared__ int s_above[4];
  __shared__ key_t s_bound[4];
  __shared__ int s_n;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int64_t row = blockIdx.x;
  const Stats* st = (const Stats*)c.stats + row * c.slices;
  const key_t* keys = (const key_t*)c.keys + row * c.slices * (int64_t)c.top;
  if (t == 0) s_n = 0;
  float m = -INFINITY;
  key_t bound = 0;  // every slice holds `top` keys no smaller than its last one
  for (int i = t; i < c.slices; i += 256) {
    m = fmaxf(m, st[i].m);
    if (c.top > 0) {
      const key_t k = keys[(int64_t)i * c.top + c.top - 1];
      bound = k > bound ? k : bound;
    }
  }
  m = wave_max(m);
  bound = wave_max_key(bound);
  if (lane == 0) {
    s_m[wave] = m;
    s_bound[wave] = bound;
  }
  __syncthreads();
  m = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
#pragma unroll
  for (int w = 0; w < 4; w++) bound = s_bound[w] > bound ? s_bound[w] : bound;
  float l = 0.f, s = 0.f;
  int above = 0;
  for (int i = t; i < c.slices; i += 256) {
    const Stats p = st[i];
    const float d = p.m == -INFINITY ? 0.f : (p.m - m) * kLog2e;  // a slice of -inf alone has l = s = 0
    const float f = __builtin_amdgcn_exp2f(d);
    l = fmaf(p.l, f, l);
    s = fmaf(fmaf(p.l, fmaxf(d, kLeast), p.s), f, s);
    above += p.above;
  }
  l = wave_sum(l);
  s = wave_sum(s);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) above += __shfl_xor(above, o, 64);
  if (lane == 0) {
    s_l[wave] = l;
    s_s[wave] = s;
    s_above[wave] = above;
  }
  if (c.top > 0)
    for (int i = t; i < c.slices * c.top; i += 256) {
      const key_t k = keys[i];
      if (k >= bound && k) s_keys[atomicAdd(&s_n, 1)] = k;
    }
  __syncthreads();
  l = ((s_l[0] + s_l[1]) + s_l[2]) + s_l[3];
  s = ((s_s[0] + s_s[1]) + s_s[2]) + s_s[3];
  // no distribution: a NaN or +inf among the logits, or nothing above -inf
  const bool none = !(l > 0.f) || m == INFINITY;
  const float logl = logf(l);
  auto logprob = [&](float v) { return none ? NAN : (v - m) - logl; };
  if (t == 0) {
    if (c.entropy) c.entropy[row] = none ? NAN : fmaf(-(s / l), kLn2, logl);
    const int tgt = c.targets ? c.targets[row] : -1;
    const bool given = tgt >= 0 && tgt < c.vocab;
    if (c.logprob) {
      float v = NAN;
      if (given) {
        const uintptr_t base = (uintptr_t)c.logits + (uintptr_t)(row * c.stride) * (F32 ? 4 : 2);
        v = logprob(F32 ? ((const float*)base)[tgt] : bf2f(((const uint16_t*)base)[tgt]));
      }
      c.logprob[row] = v;
    }
    if (c.rank) c.rank[row] = given && !none ? s_above[0] + s_above[1] + s_above[2] + s_above[3] : -1;
  }
  const int n = s_n;
  int32_t* ids = c.top_ids + row * c.top;
  float* lps = c.top_logprobs + row * c.top;
  if (none) {
    for (int i = t; i < c.top; i += 256) {
      ids[i] = -1;
      lps[i] = NAN;
    }
    return;
  }
  for (int i = t; i < n; i += 256) {
    const key_t mine = s_keys[i];
    int rank = 0;
    for (int j = 0; j < n; j++) rank += s_keys[j] > mine;
    if (rank < c.top) {
      ids[rank] = key_index(mine);
      lps[rank] = logprob(key_value(mine));
    }
  }
}

}  // namespace

int logprob_slices(int vocab, bool f32) { return (int)(((int64_t)vocab + (f32 ? 3 : 7) + kSlice - 1) / kSlice); }

size_t logprob_ws_bytes(int rows, int vocab, int top) {
  const size_t parts = (size_t)rows * std::max(logprob_slices(vocab, true), logprob_slices(vocab, false));
  return parts * (sizeof(Stats) + (size_t)top * sizeof(key_t));
}

hipError_t launch_logprobs(LogprobCall c, hipStream_t s) {
  if (c.rows <= 0) return hipSuccess;
  c.slices = logprob_slices(c.vocab, c.f32);
  c.stats = c.ws;
  c.keys = (char*)c.ws + (size_t)c.rows * c.slices * sizeof(Stats);
  const size_t lds = (size_t)c.slices * c.top * sizeof(key_t);
  const dim3 grid((unsigned)((int64_t)c.rows * c.slices));
  if (c.f32) {
    k_logprob_slice<true><<<grid, 256, 0, s>>>(c);
    k_logprob_join<true><<<c.rows, 256, lds, s>>>(c);
  } else {
    k_logprob_slice<false><<<grid, 256, 0, s>>>(c);
    k_logprob_join<false><<<c.rows, 256, lds, s>>>(c);
  }
  return hipGetLastError();
}

}  // namespace sidp
