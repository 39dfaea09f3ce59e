// A token of each row of logits, drawn by temperature, top-k, top-p and min-p from a
// given random number.
//
// Tokens are in order of their logits, of equal ones the lowest first. With the largest
// logit m and weights w_i = exp((x_i - m) / T), each setting keeps a front of that order:
//   top-k  its first k tokens, of weight K together
//   top-p  those with less than p K in front of them (the first one always)
//   min-p  those with w_i >= min_p
// and the token drawn is the first of the n that all keep at which their running weight
// exceeds u times their weight together.
//
// Weights are whole multiples of 2^-43 of the largest, from exponents in 64 bits, so that
// sums are exact in any order, and a draw is the same however a row is read. (With sums
// of 32 bits one draw in a hundred or so over 10^5 alike tokens would be a neighbour's.)
//
// No row is sorted. A histogram over the exponents, 2048 bins of counts and weights, says
// in which bin a count or a weight is reached; only that bin's tokens, or those of all
// bins up to it where they are few, are picked out and put in order. A bin with too many
// (equal logits) is divided by its tokens' order until it has few.
#include <type_traits>

#include "common.h"
#include "internal.h"

namespace sidp {

namespace {

typedef unsigned long long u64;

constexpr int kThreads = 1024, kWavesOf = kThreads / 64;
constexpr int kBins = 2048;
constexpr float kReach = 44.f;   // weights of 2^-kReach and less are 0
constexpr int kUnit = 43;        // bits behind the point of a weight: 2^20 tokens of 2^43 are 2^63
constexpr int kList = 4096;      // tokens picked out of a row at once
constexpr int kSub = 1024;       // tokens of a bin that are put in order

// The order of tokens: larger keys first.
__device__ __forceinline__ u64 make_key(float x, int index) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // -0 becomes +0: equal logits, equal order
  const uint32_t o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return (u64)o << 32 | (uint32_t)~index;
}
__device__ __forceinline__ int key_index(u64 k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_value(u64 k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}

// A row's settings, and what a logit weighs under them.
struct Scale {
  float m;
  double c;     // log2(e) / T
  float bins;   // bins a unit of x
  double most;  // the largest exponent that min_p keeps
  __device__ __forceinline__ double exponent(float x) const { return ((double)m - (double)x) * c; }
  // Bins follow the order: each step is monotone.
  __device__ __forceinline__ int bin(float x) const { return (int)fminf((m - x) * bins, (float)(kBins - 1)); }
};

// 2^-d in units of 2^-kUnit, to the nearest; d >= 0. The fraction by Taylor's series of exp: the first term left out is
// (ln 2 / 2)^11 / 11! < 2^-42 of the weight.
__device__ __forceinline__ u64 weight_of(double d) {
  if (!(d < kReach + 0.5)) return 0;
  const double n = __builtin_rint(d), f = (n - d) * 0.6931471805599453;
  double p = 1.0 / 3628800;
  p = __builtin_fma(p, f, 1.0 / 362880);
  p = __builtin_fma(p, f, 1.0 / 40320);
  p = __builtin_fma(p, f, 1.0 / 5040);
  p = __builtin_fma(p, f, 1.0 / 720);
  p = __builtin_fma(p, f, 1.0 / 120);
  p = __builtin_fma(p, f, 1.0 / 24);
  p = __builtin_fma(p, f, 1.0 / 6);
  p = __builtin_fma(p, f, 0.5);
  p = __builtin_fma(p, f, 1.0);
  p = __builtin_fma(p, f, 1.0);
  p = __builtin_amdgcn_ldexp(p, kUnit - (int)n) + 0x1p52;  // the sum's last bit is one unit
  return (u64)__builtin_bit_cast(int64_t, p) & ((1ull << 52) - 1);
}

// f(logit, index) for every logit of a row, 16 bytes a load where its address allows.
template <bool F32, class F>
__device__ __forceinline__ void each_logit(const void* row, int n, const F& f) {
  constexpr int kSize = F32 ? 4 : 2, V = 16 / kSize, U = 4;
  const int t = threadIdx.x;
  auto at = [&](int i) { return F32 ? ((const float*)row)[i] : bf2f(((const uint16_t*)row)[i]); };
  const int head = min(n, (int)(-(uintptr_t)row & 15) / kSize), vectors = (n - head) / V, tail = head + vectors * V;
  if (t < head) f(at(t), t);
  const u32x4_t* v = (const u32x4_t*)((const char*)row + head * kSize);
  for (int j0 = 0; j0 < vectors; j0 += kThreads * U) {
    u32x4_t w[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int j = j0 + u * kThreads + t;
      if (j < vectors) w[u] = v[j];
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int j = j0 + u * kThreads + t;
      if (j < vectors) {
#pragma unroll
        for (int k = 0; k < V; k++) {
          const float x = F32 ? __uint_as_float(w[u][k % 4]) : __uint_as_float(k % 2 ? w[u][k / 2] & 0xffff0000u : w[u][k / 2] << 16);
          f(x, head + j * V + k);
        }
      }
    }
  }
  if (t < n - tail) f(at(tail + t), tail + t);
}

struct Histogram {
  u64 weight[kBins];
  uint32_t count[kBins];
};
struct Memory {
  Histogram all;  // running sums, once they are made
  union {
    u64 list[kList];
    Histogram part;  // of one bin that has too many tokens
  };
  u64 sub[kSub], sub_weight[kSub];
  u64 wave_a[kWavesOf], wave_b[kWavesOf];
  u64 found_key, found_weight;
  uint32_t found_count, filled, listed;
  int bin;
};
// LDS is addressed as such, through its own name in code that is inlined: a flat access decides by its address register alone
// whether it goes to LDS, and the compiler may put a register 8 bytes in front of what it addresses.
__device__ __forceinline__ Memory& memory() {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  return *(Memory*)smem;
}
// a place in the order: its token, and the tokens and weight up to and with it
struct Place {
  u64 key, weight;
  uint32_t count;
};

__device__ __forceinline__ u64 wave_max_u64(u64 v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const u64 w = __shfl_xor(v, o, 64);
    v = w > v ? w : v;
  }
  return v;
}
// The largest of all threads' values; every thread calls.
__device__ __forceinline__ u64 group_max(u64 v) {
  Memory& m = memory();
  v = wave_max_u64(v);
  if ((threadIdx.x & 63) == 0) m.wave_a[threadIdx.x >> 6] = v;
  __syncthreads();
  for (int w = 0; w < kWavesOf; w++) v = m.wave_a[w] > v ? m.wave_a[w] : v;
  __syncthreads();
  return v;
}

__device__ __forceinline__ void clear(Histogram& h) {
  for (int i = threadIdx.x; i < kBins; i += kThreads) h.weight[i] = 0, h.count[i] = 0;
}
// A histogram's running sums, in its place.
__device__ __forceinline__ void run_up(Histogram& h) {
  Memory& m = memory();
  constexpr int kPer = kBins / kThreads;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  u64 w[kPer], sw = 0;
  uint32_t c[kPer], sc = 0;
#pragma unroll
  for (int i = 0; i < kPer; i++) {
    w[i] = sw += h.weight[t * kPer + i];
    c[i] = sc += h.count[t * kPer + i];
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 a = __shfl_up(sw, o, 64);
    const uint32_t b = (uint32_t)__shfl_up((int)sc, o, 64);
    if (lane >= o) sw += a, sc += b;
  }
  if (lane == 63) m.wave_a[wave] = sw, m.wave_b[wave] = sc;
  sw -= w[kPer - 1];
  sc -= c[kPer - 1];
  __syncthreads();
  for (int i = 0; i < wave; i++) sw += m.wave_a[i], sc += (uint32_t)m.wave_b[i];
#pragma unroll
  for (int i = 0; i < kPer; i++) h.weight[t * kPer + i] = sw + w[i], h.count[t * kPer + i] = sc + c[i];
  __syncthreads();
}
// The bin of running sums `h` in which `target` is reached, by count or by weight. It is, in one.
__device__ __forceinline__ int bin_of(const Histogram& h, bool by_count, u64 target) {
  Memory& m = memory();
  for (int i = threadIdx.x; i < kBins; i += kThreads) {
    const u64 to = by_count ? h.count[i] : h.weight[i], from = i == 0 ? 0 : by_count ? h.count[i - 1] : h.weight[i - 1];
    if (from < target && target <= to) m.bin = i;
  }
  __syncthreads();
  const int b = m.bin;
  __syncthreads();
  return b;
}

// Where the count or the weight, in order, reaches `target`, which it does. listed_to: the last of the bins, from 0 on, whose tokens
// the list holds; -1: none.
template <bool F32>
__device__ __forceinline__ Place find(const void* row, int n, const Scale& s, bool by_count, u64 target, int& listed_to) {
  Memory& m = memory();
  const int b = bin_of(m.all, by_count, target);
  uint32_t base_c = b ? m.all.count[b - 1] : 0, in_bin = m.all.count[b] - base_c;
  u64 base_w = b ? m.all.weight[b - 1] : 0;
  if (threadIdx.x == 0) m.filled = 0;
  __syncthreads();
  if (in_bin <= kSub) {
    auto take = [&](u64 key) { m.sub[atomicAdd(&m.filled, 1u)] = key; };
    if (listed_to < 0 && m.all.count[b] <= kList) {  // the first time: what later places can ask for, too
      if (threadIdx.x == 0) m.listed = 0;
      __syncthreads();
      each_logit<F32>(row, n, [&](float x, int i) {
        if (x > -INFINITY && s.bin(x) <= b) m.list[atomicAdd(&m.listed, 1u)] = make_key(x, i);
      });
      listed_to = b;
      __syncthreads();
    }
    if (b <= listed_to) {
      for (uint32_t i = threadIdx.x; i < m.listed; i += kThreads)
        if (s.bin(key_value(m.list[i])) == b) take(m.list[i]);
    } else {
      each_logit<F32>(row, n, [&](float x, int i) {
        if (x > -INFINITY && s.bin(x) == b) take(make_key(x, i));
      });
    }
  } else {
    // keys in lo .. hi of the bin, divided by the leading bits in which they differ
    u64 lo = 0, hi = ~0ull;
    listed_to = -1;
    while (in_bin > kSub) {
      u64 most = 0, least = 0;  // of ~key
      each_logit<F32>(row, n, [&](float x, int i) {
        if (x > -INFINITY && s.bin(x) == b) {
          const u64 k = make_key(x, i);
          if (k >= lo && k <= hi) {
            most = k > most ? k : most;
            least = ~k > least ? ~k : least;
          }
        }
      });
      hi = group_max(most);
      lo = ~group_max(least);
      const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - 11);
      clear(m.part);
      __syncthreads();
      each_logit<F32>(row, n, [&](float x, int i) {
        if (x > -INFINITY && s.bin(x) == b) {
          const u64 k = make_key(x, i);
          if (k >= lo && k <= hi) {
            const int p = (int)((hi - k) >> shift);
            atomicAdd(&m.part.count[p], 1u);
            atomicAdd(&m.part.weight[p], weight_of(s.exponent(x)));
          }
        }
      });
      __syncthreads();
      run_up(m.part);
      const int p = bin_of(m.part, by_count, target - (by_count ? base_c : base_w));
      const uint32_t c0 = p ? m.part.count[p - 1] : 0;
      in_bin = m.part.count[p] - c0;
      base_w += p ? m.part.weight[p - 1] : 0;
      base_c += c0;
      const u64 top = hi - ((u64)p << shift), bottom = top - ((1ull << shift) - 1);
      lo = bottom > lo ? bottom : lo;
      hi = top;
      __syncthreads();
    }
    each_logit<F32>(row, n, [&](float x, int i) {
      if (x > -INFINITY && s.bin(x) == b) {
        const u64 k = make_key(x, i);
        if (k >= lo && k <= hi) m.sub[atomicAdd(&m.filled, 1u)] = k;
      }
    });
  }
  __syncthreads();
  const int filled = (int)m.filled, t = threadIdx.x;
  const u64 key = t < filled ? m.sub[t] : 0, w = t < filled ? weight_of(s.exponent(key_value(key))) : 0;
  if (t < filled) m.sub_weight[t] = w;
  __syncthreads();
  if (t < filled) {
    uint32_t c = base_c + 1;
    u64 sum = base_w + w;
    for (int j = 0; j < filled; j++) {
      const bool before = m.sub[j] > key;
      c += before;
      sum += before ? m.sub_weight[j] : 0;
    }
    if (by_count ? c == target : sum >= target && sum - w < target) m.found_key = key, m.found_weight = sum, m.found_count = c;
  }
  __syncthreads();
  const Place p = {m.found_key, m.found_weight, m.found_count};
  __syncthreads();
  return p;
}

template <bool F32>
__global__ void __launch_bounds__(kThreads) k_sample(SampleCall c) {
  Memory& m = memory();
  const int64_t r = blockIdx.x;
  const int t = threadIdx.x;
  const void* row = (const char*)c.logits + r * c.stride * (F32 ? 4 : 2);
  const float T = c.temperatures ? c.temperatures[r] : 1.f, top_p = c.top_ps ? c.top_ps[r] : 1.f, min_p = c.min_ps ? c.min_ps[r] : 0.f;
  const float u = c.uniforms[r];
  const int top_k = c.top_ks ? c.top_ks[r] : 0;
  auto answer = [&](int token, double logprob, int kept) {
    if (t == 0) {
      c.tokens[r] = token;
      if (c.logprobs) c.logprobs[r] = (float)logprob;
      if (c.kept) c.kept[r] = kept;
    }
  };
  if (!(T >= 0.f && T < INFINITY && top_p >= 0.f && min_p >= 0.f && min_p <= 1.f && u >= 0.f && u < 1.f)) return answer(-1, NAN, 0);

  float most = -INFINITY;
  bool bad = false;
  each_logit<F32>(row, c.vocab, [&](float x, int) {
    most = fmaxf(most, x);
    bad |= !(x < INFINITY);
  });
  // the largest in order, a bad row above all
  const u64 first = group_max(bad ? ~0ull : make_key(most, 0));
  const float top = key_value(first);
  if (first == ~0ull || top == -INFINITY) return answer(-1, NAN, 0);
  if (T == 0.f || top_k == 1) {
    u64 key = 0;
    each_logit<F32>(row, c.vocab, [&](float x, int i) {
      if (x == top) key = max(key, make_key(x, i));
    });
    return answer(key_index(group_max(key)), 0.0, 1);
  }

  Scale s;
  s.m = top;
  s.c = 1.4426950408889634 / (double)T;
  s.bins = (float)fmin(fmax(s.c * ((kBins - 1) / (double)kReach), (double)1.17549435e-38f), (double)3.40282347e+38f);
  s.most = min_p > 0.f ? -log2((double)min_p) : INFINITY;
  clear(m.all);
  if (t == 0) m.bin = 0;
  __syncthreads();
  uint32_t likely = 0;  // tokens that min_p keeps
  each_logit<F32>(row, c.vocab, [&](float x, int) {
    if (x > -INFINITY) {
      const double d = s.exponent(x);
      const u64 w = weight_of(d);
      const int b = s.bin(x);
      atomicAdd(&m.all.count[b], 1u);
      if (w) atomicAdd(&m.all.weight[b], w);
      likely += d <= s.most;
    }
  });
  __syncthreads();
  run_up(m.all);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) likely += (uint32_t)__shfl_xor((int)likely, o, 64);
  if ((t & 63) == 0) m.wave_a[t >> 6] = likely;
  __syncthreads();
  likely = 0;
  for (int w = 0; w < kWavesOf; w++) likely += (uint32_t)m.wave_a[w];
  __syncthreads();

  const uint32_t all = m.all.count[kBins - 1];
  const uint32_t k = top_k > 0 && (uint32_t)top_k < all ? (uint32_t)top_k : all;
  const bool cut = top_p < 1.f;
  u64 weight = m.all.weight[kBins - 1];  // of the first `weighed` tokens
  uint32_t weighed = all, kept = cut ? k : min(k, likely);
  Place p;
  int listed_to = -1;
  // the places asked for, one after the other: top-k's, top-p's, the last one that is kept, the draw
  for (int step = cut ? 0 : 2; step < 4; step++) {
    if (step % 2 == 0 && kept == weighed) continue;
    u64 target = kept;
    if (step == 1) target = max((u64)1, (u64)ceil((double)top_p * (double)weight));
    if (step == 3) target = min((u64)((double)u * (double)weight), weight - 1) + 1;
    p = find<F32>(row, c.vocab, s, step % 2 == 0, target, listed_to);
    if (step == 3) break;
    weight = p.weight;
    weighed = p.count;
    if (step == 1) kept = min(weighed, likely);
  }
  answer(key_index(p.key), -s.exponent(key_value(p.key)) * 0.6931471805599453 - log((double)weight * 0x1p-43), (int)kept);
}

}  // namespace

size_t sample_ws_bytes(int rows, int vocab) { return 16; }

hipError_t launch_sample(const SampleCall& c, hipStream_t s) {
  if (c.rows <= 0) return hipSuccess;
  const void* kernel = c.f32 ? (const void*)k_sample<true> : (const void*)k_sample<false>;
  const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Memory));
  if (e != hipSuccess) return e;
  if (c.f32) k_sample<true><<<c.rows, kThreads, sizeof(Memory), s>>>(c);
  else k_sample<false><<<c.rows, kThreads, sizeof(Memory), s>>>(c);
  return hipGetLastError();
}

}  // namespace sidp
