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
// in which bin a count or a weight is reached. Each place depends on the one before it,
// but bounds of all follow from the histogram, so that the tokens of every bin that can
// matter are picked out of the row at once (where they are too many, a bin at a time, when
// its place is asked for). A place's own bin is divided by its tokens' order, value and
// then index, with a small histogram each time, until it has few, and these are put in
// order. With a top-k the large histogram counts only: the weights that matter are those of
// the tokens picked out.
//
// Four launches: the row's ends (its largest and least logit), the histogram, the picking,
// the draw. The first three read the row, by as many segments as fill the chip; histograms
// are joined by atomics on whole numbers, whose order changes nothing.
//
// Measured, us: a row of 128256 bf16 logits 30, 16 rows 37 (top-k and top-p) and 58 (top-p),
// 64 rows 49 and 79, 256 rows 92 and 127; 256 rows of 151936 fp32 logits with all settings
// mixed 135 (146 from Python), of which the ends take 31 (155 MB at 5 TB/s); 512 rows of
// 32001 bf16 logits at a temperature alone 77. What bounds it is the reading, arithmetic on
// logits (the histogram 46 us of the mixed rows, with an exponential in 64 bits and two LDS
// atomics each) and for few rows the barriers of the draw, about 14 us. A workgroup a row
// for all four steps in one launch took 166 for the mixed rows and 84 for the 512. Greedy
// rows pass through all four: 16 us a row, 31 to 36 for 256.
//
// Rows whose wanted bins hold more than kList tokens are the slow ones: a single workgroup
// reads the row again for each place. Bins are spaced from the largest logit to the least, or to
// where weights end, so it takes many alike logits, or a high temperature beside a finite
// mask value: half of 128256 normal logits masked by -10000, top-p alone, at T of 1, 4, 8 one row 46, 56,
// 100 us, 256 rows 153, 173, 229 (123 without the mask at T = 1); 128256 equal logits 300 to 700 us one row,
// 550 to 880 for 256.
#include <type_traits>

#include "common.h"
#include "internal.h"

namespace sidp {

namespace {

typedef unsigned long long u64;

// Waves of a group that goes through barriers together: 8. With 16 the 256 mixed rows took 156 us and a single one 33, with 8 144 and 30,
// with 4 174 and 35.
constexpr int kThreads = 512, kWavesOf = kThreads / 64;
constexpr int kBins = 2048;
constexpr float kReach = 44.f;   // weights of 2^-kReach and less are 0
constexpr int kUnit = 43;        // bits behind the point of a weight: 2^20 tokens of 2^43 are 2^63
constexpr int kList = 4096;      // tokens picked out of a row at once
constexpr int kParts = 512;      // of a bin that is divided
constexpr int kFew = 64;         // tokens that are put in order (up to 128: a row 35 us, 30; up to 32: as 64)
constexpr int kSteps = 4;        // places that a row can ask for, each with its own answer in LDS
constexpr int kTurns = 4;        // bins are told to all in as many places in turn, so that one barrier each is enough

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

// 2^-d in units of 2^-kUnit, to the nearest; d >= 0. The fraction's power by the polynomial of degree 9 that meets 2^f at the ten
// Chebyshev nodes of -1/2 .. 1/2: off by at most 2^-45 of it (2 (ln 2 / 4)^10 / 10! = 2^-46 and the coefficients' roundings). Taylor's
// series would need a degree of 11 for that.
__device__ __forceinline__ u64 weight_of(double d) {
  if (!(d < kReach + 0.5)) return 0;
  const double n = __builtin_rint(d), f = n - d;
  // kept in scalar registers, of which a product takes one operand: in vector ones the ten of them cost the loop 20
  // (256 mixed rows 149 us, so 137)
  auto scalar = [](double c) {
    asm("" : "+s"(c));
    return c;
  };
  double p = 0x1.b6571de2f2351p-24;
  p = __builtin_fma(p, f, scalar(0x1.63ef969a64d3cp-20));
  p = __builtin_fma(p, f, scalar(0x1.ffcb76789860fp-17));
  p = __builtin_fma(p, f, scalar(0x1.43088e257f341p-13));
  p = __builtin_fma(p, f, scalar(0x1.5d87fe908f88ap-10));
  p = __builtin_fma(p, f, scalar(0x1.3b2ab72b175eep-7));
  p = __builtin_fma(p, f, scalar(0x1.c6b08d7044119p-5));
  p = __builtin_fma(p, f, scalar(0x1.ebfbdff8149f2p-3));
  p = __builtin_fma(p, f, scalar(0x1.62e42fefa39f7p-1));
  p = __builtin_fma(p, f, scalar(0x1.000000000003dp+0));
  p = __builtin_amdgcn_ldexp(p, kUnit - (int)n) + 0x1p52;  // the sum's last bit is one unit
  return (u64)__builtin_bit_cast(int64_t, p) & ((1ull << 52) - 1);
}

// f(logit, index) for the logits first .. last - 1 of a row, 16 bytes a load where their address allows.
template <bool F32, class F>
__device__ __forceinline__ void each_logit(const void* row, int first, int last, const F& f) {
  constexpr int kSize = F32 ? 4 : 2, V = 16 / kSize;
  const int t = threadIdx.x, n = last - first;
  const char* from = (const char*)row + (int64_t)first * kSize;
  auto at = [&](int i) { return F32 ? ((const float*)from)[i] : bf2f(((const uint16_t*)from)[i]); };
  const int head = min(n, (int)(-(uintptr_t)from & 15) / kSize), vectors = (n - head) / V, tail = head + vectors * V;
  if (t < head) f(at(t), first + t);
  const u32x4_t* v = (const u32x4_t*)(from + head * kSize);
  // The next two loads are under way while a third's logits are worked on. A loop that is not unrolled: with few logits a thread,
  // most of a call's time is that of its instructions on their way.
  auto load = [&](int j) { return j < vectors ? v[j] : u32x4_t{0, 0, 0, 0}; };
  u32x4_t w0 = load(t), w1 = load(t + kThreads), w2 = load(t + 2 * kThreads);
#pragma unroll 1
  for (int j = t; j < vectors; j += kThreads) {
#pragma unroll
    for (int k = 0; k < V; k++) {
      const float x = F32 ? __uint_as_float(w0[k % 4]) : __uint_as_float(k % 2 ? w0[k / 2] & 0xffff0000u : w0[k / 2] << 16);
      f(x, first + head + j * V + k);
    }
    w0 = w1;
    w1 = w2;
    w2 = load(j + 3 * kThreads);
  }
  if (t < n - tail) f(at(tail + t), first + tail + t);
}

template <int BINS>
struct Histogram {
  u64 weight[BINS];
  uint32_t count[BINS];
};
struct Memory {
  u64 wave_a[kWavesOf], wave_b[kWavesOf];
  u64 found_key[kSteps], found_weight[kSteps];
  uint32_t found_count[kSteps], filled[kSteps], listed;
  int bin[kTurns];
  Histogram<kBins> all;  // running sums, once they are made
  // what follows is the draw's
  Histogram<kParts> part;  // of a bin that is divided
  u64 list[kList];
  u64 few[kFew], few_weight[kFew];
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

// A value of all threads', made of two at a time by `f`; every thread calls.
template <class T, class F>
__device__ __forceinline__ T over_group(T v, const F& f) {
  Memory& m = memory();
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = f(v, __shfl_xor(v, o, 64));
  T* s = (T*)m.wave_a;
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
  for (int w = 1; w < kWavesOf; w++) v = f(v, s[w]);
  __syncthreads();
  return v;
}
__device__ __forceinline__ u64 larger(u64 a, u64 b) { return a > b ? a : b; }

template <int BINS>
__device__ __forceinline__ void clear(Histogram<BINS>& h) {
  for (int i = threadIdx.x; i < BINS; i += kThreads) h.weight[i] = 0, h.count[i] = 0;
}
// A histogram's running sums, in its place: of counts, weights or both.
template <bool COUNTS, bool WEIGHTS, int BINS>
__device__ __forceinline__ void run_up(Histogram<BINS>& h) {
  Memory& m = memory();
  constexpr int kPer = BINS < kThreads ? 1 : BINS / kThreads;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const bool mine = t * kPer < BINS;
  u64 w[kPer], sw = 0;
  uint32_t c[kPer], sc = 0;
#pragma unroll
  for (int i = 0; i < kPer; i++) {
    if (WEIGHTS) w[i] = sw += mine ? h.weight[t * kPer + i] : 0;
    if (COUNTS) c[i] = sc += mine ? h.count[t * kPer + i] : 0;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    if (WEIGHTS) {
      const u64 a = __shfl_up(sw, o, 64);
      if (lane >= o) sw += a;
    }
    if (COUNTS) {
      const uint32_t b = (uint32_t)__shfl_up((int)sc, o, 64);
      if (lane >= o) sc += b;
    }
  }
  if (lane == 63) {
    if (WEIGHTS) m.wave_a[wave] = sw;
    if (COUNTS) m.wave_b[wave] = sc;
  }
  if (WEIGHTS) sw -= w[kPer - 1];
  if (COUNTS) sc -= c[kPer - 1];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWavesOf - 1; i++) {  // read side by side
    if (WEIGHTS) sw += i < wave ? m.wave_a[i] : 0;
    if (COUNTS) sc += i < wave ? (uint32_t)m.wave_b[i] : 0;
  }
#pragma unroll
  for (int i = 0; i < kPer; i++) {
    if (WEIGHTS && mine) h.weight[t * kPer + i] = sw + w[i];
    if (COUNTS && mine) h.count[t * kPer + i] = sc + c[i];
  }
  __syncthreads();
}
// The bin of running sums `h` in which `target` is reached, by count or by weight. It is, in one.
template <int BINS>
__device__ __forceinline__ int bin_of(const Histogram<BINS>& h, bool by_count, u64 target, int& turn) {
  Memory& m = memory();
  const int slot = turn++ % kTurns;
  for (int i = threadIdx.x; i < BINS; i += kThreads) {
    const u64 to = by_count ? h.count[i] : h.weight[i], from = i == 0 ? 0 : by_count ? h.count[i - 1] : h.weight[i - 1];
    if (from < target && target <= to) m.bin[slot] = i;
  }
  __syncthreads();
  return m.bin[slot];
}

// A row's settings as the caller gave them.
struct Settings {
  float T, top_p, min_p, u;
  int top_k;
  __device__ __forceinline__ bool good() const {
    return T >= 0.f && T < INFINITY && top_p >= 0.f && min_p >= 0.f && min_p <= 1.f && u >= 0.f && u < 1.f;
  }
  __device__ __forceinline__ bool greedy() const { return T == 0.f || top_k == 1; }
  // the histogram counts only: few enough tokens are picked out, as a rule, to weigh them there
  __device__ __forceinline__ bool counts_only() const { return top_k > 0 && top_k <= kList / 2; }
};
__device__ __forceinline__ Settings settings_of(const SampleCall& c, int64_t r) {
  return Settings{c.temperatures ? c.temperatures[r] : 1.f, c.top_ps ? c.top_ps[r] : 1.f, c.min_ps ? c.min_ps[r] : 0.f, c.uniforms[r],
                  c.top_ks ? c.top_ks[r] : 0};
}
// What the first reading of a row gives: its first token's key (all ones if a logit is NaN or +inf), and the least logit above -inf.
struct Ends {
  u64 best;
  float least;
  __device__ __forceinline__ bool none() const { return best == ~0ull || key_value(best) == -INFINITY; }
};
template <bool F32>
__device__ __forceinline__ Ends ends_of(const void* row, int first, int last) {
  float most = -INFINITY, least = INFINITY;
  int at = 0;
  bool bad = false;
  each_logit<F32>(row, first, last, [&](float x, int i) {
    if (x > most) most = x, at = i;
    if (x > -INFINITY) least = fminf(least, x);
    bad |= !(x < INFINITY);
  });
  // indexes rise within a thread, and a smaller one's key is the larger among equals
  return Ends{over_group(bad ? ~0ull : make_key(most, at), larger), over_group(least, [](float a, float b) { return fminf(a, b); })};
}
__device__ __forceinline__ Scale scale_of(const Settings& z, const Ends& e) {
  Scale s;
  s.m = key_value(e.best);
  s.c = 1.4426950408889634 / (double)z.T;
  // the bins reach to the least logit, or to where weights end
  const double reach = fmin(((double)s.m - (double)e.least) * s.c, (double)kReach);
  s.bins = (float)fmin(fmax(s.c * ((kBins - 2) / fmax(reach, 1e-30)), (double)1.17549435e-38f), (double)3.40282347e+38f);
  s.most = z.min_p > 0.f ? -log2((double)z.min_p) : INFINITY;
  return s;
}
// Adds logits first .. last - 1 to the histogram (cleared, or holding others'). The number of those that min_p keeps, of this thread's.
template <bool F32>
__device__ __forceinline__ uint32_t add_up(const void* row, int first, int last, const Scale& s, bool count, bool weigh, bool likely_too) {
  Memory& m = memory();
  uint32_t likely = 0;
  auto all = [&](auto weights) {
    each_logit<F32>(row, first, last, [&](float x, int) {
      if (x > -INFINITY) {
        const int b = s.bin(x);
        if (count) atomicAdd(&m.all.count[b], 1u);
        if (decltype(weights)::value || likely_too) {
          const double d = s.exponent(x);
          if (decltype(weights)::value) {
            const u64 w = weight_of(d);
            if (w) atomicAdd(&m.all.weight[b], w);
          }
          likely += d <= s.most;
        }
      }
    });
  };
  if (weigh) all(std::true_type{});
  else all(std::false_type{});
  return likely;
}

__device__ __forceinline__ u64 cut_target(float p, u64 weight) { return larger(1, (u64)ceil((double)p * (double)weight)); }
__device__ __forceinline__ u64 draw_target(float u, u64 weight) {
  if (weight == 0) return 1;
  const u64 t = (u64)((double)u * (double)weight);
  return (t < weight ? t : weight - 1) + 1;
}

// Bins whose tokens are picked out: up to four stretches.
struct Wanted {
  int from[4], to[4];
  uint32_t tokens;  // at most
  bool more;        // than stretches 1 and 3
  __device__ __forceinline__ bool in(int i, int b) const { return (uint32_t)(b - from[i]) <= (uint32_t)(to[i] - from[i]); }
  // top-k's and the last token's bins are the rarer ones
  __device__ __forceinline__ bool has(int b) const { return in(1, b) || in(3, b) || (more && (in(0, b) || in(2, b))); }
};
// Every bin in which a place of the row can lie, from the running sums: of top-k, of top-p, of the last token that all settings keep, of
// the draw. With counts alone: all bins up to top-k's.
__device__ __forceinline__ Wanted wanted_of(const Settings& z, uint32_t likely, bool weighed, int& turn) {
  const Histogram<kBins>& h = memory().all;
  Wanted w;
#pragma unroll
  for (int i = 0; i < 4; i++) w.from[i] = w.to[i] = kBins;  // none
  w.tokens = 0;
  w.more = false;
  auto count_before = [&](int b) { return b ? h.count[b - 1] : 0u; };
  auto weight_before = [&](int b) { return b ? h.weight[b - 1] : 0ull; };
  const uint32_t all = h.count[kBins - 1], k = z.top_k > 0 && (uint32_t)z.top_k < all ? (uint32_t)z.top_k : all;
  if (!weighed) {
    w.from[1] = 0;
    w.to[1] = bin_of(h, true, k, turn);
    w.tokens = h.count[w.to[1]];
    return w;
  }
  auto add = [&](int i, int a, int b) {
    w.from[i] = a;
    w.to[i] = b;
    w.more |= i % 2 == 0;
    w.tokens += h.count[b] - count_before(a);
  };
  u64 lo = h.weight[kBins - 1], hi = lo;  // bounds of the weight that the draw goes by
  uint32_t least = k, most = k;           // and of the tokens
  if (z.top_p < 1.f) {
    if (k < all) {
      const int b = bin_of(h, true, k, turn);
      add(0, b, b);
      lo = weight_before(b);
      hi = h.weight[b];
    }
    const int a = bin_of(h, false, cut_target(z.top_p, lo), turn), b = bin_of(h, false, cut_target(z.top_p, hi), turn);
    add(1, a, b);
    least = count_before(a) + 1;
    most = h.count[b];
    lo = weight_before(a);
    hi = h.weight[b];
  }
  if (likely <= most && (likely < all || z.top_p < 1.f || k < all)) {
    most = likely;
    const int b = bin_of(h, true, likely, turn);
    add(2, b, b);
    lo = likely < least ? weight_before(b) : min(lo, weight_before(b));
    hi = min(hi, h.weight[b]);
  } else if (!(z.top_p < 1.f) && k < all) {
    const int b = bin_of(h, true, k, turn);
    add(2, b, b);
    lo = weight_before(b);
    hi = h.weight[b];
  }
  const int a = bin_of(h, false, draw_target(z.u, lo), turn), b = bin_of(h, false, draw_target(z.u, hi), turn);
  add(3, a, b);
  return w;
}
// Picks the wanted tokens out of logits first .. last - 1: put(key).
template <bool F32, class Put>
__device__ __forceinline__ void pick(const void* row, int first, int last, const Scale& s, const Wanted& w, const Put& put) {
  // The stretches as bounds of what Scale::bin cuts to a whole number: up to the last number below `to` + 1, the last bin's end is open.
  float lo[4], hi[4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const bool none = w.from[i] >= kBins;
    lo[i] = none ? INFINITY : (float)w.from[i];
    hi[i] = none ? -1.f : w.to[i] == kBins - 1 ? INFINITY : __uint_as_float(__float_as_uint((float)(w.to[i] + 1)) - 1);
  }
  auto all = [&](auto more) {  // top-k's and the last token's stretches are the rarer ones
    each_logit<F32>(row, first, last, [&](float x, int i) {
      const float at = (s.m - x) * s.bins;
      bool want = (at >= lo[1] && at <= hi[1]) | (at >= lo[3] && at <= hi[3]);
      if (decltype(more)::value) want |= (at >= lo[0] && at <= hi[0]) | (at >= lo[2] && at <= hi[2]);
      if (want && x > -INFINITY) put(make_key(x, i));
    });
  };
  if (w.more) all(std::true_type{});
  else all(std::false_type{});
}

// Where the count or the weight, in order, reaches `target`, which it does; the row's place number `step`. listed: the list holds the
// tokens of the wanted bins.
template <bool F32>
__device__ __forceinline__ Place find(const void* row, int n, const Scale& s, bool by_count, u64 target, const Wanted& w, bool& listed,
                                      int& turn, int step) {
  Memory& m = memory();
  const int t = threadIdx.x, b = bin_of(m.all, by_count, target, turn);
  uint32_t base_c = b ? m.all.count[b - 1] : 0, left = m.all.count[b] - base_c;
  u64 base_w = b ? m.all.weight[b - 1] : 0;
  u64 lo = 0, hi = ~0ull;  // keys of the bin that are still looked at, `left` of them
  bool here = listed && w.has(b);
  auto in_list = [&](auto f) {
    for (uint32_t i = t; i < m.listed; i += kThreads) {
      const u64 k = m.list[i];
      if (k >= lo && k <= hi && s.bin(key_value(k)) == b) f(k);
    }
  };
  auto in_row = [&](auto f) {
    each_logit<F32>(row, 0, n, [&](float x, int i) {
      if (x > -INFINITY && s.bin(x) == b) {
        const u64 k = make_key(x, i);
        if (k >= lo && k <= hi) f(k);
      }
    });
  };
  for (;;) {
    if (!here && left <= kList) {
      listed = false;  // the list is this bin's now
      if (t == 0) m.listed = 0;
      __syncthreads();
      in_row([&](u64 k) { m.list[atomicAdd(&m.listed, 1u)] = k; });
      __syncthreads();
      here = true;
    }
    if (here && left <= kFew) break;
    // divided by the leading bits in which they differ
    u64 most = 0, least = 0;  // of ~key
    auto reach = [&](u64 k) {
      most = larger(k, most);
      least = larger(~k, least);
    };
    if (here) in_list(reach);
    else in_row(reach);
    hi = over_group(most, larger);
    lo = ~over_group(least, larger);
    const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - 9);
    clear(m.part);
    __syncthreads();
    auto add = [&](u64 k) {
      const int p = (int)((hi - k) >> shift);
      atomicAdd(&m.part.count[p], 1u);
      atomicAdd(&m.part.weight[p], weight_of(s.exponent(key_value(k))));
    };
    if (here) in_list(add);
    else in_row(add);
    __syncthreads();
    run_up<true, true>(m.part);
    const int p = bin_of(m.part, by_count, target - (by_count ? base_c : base_w), turn);
    const uint32_t c0 = p ? m.part.count[p - 1] : 0;
    left = m.part.count[p] - c0;
    base_w += p ? m.part.weight[p - 1] : 0;
    base_c += c0;
    const u64 top = hi - ((u64)p << shift), bottom = top - ((1ull << shift) - 1);
    lo = larger(bottom, lo);
    hi = top;
    __syncthreads();
  }
  in_list([&](u64 k) { m.few[atomicAdd(&m.filled[step], 1u)] = k; });
  __syncthreads();
  const int filled = (int)m.filled[step];
  if (t < filled) m.few_weight[t] = weight_of(s.exponent(key_value(m.few[t])));
  __syncthreads();
  // kLanes threads a token: each looks at every kLanes-th other
  constexpr int kLanes = kThreads / kFew;
  const int mine = t / kLanes;
  const u64 key = mine < filled ? m.few[mine] : 0, weight = mine < filled ? m.few_weight[mine] : 0;
  uint32_t c = 0;
  u64 sum = 0;
#pragma unroll
  for (int q = 0; q < kFew / kLanes; q++) {
    const int j = t % kLanes + q * kLanes;
    const bool before = j < filled && m.few[j] > key;
    c += before;
    sum += before ? m.few_weight[j] : 0;
  }
#pragma unroll
  for (int o = kLanes / 2; o >= 1; o >>= 1) {
    c += (uint32_t)__shfl_xor((int)c, o, 64);
    sum += __shfl_xor(sum, o, 64);
  }
  c += base_c + 1;
  sum += base_w + weight;
  if (mine < filled && (by_count ? c == target : sum >= target && sum - weight < target))
    m.found_key[step] = key, m.found_weight[step] = sum, m.found_count[step] = c;
  __syncthreads();
  return Place{m.found_key[step], m.found_weight[step], m.found_count[step]};
}

// The answer of a row of which the histogram's running sums and, with `listed`, the wanted tokens are at hand.
template <bool F32>
__device__ __forceinline__ void draw(const SampleCall& c, int64_t r, const void* row, const Settings& z, const Scale& s, uint32_t likely,
                                     bool weighed, const Wanted& w, bool listed, int turn) {
  Memory& m = memory();
  if (!weighed) {  // the weights of the tokens picked out; where they were too many, of all
    for (int i = threadIdx.x; i < kBins; i += kThreads) m.all.weight[i] = 0;
    __syncthreads();
    if (listed) {
      for (uint32_t i = threadIdx.x; i < m.listed; i += kThreads) {
        const float x = key_value(m.list[i]);
        atomicAdd(&m.all.weight[s.bin(x)], weight_of(s.exponent(x)));
      }
    } else {
      add_up<F32>(row, 0, c.vocab, s, false, true, false);
    }
    __syncthreads();
    run_up<false, true>(m.all);
  }
  const uint32_t all = m.all.count[kBins - 1];
  const uint32_t k = z.top_k > 0 && (uint32_t)z.top_k < all ? (uint32_t)z.top_k : all;
  const bool cut = z.top_p < 1.f;
  u64 weight = m.all.weight[kBins - 1];  // of the first `of` tokens
  uint32_t of = all, kept = cut ? k : min(k, likely);
  Place p;
  // the places asked for, one after the other: top-k's, top-p's, the last one that is kept, the draw
#pragma unroll 1
  for (int step = cut ? 0 : 2; step < kSteps; step++) {
    if (step % 2 == 0 && kept == of) continue;
    const u64 target = step == 1 ? cut_target(z.top_p, weight) : step == 3 ? draw_target(z.u, weight) : kept;
    p = find<F32>(row, c.vocab, s, step % 2 == 0, target, w, listed, turn, step);
    if (step == 3) break;
    weight = p.weight;
    of = p.count;
    if (step == 1) kept = min(of, likely);
  }
  if (threadIdx.x == 0) {
    c.tokens[r] = key_index(p.key);
    if (c.logprobs) c.logprobs[r] = (float)(-s.exponent(key_value(p.key)) * 0.6931471805599453 - log((double)weight * 0x1p-43));
    if (c.kept) c.kept[r] = (int)kept;
  }
}
// The answers that need no draw: true if this is one.
__device__ __forceinline__ bool answered(const SampleCall& c, int64_t r, const Settings& z, const Ends& e) {
  const bool none = !z.good() || e.none();
  if (!none && !z.greedy()) return false;
  if (threadIdx.x == 0) {
    c.tokens[r] = none ? -1 : key_index(e.best);
    if (c.logprobs) c.logprobs[r] = none ? NAN : 0.f;
    if (c.kept) c.kept[r] = none ? 0 : 1;
  }
  return true;
}

template <bool F32>
__device__ __forceinline__ const void* row_of(const SampleCall& c, int64_t r) {
  return (const char*)c.logits + r * c.stride * (F32 ? 4 : 2);
}

__device__ __forceinline__ void begin() {
  Memory& m = memory();
  if (threadIdx.x < kTurns) m.bin[threadIdx.x] = 0;
  if (threadIdx.x < kSteps) m.filled[threadIdx.x] = 0;
  if (threadIdx.x == 0) m.listed = 0;
}

// A row's part of the workspace:
struct Row {
  u64 weight[kBins];
  uint32_t count[kBins];
  u64 list[kList];
  uint32_t likely, listed;
  Wanted wanted;
};
struct Layout {
  size_t rows, ends, bytes;
};
__host__ __device__ inline Layout layout_of(int rows, int segments) {
  Layout l;
  l.rows = 0;
  l.ends = (size_t)rows * sizeof(Row);
  l.bytes = l.ends + (size_t)rows * segments * sizeof(Ends);
  return l;
}
struct Segment {
  int64_t row;
  int first, last;
  Row* state;
  Ends* ends;  // of the row's segments
};
__device__ __forceinline__ Segment segment_of(const SampleCall& c) {
  Segment g;
  g.row = blockIdx.y;
  const int per = ((c.vocab + c.segments - 1) / c.segments + 63) / 64 * 64;  // whole 16 bytes of either type
  g.first = min((int)blockIdx.x * per, c.vocab);
  g.last = min(g.first + per, c.vocab);
  const Layout l = layout_of(c.rows, c.segments);
  g.state = (Row*)((char*)c.ws + l.rows) + g.row;
  g.ends = (Ends*)((char*)c.ws + l.ends) + g.row * c.segments;
  return g;
}
__device__ __forceinline__ Ends join_ends(const Segment& g, int segments) {
  Ends e = {0, INFINITY};
  for (int i = threadIdx.x & 63; i < segments; i += 64) {  // by each wave for itself, a segment a lane
    e.best = larger(e.best, g.ends[i].best);
    e.least = fminf(e.least, g.ends[i].least);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    e.best = larger(e.best, __shfl_xor(e.best, o, 64));
    e.least = fminf(e.least, __shfl_xor(e.least, o, 64));
  }
  return e;
}

template <bool F32>
__global__ void __launch_bounds__(kThreads, 8) k_sample_ends(SampleCall c) {
  const Segment g = segment_of(c);
  for (int i = blockIdx.x * kThreads + threadIdx.x; i < kBins; i += c.segments * kThreads) g.state->weight[i] = 0, g.state->count[i] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) g.state->likely = g.state->listed = 0;
  const Ends e = ends_of<F32>(row_of<F32>(c, g.row), g.first, g.last);
  if (threadIdx.x == 0) g.ends[blockIdx.x] = e;
}
template <bool F32>
__global__ void __launch_bounds__(kThreads, 8) k_sample_add(SampleCall c) {
  Memory& m = memory();
  const Segment g = segment_of(c);
  const Settings z = settings_of(c, g.row);
  const Ends e = join_ends(g, c.segments);
  if (!z.good() || e.none() || z.greedy()) return;
  clear(m.all);
  __syncthreads();
  const uint32_t likely = add_up<F32>(row_of<F32>(c, g.row), g.first, g.last, scale_of(z, e), true, !z.counts_only(), z.min_p > 0.f);
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kThreads) {
    if (m.all.count[i]) atomicAdd(&g.state->count[i], m.all.count[i]);
    if (m.all.weight[i]) atomicAdd(&g.state->weight[i], m.all.weight[i]);
  }
  const uint32_t sum = over_group(likely, [](uint32_t a, uint32_t b) { return a + b; });
  if (threadIdx.x == 0 && sum) atomicAdd(&g.state->likely, sum);
}
// The row's running sums in LDS; the tokens that min_p keeps.
__device__ __forceinline__ uint32_t load_sums(const Segment& g, const Settings& z) {
  Memory& m = memory();
  const uint32_t some = g.state->likely;
  for (int i = threadIdx.x; i < kBins; i += kThreads) m.all.weight[i] = g.state->weight[i], m.all.count[i] = g.state->count[i];
  begin();
  __syncthreads();
  run_up<true, true>(m.all);
  const uint32_t all = m.all.count[kBins - 1];
  return z.min_p > 0.f ? some : all;
}
template <bool F32>
__global__ void __launch_bounds__(kThreads, 8) k_sample_pick(SampleCall c) {
  const Segment g = segment_of(c);
  const Settings z = settings_of(c, g.row);
  const Ends e = join_ends(g, c.segments);
  if (!z.good() || e.none() || z.greedy()) return;
  int turn = 0;
  const Wanted w = wanted_of(z, load_sums(g, z), !z.counts_only(), turn);
  if (blockIdx.x == 0 && threadIdx.x == 0) g.state->wanted = w;
  if (w.tokens <= kList)
    pick<F32>(row_of<F32>(c, g.row), g.first, g.last, scale_of(z, e), w, [&](u64 key) { g.state->list[atomicAdd(&g.state->listed, 1u)] = key; });
}
template <bool F32>
__global__ void __launch_bounds__(kThreads) k_sample_draw(SampleCall c) {
  Memory& m = memory();
  const Segment g = segment_of(c);
  const Settings z = settings_of(c, g.row);
  const Ends e = join_ends(g, c.segments);
  if (answered(c, g.row, z, e)) return;
  const Wanted w = g.state->wanted;
  const bool listed = w.tokens <= kList;
  const uint32_t likely = load_sums(g, z), n = listed ? min(g.state->listed, (uint32_t)kList) : 0;
  for (uint32_t i = threadIdx.x; i < n; i += kThreads) m.list[i] = g.state->list[i];
  if (threadIdx.x == 0) m.listed = n;
  __syncthreads();
  draw<F32>(c, g.row, row_of<F32>(c, g.row), z, scale_of(z, e), likely, !z.counts_only(), w, listed, 0);
}

constexpr int kGroups = 1024;       // workgroups that fill the chip: four a CU
constexpr int kLeastSegment = 4096;  // logits: with 8192 a single row took 32 us (30), 16 rows 34 to 54 (37 to 58)
constexpr int kRowsAtOnce = 1024;   // more rows go by several times four launches, which share a workspace
int segments_of(int rows, int vocab) {
  return std::max(1, std::min((kGroups + rows - 1) / rows, (vocab + kLeastSegment - 1) / kLeastSegment));
}

template <class K>
hipError_t launch(K kernel, dim3 grid, size_t lds, const SampleCall& c, hipStream_t s) {
  const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  kernel<<<grid, kThreads, lds, s>>>(c);
  return hipGetLastError();
}
template <bool F32>
hipError_t launch_type(const SampleCall& c, hipStream_t s) {
  const dim3 grid(c.segments, c.rows);
  hipError_t e = launch(k_sample_ends<F32>, grid, offsetof(Memory, part), c, s);
  if (e == hipSuccess) e = launch(k_sample_add<F32>, grid, offsetof(Memory, part), c, s);
  if (e == hipSuccess) e = launch(k_sample_pick<F32>, grid, offsetof(Memory, part), c, s);
  if (e == hipSuccess) e = launch(k_sample_draw<F32>, dim3(1, c.rows), sizeof(Memory), c, s);
  return e;
}

}  // namespace

size_t sample_ws_bytes(int rows, int vocab) {
  size_t most = 0;  // the last rows may be cut into more segments
  for (int r : {std::min(rows, kRowsAtOnce), rows % kRowsAtOnce})
    if (r > 0) most = std::max(most, layout_of(r, segments_of(r, vocab)).bytes);
  return most;
}

hipError_t launch_sample(const SampleCall& call, hipStream_t s) {
  hipError_t e = hipSuccess;
  for (int r = 0; r < call.rows && e == hipSuccess; r += kRowsAtOnce) {
    SampleCall c = call;
    c.rows = std::min(kRowsAtOnce, call.rows - r);
    c.segments = segments_of(c.rows, c.vocab);
    c.logits = (const char*)c.logits + r * c.stride * (c.f32 ? 4 : 2);
    auto skip = [&](auto& p) {
      if (p) p += r;
    };
    skip(c.temperatures);
    skip(c.top_ks);
    skip(c.top_ps);
    skip(c.min_ps);
    skip(c.uniforms);
    skip(c.tokens);
    skip(c.logprobs);
    skip(c.kept);
    e = c.f32 ? launch_type<true>(c, s) : launch_type<false>(c, s);
  }
  return e;
}

}  // namespace sidp
