// A tile of (token, query head) pairs that share one KV head, over a run of the keys
// they see in the paged cache: the attention of several new tokens a sequence, by one
// workgroup of four waves. How it goes about it stands in k_attn_rows.hip; this is its
// text, for every kernel whose items are such tiles.
//
// Over the 8-bit cache (TYPE other than 0) the same products run on the codes as bf16,
// which holds them exactly: the scale of a key's token multiplies its scores, with the
// softmax's own factor, and the scale of a value's token its weights, so that no value
// is rounded on the way. Chunks come through registers (two of K and one of V on their
// way) and are spread out to bf16 as they are put into LDS, a turn before their scores
// are made or their values added.
#pragma once
#include <type_traits>

#include "common.h"
#include "internal.h"
#include "kv8.h"

namespace sidp {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kChunk = 32;        // tokens staged at a time
constexpr int kChunkBlocks = kChunk / kBlockTokens;
constexpr float kMost = 4096.f;
constexpr int kWaves = 4;
constexpr int kTileRows = 32 * kWaves;  // (token, head) pairs of a tile

typedef const __attribute__((address_space(4))) int32_t cint32_t;

__host__ __device__ inline int tile_tokens(int group) { return kTileRows / group; }

// Chunks of K, and of V, in LDS; bytes of LDS.
template <int TYPE>
constexpr int ring_of() { return TYPE ? 2 : 4; }
template <int D, int TYPE>
constexpr int tile_lds() { return 2 * ring_of<TYPE>() * kChunk * D * 2 + (TYPE ? 2 * kChunk * 2 * (int)sizeof(float) : 0); }

// The tile of an item. CAUSAL: token i, at position first_pos + i, sees the keys up to its own; else, by `step`, that (1) or the
// first first_pos + 1 whatever i is (0).
template <bool CAUSAL>
struct AttnTile {
  int b;          // the sequence whose block table it reads
  int row0;       // its first row
  int tokens;     // rows
  int first_pos;
  int kv_end;     // keys that its rows see together
  int c0, c1;     // chunks of this item
  int g;          // KV head
  bool one_tile;  // of all rows that read these keys
  int step = 1;
};

// What a lane has of the result: dims 32 dt + 8 i + from .. + 3 of its pair, in o[dt][4 i .. 4 i + 3], not yet divided by `sum`; the
// reference of the sum's weights (-inf where the pair saw nothing).
template <int D>
struct AttnOut {
  int at, tok, head, from;
  int64_t row;  // of out, in heads
  const f32x16_t (&o)[D / 32];
  float sum, ref;
  __device__ __forceinline__ void rows(uint16_t* out) const {
    const float inv = 1.f / sum;
    uint16_t* op = out + row * D + from;
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
      for (int i = 0; i < 4; i++)
        *(u32x2_t*)(op + dt * 32 + i * 8) = u32x2_t{pack_bf2(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv),
                                                    pack_bf2(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv)};
  }
  // r: the pair's D floats; ml: its reference and sum
  __device__ __forceinline__ void record(float* r, float* ml) const {
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
      for (int i = 0; i < 4; i++)
        *(f32x4_t*)(r + dt * 32 + i * 8 + from) = f32x4_t{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
    if (from == 0) *(float2*)ml = make_float2(ref, sum);
  }
};

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

// 16, 8 or 4 bytes a lane of a block, to registers. Buffer loads, whose address is one register a lane.
template <int BYTES>
__device__ __forceinline__ u32x4_t load16(const void* block, uint32_t offset, bool once) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(block), (short)0, BYTES, 0x00020000);
  return once ? __builtin_amdgcn_raw_buffer_load_b128(r, offset, 0, 2) : __builtin_amdgcn_raw_buffer_load_b128(r, offset, 0, 0);
}
template <int BYTES>
__device__ __forceinline__ u32x2_t load8(const void* block, uint32_t offset, bool once) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(block), (short)0, BYTES, 0x00020000);
  return once ? __builtin_amdgcn_raw_buffer_load_b64(r, offset, 0, 2) : __builtin_amdgcn_raw_buffer_load_b64(r, offset, 0, 0);
}
template <int BYTES>
__device__ __forceinline__ float load4(const void* block, uint32_t offset) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(block), (short)0, BYTES, 0x00020000);
  return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, offset, 0, 0));
}

// The larger of a lane's value and its counterpart's in the other half of the wave.
__device__ __forceinline__ float max_halves(float v) {
  const u32x2_t r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// emit: called by every lane that has a pair, with an AttnOut.
template <int D, int TYPE, bool CAUSAL, class Call, class Emit>
__device__ __forceinline__ void attn_tile(const Call& c, const AttnTile<CAUSAL>& x, const Emit& emit) {
  constexpr int KK = D / 16, DT = D / 32;
  constexpr int kBlockBytes = kBlockTokens * D * 2;
  constexpr int kSide = kChunkBlocks * kBlockBytes;  // K or V of a chunk
  constexpr int kBlockWaves = D / 32;                // waves that load a block's K (and V), 16 bytes a lane
  constexpr int kPieces = kChunkBlocks * kBlockWaves / kWaves;
  constexpr int kGroupChunks = 64 / kChunkBlocks;    // chunks whose block ids a wave holds, one a lane
  constexpr int kRing = ring_of<TYPE>();
  extern __shared__ __attribute__((aligned(16))) char smem[];  // the rings of K and of V
  // TYPE 0: whether an edge chunk held values that are not finite; else the first token without a scale
  __shared__ int s_odd;
  __shared__ int s_first[3][D];  // and the first tokens that hold +inf, -inf and NaN, of each dim

  const int t = threadIdx.x, lane = t & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int hkv = c.kv.hkv, group = c.hq / hkv;
  const int g = x.g, b = x.b, c0 = x.c0, c1 = x.c1, row0 = x.row0, tokens = x.tokens, first_pos = x.first_pos;
  // A sequence of one tile reads its keys and values once: loads that leave nothing in the caches reach more of HBM's rate (16
  // sequences of 4 rows 69 us, 77 without), but more tiles of a sequence share what one leaves there (8192 rows 1020 us, 1054).
  // Beside such loads there is time for P in two parts.
  const bool one_tile = x.one_tile;
  const int kv_end = x.kv_end;
  const int step = CAUSAL ? 1 : x.step;
  const int blocks = (kv_end + kBlockTokens - 1) / kBlockTokens;
  const int32_t* bt = c.block_tables + (int64_t)b * c.max_blocks;
  const float scale = kLog2e / sqrtf((float)D);
  if (TYPE == 0) {
    if (t == 0) s_odd = 0;
    for (int i = t; i < 3 * D; i += 256) (&s_first[0][0])[i] = 0x7fffffff;
  }

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
  const int limit = live ? first_pos + step * own.tok + 1 : 0;
  bf16x8_t q[KK];
  {
    const uint16_t* qp = c.q + ((int64_t)(row0 + (live ? own.tok : 0)) * c.hq + g * group + (live ? own.head : 0)) * D + half * 8;
#pragma unroll
    for (int kk = 0; kk < KK; kk++) q[kk] = as_bf16x8(*(const u32x4_t*)(qp + kk * 16));
  }
  // pairs of a wave are in token order: the fewest and the most keys that its pairs see
  const int wave_first = wave * 32 / group;
  const bool wave_live = wave_first < tokens;
  const int wave_least = first_pos + step * wave_first + 1;
  const int wave_most = wave_live ? first_pos + (step ? min(tokens, (wave * 32 + 31) / group + 1) : 1) : 0;

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
  // The 8-bit cache's scales of a chunk in LDS, [block][K, V][token]: registers 4 j .. 4 j + 3. K's are times the softmax's factor.
  float* const s_scales = (float*)(smem + 2 * kRing * kSide);
  auto scales_at = [&](int slot, int value, int j) -> const f32x4_t& {
    return *(const f32x4_t*)(s_scales + slot * (2 * kChunk) + j / 2 * (2 * kBlockTokens) + value * kBlockTokens + half * 8 + j % 2 * 4);
  };
  auto scales_of = [&](int slot, int value, int j) { return scales_at(slot, value, j); };
  // Where a pair's weights of a chunk have grown too large for its reference (or it has none): the reference moves to the chunk's
  // largest score, the sums with it, and the weights are made again.
  auto weigh = [&](auto parts, int slot, const f32x16_t& s, bf16x8_t (&p)[4], float sum) {
    if (__any(sum > most)) {
      float cm;
      if (TYPE) {
        cm = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const f32x4_t f = scales_of(slot, 0, j);
#pragma unroll
          for (int i = 0; i < 4; i++) cm = fmaxf(cm, s[4 * j + i] * f[i]);
        }
        cm = max_halves(cm);
      } else {
        cm = s[0];
#pragma unroll
        for (int r = 1; r < 16; r++) cm = fmaxf(cm, s[r]);
        cm = max_halves(cm) * scale;
      }
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
        for (int j = 0; j < 2; j++) {
          f32x4_t kf, vf;
          if (TYPE) {
            kf = scales_of(slot, 0, 2 * k + j);
            vf = scales_of(slot, 1, 2 * k + j);
          }
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const int r = 4 * j + i;
            e[r] = __builtin_amdgcn_exp2f(fmaf(s[8 * k + r], TYPE ? kf[i] : scale, base));
            sum += e[r];
            if (TYPE) e[r] *= vf[i];
          }
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
    // scales, the next few registers' ahead: V's four at a time, K's too where there are registers left for it
    constexpr int kFew = D == 64 ? 4 : 2;
    float kf[2][kFew];
    f32x4_t vf[2];
    auto key_scales = [&](int i) {
      const float* from = (const float*)&scales_at(slot, 0, i * kFew / 4) + i * kFew % 4;
      if (kFew == 4) *(f32x4_t*)kf[i % 2] = *(const f32x4_t*)from;
      else *(float2*)kf[i % 2] = *(const float2*)from;
    };
    if (TYPE) {
      key_scales(0);
      vf[0] = scales_of(slot, 1, 0);
    }
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
        if (TYPE && r % kFew == 0 && r + kFew < 16) key_scales(r / kFew + 1);
        if (TYPE && r % 4 == 1 && r < 12) vf[(r / 4 + 1) % 2] = scales_of(slot, 1, r / 4 + 1);  // behind the last use of the quad before
        e[r] = __builtin_amdgcn_exp2f(fmaf(s[r], TYPE ? kf[r / kFew % 2][r % kFew] : scale, base));
        if (TYPE == 0) {
          if (r > 0) sum += e[r - 1];  // a step late: nothing waits for the exponential
        } else {
          if (r % 8 != 0) sum += e[r - 1], e[r - 1] *= vf[(r - 1) / 4 % 2][(r - 1) % 4];
          if (r % 8 == 7) sum += e[r], e[r] *= vf[r / 4 % 2][r % 4];
        }
        if (r % 8 == 7) to_bf16(parts, e + r - 7, p, r / 8);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    weigh(parts, slot, s, p, TYPE ? sum : sum + e[15]);
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
  if constexpr (TYPE != 0) {
    // The 8-bit cache. A thread below 2 D carries 16 bytes of a chunk's K and of its V; the last wave carries the scales.
    const int n_end = c1 - c0, code_blk = min(wave * 64 / D, kChunkBlocks - 1), code_at = t % D;
    const bool carries = kChunkBlocks * D == 64 * kWaves || t < kChunkBlocks * D;
    u32x4_t k_in[2], v_in;
    float s_in;
    auto load_codes = [&](const uint8_t* cache, int at, int n, u32x4_t& v) {
      const int place = __builtin_amdgcn_readlane(at, n % kGroupChunks * kChunkBlocks + code_blk);
      if (!carries) return;
      v = load16<kBlockTokens * D>(cache + (int64_t)place * (kBlockTokens * D), 16 * code_at, false);
    };
    auto load_k = [&](int n, u32x4_t& v) {
      if (n > 0 && n % kGroupChunks == 0) {
        at_k = places(ids_next);
        ids_next = load_ids(c0 + n + kGroupChunks);
      }
      load_codes(c.kv8.k, at_k, n, v);
    };
    int at_s = at_k;
    auto load_v = [&](int n, u32x4_t& v) {
      if (n % kGroupChunks == 0) at_v = at_k;
      load_codes(c.kv8.v, at_v, n, v);
    };
    auto load_s = [&](int n, float& v) {
      if (n % kGroupChunks == 0) at_s = at_k;
      if (wave != kWaves - 1) return;
      const int first = n % kGroupChunks * kChunkBlocks;
      const int p0 = __builtin_amdgcn_readlane(at_s, first), p1 = __builtin_amdgcn_readlane(at_s, first + 1);
      if (half) v = load4<2 * kBlockTokens * 4>(c.kv8.scales + (int64_t)p1 * (2 * kBlockTokens), 4 * col);
      else v = load4<2 * kBlockTokens * 4>(c.kv8.scales + (int64_t)p0 * (2 * kBlockTokens), 4 * col);
    };
    auto spread = [&](u32x4_t w, char* to, int next) {  // 16 codes as bf16: eight here, eight `next` bytes on
      const u32x2_t a = kv8_bf16<TYPE>(w[0]), b = kv8_bf16<TYPE>(w[1]), d = kv8_bf16<TYPE>(w[2]), e = kv8_bf16<TYPE>(w[3]);
      *(u32x4_t*)to = u32x4_t{a[0], a[1], b[0], b[1]};
      *(u32x4_t*)(to + next) = u32x4_t{d[0], d[1], e[0], e[1]};
    };
    auto store_k = [&](u32x4_t w, int slot) {  // a token's 16 dims
      if (carries) spread(w, smem + slot * kSide + code_blk * kBlockBytes + code_at / 16 * 512 + code_at % 16 * 16, 256);
    };
    auto store_v = [&](auto plain, u32x4_t w, int slot, int ch) {  // a dim's 16 tokens; those past kv_end become zeros (anything may stand there)
      if (!decltype(plain)::value && (ch + 1) * kChunk > kv_end) {
        const int left = kv_end - ch * kChunk - code_blk * kBlockTokens;
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = left >= 4 * i + 4 ? w[i] : left <= 4 * i ? 0u : w[i] & ((1u << 8 * (left - 4 * i)) - 1u);
      }
      if (carries) spread(w, smem + (kRing + slot) * kSide + code_blk * kBlockBytes + code_at * 16, D * 16);
    };
    // A token without a scale gets one: the rows that see it are NaN at the end.
    auto store_s = [&](float v, int slot, int ch) {
      if (wave != kWaves - 1) return;
      int at = threadIdx.x;
      asm volatile("" : "+v"(at));  // made again rather than kept, as no register is left for it
      const int token = ch * kChunk + (at >> 5 & 1) * kBlockTokens + at % kBlockTokens;
      const bool value = at & kBlockTokens;
      if ((ch + 1) * kChunk > kv_end && token >= kv_end) v = 1.f;  // of a zero, or masked
      if (__any(v != v)) {
        if (v != v) {
          atomicMin(&s_odd, token);
          v = 0.f;
        }
      }
      // not so small that it is flushed: a masked score stays -inf
      s_scales[slot * (2 * kChunk) + lane] = value ? v : fmaxf(v * scale, 0x1p-126f);
    };
    // P in one part, and loads that leave what they read in the caches: the fewer pairs that HBM bounds go by attn_few.h.
    constexpr auto single = std::false_type{};
    // A turn for chunk c0 + n: K(n + 2), V(n) and the scales of n + 1 go to LDS, into the places of K(n), V(n - 2) and the scales of
    // n - 1, and the registers that held them take K(n + 4), V(n + 1) and the scales of n + 2, these first: all but K's are waited
    // for a turn later. odd: n's last bit. plain: every row sees the chunk whole, and there are those to fetch.
    auto turn8 = [&](auto first, auto plain, auto odd, int n, f32x16_t& s, f32x16_t& s_next, bf16x8_t (&p_last)[4], bf16x8_t (&p)[4]) {
      constexpr bool kFirst = decltype(first)::value, kPlain = decltype(plain)::value;
      constexpr int kOdd = decltype(odd)::value;
      const int ch = c0 + n;
      if (kPlain || n + 2 < n_end) store_k(k_in[kOdd], kOdd);
      __builtin_amdgcn_sched_barrier(0);
      store_v(plain, v_in, kOdd, ch);
      __builtin_amdgcn_sched_barrier(0);
      if (kPlain || n + 1 < n_end) store_s(s_in, 1 - kOdd, ch + 1);
      if (kPlain || n + 2 < n_end) load_s(n + 2, s_in);
      if (kPlain || n + 1 < n_end) load_v(n + 1, v_in);
      if (kPlain || n + 4 < n_end) load_k(n + 4, k_in[kOdd]);
      if (kPlain ? wave_live : ch * kChunk < wave_most) {
        if (!kPlain) mask(ch, s);
        products(first, single, kOdd, s, s_next, p_last, p);
      } else if (!kPlain && !kFirst && (ch - 1) * kChunk < wave_most) {
        add_values(single, 1 - kOdd, p_last);
      }
      meet();
    };
    constexpr auto yes = std::true_type{};
    constexpr auto no = std::false_type{};
    constexpr auto even = std::integral_constant<int, 0>{};
    constexpr auto odd = std::integral_constant<int, 1>{};
    f32x16_t sa, sb;
    bf16x8_t pa[4], pb[4];
    if (t == 64 * (kWaves - 1)) s_odd = 0x7fffffff;  // by the wave that changes it
    load_s(0, s_in);
    load_k(0, k_in[0]);
    if (1 < n_end) load_k(1, k_in[1]);
    load_v(0, v_in);
    store_k(k_in[0], 0);
    store_s(s_in, 0, c0);
    if (1 < n_end) load_s(1, s_in);
    if (1 < n_end) store_k(k_in[1], 1);
    if (2 < n_end) load_k(2, k_in[0]);
    if (3 < n_end) load_k(3, k_in[1]);
    meet();
    if (c0 * kChunk < wave_most) {
      const char* kb = smem + k_lane;
#pragma unroll
      for (int r = 0; r < 16; r++) sa[r] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; kk++)
        sa = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*(const u32x4_t*)(kb + kk * 512)), q[kk], sa, 0, 0, 0);
    }
    meet();  // K(0) is read
    turn8(yes, no, even, 0, sa, sb, pb, pa);
    int n = 1;
    const int plain_end = min(n_end - 4, (first_pos + 1) / kChunk - c0);
    for (; n + 1 < plain_end; n += 2) {
      turn8(no, yes, odd, n, sb, sa, pa, pb);
      turn8(no, yes, even, n + 1, sa, sb, pb, pa);
    }
    for (; n < n_end; n += 2) {
      turn8(no, no, odd, n, sb, sa, pa, pb);
      if (n + 1 < n_end) turn8(no, no, even, n + 1, sa, sb, pb, pa);
    }
    if ((c1 - 1) * kChunk < wave_most) {
      if (n_end & 1) add_values(single, (n_end - 1) % kRing, pa);
      else add_values(single, (n_end - 1) % kRing, pb);
    }
  } else {
    if (one_tile) chunks(std::true_type{});
    else chunks(std::false_type{});
  }
  if (bad) atomicOr(c.err, SIDP_DEVERR_BLOCK);

  // Register r of O^T's tile dt is dim 32 dt + 8 (r / 4) + 4 half + r % 4.
  if (TYPE) {
    if (s_odd < limit) {
#pragma unroll
      for (int dt = 0; dt < DT; dt++)
#pragma unroll
        for (int r = 0; r < 16; r++) o[dt][r] = NAN;
    }
  } else if (s_odd) {
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
  emit(AttnOut<D>{out.at, out.tok, out.head, from, (int64_t)(row0 + out.tok) * c.hq + g * group + out.head, o, sum,
                  most < 0.f ? -INFINITY : -base});
}

}  // namespace

}  // namespace sidp
