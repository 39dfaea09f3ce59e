// A tile of few (token, query head) pairs over a run of keys of the 8-bit cache: the
// rows of attn_tile.h where HBM is what bounds them.
//
// The waves of a workgroup share the keys out instead of the pairs: each takes every
// 4th (2nd) chunk of 32 tokens by itself, without a barrier until the end, where their
// parts are joined through LDS. Codes go from HBM to registers, as the fragments that
// the products want, and become bf16 there:
//   S[token][pair]  = K[token][:] . Q^T[:][pair]    (v_mfma_f32_16x16x32_bf16)
//   O^T[dim][pair] += V^T[dim][token] . P[token][pair]
// A lane's 16 bytes of K are 16 dims of its token, which make two of the products' steps,
// Q's dims being dealt out alike. Its 16 bytes of V are a dim's 16 tokens; four lanes
// with dims of four tiles exchange theirs, so that each has four tokens of all four, the
// ones whose scores it made. Scales and softmax are those of attn_tile.h, and P has 16
// bits: it is cut to bf16 and what the cut leaves is multiplied as well.
#pragma once
#include "attn_tile.h"

namespace sidp {

namespace {

template <int D, int NT>
constexpr int few_lds() { return kWaves * 16 * NT * (D + 4 + 2) * (int)sizeof(float); }

// NT: tiles of 16 pairs of a wave. sides: 1, 2 or 4 groups of waves, each with pairs of its own; 4 / sides waves share the keys.
// emit(token, head, dim, values of dims dim .. dim + 3 not yet divided, sum, reference).
template <int D, int TYPE, int NT, class Call, class Emit>
__device__ __forceinline__ void attn_few8(const Call& c, const AttnTile<false>& x, int sides, const Emit& emit) {
  constexpr bool kTwo = NT == 1;     // P in two parts
  constexpr int J = D / 64;          // loads of 16 bytes a lane of a block's K, and of its V
  constexpr int kGroupChunks = 32;   // chunks whose block ids a wave holds, two lanes each
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int t = threadIdx.x, lane = t & 63, col = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), side = wave % sides, turn = wave / sides, turns = kWaves / sides;
  const int hkv = c.kv.hkv, group = c.hq / hkv, g = x.g;
  const int pair0 = side * 16 * NT;

  int limit[NT];
  bf16x8_t q[NT][2 * J];
#pragma unroll
  for (int nt = 0; nt < NT; nt++) {
    const int pair = pair0 + nt * 16 + col, tok = pair / group;
    const bool live = tok < x.tokens;
    limit[nt] = live ? x.first_pos + x.step * tok + 1 : 0;
    const uint16_t* qp = c.q + ((int64_t)(x.row0 + (live ? tok : 0)) * c.hq + g * group + (live ? pair - tok * group : 0)) * D;
#pragma unroll
    for (int j = 0; j < J; j++)
#pragma unroll
      for (int h = 0; h < 2; h++) q[nt][2 * j + h] = as_bf16x8(*(const u32x4_t*)(qp + (kg + 4 * j) * 16 + h * 8));
  }
  const int least = x.first_pos + x.step * (pair0 / group) + 1;  // keys that every pair of this wave sees

  f32x4_t o[NT][4 * J];
  float base[NT], most[NT], l[NT];
#pragma unroll
  for (int nt = 0; nt < NT; nt++) {
    base[nt] = 0.f;
    most[nt] = limit[nt] > 0 ? -1.f : kMost;
    l[nt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 4 * J; dt++) o[nt][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // This wave's chunks: c0 + turn + n turns. Block ids as in attn_tile.h.
  const int32_t* bt = c.block_tables + (int64_t)x.b * c.max_blocks;
  const int blocks = (x.kv_end + kBlockTokens - 1) / kBlockTokens;
  const int first = x.c0 + turn, count = first < x.c1 ? (x.c1 - first + turns - 1) / turns : 0;
  const int place0 = c.region * c.kv.nblk;
  bool bad = false;
  auto load_ids = [&](int n) { return bt[min((first + (n + lane / 2) * turns) * kChunkBlocks + lane % 2, blocks - 1)]; };
  auto places = [&](int id) {
    const bool ok = id >= 0 && id < c.kv.nblk;
    bad |= !ok;
    return (place0 + (ok ? id : 0)) * hkv + g;
  };
  int at = 0, ids_next = 0;
  if (count > 0) {
    at = places(load_ids(0));
    ids_next = load_ids(kGroupChunks);
  }
  // Codes of kDepth chunks on their way, a chunk's K refilled as soon as its scores are made, its V as soon as its values are added.
  // With two tiles of pairs the registers hold one chunk's: 16 x 8 rows over 4000 66 us with two, some of them spilled, 61 with one.
  constexpr int kDepth = NT == 1 ? 2 : 1;
  struct Codes {
    u32x4_t code[kChunkBlocks][J];
    f32x4_t scale[kChunkBlocks];
  };
  Codes kw[kDepth], vw[kDepth];
  int at_v = at;
  auto load = [&](auto single, int n, int places, const uint8_t* codes, const float* scales, Codes& w) {
    constexpr bool once = decltype(single)::value;
#pragma unroll
    for (int b = 0; b < kChunkBlocks; b++) {
      const int64_t place = __builtin_amdgcn_readlane(places, n % kGroupChunks * kChunkBlocks + b);
#pragma unroll
      for (int j = 0; j < J; j++) w.code[b][j] = load16<kBlockTokens * D>(codes + place * (kBlockTokens * D), 1024 * j + 16 * lane, once);
      w.scale[b] = __builtin_bit_cast(f32x4_t, load16<kBlockTokens * 4>(scales + place * (2 * kBlockTokens), 16 * kg, false));
    }
  };
  auto fetch_k = [&](auto single, int n, Codes& w) {
    if (n > 0 && n % kGroupChunks == 0) {
      at = places(ids_next);
      ids_next = load_ids(n + kGroupChunks);
    }
    load(single, n, at, c.kv8.k, c.kv8.scales, w);
  };
  auto fetch_v = [&](auto single, int n, Codes& w) {
    if (n % kGroupChunks == 0) at_v = at;
    load(single, n, at_v, c.kv8.v, c.kv8.scales + kBlockTokens, w);
  };
  const float scale = kLog2e / sqrtf((float)D);
  // The largest of the four lanes that hold a pair's scores.
  auto max_pair = [&](float v) {
    const u32x2_t a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const u32x2_t b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
  };
  auto chunk = [&](auto single, int n, Codes& wk, Codes& wv) {
    const int token0 = (first + n * turns) * kChunk;
    const bool edge = token0 + kChunk > least;
    // scores; register r of block b is token 16 b + 4 kg + r
    f32x4_t s[NT][kChunkBlocks];
#pragma unroll
    for (int b = 0; b < kChunkBlocks; b++) {
#pragma unroll
      for (int nt = 0; nt < NT; nt++) s[nt][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < J; j++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
          const u32x2_t lo = kv8_bf16<TYPE>(wk.code[b][j][2 * h]), hi = kv8_bf16<TYPE>(wk.code[b][j][2 * h + 1]);
          const bf16x8_t k = as_bf16x8(u32x4_t{lo[0], lo[1], hi[0], hi[1]});
#pragma unroll
          for (int nt = 0; nt < NT; nt++) s[nt][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[nt][2 * j + h], s[nt][b], 0, 0, 0);
          if (TYPE == kInt8) __builtin_amdgcn_sched_barrier(0);  // or all codes are spread out at once, past the registers
        }
    }
    float ks[8];
#pragma unroll
    for (int i = 0; i < 8; i++) ks[i] = wk.scale[i / 4][i % 4] * scale;
    if (n + kDepth < count) fetch_k(single, n + kDepth, wk);
    bf16x8_t p[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      auto seen = [&](int i) { return token0 + i / 4 * kBlockTokens + kg * 4 + i % 4 < limit[nt]; };
      float e[8], sum = 0.f;
      auto weigh = [&] {
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; i++) e[i] = fmaf(s[nt][i / 4][i % 4], ks[i], base[nt]);
        if (edge) {
#pragma unroll
          for (int i = 0; i < 8; i++) e[i] = seen(i) ? e[i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
          e[i] = __builtin_amdgcn_exp2f(e[i]);
          sum += e[i];
        }
      };
      weigh();
      // The reference moves as in attn_tile.h: where a lane's weights of a chunk have grown too large for it, or there is none.
      if (__any(sum > most[nt])) {
        float cm = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; i++) cm = fmaxf(cm, !edge || seen(i) ? s[nt][i / 4][i % 4] * ks[i] : -INFINITY);
        cm = max_pair(cm);
        const float old = most[nt] < 0.f ? -INFINITY : -base[nt], now = fmaxf(old, cm);
        if (now > -INFINITY) {
          const float alpha = __builtin_amdgcn_exp2f(old - now);
          base[nt] = -now;
          most[nt] = kMost;
          l[nt] *= alpha;
#pragma unroll
          for (int dt = 0; dt < 4 * J; dt++) o[nt][dt] *= alpha;
        }
        weigh();
      }
      l[nt] += sum;
#pragma unroll
      for (int i = 0; i < 8; i++) e[i] *= wv.scale[i / 4][i % 4];
      if (edge) {  // a token that the pair does not see may have no scale
#pragma unroll
        for (int i = 0; i < 8; i++) e[i] = seen(i) ? e[i] : 0.f;
      }
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; i++) {
        if (!kTwo) {
          hi[i] = pack_bf2(e[2 * i], e[2 * i + 1]);
          continue;
        }
        const uint32_t a = __float_as_uint(e[2 * i]), b = __float_as_uint(e[2 * i + 1]);
        hi[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);  // the upper halves
        lo[i] = pack_bf2(e[2 * i] - __uint_as_float(a & 0xffff0000u), e[2 * i + 1] - __uint_as_float(b & 0xffff0000u));
      }
      p[nt][0] = as_bf16x8(u32x4_t{hi[0], hi[1], hi[2], hi[3]});
      if (kTwo) p[nt][1] = as_bf16x8(u32x4_t{lo[0], lo[1], lo[2], lo[3]});
    }
#pragma unroll
    for (int j = 0; j < J; j++) {
#pragma unroll
      for (int b = 0; b < kChunkBlocks; b++) {
        u32x4_t& v = wv.code[b][j];
        // word i of lane group kg, tokens 4 i of dim tile kg, becomes tokens 4 kg of dim tile i
        u32x2_t a = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false), d = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
        const u32x2_t e = __builtin_amdgcn_permlane16_swap(a[0], d[0], false, false), f = __builtin_amdgcn_permlane16_swap(a[1], d[1], false, false);
        v = u32x4_t{e[0], e[1], f[0], f[1]};
        if (token0 + kChunk > x.kv_end) {  // anything may stand past the last key
          const int left = x.kv_end - token0 - b * kBlockTokens - kg * 4;
          const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << 8 * left) - 1u;
#pragma unroll
          for (int i = 0; i < 4; i++) v[i] &= keep;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const u32x2_t lo = kv8_bf16<TYPE>(wv.code[0][j][i]), hi = kv8_bf16<TYPE>(wv.code[1][j][i]);
        const bf16x8_t v = as_bf16x8(u32x4_t{lo[0], lo[1], hi[0], hi[1]});
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
          o[nt][4 * j + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[nt][0], o[nt][4 * j + i], 0, 0, 0);
          if (kTwo) o[nt][4 * j + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[nt][1], o[nt][4 * j + i], 0, 0, 0);
        }
        if (TYPE == kInt8) __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (n + kDepth < count) fetch_v(single, n + kDepth, wv);
  };
  auto chunks = [&](auto single) {
#pragma unroll
    for (int d = 0; d < kDepth; d++)
      if (d < count) {
        fetch_k(single, d, kw[d]);
        fetch_v(single, d, vw[d]);
      }
    for (int n = 0; n < count; n += kDepth)
#pragma unroll
      for (int d = 0; d < kDepth; d++)
        if (n + d < count) chunk(single, n + d, kw[d], vw[d]);
  };
  if (NT == 1 || x.one_tile && sides == 1) chunks(std::true_type{});
  else chunks(std::false_type{});
  if (bad) atomicOr(c.err, SIDP_DEVERR_BLOCK);

  // The waves' parts, [wave][pair][dim] and their references and sums. Register r of O^T's tile dt is dim 16 dt + 4 kg + r.
  constexpr int kRow = D + 4;
  float* const parts = (float*)smem;
  float* const sums = parts + kWaves * 16 * NT * kRow;
#pragma unroll
  for (int nt = 0; nt < NT; nt++) {
    float sum = l[nt];
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    const int at_pair = wave * 16 * NT + nt * 16 + col;
#pragma unroll
    for (int dt = 0; dt < 4 * J; dt++) *(f32x4_t*)(parts + at_pair * kRow + dt * 16 + kg * 4) = o[nt][dt];
    if (kg == 0) *(float2*)(sums + 2 * at_pair) = make_float2(most[nt] < 0.f ? -INFINITY : -base[nt], sum);
  }
  __syncthreads();
  for (int i = t; i < sides * 16 * NT * (D / 4); i += 256) {
    const int pair = i / (D / 4), dim = i % (D / 4) * 4, tok = pair / group;
    if (tok >= x.tokens) break;
    float M = -INFINITY, L = 0.f;
    f32x4_t O = {0.f, 0.f, 0.f, 0.f};
    const int mine = pair / (16 * NT), in_wave = pair % (16 * NT);
    for (int w = mine; w < kWaves; w += sides) M = fmaxf(M, sums[2 * (w * 16 * NT + in_wave)]);
    for (int w = mine; w < kWaves; w += sides) {
      const float2 r = *(const float2*)(sums + 2 * (w * 16 * NT + in_wave));
      const float f = r.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(r.x - M);
      L = fmaf(r.y, f, L);
      O += *(const f32x4_t*)(parts + (w * 16 * NT + in_wave) * kRow + dim) * f;
    }
    emit(tok, pair - tok * group, dim, O, L, M);
  }
}

}  // namespace

}  // namespace sidp
