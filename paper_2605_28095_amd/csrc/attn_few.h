// A tile of few (token, query head) pairs over a run of keys: the rows of attn_tile.h
// where HBM is what bounds them.
//
// The waves of a workgroup share the keys out instead of the pairs: each takes every
// 4th (2nd) chunk of 32 tokens by itself, without a barrier until the end, where their
// parts are joined through LDS; or, where sequences are many and short, each takes an
// item of its own. Keys and values go from HBM to registers, as the fragments that the
// products want:
//   S[token][pair]  = K[token][:] . Q^T[:][pair]    (v_mfma_f32_16x16x32_bf16)
//   O^T[dim][pair] += V^T[dim][token] . P[token][pair]
// bf16 ones as they are. Of codes a lane's 16 bytes of K are 16 dims of its token, which
// make two of the products' steps, Q's dims being dealt out alike; its 16 bytes of V are
// a dim's 16 tokens: four lanes with dims of four tiles exchange theirs, so that each has
// four tokens of all four, the ones whose scores it made, and they become bf16 there.
// Scales and softmax are those of attn_tile.h. With one tile of 16 pairs, where there is
// time for it, P has 16 bits: it is cut to bf16 and what the cut leaves is multiplied as
// well; with two it is rounded to bf16.
//
// bf16 tiles here are of pairs that all see the same keys: a value that is not finite is
// then nobody's to be kept from, and is in both products what it is.
#pragma once
#include "attn_tile.h"

namespace sidp {

namespace {

template <int D, int NT>
constexpr int few_lds() { return kWaves * 16 * NT * (D + 4 + 2) * (int)sizeof(float); }

// NT: tiles of 16 pairs of a wave. sides: 1 or 2 groups of waves, each with pairs of its own; 4 / sides waves share the keys; 0: the
// item is this wave's own. emit(token, head, dim, values of dims dim .. dim + 3 not yet divided, sum, reference).
template <int D, int TYPE, int NT, class Call, class Emit>
__device__ __forceinline__ void attn_few(const Call& c, const AttnTile<false>& x, int sides, const Emit& emit) {
  constexpr bool kTwo = NT == 1;     // P in two parts
  // of bf16 the second part gets 2^-23 of the weight more, as in attn_tile.h: a cut that leaves nothing (of a weight of 1, say) would
  // make 0 * inf of an infinite value. Codes are finite.
  constexpr float kRest = TYPE ? 1.f : 1.f + 0x1p-23f;
  constexpr int J = D / 64;
  constexpr int kGroupChunks = 32;   // chunks whose block ids a wave holds, two lanes each
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int t = threadIdx.x, lane = t & 63, col = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), side = sides == 2 ? wave % 2 : 0;
  const int turn = sides == 0 ? 0 : wave / sides, turns = sides == 0 ? 1 : kWaves / sides;
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
      for (int h = 0; h < 2; h++)  // bf16: 32 dims a step; codes: 64 dims' halves
        q[nt][2 * j + h] = as_bf16x8(*(const u32x4_t*)(qp + (TYPE ? (kg + 4 * j) * 16 + h * 8 : (2 * j + h) * 32 + kg * 8)));
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
  // Keys and values of kDepth chunks on their way, a chunk's K refilled as soon as its scores are made, its V as soon as its values
  // are added: two of codes, 8 KB each, where the registers hold them (16 x 8 rows of codes over 4000 66 us with two, some of them
  // spilled, 61 with one), one of bf16, 16 KB.
  constexpr int kDepth = TYPE && NT == 1 ? 2 : 1;
  constexpr int kLoads = TYPE ? J : 2 * J;  // of 16 bytes a lane, of a block's K or V
  struct Piece {
    u32x4_t code[kChunkBlocks][kLoads];
    f32x4_t scale[kChunkBlocks];  // of codes
  };
  Piece kw[kDepth], vw[kDepth];
  int at_v = at;
  auto load = [&](auto single, auto value, int n, int places, Piece& w) {
    constexpr bool once = decltype(single)::value, kValue = decltype(value)::value;
#pragma unroll
    for (int b = 0; b < kChunkBlocks; b++) {
      const int64_t place = __builtin_amdgcn_readlane(places, n % kGroupChunks * kChunkBlocks + b);
      if constexpr (TYPE != 0) {
        const uint8_t* from = (kValue ? c.kv8.v : c.kv8.k) + place * (kBlockTokens * D);
#pragma unroll
        for (int j = 0; j < J; j++) w.code[b][j] = load16<kBlockTokens * D>(from, 1024 * j + 16 * lane, once);
        const float* scales = c.kv8.scales + place * (2 * kBlockTokens) + (kValue ? kBlockTokens : 0);
        w.scale[b] = __builtin_bit_cast(f32x4_t, load16<kBlockTokens * 4>(scales, 16 * kg, false));
      } else {
        const uint16_t* from = (kValue ? c.kv.v : c.kv.k) + place * (kBlockTokens * D);
#pragma unroll
        for (int j = 0; j < kLoads; j++) {
          if (kValue) {  // tokens 4 kg .. of a dim of tile 2 j, and of tile 2 j + 1
            const u32x2_t lo = load8<kBlockTokens * D * 2>(from, 1024 * j + 32 * col + 8 * kg, once);
            const u32x2_t hi = load8<kBlockTokens * D * 2>(from, 1024 * j + 512 + 32 * col + 8 * kg, once);
            w.code[b][j] = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
          } else {
            w.code[b][j] = load16<kBlockTokens * D * 2>(from, 1024 * j + 16 * lane, once);
          }
        }
      }
    }
  };
  auto fetch_k = [&](auto single, int n, Piece& w) {
    if (n > 0 && n % kGroupChunks == 0) {
      at = places(ids_next);
      ids_next = load_ids(n + kGroupChunks);
    }
    load(single, std::false_type{}, n, at, w);
  };
  auto fetch_v = [&](auto single, int n, Piece& w) {
    if (n % kGroupChunks == 0) at_v = at;
    load(single, std::true_type{}, n, at_v, w);
  };
  const float scale = kLog2e / sqrtf((float)D);
  // The largest of the four lanes that hold a pair's scores.
  auto max_pair = [&](float v) {
    const u32x2_t a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const u32x2_t b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
  };
  auto chunk = [&](auto single, int n, Piece& wk, Piece& wv) {
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
          bf16x8_t k;
          if constexpr (TYPE != 0) {
            const u32x2_t lo = kv8_bf16<TYPE>(wk.code[b][j][2 * h]), hi = kv8_bf16<TYPE>(wk.code[b][j][2 * h + 1]);
            k = as_bf16x8(u32x4_t{lo[0], lo[1], hi[0], hi[1]});
          } else {
            k = as_bf16x8(wk.code[b][2 * j + h]);
          }
#pragma unroll
          for (int nt = 0; nt < NT; nt++) s[nt][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[nt][2 * j + h], s[nt][b], 0, 0, 0);
          if (TYPE == kInt8) __builtin_amdgcn_sched_barrier(0);  // or all codes are spread out at once, past the registers
        }
    }
    float ks[8];
#pragma unroll
    for (int i = 0; i < 8; i++) ks[i] = TYPE ? wk.scale[i / 4][i % 4] * scale : scale;
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
      for (int i = 0; i < 8; i++)
        if (TYPE) e[i] *= wv.scale[i / 4][i % 4];
      if (TYPE && edge) {  // a token that the pair does not see may have no scale
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
        lo[i] = pack_bf2(fmaf(e[2 * i], kRest, -__uint_as_float(a & 0xffff0000u)), fmaf(e[2 * i + 1], kRest, -__uint_as_float(b & 0xffff0000u)));
      }
      p[nt][0] = as_bf16x8(u32x4_t{hi[0], hi[1], hi[2], hi[3]});
      if (kTwo) p[nt][1] = as_bf16x8(u32x4_t{lo[0], lo[1], lo[2], lo[3]});
    }
#pragma unroll
    for (int j = 0; j < J; j++) {
      u32x2_t words[kChunkBlocks][4];  // tokens 4 kg .. 4 kg + 3 of a dim of tiles 4 j .. 4 j + 3 as bf16
#pragma unroll
      for (int b = 0; b < kChunkBlocks; b++) {
        const int left = x.kv_end - token0 - b * kBlockTokens - kg * 4;  // anything may stand past the last key
        if constexpr (TYPE != 0) {
          u32x4_t& v = wv.code[b][j];
          // word i of lane group kg, tokens 4 i of dim tile kg, becomes tokens 4 kg of dim tile i
          const u32x2_t a = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false), d = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
          const u32x2_t e = __builtin_amdgcn_permlane16_swap(a[0], d[0], false, false), f = __builtin_amdgcn_permlane16_swap(a[1], d[1], false, false);
          v = u32x4_t{e[0], e[1], f[0], f[1]};
          if (token0 + kChunk > x.kv_end) {
            const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << 8 * left) - 1u;
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] &= keep;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const u32x4_t v = wv.code[b][2 * j + i / 2];
            words[b][i] = u32x2_t{v[i % 2 * 2], v[i % 2 * 2 + 1]};
            if (token0 + kChunk > x.kv_end) {
              words[b][i][0] &= left >= 2 ? ~0u : left == 1 ? 0xffffu : 0u;
              words[b][i][1] &= left >= 4 ? ~0u : left == 3 ? 0xffffu : 0u;
            }
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; i++) {
        if constexpr (TYPE != 0) {
#pragma unroll
          for (int b = 0; b < kChunkBlocks; b++) words[b][i] = kv8_bf16<TYPE>(wv.code[b][j][i]);
        }
        const bf16x8_t v = as_bf16x8(u32x4_t{words[0][i][0], words[0][i][1], words[1][i][0], words[1][i][1]});
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
  if (NT == 1 || (x.one_tile && sides == 1)) chunks(std::true_type{});
  else chunks(std::false_type{});
  if (bad) atomicOr(c.err, SIDP_DEVERR_BLOCK);

  if (sides == 0) {
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      float sum = l[nt];
      sum += __shfl_xor(sum, 16, 64);
      sum += __shfl_xor(sum, 32, 64);
      const int pair = nt * 16 + col, tok = pair / group;
      if (tok < x.tokens) {
#pragma unroll
        for (int dt = 0; dt < 4 * J; dt++)
          emit(tok, pair - tok * group, dt * 16 + kg * 4, o[nt][dt], sum, most[nt] < 0.f ? -INFINITY : -base[nt]);
      }
    }
    return;
  }
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
