// Rotation of a head held 8 consecutive dims a lane, D / 8 lanes a head: pairs
// (i, i + rot / 2) or (2 i, 2 i + 1) of the leading `rot` dims, the rest unturned.
// Shared by the KV append kernels. rot is a multiple of 16, so a lane's 8 dims lie
// wholly in one half of the pairs, or behind them.
#pragma once
#include "common.h"
#include "internal.h"

namespace sidp {

// 8 bf16 values; ALIGNED: 16-byte aligned, one load.
template <bool ALIGNED>
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  if (ALIGNED) {
    const u32x4_t u = *(const u32x4_t*)p;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      v[2 * i] = bf2f((uint16_t)(u[i] & 0xffffu));
      v[2 * i + 1] = bf2f((uint16_t)(u[i] >> 16));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = bf2f(p[i]);
  }
}

// The sum of a head's squares, on each of its D / 8 lanes: rotate-half pairs (i, i +
// D/2) first, then pairs of i that differ in their highest bit, and so on down, so
// that the roundings are those of one pair per lane and a butterfly over the lanes.
// Each of the first steps hands half of a lane's sums over and keeps the other half.
template <int D>
__device__ __forceinline__ float head_sum_sq(const float (&x)[8], int sub) {
  constexpr int kLanes = D / 8;
  const bool h4 = sub & (kLanes / 2), h2 = sub & (kLanes / 4), h1 = sub & (kLanes / 8);
  float t[4], u[2];
#pragma unroll
  for (int j = 0; j < 4; j++) {  // dims j of the lane's eight in its first half, 4 + j in its second
    const float own = h4 ? x[4 + j] : x[j];
    const float other = __shfl_xor(h4 ? x[j] : x[4 + j], kLanes / 2, 64);
    const float lo = h4 ? other : own, hi = h4 ? own : other;
    t[j] = fmaf(hi, hi, lo * lo);
  }
#pragma unroll
  for (int j = 0; j < 2; j++) u[j] = (h2 ? t[2 + j] : t[j]) + __shfl_xor(h2 ? t[j] : t[2 + j], kLanes / 4, 64);
  float v = (h1 ? u[1] : u[0]) + __shfl_xor(h1 ? u[0] : u[1], kLanes / 8, 64);
  if (D == 128) v += __shfl_xor(v, 1, 64);
#pragma unroll
  for (int o = kLanes / 2; o >= kLanes / 8; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// One lane's part of a position's angles, for every head of a row.
struct Turn {
  float c[8], s[8];  // cos and signed sin of each dim's pair
  int partner;       // half layout: lane (within the wave) that holds the pairs' other dims
  bool on;           // the lane's dims are turned
};

// cos, sin: the position's row of the tables (rot / 2 entries used). `lane`
// within the wave, `sub` within the head.
__device__ __forceinline__ void load_turn(const float* cos, const float* sin, int rot, bool interleaved, int lane,
                                          int sub, Turn& t) {
  const int d0 = sub * 8;
  t.on = d0 < rot;
  t.partner = lane;
  if (!t.on) return;
  if (interleaved) {
    const f32x4_t cv = *(const f32x4_t*)(cos + d0 / 2), sv = *(const f32x4_t*)(sin + d0 / 2);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      t.c[2 * i] = t.c[2 * i + 1] = cv[i];
      t.s[2 * i] = -sv[i];
      t.s[2 * i + 1] = sv[i];
    }
  } else {
    const bool low = d0 < rot / 2;
    const int i0 = low ? d0 : d0 - rot / 2;
    t.partner = low ? lane + rot / 16 : lane - rot / 16;
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const f32x4_t cv = *(const f32x4_t*)(cos + i0 + i), sv = *(const f32x4_t*)(sin + i0 + i);
#pragma unroll
      for (int j = 0; j < 4; j++) {
        t.c[i + j] = cv[j];
        t.s[i + j] = low ? -sv[j] : sv[j];
      }
    }
  }
}

// The turned dims. Every lane of the wave takes part.
template <bool INTERLEAVED>
__device__ __forceinline__ void turn_dims(const float (&x)[8], const Turn& t, float (&o)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const float other = INTERLEAVED ? x[i ^ 1] : __shfl(x[i], t.partner, 64);
    o[i] = t.on ? fmaf(x[i], t.c[i], other * t.s[i]) : x[i];
  }
}

// The same as bf16.
template <bool INTERLEAVED>
__device__ __forceinline__ u32x4_t turned(const float (&x)[8], const Turn& t) {
  float o[8];
  turn_dims<INTERLEAVED>(x, t, o);
  return u32x4_t{pack_bf2(o[0], o[1]), pack_bf2(o[2], o[3]), pack_bf2(o[4], o[5]), pack_bf2(o[6], o[7])};
}

}  // namespace sidp
