// Kernel launchers shared between the kernel sources and the host runtime.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/sidp.h"

namespace sidp {

struct LinearCall {
  const void* x;
  int m, k;
  const void* packed;
  int n;
  int epilogue;
  const void* bias;
  const float* residual;
  void* out;
  float* ws;
  size_t ws_bytes;
  int num_cus;
  // optional RMSNorm of the result (EPI_RESID in place only): norm_out = bf16(rmsnorm(out) * norm_gain)
  const void* norm_gain = nullptr;
  float norm_eps = 0.f;
  void* norm_out = nullptr;
  // leave split-K partials in ws for the consumer to reduce (it must sum them
  // in split order and apply the epilogue); ignored when there is one split
  bool defer_reduce = false;
  // the call runs beside a slot fill (a streamed step)
  bool beside_fill = false;
};

size_t packed_bytes(int n, int k);
bool gemm_fits(int m, int n_cols_packed, int k);  // within the kernels' 32-bit buffer offsets
int gemm_splits(int M, int n_cols_packed, int K, int num_cus);
size_t gemm_ws_bytes(int M, int n_cols_packed, int K, int num_cus);
// The launch launch_linear makes for an [m, k] x [n, k]^T projection: kernel
// 0 = weights into registers (k_gemm_deep, or k_gemm beside a slot fill, on
// unaligned activations and where it is the faster one), 1 = k_gemm_lw (256-row
// workgroups, weight tiles staged in LDS); waves and rows per workgroup;
// split-K count; workgroups launched; bytes of fp32 partials (0 without a split).
struct GemmPlan {
  int kernel, waves, rows, splits, workgroups;
  size_t ws_bytes;
};
GemmPlan plan_linear(int m, int n, int k, int epilogue, int num_cus);
hipError_t launch_pack_linear(const void* w, int n, int k, void* packed, hipStream_t s);
// W_q [nq, k], W_k and W_v [nkv, k] packed as the one stacked matrix [nq + 2 nkv, k]
hipError_t launch_pack_qkv(const void* wq, const void* wk, const void* wv, int nq, int nkv, int k, void* packed,
                           hipStream_t s);
hipError_t launch_pack_gate_up(const void* wg, const void* wu, int f, int k, void* packed, hipStream_t s);
hipError_t launch_linear(const LinearCall& c, hipStream_t s);

hipError_t launch_rmsnorm(const float* x, const void* gain, float eps, void* out, int rows, int n, hipStream_t s);
bool reduce_resid_norm_fits(int n);
hipError_t launch_reduce_resid_norm(const float* ws, int splits, int M, int NP, int n, float* x, const void* gain,
                                    float eps, void* h, hipStream_t s);

struct KvView {
  uint16_t* k;            // [regions][nblk][Hkv][D / 8][bs][8]
  uint16_t* v;            // [regions][nblk][Hkv][D][bs]
  int nblk, regions;
  int hkv, d, bs;
};

struct RopeCall {
  const uint16_t* qkv;    // bf16 projection output [B][heads * D], or
  const float* ws;        // its split-K partials [splits][B][ws_np] (reduced here, in split order, + bias)
  int splits, ws_np;
  const uint16_t* bias;   // with ws only
  const int32_t* positions;
  const int32_t* block_tables;
  int max_blocks, batch;
  int hq, hkv, d;
  const uint16_t* g_q;
  const uint16_t* g_k;
  float qk_eps;
  const float* rope_cos;  // [max_seq][D/2]
  const float* rope_sin;
  int max_seq;
  int rot;                // leading dims that are turned, a multiple of 16
  bool interleaved;       // pairs (2 i, 2 i + 1) instead of (i, i + rot / 2)
  KvView kv;
  int region;
  uint16_t* q_out;
  uint32_t* err;
  bool beside_fill = false;  // the call runs beside a slot fill (a streamed step)
};
hipError_t launch_rope_append(const RopeCall& c, hipStream_t s);
hipError_t launch_slot_mapping(const int32_t* positions, const int32_t* bt, int max_blocks, int batch, int bs,
                               int nblk, int32_t* slots, uint32_t* err, hipStream_t s);

// Many rows at given positions and cache slots: see sidp_rope_append_rows.
struct RopeRowsCall {
  const uint16_t* qkv;       // [rows][stride]
  int64_t stride;
  int rows;
  const int32_t* row_count;  // rows in use, or null
  const int32_t* positions;
  const int32_t* slots;
  int hq;
  const uint16_t* g_q;
  const uint16_t* g_k;
  float qk_eps;
  const float* rope_cos;
  const float* rope_sin;
  int max_seq, rot;
  bool interleaved;
  KvView kv;
  int region;
  uint16_t* q_out;
  uint32_t* err;
};
bool rope_rows_fit(int rows, int hkv);  // in one launch
hipError_t launch_rope_rows(const RopeRowsCall& c, hipStream_t s);

// The 8-bit cache: codes, and the scales of each block's K and V tokens.
struct Kv8View {
  uint8_t* k;     // [regions][nblk][Hkv][D / 16][bs][16]
  uint8_t* v;     // [regions][nblk][Hkv][D][bs]
  float* scales;  // [regions][nblk][Hkv][2][bs]
  int type;       // SIDP_KV_E4M3 or SIDP_KV_INT8
  int nblk, regions;
  int hkv, d;
};
// kv: its counts only
struct RopeRows8Call : RopeRowsCall {
  Kv8View kv8;
};
hipError_t launch_rope_rows8(const RopeRows8Call& c, hipStream_t s);
struct Kv8ReadCall {
  Kv8View kv8;
  int region;
  int rows;
  const int32_t* row_count;
  const int32_t* slots;
  uint16_t* k_out;  // [rows][Hkv][D] or null
  uint16_t* v_out;
  uint32_t* err;
};
bool kv8_read_fits(int rows, int hkv);  // in one launch
hipError_t launch_kv8_read(const Kv8ReadCall& c, hipStream_t s);

// Angle per position of the rot / 2 pairs, in turning order, and the factor on
// cos and sin (host only). False for a rope that a head of `head_dim` cannot have.
bool rope_frequencies(const sidp_rope& r, int head_dim, double* freqs, double* scale);
// cos and sin tables [positions][head_dim / 2] (host): entry p, i is the cosine of
// p * freqs[i] in double precision, times scale, stored as fp32; 0 from `pairs` on.
void rope_tables(const double* freqs, int pairs, double scale, int positions, int head_dim, float* cos, float* sin);

constexpr int kBlockTokens = 16;  // tokens of a KV block

struct ExtendCall {
  const int32_t* ctx_lens;
  const int32_t* new_lens;
  int batch;
  const int32_t* free_blocks;
  int num_free;
  const int32_t* taken;
  int32_t* taken_out;
  int32_t* block_tables;
  int max_blocks;
  int max_rows;
  int nblk;
  int32_t* row_starts;
  int32_t* positions;
  int32_t* slots;
  uint32_t* err;
};
hipError_t launch_kv_extend(ExtendCall c, hipStream_t s);

struct LogprobCall {
  const void* logits;
  bool f32;
  int rows, vocab;
  int64_t stride;
  const int32_t* targets;
  int top;
  float* logprob;
  int32_t* rank;
  float* entropy;
  int32_t* top_ids;
  float* top_logprobs;
  void* ws;
  // set by launch_logprobs
  int segments = 0;
  void* stats = nullptr;
  void* keys = nullptr;
};
size_t logprob_ws_bytes(int rows, int vocab, int top);
hipError_t launch_logprobs(LogprobCall c, hipStream_t s);

struct SampleCall {
  const void* logits;
  bool f32;
  int rows, vocab;
  int64_t stride;
  const float* temperatures;
  const int32_t* top_ks;
  const float* top_ps;
  const float* min_ps;
  const float* uniforms;
  int32_t* tokens;
  float* logprobs;
  int32_t* kept;
  void* ws;
  // set by launch_sample
  int segments = 1;
};
size_t sample_ws_bytes(int rows, int vocab);
hipError_t launch_sample(const SampleCall& c, hipStream_t s);

struct AttnCall {
  const uint16_t* q;  // [B][Hq][D]
  const int32_t* positions;
  const int32_t* block_tables;
  int max_blocks, batch;
  int hq, hkv, d;
  KvView kv;
  int region;
  uint16_t* out;      // [B][Hq][D]
  float* part;        // partials: one record per item of Hq/Hkv*D + 32 floats: o[Hq/Hkv][D], (m, l) per head, pad
  uint32_t* err;
  int num_cus;
  int32_t* plan;      // work list written by launch_attn_plan
};
size_t attn_ws_bytes(int max_batch, int hq, int hkv, int d, int max_seq, int num_cus);
size_t attn_plan_bytes(int max_batch, int num_cus);
// What k_attn_plan and launch_attention make of these positions (host memory).
struct AttnPlan {
  int part_tokens;  // partition length; 2^20 where sequences stay whole
  int items;        // (sequence, partition, KV head)
  bool wave_items;  // a wave takes an item by itself
  bool combine;     // partial records and the combine kernel
};
AttnPlan plan_attention(const int32_t* positions, int batch, int max_tokens, int hkv, int num_cus);
// Builds the work list from positions; needed once per set of positions (a
// decode step shares it across its layers). Reads positions, batch, hkv,
// num_cus, max_blocks, kv.bs, plan, err.
hipError_t launch_attn_plan(const AttnCall& c, hipStream_t s);
// With `start`/`stop`, the events take the start time of the attention's
// first kernel and the end time of its last from those kernels' own
// dispatches (no marker packets between the kernels of the stream).
hipError_t launch_attention(const AttnCall& c, hipStream_t s, hipEvent_t start = nullptr,
                            hipEvent_t stop = nullptr);

// Several new tokens a sequence: see sidp_attention_rows.
struct AttnRowsCall {
  const uint16_t* q;  // [rows][Hq][D]
  const int32_t* row_starts;
  const int32_t* ctx_lens;
  const int32_t* block_tables;
  int max_blocks, batch, max_rows, max_seq;
  int hq;
  KvView kv;
  int region;
  uint16_t* out;
  void* ws;
  uint32_t* err;
  int num_cus;
};
size_t attn_rows_ws_bytes(int batch, int max_rows, int hq, int hkv, int d, int max_seq, int num_cus);
hipError_t launch_attention_rows(const AttnRowsCall& c, hipStream_t s);

// The same over the 8-bit cache (kv8.type other than 0; kv its counts only), or where groups of sequences share their first blocks:
// see sidp_attention_rows8 and sidp_attention_shared.
struct AttnPartsCall : AttnRowsCall {
  Kv8View kv8;
  const int32_t* group_starts;  // [groups + 1]
  const int32_t* shared_lens;   // [groups]
  int groups;
};
size_t attn_parts_ws_bytes(int batch, int max_rows, int hq, int hkv, int d, int num_cus, bool groups);
hipError_t launch_attention_parts(const AttnPartsCall& c, hipStream_t s);

hipError_t launch_copy(const void* src, void* dst, size_t bytes, int grid, hipStream_t s);

// Rows moved between per-replica buffers and one contiguous staging buffer:
// staging row i belongs to replica r with row_off[r] <= i < row_off[r + 1].
constexpr int kMaxReplicas = 16;
struct RowMove {
  void* rep[kMaxReplicas];
  int row_off[kMaxReplicas + 1];
  int n;             // replicas listed
  size_t row_bytes;  // a multiple of 16
  void* staging;
  int gather;        // 1: replicas -> staging; 0: staging -> replicas
};
hipError_t launch_rows_move(const RowMove& m, hipStream_t s);
// loads: 16-byte loads in flight per lane (2, 4 or 8): how hard the fill
// presses on HBM while it shares the chip with the layer kernels
hipError_t launch_fill_bg(const void* src, void* dst, size_t bytes, int num_cus, int loads, hipStream_t s);
hipError_t launch_poison(void* dst, size_t bytes, hipStream_t s);
hipError_t launch_spin(int64_t cycles, hipStream_t s);

}  // namespace sidp
