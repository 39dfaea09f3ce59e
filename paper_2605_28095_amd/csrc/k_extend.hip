// Block tables, row starts, positions and cache slots of one iteration, from
// request lengths: sequence b has ctx tokens cached and brings `new` more, so it
// needs ceil((ctx + new) / 16) - ceil(ctx / 16) further blocks, which are dealt out
// of the free list in batch order; its i-th new token takes position ctx + i and
// slot table[position / 16] * 16 + position % 16.
//
// Latency alone bounds it (8 bytes written a row): 1 sequence 2.2-2.5 us on the GPU, 256
// with a token each 6.8-7.2, 512 prompts of up to 511 tokens 8.9-9.2, where a call takes 10.5.
// One launch: every workgroup sums all lengths for itself (as k_attn_plan does; a
// second launch or a wait between workgroups would cost more than re-reading 8 bytes a
// sequence from L2), then takes 256 rows, each of which finds its sequence by bisection
// of the row starts in LDS. The row at a block's first position writes the block's
// table entry, so no row waits for another.
#include "common.h"
#include "internal.h"

namespace sidp {

namespace {

// Sums stop here: more rows or blocks than any call has, and twice it is still an int.
constexpr int kFull = (1 << 30) - 1;
__device__ __forceinline__ int add_up(int a, int b) { return min(a + b, kFull); }

__device__ __forceinline__ int wave_scan(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, 64);
    if (lane >= o) v = add_up(v, u);
  }
  return v;
}

__global__ void __launch_bounds__(256) k_kv_extend(ExtendCall c) {
  extern __shared__ int32_t s_lds[];
  int32_t* s_start = s_lds;                // [batch + 1] first row of each sequence
  int32_t* s_block = s_start + c.batch + 1;  // [batch] place in the free list of its first new block
  int32_t* s_ctx = s_block + c.batch;        // [batch] its cached tokens
  __shared__ int s_rows[4], s_blocks[4];
  __shared__ int s_all_rows, s_all_blocks;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int per = (c.batch + 255) / 256;  // thread t sums sequences [b0, b1)
  const int b0 = min(t * per, c.batch), b1 = min(b0 + per, c.batch);
  const int taken = c.taken[0];
  // a cursor outside the list hands out nothing
  const bool in_list = taken >= 0 && taken <= c.num_free;
  const int left = in_list ? c.num_free - taken : 0;
  uint32_t bad = in_list ? 0u : SIDP_DEVERR_POSITION;
  struct Need {
    int rows, blocks;
    bool ok;
  };
  auto need_of = [&](int b) {
    const int ctx = c.ctx_lens[b], n = c.new_lens[b];
    s_ctx[b] = ctx;
    const bool ok = ctx >= 0 && n >= 0 && (int64_t)ctx + n <= (int64_t)c.max_blocks * kBlockTokens;
    const int blocks = ok ? (ctx + n + kBlockTokens - 1) / kBlockTokens - (ctx + kBlockTokens - 1) / kBlockTokens : 0;
    return Need{ok ? n : 0, blocks, ok};
  };
  // a thread's first sequence stays in registers: up to 256 sequences it is its only one
  const Need own = b0 < b1 ? need_of(b0) : Need{0, 0, true};
  int rows = own.rows, blocks = own.blocks;
  bool ok = own.ok;
  for (int b = b0 + 1; b < b1; b++) {
    const Need n = need_of(b);
    rows = add_up(rows, n.rows);
    blocks = add_up(blocks, n.blocks);
    ok &= n.ok;
  }
  if (!ok) bad |= SIDP_DEVERR_POSITION;
  if (t == 0) s_all_rows = s_all_blocks = 0;
  // exclusive sums: of the lanes before this one, then of the waves
  const int rows_end = wave_scan(rows, lane), blocks_end = wave_scan(blocks, lane);
  int r_at = __shfl_up(rows_end, 1, 64), k_at = __shfl_up(blocks_end, 1, 64);
  if (lane == 0) r_at = k_at = 0;
  if (lane == 63) {
    s_rows[wave] = rows_end;
    s_blocks[wave] = blocks_end;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 3; w++)
    if (w < wave) {
      r_at = add_up(r_at, s_rows[w]);
      k_at = add_up(k_at, s_blocks[w]);
    }
  // Sequences fit in batch order: the sums only grow, so the first that does not
  // fit ends it for all behind it, and it alone says why (what those behind it would
  // have met says nothing: the sums go on with rows and blocks that nobody gets).
  int fit_rows = 0, fit_blocks = 0;
  for (int b = b0; b < b1; b++) {
    const Need n = b == b0 ? own : need_of(b);
    const bool open = r_at <= c.max_rows && k_at <= left;
    s_start[b] = min(r_at, c.max_rows);
    s_block[b] = min(k_at, left);
    r_at = add_up(r_at, n.rows);
    k_at = add_up(k_at, n.blocks);
    if (r_at <= c.max_rows && k_at <= left) {
      fit_rows = r_at;
      fit_blocks = k_at;
    } else if (open) {
      bad |= r_at > c.max_rows ? SIDP_DEVERR_POSITION : SIDP_DEVERR_NOBLOCKS;
    }
  }
  if (fit_rows) atomicMax(&s_all_rows, fit_rows);
  if (fit_blocks) atomicMax(&s_all_blocks, fit_blocks);
  __syncthreads();
  const int total = s_all_rows;
  if (t == 0) s_start[c.batch] = total;
  if (blockIdx.x == 0) {
    for (int b = t; b <= c.batch; b += 256) c.row_starts[b] = b < c.batch ? min(s_start[b], total) : total;
    if (t == 0 && c.taken_out) c.taken_out[0] = taken + s_all_blocks;
  }

  const int row = blockIdx.x * 256 + t;
  if (row < total) {
    int lo = 0, hi = c.batch;  // the last sequence that starts at or before the row
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_start[mid] <= row) lo = mid;
      else hi = mid;
    }
    const int ctx = s_ctx[lo], pos = ctx + row - s_start[lo];
    const int have = (ctx + kBlockTokens - 1) / kBlockTokens, j = pos / kBlockTokens;
    int32_t* entry = c.block_tables + (int64_t)lo * c.max_blocks + j;
    int blk = j >= have ? c.free_blocks[taken + s_block[lo] + (j - have)] : *entry;
    if (blk < 0 || blk >= c.nblk) {
      blk = -1;
      bad |= SIDP_DEVERR_BLOCK;
    }
    if (j >= have && pos % kBlockTokens == 0) *entry = blk;
    c.positions[row] = pos;
    c.slots[row] = blk < 0 ? -1 : blk * kBlockTokens + pos % kBlockTokens;
  }
  if (bad) atomicOr(c.err, bad);
}

// The cursor alone, behind a launch that read it (taken_out may be taken itself).
__global__ void k_move_cursor(const int32_t* __restrict__ ctx_lens, const int32_t* __restrict__ row_starts, int batch,
                              int32_t* taken) {
  const int lane = threadIdx.x;
  int n = 0;
  for (int b = lane; b < batch; b += 64) {
    const int rows = row_starts[b + 1] - row_starts[b];
    const int ctx = rows > 0 ? ctx_lens[b] : 0;
    n += (ctx + rows + kBlockTokens - 1) / kBlockTokens - (ctx + kBlockTokens - 1) / kBlockTokens;
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) n += __shfl_xor(n, o, 64);
  if (lane == 0) *taken += n;
}

}  // namespace

hipError_t launch_kv_extend(ExtendCall c, hipStream_t s) {
  const bool in_place = c.taken == c.taken_out;
  if (in_place) c.taken_out = nullptr;
  const int64_t groups = std::max<int64_t>(1, ((int64_t)c.max_rows + 255) / 256);
  k_kv_extend<<<(unsigned)groups, 256, (3 * (size_t)c.batch + 1) * sizeof(int32_t), s>>>(c);
  if (in_place) k_move_cursor<<<1, 64, 0, s>>>(c.ctx_lens, c.row_starts, c.batch, const_cast<int32_t*>(c.taken));
  return hipGetLastError();
}

}  // namespace sidp
