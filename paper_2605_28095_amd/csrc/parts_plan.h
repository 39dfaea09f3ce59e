// The arithmetic of the plan of k_attn_parts.hip: the runs that tiles are cut into, and
// the most items and records that a call can have. Whole numbers alone, the same on the
// host and on the GPU.
#pragma once
#include <cstdint>

namespace sidp {

constexpr int kSlotsPerCu = 2;  // workgroups a CU holds
// Runs that a tile is cut into: at least this many chunks, at most this many runs, and only where the longest item is this much
// longer than the runs would be (as in k_attn_rows.hip, which has both sides).
constexpr int kMinRun = 8, kMaxRuns = 32;
constexpr float kCutFrom = 1.75f;
constexpr int kTries = 8;
constexpr int kLeastShared = 4;  // chunks
// Wave items: of at most kWaveShare / 4 of the chunks that a wave has on average, or kWaveLeast.
constexpr int kWaveShare = 5, kWaveLeast = 4;

// Chunks of all tiles: a million rows of 4 a tile are 2^18 tiles, of up to 2^15 chunks each.
typedef uint64_t ChunkSum;

constexpr int larger_of(int a, int b) { return a > b ? a : b; }
constexpr int smaller_of(int a, int b) { return a < b ? a : b; }
constexpr int at_most(ChunkSum n, int most) { return n < (ChunkSum)most ? (int)n : most; }

// For one KV head's items.
constexpr int slots_of(int num_cus, int hkv) { return kSlotsPerCu * larger_of(num_cus, 1) / hkv; }

// A group shares its prefix where its tiles are at most half of its sequences'.
constexpr bool group_shares(int shared_chunks, int group_rows, int own_tiles, int tm) {
  return shared_chunks >= kLeastShared && own_tiles > 0 && 2 * ((group_rows + tm - 1) / tm) <= own_tiles;
}

// Fewer tiles than slots: runs of at most try_run(j, ..) chunks, the shortest of kTries lengths of which no more runs than slots
// come, between an even share of all chunks and one that cannot give more.
constexpr int least_run(ChunkSum total, int slots, int longest) {
  return larger_of(larger_of((int)((total + slots - 1) / slots), kMinRun), (longest + kMaxRuns - 1) / kMaxRuns);
}
constexpr bool tiles_are_cut(int longest, int least) { return longest >= kCutFrom * least; }
constexpr int safe_run(ChunkSum total, int slots, int tiles, int least) {
  return larger_of((int)((total + slots - tiles - 1) / (slots - tiles)), least);
}
constexpr int try_run(int j, int least, int safe) { return least + (safe - least) * j / (kTries - 1); }

// As many tiles as slots, or more: groups' tiles in runs of an even share of all chunks; `slots` of them more than tiles at most.
constexpr int group_run(ChunkSum total, int slots, int longest) {
  return smaller_of(longest, larger_of(at_most(total / slots, longest) + 1, kMinRun));
}
// Chunks of the longest item of a wave.
constexpr int wave_item(ChunkSum total, int waves, int slots, int longest) {
  return larger_of(at_most(total / (waves * larger_of(slots, 1)) * kWaveShare / 4, longest), kWaveLeast);
}

// The most tiles of sequences, items, joined tiles and rows of records.
struct PartsCaps {
  int tiles, entries, cuts, recs;
};
constexpr PartsCaps parts_caps(int batch, int max_rows, int tm, int slots, bool groups) {
  PartsCaps l = {};
  l.tiles = smaller_of(max_rows, max_rows / tm + smaller_of(batch, max_rows));
  // A group's tiles are at most half of its sequences'. With fewer tiles than slots runs are chosen so that they fit the slots;
  // with more only shared tiles are cut, into runs of an even share of all chunks or more.
  l.entries = larger_of(l.tiles, slots) + (groups ? l.tiles / 2 + slots : 0);
  l.cuts = groups ? l.tiles : smaller_of(l.tiles, larger_of(slots, 0));
  // 2 ceil(R / tm) <= sum ceil(rows / tm) <= R / tm + sequences: R of the groups that share is at most tm a sequence
  const int shared = groups ? 2 * at_most((ChunkSum)batch * tm, max_rows) : 0;
  l.recs = shared + slots * smaller_of(tm, max_rows);
  return l;
}

}  // namespace sidp
