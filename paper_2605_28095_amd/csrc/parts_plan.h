// The arithmetic of the plan of k_attn_parts.hip: the runs that tiles are cut into, and
// the most items and records that a call can have. Whole numbers alone, the same on the
// host and on the GPU.
#pragma once
#include <cstdint>

namespace sidp {

constexpr int kSlotsPerCu = 2;  // workgroups a CU holds
// Runs that a tile is cut into: at least kMinRun chunks, at most kMaxRuns runs, and only where the longest item is kCutFrom times as
// long as the runs would be (k_attn_rows.hip has both sides of that). Runs of at least 8 chunks, of 16 and of 4, us a call:
// 4 sequences under 1024 shared bf16 tokens 25, 29, 24; 8 under 2048 28, 31, 28; 32 under 1024 28, 30, 29; over e4m3 1 row of 1000
// 18, 20, 18; 4 x 40 rows of 2000 46, 48, 45; but 16 x 1 of 500 20, 18, 20 and 4 x 1 of 4000 25, 23, 25; longer ones alike. At most
// 32 runs, 16 and 64: over e4m3 1 row of 32000 34, 37, 41, 5 rows 45, 57, 49; 8 rows under 32000 shared bf16 tokens 52, 62, 62; but 1
// row of 8000 26, 24, 25.
constexpr int kMinRun = 8, kMaxRuns = 32;
constexpr float kCutFrom = 1.75f;
constexpr int kTries = 8;
// Chunks of the shortest prefix that is shared. What sharing costs is the join and the group's items (1 to 11 us); what it saves are
// the bytes of the prefix for all rows but one tile's, so that 128 tokens are about where it begins to pay, in calls with many KV
// heads and rows, and few sequences want far more. Shared and not, us a call: 256 rows in 8 groups, 16 heads of 64, bf16, under 128
// 66.5 and 67.5, 192 67 and 73, 256 67 and 77; 256 rows in 32 groups, 8 KV heads of 128, bf16, under 128 75 and 76, 192 78 and 87,
// 1024 95 and 193; the same over e4m3 under 128 57 and 50, 256 60 and 63, 1024 61 and 107; 64 rows in 8, bf16, under 256 34 and 28,
// 768 35 and 37, 2048 45 and 65; 8 rows in 1 under 256 27 and 21, 2048 28 and 25.
constexpr int kLeastShared = 4;
// Wave items: of at most kWaveShare / 4 of the chunks that a wave has on average, or kWaveLeast. With them and without, us a call,
// rows of one with so many keys each: e4m3 512 of 0-300 53 and 63, 256 of 200 34 and 41, 256 of 0-1000 69 and 68; 256 under 8192
// shared bf16 tokens 143 and 150; but with few items, some of them about as long as a wave's share, e4m3 128 of 500-1500 68 and 58,
// 128 of 0-8000 195 and 181. With 3 / 4 of the average 57, 41 and 70, 58 and 183; with 10 / 4 53, 34 and 73, 69 and 258.
constexpr int kWaveShare = 5, kWaveLeast = 4;

// Chunks of all tiles: a million rows of 8 a tile are more than 2^17 tiles, of up to 2^15 chunks each.
typedef uint64_t ChunkSum;

constexpr int larger_of(int a, int b) { return a > b ? a : b; }
constexpr int smaller_of(int a, int b) { return a < b ? a : b; }
constexpr int at_most(ChunkSum n, int most) { return n < (ChunkSum)most ? (int)n : most; }

// For one KV head's items.
constexpr int slots_of(int num_cus, int hkv) { return kSlotsPerCu * larger_of(num_cus, 1) / hkv; }

// A group shares its prefix where its tiles are at most half of its sequences'. Shared all the same, which halves nothing but leaves
// records of every row, 32 sequences of 9 rows (18 tiles, not 32) take 41, 52 and 96 us under 256, 1024 and 4096 bf16 tokens and 43,
// 62 and 134 over e4m3; not shared 27, 59, 110 and 25, 54, 99. 16 sequences 30, 40, 53 and 32, 43, 61; not shared 26, 43, 68 and 24,
// 40, 62.
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
