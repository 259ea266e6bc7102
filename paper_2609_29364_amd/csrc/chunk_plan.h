// How a batch of chunk_attention becomes items (at most 128 rows of a KV head) and parts of them:
// the host's bounds, which size the grid and the workspace, and the device's rules, by which every
// wave finds its piece from the batch's lengths (no device types, so that the counts can be checked
// by themselves).
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace {

constexpr int kMaxBatch = 8192;
constexpr int kWaves = 4;
constexpr int kWaveRows = 32;
constexpr int kRows = kWaves * kWaveRows;    // query rows (token, head of the group) of an item, at most
constexpr int kStage = 64;                   // tokens of a stage
constexpr int kSlots = 512;                  // workgroups resident on 256 CUs, two each
constexpr int kPerLane = 4;                  // requests a lane looks at where the batch is parted
constexpr int kPartedBatch = 64 * kPerLane;
constexpr int kMaxSplits = 64;

// The most stages a part has.  A slot's fair share of the batch is total / (kSlots / hkv) stages.
// Where the items are fewer than the slots, they are split so that all pieces run in one round
// (the parts beyond the first of each are fewer than total / limit); where they are more, only
// one of more than 1.5 shares is: a part costs its rows' partial results, written and read.
constexpr float split_limit(int items, float total, int hkv) {
  const float slots = (float)kSlots / hkv;
  const float limit = items < slots ? total / (slots - 0.5f * items) : 1.5f * total / slots;
  return limit > 4.f ? limit : 4.f;
}

// Parts of an item of `stages` stages.
constexpr int parts_of(int stages, float limit) {
  const float x = stages / limit;
  const int n = (int)x;
  return std::max(1, std::min(n + (n < x), kMaxSplits));
}

// Where none is split so, the items that would begin a last round less than half full are split
// to fill it: two ragged chunks (193 items a head) 2897 -> 2530 us, 8300 tokens after 24000 3712
// -> 3400.
struct Tail {
  int items, parts;
};
constexpr Tail last_round(int items, int hkv) {
  const int round = kSlots / hkv, over = round ? items % round : 0;
  if (items <= round || over == 0 || 2 * over > round) return Tail{0, 1};
  return Tail{over, std::min(round / over, 16)};
}

// The most parts of a batch, per KV head (see plan()).
int64_t most_places(int32_t hkv) { return 2 * kSlots / hkv + 1; }

// Bounds per KV head: a batch's items, the split ones of them and their parts.
struct Plan {
  int tile;        // rows of an item
  int64_t items;
  int split_items, places;
};

Plan plan(int32_t bs, int32_t total_q, int32_t hq, int32_t hkv, int32_t max_len) {
  Plan p;
  const int64_t stages = ((int64_t)max_len + kStage - 1) / kStage;
  // Where items of 32 or 64 rows still run all at once, their waves part the tokens of short
  // contexts: up to 2048 tokens that is faster than 128 rows after one another (512 tokens of a
  // new request 15.5 -> 13.1 us, four of 350-900 at head_dim 64 20.1 -> 13.6), beyond it the
  // planes are read too often (512 after 8000 88 -> 131 us).
  p.tile = kRows;
  while (stages <= 32 && p.tile > kWaveRows &&
         ((int64_t)total_q * (hq / hkv) / (p.tile / 2) + bs) * hkv <= kSlots)
    p.tile /= 2;
  p.items = (int64_t)total_q * (hq / hkv) / p.tile + bs;
  // Where the items make two rounds or more, parts, their order and the second launch win only if
  // one context is much longer than the rest (us without -> with them, the longest context 4000
  // / 8000 tokens: one single token after it among 200 after 64 48 -> 50 / 86 -> 50, one of 256
  // chunks of 100 tokens 51 -> 32 / 94 -> 32).  Single tokens after a quarter of it to all of it
  // lose 324 -> 331 / 633 -> 636, in windows of 512 86 -> 94 / 84 -> 92; prompts of like lengths 509
  // -> 517 / 1887 -> 1904, ragged ones 541 -> 555 / 1308 -> 1335, of packed documents 206 -> 219 /
  // 367 -> 407.  The host knows the longest context alone: the lone one counts beyond 8192 tokens.
  // Where all contexts are short nothing is split.
  p.split_items = p.places = 0;
  if (bs > kPartedBatch || stages <= (p.items * hkv > 2 * kSlots ? 8192 / kStage : 12)) return p;
  // A tile of s stages has at most 1 + s / limit <= 2 s / limit parts if it is split, and the
  // tiles' s sum to the total: at most 2 total / limit places, where limit is at least the
  // share total / (kSlots / hkv); also at most kMaxSplits and ceil(stages / 4) a tile.
  const int64_t each = std::min<int64_t>(kMaxSplits, (stages + 3) / 4);
  p.places = (int)std::min(most_places(hkv), p.items * each);
  p.split_items = (int)std::min<int64_t>(p.places / 2, p.items);
  if (p.split_items == 0) p.places = 0;   // (more KV heads than workgroups to split for)
  return p;
}

size_t workspace_bytes(const Plan& p, int32_t hkv, int32_t d) {
  // the count, the records, then (max, sum) and rows of every place
  return p.places ? 16 + (size_t)p.split_items * hkv * 16 +
                        (size_t)p.places * hkv * kRows * (8 + (size_t)d * 4) : 0;
}

// What workspace_bytes() is at most for any batch of these heads.  (It does not rise with the batch:
// one token after 4096 is split for every slot of the device, 256 of them are not.)
size_t workspace_bound(int32_t hkv, int32_t d) {
  Plan p{};
  p.places = (int)most_places(hkv);
  p.split_items = p.places / 2;
  if (p.split_items == 0) p.places = 0;
  return workspace_bytes(p, hkv, d);
}

// Workgroups per KV head: the items, and parts beyond the first of each, which are fewer than
// total / limit.
int64_t pieces(const Plan& p, int32_t hkv) {
  return p.items + std::min(p.places, kSlots / hkv + 1);
}

}  // namespace
