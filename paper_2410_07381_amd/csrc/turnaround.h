// How soon preempted workers hand the execution units over, estimated from a kernel's measured time.  Plain C++
// beside the kernels: the estimates can be looked at without a GPU.
#pragma once
#include <stdint.h>

#include "../../include/tally.h"

namespace tally {

// Eq. 1: the time of the blocks of one fetch, if all blocks last as long.
inline double eq1_turnaround_ms(double latency_ms, uint32_t workers, uint32_t chunk, uint64_t blocks) {
  return blocks == 0 ? 0.0 : latency_ms * (double)workers * (double)(chunk ? chunk : 1) / (double)blocks;
}

// Of workers that pause after `share` of an average block: Eq. 1 with one block, whatever the chunk, times that share.
// (One that is 1, the share of a body that stops between blocks alone, counts the whole fetch.)
inline double workers_turnaround_ms(double latency_ms, uint32_t workers, uint32_t chunk, uint64_t blocks, double share) {
  return eq1_turnaround_ms(latency_ms, workers, share < 1.0 ? 1 : chunk, blocks) * share;
}

// ---- prompts ---------------------------------------------------------------------------------
constexpr uint32_t kPromptRows = 128;                      // rows of a logical block
constexpr uint32_t kPromptTile = 64;                       // tokens of a tile

// Slots for blocks of one head (PromptBodyT): enough wherever the sequences begin.
inline uint32_t prompt_slots(const tally_attn_prompt_args &a) { return a.total / kPromptRows + a.n_seqs; }

// Share of the average block between two looks at the pause word, `every` tiles apart, and the tile after, in
// which the answer is acted on.  How long sequences are is known on the device alone.  A single one is taken to have
// all tokens: its blocks have 2, 4, 6 ... tiles, one of the rows that are left all of them, and without such rows a
// slot has none.  Of several a block may have fewer tiles than lie between two looks, and only ends.
inline double prompt_pause_share(const tally_attn_prompt_args &a, uint32_t every) {
  if (a.n_seqs != 1) return 1.0;
  const uint64_t whole = a.total / kPromptRows, rest = a.total % kPromptRows;
  const uint64_t tiles = whole * (whole + 1) + (rest ? (a.total + (uint64_t)kPromptTile - 1) / kPromptTile : 0);
  const double share = (double)(every + 1) * (double)prompt_slots(a) / (double)tiles;
  return share < 1.0 ? share : 1.0;
}

}  // namespace tally
