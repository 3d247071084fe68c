// weights.h -- tables of the key weights' kernels (msa_kv_weights), made with the plan.
#pragma once

#include <cstdint>

namespace msa {

constexpr int kPairs = 32;        // (row, query head of a KV head) pairs of a tile
constexpr int kGroupKeys = 256;   // keys of a workgroup

// Keys of a sequence of up to kPairs pairs for the four waves of a workgroup (for every KV head):
// wave w takes key0 + w wave_keys and the wave_keys - 1 after it, as far as `last`.
struct StreamItem {
  int32_t seq;
  int32_t row0, nrows;  // the sequence's packed rows
  int32_t last;         // position of the last of them
  int32_t key0;
  int32_t wave_keys;    // a multiple of 32, at most kStreamMost
};
constexpr int kStreamMost = 1024;  // a lane holds the id of one of a wave's blocks

// Tiles tile0 .. tile1 - 1 of a sequence's pairs against 256 of its keys (for every KV head).
struct WeightsItem {
  int32_t seq;
  int32_t key0;
  int32_t row0, nrows;  // the sequence's packed rows
  int32_t tile0, tile1;
  int32_t slot;         // -1: these are all tiles that see the keys; else where the sums go
  int32_t last;         // position of the sequence's last row
};
static_assert(sizeof(WeightsItem) == 32, "loaded as 8 int32");

// Keys whose tiles are in several items: the sums of slots slot0 .. slot0 + parts - 1, in order.
struct WeightsJoin {
  int32_t seq;
  int32_t key0;
  int32_t slot0;
  int32_t parts;
};

}  // namespace msa
