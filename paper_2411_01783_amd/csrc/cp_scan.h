// Prefix sums over lanes, and the sequence that a block of work belongs to.
#pragma once

#include "cp_common.h"

namespace cp {

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) {
  return x < lo ? lo : x > hi ? hi : x;
}

// Sequences of a call whose workgroups (and, of trees, rows) all walk the batch, 64 sequences a step: beyond it that walk
// is what a call does (at 2^20 sequences of one node it would be half a minute).
constexpr int32_t kMaxWalkedBatch = 65535;

// Inclusive prefix sums on the vector pipe (data-parallel moves between lanes; a __shfl is a round
// trip through LDS): over 16 lanes, over the wavefront.
template <int CTRL, int ROWS>
__device__ __forceinline__ int lanes_moved(int x) {   // 0 where no lane moves here
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, true);
}
__device__ __forceinline__ int row_scan(int x) {
  x += lanes_moved<0x111, 0xf>(x);   // row_shr:1, 2, 4, 8
  x += lanes_moved<0x112, 0xf>(x);
  x += lanes_moved<0x114, 0xf>(x);
  x += lanes_moved<0x118, 0xf>(x);
  return x;
}
__device__ __forceinline__ int wave_scan(int x) {
  x = row_scan(x);
  x += lanes_moved<0x142, 0xa>(x);   // lane 15 of a row to the next one: rows 1 and 3
  x += lanes_moved<0x143, 0xc>(x);   // lane 31 to the upper half
  return x;
}

// The sequence that block x of the line of all sequences' blocks belongs to; -1: behind the last one.
// Lane l of a step describes sequence b0 + l by load(b) and the number of its blocks by
// count(description); the description found is spread by its of_lane(l), and *begin is its first
// block. One round trip to memory for up to 64 sequences.
template <typename Seq, typename Load, typename Count>
__device__ __forceinline__ int find_sequence_of_block(int batch, int x, int* begin, Seq* found, Load load,
                                                      Count count) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int b0 = 0; b0 < batch; b0 += 64) {
    const bool in = b0 + lane < batch;
    const Seq mine = load(in ? b0 + lane : b0);
    const int c = in ? count(mine) : 0;
    const int end = wave_scan(c);
    const uint64_t behind = __builtin_amdgcn_ballot_w64(base + end > x);
    if (behind != 0) {
      const int l = __builtin_ctzll(behind);
      *begin = base + __builtin_amdgcn_readlane(end - c, l);
      *found = mine.of_lane(l);
      return b0 + l;
    }
    base += __builtin_amdgcn_readlane(end, 63);
  }
  return -1;
}

}  // namespace cp
