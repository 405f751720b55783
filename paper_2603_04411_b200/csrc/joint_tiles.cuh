// Joint K tiles: the partly full tiles of one sequence, laid together for the K-score kernels.
#pragma once
#include "twkv_dev.h"

namespace twkv {

// Joint tiles.  A key (sequence, class) ends with a tile that is partly full, and sixteen of those cost a short sequence several times
// its tokens: the K-score kernel pays for a tile, not for its rows.  The last tiles of a sequence are therefore laid together, from the
// widest class to the narrowest, as long as their rows (rounded up to boxes of sixteen) fit one tile; it has the class of its first, and
// the narrower ones' missing panels are zeros.  Every row is computed as in a tile of its own, so the scores are the same bit for bit.
// A decode call in us, a tile per class / joint tiles: 16 x 500 82.7 / 60.5, 64 x 1000 216 / 146, 37 x 700 of any rank 140 / 105,
// 32 x 2000 139 / 111, 4 x 1000 44.7 / 41.7, 8 x 5000 74.3 / 72.2; long sequences, whose tiles are nearly all full, pay for the tables:
// 1 x 30000 62.4 / 64.6, 4 x 8192 61.0 / 62.7.
// Returns the classes (bit class - 1) at which a joint tile starts, and << 16 the classes that lie in one.
__device__ inline unsigned joint_masks(const DevView& v, int layer, int seq) {
  const int* fill = v.fill_l(layer) + (size_t)seq * v.NC;
  int boxes[TWKV_MAX_CLASSES];
#pragma unroll
  for (int k = 0; k < TWKV_MAX_CLASSES; ++k) boxes[k] = k < v.NC ? ((fill[k] & (TILE - 1)) + JOINT_ROWS - 1) / JOINT_ROWS : 0;
  unsigned starts = 0u, joined = 0u, run = 0u, first = 0u;       // of the run being laid together: its classes, the widest
  int used = 0;
#pragma unroll
  for (int k = TWKV_MAX_CLASSES - 1; k >= 0; --k) {
    const int b = boxes[k];
    if (b == 0 || b == TILE / JOINT_ROWS) continue;
    if (used + b > TILE / JOINT_ROWS) {
      if (run != first) { starts |= first; joined |= run; }
      run = 0u; used = 0;
    }
    if (run == 0u) first = 1u << k;
    run |= 1u << k;
    used += b;
  }
  if (run != first) { starts |= first; joined |= run; }
  return starts | (joined << 16);
}

// One warp writes the tables of the joint tile of sequence `seq` that starts at class index k0 (bit k0 of the masks).
__device__ inline void joint_tile(const DevView& v, int layer, int seq, unsigned masks, int k0, int id) {
  const int lane = threadIdx.x & 31;
  const unsigned below = masks & ((1u << k0) - 1u);               // the next joint tile's first class, if any, ends this one
  unsigned members = (masks >> 16) & ((2u << k0) - 1u);
  if (below) members &= ~((2u << (31 - __clz(below))) - 1u);
  const bool in = lane < TWKV_MAX_CLASSES && ((members >> lane) & 1u);
  const int key = seq * v.NC + lane;
  const int rest = in ? v.fill_l(layer)[key] & (TILE - 1) : 0, tile = in ? v.key_last_l(layer)[key] : 0;
  const int block = in ? v.desc(layer, 0)[tile].w : 0, room = (rest + JOINT_ROWS - 1) / JOINT_ROWS * JOINT_ROWS;
  int at = room;                                                  // wide classes first: the rooms of the lanes above
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_down_sync(0xffffffffu, at, o);
    if (lane + o < 32) at += u;
  }
  at -= room;
  int slot[4] = {-1, -1, -1, -1};
  unsigned box = 0u;
  for (unsigned m = members; m; m &= m - 1) {
    const int k = __ffs(m) - 1;
    const int a = __shfl_sync(0xffffffffu, at, k), n = __shfl_sync(0xffffffffu, rest, k), rm = __shfl_sync(0xffffffffu, room, k);
    const int t = __shfl_sync(0xffffffffu, tile, k), b = __shfl_sync(0xffffffffu, block, k);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = 32 * j + lane - a;
      if (r >= 0 && r < n) slot[j] = t * TILE + r;
    }
    const int r = JOINT_ROWS * lane - a;
    if (r >= 0 && r < rm) box = (unsigned)((b * TILE + r) / JOINT_ROWS) << 5 | (unsigned)(k + 1);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v.joint_rows()[(size_t)id * TILE + 32 * j + lane] = slot[j];
    v.joint_pos()[(size_t)id * TILE + 32 * j + lane] = slot[j] >= 0 ? v.aux(layer, 0)[slot[j]] : 0;
  }
  if (lane < TILE / JOINT_ROWS) v.joint_boxes()[(size_t)id * (TILE / JOINT_ROWS) + lane] = box;
}

}  // namespace twkv
