// Device-side pieces shared by the sliding-window attention kernels: which
// tiles a row block visits, what a tile's mask needs, and the order of heads.
//
// Query i sees key j iff j <= i and (i - j < window or j < sinks), both below
// the sequence's length n (lens[b], or S).
#pragma once

#include "attn_device.h"
#include "block_launch.h"

namespace cattn {

// Tokens of sequence b.
__device__ __forceinline__ int swa_len(const int* lens, int b, int S) { return lens ? min(max(lens[b], 0), S) : S; }

// The i-th head of n in the order work groups take them: with n a multiple of
// 8, work group i runs on chiplet i % 8, and each chiplet takes n / 8
// consecutive heads, so that the query heads of a key/value head share its
// tiles in one L2.
__device__ __forceinline__ int swa_head(int i, int n) { return n % 8 == 0 ? (i & 7) * (n >> 3) + (i >> 3) : i; }

// Masks are selects of conditions joined by & and |.  With && and || the compiler
// (ROCm 7.2's) made branches of them, and in one kernel lost the assignment of an
// accumulator's first element in the branch: hidden pairs kept their score.
__device__ __forceinline__ bool swa_sees(int query, int key, int window, int sinks) {
  return (key <= query) & ((query - key < window) | (key < sinks));
}
__device__ __forceinline__ float swa_masked(bool seen, float score) { return seen ? score : -INFINITY; }

// The 32-key tiles that queries [q0, q1) see: the sinks' tiles 0 .. sink_tiles-1,
// then first .. first + n - sink_tiles - 1.
struct KeyTiles {
  int sink_tiles, first, n;
  __device__ __forceinline__ KeyTiles(int q0, int q1, int window, int sinks) {
    const int last = (q1 - 1) / 32;
    first = max(q0 - window + 1, 0) / 32;
    sink_tiles = min((min(sinks, q1) + 31) / 32, first);
    n = sink_tiles + last - first + 1;
  }
  __device__ __forceinline__ int tile(int x) const { return x < sink_tiles ? x : x - sink_tiles + first; }
};

// Whether queries [q, q + 32) see any key of the tile at k0, and whether any
// pair of the two is hidden.
__device__ __forceinline__ bool swa_tile_seen(int q, int k0, int window, int sinks) {
  return k0 <= q + 31 && (q - (k0 + 31) < window || k0 < sinks);
}
__device__ __forceinline__ bool swa_tile_masked(int q, int k0, int window, int sinks) {
  return k0 + 31 > q || (q + 31 - k0 >= window && k0 + 32 > sinks);
}

// Where the partial sums of a sink key's dK (and, 32 D floats on, dV) start:
// [B * Hkv][sink tile][1 + parts][dK, dV][32][D].
__device__ __forceinline__ float* swa_far_slot(const SwaArgs& a, int bkv, int key, int slot, int parts) {
  const int64_t tile = (int64_t)bkv * swa_sink_tiles(a.S, a.sinks) + key / 32;
  return a.far + ((tile * (1 + parts) + slot) * 2 * 32 + key % 32) * a.D;
}

}  // namespace cattn
