// Device-side pieces shared by the sliding-window attention kernels: which
// tiles a row block visits, what a tile's mask needs, and the order of heads.
//
// Query i sees key j iff j <= i and (i - j < window or j < sinks), both below
// the sequence's length n (lens[b], or S).
#pragma once

#include "attn_device.h"
#include "block_launch.h"

namespace cattn {

// A value that is the same in every lane, into a scalar register (the compiler
// leaves what a division gives in vector ones, and all that follows from it).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// x, by a way the compiler cannot see through: what is formed from it in a rare
// branch is not formed before the loop and kept in registers.
__device__ __forceinline__ int opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Tokens of sequence b.
__device__ __forceinline__ int swa_len(const int* lens, int b, int S) { return lens ? min(max(lens[b], 0), S) : S; }

// The i-th query head of n in the order work groups take them.  Work group i runs
// on chiplet i % 8.  With a multiple of 8 key/value heads, each chiplet takes every
// eighth of them, with all its query heads (which share its tiles in one L2): the
// heads of one sequence, which in a padded batch may be short, are then spread
// over the chiplets (B8 H12 S1024 D64, lengths 512 .. 1024, window 256, forward and
// backward: 65.4 -> 62.9 us against a sequence per chiplet).  With fewer, n / 8
// consecutive heads.
__device__ __forceinline__ int swa_head(int i, int n, int group) {
  if (n / group % 8 == 0) return (i & 7) * group + (i >> 3) / group * 8 * group + (i >> 3) % group;
  return n % 8 == 0 ? (i & 7) * (n >> 3) + (i >> 3) : i;
}

// Masks of a score block.  Its 16 elements of a lane are rows base + acc_row(e, 0)
// of a tile, base = first row + 4 half: bits 0 .. 27 of a word, set where the pair
// is seen, formed once per lane and tile from the ends of what its column sees; an
// element then takes two instructions (bit to all ones, bitwise select).  With
// comparisons per element, six, a masked tile cost a wave 450 cycles: B8 H12 S1024
// D64 window 32 / 256, forward 16.1 / 20.7 -> 14.9 / 19.6 us; B4 H16 S2048 D128 window
// 256 46.9 -> 44.7.
__device__ __forceinline__ unsigned bits_below(int n) { return (1u << min(max(n, 0), 31)) - 1; }  // bits 0 .. n - 1 (of 28)
// Keys from key0 on that `query` sees.
__device__ __forceinline__ unsigned swa_keys(int query, int key0, int window, int sinks) {
  const int n = query - key0 + 1;
  return bits_below(n) & (~bits_below(n - window) | bits_below(sinks - key0));
}
// Queries lo .. hi - 1, from query0 on.
__device__ __forceinline__ unsigned swa_queries(int lo, int hi, int query0) {
  return bits_below(hi - query0) & ~bits_below(lo - query0);
}
__device__ __forceinline__ void swa_mask(f32x16& s, unsigned seen) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float score = s[e];  // (a bit cast of the element itself reads element 0)
    const int keep = __builtin_amdgcn_sbfe(seen, acc_row(e, 0), 1), bits = __builtin_bit_cast(int, score);
    s[e] = __builtin_bit_cast(float, (keep & bits) | (~keep & (int)0xff800000));  // or -inf
  }
}

// The 32-key tiles that queries [q0, q1) see: the sinks' tiles 0 .. sink_tiles-1,
// then first .. first + n - sink_tiles - 1.
struct KeyTiles {
  int sink_tiles, first, n;
  int with_sinks;  // indexes below hold sinks, wherever the window begins
  __device__ __forceinline__ KeyTiles(int q0, int q1, int window, int sinks) {
    const int last = (q1 - 1) / 32;
    first = max(q0 - window + 1, 0) / 32;
    with_sinks = (min(sinks, q1) + 31) / 32;
    sink_tiles = min(with_sinks, first);
    n = sink_tiles + last - first + 1;
  }
  __device__ __forceinline__ int tile(int x) const { return x < sink_tiles ? x : x - sink_tiles + first; }
};

// Of a work group's tiles, by index x: which a wave with queries [q, q + 32) below
// `len` sees any key of (those with sinks, and [lo, hi]), and which hold a pair
// that is hidden (below edge: outside the window of some query, the sinks' tiles
// before the window with them; from diag on: the diagonal).  Compares against
// indexes formed once.
struct WaveTiles {
  int with_sinks, lo, hi, edge, diag;
  __device__ __forceinline__ WaveTiles(const KeyTiles& kt, int q, int len, int window) {
    const int shift = kt.sink_tiles - kt.first;
    with_sinks = kt.with_sinks;
    lo = max(q - window + 1, 0) / 32 + shift;
    hi = q < len ? (min(q + 32, len) - 1) / 32 + shift : -1;
    edge = (max(q + 32 - window, 0) + 31) / 32 + shift;
    diag = q / 32 + shift;
  }
  __device__ __forceinline__ bool seen(int x) const { return x <= hi && (x >= lo || x < with_sinks); }
  __device__ __forceinline__ bool masked(int x) const { return x < edge || x >= diag; }
};

// Whether any pair of queries [q, q + 32) and the tile at k0 is hidden.
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
