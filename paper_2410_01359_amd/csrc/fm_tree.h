// Trees of drafted tokens, and the chunk of a sequence's keys that a workgroup works on.
#pragma once
#include "fm_cache_math.h"
#include "fm_serving.h"

namespace fm {

// Token t follows token parents[t] < t, or the sequence itself (any other value).  Its row is as many rows behind the first
// new one as it has ancestors in the tree, and of the drafted tokens it sees those and itself.
template <int MOST>
struct TreeOf {
  unsigned ancestors[MOST][MOST / 32];   // of a token, itself among them
  int depth[MOST];
  __device__ __forceinline__ bool on_path(int t, int u) const { return ancestors[t][u / 32] >> (u % 32) & 1; }
};
using Tree = TreeOf<FM_MOST_NEW_TOKENS>;
using SmallTree = TreeOf<64>;

// Of up to 64 tokens, by a wave for itself: lane t has token t's parent.  Lines double their reach in each turn.  Waves that share the tree write the same,
// so that none waits for another (8 trees of 60 tokens over ragged caches of 3000, 8 heads of 64, by decode_kernel: 25.5 us by all waves together ahead of
// everything, 21.1 so).
__device__ __forceinline__ void plant_small(SmallTree& tree, int parent, int T) {
  const int lane = threadIdx.x & 63;
  int ahead = lane < T && parent >= 0 && parent < lane ? parent : -1;   // the first of the line that is not among the bits
  unsigned long long line = 1ull << lane;
  while (__any(ahead >= 0)) {
    const int from = ahead >= 0 ? ahead : lane;
    const unsigned low = __shfl((unsigned)line, from), high = __shfl((unsigned)(line >> 32), from);
    const int next = __shfl(ahead, from);
    if (ahead >= 0) {
      line |= (unsigned long long)high << 32 | low;
      ahead = next;
    }
  }
  tree.ancestors[lane][0] = (unsigned)line;
  tree.ancestors[lane][1] = (unsigned)(line >> 32);
  tree.depth[lane] = __popcll(line) - 1;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // LDS serves a wave in order
}

// By a workgroup of at least T threads.  Every token walks up its line; parents come before their children, so that ends.
__device__ __forceinline__ void plant(Tree& tree, const int* parents, int T) {
  const int t = threadIdx.x;
  if (t < T) {
    const int p = parents[t];
    tree.depth[t] = p >= 0 && p < t ? p : -1;
#pragma unroll
    for (int w = 0; w < FM_MOST_NEW_TOKENS / 32; ++w) tree.ancestors[t][w] = 0;
  }
  barrier_nofence();
  int depth = -1;
  if (t < T)
    for (int u = t; u >= 0; u = tree.depth[u], ++depth) tree.ancestors[t][u / 32] |= 1u << (u % 32);
  barrier_nofence();
  if (t < T) tree.depth[t] = depth;
  barrier_nofence();
}

// A chunk of a sequence's keys, by the cut that fm_cache_index.h describes: all sequences' keys in about `meant` pieces of one size, at least `least` and
// a multiple of `round` groups, each sequence in whole ones.
struct Chunk {
  int b, number, of, slot;   // sequence, which of its chunks, first partial result of the sequence
  int len, begin, end;       // tokens of the sequence; keys
};
// Unit `unit` of such a cut; false: there are fewer.  groups_of(len): groups of a sequence; every wave works this out for itself, 64 sequences at a time.
// ONCE: up to 64 sequences in `meant` pieces at most, where pieces of up to twice the size allow that: as many as run at once.
template <bool ONCE, class Groups>
__device__ __forceinline__ bool find_chunk(const int* lens, int B, const FmDivisor& meant, int least, int round, int unit, const Groups& groups_of,
                                           Chunk& chunk) {
  const int lane = threadIdx.x & 63;
  int lane_len = lane < B ? lens[lane] : 0;
  const auto lane_groups = [&](int base) {
    if (B > 64) lane_len = base + lane < B ? lens[base + lane] : 0;
    return groups_of(lane_len);
  };
  unsigned total = 0;
  for (int base = 0; base < B; base += 64) total += wave_last(wave_scan(lane_groups(base)));
  int size = fm_chunk_groups(total, meant, least, round);
  if (ONCE && B <= 64) {
    const int groups = lane < B ? lane_groups(0) : 0;
    const auto pieces = [&](int size) { return wave_last(wave_scan(lane < B ? fm_chunks_of(groups, size) : 0)); };
    if (pieces(size) > (int)meant.n && pieces(2 * size) <= (int)meant.n) {
      int low = size, high = 2 * size;   // too many, few enough
      while (high - low > round) {
        const int middle = low + (high - low) / (2 * round) * round;
        if (pieces(middle) > (int)meant.n) low = middle;
        else high = middle;
      }
      size = high;
    }
  }
  for (int units = 0, slots = 0, base = 0; base < B; base += 64) {
    const int n = base + lane < B ? fm_chunks_of(lane_groups(base), size) : 0;
    const int upto = wave_scan(n), upto_slots = wave_scan(n > 1 ? n : 0);
    const unsigned long long behind = __ballot(units + upto > unit);
    if (behind) {
      const int at = __builtin_ctzll(behind);
      chunk.b = base + at;
      chunk.of = __builtin_amdgcn_readlane(n, at);
      chunk.number = unit - (units + __builtin_amdgcn_readlane(upto, at) - chunk.of);
      chunk.slot = slots + __builtin_amdgcn_readlane(upto_slots, at) - (chunk.of > 1 ? chunk.of : 0);
      chunk.len = __builtin_amdgcn_readlane(lane_len, at);
      return true;
    }
    units += wave_last(upto);
    slots += wave_last(upto_slots);
  }
  return false;
}

}  // namespace fm
