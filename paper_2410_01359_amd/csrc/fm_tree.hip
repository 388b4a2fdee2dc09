// Attention of trees of drafted tokens whose query rows are many to a K/V head (flashmask_decode_tree; few rows go through decode_kernel).
//
// A workgroup has 128 of the H / Hk * T query rows that share a K/V head, a wave 32 of them, and all waves go over the same keys, 64 at a time through
// LDS: read, and of 8 bits widened, once for 128 rows.  With 32x32x16 products
//     S^T = K Q^T (a lane has 16 keys of each half of the tile, of one query), O^T += V^T P^T (V^T by transpose reads),
// softmax statistics are per lane, a lane's probabilities are the second product's operand as they are, and enter it as sums of two 16-bit values
// (see split2).  Tiles without a masked pair take a short way.
// 16 trees of 63 tokens, 32 heads on 8 of 128, ragged caches of up to 8192 tokens (208 MB): 101 us and the join, of which power takes a part (the clock falls
// to 1.6 - 1.8 GHz).  256 rows to a workgroup of eight waves, half of them at the scores while the others are at the products with the values: the same.
#include <algorithm>

#include "fm_cache_math.h"
#include "fm_common.h"
#include "fm_serving.h"
#include "fm_tree.h"

namespace fm {

constexpr int kTile = 64, kWaveRows = 32, kWaves = 4, kBlockRows = kWaveRows * kWaves, kThreads = 64 * kWaves, kPanelTiles = 64;

template <bool F16>
__device__ __forceinline__ f32x16 mfma_rows(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return mfma32(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c);
}

template <int D>
struct TreeShared {
  alignas(16) char k[2][kTile * TileLayout<D>::RS], v[2][kTile * TileLayout<D>::RS];
  i32x4 bound[kTile];   // of a masked tile
  Tree tree;
  int deepest;
  int flag[kPanelTiles];
  unsigned odd[3][2];   // keys of a masked tile whose values have an infinity or NaN
};

template <int D, bool F16, bool E4M3>
__global__ __launch_bounds__(kThreads, 2) void tree_kernel(FmTreeArgs a, FmDivisor inner, FmDivisor row_blocks, FmDivisor tokens, FmDivisor chunks_meant) {
  using L = TileLayout<D>;
  constexpr int STEPS = D / 16, NDB = D / 32;
  __shared__ TreeShared<D> sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, half = lane >> 5;
  const int workgroup = a.first_workgroup + blockIdx.x, deal = fm_div(workgroup >> 3, inner), member = (workgroup >> 3) - deal * (int)inner.n;
  const int hk = fm_div(member, row_blocks), rb = member - hk * (int)row_blocks.n;
  constexpr int ROUND = FM_TREE_ROUND;
  static_assert(ROUND * FM_KEY_GROUP == kTile);
  const int unit = deal * 8 + (workgroup & 7);
  const auto range_of = [&](int n) { return fm_key_range(n, a.T, a.window, a.columns * a.page_tokens); };
  Chunk chunk = {unit, 0, 1, 0, 0, 0, 0};
  if (a.units) {
    const FM_CONSTANT int* entry = (const FM_CONSTANT int*)(a.units + unit);
    chunk = Chunk{entry[0], entry[2] & 0xffff, entry[2] >> 16, entry[3], entry[1], 0, 0};
    if (chunk.b < 0) return;
  } else if (a.plan) {
    if (!find_chunk<true>(a.lens, a.B, chunks_meant, a.cut.least, ROUND, unit, [&](int n) { return fm_key_groups(range_of(n)); }, chunk)) return;
  } else {
    if (unit >= a.B) return;
    chunk.len = a.lens[unit];
  }
  const FmKeyRange range = range_of(chunk.len);
  const int size = chunk.of > 1 ? fm_even_chunk(fm_key_groups(range), chunk.of, ROUND) * FM_KEY_GROUP : range.hi;
  // (known to be the same in all lanes)
  const int begin = __builtin_amdgcn_readfirstlane(range.lo + chunk.number * size), end = __builtin_amdgcn_readfirstlane(min(range.hi, begin + size));
  if (a.plan && !a.units && chunk.number == 0 && member == 0 && threadIdx.x == 0) a.plan[chunk.b] = int2{chunk.slot, chunk.of};
  const int b = __builtin_amdgcn_readfirstlane(chunk.b), first_row = __builtin_amdgcn_readfirstlane(range.len - a.T);

  // Queries
  const int G = a.H / a.Hk, R = G * a.T, r = rb * kBlockRows + wave * kWaveRows + c;
  const bool real = r < R;
  const int hq = fm_div(min(r, R - 1), tokens), t = min(r, R - 1) - hq * a.T;
  const bool idle = rb * kBlockRows + wave * kWaveRows >= R;   // the wave has no rows
  u32x4 q[STEPS];
  {
    const char* p = (const char*)a.q + 2 * ((long long)b * a.sq.b + (long long)(hk * G + hq) * a.sq.h + (long long)t * a.sq.n);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) q[s] = ldg16(p + 2 * (16 * s + 8 * half));
  }
  const float scale = a.scale * kLog2e * (E4M3 ? a.k_scale[hk] : 1.f);

  const char* k_head = a.k.base + (long long)hk * a.k.head;
  const char* v_head = a.v.base + (long long)hk * a.v.head;
  // Pages of a panel's tiles, a lane to a tile: of each of its groups of 16 keys, -1 where there is none or no key
  int entry[kTile / FM_KEY_GROUP];
  const auto page_of = [&](int tile, int group) { return __builtin_amdgcn_readlane(entry[group], tile); };
  // 16 bits: a wave copies its 16 rows of the tile straight to LDS.  8 bits: a thread has piece i of row i * ROWS + thread / PIECES, and widens it.
  constexpr int PIECES = D / 16, ROWS = kThreads / PIECES, LOADS = E4M3 ? kTile / ROWS : 1;
  static_assert(64 / PIECES <= FM_KEY_GROUP);
  const auto group_of = [&](int i) { return E4M3 ? (i * ROWS + wave * (64 / PIECES)) / FM_KEY_GROUP : wave; };   // that piece i of the wave is of
  int mine[LOADS];   // entry[group_of(i)]
  // First row of that group in its page (of one without a page: rows that are there, and not used)
  const auto rows_of = [&](const char* head, const FmPages& p, int panel, int tile, int i) {
    const int page = __builtin_amdgcn_readlane(mine[i], tile), j = panel + tile * kTile + group_of(i) * FM_KEY_GROUP;
    const int slot = page < 0 ? 0 : j - fm_div(j, a.page) * (int)a.page.n;
    return head + std::max(page, 0) * p.page + (unsigned)slot * (unsigned long long)p.token;
  };
  CopyLanes<D> k_lanes, v_lanes;
  if constexpr (!E4M3) {
    k_lanes.init(lane, a.k.token);
    v_lanes.init(lane, a.v.token);
  }
  u32x4 kraw[LOADS], vraw[LOADS];
  i32x4 bound_raw;
  const auto copy_keys = [&](int buffer, int panel, int tile) {
    tile_load_async<D>(rows_of(k_head, a.k, panel, tile, 0) - CopyLanes<D>::BIAS, k_lanes, sh.k[buffer], wave);
  };
  const auto copy_values = [&](int buffer, int panel, int tile) {
    tile_load_async<D>(rows_of(v_head, a.v, panel, tile, 0) - CopyLanes<D>::BIAS, v_lanes, sh.v[buffer], wave);
  };
  const auto load = [&](int buffer, int panel, int tile) {
    if constexpr (E4M3) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const unsigned row = (i * ROWS + wave * (64 / PIECES)) % FM_KEY_GROUP + lane / PIECES, at = lane % PIECES * 16;
        kraw[i] = ldg16(rows_of(k_head, a.k, panel, tile, i) + (row * a.k.token + at));
        vraw[i] = ldg16(rows_of(v_head, a.v, panel, tile, i) + (row * a.v.token + at));
      }
    } else {
      copy_keys(buffer, panel, tile);
      copy_values(buffer, panel, tile);
    }
  };
  const auto load_bounds = [&](int start) {
    bound_raw = i32x4{0, 0, 0, 0};
    const int j = start + (int)threadIdx.x;
    if (threadIdx.x < kTile && j < a.bound_columns) {
#pragma unroll
      for (int w = 0; w < 4; ++w) bound_raw[w] = a.bounds[w][(size_t)b * a.bound_columns + j];
    }
  };
  // What was loaded is in LDS behind the next barrier.
  const auto store = [&](int buffer) {
    if constexpr (E4M3) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const u32x4 raw = w ? vraw[i] : kraw[i];
          const u32x2 x0 = widen4<F16>(raw[0]), x1 = widen4<F16>(raw[1]), x2 = widen4<F16>(raw[2]), x3 = widen4<F16>(raw[3]);
          char* to = w ? sh.v[buffer] : sh.k[buffer];
          const int key = i * ROWS + (int)threadIdx.x / PIECES, at = threadIdx.x % PIECES * 32;
          *(u32x4*)(to + L::off(key, at)) = u32x4{x0[0], x0[1], x1[0], x1[1]};
          *(u32x4*)(to + L::off(key, at + 16)) = u32x4{x2[0], x2[1], x3[0], x3[1]};
        }
    }
    async_wait<0>();
  };
  const auto pages_of = [&](int tile) {   // which groups have one
    unsigned pages = 0;
#pragma unroll
    for (int g = 0; g < kTile / FM_KEY_GROUP; ++g) pages |= (page_of(tile, g) >= 0 ? 1u : 0u) << g;
    return pages;
  };
  // The values of a masked tile: 0 where there is no key or no page, and where they are infinite or NaN; the keys of the latter are noted.
  const auto clean = [&](int buffer, int turn, int start, int tile) {
    constexpr int ALL = kTile * D / 8;
    const unsigned pages = pages_of(tile);
    for (int i = threadIdx.x; i < ALL; i += kThreads) {
      const int key = i / (D / 8);
      u32x4* at = (u32x4*)(sh.v[buffer] + L::off(key, i % (D / 8) * 16));
      u32x4 v = *at;
      const bool odd = odd_words<F16>(v), none = start + key >= end || !(pages >> (key / FM_KEY_GROUP) & 1);
      if (odd || none) *at = none ? u32x4{0, 0, 0, 0} : without_odd<F16>(v);
      if (odd && !none) atomicOr(&sh.odd[turn][key / 32], 1u << (key % 32));
    }
    barrier_nofence();
  };

  float m = -INFINITY, l = 0.f;
  f32x16 acc[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) acc[db] = f32x16{};
  const int k_off = L::off(c, 16 * half);
  int v_off[2];   // transpose reads: row 4 half + i16 / 4 (+ 8), bytes 32 of the lane's 16 and 8 of its place among them
#pragma unroll
  for (int hi = 0; hi < 2; ++hi) v_off[hi] = L::off(4 * half + ((lane & 15) >> 2) + 8 * hi, (16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2);

  // The lane's row, and where all of them are, [first_row, rows_end): for chunks that need it (plant_tree)
  int row_i = 0, rows_end = 0;
  // Which of the lane's keys of a tile (bit 16 n + 4 q + e: key 32 n + 8 q + 4 half + e) its query sees.  Drafted tokens lie in the order of the bits that
  // their tree has of them: a tile's 64 are a shift of three words, ahead of them everything is seen.
  const auto seen_keys = [&](int buffer, int start, int tile) {
    if (!real || first_row + t < 0) return 0u;
    const int ahead = first_row - start, left = end - start;   // keys that are not drafted ones, and keys
    const int word = -ahead >> 5, shift = -ahead & 31;
    unsigned x[3];
#pragma unroll
    for (int w = 0; w < 3; ++w) {
      const int at = word + w;
      x[w] = at >= 0 && at < FM_MOST_NEW_TOKENS / 32 ? sh.tree.ancestors[t][at] : 0u;
    }
    unsigned long long keys = (unsigned long long)__builtin_amdgcn_alignbit(x[2], x[1], shift) << 32 | __builtin_amdgcn_alignbit(x[1], x[0], shift);
    const auto below = [](int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1ull; };
    unsigned long long prefix = below(ahead);
    if (a.window > 0) prefix &= ~below(row_i - a.window + 1 - start);
    keys = (keys | prefix) & below(left);
    // nibbles of this half, of each 32
    unsigned seen = 0;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      unsigned y = (unsigned)(keys >> (32 * n + 4 * half)) & 0x0f0f0f0fu;
      y = (y | y >> 4) & 0x00ff00ffu;
      seen |= ((y | y >> 8) & 0xffffu) << (16 * n);
    }
    // bounds, and windows that end inside the tree
    if (a.bounds[0] || (a.window > 0 && first_row + a.window < rows_end)) {
#pragma unroll 1
      for (int n = 0; n < 8; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = 8 * n + 4 * half + e, u = start + key - first_row, at = min(max(u, 0), a.T - 1);
          bool sees = a.window <= 0 || u < 0 || sh.tree.depth[t] - sh.tree.depth[at] < a.window;
          if (a.bounds[0]) sees &= !hides(sh.bound[key], row_i);
          if (!sees) seen &= ~(1u << (4 * n + e));
        }
      }
    }
    // keys without a page: their values are 0, and so are their scores
    const unsigned pages = pages_of(tile);
#pragma unroll
    for (int g = 0; g < kTile / FM_KEY_GROUP; ++g)
      if (!(pages >> g & 1)) seen &= ~(0xffu << (8 * g));
    return seen;
  };

  // half_way() is called by waves without rows, too, by itself.
  const auto compute = [&](auto with_mask, int buffer, int turn, int start, int tile, const auto& half_way) {
    constexpr bool MASKED = decltype(with_mask)::value;
    // operands from LDS a few products ahead
    f32x16 s[2] = {};
    {
      constexpr int RING = 4;
      u32x4 ring[RING];
      const auto fetch = [&](int i) { ring[i % RING] = *(const u32x4*)(sh.k[buffer] + L::add_col(k_off, 32 * (i / 2)) + 32 * (i % 2) * L::RS); };
#pragma unroll
      for (int i = 0; i < RING - 1; ++i) fetch(i);
#pragma unroll
      for (int i = 0; i < 2 * STEPS; ++i) {
        if (i + RING - 1 < 2 * STEPS) fetch(i + RING - 1);
        s[i % 2] = mfma_rows<F16>(ring[i % RING], q[i / 2], s[i % 2]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    half_way();
    unsigned seen = ~0u;
    if constexpr (MASKED) {
      seen = seen_keys(buffer, start, tile);
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[n][e] = seen >> (16 * n + e) & 1 ? s[n][e] : -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[n][e]);
    top = fmaxf(top, partner32(top)) * scale;
    // seldom, after the first tiles: bf16 has room for probabilities of up to 2^8 times those at the reference
    constexpr float kGap = F16 ? 0.f : 8.f;
    if (__any(top > m + kGap)) {
      const float now = fmaxf(top, m), alpha = fast_exp2(m - reference(now));
      m = now;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db) acc[db] *= alpha;
    }
    const float ref = reference(m) - kShift<F16>;
    float sum = 0.f;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[n][e] = fast_exp2(fmaf(s[n][e], scale, -ref));
        sum += s[n][e];
      }
    l += sum;
    {
      constexpr int RING = 4;
      u32x4 ring[RING], hi, lo;
      const auto fetch = [&](int i) {
        const char* rows = sh.v[buffer] + i / NDB * 16 * L::RS;
        const auto part = [&](int hi) { return lds_read_tr16(rows + L::add_col(v_off[hi], i % NDB * 64)); };
        ring[i % RING] = __builtin_bit_cast(u32x4, cat4(part(0), part(1)));
      };
      fetch(0);
      fetch(1);
#pragma unroll
      for (int i = 0; i < 4 * NDB; ++i) {
        const int n = i / NDB;   // of 16 keys
        if (i % NDB == 0) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            unsigned x, y;
            split2<F16>(s[n / 2][8 * (n % 2) + 2 * w], s[n / 2][8 * (n % 2) + 2 * w + 1], x, y);
            hi[w] = x;
            lo[w] = y;
          }
        }
        if (i + 2 < 4 * NDB) fetch(i + 2);
        if (i % 2 == 1) {   // two results in turn
          acc[i % NDB - 1] = mfma_rows<F16>(ring[(i - 1) % RING], lo, acc[i % NDB - 1]);
          acc[i % NDB] = mfma_rows<F16>(ring[i % RING], lo, acc[i % NDB]);
          acc[i % NDB - 1] = mfma_rows<F16>(ring[(i - 1) % RING], hi, acc[i % NDB - 1]);
          acc[i % NDB] = mfma_rows<F16>(ring[i % RING], hi, acc[i % NDB]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if constexpr (MASKED) {
      // Infinite and NaN values reach the rows that see them, and no others
      for (int w = 0; w < 2; ++w) {
        for (unsigned keys = __builtin_amdgcn_readfirstlane(sh.odd[turn][w]); keys; keys &= keys - 1) {
          const int key = 32 * w + __builtin_ctz(keys), at = key / 8 * 4 + key % 4, j = start + key;   // `at` of the half key / 4 % 2
          float p = 0.f;
#pragma unroll
          for (int e = 0; e < 32; ++e) p = e == at ? s[e / 16][e % 16] : p;
          if (!(seen >> at & 1)) p = -1.f;
          const float other = partner32(p);
          if (half != key / 4 % 2) p = other;
          if (p < 0.f) continue;
          p = fmaxf(p, 0x1p-126f);
          const int group = key / FM_KEY_GROUP;   // it has a page: without one the value is 0
          const int page = group == 0 ? page_of(tile, 0) : group == 1 ? page_of(tile, 1) : group == 2 ? page_of(tile, 2) : page_of(tile, 3);
          const char* row = v_head + page * a.v.page + (j - fm_div(j, a.page) * (int)a.page.n) * (long long)a.v.token;
#pragma unroll
          for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int d = 32 * db + 8 * (e / 4) + 4 * half + e % 4;
              float x;
              if constexpr (E4M3) x = (((const unsigned char*)row)[d] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.f;
              else if constexpr (F16) x = (float)((const _Float16*)row)[d];
              else x = (float)((const __bf16*)row)[d];
              if (!(fabsf(x) < INFINITY)) acc[db][e] += p * x;
            }
        }
      }
    }
  };

  const auto plant_tree = [&] {
    plant(sh.tree, a.parents + (size_t)b * a.T, a.T);
    if (threadIdx.x < 64) {   // every depth up to the largest occurs: a token's ancestors have the smaller ones
      int depth = 0;
      for (int u = lane; u < a.T; u += 64) depth = max(depth, sh.tree.depth[u]);
#pragma unroll
      for (int k = 1; k < 64; k *= 2) depth = max(depth, __shfl_xor(depth, k));
      if (lane == 0) sh.deepest = depth;
    }
    if (threadIdx.x < 6) sh.odd[threadIdx.x / 2][threadIdx.x % 2] = 0;
    barrier_nofence();
    row_i = first_row + sh.tree.depth[t];
    rows_end = first_row + __builtin_amdgcn_readfirstlane(sh.deepest) + 1;
  };
  // Tiles of a panel: the next one's copies are in flight while one is worked on.
  int buffer = 0, turn = 0;
  const auto run = [&](auto with_mask, int panel, unsigned long long tiles) {
    constexpr bool MASKED = decltype(with_mask)::value;
    int tile = __builtin_ctzll(tiles);
    tiles &= tiles - 1;
    load(buffer, panel, tile);
    store(buffer);
    barrier_nofence();
    while (true) {
      const int now = tile, start = panel + now * kTile;
      const bool more = tiles != 0;
      if (more) {
        tile = __builtin_ctzll(tiles);
        tiles &= tiles - 1;
        load(buffer ^ 1, panel, tile);
      }
      if constexpr (MASKED) {
        if (threadIdx.x < 2) sh.odd[turn == 0 ? 2 : turn - 1][threadIdx.x] = 0;   // of the tile before, for the one after the next
        if (a.bounds[0]) {
          load_bounds(start);
          if (threadIdx.x < kTile) sh.bound[threadIdx.x] = bound_raw;
        }
        clean(buffer, turn, start, now);
      }
      if (!idle) compute(with_mask, buffer, turn, start, now, [] {});
      buffer ^= 1;
      if (MASKED) turn = turn == 2 ? 0 : turn + 1;   // of masked tiles alone, so that each clears what the one before has noted
      if (more) store(buffer);
      barrier_nofence();
      if (!more) break;
    }
  };
  // The same of unmasked tiles of 16 bits, with a tile and a half ahead: keys are copied where the products with those before the last are done, values
  // where the tile before is done.  (All a tile ahead: 16 trees of 63 tokens 106 us, so 102.)
  const auto run_far = [&](int panel, unsigned long long tiles) {
    constexpr int COPIES = CopyLanes<D>::NINST;
    const auto take = [&] {
      const int tile = tiles ? __builtin_ctzll(tiles) : -1;
      tiles &= tiles - 1;
      return tile;
    };
    // what comes by ordinary loads is there before the first copy, so that no wait for it counts the copies
#pragma unroll
    for (int g = 0; g < kTile / FM_KEY_GROUP; ++g) settle(entry[g]);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) settle(q[s]);
    int now = take(), next = take();
    buffer = 0;
    copy_keys(0, panel, now);
    copy_values(0, panel, now);
    if (next >= 0) copy_keys(1, panel, next);
    while (now >= 0) {
      const int far = take();
      if (next >= 0) async_wait<2 * COPIES>();
      else async_wait<COPIES>();
      barrier_nofence();   // the keys are there, the values before have been read
      if (next >= 0) copy_values(buffer ^ 1, panel, next);
      const auto half_way = [&] {
        if (next >= 0) async_wait<2 * COPIES>();
        else async_wait<0>();
        barrier_nofence();   // the values are there, the keys have been read
        if (far >= 0) copy_keys(buffer, panel, far);
      };
      if (idle) half_way();
      else compute(std::false_type(), buffer, 0, panel + now * kTile, now, half_way);
      now = next;
      next = far;
      buffer ^= 1;
    }
    barrier_nofence();
  };
  if (a.bounds[0] || a.window > 0) plant_tree();
  for (int panel = begin; panel < end; panel += kPanelTiles * kTile) {
    const int panel_end = min(end, panel + kPanelTiles * kTile), tiles = (panel_end - panel + kTile - 1) / kTile;
    bool hole = false;
#pragma unroll
    for (int g = 0; g < kTile / FM_KEY_GROUP; ++g) {
      const int j = panel + lane * kTile + g * FM_KEY_GROUP;
      entry[g] = j < panel_end ? fm_known_page(a.table[(size_t)b * a.columns + fm_div(j, a.page)], a.num_pages) : -1;
      hole |= j < panel_end && entry[g] < 0;
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int group = group_of(i);
      mine[i] = group == 0 ? entry[0] : group == 1 ? entry[1] : group == 2 ? entry[2] : entry[3];
    }
    unsigned long long live, partly;
    if (a.bounds[0]) {
      for (int i = wave; i < tiles; i += kWaves) {
        const int j = panel + i * kTile + lane;
        int seen = 0;
        if (j < panel_end) {
          i32x4 bound = {0, 0, 0, 0};
          if (j < a.bound_columns) {
#pragma unroll
            for (int w = 0; w < 4; ++w) bound[w] = a.bounds[w][(size_t)b * a.bound_columns + j];
          }
          const int last = a.window > 0 ? (int)std::min<long long>(rows_end, (long long)j + a.window) : rows_end;
          seen = j >= first_row ? -1 : rows_left(first_row, last, bound);
        }
        const bool some = __any(seen != 0), all = __all(seen == rows_end - first_row);
        if (lane == 0) sh.flag[i] = some ? all ? 1 : 2 : 0;
      }
      barrier_nofence();
      const int flag = lane < tiles ? sh.flag[lane] : 0;
      live = __ballot(flag != 0);
      partly = __ballot(flag == 2 || hole);
      barrier_nofence();   // the flags have been read
    } else {
      const int start = panel + lane * kTile;
      live = __ballot(lane < tiles);
      partly = __ballot(hole || start + kTile > panel_end || start + kTile > first_row || (a.window > 0 && start <= rows_end - 1 - a.window));
    }
    if (live & ~partly) {
      if constexpr (E4M3) run(std::false_type(), panel, live & ~partly);
      else run_far(panel, live & ~partly);
    }
    if (live & partly) {
      if (!a.bounds[0] && a.window <= 0) plant_tree();
      run(std::true_type(), panel, live & partly);
    }
  }

  // Results: a lane has elements 32 db + 8 q + 4 half + 0..3 of its row
  const float total = l + partner32(l);
  if (chunk.of > 1) {
    // Rows of d floats to a wave's piece of LDS, 16-byte pieces of a row in an order that spreads them over the banks, and from there whole rows to memory
    constexpr int ROW_PIECES = D / 4;
    char* stage = (wave < 2 ? sh.k[wave] : sh.v[wave - 2]);
    static_assert(kWaveRows * D * 4 <= sizeof(sh.k[0]));
    if (!idle) {
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          *(f32x4*)(stage + (c * ROW_PIECES + ((8 * db + 2 * x + half) ^ c % ROW_PIECES)) * 16) =
              f32x4{acc[db][4 * x], acc[db][4 * x + 1], acc[db][4 * x + 2], acc[db][4 * x + 3]};
      const size_t at = ((size_t)(chunk.slot + chunk.number) * a.Hk + hk) * R;
      const int first = rb * kBlockRows + wave * kWaveRows;
#pragma unroll
      for (int i = 0; i < kWaveRows * ROW_PIECES / 64; ++i) {
        const int row = (i * 64 + lane) / ROW_PIECES, piece = lane % ROW_PIECES;
        const f32x4 x = *(const f32x4*)(stage + (row * ROW_PIECES + (piece ^ row % ROW_PIECES)) * 16);
        if (first + row < R) *(f32x4*)(a.part + (at + first + row) * D + 4 * piece) = x;
      }
      if (half == 0 && real) a.stat[at + r] = float2{m, total};
    }
  } else if (real) {
    const int h = hk * G + hq;
    const float factor = total == 0.f ? 0.f : (E4M3 ? a.v_scale[hk] : 1.f) / total;
    char* o = (char*)a.out + 2 * ((long long)b * a.so.b + (long long)h * a.so.h + (long long)t * a.so.n);
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *(u32x2*)(o + 2 * (32 * db + 8 * x + 4 * half)) = u32x2{pack2<F16>(acc[db][4 * x] * factor, acc[db][4 * x + 1] * factor),
                                                                pack2<F16>(acc[db][4 * x + 2] * factor, acc[db][4 * x + 3] * factor)};
    if (half == 0) a.lse[((size_t)b * a.H + h) * a.T + t] = total == 0.f ? -INFINITY : (m + fast_log2(total * kUnshift<F16>)) * kLn2;
  }
}

// Joins the chunks of split sequences where they are few and rows many (fm_tree_joins_by_lanes): D / 4 lanes to a row, four chunks at a time.
template <int D, bool F16>
__global__ __launch_bounds__(kThreads) void tree_join_kernel(FmTreeArgs a, FmDivisor rows, FmDivisor tokens) {
  constexpr int LANES = D / 4, BATCH = 4;
  const int G = a.H / a.Hk, R = G * a.T, b = blockIdx.y, lane = threadIdx.x % LANES, row = blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES;
  const int2 plan = a.plan[b];
  if (plan.y <= 1 || row >= a.Hk * R) return;
  const int hk = fm_div(row, rows), r = row - hk * R;
  const size_t first = ((size_t)plan.x * a.Hk + hk) * R + r, step = (size_t)a.Hk * R;
  float m = -INFINITY, l = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int base = 0; base < plan.y; base += BATCH) {
    f32x4 v[BATCH];
    float2 s[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const size_t at = first + std::min(base + i, plan.y - 1) * step;
      s[i] = a.stat[at];
      v[i] = *(const f32x4*)(a.part + at * D + 4 * lane);
      if (base + i >= plan.y) s[i] = float2{-INFINITY, 0.f};
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) top = fmaxf(top, s[i].x);
    const float alpha = fast_exp2(m - reference(top));
    m = top;
    l *= alpha;
    x *= alpha;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      if (base + i >= plan.y) continue;
      const float w = fast_exp2(s[i].x - reference(top));
      l += w * s[i].y;
      x += w * v[i];
    }
  }
  const int hq = fm_div(r, tokens), t = r - hq * a.T, h = hk * G + hq;
  const float factor = l == 0.f ? 0.f : (a.v_scale ? a.v_scale[hk] : 1.f) / l;
  char* o = (char*)a.out + 2 * ((long long)b * a.so.b + (long long)h * a.so.h + (long long)t * a.so.n + 4 * lane);
  *(u32x2*)o = u32x2{pack2<F16>(x[0] * factor, x[1] * factor), pack2<F16>(x[2] * factor, x[3] * factor)};
  if (lane == 0) a.lse[((size_t)b * a.H + h) * a.T + t] = l == 0.f ? -INFINITY : (m + fast_log2(l * kUnshift<F16>)) * kLn2;
}

template <int D, bool F16, bool E4M3>
static void launch(FmTreeArgs a, hipStream_t stream) {
  constexpr int kMost = 1 << 23;   // workgroups of a launch, which has fewer than 2^32 lanes
  const FmDecodeCut& cut = a.cut;
  const int units = a.plan ? fm_listed_units(cut.chunks, a.B) : (a.B + 7) / 8 * 8, workgroups = units * cut.workgroups;
  if (a.units) fm_launch_decode_list(a, FM_TREE_ROUND, stream);
  for (a.first_workgroup = 0; a.first_workgroup < workgroups; a.first_workgroup += kMost)
    hipLaunchKernelGGL((tree_kernel<D, F16, E4M3>), dim3((unsigned)std::min(workgroups - a.first_workgroup, kMost)), dim3(kThreads), 0, stream, a,
                       fm_divisor(cut.workgroups), fm_divisor(cut.row_blocks), fm_divisor(a.T), fm_divisor(cut.chunks));
  if (a.plan && !a.split && fm_tree_joins_by_lanes((long long)a.H * a.T, a.B, cut.chunks, cut.least, (long long)a.columns * a.page_tokens)) {
    const int R = a.H / a.Hk * a.T, each = kThreads / (D / 4);
    hipLaunchKernelGGL((tree_join_kernel<D, F16>), dim3((a.Hk * R + each - 1) / each, a.B), dim3(kThreads), 0, stream, a, fm_divisor(R), fm_divisor(a.T));
  } else if (a.plan) {
    fm_launch_decode_join(a, F16, stream);
  }
}

}  // namespace fm

FmDecodeCut fm_tree_cut(int H, int Hk, int T, int d, int B, int cus) {
  FmDecodeCut cut;
  const int R = H / Hk * T;
  cut.block_rows = fm::kBlockRows;
  cut.row_blocks = (R + fm::kBlockRows - 1) / fm::kBlockRows;
  cut.teams = 1;
  cut.workgroups = cut.row_blocks * Hk;
  // Chunks that give every compute unit its two workgroups once, for more sequences than that twice, as where few rows are (fm_decode_cut); two tiles
  // at least, and partial results in 96 MiB.
  const long long at_once = std::max(1, 2 * (cus > 0 ? cus : 256) / cut.workgroups), wanted = B <= at_once ? at_once : 2 * at_once;
  const long long room = (96ll << 20) / ((long long)Hk * R * (d + 2) * 4), most = room / 2 < B ? room / 2 : room - B;   // see fm_most_slots
  cut.chunks = (int)std::max<long long>(1, std::min({wanted, most, 256ll}));
  cut.least = 2 * FM_TREE_ROUND;
  cut.slots = fm_most_slots(cut.chunks, B);
  cut.listed = (B + 63) / 64 * (long long)B * cut.workgroups > 4 * 2ll * (cus > 0 ? cus : 256);
  return cut;
}

hipError_t fm_launch_tree_wide(const FmTreeArgs& a, bool f16, bool e4m3, hipStream_t stream) {
  if (a.d == 64) {
    if (f16) e4m3 ? fm::launch<64, true, true>(a, stream) : fm::launch<64, true, false>(a, stream);
    else e4m3 ? fm::launch<64, false, true>(a, stream) : fm::launch<64, false, false>(a, stream);
  } else {
    if (f16) e4m3 ? fm::launch<128, true, true>(a, stream) : fm::launch<128, true, false>(a, stream);
    else e4m3 ? fm::launch<128, false, true>(a, stream) : fm::launch<128, false, false>(a, stream);
  }
  return hipGetLastError();
}
