// Attention weight of keys: of a prompt's (flashmask_weights) and of a paged cache's (flashmask_cache_weights).
//
//     w[j] = sum over the query rows i that see j, of all query heads of the K/V head, of exp(scale * q_i k_j - lse_i)
//
// Scores as S = Q K^T with keys on lanes: a lane's results are rows of one key, which it adds up in registers; lanes meet once per key at the
// end.  exp(s - lse) is exp2(s * scale * log2 e - lse * log2 e), one multiply-add and one exponential.
#include <algorithm>

#include "fm_cache_math.h"
#include "fm_common.h"
#include "fm_serving.h"
#include "fm_tree.h"

namespace fm {

// What is added to a row's score: -lse in the log2 domain, and -inf for a row that gives nothing (lse = -inf), for no other.  Such a row's scores may be infinite
// or NaN, which the sum alone does not take away: it goes the way of rows that do not see a key.
__device__ __forceinline__ float minus_lse(float lse) {
  const float x = -lse * kLog2e;
  return lse == -INFINITY ? -INFINITY : x < -3.0e38f ? -3.0e38f : x;
}

// --- a prompt --------------------------------------------------------------------------------------------------
// A workgroup has 256 keys of a K/V head, a wave 64 of them, whose fragments stay in registers (B operands of 32x32x16 products); 64 query rows at
// a time come through LDS, copied two tiles ahead.  Row tiles of all query heads of the group, one behind
// the other, are cut into `parts`; Equation 4 tells for the workgroup's and for the wave's keys which are skipped and which
// take the element mask.
// An element costs its product, a multiply-add, an exponential (8 cycles of a wave) and an addition: 64 of them as many cycles as their 32 products.
// 16384 tokens with answers (32 heads on 8, d = 128): 890 us, with zeros for q and k 729: power.  The last 64 rows of 131072 tokens: 106 to 114 us, 56
// without the loop over the rows.  With 32 keys to a wave and three workgroups to a compute unit 983 and 124.
constexpr int kKeys = 256, kTile = 64, kPanel = 2048;   // kPanel: row tiles that are listed together

template <int D>
struct WeightsShared {
  alignas(16) char q[3][kTile * TileLayout<D>::RS];
  alignas(16) float lse[4][4][kTile];   // each wave's own; one more: a wave has use for the rows before
  int minmax[4][8];
  int list[kPanel], wave_count[4];   // row tiles that some key of the workgroup's sees: tile | class for wave w << (16 + 2 w)
};

// Maximum, minimum over the 32 lanes of a wave's half (all halves alike).
__device__ __forceinline__ int half_max(int x) {
  x = row16_max(x);
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return __builtin_amdgcn_readfirstlane(max((int)r[0], (int)r[1]));
}
__device__ __forceinline__ int half_min(int x) {
  x = row16_min(x);
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return __builtin_amdgcn_readfirstlane(min((int)r[0], (int)r[1]));
}

template <int D>
__global__ __launch_bounds__(256, 2) void weights_kernel(FmWeightsArgs a) {
  using L = TileLayout<D>;
  constexpr int STEPS = D / 16;
  __shared__ WeightsShared<D> sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, half = lane >> 5;
  // Slices go round: workgroup x runs on XCD x % 8, so that up to eight slices' query rows stay in few L2s.
  const int rest = fm_div(blockIdx.x, a.slices), slice = blockIdx.x - rest * (int)a.slices.n;
  const int block = fm_div(rest, a.by_part), part = rest - block * a.parts;
  const int b = fm_div(slice, a.by_head), hk = slice - b * a.Hk;
  const int key0 = block * kKeys + wave * 64, G = a.H / a.Hk;

  bf16x8 k[2][STEPS];
  i32x4 bound[2];
  const unsigned row_part = L::off(c, 16 * half);
  const char* k_rows = (const char*)a.k + 2 * ((long long)b * a.sk.b + (long long)hk * a.sk.h);
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int key = min(key0 + 32 * n + c, a.N - 1);   // a lane past the last key works on a copy of it
#pragma unroll
    for (int w = 0; w < 4; ++w) bound[n][w] = min(max(a.bounds[w][(size_t)b * a.N + key], 0), a.N);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) k[n][s] = __builtin_bit_cast(bf16x8, ldg16(k_rows + 2 * (key * a.sk.n + 16 * s + 8 * half)));
  }
  MinMax8 mine, all;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    mine.v[2 * w] = half_max(max(bound[0][w], bound[1][w]));
    mine.v[2 * w + 1] = half_min(min(bound[0][w], bound[1][w]));
  }
  if (lane == 0) {
#pragma unroll
    for (int w = 0; w < 8; ++w) sh.minmax[wave][w] = mine.v[w];
  }
  barrier_nofence();
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    int x = sh.minmax[0][w];
#pragma unroll
    for (int i = 1; i < 4; ++i) x = w % 2 ? min(x, sh.minmax[i][w]) : max(x, sh.minmax[i][w]);
    all.v[w] = x;
  }
  CopyLanes<D> lanes;
  lanes.init(lane, 2 * (int)a.sq.n);
  // To LDS, by each wave 16 rows, and every row's lse for itself; a tile's rows past the last are copies of it.
  constexpr int COPIES = CopyLanes<D>::NINST + 1;
  const int row_bytes = 2 * (int)a.sq.n;
  const auto load = [&](const char* rows, const float* lse, int tile, int last, int slot, int turn) {
    async_copy4(lse + min(tile * kTile + lane, last), lds_address(sh.lse[wave][turn]));
    if (tile * kTile + kTile - 1 <= last) {
      const char* source = CopyLanes<D>::wave_base(rows, wave, row_bytes) + (unsigned long long)(unsigned)tile * (unsigned)(kTile * row_bytes);
      tile_load_async<D>(source, lanes, sh.q[slot], wave);
    } else {
      tile_load_async_clamped<D>((const __bf16*)rows, tile * kTile, last + 1, sh.q[slot], wave, lane, row_bytes);
    }
  };

  const float scale = a.scale * kLog2e;
  float sum[2] = {0.f, 0.f};
  // Products of half m of a tile with the keys, and (OLD) beside them the exponentials of the 32 rows before: two elements (d = 64: four) to a
  // product, each a multiply-add, an exponential and, a product later each, an addition.
  // Sums of 32 rows first keep the error of long sums down.
  const auto scores = [&](auto with_old, int m, const char* rows, f32x16 (&s)[2], const f32x16 (&old)[2], const float* old_lse) {
    constexpr bool OLD = decltype(with_old)::value;
    constexpr int RING = 3, EACH = 16 / STEPS;   // elements to a product; element e: row e / 2 of the lane's 16, key e % 2
    bf16x8 ring[RING];
    f32x4 lse[4];
    float x[2][EACH], tile[2] = {0.f, 0.f};
    const auto fetch = [&](int step) { ring[step % RING] = *(const bf16x8*)(rows + L::add_col(row_part, 32 * step) + 32 * m * L::RS); };
    fetch(0);
    fetch(1);
    if constexpr (OLD) {
#pragma unroll
      for (int q = 0; q < 4; ++q) lse[q] = *(const f32x4*)(old_lse + 8 * q + 4 * half);
    }
    s[0] = s[1] = f32x16{};
#pragma unroll
    for (int i = 0; i < 2 * STEPS + 2; ++i) {
      if (i < 2 * STEPS) {
        if (i % 2 == 0 && i / 2 + 2 < STEPS) fetch(i / 2 + 2);
        s[i % 2] = mfma32(ring[i / 2 % RING], k[i % 2][i / 2], s[i % 2]);
      }
      if constexpr (OLD) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
          if (i > 1) {
            tile[e % 2] += x[i % 2][e];
            settle(tile[e % 2]);
          }
          if (i < 2 * STEPS) {
            const int at = i * EACH + e, row = at / 2;
            x[i % 2][e] = fmaf(old[at % 2][row], scale, lse[row / 4][row % 4]);
            settle(x[i % 2][e]);
          }
          if (i > 0 && i < 2 * STEPS + 1) {
            x[(i - 1) % 2][e] = fast_exp2(x[(i - 1) % 2][e]);
            settle(x[(i - 1) % 2][e]);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (OLD) {
      sum[0] += tile[0];
      sum[1] += tile[1];
    }
  };
  constexpr std::true_type with_old;
  constexpr std::false_type alone;
  // The same exponentials by themselves; hides(x, n, q) puts -inf where rows 8 q + 4 half + (0..3) do not see key n.
  const auto add = [&](const f32x16 (&s)[2], const float* lses, const auto& hides) {
    float tile[2] = {0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 lse = *(const f32x4*)(lses + 8 * q + 4 * half);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = fmaf(s[n][4 * q + r], scale, lse[r]);
        hides(x, n, q);
#pragma unroll
        for (int r = 0; r < 4; ++r) tile[n] += fast_exp2(x[r]);
      }
    }
    sum[0] += tile[0];
    sum[1] += tile[1];
  };
  const auto none = [](f32x4&, int, int) {};

  f32x16 upper[2], lower[2];   // scores of a tile's halves; those of `lower` wait for the next products
  const float* waiting = nullptr;   // their rows' lse
  int slot = 0, turn = 0;   // of the tile at hand
  for (int panel = 0; panel < a.row_tiles; panel += kPanel) {
    const int panel_row = a.first_row + panel * kTile, tiles = min(kPanel, a.row_tiles - panel);
    int listed = 0;
    barrier_nofence();   // the list before has been read
    for (int base = 0; base < tiles; base += 256) {
      const int tile = base + threadIdx.x, r0 = panel_row + tile * kTile, r1 = min(r0 + kTile, a.N);
      int entry = tile;
      bool live = false;
      if (tile < tiles && classify_tile(r0, r1, all) != T_FULLY) {
        live = true;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          MinMax8 x;
#pragma unroll
          for (int i = 0; i < 8; ++i) x.v[i] = sh.minmax[w][i];
          entry |= (classify_tile(r0, r1, x) & 3) << (16 + 2 * w);
        }
      }
      append_live(live, entry, sh.list, sh.wave_count, listed);
    }
    // this part's share of the heads' tiles
    const int items = G * listed, each = fm_div(items, a.by_part), more = items - each * a.parts;
    int left = each + (part < more);
    if (left == 0) continue;
    const int first = part * each + min(part, more);
    const int h = first / listed;
    int at = first - h * listed;
    const char* head_rows = (const char*)a.q + 2 * ((long long)b * a.sq.b + (long long)(hk * G + h) * a.sq.h + panel_row * a.sq.n);
    const float* head_lse = a.lse + ((size_t)b * a.H + hk * G + h) * a.N + panel_row;
    // What comes from outside asynchronous copies has to be there before the loop: a wait for it in there would be one for the copies, too.
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      settle(bound[n]);
#pragma unroll
      for (int s = 0; s < STEPS; ++s) settle(k[n][s]);
    }
    // Copies run two tiles ahead: ahead[0] is the tile at hand, ahead[1] the next.
    int ahead[2];
    const auto begin = [&](int entry, int far) {
      load(head_rows, head_lse, entry & 0xffff, a.N - 1 - panel_row, slot + far - (slot + far > 2 ? 3 : 0), (turn + far) & 3);
      if (++at == listed) {
        at = 0;
        head_rows += 2 * a.sq.h;
        head_lse += a.N;
      }
      return entry;
    };
    ahead[0] = begin(__builtin_amdgcn_readfirstlane(sh.list[at]), 0);
    ahead[1] = left > 1 ? begin(__builtin_amdgcn_readfirstlane(sh.list[at]), 1) : 0;
    int listed_next = sh.list[at];
    for (; left > 0; --left) {
      const char* rows = sh.q[slot];
      float* lses = sh.lse[wave][turn];
      if (left > 1) async_wait<COPIES>();
      else async_wait<0>();
      barrier_nofence();   // the tile is there, and the one before has been read
      const float mine = minus_lse(lses[lane]);
      lses[lane] = mine;
      const unsigned long long silent = __ballot(mine == -INFINITY);
      const int row = panel_row + (ahead[0] & 0xffff) * kTile, cls = ahead[0] >> (16 + 2 * wave) & 3;
      ahead[0] = ahead[1];
      if (left > 2) {
        ahead[1] = begin(__builtin_amdgcn_readfirstlane(listed_next), 2);
        listed_next = sh.list[at];
      }
      slot = slot == 2 ? 0 : slot + 1;
      turn = (turn + 1) & 3;

      if (cls == T_FULLY) {   // what waits does not wait longer than a tile
        if (waiting) add(lower, waiting, none);
        waiting = nullptr;
        continue;
      }
      if (waiting) scores(with_old, 0, rows, upper, lower, waiting);
      else scores(alone, 0, rows, upper, upper, lses);
      if (cls == T_UNMASKED && row + kTile <= a.N && !silent) {
        scores(with_old, 1, rows, lower, upper, lses);
        waiting = lses + 32;
        continue;
      }
      // The tile's rows that do not see a key are bits, spread over the elements with a bit-field extract each.  (With comparisons at every
      // element a masked tile takes 1000 instructions instead of 550.)
      unsigned hidden[2][2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const auto below = [&](int i) { return i - row >= 64 ? ~0ull : i <= row ? 0ull : (1ull << (i - row)) - 1; };
        const unsigned long long x =
            (below(bound[n][1]) & ~below(bound[n][0])) | (below(bound[n][3]) & ~below(bound[n][2])) | ~below(a.N) | silent;
        hidden[0][n] = (unsigned)x >> 4 * half;
        hidden[1][n] = (unsigned)(x >> 32) >> 4 * half;
      }
      const auto masked = [&](int m) {
        return [&, m](f32x4& x, int n, int q) {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            int hide = __builtin_amdgcn_sbfe(hidden[m][n], 8 * q + r, 1);
            settle(hide);   // no comparison
            x[r] = __int_as_float((__float_as_int(x[r]) & ~hide) | (hide & 0xff800000));
          }
        };
      };
      add(upper, lses, masked(0));
      scores(alone, 1, rows, lower, lower, lses);
      add(lower, lses + 32, masked(1));
      waiting = nullptr;
    }
    if (waiting) add(lower, waiting, none);
    waiting = nullptr;
  }
#pragma unroll
  for (int n = 0; n < 2; ++n) sum[n] += partner32(sum[n]);
  const int key = key0 + lane;
  if (key < a.N) a.part[((size_t)part * a.B * a.Hk + slice) * a.N + key] = half ? sum[1] : sum[0];
}

// Sums of the parts, in their order.
__global__ __launch_bounds__(256) void join_weights_kernel(const float* __restrict__ part, float* __restrict__ weights, size_t n, int parts) {
  for (size_t i = blockIdx.x * 256ull + threadIdx.x; i < n; i += 256ull * gridDim.x) {
    float x = part[i];
    for (int p = 1; p < parts; ++p) x += part[p * n + i];
    weights[i] = x;
  }
}

// --- a cache ---------------------------------------------------------------------------------------------------
// Keys in steps of 64 to a wave, four groups of 16 (B operands of 16x16x32 products: a lane has a key of each group); 16 query rows are the A operand,
// so that a lane's results are four rows of its keys.  A wave has the next step's keys in flight.  Of up to 16 rows to a K/V head the
// operand stays in registers and reading the keys is what takes the time; of more, 256 at a time lie in LDS.
// Chunks of keys are dealt as in attention over the cache: all sequences' keys in as many pieces as the chip has places, each sequence in whole ones.
// 64 ragged sequences of up to 8192 keys of 128 elements, one new token: 82 us, 4.6 TB/s, of 8 bits 40 us, 4.8; of 64 elements 36 us, 5.3, and 26 us, 3.9 (4 KiB
// of a wave in flight); 32 new tokens of four sequences, 256 rows to a K/V head, 8 bits: 20 us.
// With bounds every lane first works out for its own key how many of the T rows see it: steps that none sees are not read, and only steps with keys that
// some rows do not see take the element mask.
constexpr int kStep = 64, kGroups = kStep / FM_KEY_GROUP, kWaves = 4, kSteps = 64, kRows = 256;   // kSteps: of a panel, whose flags lie together

template <int D, bool ONE>
struct CacheWeightsShared {
  int flag[kSteps];
  alignas(16) char q[ONE ? 16 : kRows * TileLayout<D>::RS];
  alignas(16) float lse[ONE ? 4 : kRows];
  float part[ONE ? 1 : kWaves][ONE ? 1 : kStep];   // sums of waves that share a step
  alignas(4) unsigned char token[ONE ? 4 : kRows];   // which of the T a row is
};

// ONE: the rows of a K/V head are 16 at most.
template <int D, bool F16, bool E4M3, bool ONE>
__global__ __launch_bounds__(64 * kWaves, 2) void cache_weights_kernel(FmCacheWeightsArgs a) {
  using L = TileLayout<D>;
  constexpr int BYTES = E4M3 ? 1 : 2, STEPS = D / 32, LOADS = D * BYTES / 64;
  __shared__ CacheWeightsShared<D, ONE> sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, c = lane & 15;
  // all heads of a chunk on one XCD: they share table entries and bounds, and cache lines where heads lie side by side
  const int turn = fm_div(blockIdx.x >> 3, a.by_head), hk = (blockIdx.x >> 3) - turn * a.Hk, unit = turn * 8 + (blockIdx.x & 7);
  int b, len, begin, end;
  if (a.dealt) {
    const auto groups_of = [&](int n) { return (min(max(n, 0), a.places) + FM_KEY_GROUP - 1) / FM_KEY_GROUP; };
    Chunk chunk;
    constexpr int least = ONE ? kWaves * kGroups : kGroups;
    if (!find_chunk<false>(a.lens, a.B, a.chunks, least, least, unit, groups_of, chunk)) return;
    b = chunk.b;
    len = chunk.len;
    const int keys = fm_even_chunk(groups_of(len), chunk.of, kGroups) * FM_KEY_GROUP;
    begin = chunk.number * keys;
    end = begin + keys;
  } else {
    b = fm_div(unit, a.chunks);
    if (b >= a.B) return;
    len = a.lens[b];
    begin = (unit - b * (int)a.chunks.n) * a.chunk_keys;
    end = begin + a.chunk_keys;
  }
  len = max(len, 0);
  end = min(end, min(len, a.places));
  if (begin >= end) return;
  const int first_row = len - a.T;
  const FM_CONSTANT int* table = (const FM_CONSTANT int*)(a.table + (size_t)b * a.columns);
  const size_t row_of_weights = ((size_t)b * a.Hk + hk) * a.weight_columns;
  const auto old = [&](int j) { return a.before && j < first_row ? a.decay * a.before[row_of_weights + j] : 0.f; };
  const auto bound_of = [&](int j) {
    i32x4 x = {0, 0, 0, 0};
    if (j < a.bound_columns) {
#pragma unroll
      for (int w = 0; w < 4; ++w) x[w] = a.bounds[w][(size_t)b * a.bound_columns + j];
    }
    return x;
  };
  const auto rows_end = [&](int j) { return a.window > 0 ? (int)std::min<long long>(len, (long long)j + a.window) : len; };   // behind the last that sees j

  // Queries: rows hq * T + t of the K/V head, 16 at a time; rows past the last are copies that give nothing
  const int G = a.H / a.Hk, R = G * a.T;
  const auto query = [&](int r) {
    const int hq = fm_div(r, a.tokens);
    return (const char*)a.q + 2 * ((long long)b * a.sq.b + (long long)(hk * G + hq) * a.sq.h + (long long)(r - hq * a.T) * a.sq.n);
  };
  const auto lse_of = [&](int r) { return r < R ? minus_lse(a.lse[((size_t)b * a.H + hk * G) * a.T + r]) : -INFINITY; };   // [b, head, t] is contiguous
  // Which of the T a row is; of one past the last, what the last one is.
  const auto token_of = [&](int r) {
    const int at = min(r, R - 1);
    return at - fm_div(at, a.tokens) * a.T;
  };
  u32x4 q[STEPS];
  f32x4 lse;
  int silent = 0;   // some of the rows at hand have lse = -inf (known to be the same in all lanes)
  if constexpr (ONE) {
    const char* p = query(min(c, R - 1));
    bool some = false;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) q[s] = ldg16(p + 2 * (E4M3 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g));
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      lse[r] = lse_of(4 * g + r);
      some |= 4 * g + r < R && lse[r] == -INFINITY;
    }
    silent = __builtin_amdgcn_readfirstlane(__any(some));
  }

  const char* k_head = a.k.base + (long long)hk * a.k.head;
  u32x4 kraw[kGroups][LOADS];
  unsigned there = 0;   // groups that have a page, of the step that was loaded last
  const auto load_keys = [&](int start) {
    there = 0;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const int j = start + i * FM_KEY_GROUP, at = j < end ? j : start, column = fm_div(at, a.page);
      const int page = j < end ? fm_known_page(table[column], a.num_pages) : -1;
      const char* base = k_head + std::max(page, 0) * a.k.page + (unsigned)(at - column * (int)a.page.n) * (unsigned long long)a.k.token;
      there |= (page >= 0 ? 1u : 0u) << i;
      // a descriptor of no bytes where there is no page: such loads give 0 and touch no memory
      const auto rows = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, __builtin_amdgcn_readfirstlane(page < 0 ? 0 : -1), 0x00020000);
#pragma unroll
      for (int s = 0; s < LOADS; ++s)
        kraw[i][s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, c * a.k.token + 16 * g + 64 * s, 0, 0));
    }
  };
  const float scale = a.scale * kLog2e * (E4M3 ? a.k_scale[hk] : 1.f);

  for (int row0 = 0; row0 < R; row0 += ONE ? 16 : kRows) {
    const int blocks = ONE ? 1 : (min(R - row0, kRows) + 15) / 16;
    if constexpr (!ONE) {
      constexpr int PIECES = D / 8;
      __syncthreads();   // the rows before have been read
      for (int i = threadIdx.x; i < blocks * 16 * PIECES; i += 64 * kWaves) {
        const int r = i / PIECES, to = i % PIECES;
        // e4m3: which elements of d a product takes together follows the order of the keys' bytes
        const int from = E4M3 ? 8 * (to / 8) + 2 * (to % 4) + to / 4 % 2 : to;
        *(u32x4*)(sh.q + L::off(r, 16 * to)) = ldg16(query(min(row0 + r, R - 1)) + 16 * from);
      }
      if ((int)threadIdx.x < blocks * 16) {
        sh.lse[threadIdx.x] = lse_of(row0 + threadIdx.x);
        sh.token[threadIdx.x] = (unsigned char)token_of(row0 + threadIdx.x);
      }
      __syncthreads();
      const f32x4 four = *(const f32x4*)&sh.lse[4 * lane];
      bool some = false;
#pragma unroll
      for (int r = 0; r < 4; ++r) some |= 4 * lane + r < min(R - row0, kRows) && four[r] == -INFINITY;
      silent = __builtin_amdgcn_readfirstlane(__any(some));
    }
    for (int panel = begin; panel < end; panel += kSteps * kStep) {
      const int panel_end = min(end, panel + kSteps * kStep), steps = (panel_end - panel + kStep - 1) / kStep;
      unsigned long long left, partly;
      if (a.bound_columns) {
        __syncthreads();   // the flags before have been read
        for (int s = wave; s < steps; s += kWaves) {
          const int j = panel + s * kStep + lane;
          const int seen = j < panel_end ? rows_left(max(first_row, j), rows_end(j), bound_of(j)) : 0;
          const bool some = __any(seen > 0), all = __all(seen == a.T);
          if (lane == 0) sh.flag[s] = some ? all ? 1 : 2 : 0;
        }
        __syncthreads();
        const int flag = lane < steps ? sh.flag[lane] : 0;
        left = __ballot(flag != 0);
        partly = __ballot(flag == 2);
      } else {
        const int start = panel + lane * kStep, first = a.window > 0 ? first_row - a.window + 1 : 0;
        left = __ballot(lane < steps && start + kStep > first);
        partly = __ballot(start + kStep > panel_end || start + kStep - 1 > first_row || (a.window > 0 && start <= len - 1 - a.window));
      }
      // what no row sees has its old weight alone
      if (row0 == 0)
        for (unsigned long long none = ~left & (steps < 64 ? (1ull << steps) - 1ull : ~0ull); none; none &= none - 1) {
          const int s = __builtin_ctzll(none), j = panel + s * kStep + lane;
          if (s % kWaves == wave && j < panel_end) a.weights[row_of_weights + j] = old(j);
        }
      // The wave takes every fourth of the others; where they are one or two, waves share one, each with some of the rows (32 new tokens of one
      // sequence of 2000 keys 12.8 -> 9.5 us).
      const int live = __popcll(left), share = ONE || live > 2 ? 1 : live == 2 ? 2 : 4, sharer = wave % share;
      for (int i = 0; i < wave / share; ++i) left &= left - 1;
      if (!left) continue;
      int step = __builtin_ctzll(left);
      load_keys(panel + step * kStep);
      while (left) {
        const int start = panel + step * kStep, j = start + lane;
        const unsigned pages = there;
        const bool masked = (partly >> step & 1) || pages != (1u << kGroups) - 1u || silent;
        u32x4 keys[kGroups][STEPS];
#pragma unroll
        for (int i = 0; i < kGroups; ++i)
#pragma unroll
          for (int s = 0; s < STEPS; ++s) {
            if constexpr (E4M3) {
              const u32x4 raw = kraw[i][s / 2];
              const u32x2 x = widen4<F16>(raw[s % 2 * 2]), y = widen4<F16>(raw[s % 2 * 2 + 1]);
              keys[i][s] = u32x4{x[0], x[1], y[0], y[1]};
            } else {
              keys[i][s] = kraw[i][s];
            }
          }
        const float before = j >= panel_end ? 0.f : row0 == 0 ? old(j) : a.weights[row_of_weights + j];
        for (int i = 0; i < kWaves / share; ++i) left &= left - 1;
        if (left) {
          step = __builtin_ctzll(left);
          load_keys(panel + step * kStep);
        }
        float sum[kGroups] = {};
        const auto block = [&](const u32x4 (&q)[STEPS], const f32x4& lse, const int (&token)[4], const auto& mask) {
          f32x4 score[kGroups];
#pragma unroll
          for (int i = 0; i < kGroups; ++i) score[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int i = 0; i < kGroups; ++i) score[i] = mfma_keys<F16>(q[s], keys[i][s], score[i]);
#pragma unroll
          for (int i = 0; i < kGroups; ++i) {
            f32x4 x;
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = fmaf(score[i][r], scale, lse[r]);
            mask(x, i, token, lse);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = fast_exp2(x[r]);
            sum[i] += (x[0] + x[1]) + (x[2] + x[3]);
          }
        };
        const auto all_blocks = [&](const auto& mask) {
          if constexpr (ONE) {
            block(q, lse, {token_of(4 * g), token_of(4 * g + 1), token_of(4 * g + 2), token_of(4 * g + 3)}, mask);
          } else {
            for (int n = blocks * sharer / share; n < blocks * (sharer + 1) / share; ++n) {
              u32x4 rows[STEPS];
#pragma unroll
              for (int s = 0; s < STEPS; ++s) rows[s] = *(const u32x4*)(sh.q + L::off(c, 16 * g) + n * 16 * L::RS + s * 1024);
              const unsigned token = *(const unsigned*)&sh.token[n * 16 + 4 * g];
              const f32x4 lse = *(const f32x4*)&sh.lse[n * 16 + 4 * g];   // a copy: what is read in place is read again behind every settle
              block(rows, lse, {(int)(token & 255), (int)(token >> 8 & 255), (int)(token >> 16 & 255), (int)(token >> 24)}, mask);
            }
          }
        };
        if (masked) {
          i32x4 bound[kGroups];
          int key[kGroups], behind[kGroups];   // rows from key on and before `behind` see it, bounds apart
#pragma unroll
          for (int i = 0; i < kGroups; ++i) {
            const int at = start + i * FM_KEY_GROUP + c;
            const bool real = at < panel_end && (pages >> i & 1);
            bound[i] = a.bound_columns ? bound_of(at) : i32x4{0, 0, 0, 0};
            key[i] = at;
            behind[i] = real ? rows_end(at) : 0;
          }
          if (ONE || a.T <= 64) {
            // The tokens that see a key are bits, one extracted for each element, of a row with lse = -inf none.  (With comparisons at every element 16
            // rows of a masked step take 320 instructions instead of 150, the last rows of four prompts 29 us instead of 20.)
            unsigned seen[kGroups][2];
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
              const auto below = [&](int row) {
                const int n = min(max(row, 0), len) - first_row;   // T at most: no row is behind the sequence
                return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
              };
              const unsigned long long x = below(behind[i]) & ~(below(key[i]) | (below(bound[i][1]) & ~below(bound[i][0])) |
                                                                (below(bound[i][3]) & ~below(bound[i][2])));
              seen[i][0] = (unsigned)x;
              seen[i][1] = (unsigned)(x >> 32);
            }
            all_blocks([&](f32x4& x, int i, const int (&token)[4], const f32x4& lse) {
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                int sees = __builtin_amdgcn_sbfe(ONE || token[r] < 32 ? seen[i][0] : seen[i][1], token[r] & 31, lse[r] == -INFINITY ? 0 : 1);
                settle(sees);   // no comparison
                x[r] = __int_as_float((__float_as_int(x[r]) & sees) | (~sees & 0xff800000));
              }
            });
          } else if constexpr (!ONE) {
            all_blocks([&](f32x4& x, int i, const int (&token)[4], const f32x4& lse) {
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const int row = lse[r] == -INFINITY ? -1 : first_row + token[r];
                const bool gone = (row < key[i]) | (row >= behind[i]) | ((bound[i][0] <= row) & (row < bound[i][1])) | ((bound[i][2] <= row) & (row < bound[i][3]));
                x[r] = gone ? -INFINITY : x[r];
              }
            });
          }
        } else {
          all_blocks([](f32x4&, int, const int (&)[4], const f32x4&) {});
        }
        float mine = 0.f;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
          const float x = quad_sum(sum[i]);
          if (i == g) mine = x;
        }
        if constexpr (!ONE) {
          if (share > 1) {   // all waves come here, once in a panel
            __syncthreads();   // the sums of the panel before have been read
            sh.part[wave][lane] = mine;
            __syncthreads();
            if (sharer != 0) break;
            for (int p = 1; p < share; ++p) mine += sh.part[wave + p][lane];
          }
        }
        if (j < panel_end) a.weights[row_of_weights + j] = before + mine;
      }
    }
  }
}

template <int D, bool F16, bool E4M3>
static void launch(const FmCacheWeightsArgs& a, unsigned workgroups, hipStream_t stream) {
  if (a.H / a.Hk * a.T <= 16) hipLaunchKernelGGL((cache_weights_kernel<D, F16, E4M3, true>), dim3(workgroups), dim3(64 * kWaves), 0, stream, a);
  else hipLaunchKernelGGL((cache_weights_kernel<D, F16, E4M3, false>), dim3(workgroups), dim3(64 * kWaves), 0, stream, a);
}

}  // namespace fm

FmWeightsCut fm_weights_cut(int B, int H, int Hk, int N, int first_row, int cus) {
  FmWeightsCut cut;
  cut.row_tiles = (N - first_row + fm::kTile - 1) / fm::kTile;
  cut.key_blocks = (N + fm::kKeys - 1) / fm::kKeys;
  // Eight rounds of the places that the chip has, with parts of 16 tiles at least; where that leaves places empty, parts of 2 tiles.
  const long long units = (long long)B * Hk * cut.key_blocks, places = 2ll * (cus > 0 ? cus : 256), all = (long long)H / Hk * cut.row_tiles;
  const long long rounds = std::min((8 * places + units - 1) / units, all / 16), once = std::min((places + units - 1) / units, (all + 1) / 2);
  cut.parts = (int)std::max({rounds, once, 1ll});
  return cut;
}

hipError_t fm_launch_weights(FmWeightsArgs a, float* weights, const FmWeightsCut& cut, hipStream_t stream) {
  a.row_tiles = cut.row_tiles;
  a.parts = cut.parts;
  a.slices = fm_divisor(a.B * a.Hk);
  a.by_part = fm_divisor(cut.parts);
  a.by_head = fm_divisor(a.Hk);
  float* parts = a.part;
  if (cut.parts == 1) a.part = weights;
  const unsigned workgroups = (unsigned)a.B * a.Hk * cut.key_blocks * cut.parts;
  if (a.d == 64) hipLaunchKernelGGL(fm::weights_kernel<64>, dim3(workgroups), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(fm::weights_kernel<128>, dim3(workgroups), dim3(256), 0, stream, a);
  if (cut.parts > 1) {
    const size_t n = (size_t)a.B * a.Hk * a.N;
    hipLaunchKernelGGL(fm::join_weights_kernel, dim3((unsigned)std::min<size_t>((n + 255) / 256, 4096)), dim3(256), 0, stream, parts, weights, n, cut.parts);
  }
  return hipGetLastError();
}

bool fm_cut_cache_weights(FmCacheWeightsArgs& a, int cus) {
  // Every workgroup goes over all lengths, 64 at a time and about 1 us each; more sequences fill the chip by themselves.
  a.dealt = a.B <= 512;
  a.chunk_keys = std::min(a.places, 8192);
  // Up to 16 rows: four rounds of the two workgroups that a compute unit holds: there is nothing to join, and 64 ragged sequences take 82 us, with one,
  // two, three and eight rounds 90, 87, 83 and 85.  More rows, which every workgroup lays into LDS: one round of three.  One, two, three, four, eight
  // workgroups to a compute unit: 32 new tokens of four sequences, 8 heads to a K/V head, ragged caches of 20000 8-bit keys 23.6 21.8 19.2 21.0 23.1 us, of
  // one sequence 15.5 13.2 12.8 12.7 16.4; 63 of 16 ragged sequences of 8192 keys, 4 heads, from two on 66 63 72 76.
  const int workgroups = (a.H / a.Hk * a.T > 16 ? 3 : 8) * (cus > 0 ? cus : 256);
  a.chunks = fm_divisor(a.dealt ? std::max(1, workgroups / a.Hk) : (a.places + a.chunk_keys - 1) / a.chunk_keys);
  const long long units = a.dealt ? fm_most_units((int)a.chunks.n, a.B) : (long long)a.B * a.chunks.n;
  return (units + 8) * a.Hk < 1 << 24;   // a launch has fewer than 2^32 lanes
}

hipError_t fm_launch_cache_weights(const FmCacheWeightsArgs& a, bool f16, bool e4m3, hipStream_t stream) {
  const long long units = a.dealt ? fm_most_units((int)a.chunks.n, a.B) : (long long)a.B * a.chunks.n;
  const unsigned workgroups = (unsigned)((units + 7) / 8 * 8 * a.Hk);
  if (a.d == 64) {
    if (f16) e4m3 ? fm::launch<64, true, true>(a, workgroups, stream) : fm::launch<64, true, false>(a, workgroups, stream);
    else e4m3 ? fm::launch<64, false, true>(a, workgroups, stream) : fm::launch<64, false, false>(a, workgroups, stream);
  } else {
    if (f16) e4m3 ? fm::launch<128, true, true>(a, workgroups, stream) : fm::launch<128, true, false>(a, workgroups, stream);
    else e4m3 ? fm::launch<128, false, true>(a, workgroups, stream) : fm::launch<128, false, false>(a, workgroups, stream);
  }
  return hipGetLastError();
}
