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

namespace fm {

// What is added to a row's score: -lse in the log2 domain.  A row that sees nothing (lse = -inf) gives nothing.
__device__ __forceinline__ float minus_lse(float lse) { return lse == -INFINITY ? -INFINITY : -lse * kLog2e; }

// --- a prompt --------------------------------------------------------------------------------------------------
// A workgroup has 256 keys of a K/V head, a wave 64 of them, whose fragments stay in registers (B operands of 32x32x16 products); 64 query rows at
// a time come through LDS, two buffers, their loads in flight over the tile before.  Row tiles of all query heads of the group, one behind
// the other, are cut into `parts`; Equation 4 tells for the workgroup's and for the wave's keys which are skipped and which
// take the element mask.
constexpr int kKeys = 256, kTile = 64, kPanel = 2048;   // kPanel: row tiles that are listed together

template <int D>
struct WeightsShared {
  alignas(16) char q[2][kTile * TileLayout<D>::RS];
  alignas(16) float lse[3][kTile];   // one more: a wave may still be at the rows before the last
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
  constexpr int STEPS = D / 16, PIECES = D / 8, LOADS = kTile * PIECES / 256;
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
    for (int w = 0; w < 4; ++w) bound[n][w] = a.bounds[w][(size_t)b * a.N + key];
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
  u32x4 staged[LOADS];
  float staged_lse = 0.f;
  const auto load = [&](int h, int first) {
    const char* rows = (const char*)a.q + 2 * ((long long)b * a.sq.b + (long long)(hk * G + h) * a.sq.h);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int piece = i * 256 + threadIdx.x, row = min(first + piece / PIECES, a.N - 1);
      staged[i] = ldg16(rows + 2 * ((long long)row * a.sq.n + piece % PIECES * 8));
    }
    if (threadIdx.x < kTile) staged_lse = a.lse[((size_t)b * a.H + hk * G + h) * a.N + min(first + (int)threadIdx.x, a.N - 1)];
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
          if (i > 1) tile[e % 2] += x[i % 2][e];
          if (i < 2 * STEPS) {
            const int at = i * EACH + e, row = at / 2;
            x[i % 2][e] = fmaf(old[at % 2][row], scale, lse[row / 4][row % 4]);
          }
          if (i > 0 && i < 2 * STEPS + 1) x[(i - 1) % 2][e] = fast_exp2(x[(i - 1) % 2][e]);
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
  // The same exponentials by themselves; hides(n, r): rows r that do not see key n.
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
        hides(x, n, 8 * q + 4 * half);
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
  int buffer = 0, turn = 0;
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
    const long long items = (long long)G * listed;
    int left = (int)(items * (part + 1) / a.parts - items * part / a.parts);
    if (left == 0) continue;
    const long long first = items * part / a.parts;
    int h = (int)(first / listed), at = (int)(first - (long long)h * listed);
    int entry = __builtin_amdgcn_readfirstlane(sh.list[at]);
    load(h, panel_row + (entry & 0xffff) * kTile);
    for (; left > 0; --left) {
      const char* rows = sh.q[buffer];
      float* lses = sh.lse[turn];
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int piece = i * 256 + threadIdx.x;
        *(u32x4*)(sh.q[buffer] + L::off(piece / PIECES, piece % PIECES * 16)) = staged[i];
      }
      if (threadIdx.x < kTile) lses[threadIdx.x] = minus_lse(staged_lse);
      const int row = panel_row + (entry & 0xffff) * kTile, cls = entry >> (16 + 2 * wave) & 3;
      if (left > 1) {
        if (++at == listed) {
          at = 0;
          ++h;
        }
        entry = __builtin_amdgcn_readfirstlane(sh.list[at]);
        load(h, panel_row + (entry & 0xffff) * kTile);
      }
      buffer ^= 1;
      turn = turn == 2 ? 0 : turn + 1;
      barrier_nofence();   // the next tile's loads stay in flight

      if (cls == T_FULLY) {   // what waits does not wait longer than a tile
        if (waiting) add(lower, waiting, none);
        waiting = nullptr;
        continue;
      }
      if (waiting) scores(with_old, 0, rows, upper, lower, waiting);
      else scores(alone, 0, rows, upper, upper, lses);
      if (cls == T_UNMASKED && row + kTile <= a.N) {
        scores(with_old, 1, rows, lower, upper, lses);
        waiting = lses + 32;
        continue;
      }
      const auto masked = [&](int m) {
        return [&, m](f32x4& x, int n, int r0) {
          hide4(x, 0, [&](int r) {
            const int i = row + 32 * m + r0 + r;
            return (i >= a.N) | ((bound[n][0] <= i) & (i < bound[n][1])) | ((bound[n][2] <= i) & (i < bound[n][3]));
          });
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
// so that a lane's results are four rows of its keys.  A workgroup has a chunk of a sequence's keys of one K/V head.  First every lane works
// out for its own key how many of the T rows see it: steps that none sees are not read, and only steps of keys that some
// rows do not see take the element mask.
constexpr int kStep = 64, kGroups = kStep / FM_KEY_GROUP, kWaves = 4;

// Rows of [lo, hi) that an interval pair leaves.
__device__ __forceinline__ int rows_left(int lo, int hi, const i32x4& bound) {
  if (lo >= hi) return 0;
  const int a0 = max(bound[0], lo), b0 = min(bound[1], hi), a1 = max(bound[2], lo), b1 = min(bound[3], hi);
  return hi - lo - max(b0 - a0, 0) - max(b1 - a1, 0) + max(min(b0, b1) - max(a0, a1), 0);
}

// ONE: the rows of a K/V head are 16 at most and stay in registers.
template <int D, bool F16, bool E4M3, bool ONE>
__global__ __launch_bounds__(64 * kWaves, 2) void cache_weights_kernel(FmCacheWeightsArgs a) {
  constexpr int BYTES = E4M3 ? 1 : 2, STEPS = D / 32, LOADS = D * BYTES / 64;
  __shared__ int flags[FM_WEIGHTS_CHUNK / kStep];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, c = lane & 15;
  // all heads of a chunk on one XCD: they share table entries and bounds, and cache lines where heads lie side by side
  const int turn = fm_div(blockIdx.x >> 3, a.by_head), hk = (blockIdx.x >> 3) - turn * a.Hk, unit = turn * 8 + (blockIdx.x & 7);
  const int b = fm_div(unit, a.chunks), chunk = unit - b * (int)a.chunks.n;
  if (b >= a.B) return;
  const int len = max(a.lens[b], 0), end = min(len, a.places), j0 = chunk * FM_WEIGHTS_CHUNK, j1 = min(j0 + FM_WEIGHTS_CHUNK, end);
  if (j0 >= j1) return;
  const int first_row = len - a.T, steps = (j1 - j0 + kStep - 1) / kStep;
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
  const auto last_row = [&](int j) { return a.window > 0 ? (int)std::min<long long>(len, (long long)j + a.window) : len; };   // that sees j, and one

  for (int s = wave; s < steps; s += kWaves) {
    const int j = j0 + s * kStep + lane;
    int seen = 0;
    if (j < j1 && fm_known_page(a.table[(size_t)b * a.columns + fm_div(j, a.page)], a.num_pages) >= 0)
      seen = rows_left(max(first_row, j), last_row(j), a.bound_columns ? bound_of(j) : i32x4{0, 0, 0, 0});
    const bool some = __any(seen > 0), all = __all(seen == a.T);
    if (lane == 0) flags[s] = some ? all ? 1 : 2 : 0;
    if (!some && j < j1) a.weights[row_of_weights + j] = old(j);
  }
  __syncthreads();
  const int flag = lane < steps ? flags[lane] : 0;
  unsigned long long left = __ballot(flag != 0);
  const unsigned long long partly = __ballot(flag == 2);
  const auto skip = [&](int n) {
    for (int i = 0; i < n; ++i) left &= left - 1;
  };
  skip(wave);
  if (!left) return;

  // Queries: rows hq * T + t of the K/V head, 16 at a time; rows past the last are copies that give nothing
  const int G = a.H / a.Hk, R = G * a.T, blocks = ONE ? 1 : (R + 15) / 16;
  const auto load_rows = [&](int block, u32x4 (&q)[STEPS], f32x4& lse) {
    const int r = min(block * 16 + c, R - 1), hq = fm_div(r, a.tokens);
    const char* p = (const char*)a.q + 2 * ((long long)b * a.sq.b + (long long)(hk * G + hq) * a.sq.h + (long long)(r - hq * a.T) * a.sq.n);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) q[s] = ldg16(p + 2 * (E4M3 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = block * 16 + 4 * g + i;   // [b, head, t] is contiguous
      lse[i] = a.lse[((size_t)b * a.H + hk * G) * a.T + min(at, R - 1)];
      if (at >= R) lse[i] = -INFINITY;
    }
  };
  u32x4 q[STEPS];
  f32x4 lse;
  load_rows(0, q, lse);

  const char* k_head = a.k.base + (long long)hk * a.k.head;
  u32x4 kraw[kGroups][LOADS];
  const auto load_keys = [&](int step) {
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const int j = j0 + step * kStep + i * FM_KEY_GROUP, at = min(j, j1 - 1), column = fm_div(at, a.page), slot = at - column * (int)a.page.n;
      const int page = j < j1 ? fm_known_page(table[column], a.num_pages) : -1;
      // slot: of the group's first key, a multiple of 16
      const char* base = k_head + std::max(page, 0) * a.k.page + (unsigned)(slot & ~(FM_KEY_GROUP - 1)) * (unsigned long long)a.k.token;
      // a descriptor of no bytes where there is no page: such loads give 0 and touch no memory
      const auto rows = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, __builtin_amdgcn_readfirstlane(page < 0 ? 0 : -1), 0x00020000);
#pragma unroll
      for (int s = 0; s < LOADS; ++s)
        kraw[i][s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, c * a.k.token + 16 * g + 64 * s, 0, 0));
    }
  };
  const float scale = a.scale * kLog2e * (E4M3 ? a.k_scale[hk] : 1.f);

  int step = __builtin_ctzll(left);
  load_keys(step);
  while (left) {
    const bool masked = partly >> step & 1;
    const int start = j0 + step * kStep;
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
    const int j = start + lane;
    const float before = j < j1 ? old(j) : 0.f;
    skip(kWaves);
    if (left) {
      step = __builtin_ctzll(left);
      load_keys(step);
    }
    i32x4 bound[kGroups];
    bool there[kGroups];
    if (masked) {
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const int key = start + i * FM_KEY_GROUP + c;
        bound[i] = a.bound_columns ? bound_of(key) : i32x4{0, 0, 0, 0};
        there[i] = key < j1 && fm_known_page(a.table[(size_t)b * a.columns + fm_div(min(key, j1 - 1), a.page)], a.num_pages) >= 0;
      }
    }
    float sum[kGroups] = {};
    for (int block = 0; block < blocks; ++block) {
      if constexpr (!ONE) load_rows(block, q, lse);
      f32x4 score[kGroups];
#pragma unroll
      for (int i = 0; i < kGroups; ++i) score[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int i = 0; i < kGroups; ++i) score[i] = mfma_keys<F16>(q[s], keys[i][s], score[i]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float minus = minus_lse(lse[r]);
        int row = 0;
        if (masked) {
          const int at = min(block * 16 + 4 * g + r, R - 1);
          row = first_row + at - fm_div(at, a.tokens) * a.T;
        }
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
          float x = fmaf(score[i][r], scale, minus);
          if (masked) {
            const int key = start + i * FM_KEY_GROUP + c;
            const bool sees = there[i] && key <= row && row < last_row(key) && !hides(bound[i], row);
            if (!sees) x = -INFINITY;
          }
          sum[i] += fast_exp2(x);
        }
      }
    }
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const float x = quad_sum(sum[i]);
      if (i == g) mine = x;
    }
    if (j < j1) a.weights[row_of_weights + j] = before + mine;
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

hipError_t fm_launch_cache_weights(const FmCacheWeightsArgs& a, bool f16, bool e4m3, hipStream_t stream) {
  const unsigned workgroups = (unsigned)(((long long)a.B * a.chunks.n + 7) / 8 * 8 * a.Hk);
  if (a.d == 64) {
    if (f16) e4m3 ? fm::launch<64, true, true>(a, workgroups, stream) : fm::launch<64, true, false>(a, workgroups, stream);
    else e4m3 ? fm::launch<64, false, true>(a, workgroups, stream) : fm::launch<64, false, false>(a, workgroups, stream);
  } else {
    if (f16) e4m3 ? fm::launch<128, true, true>(a, workgroups, stream) : fm::launch<128, true, false>(a, workgroups, stream);
    else e4m3 ? fm::launch<128, false, true>(a, workgroups, stream) : fm::launch<128, false, false>(a, workgroups, stream);
  }
  return hipGetLastError();
}
