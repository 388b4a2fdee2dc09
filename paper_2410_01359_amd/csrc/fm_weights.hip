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
constexpr int kKeys = 256, kTile = 64;

template <int D>
struct WeightsShared {
  alignas(16) char q[2][kTile * TileLayout<D>::RS];
  alignas(16) float lse[2][kTile];
  int minmax[4][8];
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
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    int x = sh.minmax[0][w];
#pragma unroll
    for (int i = 1; i < 4; ++i) x = w % 2 ? min(x, sh.minmax[i][w]) : max(x, sh.minmax[i][w]);
    all.v[w] = __builtin_amdgcn_readfirstlane(x);
  }

  // Tiles of this part: head h, tile t of its rows
  struct Tile {
    int at, h, row;
  };
  const int last = min((part + 1) * a.part_tiles, G * a.row_tiles);
  const auto live = [&](Tile t) {   // the first live one from t on
    while (t.at < last && classify_tile(t.row, min(t.row + kTile, a.N), all) == T_FULLY) {
      ++t.at;
      t.row += kTile;
      if (t.row >= a.N) {
        t.row = a.first_row;
        ++t.h;
      }
    }
    return t;
  };
  const auto behind = [&](Tile t) {
    ++t.at;
    t.row += kTile;
    if (t.row >= a.N) {
      t.row = a.first_row;
      ++t.h;
    }
    return live(t);
  };
  u32x4 staged[LOADS];
  float staged_lse = 0.f;
  const auto load = [&](const Tile& t) {
    const char* rows = (const char*)a.q + 2 * ((long long)b * a.sq.b + (long long)(hk * G + t.h) * a.sq.h);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int piece = i * 256 + threadIdx.x, row = min(t.row + piece / PIECES, a.N - 1);
      staged[i] = ldg16(rows + 2 * ((long long)row * a.sq.n + piece % PIECES * 8));
    }
    if (threadIdx.x < kTile) staged_lse = a.lse[((size_t)b * a.H + hk * G + t.h) * a.N + min(t.row + (int)threadIdx.x, a.N - 1)];
  };

  const float scale = a.scale * kLog2e;
  float sum[2] = {0.f, 0.f};
  Tile t;
  t.at = part * a.part_tiles;
  t.h = fm_div(t.at, a.by_tile);
  t.row = a.first_row + (t.at - t.h * a.row_tiles) * kTile;
  t = live(t);
  if (t.at < last) load(t);
  for (int buffer = 0; t.at < last; buffer ^= 1) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int piece = i * 256 + threadIdx.x;
      *(u32x4*)(sh.q[buffer] + L::off(piece / PIECES, piece % PIECES * 16)) = staged[i];
    }
    if (threadIdx.x < kTile) sh.lse[buffer][threadIdx.x] = minus_lse(staged_lse);
    const Tile now = t;
    t = behind(t);
    if (t.at < last) load(t);
    barrier_nofence();   // the next tile's loads stay in flight

    const int cls = classify_tile(now.row, min(now.row + kTile, a.N), mine);
    if (cls == T_FULLY) continue;
    const auto scores = [&](int m, f32x16 (&s)[2]) {
      s[0] = s[1] = f32x16{};
#pragma unroll
      for (int step = 0; step < STEPS; ++step) {
        const bf16x8 rows = *(const bf16x8*)(sh.q[buffer] + L::add_col(row_part, 32 * step) + 32 * m * L::RS);
        s[0] = mfma32(rows, k[0][step], s[0]);
        s[1] = mfma32(rows, k[1][step], s[1]);
      }
    };
    // a tile's sums first: partial sums of 32 rows keep the error of long ones down
    const auto add = [&](int m, const f32x16 (&s)[2]) {
      float tile[2] = {0.f, 0.f};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 lse = *(const f32x4*)&sh.lse[buffer][32 * m + 8 * q + 4 * half];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) tile[n] += fast_exp2(fmaf(s[n][4 * q + r], scale, lse[r]));
      }
      sum[0] += tile[0];
      sum[1] += tile[1];
    };
    if (cls == T_UNMASKED && now.row + kTile <= a.N) {
      f32x16 s[2][2];
      scores(0, s[0]);
      scores(1, s[1]);
      add(0, s[0]);
      add(1, s[1]);
    } else {
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        f32x16 s[2];
        scores(m, s);
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            hide4(s[n], 4 * q, [&](int r) {
              const int i = now.row + 32 * m + 8 * q + 4 * half + r;
              return (i >= a.N) | ((bound[n][0] <= i) & (i < bound[n][1])) | ((bound[n][2] <= i) & (i < bound[n][3]));
            });
        add(m, s);
      }
    }
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
  const int tiles = (N - first_row + fm::kTile - 1) / fm::kTile, all = H / Hk * tiles;
  cut.row_tiles = tiles;
  cut.key_blocks = (N + fm::kKeys - 1) / fm::kKeys;
  // eight rounds of the places that the chip has, parts of 16 tiles at least
  const long long units = (long long)B * Hk * cut.key_blocks, wanted = 16ll * (cus > 0 ? cus : 256);
  long long parts = std::max<long long>(1, std::min<long long>((wanted + units - 1) / units, all / 16));
  cut.part_tiles = (int)((all + parts - 1) / parts);
  cut.parts = (all + cut.part_tiles - 1) / cut.part_tiles;
  return cut;
}

hipError_t fm_launch_weights(FmWeightsArgs a, float* weights, const FmWeightsCut& cut, hipStream_t stream) {
  a.row_tiles = cut.row_tiles;
  a.parts = cut.parts;
  a.part_tiles = cut.part_tiles;
  a.slices = fm_divisor(a.B * a.Hk);
  a.by_part = fm_divisor(cut.parts);
  a.by_head = fm_divisor(a.Hk);
  a.by_tile = fm_divisor(cut.row_tiles);
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
