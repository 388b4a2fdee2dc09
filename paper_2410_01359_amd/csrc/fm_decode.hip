// Attention of the last tokens of every sequence over a paged cache (flashmask_decode).
//
// The H / Hk * T query rows that share a K/V head are the columns of both products: with 16-row groups of keys
//     S^T = K Q^T   (16 keys x 16 queries: a lane has keys 4 g + r of query c, g = lane / 16, c = lane % 16)
//     O^T = V^T P^T (16 elements of d x 16 queries, contraction over 32 keys)
// by the 16x16x32 matrix instruction.  Softmax statistics are per column, so rescaling and the final division stay in the lane.
// Keys and values go straight from memory to the operands, without LDS:
//  - K: lane (g, c) loads 16 bytes of key c; which elements of d a product takes together is free, as long as Q has them in the
//    same order.
//  - V: lane (g, c) loads the same piece of d (D / 16 elements, piece c) of the eight keys whose probabilities it holds of its
//    column, and the eight 16-bit values of each element are gathered by byte permutes: product e has as its rows the
//    elements D / 16 * m + e, m = 0..15.  The lane's results are then 4 * D / 16 consecutive elements of its query's row.
// The probabilities go into the second product as sums of two 16-bit values, which the matrix pipe has room for.
// Bound by memory: every wave has the next step's 16 KiB of keys and values in flight while it works on this one's.  131072 tokens, 8
// heads of 128 elements: 94 us, 5.7 TB/s of the 6.4 that a plain reading loop reaches here, and 5 for the join.
#include <algorithm>

#include "fm_cache_math.h"
#include "fm_common.h"
#include "fm_serving.h"
#include "fm_tree.h"

namespace fm {

constexpr int kGroup = FM_KEY_GROUP;
constexpr int kWaves = 4;

template <int D, bool F16, bool E4M3, int NB>
struct Decode {
  static constexpr int BYTES = E4M3 ? 1 : 2;
  // keys of a wave's step: 16 KiB of K and V, fewer where the scores of NB query blocks would not fit the registers
  static constexpr int KT = std::min(16384 / (64 * D * BYTES), std::max(256 / (D * NB), 1)), GROUPS = 2 * KT, KEYS = 32 * KT;
  static constexpr int KSTEPS = D / 32;             // products of S^T
  static constexpr int KLOADS = D * BYTES / 64;     // 16-byte loads of a lane per group of keys
  static constexpr int E = D / 16;                  // products of O^T; elements of d in a lane's piece of a value row
  static constexpr int VWORDS = E * BYTES / 4;      // words of that piece
  static constexpr int ROWS = 16 * NB;              // query rows
  static constexpr int PANEL = 2048, LIST = PANEL / KEYS;   // keys, and steps, whose bounds are looked at together
  typedef __attribute__((ext_vector_type(VWORDS))) unsigned vpiece;
  struct Shared {
    union {
      struct {
        i32x4 bound[PANEL];
        int list[LIST], flag[LIST], count;
      };
      float out[kWaves][16][D + 4];
    };
    float2 stat[kWaves][16];
    int odd;   // an infinity or NaN among values that some rows see and others do not
  };
};

template <class Args>
constexpr bool kTree = std::is_same_v<Args, FmTreeArgs>;

// TEAMS > 1: the workgroup's waves are teams that go over the same keys together, for blocks of query rows, which find in the caches what
// the first of them loads, or for heads whose rows lie side by side.
// FmTreeArgs: the new tokens are a tree.
template <int D, bool F16, bool E4M3, int NB, int TEAMS, class Args>
__global__ __launch_bounds__(64 * kWaves, 2) void decode_kernel(Args a, int members, FmDivisor inner, FmDivisor row_blocks,
                                                              FmDivisor tokens, FmDivisor chunks_meant) {
  constexpr int TW = kWaves / TEAMS;   // waves of a team
  using C = Decode<D, F16, E4M3, NB>;
  __shared__ typename C::Shared sh;
  __shared__ std::conditional_t<kTree<Args>, SmallTree, char> tree;   // of few tokens (fm_tree_is_wide)
  // Barriers here order LDS alone (barrier_nofence): loads stay in flight across them.
  // The launch arguments that come first, read together: left where they are first needed they are six round trips in a row.
  asm volatile("" ::"s"(a.units), "s"(a.plan), "s"(a.lens), "s"(a.B), "s"(a.T), "s"(a.window), "s"(a.columns), "s"(a.page_tokens), "s"(a.cut.least),
               "s"(a.first_workgroup), "s"(inner.factor), "s"(row_blocks.factor), "s"(chunks_meant.factor), "s"(members));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, c = lane & 15;
  // Workgroup -> chunk of a sequence, K/V head, block of query rows.  Workgroup x runs on XCD x % 8: all heads of a chunk on one,
  // one behind the other, because they share page table entries, bounds, and cache lines where heads lie next to each other.
  const int workgroup = a.first_workgroup + blockIdx.x, slot_of_xcd = workgroup >> 3;
  const int turn = fm_div(slot_of_xcd, inner), pair = slot_of_xcd - turn * (int)inner.n;
  const int unit = turn * 8 + (workgroup & 7);
  const int team = wave % TEAMS, team_wave = wave / TEAMS, team_thread = team_wave * 64 + lane;
  const bool idle = pair * TEAMS + team >= members;   // a last team without a partner
  const int member = idle ? members - 1 : pair * TEAMS + team;
  const int hk = fm_div(member, row_blocks), rb = member - hk * (int)row_blocks.n;

  // Chunk: all sequences' keys together are cut into about a.cut.chunks pieces, each sequence into whole ones of that size.  Every wave works
  // this out for itself, 64 sequences at a time; up to 64 their lengths are read once.  Where that is too much work the list of units has it.
  int b = unit, chunk = 0, chunks = 1, slot = 0, size = 1 << 26, len;   // size: in groups, more than any table's
  if (a.units) {
    const FM_CONSTANT int* entry = (const FM_CONSTANT int*)(a.units + unit);
    b = entry[0];
    if (b < 0) return;
    len = entry[1];
    chunk = entry[2] & 0xffff;
    chunks = entry[2] >> 16;
    slot = entry[3];
  } else if (a.plan) {
    int lane_len = lane < a.B ? a.lens[lane] : 0;
    const auto lane_groups = [&](int base) {
      if (a.B > 64) lane_len = base + lane < a.B ? a.lens[base + lane] : 0;
      return fm_key_groups(fm_key_range(lane_len, a.T, a.window, a.columns * a.page_tokens));
    };
    unsigned total = 0;
    for (int base = 0; base < a.B; base += 64) total += wave_last(wave_scan(lane_groups(base)));
    size = fm_chunk_groups(total, chunks_meant, a.cut.least, TW * C::GROUPS);
    int units = 0, slots = 0, base = 0;
    while (true) {
      const int n = base + lane < a.B ? fm_chunks_of(lane_groups(base), size) : 0;
      const int upto = wave_scan(n), upto_slots = wave_scan(n > 1 ? n : 0);
      const unsigned long long behind = __ballot(units + upto > unit);
      if (behind) {
        const int at = __builtin_ctzll(behind);
        b = base + at;
        chunks = __builtin_amdgcn_readlane(n, at);
        chunk = unit - (units + __builtin_amdgcn_readlane(upto, at) - chunks);
        slot = slots + __builtin_amdgcn_readlane(upto_slots, at) - (chunks > 1 ? chunks : 0);
        len = __builtin_amdgcn_readlane(lane_len, at);
        break;
      }
      units += wave_last(upto);
      slots += wave_last(upto_slots);
      base += 64;
      if (base >= a.B) return;
    }
    if (chunk == 0 && pair == 0 && threadIdx.x == 0) a.plan[b] = int2{slot, chunks};
  } else {
    if (b >= a.B) return;
    len = a.lens[b];
  }
  const FmKeyRange range = fm_key_range(len, a.T, a.window, a.columns * a.page_tokens);
  // a sequence's chunks alike, instead of a last short one: 64 ragged sequences 88 -> 82 us, windows 46 -> 43
  if (chunks > 1) size = fm_even_chunk(fm_key_groups(range), chunks, C::GROUPS);
  const int j_begin = range.lo + chunk * size * kGroup;
  const int j_end = (int)std::min<long long>(range.hi, j_begin + (long long)size * kGroup);
  const int first_row = range.len - a.T;   // row of query 0
  // The tree is planted where it is first needed, which not all chunks do: its parents are asked for here
  int parent = -1;
  bool planted = false;
  if constexpr (kTree<Args>) {
    static_assert(fm_tree_is_wide(1, 64, D, E4M3));   // SmallTree
    if (lane < a.T) parent = a.parents[(size_t)b * a.T + lane];
  }
  const auto plant_tree = [&] {
    if constexpr (kTree<Args>) {
      if (!planted) plant_small(tree, parent, a.T);
      planted = true;
    }
  };
  if (a.bounds[0]) plant_tree();
  // Row of query t, and whether it sees key j, bounds apart
  const auto row_of = [&](int t) {
    if constexpr (kTree<Args>) return first_row + tree.depth[t];
    else return first_row + t;
  };
  const auto reaches = [&](int j, int t) {
    const int i = row_of(t);
    if constexpr (kTree<Args>) {
      const int u = j - first_row;
      if (first_row + t < 0) return false;   // not there
      return u < 0 ? a.window <= 0 || j > i - a.window : u < a.T && tree.on_path(t, u) && (a.window <= 0 || tree.depth[t] - tree.depth[u] < a.window);
    } else {
      return j <= i && (a.window <= 0 || j > i - a.window);
    }
  };

  // Queries
  const int G = a.H / a.Hk, R = G * a.T;
  u32x4 q[NB][C::KSTEPS];
  int column_token[NB];   // query t of the lane's column, -1: none
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = rb * C::ROWS + nb * 16 + c;
    column_token[nb] = -1;
#pragma unroll
    for (int s = 0; s < C::KSTEPS; ++s) q[nb][s] = u32x4{0, 0, 0, 0};
    if (r < R) {
      const int hq = fm_div(r, tokens), t = r - hq * a.T;
      column_token[nb] = kTree<Args> && first_row + t < 0 ? -1 : t;
      const char* p = (const char*)a.q + 2 * ((long long)b * a.sq.b + (long long)(hk * G + hq) * a.sq.h + (long long)t * a.sq.n);
#pragma unroll
      for (int s = 0; s < C::KSTEPS; ++s)
        q[nb][s] = ldg16(p + 2 * (E4M3 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g));
    }
  }
  const float scale = a.scale * kLog2e * (E4M3 ? a.k_scale[hk] : 1.f);

  // Where the lane's pieces of a group of keys lie
  const char* k_head = a.k.base + (long long)hk * a.k.head;
  const char* v_head = a.v.base + (long long)hk * a.v.head;
  const unsigned k_lane = c * a.k.token + 16 * g;
  unsigned v_lane[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) v_lane[t] = (4 * g + t) * a.v.token + c * (C::E * C::BYTES);
  // The table is read through the scalar cache (nothing here writes it): a vector load would come back behind the keys and values asked
  // for before it, and waiting for it meant waiting for them (64 ragged sequences 88 -> 81 us).
  const FM_CONSTANT int* row = (const FM_CONSTANT int*)(a.table + (size_t)b * a.columns);

  // A step's groups: their table entries, as read (a step ahead: nothing waits for them here), and slots, -1 behind the last key
  struct Step {
    int entry[C::GROUPS], slot[C::GROUPS];
    int num_pages;
    __device__ __forceinline__ int page(int i) const { return fm_known_page(slot[i] < 0 ? -1 : entry[i], num_pages); }
  };
  const auto pages_of = [&](int start) {
    Step p;
    p.num_pages = a.num_pages;
#pragma unroll
    for (int i = 0; i < C::GROUPS; ++i) {
      const int key = start + i * kGroup, at = key < j_end ? key : j_begin, column = fm_div(at, a.page);
      p.entry[i] = row[column];
      p.slot[i] = key < j_end ? at - column * (int)a.page.n : -1;
    }
    return p;
  };
  u32x4 kraw[C::GROUPS][C::KLOADS];
  typename C::vpiece vraw[C::KT][8];
  // Through buffer descriptors of no bytes where there is no page (its sign is set), or no step (`there` = 0, not -1): such loads give 0 and
  // touch no memory, and the loop's loads need no branch, behind which the compiler would wait for all of them at the first
  // use of any.
  const auto descriptor = [](const char* base, int page, int there) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, __builtin_amdgcn_readfirstlane(~(page >> 31) & there), 0x00020000);
  };
  const auto load_k = [&](const Step& p, int there) {
#pragma unroll
    for (int i = 0; i < C::GROUPS; ++i) {
      const int page = p.page(i);
      const auto rows = descriptor(k_head + std::max(page, 0) * a.k.page + (unsigned)std::max(p.slot[i], 0) * (unsigned long long)a.k.token,
                                   page, there);
#pragma unroll
      for (int s = 0; s < C::KLOADS; ++s)
        kraw[i][s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, k_lane + 64 * s, 0, 0));
    }
  };
  const auto load_v = [&](const Step& p, int there) {
#pragma unroll
    for (int i = 0; i < C::GROUPS; ++i) {
      const int page = p.page(i);
      const auto rows = descriptor(v_head + std::max(page, 0) * a.v.page + (unsigned)std::max(p.slot[i], 0) * (unsigned long long)a.v.token,
                                   page, there);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        typename C::vpiece& x = vraw[i / 2][i % 2 * 4 + t];
        if constexpr (C::VWORDS == 4) x = __builtin_bit_cast(typename C::vpiece, __builtin_amdgcn_raw_buffer_load_b128(rows, v_lane[t], 0, 0));
        else if constexpr (C::VWORDS == 2) x = __builtin_bit_cast(typename C::vpiece, __builtin_amdgcn_raw_buffer_load_b64(rows, v_lane[t], 0, 0));
        else x[0] = __builtin_amdgcn_raw_buffer_load_b32(rows, v_lane[t], 0, 0);
      }
    }
  };

  // Which of the lane's keys (bit 4 i + r: key 4 g + r of group i) query t sees
  const auto seen_keys = [&](int start, int panel, unsigned pages_there, int t) {
    unsigned seen = 0;
    const int row_i = row_of(t);
    unsigned long long line = 0;   // drafted tokens that a drafted one sees, windows apart
    if constexpr (kTree<Args>) line = (unsigned long long)tree.ancestors[t][1] << 32 | tree.ancestors[t][0];
    const int last = min(j_end - 1, row_i), first = a.window > 0 ? row_i - a.window + 1 : 0;
#pragma unroll 1
    for (int i = 0; i < C::GROUPS; ++i) {
      const int j = start + i * kGroup + 4 * g;
      unsigned four = 0;
      if (kTree<Args> && a.window <= 0) {
        const int u = j - first_row, left = j_end - j;   // the first of the four keys as a drafted token, and keys
        four = u >= 64 ? 0u : u >= 0 ? (unsigned)(line >> u) : u > -4 ? (unsigned)line << -u | ((1u << -u) - 1u) : 15u;
        four &= left >= 4 ? 15u : left > 0 ? (1u << left) - 1u : 0u;
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if constexpr (kTree<Args>) four |= (j + r < j_end && reaches(j + r, t) ? 1u : 0u) << r;
          else four |= (j + r <= last && j + r >= first ? 1u : 0u) << r;
        }
      }
      if (a.bounds[0]) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (hides(sh.bound[min(j + r - panel, C::PANEL - 1)], row_i)) four &= ~(1u << r);
      }
      seen |= (pages_there >> i & 1 ? four : 0u) << (4 * i);
    }
    return seen;
  };

  // Columns are worked on together.  A value that one row sees and another does not enters the other's sum times 0, so an infinity or
  // NaN among those would reach rows that do not see it: where one turns up, the workgroup begins again and takes the
  // rows of one query t at a time, which all see the same keys.
  if (threadIdx.x == 0) sh.odd = 0;
  for (int only = -1, rounds = 1; rounds > 0; --rounds) {
    int row_token[NB];
    float m[NB], l[NB];
    f32x4 acc[NB][C::E];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      row_token[nb] = only < 0 || column_token[nb] == only ? column_token[nb] : -1;
      m[nb] = -INFINITY;
      l[nb] = 0.f;
#pragma unroll
      for (int e = 0; e < C::E; ++e) acc[nb][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    barrier_nofence();

    for (int panel = j_begin; panel < j_end; panel = fm_next_panel(panel, j_end, a.bounds[0] ? C::PANEL : 0)) {
      int steps;
      if (a.bounds[0]) {
        // the steps of which some row sees a key, and whether it takes the element mask
        const int end = min(j_end, panel + C::PANEL), all = (end - panel + C::KEYS - 1) / C::KEYS;
        for (int i = threadIdx.x; i < all; i += 64 * kWaves) sh.flag[i] = 0;
        barrier_nofence();
        for (int j = panel + threadIdx.x; j < end; j += 64 * kWaves) {
          i32x4 bound = {0, 0, 0, 0};
          if (j < a.bound_columns) {
#pragma unroll
            for (int w = 0; w < 4; ++w) bound[w] = a.bounds[w][(size_t)b * a.bound_columns + j];
          }
          sh.bound[j - panel] = bound;
          int flag = 0;
          for (int t = 0; t < a.T; ++t) {
            flag |= reaches(j, t) && !hides(bound, row_of(t)) ? 1 : 2;
          }
          atomicOr(&sh.flag[(j - panel) / C::KEYS], flag);
        }
        barrier_nofence();
        if (wave == 0) {
          int count = 0;
          for (int base = 0; base < all; base += 64) {
            const int flag = base + lane < all ? sh.flag[base + lane] : 0;
            const unsigned long long live = __ballot(flag & 1);
            if (flag & 1) sh.list[count + __popcll(live & ((1ull << lane) - 1ull))] = (base + lane) * 4 + flag;
            count += __popcll(live);
          }
          if (lane == 0) sh.count = count;
        }
        barrier_nofence();
        steps = __builtin_amdgcn_readfirstlane(sh.count);
      } else {
        steps = (j_end - panel + C::KEYS - 1) / C::KEYS;
      }
      const auto entry_of = [&](int s) { return a.bounds[0] ? __builtin_amdgcn_readfirstlane(sh.list[s]) : s * 4; };

      if (team_wave < steps && !idle) {
        int entry = entry_of(team_wave);
        Step now = pages_of(panel + entry / 4 * C::KEYS);
        load_k(now, -1);
        load_v(now, -1);
        int next_entry = team_wave + TW < steps ? entry_of(team_wave + TW) : entry;
        Step next = pages_of(panel + next_entry / 4 * C::KEYS);
        for (int s = team_wave; s < steps; s += TW) {
          const int more = (s + TW - steps) >> 31;   // -1: another step follows
          const int start = panel + entry / 4 * C::KEYS;
          bool masked = (entry & 2) || start + C::KEYS > j_end || start + C::KEYS - 1 > first_row - (kTree<Args> ? 1 : 0) ||
                        (a.window > 0 && start <= range.len - 1 - a.window);
#pragma unroll
          for (int i = 0; i < C::GROUPS; ++i) masked |= now.page(i) < 0;

          // scores
          f32x4 p[NB][C::GROUPS];
#pragma unroll
          for (int i = 0; i < C::GROUPS; ++i) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) p[nb][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < C::KSTEPS; ++k) {
              u32x4 op;
              if constexpr (E4M3) {
                const u32x4 raw = kraw[i][k / 2];
                const u32x2 x = widen4<F16>(raw[k % 2 * 2]), y = widen4<F16>(raw[k % 2 * 2 + 1]);
                op = u32x4{x[0], x[1], y[0], y[1]};
              } else {
                op = kraw[i][k];
              }
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) p[nb][i] = mfma_keys<F16>(op, q[nb][k], p[nb][i]);
            }
          }
          load_k(next, more);

#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < C::GROUPS; ++i) p[nb][i] *= scale;

          // element mask; values that no row sees become 0 (the keys of a lane's scores are those of its value pieces).  Which of its
          // keys a column sees is gathered as bits by a loop: unrolled, the bounds' addresses alone would fill the registers.
          if (masked) {
            plant_tree();
            unsigned pages_there = 0;
#pragma unroll
            for (int i = 0; i < C::GROUPS; ++i) pages_there |= (now.page(i) >= 0 ? 1u : 0u) << i;
            unsigned any = 0, every = ~0u;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const bool real = row_token[nb] >= 0;
              const unsigned seen = real ? seen_keys(start, panel, pages_there, row_token[nb]) : 0u;
              any |= row16_or(seen);
              every &= ~row16_or(real ? ~seen : 0u);
#pragma unroll
              for (int i = 0; i < C::GROUPS; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                  if (!(seen >> (4 * i + r) & 1)) p[nb][i][r] = -INFINITY;
            }
            if (__any((any & ~every) != 0)) {
              bool odd = false;
#pragma unroll
              for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
                for (int t = 0; t < 8; ++t)
#pragma unroll
                  for (int w = 0; w < C::VWORDS; ++w) odd |= (any & ~every) >> (8 * kt + t) & 1 && odd_word<F16, E4M3>(vraw[kt][t][w]);
              if (odd) sh.odd = 1;
            }
#pragma unroll
            for (int i = 0; i < C::GROUPS; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (!(any >> (4 * i + r) & 1)) vraw[i / 2][i % 2 * 4 + r] = (typename C::vpiece)(0u);
          }

          // softmax
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float top = p[nb][0][0];
#pragma unroll
            for (int i = 0; i < C::GROUPS; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) top = fmaxf(top, p[nb][i][r]);
            top = fmaxf(quad_max(top), m[nb]);
            const float ref = reference(top), alpha = fast_exp2(m[nb] - ref);
            m[nb] = top;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < C::GROUPS; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                p[nb][i][r] = fast_exp2(p[nb][i][r] - (ref - kShift<F16>));
                sum += p[nb][i][r];
              }
            l[nb] = l[nb] * alpha + sum;
            if (__any(alpha != 1.f)) {   // seldom, after the first steps
#pragma unroll
              for (int e = 0; e < C::E; ++e) acc[nb][e] *= alpha;
            }
          }

          // products with the values
#pragma unroll
          for (int kt = 0; kt < C::KT; ++kt) {
            u32x4 hi[NB], lo[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                unsigned h, o;
                split2<F16>(p[nb][2 * kt + w / 2][2 * (w % 2)], p[nb][2 * kt + w / 2][2 * (w % 2) + 1], h, o);
                hi[nb][w] = h;
                lo[nb][w] = o;
              }
            unsigned v[8][C::E / 2];
#pragma unroll
            for (int t = 0; t < 8; ++t) {
              if constexpr (E4M3) {
#pragma unroll
                for (int w = 0; w < C::VWORDS; ++w) {
                  const u32x2 x = widen4<F16>(vraw[kt][t][w]);
                  v[t][2 * w] = x[0];
                  v[t][2 * w + 1] = x[1];
                }
              } else {
#pragma unroll
                for (int w = 0; w < C::VWORDS; ++w) v[t][w] = vraw[kt][t][w];
              }
            }
#pragma unroll
            for (int e = 0; e < C::E; ++e) {
              u32x4 op;
#pragma unroll
              for (int w = 0; w < 4; ++w) op[w] = pair_of(v[2 * w][e / 2], v[2 * w + 1][e / 2], e % 2);
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) {
                acc[nb][e] = mfma_keys<F16>(op, lo[nb], acc[nb][e]);
                acc[nb][e] = mfma_keys<F16>(op, hi[nb], acc[nb][e]);
              }
            }
          }
          load_v(next, more);
          entry = next_entry;
          now = next;
          next_entry = s + 2 * TW < steps ? entry_of(s + 2 * TW) : entry;
          next = pages_of(panel + next_entry / 4 * C::KEYS);
        }
      }
      if (a.bounds[0]) barrier_nofence();
    }

    barrier_nofence();
    if (only < 0 && __builtin_amdgcn_readfirstlane(sh.odd)) {
      only = 0;
      rounds = a.T + 1;
      continue;
    }

    // A team's sums meet in LDS, 16 rows at a time
    constexpr int PER = 16 * D / (64 * TW);   // elements of a thread: neighbours of one row
    const int my_row = team_thread * PER / D, my_col = team_thread * PER % D;
    const float v_scale = E4M3 ? a.v_scale[hk] : 1.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float sum = quad_sum(l[nb]);
      if (g == 0) sh.stat[wave][c] = float2{m[nb], sum};
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < C::E; e += 4)
          *(f32x4*)&sh.out[wave][c][4 * C::E * g + C::E * r + e] =
              f32x4{acc[nb][e][r], acc[nb][e + 1][r], acc[nb][e + 2][r], acc[nb][e + 3][r]};
      barrier_nofence();
      float top = -INFINITY, total = 0.f, x[PER];
#pragma unroll
      for (int w = 0; w < TW; ++w) top = fmaxf(top, sh.stat[w * TEAMS + team][my_row].x);
#pragma unroll
      for (int e = 0; e < PER; ++e) x[e] = 0.f;
#pragma unroll
      for (int w = 0; w < TW; ++w) {
        const float2 stat = sh.stat[w * TEAMS + team][my_row];
        const float weight = fast_exp2(stat.x - reference(top));
        total += weight * stat.y;
#pragma unroll
        for (int e = 0; e < PER; ++e) x[e] += weight * sh.out[w * TEAMS + team][my_row][my_col + e];
      }
      const int r = rb * C::ROWS + nb * 16 + my_row;
      if (r < R && !idle && (only < 0 || r % a.T == only)) {
        if (chunks > 1) {
          const size_t at = ((size_t)(slot + chunk) * a.Hk + hk) * R + r;
#pragma unroll
          for (int e = 0; e < PER; e += 4) *(f32x4*)(a.part + at * D + my_col + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
          if (my_col == 0) a.stat[at] = float2{top, total};
        } else {
          const int hq = fm_div(r, tokens), t = r - hq * a.T, h = hk * G + hq;
          const float factor = total == 0.f ? 0.f : v_scale / total;
          char* o = (char*)a.out + 2 * ((long long)b * a.so.b + (long long)h * a.so.h + (long long)t * a.so.n + my_col);
#pragma unroll
          for (int e = 0; e < PER; e += 2) *(unsigned*)(o + 2 * e) = pack2<F16>(x[e] * factor, x[e + 1] * factor);
          if (my_col == 0) a.lse[((size_t)b * a.H + h) * a.T + t] = total == 0.f ? -INFINITY : (top + fast_log2(total * kUnshift<F16>)) * kLn2;
        }
      }
      barrier_nofence();
    }
    if (only >= 0) ++only;
  }
}

// The list of units: one workgroup goes over the lengths twice, 1024 at a time, and lists each sequence's chunks, for workgroups that do not go
// over all lengths themselves, which takes a call time with the square of its sequences.
constexpr int kPlanThreads = 1024;
__global__ __launch_bounds__(kPlanThreads) void plan_units_kernel(FmDecodeArgs a, FmDivisor chunks_meant, int round, int units, int splits) {
  __shared__ int sums[2][3][kPlanThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const auto groups_of = [&](int len) { return fm_key_groups(fm_key_range(len, a.T, a.window, a.columns * a.page_tokens)); };
  int mine = 0;
  for (int b = tid; b < a.B; b += kPlanThreads) mine += groups_of(a.lens[b]);
  const int upto = wave_scan(mine);
  if (lane == 63) sums[1][0][wave] = upto;
  __syncthreads();
  unsigned total = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) total += sums[1][0][w];
  const int size = fm_chunk_groups(total, chunks_meant, a.cut.least, round);
  int before[3] = {0, 0, 0};   // units, slots, split sequences
  for (int base = 0, turn = 0; base < a.B; base += kPlanThreads, turn ^= 1) {
    const int b = base + tid, len = b < a.B ? a.lens[b] : 0, n = b < a.B ? fm_chunks_of(groups_of(len), size) : 0;
    const int x[3] = {n, n > 1 ? n : 0, n > 1};
    int at[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      at[i] = wave_scan(x[i]);
      if (lane == 63) sums[turn][i][wave] = at[i];
    }
    __syncthreads();   // the other turn's sums have been read before this one's are written again
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      at[i] += before[i] - x[i];
#pragma unroll
      for (int w = 0; w < kPlanThreads / 64; ++w) {
        const int sum = sums[turn][i][w];
        if (w < wave) at[i] += sum;
        before[i] += sum;
      }
    }
    for (int c = 0; c < n; ++c) a.units[at[0] + c] = int4{b, len, c | n << 16, at[1]};
    if (n > 1) {
      a.plan[b] = int2{at[1], n};
      a.split[at[2]] = b;
    }
  }
  for (int i = before[0] + tid; i < units; i += kPlanThreads) a.units[i] = int4{-1, 0, 0, 0};
  for (int i = before[2] + tid; i < splits; i += kPlanThreads) a.split[i] = -1;
}

// Joins the chunks of a row of a split sequence: D / 4 lanes take a chunk's sums of p v, the workgroup 1024 / D chunks at a time.  Bound by
// its chain of round trips, 4 to 5 us.
template <int D, bool F16>
__global__ __launch_bounds__(256) void join_kernel(FmDecodeArgs a, FmDivisor rows, FmDivisor tokens) {
  constexpr int LANES = D / 4, TEAMS = 256 / LANES, BATCH = 4;
  asm volatile("" ::"s"(a.split), "s"(a.plan), "s"(a.part), "s"(a.stat), "s"(a.H), "s"(rows.factor));   // read together
  const int G = a.H / a.Hk, R = G * a.T;
  const int b = a.split ? a.split[blockIdx.y] : blockIdx.y, hk = fm_div(blockIdx.x, rows), r = blockIdx.x - hk * R;   // row of the K/V head
  if (b < 0) return;
  const int2 plan = a.plan[b];
  if (plan.y <= 1) return;
  const int team = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  float m = -INFINITY, l = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int base = team; base < plan.y; base += TEAMS * BATCH) {
    f32x4 v[BATCH];
    float2 s[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int c = base + i * TEAMS;
      s[i] = float2{-INFINITY, 0.f};
      v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (c < plan.y) {
        const size_t at = ((size_t)(plan.x + c) * a.Hk + hk) * R + r;
        s[i] = a.stat[at];
        v[i] = *(const f32x4*)(a.part + at * D + 4 * lane);
      }
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
      const float w = fast_exp2(s[i].x - reference(top));
      l += w * s[i].y;
      x += w * v[i];
    }
  }
  __shared__ f32x4 sums[TEAMS][LANES];
  __shared__ float2 stats[TEAMS];
  sums[team][lane] = x;
  if (lane == 0) stats[team] = float2{m, l};
  __syncthreads();
  if (team > 0) return;
  float top = -INFINITY, total = 0.f;
#pragma unroll
  for (int w = 0; w < TEAMS; ++w) top = fmaxf(top, stats[w].x);
  x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < TEAMS; ++w) {
    const float weight = fast_exp2(stats[w].x - reference(top));
    total += weight * stats[w].y;
    x += weight * sums[w][lane];
  }
  const int hq = fm_div(r, tokens), t = r - hq * a.T, h = hk * G + hq;
  const float factor = total == 0.f ? 0.f : (a.v_scale ? a.v_scale[hk] : 1.f) / total;
  char* o = (char*)a.out + 2 * ((long long)b * a.so.b + (long long)h * a.so.h + (long long)t * a.so.n + 4 * lane);
  *(u32x2*)o = u32x2{pack2<F16>(x[0] * factor, x[1] * factor), pack2<F16>(x[2] * factor, x[3] * factor)};
  if (lane == 0) a.lse[((size_t)b * a.H + h) * a.T + t] = total == 0.f ? -INFINITY : (top + fast_log2(total * kUnshift<F16>)) * kLn2;
}

static void launch_list(const FmDecodeArgs& a, int round, hipStream_t stream) {
  hipLaunchKernelGGL(plan_units_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a, fm_divisor(a.cut.chunks), round,
                     fm_listed_units(a.cut.chunks, a.B), fm_most_splits(a.cut.chunks, a.B));
}
template <int D, bool F16>
static void launch_join(const FmDecodeArgs& a, hipStream_t stream) {
  const int R = a.H / a.Hk * a.T;
  hipLaunchKernelGGL((join_kernel<D, F16>), dim3(a.Hk * R, a.split ? fm_most_splits(a.cut.chunks, a.B) : a.B), dim3(256), 0, stream, a, fm_divisor(R),
                     fm_divisor(a.T));
}

template <int D, bool E4M3>
static int round_groups(const FmDecodeCut& cut) {
  return kWaves / cut.teams * (cut.block_rows == 16 ? Decode<D, false, E4M3, 1>::GROUPS : Decode<D, false, E4M3, 2>::GROUPS);
}

template <int D, bool F16, bool E4M3, class Args>
static void launch(Args a, hipStream_t stream) {
  constexpr int kMost = 1 << 23;   // workgroups of a launch, which has fewer than 2^32 lanes
  const FmDecodeCut& cut = a.cut;
  const int units = a.plan ? fm_listed_units(cut.chunks, a.B) : (a.B + 7) / 8 * 8, workgroups = units * cut.workgroups;
  const FmDivisor di = fm_divisor(cut.workgroups), dr = fm_divisor(cut.row_blocks), dt = fm_divisor(a.T), dc = fm_divisor(cut.chunks);
#define FM_DECODE(NB, TEAMS)                                                                                                      \
  hipLaunchKernelGGL((decode_kernel<D, F16, E4M3, NB, TEAMS, Args>), dim3((unsigned)std::min(workgroups - a.first_workgroup, kMost)), \
                     dim3(64 * kWaves), 0, stream, a, cut.row_blocks * a.Hk, di, dr, dt, dc)
  if (a.units) launch_list(a, round_groups<D, E4M3>(cut), stream);
  for (a.first_workgroup = 0; a.first_workgroup < workgroups; a.first_workgroup += kMost) {
    if (cut.block_rows == 16) {
      if constexpr (E4M3 || D == 64) {   // rows of less than 256 bytes, which may go together
        if (cut.teams == 2) FM_DECODE(1, 2);
        else FM_DECODE(1, 1);
      } else {
        FM_DECODE(1, 1);
      }
    } else {
      if (cut.teams == 2) FM_DECODE(2, 2);
      else FM_DECODE(2, 1);
    }
  }
#undef FM_DECODE
  if (a.plan) launch_join<D, F16>(a, stream);
}

}  // namespace fm

FmDecodeCut fm_decode_cut(int H, int Hk, int T, int d, int B, int together, int cus) {
  FmDecodeCut cut;
  const int R = H / Hk * T;
  cut.block_rows = R <= 16 ? 16 : 32;
  cut.row_blocks = (R + cut.block_rows - 1) / cut.block_rows;
  const int members = cut.row_blocks * Hk;
  cut.teams = members > 1 && (together > 1 || cut.row_blocks > 1) ? 2 : 1;
  cut.workgroups = (members + cut.teams - 1) / cut.teams;
  // Chunks that give every compute unit its two workgroups once (131072 keys 102 us, twice as many chunks 105; 64 sequences of 1536, 8 heads,
  // 76 and 79, ragged ones 23 and 24), but for more sequences than that, whose lengths leave more of them over (128 ragged ones
  // of up to 4096 103 and 95, with 16 heads 197 and 181).  Partial results in 48 MiB, and 256 to a row, which its join goes through
  // in a few steps.
  const long long at_once = std::max(1, 2 * (cus > 0 ? cus : 256) / cut.workgroups), wanted = B <= at_once ? at_once : 2 * at_once;
  const long long bytes = (long long)Hk * R * (d + 2) * 4, room = (48ll << 20) / (2 * bytes);
  cut.chunks = (int)std::max<long long>(1, std::min({wanted, room, 256ll}));
  // A chunk's partial sums cost a join more per query row than a key does: 8 keys to a row at least (64 rows, 16 ragged sequences of up to 8192,
  // 43 us, with 4 and 16 keys 53 and 48), and two steps of the workgroup.
  cut.least = std::max(128, 8 * R) / FM_KEY_GROUP;
  cut.slots = fm_most_slots(cut.chunks, B);
  // A workgroup goes over all lengths in rounds of 64, about 1 us each; the list of units takes a launch of 3 us before them all.  Rounds of all
  // workgroups over their 2 * cus places, without and with the list: 8 heads and 128 / 192 / 1024 / 8192 sequences of up to 40
  // keys (4, 9, 256, 16384) 18.7, 26.5, 187, 6821 us and 17.8, 22.4, 80, 611; of 400 to 1100 keys 81, 111, 541 and 85, 115, 527; a single head,
  // 384 and 512 of up to 200 (4.5, 8) 15.2, 19.3 and 15.9, 16.5; 32 and 64 heads, 64 sequences of up to 200 (4, 8) 36, 61 and 37, 60.
  cut.listed = (B + 63) / 64 * (long long)B * cut.workgroups > 4 * 2ll * (cus > 0 ? cus : 256);
  return cut;
}

int fm_decode_round_groups(int d, bool e4m3, const FmDecodeCut& cut) {
  if (d == 64) return e4m3 ? fm::round_groups<64, true>(cut) : fm::round_groups<64, false>(cut);
  return e4m3 ? fm::round_groups<128, true>(cut) : fm::round_groups<128, false>(cut);
}

template <class Args>
static hipError_t launch_decode(const Args& a, bool f16, bool e4m3, hipStream_t stream) {
  if (a.d == 64) {
    if (f16) e4m3 ? fm::launch<64, true, true>(a, stream) : fm::launch<64, true, false>(a, stream);
    else e4m3 ? fm::launch<64, false, true>(a, stream) : fm::launch<64, false, false>(a, stream);
  } else {
    if (f16) e4m3 ? fm::launch<128, true, true>(a, stream) : fm::launch<128, true, false>(a, stream);
    else e4m3 ? fm::launch<128, false, true>(a, stream) : fm::launch<128, false, false>(a, stream);
  }
  return hipGetLastError();
}
hipError_t fm_launch_decode(const FmDecodeArgs& a, bool f16, bool e4m3, hipStream_t stream) { return launch_decode(a, f16, e4m3, stream); }
hipError_t fm_launch_decode_tree(const FmTreeArgs& a, bool f16, bool e4m3, hipStream_t stream) { return launch_decode(a, f16, e4m3, stream); }
void fm_launch_decode_list(const FmDecodeArgs& a, int round, hipStream_t stream) { fm::launch_list(a, round, stream); }
void fm_launch_decode_join(const FmDecodeArgs& a, bool f16, hipStream_t stream) {
  if (a.d == 64) f16 ? fm::launch_join<64, true>(a, stream) : fm::launch_join<64, false>(a, stream);
  else f16 ? fm::launch_join<128, true>(a, stream) : fm::launch_join<128, false>(a, stream);
}
