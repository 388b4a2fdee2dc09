// Which tokens of a cache stay and where they go: eviction of the lightest (flashmask_cache_evict), the accepted path of a tree of
// drafted tokens (flashmask_cache_accept).
#include <algorithm>

#include "fm_common.h"
#include "fm_serving.h"

namespace fm {

// --- eviction --------------------------------------------------------------------------------------------------
// The m heaviest of the tokens between the first and the last ones: the m-th heaviest weight is found digit by digit (11, 11, 10 bits) from
// histograms of the digits of those that agree with it so far, of weights as whole numbers of the same order.  What is heavier
// stays, and of what is as heavy the first ones.  A workgroup takes 8192 places at a time, eight to a thread with their loads in flight together; a row
// of no more stays in registers.  A chain of steps between barriers: 384 rows of up to 6000 take 14 us, one of 300 11 (digits counted in four banks by
// lane: 15).
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kEach = 8, kChunk = kSelectThreads * kEach;
constexpr int kDigitBits = 11, kDigits = 1 << kDigitBits, kStages = 3;
__device__ __forceinline__ int digit_shift(int stage) { return stage == 0 ? 21 : stage == 1 ? 10 : 0; }

// Weights in order as whole numbers, 0 and -0 alike, NaN below all others.
__device__ __forceinline__ unsigned ordered(float w) {
  if (w != w) return 0;
  const unsigned x = __builtin_bit_cast(unsigned, w + 0.f);
  return x >> 31 ? ~x : x | 0x80000000u;
}

// A row of weights: its tokens, the candidates [first, last), how many of them stay.
struct Row {
  const float* weights;
  float* weights_out;
  int* kept;
  int n, first, last, wanted, columns, keep;
  bool evicts;
  __device__ __forceinline__ Row(const FmEvictArgs& a, int b, int h) {
    n = min(max(a.lens[b], 0), (int)a.page.n * a.columns);
    evicts = n > a.keep;
    const size_t row = (size_t)b * a.weight_heads + h;
    columns = a.weight_columns;
    keep = a.keep;
    weights = a.weights + row * columns;
    weights_out = a.weights_out + row * columns;
    kept = a.kept + row * keep;
    first = a.first;
    last = n - a.recent;
    wanted = a.keep - a.first - a.recent;
  }
  // of places base + 1024 i + thread, 0 from `end` on and where there is no weight
  __device__ __forceinline__ void load(float (&w)[kEach], int base, int end) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int j = base + i * kSelectThreads + (int)threadIdx.x;
      w[i] = j < end && j < columns ? weights[j] : 0.f;
    }
  }
};
struct SelectShared {
  unsigned count[kDigits], chosen[2];
  int wave_sum[kSelectWaves], ranks[kEach * kSelectWaves], total;
};

__device__ __forceinline__ void clear(SelectShared& sh) {
#pragma unroll
  for (int i = 0; i < kDigits / kSelectThreads; ++i) sh.count[i * kSelectThreads + threadIdx.x] = 0;
  __syncthreads();
}
// Counts the digits of the candidates of [base, end) that agree with `prefix` so far.
__device__ __forceinline__ void count_digits(SelectShared& sh, const Row& row, const float (&w)[kEach], int base, int end, int stage, unsigned prefix) {
  const int shift = digit_shift(stage);
  const unsigned known = stage == 0 ? 0u : ~0u << digit_shift(stage - 1), mask = stage == 2 ? 1023u : 2047u;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int j = base + i * kSelectThreads + (int)threadIdx.x;
    const unsigned x = ordered(w[i]);
    if (j >= row.first && j < min(row.last, end) && (x & known) == prefix) atomicAdd(&sh.count[x >> shift & mask], 1u);
  }
}
// The digit of the `wanted`-th largest of what was counted, and how many have a larger one.
__device__ __forceinline__ void pick(SelectShared& sh, unsigned wanted, unsigned& digit, unsigned& larger) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // digits from the largest down, two to a thread
  const int at = kDigits - 2 - 2 * tid;
  const unsigned upper = sh.count[at + 1], lower = sh.count[at], both = upper + lower;
  unsigned upto = both;
#pragma unroll
  for (int k = 1; k < 64; k *= 2) {
    const unsigned other = __shfl_up(upto, k);
    if (lane >= k) upto += other;
  }
  if (lane == 63) sh.wave_sum[wave] = (int)upto;
  __syncthreads();
  unsigned ahead = upto - both;
#pragma unroll
  for (int w = 0; w < kSelectWaves; ++w) ahead += w < wave ? sh.wave_sum[w] : 0;
  if (ahead < wanted && wanted <= ahead + both) {
    const bool top = wanted <= ahead + upper;
    sh.chosen[0] = top ? at + 1 : at;
    sh.chosen[1] = top ? ahead : ahead + upper;
  }
  __syncthreads();
  digit = sh.chosen[0];
  larger = sh.chosen[1];
}
// The sum of all threads' x, in every thread.
__device__ __forceinline__ int sum_of_all(SelectShared& sh, int x) {
#pragma unroll
  for (int k = 1; k < 64; k *= 2) x += __shfl_xor(x, k);
  __syncthreads();   // what was there has been read
  if ((threadIdx.x & 63) == 0) sh.wave_sum[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int w = 0; w < kSelectWaves; ++w) x += sh.wave_sum[w];
  return x;
}
// Writes what stays of [base, end), at most 8192 places: all that is heavier than `limit`, and the first `equal` of all that are as heavy.
// stayed, equals: of the places before.
__device__ __forceinline__ void keep_places(SelectShared& sh, const Row& row, const float (&w)[kEach], int base, int end, unsigned limit, int equal,
                                            int& stayed, int& equals) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const unsigned long long below = (1ull << lane) - 1ull;
  int kind[kEach], rank[kEach];   // kind 2: stays, 1: as heavy as the limit, 0: goes; rank among the wave's lanes: stays | as heavy << 16
  __syncthreads();   // the ranks before have been read
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int j = base + i * kSelectThreads + tid;
    const unsigned x = ordered(w[i]);
    kind[i] = j >= end ? 0 : j < row.first || j >= row.last ? 2 : row.wanted == 0 ? 0 : x > limit ? 2 : x == limit ? 1 : 0;
    const unsigned long long sure = __ballot(kind[i] == 2), even = __ballot(kind[i] == 1);
    rank[i] = __popcll(sure & below) | __popcll(even & below) << 16;
    if (lane == 0) sh.ranks[i * kSelectWaves + wave] = __popcll(sure) | __popcll(even) << 16;
  }
  __syncthreads();
  if (wave == 0) {   // ahead of each 64: two entries to a lane; sums of at most 8192
    static_assert(kEach * kSelectWaves == 128);
    const int one = sh.ranks[2 * lane], two = sh.ranks[2 * lane + 1];
    int upto = one + two;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
      const int other = __shfl_up(upto, k);
      if (lane >= k) upto += other;
    }
    sh.ranks[2 * lane] = upto - one - two;
    sh.ranks[2 * lane + 1] = upto - two;
    if (lane == 63) sh.total = upto;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = rank[i] + sh.ranks[i * kSelectWaves + wave], even = equals + (at >> 16);
    if (kind[i] == 2 || (kind[i] == 1 && even < equal)) {
      const int to = stayed + (at & 0xffff) + min(even, equal);
      row.kept[to] = base + i * kSelectThreads + tid;
      if (to < row.columns) row.weights_out[to] = w[i];
    }
  }
  stayed += sh.total & 0xffff;
  equals += sh.total >> 16;
}
// What does not depend on the selection, by workgroup `part` of `parts`: the row of the table, the length, what is behind the kept tokens, and
// a row that is not evicted from.
__device__ __forceinline__ void write_rest(const FmEvictArgs& a, const Row& row, int b, int h, int part, int parts) {
  const int at = part * kSelectThreads + threadIdx.x, step = parts * kSelectThreads;
  if (h == 0) {
    const int* from = a.table + (size_t)b * a.columns;
    const int* fresh = a.new_table + (size_t)b * a.new_columns;
    const int pages = (int)((a.keep + a.page.n - 1) / a.page.n);
    for (int c = at; c < a.columns; c += step) a.table_out[(size_t)b * a.columns + c] = row.evicts ? c < pages ? fresh[c] : -1 : from[c];
    if (at == 0) a.lens_out[b] = row.evicts ? a.keep : a.lens[b];
  }
  for (int j = (row.evicts ? row.keep : row.n) + at; j < row.columns; j += step) row.weights_out[j] = 0.f;
  if (row.evicts) return;
  for (int j = at; j < row.keep; j += step) row.kept[j] = j < row.n ? j : -1;
  for (int j = at; j < min(row.n, row.columns); j += step) row.weights_out[j] = row.weights[j];
}

// Rows of the tokens that stay go to their new places, keys and values, 16 bytes a lane.  A token without a page becomes zeros.  Memory: 2048 tokens of 256
// bytes of 8 heads of up to 48 sequences 52 us, 5.9 TB/s.
template <int TOKENS>
struct Moves {
  long long from[TOKENS], to[TOKENS];   // page << 32 | slot, -1: none
  // Of a head's kept tokens [first, first + count), by a workgroup; pieces: of 16 bytes of a row.
  template <int THREADS>
  __device__ __forceinline__ void run(const FmEvictArgs& a, int b, int h, const int* kept, int first, int count, const FmDivisor& pieces) {
    static_assert(TOKENS <= THREADS);
    if ((int)threadIdx.x < count) {
      const auto place = [&](const int* row, int j) {
        const int column = fm_div(j, a.page), page = fm_known_page(row[column], a.num_pages);
        return page < 0 ? -1ll : (long long)page << 32 | (j - column * (int)a.page.n);
      };
      const int i = first + threadIdx.x;
      from[threadIdx.x] = place(a.table + (size_t)b * a.columns, kept[i]);
      to[threadIdx.x] = place(a.new_table + (size_t)b * a.new_columns, i);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < count * (int)pieces.n; i += THREADS) {
      const int token = fm_div(i, pieces), piece = i - token * (int)pieces.n;
      const long long source = from[token], target = to[token];
      if (target < 0) continue;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const FmPages& p = a.cache[w];
        const auto at = [&](long long x) { return p.base + (x >> 32) * p.page + h * p.head + (unsigned)x * (long long)p.token + piece * 16; };
        u32x4 v = {0, 0, 0, 0};
        if (source >= 0) v = ldg16(at(source));
        *(u32x4*)at(target) = v;
      }
    }
  }
};

// One workgroup to a row.  MOVE: it moves the tokens that stay, too, of its one head, one to a thread at most.
template <bool MOVE>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(FmEvictArgs a, FmDivisor pieces) {
  __shared__ SelectShared sh;
  __shared__ Moves<MOVE ? kSelectThreads : 1> moves;
  const int b = blockIdx.y, h = blockIdx.x;
  const Row row(a, b, h);
  float w[kEach];
  if (row.evicts) row.load(w, 0, row.n);
  write_rest(a, row, b, h, 0, 1);
  if (!row.evicts) return;
  unsigned prefix = 0, wanted = row.wanted;
  for (int stage = 0; stage < kStages && wanted > 0; ++stage) {
    clear(sh);
    for (int base = 0; base < row.n; base += kChunk) {
      if (row.n > kChunk) row.load(w, base, row.n);
      count_digits(sh, row, w, base, row.n, stage, prefix);
    }
    __syncthreads();
    unsigned digit, larger;
    pick(sh, wanted, digit, larger);
    prefix |= digit << digit_shift(stage);
    wanted -= larger;
  }
  int stayed = 0, equals = 0;
  for (int base = 0; base < row.n; base += kChunk) {
    if (row.n > kChunk) row.load(w, base, row.n);
    keep_places(sh, row, w, base, row.n, prefix, (int)wanted, stayed, equals);
  }
  if constexpr (MOVE) {
    __syncthreads();   // the list is there
    moves.template run<kSelectThreads>(a, b, h, row.kept, 0, row.keep, pieces);
  }
}

// Sixteen workgroups to a row, each with a run of its places, and a launch for each digit and one that writes: a launch finds the digit that the one
// before counted from the sum of the runs' histograms.  One row of 131072 tokens: 29 us, by one workgroup 196.
struct SplitState {
  unsigned prefix, wanted;
};
struct SplitSpace {   // of a row, in words
  static constexpr int kHeavier = kStages * FM_EVICT_PARTS * kDigits;   // behind the histograms [stage][part][digit]; [stage][part] of the part's candidates
  static constexpr int kState = kHeavier + kStages * FM_EVICT_PARTS;    // [stage]
  static constexpr int kWords = (kState + kStages * 2 + 63) / 64 * 64;
};
template <int STAGE>
__global__ __launch_bounds__(kSelectThreads) void split_kernel(FmEvictArgs a) {
  __shared__ SelectShared sh;
  const int b = blockIdx.z, h = blockIdx.y, part = blockIdx.x, tid = threadIdx.x;
  const Row row(a, b, h);
  if (STAGE == 0) write_rest(a, row, b, h, part, FM_EVICT_PARTS);
  if (!row.evicts) return;
  unsigned* space = a.scratch + ((size_t)b * a.weight_heads + h) * SplitSpace::kWords;
  const auto histogram = [&](int stage, int p) { return space + (stage * FM_EVICT_PARTS + p) * kDigits; };
  unsigned* heavier = space + SplitSpace::kHeavier;
  SplitState* states = (SplitState*)(space + SplitSpace::kState);
  const int run = (row.n + FM_EVICT_PARTS * kSelectThreads - 1) / (FM_EVICT_PARTS * kSelectThreads) * kSelectThreads;
  const int begin = (int)std::min<long long>((long long)part * run, row.n), end = (int)std::min<long long>((long long)begin + run, row.n);
  float w[kEach];
  row.load(w, begin, end);

  SplitState now = {0u, (unsigned)row.wanted};
  int stayed = std::min(begin, row.first) + std::max(begin - row.last, 0), equals = 0;   // ahead of the run (the last stage)
  if (STAGE > 0 && row.wanted > 0) {
    if (STAGE > 1) now = states[STAGE - 2];
    unsigned own[kDigits / kSelectThreads];
#pragma unroll
    for (int i = 0; i < kDigits / kSelectThreads; ++i) {
      const int d = i * kSelectThreads + tid;
      unsigned sum = 0;
#pragma unroll
      for (int p = 0; p < FM_EVICT_PARTS; ++p) sum += histogram(STAGE - 1, p)[d];
      sh.count[d] = sum;
      own[i] = histogram(STAGE - 1, part)[d];
    }
    __syncthreads();
    unsigned digit, larger;
    pick(sh, now.wanted, digit, larger);
    now.prefix |= digit << digit_shift(STAGE - 1);
    now.wanted -= larger;
    if constexpr (STAGE < kStages) {
      int mine = 0;
#pragma unroll
      for (int i = 0; i < kDigits / kSelectThreads; ++i) mine += i * kSelectThreads + tid > (int)digit ? own[i] : 0;
      mine = sum_of_all(sh, mine);
      if (tid == 0) heavier[(STAGE - 1) * FM_EVICT_PARTS + part] = mine;
      if (part == 0 && tid == 0) states[STAGE - 1] = now;
    } else {
      int ahead = 0, even = 0;
#pragma unroll
      for (int i = 0; i < kDigits / kSelectThreads; ++i) {
        const int d = i * kSelectThreads + tid;
        int before = 0;
#pragma unroll
        for (int p = 0; p < FM_EVICT_PARTS; ++p) before += p < part ? histogram(STAGE - 1, p)[d] : 0;
        if (d > (int)digit) ahead += before;
        if (d == (int)digit) even += before;
      }
      if (tid < 2 * FM_EVICT_PARTS && tid % FM_EVICT_PARTS < part) ahead += heavier[tid];
      stayed += sum_of_all(sh, ahead);
      equals = sum_of_all(sh, even);
    }
  }
  if constexpr (STAGE < kStages) {
    __syncthreads();
    clear(sh);
    for (int base = begin; base < end; base += kChunk) {
      if (base > begin) row.load(w, base, end);
      count_digits(sh, row, w, base, end, STAGE, now.prefix);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kDigits / kSelectThreads; ++i) histogram(STAGE, part)[i * kSelectThreads + tid] = sh.count[i * kSelectThreads + tid];
  } else {
    for (int base = begin; base < end; base += kChunk) {
      if (base > begin) row.load(w, base, end);
      keep_places(sh, row, w, base, end, now.prefix, (int)now.wanted, stayed, equals);
    }
  }
}

constexpr int kGatherTokens = 64;
__global__ __launch_bounds__(256) void gather_kernel(FmEvictArgs a, FmDivisor pieces) {
  __shared__ Moves<kGatherTokens> moves;
  const int b = blockIdx.z, h = blockIdx.y, first = blockIdx.x * kGatherTokens;
  const int places = (int)a.page.n * a.columns;
  if (min(max(a.lens[b], 0), places) <= a.keep) return;
  const int* kept = a.kept + ((size_t)b * a.weight_heads + (a.weight_heads > 1 ? h : 0)) * a.keep;
  moves.run<256>(a, b, h, kept, first, min(kGatherTokens, a.keep - first), pieces);
}

// --- the accepted path -----------------------------------------------------------------------------------------
// Token path[i] of the drafted ones goes to the place of the i-th.  A path ascends, so path[i] >= i: a lane that moves its 16 bytes of the
// rows one behind the other, all of a batch's loads ahead of its stores, never reads what it has written.  128 sequences, 24 pools: 6.7 us, a chain of four loads.
constexpr int kBatch = 8;
__global__ __launch_bounds__(256) void accept_kernel(FmPools pools, FmAcceptArgs a, bool first_launch) {
  __shared__ int line[FM_MOST_NEW_TOKENS], count;
  __shared__ long long from[FM_MOST_NEW_TOKENS], to[FM_MOST_NEW_TOKENS];   // bytes from the pool's begin, -1: none
  const int tid = threadIdx.x, b = blockIdx.y, len = a.lens[b], start = len - a.T;
  const bool drafted = len >= a.T;
  if (tid == 0) count = a.path_columns;
  int t = -1;
  if (tid < a.path_columns) line[tid] = t = a.path[(size_t)b * a.path_columns + tid];
  __syncthreads();
  if (tid < a.path_columns && !(t >= 0 && t < a.T && (tid == 0 || t > line[tid - 1]))) atomicMin(&count, tid);
  const auto offset = [&](int j) {
    const FmPlace p = fm_place(j, a.page, a.columns);
    const int page = p.column < 0 ? -1 : fm_known_page(a.table[(size_t)b * a.columns + p.column], a.num_pages);
    return page < 0 ? -1ll : page * a.page_bytes + p.slot * (long long)a.token_bytes;
  };
  if (tid < a.path_columns && drafted && t >= 0 && t < a.T) {
    from[tid] = offset(start + t);
    to[tid] = t == tid ? -1 : offset(start + tid);
  }
  __syncthreads();
  const int n = drafted ? count : 0;
  if (first_launch && blockIdx.x == 0 && blockIdx.z == 0 && tid == 0) a.lens_out[b] = drafted ? start + n : len;
  const int pieces = a.row_bytes / 16, item = blockIdx.x * 256 + tid;
  if (item >= a.heads * pieces) return;
  const int head = item / pieces;
  char* base = pools.p[blockIdx.z] + head * a.head_bytes + (item - head * pieces) * 16;
  for (int i = 0; i < n; i += kBatch) {
    u32x4 x[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      x[k] = u32x4{0, 0, 0, 0};
      if (i + k < n && to[i + k] >= 0 && from[i + k] >= 0) x[k] = ldg16(base + from[i + k]);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (i + k < n && to[i + k] >= 0) *(u32x4*)(base + to[i + k]) = x[k];
  }
}

}  // namespace fm

size_t fm_evict_bytes(int sequences, int weight_heads, int weight_columns) {
  const long long rows = (long long)sequences * weight_heads;
  // Split rows pay four launches of 4 us; whole ones 8 us for every 8192 places, 256 rows at a time.
  return weight_columns > 2 * fm::kChunk && rows <= 128 ? rows * fm::SplitSpace::kWords * sizeof(unsigned) : 0;
}

hipError_t fm_launch_evict(const FmEvictArgs& a, hipStream_t stream) {
  const FmDivisor pieces = fm_divisor(a.row_bytes / 16);
  if (fm_evict_bytes(a.B, a.weight_heads, a.weight_columns)) {
    const dim3 grid(FM_EVICT_PARTS, a.weight_heads, a.B), threads(fm::kSelectThreads);
    hipLaunchKernelGGL(fm::split_kernel<0>, grid, threads, 0, stream, a);
    hipLaunchKernelGGL(fm::split_kernel<1>, grid, threads, 0, stream, a);
    hipLaunchKernelGGL(fm::split_kernel<2>, grid, threads, 0, stream, a);
    hipLaunchKernelGGL(fm::split_kernel<3>, grid, threads, 0, stream, a);
  } else {
    // A launch less, and no more workgroups than rows: up to 64 KiB of keys to a row.  One launch / two, us: 4 heads of 100 tokens of 128 bytes 13.7 / 16.0, 32 of 250
    // of 256 bytes 14.9 / 16.7, of 500 17.1 / 16.4, of 1000 25 / 18.
    static_assert((64 << 10) / 64 <= fm::kSelectThreads);   // rows have 64 bytes at least
    const bool move = a.weight_heads == a.Hk && (long long)a.keep * a.row_bytes <= 64 << 10;
    hipLaunchKernelGGL(move ? fm::select_kernel<true> : fm::select_kernel<false>, dim3(a.weight_heads, a.B), dim3(fm::kSelectThreads), 0, stream, a, pieces);
    if (move) return hipGetLastError();
  }
  hipLaunchKernelGGL(fm::gather_kernel, dim3((a.keep + fm::kGatherTokens - 1) / fm::kGatherTokens, a.Hk, a.B), dim3(256), 0, stream, a, pieces);
  return hipGetLastError();
}

hipError_t fm_launch_accept(void* const* pools, int num_pools, const FmAcceptArgs& a, hipStream_t stream) {
  const int blocks = (a.heads * (a.row_bytes / 16) + 255) / 256;
  for (int at = 0; at < num_pools; at += FM_POOLS) {
    FmPools group = {};
    const int n = std::min(num_pools - at, FM_POOLS);
    for (int i = 0; i < n; ++i) group.p[i] = (char*)pools[at + i];
    hipLaunchKernelGGL(fm::accept_kernel, dim3(blocks, a.B, n), dim3(256), 0, stream, group, a, at == 0);
  }
  return hipGetLastError();
}
