// Which tokens of a cache stay and where they go: eviction of the lightest (flashmask_cache_evict), the accepted path of a tree of
// drafted tokens (flashmask_cache_accept).
#include <algorithm>

#include "fm_common.h"
#include "fm_serving.h"

namespace fm {

// --- eviction --------------------------------------------------------------------------------------------------
// The m heaviest of the tokens between the first and the last ones: the m-th heaviest weight is found digit by digit from histograms of
// the digits of those that agree with it so far, of weights as whole numbers of the same order.  What is heavier stays, and of
// what is as heavy the first ones.
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kDigitBits = 11, kDigits = 1 << kDigitBits;

// Weights in order as whole numbers, 0 and -0 alike, NaN below all others.
__device__ __forceinline__ unsigned ordered(float w) {
  if (w != w) return 0;
  const unsigned x = __builtin_bit_cast(unsigned, w + 0.f);
  return x >> 31 ? ~x : x | 0x80000000u;
}

__global__ __launch_bounds__(kSelectThreads) void select_kernel(FmEvictArgs a) {
  __shared__ unsigned count[kDigits];
  __shared__ int wave_sum[2][kSelectWaves];
  __shared__ unsigned chosen[2];   // digit, how many have a larger one
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.y, h = blockIdx.x;
  const int places = (int)a.page.n * a.columns, len = max(a.lens[b], 0), n = min(len, places);
  const bool evicts = n > a.keep;
  const size_t row = (size_t)b * a.weight_heads + h;
  const float* weights = a.weights + row * a.weight_columns;
  const auto weight = [&](int j) { return j < a.weight_columns ? weights[j] : 0.f; };
  float* weights_out = a.weights_out + row * a.weight_columns;
  int* kept = a.kept + row * a.keep;
  if (h == 0) {
    const int* from = a.table + (size_t)b * a.columns;
    const int* fresh = a.new_table + (size_t)b * a.new_columns;
    const int pages = (int)((a.keep + a.page.n - 1) / a.page.n);
    for (int c = tid; c < a.columns; c += kSelectThreads)
      a.table_out[(size_t)b * a.columns + c] = evicts ? c < pages ? fresh[c] : -1 : from[c];
    if (tid == 0) a.lens_out[b] = evicts ? a.keep : a.lens[b];
  }
  for (int j = (evicts ? a.keep : n) + tid; j < a.weight_columns; j += kSelectThreads) weights_out[j] = 0.f;
  if (!evicts) {
    for (int j = tid; j < a.keep; j += kSelectThreads) kept[j] = j < n ? j : -1;
    for (int j = tid; j < min(n, a.weight_columns); j += kSelectThreads) weights_out[j] = weights[j];
    return;
  }
  const int last = n - a.recent;   // candidates are those of [first, last)
  int wanted = a.keep - a.first - a.recent;
  unsigned prefix = 0, known = 0;
  if (wanted > 0) {
    for (int shift = 32 - kDigitBits, bits = kDigitBits;;) {
      for (int i = tid; i < kDigits; i += kSelectThreads) count[i] = 0;
      __syncthreads();
      for (int j = a.first + tid; j < last; j += kSelectThreads) {
        const unsigned x = ordered(weight(j));
        if ((x & known) == prefix) atomicAdd(&count[x >> shift & ((1u << bits) - 1)], 1u);
      }
      __syncthreads();
      // digits from the largest down, two to a thread
      const int at = kDigits - 2 - 2 * tid;
      const unsigned upper = count[at + 1], lower = count[at], both = upper + lower;
      unsigned upto = both;
#pragma unroll
      for (int k = 1; k < 64; k *= 2) {
        const unsigned other = __shfl_up(upto, k);
        if (lane >= k) upto += other;
      }
      if (lane == 63) wave_sum[0][wave] = (int)upto;
      __syncthreads();
      unsigned larger = upto - both;
      for (int w = 0; w < wave; ++w) larger += wave_sum[0][w];
      if (larger < (unsigned)wanted && (unsigned)wanted <= larger + both) {
        const bool top = (unsigned)wanted <= larger + upper;
        chosen[0] = top ? at + 1 : at;
        chosen[1] = top ? larger : larger + upper;
      }
      __syncthreads();
      prefix |= chosen[0] << shift;
      known |= ((1u << bits) - 1) << shift;
      wanted -= (int)chosen[1];
      if (shift == 0) break;
      bits = std::min(kDigitBits, shift);
      shift -= bits;
      __syncthreads();
    }
  }
  // Now `wanted` of those that equal `prefix` stay, the first ones.  Every wave has a run of places; counts first, then ranks.
  const int all = wanted > 0 ? 1 : 0, run = ((n + kSelectWaves - 1) / kSelectWaves + 63) / 64 * 64, begin = min(wave * run, n), end = min(begin + run, n);
  const auto kind = [&](int j) {   // 2: stays, 1: equals, 0: goes
    if (j < a.first || j >= last) return 2;
    if (!all) return 0;
    const unsigned x = ordered(weight(j));
    return x > prefix ? 2 : x == prefix ? 1 : 0;
  };
  int stay = 0, equal = 0;
  for (int base = begin; base < end; base += 64) {
    const int k = base + lane < end ? kind(base + lane) : 0;
    stay += __popcll(__ballot(k == 2));
    equal += __popcll(__ballot(k == 1));
  }
  if (lane == 0) {
    wave_sum[0][wave] = stay;
    wave_sum[1][wave] = equal;
  }
  __syncthreads();
  int stayed = 0, equals = 0;
  for (int w = 0; w < wave; ++w) {
    stayed += wave_sum[0][w];
    equals += wave_sum[1][w];
  }
  const unsigned long long below = (1ull << lane) - 1ull;
  for (int base = begin; base < end; base += 64) {
    const int j = base + lane, k = j < end ? kind(j) : 0;
    const unsigned long long sure = __ballot(k == 2), even = __ballot(k == 1);
    const int rank = equals + __popcll(even & below), before = min(rank, wanted);
    if (k == 2 || (k == 1 && rank < wanted)) {
      const int to = stayed + __popcll(sure & below) + before;
      kept[to] = j;
      if (to < a.weight_columns) weights_out[to] = weight(j);
    }
    stayed += __popcll(sure);
    equals += __popcll(even);
  }
}

// Rows of the tokens that stay go to their new places, keys and values, 16 bytes a lane.  A token without a page becomes zeros.
constexpr int kGatherTokens = 64;
__global__ __launch_bounds__(256) void gather_kernel(FmEvictArgs a, int pieces) {
  __shared__ long long from[kGatherTokens], to[kGatherTokens];   // page << 32 | slot, -1: none
  const int b = blockIdx.z, h = blockIdx.y, first = blockIdx.x * kGatherTokens;
  const int places = (int)a.page.n * a.columns;
  if (min(max(a.lens[b], 0), places) <= a.keep) return;
  const int count = min(kGatherTokens, a.keep - first);
  const int* kept = a.kept + ((size_t)b * a.weight_heads + (a.weight_heads > 1 ? h : 0)) * a.keep;
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
  for (int i = threadIdx.x; i < count * pieces; i += 256) {
    const int token = i / pieces, piece = i - token * pieces;
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

// --- the accepted path -----------------------------------------------------------------------------------------
// Token path[i] of the drafted ones goes to the place of the i-th.  A path ascends, so path[i] >= i: a lane that moves its 16 bytes of the
// rows one behind the other, all of a batch's loads ahead of its stores, never reads what it has written.
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

hipError_t fm_launch_evict(const FmEvictArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(fm::select_kernel, dim3(a.weight_heads, a.B), dim3(fm::kSelectThreads), 0, stream, a);
  hipLaunchKernelGGL(fm::gather_kernel, dim3((a.keep + fm::kGatherTokens - 1) / fm::kGatherTokens, a.Hk, a.B), dim3(256), 0, stream, a, a.row_bytes / 16);
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
