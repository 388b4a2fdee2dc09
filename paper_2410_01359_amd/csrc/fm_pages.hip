// Pages of the key-value cache: forks of sequences, list of free pages, compaction.
#include <algorithm>

#include "fm_common.h"
#include "fm_serving.h"

namespace fm {

// Bytes of a page that a workgroup moves at a time, two 16-byte loads of a lane in flight.  Copies go past the L2, which has no
// use for them.  256 children of 64 prompts, six layers: 99 us with four loads and ordinary stores, 90 past the L2, 88 with two loads,
// 95 with one.
constexpr int kLoads = 2, kPart = 4096 * kLoads;

__device__ __forceinline__ void copy_part(const char* from, char* to, size_t page_bytes, int part) {
  const size_t at = (size_t)part * kPart + threadIdx.x * 16;
  u32x4 x[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i)
    if (at + i * 4096 < page_bytes) x[i] = ldg16(from + at + i * 4096);
#pragma unroll
  for (int i = 0; i < kLoads; ++i)
    if (at + i * 4096 < page_bytes) __builtin_nontemporal_store(x[i], (u32x4*)(to + at + i * 4096));
}

// Workgroups (x, child): x = 0 writes the child's row (tables == true), the others a part of the last page in a pool each.
__global__ __launch_bounds__(256) void fork_kernel(FmPools pools, int parts, size_t page_bytes, int num_pages,
                                                   const int* __restrict__ table, const int* __restrict__ lens,
                                                   const int* __restrict__ parents, const int* __restrict__ new_pages,
                                                   int* __restrict__ table_out, int* __restrict__ lens_out, int sequences,
                                                   int columns, FmDivisor page, bool tables) {
  const int child = blockIdx.y;
  const int parent = parents[child], fresh = new_pages[child];
  const bool known = parent >= 0 && parent < sequences;
  const int len = known ? lens[parent] : 0;
  const FmFork fork = fm_fork(len, page);
  const int* row = table + (size_t)(known ? parent : 0) * columns;
  int x = blockIdx.x;
  if (tables && x-- == 0) {
    for (int c = threadIdx.x; c < columns; c += 256) {
      table_out[(size_t)child * columns + c] = fm_fork_entry(fork, c, known ? row[c] : -1, fresh);
    }
    if (threadIdx.x == 0) lens_out[child] = len;
    return;
  }
  if (!known || fm_known_page(fresh, num_pages) < 0 || !fork.partly || fork.last >= columns) return;
  const int from = fm_known_page(row[fork.last], num_pages);
  if (from < 0) return;
  char* pool = pools.p[x / parts];
  copy_part(pool + from * page_bytes, pool + fresh * page_bytes, page_bytes, x % parts);
}

// --- which pages are in use -----------------------------------------------------------------------------------
// One workgroup marks the pages that the table names in a bit map, counts the bits in front of each word, and deals every
// page its number among the used or the unused ones.  Map and counts lie in LDS where they fit 32 KiB; a larger map, or one of many words
// with a table that a workgroup alone reads for longer, lies in global memory and is marked by the whole chip first.  us in LDS / global memory:
// 2^17 pages, 2^17 / 2^18 / 2^20 entries 46/51, 66/58, 186/84; 2^16 pages 35/37, 54/48, 169/102; 2^14 pages, where the marks of a word
// wait for each other, 26/40, 45/69, 159/240.
constexpr int kPlanThreads = 1024;
constexpr int kMapPages = 1 << 17;                                // LDS up to these,
constexpr int kMarkedPages = 1 << 16, kMarkedEntries = 1 << 17;   // but from these pages on with more entries than these

struct PlanArgs {
  const int* table;
  int entries, num_pages;
  unsigned *map, *before;   // global memory; NULL: LDS
  int *free_pages, *count;  // list of free pages and its length, or
  int *place, *source, *target, *moves, *used;   // the moves of a compaction
};

__global__ void clear_map_kernel(unsigned* map, int words) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < words; i += gridDim.x * 256) map[i] = 0;
}
__global__ void mark_kernel(const int* __restrict__ table, int entries, int num_pages, unsigned* map) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < entries; i += gridDim.x * 256) {
    const int p = table[i];
    if (fm_known_page(p, num_pages) >= 0) atomicOr(map + p / 32, 1u << (p % 32));
  }
}

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a) {
  extern __shared__ unsigned lds_map[];
  __shared__ int wave_sum[kPlanThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int words = (a.num_pages + 31) / 32;
  unsigned* map = a.map ? a.map : lds_map;
  unsigned* before = a.map ? a.before : lds_map + words;
  if (!a.map) {
    for (int i = tid; i < words; i += kPlanThreads) map[i] = 0;
    __syncthreads();
    constexpr int BATCH = 8;   // loads in flight
    for (int base = 0; base < a.entries; base += BATCH * kPlanThreads) {
      int p[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int at = base + i * kPlanThreads + tid;
        p[i] = at < a.entries ? a.table[at] : -1;
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i)
        if (fm_known_page(p[i], a.num_pages) >= 0) atomicOr(map + p[i] / 32, 1u << (p[i] % 32));
    }
    __syncthreads();
  }
  // used pages in front of each word: every thread adds up a run of words
  const int run = (words + kPlanThreads - 1) / kPlanThreads, w0 = min(tid * run, words), w1 = min(w0 + run, words);
  int sum = 0;
  for (int w = w0; w < w1; ++w) sum += __popc(map[w]);
  int upto = sum;
#pragma unroll
  for (int k = 1; k < 64; k *= 2) {
    const int other = __shfl_up(upto, k);
    if (lane >= k) upto += other;
  }
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  int used = 0, ahead = upto - sum;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) ahead += wave_sum[w];
    used += wave_sum[w];
  }
  for (int w = w0; w < w1; ++w) {
    before[w] = ahead;
    ahead += __popc(map[w]);
  }
  __syncthreads();
  const auto rank = [&](int p) { return (int)before[p / 32] + __popc(map[p / 32] & ((1u << (p % 32)) - 1u)); };
  if (a.free_pages) {
    for (int p = tid; p < a.num_pages; p += kPlanThreads) {
      if (!(map[p / 32] >> (p % 32) & 1)) a.free_pages[p - rank(p)] = p;
      if (p >= a.num_pages - used) a.free_pages[p] = -1;
    }
    if (tid == 0) *a.count = a.num_pages - used;
    return;
  }
  const int kept = used < a.num_pages ? rank(used) : used;   // used pages that stay where they are
  for (int p = tid; p < a.num_pages; p += kPlanThreads) {
    const int r = rank(p);
    const bool in_use = map[p / 32] >> (p % 32) & 1;
    if (in_use && p >= used) {
      a.source[r - kept] = p;
      a.place[p] = -1 - (r - kept);   // the move that takes it
    } else {
      a.place[p] = p;
      if (!in_use && p < used) a.target[p - r] = p;
    }
  }
  if (tid == 0) {
    *a.moves = used - kept;
    *a.used = used;
  }
}

// The moves of a compaction, in every pool: workgroups go through (move, pool, part) with the stride of the launch.  The first launch
// of a call also rewrites the table.
__global__ __launch_bounds__(256) void move_kernel(FmPools pools, int num_pools, int parts, size_t page_bytes, int num_pages,
                                                   const int* __restrict__ moves, const int* __restrict__ source,
                                                   const int* __restrict__ target, const int* __restrict__ place,
                                                   const int* __restrict__ table, int entries, int* __restrict__ table_out) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < entries; i += gridDim.x * 256) {
    int p = table[i];
    if (fm_known_page(p, num_pages) >= 0) {
      const int to = place[p];
      p = to < 0 ? target[-1 - to] : to;
    }
    table_out[i] = p;
  }
  const long long all = (long long)*moves * num_pools * parts;
  for (long long i = blockIdx.x; i < all; i += gridDim.x) {
    const int part = (int)(i % parts), pool = (int)(i / parts % num_pools), m = (int)(i / parts / num_pools);
    char* p = pools.p[pool];
    copy_part(p + source[m] * page_bytes, p + target[m] * page_bytes, page_bytes, part);
  }
}

static size_t words_bytes(int num_pages) { return ((size_t)(num_pages + 31) / 32 * 4 + 255) / 256 * 256; }
static size_t pages_bytes(int num_pages) { return ((size_t)num_pages * 4 + 255) / 256 * 256; }

static hipError_t launch_plan(PlanArgs a, char* workspace, hipStream_t stream) {
  const int words = (a.num_pages + 31) / 32;
  size_t lds = (size_t)words * 8;
  if (a.num_pages > kMapPages || (a.num_pages >= kMarkedPages && a.entries > kMarkedEntries)) {
    a.map = (unsigned*)workspace;
    a.before = (unsigned*)(workspace + words_bytes(a.num_pages));
    lds = 0;
    hipLaunchKernelGGL(clear_map_kernel, dim3(std::min((words + 255) / 256, 1024)), dim3(256), 0, stream, a.map, words);
    hipLaunchKernelGGL(mark_kernel, dim3(std::min((a.entries + 255) / 256, 2048)), dim3(256), 0, stream, a.table, a.entries,
                       a.num_pages, a.map);
  }
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), lds, stream, a);
  return hipGetLastError();
}

// launch(pools, their number, whether they are the call's first) for groups of pools; once where there are none.
template <class Launch>
static void pool_groups(void* const* pools, int num_pools, const Launch& launch) {
  int at = 0;
  do {
    FmPools group = {};
    const int n = std::min(num_pools - at, FM_POOLS);
    for (int i = 0; i < n; ++i) group.p[i] = (char*)pools[at + i];
    launch(group, n, at == 0);
    at += FM_POOLS;
  } while (at < num_pools);
}

}  // namespace fm

size_t fm_plan_bytes(int num_pages) {
  return 2 * fm::words_bytes(num_pages) + 3 * fm::pages_bytes(num_pages) + 256;
}

hipError_t fm_launch_fork(void* const* pools, int num_pools, size_t page_bytes, int num_pages, const int* table,
                          const int* lens, const int* parents, const int* new_pages, int* table_out, int* lens_out,
                          int sequences, int columns, int page, int children, hipStream_t stream) {
  const int parts = (int)((page_bytes + fm::kPart - 1) / fm::kPart);
  fm::pool_groups(pools, num_pools, [&](const FmPools& group, int n, bool first) {
    hipLaunchKernelGGL(fm::fork_kernel, dim3(parts * n + first, children), dim3(256), 0, stream, group, parts, page_bytes,
                       num_pages, table, lens, parents, new_pages, table_out, lens_out, sequences, columns, fm_divisor(page), first);
  });
  return hipGetLastError();
}

hipError_t fm_launch_free_list(const int* table, int entries, int num_pages, int* free_pages, int* count, void* workspace,
                               hipStream_t stream) {
  fm::PlanArgs a = {};
  a.table = table; a.entries = entries; a.num_pages = num_pages;
  a.free_pages = free_pages; a.count = count;
  return fm::launch_plan(a, (char*)workspace, stream);
}

hipError_t fm_launch_compact(void* const* pools, int num_pools, size_t page_bytes, int num_pages, const int* table,
                             int entries, int* table_out, int* used, void* workspace, hipStream_t stream) {
  fm::PlanArgs a = {};
  char* ws = (char*)workspace;
  char* lists = ws + 2 * fm::words_bytes(num_pages);
  const size_t step = fm::pages_bytes(num_pages);
  a.table = table; a.entries = entries; a.num_pages = num_pages;
  a.place = (int*)lists; a.source = (int*)(lists + step); a.target = (int*)(lists + 2 * step); a.moves = (int*)(lists + 3 * step);
  a.used = used;
  if (hipError_t e = fm::launch_plan(a, ws, stream); e != hipSuccess) return e;
  const int parts = (int)((page_bytes + fm::kPart - 1) / fm::kPart);
  fm::pool_groups(pools, num_pools, [&](const FmPools& group, int n, bool first) {
    // At most every second page moves; how many do is known on the device alone.  Many workgroups that take few parts each keep
    // the memory busiest: six layers (a page of 128 KiB) 324, 320, 298 us with 16, 32, 256 to a compute unit; pages of 1 KiB 143, 141, 131 and
    // again 143 with 512.
    const long long most = (long long)(num_pages / 2) * n * parts, rows = first ? (entries + 255) / 256 : 0;
    const int workgroups = (int)std::min<long long>(std::max<long long>(std::max(most, rows), 1), 256ll * fm_compute_units());
    hipLaunchKernelGGL(fm::move_kernel, dim3(workgroups), dim3(256), 0, stream, group, n, parts, page_bytes, num_pages, a.moves,
                       a.source, a.target, a.place, table, first ? entries : 0, table_out);
  });
  return hipGetLastError();
}
