// Launchers of the kernels around the attention call: rotary positions, the paged cache, attention over it (internal).
#pragma once
#include "fm_cache_index.h"
#include "fm_kernels.h"

// Keeps the text of a HIP error for flashmask_last_hip_error; returns FM_ERR_HIP.
int fm_hip_error(hipError_t e);

constexpr int FM_MOST_HEADS = 16384;
constexpr int FM_MOST_NEW_TOKENS = 256;   // of a sequence in flashmask_decode

// q, k [B, heads, N, d] -> q_out, k_out; strides in elements, in this order.
struct FmRopeArgs {
  const void* in[2];
  void* out[2];
  FmStride si[2], so[2];
  const double* freqs;
  const int* positions;   // NULL: 0 .. N - 1
  double amp;
  int B, heads[2], N, d, rot;
  int span, group;        // tokens and heads of a workgroup
  FmDivisor rows;         // N
};
hipError_t fm_launch_rope(FmRopeArgs a, int type, bool interleaved, bool backward, hipStream_t stream);

// Strides in bytes.
struct FmPages {
  char* base;
  long long page, head;
  unsigned token;
};

struct FmAppendArgs {
  const void* in[3];      // q, k, v; strides in elements
  FmStride si[3];
  void* q_out;
  FmStride so;
  FmPages cache[2];       // k, v
  const float* scale[2];
  const int *table, *seqs, *positions;
  const double* freqs;
  double amp;
  int tokens, heads[3], d, rot, sequences, columns, num_pages;
  int span, group;        // tokens and heads of a workgroup
  FmDivisor page;
};
hipError_t fm_launch_append(FmAppendArgs a, bool f16, bool e4m3, bool interleaved, hipStream_t stream);

// How a call is cut for `cus` compute units.
struct FmDecodeCut {
  int row_blocks, block_rows;   // of the H / Hk * T query rows that share a K/V head
  int teams, workgroups;        // heads and row blocks that a workgroup takes, workgroups to a chunk of keys
  int chunks, slots;            // that all keys of a head are meant to be cut into; partial results of a head at most
  int least;                    // groups of keys of a chunk at least
  bool listed;                  // whether a launch of its own lists the chunks of split calls
};
// together: heads, 1 or 2, whose rows of a token make up a run of memory that is best read together.
FmDecodeCut fm_decode_cut(int H, int Hk, int T, int d, int B, int together, int cus);
// Groups of 16 keys that the waves of a team take in one step.
int fm_decode_round_groups(int d, bool e4m3, const FmDecodeCut& cut);
struct FmDecodeArgs {
  const void* q;
  void* out;
  float* lse;
  FmStride sq, so;        // elements
  FmPages k, v;
  const float *k_scale, *v_scale;
  const int *table, *lens;
  const int* bounds[4];   // all or none
  float scale;
  int B, H, Hk, T, d, columns, num_pages, page_tokens, bound_columns, window;
  FmDivisor page;
  // scratch of split sequences: {first slot, chunks} of a sequence; per slot and K/V head the rows' sums of p v, and {max, sum of p}
  int2* plan;
  int4* units;            // (cut.listed) {sequence, length, chunk | chunks << 16, first slot}, sequence = -1: none
  int* split;             // and the split sequences, -1 behind them
  float* part;
  float2* stat;
  FmDecodeCut cut;
  int first_workgroup;    // of the launch
};
hipError_t fm_launch_decode(const FmDecodeArgs& a, bool f16, bool e4m3, hipStream_t stream);

// Attention over a cache and a tree of drafted tokens.
struct FmTreeArgs : FmDecodeArgs {
  const int* parents;     // [B, T]
};
hipError_t fm_launch_decode_tree(const FmTreeArgs& a, bool f16, bool e4m3, hipStream_t stream);
// Trees of many query rows to a K/V head (fm_tree_is_wide) go through a kernel of their own, cut by fm_tree_cut in multiples of FM_TREE_ROUND groups of keys.
constexpr int FM_TREE_ROUND = 4;
FmDecodeCut fm_tree_cut(int H, int Hk, int T, int d, int B, int cus);
hipError_t fm_launch_tree_wide(const FmTreeArgs& a, bool f16, bool e4m3, hipStream_t stream);
// What split calls launch before and behind their loop: the list of chunks, cut in multiples of `round` groups, where there is one, and the join.
void fm_launch_decode_list(const FmDecodeArgs& a, int round, hipStream_t stream);
void fm_launch_decode_join(const FmDecodeArgs& a, bool f16, hipStream_t stream);

// How a call on a prompt is cut: row tiles of a head, blocks of keys, parts that the tiles of a block and a group's heads are cut into.
struct FmWeightsCut {
  int row_tiles, key_blocks, parts;
};
FmWeightsCut fm_weights_cut(int B, int H, int Hk, int N, int first_row, int cus);
struct FmWeightsArgs {
  const void *q, *k;
  const float* lse;
  const int* bounds[4];
  float* part;            // [parts, B, Hk, N]
  FmStride sq, sk;        // elements
  float scale;
  int B, H, Hk, N, d, first_row;
  int row_tiles, parts;
  FmDivisor slices, by_part, by_head;
};
// a.part: scratch where there are several parts.
hipError_t fm_launch_weights(FmWeightsArgs a, float* weights, const FmWeightsCut& cut, hipStream_t stream);

struct FmCacheWeightsArgs {
  const void* q;
  const float* lse;       // [B, H, T]
  FmStride sq;            // elements
  FmPages k;
  const float* k_scale;
  const int *table, *lens;
  const int* bounds[4];
  const float* before;    // [B, Hk, weight_columns], NULL: 0
  float* weights;
  float scale, decay;
  int B, H, Hk, T, d, columns, num_pages, bound_columns, window, weight_columns;
  int places;             // that have a page and a weight
  FmDivisor page, tokens, by_head;   // tokens of a page, T, Hk
  bool dealt;             // all sequences' keys into `chunks` pieces, by their lengths; else each sequence's places into `chunks` of chunk_keys
  FmDivisor chunks;
  int chunk_keys;
};
// Cuts a call's work for `cus` compute units; false: too many workgroups.
bool fm_cut_cache_weights(FmCacheWeightsArgs& a, int cus);
hipError_t fm_launch_cache_weights(const FmCacheWeightsArgs& a, bool f16, bool e4m3, hipStream_t stream);

constexpr int FM_EVICT_PARTS = 16;   // workgroups that a long row is split over
struct FmEvictArgs {
  FmPages cache[2];       // k, v
  const int *table, *lens, *new_table;
  const float* weights;   // [B, weight_heads, weight_columns]
  float* weights_out;
  int *kept, *table_out, *lens_out;   // kept [B, weight_heads, keep]
  unsigned* scratch;
  int B, Hk, weight_heads, weight_columns, keep, first, recent, columns, new_columns, num_pages, row_bytes;
  FmDivisor page;
};
// Scratch, 0 where no row is split.
size_t fm_evict_bytes(int sequences, int weight_heads, int weight_columns);
hipError_t fm_launch_evict(const FmEvictArgs& a, hipStream_t stream);

// Strides in bytes; pools go by their numbers.
struct FmAcceptArgs {
  long long page_bytes, head_bytes;
  unsigned token_bytes;
  int heads, row_bytes, num_pages;
  const int *table, *lens, *path;
  int* lens_out;
  int B, columns, T, path_columns;
  FmDivisor page;
};
hipError_t fm_launch_accept(void* const* pools, int num_pools, const FmAcceptArgs& a, hipStream_t stream);

constexpr int FM_POOLS = 64;   // pools of one launch
struct FmPools {
  char* p[FM_POOLS];
};
hipError_t fm_launch_fork(void* const* pools, int num_pools, size_t page_bytes, int num_pages, const int* table,
                          const int* lens, const int* parents, const int* new_pages, int* table_out, int* lens_out,
                          int sequences, int columns, int page, int children, hipStream_t stream);
// Scratch of the two below.
size_t fm_plan_bytes(int num_pages);
hipError_t fm_launch_free_list(const int* table, int entries, int num_pages, int* free_pages, int* count, void* workspace,
                               hipStream_t stream);
hipError_t fm_launch_compact(void* const* pools, int num_pools, size_t page_bytes, int num_pages, const int* table,
                             int entries, int* table_out, int* used, void* workspace, hipStream_t stream);
