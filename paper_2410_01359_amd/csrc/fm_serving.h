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
