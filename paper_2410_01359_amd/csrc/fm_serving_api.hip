// C ABI of the entry points around the attention call: argument validation, scratch, launches.
#include <algorithm>

#include "../../include/flashmask.h"
#include "fm_serving.h"

namespace {

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline bool bad_workspace(const void* p, size_t bytes, size_t need) {
  return !p || bytes < need || (reinterpret_cast<uintptr_t>(p) & 255u);
}
inline int element_bytes(int type) { return type == FM_TYPE_F32 ? 4 : type == FM_TYPE_E4M3 ? 1 : 2; }
FmStride to_kernel(const flashmask_strides& s) { return FmStride{s.batch, s.head, s.row}; }
int done(hipError_t e) { return e == hipSuccess ? FM_OK : fm_hip_error(e); }

// Strides of rows of `d` elements: 16-byte pieces stay aligned, offsets of a few rows fit 32 bits.  An axis of size 1 may have any stride.
int check_strides(const flashmask_strides& s, int type, long long batches, int heads, long long rows, int d) {
  const int unit = 16 / element_bytes(type);
  if ((batches > 1 && s.batch % unit) || (heads > 1 && s.head % unit) || (rows > 1 && s.row % unit)) return FM_ERR_ALIGN;
  if ((batches > 1 && s.batch <= 0) || (heads > 1 && s.head <= 0) || (rows > 1 && (s.row < d || s.row >= (1 << 24)))) return FM_ERR_SHAPE;
  return FM_OK;
}
bool bad_head_dim(int d) { return d != 64 && d != 128; }

// The parts of rope and append that are alike.
int check_rotation(int layout, double amp, int d, int rot) {
  if (layout != FM_ROPE_HALF && layout != FM_ROPE_INTERLEAVED) return FM_ERR_ARG;
  if (!(amp > -3.0e38) || !(amp < 3.0e38)) return FM_ERR_ARG;
  return rot <= 0 || rot > d || rot % 16 ? FM_ERR_SHAPE : FM_OK;
}

int rope(const void* q, const void* k, void* q_out, void* k_out, const double* freqs, const int32_t* positions, int type, int layout,
         double amp, int B, int H, int Hk, int N, int d, int rot, const flashmask_strides* strides, bool backward, void* hip_stream) {
  if (!q || !k || !q_out || !k_out || !freqs || !strides) return FM_ERR_NULL;
  if (type != FM_TYPE_BF16 && type != FM_TYPE_F16 && type != FM_TYPE_F32) return FM_ERR_ARG;
  if (B <= 0 || H <= 0 || Hk <= 0 || N <= 0 || bad_head_dim(d) || H > FM_MOST_HEADS || Hk > FM_MOST_HEADS) return FM_ERR_SHAPE;
  if ((long long)B * N > (1ll << 31) / 16 - 256) return FM_ERR_SHAPE;
  if (int rc = check_rotation(layout, amp, d, rot)) return rc;
  for (int t = 0; t < 4; ++t)
    if (int rc = check_strides(strides[t], type, B, t % 2 ? Hk : H, N, d)) return rc;
  if (misaligned(q) || misaligned(k) || misaligned(q_out) || misaligned(k_out)) return FM_ERR_ALIGN;
  FmRopeArgs a;
  a.in[0] = q; a.in[1] = k; a.out[0] = q_out; a.out[1] = k_out;
  for (int t = 0; t < 2; ++t) { a.si[t] = to_kernel(strides[t]); a.so[t] = to_kernel(strides[2 + t]); }
  a.freqs = freqs; a.positions = positions; a.amp = amp;
  a.B = B; a.heads[0] = H; a.heads[1] = Hk; a.N = N; a.d = d; a.rot = rot;
  a.rows = fm_divisor(N);
  return done(fm_launch_rope(a, type, layout == FM_ROPE_INTERLEAVED, backward, (hipStream_t)hip_stream));
}

int check_cache(const flashmask_cache* c) {
  if (!c || !c->k || !c->v || !c->table) return FM_ERR_NULL;
  if (c->type != FM_TYPE_BF16 && c->type != FM_TYPE_F16 && c->type != FM_TYPE_E4M3) return FM_ERR_ARG;
  if ((c->type == FM_TYPE_E4M3) != (c->k_scale != nullptr) || (c->type == FM_TYPE_E4M3) != (c->v_scale != nullptr)) return FM_ERR_NULL;
  if (c->heads <= 0 || c->heads > FM_MOST_HEADS || bad_head_dim(c->d) || c->num_pages <= 0 || c->page <= 0 || c->page % 16 || c->page > (1 << 20) ||
      c->sequences <= 0 || c->columns <= 0 || (long long)c->columns * c->page > (1 << 30))
    return FM_ERR_SHAPE;
  for (const flashmask_strides* s : {&c->sk, &c->sv})
    if (int rc = check_strides(*s, c->type, c->num_pages, c->heads, c->page, c->d)) return rc;
  return misaligned(c->k) || misaligned(c->v) ? FM_ERR_ALIGN : FM_OK;
}
FmPages pages(void* base, const flashmask_strides& s, int type) {
  const int bytes = element_bytes(type);
  return FmPages{(char*)base, s.batch * bytes, s.head * bytes, (unsigned)(s.row * bytes)};
}
// Rows of `type` go with the cache.
int check_row_type(int type, const flashmask_cache& c) {
  if (type != FM_TYPE_BF16 && type != FM_TYPE_F16) return FM_ERR_ARG;
  return c.type == FM_TYPE_E4M3 || c.type == type ? FM_OK : FM_ERR_ARG;
}

// How calls of a shape are cut whose workgroups take one head, and two together; the cache decides which.
struct DecodeCuts {
  FmDecodeCut of[2];
};
// Shapes that flashmask_decode's indexing and its launches have room for, whatever the cache: of workgroups that take two heads together where
// there are several; those that take one are up to twice as many.
int check_decode_shape(int sequences, int H, int Hk, int T, int d, DecodeCuts& cuts) {
  if (sequences <= 0 || H <= 0 || H > FM_MOST_HEADS || Hk <= 0 || H % Hk || T <= 0 || T > FM_MOST_NEW_TOKENS || bad_head_dim(d)) return FM_ERR_SHAPE;
  if ((long long)H * T > (1 << 24) || sequences > 65535 || (long long)H * T * sequences > (1ll << 30)) return FM_ERR_SHAPE;
  for (int i = 0; i < 2; ++i) cuts.of[i] = fm_decode_cut(H, Hk, T, d, sequences, 1 + i, fm_compute_units());
  if ((fm_most_units(cuts.of[1].chunks, sequences) + 8ll) * cuts.of[1].workgroups >= 1 << 24) return FM_ERR_SHAPE;
  return FM_OK;
}
struct DecodeSpace {
  size_t units, split, stat, part, total;   // behind the plan, which comes first
};
DecodeSpace decode_space(const FmDecodeCut& cut, int sequences, int H, int T, int d) {
  const size_t rows = (size_t)cut.slots * H * T;
  DecodeSpace s;
  s.units = ((size_t)sequences * sizeof(int2) + 255) / 256 * 256;
  s.split = s.units + (cut.listed ? (size_t)fm_listed_units(cut.chunks, sequences) * sizeof(int4) : 0);
  s.stat = (s.split + (cut.listed ? (size_t)fm_most_splits(cut.chunks, sequences) * sizeof(int) : 0) + 255) / 256 * 256;
  s.part = (s.stat + rows * sizeof(float2) + 255) / 256 * 256;
  s.total = s.part + rows * d * sizeof(float);
  return s;
}
// Of whatever cache.
size_t decode_bytes(const DecodeCuts& cuts, int sequences, int H, int T, int d) {
  return std::max(decode_space(cuts.of[0], sequences, H, T, d).total, decode_space(cuts.of[1], sequences, H, T, d).total);
}

// Of a tree's call over a cache of 8 or 16 bits: that of many query rows to a K/V head has a cut of its own.
int check_tree_shape(int sequences, int H, int Hk, int T, int d, bool e4m3, DecodeCuts& cuts, bool& is_wide, FmDecodeCut& wide) {
  if (int rc = check_decode_shape(sequences, H, Hk, T, d, cuts)) return rc;
  is_wide = fm_tree_is_wide((long long)H / Hk * T, T, d, e4m3);
  if (!is_wide) return FM_OK;
  wide = fm_tree_cut(H, Hk, T, d, sequences, fm_compute_units());
  return (fm_most_units(wide.chunks, sequences) + 8ll) * wide.workgroups < 1 << 24 ? FM_OK : FM_ERR_SHAPE;
}

// Checks of a decoding call and its launch arguments.  wide: whether a tree's has many query rows to a K/V head.
int decode_args(bool tree, const flashmask_cache* cache, const void* q, const int32_t* lens, const int32_t* lts, const int32_t* lte, const int32_t* uts,
                const int32_t* ute, int bound_columns, int window, float scale, void* out, float* lse, int type, int H, int T,
                const flashmask_strides* strides, void* workspace, size_t workspace_bytes, FmDecodeArgs& a, bool& wide) {
  if (int rc = check_cache(cache)) return rc;
  if (!q || !lens || !out || !lse || !strides) return FM_ERR_NULL;
  const bool bounds = lts || lte || uts || ute;
  if (bounds && (!lts || !lte || !uts || !ute)) return FM_ERR_NULL;
  if (int rc = check_row_type(type, *cache)) return rc;
  DecodeCuts cuts;
  wide = false;
  if (int rc = tree ? check_tree_shape(cache->sequences, H, cache->heads, T, cache->d, cache->type == FM_TYPE_E4M3, cuts, wide, a.cut)
                    : check_decode_shape(cache->sequences, H, cache->heads, T, cache->d, cuts)) return rc;
  if (bounds && bound_columns <= 0) return FM_ERR_SHAPE;
  if ((long long)cache->sequences * cache->columns * cache->page > 1ll << 34) return FM_ERR_SHAPE;   // groups of 16 keys are added up in 32 bits
  if (!(scale > 0.f) || !(scale < 3.0e38f) || window < 0) return FM_ERR_ARG;
  for (int t = 0; t < 2; ++t)
    if (int rc = check_strides(strides[t], type, cache->sequences, H, T, cache->d)) return rc;
  if (misaligned(q) || misaligned(out)) return FM_ERR_ALIGN;
  if (bad_workspace(workspace, workspace_bytes, wide ? decode_space(a.cut, cache->sequences, H, T, cache->d).total
                                                     : decode_bytes(cuts, cache->sequences, H, T, cache->d))) return FM_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  a.q = q; a.out = out; a.lse = lse; a.sq = to_kernel(strides[0]); a.so = to_kernel(strides[1]);
  a.k = pages(cache->k, cache->sk, cache->type);
  a.v = pages(cache->v, cache->sv, cache->type);
  a.k_scale = cache->k_scale; a.v_scale = cache->v_scale;
  a.table = cache->table; a.lens = lens;
  a.bounds[0] = lts; a.bounds[1] = lte; a.bounds[2] = uts; a.bounds[3] = ute;
  a.scale = scale;
  a.B = cache->sequences; a.H = H; a.Hk = cache->heads; a.T = T; a.d = cache->d;
  a.columns = cache->columns; a.num_pages = cache->num_pages; a.page_tokens = cache->page;
  a.bound_columns = bounds ? bound_columns : 0;
  a.window = window < (1 << 30) ? window : 0;   // no table holds more keys
  a.page = fm_divisor(cache->page);
  // Pages stored token by token have the rows of all heads side by side: a workgroup takes two of less than 256 bytes together.
  const int row = cache->d * element_bytes(cache->type);
  const bool side_by_side = a.k.head < 256 && a.v.head < 256;
  if (!wide) a.cut = cuts.of[side_by_side && row < 256];
  const int round = wide ? FM_TREE_ROUND : fm_decode_round_groups(cache->d, cache->type == FM_TYPE_E4M3, a.cut);
  const bool split = (long long)cache->columns * cache->page >
                     fm_whole_keys(round, (long long)cache->sequences * a.cut.workgroups,
                                   a.cut.least, fm_compute_units());
  const DecodeSpace space = decode_space(a.cut, cache->sequences, H, T, cache->d);
  const bool listed = split && a.cut.listed;
  a.plan = split ? (int2*)ws : nullptr;
  a.units = listed ? (int4*)(ws + space.units) : nullptr;
  a.split = listed ? (int*)(ws + space.split) : nullptr;
  a.stat = (float2*)(ws + space.stat);
  a.part = (float*)(ws + space.part);
  return FM_OK;
}

// Of a call on a prompt's weights: launches have fewer than 2^32 lanes.
int check_weights_shape(int B, int H, int Hk, int N, int d, int first_row, FmWeightsCut& cut) {
  if (B <= 0 || H <= 0 || H > FM_MOST_HEADS || Hk <= 0 || H % Hk || N <= 0 || N > (1 << 30) || bad_head_dim(d) || first_row < 0 || first_row >= N)
    return FM_ERR_SHAPE;
  if ((long long)B * Hk > 1 << 22 || (long long)H / Hk * ((N - first_row + 63) / 64) > 1 << 30) return FM_ERR_SHAPE;
  cut = fm_weights_cut(B, H, Hk, N, first_row, fm_compute_units());
  return (long long)B * Hk * cut.key_blocks * cut.parts < 1 << 24 ? FM_OK : FM_ERR_SHAPE;
}
size_t weights_bytes(const FmWeightsCut& cut, int B, int Hk, int N) {
  return cut.parts == 1 ? 256 : (size_t)cut.parts * B * Hk * N * sizeof(float);
}

int check_pools(void* const* pools, int num_pools, size_t page_bytes, int num_pages) {
  if (num_pools < 0 || num_pages <= 0) return FM_ERR_SHAPE;
  if (num_pools == 0) return FM_OK;
  if (!pools) return FM_ERR_NULL;
  if (page_bytes == 0 || page_bytes % 16 || page_bytes > (1u << 30)) return FM_ERR_SHAPE;
  for (int i = 0; i < num_pools; ++i) {
    if (!pools[i]) return FM_ERR_NULL;
    if (misaligned(pools[i])) return FM_ERR_ALIGN;
  }
  return FM_OK;
}

}  // namespace

extern "C" {

int flashmask_rope(const void* q, const void* k, void* q_out, void* k_out, const double* freqs, const int32_t* positions,
                   int type, int layout, double amp, int B, int H, int H_kv, int N, int d, int rot,
                   const flashmask_strides* strides, void* hip_stream) {
  return rope(q, k, q_out, k_out, freqs, positions, type, layout, amp, B, H, H_kv, N, d, rot, strides, false, hip_stream);
}

int flashmask_rope_bwd(const void* dq_out, const void* dk_out, void* dq, void* dk, const double* freqs,
                       const int32_t* positions, int type, int layout, double amp, int B, int H, int H_kv, int N, int d,
                       int rot, const flashmask_strides* strides, void* hip_stream) {
  return rope(dq_out, dk_out, dq, dk, freqs, positions, type, layout, amp, B, H, H_kv, N, d, rot, strides, true, hip_stream);
}

int flashmask_cache_append(const flashmask_cache* cache, const void* q, const void* k, const void* v, void* q_out,
                           const int32_t* seqs, const int32_t* positions, const double* freqs, int type, int layout,
                           double amp, int tokens, int H, int rot, const flashmask_strides* strides, void* hip_stream) {
  if (int rc = check_cache(cache)) return rc;
  if (!k || !v || !seqs || !positions || !strides || (q && (!q_out || !freqs))) return FM_ERR_NULL;
  if (int rc = check_row_type(type, *cache)) return rc;
  if (tokens <= 0 || tokens > (1 << 27) || (q && (H <= 0 || H > FM_MOST_HEADS))) return FM_ERR_SHAPE;
  if (freqs)
    if (int rc = check_rotation(layout, amp, cache->d, rot)) return rc;
  for (int t = q ? 0 : 1; t < (q ? 4 : 3); ++t)
    if (int rc = check_strides(strides[t], type, 1, t % 3 ? cache->heads : H, tokens, cache->d)) return rc;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(q_out)) return FM_ERR_ALIGN;
  FmAppendArgs a;
  a.in[0] = q; a.in[1] = k; a.in[2] = v; a.q_out = q_out;
  for (int t = 0; t < 3; ++t) a.si[t] = to_kernel(strides[t]);
  a.so = to_kernel(strides[3]);
  a.cache[0] = pages(cache->k, cache->sk, cache->type);
  a.cache[1] = pages(cache->v, cache->sv, cache->type);
  a.scale[0] = cache->k_scale; a.scale[1] = cache->v_scale;
  a.table = cache->table; a.seqs = seqs; a.positions = positions; a.freqs = freqs; a.amp = amp;
  a.tokens = tokens; a.heads[0] = q ? H : 0; a.heads[1] = a.heads[2] = cache->heads;
  a.d = cache->d; a.rot = freqs ? rot : 0;
  a.sequences = cache->sequences; a.columns = cache->columns; a.num_pages = cache->num_pages;
  a.page = fm_divisor(cache->page);
  return done(fm_launch_append(a, type == FM_TYPE_F16, cache->type == FM_TYPE_E4M3, layout == FM_ROPE_INTERLEAVED, (hipStream_t)hip_stream));
}

size_t flashmask_decode_workspace_bytes(int sequences, int H, int H_kv, int T, int d) {
  DecodeCuts cuts;
  return check_decode_shape(sequences, H, H_kv, T, d, cuts) == FM_OK ? decode_bytes(cuts, sequences, H, T, d) : 0;
}

int flashmask_decode(const flashmask_cache* cache, const void* q, const int32_t* lens, const int32_t* lts,
                     const int32_t* lte, const int32_t* uts, const int32_t* ute, int bound_columns, int window, float scale,
                     void* out, float* lse, int type, int H, int T, const flashmask_strides* strides, void* workspace,
                     size_t workspace_bytes, void* hip_stream) {
  FmDecodeArgs a;
  bool wide;
  if (int rc = decode_args(false, cache, q, lens, lts, lte, uts, ute, bound_columns, window, scale, out, lse, type, H, T, strides, workspace,
                           workspace_bytes, a, wide)) return rc;
  return done(fm_launch_decode(a, type == FM_TYPE_F16, cache->type == FM_TYPE_E4M3, (hipStream_t)hip_stream));
}

size_t flashmask_decode_tree_workspace_bytes(int sequences, int H, int H_kv, int T, int d) {
  size_t most = 0;   // of whatever cache
  for (const bool e4m3 : {false, true}) {
    DecodeCuts cuts;
    FmDecodeCut cut;
    bool wide;
    if (check_tree_shape(sequences, H, H_kv, T, d, e4m3, cuts, wide, cut) != FM_OK) return 0;
    most = std::max(most, wide ? decode_space(cut, sequences, H, T, d).total : decode_bytes(cuts, sequences, H, T, d));
  }
  return most;
}

int flashmask_decode_tree(const flashmask_cache* cache, const void* q, const int32_t* lens, const int32_t* parents, const int32_t* lts,
                          const int32_t* lte, const int32_t* uts, const int32_t* ute, int bound_columns, int window, float scale,
                          void* out, float* lse, int type, int H, int T, const flashmask_strides* strides, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
  if (!parents) return FM_ERR_NULL;
  FmTreeArgs a;
  bool wide;
  if (int rc = decode_args(true, cache, q, lens, lts, lte, uts, ute, bound_columns, window, scale, out, lse, type, H, T, strides, workspace,
                           workspace_bytes, a, wide)) return rc;
  a.parents = parents;
  return done((wide ? fm_launch_tree_wide : fm_launch_decode_tree)(a, type == FM_TYPE_F16, cache->type == FM_TYPE_E4M3, (hipStream_t)hip_stream));
}

size_t flashmask_weights_workspace_bytes(int B, int H, int H_kv, int N, int d, int first_row) {
  FmWeightsCut cut;
  return check_weights_shape(B, H, H_kv, N, d, first_row, cut) == FM_OK ? weights_bytes(cut, B, H_kv, N) : 0;
}

int flashmask_weights(const void* q, const void* k, const float* lse, const int32_t* lts, const int32_t* lte, const int32_t* uts,
                      const int32_t* ute, float scale, float* weights, int B, int H, int H_kv, int N, int d, int first_row,
                      const flashmask_strides* strides, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!q || !k || !lse || !lts || !lte || !uts || !ute || !weights || !strides) return FM_ERR_NULL;
  FmWeightsCut cut;
  if (int rc = check_weights_shape(B, H, H_kv, N, d, first_row, cut)) return rc;
  if (!(scale > 0.f) || !(scale < 3.0e38f)) return FM_ERR_ARG;
  for (int t = 0; t < 2; ++t)
    if (int rc = check_strides(strides[t], FM_TYPE_BF16, B, t ? H_kv : H, N, d)) return rc;
  if (misaligned(q) || misaligned(k)) return FM_ERR_ALIGN;
  if (bad_workspace(workspace, workspace_bytes, weights_bytes(cut, B, H_kv, N))) return FM_ERR_WORKSPACE;
  FmWeightsArgs a;
  a.q = q; a.k = k; a.lse = lse; a.part = (float*)workspace;
  a.bounds[0] = lts; a.bounds[1] = lte; a.bounds[2] = uts; a.bounds[3] = ute;
  a.sq = to_kernel(strides[0]); a.sk = to_kernel(strides[1]);
  a.scale = scale;
  a.B = B; a.H = H; a.Hk = H_kv; a.N = N; a.d = d; a.first_row = first_row;
  return done(fm_launch_weights(a, weights, cut, (hipStream_t)hip_stream));
}

int flashmask_cache_weights(const flashmask_cache* cache, const void* q, const int32_t* lens, const int32_t* lts, const int32_t* lte,
                            const int32_t* uts, const int32_t* ute, int bound_columns, int window, float scale, const float* lse,
                            const float* before, float decay, float* weights, int weight_columns, int type, int H, int T,
                            const flashmask_strides* strides, void* hip_stream) {
  if (int rc = check_cache(cache)) return rc;
  if (!q || !lens || !lse || !weights || !strides) return FM_ERR_NULL;
  const bool bounds = lts || lte || uts || ute;
  if (bounds && (!lts || !lte || !uts || !ute)) return FM_ERR_NULL;
  if (int rc = check_row_type(type, *cache)) return rc;
  const int B = cache->sequences, Hk = cache->heads;
  if (H <= 0 || H > FM_MOST_HEADS || H % Hk || T <= 0 || T > FM_MOST_NEW_TOKENS || B > 65535 || (long long)H * T > (1 << 24) ||
      (long long)H * T * B > (1ll << 30) || weight_columns <= 0 || weight_columns > (1 << 30) || (bounds && bound_columns <= 0))
    return FM_ERR_SHAPE;
  if (!(scale > 0.f) || !(scale < 3.0e38f) || window < 0 || !(decay >= 0.f) || !(decay < 3.0e38f)) return FM_ERR_ARG;
  if (int rc = check_strides(strides[0], type, B, H, T, cache->d)) return rc;
  if (misaligned(q)) return FM_ERR_ALIGN;
  FmCacheWeightsArgs a;
  a.places = (int)std::min<long long>((long long)cache->columns * cache->page, weight_columns);
  if ((long long)B * a.places > 1ll << 34) return FM_ERR_SHAPE;   // groups of 16 keys are added up in 32 bits
  a.q = q; a.lse = lse; a.sq = to_kernel(strides[0]);
  a.k = pages(cache->k, cache->sk, cache->type);
  a.k_scale = cache->k_scale;
  a.table = cache->table; a.lens = lens;
  a.bounds[0] = lts; a.bounds[1] = lte; a.bounds[2] = uts; a.bounds[3] = ute;
  a.before = decay > 0.f ? before : nullptr;
  a.weights = weights;
  a.scale = scale; a.decay = decay;
  a.B = B; a.H = H; a.Hk = Hk; a.T = T; a.d = cache->d; a.columns = cache->columns; a.num_pages = cache->num_pages;
  a.bound_columns = bounds ? bound_columns : 0;
  a.window = window < (1 << 30) ? window : 0;   // no table holds more keys
  a.weight_columns = weight_columns;
  a.page = fm_divisor(cache->page); a.tokens = fm_divisor(T); a.by_head = fm_divisor(Hk);
  if (!fm_cut_cache_weights(a, fm_compute_units())) return FM_ERR_SHAPE;
  return done(fm_launch_cache_weights(a, type == FM_TYPE_F16, cache->type == FM_TYPE_E4M3, (hipStream_t)hip_stream));
}

size_t flashmask_cache_evict_workspace_bytes(int sequences, int weight_heads, int weight_columns) {
  if (sequences <= 0 || sequences > 65535 || weight_heads <= 0 || weight_heads > FM_MOST_HEADS || weight_columns <= 0 || weight_columns > (1 << 30)) return 0;
  return std::max<size_t>(fm_evict_bytes(sequences, weight_heads, weight_columns), 256);
}

int flashmask_cache_evict(const flashmask_cache* cache, const int32_t* lens, const float* weights, int weight_heads, int weight_columns,
                          int keep, int first, int recent, const int32_t* new_table, int new_columns, int32_t* table_out, int32_t* lens_out,
                          float* weights_out, int32_t* kept, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_cache(cache)) return rc;
  if (!lens || !weights || !new_table || !table_out || !lens_out || !weights_out || !kept) return FM_ERR_NULL;
  if (weight_columns <= 0 || weight_columns > (1 << 30) || (weight_heads != 1 && weight_heads != cache->heads) || cache->sequences > 65535 ||
      keep <= 0 || keep > (1 << 30) - 64 || first < 0 || recent < 0 || (long long)first + recent > keep || new_columns <= 0)
    return FM_ERR_SHAPE;
  const int pages_kept = (keep + cache->page - 1) / cache->page;
  if (new_columns < pages_kept || cache->columns < pages_kept) return FM_ERR_SHAPE;
  if (bad_workspace(workspace, workspace_bytes, flashmask_cache_evict_workspace_bytes(cache->sequences, weight_heads, weight_columns))) return FM_ERR_WORKSPACE;
  FmEvictArgs a;
  a.cache[0] = pages(cache->k, cache->sk, cache->type);
  a.cache[1] = pages(cache->v, cache->sv, cache->type);
  a.table = cache->table; a.lens = lens; a.new_table = new_table; a.weights = weights; a.weights_out = weights_out;
  a.kept = kept; a.table_out = table_out; a.lens_out = lens_out; a.scratch = (unsigned*)workspace;
  a.B = cache->sequences; a.Hk = cache->heads; a.weight_heads = weight_heads; a.weight_columns = weight_columns;
  a.keep = keep; a.first = first; a.recent = recent; a.columns = cache->columns; a.new_columns = new_columns; a.num_pages = cache->num_pages;
  a.row_bytes = cache->d * element_bytes(cache->type);
  a.page = fm_divisor(cache->page);
  return done(fm_launch_evict(a, (hipStream_t)hip_stream));
}

int flashmask_cache_accept(void* const* pools, int num_pools, const flashmask_strides* strides, int type, int heads, int d, int num_pages,
                           int page, const int32_t* table, const int32_t* lens, const int32_t* path, int32_t* lens_out, int sequences,
                           int columns, int T, int path_columns, void* hip_stream) {
  if (!pools || !strides || !table || !lens || !path || !lens_out) return FM_ERR_NULL;
  if (type != FM_TYPE_BF16 && type != FM_TYPE_F16 && type != FM_TYPE_E4M3) return FM_ERR_ARG;
  if (num_pools <= 0 || heads <= 0 || heads > FM_MOST_HEADS || bad_head_dim(d) || num_pages <= 0 || page <= 0 || page % 16 || page > (1 << 20) ||
      sequences <= 0 || sequences > 65535 || columns <= 0 || (long long)columns * page > (1 << 30) || T <= 0 || T > FM_MOST_NEW_TOKENS ||
      path_columns <= 0 || path_columns > T)
    return FM_ERR_SHAPE;
  if (int rc = check_strides(*strides, type, num_pages, heads, page, d)) return rc;
  for (int i = 0; i < num_pools; ++i) {
    if (!pools[i]) return FM_ERR_NULL;
    if (misaligned(pools[i])) return FM_ERR_ALIGN;
  }
  const int bytes = element_bytes(type);
  FmAcceptArgs a;
  a.page_bytes = strides->batch * bytes; a.head_bytes = strides->head * bytes; a.token_bytes = (unsigned)(strides->row * bytes);
  a.heads = heads; a.row_bytes = d * bytes; a.num_pages = num_pages;
  a.table = table; a.lens = lens; a.path = path; a.lens_out = lens_out;
  a.B = sequences; a.columns = columns; a.T = T; a.path_columns = path_columns;
  a.page = fm_divisor(page);
  return done(fm_launch_accept(pools, num_pools, a, (hipStream_t)hip_stream));
}

int flashmask_cache_fork(void* const* pools, int num_pools, size_t page_bytes, int num_pages, const int32_t* table,
                         const int32_t* lens, const int32_t* parents, const int32_t* new_pages, int32_t* table_out,
                         int32_t* lens_out, int sequences, int columns, int page, int children, void* hip_stream) {
  if (!table || !lens || !parents || !new_pages || !table_out || !lens_out) return FM_ERR_NULL;
  if (int rc = check_pools(pools, num_pools, page_bytes, num_pages)) return rc;
  if (sequences <= 0 || columns <= 0 || page <= 0 || children <= 0 || children > 65535) return FM_ERR_SHAPE;
  return done(fm_launch_fork(pools, num_pools, page_bytes, num_pages, table, lens, parents, new_pages, table_out, lens_out, sequences,
                             columns, page, children, (hipStream_t)hip_stream));
}

size_t flashmask_cache_plan_bytes(int num_pages) { return num_pages > 0 && num_pages <= (1 << 30) ? fm_plan_bytes(num_pages) : 0; }

int flashmask_cache_free_list(const int32_t* table, int entries, int num_pages, int32_t* free_pages, int32_t* count,
                              void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!table || !free_pages || !count) return FM_ERR_NULL;
  if (entries <= 0 || entries > (1 << 30) || num_pages <= 0 || num_pages > (1 << 30)) return FM_ERR_SHAPE;
  if (bad_workspace(workspace, workspace_bytes, fm_plan_bytes(num_pages))) return FM_ERR_WORKSPACE;
  return done(fm_launch_free_list(table, entries, num_pages, free_pages, count, workspace, (hipStream_t)hip_stream));
}

int flashmask_cache_compact(void* const* pools, int num_pools, size_t page_bytes, int num_pages, const int32_t* table,
                            int entries, int32_t* table_out, int32_t* used, void* workspace, size_t workspace_bytes,
                            void* hip_stream) {
  if (!table || !table_out || !used) return FM_ERR_NULL;
  if (entries <= 0 || entries > (1 << 30) || num_pages > (1 << 30)) return FM_ERR_SHAPE;
  if (int rc = check_pools(pools, num_pools, page_bytes, num_pages)) return rc;
  if (bad_workspace(workspace, workspace_bytes, fm_plan_bytes(num_pages))) return FM_ERR_WORKSPACE;
  return done(fm_launch_compact(pools, num_pools, page_bytes, num_pages, table, entries, table_out, used, workspace, (hipStream_t)hip_stream));
}

}  // extern "C"
