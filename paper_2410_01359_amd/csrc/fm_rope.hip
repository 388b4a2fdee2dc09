// Rotary positions: rows turned in place of the tensor (flashmask_rope), or on their way to the cache (flashmask_cache_append).
#include <algorithm>

#include "fm_common.h"
#include "fm_serving.h"

namespace fm {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

// Cosine and sine of an angle in 64 bits: reduced to [-pi/4, pi/4] in two steps (pi/2 as a sum of two doubles), then the
// Taylor series, cut where the next term is below 2^-32.
__device__ __forceinline__ void cos_sin(double angle, double& c, double& s) {
  constexpr double kHalfPi = 1.57079632679489661923, kHalfPiRest = 6.12323399573676603587e-17;
  const double turns = __builtin_rint(angle * (1.0 / kHalfPi));
  double r = __builtin_fma(-turns, kHalfPi, angle);
  r = __builtin_fma(-turns, kHalfPiRest, r);
  const int quadrant = (int)(turns - 4.0 * __builtin_floor(turns * 0.25));
  const double z = r * r;
  double sp = __builtin_fma(z, -1.0 / 39916800, 1.0 / 362880);
  sp = __builtin_fma(z, sp, -1.0 / 5040);
  sp = __builtin_fma(z, sp, 1.0 / 120);
  sp = __builtin_fma(z, sp, -1.0 / 6);
  sp = __builtin_fma(z * r, sp, r);
  double cp = __builtin_fma(z, -1.0 / 3628800, 1.0 / 40320);
  cp = __builtin_fma(z, cp, -1.0 / 720);
  cp = __builtin_fma(z, cp, 1.0 / 24);
  cp = __builtin_fma(z, cp, -0.5);
  cp = __builtin_fma(z, cp, 1.0);
  c = quadrant & 1 ? sp : cp;
  s = quadrant & 1 ? cp : sp;
  if (quadrant == 1 || quadrant == 2) c = -c;
  if (quadrant >= 2) s = -s;
}

// 16 bytes of a row as floats and back.
template <class T>
struct Vec;
template <>
struct Vec<__bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(u32x4 raw, float (&x)[8]) {
    const bf16x8 h = __builtin_bit_cast(bf16x8, raw);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)h[e];
  }
  static __device__ __forceinline__ u32x4 put(const float (&x)[8]) {
    bf16x8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (__bf16)x[e];
    return __builtin_bit_cast(u32x4, h);
  }
};
template <>
struct Vec<_Float16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(u32x4 raw, float (&x)[8]) {
    const f16x8 h = __builtin_bit_cast(f16x8, raw);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)h[e];
  }
  static __device__ __forceinline__ u32x4 put(const float (&x)[8]) {
    f16x8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (_Float16)x[e];
    return __builtin_bit_cast(u32x4, h);
  }
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(u32x4 raw, float (&x)[4]) {
    const f32x4 h = __builtin_bit_cast(f32x4, raw);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = h[e];
  }
  static __device__ __forceinline__ u32x4 put(const float (&x)[4]) {
    f32x4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = x[e];
    return __builtin_bit_cast(u32x4, h);
  }
};

// What a lane has of a row: two 16-byte pieces whose elements are turned with each other (halves) or each with its neighbour
// (interleaved), V angles for both.  Lane u of the D / (2 V) that share a row; the pieces behind the turned part come in pairs too.
template <class T, bool INTER>
struct Pieces {
  static constexpr int V = Vec<T>::N;
  int at[2];
  bool turned[2];

  __device__ __forceinline__ void place(int u, int d, int rot) {
    const int pieces = rot / V, pairs = d / (2 * V);
    if (INTER) {
      // u and u + pairs: neighbouring lanes read neighbouring pieces
      at[0] = u;
      at[1] = u + pairs;
      turned[0] = at[0] < pieces;
      turned[1] = at[1] < pieces;
    } else {
      const bool head = u < pieces / 2;
      at[0] = head ? u : pieces + 2 * (u - pieces / 2);
      at[1] = head ? u + pieces / 2 : at[0] + 1;
      turned[0] = turned[1] = head;
    }
  }
  // turns: cosines and sines of the row's angles
  __device__ __forceinline__ void apply(float (&x)[V], float (&y)[V], const float2* turns) const {
    if (INTER) {
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        if (!turned[w]) continue;
        float(&z)[V] = w ? y : x;
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
          const float2 t = turns[at[w] * (V / 2) + e];
          const float a = z[2 * e], b = z[2 * e + 1];
          z[2 * e] = a * t.x - b * t.y;
          z[2 * e + 1] = b * t.x + a * t.y;
        }
      }
    } else if (turned[0]) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float2 t = turns[at[0] * V + e];
        const float a = x[e], b = y[e];
        x[e] = a * t.x - b * t.y;
        y[e] = b * t.x + a * t.y;
      }
    }
  }
};

// Tokens of a workgroup at most.  Their angles are worked out once, one to a lane, and kept in LDS for all heads.
constexpr int kMostTokens = 32;
struct Turns {
  float2 of[kMostTokens][64];
};
template <class Position>
__device__ __forceinline__ void fill_turns(Turns& turns, const double* freqs, double amp, int half, bool backward, int tokens, const Position& position) {
  for (int i = threadIdx.x; i < tokens * 64; i += 256) {
    const int token = i / 64, e = i % 64;
    if (e >= half) continue;
    double c, s;
    cos_sin(position(token) * freqs[e], c, s);
    turns.of[token][e] = float2{(float)(c * amp), (float)(backward ? -s * amp : s * amp)};
  }
}

// The rows of `heads` heads of the workgroup's tokens, numbered in the order in which they lie in memory: token by token
// ([B,N,H,d] storage) or head by head.  (heads <= FM_MOST_HEADS: the product below is exact up to 2^32 / heads rows.)
struct RowOrder {
  bool by_token;
  unsigned inner, factor;
  __device__ __forceinline__ RowOrder(bool by_token_, int heads, int tokens) : by_token(by_token_), inner(by_token_ ? heads : tokens) {
    factor = 0xffffffffu / inner + 1;   // row / inner = row * factor / 2^32 (0: inner = 1)
  }
  __device__ __forceinline__ void at(unsigned row, int& token, int& head) const {
    const unsigned outer = factor ? __umulhi(row, factor) : row, rest = row - outer * inner;
    token = by_token ? outer : rest;
    head = by_token ? rest : outer;
  }
};

// Rows whose loads a lane has in flight.  Bound by memory, the two kernels are fastest with all eight waves of a SIMD and little
// work each: against four rows at five waves, 263 -> 247 us for 32768 tokens of 40 heads, d = 128, forward and back (stored by token).
constexpr int kBatch = 2;
// Results go past the L2, which has no use for them before they are pushed out: 247 -> 239 us there; prompts into an 8-bit cache at
// d = 64 45 -> 41.  (Loads past it, too, are 231 there, but 129 instead of 120 where a call's data fit the last-level cache.)
template <class V, class P>
__device__ __forceinline__ void stream_out(P* p, V v) {
  __builtin_nontemporal_store(v, (V*)p);
}

// A workgroup turns the rows of `span` tokens of `group` heads, in the order in which they lie in memory.  Bound by memory: each
// element is read and written once.
template <class T, bool INTER>
__global__ __launch_bounds__(256, 8) void rope_kernel(FmRopeArgs a, bool backward) {
  using VT = Vec<T>;
  __shared__ Turns turns;
  __shared__ long long start[4][kMostTokens];   // of the tokens in q, k, q_out, k_out
  const int all = a.B * a.N, token0 = blockIdx.x * a.span, tokens = min(a.span, all - token0);
  if (threadIdx.x < 4 * kMostTokens) {
    const int token = threadIdx.x % kMostTokens, which = threadIdx.x / kMostTokens, row = min(token0 + token, all - 1);
    const int b = fm_div(row, a.rows), n = row - b * a.N;
    const FmStride s = which == 0 ? a.si[0] : which == 1 ? a.si[1] : which == 2 ? a.so[0] : a.so[1];
    start[which][token] = b * s.b + n * s.n;
  }
  fill_turns(turns, a.freqs, a.amp, a.rot / 2, backward, tokens, [&](int token) {
    const int row = token0 + token;
    return (double)(a.positions ? a.positions[row] : row - fm_div(row, a.rows) * a.N);
  });
  __syncthreads();
  const int lanes = a.d / (2 * VT::N), shift = 31 - __builtin_clz(lanes), step = 256 >> shift;   // to a row: a power of two
  Pieces<T, INTER> pieces;
  pieces.place(threadIdx.x & (lanes - 1), a.d, a.rot);
  const int first = blockIdx.y * a.group, last = min(first + a.group, a.heads[0] + a.heads[1]);
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int h0 = max(w ? first - a.heads[0] : first, 0), h1 = min(w ? last - a.heads[0] : last, a.heads[w]);
    if (h0 >= h1) continue;
    const RowOrder order(a.si[w].h < a.si[w].n, h1 - h0, a.span);
    const int rows = (h1 - h0) * a.span;
    for (int base = threadIdx.x >> shift; base < rows; base += kBatch * step) {
      u32x4 raw[kBatch][2];
      int token[kBatch], head[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        order.at(base + j * step, token[j], head[j]);
        if (base + j * step >= rows || token[j] >= tokens) {
          token[j] = -1;
          continue;
        }
        const T* p = (const T*)a.in[w] + start[w][token[j]] + (h0 + head[j]) * a.si[w].h;
        raw[j][0] = ldg16(p + pieces.at[0] * VT::N);
        raw[j][1] = ldg16(p + pieces.at[1] * VT::N);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (token[j] < 0) continue;
        float x[VT::N], y[VT::N];
        VT::get(raw[j][0], x);
        VT::get(raw[j][1], y);
        pieces.apply(x, y, turns.of[token[j]]);
        T* p = (T*)a.out[w] + start[2 + w][token[j]] + (h0 + head[j]) * a.so[w].h;
        stream_out<u32x4>(p + pieces.at[0] * VT::N, VT::put(x));
        stream_out<u32x4>(p + pieces.at[1] * VT::N, VT::put(y));
      }
    }
  }
}

// Eight values over a scale to 8 bits each, held to what the type has (NaN stays NaN).
__device__ __forceinline__ u32x2 to_e4m3(const float (&x)[8], float scale) {
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] = x[e] / scale;
    y[e] = y[e] > 448.f ? 448.f : y[e];
    y[e] = y[e] < -448.f ? -448.f : y[e];
  }
  u32x2 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    int word = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
    r[w] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], word, true);
  }
  return r;
}

// The rows of a workgroup's tokens as in rope_kernel: its queries to q_out, its keys and values to their place in the cache.
template <class T, bool E4M3, bool INTER>
__global__ __launch_bounds__(256, 8) void append_kernel(FmAppendArgs a) {
  using VT = Vec<T>;
  __shared__ Turns turns;
  __shared__ int page[kMostTokens], slot[kMostTokens];
  const int token0 = blockIdx.x * a.span, tokens = min(a.span, a.tokens - token0);
  const int first = blockIdx.y * a.group, last = min(first + a.group, a.heads[0] + 2 * a.heads[1]);
  if (threadIdx.x < tokens) {
    const int token = token0 + threadIdx.x, seq = a.seqs[token];
    const FmPlace place = fm_place(a.positions[token], a.page, a.columns);
    page[threadIdx.x] = seq >= 0 && seq < a.sequences && place.column >= 0
                            ? fm_known_page(a.table[(size_t)seq * a.columns + place.column], a.num_pages) : -1;
    slot[threadIdx.x] = place.slot;
  }
  if (first < a.heads[0] + a.heads[1])
    fill_turns(turns, a.freqs, a.amp, a.rot / 2, false, tokens, [&](int token) { return (double)a.positions[token0 + token]; });
  __syncthreads();
  const int lanes = a.d / 16, shift = 31 - __builtin_clz(lanes), step = 256 >> shift;
  Pieces<T, INTER> pieces;
  pieces.place(threadIdx.x & (lanes - 1), a.d, a.rot);
#pragma unroll
  for (int w = 0; w < 3; ++w) {
    const int before = w == 0 ? 0 : a.heads[0] + (w - 1) * a.heads[1];
    const int h0 = max(first - before, 0), h1 = min(last - before, a.heads[w]);
    if (h0 >= h1) continue;
    const RowOrder order(a.si[w].h < a.si[w].n, h1 - h0, a.span);
    const int rows = (h1 - h0) * a.span;
    for (int base = threadIdx.x >> shift; base < rows; base += kBatch * step) {
      u32x4 raw[kBatch][2];
      int token[kBatch], head[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        order.at(base + j * step, token[j], head[j]);
        if (base + j * step >= rows || token[j] >= tokens || (w > 0 && page[token[j]] < 0)) {
          token[j] = -1;
          continue;
        }
        const T* p = (const T*)a.in[w] + (token0 + token[j]) * a.si[w].n + (h0 + head[j]) * a.si[w].h;
        raw[j][0] = ldg16(p + pieces.at[0] * 8);
        raw[j][1] = ldg16(p + pieces.at[1] * 8);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (token[j] < 0) continue;
        const int h = h0 + head[j];
        float x[8], y[8];
        VT::get(raw[j][0], x);
        VT::get(raw[j][1], y);
        if (w < 2) pieces.apply(x, y, turns.of[token[j]]);
        if (w == 0) {
          T* o = (T*)a.q_out + (token0 + token[j]) * a.so.n + h * a.so.h;
          stream_out<u32x4>(o + pieces.at[0] * 8, VT::put(x));
          stream_out<u32x4>(o + pieces.at[1] * 8, VT::put(y));
        } else {
          const FmPages& c = a.cache[w - 1];
          char* o = c.base + page[token[j]] * c.page + h * c.head + (size_t)slot[token[j]] * c.token;
          if (E4M3) {
            const float scale = a.scale[w - 1][h];
            stream_out<u32x2>(o + pieces.at[0] * 8, to_e4m3(x, scale));
            stream_out<u32x2>(o + pieces.at[1] * 8, to_e4m3(y, scale));
          } else {
            stream_out<u32x4>(o + pieces.at[0] * 16, VT::put(x));
            stream_out<u32x4>(o + pieces.at[1] * 16, VT::put(y));
          }
        }
      }
    }
  }
}

// Tokens and heads of a workgroup, `lanes` to a row.  All heads share the tokens' angles.  Stored by token, all heads of a token are one
// run of memory, and few tokens do: about one row to a lane, 32768 tokens of 40 heads 273, 261, 247, 240 us with 16, 8, 4, 2 of
// them; 6 heads 153, 149, 169, 284.  Stored by head, a head's tokens are: 293, 260, 259 us with 8, 16, 32 of them (40 heads), a single
// head 87, 56, 67.  A call of few tokens deals out the heads, too.
static dim3 share_out(long long tokens, int heads, int lanes, bool by_token, int& span, int& group) {
  span = 16;
  if (by_token)
    for (span = 2; span < kMostTokens && span * heads * lanes < 320;) span *= 2;
  if (tokens > (1 << 23)) span = kMostTokens;   // a launch has fewer than 2^32 lanes
  const long long workgroups = (tokens + span - 1) / span, wanted = 8ll * fm_compute_units();
  const int groups = (int)std::max<long long>(1, std::min<long long>(heads, wanted / workgroups));
  group = std::max((heads + groups - 1) / groups, 256 / (span * lanes));
  return dim3((unsigned)workgroups, (heads + group - 1) / group);
}

}  // namespace fm

hipError_t fm_launch_rope(FmRopeArgs a, int type, bool interleaved, bool backward, hipStream_t stream) {
  const dim3 grid = fm::share_out((long long)a.B * a.N, a.heads[0] + a.heads[1], a.d / (type == 2 ? 8 : 16), a.si[0].h < a.si[0].n, a.span, a.group), block(256);
#define FM_ROPE(T)                                                                                             \
  if (interleaved) hipLaunchKernelGGL((fm::rope_kernel<T, true>), grid, block, 0, stream, a, backward);        \
  else hipLaunchKernelGGL((fm::rope_kernel<T, false>), grid, block, 0, stream, a, backward)
  if (type == 0) { FM_ROPE(__bf16); }
  else if (type == 1) { FM_ROPE(_Float16); }
  else { FM_ROPE(float); }
#undef FM_ROPE
  return hipGetLastError();
}

hipError_t fm_launch_append(FmAppendArgs a, bool f16, bool e4m3, bool interleaved, hipStream_t stream) {
  const dim3 grid = fm::share_out(a.tokens, a.heads[0] + 2 * a.heads[1], a.d / 16, a.si[1].h < a.si[1].n, a.span, a.group), block(256);
#define FM_APPEND(T, E)                                                                                  \
  if (interleaved) hipLaunchKernelGGL((fm::append_kernel<T, E, true>), grid, block, 0, stream, a);       \
  else hipLaunchKernelGGL((fm::append_kernel<T, E, false>), grid, block, 0, stream, a)
  if (f16 && e4m3) { FM_APPEND(_Float16, true); }
  else if (f16) { FM_APPEND(_Float16, false); }
  else if (e4m3) { FM_APPEND(__bf16, true); }
  else { FM_APPEND(__bf16, false); }
#undef FM_APPEND
  return hipGetLastError();
}
