// Rotary positions: rows turned in place of the tensor (flashmask_rope), or on their way to the cache (flashmask_cache_append).
#include <algorithm>

#include "fm_common.h"
#include "fm_serving.h"

namespace fm {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(8))) float f32x8;

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
struct Turn {
  static constexpr int V = Vec<T>::N;
  int piece[2];
  bool turned[2];
  float c[V], s[V];

  __device__ __forceinline__ void place(int u, int d, int rot) {
    const int pieces = rot / V, pairs = d / (2 * V);
    if (INTER) {
      // u and u + pairs: neighbouring lanes read neighbouring pieces
      piece[0] = u;
      piece[1] = u + pairs;
      turned[0] = piece[0] < pieces;
      turned[1] = piece[1] < pieces;
    } else {
      const bool head = u < pieces / 2;
      piece[0] = head ? u : pieces + 2 * (u - pieces / 2);
      piece[1] = head ? u + pieces / 2 : piece[0] + 1;
      turned[0] = turned[1] = head;
    }
  }
  __device__ __forceinline__ void angles(double position, const double* freqs, double amp, bool backward) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int i = INTER ? piece[e / (V / 2)] * (V / 2) + e % (V / 2) : piece[0] * V + e;
      c[e] = 1.f;
      s[e] = 0.f;
      if (turned[INTER ? e / (V / 2) : 0]) {
        double cd, sd;
        cos_sin(position * freqs[i], cd, sd);
        c[e] = (float)(cd * amp);
        s[e] = (float)(backward ? -sd * amp : sd * amp);
      }
    }
  }
  __device__ __forceinline__ void apply(float (&x)[V], float (&y)[V]) const {
    if (INTER) {
#pragma unroll
      for (int e = 0; e < V / 2; ++e) {
        const float a = x[2 * e], b = x[2 * e + 1], p = y[2 * e], q = y[2 * e + 1];
        if (turned[0]) {
          x[2 * e] = a * c[e] - b * s[e];
          x[2 * e + 1] = b * c[e] + a * s[e];
        }
        if (turned[1]) {
          y[2 * e] = p * c[V / 2 + e] - q * s[V / 2 + e];
          y[2 * e + 1] = q * c[V / 2 + e] + p * s[V / 2 + e];
        }
      }
    } else if (turned[0]) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float a = x[e], b = y[e];
        x[e] = a * c[e] - b * s[e];
        y[e] = b * c[e] + a * s[e];
      }
    }
  }
};

// A lane computes its angles once and turns its part of the row of `group` heads by them, HEADS at a time so that their loads
// are in flight together.  Bound by memory: each element is read and written once.
template <class T, bool INTER>
__global__ __launch_bounds__(256) void rope_kernel(FmRopeArgs a, bool backward) {
  constexpr int HEADS = 4;
  using VT = Vec<T>;
  const int lanes = a.d / (2 * VT::N);   // to a row: a power of two
  const int at = (int)blockIdx.x * 256 + threadIdx.x;
  const int row = at / lanes, u = at % lanes;
  if (row >= a.B * a.N) return;
  const int b = fm_div(row, a.rows), n = row - b * a.N;
  Turn<T, INTER> turn;
  turn.place(u, a.d, a.rot);
  turn.angles(a.positions ? a.positions[row] : n, a.freqs, a.amp, backward);
  const int first = blockIdx.y * a.group, last = min(first + a.group, a.heads[0] + a.heads[1]);
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int h0 = max(w ? first - a.heads[0] : first, 0), h1 = min(w ? last - a.heads[0] : last, a.heads[w]);
    const T* in = (const T*)a.in[w] + (size_t)b * a.si[w].b + (size_t)n * a.si[w].n;
    T* out = (T*)a.out[w] + (size_t)b * a.so[w].b + (size_t)n * a.so[w].n;
    for (int h = h0; h < h1; h += HEADS) {
      u32x4 raw[HEADS][2];
#pragma unroll
      for (int j = 0; j < HEADS; ++j)
        if (h + j < h1) {
          const T* p = in + (size_t)(h + j) * a.si[w].h;
          raw[j][0] = ldg16(p + turn.piece[0] * VT::N);
          raw[j][1] = ldg16(p + turn.piece[1] * VT::N);
        }
#pragma unroll
      for (int j = 0; j < HEADS; ++j)
        if (h + j < h1) {
          float x[VT::N], y[VT::N];
          VT::get(raw[j][0], x);
          VT::get(raw[j][1], y);
          turn.apply(x, y);
          T* p = out + (size_t)(h + j) * a.so[w].h;
          *(u32x4*)(p + turn.piece[0] * VT::N) = VT::put(x);
          *(u32x4*)(p + turn.piece[1] * VT::N) = VT::put(y);
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

// The rows of a token as in rope_kernel: its queries to q_out, its keys and values to their place in the cache.
template <class T, bool E4M3, bool INTER>
__global__ __launch_bounds__(256) void append_kernel(FmAppendArgs a) {
  using VT = Vec<T>;
  const int lanes = a.d / 16;
  const int at = (int)blockIdx.x * 256 + threadIdx.x;
  const int token = at / lanes, u = at % lanes;
  if (token >= a.tokens) return;
  const int first = blockIdx.y * a.group, last = min(first + a.group, a.heads[0] + 2 * a.heads[1]);
  const int position = a.positions[token];
  Turn<T, INTER> turn;
  turn.place(u, a.d, a.rot);
  if (first < a.heads[0] + a.heads[1]) turn.angles(position, a.freqs, a.amp, false);
  int page = -1, slot = 0;
  if (last > a.heads[0]) {
    const int seq = a.seqs[token];
    const FmPlace place = fm_place(position, a.page, a.columns);
    if (seq >= 0 && seq < a.sequences && place.column >= 0)
      page = fm_known_page(a.table[(size_t)seq * a.columns + place.column], a.num_pages);
    slot = place.slot;
  }
#pragma unroll
  for (int w = 0; w < 3; ++w) {
    const int before = w == 0 ? 0 : a.heads[0] + (w - 1) * a.heads[1];
    const int h0 = max(first - before, 0), h1 = min(last - before, a.heads[w]);
    if (w > 0 && page < 0) continue;
    const T* in = (const T*)a.in[w] + (size_t)token * a.si[w].n;
    for (int h = h0; h < h1; ++h) {
      float x[8], y[8];
      const T* p = in + (size_t)h * a.si[w].h;
      const u32x4 r0 = ldg16(p + turn.piece[0] * 8), r1 = ldg16(p + turn.piece[1] * 8);
      VT::get(r0, x);
      VT::get(r1, y);
      if (w < 2) turn.apply(x, y);
      if (w == 0) {
        T* o = (T*)a.q_out + (size_t)token * a.so.n + (size_t)h * a.so.h;
        *(u32x4*)(o + turn.piece[0] * 8) = VT::put(x);
        *(u32x4*)(o + turn.piece[1] * 8) = VT::put(y);
      } else {
        const FmPages& c = a.cache[w - 1];
        char* o = c.base + (long long)page * c.page + h * c.head + (size_t)slot * c.token;
        if (E4M3) {
          const float scale = a.scale[w - 1][h];
          *(u32x2*)(o + turn.piece[0] * 8) = to_e4m3(x, scale);
          *(u32x2*)(o + turn.piece[1] * 8) = to_e4m3(y, scale);
        } else {
          *(u32x4*)(o + turn.piece[0] * 16) = VT::put(x);
          *(u32x4*)(o + turn.piece[1] * 16) = VT::put(y);
        }
      }
    }
  }
}

// Heads to a workgroup: all of them share a row's angles, but a call of few rows has to give every compute unit some.
static int head_group(long long row_lanes, int heads) {
  const long long workgroups = (row_lanes + 255) / 256, wanted = 8ll * fm_compute_units();
  int groups = (int)std::min<long long>(heads, (wanted + workgroups - 1) / workgroups);
  return (heads + groups - 1) / groups;
}

}  // namespace fm

hipError_t fm_launch_rope(FmRopeArgs a, int type, bool interleaved, bool backward, hipStream_t stream) {
  const int heads = a.heads[0] + a.heads[1];
  const long long lanes = (long long)a.B * a.N * (a.d / (type == 2 ? 8 : 16));
  a.group = fm::head_group(lanes, heads);
  const dim3 grid((unsigned)((lanes + 255) / 256), (heads + a.group - 1) / a.group), block(256);
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
  const int heads = a.heads[0] + 2 * a.heads[1];
  const long long lanes = (long long)a.tokens * (a.d / 16);
  a.group = fm::head_group(lanes, heads);
  const dim3 grid((unsigned)((lanes + 255) / 256), (heads + a.group - 1) / a.group), block(256);
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
