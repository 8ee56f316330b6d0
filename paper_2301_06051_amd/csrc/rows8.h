// Rows in 8 bits (dsvt_rows8): a row of C values v is C codes from -127 to 127 and a scale.  With m the largest |v| of the row, in 32 bits and
// every operation rounded once:
//   scale = m / 127 (or the float below it, should 127 times it pass 32 bits), code = v * (127 / m) rounded to the nearest whole number, ties to the
//   even one; the row stands for code * scale.
// m < 2^-118: scale and codes 0 (127 / m would pass 32 bits).  An infinity or a NaN in the row: scale NaN, codes 0, so that nothing that is made
// of the row is finite.
#pragma once
#include "rows.h"

namespace {

constexpr float kSmallestTop = 0x1p-118f;
constexpr float kLargestScale = 0x1.020406p+121f; // the largest whose product with 127 is a number

template <int V> struct Codes { typedef uint32_t type __attribute__((ext_vector_type(V / 4))); };
template <> struct Codes<4> { typedef uint32_t type; };
template <> struct Codes<1> { typedef uint8_t type; };

__device__ __forceinline__ int8_t byte_of(uint32_t p, int i) { return (int8_t)(p >> 8 * i); }
__device__ __forceinline__ int8_t byte_of(Codes<8>::type p, int i) { return byte_of(i < 4 ? p.x : p.y, i & 3); }

// One code of four as a float, in one instruction (the compiler takes two: it cuts the byte out first).
template <int kByte> __device__ __forceinline__ float code_of(uint32_t four) {
  float f;
  if constexpr (kByte == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(four));
  else if constexpr (kByte == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(four));
  else if constexpr (kByte == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(four));
  else asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(four));
  return f;
}
// codes times scale
template <int V> __device__ __forceinline__ void values_of(typename Codes<V>::type p, float scale, float (&f)[V]) {
  if constexpr (V <= 4) {
    f[0] = code_of<0>(p) * scale;
    if constexpr (V > 1) {
      f[1] = code_of<1>(p) * scale;
      f[2] = code_of<2>(p) * scale;
      f[3] = code_of<3>(p) * scale;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      float four[4];
      values_of<4>(p[i / 4], scale, four);
#pragma unroll
      for (int k = 0; k < 4; ++k) f[i + k] = four[k];
    }
  }
}

// Sizes as whole numbers: of infinities above those of numbers, of NaN above all.
__device__ __forceinline__ uint32_t size_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// The largest size of three, NaN if one is.
__device__ __forceinline__ float largest_size(float a, float b, float c) {
  float r;
  asm("v_maximum3_f32 %0, |%1|, |%2|, |%3|" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

struct RowScale {
  float scale, to_codes;                          // codes are v * to_codes, rounded; of a row without a scale 0
  bool plain;                                     // the row is numbers that are not too small
  __device__ __forceinline__ explicit RowScale(uint32_t top_bits) {
    const float top = __uint_as_float(top_bits);
    const bool numbers = top_bits < 0x7f800000u;
    plain = numbers && top >= kSmallestTop;
    scale = plain ? fminf(top / 127.f, kLargestScale) : numbers ? 0.f : __uint_as_float(0x7fc00000u);
    to_codes = plain ? 127.f / top : 0.f;
  }
  // The code is the low byte.  With 1.5 * 2^23 added, a number's low bits are those of the nearest whole one, ties to the even one; the product is
  // rounded first (the compiler would make one fma of the two, which could decide a tie otherwise).
  __device__ __forceinline__ uint32_t code_bits(float v) const {
    float r;
    asm("v_add_f32 %0, %1, %2" : "=v"(r) : "s"(12582912.f), "v"(v * to_codes));
    return __float_as_uint(r);
  }
  __device__ __forceinline__ int8_t code(float v) const { return plain ? (int8_t)code_bits(v) : (int8_t)0; }
  // (what is not plain may be no number: its bits are cleared)
  template <int V> __device__ __forceinline__ typename Codes<V>::type codes(const float (&v)[V]) const {
    typename Codes<V>::type p;
    if constexpr (V == 1) p = (uint8_t)code(v[0]);
    else if constexpr (V == 4) {
      const uint32_t low = __builtin_amdgcn_perm(code_bits(v[1]), code_bits(v[0]), 0x0c0c0400u);
      const uint32_t high = __builtin_amdgcn_perm(code_bits(v[3]), code_bits(v[2]), 0x0c0c0400u);
      p = plain ? __builtin_amdgcn_perm(high, low, 0x05040100u) : 0u;
    } else {
#pragma unroll
      for (int k = 0; k < V; k += 4) {
        const float four[4] = {v[k], v[k + 1], v[k + 2], v[k + 3]};
        p[k / 4] = codes<4>(four);
      }
    }
    return p;
  }
};

// 16 bytes less their first `bits` bits, zeros behind them.
template <typename P> __device__ __forceinline__ P shifted(P p, int bits) {
  typedef uint64_t Two __attribute__((ext_vector_type(2)));
  Two v = __builtin_bit_cast(Two, p);
  if (bits >= 64) v = Two{v.y >> (bits - 64), 0};
  else if (bits > 0) v = Two{v.x >> bits | v.y << (64 - bits), v.y >> bits};
  return __builtin_bit_cast(P, v);
}

// Results on their way out.  Where a call writes more rows of whole cache lines than half of the 256 MB of the memory-side cache, they are marked to
// leave the caches first, so that its other rows stay: a norm of 800,000 rows of 192 bf16 that also writes its sum 235 -> 229 us, with the call that
// reads the results 362 -> 346; 200,000 rows of 384 read back from 8 bits 46 -> 37.5.  Of fewer, the next call finds them there: two norms of
// 100,000 rows one after the other 48.7 us, marked 51.3.
template <typename P> __device__ __forceinline__ void write_out(P* to, P p, bool leaves) {
  if (leaves) {
    asm volatile("");                             // (else the compiler makes one plain store of both)
    __builtin_nontemporal_store(p, to);
    asm volatile("");
  } else *to = p;
}
// all: addresses and strides in bytes of the results, joined
inline bool leaves_caches(uintptr_t all, int64_t n, int32_t C, int arrays, int elem) {
  return (all & 127u) == 0 && n * C * arrays * elem > (128 << 20);
}

// The pieces of one row that a lane holds: piece r is number r * kLanes + part, past the row's end zero.  kLoose: rows begin on any value, and the last
// piece may hold fewer than V of them (a row holds V at least); it is read so that it ends with the row, shifted, and written value by value.  Of
// the first whole_pieces() every lane has a whole one, as launch_form takes no more pieces a lane than it has to, but for four where three would do and so on.
template <int kLanes, int R> constexpr int whole_pieces() { return kLanes == kThreads && R >= kVectors ? R - 2 : R - 1; }
template <typename T, int V, int kLanes, int R, bool kLoose> struct RowOf {
  typedef typename Piece<T, V>::type P;
  typedef T Anywhere __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  P p[R];
  __device__ __forceinline__ void load(const void* base, int64_t at, int part, int C) {
    const T* row = static_cast<const T*>(base) + at;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int first = (r * kLanes + part) * V;
      P zero = {};
      if constexpr (!kLoose) p[r] = first < C ? *reinterpret_cast<const P*>(row + first) : zero;
      else if (r < whole_pieces<kLanes, R>()) p[r] = *reinterpret_cast<const Anywhere*>(row + first);
      else {
        const int past = first < C && first + V > C ? first + V - C : 0;
        p[r] = first < C ? (P)*reinterpret_cast<const Anywhere*>(row + (first - past)) : zero;
        if (past) p[r] = shifted<P>(p[r], 8 * (int)sizeof(T) * past);
      }
    }
  }
  __device__ __forceinline__ static void store(void* base, int64_t at, int part, int C, const float (&f)[R][V], bool leaves) {
    T* row = static_cast<T*>(base) + at;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int first = (r * kLanes + part) * V;
      const P q = narrow<T, V>(f[r]);
      if constexpr (!kLoose) {
        if (first < C) write_out(reinterpret_cast<P*>(row + first), q, leaves);
      } else if (r < whole_pieces<kLanes, R>() || first + V <= C) *reinterpret_cast<Anywhere*>(row + first) = q;
      else {
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
          if (first + i < C) row[first + i] = q[i];
      }
    }
  }
};
template <int V, int kLanes, int R, bool kLoose> __device__ __forceinline__ void load_values(const float* v, int part, int C, float (&f)[R][V]) {
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int first = (r * kLanes + part) * V, at = kLoose ? first + i : first;
      f[r][i] = at < C ? v[first + i] : 0.f;
    }
}

// What pieces a call's rows go in: of 16 bytes, if all rows begin on 16 and are whole pieces (kPieces) or begin and end on any value (kLooseEnds: norm
// backward of 300,000 rows of 191 bf16 464 us in values, 104 in pieces, of 192 91); rows of fewer values than a piece value by value.
enum RowForm { kPieces, kLooseEnds, kValues };
inline RowForm row_form(uintptr_t all, int32_t C, int e) { return C * e < 16 ? kValues : (all & 15u) == 0 && C * e % 16 == 0 ? kPieces : kLooseEnds; }
// Lanes of a row, none if registers do not hold it: a lane takes 32 values at most, which are eight pieces in 32 bits (8,000 rows of 8,192, norm backward:
// 1,007 us read again, 204 held).  Rows of four pieces at most take four lanes (2,000,000 of 32 bf16, GELU 122 -> 64 us).
inline int form_lanes(RowForm form, int32_t C, int e) {
  const int32_t pieces = (int32_t)dsvt_ceil_div(C, 16 / e);
  return form == kValues ? 8 : pieces <= 4 ? 4 : e == 4 && pieces > kThreads * kVectors && pieces <= 2 * kThreads * kVectors ? kThreads : row_lanes(pieces, 16);
}
template <typename Kernel, typename T, typename Args> void launch_form(const Args& a, int lanes, unsigned groups, hipStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);
  if constexpr (sizeof(T) == 4) {
    const int64_t r = dsvt_ceil_div(dsvt_ceil_div(a.C, V), lanes);
    if (r > kVectors && r <= 6) return Kernel::template rows<T, V, kThreads, 6>(a, groups, st);
    if (r > 6) return Kernel::template rows<T, V, kThreads, 2 * kVectors>(a, groups, st);
  }
  if (lanes == 4) Kernel::template rows<T, V, 4, 1>(a, groups, st);
  else launch_pieces<Kernel, T, V>(a, lanes, groups, st);
}
// Launches Kernel<kLoose>::rows<T, V, kLanes, R>(a, groups, st).
template <template <bool> class Kernel, typename T, typename Args> void launch_form(const Args& a, RowForm form, int lanes, unsigned groups, hipStream_t st) {
  if (form == kPieces) launch_form<Kernel<false>, T>(a, lanes, groups, st);
  else if (form == kLooseEnds) launch_form<Kernel<true>, T>(a, lanes, groups, st);
  else Kernel<false>::template rows<T, 1, 8, 1>(a, groups, st);
}

// The row's pieces v in 8 bits: what its kLanes lanes hold of it goes to `codes`, its scale to *scale.
template <int V, int kLanes, int R, bool kLoose>
__device__ __forceinline__ void store_codes(const float (&v)[R][V], int part, int C, int8_t* codes, float* scale, uint32_t* s) {
  float top = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if constexpr (V == 1) top = largest_size(top, v[r][0], v[r][0]);
    else {
#pragma unroll
      for (int i = 0; i < V; i += 2) top = largest_size(top, v[r][i], v[r][i + 1]);
    }
  }
  const RowScale by(lane_join<kLanes>(size_bits(top), s, [](uint32_t a, uint32_t b) { return a > b ? a : b; }));
  if (part == 0) *scale = by.scale;
  typedef typename Codes<V>::type P;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int first = (r * kLanes + part) * V;
    const P q = by.template codes<V>(v[r]);
    if (!kLoose ? first < C : r < whole_pieces<kLanes, R>() || first + V <= C) *reinterpret_cast<P*>(codes + first) = q;
    else if constexpr (kLoose) {
#pragma unroll
      for (int i = 0; i < V - 1; ++i)
        if (first + i < C) codes[first + i] = byte_of(q, i);
    }
  }
}

// GELU, x Phi(x), and its slope Phi(x) + x phi(x).  Phi(-|x|) = phi-like exponential times a polynomial of 1 / (1 + p z), z = |x| / sqrt 2
// (Abramowitz & Stegun 7.1.26, off by at most 1.5e-7 in erf and so 7.5e-8 in Phi); the slope needs the same exponential.
struct Normal {
  float below, density;                           // Phi(-|x|), phi(x)
  __device__ __forceinline__ explicit Normal(float x) {
    const float e = __builtin_amdgcn_exp2f(x * x * -0.72134752044448170368f);             // exp(-x^2 / 2)
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.3275911f * 0.70710678118654752440f, 1.f));
    float p = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
    p = fmaf(t, p, 0.5f * 1.421413741f);
    p = fmaf(t, p, 0.5f * -0.284496736f);
    p = fmaf(t, p, 0.5f * 0.254829592f);
    below = t * p * e;
    density = e * 0.39894228040143267794f;
  }
};
__device__ __forceinline__ float gelu(float x) {
  const float positive = x < 0.f ? 0.f : x;       // (a NaN stays one)
  return fmaf(-fabsf(x), Normal(x).below, positive);
}
__device__ __forceinline__ float gelu_slope(float x) {
  const Normal n(x);
  return fmaf(x, n.density, x < 0.f ? n.below : 1.f - n.below);
}

// n rows of C codes and their scales.  Rows of `ld` bytes, begin on 16.
inline bool bad_rows8(const dsvt_rows8* r, int32_t C) {
  return !r || !r->codes || !r->scale || ((uintptr_t)r->codes & 15u) != 0 || ((uintptr_t)r->scale & 3u) != 0 || r->ld < C || r->ld % 16 != 0;
}
}  // namespace
