// What kernels that go over rows share (norm.hip, rms.hip, rows8.hip): a row sits in the registers of kLanes neighbouring lanes (4 to 64, or a
// workgroup's 256), in pieces of up to 16 bytes; sums over a row across lanes; which pieces and lanes a call's rows take.
#pragma once
#include "common.h"
#include "mma.h"

namespace {

constexpr int kThreads = 256;
constexpr int kVectors = 4;                       // 16-byte pieces of a row in one lane, at most (of the longest rows of 32 bits twice as many: rows8.h)
constexpr int narrow_max(int bytes) { return bytes == 8 ? 8 : 16; }      // and smaller ones
constexpr int kBackwardGroups = 512;              // workgroups of a pass that sums over rows, at most: two a compute unit
constexpr int kForwardGroups = 2048;

template <typename T, int V> struct Piece { typedef T type __attribute__((ext_vector_type(V))); };
template <typename T> struct Piece<T, 1> { typedef T type; };

template <typename T, int V> __device__ __forceinline__ void widen(const typename Piece<T, V>::type& p, float (&f)[V]) {
  if constexpr (V == 1) f[0] = (float)p;
  else {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = (float)p[i];
  }
}
template <typename T, int V> __device__ __forceinline__ typename Piece<T, V>::type narrow(const float (&f)[V]) {
  typename Piece<T, V>::type p;
  if constexpr (V == 1) p = (T)f[0];
  else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = (T)f[i];
  }
  return p;
}

// A value combined over kLanes neighbouring lanes, or over the workgroup (kLanes = kThreads, `s` holds a value per wavefront); every lane gets it.
template <int kLanes, typename V, typename Op> __device__ __forceinline__ V lane_join(V v, V* s, Op op) {
#pragma unroll
  for (int d = 1; d < (kLanes < 64 ? kLanes : 64); d *= 2) v = op(v, __shfl_xor(v, d, 64));
  if constexpr (kLanes > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s[0];
#pragma unroll
    for (int k = 1; k < kThreads / 64; ++k) v = op(v, s[k]);
  }
  return v;
}
template <int kLanes> __device__ __forceinline__ float lane_sum(float v, float* s) {
  return lane_join<kLanes>(v, s, [](float a, float b) { return a + b; });
}

// The pieces of one row that a lane holds: piece r is number r * kLanes + lane, past the row's end zero.
template <typename T, int V, int kLanes, int R> struct RowPieces {
  typedef typename Piece<T, V>::type P;
  P p[R];
  __device__ __forceinline__ void load(const void* base, int64_t at, int part, int pieces, bool there) {
    const P* row = reinterpret_cast<const P*>(static_cast<const T*>(base) + at);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      P zero = {};
      p[r] = there && r * kLanes + part < pieces ? row[r * kLanes + part] : zero;
    }
  }
};

template <int V, int kLanes, int R>
__device__ __forceinline__ void load_vector(const float* v, int part, int pieces, float (&f)[R][V]) {
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) f[r][i] = r * kLanes + part < pieces ? v[(r * kLanes + part) * V + i] : 0.f;
}

// The widest pieces of 16, 8, 4 or 2 bytes on which every row of every array starts and of which C is a whole number (`all`: the addresses and the
// strides in bytes of the arrays, joined); then the fewest lanes a row that hold it.  0: none do.
inline int piece_elems(uintptr_t all, int32_t C, int e) {
  for (int bytes = 16; bytes > e; bytes /= 2)
    if (C % (bytes / e) == 0 && (all & (uintptr_t)(bytes - 1)) == 0) return bytes / e;
  return 1;
}
inline int row_lanes(int32_t pieces, int bytes) {
  for (int l = 8; l <= 64; l *= 2)
    if (pieces <= l * kVectors) return l;
  return bytes == 16 ? (pieces <= kThreads * kVectors ? kThreads : 0) : (pieces <= 64 * narrow_max(bytes) ? 64 : 0);
}

// Launches Kernel::rows<T, V, kLanes, R>(a, groups, st) for rows of a.C values in pieces of V on `lanes` lanes, as piece_elems and row_lanes say.
template <typename Kernel, typename T, int V, typename Args> void launch_pieces(const Args& a, int lanes, unsigned groups, hipStream_t st) {
  const int r = (int)dsvt_ceil_div(dsvt_ceil_div(a.C, V), lanes);
  if (lanes == 8) {
    if (r == 1) Kernel::template rows<T, V, 8, 1>(a, groups, st);
    else if (r == 2) Kernel::template rows<T, V, 8, 2>(a, groups, st);
    else if (r == 3) Kernel::template rows<T, V, 8, 3>(a, groups, st);
    else Kernel::template rows<T, V, 8, 4>(a, groups, st);
  } else if (lanes == 16) {                       // more than 4 * 8 pieces: three or four of 16 lanes, and so on
    if (r == 3) Kernel::template rows<T, V, 16, 3>(a, groups, st);
    else Kernel::template rows<T, V, 16, 4>(a, groups, st);
  } else if (lanes == 32) {
    if (r == 3) Kernel::template rows<T, V, 32, 3>(a, groups, st);
    else Kernel::template rows<T, V, 32, 4>(a, groups, st);
  } else if (lanes == 64) {
    if (r == 3) Kernel::template rows<T, V, 64, 3>(a, groups, st);
    else if (r == 4) Kernel::template rows<T, V, 64, 4>(a, groups, st);
    else if constexpr (V * sizeof(T) < 16) {
      if (r <= 6) Kernel::template rows<T, V, 64, 6>(a, groups, st);
      else if (r <= 8) Kernel::template rows<T, V, 64, 8>(a, groups, st);
      else if constexpr (V * sizeof(T) < 8) {
        if (r <= 12) Kernel::template rows<T, V, 64, 12>(a, groups, st);
        else Kernel::template rows<T, V, 64, 16>(a, groups, st);
      }
    }
  } else if constexpr (V * sizeof(T) == 16) {
    if (r <= 2) Kernel::template rows<T, V, kThreads, 2>(a, groups, st);
    else Kernel::template rows<T, V, kThreads, kVectors>(a, groups, st);
  }
}
template <typename Kernel, typename T, typename Args> void launch_rows(const Args& a, int v, int lanes, unsigned groups, hipStream_t st) {
  if (v == 1) launch_pieces<Kernel, T, 1>(a, lanes, groups, st);
  else if (v == 2) launch_pieces<Kernel, T, 2>(a, lanes, groups, st);
  else if (v * sizeof(T) == 8) launch_pieces<Kernel, T, 8 / (int)sizeof(T)>(a, lanes, groups, st);
  else launch_pieces<Kernel, T, 16 / (int)sizeof(T)>(a, lanes, groups, st);
}

inline bool bad_rows(const void* p, int64_t ld, int32_t C, int e) { return !p || ((uintptr_t)p % (uintptr_t)e) != 0 || ld < C; }

}  // namespace
