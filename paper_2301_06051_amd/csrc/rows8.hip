// Rows in 8 bits (rows8.h): dsvt_keep_rows8 writes them, dsvt_read_rows8 reads them back; dsvt_gelu_rows8 and dsvt_gelu_rows8_backward
// are the activation of an MLP whose input is kept in 8 bits for the backward pass.
//
//   forward   out = codes of gelu(h), kept = codes of h          gelu(h) = h Phi(h)
//   backward  dh = dy (Phi(k) + k phi(k)), k = code * scale
//
// All are bound by the bytes of their rows: writers hold a row in registers (rows.h), as its largest value is wanted before its first code; 27
// instructions a value of GELU into two sets of codes take as long as its bytes.  Rows of 384 bf16: 200,000 through GELU into both sets of codes 72 us (4.3
// TB/s), read back 37.5 (6.1, the codes from the caches), 800,000 backward 284 (5.4).  Fetching the next row ahead: 78 instead of 74.
#include "rows8.h"

namespace {

struct Rows8Args {
  const void *x, *dy;                             // rows of the type: writers' input; dy of the backward pass
  void* y;                                        // readers' output
  int8_t *out, *kept;                             // writers: codes of gelu(x) (or of x itself) and of x; either may be null.  Readers: kept
  float *out_scale, *kept_scale;
  int64_t ld_x, ld_dy, ld_y, ld_out, ld_kept;
  int32_t n, C;
  bool leaves;                                    // readers: write_out
};

template <bool kGelu, typename T, int V, int kLanes, int R, bool kLoose>
__global__ __launch_bounds__(kThreads) void k_write_rows8(Rows8Args a) {
  constexpr int kRows = kThreads / kLanes;
  __shared__ uint32_t s[kThreads / 64];
  const int part = threadIdx.x % kLanes;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes; row < a.n; row += (int64_t)gridDim.x * kRows) {
    RowOf<T, V, kLanes, R, kLoose> x;
    x.load(a.x, row * a.ld_x, part, a.C);
    float v[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r) widen<T, V>(x.p[r], v[r]);
    if (a.kept) store_codes<V, kLanes, R, kLoose>(v, part, a.C, a.kept + row * a.ld_kept, a.kept_scale + row, s);
    if constexpr (kGelu) {
      if (!a.out) continue;
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) v[r][i] = gelu(v[r][i]);
      store_codes<V, kLanes, R, kLoose>(v, part, a.C, a.out + row * a.ld_out, a.out_scale + row, s);
    }
  }
}

// Rows that registers do not hold: a workgroup a row, read twice.
template <bool kGelu, typename T> __global__ __launch_bounds__(kThreads) void k_write_rows8_long(Rows8Args a) {
  __shared__ uint32_t s[2][kThreads / 64];
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
    uint32_t top = 0, top_out = 0;
    const auto larger = [](uint32_t p, uint32_t q) { return p > q ? p : q; };
    for (int c = threadIdx.x; c < a.C; c += kThreads) {
      const float v = (float)x[c];
      top = larger(top, size_bits(v));
      if constexpr (kGelu) top_out = larger(top_out, size_bits(gelu(v)));
    }
    const RowScale by(lane_join<kThreads>(top, s[0], larger)), by_out(lane_join<kThreads>(top_out, s[1], larger));
    if (threadIdx.x == 0) {
      if (a.kept) a.kept_scale[row] = by.scale;
      if (kGelu && a.out) a.out_scale[row] = by_out.scale;
    }
    for (int c = threadIdx.x; c < a.C; c += kThreads) {
      const float v = (float)x[c];
      if (a.kept) a.kept[row * a.ld_kept + c] = by.code(v);
      if (kGelu && a.out) a.out[row * a.ld_out + c] = by_out.code(gelu(v));
    }
  }
}

// kLanes lanes go along a row of any length.
template <bool kGelu, typename T, int V, int kLanes, bool kLoose> __global__ __launch_bounds__(kThreads) void k_read_rows8(Rows8Args a) {
  constexpr int kAtOnce = kGelu ? 2 : 1;          // pieces asked for before one is used: 800,000 rows of 384 backward 289 us with one, 284 with two
  constexpr int kRows = kThreads / kLanes;
  typedef RowOf<T, V, 1, 1, kLoose> Row;          // (a piece by itself)
  typedef typename Codes<V>::type Q;
  const int part = threadIdx.x % kLanes, pieces = (a.C + V - 1) / V;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes; row < a.n; row += (int64_t)gridDim.x * kRows) {
    const Q* codes = reinterpret_cast<const Q*>(a.kept + row * a.ld_kept);
    const float scale = a.kept_scale[row];
    for (int p0 = part; p0 < pieces; p0 += kAtOnce * kLanes) {
      Q q[kAtOnce];
      Row d[kGelu ? kAtOnce : 1];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int p = p0 + u * kLanes < pieces ? p0 + u * kLanes : p0;
        q[u] = codes[p];
        if constexpr (kGelu) d[u].load(a.dy, row * a.ld_dy, p, a.C);
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int p = p0 + u * kLanes;
        if (p >= pieces) break;
        float f[1][V];
        values_of<V>(q[u], scale, f[0]);
        if constexpr (kGelu) {
          float g[V];
          widen<T, V>(d[u].p[0], g);
#pragma unroll
          for (int i = 0; i < V; ++i) f[0][i] = g[i] * gelu_slope(f[0][i]);
        }
        Row::store(a.y, row * a.ld_y, p, a.C, f, a.leaves);
      }
    }
  }
}

// The same for rows that begin and end on any value: a lane asks for all its pieces before it uses one.
template <bool kGelu, typename T, int V, int kLanes, int R> __global__ __launch_bounds__(kThreads) void k_read_rows8_loose(Rows8Args a) {
  constexpr int kRows = kThreads / kLanes;
  typedef RowOf<T, V, kLanes, R, true> Row;
  typedef typename Codes<V>::type Q;
  const int part = threadIdx.x % kLanes, last = (a.C - 1) / V * V;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes; row < a.n; row += (int64_t)gridDim.x * kRows) {
    const int8_t* codes = a.kept + row * a.ld_kept;
    const float scale = a.kept_scale[row];
    Q q[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int first = (r * kLanes + part) * V;
      q[r] = *reinterpret_cast<const Q*>(codes + (first < last ? first : last));
    }
    Row d;
    if constexpr (kGelu) d.load(a.dy, row * a.ld_dy, part, a.C);
    float f[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      values_of<V>(q[r], scale, f[r]);
      if constexpr (kGelu) {
        float g[V];
        widen<T, V>(d.p[r], g);
#pragma unroll
        for (int i = 0; i < V; ++i) f[r][i] = g[i] * gelu_slope(f[r][i]);
      }
    }
    Row::store(a.y, row * a.ld_y, part, a.C, f, false);
  }
}

template <bool kGelu> struct Read {
  template <typename T, int V, int kLanes, int R> static void rows(const Rows8Args& a, unsigned groups, hipStream_t st) {
    k_read_rows8_loose<kGelu, T, V, kLanes, R><<<groups, kThreads, 0, st>>>(a);
  }
};
template <bool kGelu> struct Write {
  template <bool kLoose> struct Kernel {
    template <typename T, int V, int kLanes, int R> static void rows(const Rows8Args& a, unsigned groups, hipStream_t st) {
      k_write_rows8<kGelu, T, V, kLanes, R, kLoose><<<groups, kThreads, 0, st>>>(a);
    }
  };
};
template <bool kGelu, typename T> void launch_write(const Rows8Args& a, RowForm form, int lanes, unsigned groups, hipStream_t st) {
  if (lanes == 0) k_write_rows8_long<kGelu, T><<<groups, kThreads, 0, st>>>(a);
  else launch_form<Write<kGelu>::template Kernel, T>(a, form, lanes, groups, st);
}
template <bool kGelu, typename T, int V, int kLanes, bool kLoose> void launch_read(const Rows8Args& a, hipStream_t st) {
  const int64_t all = dsvt_ceil_div(a.n, kThreads / kLanes);
  k_read_rows8<kGelu, T, V, kLanes, kLoose><<<(unsigned)(all < 2 * kForwardGroups ? all : 2 * kForwardGroups), kThreads, 0, st>>>(a);
}
template <bool kGelu, typename T> void launch_read(const Rows8Args& a, RowForm form, hipStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);
  if (form == kPieces) {
    int lanes = a.C <= 4 * V ? 4 : 8;
    while (lanes > 4 && lanes < 64 && lanes * 4 < a.C / V) lanes *= 2;
    if (lanes == 4) launch_read<kGelu, T, V, 4, false>(a, st);
    else if (lanes == 8) launch_read<kGelu, T, V, 8, false>(a, st);
    else if (lanes == 16) launch_read<kGelu, T, V, 16, false>(a, st);
    else if (lanes == 32) launch_read<kGelu, T, V, 32, false>(a, st);
    else launch_read<kGelu, T, V, 64, false>(a, st);
  } else if (form == kLooseEnds) {
    const int lanes = form_lanes(form, a.C, sizeof(T));
    const int64_t all = dsvt_ceil_div(a.n, lanes ? kThreads / lanes : 1);
    if (lanes == 0) launch_read<kGelu, T, V, 64, true>(a, st);   // (longer ones)
    else launch_form<Read<kGelu>, T>(a, lanes, (unsigned)(all < kForwardGroups ? all : kForwardGroups), st);
  } else launch_read<kGelu, T, 1, 8, false>(a, st);
}

int check(int32_t C, int32_t dtype, int32_t n_rows) {
  if (C <= 0 || n_rows < 0 || (dtype != DSVT_F32 && dtype != DSVT_BF16)) return DSVT_EINVAL;
  return C > DSVT_LN_MAX_C ? DSVT_EUNSUPPORTED : DSVT_OK;
}

int write(bool with_gelu, int32_t C, int32_t dtype, const void* x, int64_t ld_x, int32_t n_rows, const dsvt_rows8* out, const dsvt_rows8* kept,
          void* stream) {
  if (const int rc = check(C, dtype, n_rows)) return rc;
  if (n_rows == 0) return DSVT_OK;
  const int e = dtype == DSVT_BF16 ? 2 : 4;
  if (bad_rows(x, ld_x, C, e) || (!out && !kept) || (out && bad_rows8(out, C)) || (kept && bad_rows8(kept, C))) return DSVT_EINVAL;
  if (out && kept && (out->codes == kept->codes || out->scale == kept->scale)) return DSVT_EINVAL;
  Rows8Args a = {};
  a.x = x; a.ld_x = ld_x; a.n = n_rows; a.C = C;
  if (out) { a.out = out->codes; a.out_scale = out->scale; a.ld_out = out->ld; }
  if (kept) { a.kept = kept->codes; a.kept_scale = kept->scale; a.ld_kept = kept->ld; }
  const RowForm form = row_form((uintptr_t)x | (uintptr_t)(ld_x * e), C, e);
  const int lanes = form_lanes(form, C, e);
  const int64_t all = dsvt_ceil_div(n_rows, lanes ? kThreads / lanes : 1);
  const unsigned groups = (unsigned)(all < kForwardGroups ? all : kForwardGroups);
  hipStream_t st = (hipStream_t)stream;
  {
    dsvt_prof_scope ps(DSVT_K_ROWS8_WRITE, st);
    if (dtype == DSVT_BF16) with_gelu ? launch_write<true, bf16_t>(a, form, lanes, groups, st) : launch_write<false, bf16_t>(a, form, lanes, groups, st);
    else with_gelu ? launch_write<true, float>(a, form, lanes, groups, st) : launch_write<false, float>(a, form, lanes, groups, st);
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}

int read(bool with_gelu, int32_t C, int32_t dtype, const dsvt_rows8* kept, const void* dy, int64_t ld_dy, int32_t n_rows, void* y, int64_t ld_y,
         void* stream) {
  if (const int rc = check(C, dtype, n_rows)) return rc;
  if (n_rows == 0) return DSVT_OK;
  const int e = dtype == DSVT_BF16 ? 2 : 4;
  if (bad_rows8(kept, C) || bad_rows(y, ld_y, C, e) || (with_gelu && bad_rows(dy, ld_dy, C, e))) return DSVT_EINVAL;
  Rows8Args a = {};
  a.dy = dy; a.ld_dy = ld_dy; a.y = y; a.ld_y = ld_y; a.kept = kept->codes; a.kept_scale = kept->scale; a.ld_kept = kept->ld; a.n = n_rows; a.C = C;
  const RowForm form = row_form((uintptr_t)dy | (uintptr_t)y | (uintptr_t)((ld_dy | ld_y) * e), C, e);
  a.leaves = leaves_caches((uintptr_t)y | (uintptr_t)(ld_y * e), n_rows, C, 1, e);
  hipStream_t st = (hipStream_t)stream;
  {
    dsvt_prof_scope ps(DSVT_K_ROWS8_READ, st);
    if (dtype == DSVT_BF16) with_gelu ? launch_read<true, bf16_t>(a, form, st) : launch_read<false, bf16_t>(a, form, st);
    else with_gelu ? launch_read<true, float>(a, form, st) : launch_read<false, float>(a, form, st);
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}

}  // namespace

extern "C" int dsvt_keep_rows8(int32_t C, int32_t dtype, const void* x, int64_t ld_x, int32_t n_rows, const dsvt_rows8* kept, void* stream) {
  return write(false, C, dtype, x, ld_x, n_rows, nullptr, kept, stream);
}
extern "C" int dsvt_gelu_rows8(int32_t C, int32_t dtype, const void* h, int64_t ld_h, int32_t n_rows, const dsvt_rows8* out,
                               const dsvt_rows8* kept, void* stream) {
  return write(true, C, dtype, h, ld_h, n_rows, out, kept, stream);
}
extern "C" int dsvt_read_rows8(int32_t C, int32_t dtype, const dsvt_rows8* rows, int32_t n_rows, void* x, int64_t ld_x, void* stream) {
  return read(false, C, dtype, rows, nullptr, 0, n_rows, x, ld_x, stream);
}
extern "C" int dsvt_gelu_rows8_backward(int32_t C, int32_t dtype, const dsvt_rows8* kept, const void* dy, int64_t ld_dy, int32_t n_rows, void* dh,
                                        int64_t ld_dh, void* stream) {
  return read(true, C, dtype, kept, dy, ld_dy, n_rows, dh, ld_dh, stream);
}
