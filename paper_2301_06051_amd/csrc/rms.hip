// dsvt_rms_norm / dsvt_rms_norm_backward: the root-mean-square norm of a residual sum, with its gradients.
//
//   forward   z = x + res, n = z * rsqrt(mean z^2 + eps), y = n * gamma, as rows of the type, in 8 bits (rows8.h), or both
//   backward  w = dy * gamma, dx = rsqrt(mean z^2 + eps) * (w - n * mean(w * n)) + d_sum, d_gamma = sum of dy * n over the rows
//
// Both passes are bound by the bytes of their rows, which sit in registers and are read once (rows.h).  The sum z is formed again in the backward pass if
// it was not written, and its gradient d_sum, which comes past the branch, is added in the same pass.  800,000 rows of 192 bf16 with a branch: forward
// with y and z 228 us (5.4 TB/s), backward with d_sum 287 (5.3); 30,000 rows backward 15.4 with 512 workgroups, 18.4 with 768, 19.0 with 1,024.
#include "rows8.h"
#include "sum_parts.h"

namespace {

struct RmsArgs {
  const void *x, *res, *dy, *d_sum;               // res, d_sum: may be null; dy, d_sum: backward only
  void *z, *y;                                    // forward: either may be null; backward: y is dx
  int8_t* codes;                                  // forward: may be null
  float* scale;
  const float* gamma;
  float *partial, *d_gamma;                       // [groups][C]; d_gamma: null when partial sums are to be added up by k_sum_parts
  int64_t ld_x, ld_res, ld_dy, ld_dsum, ld_z, ld_y, ld_codes;
  int32_t n, C;
  float eps;
  bool leaves;                                    // write_out
};

// z = x + res in 32 bits; returns rsqrt(mean z^2 + eps)
template <typename T, int V, int kLanes, int R, bool kLoose>
__device__ __forceinline__ float sum_row(const RowOf<T, V, kLanes, R, kLoose>& x, const RowOf<T, V, kLanes, R, kLoose>& res, bool with_res, float inv_c,
                                         float eps, float (&z)[R][V], float* s) {
  float sq = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    widen<T, V>(x.p[r], z[r]);
    if (with_res) {
      float f[V];
      widen<T, V>(res.p[r], f);
#pragma unroll
      for (int i = 0; i < V; ++i) z[r][i] += f[i];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) sq = fmaf(z[r][i], z[r][i], sq);
  }
  return 1.f / sqrtf(lane_sum<kLanes>(sq, s) * inv_c + eps);
}

template <typename T, int V, int kLanes, int R, bool kLoose>
__global__ __launch_bounds__(kThreads) void k_rms_forward(RmsArgs a) {
  typedef RowOf<T, V, kLanes, R, kLoose> Row;
  constexpr int kRows = kThreads / kLanes;
  __shared__ float s[kThreads / 64];
  __shared__ uint32_t st[kThreads / 64];
  const int part = threadIdx.x % kLanes;
  const float inv_c = 1.f / (float)a.C;
  float gamma[R][V];
  load_values<V, kLanes, R, kLoose>(a.gamma, part, a.C, gamma);
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes; row < a.n; row += (int64_t)gridDim.x * kRows) {
    Row x, res;
    x.load(a.x, row * a.ld_x, part, a.C);
    if (a.res) res.load(a.res, row * a.ld_res, part, a.C);
    float z[R][V];
    const float rs = sum_row<T, V, kLanes, R, kLoose>(x, res, a.res != nullptr, inv_c, a.eps, z, s);
    if (a.z) Row::store(a.z, row * a.ld_z, part, a.C, z, a.leaves);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < V; ++i) z[r][i] *= rs * gamma[r][i];
    if (a.y) Row::store(a.y, row * a.ld_y, part, a.C, z, a.leaves);
    if (a.codes) store_codes<V, kLanes, R, kLoose>(z, part, a.C, a.codes + row * a.ld_codes, a.scale + row, st);
  }
}

template <typename T, int V, int kLanes, int R, bool kLoose>
__global__ __launch_bounds__(kThreads) void k_rms_backward(RmsArgs a) {
  typedef RowOf<T, V, kLanes, R, kLoose> Row;
  constexpr int kRows = kThreads / kLanes;
  __shared__ float s[kThreads / 64];
  const int part = threadIdx.x % kLanes;
  const float inv_c = 1.f / (float)a.C;
  float gamma[R][V], dg[R][V] = {};
  load_values<V, kLanes, R, kLoose>(a.gamma, part, a.C, gamma);
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes; row < a.n; row += (int64_t)gridDim.x * kRows) {
    Row x, res, dy, more;
    x.load(a.x, row * a.ld_x, part, a.C);
    if (a.res) res.load(a.res, row * a.ld_res, part, a.C);
    dy.load(a.dy, row * a.ld_dy, part, a.C);
    if (a.d_sum) more.load(a.d_sum, row * a.ld_dsum, part, a.C);
    float n[R][V], w[R][V];
    const float rs = sum_row<T, V, kLanes, R, kLoose>(x, res, a.res != nullptr, inv_c, a.eps, n, s);
    float sum_wn = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      widen<T, V>(dy.p[r], w[r]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        n[r][i] *= rs;
        dg[r][i] = fmaf(w[r][i], n[r][i], dg[r][i]);
        w[r][i] *= gamma[r][i];
        sum_wn = fmaf(w[r][i], n[r][i], sum_wn);
      }
    }
    const float mean_wn = lane_sum<kLanes>(sum_wn, s) * inv_c;
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 0; i < V; ++i) n[r][i] = rs * (w[r][i] - n[r][i] * mean_wn);
      if (a.d_sum) {
        float f[V];
        widen<T, V>(more.p[r], f);
#pragma unroll
        for (int i = 0; i < V; ++i) n[r][i] += f[i];
      }
    }
    Row::store(a.y, row * a.ld_y, part, a.C, n, a.leaves);
  }
  // the workgroup's sums: over the rows of a wavefront across lanes, over its wavefronts in LDS
  constexpr int kCopies = kLanes > 64 ? 1 : kThreads / 64;
  __shared__ float sums[kCopies][kLanes * R * V];
  const int lane = threadIdx.x & 63, copy = kLanes > 64 ? 0 : threadIdx.x >> 6;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int d = kLanes; d < 64; d *= 2) dg[r][i] += __shfl_xor(dg[r][i], d, 64);
      if (lane < kLanes || kLanes > 64) sums[copy][(r * kLanes + part) * V + i] = dg[r][i];
    }
  __syncthreads();
  for (int c = threadIdx.x; c < a.C; c += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kCopies; ++k) v += sums[k][c];
    if (a.d_gamma) a.d_gamma[c] = v;
    else a.partial[(int64_t)blockIdx.x * a.C + c] = v;
  }
}

template <typename T> __device__ __forceinline__ float sum_at(const RmsArgs& a, int64_t row, int c) {
  float z = (float)static_cast<const T*>(a.x)[row * a.ld_x + c];
  if (a.res) z += (float)static_cast<const T*>(a.res)[row * a.ld_res + c];
  return z;
}

// Rows that registers do not hold: a workgroup a row, which is read again, from the caches, for its sum, its largest value and its results.
// Workgroups take consecutive rows, `rows` of them.
template <typename T, bool kBackward>
__global__ __launch_bounds__(kThreads) void k_rms_long(RmsArgs a, int32_t rows) {
  __shared__ float s[kThreads / 64];
  __shared__ uint32_t st[kThreads / 64];
  const float inv_c = 1.f / (float)a.C;
  const int64_t first = (int64_t)blockIdx.x * rows, last = first + rows < a.n ? first + rows : a.n;
  float* part_g = kBackward ? (a.d_gamma ? a.d_gamma : a.partial + (int64_t)blockIdx.x * a.C) : nullptr;
  for (int64_t row = first; row < last; ++row) {
    float v = 0.f;
    for (int c = threadIdx.x; c < a.C; c += kThreads) {
      const float z = sum_at<T>(a, row, c);
      v = fmaf(z, z, v);
    }
    const float rs = 1.f / sqrtf(lane_sum<kThreads>(v, s) * inv_c + a.eps);
    if constexpr (kBackward) {
      const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
      float sum_wn = 0.f;
      for (int c = threadIdx.x; c < a.C; c += kThreads) sum_wn = fmaf((float)dy[c] * a.gamma[c], sum_at<T>(a, row, c) * rs, sum_wn);
      const float mean_wn = lane_sum<kThreads>(sum_wn, s) * inv_c;
      T* out = static_cast<T*>(a.y) + row * a.ld_y;
      const T* more = a.d_sum ? static_cast<const T*>(a.d_sum) + row * a.ld_dsum : nullptr;
      for (int c = threadIdx.x; c < a.C; c += kThreads) {
        const float d = (float)dy[c], n = sum_at<T>(a, row, c) * rs;
        float dx = rs * (d * a.gamma[c] - n * mean_wn);
        if (more) dx += (float)more[c];
        out[c] = (T)dx;
        part_g[c] = (row == first ? 0.f : part_g[c]) + d * n;     // a column is always the same thread's
      }
    } else {
      uint32_t top = 0;
      if (a.codes) {
        for (int c = threadIdx.x; c < a.C; c += kThreads) {
          const uint32_t b = size_bits(sum_at<T>(a, row, c) * (rs * a.gamma[c]));
          top = b > top ? b : top;
        }
        top = lane_join<kThreads>(top, st, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
      }
      const RowScale by(top);
      if (a.codes && threadIdx.x == 0) a.scale[row] = by.scale;
      for (int c = threadIdx.x; c < a.C; c += kThreads) {
        const float z = sum_at<T>(a, row, c), y = z * (rs * a.gamma[c]);
        if (a.z) static_cast<T*>(a.z)[row * a.ld_z + c] = (T)z;
        if (a.y) static_cast<T*>(a.y)[row * a.ld_y + c] = (T)y;
        if (a.codes) a.codes[row * a.ld_codes + c] = by.code(y);
      }
    }
  }
}

// Rows that one workgroup sums up by itself: a second launch takes longer than the three more turns of rows.
constexpr int kTurnsAlone = 4;

uintptr_t starts(const RmsArgs& a, int e) {
  return (uintptr_t)a.x | (uintptr_t)a.res | (uintptr_t)a.dy | (uintptr_t)a.d_sum | (uintptr_t)a.z | (uintptr_t)a.y |
         (uintptr_t)((a.ld_x | a.ld_res | a.ld_dy | a.ld_dsum | a.ld_z | a.ld_y) * e);
}

template <bool kLoose> struct Forward {
  template <typename T, int V, int kLanes, int R> static void rows(const RmsArgs& a, unsigned groups, hipStream_t st) {
    k_rms_forward<T, V, kLanes, R, kLoose><<<groups, kThreads, 0, st>>>(a);
  }
};
template <bool kLoose> struct Backward {
  template <typename T, int V, int kLanes, int R> static void rows(const RmsArgs& a, unsigned groups, hipStream_t st) {
    k_rms_backward<T, V, kLanes, R, kLoose><<<groups, kThreads, 0, st>>>(a);
  }
};
template <typename T> void launch(const RmsArgs& a, bool back, RowForm form, int lanes, unsigned groups, int32_t rows, hipStream_t st) {
  if (lanes == 0) {
    if (back) k_rms_long<T, true><<<groups, kThreads, 0, st>>>(a, rows);
    else k_rms_long<T, false><<<groups, kThreads, 0, st>>>(a, rows);
  } else if (back) launch_form<Backward, T>(a, form, lanes, groups, st);
  else launch_form<Forward, T>(a, form, lanes, groups, st);
}

int check(const dsvt_rms_cfg* cfg, int32_t n_rows) {
  if (!cfg || !cfg->gamma || cfg->C <= 0 || n_rows < 0) return DSVT_EINVAL;
  if (cfg->dtype != DSVT_F32 && cfg->dtype != DSVT_BF16) return DSVT_EINVAL;
  if (!(cfg->eps >= 0.f)) return DSVT_EINVAL;
  if (cfg->C > DSVT_LN_MAX_C) return DSVT_EUNSUPPORTED;
  return DSVT_OK;
}

}  // namespace

extern "C" int dsvt_rms_norm(const dsvt_rms_cfg* cfg, const void* x, int64_t ld_x, const void* res, int64_t ld_res, int32_t n_rows, void* z,
                             int64_t ld_z, void* y, int64_t ld_y, const dsvt_rows8* rows8, void* stream) {
  if (const int rc = check(cfg, n_rows)) return rc;
  if (n_rows == 0) return DSVT_OK;
  const int e = cfg->dtype == DSVT_BF16 ? 2 : 4;
  if ((!y && !rows8) || (z && z == y)) return DSVT_EINVAL;
  if (bad_rows(x, ld_x, cfg->C, e) || (res && bad_rows(res, ld_res, cfg->C, e)) || (z && bad_rows(z, ld_z, cfg->C, e)) ||
      (y && bad_rows(y, ld_y, cfg->C, e)) || (rows8 && bad_rows8(rows8, cfg->C))) return DSVT_EINVAL;
  RmsArgs a = {};
  a.x = x; a.res = res; a.z = z; a.y = y; a.gamma = cfg->gamma;
  a.ld_x = ld_x; a.ld_res = res ? ld_res : 0; a.ld_z = z ? ld_z : 0; a.ld_y = y ? ld_y : 0; a.n = n_rows; a.C = cfg->C; a.eps = cfg->eps;
  if (rows8) { a.codes = rows8->codes; a.scale = rows8->scale; a.ld_codes = rows8->ld; }
  const RowForm form = row_form(starts(a, e), a.C, e);
  const int lanes = form_lanes(form, a.C, e);
  a.leaves = leaves_caches((uintptr_t)z | (uintptr_t)y | (uintptr_t)((a.ld_z | a.ld_y) * e), n_rows, cfg->C, (z != nullptr) + (y != nullptr), e);
  const int64_t per = lanes ? kThreads / lanes : 1, all = dsvt_ceil_div(n_rows, per);
  const unsigned groups = (unsigned)(all < kForwardGroups ? all : kForwardGroups);
  const int32_t rows = (int32_t)dsvt_ceil_div(n_rows, groups);
  hipStream_t st = (hipStream_t)stream;
  {
    dsvt_prof_scope ps(DSVT_K_RMS_FORWARD, st);
    if (cfg->dtype == DSVT_BF16) launch<bf16_t>(a, false, form, lanes, groups, rows, st);
    else launch<float>(a, false, form, lanes, groups, rows, st);
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}

extern "C" int dsvt_rms_norm_backward_workspace_size(const dsvt_rms_cfg* cfg, int32_t n_rows, size_t* bytes) {
  if (!bytes) return DSVT_EINVAL;
  if (const int rc = check(cfg, n_rows)) return rc;
  *bytes = n_rows <= 1 ? 0 : (size_t)(n_rows < kBackwardGroups ? n_rows : kBackwardGroups) * (size_t)cfg->C * sizeof(float);
  return DSVT_OK;
}

extern "C" int dsvt_rms_norm_backward(const dsvt_rms_cfg* cfg, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const void* res,
                                      int64_t ld_res, const void* d_sum, int64_t ld_dsum, int32_t n_rows, void* dx, int64_t ld_dx,
                                      float* d_gamma, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  if (const int rc = dsvt_rms_norm_backward_workspace_size(cfg, n_rows, &need)) return rc;
  if (!d_gamma) return DSVT_EINVAL;
  const int e = cfg->dtype == DSVT_BF16 ? 2 : 4;
  if (n_rows > 0 && (bad_rows(dy, ld_dy, cfg->C, e) || bad_rows(x, ld_x, cfg->C, e) || bad_rows(dx, ld_dx, cfg->C, e) ||
                     (res && bad_rows(res, ld_res, cfg->C, e)) || (d_sum && bad_rows(d_sum, ld_dsum, cfg->C, e)))) return DSVT_EINVAL;
  if (need > 0 && (!ws || ((uintptr_t)ws & 15u))) return DSVT_EINVAL;
  if (ws_bytes < need) return DSVT_ENOSPC;
  hipStream_t st = (hipStream_t)stream;
  int32_t groups = 0;
  if (n_rows > 0) {
    RmsArgs a = {};
    a.x = x; a.res = res; a.dy = dy; a.d_sum = d_sum; a.y = dx; a.gamma = cfg->gamma;
    a.ld_x = ld_x; a.ld_res = res ? ld_res : 0; a.ld_dy = ld_dy; a.ld_dsum = d_sum ? ld_dsum : 0; a.ld_y = ld_dx;
    a.n = n_rows; a.C = cfg->C; a.eps = cfg->eps;
    a.partial = static_cast<float*>(ws);
    const RowForm form = row_form(starts(a, e), a.C, e);
    const int lanes = form_lanes(form, a.C, e);
    a.leaves = leaves_caches((uintptr_t)dx | (uintptr_t)(ld_dx * e), n_rows, cfg->C, 1, e);
    const int64_t per = lanes ? kThreads / lanes : 1, all = dsvt_ceil_div(n_rows, per);
    groups = (int32_t)(all <= kTurnsAlone ? 1 : all < kBackwardGroups ? all : kBackwardGroups);
    const int32_t rows = (int32_t)dsvt_ceil_div(n_rows, groups);
    if (lanes == 0) groups = (int32_t)dsvt_ceil_div(n_rows, rows);       // every workgroup has a row
    if (groups == 1) a.d_gamma = d_gamma;
    dsvt_prof_scope ps(DSVT_K_RMS_BACKWARD, st);
    if (cfg->dtype == DSVT_BF16) launch<bf16_t>(a, true, form, lanes, (unsigned)groups, rows, st);
    else launch<float>(a, true, form, lanes, (unsigned)groups, rows, st);
  }
  if (groups != 1) {
    dsvt_prof_scope ps(DSVT_K_RMS_SUM, st);
    k_sum_parts<<<(unsigned)dsvt_ceil_div(cfg->C, 32), 1024, 0, st>>>(static_cast<const float*>(ws), groups, cfg->C, cfg->C, d_gamma, nullptr);
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}
