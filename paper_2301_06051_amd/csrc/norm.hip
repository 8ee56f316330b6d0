// dsvt_layer_norm / dsvt_layer_norm_backward: the residual sum and LayerNorm of a DSVT layer (Eq. 5) as calls of their
// own, with their gradients.
//
//   forward   z = x + res, n = (z - mean z) * rsqrt(var z + eps), y = n * gamma + beta
//   backward  w = dy * gamma, dz = rsqrt(var z + eps) * (w - mean w - n * mean(w * n)), d_gamma = sum of dy * n over
//             the rows, d_beta = sum of dy
// z, its mean and its variance are formed again in the backward pass instead of being kept: x and res hold the sum
// exactly, where a z kept in bf16 would not, and one more row read is one row less written by the forward pass.
//
// Both passes are bound by the bytes of their rows.  A row sits in the registers of kLanes neighbouring lanes (8 to 64, or a workgroup's
// 256, up to four 16-byte pieces each), so it is read once, and its sums take three to eight steps across lanes.  Workgroups stay and
// take rows in turn: gamma and beta are read once a workgroup, and the backward pass adds d_gamma and d_beta up in
// registers, then in LDS and in one row of partial sums a workgroup, which k_sum_parts adds in their order.  All sums are
// held in 32 bits, that over the workgroups in 64, and none depends on the order in which workgroups run.  800,000 rows of 192 bf16 with a
// branch: forward 175 us, backward 233 (5.3 TB/s each; a copy of 2 GiB reaches 4.8 on the same card).
#include "rows.h"
#include "sum_parts.h"

namespace {

struct LnArgs {
  const void *x, *res, *dy;                       // res: may be null; dy: backward only
  void* out;                                      // y or dx
  const float *gamma, *beta;
  float *partial, *d_gamma, *d_beta;              // [groups][2][C]; d_*: null when partial sums are to be added up by k_sum_parts
  int64_t ld_x, ld_res, ld_dy, ld_out;
  int32_t n, C;
  float eps;
};

// z = x + res in 32 bits, normed in place: returns rsqrt(var + eps).  The mean is subtracted before the squares are summed.
template <typename T, int V, int kLanes, int R>
__device__ __forceinline__ float norm_row(const RowPieces<T, V, kLanes, R>& x, const RowPieces<T, V, kLanes, R>& res, bool with_res, int part,
                                          int pieces, float inv_c, float eps, float (&z)[R][V], float* s) {
  float sum = 0.f;
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
    for (int i = 0; i < V; ++i) sum += z[r][i];
  }
  const float mean = lane_sum<kLanes>(sum, s) * inv_c;
  float sq = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool there = r * kLanes + part < pieces;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      z[r][i] = there ? z[r][i] - mean : 0.f;
      sq = fmaf(z[r][i], z[r][i], sq);
    }
  }
  const float rs = 1.f / sqrtf(lane_sum<kLanes>(sq, s) * inv_c + eps);
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) z[r][i] *= rs;
  return rs;
}

template <typename T, int V, int kLanes, int R>
__global__ __launch_bounds__(kThreads) void k_ln_forward(LnArgs a) {
  constexpr int kRows = kThreads / kLanes;
  __shared__ float s[kThreads / 64];
  const int part = threadIdx.x % kLanes, pieces = a.C / V;
  const float inv_c = 1.f / (float)a.C;
  float gamma[R][V], beta[R][V];
  load_vector<V, kLanes, R>(a.gamma, part, pieces, gamma);
  load_vector<V, kLanes, R>(a.beta, part, pieces, beta);
  typedef typename Piece<T, V>::type P;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes; row < a.n; row += (int64_t)gridDim.x * kRows) {
    RowPieces<T, V, kLanes, R> x, res;
    x.load(a.x, row * a.ld_x, part, pieces, true);
    if (a.res) res.load(a.res, row * a.ld_res, part, pieces, true);
    float z[R][V];
    norm_row<T, V, kLanes, R>(x, res, a.res != nullptr, part, pieces, inv_c, a.eps, z, s);
    P* out = reinterpret_cast<P*>(static_cast<T*>(a.out) + row * a.ld_out);
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 0; i < V; ++i) z[r][i] = fmaf(z[r][i], gamma[r][i], beta[r][i]);
      if (r * kLanes + part < pieces) out[r * kLanes + part] = narrow<T, V>(z[r]);
    }
  }
}

template <typename T, int V, int kLanes, int R>
__global__ __launch_bounds__(kThreads) void k_ln_backward(LnArgs a) {
  constexpr int kRows = kThreads / kLanes;
  __shared__ float s[kThreads / 64];
  const int part = threadIdx.x % kLanes, pieces = a.C / V;
  const float inv_c = 1.f / (float)a.C;
  float gamma[R][V], dg[R][V] = {}, db[R][V] = {};
  load_vector<V, kLanes, R>(a.gamma, part, pieces, gamma);
  typedef typename Piece<T, V>::type P;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes; row < a.n; row += (int64_t)gridDim.x * kRows) {
    RowPieces<T, V, kLanes, R> x, res, dy;
    x.load(a.x, row * a.ld_x, part, pieces, true);
    if (a.res) res.load(a.res, row * a.ld_res, part, pieces, true);
    dy.load(a.dy, row * a.ld_dy, part, pieces, true);
    float z[R][V], w[R][V];
    const float rs = norm_row<T, V, kLanes, R>(x, res, a.res != nullptr, part, pieces, inv_c, a.eps, z, s);
    float sum_w = 0.f, sum_wn = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      widen<T, V>(dy.p[r], w[r]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        dg[r][i] = fmaf(w[r][i], z[r][i], dg[r][i]);
        db[r][i] += w[r][i];
        w[r][i] *= gamma[r][i];
        sum_w += w[r][i];
        sum_wn = fmaf(w[r][i], z[r][i], sum_wn);
      }
    }
    const float mean_w = lane_sum<kLanes>(sum_w, s) * inv_c, mean_wn = lane_sum<kLanes>(sum_wn, s) * inv_c;
    P* out = reinterpret_cast<P*>(static_cast<T*>(a.out) + row * a.ld_out);
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 0; i < V; ++i) z[r][i] = rs * (w[r][i] - mean_w - z[r][i] * mean_wn);
      if (r * kLanes + part < pieces) out[r * kLanes + part] = narrow<T, V>(z[r]);
    }
  }
  // the workgroup's sums: over the rows of a wavefront across lanes, over its wavefronts in LDS
  constexpr int kCopies = kLanes > 64 ? 1 : kThreads / 64;
  __shared__ float sums[kCopies][2][kLanes * R * V];
  const int lane = threadIdx.x & 63, copy = kLanes > 64 ? 0 : threadIdx.x >> 6;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int d = kLanes; d < 64; d *= 2) {
        dg[r][i] += __shfl_xor(dg[r][i], d, 64);
        db[r][i] += __shfl_xor(db[r][i], d, 64);
      }
      if (lane < kLanes) {
        sums[copy][0][(r * kLanes + part) * V + i] = dg[r][i];
        sums[copy][1][(r * kLanes + part) * V + i] = db[r][i];
      }
    }
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * a.C; c += kThreads) {
    const int which = c >= a.C, col = c - which * a.C;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kCopies; ++k) v += sums[k][which][col];
    if (a.d_gamma) (which ? a.d_beta : a.d_gamma)[col] = v;
    else a.partial[(int64_t)blockIdx.x * 2 * a.C + c] = v;
  }
}

template <typename T> __device__ __forceinline__ float sum_at(const LnArgs& a, int64_t row, int c) {
  float z = (float)static_cast<const T*>(a.x)[row * a.ld_x + c];
  if (a.res) z += (float)static_cast<const T*>(a.res)[row * a.ld_res + c];
  return z;
}

// Rows that registers do not hold: a workgroup a row, which is read again, from the caches, for each of its sums.  Workgroups take
// consecutive rows, `rows` of them.
template <typename T, bool kBackward>
__global__ __launch_bounds__(kThreads) void k_ln_long(LnArgs a, int32_t rows) {
  __shared__ float s[kThreads / 64];
  const float inv_c = 1.f / (float)a.C;
  const int64_t first = (int64_t)blockIdx.x * rows, last = first + rows < a.n ? first + rows : a.n;
  float* part_g = kBackward ? (a.d_gamma ? a.d_gamma : a.partial + (int64_t)blockIdx.x * 2 * a.C) : nullptr;
  float* part_b = kBackward ? (a.d_gamma ? a.d_beta : part_g + a.C) : nullptr;
  for (int64_t row = first; row < last; ++row) {
    float v = 0.f;
    for (int c = threadIdx.x; c < a.C; c += kThreads) v += sum_at<T>(a, row, c);
    const float mean = lane_sum<kThreads>(v, s) * inv_c;
    v = 0.f;
    for (int c = threadIdx.x; c < a.C; c += kThreads) {
      const float z = sum_at<T>(a, row, c) - mean;
      v = fmaf(z, z, v);
    }
    const float rs = 1.f / sqrtf(lane_sum<kThreads>(v, s) * inv_c + a.eps);
    T* out = static_cast<T*>(a.out) + row * a.ld_out;
    if (!kBackward) {
      for (int c = threadIdx.x; c < a.C; c += kThreads) out[c] = (T)fmaf((sum_at<T>(a, row, c) - mean) * rs, a.gamma[c], a.beta[c]);
      continue;
    }
    const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
    float sum_w = 0.f, sum_wn = 0.f;
    for (int c = threadIdx.x; c < a.C; c += kThreads) {
      const float w = (float)dy[c] * a.gamma[c];
      sum_w += w;
      sum_wn = fmaf(w, (sum_at<T>(a, row, c) - mean) * rs, sum_wn);
    }
    const float mean_w = lane_sum<kThreads>(sum_w, s) * inv_c, mean_wn = lane_sum<kThreads>(sum_wn, s) * inv_c;
    for (int c = threadIdx.x; c < a.C; c += kThreads) {
      const float d = (float)dy[c], n = (sum_at<T>(a, row, c) - mean) * rs;
      out[c] = (T)(rs * (d * a.gamma[c] - mean_w - n * mean_wn));
      part_g[c] = (row == first ? 0.f : part_g[c]) + d * n;       // a column is always the same thread's
      part_b[c] = (row == first ? 0.f : part_b[c]) + d;
    }
  }
}

// All of a row's arrays, as piece_elems wants them.
uintptr_t starts(const LnArgs& a, int e) {
  return (uintptr_t)a.x | (uintptr_t)a.res | (uintptr_t)a.dy | (uintptr_t)a.out | (uintptr_t)((a.ld_x | a.ld_res | a.ld_dy | a.ld_out) * e);
}

struct Forward {
  template <typename T, int V, int kLanes, int R> static void rows(const LnArgs& a, unsigned groups, hipStream_t st) {
    k_ln_forward<T, V, kLanes, R><<<groups, kThreads, 0, st>>>(a);
  }
};
struct Backward {
  template <typename T, int V, int kLanes, int R> static void rows(const LnArgs& a, unsigned groups, hipStream_t st) {
    k_ln_backward<T, V, kLanes, R><<<groups, kThreads, 0, st>>>(a);
  }
};
template <typename T> void launch(const LnArgs& a, bool back, int v, int lanes, unsigned groups, int32_t rows, hipStream_t st) {
  if (lanes == 0) {
    if (back) k_ln_long<T, true><<<groups, kThreads, 0, st>>>(a, rows);
    else k_ln_long<T, false><<<groups, kThreads, 0, st>>>(a, rows);
  } else if (back) launch_rows<Backward, T>(a, v, lanes, groups, st);
  else launch_rows<Forward, T>(a, v, lanes, groups, st);
}

int check(const dsvt_ln_cfg* cfg, int32_t n_rows) {
  if (!cfg || !cfg->gamma || cfg->C <= 0 || n_rows < 0) return DSVT_EINVAL;
  if (cfg->dtype != DSVT_F32 && cfg->dtype != DSVT_BF16) return DSVT_EINVAL;
  if (!(cfg->eps >= 0.f)) return DSVT_EINVAL;
  if (cfg->C > DSVT_LN_MAX_C) return DSVT_EUNSUPPORTED;
  return DSVT_OK;
}
// Workgroups of a backward pass, and so rows of partial sums: bounded by the rows alone, so that the workspace goes by n_rows and C only.
int32_t backward_groups(int32_t n_rows) { return n_rows < kBackwardGroups ? n_rows : kBackwardGroups; }

}  // namespace

extern "C" int dsvt_layer_norm(const dsvt_ln_cfg* cfg, const void* x, int64_t ld_x, const void* res, int64_t ld_res, int32_t n_rows, void* y,
                               int64_t ld_y, void* stream) {
  if (const int rc = check(cfg, n_rows)) return rc;
  if (!cfg->beta) return DSVT_EINVAL;
  if (n_rows == 0) return DSVT_OK;
  const int e = cfg->dtype == DSVT_BF16 ? 2 : 4;
  if (bad_rows(x, ld_x, cfg->C, e) || bad_rows(y, ld_y, cfg->C, e) || (res && bad_rows(res, ld_res, cfg->C, e))) return DSVT_EINVAL;
  LnArgs a = {};
  a.x = x; a.res = res; a.out = y; a.gamma = cfg->gamma; a.beta = cfg->beta;
  a.ld_x = ld_x; a.ld_res = res ? ld_res : 0; a.ld_out = ld_y; a.n = n_rows; a.C = cfg->C; a.eps = cfg->eps;
  const int v = piece_elems(starts(a, e), a.C, e), lanes = row_lanes(cfg->C / v, v * e);
  const int64_t per = lanes ? kThreads / lanes : 1, all = dsvt_ceil_div(n_rows, per);
  const unsigned groups = (unsigned)(all < kForwardGroups ? all : kForwardGroups);
  const int32_t rows = (int32_t)dsvt_ceil_div(n_rows, groups);
  hipStream_t st = (hipStream_t)stream;
  {
    dsvt_prof_scope ps(DSVT_K_LN_FORWARD, st);
    if (cfg->dtype == DSVT_BF16) launch<bf16_t>(a, false, v, lanes, groups, rows, st);
    else launch<float>(a, false, v, lanes, groups, rows, st);
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}

extern "C" int dsvt_layer_norm_backward_workspace_size(const dsvt_ln_cfg* cfg, int32_t n_rows, size_t* bytes) {
  if (!bytes) return DSVT_EINVAL;
  if (const int rc = check(cfg, n_rows)) return rc;
  *bytes = n_rows <= 1 ? 0 : (size_t)backward_groups(n_rows) * 2 * (size_t)cfg->C * sizeof(float);
  return DSVT_OK;
}

extern "C" int dsvt_layer_norm_backward(const dsvt_ln_cfg* cfg, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const void* res,
                                        int64_t ld_res, int32_t n_rows, void* dx, int64_t ld_dx, float* d_gamma, float* d_beta, void* ws,
                                        size_t ws_bytes, void* stream) {
  size_t need = 0;
  if (const int rc = dsvt_layer_norm_backward_workspace_size(cfg, n_rows, &need)) return rc;
  if (!d_gamma || !d_beta) return DSVT_EINVAL;
  const int e = cfg->dtype == DSVT_BF16 ? 2 : 4;
  if (n_rows > 0 && (bad_rows(dy, ld_dy, cfg->C, e) || bad_rows(x, ld_x, cfg->C, e) || bad_rows(dx, ld_dx, cfg->C, e) ||
                     (res && bad_rows(res, ld_res, cfg->C, e)))) return DSVT_EINVAL;
  if (need > 0 && (!ws || ((uintptr_t)ws & 15u))) return DSVT_EINVAL;
  if (ws_bytes < need) return DSVT_ENOSPC;
  hipStream_t st = (hipStream_t)stream;
  int32_t groups = 0;
  if (n_rows > 0) {
    LnArgs a = {};
    a.x = x; a.res = res; a.dy = dy; a.out = dx; a.gamma = cfg->gamma;
    a.ld_x = ld_x; a.ld_res = res ? ld_res : 0; a.ld_dy = ld_dy; a.ld_out = ld_dx; a.n = n_rows; a.C = cfg->C; a.eps = cfg->eps;
    a.partial = static_cast<float*>(ws);
    const int v = piece_elems(starts(a, e), a.C, e), lanes = row_lanes(cfg->C / v, v * e);
    const int64_t per = lanes ? kThreads / lanes : 1, all = dsvt_ceil_div(n_rows, per);
    groups = (int32_t)(all < kBackwardGroups ? all : kBackwardGroups);
    const int32_t rows = (int32_t)dsvt_ceil_div(n_rows, groups);
    if (lanes == 0) groups = (int32_t)dsvt_ceil_div(n_rows, rows);       // every workgroup has a row
    if (groups == 1) { a.d_gamma = d_gamma; a.d_beta = d_beta; }
    dsvt_prof_scope ps(DSVT_K_LN_BACKWARD, st);
    if (cfg->dtype == DSVT_BF16) launch<bf16_t>(a, true, v, lanes, (unsigned)groups, rows, st);
    else launch<float>(a, true, v, lanes, (unsigned)groups, rows, st);
  }
  if (groups != 1) {
    dsvt_prof_scope ps(DSVT_K_LN_SUM, st);
    k_sum_parts<<<(unsigned)dsvt_ceil_div(2 * (int64_t)cfg->C, 32), 1024, 0, st>>>(static_cast<const float*>(ws), groups, 2 * cfg->C, cfg->C, d_gamma,
                                                                                   d_beta);
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}
