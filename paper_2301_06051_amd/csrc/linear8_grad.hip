// dsvt_linear_rows8_weight_grad: the gradients of a linear layer's weights and bias from its input as it was kept in 8 bits (rows8.h).
//
//   d_w[o][c] = sum_n dy[n][o] s_n x[n][c],  d_b[o] = sum_n dy[n][o]
//
// The sums run over the rows: workgroups take a tile of outputs and columns and a slice of the rows each, and leave partial sums in 32 bits, which
// are added up in their order.
#include "rows8.h"

namespace {

struct Grad8Args {
  const int8_t* x;
  const float* s;
  const void* dy;
  float *partial, *bias_partial;                  // [slices][O][C], [slices][O] (null: no gradient of the bias)
  int64_t ld_x, ld_dy;
  int32_t n, C, O;
  int32_t slice;                                  // rows of a slice
};

constexpr int kTile = 64, kStep = 16;

// 256 threads, four by four values each
template <typename T> __global__ __launch_bounds__(256) void k_linear8_grad(Grad8Args a) {
  __shared__ float dy[kStep][kTile + 4], x[kStep][kTile + 4];
  const int o0 = blockIdx.x * kTile, c0 = blockIdx.y * kTile, to = threadIdx.x >> 4, tc = threadIdx.x & 15;
  const int64_t first = (int64_t)blockIdx.z * a.slice, last = first + a.slice < a.n ? first + a.slice : a.n;
  float acc[4][4] = {}, db[4] = {};
  for (int64_t row0 = first; row0 < last; row0 += kStep) {
    __syncthreads();
    for (int k = threadIdx.x; k < kStep * kTile; k += 256) {
      const int64_t row = row0 + k / kTile;
      const int j = k % kTile;
      dy[k / kTile][j] = row < last && o0 + j < a.O ? (float)static_cast<const T*>(a.dy)[row * a.ld_dy + o0 + j] : 0.f;
      x[k / kTile][j] = row < last && c0 + j < a.C ? (float)a.x[row * a.ld_x + c0 + j] * a.s[row] : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < kStep; ++k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        db[i] += dy[k][4 * to + i];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(dy[k][4 * to + i], x[k][4 * tc + j], acc[i][j]);
      }
    }
  }
  for (int i = 0; i < 4; ++i) {
    const int o = o0 + 4 * to + i;
    if (o >= a.O) break;
    for (int j = 0; j < 4; ++j)
      if (c0 + 4 * tc + j < a.C) a.partial[((int64_t)blockIdx.z * a.O + o) * a.C + c0 + 4 * tc + j] = acc[i][j];
    if (a.bias_partial && blockIdx.y == 0 && tc == 0) a.bias_partial[(int64_t)blockIdx.z * a.O + o] = db[i];
  }
}

// d_w: the slices' sums added in their order, in 32 bits (few slices).
template <typename T> __global__ __launch_bounds__(256) void k_linear8_grad_join(const float* __restrict__ partial, int32_t slices, int32_t O, int32_t C,
                                                                                 T* __restrict__ d_w, int64_t ld) {
  const int64_t all = (int64_t)O * C;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    float v = 0.f;
    for (int k = 0; k < slices; ++k) v += partial[k * all + i];
    d_w[i / C * ld + i % C] = (T)v;
  }
}

struct Plan { int32_t slices, slice; };
Plan make_plan(int32_t C, int32_t O, int32_t n) {
  const int64_t tiles = dsvt_ceil_div(O, kTile) * dsvt_ceil_div(C, kTile);
  int64_t slices = dsvt_ceil_div(1024, tiles);
  const int64_t most = dsvt_ceil_div(n, 64);
  slices = slices < most ? slices : most;
  slices = slices < 1 ? 1 : slices;
  const int32_t slice = (int32_t)dsvt_ceil_div(n > 0 ? n : 1, slices);
  return {(int32_t)(n > 0 ? dsvt_ceil_div(n, slice) : 0), slice};
}

int check(int32_t C, int32_t O, int32_t dtype, int32_t n_rows) {
  if (C <= 0 || O <= 0 || n_rows < 0 || (dtype != DSVT_F32 && dtype != DSVT_BF16)) return DSVT_EINVAL;
  return C > DSVT_LN_MAX_C || O > DSVT_LN_MAX_C ? DSVT_EUNSUPPORTED : DSVT_OK;
}

}  // namespace

extern "C" int dsvt_linear_rows8_weight_grad_workspace_size(int32_t C, int32_t out, int32_t dtype, int32_t n_rows, size_t* bytes) {
  if (!bytes) return DSVT_EINVAL;
  if (const int rc = check(C, out, dtype, n_rows)) return rc;
  const Plan p = make_plan(C, out, n_rows);
  *bytes = (size_t)p.slices * (size_t)out * ((size_t)C + 1) * sizeof(float);
  return DSVT_OK;
}

extern "C" int dsvt_linear_rows8_weight_grad(int32_t C, int32_t out, int32_t dtype, const dsvt_rows8* x, const void* dy, int64_t ld_dy,
                                             int32_t n_rows, void* d_w, int64_t ld_dw, float* d_b, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  if (const int rc = dsvt_linear_rows8_weight_grad_workspace_size(C, out, dtype, n_rows, &need)) return rc;
  const int e = dtype == DSVT_BF16 ? 2 : 4;
  if (bad_rows(d_w, ld_dw, C, e) || ((uintptr_t)d_b & 3u) != 0) return DSVT_EINVAL;
  if (n_rows > 0 && (bad_rows8(x, C) || bad_rows(dy, ld_dy, out, e))) return DSVT_EINVAL;
  if (need > 0 && (!ws || ((uintptr_t)ws & 15u))) return DSVT_EINVAL;
  if (ws_bytes < need) return DSVT_ENOSPC;
  const Plan p = make_plan(C, out, n_rows);
  hipStream_t st = (hipStream_t)stream;
  Grad8Args a = {};
  a.dy = dy; a.ld_dy = ld_dy; a.n = n_rows; a.C = C; a.O = out; a.slice = p.slice;
  a.partial = static_cast<float*>(ws);
  a.bias_partial = d_b ? a.partial + (int64_t)p.slices * out * C : nullptr;
  if (n_rows > 0) {
    a.x = x->codes; a.s = x->scale; a.ld_x = x->ld;
    const dim3 grid((unsigned)dsvt_ceil_div(out, kTile), (unsigned)dsvt_ceil_div(C, kTile), (unsigned)p.slices);
    dsvt_prof_scope ps(DSVT_K_LINEAR8_GRAD, st);
    if (dtype == DSVT_BF16) k_linear8_grad<bf16_t><<<grid, 256, 0, st>>>(a);
    else k_linear8_grad<float><<<grid, 256, 0, st>>>(a);
  }
  {
    dsvt_prof_scope ps(DSVT_K_LINEAR8_JOIN, st);
    const int64_t blocks = dsvt_ceil_div((int64_t)out * C, 256);
    const unsigned grid = (unsigned)(blocks < 4096 ? blocks : 4096);
    if (dtype == DSVT_BF16) k_linear8_grad_join<bf16_t><<<grid, 256, 0, st>>>(a.partial, p.slices, out, C, static_cast<bf16_t*>(d_w), ld_dw);
    else k_linear8_grad_join<float><<<grid, 256, 0, st>>>(a.partial, p.slices, out, C, static_cast<float*>(d_w), ld_dw);
    if (d_b) k_sum_parts<<<(unsigned)dsvt_ceil_div(out, 32), 1024, 0, st>>>(a.bias_partial, p.slices, out, out, d_b, nullptr);
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}
