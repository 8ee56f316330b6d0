// dsvt_linear_rows8: a linear layer on rows and weights in 8 bits (rows8.h).
//
//   y[n][o] = act(s_n t_o sum_c x[n][c] w[o][c] + b[o])
//
// The sum is of whole numbers, in 32 bits and exact (127^2 C < 2^31), whatever its order.
#include "rows8.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct Linear8Args {
  const int8_t *x, *w;
  const float *s, *t, *bias;                      // bias: may be null
  void* y;
  int64_t ld_x, ld_w, ld_y;
  int32_t n, C, O;
  int32_t act;
};

// The first `left` bytes of p, zeros behind them.
__device__ __forceinline__ i32x4 first_bytes(i32x4 p, int left) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int b = left - 4 * k;
    p[k] = b >= 4 ? p[k] : b <= 0 ? 0 : p[k] & (int)((1u << (8 * b)) - 1u);
  }
  return p;
}

// A workgroup takes 16 rows and 16 outputs; its wavefronts share the columns.
template <typename T> __global__ __launch_bounds__(256) void k_linear8_few(Linear8Args a) {
  __shared__ i32x4 sums[3][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  const int64_t row = (int64_t)blockIdx.x * 16 + m;
  const int o = blockIdx.y * 16 + m;
  const i32x4* x = reinterpret_cast<const i32x4*>(a.x + (row < a.n ? row : 0) * a.ld_x);
  const i32x4* w = reinterpret_cast<const i32x4*>(a.w + (int64_t)(o < a.O ? o : 0) * a.ld_w);
  i32x4 acc = {};
  for (int k = 64 * wave + 16 * g; k < a.C + 16 * g; k += 256) {
    const i32x4 zero = {};
    const i32x4 p = k < a.C ? first_bytes(w[k >> 4], a.C - k) : zero, q = k < a.C ? x[k >> 4] : zero;
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(p, q, acc, 0, 0, 0);
  }
  if (wave) sums[wave - 1][lane] = acc;
  __syncthreads();
  if (wave || row >= a.n) return;
#pragma unroll
  for (int k = 0; k < 3; ++k) acc += sums[k][lane];
  const float s = a.s[row];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int out = blockIdx.y * 16 + 4 * g + i;
    if (out >= a.O) break;
    float y = (float)acc[i] * s * a.t[out];
    if (a.bias) y += a.bias[out];
    if (a.act) y = gelu(y);
    static_cast<T*>(a.y)[row * a.ld_y + out] = (T)y;
  }
}

}  // namespace

extern "C" int dsvt_linear_rows8(const dsvt_linear8_cfg* cfg, const dsvt_rows8* x, int32_t n_rows, void* y, int64_t ld_y, void* stream) {
  if (!cfg || cfg->C <= 0 || cfg->out <= 0 || n_rows < 0) return DSVT_EINVAL;
  if (cfg->dtype != DSVT_F32 && cfg->dtype != DSVT_BF16) return DSVT_EINVAL;
  if (cfg->act != DSVT_ACT_NONE && cfg->act != DSVT_ACT_GELU) return DSVT_EINVAL;
  if (cfg->C > DSVT_LN_MAX_C || cfg->out > DSVT_LN_MAX_C) return DSVT_EUNSUPPORTED;
  if (bad_rows8(&cfg->w, cfg->C)) return DSVT_EINVAL;
  if (n_rows == 0) return DSVT_OK;
  if (bad_rows8(x, cfg->C) || bad_rows(y, ld_y, cfg->out, cfg->dtype == DSVT_BF16 ? 2 : 4)) return DSVT_EINVAL;
  Linear8Args a = {};
  a.x = x->codes; a.s = x->scale; a.ld_x = x->ld; a.w = cfg->w.codes; a.t = cfg->w.scale; a.ld_w = cfg->w.ld; a.bias = cfg->bias;
  a.y = y; a.ld_y = ld_y; a.n = n_rows; a.C = cfg->C; a.O = cfg->out; a.act = cfg->act;
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid((unsigned)dsvt_ceil_div(n_rows, 16), (unsigned)dsvt_ceil_div(a.O, 16));
  {
    dsvt_prof_scope ps(DSVT_K_LINEAR8, st);
    if (cfg->dtype == DSVT_BF16) k_linear8_few<bf16_t><<<grid, 256, 0, st>>>(a);
    else k_linear8_few<float><<<grid, 256, 0, st>>>(a);
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}
