// dsvt_linear_rows8: a linear layer on rows and weights in 8 bits (rows8.h).
//
//   y[n][o] = act(s_n t_o sum_c x[n][c] w[o][c] + b[o])
//
// The sum is of whole numbers, in 32 bits and exact (127^2 C < 2^31), whatever its order.
#include "rows8.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

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

// Tiles of kRowsT rows and kOutsT outputs, shared by kM x kN wavefronts; 128 columns at a time go from memory through registers into one of two
// buffers in LDS while the other is multiplied.
//
// The matrix instruction takes 32 outputs, 32 rows and 32 columns: lane 32 h + m holds 16 codes of row m, from column 16 h on.  In LDS a row's
// 16-byte pieces are permuted, piece j of row r being at j ^ (r / 2 mod 8): the 16 lanes whose reads are served together (0-3, 12-15 and 20-27, or 4-11,
// 16-19 and 28-31 of a half) then hit all banks once.  Weights are read in another order of their rows, so that a lane's 16 sums of a tile are 16
// neighbouring outputs of one row.
constexpr int kColumns = 128, kPieces = kColumns / 16;

template <int kRowsT, int kOutsT> constexpr size_t tiles_lds() { return (size_t)2 * (kRowsT + kOutsT) * kColumns; }

template <typename T, int kRowsT, int kOutsT, int kM, int kN> __global__ __launch_bounds__(64 * kM * kN) void k_linear8_tiles(Linear8Args a) {
  constexpr int kAll = 64 * kM * kN, TM = kRowsT / kM / 32, TN = kOutsT / kN / 32, kPer = kAll / kPieces;       // kPer: rows that all threads fetch at once
  constexpr int PX = kRowsT / kPer, PW = kOutsT / kPer;
  static_assert(kRowsT % kPer == 0 && kOutsT % kPer == 0, "rows are fetched by all threads together");
  extern __shared__ i32x4 lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave % kM, wn = wave / kM, m = lane & 31, h = lane >> 5;
  // workgroups of one XCD (every eighth) take neighbouring tiles: eight along the rows, then the next outputs
  const int tiles_m = (a.n + kRowsT - 1) / kRowsT, tiles_n = (a.O + kOutsT - 1) / kOutsT, all = tiles_m * tiles_n;
  const int per = (all + 7) >> 3;
  int id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per || id >= all) return;
  const int band = id / (8 * tiles_n), bm = tiles_m - 8 * band < 8 ? tiles_m - 8 * band : 8;
  id -= band * 8 * tiles_n;
  const int64_t row0 = (int64_t)(8 * band + id % bm) * kRowsT;
  const int out0 = id / bm * kOutsT;

  // what this thread fetches: piece `piece` of rows tid / 8 + kPer i (past the last row the last one again)
  const int piece = tid % kPieces;
  const int8_t *x = a.x + row0 * a.ld_x, *w = a.w + (int64_t)out0 * a.ld_w;
  uint32_t off[PX + PW];
  const int last_x = (int)(a.n - row0 < kRowsT ? a.n - row0 : kRowsT) - 1, last_w = (a.O - out0 < kOutsT ? a.O - out0 : kOutsT) - 1;
#pragma unroll
  for (int i = 0; i < PX + PW; ++i) {
    const int r = tid / kPieces + kPer * (i < PX ? i : i - PX), last = i < PX ? last_x : last_w;
    off[i] = (uint32_t)(r < last ? r : last) * (uint32_t)(i < PX ? a.ld_x : a.ld_w) + 16u * piece;
  }
  i32x4 stage[PX + PW];
  const auto fetch = [&](int k0) {
    const int left = a.C - k0 - 16 * piece;
    if (k0 + kColumns <= a.C) {
#pragma unroll
      for (int i = 0; i < PX + PW; ++i) stage[i] = *reinterpret_cast<const i32x4*>((i < PX ? x : w) + k0 + off[i]);
    } else {
#pragma unroll
      for (int i = 0; i < PX + PW; ++i) {
        const i32x4 zero = {};
        stage[i] = zero;
        if (left > 0) stage[i] = *reinterpret_cast<const i32x4*>((i < PX ? x : w) + k0 + off[i]);
        if (i >= PX) stage[i] = first_bytes(stage[i], left);              // what lies past a row's end may be anything; zeros in one operand do
      }
    }
  };
  i32x4* const mine = lds + tid / kPieces * kPieces;
  const auto put = [&](int buffer) {
#pragma unroll
    for (int i = 0; i < PX + PW; ++i) {
      const int r = tid / kPieces;                // (kPer is a multiple of 16, so the permutation is that of row r)
      mine[buffer * (kRowsT + kOutsT) * kPieces + kPer * i * kPieces + (piece ^ (r >> 1 & 7))] = stage[i];
    }
  };
  static_assert(kPer % 16 == 0, "see put");

  i32x16 acc[TM][TN] = {};
  const int turn = m >> 1 & 7, out_m = (m >> 2 & 1) * 16 + (m >> 3) * 4 + (m & 3), out_turn = out_m >> 1 & 7;
  const i32x4* const xs = lds + (wm * TM * 32 + m) * kPieces;
  const i32x4* const ws = lds + (kRowsT + wn * TN * 32 + out_m) * kPieces;
  const auto multiply = [&](int buffer, int k) {
    i32x4 p[TN], q[TM];
#pragma unroll
    for (int t = 0; t < TN; ++t) p[t] = ws[buffer * (kRowsT + kOutsT) * kPieces + t * 32 * kPieces + ((2 * k + h) ^ out_turn)];
#pragma unroll
    for (int t = 0; t < TM; ++t) q[t] = xs[buffer * (kRowsT + kOutsT) * kPieces + t * 32 * kPieces + ((2 * k + h) ^ turn)];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(p[j], q[i], acc[i][j], 0, 0, 0);
  };

  fetch(0);
  put(0);
  if (kColumns < a.C) fetch(kColumns);
  lds_barrier();
  int buffer = 0;
  int k0 = 0;
  for (; k0 + kColumns < a.C; k0 += kColumns, buffer ^= 1) {
    multiply(buffer, 0);
    multiply(buffer, 1);
    put(buffer ^ 1);
    if (k0 + 2 * kColumns < a.C) fetch(k0 + 2 * kColumns);
    multiply(buffer, 2);
    multiply(buffer, 3);
    lds_barrier();
  }
  for (int k = 0; k < 4 && k0 + 32 * k < a.C; ++k) multiply(buffer, k);

  const bool wide = ((uintptr_t)a.y & 15u) == 0 && a.ld_y * (int64_t)sizeof(T) % 16 == 0;
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int out = out0 + (wn * TN + j) * 32 + 16 * h;
    if (out >= a.O) continue;
    float t[16], b[16];
    if (out + 16 <= a.O) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        t[e] = a.t[out + e];
        b[e] = a.bias ? a.bias[out + e] : 0.f;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        t[e] = out + e < a.O ? a.t[out + e] : 0.f;
        b[e] = out + e < a.O && a.bias ? a.bias[out + e] : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t row = row0 + (wm * TM + i) * 32 + m;
      if (row >= a.n) continue;
      const float s = a.s[row];
      T* y = static_cast<T*>(a.y) + row * a.ld_y + out;
      float v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        v[e] = (float)acc[i][j][e] * s * t[e];
        if (a.bias) v[e] += b[e];
        if (a.act) v[e] = gelu(v[e]);
      }
      if (wide && out + 16 <= a.O) {
        constexpr int V = 16 / sizeof(T);
        typedef typename Piece<T, V>::type P;
#pragma unroll
        for (int e = 0; e < 16; e += V) {
          float f[V];
#pragma unroll
          for (int k = 0; k < V; ++k) f[k] = v[e + k];
          reinterpret_cast<P*>(y)[e / V] = narrow<T, V>(f);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (out + e < a.O) y[e] = (T)v[e];
      }
    }
  }
}

template <typename T, int kRowsT, int kOutsT, int kM, int kN> int launch_tiles(const Linear8Args& a, hipStream_t st) {
  static std::atomic<uint64_t> allowed;
  const auto kernel = k_linear8_tiles<T, kRowsT, kOutsT, kM, kN>;
  constexpr size_t lds = tiles_lds<kRowsT, kOutsT>();
  if (const int rc = dsvt_allow_lds(reinterpret_cast<const void*>(kernel), lds, allowed)) return rc;
  const int64_t all = dsvt_ceil_div(a.n, kRowsT) * dsvt_ceil_div(a.O, kOutsT);
  kernel<<<(unsigned)(dsvt_ceil_div(all, 8) * 8), 64 * kM * kN, lds, st>>>(a);
  return DSVT_OK;
}
template <typename T> int launch(const Linear8Args& a, hipStream_t st) {
  const auto tiles = [&](int rows, int outs) { return dsvt_ceil_div(a.n, rows) * dsvt_ceil_div(a.O, outs); };
  // (a tile's rows are 2^31 bytes apart at most)
  if (a.n <= 32 || a.ld_x >= (1 << 23) || a.ld_w >= (1 << 23)) {
    const dim3 grid((unsigned)dsvt_ceil_div(a.n, 16), (unsigned)dsvt_ceil_div(a.O, 16));
    k_linear8_few<T><<<grid, 256, 0, st>>>(a);
    return DSVT_OK;
  }
  if (tiles(256, 256) >= 256) return launch_tiles<T, 256, 256, 2, 4>(a, st);
  if (tiles(128, 128) >= 256) return launch_tiles<T, 128, 128, 2, 2>(a, st);
  return launch_tiles<T, 64, 64, 2, 2>(a, st);
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
  {
    dsvt_prof_scope ps(DSVT_K_LINEAR8, st);
    if (const int rc = cfg->dtype == DSVT_BF16 ? launch<bf16_t>(a, st) : launch<float>(a, st)) return rc;
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}
