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
  // What is fetched does not hang on a condition, which would have to wait for it: pieces past a row's end are its last one.
  i32x4 stage[PX + PW];
  const int last_piece = (a.C - 1) >> 4 << 4;
  const auto fetch = [&](int k0) {
    const int back = k0 + 16 * piece > last_piece ? k0 + 16 * piece - last_piece : 0;
#pragma unroll
    for (int i = 0; i < PX + PW; ++i) stage[i] = *reinterpret_cast<const i32x4*>((i < PX ? x : w) + k0 + (int64_t)off[i] - back);
  };
  i32x4* const mine = lds + tid / kPieces * kPieces;
  const auto put = [&](int buffer, int k0) {
    if (k0 + kColumns > a.C) {                    // what lies past a row's end may be anything; zeros in one operand do
#pragma unroll
      for (int i = PX; i < PX + PW; ++i) stage[i] = first_bytes(stage[i], a.C - k0 - 16 * piece);
    }
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
  struct Frags { i32x4 p[TN], q[TM]; } now, next;
  const auto read = [&](Frags& f, int buffer, int k) {
#pragma unroll
    for (int t = 0; t < TN; ++t) f.p[t] = ws[buffer * (kRowsT + kOutsT) * kPieces + t * 32 * kPieces + ((2 * k + h) ^ out_turn)];
#pragma unroll
    for (int t = 0; t < TM; ++t) f.q[t] = xs[buffer * (kRowsT + kOutsT) * kPieces + t * 32 * kPieces + ((2 * k + h) ^ turn)];
  };
  const auto multiply = [&](const Frags& f) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.p[j], f.q[i], acc[i][j], 0, 0, 0);
  };

  // The fragments of a product are read while the one before is under way, the first ones of a buffer behind the barrier that the other
  // wavefronts' part of it is waited for at, during the last product of the buffer before.
  fetch(0);
  put(0, 0);
  fetch(kColumns);
  lds_barrier();
  read(now, 0, 0);
  int buffer = 0;
  int k0 = 0;
  for (; k0 + kColumns < a.C; k0 += kColumns, buffer ^= 1) {
    read(next, buffer, 1);
    multiply(now);
    put(buffer ^ 1, k0 + kColumns);
    fetch(k0 + 2 * kColumns);
    read(now, buffer, 2);
    multiply(next);
    read(next, buffer, 3);
    multiply(now);
    lds_barrier();
    read(now, buffer ^ 1, 0);
    multiply(next);
  }
  for (int k = 0; k < 4 && k0 + 32 * k < a.C; ++k) {
    if (k) read(now, buffer, k);
    multiply(now);
  }

  // Results go through LDS, 32 rows of a wavefront at a time, so that a row's are written side by side: as they come out of the product, a store would
  // write 32 pieces of 64 bytes.
  constexpr int kWide = TN * 32, V = 16 / (int)sizeof(T), PR = kWide / V;
  static_assert(PR == 4 || PR == 8 || PR == 16, "pieces of a row are permuted within 4 or 8");
  const auto spot = [](int row, int p) { return row * PR + (p ^ (PR == 4 ? row >> 1 & 3 : row & 7)); };
  typedef typename Piece<T, V>::type P;
  static_assert(kM * kN * 32 * PR <= 2 * (kRowsT + kOutsT) * kPieces, "the results of all wavefronts fit the buffers");
  P* const out = reinterpret_cast<P*>(lds) + wave * 32 * PR;
  const int first_out = out0 + wn * kWide, outs = a.O - first_out < kWide ? a.O - first_out : kWide;
  const bool wide = outs % V == 0 && ((uintptr_t)a.y & 15u) == 0 && a.ld_y * (int64_t)sizeof(T) % 16 == 0;
  float t[TN][16], bias[TN][16];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int at = j * 32 + 16 * h + e, there = first_out + (at < outs ? at : 0);
      t[j][e] = outs > 0 ? a.t[there] : 0.f;
      bias[j][e] = outs > 0 && a.bias ? a.bias[there] : 0.f;
    }
  lds_barrier();                                  // all wavefronts are done with the buffers
  if (outs <= 0) return;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t from = row0 + (wm * TM + i) * 32;
    const int rows = (int)(a.n - from < 32 ? a.n - from : 32);
    if (rows <= 0) break;
    const float s = a.s[from + (m < rows ? m : 0)];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += V) {
        float f[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
          f[k] = (float)acc[i][j][e + k] * s * t[j][e + k];
          if (a.bias) f[k] += bias[j][e + k];
          if (a.act) f[k] = gelu(f[k]);
        }
        out[spot(m, (32 * j + 16 * h + e) / V)] = narrow<T, V>(f);
      }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    T* y = static_cast<T*>(a.y) + from * a.ld_y + first_out;
    if (wide) {
      constexpr int kAtOnce = 64 / PR;            // rows of a store
#pragma unroll
      for (int r = 0; r < 32; r += kAtOnce) {
        const int row = r + lane / PR, p = lane % PR;
        if (row < rows && p * V < outs) *reinterpret_cast<P*>(y + row * a.ld_y + p * V) = out[spot(row, p)];
      }
    } else {
      constexpr int kAtOnce = 64 / kWide;
      for (int r = 0; r < 32; r += kAtOnce) {
        const int row = r + lane / kWide, c = lane % kWide;
        if (row < rows && c < outs) y[row * a.ld_y + c] = reinterpret_cast<const T*>(out + spot(row, c / V))[c % V];
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
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
