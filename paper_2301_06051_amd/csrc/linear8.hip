// dsvt_linear_rows8: a linear layer on rows and weights in 8 bits (rows8.h).
//
//   y[n][o] = act(s_n t_o sum_c x[n][c] w[o][c] + b[o])
//
// The sum is of whole numbers, in 32 bits and exact (127^2 C < 2^31), whatever its order.
#include "rows8.h"
#include <type_traits>

namespace {

constexpr int kComputeUnits = 256;                // MI355X

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

// Few rows: the weights are what there is to read, and all of them should be on their way at once.  A workgroup takes 16 outputs and 16 kTiles rows; its
// eight wavefronts share the columns, in runs of 64, of which each has kAtOnce on their way.  Lane 16 g + m holds 16 codes of row m, from column 16 g of
// a run on.
constexpr int kFewWaves = 8;

template <typename T, int kTiles, int kAtOnce> __global__ __launch_bounds__(64 * kFewWaves) void k_linear8_few(Linear8Args a) {
  __shared__ i32x4 sums[kFewWaves - 1][kTiles][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4, out0 = blockIdx.x * 16;
  const int64_t row0 = (int64_t)blockIdx.y * 16 * kTiles;
  const int8_t* const w = a.w + (int64_t)(out0 + m < a.O ? out0 + m : a.O - 1) * a.ld_w;
  const int8_t* x[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int64_t row = row0 + 16 * t + m;
    x[t] = a.x + (row < a.n ? row : a.n - 1) * a.ld_x;
  }
  const int last_piece = (a.C - 1) >> 4 << 4, runs = ((a.C + 63) / 64 + kFewWaves - 1) / kFewWaves;
  const int from = 64 * runs * wave, to = from + 64 * runs < a.C ? from + 64 * runs : a.C;
  i32x4 acc[kTiles] = {};
  for (int k0 = from; k0 < to; k0 += 64 * kAtOnce) {
    i32x4 p[kAtOnce], q[kAtOnce][kTiles];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int k = k0 + 64 * u + 16 * g, at = k < last_piece ? k : last_piece;
      p[u] = *reinterpret_cast<const i32x4*>(w + at);
#pragma unroll
      for (int t = 0; t < kTiles; ++t) q[u][t] = *reinterpret_cast<const i32x4*>(x[t] + at);
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      // (past a row's end there may be anything, and past `to` there are the next wavefront's columns)
      if (k0 + 64 * (u + 1) > to) p[u] = first_bytes(p[u], to - (k0 + 64 * u + 16 * g));
#pragma unroll
      for (int t = 0; t < kTiles; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(p[u], q[u][t], acc[t], 0, 0, 0);
    }
  }
  if (wave) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) sums[wave - 1][t][lane] = acc[t];
  }
  // lane 16 g + m: outputs 4 g .. 4 g + 3 of row m
  const int out = out0 + 4 * g;
  float scale[4], bias[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = out + i < a.O ? out + i : a.O - 1;
    scale[i] = a.t[at];
    bias[i] = a.bias ? a.bias[at] : 0.f;
  }
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int64_t row = row0 + 16 * t + m;
    if (row >= a.n) continue;
#pragma unroll
    for (int k = 0; k < kFewWaves - 1; ++k) acc[t] += sums[k][t][lane];
    const float s = a.s[row];
    T* y = static_cast<T*>(a.y) + row * a.ld_y + out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = fmaf((float)acc[t][i] * s, scale[i], bias[i]);
      if (out + i < a.O) y[i] = (T)(a.act ? gelu(v) : v);
    }
  }
}

// 16 bytes a lane from memory, at base + off, straight into LDS, where the wavefront's 64 pieces lie one behind the other from `to` on.  Counted by
// vmcnt like other loads; the compiler does not know of it, so that only wait_for_stage() says when the data is there.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "m0");
}
// Until at most kLater loads of this wavefront are on their way and its LDS reads are done; then until all wavefronts are there.
template <int kLater> __device__ __forceinline__ void wait_for_stage() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLater) : "memory");
}

// Tiles of kRowsT rows and kOutsT outputs, shared by kM x kN wavefronts.  kColumns columns at a time go from memory into one of kBuffers buffers in
// LDS, kBuffers - 1 steps ahead.
//
// The matrix instruction takes 32 outputs, 32 rows and 32 columns: lane 32 h + m holds 16 codes of row m, from column 16 h on.  In LDS a row's
// 16-byte pieces are permuted, piece j of row r being at j ^ turn_of(r): the 16 lanes whose reads are served together (0-3, 12-15 and 20-27, or 4-11,
// 16-19 and 28-31 of a half) then hit all banks once.  Weights are read in another order of their rows, so that a lane's 16 sums of a tile are 16
// neighbouring outputs of one row.
template <int kRowsT, int kOutsT, int kColumns, int kBuffers> constexpr size_t tiles_lds() {
  return (size_t)kBuffers * (kRowsT + kOutsT) * kColumns + (2 * kOutsT + kRowsT) * sizeof(float);
}

template <typename T, int kRowsT, int kOutsT, int kM, int kN, int kColumns, int kBuffers>
__global__ __launch_bounds__(64 * kM * kN) void k_linear8_tiles(Linear8Args a) {
  constexpr int kWaves = kM * kN, TM = kRowsT / kM / 32, TN = kOutsT / kN / 32, kPieces = kColumns / 16, kSteps = kColumns / 32;
  constexpr int kAtOnceRows = 64 / kPieces;       // rows of one load of a wavefront
  constexpr int kLoads = (kRowsT + kOutsT) / (kWaves * kAtOnceRows), kLoadsX = kRowsT / (kWaves * kAtOnceRows);
  static_assert(kRowsT % (kWaves * kAtOnceRows) == 0 && kOutsT % (kWaves * kAtOnceRows) == 0, "rows are fetched by all wavefronts together");
  constexpr int kBuffer = (kRowsT + kOutsT) * kPieces;        // pieces of a buffer
  const auto turn_of = [](int r) { return kPieces == 4 ? r >> 2 & 3 : r >> 1 & 7; };
  extern __shared__ i32x4 lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % kM, wn = wave / kM, m = lane & 31, h = lane >> 5;
  // workgroups of one XCD (every eighth) take neighbouring tiles: eight along the rows, then the next outputs
  const int tiles_m = (a.n + kRowsT - 1) / kRowsT, tiles_n = (a.O + kOutsT - 1) / kOutsT, all = tiles_m * tiles_n;
  const int per = (all + 7) >> 3;
  int id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per || id >= all) return;
  const int band = id / (8 * tiles_n), bm = tiles_m - 8 * band < 8 ? tiles_m - 8 * band : 8;
  id -= band * 8 * tiles_n;
  const int64_t row0 = (int64_t)(8 * band + id % bm) * kRowsT;
  const int out0 = id / bm * kOutsT;

  // What this lane fetches: rows (i kWaves + wave) kAtOnceRows + lane / kPieces, past the last row the last one again, and of them the piece whose
  // place in LDS is the lane's.  Pieces past a row's end are its last one.
  const int8_t *x = a.x + row0 * a.ld_x, *w = a.w + (int64_t)out0 * a.ld_w;
  uint32_t off[kLoads];
  const int last_x = (int)(a.n - row0 < kRowsT ? a.n - row0 : kRowsT) - 1, last_w = (a.O - out0 < kOutsT ? a.O - out0 : kOutsT) - 1;
  const int piece = (lane % kPieces) ^ turn_of(wave * kAtOnceRows + lane / kPieces);
  static_assert(kWaves * kAtOnceRows % 16 == 0, "rows of one lane have one permutation");
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int r = ((i < kLoadsX ? i : i - kLoadsX) * kWaves + wave) * kAtOnceRows + lane / kPieces, last = i < kLoadsX ? last_x : last_w;
    off[i] = (uint32_t)(r < last ? r : last) * (uint32_t)(i < kLoadsX ? a.ld_x : a.ld_w) + 16u * piece;
  }
  const int last_piece = (a.C - 1) >> 4 << 4, last_step = (a.C - 1) / kColumns * kColumns;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)lds + 1024u * wave;
  const auto fetch = [&](int k0, int buffer) {
    k0 = k0 < last_step ? k0 : last_step;
    const uint32_t back = k0 + 16 * piece > last_piece ? k0 + 16 * piece - last_piece : 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_to_lds((i < kLoadsX ? x : w) + k0, off[i] - back, lds0 + 16u * kBuffer * buffer + 1024u * kWaves * i);
  };

#pragma unroll
  for (int k = 0; k < kBuffers - 1; ++k) fetch(k * kColumns, k);

  // the scales and biases of the tile, for its end
  float* const ends = reinterpret_cast<float*>(lds + kBuffers * kBuffer);
  for (int k = tid; k < kOutsT; k += 64 * kWaves) {
    const int at = out0 + (k < last_w ? k : last_w);
    ends[k] = a.t[at];
    ends[kOutsT + k] = a.bias ? a.bias[at] : 0.f;
  }
  for (int k = tid; k < kRowsT; k += 64 * kWaves) ends[2 * kOutsT + k] = a.s[row0 + (k < last_x ? k : last_x)];

  i32x16 acc[TM][TN] = {};
  const int out_m = (m >> 2 & 1) * 16 + (m >> 3) * 4 + (m & 3);
  const i32x4* const xs = lds + (wm * TM * 32 + m) * kPieces;
  const i32x4* const ws = lds + (kRowsT + wn * TN * 32 + out_m) * kPieces;
  struct Frags { i32x4 p[TN], q[TM]; } frags[2];
  const auto read = [&](Frags& f, int buffer, int k) {
#pragma unroll
    for (int t = 0; t < TN; ++t) f.p[t] = ws[buffer * kBuffer + t * 32 * kPieces + ((2 * k + h) ^ turn_of(out_m))];
#pragma unroll
    for (int t = 0; t < TM; ++t) f.q[t] = xs[buffer * kBuffer + t * 32 * kPieces + ((2 * k + h) ^ turn_of(m))];
  };
  const auto multiply = [&](const Frags& f) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.p[j], f.q[i], acc[i][j], 0, 0, 0);
  };

  // The fragments of a product are read while the one before is under way, the first ones of a buffer behind the barrier at which it is waited for.
  wait_for_stage<(kBuffers - 2) * kLoads>();
  fetch((kBuffers - 1) * kColumns, kBuffers - 1);
  read(frags[0], 0, 0);
  int buffer = 0, k0 = 0;
  for (; k0 < last_step; k0 += kColumns) {
#pragma unroll
    for (int k = 0; k < kSteps - 1; ++k) {
      read(frags[(k + 1) & 1], buffer, k + 1);
      multiply(frags[k & 1]);
    }
    const int free = buffer;
    buffer = buffer + 1 < kBuffers ? buffer + 1 : 0;
    wait_for_stage<(kBuffers - 2) * kLoads>();
    fetch(k0 + kBuffers * kColumns, free);
    read(frags[0], buffer, 0);
    multiply(frags[1]);
  }
  // what lies past a row's end may be anything; zeros in one operand do
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    if (k0 + 32 * k >= a.C) break;
    if (k) read(frags[0], buffer, k);
#pragma unroll
    for (int t = 0; t < TN; ++t) frags[0].p[t] = first_bytes(frags[0].p[t], a.C - k0 - 32 * k - 16 * h);
    multiply(frags[0]);
  }
  static_assert(kSteps % 2 == 0, "fragments change places");

  // Results go through LDS, 32 rows of a wavefront at a time, so that a row's are written side by side: as they come out of the product, a store would
  // write 32 pieces of 64 bytes.
  constexpr int kWide = TN * 32, V = 16 / (int)sizeof(T), PR = kWide / V;
  static_assert(PR == 4 || PR == 8 || PR == 16, "pieces of a row are permuted within 4 or 8");
  const auto spot = [](int row, int p) { return row * PR + (p ^ (PR == 4 ? row >> 1 & 3 : row & 7)); };
  typedef typename Piece<T, V>::type P;
  static_assert(kWaves * 32 * PR <= kBuffers * kBuffer, "the results of all wavefronts fit the buffers");
  P* const out = reinterpret_cast<P*>(lds) + wave * 32 * PR;
  const int first_out = out0 + wn * kWide, outs = a.O - first_out < kWide ? a.O - first_out : kWide;
  const bool wide = outs % V == 0 && ((uintptr_t)a.y & 15u) == 0 && a.ld_y * (int64_t)sizeof(T) % 16 == 0;
  wait_for_stage<0>();                            // nothing is on its way to the buffers, and all wavefronts are done with them
  if (outs <= 0) return;
  float t[TN][16], bias[TN][16];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int at = wn * kWide + j * 32 + 16 * h + e;
      const f32x4 t4 = *reinterpret_cast<const f32x4*>(ends + at), b4 = *reinterpret_cast<const f32x4*>(ends + kOutsT + at);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        t[j][e + k] = t4[k];
        bias[j][e + k] = b4[k];
      }
    }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t from = row0 + (wm * TM + i) * 32;
    const int rows = (int)(a.n - from < 32 ? a.n - from : 32);
    if (rows <= 0) break;
    const float s = ends[2 * kOutsT + (wm * TM + i) * 32 + m];
    const auto results = [&](auto act) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; e += V) {
          float f[V];
#pragma unroll
          for (int k = 0; k < V; ++k) f[k] = act(fmaf((float)acc[i][j][e + k] * s, t[j][e + k], bias[j][e + k]));
          out[spot(m, (32 * j + 16 * h + e) / V)] = narrow<T, V>(f);
        }
    };
    if (a.act) results([](float v) { return gelu(v); });
    else results([](float v) { return v; });
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

template <typename T, int kRowsT, int kOutsT, int kM, int kN, int kColumns, int kBuffers> int launch_tiles(const Linear8Args& a, hipStream_t st) {
  static std::atomic<uint64_t> allowed;
  const auto kernel = k_linear8_tiles<T, kRowsT, kOutsT, kM, kN, kColumns, kBuffers>;
  constexpr size_t lds = tiles_lds<kRowsT, kOutsT, kColumns, kBuffers>();
  if (const int rc = dsvt_allow_lds(reinterpret_cast<const void*>(kernel), lds, allowed)) return rc;
  const int64_t all = dsvt_ceil_div(a.n, kRowsT) * dsvt_ceil_div(a.O, kOutsT);
  kernel<<<(unsigned)(dsvt_ceil_div(all, 8) * 8), 64 * kM * kN, lds, st>>>(a);
  return DSVT_OK;
}
template <typename T> int launch(const Linear8Args& a, hipStream_t st) {
  const auto tiles = [&](int rows, int outs) { return dsvt_ceil_div(a.n, rows) * dsvt_ceil_div(a.O, outs); };
  // (rows of a tile, of either kind, are less than 2^31 bytes apart)
  if (a.n <= 64 || a.ld_x >= (1 << 23) || a.ld_w >= (1 << 23)) {
    const auto few = [&](auto rows, auto at_once) {
      constexpr int kTiles = decltype(rows)::value;
      const dim3 grid((unsigned)dsvt_ceil_div(a.O, 16), (unsigned)dsvt_ceil_div(a.n, 16 * kTiles));
      k_linear8_few<T, kTiles, decltype(at_once)::value><<<grid, 64 * kFewWaves, 0, st>>>(a);
    };
    const bool long_rows = a.C > 64 * kFewWaves * 2;
    if (a.n <= 16) long_rows ? few(std::integral_constant<int, 1>(), std::integral_constant<int, 8>()) : few(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
    else if (a.n <= 32) long_rows ? few(std::integral_constant<int, 2>(), std::integral_constant<int, 4>()) : few(std::integral_constant<int, 2>(), std::integral_constant<int, 2>());
    else few(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
    return DSVT_OK;
  }
  // The largest tiles that leave little of a last round over the 256 compute units empty: they read least from LDS and memory for a product.  (8,192 x
  // 4,096 -> 4,096: 149 us, 157 in tiles of 128, 301 of 64; 30,000 x 192 -> 576, 354 of the largest tiles: 20.1, 18.7 of 128, 19.0 of 64; 1,024 x 2,048 ->
  // 2,048, 128 tiles of 128: 14.3, 11.2 of 64.)
  const int64_t large = tiles(256, 256), rounds = dsvt_ceil_div(large, kComputeUnits);
  if (10 * large >= 8 * rounds * kComputeUnits) return launch_tiles<T, 256, 256, 2, 4, 128, 2>(a, st);
  if (tiles(128, 128) >= 2 * kComputeUnits) return launch_tiles<T, 128, 128, 2, 2, 128, 2>(a, st);
  return launch_tiles<T, 64, 64, 2, 2, 64, 3>(a, st);
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
