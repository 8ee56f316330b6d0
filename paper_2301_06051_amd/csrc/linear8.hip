// dsvt_linear_rows8: a linear layer on rows and weights in 8 bits (rows8.h).
//
//   y[n][o] = act(s_n t_o sum_c x[n][c] w[o][c] + b[o])
//
// The sum is of whole numbers, in 32 bits and exact (127^2 C < 2^31), whatever its order.
//
// Long rows are bound by the matrix cores, which three things feed at about the same rate: LDS (a wavefront of 128 x 64 reads 6 KB for eight
// products of 32 clocks), the loads of the next step, and the barrier of a step.  4,096 x 16,384 -> 4,096: 230 us, 2,390 TOP/s (the library's product
// of 8,192^3 in 8 bits 2,284 on the same card), 8,192 x 4,096 -> 4,096 with its 67 MB of results 120 to 130.  Short rows are bound by their results, whose
// instructions (a conversion, a product and an fma each) and stores have to run beside the products: 800,000 x 192 -> 576 183 us, 5.9 TB/s, by wavefronts
// on their own; 280 in tiles, whose workgroups do one after the other (220 without the results' instructions, 250 without their stores).
#include "rows8.h"
#include <cmath>
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
  bool leaves;                                    // rows_out
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

// GELU with its limits at the infinities, which a result may be (a row in 8 bits may not).
__device__ __forceinline__ float activation(float v) { return fabsf(v) == INFINITY ? fmaxf(v, 0.f) : gelu(v); }

// A result before its activation.  A sum is up to 2^30, so its product with a row's scale above 2^98 may pass 32 bits though that with the other scale, and so
// the result, does not: of rows whose scale is above kHuge the sum is multiplied by the other scale first, which passes 32 bits only if the result does.
constexpr float kHuge = 0x1p90f;
struct PlainRow {
  static __device__ __forceinline__ float result(int sum, float s, float t, float bias) { return fmaf((float)sum * s, t, bias); }
};
struct HugeRow {
  static __device__ __forceinline__ float result(int sum, float s, float t, float bias) { return fmaf((float)sum * t, s, bias); }
};
struct AnyRow {
  static __device__ __forceinline__ float result(int sum, float s, float t, float bias) { return fmaf((float)sum * (s > kHuge ? t : s), s > kHuge ? s : t, bias); }
};
// results(kind of row, activation) for a lane whose row's scale is s.  kBranch: huge rows have code of their own, which costs the others nothing but the
// registers that it takes.  (800,000 x 192 -> 576 207 us, as without huge rows; 214 with AnyRow's choice at every result; but 8,192 x 4,096 -> 4,096 of 32 bits 136
// without, 138 with the choice, 242 with code of their own, as registers go through memory then.)
template <bool kBranch, typename Results> __device__ __forceinline__ void with_activation(int act, float s, const Results& results) {
  const auto of = [&](auto row) {
    if (act) results(row, [](float v) { return activation(v); });
    else results(row, [](float v) { return v; });
  };
  if constexpr (!kBranch) of(AnyRow());
  else if (s > kHuge) of(HugeRow());
  else of(PlainRow());
}

// Few rows: the weights are what there is to read, and all of them should be on their way at once.  A workgroup takes 16 outputs and 16 kTiles rows; its
// eight wavefronts share the columns, in runs of 64, of which each has kAtOnce on their way.  Lane 16 g + m holds 16 codes of row m, from column 16 g of
// a run on.
constexpr int kFewWaves = 8;

template <typename T, int kTiles, int kAtOnce> __global__ __launch_bounds__(64 * kFewWaves) void k_linear8_few(Linear8Args a) {
  __shared__ i32x4 sums[kFewWaves - 1][kTiles][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4, out0 = blockIdx.y * 16;
  const int64_t row0 = (int64_t)blockIdx.x * 16 * kTiles;
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
      const float v = AnyRow::result(acc[t][i], s, scale[i], bias[i]);
      if (out + i < a.O) y[i] = (T)(a.act ? activation(v) : v);
    }
  }
}

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"    // m0 is the compiler's to reserve; it keeps nothing in it from one instruction to another
// 16 bytes a lane from memory, at base + off, straight into LDS, where the wavefront's 64 pieces lie one behind the other from `to` on.  Counted by
// vmcnt like other loads; the compiler does not know of it, so that only wait_for_stage() says when the data is there.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "m0");
}
// 4 bytes a lane likewise.
__device__ __forceinline__ void float_to_lds(const float* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(off), "s"(base) : "m0");
}
#pragma clang diagnostic pop
// Until at most kLater loads of this wavefront are on their way and its LDS reads are done; then until all wavefronts are there.
template <int kLater> __device__ __forceinline__ void wait_for_stage() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLater) : "memory");
}

// Results on their way out: kRowsOut rows of kWide values lie in a wavefront's LDS in pieces of 16 bytes, those of a row permuted, and are written row by
// row, in pieces that begin on any value.  Where rows are whole cache lines, stores are marked to leave the caches first (`leaves`), as rows and weights
// are to stay: 200,000 x 256 -> 1,024 132 -> 114 us, 100,000 x 384 -> 192 27 -> 24, and with a call that reads the results behind it 100,000 x 192 -> 576
// 84 -> 79 (30,000 the same).  Where they are not, lines would leave in parts: 400,000 x 200 -> 131 107 us marked, 72 not, 84 a value at a time.
template <int PR> __device__ __forceinline__ int spot(int row, int p) { return row * PR + (p ^ (PR == 4 ? row >> 1 & 3 : row & 7)); }
template <typename T, int kWide, int kRowsOut>
__device__ __forceinline__ void rows_out(const typename Piece<T, 16 / sizeof(T)>::type* out, T* y, int64_t ld_y, int rows, int outs, bool leaves, int lane) {
  constexpr int V = 16 / (int)sizeof(T), PR = kWide / V, kAtOnce = 64 / PR;     // rows of a store
  typedef typename Piece<T, V>::type P;
  typedef T Anywhere __attribute__((ext_vector_type(V), aligned(sizeof(T))));   // (rows begin on their type's alignment)
  const int row = lane / PR, c = lane % PR * V;
  T* const to = y + row * ld_y + c;
  const auto store = [&](int r, P p) {
    Anywhere* const at = reinterpret_cast<Anywhere*>(to + r * ld_y);
    if (leaves) {
      asm volatile("");                           // (as in write_out)
      __builtin_nontemporal_store((Anywhere)p, at);
      asm volatile("");
    } else *at = p;
  };
  if (rows == kRowsOut && outs == kWide) {
#pragma unroll
    for (int r = 0; r < kRowsOut; r += kAtOnce) store(r, out[spot<PR>(r + row, lane % PR)]);
  } else {
#pragma unroll
    for (int r = 0; r < kRowsOut; r += kAtOnce) {
      if (r + row >= rows || c >= outs) continue;
      const P p = out[spot<PR>(r + row, lane % PR)];
      if (c + V <= outs) store(r, p);
      else {
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
          if (c + i < outs) to[r * ld_y + i] = p[i];
      }
    }
  }
}

// Short rows: the weights of 64 outputs stay in a wavefront's registers, and it goes through blocks of 32 rows, which it reads straight into
// fragments, one block ahead.  Nothing is waited for together, so that one wavefront's products, results and stores run beside those of others.
// Wavefronts of the same rows are neighbours.  kSteps: of 32 columns, of which kWhole lie in the row for certain.
constexpr int kShortWaves = 4;
// Wavefronts a SIMD: two, a third one where registers allow it and it measured better (800,000 x 192 -> 576 198 -> 186 us; 100,000 x 64 -> 128 6.9 -> 8.7).
constexpr int short_simd(int steps, int elem) { return steps == 6 && elem == 2 ? 3 : 2; }

template <typename T, int kSteps, int kWhole>
__global__ __launch_bounds__(64 * kShortWaves, short_simd(kSteps, sizeof(T))) void k_linear8_short(Linear8Args a, int shares) {
  constexpr int V = 16 / (int)sizeof(T), PR = 64 / V, kRowsOut = sizeof(T) == 2 ? 32 : 16;
  typedef typename Piece<T, V>::type P;
  __shared__ P all_out[kShortWaves][kRowsOut * PR];
  __shared__ float all_ends[kShortWaves][2][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 31, h = lane >> 5;
  const int blocks_n = (a.O + 63) / 64, blocks_m = (a.n - 1) / 32 + 1;         // (n + 31 may pass 32 bits)
  const int groups = gridDim.x >> 3, at = ((blockIdx.x & 7) * groups + (blockIdx.x >> 3)) * kShortWaves + wave, share = at / blocks_n;
  if (share >= shares) return;
  const int out0 = at % blocks_n * 64, outs = a.O - out0 < 64 ? a.O - out0 : 64;
  const int last_piece = (a.C - 1) >> 4 << 4;

  i32x4 x[kSteps];
  float s;
  const auto fetch = [&](int block) {
    const int64_t row0 = (int64_t)block * 32;
    const int8_t* const base = a.x + row0 * a.ld_x;
    const uint32_t row = a.n - row0 > m ? m : (uint32_t)(a.n - row0) - 1u, off = row * (uint32_t)a.ld_x;
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const int c = 32 * k + 16 * h;
      x[k] = *reinterpret_cast<const i32x4*>(base + (off + (k < kWhole || c < last_piece ? c : last_piece)));
    }
    s = a.s[row0 + row];
  };
  // The first rows, scales, biases and weights are on their way together.  (There are no more shares than blocks.)
  int block = share;
  fetch(block);
  const int end = out0 + (lane < outs ? lane : outs - 1);
  const float scale_out = a.t[end], bias_out = a.bias ? a.bias[end] : 0.f;
  i32x4 w[2][kSteps];
  const int out_m = (m >> 2 & 1) * 16 + (m >> 3) * 4 + (m & 3);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int o = 32 * j + out_m;
    const int8_t* row = a.w + (int64_t)(out0 + (o < outs ? o : outs - 1)) * a.ld_w;
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const int c = 32 * k + 16 * h;
      w[j][k] = *reinterpret_cast<const i32x4*>(row + (k < kWhole || c < last_piece ? c : last_piece));
    }
  }
  float* const ends = all_ends[wave][0];
  ends[lane] = scale_out;
  ends[64 + lane] = bias_out;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int k = kWhole; k < kSteps; ++k) w[j][k] = first_bytes(w[j][k], a.C - 32 * k - 16 * h);
  P* const out = all_out[wave];
  const auto in_order = []() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  in_order();
  for (; block < blocks_m; block += shares) {
    i32x16 acc[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      acc[j] = i32x16{};
#pragma unroll
      for (int k = 0; k < kSteps; ++k) acc[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[j][k], x[k], acc[j], 0, 0, 0);
    }
    const float scale = s;
    fetch(block + shares < blocks_m ? block + shares : block);
    const int64_t row0 = (int64_t)block * 32;
#pragma unroll
    for (int part = 0; part < 32 / kRowsOut; ++part) {
      const int left = (int)(a.n - row0 - kRowsOut * part < kRowsOut ? a.n - row0 - kRowsOut * part : kRowsOut);
      if (left <= 0) break;
      if (m / kRowsOut == part) {
        const auto results = [&](auto row, auto act) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            int from = 32 * j + 16 * h;
            asm volatile("" : "+v"(from));        // (read again for every block: registers hold the weights)
#pragma unroll
            for (int e = 0; e < 16; e += V) {
              float f[V];
#pragma unroll
              for (int k = 0; k < V; k += 4) {
                const f32x4 t = *reinterpret_cast<const f32x4*>(ends + from + e + k), bias = *reinterpret_cast<const f32x4*>(ends + 64 + from + e + k);
#pragma unroll
                for (int u = 0; u < 4; ++u) f[k + u] = act(row.result(acc[j][e + k + u], scale, t[u], bias[u]));
              }
              out[spot<PR>(m % kRowsOut, (32 * j + 16 * h + e) / V)] = narrow<T, V>(f);
            }
          }
        };
        with_activation<true>(a.act, scale, results);
      }
      in_order();
      rows_out<T, 64, kRowsOut>(out, static_cast<T*>(a.y) + (row0 + kRowsOut * part) * a.ld_y + out0, a.ld_y, left, outs, a.leaves, lane);
      in_order();
    }
  }
}

// Tiles of kRowsT rows and kOutsT outputs, shared by kM x kN wavefronts.  Their columns, kColumns at a time, go from memory into one of kBuffers
// buffers in LDS, kBuffers - 1 steps ahead.  kStay: a workgroup stays and takes tiles in turn, and the steps ahead go over the tiles' borders: while
// one tile's results are written, the next one's rows and weights are on their way.
//
// The matrix instruction takes 32 outputs, 32 rows and 32 columns: lane 32 h + m holds 16 codes of row m, from column 16 h on.  In LDS a row's
// 16-byte pieces are permuted, piece j of row r being at j ^ turn_of(r): the 16 lanes whose reads are served together (0-3, 12-15 and 20-27, or 4-11,
// 16-19 and 28-31 of a half) then hit all banks once.  Weights are read in another order of their rows, so that a lane's 16 sums of a tile are 16
// neighbouring outputs of one row.
template <typename T, int kRowsT, int kOutsT, int kM, int kN, int kColumns, int kBuffers> struct Tiles {
  static constexpr int kWaves = kM * kN, TM = kRowsT / kM / 32, TN = kOutsT / kN / 32, kPieces = kColumns / 16, kSteps = kColumns / 32;
  static constexpr int kAtOnceRows = 64 / kPieces;            // rows of one load of a wavefront
  static constexpr int kLoads = (kRowsT + kOutsT) / (kWaves * kAtOnceRows), kLoadsX = kRowsT / (kWaves * kAtOnceRows);
  static_assert(kRowsT % (kWaves * kAtOnceRows) == 0 && kOutsT % (kWaves * kAtOnceRows) == 0, "rows are fetched by all wavefronts together");
  static_assert(kWaves * kAtOnceRows % 16 == 0, "rows of one lane have one permutation");
  static constexpr int kBuffer = (kRowsT + kOutsT) * kPieces;              // pieces of a buffer
  // results of a wavefront on their way out: kRowsOut rows of kWide values, V to a piece
  static constexpr int kRowsOut = sizeof(T) == 2 ? 32 : 16, kWide = TN * 32, V = 16 / (int)sizeof(T), PR = kWide / V, kOut = kRowsOut * PR;
  static_assert(PR == 4 || PR == 8 || PR == 16, "pieces of a row are permuted within 4 or 8");
  static constexpr int kEnds = 2 * kOutsT + kRowsT;           // scales of outputs, their biases, scales of rows
  static constexpr int kEndLoads = (kEnds + 64 * kWaves - 1) / (64 * kWaves);
  static constexpr int kEndPlaces = kEndLoads * 64 * kWaves;
  static_assert(kWaves * kOut <= kBuffer, "the results of all wavefronts fit a buffer");
  static constexpr int kStores = TM * 32 / (64 / PR);         // of a wavefront, of whole rows
  static constexpr size_t lds() { return (size_t)kBuffers * (16 * kBuffer + 4 * kEndPlaces); }
};

template <typename T, int kRowsT, int kOutsT, int kM, int kN, int kColumns, int kBuffers, bool kStay>
__global__ __launch_bounds__(64 * kM * kN) void k_linear8_tiles(Linear8Args a) {
  typedef Tiles<T, kRowsT, kOutsT, kM, kN, kColumns, kBuffers> S;
  constexpr int kWaves = S::kWaves, TM = S::TM, TN = S::TN, kPieces = S::kPieces, kSteps = S::kSteps, kLoads = S::kLoads, kLoadsX = S::kLoadsX;
  constexpr int kBuffer = S::kBuffer, V = S::V, PR = S::PR, kWide = S::kWide, kRowsOut = S::kRowsOut;
  const auto turn_of = [](int r) { return kPieces == 4 ? r >> 2 & 3 : r >> 1 & 7; };
  extern __shared__ i32x4 lds[];
  float* const all_ends = reinterpret_cast<float*>(lds + kBuffers * kBuffer);
  typedef typename Piece<T, V>::type P;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % kM, wn = wave / kM, m = lane & 31, h = lane >> 5;

  // Workgroups of one XCD (every eighth) take neighbouring tiles side by side: eight along the rows, then the next outputs.
  const int tiles_m = (a.n - 1) / kRowsT + 1, tiles_n = (a.O + kOutsT - 1) / kOutsT, all = tiles_m * tiles_n;
  const int share = (all + 7) >> 3, first = (blockIdx.x & 7) * share, end = first + share < all ? first + share : all, step = gridDim.x >> 3;
  int id = first + (blockIdx.x >> 3);
  if (id >= end) return;
  struct Place { int64_t row0; int out0; };
  const auto place_of = [&](int i) {
    const int band = i / (8 * tiles_n), rest = tiles_m - 8 * band, bm = rest < 8 ? rest : 8;
    i -= band * 8 * tiles_n;
    return Place{(int64_t)(8 * band + i % bm) * kRowsT, i / bm * kOutsT};
  };

  // The fetching side, ahead of the other: its tile and column.  A lane fetches rows (i kWaves + wave) kAtOnceRows + lane / kPieces, past the last row
  // the last one again, and of them the piece whose place in LDS is the lane's; pieces past a row's end are its last one.  Behind the last
  // tile it goes on with that one.
  const int last_piece = (a.C - 1) >> 4 << 4, last_step = (a.C - 1) / kColumns * kColumns;
  const int piece = (lane % kPieces) ^ turn_of(wave * S::kAtOnceRows + lane / kPieces);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)lds;
  int next_id = id, next_k = 0, next_buffer = 0, next_ends = 0;
  const int8_t *x, *w;
  uint32_t off[kLoads];
  const auto fetch = [&](bool begin) {
    if (kStay ? next_k == 0 : begin) {
      const Place at = place_of(next_id);
      x = a.x + at.row0 * a.ld_x;
      w = a.w + (int64_t)at.out0 * a.ld_w;
      const int last_x = (int)(a.n - at.row0 < kRowsT ? a.n - at.row0 : kRowsT) - 1, last_w = (a.O - at.out0 < kOutsT ? a.O - at.out0 : kOutsT) - 1;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = ((i < kLoadsX ? i : i - kLoadsX) * kWaves + wave) * S::kAtOnceRows + lane / kPieces, last = i < kLoadsX ? last_x : last_w;
        off[i] = (uint32_t)(r < last ? r : last) * (uint32_t)(i < kLoadsX ? a.ld_x : a.ld_w) + 16u * piece;
      }
      // scales and biases: 64 values a wavefront and load (without biases some that are not used)
#pragma unroll
      for (int i = 0; i < S::kEndLoads; ++i) {
        const int from = (i * kWaves + wave) * 64;            // (kOutsT and kRowsT are multiples of 64)
        const float* base = from < kOutsT ? a.t + at.out0 : from < 2 * kOutsT && a.bias ? a.bias + at.out0 : from < 2 * kOutsT ? a.t + at.out0 : a.s + at.row0;
        const int at_end = from < kOutsT ? from : from < 2 * kOutsT ? from - kOutsT : from < S::kEnds ? from - 2 * kOutsT : 0, most = from < 2 * kOutsT ? last_w : last_x;
        const int k = at_end + lane;
        float_to_lds(base, 4u * (uint32_t)(k < most ? k : most), lds0 + 16u * kBuffers * kBuffer + 4u * (next_ends * S::kEndPlaces + from));
      }
      next_ends = next_ends + 1 < kBuffers ? next_ends + 1 : 0;
    }
    const uint32_t back = next_k + 16 * piece > last_piece ? next_k + 16 * piece - last_piece : 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      load_to_lds((i < kLoadsX ? x : w) + next_k, off[i] - back, lds0 + 16u * kBuffer * next_buffer + 1024u * (kWaves * i + wave));
    next_buffer = next_buffer + 1 < kBuffers ? next_buffer + 1 : 0;
    next_k += kColumns;
    if (next_k > last_step) {
      next_k = kStay ? 0 : last_step;
      next_id = next_id + step < end ? next_id + step : next_id;
    }
  };

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
  i32x16 acc[TM][TN];
  const auto multiply = [&](const Frags& f) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.p[j], f.q[i], acc[i][j], 0, 0, 0);
  };
  static_assert(kSteps % 2 == 0, "fragments change places");

  // The fragments of a product are read while the one before is under way, the first ones of a buffer behind the barrier at which it is waited for.
  // At that barrier all wavefronts are done with the buffer before, which is then fetched into.
#pragma unroll
  for (int k = 0; k < kBuffers - 1; ++k) fetch(k == 0);
  // Stores are counted with the loads.  Behind a whole tile's, which are as many for every such tile, the next kBuffers - 1 steps were fetched before
  // them: waiting for those is not waiting for the stores.
  int buffer = 0, ends_at = 0, stored = 0;
  const auto wait = [&]() {
    constexpr int kLater = (kBuffers - 2) * kLoads;
    if (kStay && stored > 0 && kLater + S::kStores < 63) wait_for_stage<(kLater + S::kStores < 63 ? kLater + S::kStores : 0)>();
    else wait_for_stage<kLater>();
    --stored;
  };
  for (; id < end; id += step) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = i32x16{};
    wait();
    fetch(false);
    read(frags[0], buffer, 0);
    int k0 = 0;
    for (; k0 < last_step; k0 += kColumns) {
#pragma unroll
      for (int k = 0; k < kSteps - 1; ++k) {
        read(frags[(k + 1) & 1], buffer, k + 1);
        multiply(frags[k & 1]);
      }
      buffer = buffer + 1 < kBuffers ? buffer + 1 : 0;
      wait();
      fetch(false);
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

    // Results go through LDS, kRowsOut rows of a wavefront at a time, so that a row's are written side by side: as they come out of the product, a store
    // would write 32 pieces of 64 bytes.  There the buffer is free that was multiplied last, once all wavefronts are done with it.
    lds_barrier();
    P* const out = reinterpret_cast<P*>(lds + buffer * kBuffer) + wave * S::kOut;
    buffer = buffer + 1 < kBuffers ? buffer + 1 : 0;
    const Place at = place_of(id);
    const float* const ends = all_ends + ends_at * S::kEndPlaces;
    ends_at = ends_at + 1 < kBuffers ? ends_at + 1 : 0;
    const int first_out = at.out0 + wn * kWide, outs = a.O - first_out < kWide ? a.O - first_out : kWide;
    const bool whole = a.n - at.row0 >= kRowsT && outs == kWide;
    stored = whole ? kBuffers - 1 : 0;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t from = at.row0 + (wm * TM + i) * 32;
      const float s = ends[2 * kOutsT + (wm * TM + i) * 32 + m];
#pragma unroll
      for (int part = 0; part < 32 / kRowsOut; ++part) {
        const int rows = (int)(a.n - from - kRowsOut * part < kRowsOut ? a.n - from - kRowsOut * part : kRowsOut);
        if (rows <= 0 || outs <= 0) break;
        if (m / kRowsOut == part) {
          const auto results = [&](auto row, auto act) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
              for (int e = 0; e < 16; e += V) {
                float f[V];
#pragma unroll
                for (int k = 0; k < V; k += 4) {
                  const int o = wn * kWide + j * 32 + 16 * h + e + k;
                  const f32x4 t = *reinterpret_cast<const f32x4*>(ends + o);
                  f32x4 bias = {0.f, 0.f, 0.f, 0.f};
                  if (a.bias) bias = *reinterpret_cast<const f32x4*>(ends + kOutsT + o);
#pragma unroll
                  for (int u = 0; u < 4; ++u) f[k + u] = act(row.result(acc[i][j][e + k + u], s, t[u], bias[u]));
                }
                out[spot<PR>(m % kRowsOut, (32 * j + 16 * h + e) / V)] = narrow<T, V>(f);
              }
          };
          with_activation<!(sizeof(T) == 4 && kRowsT == 256)>(a.act, s, results);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        T* y = static_cast<T*>(a.y) + (from + kRowsOut * part) * a.ld_y + first_out;
        rows_out<T, kWide, kRowsOut>(out, y, a.ld_y, rows, outs, a.leaves, lane);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
    }
    if (!kStay) break;
  }
  wait_for_stage<0>();                            // nothing is on its way to LDS any more that will be another workgroup's
}

// stay: as many workgroups a compute unit; 0: one a tile
template <typename T, int kRowsT, int kOutsT, int kM, int kN, int kColumns, int kBuffers, int kStay> int launch_tiles(const Linear8Args& a, hipStream_t st) {
  typedef Tiles<T, kRowsT, kOutsT, kM, kN, kColumns, kBuffers> S;
  static std::atomic<uint64_t> allowed;
  const auto kernel = k_linear8_tiles<T, kRowsT, kOutsT, kM, kN, kColumns, kBuffers, kStay != 0>;
  if (const int rc = dsvt_allow_lds(reinterpret_cast<const void*>(kernel), S::lds(), allowed)) return rc;
  const int64_t all = dsvt_ceil_div(dsvt_ceil_div(a.n, kRowsT) * dsvt_ceil_div(a.O, kOutsT), 8) * 8, at_once = (int64_t)kComputeUnits * kStay;
  kernel<<<(unsigned)(kStay == 0 || all < at_once ? all : at_once), 64 * kM * kN, S::lds(), st>>>(a);
  return DSVT_OK;
}
template <typename T> int launch(const Linear8Args& a, hipStream_t st) {
  const auto tiles = [&](int rows, int outs) { return dsvt_ceil_div(a.n, rows) * dsvt_ceil_div(a.O, outs); };
  // Long rows whose tiles would be too few to fetch the weights at once: 64 x 4,096 -> 192 13.1 us in tiles of 64, 8.4 here; -> 4,096 (64 tiles) 14.5 and 14.3.
  // (Rows of a tile, of either kind, are less than 2^31 bytes apart.)
  const bool long_rows = a.C > 64 * kFewWaves * 2;
  if (a.n <= 32 || (long_rows && tiles(64, 64) < 64) || a.ld_x >= (1 << 23) || a.ld_w >= (1 << 23)) {
    const auto few = [&](auto rows, auto at_once) {
      constexpr int kTiles = decltype(rows)::value;
      const dim3 grid((unsigned)dsvt_ceil_div(a.n, 16 * kTiles), (unsigned)dsvt_ceil_div(a.O, 16));
      k_linear8_few<T, kTiles, decltype(at_once)::value><<<grid, 64 * kFewWaves, 0, st>>>(a);
    };
    if (a.n <= 16) long_rows ? few(std::integral_constant<int, 1>(), std::integral_constant<int, 8>()) : few(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
    else long_rows ? few(std::integral_constant<int, 2>(), std::integral_constant<int, 4>()) : few(std::integral_constant<int, 2>(), std::integral_constant<int, 2>());
    return DSVT_OK;
  }
  // Short rows of which every wavefront has two blocks at least; with results of 32 bits or GELU, which cost more, rows up to 256.  us by wavefronts on their
  // own and in the best tiles: 800,000 x 192 -> 576 183 and 279, 30,000 11.7 and 13.0, 100,000 x 64 -> 128 6.9 and 10.2, 200,000 x 256 -> 1,024 122 and 112, of 32
  // bits 155 and 177, with GELU 182 and 195, 100,000 x 384 -> 192 27 and 22; with one block 9,973 x 99 -> 130 5.9 and 5.0.
  const bool costly = a.act || sizeof(T) == 4;       // results
  if (a.C <= (costly ? 256 : 192)) {
    const int64_t blocks_n = dsvt_ceil_div(a.O, 64), blocks_m = dsvt_ceil_div(a.n, 32);
    const auto go = [&](auto steps, auto whole) {
      constexpr int kSteps = decltype(steps)::value;
      const int64_t at_once = (int64_t)kComputeUnits * 4 * short_simd(kSteps, sizeof(T)) / blocks_n, rounds = dsvt_ceil_div(blocks_m, at_once);
      if (rounds < 2) return false;
      const int64_t shares = rounds <= 3 ? dsvt_ceil_div(blocks_m, rounds) : at_once;
      const unsigned grid = (unsigned)dsvt_ceil_div(dsvt_ceil_div(shares * blocks_n, kShortWaves), 8) * 8;
      k_linear8_short<T, kSteps, decltype(whole)::value><<<grid, 64 * kShortWaves, 0, st>>>(a, (int)shares);
      return true;
    };
    if (a.C <= 64 ? go(std::integral_constant<int, 2>(), std::integral_constant<int, 0>())
        : a.C <= 128 ? go(std::integral_constant<int, 4>(), std::integral_constant<int, 2>())
        : a.C <= 192 ? go(std::integral_constant<int, 6>(), std::integral_constant<int, 4>())
                     : go(std::integral_constant<int, 8>(), std::integral_constant<int, 6>()))
      return DSVT_OK;
  }
  // The largest tiles that leave little of a last round over the 256 compute units empty: they read least from LDS and memory for a product.  us a
  // call with tiles of 256 x 256, 128 x 128, 128 x 64, 64 x 64 (the first two stay): 8,192 x 4,096 -> 4,096 125, 150, 172, 300; 10,000 x 512 -> 2,048 26.6, 20.2,
  // 24.4, 30.2; 30,000 x 384 -> 192 12.0, 9.0, 8.1, 9.9; 1,024 x 2,048 -> 2,048 27.2, 14.8, 12.3, 10.6; 200,000 x 512 -> 64 49, 32, 30.5; 100,000 x 1,024 -> 320 72, 58, 60.
  // A workgroup alone on its compute unit does nothing beside results that cost more: 200,000 x 256 -> 1,024 112, 126, 156, but of 32 bits 191, 177, 209, with
  // GELU 209, 195, 211; 16,384 x 512 -> 4,096 of 32 bits 75, 82, with GELU 86, 86.
  // Of long rows a round of the largest tiles may leave more of the chip empty: 28,652 x 4,153 -> 384 70, 84, 90, 136; 20,000 x 4,096 -> 512 57, 62, 66, 105;
  // 6,000 x 4,096 -> 2,048 58, 60, 67, 121; 2,000 x 4,096 -> 4,096 52, 40, 50, 82; 30,000 x 1,024 -> 1,152 59, 52, 59, 88.
  const bool more = a.C >= 2048;
  const int64_t rounds = dsvt_ceil_div(tiles(256, 256), kComputeUnits);
  if ((int64_t)a.n * a.O >= rounds * (kComputeUnits * 256 * 256 / 10 * (more ? 6 : 8)) && !(costly && a.C < 512))
    return launch_tiles<T, 256, 256, 2, 4, 128, 2, 1>(a, st);
  if (tiles(128, 128) >= kComputeUnits * (more ? 3 : 8) / 2 && a.O > 64) return launch_tiles<T, 128, 128, 4, 2, 128, 2, 2>(a, st);
  if (tiles(128, 64) >= 2 * kComputeUnits) return launch_tiles<T, 128, 64, 4, 1, 128, 2, 0>(a, st);
  return launch_tiles<T, 64, 64, 2, 2, 64, 3, 0>(a, st);
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
  a.leaves = (((uintptr_t)y | (uintptr_t)(ld_y * (cfg->dtype == DSVT_BF16 ? 2 : 4))) & 127u) == 0;
  a.y = y; a.ld_y = ld_y; a.n = n_rows; a.C = cfg->C; a.O = cfg->out; a.act = cfg->act;
  hipStream_t st = (hipStream_t)stream;
  {
    dsvt_prof_scope ps(DSVT_K_LINEAR8, st);
    if (const int rc = cfg->dtype == DSVT_BF16 ? launch<bf16_t>(a, st) : launch<float>(a, st)) return rc;
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}
