// dsvt_linear_rows8_weight_grad: the gradients of a linear layer's weights and bias from its input as it was kept in 8 bits (rows8.h).
//
//   d_w[o][c] = sum_n dy[n][o] s_n x[n][c],  d_b[o] = sum_n dy[n][o]
//
// The sums run over the rows: workgroups take a tile of outputs and columns and a slice of the rows each, and leave partial sums in 32 bits, which
// a second kernel adds up in the slices' order; one slice writes the results itself.  Rows go from memory through registers into one of two buffers in
// LDS, the kept ones as s_n x[n][c].  Products of 32-bit operands run at a sixteenth of the rate of bf16, of which one would round s_n x[n][c] to 8 bits; it is
// taken as two, its first bits and the rest, at twice the products: the result is off by its own rounding, 1.7e-3 of its norm (2.3e-3 with one
// operand, and no number where that passes bf16), for 1.1 to 1.6 times the time.
//
// Both operands run along the rows, so both have to be turned round, which the LDS loads do (bf16).  With tiles of 256 a step of 32 rows is 2,048 clocks of
// the matrix cores, 1,400 of LDS and some 900 of the making of values from codes, only partly at once: 65,536 rows of 1,024 -> 2,048 475 to 480 us (1,190 TFLOP/s
// of products; the library's of 8,192^3 in bf16 1,362).  Few columns leave the partial sums and a step's latency: 30,000 rows of 192 -> 576 28 us, five of them the
// second kernel.
#include "rows8.h"
#include <cmath>

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef double f64x4 __attribute__((ext_vector_type(4)));
typedef short short4_t __attribute__((ext_vector_type(4)));

struct Grad8Args {
  const int8_t* x;
  const float* s;
  const void* dy;
  void* d_w;                                      // written if there is one slice
  float *d_b, *partial, *bias_partial;            // d_b: null if not wanted; [slices] tiles, squares of 32 as lanes hold them; [slices][O]
  int64_t ld_x, ld_dy, ld_dw;
  int32_t n, C, O;
  int32_t slices, slice;                          // slices, rows of one (a multiple of a step's)
};

// Operand fragments out of LDS, where rows lie one after the other: 32 neighbouring columns, and the rows of one matrix instruction.
template <typename T> struct Columns;
template <> struct Columns<bf16_t> {
  static constexpr int kStep = 16, kTerms = 2;    // rows of an instruction; operands that a kept value is taken as
  static constexpr int kPad = 64;                 // bytes that pad a row in LDS: a fragment's four rows then lie in all banks
  typedef bf16x8 Frag;
  static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  // Lane 32 h + m gets rows 8 h .. 8 h + 7 of column m.  Of 16 lanes, the load takes four rows of four pieces of four columns, and hands lane i the
  // rows of column i % 4 of piece i / 4.  kTurn: which piece is which, so that lane m holds column 16 (m / 4 % 2) + 4 (m / 8) + m % 4.
  template <bool kTurn> static __device__ __forceinline__ Frag load(const char* p, int pitch) {
    const int lane = threadIdx.x & 63, h = lane >> 5, a = lane >> 4 & 1, j = lane >> 2 & 3, q = lane & 3;
    const int quad = kTurn ? 4 * (q & 1) + 2 * a + (q >> 1) : 4 * a + q;
    const char* at = p + (8 * h + j) * pitch + 8 * quad;
    typedef __attribute__((address_space(3))) short4_t lds_short4;
    const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(uintptr_t)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)at);
    const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(uintptr_t)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)(at + 4 * pitch));
    return __builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};
template <> struct Columns<float> {
  static constexpr int kStep = 2, kTerms = 1, kPad = 128;
  typedef float Frag;
  static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
  template <bool kTurn> static __device__ __forceinline__ Frag load(const char* p, int pitch) {
    const int lane = threadIdx.x & 63, h = lane >> 5, m = lane & 31;
    const int column = kTurn ? 16 * (m >> 2 & 1) + 4 * (m >> 3) + (m & 3) : m;
    return *reinterpret_cast<const float*>(p + h * pitch + 4 * column);
  }
};

// How rows of dy end: with a whole piece of 16 bytes; within one, which is then fetched so that it ends there, and shifted; or before the first one
// does, in which case values are fetched one by one.
enum Ends { kWhole, kShifted, kSingly };

// A tile of kO outputs and kC columns, shared by kWO x kWC wavefronts, each of which has TO x TC squares of 32.
struct Shape { int kO, kC, kWO, TO, TC; };

// kN rows at a time; those of kAhead steps are on their way.
template <typename T, int kO, int kC, int kWO, int kWC, int kN, int kAhead> struct Tile {
  static constexpr int kAll = 64 * kWO * kWC, TO = kO / kWO / 32, TC = kC / kWC / 32, V = 16 / (int)sizeof(T);
  static constexpr int kPitchO = kO * (int)sizeof(T) + Columns<T>::kPad, kPlaneC = kC * (int)sizeof(T), kPitchC = Columns<T>::kTerms * kPlaneC + Columns<T>::kPad;
  static constexpr int kBuffer = kN * (kPitchO + kPitchC);
  static constexpr int kRowsO = kAll / (kO / V), kRowsC = kAll / (kC / 8);      // rows that all threads fetch at once, in pieces of 16 bytes of dy and 8 codes
  static constexpr int PO = kN / kRowsO, PC = kN / kRowsC;
  static_assert(kAll % (kO / V) == 0 && kAll % (kC / 8) == 0 && kN % kRowsO == 0 && kN % kRowsC == 0, "rows are fetched by all threads together");
  static constexpr size_t lds() { return 2 * (size_t)kBuffer > (size_t)kRowsO * kO * 4 ? 2 * (size_t)kBuffer : (size_t)kRowsO * kO * 4; }
};

// The first `left` of V values (all if there are more) to neighbouring places that begin on any value.
template <typename T, int V> __device__ __forceinline__ void write_some(T* to, const float (&f)[V], int left) {
  typedef T Anywhere __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  const typename Piece<T, V>::type p = narrow<T, V>(f);
  if (left >= V) *reinterpret_cast<Anywhere*>(to) = p;
  else {
#pragma unroll
    for (int k = 0; k < V - 1; ++k)
      if (k < left) to[k] = p[k];
  }
}

extern __shared__ __attribute__((aligned(16))) char grad_lds[];

template <typename T, int kO, int kC, int kWO, int kWC, int kN, int kAhead, Ends kEnds> __global__ __launch_bounds__(64 * kWO * kWC) void k_linear8_grad(Grad8Args a) {
  typedef Tile<T, kO, kC, kWO, kWC, kN, kAhead> S;
  typedef Columns<T> F;
  constexpr int V = S::V, TO = S::TO, TC = S::TC, PO = S::PO, PC = S::PC;
  typedef typename Piece<T, V>::type P;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wo = wave % kWO, wc = wave / kWO, m = lane & 31, h = lane >> 5;
  // workgroups of one XCD (every eighth) take the tiles of one slice, then of the next
  const int tiles_c = (a.C + kC - 1) / kC, tiles_o = (a.O + kO - 1) / kO, tiles = tiles_c * tiles_o, all = tiles * a.slices, per = (all + 7) >> 3;
  const int id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per || id >= all) return;
  const int slice = id / tiles, tile = id - slice * tiles, o0 = tile / tiles_c * kO, c0 = (tile - tile / tiles_c * tiles_c) * kC;
  const int64_t first = (int64_t)slice * a.slice, last = first + a.slice < a.n ? first + a.slice : a.n;
  const bool sums = a.d_b && c0 == 0;

  // Threads past the last output or column fetch the first ones of the tile.  A step whose rows would pass the slice's last takes the last kN ones,
  // of which those of the step before count as zeros: what is fetched, and from where, hangs on no condition, which would have to wait for it.
  const int piece_o = tid % (kO / V), row_o = tid / (kO / V), piece_c = tid % (kC / 8), row_c = tid / (kC / 8);
  // (a piece that would pass a row's end is fetched so that it ends there, and shifted when it is put into LDS)
  const int want_o = V * piece_o < a.O - o0 ? V * piece_o : 0, most_o = a.O - o0 - V, o = kEnds != kShifted || want_o < most_o ? want_o : most_o;
  const int shift = 8 * (int)sizeof(T) * (want_o - o), c = 8 * piece_c < a.C - c0 ? 8 * piece_c : 0;
  const int rows = (int)(last - first < kN ? last - first : kN);
  const int64_t last_step = last - rows;
  uint32_t off_o[PO], off_c[PC], off_s[PC];
#pragma unroll
  for (int i = 0; i < PO; ++i) {
    const int r = row_o + i * S::kRowsO;
    off_o[i] = (uint32_t)(r < rows ? r : rows - 1) * (uint32_t)a.ld_dy + (uint32_t)o;
  }
#pragma unroll
  for (int i = 0; i < PC; ++i) {
    const int r = row_c + i * S::kRowsC;
    off_s[i] = r < rows ? r : rows - 1;
    off_c[i] = off_s[i] * (uint32_t)a.ld_x + c;
  }
  struct Stage {                                  // what this thread has fetched of the rows of one step
    P dy[PO];
    uint2 x[PC];
    float s[PC];
  } stages[kAhead];
  const auto fetch = [&](Stage& g, int64_t n0) {
    const int64_t from = n0 < last_step ? n0 : last_step;
    const int8_t* x = a.x + from * a.ld_x + c0;
    const float* s = a.s + from;
    const T* dy = static_cast<const T*>(a.dy) + from * a.ld_dy + o0;
#pragma unroll
    for (int i = 0; i < PC; ++i) {
      g.x[i] = *reinterpret_cast<const uint2*>(x + off_c[i]);
      g.s[i] = s[off_s[i]];
    }
#pragma unroll
    for (int i = 0; i < PO; ++i) {
      const T* p = dy + (int32_t)off_o[i];
      if constexpr (kEnds == kSingly) {
#pragma unroll
        for (int e = 0; e < V; ++e) g.dy[i][e] = p[o + e < a.O ? e : 0];
      } else __builtin_memcpy(&g.dy[i], p, 16);   // (on any element)
    }
  };
  // Of what was fetched, part k of kSteps goes to LDS.
  constexpr int kSteps = kN / F::kStep;
  float db[V] = {};
  const auto put = [&](Stage& g, int64_t n0, int buffer, int k) {
    char* to = grad_lds + buffer * S::kBuffer;
    const int before = n0 > last_step ? (int)(n0 - last_step < kN ? n0 - last_step : kN) : 0;     // rows of the step before
#pragma unroll
    for (int i = k; i < PC; i += kSteps) {
      // (the compiler would take the bytes apart, and wait for them, where they are fetched)
      asm volatile("" : "+v"(g.x[i].x), "+v"(g.x[i].y), "+v"(g.s[i]));
      const int r = row_c + i * S::kRowsC;
      const typename Codes<8>::type codes = {g.x[i].x, g.x[i].y};
      const float scale = r >= before && r < rows ? g.s[i] : 0.f;
      typedef typename Piece<T, 8>::type P8;
      P8* const at = reinterpret_cast<P8*>(to + kN * S::kPitchO + r * S::kPitchC + 8 * (int)sizeof(T) * piece_c);
      float f[8];
      if constexpr (F::kTerms == 1) {
        values_of<8>(codes, scale, f);
        *at = narrow<T, 8>(f);
      } else {
        // The value is taken as the first 8 bits of one a little smaller, and the rest, at most 2^-7 of it, rounded to bf16: off by 2^-15 of it.  The first
        // term then is never past bf16's numbers, and the second is zero only if the value is, and of its sign: the products with an infinity are one.
        const float below = scale * (1.f - 0x1p-21f);
        values_of<8>(codes, 1.f, f);
        uint32_t firsts[4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const uint32_t p = __float_as_uint(f[e] * below), q = __float_as_uint(f[e + 1] * below);
          firsts[e / 2] = __builtin_amdgcn_perm(q, p, 0x07060302u);
          f[e] = fmaf(f[e], scale, -__uint_as_float(p & 0xffff0000u));
          f[e + 1] = fmaf(f[e + 1], scale, -__uint_as_float(q & 0xffff0000u));
        }
        *at = __builtin_bit_cast(P8, firsts);
        at[S::kPlaneC / 16] = narrow<T, 8>(f);
      }
    }
#pragma unroll
    for (int i = k; i < PO; i += kSteps) {
      const int r = row_o + i * S::kRowsO;
      const P zero = {};
      g.dy[i] = r >= before && r < rows ? g.dy[i] : zero;
      if constexpr (kEnds == kShifted) g.dy[i] = shifted<P>(g.dy[i], shift);
      *reinterpret_cast<P*>(to + r * S::kPitchO + 16 * piece_o) = g.dy[i];
    }
    if (k == kSteps - 1 && sums) {
#pragma unroll
      for (int i = 0; i < PO; ++i) {
        float f[V];
        widen<T, V>(g.dy[i], f);
#pragma unroll
        for (int e = 0; e < V; ++e) db[e] += f[e];
      }
    }
  };

  f32x16 acc[TO][TC] = {};
  struct Frags { typename F::Frag p[F::kTerms][TC], q[TO]; } frags[2];
  const auto read = [&](Frags& f, int buffer, int step) {
    const char* dys = grad_lds + buffer * S::kBuffer + wo * TO * 32 * (int)sizeof(T) + step * F::kStep * S::kPitchO;
    const char* xs = grad_lds + buffer * S::kBuffer + kN * S::kPitchO + wc * TC * 32 * (int)sizeof(T) + step * F::kStep * S::kPitchC;
#pragma unroll
    for (int u = 0; u < F::kTerms; ++u)
#pragma unroll
      for (int t = 0; t < TC; ++t) f.p[u][t] = F::template load<true>(xs + u * S::kPlaneC + t * 32 * (int)sizeof(T), S::kPitchC);
#pragma unroll
    for (int t = 0; t < TO; ++t) f.q[t] = F::template load<false>(dys + t * 32 * (int)sizeof(T), S::kPitchO);
  };
  const auto multiply = [&](const Frags& f) {
#pragma unroll
    for (int u = F::kTerms - 1; u >= 0; --u)
#pragma unroll
      for (int i = 0; i < TO; ++i)
#pragma unroll
        for (int j = 0; j < TC; ++j) acc[i][j] = F::mma(f.p[u][j], f.q[i], acc[i][j]);
  };

  // The fragments of a product are read while the one before is under way, and so goes what was fetched to LDS; the first fragments of a
  // buffer are read behind the barrier that all wavefronts' parts of it are waited for at, during the last product of the buffer before.
  static_assert(kSteps % 2 == 0, "fragments change places");
#pragma unroll
  for (int k = 0; k < kAhead; ++k) fetch(stages[k], first + k * kN);
#pragma unroll
  for (int k = 0; k < kSteps; ++k) put(stages[0], first, 0, k);
  fetch(stages[0], first + kAhead * kN);
  lds_barrier();
  read(frags[0], 0, 0);
  int buffer = 0;
  for (int64_t n0 = first; n0 < last; n0 += kAhead * kN) {
#pragma unroll
    for (int d = 0; d < kAhead; ++d) {            // the rows from n0 + d kN on; those of the next kAhead steps are on their way
      Stage& g = stages[(d + 1) % kAhead];
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        if (k < kSteps - 1) read(frags[(k + 1) & 1], buffer, k + 1);
        put(g, n0 + (d + 1) * kN, buffer ^ 1, k);
        if (k < kSteps - 1) multiply(frags[k & 1]);
      }
      fetch(g, n0 + (d + 1 + kAhead) * kN);
      lds_barrier();
      buffer ^= 1;
      read(frags[0], buffer, 0);
      multiply(frags[1]);
    }
  }
  lds_barrier();

#pragma unroll
  for (int i = 0; i < TO; ++i)
#pragma unroll
    for (int j = 0; j < TC; ++j) {
      const int out = o0 + (wo * TO + i) * 32 + m, col = c0 + (wc * TC + j) * 32 + 16 * h;
      if (a.slices > 1) {                         // partial sums as the lanes hold them: whole lines, which the second kernel finds its way in
        if (out - m >= a.O || col - 16 * h >= a.C) continue;
        f32x4* to = reinterpret_cast<f32x4*>(a.partial) + (((int64_t)(slice * tiles + tile) * (kWO * kWC) + wave) * (TO * TC) + i * TC + j) * 256 + lane;
#pragma unroll
        for (int e = 0; e < 16; e += 4) to[16 * e] = f32x4{acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
      } else if (out < a.O) {
        T* to = static_cast<T*>(a.d_w) + out * a.ld_dw + col;
#pragma unroll
        for (int e = 0; e < 16; e += V) {
          float f[V];
#pragma unroll
          for (int k = 0; k < V; ++k) f[k] = acc[i][j][e + k];
          write_some<T, V>(to + e, f, a.C - col - e);
        }
      }
    }
  if (!sums) return;
  float* red = reinterpret_cast<float*>(grad_lds);
#pragma unroll
  for (int e = 0; e < V; ++e) red[row_o * kO + V * piece_o + e] = db[e];
  __syncthreads();
  for (int k = tid; k < kO; k += S::kAll) {
    double v = 0.;
    for (int r = 0; r < S::kRowsO; ++r) v += (double)red[r * kO + k];
    if (o0 + k < a.O) (a.slices > 1 ? a.bias_partial + (int64_t)slice * a.O : a.d_b)[o0 + k] = (float)v;
  }
}

// The slices' partial sums, added in 64 bits in an order of their numbers: a workgroup takes 32 outputs and columns, or 256 outputs of the bias; where there
// are few such workgroups, four quarters of it take every fourth slice each (kJoiners).  No slices: zeros.
template <typename T, int kJoiners> __global__ __launch_bounds__(256 * kJoiners) void k_linear8_grad_join(Grad8Args a, Shape t) {
  __shared__ f64x4 parts[kJoiners][256];
  const int tid = threadIdx.x & 255, part = threadIdx.x >> 8, tiles_c = (a.C + t.kC - 1) / t.kC, tiles = tiles_c * ((a.O + t.kO - 1) / t.kO);
  const int inner = t.kO * t.kC / 1024;           // squares of 32 of a tile
  const int tile = blockIdx.x / inner, square = blockIdx.x - tile * inner, wave = square / (t.TO * t.TC), of_wave = square - wave * (t.TO * t.TC);
  const int i = of_wave / t.TC, j = of_wave - i * t.TC, wo = wave % t.kWO, wc = wave / t.kWO;
  const int out0 = tile / tiles_c * t.kO + (wo * t.TO + i) * 32, col0 = (tile - tile / tiles_c * tiles_c) * t.kC + (wc * t.TC + j) * 32;
  const bool weights = tile < tiles;
  if (weights && (out0 >= a.O || col0 >= a.C)) return;             // (no workgroup wrote it)
  f64x4 v = {};
  if (weights) {
    const f32x4* from = reinterpret_cast<const f32x4*>(a.partial) + (int64_t)blockIdx.x * 256 + tid;
    const int64_t step = (int64_t)tiles * inner * 256;
    int k = part;
    for (; k + 7 * kJoiners < a.slices; k += 8 * kJoiners) {       // eight loads on their way at a time
      f32x4 f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = from[(k + j * kJoiners) * step];
#pragma unroll
      for (int j = 0; j < 8; ++j) v += __builtin_convertvector(f[j], f64x4);
    }
#pragma unroll 4
    for (; k < a.slices; k += kJoiners) v += __builtin_convertvector(from[k * step], f64x4);
  } else if (const int o = ((int)blockIdx.x - tiles * inner) * 256 + tid; o < a.O) {
#pragma unroll 4
    for (int k = part; k < a.slices; k += kJoiners) v[0] += (double)a.bias_partial[(int64_t)k * a.O + o];
  }
  if constexpr (kJoiners > 1) {
    parts[part][tid] = v;
    __syncthreads();
    if (part) return;
#pragma unroll
    for (int k = 1; k < kJoiners; ++k) v += parts[k][tid];
  }
  if (weights) {
    const int lane = tid & 63, out = out0 + (lane & 31), col = col0 + 16 * (lane >> 5) + 4 * (tid >> 6);
    const float f[4] = {(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
    if (out < a.O) write_some<T, 4>(static_cast<T*>(a.d_w) + out * a.ld_dw + col, f, a.C - col);
  } else if (const int o = ((int)blockIdx.x - tiles * inner) * 256 + tid; o < a.O) a.d_b[o] = (float)v[0];
}

// What tiles a call takes and how many slices.  A form's steps of 64 rows take `step` us with all its workgroups on the chip (`at_once`), its beginning
// `begin` more than that of the smallest tiles, and a slice costs the writing and reading of its partial sums, at 4.5 TB/s; the form and number of slices
// of the smallest sum are taken.  Measured, each form at its best, bf16, tiles of 64, 128, 192, 256 and 192 x 64, whose many rows at a time share a
// column's values among more outputs: 30,000 rows of 192 -> 576 33.2 us, 35.7, 32.1, 36.6, 28.0; 8,000 of 192 -> 192 12.9, 16.8, 20.0, 21.6, 14.5; 800,000 of
// 192 -> 576 604, 622, 431, 561, 497; 16,384 of 1,024 -> 1,024 116, 87, 103, 78, 121; 65,536 of 1,024 -> 2,048 872, 612, 771, 475, 845; fp32, tiles of 64 and 128:
// 30,000 of 192 -> 576 74, 105; 65,536 of 1,024 -> 2,048 2,551, 2,304.
constexpr int kRowsStep = 64;
// Rows that one slice adds up at most, of fp32 and bf16: each of its sums is a chain of additions in 32 bits, of which d_b has one for every 16 rows or more.
constexpr int kLongest[2] = {16384, 65536};
struct Form {
  Shape tile;
  int at_once;
  float step, begin;
};
constexpr int kWideForms = 5;                     // of bf16
constexpr Form kForms[2][kWideForms] = {
    {{{64, 64, 2, 1, 1}, 1024, 1.72f, 0.f}, {{128, 128, 2, 2, 2}, 512, 2.35f, 0.f}, {{192, 192, 3, 2, 3}, 256, 2.8f, 0.f}, {{256, 256, 2, 4, 2}, 256, 3.5f, 0.f},
     {{192, 64, 6, 1, 1}, 256, 1.06f, 4.f}},
    {{{64, 64, 2, 1, 1}, 768, 3.8f, 0.f}, {{128, 128, 2, 2, 2}, 512, 9.1f, 0.f}, {}, {}, {}}};

struct Plan {
  int form;                                       // of kForms
  int32_t slices, slice;
};
int64_t tile_values(const Shape& t, int32_t O, int32_t C) { return dsvt_ceil_div(O, t.kO) * dsvt_ceil_div(C, t.kC) * t.kO * t.kC; }
Plan make_plan(int32_t C, int32_t O, int32_t dtype, int32_t n) {
  Plan p = {0, 0, kRowsStep};
  if (n <= 0) return p;
  const bool narrow = dtype == DSVT_BF16;
  const int64_t steps = dsvt_ceil_div(n, kRowsStep), least = dsvt_ceil_div(n, kLongest[narrow]);
  double best = 0.;
  const int forms = O < (narrow ? 8 : 4) ? 1 : narrow ? kWideForms : 2;           // (fewer outputs than a piece: the first form)
  for (int f = 0; f < forms; ++f) {
    const Form& form = kForms[!narrow][f];
    const int64_t tiles = dsvt_ceil_div(O, form.tile.kO) * dsvt_ceil_div(C, form.tile.kC);
    const double slice_us = (double)tile_values(form.tile, O, C) * 8. / 4.5e6;
    int64_t most = form.at_once / tiles, slices = (int64_t)sqrt((double)steps * form.step / slice_us);
    most = most < steps / 4 ? most : steps / 4;    // (a slice of fewer steps is mostly its beginning and end)
    slices = slices < most ? slices : most;
    slices = slices > least ? slices : least;      // (one at least)
    const int64_t per = dsvt_ceil_div(steps, slices);
    slices = dsvt_ceil_div(steps, per);
    const double turns = tiles * slices > form.at_once ? (double)(tiles * slices) / form.at_once : 1.;
    const double us = (double)per * form.step * turns + (slices > 1 ? slices * slice_us + 4. : 0.) + form.begin;
    if (f > 0 && us >= best) continue;
    best = us;
    p = {f, (int32_t)slices, (int32_t)(per * kRowsStep)};
  }
  return p;
}

template <typename T, int kForm, int kN, int kAhead> int launch_tile(const Grad8Args& a, hipStream_t st) {
  constexpr Shape t = kForms[sizeof(T) == 4][kForm].tile;
  constexpr int kO = t.kO, kC = t.kC, kWO = t.kWO, kWC = t.kC / 32 / t.TC;
  typedef Tile<T, kO, kC, kWO, kWC, kN, kAhead> S;
  static_assert(S::TO == t.TO && S::TC == t.TC, "the second kernel goes by the form's tile");
  static std::atomic<uint64_t> allowed[3];
  const Ends ends = a.O % S::V == 0 ? kWhole : a.O > S::V ? kShifted : kSingly;
  auto kernel = ends == kWhole ? k_linear8_grad<T, kO, kC, kWO, kWC, kN, kAhead, kWhole> : k_linear8_grad<T, kO, kC, kWO, kWC, kN, kAhead, kShifted>;
  if constexpr (kForm == 0) {
    if (ends == kSingly) kernel = k_linear8_grad<T, kO, kC, kWO, kWC, kN, kAhead, kSingly>;
  }
  if (const int rc = dsvt_allow_lds(reinterpret_cast<const void*>(kernel), S::lds(), allowed[ends])) return rc;
  const int64_t all = dsvt_ceil_div(a.O, kO) * dsvt_ceil_div(a.C, kC) * a.slices;
  dsvt_prof_scope ps(DSVT_K_LINEAR8_GRAD, st);
  kernel<<<(unsigned)(dsvt_ceil_div(all, 8) * 8), S::kAll, S::lds(), st>>>(a);
  return DSVT_OK;
}
template <typename T> int launch(const Grad8Args& a, int form, hipStream_t st) {
  if (a.slices > 0) {
    int rc = DSVT_OK;
    if constexpr (sizeof(T) == 2) {
      rc = form == 4   ? launch_tile<T, 4, 96, 2>(a, st)
           : form == 3 ? launch_tile<T, 3, 32, 1>(a, st)
           : form == 2 ? launch_tile<T, 2, 32, 2>(a, st)
           : form == 1 ? launch_tile<T, 1, 32, 2>(a, st)
                       : launch_tile<T, 0, 32, 2>(a, st);
    } else {
      rc = form == 1 ? launch_tile<T, 1, 32, 1>(a, st) : launch_tile<T, 0, 32, 1>(a, st);
    }
    if (rc) return rc;
  }
  if (a.slices == 1) return DSVT_OK;
  const Shape& t = kForms[sizeof(T) == 4][form].tile;
  const int64_t blocks = tile_values(t, a.O, a.C) / 1024 + (a.d_b ? dsvt_ceil_div(a.O, 256) : 0);
  dsvt_prof_scope ps(DSVT_K_LINEAR8_JOIN, st);
  if (blocks < 4 * 256) k_linear8_grad_join<T, 4><<<(unsigned)blocks, 1024, 0, st>>>(a, t);
  else k_linear8_grad_join<T, 1><<<(unsigned)blocks, 256, 0, st>>>(a, t);
  return DSVT_OK;
}

int check(int32_t C, int32_t O, int32_t dtype, int32_t n_rows) {
  if (C <= 0 || O <= 0 || n_rows < 0 || (dtype != DSVT_F32 && dtype != DSVT_BF16)) return DSVT_EINVAL;
  return C > DSVT_LN_MAX_C || O > DSVT_LN_MAX_C ? DSVT_EUNSUPPORTED : DSVT_OK;
}

}  // namespace

extern "C" int dsvt_linear_rows8_weight_grad_workspace_size(int32_t C, int32_t out, int32_t dtype, int32_t n_rows, size_t* bytes) {
  if (!bytes) return DSVT_EINVAL;
  if (const int rc = check(C, out, dtype, n_rows)) return rc;
  const Plan p = make_plan(C, out, dtype, n_rows);
  *bytes = p.slices > 1 ? (size_t)p.slices * ((size_t)tile_values(kForms[dtype == DSVT_F32][p.form].tile, out, C) + (size_t)out) * sizeof(float) : 0;
  return DSVT_OK;
}

extern "C" int dsvt_linear_rows8_weight_grad(int32_t C, int32_t out, int32_t dtype, const dsvt_rows8* x, const void* dy, int64_t ld_dy,
                                             int32_t n_rows, void* d_w, int64_t ld_dw, float* d_b, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  if (const int rc = dsvt_linear_rows8_weight_grad_workspace_size(C, out, dtype, n_rows, &need)) return rc;
  const int e = dtype == DSVT_BF16 ? 2 : 4;
  if (bad_rows(d_w, ld_dw, C, e) || ((uintptr_t)d_b & 3u) != 0) return DSVT_EINVAL;
  if (n_rows > 0 && (bad_rows8(x, C) || bad_rows(dy, ld_dy, out, e))) return DSVT_EINVAL;
  if (n_rows > 0 && (x->ld >= (1 << 24) || ld_dy >= (1 << 24))) return DSVT_EUNSUPPORTED;        // (the rows of a step are less than 2^31 apart)
  if (need > 0 && (!ws || ((uintptr_t)ws & 15u))) return DSVT_EINVAL;
  if (ws_bytes < need) return DSVT_ENOSPC;
  const Plan p = make_plan(C, out, dtype, n_rows);
  Grad8Args a = {};
  a.dy = dy; a.ld_dy = ld_dy; a.n = n_rows; a.C = C; a.O = out; a.slices = p.slices; a.slice = p.slice;
  a.d_w = d_w; a.ld_dw = ld_dw; a.d_b = d_b;
  a.partial = static_cast<float*>(ws);
  a.bias_partial = a.partial + p.slices * tile_values(kForms[e == 4][p.form].tile, out, C);
  if (n_rows > 0) { a.x = x->codes; a.s = x->scale; a.ld_x = x->ld; }
  hipStream_t st = (hipStream_t)stream;
  if (const int rc = dtype == DSVT_BF16 ? launch<bf16_t>(a, p.form, st) : launch<float>(a, p.form, st)) return rc;
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}
