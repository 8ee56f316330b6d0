// dsvt_linear_rows8_weight_grad: the gradients of a linear layer's weights and bias from its input as it was kept in 8 bits (rows8.h).
//
//   d_w[o][c] = sum_n dy[n][o] s_n x[n][c],  d_b[o] = sum_n dy[n][o]
//
// The sums run over the rows: workgroups take a tile of outputs and columns and a slice of the rows each, and leave partial sums in 32 bits, which
// a second kernel adds up in the slices' order; one slice writes the results itself.  Rows go from memory through registers into one of two buffers in
// LDS, the kept ones as s_n x[n][c]; in bf16 that is rounded to bf16, as an operand of the product (products of 32-bit operands run at a sixteenth of
// the rate; the result, itself rounded, is off by 2.3e-3 of its norm instead of 1.7e-3).
#include "rows8.h"
#include <cstdlib>

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short short4_t __attribute__((ext_vector_type(4)));

struct Grad8Args {
  const int8_t* x;
  const float* s;
  const void* dy;
  void* d_w;                                      // written if there is one slice
  float *d_b, *partial, *bias_partial;            // d_b: null if not wanted; [slices][O][C], [slices][O]
  int64_t ld_x, ld_dy, ld_dw;
  int32_t n, C, O;
  int32_t slices, slice;                          // slices, rows of one (a multiple of a step's)
};

// Operand fragments out of LDS, where rows lie one after the other: 32 neighbouring columns, and the rows of one matrix instruction.
template <typename T> struct Columns;
template <> struct Columns<bf16_t> {
  static constexpr int kStep = 16, kPad = 64;     // rows of an instruction; bytes that pad a row in LDS: a fragment's four rows then lie in all banks
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
  static constexpr int kStep = 2, kPad = 128;
  typedef float Frag;
  static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
  template <bool kTurn> static __device__ __forceinline__ Frag load(const char* p, int pitch) {
    const int lane = threadIdx.x & 63, h = lane >> 5, m = lane & 31;
    const int column = kTurn ? 16 * (m >> 2 & 1) + 4 * (m >> 3) + (m & 3) : m;
    return *reinterpret_cast<const float*>(p + h * pitch + 4 * column);
  }
};

// kO outputs and kC columns, shared by kWO x kWC wavefronts; kN rows at a time.
template <typename T, int kO, int kC, int kWO, int kWC, int kN, int kAhead> struct Tile {
  static constexpr int kAll = 64 * kWO * kWC, TO = kO / kWO / 32, TC = kC / kWC / 32, V = 16 / (int)sizeof(T);
  static constexpr int kPitchO = kO * (int)sizeof(T) + Columns<T>::kPad, kPitchC = kC * (int)sizeof(T) + Columns<T>::kPad;
  static constexpr int kBuffer = kN * (kPitchO + kPitchC);
  static constexpr int kRowsO = kAll / (kO / V), kRowsC = kAll / (kC / 8);      // rows that all threads fetch at once, in pieces of 16 bytes of dy and 8 codes
  static constexpr int PO = kN / kRowsO, PC = kN / kRowsC;
  static_assert(kAll % (kO / V) == 0 && kAll % (kC / 8) == 0 && kN % kRowsO == 0 && kN % kRowsC == 0, "rows are fetched by all threads together");
  static constexpr size_t lds() { return 2 * (size_t)kBuffer > (size_t)kRowsO * kO * 4 ? 2 * (size_t)kBuffer : (size_t)kRowsO * kO * 4; }
};

extern __shared__ __attribute__((aligned(16))) char grad_lds[];

template <typename T, int kO, int kC, int kWO, int kWC, int kN, int kAhead> __global__ __launch_bounds__(64 * kWO * kWC) void k_linear8_grad(Grad8Args a) {
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
  const int o = V * piece_o < a.O - o0 ? V * piece_o : 0, c = 8 * piece_c < a.C - c0 ? 8 * piece_c : 0;
  const bool cut = a.O % V != 0 && o0 + kO > a.O;             // a piece of this tile's outputs does not end within them
  const int rows = (int)(last - first < kN ? last - first : kN);
  const int64_t last_step = last - rows;
  uint32_t off_o[PO], off_c[PC], off_s[PC];
#pragma unroll
  for (int i = 0; i < PO; ++i) {
    const int r = row_o + i * S::kRowsO;
    off_o[i] = (uint32_t)(r < rows ? r : rows - 1) * (uint32_t)a.ld_dy + o;
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
      const T* p = dy + off_o[i];
      if (cut) {
#pragma unroll
        for (int e = 0; e < V; ++e) g.dy[i][e] = p[o0 + o + e < a.O ? e : 0];
      } else __builtin_memcpy(&g.dy[i], p, 16);   // (on any element)
    }
  };
  float db[V] = {};
  const auto put = [&](const Stage& g, int64_t n0, int buffer) {
    char* to = grad_lds + buffer * S::kBuffer;
    const int before = n0 > last_step ? (int)(n0 - last_step < kN ? n0 - last_step : kN) : 0;     // rows of the step before
#pragma unroll
    for (int i = 0; i < PC; ++i) {
      typename Codes<8>::type codes;
      codes[0] = g.x[i].x;
      codes[1] = g.x[i].y;
      float f[8];
      widen_codes<8>(codes, f);
      const int r = row_c + i * S::kRowsC;
      const float s = r >= before && r < rows ? g.s[i] : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= s;
      typedef typename Piece<T, 8>::type P8;
      *reinterpret_cast<P8*>(to + kN * S::kPitchO + r * S::kPitchC + 8 * (int)sizeof(T) * piece_c) = narrow<T, 8>(f);
    }
#pragma unroll
    for (int i = 0; i < PO; ++i) {
      const int r = row_o + i * S::kRowsO;
      const P zero = {}, p = r >= before && r < rows ? g.dy[i] : zero;
      *reinterpret_cast<P*>(to + r * S::kPitchO + 16 * piece_o) = p;
      if (sums) {
        float f[V];
        widen<T, V>(p, f);
#pragma unroll
        for (int e = 0; e < V; ++e) db[e] += f[e];
      }
    }
  };

  f32x16 acc[TO][TC] = {};
  const auto multiply = [&](int buffer, int step) {
    const char* from = grad_lds + buffer * S::kBuffer + wo * TO * 32 * (int)sizeof(T) + step * F::kStep * S::kPitchO;
    const char* xs = grad_lds + buffer * S::kBuffer + kN * S::kPitchO + wc * TC * 32 * (int)sizeof(T) + step * F::kStep * S::kPitchC;
    typename F::Frag p[TC], q[TO];
#pragma unroll
    for (int t = 0; t < TC; ++t) p[t] = F::template load<true>(xs + t * 32 * (int)sizeof(T), S::kPitchC);
#pragma unroll
    for (int t = 0; t < TO; ++t) q[t] = F::template load<false>(from + t * 32 * (int)sizeof(T), S::kPitchO);
#pragma unroll
    for (int i = 0; i < TO; ++i)
#pragma unroll
      for (int j = 0; j < TC; ++j) acc[i][j] = F::mma(p[j], q[i], acc[i][j]);
  };

  constexpr int kSteps = kN / F::kStep;
#pragma unroll
  for (int k = 0; k < kAhead; ++k) fetch(stages[k], first + k * kN);
  put(stages[0], first, 0);
  fetch(stages[0], first + kAhead * kN);
  lds_barrier();
  int buffer = 0;
  for (int64_t n0 = first; n0 < last; n0 += kAhead * kN) {
#pragma unroll
    for (int d = 0; d < kAhead; ++d) {            // the rows from n0 + d kN on; those of the next kAhead steps are on their way
#pragma unroll
      for (int k = 0; k < kSteps / 2; ++k) multiply(buffer, k);
      put(stages[(d + 1) % kAhead], n0 + (d + 1) * kN, buffer ^ 1);
      fetch(stages[(d + 1) % kAhead], n0 + (d + 1 + kAhead) * kN);
#pragma unroll
      for (int k = kSteps / 2; k < kSteps; ++k) multiply(buffer, k);
      lds_barrier();
      buffer ^= 1;
    }
  }

#pragma unroll
  for (int i = 0; i < TO; ++i) {
    const int out = o0 + (wo * TO + i) * 32 + m;
    if (out >= a.O) continue;
#pragma unroll
    for (int j = 0; j < TC; ++j) {
      const int col = c0 + (wc * TC + j) * 32 + 16 * h;
      if (col >= a.C) continue;
      if (a.slices > 1) {
        float* to = a.partial + ((int64_t)slice * a.O + out) * a.C + col;
        if (a.C % 4 == 0 && col + 16 <= a.C) {
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            reinterpret_cast<f32x4*>(to)[e / 4] = f32x4{acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) if (col + e < a.C) to[e] = acc[i][j][e];
        }
      } else {
        T* to = static_cast<T*>(a.d_w) + out * a.ld_dw + col;
#pragma unroll
        for (int e = 0; e < 16; ++e) if (col + e < a.C) to[e] = (T)acc[i][j][e];
      }
    }
  }
  if (!sums) return;
  float* red = reinterpret_cast<float*>(grad_lds);            // (the last barrier is behind all reads)
#pragma unroll
  for (int e = 0; e < V; ++e) red[row_o * kO + V * piece_o + e] = db[e];
  __syncthreads();
  for (int k = tid; k < kO; k += S::kAll) {
    float v = 0.f;
    for (int r = 0; r < S::kRowsO; ++r) v += red[r * kO + k];
    if (o0 + k < a.O) (a.slices > 1 ? a.bias_partial + (int64_t)slice * a.O : a.d_b)[o0 + k] = v;
  }
}

// The slices' sums added in their order, in 32 bits (there are few of them), those of the bias behind those of the weights.  No slices: zeros.
template <typename T> __global__ __launch_bounds__(256) void k_linear8_grad_join(Grad8Args a) {
  const int64_t all = (int64_t)a.O * a.C, end = all + (a.d_b ? a.O : 0);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < end; i += (int64_t)gridDim.x * 256) {
    const float* from = i < all ? a.partial + i : a.bias_partial + (i - all);
    const int64_t step = i < all ? all : a.O;
    float v = 0.f;
    int k = 0;
    for (; k + 8 <= a.slices; k += 8) {           // eight loads on their way at a time
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = from[(k + j) * step];
#pragma unroll
      for (int j = 0; j < 8; ++j) v += f[j];
    }
    for (; k < a.slices; ++k) v += from[k * step];
    if (i < all) static_cast<T*>(a.d_w)[i / a.C * a.ld_dw + i % a.C] = (T)v;
    else a.d_b[i - all] = v;
  }
}

constexpr int kRowsStep = 64;                     // of every form's rows at a time a multiple

struct Plan {
  int form;                                       // 0: tiles of 64, 1: of 128, 2: of 256
  int32_t slices, slice;
};
Plan make_plan(int32_t C, int32_t O, int32_t dtype, int32_t n) {
  const auto tiles = [&](int t) { return dsvt_ceil_div(O, t) * dsvt_ceil_div(C, t); };
  const int64_t steps = dsvt_ceil_div(n, kRowsStep);
  Plan p = {0, 0, kRowsStep};
  if (n <= 0) return p;
  int64_t slices;
  if (dtype == DSVT_BF16 && tiles(256) * steps >= 256 * 16 && tiles(256) >= 8) {
    p.form = 2;
    slices = dsvt_ceil_div(256, tiles(256));
  } else if (tiles(128) >= 8 && tiles(128) * steps >= 512 * 8) {
    p.form = 1;
    slices = dsvt_ceil_div(512, tiles(128));
  } else {
    slices = dsvt_ceil_div(512, tiles(64));
  }
  if (getenv("G8_FORM")) { p.form = atoi(getenv("G8_FORM")); const int fo[] = {64, 128, 256, 192, 192, 192, 64, 64, 96}, fc[] = {64, 128, 256, 192, 64, 96, 192, 64, 192}; slices = atoi(getenv("G8_WGS")) / (dsvt_ceil_div(O, fo[p.form]) * dsvt_ceil_div(C, fc[p.form])); if (slices < 1) slices = 1; }
  const int64_t most = dsvt_ceil_div(steps, 4);
  slices = slices < most ? slices : most;
  const int64_t per = dsvt_ceil_div(steps, slices);
  p.slice = (int32_t)(per * kRowsStep);
  p.slices = (int32_t)dsvt_ceil_div(steps, per);
  return p;
}

template <typename T, int kO, int kC, int kWO, int kWC, int kN, int kAhead> int launch_tile(const Grad8Args& a, hipStream_t st) {
  typedef Tile<T, kO, kC, kWO, kWC, kN, kAhead> S;
  static std::atomic<uint64_t> allowed;
  const auto kernel = k_linear8_grad<T, kO, kC, kWO, kWC, kN, kAhead>;
  if (const int rc = dsvt_allow_lds(reinterpret_cast<const void*>(kernel), S::lds(), allowed)) return rc;
  const int64_t all = dsvt_ceil_div(a.O, kO) * dsvt_ceil_div(a.C, kC) * a.slices;
  dsvt_prof_scope ps(DSVT_K_LINEAR8_GRAD, st);
  kernel<<<(unsigned)(dsvt_ceil_div(all, 8) * 8), S::kAll, S::lds(), st>>>(a);
  return DSVT_OK;
}
template <typename T> int launch(const Grad8Args& a, int form, hipStream_t st) {
  if (a.slices > 0) {
    int rc;
    if constexpr (sizeof(T) == 2) {
      const int dd = getenv("G8_D") ? atoi(getenv("G8_D")) : 1;
      if (form == 2) rc = dd == 1 ? launch_tile<T, 256, 256, 2, 4, 64, 1>(a, st) : dd == 4 ? launch_tile<T, 256, 256, 2, 4, 32, 2>(a, st) : dd == 3 ? launch_tile<T, 256, 256, 2, 4, 32, 3>(a, st) : launch_tile<T, 256, 256, 2, 4, 32, 1>(a, st);
      else if (form == 0) rc = dd == 1 ? launch_tile<T, 64, 64, 2, 2, 64, 1>(a, st) : dd == 2 ? launch_tile<T, 64, 64, 2, 2, 64, 2>(a, st) : dd == 3 ? launch_tile<T, 64, 64, 2, 2, 64, 3>(a, st) : launch_tile<T, 64, 64, 2, 2, 64, 4>(a, st);
      else if (form == 3) rc = dd == 1 ? launch_tile<T, 192, 192, 3, 2, 32, 1>(a, st) : dd == 2 ? launch_tile<T, 192, 192, 3, 2, 32, 2>(a, st) : launch_tile<T, 192, 192, 3, 2, 32, 3>(a, st);
      else if (form == 4) rc = dd == 1 ? launch_tile<T, 192, 64, 3, 2, 48, 1>(a, st) : dd == 2 ? launch_tile<T, 192, 64, 3, 2, 48, 2>(a, st) : launch_tile<T, 192, 64, 3, 2, 48, 3>(a, st);
      else rc = dd == 1 ? launch_tile<T, 128, 128, 2, 2, 64, 1>(a, st) : dd == 2 ? launch_tile<T, 128, 128, 2, 2, 64, 2>(a, st) : launch_tile<T, 128, 128, 2, 2, 32, 3>(a, st);
    } else {
      rc = form == 1 ? launch_tile<T, 128, 128, 2, 2, 32, 1>(a, st) : launch_tile<T, 64, 64, 2, 2, 32, 1>(a, st);
    }
    if (rc) return rc;
  }
  if (a.slices == 1) return DSVT_OK;
  const int64_t blocks = dsvt_ceil_div((int64_t)a.O * a.C + a.O, 256);
  dsvt_prof_scope ps(DSVT_K_LINEAR8_JOIN, st);
  k_linear8_grad_join<T><<<(unsigned)(blocks < 8192 ? blocks : 8192), 256, 0, st>>>(a);
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
  *bytes = p.slices > 1 ? (size_t)p.slices * (size_t)out * ((size_t)C + 1) * sizeof(float) : 0;
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
  const Plan p = make_plan(C, out, dtype, n_rows);
  Grad8Args a = {};
  a.dy = dy; a.ld_dy = ld_dy; a.n = n_rows; a.C = C; a.O = out; a.slices = p.slices; a.slice = p.slice;
  a.d_w = d_w; a.ld_dw = ld_dw; a.d_b = d_b;
  a.partial = static_cast<float*>(ws);
  a.bias_partial = a.partial + (int64_t)p.slices * out * C;
  if (n_rows > 0) { a.x = x->codes; a.s = x->scale; a.ld_x = x->ld; }
  hipStream_t st = (hipStream_t)stream;
  if (const int rc = dtype == DSVT_BF16 ? launch<bf16_t>(a, p.form, st) : launch<float>(a, p.form, st)) return rc;
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}
