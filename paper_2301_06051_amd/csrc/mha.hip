// dsvt_set_mha / dsvt_set_mha_backward: multi-head attention inside every set (Eq. 5, second line) on rows that are already
// projected, with a learned relative position bias per offset or per bucket of offsets, and its gradients.  With g = d out,
// sigma = 1/sqrt(d), m_j the weight of voxel j as a key (1, or the number of its slots), B the bucket of an offset:
//
//   s_ij = sigma q_i.k_j + bias[B(c_i - c_j)]    P_ij = m_j exp(s_ij) / sum_j m_j exp(s_ij)    out_i = sum_j P_ij v_j
//   t_ij = g_i.v_j    ds_ij = P_ij (t_ij - sum_j P_ij t_ij)
//   dq_i = sigma sum_j ds_ij k_j    dk_j = sigma sum_i ds_ij q_i    dv_j = sum_i P_ij g_i    d bias[u] = sum of ds_ij with B = u
//
// A set is at most 96 voxels and every voxel is in one set, so a set's attention is a problem of its own that fits on chip: the
// backward pass forms the probabilities again and needs nothing from the forward pass, and no two sets write one row.
//
// A wavefront takes one (set, head) at a time; the wavefronts of a workgroup take the heads of one set side by side, so
// that the cache lines its heads share are fetched once.  Rows go from memory straight into matrix fragments: with the keys as
// rows and the queries as columns of the logits, lane 16 g + m holds query m and keys 4 g .. 4 g + 3 of a tile, which is how
// the next product wants its operand.  Operands that have to be turned round (V, and in the backward pass K, Q, g, P, ds) are
// multiplied by the unit matrix, which is exact (one factor is 1, the others are 0; a row with an infinity or a NaN
// becomes NaN in all of its channels).  LDS holds no tile, only the position codes and tables.
#include "common.h"
#include "mma.h"
#include <cfloat>
#include <cmath>

namespace {

constexpr int kSetMax = 96;                       // slots, and so voxels, of a set
constexpr int kTiles = kSetMax / 16;
constexpr int kWavesMax = 8;                      // wavefronts of a workgroup: heads taken side by side
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kGroups = 512;                      // workgroups that a launch aims at: two a compute unit
constexpr int kSetsPerPart = 256;                 // of a backward workgroup, at most: more would cost its 32-bit sums digits
constexpr size_t kTableLds = 64 << 10;            // a bias table of this size is kept in LDS
constexpr size_t kBinsLds = 140 << 10;            // the sums of a workgroup's heads in the backward pass, at most

struct MhaArgs {
  const int32_t *set_inds, *n_sets;
  const int4* coords;
  const void *qkv, *d_out;
  void* out;                                      // forward: the output rows; backward: d_qkv
  const float* bias;                              // [heads][n_rel] or null
  const int32_t* bucket;                          // [n_off] or null
  float* partial;                                 // backward: [parts][heads][n_off]; null: no gradient of the table
  int64_t ld_qkv, ld_dout, ld_out;
  int32_t n_voxels, max_sets, tau, heads, hd, n_off, n_rel, centre;
  int32_t w2, h2;                                 // 2W - 1, 2H - 1
  int32_t dup, hs, groups, parts;                 // heads of a workgroup, groups of heads, workgroups a group
  int32_t table_lds;
  float scale;
};

typedef short short4_t __attribute__((ext_vector_type(4)));

// Matrix fragments.  A row fragment covers 4 * KL channels: lane 16 g + m holds channels KL g .. KL g + KL - 1 of row m.  A
// tile fragment covers 16: lane 16 g + m holds elements 4 g .. 4 g + 3 of row (or column) m.
template <typename T, int HDP> struct Frag;
template <int HDP> struct Frag<bf16_t, HDP> {
  static constexpr int KL = HDP == 16 ? 4 : 8, NC = HDP / (4 * KL), NT = HDP / 16, PER = KL / 4;
  typedef bf16_t Row __attribute__((ext_vector_type(KL)));
  typedef bf16x4 Tile;
  static __device__ __forceinline__ f32x4 tile_mma(Tile a, Tile b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(short4_t, a), __builtin_bit_cast(short4_t, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 row_mma(Row a, Row b, f32x4 c) {
    if constexpr (KL == 8) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else return tile_mma(a, b, c);
  }
  static __device__ __forceinline__ Tile tile(f32x4 v) { return Tile{(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]}; }
};
template <int HDP> struct Frag<float, HDP> {
  static constexpr int KL = 4, NC = HDP / 16, NT = HDP / 16, PER = 1;
  typedef f32x4 Row;
  typedef f32x4 Tile;
  static __device__ __forceinline__ f32x4 tile_mma(Tile a, Tile b, f32x4 c) { return Mma<float>::mma(a, b, c); }
  static __device__ __forceinline__ f32x4 row_mma(Row a, Row b, f32x4 c) { return Mma<float>::mma(a, b, c); }
  static __device__ __forceinline__ Tile tile(f32x4 v) { return v; }
};

// Lanes 16 apart hold the same query's other keys.
__device__ __forceinline__ float across_sum(float v) { v += __shfl_xor(v, 16, 64); return v + __shfl_xor(v, 32, 64); }
__device__ __forceinline__ float across_max(float v) { v = fmaxf(v, __shfl_xor(v, 16, 64)); return fmaxf(v, __shfl_xor(v, 32, 64)); }

// A finite bias stays finite in units of log2 e.
__device__ __forceinline__ float to_log2(float b) {
  const float f = b * kLog2e;
  return fabsf(b) <= FLT_MAX ? fminf(fmaxf(f, -3.0e38f), 3.0e38f) : f;
}

// What a wavefront knows of its set, in LDS: row r's voxel (-1 past the last), position code and weight as a key (0 past the last).
struct SetRows {
  int32_t vox[kSetMax], code[kSetMax], weight[kSetMax];
};

// The set's distinct voxels in slot order: the first slot of every run of equal ones.  Slots outside 0 .. n_voxels - 1 hold none.
__device__ __forceinline__ int load_set(const MhaArgs& a, int32_t s, SetRows& rows) {
  const int lane = threadIdx.x & 63;
  const int32_t* inds = a.set_inds + (int64_t)s * a.tau;
  int32_t v[2];
  uint64_t first[2], change[2];
  int32_t before = -1;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int slot = 64 * k + lane;
    v[k] = slot < a.tau ? inds[slot] : -1;
    if ((uint32_t)v[k] >= (uint32_t)a.n_voxels) v[k] = -1;
    int32_t prev = __shfl_up(v[k], 1, 64);
    if (lane == 0) prev = before;
    before = __shfl(v[k], 63, 64);
    change[k] = __ballot(v[k] != prev || slot >= a.tau);
    first[k] = __ballot(v[k] != prev && v[k] >= 0);
  }
  const int n0 = __popcll(first[0]), n = n0 + __popcll(first[1]);
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (first[k] >> lane & 1) {
      const int r = (k ? n0 : 0) + __popcll(first[k] & ((1ull << lane) - 1));
      const uint64_t later = lane == 63 ? 0 : change[k] >> (lane + 1);      // slots to the next change
      int run;
      if (later) run = 1 + __builtin_ctzll(later);
      else if (k == 0) run = 64 - lane + (change[1] ? __builtin_ctzll(change[1]) : 64);
      else run = 64 - lane;
      const int4 c = a.coords[v[k]];
      rows.vox[r] = v[k];
      rows.code[r] = (c.y * a.w2 + c.z) * a.h2 + c.w;
      rows.weight[r] = a.dup ? run : 1;
    }
  const int pad = (n + 15) & ~15;
  if (n + lane < pad) {
    rows.vox[n + lane] = -1;
    rows.code[n + lane] = 0;
    rows.weight[n + lane] = 0;
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  return n;
}

template <typename T, int HDP> struct Head {
  typedef Frag<T, HDP> F;
  typedef typename F::Row Row;
  typedef typename F::Tile Tile;
  const MhaArgs& a;
  const SetRows& rows;
  const float* table;                             // LDS: this head's n_off + 1 biases in units of log2 e; null: read from memory
  const float* bias;                              // memory: this head's n_rel biases
  int lane, m, g, h;
  float scale2;                                   // sigma log2 e

  __device__ __forceinline__ Head(const MhaArgs& a_, const SetRows& rows_, const float* table_, int h_)
      : a(a_), rows(rows_), table(table_), bias(a_.bias ? a_.bias + (int64_t)h_ * a_.n_rel : nullptr), lane(threadIdx.x & 63), m(lane & 15), g(lane >> 4),
        h(h_), scale2(a_.scale * kLog2e) {}

  // rows of tile t of an array of head vectors (which: 0 q, 1 k, 2 v of a qkv row; 0 of an output row)
  __device__ __forceinline__ void load(const void* base, int64_t ld, int which, int t, Row (&f)[F::NC]) const {
    const int32_t v = rows.vox[16 * t + m];
    const T* p = static_cast<const T*>(base) + (v < 0 ? 0 : v) * ld + (int64_t)which * a.heads * a.hd + h * a.hd;
#pragma unroll
    for (int c = 0; c < F::NC; ++c) {
      const int d = (4 * c + g) * F::KL;
      Row zero = {};
      f[c] = v >= 0 && d < a.hd ? *reinterpret_cast<const Row*>(p + d) : zero;
    }
  }
  // the other way round: element 4 g' + i of column m of the result lies with row 4 g + i of a 16-column tile
  __device__ __forceinline__ void store(void* base, int64_t ld, int which, int t, const f32x4 (&o)[F::NT], float scale) const {
    const int32_t v = rows.vox[16 * t + m];
    if (v < 0) return;
    T* p = static_cast<T*>(base) + v * ld + (int64_t)which * a.heads * a.hd + h * a.hd;
#pragma unroll
    for (int c = 0; c < F::NC; ++c) {
      const int d = (4 * c + g) * F::KL;
      if (d >= a.hd) continue;
      Row r;
#pragma unroll
      for (int e = 0; e < F::KL; ++e) r[e] = (T)(o[c * F::PER + e / 4][e % 4] * scale);
      *reinterpret_cast<Row*>(p + d) = r;
    }
  }
  // The unit matrix that picks channels of part `half` of a row fragment: column m is channel 8 (m / 4) + 4 half + m % 4 (KL = 8) or m.
  __device__ __forceinline__ Row unit(int half) const {
    Row u;
    const int d = F::KL == 8 ? 8 * (m >> 2) + 4 * half + (m & 3) : m;
#pragma unroll
    for (int e = 0; e < F::KL; ++e) u[e] = (T)(F::KL * g + e == d ? 1.f : 0.f);
    return u;
  }
  __device__ __forceinline__ Tile tile_unit() const {
    Tile u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = (T)(4 * g + e == m ? 1.f : 0.f);
    return u;
  }
  // rows -> NT tile fragments: lane holds channel (of tile n) m, rows 4 g .. 4 g + 3
  __device__ __forceinline__ void turn(const Row (&f)[F::NC], Tile (&o)[F::NT]) const {
#pragma unroll
    for (int n = 0; n < F::NT; ++n) o[n] = F::tile(F::row_mma(f[n / F::PER], unit(n % F::PER), f32x4{0.f, 0.f, 0.f, 0.f}));
  }
  __device__ __forceinline__ Tile turn(Tile f) const { return F::tile(F::tile_mma(f, tile_unit(), f32x4{0.f, 0.f, 0.f, 0.f})); }

  // logits of key tile kt and query tile qt in units of log2 e, -inf where there is no key
  __device__ __forceinline__ f32x4 logits(const Row (&k)[F::NC], const Row (&q)[F::NC], int kt, int qt) const {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < F::NC; ++c) s = F::row_mma(k[c], q[c], s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float b = 0.f;
      if (a.bias) {
        const unsigned at = offset(kt, qt, i);
        if (table) b = table[at];
        else if (at < (unsigned)a.n_off) {
          const unsigned u = a.bucket ? (unsigned)a.bucket[at] : at;
          b = u < (unsigned)a.n_rel ? to_log2(bias[u]) : 0.f;
        }
      }
      s[i] = rows.weight[16 * kt + 4 * g + i] ? fmaf(s[i], scale2, b) : -INFINITY;
    }
    return s;
  }
  // number of the offset query m - key 4 g + i; n_off: none (the coordinates are further apart than a window)
  __device__ __forceinline__ unsigned offset(int kt, int qt, int i) const {
    const unsigned at = (unsigned)(rows.code[16 * qt + m] - rows.code[16 * kt + 4 * g + i] + a.centre);
    return at < (unsigned)a.n_off ? at : (unsigned)a.n_off;
  }
  __device__ __forceinline__ f32x4 weighted_exp(f32x4 s, float top, int kt) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] - top) * (float)rows.weight[16 * kt + 4 * g + i];
    return s;
  }
};

// Workgroup b takes group of heads b / 8 % groups and is part (b / 8 / groups) * 8 + b % 8 of it: workgroups that take other heads of
// the same sets are a multiple of 8 apart and so on one XCD, whose L2 they share.
struct Share {
  int group, part;
  __device__ __forceinline__ Share(const MhaArgs& a) {
    const int r = blockIdx.x >> 3;
    group = r % a.groups;
    part = r / a.groups * 8 + (blockIdx.x & 7);
  }
};

// The heads' biases by offset; one more entry, 0, for pairs that are further apart than a window.
__device__ __forceinline__ void fill_table(const MhaArgs& a, int h0, float* table) {
  for (int h = 0; h < a.hs; ++h)
    for (int u = threadIdx.x; u <= a.n_off; u += blockDim.x) {
      const unsigned r = u == a.n_off ? ~0u : a.bucket ? (unsigned)a.bucket[u] : (unsigned)u;
      table[h * (a.n_off + 1) + u] = r < (unsigned)a.n_rel ? to_log2(a.bias[(int64_t)(h0 + h) * a.n_rel + r]) : 0.f;
    }
}

__device__ __forceinline__ int32_t sets_of(const MhaArgs& a) {
  const int32_t n = *a.n_sets;
  return n < 0 ? 0 : (n > a.max_sets ? a.max_sets : n);
}

extern __shared__ float lds[];

template <typename T, int HDP>
__global__ __launch_bounds__(64 * kWavesMax) void k_mha_forward(MhaArgs a) {
  typedef Frag<T, HDP> F;
  __shared__ SetRows set_rows[kWavesMax];
  const Share share(a);
  const int wave = threadIdx.x >> 6, h = share.group * a.hs + wave;
  if (a.table_lds) {
    fill_table(a, share.group * a.hs, lds);
    __syncthreads();
  }
  SetRows& rows = set_rows[wave];
  Head<T, HDP> head(a, rows, a.table_lds ? lds + wave * (a.n_off + 1) : nullptr, h);
  const int32_t n_sets = sets_of(a);
  for (int32_t s = share.part; s < n_sets; s += a.parts) {
    const int n = load_set(a, s, rows), nt = (n + 15) >> 4;
    for (int qt = 0; qt < nt; ++qt) {
      typename F::Row q[F::NC];
      head.load(a.qkv, a.ld_qkv, 0, qt, q);
      f32x4 p[kTiles];
      float top = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < kTiles; ++kt)
        if (kt < nt) {
          typename F::Row k[F::NC];
          head.load(a.qkv, a.ld_qkv, 1, kt, k);
          p[kt] = head.logits(k, q, kt, qt);
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, p[kt][i]);
        }
      top = across_max(top);
      if (top == -INFINITY) top = 0.f;            // every key is masked: no probabilities, an output of zeros
      float sum = 0.f;
      f32x4 o[F::NT] = {};
#pragma unroll
      for (int kt = 0; kt < kTiles; ++kt)
        if (kt < nt) {
          p[kt] = head.weighted_exp(p[kt], top, kt);
#pragma unroll
          for (int i = 0; i < 4; ++i) sum += p[kt][i];
          typename F::Row v[F::NC];
          typename F::Tile vt[F::NT];
          head.load(a.qkv, a.ld_qkv, 2, kt, v);
          head.turn(v, vt);
#pragma unroll
          for (int t = 0; t < F::NT; ++t) o[t] = F::tile_mma(vt[t], F::tile(p[kt]), o[t]);
        }
      sum = across_sum(sum);
      head.store(a.out, a.ld_out, 0, qt, o, sum == 0.f ? 0.f : 1.f / sum);
    }
  }
}

template <typename T, int HDP>
__global__ __launch_bounds__(64 * kWavesMax) void k_mha_backward(MhaArgs a) {
  typedef Frag<T, HDP> F;
  typedef typename F::Row Row;
  typedef typename F::Tile Tile;
  __shared__ SetRows set_rows[kWavesMax];
  __shared__ float stats[kWavesMax][3][kSetMax];  // per query: the largest logit, 1 / sum, sum of P t
  const Share share(a);
  const int wave = threadIdx.x >> 6, h0 = share.group * a.hs, h = h0 + wave;
  float* bins = lds;                              // [hs][n_off], if the table's gradient is wanted
  float* table = a.partial ? lds + a.hs * a.n_off : lds;
  if (a.table_lds) fill_table(a, h0, table);
  if (a.partial)
    for (int u = threadIdx.x; u < a.hs * a.n_off; u += blockDim.x) bins[u] = 0.f;
  __syncthreads();
  bins += wave * a.n_off;
  SetRows& rows = set_rows[wave];
  float(&st)[3][kSetMax] = stats[wave];
  Head<T, HDP> head(a, rows, a.table_lds ? table + wave * (a.n_off + 1) : nullptr, h);
  const int m = head.m, g = head.g;
  const int32_t n_sets = sets_of(a);
  for (int32_t s = share.part; s < n_sets; s += a.parts) {
    const int n = load_set(a, s, rows), nt = (n + 15) >> 4;
    // by queries: statistics, dq, the table's gradient
    for (int qt = 0; qt < nt; ++qt) {
      Row q[F::NC], go[F::NC];
      head.load(a.qkv, a.ld_qkv, 0, qt, q);
      head.load(a.d_out, a.ld_dout, 0, qt, go);
      f32x4 p[kTiles], t[kTiles];
      float top = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < kTiles; ++kt)
        if (kt < nt) {
          Row k[F::NC], v[F::NC];
          head.load(a.qkv, a.ld_qkv, 1, kt, k);
          head.load(a.qkv, a.ld_qkv, 2, kt, v);
          p[kt] = head.logits(k, q, kt, qt);
          t[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < F::NC; ++c) t[kt] = F::row_mma(v[c], go[c], t[kt]);
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, p[kt][i]);
        }
      top = across_max(top);
      if (top == -INFINITY) top = 0.f;
      float sum = 0.f, dot = 0.f;
#pragma unroll
      for (int kt = 0; kt < kTiles; ++kt)
        if (kt < nt) {
          p[kt] = head.weighted_exp(p[kt], top, kt);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sum += p[kt][i];
            dot = fmaf(p[kt][i], t[kt][i], dot);
          }
        }
      sum = across_sum(sum);
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      dot = across_sum(dot) * inv;
      if (g == 0) {
        st[0][16 * qt + m] = top;
        st[1][16 * qt + m] = inv;
        st[2][16 * qt + m] = dot;
      }
      f32x4 dq[F::NT] = {};
      const bool query = 16 * qt + m < n;
#pragma unroll
      for (int kt = 0; kt < kTiles; ++kt)
        if (kt < nt) {
          f32x4 ds;
#pragma unroll
          for (int i = 0; i < 4; ++i) ds[i] = p[kt][i] * inv * (t[kt][i] - dot);
          if (a.partial && query) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const unsigned at = head.offset(kt, qt, i);
              if (rows.weight[16 * kt + 4 * g + i] && at < (unsigned)a.n_off) unsafeAtomicAdd(&bins[at], ds[i]);
            }
          }
          Row k[F::NC];
          Tile ktt[F::NT];
          head.load(a.qkv, a.ld_qkv, 1, kt, k);
          head.turn(k, ktt);
#pragma unroll
          for (int c = 0; c < F::NT; ++c) dq[c] = F::tile_mma(ktt[c], F::tile(ds), dq[c]);
        }
      head.store(a.out, a.ld_out, 0, qt, dq, a.scale);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    // by keys: dk, dv
    for (int kt = 0; kt < nt; ++kt) {
      Row k[F::NC], v[F::NC];
      head.load(a.qkv, a.ld_qkv, 1, kt, k);
      head.load(a.qkv, a.ld_qkv, 2, kt, v);
      f32x4 dk[F::NT] = {}, dv[F::NT] = {};
      for (int qt = 0; qt < nt; ++qt) {
        Row q[F::NC], go[F::NC];
        head.load(a.qkv, a.ld_qkv, 0, qt, q);
        head.load(a.d_out, a.ld_dout, 0, qt, go);
        f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < F::NC; ++c) t = F::row_mma(v[c], go[c], t);
        f32x4 p = head.weighted_exp(head.logits(k, q, kt, qt), st[0][16 * qt + m], kt), ds;
        const float inv = st[1][16 * qt + m], dot = st[2][16 * qt + m];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] *= inv;
          ds[i] = p[i] * (t[i] - dot);
        }
        const Tile pt = head.turn(F::tile(p)), dst = head.turn(F::tile(ds));
        Tile qtt[F::NT], gt[F::NT];
        head.turn(q, qtt);
        head.turn(go, gt);
#pragma unroll
        for (int c = 0; c < F::NT; ++c) {
          dk[c] = F::tile_mma(qtt[c], dst, dk[c]);
          dv[c] = F::tile_mma(gt[c], pt, dv[c]);
        }
      }
      head.store(a.out, a.ld_out, 1, kt, dk, a.scale);
      head.store(a.out, a.ld_out, 2, kt, dv, 1.f);
    }
  }
  if (!a.partial) return;
  __syncthreads();
  if (share.part < n_sets)                        // k_mha_offsets reads the parts that had a set
    for (int u = threadIdx.x; u < a.hs * a.n_off; u += blockDim.x)
      a.partial[((int64_t)share.part * a.heads + h0) * a.n_off + u] = lds[u];
}

// The table's gradient by offset: the parts' sums added in their order, 64 columns of [heads * n_off] a workgroup, 16 slices of the parts.
__global__ __launch_bounds__(1024) void k_mha_offsets(const float* __restrict__ partial, const int32_t* __restrict__ n_sets, int32_t parts,
                                                      int64_t cols, float* __restrict__ out) {
  __shared__ double s[16][64];
  const int32_t n = *n_sets < parts ? *n_sets : parts;       // parts without a set left no sums
  const int col = threadIdx.x & 63, slice = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + col;
  double v = 0.;
  if (c < cols)
    for (int k = slice; k < n; k += 16) v += (double)partial[k * cols + c];
  s[slice][col] = v;
  __syncthreads();
  if (slice || c >= cols) return;
  v = 0.;
#pragma unroll
  for (int k = 0; k < 16; ++k) v += s[k][col];
  out[c] = (float)v;
}

// From offsets to buckets: a wavefront adds a stretch of a head's offsets to a copy of its buckets in LDS, in their order, and the
// copies are added in theirs.
__global__ __launch_bounds__(1024) void k_mha_buckets(const float* __restrict__ by_offset, const int32_t* __restrict__ bucket, int32_t n_off,
                                                      int32_t n_rel, float* __restrict__ d_bias) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  for (int u = threadIdx.x; u < waves * n_rel; u += blockDim.x) lds[u] = 0.f;
  __syncthreads();
  float* mine = lds + wave * n_rel;
  const int per = ((n_off + waves - 1) / waves + 63) & ~63, end = (wave + 1) * per < n_off ? (wave + 1) * per : n_off;
  for (int u = wave * per + lane; u < end; u += 64) {
    const unsigned b = (unsigned)bucket[u];
    if (b < (unsigned)n_rel) unsafeAtomicAdd(&mine[b], by_offset[(int64_t)blockIdx.x * n_off + u]);
  }
  __syncthreads();
  for (int u = threadIdx.x; u < n_rel; u += blockDim.x) {
    double v = 0.;
    for (int w = 0; w < waves; ++w) v += (double)lds[w * n_rel + u];
    d_bias[(int64_t)blockIdx.x * n_rel + u] = (float)v;
  }
}

__global__ void k_mha_zero(float* __restrict__ p, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

struct Plan {
  int32_t hs, parts, n_off, padded;               // padded: channels of a head, rounded up to 16, 32 or 64
  size_t lds, ws;
  bool table_lds;
};

int64_t offsets_of(const dsvt_mha_cfg* c) {
  return (int64_t)(2 * (int64_t)c->win[0] - 1) * (2 * (int64_t)c->win[1] - 1) * (2 * (int64_t)c->win[2] - 1);
}

int make_plan(const dsvt_mha_cfg* c, int32_t max_sets, int32_t tau, bool back, bool d_bias, Plan* p) {
  if (!c || c->C <= 0 || c->heads <= 0 || max_sets < 0 || tau <= 0) return DSVT_EINVAL;
  if (c->dtype != DSVT_F32 && c->dtype != DSVT_BF16) return DSVT_EINVAL;
  if (c->dup_mode != 0 && c->dup_mode != 1) return DSVT_EINVAL;
  if (c->C % c->heads != 0) return DSVT_EINVAL;
  for (int i = 0; i < 3; ++i) if (c->win[i] <= 0 || c->win[i] > 4096) return DSVT_EINVAL;
  if (c->rel_bias && c->n_rel <= 0) return DSVT_EINVAL;
  const int64_t n_off = c->rel_bias ? offsets_of(c) : 0;
  if (c->rel_bias && !c->rel_bucket && c->n_rel != n_off) return DSVT_EINVAL;
  if (d_bias && !c->rel_bias) return DSVT_EINVAL;
  const int hd = c->C / c->heads;
  if (hd % 8 != 0 || hd > 64 || tau > kSetMax || n_off >= (1 << 24)) return DSVT_EUNSUPPORTED;
  if (d_bias && ((size_t)n_off * 4 > kBinsLds || (c->rel_bucket && (size_t)c->n_rel * 4 > kBinsLds))) return DSVT_EUNSUPPORTED;
  p->padded = hd <= 16 ? 16 : hd <= 32 ? 32 : 64;
  p->n_off = (int32_t)n_off;
  p->hs = 1;
  for (int h = 1; h <= kWavesMax; ++h)
    if (c->heads % h == 0 && (!d_bias || (size_t)h * n_off * 4 <= kBinsLds)) p->hs = h;
  const size_t bins = d_bias ? (size_t)p->hs * n_off * 4 : 0, table = (size_t)p->hs * (n_off + 1) * 4;
  p->table_lds = c->rel_bias && bins + table <= kTableLds;
  p->lds = bins + (p->table_lds ? table : 0);
  const int32_t groups = c->heads / p->hs;
  int64_t parts = dsvt_ceil_div(kGroups, groups);
  if (back && parts < dsvt_ceil_div(max_sets, kSetsPerPart)) parts = dsvt_ceil_div(max_sets, kSetsPerPart);
  if (parts > max_sets) parts = max_sets;
  p->parts = (int32_t)dsvt_align_up((size_t)(parts > 0 ? parts : 1), 8);
  p->ws = d_bias ? ((size_t)p->parts + (c->rel_bucket ? 1 : 0)) * c->heads * (size_t)n_off * 4 : 0;
  return DSVT_OK;
}

bool bad_rows(const void* p, int64_t ld, int64_t width, int e) {
  return !p || ((uintptr_t)p & 15u) != 0 || ld < width || (ld * e) % 16 != 0;
}

int check_maps(const dsvt_maps* maps) {
  if (!maps || maps->n_voxels < 0 || maps->max_sets < 0 || maps->tau <= 0) return DSVT_EINVAL;
  if (maps->n_voxels > 0 && (!maps->set_inds || !maps->n_sets)) return DSVT_EINVAL;
  return DSVT_OK;
}

MhaArgs make_args(const dsvt_mha_cfg* c, const dsvt_maps* maps, const int32_t* coords, const Plan& p) {
  MhaArgs a = {};
  a.set_inds = maps->set_inds; a.n_sets = maps->n_sets; a.coords = reinterpret_cast<const int4*>(coords);
  a.bias = c->rel_bias; a.bucket = c->rel_bias ? c->rel_bucket : nullptr;
  a.n_voxels = maps->n_voxels; a.max_sets = maps->max_sets; a.tau = maps->tau; a.heads = c->heads; a.hd = c->C / c->heads;
  a.n_off = p.n_off; a.n_rel = c->n_rel; a.w2 = 2 * c->win[1] - 1; a.h2 = 2 * c->win[2] - 1;
  a.centre = ((c->win[0] - 1) * a.w2 + c->win[1] - 1) * a.h2 + c->win[2] - 1;
  a.dup = c->dup_mode; a.hs = p.hs; a.groups = c->heads / p.hs; a.parts = p.parts; a.table_lds = p.table_lds;
  a.scale = 1.f / sqrtf((float)a.hd);
  return a;
}

template <typename T, int HDP> int launch(const MhaArgs& a, const Plan& p, bool back, hipStream_t st) {
  static std::atomic<uint64_t> allowed[2];
  const void* k = back ? reinterpret_cast<const void*>(k_mha_backward<T, HDP>) : reinterpret_cast<const void*>(k_mha_forward<T, HDP>);
  if (const int rc = dsvt_allow_lds(k, kBinsLds, allowed[back])) return rc;
  const unsigned grid = (unsigned)(a.groups * a.parts), threads = 64 * a.hs;
  dsvt_prof_scope ps(back ? DSVT_K_MHA_BACKWARD : DSVT_K_MHA_FORWARD, st);
  if (back) k_mha_backward<T, HDP><<<grid, threads, p.lds, st>>>(a);
  else k_mha_forward<T, HDP><<<grid, threads, p.lds, st>>>(a);
  return DSVT_OK;
}
int launch(const MhaArgs& a, const Plan& p, int32_t dtype, bool back, hipStream_t st) {
  if (dtype == DSVT_BF16)
    return p.padded == 16 ? launch<bf16_t, 16>(a, p, back, st) : p.padded == 32 ? launch<bf16_t, 32>(a, p, back, st) : launch<bf16_t, 64>(a, p, back, st);
  return p.padded == 16 ? launch<float, 16>(a, p, back, st) : p.padded == 32 ? launch<float, 32>(a, p, back, st) : launch<float, 64>(a, p, back, st);
}

}  // namespace

extern "C" int dsvt_rel_buckets(const int32_t win[3], int32_t n_exact, int32_t n_side, int32_t* bucket, int32_t* n_rel) {
  if (!win || !n_rel || n_exact <= 0 || n_side < n_exact) return DSVT_EINVAL;
  int64_t total = 1, most[3];
  for (int i = 0; i < 3; ++i) {
    if (win[i] <= 0 || win[i] > 4096) return DSVT_EINVAL;
    most[i] = n_side < win[i] ? n_side : win[i];
    total *= 2 * most[i] - 1;
  }
  if (total >= (1 << 24)) return DSVT_EUNSUPPORTED;
  *n_rel = (int32_t)total;
  if (!bucket) return DSVT_OK;
  const auto along = [&](int axis, int32_t d) {               // bucket of a signed distance, 0 .. 2 most - 2
    const int64_t a = d < 0 ? -d : d, b = most[axis];
    int64_t k = a;
    if (a >= n_exact && win[axis] > n_exact)
      k = n_exact + (int64_t)floor((double)(b - n_exact) * (log((double)a / n_exact) / log((double)win[axis] / n_exact)));
    k = k < b - 1 ? k : b - 1;
    return b - 1 + (d < 0 ? -k : k);
  };
  int64_t at = 0;
  for (int32_t x = 1 - win[0]; x < win[0]; ++x)
    for (int32_t y = 1 - win[1]; y < win[1]; ++y)
      for (int32_t z = 1 - win[2]; z < win[2]; ++z)
        bucket[at++] = (int32_t)((along(0, x) * (2 * most[1] - 1) + along(1, y)) * (2 * most[2] - 1) + along(2, z));
  return DSVT_OK;
}

extern "C" int dsvt_set_mha(const dsvt_mha_cfg* cfg, const dsvt_maps* maps, const int32_t* coords, const void* qkv, int64_t ld_qkv, void* out,
                            int64_t ld_out, void* stream) {
  if (const int rc = check_maps(maps)) return rc;
  Plan p;
  if (const int rc = make_plan(cfg, maps->max_sets, maps->tau, false, false, &p)) return rc;
  if (maps->n_voxels == 0 || maps->max_sets == 0) return DSVT_OK;
  const int e = cfg->dtype == DSVT_BF16 ? 2 : 4;
  if (!coords || ((uintptr_t)coords & 15u) || bad_rows(qkv, ld_qkv, 3 * (int64_t)cfg->C, e) || bad_rows(out, ld_out, cfg->C, e)) return DSVT_EINVAL;
  MhaArgs a = make_args(cfg, maps, coords, p);
  a.qkv = qkv; a.ld_qkv = ld_qkv; a.out = out; a.ld_out = ld_out;
  if (const int rc = launch(a, p, cfg->dtype, false, (hipStream_t)stream)) return rc;
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}

extern "C" int dsvt_set_mha_backward_workspace_size(const dsvt_mha_cfg* cfg, const dsvt_maps* maps, size_t* bytes) {
  if (!bytes) return DSVT_EINVAL;
  if (const int rc = check_maps(maps)) return rc;
  Plan p;
  if (const int rc = make_plan(cfg, maps->max_sets, maps->tau, true, cfg && cfg->rel_bias, &p)) return rc;
  *bytes = p.ws;
  return DSVT_OK;
}

extern "C" int dsvt_set_mha_backward(const dsvt_mha_cfg* cfg, const dsvt_maps* maps, const int32_t* coords, const void* qkv, int64_t ld_qkv,
                                     const void* d_out, int64_t ld_dout, void* d_qkv, int64_t ld_dqkv, float* d_rel_bias, void* ws,
                                     size_t ws_bytes, void* stream) {
  if (const int rc = check_maps(maps)) return rc;
  Plan p;
  if (const int rc = make_plan(cfg, maps->max_sets, maps->tau, true, d_rel_bias != nullptr, &p)) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (maps->n_voxels == 0 || maps->max_sets == 0) {
    if (d_rel_bias) {
      const int64_t n = (int64_t)cfg->heads * cfg->n_rel;
      k_mha_zero<<<(unsigned)dsvt_ceil_div(n, 256), 256, 0, st>>>(d_rel_bias, n);
      DSVT_HIP_TRY(hipGetLastError());
    }
    return DSVT_OK;
  }
  const int e = cfg->dtype == DSVT_BF16 ? 2 : 4;
  const int64_t C = cfg->C;
  if (!coords || ((uintptr_t)coords & 15u) || bad_rows(qkv, ld_qkv, 3 * C, e) || bad_rows(d_out, ld_dout, C, e) || bad_rows(d_qkv, ld_dqkv, 3 * C, e))
    return DSVT_EINVAL;
  if (p.ws > 0 && (!ws || ((uintptr_t)ws & 15u))) return DSVT_EINVAL;
  if (ws_bytes < p.ws) return DSVT_ENOSPC;
  MhaArgs a = make_args(cfg, maps, coords, p);
  a.qkv = qkv; a.ld_qkv = ld_qkv; a.d_out = d_out; a.ld_dout = ld_dout; a.out = d_qkv; a.ld_out = ld_dqkv;
  a.partial = d_rel_bias ? static_cast<float*>(ws) : nullptr;
  static std::atomic<uint64_t> allowed;
  if (d_rel_bias && cfg->rel_bucket)
    if (const int rc = dsvt_allow_lds(reinterpret_cast<const void*>(k_mha_buckets), kBinsLds, allowed)) return rc;
  if (const int rc = launch(a, p, cfg->dtype, true, st)) return rc;
  if (d_rel_bias) {
    const int64_t cols = (int64_t)cfg->heads * p.n_off;
    float* by_offset = cfg->rel_bucket ? a.partial + p.parts * cols : d_rel_bias;
    dsvt_prof_scope ps(DSVT_K_MHA_REL, st);
    k_mha_offsets<<<(unsigned)dsvt_ceil_div(cols, 64), 1024, 0, st>>>(a.partial, maps->n_sets, p.parts < maps->max_sets ? p.parts : maps->max_sets, cols, by_offset);
    if (cfg->rel_bucket) {
      size_t waves = kBinsLds / ((size_t)cfg->n_rel * 4);
      waves = waves > 16 ? 16 : waves;
      k_mha_buckets<<<(unsigned)cfg->heads, (unsigned)(64 * waves), waves * cfg->n_rel * 4, st>>>(by_offset, cfg->rel_bucket, p.n_off, cfg->n_rel, d_rel_bias);
    }
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}
