// What the kernels of dsvt_set_mha and dsvt_set_mha_backward share (mha_forward.h, mha_backward.h); the entry points are
// in mha.hip.  Multi-head attention inside every set (Eq. 5, second line) on rows that are already projected, with a learned
// relative position bias per offset or per bucket of offsets, and its gradients.  With g = d out, sigma = 1/sqrt(d), m_j the
// weight of voxel j as a key (1, or the number of its slots), B the bucket of an offset:
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
// becomes NaN in all of its channels).  LDS holds no tile, only what is known of the sets, and the tables.
#pragma once
#include "common.h"
#include "mma.h"
#include <cfloat>
#include <cmath>
#include <type_traits>

constexpr int kSetMax = 96;                       // slots, and so voxels, of a set
constexpr int kMhaWavesMax = 8;                   // wavefronts of a workgroup, and so sets that it looks up together
constexpr float kLog2e = 1.44269504088896340736f;

// Where a pair's bias is found.  By offset: LDS holds a value for every offset and head.  By bucket: LDS holds the offsets' buckets
// (16 bits, one past the last for offsets without a bias) and a value for every bucket and head.  In memory: biases and buckets are read
// where they lie.
enum TableForm { kByOffset, kByBucket, kInMemory };

struct MhaArgs {
  const int32_t *set_inds, *n_sets;
  const int4* coords;
  const void *qkv, *d_out;
  void* out;                                      // forward: the output rows; backward: d_qkv
  const float* bias;                              // [heads][n_rel] or null
  const int32_t* bucket;                          // [n_off] or null
  float* partial;                                 // backward: [parts][heads][entries]; null: no gradient of the table
  uint32_t ld_qkv, ld_dout, ld_out;               // row strides in bytes
  int32_t n_voxels, max_sets, tau, heads, hd;
  int32_t n_off, n_rel, entries;                  // offsets; biases of a head; values of a head in LDS
  int32_t w[3], centre;                           // the window; the number of offset 0
  int32_t dup, hs, slots, groups, parts;          // heads of a workgroup, sets it takes side by side, groups of heads, workgroups a group
  int32_t ranges;                                 // backward: workgroups that share a head's entries (each goes through all sets)
  float scale;
};

typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) float lds_float;
typedef __attribute__((address_space(3))) const uint16_t lds_u16;

// Matrix fragments.  A row fragment covers 4 * KL channels: lane 16 g + m holds channels KL g .. KL g + KL - 1 of row m.  A
// tile fragment covers 16: lane 16 g + m holds elements 4 g .. 4 g + 3 of row (or column) m.
template <typename T, int HDP> struct Frag;
template <int HDP> struct Frag<bf16_t, HDP> {
  static constexpr int KL = HDP == 16 ? 4 : 8, NC = HDP / (4 * KL), NT = HDP / 16, PER = KL / 4;
  typedef bf16_t Row __attribute__((ext_vector_type(KL)));
  typedef short4_t Tile;
  static __device__ __forceinline__ f32x4 tile_mma(Tile a, Tile b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x4 row_mma(Row a, Row b, f32x4 c) {
    if constexpr (KL == 8) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else return tile_mma(__builtin_bit_cast(Tile, a), __builtin_bit_cast(Tile, b), c);
  }
  // P and ds of bf16 rows are rounded to bf16 here, as operands: the products of 32-bit operands run at a sixteenth of the rate.  With the
  // rounding of the results the forward call is off by 2.0e-3 of its norm instead of 1.7e-3, the backward call by 2.4e-3.
  // (pairs in 32-bit words: on vectors of four that become operands the compiler converts one by one)
  static __device__ __forceinline__ unsigned pair(float a, float b) {
    typedef float F2 __attribute__((ext_vector_type(2)));
    typedef bf16_t B2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_convertvector(F2{a, b}, B2));
  }
  static __device__ __forceinline__ Tile tile(f32x4 v) { return __builtin_bit_cast(Tile, make_uint2(pair(v[0], v[1]), pair(v[2], v[3]))); }
  // of values that are bf16 already: their upper halves
  static __device__ __forceinline__ Tile exact_tile(f32x4 v) {
    const auto upper = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };
    return __builtin_bit_cast(Tile, make_uint2(upper(v[0], v[1]), upper(v[2], v[3])));
  }
};
template <int HDP> struct Frag<float, HDP> {
  static constexpr int KL = 4, NC = HDP / 16, NT = HDP / 16, PER = 1;
  typedef f32x4 Row;
  typedef f32x4 Tile;
  static __device__ __forceinline__ f32x4 tile_mma(Tile a, Tile b, f32x4 c) { return Mma<float>::mma(a, b, c); }
  static __device__ __forceinline__ f32x4 row_mma(Row a, Row b, f32x4 c) { return Mma<float>::mma(a, b, c); }
  static __device__ __forceinline__ Tile tile(f32x4 v) { return v; }
  static __device__ __forceinline__ Tile exact_tile(f32x4 v) { return v; }
};

// Lanes 16 apart hold the same query's other keys: every lane gets the sum (largest) of its four.
template <typename Op> __device__ __forceinline__ float across(float v, Op op) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float across_sum(float v) { return across(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float across_max(float v) { return across(v, raw_max); }

// 1 / sum of probabilities: the instruction's value and one Newton step, half a dozen instructions less than a division.  0 for 0.
__device__ __forceinline__ float inverse(float sum) {
  const float r = __builtin_amdgcn_rcpf(sum);
  return sum == 0.f ? 0.f : fmaf(fmaf(-sum, r, 1.f), r, r);
}

// The logits are formed in units of sigma, so that a bias is what the product of q and k starts from.  A finite bias stays finite.
__device__ __forceinline__ float to_units(float b, float root) {
  return fabsf(b) <= FLT_MAX ? fminf(fmaxf(b, -1.0e37f), 1.0e37f) * root : b;
}

// What a workgroup knows of a set, in LDS.  Row r is the set's r-th voxel; rows up to the next multiple of 16 repeat row 0 with
// weight 0: they are read like others, and masked where they would count.  code: the cell's number times the bytes of an entry, so that the
// difference of two codes is an offset's place in a table.
template <int kMax> struct alignas(16) SetRows {
  int32_t vox[kMax], code[kMax], weight[kMax];
  int32_t n;
};
// four neighbouring values from the `at`-th on, a multiple of four
__device__ __forceinline__ int4 four(const int32_t* values, int at) { return *reinterpret_cast<const int4*>(values + at); }

// Largest of the wavefront's values, by shifts over 1, 2, 4, 8 lanes of a row and row broadcasts; in the last lane, from where all get it.
__device__ __forceinline__ int wave_max(int v) {
  const auto step = [](int a, int b) { return a > b ? a : b; };
  v = step(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x111, 0xF, 0xF, false));
  v = step(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x112, 0xF, 0xF, false));
  v = step(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x114, 0xF, 0xF, false));
  v = step(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x118, 0xF, 0xF, false));
  v = step(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x142, 0xA, 0xF, false));
  v = step(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x143, 0xC, 0xF, false));
  return __builtin_amdgcn_readlane(v, 63);
}

// A wavefront looks a set's distinct voxels up, in slot order: the first slot of every run of equal ones.  Slots outside
// 0 .. n_voxels - 1 hold none.  In three steps, so that their loads travel while sets that were looked up before are computed: the
// slots, the cells of the first slots, the rows in LDS.
template <int kMax> struct Lookup {
  static constexpr int kWords = kMax > 64 ? 2 : 1;             // slots of a lane
  int32_t v[kWords];
  int4 c[kWords];
  uint64_t first[kWords], change[kWords];

  __device__ __forceinline__ void slots(const MhaArgs& a, int32_t s) {
    const int32_t* inds = a.set_inds + (int64_t)s * a.tau;
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      const int slot = 64 * k + (int)(threadIdx.x & 63);
      v[k] = slot < a.tau ? inds[slot] : -1;
    }
  }
  __device__ __forceinline__ void cells(const MhaArgs& a) {
    const int lane = threadIdx.x & 63;
    int32_t before = -1;
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      if ((uint32_t)v[k] >= (uint32_t)a.n_voxels) v[k] = -1;
      int32_t prev = __shfl_up(v[k], 1, 64);
      if (lane == 0) prev = before;
      before = __shfl(v[k], 63, 64);
      change[k] = __ballot(v[k] != prev || 64 * k + lane >= a.tau);
      first[k] = __ballot(v[k] != prev && v[k] >= 0);
      c[k] = make_int4(0, 0, 0, 0);
      if (first[k] >> lane & 1) c[k] = a.coords[v[k]];
    }
  }
  // Voxels that do not fit one window (the maps are another window's) all get code 0, so that every offset formed from two codes is in
  // the table.
  __device__ __forceinline__ void rows(const MhaArgs& a, int entry_bytes, SetRows<kMax>& out) {
    const int lane = threadIdx.x & 63;
    int lo[3], hi[3], n = 0;
#pragma unroll
    for (int x = 0; x < 3; ++x) lo[x] = hi[x] = INT32_MIN;
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      n += __popcll(first[k]);
      if (first[k] >> lane & 1) {
        const int at[3] = {c[k].y, c[k].z, c[k].w};
#pragma unroll
        for (int x = 0; x < 3; ++x) {
          hi[x] = at[x] > hi[x] ? at[x] : hi[x];
          lo[x] = -1 - at[x] > lo[x] ? -1 - at[x] : lo[x];
        }
      }
    }
    if (lane == 0) out.n = n;
    if (n == 0) return;
    // highest + 1 - lowest <= window along every axis (the lowest is kept as the highest of -1 - x)
    bool fits = a.bias != nullptr;
#pragma unroll
    for (int x = 0; x < 3; ++x) fits = fits && (int64_t)wave_max(hi[x]) + wave_max(lo[x]) + 2 <= a.w[x];
    const uint32_t w2 = 2 * a.w[1] - 1, h2 = 2 * a.w[2] - 1;
    uint32_t code[kWords];
    int before = 0;
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      // (unsigned: a far cell's number may pass 32 bits, the differences inside a window do not)
      code[k] = fits ? (((uint32_t)c[k].y * w2 + (uint32_t)c[k].z) * h2 + (uint32_t)c[k].w) * entry_bytes : 0;
      if (first[k] >> lane & 1) {
        const int r = before + __popcll(first[k] & ((1ull << lane) - 1));
        const uint64_t later = lane == 63 ? 0 : change[k] >> (lane + 1);    // slots to the next change
        int run = later ? 1 + __builtin_ctzll(later) : 64 - lane;
        if (kWords > 1 && k == 0 && !later) run += change[kWords - 1] ? __builtin_ctzll(change[kWords - 1]) : 64;
        out.vox[r] = v[k];
        out.code[r] = (int32_t)code[k];
        out.weight[r] = a.dup ? run : 1;
      }
      before += __popcll(first[k]);
    }
    const int k0 = first[0] ? 0 : kWords - 1, l0 = __builtin_ctzll(first[k0]);
    const int32_t vox0 = __shfl(k0 ? v[kWords - 1] : v[0], l0, 64), code0 = __shfl((int32_t)(k0 ? code[kWords - 1] : code[0]), l0, 64);
    if (n + lane < ((n + 15) & ~15)) {
      out.vox[n + lane] = vox0;
      out.code[n + lane] = code0;
      out.weight[n + lane] = 0;
    }
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

__device__ __forceinline__ int32_t sets_of(const MhaArgs& a) {
  const int32_t n = *a.n_sets;
  return n < 0 ? 0 : (n > a.max_sets ? a.max_sets : n);
}

// Where in LDS p points, as the LDS instructions want it.
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }

// The heads' biases in units of sigma, and by bucket the offsets' buckets; offsets without a bias get 0.  A thread fetches two entries of all
// heads, 16 of one head, or eight buckets, before it stores any: one after the other they were half of a forward call on 30,000 voxels.
template <TableForm kForm> __device__ __forceinline__ void fill_tables(const MhaArgs& a, int h0, float* table, uint16_t* map) {
  if constexpr (kForm == kInMemory) return;
  const float root = sqrtf((float)a.hd);
  const float* bias = a.bias + (int64_t)h0 * a.n_rel;
  const int step = blockDim.x;
  // kHeads heads from h1 on, kEntries entries of each
  const auto fetch = [&](auto heads, auto entries, int h1) {
    constexpr int kHeads = decltype(heads)::value, kEntries = decltype(entries)::value;
    for (int u = threadIdx.x; u < a.entries; u += kEntries * step) {
      float f[kEntries][kHeads] = {};
      if (a.bias) {
#pragma unroll
        for (int j = 0; j < kEntries; ++j) {
          const int at = u + j * step, r = at < a.n_rel ? at : a.n_rel - 1;                // (fetched where there is none, and cleared below)
#pragma unroll
          for (int h = 0; h < kHeads; ++h) f[j][h] = bias[(int64_t)(h1 + h < a.hs ? h1 + h : 0) * a.n_rel + r];
        }
      }
#pragma unroll
      for (int j = 0; j < kEntries; ++j) {
        const int at = u + j * step;
#pragma unroll
        for (int h = 0; h < kHeads; ++h)
          if (h1 + h < a.hs && at < a.entries) table[(h1 + h) * a.entries + at] = at < a.n_rel ? to_units(f[j][h], root) : 0.f;
      }
    }
  };
  if (a.hs > 2) fetch(std::integral_constant<int, kMhaWavesMax>(), std::integral_constant<int, 2>(), 0);
  else
    for (int h = 0; h < a.hs; ++h) fetch(std::integral_constant<int, 1>(), std::integral_constant<int, 16>(), h);
  if constexpr (kForm == kByBucket) {
    constexpr int kAtOnce = 8;
    for (int u = threadIdx.x; u < a.n_off; u += kAtOnce * blockDim.x) {
      unsigned r[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int at = u + j * (int)blockDim.x;
        r[j] = (unsigned)a.bucket[at < a.n_off ? at : u];
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int at = u + j * (int)blockDim.x;
        if (at < a.n_off) map[at] = (uint16_t)(r[j] < (unsigned)a.n_rel ? r[j] : a.n_rel);
      }
    }
  }
}

// One wavefront's head: where its rows and biases are, and its part of the matrix fragments.
template <typename T, int HDP, TableForm kForm, int kMax> struct Head {
  typedef Frag<T, HDP> F;
  typedef SetRows<kMax> Rows;
  typedef typename F::Row Row;
  typedef typename F::Tile Tile;
  const MhaArgs& a;
  uint32_t table, map;                            // LDS: this head's values, the offsets' buckets
  const float* bias;                              // memory: this head's biases
  int m, g, h;
  float root, scale2;                             // 1 / sigma, sigma log2 e

  __device__ __forceinline__ Head(const MhaArgs& a_, const float* table_, const uint16_t* map_, int h_)
      : a(a_), table(lds_address(table_)), map(lds_address(map_)), bias(a_.bias + (int64_t)h_ * a_.n_rel), m(threadIdx.x & 15),
        g(threadIdx.x >> 4 & 3), h(h_), root(sqrtf((float)a_.hd)), scale2(a_.scale * kLog2e) {}
  static constexpr int entry_bytes() { return kForm == kByBucket ? 2 : 4; }

  // A lane's first channel of part c of a row fragment; lanes past the head's last channel take its first ones.
  __device__ __forceinline__ int channel(int c) const {
    const int d = (4 * c + g) * F::KL;
    return d < a.hd ? d : 0;
  }
  __device__ __forceinline__ const char* row(const Rows& rows, const void* base, uint32_t ld, int which, int t) const {
    return static_cast<const char*>(base) + (int64_t)(which * a.heads + h) * a.hd * (int)sizeof(T) + (uint64_t)(uint32_t)rows.vox[16 * t + m] * ld;
  }
  // Rows of tile t of an array of head vectors (which: 0 q, 1 k, 2 v of a qkv row; 0 of an output row).
  __device__ __forceinline__ void load(const Rows& rows, const void* base, uint32_t ld, int which, int t, Row (&f)[F::NC]) const {
    const char* p = row(rows, base, ld, which, t);
#pragma unroll
    for (int c = 0; c < F::NC; ++c) f[c] = *reinterpret_cast<const Row*>(p + channel(c) * (int)sizeof(T));
  }
  // Zeros past the head's last channel: in one of two operands whose product runs over the channels.
  __device__ __forceinline__ void clear_past_last(Row (&f)[F::NC]) const {
    const Row zero = {};
#pragma unroll
    for (int c = 0; c < F::NC; ++c) f[c] = (4 * c + g) * F::KL < a.hd ? f[c] : zero;
  }
  // tiles of the transposed result, column m = row m of tile t, if `there`: a lane holds the channels that it holds of a row fragment
  __device__ __forceinline__ void store(const Rows& rows, void* base, uint32_t ld, int which, int t, bool there, const f32x4 (&o)[F::NT],
                                        float scale) const {
    char* p = const_cast<char*>(row(rows, base, ld, which, t));
#pragma unroll
    for (int c = 0; c < F::NC; ++c) {
      typedef float Wide __attribute__((ext_vector_type(F::KL)));
      Wide r;
#pragma unroll
      for (int e = 0; e < F::KL; ++e) r[e] = o[c * F::PER + e / 4][e % 4] * scale;
      if (there && (4 * c + g) * F::KL < a.hd) *reinterpret_cast<Row*>(p + channel(c) * (int)sizeof(T)) = __builtin_convertvector(r, Row);
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
    f32x4 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = 4 * g + e == m ? 1.f : 0.f;
    return F::exact_tile(u);
  }
  // rows -> NT tile fragments: lane holds channel (of tile n) m, rows 4 g .. 4 g + 3
  __device__ __forceinline__ void turn(const Row (&f)[F::NC], Tile (&o)[F::NT]) const {
#pragma unroll
    for (int n = 0; n < F::NT; ++n) o[n] = F::exact_tile(F::row_mma(f[n / F::PER], unit(n % F::PER), f32x4{0.f, 0.f, 0.f, 0.f}));
  }
  __device__ __forceinline__ Tile turn(Tile f) const { return F::exact_tile(F::tile_mma(f, tile_unit(), f32x4{0.f, 0.f, 0.f, 0.f})); }

  // LDS address (in memory: byte offset in the head's table) of the entry of an offset, given as the difference of two codes plus `from`
  __device__ __forceinline__ uint32_t from() const {
    return (uint32_t)(a.centre * entry_bytes()) + (kForm == kByOffset ? table : kForm == kByBucket ? map : 0u);
  }
  // entry of the four pairs of query code `at` (plus from()) and the keys 16 t + 4 g .. + 3
  __device__ __forceinline__ void entries(const Rows& rows, uint32_t at, int t, uint32_t (&e)[4]) const {
    const int4 key = four(rows.code, 16 * t + 4 * g);
    e[0] = entry(at - (uint32_t)key.x);
    e[1] = entry(at - (uint32_t)key.y);
    e[2] = entry(at - (uint32_t)key.z);
    e[3] = entry(at - (uint32_t)key.w);
  }
  __device__ __forceinline__ uint32_t entry(uint32_t at) const {
    if constexpr (kForm == kByBucket) return table + 4u * *(lds_u16*)(uintptr_t)at;
    if constexpr (kForm == kInMemory)
      if (a.bucket) {
        const unsigned r = (unsigned)*reinterpret_cast<const int32_t*>(reinterpret_cast<const char*>(a.bucket) + at);
        return 4u * (r < (unsigned)a.n_rel ? r : (unsigned)a.n_rel);
      }
    return at;
  }
  __device__ __forceinline__ float value(uint32_t entry) const {
    if constexpr (kForm == kInMemory)
      return entry < 4u * (unsigned)a.n_rel ? to_units(*reinterpret_cast<const float*>(reinterpret_cast<const char*>(bias) + entry), root) : 0.f;
    return *(lds_float*)(uintptr_t)entry;
  }

  // Probabilities of one query tile before their division by the sum: p holds the logits of kTiles key tiles in units of sigma.  Returns
  // this lane's part of the sum.
  template <int kTiles> __device__ __forceinline__ float exponentials(const Rows& rows, f32x4 (&p)[kTiles]) const {
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < kTiles; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, p[k][i]);
    top = across_max(top);
    if (top == -INFINITY) top = 0.f;              // every key is masked: no probabilities
    const float shift = top * scale2;
    // One fma an exponent.  Its error, half a step of `shift`, is the same for all keys of the query and so falls out; it has to
    // be small only against the range of exp2.
    if (__any(fabsf(shift) > 16777216.f)) {
#pragma unroll
      for (int k = 0; k < kTiles; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[k][i] = __builtin_amdgcn_exp2f((p[k][i] - top) * scale2);
    } else {
#pragma unroll
      for (int k = 0; k < kTiles; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[k][i] = __builtin_amdgcn_exp2f(fmaf(p[k][i], scale2, -shift));
    }
    if (a.dup) {
#pragma unroll
      for (int k = 0; k < kTiles; ++k) {
        const int4 w = four(rows.weight, 16 * k + 4 * g);
        p[k] *= f32x4{(float)w.x, (float)w.y, (float)w.z, (float)w.w};
      }
    }
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < kTiles; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += p[k][i];
    return sum;
  }
};

// Launchers; `form` as the tables are laid out (mha.hip chooses it), `lds` bytes of dynamic LDS.
int mha_forward_bf16(const MhaArgs& a, TableForm form, size_t lds, hipStream_t st);
int mha_forward_f32(const MhaArgs& a, TableForm form, size_t lds, hipStream_t st);
int mha_backward_bf16(const MhaArgs& a, TableForm form, size_t lds, hipStream_t st);
int mha_backward_f32(const MhaArgs& a, TableForm form, size_t lds, hipStream_t st);

// Wavefronts of a workgroup: eight; four where a wavefront needs more than half of its SIMD's registers.
__host__ __device__ constexpr int mha_waves(bool back, int element, int padded, int tau) {
  return padded == 64 || (padded == 32 && tau > 48 && (back || element == 4)) ? 4 : 8;
}
// Workgroups of a compute unit: two where a quarter of the registers does, else one.
__host__ __device__ constexpr int mha_per_cu(bool back, int element, int padded, int tau) { return !back && padded * element <= 64 && tau <= 48 ? 2 : 1; }
__host__ __device__ constexpr int mha_per_simd(bool back, int element, int padded, int tau) {
  return mha_waves(back, element, padded, tau) * mha_per_cu(back, element, padded, tau) / 4;
}
// Dynamic LDS of a workgroup, at most: 160 KB less what its sets take (14 KB of up to 48 voxels, 28 KB of up to 96), or half of it.  (What
// small sets leave more: 120,000 voxels, 12 x 12 x 12 windows with an entry an offset, backward 200 us, 345 with 131 KB and the table in memory.)
__host__ __device__ constexpr size_t mha_lds_max(int tau, int per_cu) { return (per_cu == 2 ? 65 : tau <= 48 ? 146 : 131) << 10; }

extern __shared__ double mha_lds[];
