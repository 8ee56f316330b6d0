// The backward kernel of dsvt_set_mha_backward (see mha.h), for the two types' own files.
//
// With the queries as columns, P and ds of one query tile and all keys are in registers; dq comes from them as they are, dk and dv, which
// run over the queries, from P and ds turned round, summed up over the query tiles in registers.  That takes half of a SIMD's registers, so two
// wavefronts share it, and what bounds a large call is a set's chain of steps at that: C = 192, 8 heads, bf16, 800,000 voxels in full sets of
// 36 with 2,197 buckets 1,005 us (2.15 GB: 2.1 TB/s); 708 with all rows in the caches and additions in any order, 488 without additions and
// stores.  30,000 voxels 33.5 us a pass, 4.5 of them the last step of the table's gradient.
#pragma once
#include "mha.h"

namespace {

// The order in which a workgroup's wavefronts add to the sums of one head, so that the sums do not depend on their speed: by the
// place of their set in the part's sequence (`slots` sets are taken side by side, each in `tiles` query tiles) -- round, then query
// tile, then slot.  A wavefront waits until the turn is its own; it hands on the turns of tiles that its set does not
// have.  Every wavefront takes its turns in rising order, so the one whose turn is lowest never waits for another.  With one slot a
// head's sums belong to one wavefront and nothing waits.
typedef volatile __attribute__((address_space(3))) int lds_turn;
struct Turns {
  lds_turn* next;                                 // LDS: this head's turn
  bool wanted;                                    // more than one slot
  int slots, slot, tiles, done;                   // done: turns of this wavefront that are over
  __device__ __forceinline__ int turn() const { return done * slots + slot; }
  __device__ __forceinline__ void wait() const {
    if (!wanted) return;
    while (*next != turn()) {}
    asm volatile("" ::: "memory");
  }
  __device__ __forceinline__ void hand_on() {
    if (!wanted) return;
    asm volatile("" ::: "memory");                // (LDS does a wavefront's operations in their order: the additions before this)
    if ((threadIdx.x & 63) == 0) *next = turn() + 1;
    ++done;
  }
  // up to the first turn of round r
  __device__ __forceinline__ void skip_to(int r) {
    if (!wanted) return;
    while (done < r * tiles) {
      wait();
      hand_on();
    }
  }
};

// A head's sums of the table's gradient in LDS, 64 bits each: the additions of a wavefront take 9 to 26 clocks of the LDS, those of
// 32-bit floats take 193 (1 lane in three clocks), read with 64 lanes on consecutive up to random entries.
struct Bins {
  uint32_t base;                                  // LDS address of the sum of entry address 0 (modulo 2^32)
  uint32_t lo, span;                              // kInMemory: the entries' bytes that this workgroup adds up
  bool rows_too;                                  // this workgroup writes the rows
  template <TableForm kForm> __device__ __forceinline__ void add(uint32_t entry, float v) const {
    typedef __attribute__((address_space(3))) double lds_double;
    if constexpr (kForm == kInMemory) {
      entry -= lo;
      if (entry >= span) return;
    }
    __hip_atomic_fetch_add((lds_double*)(uintptr_t)(base + 2 * entry), (double)v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
};

// A set's rows of one head as fragments.  Of sets of up to three tiles of narrow heads they all sit in registers, and the next set's are
// fetched as soon as this one's are used up; else they are read as they are needed, again for each query
// tile, from the caches.
template <typename T, int HDP, int kMax> constexpr bool hold_rows() { return HDP * sizeof(T) <= 64 && kMax <= 48; }
template <typename T, int HDP, int kMax> struct Held {
  static constexpr int kTiles = hold_rows<T, HDP, kMax>() ? kMax / 16 : 1;
  typename Frag<T, HDP>::Row q[kTiles][Frag<T, HDP>::NC], k[kTiles][Frag<T, HDP>::NC], v[kTiles][Frag<T, HDP>::NC], g[kTiles][Frag<T, HDP>::NC];
  template <TableForm kForm> __device__ __forceinline__ void fetch_kv(const Head<T, HDP, kForm, kMax>& head, const SetRows<kMax>& rows) {
    if constexpr (hold_rows<T, HDP, kMax>()) {
      const MhaArgs& a = head.a;
      const int tiles = (__builtin_amdgcn_readfirstlane(rows.n) + 15) >> 4;
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
        if (t < tiles) {
          head.load(rows, a.qkv, a.ld_qkv, 1, t, k[t]);
          head.load(rows, a.qkv, a.ld_qkv, 2, t, v[t]);
        }
    }
  }
  // tiles kFirst .. kEnd - 1
  template <int kFirst, int kEnd, TableForm kForm> __device__ __forceinline__ void fetch_qg(const Head<T, HDP, kForm, kMax>& head, const SetRows<kMax>& rows) {
    if constexpr (hold_rows<T, HDP, kMax>()) {
      const MhaArgs& a = head.a;
      const int tiles = (__builtin_amdgcn_readfirstlane(rows.n) + 15) >> 4;
#pragma unroll
      for (int t = kFirst; t < (kEnd < kTiles ? kEnd : kTiles); ++t)
        if (t < tiles) {
          head.load(rows, a.qkv, a.ld_qkv, 0, t, q[t]);
          head.load(rows, a.d_out, a.ld_dout, 0, t, g[t]);
        }
    }
  }
  template <TableForm kForm> __device__ __forceinline__ void fetch(const Head<T, HDP, kForm, kMax>& head, const SetRows<kMax>& rows) {
    fetch_qg<0, kTiles>(head, rows);
    fetch_kv(head, rows);
  }
};

template <int kTiles, typename T, int HDP, TableForm kForm, int kMax>
__device__ __forceinline__ void backward_set(const Head<T, HDP, kForm, kMax>& head, const SetRows<kMax>& rows, int n, const Bins& bins, Turns& turns,
                                             Held<T, HDP, kMax>& held, const SetRows<kMax>* next) {
  typedef Frag<T, HDP> F;
  typedef typename F::Row Row;
  typedef typename F::Tile Tile;
  constexpr bool kHold = hold_rows<T, HDP, kMax>();
  const MhaArgs& a = head.a;
  const int m = head.m, g = head.g;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  auto &k = held.k, &v = held.v;
  Tile turned_k[kHold ? kTiles : 1][F::NT];
  f32x4 dk[kTiles][F::NT] = {}, dv[kTiles][F::NT] = {};
#pragma unroll kHold ? kTiles : 1
  for (int qt = 0; qt < kTiles; ++qt) {
    Row (&q)[F::NC] = held.q[kHold ? qt : 0], (&go)[F::NC] = held.g[kHold ? qt : 0];
    if constexpr (!kHold) {
      head.load(rows, a.qkv, a.ld_qkv, 0, qt, q);
      head.load(rows, a.d_out, a.ld_dout, 0, qt, go);
    }
    head.clear_past_last(q);
    head.clear_past_last(go);
    const uint32_t at = (uint32_t)rows.code[16 * qt + m] + head.from();
    f32x4 p[kTiles], s[kTiles];                   // p: logits, then probabilities; s: t, then ds
    uint32_t entry[kTiles][4];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      if constexpr (!kHold) {
        head.load(rows, a.qkv, a.ld_qkv, 1, t, k[0]);
        head.load(rows, a.qkv, a.ld_qkv, 2, t, v[0]);
      }
      head.entries(rows, at, t, entry[t]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[t][i] = head.value(entry[t][i]);
        if (t == kTiles - 1 && 16 * t + 4 * g + i >= n) p[t][i] = -INFINITY;
      }
      s[t] = zero;
#pragma unroll
      for (int c = 0; c < F::NC; ++c) {
        p[t] = F::row_mma(k[kHold ? t : 0][c], q[c], p[t]);
        s[t] = F::row_mma(v[kHold ? t : 0][c], go[c], s[t]);
      }
    }
    if constexpr (kHold) {
      if (qt == 0) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) head.turn(k[t], turned_k[t]);
      }
      if (qt == kTiles - 1 && next) {             // what this set does not need any more
        held.fetch_kv(head, *next);
        held.template fetch_qg<0, kTiles - 1>(head, *next);
      }
    }
    const bool query = qt + 1 < kTiles || 16 * qt + m < n;
    float sum = head.template exponentials<kTiles>(rows, p), dot = 0.f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) dot = fmaf(p[t][i], s[t][i], dot);
    sum = across_sum(sum);
    const float inv = query ? inverse(sum) : 0.f;
    dot = across_sum(dot) * inv;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[t][i] *= inv;
        s[t][i] = p[t][i] * (s[t][i] - dot);
      }
    if (a.partial) {
      turns.wait();
      if (query) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (t + 1 < kTiles || 16 * t + 4 * g + i < n) bins.template add<kForm>(entry[t][i], s[t][i]);
      }
      turns.hand_on();
      if (!bins.rows_too) continue;               // another workgroup writes the rows
    }
    f32x4 dq[F::NT] = {};
    Tile turned_q[F::NT], turned_g[F::NT];
    head.turn(q, turned_q);
    head.turn(go, turned_g);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      if constexpr (!kHold) {
        head.load(rows, a.qkv, a.ld_qkv, 1, t, k[0]);
        head.turn(k[0], turned_k[0]);
      }
      const Tile ds = F::tile(s[t]), ds_t = head.turn(ds), p_t = head.turn(F::tile(p[t]));
#pragma unroll
      for (int c = 0; c < F::NT; ++c) {
        dq[c] = F::tile_mma(turned_k[kHold ? t : 0][c], ds, dq[c]);
        dk[t][c] = F::tile_mma(turned_q[c], ds_t, dk[t][c]);
        dv[t][c] = F::tile_mma(turned_g[c], p_t, dv[t][c]);
      }
    }
    head.store(rows, a.out, a.ld_out, 0, qt, query, dq, a.scale);
  }
  if (next) held.template fetch_qg<kTiles - 1, kMax>(head, *next);
  if (!bins.rows_too) return;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const bool there = t + 1 < kTiles || 16 * t + m < n;
    head.store(rows, a.out, a.ld_out, 1, t, there, dk[t], a.scale);
    head.store(rows, a.out, a.ld_out, 2, t, there, dv[t], 1.f);
  }
}

// Dynamic LDS: the sums of the table's gradient [hs][entries of the range] if they are wanted, the table [hs][entries] unless it stays in
// memory, the offsets' buckets.
template <typename T, int HDP, TableForm kForm, int kTilesMax>
__global__ __launch_bounds__(64 * mha_waves(true, sizeof(T), HDP, 16 * kTilesMax), mha_per_simd(true, sizeof(T), HDP, 16 * kTilesMax)) void k_mha_backward(MhaArgs a) {
  constexpr int kMax = 16 * kTilesMax;
  __shared__ SetRows<kMax> sets[3][kMhaWavesMax];
  __shared__ int next_turn[8];
  const Share share(a);
  const int wave = threadIdx.x >> 6, range = share.group % a.ranges, h0 = share.group / a.ranges * a.hs, all = a.hs * a.entries;
  // entries of a head that this workgroup adds up: all, or its range of them (then hs = 1)
  const int per = (a.entries + a.ranges - 1) / a.ranges, lo = range * per, mine = lo + per < a.entries ? per : (a.entries > lo ? a.entries - lo : 0);
  float* table = reinterpret_cast<float*>(mha_lds + (a.partial ? a.hs * per : 0));
  uint16_t* map = reinterpret_cast<uint16_t*>(table + all);
  const int slot = wave / a.hs, hl = wave - slot * a.hs;
  const Head<T, HDP, kForm, kMax> head(a, table + hl * a.entries, map, h0 + hl);
  const Bins bins = {lds_address(mha_lds + hl * per) - (kForm == kInMemory ? 0u : 2 * lds_address(table + hl * a.entries)), 4u * lo, 4u * mine, range == 0};
  Turns turns = {(lds_turn*)(next_turn + hl), a.partial && a.slots > 1, a.slots, slot, (a.tau + 15) >> 4, 0};
  int round = 0;                                  // of `slots` sets, over all batches (a batch is a whole number of rounds)
  Lookup<kMax> lookup;
  // A batch is as many sets as there are wavefronts, each looked up by one, two batches ahead: beside this batch's sets where registers
  // allow it, else after them.
  constexpr bool kBeside = kTilesMax <= 3;
  const int waves = blockDim.x >> 6;
  const auto number = [&](int32_t batch, int b) { return share.part + (batch * waves + b) * a.parts; };       // a set's
  // (slots of sets past n_sets may be fetched, not used: their loads do not wait for n_sets, nor the tables' for them)
  Lookup<kMax> second;
  if (number(0, wave) < a.max_sets) lookup.slots(a, number(0, wave));
  if (number(1, wave) < a.max_sets) second.slots(a, number(1, wave));
  fill_tables<kForm>(a, h0, table, map);
  if (a.partial)
    for (int u = threadIdx.x; u < a.hs * per; u += blockDim.x) mha_lds[u] = 0.;
  if (threadIdx.x < 8) next_turn[threadIdx.x] = 0;
  const int32_t n_sets = sets_of(a);
  if (number(0, wave) < n_sets) lookup.cells(a);
  if (number(1, wave) < n_sets) second.cells(a);
  if (number(0, wave) < n_sets) lookup.rows(a, head.entry_bytes(), sets[0][wave]);
  if (number(1, wave) < n_sets) second.rows(a, head.entry_bytes(), sets[1][wave]);
  __syncthreads();
  Held<T, HDP, kMax> held;
  if (number(0, slot) < n_sets) held.fetch(head, sets[0][slot]);
  int now = 0;                                    // batch modulo 3
  for (int32_t batch = 0; number(batch, 0) < n_sets; ++batch) {
    const int after = now == 2 ? 0 : now + 1, last = after == 2 ? 0 : after + 1;
    const bool more = number(batch + 2, wave) < n_sets;
    if (kBeside && more) lookup.slots(a, number(batch + 2, wave));
    for (int b = slot; b < waves && number(batch, b - slot) < n_sets; b += a.slots, ++round) {
      turns.skip_to(round);
      const bool there = number(batch, b) < n_sets;
      const SetRows<kMax>& rows = sets[now][there ? b : b - slot];
      const int n = there ? __builtin_amdgcn_readfirstlane(rows.n) : 0;
      const SetRows<kMax>* next = b + a.slots < waves ? (number(batch, b + a.slots) < n_sets ? &sets[now][b + a.slots] : nullptr)
                                                      : (number(batch + 1, slot) < n_sets ? &sets[after][slot] : nullptr);
      switch ((n + 15) >> 4) {
        case 0: if (next) held.fetch(head, *next); break;
        case 1: backward_set<1>(head, rows, n, bins, turns, held, next); break;
        case 2: backward_set<2>(head, rows, n, bins, turns, held, next); break;
        case 3: backward_set<3>(head, rows, n, bins, turns, held, next); break;
        case 4: if constexpr (kTilesMax > 3) backward_set<4>(head, rows, n, bins, turns, held, next); break;
        case 5: if constexpr (kTilesMax > 3) backward_set<5>(head, rows, n, bins, turns, held, next); break;
        case 6: if constexpr (kTilesMax > 3) backward_set<6>(head, rows, n, bins, turns, held, next); break;
      }
      if (kBeside && b == slot && more) lookup.cells(a);
    }
    if (!kBeside && more) {
      lookup.slots(a, number(batch + 2, wave));
      lookup.cells(a);
    }
    if (more) lookup.rows(a, head.entry_bytes(), sets[last][wave]);
    turns.skip_to(round);                         // nobody waits for this wavefront at the barrier
    __syncthreads();
    now = after;
  }
  if (!a.partial) return;
  if (share.part < n_sets)                        // k_mha_entries reads the parts that had a set
    for (int u = threadIdx.x; u < a.hs * mine; u += blockDim.x)
      a.partial[((int64_t)share.part * a.heads + h0) * a.entries + lo + u] = (float)mha_lds[u];
}

template <typename T, int HDP, TableForm kForm, int kTilesMax> int launch(const MhaArgs& a, size_t lds, hipStream_t st) {
  static std::atomic<uint64_t> allowed;
  if (const int rc = dsvt_allow_lds(reinterpret_cast<const void*>(k_mha_backward<T, HDP, kForm, kTilesMax>), mha_lds_max(16 * kTilesMax, 1), allowed)) return rc;
  dsvt_prof_scope ps(DSVT_K_MHA_BACKWARD, st);
  k_mha_backward<T, HDP, kForm, kTilesMax><<<(unsigned)(a.groups * a.parts), 64 * a.hs * a.slots, lds, st>>>(a);
  return DSVT_OK;
}
template <typename T, int HDP> int launch(const MhaArgs& a, TableForm form, size_t lds, hipStream_t st) {
  if (a.tau <= 48)
    return form == kByOffset ? launch<T, HDP, kByOffset, 3>(a, lds, st) : form == kByBucket ? launch<T, HDP, kByBucket, 3>(a, lds, st)
                                                                                            : launch<T, HDP, kInMemory, 3>(a, lds, st);
  return form == kByOffset ? launch<T, HDP, kByOffset, 6>(a, lds, st) : form == kByBucket ? launch<T, HDP, kByBucket, 6>(a, lds, st)
                                                                                          : launch<T, HDP, kInMemory, 6>(a, lds, st);
}
template <typename T> int launch(const MhaArgs& a, TableForm form, size_t lds, hipStream_t st) {
  return a.hd <= 16 ? launch<T, 16>(a, form, lds, st) : a.hd <= 32 ? launch<T, 32>(a, form, lds, st) : launch<T, 64>(a, form, lds, st);
}

}  // namespace
