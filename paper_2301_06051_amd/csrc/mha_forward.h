// The forward kernel of dsvt_set_mha (see mha.h), for the two types' own files.
//
// Bound by latency: of a set's chain (rows, logits, probabilities, product), which four wavefronts a SIMD (128 registers) hide in part, and of
// the first look-ups.  C = 192, 8 heads, bf16: 30,000 voxels in sets of up to 36 take 16.5 us (46 MB: 2.8 TB/s; of a
// workgroup's 24 k clocks 7.4 k until its first sets), 120,000 in sets of up to 48 with 2,475 buckets 74 us (187 MB: 2.5 TB/s; 17 of 131 k).
#pragma once
#include "mha.h"

namespace {

// All of a set's rows of one head sit in registers: n voxels, kTiles tiles of 16.
template <int kTiles, typename T, int HDP, TableForm kForm, int kMax>
__device__ __forceinline__ void forward_set(const Head<T, HDP, kForm, kMax>& head, const SetRows<kMax>& rows, int n) {
  typedef Frag<T, HDP> F;
  const MhaArgs& a = head.a;
  const int m = head.m, g = head.g;
  typename F::Row k[kTiles][F::NC], v[kTiles][F::NC], q[F::NC], next[F::NC];
  typename F::Tile vt[kTiles][F::NT];
  head.load(rows, a.qkv, a.ld_qkv, 0, 0, q);
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    head.load(rows, a.qkv, a.ld_qkv, 1, t, k[t]);
    head.load(rows, a.qkv, a.ld_qkv, 2, t, v[t]);
  }
#pragma unroll
  for (int t = 0; t < kTiles; ++t) head.turn(v[t], vt[t]);
#pragma unroll 1
  for (int qt = 0; qt < kTiles; ++qt) {
    head.load(rows, a.qkv, a.ld_qkv, 0, qt + 1 < kTiles ? qt + 1 : qt, next);
    const uint32_t at = (uint32_t)rows.code[16 * qt + m] + head.from();
    head.clear_past_last(q);
    f32x4 p[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      uint32_t entry[4];
      head.entries(rows, at, t, entry);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[t][i] = head.value(entry[i]);
        if (t == kTiles - 1 && 16 * t + 4 * g + i >= n) p[t][i] = -INFINITY;
      }
#pragma unroll
      for (int c = 0; c < F::NC; ++c) p[t] = F::row_mma(k[t][c], q[c], p[t]);
    }
    const float sum = across_sum(head.template exponentials<kTiles>(rows, p));
    f32x4 o[F::NT] = {};
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int c = 0; c < F::NT; ++c) o[c] = F::tile_mma(vt[t][c], F::tile(p[t]), o[c]);
    head.store(rows, a.out, a.ld_out, 0, qt, 16 * qt + m < n, o, inverse(sum));
#pragma unroll
    for (int c = 0; c < F::NC; ++c) q[c] = next[c];
  }
}

template <typename T, int HDP, TableForm kForm, int kTilesMax>
__global__ __launch_bounds__(64 * mha_waves(false, sizeof(T), HDP, 16 * kTilesMax), mha_per_simd(false, sizeof(T), HDP, 16 * kTilesMax)) void k_mha_forward(MhaArgs a) {
  constexpr int kMax = 16 * kTilesMax;
  __shared__ SetRows<kMax> sets[2][kMhaWavesMax];
  const Share share(a);
  const int wave = threadIdx.x >> 6, h0 = share.group * a.hs;
  float* table = reinterpret_cast<float*>(mha_lds);
  uint16_t* map = reinterpret_cast<uint16_t*>(table + a.hs * a.entries);
  const int slot = wave / a.hs, hl = wave - slot * a.hs;
  const Head<T, HDP, kForm, kMax> head(a, table + hl * a.entries, map, h0 + hl);
  Lookup<kMax> lookup;
  // A batch is as many sets as there are wavefronts, each looked up by one.  The look-up of the next batch runs beside this one's sets where
  // registers allow it.
  constexpr bool kBeside = kTilesMax <= 3;
  const int waves = blockDim.x >> 6;
  const auto number = [&](int32_t batch, int b) { return share.part + (batch * waves + b) * a.parts; };       // a set's
  // (slots of sets past n_sets may be fetched, not used: their loads do not wait for n_sets, nor the tables' for them)
  if (number(0, wave) < a.max_sets) lookup.slots(a, number(0, wave));
  fill_tables<kForm>(a, h0, table, map);
  const int32_t n_sets = sets_of(a);
  const auto looks = [&](int32_t batch) { return number(batch, wave) < n_sets; };
  if (looks(0)) {
    lookup.cells(a);
    lookup.rows(a, head.entry_bytes(), sets[0][wave]);
  }
  for (int32_t batch = 0; number(batch, 0) < n_sets; ++batch) {
    __syncthreads();
    const bool more = looks(batch + 1);
    if (kBeside && more) lookup.slots(a, number(batch + 1, wave));
    for (int b = slot; b < waves && number(batch, b) < n_sets; b += a.slots) {
      const SetRows<kMax>& rows = sets[batch & 1][b];
      const int n = __builtin_amdgcn_readfirstlane(rows.n);
      switch ((n + 15) >> 4) {
        case 1: forward_set<1>(head, rows, n); break;
        case 2: forward_set<2>(head, rows, n); break;
        case 3: forward_set<3>(head, rows, n); break;
        case 4: if constexpr (kTilesMax > 3) forward_set<4>(head, rows, n); break;
        case 5: if constexpr (kTilesMax > 3) forward_set<5>(head, rows, n); break;
        case 6: if constexpr (kTilesMax > 3) forward_set<6>(head, rows, n); break;
      }
      if (kBeside && b == slot && more) lookup.cells(a);
    }
    if (!kBeside && more) {
      lookup.slots(a, number(batch + 1, wave));
      lookup.cells(a);
    }
    if (more) lookup.rows(a, head.entry_bytes(), sets[(batch + 1) & 1][wave]);
  }
}

template <typename T, int HDP, TableForm kForm, int kTilesMax> int launch(const MhaArgs& a, size_t lds, hipStream_t st) {
  static std::atomic<uint64_t> allowed;
  if (const int rc = dsvt_allow_lds(reinterpret_cast<const void*>(k_mha_forward<T, HDP, kForm, kTilesMax>), mha_lds_max(16 * kTilesMax, 1), allowed)) return rc;
  dsvt_prof_scope ps(DSVT_K_MHA_FORWARD, st);
  k_mha_forward<T, HDP, kForm, kTilesMax><<<(unsigned)(a.groups * a.parts), 64 * a.hs * a.slots, lds, st>>>(a);
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
