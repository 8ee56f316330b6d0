// dsvt_set_mha, dsvt_set_mha_backward, dsvt_rel_buckets: what the calls check and how they lay the work out (kernels: mha_forward.h,
// mha_backward.h; mathematics: mha.h), and the last step of the bias table's gradient.
#include "mha.h"

namespace {

constexpr int kComputeUnits = 256;                // MI355X

// The parts' sums of the table's gradient added in their order: 64 columns of [heads * entries] a workgroup, 16 slices of the parts.  Entries
// from n_out on (pairs without a bias) are dropped.
__global__ __launch_bounds__(1024) void k_mha_entries(const float* __restrict__ partial, const int32_t* __restrict__ n_sets, int32_t parts,
                                                      int32_t heads, int32_t entries, int32_t n_out, float* __restrict__ out) {
  __shared__ double s[16][64];
  const int32_t n = *n_sets < parts ? *n_sets : parts;       // parts without a set left no sums
  const int col = threadIdx.x & 63, slice = threadIdx.x >> 6;
  const int64_t cols = (int64_t)heads * entries, c = (int64_t)blockIdx.x * 64 + col;
  double v = 0.;
  if (c < cols) {
    int k = slice;
    for (; k + 7 * 16 < n; k += 8 * 16) {         // eight loads on their way at a time
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = partial[(k + j * 16) * cols + c];
#pragma unroll
      for (int j = 0; j < 8; ++j) v += (double)f[j];
    }
    for (; k < n; k += 16) v += (double)partial[k * cols + c];
  }
  s[slice][col] = v;
  __syncthreads();
  if (slice || c >= cols) return;
  v = 0.;
#pragma unroll
  for (int k = 0; k < 16; ++k) v += s[k][col];
  const int32_t h = (int32_t)(c / entries), u = (int32_t)(c - (int64_t)h * entries);
  if (u < n_out) out[(int64_t)h * n_out + u] = (float)v;
}

__global__ void k_mha_zero(float* __restrict__ p, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

struct Plan {
  TableForm form;
  int32_t hs, slots, ranges, parts, n_off, entries;
  size_t lds, ws;
};

int64_t offsets_of(const dsvt_mha_cfg* c) {
  return (2 * (int64_t)c->win[0] - 1) * (2 * (int64_t)c->win[1] - 1) * (2 * (int64_t)c->win[2] - 1);
}

// LDS of a workgroup of hs heads with its table in this form; bins: sums of this many entries a head.
size_t lds_bytes(TableForm form, int hs, int64_t bins, int64_t entries, int64_t n_off) {
  return (size_t)hs * bins * 8 + (form == kInMemory ? 0 : (size_t)hs * entries * 4) + (form == kByBucket ? dsvt_align_up((size_t)n_off * 2, 4) : 0);
}

int make_plan(const dsvt_mha_cfg* c, int32_t max_sets, int32_t tau, bool back, bool d_bias, Plan* p) {
  if (!c || c->C <= 0 || c->heads <= 0 || max_sets < 0 || tau <= 0) return DSVT_EINVAL;
  if (c->dtype != DSVT_F32 && c->dtype != DSVT_BF16) return DSVT_EINVAL;
  if (c->dup_mode != 0 && c->dup_mode != 1) return DSVT_EINVAL;
  if (c->C % c->heads != 0) return DSVT_EINVAL;
  for (int i = 0; i < 3; ++i) if (c->win[i] <= 0 || c->win[i] > 4096) return DSVT_EINVAL;
  if (c->rel_bias && c->n_rel <= 0) return DSVT_EINVAL;
  const int64_t n_off = c->rel_bias ? offsets_of(c) : 1;
  if (c->rel_bias && !c->rel_bucket && c->n_rel != n_off) return DSVT_EINVAL;
  if (d_bias && !c->rel_bias) return DSVT_EINVAL;
  const int hd = c->C / c->heads;
  if (hd % 8 != 0 || hd > 64 || tau > kSetMax || n_off >= (1 << 24) || (c->rel_bias && c->n_rel >= (1 << 24))) return DSVT_EUNSUPPORTED;
  const bool by_bucket = c->rel_bias && c->rel_bucket;
  const int element = c->dtype == DSVT_BF16 ? 2 : 4, padded = hd <= 16 ? 16 : hd <= 32 ? 32 : 64;
  const int waves = mha_waves(back, element, padded, tau);
  int per_cu = mha_per_cu(back, element, padded, tau);
  // In LDS if it fits there for one head, for as many heads as fit: heads of one set in one workgroup share cache lines.  (Buckets could also be
  // summed up by offset and folded afterwards: 30,000 pillars, 81 buckets, backward 38.9 us where by bucket takes 37.3, 2,000 voxels 19.6
  // and 17.1; two lookups a pair cost less than larger tables and one more kernel.)
  p->hs = 0;
  p->form = by_bucket ? kByBucket : kByOffset;
  const int64_t entries = by_bucket ? (int64_t)c->n_rel + 1 : n_off;
  const auto most_heads = [&](size_t most) {
    int hs = 0;
    for (int h = 1; h <= waves; ++h)
      if (c->heads % h == 0 && lds_bytes(p->form, h, d_bias ? entries : 0, entries, n_off) <= most) hs = h;
    return hs;
  };
  if (by_bucket && c->n_rel > 65535) p->form = kInMemory;
  p->hs = most_heads(mha_lds_max(tau, per_cu));
  if (p->hs == 0) p->hs = most_heads(mha_lds_max(tau, 1));      // (one workgroup a compute unit after all, see below)
  if (p->hs == 0) {
    p->form = kInMemory;
    p->hs = most_heads(mha_lds_max(tau, 1));
  }
  p->entries = (int32_t)entries;
  // Sums that the LDS of a workgroup does not hold for one head: workgroups of a head share its entries, and each goes through all sets.
  p->ranges = 1;
  if (p->hs == 0) {
    p->hs = 1;
    p->ranges = (int32_t)dsvt_ceil_div((int64_t)p->entries * 8, mha_lds_max(tau, 1));
  }
  p->n_off = (int32_t)n_off;
  p->lds = lds_bytes(p->form, p->hs, d_bias ? dsvt_ceil_div(p->entries, p->ranges) : 0, p->entries, n_off);
  // (120,000 voxels, 12 x 12 x 32 windows with an entry an offset, 133 KB: forward 92 us, 99 with workgroups for two a compute unit)
  if (p->lds > mha_lds_max(tau, per_cu)) per_cu = 1;
  p->slots = 1;
  while (2 * p->slots * p->hs <= waves) p->slots *= 2;
  // Parts by eights (see Share), and no more workgroups than fit the chip at once: one part too many is a second round of all of them.
  // (120,000 voxels, 24 heads of 16, three groups: backward 248 us, 403 rounded up.)  At least eight; one a set where there are fewer sets.
  const int64_t fit = kComputeUnits * per_cu / (c->heads / p->hs * p->ranges) / 8 * 8, parts = fit > 8 ? fit : 8;
  const int64_t sets = (int64_t)dsvt_align_up((size_t)(max_sets > 0 ? max_sets : 1), 8);
  p->parts = (int32_t)(parts < sets ? parts : sets);
  p->ws = d_bias ? (size_t)p->parts * c->heads * (size_t)p->entries * 4 : 0;
  return DSVT_OK;
}

bool bad_rows(const void* p, int64_t ld, int64_t width, int e) {
  return !p || ((uintptr_t)p & 15u) != 0 || ld < width || ld > UINT32_MAX / e || (ld * e) % 16 != 0;
}

// Whether two arrays of n rows share a byte (strides and widths in bytes).  Rows of one stride may lie between each other, as slices of a
// wider array do; of two strides the arrays have to lie apart as a whole.
bool overlap(const void* p, int64_t ld_p, int64_t w_p, const void* q, int64_t ld_q, int64_t w_q, int32_t n) {
  const uint64_t a = (uintptr_t)p, b = (uintptr_t)q;
  if (a + (uint64_t)(n - 1) * ld_p + w_p <= b || b + (uint64_t)(n - 1) * ld_q + w_q <= a) return false;
  if (ld_p != ld_q) return true;
  // row j of q begins d + (j - i) ld behind row i of p: r behind the one that begins before it, ld - r before the next
  const int64_t d = (int64_t)(b - a), ld = ld_p, r = (d % ld + ld) % ld, k = (r - d) / ld;
  return (r < w_p && k < n && k > -n) || (ld - r < w_q && k - 1 < n && k - 1 > -n);
}

int check_maps(const dsvt_maps* maps) {
  if (!maps || maps->n_voxels < 0 || maps->max_sets < 0 || maps->max_sets > (1 << 30) || maps->tau <= 0) return DSVT_EINVAL;
  if (maps->n_voxels > 0 && (!maps->set_inds || !maps->n_sets)) return DSVT_EINVAL;
  return DSVT_OK;
}

MhaArgs make_args(const dsvt_mha_cfg* c, const dsvt_maps* maps, const int32_t* coords, const Plan& p) {
  MhaArgs a = {};
  a.set_inds = maps->set_inds; a.n_sets = maps->n_sets; a.coords = reinterpret_cast<const int4*>(coords);
  a.bias = c->rel_bias; a.bucket = c->rel_bias ? c->rel_bucket : nullptr;
  a.n_voxels = maps->n_voxels; a.max_sets = maps->max_sets; a.tau = maps->tau; a.heads = c->heads; a.hd = c->C / c->heads;
  a.n_off = p.n_off; a.n_rel = c->rel_bias ? c->n_rel : 0; a.entries = p.entries;
  for (int i = 0; i < 3; ++i) a.w[i] = c->win[i];
  a.centre = c->rel_bias ? ((c->win[0] - 1) * (2 * c->win[1] - 1) + c->win[1] - 1) * (2 * c->win[2] - 1) + c->win[2] - 1 : 0;
  a.dup = c->dup_mode; a.hs = p.hs; a.slots = p.slots; a.groups = c->heads / p.hs * p.ranges; a.ranges = p.ranges; a.parts = p.parts;
  a.scale = 1.f / sqrtf((float)a.hd);
  return a;
}

}  // namespace

extern "C" int dsvt_rel_buckets(const int32_t win[3], int32_t n_exact, int32_t n_side, int32_t* bucket, int32_t* n_rel) {
  if (!win || !n_rel || n_exact <= 0 || n_side < n_exact) return DSVT_EINVAL;
  int64_t total = 1, offsets = 1, most[3];
  for (int i = 0; i < 3; ++i) {
    if (win[i] <= 0 || win[i] > 4096) return DSVT_EINVAL;
    most[i] = n_side < win[i] ? n_side : win[i];
    total *= 2 * most[i] - 1;
    offsets *= 2 * (int64_t)win[i] - 1;
  }
  if (offsets >= (1 << 24)) return DSVT_EUNSUPPORTED;
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
  if (overlap(out, ld_out * e, (int64_t)cfg->C * e, qkv, ld_qkv * e, 3 * (int64_t)cfg->C * e, maps->n_voxels)) return DSVT_EINVAL;
  MhaArgs a = make_args(cfg, maps, coords, p);
  a.qkv = qkv; a.ld_qkv = (uint32_t)(ld_qkv * e); a.out = out; a.ld_out = (uint32_t)(ld_out * e);
  hipStream_t st = (hipStream_t)stream;
  if (const int rc = cfg->dtype == DSVT_BF16 ? mha_forward_bf16(a, p.form, p.lds, st) : mha_forward_f32(a, p.form, p.lds, st)) return rc;
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
  // (rows are read ahead, read again, and read by workgroups that do not write them)
  if (overlap(d_qkv, ld_dqkv * e, 3 * C * e, qkv, ld_qkv * e, 3 * C * e, maps->n_voxels) ||
      overlap(d_qkv, ld_dqkv * e, 3 * C * e, d_out, ld_dout * e, C * e, maps->n_voxels)) return DSVT_EINVAL;
  MhaArgs a = make_args(cfg, maps, coords, p);
  a.qkv = qkv; a.ld_qkv = (uint32_t)(ld_qkv * e); a.d_out = d_out; a.ld_dout = (uint32_t)(ld_dout * e); a.out = d_qkv; a.ld_out = (uint32_t)(ld_dqkv * e);
  a.partial = d_rel_bias ? static_cast<float*>(ws) : nullptr;
  if (const int rc = cfg->dtype == DSVT_BF16 ? mha_backward_bf16(a, p.form, p.lds, st) : mha_backward_f32(a, p.form, p.lds, st)) return rc;
  if (d_rel_bias) {
    const int64_t cols = (int64_t)cfg->heads * p.entries;
    dsvt_prof_scope ps(DSVT_K_MHA_REL, st);
    k_mha_entries<<<(unsigned)dsvt_ceil_div(cols, 64), 1024, 0, st>>>(a.partial, maps->n_sets, p.parts < maps->max_sets ? p.parts : maps->max_sets, cfg->heads,
                                                                     p.entries, cfg->n_rel, d_rel_bias);
  }
  DSVT_HIP_TRY(hipGetLastError());
  return DSVT_OK;
}
