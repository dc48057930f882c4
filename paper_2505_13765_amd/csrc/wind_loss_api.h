// Host side of the losses over the output layer: argument checks, workspace, launches.  Included by wind_api.hip.
#pragma once
#include "wind_loss_lattice.h"

namespace {

using LossBig = LossTile<4, 4, 5>;     // 256 x 256 outputs, one workgroup per CU
using LossMid = LossTile<2, 2, 4>;     // 128 x 128
using LossSmall = LossTile<1, 1, 4>;   // 64 x 64

constexpr size_t kLossChunkBytes = 512u << 20;   // dx and rows of a chunk, about
constexpr int kLossMaxEntries = 1024;

// the bf16 planes that make up a stored value of each type, and the sum of two bf16 values (hidden rows of the lattice)
int loss_planes(int dtype) { return dtype == WIND_BF16 ? 1 : 3; }
int lattice_planes(int dtype) { return dtype == WIND_BF16 ? 2 : 3; }

SegmentsDev loss_segments(int pa, int pb) {
  SegmentsDev s{0, 0};
  for (int sum = std::max(pa, pb) - 1; sum >= 0; --sum)
    for (int i = 0; i < pa; ++i) {
      const int j = sum - i;
      if (j < 0 || j >= pb) continue;
      s.list |= (uint32_t)(i | (j << 2)) << (4 * s.n);
      ++s.n;
    }
  return s;
}

// Tile of a product of m x n outputs: the largest whose tiles still reach every CU.
int loss_tile_size(long long m, long long n) {
  auto tiles = [&](int t) { return ((m + t - 1) / t) * ((n + t - 1) / t); };
  return tiles(256) >= 256 ? 256 : tiles(128) >= 256 ? 128 : 64;
}
int loss_tile_cols(int tile) { return tile / 2; }   // columns of a wave's block

struct LossPlan {
  int kind, dtype, V1, H, K;
  long long N;                       // rows at most
  bool grads;
  int B, T, U;                       // lattice
  // derived
  int R, chunks, vblk, hblk, hd, pa, pw, pd;
  int tile_x, tile_z, tile_w, splits;
  // offsets into the workspace
  size_t idx, count, w, rows, label, value, coef, scale, lse2, logit, part, dx, colsum, dw, total;
  size_t off, tb, ub, from, nblank, nlabel, nlse2, alpha, beta, dz, de, dp;
};

void loss_plan(LossPlan &p) {
  p.vblk = (p.V1 + 31) / 32;
  p.hblk = (p.H + 31) / 32;
  p.hd = (p.H + 3) / 4 * 4;
  p.pw = p.pd = loss_planes(p.dtype);
  p.pa = p.kind == kLossLattice ? lattice_planes(p.dtype) : loss_planes(p.dtype);
  const size_t row = (size_t)p.pa * p.hblk * 64 + (p.grads ? (size_t)p.pd * p.vblk * 64 : 0) + (p.kind == kLossLattice && p.grads ? (size_t)p.hd * 4 : 0);
  const long long N = std::max(p.N, 1ll);
  const long long most = std::max<long long>((long long)(kLossChunkBytes / row) / 256 * 256, 256);
  p.chunks = (int)((N + most - 1) / most);
  p.R = (int)round_up((size_t)((N + p.chunks - 1) / p.chunks), 256);
  p.chunks = (int)((N + p.R - 1) / p.R);
  p.tile_x = loss_tile_size(std::min<long long>(p.R, N), p.V1);
  p.tile_z = loss_tile_size(std::min<long long>(p.R, N), p.H);
  p.tile_w = loss_tile_size((long long)p.V1 * 4, p.H);
  const long long tiles = ((p.V1 + p.tile_w - 1) / p.tile_w) * (long long)((p.H + p.tile_w - 1) / p.tile_w);
  p.splits = (int)std::max<long long>(1, std::min<long long>((p.tile_w == 256 ? 256 : 512) / tiles, p.R / 256));
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += round_up(bytes, 256);
    return here;
  };
  const size_t R = (size_t)p.R, n = (size_t)N;
  p.count = take(4);
  p.w = take((size_t)p.pw * p.vblk * 32 * p.hblk * 64);
  p.rows = take((size_t)p.pa * R * p.hblk * 64);
  p.label = take(R * p.K * 4);
  p.logit = take(R * p.K * 4);
  p.coef = take(R * p.K * 4);
  p.scale = take(R * 4);
  p.lse2 = take(R * 4);
  p.part = take(R * 8 * ((p.V1 + loss_tile_cols(p.tile_x) - 1) / loss_tile_cols(p.tile_x)));
  if (p.kind != kLossLattice) p.idx = take(n * 4);
  if (p.kind == kLossDistill) p.value = take(R * p.K * 4);
  if (p.kind == kLossLattice) {
    p.off = take(((size_t)p.B + 1) * 4);
    p.tb = take((size_t)p.B * 4);
    p.ub = take((size_t)p.B * 4);
    p.from = take(R * 8);
    p.nblank = take(n * 4);
    p.nlabel = take(n * 4);
    p.nlse2 = take(n * 4);
  }
  if (p.grads) {
    p.dx = take((size_t)p.pd * R * p.vblk * 64);
    p.colsum = take(2 * ((R + p.tile_x - 1) / p.tile_x) * p.vblk * 128);
    p.dw = take((size_t)p.splits * p.V1 * p.hd * 4);
    if (p.kind == kLossLattice) {
      p.alpha = take(n * 8);
      p.beta = take(n * 8);
      p.dz = take(R * p.hd * 4);
      p.de = take((size_t)p.B * p.T * p.hd * 4);
      p.dp = take((size_t)p.B * (p.U + 1) * p.hd * 4);
    }
  }
  p.total = at;
}

int loss_layer_check(const wind_output_layer *l) {
  if (!l || !l->w) return fail(WIND_ERR_ARG, "null argument");
  if (l->V1 < 2 || l->H < 1) return fail(WIND_ERR_ARG, "V1 >= 2 and H >= 1 required");
  if (l->dtype != WIND_F32 && l->dtype != WIND_BF16) return fail(WIND_ERR_ARG, "dtype must be WIND_F32 or WIND_BF16");
  if (l->w_stride < l->H) return fail(WIND_ERR_ARG, "w_stride must be at least H");
  if ((uintptr_t)l->w % (l->dtype ? 2 : 4) || (uintptr_t)l->b % 4) return fail(WIND_ERR_ARG, "w or b is not aligned to its type");
  if ((long long)((l->V1 + 31) / 32 * 32) * ((l->H + 31) / 32 * 32) >= 1ll << 31) return fail(WIND_ERR_UNSUPPORTED, "V1 * H must be below 2^31");
  return WIND_OK;
}
int loss_workspace_check(const LossPlan &p, const void *ws, size_t bytes) {
  if (!ws) return fail(WIND_ERR_ARG, "workspace is null");
  if ((uintptr_t)ws % 256) return fail(WIND_ERR_ARG, "workspace must be 256-byte aligned");
  if (bytes < p.total)
    return fail(WIND_ERR_ARG, "workspace of " + std::to_string(bytes) + " bytes is too small: this call needs " + std::to_string(p.total));
  return WIND_OK;
}
int loss_rows_limits(const LossPlan &p) {
  if (p.K > kLossMaxEntries) return fail(WIND_ERR_UNSUPPORTED, "K must be at most 1024");
  if ((unsigned long long)p.R * std::max(p.vblk, p.hblk) * 64 >= 1ull << 32) return fail(WIND_ERR_UNSUPPORTED, "V1 and H must be below 2^24");
  return WIND_OK;
}

unsigned loss_blocks(size_t items, size_t per = 256, size_t most = 4096) { return (unsigned)std::max<size_t>(1, std::min(most, (items + per - 1) / per)); }
unsigned loss_grid(long long rt, long long ct) { return (unsigned)((rt * ct + 7) / 8 * 8); }

template <class F>
void loss_with_tile(int tile, F &&f) {
  if (tile == 256) f(LossBig{});
  else if (tile == 128) f(LossMid{});
  else f(LossSmall{});
}

struct LossRun {                     // what the launches of one call share
  LossPlan p;
  char *ws;
  hipStream_t s;
  const wind_output_layer *layer;
  LossRowsDev rows;
  LossChunk chunk;
  PanelsDev w, x;
  template <class U>
  U *at(size_t offset) const { return reinterpret_cast<U *>(ws + offset); }
};

void loss_begin(LossRun &r) {
  const LossPlan &p = r.p;
  r.w = PanelsDev{r.at<bf16_t>(p.w), (size_t)p.vblk * 32 * p.hblk * 32, (uint32_t)p.vblk * 32, (uint32_t)p.hblk};
  r.x = PanelsDev{r.at<bf16_t>(p.rows), (size_t)p.R * p.hblk * 32, (uint32_t)p.R, (uint32_t)p.hblk};
  LossChunk &k = r.chunk;
  k.R = p.R;
  k.count = r.at<int>(p.count);
  k.K = p.K;
  k.label = r.at<int>(p.label);
  k.value = p.kind == kLossDistill ? r.at<float>(p.value) : nullptr;
  k.coef = r.at<float>(p.coef);
  k.scale = r.at<float>(p.scale);
  k.lse2 = r.at<float>(p.lse2);
  k.logit = r.at<float>(p.logit);
  k.part = r.at<float2>(p.part);
  k.c = kLog2e * r.rows.inv_tau;
  const wind_output_layer &l = *r.layer;
  LossPack w{};
  w.src = l.w;
  w.stride = (size_t)l.w_stride;
  w.dtype = l.dtype;
  w.rows = l.V1;
  w.cols = l.H;
  w.dst = r.at<bf16_t>(p.w);
  w.plane = r.w.plane;
  w.dst_rows = p.vblk * 32;
  w.blocks = p.hblk;
  w.planes = p.pw;
  w.vec = (uintptr_t)l.w % 16 == 0 && l.w_stride % 8 == 0;
  loss_pack_kernel<<<loss_blocks((size_t)w.dst_rows * p.hblk * 4), 256, 0, r.s>>>(w);
}

LossProduct loss_logits(const LossRun &r) {
  const LossPlan &p = r.p;
  return LossProduct{r.x, r.w, loss_segments(p.pa, p.pw), p.hblk, p.V1, (p.V1 + p.tile_x - 1) / p.tile_x, 8};
}
void loss_stats(const LossRun &r, LossNodes nodes) {
  const LossPlan &p = r.p;
  const LossProduct g = loss_logits(r);
  loss_with_tile(p.tile_x, [&](auto t) {
    using T = decltype(t);
    loss_stats_kernel<T><<<loss_grid((p.R + T::BM - 1) / T::BM, g.ct), 256, 0, r.s>>>(g, r.chunk, r.layer->b);
  });
  loss_rows_done_kernel<<<p.R / 64, 256, 0, r.s>>>(r.rows, r.chunk, (p.V1 + loss_tile_cols(p.tile_x) - 1) / loss_tile_cols(p.tile_x), nodes);
}
// dx and what follows from it
void loss_gradients(const LossRun &r, LossOut *dz, bool dw, float *db, bool add) {
  const LossPlan &p = r.p;
  const LossProduct g = loss_logits(r);
  const LossDx d{r.at<bf16_t>(p.dx), (size_t)p.R * p.vblk * 32, p.pd, p.vblk, db ? r.at<float>(p.colsum) : nullptr};
  loss_with_tile(p.tile_x, [&](auto t) {
    using T = decltype(t);
    loss_dx_kernel<T><<<loss_grid((p.R + T::BM - 1) / T::BM, g.ct), 256, 0, r.s>>>(g, r.chunk, r.layer->b, d);
  });
  if (db)
    loss_db_kernel<<<(p.V1 + 63) / 64, 1024, 0, r.s>>>(d.colsum, p.vblk * 32, p.V1, p.tile_x, r.chunk, add, db);
  const PanelsDev dx{d.dx, d.plane, (uint32_t)p.R, (uint32_t)p.vblk};
  if (dz) {
    const LossProduct q{dx, r.w, loss_segments(p.pd, p.pw), p.vblk, p.H, (p.H + p.tile_z - 1) / p.tile_z, 8};
    loss_with_tile(p.tile_z, [&](auto t) {
      using T = decltype(t);
      loss_dz_kernel<T><<<loss_grid((p.R + T::BM - 1) / T::BM, q.ct), 256, 0, r.s>>>(q, r.chunk, *dz);
    });
  }
  if (dw) {
    const LossProduct q{dx, r.x, loss_segments(p.pd, p.pw), 0, p.V1, (p.H + p.tile_w - 1) / p.tile_w, 8};
    const int rt = (p.V1 + p.tile_w - 1) / p.tile_w;
    const LossOut o{r.at<float>(p.dw), (size_t)p.hd, 0, p.H, 1, nullptr, nullptr, 0, add};
    loss_with_tile(p.tile_w, [&](auto t) {
      using T = decltype(t);
      loss_dw_kernel<T><<<loss_grid(rt, q.ct) * p.splits, 256, 0, r.s>>>(q, r.chunk, o, rt, p.splits, (size_t)p.V1 * p.hd);
    });
  }
}
void loss_dw_done(const LossRun &r, void *dw) {
  const LossPlan &p = r.p;
  loss_dw_done_kernel<<<loss_blocks((size_t)p.V1 * (p.hd / 4)), 256, 0, r.s>>>(r.at<float>(p.dw), p.splits, (size_t)p.V1 * p.hd, (size_t)p.hd, p.V1, p.H,
                                                                            p.dtype, dw);
}

int loss_rows_call(const char *name, const wind_output_layer *layer, const void *h, long long h_stride, LossRowsDev rows, long long N, void *dh, void *dw,
                   float *db, void *workspace, size_t workspace_bytes, hipStream_t s) {
  LossRun r{};
  r.p.kind = rows.kind;
  r.p.dtype = layer->dtype;
  r.p.V1 = layer->V1;
  r.p.H = layer->H;
  r.p.K = rows.K;
  r.p.N = N;
  r.p.grads = dh || dw || db;
  loss_plan(r.p);
  int rc = loss_rows_limits(r.p);
  if (rc == WIND_OK) rc = loss_workspace_check(r.p, workspace, workspace_bytes);
  if (rc) return rc;
  const LossPlan &p = r.p;
  r.ws = (char *)workspace;
  r.s = s;
  r.layer = layer;
  rows.N = (int)N;
  rows.V1 = layer->V1;
  rows.idx = r.at<int>(p.idx);
  rows.count = r.at<int>(p.count);
  r.rows = rows;
  loss_rows_kernel<<<1, 1024, 0, s>>>(rows);
  if (dh && N) loss_zero_rows_kernel<<<(unsigned)((N + 3) / 4), 256, 0, s>>>(rows, dh, p.dtype, p.H);
  loss_begin(r);
  LossPack k{};
  k.src = h;
  k.stride = (size_t)h_stride;
  k.dtype = p.dtype;
  k.cols = p.H;
  k.idx = rows.idx;
  k.count = rows.count;
  k.dst = r.at<bf16_t>(p.rows);
  k.plane = r.x.plane;
  k.dst_rows = p.R;
  k.blocks = p.hblk;
  k.planes = p.pa;
  k.vec = (uintptr_t)h % 16 == 0 && h_stride % 8 == 0;
  LossOut dz{dh, (size_t)p.H, p.dtype, p.H, dh && (uintptr_t)dh % 16 == 0 && p.H % 4 == 0, nullptr, nullptr, 0, 0};
  for (int c = 0; c < p.chunks; ++c) {
    k.c0 = r.chunk.c0 = c * p.R;
    loss_pack_kernel<<<loss_blocks((size_t)p.R * p.hblk * 4), 256, 0, s>>>(k);
    loss_entries_kernel<<<p.R / 256, 256, 0, s>>>(rows, r.chunk);
    loss_stats(r, LossNodes{});
    if (!p.grads) continue;
    dz.idx = rows.idx + k.c0;
    loss_gradients(r, dh ? &dz : nullptr, dw != nullptr, db, c > 0);
  }
  if (dw) loss_dw_done(r, dw);
  return check_launch(name);
}

int loss_rows_check(const wind_output_layer *layer, const void *h, long long h_stride, const int32_t *labels, long long N, const float *loss, const void *dh,
                    const void *dw) {
  int rc = loss_layer_check(layer);
  if (rc) return rc;
  if (N < 0 || N >= 1ll << 31) return fail(WIND_ERR_ARG, "0 <= N < 2^31 required");
  if (N && (!h || !labels || !loss)) return fail(WIND_ERR_ARG, "null argument");
  if (h_stride < layer->H) return fail(WIND_ERR_ARG, "h_stride must be at least H");
  const uintptr_t size = layer->dtype ? 2 : 4;
  if ((uintptr_t)h % size || (uintptr_t)dh % size || (uintptr_t)dw % size) return fail(WIND_ERR_ARG, "a pointer is not aligned to its type");
  return WIND_OK;
}

int lattice_plan(LossPlan &p, const wind_output_layer *layer, int B, int T, int U, bool grads) {
  int rc = loss_layer_check(layer);
  if (rc) return rc;
  if (B < 1 || T < 0 || U < 0) return fail(WIND_ERR_ARG, "B >= 1, T >= 0 and U >= 0 required");
  if (U > 4095) return fail(WIND_ERR_UNSUPPORTED, "U must be at most 4095");
  if ((double)B * T * (U + 1.0) >= 2147483648.0) return fail(WIND_ERR_UNSUPPORTED, "B * T * (U + 1) must be below 2^31");
  p.kind = kLossLattice;
  p.dtype = layer->dtype;
  p.V1 = layer->V1;
  p.H = layer->H;
  p.K = 2;
  p.B = B;
  p.T = T;
  p.U = U;
  p.N = (long long)B * T * (U + 1);
  p.grads = grads;
  loss_plan(p);
  return loss_rows_limits(p);
}

}  // namespace

extern "C" {

int wind_row_loss_workspace_bytes(const wind_output_layer *layer, int64_t N, int K, int grads, size_t *bytes) try {
  if (!bytes) return fail(WIND_ERR_ARG, "null argument");
  int rc = loss_layer_check(layer);
  if (rc) return rc;
  if (N < 0 || N >= 1ll << 31 || K < 1) return fail(WIND_ERR_ARG, "0 <= N < 2^31 and K >= 1 required");
  LossPlan p{};
  p.kind = kLossDistill;   // the larger of the two
  p.dtype = layer->dtype;
  p.V1 = layer->V1;
  p.H = layer->H;
  p.K = K;
  p.N = N;
  p.grads = grads != 0;
  loss_plan(p);
  rc = loss_rows_limits(p);
  if (rc) return rc;
  *bytes = p.total;
  return WIND_OK;
} catch (const std::exception &e) {
  return fail(WIND_ERR_HIP, std::string("wind_row_loss_workspace_bytes: ") + e.what());
}

int wind_label_loss(const wind_output_layer *layer, const void *h, int64_t h_stride, const int32_t *labels, const float *weights, int64_t N, float *loss,
                    void *dh, void *dw, float *db, void *workspace, size_t workspace_bytes, void *stream) try {
  int rc = loss_rows_check(layer, h, h_stride, labels, N, loss, dh, dw);
  if (rc) return rc;
  LossRowsDev rows{};
  rows.kind = kLossLabel;
  rows.K = 1;
  rows.labels = labels;
  rows.weights = weights;
  rows.tau = rows.inv_tau = 1.f;
  rows.loss = loss;
  return loss_rows_call("label loss", layer, h, h_stride, rows, N, dh, dw, db, workspace, workspace_bytes, (hipStream_t)stream);
} catch (const std::exception &e) {
  return fail(WIND_ERR_HIP, std::string("wind_label_loss: ") + e.what());
}

int wind_distill_loss(const wind_output_layer *layer, const void *h, int64_t h_stride, const int32_t *teacher_labels, const float *teacher_logits, int K,
                      float temperature, const float *weights, int64_t N, float *loss, void *dh, void *dw, float *db, void *workspace,
                      size_t workspace_bytes, void *stream) try {
  int rc = loss_rows_check(layer, h, h_stride, teacher_labels, N, loss, dh, dw);
  if (rc) return rc;
  if (N && !teacher_logits) return fail(WIND_ERR_ARG, "null argument");
  if (K < 1) return fail(WIND_ERR_ARG, "K >= 1 required");
  if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(1.f / temperature))
    return fail(WIND_ERR_ARG, "temperature must be positive and finite");
  LossRowsDev rows{};
  rows.kind = kLossDistill;
  rows.K = K;
  rows.labels = teacher_labels;
  rows.logits = teacher_logits;
  rows.weights = weights;
  rows.tau = temperature;
  rows.inv_tau = 1.f / temperature;
  rows.loss = loss;
  return loss_rows_call("distillation loss", layer, h, h_stride, rows, N, dh, dw, db, workspace, workspace_bytes, (hipStream_t)stream);
} catch (const std::exception &e) {
  return fail(WIND_ERR_HIP, std::string("wind_distill_loss: ") + e.what());
}

int wind_transducer_loss_workspace_bytes(const wind_output_layer *layer, int B, int T, int U, int grads, size_t *bytes) try {
  if (!bytes) return fail(WIND_ERR_ARG, "null argument");
  LossPlan p{};
  const int rc = lattice_plan(p, layer, B, T, U, grads != 0);
  if (rc) return rc;
  *bytes = p.total;
  return WIND_OK;
} catch (const std::exception &e) {
  return fail(WIND_ERR_HIP, std::string("wind_transducer_loss_workspace_bytes: ") + e.what());
}

int wind_transducer_loss(const wind_output_layer *layer, const void *e, int64_t e_stride_b, int64_t e_stride_t, const void *p_, int64_t p_stride_b,
                         int64_t p_stride_u, const int32_t *labels, const int32_t *frames, const int32_t *label_counts, const float *weights, int B, int T,
                         int U, float *loss, void *de, void *dp, void *dw, float *db, void *workspace, size_t workspace_bytes, void *stream) try {
  LossRun r{};
  int rc = lattice_plan(r.p, layer, B, T, U, de || dp || dw || db);
  if (rc) return rc;
  if ((T && !e) || !p_ || (U && !labels) || !frames || !label_counts || !loss) return fail(WIND_ERR_ARG, "null argument");
  if (e_stride_t < 0 || e_stride_b < 0 || p_stride_u < 0 || p_stride_b < 0) return fail(WIND_ERR_ARG, "strides must not be negative");
  const uintptr_t size = layer->dtype ? 2 : 4;
  if ((uintptr_t)e % size || (uintptr_t)p_ % size || (uintptr_t)de % size || (uintptr_t)dp % size || (uintptr_t)dw % size)
    return fail(WIND_ERR_ARG, "a pointer is not aligned to its type");
  rc = loss_workspace_check(r.p, workspace, workspace_bytes);
  if (rc) return rc;
  const LossPlan &p = r.p;
  hipStream_t s = (hipStream_t)stream;
  r.ws = (char *)workspace;
  r.s = s;
  r.layer = layer;
  r.rows.kind = kLossLattice;
  r.rows.tau = r.rows.inv_tau = 1.f;
  LatticeDev l{};
  l.B = B;
  l.T = T;
  l.U = U;
  l.V1 = p.V1;
  l.H = p.H;
  l.dtype = p.dtype;
  l.e = e;
  l.p = p_;
  l.e_b = e_stride_b;
  l.e_t = e_stride_t;
  l.p_b = p_stride_b;
  l.p_u = p_stride_u;
  l.labels = labels;
  l.frames = frames;
  l.counts = label_counts;
  l.weights = weights;
  l.loss = loss;
  l.off = r.at<int>(p.off);
  l.tb = r.at<int>(p.tb);
  l.ub = r.at<int>(p.ub);
  l.count = r.at<int>(p.count);
  l.nodes = LossNodes{r.at<float>(p.nblank), r.at<float>(p.nlabel), r.at<float>(p.nlse2)};
  if (p.grads) {
    l.alpha = r.at<float2>(p.alpha);
    l.beta = r.at<float2>(p.beta);
  }
  lattice_rows_kernel<<<1, 1024, 0, s>>>(l);
  loss_begin(r);
  int2 *from = r.at<int2>(p.from);
  const int vec = (uintptr_t)e % 16 == 0 && (uintptr_t)p_ % 16 == 0 && e_stride_b % 8 == 0 && e_stride_t % 8 == 0 && p_stride_b % 8 == 0 && p_stride_u % 8 == 0;
  auto rows_of_chunk = [&](int c, int grad) {
    r.chunk.c0 = c * p.R;
    lattice_entries_kernel<<<p.R / 256, 256, 0, s>>>(l, r.chunk, from, grad);
    lattice_z_kernel<<<loss_blocks((size_t)p.R * p.hblk * 4), 256, 0, s>>>(l, r.chunk, from, r.at<bf16_t>(p.rows), r.x.plane, p.hblk, p.pa, vec);
  };
  for (int c = 0; c < p.chunks; ++c) {
    rows_of_chunk(c, 0);
    loss_stats(r, l.nodes);
  }
  const int both = p.grads, lanes = U + 1;
  if (lanes <= 1024) lattice_sums_kernel<1, 8><<<B << both, (unsigned)round_up((size_t)lanes, 64), 0, s>>>(l, both);
  else if (lanes <= 2048) lattice_sums_kernel<2, 4><<<B << both, (unsigned)round_up((size_t)(lanes + 1) / 2, 64), 0, s>>>(l, both);
  else lattice_sums_kernel<4, 2><<<B << both, (unsigned)round_up((size_t)(lanes + 3) / 4, 64), 0, s>>>(l, both);
  if (p.grads) {
    float *dz = r.at<float>(p.dz), *de32 = r.at<float>(p.de), *dp32 = r.at<float>(p.dp);
    LossOut o{dz, (size_t)p.hd, 0, p.H, 1, nullptr, r.at<bf16_t>(p.rows), (size_t)p.R, 0};
    const unsigned across = (unsigned)((p.hd + 255) / 256);
    for (int c = 0; c < p.chunks; ++c) {
      rows_of_chunk(c, 1);
      loss_gradients(r, de || dp ? &o : nullptr, dw != nullptr, db, c > 0);
      if (de && T) lattice_fold_kernel<<<dim3((unsigned)B * (unsigned)T, across), 256, 0, s>>>(l, r.chunk, dz, p.hd, 0, de32);
      if (dp) lattice_fold_kernel<<<dim3((unsigned)B * (unsigned)(U + 1), across), 256, 0, s>>>(l, r.chunk, dz, p.hd, 1, dp32);
    }
    if (de && T) lattice_fold_done_kernel<<<loss_blocks((size_t)B * T * p.H), 256, 0, s>>>(l, de32, p.hd, 0, de);
    if (dp) lattice_fold_done_kernel<<<loss_blocks((size_t)B * (U + 1) * p.H), 256, 0, s>>>(l, dp32, p.hd, 1, dp);
    if (dw) loss_dw_done(r, dw);
  }
  return check_launch("transducer loss");
} catch (const std::exception &ex) {
  return fail(WIND_ERR_HIP, std::string("wind_transducer_loss: ") + ex.what());
}

}  // extern "C"
