// Host side of the losses over the output layer: argument checks, workspace, launches.  Included by wind_api.hip.
#pragma once
#include "wind_loss_lattice.h"

namespace {

// Tiles of the logits.  rate: of a full chip of them, in parts of kLossRate; alone: the part of that left when a CU has one workgroup of them instead of
// two; start: a tile's start and results, in slabs.  256 x 128 outputs in two workgroups per CU against 256 x 256 in one, sums over 640: 34 us instead
// of 50 for 5700 rows and 4097 outputs (one's start and results behind the other's products), 1 to 5 % less over 2048.
struct LossShape { int bm, bn; double rate, alone, start; };
constexpr LossShape kLossShapes[] = {{256, 256, 0.9, 1.0, 12}, {256, 128, 1.0, 0.65, 6}, {128, 128, 0.87, 0.55, 6}, {64, 64, 0.35, 1.0, 8}};
constexpr LossShape kLossShapesF32[] = {{128, 128, 0.75, 1.0, 12}, {64, 64, 0.6, 0.65, 8}};
constexpr double kLossRate = 1.2e15 / 256 / 1e6;   // operations per microsecond and CU
// the tile of each shape for operands of PA and PB planes
template <int PA, int PB>
struct LossTiles;
template <>
struct LossTiles<1, 1> {
  using T0 = LossTile<4, 4, 1, 1, 1, 5, 1>;
  using T1 = LossTile<4, 2, 1, 1, 1, 3, 2>;
  using T2 = LossTile<2, 2, 1, 1, 1, 4, 2>;
  using T3 = LossTile<1, 1, 1, 1, 4, 3, 1>;
};
template <>
struct LossTiles<2, 1> {
  using T0 = LossTile<4, 4, 2, 1, 1, 3, 1>;
  using T1 = LossTile<4, 2, 2, 1, 1, 2, 2>;
  using T2 = LossTile<2, 2, 2, 1, 1, 3, 2>;
  using T3 = LossTile<1, 1, 2, 1, 2, 3, 1>;
};
template <>
struct LossTiles<3, 3> {
  using T0 = LossTile<2, 2, 3, 3, 1, 3, 1>;
  using T1 = LossTile<1, 1, 3, 3, 1, 3, 2>;
};

// dx and rows of a chunk, about, and what its rows' statistics and entries may take beside (65537 outputs: 16 KB a row at most, as do 1024 entries).  A chunk of 2700
// rows of 65537 outputs (512 MB) left the products of few tiles: 8.9 ms for 7373 rows, one chunk 7.4
constexpr size_t kLossChunkBytes = 1200u << 20, kLossStatBytes = 512u << 20;
constexpr int kLossMaxEntries = 1024;
constexpr int kLossJoinBlocks = 2048;   // workgroups, at most, that add up dW's parts
// Entries (of all rows) and column blocks up to which a row tile's last workgroup joins its column blocks: one launch less, 36 -> 31 us for 16 rows of 1025
// outputs.  With more, that workgroup is what the others' results wait for (3001 rows of 64 entries: 73 us against 51 and 6).
constexpr long long kLossJoinEntries = 4096;
constexpr int kLossJoinParts = 128;
// Entries x column blocks from which entries are sorted by column block: a launch of 6 to 8 us against every tile looking at all of its rows' entries (12000 rows,
// 16 entries, 130 blocks: 838 -> 788 us a step; 3476, 23, 112, fp32 losses: 143 -> 137; 3001, 64, 18: even).
constexpr double kLossSortWork = 4e6;
// Sums of dz that 16 threads share instead of 4: of at least kLatticeLong rows, where 4 would leave the chip short of workgroups (240 frames of 2 labels, 24
// utterances: 56 us for 96 of them; with thousands, 750 frames of 121, 16 threads cost 6 % of the whole step).
constexpr int kLatticeLong = 64;
constexpr long long kLatticeOnce = 64ll << 20;   // bytes of dz from which it is read once for both folds, at the price of a launch
constexpr long long kLatticeFew = 1024;

// the bf16 planes that make up a stored value of each type, and the sum of two bf16 values (hidden rows of the lattice)
int loss_planes(int dtype) { return dtype == WIND_BF16 ? 1 : 3; }
int lattice_planes(int dtype) { return dtype == WIND_BF16 ? 2 : 3; }

// A last column of tiles with at most 64 columns takes a tile of that width (0.45 of the time), where it is one of few: V1 is often a multiple of 128 and
// one for blank.  184000 rows of 1025 outputs over 640: 325 -> 299 us a chunk; with 33 columns of tiles the second form of tile in the kernel costs what
// it saves, and more.
bool loss_narrow(const LossShape &s, long long n) { return s.bn >= 128 && n % s.bn > 0 && n % s.bn <= 64 && n / s.bn <= 16; }

struct LossPick { int shape, splits, bm, bn; };
// Shape of the logits' tiles, m x n outputs over `slabs` slabs of 32: the least time of the fullest CU, where a tile costs its operations, its start
// and its results.
LossPick loss_pick(int planes, long long m, long long n, long long slabs) {
  const LossShape *shapes = planes == 3 ? kLossShapesF32 : kLossShapes;
  const int count = planes == 3 ? 2 : 4, products = planes == 3 ? 6 : planes;
  LossPick best{0, 1, 0, 0};
  double least = 1e300;
  for (int t = 0; t < count; ++t) {
    const LossShape &s = shapes[t];
    const long long tiles = ((m + s.bm - 1) / s.bm) * ((n + s.bn - 1) / s.bn);
    const double fullest = std::ceil((loss_narrow(s, n) ? tiles - 0.55 * ((m + s.bm - 1) / s.bm) : (double)tiles) / 256);
    const double time = fullest * ((double)slabs * products + s.start) * s.bm * s.bn * 64 / (kLossRate * s.rate * (fullest == 1 ? s.alone : 1.0));
    if (time < least) {
      least = time;
      best = LossPick{t, 1, s.bm, s.bn};
    }
  }
  return best;
}

// Tiles of the products of dx: dz (rows x H over outputs) and dW (outputs x H over rows) go in one launch on tiles of one shape, dz first, where dW's
// tiles fill what dz's leave free.  rate: operations per microsecond of a CU with `pair` workgroups; alone: a workgroup's own rate on a CU of its own
// against the two; start: as above; chip: operations per microsecond of the whole chip, whose clock falls with its load.  From the times of 70 problems (1
// to 180000 rows, 33 to 65537 outputs, 50 to 2048 units) on each shape with 1 to 64 parts: what this picks takes 1 % more than the best of each,
// shapes picked for each product by itself took 4 %.  10000 rows of 8193 outputs over 1024: 752 -> 692 us a step, 2000 of 5615 over 147: 267 -> 216.
struct ProductShape { int bm, bn, pair; double rate, alone, start, chip; };
constexpr ProductShape kProductShapes[] = {
    {256, 256, 1, 7.0e6, 1.0, 12, 3.2e9}, {256, 128, 2, 8.7e6, 0.73, 10, 1.53e9}, {128, 128, 2, 8.2e6, 0.81, 12, 1.17e9}, {64, 64, 1, 2.2e6, 1.0, 10, 1.6e9}};
constexpr ProductShape kProductShapesF32[] = {{128, 128, 1, 7.6e6, 1.0, 37, 1.64e9}, {64, 64, 2, 6.5e6, 0.56, 18, 1.1e9}};
constexpr int kProductParts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
constexpr size_t kLossPartBytes = 80u << 20;   // parts of a sum, at most (of 600 problems, 1 to 16384 rows or 90000 nodes, 33 to 65537 outputs, 48 to 2048 units, none was picked that takes more than 70 MB)

// when `slots` workgroups at a time end that take nz tiles of time a each, then nw of time b
double products_end(long long nz, double a, long long nw, double b, long long slots) {
  const long long late = nz % slots;                               // slots with one tile of dz more
  const double lo = (double)(nz / slots) * a, hi = late ? lo + a : lo;
  const double even = ((double)nw * b + lo * (double)(slots - late) + hi * (double)late) / (double)slots;
  double end = even + b;
  for (const double from : {lo, hi}) {                             // the least end, a whole number of dW's tiles behind lo or hi, by which nw are done
    const double k = std::max(0.0, std::floor((even - from) / b));
    for (int i = 0; i < 2; ++i) {
      const double t = from + (k + i) * b;
      const double done = (double)late * std::max(0.0, std::floor((t - hi) / b + 1e-6)) + (double)(slots - late) * std::max(0.0, std::floor((t - lo) / b + 1e-6));
      if (done >= (double)nw) end = std::min(end, t);
    }
  }
  return std::max(end, hi);
}
void products_pick(int planes, long long m, long long V1, long long H, size_t z_part, size_t w_part, LossPick &z, LossPick &w) {
  const ProductShape *shapes = planes == 3 ? kProductShapesF32 : kProductShapes;
  const int count = planes == 3 ? 2 : 4, products = planes == 3 ? 6 : planes;
  const long long z_slabs = (V1 + 31) / 32, w_slabs = (m + 31) / 32;
  // parts: what their sums cost to write and read
  const double once = planes == 3 ? 1.7 : 2.8, rate = planes == 3 ? 3.6e6 : 4.5e6;
  auto join = [&](int parts, long long rows) { return parts > 1 ? once + parts * (double)rows * (double)H * 8 / rate : 0.0; };
  double least = 1e300;
  for (int t = planes == 2 ? 2 : 0; t < count; ++t) {   // (two planes: of few rows, for which the small tiles are enough)
    const ProductShape &s = shapes[t];
    const long long across = (H + s.bn - 1) / s.bn, z_tiles = (m + s.bm - 1) / s.bm * across, w_tiles = (V1 + s.bm - 1) / s.bm * across;
    const double slab = (double)s.bm * s.bn * 64 / s.rate, chip = 4.0 * (double)m * (double)H * (double)V1 * products / s.chip;
    const long long most = 1024 * s.pair;
    for (const int pz : kProductParts) {
      if (pz > 1 && (z_slabs / pz < 8 || z_tiles * pz > most || pz * z_part > kLossPartBytes)) break;
      const double a = ((double)((z_slabs + pz - 1) / pz) * products + s.start) * slab, z_join = join(pz, m);
      for (const int pw : kProductParts) {
        if (pw > 1 && (w_slabs / pw < 8 || w_tiles * pw > most || pw * w_part > kLossPartBytes)) break;
        const double b = ((double)((w_slabs + pw - 1) / pw) * products + s.start) * slab;
        const long long nz = z_tiles * pz, nw = w_tiles * pw;
        double time = s.pair == 1      ? products_end(nz, a, nw, b, 256)
                      : nz + nw <= 256 ? std::max(a, b) / s.alone
                                       : products_end(nz, 2 * a, nw, 2 * b, 512);
        time = std::max(time, chip) + 0.1 * std::min(time, chip) + z_join + join(pw, V1);   // (a chip at its own limit still wants its CUs busy to the end)
        if (time < least) {
          least = time;
          z = LossPick{t, pz, s.bm, s.bn};
          w = LossPick{t, pw, s.bm, s.bn};
        }
      }
    }
  }
}

struct LossPlan {
  int kind, dtype, V1, H, K;
  long long N;                       // rows at most
  bool grads;
  int B, T, U, cells, skew;          // lattice
  size_t places;                     // of the lattice's nodes, at most
  // derived
  int R, chunks, vblk, hblk, hd, pa, pw, pd;
  LossPick x, z, w;                  // logits, dz, dW
  bool dw_direct, dz_direct;         // written by their products: one chunk and one part; one part
  int parts;                         // column blocks of a row
  bool narrow;                       // loss_narrow of the logits' tiles
  bool fold_once;                    // dz is read once for both of its folds
  bool sort;                         // entries sorted by column block
  bool join;                         // joined by the launch that makes them
  // offsets into the workspace
  size_t idx, state, count, ticket, wp, rows, label, value, coef, scale, top, norm, logit, part, sorted, begin, dx, colsum, dw, total;
  size_t off, place, part8, once, tb, ub, slot, arcs, nnorm, alpha, beta, dz, de, dp;
};

void loss_plan(LossPlan &p) {
  p.vblk = (p.V1 + 31) / 32;
  p.hblk = (p.H + 31) / 32;
  p.hd = (p.H + 3) / 4 * 4;
  p.pw = p.pd = loss_planes(p.dtype);
  if (p.dtype == WIND_BF16 && p.N <= kLossFineRows) p.pd = 2;
  p.pa = p.kind == kLossLattice ? lattice_planes(p.dtype) : loss_planes(p.dtype);
  // A chunk holds as many rows without gradients as with them: no panel of it has 2^32 bytes, and losses alone need less memory than a step.
  const size_t row = (size_t)p.pa * p.hblk * 64 + (size_t)p.pd * p.vblk * 64 + (p.kind == kLossLattice ? (size_t)p.hd * 4 : 0);
  const size_t stat = (size_t)(p.V1 + 63) / 64 * 16 + (size_t)p.K * 16;
  const long long N = std::max(p.N, 1ll);
  const long long most = std::max<long long>((long long)std::min(kLossChunkBytes / row, kLossStatBytes / stat) / 256 * 256, 256);
  p.chunks = (int)((N + most - 1) / most);
  p.R = (int)round_up((size_t)((N + p.chunks - 1) / p.chunks), 256);
  p.chunks = (int)((N + p.R - 1) / p.R);
  const long long m = std::min<long long>(p.R, N);
  p.x = loss_pick(p.pa, m, p.V1, p.hblk);
  // (of the cells of a padded batch about two thirds count, where its utterances' lengths lie between half of the longest and the whole; chunks but
  // the last are full of cells that count)
  if (p.grads) products_pick(p.pd, p.kind == kLossLattice && p.B > 1 && p.chunks == 1 ? std::max(m * 2 / 3, 1ll) : m, p.V1, p.H, (size_t)p.R * p.hd * 4, (size_t)p.V1 * p.hd * 4, p.z, p.w);
  p.parts = 2 * ((p.V1 + p.x.bn - 1) / p.x.bn);
  p.narrow = loss_narrow((p.pd == 3 ? kLossShapesF32 : kLossShapes)[p.x.shape], p.V1);
  p.fold_once = p.kind == kLossLattice && N * p.hd * 4 >= kLatticeOnce;
  const bool may_sort = p.kind == kLossDistill && p.K > 2 && p.K <= kLossSortMost && N * p.K > kLossSmall;
  p.sort = may_sort && (double)N * p.K * p.parts >= kLossSortWork;
  // (one chunk: the tickets by which a row tile's last workgroup is known are cleared once per call)
  p.join = p.chunks == 1 && !p.narrow && !p.sort && N * p.K <= kLossJoinEntries && p.parts <= kLossJoinParts;
  p.dw_direct = p.chunks == 1 && p.w.splits == 1;
  p.dz_direct = p.kind != kLossLattice && p.z.splits == 1;
  // The workspace.  Its size does not fall where N (or B, T, U) rises: what depends on the tiles picked is taken at its most for any number of rows up to N, a chunk's rows
  // likewise, so that a caller's buffer for the largest call serves the others.
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += round_up(bytes, 256);
    return here;
  };
  const size_t R = std::min<size_t>(round_up((size_t)N, 256), (size_t)most), n = (size_t)N, parts = (size_t)(p.V1 + 63) / 64 * 2;
  // parts of a sum of `slabs` of which one has `bytes`
  auto split = [&](size_t slabs, size_t bytes) { return slabs >= 16 ? std::min(std::min<size_t>(slabs / 8, 64) * bytes, kLossPartBytes) : 0; };
  p.count = take(4);
  p.ticket = take(R / 64 * 4);
  p.wp = take((size_t)p.pw * p.vblk * 32 * p.hblk * 64);
  p.rows = take((size_t)p.pa * R * p.hblk * 64);
  p.label = take(R * p.K * 4);
  p.logit = take(R * p.K * 4);
  p.coef = take(R * p.K * 4);
  p.scale = take(R * 4);
  p.top = take(R * 4);
  p.norm = take(R * 4);
  p.part = take(R * 8 * parts);
  if (may_sort) {
    p.sorted = take(R * p.K * 4);
    p.begin = take(R / 32 * (parts + 1) * 4);
  }
  if (p.kind != kLossLattice) {
    p.idx = take(n * 4);
    p.state = take(n);
  }
  if (p.kind == kLossDistill) p.value = take(R * p.K * 4);
  if (p.kind == kLossLattice) {
    p.off = take(((size_t)p.B + 1) * 4);
    p.tb = take((size_t)p.B * 4);
    p.ub = take((size_t)p.B * 4);
    p.place = take((size_t)p.B * 4);
    p.part8 = take((size_t)p.B * 4);
    p.slot = take(R * 4);
    p.arcs = take(p.places * 16);
    p.nnorm = take(n * 8);
  }
  if (p.grads) {
    p.dx = take((p.dtype == WIND_BF16 ? std::max<size_t>(R, 2 * kLossFinePanel) : 3 * R) * p.vblk * 64);
    p.colsum = take(R / 64 * 2 * p.vblk * 128);
    const size_t dw = (size_t)p.V1 * p.hd * 4, dz = R * p.hd * 4;
    p.dw = take(std::max(n > R ? dw : 0, split(R / 32, dw)));
    p.dz = take(std::max(p.kind == kLossLattice ? dz : 0, split(p.vblk, dz)));
    if (p.kind == kLossLattice) {
      if (p.fold_once) p.once = take((R / kFoldFrames + (size_t)(p.B + 2) * (p.U + 1)) * p.hd * 4);
      p.alpha = take(p.places * 8);
      p.beta = take(p.places * 8);
      if (n > R) {
        p.de = take((size_t)p.B * p.T * p.hd * 4);
        p.dp = take((size_t)p.B * (p.U + 1) * p.hd * 4);
      }
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
  if ((l->V1 + 31ll) / 32 * 32 * ((l->H + 31ll) / 32 * 32) >= 1ll << 31) return fail(WIND_ERR_UNSUPPORTED, "V1 * H must be below 2^31");
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
  if ((unsigned long long)p.R * std::max(p.vblk, p.hblk) * 64 >= 1ull << 32) return fail(WIND_ERR_UNSUPPORTED, "V1 and H must be at most 2^23 - 32");   // (a panel of 256 rows)
  return WIND_OK;
}

unsigned loss_blocks(size_t items, size_t per = 256, size_t most = 4096) { return (unsigned)std::max<size_t>(1, std::min(most, (items + per - 1) / per)); }
unsigned loss_grid(long long rt, long long ct, int splits = 1) { return (unsigned)((rt * ct * splits + 7) / 8 * 8); }

template <class F>
void loss_with_tile(int pa, int shape, F &&f) {
  if (pa == 3) {
    if (shape == 0) f(LossTiles<3, 3>::T0{});
    else f(LossTiles<3, 3>::T1{});
  } else if (pa == 2) {
    if (shape == 0) f(LossTiles<2, 1>::T0{});
    else if (shape == 1) f(LossTiles<2, 1>::T1{});
    else if (shape == 2) f(LossTiles<2, 1>::T2{});
    else f(LossTiles<2, 1>::T3{});
  } else {
    if (shape == 0) f(LossTiles<1, 1>::T0{});
    else if (shape == 1) f(LossTiles<1, 1>::T1{});
    else if (shape == 2) f(LossTiles<1, 1>::T2{});
    else f(LossTiles<1, 1>::T3{});
  }
}
// products of dx: the tile, and that for dx on two planes where few rows turn out to count
template <class F>
void loss_with_dx_tile(int pd, int shape, F &&f) {
  using One = LossTiles<1, 1>;
  using Two = LossTiles<2, 1>;
  using Three = LossTiles<3, 3>;
  if (pd == 3) {
    if (shape == 0) f(Three::T0{}, Three::T0{});
    else f(Three::T1{}, Three::T1{});
  } else if (pd == 2) {
    if (shape == 2) f(Two::T2{}, Two::T2{});
    else f(Two::T3{}, Two::T3{});
  } else if (shape == 0) f(One::T0{}, Two::T0{});
  else if (shape == 1) f(One::T1{}, Two::T1{});
  else if (shape == 2) f(One::T2{}, Two::T2{});
  else f(One::T3{}, Two::T3{});
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

// what the launches of a call share; the packing of W, which its first one does
LossPack loss_begin(LossRun &r) {
  const LossPlan &p = r.p;
  r.w = PanelsDev{r.at<bf16_t>(p.wp), (size_t)p.vblk * 32 * p.hblk * 32, (uint32_t)p.vblk * 32, (uint32_t)p.hblk};
  r.x = PanelsDev{r.at<bf16_t>(p.rows), (size_t)p.R * p.hblk * 32, (uint32_t)p.R, (uint32_t)p.hblk};
  LossChunk &k = r.chunk;
  k.R = p.R;
  k.count = r.at<int>(p.count);
  k.K = p.K;
  k.label = r.at<int>(p.label);
  k.value = p.kind == kLossDistill ? r.at<float>(p.value) : nullptr;
  k.coef = r.at<float>(p.coef);
  k.scale = r.at<float>(p.scale);
  k.top = r.at<float>(p.top);
  k.norm = r.at<float>(p.norm);
  k.logit = r.at<float>(p.logit);
  k.part = r.at<float2>(p.part);
  k.parts = p.parts;
  if (p.sort) {
    k.sorted = r.at<uint32_t>(p.sorted);
    k.begin = r.at<int>(p.begin);
  }
  k.c = kLog2e * r.rows.inv_tau;
  const wind_output_layer &l = *r.layer;
  LossPack w{};
  w.src = l.w;
  w.stride = (size_t)l.w_stride;
  w.dtype = l.dtype;
  w.rows = l.V1;
  w.cols = l.H;
  w.dst = r.at<bf16_t>(p.wp);
  w.plane = r.w.plane;
  w.dst_rows = p.vblk * 32;
  w.blocks = p.hblk;
  w.planes = p.pw;
  return w;
}

LossProduct loss_logits(const LossRun &r) { return LossProduct{r.x, r.w, r.p.hblk, r.p.V1, (r.p.V1 + r.p.x.bn - 1) / r.p.x.bn}; }
void loss_stats(const LossRun &r, LossNodes nodes) {
  const LossPlan &p = r.p;
  const LossProduct g = loss_logits(r);
  unsigned *ticket = r.at<unsigned>(p.ticket);
  loss_with_tile(p.pa, p.x.shape, [&](auto t) {
    using T = decltype(t);
    const unsigned grid = loss_grid((p.R + T::BM - 1) / T::BM, g.ct);
    if (p.join) loss_stats_kernel<T, true, false><<<grid, 256, 0, r.s>>>(g, r.chunk, r.layer->b, r.rows, nodes, ticket);
    else if (T::NI > 1 && p.narrow) loss_stats_kernel<T, false, (T::NI > 1)><<<grid, 256, 0, r.s>>>(g, r.chunk, r.layer->b, r.rows, nodes, ticket);
    else loss_stats_kernel<T, false, false><<<grid, 256, 0, r.s>>>(g, r.chunk, r.layer->b, r.rows, nodes, ticket);
  });
  if (p.join) return;
  if (p.parts > 256 && p.R <= 4096) loss_rows_done_kernel<4><<<p.R / 4, 256, 0, r.s>>>(r.rows, r.chunk, p.parts, nodes);
  else loss_rows_done_kernel<16><<<p.R / 16, 256, 0, r.s>>>(r.rows, r.chunk, p.parts, nodes);
}
// dx and its products; what the chunk's last launch has to do then.  dz: the output of one part (label and distillation rows).
LossFinish loss_gradients(const LossRun &r, int chunk, bool dz, LossOut dz_out, void *dw, float *db) {
  const LossPlan &p = r.p;
  const LossProduct g = loss_logits(r);
  const LossDx d{r.at<bf16_t>(p.dx), (size_t)p.R * p.vblk * 32, p.pd, p.vblk, db ? r.at<float>(p.colsum) : nullptr, p.pd == 1};
  loss_with_tile(p.pa, p.x.shape, [&](auto t) {
    using T = decltype(t);
    const unsigned grid = loss_grid((p.R + T::BM - 1) / T::BM, g.ct);
    if (T::NI > 1 && p.narrow) loss_dx_kernel<T, (T::NI > 1)><<<grid, 256, 0, r.s>>>(g, r.chunk, r.layer->b, d);
    else loss_dx_kernel<T, false><<<grid, 256, 0, r.s>>>(g, r.chunk, r.layer->b, d);
  });
  LossFinish f{};
  if (db) {
    f.db = LossDb{d.colsum, p.vblk * 32, p.V1, p.x.bm, chunk > 0, p.pd == 1, db};
    f.n_db = (p.V1 + 15) / 16;
  }
  const PanelsDev dx{d.dx, d.plane, (uint32_t)p.R, (uint32_t)p.vblk};
  LossOut zo = dz_out, wo{};
  if (dz && !p.dz_direct) {
    zo = LossOut{r.at<float>(p.dz), (size_t)p.hd, 0, p.H, nullptr, 0, p.z.splits, (size_t)p.R * p.hd};
    if (p.kind != kLossLattice) {
      f.dz = LossJoin{r.at<float>(p.dz), p.z.splits, zo.part, zo.ld, 0, p.H, p.dtype, dz_out.idx, dz_out.p};
      f.n_dz = (int)loss_blocks((size_t)p.R * (p.hd / 4), 256, 1024);
    }
  }
  if (dw) {
    wo = LossOut{r.at<float>(p.dw), (size_t)p.hd, 0, p.H, nullptr, chunk > 0, p.w.splits, (size_t)p.V1 * p.hd};
    if (p.dw_direct) wo = LossOut{dw, (size_t)p.H, p.dtype, p.H, nullptr, 0, 1, 0};
    else if (chunk + 1 == p.chunks) {
      f.dw = LossJoin{r.at<float>(p.dw), p.w.splits, wo.part, wo.ld, p.V1, p.H, p.dtype, nullptr, dw};
      f.n_dw = (int)loss_blocks((size_t)p.V1 * (p.hd / 4), 256, kLossJoinBlocks);
    }
  }
  const LossProduct z{dx, r.w, p.vblk, p.H, (p.H + p.z.bn - 1) / p.z.bn}, w{dx, r.x, 0, p.V1, (p.H + p.w.bn - 1) / p.w.bn};
  const unsigned z_blocks = dz ? loss_grid((p.R + p.z.bm - 1) / p.z.bm, z.ct, zo.splits) : 0;
  const unsigned w_blocks = dw ? loss_grid((p.V1 + p.w.bm - 1) / p.w.bm, w.ct, wo.splits) : 0;
  if (dz || dw)
    loss_with_dx_tile(p.pd, p.z.shape, [&](auto t, auto fine) {
      loss_products_kernel<decltype(t), decltype(fine)><<<z_blocks + w_blocks, 256, 0, r.s>>>(z, zo, (int)z_blocks, w, wo, r.chunk);
    });
  return f;
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
  rows.state = r.at<unsigned char>(p.state);
  r.rows = rows;
  const LossPack w = loss_begin(r);
  const unsigned w_blocks = loss_blocks((size_t)w.dst_rows * p.hblk * 4);
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
  LossOut dz{dh, (size_t)p.H, p.dtype, p.H, nullptr, 0, 1, 0};
  const bool small = p.chunks == 1 && N * p.K <= kLossSmall;
  if (small) {
    const unsigned across = std::min<unsigned>((unsigned)p.hblk, std::max(1u, 512u / (unsigned)(p.R / 64)));
    loss_small_kernel<<<w_blocks + (unsigned)(p.R / 64) * across, 256, 0, s>>>(w, (int)w_blocks, rows, k, r.chunk, (int)across, dh, r.at<unsigned>(p.ticket), p.R / 64);
  } else {
    const unsigned states = loss_blocks((size_t)N * std::min(p.K, 64), 256, 1024);
    loss_begin_kernel<<<w_blocks + states, 256, 0, s>>>(w, (int)w_blocks, rows, dh);
    loss_compact_kernel<<<1, 1024, 0, s>>>(rows, r.at<unsigned>(p.ticket), p.R / 64);
  }
  for (int c = 0; c < p.chunks; ++c) {
    k.c0 = r.chunk.c0 = c * p.R;
    const unsigned packs = loss_blocks((size_t)p.R * p.hblk * 4), entries = loss_blocks((size_t)p.R * std::min(p.K, 64), 256, 1024);
    if (!small) loss_chunk_kernel<<<packs + entries, 256, 0, s>>>(k, (int)packs, rows, r.chunk);
    if (p.sort) loss_sort_kernel<<<p.R / 32, 256, 0, s>>>(r.chunk, LossBlocks{p.x.bn, (p.V1 + p.x.bn - 1) / p.x.bn, p.narrow});
    loss_stats(r, LossNodes{});
    if (!p.grads) continue;
    dz.idx = rows.idx + k.c0;
    const LossFinish f = loss_gradients(r, c, dh != nullptr, dz, dw, db);
    if (f.n_db + f.n_dw + f.n_dz) loss_finish_kernel<<<(unsigned)(f.n_db + f.n_dw + f.n_dz), 256, 0, s>>>(f, r.chunk);
  }
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
  if ((double)T * (U + 1.0) >= 134217728.0) return fail(WIND_ERR_UNSUPPORTED, "T * (U + 1) must be below 2^27");
  if ((double)B * T * (U + 1.0) >= 2147483648.0 || (double)B * (U + 64.0) >= 2147483648.0) return fail(WIND_ERR_UNSUPPORTED, "B * T * (U + 1) and B * (U + 64) must be below 2^31");
  // (the largest launch, lattice_finish_kernel's, has fewer than 2^24 workgroups of 256 threads: a column block of a frame or prediction row each, db's and dW's)
  if (grads && (double)B * ((double)T + U + 1.0) * ((layer->H + 255ll) / 256) + (layer->V1 + 15ll) / 16 + kLossJoinBlocks >= 16777216.0)
    return fail(WIND_ERR_UNSUPPORTED, "gradients need B * (T + U + 1) * ceil(H / 256) + ceil(V1 / 16) + 2048 below 2^24");
  p.kind = kLossLattice;
  p.dtype = layer->dtype;
  p.V1 = layer->V1;
  p.H = layer->H;
  p.K = 2;
  p.B = B;
  p.T = T;
  p.U = U;
  p.N = (long long)B * T * (U + 1);
  p.cells = U < 64 ? 1 : U < 128 ? 2 : U < 256 ? 4 : U < 1024 ? 1 : 4;   // of a thread of lattice_sums_kernel
  p.skew = U <= T && (long long)B * (T + U / p.cells) * (U + 1) < 1ll << 31;
  p.places = (size_t)B * ((size_t)T + std::min(T, U)) * ((size_t)U + 1);   // (skewed or not, and whatever the cells of a thread)
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
  if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(kLog2e * (1.f / temperature)))
    return fail(WIND_ERR_ARG, "temperature must be positive and finite, and so must log2(e) / temperature");
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
  l.nodes = LossNodes{r.at<float4>(p.arcs), r.at<int>(p.slot), r.at<float2>(p.nnorm)};
  l.place = r.at<int>(p.place);
  l.part = r.at<int>(p.part8);
  l.cells = p.cells;
  l.skew = p.skew;
  if (p.grads) {
    l.alpha = r.at<float2>(p.alpha);
    l.beta = r.at<float2>(p.beta);
  }
  const LossPack w = loss_begin(r);
  const unsigned w_blocks = loss_blocks((size_t)w.dst_rows * p.hblk * 4);
  // a workgroup's 64 rows are shared by as many as it takes to fill the chip
  const unsigned across = std::min<unsigned>((unsigned)p.hblk, std::max(1u, 1024u / (unsigned)(p.R / 64)));
  const LatticeRows z{r.at<bf16_t>(p.rows), r.x.plane, p.hblk, p.pa, (int)across};
  const bool small = p.chunks == 1 && B <= 256 && (long long)B * U <= kLatticeSmall && p.R <= 16384;
  if (small)
    lattice_small_kernel<<<w_blocks + (unsigned)(p.R / 64) * across, 256, 0, s>>>(w, (int)w_blocks, l, r.chunk, z, r.at<unsigned>(p.ticket), p.R / 64);
  else lattice_begin_kernel<<<1 + w_blocks, 256, 0, s>>>(w, l, r.at<unsigned>(p.ticket), p.R / 64);
  auto rows_of_chunk = [&](int c) {
    r.chunk.c0 = c * p.R;
    lattice_chunk_kernel<<<dim3((unsigned)(p.R / 64), across), 256, 0, s>>>(l, r.chunk, z);
  };
  for (int c = p.chunks - 1; c >= 0; --c) {   // the first chunk last: its rows are then there when the gradient begins with it
    if (!small) rows_of_chunk(c);
    loss_stats(r, l.nodes);
  }
  const int both = p.grads, cells = U + 1;
  const unsigned runs = (unsigned)B << both;
  if (cells <= 64) lattice_sums_kernel<1, 8, false><<<runs, 64, 0, s>>>(l, both);
  else if (cells <= 128) lattice_sums_kernel<2, 8, false><<<runs, 64, 0, s>>>(l, both);
  else if (cells <= 256) lattice_sums_kernel<4, 4, false><<<runs, 64, 0, s>>>(l, both);
  else if (cells <= 1024) lattice_sums_kernel<1, 4, true><<<runs, (unsigned)round_up((size_t)cells, 64), 0, s>>>(l, both);
  else lattice_sums_kernel<4, 1, true><<<runs, (unsigned)round_up((size_t)(cells + 3) / 4, 64), 0, s>>>(l, both);
  if (p.grads) {
    const bool whole = p.chunks == 1;
    LatticeFold fold{r.at<float>(p.dz), p.hd, p.z.splits, (size_t)p.R * p.hd, {nullptr, nullptr}, {T ? de : nullptr, dp}, {0, 0}};
    const long long over = (p.hd + 255) / 256;
    fold.wide[0] = U + 1 >= kLatticeLong && over * B * T <= kLatticeFew ? 64 : 256;
    fold.wide[1] = T >= kLatticeLong && over * B * (U + 1) <= kLatticeFew ? 64 : 256;
    if (!whole) {
      fold.sum[0] = r.at<float>(p.de);
      fold.sum[1] = r.at<float>(p.dp);
    }
    auto columns = [&](int which) { return (p.hd + fold.wide[which] - 1) / fold.wide[which]; };
    const int n_e = fold.out[0] ? B * T * columns(0) : 0, n_p = fold.out[1] ? B * (U + 1) * columns(1) : 0;
    for (int c = 0; c < p.chunks; ++c) {
      if (c > 0) rows_of_chunk(c);
      lattice_counts_kernel<<<p.R / 256, 256, 0, s>>>(l, r.chunk);
      const LossFinish f = loss_gradients(r, c, n_e + n_p > 0, LossOut{}, dw, db);
      if (p.fold_once && n_e && n_p) {
        const LatticeOnce once{r.at<float>(p.once), B * ((T + kFoldFrames - 1) / kFoldFrames) * (int)over};
        lattice_finish_once_kernel<<<(unsigned)(f.n_db + f.n_dw + once.n), 256, 0, s>>>(f, r.chunk, l, fold, once);
        lattice_parts_kernel<<<dim3((unsigned)B * (unsigned)(U + 1), (unsigned)over), 256, 0, s>>>(l, r.chunk, fold, once);
        continue;
      }
      const int blocks = f.n_db + f.n_dw + n_e + n_p;
      if (blocks) lattice_finish_kernel<<<(unsigned)blocks, 256, 0, s>>>(f, r.chunk, l, fold, n_e);
    }
    if (!whole && n_e + n_p) lattice_done_kernel<<<loss_blocks(((size_t)B * (T + U + 1)) * (p.hd / 4)), 256, 0, s>>>(l, fold);
  }
  return check_launch("transducer loss");
} catch (const std::exception &ex) {
  return fail(WIND_ERR_HIP, std::string("wind_transducer_loss: ") + ex.what());
}

}  // extern "C"
