// The transducer loss (include/wind.h: wind_transducer_loss): the rows of all utterances' lattices, the sums over their paths, and the
// gradient's way back to encoder and prediction rows.
//
// Node (t, u) of utterance b: u labels emitted, frame t looked at; its row z = relu(e[b, t] + p[b, u]) gives blank (to (t + 1, u)) and label y[u]
// (to (t, u + 1)) their probabilities.  alpha(t, u) is the probability of reaching it, beta(t, u) of finishing from it, P = beta(0, 0); an arc's
// expected count is alpha(from) p(arc) beta(to) / P, and these are the scale and the coefficients of the node's row.
// Only nodes with t < frames[b], u <= counts[b] are rows; they are numbered b by b, t by t.  What the recursions read and write (arcs, alpha, beta) lies
// in another order where there are at least as many frames as labels: diagonal by diagonal of the threads that run them, so that what a wave asks for
// at a time is consecutive memory (by rows, 64 lanes touch 64 cache lines).
//
// Numbers.  A cell is a mantissa and an exponent of its own (m 2^e, 0.5 <= m < 1, an arc's 1 <= m < 2, e a 32-bit integer of -2^28 or more: what is
// below 2^-2^28 counts as zero).  A step of the recursion is then two
// products and one addition in fp32, relative error 2^-23 per step however improbable the cell, and no logarithm or exponential on
// the chain.  Logarithms of probabilities in fp32 lose 2^-24 of their size at every step, at -2000 a ten-thousandth of the probability.
#pragma once
#include "wind_loss_kernels.h"

namespace wind {

struct LatticeDev {
  int B, T, U, V1, H, dtype;
  const void *e, *p;                          // e [B, T, H], p [B, U + 1, H]
  long long e_b, e_t, p_b, p_u;               // strides in values
  const int *labels, *frames, *counts;        // [B, U], [B], [B]
  const float *weights;                       // [B] or null
  float *loss;                                // [B]
  int *tb, *ub, *off, *place, *part, *count;  // frames (0: left out) and labels as they are used, first row, place and part of dp, rows in all
  int cells, skew;                            // cells of a thread; 1: places lie diagonal by diagonal
  LossNodes nodes;
  float2 *alpha, *beta;                       // per place: mantissa, exponent (int bits)
};
constexpr int kFoldFrames = 8;         // frames whose dz a workgroup folds at a time
// places of T frames of U1 nodes; that of node (0, u), from which those of the later frames follow U1 apart
__device__ __forceinline__ int lattice_places(const LatticeDev &l, int T, int U1) { return T ? (T + (l.skew ? (U1 - 1) / l.cells : 0)) * U1 : 0; }
__device__ __forceinline__ int lattice_place(const LatticeDev &l, int first, int U1, int u) { return first + u + (l.skew ? u / l.cells * U1 : 0); }
__device__ __forceinline__ const char *lattice_e(const LatticeDev &l, int b, int t) { return (const char *)l.e + (b * l.e_b + t * l.e_t) * (l.dtype ? 2 : 4); }
__device__ __forceinline__ const char *lattice_p(const LatticeDev &l, int b, int u) { return (const char *)l.p + (b * l.p_b + u * l.p_u) * (l.dtype ? 2 : 4); }

// One workgroup: which utterances count, and where their rows begin; returns the number of rows.
__device__ __forceinline__ int lattice_rows(const LatticeDev &l) {
  __shared__ int wave_sum_[3][4], total_[3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // the lanes of a group look through an utterance's labels
  int group = 1;
  while (group < 64 && group < l.U) group <<= 1;
  const int at_once = 256 / group, g = tid / group, x = tid & (group - 1);
  for (int b0 = 0; b0 < l.B; b0 += at_once) {
    const int b = b0 + g;
    int T = 0, U = 0;
    bool bad = false;
    if (b < l.B) {
      T = min(max(l.frames[b], 0), l.T);
      U = min(max(l.counts[b], 0), l.U);
#pragma unroll 2
      for (int u = x; u < U; u += group) {
        const int y = l.labels[(size_t)b * l.U + u];
        bad |= y < 0 || y >= l.V1 - 1;
      }
    }
    for (int d = 1; d < group; d <<= 1) bad |= __shfl_xor((int)bad, d) != 0;
    if (b < l.B && x == 0) {
      const bool wrong = bad && T > 0;
      l.tb[b] = wrong ? 0 : T;
      l.ub[b] = U;
      if (wrong || T == 0) l.loss[b] = wrong ? __builtin_nanf("") : 0.f;
    }
  }
  __syncthreads();
  if (tid < 3) total_[tid] = 0;
  __syncthreads();
  for (int base = 0; base < l.B; base += 256) {
    const int b = base + tid;
    int n[3] = {0, 0, 0}, sum[3], at[3];
    if (b < l.B) {
      n[0] = l.tb[b] * (l.ub[b] + 1);
      n[1] = lattice_places(l, l.tb[b], l.ub[b] + 1);
      n[2] = (l.tb[b] + kFoldFrames - 1) / kFoldFrames * (l.ub[b] + 1);
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      sum[q] = n[q];
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(sum[q], d);
        if (lane >= d) sum[q] += o;
      }
      if (lane == 63) wave_sum_[q][wave] = sum[q];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      at[q] = total_[q];
      for (int w = 0; w < wave; ++w) at[q] += wave_sum_[q][w];
      if (b < l.B) (q == 0 ? l.off : q == 1 ? l.place : l.part)[b] = at[q] + sum[q] - n[q];
    }
    __syncthreads();
    if (tid == 255) {
      total_[0] = at[0] + sum[0];
      total_[1] = at[1] + sum[1];
      total_[2] = at[2] + sum[2];
    }
    __syncthreads();
  }
  if (tid == 0) {
    l.off[l.B] = total_[0];
    *l.count = total_[0];
  }
  __syncthreads();
  return total_[0];
}
// The first launch of a call: the rows, and W into panels.
__global__ __launch_bounds__(256) void lattice_begin_kernel(LossPack w, LatticeDev l, unsigned *ticket, int tickets) {
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i < tickets; i += 256) ticket[i] = 0u;
    lattice_rows(l);
  }
  else loss_pack(w, (int)blockIdx.x - 1, (int)gridDim.x - 1);
}

// a + b.  An exponent never falls below that of zero, so that sums of exponents stay in range.
__device__ __forceinline__ Cell cell_sum(Cell a, Cell b) {
  const int e = max(max(a.e, b.e), kCellZero);
  const float m = __builtin_amdgcn_ldexpf(a.m, a.e - e) + __builtin_amdgcn_ldexpf(b.m, b.e - e);
  return Cell{__builtin_amdgcn_frexp_mantf(m), e + __builtin_amdgcn_frexp_expf(m)};
}
__device__ __forceinline__ Cell cell_product(Cell a, Cell b) { return Cell{a.m * b.m, a.e + b.e}; }
__device__ __forceinline__ float2 cell_pack(Cell c) { return make_float2(c.m, __int_as_float(c.e)); }
__device__ __forceinline__ Cell cell_unpack(float2 v) { return Cell{v.x, __float_as_int(v.y)}; }

// One workgroup runs one utterance's recursion, alpha (FWD) or beta (mirrored: t' = T - 1 - t, u' = U - u), along diagonals: thread i owns C
// consecutive u, is one frame behind thread i - 1, and takes what its neighbour's last cell hands on from the lane before it, or, in a
// workgroup of several waves (MULTI), from LDS at a wave's edge.  Cells outside the lattice need no branch: before its first frame a
// thread's inputs are zero, and what is computed past the last frame or label reaches no cell that counts.  The next AHEAD
// frames' arcs are on their way while the present ones are worked off.
// The time is the number of diagonals, T + U / C, times C dependent steps and their issue by one wave.
template <int C, int AHEAD, bool MULTI, bool FWD>
__device__ __forceinline__ void lattice_run(const LatticeDev &l, int b, bool keep, float2 (&edge)[2][17]) {
  const int T = l.tb[b], U1 = l.ub[b] + 1, first = l.place[b], tid = threadIdx.x, wave = tid >> 6;
  const int steps = T + (U1 + C - 1) / C - 1;
  const char *const arcs_at = (const char *)(l.nodes.arcs + first);
  char *const keep_at = (char *)((FWD ? l.alpha : l.beta) + first);
  // byte offsets of this thread's nodes, cells (t', u' = tid C + j), for the next arcs to ask for and for the present cell (half as far)
  uint32_t ask[C], put[C];
  bool mine[C];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int u = min(tid * C + j, U1 - 1);
    mine[j] = tid * C + j < U1;
    ask[j] = (uint32_t)(lattice_place(l, 0, U1, FWD ? u : U1 - 1 - u) + (FWD ? 0 : (T - 1) * U1)) * 16u;
    put[j] = ask[j] / 2;
  }
  const uint32_t row = (uint32_t)U1 * 16u;
  int t_ask = -tid, t = -tid;
  Cell up[C], out{0.f, kCellZero}, last{0.f, kCellZero};   // what comes from the frame before; what the last cell hands on; beta(0, 0)
#pragma unroll
  for (int j = 0; j < C; ++j) up[j] = (tid == 0 && j == 0) ? Cell{0.5f, 1} : Cell{0.f, kCellZero};
  float4 arcs[2][AHEAD][C];
  auto request = [&](int set) {
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
#pragma unroll
      for (int j = 0; j < C; ++j) arcs[set][s][j] = *reinterpret_cast<const float4 *>(arcs_at + ask[j]);
      const uint32_t step = (unsigned)t_ask++ < (unsigned)(T - 1) ? row : 0u;   // stays on the first and on the last frame
#pragma unroll
      for (int j = 0; j < C; ++j) ask[j] = FWD ? ask[j] + step : ask[j] - step;
    }
  };
  auto work = [&](int set, int d0) {
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      Cell left;                          // the neighbour's, one diagonal ago
      left.m = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, out.m), 0x138, 0xF, 0xF, false));
      left.e = __builtin_amdgcn_update_dpp(kCellZero, out.e, 0x138, 0xF, 0xF, false);
      if (MULTI) {
        const int d = (d0 + s) & 1;
        if ((tid & 63) == 63) edge[d][wave + 1] = cell_pack(out);
        __syncthreads();
        if ((tid & 63) == 0) left = cell_unpack(edge[d][wave]);
      }
      const bool here = (unsigned)t < (unsigned)T;
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const float4 a = arcs[set][s][j];
        const Cell stay{a.x, __float_as_int(a.y)}, take{a.z, __float_as_int(a.w)};
        Cell v;
        if (FWD) {                        // hands on what its own arcs make of it
          v = cell_sum(up[j], left);
          up[j] = cell_product(v, stay);
          left = cell_product(v, take);
        } else {                          // its own arcs make it of what it is handed
          v = cell_sum(cell_product(up[j], stay), cell_product(left, take));
          up[j] = left = v;
          if (t == T - 1 && tid * C + j == U1 - 1) last = v;
        }
        if (keep && here && mine[j]) *reinterpret_cast<float2 *>(keep_at + put[j]) = cell_pack(v);
      }
      out = left;
      const uint32_t step = (unsigned)t++ < (unsigned)(T - 1) ? row / 2 : 0u;
#pragma unroll
      for (int j = 0; j < C; ++j) put[j] = FWD ? put[j] + step : put[j] - step;
    }
  };
  if (MULTI && tid < 34) edge[tid & 1][tid >> 1] = make_float2(0.f, __int_as_float(kCellZero));
  request(0);
  if (MULTI) __syncthreads();
  for (int d0 = 0; d0 < steps; d0 += 2 * AHEAD) {
    request(1);
    work(0, d0);
    request(0);
    work(1, d0 + AHEAD);
  }
  if (!FWD && tid == (U1 - 1) / C) l.loss[b] = (float)(-(log2((double)last.m) + (double)last.e) * kLn2);
}
template <int C, int AHEAD, bool MULTI>
__global__ __launch_bounds__(MULTI ? 1024 : 64) void lattice_sums_kernel(LatticeDev l, int both) {
  __shared__ float2 edge[2][17];
  const int b = both ? (int)blockIdx.x >> 1 : (int)blockIdx.x;
  if (l.tb[b] == 0) return;
  if (both && (blockIdx.x & 1)) lattice_run<C, AHEAD, MULTI, true>(l, b, true, edge);
  else lattice_run<C, AHEAD, MULTI, false>(l, b, both, edge);
}

// A chunk's rows, 64 from i0 on and four threads each: z = relu(e + p) in panels (of the panels, every `across`-th from `part` on), and their two
// entries (0: blank, 1: the next label).
struct LatticeRows {
  bf16_t *dst;
  size_t plane;
  int blocks, planes, across;
};
struct LatticeNode { int b, t, u, U1, place; };
__device__ __forceinline__ LatticeNode lattice_node(const LatticeDev &l, int n) {
  int lo = 0, hi = l.B;          // the last utterance whose first row is at or before n: it has rows
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.off[mid] <= n) lo = mid;
    else hi = mid;
  }
  LatticeNode d;
  d.b = lo;
  d.U1 = l.ub[lo] + 1;
  const int at = n - l.off[lo];
  d.t = at / d.U1;
  d.u = at - d.t * d.U1;
  d.place = lattice_place(l, l.place[lo], d.U1, d.u) + d.t * d.U1;
  return d;
}
__device__ __forceinline__ void lattice_chunk(const LatticeDev &l, const LossChunk &k, const LatticeRows &z, int live, int i0, int part) {
  const int used = min((live + 255) & ~255, k.R), i = i0 + (threadIdx.x >> 2), q = threadIdx.x & 3;
  if (i >= used) return;
  bf16_t *to = z.dst + (size_t)i * 32 + q * 8;
  if (i >= live) {
    const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int blk = part; blk < z.blocks; blk += z.across) loss_split8(none, z.planes, to + (size_t)blk * k.R * 32, z.plane);
    if (q == 0 && part == 0) {
      k.label[i] = k.label[k.R + i] = -1;
      k.scale[i] = 0.f;
      k.top[i] = 0.f;
      k.norm[i] = __builtin_inff();
    }
    return;
  }
  const LatticeNode d = lattice_node(l, k.c0 + i);
  LossPack e{}, p{};
  e.dtype = p.dtype = l.dtype;
  e.cols = p.cols = l.H;
  e.src = lattice_e(l, d.b, d.t);
  p.src = lattice_p(l, d.b, d.u);
  for (int blk = part; blk < z.blocks; blk += z.across) {
    const int c = blk * 32 + q * 8;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < l.H) {
      float y[8];
      loss_load8(e, 0, c, x);
      loss_load8(p, 0, c, y);
#pragma unroll
      for (int j = 0; j < 8; ++j) { x[j] += y[j]; x[j] = x[j] > 0.f || x[j] != x[j] ? x[j] : 0.f; }   // NaN stays
    }
    loss_split8(x, z.planes, to + (size_t)blk * k.R * 32, z.plane);
  }
  if (q || part) return;
  l.nodes.slot[i] = d.place;
  k.label[i] = l.V1 - 1;
  k.label[k.R + i] = d.u + 1 < d.U1 ? l.labels[(size_t)d.b * l.U + d.u] : -1;
}
__global__ __launch_bounds__(256) void lattice_chunk_kernel(LatticeDev l, LossChunk k, LatticeRows z) {
  lattice_chunk(l, k, z, chunk_rows(k), (int)blockIdx.x * 64, (int)blockIdx.y);
}
// Few utterances with few labels, in one launch: W into panels, and the rows, which every workgroup counts for itself.
constexpr int kLatticeSmall = 1024;   // B * U
__global__ __launch_bounds__(256) void lattice_small_kernel(LossPack w, int w_blocks, LatticeDev l, LossChunk k, LatticeRows z, unsigned *ticket, int tickets) {
  if ((int)blockIdx.x < w_blocks) {
    loss_pack(w, (int)blockIdx.x, w_blocks);
    return;
  }
  const int block = (int)blockIdx.x - w_blocks;
  if (block == 0)
    for (int i = threadIdx.x; i < tickets; i += 256) ticket[i] = 0u;
  const int rows = lattice_rows(l);
  lattice_chunk(l, k, z, min(rows, k.R), block / z.across * 64, block % z.across);
}

// The gradient's scales and coefficients of a chunk's rows: the arcs' expected counts, times the utterance's weight.
__global__ __launch_bounds__(256) void lattice_counts_kernel(LatticeDev l, LossChunk k) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= chunk_rows(k)) return;
  const int n = k.c0 + i;
  const LatticeNode d = lattice_node(l, n);
  const Cell P = cell_unpack(l.beta[l.place[d.b]]), a = cell_unpack(l.alpha[d.place]);
  const float4 arcs = l.nodes.arcs[d.place];
  const float w = l.weights ? l.weights[d.b] : 1.f;
  auto share = [&](float m, float e_bits, Cell next) {
    return P.m == 0.f ? 0.f : w * __builtin_amdgcn_ldexpf(a.m * m * next.m / P.m, a.e + __float_as_int(e_bits) + next.e - P.e);
  };
  const bool last = d.t + 1 == l.tb[d.b], more = d.u + 1 < d.U1;
  const float by_blank = last ? (more ? 0.f : share(arcs.x, arcs.y, Cell{0.5f, 1})) : share(arcs.x, arcs.y, cell_unpack(l.beta[d.place + d.U1]));
  const float by_label = more ? share(arcs.z, arcs.w, cell_unpack(l.beta[lattice_place(l, l.place[d.b], d.U1, d.u + 1) + d.t * d.U1])) : 0.f;
  k.coef[i] = by_blank;
  k.coef[k.R + i] = by_label;
  k.scale[i] = by_blank + by_label;
  const float2 norm = l.nodes.norm[n];
  k.top[i] = norm.x;
  k.norm[i] = norm.y;
}

// Sums of dz, where z is above zero, over the chunk's rows of one frame (which = 0) or of one prediction row (which = 1): a workgroup takes 256 columns
// with 4 threads each, or, for few long sums, 64 with 16.  The whole lattice in one chunk: the sums are rounded and stored, rows that no utterance has as zeros.  Else the
// chunk that holds the first of a sum's rows writes, later ones add, and lattice_done_kernel rounds.
struct LatticeFold {
  const float *dz;
  int ld, splits;
  size_t part;
  float *sum[2];               // [B T, ld], [B (U + 1), ld], or null
  void *out[2];                // the gradients de, dp, or null
  int wide[2];                 // columns of a workgroup: 256 or 64
};
__device__ __forceinline__ f32x4 lattice_load4(const LatticeDev &l, const char *row, int c) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (l.dtype) {
    const bf16_t *s = (const bf16_t *)row + c;
    if (c + 4 <= l.H) {
      const u32x2 w = load_any<u32x2>(s);
      v = f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u), __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xFFFF0000u)};
    } else
      for (int j = 0; j < 4; ++j) v[j] = c + j < l.H ? bf16_bits_to_f32(s[j]) : 0.f;
  } else {
    const float *s = (const float *)row + c;
    if (c + 4 <= l.H) v = load_any<f32x4>(s);
    else
      for (int j = 0; j < 4; ++j) v[j] = c + j < l.H ? s[j] : 0.f;
  }
  return v;
}
__device__ __forceinline__ void lattice_store4(const LatticeDev &l, void *out, size_t row, int c, f32x4 v) {
  if (c + 4 <= l.H) {
    if (l.dtype) store_any((bf16_t *)out + row * l.H + c, u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])});
    else store_any((float *)out + row * l.H + c, v);
    return;
  }
  for (int j = 0; j < 4 && c + j < l.H; ++j) {
    if (l.dtype) ((bf16_t *)out)[row * l.H + c + j] = (bf16_t)f32_to_bf16_bits(v[j]);
    else ((float *)out)[row * l.H + c + j] = v[j];
  }
}
template <int WIDE>
__device__ __forceinline__ void lattice_fold(const LatticeDev &l, const LossChunk &k, const LatticeFold &f, int which, int block) {
  __shared__ f32x4 sums[256];
  constexpr int lanes = WIDE / 4, groups = 256 / lanes;
  const int across = (f.ld + WIDE - 1) / WIDE, row = block / across, per = which ? l.U + 1 : l.T;
  const int live = chunk_rows(k), b = row / per, x = row - b * per;
  const int lane = threadIdx.x & (lanes - 1), wave = threadIdx.x / lanes, c = (block - row * across) * WIDE + lane * 4;
  const int T = l.tb[b], U1 = l.ub[b] + 1;
  const bool whole = f.sum[which] == nullptr;
  if (T == 0 || x >= (which ? U1 : T)) {
    if (whole && wave == 0 && c < l.H) lattice_store4(l, f.out[which], row, c, f32x4{0.f, 0.f, 0.f, 0.f});
    return;
  }
  // rows first + step * j, j = 0 .. n - 1
  const int first = l.off[b] + (which ? x : x * U1), step = which ? U1 : 1, n = which ? T : U1;
  const int j0 = first >= k.c0 ? 0 : (k.c0 - first + step - 1) / step;
  const int over = k.c0 + live - first;                       // rows below this are in the chunk or before it
  const int j1 = over <= 0 ? 0 : min(n, (over + step - 1) / step);
  if (j0 >= j1) return;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (c < l.H) {
    const f32x4 own = lattice_load4(l, which ? lattice_p(l, b, x) : lattice_e(l, b, x), c);
#pragma unroll 4
    for (int j = j0 + wave; j < j1; j += groups) {
      const float *at = f.dz + (size_t)(first + j * step - k.c0) * f.ld + c;
      f32x4 v = *reinterpret_cast<const f32x4 *>(at);
      const f32x4 other = lattice_load4(l, which ? lattice_e(l, b, j) : lattice_p(l, b, j), c);
      for (int q = 1; q < f.splits; ++q) v += *reinterpret_cast<const f32x4 *>(at + (size_t)q * f.part);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] += own[i] + other[i] > 0.f ? v[i] : 0.f;
    }
  }
  sums[threadIdx.x] = s;
  __syncthreads();
  if (wave || c >= l.H) return;
#pragma unroll
  for (int q = 1; q < groups; ++q) s += sums[q * lanes + lane];
  if (whole) {
    lattice_store4(l, f.out[which], row, c, s);
    return;
  }
  f32x4 *o = reinterpret_cast<f32x4 *>(f.sum[which] + (size_t)row * f.ld + c);
  *o = j0 > 0 ? *o + s : s;
}
// Both folds in one reading of dz, for large lattices: a workgroup takes 8 frames of an utterance and 256 columns, its waves every fourth u.  A frame's sum
// over u is done with that; a prediction row's is of 8 frames and goes to a part of dp, an eighth of dz, which lattice_parts_kernel adds up.  (165000 nodes
// of 640: 150 us for the folds apart, 90 so.)
struct LatticeOnce {
  float *parts;                // per utterance that the chunk meets [frames / 8][U1][ld]
  int n;                       // workgroups (0: the folds apart)
};
// the chunk's first part, as an utterance's parts are numbered
__device__ __forceinline__ int lattice_first_part(const LatticeDev &l, int c0) {
  const LatticeNode d = lattice_node(l, c0);
  return l.part[d.b] + d.t / kFoldFrames * d.U1;
}
__device__ __forceinline__ void lattice_fold_once(const LatticeDev &l, const LossChunk &k, const LatticeFold &f, const LatticeOnce &o, int block) {
  __shared__ f32x4 sums[4][kFoldFrames][64];
  const int across = (f.ld + 255) / 256, row = block / across, blocks = (l.T + kFoldFrames - 1) / kFoldFrames;
  const int b = row / blocks, t0 = (row - b * blocks) * kFoldFrames, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (block - row * across) * 256 + lane * 4;
  const int live = chunk_rows(k), T = l.tb[b], U1 = l.ub[b] + 1, first = l.off[b] + t0 * U1;
  const bool whole = f.sum[0] == nullptr;
  const int frames = min(kFoldFrames, T - t0);                // of the utterance
  if (whole)
    for (int i = wave; i < min(kFoldFrames, l.T - t0); i += 4)
      if (i >= frames && c < l.H) lattice_store4(l, f.out[0], (size_t)b * l.T + t0 + i, c, f32x4{0.f, 0.f, 0.f, 0.f});
  if (frames <= 0 || first >= k.c0 + live || first + frames * U1 <= k.c0) return;
  f32x4 e[kFoldFrames], de[kFoldFrames];
#pragma unroll
  for (int i = 0; i < kFoldFrames; ++i) {
    de[i] = e[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (i < frames && c < l.H) e[i] = lattice_load4(l, lattice_e(l, b, t0 + i), c);
  }
  float *const parts = o.parts + (size_t)(l.part[b] + t0 / kFoldFrames * U1 - lattice_first_part(l, k.c0)) * f.ld + c;
  if (c < l.H)
    for (int u = wave; u < U1; u += 4) {
      f32x4 v[kFoldFrames], s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kFoldFrames; ++i) {
        const int n = first + i * U1 + u - k.c0;
        v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (i < frames && n >= 0 && n < live) {
          const float *at = f.dz + (size_t)n * f.ld + c;
          v[i] = *reinterpret_cast<const f32x4 *>(at);
          for (int q = 1; q < f.splits; ++q) v[i] += *reinterpret_cast<const f32x4 *>(at + (size_t)q * f.part);
        }
      }
      const f32x4 p = lattice_load4(l, lattice_p(l, b, u), c);
#pragma unroll
      for (int i = 0; i < kFoldFrames; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x = e[i][j] + p[j] > 0.f ? v[i][j] : 0.f;
          de[i][j] += x;
          s[j] += x;
        }
      *reinterpret_cast<f32x4 *>(parts + (size_t)u * f.ld) = s;
    }
#pragma unroll
  for (int i = 0; i < kFoldFrames; ++i) sums[wave][i][lane] = de[i];
  __syncthreads();
  for (int i = wave; i < frames; i += 4) {
    const int n = first + i * U1;                             // the frame's first row
    if (c >= l.H || n >= k.c0 + live || n + U1 <= k.c0) continue;
    const f32x4 s = (sums[0][i][lane] + sums[1][i][lane]) + (sums[2][i][lane] + sums[3][i][lane]);
    const size_t to = (size_t)b * l.T + t0 + i;
    if (whole) lattice_store4(l, f.out[0], to, c, s);
    else {
      f32x4 *at = reinterpret_cast<f32x4 *>(f.sum[0] + to * f.ld + c);
      *at = n < k.c0 ? *at + s : s;
    }
  }
}
// A prediction row's parts of the chunk: a workgroup one row and 256 columns.
__global__ __launch_bounds__(256) void lattice_parts_kernel(LatticeDev l, LossChunk k, LatticeFold f, LatticeOnce o) {
  __shared__ f32x4 sums[4][64];
  const int live = chunk_rows(k), row = blockIdx.x, b = row / (l.U + 1), u = row - b * (l.U + 1);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (int)blockIdx.y * 256 + lane * 4;
  const int T = l.tb[b], U1 = l.ub[b] + 1, first = l.off[b];
  const bool whole = f.sum[1] == nullptr;
  if (T == 0 || u >= U1) {
    if (whole && wave == 0 && c < l.H) lattice_store4(l, f.out[1], row, c, f32x4{0.f, 0.f, 0.f, 0.f});
    return;
  }
  if (first + u >= k.c0 + live || first + T * U1 <= k.c0) return;
  // blocks of 8 frames that the chunk meets
  const int step = kFoldFrames * U1, x0 = max(0, k.c0 - first) / step, x1 = min((T + kFoldFrames - 1) / kFoldFrames, (k.c0 + live - first + step - 1) / step);
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (c < l.H) {
    const int base = l.part[b] - lattice_first_part(l, k.c0) + u;   // (+ x U1: not below zero from x0 on)
#pragma unroll 4
    for (int x = x0 + wave; x < x1; x += 4) s += *reinterpret_cast<const f32x4 *>(o.parts + (size_t)(base + x * U1) * f.ld + c);
  }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave || c >= l.H) return;
  s = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
  if (whole) {
    lattice_store4(l, f.out[1], row, c, s);
    return;
  }
  f32x4 *to = reinterpret_cast<f32x4 *>(f.sum[1] + (size_t)row * f.ld + c);
  *to = first + u < k.c0 ? *to + s : s;
}
// The last launch of a chunk: db, the sums over parts of dW, and what dz gives to encoder and prediction rows.
__global__ __launch_bounds__(256) void lattice_finish_kernel(LossFinish f, LossChunk k, LatticeDev l, LatticeFold fold, int n_e) {
  int block = (int)blockIdx.x;
  if (loss_finish(f, k, block)) return;
  const int which = block < n_e ? 0 : 1;
  if (which) block -= n_e;
  if (fold.wide[which] == 256) lattice_fold<256>(l, k, fold, which, block);
  else lattice_fold<64>(l, k, fold, which, block);
}

// The same of a large lattice.
__global__ __launch_bounds__(256) void lattice_finish_once_kernel(LossFinish f, LossChunk k, LatticeDev l, LatticeFold fold, LatticeOnce o) {
  int block = (int)blockIdx.x;
  if (!loss_finish(f, k, block)) lattice_fold_once(l, k, fold, o, block);
}

// The sums of several chunks, rounded once; rows that no utterance has are zero.
__global__ __launch_bounds__(256) void lattice_done_kernel(LatticeDev l, LatticeFold f) {
  const int per_row = (l.H + 3) / 4;
  const size_t rows_e = f.out[0] ? (size_t)l.B * l.T : 0, rows = rows_e + (f.out[1] ? (size_t)l.B * (l.U + 1) : 0);
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < rows * per_row; i += (size_t)gridDim.x * 256) {
    size_t row = i / per_row;
    const int c = (int)(i - row * per_row) * 4, which = row >= rows_e;
    if (which) row -= rows_e;
    const int per = which ? l.U + 1 : l.T, b = (int)(row / per), x = (int)(row - (size_t)b * per);
    const bool there = l.tb[b] > 0 && x < (which ? l.ub[b] + 1 : l.tb[b]);
    lattice_store4(l, f.out[which], row, c, there ? *reinterpret_cast<const f32x4 *>(f.sum[which] + row * f.ld + c) : f32x4{0.f, 0.f, 0.f, 0.f});
  }
}

}  // namespace wind
