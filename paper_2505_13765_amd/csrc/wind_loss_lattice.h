// The transducer loss (include/wind.h: wind_transducer_loss): the rows of all utterances' lattices, the sums over their paths, and the
// gradient's way back to encoder and prediction rows.
//
// Node (t, u) of utterance b: u labels emitted, frame t looked at; its row z = relu(e[b, t] + p[b, u]) gives blank (to (t + 1, u)) and label y[u]
// (to (t, u + 1)) their probabilities.  alpha(t, u) is the probability of reaching it, beta(t, u) of finishing from it, P = beta(0, 0); an arc's
// expected count is alpha(from) p(arc) beta(to) / P, and these are the scale and the coefficients of the node's row.
// Only nodes with t < frames[b], u <= counts[b] are rows; they are numbered b by b, t by t.
//
// Numbers.  A cell is a mantissa and an exponent of its own (m 2^e, 0.5 <= m < 1, e a 32-bit integer).  A step of the recursion is then two
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
  int *tb, *ub, *off, *count;                 // frames (0: left out) and labels as they are used, first row, rows in all
  LossNodes nodes;
  float2 *alpha, *beta;                       // per node: mantissa, exponent (int bits)
};

__global__ __launch_bounds__(1024) void lattice_rows_kernel(LatticeDev l) {
  __shared__ int wave_sum_[16], total_;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int b = wave; b < l.B; b += 16) {
    const int T = min(max(l.frames[b], 0), l.T), U = min(max(l.counts[b], 0), l.U);
    bool bad = false;
    for (int u = lane; u < U; u += 64) {
      const int y = l.labels[(size_t)b * l.U + u];
      bad |= y < 0 || y >= l.V1 - 1;
    }
    const bool wrong = __any(bad) && T > 0;
    if (lane == 0) {
      l.tb[b] = wrong ? 0 : T;
      l.ub[b] = U;
      if (wrong || T == 0) l.loss[b] = wrong ? __builtin_nanf("") : 0.f;
    }
  }
  if (tid == 0) total_ = 0;
  __syncthreads();
  for (int base = 0; base < l.B; base += 1024) {
    const int b = base + tid;
    const int n = b < l.B ? l.tb[b] * (l.ub[b] + 1) : 0;
    int sum = n;
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(sum, d);
      if (lane >= d) sum += o;
    }
    if (lane == 63) wave_sum_[wave] = sum;
    __syncthreads();
    int at = total_;
    for (int w = 0; w < wave; ++w) at += wave_sum_[w];
    if (b < l.B) l.off[b] = at + sum - n;
    __syncthreads();
    if (tid == 1023) total_ = at + sum;
    __syncthreads();
  }
  if (tid == 0) {
    l.off[l.B] = total_;
    *l.count = total_;
  }
}

struct Cell { float m; int e; };
constexpr int kCellZero = -(1 << 28);
__device__ __forceinline__ Cell cell_of_log2(float l) {   // 2^l
  const float f = floorf(l);
  if (l == -__builtin_inff()) return Cell{0.f, kCellZero};
  return Cell{__builtin_amdgcn_exp2f(l - f), (int)f};
}
__device__ __forceinline__ Cell cell_step(Cell a, Cell pa, Cell b, Cell pb) {   // a pa + b pb
  const float m1 = a.m * pa.m, m2 = b.m * pb.m;
  const int e1 = a.e + pa.e, e2 = b.e + pb.e, e = max(e1, e2);
  const float m = ldexpf(m1, e1 - e) + ldexpf(m2, e2 - e);
  return Cell{__builtin_amdgcn_frexp_mantf(m), m == 0.f ? kCellZero : e + __builtin_amdgcn_frexp_expf(m)};
}
__device__ __forceinline__ float2 cell_pack(Cell c) { return make_float2(c.m, __int_as_float(c.e)); }
__device__ __forceinline__ Cell cell_unpack(float2 v) { return Cell{v.x, __float_as_int(v.y)}; }

// One workgroup runs one utterance's recursion, alpha or beta (mirrored: t' = T - 1 - t, u' = U - u), along diagonals: thread i owns C
// consecutive u, is one frame behind thread i - 1, and takes its neighbour's last cell from LDS.  The nodes' probabilities of the
// next AHEAD frames are requested before the present ones are worked off.
template <int C, int AHEAD>
__global__ __launch_bounds__(1024) void lattice_sums_kernel(LatticeDev l, int both) {
  __shared__ float2 edge[2][1025];
  const int b = both ? (int)blockIdx.x >> 1 : (int)blockIdx.x;
  const bool fwd = both && (blockIdx.x & 1);
  const int T = l.tb[b], U1 = l.ub[b] + 1, off = l.off[b], tid = threadIdx.x;
  if (T == 0) return;
  const int lanes = (U1 + C - 1) / C, steps = T + lanes - 1;
  // arcs that lead into cell (t', u') of this direction
  auto arcs = [&](int t, int j, float &up, float &left) {
    const int u = tid * C + j;
    up = left = -__builtin_inff();
    if (t < 0 || t >= T || u >= U1) return;
    if (fwd) {
      if (t > 0) up = l.nodes.blank[off + (t - 1) * U1 + u];
      else if (u == 0) up = 0.f;
      if (u > 0) left = l.nodes.label[off + t * U1 + u - 1];
    } else {
      const int n = off + (T - 1 - t) * U1 + (U1 - 1 - u);
      if (t > 0 || u == 0) up = l.nodes.blank[n];
      if (u > 0) left = l.nodes.label[n];
    }
  };
  Cell row[C];   // cells (t - 1, .) of this thread
#pragma unroll
  for (int j = 0; j < C; ++j) row[j] = (tid == 0 && j == 0) ? Cell{0.5f, 1} : Cell{0.f, kCellZero};
  float up[2][AHEAD][C], left[2][AHEAD][C];
  auto request = [&](int set, int d0) {
#pragma unroll
    for (int s = 0; s < AHEAD; ++s)
#pragma unroll
      for (int j = 0; j < C; ++j) arcs(d0 + s - tid, j, up[set][s][j], left[set][s][j]);
  };
  auto work = [&](int set, int d0) {
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int d = d0 + s, t = d - tid;
      const bool here = t >= 0 && t < T;
      Cell before = (tid > 0) ? cell_unpack(edge[d & 1][tid]) : Cell{0.f, kCellZero};
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const int u = tid * C + j;
        const Cell v = cell_step(row[j], cell_of_log2(up[set][s][j]), before, cell_of_log2(left[set][s][j]));
        if (here && u < U1) {
          row[j] = v;
          if (fwd) l.alpha[off + t * U1 + u] = cell_pack(v);
          else if (both) l.beta[off + (T - 1 - t) * U1 + (U1 - 1 - u)] = cell_pack(v);
          if (!fwd && t == T - 1 && u == U1 - 1)
            l.loss[b] = (float)(-(log2((double)v.m) + (double)v.e) * kLn2);
          before = v;
        }
      }
      edge[(d + 1) & 1][tid + 1] = cell_pack(before);
      __syncthreads();
    }
  };
  edge[0][tid] = edge[1][tid] = make_float2(0.f, __int_as_float(kCellZero));
  request(0, 0);
  __syncthreads();
  for (int d0 = 0; d0 < steps; d0 += 2 * AHEAD) {
    request(1, d0 + AHEAD);
    work(0, d0);
    request(0, d0 + 2 * AHEAD);
    work(1, d0 + AHEAD);
  }
}

// A chunk's rows: where they take e and p from, their two entries (0: blank, 1: the next label), and for the gradient the arcs' expected counts.
__global__ __launch_bounds__(256) void lattice_entries_kernel(LatticeDev l, LossChunk k, int2 *from, int grad) {
  const int live = chunk_rows(k), used = min((live + 255) & ~255, k.R);
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= used) return;
  if (i >= live) {
    from[i] = make_int2(-1, -1);
    k.label[i] = k.label[k.R + i] = -1;
    k.scale[i] = 0.f;
    k.lse2[i] = __builtin_inff();
    return;
  }
  const int n = k.c0 + i;
  int lo = 0, hi = l.B;          // the last utterance whose first row is at or before n and that has rows
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.off[mid] <= n) lo = mid;
    else hi = mid;
  }
  const int b = lo, U1 = l.ub[b] + 1, at = n - l.off[b], t = at / U1, u = at - t * U1;
  from[i] = make_int2(b * l.T + t, b * (l.U + 1) + u);
  k.label[i] = l.V1 - 1;
  k.label[k.R + i] = u + 1 < U1 ? l.labels[(size_t)b * l.U + u] : -1;
  if (!grad) return;
  const Cell P = cell_unpack(l.beta[l.off[b]]), a = cell_unpack(l.alpha[n]);
  const float w = l.weights ? l.weights[b] : 1.f;
  auto share = [&](float arc, Cell to) {   // expected count of an arc, times the utterance's weight
    const Cell q = cell_of_log2(arc);
    return P.m == 0.f ? 0.f : w * ldexpf(a.m * q.m * to.m / P.m, a.e + q.e + to.e - P.e);
  };
  const bool last = t + 1 == l.tb[b];
  const float by_blank = last ? (u + 1 == U1 ? share(l.nodes.blank[n], Cell{0.5f, 1}) : 0.f) : share(l.nodes.blank[n], cell_unpack(l.beta[n + U1]));
  const float by_label = u + 1 < U1 ? share(l.nodes.label[n], cell_unpack(l.beta[n + 1])) : 0.f;
  k.coef[i] = by_blank;
  k.coef[k.R + i] = by_label;
  k.scale[i] = by_blank + by_label;
  k.lse2[i] = l.nodes.lse2[n];
}

// z = relu(e + p) of a chunk's rows, in panels.
__global__ __launch_bounds__(256) void lattice_z_kernel(LatticeDev l, LossChunk k, const int2 *from, bf16_t *dst, size_t plane, int blocks, int planes, int vec) {
  const int live = chunk_rows(k), used = min((live + 255) & ~255, k.R);
  const size_t total = (size_t)used * blocks * 4;
  LossPack e{}, p{};
  e.dtype = p.dtype = l.dtype;
  e.cols = p.cols = l.H;
  e.vec = p.vec = vec;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
    const int q = (int)(i & 3);
    const size_t rest = i >> 2;
    const int row = (int)(rest % used), blk = (int)(rest / used), c = blk * 32 + q * 8;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (row < live && c < l.H) {
      const int2 f = from[row];
      const int b = f.x / l.T, t = f.x - b * l.T, u = f.y - b * (l.U + 1);
      float y[8];
      const size_t size = l.dtype ? 2 : 4;
      e.src = (const char *)l.e + (b * l.e_b + t * l.e_t) * size;
      p.src = (const char *)l.p + (b * l.p_b + u * l.p_u) * size;
      loss_load8(e, 0, c, x);
      loss_load8(p, 0, c, y);
#pragma unroll
      for (int j = 0; j < 8; ++j) { x[j] += y[j]; x[j] = x[j] > 0.f || x[j] != x[j] ? x[j] : 0.f; }   // NaN stays
    }
    loss_split8(x, planes, dst + (size_t)blk * k.R * 32 + (size_t)row * 32 + q * 8, plane);
  }
}

// Sums of dz over the chunk's rows of one frame (which = 0) or of one prediction row (which = 1): a workgroup 256 columns, its waves share the rows.
// The chunk that holds the first of them writes, later ones add.
__global__ __launch_bounds__(256) void lattice_fold_kernel(LatticeDev l, LossChunk k, const float *dz, int ld, int which, float *out) {
  __shared__ f32x4 sums[4][64];
  const int live = chunk_rows(k), per = which ? l.U + 1 : l.T;
  const int b = blockIdx.x / per, x = blockIdx.x - b * per;
  const int T = l.tb[b], U1 = l.ub[b] + 1;
  if (T == 0 || x >= (which ? U1 : T)) return;
  // rows first + step * j, j = 0 .. n - 1
  const int first = l.off[b] + (which ? x : x * U1), step = which ? U1 : 1, n = which ? T : U1;
  const int j0 = first >= k.c0 ? 0 : (k.c0 - first + step - 1) / step;
  const int over = k.c0 + live - first;                       // rows below this are in the chunk or before it
  const int j1 = over <= 0 ? 0 : min(n, (over + step - 1) / step);
  if (j0 >= j1) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.y * 256 + lane * 4;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (c < ld)
    for (int j = j0 + wave; j < j1; j += 4) s += *reinterpret_cast<const f32x4 *>(dz + (size_t)(first + j * step - k.c0) * ld + c);
  sums[wave][lane] = s;
  __syncthreads();
  if (wave || c >= ld) return;
  s = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
  f32x4 *o = reinterpret_cast<f32x4 *>(out + (size_t)blockIdx.x * ld + c);
  *o = j0 > 0 ? *o + s : s;
}

// Rounded once; rows that no utterance has are zero.
__global__ __launch_bounds__(256) void lattice_fold_done_kernel(LatticeDev l, const float *in, int ld, int which, void *out) {
  const int per = which ? l.U + 1 : l.T;
  const size_t total = (size_t)l.B * per * l.H;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
    const size_t row = i / l.H;
    const int h = (int)(i - row * l.H), b = (int)(row / per), x = (int)(row - (size_t)b * per);
    const bool there = l.tb[b] > 0 && x < (which ? l.ub[b] + 1 : l.tb[b]);
    const float v = there ? in[row * ld + h] : 0.f;
    if (l.dtype) ((bf16_t *)out)[i] = (bf16_t)f32_to_bf16_bits(v);
    else ((float *)out)[i] = v;
  }
}

}  // namespace wind
