// Losses over the output layer, with their gradients (include/wind.h: wind_label_loss, wind_distill_loss, wind_transducer_loss).
//
// Rows.  All three losses are sums over rows of the joiner's last layer: a hidden vector z, logits x = W z + b over V1 outputs, p = softmax(x / tau),
// and a few outputs the row is compared with ("entries": one label, K teacher labels, or a node's blank and next label).  The
// objective's gradient has one form for all of them,
//     dx_v = s p_v - sum_k c_k [v = label_k],
// with a row's scale s and its entries' coefficients c: label loss s = c = w; distillation s = w tau, c_k = w tau q_k; a lattice node s = the
// sum of its two arcs' expected counts, c the counts.  From dx follow dz = dx W, dW = sum dx z^T, db = sum dx.
//
// No logit is kept.  Forward: the product's epilogue reduces a tile to (max, sum of exp2) per row and picks out the entries' logits
// (loss_stats_kernel); loss_rows_done_kernel joins the column blocks of a row.  Backward: the product is formed again and its epilogue turns
// logits into dx (loss_dx_kernel), in bf16 panels for as many rows as a chunk holds; two more products take it from there.
// Everything runs chunk by chunk over the rows that count: rows without a label, or utterances' padding, are left out on the device
// (how many remain is known there only: workgroups past the end leave at once).
//
// Powers of two.  Row statistics are kept in units of log2: with c = log2(e) / tau the largest logit of a block is m = fl(x c), every sum
// is of exp2(fma(x, c, -m)), and lse2 = m + log2(sum), so that the rounding of m cancels.
#pragma once
#include "wind_loss_gemm.h"

namespace wind {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr double kLn2 = 0.69314718055994530942;

// ---- rows that count ----------------------------------------------------------------------------
enum LossKind { kLossLabel = 0, kLossDistill = 1, kLossLattice = 2 };

struct LossRowsDev {           // what the caller gave for every row (label loss: K = 1, logits null)
  int kind, N, K, V1;
  const int *labels;           // [N, K]
  const float *logits;         // [N, K]
  const float *weights;        // [N] or null
  float inv_tau, tau;
  float *loss;                 // [N]
  int *idx, *count;            // rows that count, ascending, and their number
};

// 0: row n counts; 1: it has no label; 2: it names an output that does not exist
__device__ __forceinline__ int loss_row_state(const LossRowsDev &r, int n) {
  if (r.kind == kLossLabel) {
    const int l = r.labels[n];
    return l < 0 ? 1 : l < r.V1 ? 0 : 2;
  }
  bool some = false;
  for (int k = 0; k < r.K; ++k) {
    const int l = r.labels[(size_t)n * r.K + k];
    if (l >= r.V1) return 2;
    some |= l >= 0 && r.logits[(size_t)n * r.K + k] != -__builtin_inff();
  }
  return some ? 0 : 1;
}

// One workgroup: the rows that count, in order; the others' losses.
__global__ __launch_bounds__(1024) void loss_rows_kernel(LossRowsDev r) {
  __shared__ int wave_sum_[16], total_;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) total_ = 0;
  __syncthreads();
  for (int base = 0; base < r.N; base += 1024) {
    const int n = base + tid;
    const int state = n < r.N ? loss_row_state(r, n) : 1;
    const unsigned long long mk = __ballot(state == 0);
    if (lane == 0) wave_sum_[wave] = __popcll(mk);
    __syncthreads();
    int at = total_;
    for (int w = 0; w < wave; ++w) at += wave_sum_[w];
    if (state == 0) r.idx[at + __popcll(mk & ((1ull << lane) - 1ull))] = n;
    else if (n < r.N) r.loss[n] = state == 1 ? 0.f : __builtin_nanf("");
    __syncthreads();
    if (tid == 1023) total_ = at + wave_sum_[15];
    __syncthreads();
  }
  if (tid == 0) *r.count = total_;
}

// Rows of the gradient that do not count: zero.
__global__ __launch_bounds__(256) void loss_zero_rows_kernel(LossRowsDev r, void *dh, int dtype, int H) {
  const int n = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= r.N || loss_row_state(r, n) == 0) return;
  for (int h = threadIdx.x & 63; h < H; h += 64) {
    if (dtype) ((bf16_t *)dh)[(size_t)n * H + h] = 0;
    else ((float *)dh)[(size_t)n * H + h] = 0.f;
  }
}

// ---- panels -------------------------------------------------------------------------------------
struct LossPack {
  const void *src;
  size_t stride;               // values between rows
  int dtype, rows, cols;       // rows of the source (or of the chunk: see idx)
  const int *idx, *count;      // null, or: row i is row idx[c0 + i] of the source for i < *count - c0, else zeros
  int c0;
  bf16_t *dst;
  size_t plane;
  int dst_rows, blocks, planes;
  int vec;                     // rows are 16-byte aligned
};

// 8 values as up to three planes
__device__ __forceinline__ void loss_split8(const float (&v)[8], int planes, bf16_t *dst, size_t plane) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = v[i];
  for (int p = 0; p < planes; ++p) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(rest[2 * i], rest[2 * i + 1]);
    *reinterpret_cast<u32x4 *>(dst + (size_t)p * plane) = w;
    if (p + 1 < planes) {
#pragma unroll
      for (int i = 0; i < 8; ++i) rest[i] -= __uint_as_float((i & 1) ? (w[i >> 1] & 0xFFFF0000u) : (w[i >> 1] << 16));
    }
  }
}
__device__ __forceinline__ void loss_load8(const LossPack &k, size_t row, int c, float (&v)[8]) {
  if (k.dtype) {
    const bf16_t *s = (const bf16_t *)k.src + row * k.stride + c;
    if (k.vec && c + 8 <= k.cols) {
      const u32x4 w = *reinterpret_cast<const u32x4 *>(s);
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + i < k.cols ? bf16_bits_to_f32(s[i]) : 0.f;
    }
  } else {
    const float *s = (const float *)k.src + row * k.stride + c;
    if (k.vec && c + 8 <= k.cols) {
      const f32x4 a = *reinterpret_cast<const f32x4 *>(s), b = *reinterpret_cast<const f32x4 *>(s + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + i < k.cols ? s[i] : 0.f;
    }
  }
}

// Matrix rows into panels: a thread moves 8 values, four threads a row's 64 bytes of a panel.
__global__ __launch_bounds__(256) void loss_pack_kernel(LossPack k) {
  const int live = k.idx ? min(max(*k.count - k.c0, 0), k.dst_rows) : k.rows;
  const int used = k.idx ? min((live + 255) & ~255, k.dst_rows) : k.dst_rows;   // rows that the products of this chunk read
  const int chunks = k.blocks * 4;
  const size_t total = (size_t)used * chunks;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
    const int q = (int)(i & 3);
    const size_t rest = i >> 2;
    const int row = (int)(rest % used), blk = (int)(rest / used);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int c = blk * 32 + q * 8;
    if (row < live && c < k.cols) loss_load8(k, k.idx ? (size_t)k.idx[k.c0 + row] : (size_t)row, c, v);
    loss_split8(v, k.planes, k.dst + (size_t)blk * k.dst_rows * 32 + (size_t)row * 32 + q * 8, k.plane);
  }
}

// ---- a chunk's rows: entries and statistics -----------------------------------------------------
struct LossChunk {
  int c0, R;                   // first row, rows (a multiple of 256)
  const int *count;            // rows that count in all
  int K;                       // entries per row
  int *label;                  // [K][R], -1: none
  float *value;                // [K][R] log2 of the teacher's probability (distillation)
  float *coef;                 // [K][R]
  float *scale;                // [R]
  float *lse2;                 // [R] (+inf: row does not count)
  float *logit;                // [K][R] the entries' logits
  float2 *part;                // [column blocks][R] (largest, sum)
  float c;                     // log2(e) / tau
};
__device__ __forceinline__ int chunk_rows(const LossChunk &k) { return min(max(*k.count - k.c0, 0), k.R); }

// Entries of label and distillation rows.  A thread a row.
__global__ __launch_bounds__(256) void loss_entries_kernel(LossRowsDev r, LossChunk k) {
  const int live = chunk_rows(k), used = min((live + 255) & ~255, k.R);
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= used) return;
  if (i >= live) {
    for (int e = 0; e < k.K; ++e) k.label[(size_t)e * k.R + i] = -1;
    k.scale[i] = 0.f;
    k.lse2[i] = __builtin_inff();
    return;
  }
  const int n = r.idx[k.c0 + i];
  const float w = r.weights ? r.weights[n] : 1.f;
  if (r.kind == kLossLabel) {
    k.label[i] = r.labels[n];
    k.coef[i] = k.scale[i] = w;
    return;
  }
  const int *lab = r.labels + (size_t)n * r.K;
  const float *lg = r.logits + (size_t)n * r.K;
  float m = -__builtin_inff();
  for (int e = 0; e < r.K; ++e)
    if (lab[e] >= 0) m = fmaxf(m, lg[e]);
  float sum = 0.f;
  for (int e = 0; e < r.K; ++e)
    if (lab[e] >= 0) sum += exp2f((lg[e] - m) * k.c);
  const float l2 = log2f(sum), wt = w * r.tau;
  for (int e = 0; e < r.K; ++e) {
    const bool there = lab[e] >= 0 && lg[e] != -__builtin_inff();
    const float v = there ? (lg[e] - m) * k.c - l2 : -__builtin_inff();
    k.label[(size_t)e * k.R + i] = there ? lab[e] : -1;
    k.value[(size_t)e * k.R + i] = v;
    k.coef[(size_t)e * k.R + i] = wt * exp2f(v);
  }
  k.scale[i] = wt;
}

// ---- logits: statistics, and the gradient's logits ----------------------------------------------
struct LossProduct {
  PanelsDev a, b;
  SegmentsDev seg;
  int stages;                  // K stages of a segment
  int cols;                    // outputs (V1)
  int ct, group;               // column tiles, tile rows of a group (loss_tile)
};

// A wave's 32 rows x 32 NI columns of logits in LDS, row-major, for entries that name columns.
template <class T>
__device__ __forceinline__ void loss_tile_out(const f32x16 (&acc)[T::NI], float *tile) {
  const int lane = threadIdx.x & 63;
  float *row = tile + (lane & 31) * T::PITCH + 4 * (lane >> 5);
#pragma unroll
  for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = acc[ni][4 * q + j];
      *reinterpret_cast<f32x4 *>(row + 32 * ni + 8 * q) = v;
    }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// whether one of the wave's rows has an entry among its columns
template <class T>
__device__ __forceinline__ bool loss_entry_here(const LossChunk &k, int i, int col0) {
  bool hit = false;
  for (int e = 0; e < k.K; ++e) hit |= (unsigned)(k.label[(size_t)e * k.R + i] - col0) < (unsigned)(32 * T::NI);
  return __any(hit);
}
// accumulators that start as the bias; columns past the end as -inf, which exp2 turns into nothing
template <class T>
__device__ __forceinline__ void loss_bias(const float *bias, int cols, int col0, f32x16 (&acc)[T::MI][T::NI]) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int v = col0 + 32 * ni + 8 * (r >> 2) + 4 * half + (r & 3);
      const float x = v < cols ? (bias ? bias[v] : 0.f) : -__builtin_inff();
#pragma unroll
      for (int mi = 0; mi < T::MI; ++mi) acc[mi][ni][r] = x;
    }
}

template <class T>
__global__ __launch_bounds__(256, 1) void loss_stats_kernel(LossProduct g, LossChunk k, const float *bias) {
  __shared__ __attribute__((aligned(256))) unsigned char smem[T::SMEM];
  const int live = chunk_rows(k);
  int ti, tj;
  if (!loss_tile((int)blockIdx.x, (live + T::BM - 1) / T::BM, g.ct, g.group, ti, tj)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int col0 = tj * T::BN + (wave & 1) * 32 * T::NI;
  f32x16 acc[T::MI][T::NI];
  loss_bias<T>(bias, g.cols, col0, acc);
  loss_mainloop<T, false, false>(g.a, g.b, g.seg, ti * T::BM, tj * T::BN, 0, g.stages, smem, acc);
  float *tile = reinterpret_cast<float *>(smem) + wave * 32 * T::PITCH;
#pragma unroll
  for (int mi = 0; mi < T::MI; ++mi) {
    const int i = ti * T::BM + ((wave >> 1) * T::MI + mi) * 32 + (lane & 31);
    float m = -__builtin_inff();
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) m = fmaxf(m, acc[mi][ni][r]);
    m = fmaxf(m, xor32_f32(m));
    const float mc = m * k.c, ref = m == -__builtin_inff() ? 0.f : mc;
    float sum = 0.f;
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[mi][ni][r], k.c, -ref));
    sum += xor32_f32(sum);
    if (lane < 32 && col0 < g.cols) k.part[(size_t)(col0 / (32 * T::NI)) * k.R + i] = make_float2(mc, sum);
    if (loss_entry_here<T>(k, i, col0)) {
      loss_tile_out<T>(acc[mi], tile);
      for (int e = lane >> 5; e < k.K; e += 2) {   // a row's entries are shared by its two lanes
        const int at = k.label[(size_t)e * k.R + i] - col0;
        if ((unsigned)at < (unsigned)(32 * T::NI)) k.logit[(size_t)e * k.R + i] = tile[(lane & 31) * T::PITCH + at];
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Joins a row's column blocks: 64 rows a workgroup, four threads a row.
struct LossNodes { float *blank, *label, *lse2; };   // per lattice node: log2 probabilities of its arcs, lse2
__global__ __launch_bounds__(256) void loss_rows_done_kernel(LossRowsDev r, LossChunk k, int parts, LossNodes nodes) {
  __shared__ float sm[4][64], ss[4][64];
  const int live = chunk_rows(k), lane = threadIdx.x & 63, grp = threadIdx.x >> 6;
  if ((int)blockIdx.x * 64 >= live) return;
  const int i = blockIdx.x * 64 + lane;
  float m = -__builtin_inff(), s = 0.f;
  if (i < live) {
    for (int p = grp; p < parts; p += 4) {
      const float2 v = k.part[(size_t)p * k.R + i];
      const float top = fmaxf(m, v.x), ref = top == -__builtin_inff() ? 0.f : top;
      s = s * __builtin_amdgcn_exp2f(m - ref) + v.y * __builtin_amdgcn_exp2f(v.x - ref);
      m = top;
    }
  }
  sm[grp][lane] = m;
  ss[grp][lane] = s;
  __syncthreads();
  if (grp || i >= live) return;
  float top = fmaxf(fmaxf(sm[0][lane], sm[1][lane]), fmaxf(sm[2][lane], sm[3][lane]));
  const float ref = top == -__builtin_inff() ? 0.f : top;
  s = 0.f;
#pragma unroll
  for (int q = 0; q < 4; ++q) s += ss[q][lane] * __builtin_amdgcn_exp2f(sm[q][lane] - ref);
  const float ls = log2f(s), lse2 = top + ls;
  k.lse2[i] = lse2;
  if (r.kind == kLossLattice) {
    const int n = k.c0 + i;
    nodes.lse2[n] = lse2;
    nodes.blank[n] = -(__builtin_fmaf(-k.logit[i], k.c, top) + ls);
    nodes.label[n] = k.label[(size_t)k.R + i] < 0 ? -__builtin_inff() : -(__builtin_fmaf(-k.logit[(size_t)k.R + i], k.c, top) + ls);
    return;
  }
  const int n = r.idx[k.c0 + i];
  if (r.kind == kLossLabel) {
    r.loss[n] = (__builtin_fmaf(-k.logit[i], k.c, top) + ls) * (float)kLn2;
    return;
  }
  float sum = 0.f;
  for (int e = 0; e < k.K; ++e) {
    if (k.label[(size_t)e * k.R + i] < 0) continue;
    const float lq = k.value[(size_t)e * k.R + i], q = exp2f(lq);
    if (q != 0.f) sum += q * (lq + (__builtin_fmaf(-k.logit[(size_t)e * k.R + i], k.c, top) + ls));
  }
  r.loss[n] = sum * (float)kLn2 * r.tau * r.tau;
}

// dx of a chunk, in panels, and its column sums.
struct LossDx {
  bf16_t *dx;
  size_t plane;
  int planes, blocks;
  float *colsum;               // [2 row tiles][blocks * 32] sums over a wave's rows, or null
};

template <class T>
__global__ __launch_bounds__(256, 1) void loss_dx_kernel(LossProduct g, LossChunk k, const float *bias, LossDx d) {
  __shared__ __attribute__((aligned(256))) unsigned char smem[T::SMEM];
  const int live = chunk_rows(k);
  int ti, tj;
  if (!loss_tile((int)blockIdx.x, (live + T::BM - 1) / T::BM, g.ct, g.group, ti, tj)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), half = lane >> 5;
  const int col0 = tj * T::BN + (wave & 1) * 32 * T::NI;
  f32x16 acc[T::MI][T::NI];
  loss_bias<T>(bias, g.cols, col0, acc);
  loss_mainloop<T, false, false>(g.a, g.b, g.seg, ti * T::BM, tj * T::BN, 0, g.stages, smem, acc);
  float *tile = reinterpret_cast<float *>(smem) + wave * 32 * T::PITCH;
#pragma unroll
  for (int mi = 0; mi < T::MI; ++mi) {
    const int i = ti * T::BM + ((wave >> 1) * T::MI + mi) * 32 + (lane & 31);
    const float s = k.scale[i], lse2 = k.lse2[i];
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[mi][ni][r] = s * __builtin_amdgcn_exp2f(__builtin_fmaf(acc[mi][ni][r], k.c, -lse2));
    if (loss_entry_here<T>(k, i, col0)) {
      loss_tile_out<T>(acc[mi], tile);
      float *row = tile + (lane & 31) * T::PITCH;
      if (lane < 32)   // one lane a row: an output that is named twice is taken off twice, in order
        for (int e = 0; e < k.K; ++e) {
          const int at = k.label[(size_t)e * k.R + i] - col0;
          if ((unsigned)at < (unsigned)(32 * T::NI)) row[at] -= k.coef[(size_t)e * k.R + i];
        }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 v = *reinterpret_cast<const f32x4 *>(row + 32 * ni + 8 * q + 4 * half);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[mi][ni][4 * q + j] = v[j];
        }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    // two lanes hold a row's columns in runs of four: they swap runs so that each stores eight
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni) {
      const int blk = col0 / 32 + ni;
      if (blk >= d.blocks) continue;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float rest[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) rest[j] = acc[mi][ni][8 * q + j];
        for (int p = 0; p < d.planes; ++p) {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(rest[2 * j], rest[2 * j + 1]);
          if (p + 1 < d.planes) {
#pragma unroll
            for (int j = 0; j < 8; ++j) rest[j] -= __uint_as_float((j & 1) ? (w[j >> 1] & 0xFFFF0000u) : (w[j >> 1] << 16));
          }
          const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
          const auto y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
          const u32x4 out = {(uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1]};
          *reinterpret_cast<u32x4 *>(d.dx + (size_t)p * d.plane + (size_t)blk * k.R * 32 + (size_t)i * 32 + (2 * q + half) * 8) = out;
        }
      }
    }
  }
  if (!d.colsum) return;
  // sums over the wave's rows: down the registers, then over the 32 lanes of a half
  float keep[(T::NI + 1) / 2];
#pragma unroll
  for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float v = acc[0][ni][r];
#pragma unroll
      for (int mi = 1; mi < T::MI; ++mi) v += acc[mi][ni][r];
      v = row16_sum_f32(v);
      const auto o = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
      v = __uint_as_float(o[0]) + __uint_as_float(o[1]);
      if ((lane & 31) == (ni & 1) * 16 + r) keep[ni >> 1] = v;
    }
  float *out = d.colsum + (size_t)(2 * ti + (wave >> 1)) * d.blocks * 32;
#pragma unroll
  for (int j = 0; j < (T::NI + 1) / 2; ++j) {
    const int ni = 2 * j + ((lane & 31) >> 4), r = lane & 15, v = col0 + 32 * ni + 8 * (r >> 2) + 4 * half + (r & 3);
    if (ni < T::NI && v < d.blocks * 32) out[v] = keep[j];
  }
}

// db: the column sums of all row tiles, 64 columns a workgroup, 16 threads a column.
__global__ __launch_bounds__(1024) void loss_db_kernel(const float *colsum, int width, int cols, int tile_rows, LossChunk k, int add, float *db) {
  __shared__ float sums[16][64];
  const int live = chunk_rows(k);
  const int parts = 2 * ((live + tile_rows - 1) / tile_rows);
  const int lane = threadIdx.x & 63, grp = threadIdx.x >> 6, v = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (v < cols)
    for (int p = grp; p < parts; p += 16) s += colsum[(size_t)p * width + v];
  sums[grp][lane] = s;
  __syncthreads();
  if (grp || v >= cols) return;
  s = 0.f;
  for (int q = 0; q < 16; ++q) s += sums[q][lane];
  db[v] = add ? db[v] + s : s;
}

// ---- products of dx -----------------------------------------------------------------------------
struct LossOut {
  void *p;
  size_t ld;                   // values between rows
  int dtype;                   // 0: fp32, 1: bf16
  int cols;
  int vec;                     // four values of a row can be stored at once
  const int *idx;              // null, or row i goes to row idx[i]
  const bf16_t *mask;          // null, or panels (of mask_rows rows): where they are not above zero, the output is zero
  size_t mask_rows;
  int add;                     // fp32: added to what is there
};
template <class T>
__device__ __forceinline__ void loss_store(const LossOut &o, const f32x16 (&acc)[T::MI][T::NI], int i0, int rows, int j0) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), half = lane >> 5;
#pragma unroll
  for (int mi = 0; mi < T::MI; ++mi) {
    const int i = i0 + ((wave >> 1) * T::MI + mi) * 32 + (lane & 31);
    if (i >= rows) continue;
    const size_t at = (size_t)(o.idx ? o.idx[i] : i) * o.ld;
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j = j0 + ((wave & 1) * T::NI + ni) * 32 + 8 * q + 4 * half;
        if (j >= o.cols) continue;
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[mi][ni][4 * q + e];
        if (o.mask) {
          const u32x2 m = *reinterpret_cast<const u32x2 *>(o.mask + (size_t)(j >> 5) * o.mask_rows * 32 + (size_t)i * 32 + (j & 31));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t bits = (e & 1) ? m[e >> 1] >> 16 : m[e >> 1] & 0xFFFFu;
            if (bits == 0) v[e] = 0.f;   // z = relu(..): never below zero
          }
        }
        if (o.dtype) {
          bf16_t *d = (bf16_t *)o.p + at + j;
          if (o.vec && j + 4 <= o.cols) *reinterpret_cast<u32x2 *>(d) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
          else
            for (int e = 0; e < 4 && j + e < o.cols; ++e) d[e] = (bf16_t)f32_to_bf16_bits(v[e]);
        } else {
          float *d = (float *)o.p + at + j;
          if (o.vec && j + 4 <= o.cols) {
            f32x4 *w = reinterpret_cast<f32x4 *>(d);
            *w = o.add ? *w + v : v;
          } else {
            for (int e = 0; e < 4 && j + e < o.cols; ++e) d[e] = o.add ? d[e] + v[e] : v[e];
          }
        }
      }
  }
}

// dz = dx W: rows of the chunk against columns of W's panels.
template <class T>
__global__ __launch_bounds__(256, 1) void loss_dz_kernel(LossProduct g, LossChunk k, LossOut o) {
  __shared__ __attribute__((aligned(256))) unsigned char smem[T::SMEM];
  const int live = chunk_rows(k);
  int ti, tj;
  if (!loss_tile((int)blockIdx.x, (live + T::BM - 1) / T::BM, g.ct, g.group, ti, tj)) return;
  f32x16 acc[T::MI][T::NI];
#pragma unroll
  for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = f32x16{};
  loss_mainloop<T, false, true>(g.a, g.b, g.seg, ti * T::BM, tj * T::BN, 0, g.stages, smem, acc);
  loss_store<T>(o, acc, ti * T::BM, live, tj * T::BN);
}

// dW = dx^T z: columns of dx's panels against columns of z's, summed over the chunk's rows, which `splits` workgroups share.
template <class T>
__global__ __launch_bounds__(256, 1) void loss_dw_kernel(LossProduct g, LossChunk k, LossOut o, int rt, int splits, size_t part) {
  __shared__ __attribute__((aligned(256))) unsigned char smem[T::SMEM];
  const int live = chunk_rows(k), stages = (live + 31) / 32;
  if (o.add && live == 0) return;
  const int split = (int)blockIdx.x % splits;
  int ti, tj;
  if (!loss_tile((int)blockIdx.x / splits, rt, g.ct, g.group, ti, tj)) return;
  const int per = (stages + splits - 1) / splits, s0 = min(split * per, stages), s1 = min(s0 + per, stages);
  f32x16 acc[T::MI][T::NI];
#pragma unroll
  for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = f32x16{};
  if (s0 < s1) loss_mainloop<T, true, true>(g.a, g.b, g.seg, ti * T::BM, tj * T::BN, s0, s1, smem, acc);
  o.p = (float *)o.p + (size_t)split * part;
  loss_store<T>(o, acc, ti * T::BM, g.cols, tj * T::BN);
}

// The splits' sums, rounded once.
__global__ __launch_bounds__(256) void loss_dw_done_kernel(const float *parts, int splits, size_t part, size_t ld, int rows, int cols, int dtype, void *dw) {
  const int per_row = (cols + 3) / 4;
  const size_t total = (size_t)rows * per_row;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
    const size_t v = i / per_row;
    const int h = (int)(i - v * per_row) * 4;
    f32x4 s = *reinterpret_cast<const f32x4 *>(parts + v * ld + h);
    for (int q = 1; q < splits; ++q) s += *reinterpret_cast<const f32x4 *>(parts + (size_t)q * part + v * ld + h);
    for (int e = 0; e < 4 && h + e < cols; ++e) {
      if (dtype) ((bf16_t *)dw)[v * cols + h + e] = (bf16_t)f32_to_bf16_bits(s[e]);
      else ((float *)dw)[v * cols + h + e] = s[e];
    }
  }
}

}  // namespace wind
