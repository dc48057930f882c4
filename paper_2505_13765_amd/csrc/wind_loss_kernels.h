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
// Exponentials.  A row's statistics are its largest logit m and s = sum exp2((x - m) c), c = log2(e) / tau: the difference is taken before it is scaled, so
// that the largest term is 1 whatever the logits' size (a block of outputs that the bias masks with -1e30 had a sum of exp2 of m c's rounding, and with the lowest
// value m c was infinite).  -log2 p = (m - x) c + log2 s, and p itself is exp2((x - m) c - log2 s).
#pragma once
#include "wind_loss_gemm.h"

namespace wind {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr double kLn2 = 0.69314718055994530942;

// Vectors at any address: the hardware takes them at every alignment (a row of 654 bf16 values begins at 4-byte steps; by single values W of 43250 such
// rows was packed in 58 us).
template <class V>
__device__ __forceinline__ V load_any(const void *p) {
  V v;
  __builtin_memcpy(&v, p, sizeof(V));
  return v;
}
template <class V>
__device__ __forceinline__ void store_any(void *p, V v) {
  __builtin_memcpy(p, &v, sizeof(V));
}

// ---- rows that count ----------------------------------------------------------------------------
enum LossKind { kLossLabel = 0, kLossDistill = 1, kLossLattice = 2 };

struct LossRowsDev {           // what the caller gave for every row (label loss: K = 1, logits null)
  int kind, N, K, V1;
  const int *labels;           // [N, K]
  const float *logits;         // [N, K]
  const float *weights;        // [N] or null
  float inv_tau, tau;
  float *loss;                 // [N]
  unsigned char *state;        // [N]
  int *idx, *count;            // rows that count, ascending, and their number
};

// Lanes that share a row's K entries: a power of two, at most a wave.
__device__ __forceinline__ int loss_group(int K) { return K <= 1 ? 1 : K >= 33 ? 64 : 1 << (32 - __builtin_clz((unsigned)(K - 1))); }
__device__ __forceinline__ float group_max(float v, int group) {
  for (int d = 1; d < group; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float group_sum(float v, int group) {
  for (int d = 1; d < group; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

// A wave clears a row of the gradient.
__device__ __forceinline__ void loss_clear_row(void *dh, size_t n, int dtype, int H) {
  const size_t bytes = (size_t)H * (dtype ? 2 : 4);
  char *row = (char *)dh + n * bytes;
  for (size_t c = (threadIdx.x & 63) * 16; c < bytes; c += 1024) {
    if (c + 16 <= bytes) store_any(row + c, u32x4{0u, 0u, 0u, 0u});
    else
      for (size_t x = c; x < bytes; x += 2) *reinterpret_cast<uint16_t *>(row + x) = 0;
  }
}

// Which rows count: state 1, else 0 and the row's loss (0, or NaN if it names an output that does not exist) and gradient (zeros).
__device__ __forceinline__ void loss_states(const LossRowsDev &r, int block, int nblocks, void *dh, int dtype, int H) {
  const int group = r.kind == kLossLabel ? 1 : loss_group(r.K), rows = 256 / group;
  const int l = threadIdx.x & (group - 1);
  for (long long n0 = (long long)block * rows; n0 < r.N; n0 += (long long)nblocks * rows) {
    const long long n = n0 + threadIdx.x / group;
    bool some = false, wrong = false;
    if (n < r.N)
      for (int k = l; k < r.K; k += group) {
        const int y = r.labels[(size_t)n * r.K + k];
        wrong |= y >= r.V1;
        some |= y >= 0 && (r.kind == kLossLabel || r.logits[(size_t)n * r.K + k] != -__builtin_inff());
      }
    for (int d = 1; d < group; d <<= 1) {
      some |= __shfl_xor((int)some, d) != 0;
      wrong |= __shfl_xor((int)wrong, d) != 0;
    }
    const bool counts = some && !wrong;
    if (n < r.N && l == 0) {
      r.state[n] = counts ? 1 : 0;
      if (!counts) r.loss[n] = wrong ? __builtin_nanf("") : 0.f;
    }
    if (!dh) continue;
    unsigned long long out = __ballot(n < r.N && l == 0 && !counts);   // the wave clears its rows one after the other
    while (out) {
      const int at = __builtin_ctzll(out);
      out &= out - 1;
      loss_clear_row(dh, (size_t)(n0 + ((threadIdx.x & ~63) + at) / group), dtype, H);
    }
  }
}

// One workgroup: the rows that count, in order.  A thread looks at 16 rows at a time.
__global__ __launch_bounds__(1024) void loss_compact_kernel(LossRowsDev r, unsigned *ticket, int tickets) {
  __shared__ int wave_sum_[16], total_;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < tickets; i += 1024) ticket[i] = 0u;
  if (tid == 0) total_ = 0;
  __syncthreads();
  for (long long base = 0; base < r.N; base += 16384) {
    const long long n = base + tid * 16;
    u32x4 st = {0u, 0u, 0u, 0u};
    if (n < r.N) st = *reinterpret_cast<const u32x4 *>(r.state + n);   // (whole sixteens are allocated)
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) bits |= ((st[i >> 2] >> (8 * (i & 3))) & 1u) << i;
    if (n + 16 > r.N) bits &= n < r.N ? (1u << (r.N - n)) - 1u : 0u;
    const int mine = __popc(bits);
    int sum = mine;
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(sum, d);
      if (lane >= d) sum += o;
    }
    if (lane == 63) wave_sum_[wave] = sum;
    __syncthreads();
    int at = total_;
    for (int w = 0; w < wave; ++w) at += wave_sum_[w];
    int put = at + sum - mine;
    while (bits) {
      r.idx[put++] = (int)n + __builtin_ctz(bits);
      bits &= bits - 1;
    }
    __syncthreads();
    if (tid == 1023) total_ = at + sum;
    __syncthreads();
  }
  if (tid == 0) *r.count = total_;
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
    if (c + 8 <= k.cols) {
      const u32x4 w = load_any<u32x4>(s);
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + i < k.cols ? bf16_bits_to_f32(s[i]) : 0.f;
    }
  } else {
    const float *s = (const float *)k.src + row * k.stride + c;
    if (c + 8 <= k.cols) {
      const f32x4 a = load_any<f32x4>(s), b = load_any<f32x4>(s + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + i < k.cols ? s[i] : 0.f;
    }
  }
}

// Matrix rows into panels: a thread moves 8 values, four threads a row's 64 bytes of a panel.
__device__ __forceinline__ void loss_pack(const LossPack &k, int block, int nblocks) {
  const int live = k.idx ? min(max(*k.count - k.c0, 0), k.dst_rows) : k.rows;
  const int used = k.idx ? min((live + 255) & ~255, k.dst_rows) : k.dst_rows;   // rows that the products of this chunk read
  const int chunks = k.blocks * 4;
  const size_t total = (size_t)used * chunks;
  for (size_t i = (size_t)block * 256 + threadIdx.x; i < total; i += (size_t)nblocks * 256) {
    const int q = (int)(i & 3);
    const size_t rest = i >> 2;
    const int row = (int)(rest % used), blk = (int)(rest / used);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int c = blk * 32 + q * 8;
    if (row < live && c < k.cols) loss_load8(k, k.idx ? (size_t)k.idx[k.c0 + row] : (size_t)row, c, v);
    loss_split8(v, k.planes, k.dst + (size_t)blk * k.dst_rows * 32 + (size_t)row * 32 + q * 8, k.plane);
  }
}

// The first launch of a call: W into panels, and behind it which rows count.
__global__ __launch_bounds__(256) void loss_begin_kernel(LossPack w, int pack_blocks, LossRowsDev r, void *dh) {
  if ((int)blockIdx.x < pack_blocks) loss_pack(w, (int)blockIdx.x, pack_blocks);
  else loss_states(r, (int)blockIdx.x - pack_blocks, (int)gridDim.x - pack_blocks, dh, w.dtype, w.cols);
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
  float *top, *norm;           // [R] largest logit, log2 of the sum (0, +inf: row does not count)
  float *logit;                // [K][R] the entries' logits
  float2 *part;                // [column blocks][R] (largest, sum)
  // many entries (else null): those of 32 rows by column block, and where each block's begin
  uint32_t *sorted;            // [R / 32][32 K]: column within its block << 18 | row << 12 | entry
  int *begin;                  // [R / 32][parts + 1]
  int parts;
  float c;                     // log2(e) / tau
};
__device__ __forceinline__ int chunk_rows(const LossChunk &k) { return min(max(*k.count - k.c0, 0), k.R); }

// Entries of label and distillation rows `begin` to `end` of a chunk, of which `live` count.
__device__ __forceinline__ void loss_entries(const LossRowsDev &r, const LossChunk &k, int live, int begin, int end, int stride) {
  const int group = r.kind == kLossLabel ? 1 : loss_group(r.K), rows = 256 / group, l = threadIdx.x & (group - 1);
  for (int i0 = begin; i0 < end; i0 += stride * rows) {
    const int i = i0 + (int)threadIdx.x / group;
    if (i >= end) continue;
    if (i >= live) {
      for (int e = l; e < k.K; e += group) k.label[(size_t)e * k.R + i] = -1;
      if (l == 0) {
        k.scale[i] = 0.f;
        k.top[i] = 0.f;
        k.norm[i] = __builtin_inff();
      }
      continue;
    }
    const int n = r.idx[k.c0 + i];
    const float w = r.weights ? r.weights[n] : 1.f;
    if (r.kind == kLossLabel) {
      k.label[i] = r.labels[n];
      k.coef[i] = k.scale[i] = w;
      continue;
    }
    const int *lab = r.labels + (size_t)n * r.K;
    const float *lg = r.logits + (size_t)n * r.K;
    float m = -__builtin_inff(), sum = 0.f;
    for (int e = l; e < r.K; e += group)
      if (lab[e] >= 0) m = fmaxf(m, lg[e]);
    m = group_max(m, group);
    for (int e = l; e < r.K; e += group)
      if (lab[e] >= 0) sum += exp2f((lg[e] - m) * k.c);
    const float l2 = log2f(group_sum(sum, group)), wt = w * r.tau;
    for (int e = l; e < r.K; e += group) {
      const bool there = lab[e] >= 0 && lg[e] != -__builtin_inff();
      const float v = there ? (lg[e] - m) * k.c - l2 : -__builtin_inff();
      k.label[(size_t)e * k.R + i] = there ? lab[e] : -1;
      k.value[(size_t)e * k.R + i] = v;
      k.coef[(size_t)e * k.R + i] = wt * exp2f(v);
    }
    if (l == 0) k.scale[i] = wt;
  }
}

// The first launch of a chunk: its rows into panels, and their entries.
__global__ __launch_bounds__(256) void loss_chunk_kernel(LossPack h, int pack_blocks, LossRowsDev r, LossChunk k) {
  if ((int)blockIdx.x < pack_blocks) {
    loss_pack(h, (int)blockIdx.x, pack_blocks);
    return;
  }
  const int live = chunk_rows(k), block = (int)blockIdx.x - pack_blocks, group = r.kind == kLossLabel ? 1 : loss_group(r.K);
  loss_entries(r, k, live, block * (256 / group), min((live + 255) & ~255, k.R), (int)gridDim.x - pack_blocks);
}

// Entries of 32 rows sorted by column block, column, row and entry, so that a tile of logits finds its own without looking at the others' and an output that a
// row names again follows itself (39 entries a row over 10169 outputs: gradient of the logits 102 us, looking at all).  Bitonic, in LDS.
constexpr int kLossSortMost = 128;     // entries a row
struct LossBlocks { int bn, ct, narrow; };   // columns of a tile, tiles, and whether the last one is narrow: two blocks a tile
__global__ __launch_bounds__(256) void loss_sort_kernel(LossChunk k, LossBlocks b) {
  __shared__ unsigned long long key[32 * kLossSortMost];   // block << 32 | column << 18 | row << 12 | entry
  const int rows0 = blockIdx.x * 32, tid = threadIdx.x, n = 32 * k.K;
  if (rows0 >= ((chunk_rows(k) + 255) & ~255)) return;
  int size = 64;
  while (size < n) size <<= 1;
  for (int x = tid; x < size; x += 256) {
    const int row = x & 31, e = x >> 5, y = x < n ? k.label[(size_t)e * k.R + rows0 + row] : -1;
    unsigned long long v = ~0ull;
    if (y >= 0) {
      const int tile = y / b.bn, width = b.narrow && tile + 1 == b.ct ? 32 : b.bn / 2, in = y - tile * b.bn, half = in / width;
      v = (unsigned long long)(2 * tile + half) << 32 | (unsigned)((in - half * width) << 18 | row << 12 | e);
    }
    key[x] = v;
  }
  __syncthreads();
  for (int run = 2; run <= size; run <<= 1)
    for (int step = run >> 1; step > 0; step >>= 1) {
      for (int t = tid; t < size / 2; t += 256) {
        const int i = 2 * t - (t & (step - 1)), j = i + step;
        const unsigned long long u = key[i], v = key[j];
        if ((u > v) == ((i & run) == 0)) {
          key[i] = v;
          key[j] = u;
        }
      }
      __syncthreads();
    }
  for (int x = tid; x < n; x += 256) k.sorted[(size_t)blockIdx.x * n + x] = (uint32_t)key[x];
  for (int p = tid; p <= k.parts; p += 256) {   // the first key of block p or above
    int lo = 0, hi = size;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if ((key[mid] >> 32) < (unsigned long long)p) lo = mid + 1;
      else hi = mid;
    }
    k.begin[(size_t)blockIdx.x * (k.parts + 1) + p] = min(lo, n);
  }
}

// Few rows, in one launch: W into panels, which rows count, and the rows' panels and entries.  Every workgroup of rows looks at all labels itself
// (kLossSmall of them at most) and finds the places of its 64 rows among those that count; `across` of them share the 64 rows' panels.
constexpr int kLossSmall = 16384;
__global__ __launch_bounds__(256) void loss_small_kernel(LossPack w, int w_blocks, LossRowsDev r, LossPack h, LossChunk k, int across, void *dh, unsigned *ticket,
                                                         int tickets) {
  __shared__ __attribute__((aligned(16))) unsigned char state[kLossSmall];
  __shared__ int sums[4];
  if ((int)blockIdx.x < w_blocks) {
    loss_pack(w, (int)blockIdx.x, w_blocks);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, block = (int)blockIdx.x - w_blocks, i0 = block / across * 64, part = block % across;
  if (block == 0)
    for (int i = tid; i < tickets; i += 256) ticket[i] = 0u;
  // states of all rows; of the block's own source rows also what does not count
  const int each = (r.N + 4095) / 4096 * 16;   // rows a thread looks at for their places, in sixteens
  for (int n = r.N + tid; n < each * 256; n += 256) state[n] = 0;
  auto settle = [&](int n, bool counts, bool wrong) {
    state[n] = counts;
    if (part == 0 && n >= i0 && n < i0 + 64 && !counts) r.loss[n] = wrong ? __builtin_nanf("") : 0.f;
  };
  if (r.kind == kLossLabel) {
#pragma unroll 2
    for (int n0 = tid * 4; n0 < r.N; n0 += 1024) {
      i32x4 y = {-1, -1, -1, -1};
      if (n0 + 4 <= r.N) y = load_any<i32x4>(r.labels + n0);
      else
        for (int j = 0; n0 + j < r.N; ++j) y[j] = r.labels[n0 + j];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n0 + j < r.N) settle(n0 + j, y[j] >= 0 && y[j] < r.V1, y[j] >= r.V1);
    }
  } else {
    const int group = loss_group(r.K), rows = 256 / group, l = tid & (group - 1);
    for (int n0 = 0; n0 < r.N; n0 += rows) {
      const int n = n0 + tid / group;
      bool some = false, wrong = false;
      if (n < r.N)
        for (int e = l; e < r.K; e += group) {
          const int y = r.labels[(size_t)n * r.K + e];
          wrong |= y >= r.V1;
          some |= y >= 0 && r.logits[(size_t)n * r.K + e] != -__builtin_inff();
        }
      for (int d = 1; d < group; d <<= 1) {
        some |= __shfl_xor((int)some, d) != 0;
        wrong |= __shfl_xor((int)wrong, d) != 0;
      }
      if (n < r.N && l == 0) settle(n, some && !wrong, wrong);
    }
  }
  __syncthreads();
  // the places of a thread's rows
  auto bits_of = [&](int i) {
    const u32x4 st = *reinterpret_cast<const u32x4 *>(state + tid * each + i);
    uint32_t bits = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) bits |= ((st[j >> 2] >> (8 * (j & 3))) & 1u) << j;
    return bits;
  };
  int mine = 0;
  for (int i = 0; i < each; i += 16) mine += __popc(bits_of(i));
  int sum = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(sum, d);
    if (lane >= d) sum += o;
  }
  if (lane == 63) sums[wave] = sum;
  __syncthreads();
  int put = sum - mine, live = 0;
  for (int w2 = 0; w2 < 4; ++w2) {
    if (w2 < wave) put += sums[w2];
    live += sums[w2];
  }
  if (block == 0 && tid == 0) *r.count = live;
  if (put < i0 + 64 && put + mine > i0)
    for (int i = 0; i < each; i += 16)
      for (uint32_t bits = bits_of(i); bits; bits &= bits - 1, ++put)   // (the blocks of the same rows write the same)
        if (put >= i0 && put < i0 + 64) r.idx[put] = tid * each + i + __builtin_ctz(bits);
  __syncthreads();
  const int used = min((live + 255) & ~255, k.R);
  if (part == 0) loss_entries(r, k, live, i0, min(i0 + 64, used), 1);
  if (i0 < used) {   // 64 rows, four threads each
    const int row = i0 + (tid >> 2), q = tid & 3;
    const size_t src = row < live ? (size_t)r.idx[row] : 0;
    for (int blk = part; blk < h.blocks; blk += across) {
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      const int c = blk * 32 + q * 8;
      if (row < live && c < h.cols) loss_load8(h, src, c, v);
      loss_split8(v, h.planes, h.dst + (size_t)blk * h.dst_rows * 32 + (size_t)row * 32 + q * 8, h.plane);
    }
  }
  if (!dh) return;
  for (int n = i0 + wave + 4 * part; n < min(i0 + 64, r.N); n += 4 * across) {   // gradients of rows that do not count
    if (state[n]) continue;
    loss_clear_row(dh, n, h.dtype, h.cols);
  }
}

// ---- logits: statistics, and the gradient's logits ----------------------------------------------
struct LossProduct {
  PanelsDev a, b;
  int slabs;                   // of K, 32 each
  int cols;                    // outputs (V1)
  int ct;                      // column tiles
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
// The first two entries of the lane's rows, and which 32-row blocks of the wave have an entry among its columns.
template <class T>
struct LossEntries {
  int label[T::MI][2];
  int first[T::MI], end[T::MI];   // sorted entries of a block
  unsigned hit;
  __device__ __forceinline__ void load(const LossChunk &k, int i0, int col0, int part) {
    if (k.sorted) {
      hit = 0;
#pragma unroll
      for (int mi = 0; mi < T::MI; ++mi) {
        const int *begin = k.begin + (size_t)(i0 / 32 + mi) * (k.parts + 1) + part;
        first[mi] = __builtin_amdgcn_readfirstlane(begin[0]);
        end[mi] = __builtin_amdgcn_readfirstlane(begin[1]);
        hit |= end[mi] > first[mi] ? 1u << mi : 0u;
      }
      return;
    }
    bool in[T::MI];
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi) {
      label[mi][0] = k.label[i0 + 32 * mi];
      label[mi][1] = k.K > 1 ? k.label[k.R + i0 + 32 * mi] : -1;
      in[mi] = inside(label[mi][0] - col0) || inside(label[mi][1] - col0);
    }
#pragma unroll 4
    for (int e = 2 + ((threadIdx.x & 63) >> 5); e < k.K; e += 2)   // a row's two lanes share them
#pragma unroll
      for (int mi = 0; mi < T::MI; ++mi) in[mi] |= inside(k.label[(size_t)e * k.R + i0 + 32 * mi] - col0);
    hit = 0;
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi) hit |= __any(in[mi]) ? 1u << mi : 0u;
  }
  static __device__ __forceinline__ bool inside(int at) { return (unsigned)at < (unsigned)(32 * T::NI); }
  // More entries of row i, from e0 on: eight a lane, the row's two lanes one after the other.  at: column, or anything that is not
  // inside.  (All of a batch are asked for together: one by one, 64 entries a row cost as much again as the product of fp32 rows of 640.)
  static constexpr int kBatch = 16;
  __device__ __forceinline__ void batch(const LossChunk &k, int i, int e0, int col0, int (&at)[8]) const {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int x = 0; x < 8; ++x) at[x] = -1;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const int e = e0 + 8 * half + x;
      if (e < k.K) at[x] = k.label[(size_t)e * k.R + i] - col0;
    }
  }
};
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

// A probability as mantissa and exponent, m 2^e (wind_loss_lattice.h); zero has an exponent below every other's.
struct Cell { float m; int e; };
constexpr int kCellZero = -(1 << 28);
// 2^l, 1 <= m < 2.  Below 2^kCellZero (an output masked by -1e30, say) it is zero: sums of three exponents that began lower would leave the integers' range.
__device__ __forceinline__ Cell cell_of_log2(float l) {
  const float f = fmaxf(floorf(l), (float)kCellZero);
  return Cell{__builtin_amdgcn_exp2f(l - f), (int)f};
}
struct LossNodes {
  float4 *arcs;                // per place of a lattice node: the probabilities of blank and of its label (m, e, m, e; e as bits)
  int *slot;                   // [R] places of the chunk's nodes
  float2 *norm;                // per node: top and norm as in LossChunk
};
// What the workgroups of a row tile leave for the one that joins it (JOIN) goes past their L2s, which do not see each other's.
template <bool JOIN, class U>
__device__ __forceinline__ void loss_leave(U *p, U v) {
  if (JOIN) __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  else *p = v;
}
template <bool JOIN, class U>
__device__ __forceinline__ U loss_take(const U *p) {
  if (JOIN) return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return *p;
}
// Joins the column blocks of ROWS rows from i0 on, 256 / ROWS threads a row.  sm: 512 floats of LDS.
template <int ROWS, bool JOIN>
__device__ __forceinline__ void loss_rows_done(const LossRowsDev &r, const LossChunk &k, int live, int parts, const LossNodes &nodes, int i0, float *sm) {
  constexpr int G = 256 / ROWS;
  float *const ss = sm + 256;
  const int lane = threadIdx.x % ROWS, grp = threadIdx.x / ROWS, i = i0 + lane;
  float m = -__builtin_inff(), s = 0.f;
  if (i < live) {
#pragma unroll 4
    for (int p = grp; p < parts; p += G) {
      const float2 v = __builtin_bit_cast(float2, loss_take<JOIN>(reinterpret_cast<const unsigned long long *>(k.part) + (size_t)p * k.R + i));
      const float top = fmaxf(m, v.x), ref = top == -__builtin_inff() ? 0.f : top;
      s = s * __builtin_amdgcn_exp2f((m - ref) * k.c) + v.y * __builtin_amdgcn_exp2f((v.x - ref) * k.c);
      m = top;
    }
  }
  sm[threadIdx.x] = m;
  ss[threadIdx.x] = s;
  __syncthreads();
  float top = sm[lane];
#pragma unroll 16
  for (int q = 1; q < G; ++q) top = fmaxf(top, sm[q * ROWS + lane]);
  const float ref = top == -__builtin_inff() ? 0.f : top;
  s = 0.f;
#pragma unroll 16
  for (int q = 0; q < G; ++q) s += ss[q * ROWS + lane] * __builtin_amdgcn_exp2f((sm[q * ROWS + lane] - ref) * k.c);
  const float ls = log2f(s);
  // how far below the largest logit entry e's is: -log2 p = below c + ls, -log p = below / tau + ls ln 2
  auto below = [&](int e) { return top - loss_take<JOIN>(k.logit + (size_t)e * k.R + i); };
  auto cost = [&](int e) { return __builtin_fmaf(below(e), r.inv_tau, ls * (float)kLn2); };
  const bool first = grp == 0 && i < live;
  if (first) {
    k.top[i] = top;
    k.norm[i] = ls;
  }
  float sum = 0.f;
  if (r.kind == kLossLattice) {
    if (first) {
      auto arc = [&](int e) { return cell_of_log2(-__builtin_fmaf(below(e), k.c, ls)); };
      const Cell stay = arc(0), take = k.label[(size_t)k.R + i] < 0 ? Cell{0.f, kCellZero} : arc(1);
      nodes.norm[k.c0 + i] = make_float2(top, ls);
      nodes.arcs[nodes.slot[i]] = make_float4(stay.m, __int_as_float(stay.e), take.m, __int_as_float(take.e));
    }
  } else if (r.kind == kLossLabel) {
    if (first) r.loss[r.idx[k.c0 + i]] = cost(0);
  } else {
    if (i < live) {
#pragma unroll 4
      for (int e = grp; e < k.K; e += G) {
        const float lq = k.value[(size_t)e * k.R + i], q = exp2f(lq);   // (an entry that is not there has q = 0)
        if (q != 0.f) sum += q * __builtin_fmaf(lq, (float)kLn2, cost(e));
      }
    }
    __syncthreads();
    sm[threadIdx.x] = sum;
    __syncthreads();
    if (first) {
#pragma unroll 16
      for (int q = 1; q < G; ++q) sum += sm[q * ROWS + lane];
      r.loss[r.idx[k.c0 + i]] = sum * r.tau * r.tau;
    }
  }
  __syncthreads();
}
template <int ROWS>
__global__ __launch_bounds__(256) void loss_rows_done_kernel(LossRowsDev r, LossChunk k, int parts, LossNodes nodes) {
  __shared__ float sm[512];
  const int live = chunk_rows(k);
  if ((int)blockIdx.x * ROWS < live) loss_rows_done<ROWS, false>(r, k, live, parts, nodes, (int)blockIdx.x * ROWS, sm);
}

// Row statistics.  NARROW: the last column of tiles has at most 64 columns and takes a tile of that width.  JOIN: the last workgroup of a row tile (by a ticket, zero at launch) joins its column blocks itself; few rows and column blocks,
// where a launch of its own costs more.
template <class T, bool JOIN>
__device__ __forceinline__ void loss_stats(const LossProduct &g, const LossChunk &k, const float *bias, int row0, int j0, int part0, unsigned char *smem) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int col0 = j0 + (wave & 1) * 32 * T::NI, part = part0 + (wave & 1);
  const int i0 = row0 + (wave >> 1) * 32 * T::MI + (lane & 31);
  f32x16 acc[T::MI][T::NI];
  LossEntries<T> entries;
  loss_mainloop<T, false, false>(g.a, g.b, row0, j0, 0, g.slabs, smem, acc, [&]() {
    entries.load(k, i0, col0, part);
    loss_bias<T>(bias, g.cols, col0, acc);
  });
  float *tile = reinterpret_cast<float *>(smem) + wave * 32 * T::PITCH;
#pragma unroll
  for (int mi = 0; mi < T::MI; ++mi) {
    const int i = i0 + 32 * mi;
    float m = -__builtin_inff();
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) m = fmaxf(m, acc[mi][ni][r]);
    m = fmaxf(m, xor32_f32(m));
    const float ref = m == -__builtin_inff() ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f((acc[mi][ni][r] - ref) * k.c);
    sum += xor32_f32(sum);
    if (lane < 32)
      loss_leave<JOIN>(reinterpret_cast<unsigned long long *>(k.part) + (size_t)part * k.R + i,
                       __builtin_bit_cast(unsigned long long, make_float2(m, sum)));
    if (entries.hit >> mi & 1u) {
      loss_tile_out<T>(acc[mi], tile);
      if (k.sorted) {
        const uint32_t *list = k.sorted + (size_t)(i0 / 32 + mi) * 32 * k.K;
        for (int x = entries.first[mi] + lane; x < entries.end[mi]; x += 64) {
          const uint32_t w = list[x];
          const int row = (int)(w >> 12) & 31, e = (int)(w & 4095u);
          loss_leave<JOIN>(k.logit + (size_t)e * k.R + (i - (lane & 31)) + row, tile[row * T::PITCH + (int)(w >> 18)]);
        }
      } else if (k.K <= 2) {   // a lane each
        const int at = (lane < 32 ? entries.label[mi][0] : entries.label[mi][1]) - col0;
        if (entries.inside(at)) loss_leave<JOIN>(k.logit + (size_t)(lane >> 5) * k.R + i, tile[(lane & 31) * T::PITCH + at]);
      } else for (int e0 = 0; e0 < k.K; e0 += entries.kBatch) {
        int at[8];
        entries.batch(k, i, e0, col0, at);
#pragma unroll
        for (int x = 0; x < 8; ++x)
          if (entries.inside(at[x])) loss_leave<JOIN>(k.logit + (size_t)(e0 + 8 * (lane >> 5) + x) * k.R + i, tile[(lane & 31) * T::PITCH + at[x]]);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}
template <class T, bool JOIN, bool NARROW>
__global__ __launch_bounds__(256, T::W) void loss_stats_kernel(LossProduct g, LossChunk k, const float *bias, LossRowsDev r, LossNodes nodes, unsigned *ticket) {
  __shared__ __attribute__((aligned(256))) unsigned char smem[T::SMEM];
  const int live = chunk_rows(k);
  int ti, tj, split;
  if (!loss_place((int)blockIdx.x, (live + T::BM - 1) / T::BM, g.ct, 1, ti, tj, split)) return;
  if (NARROW && tj + 1 == g.ct) loss_stats<typename T::Narrow, JOIN>(g, k, bias, ti * T::BM, tj * T::BN, 2 * tj, smem);
  else loss_stats<T, JOIN>(g, k, bias, ti * T::BM, tj * T::BN, 2 * tj, smem);
  if (!JOIN) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // what this wave leaves has arrived
  int &last = *reinterpret_cast<int *>(smem + 4096);
  __syncthreads();
  if (threadIdx.x == 0) last = __hip_atomic_fetch_add(ticket + ti, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)g.ct - 1u;
  __syncthreads();
  if (!last) return;
  const int end = min(live, (ti + 1) * T::BM), parts = 2 * g.ct;
  float *const sm = reinterpret_cast<float *>(smem);
  if (end - ti * T::BM <= 16) loss_rows_done<16, true>(r, k, end, parts, nodes, ti * T::BM, sm);
  else
    for (int i = ti * T::BM; i < end; i += 64) loss_rows_done<64, true>(r, k, end, parts, nodes, i, sm);
}

// Rows that count in all up to which dx of bf16 operands is kept on 16 bits (two planes) for its products: gradients of few rows are decided by a few values of it, whose
// roundings to 8 bits do not average out (13 rows of 29052 outputs: error of dz 0.0037 of its norm with one plane, 0.0016, the result's own rounding, with two).  The
// second plane costs 0 to 7 % of a step up to 128 rows, 15 % of one of 256 rows of 65537.
constexpr int kLossFineRows = 128;

// dx of a chunk, in panels, and its column sums.
struct LossDx {
  bf16_t *dx;
  size_t plane;
  int planes, blocks;
  float *colsum;               // [2 row tiles][blocks * 32] sums over a wave's rows, or null
  int may_fine;                // one plane; two, of 256 rows each, where no more rows count than kLossFineRows
};
// The row tiles of few rows end at 256 at the latest, and the space of one plane of all rows (512 at least) holds both of theirs.
constexpr int kLossFinePanel = 256;
__device__ __forceinline__ bool loss_fine(int may_fine, const LossChunk &k) { return may_fine && *k.count <= kLossFineRows; }
// What dx on one plane is kept in units of: the mantissa (1 <= unit < 2) of the first scale that is not zero, of the chunk's first 64.  A weight that all rows share (1 / N)
// is then not part of what is rounded: most rows' label has p - 1, near -1, and times such a weight all of them were rounded the same way, up to 2^-8 of the whole
// gradient (971 rows of weight 1 / 971: error of dz 0.0027 of its norm, in units 0.0020; 466 rows 0.0035, 0.0019; the result's own rounding 0.0017).  The products' results are multiplied by it.
__device__ __forceinline__ float loss_unit(const LossChunk &k, int live) {
  const int lane = threadIdx.x & 63;
  const float s = lane < live ? fabsf(k.scale[lane]) : 0.f;
  const unsigned long long some = __ballot(s >= 1.17549435e-38f && s < __builtin_inff());
  if (!some) return 1.f;
  const unsigned bits = (unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(s), __builtin_ctzll(some));
  return __uint_as_float(0x3F800000u | (bits & 0x007FFFFFu));
}

template <class T>
__device__ __forceinline__ void loss_dx(const LossProduct &g, const LossChunk &k, const float *bias, const LossDx &d, int row0, int j0, int part0, unsigned char *smem) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), half = lane >> 5;
  const int col0 = j0 + (wave & 1) * 32 * T::NI, part = part0 + (wave & 1);
  const int i0 = row0 + (wave >> 1) * 32 * T::MI + (lane & 31);
  f32x16 acc[T::MI][T::NI];
  LossEntries<T> entries;
  loss_mainloop<T, false, false>(g.a, g.b, row0, j0, 0, g.slabs, smem, acc, [&]() {
    entries.load(k, i0, col0, part);
    loss_bias<T>(bias, g.cols, col0, acc);
  });
  float *tile = reinterpret_cast<float *>(smem) + wave * 32 * T::PITCH;
  constexpr bool F32 = T::PA == 3;   // (three planes always)
  const bool fine = !F32 && loss_fine(d.may_fine, k);
  const float per_unit = !F32 && d.may_fine && !fine ? 1.f / loss_unit(k, chunk_rows(k)) : 1.f;
  const int planes = fine ? 2 : d.planes;
  const size_t panel = (size_t)(fine ? kLossFinePanel : k.R) * 32, plane = fine ? panel * d.blocks : d.plane;
#pragma unroll
  for (int mi = 0; mi < T::MI; ++mi) {
    const int i = i0 + 32 * mi;
    const float s = k.scale[i] * per_unit, top = k.top[i], norm = k.norm[i];
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[mi][ni][r] = s * __builtin_amdgcn_exp2f(__builtin_fmaf(acc[mi][ni][r] - top, k.c, -norm));
    if (entries.hit >> mi & 1u) {
      loss_tile_out<T>(acc[mi], tile);
      float *row = tile + (lane & 31) * T::PITCH;
      if (k.sorted) {
        const int n = entries.end[mi] - entries.first[mi];
        const uint32_t *list = k.sorted + (size_t)(i0 / 32 + mi) * 32 * k.K + entries.first[mi];
        const float *coef = k.coef + (i - (lane & 31));
        for (int x = lane; x < n; x += 64) {   // the first of an output's entries takes all of them off, in order
          const uint32_t w = list[x];
          if (x > 0 && list[x - 1] >> 12 == w >> 12) continue;
          const int row_x = (int)(w >> 12) & 31;
          float &at = tile[row_x * T::PITCH + (int)(w >> 18)];
          float v = at - coef[(size_t)(w & 4095u) * k.R + row_x] * per_unit;
          for (int y = x + 1; y < n && list[y] >> 12 == w >> 12; ++y) v -= coef[(size_t)(list[y] & 4095u) * k.R + row_x] * per_unit;
          at = v;
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
      } else if (k.K <= 2) {
        const int at[2] = {entries.label[mi][0] - col0, entries.label[mi][1] - col0};
        const float c[2] = {k.coef[i] * per_unit, k.K > 1 ? k.coef[k.R + i] * per_unit : 0.f};
        if (half == 0) {
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (entries.inside(at[e])) row[at[e]] -= c[e];
        }
      } else for (int e0 = 0; e0 < k.K; e0 += entries.kBatch) {
        int at[8];
        float c[8];
        entries.batch(k, i, e0, col0, at);
#pragma unroll
        for (int x = 0; x < 8; ++x) c[x] = e0 + 8 * half + x < k.K ? k.coef[(size_t)(e0 + 8 * half + x) * k.R + i] * per_unit : 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {   // one lane of a row after the other: an output that is named twice is taken off twice, in order
          if (half == h) {
#pragma unroll
            for (int x = 0; x < 8; ++x)
              if (entries.inside(at[x])) row[at[x]] -= c[x];
          }
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
          __builtin_amdgcn_wave_barrier();
        }
      }
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
        for (int p = 0; p < planes; ++p) {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(rest[2 * j], rest[2 * j + 1]);
          if (p + 1 < planes) {
#pragma unroll
            for (int j = 0; j < 8; ++j) rest[j] -= __uint_as_float((j & 1) ? (w[j >> 1] & 0xFFFF0000u) : (w[j >> 1] << 16));
          }
          const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
          const auto y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
          const u32x4 out = {(uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1]};
          *reinterpret_cast<u32x4 *>(d.dx + (size_t)p * plane + (size_t)blk * panel + (size_t)i * 32 + (2 * q + half) * 8) = out;
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
  float *out = d.colsum + (size_t)(2 * (row0 / T::BM) + (wave >> 1)) * d.blocks * 32;
#pragma unroll
  for (int j = 0; j < (T::NI + 1) / 2; ++j) {
    const int ni = 2 * j + ((lane & 31) >> 4), r = lane & 15, v = col0 + 32 * ni + 8 * (r >> 2) + 4 * half + (r & 3);
    if (ni < T::NI && v < d.blocks * 32) out[v] = keep[j];
  }
}

template <class T, bool NARROW>
__global__ __launch_bounds__(256, T::W) void loss_dx_kernel(LossProduct g, LossChunk k, const float *bias, LossDx d) {
  __shared__ __attribute__((aligned(256))) unsigned char smem[T::SMEM];
  const int live = chunk_rows(k);
  int ti, tj, split;
  if (!loss_place((int)blockIdx.x, (live + T::BM - 1) / T::BM, g.ct, 1, ti, tj, split)) return;
  if (NARROW && tj + 1 == g.ct) loss_dx<typename T::Narrow>(g, k, bias, d, ti * T::BM, tj * T::BN, 2 * tj, smem);
  else loss_dx<T>(g, k, bias, d, ti * T::BM, tj * T::BN, 2 * tj, smem);
}

// ---- products of dx -----------------------------------------------------------------------------
struct LossOut {
  void *p;
  size_t ld;                   // values between rows
  int dtype;                   // 0: fp32, 1: bf16
  int cols;
  const int *idx;              // null, or row i goes to row idx[i]
  int add;                     // fp32: added to what is there
  int splits;                  // > 1: fp32, the s-th part of the sum goes to p + s part
  size_t part;
};
// 32 rows of results from LDS, RUN values of a row per lane
template <int RUN>
__device__ __forceinline__ void loss_store_rows(const LossOut &o, const float *tile, int pitch, int width, int i0, int rows, int j0, size_t base, float unit) {
  const int lane = threadIdx.x & 63, per = width / RUN;
  for (int u = lane; u < 32 * per; u += 64) {
    const int r = u / per, c = (u - r * per) * RUN, i = i0 + r, j = j0 + c;
    if (i >= rows || j >= o.cols) continue;
    const size_t at = base + (size_t)(o.idx ? o.idx[i] : i) * o.ld + j;
    float v[RUN];
#pragma unroll
    for (int e = 0; e < RUN; ++e) v[e] = tile[r * pitch + c + e] * unit;
    const bool whole = j + RUN <= o.cols;
    if constexpr (RUN == 8) {
      bf16_t *d = (bf16_t *)o.p + at;
      if (whole) store_any(d, u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])});
      else
#pragma unroll
        for (int e = 0; e < RUN; ++e)
          if (j + e < o.cols) d[e] = (bf16_t)f32_to_bf16_bits(v[e]);
    } else {
      float *d = (float *)o.p + at;
      if (whole) {
        const f32x4 x = {v[0], v[1], v[2], v[3]};
        store_any(d, o.add ? load_any<f32x4>(d) + x : x);
      } else
#pragma unroll
        for (int e = 0; e < RUN; ++e)
          if (j + e < o.cols) d[e] = o.add ? d[e] + v[e] : v[e];
    }
  }
}
// A wave's results, 32 rows at a time through LDS: what a store instruction writes is then whole lines of a few rows, not a piece of 32 of them
// (dW of 43250 x 654 for 9 rows: 89 us by pieces).
template <class T>
__device__ __forceinline__ void loss_store(const LossOut &o, const f32x16 (&acc)[T::MI][T::NI], int i0, int rows, int j0, int split, float unit, unsigned char *smem) {
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  float *tile = reinterpret_cast<float *>(smem) + wave * 32 * T::PITCH;
  const int j = j0 + (wave & 1) * 32 * T::NI;
  if (j >= o.cols) return;
#pragma unroll
  for (int mi = 0; mi < T::MI; ++mi) {
    const int i = i0 + ((wave >> 1) * T::MI + mi) * 32;
    if (i >= rows) break;
    loss_tile_out<T>(acc[mi], tile);
    const size_t base = (size_t)split * o.part;
    if (o.dtype) loss_store_rows<8>(o, tile, T::PITCH, 32 * T::NI, i, rows, j, base, unit);
    else loss_store_rows<4>(o, tile, T::PITCH, 32 * T::NI, i, rows, j, base, unit);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

template <class T>
__device__ __forceinline__ void loss_clear(f32x16 (&acc)[T::MI][T::NI]) {
#pragma unroll
  for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = f32x16{};
}

// A product whose K axis several workgroups may share: tiles of o.splits parts.
template <class T, bool TA, bool TB>
__device__ __forceinline__ void loss_product(int bid, const LossProduct &g, const LossOut &o, int rows, int slabs, float unit, unsigned char *smem) {
  int ti, tj, split;
  if (!loss_place(bid, (rows + T::BM - 1) / T::BM, g.ct, o.splits, ti, tj, split)) return;
  const int per = (slabs + o.splits - 1) / o.splits, s0 = min(split * per, slabs), s1 = min(s0 + per, slabs);
  f32x16 acc[T::MI][T::NI];
  if (s0 < s1) loss_mainloop<T, TA, TB>(g.a, g.b, ti * T::BM, tj * T::BN, s0, s1, smem, acc, [&]() { loss_clear<T>(acc); });
  else loss_clear<T>(acc);
  loss_store<T>(o, acc, ti * T::BM, rows, tj * T::BN, split, unit, smem);
}
// dz = dx W: rows of the chunk against columns of W's panels, summed over outputs.  dW = dx^T z: columns of dx's panels against columns of z's, summed over
// the chunk's rows.  In one launch, on tiles of one shape.
template <class T>
__device__ __forceinline__ void loss_products(const LossProduct &z, const LossOut &zo, int z_blocks, const LossProduct &w, const LossOut &wo, int live, float unit, unsigned char *smem) {
  if ((int)blockIdx.x < z_blocks) loss_product<T, false, true>((int)blockIdx.x, z, zo, live, z.slabs, unit, smem);
  else if (!wo.add || live) loss_product<T, true, true>((int)blockIdx.x - z_blocks, w, wo, w.cols, (live + 31) / 32, unit, smem);
}
// F: the tile of the same shape for dx on two planes, where that is decided by the rows that count; else T.
template <class T, class F>
__global__ __launch_bounds__(256, T::W) void loss_products_kernel(LossProduct z, LossOut zo, int z_blocks, LossProduct w, LossOut wo, LossChunk k) {
  static_assert(F::BM == T::BM && F::BN == T::BN && F::W == T::W, "one grid for both");
  __shared__ __attribute__((aligned(256))) unsigned char smem[F::SMEM > T::SMEM ? F::SMEM : T::SMEM];
  const int live = chunk_rows(k);
  if constexpr (F::PA != T::PA) {
    if (loss_fine(1, k)) {
      z.a.rows = w.a.rows = kLossFinePanel;
      z.a.plane = w.a.plane = (size_t)kLossFinePanel * 32 * z.a.blocks;
      loss_products<F>(z, zo, z_blocks, w, wo, live, 1.f, smem);
      return;
    }
    loss_products<T>(z, zo, z_blocks, w, wo, live, loss_unit(k, live), smem);
  } else loss_products<T>(z, zo, z_blocks, w, wo, live, 1.f, smem);
}

// ---- the last launch of a chunk -----------------------------------------------------------------
// db: the column sums of all row tiles.  A workgroup takes 16 columns, 16 threads each.
struct LossDb {
  const float *colsum;
  int width, cols, tile_rows, add, may_fine;
  float *db;
};
__device__ __forceinline__ void loss_db(const LossDb &d, const LossChunk &k, int block) {
  __shared__ float sums[16][16];
  const int live = chunk_rows(k);
  const float unit = d.may_fine && !loss_fine(1, k) ? loss_unit(k, live) : 1.f;
  const int parts = 2 * ((live + d.tile_rows - 1) / d.tile_rows);
  const int lane = threadIdx.x & 15, grp = threadIdx.x >> 4, v = block * 16 + lane;
  float s = 0.f;
  if (v < d.cols) {
#pragma unroll 8
    for (int p = grp; p < parts; p += 16) s += d.colsum[(size_t)p * d.width + v];
  }
  sums[grp][lane] = s;
  __syncthreads();
  if (grp || v >= d.cols) return;
  s = 0.f;
#pragma unroll
  for (int q = 0; q < 16; ++q) s += sums[q][lane];
  s *= unit;
  d.db[v] = d.add ? d.db[v] + s : s;
}

// Sums of a product's parts, rounded once (rows: as many as count where idx is given).
struct LossJoin {
  const float *parts;
  int splits;
  size_t part, ld;
  int rows, cols, dtype;
  const int *idx;
  void *out;                   // [.., cols]
};
__device__ __forceinline__ void loss_join(const LossJoin &j, int rows, int block, int nblocks) {
  const int per_row = (j.cols + 3) / 4;
  const size_t total = (size_t)rows * per_row;
  for (size_t i = (size_t)block * 256 + threadIdx.x; i < total; i += (size_t)nblocks * 256) {
    const size_t v = i / per_row;
    const int h = (int)(i - v * per_row) * 4;
    f32x4 s = *reinterpret_cast<const f32x4 *>(j.parts + v * j.ld + h);
    for (int q = 1; q < j.splits; ++q) s += *reinterpret_cast<const f32x4 *>(j.parts + (size_t)q * j.part + v * j.ld + h);
    const size_t to = (j.idx ? (size_t)j.idx[v] : v) * j.cols + h;
    if (h + 4 <= j.cols) {
      if (j.dtype) store_any((bf16_t *)j.out + to, u32x2{pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3])});
      else store_any((float *)j.out + to, s);
      continue;
    }
    for (int e = 0; e < 4 && h + e < j.cols; ++e) {
      if (j.dtype) ((bf16_t *)j.out)[to + e] = (bf16_t)f32_to_bf16_bits(s[e]);
      else ((float *)j.out)[to + e] = s[e];
    }
  }
}

// What is left of a chunk of label or distillation rows: db, and the sums over parts of dW (with the last chunk) and dz.
struct LossFinish {
  LossDb db;
  LossJoin dw, dz;
  int n_db, n_dw, n_dz;        // workgroups of each
};
// false: the workgroup's number, less those taken, is left in `block`
__device__ __forceinline__ bool loss_finish(const LossFinish &f, const LossChunk &k, int &block) {
  if (block < f.n_db) { loss_db(f.db, k, block); return true; }
  block -= f.n_db;
  if (block < f.n_dw) { loss_join(f.dw, f.dw.rows, block, f.n_dw); return true; }
  block -= f.n_dw;
  if (block < f.n_dz) { loss_join(f.dz, chunk_rows(k), block, f.n_dz); return true; }
  block -= f.n_dz;
  return false;
}
__global__ __launch_bounds__(256) void loss_finish_kernel(LossFinish f, LossChunk k) {
  int block = (int)blockIdx.x;
  loss_finish(f, k, block);
}

}  // namespace wind
