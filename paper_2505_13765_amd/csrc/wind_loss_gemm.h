// Matrix products of the losses over the output layer (wind_loss_kernels.h): bf16 MFMA tiles whose operands lie in panels.
//
// Panels.  A matrix X of R rows and C columns is kept as P[C / 32][R][32]: a panel is 32 columns of all rows, 64 bytes per row, R a
// multiple of 32, columns and rows past the matrix hold zeros.  The loss needs every matrix in two products that sum over different
// axes (logits = H W^T sums over hidden units, dH = D W and dW = D^T H over outputs and over rows), and a panel serves both:
//   summed over its columns   a K stage of 32 is 64 consecutive bytes of every row of one panel;
//   summed over its rows      a K stage of 32 is 32 consecutive rows = 2 KB of every panel, and the matrix operand, which wants 8
//                             consecutive K values per lane, is read from LDS by the transposing read (ds_read_b64_tr_b16: the 16 lanes of a
//                             group name 4 rows of 16 values and each receives one column's 4).
// Either way a wave-wide load of 1 KB is dense memory, and no matrix is ever stored twice or transposed in memory.
//
// More than 16 bits.  A value may be kept as a sum of bf16 planes (x = hi + mid + lo, each the rounding of what the ones before leave: 8,
// 16 or 24 bits).  A product of two such matrices is a sum of products of planes, computed as one product with a longer K: a list of
// plane pairs ("segments"), the smallest first.  fp32 operands take the six pairs that reach 2^-24 of the product: 2.5 PFLOP/s over six is
// 2.6 times the rate of the fp32 matrix instructions.
//
// Schedule of a wave, as in the wide core (wind_mfma_wide.h): a ring of stages filled by direct-to-LDS buffer loads, S stages ahead.  The
// MFMAs of a stage's first K step run with the fragment reads of the second woven in; then the wave waits for its own loads of the
// next stage and its own reads, and meets the others at one barrier; the MFMAs of the second step follow with the next stage's first
// reads and the loads that refill the stage just left.
#pragma once
#include "wind_mfma_wide.h"

namespace wind {

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// One operand: panels of `rows` rows, `blocks` panels, planes `plane` values apart.
struct PanelsDev {
  const bf16_t *p;
  size_t plane;
  uint32_t rows, blocks;
};
// Plane pairs of a product: 4 bits each, a in the lower two, b in the upper two; the first pair lowest.
struct SegmentsDev {
  uint32_t list;
  int n;
};

// 64 MI x 64 NI outputs on four waves (2 x 2), a ring of S stages of 32 K values.
template <int MI_, int NI_, int S_>
struct LossTile {
  static constexpr int MI = MI_, NI = NI_, S = S_;
  static constexpr int BM = 64 * MI_, BN = 64 * NI_, NT = 256;
  static constexpr int STA = BM * 64, STB = BN * 64, RING = S_ * (STA + STB);
  static constexpr int PITCH = 32 * NI_ + 4;                 // floats per row of a wave's tile of logits in LDS
  static constexpr int TILE = 4 * 32 * PITCH * 4;            // all four waves', 32 rows each
  static constexpr int SMEM = RING > TILE ? RING : TILE;
  static constexpr int L = MI_ + NI_;                        // loads per wave and stage
  static_assert(SMEM <= 160 * 1024 && (S_ - 1) * L < 64 && S_ >= 2 && S_ <= 5, "LDS, vmcnt range");
};

// acc += A[i0 .., :] B[j0 .., :]^T over K stages s0 .. s1 - 1 of every segment.  TA / TB: the operand's K axis is its panels' rows (its tile
// rows are columns of the matrix: a multiple of 32 from i0 / j0).  Rows past the end of an operand are read as its last ones: the caller
// does not use those outputs.  At least one stage (s0 < s1).  The transposed block is accumulated: acc[mi][ni][r] holds A row 32 mi + (lane & 31) and B row
// 32 ni + 8 (r / 4) + 4 (lane / 32) + r % 4 of the wave's block.  Leaves LDS free for the caller (all waves have passed).
template <class T, bool TA, bool TB>
__device__ __forceinline__ void loss_mainloop(const PanelsDev &a, const PanelsDev &b, const SegmentsDev &seg, int i0, int j0, int s0, int s1,
                                              unsigned char *smem, f32x16 (&acc)[T::MI][T::NI]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int wm = wave >> 1, wn = wave & 1;
  const int stages = (s1 - s0) * seg.n;
  unsigned char *const lds_a = smem, *const lds_b = smem + T::S * T::STA;

  // where a lane's 16 bytes of load group g (1 KB) lie in a stage
  auto offset = [&](bool trans, const PanelsDev &x, int row0, int g) -> uint32_t {
    if (trans) {
      uint32_t blk = (uint32_t)(row0 >> 5) + (g >> 1);
      blk = blk < x.blocks ? blk : x.blocks - 1;
      return blk * (x.rows * 64u) + (uint32_t)((g & 1) * 1024 + lane * 16);
    }
    const int r = 16 * g + (lane >> 2);
    uint32_t row = (uint32_t)(row0 + r);
    row = row < x.rows ? row : x.rows - 1;
    return row * 64u + (uint32_t)(((lane & 3) ^ ((r >> 2) & 3)) * 16);
  };
  uint32_t va[T::MI], vb[T::NI];
#pragma unroll
  for (int i = 0; i < T::MI; ++i) va[i] = offset(TA, a, i0, 4 * i + wave);
#pragma unroll
  for (int i = 0; i < T::NI; ++i) vb[i] = offset(TB, b, j0, 4 * i + wave);
  const uint32_t step_a = TA ? 2048u : a.rows * 64u, step_b = TB ? 2048u : b.rows * 64u;
  const uint32_t bytes_a = a.rows * 64u * a.blocks, bytes_b = b.rows * 64u * b.blocks;

  // the next stage to fetch
  int f_seg = 0, f_s = s0;
  i32x4 rs_a, rs_b;
  uint32_t so_a, so_b;
  auto open_segment = [&]() {
    const uint32_t pair = (seg.list >> (4 * f_seg)) & 15u;
    rs_a = wide_rsrc(a.p + (size_t)(pair & 3u) * a.plane, bytes_a);
    rs_b = wide_rsrc(b.p + (size_t)(pair >> 2) * b.plane, bytes_b);
    so_a = (uint32_t)s0 * step_a;
    so_b = (uint32_t)s0 * step_b;
  };
  open_segment();
  auto fetch = [&](int q, int slot) {   // load q of a stage
    if (q < T::MI) wide_load(rs_a, lds_a + slot * T::STA + (4 * q + wave) * 1024, va[q < T::MI ? q : 0], so_a);
    else wide_load(rs_b, lds_b + slot * T::STB + (4 * (q - T::MI) + wave) * 1024, vb[q >= T::MI ? q - T::MI : 0], so_b);
  };
  // Past the last stage the descriptors are empty: such loads touch no memory (zeros arrive in LDS), and the counts that the wave waits
  // for stay the same in every stage, without a branch in the loop.
  auto fetched = [&]() {
    so_a += step_a;
    so_b += step_b;
    if (++f_s == s1) {
      f_s = s0;
      if (++f_seg < seg.n) open_segment();
      else rs_a[2] = rs_b[2] = 0;
    }
  };
#pragma unroll
  for (int s = 0; s < T::S; ++s) {
#pragma unroll
    for (int q = 0; q < T::L; ++q) fetch(q, s);
    fetched();
  }

  bf16x8 af[2][T::MI], bfr[2][T::NI];
  const int frow = lane & 31, half = lane >> 5;
  const int c0 = (half ^ ((frow >> 2) & 3)) * 16;                                          // K step 1: bit 5 flipped
  const int t0 = (8 * half + ((lane & 15) >> 2)) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;   // K step 1: + 1024
  auto frag = [&](bool trans, const unsigned char *stage, int blk, int ks) -> bf16x8 {
    const unsigned char *at = stage + blk * 2048;
    if (trans) {
      union { s16x4 h[2]; bf16x8 v; } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + t0 + ks * 1024));
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + t0 + ks * 1024 + 256));
      return u.v;
    }
    return *reinterpret_cast<const bf16x8 *>(at + frow * 64 + (c0 ^ (ks * 32)));
  };
  constexpr int NREAD = T::MI + T::NI, NMFMA = T::MI * T::NI;
  auto read_frag = [&](int q, int set, int slot, int ks) {   // in the order the MFMAs want them
    if (q == 0) af[set][0] = frag(TA, lds_a + slot * T::STA, wm * T::MI, ks);
    else if (q <= T::NI) bfr[set][q - 1] = frag(TB, lds_b + slot * T::STB, wn * T::NI + q - 1, ks);
    else af[set][q - T::NI] = frag(TA, lds_a + slot * T::STA, wm * T::MI + q - T::NI, ks);
  };
  // the MFMAs on register set `set`, the reads of K step ks of the stage in `slot` into the other one (if any), `load(x)` behind MFMA x
  auto kstep = [&](int set, bool reads, int slot, int ks, auto &&load) {
    constexpr int PER = (NREAD + NMFMA - 1) / NMFMA;
#pragma unroll
    for (int x = 0; x < NMFMA; ++x) {
      const int mi = x / T::NI, ni = x % T::NI;
      acc[mi][ni] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bfr[set][ni], af[set][mi], acc[mi][ni], 0, 0, 0);
      if (reads) {
#pragma unroll
        for (int y = 0; y < PER; ++y)
          if (x * PER + y < NREAD) read_frag(x * PER + y, set ^ 1, slot, ks);
      }
      load(x);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto none = [](int) {};
  wait_vmcnt<(T::S - 1) * T::L>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int q = 0; q < NREAD; ++q) read_frag(q, 0, 0, 0);
  int slot = 0;
  for (int j = 1; j < stages; ++j) {
    kstep(0, true, slot, 1, none);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // my reads of this stage are complete
    wait_vmcnt<(T::S - 2) * T::L>();                     // my loads of the next one have landed
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int next = slot + 1 == T::S ? 0 : slot + 1;
    kstep(1, true, next, 0, [&](int x) {
      constexpr int EVERY = NMFMA >= T::L ? NMFMA / T::L : 1, PER = (T::L + NMFMA - 1) / NMFMA;
      if (x % EVERY == EVERY - 1) {
#pragma unroll
        for (int y = 0; y < PER; ++y)
          if ((x / EVERY) * PER + y < T::L) fetch((x / EVERY) * PER + y, slot);
      }
    });
    fetched();
    slot = next;
  }
  kstep(0, true, slot, 1, none);
  kstep(1, false, slot, 0, none);
  wait_vmcnt<0>();
  __syncthreads();
}

// Tile number of a workgroup: workgroups reach the XCDs in turn, so that number b of XCD b % 8 takes the (b / 8)-th of a consecutive
// eighth of the tiles, in groups of `group` tile rows column by column: what one XCD works on at a time shares rows and columns in its L2.
// Returns false for a workgroup without a tile.
__device__ __forceinline__ bool loss_tile(int bid, int rt, int ct, int group, int &ti, int &tj) {
  const long long tiles = (long long)rt * ct, per = (tiles + 7) / 8, at = (bid & 7) * per + (bid >> 3);
  if ((bid >> 3) >= per || at >= tiles) return false;
  const long long span = (long long)group * ct;
  const int g = (int)(at / span), in = (int)(at - g * span);
  const int rows = rt - g * group < group ? rt - g * group : group;
  ti = g * group + in % rows;
  tj = in / rows;
  return true;
}

}  // namespace wind
