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
// 16 or 24 bits).  A product of two such matrices is a sum of products of planes, the smallest first; a stage holds all planes of its K
// values, so that each is fetched once.  fp32 operands (three planes each) take the six products that reach 2^-24 of the whole: the bf16
// matrix rate over six is 2.6 times that of the fp32 matrix instructions.  Hidden rows that are sums of two bf16 values take two planes.
//
// Schedule of a wave, as in the wide core (wind_mfma_wide.h): a ring of stages filled by direct-to-LDS buffer loads, S stages ahead.  The
// MFMAs of one K step of 16 run with the fragment reads of the next woven in; before a stage's last K step the wave waits for its own loads
// of the next stage and its own reads, and meets the others at one barrier; the MFMAs of that step come with the next stage's first reads
// and the loads that refill the stage just left.
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

// 64 MI x 64 NI outputs on four waves (2 x 2); PA / PB planes of the operands; a ring of S stages of 32 KPS K values.  W workgroups of it
// share a CU: while one starts or writes its results, the others multiply.
template <int MI_, int NI_, int PA_, int PB_, int KPS_, int S_, int W_>
struct LossTile {
  static constexpr int MI = MI_, NI = NI_, PA = PA_, PB = PB_, KPS = KPS_, S = S_, W = W_;
  static constexpr int BM = 64 * MI_, BN = 64 * NI_, NT = 256;
  static constexpr int SLAB = (PA_ * BM + PB_ * BN) * 64, STAGE = KPS_ * SLAB, RING = S_ * STAGE;
  static constexpr int PITCH = 32 * NI_ + 4;                 // floats per row of a wave's tile of logits in LDS
  static constexpr int TILE = 4 * 32 * PITCH * 4;            // all four waves', 32 rows each
  static constexpr int SMEM = RING > TILE ? RING : TILE;
  static constexpr int LS = PA_ * MI_ + PB_ * NI_, L = KPS_ * LS;   // loads per wave and slab, and stage
  static constexpr int PAIRS = PA_ == 3 && PB_ == 3 ? 6 : PA_ * PB_;
  using Narrow = LossTile<MI_, 1, PA_, PB_, KPS_, S_, W_>;   // for a last column of tiles of at most 64 columns
  static_assert(PAIRS == 6 || PB_ == 1, "products of planes");
  static_assert(W_ * SMEM <= 160 * 1024 && (S_ - 1) * L < 64 && S_ >= 2, "LDS, vmcnt range");
};

// acc += A[i0 .., :] B[j0 .., :]^T over K slabs (of 32) s0 .. s1 - 1.  TA / TB: the operand's K axis is its panels' rows (its tile
// rows are columns of the matrix: a multiple of 32 from i0 / j0).  Rows past the end of an operand are read as its last ones: the caller
// does not use those outputs.  acc is set by `init`, which runs behind the first loads.  At least one slab (s0 < s1).  The transposed block is
// accumulated: acc[mi][ni][r] holds A row 32 mi + (lane & 31) and B row 32 ni + 8 (r / 4) + 4 (lane / 32) + r % 4 of the wave's block.  Leaves
// LDS free for the caller (all waves have passed).
template <class T, bool TA, bool TB, class Init>
__device__ __forceinline__ void loss_mainloop(const PanelsDev &a, const PanelsDev &b, int i0, int j0, int s0, int s1, unsigned char *smem,
                                              f32x16 (&acc)[T::MI][T::NI], Init init) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int wm = wave >> 1, wn = wave & 1;
  const int stages = (s1 - s0 + T::KPS - 1) / T::KPS;

  // where a lane's 16 bytes of load group g (1 KB) lie in a slab
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
  i32x4 rs_a[T::PA], rs_b[T::PB];
#pragma unroll
  for (int p = 0; p < T::PA; ++p) rs_a[p] = wide_rsrc(a.p + (size_t)p * a.plane, bytes_a);
#pragma unroll
  for (int p = 0; p < T::PB; ++p) rs_b[p] = wide_rsrc(b.p + (size_t)p * b.plane, bytes_b);

  // Load q of the wave's part of a stage whose first slab is f_s.  Past the last slab the descriptor is empty: such a load touches no memory
  // (zeros arrive in LDS), and the counts that the wave waits for stay the same in every stage, without a branch in the loop.
  int f_s = s0;
  uint32_t so_a = (uint32_t)s0 * step_a, so_b = (uint32_t)s0 * step_b;
  auto fetch = [&](int q, int slot) {
    const int k = q / T::LS, x = q % T::LS;
    unsigned char *const at = smem + slot * T::STAGE + k * T::SLAB + wave * 1024;
    if (x < T::PA * T::MI) {
      const int p = x / T::MI, i = x % T::MI;
      i32x4 rs = rs_a[p];
      rs[2] = f_s + k < s1 ? rs[2] : 0;
      wide_load(rs, at + p * (T::BM * 64) + i * 4096, va[i], so_a + (uint32_t)k * step_a);
    } else {
      const int y = x - T::PA * T::MI, p = y / T::NI, i = y % T::NI;
      i32x4 rs = rs_b[p];
      rs[2] = f_s + k < s1 ? rs[2] : 0;
      wide_load(rs, at + T::PA * (T::BM * 64) + p * (T::BN * 64) + i * 4096, vb[i], so_b + (uint32_t)k * step_b);
    }
  };
  auto fetched = [&]() {
    f_s += T::KPS;
    so_a += T::KPS * step_a;
    so_b += T::KPS * step_b;
  };
#pragma unroll
  for (int s = 0; s < T::S; ++s) {
#pragma unroll
    for (int q = 0; q < T::L; ++q) fetch(q, s);
    fetched();
  }
  init();
  // Of six products the five smaller ones have sums of their own: added to the large one they would round it six times a K step instead of once
  // (1952 hidden units: db of a lattice off by 4e-6 relative).
  constexpr bool SIX = T::PAIRS == 6;
  f32x16 low[SIX ? T::MI : 1][SIX ? T::NI : 1] = {};

  bf16x8 af[2][T::PA][T::MI], bfr[2][T::PB][T::NI];
  const int frow = lane & 31, half = lane >> 5;
  const int c0 = (half ^ ((frow >> 2) & 3)) * 16;                                                  // K step 1: bit 5 flipped
  const int t0 = (8 * half + ((lane & 15) >> 2)) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;   // K step 1: + 1024
  auto frag = [&](bool trans, const unsigned char *base, int blk, int ks) -> bf16x8 {
    const unsigned char *at = base + blk * 2048;
    if (trans) {
      union { s16x4 h[2]; bf16x8 v; } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + t0 + ks * 1024));
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + t0 + ks * 1024 + 256));
      return u.v;
    }
    return *reinterpret_cast<const bf16x8 *>(at + frow * 64 + (c0 ^ (ks * 32)));
  };
  constexpr int NREAD = T::LS, NMFMA = T::PAIRS * T::MI * T::NI, STEPS = 2 * T::KPS;
  // fragment q of K step `step` of the stage in `slot`
  auto read_frag = [&](int q, int set, int slot, int step) {
    const unsigned char *at = smem + slot * T::STAGE + (step >> 1) * T::SLAB;
    if (q < T::PB * T::NI) bfr[set][q / T::NI][q % T::NI] = frag(TB, at + T::PA * (T::BM * 64) + (q / T::NI) * (T::BN * 64), wn * T::NI + q % T::NI, step & 1);
    else {
      const int x = q - T::PB * T::NI;
      af[set][x / T::MI][x % T::MI] = frag(TA, at + (x / T::MI) * (T::BM * 64), wm * T::MI + x % T::MI, step & 1);
    }
  };
  // the MFMAs on register set `set`, the reads of K step `step` of the stage in `slot` into the other one (if any), `load(x)` behind MFMA x
  auto kstep = [&](int set, bool reads, int slot, int step, auto &&load) {
    constexpr int PER = (NREAD + NMFMA - 1) / NMFMA;
#pragma unroll
    for (int x = 0; x < NMFMA; ++x) {
      const int pair = x / (T::MI * T::NI), mi = x % (T::MI * T::NI) / T::NI, ni = x % T::NI;
      // planes of the pair, the smallest product first: (2, 0) (0, 2) (1, 1) (1, 0) (0, 1) (0, 0), or (1, 0) (0, 0)
      const int pa = T::PAIRS == 6 ? (pair == 0 ? 2 : pair == 2 || pair == 3 ? 1 : 0) : T::PA - 1 - pair;
      const int pb = T::PAIRS == 6 ? (pair == 1 ? 2 : pair == 2 || pair == 4 ? 1 : 0) : 0;
      f32x16 &to = SIX && pair < 5 ? low[SIX ? mi : 0][SIX ? ni : 0] : acc[mi][ni];
      to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bfr[set][pb][ni], af[set][pa][mi], to, 0, 0, 0);
      if (reads) {
#pragma unroll
        for (int y = 0; y < PER; ++y)
          if (x * PER + y < NREAD) read_frag(x * PER + y, set ^ 1, slot, step);
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
#pragma unroll
    for (int step = 0; step + 1 < STEPS; ++step) kstep(step & 1, true, slot, step + 1, none);
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
#pragma unroll
  for (int step = 0; step + 1 < STEPS; ++step) kstep(step & 1, true, slot, step + 1, none);
  kstep(1, false, slot, 0, none);
  if (SIX) {
#pragma unroll
    for (int x = 0; x < T::MI * T::NI; ++x) acc[x / T::NI][x % T::NI] += low[SIX ? x / T::NI : 0][SIX ? x % T::NI : 0];
  }
  wait_vmcnt<0>();
  __syncthreads();
}

// Tile of a workgroup.  Workgroups reach the XCDs in turn, so that number b of XCD b % 8 takes the (b / 8)-th of a consecutive eighth of
// the work: part by part of the summed axis (`splits`), in each the tiles in groups of 8 tile rows column by column.  What one XCD works on at
// a time then shares rows, columns and K in its L2.  Returns false for a workgroup without a tile.
__device__ __forceinline__ bool loss_place(int bid, int rt, int ct, int splits, int &ti, int &tj, int &split) {
  const long long tiles = (long long)rt * ct, work = tiles * splits, per = (work + 7) / 8, at = (bid & 7) * per + (bid >> 3);
  if ((bid >> 3) >= per || at >= work) return false;
  split = (int)(at / tiles);
  const long long in = at - split * tiles, span = 8ll * ct;
  const int g = (int)(in / span), rest = (int)(in - g * span), rows = rt - 8 * g < 8 ? rt - 8 * g : 8;
  ti = 8 * g + rest % rows;
  tj = rest / rows;
  return true;
}

}  // namespace wind
