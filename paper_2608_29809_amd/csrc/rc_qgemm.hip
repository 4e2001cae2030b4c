// Product of block-scaled 8-bit matrices: Y[M][N] = act(A[M][K] . W[N][K]^T + bias),
// A with a scale for each row and 128 of K, W with one for each 128 x 128 tile.
//
// bfloat16 results: 16x16x128 matrix instructions on the 8-bit operands.  A
// block of 128 of K is one instruction, whose scale operands are the blocks'
// exponent bytes, so the sum over blocks stays in the accumulator and no
// vector instruction is spent on scales.  Inside an instruction the sum over
// its 128 products is held to about 17 bits (measured: 1.3e-5 of the result's
// norm, against 2.0e-3 for rounding it to bfloat16).
// float32 results: the operands become bfloat16 with their scales applied
// (exactly from 2^-133 on), for 16x16x32 instructions whose sums keep float32's precision
// (8e-8 of the result's norm over 36 blocks, as a float32 library product).
//
// W is operand A of the matrix instruction, so a lane's accumulators are four
// consecutive columns of one row.  Lane (l16, lq) of an operand supplies, of
// row l16, the 16-byte chunks lq and lq + 4 of the block's eight, in either
// matrix (the order of K inside a block is free).
#include "rc_common.h"
#include "rc_launch.h"
#include "rc_quant.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace rc {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kQMaxBlocks = kQMaxCols / kQBlock;

template <int N> __device__ __forceinline__ void wait_vm_q() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// The products of one block of K: acc += w a, scale bytes ew (uniform) and ea.
template <bool F32> __device__ __forceinline__ f32x4 q_mma(i32x8 w, i32x8 a, f32x4 acc, int ew, int ea) {
  if constexpr (!F32) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, acc, 0, 0, 0, ew, 0, ea);
#pragma unroll
  for (int q = 0; q < 4; ++q)
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
        q_bf16x8(u32x2{(uint32_t)w[2 * q], (uint32_t)w[2 * q + 1]}, q_factor(ew)),
        q_bf16x8(u32x2{(uint32_t)a[2 * q], (uint32_t)a[2 * q + 1]}, q_factor(ea)), acc, 0, 0, 0);
  return acc;
}

template <typename OUT> __device__ __forceinline__ void q_store4(OUT *o, const f32x4 v, bool vec, int left) {
  typedef OUT out4 __attribute__((ext_vector_type(4)));
  if (vec && left >= 4) {
    *(out4 *)o = out4{(OUT)v[0], (OUT)v[1], (OUT)v[2], (OUT)v[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) o[e] = (OUT)v[e];
  }
}

// ------------------------------------------------------------------ few tiles

// A workgroup's KG waves each take every KG-th block of K of the same tile of
// 16 FM x 16 FN results, from memory to registers without LDS (no operand is
// shared between waves), and their sums are joined in LDS in a fixed order.
template <int FM, int FN, int KG, bool GELU, typename OUT>
__global__ __launch_bounds__(64 * KG) void qgemm_split_kernel(QGemmArgs g) {
  constexpr bool F32 = sizeof(OUT) == 4;
  constexpr int BM = 16 * FM, BN = 16 * FN, LD = BN + 4;
  __shared__ __attribute__((aligned(16))) float part[KG * BM * LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, lq = lane >> 4;
  const int tiles_m = (g.M + BM - 1) / BM, L = xcd_logical_id(blockIdx.x, gridDim.x);
  const int tn = L / tiles_m, tm = L - tn * tiles_m, m0 = tm * BM, n0 = tn * BN;
  const int nk = (g.K + kQBlock - 1) / kQBlock;
  const uint8_t *pa[FM], *pw[FN];
  int ra[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    ra[i] = min(m0 + i * 16 + l16, g.M - 1);
    pa[i] = g.a + ra[i] * g.lda;
  }
#pragma unroll
  for (int j = 0; j < FN; ++j) pw[j] = g.w + min(n0 + j * 16 + l16, g.N - 1) * g.ldw;
  const uint8_t *ws = g.ws + n0 / kQBlock;  // (a tile's columns share their scales)
  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  struct Block {
    i32x4 a[FM][2], w[FN][2];
    int ea[FM], ew;
  };
  auto load = [&](Block &b, int kb) {
    const int k0 = kb * kQBlock, c0 = min(k0 + lq * 16, g.K - 16), c1 = min(k0 + lq * 16 + 64, g.K - 16);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      b.w[j][0] = *(const i32x4 *)(pw[j] + c0);
      b.w[j][1] = *(const i32x4 *)(pw[j] + c1);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      b.a[i][0] = *(const i32x4 *)(pa[i] + c0);
      b.a[i][1] = *(const i32x4 *)(pa[i] + c1);
      b.ea[i] = g.as[(size_t)kb * g.as_ld + ra[i]];
    }
    b.ew = ws[(size_t)kb * g.ws_ld];
  };
  auto multiply = [&](Block &b, int kb) {
    const int left = (g.K - kb * kQBlock) / 16;  // chunks of 16 that exist: zeros for the others
    if (left < 8) {
      const i32x4 zero = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        b.w[j][0] = lq < left ? b.w[j][0] : zero;
        b.w[j][1] = lq + 4 < left ? b.w[j][1] : zero;
      }
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        b.a[i][0] = lq < left ? b.a[i][0] : zero;
        b.a[i][1] = lq + 4 < left ? b.a[i][1] : zero;
      }
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
        acc[i][j] = q_mma<F32>(__builtin_shufflevector(b.w[j][0], b.w[j][1], 0, 1, 2, 3, 4, 5, 6, 7),
                               __builtin_shufflevector(b.a[i][0], b.a[i][1], 0, 1, 2, 3, 4, 5, 6, 7), acc[i][j], b.ew, b.ea[i]);
  };
  Block b0, b1;
  if (wave < nk) load(b0, wave);
  for (int kb = wave; kb < nk; kb += 2 * KG) {
    if (kb + KG < nk) load(b1, kb + KG);
    multiply(b0, kb);
    if (kb + KG >= nk) break;
    if (kb + 2 * KG < nk) load(b0, kb + 2 * KG);
    multiply(b1, kb + KG);
  }
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) *(f32x4 *)(part + (wave * BM + i * 16 + l16) * LD + j * 16 + lq * 4) = acc[i][j];
  __syncthreads();
  OUT *out = (OUT *)g.out;
  const bool vec = (g.ldo & 3) == 0;
#pragma nounroll
  for (int c = tid; c < BM * BN / 4; c += 64 * KG) {
    const int r = c / (BN / 4), n = (c - r * (BN / 4)) * 4;
    f32x4 v = *(const f32x4 *)(part + r * LD + n);
#pragma unroll
    for (int w = 1; w < KG; ++w) {
      const f32x4 p = *(const f32x4 *)(part + (w * BM + r) * LD + n);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += p[e];
    }
    if (m0 + r >= g.M) break;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (g.bias) v[e] += g.bias[min(n0 + n + e, g.N - 1)];
      if (GELU) v[e] = gelu_tanh(v[e]);
    }
    q_store4(out + (m0 + r) * g.ldo + n0 + n, v, vec, g.N - n0 - n);
  }
}

// ------------------------------------------------------------------ many tiles

// Wave tiles of 16 FM rows x 16 FN columns; WGM x WGN waves share a ring of S
// stages of one block of K, KG such groups take every KG-th block each.
// * Operands move global -> LDS by direct copies of 1 KB per wave, eight rows of
//   128 bytes (stages of half a block, half rows, take as many requests: 137
//   instead of 101 us for 16384 x 1152 x 4608); the 16-byte chunks of a row are
//   swizzled so that a fragment read of 16 rows touches every bank once.
// * KG = 1: a step waits for its stage, and the next ones' copies run beside its
//   products; W fragments are read one ahead.  Two workgroups per CU cover each
//   other's waits and epilogues.
// * KG > 1, one wave per group, for few tiles: nothing but its own copies is
//   waited for, a block's fragments are read while the block before is
//   multiplied, in the registers that its fragments leave, and the groups' sums
//   are joined in LDS in a fixed order.  A step waits for the next block before
//   it sends for the one after that, so S - 1 blocks are on their way at most.
// What bounds it: with 128 x 128 tiles (4096 x 4608 x 1152 with GELU: 38 us, 1.1
// PFLOP/s) LDS, which gives 128 bytes per clock and takes 187 for 64 x 64 wave
// tiles with their copies, then the epilogues; with KG = 4 the copies' latency,
// a whole one each step at S = 2 (723 x 1152 x 4608, 64 x 64 tiles: nine steps in
// 14.5 us).
template <int FM, int FN, int WGM, int WGN, int KG, int S, int EPI, typename OUT>
__global__ __launch_bounds__(64 * WGM * WGN * KG, 2) void qgemm_kernel(QGemmArgs g) {
  constexpr int NG = WGM * WGN, NW = NG * KG, BM = 16 * FM * WGM, BN = 16 * FN * WGN;
  static_assert(KG == 1 || NG == 1, "groups of one wave");
  constexpr bool F32 = EPI <= QG_GELU && sizeof(OUT) == 4, GELU = EPI == QG_GELU || EPI == QG_GELU8;
  constexpr int STAGE = (BM + BN) * kQBlock, NL = STAGE / 1024 / NG, NA = BM * kQBlock / 1024 / NG;
  static_assert(STAGE % (1024 * NG) == 0 && BM * kQBlock % (1024 * NG) == 0 && kQBlock % (16 * FN) == 0, "tile");
  constexpr int NB = (BN + kQBlock - 1) / kQBlock;
  constexpr int RING = KG * S * STAGE;
  // results on their way out, float32: a band of 16 rows per wave, or every group's tile
  constexpr int WN = 16 * FN, CLD = (KG == 1 ? WN : BN) + 4;
  static_assert((KG == 1 ? NW * 16 : KG * BM) * CLD * 4 <= RING, "the results fit the ring");
  __shared__ __attribute__((aligned(1024))) char lds[RING + KG * S * BM];
  __shared__ uint8_t sw[NB][kQMaxBlocks];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  __builtin_assume(wave >= 0 && wave < NW);
  const int grp = wave / NG, wg = wave % NG, wm = wg / WGN, wn = wg % WGN, l16 = lane & 15, lq = lane >> 4;
  const int tiles_m = (g.M + BM - 1) / BM, tiles_n = (g.N + BN - 1) / BN, L = xcd_logical_id(blockIdx.x, gridDim.x);
  // bands of GM row tiles: the tiles in flight share rows and columns
  constexpr int GM = 2048 / BM;
  const int band0 = L / (GM * tiles_n), gm = min(GM, tiles_m - band0 * GM), idx = L - band0 * GM * tiles_n;
  const int m0 = (band0 * GM + idx % gm) * BM, n0 = idx / gm * BN;
  const int blocks = (g.K + kQBlock - 1) / kQBlock, tail = g.K - (blocks - 1) * kQBlock;
  const int n = (blocks - grp + KG - 1) / KG;  // this group's: grp + KG i

  // rows past the last are clamped to it and never stored; columns of K past
  // the last are copies of its last 16 and multiplied as zeros
  const int row8 = wg * 8 + (lane >> 3), chunk = ((lane & 7) ^ ((row8 >> 1) & 7)) * 16;
  const uint8_t *a0 = g.a + m0 * g.lda, *w0 = g.w + n0 * g.ldw;
  unsigned off[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i)
    off[i] = i < NA ? (unsigned)min(row8 + i * NG * 8, g.M - 1 - m0) * (unsigned)g.lda
                    : (unsigned)min(row8 + (i - NA) * NG * 8, g.N - 1 - n0) * (unsigned)g.ldw;
  char *ring = lds + grp * S * STAGE, *scales = lds + RING + grp * S * BM;
  const unsigned ring0 = lds_address(ring) + wg * 1024, scales0 = lds_address(scales);
  // (row scales: 16 a lane, by the group's first wave, up to a multiple of 16 rows)
  const unsigned sc_off = (unsigned)min(lane * 16, (g.M - 1 - m0) & ~15);
  auto issue = [&](int slot, int i) {
    const int kb = grp + KG * i;
#pragma unroll
    for (int q = 0; q < NL; ++q) {
      unsigned c = NG == 1 && (q & 1) ? chunk ^ 64 : chunk;  // (rows 8 further: the other half of the swizzle)
      if (kb == blocks - 1) c = min((int)c, tail - 16);
      lds_dma16s((q < NA ? a0 : w0) + (size_t)kb * kQBlock, off[q] + c, ring0 + slot * STAGE + q * NG * 1024);
    }
    if (wg == 0 && lane < BM / 16) lds_dma16s(g.as + (size_t)kb * g.as_ld + m0, sc_off, scales0 + slot * BM);
  };
  auto wait_blocks = [&](int later) {  // at most `later` younger blocks' copies are in flight
    if (S > 2 && later >= 2) {
      if (wg == 0) wait_vm_q<2 * NL + 2>();
      else wait_vm_q<2 * NL>();
    } else if (later >= 1) {
      if (wg == 0) wait_vm_q<NL + 1>();
      else wait_vm_q<NL>();
    } else {
      wait_vm_q<0>();
    }
  };
  for (int i = tid; i < blocks; i += 64 * NW)
#pragma unroll
    for (int j = 0; j < NB; ++j) sw[j][i] = g.ws[(size_t)i * g.ws_ld + min(n0 / kQBlock + j, (g.N - 1) / kQBlock)];
  __syncthreads();

  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int sz = (l16 >> 1) & 7, c_lo = l16 * kQBlock + ((lq ^ sz) << 4), c_hi = l16 * kQBlock + (((lq + 4) ^ sz) << 4);
  constexpr int RW = KG > 1 ? FN : 2;  // W fragments held
  i32x8 a[FM], w[RW];
  int ea[FM];
  auto frag = [&](const char *rows, bool last) {
    i32x4 lo = *(const i32x4 *)(rows + c_lo), hi = *(const i32x4 *)(rows + c_hi);
    if (last) {
      if (lq >= tail / 16) lo = i32x4{0, 0, 0, 0};
      if (lq + 4 >= tail / 16) hi = i32x4{0, 0, 0, 0};
    }
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto read_a = [&](int slot, int i, bool last) {
    a[i] = frag(ring + slot * STAGE + (wm * FM + i) * 16 * kQBlock, last);
    ea[i] = *(const uint8_t *)(scales + slot * BM + (wm * FM + i) * 16 + l16);
  };
  auto read_w = [&](int slot, int j, bool last) { w[j % RW] = frag(ring + slot * STAGE + (BM + wn * WN + j * 16) * kQBlock, last); };

  if constexpr (KG > 1) {
#pragma unroll
    for (int i = 0; i < S; ++i)
      if (i < n) issue(i, i);
    wait_blocks(min(n - 1, S - 1));
    const bool last0 = grp == blocks - 1 && tail < kQBlock;
#pragma unroll
    for (int i = 0; i < FM; ++i) read_a(0, i, last0);
#pragma unroll
    for (int j = 0; j < FN; ++j) read_w(0, j, last0);
    int slot = 0;
#pragma nounroll
    for (int i = 0; i < n; ++i) {
      const int kb = grp + KG * i, ns = slot == S - 1 ? 0 : slot + 1;
      const int ew = sw[wn * WN / kQBlock][kb];
      if (i + 1 < n) {
        wait_blocks(min(n - 2 - i, S - 2));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (i + S < n) issue(slot, i + S);
      }
      // (the last step's reads of a stale slot are never used)
      const bool last = kb + KG == blocks - 1 && tail < kQBlock;
      __builtin_amdgcn_sched_barrier(0);
      constexpr int JT = FN > 2 ? FN - 2 : 1;  // from this column block on, row by row
#pragma unroll
      for (int j = 0; j < JT; ++j) {
#pragma unroll
        for (int q = 0; q < FM; ++q) acc[q][j] = q_mma<F32>(w[j], a[q], acc[q][j], ew, ea[q]);
        read_w(ns, j, last);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int q = 0; q < FM; ++q) {
#pragma unroll
        for (int j = JT; j < FN; ++j) acc[q][j] = q_mma<F32>(w[j], a[q], acc[q][j], ew, ea[q]);
        read_a(ns, q, last);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = JT; j < FN; ++j) read_w(ns, j, last);
      __builtin_amdgcn_sched_barrier(0);
      slot = ns;
    }
  } else {
#pragma unroll
    for (int i = 0; i < S - 1; ++i)
      if (i < n) issue(i, i);
    int slot = 0;
#pragma nounroll
    for (int i = 0; i < n; ++i) {
      wait_blocks(min(n - 1 - i, S - 2));
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (i + S - 1 < n) issue(slot == 0 ? S - 1 : slot - 1, i + S - 1);
      const bool last = i == blocks - 1 && tail < kQBlock;
      const int ew = sw[wn * WN / kQBlock][i];
      read_w(slot, 0, last);
#pragma unroll
      for (int q = 0; q < FM; ++q) read_a(slot, q, last);
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        if (j + 1 < FN) read_w(slot, j + 1, last);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < FM; ++q) acc[q][j] = q_mma<F32>(w[j & 1], a[q], acc[q][j], ew, ea[q]);
        __builtin_amdgcn_sched_barrier(0);
      }
      slot = slot == S - 1 ? 0 : slot + 1;
    }
  }

  // The results pass through LDS so that WN / 8 lanes (or BN / 8) store a row's
  // columns and the code is a short loop (run once, each instruction of it is
  // fetched from memory).
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  if constexpr (EPI == QG_GELU8) {
    // 64 rows at a time, whole blocks of 128 columns: sixteen lanes a row
    static_assert(EPI != QG_GELU8 || (KG == 1 && BN == kQBlock && FM == 4 && 64 * (BN + 4) * 4 <= RING), "blocks of 128 columns");
    float *tile = (float *)lds;
    const int c8 = (tid & 15) * 8;
    float bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = g.bias[n0 + c8 + e];
#pragma nounroll
    for (int pass = 0; pass < WGM; ++pass) {
      if (wm == pass)
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) *(f32x4 *)(tile + (i * 16 + l16) * (BN + 4) + wn * WN + j * 16 + lq * 4) = acc[i][j];
      __syncthreads();
#pragma nounroll
      for (int r = tid >> 4; r < 64; r += 4 * NW) {
        float v[8], m = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 x = *(const f32x4 *)(tile + r * (BN + 4) + c8 + 4 * h);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[4 * h + e] = gelu_tanh(x[e] + bias[4 * h + e]);
            m = fmaxf(m, q_magnitude(v[4 * h + e]));
          }
        }
        const int ex = q_exponent(row16_max(m)), row = m0 + pass * 64 + r;
        if (row >= g.M) continue;
        *(u32x2 *)((uint8_t *)g.out + row * g.ldo + n0 + c8) = u32x2{q_pack4(v, q_inverse(ex)), q_pack4(v + 4, q_inverse(ex))};
        if ((tid & 15) == 0) g.out_scales[(size_t)(n0 / kQBlock) * g.out_scale_ld + row] = (uint8_t)ex;
      }
      __syncthreads();
    }
    return;
  }
  // Rows that are a multiple of 16 bytes apart: eight columns a lane.  Others:
  // one column a lane, so that a store covers whole lines all the same.
  float *res = (float *)lds;
  constexpr int ROWS = KG == 1 ? 16 : BM, COLS = KG == 1 ? WN : BN, WHO = KG == 1 ? 64 : 64 * KG;
  const int who = KG == 1 ? lane : tid, col0 = n0 + (KG == 1 ? wn * WN : 0);
  OUT *out = (OUT *)g.out;
  const bool vec = EPI == QG_RESID || (g.ldo & 7) == 0;
  const int c8 = vec ? who % (COLS / 8) * 8 : who % COLS, col = col0 + c8;
  float bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = g.bias ? g.bias[min(col + e, g.N - 1)] : 0.0f;
  float gate[8];
  if (EPI == QG_RESID)
#pragma unroll
    for (int e = 0; e < 8; ++e) gate[e] = g.gate[min(col + e, g.N - 1)] + g.gate2[min(col + e, g.N - 1)];
  // rows row0 .. + ROWS of the result from `tile`, the groups' sums joined in order
  auto put = [&](const float *tile, int row0) {
    if (vec) {
#pragma nounroll
      for (int r = who / (COLS / 8); r < ROWS; r += WHO / (COLS / 8)) {
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4 x = *(const f32x4 *)(tile + r * CLD + c8 + 4 * h);
#pragma unroll
          for (int q = 1; q < KG; ++q) {
            const f32x4 y = *(const f32x4 *)(tile + (q * BM + r) * CLD + c8 + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] += y[e];
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[4 * h + e] = x[e] + bias[4 * h + e];
            if (GELU) v[4 * h + e] = gelu_tanh(v[4 * h + e]);
          }
        }
        if (row0 + r >= g.M) break;
        if constexpr (EPI == QG_RESID) {
          if (col >= g.N) break;
          f32x4 *x = (f32x4 *)(g.X + (size_t)(row0 + r) * g.N + col);
          const f32x4 x0 = x[0], x1 = x[1];
          const int pk = g.packed[row0 + r];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = (e < 4 ? x0[e] : x1[e - 4]) + gate[e] * v[e];
          x[0] = f32x4{v[0], v[1], v[2], v[3]};
          x[1] = f32x4{v[4], v[5], v[6], v[7]};
          *(bf16x8 *)(g.hslot + row_chain(pk) * g.chain_stride + (size_t)row_token(pk) * g.N + col) =
              bf16x8{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3], (bf16)v[4], (bf16)v[5], (bf16)v[6], (bf16)v[7]};
          continue;
        }
        OUT *o = out + (row0 + r) * g.ldo + col;
        if (col + 8 <= g.N) {
          // (past the L2, which the operands need: 134 instead of 165 us for 16384 x 4608 x 1152 with GELU)
          if constexpr (F32) {
            __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, (f32x4 *)o);
            __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, (f32x4 *)(o + 4));
          } else {
            __builtin_nontemporal_store(
                bf16x8{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3], (bf16)v[4], (bf16)v[5], (bf16)v[6], (bf16)v[7]}, (bf16x8 *)o);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (col + e < g.N) o[e] = (OUT)v[e];
        }
      }
    } else {
#pragma nounroll
      for (int r = who / COLS; r < ROWS; r += WHO / COLS) {
        float v = tile[r * CLD + c8];
#pragma unroll
        for (int q = 1; q < KG; ++q) v += tile[(q * BM + r) * CLD + c8];
        v += bias[0];
        if (GELU) v = gelu_tanh(v);
        if (row0 + r < g.M && col < g.N) out[(row0 + r) * g.ldo + col] = (OUT)v;
      }
    }
  };
  if constexpr (KG == 1) {
    float *band = res + wave * 16 * CLD;
#pragma nounroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int q = 0; q < FM; ++q)
        if (i == q)
#pragma unroll
          for (int j = 0; j < FN; ++j) *(f32x4 *)(band + l16 * CLD + j * 16 + lq * 4) = acc[q][j];
      put(band, m0 + (wm * FM + i) * 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) *(f32x4 *)(res + (grp * BM + i * 16 + l16) * CLD + j * 16 + lq * 4) = acc[i][j];
    __syncthreads();
    put(res, m0);
  }
}

// ------------------------------------------------------------------ whole chip

// Lane groups 1 and 3 (of 16) of x change places with groups 0 and 2 of y.
__device__ __forceinline__ void q_swap16(uint32_t &x, uint32_t &y) {
  const auto r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
  x = r[0];
  y = r[1];
}
// Lane groups 2 and 3 of x change places with groups 0 and 1 of y.
__device__ __forceinline__ void q_swap32(uint32_t &x, uint32_t &y) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
  x = r[0];
  y = r[1];
}

// gelu_tanh with one multiplication less.
__device__ __forceinline__ float q_gelu(float x) {
  constexpr float k = -2.0f * 0.7978845608028654f * 1.4426950408889634f;
  return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * __builtin_fmaf(x * x, 0.044715f * k, k)));
}
// A copy of 4 bytes per lane to LDS.
__device__ __forceinline__ void lds_dma4s(const void *from, unsigned lane_off, unsigned to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, %2" ::"v"(lane_off), "s"(to), "s"(from) : "memory", "m0");
}
// A copy of 16 bytes per lane to LDS base + PLACE (uniform), in as few instructions as fit between two products.
template <int PLACE> __device__ __forceinline__ void lds_copy16(const void *from, unsigned lane_off, unsigned base) {
  asm volatile("s_add_u32 m0, %1, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %3" ::"v"(lane_off), "s"(base), "n"(PLACE),
               "s"(from) : "memory", "m0", "scc");
}
// 256 x 256 tiles, one workgroup of four waves per CU, 128 x 128 results per
// wave (all 256 accumulation registers): a step of K, 64 matrix instructions or
// 2048 clocks, takes 32 KB of fragments a wave and 64 KB of copies from memory,
// where 128 x 128 tiles of 64 x 64 per wave take all that LDS gives and twice
// the copies.  (FM = 6: 192 x 256, three quarters of the work in 0.86 of the time,
// where that saves a part of a round of workgroups.)  With one wave per SIMD
// nothing but the order of instructions covers latency:
// * stages of 128 of K in a ring of two.  A step's first half multiplies column
//   by column and reads the rest of its W fragments at once; then the stage is
//   in registers and its place takes the stage after next.  The second half
//   multiplies row by row and reads the next stage's fragments into the
//   registers of the rows that are done with.
// * Copies are issued one between two products, every second or third (all at
//   once they hold a wave up for 1100 clocks a step; with a branch each, 400).
// * The steps of a workgroup's tiles are one sequence: the last two steps of a
//   tile copy the next one's first stages, which are on their way when the
//   epilogue begins.  It needs no LDS: lanes exchange registers until they hold
//   whole stores.  (It does not overlap them: 4 to 15 registers are spilled,
//   some are read back where the epilogue begins, and the wait for those is one
//   for every copy too.  Spills are no danger to the counted waits: vector memory
//   operations end in order, so one more between a copy and its wait can only
//   make the wait longer.)
// 2330 clocks a step where few CUs work; with all of them the power limit leaves
// 1.8 GHz.  A tile's epilogue takes 6500 clocks, 17500 with GELU, of nine steps'
// 21000 at K = 1152, and nothing covers it (accumulators of a second tile find
// no registers).  16384 x 4608 x 1152: 98 to 100 us (128 x 128 tiles 118), 102 to
// 111 with GELU (134), by card; 8192 x 8192 x 9216: 462 us, 2.7 PFLOP/s.
template <int FM, int EPI>
__global__ __launch_bounds__(256, 1) void qgemm_large_kernel(QGemmArgs g, int tiles) {
  constexpr int FN = 8, BM = 32 * FM, BN = 32 * FN, W0 = BM * kQBlock, STAGE = W0 + BN * kQBlock;
  constexpr int NA = FM, NW = FN;  // copies of a stage: rows, W
  constexpr bool GELU = EPI == QG_GELU || EPI == QG_GELU8;
  // per slot: rows, W; behind the ring, per slot: the rows' scales, W's four; for
  // three tiles: the bias (the next one's is copied before the last two steps of
  // a tile, which are all of them if K = 256: another wave may still be in the
  // epilogue of the tile before)
  constexpr int SCALES = 2 * STAGE, BIAS = SCALES + 2 * 512;
  __shared__ __attribute__((aligned(1024))) char lds[BIAS + 3 * 4 * BN];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  __builtin_assume(wave >= 0 && wave < 4);
  const int wm = wave >> 1, wn = wave & 1, l16 = lane & 15, lq = lane >> 4;
  const int tiles_m = (g.M + BM - 1) / BM, tiles_n = (g.N + BN - 1) / BN, n = g.K / kQBlock;
  // bands of GM row tiles, as above
  constexpr int GM = 2048 / BM;
  auto place = [&](int p, int &m0, int &n0) {
    const int L = xcd_logical_id(p, tiles);
    const int band0 = L / (GM * tiles_n), gm = min(GM, tiles_m - band0 * GM), idx = L - band0 * GM * tiles_n;
    m0 = __builtin_amdgcn_readfirstlane((band0 * GM + idx % gm) * BM);
    n0 = __builtin_amdgcn_readfirstlane(idx / gm * BN);
  };

  const unsigned ring0 = __builtin_amdgcn_readfirstlane(lds_address(lds)), mine = ring0 + wave * 1024;

  // The next stage to be copied: rows, W, their scales.
  const int row8 = wave * 8 + (lane >> 3), chunk = ((lane & 7) ^ ((row8 >> 1) & 7)) * 16;
  const uint8_t *c_a, *c_w, *c_as, *c_ws;
  unsigned off_a[NA], off_w[NW];
  int c_rows, by = kQBlock, as_by = g.as_ld, ws_by = g.ws_ld;
  auto enter = [&](int m0, int n0) {  // a tile's first
    c_a = g.a + m0 * g.lda;
    c_w = g.w + n0 * g.ldw;
    c_as = g.as + m0;
    c_ws = g.ws + (n0 / kQBlock & ~3);
    c_rows = g.M - 1 - m0;
    // (rows behind the last are copies of it)
#pragma unroll
    for (int q = 0; q < NA; ++q) off_a[q] = __umul24((unsigned)min(row8 + q * 32, c_rows), (unsigned)g.lda) + chunk;
#pragma unroll
    for (int q = 0; q < NW; ++q) off_w[q] = __umul24((unsigned)min(row8 + q * 32, g.N - 1 - n0), (unsigned)g.ldw) + chunk;
  };
  auto copy_bias = [&](int n0, int which) {  // (a wave's 64 columns)
    lds_dma4s(g.bias, (unsigned)min(n0 + wave * 64 + lane, g.N - 1) * 4u, ring0 + BIAS + which * 4 * BN + wave * 256);
  };
  auto advance = [&]() {
    c_a += by;
    c_w += by;
    c_as += as_by;
    c_ws += ws_by;
  };
  // (the same by every wave, so that every wave has the same copies in flight)
  auto copy_scales = [&](int slot) {
    const unsigned to = ring0 + SCALES + slot * 512;
    lds_dma4s(c_as, (unsigned)min(lane * 4, c_rows & ~3), to);
    lds_dma4s(c_ws, 0, to + 256);
  };
  auto copy = [&](int slot, int c) {  // the rows' copies, then W's
    switch (c) {
#define RC_CASE(Q) \
  case Q: return lds_copy16<Q * 4096>(Q < NA ? c_a : c_w, Q < NA ? off_a[Q < NA ? Q : 0] : off_w[Q < NA ? 0 : Q - NA], mine + slot * STAGE);
      RC_CASE(0) RC_CASE(1) RC_CASE(2) RC_CASE(3) RC_CASE(4) RC_CASE(5) RC_CASE(6) RC_CASE(7)
      RC_CASE(8) RC_CASE(9) RC_CASE(10) RC_CASE(11) RC_CASE(12) RC_CASE(13)
#undef RC_CASE
    }
    if constexpr (NA + NW == 16) {
      if (c == 14) lds_copy16<14 * 4096>(c_w, off_w[NW - 2], mine + slot * STAGE);
      if (c == 15) lds_copy16<15 * 4096>(c_w, off_w[NW - 1], mine + slot * STAGE);
    }
  };

  f32x4 acc[FM][FN];
  const int sz = (l16 >> 1) & 7, c_lo = l16 * kQBlock + ((lq ^ sz) << 4), c_hi = l16 * kQBlock + (((lq + 4) ^ sz) << 4);
  i32x8 a[FM], w[FN];
  int ea[FM], ew, ew_next;
  auto frag = [&](const char *rows) {
    return __builtin_shufflevector(*(const i32x4 *)(rows + c_lo), *(const i32x4 *)(rows + c_hi), 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto read_a = [&](int slot, int i) {
    a[i] = frag(lds + slot * STAGE + (wm * FM + i) * 16 * kQBlock);
    ea[i] = *(const uint8_t *)(lds + SCALES + slot * 512 + (wm * FM + i) * 16 + l16);
  };
  auto read_w = [&](int slot, int j) { w[j] = frag(lds + slot * STAGE + W0 + (wn * FN + j) * 16 * kQBlock); };
  auto read_ew = [&](int slot, int byte) { return (int)*(const uint8_t *)(lds + SCALES + slot * 512 + 256 + byte); };

  int m0, n0;
  place(blockIdx.x, m0, n0);
  enter(m0, n0);
  if (g.bias) copy_bias(n0, 0);
  else if (tid < 3 * BN / 4) *(f32x4 *)(lds + BIAS + tid * 16) = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    copy_scales(s);
#pragma unroll
    for (int c = 0; c < NA + NW; ++c) copy(s, c);
    advance();
  }
  wait_vm_q<2 + NA + NW>();
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  ew = read_ew(0, (n0 / kQBlock & 3) + wn);
#pragma unroll
  for (int j = 0; j < FN / 2; ++j) read_w(0, j);
#pragma unroll
  for (int i = 0; i < FM; ++i) read_a(0, i);

  int slot = 0, which = 0;
  auto multiply = [&](int q, int j) {
    acc[q][j] = q_mma<false>(w[j], a[q], acc[q][j], ew, ea[q]);
    asm volatile("" : "+a"(acc[q][j]));  // (in its place)
  };
  constexpr int HALF = FM * FN / 2, FROM = 13, EVERY = FM == 8 ? 3 : 2;  // products before the first copy, and between two
  static_assert(FROM + EVERY * (NA + NW - 1) < 2 * HALF, "a step issues all copies of a stage");
  auto step = [&](int byte) {  // byte: W's scale of the next stage
#pragma unroll
    for (int t8 = 0; t8 < FM; ++t8)
#pragma unroll
      for (int t1 = 0; t1 < FN; ++t1) {
        const int t = t8 * FN + t1;
        // the first half column by column, the second row by row
        const int q = t < HALF ? t % FM : (t - HALF) / 4, j = t < HALF ? t / FM : 4 + t % 4;
        multiply(q, j);
        if (t < 4) read_w(slot, 4 + t);
        if (t == 11) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // every wave has all of this stage
        if (t == 12) copy_scales(slot);
        if (t >= FROM && (t - FROM) % EVERY == 0 && (t - FROM) / EVERY < NA + NW) copy(slot, (t - FROM) / EVERY);
        if (t == HALF - 1) {  // the next stage is there
          wait_vm_q<2 + (HALF - FROM + EVERY - 1) / EVERY>();
          asm volatile("s_barrier" ::: "memory");
        }
        if (t >= HALF && (t - HALF) % FM == 1) read_w(slot ^ 1, (t - HALF) / FM);
        if (t == 2 * HALF - 11) ew_next = read_ew(slot ^ 1, byte);
        if (t >= HALF && j == 7) read_a(slot ^ 1, q);  // (behind the last stage: stale, never used)
        __builtin_amdgcn_sched_barrier(0);
      }
    ew = ew_next;
    advance();
    slot ^= 1;
  };

#pragma nounroll
  for (int t = blockIdx.x; t < tiles; t += gridDim.x) {
    int next_m0 = m0, next_n0 = n0;
    if (t + (int)gridDim.x < tiles) place(t + gridDim.x, next_m0, next_n0);
    const int byte = (n0 / kQBlock & 3) + wn, next_byte = (next_n0 / kQBlock & 3) + wn;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        asm volatile("" : "+a"(acc[i][j]));
      }
    // (all but the last two steps copy from this tile, those from the next)
    int i = 0;
#pragma nounroll
    for (int last = n - 2; i < n; last = n) {
#pragma nounroll
      for (; i < last; ++i) step(i + 1 < n ? byte : next_byte);
      if (i < n) {
        if (t + (int)gridDim.x < tiles) {
          enter(next_m0, next_n0);
          if (g.bias) copy_bias(next_n0, which == 2 ? 0 : which + 1);
        } else {  // no next one: the last stage again
          c_a -= by;
          c_w -= by;
          c_as -= as_by;
          c_ws -= ws_by;
          by = as_by = ws_by = 0;
        }
      }
    }

    // lane (l16, lq) holds, of row i * 16 + l16, columns j * 16 + lq * 4 .. + 3
    int my = lane;
    asm volatile("" : "+v"(my));  // (nothing that follows is made ahead and kept)
    const int lq = my >> 4, col0 = n0 + wn * 128, row0 = m0 + wm * (16 * FM) + (my & 15);
    const char *bias_at = lds + BIAS + which * 4 * BN + (wn * 128 + lq * 4) * 4;
    m0 = next_m0;
    n0 = next_n0;
    which = which == 2 ? 0 : which + 1;
    if constexpr (EPI == QG_RESID) {
      // half a row block of 16 at a time, its X and place loaded one half ahead
      // (rows and columns behind the last: any valid ones)
      constexpr int H = FN / 2;
      f32x4 gate[FN], x[2][H];
      int packed[2];
      auto load = [&](int u) {
        const int row = min(row0 + u / 2 * 16, g.M - 1);
        packed[u & 1] = g.packed[row];
#pragma unroll
        for (int j = 0; j < H; ++j)
          x[u & 1][j] = *(const f32x4 *)(g.X + (size_t)row * g.N + min(col0 + (u % 2 * H + j) * 16 + lq * 4, g.N - 4));
      };
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int col = min(col0 + j * 16 + lq * 4, g.N - 4);
        gate[j] = *(const f32x4 *)(g.gate + col) + *(const f32x4 *)(g.gate2 + col);
      }
      load(0);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int u = i * 2 + half, row = row0 + i * 16;
          __builtin_amdgcn_sched_barrier(0);
          if (u + 1 < 2 * FM) load(u + 1);
          bf16 *h = g.hslot + row_chain(packed[u & 1]) * g.chain_stride + (size_t)row_token(packed[u & 1]) * g.N;
#pragma unroll
          for (int j = half * H; j < half * H + H; j += 2) {
            uint32_t y[2][2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int col = col0 + (j + k) * 16 + lq * 4;
              const f32x4 bias = *(const f32x4 *)(bias_at + (j + k) * 64);
              f32x4 v;
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = x[u & 1][j + k - half * H][e] + gate[j + k][e] * (acc[i][j + k][e] + bias[e]);
              if (row < g.M && col < g.N) *(f32x4 *)(g.X + (size_t)row * g.N + col) = v;
              y[k][0] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)v[0], (bf16)v[1]});
              y[k][1] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)v[2], (bf16)v[3]});
            }
            q_swap16(y[0][0], y[1][0]);
            q_swap16(y[0][1], y[1][1]);
            const int col = col0 + (j + (lq & 1)) * 16 + (lq >> 1) * 8;
            if (row < g.M && col < g.N) __builtin_nontemporal_store(u32x4{y[0][0], y[0][1], y[1][0], y[1][1]}, (u32x4 *)(h + col));
          }
        }
    } else {
      f32x4 bias[FN];
#pragma unroll
      for (int j = 0; j < FN; ++j) bias[j] = *(const f32x4 *)(bias_at + j * 64);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int row = row0 + i * 16;
        float v[FN][4];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[j][e] = acc[i][j][e] + bias[j][e];
            if (GELU) v[j][e] = q_gelu(v[j][e]);
          }
        }
        if constexpr (EPI == QG_GELU8) {
          float m = 0.0f;
#pragma unroll
          for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) m = fmaxf(m, q_magnitude(v[j][e]));
          uint32_t m0_ = __float_as_uint(m), m1_ = m0_;
          q_swap16(m0_, m1_);
          m = half_swap_max(fmaxf(__uint_as_float(m0_), __uint_as_float(m1_)));
          const int ex = q_exponent(m);
          const float inv = q_inverse(ex);
#pragma unroll
          for (int h = 0; h < FN; h += 4) {  // four blocks of 16 columns: lane group lq gets block h + lq
            uint32_t d[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) d[k] = q_pack4(v[h + k], inv);
            q_swap16(d[0], d[1]);
            q_swap16(d[2], d[3]);
            q_swap32(d[0], d[2]);
            q_swap32(d[1], d[3]);
            if (row < g.M && col0 < g.N)
              *(u32x4 *)((uint8_t *)g.out + row * g.ldo + col0 + (h + lq) * 16) = u32x4{d[0], d[1], d[2], d[3]};
          }
          if (lq == 0 && row < g.M && col0 < g.N) g.out_scales[(size_t)(col0 / kQBlock) * g.out_scale_ld + row] = (uint8_t)ex;
        } else {
#pragma unroll
          for (int j = 0; j < FN; j += 2) {  // two blocks of 16 columns: eight in a row for each lane
            uint32_t u[2][2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              u[k][0] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)v[j + k][0], (bf16)v[j + k][1]});
              u[k][1] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)v[j + k][2], (bf16)v[j + k][3]});
            }
            q_swap16(u[0][0], u[1][0]);
            q_swap16(u[0][1], u[1][1]);
            const int col = col0 + (j + (lq & 1)) * 16 + (lq >> 1) * 8;
            if (row < g.M && col < g.N)
              __builtin_nontemporal_store(u32x4{u[0][0], u[0][1], u[1][0], u[1][1]}, (u32x4 *)((bf16 *)g.out + row * g.ldo + col));
          }
        }
      }
    }
  }
  wait_vm_q<0>();  // (the copies behind the last stage)
}

template <int EPI, typename OUT> static hipError_t launch_qg(const QGemmArgs &a, const QGemmPlan &p, hipStream_t s) {
  const long long n = ((long long)a.M + p.bm - 1) / p.bm * (((long long)a.N + p.bn - 1) / p.bn);
  if (n > 1 << 22) return hipErrorInvalidValue;  // (a grid holds fewer than 2^32 threads)
  const unsigned tiles = (unsigned)n;
#define RC_QG_SPLIT(FM, FN, KG) \
  return rc_launch(qgemm_split_kernel<FM, FN, KG, EPI == QG_GELU, OUT>, dim3(tiles), dim3(64 * KG), 0, s, a)
#define RC_QG(FM, FN, WGM, WGN, KG, S) \
  return rc_launch(qgemm_kernel<FM, FN, WGM, WGN, KG, S, EPI, OUT>, dim3(tiles), dim3(64 * WGM * WGN * KG), 0, s, a)
  const int tile = p.bm * 1000 + p.bn;
  if constexpr (EPI <= QG_GELU) {
    if (tile == 16016) RC_QG_SPLIT(1, 1, 8);
    if (tile == 32032) RC_QG_SPLIT(2, 2, 8);
  }
  if constexpr (EPI != QG_GELU8) {
    if (tile == 64032) RC_QG(4, 2, 1, 1, 4, 3);
    if (tile == 64064) RC_QG(4, 4, 1, 1, 4, 2);
  }
  if (tile == 64128) RC_QG(4, 2, 1, 4, 1, 3);
  if (tile == 128128) RC_QG(4, 4, 2, 2, 1, 2);
  if constexpr (sizeof(OUT) == 2)
    if (p.bn == 256) {
      if (a.K % kQBlock || a.K < 2 * kQBlock || a.N % 8 || a.ldo % 8) return hipErrorInvalidValue;
      const dim3 grid(std::min(tiles, 256u));
      if (p.bm == 192) return rc_launch(qgemm_large_kernel<6, EPI>, grid, dim3(256), 0, s, a, (int)tiles);
      if (p.bm == 256) return rc_launch(qgemm_large_kernel<8, EPI>, grid, dim3(256), 0, s, a, (int)tiles);
    }
#undef RC_QG
#undef RC_QG_SPLIT
  return hipErrorInvalidValue;
}

// The tile with the least estimated time: 5 us of ends, and for every tile that
// a CU has to do a time for each step of K and an end.  Workgroups of small
// tiles (kg 8) share a CU; those of kg 1 count as pairs where there are few.
// Measured, us (kernels alone): 16 x 16, 32 x 32, 64 x 32 and 64 x 64 tiles 1 x
// 4608 x 1152 4.6, 4.6, 6.0, 7.2; 16 x 1152 x 4608 7.4, 9.6, 10.4, 13.0; 64 x 4608
// x 1152 8.7, 7.3, 6.0, 7.4; 200 x 1152 x 640 5.9, 4.4, 5.4, 6.5; 200 x 1152 x
// 4608 19.7, 12.0, 11.4, 13.6; 723 x 1152 x 4608 -, -, 21, 15 (64 x 128 24), 1517
// x 1152 x 4608 -, -, 44, 31 (28).  With launches, 64 x 128, 128 x 128, 192 x 256
// and 256 x 256: 723 x 4608 x 1152 13.3, 14.9, -, -; 1639 x 4608 x 1152 22.5,
// 16.4, 18.6, 21.0; 2401 x 4608 x 1152 31.5, 26.2, 19.7, 22.1; 3500 x 4608 x 1152
// 42, 31, 34, 24.8 (342 and 252 of the large tiles for 256 CUs); 3500 x 1152 x
// 4608 30.9, 31.5, 38.8, 43.7; 4096 x 4608 x 1152 48, 39, 35, 41; 8192 x 1152 x
// 4608 76, 66, 46.7, 48.9; 16384 x 4608 x 1152 171, 132, 119, 107; 16384 x 1152 x
// 4608 146, 121, 90, 100.
QGemmPlan plan_qgemm(int M, int N, int K, QGemmEpi epi, bool large) {
  struct Tile { int bm, bn, kg; double per, end; };  // us a step, a tile
  static constexpr Tile tiles[] = {{16, 16, 8, 1.0, 0.0}, {32, 32, 8, 1.7, 0.0}, {64, 32, 4, 0.65, 1.2}, {64, 64, 4, 1.0, 2.5},
                                   {64, 128, 1, 0.33, 0.6}, {128, 128, 1, 0.44, 1.0}, {192, 256, 0, 1.0, 5.9}, {256, 256, 0, 1.1, 7.5}};
  const int blocks = (K + kQBlock - 1) / kQBlock;
  QGemmPlan best{128, 128};
  double best_us = 1e30;
  for (const Tile &t : tiles) {
    if ((epi == QG_GELU8 && t.bn % kQBlock) || (epi == QG_RESID && t.bm < 64)) continue;  // (tiles that have the epilogue)
    if (t.kg == 0 && (!large || K % kQBlock || K < 2 * kQBlock)) continue;
    const double wgs = std::ceil((double)M / t.bm) * std::ceil((double)N / t.bn) / 256;
    const double load = t.kg == 8   ? std::max(1.3 * wgs, 1.0)
                        : t.kg != 1 ? std::ceil(wgs)
                        : wgs <= 1.0 ? 1.7 : wgs <= 2.0 ? 2.0 : std::max(1.35 * wgs, 3.2);
    const double steps = t.kg > 1 ? (blocks + t.kg - 1) / t.kg : blocks;
    const double us = 5.0 + load * (steps * t.per + t.end);
    if (us < best_us) {
      best_us = us;
      best = QGemmPlan{t.bm, t.bn};
    }
  }
  return best;
}

hipError_t launch_qgemm(const QGemmArgs &a, const QGemmPlan &p, QGemmEpi epi, bool f32_out, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  if (a.K > kQMaxCols || a.K % 16) return hipErrorInvalidValue;
  hipError_t e = hipErrorInvalidValue;
  if (epi == QG_GELU8) {
    if (a.N % kQBlock == 0 && a.bias) e = launch_qg<QG_GELU8, bf16>(a, p, s);
  } else if (epi == QG_RESID) {
    if (a.N % 8 == 0) e = launch_qg<QG_RESID, bf16>(a, p, s);
  } else if (epi == QG_GELU) {
    e = f32_out ? launch_qg<QG_GELU, float>(a, p, s) : launch_qg<QG_GELU, bf16>(a, p, s);
  } else {
    e = f32_out ? launch_qg<QG_STORE, float>(a, p, s) : launch_qg<QG_STORE, bf16>(a, p, s);
  }
  return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace rc
