// Product of int8 matrices: Y[M][N] = act((A[M][K] . W[N][K]^T) sa[m] sw[n] + bias[n]),
// 16x16x64 matrix instructions in the tiles of rc_qgemm_tiles.h.  Sums are 32-bit
// integers, exact for any order (at most 2^14 K < 2^31), so that K may be split
// as it suits; they are rounded once, to float32, before the two scales.
//
// Two kinds of tiles: those of rc_qgemm_tiles.h for any shape and type, and those of
// igemm_step_kernel below.  In a captured graph, one call behind the other, us: 1 x 4608 x
// 1152 3.5; 400 x 4608 x 1152 5.7; 723 x 1152 x 4608 9.5; 723 x 4608 x 1152 with GELU 8.2; 4096 x
// 1152 x 4608 24; 4096 x 4608 x 1152 with GELU 30; 16384 x 4608 x 1152 87, 100 with GELU; 16384 x
// 1152 x 4608 80; 8192 x 8192 x 8192 365, 3.0 POP/s (PyTorch's int8 product 520).
//
// float32 results take the tiles of rc_qgemm_tiles.h up to 128 x 128 only: the others' epilogues
// pack bfloat16, which the steps and a next quantisation take.  The same calls: 400 x 4608 x 1152
// 8.1; 723 x 1152 x 4608 11.2; 723 x 4608 x 1152 10.8 (bfloat16 7.4); 4096 x 1152 x 4608 34; 16384 x
// 4608 x 1152 131, whose 302 MB of results alone are 59 at a copy's rate; 8192 x 8192 x 8192 546.
#include "rc_common.h"
#include "rc_int8.h"
#include "rc_launch.h"
#include "rc_qgemm_tiles.h"
#include "rc_quant.h"

#include <algorithm>

namespace rc {

// Tiles of 32 FM x 32 FN results, four waves of 16 FM x 16 FN each, whole blocks of
// 128 of K, bfloat16 results whose rows begin at 16 bytes.  One wave per SIMD (two
// where two workgroups' rings fit a CU), so the order of instructions covers latency:
// * A ring of S stages.  A step's first half multiplies column by column and reads
//   the rest of its W fragments at once; then the stage is in registers, every
//   wave says so at the step's only barrier, and its place takes the stage S steps
//   on.  The second half multiplies row by row and reads the next stage's fragments
//   into the registers of the rows that are done with.
// * The copies of a stage go out one after another between products; with S = 3
//   those that the barrier waits for are a whole step old.
// * The epilogue needs no LDS: lanes exchange registers until they hold whole stores.
// A step of 128 x 192 takes LDS 960 clocks (fragments 640, copies 320), its products
// 770, a CU's share of the L2 640.  Tiles of 128 x 128 in the rings above wait for LDS
// reads and copies within each step, and two workgroups of them are needed to cover
// that: 4096 x 1152 x 4608 34.5 us, 23.5 here; 2401 x 1152 x 4608 24.2 -> 16.4 (96 x 128);
// 723 x 4608 x 1152 with GELU 10.4 -> 8.7 (128 x 128); 400 x 4608 x 1152 8.7 -> 6.9 (64 x 128).
// With two stages two workgroups of 128 x 128 or 96 x 192 fit a CU and cover each
// other's waits and epilogues, which pays for several rounds and short K: 8192 x 4608 x
// 1152 with GELU 65 (128 x 192, S = 3) -> 57, 1639 x 4608 x 1152 16.5 -> 13.8; but 4096 x 1152
// x 4608 25 -> 29.  A ring of four or six took longer where it keeps a second workgroup off
// the CU (4096 x 4608 x 1152, 64 x 128: 33.5 -> 47), else the same within 3 %.
template <int FM, int FN, int S, int EPI> __global__ __launch_bounds__(256, 1) void igemm_step_kernel(IGemmArgs g) {
  constexpr int BM = 32 * FM, BN = 32 * FN, W0 = BM * kQBlock, STAGE = W0 + BN * kQBlock, NA = FM, NW = FN, NL = NA + NW;
  constexpr int ENDS = S * STAGE;  // the columns' bias and scales, the rows' scales
  static_assert(FN % 2 == 0 && S >= 2 && BN <= 256 && BM <= 256, "tile");
  __shared__ __attribute__((aligned(1024))) char lds[ENDS + 8 * BN + 4 * ((BM + 63) / 64 * 64)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  __builtin_assume(wave >= 0 && wave < 4);
  const int wm = wave >> 1, wn = wave & 1, l16 = lane & 15, lq = lane >> 4;
  const int tiles_m = (g.M + BM - 1) / BM, tiles_n = (g.N + BN - 1) / BN, n = g.K / kQBlock;
  constexpr int GM = 2048 / BM;  // bands of row tiles, as in the other kernels
  const int L = xcd_logical_id(blockIdx.x, gridDim.x);
  const int band0 = L / (GM * tiles_n), gm = min(GM, tiles_m - band0 * GM), idx = L - band0 * GM * tiles_n;
  const int m0 = __builtin_amdgcn_readfirstlane((band0 * GM + idx % gm) * BM), n0 = __builtin_amdgcn_readfirstlane(idx / gm * BN);

  // copies of 1 KB per wave, eight rows of 128 bytes (those behind the last are copies of it)
  const unsigned ring0 = __builtin_amdgcn_readfirstlane(lds_address(lds)), mine = ring0 + wave * 1024;
  const int row8 = wave * 8 + (lane >> 3), chunk = ((lane & 7) ^ ((row8 >> 1) & 7)) * 16;
  const uint8_t *c_a = g.a + m0 * g.lda, *c_w = g.w + n0 * g.ldw;  // the next stage to be copied
  unsigned off_a[NA], off_w[NW];
#pragma unroll
  for (int q = 0; q < NA; ++q) off_a[q] = __umul24((unsigned)min(row8 + q * 32, g.M - 1 - m0), (unsigned)g.lda) + chunk;
#pragma unroll
  for (int q = 0; q < NW; ++q) off_w[q] = __umul24((unsigned)min(row8 + q * 32, g.N - 1 - n0), (unsigned)g.ldw) + chunk;
  auto copy = [&](unsigned to, int c) {  // the rows' copies, then W's
    switch (c) {
#define RC_CASE(Q)                                                                                                     \
  case Q:                                                                                                              \
    if constexpr (Q < NL)                                                                                              \
      lds_copy16<Q * 4096>(Q < NA ? c_a : c_w, Q < NA ? off_a[Q < NA ? Q : 0] : off_w[Q < NA || Q >= NL ? 0 : Q - NA], to); \
    return;
      RC_CASE(0) RC_CASE(1) RC_CASE(2) RC_CASE(3) RC_CASE(4) RC_CASE(5) RC_CASE(6) RC_CASE(7) RC_CASE(8) RC_CASE(9)
#undef RC_CASE
    }
  };
  static_assert(NL <= 10, "copies of a stage");
  auto advance = [&](int stage) {  // (behind the last one: the last again, never used)
    if (stage < n - 1) {
      c_a += kQBlock;
      c_w += kQBlock;
    }
  };
  // a wave has 64 columns and 64 rows of what the epilogue takes
  const unsigned ends = __builtin_amdgcn_readfirstlane(ring0 + ENDS + wave * 256);
  if (wave * 64 < BN) {
    if (g.bias) lds_dma4s(g.bias, (unsigned)min(n0 + wave * 64 + lane, g.N - 1) * 4u, ends);
    else *(float *)(lds + ENDS + threadIdx.x * 4) = 0.0f;
    lds_dma4s(g.ws, (unsigned)min(n0 + wave * 64 + lane, g.N - 1) * 4u, ends + 4 * BN);
  }
  if (wave * 64 < BM) lds_dma4s(g.as + m0, (unsigned)min(wave * 64 + lane, g.M - 1 - m0) * 4u, ends + 8 * BN);
#pragma unroll
  for (int s = 0; s < S; ++s) {
#pragma unroll
    for (int c = 0; c < NL; ++c) copy(mine + s * STAGE, c);
    advance(s);
  }

  i32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      acc[i][j] = i32x4{0, 0, 0, 0};
      asm volatile("" : "+a"(acc[i][j]));
    }
  const int sz = (l16 >> 1) & 7, c_lo = l16 * kQBlock + ((lq ^ sz) << 4), c_hi = l16 * kQBlock + (((lq + 4) ^ sz) << 4);
  i32x8 a[FM], w[FN];
  auto frag = [&](const char *rows) {
    return __builtin_shufflevector(*(const i32x4 *)(rows + c_lo), *(const i32x4 *)(rows + c_hi), 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto read_a = [&](int at, int i) { a[i] = frag(lds + at + (wm * FM + i) * 16 * kQBlock); };
  auto read_w = [&](int at, int j) { w[j] = frag(lds + at + W0 + (wn * FN + j) * 16 * kQBlock); };
  constexpr int H = FN / 2, HALF = FM * H, PER = (NL + HALF - 1) / HALF;  // copies between two products
  wait_vm_q<(S - 1) * NL>();
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
  for (int j = 0; j < H; ++j) read_w(0, j);
#pragma unroll
  for (int i = 0; i < FM; ++i) read_a(0, i);
  int at = 0;  // the stage's place
#pragma nounroll
  for (int k = 0; k < n; ++k) {
    const int next = at == (S - 1) * STAGE ? 0 : at + STAGE;
#pragma unroll
    for (int t = 0; t < 2 * HALF; ++t) {
      const int q = t < HALF ? t % FM : (t - HALF) / H, j = t < HALF ? t / FM : H + (t - HALF) % H;
      acc[q][j] = q_mma<false>(w[j], a[q], acc[q][j], 0, 0);
      asm volatile("" : "+a"(acc[q][j]));  // (in its place)
      if (t < H) read_w(at, H + t);
      if (t == HALF - 1) {  // every wave has all of this stage, and the next one is there
        wait_vm_q<(S - 2) * NL>();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      }
      if (t >= HALF) {
        const int u = t - HALF;
#pragma unroll
        for (int c = u * PER; c < u * PER + PER; ++c)
          if (c < NL) copy(mine + at, c);
        if (u % FM == 1 && u / FM < H) read_w(next, u / FM);
        if (j == FN - 1) read_a(next, q);  // (behind the last stage: never used)
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    advance(k + S);
    at = next;
  }

  // lane (l16, lq) holds, of row i * 16 + l16, columns j * 16 + lq * 4 .. + 3
  const int col0 = n0 + wn * 16 * FN, row0 = m0 + wm * 16 * FM + l16;
  const char *bias_at = lds + ENDS + (wn * 16 * FN + lq * 4) * 4, *rows_at = lds + ENDS + 8 * BN + (wm * 16 * FM + l16) * 4;
  f32x4 gate[EPI == QG_RESID ? FN : 1];
  if constexpr (EPI == QG_RESID)
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int col = min(col0 + j * 16 + lq * 4, g.N - 4);
      gate[j] = *(const f32x4 *)(g.gate + col) + *(const f32x4 *)(g.gate2 + col);
    }
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int row = row0 + i * 16;
    const float row_scale = *(const float *)(rows_at + i * 64);
    bf16 *out = (bf16 *)g.out + row * g.ldo;
    f32x4 x[EPI == QG_RESID ? FN : 1];
    if constexpr (EPI == QG_RESID) {  // (rows and columns behind the last: any valid ones)
      const int r = min(row, g.M - 1), packed = g.packed[r];
      out = g.hslot + row_chain(packed) * g.chain_stride + (size_t)row_token(packed) * g.N;
#pragma unroll
      for (int j = 0; j < FN; ++j) x[j] = *(const f32x4 *)(g.X + (size_t)r * g.N + min(col0 + j * 16 + lq * 4, g.N - 4));
    }
#pragma unroll
    for (int j = 0; j < FN; j += 2) {  // two blocks of 16 columns: eight in a row for each lane
      uint32_t y[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 bias = *(const f32x4 *)(bias_at + (j + h) * 64), cs = *(const f32x4 *)(bias_at + 4 * BN + (j + h) * 64);
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = q_biased(acc[i][j + h][e], row_scale, cs[e], bias[e]);
          if (EPI == QG_GELU) v[e] = q_gelu(v[e]);
          if constexpr (EPI == QG_RESID) v[e] = x[j + h][e] + gate[j + h][e] * v[e];
        }
        if constexpr (EPI == QG_RESID) {
          const int col = col0 + (j + h) * 16 + lq * 4;
          if (row < g.M && col < g.N) *(f32x4 *)(g.X + (size_t)row * g.N + col) = v;
        }
        y[h][0] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)v[0], (bf16)v[1]});
        y[h][1] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)v[2], (bf16)v[3]});
      }
      q_swap16(y[0][0], y[1][0]);
      q_swap16(y[0][1], y[1][1]);
      const int col = col0 + (j + (lq & 1)) * 16 + (lq >> 1) * 8;
      if (row < g.M && col < g.N) __builtin_nontemporal_store(u32x4{y[0][0], y[0][1], y[1][0], y[1][1]}, (u32x4 *)(out + col));
    }
  }
  wait_vm_q<0>();  // (the copies behind the last stage)
}

template <int EPI, typename OUT> static hipError_t launch_ig(const IGemmArgs &a, const IGemmPlan &p, hipStream_t s) {
  const long long n = ((long long)a.M + p.bm - 1) / p.bm * (((long long)a.N + p.bn - 1) / p.bn);
  if (n > 1 << 22) return hipErrorInvalidValue;  // (a grid holds fewer than 2^32 threads)
  const unsigned tiles = (unsigned)n;
#define RC_IG_SPLIT(FM, FN, KG) \
  return rc_launch(qgemm_split_kernel<FM, FN, KG, EPI == QG_GELU, OUT, IGemmArgs>, dim3(tiles), dim3(64 * KG), 0, s, a)
#define RC_IG(FM, FN, WGM, WGN, KG, S) \
  return rc_launch(qgemm_kernel<FM, FN, WGM, WGN, KG, S, EPI, OUT, IGemmArgs>, dim3(tiles), dim3(64 * WGM * WGN * KG), 0, s, a)
  const int tile = p.bm * 1000 + p.bn;
  if constexpr (sizeof(OUT) == 2)
    if (p.ring) {
      if (a.K % kQBlock || a.N % 8 || a.ldo % 8) return hipErrorInvalidValue;
#define RC_IG_STEP(FM, FN, S) \
  if (tile == 32 * FM * 1000 + 32 * FN && p.ring == S) return rc_launch(igemm_step_kernel<FM, FN, S, EPI>, dim3(tiles), dim3(256), 0, s, a)
      RC_IG_STEP(2, 2, 4);
      RC_IG_STEP(2, 4, 3);
      RC_IG_STEP(3, 4, 3);
      RC_IG_STEP(4, 4, 3);
      RC_IG_STEP(4, 6, 3);
      RC_IG_STEP(3, 6, 2);
      RC_IG_STEP(4, 4, 2);
#undef RC_IG_STEP
      return hipErrorInvalidValue;
    }
  if (p.ring) return hipErrorInvalidValue;
  if constexpr (EPI <= QG_GELU) {
    if (tile == 16016) RC_IG_SPLIT(1, 1, 8);
    if (tile == 32032) RC_IG_SPLIT(2, 2, 8);
  }
  if (tile == 64032) RC_IG(4, 2, 1, 1, 4, 3);
  if constexpr (EPI <= QG_GELU) {  // (a residual's K, the model's inner width, is a multiple of 128)
    if (tile == 64064) RC_IG(4, 4, 1, 1, 4, 2);
    if (tile == 64128) RC_IG(4, 2, 1, 4, 1, 3);
    if (tile == 128128) RC_IG(4, 4, 2, 2, 1, 2);
  }
  if constexpr (sizeof(OUT) == 2) {
    if (p.bn == 256) {
      if (a.K % kQBlock || a.K < 2 * kQBlock || a.N % 8 || a.ldo % 8) return hipErrorInvalidValue;
      const dim3 grid(std::min(tiles, 256u));
      if (p.bm == 192) return rc_launch(qgemm_large_kernel<6, EPI, IGemmArgs>, grid, dim3(256), 0, s, a, (int)tiles);
      if (p.bm == 256) return rc_launch(qgemm_large_kernel<8, EPI, IGemmArgs>, grid, dim3(256), 0, s, a, (int)tiles);
    }
  }
#undef RC_IG
#undef RC_IG_SPLIT
  return hipErrorInvalidValue;
}

// The tile with the least estimate, a launch and rounds of workgroups of so many
// steps and an end each (fitted to what 281 sizes of 1 to 16384 rows took in every
// tile; the choice takes 1.03 times the best tile's time in the mean, 1.3 at most:
// 108 x 1152 x 4096, 32 x 32 tiles 10.1 us, 64 x 32 ones 7.7).  Without the tiles of
// igemm_step_kernel the best of the others takes 1.10 times as long in the mean, 1.5 at most.
IGemmPlan plan_igemm(int M, int N, int K, QGemmEpi epi, bool large) {
  struct Tile {
    int bm, bn, kg;       // groups of waves that share K (0: whole chip)
    int ring;
    double per, end;      // us a step, a tile
    double least, whole;  // more than one round: at least so many, and how much of the last one counts as whole
  };
  static constexpr Tile tiles[] = {
      {16, 16, 8, 0, 0.38, 0.0, 0, 1.38},     {32, 32, 8, 0, 0.8, 0.0, 0, 1.94},      {64, 32, 4, 0, 0.55, 0.4, 1.2, 1},
      {64, 64, 4, 0, 0.79, 1.0, 1.2, 1},      {64, 128, 1, 0, 0.37, 1.1, 1.2, 0.31},  {128, 128, 1, 0, 0.54, 2.1, 1.1, 0.36},
      {192, 256, 0, 0, 0.95, 6.6, 1, 0.83},   {256, 256, 0, 0, 1.44, 6.3, 1, 0.33},   {64, 64, 1, 4, 0.173, 0.4, 2, 1},
      {64, 128, 1, 3, 0.276, 0.8, 1.7, 1},    {96, 128, 1, 3, 0.35, 1.3, 1.6, 1},     {128, 128, 1, 3, 0.42, 1.8, 1.3, 1},
      {128, 192, 1, 3, 0.61, 2.6, 1.6, 1},    {96, 192, 1, 2, 0.48, 1.7, 1.6, 0.61},  {128, 128, 1, 2, 0.47, 1.6, 1, 0.47}};
  const int blocks = (K + kQBlock - 1) / kQBlock;
  const bool rows16 = large && K % kQBlock == 0;  // what the step's and the largest tiles need
  IGemmPlan best{64, 32, 0};
  double best_us = 1e30;
  for (const Tile &t : tiles) {
    if (epi == QG_RESID && !t.ring && t.kg != 0 && !(t.bm == 64 && t.bn == 32)) continue;  // (tiles that have the epilogue)
    if ((t.ring || t.kg == 0) && !rows16) continue;
    if (t.kg == 0 && K < 2 * kQBlock) continue;
    const double wgs = std::ceil((double)M / t.bm) * std::ceil((double)N / t.bn) / 256, rounds = std::ceil(wgs);
    const double load = t.kg == 8     ? std::max(t.whole * wgs, 1.0)  // (many on a CU)
                        : wgs <= 1.0 ? 1.0
                                     : std::max(t.least, t.whole * rounds + (1 - t.whole) * wgs);
    const double us = 3.0 + load * ((t.kg > 1 ? (blocks + t.kg - 1) / t.kg : blocks) * t.per + t.end);
    if (us < best_us) {
      best_us = us;
      best = IGemmPlan{t.bm, t.bn, t.ring};
    }
  }
  return best;
}

hipError_t launch_igemm(const IGemmArgs &a, const IGemmPlan &p, QGemmEpi epi, bool f32_out, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  if (a.K > kI8MaxCols || a.K % 16) return hipErrorInvalidValue;
  hipError_t e = hipErrorInvalidValue;
  if (epi == QG_GELU) e = f32_out ? launch_ig<QG_GELU, float>(a, p, s) : launch_ig<QG_GELU, bf16>(a, p, s);
  else if (epi == QG_RESID) e = a.N % 8 == 0 ? launch_ig<QG_RESID, bf16>(a, p, s) : hipErrorInvalidValue;
  else if (epi == QG_STORE) e = f32_out ? launch_ig<QG_STORE, float>(a, p, s) : launch_ig<QG_STORE, bf16>(a, p, s);
  return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace rc
