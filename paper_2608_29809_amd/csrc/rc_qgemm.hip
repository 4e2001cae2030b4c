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
// (exactly), for 16x16x32 instructions whose sums keep float32's precision
// (8e-8 of the result's norm over 36 blocks, as a float32 library product).
#include "rc_common.h"
#include "rc_launch.h"
#include "rc_quant.h"

namespace rc {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kQMaxBlocks = kQMaxCols / kQBlock;

// Workgroup tile of 16 FM WGM rows and 16 FN WGN columns.  W is operand A of
// the matrix instruction, so a lane's accumulators are four consecutive
// columns of one row.
template <int FM, int FN, int WGM, int WGN, bool GELU, typename OUT>
__global__ __launch_bounds__(64 * WGM * WGN) void qgemm_kernel(QGemmArgs g) {
  constexpr int NW = WGM * WGN, BM = 16 * FM * WGM, BN = 16 * FN * WGN;
  constexpr bool F32 = sizeof(OUT) == 4;
  constexpr int STAGE = (BM + BN) * kQBlock, TC = STAGE / 1024;  // wave copies of 1 KB: eight rows
  static_assert(TC % NW == 0 && kQBlock % (16 * FN) == 0 && BM % 64 == 0, "tile");
  constexpr int NL = TC / NW;
  __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];
  __shared__ uint8_t sa[2][BM], sw[(BN + kQBlock - 1) / kQBlock][kQMaxBlocks];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WGN, wn = wave % WGN, l16 = lane & 15, lq = lane >> 4;
  const int tiles_n = (g.N + BN - 1) / BN, L = xcd_logical_id(blockIdx.x, gridDim.x);
  const int tm = L / tiles_n, tn = L - tm * tiles_n, m0 = tm * BM, n0 = tn * BN;
  const int nk = (g.K + kQBlock - 1) / kQBlock;

  // rows past the last are clamped to it and never stored; columns of K past
  // the last are copies of its last 16 and multiplied as zeros
  const uint8_t *src[NL];
  int col[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int row = (i * NW + wave) * 8 + (lane >> 3);
    col[i] = ((lane & 7) ^ ((row >> 1) & 7)) * 16;
    src[i] = row < BM ? g.a + min(m0 + row, g.M - 1) * g.lda : g.w + min(n0 + row - BM, g.N - 1) * g.ldw;
  }
  auto issue = [&](int slot, int kt) {
#pragma unroll
    for (int i = 0; i < NL; ++i)
      lds_dma16(src[i] + min(kt * kQBlock + col[i], g.K - 16), lds + slot * STAGE + (i * NW + wave) * 1024);
  };
  auto row_scales = [&](int slot, int kt) {
    for (int r = tid; r < BM; r += 64 * NW) sa[slot][r] = g.as[(size_t)kt * g.as_ld + min(m0 + r, g.M - 1)];
  };
  for (int i = tid; i < nk; i += 64 * NW)
#pragma unroll
    for (int j = 0; j < (BN + kQBlock - 1) / kQBlock; ++j)
      sw[j][i] = g.ws[(size_t)i * g.ws_ld + min(n0 / kQBlock + j, (g.N - 1) / kQBlock)];

  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int fr = l16 * kQBlock, sz = (l16 >> 1) & 7;
  auto frag = [&](const char *tile, int block, int kt) {
    const char *p = tile + block * 16 * kQBlock + fr;
    i32x4 lo = *(const i32x4 *)(p + ((lq ^ sz) << 4)), hi = *(const i32x4 *)(p + (((lq + 4) ^ sz) << 4));
    if (kt * kQBlock + kQBlock > g.K) {
      const int left = (g.K - kt * kQBlock) / 16;  // chunks of 16 that exist
      if (lq >= left) lo = i32x4{0, 0, 0, 0};
      if (lq + 4 >= left) hi = i32x4{0, 0, 0, 0};
    }
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };

  issue(0, 0);
  row_scales(0, 0);
  for (int kt = 0; kt < nk; ++kt) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (kt + 1 < nk) {
      issue((kt + 1) & 1, kt + 1);
      row_scales((kt + 1) & 1, kt + 1);
    }
    const char *st = lds + (kt & 1) * STAGE;
    const int ew = sw[wn * FN * 16 / kQBlock][kt];
    i32x8 w[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) w[j] = frag(st + BM * kQBlock, wn * FN + j, kt);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const i32x8 a = frag(st, wm * FM + i, kt);
      const int ea = sa[kt & 1][(wm * FM + i) * 16 + l16];
      if constexpr (!F32) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[j], a, acc[i][j], 0, 0, 0, ew, 0, ea);
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const bf16x8 av = q_bf16x8(u32x2{(uint32_t)a[2 * q], (uint32_t)a[2 * q + 1]}, q_factor(ea));
#pragma unroll
          for (int j = 0; j < FN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                q_bf16x8(u32x2{(uint32_t)w[j][2 * q], (uint32_t)w[j][2 * q + 1]}, q_factor(ew)), av, acc[i][j], 0, 0, 0);
        }
      }
    }
  }

  OUT *out = (OUT *)g.out;
  const bool vec = (g.ldo & 3) == 0;
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int m = m0 + (wm * FM + i) * 16 + l16;
    if (m >= g.M) continue;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int n = n0 + (wn * FN + j) * 16 + lq * 4;
      f32x4 v = acc[i][j];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (g.bias) v[e] += g.bias[min(n + e, g.N - 1)];
        if (GELU) v[e] = gelu_tanh(v[e]);
      }
      OUT *o = out + m * g.ldo + n;
      typedef OUT out4 __attribute__((ext_vector_type(4)));
      if (vec && n + 3 < g.N) {
        *(out4 *)o = out4{(OUT)v[0], (OUT)v[1], (OUT)v[2], (OUT)v[3]};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < g.N) o[e] = (OUT)v[e];
      }
    }
  }
}

template <bool GELU, typename OUT> static void launch_qg(const QGemmArgs &a, hipStream_t s) {
  constexpr int BM = 128, BN = 128;
  const long long tiles = (long long)((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN);
  rc_launch(qgemm_kernel<4, 4, 2, 2, GELU, OUT>, dim3((unsigned)tiles), dim3(256), 0, s, a);
}

size_t qgemm_scratch(int, int, int) { return 0; }

hipError_t launch_qgemm(const QGemmArgs &a, bool gelu, bool f32_out, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  if (a.K > kQMaxBlocks * kQBlock || a.K % 16) return hipErrorInvalidValue;
  if (f32_out) gelu ? launch_qg<true, float>(a, s) : launch_qg<false, float>(a, s);
  else gelu ? launch_qg<true, bf16>(a, s) : launch_qg<false, bf16>(a, s);
  return hipGetLastError();
}

}  // namespace rc
