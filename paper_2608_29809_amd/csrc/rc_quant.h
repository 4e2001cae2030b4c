// Launch interface of the 8-bit operators: block quantisation, the product of
// block-scaled matrices, the 8-bit cache of keys and values.
//
// Values are e4m3.  A block's scale is a power of two held as one byte e,
// 2^(e - 127): the least with which its largest finite magnitude is at most
// 448, and e >= 1.  A floating-point format loses no precision to a power of
// two (only range), dequantised values are exact in bfloat16 (but for e <= 2,
// where those below 2^-133 are beneath its range), a block's other values are
// exact under a change of its scale (unless they become subnormal), and the
// matrix instructions take the byte as it is.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_common.h"

namespace rc {

constexpr int kQBlock = 128;    // columns that share a scale (rows too, of a weight)
constexpr int kQMaxCols = 65536;
constexpr int kQTokens = 64;    // tokens of a cache block
constexpr int kQTileBytes = kQTokens * kHeadDim;  // a block's keys or values

struct QuantArgs {
  const void *x;
  long long ldx;  // elements
  int rows, cols;
  uint8_t *q;
  long long ldq;
  uint8_t *scales;  // [column blocks][scale_ld]
  int scale_ld;
};
template <typename T> hipError_t launch_quantize(const QuantArgs &a, int block_rows, hipStream_t s);

// LayerNorm + modulation of a step's rows, into 8 bits.
struct NormQuantArgs {
  const float *X;           // [rows][C]
  int rows, C;
  const float *sst, *t0;    // shift and scale: rows shift_row and shift_row + 1 of sst + t0
  int shift_row;
  float eps;
  uint8_t *q;               // [rows][C]
  uint8_t *scales;          // [C / 128][scale_ld]
  int scale_ld;
};
hipError_t launch_norm_quantize(const NormQuantArgs &a, hipStream_t s);

enum QGemmEpi {
  QG_STORE = 0,  // out = acc + bias, bfloat16 or float32
  QG_GELU = 1,   // out = gelu_tanh(acc + bias), bfloat16 or float32
  QG_GELU8 = 2,  // the same in 8 bits with a scale for each row and 128 columns (N a multiple of 128)
  QG_RESID = 3,  // X += (gate + gate2) (acc + bias), and the new X in bfloat16 into the rows' places in hslot (N a multiple of 8)
};
struct QGemmArgs {
  const uint8_t *a, *w;     // [M][K], [N][K]
  const uint8_t *as, *ws;   // scales: [K blocks][as_ld], [K blocks][ws_ld]
  long long lda, ldw;
  int as_ld, ws_ld;
  int M, N, K;
  const float *bias;        // [N] or null
  void *out;                // QG_GELU8: e4m3
  long long ldo;            // elements
  // QG_GELU8
  uint8_t *out_scales;      // [N / 128][out_scale_ld]
  int out_scale_ld;
  // QG_RESID
  float *X;                 // [M][N]
  const float *gate, *gate2;
  const int *packed;        // (chain << 16) | token per row
  bf16 *hslot;              // H of chain 0's slot
  long long chain_stride;   // elements
};
struct QGemmPlan { int bm, bn; };  // workgroup tile
// large: bfloat16 or 8-bit results, N and their row stride multiples of 8 (what 256 x 256 tiles need)
QGemmPlan plan_qgemm(int M, int N, int K, QGemmEpi epi, bool large);
hipError_t launch_qgemm(const QGemmArgs &a, const QGemmPlan &p, QGemmEpi epi, bool f32_out, hipStream_t s);

struct QCacheArgs {
  uint8_t *data;            // [heads][tokens / 64][2][64][72] per chain: keys, then values, of a block
  uint8_t *scales;          // [heads][tokens / 64][2] per chain
  long long chain_stride, scale_chain_stride;  // bytes
  int heads, tokens;
};
// Row ranges of the chains: the first ones by value, the others from device memory.
constexpr int kQArgChains = 16;
struct ChainRows {
  const int *offsets;
  int n_arg;
  int arg[kQArgChains + 1];
};
__device__ __forceinline__ int2 chain_rows(const ChainRows &a, int b) {
  if (b < a.n_arg) return make_int2(a.arg[b], a.arg[b + 1]);
  return make_int2(a.offsets[b], a.offsets[b + 1]);
}
struct QStoreArgs {
  QCacheArgs c;
  ChainRows rows;
  const int *idx;           // or null: every token of every chain
  const void *k, *v;        // [rows][heads * 72]
  long long ld;             // elements
};
template <typename T> hipError_t launch_qcache_store(const QStoreArgs &a, int chains, int max_rows, hipStream_t s);

struct QAttnArgs {
  QCacheArgs c;
  ChainRows rows;
  const int *key_len;       // [chains] or null (all tokens)
  const bf16 *q;
  long long ldq;
  float scale_log2;         // softmax scale times log2(e)
  bf16 *out;
  long long ldo;
  int chains;               // (set by launch_qattention)
  int splits;
  float *part;              // [splits][rows][heads * 72] (splits > 1)
  float *ml;                // [splits][rows][heads][2]: log2-domain reference and denominator
  int total_rows;
};
constexpr int kQMaxSplits = 16;
constexpr long kQMaxSplitRows = 1L << 18;  // rows x heads x splits of a split plan
constexpr long long kQMaxWorkgroups = 1LL << 23;  // of one launch (a grid holds fewer than 2^32 threads)
struct QAttnPlan {
  int qh, splits;        // qh: 32-query halves per wave, or 0: 16 queries per workgroup
  long long workgroups;  // a plan of more than kQMaxWorkgroups is not launched
};
// Query rows of the chains: offsets [chains + 1] on the host, or null: `tokens` rows each.
QAttnPlan plan_qattention(const int *offsets, int chains, int heads, int tokens);
hipError_t launch_qattention(const QAttnArgs &a, int chains, const QAttnPlan &p, hipStream_t s);
hipError_t launch_qattention_combine(const QAttnArgs &a, hipStream_t s);  // (splits > 1)

// ------------------------------------------------------------------ device side

// Scale byte of a block whose largest finite magnitude is amax >= 0.
__device__ __forceinline__ int q_exponent(float amax) {
  const unsigned u = __float_as_uint(amax);
  return max((int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0), 1);
}
// 2^(127 - e): what a value is multiplied by before it is rounded (e in 1..247: 2^126 .. 2^-120, exact).
__device__ __forceinline__ float q_inverse(int e) { return __uint_as_float((unsigned)(254 - e) << 23); }
// 2^(e - 127) as the scale operand of a conversion (of which only the exponent counts).
__device__ __forceinline__ float q_factor(int e) { return __uint_as_float((unsigned)e << 23); }
// |x|, or 0 where x is not finite.
__device__ __forceinline__ float q_magnitude(float x) {
  const float m = fabsf(x);
  return m <= 3.402823466e38f ? m : 0.0f;
}
// Four values to e4m3, nearest even; not finite: NaN (the conversion of an
// infinity would depend on the wave's clamp mode).
__device__ __forceinline__ uint32_t q_pack4(const float *x, float inv) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = fabsf(x[i]) <= 3.402823466e38f ? x[i] * inv : __builtin_nanf("");
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
  return (uint32_t)r;
}
// Maximum over the 16 lanes of a DPP row.
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, dpp_mov<0xB1>(v));
  v = fmaxf(v, dpp_mov<0x4E>(v));
  v = fmaxf(v, dpp_mov<0x141>(v));
  return fmaxf(v, dpp_mov<0x140>(v));
}

typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Eight e4m3 values times a power of two, in bfloat16 (exact from 2^-133 on).
__device__ __forceinline__ bf16x8 q_bf16x8(u32x2 v, float factor) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[0], factor, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[0], factor, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[1], factor, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[1], factor, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
// The same in float32.
__device__ __forceinline__ void q_f32x8(u32x2 v, float factor, float *x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i], true);
    x[4 * i] = a[0] * factor;
    x[4 * i + 1] = a[1] * factor;
    x[4 * i + 2] = b[0] * factor;
    x[4 * i + 3] = b[1] * factor;
  }
}

}  // namespace rc
