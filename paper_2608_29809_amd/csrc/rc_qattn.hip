// Attention of bfloat16 queries over an 8-bit cache (head dim 72): queries of
// one (chain, head) against the first key_len keys of the chain, key ranges
// (splits) joined by a second kernel.
//
// Scores are formed transposed (S^T = K Q^T), so a lane owns one query and its
// probabilities are in registers the B operand of O^T = V^T P^T.  Keys and
// values become bfloat16 with their block's scale as they are read from LDS
// (exact: e4m3 times a power of two), so the products are those of the
// bfloat16 attention; values are transposed by 8-bit transpose reads.  The
// probabilities are rounded to bfloat16 (2^-9 relative each, averaged by the
// sum), the denominator sums the rounded ones.
#include "rc_common.h"
#include "rc_launch.h"
#include "rc_quant.h"

#include <algorithm>
#include <cmath>

namespace rc {

// key that lane m of a 32-key operand supplies, so that accumulator
// e = c*8 + k of lane group g is key c*16 + g*8 + k
__device__ __forceinline__ int key_perm8(int m) {
  return ((m >> 4) & 1) * 16 + ((m >> 2) & 1) * 8 + ((m >> 3) & 1) * 4 + (m & 3);
}

__global__ __launch_bounds__(256) void qattn_kernel(QAttnArgs a) {
  constexpr int D = kHeadDim;
  __shared__ __attribute__((aligned(16))) char tile[2 * kQTileBytes];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 5, r32 = lane & 31;
  const int heads = a.c.heads, qt = blockIdx.x, h = blockIdx.y % heads, split = blockIdx.y / heads, b = blockIdx.z;
  const int2 rr = chain_rows(a.rows, b);
  const int q0 = rr.x + qt * 128;
  if (q0 >= rr.y) return;
  const int keys = a.key_len ? max(0, min(a.key_len[b], a.c.tokens)) : a.c.tokens;
  const int n_tiles = (keys + kQTokens - 1) / kQTokens;
  const int t0 = (int)((long long)split * n_tiles / a.splits), t1 = (int)((long long)(split + 1) * n_tiles / a.splits);
  const uint8_t *data = a.c.data + b * a.c.chain_stride + (size_t)h * (a.c.tokens / kQTokens) * 2 * kQTileBytes;
  const uint8_t *scales = a.c.scales + b * a.c.scale_chain_stride + (size_t)h * (a.c.tokens / kQTokens) * 2;
  const int my_q = q0 + wave * 32 + r32;
  const bf16 *qrow = a.q + min(my_q, rr.y - 1) * a.ldq + h * D;
  bf16x8 qf[5];
#pragma unroll
  for (int c = 0; c < 5; ++c) {
    const int d0 = c * 16 + g * 8;
    qf[c] = Mfma<bf16>::zero();
    if (d0 < D) qf[c] = *(const bf16x8 *)(qrow + d0);
  }
  const f32x16 zero16 = {};
  f32x16 o[3] = {zero16, zero16, zero16};  // dims 0..95 (72: the denominator's row)
  float m_run = -INFINITY;
  const int tw = lane >> 4, tj = lane & 15;
  typedef int v2i __attribute__((ext_vector_type(2)));
  for (int t = t0; t < t1; ++t) {
    __syncthreads();
    for (int c = tid; c < 2 * kQTileBytes / 16; c += 256) {
      u32x4 v = *(const u32x4 *)(data + (size_t)t * 2 * kQTileBytes + c * 16);
      *(u32x4 *)(tile + c * 16) = v;
    }
    __syncthreads();
    const int left = keys - t * kQTokens;
    if (left < kQTokens) {  // values of masked keys may be anything: zeros
      for (int i = left * D + tid; i < kQTileBytes; i += 256) tile[kQTileBytes + i] = 0;
      __syncthreads();
    }
    const float fk = q_factor(scales[2 * t]), fv = q_factor(scales[2 * t + 1]);
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      const char *krow = tile + (st * 32 + key_perm8(r32)) * D + g * 8;
      f32x16 s = zero16;
#pragma unroll
      for (int c = 0; c < 5; ++c) {
        bf16x8 kf = Mfma<bf16>::zero();
        if (c * 16 + g * 8 < D) kf = q_bf16x8(*(const u32x2 *)(krow + c * 16), fk);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[c], s, 0, 0, 0);
      }
      float m = m_run;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = st * 32 + (e >> 3) * 16 + g * 8 + (e & 7);
        s[e] = key < left ? s[e] * a.scale_log2 : -INFINITY;
        m = fmaxf(m, s[e]);
      }
      m = half_swap_max(m);
      const float ref = m == -INFINITY ? 0.0f : m, f = exp2f(m_run - ref);
      m_run = m;
      bf16x8 pf[2];
#pragma unroll
      for (int e = 0; e < 16; ++e) pf[e >> 3][e & 7] = (bf16)exp2f(s[e] - ref);
#pragma unroll
      for (int d = 0; d < 3; ++d) {
        o[d] *= f;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int key = st * 32 + c * 16 + g * 8 + (tj >> 1), dim = d * 32 + 16 * (tw & 1) + 8 * (tj & 1);
          const v2i raw = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
              (__attribute__((address_space(3))) v2i *)(tile + kQTileBytes + key * D + min(dim, D - 8)));
          bf16x8 vf = q_bf16x8(u32x2{(uint32_t)raw[0], (uint32_t)raw[1]}, fv);
          if (d == 2 && r32 >= 8) {
#pragma unroll
            for (int k = 0; k < 8; ++k) vf[k] = (bf16)(r32 == 8 ? 1.0f : 0.0f);
          }
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[c], o[d], 0, 0, 0);
        }
      }
    }
  }
  // dim 72 is row 8 of the last block: element 4 of lane group 0
  const float den = __shfl(o[2][4], r32, 64), inv = den > 0.0f ? 1.0f / den : den == 0.0f ? 0.0f : den;
  if (my_q >= rr.y) return;
#pragma unroll
  for (int d = 0; d < 3; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int dim = d * 32 + i * 8 + g * 4;
      if (dim >= D) continue;
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = o[d][i * 4 + e] * inv;
      if (a.splits == 1) {
        *(bf16x4 *)(a.out + my_q * a.ldo + h * D + dim) = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
      } else {
        *(f32x4 *)(a.part + ((size_t)split * a.total_rows + my_q) * heads * D + h * D + dim) = v;
      }
    }
  if (a.splits > 1 && g == 0) {
    float *ml = a.ml + (((size_t)split * a.total_rows + my_q) * heads + h) * 2;
    ml[0] = m_run;
    ml[1] = den;
  }
}

// O = sum_s w_s O_s / sum_s w_s, w_s = 2^(m_s - max m) l_s, in split order.  A
// range without keys has m = -inf and weight 0; a row without keys is 0.
__global__ __launch_bounds__(64) void qattn_combine_kernel(QAttnArgs a) {
  constexpr int G = kHeadDim / 4;
  const int heads = a.c.heads, C = heads * kHeadDim;
  const long long i = (long long)blockIdx.x * 64 + threadIdx.x;
  if (i >= (long long)a.total_rows * heads * G) return;
  const int r = (int)(i / (heads * G)), rem = (int)(i - (long long)r * heads * G), h = rem / G, d = (rem - h * G) * 4;
  float M = -INFINITY;
  for (int s = 0; s < a.splits; ++s) M = fmaxf(M, a.ml[(((size_t)s * a.total_rows + r) * heads + h) * 2]);
  f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
  float den = 0.0f;
  for (int s = 0; s < a.splits; ++s) {
    const float *ml = a.ml + (((size_t)s * a.total_rows + r) * heads + h) * 2;
    const float w = ml[0] == -INFINITY ? 0.0f : exp2f(ml[0] - M) * ml[1];
    num += w * *(const f32x4 *)(a.part + ((size_t)s * a.total_rows + r) * C + h * kHeadDim + d);
    den += w;
  }
  const float inv = den > 0.0f ? 1.0f / den : den == 0.0f ? 0.0f : den;
  *(bf16x4 *)(a.out + r * a.ldo + h * kHeadDim + d) =
      bf16x4{(bf16)(num[0] * inv), (bf16)(num[1] * inv), (bf16)(num[2] * inv), (bf16)(num[3] * inv)};
}

QAttnPlan plan_qattention(const int *offsets, int chains, int heads, int tokens) {
  long tiles = 0;
  for (int b = 0; b < chains; ++b) tiles += (offsets[b + 1] - offsets[b] + 127) / 128;
  const int n_tiles = tokens / kQTokens;
  int splits = 1;
  while (splits < 16 && splits * 2 <= n_tiles && tiles * heads * splits < 512) splits *= 2;
  return QAttnPlan{splits};
}

hipError_t launch_qattention(const QAttnArgs &a, int chains, int max_rows, hipStream_t s) {
  if (max_rows <= 0 || a.total_rows <= 0) return hipSuccess;
  rc_launch(qattn_kernel, dim3((max_rows + 127) / 128, a.c.heads * a.splits, chains), dim3(256), 0, s, a);
  if (a.splits > 1) {
    const long long n = (long long)a.total_rows * a.c.heads * (kHeadDim / 4);
    rc_launch(qattn_combine_kernel, dim3((unsigned)((n + 63) / 64)), dim3(64), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace rc
