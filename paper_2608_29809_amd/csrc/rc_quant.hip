// Block quantisation to e4m3 with power-of-two scales, and the merge of fresh
// keys and values into an 8-bit cache.
#include "rc_common.h"
#include "rc_launch.h"
#include "rc_quant.h"

namespace rc {

template <typename T> __device__ __forceinline__ void q_load8(const T *p, float *v);
template <> __device__ __forceinline__ void q_load8<float>(const float *p, float *v) {
  const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}
template <> __device__ __forceinline__ void q_load8<bf16>(const bf16 *p, float *v) {
  const bf16x8 a = *(const bf16x8 *)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
}

// A scale for each row and 128 columns: sixteen lanes take a block, eight
// columns each, so that its maximum is four lane exchanges and nothing is read
// twice.  Bound by its bytes: 16384 x 4608 bfloat16 values 43 us (5.3 TB/s), 723 x
// 1152 2.8 us, most of it one load's latency.
template <typename T> __global__ __launch_bounds__(256) void quantize_rows_kernel(QuantArgs a, int cb) {
  const long long unit = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int row = (int)(unit / cb), kb = (int)(unit - (long long)row * cb), l = threadIdx.x & 15;
  if (row >= a.rows) return;
  const int col = kb * kQBlock + l * 8;
  float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  if (col < a.cols) q_load8<T>((const T *)a.x + row * a.ldx + col, v);
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, q_magnitude(v[i]));
  const int e = q_exponent(row16_max(m));
  const float inv = q_inverse(e);
  if (col < a.cols) *(u32x2 *)(a.q + row * a.ldq + col) = u32x2{q_pack4(v, inv), q_pack4(v + 4, inv)};
  if (l == 0) a.scales[(size_t)kb * a.scale_ld + row] = (uint8_t)e;
}

// A scale for each 128 x 128 tile: one workgroup each, 64 values per thread, held
// in registers from the maximum to the rounding.  Bound by its bytes: 16384 x
// 4608 float32 values 70 us (5.4 TB/s), 4608 x 1152 8 us (324 workgroups).
template <typename T> __global__ __launch_bounds__(256) void quantize_tiles_kernel(QuantArgs a, int cb) {
  __shared__ float red[4];
  const int rb = blockIdx.x / cb, kb = blockIdx.x - rb * cb, tid = threadIdx.x;
  const int col = kb * kQBlock + (tid & 15) * 8, row0 = rb * kQBlock + (tid >> 4);
  float v[8][8], m = 0.0f;
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int row = row0 + p * 16;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[p][i] = 0.0f;
    if (row < a.rows && col < a.cols) q_load8<T>((const T *)a.x + row * a.ldx + col, v[p]);
  }
#pragma unroll
  for (int p = 0; p < 8; ++p)
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, q_magnitude(v[p][i]));
  m = wave_max(m);
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
  const int e = q_exponent(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
  const float inv = q_inverse(e);
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int row = row0 + p * 16;
    if (row < a.rows && col < a.cols)
      *(u32x2 *)(a.q + row * a.ldq + col) = u32x2{q_pack4(v[p], inv), q_pack4(v[p] + 4, inv)};
  }
  if (tid == 0) a.scales[(size_t)kb * a.scale_ld + rb] = (uint8_t)e;
}

template <typename T> hipError_t launch_quantize(const QuantArgs &a, int block_rows, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  const int cb = (a.cols + kQBlock - 1) / kQBlock;
  if (block_rows == 1) {
    const long long units = (long long)a.rows * cb;
    rc_launch(quantize_rows_kernel<T>, dim3((unsigned)((units + 15) / 16)), dim3(256), 0, s, a, cb);
  } else {
    rc_launch(quantize_tiles_kernel<T>, dim3((unsigned)((a.rows + kQBlock - 1) / kQBlock * cb)), dim3(256), 0, s, a, cb);
  }
  return hipGetLastError();
}
template hipError_t launch_quantize<bf16>(const QuantArgs &, int, hipStream_t);
template hipError_t launch_quantize<float>(const QuantArgs &, int, hipStream_t);

// One workgroup per row; a block of 128 columns is 32 lanes of four.  Bound by
// its bytes and the two sums' round trips: 16384 rows of 1152 24 us (3.9 TB/s),
// 676 rows 4.1 us.
__global__ __launch_bounds__(256) void norm_quantize_kernel(NormQuantArgs a) {
  __shared__ float red[4];
  const int r = blockIdx.x, t = threadIdx.x, C4 = a.C >> 2;
  constexpr int MAXV = 2;  // C <= 4 * 256 * MAXV
  const float *X = a.X + (size_t)r * a.C;
  const f32x4 zero4 = {0.0f, 0.0f, 0.0f, 0.0f};
  f32x4 x[MAXV], shift[MAXV], scale[MAXV];
  const float *sh = a.sst + (size_t)a.shift_row * a.C, *tsh = a.t0 + (size_t)a.shift_row * a.C;
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < MAXV; ++i) {
    const int n = (t + 256 * i) * 4;
    const bool in = n < a.C;
    x[i] = in ? *(const f32x4 *)(X + n) : zero4;
    shift[i] = in ? *(const f32x4 *)(sh + n) + *(const f32x4 *)(tsh + n) : zero4;
    scale[i] = in ? *(const f32x4 *)(sh + a.C + n) + *(const f32x4 *)(tsh + a.C + n) : zero4;
    s += (x[i][0] + x[i][1]) + (x[i][2] + x[i][3]);
  }
  const float mean = block4_sum(s, red) / a.C;
  float d2 = 0.0f;
#pragma unroll
  for (int i = 0; i < MAXV; ++i)
    if (t + 256 * i < C4)
#pragma unroll
      for (int e = 0; e < 4; ++e) d2 += (x[i][e] - mean) * (x[i][e] - mean);
  const float rstd = rsqrtf(block4_sum(d2, red) / a.C + a.eps);
#pragma unroll
  for (int i = 0; i < MAXV; ++i) {
    const int n = (t + 256 * i) * 4;
    float v[4], m = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = (x[i][e] - mean) * rstd * (1.0f + scale[i][e]) + shift[i][e];
      m = fmaxf(m, q_magnitude(v[e]));
    }
    m = row16_max(m);
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    const int e8 = q_exponent(m);
    if (n >= a.C) continue;
    *(uint32_t *)(a.q + (size_t)r * a.C + n) = q_pack4(v, q_inverse(e8));
    if ((t & 31) == 0) a.scales[(size_t)(n / kQBlock) * a.scale_ld + r] = (uint8_t)e8;
  }
}

hipError_t launch_norm_quantize(const NormQuantArgs &a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  if (a.C % kQBlock || a.C > 2048) return hipErrorInvalidValue;
  rc_launch(norm_quantize_kernel, dim3(a.rows), dim3(256), 0, s, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------ cache store

// A workgroup takes one head's keys or values in the blocks of 64 tokens whose
// first active row is among its `chunk` rows of the list.  A block's fresh rows
// take the places of their tokens, the others keep their values; the scale is
// that of the merged tile.  Bound by latency for a region (the list, then the
// values and the old tile: 729 tokens of a 4096-token cache 6.8 us), by its bytes
// for every token of a dense step (idx null: workgroup x takes block x): two
// chains of 16384 tokens from float32 73 us, 5.2 TB/s.
template <typename T> __global__ __launch_bounds__(192) void qcache_store_kernel(QStoreArgs a, int chunk) {
  constexpr int CPR = kHeadDim / 8;  // chunks of eight values per token
  __shared__ int row_of[kQTokens];
  __shared__ float red[3];
  const int tid = threadIdx.x, lane = tid & 63, head = blockIdx.y >> 1, which = blockIdx.y & 1, b = blockIdx.z;
  const int2 rr = chain_rows(a.rows, b);
  const int blocks = a.c.tokens / kQTokens, r0 = rr.x + (int)blockIdx.x * chunk;
  // list entries r0 - 1 + lane and r0 + 63 + lane (the same in every wave); the
  // blocks that begin here (its first lanes of them)
  int tok0 = -1, tok1 = -1;
  unsigned long long first = 1;
  if (a.idx) {
    if (r0 >= rr.y) return;
    const int at = r0 - 1 + lane;
    if (at >= rr.x && at < rr.y) tok0 = a.idx[at];
    if (at + 64 < rr.y) tok1 = a.idx[at + 64];
    const int before = __shfl_up(tok0, 1, 64);
    first = __ballot(lane >= 1 && lane <= chunk && tok0 >= 0 && (before < 0 || (before >> 6) != (tok0 >> 6)));
  }
  for (; first; first &= first - 1) {
    const int pos = __ffsll((long long)first) - 1;
    const int blk = a.idx ? __shfl(tok0, pos, 64) >> 6 : (int)blockIdx.x;
    if (blk >= blocks) break;  // (an invalid list: nothing is written)
    // rows of the block (contiguous, from any_row on; all of it: a dense step's)
    const int any_row = a.idx ? r0 - 1 + pos : rr.x + blk * kQTokens;
    const bool full = !a.idx || __popcll(__ballot(tok0 >= 0 && tok0 >> 6 == blk && lane >= pos)) +
                                        __popcll(__ballot(tok1 >= 0 && tok1 >> 6 == blk)) == kQTokens;
    __syncthreads();           // the block before is done with row_of and red
    if (tid < 64) {
      row_of[lane] = a.idx ? -1 : rr.x + blk * kQTokens + lane;
      __builtin_amdgcn_wave_barrier();
      if (a.idx) {
        if (lane >= pos && tok0 >= 0 && tok0 >> 6 == blk) row_of[tok0 & 63] = r0 - 1 + lane;
        if (tok1 >= 0 && tok1 >> 6 == blk) row_of[tok1 & 63] = r0 + 63 + lane;
      }
    }
    __syncthreads();
    const size_t tile = ((size_t)head * blocks + blk) * 2 + which;
    uint8_t *data = a.c.data + b * a.c.chain_stride + tile * kQTileBytes;
    uint8_t *scale = a.c.scales + b * a.c.scale_chain_stride + tile;
    const T *src = (const T *)(which ? a.v : a.k) + head * kHeadDim;
    // every load before the first use: fresh rows (kept tokens read the block's
    // first one), and the old tile unless every token is fresh
    float v[3][8], old = 0.0f, m = 0.0f;
    u32x2 kept[3];
    int r[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const int c = tid + i * 192, tok = c / CPR, d = (c - tok * CPR) * 8;
      r[i] = row_of[tok];
      kept[i] = u32x2{0u, 0u};
      if (!full) kept[i] = *(const u32x2 *)(data + c * 8);
      q_load8<T>(src + (r[i] >= 0 ? r[i] : any_row) * a.ld + d, v[i]);
    }
    if (!full) old = q_factor(*scale);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      float w[8];
      q_f32x8(kept[i], old, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[i][k] = r[i] >= 0 ? v[i][k] : w[k];
        m = fmaxf(m, q_magnitude(v[i][k]));
      }
    }
    m = wave_max(m);
    if (lane == 0) red[tid >> 6] = m;
    __syncthreads();
    const int e = q_exponent(fmaxf(fmaxf(red[0], red[1]), red[2]));
    const float inv = q_inverse(e);
#pragma unroll
    for (int i = 0; i < 3; ++i) *(u32x2 *)(data + (tid + i * 192) * 8) = u32x2{q_pack4(v[i], inv), q_pack4(v[i] + 4, inv)};
    if (tid == 0) *scale = (uint8_t)e;
  }
}

// Rows per workgroup: as few (down to 1, at most 32) as leave no more workgroups
// than run at once, about 1536, so that scattered tokens, each with a block of
// its own, are spread too.
template <typename T> hipError_t launch_qcache_store(const QStoreArgs &a, int chains, int max_rows, hipStream_t s) {
  if (chains <= 0 || max_rows <= 0) return hipSuccess;
  int chunk = 1;
  while (chunk < 32 && (long long)(max_rows + chunk - 1) / chunk * 2 * a.c.heads * chains > 1536) chunk *= 2;
  const int x = a.idx ? (max_rows + chunk - 1) / chunk : a.c.tokens / kQTokens;
  rc_launch(qcache_store_kernel<T>, dim3(x, 2 * a.c.heads, chains), dim3(192), 0, s, a, chunk);
  return hipGetLastError();
}
template hipError_t launch_qcache_store<bf16>(const QStoreArgs &, int, int, hipStream_t);
template hipError_t launch_qcache_store<float>(const QStoreArgs &, int, int, hipStream_t);

}  // namespace rc
