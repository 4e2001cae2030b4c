// Quantisation of rows to int8.
#include "rc_common.h"
#include "rc_int8.h"
#include "rc_launch.h"

namespace rc {

template <typename T> struct I8Raw;
template <> struct I8Raw<float> {
  f32x4 w[2];
  __device__ __forceinline__ void load(const float *p) {
    w[0] = *(const f32x4 *)p;
    w[1] = *(const f32x4 *)(p + 4);
  }
  __device__ __forceinline__ float value(int e) const { return w[e >> 2][e & 3]; }
};
template <> struct I8Raw<bf16> {
  bf16x8 w;
  __device__ __forceinline__ void load(const bf16 *p) { w = *(const bf16x8 *)p; }
  __device__ __forceinline__ float value(int e) const { return (float)w[e]; }
};

// One pass over the data: a row stays in the registers of the threads that share
// it, eight columns times U each, from the maximum to the rounding: sixteen lanes
// (L = 16), a wave (L = 64) or a workgroup of as many waves as it takes (L = 0).
// Columns behind the last are copies of the last eight and not stored.  Bound by
// its bytes for many rows: 16384 x 4608 bfloat16 values 42-45 us (5.0-5.4 TB/s), 4096 x 4608
// 12.5-14.5, 4608 x 1152 float32 6.5; by latency for few: 723 x 4608 4.6, of which a
// launch is 3.  Rows one after another by fewer workgroups, the next one sent for
// ahead, were slower (4096 x 4608: 18.7 us), as was a unit a thread (18.6): what the
// threads of a row do once, the exchanges, is spread over more values.
template <int L, int U, typename T>
__global__ __launch_bounds__(L ? 256 : 1024) void quantize_int8_kernel(QuantInt8Args a, int chunk) {
  constexpr int G = L ? 256 / L : 1, LANES = L == 16 ? 16 : 64;
  __shared__ uint32_t tops[2][16];
  const int lane = threadIdx.x & 63, wave = L ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = L ? 1 : blockDim.x >> 6, t = threadIdx.x & (LANES - 1);
  long long first = (long long)blockIdx.x * G * chunk;
  if (L == 64) first += __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * chunk;
  if (L == 16) first += threadIdx.x / 16 * chunk;
  const long long end = min(first + chunk, (long long)a.rows);
  int col[U];
  bool mine[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = wave * 512 * U + (u * LANES + t) * 8;
    mine[u] = c < a.cols;
    col[u] = min(c, a.cols - 8);
  }
  I8Raw<T> raw[U];
  auto load = [&](long long row) {
    const T *x = (const T *)a.x + row * a.ldx;
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u].load(x + col[u]);
  };
  int odd = 0;
#pragma nounroll
  for (long long r = first; r < end; ++r, odd ^= 1) {
    load(r);
    float v[U][8];
    uint32_t m = 0;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[u][e] = raw[u].value(e);
        m = max(m, i8_magnitude(v[u][e]));
      }
    m = lanes_umax<LANES>(m);
    if constexpr (L == 0) {
      if (lane == 0) tops[odd][wave] = m;
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      m = row16_umax(tops[odd][min(lane & 15, waves - 1)]);
    }
    const float s = i8_scale(m), inv = i8_inverse(s);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t q[2];
      i8_pack8(v[u], s, inv, q);
      if (mine[u]) *(u32x2 *)(a.q + r * a.ldq + col[u]) = u32x2{q[0], q[1]};
    }
    if (wave == 0 && t == 0) a.scales[r] = s;
  }
}

template <typename T> hipError_t launch_quantize_int8(const QuantInt8Args &a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  auto run = [&](auto kernel, int threads, int rows_at_once) {
    const long long groups = ((long long)a.rows + rows_at_once - 1) / rows_at_once;
    const int chunk = (int)((groups + (1 << 21) - 1) >> 21);  // (a grid holds fewer than 2^32 threads)
    rc_launch(kernel, dim3((unsigned)((groups + chunk - 1) / chunk)), dim3(threads), 0, s, a, chunk);
    return hipGetLastError();
  };
  if (a.cols <= 128) return run(quantize_int8_kernel<16, 1, T>, 256, 16);
  if (a.cols <= 512) return run(quantize_int8_kernel<64, 1, T>, 256, 4);
  if (a.cols <= 1024) return run(quantize_int8_kernel<64, 2, T>, 256, 4);
  if (a.cols <= 1536) return run(quantize_int8_kernel<64, 3, T>, 256, 4);
  if (a.cols <= 16384) return run(quantize_int8_kernel<0, 2, T>, (a.cols + 1023) / 1024 * 64, 1);
  return run(quantize_int8_kernel<0, 8, T>, (a.cols + 4095) / 4096 * 64, 1);
}
template hipError_t launch_quantize_int8<bf16>(const QuantInt8Args &, hipStream_t);
template hipError_t launch_quantize_int8<float>(const QuantInt8Args &, hipStream_t);

}  // namespace rc
