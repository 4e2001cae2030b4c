// Norms before and after a block, with the gated residual update between them.
#include "rc_norm.h"

#include <algorithm>
#include <type_traits>

#include "rc_common.h"
#include "rc_int8.h"
#include "rc_launch.h"

namespace rc {

// How a row's columns are loaded, eight to a thread: rows and vectors at
// multiples of 16 bytes and whole units of eight; at any element, the last unit's
// columns being the row's last eight, of which it ignores those that the unit
// before has; rows of less than eight columns, one by one.
enum NormForm { NF_WHOLE = 0, NF_ANY = 1, NF_TINY = 2 };

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));

// Eight values as they lie in memory.
template <typename T> struct Raw8;
template <> struct Raw8<float> {
  f32x4 w[2];
  __device__ __forceinline__ void values(float *v) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = w[e >> 2][e & 3];
  }
};
template <> struct Raw8<bf16> {
  bf16x8 w;
  __device__ __forceinline__ void values(float *v) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)w[e];
  }
};
template <> struct Raw8<void> {};
template <int FORM> __device__ __forceinline__ void n_load8(Raw8<float> &r, const float *p, int n) {
  if constexpr (FORM == NF_WHOLE) {
    r.w[0] = *(const f32x4 *)p;
    r.w[1] = *(const f32x4 *)(p + 4);
  } else if constexpr (FORM == NF_ANY) {
    r.w[0] = *(const f32x4_any *)p;
    r.w[1] = *(const f32x4_any *)(p + 4);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.w[e >> 2][e & 3] = p[min(e, n - 1)];
  }
}
template <int FORM> __device__ __forceinline__ void n_load8(Raw8<bf16> &r, const bf16 *p, int n) {
  if constexpr (FORM == NF_WHOLE) {
    r.w = *(const bf16x8 *)p;
  } else if constexpr (FORM == NF_ANY) {
    r.w = *(const bf16x8_any *)p;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.w[e] = p[min(e, n - 1)];
  }
}
// Those from value `from` on (tiny rows: of n).
template <int FORM, typename T> __device__ __forceinline__ void n_store8(T *p, const float *v, int from, int n) {
  if (FORM != NF_TINY && from == 0) {
    if constexpr (std::is_same<T, bf16>::value) {
      const bf16x8 a = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3], (bf16)v[4], (bf16)v[5], (bf16)v[6], (bf16)v[7]};
      if constexpr (FORM == NF_WHOLE) *(bf16x8 *)p = a;
      else *(bf16x8_any *)p = a;
    } else {
      const f32x4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
      if constexpr (FORM == NF_WHOLE) {
        *(f32x4 *)p = a;
        *(f32x4 *)(p + 4) = b;
      } else {
        *(f32x4_any *)p = a;
        *(f32x4_any *)(p + 4) = b;
      }
    }
  } else if (FORM != NF_WHOLE) {
    if (FORM == NF_ANY) asm volatile("" : "+v"(from));
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= from && (FORM == NF_ANY || e < n)) p[e] = (T)v[e];
  }
}

// Sum over the lanes that share a row (L = 16: a DPP row, else the wave), the
// same in all of them and in the same order every time.
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
  v = row16_sum(v);
  if constexpr (L == 64) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(q[0]) + __uint_as_float(q[1]);
  }
  return v;
}
constexpr int kNormWaves = 16;  // most that share a row
template <typename H> constexpr bool kUpdate = !std::is_same<H, void>::value;  // h of type H, or none
// Waves of a SIMD that the registers leave: 6 (80 registers) where a wave or more share a row, one
// unit each; not 16 lanes' chains, which differ within a wave, nor, at 4, theirs with an update.  No
// vector register is spilled but two of <0, 1, NF_ANY, float, void>; scalar ones are, to lanes of a
// vector register: up to 22 with an update, of rows under eight columns 42, and 109 to 123 with one.
template <int L, int U, typename H> constexpr int kNormResident = L == 16 ? (kUpdate<H> ? 3 : 4) : U == 1 && !kUpdate<H> ? 6 : 4;

// One pass over the data: a row stays in the registers of the threads that share
// it, 8 U values each: sixteen lanes (L = 16), a wave (L = 64) or a workgroup of
// as many waves as 512 U columns each ask for (L = 0).  A workgroup takes `chunk`
// rows one after another; the next one's values are sent for before the row is
// worked on, and the vectors stay in registers (KEEP) while the chain does.
//
// A wave's variance is that of differences from its own mean; waves are joined by
// sum_w (M_w + n_w (m_w - mean)^2), which needs one exchange through LDS where
// mean and variance one after another would need two, and does not cancel as
// sums of squares do.
//
// Bound by its bytes for many rows: an update of 16384 x 1152 float32 values by
// bfloat16 ones with the next norm 49 us (4.6 TB/s), alone 41; a norm of them to bfloat16
// 22.5 (5.0 TB/s); by instructions and the exchanges' waits where results are 8 bits (4096 x
// 4608 bfloat16 to e4m3 17-18 us, to int8 21-22.5; with an update to e4m3 28, but to int8 47:
// one workgroup a CU, which waits at two exchanges a row); by latency for few rows (723 x
// 1152 to int8 4.5 us, with an update 5.4; one row 2.6, a launch).  One row a workgroup
// without `chunk` loads the vectors for each (16384 x 1152: 30 us where it then took 24.5 with
// it); two rows at a time, whose exchanges are one, were slower (26).
template <int L, int U, int FORM, typename X, typename H>
__global__ __launch_bounds__(L ? 256 : 1024, (kNormResident<L, U, H>)) void norm_kernel(NormArgs a, int chunk) {
  constexpr bool RES = kUpdate<H>;
  constexpr int G = L ? 256 / L : 1, LANES = L == 16 ? 16 : 64;  // rows of a workgroup at a time; lanes of a wave that share a row
  __shared__ float2 parts[L ? 1 : 2][2][kNormWaves];             // of post, pre; rows of even and odd number
  __shared__ uint32_t tops[L ? 1 : 2][kNormWaves];
  const int lane = threadIdx.x & 63, wave = L ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cols = a.cols, waves = L ? 1 : blockDim.x >> 6, t = threadIdx.x & (LANES - 1);
  const int n_wave = min(LANES * 8 * U, cols - wave * 512 * U);  // values of this wave
  const float per_wave = 1.0f / n_wave, per_row = 1.0f / cols;
  long long first = (long long)blockIdx.x * G * chunk;
  if (L == 64) first += __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * chunk;
  if (L == 16) first += threadIdx.x / 16 * chunk;

  // The thread's units: columns col[u] .. + 7, of which it has those from skip[u]
  // on (none from 8 on; the others are another thread's).
  int col[U], skip[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = wave * 512 * U + (u * LANES + t) * 8;
    col[u] = FORM == NF_TINY ? 0 : min(c, cols - 8);
    skip[u] = FORM == NF_TINY ? c : c - col[u];
  }
  auto none = [&](int u) { return FORM == NF_WHOLE ? skip[u] != 0 : skip[u] >= 8; };
  auto drop = [&](int u, float *v) {  // zeros where another thread, or none, has the value
    if constexpr (FORM != NF_WHOLE)
      if (FORM == NF_TINY || skip[u]) {
        int from = skip[u];
        if (FORM == NF_ANY) asm volatile("" : "+v"(from));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e >= from && (FORM != NF_TINY || e < cols) ? v[e] : 0.0f;
      }
  };

  // v becomes its difference from the wave's mean; that from the row's is v + off.
  auto statistics = [&](const NormSpec &n, float (&v)[U][8], float2 *part, float &off, float &rstd) {
    float mean = 0.0f;
    if (n.kind == NORM_LAYER) {
      float s = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        drop(u, v[u]);
        const float p = ((v[u][0] + v[u][1]) + (v[u][2] + v[u][3])) + ((v[u][4] + v[u][5]) + (v[u][6] + v[u][7]));
        s += FORM == NF_WHOLE && none(u) ? 0.0f : p;
      }
      mean = lanes_sum<LANES>(s) * per_wave;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] -= mean;
    }
    float q = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      drop(u, v[u]);
      float p = v[u][0] * v[u][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) p = __builtin_fmaf(v[u][e], v[u][e], p);
      q += FORM == NF_WHOLE && none(u) ? 0.0f : p;
    }
    q = lanes_sum<LANES>(q);
    off = 0.0f;
    if constexpr (L == 0) {
      if (lane == 0) part[wave] = make_float2(mean, q);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      const int w = lane & 15;
      const float n_w = w < waves ? (float)min(512 * U, cols - w * 512 * U) : 0.0f;
      const float2 p = part[min(w, waves - 1)];
      const float all = row16_sum(p.x * n_w) * per_row, d = p.x - all;
      q = row16_sum(w < waves ? __builtin_fmaf(d * d, n_w, p.y) : 0.0f);
      off = mean - all;
    }
    rstd = rsqrtf(q * per_row + n.eps);
  };

  // What the norm of the thread's columns is multiplied by and what is added:
  // weight and bias, and the modulation 1 + scale and shift, or the gate.
  typedef Raw8<float> Vec;
  struct Vectors {
    Vec weight, bias, factor, shift;
  };
  auto load_vectors = [&](int has, const NormSpec &n, const float *factor, const float *shift, int u, Vectors &v) {
    if (has & NV_WEIGHT) n_load8<FORM>(v.weight, n.weight + col[u], cols);
    if (has & NV_BIAS) n_load8<FORM>(v.bias, n.bias + col[u], cols);
    if (has & NV_FACTOR) n_load8<FORM>(v.factor, factor + col[u], cols);
    if (has & NV_SHIFT) n_load8<FORM>(v.shift, shift + col[u], cols);
  };
  auto join_vectors = [&](int has, const Vectors &v, float one, float *mul, float *add) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      mul[e] = has & NV_FACTOR ? one + v.factor.w[e >> 2][e & 3] : 1.0f;
      add[e] = has & NV_BIAS ? mul[e] * v.bias.w[e >> 2][e & 3] : 0.0f;
      if (has & NV_WEIGHT) mul[e] *= v.weight.w[e >> 2][e & 3];
      if (has & NV_SHIFT) add[e] += v.shift.w[e >> 2][e & 3];
    }
  };
  constexpr bool KEEP = U == 1 || !RES;  // (of an update, two units' vectors and a next row do not fit 128 registers)
  float mul[U][8], add[U][8], post_mul[U][8], post_add[U][8];
  auto vectors = [&](int b, bool post, bool pre) {
    int of_h = a.post_has, of_x = a.pre_has;
    asm volatile("" : "+s"(of_h), "+s"(of_x));  // (decided here: ahead of the loop every bit would be a pair of registers, spilled: 0.5 us)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Vectors of_post, of_pre;  // (all are sent for before the first is waited for)
      if (post) load_vectors(of_h, a.post, a.gate + b * a.gate_stride, nullptr, u, of_post);
      if (pre) load_vectors(of_x, a.pre, a.scale + b * a.scale_stride, a.shift + b * a.shift_stride, u, of_pre);
      if (post) join_vectors(of_h, of_post, 0.0f, post_mul[u], post_add[u]);
      if (pre) join_vectors(of_x, of_pre, 1.0f, mul[u], add[u]);
    }
  };
  Raw8<X> raw_x[U];
  Raw8<H> raw_h[U];
  auto load = [&](long long row) {
    const X *px = (const X *)a.x + row * a.ldx;
#pragma unroll
    for (int u = 0; u < U; ++u) n_load8<FORM>(raw_x[u], px + col[u], cols);
    if constexpr (RES) {
      const H *ph = (const H *)a.h + row * a.ldh;
#pragma unroll
      for (int u = 0; u < U; ++u) n_load8<FORM>(raw_h[u], ph + col[u], cols);
    }
  };
  const long long last = a.rows - 1;
  if (L != 16 && first > last) return;
  if constexpr (KEEP) load(min(first, last));
  int chain = -1;
  int chain_end = 0;  // the first row of the next one
#pragma nounroll
  for (int i = 0; i < chunk; ++i) {
    const bool live = first + i <= last;
    if (L != 16 && !live) break;  // (of sixteen lanes, the wave's other rows need them all)
    const int r = (int)min(first + i, last);
    if (r >= chain_end) {
      int b = 0;
      chain_end = a.rows;
      if (a.chains > kQArgChains) {
        for (int hi = a.chains - 1; b < hi;) {
          const int mid = (b + hi) >> 1;
          if (a.chain.offsets[mid + 1] <= r) b = mid + 1;
          else hi = mid;
        }
        if (b < a.chains - 1) chain_end = a.chain.offsets[b + 1];
      } else if (a.chains > 1) {
#pragma unroll
        for (int k = 1; k < kQArgChains; ++k) {  // (behind the last chain: the rows' end)
          const int at = a.chain.arg[k];
          b += at <= r ? 1 : 0;
          chain_end = min(chain_end, at > r ? at : 0x7fffffff);
        }
      }
      if (KEEP && b != chain) vectors(b, RES, a.out_kind != NO_NONE);
      chain = b;
    }
    if constexpr (!KEEP) load(r);
    float x[U][8], h[U][8], off, rstd;
#pragma unroll
    for (int u = 0; u < U; ++u) raw_x[u].values(x[u]);
    if constexpr (RES)
#pragma unroll
      for (int u = 0; u < U; ++u) raw_h[u].values(h[u]);
    if (KEEP && i + 1 < chunk) load(min(first + i + 1, last));
    int kind = a.out_kind;
    if (L != 16) asm volatile("" : "+s"(kind));
    if constexpr (RES) {
      if constexpr (!KEEP) vectors(chain, true, false);
      off = 0.0f;
      rstd = 1.0f;
      if (a.post.kind != NORM_NONE) statistics(a.post, h, parts[0][i & 1], off, rstd);
      off *= rstd;
      X *px = (X *)a.x + r * a.ldx;
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = __builtin_fmaf(__builtin_fmaf(h[u][e], rstd, off), post_mul[u][e], post_add[u][e]);
          x[u][e] = __builtin_fmaf(a.residual_scale, x[u][e], p);
        }
        if (live && !none(u)) n_store8<FORM>(px + col[u], x[u], skip[u], cols);
      }
    }
    if (kind == NO_NONE) continue;
    if constexpr (!KEEP) vectors(chain, false, true);
    statistics(a.pre, x, parts[L ? 0 : 1][i & 1], off, rstd);
    off *= rstd;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[u][e] = __builtin_fmaf(__builtin_fmaf(x[u][e], rstd, off), mul[u][e], add[u][e]);
    if (kind == NO_F32) {
      float *po = (float *)a.out + r * a.ldo;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (live && !none(u)) n_store8<FORM>(po + col[u], x[u], skip[u], cols);
      continue;
    }
    if (kind == NO_BF16) {
      bf16 *po = (bf16 *)a.out + r * a.ldo;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (live && !none(u)) n_store8<FORM>(po + col[u], x[u], skip[u], cols);
      continue;
    }
    // (eight bits: the columns are a multiple of 16, units whole)
    if constexpr (FORM != NF_TINY) {
      uint8_t *po = (uint8_t *)a.out + r * a.ldo;
      uint32_t m[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        m[u] = i8_magnitude(x[u][0]);
#pragma unroll
        for (int e = 1; e < 8; ++e) m[u] = max(m[u], i8_magnitude(x[u][e]));
        if (none(u)) m[u] = 0;
      }
      if (kind == NO_E4M3) {  // sixteen threads have a block of 128 columns
#pragma unroll
        for (int u = 0; u < U; ++u) {
          uint32_t top = row16_umax(m[u]);
          if (__builtin_amdgcn_ballot_w64(top >= kI8NotFinite)) {  // what is not finite does not count
            float big = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) big = fmaxf(big, q_magnitude(x[u][e]));
            top = __float_as_uint(row16_max(none(u) ? 0.0f : big));
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] = fabsf(x[u][e]) <= 3.402823466e38f ? x[u][e] : __builtin_nanf("");
          }
          const int ex = q_exponent(__uint_as_float(top));
          const float inv = q_inverse(ex);
          uint32_t q[2];
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[u][4 * p] * inv, x[u][4 * p + 1] * inv, 0, false);
            q[p] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[u][4 * p + 2] * inv, x[u][4 * p + 3] * inv, lo, true);
          }
          if (live && !none(u)) {
            *(u32x2 *)(po + col[u]) = u32x2{q[0], q[1]};
            if ((lane & 15) == 0) ((uint8_t *)a.scales)[(size_t)(col[u] / kQBlock) * a.scale_ld + r] = (uint8_t)ex;
          }
        }
      } else {
        uint32_t top = m[0];
#pragma unroll
        for (int u = 1; u < U; ++u) top = max(top, m[u]);
        top = lanes_umax<LANES>(top);
        if constexpr (L == 0) {
          uint32_t *of_waves = tops[i & 1];
          if (lane == 0) of_waves[wave] = top;
          asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
          top = row16_umax(of_waves[min(lane & 15, waves - 1)]);
        }
        const float s = i8_scale(top), inv = i8_inverse(s);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          uint32_t q[2];
          i8_pack8(x[u], s, inv, q);
          if (live && !none(u)) *(u32x2 *)(po + col[u]) = u32x2{q[0], q[1]};
        }
        if (live && wave == 0 && t == 0) ((float *)a.scales)[r] = s;
      }
    }
  }
}

// Rows of a workgroup: as many as leave no more workgroups than run at once, a
// power of two a CU (2560 columns with an update: 2 or 3 a CU 25.6, 29.4 us).
// Two units a thread for many int8 results, whose second exchange is a wait more
// for every row (16384 x 1152 float32 29.6 -> 26.1 us, 4096 x 4608 bfloat16 29.0 -> 23.0,
// 2048 x 1152 7.6 -> 7.1; but 1376 x 1152 6.6 -> 6.8, 256 x 1152 4.1 -> 4.6, and with e4m3
// results 22.9 -> 24.4, 19.2 -> 19.5).
template <int FORM, typename X, typename H> static hipError_t launch_norm_form(const NormArgs &a, hipStream_t s) {
  auto run = [&](auto kernel, int threads, int rows_at_once, int per_cu) {
    const long long groups = ((long long)a.rows + rows_at_once - 1) / rows_at_once, resident = 256LL * per_cu;
    const int chunk = (int)((groups + resident - 1) / resident);
    return rc_launch(kernel, dim3((unsigned)((groups + chunk - 1) / chunk)), dim3(threads), 0, s, a, chunk);
  };
  auto whole = [&](auto kernel, int units, int waves_of_cu) {  // a workgroup a row
    const int waves = (a.cols + 512 * units - 1) / (512 * units);
    int per_cu = 8;
    while (per_cu > 1 && per_cu * waves > waves_of_cu) per_cu /= 2;
    return run(kernel, 64 * waves, 1, per_cu);
  };
  if constexpr (FORM == NF_TINY) {
    return run(norm_kernel<16, 1, FORM, X, H>, 256, 16, 4);
  } else {
    if (a.cols <= 128) return run(norm_kernel<16, 1, FORM, X, H>, 256, 16, 4);
    if (a.cols <= 512) return run(norm_kernel<64, 1, FORM, X, H>, 256, 4, 8);
    if (a.cols > 8192) return whole(norm_kernel<0, 2, FORM, X, H>, 2, 16);
    if (!kUpdate<H> && a.out_kind == NO_INT8 && (long long)a.rows * a.cols >= 1 << 21) return whole(norm_kernel<0, 2, FORM, X, H>, 2, 16);
    return whole(norm_kernel<0, 1, FORM, X, H>, 1, kUpdate<H> ? 16 : 24);  // (registers)
  }
}
template <typename X, typename H> static hipError_t launch_norm_types(const NormArgs &a, hipStream_t s) {
  return a.cols < 8 ? launch_norm_form<NF_TINY, X, H>(a, s) : a.vec ? launch_norm_form<NF_WHOLE, X, H>(a, s) : launch_norm_form<NF_ANY, X, H>(a, s);
}

hipError_t launch_norm(const NormArgs &args, hipStream_t s) {
  if (args.rows <= 0) return hipSuccess;
  if (args.cols > kNormMaxCols) return hipErrorInvalidValue;
  NormArgs a = args;
  auto has = [](const NormSpec &n, const float *factor, const float *shift) {
    return (n.weight ? NV_WEIGHT : 0) | (n.bias ? NV_BIAS : 0) | (factor ? NV_FACTOR : 0) | (shift ? NV_SHIFT : 0);
  };
  a.post_has = has(a.post, a.gate, nullptr);
  a.pre_has = has(a.pre, a.scale, a.shift);
  for (int k = a.chains; k <= kQArgChains; ++k) a.chain.arg[k] = a.rows;
  hipError_t e;
  if (!a.h) e = a.x_bf16 ? launch_norm_types<bf16, void>(a, s) : launch_norm_types<float, void>(a, s);
  else if (a.h_bf16) e = a.x_bf16 ? launch_norm_types<bf16, bf16>(a, s) : launch_norm_types<float, bf16>(a, s);
  else e = a.x_bf16 ? launch_norm_types<bf16, float>(a, s) : launch_norm_types<float, float>(a, s);
  return e != hipSuccess ? e : hipGetLastError();
}

__global__ __launch_bounds__(256) void modulation_kernel(ModulationArgs a) {
  const int i = (blockIdx.x * 256 + threadIdx.x) * 4, l = blockIdx.y;
  if (i < a.n) *(f32x4 *)(a.out + (size_t)l * a.n + i) = *(const f32x4 *)(a.sst[l] + i) + *(const f32x4 *)(a.t0 + i);
}

hipError_t launch_modulation(const ModulationArgs &a, int layers, hipStream_t s) {
  rc_launch(modulation_kernel, dim3((a.n / 4 + 255) / 256, layers), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace rc
