// Root-mean-square norm of rows, with the residual's addition, and its gradient.
//   s = x + r;  q = 1 / sqrt(mean(s^2) + eps);  y = s q gamma
//   8-bit output: per block of a row (or per row) scale = max |y| / 448, codes e4m3(y / scale)
//   gradient: a = dy gamma;  dx = q (a - s q^2 mean(a s)) + dsum;  dgamma = sum over rows of dy s q
// All of it is computed in 32 bits from the unrounded sum s and rounded once, when a result is stored.
// Bound by memory: a row is read once, kept in registers over its reductions, and written once; the gradient sums dgamma in
// registers over a workgroup's rows and then over the workgroups in a fixed order.  A large copy moves 5.08 TB/s on this card;
// measured: 2000 rows of 9216 fp32 values to 8 bits 18.4 us (5.0 TB/s; a scale for every 32, 64 or 128 values: the same), 8191
// unaligned rows of 2047 fp16 values with residual 28.1 us (4.8), the gradient of 32000 rows of 4096 bf16 values with dsum 207 us
// (5.1).
#include <hip/hip_runtime.h>

#include "head.h"

namespace dn {
namespace head {
namespace {

// Sum (or maximum) of K values per thread over the threads of a row, in every one of them: a wave (WAVE), or the whole
// workgroup, whose waves' sums meet in LDS.  `buf` alternates between calls, so that one barrier separates a call's reads
// from the next but one's writes.
constexpr int MAX_WAVES = 16;
template <bool WAVE, int K, bool MAX = false>
__device__ inline void row_reduce(float (&v)[K], float (*buf)[MAX_WAVES]) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = MAX ? lanes_max<64>(v[k]) : lanes_sum<64>(v[k]);
  if constexpr (!WAVE) {
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) buf[k][wave] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float t = buf[k][0];
      for (int w = 1; w < waves; ++w) t = MAX ? fmaxf(t, buf[k][w]) : t + buf[k][w];
      v[k] = t;
    }
  }
}

// Eight values of a row as they are stored, 0 past its end.
template <typename T>
using Raw = typename Vec8<T>::type;
template <typename T>
__device__ inline Raw<T> load_raw(const T* row, int i, int C) {
  if (i + 8 <= C) return *(const Raw<T>*)(row + i);
  Raw<T> r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = i + j < C ? row[i + j] : (T)0.f;
  return r;
}

// Thread t of a row's TPR threads holds elements 8 (k TPR + t) .. + 7, k < NV: 16-byte accesses of consecutive threads.
// WAVE: a wave per row, four rows per workgroup, no barriers; else the workgroup.
// THREADS: the most threads of a workgroup of this shape.
template <typename T, typename O, bool WAVE, int NV, int THREADS>
__global__ __launch_bounds__(THREADS) void rms_norm_kernel(NormArgs a) {
  __shared__ float s_buf[2][1][MAX_WAVES];
  const int TPR = WAVE ? 64 : blockDim.x, t = WAVE ? threadIdx.x & 63 : threadIdx.x, C = a.C;
  const int64_t row = WAVE ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (row >= a.n) return;  // whole waves, and only where WAVE (no barriers)
  const T* x = (const T*)a.x + row * a.x_stride;
  const T* res = (const T*)a.res + row * a.res_stride;
  Raw<T> xr[NV], rr[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) xr[k] = load_raw(x, 8 * (k * TPR + t), C);
  if (a.res)
#pragma unroll
    for (int k = 0; k < NV; ++k) rr[k] = load_raw(res, 8 * (k * TPR + t), C);
  float v[NV][8], w[NV][8];
  if (a.gamma)
#pragma unroll
    for (int k = 0; k < NV; ++k) load8(a.gamma, 8 * (k * TPR + t), C, w[k]);
  float ss[1] = {0.f};
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[k][j] = a.res ? (float)xr[k][j] + (float)rr[k][j] : (float)xr[k][j];
      ss[0] += v[k][j] * v[k][j];
    }
  if (a.sum)
#pragma unroll
    for (int k = 0; k < NV; ++k)
      store8((T*)a.sum + row * a.sum_stride, 8 * (k * TPR + t), C, v[k]);
  row_reduce<WAVE>(ss, s_buf[0]);
  const float q = 1.f / sqrtf(ss[0] / (float)C + a.eps);
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[k][j] = v[k][j] * q * (a.gamma ? w[k][j] : 1.f);
  O* y = (O*)a.y + row * a.y_stride;
  if constexpr (std::is_same<O, F8>::value) {
    float top[NV];  // of the block that the thread's k-th eight values lie in
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      top[k] = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) top[k] = fmaxf(top[k], fabsf(v[k][j]));
    }
    if (a.block == 0) {
      float m[1] = {top[0]};
#pragma unroll
      for (int k = 1; k < NV; ++k) m[0] = fmaxf(m[0], top[k]);
      row_reduce<WAVE, 1, true>(m, s_buf[1]);
#pragma unroll
      for (int k = 0; k < NV; ++k) top[k] = m[0];
      if (t == 0) a.scale[row] = m[0] * (1.f / 448.f);
    } else {
      const int lanes = a.block / 8, blocks = (C + a.block - 1) / a.block;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        for (int d = 1; d < lanes; d *= 2) top[k] = fmaxf(top[k], __shfl_xor(top[k], d));
        const int b = (k * TPR + t) / lanes;
        if (t % lanes == 0 && b < blocks) a.scale[row * blocks + b] = top[k] * (1.f / 448.f);
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      // 448 / top of a block of zeros, or of values below 1e-36 (whose reciprocal is past fp32's range), is taken as
      // 0.  The largest value becomes 448 within a rounding, which e4m3 rounds to 448; a NaN stays one.
      const float inv = top[k] > 1.4e-36f ? 448.f / top[k] : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[k][j] *= inv;
    }
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) store8(y, 8 * (k * TPR + t), C, v[k]);
}

// Gradient: a workgroup (WAVE: each of its waves) takes rows at a fixed distance, loads a row while it works on the one
// before (AHEAD), keeps its sums of dy s q per column in registers over them, and writes them as one row of part.
// THREADS: the most threads of a workgroup of this shape, which bounds its registers.
template <typename T, typename D, bool WAVE, int NV, int THREADS, bool AHEAD>
__global__ __launch_bounds__(THREADS) void rms_norm_back_kernel(NormBackArgs a) {
  constexpr bool HOLD = NV < 4;  // gamma stays in registers
  __shared__ float s_buf[2][2][MAX_WAVES];
  const int TPR = WAVE ? 64 : blockDim.x, t = WAVE ? threadIdx.x & 63 : threadIdx.x, C = a.C;
  const int64_t first = WAVE ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  const int64_t step = a.groups;
  float dg[NV][8], held[HOLD ? NV : 1][8];
  auto gamma = [&](int k, float (&w)[8]) {
    if (a.gamma) {
      load8(a.gamma, 8 * (k * TPR + t), C, w);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = 1.f;
    }
  };
#pragma unroll
  for (int k = 0; k < NV; ++k) {
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[k][j] = 0.f;
    if constexpr (HOLD) gamma(k, held[k]);
  }
  struct Row {
    Raw<T> s[NV], e[NV];
    Raw<D> d[NV];
  };
  auto load = [&](int64_t row, Row& r) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = 8 * (k * TPR + t);
      r.s[k] = load_raw((const T*)a.s + row * a.s_stride, i, C);
      r.d[k] = load_raw((const D*)a.dy + row * a.dy_stride, i, C);
      if (a.dsum) r.e[k] = load_raw((const T*)a.dsum + row * a.dsum_stride, i, C);
    }
  };
  Row next;
  if (AHEAD && first < a.n) load(first, next);
  int turn = 0;
  for (int64_t row = first; row < a.n; row += step, turn ^= 1) {
    Row r;
    if constexpr (AHEAD) r = next;
    else load(row, r);
    float z[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float w[8];
      if constexpr (!HOLD) gamma(k, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = (float)r.s[k][j];
        z[0] += v * v;
        z[1] += (float)r.d[k][j] * (HOLD ? held[HOLD ? k : 0][j] : w[j]) * v;
      }
    }
    if (AHEAD && row + step < a.n) load(row + step, next);
    row_reduce<WAVE>(z, s_buf[turn]);
    const float q = 1.f / sqrtf(z[0] / (float)C + a.eps), f = q * q * (z[1] / (float)C);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float w[8], x[8];
      if constexpr (!HOLD) gamma(k, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = (float)r.s[k][j], g = (float)r.d[k][j];
        dg[k][j] += g * (v * q);
        x[j] = q * (g * (HOLD ? held[HOLD ? k : 0][j] : w[j]) - v * f);
        if (a.dsum) x[j] += (float)r.e[k][j];
      }
      store8((T*)a.dx + row * a.dx_stride, 8 * (k * TPR + t), C, x);
    }
  }
  if (a.dgamma)
#pragma unroll
    for (int k = 0; k < NV; ++k) store8(a.part + first * C, 8 * (k * TPR + t), C, dg[k]);
}

// Sums of the columns of part ([rows][C]), always in the same order: 32 columns per workgroup, 8 rows at a time.
__global__ __launch_bounds__(256) void column_sum_kernel(const float* __restrict__ part, float* __restrict__ out, int rows,
                                                         int C) {
  __shared__ float s_sum[8][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), r0 = threadIdx.x >> 5;
  float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
  if (c < C) {
    int r = r0;
    for (; r + 24 < rows; r += 32) {
      s0 += part[(int64_t)r * C + c];
      s1 += part[(int64_t)(r + 8) * C + c];
      s2 += part[(int64_t)(r + 16) * C + c];
      s3 += part[(int64_t)(r + 24) * C + c];
    }
    for (; r < rows; r += 8) s0 += part[(int64_t)r * C + c];
  }
  s_sum[r0][threadIdx.x & 31] = (s0 + s1) + (s2 + s3);
  __syncthreads();
  if (r0 == 0 && c < C) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += s_sum[i][threadIdx.x & 31];
    out[c] = s;
  }
}

// The most threads of a workgroup whose threads hold NV times eight values of rows of up to C.
template <bool WAVE_, int NV_, int C>
struct Shape {
  static constexpr bool wave = WAVE_;
  static constexpr int nv = NV_, most = WAVE_ ? 256 : C / (8 * NV_);
  // whole waves that hold a row of C_ values
  static int threads(int C_) { return WAVE_ ? 256 : (C_ + 512 * NV_ - 1) / (512 * NV_) * 64; }
};
template <typename F>
int with_type(dn_dtype dt, F&& f) {
  if (dt == DN_F32) return f(float{});
  if (dt == DN_F16) return f(_Float16{});
  return f(__bf16{});
}

}  // namespace

// A wave per row where its lanes can hold it in up to four times eight values each, else a workgroup (8191 unaligned rows of
// 2047 fp16 values: 27 us, a workgroup per row 35).  More rows than a launch can have threads for (2^26 by waves) go in several.
int launch_rms_norm(const NormArgs& a, dn_dtype dt, dn_dtype y_dt, void* stream) {
  const auto with = [&](auto shape) {
    using S = decltype(shape);
    return with_type(dt, [&](auto x) {
      using T = decltype(x);
      const int threads = S::threads(a.C);
      const int64_t per = S::wave ? 4 : 1, most = MAX_LAUNCH_THREADS / threads * per;  // rows of a workgroup, of a launch
      const int64_t y_size = y_dt == DN_F8 ? 1 : (int64_t)dtype_size(y_dt);
      const int64_t scales = a.block ? (a.C + a.block - 1) / a.block : 1;
      for (int64_t at = 0; at < a.n; at += most) {
        NormArgs b = a;
        b.n = std::min(a.n - at, most);
        b.x = (const T*)a.x + at * a.x_stride;
        if (a.res) b.res = (const T*)a.res + at * a.res_stride;
        if (a.sum) b.sum = (T*)a.sum + at * a.sum_stride;
        b.y = (char*)a.y + at * a.y_stride * y_size;
        if (a.scale) b.scale = a.scale + at * scales;
        const dim3 grid((unsigned)((b.n + per - 1) / per));
        if (y_dt == DN_F8)
          rms_norm_kernel<T, F8, S::wave, S::nv, S::most><<<grid, threads, 0, (hipStream_t)stream>>>(b);
        else
          with_type(y_dt, [&](auto y) {
            rms_norm_kernel<T, decltype(y), S::wave, S::nv, S::most><<<grid, threads, 0, (hipStream_t)stream>>>(b);
            return 0;
          });
        if (const int err = (int)hipGetLastError()) return err;
      }
      return 0;
    });
  };
  if (a.C <= 512) return with(Shape<true, 1, 512>{});
  if (a.C <= 1024) return with(Shape<true, 2, 1024>{});
  if (a.C <= 2048) return with(Shape<true, 4, 2048>{});
  if (a.C <= 8192) return with(Shape<false, 2, 8192>{});
  if (a.C <= 16384) return with(Shape<false, 2, 16384>{});
  return with(Shape<false, 4, DN_MAX_NORM_C>{});
}

// Rows of part: one per workgroup (or wave) of the gradient's launch.  More workgroups cover each other's waits, and each
// costs a row of part: 2 to 4 per CU (of 512, 768, 1024 and 2048 workgroups, 32000 rows of 4096 took 217, 211, 211 and 234 us).
int32_t norm_back_groups(int64_t n, int32_t C) {
  const int64_t rows = C <= 1024 ? 4 : 1, most = C <= 1024 || C > 4096 ? 512 : 768;
  return (int32_t)(std::min((n + rows - 1) / rows, most) * rows);
}

int launch_rms_norm_backward(const NormBackArgs& a, dn_dtype dt, dn_dtype dy_dt, void* stream) {
  const auto with = [&](auto shape) {
    using S = decltype(shape);
    return with_type(dt, [&](auto x) {
      return with_type(dy_dt, [&](auto d) {
        using T = decltype(x);
        using D = decltype(d);
        // a second row in registers where they suffice: fp32 rows of over 12288 values, and rows of over 16384, would spill (6000
        // rows of 9216 fp32 values took 118 us, and 197 when compiled for half the registers)
        constexpr bool AHEAD = S::nv < 4 && (S::most <= 768 || sizeof(T) == 2);
        rms_norm_back_kernel<T, D, S::wave, S::nv, S::most, AHEAD>
            <<<dim3((unsigned)(a.groups / (S::wave ? 4 : 1))), S::threads(a.C), 0, (hipStream_t)stream>>>(a);
        return (int)hipGetLastError();
      });
    });
  };
  int err = 0;
  if (a.n == 0) err = 0;
  else if (a.C <= 512) err = with(Shape<true, 1, 512>{});
  else if (a.C <= 1024) err = with(Shape<true, 2, 1024>{});
  else if (a.C <= 2048) err = with(Shape<false, 1, 2048>{});
  else if (a.C <= 8192) err = with(Shape<false, 2, 8192>{});
  else if (a.C <= 12288) err = with(Shape<false, 2, 12288>{});
  else if (a.C <= 16384) err = with(Shape<false, 2, 16384>{});
  else err = with(Shape<false, 4, DN_MAX_NORM_C>{});
  if (err || !a.dgamma) return err;
  column_sum_kernel<<<dim3((unsigned)((a.C + 31) / 32)), 256, 0, (hipStream_t)stream>>>(a.part, a.dgamma, a.groups, a.C);
  return (int)hipGetLastError();
}

}  // namespace head
}  // namespace dn
