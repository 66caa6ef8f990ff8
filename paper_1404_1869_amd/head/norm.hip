// Root-mean-square norm of rows, with the residual's addition, and its gradient.
//   s = x + r;  q = 1 / sqrt(mean(s^2) + eps);  y = s q gamma
//   8-bit output: per block of a row (or per row) scale = max |y| / 448, codes e4m3(y / scale)
//   gradient: a = dy gamma;  dx = q (a - s q^2 mean(a s)) + dsum;  dgamma = sum over rows of dy s q
// All of it is computed in 32 bits from the unrounded sum s and rounded once, when a result is stored.
// Bound by memory: a row is read once, kept in registers over its reductions, and written once.
#include <hip/hip_runtime.h>

#include "head.h"

namespace dn {
namespace head {
namespace {

// Sum of K values per thread over the TPR threads of a row, in every one of them.  TPR = 64: a wave.  Else the
// waves' sums meet in LDS; `buf` alternates between calls, so that one barrier separates a call's reads from the
// next but one's writes.
template <int TPR, int K, bool MAX = false>
__device__ inline void row_reduce(float (&v)[K], float (*buf)[TPR / 64]) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = MAX ? lanes_max<64>(v[k]) : lanes_sum<64>(v[k]);
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) buf[k][wave] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float t = buf[k][0];
#pragma unroll
      for (int w = 1; w < TPR / 64; ++w) t = MAX ? fmaxf(t, buf[k][w]) : t + buf[k][w];
      v[k] = t;
    }
  }
}

// Threads of a workgroup: TPR per row, at least 256.
template <int TPR>
constexpr int threads() { return TPR < 256 ? 256 : TPR; }

// Thread t of a row holds elements 8 (k TPR + t) .. + 7, k < NV: 16-byte accesses of consecutive threads.
template <typename T, typename O, int TPR, int NV>
__global__ __launch_bounds__(threads<TPR>()) void rms_norm_kernel(NormArgs a) {
  constexpr int ROWS = threads<TPR>() / TPR;
  __shared__ float s_buf[2][1][TPR / 64];
  const int t = threadIdx.x % TPR, C = a.C;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  if (row >= a.n) return;  // whole waves, and only where TPR = 64 (no barriers)
  const T* x = (const T*)a.x + row * a.x_stride;
  const T* res = (const T*)a.res + row * a.res_stride;
  float v[NV][8], r[NV][8], w[NV][8];
#pragma unroll
  for (int k = 0; k < NV; ++k) load8(x, 8 * (k * TPR + t), C, v[k]);
  if (a.res)
#pragma unroll
    for (int k = 0; k < NV; ++k) load8(res, 8 * (k * TPR + t), C, r[k]);
  if (a.gamma)
#pragma unroll
    for (int k = 0; k < NV; ++k) load8(a.gamma, 8 * (k * TPR + t), C, w[k]);
  if (a.res)
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[k][j] += r[k][j];
  if (a.sum)
#pragma unroll
    for (int k = 0; k < NV; ++k)
      store8((T*)a.sum + row * a.sum_stride, 8 * (k * TPR + t), C, v[k]);
  float ss[1] = {0.f};
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) ss[0] += v[k][j] * v[k][j];
  row_reduce<TPR>(ss, s_buf[0]);
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
      row_reduce<TPR, 1, true>(m, s_buf[1]);
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

// Gradient: a workgroup takes rows blockIdx.x, blockIdx.x + gridDim.x, ... (groups of ROWS rows), keeps its sums of
// dy s q per column in registers over them, and writes them as one row of part (ROWS rows of it where TPR = 64).
template <typename T, typename D, int TPR, int NV>
__global__ __launch_bounds__(threads<TPR>()) void rms_norm_back_kernel(NormBackArgs a) {
  constexpr int ROWS = threads<TPR>() / TPR;
  __shared__ float s_buf[2][2][TPR / 64];
  const int t = threadIdx.x % TPR, C = a.C, sub = threadIdx.x / TPR;
  float dg[NV][8], w[NV][8];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[k][j] = 0.f, w[k][j] = 1.f;
    if (a.gamma) load8(a.gamma, 8 * (k * TPR + t), C, w[k]);
  }
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + sub; row < a.n; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
    const T* s = (const T*)a.s + row * a.s_stride;
    const D* dy = (const D*)a.dy + row * a.dy_stride;
    float v[NV][8], d[NV][8], e[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      load8(s, 8 * (k * TPR + t), C, v[k]);
      load8(dy, 8 * (k * TPR + t), C, d[k]);
      if (a.dsum) load8((const T*)a.dsum + row * a.dsum_stride, 8 * (k * TPR + t), C, e[k]);
    }
    float z[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        z[0] += v[k][j] * v[k][j];
        z[1] += d[k][j] * w[k][j] * v[k][j];
      }
    row_reduce<TPR>(z, s_buf[turn]);
    const float q = 1.f / sqrtf(z[0] / (float)C + a.eps), f = q * q * (z[1] / (float)C);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dg[k][j] += d[k][j] * (v[k][j] * q);
        const float g = q * (d[k][j] * w[k][j] - v[k][j] * f);
        v[k][j] = a.dsum ? g + e[k][j] : g;
      }
      store8((T*)a.dx + row * a.dx_stride, 8 * (k * TPR + t), C, v[k]);
    }
  }
  if (a.dgamma)
#pragma unroll
    for (int k = 0; k < NV; ++k)
      store8(a.part + ((int64_t)blockIdx.x * ROWS + sub) * C, 8 * (k * TPR + t), C, dg[k]);
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

// The fewest threads and registers that hold a row: f(integral_constant TPR, integral_constant NV).
template <int TPR, int NV>
struct Shape {
  static constexpr int tpr = TPR, nv = NV;
};
template <typename F>
int with_shape(int C, F&& f) {
  if (C <= 512) return f(Shape<64, 1>{});
  if (C <= 1024) return f(Shape<64, 2>{});
  if (C <= 2048) return f(Shape<256, 1>{});
  if (C <= 4096) return f(Shape<256, 2>{});
  if (C <= 8192) return f(Shape<512, 2>{});
  if (C <= 12288) return f(Shape<512, 3>{});
  if (C <= 16384) return f(Shape<1024, 2>{});
  return f(Shape<1024, 4>{});
}
template <typename F>
int with_type(dn_dtype dt, F&& f) {
  if (dt == DN_F32) return f(float{});
  if (dt == DN_F16) return f(_Float16{});
  return f(__bf16{});
}

}  // namespace

int launch_rms_norm(const NormArgs& a, dn_dtype dt, dn_dtype y_dt, void* stream) {
  return with_shape(a.C, [&](auto shape) {
    constexpr int TPR = decltype(shape)::tpr, NV = decltype(shape)::nv, ROWS = threads<TPR>() / TPR;
    return with_type(dt, [&](auto x) {
      using T = decltype(x);
      const dim3 grid((unsigned)((a.n + ROWS - 1) / ROWS));
      if (y_dt == DN_F8)
        rms_norm_kernel<T, F8, TPR, NV><<<grid, threads<TPR>(), 0, (hipStream_t)stream>>>(a);
      else
        with_type(y_dt, [&](auto y) {
          rms_norm_kernel<T, decltype(y), TPR, NV><<<grid, threads<TPR>(), 0, (hipStream_t)stream>>>(a);
          return 0;
        });
      return (int)hipGetLastError();
    });
  });
}

// Rows of part: one per workgroup (or wave) of the gradient's launch.
int32_t norm_back_groups(int64_t n, int32_t C) {
  const int64_t rows = C <= 1024 ? 4 : 1, most = 1024;
  return (int32_t)(std::min((n + rows - 1) / rows, most) * rows);
}

int launch_rms_norm_backward(const NormBackArgs& a, dn_dtype dt, dn_dtype dy_dt, void* stream) {
  const int err = a.n == 0 ? 0 : with_shape(a.C, [&](auto shape) {
    constexpr int TPR = decltype(shape)::tpr, NV = decltype(shape)::nv, ROWS = threads<TPR>() / TPR;
    return with_type(dt, [&](auto x) {
      return with_type(dy_dt, [&](auto d) {
        rms_norm_back_kernel<decltype(x), decltype(d), TPR, NV>
            <<<dim3((unsigned)(a.groups / ROWS)), threads<TPR>(), 0, (hipStream_t)stream>>>(a);
        return (int)hipGetLastError();
      });
    });
  });
  if (err || !a.dgamma) return err;
  column_sum_kernel<<<dim3((unsigned)((a.C + 31) / 32)), 256, 0, (hipStream_t)stream>>>(a.part, a.dgamma, a.groups, a.C);
  return (int)hipGetLastError();
}

}  // namespace head
}  // namespace dn
