// Internal declarations of the head's operators (norm, loss, optimiser): the launchers, and the device helpers they
// share.  Conventions (errors, streams, ownership) are the library's: see densenet.h.
#pragma once

#include "common.h"

namespace dn {
namespace head {

// HIP counts a launch's threads in 32 bits: of 2^32 and more it runs fewer workgroups than were asked for, and says nothing.
constexpr int64_t MAX_LAUNCH_THREADS = (1LL << 32) - 1;

// ---------------------------------------------------------------------------------------------
// Launchers.  Every launcher enqueues on `stream` and returns hipGetLastError() as an int (0 = success).
// ---------------------------------------------------------------------------------------------
struct NormArgs {  // strides in elements of the operand's own type
  const void *x, *res;
  const float* gamma;
  void *sum, *y;
  float* scale;
  int64_t x_stride, res_stride, sum_stride, y_stride;
  int64_t n;
  int32_t C, block;
  float eps;
};
int launch_rms_norm(const NormArgs& a, dn_dtype dt, dn_dtype y_dt, void* stream);

struct NormBackArgs {
  const void *dy, *s, *dsum;
  const float* gamma;
  void* dx;
  float *dgamma, *part;
  int64_t dy_stride, s_stride, dsum_stride, dx_stride;
  int64_t n;
  int32_t C, groups;  // groups: workgroups, one row of part each
  float eps;
};
int32_t norm_back_groups(int64_t n, int32_t C);
int launch_rms_norm_backward(const NormBackArgs& a, dn_dtype dt, dn_dtype dy_dt, void* stream);

// Tensors of one AdamW launch, passed by value.
constexpr int ADAMW_TENSORS = 72;
constexpr int ADAMW_BLOCK = 256;   // values that share a scale in 8-bit states
constexpr int ADAMW_TILE = 2048;   // values of one workgroup
struct AdamWTensor {
  void* p;
  const void* g;
  void* copy;
  int64_t n, state;  // values; first value in the states
  int64_t first;     // first workgroup of the tensor in its launch
};
struct AdamWArgs {
  AdamWTensor t[ADAMW_TENSORS];
  int32_t count;
  uint32_t seed;
  void *m, *v;
  float *m_scale, *v_scale;
  float beta1, beta2, one_beta1, one_beta2, rate, root, eps, decay, grad_scale;
};
int launch_adamw(const AdamWArgs& a, int64_t groups, dn_dtype p_dt, dn_dtype g_dt, dn_dtype copy_dt, int bits,
                 void* stream);

// Softmax loss of rows h [n][C] over the products with w [V][C].  Strides in elements.
struct LossArgs {
  const void *h, *w;
  const int64_t* label;
  int64_t h_stride, w_stride;
  int64_t n;
  int32_t C, V;
  float *loss, *lse;  // the forward pass's results
  // gradient: lse is read
  const float *lse_in, *dloss;
  void *dh, *dw;
  int64_t dh_stride, dw_stride;
  float scale;
};
size_t softmax_loss_bytes(const LossArgs& a, dn_dtype dt);
int launch_softmax_loss(const LossArgs& a, dn_dtype dt, void* d_work, void* stream);
size_t softmax_loss_backward_bytes(const LossArgs& a, dn_dtype dt);
int launch_softmax_loss_backward(const LossArgs& a, dn_dtype dt, void* d_work, void* stream);

}  // namespace head
}  // namespace dn

#if defined(__HIPCC__)
namespace dn {
namespace head {

struct F8 {  // e4m3 (OCP), a storage type
  uint8_t bits;
};

// Eight values of a type at any address that its elements may have: one or two 16-byte accesses (the hardware takes
// them at the alignment of one element).
template <typename T>
struct Vec8 {
  typedef T type __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};
template <typename T>
__device__ inline void load8(const T* p, float (&v)[8]) {
  const typename Vec8<T>::type t = *(const typename Vec8<T>::type*)p;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)t[j];
}
template <typename T>
__device__ inline void store8(T* p, const float (&v)[8]) {
  typename Vec8<T>::type t;
#pragma unroll
  for (int j = 0; j < 8; ++j) t[j] = (T)v[j];
  *(typename Vec8<T>::type*)p = t;
}
// Eight values of a row from element i on, 0 past its C elements.
template <typename T>
__device__ inline void load8(const T* row, int i, int C, float (&v)[8]) {
  if (i + 8 <= C) {
    load8(row + i, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = i + j < C ? (float)row[i + j] : 0.f;
  }
}
template <typename T>
__device__ inline void store8(T* row, int i, int C, const float (&v)[8]) {
  if (i + 8 <= C) {
    store8(row + i, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j < C) row[i + j] = (T)v[j];
  }
}
// Two values as e4m3 in the low (HI = false) or high half of `old`, rounded to nearest even.
template <bool HI>
__device__ inline uint32_t f8_pair(float a, float b, uint32_t old) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, HI);
}
__device__ inline void f8_pack(const float (&v)[8], uint32_t (&w)[2]) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
    w[k] = f8_pair<true>(v[4 * k + 2], v[4 * k + 3], f8_pair<false>(v[4 * k], v[4 * k + 1], 0));
}
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
__device__ inline void store8(F8* row, int i, int C, const float (&v)[8]) {
  uint32_t w[2];
  f8_pack(v, w);
  if (i + 8 <= C) {
    *(u32x2_any*)(row + i) = u32x2_any{w[0], w[1]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j < C) row[i + j].bits = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
  }
}

// Sum (or maximum) over the W consecutive lanes that a lane is among, in every one of them.
template <int W>
__device__ inline float lanes_sum(float v) {
#pragma unroll
  for (int d = 1; d < W; d *= 2) v += __shfl_xor(v, d);
  return v;
}
template <int W>
__device__ inline float lanes_max(float v) {
#pragma unroll
  for (int d = 1; d < W; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

}  // namespace head
}  // namespace dn
#endif
