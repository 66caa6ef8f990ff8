// One AdamW step over many tensors at once, states in 32 or in 8 bits.
//   g' = g grad_scale;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2
//   p = p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v) / sqrt(1 - b2^t) + eps)
// computed in 32 bits; the 16-bit copy is the new p, rounded.
// 8-bit states: blocks of 256 values hold m and r = sqrt(v) as e4m3 codes of m 448 / max |m| and r 448 / max r, with
// max / 448 as the block's scale.  r rather than v: the codes' range of 2^18 is then one of 2^36 in v.  A code is the
// e4m3 value below or above, above with the chance of its place between the two, so that a step's small part
// (1 - b2 = 0.001 of v, where neighbouring codes are 6 to 12 % apart) is kept on average: to nearest it would be lost
// every time.  The chance comes from a multiplicative hash of the value's place and the seed, 16 bits for m and 16 for r: shifts
// and multipliers of low bias that C. Wellons published ("Prospecting for Hash Functions", 2018).  An r above 0 is never
// stored as 0 (it divides).  The step itself uses the unrounded m and r.
// Bound by memory: every value is read and written once, eight of them a thread.  64 M fp32 values with bf16 gradients and
// copies in 160 tensors: 342 to 352 us with 32-bit states (28 bytes a value, 5.2 TB/s), 212 us with 8-bit ones (16 bytes, 4.8 TB/s),
// against 5.08 TB/s of a large copy.
#include <hip/hip_runtime.h>

#include "head.h"

namespace dn {
namespace head {
namespace {

__device__ inline uint32_t noise(uint32_t i, uint32_t seed) {
  uint32_t x = i * 0x9E3779B1u + seed;
  x = (x ^ (x >> 15)) * 0x2C1B3C6Du;
  x = (x ^ (x >> 12)) * 0x297A2D39u;
  return x ^ (x >> 15);
}

// a in [0, 448] to the e4m3 value below or above.  From 2^-6 on e4m3 keeps 3 of the 23 mantissa bits: the chance is
// added below them and the rest cut off.  Below, its values are the multiples of 2^-9.  NaN stays NaN.
__device__ inline float round8(float a, uint32_t chance) {
  const float small = floorf(a * 512.f + (float)chance * (1.f / 65536.f)) * (1.f / 512.f);
  const float large = __uint_as_float((__float_as_uint(a) + (chance << 4)) & ~0xFFFFFu);
  return a != a ? a : a < 0.015625f ? small : large;
}

__device__ inline void f8_unpack(const uint32_t (&w)[2], float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
    v[4 * k] = lo[0], v[4 * k + 1] = lo[1], v[4 * k + 2] = hi[0], v[4 * k + 3] = hi[1];
  }
}

// A block's 256 values lie in 32 consecutive lanes, eight each.  States are padded to whole blocks per tensor, so
// their accesses are whole and aligned.
template <typename P, typename G, bool BITS8, typename Q>
__global__ __launch_bounds__(256) void adamw_kernel(AdamWArgs a) {
#pragma clang fp contract(off)
  int lo = 0, hi = a.count - 1;  // the tensor of this workgroup: the last whose first is at most blockIdx.x
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.t[mid].first <= (int64_t)blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const AdamWTensor& t = a.t[lo];
  const int64_t base = ((int64_t)blockIdx.x - t.first) * ADAMW_TILE, at = base + threadIdx.x * 8;
  const int left = (int)std::min<int64_t>(t.n - base, ADAMW_TILE);  // values of the tensor in this tile
  const int i = threadIdx.x * 8;
  if ((i & ~(ADAMW_BLOCK - 1)) >= left) return;  // whole blocks past the end
  P* p_at = (P*)t.p + base;
  const int64_t st = t.state + at;
  float g[8], p[8], m[8], r[8];
  load8((const G*)t.g + base, i, left, g);
  load8((const P*)p_at, i, left, p);
  if constexpr (BITS8) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 mw = *(const u32x2*)((const uint8_t*)a.m + st), vw = *(const u32x2*)((const uint8_t*)a.v + st);
    const float ms = a.m_scale[st / ADAMW_BLOCK], vs = a.v_scale[st / ADAMW_BLOCK];
    const uint32_t mq[2] = {mw[0], mw[1]}, vq[2] = {vw[0], vw[1]};
    f8_unpack(mq, m);
    f8_unpack(vq, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) m[j] *= ms, r[j] *= vs;
  } else {
    load8((const float*)a.m + st, m);
    load8((const float*)a.v + st, r);
  }
  if (i + 8 > left)  // what lies past the tensor's end in its last block counts as 0
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j >= left) m[j] = r[j] = 0.f;
  float m_top = 0.f, r_top = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float gj = g[j] * a.grad_scale;
    m[j] = a.beta1 * m[j] + a.one_beta1 * gj;
    const float v = a.beta2 * (BITS8 ? r[j] * r[j] : r[j]) + a.one_beta2 * (gj * gj);
    const float root = sqrtf(v);
    r[j] = BITS8 ? root : v;
    p[j] = p[j] * a.decay - a.rate * m[j] / (root * a.root + a.eps);
    if constexpr (BITS8) {  // an infinity is stored as NaN, and counts for no scale: it would take its whole block along
      m[j] = fabsf(m[j]) < INFINITY ? m[j] : NAN;
      r[j] = r[j] < INFINITY ? r[j] : NAN;
      m_top = fmaxf(m_top, fabsf(m[j]));
      r_top = fmaxf(r_top, r[j]);
    }
  }
  store8(p_at, i, left, p);
  if (t.copy) store8((Q*)t.copy + base, i, left, p);
  if constexpr (BITS8) {
    m_top = lanes_max<32>(m_top);
    r_top = lanes_max<32>(r_top);
    // 448 / top of a block of zeros, or of values below 1e-36 (whose reciprocal is past fp32's range), is taken as 0
    const float mi = m_top > 1.4e-36f ? 1.f / m_top * 448.f : 0.f, ri = r_top > 1.4e-36f ? 1.f / r_top * 448.f : 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t h = noise((uint32_t)(st + j), a.seed);
      float am = fabsf(m[j]) * mi, ar = r[j] * ri;
      am = am > 448.f ? 448.f : am, ar = ar > 448.f ? 448.f : ar;
      const float q = round8(ar, h & 0xFFFFu);
      r[j] = r[j] > 0.f && q < 0.001953125f ? 0.001953125f : q;
      m[j] = __builtin_copysignf(round8(am, h >> 16), m[j]);
    }
    uint32_t w[2];
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    f8_pack(m, w);
    *(u32x2*)((uint8_t*)a.m + st) = u32x2{w[0], w[1]};
    f8_pack(r, w);
    *(u32x2*)((uint8_t*)a.v + st) = u32x2{w[0], w[1]};
    if ((threadIdx.x & 31) == 0) {
      a.m_scale[st / ADAMW_BLOCK] = m_top * (1.f / 448.f);
      a.v_scale[st / ADAMW_BLOCK] = r_top * (1.f / 448.f);
    }
  } else {
    store8((float*)a.m + st, m);
    store8((float*)a.v + st, r);
  }
}

template <typename F>
int with_type(dn_dtype dt, F&& f) {
  if (dt == DN_F32) return f(float{});
  if (dt == DN_F16) return f(_Float16{});
  return f(__bf16{});
}

}  // namespace

int launch_adamw(const AdamWArgs& a, int64_t groups, dn_dtype p_dt, dn_dtype g_dt, dn_dtype copy_dt, int bits,
                 void* stream) {
  return with_type(p_dt, [&](auto p) {
    return with_type(g_dt, [&](auto g) {
      using P = decltype(p);
      using G = decltype(g);
      const dim3 grid((unsigned)groups);
      const hipStream_t st = (hipStream_t)stream;
      if (copy_dt == DN_F16) {
        if (bits == 8) adamw_kernel<P, G, true, _Float16><<<grid, 256, 0, st>>>(a);
        else adamw_kernel<P, G, false, _Float16><<<grid, 256, 0, st>>>(a);
      } else {
        if (bits == 8) adamw_kernel<P, G, true, __bf16><<<grid, 256, 0, st>>>(a);
        else adamw_kernel<P, G, false, __bf16><<<grid, 256, 0, st>>>(a);
      }
      return (int)hipGetLastError();
    });
  });
}

}  // namespace head
}  // namespace dn
