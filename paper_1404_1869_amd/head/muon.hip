// Muon: a matrix's momentum, orthogonalised by Newton-Schulz steps, as its update.
//   m = beta m + g';  u = g' + beta m (nesterov) or m;  X = u / (|u| + eps)
//   per step: A = X X',  P = b A + c A^2,  X = a X + P X   (of a tall X: A = X' X,  X = a X + X P)
//   p = p (1 - lr weight_decay) - lr rate X
// A, P and A^2 have the smaller side r of the matrix, and are symmetric: half their tiles are computed and mirrored.  A step is
// 3 r^2 c + r^3 operations (c: the larger side), on the matrix cores, in one or two fp16 parts of every value:
//   X, A are held times 2^13, P times a power of two that its coefficients allow, all of them below fp16's largest (the singular
//   values of X are at most about 1.2 with the usual coefficients).  One part is 11 bits of a value down to 2^-27: the steps'
//   roundings are of either sign and come to about 2^-11 of the update in all, below half a unit of a bf16 weight.  Two parts
//   (fp32 and fp16 weights) are 22 bits, in three products of parts, as the loss's logits in fp32.
// All matrices of a call go through the same launches.  Sums over k go to slabs in fp32, one for each split, and a launch adds
// them in order, so results do not depend on what ran first.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "tiles.h"

namespace dn {
namespace head {
namespace {

constexpr int XS = 13;  // X and A are held times 2^XS
constexpr int T = 128;  // a tile's sides
constexpr int SUMS = 1024;  // partial sums of a matrix's norm

// A matrix in a launch, passed by value.
struct Mat {
  const void* g;
  float* m;
  void *p, *copy;
  int64_t x[2], a, poly, slab;  // offsets in the workspace: X (two buffers), A, P, slabs (fp32)
  int32_t rows, cols, first, splits;  // first: workgroup (or unit) of the launch that the matrix starts at
  int32_t sums;                       // partial sums of its norm, from norm on
  int32_t norm;
  float rate;
};
constexpr int MATS = 32;  // 96 bytes each
struct MuonLaunch {
  Mat t[MATS];
  int32_t count;
  char* work;
  float* sums;
  float beta, grad_scale, eps, lr, decay;
  float a, b, c;  // of the step
  int32_t poly_shift;  // P is held times 2^poly_shift
  int32_t nesterov, from;  // from: the buffer that X is in
};

__host__ __device__ inline int32_t up8(int32_t x) { return (x + 7) / 8 * 8; }
__device__ inline const Mat& mat_of(const MuonLaunch& l, int block) {
  int k = 0;
  for (int i = 1; i < l.count; ++i) k = block >= l.t[i].first ? i : k;
  return l.t[__builtin_amdgcn_readfirstlane(k)];
}

// u from the gradient and the momentum after its step.
template <typename G>
__device__ inline void update_of(const MuonLaunch& l, const G* g, const float* m, const float (&gv)[8], const float (&mv)[8], float (&u)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float x = gv[j] * l.grad_scale;
    u[j] = !m ? x : l.nesterov ? __builtin_fmaf(l.beta, mv[j], x) : mv[j];
  }
}

// Momentum, and partial sums of u's squares: `sums` workgroups a matrix, each every sums-th piece of 2048 values.
template <typename G>
__global__ __launch_bounds__(256) void momentum_kernel(MuonLaunch l) {
  __shared__ float s_sum[4];
  const Mat& t = mat_of(l, blockIdx.x);
  const int part = blockIdx.x - t.first;
  const int64_t n = (int64_t)t.rows * t.cols;
  float ss = 0.f;
  for (int64_t i0 = (int64_t)part * 2048; i0 < n; i0 += (int64_t)t.sums * 2048) {
    const int64_t i = i0 + 8 * threadIdx.x;
    if (i >= n) break;
    const int left = (int)std::min<int64_t>(n - i, 8);
    float g[8], m[8] = {}, u[8];
    load8((const G*)t.g + i, 0, left, g);
    if (t.m) {
      load8(t.m + i, 0, left, m);
#pragma unroll
      for (int j = 0; j < 8; ++j) m[j] = __builtin_fmaf(l.beta, m[j], g[j] * l.grad_scale);
      store8(t.m + i, 0, left, m);
    }
    update_of(l, (const G*)t.g, t.m, g, m, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += u[j] * u[j];
  }
  ss = lanes_sum<64>(ss);
  if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = ss;
  __syncthreads();
  if (threadIdx.x == 0) l.sums[t.norm + part] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}

// Eight values as one or two fp16 parts, `part` elements apart.  A value has to be one fp32 number for both parts: the compiler
// fuses the operation that made it into the conversion (one rounding), and into the other part's (another), which then and now
// leaves a whole unit of the first part between them.  The empty statement keeps it from that.
template <int PARTS>
__device__ inline void store_parts(_Float16* to, int64_t part, const float (&v)[8]) {
  float lo[8];
  typename Vec8<_Float16>::type hi;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    lo[j] = v[j];
    asm("" : "+v"(lo[j]));
    hi[j] = (_Float16)lo[j];
    lo[j] -= (float)hi[j];
  }
  *(typename Vec8<_Float16>::type*)to = hi;
  if constexpr (PARTS == 2) store8(to + part, lo);
}

// X = u / (|u| + eps), in rows of up8(cols); units of eight values.
template <typename G, int PARTS>
__global__ __launch_bounds__(256) void start_kernel(MuonLaunch l) {
  __shared__ float s_sum[4];
  const Mat& t = mat_of(l, blockIdx.x);
  float ss = 0.f;
  for (int i = threadIdx.x; i < t.sums; i += 256) ss += l.sums[t.norm + i];
  ss = lanes_sum<64>(ss);
  if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = ss;
  __syncthreads();
  ss = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
  const float mul = ldexpf(1.f / (sqrtf(ss) + l.eps), XS);
  const int ld = up8(t.cols), per = ld / 8;
  const int64_t part = (int64_t)t.rows * ld, total = (int64_t)t.rows * per;
#pragma unroll 1
  for (int k = 0; k < 4; ++k) {
    const int64_t unit = ((int64_t)(blockIdx.x - t.first) * 4 + k) * 256 + threadIdx.x;
    if (unit >= total) return;
    const int64_t row = unit / per;
    const int c = (int)(unit - row * per) * 8;
    float g[8], m[8] = {}, u[8];
    load8((const G*)t.g + row * t.cols, c, t.cols, g);
    if (t.m) load8(t.m + row * t.cols, c, t.cols, m);
    update_of(l, (const G*)t.g, t.m, g, m, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] *= mul;
    store_parts<PARTS>((_Float16*)(l.work + t.x[0]) + row * ld + c, part, u);
  }
}

// A = X X' (SQUARE: A A) into slabs [splits][r][up(r, T)]: the tiles of the lower half.  TALL: X' X.
template <bool TALL, bool SQUARE, int PARTS>
__global__ __launch_bounds__(256) void gram_kernel(MuonLaunch l) {
  constexpr int NST = 2, STAGE = 2 * T * BK * 2, OUT_ROW = 64 * 4 + 16;
  __shared__ __align__(1024) char s_mem[NST * STAGE > 4 * 32 * OUT_ROW ? NST * STAGE : 4 * 32 * OUT_ROW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int all = gridDim.x, xcd = blockIdx.x % 8, per = all / 8, rem = all % 8;
  const int job = xcd * per + min(xcd, rem) + blockIdx.x / 8;  // each XCD takes a contiguous range
  const Mat& t = mat_of(l, job);
  const int r = min(t.rows, t.cols), tiles = (r + T - 1) / T, half_tiles = tiles * (tiles + 1) / 2;
  const int in = job - t.first, split = in / half_tiles, id = in - split * half_tiles;
  int tm = (int)((sqrtf(8.f * id + 1.f) - 1.f) * 0.5f);  // id = tm (tm + 1) / 2 + tn, tn <= tm
  while (tm * (tm + 1) / 2 > id) --tm;
  while ((tm + 1) * (tm + 2) / 2 <= id) ++tm;
  const int tn = id - tm * (tm + 1) / 2, m0 = tm * T, n0 = tn * T;
  const int ld = up8(SQUARE ? r : t.cols);
  const int64_t part = (int64_t)(SQUARE ? r : t.rows) * ld;
  const void* x = l.work + (SQUARE ? t.a : t.x[l.from]);
  const int rows = SQUARE ? r : TALL ? ld : t.rows, K = SQUARE ? r : TALL ? t.rows : t.cols;
  f32x16 acc[2][2];
  multiply<_Float16, TALL, TALL, T, T, 2, 2, NST, PARTS == 2>(
      s_mem, Multiplied{x, x, ld, ld, part, part, rows, rows, TALL ? K : up8(K), PARTS == 2 ? 3 : 1}, m0, n0, split, t.splits, wave, lane, acc);

  const int l32 = lane & 31, half = lane >> 5, wm = wave % 2, wn = wave / 2;
  const int64_t slab_ld = (int64_t)tiles * T;
  float* out = (float*)(l.work + t.slab) + split * r * slab_ld;
  __syncthreads();
  char* stg = s_mem + wave * 32 * OUT_ROW;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][b][4 * q + e];
        *(f32x4*)(stg + l32 * OUT_ROW + (32 * i + 8 * q + 4 * half) * 4) = v;
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int line = 4 * k + (lane >> 4), n = n0 + wn * 64 + 32 * b + line, m = m0 + wm * 64 + (lane & 15) * 4;
      if (n < r) *(f32x4*)(out + n * slab_ld + m) = *(const f32x4*)(stg + line * OUT_ROW + (lane & 15) * 16);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Adds the slabs of a 64 x 64 block and its mirror: A (POLY: P = b A + c A^2), in parts, both blocks.
template <bool POLY, int PARTS>
__global__ __launch_bounds__(256) void mirror_kernel(MuonLaunch l) {
  __shared__ float s_v[64][65];
  const Mat& t = mat_of(l, blockIdx.x);
  const int r = min(t.rows, t.cols), id = blockIdx.x - t.first;
  int bm = (int)((sqrtf(8.f * id + 1.f) - 1.f) * 0.5f);
  while (bm * (bm + 1) / 2 > id) --bm;
  while ((bm + 1) * (bm + 2) / 2 <= id) ++bm;
  const int bn = id - bm * (bm + 1) / 2;
  const int64_t slab_ld = (r + T - 1) / T * T;
  const float* slab = (const float*)(l.work + t.slab);
  const int c4 = (threadIdx.x & 15) * 4, row0 = threadIdx.x >> 4;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int rr = row0 + 16 * k, n = bn * 64 + rr;
    f32x4 v{};
    if (n < r)
#pragma unroll 4
      for (int s = 0; s < t.splits; ++s) v += *(const f32x4*)(slab + (s * (int64_t)r + n) * slab_ld + bm * 64 + c4);
#pragma unroll
    for (int e = 0; e < 4; ++e) s_v[rr][c4 + e] = v[e];
  }
  __syncthreads();
  const int ld = up8(r);
  const int64_t part = (int64_t)r * ld;
  const _Float16* A = (const _Float16*)(l.work + t.a);
  _Float16* to = (_Float16*)(l.work + (POLY ? t.poly : t.a));
  // block (bn, bm) as it lies, then (bm, bn): rows of 64 in units of eight
  for (int side = 0; side < (bm == bn ? 1 : 2); ++side) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int unit = threadIdx.x + 256 * k, rr = unit >> 3, cc = (unit & 7) * 8;
      const int n = (side ? bm : bn) * 64 + rr, m = (side ? bn : bm) * 64 + cc;
      if (n >= r || m >= ld) continue;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // a block on the diagonal is symmetric to the bit too: the half with the larger column counts
        const bool swap = side || (bm == bn && cc + j < rr);
        const float x = swap ? s_v[cc + j][rr] : s_v[rr][cc + j];
        v[j] = m + j < r ? x : 0.f;
      }
      const int64_t at = (int64_t)n * ld + m;
      if constexpr (POLY) {
        float a[8];
        load8(A + at, a);
        if constexpr (PARTS == 2) {
          float lo[8];
          load8(A + part + at, lo);
#pragma unroll
          for (int j = 0; j < 8; ++j) a[j] += lo[j];
        }
        const float fa = ldexpf(l.b, l.poly_shift - XS), fs = ldexpf(l.c, l.poly_shift - 2 * XS);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __builtin_fmaf(fa, a[j], fs * v[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = ldexpf(v[j], -XS);
      }
      store_parts<PARTS>(to + at, part, v);
    }
  }
}

// X = a X + P X (TALL: a X + X P), into the other buffer, or (LAST) p's step.
template <bool TALL, int PARTS, bool LAST, typename P, typename O>
__global__ __launch_bounds__(256) void update_kernel(MuonLaunch l) {
  constexpr int NST = 2, STAGE = 2 * T * BK * 2, OUT_ROW = 64 * 4 + 16;
  __shared__ __align__(1024) char s_mem[NST * STAGE > 4 * 32 * OUT_ROW ? NST * STAGE : 4 * 32 * OUT_ROW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int all = gridDim.x, xcd = blockIdx.x % 8, per = all / 8, rem = all % 8;
  const int job = xcd * per + min(xcd, rem) + blockIdx.x / 8;
  const Mat& t = mat_of(l, job);
  const int r = min(t.rows, t.cols), tiles_m = (t.cols + T - 1) / T, tiles_n = (t.rows + T - 1) / T;
  constexpr int COL = 6;
  const int id = job - t.first, col = id / (COL * tiles_m), width = min(COL, tiles_n - col * COL), in = id - col * COL * tiles_m;
  const int m0 = in / width * T, n0 = (col * COL + in % width) * T;  // m: columns of X, n: rows
  const int ld = up8(t.cols), ldp = up8(r);
  const int64_t part = (int64_t)t.rows * ld, ppart = (int64_t)r * ldp;
  const _Float16* x = (const _Float16*)(l.work + t.x[l.from]);
  const void* poly = l.work + t.poly;
  f32x16 acc[2][2];
  const Multiplied wide{x, poly, ld, ldp, part, ppart, ld, r, r, PARTS == 2 ? 3 : 1};
  const Multiplied tall{poly, x, ldp, ld, ppart, part, r, t.rows, ldp, PARTS == 2 ? 3 : 1};
  multiply<_Float16, !TALL, false, T, T, 2, 2, NST, PARTS == 2>(s_mem, TALL ? tall : wide, m0, n0, 0, 1, wave, lane, acc);

  const int l32 = lane & 31, half = lane >> 5, wm = wave % 2, wn = wave / 2;
  const float unscale = ldexpf(1.f, -l.poly_shift), rate = ldexpf(l.lr * t.rate, -XS);
  _Float16* to = (_Float16*)(l.work + t.x[l.from ^ 1]);
  __syncthreads();
  char* stg = s_mem + wave * 32 * OUT_ROW;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][b][4 * q + e];
        *(f32x4*)(stg + l32 * OUT_ROW + (32 * i + 8 * q + 4 * half) * 4) = v;
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int k = 0; k < 4; ++k) {  // eight columns of a row
      const int line = 8 * k + (lane >> 3), n = n0 + wn * 64 + 32 * b + line, c = (lane & 7) * 8, m = m0 + wm * 64 + c;
      if (n >= t.rows || m >= ld) continue;
      float v[8], old[8];
      const f32x4 lo = *(const f32x4*)(stg + line * OUT_ROW + c * 4), hi = *(const f32x4*)(stg + line * OUT_ROW + c * 4 + 16);
      const int64_t at = (int64_t)n * ld + m;
      load8(x + at, old);
      if constexpr (PARTS == 2) {
        float rest[8];
        load8(x + part + at, rest);
#pragma unroll
        for (int j = 0; j < 8; ++j) old[j] += rest[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __builtin_fmaf(l.a, old[j], (j < 4 ? lo[j & 3] : hi[j & 3]) * unscale);
      if constexpr (!LAST) {
        store_parts<PARTS>(to + at, part, v);
      } else {
        P* p = (P*)t.p + (int64_t)n * t.cols;
        float w[8];
        load8(p, m, t.cols, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = __builtin_fmaf(-rate, v[j], w[j] * l.decay);
        store8(p, m, t.cols, w);
        if (t.copy) store8((O*)t.copy + (int64_t)n * t.cols, m, t.cols, w);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

template <typename F>
int with_type(dn_dtype dt, F&& f) {
  if (dt == DN_F32) return f(float{});
  if (dt == DN_F16) return f(_Float16{});
  return f(__bf16{});
}
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
struct Work {  // offsets in the workspace, 256-byte aligned
  size_t total = 0;
  size_t take(size_t bytes) {
    const size_t at = total;
    total += up((int64_t)bytes, 256);
    return at;
  }
};

int parts_of(const dn_muon_params& k, dn_dtype p_dt) { return k.parts ? k.parts : p_dt == DN_BF16 ? 1 : 2; }
int64_t half_tiles(int64_t r, int64_t side) {
  const int64_t tiles = (r + side - 1) / side;
  return tiles * (tiles + 1) / 2;
}
int splits_of(int64_t tiles, int64_t stages) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({512 / std::max<int64_t>(tiles, 1), stages / 8, 16}));
}

// A group of matrices that share launches, laid out in the workspace.
struct Group {
  MuonLaunch l;
  int32_t gram_splits[MATS], square_splits[MATS];
  size_t total;
};
void plan_group(const dn_muon_tensor* ts, int count, int parts, Group& gr) {
  gr.l = MuonLaunch{};
  Work w;
  int64_t tiles = 0;
  for (int i = 0; i < count; ++i) tiles += half_tiles(std::min(ts[i].rows, ts[i].cols), T);
  int32_t sums = 0;
  for (int i = 0; i < count; ++i) {
    Mat& t = gr.l.t[i];
    t.g = ts[i].g, t.m = ts[i].m, t.p = ts[i].p, t.copy = ts[i].copy;
    t.rows = (int32_t)ts[i].rows, t.cols = (int32_t)ts[i].cols, t.rate = (float)ts[i].rate;
    const int64_t r = std::min(t.rows, t.cols), c = std::max(t.rows, t.cols);
    for (int b = 0; b < 2; ++b) t.x[b] = w.take((size_t)parts * t.rows * up8(t.cols) * 2);
    t.a = w.take((size_t)parts * r * up8((int32_t)r) * 2), t.poly = w.take((size_t)parts * r * up8((int32_t)r) * 2);
    const int products = parts == 2 ? 3 : 1;
    gr.gram_splits[i] = splits_of(tiles, (c + BK - 1) / BK * products), gr.square_splits[i] = splits_of(tiles, (r + BK - 1) / BK * products);
    t.slab = w.take((size_t)std::max(gr.gram_splits[i], gr.square_splits[i]) * r * up(r, T) * 4);
    t.sums = (int32_t)std::min<int64_t>(SUMS, ((int64_t)t.rows * t.cols + 2047) / 2048);
    t.norm = sums, sums += t.sums;
  }
  gr.l.count = count;
  gr.l.sums = (float*)w.take((size_t)sums * 4);  // (an offset: the workspace's address is added)
  gr.total = w.total;
}

// The launch of those matrices that `take` chooses, each with `units` workgroups and `splits` splits.
template <typename Take, typename Units>
int64_t select(const MuonLaunch& all, MuonLaunch& l, Take&& take, Units&& units) {
  l = all;
  l.count = 0;
  int64_t total = 0;
  for (int i = 0; i < all.count; ++i)
    if (take(i)) {
      Mat& t = l.t[l.count++];
      t = all.t[i];
      t.first = (int32_t)total;
      total += units(i, t);
    }
  return total;
}

template <int PARTS>
int run_group(Group& gr, const dn_muon_params& k, dn_dtype p_dt, dn_dtype g_dt, dn_dtype copy_dt, hipStream_t st) {
  MuonLaunch l;
  const auto any = [](int) { return true; };
  int64_t n = select(gr.l, l, any, [](int, const Mat& t) { return (int64_t)t.sums; });
  with_type(g_dt, [&](auto g) {
    momentum_kernel<decltype(g)><<<dim3((unsigned)n), 256, 0, st>>>(l);
    return 0;
  });
  if (const int err = (int)hipGetLastError()) return err;
  n = select(gr.l, l, any, [](int, const Mat& t) { return ((int64_t)t.rows * (up8(t.cols) / 8) + 1023) / 1024; });
  with_type(g_dt, [&](auto g) {
    start_kernel<decltype(g), PARTS><<<dim3((unsigned)n), 256, 0, st>>>(l);
    return 0;
  });
  if (const int err = (int)hipGetLastError()) return err;
  const auto tall = [&](int i) { return gr.l.t[i].rows > gr.l.t[i].cols; };
  const auto wide = [&](int i) { return !tall(i); };
  const auto side = [](const Mat& t) { return std::min(t.rows, t.cols); };
  for (int s = 0; s < k.steps; ++s) {
    gr.l.a = (float)k.coefficients[s][0], gr.l.b = (float)k.coefficients[s][1], gr.l.c = (float)k.coefficients[s][2];
    // |P| <= |b| |A| + |c| |A|^2, which is at most 2.25 |c| + 1.5 |b| for singular values up to 1.22, and twice that to spare
    const double most = 2 * (1.5 * std::fabs(k.coefficients[s][1]) + 2.25 * std::fabs(k.coefficients[s][2]));
    gr.l.poly_shift = std::min(XS, (int)std::floor(std::log2(65504 / std::max(most, 1e-6))));
    gr.l.from = s & 1;
    const auto gram = [&](int i, Mat& t) {
      t.splits = gr.gram_splits[i];
      return half_tiles(side(t), T) * t.splits;
    };
    if ((n = select(gr.l, l, wide, gram))) gram_kernel<false, false, PARTS><<<dim3((unsigned)n), 256, 0, st>>>(l);
    if ((n = select(gr.l, l, tall, gram))) gram_kernel<true, false, PARTS><<<dim3((unsigned)n), 256, 0, st>>>(l);
    n = select(gr.l, l, any, [&](int i, Mat& t) { return t.splits = gr.gram_splits[i], half_tiles(side(t), 64); });
    mirror_kernel<false, PARTS><<<dim3((unsigned)n), 256, 0, st>>>(l);
    n = select(gr.l, l, any, [&](int i, Mat& t) {
      t.splits = gr.square_splits[i];
      return half_tiles(side(t), T) * t.splits;
    });
    gram_kernel<false, true, PARTS><<<dim3((unsigned)n), 256, 0, st>>>(l);
    n = select(gr.l, l, any, [&](int i, Mat& t) { return t.splits = gr.square_splits[i], half_tiles(side(t), 64); });
    mirror_kernel<true, PARTS><<<dim3((unsigned)n), 256, 0, st>>>(l);
    const auto update = [&](int, Mat& t) { return (int64_t)((t.rows + T - 1) / T) * ((t.cols + T - 1) / T); };
    for (int shape = 0; shape < 2; ++shape) {
      n = shape ? select(gr.l, l, tall, update) : select(gr.l, l, wide, update);
      if (!n) continue;
      const dim3 grid((unsigned)n);
      if (s + 1 < k.steps) {
        if (shape) update_kernel<true, PARTS, false, float, __bf16><<<grid, 256, 0, st>>>(l);
        else update_kernel<false, PARTS, false, float, __bf16><<<grid, 256, 0, st>>>(l);
        continue;
      }
      with_type(p_dt, [&](auto p) {
        using P = decltype(p);
        const auto go = [&](auto o) {
          using O = decltype(o);
          if (shape) update_kernel<true, PARTS, true, P, O><<<grid, 256, 0, st>>>(l);
          else update_kernel<false, PARTS, true, P, O><<<grid, 256, 0, st>>>(l);
        };
        if (copy_dt == DN_F16) go(_Float16{});
        else go(__bf16{});
        return 0;
      });
    }
    if (const int err = (int)hipGetLastError()) return err;
  }
  return 0;
}

}  // namespace

size_t muon_bytes(const dn_muon_tensor* tensors, int32_t count, dn_dtype p_dt, const dn_muon_params& k) {
  size_t most = 256;
  Group gr;
  for (int32_t at = 0; at < count; at += MATS) {
    plan_group(tensors + at, std::min(count - at, MATS), parts_of(k, p_dt), gr);
    most = std::max(most, gr.total);
  }
  return most;
}

int launch_muon(const dn_muon_tensor* tensors, int32_t count, dn_dtype p_dt, dn_dtype g_dt, dn_dtype copy_dt, const dn_muon_params& k,
                void* d_work, void* stream) {
  for (int32_t at = 0; at < count; at += MATS) {  // groups share the workspace: the stream keeps them apart
    Group gr;
    const int parts = parts_of(k, p_dt);
    plan_group(tensors + at, std::min(count - at, MATS), parts, gr);
    gr.l.work = (char*)d_work;
    gr.l.sums = (float*)((char*)d_work + (size_t)gr.l.sums);
    gr.l.beta = (float)k.momentum, gr.l.grad_scale = (float)k.grad_scale, gr.l.eps = (float)k.eps, gr.l.lr = (float)k.lr;
    gr.l.decay = (float)(1 - k.lr * k.weight_decay), gr.l.nesterov = k.nesterov;
    const int err = parts == 2 ? run_group<2>(gr, k, p_dt, g_dt, copy_dt, (hipStream_t)stream)
                               : run_group<1>(gr, k, p_dt, g_dt, copy_dt, (hipStream_t)stream);
    if (err) return err;
  }
  return 0;
}

}  // namespace head
}  // namespace dn
