// Muon: a matrix's momentum, orthogonalised by Newton-Schulz steps, as its update.
//   m = beta m + g';  u = g' + beta m (nesterov) or m;  X = u / (|u| + eps)
//   per step: A = X X',  P = b A + c A^2,  X = a X + P X   (of a tall X: A = X' X,  X = a X + X P)
//   p = p (1 - lr weight_decay) - lr rate X
// A, P and A^2 have the smaller side r of the matrix, and are symmetric: half their tiles are computed and mirrored.  A step is
// 3 r^2 c + r^3 operations (c: the larger side), on the matrix cores, in one or two fp16 parts of every value:
//   X is held times 2^13, A and P times powers of two that the singular values of X and the coefficients allow (steps_of), all of
//   them below fp16's largest (singular values are at most about 1.2 with the usual coefficients, and A times 2^13 too).  One part is 11 bits of a value down to 2^-27: the steps'
//   roundings are of either sign and come to about 2^-11 of the update in all, below half a unit of a bf16 weight.  Two parts
//   (fp32 and fp16 weights) are 22 bits, in three products of parts, as the loss's logits in fp32.
// Bound by the matrix cores: six matrices of 2048 x 8192 in bf16 take 3.7 to 4.2 ms by machine and clock (0.89 to 0.79 PFLOP/s), one of
// 1000 x 9216 in two parts 0.75 to 0.83 ms (0.57 to 0.52: its 144 tiles leave CUs idle), four of 512 x 512 278 us in two parts and 164 in one, which are launches more than work.
// All matrices of a call go through the same launches.  Sums over k go to slabs in fp32, one for each split, and a launch adds
// them in order, so results do not depend on what ran first.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "tiles.h"

namespace dn {
namespace head {
namespace {

constexpr int XS = 13;  // X is held times 2^XS, which singular values below 4 allow
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
constexpr int MATS = 32;
struct MuonLaunch {
  Mat t[MATS];
  int32_t count;
  char* work;
  float* sums;
  float beta, grad_scale, eps, lr, decay;
  float a, b, c;  // of the step
  int32_t a_shift, poly_shift;  // A and P are held times 2^these
  int32_t nesterov, from;  // from: the buffer that X is in
};
constexpr size_t MAX_ARGUMENTS = 4096;  // bytes of a launch
static_assert(sizeof(MuonLaunch) <= MAX_ARGUMENTS, "the matrices of a launch are its arguments");

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

// Tile shapes: 256 x 256 by eight waves, a workgroup per CU, 128 x 128 by four, two per CU, or 128 x 64 by four, three per CU.
template <int BM, int BN = BM>
struct Shape {
  static constexpr int WM = 2, WN = BM == 256 ? 4 : 2, NW = WM * WN, NST = 2, STAGE = (BM + BN) * BK * 2;
  static constexpr int WCOLS = BM / WM, WROWS = BN / WN, TM = WCOLS / 32, TN = WROWS / 32;
  static constexpr int OUT_ROW = WCOLS * 4 + 16, OUT = NW * 32 * OUT_ROW;
  static constexpr int LDS = NST * STAGE > OUT ? NST * STAGE : OUT;
};
// The tile's rows n on their way out, through LDS: `row(n, c, v)` gets eight values of row n of the tile from column c on.
template <typename S, typename F>
__device__ inline void rows_out(char* s_mem, int wave, int lane, const f32x16 (&acc)[S::TM][S::TN], F&& row) {
  const int l32 = lane & 31, half = lane >> 5, wm = wave % S::WM, wn = wave / S::WM;
  constexpr int LANES = S::WCOLS / 8, LINES = 64 / LANES;
  __syncthreads();
  char* stg = s_mem + wave * 32 * S::OUT_ROW;
#pragma unroll
  for (int b = 0; b < S::TN; ++b) {
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][b][4 * q + e];
        *(f32x4*)(stg + l32 * S::OUT_ROW + (32 * i + 8 * q + 4 * half) * 4) = v;
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int k = 0; k < 32 / LINES; ++k) {
      const int line = LINES * k + lane / LANES, c = lane % LANES * 8;
      const f32x4 lo = *(const f32x4*)(stg + line * S::OUT_ROW + c * 4), hi = *(const f32x4*)(stg + line * S::OUT_ROW + c * 4 + 16);
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < 4 ? lo[j & 3] : hi[j & 3];
      row(wn * S::WROWS + 32 * b + line, wm * S::WCOLS + c, v);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// The tile's columns m on their way out as rows: `row(m, n, v)` gets eight values of column m from row n on.
template <int T, typename F>
__device__ inline void columns_out(char* s_mem, int wave, int lane, const f32x16 (&acc)[Shape<T>::TM][Shape<T>::TN], F&& row) {
  using S = Shape<T>;
  const int l32 = lane & 31, half = lane >> 5, wm = wave % S::WM, wn = wave / S::WM;
  constexpr int ROW = S::WROWS * 4 + 16, LANES = S::WROWS / 8, LINES = 64 / LANES;
  static_assert(S::NW * 32 * ROW <= S::LDS, "a wave's 32 columns fit");
  __syncthreads();
  char* stg = s_mem + wave * 32 * ROW;
#pragma unroll
  for (int i = 0; i < S::TM; ++i) {
#pragma unroll
    for (int b = 0; b < S::TN; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) *(float*)(stg + (8 * (e / 4) + 4 * half + e % 4) * ROW + (32 * b + l32) * 4) = acc[i][b][e];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int k = 0; k < 32 / LINES; ++k) {
      const int line = LINES * k + lane / LANES, c = lane % LANES * 8;
      const f32x4 lo = *(const f32x4*)(stg + line * ROW + c * 4), hi = *(const f32x4*)(stg + line * ROW + c * 4 + 16);
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < 4 ? lo[j & 3] : hi[j & 3];
      row(wm * S::WCOLS + 32 * i + line, wn * S::WROWS + c, v);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Eight values of a matrix held in parts.
template <int PARTS>
__device__ inline void load_parts(const _Float16* p, int64_t part, float (&v)[8]) {
  load8(p, v);
  if constexpr (PARTS == 2) {
    float lo[8];
    load8(p + part, lo);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += lo[j];
  }
}
// An entry of A from X X', or (SQUARE) of P = b A + c A^2 from A's and A A's.
template <bool SQUARE>
struct Entry {
  float fa, fs;
  __device__ inline Entry(const MuonLaunch& l) {
    fa = SQUARE ? ldexpf(l.b, l.poly_shift - l.a_shift) : 0.f;
    fs = SQUARE ? ldexpf(l.c, l.poly_shift - 2 * l.a_shift) : ldexpf(1.f, l.a_shift - 2 * XS);
  }
  __device__ inline float operator()(float sum, float a) const { return SQUARE ? __builtin_fmaf(fa, a, fs * sum) : fs * sum; }
};

// A = X X' (of a tall matrix X' X), or (SQUARE) P = b A + c A A: the tiles of the lower half, written in both places.  SLABS: their
// sums alone, a slab [r][up(r, T)] for each split; mirror_kernel does the rest.
template <bool SQUARE, int PARTS, int T, bool SLABS>
__global__ __launch_bounds__(64 * Shape<T>::NW) void gram_kernel(MuonLaunch l) {
  using S = Shape<T>;
  __shared__ __align__(1024) char s_mem[S::LDS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int all = gridDim.x, xcd = blockIdx.x % 8, per = all / 8, rem = all % 8;
  const int job = xcd * per + min(xcd, rem) + blockIdx.x / 8;  // each XCD takes a contiguous range
  const Mat& t = mat_of(l, job);
  const int r = min(t.rows, t.cols), tiles = (r + T - 1) / T, half_tiles = tiles * (tiles + 1) / 2;
  const int in = job - t.first, split = SLABS ? in / half_tiles : 0, id = in - split * half_tiles;
  int tm = (int)((sqrtf(8.f * id + 1.f) - 1.f) * 0.5f);  // id = tm (tm + 1) / 2 + tn, tn <= tm
  while (tm * (tm + 1) / 2 > id) --tm;
  while ((tm + 1) * (tm + 2) / 2 <= id) ++tm;
  const int tn = id - tm * (tm + 1) / 2, m0 = tm * T, n0 = tn * T;
  const int ld = up8(SQUARE ? r : t.cols);
  const int64_t part = (int64_t)(SQUARE ? r : t.rows) * ld;
  const _Float16* x = (const _Float16*)(l.work + (SQUARE ? t.a : t.x[l.from]));
  f32x16 acc[S::TM][S::TN];
  Multiplied op{x, x, ld, ld, part, part, SQUARE ? r : t.rows, SQUARE ? r : t.rows, ld, PARTS == 2 ? 3 : 1};
  const int splits = SLABS ? t.splits : 1;
  if (SQUARE || t.rows <= t.cols) {
    multiply<_Float16, false, false, T, T, S::WM, S::WN, S::NST, PARTS == 2>(s_mem, op, m0, n0, split, splits, wave, lane, acc);
  } else if constexpr (!SQUARE) {
    op.a_rows = op.b_rows = ld, op.K = t.rows;
    multiply<_Float16, true, true, T, T, S::WM, S::WN, S::NST, PARTS == 2>(s_mem, op, m0, n0, split, splits, wave, lane, acc);
  }
  if constexpr (SLABS) {
    const int64_t slab_ld = (int64_t)tiles * T;
    float* out = (float*)(l.work + t.slab) + split * r * slab_ld;
    rows_out<S>(s_mem, wave, lane, acc, [&](int n, int m, const float (&v)[8]) {
      if (n0 + n < r) store8(out + (n0 + n) * slab_ld + m0 + m, v);
    });
  } else {
    const int lda = up8(r);
    const int64_t apart = (int64_t)r * lda;
    _Float16* to = (_Float16*)(l.work + (SQUARE ? t.poly : t.a));
    const Entry<SQUARE> entry(l);
    if (tm != tn)  // the mirrored tile (one on the diagonal is its own mirror, within roundings)
      columns_out<T>(s_mem, wave, lane, acc, [&](int m, int n, float (&v)[8]) {
        n += n0, m += m0;  // (n is below r: its tile is a whole one)
        if (m >= r) return;
        const int64_t at = (int64_t)m * lda + n;
        float a[8] = {};
        if constexpr (SQUARE) load_parts<PARTS>(x + at, apart, a);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = entry(v[j], a[j]);
        store_parts<PARTS>(to + at, apart, v);
      });
    rows_out<S>(s_mem, wave, lane, acc, [&](int n, int m, float (&v)[8]) {
      n += n0, m += m0;
      if (n >= r || m >= lda) return;
      const int64_t at = (int64_t)n * lda + m;
      float a[8] = {};
      if constexpr (SQUARE) load_parts<PARTS>(x + at, apart, a);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = entry(v[j], a[j]);  // (0 past column r)
      store_parts<PARTS>(to + at, apart, v);
    });
  }
}

// Adds the slabs of a 64 x 64 block and its mirror: A (POLY: P = b A + c A^2), in parts, both blocks.  T: the slabs' tiles.  (A
// thread has four values of a slab: there are few blocks, and each waits for memory.)
template <bool POLY, int PARTS, int T>
__global__ __launch_bounds__(1024) void mirror_kernel(MuonLaunch l) {
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
  f32x4 sum{};
  if (bn * 64 + row0 < r)
#pragma unroll 8
    for (int s = 0; s < t.splits; ++s) sum += *(const f32x4*)(slab + (s * (int64_t)r + bn * 64 + row0) * slab_ld + bm * 64 + c4);
#pragma unroll
  for (int e = 0; e < 4; ++e) s_v[row0][c4 + e] = sum[e];
  __syncthreads();
  const int ld = up8(r);
  const int64_t part = (int64_t)r * ld;
  const _Float16* A = (const _Float16*)(l.work + t.a);
  _Float16* to = (_Float16*)(l.work + (POLY ? t.poly : t.a));
  const Entry<POLY> entry(l);
  // the first half of the threads: block (bn, bm) as it lies, the other: (bm, bn); rows of 64 in units of eight
  const int side = threadIdx.x >> 9, unit = threadIdx.x & 511, rr = unit >> 3, cc = (unit & 7) * 8;
  const int n = (side ? bm : bn) * 64 + rr, m = (side ? bn : bm) * 64 + cc;
  if (n >= r || m >= ld || (side && bm == bn)) return;
  float v[8], own[8] = {};
  const int64_t at = (int64_t)n * ld + m;
  if constexpr (POLY) load_parts<PARTS>(A + at, part, own);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    // a block on the diagonal is symmetric to the bit too: the half with the larger column counts
    const bool swap = side || (bm == bn && cc + j < rr);
    const float x = swap ? s_v[cc + j][rr] : s_v[rr][cc + j];
    v[j] = entry(m + j < r ? x : 0.f, own[j]);
  }
  store_parts<PARTS>(to + at, part, v);
}

// X = a X + P X (of a tall matrix a X + X P), into the other buffer, or (LAST) p's step.
template <int PARTS, int BM, int BN, bool LAST, typename P, typename O>
__global__ __launch_bounds__((64 * Shape<BM, BN>::NW)) void update_kernel(MuonLaunch l) {
  using S = Shape<BM, BN>;
  __shared__ __align__(1024) char s_mem[S::LDS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int all = gridDim.x, xcd = blockIdx.x % 8, per = all / 8, rem = all % 8;
  const int job = xcd * per + min(xcd, rem) + blockIdx.x / 8;
  const Mat& t = mat_of(l, job);
  const int r = min(t.rows, t.cols), tiles_m = (t.cols + BM - 1) / BM, tiles_n = (t.rows + BN - 1) / BN;
  constexpr int COL = 6;
  const int id = job - t.first, col = id / (COL * tiles_m), width = min(COL, tiles_n - col * COL), in = id - col * COL * tiles_m;
  const int m0 = in / width * BM, n0 = (col * COL + in % width) * BN;  // m: columns of X, n: rows
  const int ld = up8(t.cols), ldp = up8(r);
  const int64_t part = (int64_t)t.rows * ld, ppart = (int64_t)r * ldp;
  const _Float16* x = (const _Float16*)(l.work + t.x[l.from]);
  const void* poly = l.work + t.poly;
  f32x16 acc[S::TM][S::TN];
  if (t.rows <= t.cols)
    multiply<_Float16, true, false, BM, BN, S::WM, S::WN, S::NST, PARTS == 2>(
        s_mem, Multiplied{x, poly, ld, ldp, part, ppart, ld, r, r, PARTS == 2 ? 3 : 1}, m0, n0, 0, 1, wave, lane, acc);
  else
    multiply<_Float16, false, false, BM, BN, S::WM, S::WN, S::NST, PARTS == 2>(
        s_mem, Multiplied{poly, x, ldp, ld, ppart, part, r, t.rows, ldp, PARTS == 2 ? 3 : 1}, m0, n0, 0, 1, wave, lane, acc);

  const float unscale = ldexpf(1.f, -l.poly_shift), rate = ldexpf(l.lr * t.rate, -XS);
  _Float16* to = (_Float16*)(l.work + t.x[l.from ^ 1]);
  rows_out<S>(s_mem, wave, lane, acc, [&](int n, int m, float (&v)[8]) {
    n += n0, m += m0;
    if (n >= t.rows || m >= ld) return;
    const int64_t at = (int64_t)n * ld + m;
    float old[8];
    load_parts<PARTS>(x + at, part, old);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __builtin_fmaf(l.a, old[j], v[j] * unscale);
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
  });
}

// A small matrix's whole step by one workgroup, X and A in LDS (a tall one turned, so that rows are the smaller side): of the general
// path's 17 launches each takes 8 us and more for next to no work (four matrices of 96 x 256 in fp32: 178 us, so 81).
// X: [r32][c32 + 8] in parts, zeros past r and c; A, and P over it: [r32][r32 + 8].  Rows 16 bytes longer than a multiple of 64
// spread over the banks.  Waves take 32 x 32 tiles of A and A A, and columns of 32 of P X, whose rows they replace.
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
constexpr int SMALL_WAVES = 16, SMALL_LDS = 159 * 1024;
__host__ __device__ inline int up32(int x) { return (x + 31) / 32 * 32; }
__host__ __device__ inline int64_t small_bytes(int64_t rows, int64_t cols, int parts) {
  const int64_t r = (rows < cols ? rows : cols), c = rows < cols ? cols : rows;
  if (r > 128 || c > 4096) return SMALL_LDS + 1;
  return (int64_t)parts * 2 * up32((int)r) * (up32((int)c) + 8 + up32((int)r) + 8);
}
struct SmallMat {
  const void* g;
  float* m;
  void *p, *copy;
  int32_t rows, cols;
  float rate;
};
constexpr int SMALL_MATS = 48;
struct SmallLaunch {
  SmallMat t[SMALL_MATS];
  float beta, grad_scale, eps, lr, decay;
  int32_t nesterov, steps;
  float coef[DN_MAX_NS_STEPS][3];
  int32_t a_shift[DN_MAX_NS_STEPS], poly_shift[DN_MAX_NS_STEPS];
};
static_assert(sizeof(SmallLaunch) <= MAX_ARGUMENTS, "the matrices of a launch are its arguments");
template <int PARTS, typename P, typename G, typename O>
__global__ __launch_bounds__(64 * SMALL_WAVES) void small_kernel(SmallLaunch l) {
  extern __shared__ __align__(16) char s_mem[];
  __shared__ float s_sum[SMALL_WAVES];
  const SmallMat& t = l.t[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
  const bool tall = t.rows > t.cols;
  const int r = tall ? t.cols : t.rows, c = tall ? t.rows : t.cols, r32 = up32(r), c32 = up32(c), lx = c32 + 8, la = r32 + 8;
  const int xpart = r32 * lx, apart = r32 * la;
  _Float16 *X = (_Float16*)s_mem, *A = X + PARTS * xpart;
  const int n = t.rows * t.cols;
  const auto put = [&](_Float16* at, int part, float v) {
    asm("" : "+v"(v));  // (see store_parts)
    const _Float16 hi = (_Float16)v;
    *at = hi;
    if constexpr (PARTS == 2) at[part] = (_Float16)(v - (float)hi);
  };
  const auto get = [&](const _Float16* at, int part) { return PARTS == 2 ? (float)at[0] + (float)at[part] : (float)at[0]; };
  // u of eight values at a time, whose loads go out together; `first`: momentum makes its step
  constexpr int STEP = 64 * SMALL_WAVES;
  const auto updates = [&](int i0, bool first, float (&u)[8]) {
    float m[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = min(i0 + j * STEP, n - 1);
      u[j] = (float)((const G*)t.g)[i] * l.grad_scale, m[j] = t.m ? t.m[i] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (first) m[j] = __builtin_fmaf(l.beta, m[j], u[j]);
      if (first && t.m && i0 + j * STEP < n) t.m[i0 + j * STEP] = m[j];
      if (t.m) u[j] = l.nesterov ? __builtin_fmaf(l.beta, m[j], u[j]) : m[j];
    }
  };
  float ss = 0.f;
  for (int i = threadIdx.x; i < n; i += 8 * STEP) {
    float u[8];
    updates(i, true, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += i + j * STEP < n ? u[j] * u[j] : 0.f;
  }
  ss = lanes_sum<64>(ss);
  if (lane == 0) s_sum[wave] = ss;
  for (int i = threadIdx.x; i < PARTS * xpart / 8; i += 64 * SMALL_WAVES) *(f32x4*)(X + 8 * i) = f32x4{};
  __syncthreads();
  ss = 0.f;
  for (int w = 0; w < SMALL_WAVES; ++w) ss += s_sum[w];
  const float mul = ldexpf(1.f / (sqrtf(ss) + l.eps), XS);
  for (int i0 = threadIdx.x; i0 < n; i0 += 8 * STEP) {  // (a thread reads the momentum that it wrote)
    float u[8];
    updates(i0, false, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = i0 + j * STEP, row = i / t.cols, col = i - row * t.cols;
      if (i < n) put(X + (tall ? col * lx + row : row * lx + col), xpart, u[j] * mul);
    }
  }
  __syncthreads();
  const int tiles = r32 / 32;
  const int ways = c32 / 32 * tiles <= SMALL_WAVES ? tiles : tiles > 1 && c32 / 32 * 2 <= SMALL_WAVES ? 2 : 1;  // waves to 32 columns of X
  const int each = (tiles + ways - 1) / ways;
  // a tile's products of k from rows of p (rows from i0) and of q (from j0): D[i][j]
  const auto rows_product = [&](const _Float16* p, int ld, int part, int i0, int j0, int k, f32x16& acc) {
#pragma unroll
    for (int pr = PARTS == 2 ? 0 : 2; pr < 3; ++pr) {  // parts (1, 0), (0, 1), (0, 0)
      const _Float16* a = p + (pr == 0 ? part : 0) + (i0 + l32) * ld + 8 * half;
      const _Float16* b = p + (pr == 1 ? part : 0) + (j0 + l32) * ld + 8 * half;
#pragma unroll 4
      for (int k0 = 0; k0 < k; k0 += 16) acc = Mfma<_Float16>::mma(*(const f16x8*)(a + k0), *(const f16x8*)(b + k0), acc);
    }
  };
  for (int s = 0; s < l.steps; ++s) {
    // A = X X', all tiles (the mirrored ones too: there are waves to spare)
    for (int id = wave; id < tiles * tiles; id += SMALL_WAVES) {
      const int i0 = id / tiles * 32, j0 = id % tiles * 32;
      f32x16 acc{};
      rows_product(X, lx, xpart, i0, j0, c32, acc);
#pragma unroll
      for (int e = 0; e < 16; ++e) put(A + (i0 + 8 * (e / 4) + 4 * half + e % 4) * la + j0 + l32, apart, ldexpf(acc[e], l.a_shift[s] - 2 * XS));
    }
    __syncthreads();
    // P = b A + c A A, over A once all waves have read it (16 waves: a tile each)
    f32x16 square{};
    const int i0 = wave / tiles * 32, j0 = wave % tiles * 32;
    const bool is = wave < tiles * tiles;
    if (is) rows_product(A, la, apart, i0, j0, r32, square);
    __syncthreads();
    if (is) {
      const float fa = ldexpf(l.coef[s][1], l.poly_shift[s] - l.a_shift[s]), fs = ldexpf(l.coef[s][2], l.poly_shift[s] - 2 * l.a_shift[s]);
      const auto place = [&](int e) { return A + (i0 + 8 * (e / 4) + 4 * half + e % 4) * la + j0 + l32; };
#pragma unroll
      for (int e = 0; e < 16; ++e) square[e] = __builtin_fmaf(fa, get(place(e), apart), fs * square[e]);
#pragma unroll
      for (int e = 0; e < 16; ++e) put(place(e), apart, square[e]);
    }
    __syncthreads();
    // X = a X + P X: `each` blocks of 32 rows of 32 columns a wave, D[m][n] = sum_k X[k][m] P[n][k]
    const float unscale = ldexpf(1.f, -l.poly_shift[s]);
    for (int first = 0; first < c32; first += SMALL_WAVES / ways * 32) {
      const int m0 = first + wave / ways * 32, b0 = wave % ways * each, count = m0 < c32 ? min(each, tiles - b0) : 0;
      f32x16 acc[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) acc[b] = f32x16{};
#pragma unroll
      for (int pr = PARTS == 2 ? 0 : 2; pr < 3; ++pr) {
        const _Float16* x = X + (pr == 0 ? xpart : 0) + m0;
        const _Float16* q = A + (pr == 1 ? apart : 0);
        if (count <= 0) continue;
#pragma unroll 2
        for (int k0 = 0; k0 < r32; k0 += 16) {
          f16x8 a;
#pragma unroll
          for (int j = 0; j < 8; ++j) a[j] = x[(k0 + 8 * half + j) * lx + l32];
#pragma unroll
          for (int b = 0; b < 4; ++b)
            if (b < count) acc[b] = Mfma<_Float16>::mma(a, *(const f16x8*)(q + (32 * (b0 + b) + l32) * la + k0 + 8 * half), acc[b]);
        }
      }
      if (ways > 1) __syncthreads();  // other waves read these columns too
      // element e of acc[b]: column m0 + 8 (e / 4) + 4 half + e % 4 of row 32 (b0 + b) + l32
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (b >= count) continue;
        const int row = 32 * (b0 + b) + l32, col0 = m0 + 4 * half;
        _Float16* mine = X + row * lx + col0;
        // (all of X's old values before the first is written)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const f16x4 hi = *(const f16x4*)(mine + 2 * e), lo = PARTS == 2 ? *(const f16x4*)(mine + xpart + 2 * e) : f16x4{};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[b][e + j] = __builtin_fmaf(l.coef[s][0], (float)hi[j] + (float)lo[j], acc[b][e + j] * unscale);
        }
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          f16x4 hi, lo;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float v = acc[b][e + j];
            asm("" : "+v"(v));
            hi[j] = (_Float16)v, lo[j] = (_Float16)(v - (float)hi[j]);
          }
          *(f16x4*)(mine + 2 * e) = hi;
          if constexpr (PARTS == 2) *(f16x4*)(mine + xpart + 2 * e) = lo;
        }
      }
    }
    __syncthreads();
  }
  // the weights, in their own order (from the accumulators, each lane with values of its own row, this took 29 us more)
  const float rate = ldexpf(l.lr * t.rate, -XS);
  for (int i0 = threadIdx.x; i0 < n; i0 += 8 * STEP) {
    float w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = (float)((const P*)t.p)[min(i0 + j * STEP, n - 1)];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = i0 + j * STEP, row = i / t.cols, col = i - row * t.cols;
      if (i >= n) continue;
      w[j] = __builtin_fmaf(-rate, get(X + (tall ? col * lx + row : row * lx + col), xpart), w[j] * l.decay);
      ((P*)t.p)[i] = (P)w[j];
      if (t.copy) ((O*)t.copy)[i] = (O)w[j];
    }
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

// Powers of two that each step's A and P are held times, so that fp16 holds the largest that they can be.  X's singular values are at
// most 1 before the first step, and after a step at most the largest |a s + b s^3 + c s^5| of those before it (and 4, by what
// coefficients have to keep); |A| is at most the largest of them squared, and |P| the largest |b t + c t^2| up to there.  2 % are left
// for roundings, and P has at least twice 1.5 |b| + 2.25 |c|, which is more than the usual coefficients need.
struct StepShifts {
  int32_t a, poly;
};
void steps_of(const dn_muon_params& k, StepShifts (&to)[DN_MAX_NS_STEPS]) {
  const auto shift = [](double most) { return (int32_t)std::min<double>(XS, std::floor(std::log2(65504 / std::max(most, 1e-6)))); };
  double top = 1;
  for (int32_t i = 0; i < k.steps; ++i) {
    const double a = k.coefficients[i][0], b = k.coefficients[i][1], c = k.coefficients[i][2], t = top * top;
    const auto p = [&](double t) { return std::fabs(b * t + c * t * t); };
    const auto x = [&](double t) { return std::sqrt(t) * std::fabs(a + b * t + c * t * t); };
    double most_p = p(t), most_x = x(t);
    const auto inside = [&](double at) { return at > 0 && at < t; };  // (false for NaN)
    if (const double at = -b / (2 * c); inside(at)) most_p = std::max(most_p, p(at));
    // where a + 3 b t + 5 c t^2, the derivative by the singular value, is 0
    const double root = std::sqrt(9 * b * b - 20 * a * c);
    for (const double at : {(-3 * b + root) / (10 * c), (-3 * b - root) / (10 * c), -a / (3 * b)})
      if (inside(at)) most_x = std::max(most_x, x(at));
    to[i].a = shift(1.02 * t);
    to[i].poly = shift(std::max(1.02 * most_p, 2 * (1.5 * std::fabs(b) + 2.25 * std::fabs(c))));
    top = std::min(4.0, 1.01 * most_x);
  }
}

int parts_of(const dn_muon_params& k, dn_dtype p_dt) { return k.parts ? k.parts : p_dt == DN_BF16 ? 1 : 2; }
int64_t half_tiles(int64_t r, int64_t side) {
  const int64_t tiles = (r + side - 1) / side;
  return tiles * (tiles + 1) / 2;
}
// The update's tiles: 256 x 256, or 64 rows x 128 columns, of which three workgroups share a CU (one of 512 x 512 in two parts 231 us a
// step, with tiles of 128 x 128 251; 1000 x 1000 391 and 431).
enum Update { U256, U64 };
int64_t update_tiles(Update u, int64_t rows, int64_t cols) {
  const int64_t m = u == U256 ? 256 : 128, n = u == U256 ? 256 : 64;
  return (rows + n - 1) / n * ((cols + m - 1) / m);
}

// The time of a launch of `jobs` tiles of `stages` of 64 k in us, by what launches of many shapes took: a stage of 256 x 256 takes
// 1.25 us on an idle chip and 1.75 on a full one, of 128 x 128 0.62 alone on a CU and 1.15 for two, of 128 x 64
// 0.4 and 0.8 for three.
double launch_us(int T, double jobs, double stages) {
  if (T == 256) return std::ceil(jobs / 256) * (stages * (1.25 + 0.5 * std::min(1.0, jobs / 256)) + 8);
  if (T == 64) return std::ceil(jobs / 768) * (stages * (0.4 + 0.4 * std::min(1.0, jobs / 768)) + 5);
  if (jobs <= 256) return stages * (0.62 + 0.25 * jobs / 256) + 5;
  return std::ceil(jobs / 512) * (stages * 1.15 + 6);
}
struct Tiling {
  int T, splits;
};
// Of products of half the tiles of r x r over `stages`: tiles and splits with the least time.  Splits cost the slabs' way through
// memory and a launch more.
Tiling choose(const dn_muon_tensor* ts, int count, int products, bool square) {
  Tiling best{128, 1};
  double least = 1e300;
  for (const int T : {256, 128})
    for (int s = 1; s <= 16; ++s) {
      double jobs = 0, stages = 0, area = 0;
      for (int i = 0; i < count; ++i) {
        const int64_t r = std::min(ts[i].rows, ts[i].cols), k = square ? r : std::max(ts[i].rows, ts[i].cols);
        jobs += (double)half_tiles(r, T) * s, area += (double)half_tiles(r, T) * T * T;
        stages = std::max(stages, (double)((k + BK - 1) / BK * products));
      }
      if (s > 1 && stages / s < 4) break;
      const double us = launch_us(T, jobs, std::ceil(stages / s)) + (s > 1 ? 5 + s * area * 8 / 6e6 : 0);
      if (us < least * 0.999) least = us, best = Tiling{T, s};
    }
  return best;
}

// A group of matrices that share launches, laid out in the workspace.
struct Group {
  MuonLaunch l;
  Tiling gram, square;
  Update update;
  size_t total;
};
void plan_group(const dn_muon_tensor* ts, int count, int parts, Group& gr) {
  gr.l = MuonLaunch{};
  Work w;
  const int products = parts == 2 ? 3 : 1;
  gr.gram = choose(ts, count, products, false), gr.square = choose(ts, count, products, true);
  double least = 1e300;
  for (const Update u : {U256, U64}) {
    double jobs = 0, stages = 0;
    for (int i = 0; i < count; ++i) {
      jobs += (double)update_tiles(u, ts[i].rows, ts[i].cols);
      stages = std::max(stages, (double)((std::min(ts[i].rows, ts[i].cols) + BK - 1) / BK * products));
    }
    const double us = launch_us(u == U256 ? 256 : 64, jobs, stages);
    if (us < least) least = us, gr.update = u;
  }
  int32_t sums = 0;
  for (int i = 0; i < count; ++i) {
    Mat& t = gr.l.t[i];
    t.g = ts[i].g, t.m = ts[i].m, t.p = ts[i].p, t.copy = ts[i].copy;
    t.rows = (int32_t)ts[i].rows, t.cols = (int32_t)ts[i].cols, t.rate = (float)ts[i].rate;
    const int64_t r = std::min(t.rows, t.cols);
    for (int b = 0; b < 2; ++b) t.x[b] = w.take((size_t)parts * t.rows * up8(t.cols) * 2);
    t.a = w.take((size_t)parts * r * up8((int32_t)r) * 2), t.poly = w.take((size_t)parts * r * up8((int32_t)r) * 2);
    size_t slab = 0;
    for (const Tiling& k : {gr.gram, gr.square})
      if (k.splits > 1) slab = std::max(slab, (size_t)k.splits * r * up(r, k.T) * 4);
    t.slab = w.take(slab);
    t.sums = (int32_t)std::min<int64_t>(SUMS, ((int64_t)t.rows * t.cols + 2047) / 2048);
    t.norm = sums, sums += t.sums;
  }
  gr.l.count = count;
  gr.l.sums = (float*)w.take((size_t)sums * 4);  // (an offset: the workspace's address is added)
  gr.total = w.total;
}

// A launch of all matrices, each with `units` workgroups.
template <typename Units>
int64_t spread(MuonLaunch& l, Units&& units) {
  int64_t total = 0;
  for (int i = 0; i < l.count; ++i) {
    l.t[i].first = (int32_t)total;
    total += units(l.t[i]);
  }
  return total;
}

template <bool SQUARE, int PARTS>
int run_gram(MuonLaunch& l, const Tiling& k, hipStream_t st) {
  const auto side = [](const Mat& t) { return std::min(t.rows, t.cols); };
  const dim3 grid((unsigned)spread(l, [&](Mat& t) { return t.splits = k.splits, half_tiles(side(t), k.T) * k.splits; }));
  if (k.splits == 1) {
    if (k.T == 256) gram_kernel<SQUARE, PARTS, 256, false><<<grid, 512, 0, st>>>(l);
    else gram_kernel<SQUARE, PARTS, 128, false><<<grid, 256, 0, st>>>(l);
    return (int)hipGetLastError();
  }
  if (k.T == 256) gram_kernel<SQUARE, PARTS, 256, true><<<grid, 512, 0, st>>>(l);
  else gram_kernel<SQUARE, PARTS, 128, true><<<grid, 256, 0, st>>>(l);
  if (const int err = (int)hipGetLastError()) return err;
  const dim3 blocks((unsigned)spread(l, [&](Mat& t) { return half_tiles(side(t), 64); }));
  if (k.T == 256) mirror_kernel<SQUARE, PARTS, 256><<<blocks, 1024, 0, st>>>(l);
  else mirror_kernel<SQUARE, PARTS, 128><<<blocks, 1024, 0, st>>>(l);
  return (int)hipGetLastError();
}
template <int PARTS, bool LAST, typename P, typename O>
int run_update(MuonLaunch& l, Update u, hipStream_t st) {
  const dim3 grid((unsigned)spread(l, [&](const Mat& t) { return update_tiles(u, t.rows, t.cols); }));
  if (u == U256) update_kernel<PARTS, 256, 256, LAST, P, O><<<grid, 512, 0, st>>>(l);
  else update_kernel<PARTS, 128, 64, LAST, P, O><<<grid, 256, 0, st>>>(l);
  return (int)hipGetLastError();
}

template <int PARTS>
int run_group(Group& gr, const dn_muon_params& k, dn_dtype p_dt, dn_dtype g_dt, dn_dtype copy_dt, hipStream_t st) {
  MuonLaunch& l = gr.l;
  int err = with_type(g_dt, [&](auto g) {
    const int64_t n = spread(l, [](const Mat& t) { return (int64_t)t.sums; });
    momentum_kernel<decltype(g)><<<dim3((unsigned)n), 256, 0, st>>>(l);
    return (int)hipGetLastError();
  });
  if (err) return err;
  err = with_type(g_dt, [&](auto g) {
    const int64_t n = spread(l, [](const Mat& t) { return ((int64_t)t.rows * (up8(t.cols) / 8) + 1023) / 1024; });
    start_kernel<decltype(g), PARTS><<<dim3((unsigned)n), 256, 0, st>>>(l);
    return (int)hipGetLastError();
  });
  StepShifts shifts[DN_MAX_NS_STEPS];
  steps_of(k, shifts);
  for (int s = 0; s < k.steps && !err; ++s) {
    l.a = (float)k.coefficients[s][0], l.b = (float)k.coefficients[s][1], l.c = (float)k.coefficients[s][2];
    l.a_shift = shifts[s].a, l.poly_shift = shifts[s].poly;
    l.from = s & 1;
    if ((err = run_gram<false, PARTS>(l, gr.gram, st)) || (err = run_gram<true, PARTS>(l, gr.square, st))) return err;
    err = s + 1 < k.steps ? run_update<PARTS, false, float, __bf16>(l, gr.update, st) : with_type(p_dt, [&](auto p) {
      using P = decltype(p);
      return copy_dt == DN_F16 ? run_update<PARTS, true, P, _Float16>(l, gr.update, st) : run_update<PARTS, true, P, __bf16>(l, gr.update, st);
    });
  }
  return err;
}

// Whether a matrix is a workgroup's own.
bool is_small(const dn_muon_tensor& t, int parts) { return small_bytes(t.rows, t.cols, parts) <= SMALL_LDS; }

template <int PARTS>
int run_small(const dn_muon_tensor* const* ts, int count, const dn_muon_params& k, dn_dtype p_dt, dn_dtype g_dt, dn_dtype copy_dt,
              hipStream_t st) {
  SmallLaunch l{};
  l.beta = (float)k.momentum, l.grad_scale = (float)k.grad_scale, l.eps = (float)k.eps, l.lr = (float)k.lr;
  l.decay = (float)(1 - k.lr * k.weight_decay), l.nesterov = k.nesterov, l.steps = k.steps;
  StepShifts shifts[DN_MAX_NS_STEPS];
  steps_of(k, shifts);
  for (int s = 0; s < k.steps; ++s) {
    for (int j = 0; j < 3; ++j) l.coef[s][j] = (float)k.coefficients[s][j];
    l.a_shift[s] = shifts[s].a, l.poly_shift[s] = shifts[s].poly;
  }
  int64_t bytes = 0;
  for (int i = 0; i < count; ++i) {
    const dn_muon_tensor& t = *ts[i];
    l.t[i] = SmallMat{t.g, t.m, t.p, t.copy, (int32_t)t.rows, (int32_t)t.cols, (float)t.rate};
    bytes = std::max(bytes, small_bytes(t.rows, t.cols, PARTS));
  }
  return with_type(p_dt, [&](auto p) {
    return with_type(g_dt, [&](auto g) {
      const auto go = [&](auto o) {
        const auto kernel = small_kernel<PARTS, decltype(p), decltype(g), decltype(o)>;
        // (more than 64 KB has to be asked for, each time: which device this is may change)
        if (const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, SMALL_LDS)) return (int)e;
        kernel<<<dim3((unsigned)count), 64 * SMALL_WAVES, (size_t)bytes, st>>>(l);
        return (int)hipGetLastError();
      };
      return copy_dt == DN_F16 ? go(_Float16{}) : go(__bf16{});
    });
  });
}

}  // namespace

size_t muon_bytes(const dn_muon_tensor* tensors, int32_t count, dn_dtype p_dt, const dn_muon_params& k) {
  size_t most = DN_NO_WORKSPACE;  // (a group's is more: it has five pieces of 256 bytes at least)
  Group gr;
  const int parts = parts_of(k, p_dt);
  dn_muon_tensor large[MATS];
  int held = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (!is_small(tensors[i], parts)) large[held++] = tensors[i];
    if (held == MATS || (i + 1 == count && held)) {
      plan_group(large, held, parts, gr);
      most = std::max(most, gr.total), held = 0;
    }
  }
  return most;
}

int launch_muon(const dn_muon_tensor* tensors, int32_t count, dn_dtype p_dt, dn_dtype g_dt, dn_dtype copy_dt, const dn_muon_params& k,
                void* d_work, void* stream) {
  const int parts = parts_of(k, p_dt);
  const hipStream_t st = (hipStream_t)stream;
  const dn_muon_tensor* small[SMALL_MATS];
  dn_muon_tensor large[MATS];
  int n_small = 0, n_large = 0;
  for (int32_t i = 0; i < count; ++i) {  // groups share the workspace: the stream keeps them apart
    if (is_small(tensors[i], parts)) small[n_small++] = &tensors[i];
    else large[n_large++] = tensors[i];
    const bool end = i + 1 == count;
    if (n_small == SMALL_MATS || (end && n_small)) {
      const int err = parts == 2 ? run_small<2>(small, n_small, k, p_dt, g_dt, copy_dt, st) : run_small<1>(small, n_small, k, p_dt, g_dt, copy_dt, st);
      if (err) return err;
      n_small = 0;
    }
    if (n_large == MATS || (end && n_large)) {
      Group gr;
      plan_group(large, n_large, parts, gr);
      gr.l.work = (char*)d_work;
      gr.l.sums = (float*)((char*)d_work + (size_t)gr.l.sums);
      gr.l.beta = (float)k.momentum, gr.l.grad_scale = (float)k.grad_scale, gr.l.eps = (float)k.eps, gr.l.lr = (float)k.lr;
      gr.l.decay = (float)(1 - k.lr * k.weight_decay), gr.l.nesterov = k.nesterov;
      const int err = parts == 2 ? run_group<2>(gr, k, p_dt, g_dt, copy_dt, st) : run_group<1>(gr, k, p_dt, g_dt, copy_dt, st);
      if (err) return err;
      n_large = 0;
    }
  }
  return 0;
}

}  // namespace head
}  // namespace dn
