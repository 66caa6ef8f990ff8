// Rows in 8 bits with a scale for every block of 128, and matrix products of such operands.
//   quantize: scale = max |x| / 448 over a block (128 values of a row, or a square of 128 x 128), code = e4m3(x / scale), along
//     the rows, and turned ([C][n], blocks along n) from the same reading
//   product: y_nv = sum over blocks b of a_scale[n][b] w_scale[v / 128][b] (sum over c in b of a_nc w_vc)
// Quantising is bound by memory: a tile of 128 x 128 stays in registers, and its turned codes leave through LDS in whole lines.
// A product's block of 128 is two MFMAs of 64 k into fresh registers (the matrix cores' 8-bit rate is twice that of 16 bits),
// whose 32-bit sums are multiplied by both scales and added to the result's: 16 multiply-adds for 128 cycles of MFMA.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "tiles.h"

namespace dn {
namespace head {
namespace {

constexpr int B = DN_SCALE_BLOCK;  // 128
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------------------------------------------------------------
// Quantising.  A workgroup takes a tile of 128 x 128; thread t holds 8 rows from 8 (t / 16) on of 8 columns from 8 (t % 16) on.
// ---------------------------------------------------------------------------------------------------------------------
// 448 / top, and 0 for a block of zeros or of values below 1.4e-36, whose reciprocal is past fp32's range.
__device__ inline float inverse(float top) { return top > 1.4e-36f ? 448.f / top : 0.f; }

template <typename T, bool SQUARE, bool TURNED>
__global__ __launch_bounds__(256) void quantize_kernel(QuantArgs a) {
  __shared__ __align__(16) uint8_t s_tile[TURNED ? B * B : 16];
  __shared__ float s_top[4][TURNED && !SQUARE ? B : 1];
  const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4;
  const int blocks_c = (a.C + B - 1) / B;
  const int64_t blocks_n = (a.n + B - 1) / B;
  const int64_t br = blockIdx.x / blocks_c;
  const int bc = (int)(blockIdx.x - br * blocks_c);
  const int64_t r0 = br * B;
  const int c0 = bc * B, c = c0 + 8 * cg;
  const int rows = (int)std::min<int64_t>(B, a.n - r0);  // of the tile
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = 8 * rg + i;
    if (r < rows && c < a.C) {
      load8((const T*)a.x + (r0 + r) * a.x_stride, c, a.C, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
  }
  float row_top[8], col_top[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) row_top[j] = col_top[j] = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // an infinity is stored as a NaN; neither counts for a maximum
      v[i][j] = fabsf(v[i][j]) < INFINITY ? v[i][j] : __uint_as_float(0x7fc00000u);
      row_top[i] = fmaxf(row_top[i], fabsf(v[i][j]));
      if (TURNED && !SQUARE) col_top[j] = fmaxf(col_top[j], fabsf(v[i][j]));
    }
  float inv[8];  // of the thread's rows
  if constexpr (SQUARE) {
    float top = row_top[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, row_top[i]);
    top = lanes_max<64>(top);
    if ((tid & 63) == 0) s_top[tid >> 6][0] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_top[0][0], s_top[1][0]), fmaxf(s_top[2][0], s_top[3][0]));
    if (tid == 0) {
      if (a.codes) a.scale[br * blocks_c + bc] = top * (1.f / 448.f);
      if (TURNED) a.turned_scale[bc * blocks_n + br] = top * (1.f / 448.f);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) inv[i] = inverse(top);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float top = lanes_max<16>(row_top[i]);
      inv[i] = inverse(top);
      if (a.codes && cg == 0 && 8 * rg + i < rows) a.scale[(r0 + 8 * rg + i) * blocks_c + bc] = top * (1.f / 448.f);
    }
  }
  if (a.codes)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = v[i][j] * inv[i];
      if (8 * rg + i < rows && c < a.C) store8((F8*)a.codes + (r0 + 8 * rg + i) * a.codes_stride, c, a.C, q);
    }
  if constexpr (TURNED) {
    float cinv[8];  // of the thread's columns
    if constexpr (SQUARE) {
#pragma unroll
      for (int j = 0; j < 8; ++j) cinv[j] = inv[0];
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        col_top[j] = fmaxf(col_top[j], __shfl_xor(col_top[j], 16));
        col_top[j] = fmaxf(col_top[j], __shfl_xor(col_top[j], 32));
        if ((tid & 48) == 0) s_top[tid >> 6][8 * cg + j] = col_top[j];
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = 8 * cg + j;
        const float top = fmaxf(fmaxf(s_top[0][k], s_top[1][k]), fmaxf(s_top[2][k], s_top[3][k]));
        cinv[j] = inverse(top);
        if (rg == 0 && c + j < a.C) a.turned_scale[(int64_t)(c + j) * blocks_n + br] = top * (1.f / 448.f);
      }
    }
    // Column k's 128 rows lie in 8 pieces of 16, piece s at place s ^ k / 8 % 8: a wave's writes spread over the banks.
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float q[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = v[i][j] * cinv[j];
      uint32_t w[2];
      f8_pack(q, w);
      *(uint2*)(s_tile + (8 * cg + j) * B + (((rg >> 1) ^ (cg & 7)) * 16 + (rg & 1) * 8)) = make_uint2(w[0], w[1]);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int col = (tid + 256 * k) >> 3, s = tid & 7;
      if (c0 + col >= a.C) break;
      const u32x4 w = *(const u32x4*)(s_tile + col * B + ((s ^ (col >> 3 & 7)) * 16));
      uint8_t* to = a.turned + (int64_t)(c0 + col) * a.turned_stride + r0 + 16 * s;
      if (16 * s + 16 <= rows) {
        *(u32x4_any*)to = w;
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (16 * s + e < rows) to[e] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Products.  D[m][n] = y[n][m]: M runs over w's rows, N over a's, so that a lane's results are neighbours in a row of y.
// ---------------------------------------------------------------------------------------------------------------------
struct P8Args {
  const uint8_t *w, *a;
  int64_t ldw, lda;
  const float *w_scale, *a_scale;
  int32_t M, N, K, blocks;  // blocks: of K, the scales' row length
  int32_t tiles_m, tiles_n, splits;
  void* out;  // [N][ldo]; a split's sums in fp32 at out + split * out_split
  int64_t ldo, out_split;
};

// A tile of R rows x 128 codes in LDS, loaded straight from memory in 16-byte slots; slot s of row r at place s ^ (r / 2) % 8
// (16 consecutive rows' reads of one slot meet 16 different places modulo 256 bytes).
template <int R, int NW>
struct Codes {
  static constexpr int BYTES = R * B, PIECES = BYTES / 1024, PER = PIECES / NW;
  static_assert(PIECES % NW == 0 && NW % 2 == 0, "whole pieces per wave");
  uint32_t voff[PER];
  const uint8_t* base;
  int place;  // first k of this lane's slot: the same in each piece, since those are 8 rows each and NW is even
  __device__ inline void init(const uint8_t* p, int64_t ld, int row0, int rows, int wave, int lane) {
    base = p + (int64_t)row0 * ld;
    const int line = lane >> 3;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int row = (wave + i * NW) * 8 + line, s = (lane & 7) ^ ((row >> 1) & 7);
      voff[i] = row0 + row < rows ? (uint32_t)(row * ld + s * 16) : OOB;
      place = s * 16;
    }
  }
  __device__ inline void load(char* lds, int k0, int K, int wave, int lane) const {
    const __amdgpu_buffer_rsrc_t rsrc = uniform_rsrc(base, 0x7fffffffu);
    if (k0 + B <= K) {
#pragma unroll
      for (int i = 0; i < PER; ++i) direct16(rsrc, lds + (wave + i * NW) * 1024, voff[i], (uint32_t)k0);
      return;
    }
    const int k = k0 + place;
#pragma unroll
    for (int i = 0; i < PER; ++i) direct16(rsrc, lds + (wave + i * NW) * 1024, k + 16 <= K ? voff[i] : OOB, (uint32_t)k0);
    if (K & 15) {  // the slot that the row ends in, a code at a time: what lies behind it may be anything
      wait_loads<0>();
#pragma unroll 1
      for (int i = 0; i < PER; ++i) {
        if (k >= K || k + 16 <= K || voff[i] == OOB) continue;
        u32x4 v{};
#pragma unroll
        for (int e = 0; e < 15; ++e)
          if (k + e < K) v[e / 4] |= (uint32_t)base[(int64_t)voff[i] + k0 + e] << (8 * (e % 4));
        *(u32x4*)(lds + (wave + i * NW) * 1024 + lane * 16) = v;
      }
    }
  }
};

// The fragments of 32 rows from row r0 on: a lane's 64 codes of row lane % 32, for two MFMAs of 64 k.
struct Frag {
  i32x8 k[2];
};
__device__ inline void read_frag(const char* lds, int r0, int lane, Frag& f) {
  const int row = r0 + (lane & 31), half = lane >> 5;
  const char* p = lds + row * B;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const i32x4 lo = *(const i32x4*)(p + (((4 * h + 2 * half) ^ ((row >> 1) & 7)) * 16));
    const i32x4 hi = *(const i32x4*)(p + (((4 * h + 2 * half + 1) ^ ((row >> 1) & 7)) * 16));
    f.k[h] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}
// Codes 8 j .. + 7 of a lane's 32 as fp16.
__device__ inline f16x8 halves(const i32x8& k, int j) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(k[2 * j], 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(k[2 * j], 1.f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(k[2 * j + 1], 1.f, false),
              d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(k[2 * j + 1], 1.f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Sums of a block's 128 products.  The 8-bit MFMAs add the products of eight k with those bits only that lie within 2^-13 of the
// largest one's leading bit, the rest cut off (found by products of powers of two; other lengths are added in full): for results
// in 16 bits.  EXACT: codes become fp16, which they fit, for MFMAs that keep 24 bits, at half the rate: for results in fp32.
template <bool EXACT>
__device__ inline f32x16 block_sum(const Frag& a, const Frag& b) {
  f32x16 v{};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (EXACT) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v = Mfma<_Float16>::mma(halves(a.k[h], j), halves(b.k[h], j), v);
    } else {
      v = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a.k[h], b.k[h], v, 0, 0, 0, 0, 0, 0);
    }
  }
  return v;
}

// Waves: WM x WN, each (BM / WM) x (BN / WN).  NST: stages of 128 k held in LDS.  SLAB: sums in fp32, a slab a split.
template <int BM, int BN, int WM, int WN, int NST, typename O, bool SLAB, bool EXACT>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(P8Args g) {
  constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
  using OW = Codes<BM, NW>;
  using OA = Codes<BN, NW>;
  constexpr int STAGE = OW::BYTES + OA::BYTES, PER = OW::PER + OA::PER;
  constexpr int WROWS = BN / WN, WCOLS = BM / WM;
  using S = std::conditional_t<SLAB, float, O>;
  constexpr int OUT_ROW = WCOLS * (int)sizeof(S) + 16, OUT_BYTES = NW * 32 * OUT_ROW;
  constexpr int LDS = NST * STAGE > OUT_BYTES ? NST * STAGE : OUT_BYTES;
  __shared__ __align__(1024) char s_mem[LDS];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM, l32 = lane & 31, half = lane >> 5;
  // each XCD takes a contiguous range of (split, tile), tiles ordered as columns of COL along n, which share their operands in
  // its L2
  constexpr int COL = 6;
  const int all = gridDim.x, xcd = blockIdx.x % 8, per = all / 8, rem = all % 8;
  const int job = xcd * per + min(xcd, rem) + blockIdx.x / 8, nt = g.tiles_m * g.tiles_n, split = job / nt, id = job - split * nt;
  const int col = id / (COL * g.tiles_m), width = min(COL, g.tiles_n - col * COL), in = id - col * COL * g.tiles_m;
  const int tile_m = in / width, tile_n = col * COL + in % width;
  const int m0 = tile_m * BM, n0 = tile_n * BN;

  OW ow;
  OA oa;
  ow.init(g.w, g.ldw, m0, g.M, wave, lane);
  oa.init(g.a, g.lda, n0, g.N, wave, lane);
  const int s0 = (int)((int64_t)g.blocks * split / g.splits), s1 = (int)((int64_t)g.blocks * (split + 1) / g.splits);
  auto load = [&](int s, int buf) {
    char* at = s_mem + buf * STAGE;
    ow.load(at, s * B, g.K, wave, lane);
    oa.load(at + OW::BYTES, s * B, g.K, wave, lane);
  };
  // The scales: of the wave's rows of w one (its rows lie in one block of 128), of a one for each of a lane's rows.
  static_assert(WCOLS <= B && B % WCOLS == 0, "a wave's rows of w share their scales");
  const float* ws = g.w_scale + (int64_t)(std::min(m0 + wm * WCOLS, g.M - 1) / B) * g.blocks;
  const float* as[TN];
#pragma unroll
  for (int t = 0; t < TN; ++t) as[t] = g.a_scale + (int64_t)std::min(n0 + wn * WROWS + 32 * t + l32, g.N - 1) * g.blocks;
  float f[TN], next[TN];
  auto factors = [&](int s, float (&to)[TN]) {
    const float w = ws[s];
#pragma unroll
    for (int t = 0; t < TN; ++t) to[t] = as[t][s] * w;
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int t = 0; t < TN; ++t) acc[i][t] = f32x16{};

  if (s1 > s0) {
#pragma unroll
    for (int i = 0; i < NST; ++i)
      if (s0 + i < s1) load(s0 + i, i);
    factors(s0, f);
    int buf = 0;
    for (int s = s0; s < s1; ++s) {
      wait_loads<0>();
      wave_barrier();
      if (s + 1 < s1) factors(s + 1, next);
      const char* at = s_mem + buf * STAGE;
      Frag b[TN];
#pragma unroll
      for (int t = 0; t < TN; ++t) read_frag(at + OW::BYTES, wn * WROWS + 32 * t, lane, b[t]);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        Frag a;
        read_frag(at, wm * WCOLS + 32 * i, lane, a);
#pragma unroll
        for (int t = 0; t < TN; ++t) {
          const f32x16 v = block_sum<EXACT>(a, b[t]);
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][t][r] = __builtin_fmaf(v[r], f[t], acc[i][t][r]);
        }
      }
      wait_lds();
      wave_barrier();
      if (s + NST < s1) load(s + NST, buf);
#pragma unroll
      for (int t = 0; t < TN; ++t) f[t] = next[t];
      buf = buf + 1 == NST ? 0 : buf + 1;
    }
  }
  (void)PER;

  // Element r of acc[i][t]: m = m0 + wm WCOLS + 32 i + 8 (r / 4) + 4 half + r % 4, n = n0 + wn WROWS + 32 t + l32.  Results leave
  // through LDS, whole pieces of rows at a time.
  constexpr int EV = 16 / (int)sizeof(S), LANES = WCOLS / EV, LINES = 64 / LANES;
  typedef S v4 __attribute__((ext_vector_type(4)));
  typedef S vec __attribute__((ext_vector_type(EV)));
  typedef S vec_any __attribute__((ext_vector_type(EV), aligned(sizeof(S))));
  __syncthreads();
  char* stg = s_mem + wave * 32 * OUT_ROW;
  S* out = (S*)g.out + (SLAB ? split * g.out_split : 0);
#pragma unroll
  for (int t = 0; t < TN; ++t) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (S)acc[i][t][4 * q + e];
        *(v4*)(stg + l32 * OUT_ROW + (32 * i + 8 * q + 4 * half) * (int)sizeof(S)) = v;
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int c = (lane % LANES) * EV, m = m0 + wm * WCOLS + c;
#pragma unroll
    for (int k = 0; k < 32 / LINES; ++k) {
      const int line = k * LINES + lane / LANES, n = n0 + wn * WROWS + 32 * t + line;
      const vec v = *(const vec*)(stg + line * OUT_ROW + c * (int)sizeof(S));
      if (n >= g.N) continue;
      S* dst = out + (int64_t)n * g.ldo + m;
      if (SLAB || m + EV <= g.M) {  // (a slab's rows are padded to whole tiles)
        *(vec_any*)dst = v;
      } else {
#pragma unroll
        for (int e = 0; e < EV; ++e)
          if (m + e < g.M) dst[e] = v[e];
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// y = sum of the splits' slabs, rounded.
template <typename O>
__global__ __launch_bounds__(256) void join_splits_kernel(const float* __restrict__ slab, int64_t ld, int64_t stride, int splits,
                                                          int64_t rows, int C, O* __restrict__ out, int64_t ldo) {
  const int per = (C + 7) / 8;
  const int64_t total = rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per;
    const int c = (int)(i - row * per) * 8;
    float v[8] = {};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
      float w[8];
      load8(slab + s * stride + row * ld + c, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += w[j];
    }
    store8(out + row * ldo, c, C, v);
  }
}

// Codes at any address in rows of ldo (a multiple of 16), zeros past column C.
__global__ __launch_bounds__(256) void align_kernel(const uint8_t* __restrict__ in, int64_t ld, int64_t rows, int C,
                                                    uint8_t* __restrict__ out, int64_t ldo) {
  const int64_t per = ldo / 16, total = rows * per;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
    const int64_t row = u / per;
    const int c = (int)(u - row * per) * 16;
    const uint8_t* p = in + row * ld + c;
    u32x4 v{};
    if (c + 16 <= C) {
      v = *(const u32x4_any*)p;
    } else {
#pragma unroll
      for (int e = 0; e < 15; ++e)
        if (c + e < C) v[e / 4] |= (uint32_t)p[e] << (8 * (e % 4));
    }
    *(u32x4*)(out + row * ldo + c) = v;
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

enum Tile { T256, T128, T64, T32 };
int tile_m(Tile t) { return t == T256 ? 256 : 128; }
int tile_n(Tile t) { return t == T256 ? 256 : t == T128 ? 128 : t == T64 ? 64 : 32; }

struct Plan8 {
  Tile tile;
  int splits;
  bool copy_a, copy_w;
  int64_t ld, slab_ld;  // ld: of the copies
  size_t a_at, w_at, slab_at, total;
};
bool lies_well(const void* p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 16 == 0 && ld <= MAX_LD; }
Plan8 plan_product(const ProductArgs& a) {
  Plan8 p{};
  Work w;
  p.tile = a.n <= 32 ? T32 : a.n <= 64 ? T64 : T128;
  const int64_t tiles = (up(a.V, tile_m(p.tile)) / tile_m(p.tile)) * (up(a.n, tile_n(p.tile)) / tile_n(p.tile));
  const int64_t blocks = (a.C + B - 1) / B;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({512 / tiles, blocks / 4, 64}));
  p.copy_a = !lies_well(a.a, a.a_stride), p.copy_w = !lies_well(a.w, a.w_stride);
  p.ld = up(a.C, 16);
  if (p.copy_a) p.a_at = w.take((size_t)a.n * p.ld);
  if (p.copy_w) p.w_at = w.take((size_t)a.V * p.ld);
  p.slab_ld = up(a.V, 256);
  if (p.splits > 1) p.slab_at = w.take((size_t)p.splits * a.n * p.slab_ld * 4);
  p.total = w.total;
  return p;
}

template <int BM, int BN, int WM, int WN, int NST, typename O, bool SLAB, bool EXACT>
int run_product(P8Args& g, hipStream_t st) {
  g.tiles_m = (g.M + BM - 1) / BM, g.tiles_n = (g.N + BN - 1) / BN;
  product_kernel<BM, BN, WM, WN, NST, O, SLAB, EXACT>
      <<<dim3((unsigned)(g.tiles_m * g.tiles_n * g.splits)), 64 * WM * WN, 0, st>>>(g);
  return (int)hipGetLastError();
}
template <typename O, bool SLAB, bool EXACT>
int run_tile(Tile t, P8Args& g, hipStream_t st) {
  if (t == T32) return run_product<128, 32, 4, 1, 4, O, SLAB, EXACT>(g, st);
  if (t == T64) return run_product<128, 64, 2, 2, 3, O, SLAB, EXACT>(g, st);
  return run_product<128, 128, 2, 2, 2, O, SLAB, EXACT>(g, st);
}

int align(const uint8_t* in, int64_t ld, int64_t rows, int C, uint8_t* out, int64_t ldo, hipStream_t st) {
  const unsigned grid = (unsigned)std::min<int64_t>((rows * (ldo / 16) + 255) / 256, 8192);
  align_kernel<<<grid, 256, 0, st>>>(in, ld, rows, C, out, ldo);
  return (int)hipGetLastError();
}

}  // namespace

int launch_quantize_blocks(const QuantArgs& a, dn_dtype dt, void* stream) {
  const dim3 grid((unsigned)(((a.n + B - 1) / B) * ((a.C + B - 1) / B)));
  const hipStream_t st = (hipStream_t)stream;
  return with_type(dt, [&](auto v) {
    using T = decltype(v);
    if (a.rows > 1) {
      if (a.turned) quantize_kernel<T, true, true><<<grid, 256, 0, st>>>(a);
      else quantize_kernel<T, true, false><<<grid, 256, 0, st>>>(a);
    } else {
      if (a.turned) quantize_kernel<T, false, true><<<grid, 256, 0, st>>>(a);
      else quantize_kernel<T, false, false><<<grid, 256, 0, st>>>(a);
    }
    return (int)hipGetLastError();
  });
}

size_t block_product_bytes(const ProductArgs& a) { return plan_product(a).total; }

int launch_block_product(const ProductArgs& a, dn_dtype dt, void* d_work, void* stream) {
  const Plan8 p = plan_product(a);
  const hipStream_t st = (hipStream_t)stream;
  char* work = (char*)d_work;
  P8Args g{};
  g.a = a.a, g.lda = a.a_stride, g.w = a.w, g.ldw = a.w_stride, g.a_scale = a.a_scale, g.w_scale = a.w_scale;
  g.M = a.V, g.N = (int)a.n, g.K = a.C, g.blocks = (a.C + B - 1) / B, g.splits = p.splits;
  int err;
  if (p.copy_a) {
    if ((err = align(a.a, a.a_stride, a.n, a.C, (uint8_t*)work + p.a_at, p.ld, st))) return err;
    g.a = (uint8_t*)work + p.a_at, g.lda = p.ld;
  }
  if (p.copy_w) {
    if ((err = align(a.w, a.w_stride, a.V, a.C, (uint8_t*)work + p.w_at, p.ld, st))) return err;
    g.w = (uint8_t*)work + p.w_at, g.ldw = p.ld;
  }
  if (p.splits == 1) {
    g.out = a.y, g.ldo = a.y_stride;
    return with_type(dt, [&](auto v) {
      using O = decltype(v);
      return run_tile<O, false, std::is_same<O, float>::value>(p.tile, g, st);
    });
  }
  g.out = work + p.slab_at, g.ldo = p.slab_ld, g.out_split = a.n * p.slab_ld;
  if ((err = dt == DN_F32 ? run_tile<float, true, true>(p.tile, g, st) : run_tile<float, true, false>(p.tile, g, st))) return err;
  return with_type(dt, [&](auto v) {
    const unsigned grid = (unsigned)std::min<int64_t>((a.n * ((a.V + 7) / 8) + 255) / 256, 8192);
    join_splits_kernel<<<grid, 256, 0, st>>>((const float*)g.out, p.slab_ld, g.out_split, p.splits, a.n, a.V, (decltype(v)*)a.y,
                                             a.y_stride);
    return (int)hipGetLastError();
  });
}

}  // namespace head
}  // namespace dn
