// Softmax cross entropy of rows h [n][C] over a large vocabulary w [V][C], and its gradient, without keeping the logits.
//   l_nv = h_n . w_v;  lse_n = log sum_v exp l_nv;  loss_n = lse_n - l_n,label(n)
//   g_nv = c_n (exp(l_nv - lse_n) - [v = label(n)]);  dh = g w;  dw = g^T h
// The forward pass is one matrix product whose tiles end in a maximum and a sum of exponentials per row; a second launch
// joins the tiles.  The gradient goes over the vocabulary in pieces: a piece's logits are computed again and leave as g in
// 16 bits, and two more products take dh and dw from it: 6 n V C operations, the least without the logits.
// 16-bit types: products on the matrix cores, 32-bit sums.  fp32, by what the product can take:
//  logits: rows as two fp16 parts, x 2^k = a + b with 2^k such that the row's largest value lies in [2^13, 2^14), and three
//    products a a' + a b' + b a'.  a and b hold 22 bits of a value down to 2^-16 of the row's largest (half of b's smallest
//    step is 2^-25, 2^-38 of the largest); what is left out is at most 2^-22 of a product and of either sign, as an fp32
//    product's and sum's roundings.  The row factors are powers of two (a word with infinities: see split_rows_kernel).
//  dh, dw: the sums run across rows, which have no common factor: three bf16 parts of every value (h, w, g) and six products,
//    as the library's fp32 convolutions.
//  up to 64 rows, or 64 words: bound by reading w, or h, which fp32 MFMAs keep up with: all products on the values as they lie.
// Rows whose label lies outside [0, V) are masked: loss and lse 0, g and dh 0, and what their h holds reaches nothing.
//
// Why this split: the forward pass is the product alone, and its tiles' statistics (8 bytes a row and tile) are what two tiles
// have to tell each other.  The gradient needs lse before g, so the logits are computed again: a third of its operations, where
// keeping them would take 4 n V bytes.  g goes through memory once (2 n V bytes written, 4 n V read) because dh and dw sum it
// over different axes; pieces of 2^29 bytes of it (of 2^27, 28, 29, 30 bytes, 16384 rows over 65536 words took 13.0, 12.5,
// 12.4, 12.3 ms in one version).  Partial sums of splits and pieces have slabs of their own, added in order: no atomics, the
// same bits every time.
// Bound by the matrix cores at the clock that the chip's power allows: the products of 16384 x 16384 x 2048 in bf16 take 998, 898
// and 849 us (1.10, 1.22, 1.29 PFLOP/s; a library's large product 1.38), their MFMA pipes 58 to 68 % busy at 1.89 to 1.84 GHz.
// Gradients of 16384 x 2048 over 65536 words 11.0 ms (1.20 PFLOP/s), 4096 x 2048 over 32000 1.38 ms (1.17), loss of 2000 x 2048
// over 50257 words in fp16 390 us (1.06; 1576 tiles are 6.2 rounds of workgroups), of one row x 4096 over 32000 words 61 us
// (bound by memory: 4.3 TB/s), of 32000 x 9216 over 21 words 109 us (5.4 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "head.h"

namespace dn {
// fp32 fragments: a lane's 16 bytes are four k of its row (k 4 (lane / 32) .. + 3 of eight), which four MFMAs of two k
// take one after the other; A and B agree on the order of k.
template <>
struct Mfma<float> {
  typedef f32x4 frag;
  __device__ static inline f32x16 mma(frag a, frag b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

namespace head {
namespace {

typedef short i16x4 __attribute__((ext_vector_type(4)));
constexpr uint32_t OOB = 0x80000000u;  // a buffer offset past every buffer: reads as 0
constexpr int BK = 64;                 // k of one pipeline stage (of 16-bit values; fp32: 32)
constexpr int64_t MAX_LD = 1 << 22;    // elements between rows: 256 rows stay within 32-bit byte offsets

enum Epilogue { E_STATS, E_GRAD, E_SLAB, E_OUT };

// D[m][n] = sum_k A(m, k) B(n, k).  An operand lies with k along its rows ([m][k], plain) or with k across them ([k][m],
// turned); ld: elements from row to row.  Elements are 16-bit ones; fp32 operands as they lie count two for each.
struct GemmArgs {
  const void *a, *b;
  int64_t lda, ldb, a_part, b_part;  // *_part: elements between the parts of fp32 operands
  int32_t M, N, K;
  int32_t a_rows, b_rows;  // rows of the operand that may be read (turned: columns, a multiple of 8)
  const float *a_factor, *b_factor;  // of the operands' rows (both or none): D[m][n] is multiplied by both
  const int32_t* alt;                // where *alt is not 0, A lies at a_alt
  const void* a_alt;
  int64_t lda_alt;
  int32_t tiles_m, tiles_n, products, splits;
  // E_STATS, E_GRAD: M runs over the vocabulary from v0 on, N over rows
  const int64_t* label;
  int32_t v0, V;
  float2* stats;  // [tiles_m][N]: maximum, in base 2, and sum of exponentials over it
  float* at;      // [N]: the label's logit
  const float *lse, *coef;
  void* g;  // [N][ldg]
  int64_t ldg, g_part;
  // E_SLAB: sums of split s at slab + s slab_stride, [N][slab_ld]; accumulate: added to what is there
  float* slab;
  int64_t slab_ld, slab_stride;
  int32_t accumulate;
  // E_OUT: [N][ldo], times *unscale; rows with row_coef 0 are 0
  void* out;
  int64_t ldo;
  const float *unscale, *row_coef;
};

__device__ inline void direct16(__amdgpu_buffer_rsrc_t rsrc, void* lds, uint32_t voff, uint32_t soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)lds, 16, voff, soff, 0, 0);
}
// Wait until at most N (< 64) vector-memory accesses of this wave are outstanding, and all its LDS accesses are done.
template <int N>
__device__ inline void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
}
// Wait until all LDS accesses of this wave are done.
__device__ inline void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }
__device__ inline void wave_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// One operand's tile of R rows x 64 k (fp32: 32) in LDS, loaded straight from memory in 16-byte slots (a wave instruction
// fills 1 KB).  Plain: rows of 8 slots, slot s of row r at place s ^ (r / 2) % 8, so that 16 consecutive rows' reads of one k
// meet 16 different 16-byte places modulo 256 bytes.  Turned: rows are k, R / 8 slots each (fp32: R / 4), slot s of row k at
// place s ^ 4 (k % 4): the transposing reads take 32 bytes from each of four k at a time; fp32 at s ^ 8 (k / 4 % 2): the halves
// of a wave read 128 bytes each, four k apart.
template <typename T, bool TR, int R, int NW>
struct Operand {
  static constexpr int ES = TR && std::is_same<T, float>::value ? 2 : 1;  // 16-bit elements of a value (plain rows count those)
  static constexpr int BYTES = R * BK * 2, PIECES = BYTES / 1024, PER = PIECES / NW;
  static constexpr int SLOTS = TR ? R * ES / 8 : 8, LINES = 64 / SLOTS;  // slots of an LDS row, LDS rows of a piece
  static_assert(PIECES % NW == 0 && (!TR || SLOTS >= 16), "whole pieces per wave");
  uint32_t voff[PER];
  const char* base;
  int64_t ld;
  int place;  // plain: first k of this lane's slot; turned: this lane's row within a piece

  __device__ inline void init(const void* p, int64_t ld_, int row0, int rows, int wave, int lane) {
    ld = ld_;
    base = (const char*)p + (TR ? (int64_t)row0 * ES : (int64_t)row0 * ld) * 2;
    const int line = lane / SLOTS, slot = lane % SLOTS;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int row = (wave + i * NW) * LINES + line;
      if constexpr (TR) {
        const int s = slot ^ (ES == 2 ? (row & 4) << 1 : (row & 3) << 2);
        voff[i] = row0 * ES + s * 8 < rows ? (uint32_t)(row * ld * 2 + s * 16) : OOB;
      } else {
        const int s = slot ^ ((row >> 1) & 7);
        voff[i] = row0 + row < rows ? (uint32_t)(row * ld * 2 + s * 16) : OOB;
        place = s * 8;  // the same for every i: NW is even, or there is one piece
      }
    }
    if constexpr (TR) place = line;
  }
  __device__ inline void load(char* lds, int64_t part, int k0, int K, int wave) const {
    const char* p = base + part * 2 + (TR ? (int64_t)(k0 / ES) * ld * 2 : 0);
    const __amdgpu_buffer_rsrc_t rsrc = uniform_rsrc(p, 0x7fffffffu);
    const uint32_t soff = TR ? 0 : (uint32_t)k0 * 2;
    if (k0 + BK <= K) {
#pragma unroll
      for (int i = 0; i < PER; ++i) direct16(rsrc, lds + (wave + i * NW) * 1024, voff[i], soff);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int k = k0 + (TR ? ((wave + i * NW) * LINES + place) * ES : place);
        direct16(rsrc, lds + (wave + i * NW) * 1024, k < K ? voff[i] : OOB, soff);
      }
    }
  }
};

// Fragments of NT MFMA tiles (32 rows each) from row r0 of an operand's tile on: a lane's 8 k of row lane % 32.
template <typename T, bool TR, int R, int NT>
struct Fragments {
  typedef typename Mfma<T>::frag frag;
  uint32_t off[TR ? NT : 4];
  __device__ inline void init(int r0, int lane) {
    if constexpr (TR && std::is_same<T, float>::value) {
      const int half = lane >> 5;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int m = r0 + t * 32 + (lane & 31);
        off[t] = 4 * half * (R * 4) + ((m / 4) ^ (half << 3)) * 16 + (m % 4) * 4;
      }
    } else if constexpr (TR) {
      const int q = (lane & 15) >> 2;  // k of the four that this lane's address is in
      const int k = 8 * (lane >> 5) + q;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int slot = (r0 + t * 32) / 8 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
        off[t] = k * (R * 2) + (slot ^ (q << 2)) * 16 + (lane & 1) * 8;
      }
    } else {
      const int row = r0 + (lane & 31);
#pragma unroll
      for (int j = 0; j < 4; ++j) off[j] = row * 128 + (((2 * j + (lane >> 5)) ^ ((row >> 1) & 7)) * 16);
    }
  }
  // Plain, or fp32: the fragments of k-step J.
  template <int J>
  __device__ inline void read_step(const char* lds, frag (&f)[NT]) const {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if constexpr (TR) {
#pragma unroll
        for (int j = 0; j < 4; ++j) f[t][j] = *(const float*)(lds + off[t] + (8 * J + j) * (R * 4));
      } else {
        f[t] = *(const frag*)(lds + off[J] + t * 32 * 128);
      }
    }
  }
  // The fragments of k-steps 2 H and 2 H + 1.  Turned: in one block of assembly with its wait, because the compiler would
  // first wait for every load into LDS that is on its way (it takes the transposing read to depend on them).
  template <int H>
  __device__ inline void read(const char* lds, frag (&f)[2][NT]) const {
    if constexpr (TR && !std::is_same<T, float>::value) {
      constexpr int K0 = H * 32 * (R * 2), ROW4 = 4 * (R * 2);
      const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)lds;
      i16x4 v[2][NT][2];
      if constexpr (NT == 4) {
        asm volatile(
            "ds_read_b64_tr_b16 %0, %16 offset:%20\n ds_read_b64_tr_b16 %1, %16 offset:%21\n"
            "ds_read_b64_tr_b16 %2, %17 offset:%20\n ds_read_b64_tr_b16 %3, %17 offset:%21\n"
            "ds_read_b64_tr_b16 %4, %18 offset:%20\n ds_read_b64_tr_b16 %5, %18 offset:%21\n"
            "ds_read_b64_tr_b16 %6, %19 offset:%20\n ds_read_b64_tr_b16 %7, %19 offset:%21\n"
            "ds_read_b64_tr_b16 %8, %16 offset:%22\n ds_read_b64_tr_b16 %9, %16 offset:%23\n"
            "ds_read_b64_tr_b16 %10, %17 offset:%22\n ds_read_b64_tr_b16 %11, %17 offset:%23\n"
            "ds_read_b64_tr_b16 %12, %18 offset:%22\n ds_read_b64_tr_b16 %13, %18 offset:%23\n"
            "ds_read_b64_tr_b16 %14, %19 offset:%22\n ds_read_b64_tr_b16 %15, %19 offset:%23\n"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(v[0][0][0]), "=&v"(v[0][0][1]), "=&v"(v[0][1][0]), "=&v"(v[0][1][1]), "=&v"(v[0][2][0]), "=&v"(v[0][2][1]),
              "=&v"(v[0][3][0]), "=&v"(v[0][3][1]), "=&v"(v[1][0][0]), "=&v"(v[1][0][1]), "=&v"(v[1][1][0]), "=&v"(v[1][1][1]),
              "=&v"(v[1][2][0]), "=&v"(v[1][2][1]), "=&v"(v[1][3][0]), "=&v"(v[1][3][1])
            : "v"(at + off[0]), "v"(at + off[1]), "v"(at + off[2]), "v"(at + off[3]), "n"(K0), "n"(K0 + ROW4),
              "n"(K0 + 16 * (R * 2)), "n"(K0 + 16 * (R * 2) + ROW4)
            : "memory");
      } else {
        static_assert(NT == 2, "tiles of a wave");
        asm volatile(
            "ds_read_b64_tr_b16 %0, %8 offset:%10\n ds_read_b64_tr_b16 %1, %8 offset:%11\n"
            "ds_read_b64_tr_b16 %2, %9 offset:%10\n ds_read_b64_tr_b16 %3, %9 offset:%11\n"
            "ds_read_b64_tr_b16 %4, %8 offset:%12\n ds_read_b64_tr_b16 %5, %8 offset:%13\n"
            "ds_read_b64_tr_b16 %6, %9 offset:%12\n ds_read_b64_tr_b16 %7, %9 offset:%13\n"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(v[0][0][0]), "=&v"(v[0][0][1]), "=&v"(v[0][1][0]), "=&v"(v[0][1][1]), "=&v"(v[1][0][0]), "=&v"(v[1][0][1]),
              "=&v"(v[1][1][0]), "=&v"(v[1][1][1])
            : "v"(at + off[0]), "v"(at + off[1]), "n"(K0), "n"(K0 + ROW4), "n"(K0 + 16 * (R * 2)), "n"(K0 + 16 * (R * 2) + ROW4)
            : "memory");
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int t = 0; t < NT; ++t)
          f[j][t] = __builtin_bit_cast(frag, __builtin_shufflevector(v[j][t][0], v[j][t][1], 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      read_step<2 * H>(lds, f[0]);
      read_step<2 * H + 1>(lds, f[1]);
    }
  }
};

// Exponentials are taken to base 2 (the hardware's): exp x = 2^(x LOG2E).
constexpr float LOG2E = 1.44269504088896f, LN2 = 0.693147180559945f;
__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// x as three bf16 parts, each the nearest of what the ones before leave.  Finite values past bf16's largest (fp32's lowest, as
// a mask, among them) start from that: rounded to an infinity, they would make a NaN of their product with a g of 0.
__device__ inline void split3(float x, __bf16 (&p)[3]) {
  constexpr float BF16_MAX = 3.38953139e38f;
  p[0] = (__bf16)(fabsf(x) < INFINITY ? fminf(fmaxf(x, -BF16_MAX), BF16_MAX) : x);
  const float r = x - (float)p[0];
  p[1] = (__bf16)r;
  p[2] = (__bf16)(r - (float)p[1]);
}

// AT, BT: the operand is turned.  Waves: WM x WN, each (BM / WM) x (BN / WN).  NST: pipeline stages held in LDS.
// O: type of the operator's operands and results (float where T holds parts of fp32 values).
template <typename T, bool AT, bool BT, int BM, int BN, int WM, int WN, int NST, Epilogue E, typename O>
__global__ __launch_bounds__(64 * WM * WN) void gemm_kernel(GemmArgs g) {
  constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
  constexpr bool MULTI = std::is_same<O, float>::value && !std::is_same<T, float>::value;  // parts of fp32 values
  using OA = Operand<T, AT, BM, NW>;
  using OB = Operand<T, BT, BN, NW>;
  constexpr int STAGE = OA::BYTES + OB::BYTES, PER = OA::PER + OB::PER;
  constexpr int WROWS = BN / WN, WCOLS = BM / WM;
  // A wave's 32 rows x WCOLS results on their way out, rows 16 bytes apart in banks
  constexpr int OUT_SIZE = E == E_SLAB || (E == E_OUT ? std::is_same<O, float>::value : std::is_same<T, float>::value) ? 4 : 2;
  constexpr int OUT_ROW = WCOLS * OUT_SIZE + 16, OUT_BYTES = E == E_STATS ? WM * BN * 8 : NW * 32 * OUT_ROW;
  constexpr int LDS = NST * STAGE > OUT_BYTES ? NST * STAGE : OUT_BYTES;
  __shared__ __align__(1024) char s_mem[LDS];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM, l32 = lane & 31, half = lane >> 5;
  // Workgroups are dealt to the 8 XCDs in turn: each XCD takes a contiguous range of (split, tile), tiles ordered as
  // columns of 6 along n, so that those that run together share their operands in the XCD's L2 (columns of 4, 6, 8, 16 tiles:
  // 12.00, 12.04, 12.21, 12.43 ms for the gradients of 16384 x 2048 over 65536 words).
  constexpr int COL = 6;
  const int all = gridDim.x, xcd = blockIdx.x % 8, per = all / 8, rem = all % 8;
  const int job = xcd * per + min(xcd, rem) + blockIdx.x / 8, nt = g.tiles_m * g.tiles_n, split = job / nt, id = job - split * nt;
  const int col = id / (COL * g.tiles_m), width = min(COL, g.tiles_n - col * COL), in = id - col * COL * g.tiles_m;
  const int tile_m = in / width, tile_n = col * COL + in % width;
  const int m0 = tile_m * BM, n0 = tile_n * BN;

  OA oa;
  OB ob;
  const bool alt = AT && BT && g.alt && *g.alt;
  oa.init(alt ? g.a_alt : g.a, alt ? g.lda_alt : g.lda, m0, g.a_rows, wave, lane);
  ob.init(g.b, g.ldb, n0, g.b_rows, wave, lane);
  Fragments<T, AT, BM, TM> fa;
  Fragments<T, BT, BN, TN> fb;
  fa.init(wm * WCOLS, lane);
  fb.init(wn * WROWS, lane);

  const int kt = (g.K + BK - 1) / BK, total = MULTI ? kt * g.products : kt;
  const int s0 = (int)((int64_t)total * split / g.splits), s1 = (int)((int64_t)total * (split + 1) / g.splits);
  auto load = [&](int s, int buf) {
    // products of parts from the smallest to the largest, the last `products` of (2,0) (1,1) (0,2) (1,0) (0,1) (0,0)
    const int turn = MULTI ? s / kt : 0, pr = MULTI ? 6 - g.products + turn : 5, k0 = (s - turn * kt) * BK;
    const int pa = pr == 0 ? 2 : pr == 1 || pr == 3 ? 1 : 0, pb = pr == 2 ? 2 : pr == 1 || pr == 4 ? 1 : 0;
    char* at = s_mem + buf * STAGE;
    oa.load(at, pa * g.a_part, k0, g.K, wave);
    ob.load(at + OA::BYTES, pb * g.b_part, k0, g.K, wave);
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int t = 0; t < TN; ++t) acc[a][t] = f32x16{};

  typename Mfma<T>::frag a[2][TM], b[2][TN];
  auto mma = [&](int h) {
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int i = 0; i < TM; ++i) acc[i][t] = Mfma<T>::mma(a[h][i], b[h][t], acc[i][t]);
  };
  if constexpr (NW == 8) {
    // Two waves per SIMD, in turns: while waves 0..3 run the MFMAs of half a stage, waves 4..7 read their next half's
    // fragments and send off loads, and the other way round, a barrier between the turns (waves 4..7 are one turn late).
    // Turn 4 s: waves 0..3 read the first half of stage s and load stage s + 1 into the other buffer, which the last turn
    // of stage s - 1 has left; 4 s + 1: waves 4..7 do; 4 s + 3: the last reads of stage s, and the loads have come.
    const bool late = wave >= 4;
    auto turn = [&]() {
      __builtin_amdgcn_sched_barrier(0);
      wave_barrier();
      __builtin_amdgcn_sched_barrier(0);
    };
    auto compute = [&]() {
      __builtin_amdgcn_s_setprio(1);
      mma(0);
      mma(1);
      __builtin_amdgcn_s_setprio(0);
    };
    if (s1 > s0) load(s0, 0);
    wait_loads<0>();
    turn();
    if (late) turn();
    for (int s = s0; s < s1; ++s) {
      const int buf = (s - s0) & 1;
      const char* at = s_mem + buf * STAGE;
      // (the turned operands' reads end in a wait, so the loads go out first; plain ones' go after the reads: g of 16384 x 16384
      // x 2048 992 us, the other way 1075)
      if ((AT || BT) && s + 1 < s1) load(s + 1, buf ^ 1);
      fb.template read<0>(at + OA::BYTES, b);
      fa.template read<0>(at, a);
      if (!(AT || BT) && s + 1 < s1) load(s + 1, buf ^ 1);
      wait_lds();
      turn();
      compute();
      turn();
      fb.template read<1>(at + OA::BYTES, b);
      fa.template read<1>(at, a);
      if (late) wait_loads<0>();
      else wait_lds();
      turn();
      compute();
      if (!late) wait_loads<0>();
      turn();
    }
    if (!late) turn();
  } else if (s1 > s0) {
    // Stage s computes from buffer (s - s0) % NST while the next NST - 1 stages' loads are on their way.  Once every wave
    // holds the rest of the stage in registers, its buffer takes the loads of stage s + NST.  The workgroups of a CU cover
    // each other's waits.
#pragma unroll
    for (int i = 0; i < NST; ++i)
      if (s0 + i < s1) load(s0 + i, i);
    if (s1 - s0 >= NST) wait_loads<PER * (NST - 1)>();
    else wait_loads<0>();
    wave_barrier();
    auto next_stage = [&](int s, int buf) {
      if (NST > 2 && s + NST <= s1) wait_loads<PER * (NST > 2 ? NST - 2 : 0)>();
      else wait_loads<0>();
      wave_barrier();
      if (s + NST < s1) load(s + NST, buf);
    };
    int buf = 0;
    if constexpr (AT || BT) {
      for (int s = s0; s < s1; ++s) {
        const char* at = s_mem + buf * STAGE;
        fb.template read<0>(at + OA::BYTES, b);
        fa.template read<0>(at, a);
        mma(0);
        mma(1);
        fb.template read<1>(at + OA::BYTES, b);
        fa.template read<1>(at, a);
        if (s + 1 < s1) next_stage(s, buf);
        mma(0);
        mma(1);
        buf = buf + 1 == NST ? 0 : buf + 1;
      }
    } else {
      // plain operands: a wave reads the fragments of k-step j + 1 while the MFMAs of k-step j run, across stages too
      auto step = [&](auto j, const char* at) {
        constexpr int J = decltype(j)::value;
        fa.template read_step<J>(at, a[J & 1]);
        fb.template read_step<J>(at + OA::BYTES, b[J & 1]);
      };
      step(std::integral_constant<int, 0>{}, s_mem);
      for (int s = s0; s < s1; ++s) {
        const char* at = s_mem + buf * STAGE;
        const int next = buf + 1 == NST ? 0 : buf + 1;
        step(std::integral_constant<int, 1>{}, at);
        mma(0);
        step(std::integral_constant<int, 2>{}, at);
        mma(1);
        step(std::integral_constant<int, 3>{}, at);
        mma(0);
        if (s + 1 < s1) {
          next_stage(s, buf);
          step(std::integral_constant<int, 0>{}, s_mem + next * STAGE);
        }
        mma(1);
        buf = next;
      }
    }
  }

  // Element r of acc[i][t]: m = m0 + wm WCOLS + 32 i + 8 (r / 4) + 4 half + r % 4, n = n0 + wn WROWS + 32 t + l32.
  const int mw = m0 + wm * WCOLS + 4 * half, nw = n0 + wn * WROWS + l32;
  // fp32's logits from two fp16 parts: the rows' factors
  if constexpr ((E == E_STATS || E == E_GRAD || E == E_SLAB) && !AT && std::is_same<T, _Float16>::value && std::is_same<O, float>::value) {
    float fb[TN];
#pragma unroll
    for (int t = 0; t < TN; ++t) fb[t] = nw + 32 * t < g.N ? g.b_factor[nw + 32 * t] : 0.f;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int m = mw + 32 * i + 8 * q;
        f32x4 f;
        if (m + 4 <= g.M) {
          f = *(const f32x4*)(g.a_factor + m);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = m + e < g.M ? g.a_factor[m + e] : 0.f;
        }
        // (one factor at a time a sum could pass fp32's range on its way to a logit within it; an infinite product of finite
        // factors would make a NaN of a sum of 0; -infinity is the factor of a word with infinities)
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][t][4 * q + e] *= fminf(f[e] * fb[t], 3.4e38f);
      }
      __builtin_amdgcn_sched_barrier(0);  // 16 factors at a time: the registers are full of sums
    }
  }
  if constexpr (E == E_STATS) {
    float2* red = (float2*)s_mem;
    __syncthreads();
    if (m0 + BM > g.M)  // the last tile: what lies past the vocabulary counts for nothing
#pragma unroll
      for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (mw + 32 * i + 8 * (r / 4) + r % 4 >= g.M) acc[i][t][r] = -INFINITY;
#pragma unroll
    for (int t = 0; t < TN; ++t) {
      const int n = nw + 32 * t;
      const int lab = n < g.N ? (int)std::min<int64_t>(std::max<int64_t>(g.label[n], -1), g.V) - g.v0 : -1;
      // the label's logit, where the wave has one: word lab is value (i, r) of the lanes of one half
      const int d = lab - mw;
      if (__any(d >= 0 && d < WCOLS && lab < g.M && !(d & 4)))
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (d == 32 * i + 8 * (r / 4) + r % 4 && lab < g.M) g.at[n] = acc[i][t][r];
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, acc[i][t][r]);
      // the maximum in base 2, rounded: what is subtracted here is added again by the join, to the bit
      top = fmaxf(top, __shfl_xor(top, 32)) * LOG2E;
      const float ref = top == -INFINITY ? 0.f : top;
      float part[4] = {0.f, 0.f, 0.f, 0.f};  // small exponentials meet the largest, 1, in a fourth of the sums
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) part[r % 4] += exp2_of(__builtin_fmaf(acc[i][t][r], LOG2E, -ref));
      sum = (part[0] + part[1]) + (part[2] + part[3]);
      sum += __shfl_xor(sum, 32);
      if (half == 0) red[wm * BN + wn * WROWS + 32 * t + l32] = float2{top, sum};
    }
    __syncthreads();
    for (int c = threadIdx.x; c < BN; c += 64 * NW)
      if (n0 + c < g.N) {
        float top = red[c].x, sum = 0.f;
#pragma unroll
        for (int w = 1; w < WM; ++w) top = fmaxf(top, red[w * BN + c].x);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int w = 0; w < WM; ++w) {
          const float2 o = red[w * BN + c];
          sum += o.x == -INFINITY ? o.y : o.y * exp2_of(o.x - ref);
        }
        g.stats[(int64_t)tile_m * g.N + n0 + c] = float2{top, sum};
      }
  } else if constexpr (E == E_GRAD) {
    constexpr int PARTS = MULTI ? 3 : 1;
    using S = std::conditional_t<PARTS == 3, __bf16, T>;  // g as it is stored
    __syncthreads();
    char* stg = s_mem + wave * 32 * OUT_ROW;
    typedef S v4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int t = 0; t < TN; ++t) {
      const int n = nw + 32 * t;
      const bool row = n < g.N;
      const int lab = row ? (int)std::min<int64_t>(std::max<int64_t>(g.label[n], -1), g.V) - g.v0 : -1;
      const float c = row ? g.coef[n] : 0.f, lse = row ? g.lse[n] * LOG2E : 0.f;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int m = mw + 32 * i + 8 * (r / 4) + r % 4;
          const float p = exp2_of(__builtin_fmaf(acc[i][t][r], LOG2E, -lse)) - (m == lab ? 1.f : 0.f);
          acc[i][t][r] = c == 0.f ? 0.f : c * p;  // (a masked row's p may be anything)
        }
      if (m0 + BM > g.M)  // the last tile: zeros past the vocabulary
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (mw + 32 * i + 8 * (r / 4) + r % 4 >= g.M) acc[i][t][r] = 0.f;
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            v4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              o[e] = (S)acc[i][t][4 * q + e];
              if (PARTS > 1) acc[i][t][4 * q + e] -= (float)o[e];
            }
            *(v4*)(stg + l32 * OUT_ROW + (32 * i + 8 * q + 4 * half) * OUT_SIZE) = o;
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        constexpr int EV = 16 / OUT_SIZE, LANES = WCOLS / EV, LINES = 64 / LANES;  // lanes of a row, rows of an instruction
        typedef S v8 __attribute__((ext_vector_type(EV)));
        int nn = n0 + wn * WROWS + 32 * t + lane / LANES;
        S* dst = (S*)g.g + part * g.g_part + m0 + wm * WCOLS + (lane % LANES) * EV + nn * g.ldg;
#pragma unroll
        for (int k = 0; k < 32 / LINES; ++k) {
          const v8 o = *(const v8*)(stg + (k * LINES + lane / LANES) * OUT_ROW + (lane % LANES) * 16);
          if (nn < g.N) __builtin_nontemporal_store(o, (v8*)dst);  // read by later launches only
          nn += LINES, dst += LINES * g.ldg;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }
  } else {
    // Results leave through LDS, whole pieces of rows at a time (stored from the registers, four values of 32 rows at a time,
    // dh of 32000 x 9216 from 21 words took 260 us, now 154).
    using S = std::conditional_t<OUT_SIZE == 4, float, O>;
    constexpr int EV = 16 / OUT_SIZE, LANES = WCOLS / EV, LINES = 64 / LANES;
    typedef S v4 __attribute__((ext_vector_type(4)));
    typedef S vec __attribute__((ext_vector_type(EV)));
    typedef S vec_any __attribute__((ext_vector_type(EV), aligned(sizeof(S))));
    const float u = E == E_OUT ? *g.unscale : 1.f;
    __syncthreads();
    char* stg = s_mem + wave * 32 * OUT_ROW;
    const int64_t ld = E == E_OUT ? g.ldo : g.slab_ld;
    S* out = E == E_OUT ? (S*)g.out : (S*)(g.slab + split * g.slab_stride);
#pragma unroll
    for (int t = 0; t < TN; ++t) {
      const bool zero = E == E_OUT && g.row_coef && nw + 32 * t < g.N && g.row_coef[nw + 32 * t] == 0.f;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (S)(zero ? 0.f : acc[i][t][4 * q + e] * u);
          *(v4*)(stg + l32 * OUT_ROW + (32 * i + 8 * q + 4 * half) * OUT_SIZE) = v;
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const int c = (lane % LANES) * EV, m = m0 + wm * WCOLS + c;
      int n = n0 + wn * WROWS + 32 * t + lane / LANES;
      S* dst = out + n * ld + m;
#pragma unroll
      for (int k = 0; k < 32 / LINES; ++k) {
        const vec v = *(const vec*)(stg + (k * LINES + lane / LANES) * OUT_ROW + c * OUT_SIZE);
        if (n < g.N) {
          if constexpr (E == E_SLAB) {  // rows are padded to whole tiles
            *(vec*)dst = g.accumulate ? *(const vec*)dst + v : v;
          } else if (m + EV <= g.M) {
            *(vec_any*)dst = v;
          } else {
#pragma unroll
            for (int e = 0; e < EV; ++e)
              if (m + e < g.M) dst[e] = v[e];
          }
        }
        n += LINES, dst += LINES * ld;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
}

// Joins the tiles of a row: ROWS rows per workgroup, 256 / ROWS tiles at a time (16 rows share the lines that their
// statistics lie in; of a few rows each takes a workgroup: one row of 250 tiles 3.9 us, of ROWS = 16 6.6).
template <int ROWS>
__global__ __launch_bounds__(256) void join_stats_kernel(const float2* __restrict__ stats, const float* __restrict__ at,
                                                         const int64_t* __restrict__ label, int tiles, int n, int V,
                                                         float* __restrict__ loss, float* __restrict__ lse) {
  __shared__ float2 s_red[4][ROWS];
  const int row = blockIdx.x * ROWS + threadIdx.x % ROWS, t0 = threadIdx.x / ROWS;
  float top = -INFINITY, sum = 0.f;
  auto add = [&](float2 o) {  // (-inf, 0) adds nothing; a NaN sum stays
    const float m = fmaxf(top, o.x), ref = m == -INFINITY ? 0.f : m;
    sum = (top == -INFINITY ? sum : sum * exp2_of(top - ref)) + (o.x == -INFINITY ? o.y : o.y * exp2_of(o.x - ref));
    top = m;
  };
  if (row < n)
#pragma unroll 4
    for (int t = t0; t < tiles; t += 256 / ROWS) add(stats[(int64_t)t * n + row]);
#pragma unroll
  for (int d = ROWS; d < 64; d *= 2) add(float2{__shfl_xor(top, d), __shfl_xor(sum, d)});
  if ((threadIdx.x & 63) < ROWS) s_red[threadIdx.x >> 6][threadIdx.x & 63] = float2{top, sum};
  __syncthreads();
  if (threadIdx.x < ROWS && row < n) {
    for (int w = 1; w < 4; ++w) add(s_red[w][threadIdx.x]);
    const int64_t l = label[row];
    const bool has = l >= 0 && l < V;
    // the loss from the logits' difference, not from lse, whose rounding grows with the logits: of a row that is sure of its
    // label, little is left of lse - l
    const float lg = logf(sum);
    lse[row] = has ? __builtin_fmaf(top, LN2, lg) : 0.f;
    loss[row] = has ? __builtin_fmaf(__builtin_fmaf(at[row], -LOG2E, top), LN2, lg) : 0.f;
  }
}

// The few-tiles forward pass: logits of a row as `splits` partial sums; a workgroup per row, or (WAVE) a wave
// (32000 rows of 200 words: 21 us, a workgroup per row 140).
template <bool WAVE>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void join_logits_kernel(const float* __restrict__ slab, int64_t ld, int64_t stride,
                                                                        int splits, const int64_t* __restrict__ label, int64_t n, int V,
                                                                        float* __restrict__ loss, float* __restrict__ lse) {
  constexpr int TPR = WAVE ? 64 : 1024;
  __shared__ float s_top[16], s_sum[16];
  __shared__ float s_at[4];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const int64_t row = (int64_t)blockIdx.x * (WAVE ? 4 : 1) + sub;
  if (WAVE && row >= n) return;  // no barriers follow
  const int64_t l = label[row];
  float top = -INFINITY, sum = 0.f;
  for (int v = t; v < V; v += TPR) {
    float x = 0.f;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) x += slab[s * stride + row * ld + v];
    if (v == l) s_at[sub] = x;
    const float m = fmaxf(top, x), ref = m == -INFINITY ? 0.f : m;
    sum = (top == -INFINITY ? sum : sum * exp2_of((top - ref) * LOG2E)) + exp2_of((x - ref) * LOG2E);
    top = m;
  }
  float m = lanes_max<64>(top);
  const float ref = m == -INFINITY ? 0.f : m;
  float z = lanes_sum<64>(top == -INFINITY ? sum : sum * exp2_of((top - ref) * LOG2E));
  if constexpr (WAVE) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // s_at is the wave's own
  } else {
    if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = m, s_sum[threadIdx.x >> 6] = z;
    __syncthreads();
  }
  if (t == 0) {
    if constexpr (!WAVE) {
      m = s_top[0], z = 0.f;
      for (int w = 1; w < 16; ++w) m = fmaxf(m, s_top[w]);
      const float mr = m == -INFINITY ? 0.f : m;
      for (int w = 0; w < 16; ++w) z += s_top[w] == -INFINITY ? s_sum[w] : s_sum[w] * exp2_of((s_top[w] - mr) * LOG2E);
    }
    const bool has = l >= 0 && l < V;
    z = logf(z);
    lse[row] = has ? z + m : 0.f;
    loss[row] = has ? z + (m - s_at[sub]) : 0.f;  // as above
  }
}

// |g| <= FP16_BOOST: the coefficients are over the largest and |p - 1| <= 1; 65504 leaves room for p of up to 4, from an lse that
// is off.  fp16's smallest step, 2^-24, is 2^-38 of the largest weight then: a row whose weight is 1e-6 of the largest keeps
// probabilities of 5e-5 to 4 % (with 2^10 it lost them).
constexpr float FP16_BOOST = 0x1p14f;

// A row's part in the gradient, coef[n], and the factor that is left for the end, *unscale.  Without dloss every unmasked
// row counts 1 and unscale is scale / (their number).  With it the rows keep dloss / 2^e in (-2, 2) for the largest
// finite |dloss| in [2^e, 2^(e + 1)), or (by_largest, 16 bits) dloss over the largest: the heaviest row's g is then p - 1 at
// its label, nearly exact in 16 bits, where 1.02 (p - 1) would carry one rounding of up to 2^-8 into all of dh (one row of
// 5234 values over 12405 words: off by 2.9e-3 in all, 1.7e-3 now).  boost: a power of two that moves fp16's g away from its
// smallest values, FP16_BOOST.
// A workgroup of 1024 threads; returns the factor of the coefficients to all of them.
__device__ inline float weigh(const int64_t* __restrict__ label, const float* __restrict__ dloss, int64_t n, int V, float scale,
                              float boost, bool by_largest, float* __restrict__ mul, float* __restrict__ unscale,
                              int32_t* __restrict__ flag) {
  __shared__ float s_red[16];
  __shared__ float s_mul;
  float v = 0.f;
  for (int64_t i0 = threadIdx.x; i0 < n; i0 += 8 * 1024) {
    int64_t l[8];
    float d[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {  // eight loads at a time
      const int64_t i = i0 + k * 1024;
      l[k] = i < n ? label[i] : -1;
      d[k] = dloss && i < n ? fabsf(dloss[i]) : 1.f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (!(l[k] >= 0 && l[k] < V)) d[k] = 0.f;
      v = dloss ? (d[k] < INFINITY ? fmaxf(v, d[k]) : v) : v + d[k];
    }
  }
  v = dloss ? lanes_max<64>(v) : lanes_sum<64>(v);
  if ((threadIdx.x & 63) == 0) s_red[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    v = s_red[0];
    for (int w = 1; w < 16; ++w) v = dloss ? fmaxf(v, s_red[w]) : v + s_red[w];
    int e = dloss && v > 0.f ? ilogbf(v) : 0;
    e = e < -100 ? -100 : e > 100 ? 100 : e;
    // (a factor in fp32's normal range: an infinite one would make NaN of all of dh and dw)
    const float by = !dloss || v == 0.f ? 1.f : by_largest ? fminf(fmaxf(v, boost * 0x1p-126f), boost * 0x1p126f) : ldexpf(1.f, e);
    *mul = s_mul = boost / by;
    *unscale = dloss ? scale * (by / boost) : v > 0.f ? scale / (v * boost) : 0.f;
    *flag = 0;
  }
  __syncthreads();
  return s_mul;
}
__device__ inline float coef_of(const int64_t* __restrict__ label, const float* __restrict__ dloss, int64_t i, int V, float mul) {
  const bool has = label[i] >= 0 && label[i] < V;
  return has ? (dloss ? dloss[i] : 1.f) * mul : 0.f;
}
__global__ __launch_bounds__(1024) void weight_kernel(const int64_t* __restrict__ label, const float* __restrict__ dloss, int64_t n,
                                                      int V, float scale, float boost, bool by_largest, float* __restrict__ mul,
                                                      float* __restrict__ unscale, int32_t* __restrict__ flag) {
  weigh(label, dloss, n, V, scale, boost, by_largest, mul, unscale, flag);
}
__global__ __launch_bounds__(256) void coef_kernel(const int64_t* __restrict__ label, const float* __restrict__ dloss, int64_t n, int V,
                                                   const float* __restrict__ mul, float* __restrict__ coef) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) coef[i] = coef_of(label, dloss, i, V, *mul);
}

// Eight fp32 values as three bf16 parts, `part` elements apart.
__device__ inline void store_split3(__bf16* out, int64_t part, const float (&v)[8]) {
  float p[3][8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    __bf16 s[3];
    split3(v[j], s);
#pragma unroll
    for (int k = 0; k < 3; ++k) p[k][j] = (float)s[k];
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) store8(out + k * part, p[k]);
}

// Copies an operand into aligned rows of ldo elements (a multiple of 8), zeros past column C, as one 16-bit part or fp32's
// three; rows whose label is outside [0, V) become 0 (label may be null).  Units first, first + step, ... of eight values.
template <typename T>
__device__ inline void pack_rows(const T* __restrict__ in, int64_t ld, int64_t rows, int C, void* __restrict__ out, int64_t ldo,
                                 int64_t part, const int64_t* __restrict__ label, int V, int64_t first, int64_t step) {
  const int64_t per = ldo / 8, total = rows * per;
  for (int64_t u = first; u < total; u += step) {
    const int64_t row = u / per;
    const int c = (int)(u - row * per) * 8;
    float v[8];
    load8(in + row * ld, c, C, v);
    if (label && !(label[row] >= 0 && label[row] < V))
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.f;
    if constexpr (std::is_same<T, float>::value) {
      store_split3((__bf16*)out + row * ldo + c, part, v);
    } else {
      store8((T*)out + row * ldo + c, v);
    }
  }
}
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T* __restrict__ in, int64_t ld, int64_t rows, int C, void* __restrict__ out,
                                                   int64_t ldo, int64_t part, const int64_t* __restrict__ label, int V,
                                                   const int32_t* __restrict__ only_if) {
  if (only_if && !*only_if) return;
  pack_rows(in, ld, rows, C, out, ldo, part, label, V, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}
// Small calls in one launch: the first workgroup weighs the rows, the others (if any) copy h.
template <typename T>
__global__ __launch_bounds__(1024) void prepare_kernel(const int64_t* __restrict__ label, const float* __restrict__ dloss, int64_t n, int V,
                                                       float scale, float boost, float* __restrict__ mul, float* __restrict__ unscale,
                                                       int32_t* __restrict__ flag, float* __restrict__ coef, const T* __restrict__ h,
                                                       int64_t ld, int C, void* __restrict__ out, int64_t ldo) {
  if (blockIdx.x == 0) {
    const float m = weigh(label, dloss, n, V, scale, boost, sizeof(T) == 2, mul, unscale, flag);
    for (int64_t i = threadIdx.x; i < n; i += 1024) coef[i] = coef_of(label, dloss, i, V, m);
  } else {
    pack_rows(h, ld, n, C, out, ldo, n * ldo, label, V, (int64_t)(blockIdx.x - 1) * 1024 + threadIdx.x, (int64_t)(gridDim.x - 1) * 1024);
  }
}

// Sets *flag if a masked row (its label outside [0, V)) holds an infinity or a NaN: such a row alone can reach dw, as 0 times
// that.  A wave per row.
template <typename T>
__global__ __launch_bounds__(256) void masked_rows_kernel(const T* __restrict__ in, int64_t ld, int64_t rows, int C,
                                                          const int64_t* __restrict__ label, int V, int32_t* __restrict__ flag) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows || (label[row] >= 0 && label[row] < V)) return;
  bool bad = false;
  for (int c = (threadIdx.x & 63) * 8; c < C; c += 512) {
    float v[8];
    load8(in + row * ld, c, C, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) bad |= !(fabsf(v[j]) < INFINITY);
  }
  if (bad) *flag = 1;
}

// fp32 rows at any alignment as aligned ones of ldo elements, zeros past column C; masked rows become 0 (label may be null).
__global__ __launch_bounds__(256) void copy_rows_kernel(const float* __restrict__ in, int64_t ld, int64_t rows, int C,
                                                        float* __restrict__ out, int64_t ldo, const int64_t* __restrict__ label, int V,
                                                        const int32_t* __restrict__ only_if) {
  if (only_if && !*only_if) return;
  const int64_t per = ldo / 4, total = rows * per;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
    const int64_t row = u / per;
    const int c = (int)(u - row * per) * 4;
    f32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = c + j < C ? in[row * ld + c + j] : 0.f;
    if (label && !(label[row] >= 0 && label[row] < V)) v = f32x4{};
    *(f32x4*)(out + row * ldo + c) = v;
  }
}

// fp32 rows as two fp16 parts [2][rows][ldo] of x 2^k and a factor 2^-k, one workgroup per row; with `three` also as three bf16
// parts [3][rows][ldo].  Rows whose label is outside [0, V) become 0 (label may be null).  A row with a NaN keeps it.  Of a word
// (words) with infinities only these count, as +-2^13 without a second part, and the factor is infinite: logits are infinite by
// the sign of their sum, so a word masked by -infinity is one that no row reaches.  (Both signs are turned: -infinity as the
// factor tells it from products of factors past fp32's range.)  A row of h with infinities keeps them in both parts, inf and
// NaN: its logits are NaN.
__global__ __launch_bounds__(256) void split_rows_kernel(const float* __restrict__ in, int64_t ld, int C, _Float16* __restrict__ out,
                                                         int64_t ldo, int64_t part, float* __restrict__ factor,
                                                         __bf16* __restrict__ three, const int64_t* __restrict__ label, int V,
                                                         bool words) {
  __shared__ float s_top[4];
  const int64_t row = blockIdx.x;
  const float* x = in + row * ld;
  const bool zero = label && !(label[row] >= 0 && label[row] < V);
  float top = 0.f, first[8];
  for (int c = threadIdx.x * 8; c < ldo; c += 2048) {
    float v[8];
    load8(x, c, C, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[j]));
    if (c == (int)threadIdx.x * 8)
#pragma unroll
      for (int j = 0; j < 8; ++j) first[j] = v[j];
  }
  top = lanes_max<64>(top);
  if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
  int k = 0;
  if (!zero && top > 0.f && top < INFINITY) k = 13 - max(ilogbf(top), -100);
  const bool infinite = words && top == INFINITY;
  const float mul = ldexpf(1.f, k);
  if (threadIdx.x == 0) factor[row] = infinite ? -INFINITY : ldexpf(1.f, -k);
  for (int c = threadIdx.x * 8; c < ldo; c += 2048) {
    float v[8], w[8], lo[8];
    if (c == (int)threadIdx.x * 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = first[j];
    } else {
      load8(x, c, C, v);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = zero ? 0.f : v[j];
      w[j] = v[j] * mul;
      if (infinite) w[j] = v[j] != v[j] ? v[j] : fabsf(v[j]) == INFINITY ? copysignf(8192.f, -v[j]) : 0.f;
      lo[j] = w[j] - (float)(_Float16)w[j];
    }
    store8(out + row * ldo + c, w);
    store8(out + part + row * ldo + c, lo);
    if (three) store_split3(three + row * ldo + c, part, v);
  }
}

// out = unscale (sum of the slabs), rounded; rows with row_coef 0 are 0.
template <typename O>
__global__ __launch_bounds__(256) void join_slabs_kernel(const float* __restrict__ slab, int64_t ld, int64_t stride, int splits,
                                                         int64_t rows, int C, const float* __restrict__ unscale,
                                                         const float* __restrict__ row_coef, O* __restrict__ out, int64_t ldo) {
  const int per = (C + 7) / 8;
  const int64_t total = rows * per;
  const float u = *unscale;
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
    const bool zero = row_coef && row_coef[row] == 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = zero ? 0.f : v[j] * u;
    store8(out + row * ldo, c, C, v);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void zero_rows_kernel(T* __restrict__ out, int64_t ld, int64_t rows, int C) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * C; i += (int64_t)gridDim.x * 256)
    out[i / C * ld + i % C] = T{};
}

// -----------------------------------------------------------------------------------------------------------------
// Host side: which tiles, how many splits and pieces, and where things lie in the workspace.
// -----------------------------------------------------------------------------------------------------------------
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Work {  // offsets in the workspace, 256-byte aligned
  size_t total = 0;
  size_t take(size_t bytes) {
    const size_t at = total;
    total += up((int64_t)bytes, 256);
    return at;
  }
};

// Whether the loads can take an operand as it lies: rows that start on 16 bytes and hold whole 16-byte slots.
bool lies_well(const void* p, int64_t ld, int32_t C, dn_dtype dt) {
  return dt != DN_F32 && (uintptr_t)p % 16 == 0 && ld % 8 == 0 && C % 8 == 0 && ld <= MAX_LD;
}

// Tile shapes: T256 (8 waves, a workgroup per CU), T128 (4 waves, two per CU), and for the logits of few rows T64 and T32
// (128 words x 64 or 32 rows), of few words W64 and W32 (64 or 32 words x 128 rows).
enum Tile { T256, T128, T64, T32, W64, W32 };
int tile_m(Tile t) { return t == T256 ? 256 : t == W64 ? 64 : t == W32 ? 32 : 128; }
int tile_n(Tile t) { return t == T256 ? 256 : t == T64 ? 64 : t == T32 ? 32 : 128; }
// Rows or words that these are for (16 bits: 32000 rows x 9216 over 21 words 109 us, in T256 tiles 259; fp32, read as it lies:
// 64 rows x 2048 over 32000 words 92 us, laid out in parts 265, and 100 rows in parts 187).
constexpr int FEW = 64;

// The time of a product [M][N] over `stages` of 64 k in us, by what launches of many shapes took: a stage of T256 takes 1.25
// us on an idle chip and 1.75 on a full one, of T128 0.62 alone on a CU and 1.1 (turned operands: 1.2) for two, and a
// workgroup's start and end 5 to 10.  In splits, the partial sums' traffic and the launch that adds them come on top.
double product_us(Tile t, int64_t M, int64_t N, int64_t stages, int splits, bool turned) {
  const int64_t tiles = ((M + tile_m(t) - 1) / tile_m(t)) * ((N + tile_n(t) - 1) / tile_n(t)) * splits;
  const double st = (double)((stages + splits - 1) / splits), per_cu = (double)((tiles + 255) / 256);
  double us;
  if (t == T256)
    us = per_cu * (st * (1.25 + 0.5 * std::min(1.0, tiles / 256.0)) + 10);
  else if (t == T128)
    us = tiles <= 256 ? st * (0.62 + 0.25 * tiles / 256.0) + 5 : per_cu / 2 * (st * (turned ? 1.2 : 1.1) + 6);
  else  // at least the time that reading the long operand takes
    us = std::max(tiles <= 256 ? st * 0.5 + 4 : per_cu / 2 * (st * 0.6 + 4), (double)std::max(M, N) * stages * 128 / 5e6);
  return us + (splits > 1 ? 5 + (double)splits * M * N * 8 / 5e6 : 0);
}
// The only tile for the logits of few rows or words, or the number of those to choose from.
int logit_tiles(int64_t V, int64_t n, Tile (&of)[2]) {
  of[0] = T256, of[1] = T128;
  if (n > FEW && V > FEW) return 2;
  of[0] = V <= 32 && n > 32 ? W32 : n <= 32 ? T32 : n <= FEW ? T64 : W64;
  return 1;
}
// Whether a launch can have the product's workgroups.
bool fits_launch(Tile t, int64_t M, int64_t N, int splits) {
  const int64_t groups = ((M + tile_m(t) - 1) / tile_m(t)) * ((N + tile_n(t) - 1) / tile_n(t)) * splits;
  return groups <= MAX_LAUNCH_THREADS / (t == T256 ? 512 : 256);
}
// The tile and the splits with the least time (splits of at least 4 stages; one split unless `split`).  One of the tiles in one
// split fits a launch: the checks of the arguments, and forward_rows, see to it.
void choose(const Tile* of, int n_tiles, int64_t M, int64_t N, int64_t stages, bool split, bool turned, Tile& tile, int& splits) {
  double best = 1e300;
  for (int i = 0; i < n_tiles; ++i)
    for (int s = 1; s <= 64 && (s == 1 || (split && stages / s >= 4)); ++s) {
      const double us = product_us(of[i], M, N, stages, s, turned);
      if (fits_launch(of[i], M, N, s) && us < best * 0.999) best = us, tile = of[i], splits = s;
    }
}
int64_t stages_of(int64_t k, int products) { return (k + BK - 1) / BK * products; }

// An operand as a product reads it: 16-bit elements (or fp32 ones, two for each) from p on, rows ld apart, `part` between
// its parts, a factor for each row.
struct Matrix {
  const void* p;
  int64_t ld, part;
  const float* factor;
};
// How operands are laid out for products: as they lie (16-bit types; fp32 where `wide`), as three bf16 or two fp16 parts.
enum Layout { AS_IS, WIDE, THREE, TWO };
struct Pack {
  bool copy;       // laid out in the workspace
  bool words;      // w, not h
  Layout how;
  int64_t rows, ld;  // elements of a row there
  size_t at, factor_at;
};
Pack plan_pack(const void* p, int64_t ld, int64_t rows, int32_t C, dn_dtype dt, Layout how, bool always, Work& w) {
  Pack k{};
  k.how = how, k.rows = rows, k.ld = how == WIDE ? up(C, 4) * 2 : up(C, 8);
  if (how == AS_IS) k.copy = always || !lies_well(p, ld, C, dt);
  else if (how == WIDE) k.copy = always || (uintptr_t)p % 16 || ld % 4 || C % 4 || 2 * ld > MAX_LD;
  else k.copy = true;
  const int parts = how == THREE ? 3 : how == TWO ? 2 : 1;
  if (k.copy) k.at = w.take((size_t)parts * rows * k.ld * 2);
  if (how == TWO) k.factor_at = w.take((size_t)rows * 4);
  return k;
}

template <typename T>
int pack(const T* in, int64_t ld, int64_t rows, int C, void* out, int64_t ldo, const int64_t* label, int V, const int32_t* only_if,
         hipStream_t st) {
  const int64_t total = rows * (ldo / 8);
  const unsigned grid = (unsigned)std::min<int64_t>((total + 255) / 256, 8192);
  pack_kernel<T><<<grid, 256, 0, st>>>(in, ld, rows, C, out, ldo, rows * ldo, label, V, only_if);
  return (int)hipGetLastError();
}
int pack_any(dn_dtype dt, const void* in, int64_t ld, int64_t rows, int C, void* out, int64_t ldo, const int64_t* label, int V,
             const int32_t* only_if, hipStream_t st) {
  if (dt == DN_F32) return pack((const float*)in, ld, rows, C, out, ldo, label, V, only_if, st);
  if (dt == DN_F16) return pack((const _Float16*)in, ld, rows, C, out, ldo, label, V, only_if, st);
  return pack((const __bf16*)in, ld, rows, C, out, ldo, label, V, only_if, st);
}

template <typename T, bool AT, bool BT, Epilogue E, typename O, int BM, int BN, int WM, int WN, int NST>
int run_gemm(GemmArgs& g, hipStream_t st) {
  g.tiles_m = (g.M + BM - 1) / BM, g.tiles_n = (g.N + BN - 1) / BN;
  const dim3 grid((unsigned)(g.tiles_m * g.tiles_n * g.splits));
  gemm_kernel<T, AT, BT, BM, BN, WM, WN, NST, E, O><<<grid, 64 * WM * WN, 0, st>>>(g);
  return (int)hipGetLastError();
}
template <typename T, bool AT, bool BT, Epilogue E, typename O>
int run_tile(Tile t, GemmArgs& g, hipStream_t st) {
  // fp32 as it lies: few rows or words.  fp32's g from parts leaves as three parts, which T256's registers do not hold (1001
  // rows over 10007 words: 116 us, T128 99).
  constexpr bool wide = std::is_same<T, float>::value, logits = !AT && !BT;
  constexpr bool parts_out = E == E_GRAD && std::is_same<O, float>::value && !wide;
  if constexpr (!wide && !parts_out)
    if (t == T256) return run_gemm<T, AT, BT, E, O, 256, 256, 2, 4, 2>(g, st);
  if constexpr (!wide || !logits)
    if (t == T128) return run_gemm<T, AT, BT, E, O, 128, 128, 2, 2, 2>(g, st);
  if constexpr ((logits && !parts_out) || wide)
    if (t == T64) return run_gemm<T, AT, BT, E, O, 128, 64, 2, 2, 3>(g, st);
  if constexpr ((logits && !parts_out) || (wide && !BT))
    if (t == T32) return run_gemm<T, AT, BT, E, O, 128, 32, 4, 1, 4>(g, st);
  if constexpr (logits && !parts_out) {
    if (t == W64) return run_gemm<T, AT, BT, E, O, 64, 128, 1, 4, 3>(g, st);
    if (t == W32) return run_gemm<T, AT, BT, E, O, 32, 128, 1, 4, 4>(g, st);
  }
  return (int)hipErrorInvalidValue;  // no plan asks for another tile
}

struct FwdPlan {
  Layout how;
  Pack h, w;
  int products;
  Tile tile;
  int splits;
  bool logits;  // partial logits in memory (few tiles) instead of tile statistics
  int64_t tiles_m, ld;
  size_t stats_at, at_at, slab_at, total;
};
FwdPlan plan_forward(const LossArgs& a, dn_dtype dt) {
  FwdPlan f{};
  Work w;
  f.how = dt != DN_F32 ? AS_IS : a.n <= FEW || a.V <= FEW ? WIDE : TWO;
  f.h = plan_pack(a.h, a.h_stride, a.n, a.C, dt, f.how, false, w);
  f.w = plan_pack(a.w, a.w_stride, a.V, a.C, dt, f.how, false, w);
  f.w.words = true;
  f.products = f.how == TWO ? 3 : 1;
  Tile of[2];
  const int tiles = logit_tiles(a.V, a.n, of);
  choose(of, tiles, a.V, a.n, stages_of(f.w.ld, f.products), true, false, f.tile, f.splits);
  f.tiles_m = (a.V + tile_m(f.tile) - 1) / tile_m(f.tile);
  f.logits = f.splits > 1;
  f.at_at = w.take((size_t)a.n * 4);
  if (f.logits) {
    f.ld = f.tiles_m * tile_m(f.tile);
    f.slab_at = w.take((size_t)f.splits * a.n * f.ld * 4);
  } else {
    f.stats_at = w.take((size_t)f.tiles_m * a.n * 8);
  }
  f.total = w.total;
  return f;
}

struct BackPlan {
  Layout how;    // of the operands of dh and dw
  Pack h, w;
  bool h_spare;  // h is read as it lies, and from its copy only where a masked row holds an infinity or a NaN
  Layout logits;
  Pack lh, lw;   // fp32 parts: the logits' own layout, in two parts
  int parts, products, unit;  // unit: 16-bit elements of a value of g
  int64_t vc, ldg;            // words of a piece (a multiple of 256)
  Tile grad, dh, dw;
  int dh_splits, dw_splits;
  bool dh_slab, dw_slab;
  int64_t slab_ld;
  size_t coef_at, unscale_at, g_at, dh_at, dw_at, total;
};
constexpr int64_t PIECE_BYTES = 1LL << 29;  // of one part of g
constexpr int64_t SPARE_BYTES = 32 << 20;   // from here on h is looked through before it is copied (a launch against 13 us)
int logit_products(const BackPlan& b) { return b.logits == THREE ? 6 : b.logits == TWO ? 3 : 1; }
BackPlan plan_backward(const LossArgs& a, dn_dtype dt) {
  BackPlan b{};
  Work w;
  const bool few = a.n <= FEW || a.V <= FEW;
  b.how = dt != DN_F32 ? AS_IS : few ? WIDE : THREE;
  b.parts = b.how == THREE ? 3 : 1, b.products = b.how == THREE ? 6 : 1, b.unit = b.how == WIDE ? 2 : 1;
  const Pack plain = plan_pack(a.h, a.h_stride, a.n, a.C, dt, b.how, false, w);
  b.h_spare = !plain.copy && (int64_t)a.n * a.C * (int64_t)dtype_size(dt) >= SPARE_BYTES;
  b.h = plain.copy ? plain : plan_pack(a.h, a.h_stride, a.n, a.C, dt, b.how, true, w);  // masked rows become 0
  b.w = plan_pack(a.w, a.w_stride, a.V, a.C, dt, b.how, false, w);
  // fp32: from 400 rows on a second layout of w for the logits (12 bytes a value) costs less than three of the six products
  // (1001 rows x 1024 over 10007 words: 16 us against 75; of 300 rows the whole call takes 213 us with it, 210 without)
  b.logits = b.how == THREE && a.n >= 400 ? TWO : b.how;
  if (b.logits == TWO) {
    b.lh = plan_pack(a.h, a.h_stride, a.n, a.C, dt, TWO, true, w);
    b.lw = plan_pack(a.w, a.w_stride, a.V, a.C, dt, TWO, true, w);
    b.lw.words = true;
  }
  const int64_t v256 = up(a.V, 256);
  b.vc = std::min(v256, std::max<int64_t>(256, PIECE_BYTES / (2 * b.unit * a.n) / 256 * 256));
  const int64_t pieces = (v256 + b.vc - 1) / b.vc;
  b.vc = up((v256 + pieces - 1) / pieces, 256);
  b.ldg = b.vc;
  const int64_t words = std::min<int64_t>(b.vc, a.V);
  const int64_t k_c = b.logits == TWO ? b.lw.ld : b.w.ld, k_v = words * b.unit, k_n = a.n * b.unit;
  Tile of[2];
  int one, tiles = logit_tiles(words, a.n, of);
  if (b.how == THREE) of[0] = T128, tiles = 1;  // see run_tile
  choose(of, tiles, words, a.n, stages_of(k_c, logit_products(b)), false, false, b.grad, one);
  of[0] = T256, of[1] = T128, tiles = 2;
  if (b.how == WIDE) of[0] = a.n > FEW ? T128 : a.n > 32 ? T64 : T32, tiles = 1;
  choose(of, tiles, a.C, a.n, stages_of(k_v, b.products), true, true, b.dh, b.dh_splits);
  if (b.how == WIDE) of[0] = a.n > FEW ? T64 : T128;
  choose(of, tiles, a.C, words, stages_of(k_n, b.products), true, true, b.dw, b.dw_splits);
  b.dh_slab = pieces > 1 || b.dh_splits > 1;
  b.dw_slab = b.dw_splits > 1;
  b.slab_ld = up(a.C, 256);
  b.coef_at = w.take((size_t)a.n * 4);
  b.unscale_at = w.take(12);
  b.g_at = w.take((size_t)b.parts * b.unit * a.n * b.ldg * 2);
  if (b.dh_slab) b.dh_at = w.take((size_t)b.dh_splits * a.n * b.slab_ld * 4);
  if (b.dw_slab) b.dw_at = w.take((size_t)b.dw_splits * std::min<int64_t>(b.vc, a.V) * b.slab_ld * 4);
  b.total = w.total;
  return b;
}

// Lays an operand out as planned; label: rows whose label is outside [0, V) become 0.
// only_if: nothing is done where *only_if is 0.  three (two parts only): an operand's layout in three, done along with it.
int lay_out(const Pack& k, const void* p, int64_t ld, int32_t C, dn_dtype dt, const int64_t* label, int V, char* work, Matrix& m,
            hipStream_t st, const int32_t* only_if = nullptr, const Pack* three = nullptr) {
  m = Matrix{p, k.how == WIDE ? 2 * ld : ld, 0, nullptr};
  if (!k.copy) return 0;
  m.p = work + k.at, m.ld = k.ld, m.part = k.rows * k.ld;
  if (k.how == TWO) {
    m.factor = (const float*)(work + k.factor_at);
    constexpr int64_t most = MAX_LAUNCH_THREADS / 256;  // rows of a launch
    for (int64_t at = 0; at < k.rows; at += most) {
      split_rows_kernel<<<dim3((unsigned)std::min(k.rows - at, most)), 256, 0, st>>>(
          (const float*)p + at * ld, ld, C, (_Float16*)m.p + at * k.ld, k.ld, m.part, (float*)m.factor + at,
          three ? (__bf16*)(work + three->at) + at * k.ld : nullptr, label ? label + at : nullptr, V, k.words);
      if (const int err = (int)hipGetLastError()) return err;
    }
    return 0;
  }
  if (k.how == WIDE) {
    const unsigned grid = (unsigned)std::min<int64_t>((k.rows * (k.ld / 8) + 255) / 256, 8192);
    copy_rows_kernel<<<grid, 256, 0, st>>>((const float*)p, ld, k.rows, C, (float*)m.p, k.ld / 2, label, V, only_if);
    return (int)hipGetLastError();
  }
  return pack_any(dt, p, ld, k.rows, C, (void*)m.p, k.ld, label, V, only_if, st);
}

void set_operands(GemmArgs& g, const Matrix& a, int a_rows, const Matrix& b, int b_rows) {
  g.a = a.p, g.lda = a.ld, g.a_part = a.part, g.a_rows = a_rows, g.a_factor = a.factor;
  g.b = b.p, g.ldb = b.ld, g.b_part = b.part, g.b_rows = b_rows, g.b_factor = b.factor;
}

// T: type of the products' operands; O: of h and w.
template <typename T, typename O>
int forward(const LossArgs& a, dn_dtype dt, const FwdPlan& f, char* work, hipStream_t st) {
  Matrix h, w;
  int err;
  if ((err = lay_out(f.h, a.h, a.h_stride, a.C, dt, nullptr, 0, work, h, st))) return err;
  if ((err = lay_out(f.w, a.w, a.w_stride, a.C, dt, nullptr, 0, work, w, st))) return err;
  GemmArgs g{};
  set_operands(g, w, a.V, h, (int)a.n);
  g.M = a.V, g.N = (int)a.n, g.K = (int)f.w.ld, g.products = f.products, g.splits = f.splits;
  g.label = a.label, g.V = a.V;
  g.at = (float*)(work + f.at_at);
  if (f.logits) {
    g.slab = (float*)(work + f.slab_at), g.slab_ld = f.ld, g.slab_stride = a.n * f.ld;
    if ((err = run_tile<T, false, false, E_SLAB, O>(f.tile, g, st))) return err;
    if (a.V <= 2048 && a.n > FEW)
      join_logits_kernel<true><<<dim3((unsigned)((a.n + 3) / 4)), 256, 0, st>>>(g.slab, f.ld, g.slab_stride, f.splits, a.label, a.n, a.V,
                                                                               a.loss, a.lse);
    else
      join_logits_kernel<false><<<dim3((unsigned)a.n), 1024, 0, st>>>(g.slab, f.ld, g.slab_stride, f.splits, a.label, a.n, a.V, a.loss,
                                                                     a.lse);
  } else {
    g.stats = (float2*)(work + f.stats_at);
    if ((err = run_tile<T, false, false, E_STATS, O>(f.tile, g, st))) return err;
    if (a.n <= FEW)
      join_stats_kernel<1><<<dim3((unsigned)a.n), 256, 0, st>>>(g.stats, g.at, a.label, g.tiles_m, (int)a.n, a.V, a.loss, a.lse);
    else
      join_stats_kernel<16><<<dim3((unsigned)((a.n + 15) / 16)), 256, 0, st>>>(g.stats, g.at, a.label, g.tiles_m, (int)a.n, a.V,
                                                                              a.loss, a.lse);
  }
  return (int)hipGetLastError();
}

// T: type of the products' operands; O: of h, w and the results.
template <typename T, typename O>
int backward(const LossArgs& a, dn_dtype dt, const BackPlan& b, char* work, float boost, hipStream_t st) {
  float* coef = (float*)(work + b.coef_at);
  float* unscale = (float*)(work + b.unscale_at);
  int32_t* flag = (int32_t*)(unscale + 2);
  int err;
  // up to 8192 rows one workgroup weighs them in one go, and the copy of h goes along with it (64 x 512 over 1000 words: two
  // launches less, 37 -> 33 us)
  const bool two = b.logits == TWO, small = a.n <= 8192, along = small && b.how != WIDE && !b.h_spare && !two;
  if (small) {
    const int64_t units = along ? a.n * (b.h.ld / 8) : 0;
    const unsigned grid = 1 + (unsigned)std::min<int64_t>((units + 1023) / 1024, 2048);
    prepare_kernel<O><<<grid, 1024, 0, st>>>(a.label, a.dloss, a.n, a.V, a.scale, boost, unscale + 1, unscale, flag, coef,
                                            (const O*)a.h, a.h_stride, a.C, work + b.h.at, b.h.ld);
    if ((err = (int)hipGetLastError())) return err;
  } else {
    weight_kernel<<<1, 1024, 0, st>>>(a.label, a.dloss, a.n, a.V, a.scale, boost, sizeof(O) == 2, unscale + 1, unscale, flag);
    if ((err = (int)hipGetLastError())) return err;
    coef_kernel<<<dim3((unsigned)((a.n + 255) / 256)), 256, 0, st>>>(a.label, a.dloss, a.n, a.V, unscale + 1, coef);
    if ((err = (int)hipGetLastError())) return err;
  }
  Matrix h, w, lh, lw;
  if (two) {
    if ((err = lay_out(b.lh, a.h, a.h_stride, a.C, dt, a.label, a.V, work, lh, st, nullptr, &b.h))) return err;
    if ((err = lay_out(b.lw, a.w, a.w_stride, a.C, dt, nullptr, 0, work, lw, st, nullptr, &b.w))) return err;
    h = Matrix{work + b.h.at, b.h.ld, b.h.rows * b.h.ld, nullptr};
    w = Matrix{work + b.w.at, b.w.ld, b.w.rows * b.w.ld, nullptr};
  } else {
    if (b.h_spare) {
      constexpr int64_t most = MAX_LAUNCH_THREADS / 256 * 4;  // rows of a launch
      for (int64_t at = 0; at < a.n; at += most) {
        const int64_t rows = std::min(a.n - at, most);
        masked_rows_kernel<O><<<dim3((unsigned)((rows + 3) / 4)), 256, 0, st>>>((const O*)a.h + at * a.h_stride, a.h_stride, rows, a.C,
                                                                                a.label + at, a.V, flag);
        if ((err = (int)hipGetLastError())) return err;
      }
    }
    if (along)
      h = Matrix{work + b.h.at, b.h.ld, b.h.rows * b.h.ld, nullptr};
    else if ((err = lay_out(b.h, a.h, a.h_stride, a.C, dt, a.label, a.V, work, h, st, b.h_spare ? flag : nullptr)))
      return err;
    if ((err = lay_out(b.w, a.w, a.w_stride, a.C, dt, nullptr, 0, work, w, st))) return err;
    lh = b.h_spare ? Matrix{a.h, a.h_stride * b.unit, 0, nullptr} : h, lw = w;  // (a masked row's logits reach nothing)
  }
  const Matrix gm{work + b.g_at, b.ldg * b.unit, a.n * b.ldg, nullptr};
  for (int64_t v0 = 0; v0 < a.V; v0 += b.vc) {
    const int vc = (int)std::min<int64_t>(b.vc, a.V - v0);
    const auto piece = [&](Matrix m) {  // rows v0 on
      m.p = (const char*)m.p + v0 * m.ld * 2;
      if (m.factor) m.factor += v0;
      return m;
    };
    GemmArgs g{};  // the piece's logits, leaving as g
    set_operands(g, piece(lw), vc, lh, (int)a.n);
    g.M = vc, g.N = (int)a.n, g.K = (int)(b.logits == TWO ? b.lw.ld : b.w.ld), g.products = logit_products(b), g.splits = 1;
    g.label = a.label, g.v0 = (int)v0, g.V = a.V, g.lse = a.lse_in, g.coef = coef;
    g.g = work + b.g_at, g.ldg = b.ldg, g.g_part = gm.part;
    if constexpr (std::is_same<T, __bf16>::value && std::is_same<O, float>::value)
      err = b.logits == TWO ? run_tile<_Float16, false, false, E_GRAD, O>(b.grad, g, st) : run_tile<T, false, false, E_GRAD, O>(b.grad, g, st);
    else
      err = run_tile<T, false, false, E_GRAD, O>(b.grad, g, st);
    if (err) return err;

    GemmArgs d{};  // dh += g w
    set_operands(d, piece(w), (int)b.w.ld, gm, (int)a.n);
    d.M = a.C, d.N = (int)a.n, d.K = vc * b.unit, d.products = b.products, d.splits = b.dh_splits;
    d.unscale = unscale;
    if (b.dh_slab) {
      d.slab = (float*)(work + b.dh_at), d.slab_ld = b.slab_ld, d.slab_stride = a.n * b.slab_ld, d.accumulate = v0 > 0;
      err = run_tile<T, true, false, E_SLAB, O>(b.dh, d, st);
    } else {
      d.out = a.dh, d.ldo = a.dh_stride, d.row_coef = coef;
      err = run_tile<T, true, false, E_OUT, O>(b.dh, d, st);
    }
    if (err) return err;

    GemmArgs e{};  // dw = g^T h
    set_operands(e, b.h_spare ? lh : h, (int)b.h.ld, gm, (int)up(vc, 8) * b.unit);
    if (b.h_spare) e.alt = flag, e.a_alt = h.p, e.lda_alt = h.ld;
    e.M = a.C, e.N = vc, e.K = (int)a.n * b.unit, e.products = b.products, e.splits = b.dw_splits;
    e.unscale = unscale;
    O* dw = (O*)a.dw + v0 * a.dw_stride;
    if (b.dw_slab) {
      e.slab = (float*)(work + b.dw_at), e.slab_ld = b.slab_ld, e.slab_stride = std::min<int64_t>(b.vc, a.V) * b.slab_ld;
      if ((err = run_tile<T, true, true, E_SLAB, O>(b.dw, e, st))) return err;
      const unsigned grid = (unsigned)std::min<int64_t>(((int64_t)vc * ((a.C + 7) / 8) + 255) / 256, 8192);
      join_slabs_kernel<O><<<grid, 256, 0, st>>>(e.slab, e.slab_ld, e.slab_stride, b.dw_splits, vc, a.C, unscale, nullptr, dw,
                                                 a.dw_stride);
      err = (int)hipGetLastError();
    } else {
      e.out = dw, e.ldo = a.dw_stride;
      err = run_tile<T, true, true, E_OUT, O>(b.dw, e, st);
    }
    if (err) return err;
  }
  if (b.dh_slab) {
    const unsigned grid = (unsigned)std::min<int64_t>((a.n * ((a.C + 7) / 8) + 255) / 256, 8192);
    join_slabs_kernel<O><<<grid, 256, 0, st>>>((const float*)(work + b.dh_at), b.slab_ld, a.n * b.slab_ld, b.dh_splits, a.n, a.C,
                                               unscale, coef, (O*)a.dh, a.dh_stride);
    err = (int)hipGetLastError();
  }
  return err;
}

}  // namespace

// The forward pass goes over more rows than its launches have threads for in pieces: of 2^22 rows less a tile (1024 threads each
// in the join), and of 2^24 - 1 tiles of 128 x 128.
int64_t forward_rows(const LossArgs& a) {
  const int64_t most = std::min<int64_t>((1 << 22) - 128, ((1 << 24) - 1) / (((int64_t)a.V + 127) / 128) * 128);
  const int64_t pieces = (a.n + most - 1) / most;
  return std::min(most, up((a.n + pieces - 1) / pieces, 128));
}
LossArgs forward_piece(const LossArgs& a, dn_dtype dt, int64_t at, int64_t rows) {
  LossArgs p = a;
  p.h = (const char*)a.h + at * a.h_stride * (int64_t)dtype_size(dt);
  p.label = a.label + at, p.n = std::min(rows, a.n - at);
  if (a.loss) p.loss = a.loss + at;
  if (a.lse) p.lse = a.lse + at;
  return p;
}

size_t softmax_loss_bytes(const LossArgs& a, dn_dtype dt) {
  const int64_t rows = forward_rows(a), last = (a.n - 1) / rows * rows;  // all pieces but the last are alike
  return std::max(plan_forward(forward_piece(a, dt, 0, rows), dt).total, plan_forward(forward_piece(a, dt, last, rows), dt).total);
}
// (never 0, so that a caller's workspace is never the null pointer of a size query: without rows, dw is still to be written)
size_t softmax_loss_backward_bytes(const LossArgs& a, dn_dtype dt) { return a.n ? plan_backward(a, dt).total : 256; }

int launch_softmax_loss(const LossArgs& a, dn_dtype dt, void* d_work, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  const int64_t rows = forward_rows(a);
  for (int64_t at = 0; at < a.n; at += rows) {
    const LossArgs p = forward_piece(a, dt, at, rows);
    const FwdPlan f = plan_forward(p, dt);
    const int err = f.how == WIDE  ? forward<float, float>(p, dt, f, (char*)d_work, st)
                    : f.how == TWO ? forward<_Float16, float>(p, dt, f, (char*)d_work, st)
                    : dt == DN_F16 ? forward<_Float16, _Float16>(p, dt, f, (char*)d_work, st)
                                   : forward<__bf16, __bf16>(p, dt, f, (char*)d_work, st);
    if (err) return err;
  }
  return 0;
}

int launch_softmax_loss_backward(const LossArgs& a, dn_dtype dt, void* d_work, void* stream) {
  if (a.n == 0) {  // no rows: dw is 0
    const unsigned grid = (unsigned)std::min<int64_t>(((int64_t)a.V * a.C + 255) / 256, 8192);
    if (dt == DN_F32)
      zero_rows_kernel<float><<<grid, 256, 0, (hipStream_t)stream>>>((float*)a.dw, a.dw_stride, a.V, a.C);
    else
      zero_rows_kernel<uint16_t><<<grid, 256, 0, (hipStream_t)stream>>>((uint16_t*)a.dw, a.dw_stride, a.V, a.C);
    return (int)hipGetLastError();
  }
  const BackPlan b = plan_backward(a, dt);
  const hipStream_t st = (hipStream_t)stream;
  if (b.how == WIDE) return backward<float, float>(a, dt, b, (char*)d_work, 1.f, st);
  if (dt == DN_F32) return backward<__bf16, float>(a, dt, b, (char*)d_work, 1.f, st);
  if (dt == DN_F16) return backward<_Float16, _Float16>(a, dt, b, (char*)d_work, FP16_BOOST, st);
  return backward<__bf16, __bf16>(a, dt, b, (char*)d_work, 1.f, st);
}

}  // namespace head
}  // namespace dn
