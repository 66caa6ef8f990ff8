// Operand tiles of the head's matrix products: loads straight from memory into LDS, and the fragments that the matrix cores
// take from there.
#pragma once

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

typedef short i16x4 __attribute__((ext_vector_type(4)));
constexpr uint32_t OOB = 0x80000000u;  // a buffer offset past every buffer: reads as 0
constexpr int BK = 64;                 // k of one pipeline stage (of 16-bit values; fp32: 32)
constexpr int64_t MAX_LD = 1 << 22;    // elements between rows: 256 rows stay within 32-bit byte offsets

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

// The operands of a product D[m][n] = sum_k A(m, k) B(n, k).  An operand lies with k along its rows ([m][k], plain) or with k
// across them ([k][m], turned); ld: elements from row to row, *_part: between the parts of operands that are sums of parts.
struct Multiplied {
  const void *a, *b;
  int64_t lda, ldb, a_part, b_part;
  int32_t a_rows, b_rows;  // rows of the operand that may be read (turned: columns, a multiple of 8)
  int32_t K, products;
};
// acc = split `split` of `splits` of the tile's sums over k: BM x BN from (m0, n0) on, waves WM x WN, each (BM / WM) x (BN / WN).
// MULTI: the last p.products of the six products of parts.  AT, BT: the operand is turned.  NST: pipeline stages in LDS (s_mem).
template <typename T, bool AT, bool BT, int BM, int BN, int WM, int WN, int NST, bool MULTI>
__device__ __forceinline__ void multiply(char* s_mem, const Multiplied& p, int m0, int n0, int split, int splits, int wave, int lane,
                                         f32x16 (&acc)[BM / WM / 32][BN / WN / 32]) {
  constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
  using OA = Operand<T, AT, BM, NW>;
  using OB = Operand<T, BT, BN, NW>;
  constexpr int STAGE = OA::BYTES + OB::BYTES, PER = OA::PER + OB::PER;
  constexpr int WROWS = BN / WN, WCOLS = BM / WM;
  const int wm = wave % WM, wn = wave / WM;
  OA oa;
  OB ob;
  oa.init(p.a, p.lda, m0, p.a_rows, wave, lane);
  ob.init(p.b, p.ldb, n0, p.b_rows, wave, lane);
  Fragments<T, AT, BM, TM> fa;
  Fragments<T, BT, BN, TN> fb;
  fa.init(wm * WCOLS, lane);
  fb.init(wn * WROWS, lane);

  const int kt = (p.K + BK - 1) / BK, total = MULTI ? kt * p.products : kt;
  const int s0 = (int)((int64_t)total * split / splits), s1 = (int)((int64_t)total * (split + 1) / splits);
  auto load = [&](int s, int buf) {
    // products of parts from the smallest to the largest, the last `products` of (2,0) (1,1) (0,2) (1,0) (0,1) (0,0)
    const int turn = MULTI ? s / kt : 0, pr = MULTI ? 6 - p.products + turn : 5, k0 = (s - turn * kt) * BK;
    const int pa = pr == 0 ? 2 : pr == 1 || pr == 3 ? 1 : 0, pb = pr == 2 ? 2 : pr == 1 || pr == 4 ? 1 : 0;
    char* at = s_mem + buf * STAGE;
    oa.load(at, pa * p.a_part, k0, p.K, wave);
    ob.load(at + OA::BYTES, pb * p.b_part, k0, p.K, wave);
  };

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
}

}  // namespace head
}  // namespace dn
