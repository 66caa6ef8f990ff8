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

}  // namespace head
}  // namespace dn
