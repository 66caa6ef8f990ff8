// Scores of rows of logits: log probability of a given token, entropy and best alternatives, and their gradient.
//   x = scale l;  lse = log sum exp x;  logp_v = x_v - lse;  H = -sum p log p;  the `top` largest logits, lower index first among equals
//   gradient: with A = dlse - dlogp - sum dtop - dH H,  dl_v = scale (p_v (A - dH log p_v) + dlogp [v = token] + dtop_j [v = id_j])
// A row is read once (the gradient: read once and written once).  The gradient is bound by memory (4096 x 32000 in bf16 92 us, 333 x
// 50257 in fp32 with 8 alternatives 27), the scores by the vector unit (2000 x 50257 in fp16 45 us, with 5 alternatives 57), and one
// row by the chain of its two launches (131072 logits with 20 alternatives 19 to 21 us).  Every lane keeps its own maximum m, sum S of
// exp(x - m) and T of exp(x - m) (x - m) and rescales them where the maximum grows; lanes, waves and workgroups join theirs at
// the end, in a fixed order.  H = log S - T / S, and a logit's part is taken as (x - m), so large logits lose no digits.
// Alternatives: a wave keeps candidates above a bound that `top` values of the row are known to reach.  The top-th largest of the
// lanes' maxima so far is such a bound; it is looked for where a block of 1024 has a value above the last one, and the waves of a row
// tell each other theirs.  Few blocks have (of logits in no order about top ln(V / 1024)); a full buffer is ranked and cut to `top`.
// Candidates are 64-bit keys, value and then index, so no two are equal, and results do not depend on who found them first.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "head.h"

namespace dn {
namespace head {
namespace {

constexpr float LOG2E = 1.44269504088896f, LN2 = 0.693147180559945f;
constexpr int MOST = DN_MAX_TOP;  // alternatives
constexpr int CAP = 192;          // keys of a wave's buffer: `top` and two waves' worth
constexpr int EV = 16;            // values of a lane in a block, twice eight
constexpr int WAVE_BLOCK = 64 * EV;

typedef unsigned long long Key;
// Larger for larger values and, among equal ones, for lower indices.  0 and -0 are equal.
__device__ inline uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline Key key_of(float x, uint32_t index) { return (Key)ordered(x) << 32 | ~index; }
__device__ inline float value_of(Key k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
constexpr Key NOTHING = (Key)0x007fffffu << 32 | 0xffffffffu;  // key of -infinity at index 0: no key of -infinity is above it

// Maximum, sum of exponentials, and sum of exponentials times their base 2 logarithm (times scale: c = scale log2 e).
struct Stats {
  float m, s, t;
};
__device__ inline float below(float m, float top, float c) {  // base 2 logarithm of what a sum over m is worth over top
  return m == -INFINITY ? 0.f : fmaxf((m - top) * c, -1000.f);  // (finite: of a mask of the type's lowest value 0 times it is 0)
}
__device__ inline Stats join(const Stats& a, const Stats& b, float c) {
  const float m = fmaxf(a.m, b.m), da = below(a.m, m, c), db = below(b.m, m, c);
  const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
  return Stats{m, a.s * fa + b.s * fb, fa * (a.t + a.s * da) + fb * (b.t + b.s * db)};
}
__device__ inline Stats lanes_join(Stats a, float c) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) a = join(a, Stats{__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.t, d)}, c);
  // (lanes that join the same two the other way round may differ in a last bit, and equal logits would in their log probabilities)
  const auto first = [](float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); };
  return Stats{first(a.m), first(a.s), first(a.t)};
}

// A wave's candidates.  All of it is the wave's own, but for the other waves' bounds of the row: no barriers.
struct Candidates {
  Key* buf;                 // [CAP] in LDS
  volatile uint32_t* seen;  // [4] in LDS: values that the row's waves know `top` values of the row to reach (null: a row of its own)
  int count;                // wave-uniform
  Key bound;                // `top` keys above or at it have been seen (or NOTHING)
  int top;

  __device__ inline void init(Key* b, volatile uint32_t* s, int k) { buf = b, seen = s, count = 0, bound = NOTHING, top = k; }
  __device__ inline void raise(Key to) {
    if (to > bound) bound = to;
  }
  // The bound from one value per lane, the lane's largest so far: the top-th largest of these.  BITS: low bits that are 0 in T.
  template <int BITS>
  __device__ inline void raise_to(float lane_max) {
    const uint32_t o = ordered(lane_max);
    uint32_t at = 0;
#pragma unroll 4
    for (int bit = 31; bit >= BITS; --bit) {
      const uint32_t to = at | 1u << bit;
      if (__popcll(__ballot(o >= to)) >= top) at = to;
    }
    if (at) raise(((Key)at << 32) - 1);
    tell();
  }
  // (the value that `top` keys reach: the bound's own, or of a bound from lanes' maxima the one after it)
  __device__ inline void tell() {
    if (seen && (threadIdx.x & 63) == 0) seen[threadIdx.x >> 6] = (uint32_t)((bound + 1) >> 32);
  }
  __device__ inline void hear() {
    if (!seen) return;
    uint32_t v = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) v = max(v, seen[w]);
    v = __builtin_amdgcn_readfirstlane(v);
    if (v) raise(((Key)v << 32) - 1);  // equal values stay: theirs may have lower indices than what others hold
  }
  // Ranks all keys and keeps the first `top`, in order.
  __device__ inline void cut() {
    const int lane = threadIdx.x & 63;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    Key mine[CAP / 64];
    int rank[CAP / 64];
#pragma unroll
    for (int i = 0; i < CAP / 64; ++i) mine[i] = lane + 64 * i < count ? buf[lane + 64 * i] : 0, rank[i] = 0;
    if (lane < 8 && count + lane < CAP) buf[count + lane] = 0;  // eight are read at a time; no key is below 0
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int rows = (count + 63) / 64;
    for (int j = 0; j < count; j += 8) {
      Key k[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) k[e] = buf[j + e];
#pragma unroll
      for (int i = 0; i < CAP / 64; ++i)
        if (i < rows)
#pragma unroll
          for (int e = 0; e < 8; ++e) rank[i] += k[e] > mine[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < CAP / 64; ++i)
      if (lane + 64 * i < count && rank[i] < top) buf[rank[i]] = mine[i];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (count >= top) {
      count = top;
      raise(buf[top - 1]);
      tell();
    }
  }
  // One key per lane (0: none), in any order of indices.  A key at the bound is one that is held already.
  __device__ inline void offer(Key k) {
    unsigned long long hits = __ballot(k > bound);
    if (!hits) return;
    if (count + __popcll(hits) > CAP) {
      cut();
      hits = __ballot(k > bound);
    }
    const int at = count + __builtin_amdgcn_mbcnt_hi((uint32_t)(hits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hits, 0));
    if (k > bound) buf[at] = k;
    count += __popcll(hits);
  }
};

// Eight values from element i on, -infinity from element `end` on.
template <typename T>
__device__ inline typename Vec8<T>::type load_logits(const T* row, int i, int end) {
  if (i + 8 <= end) return *(const typename Vec8<T>::type*)(row + i);
  typename Vec8<T>::type r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = i + j < end ? row[i + j] : (T)-INFINITY;
  return r;
}

// Writes a row's results from its joined statistics and sorted keys (`count` of them); one wave.
__device__ inline void write_row(const ScoresArgs& a, int64_t row, const Stats& z, float logit, bool has, const Key* keys, int count) {
  const int lane = threadIdx.x & 63;
  const bool bad = !(z.s < INFINITY);  // a NaN or +infinity among the logits
  const bool empty = z.m == -INFINITY && !bad;
  const float log_s = logf(z.s), nan = __uint_as_float(0x7fc00000u);
  if (lane == 0) {
    if (a.logp) a.logp[row] = !has || empty ? 0.f : bad ? nan : (logit - z.m) * a.scale - log_s;
    if (a.entropy) a.entropy[row] = bad ? nan : empty ? 0.f : log_s - LN2 * (z.t / z.s);
    a.lse[row] = bad ? nan : empty ? -INFINITY : z.m * a.scale + log_s;
  }
  for (int j = lane; j < a.top; j += 64) {
    const bool found = j < count && !bad && !empty;
    a.top_id[row * a.top + j] = found ? (int64_t)(uint32_t)~(uint32_t)keys[j] : -1;
    a.top_logp[row * a.top + j] = found ? (value_of(keys[j]) - z.m) * a.scale - log_s : bad ? nan : -INFINITY;
  }
}

// A wave's pass over blocks first, first + step, ... of a row's elements [0, end).
template <typename T, bool TOP>
__device__ inline Stats scan(const T* row, int64_t first, int64_t step, int end, float c, Candidates& cand) {
  const int lane = threadIdx.x & 63;
  Stats z{-INFINITY, 0.f, 0.f};
  typedef typename Vec8<T>::type Raw;
  Raw next[2];
  auto load = [&](int64_t b) {
#pragma unroll
    for (int h = 0; h < 2; ++h) next[h] = load_logits(row, (int)std::min<int64_t>(b * WAVE_BLOCK + h * 512 + lane * 8, 0x7ffffff0), end);
  };
  const int64_t blocks = ((int64_t)end + WAVE_BLOCK - 1) / WAVE_BLOCK;
  if (first < blocks) load(first);
  for (int64_t b = first; b < blocks; b += step) {
    float x[EV];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 8; ++j) x[8 * h + j] = (float)next[h][j];
    if (b + step < blocks) load(b + step);
    float top = x[0];
#pragma unroll
    for (int j = 1; j < EV; ++j) top = fmaxf(top, x[j]);
    const float m = fmaxf(z.m, top), ref = m == -INFINITY ? 0.f : m;
    const float d = below(z.m, m, c), f = __builtin_amdgcn_exp2f(d);
    float s[2] = {z.s * f, 0.f}, t[2] = {f * (z.t + z.s * d), 0.f};
#pragma unroll
    for (int j = 0; j < EV; ++j) {
      const float u = (x[j] - ref) * c, e = __builtin_amdgcn_exp2f(u);
      s[j & 1] += e;
      t[j & 1] = __builtin_fmaf(e, fmaxf(u, -200.f), t[j & 1]);  // (of -infinity: 0 times that)
    }
    z.m = m, z.s = s[0] + s[1], z.t = t[0] + t[1];
    if constexpr (TOP) {
      // (a value equal to the bound's has a higher index than all that are held: blocks come in order)
      if (__any(ordered(top) > (uint32_t)(cand.bound >> 32))) {
        cand.hear();
        cand.template raise_to<std::is_same<T, float>::value ? 0 : std::is_same<T, __bf16>::value ? 16 : 13>(m);
        const float least = value_of(cand.bound);
#pragma unroll
        for (int j = 0; j < EV; ++j)
          if (__any(!(x[j] < least))) cand.offer(key_of(x[j], (uint32_t)(b * WAVE_BLOCK + (j / 8) * 512 + lane * 8 + j % 8)));
      }
    }
  }
  return z;
}

// The first `top` of four waves' sorted keys, in order; their number.  s_count is written, a barrier before.
__device__ inline int best_of(const Key (*s_keys)[CAP], const int* s_count, const Candidates& cand, Key* s_best) {
  const int lane = threadIdx.x & 63;
  int count = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) count += s_count[w];
  if (lane < cand.count) {
    const Key mine = cand.buf[lane];
    int rank = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll 8
      for (int j = 0; j < s_count[w]; ++j) rank += s_keys[w][j] > mine;
    if (rank < cand.top) s_best[rank] = mine;
  }
  __syncthreads();
  return min(count, cand.top);
}

// A workgroup of a split row leaves its statistics, and behind all rows' statistics `top` sorted keys (0: none).
__device__ inline Key* part_keys(const ScoresArgs& a, int64_t row) {
  return (Key*)((Stats*)a.work + (a.n * a.parts + 1) / 2 * 2) + row * a.parts * a.top;
}

// WAVE: a wave per row, four rows per workgroup.  Else a workgroup per row, or (SPLIT) one of `parts` workgroups of a row.
template <typename T, bool WAVE, bool SPLIT, bool TOP>
__global__ __launch_bounds__(256) void scores_kernel(ScoresArgs a) {
  __shared__ Key s_keys[TOP ? 4 : 1][TOP ? CAP : 1];
  __shared__ Key s_best[MOST];
  __shared__ uint32_t s_seen[4];
  __shared__ Stats s_stats[4];
  __shared__ int s_count[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t row = WAVE ? (int64_t)blockIdx.x * 4 + wave : SPLIT ? blockIdx.x / a.parts : blockIdx.x;
  if (row >= a.n) return;  // whole waves, only where WAVE (no barriers)
  const int part = SPLIT ? (int)(blockIdx.x - row * a.parts) : 0;
  const T* x = (const T*)a.x + row * a.x_stride;
  const float c = a.scale * LOG2E;
  Candidates cand;
  cand.init(s_keys[TOP ? wave : 0], WAVE ? nullptr : s_seen, a.top);
  if (TOP && !WAVE) {
    if (threadIdx.x < 4) s_seen[threadIdx.x] = 0;
    __syncthreads();
  }
  Stats z = scan<T, TOP>(x, WAVE ? 0 : part * 4 + wave, WAVE ? 1 : SPLIT ? 4 * a.parts : 4, a.V, c, cand);
  z = lanes_join(z, c);
  if (TOP) cand.cut();
  const int64_t token = !SPLIT && a.token ? a.token[row] : -1;
  const bool has = token >= 0 && token < a.V;
  if constexpr (WAVE) {
    write_row(a, row, z, has ? (float)x[token] : 0.f, has, cand.buf, cand.count);
    return;
  }
  if (lane == 0) s_stats[wave] = z, s_count[wave] = cand.count;
  __syncthreads();
  int count = 0;
  if constexpr (TOP) count = best_of(s_keys, s_count, cand, s_best);
  if (wave) return;
#pragma unroll
  for (int w = 1; w < 4; ++w) z = join(z, s_stats[w], c);
  if constexpr (SPLIT) {
    if (lane == 0) ((Stats*)a.work)[row * a.parts + part] = z;
    if (TOP && lane < a.top) part_keys(a, row)[part * a.top + lane] = lane < count ? s_best[lane] : 0;
  } else {
    write_row(a, row, z, has ? (float)x[token] : 0.f, has, s_best, count);
  }
}

// Joins the parts of a row: a workgroup per row, whose waves rank a quarter of the keys each (one wave with all of them took 10.5 us
// for 16 parts with 20 alternatives).
template <typename T>
__global__ __launch_bounds__(256) void join_scores_kernel(ScoresArgs a) {
  __shared__ Key s_keys[4][CAP];
  __shared__ Key s_best[MOST];
  __shared__ int s_count[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t row = blockIdx.x;
  const Stats* p = (const Stats*)a.work + row * a.parts;
  const float c = a.scale * LOG2E;
  const Stats mine = lane < a.parts ? p[lane] : Stats{-INFINITY, 0.f, 0.f};  // (at most 64 parts)
  const int64_t token = a.token ? a.token[row] : -1;
  const bool has = token >= 0 && token < a.V;
  const float logit = has ? (float)((const T*)a.x + row * a.x_stride)[token] : 0.f;
  int count = 0;
  if (a.top) {
    Candidates cand;
    cand.init(s_keys[wave], nullptr, a.top);
    const Key* keys = part_keys(a, row);
    const int all = a.parts * a.top;
    for (int i = 64 * wave; i < all; i += 1024) {  // four loads at a time
      Key k[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) k[j] = i + 256 * j + lane < all ? keys[i + 256 * j + lane] : 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) cand.offer(k[j]);
    }
    cand.cut();
    if (lane == 0) s_count[wave] = cand.count;
    __syncthreads();
    count = best_of(s_keys, s_count, cand, s_best);
  }
  if (wave) return;
  write_row(a, row, lanes_join(mine, c), logit, has, s_best, count);
}

// Gradient: a workgroup takes SEGMENT elements of a row, or (WAVE: rows of up to SEGMENT / 4) each of its waves a row.  The
// gradients of the token's and the alternatives' own logits wait in LDS at their elements' places, eights of elements that hold one
// marked in a bitmap, so that an element is written once (the result may be the logits' own memory) and no other is looked at.
// (of 4096 elements where a row has no more: 16384 x 4096 in bf16 43 us, of 8192 64).
constexpr int SEGMENT = 8192;
template <typename T, bool WAVE, int LEN>
__global__ __launch_bounds__(256) void scores_back_kernel(ScoresBackArgs a) {
  constexpr int TPR = WAVE ? 64 : 256, WORDS = LEN / 8 / 32, STEPS = LEN / 8 / TPR;
  __shared__ __align__(16) float s_own[WAVE ? 4 : 1][LEN];
  __shared__ uint32_t s_bits[WAVE ? 4 : 1][WORDS];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, t = threadIdx.x % TPR, sub = WAVE ? wave : 0;
  const int64_t row = WAVE ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x / a.segments;
  if (row >= a.n) return;  // whole waves, only where WAVE (no barriers)
  const int first = WAVE ? 0 : (int)(blockIdx.x - row * a.segments) * LEN, end = (int)std::min<int64_t>((int64_t)first + LEN, a.V);
  auto sync = [] {
    if constexpr (WAVE) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    else __syncthreads();
  };
  const T* x = (const T*)a.x + row * a.x_stride;
  T* dx = (T*)a.dx + row * a.dx_stride;
  typename Vec8<T>::type raw[STEPS];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) raw[k] = load_logits(x, std::min(first + 8 * (t + k * TPR), end), end);
  // what is asked of special places, in every wave: lane j has alternative j
  const int64_t token = a.token ? a.token[row] : -1;
  float dlogp = a.dlogp ? a.dlogp[row] : 0.f, dtop = 0.f;
  const float dH = a.dentropy ? a.dentropy[row] : 0.f, lse = a.lse[row], H = a.dentropy ? a.entropy[row] : 0.f;
  int64_t id = -1;
  if (a.dtop && lane < a.top) id = a.top_id[row * a.top + lane], dtop = a.dtop[row * a.top + lane];
  const float dlse = a.dlse ? a.dlse[row] : 0.f;
  if (token < 0 || token >= a.V) dlogp = 0.f;
  if (id < 0 || id >= a.V) dtop = 0.f;
  const float A = dlse - dlogp - lanes_sum<64>(dtop) - (dH == 0.f ? 0.f : dH * H);
  for (int i = t; i < WORDS; i += TPR) s_bits[sub][i] = 0;
  sync();
  if (t < 64) {
    const auto mark = [&](bool is, int64_t v) {
      if (!is || v < first || v >= end) return;
      const int at = (int)(v - first) & ~7;
      atomicOr(&s_bits[sub][at >> 8], 1u << (at >> 3 & 31));
      *(f32x4*)&s_own[sub][at] = f32x4{};
      *(f32x4*)&s_own[sub][at + 4] = f32x4{};
    };
    mark(dtop != 0.f, id);
    mark(lane == 0 && dlogp != 0.f, token);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // An element may be asked for more than once (an id twice, the token as an alternative): each lane adds all that its element
    // is asked for, in order, and all of them write the same sum.
    float mine = 0.f, at_token = 0.f;
    if (a.dtop)
      for (int k = 0; k < a.top; ++k) {
        const int other = __builtin_amdgcn_readlane((int)id, k);  // (of an id outside, dtop is 0)
        const float d = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, dtop), k));
        mine += other == (int)id ? d : 0.f;
        at_token += other == (int)token ? d : 0.f;
      }
    if (dlogp != 0.f && id == token) mine += dlogp;
    if (dtop != 0.f && id >= first && id < end) s_own[sub][id - first] = mine;
    if (lane == 0 && dlogp != 0.f && token >= first && token < end) s_own[sub][token - first] = at_token + dlogp;
  }
  sync();
  // a row that nothing is asked of, or may be said in (-infinity alone), gets zeros, whatever it holds
  const bool none = lse == -INFINITY || (A == 0.f && dH == 0.f && dlogp == 0.f && !__any(dtop != 0.f));
#pragma unroll
  for (int q = 0; q < STEPS; ++q) {
    const int unit = t + q * TPR, i = first + 8 * unit;
    if (i >= end) break;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float logp = __builtin_fmaf((float)raw[q][j], a.scale, -lse), p = __builtin_amdgcn_exp2f(logp * LOG2E);
      v[j] = p * (A - dH * fmaxf(logp, -200.f));
    }
    if (s_bits[sub][unit >> 5] >> (unit & 31) & 1)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += s_own[sub][8 * unit + j];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = none ? 0.f : a.scale * v[j];
    store8(dx, i, end, v);
  }
}

template <typename F>
int with_type(dn_dtype dt, F&& f) {
  if (dt == DN_F32) return f(float{});
  if (dt == DN_F16) return f(_Float16{});
  return f(__bf16{});
}

// Which rows have a wave each, not a workgroup: those of up to SHORT logits (16384 x 1000 with 5 alternatives 19 us, else 61), and
// longer ones where there are seven for a CU and more, since fewer bounds are looked for and joined (with 5 alternatives 2000 x 50257 58
// us, else 64, 5000 x 50257 103 and 136, 16384 x 8192 67 and 120; without 5000 x 50257 92 and 107).  Of fewer, SIMDs without a row
// wait as long as the last one takes (1536 x 131072 117 us, else 100).
constexpr int SHORT = 2048, MANY = 1792;
bool wave_each(int64_t n, int32_t V) { return V <= SHORT || n >= MANY; }

}  // namespace

// Workgroups of a row: enough of them for the chip where there are few rows, of at least two blocks a wave.  The launch that joins
// them costs 3 us, so only long rows are split.  In parts and in one workgroup: with 20 alternatives 8 x 50257 takes 20 and 30 us, 400
// x 50257 31 and 35, 700 x 50257 48 and 38, 8 x 16384 20 and 17; without alternatives 8 x 50257 16 and 12, 8 x 131072 16 and 16.
int32_t scores_parts(int64_t n, int32_t V, int32_t top) {
  if (V <= (top ? 1 << 15 : 1 << 17) || n >= 512 || n == 0) return 1;
  return (int32_t)std::min<int64_t>({(1024 + n - 1) / n, V / (8 * WAVE_BLOCK), 64});
}
size_t scores_bytes(int64_t n, int32_t V, int32_t top) {
  const int64_t parts = scores_parts(n, V, top);
  return parts == 1 ? 0 : sizeof(Stats) * (size_t)((n * parts + 1) / 2 * 2) + sizeof(Key) * (size_t)(n * parts) * top;
}

int launch_token_scores(const ScoresArgs& all, dn_dtype dt, void* stream) {
  return with_type(dt, [&](auto v) {
    using T = decltype(v);
    const hipStream_t st = (hipStream_t)stream;
    const bool wave = wave_each(all.n, all.V);
    const int64_t most = MAX_LAUNCH_THREADS / 256 / all.parts * (wave ? 4 : 1);
    for (int64_t at = 0; at < all.n; at += most) {  // (more than one launch's rows: never split)
      ScoresArgs a = all;
      a.n = std::min(all.n - at, most);
      a.x = (const T*)all.x + at * all.x_stride;
      a.lse = all.lse + at;
      if (all.token) a.token = all.token + at;
      if (all.logp) a.logp = all.logp + at;
      if (all.entropy) a.entropy = all.entropy + at;
      if (all.top) a.top_id = all.top_id + at * all.top, a.top_logp = all.top_logp + at * all.top;
      const auto run = [&](auto top) {
        constexpr bool TOP = decltype(top)::value;
        if (wave)
          scores_kernel<T, true, false, TOP><<<dim3((unsigned)((a.n + 3) / 4)), 256, 0, st>>>(a);
        else if (a.parts == 1)
          scores_kernel<T, false, false, TOP><<<dim3((unsigned)a.n), 256, 0, st>>>(a);
        else
          scores_kernel<T, false, true, TOP><<<dim3((unsigned)(a.n * a.parts)), 256, 0, st>>>(a);
      };
      if (a.top) run(std::true_type{});
      else run(std::false_type{});
      if (const int err = (int)hipGetLastError()) return err;
      if (a.parts > 1) {
        join_scores_kernel<T><<<dim3((unsigned)a.n), 256, 0, st>>>(a);
        if (const int err = (int)hipGetLastError()) return err;
      }
    }
    return 0;
  });
}

int launch_token_scores_backward(const ScoresBackArgs& all, dn_dtype dt, void* stream) {
  return with_type(dt, [&](auto v) {
    using T = decltype(v);
    const bool wave = all.V <= SHORT;
    const bool half = all.V <= SEGMENT / 2;
    const int64_t segments = wave ? 1 : ((int64_t)all.V + SEGMENT - 1) / SEGMENT;
    const int64_t most = MAX_LAUNCH_THREADS / 256 / segments * (wave ? 4 : 1);
    for (int64_t at = 0; at < all.n; at += most) {
      ScoresBackArgs a = all;
      a.n = std::min(all.n - at, most), a.segments = (int32_t)segments;
      a.x = (const T*)all.x + at * all.x_stride, a.dx = (T*)all.dx + at * all.dx_stride;
      a.lse = all.lse + at;
      if (all.token) a.token = all.token + at;
      if (all.entropy) a.entropy = all.entropy + at;
      if (all.dlogp) a.dlogp = all.dlogp + at;
      if (all.dentropy) a.dentropy = all.dentropy + at;
      if (all.dlse) a.dlse = all.dlse + at;
      if (all.dtop) a.dtop = all.dtop + at * all.top, a.top_id = all.top_id + at * all.top;
      if (wave)
        scores_back_kernel<T, true, SHORT><<<dim3((unsigned)((a.n + 3) / 4)), 256, 0, (hipStream_t)stream>>>(a);
      else if (half)
        scores_back_kernel<T, false, SEGMENT / 2><<<dim3((unsigned)a.n), 256, 0, (hipStream_t)stream>>>(a);
      else
        scores_back_kernel<T, false, SEGMENT><<<dim3((unsigned)(a.n * segments)), 256, 0, (hipStream_t)stream>>>(a);
      if (const int err = (int)hipGetLastError()) return err;
    }
    return 0;
  });
}

}  // namespace head
}  // namespace dn
