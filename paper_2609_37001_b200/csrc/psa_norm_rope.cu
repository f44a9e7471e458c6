// psa_qk_norm_rope and its gradient: root-mean-square norm of queries and keys and rotary positions on the frame, row and
// column axes, in one pass over the data.
//
// For x of one token and head, 128 channels:  y = R(angles) (w * x * r),  r = 1 / sqrt(mean(x^2) + eps),  R a rotation of
// every pair of channels; the mean goes over the head's channels or over those of all heads of the token.  The gradient:
// g = R(-angles) dy, h = w * g, s = mean(h * x):  dx = r * (h - x * r^2 * s),  dw = sum of g * x * r.
//
// Bound by HBM: forward moves each value in and out once, the gradient x and dy in and dx out.  A group of eight lanes takes one
// head of a token, 16 channels a lane (or kRows = 2 heads, where there are more than 64, backward 56, as a block has no more threads); a block takes one or more
// tokens of q and k, or (more than 16 heads, backward 8) of one of them, all heads, so that a mean over all heads costs one read.
// Blocks are persistent: a group's head is always the same, whose weights, and sums for dw, stay in registers.  Two more warps of
// the block, the producers, copy the next tokens' rows into shared memory (cp.async, kMaxStages sets at most), and compute cos and
// sin of their 64 pairs, once for all heads.
// The next bounds are the waits between a token's steps (sums of lanes, the barrier, the sum over heads: with the mean over all heads
// 12 heads of 2 x 32,760 tokens reach 0.70 to 0.75 of the copy rate forward, 40 of 75,600 0.70 to 0.76 backward), and the issue of
// instructions (some 100 a row in a first version where every thread loaded its own rows and computed its own angles, 65 % of the
// issue slots at 44 % of HBM): what is done for a token and not for a channel is left to the producers, eight lanes a row instead of
// 16 halve what is spent on addresses, sums over lanes and roots, and arithmetic runs on packed pairs of 32-bit values.
//
// Angles: position times frequency in 64 bits, as only the fraction of a turn counts and positions may be far; the distance
// to the nearest quarter turn then in 32 bits.  Sums, norms and rotations are in 32 bits, rounded once.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "psa_norm_rope.cuh"

namespace psa {

namespace {

constexpr int kLanes = 8;         // lanes of a group
constexpr int kPairs = kHeadDim / 2;
constexpr int kMaxThreads = 512;   // besides the producers
constexpr int kProducers = 64;     // threads: a warp that copies and one for angles
// Sets of rows in shared memory.  24 heads of 115,456 tokens on one card, us with 2, 3 and 4 sets: 1,268, 529, 469.  (copies_wait tells no more than
// three sets in flight apart: with 5 to 8 sets there are no more copies on their way than with 4, and the time is the same.)
constexpr int kMaxStages = 4;
constexpr int kMaxGroups = kMaxThreads / kLanes, kMaxBwdGroups = (16 * 32 - kProducers) / kLanes;   // of one row each
// Registers.  Forward 80, which are 24 warps an SM: with 64 and 72, 24 heads of 115,456 tokens take 606 and 522 us instead of 486 (5.8
// TB/s, 0.89 of what a copy reaches).  The gradient's sums, weights, x and dy want 128, which are 16 warps: 40 heads of 75,600 tokens with the norm over all heads
// take 939 us, and with 80, 96 and 112 registers 1,249, 1,017 and 972.  (Two rows a group: 96, so that kMaxThreads + kProducers
// threads start.)
constexpr int kRegs = 80, kBwdRegs = 128, kTwoRowsRegs = 96;
// Threads of a block besides the producers, at most: with q and k (forward and backward), with several tokens.  (A token of few heads
// keeps the producers as busy as one of many.  12 heads of 32,760 tokens backward: 120 us with blocks of one tensor, 126 with both.  1.5 million rows a
// tensor backward, norm over a head, us with blocks of both and of one: 6 heads 557 and 626, 8 heads 549 and 461, 9 heads 609 and 578, 16 heads 636 and
// 452, so that 8 heads are on the slower side of the rule as it stands.)
constexpr int kBothThreads = 256, kBothBwdThreads = 128, kSmallThreads = 64;

// ------------------------------------------------------------------------------------------------ packed pairs
typedef unsigned long long f2;    // two fp32 values, one instruction for both
__device__ __forceinline__ f2 pack(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack(f2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ f2 fma(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f2 mul(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float sum(f2 a) {
  const float2 v = unpack(a);
  return v.x + v.y;
}

// A lane's 16 channels of a row: the first (a) and second (b) channels of its eight pairs.
struct Row {
  f2 a[4], b[4];
};

// The same as it lies in memory: two runs of eight channels.  Pairs of neighbouring channels: four pairs each; channels in halves:
// the first and the second channels.
template <class T>
struct Raw {
  static constexpr int kWords = 4 * sizeof(T);
  uint32_t w[kWords];
};
template <class T>
__device__ __forceinline__ void load_row(const T* p, int c0, int c1, Raw<T>& r) {
  constexpr int kVec = sizeof(T) / 2;   // 16-byte words of a run
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    *reinterpret_cast<uint4*>(r.w + 4 * i) = reinterpret_cast<const uint4*>(p + c0)[i];
    *reinterpret_cast<uint4*>(r.w + 4 * (kVec + i)) = reinterpret_cast<const uint4*>(p + c1)[i];
  }
}
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the last `later` sets of copies have arrived.
__device__ __forceinline__ void copies_wait(int later) {
  if (later >= 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (later == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}
// Of all threads; of all but the producers.
__device__ __forceinline__ void consumer_barrier() { asm volatile("bar.sync 1, %0;" ::"r"(blockDim.x - kProducers) : "memory"); }
__device__ __forceinline__ void block_barrier() { asm volatile("bar.sync 0;" ::: "memory"); }
__device__ __forceinline__ float2 pair_of(uint32_t w, const __nv_bfloat16*) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ float2 pair_of(uint32_t w, const __half*) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
template <class T, bool kHalves>
__device__ __forceinline__ Row row_of(const Raw<T>& r) {
  float2 v[8];   // in memory order
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = make_float2(__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1]));
    else v[i] = pair_of(r.w[i], static_cast<const T*>(nullptr));
  }
  Row x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (kHalves) {
      x.a[k] = pack(v[k].x, v[k].y);
      x.b[k] = pack(v[k + 4].x, v[k + 4].y);
    } else {
      x.a[k] = pack(v[2 * k].x, v[2 * k + 1].x);
      x.b[k] = pack(v[2 * k].y, v[2 * k + 1].y);
    }
  }
  return x;
}
__device__ __forceinline__ uint32_t word_of(float2 v, const __nv_bfloat16*) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(v.x, v.y);
  return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ uint32_t word_of(float2 v, const __half*) {
  const __half2 x = __floats2half2_rn(v.x, v.y);
  return *reinterpret_cast<const uint32_t*>(&x);
}
// The channels in memory order.
template <bool kHalves>
__device__ __forceinline__ void in_order(const Row& x, float2* v) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 a = unpack(x.a[k]), b = unpack(x.b[k]);
    v[kHalves ? k : 2 * k] = kHalves ? a : make_float2(a.x, b.x);
    v[kHalves ? k + 4 : 2 * k + 1] = kHalves ? b : make_float2(a.y, b.y);
  }
}
template <class T, bool kHalves>
__device__ __forceinline__ void store_row(T* p, int c0, int c1, const Row& x) {
  float2 v[8];
  in_order<kHalves>(x, v);
  uint32_t w[Raw<T>::kWords];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (sizeof(T) == 4) {
      w[2 * i] = __float_as_uint(v[i].x);
      w[2 * i + 1] = __float_as_uint(v[i].y);
    } else {
      w[i] = word_of(v[i], static_cast<const T*>(nullptr));
    }
  }
  constexpr int kVec = sizeof(T) / 2;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    reinterpret_cast<uint4*>(p + c0)[i] = *reinterpret_cast<const uint4*>(w + 4 * i);
    reinterpret_cast<uint4*>(p + c1)[i] = *reinterpret_cast<const uint4*>(w + 4 * (kVec + i));
  }
}

// Weights of the lane's channels, from element `at` on; 1 without weights.
template <class T, bool kHalves>
__device__ __forceinline__ Row weight_of(const void* base, int at, int c0, int c1) {
  Raw<T> raw;
  load_row(static_cast<const T*>(base) + at, c0, c1, raw);
  return row_of<T, kHalves>(raw);
}
template <bool kHalves>
__device__ __forceinline__ Row load_weight(const void* base, int dtype, int at, int c0, int c1) {
  if (base == nullptr) {
    const f2 one = pack(1.f, 1.f);
    return Row{{one, one, one, one}, {one, one, one, one}};
  }
  if (dtype == PSA_FP32) return weight_of<float, kHalves>(base, at, c0, c1);
  if (dtype == PSA_FP16) return weight_of<__half, kHalves>(base, at, c0, c1);
  return weight_of<__nv_bfloat16, kHalves>(base, at, c0, c1);
}

__device__ __forceinline__ Row times(const Row& x, const Row& w) {
  Row y;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    y.a[k] = mul(x.a[k], w.a[k]);
    y.b[k] = mul(x.b[k], w.b[k]);
  }
  return y;
}
__device__ __forceinline__ Row times(const Row& x, float r) {
  const f2 rr = pack(r, r);
  Row y;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    y.a[k] = mul(x.a[k], rr);
    y.b[k] = mul(x.b[k], rr);
  }
  return y;
}
// Two sums of products, added at the end: shorter chains.
__device__ __forceinline__ float dot(const Row& x, const Row& y) {
  f2 a = mul(x.a[0], y.a[0]), b = mul(x.b[0], y.b[0]);
#pragma unroll
  for (int k = 1; k < 4; ++k) {
    a = fma(x.a[k], y.a[k], a);
    b = fma(x.b[k], y.b[k], b);
  }
  return sum(a) + sum(b);
}

// Sum over the group's lanes.
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int m = kLanes / 2; m > 0; m >>= 1) x += __shfl_xor_sync(0xffffffffu, x, m);
  return x;
}
// The sums of two values over the group's lanes, x's in the lanes below 4 and y's in the others.
__device__ __forceinline__ float lanes_sum2(float x, float y) {
  const bool upper = (threadIdx.x & 4) != 0;
  float v = (upper ? y : x) + __shfl_xor_sync(0xffffffffu, upper ? x : y, 4);
  v += __shfl_xor_sync(0xffffffffu, v, 2);
  return v + __shfl_xor_sync(0xffffffffu, v, 1);
}

// ------------------------------------------------------------------------------------------------ places and angles
// A lane's place: which channels of a row it holds, and which group of which token of the block it belongs to.
struct Place {
  int c0, c1;          // its two runs of eight channels
  int set, part;       // token and tensor of the block, group of that one
  int slot, t;         // token of the block; tensor
  bool idle;           // beyond the last group of the last token
};
template <bool kHalves>
__device__ __forceinline__ Place place_of(const NormRopeArgs& a) {
  Place p;
  const int lane = (int)threadIdx.x & (kLanes - 1), group = (int)threadIdx.x / kLanes;
  if (kHalves) {
    // runs i and i + n of the n = R / 16 runs of either half; what is not rotated goes to the lanes behind, two runs each
    const int n = a.pairs[2] / 8;
    p.c0 = 8 * (lane < n ? lane : 2 * lane);   // (2 n + 2 (lane - n) = 2 lane)
    p.c1 = lane < n ? p.c0 + a.pairs[2] : p.c0 + 8;
  } else {
    p.c0 = 8 * lane;
    p.c1 = p.c0 + 64;
  }
  p.set = group / a.parts;
  p.part = group - p.set * a.parts;
  p.idle = p.set >= a.slots * a.tensors;
  if (p.idle) p.set = p.part = 0;   // (it looks at a token's turns like the others)
  p.slot = a.tensors == 2 ? p.set >> 1 : p.set;
  p.t = a.tensors == 2 ? p.set & 1 : (int)blockIdx.y;
  return p;
}

// Token n of all batch elements: batch element and token within it.
__device__ __forceinline__ void token_of(const NormRopeArgs& a, int n, int& b, int& i) {
  b = a.n_all == a.n_tokens ? 0 : divide(n, a.by_tokens);
  i = n - b * a.n_tokens;
}

// cos and sin of x quarter turns, |x| <= 1/2: Taylor polynomials of the angle up to its 11th and 12th power, whose next terms are
// below 2^-32.
__device__ __forceinline__ void quarter_turn(float x, float& c, float& s) {
  const float t = 1.57079632679489662f * x, t2 = t * t;
  float p = fmaf(t2, -2.50521083854417188e-8f, 2.75573192239858907e-6f);
  p = fmaf(t2, p, -1.98412698412698413e-4f);
  p = fmaf(t2, p, 8.33333333333333333e-3f);
  p = fmaf(t2, p, -1.66666666666666667e-1f);
  s = fmaf(t * t2, p, t);
  float q = fmaf(t2, 2.08767569878680990e-9f, -2.75573192239858907e-7f);
  q = fmaf(t2, q, 2.48015873015873016e-5f);
  q = fmaf(t2, q, -1.38888888888888889e-3f);
  q = fmaf(t2, q, 4.16666666666666667e-2f);
  q = fmaf(t2, q, -0.5f);
  c = fmaf(t2, q, 1.f);
}

// A pair's quarter turns: per index of its axis, and at index 0.
struct Angle {
  int axis;            // 3: it does not turn
  double per, at0;
};
__device__ __forceinline__ Angle angle_of(const NormRopeArgs& a, int p) {
  const int axis = p < a.pairs[0] ? 0 : (p < a.pairs[1] ? 1 : (p < a.pairs[2] ? 2 : 3));
  return Angle{axis, axis < 3 ? a.step[axis] * a.turns[p] : 0.0, axis < 3 ? a.origin[axis] * a.turns[p] : 0.0};
}
// cos, sin and -sin of pairs p and p + 32 of the block's tokens from `first` on into shared memory, [token][3][64]; 1 and 0 where nothing
// turns.
__device__ __forceinline__ void fill_turns(const NormRopeArgs& a, const Angle* angle, int p, int first, float* turns) {
  for (int slot = 0; slot < a.slots; ++slot, turns += 3 * kPairs) {
    const int n = first + slot;
    if (n >= a.n_all || n < 0) break;
    int b, i;
    token_of(a, n, b, i);
    const bool video = a.first_token + i < a.n_video;
    const int j = video ? (int)(a.first_token + i) : 0, row = divide(j, a.by_w), t = divide(row, a.by_h);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int index = angle[k].axis == 0 ? t : (angle[k].axis == 1 ? row - t * a.H : j - row * a.W);
      const double quarters = __fma_rn(angle[k].per, (double)index, angle[k].at0);
      // the nearest whole number of quarters, in the last bits of the sum (the host bounds positions far below 2^51)
      const double shifted = quarters + 6755399441055744.0;   // 1.5 * 2^52
      const int q = __double2loint(shifted);
      float x, y;
      quarter_turn((float)(quarters - (shifted - 6755399441055744.0)), x, y);
      float c = q & 1 ? y : x, s = q & 1 ? x : y;
      c = __uint_as_float(__float_as_uint(c) ^ (uint32_t)((q + 1) & 2) << 30);
      s = __uint_as_float(__float_as_uint(s) ^ (uint32_t)(q & 2) << 30);
      const bool turned = video && angle[k].axis < 3;
      turns[p + 32 * k] = turned ? c : 1.f;
      turns[kPairs + p + 32 * k] = turned ? s : 0.f;
      turns[2 * kPairs + p + 32 * k] = turned ? -s : 0.f;
    }
  }
}

// A lane's angles at its token, and which of its pairs turn (where none does a value that is not finite stays in its channel).
struct Turn {
  f2 c[4], s[4], m[4];   // cos, sin, -sin
  uint32_t some;
  bool all;              // every pair of every lane of the warp turns
};
// turns: the token's; some: the lane's pairs that turn at video tokens.
template <bool kHalves, bool kBack>
__device__ __forceinline__ Turn turn_of(const float* turns, uint32_t some, bool video) {
  const int lane = (int)threadIdx.x & (kLanes - 1), p0 = (kHalves ? 8 : 4) * lane, p1 = kHalves ? p0 + 4 : p0 + 32;
  Turn t;
  f2* to[3] = {t.c, t.s, t.m};
#pragma unroll
  for (int k = 0; k < (kBack ? 2 : 3); ++k) {
    const float4 x = *reinterpret_cast<const float4*>(turns + k * kPairs + p0), y = *reinterpret_cast<const float4*>(turns + k * kPairs + p1);
    to[k][0] = pack(x.x, x.y); to[k][1] = pack(x.z, x.w); to[k][2] = pack(y.x, y.y); to[k][3] = pack(y.z, y.w);
  }
  if (kBack) {   // (registers are scarce there)
#pragma unroll
    for (int k = 0; k < 4; ++k) t.m[k] = t.s[k] ^ 0x8000000080000000ull;
  }
  t.some = video ? some : 0u;
  t.all = __all_sync(0xffffffffu, t.some == 255u);
  return t;
}
template <bool kHalves>
__device__ __forceinline__ uint32_t pairs_that_turn(const NormRopeArgs& a) {
  const int lane = (int)threadIdx.x & (kLanes - 1), p0 = (kHalves ? 8 : 4) * lane, p1 = kHalves ? p0 + 4 : p0 + 32;
  auto bits = [&](int from) -> uint32_t { return (1u << max(0, min(4, a.pairs[2] - from))) - 1u; };
  return bits(p0) | bits(p1) << 4;
}

// Rotates the lane's pairs, by the opposite angles for kBack.
template <bool kBack>
__device__ __forceinline__ Row rotate(const Turn& t, const Row& x) {
  Row y;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    y.a[k] = fma(x.b[k], kBack ? t.s[k] : t.m[k], mul(x.a[k], t.c[k]));
    y.b[k] = fma(x.a[k], kBack ? t.m[k] : t.s[k], mul(x.b[k], t.c[k]));
  }
  if (!t.all) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool lo = (t.some >> (2 * k)) & 1u, hi = (t.some >> (2 * k + 1)) & 1u;
      const float2 xa = unpack(x.a[k]), xb = unpack(x.b[k]), ya = unpack(y.a[k]), yb = unpack(y.b[k]);
      y.a[k] = pack(lo ? ya.x : xa.x, hi ? ya.y : xa.y);
      y.b[k] = pack(lo ? yb.x : xb.x, hi ? yb.y : xb.y);
    }
  }
  return y;
}

// Sums (of two values) over the groups of a token's tensor, which every one of them gets.  `sums`: the token's, one entry a group.
__device__ __forceinline__ float2 token_sum(const float2* sums, int parts) {
  float2 v = make_float2(0.f, 0.f);
#pragma unroll 4
  for (int j = (int)threadIdx.x & (kLanes - 1); j < parts; j += kLanes) {
    const float2 x = sums[j];
    v.x += x.x;
    v.y += x.y;
  }
  return make_float2(lanes_sum(v.x), lanes_sum(v.y));
}
__device__ __forceinline__ float token_sum(const float* sums, int parts) {
  float v = 0.f;
#pragma unroll 4
  for (int j = (int)threadIdx.x & (kLanes - 1); j < parts; j += kLanes) v += sums[j];
  return lanes_sum(v);
}

// Shared memory: the turns of two sets of tokens, sums of the groups, the sets of rows ([token][head], x and then dy).
struct Shared {
  float* turns;      // [2][tokens][cos, sin, -sin][64]
  float2* sums;      // [2][groups]
  uint8_t* rows;
};
__device__ __forceinline__ Shared carve(const NormRopeArgs& a, uint8_t* sm) {
  float* turns = reinterpret_cast<float*>(sm);
  float2* sums = reinterpret_cast<float2*>(turns + 6 * a.slots * kPairs);
  return Shared{turns, sums, reinterpret_cast<uint8_t*>(sums + 2 * kMaxGroups)};
}
// bytes: of the rows of a set of tokens
constexpr size_t shared_bytes(int slots, int bytes, int stages) {
  return (size_t)6 * slots * kPairs * sizeof(float) + 2 * kMaxGroups * sizeof(float2) + (size_t)stages * bytes;
}

// The producers' part: what lies in front of the first barrier, between two, and behind the last one.  Every block barrier of the
// others has its like here: one a set of tokens in front of it, and (a single stage) one when it has been read.
template <class T, class O>
__device__ __forceinline__ void produce(const NormRopeArgs& a, const Shared& sh, bool x_too, bool g_too) {
  const int me = (int)threadIdx.x - ((int)blockDim.x - kProducers), stride = (int)gridDim.x * a.slots;
  const int x_bytes = x_too ? kHeadDim * (int)sizeof(T) : 0, token_bytes = a.n_heads * (x_bytes + (g_too ? kHeadDim * (int)sizeof(O) : 0));
  const int stages = a.stages;
  const uint32_t rows = (uint32_t)__cvta_generic_to_shared(sh.rows);
  // 16-byte piece `me % pieces` of every (32 / pieces)-th head
  auto copy_rows = [&](const auto* from, long long head_stride, uint32_t to) {
    using E = typename std::remove_cv<typename std::remove_pointer<decltype(from)>::type>::type;
    constexpr int kPieces = kHeadDim * (int)sizeof(E) / 16, kStep = 32 / kPieces;
    const int piece = me % kPieces, h0 = me / kPieces;
    const E* p = from + h0 * head_stride + piece * (16 / (int)sizeof(E));
    to += (uint32_t)(h0 * kHeadDim * (int)sizeof(E) + piece * 16);
    const long long step = kStep * head_stride;
#pragma unroll 4
    for (int h = h0; h < a.n_heads; h += kStep, p += step, to += kStep * kHeadDim * sizeof(E)) copy16(to, p);
  };
  auto issue = [&](int first, int stage) {
    if (first < a.n_all) {
      for (int slot = 0; slot < a.slots; ++slot) {
        const int n = first + slot;
        if (n >= a.n_all || n < 0) break;
        int b, i;
        token_of(a, n, b, i);
        for (int k = 0; k < a.tensors; ++k) {
          const int t = a.tensors == 2 ? k : (int)blockIdx.y;
          const uint32_t to = rows + (uint32_t)(((stage * a.slots + slot) * a.tensors + k) * token_bytes);
          if (x_too) copy_rows(static_cast<const T*>(a.in[t]) + (b * a.in_batch + i * a.in_token), a.in_head, to);
          if (g_too) copy_rows(static_cast<const O*>(a.grad[t]) + (b * a.out_batch + i * a.out_token), a.out_head, to + (uint32_t)(a.n_heads * x_bytes));
        }
      }
    }
    copies_end();
  };
  // first tokens of the sets to be copied, and computed with; a sum that passes 2^31 is the end, too
  auto after = [&](int first) -> int { return a.n_all - first > stride ? first + stride : a.n_all; };
  int first = (int)blockIdx.x * a.slots;
  if (me >= 32) {   // the second warp: angles, those of the next tokens while these are worked on
    const int p = me - 32;
    const Angle angle[2] = {angle_of(a, p), angle_of(a, p + 32)};
    fill_turns(a, angle, p, first, sh.turns);
    for (int it = 0; first < a.n_all; ++it) {
      block_barrier();
      if (stages == 1) block_barrier();
      first = after(first);
      if (first < a.n_all) fill_turns(a, angle, p, first, sh.turns + ((it + 1) & 1) * 3 * a.slots * kPairs);
    }
    return;
  }
  int ahead = first, stage = 0;
  const int depth = stages > 1 ? stages - 1 : 1;   // sets in flight
  for (int k = 0; k < depth; ++k, ahead = after(ahead)) issue(ahead, k);
  copies_wait(depth - 1);
  for (; first < a.n_all; first = after(first)) {
    block_barrier();   // the set is there, and nobody reads the one before any more
    if (stages > 1) {
      issue(ahead, stage == 0 ? stages - 1 : stage - 1);
      stage = stage + 1 == stages ? 0 : stage + 1;
    } else {
      block_barrier();   // it has been read
      issue(ahead, 0);
    }
    ahead = after(ahead);
    copies_wait(depth - 1);
  }
  copies_wait(0);
}

// ------------------------------------------------------------------------------------------------ forward
template <class T, class O, int kNorm, bool kHalves, int kRows>
__global__ void __maxnreg__(kRows == 1 ? kRegs : kTwoRowsRegs)
norm_rope_kernel(const __grid_constant__ NormRopeArgs a) {
  extern __shared__ __align__(16) uint8_t sm[];
  const Shared sh = carve(a, sm);
  if (threadIdx.x >= blockDim.x - kProducers) {
    produce<T, O>(a, sh, true, false);
    return;
  }
  const Place p = place_of<kHalves>(a);
  const int t = p.t, group = (int)threadIdx.x / kLanes, stride = (int)gridDim.x * a.slots;
  const uint32_t some = pairs_that_turn<kHalves>(a);
  Row w[kRows];
  if constexpr (kNorm != PSA_NORM_NONE) {
#pragma unroll
    for (int u = 0; u < kRows; ++u)
      w[u] = load_weight<kHalves>(a.weight[t], a.weight_dtype, a.weight_head ? min(p.part + u * a.parts, a.n_heads - 1) * kHeadDim : 0, p.c0, p.c1);
  }
  int n = (int)blockIdx.x * a.slots + p.slot, i = 0;   // token, batches behind one another; within its batch element
  O* to = static_cast<O*>(a.out[t]);                    // where its first row goes
  auto there = [&](int u) -> bool { return !p.idle && n < a.n_all && n >= 0 && (kRows == 1 || p.part + u * a.parts < a.n_heads); };
  if (there(0)) {
    int b;
    token_of(a, n, b, i);
    to += b * a.out_batch + i * a.out_token + p.part * a.out_head;
  }
  const int over = stride / a.n_tokens, step = stride - over * a.n_tokens;   // to the block's next tokens: batch elements, tokens
  const long long to_step = over * a.out_batch + step * a.out_token;
  const T* rows = reinterpret_cast<const T*>(sh.rows) + (p.set * a.n_heads + p.part) * kHeadDim;
  const int set_step = a.slots * a.tensors * a.n_heads * kHeadDim;
  int stage = 0;
  for (int it = 0, first = (int)blockIdx.x * a.slots; first < a.n_all; ++it) {
    block_barrier();
    const Turn turn = turn_of<kHalves, false>(sh.turns + ((it & 1) * a.slots + p.slot) * 3 * kPairs, some, a.first_token + i < a.n_video);
    Row x[kRows];
    float ss[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      Raw<T> raw;
      load_row(rows + stage * set_step + (kRows == 1 ? 0 : min(u * a.parts, a.n_heads - 1 - p.part) * kHeadDim), p.c0, p.c1, raw);
      x[u] = row_of<T, kHalves>(raw);
      if (kNorm != PSA_NORM_NONE) ss[u] = lanes_sum(dot(x[u], x[u]));
    }
    if constexpr (kNorm == PSA_NORM_TOKEN) {
      float* sums = reinterpret_cast<float*>(sh.sums) + (it & 1) * kMaxGroups;
      if ((threadIdx.x & (kLanes - 1)) == 0) sums[group] = kRows == 1 ? ss[0] : ss[0] + (p.part + a.parts < a.n_heads ? ss[kRows - 1] : 0.f);
      consumer_barrier();
      ss[0] = ss[kRows - 1] = token_sum(sums + p.set * a.parts, a.parts);
    }
    if (a.stages == 1) block_barrier();
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      if (!there(u)) continue;
      if constexpr (kNorm != PSA_NORM_NONE) x[u] = times(times(x[u], w[u]), rsqrtf(ss[u] * a.inv_count + a.eps));
      store_row<O, kHalves>(to + u * a.parts * a.out_head, p.c0, p.c1, rotate<false>(turn, x[u]));
    }
    first = a.n_all - first > stride ? first + stride : a.n_all;
    n = first + p.slot;
    i += step;
    to += to_step;
    if (i >= a.n_tokens) {
      i -= a.n_tokens;
      to += a.out_batch - a.n_tokens * a.out_token;
    }
    stage = stage + 1 == a.stages ? 0 : stage + 1;
  }
}

// ------------------------------------------------------------------------------------------------ gradient
// Like the forward pass.  Every block leaves one partial sum per weight, which norm_rope_dw_kernel adds in a fixed order, in 64 bits.  A thread's own sum,
// over the tokens of its block (of 75,600 some 1,000, where a tensor has 74 blocks), is in 32: 64 bits would take twice the registers, which are all in use.
// (It is off by a half step of 32 bits of the magnitudes for each token at most, by the root of that many as a rule.)
template <class T, class O, int kNorm, bool kHalves, int kRows>
__global__ void __maxnreg__(kRows == 1 ? kBwdRegs : kTwoRowsRegs)
norm_rope_bwd_kernel(const __grid_constant__ NormRopeArgs a) {
  constexpr bool kHasNorm = kNorm != PSA_NORM_NONE;
  extern __shared__ __align__(16) uint8_t sm[];
  const Shared sh = carve(a, sm);
  const int consumers = (int)blockDim.x - kProducers;
  float* dw_part = reinterpret_cast<float*>(sm);   // (at the end) [groups][128] of one row
  Row dw[kRows];
  const Place p = place_of<kHalves>(a);
  const int t = p.t, group = (int)threadIdx.x / kLanes;
  if ((int)threadIdx.x >= consumers) {
    produce<T, O>(a, sh, kHasNorm, true);
  } else {
    const int stride = (int)gridDim.x * a.slots;
    const uint32_t some = pairs_that_turn<kHalves>(a);
      Row w[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      dw[u] = Row{{0ull, 0ull, 0ull, 0ull}, {0ull, 0ull, 0ull, 0ull}};
      if (kHasNorm) w[u] = load_weight<kHalves>(a.weight[t], a.weight_dtype, a.weight_head ? min(p.part + u * a.parts, a.n_heads - 1) * kHeadDim : 0, p.c0, p.c1);
    }
    int n = (int)blockIdx.x * a.slots + p.slot, i = 0;
    T* to = static_cast<T*>(a.out[t]);
    auto there = [&](int u) -> bool { return !p.idle && n < a.n_all && n >= 0 && (kRows == 1 || p.part + u * a.parts < a.n_heads); };
    if (there(0)) {
      int b;
      token_of(a, n, b, i);
      to += b * a.dx_batch + i * a.dx_token + p.part * a.dx_head;
    }
    const int over = stride / a.n_tokens, step = stride - over * a.n_tokens;   // to the block's next tokens: batch elements, tokens
    const long long to_step = over * a.dx_batch + step * a.dx_token;
    const int x_bytes = kHasNorm ? kHeadDim * (int)sizeof(T) : 0, g_bytes = kHeadDim * (int)sizeof(O), token_bytes = a.n_heads * (x_bytes + g_bytes);
    const uint8_t* rows = sh.rows + p.set * token_bytes;
    int stage = 0;
    for (int it = 0, first = (int)blockIdx.x * a.slots; first < a.n_all; ++it) {
      block_barrier();
      Row x[kRows], g[kRows];
      float ss[kRows], hx[kRows];
      {
        const Turn turn = turn_of<kHalves, true>(sh.turns + ((it & 1) * a.slots + p.slot) * 3 * kPairs, some, a.first_token + i < a.n_video);
        const uint8_t* set = rows + stage * a.slots * a.tensors * token_bytes;
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
          const int head = kRows == 1 ? p.part : min(p.part + u * a.parts, a.n_heads - 1);
          Raw<O> raw_g;
          load_row(reinterpret_cast<const O*>(set + a.n_heads * x_bytes + head * g_bytes), p.c0, p.c1, raw_g);
          g[u] = rotate<true>(turn, row_of<O, kHalves>(raw_g));
          if constexpr (kHasNorm) {
            Raw<T> raw_x;
            load_row(reinterpret_cast<const T*>(set + head * x_bytes), p.c0, p.c1, raw_x);
            x[u] = row_of<T, kHalves>(raw_x);
            ss[u] = dot(x[u], x[u]);
            hx[u] = dot(times(g[u], w[u]), x[u]);
            if constexpr (kNorm == PSA_NORM_HEAD) {
              ss[u] = lanes_sum(ss[u]);
              hx[u] = lanes_sum(hx[u]);
            }
          }
        }
      }
      if constexpr (kNorm == PSA_NORM_TOKEN) {
        float2* sums = sh.sums + (it & 1) * kMaxGroups;
        const bool both = kRows > 1 && p.part + a.parts < a.n_heads;
        const float s = lanes_sum2(both ? ss[0] + ss[kRows - 1] : ss[0], both ? hx[0] + hx[kRows - 1] : hx[0]);
        if ((threadIdx.x & 3) == 0) reinterpret_cast<float*>(sums + group)[(threadIdx.x >> 2) & 1] = s;
        consumer_barrier();
        const float2 v = token_sum(sums + p.set * a.parts, a.parts);
        ss[0] = ss[kRows - 1] = v.x;
        hx[0] = hx[kRows - 1] = v.y;
      }
      if (a.stages == 1) block_barrier();
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        if (!there(u)) continue;
        if constexpr (kHasNorm) {
          const float r = rsqrtf(ss[u] * a.inv_count + a.eps), coef = -r * r * (hx[u] * a.inv_count);
          const f2 rr = pack(r, r), cc = pack(coef, coef);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            dw[u].a[k] = fma(g[u].a[k], mul(x[u].a[k], rr), dw[u].a[k]);
            dw[u].b[k] = fma(g[u].b[k], mul(x[u].b[k], rr), dw[u].b[k]);
            g[u].a[k] = mul(fma(x[u].a[k], cc, mul(g[u].a[k], w[u].a[k])), rr);
            g[u].b[k] = mul(fma(x[u].b[k], cc, mul(g[u].b[k], w[u].b[k])), rr);
          }
        }
        store_row<T, kHalves>(to + u * a.parts * a.dx_head, p.c0, p.c1, g[u]);
      }
      first = a.n_all - first > stride ? first + stride : a.n_all;
      n = first + p.slot;
      i += step;
      to += to_step;
      if (i >= a.n_tokens) {
        i -= a.n_tokens;
        to += a.dx_batch - a.n_tokens * a.dx_token;
      }
      stage = stage + 1 == a.stages ? 0 : stage + 1;
    }
  }
  if (!kHasNorm || a.dw_part == nullptr) return;
  // the block's tokens, and for a shared weight its heads, in order
  if (kRows > 1 && a.weight_head == 0) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      dw[0].a[k] = fma(dw[kRows - 1].a[k], pack(1.f, 1.f), dw[0].a[k]);
      dw[0].b[k] = fma(dw[kRows - 1].b[k], pack(1.f, 1.f), dw[0].b[k]);
    }
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    if (u > 0 && a.weight_head == 0) break;
    block_barrier();
    if ((int)threadIdx.x < consumers) store_row<float, kHalves>(dw_part + group * kHeadDim, p.c0, p.c1, dw[u]);
    block_barrier();
    for (int k = 0; k < a.tensors; ++k) {
      const int tensor = a.tensors == 2 ? k : (int)blockIdx.y, per = a.tensors * a.parts * kHeadDim;   // from a token's sums to the next one's
      float* to = a.dw_part + ((long long)tensor * gridDim.x + blockIdx.x) * a.weight_cols;
      const float* from = dw_part + k * a.parts * kHeadDim;
      for (int e = (int)threadIdx.x; e < (a.weight_head == 0 ? kHeadDim : a.parts * kHeadDim); e += (int)blockDim.x) {
        const int head = e / kHeadDim + u * a.parts;
        if (head >= a.n_heads) break;
        float sum = 0.f;
        for (int j = 0; j < a.slots; ++j)
          for (int h = 0; h < (a.weight_head == 0 ? a.parts : 1); ++h) sum += from[j * per + h * kHeadDim + e];
        to[head * kHeadDim + e % kHeadDim] = sum;
      }
    }
  }
}

constexpr int kDwCols = 32, kDwGroups = 32;
__global__ void __launch_bounds__(kDwCols * kDwGroups)
norm_rope_dw_kernel(const float* __restrict__ part, int n_part, int cols, float* __restrict__ q_dw, float* __restrict__ k_dw) {
  __shared__ double red[kDwGroups][kDwCols];
  const int c = blockIdx.x * kDwCols + threadIdx.x % kDwCols, grp = threadIdx.x / kDwCols;
  const float* from = part + (long long)blockIdx.y * n_part * cols + c;
  double s = 0.0;
#pragma unroll 4
  for (int i = grp; i < n_part; i += kDwGroups) s += (double)from[(long long)i * cols];
  red[grp][threadIdx.x % kDwCols] = s;
  __syncthreads();
  if (grp == 0) {
#pragma unroll
    for (int i = 1; i < kDwGroups; ++i) s += red[i][threadIdx.x];
    (blockIdx.y == 0 ? q_dw : k_dw)[c] = (float)s;
  }
}

// Blocks of a persistent launch: as many as run at once.  The answers of the occupancy calculator (a microsecond a question) are kept
// by kernel, block and shared memory size; calls hold the library's lock.
cudaError_t blocks_at_once(void (*kernel)(NormRopeArgs), int threads, size_t smem, int n_sms, int* blocks) {
  constexpr int kKept = 32;
  static struct { void (*kernel)(NormRopeArgs); int device, threads, smem, per_sm; } kept[kKept];
  static int n_kept = 0;
  int device;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  for (int i = 0; i < (n_kept < kKept ? n_kept : kKept); ++i)
    if (kept[i].kernel == kernel && kept[i].device == device && kept[i].threads == threads && kept[i].smem == (int)smem) {
      *blocks = kept[i].per_sm * n_sms;
      return cudaSuccess;
    }
  int per_sm = 0;
  if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxSmemBytes)) != cudaSuccess) return e;
  if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem)) != cudaSuccess) return e;
  if (per_sm < 1) return cudaErrorInvalidConfiguration;
  kept[n_kept++ % kKept] = {kernel, device, threads, (int)smem, per_sm};
  *blocks = per_sm * n_sms;
  return cudaSuccess;
}

template <class T, class O, int kNorm, bool kHalves, int kRows>
cudaError_t launch_rows(NormRopeArgs& a, bool backward, int threads, int blocks, int n_sms, int* launched, cudaStream_t st) {
  auto* kernel = backward ? norm_rope_bwd_kernel<T, O, kNorm, kHalves, kRows> : norm_rope_kernel<T, O, kNorm, kHalves, kRows>;
  // as many sets of rows as fit, beside as many blocks as there are registers for
  const int bytes = a.slots * a.tensors * a.n_heads * kHeadDim * (int)(backward ? (kNorm != PSA_NORM_NONE ? sizeof(T) : 0) + sizeof(O) : sizeof(T));
  const size_t sums = backward ? (size_t)((threads - kProducers) / kLanes) * kHeadDim * sizeof(float) : 0;
  const size_t share = kMaxSmemBytes / (65536 / ((kRows > 1 ? kTwoRowsRegs : backward ? kBwdRegs : kRegs) * threads)) - 1024;
  for (a.stages = kMaxStages; a.stages > 2 && shared_bytes(a.slots, bytes, a.stages) > share; --a.stages) {}
  while (a.stages > 1 && shared_bytes(a.slots, bytes, a.stages) > kMaxSmemBytes) --a.stages;
  const size_t rows = shared_bytes(a.slots, bytes, a.stages), smem = rows > sums ? rows : sums;
  int most;
  const cudaError_t e = blocks_at_once(kernel, threads, smem, n_sms, &most);
  if (e != cudaSuccess) return e;
  const int tensors = a.out[1] && a.tensors == 1 ? 2 : 1;   // each with blocks of its own
  most = most > tensors ? most / tensors : 1;
  if (backward && most > kNormRopeBwdBlocks) most = kNormRopeBwdBlocks;
  *launched = blocks < most ? blocks : most;
  kernel<<<dim3(*launched, tensors), threads, smem, st>>>(a);
  return cudaGetLastError();
}

template <class T, class O, int kNorm, bool kHalves>
cudaError_t launch_typed(NormRopeArgs& a, bool backward, int threads, int blocks, int n_sms, int* launched, cudaStream_t st) {
  return a.parts == a.n_heads ? launch_rows<T, O, kNorm, kHalves, 1>(a, backward, threads, blocks, n_sms, launched, st)
                              : launch_rows<T, O, kNorm, kHalves, 2>(a, backward, threads, blocks, n_sms, launched, st);
}
template <class T, class O, int kNorm>
cudaError_t launch_pairs(NormRopeArgs& a, bool halves, bool backward, int threads, int blocks, int n_sms, int* launched, cudaStream_t st) {
  return halves ? launch_typed<T, O, kNorm, true>(a, backward, threads, blocks, n_sms, launched, st)
                : launch_typed<T, O, kNorm, false>(a, backward, threads, blocks, n_sms, launched, st);
}
template <class T, class O>
cudaError_t launch_norm(NormRopeArgs& a, int norm, bool halves, bool backward, int threads, int blocks, int n_sms, int* launched, cudaStream_t st) {
  switch (norm) {
    case PSA_NORM_HEAD: return launch_pairs<T, O, PSA_NORM_HEAD>(a, halves, backward, threads, blocks, n_sms, launched, st);
    case PSA_NORM_TOKEN: return launch_pairs<T, O, PSA_NORM_TOKEN>(a, halves, backward, threads, blocks, n_sms, launched, st);
    default: return launch_pairs<T, O, PSA_NORM_NONE>(a, halves, backward, threads, blocks, n_sms, launched, st);
  }
}

}  // namespace

cudaError_t launch_norm_rope(NormRopeArgs& a, const psa_qk& prob, bool halves, bool backward, int n_sms, float* q_dw, float* k_dw, cudaStream_t st,
                             int* launches) {
  // Groups a token: one a head, or one for two (1.5 million rows a tensor, norm over a head, of the copy rate: 64 heads forward 0.83, 65 to 128
  // heads 0.54 to 0.63; 56 heads backward 0.84, 57 to 128 heads 0.34 to 0.38).  Tokens a block: one, of few heads as many as make kSmallThreads threads;
  // whole warps.
  a.parts = a.n_heads <= (backward ? kMaxBwdGroups : kMaxGroups) ? a.n_heads : (a.n_heads + 1) / 2;
  a.tensors = a.out[1] && 2 * a.parts * kLanes <= (backward ? kBothBwdThreads : kBothThreads) ? 2 : 1;
  a.slots = kSmallThreads / (a.tensors * a.parts * kLanes);
  if (a.slots < 1) a.slots = 1;
  const int threads = ((a.slots * a.tensors * a.parts * kLanes + 31) & ~31) + kProducers, blocks = (int)(((long long)a.n_all + a.slots - 1) / a.slots);
  int launched = 0;
  cudaError_t e;
  const int in = prob.dtype, out = prob.out_dtype;
  if (in == PSA_BF16) e = launch_norm<__nv_bfloat16, __nv_bfloat16>(a, prob.norm, halves, backward, threads, blocks, n_sms, &launched, st);
  else if (in == PSA_FP16 && out == PSA_FP16) e = launch_norm<__half, __half>(a, prob.norm, halves, backward, threads, blocks, n_sms, &launched, st);
  else if (in == PSA_FP16) e = launch_norm<__half, __nv_bfloat16>(a, prob.norm, halves, backward, threads, blocks, n_sms, &launched, st);
  else if (out == PSA_FP32) e = launch_norm<float, float>(a, prob.norm, halves, backward, threads, blocks, n_sms, &launched, st);
  else e = launch_norm<float, __nv_bfloat16>(a, prob.norm, halves, backward, threads, blocks, n_sms, &launched, st);
  if (e != cudaSuccess) return e;
  ++*launches;
  if (backward && a.dw_part != nullptr) {
    norm_rope_dw_kernel<<<dim3(a.weight_cols / kDwCols, k_dw ? 2 : 1), kDwCols * kDwGroups, 0, st>>>(a.dw_part, launched, a.weight_cols, q_dw, k_dw);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

}  // namespace psa
