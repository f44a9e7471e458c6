// psa_qk_norm_rope and its gradient: root-mean-square norm of queries and keys and rotary positions on the frame, row and
// column axes, in one pass over the data.
//
// For x of one token and head, 128 channels:  y = R(angles) (w * x * r),  r = 1 / sqrt(mean(x^2) + eps),  R a rotation of
// every pair of channels; the mean goes over the head's channels or over those of all heads of the token.  The gradient:
// g = R(-angles) dy, h = w * g, s = mean(h * x):  dx = r * (h - x * r^2 * s),  dw = sum of g * x * r.
//
// Bound by HBM: forward moves each value in and out once, the gradient x and dy in and dx out.  A group of eight lanes takes
// up to kRows rows (heads) of one token, 16 channels a lane; several groups share a token.  Blocks are persistent, and every
// thread copies what it needs of the block's next token into shared memory (cp.async) while it works on this one: loads are
// always in flight without holding registers, a second look at a row (the mean over all heads) costs no second read, and no
// thread waits for another's copies.  The next bound is the issue of instructions (some 100 a row in a first version that
// held rows in registers, 65 % of the issue slots at 44 % of HBM): eight lanes a row instead of 16 halve what is spent on addresses,
// sums over lanes and roots, arithmetic runs on packed pairs of 32-bit values, and cos and sin of a token's 64 pairs are computed
// once for all its rows of q and k, into shared memory, while the token before is worked on.
//
// Angles: position times frequency in 64 bits, as only the fraction of a turn counts and positions may be far; the distance
// to the nearest quarter turn then in 32 bits.  Sums, norms and rotations are in 32 bits, rounded once.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "psa_norm_rope.cuh"

namespace psa {

namespace {

constexpr int kRows = 2;          // rows (heads) of a token that one group takes (more than 64 heads: twice as many going forward)
constexpr int kLanes = 8;         // lanes of a group
constexpr int kPairs = kHeadDim / 2;
constexpr int kMaxThreads = 256;  // forward; backward twice as many (kMaxHeads / kRows groups)

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
__device__ __forceinline__ f2 negate(f2 a) { return a ^ 0x8000000080000000ull; }
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
// The same by way of shared memory: word i of a thread lies at i * blockDim words of 16 bytes from its first, where only this thread
// writes and reads.
template <class T>
__device__ __forceinline__ void copy_row(uint32_t to, const T* p, int c0, int c1) {
  constexpr int kVec = sizeof(T) / 2;
  const uint32_t step = blockDim.x * 16u;
#pragma unroll
  for (int i = 0; i < 2 * kVec; ++i)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + i * step), "l"(p + (i < kVec ? c0 : c1) + (i % kVec) * (16 / (int)sizeof(T))) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLater>   // all but the last kLater sets of copies have arrived
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLater) : "memory"); }
// Zeros in all of a thread's words, for the rows that it has no head for.
__device__ __forceinline__ void clear_rows(uint4* rows, int words) {
  for (int i = 0; i < words; ++i) rows[i * blockDim.x] = make_uint4(0u, 0u, 0u, 0u);
}
template <class T>
__device__ __forceinline__ Raw<T> read_row(const uint4* from) {
  Raw<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T); ++i) *reinterpret_cast<uint4*>(r.w + 4 * i) = from[i * blockDim.x];
  return r;
}
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
  int slot, part;      // token of the block, group of that token
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
  p.slot = group / a.parts;
  p.part = group - p.slot * a.parts;
  p.idle = p.slot >= a.slots;
  if (p.idle) p.slot = p.part = 0;   // (it looks at a token's turns like the others)
  return p;
}

// n / d for n below 2^31 (NormRopeArgs::Divisor).
__device__ __forceinline__ int divide(int n, const Divisor& d) { return d.m == 0u ? n >> d.shift : (int)(__umulhi((uint32_t)n, d.m) >> d.shift); }

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

// cos and sin of the 64 pairs of the block's tokens from `first` on into shared memory, [token][cos 64, sin 64]; 1 and 0 where nothing
// turns.  angles: quarter turns of every pair, {per index, at index 0}.
__device__ __forceinline__ void fill_turns(const NormRopeArgs& a, const double2* angles, int first, float* turns) {
  for (int e = (int)threadIdx.x; e < a.slots * kPairs; e += (int)blockDim.x) {
    const int slot = e / kPairs, p = e % kPairs, n = first + slot;
    if (n >= a.n_all || n < 0) continue;
    int b, i;
    token_of(a, n, b, i);
    const long long at = a.first_token + i;
    float c = 1.f, s = 0.f;
    if (p < a.pairs[2] && at < a.n_video) {
      const int j = (int)at, row = divide(j, a.by_w), t = divide(row, a.by_h);
      const int index = p < a.pairs[0] ? t : (p < a.pairs[1] ? row - t * a.H : j - row * a.W);
      const double2 angle = angles[p];
      const double quarters = __fma_rn(angle.x, (double)index, angle.y);
      // the nearest whole number of quarters, in the last bits of the sum (the host bounds positions far below 2^51)
      const double shifted = quarters + 6755399441055744.0;   // 1.5 * 2^52
      const int q = __double2loint(shifted);
      float x, y;
      quarter_turn((float)(quarters - (shifted - 6755399441055744.0)), x, y);
      c = q & 1 ? y : x;
      s = q & 1 ? x : y;
      c = __uint_as_float(__float_as_uint(c) ^ (uint32_t)((q + 1) & 2) << 30);
      s = __uint_as_float(__float_as_uint(s) ^ (uint32_t)(q & 2) << 30);
    }
    turns[slot * 2 * kPairs + p] = c;
    turns[slot * 2 * kPairs + kPairs + p] = s;
  }
}

// A lane's angles at its token, and which of its pairs turn (where none does a value that is not finite stays in its channel).
struct Turn {
  f2 c[4], s[4];
  uint32_t some;
};
template <bool kHalves>
__device__ __forceinline__ Turn turn_of(const NormRopeArgs& a, const float* from, bool video) {
  const int lane = (int)threadIdx.x & (kLanes - 1), p0 = (kHalves ? 8 : 4) * lane, p1 = kHalves ? p0 + 4 : p0 + 32;
  const float4 c0 = *reinterpret_cast<const float4*>(from + p0), c1 = *reinterpret_cast<const float4*>(from + p1),
               s0 = *reinterpret_cast<const float4*>(from + kPairs + p0), s1 = *reinterpret_cast<const float4*>(from + kPairs + p1);
  Turn t;
  t.c[0] = pack(c0.x, c0.y); t.c[1] = pack(c0.z, c0.w); t.c[2] = pack(c1.x, c1.y); t.c[3] = pack(c1.z, c1.w);
  t.s[0] = pack(s0.x, s0.y); t.s[1] = pack(s0.z, s0.w); t.s[2] = pack(s1.x, s1.y); t.s[3] = pack(s1.z, s1.w);
  auto bits = [&](int from) -> uint32_t { return (1u << max(0, min(4, a.pairs[2] - from))) - 1u; };
  t.some = video ? bits(p0) | bits(p1) << 4 : 0u;
  return t;
}

// Rotates the lane's pairs, by the opposite angles for kBack.  all: every pair of every lane of the warp turns.
template <bool kBack>
__device__ __forceinline__ Row rotate(const Turn& t, bool all, const Row& x) {
  Row y;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const f2 sa = kBack ? t.s[k] : negate(t.s[k]), sb = kBack ? negate(t.s[k]) : t.s[k];
    y.a[k] = fma(x.b[k], sa, mul(x.a[k], t.c[k]));
    y.b[k] = fma(x.a[k], sb, mul(x.b[k], t.c[k]));
  }
  if (!all) {
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

// Sum over the groups of a token, which every one of them gets; all threads of the block.  `buf`: one float a group, not
// written again before the next barrier.
__device__ __forceinline__ float token_sum(const NormRopeArgs& a, const Place& p, const float* buf) {
  const int lane = (int)threadIdx.x & (kLanes - 1);
  float x = 0.f;
  if (!p.idle)
    for (int j = lane; j < a.parts; j += kLanes) x += buf[p.slot * a.parts + j];
  return lanes_sum(x);
}

// Shared memory: frequencies, shared weights, the turns of two sets of tokens, sums of the groups, the rows of two sets of tokens.
struct Shared {
  double2* angles; // [64]
  float* weights;  // [2][128]
  float* turns;    // [2][tokens][cos 64, sin 64]
  float* sums;     // [2][2][groups]
  uint4* rows;     // [sets][words of a thread][threads], from this thread's on
};
__device__ __forceinline__ Shared carve(const NormRopeArgs& a, double* sm) {
  float* f = reinterpret_cast<float*>(sm + 2 * kPairs) + 2 * kHeadDim;
  const int n = a.slots * 2 * kPairs, groups = (int)blockDim.x / kLanes;
  return Shared{reinterpret_cast<double2*>(sm), f - 2 * kHeadDim, f, f + 2 * n, reinterpret_cast<uint4*>(f + 2 * n + 4 * groups) + threadIdx.x};
}
// What a block keeps: the pairs' angles, and weights that all heads share (of tensors t0 .. t1 - 1).
template <bool kHasNorm>
__device__ __forceinline__ void fill_constants(const NormRopeArgs& a, const Shared& sh, int t0, int t1) {
  for (int i = (int)threadIdx.x; i < kPairs; i += (int)blockDim.x) {
    const int axis = i < a.pairs[0] ? 0 : (i < a.pairs[1] ? 1 : 2);
    sh.angles[i] = make_double2(a.step[axis] * a.turns[i], a.origin[axis] * a.turns[i]);
  }
  if (kHasNorm && a.weight_head == 0) {
    for (int i = (int)threadIdx.x; i < (t1 - t0) * kHeadDim; i += (int)blockDim.x) {
      const int t = t0 + i / kHeadDim, c = i % kHeadDim;
      const void* w = a.weight[t];
      sh.weights[t * kHeadDim + c] = w == nullptr ? 1.f
                                     : a.weight_dtype == PSA_FP32 ? static_cast<const float*>(w)[c]
                                     : a.weight_dtype == PSA_FP16 ? __half2float(static_cast<const __half*>(w)[c])
                                                                  : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[c]);
    }
  }
}
// words: of 16 bytes, of a thread and one set of tokens.  Where two sets do not fit (more than 110 heads of fp32) there is one, which is
// copied when the tokens before have been worked on: 1; else 2.
constexpr size_t shared_bytes(int slots, int threads, int words, int sets) {
  return 2 * kPairs * sizeof(double) + 2 * kHeadDim * sizeof(float) + (size_t)(4 * slots * kPairs + 4 * (threads / kLanes)) * sizeof(float) + (size_t)sets * words * threads * 16;
}
int sets_of(int slots, int threads, int words) { return shared_bytes(slots, threads, words, 2) <= kMaxSmemBytes ? 2 : 1; }

// ------------------------------------------------------------------------------------------------ forward
template <class T, class O, int kNorm, bool kHalves>
__global__ void __launch_bounds__(kMaxThreads, sizeof(T) == 4 ? 2 : 3)   // (80 registers: 24 warps an SM)
norm_rope_kernel(const __grid_constant__ NormRopeArgs a) {
  constexpr int kWords = sizeof(T);   // 16-byte words of a row and lane
  extern __shared__ __align__(16) double sm[];
  const Shared sh = carve(a, sm);
  const Place p = place_of<kHalves>(a);
  const int groups = (int)blockDim.x / kLanes, group = (int)threadIdx.x / kLanes, stride = (int)gridDim.x * a.slots;
  const int tensors = a.in[1] != nullptr ? 2 : 1, per_group = a.rows;
  const int row_step = kWords * (int)blockDim.x, tensor_step = per_group * row_step, set_step = 2 * tensor_step;   // in shared memory
  const long long in_step = a.parts * a.in_head, out_step = a.parts * a.out_head;                                  // from a row to the next
  const uint32_t rows_shared = (uint32_t)__cvta_generic_to_shared(sh.rows);
  int first = (int)blockIdx.x * a.slots;   // token, batches behind one another
  // rows of the group at token n: row u is there if u * parts is below
  auto rows_of = [&](int n) -> int { return !p.idle && n < a.n_all && n >= 0 ? a.n_heads - p.part : 0; };
  // the token copied last: its number, where its first row is and goes
  int i = 0;
  long long in_at = 0, out_at = 0;
  const long long in_stride = stride * a.in_token, out_stride = stride * a.out_token;
  const bool one_batch = a.n_all == a.n_tokens;
  auto copy = [&](int n, int set, bool again) {
    const int rows = rows_of(n);
    if (again && one_batch) {
      i += stride;
      in_at += in_stride;
      out_at += out_stride;
    } else if (rows > 0) {
      int b;
      token_of(a, n, b, i);
      in_at = b * a.in_batch + i * a.in_token + p.part * a.in_head;
      out_at = b * a.out_batch + i * a.out_token + p.part * a.out_head;
    }
    const uint32_t to = rows_shared + (uint32_t)(set * set_step) * 16u;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (t == tensors) break;
      const T* x = static_cast<const T*>(a.in[t]) + in_at;
#pragma unroll
      for (int u = 0; u < 2 * kRows; ++u, x += in_step) {
        if (u == per_group) break;
        if (u * a.parts < rows) copy_row(to + (uint32_t)(t * tensor_step + u * row_step) * 16u, x, p.c0, p.c1);
      }
    }
  };
  if (per_group * a.parts != a.n_heads) clear_rows(sh.rows, a.sets * 2 * per_group * kWords);
  copy(first + p.slot, 0, false);
  copies_end();
  fill_constants<kNorm != PSA_NORM_NONE>(a, sh, 0, tensors);
  __syncthreads();
  fill_turns(a, sh.angles, first, sh.turns);
  for (int it = 0; first < a.n_all; ++it) {
    const int next = a.n_all - first > stride ? first + stride : a.n_all, rows = rows_of(first + p.slot);
    const int i_here = i;
    const long long out_here = out_at;
    const uint4* mine = sh.rows;
    if (a.sets == 2) {
      if (next < a.n_all) copy(next + p.slot, (it + 1) & 1, true);
      copies_end();
      copies_wait<1>();
      mine += (it & 1) * set_step;
    } else {
      copies_wait<0>();
    }
    float* sums = sh.sums + (it & 1) * 2 * groups;
    if constexpr (kNorm == PSA_NORM_TOKEN) {
      float ss[2] = {0.f, 0.f};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (t == tensors) break;
        for (int u = 0; u < per_group; ++u) {
          const Row x = row_of<T, kHalves>(read_row<T>(mine + t * tensor_step + u * row_step));
          ss[t] += dot(x, x);
        }
      }
      const float s = lanes_sum2(ss[0], ss[1]);
      if ((threadIdx.x & 3) == 0) sums[((threadIdx.x >> 2) & 1) * groups + group] = s;
    }
    __syncthreads();
    if (next < a.n_all) fill_turns(a, sh.angles, next, sh.turns + ((it + 1) & 1) * a.slots * 2 * kPairs);
    const Turn turn = turn_of<kHalves>(a, sh.turns + ((it & 1) * a.slots + p.slot) * 2 * kPairs, a.first_token + i_here < a.n_video);
    const bool all = __all_sync(0xffffffffu, turn.some == 255u);
#pragma unroll 1
    for (int t = 0; t < tensors; ++t) {
      float r = 1.f;
      if constexpr (kNorm == PSA_NORM_TOKEN) r = rsqrtf(token_sum(a, p, sums + t * groups) * a.inv_count + a.eps);
      O* to = static_cast<O*>(a.out[t]) + out_here;
      const uint4* from = mine + t * tensor_step;
      Row w;
      if (kNorm != PSA_NORM_NONE && a.weight_head == 0) w = weight_of<float, kHalves>(sh.weights, t * kHeadDim, p.c0, p.c1);
#pragma unroll 1
      for (int u = 0; u < per_group; ++u, from += row_step, to += out_step) {
        Row x = row_of<T, kHalves>(read_row<T>(from));
        if constexpr (kNorm == PSA_NORM_HEAD) r = rsqrtf(lanes_sum(dot(x, x)) * a.inv_count + a.eps);
        if (u * a.parts >= rows) continue;
        if constexpr (kNorm != PSA_NORM_NONE) {
          if (a.weight_head != 0) w = load_weight<kHalves>(a.weight[t], a.weight_dtype, (p.part + u * a.parts) * kHeadDim, p.c0, p.c1);
          x = times(times(x, w), r);
        }
        store_row<O, kHalves>(to, p.c0, p.c1, rotate<false>(turn, all, x));
      }
    }
    if (a.sets == 1 && next < a.n_all) {
      copy(next + p.slot, 0, true);
      copies_end();
    }
    first = next;
  }
}

// ------------------------------------------------------------------------------------------------ gradient
// Like the forward pass, one tensor a block (blockIdx.y).  The sums for dw of a group's rows (kHeadWeights), or of all of them
// together, stay in registers; every block leaves one partial sum per weight, which norm_rope_dw_kernel adds in a fixed order.
template <class T, class O, int kNorm, bool kHalves, bool kHeadWeights>
__global__ void __launch_bounds__(2 * kMaxThreads)
norm_rope_bwd_kernel(const __grid_constant__ NormRopeArgs a) {
  constexpr bool kHasNorm = kNorm != PSA_NORM_NONE;
  constexpr int kSums = kHeadWeights ? kRows : 1;
  constexpr int kWords = kHasNorm ? sizeof(T) : 0, kGradWords = sizeof(O);   // 16-byte words of a row and lane
  extern __shared__ __align__(16) double sm[];
  const Shared sh = carve(a, sm);
  const Place p = place_of<kHalves>(a);
  const int groups = (int)blockDim.x / kLanes, group = (int)threadIdx.x / kLanes, stride = (int)gridDim.x * a.slots, t = blockIdx.y;
  const int per_group = a.rows, x_words = kWords * (int)blockDim.x, row_step = (kWords + kGradWords) * (int)blockDim.x, set_step = per_group * row_step;
  const long long x_step = a.parts * a.in_head, g_step = a.parts * a.out_head, dx_step = a.parts * a.dx_head;   // from a row to the next
  const uint32_t rows_shared = (uint32_t)__cvta_generic_to_shared(sh.rows);
  int first = (int)blockIdx.x * a.slots;
  auto rows_of = [&](int n) -> int { return !p.idle && n < a.n_all && n >= 0 ? a.n_heads - p.part : 0; };
  // the token copied last: its number, where its first rows are and go
  int i = 0;
  const T* x_at = static_cast<const T*>(a.in[t]);
  const O* g_at = static_cast<const O*>(a.grad[t]);
  T* dx_at = static_cast<T*>(a.out[t]);
  const long long x_stride = stride * a.in_token, g_stride = stride * a.out_token, dx_stride = stride * a.dx_token;
  const bool one_batch = a.n_all == a.n_tokens;
  auto copy = [&](int n, int set, bool again) {   // x of a row, then dy
    const int rows = rows_of(n);
    if (again && one_batch) {
      i += stride;
      x_at += x_stride;
      g_at += g_stride;
      dx_at += dx_stride;
    } else if (rows > 0) {
      int b;
      token_of(a, n, b, i);
      x_at = static_cast<const T*>(a.in[t]) + (b * a.in_batch + i * a.in_token + p.part * a.in_head);
      g_at = static_cast<const O*>(a.grad[t]) + (b * a.out_batch + i * a.out_token + p.part * a.out_head);
      dx_at = static_cast<T*>(a.out[t]) + (b * a.dx_batch + i * a.dx_token + p.part * a.dx_head);
    }
    const T* x = x_at;
    const O* g = g_at;
    const uint32_t to = rows_shared + (uint32_t)(set * set_step) * 16u;
#pragma unroll
    for (int u = 0; u < kRows; ++u, x += x_step, g += g_step) {
      if (u * a.parts >= rows) break;
      if constexpr (kHasNorm) copy_row(to + (uint32_t)(u * row_step) * 16u, x, p.c0, p.c1);
      copy_row(to + (uint32_t)(u * row_step + x_words) * 16u, g, p.c0, p.c1);
    }
  };
  if (per_group * a.parts != a.n_heads) clear_rows(sh.rows, a.sets * per_group * (kWords + kGradWords));
  auto weight = [&](int u) -> Row {
    if constexpr (!kHeadWeights) return weight_of<float, kHalves>(sh.weights, t * kHeadDim, p.c0, p.c1);
    return load_weight<kHalves>(a.weight[t], a.weight_dtype, min(p.part + u * a.parts, a.n_heads - 1) * kHeadDim, p.c0, p.c1);
  };
  copy(first + p.slot, 0, false);
  copies_end();
  fill_constants<kHasNorm>(a, sh, t, t + 1);
  Row dw[kSums];
#pragma unroll
  for (int u = 0; u < kSums; ++u) dw[u] = Row{{0ull, 0ull, 0ull, 0ull}, {0ull, 0ull, 0ull, 0ull}};
  __syncthreads();
  fill_turns(a, sh.angles, first, sh.turns);
  for (int it = 0; first < a.n_all; ++it) {
    const int next = a.n_all - first > stride ? first + stride : a.n_all, rows = rows_of(first + p.slot);
    const int i_here = i;
    T* to = dx_at;
    const uint4* mine = sh.rows;
    if (a.sets == 2) {
      if (next < a.n_all) copy(next + p.slot, (it + 1) & 1, true);
      copies_end();
      copies_wait<1>();
      mine += (it & 1) * set_step;
    } else {
      copies_wait<0>();
    }
    __syncthreads();   // these tokens' turns are there, and nobody reads those of the token before any more
    const Turn turn = turn_of<kHalves>(a, sh.turns + ((it & 1) * a.slots + p.slot) * 2 * kPairs, a.first_token + i_here < a.n_video);
    const bool all = __all_sync(0xffffffffu, turn.some == 255u);
    Row w;
    if (kHasNorm && !kHeadWeights) w = weight(0);
    float ss = 0.f, hx = 0.f;
    if constexpr (kNorm == PSA_NORM_TOKEN) {
#pragma unroll 1
      for (int u = 0; u < per_group; ++u) {
        const Row x = row_of<T, kHalves>(read_row<T>(mine + u * row_step));
        const Row g = rotate<true>(turn, all, row_of<O, kHalves>(read_row<O>(mine + u * row_step + x_words)));
        if constexpr (kHeadWeights) w = weight(u);
        ss += dot(x, x);
        hx += dot(times(g, w), x);
      }
      float* sums = sh.sums + (it & 1) * 2 * groups;
      const float s = lanes_sum2(ss, hx);
      if ((threadIdx.x & 3) == 0) sums[((threadIdx.x >> 2) & 1) * groups + group] = s;
      if (next < a.n_all) fill_turns(a, sh.angles, next, sh.turns + ((it + 1) & 1) * a.slots * 2 * kPairs);
      __syncthreads();
      ss = token_sum(a, p, sums);
      hx = token_sum(a, p, sums + groups);
    } else if (next < a.n_all) {
      fill_turns(a, sh.angles, next, sh.turns + ((it + 1) & 1) * a.slots * 2 * kPairs);
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u, to += dx_step) {
      if (u == per_group) break;
      Row g = rotate<true>(turn, all, row_of<O, kHalves>(read_row<O>(mine + u * row_step + x_words)));
      if constexpr (kHasNorm) {
        const Row x = row_of<T, kHalves>(read_row<T>(mine + u * row_step));
        if constexpr (kHeadWeights) w = weight(u);
        const Row h = times(g, w);
        if constexpr (kNorm == PSA_NORM_HEAD) {
          ss = lanes_sum(dot(x, x));
          hx = lanes_sum(dot(h, x));
        }
        const float r = rsqrtf(ss * a.inv_count + a.eps), coef = -r * r * (hx * a.inv_count);
        const f2 rr = pack(r, r), cc = pack(coef, coef);
        if (u * a.parts < rows) {
          Row& d = dw[kHeadWeights ? u : 0];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            d.a[k] = fma(g.a[k], mul(x.a[k], rr), d.a[k]);
            d.b[k] = fma(g.b[k], mul(x.b[k], rr), d.b[k]);
            g.a[k] = mul(fma(x.a[k], cc, h.a[k]), rr);
            g.b[k] = mul(fma(x.b[k], cc, h.b[k]), rr);
          }
        }
      }
      if (u * a.parts < rows) store_row<T, kHalves>(to, p.c0, p.c1, g);
    }
    if (a.sets == 1 && next < a.n_all) {
      copy(next + p.slot, 0, true);
      copies_end();
    }
    first = next;
  }
  if (!kHasNorm || a.dw_part == nullptr) return;
  // the block's tokens, and for a shared weight its heads, in order
  float* dw_part = reinterpret_cast<float*>(sm);   // [groups][128] of one row
  float* to = a.dw_part + ((long long)t * gridDim.x + blockIdx.x) * a.weight_cols;
#pragma unroll
  for (int u = 0; u < kSums; ++u) {
    if (u > 0 && u * a.parts >= a.n_heads) break;
    __syncthreads();
    store_row<float, kHalves>(dw_part + group * kHeadDim, p.c0, p.c1, dw[u]);
    __syncthreads();
    if (!kHeadWeights) {
      for (int c = (int)threadIdx.x; c < kHeadDim; c += (int)blockDim.x) {
        float s = 0.f;
        for (int j = 0; j < groups; ++j) s += dw_part[j * kHeadDim + c];   // (idle groups left zeros)
        to[c] = s;
      }
    } else {
      for (int k = (int)threadIdx.x; k < a.parts * kHeadDim; k += (int)blockDim.x) {
        const int head = k / kHeadDim + u * a.parts;
        if (head >= a.n_heads) break;
        float s = 0.f;
        for (int j = 0; j < a.slots; ++j) s += dw_part[j * a.parts * kHeadDim + k];
        to[head * kHeadDim + k % kHeadDim] = s;
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

template <class T, class O, int kNorm, bool kHalves, bool kHeadWeights>
cudaError_t launch_bwd(NormRopeArgs& a, int threads, int blocks, int n_sms, int* launched, cudaStream_t st) {
  auto* kernel = norm_rope_bwd_kernel<T, O, kNorm, kHalves, kHeadWeights>;
  const int words = a.rows * (int)((kNorm != PSA_NORM_NONE ? sizeof(T) : 0) + sizeof(O));
  a.sets = sets_of(a.slots, threads, words);
  const size_t rows = shared_bytes(a.slots, threads, words, a.sets),
               sums = (size_t)(threads / kLanes) * kHeadDim * sizeof(float), smem = rows > sums ? rows : sums;
  const int tensors = a.grad[1] ? 2 : 1;
  int most;
  const cudaError_t e = blocks_at_once(kernel, threads, smem, n_sms, &most);
  if (e != cudaSuccess) return e;
  most /= tensors;
  if (most > kNormRopeBwdBlocks) most = kNormRopeBwdBlocks;
  *launched = blocks < most ? blocks : most;
  kernel<<<dim3(*launched, tensors), threads, smem, st>>>(a);
  return cudaGetLastError();
}

template <class T, class O, int kNorm, bool kHalves>
cudaError_t launch_typed(NormRopeArgs& a, bool backward, int threads, int blocks, int n_sms, int* launched, cudaStream_t st) {
  if (backward) {
    if constexpr (kNorm != PSA_NORM_NONE) {
      if (a.weight_head != 0) return launch_bwd<T, O, kNorm, kHalves, true>(a, threads, blocks, n_sms, launched, st);
    }
    return launch_bwd<T, O, kNorm, kHalves, false>(a, threads, blocks, n_sms, launched, st);
  }
  const int words = 2 * a.rows * (int)sizeof(T);
  a.sets = sets_of(a.slots, threads, words);
  const size_t smem = shared_bytes(a.slots, threads, words, a.sets);
  int most;
  const cudaError_t e = blocks_at_once(norm_rope_kernel<T, O, kNorm, kHalves>, threads, smem, n_sms, &most);
  if (e != cudaSuccess) return e;
  *launched = blocks < most ? blocks : most;
  norm_rope_kernel<T, O, kNorm, kHalves><<<*launched, threads, smem, st>>>(a);
  return cudaGetLastError();
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
  // Groups a token: so many that each has at most kRows heads; one a head where there are too few tokens to fill the GPU
  // with less.  Tokens a block: blocks of some 256 threads, whole warps.
  const int most = (backward ? 2 : 1) * kMaxThreads / kLanes;   // groups of a block
  const long long by_rows = (long long)a.n_all * ((a.n_heads + kRows - 1) / kRows);
  a.parts = by_rows * kLanes < (long long)n_sms * 1024 && a.n_heads <= most ? a.n_heads : (a.n_heads + kRows - 1) / kRows;
  if (a.parts > most) a.parts = (a.n_heads + 2 * kRows - 1) / (2 * kRows);
  a.rows = (a.n_heads + a.parts - 1) / a.parts;
  a.slots = 256 / (a.parts * kLanes);
  if (a.slots < 1) a.slots = 1;
  const int threads = (a.slots * a.parts * kLanes + 31) & ~31, blocks = (int)(((long long)a.n_all + a.slots - 1) / a.slots);
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
