// psa_qk_norm_rope and its gradient: root-mean-square norm of queries and keys and rotary positions on the frame, row and
// column axes, in one pass over the data.
//
// For x of one token and head, 128 channels:  y = R(angles) (w * x * r),  r = 1 / sqrt(mean(x^2) + eps),  R a rotation of
// every pair of channels; the mean goes over the head's channels or over those of all heads of the token.  The gradient:
// g = R(-angles) dy, h = w * g, s = mean(h * x):  dx = r * (h - x * r^2 * s),  dw = sum of g * x * r.
//
// Bound by HBM: forward moves each value in and out once, the gradient x and dy in and dx out.  A half warp holds up to
// kRows rows (heads) of one token, 8 channels a lane, all in registers from load to store, so that also a mean over all
// heads costs one read; several half warps share a token.  A lane's four angles serve all its rows, of q and of k: they are
// computed where they are used (no table to read), the position times the frequency in 64 bits, as only the fraction of
// a turn counts and positions may be far, then 32 bits.  Sums, norms and rotations are in 32 bits, rounded once.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "psa_norm_rope.cuh"

namespace psa {

namespace {

constexpr int kRows = 4;          // rows (heads) of a token in one half warp's registers
constexpr int kLanes = 16;        // lanes a row
constexpr int kMaxThreads = 512;  // kMaxHeads / kRows half warps

template <class T>
struct Io {   // eight channels of a row as they lie in memory
  static constexpr int kWords = 2 * sizeof(T);
};

__device__ __forceinline__ float2 pair_of(uint32_t w, const __nv_bfloat16*) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ float2 pair_of(uint32_t w, const __half*) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ uint32_t word_of(float a, float b, const __nv_bfloat16*) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t word_of(float a, float b, const __half*) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// The two groups of four channels of a lane are neighbours (pairs of neighbouring channels), or lie half of the rotated
// channels apart.
template <class T, bool kHalves>
__device__ __forceinline__ void load_row(const T* p, int c0, int c1, uint32_t* w) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(p + c0);
    *reinterpret_cast<uint4*>(w + 4) = *reinterpret_cast<const uint4*>(p + c1);
  } else if constexpr (kHalves) {
    *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(p + c0);
    *reinterpret_cast<uint2*>(w + 2) = *reinterpret_cast<const uint2*>(p + c1);
  } else {
    *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(p + c0);
  }
}
template <class T>
__device__ __forceinline__ void unpack_row(const uint32_t* w, float* v) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = pair_of(w[i], static_cast<const T*>(nullptr));
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
}
template <class T, bool kHalves>
__device__ __forceinline__ void store_row(T* p, int c0, int c1, const float* v) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p + c0) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + c1) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = word_of(v[2 * i], v[2 * i + 1], static_cast<const T*>(nullptr));
    if constexpr (kHalves) {
      *reinterpret_cast<uint2*>(p + c0) = make_uint2(w[0], w[1]);
      *reinterpret_cast<uint2*>(p + c1) = make_uint2(w[2], w[3]);
    } else {
      *reinterpret_cast<uint4*>(p + c0) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// Weights of the lane's channels, of `head` where every head has its own; 1 without weights.
template <bool kHalves>
__device__ __forceinline__ void load_weight(const void* base, int dtype, long long at, int c0, int c1, float* w) {
  if (base == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
    return;
  }
  uint32_t raw[8];
  if (dtype == PSA_FP32) {
    load_row<float, kHalves>(static_cast<const float*>(base) + at, c0, c1, raw);
    unpack_row<float>(raw, w);
  } else if (dtype == PSA_FP16) {
    load_row<__half, kHalves>(static_cast<const __half*>(base) + at, c0, c1, raw);
    unpack_row<__half>(raw, w);
  } else {
    load_row<__nv_bfloat16, kHalves>(static_cast<const __nv_bfloat16*>(base) + at, c0, c1, raw);
    unpack_row<__nv_bfloat16>(raw, w);
  }
}

// Sum over the half warp's lanes.
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int m = kLanes / 2; m > 0; m >>= 1) x += __shfl_xor_sync(0xffffffffu, x, m);
  return x;
}

// A lane's place: which channels of a row it holds, and which half warp of which token of the block it belongs to.
struct Place {
  int c0, c1;          // its two groups of four channels
  int slot, part;      // token of the block, half warp of that token
  bool idle;           // beyond the last half warp of the last token
};
template <bool kHalves>
__device__ __forceinline__ Place place_of(const NormRopeArgs& a) {
  Place p;
  const int lane = (int)threadIdx.x & (kLanes - 1), half = (int)threadIdx.x / kLanes;
  if (kHalves) {
    // groups g and g + n of the n = R / 8 groups of either half; what is not rotated goes to the lanes behind, two groups each
    const int n = a.pairs[2] / 4;
    p.c0 = 4 * (lane < n ? lane : 2 * lane);   // (2 n + 2 (lane - n) = 2 lane)
    p.c1 = lane < n ? p.c0 + a.pairs[2] : p.c0 + 4;
  } else {
    p.c0 = 8 * lane;
    p.c1 = p.c0 + 4;
  }
  p.slot = half / a.parts;
  p.part = half - p.slot * a.parts;
  p.idle = p.slot >= a.slots;
  return p;
}

// cos and sin of the lane's four pairs (4 lane .. 4 lane + 3, in either order of channels) at token `i` of the sequence; pairs and
// tokens that are not rotated have *turned bit k of 0.
struct Turn {
  float cos[4], sin[4];
  uint32_t turned;
};
__device__ __forceinline__ Turn turn_at(const NormRopeArgs& a, long long i) {
  Turn r;
  r.turned = 0;
  const int p0 = 4 * ((int)threadIdx.x & (kLanes - 1));
  const bool video = i < a.n_video;
  const int j = video ? (int)i : 0, row = j / a.W, t = row / a.H;
  const int at[3] = {t, row - t * a.H, j - row * a.W};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int p = p0 + k, axis = p < a.pairs[0] ? 0 : (p < a.pairs[1] ? 1 : 2);
    r.cos[k] = 1.f;
    r.sin[k] = 0.f;
    if (video && p < a.pairs[2]) {
      r.turned |= 1u << k;
      const double turns = fma(axis == 0 ? a.step[0] : (axis == 1 ? a.step[1] : a.step[2]), (double)(axis == 0 ? at[0] : (axis == 1 ? at[1] : at[2])),
                               axis == 0 ? a.origin[0] : (axis == 1 ? a.origin[1] : a.origin[2])) * a.turns[p];
      // nearest quarter turn in 64 bits; the rest, at most 1/8 turn, keeps its relative precision in 32
      const double quarters = 4.0 * (turns - rint(turns)), q = rint(quarters);
      float s, c;
      sincospif(0.5f * (float)(quarters - q), &s, &c);
      const int n = (int)q & 3;
      r.cos[k] = n == 0 ? c : (n == 1 ? -s : (n == 2 ? -c : s));
      r.sin[k] = n == 0 ? s : (n == 1 ? c : (n == 2 ? -s : -c));
    }
  }
  return r;
}

// Rotates the lane's pairs, by the opposite angles for kBack.
template <bool kHalves, bool kBack>
__device__ __forceinline__ void rotate(const Turn& t, float* v) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = kHalves ? k : 2 * k, j = kHalves ? k + 4 : 2 * k + 1;
    const float c = t.cos[k], s = kBack ? -t.sin[k] : t.sin[k], x = v[i], y = v[j];
    const bool turned = (t.turned >> k) & 1u;   // (a value that is not finite stays where it is)
    v[i] = turned ? x * c - y * s : x;
    v[j] = turned ? x * s + y * c : y;
  }
}

// Sum over the half warps of a token, which every one of them gets; all threads of the block.  `buf`: one float a half warp.
__device__ __forceinline__ float token_sum(const NormRopeArgs& a, const Place& p, float mine, float* buf) {
  const int lane = (int)threadIdx.x & (kLanes - 1);
  if (lane == 0) buf[threadIdx.x / kLanes] = mine;
  __syncthreads();
  float x = 0.f;
  if (!p.idle)
    for (int j = lane; j < a.parts; j += kLanes) x += buf[p.slot * a.parts + j];
  return lanes_sum(x);
}

// ------------------------------------------------------------------------------------------------ forward
template <class T, class O, int kNorm, bool kHalves>
__global__ void __launch_bounds__(kMaxThreads)
norm_rope_kernel(const __grid_constant__ NormRopeArgs a) {
  constexpr int kWords = Io<T>::kWords;
  __shared__ float sums[2][kMaxThreads / kLanes];
  const Place p = place_of<kHalves>(a);
  const long long n = (long long)blockIdx.x * a.slots + p.slot;   // token, batches behind one another
  const bool have = !p.idle && n < a.n_all;
  const int b = have ? (int)(n / a.n_tokens) : 0;
  const long long i = have ? n - (long long)b * a.n_tokens : 0;
  uint32_t raw[2][kRows][kWords];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const T* from = static_cast<const T*>(a.in[t]) + b * a.in_batch + i * a.in_token;
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int head = p.part + u * a.parts;
      if (have && a.in[t] != nullptr && head < a.n_heads) {
        load_row<T, kHalves>(from + head * a.in_head, p.c0, p.c1, raw[t][u]);
      } else {
#pragma unroll
        for (int w = 0; w < kWords; ++w) raw[t][u][w] = 0u;
      }
    }
  }
  const Turn turn = turn_at(a, a.first_token + i);
  float r_token[2] = {1.f, 1.f};
  if constexpr (kNorm == PSA_NORM_TOKEN) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float ss = 0.f;
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        float v[8];
        unpack_row<T>(raw[t][u], v);
#pragma unroll
        for (int c = 0; c < 8; ++c) ss = fmaf(v[c], v[c], ss);
      }
      r_token[t] = rsqrtf(token_sum(a, p, lanes_sum(ss), sums[t]) * a.inv_count + a.eps);
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if (a.in[t] == nullptr) continue;
    O* to = static_cast<O*>(a.out[t]) + b * a.out_batch + i * a.out_token;
    float w[8];
    if (kNorm != PSA_NORM_NONE && a.weight_head == 0) load_weight<kHalves>(a.weight[t], a.weight_dtype, 0, p.c0, p.c1, w);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int head = p.part + u * a.parts;
      if (u > 0 && u * a.parts >= a.n_heads) break;
      float v[8];
      unpack_row<T>(raw[t][u], v);
      float r = r_token[t];
      if constexpr (kNorm == PSA_NORM_HEAD) {
        float ss = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) ss = fmaf(v[c], v[c], ss);
        r = rsqrtf(lanes_sum(ss) * a.inv_count + a.eps);
      }
      if (!have || head >= a.n_heads) continue;
      if constexpr (kNorm != PSA_NORM_NONE) {
        if (a.weight_head != 0) load_weight<kHalves>(a.weight[t], a.weight_dtype, (long long)head * kHeadDim, p.c0, p.c1, w);
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = v[c] * r * w[c];
      }
      rotate<kHalves, false>(turn, v);
      store_row<O, kHalves>(to + head * a.out_head, p.c0, p.c1, v);
    }
  }
}

// ------------------------------------------------------------------------------------------------ gradient
// Blocks (x of each tensor y) walk over the tokens and keep the sums for dw of their rows in registers; every block leaves one
// partial sum per weight, which norm_rope_dw_kernel adds in a fixed order.
template <class T, class O, int kNorm, bool kHalves>
__global__ void __launch_bounds__(kMaxThreads)
norm_rope_bwd_kernel(const __grid_constant__ NormRopeArgs a) {
  constexpr int kWords = Io<T>::kWords, kGradWords = Io<O>::kWords;
  __shared__ float sums[2][kMaxThreads / kLanes];
  extern __shared__ float dw_part[];   // [half warps][128] of one row
  const Place p = place_of<kHalves>(a);
  const int t = blockIdx.y;
  float w[8], dw[kRows][8];
#pragma unroll
  for (int u = 0; u < kRows; ++u)
#pragma unroll
    for (int c = 0; c < 8; ++c) dw[u][c] = 0.f;
  if (kNorm != PSA_NORM_NONE && a.weight_head == 0) load_weight<kHalves>(a.weight[t], a.weight_dtype, 0, p.c0, p.c1, w);
  for (long long first = (long long)blockIdx.x * a.slots; first < a.n_all; first += (long long)gridDim.x * a.slots) {
    const long long n = first + p.slot;
    const bool have = !p.idle && n < a.n_all;
    const int b = have ? (int)(n / a.n_tokens) : 0;
    const long long i = have ? n - (long long)b * a.n_tokens : 0;
    uint32_t raw_x[kRows][kWords], raw_g[kRows][kGradWords];
    const T* x_from = static_cast<const T*>(a.in[t]) + b * a.in_batch + i * a.in_token;
    const O* g_from = static_cast<const O*>(a.grad[t]) + b * a.out_batch + i * a.out_token;
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int head = p.part + u * a.parts;
      const bool row = have && head < a.n_heads;
      if (row) load_row<O, kHalves>(g_from + head * a.out_head, p.c0, p.c1, raw_g[u]);
      if (kNorm != PSA_NORM_NONE && row) load_row<T, kHalves>(x_from + head * a.in_head, p.c0, p.c1, raw_x[u]);
      if (!row) {
#pragma unroll
        for (int k = 0; k < kGradWords; ++k) raw_g[u][k] = 0u;
#pragma unroll
        for (int k = 0; k < kWords; ++k) raw_x[u][k] = 0u;
      }
    }
    const Turn turn = turn_at(a, a.first_token + i);
    float ss = 0.f, hx = 0.f;
    if constexpr (kNorm == PSA_NORM_TOKEN) {
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int head = p.part + u * a.parts;
        if (head >= a.n_heads) break;
        float x[8], g[8];
        unpack_row<T>(raw_x[u], x);
        unpack_row<O>(raw_g[u], g);
        rotate<kHalves, true>(turn, g);
        if (a.weight_head != 0) load_weight<kHalves>(a.weight[t], a.weight_dtype, (long long)head * kHeadDim, p.c0, p.c1, w);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          ss = fmaf(x[c], x[c], ss);
          hx = fmaf(g[c] * w[c], x[c], hx);
        }
      }
      __syncthreads();   // (the sums of the token before have been read)
      ss = token_sum(a, p, lanes_sum(ss), sums[0]);
      hx = token_sum(a, p, lanes_sum(hx), sums[1]);
    }
    T* to = static_cast<T*>(a.out[t]) + b * a.dx_batch + i * a.dx_token;
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int head = p.part + u * a.parts;
      if (u > 0 && u * a.parts >= a.n_heads) break;
      const bool row = have && head < a.n_heads;
      float x[8], g[8];
      unpack_row<O>(raw_g[u], g);
      rotate<kHalves, true>(turn, g);
      if constexpr (kNorm != PSA_NORM_NONE) {
        unpack_row<T>(raw_x[u], x);
        if (a.weight_head != 0 && row) load_weight<kHalves>(a.weight[t], a.weight_dtype, (long long)head * kHeadDim, p.c0, p.c1, w);
        if constexpr (kNorm == PSA_NORM_HEAD) {
          ss = hx = 0.f;
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            ss = fmaf(x[c], x[c], ss);
            hx = fmaf(g[c] * (row ? w[c] : 0.f), x[c], hx);
          }
          ss = lanes_sum(ss);
          hx = lanes_sum(hx);
        }
        const float r = rsqrtf(ss * a.inv_count + a.eps), coef = r * r * (hx * a.inv_count);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const float xc = x[c], gc = g[c];
          if (row) dw[u][c] = fmaf(gc, xc * r, dw[u][c]);
          g[c] = r * (gc * w[c] - xc * coef);
        }
      }
      if (row) store_row<T, kHalves>(to + head * a.dx_head, p.c0, p.c1, g);
    }
  }
  if (kNorm == PSA_NORM_NONE || a.dw_part == nullptr) return;
  // the block's tokens, and for a shared weight its heads, in order
  float* to = a.dw_part + ((long long)t * gridDim.x + blockIdx.x) * a.weight_cols;
  const int half = (int)threadIdx.x / kLanes, halves = (int)blockDim.x / kLanes;
  if (a.weight_head == 0) {
#pragma unroll
    for (int u = 1; u < kRows; ++u)
#pragma unroll
      for (int c = 0; c < 8; ++c) dw[0][c] += dw[u][c];
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    if (u > 0 && (a.weight_head == 0 || u * a.parts >= a.n_heads)) break;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      dw_part[half * kHeadDim + p.c0 + c] = dw[u][c];
      dw_part[half * kHeadDim + p.c1 + c] = dw[u][c + 4];
    }
    __syncthreads();
    if (a.weight_head == 0) {
      for (int c = (int)threadIdx.x; c < kHeadDim; c += (int)blockDim.x) {
        float s = 0.f;
        for (int j = 0; j < halves; ++j) s += dw_part[j * kHeadDim + c];   // (idle half warps left zeros)
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
  for (int i = grp; i < n_part; i += kDwGroups) s += (double)from[(long long)i * cols];
  red[grp][threadIdx.x % kDwCols] = s;
  __syncthreads();
  if (grp == 0) {
    for (int i = 1; i < kDwGroups; ++i) s += red[i][threadIdx.x];
    (blockIdx.y == 0 ? q_dw : k_dw)[c] = (float)s;
  }
}

template <class T, class O, int kNorm, bool kHalves>
cudaError_t launch_typed(const NormRopeArgs& a, int threads, int blocks, int bwd_blocks, cudaStream_t st) {
  if (bwd_blocks == 0) {
    norm_rope_kernel<T, O, kNorm, kHalves><<<blocks, threads, 0, st>>>(a);
  } else {
    const size_t smem = kNorm == PSA_NORM_NONE ? 0 : (size_t)(threads / kLanes) * kHeadDim * sizeof(float);
    norm_rope_bwd_kernel<T, O, kNorm, kHalves><<<dim3(bwd_blocks, a.in[1] || a.grad[1] ? 2 : 1), threads, smem, st>>>(a);
  }
  return cudaGetLastError();
}
template <class T, class O, int kNorm>
cudaError_t launch_pairs(const NormRopeArgs& a, bool halves, int threads, int blocks, int bwd_blocks, cudaStream_t st) {
  return halves ? launch_typed<T, O, kNorm, true>(a, threads, blocks, bwd_blocks, st) : launch_typed<T, O, kNorm, false>(a, threads, blocks, bwd_blocks, st);
}
template <class T, class O>
cudaError_t launch_norm(const NormRopeArgs& a, int norm, bool halves, int threads, int blocks, int bwd_blocks, cudaStream_t st) {
  switch (norm) {
    case PSA_NORM_HEAD: return launch_pairs<T, O, PSA_NORM_HEAD>(a, halves, threads, blocks, bwd_blocks, st);
    case PSA_NORM_TOKEN: return launch_pairs<T, O, PSA_NORM_TOKEN>(a, halves, threads, blocks, bwd_blocks, st);
    default: return launch_pairs<T, O, PSA_NORM_NONE>(a, halves, threads, blocks, bwd_blocks, st);
  }
}

}  // namespace

cudaError_t launch_norm_rope(NormRopeArgs& a, const psa_qk& prob, bool halves, bool backward, int n_sms, float* q_dw, float* k_dw, cudaStream_t st,
                             int* launches) {
  // Half warps a token: so many that each has at most kRows heads; one a head where there are too few tokens to fill the GPU
  // with less.  Tokens a block: blocks of some 256 threads, whole warps.
  const long long by_rows = (long long)a.n_all * ((a.n_heads + kRows - 1) / kRows);
  a.parts = by_rows * kLanes < (long long)n_sms * 1024 && a.n_heads <= kMaxThreads / kLanes ? a.n_heads : (a.n_heads + kRows - 1) / kRows;
  a.slots = 256 / (a.parts * kLanes);
  if (a.slots < 1) a.slots = 1;
  const int threads = (a.slots * a.parts * kLanes + 31) & ~31;
  const long long blocks = (a.n_all + a.slots - 1) / a.slots;
  int bwd_blocks = 0;
  if (backward) bwd_blocks = (int)(blocks < kNormRopeBwdBlocks ? blocks : kNormRopeBwdBlocks);
  cudaError_t e;
  const int in = prob.dtype, out = prob.out_dtype;
  if (in == PSA_BF16) e = launch_norm<__nv_bfloat16, __nv_bfloat16>(a, prob.norm, halves, threads, (int)blocks, bwd_blocks, st);
  else if (in == PSA_FP16 && out == PSA_FP16) e = launch_norm<__half, __half>(a, prob.norm, halves, threads, (int)blocks, bwd_blocks, st);
  else if (in == PSA_FP16) e = launch_norm<__half, __nv_bfloat16>(a, prob.norm, halves, threads, (int)blocks, bwd_blocks, st);
  else if (out == PSA_FP32) e = launch_norm<float, float>(a, prob.norm, halves, threads, (int)blocks, bwd_blocks, st);
  else e = launch_norm<float, __nv_bfloat16>(a, prob.norm, halves, threads, (int)blocks, bwd_blocks, st);
  if (e != cudaSuccess) return e;
  ++*launches;
  if (backward && a.dw_part != nullptr) {
    norm_rope_dw_kernel<<<dim3(a.weight_cols / kDwCols, k_dw ? 2 : 1), kDwCols * kDwGroups, 0, st>>>(a.dw_part, bwd_blocks, a.weight_cols, q_dw, k_dw);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

}  // namespace psa
