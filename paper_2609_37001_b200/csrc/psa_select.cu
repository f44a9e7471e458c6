// psa_select_blocks: for every query block the key blocks with the largest pooled score.
//
// Q_i, K_j: sums over the blocks' tokens; s_ij = (sum over c of Q_ic K_jc) / n_j, n_j the tokens of block j: mean key against a
// multiple of the mean query, which orders a row as the mean of all its scores q . k does.  A block keeps its `keep` largest.
// Sums and scores are in 64 bits: which blocks are kept is a matter of order, and scores next to the border have to be told apart (sums in
// 32 bits are off by some 2^-22 of the scores' spread, over which a row has hundreds of scores: by estimate a row in 10^4 would come out
// otherwise).  Equal scores go to the lowest block.
//
// Two kernels: pooling is bound by reading q and k once; scores and choice together keep the scores of eight rows in shared memory, so
// that the heads * NB^2 scores of 8 bytes never reach HBM.
#include <cuda_bf16.h>

#include "psa_common.cuh"

namespace psa {

namespace {

constexpr int kPoolThreads = 256, kPoolRows = kPoolThreads / 16;   // 16 lanes a token, 8 channels each
constexpr int kPoolAhead = 4;                                      // pairs of tokens that a thread has on their way
constexpr int kSelectThreads = 256, kSelectWarps = kSelectThreads / 32, kSelectRows = 8;
constexpr int kSumPitch = kHeadDim + 2;   // doubles a row of Q in shared memory

struct BlockOrigin {
  int t0, h0, w0, nt, nh, nw;   // first token, extents inside the grid
};
__device__ __forceinline__ BlockOrigin block_origin(const Geom& g, int b) {
  const int t = b / g.Sp, s = b - t * g.Sp, h = s / g.Wp, w = s - h * g.Wp;
  BlockOrigin o;
  o.t0 = t * g.bt; o.h0 = h * g.bh; o.w0 = w * g.bw;
  o.nt = min(g.bt, g.T - o.t0); o.nh = min(g.bh, g.H - o.h0); o.nw = min(g.bw, g.W - o.w0);
  return o;
}

// Sums over the tokens of one block of one head of q (z = 0) or k (z = 1).  Bound by HBM (q and k once) and, next to it, by the issue
// of instructions: 12 heads of 115,200 tokens 135 us, 5.2 TB/s, issue slots 75 % busy, mostly with numbers of 64 bits.  (With a
// conversion for every value the conversions' pipe was 55 % busy, and the call for 24 heads took 453 instead of 425 us.)  So of the two
// values in a 32-bit word only the lower one is converted.  The bits of the upper one are moved three places down, under the sign: read
// as the upper half of a double that is the value times 2^-896, exactly (subnormals, too), which the sum is multiplied back by.
// Infinities and NaN would become numbers; a thread that saw an exponent of 255 adds its values up again by conversion.
__device__ __forceinline__ double upper_scaled(uint32_t v) { return __hiloint2double(((int)v >> 3) & 0x8fffe000, 0); }
__device__ __forceinline__ double lower(uint32_t v) { return (double)__uint_as_float(v << 16); }
__device__ __forceinline__ double upper(uint32_t v) { return (double)__uint_as_float(v & 0xffff0000u); }
__global__ void __launch_bounds__(kPoolThreads)
pool_kernel(const __nv_bfloat16* __restrict__ q, const __nv_bfloat16* __restrict__ k, const Geom g, long long stride_head, long long stride_token,
            double* __restrict__ sums) {
  __shared__ __align__(16) union {
    uint4 copied[2 * kPoolAhead][kPoolThreads];
    double part[kPoolRows][kHeadDim];
  } sm;
  const int b = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 15, row = threadIdx.x >> 4;
  const BlockOrigin o = block_origin(g, b);
  const __nv_bfloat16* from = (blockIdx.z ? k : q) + head * stride_head + (((long long)o.t0 * g.H + o.h0) * g.W + o.w0) * stride_token + 8 * lane;
  // 16 lanes take a line of the block's tokens, or (fewer than 16 lines) a part of one, then the 16th behind it: addresses go up by one
  // token, and only a new line is looked for
  const int lines = o.nt * o.nh, log_parts = lines >= 16 ? 0 : (lines >= 8 ? 1 : (lines >= 4 ? 2 : (lines >= 2 ? 3 : 4)));
  const int part_len = (o.nw + (1 << log_parts) - 1) >> log_parts, units = lines << log_parts;
  auto len_of = [&](int u) -> int { return max(0, min(part_len, o.nw - (u & ((1 << log_parts) - 1)) * part_len)); };
  auto start_of = [&](int u) -> const __nv_bfloat16* {
    const int line = u >> log_parts, t = line / o.nh, h = line - t * o.nh;
    return from + ((long long)(t * g.H + h) * g.W + (u & ((1 << log_parts) - 1)) * part_len) * stride_token;
  };
  int total = 0;   // tokens of these lanes
  for (int u = row; u < units; u += kPoolRows) total += len_of(u);
  // two tokens at a time, kPoolAhead pairs on their way to shared memory, where each thread reads what it copied; zeros behind the last
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&sm.copied[0][threadIdx.x]);
  int unit = row, left = 0, fetched = 0;
  const __nv_bfloat16* at = from;
  auto fetch = [&](int pair) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool there = fetched < total;
      if (there && left == 0) {
        do { left = len_of(unit); unit += kPoolRows; } while (left == 0);   // (there is another token)
        at = start_of(unit - kPoolRows);
      }
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                   ::"r"(mine + (uint32_t)((2 * pair + i) * kPoolThreads) * 16u), "l"(at), "r"(there ? 16 : 0) : "memory");
      if (there) {
        ++fetched;
        if (--left > 0) at += stride_token;
      }
    }
  };
  double acc[8];
  float most[4] = {0.f, 0.f, 0.f, 0.f};   // largest magnitude among the upper values (and what lies below them in the word), or NaN
#pragma unroll
  for (int c = 0; c < 8; ++c) acc[c] = 0.0;
  auto add = [&](const uint4& x, const uint4& y) {
    const uint32_t v[4] = {x.x, x.y, x.z, x.w}, u[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      acc[2 * c] += lower(v[c]);
      acc[2 * c + 1] += upper_scaled(v[c]);
      acc[2 * c] += lower(u[c]);
      acc[2 * c + 1] += upper_scaled(u[c]);
      asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(most[c]) : "f"(fabsf(__uint_as_float(v[c]))), "f"(fabsf(__uint_as_float(u[c]))));
    }
  };
#pragma unroll
  for (int i = 0; i < kPoolAhead; ++i) {
    if (fetched < total) fetch(i);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  for (int n = 0, pair = 0; n < total; n += 2, pair = pair + 1 == kPoolAhead ? 0 : pair + 1) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kPoolAhead - 1) : "memory");
    add(sm.copied[2 * pair][threadIdx.x], sm.copied[2 * pair + 1][threadIdx.x]);
    if (fetched < total) fetch(pair);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    acc[2 * c + 1] *= 0x1p896;
    if (!(most[c] < __uint_as_float(0x7f800000u))) {
      acc[2 * c + 1] = 0.0;
      for (int u = row; u < units; u += kPoolRows) {
        const __nv_bfloat16* x = start_of(u);
        for (int n = len_of(u); n > 0; --n, x += stride_token) acc[2 * c + 1] += upper(reinterpret_cast<const uint32_t*>(x)[c]);
      }
    }
  }
  __syncthreads();   // (nobody reads copies any more)
#pragma unroll
  for (int c = 0; c < 8; ++c) sm.part[row][8 * lane + c] = acc[c];
  __syncthreads();
  if (threadIdx.x < kHeadDim) {
    double s = 0.0;
#pragma unroll
    for (int r = 0; r < kPoolRows; ++r) s += sm.part[r][threadIdx.x];
    sums[(((long long)blockIdx.z * gridDim.y + head) * g.NB + b) * kHeadDim + threadIdx.x] = s;
  }
}

// D (8 x 8) += A (8 x 4) B (4 x 8), 64 bits: lane l holds A[l / 4][l % 4], B[l % 4][l / 4], D[l / 4][2 (l % 4) + {0, 1}].
__device__ __forceinline__ void mma_f64(double* d, double a, double b) {
  asm("mma.sync.aligned.m8n8k4.row.col.f64.f64.f64.f64 {%0, %1}, {%2}, {%3}, {%0, %1};" : "+d"(d[0]), "+d"(d[1]) : "d"(a), "d"(b));
}

// Whole numbers in the order of the scores: NaN as -infinity, -0 as 0.
__device__ __forceinline__ unsigned long long order_key(double s) {
  const long long b = __double_as_longlong(s != s ? -__longlong_as_double(0x7ff0000000000000ll) : s + 0.0);
  return (unsigned long long)b ^ (b < 0 ? ~0ull : 1ull << 63);
}

// The list of one row by one warp: `n` of its keys (in shared memory) to `to`.  kHeld: 32-key pieces that a lane keeps in registers
// during the search, 0: none, it reads them every time.
template <int kHeld>
__device__ __forceinline__ void choose(const unsigned long long* row, int nb, int n, int lane, int* to) {
  unsigned long long held[kHeld ? kHeld : 1];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = lane + 32 * i < nb ? row[lane + 32 * i] : 0ull;
  // keys that f holds for, of all lanes (not for 0, which stands behind the last key)
  auto count = [&](auto f) -> int {
    int c = 0;
    if constexpr (kHeld > 0) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i) c += f(held[i]);
    } else {
      for (int j = lane; j < nb; j += 32) c += f(row[j]);
    }
    return __reduce_add_sync(0xffffffffu, c);
  };
  // the n-th largest key lies in [lo, hi]: at least n keys are >= lo, fewer are > hi.  Halved until exactly n keys are >= lo, or
  // nothing is left between.
  unsigned long long lo = ~0ull, hi = 0;
  for (int j = lane; j < nb; j += 32) {
    lo = min(lo, row[j]);
    hi = max(hi, row[j]);
  }
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) {
    lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, m));
    hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, m));
  }
  int at_least = nb;   // keys >= lo
  while (at_least != n && lo < hi) {
    const unsigned long long mid = lo + (hi - lo) / 2 + 1;   // above lo, at most hi
    const int c = count([&](unsigned long long key) { return key >= mid; });
    if (c >= n) { lo = mid; at_least = c; }
    else hi = mid - 1;
  }
  // all keys above lo, and the first ones equal to it as far as there is room (no key is 0)
  int room = at_least == n ? nb : n - count([&](unsigned long long key) { return key > lo; });
  for (int j0 = 0; j0 < nb; j0 += 32) {
    const int j = j0 + lane;
    const unsigned long long key = j < nb ? row[j] : 0ull;
    const unsigned equal = __ballot_sync(0xffffffffu, key == lo), more = __ballot_sync(0xffffffffu, key > lo);
    const unsigned below = (1u << lane) - 1u;
    const bool take = (more >> lane & 1u) || ((equal >> lane & 1u) && __popc(equal & below) < room);
    const unsigned taken = __ballot_sync(0xffffffffu, take);
    room -= min(room, __popc(equal));
    if (take) to[__popc(taken & below)] = j;
    to += __popc(taken);
  }
}

// Eight query blocks of one head: their scores against every key block, then one warp a row chooses.  Bound by the waits in both
// parts; several blocks an SM overlap them.  (16 query blocks read the key sums half as often, but only two blocks fit an SM then: 24
// heads of 450 blocks 378 instead of 371 us for the whole call; two rows a warp in turn: 395.)
__global__ void __launch_bounds__(kSelectThreads)
select_kernel(const double* __restrict__ sums, const Geom g, const __grid_constant__ SelectHeads heads, int keep_self, int* __restrict__ row_ptr,
              int* __restrict__ col_idx) {
  extern __shared__ __align__(16) double sm[];
  double* qs = sm;                                                                                   // [kSelectRows][kSumPitch]
  unsigned long long* keys = reinterpret_cast<unsigned long long*>(sm + kSelectRows * kSumPitch);   // [kSelectRows][NB]
  const int head = blockIdx.y, i0 = blockIdx.x * kSelectRows, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rows = min(kSelectRows, g.NB - i0);
  const double* q_sums = sums + ((long long)head * g.NB + i0) * kHeadDim;
  const double* k_sums = sums + ((long long)(gridDim.y + head) * g.NB) * kHeadDim;
  for (int i = threadIdx.x; i < kSelectRows * kHeadDim; i += kSelectThreads) {
    const int r = i / kHeadDim, c = i % kHeadDim;
    qs[r * kSumPitch + c] = r < rows ? q_sums[i] : 0.0;
  }
  __syncthreads();
  // scores: a warp takes 8 key blocks at a time.  Which four channels a product takes is free as long as both sides agree: lane
  // l % 4 = x takes channels 8 p + 2 x and 8 p + 2 x + 1, so that loads are of 16 bytes.
  const int x = lane & 3, y = lane >> 2;
  for (int j0 = 8 * warp; j0 < g.NB; j0 += 8 * kSelectWarps) {
    const double2* kp = reinterpret_cast<const double2*>(k_sums + (long long)min(j0 + y, g.NB - 1) * kHeadDim + 2 * x);
    double d[2] = {0.0, 0.0};
#pragma unroll 8
    for (int p = 0; p < kHeadDim / 8; ++p) {
      const double2 b = kp[4 * p], a = *reinterpret_cast<const double2*>(qs + y * kSumPitch + 8 * p + 2 * x);
      mma_f64(d, a.x, b.x);
      mma_f64(d, a.y, b.y);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int j = j0 + 2 * x + e;
      if (j >= g.NB) continue;
      const BlockOrigin o = block_origin(g, j);
      keys[y * g.NB + j] = keep_self && j == i0 + y ? ~0ull : order_key(d[e] / (double)(o.nt * o.nh * o.nw));
    }
  }
  __syncthreads();
  const int keep = heads.keep[head];
  for (int r = warp; r < rows; r += kSelectWarps) {
    const unsigned long long* mine = keys + r * g.NB;
    const int row = head * g.NB + i0 + r, base = heads.base[head] + (i0 + r) * keep;
    if (lane == 0) {
      row_ptr[row] = base;
      if (i0 + r + 1 == g.NB) row_ptr[row + 1] = base + keep;   // (the next head writes the same there)
    }
    if (g.NB <= 256) choose<8>(mine, g.NB, keep, lane, col_idx + base);
    else if (g.NB <= 512) choose<16>(mine, g.NB, keep, lane, col_idx + base);
    else choose<0>(mine, g.NB, keep, lane, col_idx + base);
  }
}

size_t select_smem(int nb) { return (size_t)kSelectRows * (kSumPitch + nb) * sizeof(double); }

}  // namespace

bool select_fits(int nb) { return select_smem(nb) <= kMaxSmemBytes; }

cudaError_t launch_select(const void* q, const void* k, const Geom& g, long long stride_head, long long stride_token, const SelectHeads& heads, int n_heads,
                          bool keep_self, double* sums, int* row_ptr, int* col_idx, cudaStream_t st, int* launches) {
  pool_kernel<<<dim3(g.NB, n_heads, 2), kPoolThreads, 0, st>>>(static_cast<const __nv_bfloat16*>(q), static_cast<const __nv_bfloat16*>(k), g, stride_head,
                                                               stride_token, sums);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ++*launches;
  const size_t smem = select_smem(g.NB);
  if (smem > 48 * 1024 && (e = cudaFuncSetAttribute(select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)) != cudaSuccess) return e;
  select_kernel<<<dim3((g.NB + kSelectRows - 1) / kSelectRows, n_heads), kSelectThreads, smem, st>>>(sums, g, heads, keep_self ? 1 : 0, row_ptr, col_idx);
  e = cudaGetLastError();
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace psa
