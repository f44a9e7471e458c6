// psa_select_blocks: for every query block the key blocks with the largest pooled score.
//
// Q_i, K_j: sums over the blocks' tokens; s_ij = (sum over c of Q_ic K_jc) / n_j, n_j the tokens of block j: mean key against a
// multiple of the mean query, which orders a row as the mean of all its scores q . k does.  A block keeps its `keep` largest.
// Sums and scores are in 64 bits: which blocks are kept is a matter of order, and scores next to the border are told apart (32 bits
// order some 1 in 10^4 rows of a 315-block head otherwise).  Equal scores (exactly, whatever the blocks: the sums are the same
// operations) go to the lowest block.
//
// Two kernels: pooling is bound by reading q and k once; scores and choice together keep a tile of rows of scores in shared memory,
// so that the heads * NB^2 scores of 8 bytes never reach HBM.
#include <cuda_bf16.h>

#include "psa_common.cuh"

namespace psa {

namespace {

constexpr int kPoolThreads = 256, kPoolRows = kPoolThreads / 16;   // 16 lanes a token, 8 channels each
constexpr int kSelectThreads = 256, kSelectWarps = kSelectThreads / 32;
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

// Sums over the tokens of one block of one head of q (z = 0) or k (z = 1).
__global__ void __launch_bounds__(kPoolThreads)
pool_kernel(const __nv_bfloat16* __restrict__ q, const __nv_bfloat16* __restrict__ k, const Geom g, long long stride_head, long long stride_token,
            double* __restrict__ sums) {
  __shared__ double part[kPoolRows][kHeadDim];
  const int b = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 15, row = threadIdx.x >> 4;
  const BlockOrigin o = block_origin(g, b);
  const __nv_bfloat16* from = (blockIdx.z ? k : q) + head * stride_head + 8 * lane;
  const int frame = o.nh * o.nw, n = o.nt * frame;
  double acc[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) acc[c] = 0.0;
#pragma unroll 4
  for (int r = row; r < n; r += kPoolRows) {
    const int t = r / frame, y = r - t * frame, h = y / o.nw, w = y - h * o.nw;
    const long long token = ((long long)(o.t0 + t) * g.H + o.h0 + h) * g.W + o.w0 + w;
    const uint4 x = *reinterpret_cast<const uint4*>(from + token * stride_token);
    const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      acc[2 * c] += (double)__uint_as_float(v[c] << 16);
      acc[2 * c + 1] += (double)__uint_as_float(v[c] & 0xffff0000u);
    }
  }
#pragma unroll
  for (int c = 0; c < 8; ++c) part[row][8 * lane + c] = acc[c];
  __syncthreads();
  if (threadIdx.x < kHeadDim) {
    double s = 0.0;
#pragma unroll
    for (int r = 0; r < kPoolRows; ++r) s += part[r][threadIdx.x];
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

// kTiles * 8 query blocks of one head: their scores against every key block, then one warp a row chooses.
template <int kTiles>
__global__ void __launch_bounds__(kSelectThreads)
select_kernel(const double* __restrict__ sums, const Geom g, const __grid_constant__ SelectHeads heads, int keep_self, int* __restrict__ row_ptr,
              int* __restrict__ col_idx) {
  constexpr int kRows = 8 * kTiles;
  extern __shared__ __align__(16) double sm[];
  double* qs = sm;                                                            // [kRows][kSumPitch]
  unsigned long long* keys = reinterpret_cast<unsigned long long*>(sm + kRows * kSumPitch);   // [kRows][NB]
  const int head = blockIdx.y, i0 = blockIdx.x * kRows, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rows = min(kRows, g.NB - i0);
  const double* q_sums = sums + ((long long)head * g.NB + i0) * kHeadDim;
  const double* k_sums = sums + ((long long)(gridDim.y + head) * g.NB) * kHeadDim;
  for (int i = threadIdx.x; i < kRows * kHeadDim; i += kSelectThreads) {
    const int r = i / kHeadDim, c = i % kHeadDim;
    qs[r * kSumPitch + c] = r < rows ? q_sums[i] : 0.0;
  }
  __syncthreads();
  // scores: a warp takes 8 key blocks at a time.  Which four channels a product takes is free as long as both sides agree: lane
  // l % 4 = x takes channels 8 p + 2 x and 8 p + 2 x + 1, so that loads are of 16 bytes.
  const int x = lane & 3, y = lane >> 2;
  for (int j0 = 8 * warp; j0 < g.NB; j0 += 8 * kSelectWarps) {
    const double2* kp = reinterpret_cast<const double2*>(k_sums + (long long)min(j0 + y, g.NB - 1) * kHeadDim + 2 * x);
    double d[kTiles][2];
#pragma unroll
    for (int m = 0; m < kTiles; ++m) d[m][0] = d[m][1] = 0.0;
#pragma unroll 8
    for (int p = 0; p < kHeadDim / 8; ++p) {
      const double2 b = kp[4 * p];
#pragma unroll
      for (int m = 0; m < kTiles; ++m) {
        const double2 a = *reinterpret_cast<const double2*>(qs + (8 * m + y) * kSumPitch + 8 * p + 2 * x);
        mma_f64(d[m], a.x, b.x);
        mma_f64(d[m], a.y, b.y);
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int j = j0 + 2 * x + e;
      if (j >= g.NB) continue;
      const BlockOrigin o = block_origin(g, j);
      const double n = (double)(o.nt * o.nh * o.nw);
#pragma unroll
      for (int m = 0; m < kTiles; ++m) {
        const int r = 8 * m + y;
        keys[r * g.NB + j] = keep_self && j == i0 + r ? ~0ull : order_key(d[m][e] / n);
      }
    }
  }
  __syncthreads();
  const int keep = heads.keep[head];
  for (int r = warp; r < rows; r += kSelectWarps) {
    const unsigned long long* mine = keys + r * g.NB;
    const int row = head * g.NB + i0 + r, base = heads.base[head] + (i0 + r) * keep;
    // the keep-th largest key lies in [lo, hi]: at least `keep` keys are >= lo, fewer are > hi.  Halved until exactly `keep` keys
    // are >= lo, or nothing is left between.
    unsigned long long lo = ~0ull, hi = 0;
    for (int j = lane; j < g.NB; j += 32) {
      lo = min(lo, mine[j]);
      hi = max(hi, mine[j]);
    }
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) {
      lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, m));
      hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, m));
    }
    int at_least = g.NB;   // keys >= lo
    while (at_least != keep && lo < hi) {
      const unsigned long long mid = lo + (hi - lo) / 2 + 1;   // above lo, at most hi
      int n = 0;
      for (int j = lane; j < g.NB; j += 32) n += mine[j] >= mid;
      n = __reduce_add_sync(0xffffffffu, n);
      if (n >= keep) { lo = mid; at_least = n; }
      else hi = mid - 1;
    }
    // all keys above lo, and the first ones equal to it as far as there is room
    int above = 0;
    if (at_least != keep) {
      for (int j = lane; j < g.NB; j += 32) above += mine[j] > lo;
      above = __reduce_add_sync(0xffffffffu, above);
    }
    int room = at_least == keep ? g.NB : keep - above, at = base;
    for (int j0 = 0; j0 < g.NB; j0 += 32) {
      const int j = j0 + lane;
      const unsigned long long key = j < g.NB ? mine[j] : 0ull;
      const unsigned equal = __ballot_sync(0xffffffffu, j < g.NB && key == lo), more = __ballot_sync(0xffffffffu, j < g.NB && key > lo);
      const unsigned below = (1u << lane) - 1u;
      const bool take = (more >> lane & 1u) || ((equal >> lane & 1u) && __popc(equal & below) < room);
      const unsigned taken = __ballot_sync(0xffffffffu, take);
      room -= min(room, __popc(equal));
      if (take) col_idx[at + __popc(taken & below)] = j;
      at += __popc(taken);
    }
    if (lane == 0) {
      row_ptr[row] = base;
      if (i0 + r + 1 == g.NB) row_ptr[row + 1] = base + keep;   // (the next head writes the same there)
    }
  }
}

size_t select_smem(int rows, int nb) { return ((size_t)rows * kSumPitch + (size_t)rows * nb) * sizeof(double); }

template <int kTiles>
cudaError_t launch_select_tiles(const double* sums, const Geom& g, const SelectHeads& heads, int n_heads, bool keep_self, int* row_ptr, int* col_idx,
                                cudaStream_t st) {
  const size_t smem = select_smem(8 * kTiles, g.NB);
  const cudaError_t e = cudaFuncSetAttribute(select_kernel<kTiles>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  select_kernel<kTiles><<<dim3((g.NB + 8 * kTiles - 1) / (8 * kTiles), n_heads), kSelectThreads, smem, st>>>(sums, g, heads, keep_self ? 1 : 0, row_ptr, col_idx);
  return cudaGetLastError();
}

}  // namespace

bool select_fits(int nb) { return select_smem(8, nb) <= kMaxSmemBytes; }

cudaError_t launch_select(const void* q, const void* k, const Geom& g, long long stride_head, long long stride_token, const SelectHeads& heads, int n_heads,
                          bool keep_self, double* sums, int* row_ptr, int* col_idx, cudaStream_t st, int* launches) {
  pool_kernel<<<dim3(g.NB, n_heads, 2), kPoolThreads, 0, st>>>(static_cast<const __nv_bfloat16*>(q), static_cast<const __nv_bfloat16*>(k), g, stride_head,
                                                               stride_token, sums);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ++*launches;
  // 16 rows a block read the key sums half as often as 8
  e = select_smem(16, g.NB) <= kMaxSmemBytes ? launch_select_tiles<2>(sums, g, heads, n_heads, keep_self, row_ptr, col_idx, st)
                                             : launch_select_tiles<1>(sums, g, heads, n_heads, keep_self, row_ptr, col_idx, st);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace psa
