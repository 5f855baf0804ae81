// Linear layers: y = act(x w^T + bias + residual), and the products its gradients are made of.
//
//   forward  y[m][n]  = sum_k x[m][k] w[n][k]      dgrad  dx[m][k] = sum_n g[m][n] w[n][k]      wgrad  dw[n][k] = sum_m g[m][n] x[m][k]
//
// All three are C[p][q] = sum_r A(p, r) B(q, r) with operands that are contiguous along r or along p / q.
#include <initializer_list>

#include "nf_act.cuh"
#include "nf_gemm.h"
#include "nf_ldst.cuh"

namespace {

// The sum at (p, q) to its place: bias and residual are added in fp32, every stored value is rounded once
template <typename T>
__device__ __forceinline__ void finish(const Epilogue& e, size_t at, int q, float v) {
  if (e.out_f32) {
    reinterpret_cast<float*>(e.out)[at] = v;
    return;
  }
  if (e.bias) v += e.bias[q];
  if (e.residual) v += ldf(reinterpret_cast<const T*>(e.residual), at);
  if (e.pre) stf(reinterpret_cast<T*>(e.pre), at, v);
  stf(reinterpret_cast<T*>(e.out), at, nf_act_value<T>(v, e.act));
}

// fp32 on the CUDA cores, for products too small for the tensor cores: 64 x 64 results per block, 4 x 4 per thread, 16 steps of r at a time; sa_p,
// sa_r: element strides of A.  gridDim.z > 1: each z sums a range of r into part[z][P][Q].  Latency bounds it: 256 x 256 x 256 9 us, launch and join included.
__global__ void __launch_bounds__(256) gemm_simple_kernel(const float* __restrict__ A, size_t sa_p, size_t sa_r, const float* __restrict__ B, size_t sb_q,
                                                          size_t sb_r, int P, int Q, int R, float* part, const Epilogue e) {
  nf_pdl_begin();
  __shared__ float As[16][68], Bs[16][68];
  const int p0 = blockIdx.x * 64, q0 = blockIdx.y * 64;
  const int r_lo = (int)((long long)R * blockIdx.z / gridDim.z), r_hi = (int)((long long)R * (blockIdx.z + 1) / gridDim.z);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[4][4] = {}, na[4], nb[4];  // the next step's operands are on their way while this one's are multiplied
  auto fetch = [&](int r0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int l = threadIdx.x + 256 * i;
      // neighbouring threads along whichever direction is contiguous
      const int pa = sa_r == 1 ? l / 16 : l % 64, ra = sa_r == 1 ? l % 16 : l / 64;
      na[i] = p0 + pa < P && r0 + ra < r_hi ? A[(size_t)(p0 + pa) * sa_p + (size_t)(r0 + ra) * sa_r] : 0.f;
      const int qb = sb_r == 1 ? l / 16 : l % 64, rb = sb_r == 1 ? l % 16 : l / 64;
      nb[i] = q0 + qb < Q && r0 + rb < r_hi ? B[(size_t)(q0 + qb) * sb_q + (size_t)(r0 + rb) * sb_r] : 0.f;
    }
  };
  fetch(r_lo);
  for (int r0 = r_lo; r0 < r_hi; r0 += 16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int l = threadIdx.x + 256 * i;
      As[sa_r == 1 ? l % 16 : l / 64][sa_r == 1 ? l / 16 : l % 64] = na[i];
      Bs[sb_r == 1 ? l % 16 : l / 64][sb_r == 1 ? l / 16 : l % 64] = nb[i];
    }
    __syncthreads();
    if (r0 + 16 < r_hi) fetch(r0 + 16);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      float a[4], b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = As[k][ty * 4 + i];
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] = Bs[k][tx * 4 + j];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(a[i], b[j], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = p0 + ty * 4 + i, q = q0 + tx * 4 + j;
      if (p >= P || q >= Q) continue;
      const size_t at = (size_t)p * Q + q;
      if (gridDim.z > 1)
        part[(size_t)blockIdx.z * P * Q + at] = acc[i][j];
      else
        finish<float>(e, at, q, acc[i][j]);
    }
}

// The partial sums of an element in LN chains (chain k takes splits k, k + LN, ...) in fp64, joined in order: one chain where there are many
// elements, eight threads to an element where there are few
template <typename T, int LN>
__global__ void __launch_bounds__(256) gemm_join_kernel(const float* __restrict__ part, int splits, size_t n, int Q, const Epilogue e) {
  nf_pdl_begin();
  constexpr int kCols = 256 / LN;
  __shared__ double sm[LN][kCols];
  const int tx = threadIdx.x % kCols, ty = threadIdx.x / kCols;
  const size_t i = (size_t)blockIdx.x * kCols + tx;
  double s = 0;
  if (i < n) {
#pragma unroll 4
    for (int z = ty; z < splits; z += LN) s += part[(size_t)z * n + i];
  }
  if constexpr (LN > 1) {
    sm[ty][tx] = s;
    __syncthreads();
    if (ty) return;
#pragma unroll
    for (int k = 1; k < LN; ++k) s += sm[k][tx];
  }
  if (i < n) finish<T>(e, i, (int)(i % Q), (float)s);
}

// A few rows of x (MR at most) through weights contiguous along r: the weights are all the traffic.  A block of 128 threads takes kThinRows
// weight rows; its threads share a row in 16-byte pieces, so that a block has 128 * kThinRows * 16 bytes on their way at a time, and each
// piece of x serves kThinRows rows of weights.  Pairs of neighbouring products are added in one packed multiply-add; threads' sums meet by shuffles
// and shared memory.  Rows that are not made of such pieces are read element by element.  One row of 4096 x 8192 bf16 weights 13 us (5.2 TB/s).
constexpr int kThinRows = 4;
// Up to four rows of bf16, 24 of fp32: beyond, the tensor cores take the product sooner (8 x 8192 x 4096 bf16 38 us here, 18 there; 32 x 2344 x 7416
// fp32 64 us there, 24 rows 49 us here)
template <typename T> constexpr int kThinMost = sizeof(T) == 4 ? 24 : 4;
template <typename T> constexpr int kThinRowsOfX = sizeof(T) == 4 ? 8 : 4;  // of one block; more rows take the weights through L2 again

// WHOLE: rows are made of 16-byte pieces; else a thread takes every 128th element, as many at a time
template <typename T, int MR, bool WHOLE>
__global__ void __launch_bounds__(128) thin_kernel(const T* __restrict__ x, const T* __restrict__ w, int M, int N, int K, const Epilogue e) {
  nf_pdl_begin();
  constexpr int V = 16 / sizeof(T), NP = V / 2;
  __shared__ float sm[4][kThinRows * MR];
  const int n0 = blockIdx.x * kThinRows, m0 = blockIdx.y * MR;
  f32x2 acc[kThinRows][MR];
#pragma unroll
  for (int j = 0; j < kThinRows; ++j)
#pragma unroll
    for (int m = 0; m < MR; ++m) acc[j][m] = 0;
  auto pairs = [&](const T* row, int k, f32x2 (&v)[NP], bool stream) {
    const T* at = row + k;
    if constexpr (!WHOLE) {
#pragma unroll
      for (int i = 0; i < NP; ++i)
        v[i] = nf_pack2(k + 256 * i < K ? ldf(at, 256 * i) : 0.f, k + 256 * i + 128 < K ? ldf(at, 256 * i + 128) : 0.f);
    } else if constexpr (sizeof(T) == 2) {
      const uint4 u = stream ? __ldcs(reinterpret_cast<const uint4*>(at)) : __ldg(reinterpret_cast<const uint4*>(at));
      const uint32_t q[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = nf_pack2(__uint_as_float(q[i] << 16), __uint_as_float(q[i] & 0xffff0000u));
    } else {
      const float4 u = stream ? __ldcs(reinterpret_cast<const float4*>(at)) : __ldg(reinterpret_cast<const float4*>(at));
      v[0] = nf_pack2(u.x, u.y);
      v[1] = nf_pack2(u.z, u.w);
    }
  };
#pragma unroll 2
  for (int k = threadIdx.x * (WHOLE ? V : 1); k < K; k += 128 * V) {
    f32x2 b[kThinRows][NP];
#pragma unroll
    for (int j = 0; j < kThinRows; ++j) pairs(w + (size_t)min(n0 + j, N - 1) * K, k, b[j], true);  // rows beyond N: the last one again, not stored
#pragma unroll
    for (int m = 0; m < MR; ++m) {
      f32x2 a[NP];
      pairs(x + (size_t)min(m0 + m, M - 1) * K, k, a, false);
#pragma unroll
      for (int j = 0; j < kThinRows; ++j)
#pragma unroll
        for (int i = 0; i < NP; ++i) acc[j][m] = nf_fma2(a[i], b[j][i], acc[j][m]);
    }
  }
#pragma unroll
  for (int j = 0; j < kThinRows; ++j)
#pragma unroll
    for (int m = 0; m < MR; ++m) {
      float lo, hi;
      nf_unpack2(acc[j][m], lo, hi);
      float v = lo + hi;
#pragma unroll
      for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (threadIdx.x % 32 == 0) sm[threadIdx.x / 32][m * kThinRows + j] = v;
    }
  __syncthreads();
  if (threadIdx.x < kThinRows * MR) {
    const int m = m0 + threadIdx.x / kThinRows, n = n0 + threadIdx.x % kThinRows;
    if (m < M && n < N) finish<T>(e, (size_t)m * N + n, n, (sm[0][threadIdx.x] + sm[1][threadIdx.x]) + (sm[2][threadIdx.x] + sm[3][threadIdx.x]));
  }
}

// Where rows come in pieces, kThinMost of them, else one block's worth.  And any product whose blocks take no longer than the launches, pipeline and join
// of the other kernels: each is about 3 ns at up to 512 long sums, 6 at 2000 (bf16 16 x 1024 x 1024 1024 blocks 5.6 us, 7.5 on the tensor cores;
// 64 x 512 x 512 2048 blocks 8.1 and 6.1; 128 x 512 x 10 2.0 and 7.3; fp32 64 x 512 x 512 1024 blocks 6.8, 14 by the simple kernel, 64 x 1024 x 1024 2048
// blocks 13.7 and 14.2; sums below 128, which that one does not split, 128 x 64 x 1024 4096 blocks 18.9 and 8.3).
template <typename T>
bool thin_pays(int P, int Q, int R) {
  const bool half = sizeof(T) == 2;
  if (P <= (R % (16 / (int)sizeof(T)) == 0 ? kThinMost<T> : kThinRowsOfX<T>)) return true;
  const double blocks = (double)((Q + kThinRows - 1) / kThinRows) * ((P + kThinRowsOfX<T> - 1) / kThinRowsOfX<T>);
  return blocks <= (half ? 1024 : R >= 128 ? 2048 : 512) && blocks * R <= (half ? 1 << 20 : 1 << 21);
}

template <typename T, bool WHOLE>
int thin_product(const T* x, const T* w, int M, int N, int K, const Epilogue& e) {
  constexpr int most = kThinRowsOfX<T>;
  auto k = M == 1 ? thin_kernel<T, 1, WHOLE> : M == 2 ? thin_kernel<T, 2, WHOLE> : M <= 4 ? thin_kernel<T, 4, WHOLE> : thin_kernel<T, most, WHOLE>;
  nf_launch(k, dim3((N + kThinRows - 1) / kThinRows, (M + most - 1) / most), 128, 0, x, w, M, N, K, e);
  NF_LAUNCHED();
  return NF_OK;
}

// A few rows of A (MR to a block) through a matrix whose rows lie along q: the input gradients of small batches.  Again the matrix is all the traffic:
// a lane keeps 16 bytes of columns, the eight warps of a block take rows r in turn, and A's values reach all lanes at once from shared memory.
// Blocks share a column's rows (gridDim.z ranges, whose sums go to part[z][P][Q]) until the SMs have enough loads on their way.
// 7 x 7416 x 2344 fp32 17 us, one row 10 us (the simple kernel 128 and 97, reading the matrix from memory 11); bf16 one or two rows 10 us, from three on
// 16 here and 13 on the tensor cores.  fp32 24 rows 39 us, 32 on the tensor cores 62.
constexpr int kAcrossRange = 256;  // rows of r whose part of A is in shared memory at a time
template <typename T> constexpr int kAcrossMost = sizeof(T) == 4 ? 24 : 2;
template <typename T> constexpr int kAcrossRows = sizeof(T) == 4 ? 8 : 2;

template <typename T, int MR>
__global__ void __launch_bounds__(256) across_kernel(const T* __restrict__ A, const T* __restrict__ B, int P, int Q, int R, float* part, const Epilogue e) {
  nf_pdl_begin();
  constexpr int V = 16 / sizeof(T), NP = V / 2, kCols = 32 * V;
  __shared__ __align__(16) float sm[8 * MR * kCols > kAcrossRange * MR ? 8 * MR * kCols : kAcrossRange * MR];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, p0 = blockIdx.y * MR, q = blockIdx.x * kCols + lane * V;
  const int lo = (int)((long long)R * blockIdx.z / gridDim.z), hi = (int)((long long)R * (blockIdx.z + 1) / gridDim.z);
  f32x2 acc[MR][NP];
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int i = 0; i < NP; ++i) acc[m][i] = 0;
  for (int c = lo; c < hi; c += kAcrossRange) {
    const int n = min(kAcrossRange, hi - c);
    __syncthreads();
    if ((int)threadIdx.x < n) {
      float a[MR];
#pragma unroll
      for (int m = 0; m < MR; ++m) a[m] = p0 + m < P ? ldf(A, (size_t)(p0 + m) * R + c + threadIdx.x) : 0.f;
#pragma unroll
      for (int m = 0; m < MR; ++m) sm[threadIdx.x * MR + m] = a[m];
    }
    __syncthreads();
    if (q < Q) {  // whole: Q is a multiple of V
#pragma unroll 8
      for (int r = warp; r < n; r += 8) {
        const T* at = B + (size_t)(c + r) * Q + q;
        f32x2 b[NP];
        if constexpr (sizeof(T) == 2) {
          const uint4 u = __ldcs(reinterpret_cast<const uint4*>(at));
          const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) b[i] = nf_pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
        } else {
          const float4 u = __ldg(reinterpret_cast<const float4*>(at));
          b[0] = nf_pack2(u.x, u.y);
          b[1] = nf_pack2(u.z, u.w);
        }
#pragma unroll
        for (int m = 0; m < MR; ++m) {
          const float a = sm[r * MR + m];
#pragma unroll
          for (int i = 0; i < NP; ++i) acc[m][i] = nf_fma2(nf_pack2(a, a), b[i], acc[m][i]);
        }
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int i = 0; i < NP; i += 2) {
      float4 v;
      nf_unpack2(acc[m][i], v.x, v.y);
      nf_unpack2(acc[m][i + 1], v.z, v.w);
      *reinterpret_cast<float4*>(&sm[(warp * MR + m) * kCols + lane * V + 2 * i]) = v;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < MR * kCols; i += 256) {
    const int p = p0 + i / kCols, col = blockIdx.x * kCols + i % kCols;
    if (p >= P || col >= Q) continue;
    float v = sm[i];
#pragma unroll
    for (int w = 1; w < 8; ++w) v += sm[w * MR * kCols + i];
    const size_t at = (size_t)p * Q + col;
    if (gridDim.z > 1) part[(size_t)blockIdx.z * P * Q + at] = v;
    else finish<T>(e, at, col, v);
  }
}

// Also any product short enough that the other kernels are waiting for launches, pipeline and join: fp32 up to 2^26 multiply-adds counted in whole columns of
// blocks (256 x 256 x 256 5.4 us, 13.9 by the simple kernel; 64 x 1024 x 1024 12.3 and 13.9; 48 x 2344 x 7416 68 and 62 on the tensor cores), bf16 below
// 2^24 (32 x 512 x 512 4.7 us, 5.6 on the tensor cores; 128 x 1000 x 100 4.2 and 7.0; at 2^24 256 x 256 x 256 6.3 and 5.3).
template <typename T>
bool across(int P, int Q, int R) {
  constexpr int kCols = 512 / sizeof(T);
  if (Q % (16 / (int)sizeof(T))) return false;
  const double work = (double)P * (double)nf_align_up(Q, kCols) * R;
  return P <= kAcrossMost<T> || (P <= 1 << 17 && (sizeof(T) == 4 ? work <= 67108864.0 : work < 16777216.0));
}
// Ranges of r: four blocks for each SM, 64 rows each at least and 4096 (512 steps of a running sum) at most
template <typename T>
int across_splits(int P, int Q, int R) {
  const int blocks = (Q + 512 / (int)sizeof(T) - 1) / (512 / (int)sizeof(T)) * ((P + kAcrossRows<T> - 1) / kAcrossRows<T>);
  int s = 592 / blocks;
  if (s > R / 64) s = R / 64;
  if (s < (R - 1) / 4096 + 1) s = (R - 1) / 4096 + 1;
  return s < 65535 ? s : 65535;
}

// Sums of few terms (R of them, RR at most): the weight gradients of small batches, where writing the result is all the traffic.  A thread keeps its four
// columns of B in registers for 16 rows of the result; A's 64 columns lie in shared memory.  7416 x 2344 of 7 rows 14 us fp32, 13 bf16 (48 and 21 before,
// writing 10.8); of 16 rows fp32 24 us (49 by the simple kernel), bf16 25 us (21 on the tensor cores, which take over from nine).
constexpr int kOuterRows = 64;
template <typename T> constexpr int kOuterMost = sizeof(T) == 4 ? 16 : 8;

template <typename T, int RR>
__global__ void __launch_bounds__(256) outer_kernel(const T* __restrict__ A, const T* __restrict__ B, int P, int Q, int R, const Epilogue e) {
  nf_pdl_begin();
  __shared__ float as[kOuterRows][RR];
  const int p0 = blockIdx.x * kOuterRows, q = blockIdx.y * 256 + threadIdx.x % 64 * 4;
  for (int i = threadIdx.x; i < kOuterRows * RR; i += 256) {
    const int r = i / kOuterRows, p = i % kOuterRows;
    as[p][r] = r < R && p0 + p < P ? ldf(A, (size_t)r * P + p0 + p) : 0.f;
  }
  f32x2 b[RR][2];
#pragma unroll
  for (int r = 0; r < RR; ++r) {
    float v[4] = {};
    if (r < R && q < Q)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = ldf(B, (size_t)r * Q + q + j);
    b[r][0] = nf_pack2(v[0], v[1]);
    b[r][1] = nf_pack2(v[2], v[3]);
  }
  __syncthreads();
  if (q >= Q) return;  // whole: Q is a multiple of four
#pragma unroll 4
  for (int p = threadIdx.x / 64; p < min(kOuterRows, P - p0); p += 4) {
    f32x2 lo = 0, hi = 0;
#pragma unroll
    for (int r = 0; r < RR; ++r) {
      const float a = as[p][r];
      lo = nf_fma2(nf_pack2(a, a), b[r][0], lo);
      hi = nf_fma2(nf_pack2(a, a), b[r][1], hi);
    }
    float4 v;
    nf_unpack2(lo, v.x, v.y);
    nf_unpack2(hi, v.z, v.w);
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(e.out) + (size_t)(p0 + p) * Q + q) = v;
  }
}

template <typename T>
int outer_product(const T* A, const T* B, int P, int Q, int R, const Epilogue& e) {
  auto k = R <= 4 ? outer_kernel<T, 4> : R <= 8 ? outer_kernel<T, 8> : outer_kernel<T, kOuterMost<T>>;
  nf_launch(k, dim3((P + kOuterRows - 1) / kOuterRows, (Q + 255) / 256), 256, 0, A, B, P, Q, R, e);
  NF_LAUNCHED();
  return NF_OK;
}

// Many rows times a small matrix (R and Q up to 64, kRowsMost in all: 1x1 convolutions of few channels), where narrow rows come slowly through TMA
// (13 cycles each).  143962 x 16 x 56 bf16 24 us (29 on the tensor cores), 96631 x 45 x 30 fp32 27 us (147); at 64 x 64 the products bound it, 200704 rows
// of bf16 128 us (32 there).  A block takes kRowTile rows, contiguous in memory, through shared memory in whole 16-byte pieces;
// the matrix lies there as fp32 [r][q]; two threads per row compute half of its results each, pairs of neighbours in one packed multiply-add; the
// results go through shared memory again, so that everything per result (residual, pre, y) is read and written in order.
constexpr int kRowTile = 128, kRowsMost = 2048;

template <typename T>
struct RowShape {  // floats in shared memory: matrix, rows of A (an odd pitch: a warp reads one column of 32 rows), results
  int Qp, pa, py;
  __host__ __device__ RowShape(int R, int Q, int QH) : Qp(2 * QH), pa(R | 1), py(Q | 1) {}
  __host__ __device__ size_t bytes(int R) const { return ((size_t)((R * Qp + kRowTile * pa + 3) & ~3) + (size_t)kRowTile * py) * 4; }
};

template <typename T, int QH>  // results per thread
__global__ void __launch_bounds__(2 * kRowTile) rows_kernel(const T* __restrict__ A, const T* __restrict__ B, int P, int Q, int R, int b_along_r,
                                                            const Epilogue e) {
  nf_pdl_begin();
  extern __shared__ __align__(16) float rsm[];
  const RowShape<T> sh(R, Q, QH);
  float* bs = rsm;
  float* as = bs + R * sh.Qp;
  float* ys = rsm + ((R * sh.Qp + kRowTile * sh.pa + 3) & ~3);
  constexpr int NT = 2 * kRowTile;
#pragma unroll 4
  for (int i = threadIdx.x; i < R * sh.Qp; i += NT) {
    const int r = i / sh.Qp, q = i - r * sh.Qp;
    bs[i] = q < Q ? ldf(B, b_along_r ? (size_t)q * R + r : (size_t)r * Q + q) : 0.f;
  }
  const int p0 = blockIdx.x * kRowTile, rows = min(kRowTile, P - p0), na = rows * R;
  const T* from = A + (size_t)p0 * R;  // a multiple of 16 bytes from the start
#pragma unroll 2
  for (int i = threadIdx.x * 8; i < na; i += NT * 8) {
    float v[8];
    if (i + 8 <= na) {
      ld8(from + i, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = i + j < na ? ldf(from, i + j) : 0.f;
    }
    int row = i / R, c = i - row * R;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (i + j < na) as[row * sh.pa + c] = v[j];
      if (++c == R) {
        c = 0;
        ++row;
      }
    }
  }
  __syncthreads();
  const int half = threadIdx.x / kRowTile, row = threadIdx.x % kRowTile;
  if (row < rows) {
    f32x2 acc[QH / 2];
#pragma unroll
    for (int i = 0; i < QH / 2; ++i) acc[i] = 0;
    const float* a = as + row * sh.pa;
    const float* b = bs + half * QH;
#pragma unroll 4
    for (int r = 0; r < R; ++r, b += sh.Qp) {
      const f32x2 aa = nf_pack2(a[r], a[r]);
#pragma unroll
      for (int i = 0; i < QH / 4; ++i) {
        const float4 w = *reinterpret_cast<const float4*>(b + 4 * i);
        acc[2 * i] = nf_fma2(aa, nf_pack2(w.x, w.y), acc[2 * i]);
        acc[2 * i + 1] = nf_fma2(aa, nf_pack2(w.z, w.w), acc[2 * i + 1]);
      }
    }
#pragma unroll
    for (int i = 0; i < QH / 2; ++i) {
      float lo, hi;
      nf_unpack2(acc[i], lo, hi);
      const int q = half * QH + 2 * i;
      if (q < Q) ys[row * sh.py + q] = lo;
      if (q + 1 < Q) ys[row * sh.py + q + 1] = hi;
    }
  }
  __syncthreads();
  const int ny = rows * Q;
  const size_t at0 = (size_t)p0 * Q;
  for (int i = threadIdx.x * 8; i < ny; i += NT * 8) {  // eight results in a row of memory
    float v[8];
    int r = i / Q, q = i - r * Q;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = i + j < ny ? ys[r * sh.py + q] + (e.bias ? e.bias[q] : 0.f) : 0.f;
      if (++q == Q) {
        q = 0;
        ++r;
      }
    }
    if (i + 8 <= ny) {
      if (e.residual) {
        float s[8];
        ld8(reinterpret_cast<const T*>(e.residual) + at0 + i, s);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += s[j];
      }
      if (e.pre) {
        float s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = v[j];
        st8(reinterpret_cast<T*>(e.pre) + at0 + i, s);
      }
      if (e.act != NF_ACT_NONE) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = nf_act_value<T>(v[j], e.act);
      }
      st8(reinterpret_cast<T*>(e.out) + at0 + i, v);
    } else {
      for (int j = 0; j < 8 && i + j < ny; ++j) {
        float t = v[0];
#pragma unroll
        for (int k = 1; k < 8; ++k) t = j == k ? v[k] : t;
        if (e.residual) t += ldf(reinterpret_cast<const T*>(e.residual), at0 + i + j);
        if (e.pre) stf(reinterpret_cast<T*>(e.pre), at0 + i + j, t);
        stf(reinterpret_cast<T*>(e.out), at0 + i + j, nf_act_value<T>(t, e.act));
      }
    }
  }
}

template <typename T>
int rows_product(const T* A, const T* B, int P, int Q, int R, bool b_along_r, const Epilogue& e) {
  const int QH = Q <= 16 ? 8 : Q <= 32 ? 16 : 32;
  auto k = QH == 8 ? rows_kernel<T, 8> : QH == 16 ? rows_kernel<T, 16> : rows_kernel<T, 32>;
  const size_t smem = RowShape<T>(R, Q, QH).bytes(R);
  static bool ready[64];
  int dev = 0;
  NF_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return NF_EUNSUPPORTED;
  if (!ready[dev]) {
    const int most = (int)RowShape<T>(64, 64, 32).bytes(64);
    NF_CUDA(cudaFuncSetAttribute(rows_kernel<T, 8>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    NF_CUDA(cudaFuncSetAttribute(rows_kernel<T, 16>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    NF_CUDA(cudaFuncSetAttribute(rows_kernel<T, 32>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    ready[dev] = true;
  }
  nf_launch(k, (unsigned)((P + kRowTile - 1) / kRowTile), 2 * kRowTile, smem, A, B, P, Q, R, (int)b_along_r, e);
  NF_LAUNCHED();
  return NF_OK;
}

// part[block][n]: sums of g over a range of rows.  V columns per thread (16 bytes of a row where rows are made of such pieces), lx threads along a
// row (a power of two), the others on the rows beside it, so that a narrow matrix keeps as many loads on their way as a wide one.  235 x 1200 fp32
// 4 us behind the weight gradient (12 with 256 threads, 32 along the row), 100000 x 32 10 (19).
constexpr int kSumThreads = 1024;

template <typename T, int V>
__global__ void __launch_bounds__(kSumThreads) column_sums_kernel(const T* __restrict__ g, int M, int N, int lx, float* __restrict__ part) {
  nf_pdl_begin();
  __shared__ __align__(16) float sm[kSumThreads * V];
  const int tx = threadIdx.x % lx, ty = threadIdx.x / lx, nty = blockDim.x / lx, n = (blockIdx.y * lx + tx) * V;
  const int m0 = (int)((long long)M * blockIdx.x / gridDim.x), m1 = (int)((long long)M * (blockIdx.x + 1) / gridDim.x);
  float s[V];
#pragma unroll
  for (int e = 0; e < V; ++e) s[e] = 0.f;
  if (n < N) {
#pragma unroll 4
    for (int m = m0 + ty; m < m1; m += nty) {
      const T* at = g + (size_t)m * N + n;
      if constexpr (V == 8) {
        float v[8];
        ld8(at, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += v[e];
      } else {
        s[0] += ldf(at, 0);
      }
    }
  }
  float* mine = sm + threadIdx.x;  // one value of every thread after another
#pragma unroll
  for (int e = 0; e < V; ++e) mine[e * kSumThreads] = s[e];
  for (int h = nty / 2; h; h /= 2) {
    __syncthreads();
    if (ty < h) {
#pragma unroll
      for (int e = 0; e < V; ++e) mine[e * kSumThreads] += mine[e * kSumThreads + h * lx];
    }
  }
  if (ty == 0 && n < N) {
#pragma unroll
    for (int e = 0; e < V; ++e) part[(size_t)blockIdx.x * N + n + e] = mine[e * kSumThreads];
  }
}

// g = dy act'(saved), eight elements a thread: memory bounds it (35 M bf16 elements of ReLU 30 us, 7.1 TB/s with part of the write left in L2; GELU 70 M 85 us)
template <typename T>
__global__ void __launch_bounds__(256) act_backward_kernel(const T* saved, const T* dy, size_t n, int act, T* g) {
  nf_pdl_begin();
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  if (i + 8 <= n) {
    float s[8], d[8];
    ld8(saved + i, s);
    ld8(dy + i, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = nf_act_dz<T>(s[e], d[e], act);
    st8(g + i, d);
  } else {
    for (size_t e = i; e < n; ++e) stf(g, e, nf_act_dz<T>(ldf(saved, e), ldf(dy, e), act));
  }
}

// Operand copies for the tensor cores: rows padded to 16 bytes, and fp32 cut into three bf16 parts whose sum is exact (each is the
// nearest bf16 to what the earlier ones leave).  Memory bounds it; both operands in one launch: a product of
// 1777 x 2048 x 1000 62 us (64 in two), 318 x 840 x 2408 24.9 (26.5).
struct PartsOf {
  const void* src;
  bf16* dst;
  size_t rows, plane;
  int len, ld;
  unsigned blocks;  // 0: this operand is taken as it lies
};

template <typename T>
__global__ void __launch_bounds__(256) parts_kernel(const PartsOf first, const PartsOf second) {  // the first blocks on one operand, the others on the other
  nf_pdl_begin();
  constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
  const bool other = blockIdx.x >= first.blocks;
  const PartsOf& o = other ? second : first;
  const size_t i = (size_t)(blockIdx.x - (other ? first.blocks : 0)) * 256 + threadIdx.x, plane = o.plane;
  const int len = o.len, ld = o.ld, per = ld / 8;
  const size_t r = i >> 32 ? i / per : (uint32_t)i / (uint32_t)per;
  const int c = (int)(i - r * per) * 8;
  if (r >= o.rows) return;
  const T* from = (const T*)o.src + r * len + c;
  bf16* dst = o.dst;
  float v[8];
  if (c + 8 <= len && len % (16 / (int)sizeof(T)) == 0) {
    ld8(from, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < len ? ldf(from, e) : 0.f;
  }
#pragma unroll
  for (int k = 0; k < kParts; ++k) {
    float h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = v[e];
    st8(dst + k * plane + r * ld + c, h);  // h: as stored
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] -= h[e];
  }
}

int pad8(int n) { return (n + 7) / 8 * 8; }

// One of the three products as the kernels see it: A [a_rows][a_len] and B [b_rows][b_len] as they lie
struct Product {
  int P, Q, R;
  bool a_along_r, b_along_r;
  int a_rows() const { return a_along_r ? P : R; }
  int a_len() const { return a_along_r ? R : P; }
  int b_rows() const { return b_along_r ? Q : R; }
  int b_len() const { return b_along_r ? R : Q; }
};

// bf16: always (a 128 x 64 x 10 product took 6 us there and 10 us on the CUDA cores).  fp32: from 2^26 multiply-adds on, counted in the 64 x 64 tiles of
// the simple kernel, where what cutting the operands into parts costs is earned back (256 x 256 x 256 16 us there, 9 us here; 512 x 512 x 512 17 us and
// 24 us) -- with a side of a few too: 100000 x 512 x 10 195 us there, 301 here, its gradients 65 and 155 us there, 149 and 350 here.
bool on_tensor_cores(int dtype, const Product& d) {
  return dtype == NF_BF16 || (double)nf_align_up(d.P, 64) * (double)nf_align_up(d.Q, 64) * d.R >= 67108864.0;
}
bool few_across(int dtype, const Product& d) {
  return d.a_along_r && !d.b_along_r && (dtype == NF_F32 ? across<float>(d.P, d.Q, d.R) : across<bf16>(d.P, d.Q, d.R));
}
bool needs_copy(int dtype, int len) { return dtype == NF_F32 || len % 8; }
size_t copy_bytes(int dtype, int rows, int len) {
  return needs_copy(dtype, len) ? nf_align_up((size_t)rows * pad8(len) * 2 * (dtype == NF_F32 ? 3 : 1), 256) : 0;
}

int simple_splits(int P, int Q, int R) {
  const long tiles = (long)((P + 63) / 64) * ((Q + 63) / 64);
  long s = 296 / tiles;
  if (s > R / 128) s = R / 128;  // eight steps of 16 at least
  return s < 1 ? 1 : (int)s;
}

// Scratch that covers a product of M rows and every one of fewer, so that what was allocated for the largest batch serves a ragged last one: fewer rows
// mean more splits, and other kernels.  Copies of operands grow with M.  Partial sums:
//  - where P is M (forward, input gradient) splits * tiles <= `places` bounds splits * P by places * side / (tiles along q), and splits and P each have a bound of
//    their own; across_splits likewise, over the P that across() takes;
//  - where R is M (weight gradient) splits grow with it; the simple kernel's as far as it is used.
size_t split_bytes(int P, int Q, long most, int side, long places) {
  const long tq = (Q + side - 1) / side;
  if (most < 2 || places / tq < 2) return 0;
  const double rows = (double)most * P, cap = (double)places * side / tq;
  return (size_t)(rows < cap ? rows : cap) * Q * 4;
}
template <typename T>
size_t across_bytes(const Product& d) {
  constexpr int cols = 512 / (int)sizeof(T);
  if (d.Q % (16 / (int)sizeof(T))) return 0;
  const double columns = (double)nf_align_up(d.Q, cols) * d.R, fit = (sizeof(T) == 4 ? 67108864.0 : 16777216.0) / columns;
  double P = fit < (double)(1 << 17) ? fit : (double)(1 << 17);
  if (P < kAcrossMost<T>) P = kAcrossMost<T>;
  if (P > d.P) P = d.P;
  const long blocks = (d.Q + cols - 1) / cols;
  double rows = 0;
  if (592 / blocks >= 2 && d.R >= 128) {
    rows = (double)(d.R / 64) * P;
    const double cap = 592.0 * kAcrossRows<T> / blocks;
    if (rows > cap) rows = cap;
  }
  const double forced = (d.R - 1) / 4096 + 1;
  if (forced > 1 && rows < forced * P) rows = forced * P;
  return (size_t)rows * d.Q * 4;
}
size_t product_bytes(int dtype, const Product& d) {
  const bool f32 = dtype == NF_F32;
  size_t sums = 0;
  auto most = [&](size_t b) { sums = b > sums ? b : sums; };
  if (d.a_along_r) {
    most(split_bytes(d.P, d.Q, nf_gemm_splits(1, 1, d.R, f32 ? 3 : 1), 128, 148));
    if (f32) most(split_bytes(d.P, d.Q, d.R / 128, 64, 296));
    if (!d.b_along_r) most(f32 ? across_bytes<float>(d) : across_bytes<bf16>(d));
  } else {
    auto whole = [&](int s) { most(s > 1 ? (size_t)s * d.P * d.Q * 4 : 0); };
    whole(nf_gemm_splits(d.P, d.Q, d.R, f32 ? 3 : 1));
    if (f32) whole(simple_splits(d.P, d.Q, d.R));
  }
  return sums + (on_tensor_cores(dtype, d) ? copy_bytes(dtype, d.a_rows(), d.a_len()) + copy_bytes(dtype, d.b_rows(), d.b_len()) : 0);
}

template <typename T>
int join(const float* part, int splits, int P, int Q, const Epilogue& e) {
  const size_t n = (size_t)P * Q;
  if (n < 148 * 1024 && splits > 4)
    nf_launch(gemm_join_kernel<T, 8>, (unsigned)((n + 31) / 32), 256, 0, part, splits, n, Q, e);
  else
    nf_launch(gemm_join_kernel<T, 1>, (unsigned)((n + 255) / 256), 256, 0, part, splits, n, Q, e);
  NF_LAUNCHED();
  return NF_OK;
}

int simple_product(const Product& d, const float* A, const float* B, float* part, const Epilogue& e) {
  const int splits = simple_splits(d.P, d.Q, d.R);
  const size_t la = d.a_len(), lb = d.b_len();
  nf_launch(gemm_simple_kernel, dim3((d.P + 63) / 64, (d.Q + 63) / 64, splits), 256, 0, A, d.a_along_r ? la : 1, d.a_along_r ? 1 : la,
            B, d.b_along_r ? lb : 1, d.b_along_r ? 1 : lb, d.P, d.Q, d.R, part, e);
  NF_LAUNCHED();
  return splits > 1 ? join<float>(part, splits, d.P, d.Q, e) : NF_OK;
}

template <typename T>
int across_product(const T* A, const T* B, float* part, const Product& d, const Epilogue& e) {
  const int splits = across_splits<T>(d.P, d.Q, d.R), cols = 512 / (int)sizeof(T);
  auto k = d.P == 1 ? across_kernel<T, 1> : d.P == 2 ? across_kernel<T, 2> : across_kernel<T, kAcrossRows<T>>;
  if constexpr (sizeof(T) == 4)
    if (d.P == 3 || d.P == 4) k = across_kernel<T, 4>;
  nf_launch(k, dim3((d.Q + cols - 1) / cols, (d.P + kAcrossRows<T> - 1) / kAcrossRows<T>, splits), 256, 0, A, B, d.P, d.Q, d.R, part, e);
  NF_LAUNCHED();
  return splits > 1 ? join<T>(part, splits, d.P, d.Q, e) : NF_OK;
}

// Where an operand will lie for the tensor cores, and what copying it takes
PartsOf operand(int dtype, const void* src, int rows, int len, bool along_r, char*& scratch, GemmOperand* o) {
  *o = {(const bf16*)src, (size_t)len, 0, along_r};
  if (!needs_copy(dtype, len)) return PartsOf{};
  const int ld = pad8(len);
  const size_t plane = (size_t)rows * ld, blocks = (plane / 8 + 255) / 256;
  const PartsOf p{src, (bf16*)scratch, (size_t)rows, plane, len, ld, blocks > 0x3fffffffull ? ~0u : (unsigned)blocks};
  *o = {(const bf16*)scratch, (size_t)ld, plane, along_r};
  scratch += copy_bytes(dtype, rows, len);
  return p;
}

template <typename T>
int product(const Product& d, const void* A, const void* B, void* scratch, const Epilogue& e) {
  const int dtype = sizeof(T) == 4 ? NF_F32 : NF_BF16;
  if ((d.Q + 63) / 64 > 65535) return NF_EUNSUPPORTED;
  if (d.a_along_r && d.R <= 64 && d.Q <= 64 && d.R * d.Q <= kRowsMost) return rows_product<T>((const T*)A, (const T*)B, d.P, d.Q, d.R, d.b_along_r, e);
  if (d.a_along_r && d.b_along_r && thin_pays<T>(d.P, d.Q, d.R))
    return d.R % (16 / (int)sizeof(T)) == 0 ? thin_product<T, true>((const T*)A, (const T*)B, d.P, d.Q, d.R, e)
                                            : thin_product<T, false>((const T*)A, (const T*)B, d.P, d.Q, d.R, e);
  if (few_across(dtype, d)) return across_product<T>((const T*)A, (const T*)B, (float*)scratch, d, e);
  if (!d.a_along_r && !d.b_along_r && e.out_f32 && d.R <= kOuterMost<T> && d.Q % 4 == 0) return outer_product<T>((const T*)A, (const T*)B, d.P, d.Q, d.R, e);
  if constexpr (sizeof(T) == 4) {
    if (!on_tensor_cores(dtype, d)) return simple_product(d, (const float*)A, (const float*)B, (float*)scratch, e);
  }
  char* s = (char*)scratch;
  GemmProblem g{};
  g.P = d.P; g.Q = d.Q; g.R = d.R;
  g.planes = dtype == NF_F32 ? 3 : 1;
  g.out_f32 = dtype == NF_F32 || e.out_f32;
  const PartsOf a = operand(dtype, A, d.a_rows(), d.a_len(), d.a_along_r, s, &g.A), b = operand(dtype, B, d.b_rows(), d.b_len(), d.b_along_r, s, &g.B);
  if (a.blocks == ~0u || b.blocks == ~0u) return NF_EUNSUPPORTED;
  if (a.blocks + b.blocks) {
    nf_launch(parts_kernel<T>, a.blocks + b.blocks, 256, 0, a, b);
    NF_LAUNCHED();
  }
  const int rc = nf_gemm_tc(g, e, (float*)s);
  const int splits = nf_gemm_splits(d.P, d.Q, d.R, g.planes);
  return rc == NF_OK && splits > 1 ? join<T>((const float*)s, splits, d.P, d.Q, e) : rc;
}

struct SumPlan {
  int V, lx, cols, threads, blocks;  // columns per thread, threads along a row, blocks along it, threads per block, ranges of rows
};
// One range, whose sums are the result, where a thread has 16 rows or fewer; else two blocks per SM, with eight rows per thread at least
SumPlan sum_plan(int M, int N) {
  SumPlan s{N % 8 == 0 ? 8 : 1, 1, 1, kSumThreads, 1};
  const int pieces = N / s.V;
  while (s.lx < 32 && s.lx < pieces) s.lx *= 2;
  s.cols = (pieces + s.lx - 1) / s.lx;
  while (s.threads > 128 && s.threads / s.lx > M / 2) s.threads /= 2;
  const int nty = s.threads / s.lx, want = (296 + s.cols - 1) / s.cols, most = M / (8 * nty);
  if (M > 16 * nty) s.blocks = want < most ? want : most;
  return s;
}

template <typename T>
void column_sums(const SumPlan& s, const T* g, int M, int N, float* part) {
  nf_launch(s.V == 8 ? column_sums_kernel<T, 8> : column_sums_kernel<T, 1>, dim3(s.blocks, s.cols), s.threads, 0, g, M, N, s.lx, part);
}

bool large(int M, int K, int N) { return M > 1 << 30 || K > 1 << 30 || N > 1 << 30; }  // positions run on beyond the last one, in 32 bits
bool sizes_ok(int dtype, int M, int K, int N) { return (dtype == NF_F32 || dtype == NF_BF16) && M >= 1 && K >= 1 && N >= 1; }

Product forward_of(int M, int K, int N) { return {M, N, K, true, true}; }
Product dgrad_of(int M, int K, int N) { return {M, K, N, true, false}; }
Product wgrad_of(int M, int K, int N) { return {N, K, M, false, false}; }

}  // namespace

extern "C" size_t nf_linear_scratch_bytes(int dtype, int M, int K, int N) {
  if (!sizes_ok(dtype, M, K, N) || large(M, K, N)) return 0;
  size_t b = 0;
  for (const Product& d : {forward_of(M, K, N), dgrad_of(M, K, N), wgrad_of(M, K, N)}) {
    const size_t n = product_bytes(dtype, d);
    if (n > b) b = n;
  }
  return b + (size_t)sum_plan(M, N).blocks * N * 4 + 256;
}

extern "C" int nf_linear_forward(int dtype, const void* x, const void* w, const float* bias, const void* residual, int M, int K, int N, int act,
                                 void* scratch, size_t scratch_bytes, void* pre, void* y) {
  if (!x || !w || !scratch || !y || !sizes_ok(dtype, M, K, N) || !nf_act_ok(act)) return NF_EINVAL;
  if (((uintptr_t)x | (uintptr_t)w | (uintptr_t)bias | (uintptr_t)residual | (uintptr_t)scratch | (uintptr_t)pre | (uintptr_t)y) & 15) return NF_EALIGN;
  const size_t es = nf_esize(dtype), xb = es * M * K, wb = es * N * K, yb = es * M * N;
  for (const void* o : {(const void*)y, (const void*)pre})
    if (nf_overlap(o, yb, x, xb) || nf_overlap(o, yb, w, wb) || nf_overlap(o, yb, residual, yb) || nf_overlap(o, yb, bias, (size_t)N * 4))
      return NF_EINVAL;
  if (nf_overlap(y, yb, pre, yb)) return NF_EINVAL;
  if (large(M, K, N)) return NF_EUNSUPPORTED;
  const size_t need = nf_linear_scratch_bytes(dtype, M, K, N);
  if (scratch_bytes < need) return NF_ENOWS;
  for (const void* t : {(const void*)y, (const void*)pre, residual})
    if (nf_overlap(scratch, need, t, yb)) return NF_EINVAL;
  if (nf_overlap(scratch, need, x, xb) || nf_overlap(scratch, need, w, wb) || nf_overlap(scratch, need, bias, (size_t)N * 4)) return NF_EINVAL;
  const Epilogue e{bias, residual, act, pre, y, 0};
  const Product d = forward_of(M, K, N);
  return dtype == NF_F32 ? product<float>(d, x, w, scratch, e) : product<bf16>(d, x, w, scratch, e);
}

extern "C" int nf_linear_dgrad(int dtype, const void* g, const void* w, int M, int K, int N, void* scratch, size_t scratch_bytes, void* dx) {
  if (!g || !w || !scratch || !dx || !sizes_ok(dtype, M, K, N)) return NF_EINVAL;
  if (((uintptr_t)g | (uintptr_t)w | (uintptr_t)scratch | (uintptr_t)dx) & 15) return NF_EALIGN;
  const size_t es = nf_esize(dtype), xb = es * M * K;
  if (nf_overlap(dx, xb, g, es * M * N) || nf_overlap(dx, xb, w, es * N * K)) return NF_EINVAL;
  if (large(M, K, N)) return NF_EUNSUPPORTED;
  const size_t need = nf_linear_scratch_bytes(dtype, M, K, N);
  if (scratch_bytes < need) return NF_ENOWS;
  if (nf_overlap(scratch, need, dx, xb) || nf_overlap(scratch, need, g, es * M * N) || nf_overlap(scratch, need, w, es * N * K)) return NF_EINVAL;
  const Epilogue e{nullptr, nullptr, NF_ACT_NONE, nullptr, dx, 0};
  const Product d = dgrad_of(M, K, N);
  return dtype == NF_F32 ? product<float>(d, g, w, scratch, e) : product<bf16>(d, g, w, scratch, e);
}

extern "C" int nf_linear_wgrad(int dtype, const void* x, const void* g, int M, int K, int N, void* scratch, size_t scratch_bytes, float* dw,
                               float* db) {
  if (!x || !g || !scratch || !dw || !sizes_ok(dtype, M, K, N)) return NF_EINVAL;
  if (((uintptr_t)x | (uintptr_t)g | (uintptr_t)scratch | (uintptr_t)dw | (uintptr_t)db) & 15) return NF_EALIGN;
  const size_t es = nf_esize(dtype), wb = (size_t)4 * N * K, bb = (size_t)4 * N;
  if (nf_overlap(dw, wb, x, es * M * K) || nf_overlap(dw, wb, g, es * M * N) || nf_overlap(db, bb, x, es * M * K) ||
      nf_overlap(db, bb, g, es * M * N) || nf_overlap(dw, wb, db, bb))
    return NF_EINVAL;
  if (large(M, K, N)) return NF_EUNSUPPORTED;
  const size_t need = nf_linear_scratch_bytes(dtype, M, K, N);
  if (scratch_bytes < need) return NF_ENOWS;
  if (nf_overlap(scratch, need, dw, wb) || nf_overlap(scratch, need, db, bb) || nf_overlap(scratch, need, x, es * M * K) ||
      nf_overlap(scratch, need, g, es * M * N))
    return NF_EINVAL;
  const SumPlan sums = sum_plan(M, N);
  if (db && (N + 31) / 32 > 65535) return NF_EUNSUPPORTED;  // blocks along a row, where a thread has one column
  const Epilogue e{nullptr, nullptr, NF_ACT_NONE, nullptr, dw, 1};
  const Product d = wgrad_of(M, K, N);
  const int rc = dtype == NF_F32 ? product<float>(d, g, x, scratch, e) : product<bf16>(d, g, x, scratch, e);
  if (rc != NF_OK || !db) return rc;
  float* part = sums.blocks > 1 ? (float*)scratch : db;  // the product's partial sums have been read by now
  if (dtype == NF_F32) column_sums(sums, (const float*)g, M, N, part);
  else column_sums(sums, (const bf16*)g, M, N, part);
  NF_LAUNCHED();
  return sums.blocks > 1 ? nf_k_sum_parts(part, sums.blocks, N, db, true) : NF_OK;
}

extern "C" int nf_act_backward(int dtype, int act, const void* saved, const void* dy, long long n, void* g) {
  if (!saved || !dy || !g || n < 1 || (dtype != NF_F32 && dtype != NF_BF16) || !nf_act_ok(act)) return NF_EINVAL;
  if (((uintptr_t)saved | (uintptr_t)dy | (uintptr_t)g) & 15) return NF_EALIGN;
  const size_t bytes = (size_t)n * nf_esize(dtype);
  if ((g != dy && nf_overlap(g, bytes, dy, bytes)) || (g != saved && nf_overlap(g, bytes, saved, bytes))) return NF_EINVAL;
  const size_t blocks = ((size_t)n + 2047) / 2048;
  if (blocks > 0x7fffffffull) return NF_EUNSUPPORTED;
  if (dtype == NF_F32)
    nf_launch(act_backward_kernel<float>, (unsigned)blocks, 256, 0, (const float*)saved, (const float*)dy, (size_t)n, act, (float*)g);
  else
    nf_launch(act_backward_kernel<bf16>, (unsigned)blocks, 256, 0, (const bf16*)saved, (const bf16*)dy, (size_t)n, act, (bf16*)g);
  NF_LAUNCHED();
  return NF_OK;
}
