// Group normalisation of channels-last maps with the activation behind it, forward and backward.
//
//   mean, var over the P pixels and C/groups channels of every (image, group);  xh = (x - mean) rstd,  z = gamma xh + beta,  y = act(z)
//   dz = dy act'(z);  dgamma = sum dz xh, dbeta = sum dz;
//   dx = rstd (gamma dz - m1 - xh m2),  m1, m2 = means over the group of gamma dz and gamma dz xh
//
// One launch does a pass over the data for the sums and a second one for the result.  A cluster of CS blocks owns one image (or one
// slice of its channels, whole groups), each block a range of its pixels; the blocks' channel sums meet through distributed
// shared memory, and the second pass finds the image in L2, so that HBM carries every tensor once.
//
// Sums: a thread adds in fp32 what it sees of its channels, after subtracting the image's first pixel of the channel (forward), so that
// a mean far from zero costs no digits; blocks, ranks and the channels of a group are joined in fp64.  xh and z are formed by
// separately rounded operations in this order in both directions, so that the gradient's ReLU mask is the forward's.
#include <cooperative_groups.h>

#include "nf_act.cuh"
#include "nf_ldst.cuh"
#include "nf_tc.h"

namespace {
namespace cg = cooperative_groups;

constexpr int kNT = 256;
constexpr int kMaxCs = 4096;       // channels of a slice: totals of all of them lie in shared memory
constexpr int kMaxCluster = 16;    // above 8 is outside the portable limit and has to be allowed per kernel
constexpr int kMaxParts = 1184;    // rows of dgamma / dbeta partials at most: 8 blocks on each of 148 SMs

struct GnArgs {
  const void *x, *dy;
  const float *gamma, *beta;
  float *mean, *rstd;  // read in the backward pass
  void* out;           // y or dx
  float* part;         // backward: [rows][2][C] partial sums of dbeta, dgamma
  int N, P, C, G, cpg;
  int slices, Cs, vpr;  // channel slices, channels and vectors per slice
  int CS, stride;       // blocks per cluster; images between two turns of a cluster
  int act;
  float eps;
};

template <typename T, int V>
__device__ __forceinline__ void ldv(const T* p, float (&v)[V]) {
  if constexpr (V == 8) {
    ld8(p, v);
  } else if constexpr (V == 4 && std::is_same<T, float>::value) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = ldf(p, e);
  }
}
template <typename T, int V>
__device__ __forceinline__ void stv(T* p, float (&v)[V]) {
  if constexpr (V == 8) {
    st8(p, v);
  } else if constexpr (V == 4 && std::is_same<T, float>::value) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) stf(p, e, v[e]);
  }
}

__device__ __forceinline__ float normalised(float x, float mean, float rstd) { return __fmul_rn(__fsub_rn(x, mean), rstd); }
__device__ __forceinline__ float affine(float xh, float g, float b) { return __fadd_rn(__fmul_rn(xh, g), b); }

// V channels per thread; threads run along the channels of a pixel first, then along the pixels
template <typename T, int V, bool BWD>
__global__ void __launch_bounds__(kNT) group_norm_kernel(const GnArgs a) {
  nf_pdl_begin();
  extern __shared__ __align__(16) float sm[];
  float* red = sm;                        // [2V][kNT] tree reduction
  float* tot = red + 2 * V * kNT;         // [2][2][Cs] this block's channel sums, two images in turn
  float* gsm = tot + 4 * a.Cs;            // [2][groups of the slice]: mean and rstd (forward), m1 and m2 (backward)
  float* acc = gsm + 2 * (a.Cs / a.cpg);  // backward: [2][Cs] sums over the images of this block
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = blockIdx.x % a.CS, cid = blockIdx.x / a.CS, slice = cid % a.slices;
  const int gps = a.Cs / a.cpg;  // groups per slice
  const int c0 = slice * a.Cs;
  const int cols = a.vpr < kNT ? a.vpr : kNT, R = kNT / cols;
  const int tc = threadIdx.x % cols, tr = threadIdx.x / cols;
  const bool on = tr < R;
  const int p0 = (int)((long long)a.P * rank / a.CS), p1 = (int)((long long)a.P * (rank + 1) / a.CS);
  const T* x = (const T*)a.x;
  const T* dy = (const T*)a.dy;
  T* out = (T*)a.out;
  if constexpr (BWD) {
    for (int i = threadIdx.x; i < 2 * a.Cs; i += kNT) acc[i] = 0.f;
  }
  int turn = 0;
  for (int n = cid / a.slices; n < a.N; n += a.stride, turn ^= 1) {
    const size_t base = (size_t)n * a.P * a.C + c0;
    float* mine = tot + turn * 2 * a.Cs;
    for (int cv0 = 0; cv0 < a.vpr; cv0 += cols) {
      const int cv = cv0 + tc;
      const bool here = on && cv < a.vpr;
      float s[V], q[V];
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] = q[e] = 0.f;
      if (here) {
        const size_t col = base + (size_t)cv * V;
        if constexpr (!BWD) {
          float k[V];
          ldv<T, V>(x + col, k);
#pragma unroll 4
          for (int p = p0 + tr; p < p1; p += R) {
            float v[V];
            ldv<T, V>(x + col + (size_t)p * a.C, v);
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float d = v[e] - k[e];
              s[e] += d;
              q[e] = fmaf(d, d, q[e]);
            }
          }
        } else {
          float mu[V], rs[V], ga[V], be[V];
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const int c = c0 + cv * V + e;
            mu[e] = a.mean[(size_t)n * a.G + c / a.cpg];
            rs[e] = a.rstd[(size_t)n * a.G + c / a.cpg];
            ga[e] = a.gamma[c];
            be[e] = a.beta[c];
          }
#pragma unroll 2
          for (int p = p0 + tr; p < p1; p += R) {
            float v[V], g[V];
            ldv<T, V>(x + col + (size_t)p * a.C, v);
            ldv<T, V>(dy + col + (size_t)p * a.C, g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float xh = normalised(v[e], mu[e], rs[e]);
              const float dz = g[e] * nf_act_grad<T>(affine(xh, ga[e], be[e]), a.act);
              s[e] += dz;
              q[e] = fmaf(dz, xh, q[e]);
            }
          }
        }
      }
      // rows of threads are folded in halves
      __syncthreads();
#pragma unroll
      for (int e = 0; e < V; ++e) {
        red[e * kNT + threadIdx.x] = s[e];
        red[(V + e) * kNT + threadIdx.x] = q[e];
      }
      for (int left = R; left > 1;) {
        const int half = (left + 1) / 2;
        __syncthreads();
        if (tr + half < left) {
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) red[e * kNT + threadIdx.x] += red[e * kNT + threadIdx.x + half * cols];
        }
        left = half;
      }
      __syncthreads();
      const int width = (a.vpr - cv0 < cols ? a.vpr - cv0 : cols) * V;  // channels of this chunk
      for (int i = threadIdx.x; i < 2 * width; i += kNT) {
        const int w = i / width, c = i - w * width;
        mine[w * a.Cs + cv0 * V + c] = red[(w * V + c % V) * kNT + c / V];
      }
    }
    cluster.sync();
    // every block joins the ranks' sums and the channels of each group: L lanes per group
    {
      int L = 1;
      while (L < a.cpg && L < 32) L *= 2;
      const int lane = threadIdx.x % L, per = kNT / L;
      for (int g0 = 0; g0 < gps; g0 += per) {
        const int g = g0 + threadIdx.x / L;
        double A = 0, B = 0;
        if (g < gps) {
          for (int i = lane; i < a.cpg; i += L) {
            const int c = g * a.cpg + i;
            double S = 0, Q = 0;
            for (int r = 0; r < a.CS; ++r) {
              const float* o = cluster.map_shared_rank(mine, r);
              S += o[c];
              Q += o[a.Cs + c];
            }
            if constexpr (!BWD) {  // mean and sum of squared deviations of the channel; the group's by their sums
              const double d = S / a.P, m = (double)ldf(x, base + c) + d;
              A += m;
              B += Q / a.P - d * d + m * m;
            } else {
              const double gm = a.gamma[c0 + c];
              A += gm * S;
              B += gm * Q;
            }
          }
        }
        for (int o = 1; o < L; o *= 2) {
          A += __shfl_xor_sync(0xffffffffu, A, o);
          B += __shfl_xor_sync(0xffffffffu, B, o);
        }
        if (g < gps && lane == 0) {
          if constexpr (!BWD) {
            const double m = A / a.cpg, var = B / a.cpg - m * m;
            const float mf = (float)m, rf = (float)(1.0 / sqrt((var > 0 ? var : var == var ? 0 : var) + (double)a.eps));
            gsm[g] = mf;
            gsm[gps + g] = rf;
            if (rank == 0) {
              a.mean[(size_t)n * a.G + slice * gps + g] = mf;
              a.rstd[(size_t)n * a.G + slice * gps + g] = rf;
            }
          } else {
            const double M = (double)a.cpg * a.P;
            gsm[g] = (float)(A / M);
            gsm[gps + g] = (float)(B / M);
          }
        }
      }
      if constexpr (BWD) {
        for (int i = threadIdx.x; i < 2 * a.Cs; i += kNT) acc[i] += mine[i];
      }
    }
    __syncthreads();
    for (int cv = tc; on && cv < a.vpr; cv += cols) {
      const size_t col = base + (size_t)cv * V;
      float mu[V], rs[V], ga[V], be[V];
      float m1[BWD ? V : 1], m2[BWD ? V : 1];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int c = cv * V + e, g = c / a.cpg;
        ga[e] = a.gamma[c0 + c];
        be[e] = a.beta[c0 + c];
        if constexpr (!BWD) {
          mu[e] = gsm[g];
          rs[e] = gsm[gps + g];
        } else {
          mu[e] = a.mean[(size_t)n * a.G + slice * gps + g];
          rs[e] = a.rstd[(size_t)n * a.G + slice * gps + g];
          m1[e] = gsm[g];
          m2[e] = gsm[gps + g];
        }
      }
#pragma unroll 2
      for (int p = p0 + tr; p < p1; p += R) {
        const size_t at = col + (size_t)p * a.C;
        float v[V];
        ldv<T, V>(x + at, v);
        if constexpr (!BWD) {
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = nf_act_value<T>(affine(normalised(v[e], mu[e], rs[e]), ga[e], be[e]), a.act);
        } else {
          float g[V];
          ldv<T, V>(dy + at, g);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float xh = normalised(v[e], mu[e], rs[e]);
            const float dz = g[e] * nf_act_grad<T>(affine(xh, ga[e], be[e]), a.act);
            v[e] = rs[e] * (fmaf(ga[e], dz, -m1[e]) - xh * m2[e]);
          }
        }
        stv<T, V>(out + at, v);
      }
    }
  }
  if constexpr (BWD) {
    __syncthreads();
    const int row = (cid / a.slices) * a.CS + rank;
    for (int i = threadIdx.x; i < 2 * a.Cs; i += kNT) {
      const int w = i / a.Cs, c = i - w * a.Cs;
      a.part[((size_t)row * 2 + w) * a.C + c0 + c] = acc[i];
    }
  }
  cluster.sync();  // no block leaves while another may still read its sums
}

// dbeta, dgamma: the rows of partials added in fp64, eight chains of every eighth row, joined in order
__global__ void __launch_bounds__(256) group_norm_param_kernel(const float* __restrict__ part, int rows, int C, float* __restrict__ dgamma,
                                                               float* __restrict__ dbeta) {
  nf_pdl_begin();
  __shared__ double sm[8][32];
  const int tx = threadIdx.x % 32, ty = threadIdx.x / 32;
  const int i = blockIdx.x * 32 + tx;
  double s = 0;
  if (i < 2 * C)
    for (int r = ty; r < rows; r += 8) s += part[(size_t)r * 2 * C + i];
  sm[ty][tx] = s;
  __syncthreads();
  if (ty == 0 && i < 2 * C) {
    for (int k = 1; k < 8; ++k) s += sm[k][tx];
    (i < C ? dbeta[i] : dgamma[i - C]) = (float)s;
  }
}

struct GnPlan {
  int V, slices, CS, clusters;
  size_t smem;
};

GnPlan plan_gn(int dtype, int N, int P, int C, int groups, bool bwd) {
  GnPlan pl;
  const int cpg = C / groups;
  const size_t es = nf_esize(dtype), image = (size_t)P * C * es;
  // 16 bytes per thread where the slices allow it, else single channels.  A slice is some whole groups: all of them, fewer where C is
  // above kMaxCs or where one image per (largest portable) cluster would leave most SMs idle, as long as a pixel of it is 64 bytes.
  for (pl.V = 16 / (int)es;; pl.V = 1) {
    pl.slices = 0;
    for (int s = 1; s <= groups; ++s) {
      if (groups % s || C / s > kMaxCs || C / s % pl.V) continue;
      if (pl.slices && ((C / s) * es < 64 || (long)N * s * 8 > 296)) break;
      pl.slices = s;
    }
    if (pl.slices || pl.V == 1) break;
  }
  const size_t slab = image / pl.slices;
  const long items = (long)N * pl.slices;
  pl.CS = 1;
  while (pl.CS < kMaxCluster && pl.CS < P && (slab / pl.CS > 65536 || (items * pl.CS < 296 && slab / pl.CS > 8192))) pl.CS *= 2;
  if (pl.CS > P) pl.CS = 1;
  long most = kMaxParts / (pl.CS * pl.slices);
  if (most < 1) most = 1;
  if (most > N) most = N;
  pl.clusters = (int)most * pl.slices;
  const int Cs = C / pl.slices;
  pl.smem = sizeof(float) * ((size_t)2 * pl.V * kNT + 4 * Cs + 2 * (Cs / cpg) + (bwd ? 2 * Cs : 0));
  return pl;
}

bool gn_args_ok(int dtype, int N, int P, int C, int groups) {
  return (dtype == NF_F32 || dtype == NF_BF16) && N >= 1 && P >= 1 && C >= 1 && groups >= 1 && C % groups == 0;
}

template <typename T, int V, bool BWD>
int launch_gn(const GnArgs& a, const GnPlan& pl) {
  static bool ready[64];
  int dev = 0;
  NF_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return NF_EUNSUPPORTED;
  auto k = group_norm_kernel<T, V, BWD>;
  if (!ready[dev]) {
    NF_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024));
    NF_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    ready[dev] = true;
  }
  nf_launch_cluster(k, (unsigned)(pl.clusters * pl.CS), kNT, pl.smem, pl.CS, a);
  NF_LAUNCHED();
  return NF_OK;
}

template <bool BWD>
int run_gn(int dtype, const GnArgs& a, const GnPlan& pl) {
  if (dtype == NF_F32) return pl.V == 4 ? launch_gn<float, 4, BWD>(a, pl) : launch_gn<float, 1, BWD>(a, pl);
  return pl.V == 8 ? launch_gn<bf16, 8, BWD>(a, pl) : launch_gn<bf16, 1, BWD>(a, pl);
}

void fill_gn(GnArgs& a, const GnPlan& pl, int N, int P, int C, int groups, int act) {
  a.N = N; a.P = P; a.C = C; a.G = groups; a.cpg = C / groups;
  a.slices = pl.slices; a.Cs = C / pl.slices; a.vpr = a.Cs / pl.V;
  a.CS = pl.CS; a.stride = pl.clusters / pl.slices;
  a.act = act;
}

}  // namespace

extern "C" int nf_group_norm_forward(int dtype, const void* x, const float* gamma, const float* beta, int N, int P, int C, int groups,
                                     float eps, int act, void* y, float* mean, float* rstd) {
  if (!x || !gamma || !beta || !y || !mean || !rstd || !gn_args_ok(dtype, N, P, C, groups) || !nf_act_ok(act) || !(eps > 0.f)) return NF_EINVAL;
  if (((uintptr_t)x | (uintptr_t)gamma | (uintptr_t)beta | (uintptr_t)y | (uintptr_t)mean | (uintptr_t)rstd) & 15) return NF_EALIGN;
  if (C / groups > kMaxCs) return NF_EUNSUPPORTED;
  const size_t bytes = (size_t)N * P * C * nf_esize(dtype);
  if (nf_overlap(x, bytes, y, bytes)) return NF_EINVAL;
  const GnPlan pl = plan_gn(dtype, N, P, C, groups, false);
  GnArgs a{};
  fill_gn(a, pl, N, P, C, groups, act);
  a.x = x; a.gamma = gamma; a.beta = beta; a.out = y; a.mean = mean; a.rstd = rstd; a.eps = eps;
  return run_gn<false>(dtype, a, pl);
}

extern "C" size_t nf_group_norm_scratch_bytes(int dtype, int N, int P, int C, int groups) {
  if (!gn_args_ok(dtype, N, P, C, groups) || C / groups > kMaxCs) return 0;
  const GnPlan pl = plan_gn(dtype, N, P, C, groups, true);
  return (size_t)pl.clusters / pl.slices * pl.CS * 2 * C * sizeof(float);
}

extern "C" int nf_group_norm_backward(int dtype, const void* x, const void* dy, const float* gamma, const float* beta, const float* mean,
                                      const float* rstd, int N, int P, int C, int groups, int act, void* scratch, size_t scratch_bytes,
                                      void* dx, float* dgamma, float* dbeta) {
  if (!x || !dy || !gamma || !beta || !mean || !rstd || !scratch || !dx || !dgamma || !dbeta || !gn_args_ok(dtype, N, P, C, groups) ||
      !nf_act_ok(act))
    return NF_EINVAL;
  if (((uintptr_t)x | (uintptr_t)dy | (uintptr_t)gamma | (uintptr_t)beta | (uintptr_t)mean | (uintptr_t)rstd | (uintptr_t)scratch |
       (uintptr_t)dx | (uintptr_t)dgamma | (uintptr_t)dbeta) & 15)
    return NF_EALIGN;
  if (C / groups > kMaxCs) return NF_EUNSUPPORTED;
  const size_t bytes = (size_t)N * P * C * nf_esize(dtype), need = nf_group_norm_scratch_bytes(dtype, N, P, C, groups);
  if (scratch_bytes < need) return NF_ENOWS;
  if (nf_overlap(x, bytes, dx, bytes) || nf_overlap(dy, bytes, dx, bytes)) return NF_EINVAL;
  const GnPlan pl = plan_gn(dtype, N, P, C, groups, true);
  GnArgs a{};
  fill_gn(a, pl, N, P, C, groups, act);
  a.x = x; a.dy = dy; a.gamma = gamma; a.beta = beta; a.out = dx; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.part = (float*)scratch;
  const int rc = run_gn<true>(dtype, a, pl);
  if (rc != NF_OK) return rc;
  nf_launch(group_norm_param_kernel, (unsigned)((2 * C + 31) / 32), 256, 0, (const float*)scratch, a.stride * pl.CS, C, dgamma, dbeta);
  NF_LAUNCHED();
  return NF_OK;
}
