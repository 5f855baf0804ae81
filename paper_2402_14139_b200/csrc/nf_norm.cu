// Group normalisation of channels-last maps with the activation behind it, forward and backward.
//
//   mean, var over the P pixels and C/groups channels of every (image, group);  xh = (x - mean) rstd,  z = gamma xh + beta,  y = act(z)
//   dz = dy act'(z);  dgamma = sum dz xh, dbeta = sum dz;
//   dx = rstd (gamma dz - m1 - xh m2),  m1, m2 = means over the group of gamma dz and gamma dz xh
//
// HBM has to carry every tensor once; the two passes over an image that the formulas need have to find it on the chip.  Two forms:
//  - where a pixel of the slice (some whole groups) is a power of two of 16-byte pieces: teams of a warp up to clusters of sixteen blocks hold a
//    slice, or as much of it as fits, in shared memory, and fill each place anew as soon as the second pass has read it, so that copies run under
//    both passes; the rest passes through a small ring of places, from HBM and then from L2.
//  - any other shape: a cluster of blocks reads its slice twice, the second time from L2.
// Parameter gradients gather in registers or shared memory over all images of a team or block, then in one row of partials each.
//
// What bounds it: HBM with ReLU or none (8602 maps of 4x4x512 backward 78 us, 5.5 TB/s, and 88 with the launch that joins dgamma and dbeta; 256 images of
// 112x112x64 forward 160 us, 5.1 TB/s, in groups of two channels 201), latency with SiLU or GELU, whose derivative is taken in both passes: the pieces of the
// ring go one at a time through a wait and the sigmoid's chain (128 images of 32x32x128 backward 42 us, 2.4 TB/s, with the special-function pipe 41%
// and the issue slots 43% busy), and for images of several MB the second reading: 64 of 224x224x64 forward 212 us, of which L2 gives back a quarter
// of what is read twice.
//
// Sums of the forward pass: a thread takes its values in runs of a few dozen, subtracts the mean of what it has seen before (of its first few pixels
// to begin with), and joins a run's mean and squared deviations to those of the runs before it; lanes, warps and blocks are joined in the same way.  A mean is
// held as two numbers, what was subtracted and the distance from it, until it is stored: rounded to one it would be off by 2^-24 of itself, and the
// squares of distances between such means by as much of their product.  So neither a mean far from zero nor a value that is not like the others costs
// digits: in any run the squares added are at most about as large as the deviations that come out.  The backward pass adds in fp32
// what a thread sees, then in fp32 or fp64 over threads and blocks; its ReLU mask is decided on xh gamma + beta with every operation rounded by itself.
#include <cooperative_groups.h>

#include <cuda.h>

#include "nf_act.cuh"
#include "nf_ldst.cuh"
#include "nf_ptx.cuh"
#include "nf_tc.h"

namespace {
namespace cg = cooperative_groups;

constexpr int kNT = 256;
constexpr int kMaxCs = 4096;       // channels of a slice: totals of all of them lie in shared memory
constexpr int kMaxCluster = 16;    // above 8 is outside the portable limit and has to be allowed per kernel
constexpr int kMaxBlocks = 1184;   // persistent blocks at most (rows of dgamma / dbeta partials): 8 on each of 148 SMs

struct GnArgs {
  const void *x, *dy;
  const float *gamma, *beta;
  float *mean, *rstd;  // read in the backward pass
  void* out;           // y or dx
  float* part;         // backward: [rows][2][C] partial sums of dbeta, dgamma
  int N, P, C, G, cpg;
  int slices, Cs, vpr;  // channel slices, channels and vectors per slice
  int CS, stride;       // blocks per cluster; images between two turns of a cluster or team
  int TS;               // threads of a team
  int rpc, hold, buffers;  // held form: pixels per block; pieces per thread and tensor; images in shared memory at a time
  int32_t* status;
  int act;
  float eps;
};

// V values of storage type T as loaded (16 bytes, or one value), and as pairs of floats
template <typename T, int V> struct Raw;
template <> struct Raw<bf16, 8> {
  uint4 u;
  __device__ __forceinline__ void load(const bf16* p) { u = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void load_last(const bf16* p) { u = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void load_shared(uint32_t at) { u = ptx::lds128(at); }
  __device__ __forceinline__ f32x2 pair(int i) const {
    const uint32_t w = i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w;
    return nf_pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
};
template <> struct Raw<float, 4> {
  float4 u;
  __device__ __forceinline__ void load(const float* p) { u = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void load_last(const float* p) { u = __ldcs(reinterpret_cast<const float4*>(p)); }
  __device__ __forceinline__ void load_shared(uint32_t at) {
    const uint4 w = ptx::lds128(at);
    u = make_float4(__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w));
  }
  __device__ __forceinline__ f32x2 pair(int i) const { return i == 0 ? nf_pack2(u.x, u.y) : nf_pack2(u.z, u.w); }
};
template <> struct Raw<bf16, 4> {
  uint2 u;
  __device__ __forceinline__ void load(const bf16* p) { u = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void load_last(const bf16* p) { u = __ldcs(reinterpret_cast<const uint2*>(p)); }
  __device__ __forceinline__ f32x2 pair(int i) const {
    const uint32_t w = i == 0 ? u.x : u.y;
    return nf_pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
};
template <> struct Raw<bf16, 2> {
  uint32_t u;
  __device__ __forceinline__ void load(const bf16* p) { u = *reinterpret_cast<const uint32_t*>(p); }
  __device__ __forceinline__ void load_last(const bf16* p) { u = __ldcs(reinterpret_cast<const uint32_t*>(p)); }
  __device__ __forceinline__ f32x2 pair(int) const { return nf_pack2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)); }
};
template <> struct Raw<float, 2> {
  float2 u;
  __device__ __forceinline__ void load(const float* p) { u = *reinterpret_cast<const float2*>(p); }
  __device__ __forceinline__ void load_last(const float* p) { u = __ldcs(reinterpret_cast<const float2*>(p)); }
  __device__ __forceinline__ f32x2 pair(int) const { return nf_pack2(u.x, u.y); }
};
template <typename T> struct Raw<T, 1> {
  float u;
  __device__ __forceinline__ void load(const T* p) { u = ldf(p, 0); }
  __device__ __forceinline__ void load_last(const T* p) { u = ldf(p, 0); }
  __device__ __forceinline__ f32x2 pair(int) const { return nf_pack2(u, 0.f); }
};
template <typename T, int V>
__device__ __forceinline__ void store(T* p, const f32x2 (&v)[(V + 1) / 2]) {
  float f[V + 1];
#pragma unroll
  for (int i = 0; i < (V + 1) / 2; ++i) nf_unpack2(v[i], f[2 * i], f[2 * i + 1]);
  if constexpr (V > 1 && sizeof(T) == 2) {
    uint32_t w[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    if constexpr (V == 8) __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
    else if constexpr (V == 4) __stcs(reinterpret_cast<uint2*>(p), make_uint2(w[0], w[1]));
    else __stcs(reinterpret_cast<uint32_t*>(p), w[0]);
  } else if constexpr (V == 2) {
    __stcs(reinterpret_cast<float2*>(p), make_float2(f[0], f[1]));
  } else if constexpr (V == 4) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
  } else {
    stf(p, 0, f[0]);
  }
}
__device__ __forceinline__ f32x2 both(float v) { return nf_pack2(v, v); }
// What is subtracted from values has to be finite: an infinity among them then gives the mean that it should
__device__ __forceinline__ float finite_or_0(float v) { return fabsf(v) <= 3.4028234663852886e38f ? v : 0.f; }
constexpr int kRun = 32;  // pixels of a thread between two joins of what it adds to its mean and squared deviations
__device__ __forceinline__ float low(f32x2 v) { float a, b; nf_unpack2(v, a, b); return a; }
__device__ __forceinline__ float high(f32x2 v) { float a, b; nf_unpack2(v, a, b); return b; }

// ACT: an nf_act known to the compiler, or kAnyAct: `act` says
constexpr int kAnyAct = -1;
// Two sigmoids; in bf16 storage as nf_sigmoid, its scaling and sum taken in pairs
template <typename T>
__device__ __forceinline__ f32x2 sigmoid2(f32x2 z) {
  float a, b;
  if constexpr (std::is_same<T, float>::value) {
    nf_unpack2(z, a, b);
    return nf_pack2(nf_sigmoid<T>(a), nf_sigmoid<T>(b));
  }
  nf_unpack2(nf_mul2(z, both(-1.4426950408889634f)), a, b);
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
  nf_unpack2(nf_add2(nf_pack2(a, b), both(1.f)), a, b);
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
  return nf_pack2(a, b);
}
template <typename T, int ACT>
__device__ __forceinline__ f32x2 act2(f32x2 z, int act) {
  if constexpr (ACT == NF_ACT_NONE) return z;
  if constexpr (ACT == NF_ACT_SILU) return nf_mul2(z, sigmoid2<T>(z));
  float a, b;
  nf_unpack2(z, a, b);
  return nf_pack2(nf_act_value<T>(a, ACT == kAnyAct ? act : ACT), nf_act_value<T>(b, ACT == kAnyAct ? act : ACT));
}
// dz = dy act'(z), z = xh ga + be.  ReLU: z > 0 is decided as the product, rounded by itself, being above -be; the sum of the two, rounded,
// has the sign of the exact one.
template <typename T, int ACT>
__device__ __forceinline__ f32x2 grad2(f32x2 xh, f32x2 ga, f32x2 be, f32x2 dy, int act) {
  if constexpr (ACT == NF_ACT_NONE) return dy;
  float a, b, c, d;
  if constexpr (ACT == NF_ACT_RELU) {
    float e, f;
    nf_unpack2(nf_mul2(xh, ga), a, b);
    nf_unpack2(be, e, f);
    nf_unpack2(dy, c, d);
    return nf_pack2(a > -e ? c : 0.f, b > -f ? d : 0.f);
  }
  if constexpr (ACT == NF_ACT_SILU) {  // s (1 + z (1 - s))
    const f32x2 z = nf_fma2(xh, ga, be), s = sigmoid2<T>(z);
    const f32x2 t = nf_fma2(nf_mul2(z, s), nf_fma2(s, both(-1.f), both(1.f)), s);
    return nf_mul2(t, dy);
  }
  const f32x2 z = ACT == kAnyAct ? nf_add_each(nf_mul2(xh, ga), be) : nf_fma2(xh, ga, be);
  nf_unpack2(z, a, b);
  nf_unpack2(dy, c, d);
  return nf_pack2(nf_act_dz<T>(a, c, ACT == kAnyAct ? act : ACT), nf_act_dz<T>(b, d, ACT == kAnyAct ? act : ACT));
}

// Parameters of a thread's V channels, as pairs.  ONE: they belong to one group
template <int V, bool ONE = false>
struct Chan {
  static constexpr int NP = (V + 1) / 2, NS = ONE ? 1 : NP;
  f32x2 nmu[NS], rs[NS], ga[NP], be[NP];
  __device__ __forceinline__ void affine(const GnArgs& a, int c) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int d = V == 1 ? c : c + 2 * i + 1;
      ga[i] = nf_pack2(a.gamma[c + 2 * i], a.gamma[d]);
      be[i] = nf_pack2(a.beta[c + 2 * i], a.beta[d]);
    }
  }
  template <typename F>
  __device__ __forceinline__ void stats(int c, int cpg, F&& at) {  // at(group) -> (mean, rstd)
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const float2 p = at((c + 2 * i) / cpg), q = V == 1 || ONE ? p : at((c + 2 * i + 1) / cpg);
      nmu[i] = nf_pack2(-p.x, -q.x);
      rs[i] = nf_pack2(p.y, q.y);
    }
  }
  __device__ __forceinline__ f32x2 scale(int i) const { return rs[ONE ? 0 : i]; }
  __device__ __forceinline__ f32x2 xh(f32x2 x, int i) const { return nf_mul2(nf_add2(x, nmu[ONE ? 0 : i]), rs[ONE ? 0 : i]); }
  // Forward: z from x as one sum and one multiply-add, the factor of a channel being gamma rstd
  __device__ __forceinline__ f32x2 z(f32x2 x, const f32x2 (&factor)[NP], int i) const { return nf_fma2(nf_add2(x, nmu[ONE ? 0 : i]), factor[i], be[i]); }
  __device__ __forceinline__ void factors(f32x2 (&factor)[NP]) const {
#pragma unroll
    for (int i = 0; i < NP; ++i) factor[i] = nf_mul2(ga[i], rs[ONE ? 0 : i]);
  }
};

// ---------------------------------------------------------------- large images
// V channels per thread; threads run along the channels of a pixel first, then along the pixels
template <typename T, int V, int ACT, bool BWD>
__global__ void __launch_bounds__(kNT, V == 8 ? 2 : 4) group_norm_kernel(const GnArgs a) {
  nf_pdl_begin();
  constexpr int NP = (V + 1) / 2, U = V < 8 || BWD ? 4 : 8;  // loads in flight per thread and tensor
  extern __shared__ __align__(16) float sm[];
  constexpr int kSums = BWD ? 2 : 3;
  float* red = sm;                        // [kSums V + 1][kNT] tree reduction
  // [2][kSums][Cs] this block's channel sums, two images in turn; forward: the mean's distance from what was subtracted, squared deviations, minus that
  float* tot = red + (kSums * V + 1) * kNT;
  float* gsm = tot + 2 * kSums * a.Cs;            // [2][groups of the slice]: mean and rstd (forward), m1 and m2 (backward)
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
  const bool one_col = a.vpr <= kNT;  // a thread's channels stay the same
  Chan<V> ch;
  if (one_col && on) ch.affine(a, c0 + tc * V);
  if constexpr (BWD) {
    for (int i = threadIdx.x; i < 2 * a.Cs; i += kNT) acc[i] = 0.f;
  }
  int turn = 0;
  for (int n = cid / a.slices; n < a.N; n += a.stride, turn ^= 1) {
    const size_t base = (size_t)n * a.P * a.C + c0;
    const size_t gbase = (size_t)n * a.G + slice * gps;
    float* mine = tot + turn * kSums * a.Cs;
    auto saved = [&](int g) { return make_float2(a.mean[gbase + g], a.rstd[gbase + g]); };
    for (int cv0 = 0; cv0 < a.vpr; cv0 += cols) {
      const int cv = cv0 + tc;
      f32x2 s[NP], q[NP];
      // Forward: minus what is subtracted, the distance from that of the mean of the pixels seen, and their squared deviations
      [[maybe_unused]] f32x2 nk[NP], mu[NP], m2[NP];
      [[maybe_unused]] float seen = 0.f;
#pragma unroll
      for (int i = 0; i < NP; ++i) s[i] = q[i] = nk[i] = mu[i] = m2[i] = 0;
      if (on && cv < a.vpr) {
        const size_t col = base + (size_t)cv * V;
        if constexpr (BWD) {
          if (!one_col) ch.affine(a, c0 + cv * V);
          ch.stats(cv * V, a.cpg, saved);
        }
        auto finite2 = [](f32x2 v) { return nf_pack2(finite_or_0(low(v)), finite_or_0(high(v))); };
        auto minus = [](f32x2 v) { return nf_mul2(v, both(-1.f)); };
        [[maybe_unused]] auto begin = [&](const Raw<T, V>* v, auto pixels) {  // the mean of the first pixels is subtracted from the first run
          constexpr int n = decltype(pixels)::value;
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            f32x2 m = 0;
#pragma unroll
            for (int u = 0; u < n; ++u) m = nf_fma2(v[u].pair(i), both(1.f / n), m);
            nk[i] = minus(finite2(m));
          }
        };
        // `pixels` have been added as distances from -nk, `seen` lie mu from there: S = s + seen mu of n, the mean lies S / n from there, and the squared
        // deviations grow by q + seen mu^2 - S^2 / n.  Then the mean, rounded, is what is subtracted.
        [[maybe_unused]] auto join = [&](int pixels) {
          const float n = seen + (float)pixels;
          const f32x2 w = both(1.f / n);
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            const f32x2 old = nf_mul2(both(seen), mu[i]), sum = nf_add2(s[i], old), d = nf_mul2(sum, w);
            m2[i] = nf_add2(m2[i], nf_fma2(minus(sum), d, nf_fma2(old, mu[i], q[i])));
            const f32x2 next = minus(finite2(nf_add2(d, minus(nk[i]))));
            mu[i] = nf_add2(d, nf_add2(next, minus(nk[i])));
            nk[i] = next;
            s[i] = q[i] = 0;
          }
          seen = n;
        };
        auto add = [&](const Raw<T, V>& v, const Raw<T, V>& g) {
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            if constexpr (BWD) {
              const f32x2 xh = ch.xh(v.pair(i), i);
              const f32x2 dz = grad2<T, ACT>(xh, ch.ga[i], ch.be[i], g.pair(i), a.act);
              s[i] = nf_add2(s[i], dz);
              q[i] = nf_fma2(dz, xh, q[i]);
            } else {
              const f32x2 d = nf_add2(v.pair(i), nk[i]);
              s[i] = nf_add2(s[i], d);
              q[i] = nf_fma2(d, d, q[i]);
            }
          }
        };
        int p = p0 + tr;
        [[maybe_unused]] int run = 0;
        [[maybe_unused]] bool begun = false;
        const size_t step = (size_t)R * a.C;
        size_t at = col + (size_t)p * a.C;
        for (; p + (U - 1) * R < p1; p += U * R, at += U * step) {
          Raw<T, V> v[U], g[BWD ? U : 1];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            v[u].load(x + at + u * step);
            if constexpr (BWD) g[u].load(dy + at + u * step);
          }
          if constexpr (!BWD) {
            if (!begun) begin(v, std::integral_constant<int, U>());
            begun = true;
          }
#pragma unroll
          for (int u = 0; u < U; ++u) add(v[u], g[BWD ? u : 0]);
          if constexpr (!BWD) {
            if ((run += U) == kRun) {
              join(run);
              run = 0;
            }
          }
        }
        for (; p < p1; p += R, at += step) {
          Raw<T, V> v, g;
          v.load(x + at);
          if constexpr (BWD) g.load(dy + at);
          else g = v;
          if constexpr (!BWD) {
            if (!begun) begin(&v, std::integral_constant<int, 1>());
            begun = true;
            ++run;
          }
          add(v, g);
        }
        if constexpr (!BWD) {
          if (run) join(run);
        }
      }
      // rows of threads are folded in halves
      __syncthreads();
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const f32x2 first = BWD ? s[i / 2] : mu[i / 2], second = BWD ? q[i / 2] : m2[i / 2];
        red[i * kNT + threadIdx.x] = i % 2 ? high(first) : low(first);
        red[(V + i) * kNT + threadIdx.x] = i % 2 ? high(second) : low(second);
      }
      if constexpr (!BWD) {
        red[3 * V * kNT + threadIdx.x] = seen;
#pragma unroll
        for (int i = 0; i < V; ++i) red[(2 * V + i) * kNT + threadIdx.x] = i % 2 ? high(nk[i / 2]) : low(nk[i / 2]);
      }
      for (int left = R; left > 1;) {
        const int half = (left + 1) / 2;
        __syncthreads();
        if (tr + half < left) {
          float* mine_at = red + threadIdx.x;
          const float* other = mine_at + half * cols;
          if constexpr (BWD) {
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) mine_at[e * kNT] += other[e * kNT];
          } else {  // (count, what was subtracted, distance of the mean, squared deviations) of both; rows further on never have more pixels
            const float na = mine_at[3 * V * kNT], nb = other[3 * V * kNT];
            if (nb > 0.f) {
              const float w = __fdividef(nb, na + nb);  // two units in the last place are enough for a weight
#pragma unroll
              for (int e = 0; e < V; ++e) {
                const float ma = mine_at[e * kNT], base_m = finite_or_0(ma);
                const float mb = (mine_at[(2 * V + e) * kNT] - other[(2 * V + e) * kNT]) + other[e * kNT], d = mb - ma;
                mine_at[e * kNT] = base_m + fmaf(mb - base_m, w, (ma - base_m) * (1.f - w));
                mine_at[(V + e) * kNT] += other[(V + e) * kNT] + d * d * (na * w);
              }
              mine_at[3 * V * kNT] = na + nb;
            }
          }
        }
        left = half;
      }
      __syncthreads();
      const int width = (a.vpr - cv0 < cols ? a.vpr - cv0 : cols) * V;  // channels of this chunk
      for (int i = threadIdx.x; i < kSums * width; i += kNT) {
        const int w = i / width, c = i - w * width;
        mine[w * a.Cs + cv0 * V + c] = red[(w * V + c % V) * kNT + c / V];
      }
    }
    cluster.sync();
    // every block joins the ranks' sums and the channels of each group: L lanes per group
    {
      int L = 1;
      while (L < a.cpg && L < 32) L *= 2;
      [[maybe_unused]] const int cs_log = 31 - __clz(a.CS);
      const int lane = threadIdx.x % L, per = kNT / L;
      for (int g0 = 0; g0 < gps; g0 += per) {
        const int g = g0 + threadIdx.x / L;
        double A = 0, B = 0, from = 0;  // forward: moments about what the first block subtracted from the group's first channel
        if (g < gps) {
          if constexpr (!BWD) from = -cluster.map_shared_rank(mine, 0)[2 * a.Cs + g * a.cpg];
          for (int i = lane; i < a.cpg; i += L) {
            const int c = g * a.cpg + i;
            double S = 0, Q = 0;
#pragma unroll 4
            for (int r = 0; r < a.CS; ++r) {
              const float* o = cluster.map_shared_rank(mine, r);
              if constexpr (BWD) {
                S += o[c];
                Q += o[a.Cs + c];
              } else {  // CS is a power of two
                const double n = (double)(int)(((long long)a.P * (r + 1) >> cs_log) - ((long long)a.P * r >> cs_log)), d = o[c] - ((double)o[2 * a.Cs + c] + from);
                S += n * d;
                Q += o[a.Cs + c] + n * d * d;
              }
            }
            if constexpr (!BWD) {
              A += S / a.P;
              B += Q / a.P;
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
            const float mf = (float)(from + m), rf = (float)(1.0 / sqrt((var > 0 ? var : var == var ? 0 : var) + (double)a.eps));
            gsm[g] = mf;
            gsm[gps + g] = rf;
            if (rank == 0) {
              a.mean[gbase + g] = mf;
              a.rstd[gbase + g] = rf;
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
      f32x2 m1[NP], m2[NP];
      if (!one_col) ch.affine(a, c0 + cv * V);
      if constexpr (!BWD) {
        ch.stats(cv * V, a.cpg, [&](int g) { return make_float2(gsm[g], gsm[gps + g]); });
      } else {
        if (!one_col) ch.stats(cv * V, a.cpg, saved);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int g = (cv * V + 2 * i) / a.cpg, h = V == 1 ? g : (cv * V + 2 * i + 1) / a.cpg;
          m1[i] = nf_pack2(-gsm[g], -gsm[h]);
          m2[i] = nf_pack2(-gsm[gps + g], -gsm[gps + h]);
        }
      }
      f32x2 factor[NP];
      if constexpr (!BWD) ch.factors(factor);
      auto result = [&](const Raw<T, V>& v, const Raw<T, V>& g, T* to) {
        f32x2 o[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          if constexpr (BWD) {
            const f32x2 xh = ch.xh(v.pair(i), i);
            const f32x2 dz = grad2<T, ACT>(xh, ch.ga[i], ch.be[i], g.pair(i), a.act);
            o[i] = nf_mul2(ch.scale(i), nf_fma2(xh, m2[i], nf_fma2(ch.ga[i], dz, m1[i])));
          } else {
            o[i] = act2<T, ACT>(ch.z(v.pair(i), factor, i), a.act);
          }
        }
        store<T, V>(to, o);
      };
      constexpr int W = V < 8 || BWD ? 4 : 8;
      int p = p0 + tr;
      const size_t step = (size_t)R * a.C;
      size_t at = col + (size_t)p * a.C;
      for (; p + (W - 1) * R < p1; p += W * R, at += W * step) {
        Raw<T, V> v[W], g[BWD ? W : 1];
#pragma unroll
        for (int u = 0; u < W; ++u) {
          v[u].load_last(x + at + u * step);
          if constexpr (BWD) g[u].load_last(dy + at + u * step);
        }
#pragma unroll
        for (int u = 0; u < W; ++u) result(v[u], g[BWD ? u : 0], out + at + u * step);
      }
      for (; p < p1; p += R, at += step) {
        Raw<T, V> v, g;
        v.load_last(x + at);
        if constexpr (BWD) g.load_last(dy + at);
        else g = v;
        result(v, g, out + at);
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

// ---------------------------------------------------------------- slices held in shared memory
// A team of TS threads works on one image's slice (in a cluster: each block's team on a range of its pixels).  A slice is `vpr` 16-byte pieces
// of a pixel, a power of two up to 32, whole groups; a thread takes pieces t, t + TS, ..., so its channels stay the same, and it alone
// copies them into shared memory (cp.async), reads them in both passes and refills their places with the image `buffers` turns on: no
// barrier guards the data.  Sums of a group (forward: means and squared deviations): shuffles; teams of several warps join one pair per warp and group
// through shared memory; blocks of a cluster send theirs to each other (st.async into slots of the receiver, counted by its barrier).  FINE: groups
// of fewer channels than a piece; MORE: the slice is larger than what is held.
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait(int behind) {  // all but the latest `behind` groups have landed
  if (behind <= 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
  else if (behind == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else if (behind == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

// Places per thread and tensor that the rest of a large image passes through: 32 KB on their way in a block, two blocks on an SM.  64 images of
// 224x224x64 forward: 4 places 7% slower, 6 and more the same.
__host__ __device__ constexpr int held_ring(bool bwd) { return bwd ? 4 : 8; }

template <typename T, int V, int ACT, bool BWD, bool FINE, bool MORE>
__global__ void __launch_bounds__(kNT, 2) group_norm_held_kernel(const GnArgs a) {
  constexpr int NT = kNT, NP = V / 2, S = FINE ? V : 1, kTensors = BWD ? 2 : 1, kRing = held_ring(BWD);
  extern __shared__ __align__(16) uint8_t held_raw[];
  __shared__ float part[NT / 32][BWD ? 2 : 3][32];      // per warp: totals of the groups
  __shared__ float2 gsm[NT / 32 * 32];                  // per team: mean and rstd, or m1 and m2
  __shared__ float2 peers[2][kMaxCluster][32];          // the blocks' totals, two items in turn
  __shared__ float peers_rest[BWD ? 1 : 2][kMaxCluster][32];  // forward: of their means, what rounding left
  __shared__ uint64_t xbar[2];
  __shared__ int abort_word;
  const int TS = a.TS, team = threadIdx.x / TS, t = threadIdx.x % TS, lane = threadIdx.x & 31, warps = TS / 32;
  const int rank = blockIdx.x % a.CS, id = blockIdx.x / a.CS * (NT / TS) + team, slice = id % a.slices;
  const int tc = t % a.vpr, tr = t / a.vpr, rows = TS / a.vpr;
  const int gps = a.Cs / a.cpg, c0 = slice * a.Cs;
  const int lo = a.cpg > V ? a.cpg / V : 1;
  const int p0 = rank * a.rpc, np = max(0, min(a.P - p0, a.rpc));
  // Turns over the slice: `whole` of them with a piece for every thread, then one where some have none.  The first a.hold are held; the rest of
  // a very large image (MORE), ks pieces of this thread, passes through a ring of kRing places twice, the second time from L2.
  const int whole = np * a.vpr / TS, kw = min(whole, a.hold);
  const bool last = t < np * a.vpr - whole * TS, last_held = last && whole < a.hold;
  const int ks = MORE ? whole - kw + (last && !last_held) : 0;
  if (a.CS > 1) {
    if (threadIdx.x == 0) {
      ptx::mbar_init(&xbar[0], 1);
      ptx::mbar_init(&xbar[1], 1);
      abort_word = 0;
      ptx::fence_mbar_init();
    }
    __syncthreads();
    ptx::cluster_sync();
  }
  nf_pdl_begin();

  const T* x = (const T*)a.x + (size_t)p0 * a.C + c0 + tc * V;
  const T* dy = (const T*)a.dy + (size_t)p0 * a.C + c0 + tc * V;
  T* out = (T*)a.out + (size_t)p0 * a.C + c0 + tc * V;
  const size_t image = (size_t)a.P * a.C, row_step = (size_t)rows * a.C;
  constexpr uint32_t kstep = NT * 16;
  const uint32_t slot0 = ptx::smem_u32(held_raw) + threadIdx.x * 16, tstep = a.hold * kstep, bstep = kTensors * tstep;
  const int first = id / a.slices;
  for (int i = 0; i < a.buffers; ++i) {
    const int n = first + i * a.stride;
    if (n < a.N) {
      size_t at = (size_t)n * image + (size_t)tr * a.C;
      uint32_t slot = slot0 + i * bstep;
      for (int k = 0; k < kw + last_held; ++k, at += row_step, slot += kstep) {
        copy16(slot, x + at);
        if constexpr (BWD) copy16(slot + tstep, dy + at);
      }
    }
    copies_end();
  }
  // The ring's loads run kRing pieces ahead of their use, through both passes and from one image to the next: (image, pass, pieces left, where).  The
  // second pass goes backwards, from what L2 has had last.
  const uint32_t ring0 = slot0 + kTensors * a.hold * kstep;
  const size_t ring_at = (size_t)tr * a.C + a.hold * row_step;
  int ring_n = first, ring_left = ks;
  bool ring_second = false;
  uint32_t ring_slot = 0;  // place of the next piece to be used
  const T* ring_x = x + (size_t)first * image + ring_at;
  const T* ring_dy = BWD ? dy + (size_t)first * image + ring_at : nullptr;
  const ptrdiff_t forth = (ptrdiff_t)row_step;
  const size_t ring_end = ks ? (ks - 1) * row_step : 0;  // its last piece, from its first
  auto ring_fill = [&](uint32_t place) {
    if (ring_n < a.N && ks) {
      copy16(ring0 + place * kstep, ring_x);
      ring_x += ring_second ? -forth : forth;
      if constexpr (BWD) {
        copy16(ring0 + (kRing + place) * kstep, ring_dy);
        ring_dy += ring_second ? -forth : forth;
      }
      if (--ring_left == 0) {
        ring_left = ks;
        if (ring_second) ring_n += a.stride;
        ring_second = !ring_second;
        const size_t at = (size_t)ring_n * image + ring_at + (ring_second ? ring_end : 0);
        ring_x = x + at;
        if constexpr (BWD) ring_dy = dy + at;
      }
    }
    copies_end();
  };
  // f(x, dy) for each of this pass's pieces, way from one to the next; join(): kRun pieces have been used, in the first of those runs `before` fewer
  auto ring_use = [&](auto&& f, ptrdiff_t way, int before, auto&& join) {
    auto step = [&](auto&& fill) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
      Raw<T, V> v, g;
      v.load_shared(ring0 + ring_slot * kstep);
      if constexpr (BWD) g.load_shared(ring0 + (kRing + ring_slot) * kstep);
      else g = v;
      f(v, g);
      fill();  // the piece has been read: what became of it depends on it
      ring_slot = (ring_slot + 1) % kRing;
    };
    auto along = [&] {  // within a pass the loads move on by rows
      copy16(ring0 + ring_slot * kstep, ring_x);
      ring_x += way;
      if constexpr (BWD) {
        copy16(ring0 + (kRing + ring_slot) * kstep, ring_dy);
        ring_dy += way;
      }
      copies_end();
    };
    const int same = ks - kRing;  // steps whose loads belong to this pass as well; the last of them is the pass's last load
    int k = 0;
    if (same > 1 && ring_n < a.N) {
      if constexpr (!std::is_same<std::decay_t<decltype(join)>, std::nullptr_t>::value) {
        for (int end = kRun - before; end <= same - 1; end += kRun) {
#pragma unroll 4
          for (; k < end; ++k) step(along);
          join();
        }
      }
#pragma unroll 4
      for (; k < same - 1; ++k) step(along);
      ring_left -= same - 1;
    }
    for (; k < ks; ++k) step([&] { ring_fill(ring_slot); });
  };
  if (MORE && ks) {
    for (uint32_t i = 0; i < kRing; ++i) ring_fill(i);
  }
  Chan<V, !FINE> ch;
  constexpr int NS = FINE ? NP : 1;
  ch.affine(a, c0 + tc * V);
  f32x2 db[NP], dg[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) db[i] = dg[i] = 0;

  // Backward: the statistics of this thread's group are read one image ahead
  [[maybe_unused]] float2 ahead = make_float2(0.f, 0.f);
  auto look = [&](int n) {
    if (!BWD || FINE || n >= a.N) return;
    const size_t g = (size_t)n * a.G + slice * gps + tc / lo;
    ahead = make_float2(a.mean[g], a.rstd[g]);
  };
  // Forward: pixels that this thread sees, values that it and the warps of its team see of a group; runs count in `unit`s
  const int own_px = whole + last, rest = np * a.vpr - whole * TS, pivots = min(kw + last_held, 4), from_lane = lane & (a.vpr - 1) & ~(lo - 1);
  auto warp_values = [&](int w) { return (float)((32 * whole + min(max(rest - 32 * w, 0), 32)) / a.vpr * a.cpg); };
  constexpr float unit = FINE ? 1.f : V;
  const float own_n = (float)(own_px * (FINE ? a.cpg : V)), own_w = own_px ? 1.f / (own_px * unit) : 0.f;
  const float warp_n = warp_values(t / 32), warp_w = warp_n > 0.f ? 1.f / warp_n : 0.f, pivot_w = pivots ? 1.f / (pivots * unit) : 0.f;
  look(first);
  int b = 0, turn = 0;
  uint32_t xph = 0;
  for (int n = first; n < a.N; n += a.stride) {
    const size_t gbase = (size_t)n * a.G + slice * gps;
    const uint32_t slot = slot0 + b * bstep;
    if constexpr (BWD) {
      if constexpr (FINE) ch.stats(tc * V, a.cpg, [&](int i) { return make_float2(a.mean[gbase + i], a.rstd[gbase + i]); });
      else ch.stats(0, 1, [&](int) { return ahead; });
    }
    look(n + a.stride);
    f32x2 s[NP], q[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) s[i] = q[i] = 0;
    // A thread's pairs added over the channels of each slot's group
    auto slots = [&](const f32x2 (&from)[NP], float (&to)[S]) {
      float v[V];
#pragma unroll
      for (int i = 0; i < NP; ++i) nf_unpack2(from[i], v[2 * i], v[2 * i + 1]);
      if constexpr (FINE) {
#pragma unroll
        for (int i = 0; i < V; ++i) to[i] = v[i];
        // channels of a group lie next to each other in the thread
        if (a.cpg >= 2) {
#pragma unroll
          for (int i = 0; i < S; i += 2) to[i] = to[i + 1 < S ? i + 1 : i] = to[i] + to[i + 1 < S ? i + 1 : i];
        }
        if (S == 8 && a.cpg >= 4) {
#pragma unroll
          for (int i = 0; i + 2 < S; i += 4) to[i] = to[i + 1] = to[i + 2] = to[i + 3] = to[i] + to[i + 2];
        }
      } else {
        to[0] = v[0];
#pragma unroll
        for (int i = 1; i < V; ++i) to[0] += v[i];
      }
    };
    // Forward: minus what is subtracted (of the group, or FINE of each channel), the distance from that of the mean of what this thread has seen, and its
    // squared deviations; seen: how much that is
    [[maybe_unused]] f32x2 nk[NS] = {}, mu2[NP], sq2[NP];
    [[maybe_unused]] float mu = 0.f, sq = 0.f, seen = 0.f;
    auto finite2 = [](f32x2 v) { return nf_pack2(finite_or_0(low(v)), finite_or_0(high(v))); };
    // Values have been added as distances from -nk: S = s + seen mu of n = 1 / w, the mean lies S / n from there, the squared deviations grow by
    // q + seen mu^2 - S^2 / n.  Then the mean, rounded, is what is subtracted.
    auto join_run = [&](float w) {
      if constexpr (FINE) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const f32x2 old = nf_mul2(both(seen), mu2[i]), sum = nf_add2(s[i], old), d = nf_mul2(sum, both(w));
          sq2[i] = nf_add2(sq2[i], nf_fma2(nf_mul2(sum, both(-1.f)), d, nf_fma2(old, mu2[i], q[i])));
          const f32x2 minus = both(-1.f), next = nf_mul2(finite2(nf_fma2(nk[i], minus, d)), minus);
          mu2[i] = nf_add2(d, nf_fma2(nk[i], minus, next));
          nk[i] = next;
        }
      } else {
        float f0[S], f1[S];
        slots(s, f0);
        slots(q, f1);
        const float old = seen * mu, sum = f0[0] + old, d = sum * w;
        sq += fmaf(-sum, d, fmaf(old, mu, f1[0]));
        const float before = -low(nk[0]), next = finite_or_0(before + d);
        mu = d - (next - before);
        nk[0] = both(-next);
      }
#pragma unroll
      for (int i = 0; i < NP; ++i) s[i] = q[i] = 0;
    };
    auto add = [&](const Raw<T, V>& v, const Raw<T, V>& g) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        if constexpr (BWD) {
          const f32x2 xh = ch.xh(v.pair(i), i);
          const f32x2 dz = grad2<T, ACT>(xh, ch.ga[i], ch.be[i], g.pair(i), a.act);
          s[i] = nf_add2(s[i], dz);
          q[i] = nf_fma2(dz, xh, q[i]);
        } else {
          const f32x2 d = nf_add2(v.pair(i), nk[FINE ? i : 0]);
          s[i] = nf_add2(s[i], d);
          q[i] = nf_fma2(d, d, q[i]);
        }
      }
    };
    const size_t own_at = (size_t)n * image + (size_t)tr * a.C;  // this thread's first piece
    if constexpr (MORE) {  // what is held was asked for before the latest kRing pieces of the ring, unless the image hardly needs it
      if (ks >= kRing) asm volatile("cp.async.wait_group %0;" ::"n"(kRing) : "memory");
      else copies_wait(ks ? 0 : a.buffers - 1);
    } else {
      copies_wait(a.buffers - 1);
    }
    {
      auto one = [&](uint32_t at) {
        Raw<T, V> v, g;
        v.load_shared(at);
        if constexpr (BWD) g.load_shared(at + tstep);
        else g = v;
        add(v, g);
      };
      uint32_t at = slot;
      int k = kw;
      if constexpr (!BWD) {  // what is subtracted to begin with: the mean of the first four pieces
        f32x2 sum[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) sum[i] = mu2[i] = sq2[i] = 0;
        auto more = [&](const Raw<T, V>& v) {
#pragma unroll
          for (int i = 0; i < NP; ++i) sum[i] = nf_fma2(v.pair(i), both(pivot_w), sum[i]);
        };
        auto begin = [&] {
          if constexpr (!FINE) {
            float m[S];
            slots(sum, m);
            nk[0] = both(-finite_or_0(m[0]));
          } else {
#pragma unroll
            for (int i = 0; i < NP; ++i) nk[i] = nf_mul2(finite2(sum[i]), both(-1.f));
          }
        };
        if (kw >= 4) {
          Raw<T, V> v[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) v[u].load_shared(slot + u * kstep);
#pragma unroll
          for (int u = 0; u < 4; ++u) more(v[u]);
          begin();
#pragma unroll
          for (int u = 0; u < 4; ++u) add(v[u], v[u]);
          at += 4 * kstep;
          k -= 4;
        } else {
          for (int u = 0; u < pivots; ++u) {
            Raw<T, V> v;
            v.load_shared(slot + u * kstep);
            more(v);
          }
          begin();
        }
      }
      for (; k >= 4; k -= 4, at += 4 * kstep) {
#pragma unroll
        for (int u = 0; u < 4; ++u) one(at + u * kstep);
      }
      for (k += last_held; k > 0; --k, at += kstep) one(at);
    }
    if constexpr (!BWD) {
      if constexpr (MORE) {
        ring_use(add, forth, kw, [&] {
          join_run(1.f / (seen + kRun * unit));
          seen += kRun * unit;
        });
      }
      join_run(own_w);
    } else if constexpr (MORE) {
      ring_use(add, forth, 0, nullptr);
    }
    if constexpr (BWD) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        db[i] = nf_add2(db[i], s[i]);
        dg[i] = nf_add2(dg[i], q[i]);
        s[i] = nf_mul2(s[i], ch.ga[i]);
        q[i] = nf_mul2(q[i], ch.ga[i]);
      }
    }
    // Over the lanes that share the group, all values side by side: shuffles stay in order, and each waits for the one before it of its own value only.
    // Forward, FINE: a group's first channel stands for it
    auto over_lanes = [&](auto& v) {
      constexpr int n = sizeof(v) / sizeof(float);
      float* w = reinterpret_cast<float*>(&v);
#pragma unroll
      for (int o = 1; o < 32; o *= 2)
        if (o < lo || o >= a.vpr) {
#pragma unroll
          for (int i = 0; i < n; ++i)
            if (BWD || !FINE || !(i & (a.cpg - 1))) w[i] += __shfl_xor_sync(0xffffffffu, w[i], o);
        }
    };
    float f[2][S];  // backward: sums; forward: distance of the mean from `origin`, squared deviations
    [[maybe_unused]] float origin[S];
    if constexpr (BWD) {
      slots(s, f[0]);
      slots(q, f[1]);
      over_lanes(f);
    } else {  // the origin: what the first lane of the group subtracted; no lane has more pixels
#pragma unroll
      for (int i = 0; i < S; ++i)
        if (!FINE || !(i & (a.cpg - 1))) origin[i] = -__shfl_sync(0xffffffffu, i % 2 ? high(nk[i / 2]) : low(nk[i / 2]), from_lane);
      auto spread = [&](float (&v)[S]) {  // from a group's first channel
        if constexpr (FINE) {
#pragma unroll
          for (int i = 1; i < S; ++i) {
            if (i % 2 && a.cpg >= 2) v[i] = v[i - 1];
            if (i % 4 == 2 && a.cpg >= 4) v[i] = v[i - 2];
          }
        }
      };
      spread(origin);
      if constexpr (FINE) {  // channels of a group: as many pixels of each
        f32x2 v[NP];
        const f32x2 w = both(1.f / a.cpg), px = both((float)own_px);
#pragma unroll
        for (int i = 0; i < NP; ++i) {  // from the origin on
          const f32x2 from = nf_add2(nk[i], nf_pack2(origin[2 * i], origin[S > 1 ? 2 * i + 1 : 0]));
          mu2[i] = nf_fma2(from, both(-1.f), mu2[i]);
          v[i] = nf_mul2(mu2[i], w);
        }
        slots(v, f[0]);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const f32x2 d = nf_add2(mu2[i], nf_pack2(-f[0][2 * i], -f[0][S > 1 ? 2 * i + 1 : 0]));
          v[i] = nf_fma2(nf_mul2(d, px), d, sq2[i]);
        }
        slots(v, f[1]);
      } else {
        f[0][0] = mu - (low(nk[0]) + origin[0]);
        f[1][0] = sq;
      }
      float m[S];
#pragma unroll
      for (int i = 0; i < S; ++i) m[i] = own_px ? own_n * f[0][i] : 0.f;
      over_lanes(m);
#pragma unroll
      for (int i = 0; i < S; ++i) {
        m[i] *= warp_w;
        const float d = f[0][i] - m[i];
        f[0][i] = m[i];
        f[1][i] = own_px ? fmaf(own_n * d, d, f[1][i]) : 0.f;
      }
      over_lanes(f[1]);
#pragma unroll
      for (int i = 0; i < S; ++i) f[1][i] = f[1][i] < 0.f ? 0.f : f[1][i];  // a NaN stays one
      spread(f[0]);
      spread(f[1]);
    }
    const float M = (float)a.P * a.cpg;
    float2 mine[S];
    if (warps == 1) {
#pragma unroll
      for (int i = 0; i < S; ++i) {
        if constexpr (BWD) {
          mine[i] = make_float2(-f[0][i] / M, -f[1][i] / M);
        } else {
          mine[i] = make_float2(origin[i] + f[0][i], 1.f / sqrtf(f[1][i] / M + a.eps));
        }
      }
      if (!BWD && tr == 0 && tc % lo == 0) {
#pragma unroll
        for (int i = 0; i < S; ++i)
          if (!FINE || i % a.cpg == 0) {
            const int g = (tc * V + i) / a.cpg;
            a.mean[gbase + g] = mine[i].x;
            a.rstd[gbase + g] = mine[i].y;
          }
      }
    } else {
      if (lane < a.vpr && lane % lo == 0) {
#pragma unroll
        for (int i = 0; i < S; ++i)
          if (!FINE || i % a.cpg == 0) {
            const int g = (tc * V + i) / a.cpg;
            part[threadIdx.x / 32][0][g] = f[0][i];
            part[threadIdx.x / 32][1][g] = f[1][i];
            if constexpr (!BWD) part[threadIdx.x / 32][2][g] = origin[i];
          }
      }
      ptx::named_barrier(1 + team, TS);
      float2* own = gsm + team * warps * 32;  // up to 32 groups per warp of the team
      // a warp per group: its lanes join the warps' sums (A in the lower half, B in the upper), then the other blocks'
      for (int g = t / 32; g < gps; g += warps) {
        float A, B;
        [[maybe_unused]] float rest_of_mean = 0.f;
        if constexpr (BWD) {
          const int w = lane & 15;
          float v = w < warps ? part[team * warps + w][lane >> 4][g] : 0.f;
#pragma unroll
          for (int o = 1; o < 16; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
          A = __shfl_sync(0xffffffffu, v, 0);
          B = __shfl_sync(0xffffffffu, v, 16);
        } else {
          const float wn = lane < warps ? warp_values(lane) : 0.f, wo = wn > 0.f ? part[team * warps + lane][2][g] : 0.f;
          const float from = __shfl_sync(0xffffffffu, wo, 0);  // no warp has more pixels than the first
          const float wm = wn > 0.f ? (wo - from) + part[team * warps + lane][0][g] : 0.f;
          A = wn * wm;
#pragma unroll
          for (int o = 1; o < NT / 32; o *= 2) A += __shfl_xor_sync(0xffffffffu, A, o);
          A = __shfl_sync(0xffffffffu, A, 0);
          if (np) A /= (float)np * a.cpg;
          B = wn > 0.f ? fmaf(wn * (wm - A), wm - A, part[team * warps + lane][1][g]) : 0.f;
#pragma unroll
          for (int o = 1; o < NT / 32; o *= 2) B += __shfl_xor_sync(0xffffffffu, B, o);
          B = __shfl_sync(0xffffffffu, B, 0);
          const float sum = from + finite_or_0(A);
          rest_of_mean = A - (sum - from);
          A = sum;
        }
        if (a.CS > 1) {
          if (t == 0 && g == 0) ptx::mbar_expect_tx(&xbar[turn], a.CS * gps * (BWD ? 8 : 12));  // once: the barrier counts one arrival
          if (lane < a.CS) {
            ptx::st_async_f2(&peers[turn][rank][g], A, B, &xbar[turn], lane);
            if constexpr (!BWD) ptx::st_async_f1(&peers_rest[turn][rank][g], rest_of_mean, &xbar[turn], lane);
          }
        } else if (!BWD) {
          A += rest_of_mean;
        }
        if (lane == 0) own[g] = make_float2(A, B);
      }
      __syncwarp();
      for (int g = t / 32; g < gps; g += warps) {
        float A = own[g].x, B = own[g].y;
        if (a.CS > 1) {
          if (g == t / 32) ptx::mbar_wait(&xbar[turn], (xph >> turn) & 1, &abort_word);  // sets the abort word itself when it gives up
          const float2 from = lane < a.CS ? peers[turn][lane][g] : make_float2(0.f, 0.f);
          const float cr = lane < a.CS ? (float)max(0, min(a.P - lane * a.rpc, a.rpc)) : 0.f;
          const float base = __shfl_sync(0xffffffffu, from.x, 0);  // forward, block 0's mean, rounded, which is finite: means are joined by their distances from it
          float d = from.x;
          if constexpr (!BWD) d = cr > 0.f ? (from.x - base) + peers_rest[turn][lane & (kMaxCluster - 1)][g] : 0.f;
          float m = BWD ? d : cr * d, M2 = from.y;
#pragma unroll
          for (int o = 1; o < kMaxCluster; o *= 2) m += __shfl_xor_sync(0xffffffffu, m, o);
          if constexpr (!BWD) {
            m /= (float)a.P;
            M2 += cr * (float)a.cpg * (d - m) * (d - m);
          }
#pragma unroll
          for (int o = 1; o < kMaxCluster; o *= 2) M2 += __shfl_xor_sync(0xffffffffu, M2, o);
          A = BWD ? m : base + m;
          B = M2;
        }
        if (lane == 0) {
          if constexpr (BWD) {
            own[g] = make_float2(-A / M, -B / M);
          } else {
            const float rf = 1.f / sqrtf(B / M + a.eps);
            own[g] = make_float2(A, rf);
            if (rank == 0) {
              a.mean[gbase + g] = A;
              a.rstd[gbase + g] = rf;
            }
          }
        }
      }
      ptx::named_barrier(1 + team, TS);
#pragma unroll
      for (int i = 0; i < S; ++i) mine[i] = own[FINE ? (tc * V + i) / a.cpg : tc / lo];
    }
    if (a.CS > 1) xph ^= 1u << turn;
    f32x2 m1[BWD ? NS : 1], m2[BWD ? NS : 1];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const float2 g = mine[FINE ? 2 * i : 0], h = mine[FINE ? 2 * i + 1 : 0];
      if constexpr (BWD) {
        m1[i] = nf_pack2(g.x, h.x);
        m2[i] = nf_pack2(g.y, h.y);
      } else {
        ch.nmu[i] = nf_pack2(-g.x, -h.x);
        ch.rs[i] = nf_pack2(g.y, h.y);
      }
    }
    f32x2 factor[NP];
    if constexpr (!BWD) ch.factors(factor);
    auto result = [&](const Raw<T, V>& v, const Raw<T, V>& g, T* to) {
      f32x2 o[NP];
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        if constexpr (BWD) {
          const f32x2 xh = ch.xh(v.pair(i), i);
          const f32x2 dz = grad2<T, ACT>(xh, ch.ga[i], ch.be[i], g.pair(i), a.act);
          o[i] = nf_mul2(ch.scale(i), nf_fma2(xh, m2[FINE ? i : 0], nf_fma2(ch.ga[i], dz, m1[FINE ? i : 0])));
        } else {
          o[i] = act2<T, ACT>(ch.z(v.pair(i), factor, i), a.act);
        }
      }
      store<T, V>(to, o);
    };
    // Pass two; a place that has been read (the stored value depends on it) is filled with the image `buffers` turns on
    auto held = [&](auto refill) {
      constexpr bool kRefill = decltype(refill)::value;
      T* to = out + own_at;
      const size_t ahead_by = (size_t)a.buffers * a.stride * image;
      const T* nx = x + own_at + ahead_by;
      [[maybe_unused]] const T* nd = dy + own_at + ahead_by;
      auto one = [&](uint32_t at) {
        Raw<T, V> v, g;
        v.load_shared(at);
        if constexpr (BWD) g.load_shared(at + tstep);
        else g = v;
        result(v, g, to);
        to += row_step;
        if constexpr (kRefill) {
          copy16(at, nx);
          nx += row_step;
          if constexpr (BWD) {
            copy16(at + tstep, nd);
            nd += row_step;
          }
        }
      };
      uint32_t at = slot;
      int k = kw;
      for (; k >= 4; k -= 4, at += 4 * kstep) {
#pragma unroll
        for (int u = 0; u < 4; ++u) one(at + u * kstep);
      }
      for (k += last_held; k > 0; --k, at += kstep) one(at);
    };
    if (n + a.buffers * a.stride < a.N) held(std::true_type());
    else held(std::false_type());
    copies_end();
    if constexpr (MORE) {
      T* to = out + own_at + a.hold * row_step + ring_end;
      ring_use([&](const Raw<T, V>& v, const Raw<T, V>& g) {
        result(v, g, to);
        to -= row_step;
      }, -forth, 0, nullptr);
    }
    if (++b == a.buffers) b = 0;
    turn ^= 1;
  }
  copies_wait(0);
  if constexpr (BWD) {  // the team's rows of threads folded in halves; a row of partials per team and rank
    float* sm = reinterpret_cast<float*>(held_raw);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sm[i * NT + threadIdx.x] = i % 2 ? high(db[i / 2]) : low(db[i / 2]);
      sm[(V + i) * NT + threadIdx.x] = i % 2 ? high(dg[i / 2]) : low(dg[i / 2]);
    }
    for (int left = TS / 2; left >= a.vpr; left /= 2) {
      __syncthreads();
      if (t < left) {
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) sm[e * NT + threadIdx.x] += sm[e * NT + threadIdx.x + left];
      }
    }
    __syncthreads();
    float* row = a.part + (size_t)(id / a.slices * a.CS + rank) * 2 * a.C + c0;
    for (int i = t; i < 2 * a.Cs; i += TS) {
      const int w = i / a.Cs, c = i - w * a.Cs;
      row[(size_t)w * a.C + c] = sm[(w * V + c % V) * NT + team * TS + c / V];
    }
  }
  if (a.CS > 1) {
    __syncthreads();
    if (threadIdx.x == 0 && abort_word) atomicOr(a.status, NF_ETIMEOUT);
    __syncwarp();
    ptx::cluster_sync();  // no block leaves while another may still send it sums
  }
}

// dbeta, dgamma: the rows of partials added in fp64, 32 chains of every 32nd row, joined in order
__global__ void __launch_bounds__(1024) group_norm_param_kernel(const float* __restrict__ part, int rows, int C, float* __restrict__ dgamma,
                                                                float* __restrict__ dbeta) {
  nf_pdl_begin();
  __shared__ double sm[32][33];
  const int tx = threadIdx.x % 32, ty = threadIdx.x / 32;
  const int i = blockIdx.x * 32 + tx;
  double s = 0;
  if (i < 2 * C) {
#pragma unroll 4
    for (int r = ty; r < rows; r += 32) s += part[(size_t)r * 2 * C + i];
  }
  sm[ty][tx] = s;
  __syncthreads();
  // a warp per column: lane k joins chain k
  double v = sm[tx][ty];
  for (int o = 1; o < 32; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
  const int j = blockIdx.x * 32 + ty;
  if (tx == 0 && j < 2 * C) (j < C ? dbeta[j] : dgamma[j - C]) = (float)v;
}

struct GnPlan {
  int V, slices, CS, blocks, rows, stride;
  int TS, rpc, hold, buffers;  // held form: TS > 0
  bool more;                   // it holds a part only
  size_t smem;
};

// Channels of a slice as the held form wants them: whole groups, a power of two of 16-byte pieces up to a warp's; false: none
bool slice_lanes(int C, int cpg, int full, int* least, int* most) {
  if (C % full) return false;
  const bool fine = cpg < full;
  if (fine ? full % cpg != 0 : cpg % full != 0 || ((cpg / full) & (cpg / full - 1)) || cpg / full > 32) return false;
  *least = *most = fine ? 1 : cpg / full;
  while (*most < 32 && C % (2 * *most * full) == 0) *most *= 2;
  return true;
}

constexpr int kHeldBytes = 92 * 1024;  // of shared memory per block, two on an SM

// The held form.  Slices are 128 bytes of a pixel at least, where it has that many: at 64 the backward pass of 1904 images of 16x16x256 took 188 us,
// at 128 145; at 32 the forward pass of 64 images of 224x224x64 608 us for 260 (other blocks read the rest of a line at other times).  One or
// two large images want more blocks than a cluster has, and their blocks run at the same time: narrower there (one image of 224x224x64 20 us in slices
// of 128 bytes, 12.7 of 64, 10.1 of 32; four images 24, 23, 28).
//   Small images: the smallest team (a warp to a block) that holds a slice in kPer pieces a thread, the slice as wide as that allows.  Larger ones: a
// block, or as few blocks as give the SMs work, since blocks that exchange sums wait for one another (512 images of 28x28x128 forward: one
// block 53 us, two 61, four 103, eight 190), even where the slice then does not fit.  But no more images are in work at a time than L2 keeps between
// their two passes, as far as up to eight blocks to an image help that (256 images of 112x112x64 forward: one block 209 us, two 198, four 186,
// eight 163, sixteen 201; 512 of 56x56x64 93, 85, 91, 113, 163; 64 of 224x224x64 319, 218, 212, 204, 215; backward 623, 387, 322, 332, 365).
bool plan_held(int N, int P, int C, int cpg, int full, bool bwd, GnPlan* pl) {
  int least, most;
  if (!slice_lanes(C, cpg, full, &least, &most)) return false;
  const int tensors = bwd ? 2 : 1, kPer = bwd ? 4 : 8;
  const int wide = most < 8 ? most : 8 > least ? 8 : least;
  const int places = kHeldBytes / (kNT * 16 * tensors);  // per thread and tensor
  auto fill = [&](int lanes, int TS, int CS) {
    pl->V = full;
    pl->TS = TS;
    pl->CS = CS;
    pl->slices = C / (lanes * full);
    pl->rpc = (P + CS - 1) / CS;
    const long all = ((long)pl->rpc * lanes + TS - 1) / TS;
    pl->more = all > places;
    pl->hold = pl->more ? places - held_ring(bwd) : (int)all;
    pl->buffers = pl->more ? 1 : places / pl->hold < 4 ? places / pl->hold : 4;
    const long used = (pl->more ? places : pl->buffers * pl->hold) * (long)kNT * 16 * tensors;
    const long teams = kNT / TS;
    long per = 296 / CS * teams / pl->slices;  // teams at a time for each slice
    if (per > N) per = N;
    if (per < 1) per = 1;
    while (per * pl->slices % teams) ++per;
    pl->stride = (int)per;
    pl->blocks = (int)(per * pl->slices / teams * CS);
    pl->rows = (int)per * CS;
    const long fold = bwd ? 2l * full * kNT * 4 : 0;
    pl->smem = (size_t)(used > fold ? used : fold);
  };
  for (int TS = 32; TS <= kNT; TS *= 2) {
    int lanes = most;
    while (lanes > wide && ((long)P * lanes > (long)TS * kPer || (long)N * (C / (lanes * full)) * TS < 296 * kNT)) lanes /= 2;
    if ((long)P * lanes > (long)TS * kPer || lanes * full / cpg > 32) continue;
    if (TS < kNT && (long)N * (C / (lanes * full)) * TS < 148 * kNT) continue;  // few images: wider teams
    fill(lanes, TS, 1);
    return true;
  }
  if (wide * full / cpg > 32) return false;
  int lanes = wide;
  while (lanes > least && lanes > 2 && (long)N * (C / (lanes * full)) < 4) lanes /= 2;
  const long items = (long)N * (C / (lanes * full)), slice = (long)P * lanes * 16 * tensors;
  int CS = 1;
  while (CS < kMaxCluster && CS < P && slice / CS > 8192 && items * CS < 128) CS *= 2;
  auto in_work = [&] { return (items < 296 / CS ? items : 296 / CS) * slice; };
  while (CS < 8 && ((items * CS < 256 && slice / CS > 4 * kHeldBytes) ||
                    (in_work() > 96l << 20 && (!bwd || CS < 4 || items >= 2 * (296 / (2 * CS))))))  // backward, eight blocks: not for a turn and a bit
    CS *= 2;
  fill(lanes, kNT, CS);
  return true;
}

GnPlan plan_gn(int dtype, int N, int P, int C, int groups, bool bwd) {
  GnPlan pl{};
  const int cpg = C / groups;
  const size_t es = nf_esize(dtype);
  if (plan_held(N, P, C, cpg, 16 / (int)es, bwd, &pl)) return pl;
  const size_t image = (size_t)P * C * es * (bwd ? 2 : 1);
  // 16 bytes per thread where the slices allow it, else fewer, down to single channels.  A slice is some whole groups: all of them, fewer where C is
  // above kMaxCs, where one image per (largest portable) cluster would leave most SMs idle, or where the images in work (two blocks
  // on each SM) would fill half of L2 -- but not below 64 bytes of a pixel.
  for (pl.V = 16 / (int)es;; pl.V /= 2) {
    pl.slices = 0;
    for (int s = 1; s <= groups; ++s) {
      if (groups % s || C / s > kMaxCs || C / s % pl.V) continue;
      if (pl.slices && ((C / s) * es < 64 || ((long)N * pl.slices * 8 >= 296 && image / pl.slices / kMaxCluster <= 200000))) break;
      pl.slices = s;
    }
    if (pl.slices || pl.V == 1) break;
  }
  const size_t slab = image / pl.slices;
  const long items = (long)N * pl.slices;
  // as few blocks to a cluster as give the SMs work: they wait for one another at every image
  pl.CS = 1;
  while (pl.CS < kMaxCluster && pl.CS < P && slab / pl.CS > 8192 && (items * pl.CS < 256 || (pl.CS < 4 && slab / pl.CS > 262144))) pl.CS *= 2;
  long most = kMaxBlocks / (pl.CS * pl.slices);
  if (most < 1) most = 1;
  if (most > N) most = N;
  pl.blocks = (int)most * pl.slices * pl.CS;
  pl.stride = (int)most;
  pl.rows = (int)most * pl.CS;
  const int Cs = C / pl.slices;
  pl.smem = sizeof(float) * ((size_t)((bwd ? 2 : 3) * pl.V + 1) * kNT + 6 * Cs + 2 * (Cs / cpg));
  return pl;
}

// Counts of images and pixels run on in steps beyond the last one, channels are doubled: all in 32 bits
bool gn_size_ok(int N, int P, int C, int groups) { return C / groups <= kMaxCs && N <= 1 << 30 && P <= 1 << 30 && C <= 1 << 24; }

// Rows of partial sums that the backward pass needs at most, for N images or fewer: what was allocated for the largest batch then serves a ragged last one
// (fewer images get more blocks each).  A plan has at most 16 blocks to an image, and more rows than 16 only for as many as there are teams (eight to a block)
// for each slice; the generic form's slices may be one.
size_t gn_rows(int dtype, int N, int C, int groups) {
  const int full = 16 / (int)nf_esize(dtype);
  int least, most;
  size_t rows = kMaxBlocks;
  if (slice_lanes(C, C / groups, full, &least, &most)) {
    const size_t held = (size_t)296 * (kNT / 32) * (most * full) / C;  // `most` lanes make the fewest slices
    const int wide = most < 8 ? most : 8 > least ? 8 : least;
    if (wide * full / (C / groups) <= 32) rows = held;
  }
  if (rows < kMaxCluster) rows = kMaxCluster;
  const size_t few = (size_t)N * kMaxCluster;
  return (few < rows ? few : rows) + kNT / 32 - 1;  // rounded up to whole blocks of teams
}

bool gn_args_ok(int dtype, int N, int P, int C, int groups) {
  return (dtype == NF_F32 || dtype == NF_BF16) && N >= 1 && P >= 1 && C >= 1 && groups >= 1 && C % groups == 0;
}

// Clusters of a kernel that are on the GPU at a time: a cluster more than that would only start when the others have done all their images
template <typename K>
int resident_clusters(K kernel, int CS, int threads, size_t smem, int* out) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = CS;
  cfg.blockDim = threads;
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = CS;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  NF_CUDA(cudaOccupancyMaxActiveClusters(out, kernel, &cfg));
  return NF_OK;
}

template <typename T, int V, int ACT, bool BWD>
int launch_gn(GnArgs& a, GnPlan& pl) {
  static bool ready[64];
  static int resident[64][2][2][5];  // [device][FINE][MORE][log2 CS]; 0: not asked yet
  int dev = 0;
  NF_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return NF_EUNSUPPORTED;
  auto allow = [](auto k, int smem) -> int {
    NF_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    NF_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    return NF_OK;
  };
  auto k = group_norm_kernel<T, V, ACT, BWD>;
  if (!ready[dev]) {
    int rc = allow(k, 200 * 1024);
    if constexpr (V * sizeof(T) == 16) {
      if (rc == NF_OK) rc = allow(group_norm_held_kernel<T, V, ACT, BWD, true, false>, kHeldBytes);
      if (rc == NF_OK) rc = allow(group_norm_held_kernel<T, V, ACT, BWD, false, false>, kHeldBytes);
      if (rc == NF_OK) rc = allow(group_norm_held_kernel<T, V, ACT, BWD, true, true>, kHeldBytes);
      if (rc == NF_OK) rc = allow(group_norm_held_kernel<T, V, ACT, BWD, false, true>, kHeldBytes);
    }
    if (rc != NF_OK) return rc;
    ready[dev] = true;
  }
  if constexpr (V * sizeof(T) == 16) {
    if (pl.TS) {
      const bool fine = a.cpg < V;
      auto held = fine ? (pl.more ? group_norm_held_kernel<T, V, ACT, BWD, true, true> : group_norm_held_kernel<T, V, ACT, BWD, true, false>)
                       : (pl.more ? group_norm_held_kernel<T, V, ACT, BWD, false, true> : group_norm_held_kernel<T, V, ACT, BWD, false, false>);
      if (pl.CS > 1) {
        int lg = 0;
        while (1 << lg < pl.CS) ++lg;
        int& most = resident[dev][fine][pl.more][lg];
        if (!most) {
          const int rc = resident_clusters(held, pl.CS, kNT, kHeldBytes, &most);
          if (rc != NF_OK) return rc;
        }
        if (most < 1) return NF_EUNSUPPORTED;
        if (pl.blocks / pl.CS > most && pl.slices <= most) {
          a.stride = most / pl.slices;
          pl.blocks = a.stride * pl.slices * pl.CS;
          pl.rows = a.stride * pl.CS;
        }
      }
      nf_launch_cluster(held, (unsigned)pl.blocks, kNT, pl.smem, pl.CS, a);
      NF_LAUNCHED();
      return NF_OK;
    }
  }
  nf_launch_cluster(k, (unsigned)pl.blocks, kNT, pl.smem, pl.CS, a);
  NF_LAUNCHED();
  return NF_OK;
}

// bf16 has a kernel per activation; fp32 and channel counts that are no multiple of eight ask at run time
template <bool BWD>
int run_gn(int dtype, GnArgs& a, GnPlan& pl) {
  if (dtype == NF_F32)
    return pl.V == 4   ? launch_gn<float, 4, kAnyAct, BWD>(a, pl)
           : pl.V == 2 ? launch_gn<float, 2, kAnyAct, BWD>(a, pl)
                       : launch_gn<float, 1, kAnyAct, BWD>(a, pl);
  if (pl.V < 8)
    return pl.V == 4   ? launch_gn<bf16, 4, kAnyAct, BWD>(a, pl)
           : pl.V == 2 ? launch_gn<bf16, 2, kAnyAct, BWD>(a, pl)
                       : launch_gn<bf16, 1, kAnyAct, BWD>(a, pl);
  switch (a.act) {
    case NF_ACT_NONE: return launch_gn<bf16, 8, NF_ACT_NONE, BWD>(a, pl);
    case NF_ACT_RELU: return launch_gn<bf16, 8, NF_ACT_RELU, BWD>(a, pl);
    case NF_ACT_SILU: return launch_gn<bf16, 8, NF_ACT_SILU, BWD>(a, pl);
    default: return launch_gn<bf16, 8, NF_ACT_GELU, BWD>(a, pl);
  }
}

int fill_gn(GnArgs& a, const GnPlan& pl, int N, int P, int C, int groups, int act) {
  a.N = N; a.P = P; a.C = C; a.G = groups; a.cpg = C / groups;
  a.slices = pl.slices; a.Cs = C / pl.slices; a.vpr = a.Cs / pl.V;
  a.CS = pl.CS; a.stride = pl.stride; a.TS = pl.TS;
  a.rpc = pl.rpc; a.hold = pl.hold; a.buffers = pl.buffers;
  a.act = act;
  return nf_tc_op_status_ptr(&a.status);
}

}  // namespace

extern "C" int nf_group_norm_forward(int dtype, const void* x, const float* gamma, const float* beta, int N, int P, int C, int groups,
                                     float eps, int act, void* y, float* mean, float* rstd) {
  if (!x || !gamma || !beta || !y || !mean || !rstd || !gn_args_ok(dtype, N, P, C, groups) || !nf_act_ok(act) || !(eps > 0.f)) return NF_EINVAL;
  if (((uintptr_t)x | (uintptr_t)gamma | (uintptr_t)beta | (uintptr_t)y | (uintptr_t)mean | (uintptr_t)rstd) & 15) return NF_EALIGN;
  if (!gn_size_ok(N, P, C, groups)) return NF_EUNSUPPORTED;
  const size_t bytes = (size_t)N * P * C * nf_esize(dtype), cb = (size_t)C * 4, sb = (size_t)N * groups * 4;
  if (nf_shared({{y, bytes}, {mean, sb}, {rstd, sb}}, {{x, bytes}, {gamma, cb}, {beta, cb}})) return NF_EINVAL;
  GnPlan pl = plan_gn(dtype, N, P, C, groups, false);
  GnArgs a{};
  if (fill_gn(a, pl, N, P, C, groups, act) != NF_OK) return NF_ECUDA;
  a.x = x; a.gamma = gamma; a.beta = beta; a.out = y; a.mean = mean; a.rstd = rstd; a.eps = eps;
  return run_gn<false>(dtype, a, pl);
}

extern "C" size_t nf_group_norm_scratch_bytes(int dtype, int N, int P, int C, int groups) {
  if (!gn_args_ok(dtype, N, P, C, groups) || !gn_size_ok(N, P, C, groups)) return 0;
  return gn_rows(dtype, N, C, groups) * 2 * C * sizeof(float);
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
  if (!gn_size_ok(N, P, C, groups)) return NF_EUNSUPPORTED;
  const size_t bytes = (size_t)N * P * C * nf_esize(dtype);
  GnPlan pl = plan_gn(dtype, N, P, C, groups, true);
  const size_t used = gn_rows(dtype, N, C, groups) * 2 * C * sizeof(float);
  if (scratch_bytes < used) return NF_ENOWS;
  const size_t cb = (size_t)C * 4, sb = (size_t)N * groups * 4;
  if (nf_shared({{dx, bytes}, {dgamma, cb}, {dbeta, cb}, {scratch, used}}, {{x, bytes}, {dy, bytes}, {gamma, cb}, {beta, cb}, {mean, sb}, {rstd, sb}}))
    return NF_EINVAL;
  GnArgs a{};
  if (fill_gn(a, pl, N, P, C, groups, act) != NF_OK) return NF_ECUDA;
  a.x = x; a.dy = dy; a.gamma = gamma; a.beta = beta; a.out = dx; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.part = (float*)scratch;
  const int rc = run_gn<true>(dtype, a, pl);
  if (rc != NF_OK) return rc;
  nf_launch(group_norm_param_kernel, (unsigned)((2 * C + 31) / 32), 1024, 0, (const float*)scratch, pl.rows, C, dgamma, dbeta);
  NF_LAUNCHED();
  return NF_OK;
}
