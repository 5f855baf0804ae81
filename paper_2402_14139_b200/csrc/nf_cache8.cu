// The activation cache in 8 bits: quantised as it is written, read back row by row.
//
// A row is cut into groups of `group` consecutive elements (channels of one pixel, or of neighbouring ones); a group keeps one fp32
// scale s = a / top, a = its largest magnitude (at least 2^-100), top = 127 (int8) or 448 (e4m3), and per element the code
// nearest to x * (top / a).  Reading back is code * s, rounded once to the output type.  int8: |x - x'| <= s / 2; e4m3: a relative
// 2^-4 at most down to 2^-6 of the code range.
//
// HBM bounds both: every element is read and every code written once.  1260 rows of 65536 bf16 written 42 us (6.0 TB/s); 1904 of 10000 rows of 65536 read
// back 61 us (6.2 TB/s).  Rows that are no multiple of 16 (write) or 8 (read) elements go element by element at about half that.
#include <cuda_fp8.h>

#include "nf_internal.h"
#include "nf_ldst.cuh"
#include "nf_tc.h"

namespace {

constexpr uint32_t kFloorBits = 27u << 23;  // 2^-100 as a float: (127 - 100) << 23
template <int F> constexpr float kTop = F == NF_Q_INT8 ? 127.f : 448.f;

// Codes of x * (top / a), whose magnitude is at most the top, or one rounding above it.  int8: adding 1.5 * 2^23 rounds to an integer,
// ties to even, and leaves it in the low byte.
template <int F>
__device__ __forceinline__ uint32_t code_of(float q) {
  if constexpr (F == NF_Q_INT8) return __float_as_uint(__fadd_rn(q, 12582912.f)) & 255u;  // not fused with the product before it
  return (uint32_t)__nv_cvt_float_to_fp8(q, __NV_SATFINITE, __NV_E4M3);
}
template <int F>
__device__ __forceinline__ uint32_t codes4(f32x2 q01, f32x2 q23) {
  float a, b, c, d;
  if constexpr (F == NF_Q_INT8) {
    const f32x2 magic = nf_pack2(12582912.f, 12582912.f);
    nf_unpack2(nf_add_each(q01, magic), a, b);
    nf_unpack2(nf_add_each(q23, magic), c, d);
    return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040), __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
  }
  nf_unpack2(q01, a, b);
  nf_unpack2(q23, c, d);
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3) |
         (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3) << 16;
}
template <int F>
__device__ __forceinline__ float value_of(uint32_t code) {
  if constexpr (F == NF_Q_INT8) return (float)(int8_t)code;
  return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3)));
}
// The values of the four codes in w.  int8: a code offset by 128 is the low byte of a float whose unit is 1.
template <int F>
__device__ __forceinline__ void values4(uint32_t w, f32x2& v01, f32x2& v23) {
  if constexpr (F == NF_Q_INT8) {
    const uint32_t u = w ^ 0x80808080u;
    const f32x2 back = nf_pack2(-8388736.f, -8388736.f);  // 2^23 + 128
    v01 = nf_add2(nf_pack2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7540)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7541))), back);
    v23 = nf_add2(nf_pack2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7542)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7543))), back);
  } else {
    const float2 a = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xffffu), __NV_E4M3)));
    const float2 b = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3)));
    v01 = nf_pack2(a.x, a.y);
    v23 = nf_pack2(b.x, b.y);
  }
}
// Scale and reciprocal from the largest magnitude's bits.  A group that holds a NaN or an infinity (whose bits are above those of every
// finite number) gets a NaN for a scale, so that all of it reads back as NaN, and raises the flag.
template <int F>
__device__ __forceinline__ float scale_of(uint32_t abits, float* r, int32_t* status) {
  if (abits >= 0x7f800000u) {
    atomicOr(status, NF_ENONFINITE);
    *r = 0.f;
    return __uint_as_float(0x7fc00000u);
  }
  const float a = __uint_as_float(abits > kFloorBits ? abits : kFloorBits);
  *r = __fdiv_rn(kTop<F>, a);
  return __fdiv_rn(a, kTop<F>);
}

// Rows of whole 16-element pieces: a thread takes one piece (16 codes = one 16-byte store), the LG = group / 16 threads of a group find
// their largest magnitude by shuffles.  pieces = rows * row_elems / 16; groups end with their row, so the last one may be short.
template <int F, typename T, int LG>
__global__ void __launch_bounds__(256) quantize_vec_kernel(const T* __restrict__ x, size_t pieces, uint32_t per_row, uint32_t groups,
                                                           uint4* __restrict__ codes, float* __restrict__ scales, int32_t* status) {
  nf_pdl_begin();
  // threads are dealt to whole groups: a short last group leaves some of its threads idle
  const size_t slot = (size_t)blockIdx.x * 256 + threadIdx.x;
  const size_t g = slot / LG;
  const size_t row = g / groups;
  const uint32_t gi = (uint32_t)(g - row * groups), k = gi * LG + (uint32_t)(slot % LG);
  const bool on = k < per_row && row * per_row < pieces;
  const size_t e = row * per_row + k;
  f32x2 v[8];
  uint32_t top = 0;
  if (on) {
    if constexpr (sizeof(T) == 2) {  // magnitudes of bf16 pairs compared as they lie
      const uint4 a = __ldcs(reinterpret_cast<const uint4*>(x + e * 16)), b = __ldcs(reinterpret_cast<const uint4*>(x + e * 16 + 8));
      const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        m = __vmaxu2(m, w[i] & 0x7fff7fffu);
        v[i] = nf_pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
      }
      top = max(m & 0xffff0000u, m << 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 a = __ldcs(reinterpret_cast<const float4*>(x + e * 16 + 4 * i));
        v[2 * i] = nf_pack2(a.x, a.y);
        v[2 * i + 1] = nf_pack2(a.z, a.w);
        top = max(top, max(max(__float_as_uint(a.x) & 0x7fffffffu, __float_as_uint(a.y) & 0x7fffffffu),
                           max(__float_as_uint(a.z) & 0x7fffffffu, __float_as_uint(a.w) & 0x7fffffffu)));
      }
    }
  }
#pragma unroll
  for (int o = 1; o < LG; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (!on) return;
  float r;
  const float s = scale_of<F>(top, &r, status);
  uint32_t w[4];
  const f32x2 rr = nf_pack2(r, r);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = codes4<F>(nf_mul2(v[2 * i], rr), nf_mul2(v[2 * i + 1], rr));
  codes[e] = make_uint4(w[0], w[1], w[2], w[3]);
  if (slot % LG == 0) scales[g] = s;
}

// Any row length: a warp takes kWarpGroups neighbouring groups of a row, a lane every 32nd element; no piece is aligned, so loads and stores
// are single elements, 32 neighbours at a time.
constexpr int kWarpGroups = 4;

template <int F, typename T, int Q>  // Q = group / 32
__global__ void __launch_bounds__(256) quantize_any_kernel(const T* __restrict__ x, uint32_t row_elems, uint32_t groups, uint32_t chunks,
                                                           uint8_t* __restrict__ codes, float* __restrict__ scales, int32_t* status) {
  nf_pdl_begin();
  const int lane = threadIdx.x & 31;
  const uint32_t row = blockIdx.x / chunks, g0 = ((blockIdx.x - row * chunks) * 8 + threadIdx.x / 32) * kWarpGroups;
  const T* from = x + (size_t)row * row_elems;
  uint8_t* to = codes + (size_t)row * row_elems;
  float v[kWarpGroups][Q];
#pragma unroll
  for (int j = 0; j < kWarpGroups; ++j)
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      const uint32_t k = (g0 + j) * (32 * Q) + 32 * i + lane;
      v[j][i] = g0 + j < groups && k < row_elems ? ldf(from, k) : 0.f;
    }
#pragma unroll
  for (int j = 0; j < kWarpGroups; ++j) {
    if (g0 + j >= groups) return;  // the whole warp
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < Q; ++i) top = max(top, __float_as_uint(v[j][i]) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
    float r;
    const float s = scale_of<F>(top, &r, status);
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      const uint32_t k = (g0 + j) * (32 * Q) + 32 * i + lane;
      if (k < row_elems) to[k] = (uint8_t)code_of<F>(__fmul_rn(v[j][i], r));
    }
    if (lane == 0) scales[(size_t)row * groups + g0 + j] = s;
  }
}

// Row r of the output from row idx[r] of the cache; indices out of range as in nf_cache_gather.  A block takes kGatherSpan elements of one
// row: pieces of 8 codes (one 16-byte store of bf16), or, where rows are not made of such pieces, single elements.
constexpr int kGatherSpan = 8192;

template <int F, typename T>
__global__ void __launch_bounds__(256) gather_vec_kernel(const uint2* __restrict__ codes, const float* __restrict__ scales,
                                                         const int32_t* __restrict__ labels, int cache_rows, const int32_t* __restrict__ idx,
                                                         uint32_t per_row, uint32_t groups, int lg_log, uint32_t chunks, T* __restrict__ out,
                                                         int32_t* __restrict__ out_labels, int32_t* status) {
  nf_pdl_begin();
  const uint32_t r = blockIdx.x / chunks, chunk = blockIdx.x - r * chunks;
  const int32_t src = idx[r];
  const bool ok = src >= 0 && src < cache_rows;
  const uint2* from = codes + (size_t)(ok ? src : 0) * per_row;
  const float* sc = scales + (size_t)(ok ? src : 0) * groups;
  T* to = out + (size_t)r * per_row * 8;
  constexpr int kTurns = kGatherSpan / 8 / 256;
  const uint32_t k0 = chunk * (kGatherSpan / 8) + threadIdx.x;
  uint2 u[kTurns];
  float s[kTurns];
#pragma unroll
  for (int j = 0; j < kTurns; ++j) {
    const uint32_t k = k0 + 256 * j;
    if (k < per_row && ok) {
      u[j] = __ldcs(from + k);
      s[j] = sc[k >> lg_log];
    }
  }
#pragma unroll
  for (int j = 0; j < kTurns; ++j) {
    const uint32_t k = k0 + 256 * j;
    if (k >= per_row) break;
    float f[8];
    if (ok) {
      f32x2 v[4];
      const f32x2 ss = nf_pack2(s[j], s[j]);
      values4<F>(u[j].x, v[0], v[1]);
      values4<F>(u[j].y, v[2], v[3]);
#pragma unroll
      for (int i = 0; i < 4; ++i) nf_unpack2(nf_mul2(v[i], ss), f[2 * i], f[2 * i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = 0.f;
    }
    st8(to + (size_t)k * 8, f);
  }
  if (chunk == 0 && threadIdx.x == 0) {
    if (out_labels) out_labels[r] = ok ? labels[src] : -1;
    if (!ok) atomicOr(status, NF_EINDEX);
  }
}

template <int F, typename T>
__global__ void __launch_bounds__(256) gather_any_kernel(const uint8_t* __restrict__ codes, const float* __restrict__ scales,
                                                         const int32_t* __restrict__ labels, int cache_rows, const int32_t* __restrict__ idx,
                                                         uint32_t row_elems, uint32_t groups, int group_log, uint32_t chunks, T* __restrict__ out,
                                                         int32_t* __restrict__ out_labels, int32_t* status) {
  nf_pdl_begin();
  const uint32_t r = blockIdx.x / chunks, chunk = blockIdx.x - r * chunks;
  const int32_t src = idx[r];
  const bool ok = src >= 0 && src < cache_rows;
  const uint8_t* from = codes + (size_t)(ok ? src : 0) * row_elems;
  const float* sc = scales + (size_t)(ok ? src : 0) * groups;
  T* to = out + (size_t)r * row_elems;
  const uint32_t end = min(row_elems, (chunk + 1) * kGatherSpan);
#pragma unroll 8
  for (uint32_t k = chunk * kGatherSpan + threadIdx.x; k < end; k += 256) stf(to, k, ok ? value_of<F>(from[k]) * sc[k >> group_log] : 0.f);
  if (chunk == 0 && threadIdx.x == 0) {
    if (out_labels) out_labels[r] = ok ? labels[src] : -1;
    if (!ok) atomicOr(status, NF_EINDEX);
  }
}

bool args_ok(int format, int dtype, long long row_elems, int group) {
  return (format == NF_Q_INT8 || format == NF_Q_E4M3) && (dtype == NF_F32 || dtype == NF_BF16) && row_elems >= 1 &&
         row_elems <= 0x7fffffffll && (group == 32 || group == 64 || group == 128);
}

template <int F, typename T>
int quantize(const T* x, int rows, long long E, int group, uint8_t* codes, float* scales, int32_t* st) {
  const size_t groups = (size_t)((E + group - 1) / group), total = groups * rows;
  if (E % 16 == 0) {
    const int LG = group / 16;
    const size_t blocks = (total * LG + 255) / 256;
    if (blocks > 0x7fffffffull) return NF_EUNSUPPORTED;
    auto k = LG == 2 ? quantize_vec_kernel<F, T, 2> : LG == 4 ? quantize_vec_kernel<F, T, 4> : quantize_vec_kernel<F, T, 8>;
    nf_launch(k, (unsigned)blocks, 256, 0, x, (size_t)rows * (E / 16), (uint32_t)(E / 16), (uint32_t)groups, (uint4*)codes, scales, st);
  } else {
    const size_t chunks = (groups + 8 * kWarpGroups - 1) / (8 * kWarpGroups), blocks = chunks * rows;
    if (blocks > 0x7fffffffull) return NF_EUNSUPPORTED;
    auto k = group == 32 ? quantize_any_kernel<F, T, 1> : group == 64 ? quantize_any_kernel<F, T, 2> : quantize_any_kernel<F, T, 4>;
    nf_launch(k, (unsigned)blocks, 256, 0, x, (uint32_t)E, (uint32_t)groups, (uint32_t)chunks, codes, scales, st);
  }
  NF_LAUNCHED();
  return NF_OK;
}

template <int F, typename T>
int gather(const uint8_t* codes, const float* scales, const int32_t* labels, int cache_rows, const int32_t* idx, int count, long long E,
           int group, T* out, int32_t* out_labels, int32_t* st) {
  const size_t groups = (size_t)((E + group - 1) / group), chunks = (size_t)(E + kGatherSpan - 1) / kGatherSpan, blocks = chunks * count;
  const int lg = group == 32 ? 5 : group == 64 ? 6 : 7;
  if (blocks > 0x7fffffffull) return NF_EUNSUPPORTED;
  if (E % 8 == 0)
    nf_launch(gather_vec_kernel<F, T>, (unsigned)blocks, 256, 0, (const uint2*)codes, scales, labels, cache_rows, idx, (uint32_t)(E / 8),
              (uint32_t)groups, lg - 3, (uint32_t)chunks, out, out_labels, st);
  else
    nf_launch(gather_any_kernel<F, T>, (unsigned)blocks, 256, 0, codes, scales, labels, cache_rows, idx, (uint32_t)E, (uint32_t)groups, lg,
              (uint32_t)chunks, out, out_labels, st);
  NF_LAUNCHED();
  return NF_OK;
}

}  // namespace

extern "C" int nf_cache_quantize(int format, int dtype, const void* x, int rows, long long row_elems, int group, void* codes, float* scales) {
  if (!x || !codes || !scales || rows < 1 || !args_ok(format, dtype, row_elems, group)) return NF_EINVAL;
  if (((uintptr_t)x | (uintptr_t)codes | (uintptr_t)scales) & 15) return NF_EALIGN;
  const size_t n = (size_t)rows * row_elems, sb = (size_t)rows * ((row_elems + group - 1) / group) * 4;
  if (nf_overlap(x, n * nf_esize(dtype), codes, n) || nf_overlap(x, n * nf_esize(dtype), scales, sb) || nf_overlap(codes, n, scales, sb))
    return NF_EINVAL;
  int32_t* st = nullptr;
  if (nf_tc_op_status_ptr(&st) != NF_OK) return NF_ECUDA;
  uint8_t* c = (uint8_t*)codes;
  if (format == NF_Q_INT8)
    return dtype == NF_F32 ? quantize<NF_Q_INT8>((const float*)x, rows, row_elems, group, c, scales, st)
                           : quantize<NF_Q_INT8>((const bf16*)x, rows, row_elems, group, c, scales, st);
  return dtype == NF_F32 ? quantize<NF_Q_E4M3>((const float*)x, rows, row_elems, group, c, scales, st)
                         : quantize<NF_Q_E4M3>((const bf16*)x, rows, row_elems, group, c, scales, st);
}

extern "C" int nf_cache_gather_quantized(int format, const void* codes, const float* scales, const int32_t* cache_labels, int cache_rows,
                                         const int32_t* idx, int count, long long row_elems, int group, int dtype, void* out,
                                         int32_t* out_labels) {
  if (!codes || !scales || !idx || !out || cache_rows < 1 || count < 1 || !args_ok(format, dtype, row_elems, group)) return NF_EINVAL;
  if ((cache_labels == nullptr) != (out_labels == nullptr)) return NF_EINVAL;
  if (((uintptr_t)codes | (uintptr_t)scales | (uintptr_t)out) & 15) return NF_EALIGN;
  if (((uintptr_t)idx | (uintptr_t)cache_labels | (uintptr_t)out_labels) & 3) return NF_EALIGN;
  const size_t ob = (size_t)count * row_elems * nf_esize(dtype), nb = (size_t)count * 4;
  if (nf_shared({{out, ob}, {out_labels, nb}}, {{codes, (size_t)cache_rows * row_elems},
                                                {scales, (size_t)cache_rows * ((row_elems + group - 1) / group) * 4},
                                                {cache_labels, (size_t)cache_rows * 4},
                                                {idx, nb}}))
    return NF_EINVAL;
  int32_t* st = nullptr;
  if (nf_tc_op_status_ptr(&st) != NF_OK) return NF_ECUDA;
  const uint8_t* c = (const uint8_t*)codes;
  if (format == NF_Q_INT8)
    return dtype == NF_F32
               ? gather<NF_Q_INT8>(c, scales, cache_labels, cache_rows, idx, count, row_elems, group, (float*)out, out_labels, st)
               : gather<NF_Q_INT8>(c, scales, cache_labels, cache_rows, idx, count, row_elems, group, (bf16*)out, out_labels, st);
  return dtype == NF_F32 ? gather<NF_Q_E4M3>(c, scales, cache_labels, cache_rows, idx, count, row_elems, group, (float*)out, out_labels, st)
                         : gather<NF_Q_E4M3>(c, scales, cache_labels, cache_rows, idx, count, row_elems, group, (bf16*)out, out_labels, st);
}
