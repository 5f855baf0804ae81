// The activation cache in 8 bits: quantised as it is written, read back row by row.
//
// A row is cut into groups of `group` consecutive elements (channels of one pixel, or of neighbouring ones); a group keeps one fp32
// scale s = a / top, a = its largest magnitude (at least 2^-100), top = 127 (int8) or 448 (e4m3), and per element the code
// nearest to x * (top / a).  Reading back is code * s, rounded once to the output type.  int8: |x - x'| <= s / 2; e4m3: a relative
// 2^-4 at most down to 2^-6 of the code range.
#include <cuda_fp8.h>

#include "nf_internal.h"
#include "nf_ldst.cuh"
#include "nf_tc.h"

namespace {

constexpr uint32_t kFloorBits = 27u << 23;  // 2^-100 as a float: (127 - 100) << 23
template <int F> constexpr float kTop = F == NF_Q_INT8 ? 127.f : 448.f;

template <int F>
__device__ __forceinline__ uint32_t code_of(float q) {  // the code of x * (top / a)
  if constexpr (F == NF_Q_INT8) return (uint32_t)(__float2int_rn(fminf(fmaxf(q, -127.f), 127.f)) & 255);
  return (uint32_t)__nv_cvt_float_to_fp8(q, __NV_SATFINITE, __NV_E4M3);
}
template <int F>
__device__ __forceinline__ float value_of(uint32_t code) {
  if constexpr (F == NF_Q_INT8) return (float)(int8_t)code;
  return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3)));
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
  float v[16];
  uint32_t top = 0;
  if (on) {
    ld8(x + e * 16, *reinterpret_cast<float(*)[8]>(v));
    ld8(x + e * 16 + 8, *reinterpret_cast<float(*)[8]>(v + 8));
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  }
#pragma unroll
  for (int o = 1; o < LG; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (!on) return;
  float r;
  const float s = scale_of<F>(top, &r, status);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[i] |= code_of<F>(v[4 * i + j] * r) << (8 * j);
  }
  codes[e] = make_uint4(w[0], w[1], w[2], w[3]);
  if (slot % LG == 0) scales[g] = s;
}

// Any row length: a warp per group
template <int F, typename T>
__global__ void __launch_bounds__(256) quantize_any_kernel(const T* __restrict__ x, size_t total_groups, size_t row_elems, uint32_t groups,
                                                           int group, uint8_t* __restrict__ codes, float* __restrict__ scales,
                                                           int32_t* status) {
  nf_pdl_begin();
  const int lane = threadIdx.x & 31;
  const size_t g = (size_t)blockIdx.x * 8 + threadIdx.x / 32;
  if (g >= total_groups) return;
  const size_t row = g / groups, first = (g - row * groups) * group;
  const int len = (int)(row_elems - first < (size_t)group ? row_elems - first : (size_t)group);
  const size_t base = row * row_elems + first;
  float v[4];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = lane + 32 * i < len ? ldf(x, base + lane + 32 * i) : 0.f;
    top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  }
#pragma unroll
  for (int o = 1; o < 32; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  float r;
  const float s = scale_of<F>(top, &r, status);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane + 32 * i < len) codes[base + lane + 32 * i] = (uint8_t)code_of<F>(v[i] * r);
  if (lane == 0) scales[g] = s;
}

// One piece of 16 elements per thread; out of range indices as in nf_cache_gather
template <int F, typename T>
__global__ void __launch_bounds__(256) gather_vec_kernel(const uint4* __restrict__ codes, const float* __restrict__ scales,
                                                         const int32_t* __restrict__ labels, int cache_rows,
                                                         const int32_t* __restrict__ idx, uint32_t per_row, uint32_t groups, int lg_log,
                                                         size_t total, T* __restrict__ out, int32_t* __restrict__ out_labels, int32_t* status) {
  nf_pdl_begin();
  const size_t e = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= total) return;
  const size_t r = e / per_row;
  const uint32_t k = (uint32_t)(e - r * per_row);
  const int32_t src = idx[r];
  const bool ok = src >= 0 && src < cache_rows;
  float v[16];
  if (ok) {
    const uint4 u = codes[(size_t)src * per_row + k];
    const float s = scales[(size_t)src * groups + (k >> lg_log)];
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = value_of<F>((w[i / 4] >> (8 * (i % 4))) & 255u) * s;
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = 0.f;
  }
  st8(out + e * 16, *reinterpret_cast<float(*)[8]>(v));
  st8(out + e * 16 + 8, *reinterpret_cast<float(*)[8]>(v + 8));
  if (k == 0) {
    if (out_labels) out_labels[r] = ok ? labels[src] : -1;
    if (!ok) atomicOr(status, NF_EINDEX);
  }
}

template <int F, typename T>
__global__ void __launch_bounds__(256) gather_any_kernel(const uint8_t* __restrict__ codes, const float* __restrict__ scales,
                                                         const int32_t* __restrict__ labels, int cache_rows,
                                                         const int32_t* __restrict__ idx, size_t row_elems, size_t groups, int group,
                                                         size_t total, T* __restrict__ out, int32_t* __restrict__ out_labels, int32_t* status) {
  nf_pdl_begin();
  const size_t e = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= total) return;
  const size_t r = e / row_elems, k = e - r * row_elems;
  const int32_t src = idx[r];
  const bool ok = src >= 0 && src < cache_rows;
  stf(out, e, ok ? value_of<F>(codes[(size_t)src * row_elems + k]) * scales[(size_t)src * groups + k / group] : 0.f);
  if (k == 0) {
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
    const size_t blocks = (total + 7) / 8;
    if (blocks > 0x7fffffffull) return NF_EUNSUPPORTED;
    nf_launch(quantize_any_kernel<F, T>, (unsigned)blocks, 256, 0, x, total, (size_t)E, (uint32_t)groups, group, codes, scales, st);
  }
  NF_LAUNCHED();
  return NF_OK;
}

template <int F, typename T>
int gather(const uint8_t* codes, const float* scales, const int32_t* labels, int cache_rows, const int32_t* idx, int count, long long E,
           int group, T* out, int32_t* out_labels, int32_t* st) {
  const size_t groups = (size_t)((E + group - 1) / group);
  const bool vec = E % 16 == 0;
  const size_t total = (size_t)count * (vec ? E / 16 : E), blocks = (total + 255) / 256;
  if (blocks > 0x7fffffffull) return NF_EUNSUPPORTED;
  if (vec)
    nf_launch(gather_vec_kernel<F, T>, (unsigned)blocks, 256, 0, (const uint4*)codes, scales, labels, cache_rows, idx, (uint32_t)(E / 16),
              (uint32_t)groups, group == 32 ? 1 : group == 64 ? 2 : 3, total, out, out_labels, st);
  else
    nf_launch(gather_any_kernel<F, T>, (unsigned)blocks, 256, 0, codes, scales, labels, cache_rows, idx, (size_t)E, groups, group, total, out,
              out_labels, st);
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
  const size_t ob = (size_t)count * row_elems * nf_esize(dtype);
  if (nf_overlap(out, ob, codes, (size_t)cache_rows * row_elems) || nf_overlap(out, ob, scales, (size_t)cache_rows * ((row_elems + group - 1) / group) * 4))
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
