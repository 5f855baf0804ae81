// Dropout from a counter-based generator: the mask is a function of (seed, offset, element index) and is never stored, so the same
// call on the output's gradient is the backward pass.
#include "nf_internal.h"
#include "nf_ldst.cuh"

namespace {

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel Random Numbers: As Easy as 1, 2, 3, 2011): four 32-bit words from a 64-bit key
// and a 128-bit counter, here (block, offset) of 64 bits each.
__device__ __forceinline__ uint4 philox(uint2 key, unsigned long long block, unsigned long long offset) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long p0 = (unsigned long long)c0 * 0xD2511F53u, p1 = (unsigned long long)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ key.x;
    c1 = (uint32_t)p1;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ key.y;
    c3 = (uint32_t)p0;
    key.x += 0x9E3779B9u;
    key.y += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// Eight elements (two blocks of the generator) per thread.  An element is dropped where its word is below `threshold`; it is then 0
// whatever it was (a product with a zero mask would keep an infinity or NaN there).
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(const T* x, size_t n, uint32_t threshold, float scale, uint2 key,
                                                      unsigned long long offset, const unsigned long long* offset_dev, T* y) {
  nf_pdl_begin();
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  if (offset_dev) offset += *offset_dev;
  const bool whole = i + 8 <= n;
  float v[8];
  if (whole) {
    ld8(x + i, v);
  } else {
    for (int e = 0; e < 8; ++e) v[e] = i + e < n ? ldf(x, i + e) : 0.f;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint4 w = philox(key, i / 4 + h, offset);
    const uint32_t bits[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * h + e] = bits[e] >= threshold ? v[4 * h + e] * scale : 0.f;
  }
  if (whole) {
    st8(y + i, v);
  } else {
    for (int e = 0; e < 8; ++e)
      if (i + e < n) stf(y, i + e, v[e]);
  }
}

}  // namespace

extern "C" int nf_dropout(int dtype, const void* x, long long n, float p, unsigned long long seed, unsigned long long offset,
                          const unsigned long long* offset_dev, void* y) {
  if (!x || !y || n < 1 || (dtype != NF_F32 && dtype != NF_BF16) || !(p >= 0.f && p < 1.f)) return NF_EINVAL;
  if (((uintptr_t)x | (uintptr_t)y) & 15 || (uintptr_t)offset_dev & 7) return NF_EALIGN;
  const size_t bytes = (size_t)n * nf_esize(dtype);
  if (x != y && nf_overlap(x, bytes, y, bytes)) return NF_EINVAL;
  const size_t blocks = ((size_t)n + 2047) / 2048;
  if (blocks > 0x7fffffffull) return NF_EUNSUPPORTED;
  const uint32_t threshold = (uint32_t)((double)p * 4294967296.0);  // p < 1 as a float is at most 1 - 2^-24
  const float scale = (float)(1.0 / (1.0 - (double)p));
  const uint2 key = make_uint2((uint32_t)seed, (uint32_t)(seed >> 32));
  if (dtype == NF_F32)
    nf_launch(dropout_kernel<float>, (unsigned)blocks, 256, 0, (const float*)x, (size_t)n, threshold, scale, key, offset, offset_dev, (float*)y);
  else
    nf_launch(dropout_kernel<bf16>, (unsigned)blocks, 256, 0, (const bf16*)x, (size_t)n, threshold, scale, key, offset, offset_dev, (bf16*)y);
  NF_LAUNCHED();
  return NF_OK;
}
