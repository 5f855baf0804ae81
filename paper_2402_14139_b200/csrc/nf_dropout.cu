// Dropout from a counter-based generator: the mask is a function of (seed, offset, element index) and is never stored, so the same
// call on the output's gradient is the backward pass.
#include "nf_internal.h"
#include "nf_ldst.cuh"

namespace {

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel Random Numbers: As Easy as 1, 2, 3, 2011): four 32-bit words from a 64-bit key
// and a 128-bit counter, here (block, offset) of 64 bits each.  The rounds' keys come ready from the host.
struct RoundKeys {
  uint32_t k0[10], k1[10];
};
__device__ __forceinline__ uint4 philox(const RoundKeys& key, uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long p0 = (unsigned long long)c0 * 0xD2511F53u, p1 = (unsigned long long)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ key.k0[r];
    c1 = (uint32_t)p1;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ key.k1[r];
    c3 = (uint32_t)p0;
  }
  return make_uint4(c0, c1, c2, c3);
}

// An element is dropped where its word is below the threshold; it is then 0 whatever it was (a product with a zero mask would keep an
// infinity or NaN there).
__device__ __forceinline__ void drop8(float (&v)[8], const uint4& a, const uint4& b, uint32_t threshold, float scale) {
  const uint32_t bits[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  const f32x2 s = nf_pack2(scale, scale);
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    nf_unpack2(nf_mul2(nf_pack2(v[e], v[e + 1]), s), v[e], v[e + 1]);
    v[e] = bits[e] >= threshold ? v[e] : 0.f;
    v[e + 1] = bits[e + 1] >= threshold ? v[e + 1] : 0.f;
  }
}

// Eight elements (two blocks of the generator) per thread.  The generator bounds bf16: about 140 instructions per thread in ten rounds that depend on one
// another, the most of them on the integer pipe, which is 59% busy, issue slots 61%; 70 M elements 64 us (4.4 TB/s), fp32 35 M 48 us (5.8 TB/s).  Blocks that stride over the tensor with the
// next pieces on their way took longer (72 us with one piece, 87 with two: fewer threads to hide the rounds' latency), and so did four pieces a
// thread (95 us).  WIDE: block numbers beyond 32 bits.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) dropout_kernel(const T* x, size_t n, uint32_t threshold, float scale, const __grid_constant__ RoundKeys key,
                                                      unsigned long long offset, const unsigned long long* offset_dev, T* y) {
  nf_pdl_begin();
  if (offset_dev) offset += *offset_dev;
  const uint32_t o0 = (uint32_t)offset, o1 = (uint32_t)(offset >> 32);
  const size_t pieces = n / 8, i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i < pieces) {
    float v[8];
    ld8(x + i * 8, v);
    const size_t block = 2 * i;
    const uint32_t hi = WIDE ? (uint32_t)(block >> 32) : 0u;
    drop8(v, philox(key, (uint32_t)block, hi, o0, o1), philox(key, (uint32_t)block + 1, hi, o0, o1), threshold, scale);
    st8(y + i * 8, v);
  }
  if (blockIdx.x == 0 && threadIdx.x < 2 && pieces * 8 + threadIdx.x * 4 < n) {  // up to seven elements behind the last piece
    const size_t at = pieces * 8 + threadIdx.x * 4, block = at / 4;
    const uint4 w = philox(key, (uint32_t)block, (uint32_t)(block >> 32), o0, o1);
    const uint32_t bits[4] = {w.x, w.y, w.z, w.w};
    for (int e = 0; e < 4 && at + e < n; ++e) stf(y, at + e, bits[e] >= threshold ? ldf(x, at + e) * scale : 0.f);
  }
}

template <typename T>
void launch_dropout(const void* x, size_t n, uint32_t threshold, float scale, const RoundKeys& key, unsigned long long offset,
                    const unsigned long long* offset_dev, void* y) {
  const size_t blocks = (n / 8 + 255) / 256;
  nf_launch(n >> 34 ? dropout_kernel<T, true> : dropout_kernel<T, false>, (unsigned)(blocks ? blocks : 1), 256, 0, (const T*)x, n, threshold, scale, key,
            offset, offset_dev, (T*)y);
}

}  // namespace

extern "C" int nf_dropout(int dtype, const void* x, long long n, float p, unsigned long long seed, unsigned long long offset,
                          const unsigned long long* offset_dev, void* y) {
  if (!x || !y || n < 1 || (dtype != NF_F32 && dtype != NF_BF16) || !(p >= 0.f && p < 1.f)) return NF_EINVAL;
  if (((uintptr_t)x | (uintptr_t)y) & 15 || (uintptr_t)offset_dev & 7) return NF_EALIGN;
  const size_t bytes = (size_t)n * nf_esize(dtype);
  if ((x != y && nf_overlap(x, bytes, y, bytes)) || nf_overlap(y, bytes, offset_dev, 8)) return NF_EINVAL;
  const uint32_t threshold = (uint32_t)((double)p * 4294967296.0);  // p < 1 as a float is at most 1 - 2^-24
  const float scale = (float)(1.0 / (1.0 - (double)p));
  if ((size_t)n / 2048 >= 0x7fffffffull) return NF_EUNSUPPORTED;
  RoundKeys key;
  for (uint32_t r = 0; r < 10; ++r) {
    key.k0[r] = (uint32_t)seed + r * 0x9E3779B9u;
    key.k1[r] = (uint32_t)(seed >> 32) + r * 0xBB67AE85u;
  }
  if (dtype == NF_F32)
    launch_dropout<float>(x, (size_t)n, threshold, scale, key, offset, offset_dev, y);
  else
    launch_dropout<bf16>(x, (size_t)n, threshold, scale, key, offset, offset_dev, y);
  NF_LAUNCHED();
  return NF_OK;
}
