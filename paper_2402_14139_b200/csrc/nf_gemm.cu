// C[p][q] = sum over r of A(p, r) B(q, r) on tcgen05.mma, bf16 operands, fp32 accumulators in tensor memory.
//
// Tiles of 256 x 256 results by a pair of blocks on neighbouring SMs (cta_group::2: each block stages 128 rows of either operand, half the
// shared-memory traffic of two single tiles), or of 128 x 128 by one block where there are too few large tiles for the SMs.  Persistent
// blocks of ten warps: one feeds a ring of 64-deep operand tiles by TMA, one issues the products, eight take finished accumulators
// out of tensor memory (two sets, so the next tile's products go on) through shared memory to TMA stores.  Operands are read
// as they lie: contiguous along r (K-major) or along p / q (MN-major), so that no transposed copy exists.
//
// The tensor core cuts low bits off its running sum at every instruction, always towards zero (about 2^-25 of it here), so a sum over
// thousands of products would lose the digits that fp32 has, and one over 2^18 of one sign a third of a bf16 step (1.5e-3 of the result).  Accumulators
// therefore change every `seg` steps of 64 and the warps add them up in registers: every 8 steps (3 of parts) for fp32 results, every 16 for bf16 ones,
// which bounds their loss at 2^-18 whatever the length (358 us instead of 354 for the input gradient of 8602 x 8192 -> 4096; sums up to 1024 need it not).  fp32 operands come as three bf16 parts, x = h + m + l exactly, and the six products
// l h, h l, m m, h m, m h, h h; what is left out is below 2^-24 of |x| |w|.  The three parts of a step of 64 lie in three stages side by side,
// so that each is brought in once for all its products.
//
// What bounds it: the tensor pipe where sums are long (gradients of 8602 x 8192 -> 4096: the two products 728 us, 1.59 PFLOP/s, the pipe 91% and 86%
// busy), the epilogue's latency where they are short (200704 x 256 x 256 with residual: 65 us, 4.7 TB/s, DRAM 51% and issue slots 26% busy), the ends of the pipeline and the join of partial
// sums where the result has few tiles (128 x 4096 x 4096: 17 us, its weights alone 5).  For those, clusters that join a tile's sums through
// distributed shared memory took 16.4 us there but 14 instead of 12 at 1000 x 1000 x 1000, and pairs of blocks on 256 x 128 tiles 10.6 there and
// 35.7 instead of 26.5 at 318 x 2408 x 840 fp32: neither is here.
#include <cuda.h>

#include "nf_act.cuh"
#include "nf_gemm.h"
#include "nf_ptx.cuh"
#include "nf_tc.h"

namespace {

constexpr int kGemmThreads = 320;  // warp 0: TMA, warp 1: products, warps 2-9: epilogue
constexpr int kBox = 64;           // r per operand tile: 128 bytes of bf16
constexpr int kSegBf16 = 16;       // bf16 results: operand tiles between two readings of an accumulator
// Tiles of 32 rows x 128 bytes per epilogue warp on their way out: two, or one where sums are long (fp32 results) and a sixth operand stage
// is worth more: the parts of the next step of 64 are then all on their way while this one's are multiplied
template <typename T> constexpr int kTiles = sizeof(T) == 4 ? 1 : 2;
template <typename T> constexpr int kStaging = 8 * kTiles<T> * 4096;

struct GemmParams {
  int P, Q, kblocks;           // operand tiles along r: 64 products each, times the parts
  int tiles_p, tiles_q, splits, planes, seg;
  int a_along_r, b_along_r;
  int tma_out;                 // rows of C are multiples of 16 bytes: TMA stores them
  Epilogue e;
  int32_t* status;
};

__device__ __forceinline__ void unit_at(const GemmParams& p, int u, int& pt, int& qt, int& sp) {
  sp = u % p.splits;
  const int t = u / p.splits, band = 8 * p.tiles_q, g = t / band, first = g * 8;
  const int rows = p.tiles_p - first < 8 ? p.tiles_p - first : 8, in = t - g * band;
  pt = first + in % rows;  // bands of eight tile rows, so that what runs at a time shares operand tiles in L2
  qt = in / rows;
}

template <typename T> struct Pack;
template <> struct Pack<bf16> {
  static constexpr int n = 8;  // values in 16 bytes
  __device__ static __forceinline__ uint4 pack(const float* v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static __forceinline__ void add(const uint4& u, float* v) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] += __uint_as_float(w[i] << 16);
      v[2 * i + 1] += __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};
template <> struct Pack<float> {
  static constexpr int n = 4;
  __device__ static __forceinline__ uint4 pack(const float* v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
  __device__ static __forceinline__ void add(const uint4& u, float* v) {
    v[0] += __uint_as_float(u.x);
    v[1] += __uint_as_float(u.y);
    v[2] += __uint_as_float(u.z);
    v[3] += __uint_as_float(u.w);
  }
};

// A warp's 32 x 128-byte tile in shared memory (16-byte pieces swizzled by row) from or to rows of C that TMA cannot address
template <typename T>
__device__ __forceinline__ void tile_from_rows(uint32_t tile, const T* src, int row0, int col0, int P, int Q, int lane) {
  constexpr int CH = 128 / sizeof(T), W = CH / 32;
  for (int r = 0; r < 32 && row0 + r < P; ++r)
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const int c = lane + 32 * k;
      if (col0 + c < Q) {
        const uint32_t at = tile + r * 128 + (((c / Pack<T>::n) ^ (r & 7)) << 4) + (c % Pack<T>::n) * sizeof(T);
        const T v = src[(size_t)(row0 + r) * Q + col0 + c];
        if constexpr (sizeof(T) == 2) asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"(__bfloat16_as_ushort(v)) : "memory");
        else asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(__float_as_uint(v)) : "memory");
      }
    }
}
template <typename T>
__device__ __forceinline__ void tile_to_rows(uint32_t tile, T* dst, int row0, int col0, int P, int Q, int lane) {
  constexpr int CH = 128 / sizeof(T), W = CH / 32;
  for (int r = 0; r < 32 && row0 + r < P; ++r)
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const int c = lane + 32 * k;
      if (col0 + c < Q) {
        const uint32_t at = tile + r * 128 + (((c / Pack<T>::n) ^ (r & 7)) << 4) + (c % Pack<T>::n) * sizeof(T);
        T* to = dst + (size_t)(row0 + r) * Q + col0 + c;
        if constexpr (sizeof(T) == 2) {
          uint16_t v;
          asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(at) : "memory");
          *to = __ushort_as_bfloat16(v);
        } else {
          uint32_t v;
          asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
          *to = __uint_as_float(v);
        }
      }
    }
}

// One branch per activation, not one per value: with the branch inside the loop the 1x1 product of 200704 x 256 x 256 took 136 us for 65
template <typename T, int CH>
__device__ __forceinline__ void activate(float (&v)[CH], int act) {
  if (act == NF_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < CH; ++j) v[j] = nf_act_value<T>(v[j], NF_ACT_RELU);
  } else if (act == NF_ACT_SILU) {
#pragma unroll
    for (int j = 0; j < CH; ++j) v[j] = nf_act_value<T>(v[j], NF_ACT_SILU);
  } else if (act == NF_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < CH; ++j) v[j] = nf_act_value<T>(v[j], NF_ACT_GELU);
  }
}

// One warp's way out: 32 rows x CH columns at a time.  `turn` counts the tiles of this warp, which take its staging tiles in turn.
template <typename T>
struct WayOut {
  static constexpr int CH = 128 / sizeof(T);
  uint32_t stage;   // shared address of this warp's two tiles
  uint8_t* stage_p;
  uint64_t* rbar;   // two barriers: residual tile has landed
  uint32_t rphase;  // parities, one bit per tile
  uint32_t turn;
  int lane;
  volatile int* abort_flag;

  // The residual tile at (row0, col0) starts on its way into staging tile `b`, once what was stored from there has been read
  __device__ __forceinline__ void fetch(const GemmParams& p, const CUtensorMap* tr, uint32_t b, int row0, int col0) {
    if (p.splits > 1 || !p.e.residual || !p.tma_out || row0 >= p.P || col0 >= p.Q) return;
    if (lane == 0) {
      ptx::tma_store_wait_read();
      ptx::mbar_expect_tx(&rbar[b], 4096);
      ptx::tma_load_3d<1>(stage_p + b * 4096, tr, &rbar[b], col0, row0, 0);
    }
  }
  // v: this lane's row of the tile at (row0, col0); the next tile of this unit starts at column next_col
  __device__ __forceinline__ void put(const GemmParams& p, const CUtensorMap* tc, const CUtensorMap* tp, const CUtensorMap* tr, int row0, int col0, int plane,
                                      int next_col, float (&v)[CH]) {
    constexpr int n = Pack<T>::n;
    const uint32_t b = turn & (kTiles<T> - 1);
    ++turn;
    if (row0 >= p.P || col0 >= p.Q) return;  // the whole warp
    const bool whole = p.splits == 1;
    const uint32_t row = stage + b * 4096 + lane * 128;
    if (whole && p.e.bias) {
      const float* bias = p.e.bias + col0;
      if (col0 + CH <= p.Q) {
#pragma unroll
        for (int j = 0; j < CH; j += 4) {
          const float4 t = __ldg(reinterpret_cast<const float4*>(bias + j));
          v[j] += t.x; v[j + 1] += t.y; v[j + 2] += t.z; v[j + 3] += t.w;
        }
      } else {
#pragma unroll
        for (int j = 0; j < CH; ++j)
          if (col0 + j < p.Q) v[j] += __ldg(bias + j);
      }
    }
    if (whole && p.e.residual) {
      if (p.tma_out) {
        if constexpr (kTiles<T> == 2) fetch(p, tr, b ^ 1, row0, next_col);
        ptx::mbar_wait(&rbar[b], (rphase >> b) & 1, abort_flag);  // sets the abort flag itself when it gives up
        rphase ^= 1u << b;
      } else {
        tile_from_rows<T>(stage + b * 4096, reinterpret_cast<const T*>(p.e.residual), row0, col0, p.P, p.Q, lane);
        __syncwarp();
      }
#pragma unroll
      for (int i = 0; i < CH / n; ++i) Pack<T>::add(ptx::lds128(row + ((i ^ (lane & 7)) << 4)), v + i * n);
    } else if (p.tma_out && lane == 0) {  // what was stored from this tile before has been read
      if constexpr (kTiles<T> == 2) ptx::tma_store_wait_read_but_one();
      else ptx::tma_store_wait_read();
    }
    __syncwarp();
    if (whole && p.e.pre) {
#pragma unroll
      for (int i = 0; i < CH / n; ++i) ptx::sts128(row + ((i ^ (lane & 7)) << 4), Pack<T>::pack(v + i * n));
      send(p, tp, reinterpret_cast<T*>(p.e.pre), b, row0, col0, 0);
      if (p.tma_out && lane == 0) ptx::tma_store_wait_read();
      __syncwarp();
    }
    if (whole) activate<T, CH>(v, p.e.act);
#pragma unroll
    for (int i = 0; i < CH / n; ++i) ptx::sts128(row + ((i ^ (lane & 7)) << 4), Pack<T>::pack(v + i * n));
    send(p, tc, reinterpret_cast<T*>(p.e.out) + (size_t)plane * p.P * p.Q, b, row0, col0, plane);
    if constexpr (kTiles<T> == 1) fetch(p, tr, b, row0, next_col);  // waits for the store just sent to have been read
  }
  __device__ __forceinline__ void send(const GemmParams& p, const CUtensorMap* m, T* dst, uint32_t b, int row0, int col0, int plane) {
    if (p.tma_out) {
      ptx::fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        ptx::tma_store_3d(m, stage_p + b * 4096, col0, row0, plane);
        ptx::tma_store_commit();
      }
    } else {
      __syncwarp();
      tile_to_rows<T>(stage + b * 4096, dst, row0, col0, p.P, p.Q, lane);
      __syncwarp();
    }
  }
};

template <int CG, int BN, typename T> constexpr int kGemmStages = (227 * 1024 - 1024 - 512 - kStaging<T>) / (128 * 128 + BN / CG * 128);
template <int CG, int BN, typename T> constexpr int kGemmSmem = 1024 + kGemmStages<CG, BN, T> * (128 * 128 + BN / CG * 128) + kStaging<T> + 512;

// SEG: the accumulators change every p.seg steps of 64, and the warps add them up in registers
template <int CG, int BN, typename T, bool SEG>
__global__ void __launch_bounds__(kGemmThreads, 1)
gemm_tc_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ CUtensorMap tm_c,
               const __grid_constant__ CUtensorMap tm_r, const __grid_constant__ CUtensorMap tm_p, const __grid_constant__ GemmParams p) {
  constexpr int kStages = kGemmStages<CG, BN, T>, kA = 128 * 128, kB = BN / CG * 128, kStage = kA + kB;
  constexpr uint32_t kCols = 2 * BN;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* staging = smem + kStages * kStage;
  uint64_t* full = reinterpret_cast<uint64_t*>(staging + kStaging<T>);
  uint64_t* empty = full + kStages;
  uint64_t* tfull = empty + kStages;
  uint64_t* tempty = tfull + 2;
  uint64_t* rbars = tempty + 2;  // [8][2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(rbars + 16);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? ptx::cluster_rank() : 0;
  const int first = blockIdx.x / CG, step = gridDim.x / CG, units = p.tiles_p * p.tiles_q * p.splits;
  auto k_range = [&](int sp, int& k0, int& k1) {  // all parts of a tile
    const int groups = p.kblocks / p.planes;
    k0 = (int)((long long)groups * sp / p.splits) * p.planes;
    k1 = (int)((long long)groups * (sp + 1) / p.splits) * p.planes;
  };

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&tfull[a], 1);
      ptx::mbar_init(&tempty[a], CG * 8);
    }
    for (int i = 0; i < 16; ++i) ptx::mbar_init(&rbars[i], 1);
    *abort_flag = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tmap(&tm_a);
    ptx::prefetch_tmap(&tm_b);
    ptx::prefetch_tmap(&tm_c);
  }
  if (warp == 1) ptx::tmem_alloc_cg<CG>(tmem_slot, kCols);
  ptx::tc_fence_before();
  __syncthreads();
  if constexpr (CG == 2) ptx::cluster_sync();  // the other block's barriers are ready
  ptx::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  nf_pdl_begin();

  if (warp == 0) {
    if (ptx::elect_one()) {
      uint32_t s = 0, ph = 0, filled = 0;
      bool ok = true;
      for (int u = first; ok && u < units; u += step) {
        int pt, qt, sp, k0, k1;
        unit_at(p, u, pt, qt, sp);
        k_range(sp, k0, k1);
        const int prow = pt * 128 * CG + (int)rank * 128, qrow = qt * BN + (int)rank * (BN / CG);
        int r0 = k0 / p.planes * kBox, j = 0;  // j counts the parts from the smallest
        for (int kb = k0; kb < k1; ++kb) {
          if (!ptx::mbar_wait(&empty[s], ph ^ 1, abort_flag)) { ok = false; break; }
          uint8_t* st = smem + s * kStage;
          const int part = p.planes - 1 - j;
          if (rank == 0) ptx::mbar_expect_tx(&full[s], CG * kStage);
          if (p.a_along_r) {
            ptx::tma_load_3d<CG>(st, &tm_a, &full[s], r0, prow, part);
          } else {
            ptx::tma_load_3d<CG>(st, &tm_a, &full[s], prow, r0, part);
            ptx::tma_load_3d<CG>(st + 8192, &tm_a, &full[s], prow + 64, r0, part);
          }
          if (p.b_along_r) {
            ptx::tma_load_3d<CG>(st + kA, &tm_b, &full[s], r0, qrow, part);
          } else {
#pragma unroll
            for (int i = 0; i < BN / CG / 64; ++i) ptx::tma_load_3d<CG>(st + kA + i * 8192, &tm_b, &full[s], qrow + 64 * i, r0, part);
          }
          if (++j == p.planes) {
            j = 0;
            r0 += kBox;
          }
          ++filled;
          if (++s == kStages) { s = 0; ph ^= 1; }
        }
      }
      // every stage has been read by the products before the block may leave
      for (uint32_t i = 0; ok && i < kStages && i < filled; ++i) {
        const uint32_t t = filled - 1 - i;  // the fill of that stage; it is released once more than it was before
        if (!ptx::mbar_wait(&empty[t % kStages], (t / kStages) & 1, abort_flag)) ok = false;
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && ptx::elect_one()) {
      const uint32_t idesc = ptx::idesc_bf16(128 * CG, BN, p.a_along_r ? 0 : 1, p.b_along_r ? 0 : 1);
      // along r: rows of 128 bytes, groups of eight 1 KB apart, 16 products = 32 bytes; else atoms of 64 columns 8 KB apart, 16 products = 16 rows
      const uint64_t hi_a = ptx::sdesc_sw128(0, p.a_along_r ? 16 : 8192, 1024), hi_b = ptx::sdesc_sw128(0, p.b_along_r ? 16 : 8192, 1024);
      const uint32_t ka = p.a_along_r ? 2 : 128, kbs = p.b_along_r ? 2 : 128;
      uint32_t s = 0, ph = 0, acc = 0, aph = 0;
      bool ok = true;
      for (int u = first; ok && u < units; u += step) {
        int pt, qt, sp, k0, k1;
        unit_at(p, u, pt, qt, sp);
        k_range(sp, k0, k1);
        for (int kb = k0; ok && kb < k1;) {
          const int end = SEG ? (kb + p.seg < k1 ? kb + p.seg : k1) : k1;
          if (!ptx::mbar_wait(&tempty[acc], aph ^ 1, abort_flag)) { ok = false; break; }
          ptx::tc_fence_after();
          const uint32_t d = tmem + acc * BN;
          uint32_t add = 0;
          auto products = [&](uint32_t a16, uint32_t b16) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              ptx::mma_f16_cg<CG>(d, hi_a | (uint64_t)(a16 + k * ka), hi_b | (uint64_t)(b16 + k * kbs), idesc, add);
              add = 1;
            }
          };
          if (SEG && p.planes == 3) {  // parts l, m, h in three stages, each given back after its last use, in the order they are filled again
            for (; ok && kb < end; kb += 3) {
              uint32_t st[3], at[3];
#pragma unroll
              for (int i = 0; i < 3; ++i) {
                st[i] = s;
                at[i] = ptx::smem_u32(smem + s * kStage) >> 4;
                ok = ok && ptx::mbar_wait(&full[s], ph, abort_flag);
                if (++s == kStages) { s = 0; ph ^= 1; }
              }
              if (!ok) break;
              ptx::tc_fence_after();
              constexpr uint32_t kB16 = kA >> 4;
              products(at[0], at[2] + kB16);  // l h
              products(at[2], at[0] + kB16);  // h l
              ptx::mma_commit_cg<CG>(&empty[st[0]]);
              products(at[1], at[1] + kB16);  // m m
              products(at[2], at[1] + kB16);  // h m
              products(at[1], at[2] + kB16);  // m h
              ptx::mma_commit_cg<CG>(&empty[st[1]]);
              products(at[2], at[2] + kB16);  // h h
              ptx::mma_commit_cg<CG>(&empty[st[2]]);
            }
          } else {
            for (; kb < end; ++kb) {
              if (!ptx::mbar_wait(&full[s], ph, abort_flag)) { ok = false; break; }
              ptx::tc_fence_after();
              const uint32_t a16 = ptx::smem_u32(smem + s * kStage) >> 4;
              products(a16, a16 + (kA >> 4));
              ptx::mma_commit_cg<CG>(&empty[s]);
              if (++s == kStages) { s = 0; ph ^= 1; }
            }
          }
          if (ok) ptx::mma_commit_cg<CG>(&tfull[acc]);
          if (++acc == 2) { acc = 0; aph ^= 1; }
        }
      }
    }
    __syncwarp();
  } else {
    constexpr int CH = 128 / sizeof(T), kChunks = BN / 2 / CH;
    const int w = warp - 2, half = w >> 2, lg = warp & 3;
    WayOut<T> out;
    out.stage_p = staging + w * kTiles<T> * 4096;
    out.stage = ptx::smem_u32(out.stage_p);
    out.rbar = rbars + 2 * w;
    out.rphase = 0;
    out.turn = 0;
    out.lane = lane;
    out.abort_flag = abort_flag;
    uint32_t acc = 0, aph = 0;
    for (int u = first; u < units && !*abort_flag; u += step) {
      int pt, qt, sp, k0, k1;
      unit_at(p, u, pt, qt, sp);
      k_range(sp, k0, k1);
      const int row0 = pt * 128 * CG + (int)rank * 128 + lg * 32, col0 = qt * BN + half * (BN / 2);
      const uint32_t taddr = tmem + ((uint32_t)(lg * 32) << 16) + half * (BN / 2);
      out.fetch(p, &tm_r, out.turn & (kTiles<T> - 1), row0, col0);
      if constexpr (SEG) {
        float sum[BN / 2];
#pragma unroll
        for (int i = 0; i < BN / 2; ++i) sum[i] = 0.f;
        bool ok = true;
        for (int kb = k0; kb < k1; kb += p.seg) {
          ok = ptx::mbar_wait(&tfull[acc], aph, abort_flag);
          if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
          ptx::tc_fence_after();
#pragma unroll
          for (int c = 0; c < BN / 32; ++c) {
            uint32_t v[16];
            ptx::tmem_ld16(taddr + acc * BN + c * 16, v);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[c * 16 + i] += __uint_as_float(v[i]);
          }
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive_rank(&tempty[acc], 0);
          if (++acc == 2) { acc = 0; aph ^= 1; }
        }
        if (!ok) break;
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
          out.put(p, &tm_c, &tm_p, &tm_r, row0, col0 + c * CH, sp, c + 1 < kChunks ? col0 + (c + 1) * CH : p.Q,
                  *reinterpret_cast<float(*)[CH]>(sum + c * CH));
      } else {
        const bool ok = ptx::mbar_wait(&tfull[acc], aph, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) break;
        ptx::tc_fence_after();
#pragma unroll 1
        for (int c = 0; c < kChunks; ++c) {
          uint32_t raw[CH / 32][32];
          float v[CH];
#pragma unroll
          for (int q = 0; q < CH / 32; ++q) ptx::tmem_ld32(taddr + acc * BN + c * CH + q * 32, raw[q]);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < CH; ++i) v[i] = __uint_as_float(raw[i / 32][i % 32]);
          if (c == kChunks - 1) {
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_rank(&tempty[acc], 0);
          }
          out.put(p, &tm_c, &tm_p, &tm_r, row0, col0 + c * CH, sp, c + 1 < kChunks ? col0 + (c + 1) * CH : p.Q, v);
        }
        if (++acc == 2) { acc = 0; aph ^= 1; }
      }
    }
    if (lane == 0) ptx::tma_store_wait_all();
  }

  ptx::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicOr(p.status, NF_ETIMEOUT);
    const unsigned long long t0 = ptx::globaltimer();
    while (ptx::globaltimer() - t0 < 2000000ull) __nanosleep(1000);
  }
  __syncwarp();
  if constexpr (CG == 2) ptx::cluster_sync();  // neither block's memory goes while the other's products or arrivals may use it
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_cg<CG>(tmem, kCols);
  }
}

int make_map3(CUtensorMap* m, const void* base, bool f32, size_t inner, size_t outer, size_t planes, size_t ld, size_t plane, int rows) {
  const size_t es = f32 ? 4 : 2;
  return nf_tc_map3(m, base, f32, inner, outer, planes, ld * es, (planes > 1 ? plane : ld * outer) * es, rows);
}

template <int CG, int BN, typename T, bool SEG>
int launch(const GemmProblem& g, const Epilogue& e, float* part, int splits) {
  GemmParams p{};
  p.P = g.P;
  p.Q = g.Q;
  p.planes = g.planes;
  p.kblocks = (g.R + kBox - 1) / kBox * p.planes;
  p.tiles_p = (g.P + 128 * CG - 1) / (128 * CG);
  p.tiles_q = (g.Q + BN - 1) / BN;
  p.splits = splits;
  // 24 products of 16 (fp32 by parts), or 32, between two readings of an accumulator: errors of 1.6e-7 and 3e-7, the running sum losing about 2^-25 of
  // itself at each.  Twice as many cost fp32 6.6e-7 for 60 us instead of 64 (1777 x 2048 x 1000).
  p.seg = p.planes == 3 ? 3 : sizeof(T) == 4 ? 8 : kSegBf16;
  p.a_along_r = g.A.along_r;
  p.b_along_r = g.B.along_r;
  p.e = e;
  if (splits > 1) p.e.out = part;
  p.tma_out = (size_t)g.Q * sizeof(T) % 16 == 0;
  if (nf_tc_op_status_ptr(&p.status) != NF_OK) return NF_ECUDA;
  CUtensorMap ta, tb, tc, tr, tp;
  auto operand = [&](CUtensorMap* m, const GemmOperand& o, int n, int rows) {
    return o.along_r ? make_map3(m, o.base, false, g.R, n, g.planes, o.ld, o.plane, rows) : make_map3(m, o.base, false, n, g.R, g.planes, o.ld, o.plane, 64);
  };
  int rc = operand(&ta, g.A, g.P, 128);
  if (rc == NF_OK) rc = operand(&tb, g.B, g.Q, BN / CG);
  if (rc == NF_OK) {
    if (p.tma_out) {
      const bool f32 = sizeof(T) == 4;
      rc = make_map3(&tc, p.e.out, f32, g.Q, g.P, splits, g.Q, (size_t)g.P * g.Q, 32);
      tr = tp = tc;
      if (rc == NF_OK && e.residual && splits == 1) rc = make_map3(&tr, e.residual, f32, g.Q, g.P, 1, g.Q, 0, 32);
      if (rc == NF_OK && e.pre && splits == 1) rc = make_map3(&tp, e.pre, f32, g.Q, g.P, 1, g.Q, 0, 32);
    } else {
      tc = tr = tp = ta;  // not used
    }
  }
  if (rc != NF_OK) return rc;
  static bool ready[64];
  int dev = 0;
  NF_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return NF_EUNSUPPORTED;
  auto k = gemm_tc_kernel<CG, BN, T, SEG>;
  if (!ready[dev]) {
    NF_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmem<CG, BN, T>));
    ready[dev] = true;
  }
  const long units = (long)p.tiles_p * p.tiles_q * splits;
  const int most = nf_tc_sm_count() / CG;
  const unsigned grid = (unsigned)((units < most ? units : most) * CG);
  nf_launch_cluster(k, grid, kGemmThreads, kGemmSmem<CG, BN, T>, CG, ta, tb, tc, tr, tp, p);
  NF_LAUNCHED();
  return NF_OK;
}

bool large_tiles(int P, int Q) { return (long)((P + 255) / 256) * ((Q + 255) / 256) >= 56; }

}  // namespace

int nf_gemm_splits(int P, int Q, int R, int planes) {
  if (large_tiles(P, Q)) return 1;
  const long tiles = (long)((P + 127) / 128) * ((Q + 127) / 128);
  long s = 148 / tiles, most = (long)R * (planes == 3 ? 6 : 1) / 1024;  // 16 steps of 64 at least: joining costs a launch and the partial sums' traffic
  if (s > most) s = most;
  if (s > 64) s = 64;
  return s < 1 ? 1 : (int)s;
}

int nf_gemm_tc(const GemmProblem& g, const Epilogue& e, float* part) {
  const long tiles = (long)((g.P + 127) / 128) * ((g.Q + 127) / 128);
  const int splits = nf_gemm_splits(g.P, g.Q, g.R, g.planes);
  if (tiles * splits > 0x3fffffffl) return NF_EUNSUPPORTED;
  const bool f32 = g.out_f32 || splits > 1;
  const bool large = large_tiles(g.P, g.Q), seg = (g.R + kBox - 1) / kBox > kSegBf16;
  if (f32) return large ? launch<2, 256, float, true>(g, e, part, 1) : launch<1, 128, float, true>(g, e, part, splits);
  if (seg) return large ? launch<2, 256, bf16, true>(g, e, part, 1) : launch<1, 128, bf16, true>(g, e, part, splits);
  return large ? launch<2, 256, bf16, false>(g, e, part, 1) : launch<1, 128, bf16, false>(g, e, part, splits);
}
