// 8-bit matrices with a scale for each block of 128 columns, and what a vocabulary head does with them: the norm of the
// backbone's output that leaves in 8 bits, and the product with the vocabulary matrix.
//
// An 8-bit matrix is [rows, ld] e4m3 with ld = K rounded up to 128 (padded with zeros) and [rows, ls] scales, one e8m0 byte a
// block (2^(byte - 127), 255 = NaN), rows padded to a multiple of 4 with 127.  Scales are powers of two: e4m3 is a
// floating format, so a finer scale would not make a value more exact, only keep 0.2 bit more of its range, and the tensor cores apply e8m0
// scales inside the product (kind::mxf8f6f4), without a pass over the accumulators for each block.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ptx.cuh"

namespace csd {

constexpr int kQuantBlock = 128;

// ------------------------------------------------------------------------------------------------------------ the norm
struct QuantRowsParams {
  int rows, K, ld, ls;
  const void* x;
  int64_t ldx;
  const void* residual;   // null: none
  int64_t ldr;
  const void* weight;     // [K], null: ones
  float eps;
  void* sum;              // x + residual, null: not wanted; may be x or residual
  int64_t lds;
  uint8_t *data, *scale;
};

template <typename T> __device__ __forceinline__ T quant_from_float(float v);
template <> __device__ __forceinline__ float quant_from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 quant_from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half quant_from_float<__half>(float v) { return __float2half_rn(v); }

// Eight elements of a row from column `col` on as they lie, zeros behind the row's end.  16-bit rows that are not 16-byte aligned
// are read as aligned vectors too, one more than the elements fill, and shifted (element by element a warp's loads touch every line eight
// times: 154 us against 117 at 8192 x 5001 bf16 with residual; fp32, where the two were 216 and 236 side by side, goes by element: 234 as the kernel stands); so do not pieces that would reach beyond the row.
template <typename T> struct QuantRaw { __align__(16) T e[8]; };
// VEC: K is a multiple of 8 and rows are 16-byte aligned, a piece is a whole one or none.
template <bool VEC, typename T>
__device__ __forceinline__ void quant_load8(const T* row, int col, int K, QuantRaw<T>& v) {
  constexpr int kQ = sizeof(T) / 2;   // 16-byte vectors
  if (VEC) {
#pragma unroll
    for (int i = 0; i < kQ; ++i) reinterpret_cast<uint4*>(v.e)[i] = col < K ? reinterpret_cast<const uint4*>(row + col)[i] : make_uint4(0, 0, 0, 0);
    return;
  }
  const uintptr_t a = reinterpret_cast<uintptr_t>(row + col);
  const int off = static_cast<int>(a & 15);
  uint32_t* out = reinterpret_cast<uint32_t*>(v.e);
  if (off == 0 && col + 8 <= K) {
#pragma unroll
    for (int i = 0; i < kQ; ++i) reinterpret_cast<uint4*>(out)[i] = reinterpret_cast<const uint4*>(row + col)[i];
  } else if (sizeof(T) == 2 && off != 0 && col > 0 && col + 8 + (16 - off) / static_cast<int>(sizeof(T)) <= K) {
    const uint4* b = reinterpret_cast<const uint4*>(a - off);
    __align__(16) uint32_t w[4 * kQ + 4];
#pragma unroll
    for (int i = 0; i <= kQ; ++i) reinterpret_cast<uint4*>(w)[i] = b[i];
    const int sh = (off & 3) * 8;
    auto shift = [&](auto first) {    // (the same for a whole row)
      constexpr int k = decltype(first)::value;
#pragma unroll
      for (int i = 0; i < 4 * kQ; ++i) out[i] = sizeof(T) == 2 && k + i + 1 < 4 * kQ + 4 ? __funnelshift_r(w[k + i], w[k + i + 1], sh) : w[k + i];
    };
    switch (off >> 2) {
      case 0: shift(std::integral_constant<int, 0>()); break;
      case 1: shift(std::integral_constant<int, 1>()); break;
      case 2: shift(std::integral_constant<int, 2>()); break;
      default: shift(std::integral_constant<int, 3>());
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v.e[i] = col + i < K ? row[col + i] : quant_from_float<T>(0.0f);
  }
}
__device__ __forceinline__ void quant_floats(const QuantRaw<float>& v, float* h) {
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = v.e[i];
}
__device__ __forceinline__ void quant_floats(const QuantRaw<__nv_bfloat16>& v, float* h) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(v.e);
#pragma unroll
  for (int i = 0; i < 4; ++i) { h[2 * i] = __uint_as_float(w[i] << 16); h[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void quant_floats(const QuantRaw<__half>& v, float* h) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 f = __half22float2(reinterpret_cast<const __half2*>(v.e)[i]); h[2 * i] = f.x; h[2 * i + 1] = f.y; }
}
__device__ __forceinline__ void quant_round(const float* h, QuantRaw<float>& v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v.e[i] = h[i];
}
__device__ __forceinline__ void quant_round(const float* h, QuantRaw<__nv_bfloat16>& v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) reinterpret_cast<__nv_bfloat162*>(v.e)[i] = __floats2bfloat162_rn(h[2 * i], h[2 * i + 1]);
}
__device__ __forceinline__ void quant_round(const float* h, QuantRaw<__half>& v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) reinterpret_cast<__half2*>(v.e)[i] = __floats2half2_rn(h[2 * i], h[2 * i + 1]);
}
template <bool VEC, typename T>
__device__ __forceinline__ void quant_store8(T* row, int col, int K, const float* h) {
  QuantRaw<T> v;
  quant_round(h, v);
  if (VEC) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) if (col < K) reinterpret_cast<uint4*>(row + col)[i] = reinterpret_cast<uint4*>(v.e)[i];
    return;
  }
  const uintptr_t a = reinterpret_cast<uintptr_t>(row + col);
  if ((a & 15) == 0 && col + 8 <= K) {
    constexpr int kQ = sizeof(T) / 2;
#pragma unroll
    for (int i = 0; i < kQ; ++i) reinterpret_cast<uint4*>(row + col)[i] = reinterpret_cast<uint4*>(v.e)[i];
  } else if (sizeof(T) == 2 && col + 8 <= K) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(v.e);
    if ((a & 3) == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(row + col)[i] = w[i];
    } else {
      row[col] = v.e[0];
#pragma unroll
      for (int i = 0; i < 3; ++i) reinterpret_cast<uint32_t*>(row + col + 1)[i] = __funnelshift_r(w[i], w[i + 1], 16);
      row[col + 7] = v.e[7];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) if (col + i < K) row[col + i] = v.e[i];
  }
}

// Eight values of a block whose largest magnitude has bits `amax`, to e4m3 under the block's scale byte: the smallest power
// of two under which 448 = 1.75 2^8 reaches it (mantissas beyond 1.75 carry into the exponent).  A block with an infinity or a NaN is NaN.
__device__ __forceinline__ uint32_t quant_scale_byte(uint32_t amax) {
  if (amax >= 0x7f800000u) return 255u;
  if (amax == 0u) return 127u;
  const int b = static_cast<int>((amax + 0x1fffffu) >> 23) - 8;
  return b > 0 ? static_cast<uint32_t>(b) : 0u;
}
// the larger one, a NaN if either is
__device__ __forceinline__ float quant_max_nan(float a, float b) { float m; asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b)); return m; }
__device__ __forceinline__ uint2 quant_pack8(const float* v, uint32_t byte) {
  if (byte == 255u) return make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
  const float inv = __uint_as_float((254u - byte) << 23);   // 2^(127 - byte), exact
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(v[4 * i + 1] * inv), "f"(v[4 * i] * inv));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(v[4 * i + 3] * inv), "f"(v[4 * i + 2] * inv));
    w[i] = static_cast<uint32_t>(lo) | (static_cast<uint32_t>(hi) << 16);
  }
  return make_uint2(w[0], w[1]);
}

// Blocks of the most threads that an SM's registers hold.  Four pieces a thread take 112 registers; two of fp32 spill a little at 64, but
// with 104 half as many blocks fit (8192 x 5000: 109 us and 152).
template <typename T, int NCH> constexpr int quant_rows_resident() { return NCH == 1 || NCH == 2 ? 2 : 1; }

// A block takes rows blockIdx.x, + gridDim.x, ...: the next row is requested before this one's reduction, so that its reads are under
// way while the block waits and writes (one block a row, without that: 79 us at 8192 x 5000 bf16 with residual, 63 as it is;
// 288 MB take 44 us at the rate of a copy, instructions bound 16-bit rows: 8192 x 4096 fp32 go at 6.4 TB/s, bf16 at 4.8).  A thread holds NCH pieces of eight columns (NCH = 0: rows too wide for that are read
// twice), 16 lanes a scale block.  Sums and the norm in fp32; the sum leaves rounded to the input's type, the norm uses it unrounded.
template <typename T, int NCH, bool NORM, bool VEC>
__global__ void __launch_bounds__(NCH > 0 ? 512 : 1024, quant_rows_resident<T, NCH>()) quant_rows_kernel(const __grid_constant__ QuantRowsParams p) {
  __shared__ float part[2][32];
  constexpr int kN = NCH > 0 ? NCH : 1;
  const int tid = threadIdx.x, T_ = blockDim.x, pieces = p.ld / 8, lane = tid & 31;
  griddep_enter();
  const T* const wt = static_cast<const T*>(p.weight);
  auto row_x = [&](int64_t r) { return static_cast<const T*>(p.x) + r * p.ldx; };
  auto row_r = [&](int64_t r) { return static_cast<const T*>(p.residual) + r * p.ldr; };
  QuantRaw<T> vx[kN], vr[kN];
  auto fetch = [&](int64_t r, int j, int c) {
    quant_load8<VEC>(row_x(r), c * 8, p.K, vx[j]);
    if (p.residual) quant_load8<VEC>(row_r(r), c * 8, p.K, vr[j]);
  };
  auto take = [&](int j, float* h) {
    quant_floats(vx[j], h);
    if (p.residual) {
      float y[8];
      quant_floats(vr[j], y);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += y[i];
    }
  };
  auto put = [&](int64_t r, int c, float* h, float rstd) {   // (whole groups of 16 lanes are inside or outside)
    if (p.sum) quant_store8<VEC>(static_cast<T*>(p.sum) + r * p.lds, c * 8, p.K, h);
    if (NORM) {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] *= rstd;
      if (wt) {
        QuantRaw<T> w;
        float y[8];
        quant_load8<VEC>(wt, c * 8, p.K, w);
        quant_floats(w, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] *= y[i];
      }
    }
    float big = fabsf(h[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) big = quant_max_nan(big, fabsf(h[i]));
    uint32_t amax = __float_as_uint(big) & 0x7fffffffu;
    const unsigned group = 0xffffu << (lane & 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(group, amax, o));
    const uint32_t byte = quant_scale_byte(amax);
    reinterpret_cast<uint2*>(p.data + r * p.ld)[c] = quant_pack8(h, byte);
    if ((lane & 15) == 0) p.scale[r * p.ls + (c >> 4)] = static_cast<uint8_t>(byte);
  };
  int turn = 0;
  auto finish = [&](float ss) -> float {
    if (!NORM) return 1.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    float* const at = part[turn];
    turn ^= 1;                                   // (two in turn: a warp is at most one row ahead of one that still reads)
    if (lane == 0) at[tid >> 5] = ss;
    __syncthreads();
    ss = lane < (T_ >> 5) ? at[lane] : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    return rsqrtf(ss / static_cast<float>(p.K) + p.eps);
  };
  const int64_t step = gridDim.x;
  int64_t r = blockIdx.x;
  if (NCH > 0) {
#pragma unroll
    for (int j = 0; j < kN; ++j) if (tid + j * T_ < pieces) fetch(r, j, tid + j * T_);
  }
  for (; r < p.rows; r += step) {
    for (int i = p.ld / kQuantBlock + tid; i < p.ls; i += T_) p.scale[r * p.ls + i] = 127;
    float ss = 0.0f;
    if (NCH > 0) {
      float h[kN][8];
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        if (tid + j * T_ < pieces) {
          take(j, h[j]);
#pragma unroll
          for (int i = 0; i < 8; ++i) ss = fmaf(h[j][i], h[j][i], ss);
        }
      }
      if (r + step < p.rows) {
#pragma unroll
        for (int j = 0; j < kN; ++j) if (tid + j * T_ < pieces) fetch(r + step, j, tid + j * T_);
      }
      const float rstd = finish(ss);
#pragma unroll
      for (int j = 0; j < kN; ++j)
        if (tid + j * T_ < pieces) put(r, tid + j * T_, h[j], rstd);
    } else {
      float h[8];
      if (NORM)
        for (int c = tid; c < pieces; c += T_) {
          fetch(r, 0, c); take(0, h);
#pragma unroll
          for (int i = 0; i < 8; ++i) ss = fmaf(h[i], h[i], ss);
        }
      const float rstd = finish(ss);
      for (int c = tid; c < pieces; c += T_) { fetch(r, 0, c); take(0, h); put(r, c, h, rstd); }
    }
  }
}

// --------------------------------------------------------------------------------------------------------- the product
// out[m, n] = sum_k a[m, k] w[n, k], both 8-bit matrices.  The vocabulary matrix is the MMA's M operand (128 rows a
// block: N is never small), the token rows its N operand (a multiple of 32 up to 224, so that two accumulators and the scales
// fit the 512 tensor-memory columns): a single token row costs what reading the weights costs.
// PAIR: two blocks of a cluster share each MMA (256 vocabulary rows, every block loads its own 128 and half of the token rows): a block of its own needs
// 107 B a cycle of operands at 192 token rows, more than an SM takes from L2; in a pair it needs 75.
//   warp 0      requests both operands by TMA, KPS blocks of 128 columns a stage: waiting for a stage and handing it back costs the issuing
//               warp 300 to 500 cycles, about what one block's MMAs take at 192 token rows and several times what they take at 32
//   warp 1      issues the MMAs (of a pair, the leader's): four of K = 32 a block under one scale byte (byte kb % 4 of the scale words)
//   warps 2..5  bring the scales into tensor memory, a word (four blocks) per row: row 32 j + i at lane i, column j, in all
//               four lane quarters; the token rows' scales into both blocks'
//   warps 6..   epilogue: a lane is a vocabulary row, a register a token.  (Two tokens' columns packed to words by an exchange between lanes, for
//               half as many stores, took 119 us where the kernel without it took 90: 576 x 65536 x 2048, bf16, which takes 79 in a short run, 94 under the power cap)
struct QuantMmaParams {
  int M, N, nkb, ls;          // token rows, vocabulary rows, blocks of 128 columns, scale bytes a row
  int bn, stages, sf_col, tmem_cols, tiles_m, tiles;
  const uint8_t *scale_a, *scale_w;
  void* out;
  int64_t ldo;
};
constexpr int kQmEpi = 8;       // epilogue warps (with four the MMAs waited for them where the sums are short: 576 x 65536 x 2048 under the power cap 101 us, 94)
constexpr int kQmThreads = 32 * (6 + kQmEpi);
constexpr int kQmABytes = 128 * kQuantBlock;
constexpr int kQmSfCols = 12;   // 4 of the weights' scales, up to 8 of the tokens'
constexpr int kQmSfRing = 4;    // groups of scales in tensor memory (with two, the MMAs waited a seventh of their time for the next)
constexpr int kQmFixed = 1024 + 256;

// (+)= with e8m0 scales from tensor memory; the scale byte is chosen by the instruction descriptor
template <bool PAIR>
__device__ __forceinline__ void umma_mxf8(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t acc) {
  if (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
        ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(acc), "r"(sfa), "r"(sfb)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
        ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(acc), "r"(sfa), "r"(sfb)
        : "memory");
}
__device__ __forceinline__ void tmem_st4(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
// Arrives on a barrier of a block of the cluster (shared::cluster address); tensor-memory stores before it are complete and fenced.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

template <typename OUT, bool PAIR, int KPS>
__global__ void __launch_bounds__(kQmThreads, 1)
quant_mma_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ QuantMmaParams p, int* err) {
  extern __shared__ uint8_t qm_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(qm_raw) + 1023) & ~uintptr_t(1023));
  const int b_rows = PAIR ? p.bn / 2 : p.bn;                      // token rows that this block loads
  const int block_bytes = kQmABytes + b_rows * kQuantBlock, stage_bytes = KPS * block_bytes, S = p.stages;
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + static_cast<size_t>(S) * stage_bytes);   // [8]
  uint64_t* empty = full + 8;       // [8]
  uint64_t* sf_full = empty + 8;    // [kQmSfRing]
  uint64_t* sf_empty = sf_full + kQmSfRing;
  uint64_t* acc_full = sf_empty + kQmSfRing;   // [2]
  uint64_t* acc_empty = acc_full + 2;  // [2]
  uint32_t* tmem_s = reinterpret_cast<uint32_t*>(acc_empty + 2);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = PAIR ? static_cast<int>(cluster_ctarank()) : 0;
  int* s_abort = reinterpret_cast<int*>(tmem_s + 1);
  if (threadIdx.x == 0) {
    *s_abort = *reinterpret_cast<volatile int*>(err);
    tma_prefetch_desc(&tm_w);
    tma_prefetch_desc(&tm_a);
    for (int s = 0; s < S; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int i = 0; i < kQmSfRing; ++i) { mbar_init(&sf_full[i], PAIR ? 8 : 4); mbar_init(&sf_empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], PAIR ? 2 * kQmEpi : kQmEpi); }
    fence_mbar_init();
  }
  __syncthreads();
  if (PAIR) {                       // both blocks go by what either has seen
    cluster_arrive(); cluster_wait();
    int peer = 0;
    if (threadIdx.x == 0) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(peer) : "r"(mapa_shared(smem_u32(s_abort), static_cast<uint32_t>(rank ^ 1))) : "memory");
    cluster_arrive(); cluster_wait();
    if (threadIdx.x == 0 && peer != 0) *s_abort = peer;
    __syncthreads();
  }
  if (*s_abort != 0) return;
  if (warp == 1) {
    if (PAIR) { tmem_alloc_pair(tmem_s, p.tmem_cols); tmem_relinquish_pair(); }
    else { tmem_alloc(tmem_s, p.tmem_cols); tmem_relinquish(); }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (PAIR) { cluster_arrive(); cluster_wait(); }
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_s;
  griddep_wait();
  if (threadIdx.x == 0) griddep_launch_dependents();
  const int first = PAIR ? blockIdx.x >> 1 : blockIdx.x, step = PAIR ? gridDim.x >> 1 : gridDim.x;
  const int groups = (p.nkb + 3) / 4, nst = (p.nkb + KPS - 1) / KPS;
  constexpr int kRows = PAIR ? 256 : 128;       // vocabulary rows of a tile
  bool ok = true;
  // a wait by a whole warp: one answer for all its lanes
  auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, ch_wait<PAIR>(bar, parity, err)) != 0; };
  if (warp == 0) {
    if (lane == 0) {
      int it = 0;
      for (int t = first; t < p.tiles && ok; t += step) {
        const int n0 = t / p.tiles_m * kRows + rank * 128, m0 = t % p.tiles_m * p.bn + rank * b_rows;
        for (int st = 0; st < nst; ++st, ++it) {
          const int s = it % S, blocks = min(KPS, p.nkb - st * KPS);
          if (it >= S && !ch_wait<PAIR>(&empty[s], ((it / S) & 1) ^ 1, err)) { ch_fail(err, 1, 9, it); ok = false; break; }
          uint8_t* dst = ring + static_cast<size_t>(s) * stage_bytes;
          if (PAIR) {
            // the leader's barrier counts the bytes of both blocks; only the leader arms it
            if (rank == 0) mbar_arrive_expect_tx(&full[s], 2 * blocks * block_bytes);
            const uint32_t lb = mapa_shared(smem_u32(&full[s]), 0);
            for (int k = 0; k < blocks; ++k) {
              tma_load_2d_pair(dst + k * block_bytes, &tm_w, lb, (st * KPS + k) * kQuantBlock, n0);
              tma_load_2d_pair(dst + k * block_bytes + kQmABytes, &tm_a, lb, (st * KPS + k) * kQuantBlock, m0);
            }
          } else {
            mbar_arrive_expect_tx(&full[s], blocks * block_bytes);
            for (int k = 0; k < blocks; ++k) {
              tma_load_2d(dst + k * block_bytes, &tm_w, &full[s], (st * KPS + k) * kQuantBlock, n0);
              tma_load_2d(dst + k * block_bytes + kQmABytes, &tm_a, &full[s], (st * KPS + k) * kQuantBlock, m0);
            }
          }
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      const bool leader = elect_one();
      // e4m3 operands, K-major, fp32 accumulator, e8m0 scales
      const uint32_t idesc = (static_cast<uint32_t>(p.bn >> 3) << 17) | (1u << 23) | (static_cast<uint32_t>(kRows >> 4) << 24);
      int it = 0, g = 0, i = 0;
      for (int t = first; t < p.tiles && ok; t += step, ++i) {
        const int ab = i & 1, use = i >> 1;
        if (use > 0 && !wait(&acc_empty[ab], (use - 1) & 1)) { if (leader) ch_fail(err, 2, 9, i); ok = false; break; }
        tc_fence_after_sync();
        const uint32_t d = tmem + ab * p.bn;
        for (int st = 0; st < nst; ++st, ++it) {
          const int s = it % S;
          if (((st * KPS) & 3) == 0 && !wait(&sf_full[g % kQmSfRing], (g / kQmSfRing) & 1)) { if (leader) ch_fail(err, 2, 10, g); ok = false; break; }
          if (!wait(&full[s], (it / S) & 1)) { if (leader) ch_fail(err, 2, 11, it); ok = false; break; }
          tc_fence_after_sync();
          const int kb0 = st * KPS;
          const bool last = ((kb0 + KPS) & 3) == 0 || st == nst - 1;     // of a group of four blocks
          if (leader) {
            const uint32_t base = smem_u32(ring + static_cast<size_t>(s) * stage_bytes);
            const uint32_t sf = tmem + p.sf_col + (g % kQmSfRing) * kQmSfCols;
#pragma unroll
            for (int j = 0; j < KPS; ++j) {
              const int kb = kb0 + j;
              if (kb >= p.nkb) break;
              const uint64_t da = umma_smem_desc_sw128(base + j * block_bytes), db = umma_smem_desc_sw128(base + j * block_bytes + kQmABytes);
              const uint32_t id = idesc | (static_cast<uint32_t>(kb & 3) << 4) | (static_cast<uint32_t>(kb & 3) << 29);
#pragma unroll
              for (int k = 0; k < 4; ++k) umma_mxf8<PAIR>(d, da + 2 * k, db + 2 * k, id, sf, sf + 4, kb > 0 || k > 0 ? 1u : 0u);
            }
            if (PAIR) { umma_commit_pair(&empty[s]); if (last) umma_commit_pair(&sf_empty[g % kQmSfRing]); }
            else { umma_commit(&empty[s]); if (last) umma_commit(&sf_empty[g % kQmSfRing]); }
          }
          if (last) ++g;
          __syncwarp();
        }
        if (ok && leader) { if (PAIR) umma_commit_pair(&acc_full[ab]); else umma_commit(&acc_full[ab]); }
        __syncwarp();
      }
    }
    __syncwarp();
  } else if (warp < 6) {
    const int q = warp & 3, nb = p.bn / 32;
    // Words of four groups at a time: a row's lie together, and shared memory leaves the L1 cache too little to keep their lines
    // from one group to the next (word by word, these loads took as much from L2 as a third of the operands).
    const bool wide = (p.ls & 15) == 0 && ((reinterpret_cast<uintptr_t>(p.scale_w) | reinterpret_cast<uintptr_t>(p.scale_a)) & 15) == 0;
    int g = 0;
    for (int t = first; t < p.tiles && ok; t += step) {
      const int n0 = t / p.tiles_m * kRows + rank * 128, m0 = t % p.tiles_m * p.bn;
      for (int j4 = 0; j4 < groups && ok; j4 += 4) {
        uint4 w[12];
#pragma unroll
        for (int i = 0; i < 12; ++i) {
          w[i] = make_uint4(0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu);
          const int row = i < 4 ? n0 + 32 * i + lane : m0 + 32 * (i - 4) + lane;
          if (i < 4 ? row < p.N : i - 4 < nb && row < p.M) {
            const uint32_t* src = reinterpret_cast<const uint32_t*>((i < 4 ? p.scale_w : p.scale_a) + static_cast<int64_t>(row) * p.ls) + j4;
            if (wide) w[i] = __ldg(reinterpret_cast<const uint4*>(src));
            else {
              w[i].x = __ldg(src);
              if (j4 + 1 < groups) w[i].y = __ldg(src + 1);
              if (j4 + 2 < groups) w[i].z = __ldg(src + 2);
              if (j4 + 3 < groups) w[i].w = __ldg(src + 3);
            }
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (j4 + k >= groups) break;
          if (g >= kQmSfRing && !wait(&sf_empty[g % kQmSfRing], ((g / kQmSfRing) & 1) ^ 1)) { if (lane == 0) ch_fail(err, 2, 12, g); ok = false; break; }
          tc_fence_after_sync();
          uint32_t x[12];
#pragma unroll
          for (int i = 0; i < 12; ++i) x[i] = k == 0 ? w[i].x : k == 1 ? w[i].y : k == 2 ? w[i].z : w[i].w;
          const uint32_t at = tmem + p.sf_col + (g % kQmSfRing) * kQmSfCols + (static_cast<uint32_t>(q * 32) << 16);
          tmem_st4(at, x);
          tmem_st4(at + 4, x + 4);
          if (nb > 4) tmem_st4(at + 8, x + 8);
          tmem_st_wait();
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) { if (PAIR) mbar_arrive_cluster(mapa_shared(smem_u32(&sf_full[g % kQmSfRing]), 0)); else mbar_arrive(&sf_full[g % kQmSfRing]); }
          ++g;
        }
      }
    }
  } else {
    const int q = warp & 3;
    int i = 0;
    OUT* out = static_cast<OUT*>(p.out);
    for (int t = first; t < p.tiles && ok; t += step, ++i) {
      const int n = t / p.tiles_m * kRows + rank * 128 + q * 32 + lane, m0 = t % p.tiles_m * p.bn;
      const int ab = i & 1, use = i >> 1;
      if (!wait(&acc_full[ab], use & 1)) { if (lane == 0) ch_fail(err, 3, 9, i); ok = false; break; }
      tc_fence_after_sync();
      auto drained = [&]() {                     // this warp has read all it needs: the MMAs may have the accumulator
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) { if (PAIR) mbar_arrive_cluster_tmem(mapa_shared(smem_u32(&acc_empty[ab]), 0)); else mbar_arrive(&acc_empty[ab]); }
      };
      const int c0 = (warp - 6) / 4 * 32;
      if (c0 >= p.bn) drained();
      for (int c = c0; c < p.bn; c += 32 * (kQmEpi / 4)) {
        float v[32];
        tmem_ld32(tmem + ab * p.bn + c + (static_cast<uint32_t>(q * 32) << 16), v);
        tmem_ld_wait();
        if (c + 32 * (kQmEpi / 4) >= p.bn) drained();
        if (n < p.N) {
          OUT* o = out + static_cast<int64_t>(m0 + c) * p.ldo + n;
          const int rows = p.M - m0 - c;
          if (rows >= 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j, o += p.ldo) *o = quant_from_float<OUT>(v[j]);
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j, o += p.ldo) if (j < rows) *o = quant_from_float<OUT>(v[j]);
          }
        }
      }
    }
  }
  if (!ok) settle();   // copies that nobody waits for any more
  __syncthreads();
  if (PAIR) { cluster_arrive(); cluster_wait(); }   // neither block leaves (or frees its columns) while the other's MMAs or arrivals may still reach it
  tc_fence_after_sync();
  if (warp == 1) { if (PAIR) tmem_dealloc_pair(tmem, p.tmem_cols); else tmem_dealloc(tmem, p.tmem_cols); }
}

}  // namespace csd
