// Categorical (vocabulary) heads: draft sampling, verification and resampling where p and q are explicit distributions over
// V tokens, the case continuous speculative decoding generalises (accept rule of Sec. 3.1, modified distribution of Eq. 5).
//
// A row's distribution is softmax(logits / temperature) restricted to its kept tokens: top-k, of these the shortest prefix in
// the order (value descending, index ascending) whose weight reaches top_p of theirs, of these all at least min_p times as
// likely as the likeliest.  All three are prefixes of one order, so the kept set is "at or before one element" (its cut) and a
// row's distribution is five numbers (kCatRow): log normaliser, cut value, highest index kept among equals of the cut, count,
// reciprocal temperature.
//
// Weights are 64-bit fixed point (2^-44 of the row's largest), formed in fp64 from scaled logits rounded once to fp32:
// integer sums do not depend on the order, so a cut or a token does not depend on how a row is spread over blocks, and the error of a
// prefix sum stays below 2^-36: which of 10^5 tokens straddles top_p or u is decided as in 64-bit arithmetic.  (With fp32 weights one
// flat row of 131072 tokens in a hundred had another count.)
//
// One cluster of 1 to 8 blocks carries a row; every pass reads the row again (DRAM the first time, L2 after): a pass from L2 costs
// about what one from shared memory would, and V is not bounded by it.
#pragma once
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <stdint.h>

#include "ptx.cuh"

namespace csd {
namespace cg = cooperative_groups;
typedef unsigned long long u64;

constexpr int kCatThreads = 512;
constexpr int kCatWarps = kCatThreads / 32;
constexpr int kCatBins = 2048;        // bins of the first histogram: 1/64 of scaled logit each, 32 below the largest
constexpr float kCatPerUnit = 64.0f;
constexpr int kCatList = 2048;        // candidates that are sorted
constexpr int kCatSub = 1024;         // bins of a refinement
constexpr int kCatSegs = 8;           // pieces of a warp's part whose sums are kept, of at least kCatUnroll rounds
constexpr int kCatPairs = 256;        // kept tokens up to which a token is found by comparing all pairs
constexpr int kCatRow = 5;            // doubles of a row's summary
constexpr int kCatMaxCluster = 8;
constexpr double kLog2e = 1.4426950408889634074;
constexpr float kCatFar = 30.5f;      // further below the largest a weight is less than 2^-44: 0

struct CatView {
  const void* data;
  int64_t ld;      // elements from row to row
};

// ------------------------------------------------------------------------------------------------ elements of a row
template <typename T> struct CatType;
template <> struct CatType<float> {
  static constexpr int kVec = 4;
  static __device__ __forceinline__ uint32_t masked() { return 0xff800000u; }
  static __device__ __forceinline__ void unpack(const uint4& r, float* l) {
    l[0] = __uint_as_float(r.x); l[1] = __uint_as_float(r.y); l[2] = __uint_as_float(r.z); l[3] = __uint_as_float(r.w);
  }
};
template <> struct CatType<__nv_bfloat16> {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ uint32_t masked() { return 0xff80ff80u; }
  static __device__ __forceinline__ void unpack(const uint4& r, float* l) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { l[2 * i] = __uint_as_float(w[i] << 16); l[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
};
template <> struct CatType<__half> {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ uint32_t masked() { return 0xfc00fc00u; }
  static __device__ __forceinline__ void unpack(const uint4& r, float* l) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      l[2 * i] = f.x; l[2 * i + 1] = f.y;
    }
  }
};
template <typename T> __device__ __forceinline__ float cat_float(T v) { return static_cast<float>(v); }
template <> __device__ __forceinline__ float cat_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float cat_float<__half>(__half v) { return __half2float(v); }

// Scaled logit: -inf where masked (-inf or NaN), finite elsewhere (a mask of the type's lowest value is an ordinary, hopeless logit).
__device__ __forceinline__ float cat_scale(float l, float inv_t) {
  const float t = fminf(fmaxf(__fmul_rn(l, inv_t), -FLT_MAX), FLT_MAX);
  return l > -INFINITY ? t : -INFINITY;
}

// A row as 16-byte vectors of its aligned memory: virtual element v is index v - head.  Vectors across the row's ends are read by element.
template <typename T> struct CatRow {
  static constexpr int kVec = CatType<T>::kVec;
  const T* base;   // aligned down to 16 bytes
  int head, V;
  __device__ __forceinline__ CatRow(const CatView& m, int64_t row, int V_) : V(V_) {
    const T* p = static_cast<const T*>(m.data) + row * m.ld;
    head = static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    base = p - head;
  }
  __device__ __forceinline__ int vecs() const { return (head + V + kVec - 1) / kVec; }
  __device__ __forceinline__ uint4 load(int v) const {
    const int first = v * kVec - head;
    if (first >= 0 && first + kVec <= V) return __ldg(reinterpret_cast<const uint4*>(base) + v);
    const uint32_t mk = CatType<T>::masked();
    uint4 r = make_uint4(mk, mk, mk, mk);
    __align__(16) T e[kVec];
    *reinterpret_cast<uint4*>(e) = r;
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (first + i >= 0 && first + i < V) e[i] = base[static_cast<int64_t>(v) * kVec + i];
    return *reinterpret_cast<uint4*>(e);
  }
};

constexpr int kCatUnroll = 4;
// This warp's part of the row: `iters` rounds of 32 vectors, parts in index order over the warps of the cluster; `len` rounds a piece.
struct CatPart {
  int first, iters, len, vecs;
  template <typename T> __device__ __forceinline__ CatPart(const CatRow<T>& r, int cs, int rank) : vecs(r.vecs()) {
    const int warps = cs * kCatWarps;
    iters = ((vecs + warps - 1) / warps + 31) / 32;
    first = (rank * kCatWarps + (threadIdx.x >> 5)) * iters * 32;
    len = max(kCatUnroll, (iters + kCatSegs - 1) / kCatSegs);
  }
};

// f(scaled logits of a vector's elements, index of the first of them) for every vector of rounds [from, to); elements outside the row are masked.
template <typename T, typename F>
__device__ __forceinline__ void cat_each(const CatRow<T>& row, const CatPart& part, float inv_t, int from, int to, F f) {
  constexpr int kVec = CatRow<T>::kVec;
  const int lane = threadIdx.x & 31;
  for (int it = from; it < to; it += kCatUnroll) {
    uint4 raw[kCatUnroll];
#pragma unroll
    for (int j = 0; j < kCatUnroll; ++j) {
      const int v = part.first + (it + j) * 32 + lane;
      if (it + j < to && v < part.vecs) raw[j] = row.load(v);
      else { const uint32_t mk = CatType<T>::masked(); raw[j] = make_uint4(mk, mk, mk, mk); }
    }
#pragma unroll
    for (int j = 0; j < kCatUnroll; ++j) {
      if (it + j >= to) break;
      float t[kVec];
      CatType<T>::unpack(raw[j], t);
#pragma unroll
      for (int i = 0; i < kVec; ++i) t[i] = cat_scale(t[i], inv_t);
      f(t, (part.first + (it + j) * 32 + lane) * kVec - row.head);
    }
  }
}

// ------------------------------------------------------------------------------------------------------ arithmetic
// Order of the tokens as one ascending key: value descending, then index.
__device__ __forceinline__ uint32_t cat_ord(float t) {
  const uint32_t b = __float_as_uint(t + 0.0f);   // -0 and 0 are equals
  return b & 0x80000000u ? b : 0x7fffffffu - b;
}
__device__ __forceinline__ u64 cat_key(float t, int idx) { return (static_cast<u64>(cat_ord(t)) << 32) | static_cast<uint32_t>(idx); }
__device__ __forceinline__ float cat_key_value(u64 k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o : 0x7fffffffu - o);
}

// 2^(t log2(e) + c) in fp64: 16 table values of 2^(j/16) and the Taylor polynomial of degree 5 on [-1/32, 1/32]
// (remainder 2^-42.6).  16 doubles lie in 16 different pairs of banks: lookups do not conflict.
__device__ __forceinline__ double cat_exp(float t, double c, const double* tab) {
  constexpr double kRound = 6755399441055744.0 / 16;   // 1.5 2^52 / 16: rounds to a multiple of 1/16
  const double y = fma(static_cast<double>(t), kLog2e, c);
  const double z = y + kRound;
  const double r = y - (z - kRound);
  const int k = __double2loint(z);
  constexpr double l = 0.69314718055994530942;
  double p = l * l * l * l * l / 120;
  p = fma(p, r, l * l * l * l / 24);
  p = fma(p, r, l * l * l / 6);
  p = fma(p, r, l * l / 2);
  p = fma(p, r, l);
  const double b = tab[k & 15];
  const double v = fma(b * r, p, b);
  return __hiloint2double(__double2hiint(v) + ((k >> 4) << 20), __double2loint(v));
}
__device__ __forceinline__ void cat_table(double* tab) {
  if (threadIdx.x < 16) tab[threadIdx.x] = exp2(threadIdx.x / 16.0);
}
// Weight relative to the largest scaled logit m (c = -m log2(e)): 2^44 exp(t - m), rounded; at most a few units above 2^44.
__device__ __forceinline__ u64 cat_weight(float t, float m, double c, const double* tab) {
  if (!(m - t <= kCatFar)) return 0;
  return static_cast<u64>(__double_as_longlong(cat_exp(t, c, tab) + 256.0) - __double_as_longlong(256.0));
}

template <typename X> __device__ __forceinline__ X cat_warp_sum(X v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Inclusive sum over the block's threads (exclusive = inclusive - v); part: kCatWarps values of shared memory.
template <typename X> __device__ __forceinline__ X cat_block_scan(X v, X* part, X* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const X w = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += w; }
  __syncthreads();
  if (lane == 31) part[warp] = v;
  __syncthreads();
  X before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kCatWarps; ++i) { const X w = part[i]; if (i < warp) before += w; all += w; }
  *total = all;
  return v + before;
}

// ---------------------------------------------------------------------------------------------------- shared memory
struct CatShared {
  uint32_t hist[kCatBins];
  u64 list[kCatList];                       // candidates; a refinement's weights
  u64 seg[kCatWarps * kCatSegs];            // sums of the pieces of the warps' parts
  u64 red[2][kCatWarps][3];                 // reductions over the cluster, two in turn
  u64 scan[kCatWarps];
  double scan_d[kCatWarps];
  double tab[16];
  float maxima[kCatWarps];
  // found by one thread, read by all (of the cluster: rank 0's)
  u64 found_key, found_sum;
  u64 found_count;
  int found_a, found_b, found_n, found_seg;
  uint32_t list_n;
};

struct CatParams {
  int R, V;
  CatView logits;
  const float* temperature;   // [R] or null: 1
  const int32_t* top_k;       // [R] or null
  const float *top_p, *min_p; // [R] or null
  const float* u;             // [R] or null: no token is drawn
  int32_t* token;             // [R]
  float* logp;                // [R] or null
  double* dist;               // [R, 5] or null
};

// Blocks of a row's cluster and the reductions between them.
struct CatTeam {
  cg::cluster_group cl;
  int cs, rank, turn;
  CatShared& sh;
  __device__ __forceinline__ explicit CatTeam(CatShared& s) : cl(cg::this_cluster()), cs(cl.num_blocks()), rank(cl.block_rank()), turn(0), sh(s) {}
  __device__ __forceinline__ void sync() { if (cs == 1) __syncthreads(); else cl.sync(); }
  template <typename X> __device__ __forceinline__ X* at(X* p, int r) { return cs == 1 ? p : cl.map_shared_rank(p, r); }
  // sums (a, b) and the maximum (c) over all threads of the cluster.  Slots are used in turn: a block is at most one
  // reduction ahead of a block that still reads.
  __device__ __forceinline__ void reduce(u64& a, u64& b, u64& c) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    a = cat_warp_sum(a); b = cat_warp_sum(b);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) { const u64 w = __shfl_xor_sync(0xffffffffu, c, o); c = w > c ? w : c; }
    u64 (*slot)[3] = sh.red[turn];
    turn ^= 1;
    if (lane == 0) { slot[warp][0] = a; slot[warp][1] = b; slot[warp][2] = c; }
    sync();
    u64 x = 0, y = 0, z = 0;
    for (int i = lane; i < cs * kCatWarps; i += 32) {
      const u64* p = at(&slot[i % kCatWarps][0], i / kCatWarps);
      x += p[0]; y += p[1]; z = p[2] > z ? p[2] : z;
    }
    a = cat_warp_sum(x); b = cat_warp_sum(y); c = z;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) { const u64 w = __shfl_xor_sync(0xffffffffu, c, o); c = w > c ? w : c; }
  }
};

// Sorts list[0, n) ascending (bitonic; padded to a power of two).  Steps within 64 neighbours stay in one warp.
__device__ __forceinline__ void cat_sort(u64* list, int n) {
  int P = 64;
  while (P < n) P <<= 1;
  for (int i = n + static_cast<int>(threadIdx.x); i < P; i += kCatThreads) list[i] = ~0ull;
  __syncthreads();
  for (int size = 2; size <= P; size <<= 1)
    for (int stride = size >> 1; stride > 0; stride >>= 1) {
      for (int i = threadIdx.x; i < P / 2; i += kCatThreads) {
        const int a = (i / stride) * 2 * stride + i % stride, b = a + stride;
        const u64 x = list[a], y = list[b];
        const bool up = (a & size) == 0;
        if ((x > y) == up) { list[a] = y; list[b] = x; }
      }
      if (stride > 32 || (stride == 1 && size >= 64)) __syncthreads(); else __syncwarp();
    }
  __syncthreads();
}

// ---------------------------------------------------------------------------------------------------- finding a token
// The token at which the cumulative weight reaches target: sums of the pieces of all warps' parts are in every block's
// sh.seg; the warp that owns the piece goes through it again.  weight(t, idx) as in the pass that formed the sums.
template <typename T, typename W>
__device__ __forceinline__ void cat_locate(CatTeam& team, const CatRow<T>& row, const CatPart& part, float inv_t, u64 target, W weight, int* token) {
  CatShared& sh = team.sh;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kVec = CatRow<T>::kVec;
  team.sync();                                     // the pieces' sums are written
  const int pieces = team.cs * kCatWarps * kCatSegs;   // at most 1024: two a thread
  const int each = (pieces + kCatThreads - 1) / kCatThreads;
  if (team.rank == 0) {
    u64 s[2] = {0, 0};
    for (int j = 0; j < each; ++j) {
      const int i = threadIdx.x * each + j;
      if (i < pieces) s[j] = *team.at(&sh.seg[i % (kCatWarps * kCatSegs)], i / (kCatWarps * kCatSegs));
    }
    u64 total;
    u64 before = cat_block_scan<u64>(s[0] + s[1], sh.scan, &total) - s[0] - s[1];
    for (int j = 0; j < each; ++j) {
      if (before < target && before + s[j] >= target) { sh.found_seg = threadIdx.x * each + j; sh.found_sum = before; }
      before += s[j];
    }
  }
  team.sync();
  const int piece = *team.at(&sh.found_seg, 0);
  u64 before = *team.at(&sh.found_sum, 0);
  if (piece / kCatSegs == team.rank * kCatWarps + warp) {
    const int from = (piece % kCatSegs) * part.len, to = min(from + part.len, part.iters);
    bool done = false;
    for (int it = from; it < to && !done; ++it) {
      cat_each(row, part, inv_t, it, it + 1, [&](const float* t, int idx) {
        u64 w[kVec], s = 0;
#pragma unroll
        for (int i = 0; i < kVec; ++i) { w[i] = weight(t[i], idx + i); s += w[i]; }
        u64 incl = s;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const u64 x = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += x; }
        u64 at = before + incl - s;
        if (at < target && at + s >= target) {
#pragma unroll
          for (int i = 0; i < kVec; ++i) { if (at < target && at + w[i] >= target) *token = idx + i; at += w[i]; }
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
        done = before >= target;
      });
    }
  }
}

// One pass that leaves the sums of the warps' pieces in sh.seg; f(t, idx) gives an element's weight.
template <typename T, typename F>
__device__ __forceinline__ u64 cat_sums(CatTeam& team, const CatRow<T>& row, const CatPart& part, float inv_t, F f) {
  constexpr int kVec = CatRow<T>::kVec;
  u64 all = 0;
  for (int s = 0; s < kCatSegs; ++s) {
    u64 sum = 0;
    cat_each(row, part, inv_t, s * part.len, min((s + 1) * part.len, part.iters), [&](const float* t, int idx) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) sum += f(t[i], idx + i);
    });
    all += sum;
    sum = cat_warp_sum(sum);
    if ((threadIdx.x & 31) == 0) team.sh.seg[(threadIdx.x >> 5) * kCatSegs + s] = sum;
  }
  return all;
}

// The weight that top-p asks for (the likeliest token is kept whatever it asks).
__device__ __forceinline__ double cat_limit(float top_p, u64 total) { return fmax(static_cast<double>(top_p) * static_cast<double>(total), 1.0); }
__device__ __forceinline__ u64 cat_target(float u, u64 total) {
  const double x = ceil(static_cast<double>(u) * static_cast<double>(total));
  u64 t = x >= 1.0 ? static_cast<u64>(x) : 1;
  return t > total ? total : t;
}

// ----------------------------------------------------------------------------------------------------- refinement
// The last element kept, where more elements than the list holds come into question: the first element in key order at which the
// running count reaches `count` (BY_WEIGHT: the running weight reaches `limit`) among keys <= last.  [a, b] should hold it.
template <bool BY_WEIGHT, typename T>
__device__ __forceinline__ u64 cat_refine(CatTeam& team, const CatRow<T>& row, const CatPart& part, float inv_t, float m, double c,
                                          u64 a, u64 b, u64 last, u64 count, double limit) {
  CatShared& sh = team.sh;
  constexpr int kVec = CatRow<T>::kVec;
  const int tid = threadIdx.x;
  for (;;) {
    const int top = 64 - __clzll(static_cast<long long>(b - a | 1));
    const int shift = top > 10 ? top - 10 : 0;
    team.sync();                                   // nobody reads the arrays below any more
    for (int i = tid; i < kCatSub; i += kCatThreads) { sh.hist[i] = 0; sh.list[i] = 0; }
    if (tid == 0) sh.list_n = 0;
    __syncthreads();
    u64 n_before = 0, w_before = 0, none = 0;
    cat_each(row, part, inv_t, 0, part.iters, [&](const float* t, int idx) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const u64 key = cat_key(t[i], idx + i);
        if (!(t[i] > -INFINITY) || key > b || key > last) continue;
        const u64 w = BY_WEIGHT ? cat_weight(t[i], m, c, sh.tab) : 0;
        if (key < a) { ++n_before; w_before += w; }
        else {
          const int s = static_cast<int>((key - a) >> shift);
          atomicAdd(&sh.hist[s], 1u);
          if (BY_WEIGHT) atomicAdd(&sh.list[s], w);
        }
      }
    });
    team.reduce(n_before, w_before, none);         // (also orders the histograms' additions before the reads below)
    uint32_t n[2];
    u64 w[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      n[j] = 0; w[j] = 0;
      for (int r = 0; r < team.cs; ++r) {
        n[j] += *team.at(&sh.hist[tid * 2 + j], r);
        if (BY_WEIGHT) w[j] += *team.at(&sh.list[tid * 2 + j], r);
      }
    }
    u64 all_n, all_w = 0;
    u64 pn = cat_block_scan<u64>(n[0] + n[1], sh.scan, &all_n) - n[0] - n[1] + n_before;
    u64 pw = w_before;
    if (BY_WEIGHT) pw += cat_block_scan<u64>(w[0] + w[1], sh.scan, &all_w) - w[0] - w[1];
    auto reached = [&](u64 cn, u64 cw) { return BY_WEIGHT ? static_cast<double>(cw) >= limit : cn >= count; };
    if (reached(n_before, w_before)) { b = a - 1; a = 0; continue; }        // not in [a, b]: before it
    if (!reached(n_before + all_n, w_before + all_w)) {                     // behind it
      if (b >= last) return last;
      a = b + 1; b = last;
      continue;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (!reached(pn, pw) && reached(pn + n[j], pw + w[j])) { sh.found_a = tid * 2 + j; sh.found_n = static_cast<int>(n[j]); sh.found_count = pn; sh.found_sum = pw; }
      pn += n[j]; pw += w[j];
    }
    __syncthreads();
    a += static_cast<u64>(sh.found_a) << shift;
    const u64 span = (1ull << shift) - 1;
    b = b - a > span ? a + span : b;
    const int inside = sh.found_n;
    pn = sh.found_count; pw = sh.found_sum;
    if (inside > kCatList) continue;
    // few enough: sorted by the first block
    team.sync();
    cat_each(row, part, inv_t, 0, part.iters, [&](const float* t, int idx) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const u64 key = cat_key(t[i], idx + i);
        if (t[i] > -INFINITY && key >= a && key <= b && key <= last) team.at(sh.list, 0)[atomicAdd(team.at(&sh.list_n, 0), 1u)] = key;
      }
    });
    team.sync();
    if (team.rank == 0) {
      cat_sort(sh.list, inside);
      if (!BY_WEIGHT) {
        if (tid == 0) sh.found_key = sh.list[count - pn - 1];
      } else {
        constexpr int kEach = kCatList / kCatThreads;
        u64 lw[kEach], s = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          const int i = tid * kEach + j;
          lw[j] = i < inside ? cat_weight(cat_key_value(sh.list[i]), m, c, sh.tab) : 0;
          s += lw[j];
        }
        u64 total;
        u64 before = cat_block_scan<u64>(s, sh.scan, &total) - s + pw;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          const int i = tid * kEach + j;
          if (i < inside && !reached(0, before) && reached(0, before + lw[j])) sh.found_key = sh.list[i];
          before += lw[j];
        }
      }
    }
    team.sync();
    return *team.at(&sh.found_key, 0);
  }
}

// ------------------------------------------------------------------------------------------- summary of a row, and a token
__device__ __forceinline__ int cat_bin(float m, float t) {   // kCatBins and more: below every bin
  const float x = fminf((m - t) * kCatPerUnit, 4095.0f);
  return __float2int_rd(x);
}

template <typename T>
__global__ void __launch_bounds__(kCatThreads, 2) cat_filter_kernel(const CatParams p) {
  __shared__ CatShared sh;
  CatTeam team(sh);
  const int tid = threadIdx.x;
  constexpr int kVec = CatRow<T>::kVec;
  const int64_t r = blockIdx.x / team.cs;
  griddep_enter();
  const float temp = p.temperature ? p.temperature[r] : 1.0f;
  const bool greedy = !(temp > 0.0f);
  const float inv_t = greedy ? 1.0f : __fdiv_rn(1.0f, temp);
  const int want = greedy ? 1 : (p.top_k ? p.top_k[r] : 0);
  const u64 k = want > 0 && want < p.V ? static_cast<u64>(want) : static_cast<u64>(p.V);
  const float tp = p.top_p ? p.top_p[r] : 1.0f, mp = p.min_p ? p.min_p[r] : 0.0f;
  const bool by_k = k < static_cast<u64>(p.V), by_p = tp < 1.0f && !greedy;
  const double min_d = mp > 0.0f ? log(static_cast<double>(fminf(mp, 1.0f))) : -INFINITY;   // kept: t - m >= min_d
  const CatRow<T> row(p.logits, r, p.V);
  const CatPart part(row, team.cs, team.rank);

  // the largest scaled logit: scaling is monotonic, so it is the largest logit's
  cat_table(sh.tab);
  for (int i = tid; i < kCatBins; i += kCatThreads) sh.hist[i] = 0;
  if (tid == 0) sh.list_n = 0;
  float m = -INFINITY;
  cat_each(row, part, inv_t, 0, part.iters, [&](const float* t, int) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) m = fmaxf(m, t[i]);
  });
  {
    u64 x = 0, y = 0, z = ~static_cast<u64>(cat_ord(m));   // ascending in m
    team.reduce(x, y, z);
    const u64 o = ~z;
    m = cat_key_value(o << 32);
  }
  double* dist = p.dist ? p.dist + r * kCatRow : nullptr;
  if (!(m > -INFINITY)) {   // nothing is left
    if (team.rank == 0 && tid == 0) {
      if (dist) { dist[0] = -INFINITY; dist[1] = INFINITY; dist[2] = -1.0; dist[3] = 0.0; dist[4] = inv_t; }
      if (p.u) { p.token[r] = -1; if (p.logp) p.logp[r] = -INFINITY; }
    }
    team.sync();
    return;
  }
  const double md = m, c = -md * kLog2e;
  auto weight = [&](float t) { return cat_weight(t, m, c, sh.tab); };
  auto likely = [&](float t) { return static_cast<double>(t) - md >= min_d; };

  u64 cut = ~0ull;          // last key kept by top-k and top-p
  bool listed = false;      // the kept tokens are the first of the first block's sorted list
  u64 kept_n = 0, kept_w = 0, kept_last = 0;
  if (by_k || by_p) {
    // counts by distance from the largest, and the sum of all weights where top-p refers to it
    const bool with_sum = by_p && k > kCatList / 2;
    u64 live = 0, sum = 0, none = 0;
    cat_each(row, part, inv_t, 0, part.iters, [&](const float* t, int) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        if (!(t[i] > -INFINITY)) continue;
        ++live;
        const int b = cat_bin(m, t[i]);
        if (b < kCatBins) atomicAdd(&sh.hist[b], 1u);
        if (with_sum) sum += weight(t[i]);
      }
    });
    team.reduce(live, sum, none);
    const bool k_counts = by_k && k < live;
    const bool p_all = by_p && !k_counts && with_sum;   // top-p refers to the whole row, whose sum is known
    // the bin where the count reaches k, or the bins between which the weight reaches top_p of the sum
    uint32_t n[4] = {0, 0, 0, 0};
    for (int q = 0; q < team.cs; ++q) {
      const uint4 h = *reinterpret_cast<const uint4*>(team.at(&sh.hist[tid * 4], q));
      n[0] += h.x; n[1] += h.y; n[2] += h.z; n[3] += h.w;
    }
    u64 binned;
    u64 cum = cat_block_scan<u64>(static_cast<u64>(n[0]) + n[1] + n[2] + n[3], sh.scan, &binned) - n[0] - n[1] - n[2] - n[3];
    double e[4], es = 0.0, et;
    const double limit = cat_limit(tp, sum);
#pragma unroll
    for (int j = 0; j < 4; ++j) { e[j] = n[j] * static_cast<double>(exp2f(-static_cast<float>(kLog2e) * (tid * 4 + j + 0.5f) / kCatPerUnit)); es += e[j]; }
    double mass = cat_block_scan<double>(es, sh.scan_d, &et) - es;
    if (tid == 0) { sh.found_a = kCatBins; sh.found_b = kCatBins; sh.found_n = 0; }
    __syncthreads();
    // a bin's weight lies within exp(+-1/128) of its count times its middle's weight (and what rounding adds)
    const double unit = 17592186044416.0;   // 2^44
    const double lo = unit * 0.99221 * 0.99999, hi = unit * 1.00785 * 1.00001;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int b = tid * 4 + j;
      if (k_counts) {
        if (cum < k && cum + n[j] >= k) { sh.found_a = b; sh.found_b = b; sh.found_n = static_cast<int>(min(cum + n[j], static_cast<u64>(INT_MAX))); }
      } else if (p_all) {
        if (mass * hi < limit && (mass + e[j]) * hi >= limit) sh.found_a = b;
        if (mass * lo < limit && (mass + e[j]) * lo >= limit) { sh.found_b = b; sh.found_n = static_cast<int>(min(cum + n[j], static_cast<u64>(INT_MAX))); }
      }
      cum += n[j]; mass += e[j];
    }
    __syncthreads();
    int bin_a = sh.found_a, bin_b = sh.found_b;
    int upto = sh.found_n;
    if (!k_counts && !p_all && live <= kCatList) { bin_b = 4096; upto = static_cast<int>(live); }   // all of them, sorted
    const bool found = bin_b != kCatBins;
    if (found && upto <= kCatList) {
      listed = true;
      cat_each(row, part, inv_t, 0, part.iters, [&](const float* t, int idx) {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
          if (t[i] > -INFINITY && cat_bin(m, t[i]) <= bin_b) team.at(sh.list, 0)[atomicAdd(team.at(&sh.list_n, 0), 1u)] = cat_key(t[i], idx + i);
      });
      team.sync();
      if (team.rank == 0) {
        cat_sort(sh.list, upto);
        constexpr int kEach = kCatList / kCatThreads;
        u64 lw[kEach], s = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          const int i = tid * kEach + j;
          lw[j] = i < upto ? weight(cat_key_value(sh.list[i])) : 0;
          s += lw[j];
        }
        u64 total;
        const u64 start = cat_block_scan<u64>(s, sh.scan, &total) - s;
        const int most = static_cast<int>(k_counts ? k : min(live, static_cast<u64>(upto)));
        u64 before = start;
        if (tid == 0) sh.found_sum = total;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kEach; ++j) { before += lw[j]; if (k_counts && tid * kEach + j == most - 1) sh.found_sum = before; }
        __syncthreads();
        const double lim = by_p ? (p_all ? limit : cat_limit(tp, sh.found_sum)) : INFINITY;
        before = start;
        int mine = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          const int i = tid * kEach + j;
          mine += i < most && (i == 0 || (static_cast<double>(before) < lim && likely(cat_key_value(sh.list[i]))));
          before += lw[j];
        }
        u64 all;
        cat_block_scan<u64>(static_cast<u64>(mine), sh.scan, &all);
        const int last = static_cast<int>(all) - 1;
        before = start;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          before += lw[j];
          if (tid * kEach + j == last) { sh.found_key = sh.list[last]; sh.found_count = all; sh.found_sum = before; }
        }
      }
      team.sync();
      cut = *team.at(&sh.found_key, 0);
      kept_n = *team.at(&sh.found_count, 0);
      kept_w = *team.at(&sh.found_sum, 0);
      kept_last = cut;
    } else {
      // many candidates (wide top-k, flat distributions, many equals)
      auto edge_a = [&](int b) { return b <= 0 ? 0ull : cat_key(nextafterf(nextafterf(m - (b - 0.02f) / kCatPerUnit, INFINITY), INFINITY), 0); };
      auto edge_b = [&](int b) { return b >= kCatBins - 1 ? ~0ull : cat_key(nextafterf(nextafterf(m - (b + 1.02f) / kCatPerUnit, -INFINITY), -INFINITY), -1); };
      if (k_counts) {
        cut = cat_refine<false>(team, row, part, inv_t, m, c, edge_a(bin_a), edge_b(bin_b), ~0ull, k, 0.0);
        bin_a = 0;
      }
      if (by_p) {
        u64 w = sum;
        if (k_counts || !with_sum) {
          u64 x = 0, y = 0;
          w = 0;
          cat_each(row, part, inv_t, 0, part.iters, [&](const float* t, int idx) {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
              if (t[i] > -INFINITY && cat_key(t[i], idx + i) <= cut) w += weight(t[i]);
          });
          team.reduce(w, x, y);
        }
        const u64 a = p_all ? edge_a(bin_a) : 0;
        u64 b = p_all ? edge_b(bin_b) : cut;
        b = b < cut ? b : cut;
        cut = cat_refine<true>(team, row, part, inv_t, m, c, a < b ? a : 0, b, cut, 0, cat_limit(tp, w));
      }
    }
  }
  auto kept_weight = [&](float t, int idx) -> u64 { return t > -INFINITY && cat_key(t, idx) <= cut && likely(t) ? weight(t) : 0; };
  const bool pairs = listed && kept_n <= kCatPairs;
  if (!listed || (p.u && !pairs)) {
    u64 n = 0, last = 0;
    u64 w = cat_sums(team, row, part, inv_t, [&](float t, int idx) -> u64 {
      if (!(t > -INFINITY)) return 0;
      const u64 key = cat_key(t, idx);
      if (key > cut || !likely(t)) return 0;
      ++n;
      last = key > last ? key : last;
      return weight(t);
    });
    team.reduce(w, n, last);
    kept_n = n; kept_w = w; kept_last = last;
  }
  const double norm = md + log(static_cast<double>(kept_w)) - 44.0 * 0.69314718055994530942;
  if (team.rank == 0 && tid == 0 && dist) {
    dist[0] = norm; dist[1] = cat_key_value(kept_last); dist[2] = static_cast<double>(static_cast<uint32_t>(kept_last)); dist[3] = static_cast<double>(kept_n); dist[4] = inv_t;
  }
  if (p.u) {
    const u64 target = cat_target(p.u[r], kept_w);
    int found = -1;
    if (pairs) {
      if (team.rank == 0) {
        const int n = static_cast<int>(kept_n);
        __syncthreads();
        u64* w = sh.list + kCatList - kCatPairs;   // (the list's own first kept_n entries stay)
        if (tid < n) w[tid] = weight(cat_key_value(sh.list[tid]));
        __syncthreads();
        if (tid < n) {
          const uint32_t idx = static_cast<uint32_t>(sh.list[tid]);
          u64 before = 0;
          for (int j = 0; j < n; ++j) before += static_cast<uint32_t>(sh.list[j]) < idx ? w[j] : 0;
          if (before < target && before + w[tid] >= target) found = static_cast<int>(idx);
        }
      }
    } else {
      cat_locate(team, row, part, inv_t, target, kept_weight, &found);
    }
    if (found >= 0) {
      p.token[r] = found;
      if (p.logp) p.logp[r] = static_cast<float>(static_cast<double>(cat_scale(cat_float(row.base[row.head + found]), inv_t)) - norm);
    }
  }
  team.sync();   // no block leaves while another may still read its shared memory
}

// ------------------------------------------------------------------------------------------------------- verification
struct CatVerifyParams {
  int B, gamma, rows, V;
  CatView q, p;
  const double *dist_q, *dist_p;   // [B gamma, 5], [B rows, 5]
  const int32_t* token;            // [B, gamma]
  const float* u;
  float* logratio;
  int32_t* n_accept;
  uint32_t* accept_mask;
};

// log probability of one token under a row's summary; -inf where it is not kept
template <typename T>
__device__ __forceinline__ double cat_log_prob(const CatView& m, int64_t row, const double* d, int token) {
  const float t = cat_scale(cat_float(static_cast<const T*>(m.data)[row * m.ld + token]), static_cast<float>(d[4]));
  const bool kept = t > d[1] || (t == d[1] && token <= d[2]);
  return kept ? static_cast<double>(t) - d[0] : -INFINITY;
}

// A warp per sequence, a lane per position: logratio = log p(x) - log q(x), accept iff log u <= logratio, n_accept = leading accepts.
template <typename TQ, typename TP>
__global__ void __launch_bounds__(128) cat_verify_kernel(const CatVerifyParams p) {
  griddep_enter();
  const int b = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (b >= p.B) return;
  bool ok = false;
  if (lane < p.gamma) {
    const int64_t r = static_cast<int64_t>(b) * p.gamma + lane, rp = static_cast<int64_t>(b) * p.rows + lane;
    const int x = p.token[r];
    double ratio = -INFINITY;
    if (x >= 0 && x < p.V) {
      const double lp = cat_log_prob<TP>(p.p, rp, p.dist_p + rp * kCatRow, x), lq = cat_log_prob<TQ>(p.q, r, p.dist_q + r * kCatRow, x);
      if (lp > -INFINITY) ratio = lq > -INFINITY ? lp - lq : INFINITY;
    }
    p.logratio[r] = static_cast<float>(ratio);
    ok = log(static_cast<double>(p.u[r])) <= ratio;
  }
  const uint32_t mask = __ballot_sync(0xffffffffu, ok);
  if (lane == 0) {
    const uint32_t rej = ~mask & (p.gamma >= 32 ? 0xffffffffu : ((1u << p.gamma) - 1u));
    p.n_accept[b] = rej ? __ffs(rej) - 1 : p.gamma;
    if (p.accept_mask) p.accept_mask[b] = mask;
  }
}

// --------------------------------------------------------------------------------------------------------- resampling
struct CatResampleParams {
  int B, gamma, rows, V;
  CatView q, p;
  const double *dist_q, *dist_p;
  const int32_t* n_accept;
  const float* w;
  int32_t* x_new;
};

// A cluster per sequence: the token of max(0, p - q) at the first rejected position (of p where that is nothing, and at the bonus
// position).  Probabilities to 2^-52, integer sums as above.
template <typename TQ, typename TP>
__global__ void __launch_bounds__(kCatThreads, 2) cat_resample_kernel(const CatResampleParams p) {
  __shared__ CatShared sh;
  CatTeam team(sh);
  const int b = blockIdx.x / team.cs;
  griddep_enter();
  cat_table(sh.tab);
  __syncthreads();
  const int n = p.n_accept[b];
  const bool residual = n < p.gamma;
  const int64_t rp = static_cast<int64_t>(b) * p.rows + n, rq = static_cast<int64_t>(b) * p.gamma + n;
  if (n < 0 || n >= p.rows || !(p.dist_p[rp * kCatRow + 3] > 0.0)) {   // (the whole cluster)
    if (team.rank == 0 && threadIdx.x == 0) p.x_new[b] = -1;
    team.sync();
    return;
  }
  const double* dp = p.dist_p + rp * kCatRow;
  const double cp = -dp[0] * kLog2e;
  const float cut_p = static_cast<float>(dp[1]), inv_p = static_cast<float>(dp[4]);
  const int last_p = static_cast<int>(dp[2]);
  double cq = 0.0;
  float cut_q = INFINITY, inv_q = 1.0f;
  int last_q = -1;
  if (residual) {
    const double* dq = p.dist_q + rq * kCatRow;
    if (dq[3] > 0.0) { cq = -dq[0] * kLog2e; cut_q = static_cast<float>(dq[1]); last_q = static_cast<int>(dq[2]); }
    inv_q = static_cast<float>(dq[4]);
  }
  const CatRow<TP> row(p.p, rp, p.V);
  const TQ* qrow = static_cast<const TQ*>(p.q.data) + (residual ? rq * p.q.ld : 0);
  const CatPart part(row, team.cs, team.rank);
  bool minus = residual;
  auto kept = [](float t, int i, float cut, int last) { return t > cut || (t == cut && i <= last); };
  auto weight = [&](float t, int idx) -> u64 {
    if (!(t > -INFINITY) || !kept(t, idx, cut_p, last_p)) return 0;
    double x = cat_exp(fmaxf(t, -FLT_MAX), cp, sh.tab);
    if (static_cast<double>(t) * kLog2e + cp < -60.0) x = 0.0;
    if (minus) {
      const float tq = cat_scale(cat_float(qrow[idx]), inv_q);
      if (kept(tq, idx, cut_q, last_q) && static_cast<double>(tq) * kLog2e + cq > -60.0) x -= cat_exp(tq, cq, sh.tab);
    }
    return x > 0.0 ? static_cast<u64>(__double_as_longlong(x + 1.0) - __double_as_longlong(1.0)) : 0;
  };
  u64 total;
  for (;;) {
    u64 none = 0, more = 0;
    total = cat_sums(team, row, part, inv_p, weight);
    team.reduce(total, none, more);
    if (total > 0 || !minus) break;
    minus = false;
    team.sync();
  }
  int found = -1;
  if (total > 0) cat_locate(team, row, part, inv_p, cat_target(p.w[b], total), weight, &found);
  if (found >= 0) p.x_new[b] = found;
  team.sync();
}

}  // namespace csd
