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
// integer sums do not depend on the order, so a cut or a token does not depend on how a row is spread over blocks, and a
// prefix sum is off by 2^-42 of itself and 2^-45 a token: which of 10^5 tokens straddles top_p or u is decided as in 64-bit arithmetic.
//
// A row that fits shared memory goes by one block (cat_row_kernel), which reads it once and does the passes there.  Other rows, few long ones and
// many that would each fill an SM, by three kernels over (row, part of the row): the largest logit (cat_top_kernel); counts by distance from it, or what needs no
// counts (cat_scan_kernel); weights and the few candidates for the cut (cat_range_kernel).  The last block of a row to arrive draws the
// conclusion for the row.  One kernel that kept a row in a cluster took 2 to 4 times as long: its passes shared 64 registers with
// everything a row's state needs, and a reduction through distributed shared memory cost 1.3 us.
//
// Bound by instructions, not by reading: 47 a token with its weight (11 of them fp64), 22 a token counted.  512 rows of 131072 fp32 with top-p take
// 306 us (the three kernels, each alone, 49, 92 and 175; reading once at the copy rate 41), 576 of 65536 bf16 with top-k 200 and top-p, with the ratios, 68 (reading 12).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <limits.h>
#include <stdint.h>

#include <type_traits>

#include "ptx.cuh"

namespace csd {
typedef unsigned long long u64;

constexpr int kCatThreads = 256;
constexpr int kCatWarps = kCatThreads / 32;
constexpr int kCatBins = 2048;        // bins of the histogram: 1/64 of scaled logit each, 32 below the largest
constexpr float kCatPerUnit = 64.0f;
constexpr int kCatFrac = 5;           // bits of a token's place within its bin
constexpr int kCatPack = 18;          // a word holds a count (above) and a sum of places of up to 2^13 tokens
constexpr int kCatList = 2048;        // candidates that are sorted
constexpr int kCatSub = 1024;         // bins of a refinement
constexpr int kCatPiece = 512;        // tokens whose weights are summed together, to find a token by its cumulative weight
constexpr int kCatRow = 5;            // doubles of a row's summary
constexpr int kCatTau = 256;          // top-k up to which its tokens are gathered by a threshold from the threads' maxima
constexpr int kCatMaxV = 1 << 19;     // sums of 2^19 weights of 2^44 stay far below 2^64
constexpr int kCatMaxPieces = kCatMaxV / kCatPiece + 1;   // (rows that do not start on 16 bytes)
constexpr double kLog2e = 1.4426950408889634074;
constexpr float kCatFloor = 32.0f;    // weights are 0 from here on down

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
  static constexpr bool kShared = false;
  using Type = T;
  __device__ __forceinline__ int pieces() const { return (head + V + kCatPiece - 1) / kCatPiece; }
  __device__ __forceinline__ T at(int i) const { return base[head + i]; }
  __device__ __forceinline__ bool whole(int v) const { const int first = v * kVec - head; return first >= 0 && first + kVec <= V; }
  __device__ __forceinline__ uint4 vec(int v) const { return __ldg(reinterpret_cast<const uint4*>(base) + v); }
  __device__ __forceinline__ bool some(int v) const { return v * kVec - head < V; }
  __device__ __forceinline__ static uint4 none() { const uint32_t mk = CatType<T>::masked(); return make_uint4(mk, mk, mk, mk); }
  __device__ __noinline__ uint4 edge(int v) const {   // across an end of the row: masked outside
    const int first = v * kVec - head;
    __align__(16) T e[kVec];
    *reinterpret_cast<uint4*>(e) = none();
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (first + i >= 0 && first + i < V) e[i] = base[static_cast<int64_t>(v) * kVec + i];
    return *reinterpret_cast<uint4*>(e);
  }
};

__device__ __forceinline__ u64 cat_warp_sum(u64 v) {   // in three pieces: 32 times 27 bits fit a word
  const uint32_t a = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(v) & 0x7ffffffu);
  const uint32_t b = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(v >> 27) & 0x7ffffffu);
  const uint32_t c = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(v >> 54));
  return a + (static_cast<u64>(b) << 27) + (static_cast<u64>(c) << 54);
}
__device__ __forceinline__ u64 cat_warp_max(u64 v) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(v >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(v >> 32) == hi ? static_cast<uint32_t>(v) : 0u);
  return (static_cast<u64>(hi) << 32) | lo;
}

// A row that lies in shared memory, as the vectors of its aligned memory with what is outside masked.
template <typename T> struct CatHeld {
  static constexpr int kVec = CatType<T>::kVec;
  static constexpr bool kShared = true;
  using Type = T;
  const uint4* data;
  int head, V, vecs;
  __device__ __forceinline__ bool whole(int v) const { return v < vecs; }
  __device__ __forceinline__ bool some(int) const { return false; }
  __device__ __forceinline__ uint4 vec(int v) const { return data[v]; }
  __device__ __forceinline__ static uint4 none() { return CatRow<T>::none(); }
  __device__ __forceinline__ uint4 edge(int) const { return none(); }
  __device__ __forceinline__ int pieces() const { return (head + V + kCatPiece - 1) / kCatPiece; }
  __device__ __forceinline__ T at(int i) const { return reinterpret_cast<const T*>(data)[head + i]; }
};
// What other blocks may have written, or this one in its own shared memory.
template <bool SHARED, typename X> __device__ __forceinline__ X cat_get(const X* p) { return SHARED ? *p : __ldcg(p); }

// f(logits, index of the first) for the vectors of pieces [p0, p1), a piece a warp; done(piece) after each.  Tokens outside the row are masked.
template <int NT, typename R, typename F, typename D>
__device__ __forceinline__ void cat_pieces(const R& row, int p0, int p1, F f, D done) {
  constexpr int kVec = R::kVec, kIts = kCatPiece / (32 * kVec), kTwo = 4 / kIts, kWarps = NT / 32;   // four vectors are requested at a time
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int p = p0 + warp; p < p1; p += kTwo * kWarps) {
    uint4 raw[4];
    bool all = true;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int q = p + j / kIts * kWarps, v = (q * kIts + j % kIts) * 32 + lane;
      const bool in = q < p1 && row.whole(v);
      all = all && in;
      if (in) raw[j] = row.vec(v);
    }
    if (!all) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int q = p + j / kIts * kWarps, v = (q * kIts + j % kIts) * 32 + lane;
        if (q >= p1 || !row.whole(v)) raw[j] = q < p1 && row.some(v) ? row.edge(v) : row.none();
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int q = p + j / kIts * kWarps;
      if (q >= p1) break;
      float l[kVec];
      CatType<typename R::Type>::unpack(raw[j], l);
      f(l, ((q * kIts + j % kIts) * 32 + lane) * kVec - row.head);
      if (j % kIts == kIts - 1) done(q);
    }
  }
}
template <int NT, typename R, typename F>
__device__ __forceinline__ void cat_each(const R& row, int p0, int p1, F f) {
  if constexpr (R::kShared) {   // vector by vector: few pieces keep all threads busy too
    constexpr int kVec = R::kVec;
#pragma unroll 2
    for (int v = p0 * (kCatPiece / kVec) + threadIdx.x; v < min(p1 * (kCatPiece / kVec), row.vecs); v += NT) {
      float l[kVec];
      CatType<typename R::Type>::unpack(row.vec(v), l);
      f(l, v * kVec - row.head);
    }
  } else {
    cat_pieces<NT>(row, p0, p1, f, [](int) {});
  }
}
// The same where f gives a vector's weight: the pieces' sums go to seg; returns this thread's own sum.
template <int NT, typename R, typename F>
__device__ __forceinline__ u64 cat_sums(const R& row, int p0, int p1, u64* seg, F f) {
  u64 all = 0, sum = 0;
  cat_pieces<NT>(row, p0, p1, [&](const float* l, int idx) { sum += f(l, idx); }, [&](int q) {
    all += sum;
    sum = cat_warp_sum(sum);
    if ((threadIdx.x & 31) == 0) seg[q] = sum;
    sum = 0;
  });
  return all;
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
  const double e = tab[k & 15];   // 2^(j/16) less j in units of the exponent / 16: adding k there leaves its whole part
  const double b = __hiloint2double(__double2hiint(e) + (k << 16), __double2loint(e));
  return fma(b * r, p, b);
}
__device__ __forceinline__ void cat_table(double* tab) {
  if (threadIdx.x < 16) {
    const double e = exp2(threadIdx.x / 16.0);
    tab[threadIdx.x] = __hiloint2double(__double2hiint(e) - static_cast<int>(threadIdx.x << 16), __double2loint(e));
  }
}
// exp(t - norm) of scaled logits t as 2^((t - base) log2(e) + c).  Where norm is so large that fp64 would lose what t - norm is, base
// is the nearest fp32 number: t - base is exact for every t that matters (within a factor of two of base).  What lies more
// than `range` below (masked tokens, -inf and NaN, too) counts as `range`: its weight rounds to 0, and no argument leaves cat_exp's domain;
// what lies above counts as norm itself, where no finite scaled logit lies.
struct CatScale {
  float base, floor, ceil;
  double c;
  __device__ __forceinline__ CatScale(double norm, float range) {
    base = fabs(norm) >= 4096.0 ? static_cast<float>(norm) : 0.0f;
    const double rest = norm - base;
    c = -rest * kLog2e;
    ceil = __double2float_ru(rest);
    floor = ceil - range;
  }
  __device__ __forceinline__ double exp(float t, const double* tab) const { return cat_exp(fminf(fmaxf(t - base, floor), ceil), c, tab); }
  // the same where base is 0: no scaled logit lies above
  __device__ __forceinline__ double exp0(float t, const double* tab) const { return cat_exp(fmaxf(t, floor), c, tab); }
};
// Weights are sums of doubles with 256 added to each: the bits of v + 256 are those of 256 plus v in units of 2^-44, so adding up
// bits and taking off 256's as often gives the integer sum.
constexpr u64 kCat256 = 0x4070000000000000ull;
__device__ __forceinline__ u64 cat_bits(double v) { return static_cast<u64>(__double_as_longlong(v + 256.0)); }
// Weight relative to the largest scaled logit: 2^44 exp(t - m), rounded; at most a few units above 2^44, 0 below 2^-45.
__device__ __forceinline__ u64 cat_weight(float t, const CatScale& s, const double* tab) { return cat_bits(s.exp(t, tab)) - kCat256; }

// Barriers of a block's first NT threads: what follows the passes over a row is dependent steps of few values, which more warps make slower.
template <int NT> __device__ __forceinline__ void cat_sync() { asm volatile("bar.sync 1, %0;" ::"n"(NT) : "memory"); }
template <int NT> __device__ __forceinline__ bool cat_sync_or(bool x) {
  uint32_t any;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.or.pred p, 1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(any) : "r"(static_cast<uint32_t>(x)), "n"(NT) : "memory");
  return any != 0;
}
// Inclusive sum over the block's threads (exclusive = inclusive - v); part: a value a warp of shared memory.
template <int NT, typename X> __device__ __forceinline__ X cat_block_scan(X v, X* part, X* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const X w = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += w; }
  cat_sync<NT>();
  if (lane == 31) part[warp] = v;
  cat_sync<NT>();
  X before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < NT / 32; ++i) { const X w = part[i]; if (i < warp) before += w; all += w; }
  *total = all;
  return v + before;
}

// ------------------------------------------------------------------------------------------------------- workspace
struct CatTop { uint32_t top, tau, live, pad; };   // of a row's part: order of the largest logit and of the threshold, tokens not masked
enum { CAT_DONE = 0, CAT_RANGE = 1, CAT_SEARCH = 2 };
struct CatState {                                  // of a row
  uint32_t ticket[2], list_n;
  int mode;                                        // what is left to do for cat_range_kernel
  float da, db, dk, de;                            // distances from the largest: listed are [da, db) and [dk, de), weights wanted below da (and below dk)
  uint32_t at_a, n1, n_mid;
  int apart, upto, ends;
};
struct CatWork {
  int rows, splits, share, pieces;                 // rows of this launch; parts of a row, pieces a part, pieces of the longest row
  CatTop* top;                                     // [rows, splits]
  CatState* state;                                 // [rows]
  uint32_t* hist;                                  // [rows, 2, kCatBins]
  u64* list;                                       // [rows, kCatList]
  u64* seg;                                        // [rows, pieces]
  u64* tot;                                        // [rows, splits, 3]
};

struct CatParams {
  int V;
  int64_t r0;                                      // first row of this launch
  CatView logits;
  const float* temperature;   // [R] or null: 1
  const int32_t* top_k;       // [R] or null
  const float *top_p, *min_p; // [R] or null
  const float* u;             // [R] or null: no token is drawn
  int32_t* token;             // [R]
  float* logp;                // [R] or null
  double* dist;               // [R, 5] or null
  CatWork w;
};

// ---------------------------------------------------------------------------------------------------- shared memory
template <int NT> struct CatShared {
  __align__(16) uint32_t hist[2 * kCatBins];  // tokens per bin, sum of their places in it; later: sums of all pieces, words of a refinement
  __align__(16) u64 list[kCatList];           // candidates
  u64 scan[NT / 32];
  uint2 scan2[NT / 32];
  u64 red[32][3];
  double tab[16];
  uint32_t rank[2 * NT];                      // of the sort
  CatTop top;
  CatState state;                             // of a row that one block holds
  // found by one thread, read by all
  u64 found_key, found_sum, found_upto, found_before[2];
  double norm;
  uint32_t found_n;
  int found_a, found_b, found_k, found_prev, found_listed, found_piece;
  float found_lo, found_hi;
  uint32_t at_a, at_b, at_k, end_k, list_n, base, last;
  __device__ __forceinline__ void append(u64 key) {
    const uint32_t i = atomicAdd(&list_n, 1u);
    if (i < kCatList) list[i] = key;
  }
};
static_assert(2 * kCatBins * sizeof(uint32_t) >= kCatMaxPieces * sizeof(u64), "the pieces' sums fit the histogram's place");
static_assert(2 * kCatBins >= 4 * kCatSub, "a refinement's words do too");

// Over the block's threads: the sums of a and b, the maximum of c.
template <int NT, int TAIL>
__device__ __forceinline__ void cat_reduce(CatShared<TAIL>& sh, u64& a, u64& b, u64& c) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  a = cat_warp_sum(a); b = cat_warp_sum(b); c = cat_warp_max(c);
  if (NT == TAIL) cat_sync<NT>(); else __syncthreads();
  if (lane == 0) { sh.red[warp][0] = a; sh.red[warp][1] = b; sh.red[warp][2] = c; }
  if (NT == TAIL) cat_sync<NT>(); else __syncthreads();
  const bool in = lane < NT / 32;
  a = cat_warp_sum(in ? sh.red[lane][0] : 0); b = cat_warp_sum(in ? sh.red[lane][1] : 0); c = cat_warp_max(in ? sh.red[lane][2] : 0);
}

// Inclusive sums of a count and a weight over the block's threads.
template <int NT>
__device__ __forceinline__ void cat_block_scan2(uint32_t& n, float& w, uint2* part, float* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, n, o);
    const float y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) { n += x; w += y; }
  }
  if (lane == 31) part[warp] = make_uint2(n, __float_as_uint(w));
  cat_sync<NT>();
  uint32_t bn = 0;
  float bw = 0.0f, all = 0.0f;
#pragma unroll
  for (int i = 0; i < NT / 32; ++i) {
    const uint2 x = part[i];
    if (i < warp) { bn += x.x; bw += __uint_as_float(x.y); }
    all += __uint_as_float(x.y);
  }
  n += bn; w += bw;
  *total = all;
}

// Sorts list[0, n) ascending: by value into as many buckets of equal width as threads, then by counting within each (1.2 k cycles at 400 entries; each counting
// all before it took 11 k, a bitonic network, whose every step is a round through shared memory, 20 k).  Where a bucket
// holds too many (equals) the network does it, padded to a power of two; steps within 64 neighbours stay in one warp.
template <int NT>
__device__ __noinline__ void cat_sort(CatShared<NT>& sh, int n) {
  u64* const list = sh.list;
  u64* const other = reinterpret_cast<u64*>(sh.hist);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kEach = kCatList / NT, kMost = 64;
  if (n <= 96) {   // few: each counts all before it
    const u64 key = tid < n ? list[tid] : 0;
    int before = 0;
    if (tid < n) {
#pragma unroll 4
      for (int j = 0; j < n; ++j) before += list[j] < key;
    }
    cat_sync<NT>();
    if (tid < n) list[before] = key;
    cat_sync<NT>();
    return;
  }
  const int each = (n + NT - 1) / NT;
  sh.rank[tid] = 0;
  uint32_t lo = 0xffffffffu, hi = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    if (j >= each) break;
    const int i = tid + j * NT;
    if (i < n) { const uint32_t o = static_cast<uint32_t>(list[i] >> 32); lo = min(lo, o); hi = max(hi, o); }
  }
  lo = __reduce_min_sync(0xffffffffu, lo); hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) sh.scan2[warp] = make_uint2(lo, hi);
  cat_sync<NT>();
#pragma unroll
  for (int i = 0; i < NT / 32; ++i) { const uint2 x = sh.scan2[i]; lo = min(lo, x.x); hi = max(hi, x.y); }
  const float first = cat_key_value(static_cast<u64>(lo) << 32), last = cat_key_value(static_cast<u64>(hi) << 32);
  const float width = fmaxf(first - last, FLT_MIN), scale = fminf(__fdividef(NT - 1.0f, width), FLT_MAX);
  uint32_t at[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    if (j >= each) break;
    const int i = tid + j * NT;
    if (i < n) {
      const uint32_t b = min(__float2uint_rd(fminf((first - cat_key_value(list[i])) * scale, NT - 1.0f)), NT - 1u);
      at[j] = b << 16 | atomicAdd(&sh.rank[b], 1u);
    }
  }
  cat_sync<NT>();
  const uint32_t own = sh.rank[tid];
  if (!cat_sync_or<NT>(own > kMost)) {
    uint32_t end = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint32_t x = __shfl_up_sync(0xffffffffu, end, o); if (lane >= o) end += x; }
    if (lane == 31) sh.scan2[warp].x = end;
    cat_sync<NT>();
#pragma unroll
    for (int i = 0; i < NT / 32; ++i) if (i < warp) end += sh.scan2[i].x;
    sh.rank[NT + tid] = end;                // where a bucket ends
    cat_sync<NT>();
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    if (j >= each) break;
      const int i = tid + j * NT;
      if (i < n) { const uint32_t b = at[j] >> 16; other[sh.rank[NT + b] - sh.rank[b] + (at[j] & 0xffffu)] = list[i]; }
    }
    cat_sync<NT>();
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    if (j >= each) break;
      const int i = tid + j * NT;
      if (i < n) {
        const u64 key = list[i];
        const uint32_t b = at[j] >> 16, to = sh.rank[NT + b], from = to - sh.rank[b];
        uint32_t before = from;
        for (uint32_t k = from; k < to; ++k) before += other[k] < key;
        at[j] = before;
      }
    }
    cat_sync<NT>();
    u64 key[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) { if (j >= each) break; const int i = tid + j * NT; if (i < n) key[j] = list[i]; }
    cat_sync<NT>();
#pragma unroll
    for (int j = 0; j < kEach; ++j) { if (j >= each) break; const int i = tid + j * NT; if (i < n) list[at[j]] = key[j]; }
    cat_sync<NT>();
    return;
  }
  int P = 128;
  while (P < n) P <<= 1;
  for (int i = n + tid; i < P; i += NT) list[i] = ~0ull;
  cat_sync<NT>();
  for (int size = 2; size <= P; size <<= 1)
    for (int stride = size >> 1; stride > 0; stride >>= 1) {
      for (int i = tid; i < P / 2; i += NT) {
        const int a = ((i & ~(stride - 1)) << 1) | (i & (stride - 1)), b = a + stride;
        const u64 x = list[a], y = list[b];
        const bool up = (a & size) == 0;
        if ((x > y) == up) { list[a] = y; list[b] = x; }
      }
      if (stride > 32 || (stride == 1 && size >= 64)) cat_sync<NT>(); else __syncwarp();
    }
  cat_sync<NT>();
}

// Whether this block is the last of its row's to come here; if so, what the others wrote before is visible to it.
template <int NT>
__device__ __forceinline__ bool cat_last(CatShared<NT>& sh, uint32_t* ticket, int splits) {
  __threadfence();
  cat_sync<NT>();
  if (threadIdx.x == 0) sh.last = splits == 1 || atomicAdd(ticket, 1u) == static_cast<uint32_t>(splits - 1);
  cat_sync<NT>();
  if (!sh.last) return false;
  __threadfence();
  return true;
}
// This block's list goes to the row's in memory, ...
template <int NT>
__device__ __forceinline__ void cat_put_list(CatShared<NT>& sh, CatState* st, u64* list, int splits) {
  cat_sync<NT>();
  const uint32_t n = sh.list_n;
  if (splits == 1) return;
  if (threadIdx.x == 0 && n > 0) sh.base = atomicAdd(&st->list_n, n);
  cat_sync<NT>();
  if (n > 0 && n <= kCatList)
    for (uint32_t i = threadIdx.x; i < n; i += NT)
      if (sh.base + i < kCatList) __stcg(list + sh.base + i, sh.list[i]);
}
// ... and comes back whole to the last block: the number of entries (more than kCatList: not all of them).
template <int NT>
__device__ __forceinline__ int cat_get_list(CatShared<NT>& sh, const CatState* st, const u64* list, int splits) {
  cat_sync<NT>();
  if (splits == 1) return static_cast<int>(min(sh.list_n, kCatList + 1u));
  const uint32_t n = min(__ldcg(&st->list_n), kCatList + 1u);
  for (uint32_t i = threadIdx.x; i < min(n, static_cast<uint32_t>(kCatList)); i += NT) sh.list[i] = __ldcg(list + i);
  cat_sync<NT>();
  return static_cast<int>(n);
}

// The weight that top-p asks for (the likeliest token is kept whatever it asks).
__device__ __forceinline__ double cat_limit(float top_p, u64 total) { return fmax(static_cast<double>(top_p) * static_cast<double>(total), 1.0); }
__device__ __forceinline__ u64 cat_target(float u, u64 total) {
  const double x = ceil(static_cast<double>(u) * static_cast<double>(total));
  u64 t = x >= 1.0 ? static_cast<u64>(x) : 1;
  return t > total ? total : t;
}

// The token at which the cumulative weight reaches target, by one block: seg has the sums of all pieces, without the weights of
// the first `extra` entries of the list (listed(key)); the piece that holds the token is gone through again, a warp a vector.
// weights(l, idx, w): of a vector's logits, as in the pass that formed the sums, listed tokens included.  One thread gets the token, the others -1;
// all get -1 where no piece reaches target.
template <int NT, typename R, typename W, typename L>
__device__ __forceinline__ int cat_locate(CatShared<NT>& sh, const R& row, const u64* seg, u64 target, int extra, L listed, W weights) {
  constexpr int kVec = R::kVec, kIts = kCatPiece / (32 * kVec), kEach = (kCatMaxPieces + NT - 1) / NT;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, pieces = row.pieces(), each = (pieces + NT - 1) / NT;
  // listed weights are added up in two words of 22 and 23 bits (a piece has 2^9 tokens)
  uint32_t *lo = sh.hist, *hi = sh.hist + kCatMaxPieces;
  cat_sync<NT>();
  if (extra > 0) {
    for (int i = tid; i < pieces; i += NT) { lo[i] = 0; hi[i] = 0; }
    cat_sync<NT>();
    for (int i = tid; i < extra; i += NT) {
      const u64 key = sh.list[i], w = listed(key);
      const int q = (static_cast<int>(static_cast<uint32_t>(key)) + row.head) / kCatPiece;
      atomicAdd(&lo[q], static_cast<uint32_t>(w) & 0x3fffffu);
      atomicAdd(&hi[q], static_cast<uint32_t>(w >> 22));
    }
    cat_sync<NT>();
  }
  u64 x[kEach], s = 0, total;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int i = tid * each + j;
    x[j] = 0;
    if (j < each && i < pieces) {
      x[j] = cat_get<R::kShared>(seg + i);
      if (extra > 0) x[j] += lo[i] + (static_cast<u64>(hi[i]) << 22);
    }
    s += x[j];
  }
  if (tid == 0) sh.found_piece = -1;
  u64 before = cat_block_scan<NT, u64>(s, sh.scan, &total) - s;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    if (before < target && before + x[j] >= target) { sh.found_piece = tid * each + j; sh.found_sum = before; }
    before += x[j];
  }
  cat_sync<NT>();
  const int piece = sh.found_piece;
  if (piece < 0) return -1;   // sums beyond 64 bits: of a summary that is not this row's
  u64 w[kVec], incl = 0;
  int idx = 0;
  if (warp < kIts) {
    const int v = (piece * kIts + warp) * 32 + lane;
    uint4 raw = row.whole(v) ? row.vec(v) : row.some(v) ? row.edge(v) : row.none();
    float l[kVec];
    CatType<typename R::Type>::unpack(raw, l);
    idx = v * kVec - row.head;
    weights(l, idx, w);
#pragma unroll
    for (int i = 0; i < kVec; ++i) incl += w[i];
    s = incl;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const u64 y = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += y; }
    if (lane == 31) sh.scan[warp] = incl;
  }
  cat_sync<NT>();
  int token = -1;
  if (warp < kIts) {
    before = sh.found_sum + incl - s;
    for (int i = 0; i < warp; ++i) before += sh.scan[i];
    if (before < target && before + s >= target) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) { if (before < target && before + w[i] >= target) token = idx + i; before += w[i]; }
    }
  }
  return token;
}

// ----------------------------------------------------------------------------------------------------- refinement
// The last element kept, where more elements than the list holds come into question (many equals, rows of tiny spread), by one block: the first
// element in key order at which the running count reaches `count` (BY_WEIGHT: the running weight reaches `limit`) among keys
// <= last, searched in ever narrower intervals [a, b] of keys.  Weights of a bin are summed in three words of 15 bits
// each: 2^17 tokens fit, so a bin that holds more adds up its carries (the words are folded whenever 2^17 tokens have been read).
template <bool BY_WEIGHT, int NT, typename R>
__device__ __noinline__ u64 cat_refine(CatShared<NT>& sh, const R& row, float inv_t, const CatScale& sc, u64 last, u64 count, double limit) {
  constexpr int kVec = R::kVec, kEach = kCatSub / NT, kFold = (1 << 17) / kCatPiece;
  const int tid = threadIdx.x, pieces = row.pieces();
  uint32_t* words = sh.hist + kCatSub;
  u64 a = 0, b = last;
  for (;;) {
    const int top = 64 - __clzll(static_cast<long long>(b - a | 1));
    const int shift = top > 10 ? top - 10 : 0;
    u64 n_before = 0, w_before = 0, none = 0, n[kEach] = {}, w[kEach] = {};
    for (int p0 = 0; p0 < pieces; p0 += kFold) {
      cat_sync<NT>();                               // nobody reads the arrays below any more
      for (int i = tid; i < 4 * kCatSub; i += NT) sh.hist[i] = 0;
      cat_sync<NT>();
      cat_each<NT>(row, p0, min(p0 + kFold, pieces), [&](const float* l, int idx) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          const float t = cat_scale(l[i], inv_t);
          const u64 key = cat_key(t, idx + i);
          if (!(t > -INFINITY) || key > b) continue;
          const u64 x = BY_WEIGHT ? cat_weight(t, sc, sh.tab) : 0;
          if (key < a) { ++n_before; w_before += x; }
          else {
            const int s = static_cast<int>((key - a) >> shift);
            atomicAdd(&sh.hist[s], 1u);
            if (BY_WEIGHT) {
              atomicAdd(&words[s], static_cast<uint32_t>(x) & 0x7fffu);
              atomicAdd(&words[kCatSub + s], static_cast<uint32_t>(x >> 15) & 0x7fffu);
              atomicAdd(&words[2 * kCatSub + s], static_cast<uint32_t>(x >> 30));
            }
          }
        }
      });
      cat_sync<NT>();
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int i = tid * kEach + j;
        n[j] += sh.hist[i];
        if (BY_WEIGHT) w[j] += words[i] + (static_cast<u64>(words[kCatSub + i]) << 15) + (static_cast<u64>(words[2 * kCatSub + i]) << 30);
      }
    }
    cat_reduce<NT>(sh, n_before, w_before, none);
    u64 own_n = 0, own_w = 0, all_n, all_w = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) { own_n += n[j]; own_w += w[j]; }
    u64 pn = cat_block_scan<NT, u64>(own_n, sh.scan, &all_n) - own_n + n_before;
    u64 pw = w_before;
    if (BY_WEIGHT) pw += cat_block_scan<NT, u64>(own_w, sh.scan, &all_w) - own_w;
    auto reached = [&](u64 cn, u64 cw) { return BY_WEIGHT ? static_cast<double>(cw) >= limit : cn >= count; };
    if (!reached(n_before + all_n, w_before + all_w)) return last;   // (all of them are kept)
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      if (!reached(pn, pw) && reached(pn + n[j], pw + w[j])) { sh.found_a = tid * kEach + j; sh.found_n = static_cast<uint32_t>(n[j]); sh.found_before[0] = pn; sh.found_before[1] = pw; }
      pn += n[j]; pw += w[j];
    }
    if (tid == 0) sh.list_n = 0;
    cat_sync<NT>();
    a += static_cast<u64>(sh.found_a) << shift;
    const u64 span = (1ull << shift) - 1;
    b = b - a > span ? a + span : b;
    const int inside = static_cast<int>(sh.found_n);
    pn = sh.found_before[0]; pw = sh.found_before[1];
    if (inside > kCatList) continue;
    // few enough to be sorted
    cat_each<NT>(row, 0, pieces, [&](const float* l, int idx) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float t = cat_scale(l[i], inv_t);
        const u64 key = cat_key(t, idx + i);
        if (t > -INFINITY && key >= a && key <= b) sh.append(key);
      }
    });
    cat_sync<NT>();
    cat_sort(sh, inside);
    if (!BY_WEIGHT) return sh.list[count - pn - 1];
    constexpr int kMine = kCatList / NT;
    u64 s = 0, total;
    for (int j = 0; j < kMine; ++j) { const int i = tid * kMine + j; if (i < inside) s += cat_weight(cat_key_value(sh.list[i]), sc, sh.tab); }
    u64 before = cat_block_scan<NT, u64>(s, sh.scan, &total) - s + pw;
    for (int j = 0; j < kMine; ++j) {
      const int i = tid * kMine + j;
      const u64 x = i < inside ? cat_weight(cat_key_value(sh.list[i]), sc, sh.tab) : 0;
      if (i < inside && !reached(0, before) && reached(0, before + x)) sh.found_key = sh.list[i];
      before += x;
    }
    cat_sync<NT>();
    return sh.found_key;
  }
}

// ------------------------------------------------------------------------------------------------------ a row's settings
// a threshold in the order of keys: kept are t > value, and t = value up to the index
struct CatBound {
  float value;
  int idx;
  __device__ __forceinline__ bool kept(float t, int i) const { return t > value || (t == value && i <= idx); }
};
// Adds in shared memory where p < limit, without a branch.
__device__ __forceinline__ void cat_add_if(uint32_t* at, uint32_t v, uint32_t p, uint32_t limit) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.u32 p, %2, %3;\n\t@p red.shared.add.u32 [%0], %1;\n\t}" ::"r"(smem_u32(at)), "r"(v), "r"(p), "r"(limit) : "memory");
}
// Distance from the largest in units of 1/64, kCatFrac bits behind the point; kCatBins and more: below every bin (masked too).
__device__ __forceinline__ uint32_t cat_place(float m, float l, float inv_t) {
  return __float2uint_rd(fminf((m - __fmul_rn(l, inv_t)) * (kCatPerUnit * (1 << kCatFrac)), 4095.0f * (1 << kCatFrac)));
}
struct CatRequest {   // what the caller asks of a row
  float inv_t, top_p;
  int want;           // top-k, 0: off
  bool by_p, few;
  __device__ __forceinline__ CatRequest(const CatParams& p, int64_t r) {
    const float temp = p.temperature ? p.temperature[r] : 1.0f;
    const bool greedy = !(temp > 0.0f);
    inv_t = greedy ? 1.0f : fminf(__fdiv_rn(1.0f, temp), FLT_MAX);   // (of a subnormal temperature: 0 times it has to be 0)
    want = greedy ? 1 : (p.top_k ? p.top_k[r] : 0);
    if (want <= 0 || want >= p.V) want = 0;
    top_p = p.top_p ? p.top_p[r] : 1.0f;
    by_p = top_p < 1.0f && !greedy;
    few = want > 0 && want <= kCatTau;
  }
  // Scaled logits have to be numbers: at an infinite temperature they are 0, but an infinite one stays beyond the range, as at every other temperature.
  __device__ __forceinline__ void at_top(float largest) { if (inv_t == 0.0f && largest == INFINITY) inv_t = __uint_as_float(1u); }
};
// The least scaled logit that min-p keeps: the smallest fp32 number not below m + log(min_p).
__device__ __forceinline__ float cat_least(const CatParams& p, int64_t r, float m) {
  const float mp = p.min_p ? p.min_p[r] : 0.0f;
  return mp > 0.0f ? __double2float_ru(static_cast<double>(m) + log(static_cast<double>(fminf(mp, 1.0f)))) : -INFINITY;
}
// All parts' tops of a row, for every thread.
template <int NT>
__device__ __forceinline__ CatTop cat_tops(CatShared<NT>& sh, const CatWork& w, int row) {
  if (threadIdx.x < 32) {
    uint32_t a = 0xffffffffu, b = 0, n = 0;
    for (int i = threadIdx.x; i < w.splits; i += 32) {
      const CatTop t = w.top[static_cast<int64_t>(row) * w.splits + i];
      a = min(a, t.top); b = max(b, t.tau); n += t.live;
    }
    a = __reduce_min_sync(0xffffffffu, a); b = __reduce_max_sync(0xffffffffu, b); n = __reduce_add_sync(0xffffffffu, n);
    if (threadIdx.x == 0) sh.top = CatTop{a, b, n, 0};
  }
  cat_sync<NT>();
  return sh.top;
}

// ------------------------------------------------------------------------------------------------------- conclusions
// What a row's cut is derived from: the list of n candidates; before the first of them n_above tokens of weight
// w_above are kept for certain; between those of the first n1 (where top-p ends) and the rest (where top-k ends, if that is apart)
// lie n_mid; w_upto is the weight of all tokens before the rest.
struct CatCut {
  int n, n1;
  uint32_t n_above, n_mid;
  u64 w_above, w_upto;
  bool by_k, by_p, apart, ends;                    // ends: nothing behind the first n1 is kept (min-p)
  uint32_t k;
  float top_p, least;
};
struct CatKept {       // the conclusion
  u64 last;            // key of the last token kept
  u64 n, w;
  int listed;          // so many of them are the first ones of the list, and not in the pieces' sums
};
// False: the list does not hold the cut.
template <int NT>
__device__ __noinline__ bool cat_resolve(CatShared<NT>& sh, const CatCut& x, const CatScale& sc, CatKept& out) {
  const int tid = threadIdx.x;
  constexpr int kEach = kCatList / NT;
  if (x.n < x.n1) return false;               // (not what was counted)
  cat_sort(sh, x.n);
  // a thread holds `each` entries in a row
  const int each = x.n <= NT ? 1 : x.n <= 2 * NT ? 2 : kEach;
  // where top-k ends in the list
  const int end_k = x.by_k ? static_cast<int>(x.k - x.n_above - x.n_mid) - 1 : x.n - 1;
  u64 s = 0, total;
  u64* lw = reinterpret_cast<u64*>(sh.hist);   // (the entries' weights; of this thread)
  for (int j = 0; j < each; ++j) {
    const int i = tid * each + j;
    const u64 v = i < x.n ? cat_weight(cat_key_value(sh.list[i]), sc, sh.tab) : 0;
    lw[i] = v;
    s += v;
  }
  const u64 start = cat_block_scan<NT, u64>(s, sh.scan, &total) - s;
  if (tid == 0) { sh.found_upto = 0; sh.found_sum = total; sh.found_listed = 0; }
  cat_sync<NT>();
  u64 before = start;
  for (int j = 0; j < each; ++j) {
    const int i = tid * each + j;
    before += lw[i];
    if (i == end_k) sh.found_sum = before;
    if (i == x.n1 - 1) sh.found_upto = before;
  }
  cat_sync<NT>();
  double limit = INFINITY;
  if (x.by_p) limit = cat_limit(x.top_p, !x.by_k ? x.w_upto : x.apart ? x.w_upto + sh.found_sum - sh.found_upto : x.w_above + sh.found_sum);
  const int most = min(end_k, x.n1 - 1);
  before = start + x.w_above;
  int mine = 0;
  for (int j = 0; j < each; ++j) {
    const int i = tid * each + j;
    mine += i <= most && ((i == 0 && x.n_above == 0) || (static_cast<double>(before) < limit && cat_key_value(sh.list[i]) >= x.least));
    before += lw[i];
  }
  mine = __reduce_add_sync(0xffffffffu, mine);
  cat_sync<NT>();                             // found_sum has been read
  if ((tid & 31) == 0) sh.rank[tid >> 5] = mine;
  cat_sync<NT>();
  int all = 0;
#pragma unroll
  for (int i = 0; i < NT / 32; ++i) all += sh.rank[i];
  const int last = all - 1;
  before = start + x.w_above;
  for (int j = 0; j < each; ++j) {
    const int i = tid * each + j;
    before += lw[i];
    // the cut is certain if the next one in the list is not kept, if top-k ends here, or if top-p's weight is reached here
    if (i == last && (last < most || last == end_k || x.ends || static_cast<double>(before) >= limit)) { sh.found_listed = all; sh.found_sum = before; }
  }
  cat_sync<NT>();
  if (sh.found_listed == 0) return false;
  out.last = sh.list[last]; out.n = x.n_above + static_cast<u64>(all); out.w = sh.found_sum; out.listed = all;
  cat_sync<NT>();
  return true;
}

// One pass over pieces: weights of the tokens that `bound` keeps, their sums by piece; for this thread their weight, number and last key.
template <int NT, typename R>
__device__ __forceinline__ u64 cat_keep(const R& row, int p0, int p1, u64* seg, float inv_t, const CatScale& sc, const double* tab, CatBound bound, u64& n, u64& last) {
  constexpr int kVec = R::kVec;
  float end_t = INFINITY;   // the last token kept: the least, the highest index of its equals
  int end_i = 0;
  uint32_t count = 0;
  const u64 w = cat_sums<NT>(row, p0, p1, seg, [&](const float* l, int idx) -> u64 {
    u64 sum = 0;
#pragma unroll
    for (int h = 0; h < kVec; h += 4) {     // four exponentials side by side
      float t[4];
      bool any = false, in[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        t[i] = cat_scale(l[h + i], inv_t);
        in[i] = bound.kept(t[i], idx + h + i);
        any = any || in[i];
        if (in[i] && t[i] <= end_t) { end_t = t[i]; end_i = idx + h + i; }   // (a thread's indexes ascend)
        count += in[i];
      }
      if (!__any_sync(0xffffffffu, any)) continue;
      double x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = sc.exp(t[i], tab);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += cat_bits(in[i] ? x[i] : 0.0);
      sum -= 4 * kCat256;
    }
    return sum;
  });
  n = count;
  last = count ? cat_key(end_t, end_i) : 0;
  return w;
}

// Writes a row's summary and draws its token.  listed < kept.n: the pieces' sums are in seg.
template <int NT, typename R>
__device__ __forceinline__ void cat_finish(CatShared<NT>& sh, const CatParams& p, int64_t r, const R& row, const u64* seg, float inv_t, const CatScale& sc, float m, const CatKept& kept) {
  const int tid = threadIdx.x;
  const CatBound bound{cat_key_value(kept.last), static_cast<int>(static_cast<uint32_t>(kept.last))};
  auto summary = [&] {   // by a thread of the warp that has least to do
    if (tid != NT - 1) return;
    // The sum in units of the largest token's own weight: 2^44 but for the rounding of CatScale's c, which all weights share and the quotient takes
    // out.  A token that is certain has the quotient 1, so the normaliser is its scaled logit and its log probability 0, exactly.
    const double norm = static_cast<double>(m) + log(static_cast<double>(kept.w) / static_cast<double>(cat_weight(m, sc, sh.tab)));
    sh.norm = norm;
    if (p.dist) {
      double* d = p.dist + r * kCatRow;
      d[0] = norm; d[1] = bound.value; d[2] = bound.idx; d[3] = static_cast<double>(kept.n); d[4] = inv_t;
    }
  };
  if (!p.u) return summary();
  const u64 target = cat_target(p.u[r], kept.w);
  int found = -1;
  if (kept.listed == static_cast<int>(kept.n) && kept.listed <= NT) {   // all of them are listed: each adds up those of smaller index
    const int n = kept.listed;
    u64* w = reinterpret_cast<u64*>(sh.hist);
    cat_sync<NT>();
    const u64 own = tid < n ? cat_weight(cat_key_value(sh.list[tid]), sc, sh.tab) : 0;
    w[tid] = own;
    cat_sync<NT>();
    summary();
    if (tid < n) {
      const uint32_t idx = static_cast<uint32_t>(sh.list[tid]);
      u64 before = 0;
      for (int j = 0; j < n; ++j) before += static_cast<uint32_t>(sh.list[j]) < idx ? w[j] : 0;
      if (before < target && before + own >= target) found = static_cast<int>(idx);
    }
  } else {
    summary();
    found = cat_locate(sh, row, seg, target, kept.listed, [&](u64 key) { return cat_weight(cat_key_value(key), sc, sh.tab); },
                       [&](const float* l, int idx, u64* w) {
#pragma unroll
      for (int i = 0; i < R::kVec; ++i) {
        const float t = cat_scale(l[i], inv_t);
        const u64 x = cat_weight(t, sc, sh.tab);
        w[i] = bound.kept(t, idx + i) ? x : 0;
      }
    });
  }
  if (!p.logp) {
    if (found >= 0) p.token[r] = found;
    return;
  }
  cat_sync<NT>();                             // the normaliser is known
  if (found >= 0) {
    p.token[r] = found;
    p.logp[r] = static_cast<float>(static_cast<double>(cat_scale(cat_float(row.at(found)), inv_t)) - sh.norm);
  }
}

// A row by one block, whatever it holds.
template <int NT, typename R>
__device__ __noinline__ void cat_search(CatShared<NT>& sh, const CatParams& p, int64_t r, const R& row, u64* seg, const CatRequest& q, bool by_k, const CatScale& sc, float m) {
  constexpr int kVec = R::kVec;
  const int pieces = row.pieces();
  u64 cut = ~0ull;
  if (by_k) cut = cat_refine<false>(sh, row, q.inv_t, sc, cut, q.want, 0.0);
  if (q.by_p) {
    u64 w = 0, none = 0, none2 = 0;
    cat_each<NT>(row, 0, pieces, [&](const float* l, int idx) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float t = cat_scale(l[i], q.inv_t);
        if (cat_key(t, idx + i) <= cut) w += cat_weight(t, sc, sh.tab);
      }
    });
    cat_reduce<NT>(sh, w, none, none2);
    cut = cat_refine<true>(sh, row, q.inv_t, sc, cut, 0, cat_limit(q.top_p, w));
  }
  const float least = cat_least(p, r, m);
  CatBound bound{-INFINITY, INT_MIN};          // (everything that is not masked)
  if (cut != ~0ull) bound = CatBound{cat_key_value(cut), static_cast<int>(static_cast<uint32_t>(cut))};
  if (bound.value < least) bound = CatBound{least, INT_MAX};
  CatKept kept{};
  u64 w = cat_keep<NT>(row, 0, pieces, seg, q.inv_t, sc, sh.tab, bound, kept.n, kept.last);
  cat_reduce<NT>(sh, w, kept.n, kept.last);
  kept.w = w;
  __threadfence();
  cat_finish(sh, p, r, row, seg, q.inv_t, sc, m, kept);
}

// ------------------------------------------------------------------------------------------------------------- kernels
// The largest logit of a part (scaling is monotonic: the largest scaled one is its scaled logit) and how many are not masked; for a
// small top-k also a threshold above which that many tokens of the row lie for certain: this part's share of them, by its threads' own maxima.
// Bound by reading the logits (512 x 131072 fp32 in 49 us, 5.5 TB/s).
template <typename T>
__global__ void __launch_bounds__(kCatThreads) cat_top_kernel(const __grid_constant__ CatParams p) {
  __shared__ uint2 part[kCatWarps];
  const int tid = threadIdx.x, row_i = blockIdx.x / p.w.splits, split = blockIdx.x % p.w.splits;
  const int64_t r = p.r0 + row_i;
  constexpr int kVec = CatRow<T>::kVec, kU = 8;
  griddep_enter();
  const CatRequest q(p, r);
  const CatRow<T> row(p.logits, r, p.V);
  if (q.want || q.by_p) {   // the row's counts start at zero
    uint4* h = reinterpret_cast<uint4*>(p.w.hist + static_cast<int64_t>(row_i) * 2 * kCatBins);
    for (int i = split * kCatThreads + tid; i < 2 * kCatBins / 4; i += p.w.splits * kCatThreads) h[i] = make_uint4(0, 0, 0, 0);
  }
  if (split == 0 && tid == 0) {
    CatState* st = p.w.state + row_i;
    st->ticket[0] = st->ticket[1] = st->list_n = 0; st->mode = CAT_DONE;
  }
  float mine = -INFINITY;
  uint32_t live = 0;
  const int v1 = (split + 1) * p.w.share * (kCatPiece / kVec);
  for (int v0 = split * p.w.share * (kCatPiece / kVec) + tid; v0 < v1; v0 += kU * kCatThreads) {
    uint4 raw[kU];
#pragma unroll
    for (int j = 0; j < kU; ++j) {
      const int v = v0 + j * kCatThreads;
      raw[j] = row.none();
      if (v < v1 && row.whole(v)) raw[j] = row.vec(v);
    }
#pragma unroll
    for (int j = 0; j < kU; ++j) {
      const int v = v0 + j * kCatThreads;
      if (v < v1 && !row.whole(v) && row.some(v)) raw[j] = row.edge(v);
      float l[kVec];
      CatType<T>::unpack(raw[j], l);
#pragma unroll
      for (int i = 0; i < kVec; ++i) { mine = fmaxf(mine, l[i]); live += l[i] > -INFINITY; }
    }
  }
  const uint32_t own = cat_ord(mine);
  uint32_t tau = 0;
  if (q.few) {
    // its share goes by its part of the row (the last one's may be short)
    const int mine_n = min(p.w.share * kCatPiece, max(p.V + row.head - split * p.w.share * kCatPiece, 0));
    const int share = static_cast<int>((static_cast<int64_t>(q.want) * mine_n + p.V - 1) / p.V);
    uint32_t lo = 0, hi = 0xff800000u;   // fewer than share at lo (none are that large), share at hi (if at all)
    while (hi - lo > 1) {
      const uint32_t at = lo + (hi - lo) / 2;
      const int n = __syncthreads_count(own <= at);
      if (n >= share) { hi = at; if (n <= share + share / 16) break; } else lo = at;
    }
    tau = hi;
  }
  const uint32_t top = __reduce_min_sync(0xffffffffu, own);
  live = __reduce_add_sync(0xffffffffu, live);
  if ((tid & 31) == 0) part[tid >> 5] = make_uint2(top, live);
  __syncthreads();
  if (tid == 0) {
    uint32_t a = 0xffffffffu, n = 0;
    for (int i = 0; i < kCatWarps; ++i) { a = min(a, part[i].x); n += part[i].y; }
    p.w.top[static_cast<int64_t>(row_i) * p.w.splits + split] = CatTop{a, tau, n, 0};
  }
}

__device__ __forceinline__ float cat_exp2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// From a row's counts: between which bins top-p ends, and in which top-k; what cat_range_kernel has to look at.
template <bool SHARED, int NT>
__device__ __noinline__ void cat_bins(CatShared<NT>& sh, const uint32_t* hist, CatState* st, const CatRequest& q, uint32_t live, float m, float least) {
  const int tid = threadIdx.x;
  constexpr int kEach = kCatBins / NT;
  const bool by_k = q.want > 0 && static_cast<uint32_t>(q.want) < live;
  const uint32_t k = q.want;
  uint32_t n[kEach], own_n = 0;
  float e[kEach], own_e = 0.0f;
  uint32_t hn[kEach], fn[kEach];
#pragma unroll
  for (int j = 0; j < kEach; j += 2) {
    const uint2 h = cat_get<SHARED>(reinterpret_cast<const uint2*>(hist) + (tid * kEach + j) / 2);
    const uint2 f = cat_get<SHARED>(reinterpret_cast<const uint2*>(hist + kCatBins) + (tid * kEach + j) / 2);
    hn[j] = h.x; hn[j + 1] = h.y; fn[j] = f.x; fn[j + 1] = f.y;
  }
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    n[j] = hn[j];
    const float c = static_cast<float>(hn[j]);
    const float place = tid * kEach + j + (hn[j] ? __fdividef(static_cast<float>(fn[j]) + 0.5f * c, c * (1 << kCatFrac)) : 0.0f);
    e[j] = q.by_p ? c * cat_exp2(-static_cast<float>(kLog2e) / kCatPerUnit * place) : 0.0f;
    own_n += n[j]; own_e += e[j];
  }
  uint32_t cum0 = own_n;
  float mass0 = own_e, all_mass;
  if (tid == 0) { sh.found_a = sh.found_b = sh.found_k = kCatBins; sh.found_prev = -1; }
  cat_block_scan2<NT>(cum0, mass0, sh.scan2, &all_mass);
  cum0 -= own_n; mass0 -= own_e;
  // the bin in which top-k ends, and bounds of the weight that top-p refers to (the thread that holds it looks for it)
  float lo = all_mass, hi = all_mass;
  if (by_k) {
    if (cum0 < k && cum0 + own_n >= k) {
      uint32_t cum = cum0;
      float mass = mass0;
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        if (cum < k && cum + n[j] >= k) {
          sh.found_k = tid * kEach + j;
          const float w = e[j] / n[j] * (k - cum);   // a part of the bin: weights within exp(+-1/64)
          sh.found_lo = mass + w * 0.984f; sh.found_hi = mass + w * 1.016f;
        }
        cum += n[j]; mass += e[j];
      }
    }
    cat_sync<NT>();
    lo = sh.found_lo; hi = sh.found_hi;
  }
  const int bin_k = sh.found_k;
  int bin_a = bin_k, bin_b = bin_k;
  if (q.by_p) {
    // A bin's weight is its count times the weight at its tokens' mean place, to (1/64)^2 / 8 = 2^-15 (its tokens' weights are within
    // exp(-1/64) of each other), 2^-6 / 64 for the places' rounding (their middle is taken), 2^-12 / 64 and 2^-20 for that of the
    // distances, the exponential and the fp32 sums.
    constexpr float kLo = 1.0f - 3.2e-4f, kHi = 1.0f + 3.5e-4f;
    constexpr float kNear = 1.0f + 1e-5f;   // (the sum up to a bin is not the same number at its end and at the next one's start)
    const float lim_lo = q.top_p * lo * kLo, lim_hi = q.top_p * hi * kHi;
    const float end0 = mass0 + own_e;
    if (((mass0 * kHi < lim_lo * kNear || tid == 0) && end0 * kHi >= lim_lo) || ((mass0 * kLo < lim_hi * kNear || tid == 0) && end0 * kLo >= lim_hi)) {
      float mass = mass0;
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int b = tid * kEach + j;
        const float end = j < kEach - 1 ? mass + e[j] : end0;
        // top-p ends in the first bin at whose end its weight is reached: not before a, not behind b
        if ((mass * kHi < lim_lo * kNear || b == 0) && end * kHi >= lim_lo) atomicMin(&sh.found_a, b);
        if ((mass * kLo < lim_hi * kNear || b == 0) && end * kLo >= lim_hi) atomicMin(&sh.found_b, b);
        mass = end;
      }
    }
    cat_sync<NT>();
    bin_a = sh.found_a; bin_b = sh.found_b;
    if (by_k && bin_b >= bin_k) { bin_b = bin_k; bin_a = min(bin_a, bin_k); }   // top-k's end lies among the bins of top-p's
  }
  bool ends = false;
  if (least > -INFINITY) {
    // min-p may end before: in the bin of its least logit, or in the last one before that holds any
    const int bin_m = static_cast<int>(cat_place(m, least, 1.0f) >> kCatFrac);
    if (bin_m <= bin_b && bin_m < kCatBins) {
      ends = true;
      bin_b = bin_m;
      bin_a = min(bin_a, bin_m);
#pragma unroll
      for (int j = 0; j < kEach; ++j) if (n[j] && tid * kEach + j < bin_a) atomicMax(&sh.found_prev, tid * kEach + j);
      cat_sync<NT>();
      if (sh.found_prev >= 0) bin_a = sh.found_prev;
    }
  }
  const bool known = bin_b < kCatBins && bin_a <= bin_b && (!by_k || bin_k < kCatBins || (ends && !q.by_p));
  if (tid == bin_a / kEach || tid == bin_b / kEach || tid == bin_k / kEach) {
    uint32_t cum = cum0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int b = tid * kEach + j;
      if (b == bin_a) sh.at_a = cum;
      if (b == bin_k) sh.at_k = cum;
      cum += n[j];
      if (b == bin_b) sh.at_b = cum;
      if (b == bin_k) sh.end_k = cum;
    }
  }
  cat_sync<NT>();
  const bool apart = by_k && q.by_p && bin_k > bin_b;   // top-k ends in a bin of its own, and top-p refers to what is before
  if (tid == 0) {
    const bool fits = known && sh.at_b - sh.at_a + (apart ? sh.end_k - sh.at_k : 0) <= kCatList;
    st->mode = fits ? CAT_RANGE : CAT_SEARCH;
    st->at_a = sh.at_a; st->n1 = sh.at_b - sh.at_a; st->n_mid = apart ? sh.at_k - sh.at_b : 0;
    st->apart = apart; st->upto = q.by_p && (apart || !by_k); st->ends = ends;
  }
  // (a token lies in a bin before b iff its distance is below b / 64: the places are products by a power of two; no token lies before bin 0, one
  // scaled beyond the range neither, whose distance from the largest is -inf where it is not cut off)
  if (tid == 0) { st->da = bin_a > 0 ? bin_a / kCatPerUnit : -INFINITY; st->db = (bin_b + 1) / kCatPerUnit; st->dk = bin_k / kCatPerUnit; st->de = (bin_k + 1) / kCatPerUnit; }
}

// Counts tokens of pieces [p0, p1) by distance from the largest, and adds up their places: for bins tid * kEach + j.  One addition a token: count and
// place in one word, taken apart before 2^13 tokens could overflow it.
template <int NT, int TAIL, typename R>
__device__ __forceinline__ void cat_count(CatShared<TAIL>& sh, const R& row, int p0, int p1, const CatRequest& q, float m, uint32_t* n, uint32_t* f) {
  constexpr int kVec = R::kVec, kEach = kCatBins / NT, kMost = (1 << 13) / kCatPiece;
  const int tid = threadIdx.x;
  uint32_t* pack = reinterpret_cast<uint32_t*>(sh.list);
  uint2* own = reinterpret_cast<uint2*>(pack) + tid * kEach / 2;
#pragma unroll
  for (int j = 0; j < kEach; j += 2) { own[j / 2] = make_uint2(0, 0); n[j] = n[j + 1] = f[j] = f[j + 1] = 0; }
  for (int q0 = p0; q0 < p1; q0 += kMost) {
    __syncthreads();
    cat_each<NT>(row, q0, min(q0 + kMost, p1), [&](const float* l, int) {
      uint32_t at[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) at[i] = cat_place(m, l[i], q.inv_t);
#pragma unroll
      for (int i = 0; i < kVec; ++i) cat_add_if(pack + (at[i] >> kCatFrac), (1u << kCatPack) | (at[i] & ((1u << kCatFrac) - 1)), at[i], kCatBins << kCatFrac);
    });
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; j += 2) {
      const uint2 x = own[j / 2];
      own[j / 2] = make_uint2(0, 0);
      n[j] += x.x >> kCatPack; f[j] += x.x & ((1u << kCatPack) - 1);
      n[j + 1] += x.y >> kCatPack; f[j + 1] += x.y & ((1u << kCatPack) - 1);
    }
  }
}

// The weights that a row's state asks for: those above the bins in question by piece, and this thread's sums of these and (where top-p refers to
// them) of all before top-k's bin; the tokens of the bins in question go to the list.
template <int NT, int TAIL, typename R>
__device__ __forceinline__ u64 cat_weights(CatShared<TAIL>& sh, const R& row, int p0, int p1, u64* seg, const CatRequest& q, const CatScale& sc, float m, const CatState& st, u64& w_upto) {
  constexpr int kVec = R::kVec;
  const float da = st.da, db = st.db, dk = st.dk, de = st.de;
  const bool apart = st.apart != 0, upto = st.upto != 0;
  if (upto && !apart && sc.base == 0.0f) {
    // top-p without top-k, the common case: every token's weight is wanted
    return cat_sums<NT>(row, p0, p1, seg, [&](const float* l, int idx) -> u64 {
      u64 above = 0;
      bool list = false;
#pragma unroll
      for (int h = 0; h < kVec; h += 4) {   // four exponentials side by side
        float t[4];
        u64 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { t[i] = __fmul_rn(l[h + i], q.inv_t); x[i] = cat_bits(sc.exp0(t[i], sh.tab)); }
        w_upto += x[0] + x[1] + x[2] + x[3] - 4 * kCat256;
        if (!(m - fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])) < db)) continue;   // few tokens make up most of a row's weight
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float d = m - t[i];
          if (d < da) above += x[i] - kCat256;
          list = list || (d < db && !(d < da));
        }
      }
      if (list) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          const float d = m - __fmul_rn(l[i], q.inv_t);
          if (d < db && !(d < da)) sh.append(cat_key(cat_scale(l[i], q.inv_t), idx + i));
        }
      }
      return above;
    });
  } else {
    const float need = upto ? dk : da;
    return cat_sums<NT>(row, p0, p1, seg, [&](const float* l, int idx) -> u64 {
      u64 above = 0;
      bool list = false;
#pragma unroll
      for (int h = 0; h < kVec; h += 4) {
        float t[4];
        bool any = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          t[i] = __fmul_rn(l[h + i], q.inv_t);
          const float d = m - t[i];
          any = any || d < need || (upto && !apart);
          list = list || (d < db && !(d < da)) || (apart && d < de && !(d < dk));
        }
        if (!__any_sync(0xffffffffu, any)) continue;
        u64 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = cat_bits(sc.exp(t[i], sh.tab)) - kCat256;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float d = m - t[i];
          if (d < da) above += x[i];
          if (upto && (!apart || d < dk)) w_upto += x[i];
        }
      }
      if (list) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          const float d = m - __fmul_rn(l[i], q.inv_t);
          if ((d < db && !(d < da)) || (apart && d < de && !(d < dk))) sh.append(cat_key(cat_scale(l[i], q.inv_t), idx + i));
        }
      }
      return above;
    });
  }
}

// A logit at or below every one whose scaled logit is that of `from` or more: neighbours become equals once scaled, and of equals the index decides, so a
// threshold found among the logits as they are has to let in all equals of its own.  They lie within half a unit in the last place of the product
// (2^-24 of it, 2^-150 at least), of which the quotient takes off more.  (Scaling the logits in the pass instead: 73 us, and 67 as it is, at 576 rows of 65536
// bf16 with top-k 200, verified.)
__device__ __forceinline__ float cat_low(float from, float inv_t) {
  const float t = cat_scale(from, inv_t);
  return fmaxf(fminf(from, __fdiv_rd(t - fabsf(t) * 0x1p-21f - 0x1p-148f, inv_t)), -FLT_MAX);   // (nothing is masked from here on up)
}
// Lists the tokens of pieces [p0, p1) whose logit is at least `from`, -FLT_MAX or more.
template <int NT, int TAIL, typename R>
__device__ __forceinline__ void cat_list_from(CatShared<TAIL>& sh, const R& row, int p0, int p1, float from, float inv_t) {
  constexpr int kVec = R::kVec;
  cat_each<NT>(row, p0, p1, [&](const float* l, int idx) {
    float big = l[0];
#pragma unroll
    for (int i = 1; i < kVec; ++i) big = fmaxf(big, l[i]);
    if (big >= from) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) if (l[i] >= from) sh.append(cat_key(cat_scale(l[i], inv_t), idx + i));
    }
  });
}

// Rows without top-k and top-p: everything that is left to do.  Rows with a small top-k: the tokens above the threshold, of which the
// row's last block derives everything.  Other rows: counts by distance from the largest.
template <typename T>
__global__ void __launch_bounds__(kCatThreads, 4) cat_scan_kernel(const __grid_constant__ CatParams p) {
  __shared__ CatShared<kCatThreads> sh;
  constexpr int NT = kCatThreads;
  const int tid = threadIdx.x, row_i = blockIdx.x / p.w.splits, split = blockIdx.x % p.w.splits;
  const int64_t r = p.r0 + row_i;
  constexpr int kVec = CatRow<T>::kVec;
  griddep_enter();
  CatRequest q(p, r);
  const CatRow<T> row(p.logits, r, p.V);
  if (tid == 0) sh.list_n = 0;
  cat_table(sh.tab);
  const CatTop top = cat_tops(sh, p.w, row_i);
  q.at_top(cat_key_value(static_cast<u64>(top.top) << 32));
  if (top.live == 0) {   // nothing is left
    if (split == 0 && tid == 0) {
      if (p.dist) { double* d = p.dist + r * kCatRow; d[0] = -INFINITY; d[1] = INFINITY; d[2] = -1.0; d[3] = 0.0; d[4] = q.inv_t; }
      if (p.u) { p.token[r] = -1; if (p.logp) p.logp[r] = -INFINITY; }
    }
    return;
  }
  const float m = cat_scale(cat_key_value(static_cast<u64>(top.top) << 32), q.inv_t);
  const bool by_k = q.want > 0 && static_cast<uint32_t>(q.want) < top.live;
  CatState* st = p.w.state + row_i;
  u64* seg = p.w.seg + static_cast<int64_t>(row_i) * p.w.pieces;
  const int p0 = split * p.w.share, p1 = min(p0 + p.w.share, row.pieces());
  if (!by_k && !q.by_p) {
    const CatScale sc(m, kCatFloor);
    const float least = cat_least(p, r, m);
    CatKept kept{};
    u64 w = cat_keep<NT>(row, p0, p1, seg, q.inv_t, sc, sh.tab, least > -INFINITY ? CatBound{least, INT_MAX} : CatBound{-INFINITY, INT_MIN}, kept.n, kept.last);
    cat_reduce<NT>(sh, w, kept.n, kept.last);
    u64* tot = p.w.tot + static_cast<int64_t>(row_i) * p.w.splits * 3;
    if (tid == 0) { __stcg(tot + split * 3, w); __stcg(tot + split * 3 + 1, kept.n); __stcg(tot + split * 3 + 2, kept.last); }
    if (!cat_last(sh, &st->ticket[0], p.w.splits)) return;
    w = 0; kept.n = 0; kept.last = 0;
    for (int i = tid; i < p.w.splits; i += kCatThreads) {
      w += __ldcg(tot + i * 3); kept.n += __ldcg(tot + i * 3 + 1);
      const u64 k = __ldcg(tot + i * 3 + 2);
      kept.last = k > kept.last ? k : kept.last;
    }
    cat_reduce<NT>(sh, w, kept.n, kept.last);
    kept.w = w;
    cat_finish(sh, p, r, row, seg, q.inv_t, sc, m, kept);
  } else if (by_k && q.few && top.tau < 0xff800000u) {
    cat_list_from<NT>(sh, row, p0, p1, cat_low(cat_key_value(static_cast<u64>(top.tau) << 32), q.inv_t), q.inv_t);
    u64* list = p.w.list + static_cast<int64_t>(row_i) * kCatList;
    cat_put_list(sh, st, list, p.w.splits);
    if (!cat_last(sh, &st->ticket[0], p.w.splits)) return;
    const CatScale sc(m, kCatFloor);
    CatCut x{};
    CatKept kept{};
    x.n = x.n1 = cat_get_list(sh, st, list, p.w.splits);
    x.by_k = true; x.by_p = q.by_p; x.k = q.want; x.top_p = q.top_p; x.least = cat_least(p, r, m);
    if (x.n <= kCatList && cat_resolve(sh, x, sc, kept)) cat_finish(sh, p, r, row, seg, q.inv_t, sc, m, kept);
    else cat_search(sh, p, r, row, seg, q, by_k, sc, m);   // (many tokens above the threshold: rows in order, many equals)
  } else {
    constexpr int kEach = kCatBins / NT;
    uint32_t n[kEach], f[kEach];               // of bins tid * kEach + j
    cat_count<NT>(sh, row, p0, p1, q, m, n, f);
    uint32_t* hist = p.w.hist + static_cast<int64_t>(row_i) * 2 * kCatBins;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (n[j]) { atomicAdd(hist + tid * kEach + j, n[j]); if (q.by_p) atomicAdd(hist + kCatBins + tid * kEach + j, f[j]); }
    if (!cat_last(sh, &st->ticket[0], p.w.splits)) return;
    cat_bins<false>(sh, hist, st, q, top.live, m, cat_least(p, r, m));
  }
}

// What cat_scan_kernel left: the weights above the bins in question (all weights where top-p refers to the whole row), piece by
// piece, and the tokens of those bins, of which the row's last block derives the cut.  Bound by instructions:
// 47 a token, 62 % of the issue slots taken, the fp64 pipe to 30 % (a third of the time is dependent fp64 steps at 32 warps an SM).
template <typename T>
__global__ void __launch_bounds__(kCatThreads, 4) cat_range_kernel(const __grid_constant__ CatParams p) {
  __shared__ CatShared<kCatThreads> sh;
  constexpr int NT = kCatThreads;
  const int tid = threadIdx.x, row_i = blockIdx.x / p.w.splits, split = blockIdx.x % p.w.splits;
  const int64_t r = p.r0 + row_i;
  griddep_enter();
  CatState* st = p.w.state + row_i;
  const int mode = st->mode;
  if (mode == CAT_DONE || (mode == CAT_SEARCH && split > 0)) return;
  CatRequest q(p, r);
  const CatRow<T> row(p.logits, r, p.V);
  if (tid == 0) sh.list_n = 0;
  cat_table(sh.tab);
  const CatTop top = cat_tops(sh, p.w, row_i);
  q.at_top(cat_key_value(static_cast<u64>(top.top) << 32));
  const float m = cat_scale(cat_key_value(static_cast<u64>(top.top) << 32), q.inv_t);
  const bool by_k = q.want > 0 && static_cast<uint32_t>(q.want) < top.live;
  u64* seg = p.w.seg + static_cast<int64_t>(row_i) * p.w.pieces;
  const CatScale sc(m, kCatFloor);
  if (mode == CAT_SEARCH) {
    cat_search(sh, p, r, row, seg, q, by_k, sc, m);
    return;
  }
  const int p0 = split * p.w.share, p1 = min(p0 + p.w.share, row.pieces());
  u64 w_upto = 0, none = 0, w_above = cat_weights<NT>(sh, row, p0, p1, seg, q, sc, m, *st, w_upto);
  cat_reduce<NT>(sh, w_above, w_upto, none);
  u64* tot = p.w.tot + static_cast<int64_t>(row_i) * p.w.splits * 3;
  if (tid == 0) { __stcg(tot + split * 3, w_above); __stcg(tot + split * 3 + 1, w_upto); }
  u64* list = p.w.list + static_cast<int64_t>(row_i) * kCatList;
  cat_put_list(sh, st, list, p.w.splits);
  if (!cat_last(sh, &st->ticket[1], p.w.splits)) return;
  w_above = 0; w_upto = 0;
  for (int i = tid; i < p.w.splits; i += kCatThreads) { w_above += __ldcg(tot + i * 3); w_upto += __ldcg(tot + i * 3 + 1); }
  cat_reduce<NT>(sh, w_above, w_upto, none);
  CatCut x{};
  CatKept kept{};
  x.n = cat_get_list(sh, st, list, p.w.splits);
  x.n1 = static_cast<int>(st->n1); x.n_above = st->at_a; x.n_mid = st->n_mid; x.w_above = w_above; x.w_upto = w_upto;
  x.by_k = by_k; x.by_p = q.by_p; x.apart = st->apart != 0; x.ends = st->ends != 0; x.k = q.want; x.top_p = q.top_p; x.least = cat_least(p, r, m);
  if (x.n <= kCatList && cat_resolve(sh, x, sc, kept)) cat_finish(sh, p, r, row, seg, q.inv_t, sc, m, kept);
  else cat_search(sh, p, r, row, seg, q, by_k, sc, m);
}

// A row that fits shared memory, by one block: read once, every step without another kernel or another block to wait for.  NB threads pass
// over the row, the first kCatThreads draw the conclusions.
__host__ __device__ constexpr size_t cat_row_fixed() { return (sizeof(CatShared<kCatThreads>) + 15) / 16 * 16; }
template <typename T, int NB>
__global__ void __launch_bounds__(NB, 1024 / NB) cat_row_kernel(const __grid_constant__ CatParams p) {
  extern __shared__ __align__(16) uint8_t cat_dyn[];
  constexpr int NT = kCatThreads;
  CatShared<NT>& sh = *reinterpret_cast<CatShared<NT>*>(cat_dyn);
  u64* const seg = reinterpret_cast<u64*>(cat_dyn + cat_row_fixed());
  uint4* const data = reinterpret_cast<uint4*>(seg + (p.w.pieces + 1) / 2 * 2);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t r = p.r0 + blockIdx.x;
  constexpr int kVec = CatRow<T>::kVec, kU = NB >= 1024 ? 4 : 8;
  griddep_enter();
  CatRequest q(p, r);
  const CatRow<T> from(p.logits, r, p.V);
  const CatHeld<T> row{data, from.head, p.V, (from.head + p.V + kVec - 1) / kVec};
  cat_table(sh.tab);
  if (tid == 0) sh.list_n = 0;
  if (tid < NT) sh.rank[tid] = 0;
  float mine = -INFINITY;
  uint32_t live = 0;
  for (int v0 = tid; v0 < row.vecs; v0 += kU * NB) {
    uint4 raw[kU];
#pragma unroll
    for (int j = 0; j < kU; ++j) if (from.whole(v0 + j * NB)) raw[j] = from.vec(v0 + j * NB);
#pragma unroll
    for (int j = 0; j < kU; ++j) {
      const int v = v0 + j * NB;
      if (v >= row.vecs) break;
      if (!from.whole(v)) raw[j] = from.edge(v);
      data[v] = raw[j];
      float l[kVec];
      CatType<T>::unpack(raw[j], l);
#pragma unroll
      for (int i = 0; i < kVec; ++i) { mine = fmaxf(mine, l[i]); live += l[i] > -INFINITY; }
    }
  }
  const uint32_t own = cat_ord(mine);
  uint32_t top = __reduce_min_sync(0xffffffffu, own), low = __reduce_max_sync(0xffffffffu, mine > -INFINITY ? own : 0u);
  live = __reduce_add_sync(0xffffffffu, live);
  if (lane == 0) { sh.red[warp][0] = (static_cast<u64>(top) << 32) | live; sh.red[warp][1] = low; }
  __syncthreads();
  {
    const u64 x = lane < NB / 32 ? sh.red[lane][0] : 0xffffffffull << 32;
    top = __reduce_min_sync(0xffffffffu, static_cast<uint32_t>(x >> 32));
    live = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(x));
    low = __reduce_max_sync(0xffffffffu, lane < NB / 32 ? static_cast<uint32_t>(sh.red[lane][1]) : 0u);
  }
  const float raw_m = cat_key_value(static_cast<u64>(top) << 32);
  q.at_top(raw_m);
  if (live == 0) {   // nothing is left
    if (tid == 0) {
      if (p.dist) { double* d = p.dist + r * kCatRow; d[0] = -INFINITY; d[1] = INFINITY; d[2] = -1.0; d[3] = 0.0; d[4] = q.inv_t; }
      if (p.u) { p.token[r] = -1; if (p.logp) p.logp[r] = -INFINITY; }
    }
    return;
  }
  const float m = cat_scale(raw_m, q.inv_t);
  const bool by_k = q.want > 0 && static_cast<uint32_t>(q.want) < live;
  const int pieces = row.pieces();
  const CatScale sc(m, kCatFloor);
  CatKept kept{};
  if (!by_k && !q.by_p) {
    const float least = cat_least(p, r, m);
    u64 w = cat_keep<NB>(row, 0, pieces, seg, q.inv_t, sc, sh.tab, least > -INFINITY ? CatBound{least, INT_MAX} : CatBound{-INFINITY, INT_MIN}, kept.n, kept.last);
    cat_reduce<NB>(sh, w, kept.n, kept.last);
    if (tid >= NT) return;
    kept.w = w;
    cat_finish(sh, p, r, row, seg, q.inv_t, sc, m, kept);
    return;
  }
  CatCut x{};
  x.by_k = by_k; x.by_p = q.by_p; x.k = q.want; x.top_p = q.top_p;
  const float width = raw_m - cat_key_value(static_cast<u64>(low) << 32);
  if (by_k && q.few && width < 1e30f) {   // (no infinity among the logits)
    // A threshold above which so many tokens lie for certain, by the threads' own maxima: these in buckets of equal width; the tokens
    // of the buckets that hold that many maxima are listed.
    const float scale = fminf(__fdividef(NT - 1.0f, fmaxf(width, 1e-30f)), FLT_MAX);
    auto bucket = [&](float l) { return fminf((raw_m - l) * scale, static_cast<float>(NT)); };   // (masked: NT, the NaN of infinities too)
    if (mine > -INFINITY) atomicAdd(&sh.rank[min(__float2uint_rd(bucket(mine)), NT - 1u)], 1u);
    __syncthreads();
    if (warp == 0) {
      constexpr int kOwn = NT / 32;
      uint32_t c[kOwn], sum = 0;
#pragma unroll
      for (int j = 0; j < kOwn; ++j) { c[j] = sh.rank[lane * kOwn + j]; sum += c[j]; }
      uint32_t before = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(0xffffffffu, before, o); if (lane >= o) before += y; }
      const uint32_t all = __shfl_sync(0xffffffffu, before, 31), want = static_cast<uint32_t>(q.want);
      if (lane == 0 && all < want) sh.found_a = -1;
      before -= sum;
#pragma unroll
      for (int j = 0; j < kOwn; ++j) { if (before < want && before + c[j] >= want) sh.found_a = lane * kOwn + j; before += c[j]; }
    }
    __syncthreads();
    const int bucket_k = sh.found_a;
    if (bucket_k >= 0) {
      // everything above the bucket's lower end, a little below where that is rounded to
      const float span = __fdividef(static_cast<float>(bucket_k + 1), scale), at = raw_m - span - (span + fabsf(raw_m)) * 1e-6f;
      cat_list_from<NB>(sh, row, 0, pieces, cat_low(fmaxf(at, -FLT_MAX), q.inv_t), q.inv_t);
      __syncthreads();
      x.n = x.n1 = static_cast<int>(min(sh.list_n, kCatList + 1u));
      if (x.n <= kCatList) {
        if (tid >= NT) return;
        x.least = cat_least(p, r, m);
        if (cat_resolve(sh, x, sc, kept)) cat_finish(sh, p, r, row, seg, q.inv_t, sc, m, kept);
        else cat_search(sh, p, r, row, seg, q, by_k, sc, m);
        return;
      }
      __syncthreads();
      if (tid == 0) sh.list_n = 0;
    }
  }
  {
    constexpr int kEach = kCatBins / NB;
    uint32_t n[kEach], f[kEach];
    cat_count<NB>(sh, row, 0, pieces, q, m, n, f);
#pragma unroll
    for (int j = 0; j < kEach; ++j) { sh.hist[tid * kEach + j] = n[j]; sh.hist[kCatBins + tid * kEach + j] = f[j]; }
    __syncthreads();
    if (tid < NT) cat_bins<true>(sh, sh.hist, &sh.state, q, live, m, cat_least(p, r, m));
    __syncthreads();
  }
  const CatState& st = sh.state;
  if (st.mode == CAT_RANGE) {
    u64 w_upto = 0, none = 0, w_above = cat_weights<NB>(sh, row, 0, pieces, seg, q, sc, m, st, w_upto);
    cat_reduce<NB>(sh, w_above, w_upto, none);
    if (tid >= NT) return;
    x.n = static_cast<int>(min(sh.list_n, kCatList + 1u));
    x.n1 = static_cast<int>(st.n1); x.n_above = st.at_a; x.n_mid = st.n_mid; x.w_above = w_above; x.w_upto = w_upto;
    x.apart = st.apart != 0; x.ends = st.ends != 0; x.least = cat_least(p, r, m);
    if (x.n <= kCatList && cat_resolve(sh, x, sc, kept)) {
      cat_finish(sh, p, r, row, seg, q.inv_t, sc, m, kept);
      return;
    }
  }
  if (tid < NT) cat_search(sh, p, r, row, seg, q, by_k, sc, m);
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

// A warp per sequence, a lane per position: logratio = log p(x) - log q(x), accept iff log u <= logratio and p keeps x, n_accept = leading accepts.
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
    ok = ratio > -INFINITY && log(static_cast<double>(p.u[r])) <= ratio;   // (a uniform of 0 accepts no token that p does not keep)
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
  int gamma, rows, V, splits, share, pieces;
  int b0;                                   // first sequence of this launch
  CatView q, p;
  const double *dist_q, *dist_p;
  const int32_t* n_accept;
  const float* w;
  int32_t* x_new;
  CatState* state;                          // [sequences]: tickets, zero between calls
  u64 *seg, *tot;                           // [sequences, pieces], [sequences, splits]
};

// The token of max(0, p - q) at the first rejected position (of p where that is nothing, and at the bonus position): probabilities to 2^-52,
// integer sums by piece over (sequence, part of the row); the last block of a sequence finds the token.
template <typename TQ, typename TP>
__global__ void __launch_bounds__(kCatThreads, 4) cat_resample_kernel(const __grid_constant__ CatResampleParams p) {
  __shared__ CatShared<kCatThreads> sh;
  constexpr int NT = kCatThreads;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, i_b = blockIdx.x / p.splits, split = blockIdx.x % p.splits, b = p.b0 + i_b;
  griddep_enter();
  cat_table(sh.tab);
  __syncthreads();
  const int n = p.n_accept[b];
  const bool residual = n < p.gamma;
  const int64_t rp = static_cast<int64_t>(b) * p.rows + n, rq = static_cast<int64_t>(b) * p.gamma + n;
  if (n < 0 || n >= p.rows || !(p.dist_p[rp * kCatRow + 3] > 0.0)) {
    if (split == 0 && tid == 0) p.x_new[b] = -1;
    return;
  }
  const double* dp = p.dist_p + rp * kCatRow;
  const CatScale sp(dp[0], 42.0f);             // probabilities below 2^-60 count as that: 0 once rounded
  const float inv_p = static_cast<float>(dp[4]);
  const CatBound kept_p{static_cast<float>(dp[1]), static_cast<int>(dp[2])};
  double norm_q = 0.0;
  CatBound kept_q{INFINITY, INT_MIN};
  float inv_q = 1.0f;
  if (residual) {
    const double* dq = p.dist_q + rq * kCatRow;
    if (dq[3] > 0.0) { norm_q = dq[0]; kept_q = CatBound{static_cast<float>(dq[1]), static_cast<int>(dq[2])}; }
    inv_q = static_cast<float>(dq[4]);
  }
  const CatScale sq(norm_q, 42.0f);
  const CatRow<TP> row(p.p, rp, p.V);
  const CatRow<TQ> qrow(p.q, residual ? rq : 0, p.V);
  constexpr int kVec = CatRow<TP>::kVec;
  // a vector's weight; y: the draft's logits of the same tokens.  PLAIN: neither normaliser is so large that it needs CatScale's base, and
  // scaled logits need no bounds either.  The tokens equal to a cut, for which the index decides, are looked for apart; what is not kept gets
  // the least exponent, whose probability rounds to 0.
  auto weights = [&](auto plain, const float* x, const float* y, int idx, bool minus) -> u64 {
    constexpr bool kPlain = decltype(plain)::value;
    u64 sum = 0;
#pragma unroll
    for (int h = 0; h < kVec; h += 4) {     // four exponentials side by side
      double a[4];
      float t[4];
      bool any = false, edge = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = kPlain ? __fmul_rn(x[h + i], inv_p) : cat_scale(x[h + i], inv_p);
        const bool in = v > kept_p.value;
        edge = edge || v == kept_p.value;
        any = any || in;
        t[i] = in ? v : -INFINITY;
      }
      if (edge) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = cat_scale(x[h + i], inv_p);
          if (v == kept_p.value && idx + h + i <= kept_p.idx) { t[i] = v; any = true; }
        }
      }
      if (!__any_sync(0xffffffffu, any)) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = kPlain ? sp.exp0(t[i], sh.tab) : sp.exp(t[i], sh.tab);
      if (minus) {
        edge = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = kPlain ? __fmul_rn(y[h + i], inv_q) : cat_scale(y[h + i], inv_q);
          edge = edge || v == kept_q.value;
          t[i] = v > kept_q.value ? v : -INFINITY;
        }
        if (edge) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = cat_scale(y[h + i], inv_q);
            if (v == kept_q.value && idx + h + i <= kept_q.idx) t[i] = v;
          }
        }
        double d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = kPlain ? sq.exp0(t[i], sh.tab) : sq.exp(t[i], sh.tab);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] -= d[i];
      }
      // 1 added: the bits behind 1's are the value in units of 2^-52; below 1's bits it was negative
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const long long bits = __double_as_longlong(a[i] + 1.0) - 0x3ff0000000000000ll;
        sum += bits > 0 ? static_cast<u64>(bits) : 0;
      }
    }
    return sum;
  };
  auto weights_of = [&](const float* x, const float* y, int idx, bool minus) {
    return sp.base == 0.0f && sq.base == 0.0f ? weights(std::true_type(), x, y, idx, minus) : weights(std::false_type(), x, y, idx, minus);
  };
  // sums of pieces [p0, p1); this thread's own
  u64* seg = p.seg + static_cast<int64_t>(i_b) * p.pieces;
  auto pass = [&](int p0, int p1, bool minus) -> u64 {
    if (minus && sizeof(TQ) == sizeof(TP) && qrow.head == row.head) {   // rows that lie alike: both as vectors
      constexpr int kIts = kCatPiece / (32 * kVec);
      u64 all = 0;
      for (int g = p0 + warp; g < p1; g += kCatWarps) {
        u64 sum = 0;
#pragma unroll
        for (int h = 0; h < kIts; h += 2) {
          uint4 a[2], d[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int v = (g * kIts + h + j) * 32 + lane;
            if (row.whole(v)) { a[j] = row.vec(v); d[j] = qrow.vec(v); }
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int v = (g * kIts + h + j) * 32 + lane;
            if (!row.whole(v)) { a[j] = row.some(v) ? row.edge(v) : row.none(); d[j] = row.some(v) ? qrow.edge(v) : qrow.none(); }
            float x[kVec], y[CatRow<TQ>::kVec > kVec ? CatRow<TQ>::kVec : kVec];
            CatType<TP>::unpack(a[j], x);
            CatType<TQ>::unpack(d[j], y);
            sum += weights_of(x, y, v * kVec - row.head, true);
          }
        }
        all += sum;
        sum = cat_warp_sum(sum);
        if (lane == 0) seg[g] = sum;
      }
      return all;
    }
    return cat_sums<NT>(row, p0, p1, seg, [&](const float* l, int idx) -> u64 {
      float y[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) y[i] = minus && idx + i >= 0 && idx + i < p.V ? cat_float(qrow.base[qrow.head + idx + i]) : -INFINITY;
      return weights_of(l, y, idx, minus);
    });
  };
  const int p0 = split * p.share, p1 = min(p0 + p.share, row.pieces());
  u64 total = pass(p0, p1, residual), none = 0, none2 = 0;
  cat_reduce<NT>(sh, total, none, none2);
  u64* tot = p.tot + static_cast<int64_t>(i_b) * p.splits;
  if (tid == 0) __stcg(tot + split, total);
  uint32_t* ticket = &p.state[i_b].ticket[0];
  if (!cat_last(sh, ticket, p.splits)) return;
  if (tid == 0) *ticket = 0;                // for the next call
  total = 0;
  for (int i = tid; i < p.splits; i += kCatThreads) total += __ldcg(tot + i);
  cat_reduce<NT>(sh, total, none, none2);
  bool minus = residual;
  if (total == 0 && minus) {                // p = q as far as 2^-52 goes: of p, by this block alone
    minus = false;
    total = pass(0, row.pieces(), false);
    cat_reduce<NT>(sh, total, none, none2);
    __threadfence();
  }
  if (tid == 0) p.x_new[b] = -1;
  if (total == 0) return;
  const int found = cat_locate(sh, row, seg, cat_target(p.w[b], total), 0, [](u64) -> u64 { return 0; }, [&](const float* l, int idx, u64* w) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const float t = cat_scale(l[i], inv_p);
      const bool in = static_cast<unsigned>(idx + i) < static_cast<unsigned>(p.V);   // (a summary whose cut is -inf keeps what is masked: outside the row too)
      double a = in && kept_p.kept(t, idx + i) ? sp.exp(t, sh.tab) : 0.0;
      if (minus && a > 0.0) {
        const float tq = cat_scale(cat_float(qrow.base[qrow.head + idx + i]), inv_q);
        if (kept_q.kept(tq, idx + i)) a -= sq.exp(tq, sh.tab);
      }
      w[i] = static_cast<u64>(__double_as_longlong(fmax(a, 0.0) + 1.0) - 0x3ff0000000000000ll);
    }
  });
  if (found >= 0) p.x_new[b] = found;
}

}  // namespace csd
