// Beam search's selection: of all tokens of all beams of a request the `picks` with the largest score + log softmax(logits).
//
// One pass over the logits.  Within a beam the order of the totals is that of the logits, so that a piece of a row is reduced to its largest logit m, the
// sum of e^(logit - m), and its `picks` best logits (beam_scan_kernel); a second, small kernel per request joins the pieces' sums to the beams' logarithms
// and takes the best of the pieces' best (beam_merge_kernel).  Sums are fp32 within a thread and fp64 behind it; totals are compared in fp64, because
// candidates of different beams come near one another.
//
// Finding the best of a piece: no sort.  A thread holds 64 bytes of a tile in registers, and knows the largest element.  The q-th largest of a warp's 32 largest
// ones, q = ceil(picks / 8), is passed by q elements in each of the block's eight warps (or as many as a short row has elements for), so that what is below the least of these cannot be among the best:
// a few dozen elements of the tile are left, and ranked by counting.  From the second tile on the last best element is the bound, and hardly any tile has one above it.
//
// 256 rows of 65536 bf16 logits and sixteen picks take 24 us (1.3 TB/s; 9.3 M warp instructions, 58 % of the issue slots, no unit full: the rest is waiting, at the ends of pieces above all), four rows 6.2, of which
// two launches are 3.  First 71 and 14: packed
// conversions and maxima, four blocks an SM for three, candidates ranked by four threads each.
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/rwkvq.h"
#include "host_util.h"

namespace rwkvq {
namespace bs {

constexpr int kThreads = 256, kWarps = kThreads / 32, kLoads = 4, kMostPicks = 64, kMostBeams = 64, kMostPieces = 64, kMostVocab = 1 << 24;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kList = 256;          // candidates that are ranked by counting; more (many equal ones) are taken out one by one

struct Args {
  const void* logits;
  const float* scores;
  const uint8_t* finished;
  float* next_scores;
  int32_t* parents;
  int32_t* tokens;
  uint8_t* finished_out;
  long long row;
  int requests, beams, vocab, picks, eos, pieces, piece_vecs;
  double* sums;            // [rows][pieces]: sum of e^(logit - m) of the piece
  float* tops;             // [rows][pieces]: m
  uint2* best;             // [rows][pieces][picks]: logit (bits), token; falling, equal ones by rising token, behind the last -inf
};

// A number by which fp32 numbers compare as whole ones; both zeros are one; NaN counts as -inf, which is left out everywhere (0).
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x > -INFINITY ? (b & 0x80000000u ? ~b : b | 0x80000000u) : 0u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ uint64_t order_of(double x) {
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
  return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double value_of(uint64_t o) { return __longlong_as_double((long long)(o >> 63 ? o & ~(1ull << 63) : ~o)); }

__device__ __forceinline__ float exp2_of(float x) {        // 2^x, 2^-126 and less as 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n add.rn.f32x2 z, x, y;\n mov.b64 {%0, %1}, z;\n}" : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mul.rn.f32x2 z, x, y;\n mov.b64 {%0, %1}, z;\n}" : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// Elements as they lie in memory: kPer to a word of 32 bits.
template <typename T> struct Raw;
template <> struct Raw<float> {
  static constexpr int kPer = 1;
  static constexpr uint32_t kNone = 0xFF800000u;        // -inf
  static __device__ __forceinline__ float value(uint32_t w, int) { return __uint_as_float(w); }
  static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }      // of a NaN and a number the number
  static __device__ __forceinline__ uint32_t word(const float* p) { return __float_as_uint(*p); }
};
template <> struct Raw<__half> {
  static constexpr int kPer = 2;
  static constexpr uint32_t kNone = 0xFC00u;
  static __device__ __forceinline__ float value(uint32_t w, int i) { return __half2float(__ushort_as_half((unsigned short)(i ? w >> 16 : w & 0xFFFFu))); }
  static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) {
    const __half2 m = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&m);
  }
  static __device__ __forceinline__ uint32_t word(const __half* p) { return __half_as_ushort(*p); }
};
template <> struct Raw<__nv_bfloat16> {
  static constexpr int kPer = 2;
  static constexpr uint32_t kNone = 0xFF80u;
  static __device__ __forceinline__ float value(uint32_t w, int i) { return __uint_as_float(i ? w & 0xFFFF0000u : w << 16); }
  static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) {
    const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&m);
  }
  static __device__ __forceinline__ uint32_t word(const __nv_bfloat16* p) { return __bfloat16_as_ushort(*p); }
};

// The 16 bytes that begin `skew` bytes behind those of a, which b follows.
__device__ __forceinline__ uint4 joined(const uint4& a, const uint4& b, uint32_t skew) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (skew & 8)
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  if (skew & 4)
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  const uint32_t bits = (skew & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}

// The q-th largest of a warp's 32 numbers (0 where fewer are above 0).
__device__ __forceinline__ uint32_t qth_of_warp(uint32_t x, int q) {
  uint32_t top = 0;
  for (int i = 0; i < q; ++i) {
    top = __reduce_max_sync(~0u, x);
    const uint32_t who = __ballot_sync(~0u, x == top);
    if ((threadIdx.x & 31) == (uint32_t)__ffs(who) - 1) x = 0;
  }
  return top;
}

// Candidates of a block: keys that are all different, larger = better.  High half: the value's order; low half: ~index.
struct Best {
  uint64_t list[kList];
  uint64_t ranked[kMostPicks];
  uint32_t warp_top[kWarps], warp_low[kWarps];
  int count;
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) beam_scan_kernel(const Args a) {
  using R = Raw<T>;
  constexpr int kWords = 4 * kLoads, kHold = kWords * R::kPer, V = 4 * R::kPer;
  __shared__ Best b;
  __shared__ float warp_m[kWarps];
  __shared__ double warp_s[kWarps];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");        // only now: the second kernel reads the beams' scores before this one is done
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long r = blockIdx.y;
  const float score = a.scores[r];
  const bool ended = a.finished && a.finished[r];
  const T* row = static_cast<const T*>(a.logits) + r * a.row;
  // Vectors of 16 bytes' elements, counted from the row's first, wherever that lies: rows with the same logits have the same sum to the last bit, and their beams tie.
  // A row that begins `skew` bytes behind a boundary of 16 has its vectors put together from two aligned ones.
  const uint32_t skew = (uint32_t)((uintptr_t)row & 15);
  const uint4* const vecs = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(row) - skew);
  const int n_vecs = (a.vocab + V - 1) / V;
  const int v0 = min((int)blockIdx.x * a.piece_vecs, n_vecs), v1 = min(v0 + a.piece_vecs, n_vecs);
  // warps that have an element for each lane in the first tile
  const int full = min(kWarps, (v1 - v0) / 32), q = full > 0 ? (a.picks + full - 1) / full : 33;
  auto load = [&](int t0, uint4 (&w)[kLoads]) {
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      const int v = t0 + l * kThreads + tid, first = v * V;
      if (skew == 0 && v < v1 && first + V <= a.vocab) {
        w[l] = vecs[v];
      } else if (skew != 0 && v < v1 && v > 0 && first + 2 * V <= a.vocab) {
        w[l] = joined(vecs[v], vecs[v + 1], skew);
      } else {
        // the ends of a row: an element at a time, all on their way together
        uint32_t e[V];
#pragma unroll
        for (int j = 0; j < V; ++j) e[j] = v < v1 && first + j < a.vocab ? R::word(row + first + j) : R::kNone;
        if constexpr (R::kPer == 2) w[l] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4 % V] | e[5 % V] << 16, e[6 % V] | e[7 % V] << 16);
        else w[l] = make_uint4(e[0], e[1], e[2], e[3]);
      }
    }
  };
  // The best of the elements [e0, e1) that are above `floor` to b.list behind the `have` best so far, one after another, where there are too many to count (equal
  // ones): the owner of the last one taken looks for its next.  Returns how many there are then.  All threads.
  auto one_by_one = [&](int e0, int e1, int have, float floor) {
    uint64_t key = 0;
    auto next = [&](uint64_t below) {
      key = 0;
#pragma unroll 1
      for (int e = e0 + tid; e < e1; e += kThreads) {
        const float x = R::value(R::word(row + e), 0);
        const uint64_t k = x > floor ? (uint64_t)order_of(x) << 32 | (uint32_t)~e : 0ull;
        if (k < below && k > key) key = k;
      }
    };
    next(~0ull);
    __syncthreads();
    int n = have;
    if (tid < have) b.list[tid] = b.ranked[tid];
    for (int i = 0; i < a.picks; ++i) {
      const uint32_t hi = __reduce_max_sync(~0u, (uint32_t)(key >> 32));
      const uint32_t lo = __reduce_max_sync(~0u, (uint32_t)(key >> 32) == hi ? (uint32_t)key : 0u);
      if (lane == 0) { b.warp_top[warp] = hi; b.warp_low[warp] = lo; }
      __syncthreads();
      uint64_t best = 0;
      for (int k = 0; k < kWarps; ++k) best = max(best, (uint64_t)b.warp_top[k] << 32 | b.warp_low[k]);
      if (best == 0) break;
      if (key == best) { b.list[have + i] = best; next(best); }
      n = have + i + 1;
      __syncthreads();
    }
    __syncthreads();
    return n;
  };
  float m = -INFINITY, s = 0.f;
  int have = 0;                     // ranked[0 .. have) are the best so far
  float floor = -INFINITY;          // value of ranked[picks - 1], once there are as many: later elements have to be above it
  int since = v0;                   // first vector whose candidates are not among these
  uint4 ahead[kLoads] = {};
  int k = 0;                        // tiles so far
  int raise = 1;                    // when the bound is raised
  const int spread = max(2, 64 / a.picks);
  for (int t0 = v0 - kThreads * kLoads; t0 < v1; t0 += kThreads * kLoads, ++k) {
    const int t1 = t0 + kThreads * kLoads;
    uint32_t w[kWords];
#pragma unroll
    for (int l = 0; l < kLoads; ++l) { w[4 * l] = ahead[l].x; w[4 * l + 1] = ahead[l].y; w[4 * l + 2] = ahead[l].z; w[4 * l + 3] = ahead[l].w; }
    if (t1 < v1) load(t1, ahead);
    if (k == 0) {
      if (!(score > -INFINITY && score < INFINITY) || ended) return;      // its candidates do not come from its logits
      continue;
    }
    uint32_t most[kLoads];
#pragma unroll
    for (int l = 0; l < kLoads; ++l) most[l] = R::most(R::most(w[4 * l], w[4 * l + 1]), R::most(w[4 * l + 2], w[4 * l + 3]));
    float top = -INFINITY;
    {
      const uint32_t x = R::most(R::most(most[0], most[1]), R::most(most[2], most[3]));
      top = fmaxf(top, fmaxf(R::value(x, 0), R::value(x, R::kPer - 1)));
    }
    if (top > -INFINITY) {
      if (top > m) { s *= exp2_of((m - top) * kLog2e); m = top; }
      const float2 shift = make_float2(-m, -m), scale = make_float2(kLog2e, kLog2e);
      float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
      for (int j = 0; j < kHold; j += 2) {
        // the difference first: m may be large, up to the type's lowest value
        const float2 x = mul2(add2(make_float2(R::value(w[j / R::kPer], 0), R::value(w[(j + 1) / R::kPer], R::kPer - 1)), shift), scale);
        part[j / 2 & 1] = add2(part[j / 2 & 1], make_float2(exp2_of(x.x), exp2_of(x.y)));
      }
      part[0] = add2(part[0], part[1]);
      float sum = part[0].x + part[0].y;
      if (!(sum < INFINITY)) {      // a NaN among the logits, which does not count, or an infinity, beside which only others do
        sum = 0.f;
#pragma unroll 1
        for (int e = 0; e < kHold; ++e) {
          const int at = (t0 + (e / V) * kThreads + tid) * V + e % V;
          const float x = at < min(v1 * V, a.vocab) ? R::value(R::word(row + at), 0) : -INFINITY;
          sum += x == m ? 1.f : x < m ? exp2_of((x - m) * kLog2e) : 0.f;
        }
      }
      s += sum;
    }
    // The first tile finds a bound; those behind it add what is above it, and the bound is raised where the tiles are `spread` times as many as at the last time, when
    // about as many times the places have come together.
    float least = -INFINITY;
    if (k == 1) {
      const uint32_t low = q <= 32 ? qth_of_warp(order_of(top), q) : 0u;
      if (lane == 0) b.warp_low[warp] = low;
      if (tid == 0) b.count = 0;
      __syncthreads();
      uint32_t l = ~0u;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) l = i < max(full, 1) ? min(l, b.warp_low[i]) : l;
      if (l) least = value_of(l);
    }
    if (top > floor && top >= least) {
#pragma unroll
      for (int l = 0; l < kLoads; ++l) {
        const float here = fmaxf(R::value(most[l], 0), R::value(most[l], R::kPer - 1));
        if (!(here > floor && here >= least)) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float x = R::value(w[4 * l + j / R::kPer], j % R::kPer);
          if (x > floor && x >= least) {
            const int at = atomicAdd(&b.count, 1);
            const uint32_t index = (uint32_t)((t0 + l * kThreads + tid) * V + j);
            if (at < kList) b.list[at] = (uint64_t)order_of(x) << 32 | (uint32_t)~index;
          }
        }
      }
    }
    if (k < raise && t1 < v1) continue;
    raise = k * spread;
    __syncthreads();
    int n = b.count;
    if (n > kList) n = one_by_one(since * V, min(min(t1, v1) * V, a.vocab), have, floor);
    since = t1;
    // ranked: how many are above each, counted by four threads
    for (int i0 = 0; i0 < n; i0 += kThreads / 4) {
      const int i = i0 + tid / 4;
      const uint64_t mine = b.list[min(i, n - 1)];
      int above = 0;
#pragma unroll 4
      for (int j = tid & 3; j < n; j += 4) above += b.list[j] > mine ? 1 : 0;
      above += __shfl_xor_sync(~0u, above, 1);
      above += __shfl_xor_sync(~0u, above, 2);
      if (i < n && above < a.picks && (tid & 3) == 0) b.ranked[above] = mine;
    }
    __syncthreads();
    have = min(n, a.picks);
    if (have == a.picks) floor = value_of((uint32_t)(b.ranked[have - 1] >> 32));
    if (t1 < v1) {
      if (tid < have) b.list[tid] = b.ranked[tid];
      if (tid == 0) b.count = have;
      __syncthreads();
    }
  }
  // the block's sum
  float M = m;
#pragma unroll
  for (int o = 16; o > 0; o /= 2) M = fmaxf(M, __shfl_xor_sync(~0u, M, o));
  if (lane == 0) warp_m[warp] = M;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWarps; ++i) M = fmaxf(M, warp_m[i]);
  double S = m > -INFINITY ? (double)(m == M ? s : s * exp2_of((m - M) * kLog2e)) : 0.0;
#pragma unroll
  for (int o = 16; o > 0; o /= 2) S += __shfl_xor_sync(~0u, S, o);
  if (lane == 0) warp_s[warp] = S;
  __syncthreads();
  const long long piece = r * a.pieces + blockIdx.x;
  if (tid == 0) {
    S = 0.0;
    for (int i = 0; i < kWarps; ++i) S += warp_s[i];
    a.sums[piece] = S;
    a.tops[piece] = M;
  }
  if (tid < a.picks) {
    const uint64_t k = tid < have ? b.ranked[tid] : 0ull;
    a.best[piece * a.picks + tid] = make_uint2(k ? __float_as_uint(value_of((uint32_t)(k >> 32))) : 0xFF800000u, ~(uint32_t)k);
  }
}

// One request: the beams' logarithms, then the best of all candidates: by their totals, and among equal ones by beam, logit (fp64 totals of tiny logits can be equal
// where these are not) and token, which are one number, larger = better.
__device__ __forceinline__ uint64_t place_of(int k, float logit, uint32_t token) {
  return (uint64_t)(kMostBeams - 1 - k) << 56 | (uint64_t)order_of(logit) << 24 | (kMostVocab - 1 - token);
}
__device__ __forceinline__ int beam_of(uint64_t place) { return kMostBeams - 1 - (int)(place >> 56); }
__device__ __forceinline__ int token_of(uint64_t place) { return kMostVocab - 1 - (int)(place & (kMostVocab - 1)); }
struct __align__(16) Candidate { uint64_t total, place; };        // total: its order
__device__ __forceinline__ bool above(const Candidate& x, const Candidate& y) { return (x.total > y.total) | ((x.total == y.total) & (x.place > y.place)); }

__global__ void __launch_bounds__(kThreads) beam_merge_kernel(const Args a) {
  constexpr int kHeld = 2;                         // candidates that a thread keeps; those behind them are made anew where they are needed
  __shared__ double offset[kMostBeams], most[kMostBeams];      // score - log(sum) and m, of which a logit's total is offset + (logit - m); of a beam that ended, its score
  __shared__ int kind[kMostBeams];                 // 0: no candidates, 1: of its logits, 2: ended, 3: of its logits, the largest of which is +inf
  __shared__ int alive[kMostBeams], n_alive;       // beams of kind 1 to 3
  __shared__ Candidate list[kList], warp_best[kWarps];
  __shared__ uint32_t warp_low[kWarps];
  __shared__ int count;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K = a.beams, P = a.picks;
  const long long r0 = (long long)blockIdx.x * K;
  // what the beams are is known before the scan is done, which let this kernel begin when all in front of it was
  if (warp == 0) {
    int kinds[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = lane + 32 * h;
      const float score = k < K ? a.scores[r0 + k] : INFINITY;
      kinds[h] = !(score > -INFINITY && score < INFINITY) ? 0 : a.finished && a.finished[r0 + k] ? 2 : 1;
      if (k < K) { kind[k] = kinds[h]; offset[k] = (double)score; }
    }
    const uint32_t bx = __ballot_sync(~0u, kinds[0]), by = __ballot_sync(~0u, kinds[1]), low = (1u << lane) - 1;
    if (kinds[0]) alive[__popc(bx & low)] = lane;
    if (kinds[1]) alive[__popc(bx) + __popc(by & low)] = lane + 32;
    if (lane == 0) { n_alive = __popc(bx) + __popc(by); count = 0; }
  }
  __syncthreads();
  // Candidate c of all: place c % (pieces * P) of the c / (pieces * P)-th beam that has any.  Each warp takes its candidates from all lists alike: neighbouring ones,
  // of one list, go to different warps; `full` warps have something for each lane.
  const int each = a.pieces * P, all = n_alive * each, full = max(1, min(kWarps, all / 32)), step = 32 * full;
  const int c0 = warp < full ? lane * full + warp : all;
  auto fetch = [&](int c, int& k) {
    const int l = c / each;
    k = alive[l];
    return kind[k] == 2 ? make_uint2(0u, c - l * each) : a.best[(r0 + k) * each + (c - l * each)];
  };
  auto candidate = [&](int k, const uint2& b, Candidate& x) {
    if (kind[k] == 2) {
      x.total = order_of(offset[k]); x.place = place_of(k, 0.f, (uint32_t)a.eos);
      return b.y == 0;
    }
    const float v = __uint_as_float(b.x);
    x.total = order_of(kind[k] == 3 ? offset[k] : offset[k] + ((double)v - most[k])); x.place = place_of(k, v, b.y);
    return kind[k] == 3 ? v == INFINITY : v > -INFINITY;
  };
  asm volatile("griddepcontrol.wait;" ::: "memory");
  uint2 held[kHeld];
  int held_k[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (c0 + i * step < all) held[i] = fetch(c0 + i * step, held_k[i]);
  // All have read what their beams are, which is written below; a barrier takes less than beams of which that stands elsewhere (32 requests 23.9 us, 24.7; odd vocabulary 11.1, 11.8).
  __syncthreads();
  for (int l = warp; l < n_alive; l += kWarps) {
    const int k = alive[l];
    if (kind[k] != 1) continue;
    const long long at = (r0 + k) * a.pieces;
    const float m0 = lane < a.pieces ? a.tops[at + lane] : -INFINITY, m1 = lane + 32 < a.pieces ? a.tops[at + lane + 32] : -INFINITY;
    const double s0 = lane < a.pieces ? a.sums[at + lane] : 0.0, s1 = lane + 32 < a.pieces ? a.sums[at + lane + 32] : 0.0;
    const float M = value_of(max(__reduce_max_sync(~0u, order_of(m0)), __reduce_max_sync(~0u, order_of(m1))));
    const bool some = __any_sync(~0u, m0 > -INFINITY || m1 > -INFINITY);
    double S = 0.0;
    if (m0 > -INFINITY) S += m0 == M ? s0 : s0 * (double)exp2_of((m0 - M) * kLog2e);
    if (m1 > -INFINITY) S += m1 == M ? s1 : s1 * (double)exp2_of((m1 - M) * kLog2e);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) S += __shfl_xor_sync(~0u, S, o);
    if (lane == 0 && some) {
      offset[k] -= log(S);
      most[k] = (double)M;
      if (M == INFINITY) kind[k] = 3;
    }
  }
  __syncthreads();
  // As in a piece: a warp's q-th best are passed by q candidates, those of all full warps by enough.  By the total rounded to fp32, which keeps the order; a total that fp32 has no
  // room for (a score and a mask of the type's lowest value) is a candidate all the same, above none at all.
  auto coarse = [](const Candidate& y) { return max(order_of((float)value_of(y.total)), 1u); };
  Candidate x[kHeld];
  uint32_t order[kHeld], top = 0, bound = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    order[i] = c0 + i * step < all && candidate(held_k[i], held[i], x[i]) ? coarse(x[i]) : 0u;
    top = max(top, order[i]);
  }
#pragma unroll 1
  for (int c = c0 + kHeld * step; c < all; c += step) {
    Candidate y;
    int k;
    const uint2 b = fetch(c, k);
    if (candidate(k, b, y)) top = max(top, coarse(y));
  }
  const int q = (P + full - 1) / full;
  if (q <= 32 && all >= 32) {
    const uint32_t low = qth_of_warp(top, q);
    if (lane == 0) warp_low[warp] = low;
    __syncthreads();
    bound = ~0u;
    for (int i = 0; i < full; ++i) bound = min(bound, warp_low[i]);
  }
  auto keep = [&](const Candidate& y) {
    const int at = atomicAdd(&count, 1);
    if (at < kList) list[at] = y;
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (order[i] && order[i] >= bound) keep(x[i]);
#pragma unroll 1
  for (int c = c0 + kHeld * step; c < all; c += step) {
    Candidate y;
    int k;
    const uint2 b = fetch(c, k);
    if (candidate(k, b, y) && coarse(y) >= bound) keep(y);
  }
  __syncthreads();
  int n = count;
  if (n > kList) {
    // too many to count (equal ones): one after another
    __syncthreads();
    Candidate mine, last = {~0ull, ~0ull};
    auto next = [&]() {
      mine = Candidate{0, 0};
#pragma unroll 1
      for (int c = c0; c < all; c += step) {
        Candidate y;
        int k;
        const uint2 b = fetch(c, k);
        if (candidate(k, b, y) && above(last, y) && above(y, mine)) mine = y;
      }
    };
    next();
    for (n = 0; n < P; ++n) {
      Candidate y = mine;
#pragma unroll
      for (int o = 16; o > 0; o /= 2) {
        const Candidate z = {__shfl_xor_sync(~0u, y.total, o), __shfl_xor_sync(~0u, y.place, o)};
        if (above(z, y)) y = z;
      }
      if (lane == 0) warp_best[warp] = y;
      __syncthreads();
      y = warp_best[0];
      for (int i = 1; i < kWarps; ++i)
        if (above(warp_best[i], y)) y = warp_best[i];
      if (y.place == 0) break;
      const bool taken = mine.place == y.place && mine.total == y.total;
      last = y;
      if (taken) next();
      if (tid == 0) list[n] = y;
      __syncthreads();
    }
    __syncthreads();
  }
  auto put = [&](int i, float total, int k, int v) {
    const long long o = (long long)blockIdx.x * P + i;
    a.next_scores[o] = total;
    a.parents[o] = k;
    a.tokens[o] = v;
    if (a.finished_out) a.finished_out[o] = (a.finished && a.finished[r0 + k]) || v == a.eos;
  };
  for (int i0 = 0; i0 < n; i0 += kThreads / 4) {
    const int i = i0 + tid / 4;
    const Candidate mine = list[min(i, n - 1)];
    int better = 0;
#pragma unroll 4
    for (int j = tid & 3; j < n; j += 4) better += above(list[j], mine) ? 1 : 0;
    better += __shfl_xor_sync(~0u, better, 1);
    better += __shfl_xor_sync(~0u, better, 2);
    if (i < n && better < P && (tid & 3) == 0) put(better, (float)value_of(mine.total), beam_of(mine.place), token_of(mine.place));
  }
  if (n < P && tid >= n && tid < P) {
    // fewer candidates than places (all of them in the list): what is left has probability zero, lowest beam and token first
    int k = 0, v = 0;
    for (int skip = tid - n;; ) {
      bool taken = false;
      for (int j = 0; j < n; ++j) taken |= beam_of(list[j].place) == k && token_of(list[j].place) == v;
      if (!taken && skip-- == 0) break;
      if (++v == a.vocab) { v = 0; ++k; }
    }
    put(tid, -INFINITY, k, v);
  }
}

// Pieces of a row: as many blocks as the SMs hold at once, but no piece so short that a block has less than a tile's share of work.
struct Plan { int pieces; size_t bytes, off_tops, off_best; };
Plan plan_of(int requests, int beams, int vocab, int picks) {
  Plan p;
  const long long rows = (long long)requests * beams;
  const int least = 2048;
  const long long want = std::max<long long>(1, 4ll * sm_count() / rows);
  p.pieces = (int)std::min<long long>({want, (vocab + least - 1) / least, kMostPieces});
  // rows * pieces is at most either of these, and both grow with the sizes: what is enough for a call is enough for smaller ones
  const size_t n = (size_t)std::min(std::max<long long>(rows, 4ll * sm_count()), rows * std::min(kMostPieces, (vocab + least - 1) / least));
  p.off_tops = n * 8;
  p.off_best = round_up_sz(p.off_tops + n * 4, 16);
  p.bytes = p.off_best + n * picks * 8;
  return p;
}

template <typename T>
cudaError_t launch(Args a, cudaStream_t s) {
  const int V = 4 * Raw<T>::kPer;
  a.piece_vecs = ((a.vocab + V - 1) / V + a.pieces - 1) / a.pieces;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.pieces, (unsigned)(a.requests * a.beams)); cfg.blockDim = dim3(kThreads); cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, beam_scan_kernel<T>, a);
  if (e != cudaSuccess) return e;
  cfg.gridDim = dim3((unsigned)a.requests);
  return cudaLaunchKernelEx(&cfg, beam_merge_kernel, a);
}

bool sizes_ok(int requests, int beams, int vocab, int picks) { return requests > 0 && beams > 0 && vocab > 0 && picks > 0 && (long long)picks <= (long long)beams * vocab; }
bool sizes_supported(int requests, int beams, int vocab, int picks) {
  return beams <= kMostBeams && picks <= kMostPicks && vocab <= kMostVocab && (long long)requests * beams <= 65535;
}

}  // namespace bs
}  // namespace rwkvq

using namespace rwkvq;

extern "C" {

size_t rwkvq_beam_select_workspace_bytes(int requests, int beams, int vocab, int picks) {
  if (!bs::sizes_ok(requests, beams, vocab, picks) || !bs::sizes_supported(requests, beams, vocab, picks)) return 0;
  return bs::plan_of(requests, beams, vocab, picks).bytes;
}

rwkvq_status rwkvq_beam_select(const rwkvq_beam_select_args* args, void* workspace, size_t workspace_bytes, void* stream) {
  if (!args) return RWKVQ_EINVAL;
  const rwkvq_beam_select_args& g = *args;
  const int es = g.dtype == RWKVQ_F32 ? 4 : g.dtype == RWKVQ_F16 || g.dtype == RWKVQ_BF16 ? 2 : 0;
  if (es == 0 || !g.logits || !g.scores || !g.next_scores || !g.parents || !g.tokens) return RWKVQ_EINVAL;
  if (!bs::sizes_ok(g.requests, g.beams, g.vocab, g.picks)) return RWKVQ_EINVAL;
  if ((g.finished || g.finished_out) && (g.eos < 0 || g.eos >= g.vocab)) return RWKVQ_EINVAL;
  if (!bs::sizes_supported(g.requests, g.beams, g.vocab, g.picks)) return RWKVQ_EUNSUPPORTED;
  if ((long long)g.requests * g.beams > 1 && g.logits_row < g.vocab) return RWKVQ_EINVAL;
  // the outputs are written while other requests' inputs may not have been read
  if (g.next_scores == g.scores || (g.finished && g.finished_out == g.finished)) return RWKVQ_EINVAL;
  if (reinterpret_cast<uintptr_t>(g.logits) % es || reinterpret_cast<uintptr_t>(g.scores) % 4 || reinterpret_cast<uintptr_t>(g.next_scores) % 4 ||
      reinterpret_cast<uintptr_t>(g.parents) % 4 || reinterpret_cast<uintptr_t>(g.tokens) % 4)
    return RWKVQ_EALIGN;
  const bs::Plan l = bs::plan_of(g.requests, g.beams, g.vocab, g.picks);
  if (!workspace || workspace_bytes < l.bytes) return RWKVQ_ENOMEM;
  if (!aligned16(workspace)) return RWKVQ_EALIGN;
  bs::Args a;
  a.logits = g.logits; a.scores = g.scores; a.finished = g.finished; a.next_scores = g.next_scores; a.parents = g.parents; a.tokens = g.tokens;
  a.finished_out = g.finished_out; a.row = (long long)g.requests * g.beams > 1 ? g.logits_row : 0;
  a.requests = g.requests; a.beams = g.beams; a.vocab = g.vocab; a.picks = g.picks; a.eos = g.eos; a.pieces = l.pieces;
  uint8_t* w = static_cast<uint8_t*>(workspace);
  a.sums = reinterpret_cast<double*>(w);
  a.tops = reinterpret_cast<float*>(w + l.off_tops);
  a.best = reinterpret_cast<uint2*>(w + l.off_best);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (g.dtype == RWKVQ_F32) return cuda_status(bs::launch<float>(a, s));
  if (g.dtype == RWKVQ_F16) return cuda_status(bs::launch<__half>(a, s));
  return cuda_status(bs::launch<__nv_bfloat16>(a, s));
}

}  // extern "C"
