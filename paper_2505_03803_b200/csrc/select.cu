// Beam search's selection: of all tokens of all beams of a request the `picks` with the largest score + log softmax(logits).
//
// One pass over the logits.  Within a beam the order of the totals is that of the logits, so that a piece of a row is reduced to its largest logit m, the
// sum of e^(logit - m), and its `picks` best logits (beam_scan_kernel); a second, small kernel per request joins the pieces' sums to the beams' logarithms
// and takes the best of the pieces' best (beam_merge_kernel).  Sums are fp32 within a thread and fp64 behind it; totals are compared in fp64, because
// candidates of different beams come near one another.
//
// Finding the best of a piece: no sort.  A thread holds 32 elements of a tile in registers, and knows the largest.  The q-th largest of a warp's 32 largest
// ones, q = ceil(picks / 8), is passed by q elements in each of the block's eight warps, so that what is below the least of these eight cannot be among the best:
// a few dozen elements of 8192 are left, and ranked by counting.  From the second tile on the last best element is the bound, and hardly any tile has one above it.
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/rwkvq.h"
#include "host_util.h"

namespace rwkvq {
namespace bs {

constexpr int kThreads = 256, kWarps = kThreads / 32, kHold = 32, kTile = kThreads * kHold, kMostPicks = 64, kMostBeams = 64, kMostPieces = 64, kMostVocab = 1 << 24;
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
  int* counts;             // [rows][pieces]: best logits that there are
  uint2* best;             // [rows][pieces][picks]: logit (bits), token; falling, equal ones by rising token
};

// A number by which fp32 numbers compare as whole ones; NaN counts as -inf, which is left out everywhere (0).
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return x > -INFINITY ? (b & 0x80000000u ? ~b : b | 0x80000000u) : 0u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }

template <typename T> struct Raw;
template <> struct Raw<float> {
  static constexpr int kVec = 4;
  static __device__ __forceinline__ void values(const uint4& w, float* f) {
    f[0] = __uint_as_float(w.x); f[1] = __uint_as_float(w.y); f[2] = __uint_as_float(w.z); f[3] = __uint_as_float(w.w);
  }
};
template <> struct Raw<__half> {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ void values(const uint4& w, float* f) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&v[i]));
      f[2 * i] = p.x; f[2 * i + 1] = p.y;
    }
  }
};
template <> struct Raw<__nv_bfloat16> {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ void values(const uint4& w, float* f) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(v[i] << 16); f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u); }
  }
};
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

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

// Candidates of a block: keys that are all different, larger = better.  hi: the value's order; lo: ~index.
struct Best {
  uint64_t list[kList + kMostPicks];
  uint64_t ranked[kMostPicks];
  uint32_t warp_top[kWarps], warp_low[kWarps];
  int count, owner;
};

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

// The first `picks` of the n keys in list, falling, to ranked, and the number of them.  All threads; n <= kList + kMostPicks.
__device__ __forceinline__ int rank(Best& b, int n, int picks) {
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t mine = b.list[i];
    int above = 0;
    for (int j = 0; j < n; ++j) above += b.list[j] > mine;
    if (above < picks) b.ranked[above] = mine;
  }
  __syncthreads();
  return min(n, picks);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) beam_scan_kernel(const Args a) {
  constexpr int V = Raw<T>::kVec, kLoads = kHold / V;
  __shared__ Best b;
  __shared__ float warp_m[kWarps];
  __shared__ double warp_s[kWarps];
  asm volatile("griddepcontrol.launch_dependents;");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long r = blockIdx.y;
  const float score = a.scores[r];
  if (!(score > -INFINITY && score < INFINITY) || (a.finished && a.finished[r])) return;      // its candidates do not come from its logits
  const T* row = static_cast<const T*>(a.logits) + r * a.row;
  // Vectors of 16 bytes' elements, counted from the row's first, wherever that lies: rows with the same logits have the same sum to the last bit, and their beams tie.
  // A row that begins `skew` bytes behind a boundary of 16 has its vectors put together from two aligned ones.
  const uint32_t skew = (uint32_t)((uintptr_t)row & 15);
  const uint4* const vecs = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(row) - skew);
  const int n_vecs = (a.vocab + V - 1) / V;
  const int v0 = min((int)blockIdx.x * a.piece_vecs, n_vecs), v1 = min(v0 + a.piece_vecs, n_vecs);
  const int q = (a.picks + kWarps - 1) / kWarps;
  float m = -INFINITY, s = 0.f;
  int have = 0;                     // ranked[0 .. have) are the best so far
  uint32_t floor_order = 0;         // order of ranked[picks - 1], once there are as many: later elements have to be above it
  for (int t0 = v0; t0 < v1; t0 += kThreads * kLoads) {
    float f[kHold];
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      const int v = t0 + l * kThreads + tid, first = v * V;
      float* x = f + l * V;
      if (skew == 0 && v < v1 && first + V <= a.vocab) {
        Raw<T>::values(__ldg(vecs + v), x);
      } else if (skew != 0 && v < v1 && v > 0 && first + 2 * V <= a.vocab) {
        Raw<T>::values(joined(__ldg(vecs + v), __ldg(vecs + v + 1), skew), x);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = v < v1 && first + j < a.vocab ? to_float(row[first + j]) : -INFINITY;
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < kHold; ++j) top = fmaxf(top, f[j]);        // of a NaN and a number the number
    if (top > -INFINITY) {
      if (top > m) { s *= m > -INFINITY ? exp2f((m - top) * 1.4426950408889634f) : 0.f; m = top; }
      float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kHold; ++j) {
        const float e = exp2f((f[j] - m) * 1.4426950408889634f);        // the difference first: m may be the type's lowest value
        part[j & 3] += m < INFINITY ? (f[j] > -INFINITY ? e : 0.f) : (f[j] == m ? 1.f : 0.f);
      }
      s += (part[0] + part[1]) + (part[2] + part[3]);
    }
    const uint32_t mine = order_of(top);
    if (!__syncthreads_or(mine > floor_order)) continue;
    uint32_t bound = floor_order;
    if (have < a.picks) {
      const uint32_t low = qth_of_warp(mine, q);
      if (lane == 0) b.warp_low[warp] = low;
    }
    if (tid < have) b.list[tid] = b.ranked[tid];
    if (tid == 0) b.count = have;
    __syncthreads();
    if (have < a.picks) {
      uint32_t low = ~0u;
      for (int w = 0; w < kWarps; ++w) low = min(low, b.warp_low[w]);
      bound = low == 0 ? 0 : low - 1;
    }
    if (mine > bound) {
#pragma unroll
      for (int j = 0; j < kHold; ++j) {
        const uint32_t o = order_of(f[j]);
        if (o > bound) {
          const int at = atomicAdd(&b.count, 1);
          const uint32_t index = (uint32_t)((t0 + (j / V) * kThreads + tid) * V + j % V);
          if (at < kList) b.list[at] = (uint64_t)o << 32 | (uint32_t)~index;
        }
      }
    }
    __syncthreads();
    int n = b.count;
    if (n > kList) {
      // too many to count: the tile's best one after another.  A thread's best key below the last one taken is looked for anew by its owner alone.
      __syncthreads();
      uint64_t key = 0;
      auto next = [&](uint64_t below) {
        key = 0;
#pragma unroll
        for (int j = 0; j < kHold; ++j) {
          const uint32_t index = (uint32_t)((t0 + (j / V) * kThreads + tid) * V + j % V);
          const uint32_t o = order_of(f[j]);
          const uint64_t k = o > floor_order ? (uint64_t)o << 32 | (uint32_t)~index : 0ull;
          if (k < below && k > key) key = k;
        }
      };
      next(~0ull);
      n = have;
      if (tid < have) b.list[tid] = b.ranked[tid];
      for (int i = 0; i < a.picks; ++i) {
        const uint32_t hi = __reduce_max_sync(~0u, (uint32_t)(key >> 32));
        const uint32_t lo = __reduce_max_sync(~0u, (uint32_t)(key >> 32) == hi ? (uint32_t)key : 0u);
        if (lane == 0) { b.warp_top[warp] = hi; b.warp_low[warp] = lo; }
        __syncthreads();
        uint64_t best = 0;
        for (int w = 0; w < kWarps; ++w) best = max(best, (uint64_t)b.warp_top[w] << 32 | b.warp_low[w]);
        if (best == 0) break;
        if (key == best) { b.list[have + i] = best; next(best); }
        n = have + i + 1;
        __syncthreads();
      }
      __syncthreads();
    }
    have = rank(b, n, a.picks);
    if (have == a.picks) floor_order = (uint32_t)(b.ranked[have - 1] >> 32);
  }
  // the block's sum
  float M = m;
#pragma unroll
  for (int o = 16; o > 0; o /= 2) M = fmaxf(M, __shfl_xor_sync(~0u, M, o));
  if (lane == 0) warp_m[warp] = M;
  __syncthreads();
  for (int w = 0; w < kWarps; ++w) M = fmaxf(M, warp_m[w]);
  double S = m > -INFINITY ? (m == M ? (double)s : (double)(s * exp2f((m - M) * 1.4426950408889634f))) : 0.0;
#pragma unroll
  for (int o = 16; o > 0; o /= 2) S += __shfl_xor_sync(~0u, S, o);
  if (lane == 0) warp_s[warp] = S;
  __syncthreads();
  const long long piece = r * a.pieces + blockIdx.x;
  if (tid == 0) {
    S = 0.0;
    for (int w = 0; w < kWarps; ++w) S += warp_s[w];
    a.sums[piece] = S;
    a.tops[piece] = M;
    a.counts[piece] = have;
  }
  if (tid < have) a.best[piece * a.picks + tid] = make_uint2(__float_as_uint(value_of((uint32_t)(b.ranked[tid] >> 32))), ~(uint32_t)b.ranked[tid]);
}

// One request: the beams' logarithms, then the best of all candidates: by their totals, and among equal ones by beam, logit (fp64 totals of tiny logits can be equal
// where these are not) and token, which are one number, larger = better.
__device__ __forceinline__ uint64_t place_of(int k, float logit, uint32_t token) {
  return (uint64_t)(kMostBeams - 1 - k) << 56 | (uint64_t)order_of(logit) << 24 | (kMostVocab - 1 - token);
}
__device__ __forceinline__ int beam_of(uint64_t place) { return kMostBeams - 1 - (int)(place >> 56); }
__device__ __forceinline__ int token_of(uint64_t place) { return kMostVocab - 1 - (int)(place & (kMostVocab - 1)); }
__device__ __forceinline__ bool better(double x, uint64_t xp, double y, uint64_t yp) { return x > y || (x == y && xp > yp); }

__global__ void __launch_bounds__(kThreads) beam_merge_kernel(const Args a) {
  __shared__ double offset[kMostBeams], most[kMostBeams];      // score - log(sum) and m, of which a logit's total is offset + (logit - m); of a beam that ended, its score
  __shared__ int kind[kMostBeams];                 // 0: no candidates, 1: of its logits, 2: ended, 3: of its logits, the largest of which is +inf
  __shared__ double list_total[kMostPicks];
  __shared__ uint64_t list_at[kMostPicks];
  __shared__ double warp_total[kWarps];
  __shared__ uint64_t warp_at[kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K = a.beams, P = a.picks;
  const long long r0 = (long long)blockIdx.x * K;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (int k = warp; k < K; k += kWarps) {
    const float score = a.scores[r0 + k];
    const bool alive = score > -INFINITY && score < INFINITY;
    const bool done = a.finished && a.finished[r0 + k];
    float M = -INFINITY;
    double S = 0.0;
    if (alive && !done) {
      for (int i = lane; i < a.pieces; i += 32) M = fmaxf(M, a.tops[(r0 + k) * a.pieces + i]);
#pragma unroll
      for (int o = 16; o > 0; o /= 2) M = fmaxf(M, __shfl_xor_sync(~0u, M, o));
      for (int i = lane; i < a.pieces; i += 32) {
        const float m = a.tops[(r0 + k) * a.pieces + i];
        if (m > -INFINITY) S += a.sums[(r0 + k) * a.pieces + i] * (m == M ? 1.0 : exp((double)m - (double)M));
      }
#pragma unroll
      for (int o = 16; o > 0; o /= 2) S += __shfl_xor_sync(~0u, S, o);
    }
    if (lane == 0) {
      kind[k] = !alive ? 0 : done ? 2 : M == INFINITY ? 3 : M > -INFINITY ? 1 : 0;
      offset[k] = !alive ? 0.0 : done ? (double)score : M > -INFINITY ? (double)score - log(S) : 0.0;
      most[k] = (double)M;
    }
  }
  __syncthreads();
  // candidate c: piece c / P, place c % P of beam c / (pieces * P)
  const int each = a.pieces * P, all = K * each;
  auto candidate = [&](int c, double& total, uint64_t& at) {
    const int k = c / each, i = c - k * each;
    if (kind[k] == 2) {
      total = offset[k]; at = place_of(k, 0.f, (uint32_t)a.eos);
      return i == 0;
    }
    if (kind[k] == 0) return false;
    const long long piece = (r0 + k) * a.pieces + i / P;
    if (i % P >= a.counts[piece]) return false;
    const uint2 b = a.best[piece * P + i % P];
    const float l = __uint_as_float(b.x);
    if (kind[k] == 3 && l < INFINITY) return false;
    total = kind[k] == 3 ? offset[k] : offset[k] + ((double)l - most[k]);
    at = place_of(k, l, b.y);
    return true;
  };
  double last = INFINITY;
  uint64_t last_at = 0;
  bool first = true;
  int n = 0;
  double mine = -INFINITY;
  uint64_t mine_at = 0;
  bool some = false;
  auto look = [&]() {
    some = false;
    for (int c = tid; c < all; c += kThreads) {
      double t;
      uint64_t at;
      if (candidate(c, t, at) && (first || better(last, last_at, t, at)) && (!some || better(t, at, mine, mine_at))) { mine = t; mine_at = at; some = true; }
    }
    if (!some) { mine = -INFINITY; mine_at = 0; }
  };
  look();
  first = false;
  for (; n < P; ++n) {
    double t = mine;
    uint64_t at = mine_at;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
      const double ot = __shfl_xor_sync(~0u, t, o);
      const uint64_t oat = __shfl_xor_sync(~0u, at, o);
      if (better(ot, oat, t, at)) { t = ot; at = oat; }
    }
    if (lane == 0) { warp_total[warp] = t; warp_at[warp] = at; }
    __syncthreads();
    t = warp_total[0]; at = warp_at[0];
    for (int w = 1; w < kWarps; ++w)
      if (better(warp_total[w], warp_at[w], t, at)) { t = warp_total[w]; at = warp_at[w]; }
    if (at == 0) break;
    last = t; last_at = at;
    if (some && mine_at == at) look();
    if (tid == 0) { list_total[n] = t; list_at[n] = at; }
    __syncthreads();
  }
  __syncthreads();
  // fewer candidates than places: what is left has probability zero, lowest beam and token first
  if (tid == 0 && n < P) {
    const int found = n;
    int k = 0, v = 0;
    for (int i = found; i < P;) {
      bool taken = false;
      for (int j = 0; j < found; ++j) taken |= beam_of(list_at[j]) == k && token_of(list_at[j]) == v;
      if (!taken) { list_total[i] = -INFINITY; list_at[i] = place_of(k, 0.f, (uint32_t)v); ++i; }
      if (++v == a.vocab) { v = 0; ++k; }
    }
  }
  __syncthreads();
  if (tid < P) {
    const long long o = (long long)blockIdx.x * P + tid;
    const int parent = beam_of(list_at[tid]), token = token_of(list_at[tid]);
    a.next_scores[o] = (float)list_total[tid];
    a.parents[o] = parent;
    a.tokens[o] = token;
    if (a.finished_out) a.finished_out[o] = (a.finished && a.finished[r0 + parent]) || token == a.eos;
  }
}

// Pieces of a row: as many blocks as the SMs hold at once, but no piece so short that a block has less than a tile's share of work.
struct Plan { int pieces, piece_vecs; size_t bytes, off_tops, off_counts, off_best; };
Plan plan_of(int requests, int beams, int vocab, int picks) {
  Plan p;
  const long long rows = (long long)requests * beams;
  const int least = 2048;
  const long long want = std::max<long long>(1, 4ll * sm_count() / rows);
  p.pieces = (int)std::min<long long>({want, (vocab + least - 1) / least, kMostPieces});
  p.piece_vecs = 0;
  // rows * pieces is at most either of these, and both grow with the sizes: what is enough for a call is enough for smaller ones
  const size_t n = (size_t)std::min(std::max<long long>(rows, 4ll * sm_count()), rows * std::min(kMostPieces, (vocab + least - 1) / least));
  p.off_tops = n * 8;
  p.off_counts = p.off_tops + n * 4;
  p.off_best = round_up_sz(p.off_counts + n * 4, 16);
  p.bytes = p.off_best + n * picks * 8;
  return p;
}

template <typename T>
cudaError_t launch(Args a, cudaStream_t s) {
  const int V = Raw<T>::kVec;
  a.piece_vecs = ((a.vocab + V - 1) / V + a.pieces - 1) / a.pieces;
  beam_scan_kernel<T><<<dim3((unsigned)a.pieces, (unsigned)(a.requests * a.beams)), kThreads, 0, s>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.requests); cfg.blockDim = dim3(kThreads); cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
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
  a.counts = reinterpret_cast<int*>(w + l.off_counts);
  a.best = reinterpret_cast<uint2*>(w + l.off_best);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (g.dtype == RWKVQ_F32) return cuda_status(bs::launch<float>(a, s));
  if (g.dtype == RWKVQ_F16) return cuda_status(bs::launch<__half>(a, s));
  return cuda_status(bs::launch<__nv_bfloat16>(a, s));
}

}  // extern "C"
