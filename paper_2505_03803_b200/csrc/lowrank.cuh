// What the kernels of low-rank adapters share: the rows of a tile, and numbers as operands of the tensor cores.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/rwkvq.h"
#include "host_util.h"
#include "tc5.cuh"

namespace rwkvq {
int* device_status_ptr();  // api_misc.cu
namespace lr {

constexpr int kThreads = 256, kWarps = 8, kRows = 16, kMostRank = 128, kMostCounted = 1024;

struct alignas(64) Args {
  rwkvq_lowrank_args a;
  const uint8_t* mu;             // index stream of the token-shift vector, or nullptr
  const uint32_t* mu_codebook;
  int mu_bits, mu_entries;
  int splits;                    // clusters to a tile
  int* status;
  int x_by_map;                  // x goes to shared memory as it is, through a map
  int y_by_map;                  // sixteen rows of y, of 32 bits, are added to through a map
  int whole;                     // columns are a multiple of 64: a box holds several pieces of 64 columns
  // A: for each sixteen of the rank, as far as it goes, boxes of so many rows; B: 64 columns x 128 rows; X: 64 columns x a tile's rows; Y: 32 columns x 16 rows
  CUtensorMap A[8], B, X, Y;
};

// ---- rows of a tile -----------------------------------------------------------------------------------------
struct Tile {
  int rows[kRows];              // of groups of single rows
  int first, n, seq, start;     // of others: row `first` on, of the sequence that begins at `start`
  int adapter, rank;
  float scale;
  int counts;                   // has an adapter of a rank above 0: written, by one thread, only when all of the block may have read n
};

// The tile that is the item-th among all tiles of kTile rows of the sequences in seq_start; t.n stays 0 where there is none.  A sequence counts whose rows exist and that
// does not begin in front of an earlier entry of the list; the others are left out.  All threads of the block, of which the first kThreads look.
template <int kTile>
__device__ __forceinline__ void find_in_list(const Args& p, long long item, Tile& t, int* scratch) {
  const rwkvq_lowrank_args& a = p.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, each = (a.n_seq + kThreads - 1) / kThreads, i0 = min(tid * each, a.n_seq), i1 = min(i0 + each, a.n_seq);
  int* const tops = scratch;             // of each warp
  int* const sums = scratch + kWarps;
  int top = 0;
#pragma unroll 1
  for (int i = i0; i < i1; ++i) top = max(top, a.seq_start[i]);
  int upto = top;                        // most of this and the threads before
#pragma unroll
  for (int o = 1; o < 32; o *= 2) { const int v = __shfl_up_sync(~0u, upto, o); if (lane >= o) upto = max(upto, v); }
  if (lane == 31 && warp < kWarps) tops[warp] = upto;
  __syncthreads();
  int before = __shfl_up_sync(~0u, upto, 1);
  if (lane == 0) before = 0;
  for (int w = 0; w < min(warp, kWarps); ++w) before = max(before, tops[w]);
  // f(i, start, end) for each sequence of this thread that counts, until it is true
  auto each_one = [&](auto f) {
    int run = before;
    bool bad = false;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
      const int s = a.seq_start[i], e = a.seq_start[i + 1];
      const bool ok = s >= run && s >= 0 && e >= s && e <= a.tokens;
      bad |= !ok;
      if (ok && f(i, s, e)) break;
      run = max(run, s);
    }
    return bad;
  };
  int sum = 0;
  if (each_one([&](int, int s, int e) { sum += (e - s + kTile - 1) / kTile; return false; })) atomicExch(p.status, (int)RWKVQ_EINVAL);
  int at = sum;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) { const int v = __shfl_up_sync(~0u, at, o); if (lane >= o) at += v; }
  if (lane == 31 && warp < kWarps) sums[warp] = at;
  __syncthreads();
  at -= sum;
  for (int w = 0; w < min(warp, kWarps); ++w) at += sums[w];
  if (item >= at && item < at + sum)
    each_one([&](int i, int s, int e) {
      const int n = (e - s + kTile - 1) / kTile;
      if (item < at + n) {
        t.seq = i; t.start = s; t.first = s + (int)(item - at) * kTile; t.n = min(kTile, e - t.first);
        return true;
      }
      at += n;
      return false;
    });
}

__host__ __device__ inline bool single_rows(const rwkvq_lowrank_args& a) { return !a.seq_start && a.n_seq > 1; }      // each row a sequence
__host__ __device__ inline bool by_groups(const rwkvq_lowrank_args& a) { return a.n_seq <= kThreads && a.n_adapters <= kMostCounted; }
// Tiles of so many rows that there can be.
inline long long most_tiles(const rwkvq_lowrank_args& a, int rows) {
  const long long whole = ((long long)a.tokens + rows - 1) / rows;
  return a.seq_start ? std::min<long long>(a.tokens, whole + a.n_seq) : !single_rows(a) ? whole : by_groups(a) ? std::min<long long>(a.n_seq, a.n_adapters + whole) : (long long)a.n_seq;
}

// The rows of a tile of up to kTile; of single rows that share an adapter (then adapter, rank and scale are known, too) or of a sequence.  All threads; t.n stays as it is behind this.
// scratch: 2 * kWarps + 2 numbers; memory: 8 * kMostCounted bytes.
template <int kTile>
__device__ __forceinline__ void find_rows(const Args& p, long long item, Tile& t, int* scratch, void* memory) {
  const rwkvq_lowrank_args& a = p.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) { t.n = t.counts = 0; t.adapter = -1; }
  if (!single_rows(a)) {
    if (a.seq_start) {
      __syncthreads();
      find_in_list<kTile>(p, item, t, scratch);
    } else if (tid == 0) {
      t.seq = t.start = 0; t.first = (int)item * kTile; t.n = min(kTile, a.tokens - t.first);
    }
    __syncthreads();
    return;
  }
  if constexpr (kTile == kRows) {
    if (by_groups(a)) {
      // Rows of the same adapter are taken sixteen at a time: the item-th of these groups, in the order of their first rows.  `table`: how many rows of an adapter each
      // warp has, a byte each, from which a row knows how many are before it.
      uint64_t* const table = static_cast<uint64_t*>(memory);
      int* const heads = scratch;
      const int mine = tid < a.n_seq ? a.adapter[tid] : -1;
      for (int i = tid; i < a.n_adapters; i += kThreads) table[i] = 0;
      const bool ok = mine >= 0 && mine < a.n_adapters;
      if (!ok && mine != -1) atomicExch(p.status, (int)RWKVQ_EINVAL);
      const int there = ok ? mine : 0;
      const int rank_there = *(a.ranks ? a.ranks + there : a.adapter);
      const float scale_there = *(a.scale ? a.scale + there : reinterpret_cast<const float*>(a.adapter));
      const int rank = a.ranks ? rank_there : a.rank;
      const float scale = a.scale ? scale_there : 1.f;
      const uint32_t same = __match_any_sync(~0u, mine), earlier = same & ((1u << lane) - 1);
      __syncthreads();
      if (ok && earlier == 0) reinterpret_cast<uint8_t*>(table + mine)[warp] = (uint8_t)__popc(same);
      __syncthreads();
      const uint64_t others = ok && warp > 0 ? table[mine] << (64 - 8 * warp) : 0ull;
      const int before = (int)((others * 0x0101010101010101ull) >> 56) + __popc(earlier);
      const bool leads = ok && before % kRows == 0;
      const uint32_t vote = __ballot_sync(~0u, leads);
      if (lane == 0) heads[warp] = __popc(vote);
      __syncthreads();
      int at = __popc(vote & ((1u << lane) - 1));
      for (int w = 0; w < warp; ++w) at += heads[w];
      if (leads && at == item) { t.adapter = mine; t.rank = rank; t.scale = scale; t.start = before; }
      __syncthreads();
      const int from = t.start;
      const bool in = ok && mine == t.adapter && before >= from && before < from + kRows;
      if (in) t.rows[before - from] = tid;
      const int n = __syncthreads_count(in);
      if (tid == 0 && t.adapter >= 0) {
        t.n = t.rank < 0 || t.rank > a.rank ? 0 : t.rank == 0 ? 0 : n;
        if (t.rank < 0 || t.rank > a.rank) atomicExch(p.status, (int)RWKVQ_EINVAL);
      }
    } else {
      // many rows: an item is a row, which takes the next fifteen of its adapter if it is the first, seventeenth, ... of these
      const int mine = a.adapter[item];
      int before = 0;
      if (tid < kThreads)
#pragma unroll 8
        for (int i = tid; i < item; i += kThreads) before += a.adapter[i] == mine;
      for (int o = 16; o > 0; o /= 2) before += __shfl_xor_sync(~0u, before, o);
      if (lane == 0 && warp < kWarps) scratch[warp] = before;
      __syncthreads();
      before = 0;
      for (int w = 0; w < kWarps; ++w) before += scratch[w];
      if (before % kRows == 0 && tid < 32 && mine != -1) {
        int n = 0;
        for (int i0 = (int)item; i0 < a.n_seq && n < kRows; i0 += 256) {
          int there[8];
#pragma unroll
          for (int h = 0; h < 8; ++h) there[h] = a.adapter[min(i0 + h * 32 + tid, a.n_seq - 1)];
#pragma unroll
          for (int h = 0; h < 8; ++h) {
            const int i = i0 + h * 32 + tid;
            const uint32_t same = __ballot_sync(~0u, i < a.n_seq && there[h] == mine);
            const int at = n + __popc(same & ((1u << tid) - 1));
            if ((same >> tid & 1) && at < kRows) t.rows[at] = i;
            n = min(kRows, n + __popc(same));
          }
        }
        if (tid == 0) { t.n = n; t.seq = (int)item; }
      }
    }
  }
  __syncthreads();
}

// Adapter, rank and scale of a tile whose rows are known, and whether they count, by one thread.  The others may be reading t.n, each for itself: it is not touched.
__device__ __forceinline__ void find_adapter(const Args& p, Tile& t) {
  const rwkvq_lowrank_args& a = p.a;
  t.counts = t.n > 0 && t.adapter >= 0;
  if (t.n == 0 || t.adapter >= 0) return;
  const int mine = a.adapter[t.seq], at = min(max(mine, 0), a.n_adapters - 1);
  // both loads at once, from where something is
  const int rank_there = *(a.ranks ? a.ranks + at : a.adapter);
  const float scale_there = *(a.scale ? a.scale + at : reinterpret_cast<const float*>(a.adapter));
  const int rank = a.ranks ? rank_there : a.rank;
  const bool bad = mine < -1 || mine >= a.n_adapters || (mine >= 0 && (rank < 0 || rank > a.rank));
  if (!bad && mine >= 0 && rank > 0) { t.adapter = mine; t.rank = rank; t.scale = a.scale ? scale_there : 1.f; t.counts = 1; }
  if (bad) atomicExch(p.status, (int)RWKVQ_EINVAL);
}

// ---- numbers and operands -----------------------------------------------------------------------------------
// The next bf16 term of x, which is left with what the term leaves.  Cut off, not rounded, so that the largest numbers do not become infinite; of an infinity or
// NaN nothing is left.
__device__ __forceinline__ __nv_bfloat16 term(float& x) {
  const uint32_t b = __float_as_uint(x);
  const float hi = __uint_as_float((b & 0x7F800000u) == 0x7F800000u ? (b & 0x007FFFFFu ? b | 0x00400000u : b) & 0xFFFF0000u : b & 0xFFFF0000u);
  x = (b & 0x7F800000u) == 0x7F800000u ? 0.f : x - hi;
  return __ushort_as_bfloat16((unsigned short)(__float_as_uint(hi) >> 16));
}

// How x goes into the tensor cores: as it is, in as many bf16 terms as its bits take, or, beside f16 weights, in f16 terms under a power of two that brings the largest number of
// a row (of those that a block has) to 2^14: bf16 in one and f32 in two, off by up to 2^-24 of it, or 2^-39 of the row's largest.
template <typename X, typename W> struct Form {
  static constexpr bool kHalf = std::is_same<W, __half>::value, kScaled = kHalf && !std::is_same<X, __half>::value;
  static constexpr int kX = std::is_same<X, W>::value ? 1 : kHalf ? (std::is_same<X, float>::value ? 2 : 1) : std::is_same<X, float>::value ? 3 : std::is_same<X, __half>::value ? 2 : 1;
};
// The power of two that brings a row's largest finite number, whose bits these are, to 2^14, and the one that takes it back.
__device__ __forceinline__ void powers_of(int top, float& by, float& back) {
  const int up = top ? max(min(141 - (top >> 23), 126), -126) : 0;
  by = __uint_as_float((uint32_t)(127 + up) << 23);
  back = __uint_as_float((uint32_t)(127 - up) << 23);
}

// Byte offset of 16 bytes (eight columns) in rows of 128 bytes under the 128-byte swizzle.
__device__ __forceinline__ uint32_t swizzled(int row, int eight) { return (uint32_t)(row * 128 + ((eight ^ row) & 7) * 16); }
// A box of a tensor map by a converged warp, of which one lane is elected by predicate: from a branch of one lane each took some 145 cycles.
__device__ __forceinline__ void tensor_g2s(uint32_t dst_smem, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n"
               " @q cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n}"
               ::"r"(dst_smem), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

// Eight columns of a row of x and of the row in front of it, as they lie in memory.  All loads come from somewhere valid and none is in a branch of its own, so that they are on their
// way together; `there` says what counts.
template <typename X> struct Eights {
  uint4 x[sizeof(X) / 2], before[sizeof(X) / 2];
  bool there, has_before;
};
// A row of x, and the one in front of it (x itself, where there is none).
template <typename X> struct RowOf {
  const X* x;
  const X* before;
  bool has_before;
};
template <typename X>
__device__ __forceinline__ RowOf<X> row_at(const Args& p, int row, int seq, bool begins) {
  const rwkvq_lowrank_args& a = p.a;
  RowOf<X> r;
  r.x = static_cast<const X*>(a.x) + (long long)row * a.x_row;
  r.before = a.x_prev ? static_cast<const X*>(a.x_prev) + (long long)row * a.x_prev_row : !begins ? r.x - a.x_row : a.xprev0 ? static_cast<const X*>(a.xprev0) + (long long)seq * a.ic : r.x;
  r.has_before = a.x_prev || !begins || a.xprev0;
  return r;
}
template <typename X, bool kMix>
__device__ __forceinline__ Eights<X> load_eights(const Args& p, const RowOf<X>& r, int col) {
  Eights<X> e;
  e.there = col < p.a.ic;
  e.has_before = r.has_before;
  col = min(col, p.a.ic - 8);
#pragma unroll
  for (int i = 0; i < (int)sizeof(X) / 2; ++i) e.x[i] = reinterpret_cast<const uint4*>(r.x + col)[i];
  if constexpr (kMix) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(X) / 2; ++i) e.before[i] = reinterpret_cast<const uint4*>(r.before + col)[i];
  }
  return e;
}
// Their indices of the token-shift vector: four are 4 * mu_bits neighbouring bits from a byte's beginning; behind the indices lies the codebook.
struct MuWords { uint32_t lo, hi; };
template <bool kMix>
__device__ __forceinline__ MuWords load_mu(const Args& p, int col) {
  MuWords m = {0, 0};
  if constexpr (kMix) {
    const uint32_t* const words = reinterpret_cast<const uint32_t*>(p.mu) + ((uint32_t)(min(col, p.a.ic - 8) >> 3) * (uint32_t)p.mu_bits >> 3);
    m.lo = __ldg(words);
    m.hi = __ldg(words + 1);
  }
  return m;
}
template <bool kMix>
__device__ __forceinline__ void mu_of(const Args& p, const uint32_t* codebook, const MuWords& w, int col, float2 (&m)[4]) {
  if constexpr (kMix) {
    const uint32_t bits = (uint32_t)p.mu_bits, f = __funnelshift_r(w.lo, w.hi, ((uint32_t)(min(col, p.a.ic - 8) >> 3) * bits >> 1 & 3u) * 8u), mask = (1u << bits) - 1u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t pair = codebook[f >> (uint32_t)j * bits & mask];
      m[j] = __half22float2(*reinterpret_cast<const __half2*>(&pair));
    }
  }
}
// Pairs of 16-bit numbers; packed conversions, which take a fraction of what single ones do.
__device__ __forceinline__ float2 pair_of(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ float2 pair_of(uint32_t w, __nv_bfloat16) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ uint32_t rounded(float2 f, __half) {
  const __half2 h = __floats2half2_rn(f.x, f.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t rounded(float2 f, __nv_bfloat16) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// A pair as its next bf16 term, cut off, and what that leaves.
__device__ __forceinline__ uint32_t cut_off(float2& f) {
  const uint32_t lo = __float_as_uint(f.x), hi = __float_as_uint(f.y);
  f.x -= __uint_as_float(lo & 0xFFFF0000u);
  f.y -= __uint_as_float(hi & 0xFFFF0000u);
  return __byte_perm(lo, hi, 0x7632);
}
__device__ __forceinline__ float2 mixed(float2 x, float2 y, float2 m) { return make_float2(fmaf(y.x - x.x, m.x, x.x), fmaf(y.y - x.y, m.y, x.y)); }

// x_mix of eight columns, rounded to X; zeros behind the last column.
template <typename X, bool kMix>
__device__ __forceinline__ void mix_eights(const Eights<X>& e, const float2 (&m)[4], float2 (&f)[4]) {
  auto counts = [](const uint4& w, bool yes) { return make_uint4(yes ? w.x : 0u, yes ? w.y : 0u, yes ? w.z : 0u, yes ? w.w : 0u); };
  if constexpr (sizeof(X) == 2) {
    const uint4 x4 = counts(e.x[0], e.there);
    const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = pair_of(x[j], X());
    if constexpr (kMix) {
      const uint4 y4 = counts(e.before[0], e.there && e.has_before);
      const uint32_t y[4] = {y4.x, y4.y, y4.z, y4.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = pair_of(rounded(mixed(f[j], pair_of(y[j], X()), m[j]), X()), X());
    }
  } else {
    const uint4 a4 = counts(e.x[0], e.there), b4 = counts(e.x[1], e.there);
    f[0] = make_float2(__uint_as_float(a4.x), __uint_as_float(a4.y)); f[1] = make_float2(__uint_as_float(a4.z), __uint_as_float(a4.w));
    f[2] = make_float2(__uint_as_float(b4.x), __uint_as_float(b4.y)); f[3] = make_float2(__uint_as_float(b4.z), __uint_as_float(b4.w));
    if constexpr (kMix) {
      const uint4 c4 = counts(e.before[0], e.there && e.has_before), d4 = counts(e.before[1], e.there && e.has_before);
      const float y[8] = {__uint_as_float(c4.x), __uint_as_float(c4.y), __uint_as_float(c4.z), __uint_as_float(c4.w), __uint_as_float(d4.x), __uint_as_float(d4.y), __uint_as_float(d4.z),
                          __uint_as_float(d4.w)};
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = mixed(f[j], make_float2(y[2 * j], y[2 * j + 1]), m[j]);
    }
  }
}
// Bits of the largest finite number among them.
__device__ __forceinline__ int top_of(const float2 (&f)[4]) {
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float x = fabsf(f[j].x), y = fabsf(f[j].y);
    top = fmaxf(top, fmaxf(x < INFINITY ? x : 0.f, y < INFINITY ? y : 0.f));
  }
  return __float_as_int(top);
}
// x_mix of eight columns, rounded to X, as operands of the tensor cores: F::kX terms, `next` bytes from one to the next; `by`: see Form.  (What the first bf16 terms leave of an
// infinity is NaN.)
template <typename X, typename F, bool kMix>
__device__ __forceinline__ void put_eights(const Eights<X>& e, const float2 (&m)[4], uint8_t* to, uint32_t next, float by) {
  float2 f[4];
  mix_eights<X, kMix>(e, m, f);
  uint32_t out[3][4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (F::kScaled) {
      f[j].x *= by; f[j].y *= by;
      out[0][j] = rounded(f[j], __half());
      const float2 hi = pair_of(out[0][j], __half());
      if constexpr (F::kX == 2) out[1][j] = rounded(make_float2(fabsf(f[j].x) < INFINITY ? f[j].x - hi.x : 0.f, fabsf(f[j].y) < INFINITY ? f[j].y - hi.y : 0.f), __half());
    } else if constexpr (F::kX == 1) {
      out[0][j] = rounded(f[j], X());
    } else {
#pragma unroll
      for (int k = 0; k < F::kX - 1; ++k) out[k][j] = cut_off(f[j]);
      out[F::kX - 1][j] = rounded(f[j], __nv_bfloat16());
    }
  }
#pragma unroll
  for (int k = 0; k < F::kX; ++k) *reinterpret_cast<uint4*>(to + k * next) = make_uint4(out[k][0], out[k][1], out[k][2], out[k][3]);
}

// [n][rows][cols] of 16-bit numbers as boxes of 64 columns x box_rows rows in the 128-byte swizzle; what lies outside reads as zero.
inline bool encode(CUtensorMap* map, const void* at, bool half, int cols, int rows, int n, int box_rows) {
  const tc5::EncodeTiledFn fn = tc5::encode_tiled();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)n}, strides[2] = {(cuuint64_t)cols * 2, (cuuint64_t)cols * 2 * (cuuint64_t)rows};
  const cuuint32_t box[3] = {64u, (cuuint32_t)box_rows, 1u}, step[3] = {1u, 1u, 1u};
  return fn(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(at), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace lr
}  // namespace rwkvq
