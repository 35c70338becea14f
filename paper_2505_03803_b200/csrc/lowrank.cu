// Low-rank adapters of many sequences beside a shared projection: y_t += s_a B_a (A_a x_t), a the adapter of t's sequence.
//
// A tile is up to sixteen rows that have the same adapter; a cluster of thread blocks works on one.  Each block multiplies its share of the columns of A
// with the rows' (token-shifted) inputs, the blocks add up their shares through distributed shared memory, and each multiplies its share of the rows of B
// with the result: one launch, no workspace, sums in a fixed order.
//
// Weights are the 16-row operand of mma.sync, straight from memory to registers: a lane reads 16 neighbouring bytes of a row, and the columns of a step are
// numbered so that these are its fragments.  Operands are exact: where the types of x and the weights differ, numbers are taken apart into bf16 terms
// (f16: two, f32: three), and so is A x, which is summed in fp32 (three terms, all of it, where y has 32 bits; two, the second rounded, where y has 16: off by up to 2^-16 of it).
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/rwkvq.h"
#include "host_util.h"

namespace cg = cooperative_groups;

namespace rwkvq {
int* device_status_ptr();  // api_misc.cu
namespace lr {

constexpr int kThreads = 256, kWarps = 8, kRows = 16, kMostRank = 128, kMostCols = 512, kMostCounted = 1024;

struct Args {
  rwkvq_lowrank_args a;
  const uint8_t* mu;             // index stream of the token-shift vector, or nullptr
  const uint32_t* mu_codebook;
  int mu_bits, mu_entries;
  int splits;                    // clusters to a tile
  int* status;
};

// ---- rows of a tile -----------------------------------------------------------------------------------------
struct Tile {
  int rows[kRows], seqs[kRows];       // seqs: of a row that is its sequence's first, else -1 - sequence
  int n, adapter, rank;
  float scale;
};

// The sequence and tile of `item` among all tiles of sixteen rows of the sequences in seq_start, or n = 0.  A sequence counts whose rows exist and that
// does not begin in front of an earlier entry of the list; the others are left out.  All threads.
__device__ void find_in_list(const Args& p, long long item, int& seq, int& first, int& last, int* scratch) {
  const rwkvq_lowrank_args& a = p.a;
  const int tid = threadIdx.x, each = (a.n_seq + kThreads - 1) / kThreads, i0 = min(tid * each, a.n_seq), i1 = min(i0 + each, a.n_seq);
  int* most = scratch;                   // [kThreads + 1]
  int* tiles = scratch + kThreads + 1;   // [kThreads + 1]
  int top = 0;
  for (int i = i0; i < i1; ++i) top = max(top, a.seq_start[i]);
  most[tid + 1] = top;
  if (tid == 0) most[0] = 0;
  __syncthreads();
  int before = 0;
  for (int t = 0; t <= tid; ++t) before = max(before, most[t]);
  int sum = 0, run = before;
  bool bad = false;
  for (int i = i0; i < i1; ++i) {
    const int s = a.seq_start[i], e = a.seq_start[i + 1];
    const bool ok = s >= run && s >= 0 && e >= s && e <= a.tokens;
    bad |= !ok;
    if (ok) sum += (e - s + kRows - 1) / kRows;
    run = max(run, s);
  }
  if (bad) atomicExch(p.status, (int)RWKVQ_EINVAL);
  tiles[tid + 1] = sum;
  if (tid == 0) tiles[0] = 0;
  __syncthreads();
  long long at = 0;
  for (int t = 0; t <= tid; ++t) at += tiles[t];
  if (tid == 0) { most[0] = -1; }
  __syncthreads();
  run = before;
  if (item >= at && item < at + sum) {
    for (int i = i0; i < i1; ++i) {
      const int s = a.seq_start[i], e = a.seq_start[i + 1];
      if (s >= run && s >= 0 && e >= s && e <= a.tokens) {
        const int n = (e - s + kRows - 1) / kRows;
        if (item < at + n) {
          most[0] = i; most[1] = s + (int)(item - at) * kRows; most[2] = min(most[1] + kRows, e);
          break;
        }
        at += n;
      }
      run = max(run, s);
    }
  }
  __syncthreads();
  seq = most[0]; first = most[1]; last = most[2];
  __syncthreads();
}

__host__ __device__ inline bool by_groups(const rwkvq_lowrank_args& a) { return a.n_seq <= kThreads && a.n_adapters <= kMostCounted; }

// scratch: 2 * kThreads + 2 numbers; memory: 8 * kMostCounted bytes.
__device__ void find_tile(const Args& p, long long item, Tile& t, int* scratch, void* memory) {
  const rwkvq_lowrank_args& a = p.a;
  const int tid = threadIdx.x;
  if (tid == 0) t.n = 0;
  __syncthreads();
  if (!a.seq_start && a.n_seq == a.tokens && a.n_seq > 1) {
    // one row a sequence.  Rows of the same adapter are taken sixteen at a time; the item-th of these groups, in the order of their first rows.
    if (by_groups(a)) {
      // how many rows of an adapter each warp has, a byte each, from which a row knows how many are before it
      uint64_t* const table = static_cast<uint64_t*>(memory);
      int* const heads = scratch;
      const int warp = tid >> 5, lane = tid & 31, mine = tid < a.n_seq ? a.adapter[tid] : -1;
      const bool ok = mine >= 0 && mine < a.n_adapters;
      if (!ok && mine != -1) atomicExch(p.status, (int)RWKVQ_EINVAL);
      const int rank = ok && a.ranks ? a.ranks[mine] : a.rank;
      const float scale = ok && a.scale ? a.scale[mine] : 1.f;
      for (int i = tid; i < a.n_adapters; i += kThreads) table[i] = 0;
      const uint32_t same = __match_any_sync(~0u, mine), earlier = same & ((1u << lane) - 1);
      __syncthreads();
      if (ok && earlier == 0) reinterpret_cast<uint8_t*>(table + mine)[warp] = (uint8_t)__popc(same);
      __syncthreads();
      const uint64_t others = ok && warp > 0 ? table[mine] << (64 - 8 * warp) : 0ull;
      const int before = (int)((others * 0x0101010101010101ull) >> 56) + __popc(earlier);
      const bool leads = ok && before % kRows == 0;
      const uint32_t vote = __ballot_sync(~0u, leads);
      if (lane == 0) heads[warp] = __popc(vote);
      if (tid == 0) t.adapter = -1;
      __syncthreads();
      int at = __popc(vote & ((1u << lane) - 1));
      for (int w = 0; w < warp; ++w) at += heads[w];
      if (leads && at == item) { t.adapter = mine; t.rank = rank; t.scale = scale; heads[kWarps] = before; }
      __syncthreads();
      if (t.adapter < 0) return;
      const int from = heads[kWarps];
      const bool in = mine == t.adapter && before >= from && before < from + kRows;
      if (in) { t.rows[before - from] = tid; t.seqs[before - from] = tid; }
      const int n = __syncthreads_count(in);
      if (tid == 0) {
        t.n = n;
        if (t.rank < 0 || t.rank > a.rank) { atomicExch(p.status, (int)RWKVQ_EINVAL); t.n = 0; }
        if (t.rank == 0) t.n = 0;
      }
      __syncthreads();
      return;
    } else {
      // many rows: an item is a row, which takes the next fifteen of its adapter if it is the first, seventeenth, ... of these
      const int mine = a.adapter[item];
      if (mine < 0 || mine >= a.n_adapters) {
        if (tid == 0 && mine != -1) atomicExch(p.status, (int)RWKVQ_EINVAL);
        return;
      }
      int before = 0;
      for (int i = tid; i < item; i += kThreads) before += a.adapter[i] == mine;
      for (int o = 16; o > 0; o /= 2) before += __shfl_xor_sync(~0u, before, o);
      if ((tid & 31) == 0) scratch[tid / 32] = before;
      __syncthreads();
      before = 0;
      for (int w = 0; w < kWarps; ++w) before += scratch[w];
      if (before % kRows) return;
      if (tid < 32) {
        int n = 0;
        for (int i0 = (int)item; i0 < a.n_seq && n < kRows; i0 += 32) {
          const int i = i0 + tid;
          const uint32_t same = __ballot_sync(~0u, i < a.n_seq && a.adapter[i] == mine);
          const int at = n + __popc(same & ((1u << tid) - 1));
          if ((same >> tid & 1) && at < kRows) { t.rows[at] = i; t.seqs[at] = i; }
          n = min(kRows, n + __popc(same));
        }
        if (tid == 0) { t.n = n; t.adapter = mine; }
      }
    }
  } else {
    int seq = 0, first = (int)item * kRows, last = min(first + kRows, a.tokens), start = 0;
    if (a.seq_start) {
      find_in_list(p, item, seq, first, last, scratch);
      if (seq < 0) return;
      start = a.seq_start[seq];
    }
    const int mine = a.adapter[seq];
    if (mine < 0 || mine >= a.n_adapters) {
      if (tid == 0 && mine != -1) atomicExch(p.status, (int)RWKVQ_EINVAL);
      return;
    }
    if (tid < last - first) { t.rows[tid] = first + tid; t.seqs[tid] = first + tid == start ? seq : -1 - seq; }
    if (tid == 0) { t.n = last - first; t.adapter = mine; }
  }
  if (tid == 0) {
    const int rank = a.ranks ? a.ranks[t.adapter] : a.rank;
    t.scale = a.scale ? a.scale[t.adapter] : 1.f;
    t.rank = rank;
    if (rank < 0 || rank > a.rank) { atomicExch(p.status, (int)RWKVQ_EINVAL); t.n = 0; }
    if (rank == 0) t.n = 0;
  }
  __syncthreads();
}

// ---- numbers and operands -----------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_float<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <typename T> struct Eight { T v[8]; };
template <typename T>
__device__ __forceinline__ void load8(const T* p, float* f) {
  if constexpr (sizeof(T) == 4) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    const Eight<T> e = *reinterpret_cast<const Eight<T>*>(&w);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = to_float<T>(e.v[i]);
  }
}

// The next bf16 term of x, which is left with what the term leaves.  Cut off, not rounded, so that the largest numbers do not become infinite; of an infinity or
// NaN nothing is left.
__device__ __forceinline__ __nv_bfloat16 term(float& x) {
  const uint32_t b = __float_as_uint(x);
  const float hi = __uint_as_float((b & 0x7F800000u) == 0x7F800000u ? (b & 0x007FFFFFu ? b | 0x00400000u : b) & 0xFFFF0000u : b & 0xFFFF0000u);
  x = (b & 0x7F800000u) == 0x7F800000u ? 0.f : x - hi;
  return __ushort_as_bfloat16((unsigned short)(__float_as_uint(hi) >> 16));
}

// A pair of f16 weights as two pairs of bf16: eleven bits are eight and three.  (Of an infinity the second is NaN.)
__device__ __forceinline__ void apart(uint32_t w, uint32_t& hi, uint32_t& lo) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  const uint32_t x = __float_as_uint(f.x), y = __float_as_uint(f.y);
  hi = __byte_perm(x, y, 0x7632);
  const __nv_bfloat162 l = __floats2bfloat162_rn(f.x - __uint_as_float(x & 0xFFFF0000u), f.y - __uint_as_float(y & 0xFFFF0000u));
  lo = *reinterpret_cast<const uint32_t*>(&l);
}

// y[at], y[at + 1] += v.  Each element of y is added to once in a call, so that a reduction in memory is as good as a load, an addition and a store, and
// nothing waits for it (it takes subnormal numbers for zeros).
__device__ __forceinline__ void add_pair(void* y, int dtype, long long at, float v0, float v1) {
  if (dtype == RWKVQ_F32) {
    asm volatile("red.relaxed.gpu.global.add.v2.f32 [%0], {%1, %2};" ::"l"(static_cast<float*>(y) + at), "f"(v0), "f"(v1) : "memory");
  } else if (dtype == RWKVQ_F16) {
    __half2* const p = reinterpret_cast<__half2*>(static_cast<__half*>(y) + at);
    const float2 f = __half22float2(*p);
    *p = __floats2half2_rn(f.x + v0, f.y + v1);
  } else {
    __nv_bfloat162* const p = reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(y) + at);
    const float2 f = __bfloat1622float2(*p);
    *p = __floats2bfloat162_rn(f.x + v0, f.y + v1);
  }
}

// How x and the weights go into the tensor cores.
template <typename X, typename W> struct Form {
  static constexpr bool kHalf = std::is_same<X, __half>::value && std::is_same<W, __half>::value;
  static constexpr int kX = std::is_same<X, W>::value ? 1 : std::is_same<X, float>::value ? 3 : std::is_same<X, __half>::value ? 2 : 1;
  static constexpr bool kApart = std::is_same<W, __half>::value && !kHalf;
};

// The token-shift vector's pairs of columns col to col + 7 (col a multiple of 8), whose indices are four times mu_bits neighbouring bits from a byte's beginning.
__device__ __forceinline__ void mu_eight(const Args& p, const uint32_t* codebook, int col, float2 (&m)[4]) {
  const uint32_t byte = (uint32_t)(col >> 3) * (uint32_t)p.mu_bits >> 1, shift = (byte & 3u) * 8u;
  const uint32_t* const words = reinterpret_cast<const uint32_t*>(p.mu) + (byte >> 2);
  const uint32_t lo = __ldg(words), hi = shift + 4u * (uint32_t)p.mu_bits > 32u ? __ldg(words + 1) : 0u, f = __funnelshift_r(lo, hi, shift), mask = (1u << p.mu_bits) - 1u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t pair = codebook[f >> (uint32_t)(j * p.mu_bits) & mask];
    m[j] = __half22float2(*reinterpret_cast<const __half2*>(&pair));
  }
}

// ---- few rows: the weights straight from memory into registers ----------------------------------------------
// A unit is sixteen rows of a weight matrix by 32 columns: lane (g, q) holds columns 8q to 8q + 7 of rows g and g + 8, the operands of four steps whose columns are
// numbered so that the first four of the eight are one step's and the others the next one's.
struct Unit { uint4 lo, hi; };        // row g, row g + 8
constexpr int kSide = 4, kDeep = 2;        // units that a warp has on their way: four side by side (blocks of rank, or tiles of B), two along the columns

template <typename W>
__device__ __forceinline__ Unit load_unit(const W* m, long long row, long long rows, long long pitch, int col, int cols) {
  Unit u;
  u.lo = u.hi = make_uint4(0, 0, 0, 0);
  if (col < cols) {
    if (row < rows) u.lo = __ldg(reinterpret_cast<const uint4*>(m + row * pitch + col));
    if (row + 8 < rows) u.hi = __ldg(reinterpret_cast<const uint4*>(m + (row + 8) * pitch + col));
  }
  return u;
}
__device__ __forceinline__ void keep(uint4& w, int n) {        // the first n of eight numbers of two bytes
  auto of = [n](int i) { return n >= 2 * i + 2 ? ~0u : n == 2 * i + 1 ? 0xFFFFu : 0u; };
  w.x &= of(0); w.y &= of(1); w.z &= of(2); w.w &= of(3);
}

// d[0], d[1]: sixteen rows of x (a: row g, b: row g + 8 of the lane's columns) by the unit's rows 0 to 7 and 8 to 15.
template <bool kHalf>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (kHalf)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <bool kHalf>
__device__ __forceinline__ void mma_unit(float (&d)[2][4], const uint4& xa, const uint4& xb, const Unit& w) {
  mma<kHalf>(d[0], xa.x, xb.x, xa.y, xb.y, w.lo.x, w.lo.y);
  mma<kHalf>(d[1], xa.x, xb.x, xa.y, xb.y, w.hi.x, w.hi.y);
  mma<kHalf>(d[0], xa.z, xb.z, xa.w, xb.w, w.lo.z, w.lo.w);
  mma<kHalf>(d[1], xa.z, xb.z, xa.w, xb.w, w.hi.z, w.hi.w);
}
__device__ __forceinline__ void apart(const uint4& w, uint4& hi, uint4& lo) {
  apart(w.x, hi.x, lo.x); apart(w.y, hi.y, lo.y); apart(w.z, hi.z, lo.z); apart(w.w, hi.w, lo.w);
}
// All terms of x (`pitch` bytes from row to row, `next` from term to term) by up to kSide units of weights, the small products first.
template <bool kHalf, bool kApart, int kTerms>
__device__ __forceinline__ void multiply(float (&d)[kSide][2][4], const uint8_t* x, uint32_t pitch, uint32_t next, int terms, const Unit* w, int units) {
#pragma unroll
  for (int k = kTerms - 1; k >= 0; --k) {
    if (k >= terms) continue;
    const uint4 xa = *reinterpret_cast<const uint4*>(x + k * next), xb = *reinterpret_cast<const uint4*>(x + k * next + 8 * pitch);
#pragma unroll
    for (int u = 0; u < kSide; ++u) {
      if (u >= units) continue;
      if constexpr (kApart) {
        Unit hi, lo;
        apart(w[u].lo, hi.lo, lo.lo); apart(w[u].hi, hi.hi, lo.hi);
        mma_unit<kHalf>(d[u], xa, xb, lo);
        mma_unit<kHalf>(d[u], xa, xb, hi);
      } else {
        mma_unit<kHalf>(d[u], xa, xb, w[u]);
      }
    }
  }
}

template <typename X, typename W>
struct Shape {
  static constexpr int kTerms = Form<X, W>::kX;
  // bytes of a row in shared memory: 16-byte reads of two neighbouring rows meet no bank twice
  static constexpr int kPitch = kMostCols * 2 + 64, kHPitch = kMostRank * 2 + 64, kPartPitch = kSide * 16 + 8;
  static constexpr int kXBytes = kTerms * kRows * kPitch, kHBytes = 3 * kRows * kHPitch, kFront = kXBytes > kHBytes ? kXBytes : kHBytes;
  static constexpr int kPart = kWarps * kRows * kPartPitch * 4;       // sums of each warp: [warp][row][64 of the rank]
  static constexpr int kShare = kRows * kMostRank * 4;
  static constexpr int kBytes = kFront + kPart + kShare + 256 * 4;
  static_assert(kPart >= 8 * kMostCounted, "room for counting the rows of adapters");
};

template <typename X, typename W>
__global__ void __launch_bounds__(kThreads, 2) lowrank_kernel(const Args p) {
  using S = Shape<X, W>;
  using F = Form<X, W>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Tile t;
  __shared__ int scratch[2 * kThreads + 2];
  uint8_t* const xs = smem;                                              // [term][row][column], then A x: [term][row][rank]
  uint8_t* const hs = smem;
  float* const part = reinterpret_cast<float*>(smem + S::kFront);
  float* const share = part + S::kPart / 4;                              // this block's share of A x: [row][rank]
  uint32_t* const codebook = reinterpret_cast<uint32_t*>(share + S::kShare / 4);
  const rwkvq_lowrank_args& a = p.a;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  if (p.mu)
    for (int i = tid; i < p.mu_entries; i += kThreads) codebook[i] = p.mu_codebook[i];
  const int id = (int)(blockIdx.x / C), item = id / p.splits, split = id - item * p.splits;
  find_tile(p, item, t, scratch, part);
  __syncthreads();
  const int n = t.n;
  if (n == 0) return;            // the same for all blocks of the cluster
  const int rank = t.rank;

  // ---- A x over this block's columns, 64 of the rank at a time.  Each warp takes every eighth unit of columns, for all of these.
  const int units = (a.ic + 31) / 32, u0 = (int)((long long)units * c / C), u1 = (int)((long long)units * (c + 1) / C);
  const W* const A = static_cast<const W*>(a.A) + (long long)t.adapter * a.rank * a.ic;
  Unit w[kDeep * kSide];
  auto load_a = [&](int uc, int r0) {
#pragma unroll
    for (int k = 0; k < kDeep; ++k)
#pragma unroll
      for (int j = 0; j < kSide; ++j) {
        const int u = uc + warp + k * kWarps;
        w[k * kSide + j] = load_unit(A, r0 + j * 16 + g, rank, a.ic, u * 32 + q * 8, u < u1 ? a.ic : 0);
      }
  };
  load_a(u0, 0);
  for (int r0 = 0; r0 < rank; r0 += kSide * 16) {
    const int side = min(kSide, (rank - r0 + 15) / 16);
    float acc[kSide][2][4] = {};
    for (int uc = u0; uc < u1 || uc == u0; uc += kMostCols / 32) {
      const int ue = min(uc + kMostCols / 32, u1), eights = (ue - uc) * 4;
      if (r0 == 0 || u1 - u0 > kMostCols / 32) {
        if (uc > u0 || r0 > 0) __syncthreads();
        for (int i = tid; i < n * eights; i += kThreads) {
          const int r = i / eights, col8 = i - r * eights, col = uc * 32 + col8 * 8;
          float x[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = 0.f;
          if (col < a.ic) {
            load8(static_cast<const X*>(a.x) + (long long)t.rows[r] * a.x_row + col, x);
            if (p.mu) {
              float y[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) y[j] = 0.f;
              const int seq = t.seqs[r];
              if (a.x_prev) load8(static_cast<const X*>(a.x_prev) + (long long)t.rows[r] * a.x_prev_row + col, y);
              else if (seq < 0) load8(static_cast<const X*>(a.x) + (long long)(t.rows[r] - 1) * a.x_row + col, y);
              else if (a.xprev0) load8(static_cast<const X*>(a.xprev0) + (long long)seq * a.ic + col, y);
              float2 m[4];
              mu_eight(p, codebook, col, m);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                x[2 * j] = to_float<X>(from_float<X>(fmaf(y[2 * j] - x[2 * j], m[j].x, x[2 * j])));
                x[2 * j + 1] = to_float<X>(from_float<X>(fmaf(y[2 * j + 1] - x[2 * j + 1], m[j].y, x[2 * j + 1])));
              }
            }
          }
#pragma unroll
          for (int k = 0; k < F::kX; ++k) {
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if constexpr (F::kHalf) {
                const __half2 h = __floats2half2_rn(x[2 * j], x[2 * j + 1]);
                v[j] = *reinterpret_cast<const uint32_t*>(&h);
              } else if constexpr (F::kX == 1) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
                v[j] = *reinterpret_cast<const uint32_t*>(&h);
              } else {
                __nv_bfloat162 h;
                h.x = term(x[2 * j]); h.y = term(x[2 * j + 1]);
                v[j] = *reinterpret_cast<const uint32_t*>(&h);
              }
            }
            *reinterpret_cast<uint4*>(xs + (k * kRows + r) * S::kPitch + col8 * 16) = make_uint4(v[0], v[1], v[2], v[3]);
          }
        }
        __syncthreads();
      }
      // rows of x behind the n-th hold whatever was there: a row meets its own outputs alone
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        const int u = uc + warp + k * kWarps;
        if (u < ue) multiply<F::kHalf, F::kApart, F::kX>(acc, xs + g * S::kPitch + ((u - uc) * 32 + q * 8) * 2, S::kPitch, kRows * S::kPitch, F::kX, w + k * kSide, side);
      }
      if (ue < u1) load_a(ue, r0);
      else if (r0 + kSide * 16 < rank) load_a(u0, r0 + kSide * 16);
    }
    if (r0 > 0) __syncthreads();
#pragma unroll
    for (int j = 0; j < kSide; ++j)
      if (j < side)
#pragma unroll
        for (int e = 0; e < 4; e += 2)
          if (g + e * 4 < n)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              *reinterpret_cast<float2*>(part + (warp * kRows + g + e * 4) * S::kPartPitch + j * 16 + h * 8 + q * 2) = make_float2(acc[j][h][e], acc[j][h][e + 1]);
    __syncthreads();
    for (int i = tid; i < n * kSide * 16; i += kThreads) {
      const int row = i / (kSide * 16), r = i % (kSide * 16);
      if (r >= side * 16) continue;
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) s += part[(k * kRows + row) * S::kPartPitch + r];
      share[row * kMostRank + r0 + r] = s;
    }
  }

  // ---- B's first units on their way, and y where it is read
  const int tiles = (a.oc + 15) / 16, all_parts = C * p.splits, part_id = split * C + c;
  const int o0 = (int)((long long)tiles * part_id / all_parts), o1 = (int)((long long)tiles * (part_id + 1) / all_parts);
  const W* const Bm = static_cast<const W*>(a.B) + (long long)t.adapter * a.oc * a.rank;
  auto load_b = [&](int o, int col0) {
#pragma unroll
    for (int k = 0; k < kDeep; ++k)
#pragma unroll
      for (int j = 0; j < kSide; ++j) {
        const int tile = o + j * kWarps, col = col0 + k * 32 + q * 8;
        Unit& u = w[k * kSide + j];
        u = load_unit(Bm, (long long)tile * 16 + g, tile < o1 ? a.oc : 0, a.rank, col, rank);
        if (col + 8 > rank) { keep(u.lo, rank - col); keep(u.hi, rank - col); }        // what lies behind the adapter's rank may be anything
      }
  };
  load_b(o0 + warp, 0);
  cluster.sync();

  // ---- all of A x, as operands
  const int last_term = a.y_dtype == RWKVQ_F32 ? 2 : 1, width = (rank + 31) / 32 * 32;
  const float scale = t.scale;
  for (int i = tid; i < n * width; i += kThreads) {
    const int row = i / width, r = i - row * width;
    float s = 0.f;
    if (r < rank) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = k < C ? cluster.map_shared_rank(share, k)[row * kMostRank + r] : 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[k];
      s *= scale;
    }
    __nv_bfloat16* const at = reinterpret_cast<__nv_bfloat16*>(hs + row * S::kHPitch + r * 2);
    at[0] = term(s);
    at[kRows * S::kHPitch / 2] = last_term == 1 ? __float2bfloat16_rn(s) : term(s);
    if (last_term == 2) at[2 * kRows * S::kHPitch / 2] = term(s);
  }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  __syncthreads();

  // ---- B (A x) for this block's rows of B
  for (int o = o0 + warp; o < o1; o += kSide * kWarps) {
    const int side = min(kSide, (o1 - o + kWarps - 1) / kWarps);
    float d[kSide][2][4] = {};
    for (int col0 = 0; col0 < rank; col0 += kDeep * 32) {
#pragma unroll
      for (int k = 0; k < kDeep; ++k)
        if (col0 + k * 32 < rank)
          multiply<false, std::is_same<W, __half>::value, 3>(d, hs + g * S::kHPitch + (col0 + k * 32 + q * 8) * 2, S::kHPitch, kRows * S::kHPitch, last_term + 1, w + k * kSide, side);
      if (col0 + kDeep * 32 < rank) load_b(o, col0 + kDeep * 32);
      else if (o + kSide * kWarps < o1) load_b(o + kSide * kWarps, 0);
    }
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      if (g + e * 4 >= n) continue;
      const long long at = (long long)t.rows[g + e * 4] * a.y_row;
#pragma unroll
      for (int j = 0; j < kSide; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int col = (o + j * kWarps) * 16 + h * 8 + q * 2;
          if (j < side && col < a.oc) add_pair(a.y, a.y_dtype, at + col, d[j][h][e], d[j][h][e + 1]);
        }
    }
  }
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");        // no block ends while another reads its share
}

template <typename X, typename W>
cudaError_t launch(Args p, long long items, cudaStream_t s) {
  using S = Shape<X, W>;
  static SmemOptIn opt_in(kCarveOut);
  cudaError_t e = opt_in((const void*)lowrank_kernel<X, W>, S::kBytes);
  if (e != cudaSuccess) return e;
  const unsigned C = 8;
  // where there are few tiles, several clusters divide a tile's rows of B, and each multiplies A x for itself
  p.splits = (int)std::max<long long>(1, std::min<long long>({2ll * sm_count() / (items * C), (p.a.oc + 16 * C * kWarps - 1) / (16 * C * kWarps), 16}));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(items * C * p.splits)); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = S::kBytes; cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, lowrank_kernel<X, W>, p);
}
template <typename X>
cudaError_t launch_x(const Args& p, long long items, cudaStream_t s) {
  return p.a.w_dtype == RWKVQ_F16 ? launch<X, __half>(p, items, s) : launch<X, __nv_bfloat16>(p, items, s);
}

int bytes_of(int dtype) { return dtype == RWKVQ_F32 ? 4 : dtype == RWKVQ_F16 || dtype == RWKVQ_BF16 ? 2 : 0; }

}  // namespace lr
}  // namespace rwkvq

using namespace rwkvq;

extern "C" {

rwkvq_status rwkvq_lowrank(const rwkvq_lowrank_args* args, const rwkvq_desc* mu_desc, const void* mu_image, void* stream) {
  if (!args) return RWKVQ_EINVAL;
  lr::Args p;
  p.a = *args;
  rwkvq_lowrank_args& a = p.a;
  const int xs = lr::bytes_of(a.x_dtype), ys = lr::bytes_of(a.y_dtype);
  if (xs == 0 || ys == 0 || (a.w_dtype != RWKVQ_F16 && a.w_dtype != RWKVQ_BF16)) return RWKVQ_EINVAL;
  if (a.tokens < 0 || a.n_seq <= 0 || a.ic <= 0 || a.oc <= 0 || a.rank <= 0 || a.n_adapters <= 0) return RWKVQ_EINVAL;
  if (!a.A || !a.B || !a.adapter || (a.tokens > 0 && (!a.x || !a.y))) return RWKVQ_EINVAL;
  if (!a.seq_start && a.n_seq != 1 && a.n_seq != a.tokens) return RWKVQ_EINVAL;
  if ((mu_image && !mu_desc) || ((a.x_prev || a.xprev0) && !mu_image) || (a.x_prev && a.xprev0)) return RWKVQ_EINVAL;
  if (a.rank > lr::kMostRank || a.n_seq > 65535 || a.tokens > (1 << 24) || a.ic > (1 << 24) || a.oc > (1 << 24)) return RWKVQ_EUNSUPPORTED;
  if (a.ic % 8 || a.oc % 8 || a.rank % 8) return RWKVQ_ESHAPE;
  if (mu_image) {
    const rwkvq_status st = check_vector_desc(mu_desc, a.ic);
    if (st != RWKVQ_OK) return st;
  }
  if (a.tokens > 1 && (a.x_row < a.ic || a.y_row < a.oc || (a.x_prev && a.x_prev_row < a.ic))) return RWKVQ_EINVAL;
  if (a.tokens > 0 && (a.y == a.x || a.y == a.x_prev || a.y == a.xprev0)) return RWKVQ_EINVAL;
  if (!aligned16(a.x) || !aligned16(a.x_prev) || !aligned16(a.xprev0) || !aligned16(a.A) || !aligned16(a.B) || !aligned16(a.y) || !aligned16(mu_image)) return RWKVQ_EALIGN;
  if (a.tokens > 1 && ((a.x_row * xs) % 16 || (a.y_row * ys) % 16 || (a.x_prev && (a.x_prev_row * xs) % 16))) return RWKVQ_EALIGN;
  if (a.tokens == 0) return RWKVQ_OK;
  p.mu = nullptr; p.mu_codebook = nullptr; p.mu_bits = 0; p.mu_entries = 0;
  if (mu_image) {
    p.mu = static_cast<const uint8_t*>(mu_image) + RWKVQ_HEADER_BYTES;
    p.mu_codebook = reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(mu_image) + vector_aux_offset(mu_desc));
    p.mu_bits = mu_desc->bits; p.mu_entries = mu_desc->entries;
  }
  p.status = device_status_ptr();
  if (!p.status) return RWKVQ_ECUDA;
  // tiles that there can be
  const long long full = ((long long)a.tokens + lr::kRows - 1) / lr::kRows;
  const long long items = a.seq_start ? std::min<long long>(a.tokens, full + a.n_seq) : a.n_seq == 1 ? full :
                          lr::by_groups(a) ? std::min<long long>(a.n_seq, a.n_adapters + full) : a.n_seq;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.x_dtype == RWKVQ_F32) return cuda_status(lr::launch_x<float>(p, items, s));
  if (a.x_dtype == RWKVQ_F16) return cuda_status(lr::launch_x<__half>(p, items, s));
  return cuda_status(lr::launch_x<__nv_bfloat16>(p, items, s));
}

}  // extern "C"
