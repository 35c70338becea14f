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

constexpr int kThreads = 256, kWarps = 8, kRows = 16, kMostRank = 128, kMostCols = 512;

struct Args {
  rwkvq_lowrank_args a;
  const uint8_t* mu;             // index stream of the token-shift vector, or nullptr
  const uint32_t* mu_codebook;
  int mu_bits, mu_entries;
  int* status;
};

// ---- rows of a tile -----------------------------------------------------------------------------------------
struct Tile {
  int rows[kRows], seqs[kRows];       // seqs: of a row that is its sequence's first, else -1 - sequence
  int n, adapter, rank;
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

__device__ void find_tile(const Args& p, long long item, Tile& t, int* scratch) {
  const rwkvq_lowrank_args& a = p.a;
  const int tid = threadIdx.x;
  if (tid == 0) t.n = 0;
  __syncthreads();
  if (!a.seq_start && a.n_seq == a.tokens && a.n_seq > 1) {
    // one row a sequence: the first, seventeenth, ... row of an adapter takes it and the next fifteen of the same adapter
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

template <bool kHalf>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&w)[4], uint32_t x0, uint32_t x1) {
  if constexpr (kHalf)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(x0), "r"(x1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(x0), "r"(x1));
}
// A pair of f16 weights as two pairs of bf16: eleven bits are eight and three.
__device__ __forceinline__ void apart(uint32_t w, uint32_t& hi, uint32_t& lo) {
  float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  __nv_bfloat162 h, l;
  h.x = term(f.x); h.y = term(f.y);
  l.x = term(f.x); l.y = term(f.y);
  hi = *reinterpret_cast<const uint32_t*>(&h); lo = *reinterpret_cast<const uint32_t*>(&l);
}

// How x and the weights go into the tensor cores.
template <typename X, typename W> struct Form {
  static constexpr bool kHalf = std::is_same<X, __half>::value && std::is_same<W, __half>::value;
  static constexpr int kX = std::is_same<X, W>::value ? 1 : std::is_same<X, float>::value ? 3 : std::is_same<X, __half>::value ? 2 : 1;
  static constexpr bool kApart = std::is_same<W, __half>::value && !kHalf;
};

__device__ __forceinline__ uint32_t mu_pair(const Args& p, const uint32_t* codebook, int pair) {
  const uint32_t bit = (uint32_t)pair * (uint32_t)p.mu_bits;
  const uint8_t* at = p.mu + (bit >> 3);
  const uint32_t two = (uint32_t)at[0] | ((bit & 7u) + p.mu_bits > 8u ? (uint32_t)at[1] << 8 : 0u);
  return codebook[(two >> (bit & 7u)) & ((1u << p.mu_bits) - 1u)];
}

template <typename X, typename W>
struct Shape {
  static constexpr int kTerms = Form<X, W>::kX;
  static constexpr int kPitch = kMostCols * 2 + 64;                   // bytes of a row of x in shared memory: 16-byte reads of two rows meet no bank twice
  static constexpr int kXBytes = kTerms * kRows * kPitch;
  static constexpr int kPart = kWarps * 16 * kRows * 4;               // partial sums: [group of warps][rank][row]
  static constexpr int kHPitch = kMostRank * 2 + 16;
  static constexpr int kHBytes = 3 * kRows * kHPitch;
  static constexpr int kBytes = kXBytes + kPart + kMostRank * kRows * 4 + kHBytes + 256 * 4;
};

template <typename X, typename W>
__global__ void __launch_bounds__(kThreads) lowrank_kernel(const Args p) {
  using S = Shape<X, W>;
  using F = Form<X, W>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Tile t;
  __shared__ int scratch[2 * kThreads + 2];
  uint8_t* const xs = smem;
  float* const part = reinterpret_cast<float*>(smem + S::kXBytes);
  float* const share = reinterpret_cast<float*>(smem + S::kXBytes + S::kPart);          // this block's share of A x: [rank][row]
  uint8_t* const hs = smem + S::kXBytes + S::kPart + kMostRank * kRows * 4;              // [term][row][rank]
  uint32_t* const codebook = reinterpret_cast<uint32_t*>(hs + S::kHBytes);
  const rwkvq_lowrank_args& a = p.a;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;

  find_tile(p, blockIdx.x / C, t, scratch);
  __syncthreads();
  const int n = t.n;
  if (n == 0) return;            // the same for all blocks of the cluster
  const int rank = t.rank, blocks = (rank + 15) / 16, blocks2 = (n + 7) / 8;
  if (p.mu)
    for (int i = tid; i < p.mu_entries; i += kThreads) codebook[i] = p.mu_codebook[i];

  // ---- A x over this block's columns
  const int units = (a.ic + 31) / 32, u0 = (int)((long long)units * c / C), u1 = (int)((long long)units * (c + 1) / C);
  // warps side by side along the rank as far as it reaches, the others along the columns
  int along = 1;
  while (along < kWarps && along < blocks) along *= 2;
  const int groups = kWarps / along, group = warp / along, wr = warp % along;
  const W* const A = static_cast<const W*>(a.A) + (long long)t.adapter * a.rank * a.ic;
  float acc[2][4] = {};
  for (int uc = u0; uc < u1; uc += kMostCols / 32) {
    const int ue = min(uc + kMostCols / 32, u1), cols = (ue - uc) * 32, eights = cols / 8;
    __syncthreads();
    for (int i = tid; i < kRows * eights; i += kThreads) {
      const int r = i / eights, col8 = i - r * eights, col = uc * 32 + col8 * 8;
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = 0.f;
      if (r < n && col < a.ic) {
        load8(static_cast<const X*>(a.x) + (long long)t.rows[r] * a.x_row + col, x);
        if (p.mu) {
          float y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = 0.f;
          const int seq = t.seqs[r];
          if (a.x_prev) load8(static_cast<const X*>(a.x_prev) + (long long)t.rows[r] * a.x_prev_row + col, y);
          else if (seq < 0) load8(static_cast<const X*>(a.x) + (long long)(t.rows[r] - 1) * a.x_row + col, y);
          else if (a.xprev0) load8(static_cast<const X*>(a.xprev0) + (long long)seq * a.ic + col, y);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t m2 = mu_pair(p, codebook, col / 2 + j);
            const float2 m = __half22float2(*reinterpret_cast<const __half2*>(&m2));
            x[2 * j] = to_float<X>(from_float<X>(fmaf(y[2 * j] - x[2 * j], m.x, x[2 * j])));
            x[2 * j + 1] = to_float<X>(from_float<X>(fmaf(y[2 * j + 1] - x[2 * j + 1], m.y, x[2 * j + 1])));
          }
        }
      }
#pragma unroll
      for (int k = 0; k < F::kX; ++k) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (F::kHalf) {
            const __half2 h = __floats2half2_rn(x[2 * j], x[2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t*>(&h);
          } else {
            __nv_bfloat162 h;
            h.x = term(x[2 * j]); h.y = term(x[2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t*>(&h);
          }
        }
        *reinterpret_cast<uint4*>(xs + (k * kRows + r) * S::kPitch + col8 * 16) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    __syncthreads();
    if (wr < blocks) {
      const int r0 = wr * 16 + g, r1 = r0 + 8;
      for (int u = uc + group; u < ue; u += groups) {
        const int col = u * 32 + q * 8;
        uint4 w0 = make_uint4(0, 0, 0, 0), w1 = w0;
        if (r0 < rank && col < a.ic) w0 = *reinterpret_cast<const uint4*>(A + (long long)r0 * a.ic + col);
        if (r1 < rank && col < a.ic) w1 = *reinterpret_cast<const uint4*>(A + (long long)r1 * a.ic + col);
        const uint32_t f[2][4] = {{w0.x, w1.x, w0.y, w1.y}, {w0.z, w1.z, w0.w, w1.w}};
        uint32_t hi[2][4], lo[2][4];
        if constexpr (F::kApart) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) apart(f[h][j], hi[h][j], lo[h][j]);
        }
#pragma unroll
        for (int k = F::kX - 1; k >= 0; --k)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            if (b >= blocks2) continue;
            const uint4 xv = *reinterpret_cast<const uint4*>(xs + (k * kRows + b * 8 + g) * S::kPitch + ((u - uc) * 32 + q * 8) * 2);
            if constexpr (F::kApart) {
              mma<false>(acc[b], lo[0], xv.x, xv.y); mma<false>(acc[b], lo[1], xv.z, xv.w);
              mma<false>(acc[b], hi[0], xv.x, xv.y); mma<false>(acc[b], hi[1], xv.z, xv.w);
            } else {
              mma<F::kHalf>(acc[b], f[0], xv.x, xv.y); mma<F::kHalf>(acc[b], f[1], xv.z, xv.w);
            }
          }
      }
    }
  }
  if (wr < blocks) {
    float* at = part + (group * along + wr) * 16 * kRows;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      *reinterpret_cast<float2*>(at + g * kRows + b * 8 + q * 2) = make_float2(acc[b][0], acc[b][1]);
      *reinterpret_cast<float2*>(at + (g + 8) * kRows + b * 8 + q * 2) = make_float2(acc[b][2], acc[b][3]);
    }
  }
  __syncthreads();
  for (int i = tid; i < blocks * 16 * kRows; i += kThreads) {
    float s = 0.f;
    for (int k = 0; k < groups; ++k) s += part[k * along * 16 * kRows + i];
    share[i] = s;
  }
  cluster.sync();

  // ---- all of A x, as operands
  const int last_term = a.y_dtype == RWKVQ_F32 ? 2 : 1;
  const float scale = a.scale ? a.scale[t.adapter] : 1.f;
  for (int i = tid; i < blocks * 16 * kRows; i += kThreads) {
    float s = 0.f;
    for (int k = 0; k < C; ++k) s += cluster.map_shared_rank(share, k)[i];
    s *= scale;
    const int r = i / kRows, row = i % kRows;
    __nv_bfloat16* const at = reinterpret_cast<__nv_bfloat16*>(hs + row * S::kHPitch + r * 2);
    at[0] = term(s);
    at[kRows * S::kHPitch / 2] = last_term == 1 ? __float2bfloat16_rn(s) : term(s);
    if (last_term == 2) at[2 * kRows * S::kHPitch / 2] = term(s);
  }
  cluster.sync();                // also: no block ends while another reads its share

  // ---- B (A x) for this block's rows of B
  const int tiles = (a.oc + 15) / 16, o0 = (int)((long long)tiles * c / C), o1 = (int)((long long)tiles * (c + 1) / C);
  const W* const Bm = static_cast<const W*>(a.B) + (long long)t.adapter * a.oc * a.rank;
  for (int o = o0 + warp; o < o1; o += kWarps) {
    const int r0 = o * 16 + g, r1 = r0 + 8;
    float d[2][4] = {};
    for (int ks = 0; ks < blocks; ++ks) {
      const int col = ks * 16 + q * 4;
      uint2 w0 = make_uint2(0, 0), w1 = w0;
      if (r0 < a.oc && col < rank) w0 = *reinterpret_cast<const uint2*>(Bm + (long long)r0 * a.rank + col);
      if (r1 < a.oc && col < rank) w1 = *reinterpret_cast<const uint2*>(Bm + (long long)r1 * a.rank + col);
      if (col + 4 > rank) {        // what lies behind the adapter's rank may be anything
        const uint32_t x = col + 2 > rank ? (col + 1 > rank ? 0u : 0xFFFFu) : ~0u, y = col + 4 > rank ? (col + 3 > rank ? 0u : 0xFFFFu) : ~0u;
        w0.x &= x; w1.x &= x; w0.y &= y; w1.y &= y;
      }
      const uint32_t f[4] = {w0.x, w1.x, w0.y, w1.y};
      uint32_t hi[4], lo[4];
      if constexpr (std::is_same<W, __half>::value) {
#pragma unroll
        for (int j = 0; j < 4; ++j) apart(f[j], hi[j], lo[j]);
      }
      for (int k = last_term; k >= 0; --k)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          if (b >= blocks2) continue;
          const uint2 h = *reinterpret_cast<const uint2*>(hs + (k * kRows + b * 8 + g) * S::kHPitch + col * 2);
          if constexpr (std::is_same<W, __half>::value) {
            mma<false>(d[b], lo, h.x, h.y);
            mma<false>(d[b], hi, h.x, h.y);
          } else {
            mma<false>(d[b], f, h.x, h.y);
          }
        }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = b * 8 + q * 2 + (j & 1), col = j < 2 ? r0 : r1;
        if (row >= n || col >= a.oc) continue;
        const long long at = (long long)t.rows[row] * a.y_row + col;
        if (a.y_dtype == RWKVQ_F32) static_cast<float*>(a.y)[at] += d[b][j];
        else if (a.y_dtype == RWKVQ_F16) static_cast<__half*>(a.y)[at] = __float2half_rn(__half2float(static_cast<__half*>(a.y)[at]) + d[b][j]);
        else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(__bfloat162float(static_cast<__nv_bfloat16*>(a.y)[at]) + d[b][j]);
      }
  }
}

template <typename X, typename W>
cudaError_t launch(const Args& p, long long items, cudaStream_t s) {
  using S = Shape<X, W>;
  static SmemOptIn opt_in(kCarveOut);
  cudaError_t e = opt_in((const void*)lowrank_kernel<X, W>, S::kBytes);
  if (e != cudaSuccess) return e;
  const unsigned C = 8;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)items * C); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = S::kBytes; cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
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
  const long long items = a.seq_start ? std::min<long long>(a.tokens, full + a.n_seq) : a.n_seq == 1 ? full : a.n_seq;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.x_dtype == RWKVQ_F32) return cuda_status(lr::launch_x<float>(p, items, s));
  if (a.x_dtype == RWKVQ_F16) return cuda_status(lr::launch_x<__half>(p, items, s));
  return cuda_status(lr::launch_x<__nv_bfloat16>(p, items, s));
}

}  // extern "C"
