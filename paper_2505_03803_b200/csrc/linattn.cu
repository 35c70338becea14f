// Linear attention with decaying state: per sequence and head, with S [N keys][N values] in fp32,
//   out_t = r_t (S + (u (.) k_t) v_t^T),   S <- diag(exp(lw_t)) S + k_t v_t^T.
//
// Single tokens and short sequences: linattn_token_kernel, the recurrence as it stands, S in registers.  One token reads and writes 2 * 4 * N * N bytes of
// state for 4 N^2 operations: HBM, and with few sequences latency, is all that counts (96 sequences, 64 heads: 33.0 us, 6.2 TB/s; one, 32 heads: 2.4).
// Prompts: chunks of sixteen tokens on the tensor cores, linattn_chunk_kernel, in two passes where a sequence is dealt out over several SMs.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/rwkvq.h"
#include "host_util.h"

namespace rwkvq {

int* device_status_ptr();  // api_misc.cu

namespace la {

// A sequence as the lists' checks leave it: rows [start, end), its state's slot (-1: none), or rows [0, 0) where it is left out.
struct Entry { int start, end, slot, unused; };

struct Args {
  rwkvq_linattn_args a;
  int* status;
  int limit;                // the token kernel takes sequences of at most so many rows, the chunk kernels the others
  // The chunk kernels' blocks: so many rows each of all heads' rows one head after the other, a head's rows `pitch` apart (more than there are, where no
  // block is to have rows of two heads).
  long long block_rows, pitch;
  Entry* entries;           // [n_seq], written by the token kernel; nullptr: one sequence, all rows, slot 0
  float* block_states;      // [blocks]: the state a block's last piece adds up, the one its sequence began with, the piece's decays
};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float f);
template <> __device__ __forceinline__ float from_f32<float>(float f) { return f; }
template <> __device__ __forceinline__ __half from_f32<__half>(float f) { return __float2half_rn(f); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float f) { return __float2bfloat16_rn(f); }

// Logarithm of the decay of row t, head h, channel c.
template <typename T>
__device__ __forceinline__ float log_decay(const rwkvq_linattn_args& a, long long t, int h, int c) {
  const long long at = t * a.logw_row + (a.decay_per_head ? h : (long long)h * a.n + c);
  return a.decay_dtype == RWKVQ_F32 ? static_cast<const float*>(a.logw)[at] : to_f32(static_cast<const T*>(a.logw)[at]);
}

// Rows [start, end) of sequence i; false (and the status word set) where seq_start is not a rising list within the rows.
__device__ __forceinline__ bool rows_of(const Args& p, int i, int& start, int& end) {
  start = 0; end = p.a.tokens;
  if (p.a.seq_start) { start = p.a.seq_start[i]; end = p.a.seq_start[i + 1]; }
  return (start >= 0) & (start <= end) & (end <= p.a.tokens);
}

constexpr int kTokenThreads = 128, kCols = 64;      // value columns of a block

// One block per sequence, head and 64 value columns.  Sixteen threads of four columns share a key row; eight such groups deal the key rows out.
template <typename T, int N>
__global__ void __launch_bounds__(kTokenThreads) linattn_token_kernel(const __grid_constant__ Args p) {
  constexpr int R = N / 8;
  __shared__ float4 rkw[N];                 // r, k, exp(lw), r * u * k
  __shared__ float vs[kCols];
  __shared__ float red[kTokenThreads / 32][kCols];
  const rwkvq_linattn_args& a = p.a;
  const int tid = threadIdx.x, h = blockIdx.x, seq = blockIdx.y, v0 = blockIdx.z * kCols;
  const int kg = tid >> 4, col = (tid & 15) * 4;
  int start, end, slot = seq;
  // (without branches on what is loaded: all loads of the lists are under way at once)
  bool bad = !rows_of(p, seq, start, end);
  if (a.slots) {
    slot = a.slots[seq];
    bad = bad | (slot < -1) | (slot >= a.n_slots);
  }
  // Sequences of a call share neither a state nor rows: one that begins in front of an entry of the list before its own could have rows of a sequence that is computed, and
  // the chunk kernels' blocks keep one state each for a sequence that goes on behind them.
  if (a.slots || a.seq_start) {
    for (int j = tid; j < seq; j += kTokenThreads) {
      const int other = a.slots ? a.slots[j] : -1, before = a.seq_start ? a.seq_start[j] : 0;
      bad = bad | (slot >= 0 && other == slot) | (before > start);
    }
  }
  bad = __syncthreads_or(bad);
  if (tid == 0 && h == 0 && v0 == 0) {
    if (bad) atomicExch(p.status, (int)RWKVQ_EINVAL);
    if (p.entries) p.entries[seq] = bad ? Entry{0, 0, -1, 0} : Entry{start, end, slot, 0};
  }
  if (bad || end - start > p.limit) return;
  const size_t at = (((size_t)max(slot, 0) * a.heads + h) * N + kg * R) * N + v0 + col;
  float4 S[R];
#pragma unroll
  for (int i = 0; i < R; ++i)
    S[i] = a.state && slot >= 0 ? __ldcs(reinterpret_cast<const float4*>(a.state + at + (size_t)i * N)) : make_float4(0.f, 0.f, 0.f, 0.f);
  for (int t = start; t < end; ++t) {
    if (tid < N) {
      const long long c = (long long)h * N + tid;
      const float r = to_f32(static_cast<const T*>(a.r)[t * a.r_row + c]), k = to_f32(static_cast<const T*>(a.k)[t * a.k_row + c]);
      const float w = expf(log_decay<T>(a, t, h, tid)), u = a.u ? a.u[c] : 1.f;
      rkw[tid] = make_float4(r, k, w, r * u * k);
    }
    if (tid < kCols) vs[tid] = to_f32(static_cast<const T*>(a.v)[t * a.v_row + (long long)h * N + v0 + tid]);
    __syncthreads();
    const float4 v = *reinterpret_cast<const float4*>(&vs[col]);
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    float b = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float4 q = rkw[kg * R + i];
      y.x = fmaf(q.x, S[i].x, y.x); y.y = fmaf(q.x, S[i].y, y.y); y.z = fmaf(q.x, S[i].z, y.z); y.w = fmaf(q.x, S[i].w, y.w);
      b += q.w;
      S[i].x = fmaf(q.z, S[i].x, q.y * v.x); S[i].y = fmaf(q.z, S[i].y, q.y * v.y);
      S[i].z = fmaf(q.z, S[i].z, q.y * v.z); S[i].w = fmaf(q.z, S[i].w, q.y * v.w);
    }
    y.x = fmaf(b, v.x, y.x); y.y = fmaf(b, v.y, y.y); y.z = fmaf(b, v.z, y.z); y.w = fmaf(b, v.w, y.w);
    y.x += __shfl_xor_sync(0xFFFFFFFFu, y.x, 16); y.y += __shfl_xor_sync(0xFFFFFFFFu, y.y, 16);
    y.z += __shfl_xor_sync(0xFFFFFFFFu, y.z, 16); y.w += __shfl_xor_sync(0xFFFFFFFFu, y.w, 16);
    if ((tid & 31) < 16) *reinterpret_cast<float4*>(&red[tid >> 5][col]) = y;
    __syncthreads();
    if (tid < kCols) {
      float o = 0.f;
#pragma unroll
      for (int i = 0; i < kTokenThreads / 32; ++i) o += red[i][tid];
      static_cast<T*>(a.out)[t * a.out_row + (long long)h * N + v0 + tid] = from_f32<T>(o);
    }
  }
  if (a.state_out && slot >= 0) {
#pragma unroll
    for (int i = 0; i < R; ++i) __stcs(reinterpret_cast<float4*>(a.state_out + at + (size_t)i * N), S[i]);
  }
}

// ---- chunks -------------------------------------------------------------------------------------------------
// Sixteen tokens at a time.  With P_t, Q_s the products of the decays from the chunk's beginning to t and from behind s to its end, D all of them:
//   out_t = (r_t P_t) S + sum_{s <= t} A[t][s] v_s,   S <- D S + sum_s (k_s Q_s) v_s^T,
//   A[t][s] = sum_i r_t k_s prod_{s < x < t} w_x  (s < t),  sum_i r_t u k_t  (s = t).
// Nothing is divided by a decay: products of decays may underflow to the zero that they mean.  The 8 x 8 block of A below the diagonal is a product of
// (r_t P'_t) and (k_s Q'_s), P' and Q' from and to the chunk's middle; the two triangles are added up in fp32 with a running product along t.
//
// The products run on mma.sync.m16n8k16 with operands of several bf16 terms (hi + lo + ...), whose exponents reach as far as fp32's: r P and S with two
// (2^-17 of each; the output is rounded to 2^-9 or 2^-12), k Q with three (all 24 bits: it goes into the fp32 state), v with as many as it has
// (bf16 one, fp16 two); fp32 inputs take three of everything.  mma.sync and not tcgen05: S stays in registers from chunk to chunk as the accumulator of
// S^T, in the layout in which the next product takes it as its operand; through tensor memory it would have to be read, split and written every 16 tokens.
//
// A block has one head at a time.  Half of its warps or more make a chunk's operands (loads, exponentials, running products, splitting, the triangles) while
// the others multiply the chunk before it; these have 16 or 32 value columns each, so that they share r P, k Q and A but no sums.  Two sets of operands and named
// barriers go between them.  (All warps doing both in turn: 77 us where this takes 69, 2048 tokens of 64 heads; 14.8 and 11.2 with 203 of 32, where latency is all.)
// Rows are cut into blocks of block_rows, dealt out over the SMs: first (kStateOnly) the state that each block's last piece adds up from zero (or from its
// sequence's own), where the sequence goes on behind the block; then all blocks at once, each beginning with what those before it left.
//
// What bounds it, 2048 tokens, 64 heads, bf16, decays fp32: 25 us the states' pass, 57 the other (ncu, cold and alone; 71 in all, call after call and one under the other), of which HBM needs 15.5.
// Of the cycles that an SM is active, shared memory's data path is busy 53 % (operands are written once and read by all multiplying warps), issue slots 49 %, the tensor pipe 28 %, with
// twelve warps in 168 registers: neither a full pipe nor enough warps to wait beside one another.  A chunk is about 3 100 warp instructions.  Taken back: parts of a block halved over a cluster in the states' pass (no gain, 203 tokens 11.3 -> 13.2), five
// stages of inputs (no gain), three or four blocks an SM (spills), the triangles through shared memory (82 us where registers took 77).
// 203 tokens, 32 heads 12.3; 5000 rows of eleven sequences, one decay a head, fp16 179; fp32, N 128, 1111 tokens of 16 heads 57 (no pipe full there either: tensor
// pipe 36 %, issue slots 34 %, data path 45 %, one block of sixteen warps an SM; in 128 registers a thread the outputs' pass spills 48 bytes, with a decay per head 24, and 68 with
// fp16, N 128 and a decay per head).

template <typename T> struct Terms;
template <> struct Terms<__nv_bfloat16> { static constexpr int R = 2, V = 1; };
template <> struct Terms<__half> { static constexpr int R = 2, V = 2; };
template <> struct Terms<float> { static constexpr int R = 3, V = 3; };
constexpr int kChunk = 16, kHalf = 8, K3 = 3;

template <typename T, int N, bool kStateOnly>
struct Shape {
  // Warps that make operands, warps that multiply: each of these has kValues tiles of 16 value columns.  Two, so that what they read of r P and k Q serves more
  // products: 72.3 -> 69.2 us (2048 tokens, 64 heads, bf16); with fp16's two terms of v it is slower, 174 -> 185 (ragged, 5000 rows), and of heads of 128 the states of two
  // would not fit the registers.
  static constexpr int kValues = N == 64 && Terms<T>::V == 1 ? 2 : 1, kThreads = 2 * N, kMulThreads = 2 * N / kValues, kAll = kThreads + kMulThreads;
  static constexpr int kTiles = N / 8, kSteps = N / 16, kMidSteps = kSteps / (kMulThreads / 32);
  static constexpr int R = Terms<T>::R, V = Terms<T>::V;
  static constexpr int kPitch = (N + 8) * 2;                      // bytes of a row of terms: an odd number of 16 bytes, no conflicts for ldmatrix
  static constexpr int kRawPitch = N * (int)sizeof(T) + 16, kDecayPitch = N * 4 + 16;
  static constexpr int kTerm = kChunk * kPitch, kHalfTerm = kHalf * kPitch, kRaw = kChunk * kRawPitch;
  // a raw stage: r (where there are outputs), k, v, logarithms of decays
  static constexpr int kStages = 3, kAhead = kStages - 2;      // chunks on their way
  static constexpr int kR = 0, kK = kStateOnly ? 0 : kRaw, kV = kK + kRaw, kL = kV + kRaw, kStage = kL + kChunk * kDecayPitch;
  // a set of operands
  static constexpr int kKt = 0, kD = kKt + K3 * kTerm, kVt = kD + N * 4, kRt = kVt + (V > 2 ? V * kTerm : 0);
  // what only outputs need
  static constexpr int kRp = kRt + R * kTerm, kKp = kRp + R * kHalfTerm, kA = kKp + R * kHalfTerm, kTriangles = (N / 64) * 2 * 64 * 4;
  static constexpr int kSet = kStateOnly ? kRt : kA + kTriangles, oSets = kStages * kStage, oMid = oSets + 2 * kSet;
  static constexpr int kBytes = oMid + (kStateOnly ? 0 : kMulThreads / 32 * 64 * 4);
  static constexpr int kStateFloats = N * N, kBlockFloats = 2 * N * N + N;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp_async16(void* dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two fp32 numbers side by side: one instruction multiplies, adds or subtracts both.
typedef unsigned long long pair;
__device__ __forceinline__ pair pair_of(float x, float y) {
  pair v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
  return v;
}
__device__ __forceinline__ float2 both(pair v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
__device__ __forceinline__ pair mul2(pair a, pair b) { pair d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ pair add2(pair a, pair b) { pair d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ pair fma2(pair a, pair b, pair c) { pair d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
// e^l of both.  Below 2^-126 it is zero (a decay of that size leaves nothing; keeping subnormal numbers takes four more instructions each).
__device__ __forceinline__ pair exp_both(pair l) {
  const float2 f = both(mul2(l, pair_of(1.4426950408889634f, 1.4426950408889634f)));
  float x, y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(f.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(f.y));
  return pair_of(x, y);
}
__device__ __forceinline__ pair ones() { return pair_of(1.f, 1.f); }
__device__ __forceinline__ pair load2(const float* p) { return *reinterpret_cast<const pair*>(p); }
__device__ __forceinline__ pair widen(uint32_t v, __half) { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v)); return pair_of(f.x, f.y); }
__device__ __forceinline__ pair widen(uint32_t v, __nv_bfloat16) { return pair_of(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)); }
template <typename T> __device__ __forceinline__ pair load2(const T* p) { return widen(*reinterpret_cast<const uint32_t*>(p), T()); }
// Four numbers.
__device__ __forceinline__ void load4(const float* p, pair (&v)[2]) { const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(p); v[0] = q.x; v[1] = q.y; }
template <typename T> __device__ __forceinline__ void load4(const T* p, pair (&v)[2]) {
  const uint2 q = *reinterpret_cast<const uint2*>(p);
  v[0] = widen(q.x, T()); v[1] = widen(q.y, T());
}
// (x, y) as n bf16 terms, x in the low half: each term is what the ones before it leave, rounded.
template <int n>
__device__ __forceinline__ void split(pair v, uint32_t (&t)[n]) {
#pragma unroll
  for (int i = 0; i < n; ++i) {
    const float2 f = both(v);
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    t[i] = *reinterpret_cast<const uint32_t*>(&h);
    if (i + 1 < n) v = fma2(widen(t[i], __nv_bfloat16()), pair_of(-1.f, -1.f), v);
  }
}
template <int n>
__device__ __forceinline__ void store_split(uint8_t* at, int term_bytes, pair v) {
  uint32_t t[n];
  split<n>(v, t);
#pragma unroll
  for (int i = 0; i < n; ++i) *reinterpret_cast<uint32_t*>(at + i * term_bytes) = t[i];
}
// Barriers of a block, by number (0 is __syncthreads).
enum { kFull = 1, kEmpty = 3, kMakers = 5, kMultipliers = 6 };
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// Where the logarithms of decays come from.
enum { DECAY_F32 = 0, DECAY_SAME = 1, DECAY_HEAD = 2 };

template <typename T, int N, int kDecay, bool kStateOnly>
struct Worker {
  using Sh = Shape<T, N, kStateOnly>;
  const Args& p;
  uint8_t* sm;
  int h, warp, lane, tid;      // tid, warp: in its role
  int count = 0, stage = 0;    // chunks so far, stage of the next one
  float S[Sh::kValues][Sh::kTiles][4];      // S^T: values 16 (kValues warp + m) + lane / 4 (+ 8: the last two), keys 8 j + 2 (lane % 4) and the next
  pair total;                  // kStateOnly: sums of the logarithms of the decays of this thread's channels
  // This thread's pieces of 16 bytes of the next chunk to fetch, and bytes from row to row.
  static constexpr int kPieces = N * (int)sizeof(T) / 16, kRowsAtOnce = Sh::kThreads / kPieces;
  static constexpr int kDecaySize = kDecay == DECAY_F32 ? 4 : (int)sizeof(T), kDecayPieces = N * kDecaySize / 16, kDecayRowsAtOnce = Sh::kThreads / kDecayPieces;
  const uint8_t *rp, *kp, *vp, *lp;
  float ahead;
  pair bonus;                  // u of this thread's channels
  int place, place2;           // bytes into a triangle of A of the entries that this lane ends up with

  __device__ __forceinline__ Worker(const Args& p_, uint8_t* sm_) : p(p_), sm(sm_), warp((threadIdx.x & (2 * N - 1)) >> 5), lane(threadIdx.x & 31),
        tid(threadIdx.x & (2 * N - 1)) {
    if (kStateOnly) return;
    const int set = (warp & 3) < 2 ? 0 : 1;
    place = entry(set, lane >> 1) * 4;
    place2 = entry(set, 16 + (lane & 1)) * 4;
  }

  __device__ __forceinline__ void fetch_from(int t0) {
    const rwkvq_linattn_args& a = p.a;
    const long long row = t0 + tid / kPieces, off = (long long)h * N * (int)sizeof(T) + tid % kPieces * 16;
    rp = static_cast<const uint8_t*>(a.r) + row * a.r_row * (int)sizeof(T) + off;
    kp = static_cast<const uint8_t*>(a.k) + row * a.k_row * (int)sizeof(T) + off;
    vp = static_cast<const uint8_t*>(a.v) + row * a.v_row * (int)sizeof(T) + off;
    if (kDecay == DECAY_HEAD) lp = static_cast<const uint8_t*>(a.logw) + ((t0 + (tid & 15)) * a.logw_row + h) * (a.decay_dtype == RWKVQ_F32 ? 4 : (int)sizeof(T));
    else lp = static_cast<const uint8_t*>(a.logw) + ((t0 + tid / kDecayPieces) * a.logw_row + (long long)h * N) * kDecaySize + tid % kDecayPieces * 16;
  }
  // One decay per head: the next chunk's, `left` rows of it in the sequence.
  __device__ __forceinline__ void head_decay(int left) {
    if (tid < kChunk && tid < left)
      ahead = p.a.decay_dtype == RWKVQ_F32 ? *reinterpret_cast<const float*>(lp) : to_f32(*reinterpret_cast<const T*>(lp));
  }
  // The next 16 rows into a raw stage, `left` of them in the sequence; zeros (no decay, nothing to add) behind.
  __device__ __forceinline__ void fetch(int stage, int left) {
    const rwkvq_linattn_args& a = p.a;
    uint8_t* dst = sm + stage * Sh::kStage + tid / kPieces * Sh::kRawPitch + tid % kPieces * 16;
    const int rb = (int)sizeof(T) * kRowsAtOnce;
#pragma unroll
    for (int i = 0; i < kChunk / kRowsAtOnce; ++i) {
      const bool there = tid / kPieces + i * kRowsAtOnce < left;
      // a row that is not there is not read: the address is one that is
      if (!kStateOnly) cp_async16(dst + i * kRowsAtOnce * Sh::kRawPitch, there ? rp : static_cast<const uint8_t*>(a.r), there);
      cp_async16(dst + i * kRowsAtOnce * Sh::kRawPitch + Sh::kK, there ? kp : static_cast<const uint8_t*>(a.k), there);
      cp_async16(dst + i * kRowsAtOnce * Sh::kRawPitch + Sh::kV, there ? vp : static_cast<const uint8_t*>(a.v), there);
      rp += a.r_row * rb; kp += a.k_row * rb; vp += a.v_row * rb;
    }
    uint8_t* lw = sm + stage * Sh::kStage + Sh::kL;
    if (kDecay == DECAY_HEAD) {
      // a plain load, one chunk ahead: what it brings is stored when the next chunk is asked for
      if (tid < kChunk) reinterpret_cast<float*>(lw)[tid] = tid < left ? ahead : 0.f;
      lp += a.logw_row * ((a.decay_dtype == RWKVQ_F32 ? 4 : (int)sizeof(T)) * kChunk);
      head_decay(left - kChunk);
    } else {
#pragma unroll
      for (int i = 0; i < kChunk / kDecayRowsAtOnce; ++i) {
        const int t = tid / kDecayPieces + i * kDecayRowsAtOnce;
        cp_async16(lw + t * Sh::kDecayPitch + tid % kDecayPieces * 16, t < left ? lp : static_cast<const uint8_t*>(a.logw), t < left);
        lp += a.logw_row * (kDecaySize * kDecayRowsAtOnce);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }

  __device__ __forceinline__ pair decay2(const uint8_t* lw, int t, int c) const {
    if (kDecay == DECAY_HEAD) { const float v = reinterpret_cast<const float*>(lw)[t]; return pair_of(v, v); }
    const uint8_t* row = lw + t * Sh::kDecayPitch;
    return kDecay == DECAY_F32 ? load2(reinterpret_cast<const float*>(row) + c) : load2(reinterpret_cast<const T*>(row) + c);
  }

  // Entry number i of 18 of a set of columns: (t, s).  Constant where i and the set are.
  static __device__ __forceinline__ int entry(int set, int i) {
    constexpr int kFirst[2][4] = {{0, 3, 5, 6}, {1, 2, 4, 7}};
    int n = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int s = kFirst[set][j], len = kHalf - s;          // the diagonal first
      if (i < n + len) return (s + i - n) * 8 + s;
      n += len;
    }
    return 0;
  }
  // This lane's part (two channels) of the entries of a set.
  template <int set>
  __device__ __forceinline__ void entries(const pair (&r)[kHalf], const pair (&k)[kHalf], const pair (&w)[kHalf], float (&v)[18]) const {
    constexpr int kFirst[2][4] = {{0, 3, 5, 6}, {1, 2, 4, 7}};
    int n = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int s = kFirst[set][j];
      pair x = k[s];
      {
        const float2 f = both(mul2(mul2(r[s], bonus), x));
        v[n++] = f.x + f.y;
      }
#pragma unroll
      for (int t = s + 1; t < kHalf; ++t) {
        const float2 f = both(mul2(r[t], x));
        v[n++] = f.x + f.y;
        if (t + 1 < kHalf) x = mul2(x, w[t]);
      }
    }
  }

  // Without outputs only k Q is needed: a warp of a group of four takes four tokens (the last first, as the sums of the decays behind them are longer).
  __device__ __forceinline__ void state_operands(int stage, uint8_t* set) {
    constexpr int kQuarter = 4;
    const uint8_t* st = sm + stage * Sh::kStage;
    const uint8_t* lw = st + Sh::kL;
    const int c = (warp >> 2) * 64 + lane * 2, t0 = (3 - (warp & 3)) * kQuarter;
    pair x[kQuarter], l[kQuarter], s = pair_of(0.f, 0.f);
#pragma unroll
    for (int t = 0; t < kQuarter; ++t) {
      x[t] = load2(reinterpret_cast<const T*>(st + Sh::kK + (t0 + t) * Sh::kRawPitch) + c);
      l[t] = decay2(lw, t0 + t, c);
    }
#pragma unroll
    for (int t = kQuarter; t < kChunk; ++t)
      if (t >= t0 + kQuarter) s = add2(s, decay2(lw, t, c));
    uint8_t* const to = set + t0 * Sh::kPitch + c * 2;
    pair v[kQuarter];
    if (Sh::V > 2) {
#pragma unroll
      for (int t = 0; t < kQuarter; ++t) v[t] = load2(reinterpret_cast<const T*>(st + Sh::kV + (t0 + t) * Sh::kRawPitch) + c);
    }
    // exponentials of sums, not products of exponentials: they do not wait for one another
#pragma unroll
    for (int t = kQuarter - 1; t >= 0; --t) {
      store_split<K3>(to + Sh::kKt + t * Sh::kPitch, Sh::kTerm, mul2(x[t], exp_both(s)));
      s = add2(s, l[t]);
    }
    if (Sh::V > 2) {
#pragma unroll
      for (int t = 0; t < kQuarter; ++t) store_split<Sh::V>(to + Sh::kVt + t * Sh::kPitch, Sh::kTerm, v[t]);
    }
    if (t0 == 0) {
      const float2 f = both(s);
      *reinterpret_cast<float2*>(set + Sh::kD + c * 4) = make_float2(expf(f.x), expf(f.y));
      total = add2(total, s);
    }
  }

  // A stage's operands.  Warps of a group of four take: r of the first eight tokens, r of the last, k of the last, k of the first; a lane two channels.
  __device__ __forceinline__ void operands(int stage, uint8_t* set) {
    const uint8_t* st = sm + stage * Sh::kStage;
    const uint8_t* lw = st + Sh::kL;
    const int role = warp & 3, c = (warp >> 2) * 64 + lane * 2;
    // All that a role reads is read before it writes: the compiler cannot tell that what is written lies elsewhere, and would wait for each read in turn.
    const int t0 = role == 0 || role == 3 ? 0 : kHalf;
    pair x[kHalf], l[kHalf], w[kHalf], s = ones(), q = ones();
#pragma unroll
    for (int t = 0; t < kHalf; ++t)
      x[t] = load2(reinterpret_cast<const T*>(st + (role < 2 ? Sh::kR : Sh::kK) + (t0 + t) * Sh::kRawPitch) + c);
#pragma unroll
    for (int t = 0; t < kHalf; ++t) l[t] = decay2(lw, t0 + t, c);
    if (role & 1) {            // the decays of the other half
      s = decay2(lw, kHalf - t0, c);
#pragma unroll
      for (int t = 1; t < kHalf; ++t) s = add2(s, decay2(lw, kHalf - t0 + t, c));
    }
#pragma unroll
    for (int t = 0; t < kHalf; ++t) w[t] = exp_both(l[t]);
    uint8_t* const to = set + t0 * Sh::kPitch + c * 2;
    if (role < 2) {
      if (role == 1) {
        pair all = s;
#pragma unroll
        for (int t = 0; t < kHalf; ++t) all = add2(all, l[t]);
        // the state's decay, over and over the same where decays do not change: the accurate exponential of the sum
        const float2 f = both(all);
        *reinterpret_cast<float2*>(set + Sh::kD + c * 4) = make_float2(expf(f.x), expf(f.y));
      }
      const pair d = role == 1 ? exp_both(s) : s;
#pragma unroll
      for (int t = 0; t < kHalf; ++t) {
        pair m = mul2(x[t], q);
        if (role == 1) {
          store_split<Sh::R>(to + Sh::kRp + (t - kHalf) * Sh::kPitch, Sh::kHalfTerm, m);
          m = mul2(m, d);
        }
        store_split<Sh::R>(to + Sh::kRt + t * Sh::kPitch, Sh::kTerm, m);
        q = mul2(q, w[t]);
      }
    } else {
      const pair d = role == 3 ? exp_both(s) : s;
#pragma unroll
      for (int t = kHalf - 1; t >= 0; --t) {
        pair m = mul2(x[t], q);
        if (role == 3) {
          store_split<Sh::R>(to + Sh::kKp + t * Sh::kPitch, Sh::kHalfTerm, m);
          m = mul2(m, d);
        }
        store_split<K3>(to + Sh::kKt + t * Sh::kPitch, Sh::kTerm, m);
        q = mul2(q, w[t]);
      }
    }
    {
      // The triangles of A: tokens 0-7 by roles 0 and 3, tokens 8-15 by 1 and 2, which have one of r and k and the decays in registers and read the other.
      // Seven columns have entries below the diagonal, 7 - s each: the warps with r take s = 0, 3, 5, 6, those with k 1, 2, 4, fourteen entries either way,
      // and four of the eight on the diagonal.
      pair y[kHalf];
#pragma unroll
      for (int t = 0; t < kHalf; ++t)
        y[t] = load2(reinterpret_cast<const T*>(st + (role < 2 ? Sh::kK : Sh::kR) + (t0 + t) * Sh::kRawPitch) + c);
      float v[18];
      if (role < 2) entries<0>(x, y, w, v);
      else entries<1>(y, x, w, v);
      // sixteen sums over the lanes, each step halves the values that a lane carries, and two more
#pragma unroll
      for (int d = 16, n = 8; d > 1; d >>= 1, n >>= 1) {
        const bool up = (lane & d) != 0;
#pragma unroll
        for (int i = 0; i < n; ++i) {
          const float keep = up ? v[i + n] : v[i], send = up ? v[i] : v[i + n];
          v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, d);
        }
      }
      v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], 1);
      {
        const bool up = (lane & 1) != 0;
        const float keep = up ? v[17] : v[16], send = up ? v[16] : v[17];
        v[16] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, 1);
      }
#pragma unroll
      for (int d = 16; d > 1; d >>= 1) v[16] += __shfl_xor_sync(0xFFFFFFFFu, v[16], d);
      // lane 2 i holds entry i, lanes 0 and 1 the last two: where these are in A
      uint8_t* A = set + Sh::kA + (warp >> 2) * 512 + (t0 >> 3) * 256;
      if ((lane & 1) == 0) *reinterpret_cast<float*>(A + place) = v[0];
      if (lane < 2) *reinterpret_cast<float*>(A + place2) = v[16];
    }
    if (Sh::V > 2 && (role & 1) == 0) {       // the warps with less to do
#pragma unroll
      for (int t = 0; t < kHalf; ++t) x[t] = load2(reinterpret_cast<const T*>(st + Sh::kV + (t0 + t) * Sh::kRawPitch) + c);
#pragma unroll
      for (int t = 0; t < kHalf; ++t) store_split<Sh::V>(to + Sh::kVt + t * Sh::kPitch, Sh::kTerm, x[t]);
    }
  }

  // Chunks of rows [begin, end), by the warps that make operands.  The next kAhead chunks are on their way while one is worked on; sets and stages go on being used in
  // turn from one piece of rows to the next, so that a piece's first chunks are made while the piece before it is multiplied.
  __device__ __forceinline__ void make(int begin, int end) {
    const int n = (end - begin + kChunk - 1) / kChunk;
    if (!kStateOnly) bonus = p.a.u ? load2(p.a.u + h * N + (warp >> 2) * 64 + lane * 2) : ones();
    fetch_from(begin);
    if (kDecay == DECAY_HEAD) head_decay(end - begin);
    int into = stage, left = end - begin;            // where the next chunk to fetch goes, and the rows from it on
    auto next_chunk = [&]() {
      fetch(into, left);
      into = into == Sh::kStages - 1 ? 0 : into + 1;
      left -= kChunk;
    };
    for (int i = 0; i < Sh::kAhead && i < n; ++i) next_chunk();
    for (int i = 0; i < n; ++i, ++count) {
      const int set = count & 1;
      if (count >= 2) bar_sync(kEmpty + set, Sh::kAll);       // the chunk before the last is done with: its set of operands, and its stage
      if (i + Sh::kAhead < n) {
        next_chunk();
        asm volatile("cp.async.wait_group %0;" ::"n"(Sh::kAhead) : "memory");
      } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      bar_sync(kMakers, Sh::kThreads);
      if (kStateOnly) state_operands(stage, sm + Sh::oSets + set * Sh::kSet);
      else operands(stage, sm + Sh::oSets + set * Sh::kSet);
      bar_arrive(kFull + set, Sh::kAll);
      stage = stage == Sh::kStages - 1 ? 0 : stage + 1;
    }
  }
  // Behind the last piece: what the other warps report is waited for, so that no barrier is left half done.
  __device__ __forceinline__ void made() {
    for (int i = max(count - 2, 0); i < count; ++i) bar_sync(kEmpty + (i & 1), Sh::kAll);
  }
  // The same chunks by the warps that multiply.
  __device__ __forceinline__ void multiply(int begin, int end) {
    const rwkvq_linattn_args& a = p.a;
    const int n = (end - begin + kChunk - 1) / kChunk, g = lane >> 2, q = lane & 3;
    for (int i = 0; i < n; ++i, ++count) {
      const int t0 = begin + i * kChunk, turn = count & 1;
      const uint8_t* set = sm + Sh::oSets + turn * Sh::kSet;
      bar_sync(kFull + turn, Sh::kAll);
      float o[Sh::kValues][2][4];
      if (!kStateOnly) {
#pragma unroll
        for (int m = 0; m < Sh::kValues; ++m)
#pragma unroll
          for (int nb = 0; nb < 2; ++nb)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[m][nb][x] = 0.f;
        {
          // the block of A below the triangles: each warp adds up its share of the keys.  Rows of r P' (lanes 0-15) and of k Q' (16-31), eight keys and the next
          float mid[4] = {0.f, 0.f, 0.f, 0.f};
          const uint32_t half = smem_u32(set + (lane < 16 ? Sh::kRp : Sh::kKp)) + (lane & 7) * Sh::kPitch + ((lane >> 3) & 1) * 16 + warp * Sh::kMidSteps * 32;
#pragma unroll
          for (int k = 0; k < Sh::kMidSteps; ++k) {
            uint32_t y[Sh::R][4];
#pragma unroll
            for (int e = 0; e < Sh::R; ++e) ldsm4(half + e * Sh::kHalfTerm + k * 32, y[e]);
#pragma unroll
            for (int e = 0; e < Sh::R; ++e)
#pragma unroll
              for (int f = 0; f < Sh::R - e; ++f) {
                const uint32_t low[4] = {0u, y[e][0], 0u, y[e][1]};
                mma(mid, low, y[f][2], y[f][3]);
              }
          }
          *reinterpret_cast<float2*>(sm + Sh::oMid + (warp * 64 + g * 8 + q * 2) * 4) = make_float2(mid[2], mid[3]);
        }
        const uint32_t rt = smem_u32(set + Sh::kRt) + (lane & 15) * Sh::kPitch + (lane >> 4) * 16;
#pragma unroll
        for (int k = 0; k < Sh::kSteps; ++k) {
          uint32_t x[Sh::R][4];
#pragma unroll
          for (int e = 0; e < Sh::R; ++e) ldsm4(rt + e * Sh::kTerm + k * 32, x[e]);
#pragma unroll
          for (int m = 0; m < Sh::kValues; ++m) {
            uint32_t b[2][2][Sh::R];
#pragma unroll
            for (int nb = 0; nb < 2; ++nb)
#pragma unroll
              for (int i2 = 0; i2 < 2; ++i2) split<Sh::R>(pair_of(S[m][2 * k + i2][2 * nb], S[m][2 * k + i2][2 * nb + 1]), b[nb][i2]);
#pragma unroll
            for (int e = 0; e < Sh::R; ++e)
#pragma unroll
              for (int f = 0; f < Sh::R - e; ++f) {
                mma(o[m][0], x[e], b[0][0][f], b[0][1][f]);
                mma(o[m][1], x[e], b[1][0][f], b[1][1][f]);
              }
          }
        }
      }
      // values of the chunk's tokens: an operand of both products that follow
      uint32_t v[Sh::kValues][Sh::V][4], wild = 0;         // wild: the top bits of halves with infinities or NaN among them
#pragma unroll
      for (int m = 0; m < Sh::kValues; ++m) {
        const int row = (lane & 7) + (lane >> 4) * 8, col = (warp * Sh::kValues + m) * 16 + ((lane >> 3) & 1) * 8;
        if constexpr (Sh::V > 2) {
          const uint32_t at = smem_u32(set + Sh::kVt) + row * Sh::kPitch + col * 2;
#pragma unroll
          for (int e = 0; e < Sh::V; ++e) ldsm4t(at + e * Sh::kTerm, v[m][e]);
#pragma unroll
          for (int j = 0; j < 4; ++j) wild |= (v[m][0][j] & 0x7F807F80u) + 0x00800080u;
        } else {
          uint32_t x[4];
          ldsm4t(smem_u32(sm + stage * Sh::kStage + Sh::kV) + row * Sh::kRawPitch + col * 2, x);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            wild |= Sh::V == 1 ? (x[j] & 0x7F807F80u) + 0x00800080u : (x[j] & 0x7C007C00u) + 0x04000400u;
            if constexpr (Sh::V == 1) v[m][0][j] = x[j];
            else {
              uint32_t t[Sh::V];
              split<Sh::V>(widen(x[j], T()), t);
#pragma unroll
              for (int e = 0; e < Sh::V; ++e) v[m][e][j] = t[e];
            }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < Sh::kTiles; ++j) {
        const pair d = *reinterpret_cast<const pair*>(set + Sh::kD + (j * 8 + q * 2) * 4);
#pragma unroll
        for (int m = 0; m < Sh::kValues; ++m) {
          float(&c)[4] = S[m][j];
          const float2 lo = both(mul2(pair_of(c[0], c[1]), d)), hi = both(mul2(pair_of(c[2], c[3]), d));
          c[0] = lo.x; c[1] = lo.y; c[2] = hi.x; c[3] = hi.y;
        }
      }
      {
        const uint32_t kt = smem_u32(set + Sh::kKt) + (lane & 15) * Sh::kPitch + (lane >> 4) * 16;
#pragma unroll
        for (int f = 0; f < K3; ++f)
#pragma unroll
          for (int k = 0; k < Sh::kSteps; ++k) {
            uint32_t b[4];
            ldsm4t(kt + f * Sh::kTerm + k * 32, b);
#pragma unroll
            for (int m = 0; m < Sh::kValues; ++m)
#pragma unroll
              for (int e = 0; e < Sh::V && e + f < K3; ++e) {
                mma(S[m][2 * k], v[m][e], b[0], b[1]);
                mma(S[m][2 * k + 1], v[m][e], b[2], b[3]);
              }
          }
      }
      const T* values = reinterpret_cast<const T*>(sm + stage * Sh::kStage + Sh::kV);
      stage = stage == Sh::kStages - 1 ? 0 : stage + 1;
      if (kStateOnly) {
        bar_arrive(kEmpty + turn, Sh::kAll);
      } else {
        bar_sync(kMultipliers, Sh::kMulThreads);          // the sums of the block below the triangles
        const float* A = reinterpret_cast<const float*>(set + Sh::kA) + g * 8 + q * 2;
        pair up = load2(A), dn = load2(A + 64);
#pragma unroll
        for (int x = 1; x < N / 64; ++x) { up = add2(up, load2(A + x * 128)); dn = add2(dn, load2(A + x * 128 + 64)); }
        pair mid = load2(reinterpret_cast<const float*>(sm + Sh::oMid) + g * 8 + q * 2);
#pragma unroll
        for (int x = 1; x < Sh::kMulThreads / 32; ++x) mid = add2(mid, load2(reinterpret_cast<const float*>(sm + Sh::oMid) + x * 64 + g * 8 + q * 2));
        if (__any_sync(0xFFFFFFFFu, (wild & 0x80008000u) != 0)) {
          // Above the diagonal A is zero, and zero times infinity or NaN is not: a token must not see what comes after it, so its sum stops at itself.
          const float* parts = reinterpret_cast<const float*>(set + Sh::kA);
          const float* mids = reinterpret_cast<const float*>(sm + Sh::oMid);
          for (int i2 = 0; i2 < 2; ++i2) {
            for (int s = 0; s <= g + 8 * i2; ++s) {
              float x = 0.f;
              if (s / 8 == i2) {
                for (int y = 0; y < N / 64; ++y) x += parts[y * 128 + i2 * 64 + g * 8 + s % 8];
              } else {
                for (int y = 0; y < Sh::kMulThreads / 32; ++y) x += mids[y * 64 + g * 8 + s];
              }
              const T* row = reinterpret_cast<const T*>(reinterpret_cast<const uint8_t*>(values) + s * Sh::kRawPitch) + warp * Sh::kValues * 16 + q * 2;
#pragma unroll
              for (int m = 0; m < Sh::kValues; ++m)
#pragma unroll
                for (int nb = 0; nb < 2; ++nb)
#pragma unroll
                  for (int e = 0; e < 2; ++e) {
                    const float y = fmaf(x, to_f32(row[m * 16 + nb * 8 + e]), i2 ? o[m][nb][2 + e] : o[m][nb][e]);
                    if (i2) o[m][nb][2 + e] = y;
                    else o[m][nb][e] = y;
                  }
            }
          }
          bar_arrive(kEmpty + turn, Sh::kAll);
        } else {
          bar_arrive(kEmpty + turn, Sh::kAll);
          uint32_t a0[Sh::R], a1[Sh::R], a3[Sh::R];
          split<Sh::R>(up, a0);
          split<Sh::R>(mid, a1);
          split<Sh::R>(dn, a3);
#pragma unroll
          for (int e = 0; e < Sh::R; ++e) {
            const uint32_t x[4] = {a0[e], a1[e], 0u, a3[e]};
#pragma unroll
            for (int f = 0; f < Sh::V && e + f < Sh::R; ++f)
#pragma unroll
              for (int m = 0; m < Sh::kValues; ++m) {
                mma(o[m][0], x, v[m][f][0], v[m][f][2]);
                mma(o[m][1], x, v[m][f][1], v[m][f][3]);
              }
          }
        }
        T* out = static_cast<T*>(a.out) + (long long)h * N + warp * Sh::kValues * 16 + q * 2;
#pragma unroll
        for (int i2 = 0; i2 < 2; ++i2) {
          const int row = t0 + g + 8 * i2;
          if (row < end) {
            T* at = out + row * a.out_row;
#pragma unroll
            for (int m = 0; m < Sh::kValues; ++m)
#pragma unroll
              for (int nb = 0; nb < 2; ++nb) {
                const float x = o[m][nb][2 * i2], y = o[m][nb][2 * i2 + 1];
                if constexpr (sizeof(T) == 4) *reinterpret_cast<float2*>(at + m * 16 + nb * 8) = make_float2(x, y);
                else {
                  const T two[2] = {from_f32<T>(x), from_f32<T>(y)};
                  *reinterpret_cast<uint32_t*>(at + m * 16 + nb * 8) = *reinterpret_cast<const uint32_t*>(two);
                }
              }
          }
        }
      }
    }
  }

  // States in the caller's layout [key][value].
  __device__ __forceinline__ void load_state(int slot) {
    const float* s = p.a.state && slot >= 0 ? p.a.state + ((size_t)slot * p.a.heads + h) * Sh::kStateFloats + warp * Sh::kValues * 16 + (lane >> 2) : nullptr;
#pragma unroll
    for (int m = 0; m < Sh::kValues; ++m)
#pragma unroll
      for (int j = 0; j < Sh::kTiles; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[m][j][e] = s ? __ldg(s + (j * 8 + (lane & 3) * 2 + (e & 1)) * N + m * 16 + (e >> 1) * 8) : 0.f;
  }
  __device__ __forceinline__ void clear_state() {
#pragma unroll
    for (int m = 0; m < Sh::kValues; ++m)
#pragma unroll
      for (int j = 0; j < Sh::kTiles; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[m][j][e] = 0.f;
  }
  __device__ __forceinline__ void store_state(int slot) {
    float* s = p.a.state_out + ((size_t)slot * p.a.heads + h) * Sh::kStateFloats + warp * Sh::kValues * 16 + (lane >> 2);
#pragma unroll
    for (int m = 0; m < Sh::kValues; ++m)
#pragma unroll
      for (int j = 0; j < Sh::kTiles; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[(j * 8 + (lane & 3) * 2 + (e & 1)) * N + m * 16 + (e >> 1) * 8] = S[m][j][e];
  }
  // States in the workspace: as the registers hold them.  which: 0 what the block's last piece comes to, 1 what its sequence began with, 2 the piece's decays.
  __device__ __forceinline__ float* block_state(int block, int which) const {
    return p.block_states + (size_t)block * Sh::kBlockFloats + which * Sh::kStateFloats;
  }
  __device__ __forceinline__ int kept_at(int m, int j) const { return ((warp * Sh::kValues + m) * Sh::kTiles + j) * 32 + lane; }
  __device__ __forceinline__ void keep(float* to) const {
#pragma unroll
    for (int m = 0; m < Sh::kValues; ++m)
#pragma unroll
      for (int j = 0; j < Sh::kTiles; ++j) reinterpret_cast<float4*>(to)[kept_at(m, j)] = make_float4(S[m][j][0], S[m][j][1], S[m][j][2], S[m][j][3]);
  }
  __device__ __forceinline__ void take(const float* from) {
#pragma unroll
    for (int m = 0; m < Sh::kValues; ++m)
#pragma unroll
      for (int j = 0; j < Sh::kTiles; ++j) {
        const float4 x = reinterpret_cast<const float4*>(from)[kept_at(m, j)];
        S[m][j][0] = x.x; S[m][j][1] = x.y; S[m][j][2] = x.z; S[m][j][3] = x.w;
      }
  }
  // A block's piece behind what is here.
  __device__ __forceinline__ void behind(const float* add, const float* decay) {
#pragma unroll
    for (int j = 0; j < Sh::kTiles; ++j) {
      const float2 d = *reinterpret_cast<const float2*>(decay + j * 8 + (lane & 3) * 2);
#pragma unroll
      for (int m = 0; m < Sh::kValues; ++m) {
        const float4 x = reinterpret_cast<const float4*>(add)[kept_at(m, j)];
        S[m][j][0] = fmaf(S[m][j][0], d.x, x.x); S[m][j][1] = fmaf(S[m][j][1], d.y, x.y);
        S[m][j][2] = fmaf(S[m][j][2], d.x, x.z); S[m][j][3] = fmaf(S[m][j][3], d.y, x.w);
      }
    }
  }
};

// A 64-bit division takes a hundred instructions, and few calls have as many rows.
__device__ __forceinline__ int quotient(long long a, long long b) { return ((a | b) >> 32) != 0 ? (int)(a / b) : (int)((uint32_t)a / (uint32_t)b); }

// The next sequence from `from` on that has rows in [row0, row1) and is longer than the limit; n_seq: none.  Called by whole warps.
__device__ __forceinline__ int next_sequence(const Args& p, int from, int row0, int row1) {
  constexpr int kAtOnce = 4;         // entries a lane has under way
  for (int base = from; base < p.a.n_seq; base += 32 * kAtOnce) {
    bool here[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int i = base + 32 * j + (int)(threadIdx.x & 31);
      const Entry e = i < p.a.n_seq ? p.entries[i] : Entry{0, 0, -1, 0};
      here[j] = e.end - e.start > p.limit && e.end > row0 && e.start < row1;
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const uint32_t found = __ballot_sync(0xFFFFFFFFu, here[j]);
      if (found) return base + 32 * j + __ffs((int)found) - 1;
    }
  }
  return p.a.n_seq;
}

constexpr int kPerSm = 2, kStatesPerSm = 3;      // thread blocks an SM holds; three of the outputs' pass spill (71 -> 74 us, 9.8 -> 11.1 of 203 tokens)
template <typename T, int N, int kDecay, bool kStateOnly>
__global__ void __launch_bounds__(Shape<T, N, kStateOnly>::kAll, N == 64 ? (kStateOnly ? kStatesPerSm : kPerSm) : 1) linattn_chunk_kernel(const __grid_constant__ Args p) {
  using Sh = Shape<T, N, kStateOnly>;
  extern __shared__ __align__(128) uint8_t smem[];
  Worker<T, N, kDecay, kStateOnly> w(p, smem);
  const bool maker = threadIdx.x < Sh::kThreads;
  const int block = blockIdx.x, tokens = p.a.tokens;
  const long long f0 = block * p.block_rows, f1 = min(f0 + p.block_rows, p.a.heads * p.pitch);
  if (kStateOnly) {
    // the blocks' pass may begin as soon as there is room for it: it waits for this one where it needs the states
    asm volatile("griddepcontrol.launch_dependents;");
  } else {
    // above the diagonals it stays zero
    for (int i = (int)threadIdx.x; i < 2 * (Sh::kTriangles / 4); i += Sh::kAll)
      reinterpret_cast<float*>(smem + Sh::oSets + Sh::kA + (i < Sh::kTriangles / 4 ? 0 : Sh::kSet - Sh::kTriangles))[i] = 0.f;
    __syncthreads();
  }
  // A block's head, or heads; of the states' pass the last one only, and of that the sequence that goes on behind the block.
  for (w.h = quotient(kStateOnly ? f1 - 1 : f0, p.pitch); w.h * p.pitch < f1; ++w.h) {
    const long long head0 = w.h * p.pitch;
    const int row0 = (int)max(f0 - head0, 0ll), row1 = (int)min(f1 - head0, (long long)tokens);
    for (int seq = 0;; ++seq) {
      Entry e = {0, tokens, 0, 0};
      if (p.entries) {
        seq = next_sequence(p, seq, row0, row1);
        if (seq >= p.a.n_seq) break;
        e = p.entries[seq];
      } else if (seq > 0) {
        break;
      }
      const int begin = max(e.start, row0), end = min(e.end, row1);
      if (kStateOnly) {
        if (e.end <= row1) continue;
        if (maker) {
          w.total = pair_of(0.f, 0.f);
          w.make(begin, end);
          w.made();
          if ((w.warp & 3) == 3) {
            const float2 f = both(w.total);
            *reinterpret_cast<float2*>(w.block_state(block, 2) + (w.warp >> 2) * 64 + w.lane * 2) = make_float2(expf(f.x), expf(f.y));
          }
          return;
        }
        if (e.start >= row0) {
          w.load_state(e.slot);
          w.keep(w.block_state(block, 1));       // for the pass that follows: by then the last of its blocks may have written the new state over it
        } else {
          w.clear_state();
        }
        w.multiply(begin, end);
        w.keep(w.block_state(block, 0));
        return;
      }
      if (maker) {
        w.make(begin, end);
        continue;
      }
      if (e.start < row0 || e.end > row1) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        // from the workspace: what the sequence began with, or what the blocks before this one make of it
        const int b0 = e.start >= row0 ? block : quotient(head0 + e.start, p.block_rows);
        w.take(w.block_state(b0, e.start >= row0 ? 1 : 0));
        for (int b = b0 + 1; b < block; ++b) w.behind(w.block_state(b, 0), w.block_state(b, 2));
      } else {
        w.load_state(e.slot);
      }
      w.multiply(begin, end);
      if (e.end <= row1 && p.a.state_out && e.slot >= 0) {
        asm volatile("griddepcontrol.wait;" ::: "memory");      // it may be written where the pass before read it
        w.store_state(e.slot);
      }
    }
  }
  if (!kStateOnly && maker) w.made();
  if (!kStateOnly) asm volatile("griddepcontrol.wait;" ::: "memory");      // a block without rows does not end before the pass in front of it, either
}

// Rows of a block and how many blocks.  A block's warps work on one head at a time; an SM holds kPerSm thread blocks of the outputs' pass with heads of 64, one with heads of 128.
struct Plan { long long block_rows, pitch; int blocks, limit; size_t entries_bytes, bytes; };
constexpr int kShortest = 8, kLeastChunks = 3, kFewMore = 16;
Plan plan_of(int tokens, int n_seq, int heads, int n) {
  Plan l = {0, 0, 0, 0x7FFFFFFF, 0, 0};
  const int sms = sm_count(), per_sm = n == 64 ? kPerSm : 1;
  const long long all = (long long)heads * tokens, most = (long long)sms * per_sm;
  if (tokens <= kShortest) return l;
  // as much as fewer tokens or sequences could ask for
  l.entries_bytes = round_up_sz((size_t)n_seq * sizeof(Entry), 256);
  l.bytes = l.entries_bytes + (size_t)std::min(most, all / (2 * kChunk) + 1) * (2 * n * n + n) * 4;
  // The lengths are on the device.  With at most two rows a sequence on average, and fewer than kFewMore more than sequences, all are taken for short ones: a batch of single tokens does not pay for launches that find
  // nothing (96 sequences of two tokens, 64 heads, 37.8 us without them, 41.0 with), and a sequence of 16 among single tokens is as fast by the recurrence.  Longer ones are not (one
  // among 95 single tokens: of 32 rows 52 us by the recurrence, 40.5 in chunks, of 96 rows 106 and 47; 299 rows among 300 tokens 370 and 129).  An empty sequence hides a row.
  if (tokens <= 2ll * n_seq && tokens < (long long)n_seq + kFewMore) return l;
  // An SM has kPerSm blocks at work, a chunk of 16 rows every so often (0.95 us with two or three, 1.05 alone: measured with bf16 and heads of 64, and taken for all; 1111 rows
  // of 16 heads of 128 in fp32 it takes for 18 us where they are 57); a sequence's last block adds up the states of
  // those before it.  Blocks of one head each, or, where that leaves SMs idle, the heads' rows cut evenly: some blocks then begin anew at a second head (2048 rows of
  // 64 heads: six blocks each 77.8 us, even 74.4; 203 of 32 heads: four each 11.1, even 16.5).
  auto chunk_time = [&](long long blocks) { return std::max(0.95 * (double)((blocks + sms - 1) / sms), 1.05); };
  double best = 0.0;
  for (int b = 1; b == 1 || ((long long)b * heads <= most && b <= 64); ++b) {
    const long long rows = ((long long)tokens + b - 1) / b, chunks = (rows + kChunk - 1) / kChunk;
    if (b > 1 && chunks < kLeastChunks) break;
    const double t = (double)chunks * chunk_time((long long)b * heads) + 0.4 * (b - 1) + (b > 1 ? 3.0 + 0.45 * (double)chunks * (b - 1) / b : 0.0);
    if (b == 1 || t < best) { best = t; l.block_rows = chunks * kChunk; l.pitch = b * l.block_rows; l.blocks = b * heads; }
  }
  const long long even = std::max<long long>(kLeastChunks * kChunk, ((all + most - 1) / most + kChunk - 1) / kChunk * kChunk), blocks = (all + even - 1) / even;
  const double t = (double)(even / kChunk + 1) * (chunk_time(blocks) + 0.45) + 0.4 * (double)(tokens / even) + 6.0;
  if (t < best) { l.block_rows = even; l.pitch = tokens; l.blocks = (int)blocks; }
  l.limit = kShortest;
  return l;
}

template <typename T, int N, int kDecay>
cudaError_t launch_chunks(const Args& p, const Plan& l, cudaStream_t s) {
  using All = Shape<T, N, false>;
  using States = Shape<T, N, true>;
  static SmemOptIn opt_state(kCarveOut), opt_all(kCarveOut);
  cudaError_t e = opt_all((const void*)linattn_chunk_kernel<T, N, kDecay, false>, All::kBytes);
  const bool two_passes = l.pitch != l.block_rows;         // else every block is a whole head
  if (e == cudaSuccess && two_passes) {
    e = opt_state((const void*)linattn_chunk_kernel<T, N, kDecay, true>, States::kBytes);
    if (e == cudaSuccess) {
      linattn_chunk_kernel<T, N, kDecay, true><<<(unsigned)l.blocks - 1, States::kAll, States::kBytes, s>>>(p);
      e = cudaGetLastError();
    }
  }
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)l.blocks); cfg.blockDim = dim3(All::kAll); cfg.dynamicSmemBytes = All::kBytes; cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = two_passes ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, linattn_chunk_kernel<T, N, kDecay, false>, p);
}
template <typename T, int N>
cudaError_t launch_n(const Args& p, const Plan& l, cudaStream_t s) {
  if (l.blocks == 0 || p.entries) {
    linattn_token_kernel<T, N><<<dim3((unsigned)p.a.heads, (unsigned)p.a.n_seq, N / kCols), kTokenThreads, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || l.blocks == 0) return e;
  }
  if (p.a.decay_per_head) return launch_chunks<T, N, DECAY_HEAD>(p, l, s);
  if (sizeof(T) == 4 || p.a.decay_dtype == RWKVQ_F32) return launch_chunks<T, N, DECAY_F32>(p, l, s);
  return launch_chunks<T, N, sizeof(T) == 4 ? DECAY_F32 : DECAY_SAME>(p, l, s);
}
template <typename T>
cudaError_t launch(const Args& p, const Plan& l, cudaStream_t s) {
  return p.a.n == 64 ? launch_n<T, 64>(p, l, s) : launch_n<T, 128>(p, l, s);
}

}  // namespace la
}  // namespace rwkvq

using namespace rwkvq;

extern "C" {

size_t rwkvq_linattn_workspace_bytes(int tokens, int n_seq, int heads, int n) {
  if (tokens < 0 || n_seq <= 0 || heads <= 0 || (n != 64 && n != 128)) return 0;
  return la::plan_of(tokens, n_seq, heads, n).bytes;
}

rwkvq_status rwkvq_linattn(const rwkvq_linattn_args* args, void* workspace, size_t workspace_bytes, void* stream) {
  if (!args) return RWKVQ_EINVAL;
  la::Args p;
  p.a = *args;
  rwkvq_linattn_args& a = p.a;
  const int es = a.dtype == RWKVQ_F32 ? 4 : a.dtype == RWKVQ_F16 || a.dtype == RWKVQ_BF16 ? 2 : 0;
  if (es == 0 || (a.decay_dtype != RWKVQ_F32 && a.decay_dtype != a.dtype)) return RWKVQ_EINVAL;
  if (a.tokens < 0 || a.n_seq <= 0 || a.heads <= 0 || a.n <= 0 || a.n_slots < 0) return RWKVQ_EINVAL;
  if (a.n != 64 && a.n != 128) return RWKVQ_EUNSUPPORTED;
  if (a.n_seq > 65535 || a.heads > 65535 || a.tokens > (1 << 30)) return RWKVQ_EUNSUPPORTED;
  if (a.tokens > 0 && (!a.r || !a.k || !a.v || !a.logw || !a.out)) return RWKVQ_EINVAL;
  if (a.tokens > 0 && (a.out == a.r || a.out == a.k || a.out == a.v || a.out == a.logw)) return RWKVQ_EINVAL;
  if (!a.seq_start && a.n_seq != 1) return RWKVQ_EINVAL;
  const bool keeps = a.state || a.state_out;
  if (a.slots && !keeps) return RWKVQ_EINVAL;
  if (keeps && a.n_slots < (a.slots ? 1 : a.n_seq)) return RWKVQ_EINVAL;
  const long long d = (long long)a.heads * a.n, dw = a.decay_per_head ? a.heads : d;
  if (a.tokens > 1 && (a.r_row < d || a.k_row < d || a.v_row < d || a.out_row < d || (a.logw_row != 0 && a.logw_row < dw))) return RWKVQ_EINVAL;
  const int ws = a.decay_dtype == RWKVQ_F32 ? 4 : es;
  if (!aligned16(a.r) || !aligned16(a.k) || !aligned16(a.v) || !aligned16(a.logw) || !aligned16(a.out) || !aligned16(a.u) || !aligned16(a.state) ||
      !aligned16(a.state_out))
    return RWKVQ_EALIGN;
  if (a.tokens > 1 && ((a.r_row * es) % 16 || (a.k_row * es) % 16 || (a.v_row * es) % 16 || (a.out_row * es) % 16 || (!a.decay_per_head && (a.logw_row * ws) % 16)))
    return RWKVQ_EALIGN;
  if (a.state && a.state_out && a.state != a.state_out) {        // the very same states, or others
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.state), y = reinterpret_cast<uintptr_t>(a.state_out);
    const size_t bytes = (size_t)a.n_slots * a.heads * a.n * a.n * 4;
    if (x < y + bytes && y < x + bytes) return RWKVQ_EINVAL;
  }
  const la::Plan l = la::plan_of(a.tokens, a.n_seq, a.heads, a.n);
  if (l.blocks > 0 && (!workspace || workspace_bytes < l.bytes)) return RWKVQ_ENOMEM;
  if (!aligned16(workspace)) return RWKVQ_EALIGN;
  p.limit = l.limit; p.block_rows = l.block_rows; p.pitch = l.pitch;
  p.entries = l.blocks > 0 && (a.seq_start || a.slots) ? static_cast<la::Entry*>(workspace) : nullptr;
  p.block_states = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + l.entries_bytes);
  p.status = device_status_ptr();
  if (!p.status) return RWKVQ_ECUDA;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.dtype == RWKVQ_F32) return cuda_status(la::launch<float>(p, l, s));
  if (a.dtype == RWKVQ_F16) return cuda_status(la::launch<__half>(p, l, s));
  return cuda_status(la::launch<__nv_bfloat16>(p, l, s));
}

}  // extern "C"
