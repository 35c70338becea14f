// Linear attention with decaying state: per sequence and head, with S [N keys][N values] in fp32,
//   out_t = r_t (S + (u (.) k_t) v_t^T),   S <- diag(exp(lw_t)) S + k_t v_t^T.
//
// Single tokens and short sequences: linattn_token_kernel, the recurrence as it stands, S in registers.  One token reads and writes 2 * 4 * N * N bytes of
// state for 4 N^2 operations: HBM, and with few sequences latency, is all that counts.
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

struct Args {
  rwkvq_linattn_args a;
  int* status;
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
  return start >= 0 && start <= end && end <= p.a.tokens;
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
  bool bad = !rows_of(p, seq, start, end);
  if (a.slots) {
    slot = a.slots[seq];
    bad = bad || slot < -1 || slot >= a.n_slots;
    for (int j = tid; j < seq; j += kTokenThreads) bad = bad || (slot >= 0 && a.slots[j] == slot);      // a state belongs to one sequence of a call
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) atomicExch(p.status, (int)RWKVQ_EINVAL);
    return;
  }
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

template <typename T>
cudaError_t launch(const Args& p, cudaStream_t s) {
  const dim3 grid((unsigned)p.a.heads, (unsigned)p.a.n_seq, (unsigned)(p.a.n / kCols));
  if (p.a.n == 64) linattn_token_kernel<T, 64><<<grid, kTokenThreads, 0, s>>>(p);
  else linattn_token_kernel<T, 128><<<grid, kTokenThreads, 0, s>>>(p);
  return cudaGetLastError();
}

}  // namespace la
}  // namespace rwkvq

using namespace rwkvq;

extern "C" {

size_t rwkvq_linattn_workspace_bytes(int tokens, int n_seq, int heads, int n) {
  (void)tokens; (void)n_seq; (void)heads; (void)n;
  return 0;
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
  if (a.n_seq > 65535 || (long long)a.heads * a.n > (1ll << 24)) return RWKVQ_EUNSUPPORTED;
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
  (void)workspace; (void)workspace_bytes;
  p.status = device_status_ptr();
  if (!p.status) return RWKVQ_ECUDA;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.dtype == RWKVQ_F32) return cuda_status(la::launch<float>(p, s));
  if (a.dtype == RWKVQ_F16) return cuda_status(la::launch<__half>(p, s));
  return cuda_status(la::launch<__nv_bfloat16>(p, s));
}

}  // extern "C"
