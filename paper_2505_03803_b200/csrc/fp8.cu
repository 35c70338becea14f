// Eight-bit floating point (e4m3) with one power-of-two scale per block of 128 columns: the quantizer and the product.
//
// Scale of a group (128 columns of one row for activations, of 128 rows for weights): the smallest 2^e with max|x| <= 448 * 2^e (448 = 1.75 * 2^8 is
// the largest e4m3 number).  A power of two, so that scaling rounds nothing: a code is x * 2^-e rounded once, and a product of two
// scales is exact.  It is stored as the eight-bit exponent e + 127, the form that the block-scaled tensor-core instruction applies itself, which
// leaves no scaling to the CUDA cores.  (Scales of 32 bits would use up to twice the range of the format, which buys a floating-point
// code nothing but its few subnormals, and cost a pass of every partial sum of 128 columns through registers.)
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "../../include/rwkvq.h"
#include "host_util.h"
#include "tc5.cuh"

namespace rwkvq {

int* device_status_ptr();  // api_misc.cu

namespace f8 {

using namespace tc5;

// ---- quantizer --------------------------------------------------------------------------------------------
__device__ __forceinline__ float2 unpack2(uint32_t v, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
__device__ __forceinline__ float2 unpack2(uint32_t v, __nv_bfloat16) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v)); }
// Eight elements as they lie in memory: between the maximum and the codes they wait in as few registers as that takes.
template <typename T>
struct Eight {
  static constexpr int kWords = sizeof(T) * 2;
  uint32_t w[kWords];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) {
      const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p) + i);
      w[4 * i] = a.x; w[4 * i + 1] = a.y; w[4 * i + 2] = a.z; w[4 * i + 3] = a.w;
    }
  }
  // The compiler is to forget what it has made of the words: kept for a second use, that takes twice the registers.
  __device__ __forceinline__ void forget() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) asm volatile("" : "+r"(w[i]));
  }
  __device__ __forceinline__ void floats(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) { f[2 * i] = __uint_as_float(w[2 * i]); f[2 * i + 1] = __uint_as_float(w[2 * i + 1]); }
      else { const float2 v = unpack2(w[i], T()); f[2 * i] = v.x; f[2 * i + 1] = v.y; }
    }
  }
};
constexpr uint32_t kInfBits = 0x7F800000u;
// Bits of the largest magnitude (as unsigned integers they sort like the numbers); NaN does not count.  kFinite: infinities do not, either, which takes
// four times the instructions and is asked for only where the first answer is infinity.
template <bool kFinite, typename T>
__device__ __forceinline__ uint32_t amax8(const Eight<T>& x) {
  float f[8], a = 0.f;
  x.floats(f);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float m = fabsf(f[i]);
    a = fmaxf(a, !kFinite || __float_as_uint(m) < kInfBits ? m : 0.f);
  }
  return __float_as_uint(a);
}
// The scale's exponent + 127 from those bits: x = m * 2^(E - 127) with m <= 1.75 fits 448 * 2^(E - 127 - 8), a larger m needs one more.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  if (amax == 0u) return 127u;
  const int e = (int)(amax >> 23) - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(e, 1);
}
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }     // 1 <= byte <= 247
// kFinite: there may be infinities, which become NaN codes (the conversion alone would saturate them).
template <bool kFinite, typename T>
__device__ __forceinline__ uint2 encode8(const Eight<T>& e, float inv) {
  float f[8];
  e.floats(f);
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float v[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float x = f[2 * i + j];
      v[j] = !kFinite || (__float_as_uint(x) & 0x7FFFFFFFu) < kInfBits ? x * inv : __uint_as_float(0x7FFFFFFFu);
    }
    uint16_t c;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(v[1]), "f"(v[0]));
    h[i] = c;
  }
  return make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
}

// Rows: a warp takes 256 columns per 16-byte load (16 lanes a group), four loads under way, and writes the eight scales together.  HBM: 8192 x 7168 bf16 in 33.4 us
// (5.3 TB/s), 2048 x 4096 in 6.7, of which HBM needs 3.9.
constexpr int kRowWarps = 8, kRowChunks = 4, kRowCols = kRowChunks * 256;
template <typename T>
__global__ void __launch_bounds__(kRowWarps * 32) fp8_rows_kernel(const T* x, long long x_row, int rows, int cols, int pieces, uint8_t* codes,
                                                                 uint8_t* scale, int pitch) {
  const long long unit = (long long)blockIdx.x * kRowWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  const long long row = unit / pieces;
  if (row >= rows) { asm volatile("griddepcontrol.wait;" ::: "memory"); return; }
  const int c0 = (int)(unit % pieces) * kRowCols + lane * 8;
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  Eight<T> f[kRowChunks];
#pragma unroll
  for (int j = 0; j < kRowChunks; ++j) {
    if (c0 + j * 256 < cols) f[j].load(x + row * x_row + c0 + j * 256);
    else f[j].zero();
  }
  uint32_t m[kRowChunks], most = 0;
#pragma unroll
  for (int j = 0; j < kRowChunks; ++j) { m[j] = amax8<false>(f[j]); most = max(most, m[j]); }
  const bool infinite = __any_sync(0xFFFFFFFFu, most >= kInfBits);
  if (infinite) {
#pragma unroll
    for (int j = 0; j < kRowChunks; ++j) m[j] = amax8<true>(f[j]);
  }
  uint32_t lo = 0, hi = 0;
#pragma unroll
  for (int j = 0; j < kRowChunks; ++j) {
    uint32_t a = m[j];
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, d));
    const uint32_t b = scale_byte(a);
    const uint32_t two = b | __shfl_down_sync(0xFFFFFFFFu, b, 16) << 8;
    if (j < 2) lo |= two << (16 * j);
    else hi |= two << (16 * (j - 2));
    if (c0 + j * 256 < cols)
      *reinterpret_cast<uint2*>(codes + row * cols + c0 + j * 256) = infinite ? encode8<true>(f[j], inverse_scale(b)) : encode8<false>(f[j], inverse_scale(b));
  }
  // the pitch is a multiple of 16, and a piece of columns begins inside it
  if (lane == 0) *reinterpret_cast<uint2*>(scale + row * pitch + (c0 >> 7)) = make_uint2(lo, hi);
}

// Blocks of 128 x 128: one thread block each, its elements in registers between the maximum and the codes.  HBM: 14336 x 4096 in 33.0 us from fp16 (5.3 TB/s), 44.6 from
// fp32 (6.6 TB/s); 47 with the codes' checks for infinities on every element and 256 threads.
constexpr int kBlockThreads = 512;
template <typename T>
__global__ void __launch_bounds__(kBlockThreads, 2) fp8_blocks_kernel(const T* x, long long x_row, int rows, int cols, int groups, uint8_t* codes,
                                                                  uint8_t* scale, int pitch) {
  __shared__ uint32_t most[kBlockThreads / 32];
  const int g = (int)(blockIdx.x % (unsigned)groups), rb = (int)(blockIdx.x / (unsigned)groups);
  const int c = g * 128 + (threadIdx.x & 15) * 8;
  const long long r0 = (long long)rb * 128 + (threadIdx.x >> 4);
  constexpr int kStepRows = kBlockThreads / 16, kSteps = 128 / kStepRows;
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int left = c < cols ? (int)min(rows - r0, (long long)128) : 0;       // rows of this thread's that are there: every kStepRows-th of so many
  Eight<T> f[kSteps];
  uint32_t a = 0;
  const T* from = x + r0 * x_row + c;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    if (i * kStepRows < left) f[i].load(from);
    else f[i].zero();
    from += kStepRows * x_row;
  }
  auto whole = [&](uint32_t v) {
    v = __reduce_max_sync(0xFFFFFFFFu, v);
    if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = v;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kBlockThreads / 32; ++i) v = max(v, most[i]);
    return v;
  };
#pragma unroll
  for (int i = 0; i < kSteps; ++i) { a = max(a, amax8<false>(f[i])); f[i].forget(); }
  a = whole(a);
  const bool infinite = a >= kInfBits;       // the same in all threads
  if (infinite) {
    a = 0;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) a = max(a, amax8<true>(f[i]));
    __syncthreads();
    a = whole(a);
  }
  const uint32_t b = scale_byte(a);
  const float inv = inverse_scale(b);
  uint8_t* to = codes + r0 * cols + c;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    if (i * kStepRows < left) *reinterpret_cast<uint2*>(to) = infinite ? encode8<true>(f[i], inv) : encode8<false>(f[i], inv);
    to += (size_t)kStepRows * cols;
  }
  if (threadIdx.x == 0) scale[(size_t)rb * pitch + g] = (uint8_t)b;
}

int blocks_of(int n) { return n / 128 + (n % 128 != 0); }
size_t scale_pitch(int cols) { return round_up_sz((size_t)blocks_of(cols), 16); }

// All launches here may begin while the kernel before them ends; the kernels wait for that end before they touch memory.
cudaLaunchConfig_t launch_config(dim3 grid, int threads, uint32_t smem, cudaStream_t s, cudaLaunchAttribute (&attr)[2]) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = dim3((unsigned)threads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cfg;
}

template <typename T>
cudaError_t quantize(const void* x, long long x_row, int rows, int cols, int block_rows, void* codes, void* scale, int pitch, cudaStream_t s) {
  cudaLaunchAttribute attr[2];
  if (block_rows == 1) {
    const int pieces = cols / kRowCols + (cols % kRowCols != 0);
    const long long blocks = ((long long)rows * pieces + kRowWarps - 1) / kRowWarps;
    const cudaLaunchConfig_t cfg = launch_config(dim3((unsigned)blocks), kRowWarps * 32, 0, s, attr);
    return cudaLaunchKernelEx(&cfg, fp8_rows_kernel<T>, static_cast<const T*>(x), x_row, rows, cols, pieces, static_cast<uint8_t*>(codes),
                              static_cast<uint8_t*>(scale), pitch);
  }
  const int groups = blocks_of(cols);
  const long long blocks = (long long)blocks_of(rows) * groups;
  const cudaLaunchConfig_t cfg = launch_config(dim3((unsigned)blocks), kBlockThreads, 0, s, attr);
  return cudaLaunchKernelEx(&cfg, fp8_blocks_kernel<T>, static_cast<const T*>(x), x_row, rows, cols, groups, static_cast<uint8_t*>(codes),
                            static_cast<uint8_t*>(scale), pitch);
}

// ---- product ----------------------------------------------------------------------------------------------
// Y[t][i] = sum_g 2^(ex[t][g] + ew[i / 128][g]) sum_{k in group g} x[t][k] w[i][k].  Weights are the 128-row operand (a tile's rows are
// one block of scales), tokens the other one, NT of them, so that a lane of an accumulator is an output channel and a warp writes 32
// consecutive outputs of one token.  Roles of a CTA's warps: (0) tensor-map copies of 128-column stages, (1) tensor-core
// instructions, (2) scales, (3) tensor memory, (4 on) epilogue.  Two accumulators: for a tile's epilogue to run under the next tile's sums, or (W = 2) for two tiles of
// weights with the same tokens.
// Scales: four groups' bytes of a row are the word that the instruction picks its byte from; warp 2 deals the words of 512 columns out in the order
// of the copy to tensor memory (32 lanes x 16 bytes, row r in line r % 32, word r / 32), where they lie once per 32-lane quarter.
//
// What bounds it.  One token: launch, the latency of the first loads and of the slices' meeting (4096 x 4096 6.5 us with weights from HBM, which needs 2.6).  Few tokens,
// large matrices: HBM (65536 x 4096, 16 tokens, 43.2 us = 6.3 TB/s).  Many: power.  2048 x 4096 x 14336 over and over takes 105 to 110 us (2.2 PFLOP/s) at 990 W, the limit,
// which leaves 1.47 of 1.97 GHz; 106 without scales, 125 with one tile of weights a block.  A stage of two brings 63 KB for 256 x 240 outputs, of one 47 KB for 128 x 240,
// and shared memory, which these pass twice (in, and to the tensor core), is then busier than the tensor core.
// Taken back: pairs of blocks (cta_group::2) that share a tile's tokens, which take in as little (2048 x 14336 x 4096 111 us with barriers of the other block's, 263 with
// relayed ones); 2 KB of epilogue buffers and a stage more (no gain); two blocks an SM for few tokens (7.5 us where one with more stages takes 7.3, 4096 x 4096); the
// scales' words 16 bytes at a time (65536 x 1024, 240 tokens, 24.3 -> 28.9); elections for every instruction of warp 1 (1000 x 4096 x 1024 9.6 us, one for all 8.8).
constexpr int kRows = 128, kStageCols = 128, kMaxTokens = 240, kMaxStages = 12, kSfSlots = 2, kMaxSlices = 8;
constexpr uint32_t kWBytes = kRows * kStageCols, kLineBytes = 512, kSfCols = 16, kOutBytes = 4096, kCtrlBytes = 512;
constexpr uint32_t kMaxSmemBytes = 232448;
// By the weights' tiles W (1 or 2) of a block's tile: their scales' lines and the tokens'; four warps of the epilogue for each.
__host__ __device__ constexpr int threads_of(int W) { return 128 + 128 * W; }
__host__ __device__ constexpr uint32_t sf_bytes(int W) { return kLineBytes * (uint32_t)(W + 2); }

struct GemmArgs {
  CUtensorMap wmap, xmap;
  const uint8_t* w_scale;
  const uint8_t* x_scale;
  void* Y;
  long long y_row;
  int oc, M, groups, pitch, NT, MT, tiles, stages, slices, y_dtype, wide;
  uint32_t tmem_cols;
  int* status;
  // For a test (rwkvq_gemm_fp8_lost), kernels of their own: the limit of a wait in polls, how many words of scales a block announces, where blocks that give up are counted.
  uint32_t poll_limit;
  int announced;
  int* lost;
};

struct Ctrl {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t sffull[kSfSlots], sfempty[kSfSlots];
  uint64_t accfull[2], accempty[2], drained;
  uint32_t tmem_base;
  int abort_flag, asked;        // asked: copies of stages
};
static_assert(sizeof(Ctrl) <= kCtrlBytes, "control block");

// Shared-memory descriptor of 32 lines of 16 bytes without a swizzle: eight lines are 128 bytes.
__device__ __forceinline__ uint64_t smem_desc_lines(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(128u >> 4) << 32 | (uint64_t)1 << 46;
}
// e4m3 x e4m3 -> fp32 with eight-bit exponents as scales, one per 32 columns, both operands K-major; `id`: the byte of the scale words.
__device__ __forceinline__ uint32_t idesc_mx(int M, int N, uint32_t id) {
  return id << 4 | (uint32_t)(N >> 3) << 17 | 1u << 23 | (uint32_t)(M >> 7) << 27 | id << 29;
}
// The four that follow are for one thread: an election for each of them would take longer than the small tiles' instructions.
__device__ __forceinline__ bool elected() {
  uint32_t q;
  asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(q));
  return q != 0;
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 lines of scales to four columns of tensor memory, once per quarter of the lanes.
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
// One stage: four instructions of 32 columns.
__device__ __forceinline__ void mma_stage(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, one;\n .reg .b64 a1, a2, a3, b1, b2, b3;\n"
      " setp.ne.b32 p, %6, 0;\n setp.eq.b32 one, 0, 0;\n"
      " add.u64 a1, %1, 2;\n add.u64 a2, %1, 4;\n add.u64 a3, %1, 6;\n add.u64 b1, %2, 2;\n add.u64 b2, %2, 4;\n add.u64 b3, %2, 6;\n"
      " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n"
      " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a1, b1, %3, [%4], [%5], one;\n"
      " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a2, b2, %3, [%4], [%5], one;\n"
      " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a3, b3, %3, [%4], [%5], one;\n}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}

template <typename T> __device__ __forceinline__ T to_out(float f);
template <> __device__ __forceinline__ float to_out<float>(float f) { return f; }
template <> __device__ __forceinline__ __half to_out<__half>(float f) { return __float2half_rn(f); }
template <> __device__ __forceinline__ __nv_bfloat16 to_out<__nv_bfloat16>(float f) { return __float2bfloat16_rn(f); }

// Two numbers rounded, the first in the low half.
__device__ __forceinline__ uint32_t two_of(uint32_t x, uint32_t y, __half) {
  const __half2 v = __floats2half2_rn(__uint_as_float(x), __uint_as_float(y));
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t two_of(uint32_t x, uint32_t y, __nv_bfloat16) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(x), __uint_as_float(y));
  return *reinterpret_cast<const uint32_t*>(&v);
}

// 32 lanes x 32 columns in the tiles of stmatrix: register 16 h + 4 n + 2 x + e of lane l = D[lane base + 16 h + 8 x + l / 4][col + 8 n + 2 (l % 4) + e].
__device__ __forceinline__ void tmem_ld_tiles_issue(uint32_t taddr, uint32_t (&r)[32]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[16 * h]), "=r"(r[16 * h + 1]), "=r"(r[16 * h + 2]), "=r"(r[16 * h + 3]), "=r"(r[16 * h + 4]), "=r"(r[16 * h + 5]), "=r"(r[16 * h + 6]),
                   "=r"(r[16 * h + 7]), "=r"(r[16 * h + 8]), "=r"(r[16 * h + 9]), "=r"(r[16 * h + 10]), "=r"(r[16 * h + 11]), "=r"(r[16 * h + 12]),
                   "=r"(r[16 * h + 13]), "=r"(r[16 * h + 14]), "=r"(r[16 * h + 15])
                 : "r"(taddr + ((uint32_t)h << 20)) : "memory");
}
// A warp's 32 output channels of a tile's tokens; `done` is arrived at when they are read.  A lane of the accumulator is a channel, and 16 bytes of Y are eight channels
// of one token: the way there is through shared memory (`stage`, 4 KB of the warp's own), for 16-bit types by stmatrix, which turns 8 x 8 numbers round at
// once (2048 x 14336 x 4096, one tile of weights a block: 110.5 us, 112.6 with a store of two bytes for each number).  The 64 bytes of a token lie in an order of 16-byte pieces that spares banks.
// Without a.wide (rows of Y begin on 16 bytes), or with fewer channels, a store for each number.
// The last 32 kHeld tokens are read before the first of them is stored: where the next tile's sums wait for `done`, the stores go on under them (three: 8192 x 7168 x 2048 124 ->
// 119 us, 2048 x 14336 x 4096 117.5 -> 115.3; five spill).
template <typename T, int kHeld>
__device__ __forceinline__ void store_tile(const GemmArgs& a, uint32_t tmem, int row0, int t0, int nt, uint8_t* stage, int lane, uint64_t* done) {
  T* y = static_cast<T*>(a.Y) + (long long)t0 * a.y_row + row0;
  const bool wide = a.wide && row0 + 32 <= a.oc;
  auto is_read = [&]() { tc_fence_before(); mbar_arrive(done); };
  uint32_t r[32];
  if constexpr (sizeof(T) == 2) {
    if (wide) {
      const uint32_t to = smem_u32(stage) + (uint32_t)((lane & 7) * 64 + ((lane >> 3 ^ lane >> 1) & 3) * 16);
      const uint8_t* from = stage + (lane >> 2) * 64 + ((lane ^ lane >> 3) & 3) * 16;
      T* at = y + (long long)(lane >> 2) * a.y_row + (lane & 3) * 8;
      auto pack = [&](uint32_t (&v)[16]) {
        tmem_ld_wait(r);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = two_of(r[2 * i], r[2 * i + 1], T());       // 8 h + 2 n + x
      };
      auto store = [&](int c, const uint32_t (&v)[16]) {
        const uint32_t half = (uint32_t)(c & 32) * 64u;        // in turn, so that no lane writes where another still reads
#pragma unroll
        for (int n = 0; n < 4; ++n)
          asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(to + half + n * 512), "r"(v[2 * n]), "r"(v[2 * n + 1]), "r"(v[8 + 2 * n]),
                       "r"(v[9 + 2 * n]) : "memory");
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 x = *reinterpret_cast<const uint4*>(from + half + i * 512);
          if (c + i * 8 + (lane >> 2) < nt) *reinterpret_cast<uint4*>(at) = x;
          at += 8 * a.y_row;
        }
      };
      uint32_t v[kHeld][16];
      int c = 0;
      tmem_ld_tiles_issue(tmem, r);
      for (; nt - c > 32 * kHeld; c += 32) {
        pack(v[0]);
        tmem_ld_tiles_issue(tmem + (uint32_t)c + 32u, r);
        store(c, v[0]);
      }
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (c + 32 * i < nt) {
          pack(v[i]);
          if (c + 32 * i + 32 < nt) tmem_ld_tiles_issue(tmem + (uint32_t)(c + 32 * i) + 32u, r);
        }
      is_read();
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (c + 32 * i < nt) store(c + 32 * i, v[i]);
      return;
    }
  }
  for (int c = 0; c < nt; c += 32) {
    tmem_ld32_issue(tmem + (uint32_t)c, r);
    tmem_ld_wait(r);
    if (c + 32 >= nt) is_read();
    if (sizeof(T) == 4 && wide) {
      uint32_t* st = reinterpret_cast<uint32_t*>(stage) + lane;
#pragma unroll
      for (int j = 0; j < 32; ++j) st[j * 32] = r[j];
      __syncwarp();
      T* at = y + (long long)(c + (lane >> 3)) * a.y_row + (lane & 7) * 4;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint4 v = *reinterpret_cast<const uint4*>(stage + i * 512 + lane * 16);
        if (c + i * 4 + (lane >> 3) < nt) *reinterpret_cast<uint4*>(at) = v;
        at += 4 * a.y_row;
      }
      __syncwarp();
    } else if (row0 + lane < a.oc) {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (c + j < nt) y[(c + j) * a.y_row + lane] = to_out<T>(__uint_as_float(r[j]));
    }
  }
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A cluster's sums added up in the order of the slices: each block takes its share of the tokens, two at a time.
template <typename T, int S>
__device__ __forceinline__ void add_slices(const GemmArgs& a, uint8_t* smem, int slice, int tile) {
  constexpr int kAtOnce = 16 / S, kStep = threads_of(1) / kRows;      // sixteen loads from the other blocks' memories under way
  const int mt = tile % a.MT, t0 = mt * a.NT, nt = min(a.NT, a.M - t0), i = threadIdx.x % kRows, row = tile / a.MT * kRows + i;
  const int c1 = nt * (slice + 1) / S;
  uint32_t from[S];
#pragma unroll
  for (int s = 0; s < S; ++s) asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from[s]) : "r"(smem_u32(smem) + (uint32_t)i * 4u), "r"(s));
  for (int c = nt * slice / S + (int)threadIdx.x / kRows; c < c1; c += kAtOnce * kStep) {
    float v[kAtOnce][S];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const int at = min(c + j * kStep, c1 - 1);
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[j][s]) : "r"(from[s] + (uint32_t)at * (kRows * 4u)));
      }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      float sum = v[j][0];
#pragma unroll
      for (int s = 1; s < S; ++s) sum += v[j][s];
      if (row < a.oc && c + j * kStep < c1) static_cast<T*>(a.Y)[(long long)(t0 + c + j * kStep) * a.y_row + row] = to_out<T>(sum);
    }
  }
}
template <typename T>
__device__ __forceinline__ void add_slices(const GemmArgs& a, uint8_t* smem, int slice, int tile) {
  if (a.slices == 2) add_slices<T, 2>(a, smem, slice, tile);
  else if (a.slices == 4) add_slices<T, 4>(a, smem, slice, tile);
  else add_slices<T, 8>(a, smem, slice, tile);
}

// A block that gives up, whichever of its roles ran out of polls, leaves only when the copies that it has asked for have arrived, one a stage in turn, and the tensor core is done
// with what it was told: until then they write to its shared and tensor memory and read it.  Called by all threads once the roles have joined; each wait has a limit, as all waits.
template <bool kLost>
__device__ __forceinline__ void leave_in_order(const GemmArgs& a, Ctrl* ctrl) {
  auto arrived = [](uint64_t* bar, uint32_t parity) {
    uint32_t it = 0;
    while (it < kPollLimit && !mbar_try_wait(bar, parity)) ++it;
    return it < kPollLimit;
  };
  if (threadIdx.x == 0) {
    bool all = true;
    for (int i = max(0, ctrl->asked - a.stages); i < ctrl->asked; ++i) all = arrived(&ctrl->full[i % a.stages], (uint32_t)(i / a.stages) & 1u) && all;
    if (kLost) { atomicAdd(a.lost, 1); atomicAdd(a.lost + 1, ctrl->asked); if (all) atomicAdd(a.lost + 2, 1); }
  }
  if (threadIdx.x >> 5 == 1 && elected()) {         // the thread that issued the instructions
    commit(smem_u32(&ctrl->drained));
    const bool done = arrived(&ctrl->drained, 0);
    if (kLost && done) atomicAdd(a.lost + 3, 1);
  }
  __syncthreads();
}

// kLost: see GemmArgs.  (A limit that is not a constant costs some 40 cycles a stage: 2048 x 14336 x 4096 113.2 -> 115.8 us.)
template <int W, bool kLost>
__global__ void __launch_bounds__(threads_of(W), 1) fp8_gemm_kernel(const __grid_constant__ GemmArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023u) & ~(uintptr_t)1023u);
  constexpr uint32_t kSfBytes = sf_bytes(W);
  const uint32_t stage_bytes = W * kWBytes + (uint32_t)a.NT * kStageCols;
  uint8_t* sf = smem + (uint32_t)a.stages * stage_bytes;
  Ctrl* ctrl = reinterpret_cast<Ctrl*>(sf + kSfSlots * kSfBytes + 4 * W * kOutBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abortp = &ctrl->abort_flag;
  const uint32_t limit = kLost ? a.poll_limit : kPollLimit;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kMaxStages; ++i) { mbar_init(&ctrl->full[i], 1); mbar_init(&ctrl->empty[i], 1); }
    for (int i = 0; i < kSfSlots; ++i) { mbar_init(&ctrl->sffull[i], 32); mbar_init(&ctrl->sfempty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&ctrl->accfull[i], 1); mbar_init(&ctrl->accempty[i], 128); }
    mbar_init(&ctrl->drained, 1);
    ctrl->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\nfence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // A cluster of `slices` blocks has one tile, each a range of its columns (whole words of scales); without slices a block goes from tile to tile.
  const int slice = a.slices > 1 ? (int)(blockIdx.x % (unsigned)a.slices) : 0, tile0 = (int)(blockIdx.x / (unsigned)a.slices);
  const int step = a.slices > 1 ? a.tiles : (int)gridDim.x;
  const int words = (a.groups + 3) / 4, k0 = words * slice / a.slices * 4, n_k = min(a.groups, words * (slice + 1) / a.slices * 4) - k0;
  auto fetch = [&](int t, int k, int st) {
    uint8_t* w = smem + (uint32_t)st * stage_bytes;
    mbar_arrive_expect_tx(&ctrl->full[st], stage_bytes);
    tensor_g2s(w, &a.wmap, (k0 + k) * kStageCols, t / a.MT * (W * kRows), &ctrl->full[st]);
    tensor_g2s(w + W * kWBytes, &a.xmap, (k0 + k) * kStageCols, t % a.MT * a.NT, &ctrl->full[st]);
  };
  // The first two stages are on their way before anything else, and copies and scales do not wait for tensor memory (one token, 4096 x 4096, 7.0 -> 6.4 us; 13 tokens, 4096 x 14336,
  // 15.2 -> 13.9).
  const int first = min(n_k, 2);               // there are at least three stages
  if (threadIdx.x == 0) {
    for (int k = 0; k < first; ++k) fetch(tile0, k, k);
  }
  // Only now: tensor memory taken while an earlier kernel still wants some would be waited for by it, and it by this one.
  if (warp == 3) tmem_alloc(&ctrl->tmem_base, a.tmem_cols);
  tc_fence_before();
  if (warp != 2 && warp != 0) asm volatile("bar.sync 1, %0;" ::"n"(threads_of(W) - 64) : "memory");
  tc_fence_after();
  asm volatile("griddepcontrol.launch_dependents;");
  const uint32_t tmem = ctrl->tmem_base;       // warps 0 and 2, which do not wait for it, have no use for it
  if (warp == 0) {
    if (lane == 0) {
      int st = first, asked = first;
      uint32_t ph = 0;
      bool ok = true;
      for (int t = tile0; ok && t < a.tiles; t += step) {
        for (int k = t == tile0 ? first : 0; k < n_k; ++k, ++asked) {
          if (!mbar_wait(&ctrl->empty[st], ph ^ 1u, abortp, a.status, limit)) { ok = false; break; }
          fetch(t, k, st);
          if (++st == a.stages) { st = 0; ph ^= 1u; }
        }
      }
      ctrl->asked = asked;
    }
    __syncwarp();
  } else if (warp == 1) {
    if (elected()) {
      int st = 0, sl = 0;
      uint32_t ph = 0, sph = 0, acc = 0, aph = 0;
      bool ok = true;
      const uint64_t wdesc = smem_desc_sw128(smem_u32(smem)), lines = smem_desc_lines(smem_u32(sf));
      const uint32_t idesc = idesc_mx(kRows, a.NT, 0), stage_step = stage_bytes >> 4;
      for (int t = tile0; ok && t < a.tiles; t += step) {
        for (int i = 0; ok && i < W; ++i) ok = mbar_wait(&ctrl->accempty[W == 1 ? acc : (uint32_t)i], aph ^ 1u, abortp, a.status, limit);
        tc_fence_after();
        for (int k = 0; ok && k < n_k; ++k) {
          const uint32_t sfa = tmem + a.tmem_cols - (uint32_t)(kSfSlots - sl) * kSfCols, sfb = sfa + 4 * W;
          if ((k & 3) == 0) {
            if (!mbar_wait(&ctrl->sffull[sl], sph, abortp, a.status, limit)) { ok = false; break; }
            tc_fence_after();
            const uint64_t src = lines + (uint32_t)sl * (kSfBytes >> 4);
#pragma unroll
            for (int i = 0; i < W; ++i) copy_scales(sfa + 4 * i, src + (uint32_t)i * (kLineBytes >> 4));
            copy_scales(sfb, src + W * (kLineBytes >> 4));
            if (a.NT > 128) copy_scales(sfb + 4, src + (W + 1) * (kLineBytes >> 4));
          }
          if (!mbar_wait(&ctrl->full[st], ph, abortp, a.status, limit)) { ok = false; break; }
          tc_fence_after();
          const uint64_t w = wdesc + (uint32_t)st * stage_step;
          const uint32_t id = idesc | (uint32_t)(k & 3) << 4 | (uint32_t)(k & 3) << 29;
#pragma unroll
          for (int i = 0; i < W; ++i) {
            mma_stage(tmem + (W == 1 ? acc : (uint32_t)i) * (uint32_t)a.NT, w + (uint32_t)i * (kWBytes >> 4), w + W * (kWBytes >> 4), id, sfa + 4 * i, sfb, k != 0);
            if (i + 1 == W) commit(smem_u32(&ctrl->empty[st]));
            if (k + 1 == n_k) commit(smem_u32(&ctrl->accfull[W == 1 ? acc : (uint32_t)i]));
          }
          if (++st == a.stages) { st = 0; ph ^= 1u; }
          if ((k & 3) == 3 || k + 1 == n_k) {
            commit(smem_u32(&ctrl->sfempty[sl]));
            if (++sl == kSfSlots) { sl = 0; sph ^= 1u; }
          }
        }
        if (W == 1) acc ^= 1u;
        if (W > 1 || acc == 0) aph ^= 1u;
      }
    }
    __syncwarp();
  } else if (warp == 2) {
    int sl = 0, said = 0;
    uint32_t sph = 0;
    bool ok = true;
    for (int t = tile0; ok && t < a.tiles; t += step) {
      const int mt = t % a.MT, rb = t / a.MT;
      const uint8_t* ws = a.w_scale + (size_t)rb * W * a.pitch;
      const bool second = W > 1 && rb * (W * kRows) + kRows < a.oc;
      for (int k = 0; k < n_k; k += 4) {
        const uint32_t ww = *reinterpret_cast<const uint32_t*>(ws + k0 + k);
        const uint32_t ww2 = second ? *reinterpret_cast<const uint32_t*>(ws + a.pitch + k0 + k) : 0x7F7F7F7Fu;
        uint32_t xw[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int r = j * 32 + lane, tok = mt * a.NT + r;
          xw[j] = r < a.NT && tok < a.M ? *reinterpret_cast<const uint32_t*>(a.x_scale + (size_t)tok * a.pitch + k0 + k) : 0x7F7F7F7Fu;
        }
        if (!mbar_wait(&ctrl->sfempty[sl], sph ^ 1u, abortp, a.status, limit)) { ok = false; break; }
        uint4* dst = reinterpret_cast<uint4*>(sf + sl * kSfBytes) + lane;
        dst[0] = make_uint4(ww, ww, ww, ww);
        if (W > 1) dst[32] = make_uint4(ww2, ww2, ww2, ww2);
        dst[32 * W] = make_uint4(xw[0], xw[1], xw[2], xw[3]);
        dst[32 * W + 32] = make_uint4(xw[4], xw[5], xw[6], xw[7]);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (!kLost || said++ < a.announced) mbar_arrive(&ctrl->sffull[sl]);
        if (++sl == kSfSlots) { sl = 0; sph ^= 1u; }
      }
    }
  } else if (warp >= 4) {
    constexpr int kHeld = W > 1 ? 3 : 1;
    uint32_t acc = W > 1 ? (uint32_t)(warp >> 2) - 1u : 0u, aph = 0;        // with two tiles of weights each has its warps
    for (int t = tile0; t < a.tiles; t += step) {
      const int mt = t % a.MT, rb = t / a.MT, t0 = mt * a.NT;
      if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctrl->accfull[acc], aph, abortp, a.status, limit))) break;        // a warp reads tensor memory as a whole or not at all
      tc_fence_after();
      const uint32_t src = tmem + acc * (uint32_t)a.NT + ((uint32_t)(warp & 3) << 21);
      const int row0 = rb * (W * kRows) + (warp - 4) * 32, nt = min(a.NT, a.M - t0);
      uint8_t* out = sf + kSfSlots * kSfBytes + (warp - 4) * kOutBytes;
      if (W == 1 && a.slices > 1) {
        // this slice's sums, where the stages were: [token][row]
        float* part = reinterpret_cast<float*>(smem) + (warp - 4) * 32 + lane;
        for (int c = 0; c < nt; c += 32) {
          uint32_t r[32];
          tmem_ld32_issue(src + (uint32_t)c, r);
          tmem_ld_wait(r);
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (c + j < nt) part[(c + j) * kRows] = __uint_as_float(r[j]);
        }
        tc_fence_before();
        mbar_arrive(&ctrl->accempty[acc]);
      } else if (a.y_dtype == RWKVQ_F32) store_tile<float, kHeld>(a, src, row0, t0, nt, out, lane, &ctrl->accempty[acc]);
      else if (a.y_dtype == RWKVQ_F16) store_tile<__half, kHeld>(a, src, row0, t0, nt, out, lane, &ctrl->accempty[acc]);
      else store_tile<__nv_bfloat16, kHeld>(a, src, row0, t0, nt, out, lane, &ctrl->accempty[acc]);
      if (W == 1) acc ^= 1u;
      if (W > 1 || acc == 0) aph ^= 1u;
    }
  }
  __syncwarp();
  if (W == 1 && a.slices > 1) {
    cluster_sync();
    if (a.y_dtype == RWKVQ_F32) add_slices<float>(a, smem, slice, tile0);
    else if (a.y_dtype == RWKVQ_F16) add_slices<__half>(a, smem, slice, tile0);
    else add_slices<__nv_bfloat16>(a, smem, slice, tile0);
    cluster_sync();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (ctrl->abort_flag) leave_in_order<kLost>(a, ctrl);
  if (warp == 3) tmem_dealloc(tmem, a.tmem_cols);
}

// codes[rows][cols] as boxes of 128 columns x box_rows rows in the 128-byte swizzle.
bool encode_codes(CUtensorMap* map, const void* codes, int rows, int cols, int box_rows) {
  EncodeTiledFn fn = encode_tiled();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)cols};
  const cuuint32_t box[2] = {(cuuint32_t)kStageCols, (cuuint32_t)box_rows}, step[2] = {1u, 1u};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles, slices and stages of a product: the cheapest by an estimate of an SM's cycles, fitted to 145 times of 29 products (1 to 4096 tokens, 512 to 14336 x
// 512 to 14336), which it gives to within a tenth (6 % on average); what it chooses is at most 3 % off the best of them, over 12 others as well.  A stage takes 290 cycles and its
// bytes at 80 a cycle, or the tensor core's 2 cycles a token where that is more, and with two tiles of weights 1.72 times as much; the epilogue 16 a token, of one tile where
// the next one's sums cover the others; slices meet in 2100 and 29 a token, and their blocks have to fit side by side (clusters of eight only up to 112 blocks); nothing is
// faster than HBM.  More tiles of fewer tokens or more slices fill SMs: 203 tokens x 7168 x 2048 8.9 us as two tiles (one: 10.5; in two slices: 12.2), 2048 x 7168 11.7 as
// two in four slices (one in four: 14.0, four in two: 13.7), one token x 4096 x 4096 6.5 in four slices, 8.6 in two, 12.3 in one.  Two tiles of weights take in a third less for
// each product, but their epilogue stands alone and they fill SMs by larger steps: 1024 x 4096 x 4096 20.8 (one: 24.9), 512 x 4096 x 4096 17.7 (one: 14.5).
struct Plan { int W, NT, MT, slices, stages; uint32_t tmem_cols, smem_bytes; };
constexpr uint32_t fixed_bytes(int W) { return 1024 + kSfSlots * sf_bytes(W) + 4 * (uint32_t)W * kOutBytes + kCtrlBytes; }
Plan plan_of(int M, int oc, int groups) {
  const int words = (groups + 3) / 4, sms = sm_count(), first = (int)(((long long)M + kMaxTokens - 1) / kMaxTokens);
  const double hbm = ((double)oc + M) * groups * 128.0 / 2750.0;
  double best = 0.0;
  Plan l = {};
  for (int i = 0; i < 12; ++i) {
    const int NT = (int)((((long long)M + first + i - 1) / (first + i) + 15) / 16 * 16), MT = (int)(((long long)M + NT - 1) / NT);
    const long long tiles = (long long)blocks_of(oc) * MT;
    const double stage = std::max(2.0 * NT, 290.0 + (kWBytes + NT * kStageCols) / 80.0);
    for (int S = 1; S <= kMaxSlices && S <= words; S *= 2) {
      if (S > 1 && tiles * S > (S == 8 ? std::min(112, sms) : sms)) break;
      const long long waves = S > 1 ? 1 : (tiles + sms - 1) / sms;
      const int stages = S > 1 ? (words + S - 1) / S * 4 : groups;
      const double cost = std::max((double)waves * stages * stage, hbm) + 16.0 * NT + (S > 1 ? 2100.0 + 29.0 * NT : 0.0);
      if (l.NT == 0 || cost < best) { best = cost; l.W = 1; l.NT = NT; l.MT = MT; l.slices = S; }
    }
    const long long tall = (blocks_of(oc) + 1) / 2 * (long long)MT;
    const double cost = std::max((double)((tall + sms - 1) / sms) * (groups * 1.72 * stage + 16.0 * NT), hbm);
    if (cost < best) { best = cost; l.W = 2; l.NT = NT; l.MT = MT; l.slices = 1; }
  }
  const uint32_t stage = (uint32_t)l.W * kWBytes + (uint32_t)l.NT * kStageCols;
  l.stages = (int)std::min<uint32_t>(kMaxStages, (kMaxSmemBytes - fixed_bytes(l.W)) / stage);
  l.smem_bytes = fixed_bytes(l.W) + (uint32_t)l.stages * stage;
  l.tmem_cols = 32;
  while (l.tmem_cols < (uint32_t)l.NT * 2u + kSfSlots * kSfCols) l.tmem_cols *= 2;
  return l;
}
long long tiles_of(const Plan& l, int oc) { return (long long)((blocks_of(oc) + l.W - 1) / l.W) * l.MT; }
int thread_blocks_of(const Plan& l, int tiles) { return l.slices > 1 ? tiles * l.slices : std::min(tiles, sm_count()); }
int element_size(int dtype) { return dtype == RWKVQ_F32 ? 4 : dtype == RWKVQ_F16 || dtype == RWKVQ_BF16 ? 2 : 0; }

}  // namespace f8
}  // namespace rwkvq

using namespace rwkvq;
using tc5::kPollLimit;

extern "C" {

size_t rwkvq_fp8_scale_pitch(int cols) { return cols > 0 ? f8::scale_pitch(cols) : 0; }

rwkvq_status rwkvq_fp8_quantize(const void* x, int dtype, int rows, int cols, long long x_row, int block_rows, void* codes, void* scale, void* stream) {
  const int es = f8::element_size(dtype);
  if (!x || !codes || !scale || es == 0 || rows <= 0 || cols <= 0 || (block_rows != 1 && block_rows != 128)) return RWKVQ_EINVAL;
  if (cols % 16) return RWKVQ_ESHAPE;
  if (x_row < cols) return RWKVQ_EINVAL;
  if (!aligned16(x) || (x_row * es) % 16 || !aligned16(codes) || !aligned16(scale)) return RWKVQ_EALIGN;
  if ((long long)rows * f8::blocks_of(cols) > (1ll << 30)) return RWKVQ_EUNSUPPORTED;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int pitch = (int)f8::scale_pitch(cols);
  if (dtype == RWKVQ_F32) return cuda_status(f8::quantize<float>(x, x_row, rows, cols, block_rows, codes, scale, pitch, s));
  if (dtype == RWKVQ_F16) return cuda_status(f8::quantize<__half>(x, x_row, rows, cols, block_rows, codes, scale, pitch, s));
  return cuda_status(f8::quantize<__nv_bfloat16>(x, x_row, rows, cols, block_rows, codes, scale, pitch, s));
}

static rwkvq_status gemm_fp8(const void* w_codes, const void* w_scale, int oc, int ic, const void* x_codes, const void* x_scale, int M, void* Y, int y_dtype,
                             long long y_row, uint32_t poll_limit, int announced, int* lost, void* stream) {
  if (!w_codes || !w_scale || !x_codes || !x_scale || !Y || oc <= 0 || ic <= 0 || M <= 0 || f8::element_size(y_dtype) == 0 || y_row < oc) return RWKVQ_EINVAL;
  if (ic % 16) return RWKVQ_ESHAPE;
  if (!aligned16(w_codes) || !aligned16(w_scale) || !aligned16(x_codes) || !aligned16(x_scale) || !aligned16(Y)) return RWKVQ_EALIGN;
  f8::GemmArgs a;
  memset(&a, 0, sizeof(a));
  a.w_scale = static_cast<const uint8_t*>(w_scale); a.x_scale = static_cast<const uint8_t*>(x_scale);
  a.Y = Y; a.y_row = y_row; a.wide = (y_row * f8::element_size(y_dtype)) % 16 == 0; a.oc = oc; a.M = M; a.y_dtype = y_dtype;
  a.groups = f8::blocks_of(ic); a.pitch = (int)f8::scale_pitch(ic);
  const f8::Plan l = f8::plan_of(M, oc, a.groups);
  const long long tiles = f8::tiles_of(l, oc);
  if (tiles > (1ll << 28)) return RWKVQ_EUNSUPPORTED;
  a.NT = l.NT; a.MT = l.MT; a.slices = l.slices; a.stages = l.stages; a.tiles = (int)tiles; a.tmem_cols = l.tmem_cols;
  a.status = device_status_ptr();
  if (!a.status) return RWKVQ_ECUDA;
  a.poll_limit = poll_limit; a.lost = lost; a.announced = announced;
  if (!f8::encode_codes(&a.wmap, w_codes, oc, ic, l.W * f8::kRows) || !f8::encode_codes(&a.xmap, x_codes, M, ic, a.NT)) return RWKVQ_ECUDA;
  static SmemOptIn opt_in[4] = {SmemOptIn(kCarveOut), SmemOptIn(kCarveOut), SmemOptIn(kCarveOut), SmemOptIn(kCarveOut)};
  const auto kernel = lost ? (l.W == 2 ? f8::fp8_gemm_kernel<2, true> : f8::fp8_gemm_kernel<1, true>)
                           : (l.W == 2 ? f8::fp8_gemm_kernel<2, false> : f8::fp8_gemm_kernel<1, false>);
  const cudaError_t e = opt_in[(lost ? 2 : 0) + l.W - 1]((const void*)kernel, (int)f8::kMaxSmemBytes);
  if (e != cudaSuccess) return cuda_status(e);
  cudaLaunchAttribute attr[2];
  const unsigned blocks = (unsigned)f8::thread_blocks_of(l, a.tiles);
  cudaLaunchConfig_t cfg = f8::launch_config(dim3(blocks), f8::threads_of(l.W), l.smem_bytes, static_cast<cudaStream_t>(stream), attr);
  if (l.slices > 1) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)l.slices; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  }
  return cuda_status(cudaLaunchKernelEx(&cfg, kernel, a));
}

rwkvq_status rwkvq_gemm_fp8(const void* w_codes, const void* w_scale, int oc, int ic, const void* x_codes, const void* x_scale, int M, void* Y, int y_dtype,
                            long long y_row, void* stream) {
  return gemm_fp8(w_codes, w_scale, oc, ic, x_codes, x_scale, M, Y, y_dtype, y_row, kPollLimit, 0, nullptr, stream);
}

rwkvq_status rwkvq_gemm_fp8_plan(int M, int oc, int ic, int32_t* plan) {
  if (!plan || M <= 0 || oc <= 0 || ic <= 0) return RWKVQ_EINVAL;
  if (ic % 16) return RWKVQ_ESHAPE;
  const f8::Plan l = f8::plan_of(M, oc, f8::blocks_of(ic));
  const long long tiles = f8::tiles_of(l, oc);
  if (tiles > (1ll << 28)) return RWKVQ_EUNSUPPORTED;
  plan[0] = l.W * f8::kRows; plan[1] = l.NT; plan[2] = l.slices; plan[3] = (int32_t)tiles; plan[4] = f8::thread_blocks_of(l, (int)tiles); plan[5] = l.stages;
  return RWKVQ_OK;
}

rwkvq_status rwkvq_gemm_fp8_lost(const void* w_codes, const void* w_scale, int oc, int ic, const void* x_codes, const void* x_scale, int M, void* Y, int y_dtype,
                                 long long y_row, uint32_t poll_limit, int announced, int32_t* lost, void* stream) {
  if (!lost || announced < 0) return RWKVQ_EINVAL;
  return gemm_fp8(w_codes, w_scale, oc, ic, x_codes, x_scale, M, Y, y_dtype, y_row, poll_limit ? poll_limit : kPollLimit, announced, lost, stream);
}

}  // extern "C"
