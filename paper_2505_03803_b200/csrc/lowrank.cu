// Low-rank adapters of many sequences beside a shared projection: y_t += s_a B_a (A_a x_t), a the adapter of t's sequence.
//
// A tile is up to sixteen rows that have the same adapter; a cluster of thread blocks works on one.  Each block multiplies its share of the columns of A
// with the rows' (token-shifted) inputs, the blocks add up their shares through distributed shared memory, and each multiplies its share of the rows of B
// with the result: one launch, no workspace, sums in a fixed order.
//
// Weights come through tensor maps into a ring of shared memory, B's on their way while A's are multiplied, and are the 16-row operand of mma.sync.  Products are
// exact: where the types of x and the weights differ, numbers are taken apart into bf16 terms (f16: two, f32: three), and so is A x, which is summed in fp32
// (three terms, all of it, where y has 32 bits; two, the second rounded, where y has 16: off by up to 2^-16 of it).
//
// What such a call takes is latency, and much of that the instructions themselves, which are fetched for the first time in each block: loops are kept short and rolled
// up (the same with weights straight to registers, unrolled for sixteen loads a lane on their way: 33 us where this takes XX, 96 rows with 64 adapters of 4096 x 4096).
#include <cooperative_groups.h>

#include "lowrank.cuh"

namespace cg = cooperative_groups;

namespace rwkvq {
namespace lr {

// ---- few rows -----------------------------------------------------------------------------------------------
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&w)[4], uint32_t x0, uint32_t x1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(x0), "r"(x1));
}
// A pair of f16 weights as two pairs of bf16: eleven bits are eight and three.  (Of an infinity the second is NaN.)
__device__ __forceinline__ void apart(uint32_t w, uint32_t& hi, uint32_t& lo) {
  float2 f = pair_of(w, __half());
  hi = cut_off(f);
  lo = rounded(f, __nv_bfloat16());
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// A slot of the ring: as many pieces of 64 columns of all rows of A as fit, or 128 rows by 64 columns of B.
constexpr int kSlotBytes = 16 << 10, kPass = 8, kXPiece = kRows * 128;      // a pass over x: pieces of 64 columns that are in shared memory at a time
constexpr int kAll = kThreads + 32;                                         // a warp that asks for copies
template <typename X>
struct Shape {
  static constexpr int kTerms = Form<X, __half>::kX, kSlots = kTerms == 1 ? 4 : 3;        // two blocks an SM
  static constexpr int kXBytes = kTerms * kPass * kXPiece, kHBytes = 3 * 2 * kXPiece, kFront = kXBytes > kHBytes ? kXBytes : kHBytes;
  static constexpr int kPart = 4 * kRows * 68 * 4;                  // sums of half of the warps: [warp][row][rank], 64 of them and four warps, or 128 and two
  static constexpr int kShare = kRows * kMostRank * 4;
  static constexpr int kBytes = 1024 + kSlots * kSlotBytes + kFront + kPart + kShare + 256 * 4;
  static_assert(kPart >= 8 * kMostCounted && kPart >= 2 * kRows * 132 * 4, "room for counting the rows of adapters, and for two warps' sums");
};
struct Ctrl {
  uint64_t full[4], empty[4];
  int abort_flag, asked;
};

// One weight fragment (16 rows x 16 columns), taken apart, by up to sixteen rows of x in kTerms terms, the small products first.
template <int kTerms>
__device__ __forceinline__ void multiply(float (&d)[2][4], const uint32_t (&w)[4], const uint32_t (&x)[kTerms][4], int terms, bool both) {
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) apart(w[i], hi[i], lo[i]);
#pragma unroll
  for (int k = kTerms - 1; k >= 0; --k) {
    if (k >= terms) continue;
    mma(d[0], lo, x[k][0], x[k][1]);
    if (both) mma(d[1], lo, x[k][2], x[k][3]);
    mma(d[0], hi, x[k][0], x[k][1]);
    if (both) mma(d[1], hi, x[k][2], x[k][3]);
  }
}

template <typename X>
__global__ void __launch_bounds__(kAll, 2) lowrank_kernel(const __grid_constant__ Args p) {
  using S = Shape<X>;
  using F = Form<X, __half>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023u) & ~(uintptr_t)1023u);
  __shared__ Tile t;
  __shared__ Ctrl ctrl;
  __shared__ int scratch[2 * kWarps + 2];
  uint8_t* const xs = smem + S::kSlots * kSlotBytes;                     // [term][piece][row][64 columns], then A x: [term][piece][row][64 of the rank]
  float* const part = reinterpret_cast<float*>(xs + S::kFront);
  float* const share = part + S::kPart / 4;                              // this block's share of A x: [row][rank]
  uint32_t* const codebook = reinterpret_cast<uint32_t*>(share + S::kShare / 4);
  const rwkvq_lowrank_args& a = p.a;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
  volatile int* const abortp = &ctrl.abort_flag;
  asm volatile("griddepcontrol.launch_dependents;");
  if (tid == 0) {
    for (int i = 0; i < S::kSlots; ++i) { tc5::mbar_init(&ctrl.full[i], 1); tc5::mbar_init(&ctrl.empty[i], kWarps); }
    ctrl.abort_flag = ctrl.asked = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\nfence.proxy.async.shared::cta;" ::: "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (p.mu)
    for (int i = tid; i < p.mu_entries; i += kAll) codebook[i] = p.mu_codebook[i];
  const int id = (int)(blockIdx.x / C), item = id / p.splits, split = id - item * p.splits;
  find_rows<kRows>(p, item, t, scratch, part);
  const int n = t.n;
  const bool both = n > 8, grouped = single_rows(a);
  const int pieces = (a.ic + 63) / 64, k0 = (int)((long long)pieces * c / C), k1 = (int)((long long)pieces * (c + 1) / C);
  const int tiles = (a.oc + 127) / 128, parts = C * p.splits, at = split * C + c;
  const int o0 = (int)((long long)tiles * at / parts), o1 = (int)((long long)tiles * (at + 1) / parts);
  const uint32_t ring = tc5::smem_u32(smem), full = tc5::smem_u32(ctrl.full), empty = tc5::smem_u32(ctrl.empty);

  // x of columns [kp, ke), pieces of 64, in operand form
  auto stage_x = [&](auto mix, int kp, int ke) {
    const int eights = (ke - kp) * 8;
#pragma unroll 1
    for (int e = tid; e < n * eights; e += kThreads) {
      const int r = e / eights, eight = e - r * eights, col = kp * 64 + eight * 8, row = grouped ? t.rows[r] : t.first + r;
      const Eights<X> raw = load_eights<X, decltype(mix)::value>(p, row_at<X>(p, row, grouped ? row : t.seq, grouped || row == t.start), col);
      const MuWords words = load_mu<decltype(mix)::value>(p, col);
      float2 mu[4];
      mu_of<decltype(mix)::value>(p, codebook, words, col, mu);
      put_eights<X, F, decltype(mix)::value>(raw, mu, xs + eight / 8 * kXPiece + swizzled(r, eight & 7), kPass * kXPiece);
    }
  };
  auto stage = [&](int kp, int ke) { if (p.mu) stage_x(std::true_type(), kp, ke); else stage_x(std::false_type(), kp, ke); };
  if (warp == kWarps) {
    if (lane == 0) find_adapter(p, t);
  } else {
    stage(k0, min(k0 + kPass, k1));
  }
  __syncthreads();
  if (t.n == 0) return;            // the same for all blocks of the cluster
  const int rank = t.rank, blocks = (rank + 15) / 16;
  // ---- the ring: pieces of A for this block's columns, then tiles of B for its rows
  const int a_slot = blocks == 1 ? 8 : blocks == 2 ? 4 : blocks <= 4 ? 2 : 1, n_a = (k1 - k0 + a_slot - 1) / a_slot;      // pieces of A in a slot
  const int wide = (rank + 63) / 64;
  bool ok = true;
  auto take = [&](int i) { ok = ok && tc5::mbar_wait(full + (uint32_t)(i % S::kSlots) * 8u, (uint32_t)(i / S::kSlots) & 1u, abortp, p.status); };
  auto give = [&](int i) {
    __syncwarp();
    if (lane == 0) tc5::mbar_arrive(empty + (uint32_t)(i % S::kSlots) * 8u);
  };
  if (warp == kWarps) {
    // This warp brings nothing to the first meeting of the cluster and does not hold it up: the slots that it waits for below are given back behind it.
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    const int total = n_a + (o1 - o0) * wide;
    int i = 0;
#pragma unroll 1
    for (; i < total; ++i) {
      const uint32_t st = (uint32_t)(i % S::kSlots), bar = full + st * 8u, dst = ring + st * kSlotBytes;
      if (i >= S::kSlots && !__all_sync(~0u, tc5::mbar_wait(empty + st * 8u, (uint32_t)(i / S::kSlots - 1) & 1u, abortp, p.status))) break;
      if (i < n_a) {
        const int first = k0 + i * a_slot, count = min(a_slot, k1 - first) * blocks;
        if (lane == 0) tc5::mbar_arrive_expect_tx(&ctrl.full[st], (uint32_t)count * 2048u);
        __syncwarp();
#pragma unroll 1
        for (int j = 0, piece = first, r = 0; j < count; ++j) {
          tensor_g2s(dst + (uint32_t)j * 2048u, &p.A[0], piece * 64, r, t.adapter, bar);
          r += 16;
          if (r >= rank) { r = 0; ++piece; }
        }
      } else {
        const int j = i - n_a, tile = j / wide;
        if (lane == 0) tc5::mbar_arrive_expect_tx(&ctrl.full[st], kSlotBytes);
        __syncwarp();
        tensor_g2s(dst, &p.B, (j - tile * wide) * 64, (o0 + tile) * 128, t.adapter, bar);
      }
    }
    if (lane == 0) ctrl.asked = i;
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;\nbarrier.cluster.arrive.release.aligned;" ::: "memory");
  } else {
    // ---- A x.  Warps side by side along the columns; two groups of them, each 64 of the rank, where it is longer
    const int deep = blocks > 4 ? 4 : 8, kw = warp % deep, r_first = warp / deep * 4, side = min(4, blocks - r_first);
    float acc[4][2][4] = {};
    const uint32_t x_at = tc5::smem_u32(xs) + (uint32_t)((lane & 7) + (lane >> 4) * 8) * 128u;
    int i = 0;
    for (int kp = k0; kp < k1; kp += kPass) {
      const int ke = min(kp + kPass, k1);
      if (kp > k0) {
        asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
        stage(kp, ke);
        asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
      }
      // rows of x behind the n-th hold whatever was there: a row meets its own outputs alone
      for (int first = kp; first < ke; first += a_slot, ++i) {
        take(i);
        const uint32_t slot = ring + (uint32_t)(i % S::kSlots * kSlotBytes);
        const int steps = min(a_slot, ke - first) * 4;
        if (ok)
#pragma unroll 1
          for (int s = kw; s < steps; s += deep) {
            const int piece = s >> 2, eight = (s & 3) * 2;
            const uint32_t at_x = x_at + (uint32_t)((first - kp + piece) * kXPiece) + (uint32_t)(((eight + (lane >> 3 & 1)) ^ lane) & 7) * 16u;
            const uint32_t at_w = slot + (uint32_t)(piece * blocks + r_first) * 2048u + swizzled(lane & 15, eight + (lane >> 4));
            uint32_t x[F::kX][4], w[4][4];
#pragma unroll
            for (int k = 0; k < F::kX; ++k) ldmatrix4(x[k], at_x + (uint32_t)k * (kPass * kXPiece));
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (j < side) ldmatrix4(w[j], at_w + (uint32_t)j * 2048u);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (j < side) multiply<F::kX>(acc[j], w[j], x, F::kX, both);
          }
        give(i);
      }
    }
    // the warps' sums added up: the second half of them to the first, then what is left of these
    const int half = deep / 2, pitch = blocks > 4 ? 132 : 68;        // pitches that spare banks
    auto each = [&](auto f) {
      float* const to = part + (kw % half) * kRows * pitch + r_first * 16 + g;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = b * 8 + q * 2 + e;
          if (row >= n) continue;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (j < side) { f(to[row * pitch + j * 16], acc[j][b][e]); f(to[row * pitch + j * 16 + 8], acc[j][b][e + 2]); }
        }
    };
    if (kw >= half) each([](float& s, float v) { s = v; });
    asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
    if (kw < half) each([](float& s, float v) { s += v; });
    asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
    for (int row = warp; row < n; row += kWarps)
      for (int r = lane; r < blocks * 16; r += 32) {
        float s = part[row * pitch + r] + part[(kRows + row) * pitch + r];
        if (half == 4) s += part[(2 * kRows + row) * pitch + r] + part[(3 * kRows + row) * pitch + r];
        share[row * kMostRank + r] = s;
      }
    cluster.sync();

    // ---- all of A x, as operands
    const int last_term = a.y_dtype == RWKVQ_F32 ? 2 : 1;
    const float scale = t.scale;
    for (int row = warp; row < n; row += kWarps)
#pragma unroll 1
      for (int r = lane; r < blocks * 16; r += 32) {
        float s = 0.f;
        if (r < rank) {
          float v[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = k < C ? cluster.map_shared_rank(share, k)[row * kMostRank + r] : 0.f;
#pragma unroll
          for (int k = 0; k < 8; ++k) s += v[k];
          s *= scale;
        }
        uint8_t* const to = xs + r / 64 * kXPiece + swizzled(row, r / 8 & 7) + (r & 7) * 2;
        *reinterpret_cast<__nv_bfloat16*>(to) = term(s);
        *reinterpret_cast<__nv_bfloat16*>(to + 2 * kXPiece) = last_term == 1 ? __float2bfloat16_rn(s) : term(s);
        if (last_term == 2) *reinterpret_cast<__nv_bfloat16*>(to + 4 * kXPiece) = term(s);
      }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");

    // ---- B (A x) for this block's rows of B, sixteen of a tile's for each warp
    i = n_a;
    for (int o = o0; o < o1; ++o) {
      float d[2][4] = {};
      for (int k = 0; k < wide; ++k, ++i) {
        take(i);
        const uint32_t slot = ring + (uint32_t)(i % S::kSlots * kSlotBytes + warp * 2048);
        const int steps = min(4, blocks - k * 4);
        if (ok)
#pragma unroll 1
          for (int s = 0; s < steps; ++s) {
            uint32_t x[3][4], w[1][4];
            ldmatrix4(w[0], slot + swizzled(lane & 15, s * 2 + (lane >> 4)));
            const uint32_t at_x = x_at + (uint32_t)(k * kXPiece) + (uint32_t)(((s * 2 + (lane >> 3 & 1)) ^ lane) & 7) * 16u;
#pragma unroll
            for (int j = 0; j < 3; ++j)
              if (j <= last_term) ldmatrix4(x[j], at_x + (uint32_t)j * (2 * kXPiece));
            const int left = rank - (k * 64 + s * 16);
            if (left < 16) {        // what lies behind the adapter's rank may be anything
              const uint32_t lo = q * 2 + 2 <= left ? ~0u : q * 2 + 1 <= left ? 0xFFFFu : 0u, hi = q * 2 + 10 <= left ? ~0u : q * 2 + 9 <= left ? 0xFFFFu : 0u;
              w[0][0] &= lo; w[0][1] &= lo; w[0][2] &= hi; w[0][3] &= hi;
            }
            multiply<3>(d, w[0], x, last_term + 1, both);
          }
        give(i);
      }
      if (!ok) break;
      // y: all that is read first, then the sums
      const int col = o * 128 + warp * 16 + g;
      auto y_at = [&](int b, int e) { const int r = b * 8 + q * 2 + (e & 1); return (long long)(grouped ? t.rows[r] : t.first + r) * a.y_row + col + (e >> 1) * 8; };
      auto there = [&](int b, int e) { return b * 8 + q * 2 + (e & 1) < n && col + (e >> 1) * 8 < a.oc; };
      if (a.y_dtype == RWKVQ_F32) {
        // Each element of y is added to once in a call, so that a reduction in memory is as good as a load, an addition and a store, and nothing waits for it (it
        // takes subnormal numbers for zeros).
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (there(b, e)) asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(static_cast<float*>(a.y) + y_at(b, e)), "f"(d[b][e]) : "memory");
      } else {
        unsigned short* const y = static_cast<unsigned short*>(a.y);
        unsigned short old[2][4];
        const long long y_at_first = (long long)(grouped ? t.rows[0] : t.first) * a.y_row;        // somewhere valid
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) old[b][e] = y[there(b, e) ? y_at(b, e) : y_at_first];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (there(b, e))
              y[y_at(b, e)] = a.y_dtype == RWKVQ_F16 ? __half_as_ushort(__float2half_rn(__half2float(__ushort_as_half(old[b][e])) + d[b][e]))
                                                     : __bfloat16_as_ushort(__float2bfloat16_rn(__bfloat162float(__ushort_as_bfloat16(old[b][e])) + d[b][e]));
      }
    }
  }
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");        // no block ends while another reads its share
  __syncthreads();
  // a block that gave up leaves when its copies have arrived
  if (ctrl.abort_flag && tid == 0)
    for (int i = max(0, ctrl.asked - S::kSlots); i < ctrl.asked; ++i)
      for (uint32_t k = 0; k < tc5::kPollLimit && !tc5::mbar_try_wait(full + (uint32_t)(i % S::kSlots) * 8u, (uint32_t)(i / S::kSlots) & 1u); ++k) {}
}

template <typename X>
cudaError_t launch(Args& p, long long items, cudaStream_t s) {
  using S = Shape<X>;
  const rwkvq_lowrank_args& a = p.a;
  if (!encode(p.A, a.A, true, a.ic, a.rank, a.n_adapters, 16) || !encode(&p.B, a.B, true, a.rank, a.oc, a.n_adapters, 128)) return cudaErrorUnknown;
  static SmemOptIn opt_in(kCarveOut);
  cudaError_t e = opt_in((const void*)lowrank_kernel<X>, S::kBytes);
  if (e != cudaSuccess) return e;
  // blocks that are there at once, two an SM: clusters as wide as that allows
  unsigned C = 8;
  while (C > 1 && items * C > 2ll * sm_count()) C /= 2;
  // where there are few tiles, several clusters divide a tile's rows of B, and each multiplies A x for itself
  p.splits = (int)std::max<long long>(1, std::min<long long>({2ll * sm_count() / (items * C), (a.oc + 128ll * C - 1) / (128 * C), 16}));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(items * C * p.splits)); cfg.blockDim = dim3(kAll); cfg.dynamicSmemBytes = S::kBytes; cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, lowrank_kernel<X>, p);
}
cudaError_t launch(Args& p, cudaStream_t s) {
  if (tiles_take(p.a.x_dtype, p.a.w_dtype)) return launch_tiles(p, s);
  const long long items = most_tiles(p.a, kRows);
  return p.a.x_dtype == RWKVQ_F32 ? launch<float>(p, items, s) : launch<__nv_bfloat16>(p, items, s);
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
  return cuda_status(lr::launch(p, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
