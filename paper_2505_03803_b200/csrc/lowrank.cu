// Low-rank adapters of many sequences beside a shared projection: y_t += s_a B_a (A_a x_t), a the adapter of t's sequence.  On the tcgen05 tensor cores, in tiles of up to 64 rows
// of a sequence, or of up to sixteen rows that share an adapter.
//
// The rows are the 16- to 64-column operand and the weights the 128-row one: A x is one accumulator of 128 (of the rank) by the tile's rows, B (A x) one for each 128 rows
// of B, whose lanes are neighbouring columns of y.  A cluster of blocks divides the columns of A and the rows of B; A x is summed over the blocks through distributed
// shared memory in their order: one launch, no workspace.  Weights come through tensor maps into a ring of seven to eleven slots, B's under the meeting of the blocks; x through a map, too, or,
// where it has to be mixed with the row before or taken apart (see Form), by the warps that read the accumulators later.
//
// A x, in fp32, goes on in three bf16 terms, which are all of it, or, where the weights are f16, in two f16 terms under a power of two per row that brings its largest number to
// 2^14 (off by up to 2^-22 of it, or 2^-38 of the row's largest).
//
// Bytes bind the large calls and latency the small ones, and what such a block does besides: one token (2048 x 2048, rank 16) 6.8 us, of which the launch is 2.5; 96 sequences with 64 adapters
// (4096 x 4096) 19 us, 2.3 TB/s of what it reads; a prompt of 2048 rows 21 us, 2.5 TB/s, floor 7.8.  As many tensor products as there are cost little: the roles are laid out so that copies never wait.  The first
// form, on mma.sync with sixteen rows a tile, took 10, 39 and 84 us.
//
// A block takes all of an SM's shared memory, so that no other one that wants tensor memory is beside it: tcgen05.alloc has no limit to its wait, and a block
// that holds tensor memory waits for the others of its cluster.
#include <cooperative_groups.h>

#include "lowrank.cuh"

namespace cg = cooperative_groups;

namespace rwkvq {
namespace lr {

using tc5::smem_u32;

constexpr int kMostRing = 11, kSlotBytes = 16 << 10, kMostGroups = 4, kMostAcc = 4;
constexpr int kSmemBytes = 224 << 10;

// Pieces of 64 columns of A that a slot holds where the rank is up to 16 * blocks.
__host__ __device__ constexpr int pieces_of(int blocks) { return blocks == 1 ? 8 : blocks == 2 ? 4 : blocks <= 4 ? 2 : 1; }

template <typename X, typename W, int NT>
struct TileShape {
  static constexpr int kTerms = Form<X, W>::kX, kTileBytes = NT * 128, kPieceBytes = kTerms * kTileBytes;      // a piece: 64 columns of the tile's rows, a tile for each term
  static constexpr int kGroup = NT == 64 ? 2 : 8, kGroups = NT == 16 ? 2 : kTerms == 1 ? 4 : kTerms == 2 ? 2 : 1;      // pieces that come at once, and how many such groups there is room for
  static constexpr int kXBytes = kGroup * kGroups * kPieceBytes, kShare = NT * kMostRank * 4;
  // Warps that make operands and read accumulators; behind them one that asks for copies, one that multiplies, two that mask.
  static constexpr int kWorkers = NT == 64 ? 16 : 8, kWork = kWorkers * 32, kAll = kWork + 128;
  static constexpr int kEights = kGroup * 8, kPer = kEights * NT / kWork;          // of a row in a group, and those of a thread where the tile is full
  // Few rows: the terms lie side by side, as more columns of one product, and are added up when they are read (a product of few columns takes as long as its 128 weight rows take to
  // read).  Many rows: one product after another into the same accumulator.
  static constexpr bool kBeside = NT == 16;
  static constexpr int kColsA = kBeside ? NT * kTerms : NT, kColsB = kBeside ? NT * 3 : NT;        // of an accumulator
  static constexpr int kAcc = 4, kTmemCols = NT == 64 ? 512 : 256;
  static_assert(kColsA + kAcc * kColsB <= kTmemCols, "tensor memory");
  // The warps that read an accumulator, sixteen of its rows' columns each: a quarter of 64 rows, or all of sixteen, of every second tile.
  static constexpr int kReaders = NT == 64 ? 16 : 4, kReadCols = 16;
  static_assert(kXBytes >= 6 * kTileBytes, "A x takes x's place");
  // as many slots as there is room for, beside the codebook and what aligning takes
  static constexpr int kFree = (kSmemBytes - 2048 - kXBytes - kShare) / kSlotBytes, kRing = kFree < kMostRing ? kFree : kMostRing;
  static_assert(kRing >= 7, "shared memory");
  static_assert(kShare >= 8 * kMostCounted || NT == 64, "room for counting the rows of adapters");
};
struct TileCtrl {
  uint64_t y_full[16], full[kMostRing], empty[kMostRing], masked[kMostRing + 1], ready, xfull[kMostGroups], xempty[kMostGroups], a_done, full_acc[kMostAcc], empty_acc[kMostAcc], drained;
  int abort_flag, asked, x_asked;
  uint32_t tmem_base;
  float back[64];                 // of each row: the power of two that its A x was divided by
  int top[64];                    // the bits of the largest finite number of a row that this block has
};
// Slots of a ring in turn.
template <int N>
struct Turn {
  uint32_t at = 0, parity = 0;
  __device__ __forceinline__ void next() { if (++at == N) { at = 0; parity ^= 1u; } }
};

// Both operands of a type (bf16, or f16), K-major -> fp32, 128 x N.
__device__ __forceinline__ constexpr uint32_t idesc_of(bool half, int N) {
  return (1u << 4) | (half ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)(N >> 3) << 17) | ((128u >> 4) << 24);
}
// Up to four steps of sixteen columns of both operands, by a converged warp: one lane is elected for all of them (a step at a time took some 100 cycles each).
__device__ __forceinline__ void umma(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, bool accumulate, int steps) {
  asm volatile(
      "{\n .reg .pred q, p, one, q1, q2, q3;\n .reg .b64 a1, a2, a3, b1, b2, b3;\n"
      " elect.sync _|q, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n setp.eq.b32 one, 0, 0;\n"
      " setp.gt.and.s32 q1, %5, 1, q;\n setp.gt.and.s32 q2, %5, 2, q;\n setp.gt.and.s32 q3, %5, 3, q;\n"
      " add.u64 a1, %1, 2;\n add.u64 a2, %1, 4;\n add.u64 a3, %1, 6;\n add.u64 b1, %2, 2;\n add.u64 b2, %2, 4;\n add.u64 b3, %2, 6;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
      " @q1 tcgen05.mma.cta_group::1.kind::f16 [%0], a1, b1, %3, one;\n"
      " @q2 tcgen05.mma.cta_group::1.kind::f16 [%0], a2, b2, %3, one;\n"
      " @q3 tcgen05.mma.cta_group::1.kind::f16 [%0], a3, b3, %3, one;\n}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"((uint32_t)accumulate), "r"(steps) : "memory");
}
// 32 lanes x kCols columns; see tc5::tmem_ld32_issue.  Waits for them.
template <int kCols>
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[kCols]) {
  static_assert(kCols == 8 || kCols == 16, "");
  if constexpr (kCols == 16) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
                   "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
                 "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
  } else {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]) :: "memory");
  }
}
__device__ __forceinline__ void tensor_g2s(uint32_t dst_smem, const CUtensorMap* map, int x, int y, int z, int v, uint32_t bar) {
  asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n"
               " @q cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n}"
               ::"r"(dst_smem), "l"(map), "r"(x), "r"(y), "r"(z), "r"(v), "r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t pair_bits(__nv_bfloat16 x, __nv_bfloat16 y) { return (uint32_t)__bfloat16_as_ushort(x) | (uint32_t)__bfloat16_as_ushort(y) << 16; }
__device__ __forceinline__ uint32_t pair_bits(__half x, __half y) { return (uint32_t)__half_as_ushort(x) | (uint32_t)__half_as_ushort(y) << 16; }

// What a warp has of each accumulator: 32 lanes, neighbouring columns of y, and a quarter of its rows (64), or all of every second tile's (16).
template <typename S>
struct Share {
  static constexpr int kCols = S::kReadCols, kStep = S::kWorkers / S::kReaders;
  static constexpr int kTurn = S::kTileBytes / 128 * kMostRank / S::kWorkers / 32;          // rows of 32 numbers that its part of the shares' place holds
  int lane, warp, quarter, col0, first, rows;            // rows: maybe none
  float* turn;
  __device__ __forceinline__ Share(int n, float* share) {
    lane = threadIdx.x & 31; warp = threadIdx.x >> 5; quarter = warp & 3;
    col0 = kStep == 1 ? (warp >> 2) * kCols : 0; first = kStep == 1 ? 0 : warp >> 2;
    rows = min(n - col0, kCols);
    turn = share + warp * (kTurn * 32);
  }
  // The o-th accumulator, added up over its terms, and given back; false where a wait gave up.
  __device__ __forceinline__ bool take(const Args& p, TileCtrl& ctrl, uint32_t acc0, int o, int last_term, bool& ok, float (&sum)[kCols]) const {
    const int acc = o % S::kAcc;
    ok = ok && tc5::mbar_wait(smem_u32(&ctrl.full_acc[acc]), (uint32_t)(o / S::kAcc) & 1u, &ctrl.abort_flag, p.status);
    if (!__all_sync(~0u, ok)) return false;
    tc5::tc_fence_after();
    const uint32_t from = acc0 + (uint32_t)(acc * S::kColsB + col0);
    uint32_t v[kCols];
    tmem_ld<kCols>(from, v);
#pragma unroll
    for (int j = 0; j < kCols; ++j) sum[j] = __uint_as_float(v[j]);
    if constexpr (S::kBeside) {
#pragma unroll 1
      for (int k = 1; k <= last_term; ++k) {
        tmem_ld<kCols>(from + (uint32_t)(k * kCols), v);
#pragma unroll
        for (int j = 0; j < kCols; ++j) sum[j] += __uint_as_float(v[j]);
      }
    }
    tc5::tc_fence_before();
    __syncwarp();
    if (lane == 0) tc5::mbar_arrive(&ctrl.empty_acc[acc]);
    return true;
  }
};

// The accumulators of tiles [o0, o1) of B to y of 32 bits: each element is added to once in a call, so that a reduction where y lies is as good as a load, an addition and a store
// (but for subnormal numbers, which it may take for zeros); 45 us where these took 49 (3001 rows of 4096 columns).
template <typename S, bool kScaled>
__device__ __forceinline__ void reduce_y(const Args& p, const Tile& t, TileCtrl& ctrl, uint32_t acc0, int o0, int o1, int n, bool grouped, float* share, int last_term, bool& ok) {
  const rwkvq_lowrank_args& a = p.a;
  using H = Share<S>;
  const H w(n, share);
#pragma unroll 1
  for (int o = w.first; o < o1 - o0; o += H::kStep) {
    float sum[H::kCols];
    if (!w.take(p, ctrl, acc0, o, last_term, ok, sum)) break;
    const int col = (o0 + o) * 128 + w.quarter * 32, bytes = min(32, a.oc - col) * 4;
    if (w.rows <= 0 || bytes <= 0) continue;
#pragma unroll
    for (int h = 0; h < H::kCols / H::kTurn; ++h) {
      if (h * H::kTurn >= w.rows) continue;
      asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
      __syncwarp();
#pragma unroll
      for (int j = 0; j < H::kTurn; ++j) {
        const float back = kScaled ? ctrl.back[min(w.col0 + h * H::kTurn + j, n - 1)] : 1.f;
        w.turn[j * 32 + w.lane] = kScaled ? sum[h * H::kTurn + j] * back : sum[h * H::kTurn + j];
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      // a box of sixteen rows, or, where there are fewer or they lie apart, row after row
      if (p.y_by_map && w.rows == H::kTurn) {
        asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n"
                     " @q cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];\n @q cp.async.bulk.commit_group;\n}"
                     ::"l"(&p.Y), "r"(col), "r"(t.first + w.col0), "r"(smem_u32(w.turn)) : "memory");
      } else if (const int r = h * H::kTurn + w.lane; w.lane < H::kTurn && r < w.rows) {
        float* const to = static_cast<float*>(a.y) + (long long)(grouped ? t.rows[r] : t.first + w.col0 + r) * a.y_row + col;
        asm volatile("cp.reduce.async.bulk.global.shared::cta.bulk_group.add.f32 [%0], [%1], %2;\ncp.async.bulk.commit_group;"
                     ::"l"(to), "r"(smem_u32(w.turn + w.lane * 32)), "r"(bytes) : "memory");
      }
    }
  }
  asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}

// The same to y of 16 bits, which is rounded once, for tiles of sixteen rows.  A lane of the accumulator is a column; the way to four neighbouring columns a lane is through shared memory, where the shares were
// (a column a lane, without that, took 32 us where this took 24 when it served 2048 rows of 4096 columns, too; what bounds it is the number of accesses).
template <typename S, typename Y, bool kScaled>
__device__ __forceinline__ void store_y(const Args& p, const Tile& t, TileCtrl& ctrl, uint32_t acc0, int o0, int o1, int n, bool grouped, float* share, int last_term, bool& ok) {
  static_assert(sizeof(Y) == 2 && S::kBeside, "");
  const rwkvq_lowrank_args& a = p.a;
  using H = Share<S>;
  const H w(n, share);
  const int quad = w.lane & 7, r_lane = w.lane >> 3;
  Y* at[H::kCols / 4];                                  // rows r_lane, r_lane + 4, ...; those behind the last are read as the last
#pragma unroll
  for (int i = 0; i < H::kCols / 4; ++i) {
    const int r = min(i * 4 + r_lane, w.rows - 1);
    at[i] = static_cast<Y*>(a.y) + (long long)(grouped ? t.rows[r] : t.first + r) * a.y_row;
  }
  // y of the next tiles is on its way while this one's is added to (into buffers that take turns, not moved: a move waits for what it moves)
  constexpr int kDepth = 3;
  uint2 buffers[kDepth][H::kCols / 4];
  auto load = [&](int o, uint2 (&to)[H::kCols / 4]) {
    const int col = min((o0 + o) * 128 + w.quarter * 32 + quad * 4, a.oc - 4);
    if (o < o1 - o0)
#pragma unroll
      for (int i = 0; i < H::kCols / 4; ++i) to[i] = *reinterpret_cast<const uint2*>(at[i] + col);
  };
#pragma unroll
  for (int k = 0; k < kDepth; ++k) load(w.first + k * H::kStep, buffers[k]);
#pragma unroll 1
  for (int round = w.first; round < o1 - o0; round += kDepth * H::kStep)
#pragma unroll
  for (int turn_of = 0; turn_of < kDepth; ++turn_of) {
    const int o = round + turn_of * H::kStep, col = (o0 + o) * 128 + w.quarter * 32 + quad * 4;
    if (o >= o1 - o0) continue;
    uint2 (&y)[H::kCols / 4] = buffers[turn_of];
    float sum[H::kCols];
    if (!w.take(p, ctrl, acc0, o, last_term, ok, sum)) return;
    // [row][column], rows of 128 bytes: each lane a column, then each quarter of a warp a row
#pragma unroll
    for (int h = 0; h < H::kCols / H::kTurn; ++h) {
      if (h * H::kTurn >= w.rows) continue;
#pragma unroll
      for (int j = 0; j < H::kTurn; ++j) w.turn[j * 32 + w.lane] = sum[h * H::kTurn + j];
      __syncwarp();
#pragma unroll
      for (int i = 0; i < H::kTurn / 4; ++i) {
        const int r = h * H::kTurn + i * 4 + r_lane;
        float4 d = *reinterpret_cast<const float4*>(w.turn + (i * 4 + r_lane) * 32 + quad * 4);
        if constexpr (kScaled) { const float back = ctrl.back[min(r, n - 1)]; d.x *= back; d.y *= back; d.z *= back; d.w *= back; }
        uint2& mine = y[h * H::kTurn / 4 + i];
        const float2 lo = pair_of(mine.x, Y()), hi = pair_of(mine.y, Y());
        mine = make_uint2(rounded(make_float2(lo.x + d.x, lo.y + d.y), Y()), rounded(make_float2(hi.x + d.z, hi.y + d.w), Y()));
        if (r < w.rows && col < a.oc) *reinterpret_cast<uint2*>(at[h * H::kTurn / 4 + i] + col) = mine;
      }
      __syncwarp();
    }
    load(o + kDepth * H::kStep, y);
  }
}

// 16 lanes x 16 columns, as a product's sums lie in registers: lane / 4 (and 8 more) by two neighbouring columns for each pair of registers.  Waits for them.
__device__ __forceinline__ void tmem_ld_pairs(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]) :: "memory");
}
// The same for rows that lie one behind the other: y comes to shared memory through a map, sixteen rows at a time for each four warps, where the shares were and behind A x (two to four tiles' worth), and lies in registers
// as the sums do when it is read transposed; it goes out in rows of 256 bytes.  Eight accesses of a warp to a tile where the way above takes 28
// (2048 rows, bf16: 20.7 us where that took 22.7, A x in two terms; in all three it takes 21.1).
template <typename S, typename Y, bool kScaled, int kTerms>
__device__ __forceinline__ void store_y_rows(const Args& p, const Tile& t, TileCtrl& ctrl, uint32_t acc0, int o0, int o1, int n, float* share, bool& ok) {
  const rwkvq_lowrank_args& a = p.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quarter = warp & 3, group = warp >> 2, tiles = o1 - o0;
  const int rows = min(n - group * 16, 16);              // of this group, maybe none
  // A x as operands, of up to 128 numbers a row, leaves room behind it
  constexpr int kY = 2 + (S::kXBytes - 2 * kTerms * S::kTileBytes) / (16 << 10);
  const uint32_t first = smem_u32(share) - (uint32_t)(kY - 2) * (16u << 10) + (uint32_t)group * 4096u, full = smem_u32(&ctrl.y_full[group * 4]);
  auto ask = [&](int o) {                                // by one warp of the group
    const int at = o % kY, row = t.first + group * 16, col = (o0 + o) * 128;
    const bool second = col + 64 < a.oc;
    if (lane == 0) tc5::mbar_arrive_expect_tx(&ctrl.y_full[group * 4 + at], second ? 4096u : 2048u);
    __syncwarp();
    const uint32_t to = first + (uint32_t)at * (16u << 10), bar = full + (uint32_t)at * 8u;
    tensor_g2s(to, &p.Y, col, row, 0, bar);
    if (second) tensor_g2s(to + 2048u, &p.Y, col + 64, row, 0, bar);
  };
  auto meet = [&] { asm volatile("bar.sync %0, 128;" ::"r"(2 + group) : "memory"); };
  int asked = 0;
  if (quarter == 0 && rows > 0) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    for (; asked < min(tiles, kY); ++asked) ask(asked);
  }
  // of the transposed 8 x 8 blocks: rows 0 to 7 and columns 0 to 7, columns 8 to 15, and the same of rows 8 to 15
  const int m = lane >> 3, token = (m >> 1) * 8 + (lane & 7);
  float back[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) back[j] = kScaled ? ctrl.back[max(min(group * 16 + (j >> 1) * 8 + (lane & 3) * 2 + (j & 1), n - 1), 0)] : 1.f;
#pragma unroll 1
  for (int o = 0; o < tiles; ++o) {
    const int acc = o % S::kAcc;
    ok = ok && tc5::mbar_wait(smem_u32(&ctrl.full_acc[acc]), (uint32_t)(o / S::kAcc) & 1u, &ctrl.abort_flag, p.status);
    ok = __all_sync(~0u, ok);                            // one that gives up goes through all the meetings
    tc5::tc_fence_after();
    uint32_t v[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) tmem_ld_pairs(acc0 + (uint32_t)(acc * S::kColsB + group * 16) + ((uint32_t)(h * 16) << 16), v[h]);
    tc5::tc_fence_before();
    __syncwarp();
    if (lane == 0) tc5::mbar_arrive(&ctrl.empty_acc[acc]);
    if (rows <= 0) continue;
    ok = ok && tc5::mbar_wait(full + (uint32_t)(o % kY) * 8u, (uint32_t)(o / kY) & 1u, &ctrl.abort_flag, p.status);
    ok = __all_sync(~0u, ok);
    const uint32_t tile = first + (uint32_t)(o % kY) * (16u << 10);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t at = tile + (uint32_t)(quarter >> 1) * 2048u + swizzled(token, (quarter & 1) * 4 + h * 2 + (m & 1));
      uint32_t y[4];
      asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]) : "r"(at) : "memory");
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float2 f = pair_of(y[j], Y());
        f.x = fmaf(__uint_as_float(v[h][2 * j]), back[(j >> 1) * 2], f.x);
        f.y = fmaf(__uint_as_float(v[h][2 * j + 1]), back[(j >> 1) * 2 + 1], f.y);
        y[j] = rounded(f, Y());
      }
      asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
    }
    meet();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = quarter * 4 + i * 2 + (lane >> 4), eight = lane & 15, col = (o0 + o) * 128 + eight * 8;
      uint4 w;
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(tile + (uint32_t)(eight >> 3) * 2048u + swizzled(row, eight & 7)) : "memory");
      if (ok && row < rows && col < a.oc) *reinterpret_cast<uint4*>(static_cast<Y*>(a.y) + (long long)(t.first + group * 16 + row) * a.y_row + col) = w;
    }
    meet();
    if (quarter == 0 && ok && asked < tiles) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      ask(asked++);
    }
  }
  // not left before its copies are there
  if (!ok && quarter == 0)
    for (int o = max(0, asked - kY); o < asked; ++o)
      for (uint32_t k = 0; k < tc5::kPollLimit && !tc5::mbar_try_wait(full + (uint32_t)(o % kY) * 8u, (uint32_t)(o / kY) & 1u); ++k) {}
}

template <typename X, typename W, int NT>
__global__ void __launch_bounds__((TileShape<X, W, NT>::kAll), 1) lowrank_tile_kernel(const __grid_constant__ Args p) {
  using S = TileShape<X, W, NT>;
  using F = Form<X, W>;
  constexpr bool kHalf = std::is_same<W, __half>::value;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023u) & ~(uintptr_t)1023u);
  __shared__ Tile t;
  __shared__ TileCtrl ctrl;
  __shared__ int scratch[2 * kWarps + 2];
  uint8_t* const xs = smem + S::kRing * kSlotBytes;                         // [slot][term][row][64 columns], then A x: [term][64 of the rank][row][64], or [64 of the rank][term][row][64]
  float* const share = reinterpret_cast<float*>(xs + S::kXBytes);        // this block's share of A x: [row][rank]
  uint32_t* const codebook = reinterpret_cast<uint32_t*>(share + S::kShare / 4);
  const rwkvq_lowrank_args& a = p.a;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  volatile int* const abortp = &ctrl.abort_flag;
  asm volatile("griddepcontrol.launch_dependents;");
  if (tid < 64) ctrl.top[tid] = 0;
  if (tid == 0) {
    for (int i = 0; i < S::kRing; ++i) { tc5::mbar_init(&ctrl.full[i], 1); tc5::mbar_init(&ctrl.empty[i], 1); }
    for (int i = 0; i <= S::kRing; ++i) tc5::mbar_init(&ctrl.masked[i], 1);
    for (int i = 0; i < S::kGroups; ++i) { tc5::mbar_init(&ctrl.xfull[i], p.x_by_map ? 1 : S::kWorkers); tc5::mbar_init(&ctrl.xempty[i], 1); }
    for (int i = 0; i < S::kAcc; ++i) { tc5::mbar_init(&ctrl.full_acc[i], 1); tc5::mbar_init(&ctrl.empty_acc[i], S::kReaders); }
    for (int i = 0; i < 16; ++i) tc5::mbar_init(&ctrl.y_full[i], 1);
    tc5::mbar_init(&ctrl.a_done, 1); tc5::mbar_init(&ctrl.ready, 1); tc5::mbar_init(&ctrl.drained, 1);
    ctrl.abort_flag = ctrl.asked = ctrl.x_asked = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\nfence.proxy.async.shared::cta;" ::: "memory");
  }
  if (tid == S::kWork) {          // the maps themselves are fetched from memory, too
    auto fetch = [](const CUtensorMap* m) { asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory"); };
    fetch(&p.A[(a.rank + 15) / 16 - 1]);
    fetch(&p.B);
    if (p.x_by_map) fetch(&p.X);
  }
  // a cluster is 1, 2, 4 or 8 blocks, and at most 128 blocks divide at most 2^17 tiles of B
  const int logC = 31 - __clz(C), id = (int)(blockIdx.x >> logC), item = (int)((unsigned)id / (unsigned)p.splits), split = id - item * p.splits;
  const int pieces = (a.ic + 63) / 64, k0 = pieces * c >> logC, np = (pieces * (c + 1) >> logC) - k0;
  const unsigned tiles = (unsigned)(a.oc + 127) / 128, parts = (unsigned)(C * p.splits), at = (unsigned)(split * C + c);
  const int o0 = (int)(tiles * at / parts), o1 = (int)(tiles * (at + 1) / parts);
  const bool grouped = NT == kRows && single_rows(a);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // the codebook is on its way while the rows are looked for, and goes to shared memory when x is asked for
  const uint32_t entry = p.mu && tid < p.mu_entries ? p.mu_codebook[tid] : 0;
  find_rows<NT>(p, item, t, scratch, share);
  const int n = t.n;
  const uint32_t ring = smem_u32(smem), xring = smem_u32(xs), full = smem_u32(ctrl.full), empty = smem_u32(ctrl.empty), xfull = smem_u32(ctrl.xfull), xempty = smem_u32(ctrl.xempty);
  bool ok = true;
  auto wait = [&](uint32_t bar, uint32_t parity) { ok = ok && tc5::mbar_wait(bar, parity, abortp, p.status); };
  auto row_of = [&](int r) { return grouped ? t.rows[r] : t.first + r; };

  // What depends on the adapter, which one thread looks up while x is on its way; false where there is none: the same for all blocks of the cluster.
  int rank = 0, blocks = 0, wide = 0, a_slot = 1, n_a = 0;
  bool masks = false;
  constexpr int last_term = kHalf ? 1 : 2;
  auto settle = [&] {
    wait(smem_u32(&ctrl.ready), 0);
    if (!t.counts) return false;
    rank = t.rank; blocks = (rank + 15) / 16; wide = (rank + 63) / 64;
    a_slot = pieces_of(blocks); n_a = (np + a_slot - 1) / a_slot;          // pieces of A in a slot, and slots
    // What lies behind the adapter's rank may be anything: in B's last sixteen columns it is masked, unless these end the rows, where a box has zeros.
    masks = rank % 16 != 0 && rank < a.rank;
    return true;
  };

  // All groups of x in operand form, by the workers: the loads of two groups are on their way while one is made (into buffers that take turns, not moved: a move
  // waits for what it moves).  A thread has kN eights of columns of a group, one where the tile has few rows.
  auto stage_all = [&](auto mix, auto per) {
    constexpr bool kMix = decltype(mix)::value;
    constexpr int kN = decltype(per)::value;
    Turn<S::kGroups> turn;
    Eights<X> raw[2][kN];
    MuWords words[2];
    // kWork is a multiple of a row's eights: the columns are the same for all rows of a thread
    const int piece = tid % S::kEights / 8, groups = (np + S::kGroup - 1) / S::kGroup;
    auto col_of = [&](int g) { return (k0 + min(g * S::kGroup + piece, np - 1)) * 64 + (tid & 7) * 8; };
    RowOf<X> rows[kN];
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const int row = row_of(min((tid + j * S::kWork) / S::kEights, n - 1));
      rows[j] = row_at<X>(p, row, grouped ? row : t.seq, grouped || row == t.start);
    }
    auto load = [&](int g, Eights<X> (&e)[kN], MuWords& m) {
      const int col = col_of(g);
      m = load_mu<kMix>(p, col);
#pragma unroll
      for (int j = 0; j < kN; ++j) e[j] = load_eights<X, kMix>(p, rows[j], col);
    };
    load(0, raw[0], words[0]);
    load(1, raw[1], words[1]);
    if constexpr (kMix) {
      if (tid < p.mu_entries) codebook[tid] = entry;
      asm volatile("bar.sync 1, %0;" ::"n"(S::kWork) : "memory");
    }
    float by[kN];
    if constexpr (F::kScaled) {          // first the largest number of each row: all groups are read twice but the first two
      int top[kN] = {};
      auto look = [&](int g, const Eights<X> (&e)[kN], const MuWords& m) {
        float2 mu[4], f[4];
        mu_of<kMix>(p, codebook, m, col_of(g), mu);
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          mix_eights<X, kMix>(e[j], mu, f);
          top[j] = max(top[j], top_of(f));
        }
      };
#pragma unroll 1
      for (int g = 2; g < groups; ++g) {
        Eights<X> e[kN];
        MuWords m;
        load(g, e, m);
        look(g, e, m);
      }
      look(0, raw[0], words[0]);
      look(1, raw[1], words[1]);
      // the lanes of a row: all of a warp, or a half
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        int best = top[j];
#pragma unroll
        for (int o = 1; o < (S::kEights < 32 ? S::kEights : 32); o *= 2) best = max(best, __shfl_xor_sync(~0u, best, o));
        if (lane % S::kEights == 0) atomicMax(&ctrl.top[(tid + j * S::kWork) / S::kEights], best);
      }
      asm volatile("bar.sync 1, %0;" ::"n"(S::kWork) : "memory");
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        float back;
        powers_of(ctrl.top[(tid + j * S::kWork) / S::kEights], by[j], back);
      }
    }
#pragma unroll 1
    for (int g0 = 0; g0 < groups; g0 += 2)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int g = g0 + h;
        if (g >= groups) continue;
        if (g >= S::kGroups) {
          if (g == S::kGroups && !settle()) return;          // nothing is multiplied where there is no adapter
          wait(xempty + turn.at * 8u, turn.parity ^ 1u);
        }
        float2 mu[4];
        mu_of<kMix>(p, codebook, words[h], col_of(g), mu);
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          const int row = (tid + j * S::kWork) / S::kEights;
          if (j * S::kWork / S::kEights >= n) continue;          // of no thread
          if (row < n) put_eights<X, F, kMix>(raw[h][j], mu, xs + (turn.at * S::kGroup + piece) * S::kPieceBytes + swizzled(row, tid & 7), S::kTileBytes, F::kScaled ? by[j] : 1.f);
        }
        if (g + 2 < groups) load(g + 2, raw[h], words[h]);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) tc5::mbar_arrive(xfull + turn.at * 8u);
        turn.next();
      }
  };
  auto stage = [&] {
    const bool few = NT == kRows && n * S::kEights <= S::kWork;
    if (p.mu) {
      if (few) stage_all(std::true_type(), std::integral_constant<int, NT == kRows ? 1 : S::kPer>());
      else stage_all(std::true_type(), std::integral_constant<int, S::kPer>());
    } else {
      if (few) stage_all(std::false_type(), std::integral_constant<int, NT == kRows ? 1 : S::kPer>());
      else stage_all(std::false_type(), std::integral_constant<int, S::kPer>());
    }
  };
  if (warp == S::kWorkers) {
    // ---- copies
    int i = 0, px = 0, gx = 0;
    Turn<S::kRing> slot;
    Turn<S::kGroups> group;
    auto ask_x = [&](int upto) {
#pragma unroll 1
      for (; px < upto; px += S::kGroup, ++gx) {
        if (gx >= S::kGroups) wait(xempty + group.at * 8u, group.parity ^ 1u);
        if (!__all_sync(~0u, ok)) return;
        const uint32_t bar = xfull + group.at * 8u, to = xring + group.at * (S::kGroup * S::kPieceBytes);
        const int count = p.whole ? S::kGroup : min(S::kGroup, np - px);
        if (lane == 0) tc5::mbar_arrive_expect_tx(&ctrl.xfull[group.at], (uint32_t)(count * S::kTileBytes));
        __syncwarp();
        if (p.whole) tensor_g2s(to, &p.X, 0, t.first, k0 + px, bar);
        else
#pragma unroll 1
          for (int j = 0; j < count; ++j) tensor_g2s(to + (uint32_t)(j * S::kTileBytes), &p.X, (k0 + px + j) * 64, t.first, 0, bar);
        group.next();
      }
    };
    if (p.x_by_map && n > 0) ask_x(min(np, S::kGroup * S::kGroups));        // as much as there is room for, whatever the adapter
    if (!settle()) {
      for (int j = 0; j < gx; ++j) wait(xfull + (uint32_t)j * 8u, 0);
      return;
    }
    // This warp and those behind it bring nothing to the meetings of the cluster, arrive relaxed (with release it took 1000 cycles) and do not hold them up: what they wait for
    // below comes behind the first.
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int total = n_a + (o1 - o0) * wide;
    // Nor does this one hold up the second by waits for slots that B had, which are given back behind that.
    auto second = [] { asm volatile("barrier.cluster.wait.acquire.aligned;\nbarrier.cluster.arrive.relaxed.aligned;" ::: "memory"); };
    bool met = false;
    const CUtensorMap* const a_map = &p.A[blocks - 1];
    const uint32_t a_bytes = (uint32_t)(a_slot * blocks) * 2048u;
#pragma unroll 1
    for (; i < n_a; ++i) {
      const uint32_t bar = full + slot.at * 8u, dst = ring + slot.at * kSlotBytes;
      if (i >= S::kRing) wait(empty + slot.at * 8u, slot.parity ^ 1u);
      if (!__all_sync(~0u, ok)) break;
      const int first = i * a_slot, count = p.whole ? a_slot : min(a_slot, np - first);
      if (lane == 0) tc5::mbar_arrive_expect_tx(&ctrl.full[slot.at], p.whole ? a_bytes : (uint32_t)(count * blocks) * 2048u);
      __syncwarp();
      if (p.whole) tensor_g2s(dst, a_map, 0, 0, k0 + first, t.adapter, bar);
      else
#pragma unroll 1
        for (int j = 0; j < count; ++j) tensor_g2s(dst + (uint32_t)(j * blocks) * 2048u, a_map, (k0 + first + j) * 64, 0, t.adapter, bar);
      slot.next();
      if (p.x_by_map) ask_x(min(np, first + a_slot + S::kGroup));        // a group ahead
    }
#pragma unroll 1
    for (int tile = o0, k = 0; i < total; ++i) {
      if (i - S::kRing >= n_a && !met) { second(); met = true; }
      const uint32_t bar = full + slot.at * 8u;
      if (i >= S::kRing) wait(empty + slot.at * 8u, slot.parity ^ 1u);
      if (!__all_sync(~0u, ok)) break;
      if (lane == 0) tc5::mbar_arrive_expect_tx(&ctrl.full[slot.at], kSlotBytes);
      __syncwarp();
      tensor_g2s(ring + slot.at * kSlotBytes, &p.B, k * 64, tile * 128, t.adapter, bar);
      if (++k == wide) { k = 0; ++tile; }
      slot.next();
    }
    if (lane == 0) { ctrl.asked = i; ctrl.x_asked = gx; }
    __syncwarp();
    if (!met) second();
  } else if (warp == S::kWorkers + 1) {
    // ---- products
    tc5::tmem_alloc(&ctrl.tmem_base, S::kTmemCols);
    tc5::tc_fence_before();
    __syncwarp();
    const bool goes_on = settle();
    tc5::tc_fence_after();
    const uint32_t tmem = *static_cast<volatile uint32_t*>(&ctrl.tmem_base);
    if (!goes_on) {
      tc5::tmem_dealloc(tmem, S::kTmemCols);
      return;
    }
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const uint64_t ring_desc = tc5::smem_desc_sw128(ring), x_desc = tc5::smem_desc_sw128(xring);
    constexpr uint32_t kA = idesc_of(F::kHalf, S::kColsA);
    const uint32_t kB = idesc_of(kHalf, S::kBeside ? NT * (last_term + 1) : NT);
    Turn<S::kRing> slot;
    {
      Turn<S::kGroups> group;
      uint32_t in_group = 0;
#pragma unroll 1
      for (int i = 0, px = 0; i < n_a; ++i) {
        wait(full + slot.at * 8u, slot.parity);
        uint64_t w = ring_desc + (slot.at * kSlotBytes >> 4);
#pragma unroll 1
        for (int j = 0; j < a_slot && px < np; ++j, ++px) {
          if (in_group == 0) wait(xfull + group.at * 8u, group.parity);
          if (!__all_sync(~0u, ok)) break;
          tc5::tc_fence_after();
          const uint64_t x = x_desc + ((group.at * S::kGroup + in_group) * S::kPieceBytes >> 4);
#pragma unroll
          for (int k = S::kBeside ? 0 : F::kX - 1; k >= 0; --k) umma(tmem, w, x + (uint32_t)(k * S::kTileBytes / 16), kA, px > 0 || (!S::kBeside && k < F::kX - 1), 4);
          w += (uint32_t)blocks * 128u;
          if (++in_group == S::kGroup) {
            tc5::umma_commit(&ctrl.xempty[group.at]);
            group.next();
            in_group = 0;
          }
        }
        if (!__all_sync(~0u, ok)) break;
        tc5::umma_commit(&ctrl.empty[slot.at]);
        slot.next();
      }
    }
    if (__all_sync(~0u, ok)) tc5::umma_commit(&ctrl.a_done);
    // the second meeting: A x is there, from all blocks
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;\nbarrier.cluster.arrive.relaxed.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");
#pragma unroll 1
    for (int o = 0; o < o1 - o0; ++o) {
      const uint32_t acc = (uint32_t)(o % S::kAcc), d = tmem + S::kColsA + acc * S::kColsB;
      wait(smem_u32(&ctrl.empty_acc[acc]), (uint32_t)(o / S::kAcc + 1) & 1u);
#pragma unroll 1
      for (int k = 0; k < wide; ++k) {
        if (masks && k + 1 == wide) {
          wait(smem_u32(&ctrl.masked[o % (S::kRing + 1)]), (uint32_t)(o / (S::kRing + 1)) & 1u);
        } else {
          wait(full + slot.at * 8u, slot.parity);
        }
        if (!__all_sync(~0u, ok)) break;
        const int steps = min(4, blocks - k * 4);
        tc5::tc_fence_after();
        const uint64_t w = ring_desc + (slot.at * kSlotBytes >> 4), h = x_desc + (uint32_t)(k * (S::kBeside ? 3 : 1) * S::kTileBytes / 16);
#pragma unroll 1
        for (int j = S::kBeside ? 0 : last_term; j >= 0; --j) umma(d, w, h + (uint32_t)(j * wide * S::kTileBytes / 16), kB, k > 0 || (!S::kBeside && j < last_term), steps);
        tc5::umma_commit(&ctrl.empty[slot.at]);
        slot.next();
      }
      if (!__all_sync(~0u, ok)) break;
      tc5::umma_commit(&ctrl.full_acc[acc]);
    }
  } else if (warp > S::kWorkers + 1) {
    // One of two warps that have nothing to do yet looks up the adapter, the other has x fetched to the second-level cache, ahead of the weights, behind which a load takes
    // some 5000 cycles, and y's rows, which are read when all else is done; but for those that come through maps of their own (x and y of 2048 rows, bf16: 22.0 us with, 20.7 without).
    auto fetch = [](const void* base, long long at, int elements, int size) {
      if (elements > 0) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(static_cast<const uint8_t*>(base) + at * size), "r"(elements * size) : "memory");
    };
    if (warp == S::kWorkers + 2) {
      if (lane == 0) {
        find_adapter(p, t);
        tc5::mbar_arrive(&ctrl.ready);
      }
      __syncwarp();
    } else if (!p.x_by_map) {
      const int columns = min((k0 + np) * 64, a.ic) - k0 * 64;
      for (int r = lane; r < n; r += 32) {
        fetch(a.x, (long long)row_of(r) * a.x_row + k0 * 64, columns, (int)sizeof(X));
        if (a.x_prev) fetch(a.x_prev, (long long)row_of(r) * a.x_prev_row + k0 * 64, columns, (int)sizeof(X));
      }
    }
    if (!settle()) return;
    if (warp == S::kWorkers + 3 && (NT == kRows || a.y_dtype == RWKVQ_F32)) {
      for (int r = lane; r < n; r += 32) fetch(a.y, (long long)row_of(r) * a.y_row + o0 * 128, min(o1 * 128, a.oc) - o0 * 128, a.y_dtype == RWKVQ_F32 ? 4 : 2);
      __syncwarp();
    }
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;\nbarrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    // ---- masks, each of two warps for every second tile of B: no more tiles ahead of the products than the ring has slots
    if (masks)
#pragma unroll 1
      for (int o = warp - S::kWorkers - 2; o < o1 - o0; o += 2) {
        const int i = n_a + o * wide + wide - 1, tail = rank - (wide - 1) * 64;
        uint8_t* const weights = smem + i % S::kRing * kSlotBytes;
        wait(full + (uint32_t)(i % S::kRing) * 8u, (uint32_t)(i / S::kRing) & 1u);
        if (!__all_sync(~0u, ok)) break;
        uint4 v[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) v[h][r] = *reinterpret_cast<const uint4*>(weights + swizzled(r * 32 + lane, min(tail / 8 + h, 7)));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int e = tail / 8 + h, keep = max(tail - e * 8, 0);
          auto of = [keep](int j) { return keep >= 2 * j + 2 ? ~0u : keep == 2 * j + 1 ? 0xFFFFu : 0u; };
          if (e * 8 >= (tail + 15) / 16 * 16) continue;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            *reinterpret_cast<uint4*>(weights + swizzled(r * 32 + lane, e)) = make_uint4(v[h][r].x & of(0), v[h][r].y & of(1), v[h][r].z & of(2), v[h][r].w & of(3));
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) tc5::mbar_arrive(&ctrl.masked[o % (S::kRing + 1)]);
      }
  } else {
    if (!p.x_by_map && np > 0 && n > 0) stage();
    if (!settle()) return;
    // ---- this block's share of A x: lanes are the rank
    constexpr int kCols = NT * 4 / S::kWorkers;
    const int quarter = warp & 3, col0 = (warp >> 2) * kCols;
    wait(smem_u32(&ctrl.a_done), 0);
    tc5::tc_fence_after();
    const uint32_t lanes = *static_cast<volatile uint32_t*>(&ctrl.tmem_base) + ((uint32_t)quarter << 21);
    if (quarter * 32 < blocks * 16) {
      float sum[kCols];
#pragma unroll
      for (int j = 0; j < kCols; ++j) sum[j] = 0.f;
      if (np > 0)
#pragma unroll
        for (int k = (S::kBeside ? F::kX : 1) - 1; k >= 0; --k) {
          uint32_t v[kCols];
          tmem_ld<kCols>(lanes + (uint32_t)(k * NT + col0), v);
#pragma unroll
          for (int j = 0; j < kCols; ++j) sum[j] += __uint_as_float(v[j]);
        }
      if constexpr (F::kScaled) {
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
          float by, back;
          powers_of(ctrl.top[col0 + j], by, back);
          sum[j] *= back;
        }
      }
#pragma unroll
      for (int j = 0; j < kCols; ++j)
        if (col0 + j < n) share[(col0 + j) * kMostRank + quarter * 32 + lane] = sum[j];
    }
    tc5::tc_fence_before();
    cluster.sync();

    // ---- A x: each block adds up a share of the rows, and gives them to all as operands.  As many lanes to a row as there are fours of the rank
    const float scale = t.scale;
    auto add_up = [&](auto blocks_of_cluster) {
      constexpr int kC = decltype(blocks_of_cluster)::value;
      const int wl = blocks == 1 ? 4 : blocks == 2 ? 8 : blocks <= 4 ? 16 : 32, r4 = lane % wl * 4, row1 = n * (c + 1) / kC;
#pragma unroll 1
      for (int row0 = n * c / kC + warp * (32 / wl); row0 < row1; row0 += S::kWorkers * (32 / wl)) {
        const int row = row0 + lane / wl;
        const bool there = row < row1 && r4 < blocks * 16;
        float h[4] = {0.f, 0.f, 0.f, 0.f};
        float4 s[kC];
#pragma unroll
        for (int k = 0; k < kC; ++k) s[k] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(share, k) + min(row, n - 1) * kMostRank + r4);
#pragma unroll
        for (int k = 0; k < kC; ++k) { h[0] += s[k].x; h[1] += s[k].y; h[2] += s[k].z; h[3] += s[k].w; }
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] = r4 + j < rank ? h[j] * scale : 0.f;
        uint8_t* const to = xs + r4 / 64 * (S::kBeside ? 3 : 1) * S::kTileBytes + swizzled(row, r4 / 8 & 7) + (r4 & 4) * 2;
        const int next = (S::kBeside ? 1 : wide) * S::kTileBytes;
        uint2 terms[3];
        float back = 1.f;
        if constexpr (kHalf) {
          float top = fmaxf(fmaxf(fabsf(h[0]), fabsf(h[1])), fmaxf(fabsf(h[2]), fabsf(h[3])));
          for (int o = 1; o < wl; o *= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
          // 2^up brings the largest number to 2^14; an infinity or NaN stays what it is
          const int up = top > 0.f && top < INFINITY ? max(min(14 - ilogbf(top), 126), -126) : 0;
          const float by = __uint_as_float((uint32_t)(127 + up) << 23);
          back = __uint_as_float((uint32_t)(127 - up) << 23);
          __half hi[4], lo[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float x = h[j] * by;
            hi[j] = __float2half_rn(x);
            lo[j] = fabsf(x) < INFINITY ? __float2half_rn(x - __half2float(hi[j])) : __float2half_rn(0.f);
          }
          terms[0] = make_uint2(pair_bits(hi[0], hi[1]), pair_bits(hi[2], hi[3]));
          terms[1] = make_uint2(pair_bits(lo[0], lo[1]), pair_bits(lo[2], lo[3]));
        } else {
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            __nv_bfloat16 b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = term(h[j]);
            terms[k] = make_uint2(pair_bits(b[0], b[1]), pair_bits(b[2], b[3]));
          }
        }
        if (there)
#pragma unroll
          for (int k = 0; k < kC; ++k) {
            uint8_t* const there_to = cluster.map_shared_rank(to, k);
            *reinterpret_cast<uint2*>(there_to) = terms[0];
            *reinterpret_cast<uint2*>(there_to + next) = terms[1];
            if (!kHalf) *reinterpret_cast<uint2*>(there_to + 2 * next) = terms[2];
            if (kHalf && r4 == 0) *cluster.map_shared_rank(&ctrl.back[row], k) = back;
          }
      }
    };
    if (C == 8) add_up(std::integral_constant<int, 8>());
    else if (C == 4) add_up(std::integral_constant<int, 4>());
    else if (C == 2) add_up(std::integral_constant<int, 2>());
    else add_up(std::integral_constant<int, 1>());
    asm volatile("fence.proxy.async;" ::: "memory");
    // the second meeting, behind which no block touches another's memory
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");

    // ---- y
    if (a.y_dtype == RWKVQ_F32) reduce_y<S, kHalf>(p, t, ctrl, lanes + S::kColsA, o0, o1, n, grouped, share, last_term, ok);
    else if constexpr (NT == 64) {
      if (a.y_dtype == RWKVQ_F16) store_y_rows<S, __half, kHalf, last_term + 1>(p, t, ctrl, lanes + S::kColsA, o0, o1, n, share, ok);
      else store_y_rows<S, __nv_bfloat16, kHalf, last_term + 1>(p, t, ctrl, lanes + S::kColsA, o0, o1, n, share, ok);
    } else {
      if (a.y_dtype == RWKVQ_F16) store_y<S, __half, kHalf>(p, t, ctrl, lanes + S::kColsA, o0, o1, n, grouped, share, last_term, ok);
      else store_y<S, __nv_bfloat16, kHalf>(p, t, ctrl, lanes + S::kColsA, o0, o1, n, grouped, share, last_term, ok);
    }
  }
  if (warp == S::kWorkers || warp > S::kWorkers + 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  tc5::tc_fence_before();
  __syncthreads();
  tc5::tc_fence_after();
  if (ctrl.abort_flag) {
    // a block that gave up leaves when its copies have arrived and the tensor core is done
    auto arrived = [](uint32_t bar, uint32_t parity) {
      for (uint32_t k = 0; k < tc5::kPollLimit && !tc5::mbar_try_wait(bar, parity); ++k) {}
    };
    if (tid == 0) {
      for (int i = max(0, ctrl.asked - S::kRing); i < ctrl.asked; ++i) arrived(full + (uint32_t)(i % S::kRing) * 8u, (uint32_t)(i / S::kRing) & 1u);
      for (int i = max(0, ctrl.x_asked - S::kGroups); i < ctrl.x_asked; ++i) arrived(xfull + (uint32_t)(i % S::kGroups) * 8u, (uint32_t)(i / S::kGroups) & 1u);
    }
    if (warp == S::kWorkers + 1) {
      tc5::umma_commit(&ctrl.drained);
      arrived(smem_u32(&ctrl.drained), 0);
    }
    __syncthreads();
  }
  if (warp == S::kWorkers + 1) tc5::tmem_dealloc(ctrl.tmem_base, S::kTmemCols);
}

template <typename X, typename W, int NT>
cudaError_t opt_in_tile() {
  static SmemOptIn opt_in(kCarveOut);
  return opt_in((const void*)lowrank_tile_kernel<X, W, NT>, kSmemBytes);
}

// Clusters of C blocks that are on the device at once; asked for once per device and kernel.  What is asked for is answered with none as long as the kernel may not have its shared
// memory, so that is seen to first: how a call is cut, and with that the order of its sums, depends on the call and the device alone, not on the calls before.
template <typename X, typename W, int NT>
cudaError_t clusters_at_once(unsigned C, long long* n) {
  static std::atomic<int> known[kMaxDevices][4];          // and one more: 0 is not known
  const int dev = current_device(), h = C == 8 ? 3 : C == 4 ? 2 : C == 2 ? 1 : 0;
  int got = dev >= 0 ? known[dev][h].load(std::memory_order_relaxed) : 0;
  if (got > 0) { *n = got - 1; return cudaSuccess; }
  cudaError_t e = opt_in_tile<X, W, NT>();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(C); cfg.blockDim = dim3(TileShape<X, W, NT>::kAll); cfg.dynamicSmemBytes = kSmemBytes;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  e = cudaOccupancyMaxActiveClusters(&got, (const void*)lowrank_tile_kernel<X, W, NT>, &cfg);
  if (e != cudaSuccess) { cudaGetLastError(); return e; }
  got = std::max(got, 0);
  if (dev >= 0) known[dev][h].store(got + 1, std::memory_order_relaxed);
  *n = got;
  return cudaSuccess;
}

// One block an SM: clusters as wide as are there at once.  Wide clusters leave SMs over (132 of 148 can be in clusters of four, 120 in clusters of eight: what is behind them starts when
// all is done).
template <typename X, typename W, int NT>
cudaError_t width_of(long long items, unsigned* C) {
  for (*C = 8; *C > 1; *C /= 2) {
    long long at_once = 0;
    const cudaError_t e = clusters_at_once<X, W, NT>(*C, &at_once);
    if (e != cudaSuccess) return e;
    if (items <= at_once) break;
  }
  return cudaSuccess;
}

template <typename X, typename W, int NT>
cudaError_t launch_tile(Args& p, long long items, unsigned C, cudaStream_t s) {
  using S = TileShape<X, W, NT>;
  const rwkvq_lowrank_args& a = p.a;
  const bool half = a.w_dtype == RWKVQ_F16;
  const tc5::EncodeTiledFn fn = tc5::encode_tiled();
  if (!fn || !encode(&p.B, a.B, half, a.rank, a.oc, a.n_adapters, 128)) return cudaErrorUnknown;
  // Where columns are whole pieces of 64, a box has several of them one behind the other, as many as a slot holds of so many rows; else one.  Boxes for every sixteen of the rank
  // that an adapter may have.
  p.whole = a.ic % 64 == 0;
  const CUtensorMapDataType type = half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  auto map = [&](CUtensorMap* m, const void* at, cuuint64_t rows, cuuint64_t row, cuuint64_t n, cuuint32_t box_rows, cuuint32_t box_pieces) {
    const cuuint64_t pieces = (cuuint64_t)a.ic / 64, dims4[4] = {64, rows, pieces, n}, strides4[3] = {row * 2, 128, row * 2 * rows};
    const cuuint64_t dims3[3] = {(cuuint64_t)a.ic, rows, n}, strides3[2] = {row * 2, row * 2 * rows};
    const cuuint32_t box4[4] = {64, box_rows, box_pieces, 1}, box3[3] = {64, box_rows, 1}, step[4] = {1, 1, 1, 1};
    return fn(m, type, p.whole ? 4 : 3, const_cast<void*>(at), p.whole ? dims4 : dims3, p.whole ? strides4 : strides3, p.whole ? box4 : box3, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  const int most = (a.rank + 15) / 16;
  for (int blocks = a.ranks ? 1 : most; blocks <= most; ++blocks)
    if (!map(&p.A[blocks - 1], a.A, (cuuint64_t)a.rank, (cuuint64_t)a.ic, (cuuint64_t)a.n_adapters, 16u * (cuuint32_t)blocks, (cuuint32_t)pieces_of(blocks))) return cudaErrorUnknown;
  p.x_by_map = !p.mu && std::is_same<X, W>::value && !(NT == kRows && single_rows(a));
  if (p.x_by_map) {
    const cuuint64_t row = (cuuint64_t)(a.tokens > 1 ? a.x_row : a.ic);
    const cuuint64_t dims[3] = {p.whole ? 64 : (cuuint64_t)a.ic, (cuuint64_t)a.tokens, p.whole ? (cuuint64_t)a.ic / 64 : 1}, strides[2] = {row * 2, p.whole ? 128 : row * 2};
    const cuuint32_t box[3] = {64, NT, p.whole ? (cuuint32_t)S::kGroup : 1}, step[3] = {1, 1, 1};
    if (fn(&p.X, type, 3, const_cast<void*>(a.x), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return cudaErrorUnknown;
  }
  p.y_by_map = NT == 64;
  if (p.y_by_map) {
    const bool wide = a.y_dtype == RWKVQ_F32;
    const cuuint64_t dims[3] = {(cuuint64_t)a.oc, (cuuint64_t)a.tokens, 1}, row = (cuuint64_t)a.y_row * (wide ? 4 : 2), strides[2] = {row, row * (cuuint64_t)a.tokens};
    const cuuint32_t box[3] = {wide ? 32u : 64u, 16, 1}, step[3] = {1, 1, 1};
    if (fn(&p.Y, wide ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : a.y_dtype == RWKVQ_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, wide ? 2 : 3, a.y, dims, strides, box, step,
           CU_TENSOR_MAP_INTERLEAVE_NONE, wide ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return cudaErrorUnknown;
  }
  long long at_once = 0;
  cudaError_t e = opt_in_tile<X, W, NT>();
  if (e == cudaSuccess) e = clusters_at_once<X, W, NT>(C, &at_once);
  if (e != cudaSuccess) return e;
  // where all clusters are as wide as can be and SMs are left, several divide a tile's rows of B and each multiplies A x for itself
  p.splits = (int)std::max<long long>(1, std::min<long long>({at_once / items, (a.oc + 128ll * C - 1) / (128 * C), 16}));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(items * C * p.splits)); cfg.blockDim = dim3(S::kAll); cfg.dynamicSmemBytes = kSmemBytes; cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, lowrank_tile_kernel<X, W, NT>, p);
}
template <typename X, typename W>
cudaError_t launch_form(Args& p, cudaStream_t s) {
  const rwkvq_lowrank_args& a = p.a;
  if (single_rows(a)) {
    const long long items = most_tiles(a, kRows);
    unsigned C = 1;
    const cudaError_t e = width_of<X, W, kRows>(items, &C);
    return e != cudaSuccess ? e : launch_tile<X, W, kRows>(p, items, C, s);
  }
  // A tile takes its time by the width of its cluster, and one of 64 rows some 1.4 times that of one of sixteen (4096 x 4096, us, sixteen / 64: prompts of 203 rows 10.0 / 11.4, 448 13.7 / 11.8, 2048
  // 42 / 22.6; f16 and rank 128, forty sequences of ten rows 29 / 42, sixty 51 / 40, 96 52 / 73), so that the wider tiles are taken where they leave room for wider clusters, or for fewer rounds.
  struct Plan { long long items; unsigned C; double cost; };
  cudaError_t e = cudaSuccess;
  auto plan = [&](auto of_rows) {
    constexpr int rows = decltype(of_rows)::value;
    const long long items = most_tiles(a, rows), filled = a.tokens / rows;
    unsigned C = 1;
    if (e == cudaSuccess) e = width_of<X, W, rows>(items, &C);
    const long long tiles = a.seq_start ? std::min<long long>(items, std::max<long long>(a.n_seq, filled + a.n_seq / 2)) : items;          // as many as are to be expected
    return Plan{items, C, (double)((tiles * C + sm_count() - 1) / sm_count()) / C};
  };
  const Plan few = plan(std::integral_constant<int, kRows>()), many = plan(std::integral_constant<int, 64>());
  if (e != cudaSuccess) return e;
  if (1.4 * many.cost < few.cost) return launch_tile<X, W, 64>(p, many.items, many.C, s);
  return launch_tile<X, W, kRows>(p, few.items, few.C, s);
}

template <typename W>
cudaError_t launch_x(Args& p, cudaStream_t s) {
  return p.a.x_dtype == RWKVQ_F32 ? launch_form<float, W>(p, s) : p.a.x_dtype == RWKVQ_F16 ? launch_form<__half, W>(p, s) : launch_form<__nv_bfloat16, W>(p, s);
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
  if (!mu_image != !mu_desc || ((a.x_prev || a.xprev0) && !mu_image) || (a.x_prev && a.xprev0)) return RWKVQ_EINVAL;
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
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  return cuda_status(a.w_dtype == RWKVQ_F16 ? lr::launch_x<__half>(p, s) : lr::launch_x<__nv_bfloat16>(p, s));
}

}  // extern "C"
