// States that follow their beams: state[slot of beam b] = state[slot of b's parent], in place, for every buffer that holds states.
//
// Nothing is computed; what has to be read is each slot that some other beam goes on from, once, and what has to be written each slot whose beam changes.
// A piece of `chunk` bytes of all beams of one request is one warp's, a block of its own: the sources' pieces are copied to shared memory, all of them, and from
// there to the slots that take them.  Pieces do not meet one another, so nothing is read behind a write of the same call and cycles need no care.
//
// HBM bounds it: 215 us, 5.7 TB/s, where four requests of eight beams have 805 MB of states (187 us at the rate of a plain copy).  Blocks take pieces in turn, all of them those of one request before
// the next one's, as requests differ in how many of their beams move (a range of pieces for each: 225 us).  One request, 17 MB: 7.5 us, of which 3.9 are the bytes'.
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/rwkvq.h"
#include "host_util.h"
#include "tc5.cuh"

namespace rwkvq {
int* device_status_ptr();  // api_misc.cu
namespace ro {

constexpr int kMostParts = 128, kMostBeams = 64;
constexpr uint32_t kBuffer = 16 << 10;          // bytes of shared memory for a block's pieces: thirteen blocks an SM (8 KB and 24 KB: no better; 32 KB: 8.4 where this takes 7.6, one request)
constexpr int kMostListed = 1 << 20;            // slots, where there is a list of them: a bit each in shared memory

struct Part { uint8_t* base; uint64_t row, bytes; };
struct Args {
  Part part[kMostParts];
  uint32_t first[kMostParts + 1];      // pieces before each part
  int n_parts, requests, beams, n_slots;
  uint32_t chunk;
  const int32_t* parents;
  const int32_t* slots;
  int* status;
};

__device__ __forceinline__ void bulk_s2g(void* dst, const void* src_smem, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(tc5::smem_u32(src_smem)), "r"(bytes) : "memory");
}

// A request's lists, beam `lane` and beam `lane + 32`: parents, slots, and which beams are copied to and from.
struct Request {
  int parent[2], slot[2];
  uint64_t sources;
  bool to[2], any;
  // Requests of one block in rising order.  A request moves nothing (and the status word is set) where a parent or slot does not exist or a slot is an earlier entry's, too: `seen` has a
  // bit for each slot of the entries before `upto`.
  __device__ __forceinline__ void take(const Args& a, int r, uint32_t* seen, int& upto) {
    const int lane = threadIdx.x & 31, K = a.beams, base = r * K;
    bool bad = false;
    if (a.slots)
      for (; upto < base; upto += 256) {
        int s[8];
#pragma unroll
        for (int h = 0; h < 8; ++h) s[h] = a.slots[min(upto + h * 32 + lane, base - 1)];          // some more than once
#pragma unroll
        for (int h = 0; h < 8; ++h)
          if ((unsigned)s[h] < (unsigned)a.n_slots) atomicOr(seen + (s[h] >> 5), 1u << (s[h] & 31));
      }
    upto = base + K;
    __syncwarp();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int b = lane + 32 * h;
      parent[h] = b < K ? a.parents[base + b] : 0;
      slot[h] = b < K ? (a.slots ? a.slots[base + b] : base + b) : -1;
      const bool there = (unsigned)slot[h] < (unsigned)a.n_slots;
      bad |= b < K && ((unsigned)parent[h] >= (unsigned)K || !there);
      if (a.slots && there) bad |= atomicOr(seen + (slot[h] >> 5), 1u << (slot[h] & 31)) >> (slot[h] & 31) & 1;
    }
    bad = __any_sync(~0u, bad);
    if (bad && lane == 0) atomicExch(a.status, (int)RWKVQ_EINVAL);
    uint64_t from = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      to[h] = !bad && lane + 32 * h < K && parent[h] != lane + 32 * h;
      if (to[h]) from |= 1ull << parent[h];
    }
    sources = (uint64_t)__reduce_or_sync(~0u, (uint32_t)(from >> 32)) << 32 | __reduce_or_sync(~0u, (uint32_t)from);
    any = sources != 0;
  }
};

__global__ void __launch_bounds__(32) state_reorder_kernel(const __grid_constant__ Args a) {
  extern __shared__ __align__(128) uint8_t buffer[];
  __shared__ __align__(8) uint64_t bar;
  __shared__ int gave_up;
  const int lane = threadIdx.x;
  if (lane == 0) {
    tc5::mbar_init(&bar, 1);
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  uint32_t* const seen = reinterpret_cast<uint32_t*>(buffer + (size_t)a.chunk * a.beams);
  if (a.slots)
    for (int k = lane; k < (a.n_slots + 31) / 32; k += 32) seen[k] = 0;
  __syncwarp();
  int upto = 0;
  const long long each = a.first[a.n_parts], all = each * a.requests;
  // One request after the other, by all blocks: requests differ in how many of their beams move.
  long long i = blockIdx.x;
  Request q;
  int r = -1;
  uint32_t parity = 0;
  while (i < all) {
    const int now = (int)(i / each);
    if (now != r) { r = now; q.take(a, r, seen, upto); }
    if (!q.any) { i += ((r + 1ll) * each - i + gridDim.x - 1) / gridDim.x * gridDim.x; continue; }
    const uint32_t c = (uint32_t)(i - r * each);
    int p = 0;
    for (int step = kMostParts / 2; step > 0; step /= 2)
      if (p + step < a.n_parts && a.first[p + step] <= c) p += step;
    const Part& part = a.part[p];
    const uint64_t at = (uint64_t)(c - a.first[p]) * a.chunk;
    const uint32_t bytes = (uint32_t)min((unsigned long long)a.chunk, (unsigned long long)(part.bytes - at));
    uint8_t* const base = part.base + at;
    if (lane == 0) tc5::mbar_arrive_expect_tx(&bar, (uint32_t)__popcll(q.sources) * bytes);
    __syncwarp();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint64_t bit = 1ull << (lane + 32 * h);
      if (q.sources & bit) tc5::bulk_g2s(buffer + (size_t)__popcll(q.sources & (bit - 1)) * a.chunk, base + (uint64_t)q.slot[h] * part.row, bytes, &bar);
    }
    if (!tc5::mbar_wait(&bar, parity, &gave_up, a.status)) {
      gave_up = 0;
      tc5::mbar_wait(&bar, parity, &gave_up, a.status);      // the copies write to this block's memory: not left before they are done
      break;
    }
    parity ^= 1;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (q.to[h]) bulk_s2g(base + (uint64_t)q.slot[h] * part.row, buffer + (size_t)__popcll(q.sources & ((1ull << q.parent[h]) - 1)) * a.chunk, bytes);
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
    i += gridDim.x;
  }
  asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

// Parts that share a byte would be gone over twice.  Sorted by their beginnings, neighbours that lie apart are told by one comparison; parts that lie between
// one another's slots (layers of one buffer) have the same distance from slot to slot and lie apart within it.
bool apart(const Part& x, const Part& y, int n_slots) {
  const uint64_t a = (uint64_t)x.base, b = (uint64_t)y.base, n = (uint64_t)n_slots - 1;
  if (a + n * x.row + x.bytes <= b || b + n * y.row + y.bytes <= a) return true;
  if (x.row != y.row) return false;
  const uint64_t d = (a < b ? b - a : a - b) % x.row;
  const Part &low = a < b ? x : y, &high = a < b ? y : x;
  return d >= low.bytes && d + high.bytes <= x.row;
}
bool all_apart(Part* p, int n, int n_slots) {
  std::sort(p, p + n, [](const Part& x, const Part& y) { return x.base < y.base; });
  for (int i = 0, known = 0; i < n; ++i) {
    int j = std::max(i + 1, known);      // those before `known` lie apart from one another
    // a run of parts within one distance of the same kind: neighbours, and the last against the first
    while (j < n && p[j].row == p[i].row && p[j].base + p[j].bytes <= p[i].base + p[i].row) {
      if (p[j - 1].base + p[j - 1].bytes > p[j].base) return false;
      ++j;
    }
    known = j;
    for (; j < n && (uint64_t)p[j].base < (uint64_t)p[i].base + (uint64_t)(n_slots - 1) * p[i].row + p[i].bytes; ++j)
      if (!apart(p[i], p[j], n_slots)) return false;
  }
  return true;
}

}  // namespace ro
}  // namespace rwkvq

using namespace rwkvq;

extern "C" {

rwkvq_status rwkvq_state_reorder(const rwkvq_state_part* parts, int n_parts, int n_slots, const int32_t* parents, const int32_t* slots, int requests,
                                 int beams, void* stream) {
  if (!parts || !parents || n_parts <= 0 || n_slots <= 0 || requests <= 0 || beams <= 0) return RWKVQ_EINVAL;
  if (beams > ro::kMostBeams || n_parts > RWKVQ_MOST_STATE_PARTS || (long long)requests * beams > (1 << 20)) return RWKVQ_EUNSUPPORTED;
  if (!slots && (long long)requests * beams > n_slots) return RWKVQ_EINVAL;
  if (slots && n_slots > ro::kMostListed) return RWKVQ_EUNSUPPORTED;
  ro::Part all[RWKVQ_MOST_STATE_PARTS];
  const uint32_t chunk = std::min<uint32_t>(ro::kBuffer / (uint32_t)beams / 128 * 128, 8192);
  for (int i = 0; i < n_parts; ++i) {
    const rwkvq_state_part& p = parts[i];
    if (!p.base || p.bytes == 0 || p.slot_row < p.bytes) return RWKVQ_EINVAL;
    if (!aligned16(p.base) || p.bytes % 16 || p.slot_row % 16) return RWKVQ_EALIGN;
    if (p.bytes / chunk >= (1u << 30) / ro::kMostParts || p.slot_row > (1ull << 47) / (uint64_t)n_slots) return RWKVQ_EUNSUPPORTED;
    all[i] = ro::Part{static_cast<uint8_t*>(p.base), p.slot_row, p.bytes};
  }
  if (!ro::all_apart(all, n_parts, n_slots)) return RWKVQ_EINVAL;
  ro::Args a;
  a.requests = requests; a.beams = beams; a.n_slots = n_slots; a.chunk = chunk; a.parents = parents; a.slots = slots;
  a.status = device_status_ptr();
  if (!a.status) return RWKVQ_ECUDA;
  const uint32_t bytes = chunk * (uint32_t)beams + (slots ? ((uint32_t)n_slots + 31) / 32 * 4 : 0);
  static SmemOptIn opt_in(kCarveOut);
  cudaError_t e = opt_in((const void*)ro::state_reorder_kernel, (int)ro::kBuffer + ro::kMostListed / 8);
  for (int at = 0; e == cudaSuccess && at < n_parts; at += ro::kMostParts) {
    a.n_parts = std::min(n_parts - at, ro::kMostParts);
    a.first[0] = 0;
    for (int i = 0; i < a.n_parts; ++i) {
      a.part[i] = all[at + i];
      a.first[i + 1] = a.first[i] + (uint32_t)((all[at + i].bytes + chunk - 1) / chunk);
    }
    const long long pieces = (long long)a.first[a.n_parts] * requests, most = (long long)sm_count() * std::max<uint32_t>(1, std::min<uint32_t>(32, (224u << 10) / (bytes + 1024)));
    const long long each = (pieces + most - 1) / most;          // as many pieces for every block
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((pieces + each - 1) / each)); cfg.blockDim = dim3(32); cfg.dynamicSmemBytes = bytes; cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, ro::state_reorder_kernel, a);
  }
  return cuda_status(e);
}

}  // extern "C"
