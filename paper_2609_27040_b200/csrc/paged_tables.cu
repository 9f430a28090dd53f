// paged_tables.cu — the bookkeeping half of the device-driven path: block tables and slot maps built on
// the GPU from request lengths (build_tables_kernel) and the scatter of new K/V rows through such a slot
// map (write_kv_kernel).
//
// build_tables_kernel. With T tokens per block, request i going from a to b tokens needs
// max(0, ceil(b/T) - ceil(a/T)) blocks; the k-th block needed (request order, then logical order) is the
// k-th id popped: ids0[free0 - 1 - k], and once the first stack is empty ids1[free1 - 1 - (k - free0)],
// whose table entry is the complement. New token t of the batch belongs to the request with
// offsets[i] <= t < offsets[i + 1], at position a + t - offsets[i]. Both prefix sums are over the
// requests, a few KB: every CTA computes them for itself (no CTA waits for another one) and fills its
// share of the token slots; the thread that fills the first token of a new block writes the block's table
// entry. Only the stacks' new tops and the blocks that shrinking requests give back must wait until every
// CTA has read the old ones: the CTA that draws the last ticket does both.
// Bound by latency: launch, one read of the lengths, the block-wide scan, one read of a table or
// stack entry, the stores. One new token for each of 256 requests: 3.9 us a launch back to back; 550 000 new tokens of
// 1000 requests: 8.3 us (6.9 MB to write, 1.1 us at the copy rate; each CTA fills two steps of 2048). What finishing requests give
// back is that one CTA's work, 512 blocks at a time, 1.3 us each (two barriers, and reads of lengths and cells that depend on one another):
// of 256 requests of 4091 tokens in blocks of 16, 4 finish: 6.5 us; 64 (16384 blocks): 46 us; all (65536): 174 us.
#include "kernels.h"
#include "ptx.cuh"

namespace ema {

namespace {

constexpr uint32_t kBuildThreads = 512;
constexpr uint32_t kBuildWarps = kBuildThreads / 32;
constexpr uint32_t kPerThread = 4;               // token slots of a thread at a time
constexpr uint32_t kBuildTokens = kBuildThreads * kPerThread;  // and of the CTA; at most that many requests have tokens in them
constexpr int64_t kNoSlot = INT64_MIN;

struct Sums {
  long long add, need, gone;  // tokens, blocks popped, blocks given back
};

__device__ __forceinline__ Sums plus(const Sums& a, const Sums& b) { return {a.add + b.add, a.need + b.need, a.gone + b.gone}; }

__device__ __forceinline__ Sums shfl_up(const Sums& a, int d) {
  return {__shfl_up_sync(0xffffffffu, a.add, d), __shfl_up_sync(0xffffffffu, a.need, d), __shfl_up_sync(0xffffffffu, a.gone, d)};
}

// Exclusive prefix of v over the CTA's threads, and the total.
__device__ Sums block_exclusive(const Sums& v, Sums* warp_sums, Sums& total) {
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  Sums inc = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const Sums o = shfl_up(inc, d);
    if (lane >= static_cast<uint32_t>(d)) inc = plus(inc, o);
  }
  __syncthreads();  // the array may still be read from an earlier call
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  Sums before = {0, 0, 0}, all = {0, 0, 0};
#pragma unroll
  for (uint32_t w = 0; w < kBuildWarps; ++w) {
    if (w == warp) before = all;
    all = plus(all, warp_sums[w]);
  }
  total = all;
  return {before.add + inc.add - v.add, before.need + inc.need - v.need, before.gone + inc.gone - v.gone};
}

__device__ uint32_t block_exclusive_u32(uint32_t v, uint32_t* warp_sums, uint32_t& total) {
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  uint32_t inc = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, inc, d);
    if (lane >= static_cast<uint32_t>(d)) inc += o;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (uint32_t w = 0; w < kBuildWarps; ++w) {
    if (w == warp) before = all;
    all += warp_sums[w];
  }
  total = all;
  return before + inc - v;
}

__device__ __forceinline__ uint32_t blocks_of(int32_t tokens, uint32_t shift) {
  return (static_cast<uint32_t>(tokens) + (1u << shift) - 1) >> shift;
}

__device__ __forceinline__ Sums sums_of(int32_t a, int32_t b, uint32_t shift) {
  const uint32_t ob = blocks_of(a, shift), nb = blocks_of(b, shift);
  return {b > a ? b - a : 0, nb > ob ? static_cast<long long>(nb - ob) : 0, ob > nb ? static_cast<long long>(ob - nb) : 0};
}

// A request whose new tokens may be among those of the CTA's step.
struct Entry {
  uint32_t seq, offset, first;  // batch position, its first new token, its first popped block
  int32_t old_len;
};

// Token slots [lo, hi), kPer of them to a thread: `list` has the requests around them, in order.
template <uint32_t kPer>
__device__ __forceinline__ void fill(const BuildTablesParams& p, const Entry* list, uint32_t entries, uint32_t lo, uint32_t hi,
                                     uint32_t tokens, int32_t free0, int32_t free1) {
  const uint32_t tid = threadIdx.x, shift = p.block_shift, mask = (1u << shift) - 1;
  // A thread's tokens together, so that their searches and their table or stack reads overlap (one after the other the reads,
  // 0.7 us each, were most of the time: 550 000 new tokens of 1000 requests took 10.3 us).
  uint32_t found[kPer];
#pragma unroll
  for (uint32_t i = 0; i < kPer; ++i) found[i] = 0;  // the last entry whose offset is <= t
  for (uint32_t step = entries > 1 ? 1u << (31 - __clz(entries - 1)) : 0; step; step >>= 1)
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) {
      const uint32_t next = found[i] + step;
      if (next < entries && list[next].offset <= lo + tid + i * kBuildThreads) found[i] = next;
    }
  int32_t pos[kPer], entry[kPer];
  const int32_t* from[kPer];
  int32_t* to[kPer];
  bool second[kPer];
#pragma unroll
  for (uint32_t i = 0; i < kPer; ++i) {
    const uint32_t t = lo + tid + i * kBuildThreads;
    from[i] = nullptr;
    to[i] = nullptr;
    pos[i] = -1;
    second[i] = false;
    if (t >= hi || t >= tokens) continue;
    const Entry en = list[found[i]];
    pos[i] = en.old_len + static_cast<int32_t>(t - en.offset);
    const uint32_t block = static_cast<uint32_t>(pos[i]) >> shift, held = blocks_of(en.old_len, shift);
    int32_t* cell = p.tables + static_cast<uint64_t>(en.seq) * p.table_stride + block;
    from[i] = cell;
    if (block >= held) {
      const uint32_t k = en.first + block - held;
      second[i] = k >= static_cast<uint32_t>(free0);
      from[i] = second[i] ? p.ids[1] + (free1 - 1 - (k - static_cast<uint32_t>(free0))) : p.ids[0] + (free0 - 1 - k);
      if ((static_cast<uint32_t>(pos[i]) & mask) == 0) to[i] = cell;
    }
  }
#pragma unroll
  for (uint32_t i = 0; i < kPer; ++i) entry[i] = from[i] ? *from[i] : 0;
#pragma unroll
  for (uint32_t i = 0; i < kPer; ++i) {
    const uint32_t t = lo + tid + i * kBuildThreads;
    if (t >= hi) continue;
    int64_t slot = kNoSlot;
    if (from[i]) {
      const int32_t e = second[i] ? ~entry[i] : entry[i];
      if (to[i]) *to[i] = e;
      const uint32_t row = static_cast<uint32_t>(pos[i]) & mask;
      slot = e >= 0 ? (static_cast<int64_t>(e) << shift) + row : ~((static_cast<int64_t>(~e) << shift) + row);
    }
    p.slots[t] = slot;
    p.positions[t] = pos[i];
  }
}

__global__ void __launch_bounds__(kBuildThreads, 1) build_tables_kernel(const BuildTablesParams p) {
  __shared__ Sums warp_sums[kBuildWarps];
  __shared__ uint32_t warp_u32[kBuildWarps];
  __shared__ Entry list[kBuildTokens];
  __shared__ uint32_t last_cta;
  __shared__ uint32_t gone_after[kBuildThreads];
  const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5;
  const uint32_t shift = p.block_shift;

  ptx::launch_dependents();
  ptx::grid_dependency_wait();

  // Every thread owns a run of requests.
  const uint32_t run = (p.nseq + kBuildThreads - 1) / kBuildThreads;
  const uint32_t r0 = min(tid * run, p.nseq), r1 = min(r0 + run, p.nseq);
  const long long room = static_cast<long long>(p.max_blocks) << shift;
  const int32_t free0 = p.free_in[0], free1 = p.free_in[1];
  Sums mine = {0, 0, 0};
  bool bad = free0 < 0 || free1 < 0 || static_cast<uint32_t>(free0) > p.capacity[0] || static_cast<uint32_t>(free1) > p.capacity[1];
  for (uint32_t i = r0; i < r1; ++i) {
    const int32_t a = p.lens[i], b = p.new_lens[i];
    if (a < 0 || b < 0 || a > room || b > room)
      bad = true;
    else
      mine = plus(mine, sums_of(a, b, shift));
  }
  bad = __syncthreads_or(bad);
  Sums total;
  const Sums before = block_exclusive(mine, warp_sums, total);
  int code = 0;
  if (bad || total.add > static_cast<long long>(p.max_tokens))
    code = kStatusInvalid;
  else if (total.need > static_cast<long long>(free0) + free1)
    code = kStatusNoSpace;
  const uint32_t tokens = code ? 0 : static_cast<uint32_t>(total.add);

  if (blockIdx.x == 0) {
    uint32_t at = code ? 0 : static_cast<uint32_t>(before.add);
    for (uint32_t i = r0; i < r1; ++i) {
      p.offsets[i] = static_cast<int32_t>(at);
      if (!code) at += static_cast<uint32_t>(sums_of(p.lens[i], p.new_lens[i], shift).add);
    }
    if (tid == 0) {
      p.offsets[p.nseq] = static_cast<int32_t>(tokens);
      if (code) ptx::report_status(p.status, code);
    }
  }

  // One CTA alone lists all requests, if they are few enough (one without new tokens has the next one's offset and is passed
  // over by the search for the last entry), which saves it a scan; else a step lists those with tokens in it.
  const bool all = p.nseq <= kBuildTokens && gridDim.x == 1;
  if (all && tokens) {
    Sums at = before;
    for (uint32_t i = r0; i < r1; ++i) {
      const int32_t a = p.lens[i];
      list[i] = {i, static_cast<uint32_t>(at.add), static_cast<uint32_t>(at.need), a};
      at = plus(at, sums_of(a, p.new_lens[i], shift));
    }
    __syncthreads();
  }
  for (uint64_t t0 = static_cast<uint64_t>(blockIdx.x) * kBuildTokens; t0 < p.max_tokens; t0 += static_cast<uint64_t>(gridDim.x) * kBuildTokens) {
    const uint32_t lo = static_cast<uint32_t>(t0), hi = min(lo + kBuildTokens, p.max_tokens);
    uint32_t entries = all ? p.nseq : 0;
    if (lo < tokens && !all) {
      // The requests with tokens in [lo, hi), in order.
      uint32_t count = 0;
      Sums at = before;
      const bool near = before.add < hi && before.add + mine.add > lo;
      if (near)
        for (uint32_t i = r0; i < r1; ++i) {
          const Sums s = sums_of(p.lens[i], p.new_lens[i], shift);
          count += s.add > 0 && at.add < hi && at.add + s.add > lo;
          at = plus(at, s);
        }
      uint32_t slot = block_exclusive_u32(count, warp_u32, entries);
      if (count) {
        at = before;
        for (uint32_t i = r0; i < r1; ++i) {
          const int32_t a = p.lens[i];
          const Sums s = sums_of(a, p.new_lens[i], shift);
          if (s.add > 0 && at.add < hi && at.add + s.add > lo)
            list[slot++] = {i, static_cast<uint32_t>(at.add), static_cast<uint32_t>(at.need), a};
          at = plus(at, s);
        }
      }
      __syncthreads();
    }
    if (hi - lo <= 2 * kBuildThreads)  // short code: on a small batch the kernel's time is that of its cold instructions
      for (uint32_t x = lo; x < hi; x += kBuildThreads) fill<1>(p, list, entries, x, min(x + kBuildThreads, hi), tokens, free0, free1);
    else
      fill<kPerThread>(p, list, entries, lo, hi, tokens, free0, free1);
    if (!all) __syncthreads();  // the list is filled again
  }

  // The rest happens once, after every CTA has read the stacks and their tops; at once where nothing that is read is
  // written: no blocks come back, and the new tops go elsewhere.
  if (gridDim.x > 1 && (code || total.gone == 0) && p.free_out != p.free_in) {
    if (blockIdx.x) return;
  } else if (gridDim.x > 1) {
    __threadfence();
    __syncthreads();
    if (tid == 0) last_cta = atomicAdd(p.work, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last_cta) return;
    __threadfence();
    if (tid == 0) *p.work = 0;
  } else {
    __syncthreads();
  }
  const int32_t popped0 = code ? 0 : static_cast<int32_t>(min(total.need, static_cast<long long>(free0)));
  const int32_t popped1 = code ? 0 : static_cast<int32_t>(total.need) - popped0;
  const uint32_t top0 = static_cast<uint32_t>(free0 - popped0), top1 = static_cast<uint32_t>(free1 - popped1);
  uint32_t given0 = 0, given1 = 0;
  if (!code && total.gone > 0) {
    // Blocks given back, requests and logical blocks in descending order: number f of that order
    // belongs to the thread run that has gone_after <= f, and there to the request found by walking down.
    const uint32_t gone = static_cast<uint32_t>(total.gone);
    gone_after[tid] = static_cast<uint32_t>(total.gone - before.gone - mine.gone);
    __syncthreads();
    for (uint32_t f0 = 0; f0 < gone; f0 += kBuildThreads) {
      const uint32_t f = f0 + tid;
      int32_t e = 0;
      const bool on = f < gone;
      if (on) {
        uint32_t b = 0, n = kBuildThreads;  // gone_after falls with the thread: the first run whose value is <= f
        while (n > 0) {
          const uint32_t half = n >> 1;
          if (gone_after[b + half] > f) {
            b += half + 1;
            n -= half + 1;
          } else {
            n = half;
          }
        }
        uint32_t left = f - gone_after[b];
        const uint32_t s0 = min(b * run, p.nseq);
        uint32_t i = min(s0 + run, p.nseq);
        while (i > s0) {
          --i;
          const int32_t a = p.lens[i];
          const uint32_t g = static_cast<uint32_t>(sums_of(a, p.new_lens[i], shift).gone);
          if (left < g) {
            e = p.tables[static_cast<uint64_t>(i) * p.table_stride + blocks_of(a, shift) - 1 - left];
            break;
          }
          left -= g;
        }
      }
      const bool first = on && e >= 0, second = on && e < 0;
      const uint32_t m0 = __ballot_sync(0xffffffffu, first), m1 = __ballot_sync(0xffffffffu, second);
      __syncthreads();
      if (lane == 0) warp_u32[warp] = __popc(m0) | (__popc(m1) << 16);
      __syncthreads();
      uint32_t rank0 = given0, rank1 = given1;
      for (uint32_t w = 0; w < kBuildWarps; ++w) {
        const uint32_t c = warp_u32[w];
        if (w < warp) {
          rank0 += c & 0xffffu;
          rank1 += c >> 16;
        }
        given0 += c & 0xffffu;
        given1 += c >> 16;
      }
      const uint32_t below = (1u << lane) - 1;
      if (first) {
        const uint64_t at = static_cast<uint64_t>(top0) + rank0 + __popc(m0 & below);
        if (at < p.capacity[0])
          p.ids[0][at] = e;
        else
          ptx::report_status(p.status, kStatusInvalid);
      }
      if (second) {
        const uint64_t at = static_cast<uint64_t>(top1) + rank1 + __popc(m1 & below);
        if (at < p.capacity[1])
          p.ids[1][at] = ~e;
        else
          ptx::report_status(p.status, kStatusInvalid);
      }
    }
  }
  if (tid == 0) {
    const uint64_t n0 = static_cast<uint64_t>(top0) + given0, n1 = static_cast<uint64_t>(top1) + given1;
    p.free_out[0] = static_cast<int32_t>(code ? n0 : (n0 < p.capacity[0] ? n0 : p.capacity[0]));
    p.free_out[1] = static_cast<int32_t>(code ? n1 : (n1 < p.capacity[1] ? n1 : p.capacity[1]));
  }
}

// Scatter of rows. A row (all KV heads of one token, K or V) is `units` 16-byte units; unit u of block row
// r is stored at unit u ^ (r & 7) of its 128 bytes. `lanes` (8, 16 or 32) neighbouring threads take a
// token together. A thread has kRows * kUnits independent loads of K and as many of V in flight: four units of
// one token where rows are long enough, else one unit of each of four tokens. Bound by HBM: the rows are read
// and written once (131071 tokens of 8 heads of 128: 164 us, 6.55 TB/s, a plain copy's rate).
constexpr uint32_t kWriteThreads = 256;

template <uint32_t kRows, uint32_t kUnits>
__global__ void __launch_bounds__(kWriteThreads) write_kv_kernel(const WriteKvParams p) {
  ptx::launch_dependents();
  ptx::grid_dependency_wait();
  const uint32_t lanes = 1u << p.lane_shift;
  const uint32_t sub = threadIdx.x & (lanes - 1);
  const uint32_t groups = kWriteThreads >> p.lane_shift, group = threadIdx.x >> p.lane_shift;
  const uint64_t plane = static_cast<uint64_t>(p.row_bytes) << p.block_shift;
  const uint32_t row_mask = (1u << p.block_shift) - 1;
  const uint64_t t0 = static_cast<uint64_t>(blockIdx.x) * groups * kRows + group;
  uint8_t* dst[kRows];
  uint32_t swz[kRows];
  int64_t slots[kRows];
#pragma unroll
  for (uint32_t j = 0; j < kRows; ++j) {
    const uint64_t t = t0 + static_cast<uint64_t>(j) * groups;
    slots[j] = t < p.ntok ? p.slots[t] : kNoSlot;
  }
#pragma unroll
  for (uint32_t j = 0; j < kRows; ++j) {
    dst[j] = nullptr;
    swz[j] = 0;
    if (slots[j] == kNoSlot) continue;
    const bool second = slots[j] < 0;
    const uint64_t at = static_cast<uint64_t>(second ? ~slots[j] : slots[j]);
    const uint64_t id = at >> p.block_shift;
    if (id >= (second ? p.blocks[1] : p.blocks[0])) {
      if (sub == 0) ptx::report_status(p.status, kStatusInvalid);
      continue;
    }
    const uint32_t r = static_cast<uint32_t>(at) & row_mask;
    dst[j] = (second ? p.base[1] + id * p.block_stride[1] : p.base[0] + id * p.block_stride[0]) + static_cast<uint64_t>(r) * p.row_bytes;
    swz[j] = r & 7u;
  }
  for (uint32_t u0 = sub; u0 < p.units; u0 += lanes * kUnits) {
    uint4 k[kRows][kUnits], v[kRows][kUnits];
#pragma unroll
    for (uint32_t j = 0; j < kRows; ++j)
#pragma unroll
      for (uint32_t i = 0; i < kUnits; ++i) {
        const uint32_t u = u0 + i * lanes;
        if (dst[j] && u < p.units) {
          const uint64_t t = t0 + static_cast<uint64_t>(j) * groups;
          k[j][i] = ptx::ld_once_v4(p.k + t * p.k_stride + u * 16);
          v[j][i] = ptx::ld_once_v4(p.v + t * p.v_stride + u * 16);
        }
      }
#pragma unroll
    for (uint32_t j = 0; j < kRows; ++j)
#pragma unroll
      for (uint32_t i = 0; i < kUnits; ++i) {
        const uint32_t u = u0 + i * lanes;
        if (dst[j] && u < p.units) {
          uint8_t* d = dst[j] + ((u & ~7u) + ((u & 7u) ^ swz[j])) * 16;
          *reinterpret_cast<uint4*>(d) = k[j][i];
          *reinterpret_cast<uint4*>(d + plane) = v[j][i];
        }
      }
  }
}

}  // namespace

cudaError_t launch_build_tables(const BuildTablesParams& p, int num_sms, cudaStream_t stream) {
  const uint64_t steps = (static_cast<uint64_t>(p.max_tokens) + kBuildTokens - 1) / kBuildTokens;
  const uint64_t most = static_cast<uint64_t>(num_sms);
  const unsigned grid = static_cast<unsigned>(steps < 1 ? 1 : steps < most ? steps : most);
  return launch_early(build_tables_kernel, grid, kBuildThreads, 0, stream, p);
}

cudaError_t launch_write_kv(WriteKvParams p, cudaStream_t stream) {
  if (p.ntok == 0) return cudaSuccess;
  p.units = p.row_bytes / 16;
  p.lane_shift = p.units >= 32 ? 5 : p.units >= 16 ? 4 : 3;
  const bool wide = p.units >= 3u << p.lane_shift;  // most of four units to a thread
  const uint32_t per_cta = (kWriteThreads >> p.lane_shift) * (wide ? 1 : 4);
  const unsigned grid = static_cast<unsigned>((static_cast<uint64_t>(p.ntok) + per_cta - 1) / per_cta);
  return wide ? launch_early(write_kv_kernel<1, 4>, grid, kWriteThreads, 0, stream, p) : launch_early(write_kv_kernel<4, 1>, grid, kWriteThreads, 0, stream, p);
}

}  // namespace ema
