// paged_pages.cu — blocks that several requests hold, rows and blocks that move: forks of requests (fork_kernel), blocks given
// up by holders (free_kernel), blocks moved out of ids that are taken away (compact_plan_kernel, compact_cells_kernel),
// the copies that these ask for (copy_rows_kernel) and accepted rows of drafted tokens (keep_rows_kernel).
//
// refs[b] counts the requests that hold block b besides the first one, so that a block that nobody shares, just popped or on a
// stack, has 0, and calls that know nothing of sharing go on as they are.
//
// Nothing here waits for another CTA: what depends on all of a launch (the stacks, their tops) is done by the CTA that draws the
// last ticket. The orders of ids on the stacks do not depend on timing: pops go in the order of the forks, and what is freed or
// moved is collected as a bit per block first and then taken in the order of ids.
#include "kernels.h"
#include "ptx.cuh"

namespace ema {

namespace {

constexpr uint32_t kThreads = 512;
constexpr uint32_t kWarps = kThreads / 32;
constexpr uint32_t kCells = 128;                 // table cells that a warp takes at a time, four to a lane

__device__ __forceinline__ uint32_t blocks_of(int32_t tokens, uint32_t shift) {
  return (static_cast<uint32_t>(tokens) + (1u << shift) - 1) >> shift;
}

// Exclusive prefix of v over the CTA's threads, and the total.
__device__ uint32_t block_exclusive(uint32_t v, uint32_t* warp_sums, uint32_t& total) {
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  uint32_t inc = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, inc, d);
    if (lane >= static_cast<uint32_t>(d)) inc += o;
  }
  __syncthreads();  // the array may still be read from an earlier call
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (uint32_t w = 0; w < kWarps; ++w) {
    if (w == warp) before = all;
    all += warp_sums[w];
  }
  total = all;
  return before + inc - v;
}

// Whether this CTA is the last one to come here (its writes and everybody's are visible to it then); the word is left 0.
__device__ bool last_cta(uint32_t* word, uint32_t* flag) {
  if (gridDim.x > 1) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) *flag = atomicAdd(word, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!*flag) return false;
    __threadfence();
    if (threadIdx.x == 0) *word = 0;
  } else {
    __syncthreads();
  }
  return true;
}

__device__ __forceinline__ bool tops_bad(const PagesParams& p, const int32_t (&top)[2]) {
  return top[0] < 0 || top[1] < 0 || static_cast<uint32_t>(top[0]) > p.capacity[0] || static_cast<uint32_t>(top[1]) > p.capacity[1];
}

__device__ __forceinline__ bool length_bad(const PagesParams& p, int32_t n) {
  return n < 0 || static_cast<uint64_t>(n) > static_cast<uint64_t>(p.max_blocks) << p.block_shift;
}

// The arena of an entry, and the block's number in it; false where it has none.
__device__ __forceinline__ bool block_of(const PagesParams& p, int32_t e, uint32_t& a, uint32_t& id) {
  a = e < 0;
  id = static_cast<uint32_t>(a ? ~e : e);
  return id < (a ? p.blocks[1] : p.blocks[0]);
}

// Blocks that requests give up: lens[i] falls to new_lens[i]. Every cell takes a holder from its block; the cell that finds no other
// holder sets the block's bit. The last CTA pushes the blocks whose bits are set, the highest ids first.
// Bound by latency: lengths, cells, counts and bits one after the other, the ticket, the bits again.
__global__ void __launch_bounds__(kThreads, 1) free_kernel(const PagesParams p) {
  __shared__ uint32_t warp_sums[kWarps], flag;
  const uint32_t tid = threadIdx.x, lane = tid & 31u;
  ptx::launch_dependents();
  ptx::grid_dependency_wait();
  const int32_t top[2] = {p.free_in[0], p.free_in[1]};
  bool bad = tops_bad(p, top);
  for (uint32_t i = tid; i < p.nseq; i += kThreads) bad |= length_bad(p, p.lens[i]) || length_bad(p, p.new_lens[i]);
  bad = __syncthreads_or(bad);
  if (!bad) {
    const uint32_t pieces = (p.max_blocks + kCells - 1) / kCells;
    const uint64_t items = static_cast<uint64_t>(p.nseq) * pieces;
    for (uint64_t x = static_cast<uint64_t>(blockIdx.x) * kWarps + (tid >> 5); x < items; x += static_cast<uint64_t>(gridDim.x) * kWarps) {
      const uint32_t i = static_cast<uint32_t>(x / pieces), at = static_cast<uint32_t>(x % pieces) * kCells;
      const uint32_t first = blocks_of(p.new_lens[i], p.block_shift), end = blocks_of(p.lens[i], p.block_shift);
      if (at >= end || at + kCells <= first) continue;
      int32_t e[kCells / 32];
      bool on[kCells / 32];
#pragma unroll
      for (uint32_t k = 0; k < kCells / 32; ++k) {
        const uint32_t j = at + k * 32 + lane;
        on[k] = j >= first && j < end;
        e[k] = on[k] ? p.tables[i * p.table_stride + j] : 0;
      }
      int32_t left[kCells / 32];
      uint32_t a[kCells / 32], id[kCells / 32];
#pragma unroll
      for (uint32_t k = 0; k < kCells / 32; ++k) {
        left[k] = 1;
        if (on[k] && !block_of(p, e[k], a[k], id[k])) {
          ptx::report_status(p.status, kStatusInvalid);
          on[k] = false;
        }
        if (on[k]) left[k] = atomicSub(p.refs[a[k]] + id[k], 1);
      }
#pragma unroll
      for (uint32_t k = 0; k < kCells / 32; ++k) {
        if (!on[k]) continue;
        if (left[k] == 0) atomicOr(p.bits[a[k]] + (id[k] >> 5), 1u << (id[k] & 31u));
        if (left[k] < 0) ptx::report_status(p.status, kStatusInvalid);  // more cells than holders; the count is put right below
      }
    }
  }
  if (!last_cta(p.work, &flag)) return;
  if (bad) {
    if (tid == 0) {
      ptx::report_status(p.status, kStatusInvalid);
      p.free_out[0] = top[0];
      p.free_out[1] = top[1];
    }
    return;
  }
  for (uint32_t a = 0; a < 2; ++a) {
    const uint32_t words = (p.blocks[a] + 31) / 32, run = (words + kThreads - 1) / kThreads;
    const uint32_t end = words - min(tid * run, words), begin = words - min(tid * run + run, words);  // the first thread has the highest ids
    uint32_t count = 0, freed;
    for (uint32_t w = begin; w < end; ++w) count += __popc(__ldcg(p.bits[a] + w));
    uint64_t at = static_cast<uint64_t>(top[a]) + block_exclusive(count, warp_sums, freed);
    for (uint32_t w = end; count && w-- > begin;) {
      uint32_t bits = __ldcg(p.bits[a] + w);
      if (!bits) continue;
      p.bits[a][w] = 0;
      for (; bits; bits &= ~(1u << (31 - __clz(bits)))) {
        const uint32_t id = w * 32 + 31 - __clz(bits);
        p.refs[a][id] = 0;
        if (at < p.capacity[a])
          p.ids[a][at] = static_cast<int32_t>(id);
        else
          ptx::report_status(p.status, kStatusInvalid);
        ++at;
      }
    }
    if (tid == 0) p.free_out[a] = static_cast<int32_t>(min(static_cast<uint64_t>(top[a]) + freed, static_cast<uint64_t>(p.capacity[a])));
  }
}

// Forks: request dst[f] gets what src[f] holds. Whole blocks are shared (their cells copied, a holder added); of a last block that
// is not full, popped in the order of the forks, the copy is asked for. Every CTA looks at all forks before anything is
// written; the last one writes what the others read (lengths, tops).
__global__ void __launch_bounds__(kThreads, 1) fork_kernel(const PagesParams p) {
  extern __shared__ uint32_t taken[];              // a bit per request: it is some fork's dst
  __shared__ uint32_t warp_sums[kWarps], flag;
  const uint32_t tid = threadIdx.x, lane = tid & 31u;
  ptx::launch_dependents();
  for (uint32_t w = tid; w < (p.nseq + 31) / 32; w += kThreads) taken[w] = 0;
  __syncthreads();
  ptx::grid_dependency_wait();
  const int32_t top[2] = {p.free_in[0], p.free_in[1]};
  bool bad = tops_bad(p, top);
  const uint32_t mask = (1u << p.block_shift) - 1;
  const uint32_t run = (p.nfork + kThreads - 1) / kThreads, f0 = min(tid * run, p.nfork), f1 = min(f0 + run, p.nfork);
  uint32_t tails = 0;
  for (uint32_t i = tid; i < p.nseq; i += kThreads) bad |= length_bad(p, p.lens[i]);
  for (uint32_t f = f0; f < f1; ++f) {
    const int32_t s = p.src[f], d = p.dst[f];
    if (d < 0) continue;
    if (s < 0 || static_cast<uint32_t>(s) >= p.nseq || static_cast<uint32_t>(d) >= p.nseq) {
      bad = true;
      continue;
    }
    const int32_t n = p.lens[s];
    bad |= p.lens[d] != 0 || (atomicOr(taken + (d >> 5), 1u << (d & 31)) >> (d & 31) & 1u);
    tails += (static_cast<uint32_t>(n) & mask) != 0;
  }
  bad = __syncthreads_or(bad);
  for (uint32_t f = f0; f < f1 && !bad; ++f)       // a source that is another fork's dst: what it holds would depend on which comes first
    bad = p.dst[f] >= 0 && (taken[p.src[f] >> 5] >> (p.src[f] & 31) & 1u);
  bad = __syncthreads_or(bad);
  uint32_t need;
  uint32_t k = block_exclusive(tails, warp_sums, need);
  const int code = bad ? kStatusInvalid : need > static_cast<uint64_t>(top[0]) + top[1] ? kStatusNoSpace : 0;
  if (!code) {
    const uint32_t pieces = (p.max_blocks + kCells - 1) / kCells;
    const uint64_t items = static_cast<uint64_t>(p.nfork) * pieces;
    for (uint64_t x = static_cast<uint64_t>(blockIdx.x) * kWarps + (tid >> 5); x < items; x += static_cast<uint64_t>(gridDim.x) * kWarps) {
      const uint32_t f = static_cast<uint32_t>(x / pieces), at = static_cast<uint32_t>(x % pieces) * kCells;
      const int32_t s = p.src[f], d = p.dst[f];
      if (d < 0) continue;
      const uint32_t whole = static_cast<uint32_t>(p.lens[s]) >> p.block_shift;
      if (at >= whole) continue;
      int32_t e[kCells / 32];
#pragma unroll
      for (uint32_t c = 0; c < kCells / 32; ++c) {
        const uint32_t j = at + c * 32 + lane;
        e[c] = j < whole ? p.tables[s * p.table_stride + j] : 0;
      }
#pragma unroll
      for (uint32_t c = 0; c < kCells / 32; ++c) {
        const uint32_t j = at + c * 32 + lane;
        if (j >= whole) continue;
        uint32_t a, id;
        p.tables[d * p.table_stride + j] = e[c];
        if (block_of(p, e[c], a, id))
          atomicAdd(p.refs[a] + id, 1);
        else
          ptx::report_status(p.status, kStatusInvalid);
      }
    }
  }
  if (!last_cta(p.work, &flag)) return;
  for (uint32_t f = f0; f < f1; ++f) {
    int32_t from = 0, to = 0, rows = 0;
    const int32_t d = p.dst[f];
    if (!code && d >= 0) {
      const int32_t s = p.src[f], n = p.lens[s];
      rows = static_cast<int32_t>(static_cast<uint32_t>(n) & mask);
      if (rows) {
        const uint32_t j = static_cast<uint32_t>(n) >> p.block_shift;
        to = k < static_cast<uint32_t>(top[0]) ? p.ids[0][top[0] - 1 - k] : ~p.ids[1][top[1] - 1 - (k - top[0])];
        from = p.tables[s * p.table_stride + j];
        p.tables[d * p.table_stride + j] = to;
        ++k;
      }
      p.new_lens_out[d] = n;  // no source's length
    }
    p.copies[3 * static_cast<uint64_t>(f)] = from;
    p.copies[3 * static_cast<uint64_t>(f) + 1] = to;
    p.copies[3 * static_cast<uint64_t>(f) + 2] = rows;
  }
  if (tid == 0) {
    if (code) ptx::report_status(p.status, code);
    const uint32_t popped0 = code ? 0 : min(need, static_cast<uint32_t>(top[0]));
    p.free_out[0] = top[0] - static_cast<int32_t>(popped0);
    p.free_out[1] = top[1] - static_cast<int32_t>(code ? 0 : need - popped0);
  }
}

// Blocks that are held and whose ids are not below their arena's limit are marked; the last CTA takes such ids off the stacks,
// gives every marked block (in the order of ids) a free id, and writes down where it goes.
__device__ __forceinline__ uint32_t limit_of(const PagesParams& p, uint32_t a) {
  const int32_t l = p.limits[a];
  return l < 0 ? 0 : min(static_cast<uint32_t>(l), p.blocks[a]);
}

__global__ void __launch_bounds__(kThreads, 1) compact_plan_kernel(const PagesParams p) {
  __shared__ uint32_t warp_sums[kWarps], flag;
  const uint32_t tid = threadIdx.x, lane = tid & 31u;
  ptx::launch_dependents();
  ptx::grid_dependency_wait();
  const int32_t top[2] = {p.free_in[0], p.free_in[1]};
  const uint32_t limit[2] = {limit_of(p, 0), limit_of(p, 1)};
  bool bad = tops_bad(p, top) || p.limits[0] < 0 || p.limits[1] < 0;
  for (uint32_t i = tid; i < p.nseq; i += kThreads) bad |= length_bad(p, p.lens[i]);
  bad = __syncthreads_or(bad);
  if (!bad) {
    const uint32_t pieces = (p.max_blocks + kCells - 1) / kCells;
    const uint64_t items = static_cast<uint64_t>(p.nseq) * pieces;
    for (uint64_t x = static_cast<uint64_t>(blockIdx.x) * kWarps + (tid >> 5); x < items; x += static_cast<uint64_t>(gridDim.x) * kWarps) {
      const uint32_t i = static_cast<uint32_t>(x / pieces), at = static_cast<uint32_t>(x % pieces) * kCells;
      const uint32_t end = blocks_of(p.lens[i], p.block_shift);
      if (at >= end) continue;
      int32_t e[kCells / 32];
#pragma unroll
      for (uint32_t k = 0; k < kCells / 32; ++k) {
        const uint32_t j = at + k * 32 + lane;
        e[k] = j < end ? p.tables[i * p.table_stride + j] : 0;
      }
#pragma unroll
      for (uint32_t k = 0; k < kCells / 32; ++k) {
        if (at + k * 32 + lane >= end) continue;
        uint32_t a, id;
        if (!block_of(p, e[k], a, id))
          ptx::report_status(p.status, kStatusInvalid);
        else if (id >= limit[a])
          atomicOr(p.bits[a] + (id >> 5), 1u << (id & 31u));
      }
    }
  }
  // How many free ids stay: every CTA counts a share of the stacks.
  for (uint32_t a = 0; !bad && a < 2; ++a) {
    uint32_t count = 0;
    // (unsigned: the sum of a place and a stride may pass 2^31)
    for (uint32_t k = blockIdx.x * kThreads + tid; k < static_cast<uint32_t>(top[a]); k += gridDim.x * kThreads) {
      const uint32_t id = static_cast<uint32_t>(p.ids[a][k]);
      count += id < limit[a];
      if (id >= p.blocks[a]) ptx::report_status(p.status, kStatusInvalid);  // dropped as well
    }
    count = __reduce_add_sync(0xffffffffu, count);
    if (lane == 0 && count) atomicAdd(p.moved + 1 + a, count);
  }
  if (!last_cta(p.work, &flag)) return;
  constexpr uint32_t kEach = 8;                    // ids of a thread at a time
  uint32_t words[2], marked[2], mine[2], before[2], kept[2];
  for (uint32_t a = 0; a < 2; ++a) {
    words[a] = (p.blocks[a] + 31) / 32;
    const uint32_t run = (words[a] + kThreads - 1) / kThreads;
    mine[a] = 0;
    for (uint32_t w = min(tid * run, words[a]), end = min(tid * run + run, words[a]); w < end; ++w) mine[a] += __popc(__ldcg(p.bits[a] + w));
    before[a] = block_exclusive(mine[a], warp_sums, marked[a]);
    kept[a] = __ldcg(p.moved + 1 + a);
  }
  __syncthreads();
  if (tid == 0) p.moved[1] = p.moved[2] = 0;
  const uint32_t need = marked[0] + marked[1];
  const int code = bad ? kStatusInvalid : need > static_cast<uint64_t>(kept[0]) + kept[1] ? kStatusNoSpace : need > p.ncopies ? kStatusInvalid : 0;
  if (!code) {
    for (uint32_t a = 0; a < 2; ++a) {
      // In place: what is written lies at or before what has been read, and the ids of a step are all read before any is written.
      uint32_t at = 0;
      for (uint32_t k0 = 0; k0 < static_cast<uint32_t>(top[a]); k0 += kThreads * kEach) {
        int32_t id[kEach];
        uint32_t count = 0, step;
#pragma unroll
        for (uint32_t c = 0; c < kEach; ++c) {
          const uint32_t k = k0 + tid * kEach + c;
          id[c] = k < static_cast<uint32_t>(top[a]) ? p.ids[a][k] : -1;
          count += static_cast<uint32_t>(id[c]) < limit[a];
        }
        uint32_t to = at + block_exclusive(count, warp_sums, step);
#pragma unroll
        for (uint32_t c = 0; c < kEach; ++c)
          if (static_cast<uint32_t>(id[c]) < limit[a]) p.ids[a][to++] = id[c];
        at += step;
      }
    }
  }
  // The marked blocks in order: their entries first, a word's by one thread, then the rest by all.
  for (uint32_t a = 0; a < 2; ++a) {
    const uint32_t run = (words[a] + kThreads - 1) / kThreads;
    uint64_t r = before[a] + (a ? marked[0] : 0);
    for (uint32_t w = min(tid * run, words[a]), end = min(tid * run + run, words[a]); mine[a] && w < end; ++w) {
      uint32_t bits = __ldcg(p.bits[a] + w);
      if (!bits) continue;
      p.bits[a][w] = 0;
      for (; bits && !code; bits &= bits - 1, ++r) {
        const int32_t id = static_cast<int32_t>(w * 32 + __ffs(bits) - 1);
        p.copies[3 * r] = a ? ~id : id;
      }
    }
  }
  __syncthreads();
  for (uint32_t r0 = 0; !code && r0 < need; r0 += kThreads * kEach) {
    int32_t from[kEach], to[kEach], refs[kEach];
#pragma unroll
    for (uint32_t c = 0; c < kEach; ++c) {
      const uint32_t r = r0 + c * kThreads + tid;
      if (r >= need) continue;
      from[c] = p.copies[3 * static_cast<uint64_t>(r)];
      to[c] = r < kept[0] ? p.ids[0][kept[0] - 1 - r] : ~p.ids[1][kept[1] - 1 - (r - kept[0])];
    }
#pragma unroll
    for (uint32_t c = 0; c < kEach; ++c)
      if (r0 + c * kThreads + tid < need) refs[c] = from[c] < 0 ? p.refs[1][~from[c]] : p.refs[0][from[c]];
#pragma unroll
    for (uint32_t c = 0; c < kEach; ++c) {
      const uint32_t r = r0 + c * kThreads + tid;
      if (r >= need) continue;
      const bool a = from[c] < 0, b = to[c] < 0;
      p.map[a][a ? ~from[c] : from[c]] = to[c];
      p.refs[b][b ? ~to[c] : to[c]] = refs[c];  // a free id's: nobody's place in this list
      p.refs[a][a ? ~from[c] : from[c]] = 0;
      p.copies[3 * static_cast<uint64_t>(r) + 1] = to[c];
      p.copies[3 * static_cast<uint64_t>(r) + 2] = 1 << p.block_shift;
    }
  }
  for (uint64_t x = 3 * static_cast<uint64_t>(code ? 0 : need) + tid; x < 3 * static_cast<uint64_t>(p.ncopies); x += kThreads) p.copies[x] = 0;
  if (tid == 0) {
    *p.moved = code ? 0 : need;
    if (code) ptx::report_status(p.status, code);
    const uint32_t popped0 = code ? 0 : min(need, kept[0]);
    p.free_out[0] = code ? top[0] : static_cast<int32_t>(kept[0] - popped0);
    p.free_out[1] = code ? top[1] : static_cast<int32_t>(kept[1] - (need - popped0));
  }
}

// The cells of blocks that move.
__global__ void __launch_bounds__(kThreads, 2) compact_cells_kernel(const PagesParams p) {
  ptx::launch_dependents();
  ptx::grid_dependency_wait();
  if (*p.moved == 0) return;
  const uint32_t lane = threadIdx.x & 31u;
  const uint32_t limit[2] = {limit_of(p, 0), limit_of(p, 1)};
  const uint32_t pieces = (p.max_blocks + kCells - 1) / kCells;
  const uint64_t items = static_cast<uint64_t>(p.nseq) * pieces;
  for (uint64_t x = static_cast<uint64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); x < items; x += static_cast<uint64_t>(gridDim.x) * kWarps) {
    const uint32_t i = static_cast<uint32_t>(x / pieces), at = static_cast<uint32_t>(x % pieces) * kCells;
    const uint32_t end = blocks_of(p.lens[i], p.block_shift);
    if (at >= end) continue;
    int32_t* row = p.tables + i * p.table_stride + at + lane;
    int32_t e[kCells / 32];
#pragma unroll
    for (uint32_t k = 0; k < kCells / 32; ++k) e[k] = at + k * 32 + lane < end ? row[k * 32] : 0;
#pragma unroll
    for (uint32_t k = 0; k < kCells / 32; ++k) {
      uint32_t a, id;
      if (at + k * 32 + lane < end && block_of(p, e[k], a, id) && id >= limit[a]) row[k * 32] = p.map[a][id];
    }
  }
}

// The first rows of blocks into other blocks, in all layers: both planes of a copy are pieces of at most kPiece bytes, each a CTA's
// work. Bound by HBM: every byte is read and written once.
constexpr uint32_t kCopyThreads = 256, kCopyEach = 4, kPiece = kCopyThreads * kCopyEach * 16;

__global__ void __launch_bounds__(kCopyThreads) copy_rows_kernel(const __grid_constant__ MoveParams p) {
  __shared__ int32_t list[kCopyThreads][3];
  __shared__ uint32_t which[kCopyThreads], count;
  const uint32_t tid = threadIdx.x;
  ptx::launch_dependents();
  ptx::grid_dependency_wait();
  const uint64_t plane = static_cast<uint64_t>(p.row_bytes) << p.block_shift;
  const uint32_t pieces = static_cast<uint32_t>((plane + kPiece - 1) / kPiece), per_copy = pieces * 2 * p.nlayers;
  const uint64_t items = static_cast<uint64_t>(p.ncopies) * per_copy;
  for (uint64_t x0 = blockIdx.x; x0 < items; x0 += static_cast<uint64_t>(gridDim.x) * kCopyThreads) {
    // The CTA's next items, as many as it has threads; those with nothing to do are passed over (a list may be mostly empty).
    __syncthreads();
    if (tid == 0) count = 0;
    __syncthreads();
    const uint64_t x = x0 + static_cast<uint64_t>(tid) * gridDim.x;
    if (x < items) {
      const uint64_t c = x / per_copy;
      const int32_t src = p.copies[3 * c], dst = p.copies[3 * c + 1], rows = p.copies[3 * c + 2];
      const uint32_t part = static_cast<uint32_t>(x % per_copy);
      if (rows != 0) {
        const uint32_t sa = src < 0, da = dst < 0;
        const uint32_t s = static_cast<uint32_t>(sa ? ~src : src), d = static_cast<uint32_t>(da ? ~dst : dst);
        const bool ok = rows > 0 && rows <= 1 << p.block_shift && s < p.blocks[sa] && d < p.blocks[da];
        if (!ok) ptx::report_status(p.status, kStatusInvalid);
        if (ok && src != dst && static_cast<uint64_t>(part % pieces) * kPiece < static_cast<uint64_t>(rows) * p.row_bytes) {
          const uint32_t at = atomicAdd(&count, 1u);  // the order of copies does not matter
          list[at][0] = src;
          list[at][1] = dst;
          list[at][2] = rows;
          which[at] = part;
        }
      }
    }
    __syncthreads();
    const uint32_t n = count;
    for (uint32_t k = 0; k < n; ++k) {
      const int32_t src = list[k][0], dst = list[k][1];
      const uint32_t part = which[k], layer = part / (2 * pieces), half = part / pieces & 1u, piece = part % pieces;
      const uint32_t sa = src < 0, da = dst < 0;
      const uint32_t bytes = static_cast<uint32_t>(list[k][2]) * p.row_bytes - piece * kPiece;
      const uint64_t off = half * plane + static_cast<uint64_t>(piece) * kPiece;
      const uint8_t* from = p.base[sa][layer] + static_cast<uint64_t>(sa ? ~src : src) * p.block_stride[sa] + off;
      uint8_t* to = p.base[da][layer] + static_cast<uint64_t>(da ? ~dst : dst) * p.block_stride[da] + off;
      uint4 v[kCopyEach];
#pragma unroll
      for (uint32_t i = 0; i < kCopyEach; ++i) {
        const uint32_t b = (i * kCopyThreads + tid) * 16;
        if (b < bytes) v[i] = ptx::ld_once_v4(from + b);
      }
#pragma unroll
      for (uint32_t i = 0; i < kCopyEach; ++i) {
        const uint32_t b = (i * kCopyThreads + tid) * 16;
        if (b < bytes) *reinterpret_cast<uint4*>(to + b) = v[i];
      }
    }
  }
}

// Accepted rows to their places: row len + j of a request takes what row len + keep[j] held, in order. keep rises, so row j of a
// list is read before it or any row behind it is written. A thread has the same 16 bytes of the row for the whole list and needs
// nobody else: a unit moves to where its new row's order has it.
constexpr uint32_t kKeepThreads = 128, kKeepStage = 64, kKeepEach = 8;

__global__ void __launch_bounds__(kKeepThreads) keep_rows_kernel(const __grid_constant__ MoveParams p) {
  struct Place {
    uint64_t off;
    uint32_t arena, swz;
  };
  __shared__ Place from[kKeepStage], to[kKeepStage];
  const uint32_t tid = threadIdx.x, i = blockIdx.x;
  ptx::launch_dependents();
  ptx::grid_dependency_wait();
  const int32_t n = p.counts[i], len = p.lens[i];
  const int64_t room = static_cast<int64_t>(p.max_blocks) << p.block_shift;
  if (n == 0) return;
  bool bad = n < 0 || static_cast<uint32_t>(n) > p.max_keep || len < 0;
  const int32_t* keep = p.keep + i * p.keep_stride;
  for (int32_t j = static_cast<int32_t>(tid); !bad && j < n; j += kKeepThreads) {
    const int32_t k = keep[j];
    // By itself, as the entries before may be anything: from j on (so that row j is in range where row k is), above the one before.
    bad = k < j || (j && k <= keep[j - 1]) || len + static_cast<int64_t>(k) >= room;
    if (bad) break;
    for (uint32_t x = 0; x < 2; ++x) {
      const int32_t e = p.tables[i * p.table_stride + ((static_cast<uint32_t>(len) + (x ? k : j)) >> p.block_shift)];
      bad |= static_cast<uint32_t>(e < 0 ? ~e : e) >= p.blocks[e < 0];
    }
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) ptx::report_status(p.status, kStatusInvalid);
    return;
  }
  const uint64_t plane = static_cast<uint64_t>(p.row_bytes) << p.block_shift;
  const uint32_t mask = (1u << p.block_shift) - 1, units = p.row_bytes / 16;
  const uint32_t x = blockIdx.y * kKeepThreads + tid;  // layer, plane, unit
  const bool on = x < p.nlayers * 2 * units;
  const uint32_t u = x % units, layer = on ? x / units / 2 : 0, half = x / units & 1u;
  for (int32_t j0 = 0; j0 < n; j0 += kKeepStage) {
    __syncthreads();
    if (tid < 2 * kKeepStage) {
      const int32_t j = j0 + static_cast<int32_t>(tid % kKeepStage);
      if (j < n) {
        const uint32_t at = static_cast<uint32_t>(len) + (tid < kKeepStage ? keep[j] : j);
        const int32_t e = p.tables[i * p.table_stride + (at >> p.block_shift)];
        Place& place = (tid < kKeepStage ? from : to)[tid % kKeepStage];
        place.arena = e < 0;
        place.off = static_cast<uint64_t>(e < 0 ? ~e : e) * p.block_stride[e < 0] + (at & mask) * static_cast<uint64_t>(p.row_bytes);
        place.swz = at & 7u;
      }
    }
    __syncthreads();
    if (!on) continue;
    const uint32_t m = static_cast<uint32_t>(min(n - j0, static_cast<int32_t>(kKeepStage)));
    for (uint32_t b = 0; b < m; b += kKeepEach) {
      uint4 v[kKeepEach];
#pragma unroll
      for (uint32_t c = 0; c < kKeepEach; ++c)
        if (b + c < m) {
          const Place& f = from[b + c];
          v[c] = ptx::ld_once_v4((f.arena ? p.base[1][layer] : p.base[0][layer]) + f.off + half * plane + ((u & ~7u) + ((u & 7u) ^ f.swz)) * 16);
        }
#pragma unroll
      for (uint32_t c = 0; c < kKeepEach; ++c)
        if (b + c < m) {
          const Place& t = to[b + c];
          *reinterpret_cast<uint4*>((t.arena ? p.base[1][layer] : p.base[0][layer]) + t.off + half * plane + ((u & ~7u) + ((u & 7u) ^ t.swz)) * 16) = v[c];
        }
    }
  }
}

// CTAs for the cells of `rows` table rows: a warp takes kCells at a time.
unsigned grid_of(uint64_t rows, uint32_t max_blocks, int num_sms) {
  const uint64_t items = rows * ((max_blocks + kCells - 1) / kCells), ctas = (items + kWarps - 1) / kWarps;
  return static_cast<unsigned>(ctas < 1 ? 1 : ctas < static_cast<uint64_t>(num_sms) ? ctas : num_sms);
}

}  // namespace

cudaError_t launch_free(const PagesParams& p, int num_sms, cudaStream_t stream) {
  return launch_ahead(free_kernel, grid_of(p.nseq, p.max_blocks, num_sms), kThreads, 0, stream, p);
}

cudaError_t launch_fork(const PagesParams& p, int num_sms, cudaStream_t stream) {
  return launch_ahead(fork_kernel, grid_of(p.nfork, p.max_blocks, num_sms), kThreads, (p.nseq + 31) / 32 * 4, stream, p);
}

cudaError_t launch_compact(const PagesParams& p, int num_sms, cudaStream_t stream) {
  const unsigned grid = grid_of(p.nseq, p.max_blocks, num_sms);
  // The stacks are looked through as well, an id to a thread.
  const uint64_t stacks = (static_cast<uint64_t>(p.capacity[0]) + p.capacity[1] + kThreads - 1) / kThreads, most = static_cast<uint64_t>(num_sms);
  const unsigned plan = static_cast<unsigned>(stacks < grid ? grid : stacks < most ? stacks : most);
  const cudaError_t e = launch_ahead(compact_plan_kernel, plan, kThreads, 0, stream, p);
  return e != cudaSuccess ? e : launch_ahead(compact_cells_kernel, grid, kThreads, 0, stream, p);
}

cudaError_t launch_copy_rows(const MoveParams& p, int num_sms, cudaStream_t stream) {
  const uint64_t plane = static_cast<uint64_t>(p.row_bytes) << p.block_shift;
  const uint64_t items = static_cast<uint64_t>(p.ncopies) * ((plane + kPiece - 1) / kPiece) * 2 * p.nlayers, most = static_cast<uint64_t>(num_sms) * 8;
  return launch_ahead(copy_rows_kernel, static_cast<unsigned>(items < most ? items : most), kCopyThreads, 0, stream, p);
}

cudaError_t launch_keep_rows(const MoveParams& p, cudaStream_t stream) {
  const uint32_t threads = p.nlayers * 2 * (p.row_bytes / 16);
  return launch_ahead(keep_rows_kernel, dim3(p.nseq, (threads + kKeepThreads - 1) / kKeepThreads), kKeepThreads, 0, stream, p);
}

}  // namespace ema
