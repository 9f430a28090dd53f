// paged_tree.cu — attention of several new tokens per request over a paged KV cache: the drafted tokens of speculative decoding (a
// tree, given as a bit mask, or a chain) and pieces of prompts; tables, lengths and offsets read from device memory.
//
//   o = softmax(s q K^T) V over the context and those of the request's new tokens that the row sees, per query head.
//
// The query rows of one KV head (tokens x heads of the group) are tiles of 128, the M side of tcgen05 products. Of a step of 128
// positions (head_dim 128: 64 KB of K and V, 2470 cycles of an SM's share of HBM at 1.67 GHz) the scores take the tensor cores 560 cycles a tile, and
// the product with V 770 or, with weights as two numbers, 1540: an operand in tensor memory takes 96 cycles where N = 128 would take 64.
//   * An item is up to two tiles of one (request, KV head). The line of all items' steps is cut into equal ranges, one to a CTA: an item
//     may be cut, and its parts are joined by a second launch.
//   * Two warps copy K and V (tiled bulk copies; the block format's order of 16-byte units within 128 bytes is the one that the tensor
//     cores want, so a tile is used as it lies in the block), one issues the products, two groups of four do the softmax, a row to a
//     thread, and four write rows out while the next item goes on. Each softmax group has a stream of its own: scores, weights and
//     sums O in tensor memory. With two tiles a stream is a tile; with one, the streams take every other step and are added at the
//     end. While one group works on its scores the tensor cores work for the other one. (head_dim 256: O takes half of the tensor
//     memory, so there is one tile, one stream with two buffers for scores, and one of the groups is idle.)
//   * Weights take the place of their scores in tensor memory. Where a request's rows of a KV head are one tile (drafted tokens, which are compared
//     with and go on as single tokens; bound by HBM), they are the sum of two 16-bit numbers (error 2^-16 for bf16), as in attention of single tokens.
//     Where they are more (prompts; bound by the products and the softmax), a weight is one rounded number, which adds an error as large as the
//     output's own rounding. One number / two: 64 requests with 24 tokens each 129 / 134 us (145 / 167 one call after the other, at the clocks that
//     power leaves), outputs off by 0.0023 / 0.0017 of their size (their own rounding is 0.0017); 200 with up to 9 tokens and a window 219 / 251; 8
//     pieces of prompts 910 / 1066, five long requests of two tiles 779 / 936. Sums of weights are taken before the rounding, in f32.
//   * O is rescaled only when a row's maximum has grown by more than 2^kSlack; until then weights are larger than 1.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>
#include <type_traits>

#include "kernels.h"
#include "ptx.cuh"
#include "tcgen05.cuh"

namespace ema {

namespace {

constexpr float kMinusInf = -INFINITY;
// Warps: one that issues the products, two that copy (and an idle one), two groups of four for the softmax, four that write rows out.
constexpr uint32_t kThreads = 512, kIssueWarp = 0, kFeedWarp = 1, kSoftWarp = 4, kOutWarp = 12;
constexpr uint32_t kNotes = 4;
// Registers of a thread: the launch has 128 for everybody (exactly: with fewer the request for more would not end); the two groups of the softmax
// get what warps 0 to 3 and those that write out give up.
constexpr uint32_t kSoftRegs = 168, kOtherRegs = 88;
static_assert(2 * kSoftRegs + 2 * kOtherRegs <= 4 * 128, "no more than the block was launched with");

template <uint32_t D>
struct Shape {
  static constexpr uint32_t kTok = D == 256 ? 64 : 128;      // positions of a step
  static constexpr uint32_t kStreams = D == 256 ? 1 : 2;     // which is also the most tiles of an item
  static constexpr uint32_t kRows = kStreams * 128;
  static constexpr uint32_t kChunks = D / 64;                // pieces of 128 bytes of a head
  static constexpr uint32_t kTileBytes = 128 * D * 2;        // of queries
  static constexpr uint32_t kSlotBytes = kTok * D * 2;       // of K or of V
  static constexpr uint32_t kSlots = D == 64 ? 12 : 5;
  static constexpr uint32_t kO = 2 * kTok;                   // columns of tensor memory: two buffers of scores, then O
  static constexpr uint32_t kPart = kRows * (D + 2);         // floats of a part: [D / 4][rows] float4, maxima, sums
  static constexpr uint32_t kItem = 2;                       // steps that an item costs besides its own
  static_assert(kO + kStreams * D <= 512, "tensor memory");
};

struct Maps {
  CUtensorMap m[2];             // K and V of either arena
  CUtensorMap q;
};

// An item, or the part of it that a CTA does. tiles == 0: there are no more.
struct Note {
  uint32_t seq, head;
  uint32_t off, m, c;           // the request's first token, how many, and the context before them
  uint32_t tok0, ntok;          // those of the item
  uint32_t hi, lo, lo_all;      // positions [lo, hi) are seen by some row; from lo_all on by all of them,
  uint32_t full;                // up to here (less than that where a mask has the say)
  uint32_t first, tiles;        // steps of kTok positions
  uint32_t before;              // steps of this CTA before them
  uint32_t q;                   // where the queries of a single tile lie
  uint32_t turn;                // stream (of one: buffer) of the item's first unit
  uint32_t slot;                // part, or ~0: the whole item
};

template <uint32_t D>
struct Control {
  using S = Shape<D>;
  uint64_t full[S::kSlots], empty[S::kSlots];
  uint64_t note_full[kNotes], note_empty[kNotes];
  uint64_t q_full[2], q_empty[2], o_done, o_empty, stats_full, stats_empty, drain;
  uint64_t s_full[2], p_full[2], group[2];
  uint64_t summed;              // of one stream: after every product with V
  Note note[kNotes];
  uint32_t seen[2][2][4][4];    // positions of a step that some row sees: the groups' own, two steps' in turn, by warps
  union {
    float2 stats[S::kStreams][128];  // references and sums of the streams' rows
    unsigned long long warp_total[kThreads / 32];  // before there are any
  };
  uint32_t tmem, dead;
};

template <uint32_t D>
constexpr uint32_t tiles_bytes() {
  return Shape<D>::kStreams * Shape<D>::kTileBytes + Shape<D>::kSlots * Shape<D>::kSlotBytes;
}

__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, uint32_t y, uint32_t chunk, uint32_t block, uint32_t bar,
                                        uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4, %5}], "
      "[%6], %7;" ::"r"(dst),
      "l"(map), "r"(0), "r"(y), "r"(chunk), "r"(block), "r"(bar), "l"(policy)
      : "memory");
}

__device__ __forceinline__ void tma_queries(uint32_t dst, const CUtensorMap* map, uint32_t x, uint32_t head, uint32_t token, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(head), "r"(token), "r"(bar)
      : "memory");
}

// Two f32 numbers in one register pair: the pipes take both at a time.
__device__ __forceinline__ uint64_t two(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 each(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

template <bool kBf16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  if constexpr (kBf16) return ptx::pack_bf16x2(lo, hi);
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <bool kBf16>
__device__ __forceinline__ float2 unpack(uint32_t v) {
  if constexpr (kBf16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&v));
}

// Weights are 2^kTop at a row's reference, and 2^(kTop + kSlack) at most: an fp16 number ends at 65504 and has no bits below 2^-24.
template <bool kBf16>
__device__ constexpr float kTop = kBf16 ? 0.f : 11.f;
template <bool kBf16>
__device__ constexpr float kSlack = kBf16 ? 8.f : 4.f;

// Bounded wait; when it runs out nobody waits any more.
template <typename Ctl>
__device__ __forceinline__ bool wait(uint64_t& bar, uint32_t parity, Ctl& ctl, int* status) {
  const uint32_t b = ptx::smem_u32(&bar);
  if (ptx::mbar_try_wait(b, parity)) return true;
  const uint64_t t0 = ptx::global_timer_ns();
  for (uint32_t polls = 1;; ++polls) {
    if (ptx::mbar_try_wait(b, parity)) return true;
    if ((polls & 63u) == 0) {
      if (*reinterpret_cast<volatile uint32_t*>(&ctl.dead)) return false;
      if (ptx::global_timer_ns() - t0 > 2000000000ull) break;
    }
  }
  *reinterpret_cast<volatile uint32_t*>(&ctl.dead) = 1;
  ptx::report_status(status, kDevTimeout);
  return false;
}

template <typename Ctl>
__device__ __forceinline__ bool warp_wait(uint64_t& bar, uint32_t parity, Ctl& ctl, int* status) {
  return __all_sync(0xffffffffu, wait(bar, parity, ctl, status));
}

__device__ __forceinline__ void arrive(uint64_t& bar) { ptx::mbar_arrive(ptx::smem_u32(&bar)); }

struct Request {
  uint32_t off, m, c;
  bool ok;                      // lengths and offsets are in range
};

__device__ __forceinline__ Request request(const TreeParams& p, uint32_t i) {
  const int32_t a = p.offsets[i], b = p.offsets[i + 1], n = p.lens[i];
  Request r{};
  r.ok = a >= 0 && b >= a && static_cast<uint32_t>(b) <= p.ntok && n >= 0 && static_cast<uint64_t>(n) <= static_cast<uint64_t>(p.max_blocks) * p.block_tokens &&
         b - a <= n;
  if (!r.ok) return r;
  r.off = static_cast<uint32_t>(a);
  r.m = static_cast<uint32_t>(b - a);
  r.c = static_cast<uint32_t>(n) - r.m;
  return r;
}

// Tokens of a tile and of an item.
__device__ __forceinline__ uint32_t tile_tokens(const TreeParams& p) { return 128 / p.group; }

struct Range {
  uint32_t lo, hi, first, tiles;
};

// Item k of a request: what its rows see.
template <uint32_t D>
__device__ __forceinline__ Range range_of(const TreeParams& p, const Request& r, uint32_t k, uint32_t each) {
  constexpr uint32_t kTok = Shape<D>::kTok;
  const uint32_t t0 = k * each, t1 = min(r.m, t0 + each);
  Range g;
  g.hi = r.c + (p.mask ? r.m : t1);
  const uint32_t pos = r.c + (p.positions ? 0 : t0);  // the least of the rows' positions, or below
  g.lo = p.window && pos + 1 > p.window ? pos + 1 - p.window : 0;
  if (p.mask) g.lo = min(g.lo, r.c);  // the mask says which new tokens are seen, however far back
  g.first = g.lo / kTok;
  g.tiles = (g.hi + kTok - 1) / kTok - g.first;
  return g;
}

// What the row of a token sees: positions [lo, end), of which a mask takes away new tokens.
struct Row {
  const uint32_t* mask;         // NULL: there is none
  uint32_t bits[2];             // its first two words (all of it for requests of up to 64 new tokens), read before they are wanted
  uint32_t lo, end;
  bool on;
};

__device__ __forceinline__ Row row_of(const TreeParams& p, const Note& n, uint32_t j, bool on) {
  Row r{};
  r.on = on;
  if (!on) return r;
  uint32_t pos = n.c + j;
  if (p.positions) pos = static_cast<uint32_t>(max(static_cast<int64_t>(n.c), min(static_cast<int64_t>(p.positions[n.off + j]), static_cast<int64_t>(n.c) + n.m - 1)));
  r.lo = p.window && pos + 1 > p.window ? pos + 1 - p.window : 0;
  r.end = n.c + j + 1;
  if (p.mask) {
    r.mask = p.mask + static_cast<uint64_t>(n.off + j) * p.mask_stride;
    const uint2 v = *reinterpret_cast<const uint2*>(r.mask);
    r.bits[0] = v.x;
    r.bits[1] = v.y;
    r.lo = min(r.lo, n.c);
    r.end = n.c + n.m;
  }
  return r;
}

__device__ __forceinline__ uint32_t below(int32_t n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

// Bit i: the row sees position t + i.
__device__ __forceinline__ uint32_t visible(const TreeParams& p, const Row& r, uint32_t c, uint32_t t) {
  if (!r.on) return 0;
  uint32_t see = below(static_cast<int32_t>(r.end - t)) & ~below(static_cast<int32_t>(r.lo - t));
  if (r.mask) {
    const int32_t b = static_cast<int32_t>(t - c), i = b >> 5;  // the first position as a new token, if it is one, and its word
    uint32_t w0, w1;
    if (p.mask_words == 2) {
      w0 = i == 0 ? r.bits[0] : i == 1 ? r.bits[1] : 0u;
      w1 = i == -1 ? r.bits[0] : i == 0 ? r.bits[1] : 0u;
    } else {
      w0 = i >= 0 && i < static_cast<int32_t>(p.mask_words) ? r.mask[i] : 0u;
      w1 = i >= -1 && i + 1 < static_cast<int32_t>(p.mask_words) ? r.mask[i + 1] : 0u;
    }
    see &= below(static_cast<int32_t>(c - t)) | __funnelshift_r(w0, w1, static_cast<uint32_t>(b) & 31u);
  }
  return see;
}

// Whether a request's rows of a KV head are more than a tile: its weights are one rounded number then.
__device__ __forceinline__ bool many_rows(const Note& n, uint32_t tile_tokens) { return n.m > tile_tokens; }

// Places in the ring of K and V tiles, in the order in which the products take them, which is the order in which they come free: of an
// item of n steps K0 V0 K1 V1 .. with two tiles of queries; with one, whose scores are a step ahead of its sums, K0 K1 V0 K2 V1 ..
// (In the order K0 V0 K1 .. a tile of V would lie there for the time of a softmax before it is used.)
__device__ __forceinline__ uint32_t k_place(uint32_t t, bool pair) { return pair ? 2 * t : t ? 2 * t - 1 : 0; }
__device__ __forceinline__ uint32_t v_place(uint32_t t, uint32_t n, bool pair) { return pair || t + 1 == n ? 2 * t + 1 : 2 * t + 2; }

// The copying warps find the CTA's items. One tells the others about them and copies queries and K, the other one copies V (one warp for both took longer
// over a step's copies than HBM: its code comes from far between the softmax warps').
template <uint32_t D, bool kV>
__device__ void feed(const TreeParams& p, const Maps& maps, Control<D>& ctl, uint8_t* queries, uint8_t* slots, const unsigned long long* before, uint32_t size) {
  using S = Shape<D>;
  constexpr uint32_t kTok = S::kTok;
  const uint32_t lane = threadIdx.x & 31u;
  const uint64_t policy = ptx::policy_evict_first();
  const uint32_t run = (p.nseq + kThreads - 1) / kThreads, each = S::kStreams * tile_tokens(p);
  const uint64_t from = static_cast<uint64_t>(blockIdx.x) * size, to = from + size;
  // The item in which the range begins.
  uint32_t x = 0, n = kThreads;
  while (n > 1) {
    const uint32_t half = n >> 1;
    if (before[x + half] <= from) x += half;
    n -= half;
  }
  uint64_t at = before[x];
  ptx::fence_proxy_async();
  asm volatile("bar.sync 1, 64;" ::: "memory");  // both have read the sums: copies may take their place
  uint32_t seq = x * run, head = 0, k = 0, items = 0;
  Request r{};
  Range g{};
  for (; seq < p.nseq; ++seq) {
    r = request(p, seq);
    items = (r.m + each - 1) / each;
    uint64_t one = 0;
    for (uint32_t i = 0; i < items; ++i) one += range_of<D>(p, r, i, each).tiles + S::kItem;
    const uint64_t all = one * p.num_kv_heads;
    if (from < at + all) {
      head = static_cast<uint32_t>((from - at) / one);
      at += head * one;
      for (;; ++k) {
        g = range_of<D>(p, r, k, each);
        if (from < at + g.tiles + S::kItem) break;
        at += g.tiles + S::kItem;
      }
      break;
    }
    at += all;
  }
  int32_t* joins = reinterpret_cast<int32_t*>(p.notes) + blockIdx.x * 8;
  uint32_t steps = 0;                       // of the items before
  uint32_t units = 0;                       // of the items before: a step with every tile of queries is one
  uint32_t q_next = 0, q_parity = 3;        // where the next single tile's queries go; parities of either place being empty
  uint32_t last = ~0u;                      // the last place that this warp has filled
  bool goes_on = false, alive = true;
  const uint32_t nb_shift = (kTok == 128 ? 7 : 6) - p.block_shift, blk = lane & ((1u << nb_shift) - 1), chunk = lane >> nb_shift;
  for (uint32_t j = 0; alive;) {
    const uint32_t cost = g.tiles + S::kItem;
    const bool have = seq < p.nseq && at < to;
    // A cut inside the item's own cost lies at its beginning.
    auto step_of = [&](uint64_t pos) { return pos <= S::kItem ? 0u : static_cast<uint32_t>(pos) - S::kItem; };
    const uint32_t a = have && from > at ? step_of(from - at) : 0, b = have && to < at + cost ? step_of(to - at) : g.tiles;
    if (!have || a < b) {
      if (!kV && j >= kNotes) alive = warp_wait(ctl.note_empty[j % kNotes], (j / kNotes - 1) & 1u, ctl, p.status);
      if (!alive) break;
      Note& note = ctl.note[j % kNotes];
      if (!have) {
        if (!kV && lane == 0) {
          note.tiles = 0;
          arrive(ctl.note_full[j % kNotes]);
        }
        break;
      }
      const uint32_t tok0 = k * each, ntok = min(each, r.m - tok0);
      const bool pair = S::kStreams == 2 && ntok > tile_tokens(p);
      if (!kV && lane == 0) {
        note.seq = seq;
        note.head = head;
        note.off = r.off;
        note.m = r.m;
        note.c = r.c;
        note.tok0 = tok0;
        note.ntok = ntok;
        note.hi = g.hi;
        note.lo = g.lo;
        const uint32_t last = r.c + (p.positions ? r.m : tok0 + ntok);  // behind the last of the rows' positions
        note.lo_all = p.window && last > p.window ? last - p.window : 0;
        note.full = r.c + (p.mask ? 0 : tok0 + 1);
        note.first = g.first + a;
        note.tiles = b - a;
        note.before = steps;
        note.q = q_next;
        note.turn = units & 1u;
        note.slot = a ? 2 * blockIdx.x : b < g.tiles ? 2 * blockIdx.x + 1 : ~0u;
        arrive(ctl.note_full[j % kNotes]);
        if (a == 0 && b < g.tiles) {
          goes_on = true;
          joins[1] = static_cast<int32_t>(r.off + tok0);
          joins[2] = static_cast<int32_t>(ntok);
          joins[3] = static_cast<int32_t>(head);
          joins[0] = static_cast<int32_t>((at + cost - 1) / size - blockIdx.x + 1);
        }
      }
      __syncwarp();
      // Queries: of a single tile, to the place that the item before the last one had; of two tiles (and of head_dim 256), when the last item's
      // scores have been done, behind the first step's copies. A tile's rows are tokens x heads of the group; rows of tokens
      // behind the item's last one are somebody's, and nobody's results.
      auto ask = [&] {
#pragma unroll
        for (uint32_t i = 0; i < S::kStreams; ++i) {
          const uint32_t place = pair ? i : q_next;
          if (i && !pair) break;
          alive = alive && warp_wait(ctl.q_empty[place], q_parity >> place & 1u, ctl, p.status);
          if (!alive) return;
          q_parity ^= 1u << place;
          if (lane == 0) ptx::mbar_arrive_expect_tx(ptx::smem_u32(&ctl.q_full[place]), S::kChunks * tile_tokens(p) * p.group * 128);
          __syncwarp();
          if (lane < S::kChunks)
            tma_queries(ptx::smem_u32(queries) + place * S::kTileBytes + lane * 16384, &maps.q, lane * 64, head * p.group,
                        r.off + tok0 + i * tile_tokens(p), ptx::smem_u32(&ctl.q_full[place]));
          __syncwarp();
        }
      };
      const bool late = pair || S::kStreams == 1;
      if (!kV && !late) ask();
      // A lane's copy of step t, and its block; the next step's entry is read before this one's copies wait.
      auto wanted = [&](uint32_t t) {
        const uint32_t pos = (g.first + t) * kTok + (blk << p.block_shift);
        return t < b && chunk < S::kChunks && pos < g.hi && pos + p.block_tokens > g.lo;
      };
      const int32_t* row = p.tables + seq * p.table_stride + blk;
      auto entry_of = [&](uint32_t t) { return row[((g.first + t) * kTok) >> p.block_shift]; };
      bool on = wanted(a);
      int32_t entry = on ? entry_of(a) : 0;
      for (uint32_t t = a; t < b; ++t) {
        const uint32_t boxes = __ballot_sync(0xffffffffu, on);
        const bool second = entry < 0;
        const uint32_t blocks = second ? p.blocks[1] : p.blocks[0];
        uint32_t id = static_cast<uint32_t>(second ? ~entry : entry);
        if (on && id >= blocks) {  // a bad page: reads as zeros (a box outside the tensor), and is reported
          ptx::report_status(p.status, kStatusInvalid);
          id = blocks ? blocks : second ? p.blocks[0] : p.blocks[1];  // of an arena without blocks the map is the other one's
        }
        const bool on_next = wanted(t + 1);
        const int32_t entry_next = on_next ? entry_of(t + 1) : 0;
        const uint32_t ring = 2 * steps + (kV ? v_place(t - a, b - a, pair) : k_place(t - a, pair)), slot = ring % S::kSlots;
        alive = warp_wait(ctl.empty[slot], (ring / S::kSlots & 1u) ^ 1u, ctl, p.status);
        if (!alive) break;
        last = ring;
        const uint32_t bar = ptx::smem_u32(&ctl.full[slot]);
        if (lane == 0) ptx::mbar_arrive_expect_tx(bar, __popc(boxes) << (p.block_shift + 7));
        __syncwarp();
        if (on)
          tma_box(ptx::smem_u32(slots) + slot * S::kSlotBytes + chunk * (kTok * 128) + ((blk << p.block_shift) << 7), second ? &maps.m[1] : &maps.m[0],
                  kV ? p.block_tokens : 0, head * S::kChunks + chunk, id, bar, policy);
        __syncwarp();
        on = on_next;
        entry = entry_next;
        if (!kV && late && t == a) {
          ask();
          if (!alive) break;
        }
      }
      steps += b - a;
      units += pair ? 2 * (b - a) : b - a;
      if (S::kStreams == 2 && !pair) q_next ^= 1;
      ++j;
    }
    // The next item.
    at += cost;
    if (++k == items) {
      k = 0;
      if (++head == p.num_kv_heads) {
        head = 0;
        // The next request with new tokens, 32 looked at together (a batch may be mostly padding).
        for (++seq; seq < p.nseq; seq += 32) {
          const uint32_t some = __ballot_sync(0xffffffffu, seq + lane < p.nseq && request(p, seq + lane).m > 0);
          if (some) {
            seq += __ffs(some) - 1;
            break;
          }
        }
        r = seq < p.nseq ? request(p, seq) : Request{};
        items = (r.m + each - 1) / each;
      }
    }
    if (seq < p.nseq) g = range_of<D>(p, r, k, each);
  }
  if (!kV && lane == 0 && !goes_on) joins[0] = 0;
  if (!alive) {
    // Copies still in flight get a bounded time to land before the CTA's shared memory is given back. (A place that is the other warp's has a phase of
    // its own: waiting for it does no harm, the wait ends.)
    for (uint32_t i = 0; i < S::kSlots && last != ~0u; ++i, --last)
      ptx::mbar_wait(ptx::smem_u32(&ctl.full[last % S::kSlots]), last / S::kSlots & 1u, nullptr, 0);
    for (uint32_t i = 0; i < 2 && !kV; ++i) ptx::mbar_wait(ptx::smem_u32(&ctl.q_full[i]), q_parity >> i & 1u, nullptr, 0);
  }
}

// Whether the phase has completed: does not wait.
__device__ __forceinline__ bool ready(uint64_t& bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(ptx::smem_u32(&bar)), "r"(parity)
      : "memory");
  return done != 0;
}

// The issuing thread. Units (a step with one tile of queries) take the two buffers of scores in turn, across items. Scores of a unit may
// be issued once the sums of the unit before the last one have been: products are done in the order in which they are issued, so
// that scores take the place of weights that were used before. Whatever has its operands goes first, scores before sums.
template <uint32_t D, bool kBf16>
__device__ void issue(const TreeParams& p, Control<D>& ctl, uint8_t* queries, uint8_t* slots) {
  using S = Shape<D>;
  constexpr uint32_t kTok = S::kTok;
  const uint32_t scores = tc::product(kBf16, kTok, false) | (p.q_flip ? 1u << 13 : 0u);  // a scale below 0: queries with the other sign
  constexpr uint32_t kSums = tc::product(kBf16, D, true);
  const uint32_t tmem = ctl.tmem, tt = tile_tokens(p);
  const uint64_t q0 = tc::operand(ptx::smem_u32(queries), 16, 1024);
  const uint64_t k0 = tc::operand(ptx::smem_u32(slots), 16, 1024), v0 = tc::operand(ptx::smem_u32(slots), kTok * 128, 1024);
  struct Cursor {
    uint32_t j, u, units, tiles, before, place, first, hi;
    bool pair, many;
  };
  Cursor a{}, b{};                // next scores, next sums: item, unit
  a.j = b.j = ~0u;
  uint32_t na = 0, nb = 0, q_parity = 0;
  bool last = false;              // there are no more items
  // The cursor's next item, if it is known.
  auto open = [&](Cursor& c) {
    const uint32_t j = c.j + 1;
    if (!ready(ctl.note_full[j % kNotes], j / kNotes & 1u)) return false;
    const Note& n = ctl.note[j % kNotes];
    c.j = j;
    c.tiles = n.tiles;
    if (n.tiles == 0) return true;  // the end: nothing else of the note has been written, the cursor's places stay where they are
    c.u = 0;
    c.pair = S::kStreams == 2 && n.ntok > tt;
    c.many = many_rows(n, tt);
    c.units = c.pair ? 2 * n.tiles : n.tiles;
    c.before = 2 * n.before;
    c.place = n.q;
    c.first = n.first;
    c.hi = n.hi;
    return true;
  };
  uint64_t t0 = ptx::global_timer_ns();
  for (uint32_t polls = 1; !last || nb < na; ++polls) {
    // What both want, asked for together and before anything is issued: what is issued runs for less time than it takes to ask.
    if (!last && a.u == a.units && open(a) && a.tiles == 0) last = true;
    if (nb < na && b.u == b.units) open(b);  // known: its scores have been issued
    const uint32_t ka = a.pair ? a.u >> 1 : a.u, qa = a.pair ? a.u & 1u : a.place, first_a = a.u < (a.pair ? 2 : 1);
    const uint32_t ring_a = a.before + k_place(ka, a.pair), slot_a = ring_a % S::kSlots, buf_a = na & 1u;
    const uint32_t kb = b.pair ? b.u >> 1 : b.u, ring_b = b.before + v_place(kb, b.tiles, b.pair), slot_b = ring_b % S::kSlots, buf_b = nb & 1u;
    const bool k_there = ready(ctl.full[slot_a], ring_a / S::kSlots & 1u), q_there = ready(ctl.q_full[qa], q_parity >> qa & 1u);
    const bool p_there = ready(ctl.p_full[buf_b], nb >> 1 & 1u), v_there = ready(ctl.full[slot_b], ring_b / S::kSlots & 1u);
    const bool o_free = b.u || b.j == 0 || ready(ctl.o_empty, (b.j - 1) & 1u);
    const bool to_score = !last && a.u < a.units && k_there && (!first_a || q_there);
    const bool to_sum = nb < na && p_there && v_there && o_free;
    bool moved = false;
    if (to_sum) {
      tc::fence_after();
      const uint32_t stream = S::kStreams == 2 ? buf_b : 0, o = tmem + S::kO + stream * D, weights = tmem + buf_b * kTok;
      const uint64_t y = v0 + slot_b * (S::kSlotBytes >> 4);
      const uint32_t t = (b.first + kb) * kTok;
      const bool add = b.u >= S::kStreams;
      auto sum = [&](uint32_t ks, uint32_t part, bool first) {
        tc::mma_ts(o, weights + ks / 2 * 32 + part * 16 + ks % 2 * 8, y + ks * (16 * 128 >> 4), kSums, !first || add);
      };
      if (t + kTok <= b.hi) {
#pragma unroll
        for (uint32_t ks = 0; ks < kTok / 16; ++ks) sum(ks, 0, ks == 0);
        if (!b.many)
#pragma unroll
          for (uint32_t ks = 0; ks < kTok / 16; ++ks) sum(ks, 1, false);
      } else {                    // positions that nobody sees are left out
        const uint32_t n = (b.hi - t + 15) / 16;
#pragma unroll 1
        for (uint32_t ks = 0; ks < n; ++ks) {
          sum(ks, 0, ks == 0);
          if (!b.many) sum(ks, 1, false);
        }
      }
      if (!b.pair || (b.u & 1u)) tc::commit(ptx::smem_u32(&ctl.empty[slot_b]));
      if (S::kStreams == 1) tc::commit(ptx::smem_u32(&ctl.summed));
      ++b.u;
      ++nb;
      if (b.u == b.units) {
        tc::commit(ptx::smem_u32(&ctl.o_done));
        arrive(ctl.note_empty[b.j % kNotes]);
      }
      moved = true;
    }
    if (to_score && na - nb < 2) {
      if (first_a) q_parity ^= 1u << qa;
      tc::fence_after();
      const uint64_t x = q0 + qa * (S::kTileBytes >> 4), y = k0 + slot_a * (S::kSlotBytes >> 4);
#pragma unroll
      for (uint32_t ks = 0; ks < D / 16; ++ks)
        tc::mma_ss(tmem + buf_a * kTok, x + (ks / 4) * (128 * 128 >> 4) + (ks % 4) * 2, y + (ks / 4) * (kTok * 128 >> 4) + (ks % 4) * 2, scores, ks != 0);
      tc::commit(ptx::smem_u32(&ctl.s_full[buf_a]));
      if (!a.pair || (a.u & 1u)) tc::commit(ptx::smem_u32(&ctl.empty[slot_a]));
      if (a.u + (a.pair ? 2 : 1) >= a.units) tc::commit(ptx::smem_u32(&ctl.q_empty[qa]));
      ++a.u;
      ++na;
      moved = true;
    }
    if (moved) {
      polls = 0;
    } else if ((polls & 63u) == 0) {
      if (*reinterpret_cast<volatile uint32_t*>(&ctl.dead)) break;
      const uint64_t t = ptx::global_timer_ns();
      if (polls == 64) t0 = t;
      if (t - t0 > 2000000000ull) {
        *reinterpret_cast<volatile uint32_t*>(&ctl.dead) = 1;
        ptx::report_status(p.status, kDevTimeout);
        break;
      }
    }
  }
  // Everything issued has been done before tensor and shared memory are given back.
  tc::commit(ptx::smem_u32(&ctl.drain));
  ptx::mbar_wait(ptx::smem_u32(&ctl.drain), 0, p.status, kDevTimeout);
}

// Registers that a load has written, from here on.
template <uint32_t N>
__device__ __forceinline__ void touch(uint32_t (&r)[N]) {
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}

// A group of four warps: the softmax of its stream, a row to a thread.
template <uint32_t D, bool kBf16>
__device__ void soften(const TreeParams& p, Control<D>& ctl, uint8_t* slots) {
  using S = Shape<D>;
  constexpr uint32_t kTok = S::kTok, kWords = kTok / 32;
  const uint32_t lane = threadIdx.x & 31u, x = (threadIdx.x >> 7) - kSoftWarp / 4, r = threadIdx.x & 127u;
  const uint32_t tmem = ctl.tmem + ((r & ~31u) << 16);  // this warp's part of tensor memory
  const uint32_t tt = tile_tokens(p), in_tile = r / p.group;
  const bool packed = r < tt * p.group;          // rows behind the tile's last token are padding
  const bool works = S::kStreams == 2 || x == 0;
  const bool simple = !p.mask && !p.positions;   // some row sees every position in [lo, hi)
  uint32_t s_parity = 0, sums_before = 0, group = 0;
  bool alive = true;
  for (uint32_t j = 0; alive; ++j) {
    alive = warp_wait(ctl.note_full[j % kNotes], j / kNotes & 1u, ctl, p.status);
    if (!alive) break;
    const Note n = ctl.note[j % kNotes];
    if (n.tiles == 0) break;
    const bool pair = S::kStreams == 2 && n.ntok > tt;
    const uint32_t tile = pair ? x ^ n.turn : 0;
    const uint32_t my_tok = tile * tt + in_tile;
    const bool mine = packed && my_tok < n.ntok;
    const Row row = row_of(p, n, n.tok0 + my_tok, mine);
    Row other{};                                 // of the second tile, whose V is the same
    if (pair && tile == 0) other = row_of(p, n, n.tok0 + tt + in_tile, packed && tt + in_tile < n.ntok);
    float top = kMinusInf, sum = 0.f;            // reference of the row's weights, and their sum
    const uint32_t units = pair ? 2 * n.tiles : n.tiles;
    const uint32_t taddr_o = tmem + S::kO + (S::kStreams == 2 ? x * D : 0);
    uint32_t done = 0;                           // units of this stream
    for (uint32_t u = S::kStreams == 2 ? x ^ n.turn : 0; works && u < units; u += S::kStreams, ++done) {
      const uint32_t buf = (u + n.turn) & 1u, kt = pair ? u >> 1 : u, t0 = (n.first + kt) * kTok;
      alive = warp_wait(ctl.s_full[buf], s_parity >> buf & 1u, ctl, p.status);
      if (!alive) break;
      s_parity ^= 1u << buf;
      tc::fence_after();
      const uint32_t scores = tmem + buf * kTok;
      const uint32_t words = t0 + kTok <= n.hi ? kWords : (n.hi - t0 + 31) / 32;  // what is left is not multiplied with V
      // Rows of V that no row of the item sees are made zeros, whatever they hold (a weight of 0 would not do). Of two tiles
      // the first one's product comes first.
      bool wipe = false, seen = false;
      if (t0 < n.lo_all || t0 + kTok > n.full || p.q_keep == 0) {
        uint32_t* by_words = ctl.seen[x][group & 1u][r >> 5];
        const bool share = !simple && tile == 0;
#pragma unroll 1
        for (uint32_t w = 0; w < words; ++w) {
          uint32_t see = visible(p, row, n.c, t0 + w * 32);
          if (!__all_sync(0xffffffffu, see == ~0u) || p.q_keep == 0) {
            uint32_t s[32];
            tc::ld32(s, scores + w * 32);
            tc::wait_ld();
            touch(s);
#pragma unroll
            for (uint32_t i = 0; i < 32; ++i) {
              if (p.q_keep == 0) s[i] = __float_as_uint(__uint_as_float(s[i]) * 0.f);  // a scale of 0: queries of zeros
              s[i] = see >> i & 1u ? s[i] : __float_as_uint(kMinusInf);
            }
            tc::st32(scores + w * 32, s);
          }
          if (share) {
            if (pair) see |= visible(p, other, n.c, t0 + w * 32);
            see = __reduce_or_sync(0xffffffffu, see);
            if (lane == 0) by_words[w] = see;
          }
        }
        __syncwarp();            // one lane has stored: the warp together again for the aligned wait
        tc::wait_st();
        if (simple) {
          wipe = t0 < n.lo || t0 + kTok > n.hi;
          seen = t0 + r >= n.lo && t0 + r < n.hi;
        } else if (share) {
          wipe = true;
          __syncwarp();
          if (lane == 0) arrive(ctl.group[x]);
          alive = warp_wait(ctl.group[x], group & 1u, ctl, p.status);
          if (!alive) break;
          const uint32_t w = r / 32 % kWords;
          const uint32_t(*by_warps)[4] = ctl.seen[x][group++ & 1u];
          seen = w < words && ((by_warps[0][w] | by_warps[1][w] | by_warps[2][w] | by_warps[3][w]) >> lane & 1u);
        }
        wipe = wipe && tile == 0;
      }
      // Twice over the scores, 32 at a time, each load waited for: in registers all at once they and their code, straight
      // through, took longer to fetch than to run, and a second buffer of 32 spilled.
      float mx[4] = {kMinusInf, kMinusInf, kMinusInf, kMinusInf};
#pragma unroll 1
      for (uint32_t w = 0; w < words; ++w) {
        uint32_t s[32];
        tc::ld32(s, scores + w * 32);
        tc::wait_ld();
        touch(s);
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) mx[i & 3u] = fmaxf(mx[i & 3u], __uint_as_float(s[i]));
      }
      const float most = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
      // (Rows of nobody's have no say: what they hold would move the others' references, and with them the rounding of their weights.)
      if (__any_sync(0xffffffffu, mine && (most - top) * p.scale_log2 > kSlack<kBf16>)) {
        const float now = fmaxf(top, most), al = now == kMinusInf ? 1.f : ptx::exp2_approx((top - now) * p.scale_log2);
        top = now;
        sum *= al;
        if (done) {
          // The stream's products so far have been done: of two streams, as the scores come after them; of one, the last may still run.
          if (S::kStreams == 1) {
            alive = warp_wait(ctl.summed, (sums_before + u - 1) & 1u, ctl, p.status);
            if (!alive) break;
            tc::fence_after();
          }
#pragma unroll 1
          for (uint32_t c = 0; c < D; c += 32) {
            uint32_t o[32];
            tc::ld32(o, taddr_o + c);
            tc::wait_ld();
            touch(o);
#pragma unroll
            for (uint32_t i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * al);
            tc::st32(taddr_o + c, o);
          }
          tc::wait_st();
        }
      }
      const float ref = top == kMinusInf ? 0.f : top;
      const uint64_t ref2 = two(-ref, -ref), scale2 = two(p.scale_log2, p.scale_log2), top2 = two(kTop<kBf16>, kTop<kBf16>), minus2 = two(-1.f, -1.f);
      uint64_t sums[2] = {0, 0};
      // In the scores' place: of 32 columns the first 16 become the weights, the others what their rounding left where that is wanted.
      auto weigh = [&](auto rest) {
        constexpr bool kRest = decltype(rest)::value;
#pragma unroll 1
        for (uint32_t w = 0; w < words; ++w) {
          uint32_t s[32], v[kRest ? 32 : 16];
          tc::ld32(s, scores + w * 32);
          tc::wait_ld();
          touch(s);
#pragma unroll
          for (uint32_t i = 0; i < 16; ++i) {
            // (The difference is taken first: of scores beyond 2^24 the rounding of a score times the scale would be more than an exponent's worth.)
            const float2 e = each(fma2(add2(two(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), ref2), scale2, top2));
            const float a = ptx::exp2_approx(e.x), b = ptx::exp2_approx(e.y);
            const uint64_t ab = two(a, b);
            sums[i & 1u] = add2(sums[i & 1u], ab);
            v[i] = pack<kBf16>(a, b);
            if constexpr (kRest) {
              const float2 h = unpack<kBf16>(v[i]), left = each(fma2(two(h.x, h.y), minus2, ab));
              v[16 + i] = pack<kBf16>(left.x, left.y);
            }
          }
          if constexpr (kRest)
            tc::st32(scores + w * 32, v);
          else
            tc::st16(scores + w * 32, v);
        }
      };
      if (many_rows(n, tt))
        weigh(std::false_type{});
      else
        weigh(std::true_type{});
      const float2 both = each(add2(sums[0], sums[1]));
      sum += both.x + both.y;
      if (wipe) {
        const uint32_t ring = 2 * n.before + v_place(kt, n.tiles, pair), slot = ring % S::kSlots;
        alive = warp_wait(ctl.full[slot], ring / S::kSlots & 1u, ctl, p.status);
        if (!alive) break;
        if (r < words * 32 && !seen) {
#pragma unroll
          for (uint32_t c = 0; c < S::kChunks; ++c)
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
              *reinterpret_cast<uint4*>(slots + slot * S::kSlotBytes + c * (kTok * 128) + r * 128 + i * 16) = make_uint4(0, 0, 0, 0);
        }
        ptx::fence_proxy_async();
      }
      __syncwarp();              // some lanes have wiped rows
      tc::wait_st();
      tc::fence_before();
      __syncwarp();
      if (lane == 0) arrive(ctl.p_full[buf]);
    }
    if (!alive) break;
    sums_before += units;
    // References and sums go to the warps that write rows out.
    if (j) alive = warp_wait(ctl.stats_empty, (j - 1) & 1u, ctl, p.status);
    if (done) ctl.stats[S::kStreams == 2 ? x : 0][r] = make_float2(top, sum);
    __syncwarp();
    if (lane == 0) {
      arrive(ctl.stats_full);
      arrive(ctl.note_empty[j % kNotes]);
    }
  }
}

// Four warps write rows out, or into the workspace where the item is cut: of one tile's two streams the sum.
template <uint32_t D, bool kBf16>
__device__ void write_rows(const TreeParams& p, Control<D>& ctl) {
  using S = Shape<D>;
  const uint32_t lane = threadIdx.x & 31u, r = threadIdx.x & 127u;
  const uint32_t tmem = ctl.tmem + ((r & ~31u) << 16) + S::kO;
  const uint32_t G = p.group, tt = tile_tokens(p), in_tile = r / G, my_head = r - in_tile * G;
  const uint32_t heads = p.num_kv_heads * G;
  bool alive = true;
  for (uint32_t j = 0; alive; ++j) {
    alive = warp_wait(ctl.note_full[j % kNotes], j / kNotes & 1u, ctl, p.status);
    if (!alive) break;
    const Note n = ctl.note[j % kNotes];
    if (n.tiles == 0) break;
    const bool pair = S::kStreams == 2 && n.ntok > tt;
    alive = warp_wait(ctl.stats_full, j & 1u, ctl, p.status);
    if (!alive) break;
    float top[2], sum[2];                        // of tiles
    float w0 = 1.f, w1 = 0.f;                    // of one tile's streams
    const bool both = !pair && S::kStreams == 2 && n.tiles > 1;
    if (pair) {
#pragma unroll
      for (uint32_t i = 0; i < 2; ++i) {
        const float2 v = ctl.stats[(i ^ n.turn) % S::kStreams][r];
        top[i] = v.x;
        sum[i] = v.y;
      }
    } else {
      const float2 a = ctl.stats[n.turn % S::kStreams][r], b = both ? ctl.stats[(n.turn ^ 1u) % S::kStreams][r] : make_float2(kMinusInf, 0.f);
      top[0] = fmaxf(a.x, b.x);
      const float ref = top[0] == kMinusInf ? 0.f : top[0];
      w0 = ptx::exp2_approx((a.x - ref) * p.scale_log2);
      w1 = ptx::exp2_approx((b.x - ref) * p.scale_log2);
      sum[0] = a.y * w0 + b.y * w1;
      top[1] = kMinusInf;
      sum[1] = 0.f;
    }
    __syncwarp();
    if (lane == 0) arrive(ctl.stats_empty);
    alive = warp_wait(ctl.o_done, j & 1u, ctl, p.status);
    if (!alive) break;
    tc::fence_after();
    float4* part = reinterpret_cast<float4*>(p.parts + static_cast<uint64_t>(n.slot) * S::kPart);
#pragma unroll 1
    for (uint32_t tile = 0; tile < (pair ? 2u : 1u); ++tile) {
      const uint32_t my_tok = tile * tt + in_tile, part_row = tile * 128 + r;
      const bool mine = r < tt * G && my_tok < n.ntok;
      const uint64_t tok = n.off + n.tok0 + my_tok;
      const float total = tile ? sum[1] : sum[0], inv = total > 0.f ? 1.f / total : total;  // no weight at all: a row of zeros; not a number stays one
      uint4* out = reinterpret_cast<uint4*>(p.out + tok * p.out_stride + static_cast<uint64_t>(n.head * G + my_head) * D * 2);
      const uint32_t o0 = S::kStreams == 2 ? ((tile ^ n.turn) & 1u) * D : 0, o1 = S::kStreams == 2 ? ((n.turn ^ 1u) & 1u) * D : 0;
      if (!__any_sync(0xffffffffu, mine)) continue;
#pragma unroll 1
      for (uint32_t c = 0; c < D; c += 16) {
        uint32_t o[16];
        __syncwarp();
        tc::ld16(o, tmem + o0 + c);
        if (both) {
          uint32_t more[16];
          tc::ld16(more, tmem + o1 + c);
          tc::wait_ld();
          touch(o);
          touch(more);
#pragma unroll
          for (uint32_t i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * w0 + __uint_as_float(more[i]) * w1);
        } else {
          tc::wait_ld();
          touch(o);
        }
        if (!mine) continue;
        if (n.slot == ~0u) {
#pragma unroll
          for (uint32_t i = 0; i < 2; ++i) {
            uint32_t v[4];
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
              v[e] = pack<kBf16>(__uint_as_float(o[i * 8 + e * 2]) * inv, __uint_as_float(o[i * 8 + e * 2 + 1]) * inv);
            out[c / 8 + i] = make_uint4(v[0], v[1], v[2], v[3]);
          }
        } else {
#pragma unroll
          for (uint32_t i = 0; i < 4; ++i)
            part[(c / 4 + i) * S::kRows + part_row] = make_float4(__uint_as_float(o[i * 4]), __uint_as_float(o[i * 4 + 1]), __uint_as_float(o[i * 4 + 2]),
                                                                 __uint_as_float(o[i * 4 + 3]));
        }
      }
      if (mine) {
        const float ref = tile ? top[1] : top[0];
        if (n.slot == ~0u) {
          if (p.lse) p.lse[tok * heads + n.head * G + my_head] = fmaf(ref, p.scale_log2, log2f(total) - kTop<kBf16>) * 0.6931471805599453f;
        } else {
          float* stats = reinterpret_cast<float*>(part) + S::kRows * D;
          stats[part_row] = ref;
          stats[S::kRows + part_row] = total;
        }
      }
    }
    tc::fence_before();
    __syncwarp();
    if (lane == 0) {
      arrive(ctl.o_empty);
      arrive(ctl.note_empty[j % kNotes]);
    }
  }
}

template <uint32_t D, bool kBf16>
__global__ void __launch_bounds__(kThreads, 1) paged_tree_kernel(const TreeParams p, const __grid_constant__ Maps maps) {
  using S = Shape<D>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* queries = smem_raw;
  uint8_t* slots = queries + S::kStreams * S::kTileBytes;
  Control<D>& ctl = *reinterpret_cast<Control<D>*>(slots + S::kSlots * S::kSlotBytes);
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
  if (tid == 0) {
    for (uint32_t s = 0; s < S::kSlots; ++s) {
      ptx::mbar_init(ptx::smem_u32(&ctl.full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.empty[s]), 1);
    }
    for (uint32_t s = 0; s < kNotes; ++s) {
      ptx::mbar_init(ptx::smem_u32(&ctl.note_full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.note_empty[s]), 13);
    }
    ptx::mbar_init(ptx::smem_u32(&ctl.o_done), 1);
    ptx::mbar_init(ptx::smem_u32(&ctl.o_empty), 4);
    ptx::mbar_init(ptx::smem_u32(&ctl.stats_full), 8);
    ptx::mbar_init(ptx::smem_u32(&ctl.stats_empty), 4);
    ptx::mbar_init(ptx::smem_u32(&ctl.summed), 1);
    ptx::mbar_init(ptx::smem_u32(&ctl.drain), 1);
    for (uint32_t s = 0; s < 2; ++s) {
      ptx::mbar_init(ptx::smem_u32(&ctl.q_full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.q_empty[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.s_full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.p_full[s]), 4);
      ptx::mbar_init(ptx::smem_u32(&ctl.group[s]), 4);
    }
    ptx::fence_barrier_init();
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.m[0]));
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.m[1]));
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.q));
    ctl.dead = 0;
  }
  __syncwarp();                   // one thread has been here, and it is the allocating warp's
  if (warp == kIssueWarp) tc::alloc(ptx::smem_u32(&ctl.tmem), 512);
  ptx::launch_dependents();
  ptx::grid_dependency_wait();

  // How the work is cut: steps before each thread's run of requests. The sums lie where the queries come later.
  unsigned long long* before = reinterpret_cast<unsigned long long*>(queries);
  const uint32_t run = (p.nseq + kThreads - 1) / kThreads, each = S::kStreams * tile_tokens(p);
  const uint32_t i0 = min(tid * run, p.nseq), i1 = min(i0 + run, p.nseq);
  unsigned long long mine = 0;
  bool bad = false;
  for (uint32_t i = i0; i < i1; ++i) {
    const Request r = request(p, i);
    bad |= !r.ok;
    unsigned long long one = 0;
    for (uint32_t k = 0; k * each < r.m; ++k) one += range_of<D>(p, r, k, each).tiles + S::kItem;
    mine += one * p.num_kv_heads;
  }
  unsigned long long inc = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned long long o = __shfl_up_sync(0xffffffffu, inc, d);
    if (lane >= static_cast<uint32_t>(d)) inc += o;
  }
  if (lane == 31) ctl.warp_total[warp] = inc;
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  unsigned long long total = 0, sum = inc - mine;
  for (uint32_t x = 0; x < kThreads / 32; ++x) {
    if (x < warp) sum += ctl.warp_total[x];
    total += ctl.warp_total[x];
  }
  before[tid] = sum;
  ptx::fence_proxy_async();       // written (and read) before bulk copies of queries write there
  // A part of less than two steps would leave a group without work.
  const unsigned long long share = (total + gridDim.x - 1) / gridDim.x;
  const uint32_t size = static_cast<uint32_t>(min(max(share, 2ull), 0xffffffffull));
  bad = __syncthreads_or(bad);

  if (warp >= kSoftWarp && warp < kOutWarp) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    soften<D, kBf16>(p, ctl, slots);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp >= kOutWarp)
      write_rows<D, kBf16>(p, ctl);
    else if (warp == kFeedWarp)
      feed<D, false>(p, maps, ctl, queries, slots, before, size);
    else if (warp == kFeedWarp + 1)
      feed<D, true>(p, maps, ctl, queries, slots, before, size);
    else if (warp == kIssueWarp && lane == 0)
      issue<D, kBf16>(p, ctl, queries, slots);
    __syncwarp();
  }

  // Requests whose length or offsets are out of range: zeros, where the offsets name rows.
  const uint32_t heads = p.num_kv_heads * p.group;
  for (uint32_t i = blockIdx.x; bad && i < p.nseq; i += gridDim.x) {
    if (request(p, i).ok) continue;
    if (tid == 0) ptx::report_status(p.status, kStatusInvalid);
    const int32_t a = p.offsets[i], b = p.offsets[i + 1];
    if (a < 0 || b < a || static_cast<uint32_t>(b) > p.ntok) continue;
    for (uint32_t t = static_cast<uint32_t>(a); t < static_cast<uint32_t>(b); ++t) {
      uint4* dst = reinterpret_cast<uint4*>(p.out + t * p.out_stride);
      for (uint32_t x = tid; x < heads * D / 8; x += kThreads) dst[x] = make_uint4(0, 0, 0, 0);
      if (p.lse)
        for (uint32_t x = tid; x < heads; x += kThreads) p.lse[static_cast<uint64_t>(t) * heads + x] = kMinusInf;
    }
  }
  tc::fence_before();
  __syncthreads();
  if (warp == kIssueWarp) tc::dealloc(ctl.tmem, 512);
}

// Items that were cut: the sum of their parts, weighted by their references, and the division. A warp takes 32 rows and 16 columns of an
// item at a time, a row to a lane, four parts in flight; of an item in many parts the CTA's warps take every eighth part each. Bound by
// latency: which items, then their parts, each a trip to L2.
constexpr uint32_t kJoinThreads = 256, kJoinWarps = kJoinThreads / 32, kJoinMany = 8;
static_assert(kTreeMaxCtas <= kJoinThreads, "a thread for every CTA's item");

template <uint32_t D, bool kBf16>
__global__ void __launch_bounds__(kJoinThreads) tree_join_kernel(const TreeParams p, const uint32_t ctas) {
  using S = Shape<D>;
  constexpr uint32_t kCols = 16, kAhead = 4;
  __shared__ uint32_t list[kTreeMaxCtas][4], warp_count[kJoinWarps];
  __shared__ float rows[kJoinWarps][kCols + 2][32];
  ptx::launch_dependents();
  ptx::grid_dependency_wait();
  const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5;
  const int4 note = tid < ctas ? reinterpret_cast<const int4*>(p.notes)[tid * 2] : make_int4(0, 0, 0, 0);
  const uint32_t ballot = __ballot_sync(0xffffffffu, note.x > 0);
  if (lane == 0) warp_count[warp] = __popc(ballot);
  __syncthreads();
  uint32_t at = __popc(ballot & ((1u << lane) - 1)), count = 0;
#pragma unroll
  for (uint32_t w = 0; w < kJoinWarps; ++w) {
    if (w < warp) at += warp_count[w];
    count += warp_count[w];
  }
  if (note.x > 0) {
    list[at][0] = tid | static_cast<uint32_t>(note.x) << 16;
    list[at][1] = static_cast<uint32_t>(note.y);
    list[at][2] = static_cast<uint32_t>(note.z);
    list[at][3] = static_cast<uint32_t>(note.w);
  }
  __syncthreads();
  const uint32_t G = p.group, tt = tile_tokens(p), heads = p.num_kv_heads * G;
  constexpr uint32_t kSlabs = S::kRows / 32, kPieces = D / kCols;
  const uint32_t tasks = count * kSlabs * kPieces;

  struct Task {
    uint32_t k, parts, row, col, head, h;
    uint64_t tok;
    bool on;
  };
  auto task_of = [&](uint32_t x) {
    const uint32_t* item = list[x / (kSlabs * kPieces)];
    Task t;
    t.k = item[0] & 0xffffu;
    t.parts = item[0] >> 16;
    t.head = item[3];
    t.col = x % kPieces;
    t.row = x / kPieces % kSlabs * 32 + lane;
    const uint32_t in_tile = (t.row & 127u) / G, tok = (t.row >> 7) * tt + in_tile;
    t.h = (t.row & 127u) - in_tile * G;
    t.tok = static_cast<uint64_t>(item[1]) + tok;
    t.on = in_tile < tt && tok < item[2];
    return t;
  };
  // Parts first, first + step, ..: a row's reference, its sum of weights and 16 columns.
  auto add_parts = [&](const Task& t, uint32_t first, uint32_t step, float& top, float& sum, float (&acc)[kCols]) {
    top = kMinusInf;
    sum = 0.f;
#pragma unroll
    for (uint32_t c = 0; c < kCols; ++c) acc[c] = 0.f;
#pragma unroll 1
    for (uint32_t i0 = first; i0 < t.parts; i0 += kAhead * step) {
      float m[kAhead], l[kAhead];
      float4 v[kAhead][kCols / 4];
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k) {
        const uint32_t i = i0 + k * step;
        const bool there = i < t.parts;
        // Part 0 lies in the second place of the CTA where the item begins, the others in the first places of the next ones.
        const float* from = p.parts + static_cast<uint64_t>(there && i ? 2 * (t.k + i) : 2 * t.k + 1) * S::kPart;
        m[k] = there ? from[S::kRows * D + t.row] : kMinusInf;
        l[k] = there ? from[S::kRows * (D + 1) + t.row] : 0.f;
#pragma unroll
        for (uint32_t c = 0; c < kCols / 4; ++c)
          v[k][c] = there ? reinterpret_cast<const float4*>(from)[(t.col * (kCols / 4) + c) * S::kRows + t.row] : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      const float now = fmaxf(fmaxf(top, m[0]), fmaxf(fmaxf(m[1], m[2]), m[3])), ref = now == kMinusInf ? 0.f : now;
      const float al = ptx::exp2_approx((top - ref) * p.scale_log2);
      top = now;
      sum *= al;
#pragma unroll
      for (uint32_t c = 0; c < kCols; ++c) acc[c] *= al;
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k) {
        const float w = ptx::exp2_approx((m[k] - ref) * p.scale_log2);
        sum = fmaf(l[k], w, sum);
#pragma unroll
        for (uint32_t c = 0; c < kCols / 4; ++c) {
          acc[4 * c] = fmaf(v[k][c].x, w, acc[4 * c]);
          acc[4 * c + 1] = fmaf(v[k][c].y, w, acc[4 * c + 1]);
          acc[4 * c + 2] = fmaf(v[k][c].z, w, acc[4 * c + 2]);
          acc[4 * c + 3] = fmaf(v[k][c].w, w, acc[4 * c + 3]);
        }
      }
    }
  };
  auto write = [&](const Task& t, float top, float sum, const float (&acc)[kCols]) {
    const float inv = sum > 0.f ? 1.f / sum : sum;
    uint4* out = reinterpret_cast<uint4*>(p.out + t.tok * p.out_stride + (static_cast<uint64_t>(t.head * G + t.h) * D + t.col * kCols) * 2);
#pragma unroll
    for (uint32_t c = 0; c < kCols; c += 8)
      out[c / 8] = make_uint4(pack<kBf16>(acc[c] * inv, acc[c + 1] * inv), pack<kBf16>(acc[c + 2] * inv, acc[c + 3] * inv),
                              pack<kBf16>(acc[c + 4] * inv, acc[c + 5] * inv), pack<kBf16>(acc[c + 6] * inv, acc[c + 7] * inv));
    if (p.lse && t.col == 0) p.lse[t.tok * heads + t.head * G + t.h] = fmaf(top, p.scale_log2, log2f(sum) - kTop<kBf16>) * 0.6931471805599453f;
  };

  float top, sum, acc[kCols];
  for (uint32_t x = blockIdx.x * kJoinWarps + warp; x < tasks; x += gridDim.x * kJoinWarps) {
    const Task t = task_of(x);
    if (!t.on || t.parts > kJoinMany) continue;
    add_parts(t, 0, 1, top, sum, acc);
    write(t, top, sum, acc);
  }
  for (uint32_t x = blockIdx.x; x < tasks; x += gridDim.x) {
    const Task t = task_of(x);
    if (t.parts <= kJoinMany || !__any_sync(0xffffffffu, t.on)) continue;  // the same for all warps
    if (t.on) add_parts(t, warp, kJoinWarps, top, sum, acc);
    __syncthreads();              // the rows may still be read
    if (t.on) {
      rows[warp][kCols][lane] = top;
      rows[warp][kCols + 1][lane] = sum;
#pragma unroll
      for (uint32_t c = 0; c < kCols; ++c) rows[warp][c][lane] = acc[c];
    }
    __syncthreads();
    if (warp || !t.on) continue;
    top = kMinusInf;
#pragma unroll
    for (uint32_t w = 0; w < kJoinWarps; ++w) top = fmaxf(top, rows[w][kCols][lane]);
    const float ref = top == kMinusInf ? 0.f : top;
    sum = 0.f;
#pragma unroll
    for (uint32_t c = 0; c < kCols; ++c) acc[c] = 0.f;
#pragma unroll 1
    for (uint32_t w = 0; w < kJoinWarps; ++w) {
      const float f = ptx::exp2_approx((rows[w][kCols][lane] - ref) * p.scale_log2);
      sum = fmaf(rows[w][kCols + 1][lane], f, sum);
#pragma unroll
      for (uint32_t c = 0; c < kCols; ++c) acc[c] = fmaf(rows[w][c][lane], f, acc[c]);
    }
    write(t, top, sum, acc);
  }
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
  static const EncodeFn fn = []() -> EncodeFn {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess)
      return nullptr;
    return reinterpret_cast<EncodeFn>(f);
  }();
  return fn;
}

template <uint32_t D, bool kBf16>
cudaError_t launch(const TreeParams& p, const Maps& maps, uint32_t grid, int dev, cudaStream_t stream) {
  constexpr size_t kSharedBytes = tiles_bytes<D>() + sizeof(Control<D>);
  static_assert(kSharedBytes <= 232448, "one CTA per SM");
  static std::atomic<bool> ready[64] = {};  // the attribute is a property of the function on one device; several threads may launch
  if (!ready[dev].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(paged_tree_kernel<D, kBf16>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSharedBytes));
    if (e != cudaSuccess) return e;
    // The second launch leaves the SMs' shared memory as the first one wants it.
    const cudaError_t c = cudaFuncSetAttribute(tree_join_kernel<D, kBf16>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (c != cudaSuccess) return c;
    ready[dev].store(true, std::memory_order_release);
  }
  const cudaError_t e = launch_ahead(paged_tree_kernel<D, kBf16>, grid, kThreads, kSharedBytes, stream, p, maps);
  if (e != cudaSuccess) return e;
  // Three CTAs of the join fit an SM. Two / three: 64 requests with 24 tokens each 146 / 140 us, with heads of 256 140 / 134, one of 8000 tokens 29.4 / 31.5.
  return launch_ahead(tree_join_kernel<D, kBf16>, grid * 3, kJoinThreads, 0, stream, p, grid);
}

template <uint32_t D>
cudaError_t launch_d(const TreeParams& p, const Maps& maps, uint32_t grid, int dev, cudaStream_t stream) {
  return p.dtype == 0 ? launch<D, true>(p, maps, grid, dev, stream) : launch<D, false>(p, maps, grid, dev, stream);
}

}  // namespace

size_t tree_workspace_bytes(uint32_t head_dim) {
  const size_t part = head_dim == 64 ? Shape<64>::kPart : head_dim == 128 ? Shape<128>::kPart : Shape<256>::kPart;
  static_assert(kTreeMaxCtas * 8 * 4 <= kTreeNotesBytes, "notes");
  return kTreeNotesBytes + 2 * kTreeMaxCtas * part * sizeof(float);
}

cudaError_t launch_tree(const TreeParams& p, int dev, int num_sms, cudaStream_t stream) {
  const EncodeFn encode = encode_fn();
  if (!encode) return cudaErrorNotSupported;
  Maps maps;
  for (int j = 0; j < 2; ++j) {
    if (j == 1 && (!p.blocks[0] || !p.blocks[1])) {  // one arena: one map serves both
      maps.m[1] = maps.m[0];
      break;
    }
    const int a = p.blocks[j] ? j : 1 - j;
    const cuuint64_t chunks = static_cast<cuuint64_t>(p.num_kv_heads) * p.head_dim / 64;
    const cuuint64_t dims[4] = {64, 2ull * p.block_tokens, chunks, p.blocks[a]};
    const cuuint64_t strides[3] = {chunks * 128, 128, p.block_stride[a]};
    const cuuint32_t box[4] = {64, p.block_tokens, 1, 1};
    const cuuint32_t elem[4] = {1, 1, 1, 1};
    auto make = [&] {
      return encode(&maps.m[j], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, p.base[a], dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    CUresult r = make();
    // A thread that has not used the GPU yet: the runtime would make its device's context current at the launch, the driver's call needs it now.
    if (r == CUDA_ERROR_INVALID_CONTEXT || r == CUDA_ERROR_NOT_INITIALIZED) {
      const cudaError_t e = cudaSetDevice(dev);
      if (e != cudaSuccess) return e;
      r = make();
    }
    if (r != CUDA_SUCCESS) return cudaErrorInvalidValue;
  }
  {
    const uint32_t heads = p.num_kv_heads * p.group;
    const cuuint64_t dims[3] = {p.head_dim, heads, p.ntok};
    // of one token there is no next one
    const cuuint64_t strides[2] = {p.head_dim * 2ull, p.ntok > 1 ? p.q_stride : static_cast<cuuint64_t>(heads) * p.head_dim * 2};
    const cuuint32_t box[3] = {64, p.group, 128 / p.group};
    const cuuint32_t elem[3] = {1, 1, 1};
    if (encode(&maps.q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<uint8_t*>(p.q), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return cudaErrorInvalidValue;
  }
  const uint32_t sms = static_cast<uint32_t>(num_sms);
  const uint32_t grid = sms < kTreeMaxCtas ? sms : kTreeMaxCtas;
  if (p.head_dim == 64) return launch_d<64>(p, maps, grid, dev, stream);
  if (p.head_dim == 128) return launch_d<128>(p, maps, grid, dev, stream);
  return launch_d<256>(p, maps, grid, dev, stream);
}

}  // namespace ema
