// paged_decode.cu — attention of one new token per sequence over a paged KV cache, everything that
// changes from step to step (tables, lengths) read from device memory; and its differential form.
//
//   o = softmax(s q K^T) V over positions max(0, len - window) .. len - 1, per query head; differential:
//   o_h = softmax(s q1 K1^T) V - lam_h softmax(s q2 K2^T) V, then optionally an RMS norm over the head.
//
// Every K and V byte is needed once and used for a handful of query rows: the kernel is bound by HBM,
// and what it does is keep enough copies in flight on every SM while the arithmetic stays hidden. Measured
// (B200, 6.45 TB/s copy rate, in a captured graph): 64 sequences of 512 to 4095 tokens, 32/8 heads of 128: 100 us, 6.0 TB/s; 5 of
// 60000 to 100001, 64/8 heads: 253 us, 6.5 TB/s; 200 with a window of 1000, 12 heads of 64: 96 us, 5.8 TB/s (102 us as called from
// Python); differential, 8 of 9000 to 40000, 16/4 heads of 256: 133 us, 6.0 TB/s; one of 8000, 32/8 heads: 19 us; one of 500: 10.9 us
// (launch, one read of the lengths, of a table cell, of the cache, one merge, each a trip to L2 or HBM).
//   * Work is cut into pieces, runs of chunks of one (sequence, KV head), an item; a chunk is 16 KB of it (64 /
//     32 / 16 tokens of K and V for head_dim 64 / 128 / 256). How items are cut (cut_of, share_of) depends on the
//     lengths alone; who computes a piece is settled by a ticket counter, because the SMs do not get equal shares of
//     HBM: with equal static ranges the first CTA had its data at 81 us, the last at 95. (Short work of few items is
//     dealt out, one range to a CTA: what counts there is that nobody's last rows wait for another join.)
//   * In a CTA, a scheduler warp draws tickets, a little ahead of the work. Consumer warps take the chunks of a
//     piece in turn, each through its own online softmax; each copies its own chunks, two at a time, into stages
//     of its own (tiled bulk copies of [tokens][head] boxes, the format's swizzled rows as they are: one warp that
//     issued the copies of all could not keep up with 16-token blocks, 143 us against 104 then). A merger
//     warp adds their rows at the end of a piece, while they are already at the next one, and writes them out.
//   * Per chunk: S^T[16 tokens x 8 rows] = K Q^T and O^T += V^T P^T on mma.sync m16n8k16 tiles (the
//     query rows are the narrow side, 1 to 16 of them: tcgen05's 64- or 128-row accumulators would
//     hold tokens for S but would need P rewritten through shared memory for O; the tensor work is a few
//     per cent of the time either way). Online softmax in f32, as powers of 2 of what is left after the maximum is taken
//     off. P enters the second product as the sum of two 16-bit numbers (error 2^-16 for bf16): one rounded P would add an
//     error as large as the output's own rounding, and the differential form subtracts two nearly equal rows.
//   * The differential form is the same pass: K heads 2g, 2g+1 of width D/2 lie side by side, so q1 is
//     padded with zeros behind and q2 in front and the 2G rows of a head run over K and V of width D. The two
//     maps of a head are neighbouring columns, which one thread holds.
//   * A cut item's pieces meet in the workspace, 16 or 32 at a time: whichever piece of a group arrives last adds
//     the group's rows, in order, and is a piece of the next level. The result does not depend on who that is.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "kernels.h"
#include "ptx.cuh"

namespace ema {

namespace {

constexpr uint32_t kStageBytes = 16384;             // K half, then V half
constexpr uint32_t kHalf = kStageBytes / 2;
constexpr uint32_t kDepth = 2;                      // stages of a consumer warp
constexpr uint32_t kNotes = 16;                     // most pieces known to the consumers at a time
// Chunks of known pieces that no copy has been started of (an item that one warp takes alone counts as one chunk): 200 sequences
// of at most 1000 attended tokens, 12 heads of 64: 92 us, with 3 95, with 24 112; 64 of up to 4095 tokens: 99 us with 3 to 24 (both before the sums of
// a piece's rows and the weights took their present forms).
constexpr uint32_t kAhead = 6;
// Items of at most two chunks are taken by one warp, which also writes them out (a merge takes longer than a chunk). Where
// pieces are many (four to every consumer warp of the grid) and this small on average, items of so many chunks are, too: 1000 sequences
// of 10 to 260 tokens 119 us, with 4 (which leaves most of them to all warps) 183. Without and with it, sequences of 10 to 240
// tokens, 8 KV heads of 128, by their number: 40: 16 / 18 us, 80: 24 / 22, 160: 41 / 32, 300: 67 / 47, 440 (the last without it): 93 / 62,
// 460 (the first with it): 95 / 64, 900: 172 / 105; 155 of up to 104, 15 KV heads, differential, heads of 64: 27 / 28, of 128: 45 / 32. So the
// rule is cautious: one warp an item pays from about half an item to a warp of the grid on.
constexpr uint32_t kSolo = 8;
constexpr uint32_t kFan = kPagedFan;                // most pieces that meet at a time
static_assert(kFan == 32, "sum_parts takes two times sixteen");
constexpr float kMinusInf = -INFINITY;

// Partial rows of eight columns: [D / 16][32 lanes] float4, then the columns' (maximum, sum) pairs.
template <uint32_t D>
__host__ __device__ constexpr uint32_t part_floats() {
  return 8 * (D + 2);
}

// NT = 2: items of 9 to 16 columns are two groups of eight. Each group has consumer warps and a merger warp of its own; the
// consumers of both take the same chunks from the same stages, which those of the first group fill. (A warp for all sixteen
// columns took 2 us a chunk, 770 instructions at 6 cycles each, hardly anything else running on its scheduler, and registers and
// partial rows left room for five of them: 40 sequences of up to 2000 tokens, 16 query heads to a KV head of 256, 141 us
// against 119, differential with 8 heads 113 against 98. Two chunks at a time in one warp gained nothing.)
// Consumer warps of a group: as many as leave room for everybody's partial rows beside the stages, and registers.
template <uint32_t D, uint32_t NT>
struct Shape {
  static constexpr uint32_t kPart = part_floats<D>();
  static constexpr uint32_t kWarps = NT == 2 ? 4 : kPart * 4 * 6 <= 26000 ? 6 : 5;
  static constexpr uint32_t kConsumers = kWarps * NT;
  static constexpr uint32_t kThreads = (kConsumers + 1 + NT) * 32;
};

struct Maps {
  CUtensorMap m[2];
};

// What a sequence asks for: tokens [lo, len), in chunks of kTok tokens from `first` on.
struct Span {
  uint32_t lo, len, first, chunks;
};

// A piece, as the scheduler tells the other warps. chunks == 0: there are no more.
struct Note {
  uint32_t seq, head;
  uint32_t lo, len;             // the sequence's span
  uint32_t chunk, chunks;       // first chunk (from the sequence's start), and how many
  uint32_t turn;                // warp of the first one; the next ones go to the next warps, in turn
  uint32_t solo;                // or all of them to the same warp, which also writes the rows out
  uint32_t index, count;        // piece `index` of the item's `count`
  uint32_t slot, step;          // piece i's part: slot + i * step; the first one's (step - 1) slots behind that
};

template <uint32_t D, uint32_t NT>
struct __align__(128) Shared {
  using S = Shape<D, NT>;
  uint8_t stage[S::kWarps][kDepth][kStageBytes];
  float part[NT][S::kWarps][S::kPart];
  float joined[NT][S::kPart];      // sum over parts of the workspace
  Note note[kNotes];
  uint64_t full[S::kWarps][kDepth];
  uint64_t left[S::kWarps][kDepth];  // the second group has read the stage
  uint64_t note_full[kNotes], note_empty[kNotes];
  uint64_t rows_full[NT], rows_empty[NT];  // the consumers' partial rows of a piece
  uint64_t job_full[NT], job_done[NT];     // sums over parts that the consumers help with when they have nothing else to do
  struct Job {
    uint32_t slot, odd, stride, count, tile;  // count 0: leave; tiles from `tile` on
  } job[NT];
  uint32_t idle[NT];
  uint32_t started;                // chunks of the CTA's pieces that copies have been started of
  uint32_t dead;                   // a bounded wait ran out: no further waiting
  int32_t open[NT];                // the mergers' arrivals, less the sizes of the groups that they found complete
  uint32_t warp_sum[S::kThreads / 32][2];
  unsigned long long warp_total[S::kThreads / 32];
  uint32_t pieces_before[S::kThreads], parts_before[S::kThreads];  // before the threads' runs of sequences
  unsigned long long chunks_before[S::kThreads];
};

__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, uint32_t x, uint32_t y, uint32_t z, uint32_t bar,
                                        uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4}], "
      "[%5], %6;" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy)
      : "memory");
}

// D(16x8, f32) += A(16x16, row) * B(16x8, col). Not volatile: products that do not depend on one another are to be
// interleaved by the compiler (all uses are in code that whole warps run through together).
template <bool kBf16>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (kBf16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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

template <uint32_t kTok>
__device__ __forceinline__ Span span_of(const PagedDecodeParams& p, uint32_t i) {
  const int32_t n = p.lens[i];
  Span s{};
  if (n <= 0 || static_cast<uint32_t>(n) > p.max_blocks * p.block_tokens) return s;
  s.len = static_cast<uint32_t>(n);
  s.lo = p.window && p.window < s.len ? s.len - p.window : 0;
  s.first = s.lo / kTok;
  s.chunks = (s.len + kTok - 1) / kTok - s.first;
  return s;
}

template <typename Sh>
__device__ __forceinline__ bool wait_on(uint64_t* bar, uint32_t parity, Sh& sh, int* status) {
  if (ptx::mbar_try_wait(ptx::smem_u32(bar), parity)) return true;
  if (*reinterpret_cast<volatile uint32_t*>(&sh.dead)) return false;
  if (ptx::mbar_wait(ptx::smem_u32(bar), parity, status, kDevTimeout)) return true;
  *reinterpret_cast<volatile uint32_t*>(&sh.dead) = 1;
  return false;
}

// The same for what the CTA's other warps do: however long that takes, as long as it goes on.
template <typename Sh>
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, Sh& sh, int* status) {
  if (ptx::mbar_try_wait(ptx::smem_u32(bar), parity)) return true;
  for (;;) {
    if (*reinterpret_cast<volatile uint32_t*>(&sh.dead)) return false;
    const uint32_t before = *reinterpret_cast<volatile uint32_t*>(&sh.started);
    if (ptx::mbar_wait(ptx::smem_u32(bar), parity, nullptr, 0)) return true;
    if (*reinterpret_cast<volatile uint32_t*>(&sh.started) == before) {
      ptx::report_status(status, kDevTimeout);
      *reinterpret_cast<volatile uint32_t*>(&sh.dead) = 1;
      return false;
    }
  }
}

// Whether the phase has completed: does not wait.
__device__ __forceinline__ bool ready(uint64_t* bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(ptx::smem_u32(bar)), "r"(parity)
      : "memory");
  return done != 0;
}

__device__ __forceinline__ void arrive(uint64_t* bar) { ptx::mbar_arrive(ptx::smem_u32(bar)); }

// The largest weight of a row is 2^kTop: an fp16 number has no bits below 2^-24, and 100 000 weights of 2^-25 beside one of 1
// are 0.3 % of the sum. With 2^15 on top, what is lost is below 2^-40 of the largest weight for each token. (bf16: exponents
// as f32 has them.)
template <bool kBf16>
__device__ constexpr float kTop = kBf16 ? 0.f : 15.f;

// Eight columns (query rows) of an item as a warp holds them: column col0 + 2 * (lane % 4) + j, dims mt * 16 + lane / 4
// and + 8; the columns' largest scores (before the scale) and sums of weights (of all lanes).
template <uint32_t D>
struct Rows {
  float o[D / 16][4];
  float m[2], l[2];
};

// Normalised, combined (differential form) and written.
template <uint32_t D, bool kBf16>
__device__ __forceinline__ void write_out(const PagedDecodeParams& p, Rows<D>& r, uint32_t seq, uint32_t head, uint32_t col0) {
  const uint32_t lane = threadIdx.x & 31u, gid = lane >> 2, tig = lane & 3u;
  constexpr uint32_t kSteps = D / 16;
  const uint32_t G = p.lam ? p.rows / 2 : p.rows;
  uint8_t* out = p.out + static_cast<uint64_t>(seq) * p.out_stride + static_cast<uint64_t>(head) * G * D * 2;
  const uint64_t first_head = (static_cast<uint64_t>(seq) * p.num_kv_heads + head) * G;
  float inv[2];
#pragma unroll
  for (uint32_t j = 0; j < 2; ++j) {
    const float s = r.l[j];
    inv[j] = s > 0.f ? 1.f / s : s;  // no weight at all: a row of zeros; not a number stays one
  }
  if (!p.lam) {
#pragma unroll
    for (uint32_t j = 0; j < 2; ++j) {
      const uint32_t g = col0 + 2 * tig + j;
      if (p.lse && gid == 0 && g < G) p.lse[first_head + g] = fmaf(r.m[j], p.scale_log2, log2f(r.l[j]) - kTop<kBf16>) * 0.6931471805599453f;
    }
    uint32_t* dst = reinterpret_cast<uint32_t*>(out + static_cast<uint64_t>(col0 + gid) * D * 2) + tig;
#pragma unroll
    for (uint32_t mt = 0; mt < kSteps; ++mt) {
      const float(&v)[4] = r.o[mt];
      // [dim][column] pairs become [column][dim] pairs
      const uint32_t a = ptx::movmatrix_trans(pack<kBf16>(v[0] * inv[0], v[1] * inv[1]));
      const uint32_t b = ptx::movmatrix_trans(pack<kBf16>(v[2] * inv[0], v[3] * inv[1]));
      if (col0 + gid < G) {
        dst[mt * 8] = a;
        dst[mt * 8 + 4] = b;
      }
    }
  } else {
    const uint32_t g = col0 / 2 + tig;  // columns 2 tig and 2 tig + 1 are the two maps of this head
    inv[1] *= g < G ? p.lam[head * G + g] : 0.f;
    float sq = 0.f;
#pragma unroll
    for (uint32_t mt = 0; mt < kSteps; ++mt) {
      float(&v)[4] = r.o[mt];
      // two rounded products (not a fused one): equal maps with a weight of 1 leave exactly nothing
      v[0] = __fsub_rn(__fmul_rn(v[0], inv[0]), __fmul_rn(v[1], inv[1]));
      v[2] = __fsub_rn(__fmul_rn(v[2], inv[0]), __fmul_rn(v[3], inv[1]));
      sq = fmaf(v[0], v[0], fmaf(v[2], v[2], sq));
    }
    float f = p.out_scale;
    if (p.norm_weight) {
#pragma unroll
      for (int s = 4; s <= 16; s <<= 1) sq += __shfl_xor_sync(0xffffffffu, sq, s);
      f *= rsqrtf(sq * (1.f / D) + p.eps);
#pragma unroll
      for (uint32_t mt = 0; mt < kSteps; ++mt) {
        r.o[mt][0] *= p.norm_weight[mt * 16 + gid];
        r.o[mt][2] *= p.norm_weight[mt * 16 + 8 + gid];
      }
    }
    // pairs (dim, dim + 8) of head tig become, in lane 8 h + 4 half + t, dims 8 half + 2 t and + 1 of head h
    uint32_t* dst = reinterpret_cast<uint32_t*>(out + static_cast<uint64_t>(col0 / 2 + (gid >> 1)) * D * 2) + (gid & 1u) * 4 + tig;
#pragma unroll
    for (uint32_t mt = 0; mt < kSteps; ++mt) {
      const uint32_t a = ptx::movmatrix_trans(pack<kBf16>(r.o[mt][0] * f, r.o[mt][2] * f));
      if (col0 / 2 + (gid >> 1) < G) dst[mt * 8] = a;
    }
  }
}

// Partial rows, as the lanes hold them. Lanes whose columns are padding neither store nor load.
template <uint32_t D>
__device__ __forceinline__ void store_part(const PagedDecodeParams& p, const Rows<D>& r, uint32_t col0, float* part) {
  const uint32_t lane = threadIdx.x & 31u, tig = lane & 3u;
  constexpr uint32_t kSteps = D / 16;
  if (col0 + 2 * tig >= p.rows) return;
#pragma unroll
  for (uint32_t mt = 0; mt < kSteps; ++mt)
    reinterpret_cast<float4*>(part)[mt * 32 + lane] = make_float4(r.o[mt][0], r.o[mt][1], r.o[mt][2], r.o[mt][3]);
  if (lane < 4)
    reinterpret_cast<float4*>(part + 8 * D)[tig] = make_float4(r.m[0], r.l[0], r.m[1], r.l[1]);
}

// r and the partial rows at `part` become the rows of both.
template <uint32_t D>
__device__ __forceinline__ void add_part(const PagedDecodeParams& p, Rows<D>& r, uint32_t col0, const float* part) {
  const uint32_t lane = threadIdx.x & 31u, tig = lane & 3u;
  constexpr uint32_t kSteps = D / 16;
  if (col0 + 2 * tig >= p.rows) return;
  const float4 ml = reinterpret_cast<const float4*>(part + 8 * D)[tig];
  const float pm[2] = {ml.x, ml.z}, pl[2] = {ml.y, ml.w};
  float mine[2], theirs[2];
#pragma unroll
  for (uint32_t j = 0; j < 2; ++j) {
    const float top = fmaxf(r.m[j], pm[j]), safe = top == kMinusInf ? 0.f : top;
    mine[j] = ptx::exp2_approx((r.m[j] - safe) * p.scale_log2);
    theirs[j] = ptx::exp2_approx((pm[j] - safe) * p.scale_log2);
    r.l[j] = r.l[j] * mine[j] + pl[j] * theirs[j];
    r.m[j] = top;
  }
#pragma unroll
  for (uint32_t mt = 0; mt < kSteps; ++mt) {
    const float4 v = reinterpret_cast<const float4*>(part)[mt * 32 + lane];
    float(&o)[4] = r.o[mt];
    o[0] = o[0] * mine[0] + v.x * theirs[0];
    o[1] = o[1] * mine[1] + v.y * theirs[1];
    o[2] = o[2] * mine[0] + v.z * theirs[0];
    o[3] = o[3] * mine[1] + v.w * theirs[1];
  }
}

template <uint32_t D>
__device__ __forceinline__ void clear(Rows<D>& r) {
  r.m[0] = r.m[1] = kMinusInf;
  r.l[0] = r.l[1] = 0.f;
#pragma unroll
  for (uint32_t mt = 0; mt < D / 16; ++mt) r.o[mt][0] = r.o[mt][1] = r.o[mt][2] = r.o[mt][3] = 0.f;
}

// Query rows as the narrow operand: column n = row of the item, 16 dims per step. A scale below 0 is applied to the
// signs here, a scale of 0 makes the rows zeros: the softmax sees a scale above 0.
template <uint32_t D>
__device__ __forceinline__ void load_q(const PagedDecodeParams& p, uint32_t seq, uint32_t head, uint32_t col0, uint32_t (&qf)[D / 16][2]) {
  const uint32_t lane = threadIdx.x & 31u, gid = lane >> 2, tig = lane & 3u;
  const bool diff = p.lam != nullptr;
  const uint32_t width = diff ? D / 2 : D;
  const uint8_t* q = p.q + static_cast<uint64_t>(seq) * p.q_stride + static_cast<uint64_t>(head) * p.rows * width * 2;
  const uint32_t n = col0 + gid;
  const uint32_t shift = diff && (n & 1u) ? D / 2 : 0;  // where the row's dims start in K
  const uint8_t* row = q + static_cast<uint64_t>(n) * width * 2;
#pragma unroll
  for (uint32_t ks = 0; ks < D / 16; ++ks)
#pragma unroll
    for (uint32_t hh = 0; hh < 2; ++hh) {
      const uint32_t d = ks * 16 + hh * 8 + tig * 2;
      qf[ks][hh] = n < p.rows && d >= shift && d - shift < width
                           ? (*reinterpret_cast<const uint32_t*>(row + (d - shift) * 2) & p.q_keep) ^ p.q_flip
                           : 0u;
    }
}

// The weight of score x (before the scale) beside the largest one, top: the difference is taken first, since of scores beyond
// 2^24 the rounding of x scale alone is more than an exponent's worth. (Against exp2(x scale - m) with a scaled
// maximum, one instruction less: 64 sequences of up to 4095 tokens 101.6 us against 101.1, one of 500 11.6 against 11.5.)
template <bool kBf16>
__device__ __forceinline__ float weight(float x, float top, float scale) {
  return ptx::exp2_approx(fmaf(x - top, scale, kTop<kBf16>));
}

// One chunk: scores, softmax, product with V. `tok0` = position of its first token. p.scale_log2 is above 0 (load_q).
template <uint32_t D, bool kBf16>
__device__ __forceinline__ void take_chunk(const PagedDecodeParams& p, uint32_t lo_tok, uint32_t end_tok, uint32_t tok0, const uint8_t* stage,
                                           const uint32_t (&qf)[D / 16][2], Rows<D>& r) {
  constexpr uint32_t kTok = kHalf / (2 * D), kSub = kTok / 16, kSteps = D / 16;
  const uint32_t lane = threadIdx.x & 31u, gid = lane >> 2, tig = lane & 3u, mj = lane >> 3, mr = lane & 7u;
  const bool whole = tok0 >= lo_tok && tok0 + kTok <= end_tok;

  // Unit 2 ks + h of row r lies at r * 2 D + (ks / 4) * 128 + ((2 (ks & 3) + h) ^ (r & 7)) * 16: the step's part of the
  // exclusive or is a constant, the rest one address per lane (rows of the sub-tiles are 16 apart: same r & 7).
  const uint32_t kaddr = ptx::smem_u32(stage) + ((mj & 1u) * 8 + mr) * (2 * D) + (((mj >> 1) ^ mr) << 4);
  const uint32_t vaddr = ptx::smem_u32(stage) + kHalf + ((mj >> 1) * 8 + mr) * (2 * D) + (((mj & 1u) ^ mr) << 4);

  // A warp has few products at a time that do not depend on one another: the dims are summed in kChains parts.
  constexpr uint32_t kChains = kSub >= 4 ? 1 : 4 / kSub;
  float s[kSub][4], more[kChains][kSub][4];
#pragma unroll
  for (uint32_t ch = 0; ch < kChains; ++ch)
#pragma unroll
    for (uint32_t sub = 0; sub < kSub; ++sub)
      more[ch][sub][0] = more[ch][sub][1] = more[ch][sub][2] = more[ch][sub][3] = 0.f;
#pragma unroll
  for (uint32_t ks = 0; ks < kSteps; ++ks)
#pragma unroll
    for (uint32_t sub = 0; sub < kSub; ++sub) {
      uint32_t f[4];
      ptx::ldmatrix_x4(f, (kaddr ^ ((ks & 3) << 5)) + (ks >> 2) * 128 + sub * 16 * 2 * D);
      mma<kBf16>(more[ks % kChains][sub], f, qf[ks][0], qf[ks][1]);
    }
#pragma unroll
  for (uint32_t sub = 0; sub < kSub; ++sub)
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
      s[sub][e] = more[0][sub][e];
#pragma unroll
      for (uint32_t ch = 1; ch < kChains; ++ch) s[sub][e] += more[ch][sub][e];
    }
  if (!whole) {
#pragma unroll
    for (uint32_t sub = 0; sub < kSub; ++sub) {
      const uint32_t ta = tok0 + sub * 16 + gid, tb = ta + 8;
      const bool in_a = ta >= lo_tok && ta < end_tok, in_b = tb >= lo_tok && tb < end_tok;
      float(&x)[4] = s[sub];
      x[0] = in_a ? x[0] : kMinusInf;
      x[1] = in_a ? x[1] : kMinusInf;
      x[2] = in_b ? x[2] : kMinusInf;
      x[3] = in_b ? x[3] : kMinusInf;
    }
  }
  float mx[2];
#pragma unroll
  for (uint32_t j = 0; j < 2; ++j) {
    mx[j] = fmaxf(s[0][j], s[0][2 + j]);
#pragma unroll
    for (uint32_t sub = 1; sub < kSub; ++sub) mx[j] = fmaxf(mx[j], fmaxf(s[sub][j], s[sub][2 + j]));
  }
#pragma unroll
  for (int x = 4; x <= 16; x <<= 1)
#pragma unroll
    for (uint32_t j = 0; j < 2; ++j) mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], x));
  bool moved = false;
#pragma unroll
  for (uint32_t j = 0; j < 2; ++j) {
    mx[j] = fmaxf(r.m[j], mx[j]);
    moved |= mx[j] != r.m[j];
  }
  if (__any_sync(0xffffffffu, moved)) {
    float al[2];
#pragma unroll
    for (uint32_t j = 0; j < 2; ++j) {
      al[j] = mx[j] == kMinusInf ? 1.f : ptx::exp2_approx((r.m[j] - mx[j]) * p.scale_log2);
      r.m[j] = mx[j];
      r.l[j] *= al[j];
    }
#pragma unroll
    for (uint32_t mt = 0; mt < kSteps; ++mt) {
      r.o[mt][0] *= al[0];
      r.o[mt][1] *= al[1];
      r.o[mt][2] *= al[0];
      r.o[mt][3] *= al[1];
    }
  }
#pragma unroll
  for (uint32_t j = 0; j < 2; ++j) mx[j] = mx[j] == kMinusInf ? 0.f : mx[j];  // no finite score so far: every weight is 0
#pragma unroll
  for (uint32_t sub = 0; sub < kSub; ++sub) {
    const uint32_t t16 = tok0 + sub * 16;
    if (!whole && (t16 >= end_tok || t16 + 16 <= lo_tok)) continue;
    uint32_t hi[2], lo[2];
    const float(&x)[4] = s[sub];
    const float p0 = weight<kBf16>(x[0], mx[0], p.scale_log2), p1 = weight<kBf16>(x[1], mx[1], p.scale_log2);
    const float p2 = weight<kBf16>(x[2], mx[0], p.scale_log2), p3 = weight<kBf16>(x[3], mx[1], p.scale_log2);
    r.l[0] += p0 + p2;  // this lane's tokens; the lanes' sums are added at the end of the piece
    r.l[1] += p1 + p3;
    const uint32_t h01 = pack<kBf16>(p0, p1), h23 = pack<kBf16>(p2, p3);
    const float2 r01 = unpack<kBf16>(h01), r23 = unpack<kBf16>(h23);
    hi[0] = ptx::movmatrix_trans(h01);
    hi[1] = ptx::movmatrix_trans(h23);
    lo[0] = ptx::movmatrix_trans(pack<kBf16>(p0 - r01.x, p1 - r01.y));
    lo[1] = ptx::movmatrix_trans(pack<kBf16>(p2 - r23.x, p3 - r23.y));
    if (whole || (t16 >= lo_tok && t16 + 16 <= end_tok)) {
#pragma unroll
      for (uint32_t mt = 0; mt < kSteps; ++mt) {
        uint32_t f[4];
        ptx::ldmatrix_x4_trans(f, (vaddr ^ ((mt & 3) << 5)) + (mt >> 2) * 128 + sub * 16 * 2 * D);
        mma<kBf16>(r.o[mt], f, hi[0], hi[1]);
        mma<kBf16>(r.o[mt], f, lo[0], lo[1]);
      }
    } else {
      // Token pairs (2 tig, 2 tig + 1) and (+8, +9): rows of V outside [lo, end) are taken as zeros, whatever they hold.
      const uint32_t tk = t16 + 2 * tig;
      auto in = [&](uint32_t x) { return x >= lo_tok && x < end_tok; };
      const uint32_t keep_lo = (in(tk) ? 0x0000ffffu : 0u) | (in(tk + 1) ? 0xffff0000u : 0u);
      const uint32_t keep_hi = (in(tk + 8) ? 0x0000ffffu : 0u) | (in(tk + 9) ? 0xffff0000u : 0u);
#pragma unroll
      for (uint32_t mt = 0; mt < kSteps; ++mt) {
        uint32_t f[4];
        ptx::ldmatrix_x4_trans(f, (vaddr ^ ((mt & 3) << 5)) + (mt >> 2) * 128 + sub * 16 * 2 * D);
        f[0] &= keep_lo;
        f[1] &= keep_lo;
        f[2] &= keep_hi;
        f[3] &= keep_hi;
        mma<kBf16>(r.o[mt], f, hi[0], hi[1]);
        mma<kBf16>(r.o[mt], f, lo[0], lo[1]);
      }
    }
  }
}

// How items are cut. The line of all chunks has three zones; an item is cut evenly into pieces of about the size of the
// zone it begins in: coarse ones first (every piece costs a merge, and every cut item a join), fine ones at the end, which
// make up for the CTAs that are behind. Items shorter than two pieces stay whole.
struct Zones {
  unsigned long long end[2];  // of the first and of the second zone
  uint32_t size[3];
};

// One sequence: heads that begin in the first zone, in the first two, and pieces of an item of each zone.
struct Cut {
  uint32_t heads[2], pieces[3];
  uint32_t all, parts;        // of all heads; and of those that are cut
};

// `at` = the line's chunk at which the sequence's first item begins.
__device__ __forceinline__ Cut cut_of(const Zones& zones, unsigned long long at, uint32_t chunks, uint32_t heads) {
  Cut c;
  c.heads[0] = c.heads[1] = heads;
  c.pieces[0] = c.pieces[1] = c.pieces[2] = chunks ? 1 : 0;
  c.all = chunks ? heads : 0;
  c.parts = 0;
  if (chunks < 2 * zones.size[2]) return c;
  const unsigned long long end = at + static_cast<unsigned long long>(chunks) * heads;
#pragma unroll
  for (uint32_t z = 0; z < 2; ++z)
    c.heads[z] = zones.end[z] <= at ? 0 : zones.end[z] >= end ? heads : static_cast<uint32_t>((zones.end[z] - at + chunks - 1) / chunks);
#pragma unroll
  for (uint32_t z = 0; z < 3; ++z) c.pieces[z] = chunks < 2 * zones.size[z] ? 1 : chunks / zones.size[z];
  const uint32_t n[3] = {c.heads[0], c.heads[1] - c.heads[0], heads - c.heads[1]};
  c.all = 0;
#pragma unroll
  for (uint32_t z = 0; z < 3; ++z) {
    c.all += n[z] * c.pieces[z];
    c.parts += c.pieces[z] > 1 ? n[z] * c.pieces[z] : 0;
  }
  return c;
}

// Pieces of the item of head `head`.
__device__ __forceinline__ uint32_t pieces_of(const Cut& c, uint32_t head) {
  return head < c.heads[0] ? c.pieces[0] : head < c.heads[1] ? c.pieces[1] : c.pieces[2];
}

// Short work of few items (fewer than two to a CTA) is dealt out evenly instead. On the line of all chunks an item takes `least`
// at least: a CTA is rather given one short item than several, each of which costs a round of its own (16 sequences of 1 to 600
// tokens, 8 KV heads: 13.6 us against 16.3; one of 30 7.3 against 13.2). CTA k takes what lies from k * size on, up to the next
// one's. A cut that would leave less than `least` chunks of an item on one side of it is moved to that end of the item.
struct Even {
  uint32_t size, least;         // size 0: not dealt out
};

__device__ __forceinline__ uint32_t room_of(uint32_t chunks, uint32_t least) { return chunks ? max(chunks, least) : 0; }

// The item of `chunks` chunks that begins at `at` of the line: it begins in CTA `owner`'s range, and goes on in that of the `cuts` next ones.
struct Share {
  uint32_t owner, cuts;
};

__device__ __forceinline__ Share share_of(const Even& even, unsigned long long at, uint32_t chunks) {
  Share r;
  r.owner = static_cast<uint32_t>((at + even.least + even.size - 1) / even.size) - 1;
  r.cuts = 0;
  if (chunks >= 2 * even.least) {
    const uint32_t last = static_cast<uint32_t>((at + chunks - even.least) / even.size);  // the last cut that is not moved to the item's end
    if (last > r.owner) r.cuts = last - r.owner;
  }
  return r;
}

// Tickets drawn at a time when so many pieces are left.
__device__ __forceinline__ uint32_t batch_of(uint32_t pieces, uint32_t most) {
  const uint32_t each = pieces / (gridDim.x * 4);
  return each < 1 ? 1 : each < most ? each : most;
}

template <uint32_t D, uint32_t NT>
__device__ void schedule(const PagedDecodeParams& p, Shared<D, NT>& sh, const Zones& zones, const Even& even, uint32_t pieces, uint32_t batch, uint32_t most, bool many) {
  using S = Shape<D, NT>;
  constexpr uint32_t kTok = kHalf / (2 * D);
  const uint32_t lane = threadIdx.x & 31u;
  const uint32_t run = (p.nseq + S::kThreads - 1) / S::kThreads;
  uint32_t number = 0, turn = 0, tail = 0;    // chunks so far; whose turn it is; the oldest piece not known to be finished
  const uint32_t first = gridDim.x * batch;   // tickets that are nobody's to draw: every CTA has a batch to begin with
  uint32_t ticket = blockIdx.x * batch, left = batch;
  // where the ticket is: sequence, head, piece of the item, and what was before the item
  uint32_t seq = 0, head = 0, index = 0, count = 0, parts = 0;
  unsigned long long at = 0;  // chunks of the line before the sequence
  Span span{};
  Cut cut{};
  bool found = false;
  for (uint32_t j = 0;; ++j) {
    // Not too far ahead: what is drawn here cannot be drawn by a CTA that is faster. The consumers count the chunks that they
    // have started copies of.
    uint64_t t0 = 0;
    uint32_t seen = 0;
    for (uint32_t polls = 0; j && !even.size; ++polls) {
      const uint32_t started = *reinterpret_cast<volatile uint32_t*>(&sh.started);
      if (static_cast<int32_t>(number - started) < static_cast<int32_t>(kAhead)) break;
      if (*reinterpret_cast<volatile uint32_t*>(&sh.dead)) return;
      if (polls == 0 || started != seen) {
        t0 = ptx::global_timer_ns();
        seen = started;
      } else if ((polls & 63u) == 63u && ptx::global_timer_ns() - t0 > 4000000000ull) {  // longer than the consumers' own waits
        *reinterpret_cast<volatile uint32_t*>(&sh.dead) = 1;
        ptx::report_status(p.status, kDevTimeout);
        return;
      }
      __nanosleep(100);
    }
    __syncwarp();
    while (j - tail >= kNotes) {
      if (!__all_sync(0xffffffffu, wait_for(&sh.note_empty[tail % kNotes], tail / kNotes & 1u, sh, p.status))) return;
      ++tail;
    }
    Note& note = sh.note[j % kNotes];
    uint32_t a, b, slot, step;
    if (even.size) {
      const uint32_t me = blockIdx.x;
      const unsigned long long from = static_cast<unsigned long long>(me) * even.size;
      unsigned long long start = 0;
      bool have = false;
      Share share{};
      while (!have) {
        if (!found) {  // the item in which the range begins
          uint32_t x = 0, n = S::kThreads;  // the last run of sequences that begins there or before
          while (n > 1) {
            const uint32_t half = n >> 1;
            if (sh.chunks_before[x + half] <= from) x += half;
            n -= half;
          }
          at = sh.chunks_before[x];
          for (seq = x * run; seq < p.nseq; ++seq) {
            span = span_of<kTok>(p, seq);
            const unsigned long long all = static_cast<unsigned long long>(room_of(span.chunks, even.least)) * p.num_kv_heads;
            if (from < at + all) break;
            at += all;
          }
          if (seq < p.nseq) head = static_cast<uint32_t>((from - at) / room_of(span.chunks, even.least));
          found = true;
        } else if (++head == p.num_kv_heads) {
          head = 0;
          at += static_cast<unsigned long long>(room_of(span.chunks, even.least)) * p.num_kv_heads;
          do {
            ++seq;
            if (seq < p.nseq) span = span_of<kTok>(p, seq);
          } while (seq < p.nseq && span.chunks == 0);
        }
        if (seq >= p.nseq) break;
        start = at + static_cast<unsigned long long>(head) * room_of(span.chunks, even.least);
        share = share_of(even, start, span.chunks);
        if (share.owner > me) break;
        index = me - share.owner;
        have = index <= share.cuts;  // else its end was moved to where the range begins
      }
      if (!have) {
        if (lane == 0) {
          note.chunks = 0;
          arrive(&sh.note_full[j % kNotes]);
        }
        return;
      }
      count = share.cuts + 1;
      a = index ? static_cast<uint32_t>(from - start) : 0;
      b = index < share.cuts ? static_cast<uint32_t>(from + even.size - start) : span.chunks;
      slot = 2 * share.owner;  // of a CTA's two: the first one for an item that goes on there, the second one for one that begins there
      step = 2;
    } else {
    if (left == 0) {
      // A draw takes longer than a small piece: several at a time, fewer as the end comes nearer.
      const uint32_t rest = pieces > ticket ? pieces - ticket : 0;
      batch = batch_of(rest, most);
      uint32_t drawn = 0;
      if (lane == 0) drawn = atomicAdd(p.counters + kPagedTicket, batch);
      ticket = first + __shfl_sync(0xffffffffu, drawn, 0);
      left = batch;
      found = false;
    }
    if (ticket >= pieces) {
      if (lane == 0) {
        note.chunks = 0;
        arrive(&sh.note_full[j % kNotes]);
      }
      return;
    }
    if (!found) {
      // The run of sequences it lies in, then the sequence, the head and the piece.
      uint32_t x = 0, n = S::kThreads;  // the last run that begins at or before the ticket
      while (n > 1) {
        const uint32_t half = n >> 1;
        if (sh.pieces_before[x + half] <= ticket) x += half;
        n -= half;
      }
      uint32_t before = sh.pieces_before[x];
      parts = sh.parts_before[x];
      at = sh.chunks_before[x];
      for (seq = x * run; seq < p.nseq; ++seq) {
        span = span_of<kTok>(p, seq);
        cut = cut_of(zones, at, span.chunks, p.num_kv_heads);
        if (ticket < before + cut.all) break;
        before += cut.all;
        parts += cut.parts;
        at += static_cast<unsigned long long>(span.chunks) * p.num_kv_heads;
      }
      if (seq == p.nseq) {  // only if the lengths have changed since they were added up: no more is read
        if (lane == 0) {
          ptx::report_status(p.status, kStatusInvalid);
          note.chunks = 0;
          arrive(&sh.note_full[j % kNotes]);
        }
        return;
      }
      head = 0;
      index = ticket - before;
#pragma unroll
      for (uint32_t z = 0; z < 3; ++z) {  // heads of the zone that come before the ticket's
        const uint32_t n = (z == 2 ? p.num_kv_heads : cut.heads[z]) - (z ? cut.heads[z - 1] : 0u);
        const uint32_t whole = min(n, index / cut.pieces[z]);
        if (head == (z ? cut.heads[z - 1] : 0u)) {
          head += whole;
          index -= whole * cut.pieces[z];
          parts += cut.pieces[z] > 1 ? whole * cut.pieces[z] : 0;
        }
      }
      count = pieces_of(cut, head);
      found = true;
    } else if (++index == count) {  // the ticket after the last one
      index = 0;
      if (count > 1) parts += count;
      if (++head == p.num_kv_heads) {
        head = 0;
        do {
          at += static_cast<unsigned long long>(span.chunks) * p.num_kv_heads;
          ++seq;
          span = seq < p.nseq ? span_of<kTok>(p, seq) : Span{0, 0, 0, 1};
        } while (span.chunks == 0);  // there is one: the ticket exists
        if (seq == p.nseq) {
          if (lane == 0) {
            ptx::report_status(p.status, kStatusInvalid);
            note.chunks = 0;
            arrive(&sh.note_full[j % kNotes]);
          }
          return;
        }
        cut = cut_of(zones, at, span.chunks, p.num_kv_heads);
      }
      count = pieces_of(cut, head);
    }
    a = static_cast<uint32_t>(static_cast<uint64_t>(span.chunks) * index / count);
    b = static_cast<uint32_t>(static_cast<uint64_t>(span.chunks) * (index + 1) / count);
    slot = parts;
    step = 1;
    ++ticket;
    --left;
    }
    if (count > 1 && (slot > kPagedMaxParts || count > (kPagedMaxParts - slot) / step)) {  // as above: never with lengths that stay as they are
      if (lane == 0) {
        ptx::report_status(p.status, kStatusInvalid);
        note.chunks = 0;
        arrive(&sh.note_full[j % kNotes]);
      }
      return;
    }
    const bool solo = count == 1 && (b <= 2 || (many && b <= kSolo));
    if (lane == 0) {
      note.seq = seq;
      note.head = head;
      note.lo = span.lo;
      note.len = span.len;
      note.chunk = span.first + a;
      note.chunks = b - a;
      note.turn = turn;
      note.solo = solo;
      note.index = index;
      note.count = count;
      note.slot = slot;
      note.step = step;
      arrive(&sh.note_full[j % kNotes]);
    }
    __syncwarp();
    number += solo ? 1 : b - a;
    turn = (turn + (solo ? 1 : b - a)) % S::kWarps;
  }
}

// A consumer warp's first chunk of a piece (none if that is not below note.chunks).
template <uint32_t kWarps>
__device__ __forceinline__ uint32_t first_chunk(const Note& note, uint32_t warp) {
  const uint32_t after = warp >= note.turn ? warp - note.turn : warp + kWarps - note.turn;
  return note.solo && after ? ~0u - 64u : after;
}

// The copying side of a consumer warp (of the first group): runs ahead of the work by up to kDepth chunks, into the next pieces as far as they
// are known. A chunk is 1, 2 or 4 copies of K and as many of V (blocks of at least its tokens: one); the lanes hold the
// next 32 copies' blocks. (Every quantity that divides is a power of two and used as a shift: the integer divisions
// were a fifth of all instructions.)
template <uint32_t D, uint32_t NT>
struct Feed {
  using S = Shape<D, NT>;
  static constexpr uint32_t kTok = kHalf / (2 * D), kTokShift = D == 64 ? 6 : D == 128 ? 5 : 4;
  uint32_t box_shift;           // log2 of the token rows of one copy
  uint32_t split;               // log2 of the copies of a chunk's half
  uint32_t j;                   // piece
  uint32_t c, chunks, step;     // next chunk of this warp in it, the piece's length, and from one of its chunks to the next
  uint32_t k;                   // c is chunk number k of those whose copies the lanes hold
  uint32_t seq, lo, len, chunk;
  uint32_t x, row;              // this lane's copy: first element and token row
  int32_t entry;                // and the table's entry for it
  uint32_t boxes;               // which lanes have one
  bool end;

  __device__ void init(const PagedDecodeParams& p) {
    box_shift = p.block_shift < kTokShift ? p.block_shift : kTokShift;
    split = kTokShift - box_shift;
  }

  __device__ void open(const Note& note, uint32_t piece) {
    j = piece;
    end = note.chunks == 0;
    chunks = note.chunks;
    seq = note.seq;
    x = note.head * D;
    lo = note.lo;
    len = note.len;
    chunk = note.chunk;
    step = note.solo ? 1u : S::kWarps;
    c = first_chunk<S::kWarps>(note, threadIdx.x >> 5);
    k = 32;
  }

  // Lane `lane` takes copy lane mod 2^split of this warp's chunk number lane >> split from c on: wanted if one of its token
  // rows is in [lo, len).
  __device__ void look(const PagedDecodeParams& p, uint32_t lane) {
    const uint32_t mine = c + (lane >> split) * step;
    const uint32_t t = (chunk + mine) * kTok + ((lane & ((1u << split) - 1)) << box_shift);
    const bool on = mine < chunks && t < len && t + (1u << box_shift) > lo;
    k = 0;
    entry = on ? p.tables[static_cast<uint64_t>(seq) * p.table_stride + (t >> p.block_shift)] : 0;
    row = t & (p.block_tokens - 1);
    boxes = __ballot_sync(0xffffffffu, on);
  }

  // Reads the entries of a piece just opened, before anything else waits.
  __device__ void prepare(const PagedDecodeParams& p) {
    if (!end && c < chunks && k >= 32u >> split) look(p, threadIdx.x & 31u);
  }

  // Starts the copies of the next chunk, if there is one yet.
  __device__ bool issue(const PagedDecodeParams& p, const Maps& maps, Shared<D, NT>& sh, uint32_t stage, uint64_t policy) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    while (!end && c >= chunks) {  // the next piece, unless it is not known yet: nobody waits for it here
      const uint32_t next = j + 1;
      if (!__all_sync(0xffffffffu, ready(&sh.note_full[next % kNotes], next / kNotes & 1u))) return false;
      open(sh.note[next % kNotes], next);
      if (!end && c < chunks) {  // its query rows will be wanted soon
        const uint32_t width = p.lam ? D / 2 : D, line = lane * 128;
        if (line < p.rows * width * 2)
          asm volatile("prefetch.global.L1 [%0];" ::"l"(p.q + static_cast<uint64_t>(seq) * p.q_stride + static_cast<uint64_t>(x / D) * p.rows * width * 2 + line));
      }
    }
    if (end) return false;
    if (k >= 32u >> split) look(p, lane);
    const uint32_t group = (boxes >> (k << split)) & ((1u << (1u << split)) - 1);
    const uint32_t bar = ptx::smem_u32(&sh.full[warp][stage]);
    if (lane == 0) {
      if (step > 1 || c == 0) atomicAdd(&sh.started, 1u);
      ptx::mbar_arrive_expect_tx(bar, static_cast<uint32_t>(__popc(group)) << (box_shift + 1) << (kTokShift == 6 ? 7 : kTokShift == 5 ? 8 : 9));
    }
    __syncwarp();
    if ((lane >> split) == k && (boxes >> lane & 1u)) {
      const uint32_t dst = ptx::smem_u32(sh.stage[warp][stage]) + (((lane & ((1u << split) - 1)) << box_shift) * (D * 2));
      const bool second = entry < 0;
      const uint32_t blocks = second ? p.blocks[1] : p.blocks[0];
      uint32_t id = static_cast<uint32_t>(second ? ~entry : entry);
      if (id >= blocks) {  // a bad page: reads as zeros (a box outside the tensor), and is reported
        ptx::report_status(p.status, kStatusInvalid);
        id = blocks ? blocks : second ? p.blocks[0] : p.blocks[1];  // of an arena without blocks the map is the other one's
      }
      const CUtensorMap* map = second ? &maps.m[1] : &maps.m[0];
      tma_box(dst, map, x, row, id, bar, policy);
      tma_box(dst + kHalf, map, x, p.block_tokens + row, id, bar, policy);
    }
    c += step;
    ++k;
    return true;
  }
};

// A group's part of a slot of the workspace.
template <uint32_t D, uint32_t NT>
__device__ __forceinline__ float* part_of(const PagedDecodeParams& p, uint32_t slot, uint32_t group) {
  return p.parts + (static_cast<uint64_t>(slot) * NT + group) * Shape<D, NT>::kPart;
}

// Adds the parts of slots slot + odd, slot + stride, slot + 2 * stride, .. (`count` of them, at most kFan) in that order: of the
// D / 16 tiles of a row, first, first + step, .. into sh.joined, and the columns' maxima and sums into m and l. `go_on` is asked
// before the tiles, two at a time. A lane reads the maxima and sums of every eighth part; the first tiles are read meanwhile.
template <uint32_t D, uint32_t NT, typename GoOn>
__device__ __forceinline__ void sum_parts(const PagedDecodeParams& p, Shared<D, NT>& sh, uint32_t group, uint32_t slot, uint32_t odd,
                                          uint32_t stride, uint32_t count, uint32_t first, uint32_t step, float (&m)[2], float (&l)[2], GoOn go_on) {
  const uint32_t lane = threadIdx.x & 31u, gid = lane >> 2, tig = lane & 3u;
  constexpr uint32_t kSteps = D / 16, kOwn = kFan / 8, kTiles = NT == 1 ? 2 : 1;  // as far as the registers go
  const bool used = group * 8 + 2 * tig < p.rows;
  auto part = [&](uint32_t c) { return reinterpret_cast<const float4*>(part_of<D, NT>(p, slot + (c ? c * stride : odd), group)); };
  float4 ml[kOwn];
#pragma unroll
  for (uint32_t i = 0; i < kOwn; ++i)
    ml[i] = used && gid + 8 * i < count ? __ldcg(part(gid + 8 * i) + 2 * D + tig) : make_float4(kMinusInf, 0.f, kMinusInf, 0.f);
  float w[kOwn][2];
  auto weigh = [&] {
    m[0] = m[1] = kMinusInf;
    l[0] = l[1] = 0.f;
#pragma unroll
    for (uint32_t i = 0; i < kOwn; ++i) {
      m[0] = fmaxf(m[0], ml[i].x);
      m[1] = fmaxf(m[1], ml[i].z);
    }
#pragma unroll
    for (int x = 4; x <= 16; x <<= 1)
#pragma unroll
      for (uint32_t j = 0; j < 2; ++j) m[j] = fmaxf(m[j], __shfl_xor_sync(0xffffffffu, m[j], x));
    const float s0 = m[0] == kMinusInf ? 0.f : m[0], s1 = m[1] == kMinusInf ? 0.f : m[1];
#pragma unroll
    for (uint32_t i = 0; i < kOwn; ++i) {
      w[i][0] = ptx::exp2_approx((ml[i].x - s0) * p.scale_log2);
      w[i][1] = ptx::exp2_approx((ml[i].z - s1) * p.scale_log2);
      l[0] = fmaf(ml[i].y, w[i][0], l[0]);
      l[1] = fmaf(ml[i].w, w[i][1], l[1]);
    }
#pragma unroll
    for (int x = 4; x <= 16; x <<= 1)
#pragma unroll
      for (uint32_t j = 0; j < 2; ++j) l[j] += __shfl_xor_sync(0xffffffffu, l[j], x);
  };
  uint32_t tile = first;
#pragma unroll 1
  for (; tile < kSteps && go_on(tile); tile += step * kTiles) {
    float4 acc[kTiles];
#pragma unroll
    for (uint32_t i = 0; i < kTiles; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (uint32_t c0 = 0; c0 < count; c0 += 16) {
      float4 v[kTiles][16];
#pragma unroll
      for (uint32_t i = 0; i < kTiles; ++i) {
        const uint32_t x = tile + i * step;
#pragma unroll
        for (uint32_t c = 0; c < 16; ++c)
          v[i][c] = used && c0 + c < count && x < kSteps ? __ldcg(part(c0 + c) + x * 32 + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      if (tile == first && c0 == 0) weigh();
#pragma unroll
      for (uint32_t c = 0; c < 16; ++c) {
        const uint32_t from = (c & 7u) * 4 + tig, k = c >> 3;
        const float w0 = __shfl_sync(0xffffffffu, c0 ? w[k + 2][0] : w[k][0], from), w1 = __shfl_sync(0xffffffffu, c0 ? w[k + 2][1] : w[k][1], from);
#pragma unroll
        for (uint32_t i = 0; i < kTiles; ++i) {
          acc[i].x = fmaf(v[i][c].x, w0, acc[i].x);
          acc[i].y = fmaf(v[i][c].y, w1, acc[i].y);
          acc[i].z = fmaf(v[i][c].z, w0, acc[i].z);
          acc[i].w = fmaf(v[i][c].w, w1, acc[i].w);
        }
      }
    }
#pragma unroll
    for (uint32_t i = 0; i < kTiles; ++i)
      if (tile + i * step < kSteps) reinterpret_cast<float4*>(sh.joined[group])[(tile + i * step) * 32 + lane] = acc[i];
  }
  if (tile == first) weigh();
}

// The consumers' rows of a piece, in the order of their chunks.
template <uint32_t D, uint32_t NT>
__device__ __forceinline__ void sum_rows(const PagedDecodeParams& p, const Shared<D, NT>& sh, uint32_t group, const Note& note, Rows<D>& r) {
  constexpr uint32_t kWarps = Shape<D, NT>::kWarps, kSteps = D / 16;
  const uint32_t lane = threadIdx.x & 31u, tig = lane & 3u;
  clear(r);
  if (group * 8 + 2 * tig >= p.rows) return;
  const float* part[kWarps];
  float w[kWarps][2], l[kWarps][2];
#pragma unroll
  for (uint32_t x = 0; x < kWarps; ++x) {
    const uint32_t warp = note.turn + x < kWarps ? note.turn + x : note.turn + x - kWarps;
    part[x] = sh.part[group][warp];
    const float4 ml = x < note.chunks ? reinterpret_cast<const float4*>(part[x] + 8 * D)[tig] : make_float4(kMinusInf, 0.f, kMinusInf, 0.f);
    w[x][0] = ml.x;
    w[x][1] = ml.z;
    l[x][0] = ml.y;
    l[x][1] = ml.w;
    r.m[0] = fmaxf(r.m[0], ml.x);
    r.m[1] = fmaxf(r.m[1], ml.z);
  }
#pragma unroll
  for (uint32_t j = 0; j < 2; ++j) {
    const float safe = r.m[j] == kMinusInf ? 0.f : r.m[j];
#pragma unroll
    for (uint32_t x = 0; x < kWarps; ++x) {
      w[x][j] = ptx::exp2_approx((w[x][j] - safe) * p.scale_log2);
      r.l[j] = fmaf(l[x][j], w[x][j], r.l[j]);
    }
  }
#pragma unroll
  for (uint32_t x = 0; x < kWarps; ++x) {
    if (x >= note.chunks) break;
#pragma unroll
    for (uint32_t mt = 0; mt < kSteps; ++mt) {
      const float4 v = reinterpret_cast<const float4*>(part[x])[mt * 32 + lane];
      float(&o)[4] = r.o[mt];
      o[0] = fmaf(v.x, w[x][0], o[0]);
      o[1] = fmaf(v.y, w[x][1], o[1]);
      o[2] = fmaf(v.z, w[x][0], o[2]);
      o[3] = fmaf(v.w, w[x][1], o[3]);
    }
  }
}

template <uint32_t D, uint32_t NT, bool kBf16>
__device__ void consume(const PagedDecodeParams& p, const Maps& maps, Shared<D, NT>& sh) {
  using S = Shape<D, NT>;
  constexpr uint32_t kTok = kHalf / (2 * D), kSteps = D / 16;
  const uint32_t lane = threadIdx.x & 31u, group = NT == 1 ? 0 : (threadIdx.x >> 5) / S::kWarps, warp = (threadIdx.x >> 5) - group * S::kWarps;
  const uint32_t col0 = group * 8;
  const uint64_t policy = ptx::policy_evict_first();
  uint32_t merges = 0;              // pieces so far whose rows went to the merger
  uint32_t issued = 0, taken = 0;   // chunks of this warp
  bool alive = true;
  Feed<D, NT> feed;
  feed.init(p);
  Rows<D> r;
  // Copies on, as far as stages are free and chunks known. Of two groups both have to have read a stage: if the other one
  // has not yet, its turn comes after the next chunk, unless there is none.
  auto copy = [&] {
    while (alive && issued - taken < kDepth) {
      const uint32_t stage = issued % kDepth;
      if (NT == 2 && issued >= kDepth) {
        uint64_t* bar = &sh.left[warp][stage];
        const uint32_t parity = (issued / kDepth - 1) & 1u;
        if (!__all_sync(0xffffffffu, ready(bar, parity))) {
          if (issued != taken) return;
          alive = __all_sync(0xffffffffu, wait_for(bar, parity, sh, p.status));
          if (!alive) return;
        }
      }
      if (!feed.issue(p, maps, sh, stage, policy)) return;
      ++issued;
    }
  };
  for (uint32_t j = 0; alive; ++j) {
    alive = __all_sync(0xffffffffu, wait_for(&sh.note_full[j % kNotes], j / kNotes & 1u, sh, p.status));
    if (!alive) break;
    const Note note = sh.note[j % kNotes];
    if (note.chunks == 0) break;
    if (group == 0 && (j == 0 || feed.j < j)) feed.open(note, j);  // nothing of the pieces before is left to copy
    const uint32_t c0 = first_chunk<S::kWarps>(note, warp), step = note.solo ? 1u : S::kWarps;
    if (c0 < note.chunks) {
      if (group == 0) feed.prepare(p);
      uint32_t qf[kSteps][2];
      load_q<D>(p, note.seq, note.head, col0, qf);
      if (group == 0) copy();
      clear(r);
      for (uint32_t c = c0; c < note.chunks && alive; c += step) {
        const uint32_t stage = taken % kDepth;
        alive = __all_sync(0xffffffffu, wait_on(&sh.full[warp][stage], (taken / kDepth) & 1u, sh, p.status));
        if (!alive) break;
        take_chunk<D, kBf16>(p, note.lo, note.len, (note.chunk + c) * kTok, sh.stage[warp][stage], qf, r);
        __syncwarp();  // every lane has read the stage
        ++taken;
        if (group == 0)
          copy();
        else if (lane == 0)
          arrive(&sh.left[warp][stage]);
      }
      if (!alive) break;
#pragma unroll
      for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1) r.l[i] += __shfl_xor_sync(0xffffffffu, r.l[i], x);
    }
    if (note.solo || (note.chunks == 1 && note.count == 1)) {
      if (c0 == 0) write_out<D, kBf16>(p, r, note.seq, note.head, col0);  // nobody else has rows of it
    } else {
      alive = __all_sync(0xffffffffu, wait_for(&sh.rows_empty[group], (merges & 1u) ^ 1u, sh, p.status));
      if (!alive) break;
      if (c0 < note.chunks) store_part<D>(p, r, col0, sh.part[group][warp]);
      __syncwarp();
      if (lane == 0) arrive(&sh.rows_full[group]);
      ++merges;
    }
    __syncwarp();
    if (lane == 0) arrive(&sh.note_empty[j % kNotes]);
  }
  if (!alive) {
    // A wait ran out: copies still in flight get a bounded time to land before the CTA's shared memory is given back.
    for (uint32_t s = 0; s < kDepth && s < issued; ++s)
      ptx::mbar_wait(ptx::smem_u32(&sh.full[warp][s]), (issued - 1 - s) / kDepth & 1u, nullptr, 0);
    return;
  }
  // Nothing left to stream: sums over parts go faster with all warps.
  if (lane == 0) atomicAdd(&sh.idle[group], 1u);
  for (uint32_t k = 0;; ++k) {
    if (!__all_sync(0xffffffffu, wait_for(&sh.job_full[group], k & 1u, sh, p.status))) return;
    const auto& job = sh.job[group];
    if (job.count == 0) return;
    sum_parts<D, NT>(p, sh, group, job.slot, job.odd, job.stride, job.count, job.tile + warp, S::kWarps, r.m, r.l, [](uint32_t) { return true; });
    __syncwarp();
    if (lane == 0) arrive(&sh.job_done[group]);
  }
}

template <uint32_t D, uint32_t NT, bool kBf16>
__device__ void merge(const PagedDecodeParams& p, Shared<D, NT>& sh, uint32_t group) {
  using S = Shape<D, NT>;
  constexpr uint32_t kSteps = D / 16;
  const uint32_t lane = threadIdx.x & 31u, col0 = group * 8;
  uint32_t merges = 0, jobs = 0;
  Rows<D> r;
  for (uint32_t j = 0;; ++j) {
    if (!__all_sync(0xffffffffu, wait_for(&sh.note_full[j % kNotes], j / kNotes & 1u, sh, p.status))) return;
    const Note note = sh.note[j % kNotes];
    if (note.chunks == 0) break;
    __syncwarp();
    if (lane == 0) arrive(&sh.note_empty[j % kNotes]);  // read: the copy is what counts from here on
    if (note.solo || (note.chunks == 1 && note.count == 1)) continue;
    if (!__all_sync(0xffffffffu, wait_for(&sh.rows_full[group], merges & 1u, sh, p.status))) return;
    ++merges;
    sum_rows<D, NT>(p, sh, group, note, r);
    __syncwarp();
    if (lane == 0) arrive(&sh.rows_empty[group]);

    // Up the tree: store the rows, and where they are their group's last ones, take the group's sum on.
    uint32_t index = note.index, count = note.count, stride = note.step;
    // Dealt-out work: a join comes at the end, with all warps (one level for 17 to 32 parts: one sequence of 20000 tokens, 8 KV
    // heads, 26.4 us against 28.2). By tickets it is mostly this warp's alone, between pieces: one of 80000 67 us against 71.
    const uint32_t fan = note.step == 1 ? kFan / 2 : kFan;
    bool mine = true;
    for (uint32_t level = 0; count > 1; ++level) {
      const uint32_t g = index / fan, n = min(fan, count - g * fan);
      const uint32_t first = note.slot + g * fan * stride, odd = g ? 0 : note.step - 1;
      store_part<D>(p, r, col0, part_of<D, NT>(p, index ? note.slot + index * stride : note.slot + odd, group));
      __threadfence();
      __syncwarp();
      uint32_t* counter = p.counters + kPagedTree + (group * 3 + level) * kPagedMaxParts + first + odd;
      uint32_t arrived = 0;
      if (lane == 0) {
        arrived = atomicAdd(counter, 1u);
        const bool complete = arrived == n - 1;
        if (complete) *counter = 0;
        sh.open[group] += complete ? 1 - static_cast<int32_t>(n) : 1;
      }
      arrived = __shfl_sync(0xffffffffu, arrived, 0);
      if (arrived != n - 1) {
        mine = false;
        break;
      }
      __threadfence();
      if (n <= 4) {
        clear(r);
        for (uint32_t c = 0; c < n; ++c) add_part<D>(p, r, col0, part_of<D, NT>(p, first + (c ? c * stride : odd), group));
      } else {
        // One warp has 8 or 16 KB of the parts in flight; as soon as the consumers have nothing else to do they take
        // the tiles that are left.
        bool given = false;
        auto give = [&](uint32_t tile) {
          if (__shfl_sync(0xffffffffu, *reinterpret_cast<volatile uint32_t*>(&sh.idle[group]), 0) != S::kWarps) return false;
          if (lane == 0) {
            sh.job[group] = {first, odd, stride, n, tile};
            arrive(&sh.job_full[group]);
          }
          given = true;
          return true;
        };
        give(0);
        sum_parts<D, NT>(p, sh, group, first, odd, stride, n, 0, 1, r.m, r.l, [&](uint32_t tile) { return !given && !give(tile); });
        if (given) {
          if (!__all_sync(0xffffffffu, wait_for(&sh.job_done[group], jobs & 1u, sh, p.status))) return;
          ++jobs;
        }
#pragma unroll
        for (uint32_t mt = 0; mt < kSteps; ++mt) {
          const float4 v = reinterpret_cast<const float4*>(sh.joined[group])[mt * 32 + lane];
          r.o[mt][0] = v.x;
          r.o[mt][1] = v.y;
          r.o[mt][2] = v.z;
          r.o[mt][3] = v.w;
        }
      }
      __syncwarp();
      index = g;
      count = (count + fan - 1) / fan;
      stride *= fan;
    }
    if (mine) write_out<D, kBf16>(p, r, note.seq, note.head, col0);
  }
  if (lane == 0) {
    sh.job[group].count = 0;
    arrive(&sh.job_full[group]);
  }
}

template <uint32_t D, uint32_t NT, bool kBf16>
__global__ void __launch_bounds__(Shape<D, NT>::kThreads, 1) paged_decode_kernel(const PagedDecodeParams p, const __grid_constant__ Maps maps) {
  using S = Shape<D, NT>;
  constexpr uint32_t kTok = kHalf / (2 * D), kAllWarps = S::kThreads / 32;
  extern __shared__ uint8_t smem_raw[];
  Shared<D, NT>& sh = *reinterpret_cast<Shared<D, NT>*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~static_cast<uintptr_t>(127));
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
  if (tid == 0) {
    for (uint32_t x = 0; x < S::kWarps; ++x)
      for (uint32_t s = 0; s < kDepth; ++s) {
        ptx::mbar_init(ptx::smem_u32(&sh.full[x][s]), 1);
        ptx::mbar_init(ptx::smem_u32(&sh.left[x][s]), 1);
      }
    for (uint32_t s = 0; s < kNotes; ++s) {
      ptx::mbar_init(ptx::smem_u32(&sh.note_full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh.note_empty[s]), S::kConsumers + NT);
    }
    for (uint32_t g = 0; g < NT; ++g) {
      ptx::mbar_init(ptx::smem_u32(&sh.rows_full[g]), S::kWarps);
      ptx::mbar_init(ptx::smem_u32(&sh.rows_empty[g]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh.job_full[g]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh.job_done[g]), S::kWarps);
      sh.idle[g] = 0;
      sh.open[g] = 0;
    }
    ptx::fence_barrier_init();
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.m[0]));
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.m[1]));
    sh.dead = sh.started = 0;
  }
  ptx::launch_dependents();
  ptx::grid_dependency_wait();

  // How the work is cut: chunks before each thread's run of sequences, then pieces, and pieces of cut items.
  const uint32_t run = (p.nseq + S::kThreads - 1) / S::kThreads;
  const uint32_t i0 = min(tid * run, p.nseq), i1 = min(i0 + run, p.nseq);
  unsigned long long mine = 0;
  constexpr uint32_t kLeast = 2 * S::kWarps;  // at least two chunks for every warp: a join costs what three take
  const bool few = static_cast<unsigned long long>(p.nseq) * p.num_kv_heads < 2 * gridDim.x;
  for (uint32_t i = i0; i < i1; ++i) mine += room_of(span_of<kTok>(p, i).chunks, few ? kLeast : 1);
  mine *= p.num_kv_heads;
  unsigned long long inc = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned long long o = __shfl_up_sync(0xffffffffu, inc, d);
    if (lane >= static_cast<uint32_t>(d)) inc += o;
  }
  if (lane == 31) sh.warp_total[warp] = inc;
  __syncthreads();
  unsigned long long before = inc - mine, total = 0;
  for (uint32_t x = 0; x < kAllWarps; ++x) {
    if (x < warp) before += sh.warp_total[x];
    total += sh.warp_total[x];
  }
  const unsigned long long share = total / gridDim.x;  // of a CTA
  Zones zones{};
  Even even{};
  uint32_t pieces = 0, most = 1, batch = 1;
  bool many = false;
  sh.chunks_before[tid] = before;
  if (few && share < 8 * kLeast) {
    // Short work: what comes after the last chunk, a merge and a join or two of 3 us each, is a good part of the time, and a
    // CTA's first piece's join is in its second one's way. One sequence of 20000 tokens, 8 KV heads: 28 us against 36 in two
    // pieces to a CTA; 16 of 3000 40 against 41.6; beyond, SMs that get less of HBM count for more: 5 of 100001 321 against 315.
    even.size = max(static_cast<uint32_t>((total + gridDim.x - 1) / gridDim.x), kLeast);
    even.least = kLeast;
    pieces = static_cast<uint32_t>((total + even.size - 1) / even.size);  // as many CTAs
  } else {
    zones.end[0] = share * gridDim.x * kPagedZone0 / 16;
    zones.end[1] = share * gridDim.x * kPagedZone1 / 16;
    // Few items are all cut, and a join over many parts takes longer than uneven ends: two pieces to a CTA throughout (one
    // sequence of 150000 tokens, 8 KV heads: 107 us, against 124 us with the finer cut; two items to a CTA and more the other
    // way round: 64 sequences of up to 4095 tokens 99 us against 103, 48 of up to 6000 differential 102 against 109).
    // (If that leaves pieces of the least size, there would be somewhat more of them than CTAs: then one to a CTA.)
    const uint32_t half = static_cast<uint32_t>(share / kPagedCut0) + 1, coarse = half >= kLeast ? half : max(static_cast<uint32_t>(share) + 1, kLeast);
    zones.size[0] = coarse;
    zones.size[1] = few ? coarse : max(static_cast<uint32_t>(share / kPagedCut1) + 1, kLeast);
    zones.size[2] = few ? coarse : max(static_cast<uint32_t>(share / kPagedCut2) + 1, kLeast);
    uint2 cut = make_uint2(0, 0);
    unsigned long long at = before;
    for (uint32_t i = i0; i < i1; ++i) {
      const uint32_t chunks = span_of<kTok>(p, i).chunks;
      const Cut c = cut_of(zones, at, chunks, p.num_kv_heads);
      cut.x += c.all;
      cut.y += c.parts;
      at += static_cast<unsigned long long>(chunks) * p.num_kv_heads;
    }
    uint2 sum = cut;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t a = __shfl_up_sync(0xffffffffu, sum.x, d), b = __shfl_up_sync(0xffffffffu, sum.y, d);
      if (lane >= static_cast<uint32_t>(d)) {
        sum.x += a;
        sum.y += b;
      }
    }
    if (lane == 31) {
      sh.warp_sum[warp][0] = sum.x;
      sh.warp_sum[warp][1] = sum.y;
    }
    __syncthreads();
    sum.x -= cut.x;
    sum.y -= cut.y;
    for (uint32_t x = 0; x < kAllWarps; ++x) {
      if (x < warp) {
        sum.x += sh.warp_sum[x][0];
        sum.y += sh.warp_sum[x][1];
      }
      pieces += sh.warp_sum[x][0];
    }
    sh.pieces_before[tid] = sum.x;
    sh.parts_before[tid] = sum.y;
    // Tickets to a draw: as many as two dozen chunks or so are.
    const uint32_t mean = pieces ? static_cast<uint32_t>(min(total / pieces, 24ull)) : 24;
    most = 24 / max(mean, 1u);
    batch = batch_of(pieces, most);
    // Items that one warp takes alone: only where every warp gets several of them (times on both sides: at kSolo).
    many = pieces >= 4 * S::kWarps * gridDim.x && total <= static_cast<unsigned long long>(pieces) * kSolo;
  }
  __syncthreads();

  if (static_cast<unsigned long long>(blockIdx.x) * batch < pieces) {
    if (warp < S::kConsumers)
      consume<D, NT, kBf16>(p, maps, sh);
    else if (warp == S::kConsumers)
      schedule<D, NT>(p, sh, zones, even, pieces, batch, most, many);
    else
      merge<D, NT, kBf16>(p, sh, warp - S::kConsumers - 1);
  }

  // Sequences without tokens: zeros, and minus infinity for the log-sum-exp.
  const uint32_t heads = p.num_kv_heads * (p.lam ? p.rows / 2 : p.rows);
  for (uint32_t i = blockIdx.x; i < p.nseq; i += gridDim.x) {
    if (span_of<kTok>(p, i).chunks) continue;
    uint4* dst = reinterpret_cast<uint4*>(p.out + static_cast<uint64_t>(i) * p.out_stride);
    for (uint32_t x = tid; x < heads * D / 8; x += S::kThreads) dst[x] = make_uint4(0, 0, 0, 0);
    if (p.lse)
      for (uint32_t x = tid; x < heads; x += S::kThreads) p.lse[static_cast<uint64_t>(i) * heads + x] = kMinusInf;
    const int32_t n = p.lens[i];
    if (tid == 0 && (n < 0 || static_cast<uint32_t>(n) > p.max_blocks * p.block_tokens)) ptx::report_status(p.status, kStatusInvalid);
  }

  // The CTA that is done last resets the ticket and done words: every CTA has drawn its last ticket and made its last arrival (each
  // got the word's old value back before it came here). The words of the trees are 0 again if every group was complete, which is
  // when arrivals and complete groups balance over all CTAs; if not (a wait ran out, or lengths changed under the call and CTAs did
  // not cut the work alike), all are cleared. (Always clearing them: one sequence of 500 10.8 -> 11.1 us.)
  __syncthreads();
  if (tid == 0) {
    long long open = 0;
    for (uint32_t g = 0; g < NT; ++g) open += sh.open[g];
    const unsigned long long mine = 1 + (static_cast<unsigned long long>(open) << 8);
    auto* done = reinterpret_cast<unsigned long long*>(p.counters + kPagedDone);
    const unsigned long long all = atomicAdd(done, mine) + mine;
    if ((all & 255u) == gridDim.x) {
      p.counters[kPagedTicket] = 0;
      *done = 0;
      if (all != gridDim.x)
        for (uint32_t x = kPagedTree; x < kPagedTree + NT * 3 * kPagedMaxParts; ++x) p.counters[x] = 0;
    }
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

template <uint32_t D, uint32_t NT, bool kBf16>
cudaError_t launch(const PagedDecodeParams& p, const Maps& maps, uint32_t grid, int dev, cudaStream_t stream) {
  constexpr size_t kSharedBytes = sizeof(Shared<D, NT>) + 128;
  static_assert(kSharedBytes <= 232448, "one CTA per SM");
  static std::atomic<bool> ready[64] = {};  // the attribute is a property of the function on one device; several threads may launch
  if (!ready[dev].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(paged_decode_kernel<D, NT, kBf16>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSharedBytes));
    if (e != cudaSuccess) return e;
    ready[dev].store(true, std::memory_order_release);
  }
  return launch_early(paged_decode_kernel<D, NT, kBf16>, grid, Shape<D, NT>::kThreads, kSharedBytes, stream, p, maps);
}

template <uint32_t D>
cudaError_t launch_d(const PagedDecodeParams& p, const Maps& maps, uint32_t grid, int dev, cudaStream_t stream) {
  if (p.dtype == 0) return p.rows <= 8 ? launch<D, 1, true>(p, maps, grid, dev, stream) : launch<D, 2, true>(p, maps, grid, dev, stream);
  return p.rows <= 8 ? launch<D, 1, false>(p, maps, grid, dev, stream) : launch<D, 2, false>(p, maps, grid, dev, stream);
}

}  // namespace

size_t paged_workspace_bytes(uint32_t rows, uint32_t head_dim) {
  const size_t part = (rows <= 8 ? 8 : 16) * (static_cast<size_t>(head_dim) + 2) * sizeof(float);
  return kPagedCounterBytes + kPagedMaxParts * part;
}

cudaError_t launch_paged_decode(const PagedDecodeParams& p, int dev, int num_sms, cudaStream_t stream) {
  if (p.nseq == 0) return cudaSuccess;
  const EncodeFn encode = encode_fn();
  if (!encode) return cudaErrorNotSupported;
  const uint32_t tok = kHalf / (2 * p.head_dim);
  const uint32_t box_rows = p.block_tokens < tok ? p.block_tokens : tok;
  Maps maps;
  // A head of 64 elements is a 128-byte piece of a token row: fetching 256 bytes would read the next head along
  // each time (200 sequences, 12 heads, window 1000: 155 us against 124).
  const CUtensorMapL2promotion promotion = p.head_dim == 64 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_256B;
  for (int j = 0; j < 2; ++j) {
    if (j == 1 && (!p.blocks[0] || !p.blocks[1])) {  // one arena: one map serves both
      maps.m[1] = maps.m[0];
      break;
    }
    const int a = p.blocks[j] ? j : 1 - j;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(p.num_kv_heads) * p.head_dim, 2ull * p.block_tokens, p.blocks[a]};
    const cuuint64_t strides[2] = {dims[0] * 2, p.block_stride[a]};
    const cuuint32_t box[3] = {p.head_dim, box_rows, 1};
    const cuuint32_t elem[3] = {1, 1, 1};
    auto make = [&] {
      return encode(&maps.m[j], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, p.base[a], dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_NONE, promotion, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
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
  const uint32_t sms = static_cast<uint32_t>(num_sms);
  const uint32_t grid = sms < kPagedMaxCtas ? sms : kPagedMaxCtas;
  if (p.head_dim == 64) return launch_d<64>(p, maps, grid, dev, stream);
  if (p.head_dim == 128) return launch_d<128>(p, maps, grid, dev, stream);
  return launch_d<256>(p, maps, grid, dev, stream);
}

}  // namespace ema
