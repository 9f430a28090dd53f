// paged_decode.cu — attention of one new token per sequence over a paged KV cache, everything that
// changes from step to step (tables, lengths) read from device memory; and its differential form.
//
//   o = softmax(s q K^T) V over positions max(0, len - window) .. len - 1, per query head; differential:
//   o_h = softmax(s q1 K1^T) V - lam_h softmax(s q2 K2^T) V, then optionally an RMS norm over the head.
//
// Every K and V byte is needed once and used for a handful of query rows: the kernel is bound by HBM,
// and what it does is keep enough copies in flight on every SM while the arithmetic stays hidden.
//   * Unit of work: a chunk, 16 KB of one KV head (64 / 32 / 16 tokens of K and V for head_dim 64 / 128 /
//     256). The chunks of all (sequence, KV head) items form one line, cut into equal ranges, one per CTA:
//     long and short sequences, few and many heads balance alike, with lengths known only on the device.
//     Every CTA derives its range from the lengths by itself (a block-wide scan).
//   * One producer warp feeds a ring of 16 KB stages by tiled bulk copies ([tokens][head] boxes of a
//     block; a box is the format's swizzled rows as they are), one consumer warp per stage: a warp takes
//     whole chunks, so between the ends of an item the warps do not wait for one another.
//   * Per chunk: S^T[16 tokens x 8 rows] = K Q^T and O^T += V^T P^T on mma.sync m16n8k16 tiles (the
//     query rows are the narrow side, 1 to 16 of them: tcgen05's 64- or 128-row accumulators would
//     hold tokens for S but would need P rewritten through shared memory for O; at one chunk per
//     ~0.35 us and SM the tensor work is a few per cent of the time either way). Online softmax in the
//     log2 domain, f32. P enters the second product as the sum of two 16-bit numbers (error 2^-17
//     for bf16): one rounded P would add an error as large as the output's own rounding, and the
//     differential form subtracts two nearly equal rows.
//   * The differential form is the same pass: K heads 2g, 2g+1 of width D/2 lie side by side, so q1 is
//     padded with zeros behind and q2 in front and the 2G rows of a head run over K and V of width D.
//   * Ends of items: the warps' partial rows are added in shared memory. An item cut by a range boundary
//     leaves its rows in the workspace; the CTA that arrives last joins them, in range order (the
//     result does not depend on who that is), and writes the output.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kernels.h"
#include "ptx.cuh"

namespace ema {

namespace {

constexpr uint32_t kWarps = 6;                      // consumer warps
constexpr uint32_t kConsumers = kWarps * 32;
constexpr uint32_t kThreads = kConsumers + 32;      // and one producer warp
constexpr uint32_t kStageBytes = 16384;             // K half, then V half
constexpr uint32_t kHalf = kStageBytes / 2;
constexpr uint32_t kStages = 12;
// A stage belongs to one warp. If another warp took it in the next round, that warp could wait for a phase of the
// stage's barrier while the copy of the phase before it is still in flight, and a parity wait would pass at once.
static_assert(kStages % kWarps == 0, "a stage is always taken by the same warp");
constexpr uint32_t kMaxRows = 16;
constexpr uint32_t kMergeBytes = 32768;             // first the warps' partial rows, 8 columns x 128 dims at a time; then the
                                                    // CTA's rows in the first half and a join's factors in the second
static_assert(kWarps * 4096 <= kMergeBytes, "partial rows of all warps");
constexpr float kMinusInf = -INFINITY;

struct Maps {
  CUtensorMap m[2];
};

struct __align__(128) Shared {
  uint8_t stage[kStages][kStageBytes];
  uint8_t merge[kMergeBytes];
  float m[kWarps][kMaxRows], l[kWarps][kMaxRows];
  float top[kMaxRows], sum[kMaxRows];
  uint64_t full[kStages], empty[kStages];
  unsigned long long warp_sum[kThreads / 32];
  unsigned long long first_before;  // chunks (one head) of the sequences before the range's first one
  uint32_t first_seq;
  uint32_t arrived;
  uint32_t dead;                    // a bounded wait ran out: no further waiting
  uint32_t issued[kStages];         // parity of the stage's last copy, plus 2; 0 before the first
};

__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory"); }

__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, uint32_t x, uint32_t y, uint32_t z, uint32_t bar,
                                        uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4}], "
      "[%5], %6;" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy)
      : "memory");
}

__device__ __forceinline__ void mma_f16_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <bool kBf16>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (kBf16)
    ptx::mma_bf16_16816(c, a, b0, b1);
  else
    mma_f16_16816(c, a, b0, b1);
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

// Offset of 16-byte unit j of token row r in a stage half of D-wide rows.
template <uint32_t D>
__device__ __forceinline__ uint32_t unit_at(uint32_t r, uint32_t j) {
  return r * (D * 2) + (j >> 3) * 128 + (((j & 7u) ^ (r & 7u)) << 4);
}

// What a sequence asks for: tokens [lo, len), in chunks of kTok tokens from `first` on.
struct Span {
  uint32_t lo, len, first, chunks;
};

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

// A CTA's walk over its range of chunks, item by item; the producer and the consumers each do one.
template <uint32_t kTok>
struct Walk {
  unsigned long long u, u1;     // chunk of the line the walk is at, end of the range
  unsigned long long item;      // first chunk of the current item
  uint32_t seq, head;
  Span span;

  __device__ void start(const PagedDecodeParams& p, const Shared& sh, unsigned long long begin, unsigned long long end) {
    u = begin;
    u1 = end;
    seq = sh.first_seq;
    span = span_of<kTok>(p, seq);
    const unsigned long long before = sh.first_before * p.num_kv_heads;
    head = static_cast<uint32_t>((u - before) / span.chunks);
    item = before + static_cast<unsigned long long>(head) * span.chunks;
  }
  // Chunks [a, b) of the current item are the range's.
  __device__ uint32_t a() const { return static_cast<uint32_t>(u - item); }
  __device__ uint32_t b() const { return u1 - item < span.chunks ? static_cast<uint32_t>(u1 - item) : span.chunks; }
  // On to the next item; false at the end of the range.
  __device__ bool next(const PagedDecodeParams& p) {
    item += span.chunks;
    u = item;
    if (u >= u1) return false;
    if (++head == p.num_kv_heads) {
      head = 0;
      do {
        span = span_of<kTok>(p, ++seq);
      } while (span.chunks == 0);  // there is one: the line is longer than u
    }
    return true;
  }
};

__device__ __forceinline__ bool wait_on(uint64_t* bar, uint32_t parity, Shared& sh, int* status) {
  if (ptx::mbar_try_wait(ptx::smem_u32(bar), parity)) return true;
  if (*reinterpret_cast<volatile uint32_t*>(&sh.dead)) return false;
  if (ptx::mbar_wait(ptx::smem_u32(bar), parity, status, kDevTimeout)) return true;
  *reinterpret_cast<volatile uint32_t*>(&sh.dead) = 1;
  return false;
}

template <uint32_t D>
__device__ void produce(const PagedDecodeParams& p, const Maps& maps, Shared& sh, unsigned long long u0, unsigned long long u1) {
  constexpr uint32_t kTok = kHalf / (2 * D);
  const uint32_t lane = threadIdx.x & 31u;
  const uint32_t box = p.block_tokens < kTok ? p.block_tokens : kTok;  // token rows of one copy
  const uint32_t per_chunk = kTok / box;                                // 1, 2 or 4 copies of K (and of V)
  const uint32_t together = 32 / per_chunk;                             // chunks whose entries the warp holds at a time
  const uint32_t mine = lane / per_chunk, part = lane % per_chunk;
  const uint32_t box_bytes = box * D * 2;
  const uint64_t policy = ptx::policy_evict_first();
  uint32_t stage = 0, phase = 1;  // the first round finds the stages empty
  Walk<kTok> w;
  w.start(p, sh, u0, u1);
  do {
    const int32_t* table = p.tables + static_cast<uint64_t>(w.seq) * p.table_stride;
    const uint32_t a = w.a(), b = w.b();
    for (uint32_t c0 = a; c0 < b; c0 += together) {
      // This lane's copy: token rows [t, t + box) of chunk c0 + mine, wanted if one of them is in [lo, len).
      const uint32_t t = (w.span.first + c0 + mine) * kTok + part * box;
      const bool on = c0 + mine < b && t < w.span.len && t + box > w.span.lo;
      uint32_t which = 0, id = 0;
      if (on) {
        const int32_t e = table[t / p.block_tokens];
        which = e < 0;
        id = static_cast<uint32_t>(which ? ~e : e);
        const uint32_t blocks = which ? p.blocks[1] : p.blocks[0];
        if (id >= blocks) {  // a bad page: reads as zeros (a box outside the tensor), and is reported
          ptx::report_status(p.status, kStatusInvalid);
          id = blocks ? blocks : which ? p.blocks[0] : p.blocks[1];  // of an arena without blocks the map is the other one's
        }
      }
      const uint32_t boxes = __ballot_sync(0xffffffffu, on);
      const uint32_t steps = min(together, b - c0);
      for (uint32_t k = 0; k < steps; ++k) {
        const uint32_t group = (boxes >> (k * per_chunk)) & ((1u << per_chunk) - 1);
        if (!wait_on(&sh.empty[stage], phase, sh, p.status)) return;
        const uint32_t bar = ptx::smem_u32(&sh.full[stage]);
        if (lane == 0) {
          sh.issued[stage] = 2 + (phase ^ 1u);
          ptx::mbar_arrive_expect_tx(bar, 2 * box_bytes * __popc(group));
        }
        __syncwarp();
        if (mine == k && on) {
          const uint32_t row = t % p.block_tokens;
          const uint32_t dst = ptx::smem_u32(sh.stage[stage]) + part * box_bytes;
          tma_box(dst, &maps.m[which], w.head * D, row, id, bar, policy);
          tma_box(dst + kHalf, &maps.m[which], w.head * D, p.block_tokens + row, id, bar, policy);
        }
        if (++stage == kStages) {
          stage = 0;
          phase ^= 1u;
        }
      }
    }
  } while (w.next(p));
}

// Rows of an item, [rows][D] f32 relative to their row maximum in sh.merge, weights' sums in sh.sum: normalised,
// combined and written out. One warp per output row.
template <uint32_t D, bool kBf16>
__device__ void write_out(const PagedDecodeParams& p, Shared& sh, uint32_t seq, uint32_t head) {
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  const float* o = reinterpret_cast<const float*>(sh.merge);
  const uint32_t G = p.lam ? p.rows / 2 : p.rows;
  constexpr uint32_t kPer = D / 32;  // neighbouring dims of a lane
  for (uint32_t g = warp; g < G; g += kWarps) {
    const uint32_t h = head * G + g;
    float v[kPer];
    if (!p.lam) {
      const float inv = sh.sum[g] > 0.f ? 1.f / sh.sum[g] : (sh.sum[g] == 0.f ? 0.f : sh.sum[g]);
#pragma unroll
      for (uint32_t e = 0; e < kPer; ++e) v[e] = o[g * D + lane * kPer + e] * inv;
      if (p.lse && lane == 0)
        p.lse[static_cast<uint64_t>(seq) * p.num_kv_heads * G + h] = (sh.top[g] + log2f(sh.sum[g])) * 0.6931471805599453f;
    } else {
      const float s1 = sh.sum[2 * g], s2 = sh.sum[2 * g + 1];
      const float i1 = s1 > 0.f ? 1.f / s1 : (s1 == 0.f ? 0.f : s1), i2 = (s2 > 0.f ? 1.f / s2 : (s2 == 0.f ? 0.f : s2)) * p.lam[h];
      float sq = 0.f;
#pragma unroll
      for (uint32_t e = 0; e < kPer; ++e) {
        // two rounded products (not a fused one): equal maps with a weight of 1 leave exactly nothing
        v[e] = __fsub_rn(__fmul_rn(o[2 * g * D + lane * kPer + e], i1), __fmul_rn(o[(2 * g + 1) * D + lane * kPer + e], i2));
        sq = fmaf(v[e], v[e], sq);
      }
      float f = p.out_scale;
      if (p.norm_weight) {
#pragma unroll
        for (int sft = 16; sft; sft >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, sft);
        f *= rsqrtf(sq * (1.f / D) + p.eps);
#pragma unroll
        for (uint32_t e = 0; e < kPer; ++e) v[e] *= p.norm_weight[lane * kPer + e];
      }
#pragma unroll
      for (uint32_t e = 0; e < kPer; ++e) v[e] *= f;
    }
    uint32_t* dst = reinterpret_cast<uint32_t*>(p.out + static_cast<uint64_t>(seq) * p.out_stride + static_cast<uint64_t>(h) * D * 2) +
                    lane * (kPer / 2);
#pragma unroll
    for (uint32_t e = 0; e < kPer / 2; ++e) dst[e] = pack<kBf16>(v[2 * e], v[2 * e + 1]);
  }
}

template <uint32_t D, uint32_t NT, bool kBf16>
__device__ void consume(const PagedDecodeParams& p, Shared& sh, unsigned long long u0, unsigned long long u1, unsigned long long per) {
  constexpr uint32_t kTok = kHalf / (2 * D);
  constexpr uint32_t kSub = kTok / 16;
  constexpr uint32_t kSteps = D / 16;
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
  const uint32_t gid = lane >> 2, tig = lane & 3u;
  const uint32_t mj = lane >> 3, mr = lane & 7u;
  const uint32_t G = p.rows;
  const bool diff = p.lam != nullptr;
  uint32_t it = 0;  // chunks of the range before the current item
  Walk<kTok> w;
  w.start(p, sh, u0, u1);
  do {
    const uint32_t a = w.a(), b = w.b();

    // Query rows as the narrow operand: column n = row of the item, 16 dims per step.
    uint32_t qf[kSteps][NT][2];
    {
      const uint32_t width = diff ? D / 2 : D;
      const uint8_t* q = p.q + static_cast<uint64_t>(w.seq) * p.q_stride + static_cast<uint64_t>(w.head) * G * width * 2;
#pragma unroll
      for (uint32_t nt = 0; nt < NT; ++nt) {
        const uint32_t n = nt * 8 + gid;
        const uint32_t shift = diff && (n & 1u) ? D / 2 : 0;  // where the row's dims start in K
        const uint8_t* row = q + static_cast<uint64_t>(n) * width * 2;
#pragma unroll
        for (uint32_t ks = 0; ks < kSteps; ++ks)
#pragma unroll
          for (uint32_t hh = 0; hh < 2; ++hh) {
            const uint32_t d = ks * 16 + hh * 8 + tig * 2;
            qf[ks][nt][hh] = n < G && d >= shift && d - shift < width ? *reinterpret_cast<const uint32_t*>(row + (d - shift) * 2) : 0u;
          }
      }
    }

    float o[kSteps][NT][4];
    float m[NT][2], l[NT][2];
#pragma unroll
    for (uint32_t nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = kMinusInf;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (uint32_t mt = 0; mt < kSteps; ++mt) o[mt][nt][0] = o[mt][nt][1] = o[mt][nt][2] = o[mt][nt][3] = 0.f;
    }

    // Chunk number `it + c - a` of the range goes to warp (number mod kWarps), stage (number mod kStages).
    for (uint32_t c = a + ((warp + kWarps - it % kWarps) % kWarps); c < b; c += kWarps) {
      const uint32_t number = it + c - a, stage = number % kStages;
      wait_on(&sh.full[stage], (number / kStages) & 1u, sh, p.status);
      const uint32_t kbase = ptx::smem_u32(sh.stage[stage]), vbase = kbase + kHalf;
      const uint32_t tok0 = (w.span.first + c) * kTok;
      const bool whole = tok0 >= w.span.lo && tok0 + kTok <= w.span.len;

      float s[kSub][NT][4];
#pragma unroll
      for (uint32_t sub = 0; sub < kSub; ++sub) {
#pragma unroll
        for (uint32_t nt = 0; nt < NT; ++nt) s[sub][nt][0] = s[sub][nt][1] = s[sub][nt][2] = s[sub][nt][3] = 0.f;
        const uint32_t row = sub * 16 + (mj & 1u) * 8 + mr;
#pragma unroll
        for (uint32_t ks = 0; ks < kSteps; ++ks) {
          uint32_t f[4];
          ptx::ldmatrix_x4(f, kbase + unit_at<D>(row, 2 * ks + (mj >> 1)));
#pragma unroll
          for (uint32_t nt = 0; nt < NT; ++nt) mma<kBf16>(s[sub][nt], f, qf[ks][nt][0], qf[ks][nt][1]);
        }
      }
      float mx[NT][2];
#pragma unroll
      for (uint32_t nt = 0; nt < NT; ++nt) mx[nt][0] = mx[nt][1] = kMinusInf;
#pragma unroll
      for (uint32_t sub = 0; sub < kSub; ++sub) {
        const uint32_t ta = tok0 + sub * 16 + gid, tb = ta + 8;
        const bool in_a = whole || (ta >= w.span.lo && ta < w.span.len), in_b = whole || (tb >= w.span.lo && tb < w.span.len);
#pragma unroll
        for (uint32_t nt = 0; nt < NT; ++nt) {
          float(&x)[4] = s[sub][nt];
          x[0] = in_a ? x[0] * p.scale_log2 : kMinusInf;
          x[1] = in_a ? x[1] * p.scale_log2 : kMinusInf;
          x[2] = in_b ? x[2] * p.scale_log2 : kMinusInf;
          x[3] = in_b ? x[3] * p.scale_log2 : kMinusInf;
          mx[nt][0] = fmaxf(mx[nt][0], fmaxf(x[0], x[2]));
          mx[nt][1] = fmaxf(mx[nt][1], fmaxf(x[1], x[3]));
        }
      }
      bool moved = false;
      float al[NT][2];
#pragma unroll
      for (uint32_t nt = 0; nt < NT; ++nt)
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) {
#pragma unroll
          for (int sh_ = 4; sh_ <= 16; sh_ <<= 1) mx[nt][j] = fmaxf(mx[nt][j], __shfl_xor_sync(0xffffffffu, mx[nt][j], sh_));
          const float mn = fmaxf(m[nt][j], mx[nt][j]);
          const float safe = mn == kMinusInf ? 0.f : mn;  // no finite score so far: every weight is 0
          al[nt][j] = ptx::exp2_approx(m[nt][j] - safe);
          moved |= mn != m[nt][j];
          m[nt][j] = mn;
          mx[nt][j] = safe;
          l[nt][j] *= al[nt][j];
        }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (uint32_t mt = 0; mt < kSteps; ++mt)
#pragma unroll
          for (uint32_t nt = 0; nt < NT; ++nt) {
            o[mt][nt][0] *= al[nt][0];
            o[mt][nt][1] *= al[nt][1];
            o[mt][nt][2] *= al[nt][0];
            o[mt][nt][3] *= al[nt][1];
          }
      }
#pragma unroll
      for (uint32_t sub = 0; sub < kSub; ++sub) {
        const uint32_t t16 = tok0 + sub * 16;
        if (!whole && (t16 >= w.span.len || t16 + 16 <= w.span.lo)) continue;
        uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
        for (uint32_t nt = 0; nt < NT; ++nt) {
          const float(&x)[4] = s[sub][nt];
          const float p0 = ptx::exp2_approx(x[0] - mx[nt][0]), p1 = ptx::exp2_approx(x[1] - mx[nt][1]);
          const float p2 = ptx::exp2_approx(x[2] - mx[nt][0]), p3 = ptx::exp2_approx(x[3] - mx[nt][1]);
          l[nt][0] += p0 + p2;
          l[nt][1] += p1 + p3;
          const uint32_t h01 = pack<kBf16>(p0, p1), h23 = pack<kBf16>(p2, p3);
          const float2 r01 = unpack<kBf16>(h01), r23 = unpack<kBf16>(h23);
          hi[nt][0] = ptx::movmatrix_trans(h01);
          hi[nt][1] = ptx::movmatrix_trans(h23);
          lo[nt][0] = ptx::movmatrix_trans(pack<kBf16>(p0 - r01.x, p1 - r01.y));
          lo[nt][1] = ptx::movmatrix_trans(pack<kBf16>(p2 - r23.x, p3 - r23.y));
        }
        // Token pairs (2 tig, 2 tig + 1) and (+8, +9): rows of V outside [lo, len) are taken as zeros, whatever
        // they hold.
        uint32_t keep_lo = 0xffffffffu, keep_hi = 0xffffffffu;
        const bool full16 = whole || (t16 >= w.span.lo && t16 + 16 <= w.span.len);
        if (!full16) {
          const uint32_t t = t16 + 2 * tig;
          auto in = [&](uint32_t x) { return x >= w.span.lo && x < w.span.len; };
          keep_lo = (in(t) ? 0x0000ffffu : 0u) | (in(t + 1) ? 0xffff0000u : 0u);
          keep_hi = (in(t + 8) ? 0x0000ffffu : 0u) | (in(t + 9) ? 0xffff0000u : 0u);
        }
        const uint32_t row = sub * 16 + (mj >> 1) * 8 + mr;
#pragma unroll
        for (uint32_t mt = 0; mt < kSteps; ++mt) {
          uint32_t f[4];
          ptx::ldmatrix_x4_trans(f, vbase + unit_at<D>(row, 2 * mt + (mj & 1u)));
          if (!full16) {
            f[0] &= keep_lo;
            f[1] &= keep_lo;
            f[2] &= keep_hi;
            f[3] &= keep_hi;
          }
#pragma unroll
          for (uint32_t nt = 0; nt < NT; ++nt) {
            mma<kBf16>(o[mt][nt], f, hi[nt][0], hi[nt][1]);
            mma<kBf16>(o[mt][nt], f, lo[nt][0], lo[nt][1]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.empty[stage]));
    }
    it += b - a;

    // The warps' rows become the CTA's: common maximum, sums, then the rows 8 columns x 128 dims at a time.
#pragma unroll
    for (uint32_t nt = 0; nt < NT; ++nt)
#pragma unroll
      for (uint32_t j = 0; j < 2; ++j) {
#pragma unroll
        for (int sh_ = 4; sh_ <= 16; sh_ <<= 1) l[nt][j] += __shfl_xor_sync(0xffffffffu, l[nt][j], sh_);
        if (gid == 0) {
          sh.m[warp][nt * 8 + tig * 2 + j] = m[nt][j];
          sh.l[warp][nt * 8 + tig * 2 + j] = l[nt][j];
        }
      }
    consumers_sync();
    float scale[NT][2];
#pragma unroll
    for (uint32_t nt = 0; nt < NT; ++nt)
#pragma unroll
      for (uint32_t j = 0; j < 2; ++j) {
        const uint32_t col = nt * 8 + tig * 2 + j;
        float top = kMinusInf;
        for (uint32_t x = 0; x < kWarps; ++x) top = fmaxf(top, sh.m[x][col]);
        const float safe = top == kMinusInf ? 0.f : top;
        scale[nt][j] = ptx::exp2_approx(m[nt][j] - safe);
        if (warp == 0 && gid == 0) {
          float sum = 0.f;
          for (uint32_t x = 0; x < kWarps; ++x) sum += sh.l[x][col] * ptx::exp2_approx(sh.m[x][col] - safe);
          sh.top[col] = top;
          sh.sum[col] = sum;
        }
      }
    constexpr uint32_t kTiles = kSteps < 8 ? kSteps : 8;         // 16-dim tiles of one pass
    constexpr uint32_t kPasses = kSteps / kTiles;
    float4* buf = reinterpret_cast<float4*>(sh.merge);
    constexpr uint32_t kQuads = kTiles * 32, kMine = (kQuads + kConsumers - 1) / kConsumers;  // float4 sums of a pass, and of a thread
    float4 got[NT][kPasses][kMine];
#pragma unroll
    for (uint32_t nt = 0; nt < NT; ++nt)
#pragma unroll
      for (uint32_t ps = 0; ps < kPasses; ++ps) {
        if (nt || ps) consumers_sync();
#pragma unroll
        for (uint32_t mt = 0; mt < kTiles; ++mt) {
          const float(&x)[4] = o[ps * kTiles + mt][nt];
          buf[warp * kQuads + mt * 32 + lane] = make_float4(x[0] * scale[nt][0], x[1] * scale[nt][1], x[2] * scale[nt][0], x[3] * scale[nt][1]);
        }
        consumers_sync();
#pragma unroll
        for (uint32_t j = 0; j < kMine; ++j) {
          const uint32_t at = j * kConsumers + tid;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          if (at < kQuads) {
#pragma unroll
            for (uint32_t x = 0; x < kWarps; ++x) {
              const float4 y = buf[x * kQuads + at];
              acc.x += y.x;
              acc.y += y.y;
              acc.z += y.z;
              acc.w += y.w;
            }
          }
          got[nt][ps][j] = acc;
        }
      }
    consumers_sync();
    float* rows = reinterpret_cast<float*>(sh.merge);            // [rows][D]
#pragma unroll
    for (uint32_t nt = 0; nt < NT; ++nt)
#pragma unroll
      for (uint32_t ps = 0; ps < kPasses; ++ps)
#pragma unroll
        for (uint32_t j = 0; j < kMine; ++j) {
          const uint32_t at = j * kConsumers + tid;              // tile at / 32 of the pass, as lane at % 32 held it
          if (at >= kQuads) continue;
          const uint32_t dim = (ps * kTiles + at / 32) * 16 + ((at % 32) >> 2), col = nt * 8 + (at & 3u) * 2;
          rows[col * D + dim] = got[nt][ps][j].x;
          rows[(col + 1) * D + dim] = got[nt][ps][j].y;
          rows[col * D + dim + 8] = got[nt][ps][j].z;
          rows[(col + 1) * D + dim + 8] = got[nt][ps][j].w;
        }
    consumers_sync();

    bool write = true;
    if (a != 0 || b != w.span.chunks) {
      // An item of several ranges: c0 .. c1 are their CTAs. A CTA's first item may have begun before its range
      // (slot 0), its last one may go on behind it (slot 1).
      const uint32_t c0 = static_cast<uint32_t>(w.item / per), c1 = static_cast<uint32_t>((w.item + w.span.chunks - 1) / per);
      const uint32_t slot = 2 * blockIdx.x + (a == 0 ? 1u : 0u);
      float* po = p.part_o + static_cast<uint64_t>(slot) * G * D;
      for (uint32_t x = tid; x < G * D / 4; x += kConsumers) __stcg(reinterpret_cast<float4*>(po) + x, reinterpret_cast<const float4*>(rows)[x]);
      if (tid < G) __stcg(reinterpret_cast<float2*>(p.part_ml) + static_cast<uint64_t>(slot) * G + tid, make_float2(sh.top[tid], sh.sum[tid]));
      __threadfence();
      consumers_sync();
      if (tid == 0) sh.arrived = atomicAdd(&p.counters[c0], 1u);
      consumers_sync();
      write = sh.arrived == c1 - c0;
      if (write) {
        __threadfence();
        if (tid == 0) p.counters[c0] = 0;
        // Range c0 left its last item (slot 1), the others their first ones (slot 0).
        const uint32_t splits = c1 - c0 + 1;
        auto at = [&](uint32_t x) { return static_cast<uint64_t>(2 * (c0 + x) + (x == 0 ? 1u : 0u)) * G; };
        const float2* ml = reinterpret_cast<const float2*>(p.part_ml);
        float* weight = reinterpret_cast<float*>(sh.merge + kMergeBytes / 2);  // [rows][splits]
        for (uint32_t r = warp; r < G; r += kWarps) {
          float top = kMinusInf;
          for (uint32_t x = lane; x < splits; x += 32) top = fmaxf(top, __ldcg(ml + at(x) + r).x);
#pragma unroll
          for (int sh_ = 16; sh_; sh_ >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, sh_));
          const float safe = top == kMinusInf ? 0.f : top;
          float sum = 0.f;
          for (uint32_t x = lane; x < splits; x += 32) {
            const float2 v = __ldcg(ml + at(x) + r);
            const float f = ptx::exp2_approx(v.x - safe);
            weight[r * splits + x] = f;
            sum += v.y * f;
          }
#pragma unroll
          for (int sh_ = 16; sh_; sh_ >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, sh_);
          if (lane == 0) {
            sh.top[r] = top;
            sh.sum[r] = sum;
          }
        }
        consumers_sync();
        // Few rows: several groups of threads take every groups-th split each, and their sums are added.
        const uint32_t quads = G * D / 4, groups = quads < kConsumers ? kConsumers / quads : 1;
        float4* out4 = reinterpret_cast<float4*>(rows);
        for (uint32_t x0 = 0; x0 < quads; x0 += kConsumers) {
          const uint32_t x = groups > 1 ? tid % quads : x0 + tid, group = groups > 1 ? tid / quads : 0;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          if (x < quads && group < groups) {
            const float* wr = weight + (x / (D / 4)) * splits;
#pragma unroll 8
            for (uint32_t y = group; y < splits; y += groups) {
              const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part_o + at(y) * D) + x);
              const float f = wr[y];
              acc.x = fmaf(v.x, f, acc.x);
              acc.y = fmaf(v.y, f, acc.y);
              acc.z = fmaf(v.z, f, acc.z);
              acc.w = fmaf(v.w, f, acc.w);
            }
            out4[group * quads + x] = acc;
          }
        }
        if (groups > 1) {
          consumers_sync();
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          if (tid < quads)
            for (uint32_t y = 0; y < groups; ++y) {
              const float4 v = out4[y * quads + tid];
              acc.x += v.x;
              acc.y += v.y;
              acc.z += v.z;
              acc.w += v.w;
            }
          consumers_sync();
          if (tid < quads) out4[tid] = acc;
        }
        consumers_sync();
      }
    }
    if (write) write_out<D, kBf16>(p, sh, w.seq, w.head);
    consumers_sync();  // sh.merge, sh.m and sh.top are used again
  } while (w.next(p));
}

template <uint32_t D, uint32_t NT, bool kBf16>
__global__ void __launch_bounds__(kThreads, 1) paged_decode_kernel(const PagedDecodeParams p, const __grid_constant__ Maps maps) {
  constexpr uint32_t kTok = kHalf / (2 * D);
  extern __shared__ uint8_t smem_raw[];
  Shared& sh = *reinterpret_cast<Shared*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~static_cast<uintptr_t>(127));
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
  if (tid == 0) {
    for (uint32_t s = 0; s < kStages; ++s) {
      ptx::mbar_init(ptx::smem_u32(&sh.full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh.empty[s]), 1);
      sh.issued[s] = 0;
    }
    ptx::fence_barrier_init();
    sh.dead = 0;
    sh.first_seq = 0xffffffffu;
  }

  // The line of chunks: total length, and where this CTA's range begins.
  const uint32_t run = (p.nseq + kThreads - 1) / kThreads;
  const uint32_t i0 = min(tid * run, p.nseq), i1 = min(i0 + run, p.nseq);
  unsigned long long mine = 0;
  for (uint32_t i = i0; i < i1; ++i) mine += span_of<kTok>(p, i).chunks;
  unsigned long long inc = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned long long o = __shfl_up_sync(0xffffffffu, inc, d);
    if (lane >= static_cast<uint32_t>(d)) inc += o;
  }
  if (lane == 31) sh.warp_sum[warp] = inc;
  __syncthreads();
  unsigned long long before = 0, total = 0;
  for (uint32_t x = 0; x < kThreads / 32; ++x) {
    if (x == warp) before = total;
    total += sh.warp_sum[x];
  }
  before += inc - mine;
  total *= p.num_kv_heads;
  const unsigned long long per = (total + gridDim.x - 1) / gridDim.x;
  const unsigned long long u0 = min(per * blockIdx.x, total), u1 = min(u0 + per, total);
  if (u0 < u1 && before * p.num_kv_heads <= u0 && u0 < (before + mine) * p.num_kv_heads) {
    unsigned long long at = before;
    uint32_t i = i0;
    for (;; ++i) {
      const uint32_t c = span_of<kTok>(p, i).chunks;
      if (u0 < (at + c) * p.num_kv_heads) break;
      at += c;
    }
    sh.first_seq = i;
    sh.first_before = at;
  }
  __syncthreads();

  if (u0 < u1) {
    if (warp == kWarps)
      produce<D>(p, maps, sh, u0, u1);
    else
      consume<D, NT, kBf16>(p, sh, u0, u1, per);
  }

  // Sequences without tokens: zeros, and minus infinity for the log-sum-exp.
  const uint32_t heads = p.num_kv_heads * (p.lam ? p.rows / 2 : p.rows);
  for (uint32_t i = blockIdx.x; i < p.nseq; i += gridDim.x) {
    if (span_of<kTok>(p, i).chunks) continue;
    uint4* dst = reinterpret_cast<uint4*>(p.out + static_cast<uint64_t>(i) * p.out_stride);
    for (uint32_t x = tid; x < heads * D / 8; x += kThreads) dst[x] = make_uint4(0, 0, 0, 0);
    if (p.lse)
      for (uint32_t x = tid; x < heads; x += kThreads) p.lse[static_cast<uint64_t>(i) * heads + x] = kMinusInf;
    const int32_t n = p.lens[i];
    if (tid == 0 && (n < 0 || static_cast<uint32_t>(n) > p.max_blocks * p.block_tokens)) ptx::report_status(p.status, kStatusInvalid);
  }

  // After a wait that ran out: copies still in flight get a bounded time to land before the CTA's shared
  // memory is given back.
  __syncthreads();
  if (sh.dead && tid < kStages && sh.issued[tid]) ptx::mbar_wait(ptx::smem_u32(&sh.full[tid]), sh.issued[tid] & 1u, nullptr, 0);
}

constexpr size_t kSharedBytes = sizeof(Shared) + 128;
static_assert(kSharedBytes <= 232448, "one CTA per SM");

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
cudaError_t launch(const PagedDecodeParams& p, const Maps& maps, uint32_t grid, cudaStream_t stream) {
  static bool ready[64] = {};  // the attribute is a property of the function on one device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!ready[dev]) {
    e = cudaFuncSetAttribute(paged_decode_kernel<D, NT, kBf16>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSharedBytes));
    if (e != cudaSuccess) return e;
    ready[dev] = true;
  }
  paged_decode_kernel<D, NT, kBf16><<<grid, kThreads, kSharedBytes, stream>>>(p, maps);
  return cudaGetLastError();
}

template <uint32_t D>
cudaError_t launch_d(const PagedDecodeParams& p, const Maps& maps, uint32_t grid, cudaStream_t stream) {
  if (p.dtype == 0) return p.rows <= 8 ? launch<D, 1, true>(p, maps, grid, stream) : launch<D, 2, true>(p, maps, grid, stream);
  return p.rows <= 8 ? launch<D, 1, false>(p, maps, grid, stream) : launch<D, 2, false>(p, maps, grid, stream);
}

}  // namespace

size_t paged_workspace_bytes(uint32_t rows, uint32_t head_dim) {
  return kPagedMaxCtas * sizeof(uint32_t) + static_cast<size_t>(2) * kPagedMaxCtas * rows * (head_dim + 2) * sizeof(float);
}

cudaError_t launch_paged_decode(const PagedDecodeParams& p, int num_sms, cudaStream_t stream) {
  if (p.nseq == 0) return cudaSuccess;
  const EncodeFn encode = encode_fn();
  if (!encode) return cudaErrorNotSupported;
  const uint32_t tok = kHalf / (2 * p.head_dim);
  const uint32_t box_rows = p.block_tokens < tok ? p.block_tokens : tok;
  Maps maps;
  for (int j = 0; j < 2; ++j) {
    const int a = p.blocks[j] ? j : 1 - j;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(p.num_kv_heads) * p.head_dim, 2ull * p.block_tokens, p.blocks[a]};
    const cuuint64_t strides[2] = {dims[0] * 2, p.block_stride[a]};
    const cuuint32_t box[3] = {p.head_dim, box_rows, 1};
    const cuuint32_t elem[3] = {1, 1, 1};
    if (encode(&maps.m[j], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, p.base[a], dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return cudaErrorInvalidValue;
  }
  const uint32_t sms = static_cast<uint32_t>(num_sms);
  const uint32_t grid = sms < kPagedMaxCtas ? sms : kPagedMaxCtas;
  if (p.head_dim == 64) return launch_d<64>(p, maps, grid, stream);
  if (p.head_dim == 128) return launch_d<128>(p, maps, grid, stream);
  return launch_d<256>(p, maps, grid, stream);
}

}  // namespace ema
