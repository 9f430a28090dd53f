// paged_api.cpp — C entry points of the device-driven path: checks of what the host can see, then one
// launch each. No state is kept between calls (apart from per-device constants), nothing is allocated.
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/emaslice.h"
#include "kernels.h"

namespace {

constexpr uint64_t kMost = 0x7fffffffu;

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

uint32_t block_shift(uint32_t tokens) { return tokens == 16 ? 4u : tokens == 32 ? 5u : tokens == 64 ? 6u : 0u; }

// Whether the cache is one the kernels support; its block strides, dense where the caller gave none.
bool cache_ok(const paged_cache_t* c, uint64_t (&stride)[2]) {
  if (!c || c->dtype > 1 || c->num_kv_heads == 0 || c->num_kv_heads > 64) return false;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return false;
  if (!block_shift(c->block_tokens)) return false;
  const uint64_t dense = 2ull * c->block_tokens * c->num_kv_heads * c->head_dim * 2;
  if (c->blocks[0] == 0 && c->blocks[1] == 0) return false;
  for (int j = 0; j < 2; ++j) {
    stride[j] = c->block_stride[j] ? c->block_stride[j] : dense;
    if (c->blocks[j] == 0) continue;
    if (!c->base[j] || !aligned(c->base[j], 16) || c->blocks[j] > kMost) return false;
    if (stride[j] < dense || (stride[j] & 15u) || stride[j] >= (1ull << 40)) return false;
  }
  return true;
}

// A failure's code. The runtime keeps it until it is asked for, and the library's other launches would report it as theirs.
int failed(int code) {
  cudaGetLastError();
  return code;
}

// The call's memory has to be reachable from the current device: memory of another one is refused.
int device_ok(const void* p, int* sms, int* device = nullptr) {
  static std::atomic<int> sms_of[64] = {};  // several threads may call at a time
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return failed(SLICE_ECUDA);
  cudaPointerAttributes at{};
  if (cudaPointerGetAttributes(&at, p) != cudaSuccess) return failed(SLICE_EINVAL);
  if (at.type == cudaMemoryTypeDevice && at.device != dev) return SLICE_EINVAL;
  if (at.type == cudaMemoryTypeUnregistered) return SLICE_EINVAL;
  *sms = sms_of[dev].load(std::memory_order_relaxed);
  if (!*sms) {
    if (cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return failed(SLICE_ECUDA);
    sms_of[dev].store(*sms, std::memory_order_relaxed);
  }
  if (device) *device = dev;
  return SLICE_OK;
}

int launched(cudaError_t e) { return e == cudaSuccess ? SLICE_OK : failed(SLICE_ECUDA); }

int decode(const paged_decode_t* a, bool diff, void* stream) {
  if (!a) return SLICE_EINVAL;
  const paged_cache_t* c = a->cache;
  uint64_t stride[2];
  if (!cache_ok(c, stride)) return SLICE_EINVAL;
  if (a->num_heads == 0 || a->num_heads % c->num_kv_heads || a->num_heads / c->num_kv_heads > (diff ? 8u : 16u)) return SLICE_EINVAL;
  const uint32_t rows = a->num_heads / c->num_kv_heads * (diff ? 2 : 1);
  if (diff ? !a->lam || a->lse || (a->norm_weight && !(a->eps >= 0.f)) : a->lam || a->norm_weight) return SLICE_EINVAL;
  if (a->nseq == 0) return SLICE_OK;
  if (!a->tables || !a->lens || !a->q || !a->out || !a->workspace || static_cast<uint64_t>(a->nseq) * c->num_kv_heads > kMost / 2)
    return SLICE_EINVAL;
  if (a->max_blocks == 0 || a->table_stride < a->max_blocks || static_cast<uint64_t>(a->max_blocks) * c->block_tokens > kMost)
    return SLICE_EINVAL;
  const uint64_t q_row = static_cast<uint64_t>(rows) * c->num_kv_heads * (diff ? c->head_dim / 2 : c->head_dim) * 2;
  const uint64_t out_row = static_cast<uint64_t>(a->num_heads) * c->head_dim * 2;
  if ((a->nseq > 1 && (a->q_stride < q_row || a->out_stride < out_row)) || ((a->q_stride | a->out_stride) & 15u)) return SLICE_EINVAL;
  if (!aligned(a->q, 16) || !aligned(a->out, 16) || !aligned(a->workspace, 16) || !aligned(a->tables, 4) || !aligned(a->lens, 4) ||
      !aligned(a->lse, 4) || !aligned(a->lam, 4) || !aligned(a->norm_weight, 4) || !aligned(a->status, 4))
    return SLICE_EINVAL;
  if (a->workspace_bytes < ema::paged_workspace_bytes(rows, c->head_dim)) return SLICE_ESCRATCH;
  int sms = 0, dev = 0;
  const int rc = device_ok(a->out, &sms, &dev);
  if (rc) return rc;
  ema::PagedDecodeParams p{};
  for (int j = 0; j < 2; ++j) {
    p.base[j] = static_cast<uint8_t*>(c->base[j]);
    p.block_stride[j] = stride[j];
    p.blocks[j] = c->blocks[j];
  }
  p.dtype = c->dtype;
  p.num_kv_heads = c->num_kv_heads;
  p.head_dim = c->head_dim;
  p.block_tokens = c->block_tokens;
  p.block_shift = block_shift(c->block_tokens);
  p.tables = a->tables;
  p.table_stride = a->table_stride;
  p.max_blocks = a->max_blocks;
  p.lens = a->lens;
  p.nseq = a->nseq;
  p.q = static_cast<const uint8_t*>(a->q);
  p.q_stride = a->q_stride;
  p.rows = rows;
  p.window = a->window;
  // The kernel works with a scale above 0: the sign goes to q, and a scale of 0 is a query of zeros. (Not a number: every
  // comparison is false, and the scale itself makes the result one.)
  p.scale_log2 = (a->sm_scale < 0.f ? -a->sm_scale : a->sm_scale) * 1.4426950408889634f;
  p.q_keep = 0xffffffffu;
  p.q_flip = a->sm_scale < 0.f ? 0x80008000u : 0u;
  if (p.scale_log2 == 0.f) {
    p.scale_log2 = 1.f;
    p.q_keep = p.q_flip = 0u;
  }
  p.out = static_cast<uint8_t*>(a->out);
  p.out_stride = a->out_stride;
  p.lse = a->lse;
  p.counters = static_cast<uint32_t*>(a->workspace);
  p.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(a->workspace) + ema::kPagedCounterBytes);
  p.lam = a->lam;
  p.norm_weight = a->norm_weight;
  p.eps = a->eps;
  p.out_scale = a->out_scale;
  p.status = a->status;
  return launched(ema::launch_paged_decode(p, dev, sms, static_cast<cudaStream_t>(stream)));
}

}  // namespace

extern "C" {

int paged_build_tables(const paged_build_tables_t* a, void* stream) {
  if (!a || !a->pool) return SLICE_EINVAL;
  const paged_pool_t& pool = *a->pool;
  if (!pool.free_in || !pool.free_out || !pool.work || !block_shift(a->block_tokens)) return SLICE_EINVAL;
  if (!aligned(pool.free_in, 4) || !aligned(pool.free_out, 4) || !aligned(pool.work, 4) || !aligned(a->status, 4)) return SLICE_EINVAL;
  for (int j = 0; j < 2; ++j)
    if ((pool.capacity[j] && !pool.ids[j]) || pool.capacity[j] > kMost || !aligned(pool.ids[j], 4)) return SLICE_EINVAL;
  if (pool.free_out == pool.free_in + 1 || pool.free_in == pool.free_out + 1) return SLICE_EINVAL;  // the same counts, or others
  if (!a->offsets || !aligned(a->offsets, 4) || a->nseq > kMost - 1 || a->max_tokens > kMost) return SLICE_EINVAL;
  if (a->nseq && (!a->lens || !a->new_lens || !a->tables || !aligned(a->lens, 4) || !aligned(a->new_lens, 4) || !aligned(a->tables, 4)))
    return SLICE_EINVAL;
  if (a->nseq && (a->max_blocks == 0 || a->table_stride < a->max_blocks || static_cast<uint64_t>(a->max_blocks) * a->block_tokens > kMost))
    return SLICE_EINVAL;
  if (a->max_tokens && (!a->slots || !a->positions || !aligned(a->slots, 8) || !aligned(a->positions, 4))) return SLICE_EINVAL;
  int sms = 0;
  const int rc = device_ok(a->offsets, &sms);
  if (rc) return rc;
  ema::BuildTablesParams p{};
  for (int j = 0; j < 2; ++j) {
    p.ids[j] = pool.ids[j];
    p.capacity[j] = pool.capacity[j];
  }
  p.free_in = pool.free_in;
  p.free_out = pool.free_out;
  p.work = pool.work;
  p.lens = a->lens;
  p.new_lens = a->new_lens;
  p.nseq = a->nseq;
  p.block_shift = block_shift(a->block_tokens);
  p.tables = a->tables;
  p.table_stride = a->table_stride;
  p.max_blocks = a->max_blocks;
  p.offsets = a->offsets;
  p.slots = a->slots;
  p.positions = a->positions;
  p.max_tokens = a->max_tokens;
  p.status = a->status;
  return launched(ema::launch_build_tables(p, sms, static_cast<cudaStream_t>(stream)));
}

int paged_write_kv(const paged_write_kv_t* a, void* stream) {
  if (!a) return SLICE_EINVAL;
  const paged_cache_t* c = a->cache;
  uint64_t stride[2];
  if (!cache_ok(c, stride)) return SLICE_EINVAL;
  if (a->ntok == 0) return SLICE_OK;
  if (!a->k || !a->v || !a->slots || a->ntok > kMost || !aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->slots, 8) ||
      !aligned(a->status, 4))
    return SLICE_EINVAL;
  const uint32_t row = c->num_kv_heads * c->head_dim * 2;
  if (((a->k_stride | a->v_stride) & 15u) || (a->ntok > 1 && (a->k_stride < row || a->v_stride < row))) return SLICE_EINVAL;
  int sms = 0;
  const int rc = device_ok(a->slots, &sms);
  if (rc) return rc;
  ema::WriteKvParams p{};
  for (int j = 0; j < 2; ++j) {
    p.base[j] = static_cast<uint8_t*>(c->base[j]);
    p.block_stride[j] = stride[j];
    p.blocks[j] = c->blocks[j];
  }
  p.block_shift = block_shift(c->block_tokens);
  p.row_bytes = row;
  p.k = static_cast<const uint8_t*>(a->k);
  p.v = static_cast<const uint8_t*>(a->v);
  p.k_stride = a->k_stride;
  p.v_stride = a->v_stride;
  p.slots = a->slots;
  p.ntok = a->ntok;
  p.status = a->status;
  return launched(ema::launch_write_kv(p, static_cast<cudaStream_t>(stream)));
}

int paged_decode_workspace(const paged_cache_t* c, uint32_t num_q_rows, uint64_t* out_bytes) {
  uint64_t stride[2];
  if (!out_bytes || !cache_ok(c, stride) || num_q_rows == 0 || num_q_rows % c->num_kv_heads || num_q_rows / c->num_kv_heads > 16)
    return SLICE_EINVAL;
  *out_bytes = ema::paged_workspace_bytes(num_q_rows / c->num_kv_heads, c->head_dim);
  return SLICE_OK;
}

int paged_decode_tables(const paged_decode_t* a, void* stream) { return decode(a, false, stream); }

int paged_decode_diff(const paged_decode_t* a, void* stream) { return decode(a, true, stream); }

}  // extern "C"
