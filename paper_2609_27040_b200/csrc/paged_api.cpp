// paged_api.cpp — C entry points of the device-driven path: checks of what the host can see, then one
// launch each. No state is kept between calls (apart from per-device constants), nothing is allocated.
#include <cuda_runtime.h>
#include <stdint.h>

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

// The call's memory has to be reachable from the current device: memory of another one is refused.
int device_ok(const void* p, int* sms) {
  static int sms_of[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SLICE_ECUDA;
  cudaPointerAttributes at{};
  if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
    cudaGetLastError();
    return SLICE_EINVAL;
  }
  if (at.type == cudaMemoryTypeDevice && at.device != dev) return SLICE_EINVAL;
  if (at.type == cudaMemoryTypeUnregistered) return SLICE_EINVAL;
  if (!sms_of[dev] && cudaDeviceGetAttribute(&sms_of[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return SLICE_ECUDA;
  *sms = sms_of[dev];
  return SLICE_OK;
}

int launched(cudaError_t e) { return e == cudaSuccess ? SLICE_OK : SLICE_ECUDA; }

int decode(const paged_cache_t* c, const int32_t* tables, uint64_t table_stride, uint32_t max_blocks, const int32_t* lens,
           uint32_t nseq, const void* q, uint64_t q_stride, uint32_t rows, uint32_t out_heads, const float* lam, float sm_scale,
           uint32_t window, const float* norm_weight, float eps, float out_scale, void* out, uint64_t out_stride, float* lse,
           void* workspace, uint64_t workspace_bytes, int32_t* status, void* stream) {
  uint64_t stride[2];
  if (!cache_ok(c, stride)) return SLICE_EINVAL;
  if (rows == 0 || rows > 16) return SLICE_EINVAL;
  if (nseq == 0) return SLICE_OK;
  if (!tables || !lens || !q || !out || !workspace || static_cast<uint64_t>(nseq) * c->num_kv_heads > kMost / 2) return SLICE_EINVAL;
  if (max_blocks == 0 || table_stride < max_blocks || static_cast<uint64_t>(max_blocks) * c->block_tokens > kMost) return SLICE_EINVAL;
  const uint64_t q_row = static_cast<uint64_t>(rows) * c->num_kv_heads * (lam ? c->head_dim / 2 : c->head_dim) * 2;
  const uint64_t out_row = static_cast<uint64_t>(out_heads) * c->head_dim * 2;
  if ((nseq > 1 && (q_stride < q_row || out_stride < out_row)) || ((q_stride | out_stride) & 15u)) return SLICE_EINVAL;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16) || !aligned(tables, 4) || !aligned(lens, 4) || !aligned(lse, 4) ||
      !aligned(lam, 4) || !aligned(norm_weight, 4) || !aligned(status, 4))
    return SLICE_EINVAL;
  if (workspace_bytes < ema::paged_workspace_bytes(rows, c->head_dim)) return SLICE_ESCRATCH;
  int sms = 0;
  const int rc = device_ok(out, &sms);
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
  p.tables = tables;
  p.table_stride = table_stride;
  p.max_blocks = max_blocks;
  p.lens = lens;
  p.nseq = nseq;
  p.q = static_cast<const uint8_t*>(q);
  p.q_stride = q_stride;
  p.rows = rows;
  p.window = window;
  // The kernel works with a scale above 0: the sign goes to q, and a scale of 0 is a query of zeros. (Not a number: every
  // comparison is false, and the scale itself makes the result one.)
  p.scale_log2 = (sm_scale < 0.f ? -sm_scale : sm_scale) * 1.4426950408889634f;
  p.q_keep = 0xffffffffu;
  p.q_flip = sm_scale < 0.f ? 0x80008000u : 0u;
  if (p.scale_log2 == 0.f) {
    p.scale_log2 = 1.f;
    p.q_keep = p.q_flip = 0u;
  }
  p.out = static_cast<uint8_t*>(out);
  p.out_stride = out_stride;
  p.lse = lse;
  p.counters = static_cast<uint32_t*>(workspace);
  p.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + ema::kPagedCounterBytes);
  p.lam = lam;
  p.norm_weight = norm_weight;
  p.eps = eps;
  p.out_scale = out_scale;
  p.status = status;
  return launched(ema::launch_paged_decode(p, sms, static_cast<cudaStream_t>(stream)));
}

}  // namespace

extern "C" {

int paged_build_tables(const paged_pool_t* pool, const int32_t* lens, const int32_t* new_lens, uint32_t nseq, uint32_t block_tokens,
                       int32_t* tables, uint64_t table_stride, uint32_t max_blocks, int32_t* offsets, int64_t* slots, int32_t* positions,
                       uint32_t max_tokens, int32_t* status, void* stream) {
  if (!pool || !pool->free_in || !pool->free_out || !pool->work || !block_shift(block_tokens)) return SLICE_EINVAL;
  if (!aligned(pool->free_in, 4) || !aligned(pool->free_out, 4) || !aligned(pool->work, 4) || !aligned(status, 4)) return SLICE_EINVAL;
  for (int j = 0; j < 2; ++j)
    if ((pool->capacity[j] && !pool->ids[j]) || pool->capacity[j] > kMost || !aligned(pool->ids[j], 4)) return SLICE_EINVAL;
  if (!offsets || !aligned(offsets, 4) || nseq > kMost - 1 || max_tokens > kMost) return SLICE_EINVAL;
  if (nseq && (!lens || !new_lens || !tables || !aligned(lens, 4) || !aligned(new_lens, 4) || !aligned(tables, 4))) return SLICE_EINVAL;
  if (nseq && (max_blocks == 0 || table_stride < max_blocks || static_cast<uint64_t>(max_blocks) * block_tokens > kMost)) return SLICE_EINVAL;
  if (max_tokens && (!slots || !positions || !aligned(slots, 8) || !aligned(positions, 4))) return SLICE_EINVAL;
  int sms = 0;
  const int rc = device_ok(offsets, &sms);
  if (rc) return rc;
  ema::BuildTablesParams p{};
  for (int j = 0; j < 2; ++j) {
    p.ids[j] = pool->ids[j];
    p.capacity[j] = pool->capacity[j];
  }
  p.free_in = pool->free_in;
  p.free_out = pool->free_out;
  p.work = pool->work;
  p.lens = lens;
  p.new_lens = new_lens;
  p.nseq = nseq;
  p.block_shift = block_shift(block_tokens);
  p.tables = tables;
  p.table_stride = table_stride;
  p.max_blocks = max_blocks;
  p.offsets = offsets;
  p.slots = slots;
  p.positions = positions;
  p.max_tokens = max_tokens;
  p.status = status;
  return launched(ema::launch_build_tables(p, sms, static_cast<cudaStream_t>(stream)));
}

int paged_write_kv(const paged_cache_t* c, const void* k, uint64_t k_stride, const void* v, uint64_t v_stride, const int64_t* slots,
                   uint32_t ntok, int32_t* status, void* stream) {
  uint64_t stride[2];
  if (!cache_ok(c, stride)) return SLICE_EINVAL;
  if (ntok == 0) return SLICE_OK;
  if (!k || !v || !slots || ntok > kMost || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8) || !aligned(status, 4)) return SLICE_EINVAL;
  const uint32_t row = c->num_kv_heads * c->head_dim * 2;
  if (((k_stride | v_stride) & 15u) || (ntok > 1 && (k_stride < row || v_stride < row))) return SLICE_EINVAL;
  int sms = 0;
  const int rc = device_ok(slots, &sms);
  if (rc) return rc;
  ema::WriteKvParams p{};
  for (int j = 0; j < 2; ++j) {
    p.base[j] = static_cast<uint8_t*>(c->base[j]);
    p.block_stride[j] = stride[j];
    p.blocks[j] = c->blocks[j];
  }
  p.block_shift = block_shift(c->block_tokens);
  p.row_bytes = row;
  p.k = static_cast<const uint8_t*>(k);
  p.v = static_cast<const uint8_t*>(v);
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.slots = slots;
  p.ntok = ntok;
  p.status = status;
  return launched(ema::launch_write_kv(p, static_cast<cudaStream_t>(stream)));
}

int paged_decode_workspace(const paged_cache_t* c, uint32_t num_q_rows, uint64_t* out_bytes) {
  uint64_t stride[2];
  if (!out_bytes || !cache_ok(c, stride) || num_q_rows == 0 || num_q_rows % c->num_kv_heads || num_q_rows / c->num_kv_heads > 16)
    return SLICE_EINVAL;
  *out_bytes = ema::paged_workspace_bytes(num_q_rows / c->num_kv_heads, c->head_dim);
  return SLICE_OK;
}

int paged_decode_tables(const paged_cache_t* c, const int32_t* tables, uint64_t table_stride, uint32_t max_blocks, const int32_t* lens,
                        uint32_t nseq, const void* q, uint64_t q_stride, uint32_t num_q_heads, float sm_scale, uint32_t window, void* out,
                        uint64_t out_stride, float* lse_or_null, void* workspace, uint64_t workspace_bytes, int32_t* status, void* stream) {
  if (!c || c->num_kv_heads == 0 || num_q_heads % c->num_kv_heads) return SLICE_EINVAL;
  return decode(c, tables, table_stride, max_blocks, lens, nseq, q, q_stride, num_q_heads / c->num_kv_heads, num_q_heads, nullptr, sm_scale,
                window, nullptr, 0.f, 1.f, out, out_stride, lse_or_null, workspace, workspace_bytes, status, stream);
}

int paged_decode_diff(const paged_cache_t* c, const int32_t* tables, uint64_t table_stride, uint32_t max_blocks, const int32_t* lens,
                      uint32_t nseq, const void* q, uint64_t q_stride, uint32_t num_heads, const float* lam, float sm_scale, uint32_t window,
                      const float* norm_weight_or_null, float eps, float out_scale, void* out, uint64_t out_stride, void* workspace,
                      uint64_t workspace_bytes, int32_t* status, void* stream) {
  if (!c || c->num_kv_heads == 0 || num_heads % c->num_kv_heads || !lam || num_heads / c->num_kv_heads > 8) return SLICE_EINVAL;
  if (norm_weight_or_null && !(eps >= 0.f)) return SLICE_EINVAL;
  return decode(c, tables, table_stride, max_blocks, lens, nseq, q, q_stride, 2 * (num_heads / c->num_kv_heads), num_heads, lam, sm_scale,
                window, norm_weight_or_null, eps, out_scale, out, out_stride, nullptr, workspace, workspace_bytes, status, stream);
}

}  // extern "C"
