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

// The kernels work with a scale above 0: the sign goes to q, and a scale of 0 is a query of zeros. (Not a number: every
// comparison is false, and the scale itself makes the result one.)
void scale_of(float sm_scale, float& scale_log2, uint32_t& q_keep, uint32_t& q_flip) {
  scale_log2 = (sm_scale < 0.f ? -sm_scale : sm_scale) * 1.4426950408889634f;
  q_keep = 0xffffffffu;
  q_flip = sm_scale < 0.f ? 0x80008000u : 0u;
  if (scale_log2 == 0.f) {
    scale_log2 = 1.f;
    q_keep = q_flip = 0u;
  }
}

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
  scale_of(a->sm_scale, p.scale_log2, p.q_keep, p.q_flip);
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

// Layers that differ in their bases only; those go to p.
bool layers_ok(const paged_cache_t* c, uint32_t n, ema::MoveParams& p) {
  uint64_t first[2], stride[2];
  if (!c || n == 0 || n > ema::kMoveLayers || !cache_ok(c, first)) return false;
  for (uint32_t l = 0; l < n; ++l) {
    if (!cache_ok(c + l, stride) || c[l].dtype != c->dtype || c[l].num_kv_heads != c->num_kv_heads || c[l].head_dim != c->head_dim ||
        c[l].block_tokens != c->block_tokens)
      return false;
    for (int j = 0; j < 2; ++j) {
      if (c[l].blocks[j] != c->blocks[j] || (c->blocks[j] && stride[j] != first[j])) return false;
      p.base[j][l] = static_cast<uint8_t*>(c[l].base[j]);
    }
  }
  for (int j = 0; j < 2; ++j) {
    p.block_stride[j] = first[j];
    p.blocks[j] = c->blocks[j];
  }
  p.nlayers = n;
  p.row_bytes = c->num_kv_heads * c->head_dim * 2;
  p.block_shift = block_shift(c->block_tokens);
  return true;
}

// The workspace of shares: words of the compaction (how many blocks moved, counters), a bit per block, then the entries that blocks move to.
constexpr uint64_t kShareWords = 16;

uint64_t bit_words(uint32_t blocks) { return (static_cast<uint64_t>(blocks) + 31) / 32; }

uint64_t share_bytes(uint32_t b0, uint32_t b1) { return 4 * (kShareWords + bit_words(b0) + bit_words(b1) + b0 + b1); }

bool pool_ok(const paged_pool_t* pool) {
  if (!pool || !pool->free_in || !pool->free_out || !pool->work) return false;
  if (!aligned(pool->free_in, 4) || !aligned(pool->free_out, 4) || !aligned(pool->work, 4)) return false;
  for (int j = 0; j < 2; ++j)
    if ((pool->capacity[j] && !pool->ids[j]) || pool->capacity[j] > kMost || !aligned(pool->ids[j], 4)) return false;
  return pool->free_out != pool->free_in + 1 && pool->free_in != pool->free_out + 1;  // the same counts, or others
}

// What the calls on shared blocks have in common. SLICE_OK, or what is to be returned.
int pages_params(const paged_pool_t* pool, const paged_shares_t* shares, const int32_t* lens, const int32_t* tables, uint64_t table_stride, const int32_t* status,
                 uint32_t nseq, uint32_t block_tokens, uint32_t max_blocks, ema::PagesParams& p) {
  if (!pool_ok(pool) || !shares || !block_shift(block_tokens) || nseq > kMost - 1 || !aligned(status, 4)) return SLICE_EINVAL;
  for (int j = 0; j < 2; ++j)
    if (shares->blocks[j] > kMost || (shares->blocks[j] && !shares->refs[j]) || !aligned(shares->refs[j], 4)) return SLICE_EINVAL;
  if (!shares->work || !aligned(shares->work, 4)) return SLICE_EINVAL;
  if (shares->work_bytes < share_bytes(shares->blocks[0], shares->blocks[1])) return SLICE_ESCRATCH;
  if (nseq && (!lens || !tables || !aligned(lens, 4) || !aligned(tables, 4) || max_blocks == 0 || table_stride < max_blocks ||
               static_cast<uint64_t>(max_blocks) * block_tokens > kMost))
    return SLICE_EINVAL;
  uint32_t* word = static_cast<uint32_t*>(shares->work);
  p.moved = word;
  word += kShareWords;
  for (int j = 0; j < 2; ++j) {
    p.bits[j] = word;
    word += bit_words(shares->blocks[j]);
  }
  for (int j = 0; j < 2; ++j) {
    p.map[j] = reinterpret_cast<int32_t*>(word);
    word += shares->blocks[j];
    p.ids[j] = pool->ids[j];
    p.capacity[j] = pool->capacity[j];
    p.refs[j] = shares->refs[j];
    p.blocks[j] = shares->blocks[j];
  }
  p.free_in = pool->free_in;
  p.free_out = pool->free_out;
  p.work = pool->work;
  p.lens = lens;
  p.tables = const_cast<int32_t*>(tables);
  p.table_stride = table_stride;
  p.nseq = nseq;
  p.max_blocks = max_blocks;
  p.block_shift = block_shift(block_tokens);
  p.status = const_cast<int32_t*>(status);
  return SLICE_OK;
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

int paged_tree_workspace(const paged_cache_t* c, uint32_t num_heads, uint64_t* out_bytes) {
  uint64_t stride[2];
  if (!out_bytes || !cache_ok(c, stride) || num_heads == 0 || num_heads % c->num_kv_heads || num_heads / c->num_kv_heads > 128) return SLICE_EINVAL;
  *out_bytes = ema::tree_workspace_bytes(c->head_dim);
  return SLICE_OK;
}

int paged_tree_attention(const paged_tree_t* a, void* stream) {
  if (!a) return SLICE_EINVAL;
  const paged_cache_t* c = a->cache;
  uint64_t stride[2];
  if (!cache_ok(c, stride)) return SLICE_EINVAL;
  if (a->num_heads == 0 || a->num_heads % c->num_kv_heads || a->num_heads / c->num_kv_heads > 128) return SLICE_EINVAL;
  if (a->mask ? a->mask_words == 0 || a->mask_words > (1u << 25) || a->mask_stride < a->mask_words || a->mask_stride >= (1ull << 40) : a->mask_words != 0)
    return SLICE_EINVAL;
  if (a->nseq == 0 || a->ntok == 0) return SLICE_OK;
  if (!a->tables || !a->lens || !a->offsets || !a->q || !a->out || !a->workspace || a->ntok > kMost || a->nseq > kMost - 1) return SLICE_EINVAL;
  if (a->max_blocks == 0 || a->table_stride < a->max_blocks || static_cast<uint64_t>(a->max_blocks) * c->block_tokens > kMost) return SLICE_EINVAL;
  const uint64_t row = static_cast<uint64_t>(a->num_heads) * c->head_dim * 2;
  if ((a->ntok > 1 && (a->q_stride < row || a->out_stride < row || a->q_stride >= (1ull << 40))) || ((a->q_stride | a->out_stride) & 15u)) return SLICE_EINVAL;
  if (!aligned(a->q, 16) || !aligned(a->out, 16) || !aligned(a->workspace, 16) || !aligned(a->tables, 4) || !aligned(a->lens, 4) ||
      !aligned(a->offsets, 4) || !aligned(a->lse, 4) || !aligned(a->mask, 8) || !aligned(a->positions, 4) || !aligned(a->status, 4))
    return SLICE_EINVAL;
  if (a->workspace_bytes < ema::tree_workspace_bytes(c->head_dim)) return SLICE_ESCRATCH;
  int sms = 0, dev = 0;
  const int rc = device_ok(a->out, &sms, &dev);
  if (rc) return rc;
  ema::TreeParams p{};
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
  p.offsets = a->offsets;
  p.nseq = a->nseq;
  p.ntok = a->ntok;
  p.q = static_cast<const uint8_t*>(a->q);
  p.q_stride = a->q_stride;
  p.out = static_cast<uint8_t*>(a->out);
  p.out_stride = a->out_stride;
  p.lse = a->lse;
  p.mask = reinterpret_cast<const uint32_t*>(a->mask);
  p.mask_stride = 2 * a->mask_stride;
  p.mask_words = 2 * a->mask_words;
  p.positions = a->positions;
  p.group = a->num_heads / c->num_kv_heads;
  p.window = a->window;
  scale_of(a->sm_scale, p.scale_log2, p.q_keep, p.q_flip);
  p.notes = static_cast<uint8_t*>(a->workspace);
  p.parts = reinterpret_cast<float*>(p.notes + ema::kTreeNotesBytes);
  p.status = a->status;
  return launched(ema::launch_tree(p, dev, sms, static_cast<cudaStream_t>(stream)));
}

int paged_keep_rows(const paged_keep_rows_t* a, void* stream) {
  if (!a) return SLICE_EINVAL;
  ema::MoveParams p{};
  if (!layers_ok(a->layers, a->nlayers, p) || !aligned(a->status, 4)) return SLICE_EINVAL;
  if (a->nseq == 0 || a->max_keep == 0) return SLICE_OK;
  if (!a->tables || !a->lens || !a->keep || !a->counts || !aligned(a->tables, 4) || !aligned(a->lens, 4) || !aligned(a->keep, 4) || !aligned(a->counts, 4))
    return SLICE_EINVAL;
  if (a->nseq > kMost || a->max_keep > kMost || a->keep_stride < a->max_keep || a->max_blocks == 0 || a->table_stride < a->max_blocks ||
      (static_cast<uint64_t>(a->max_blocks) << p.block_shift) > kMost)
    return SLICE_EINVAL;
  int sms = 0;
  const int rc = device_ok(a->counts, &sms);
  if (rc) return rc;
  p.tables = a->tables;
  p.table_stride = a->table_stride;
  p.max_blocks = a->max_blocks;
  p.lens = a->lens;
  p.keep = a->keep;
  p.keep_stride = a->keep_stride;
  p.max_keep = a->max_keep;
  p.counts = a->counts;
  p.nseq = a->nseq;
  p.status = a->status;
  return launched(ema::launch_keep_rows(p, static_cast<cudaStream_t>(stream)));
}

int paged_copy_blocks(const paged_copy_blocks_t* a, void* stream) {
  if (!a) return SLICE_EINVAL;
  ema::MoveParams p{};
  if (!layers_ok(a->layers, a->nlayers, p) || !aligned(a->status, 4)) return SLICE_EINVAL;
  if (a->ncopies == 0) return SLICE_OK;
  if (!a->copies || !aligned(a->copies, 4) || a->ncopies > kMost) return SLICE_EINVAL;
  int sms = 0;
  const int rc = device_ok(a->copies, &sms);
  if (rc) return rc;
  p.copies = a->copies;
  p.ncopies = a->ncopies;
  p.status = a->status;
  return launched(ema::launch_copy_rows(p, sms, static_cast<cudaStream_t>(stream)));
}

int paged_shares_workspace(uint32_t blocks0, uint32_t blocks1, uint64_t* out_bytes) {
  if (!out_bytes || blocks0 > kMost || blocks1 > kMost) return SLICE_EINVAL;
  *out_bytes = share_bytes(blocks0, blocks1);
  return SLICE_OK;
}

int paged_fork(const paged_fork_t* a, void* stream) {
  if (!a) return SLICE_EINVAL;
  ema::PagesParams p{};
  int rc = pages_params(a->pool, a->shares, a->lens, a->tables, a->table_stride, a->status, a->nseq, a->block_tokens, a->max_blocks, p);
  if (rc) return rc;
  if (a->nfork && (a->nseq == 0 || a->nseq > 262144 || a->nfork > kMost || !a->new_lens || !a->src || !a->dst || !a->copies || !aligned(a->new_lens, 4) ||
                   !aligned(a->src, 4) || !aligned(a->dst, 4) || !aligned(a->copies, 4)))
    return SLICE_EINVAL;
  int sms = 0;
  rc = device_ok(p.free_out, &sms);
  if (rc) return rc;
  if (a->nfork == 0) p.nseq = 0;  // the tops only
  p.new_lens_out = a->new_lens;
  p.src = a->src;
  p.dst = a->dst;
  p.nfork = a->nfork;
  p.copies = a->copies;
  return launched(ema::launch_fork(p, sms, static_cast<cudaStream_t>(stream)));
}

int paged_free(const paged_free_t* a, void* stream) {
  if (!a) return SLICE_EINVAL;
  ema::PagesParams p{};
  int rc = pages_params(a->pool, a->shares, a->lens, a->tables, a->table_stride, a->status, a->nseq, a->block_tokens, a->max_blocks, p);
  if (rc) return rc;
  if (a->nseq && (!a->new_lens || !aligned(a->new_lens, 4))) return SLICE_EINVAL;
  int sms = 0;
  rc = device_ok(p.free_out, &sms);
  if (rc) return rc;
  p.new_lens = a->new_lens;
  return launched(ema::launch_free(p, sms, static_cast<cudaStream_t>(stream)));
}

int paged_compact(const paged_compact_t* a, void* stream) {
  if (!a) return SLICE_EINVAL;
  ema::PagesParams p{};
  int rc = pages_params(a->pool, a->shares, a->lens, a->tables, a->table_stride, a->status, a->nseq, a->block_tokens, a->max_blocks, p);
  if (rc) return rc;
  if (!a->limits || !aligned(a->limits, 4) || a->max_copies > kMost || (a->max_copies && !a->copies) || !aligned(a->copies, 4)) return SLICE_EINVAL;
  int sms = 0;
  rc = device_ok(p.free_out, &sms);
  if (rc) return rc;
  p.limits = a->limits;
  p.copies = a->copies;
  p.ncopies = a->max_copies;
  return launched(ema::launch_compact(p, sms, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
