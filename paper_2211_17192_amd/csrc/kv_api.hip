// C-ABI entry points of the paged key-value cache apart from a model: rows in, rows out, attention.  See include/sd.h.
#include <hip/hip_runtime.h>
#include <cmath>
#include <cstdint>
#include <string>
#include "../../include/sd.h"
#include "kernels_kv.h"

namespace {
static_assert(SD_KV_MAX_LEN == sd::KV_MAX_RANGES * sd::KV_MAX_RANGE_KEYS, "sd.h states the longest context");
static_assert(SD_KV_MAX_GROUPS == sd::KV_TICKETS, "sd.h states the tickets of a call");

sd_status kv_fail(sd_status st, const char* what) noexcept {
  try { g_load_error = what; } catch (...) {}
  return st;
}
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

sd_status kv_cache_args(const sd_kv_cache* c, sd::KvCacheArgs& a) {
  if (!c || !c->pool || !c->page_table) return kv_fail(SD_EINVAL, "null cache, pool or page table");
  if (c->dtype != SD_BF16 && c->dtype != SD_E4M3) return kv_fail(SD_EINVAL, "a cache holds SD_BF16 or SD_E4M3");
  if (c->dtype == SD_E4M3 && !c->exps) return kv_fail(SD_EINVAL, "an SD_E4M3 cache needs exps");
  if (!aligned16(c->pool) || (c->dtype == SD_E4M3 && !aligned16(c->exps))) return kv_fail(SD_EINVAL, "pool and exps must be 16-byte aligned");
  if (c->d_head != 32 && c->d_head != 64 && c->d_head != 128) return kv_fail(SD_EINVAL, "d_head must be 32, 64 or 128");
  if (c->page_size < 16 || (c->page_size & (c->page_size - 1))) return kv_fail(SD_EINVAL, "page_size must be a power of two >= 16");
  if (c->n_pages < 1 || c->n_seq < 1 || c->table_stride < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535)
    return kv_fail(SD_EINVAL, "non-positive size of the cache, or more than 65535 kv heads");
  if ((int64_t)c->page_size * c->n_kv_heads > (1 << 28)) return kv_fail(SD_EINVAL, "a page of more than 2^28 rows");
  a.pool = c->pool; a.exps = c->exps; a.table = c->page_table; a.n_pages = c->n_pages; a.n_seq = c->n_seq;
  a.table_stride = c->table_stride; a.page_shift = __builtin_ctz((unsigned)c->page_size); a.Hkv = c->n_kv_heads;
  return SD_OK;
}

sd_status kv_rows(const sd_kv_cache* cache, const sd_kv_rows* x, const int32_t* seq, const int32_t* pos, int32_t rows, void* stream, bool append) {
  sd::KvRowsArgs a{};
  const sd_status st = kv_cache_args(cache, a.c);
  if (st != SD_OK) return st;
  if (rows < 0) return kv_fail(SD_EINVAL, "negative number of rows");
  if (rows == 0) return SD_OK;
  if (!x || !x->k || !x->v) return kv_fail(SD_EINVAL, "null rows");
  if (x->dtype != SD_F32 && x->dtype != SD_BF16) return kv_fail(SD_EINVAL, "rows are SD_F32 or SD_BF16");
  const int64_t block_rows = sd::KV_ROW_BYTES / (cache->d_head * (x->dtype == SD_F32 ? 4 : 2));
  if (((int64_t)rows + block_rows - 1) / block_rows * cache->n_kv_heads >= 1 << 24) return kv_fail(SD_ERANGE, "too many rows");      // 2^32 threads
  if (!aligned16(x->k) || !aligned16(x->v)) return kv_fail(SD_EINVAL, "rows must be 16-byte aligned");
  if ((x->k_row_stride | x->k_head_stride | x->v_row_stride | x->v_head_stride) & 7) return kv_fail(SD_EINVAL, "strides must be multiples of 8 elements");
  if (!seq && rows % cache->n_seq) return kv_fail(SD_EINVAL, "without seq every sequence has the same number of rows");
  a.seq = seq; a.pos = pos; a.rows = rows;
  a.per_seq = seq ? rows : rows / cache->n_seq;
  a.k = x->k; a.v = x->v; a.k_row = x->k_row_stride; a.k_head = x->k_head_stride; a.v_row = x->v_row_stride; a.v_head = x->v_head_stride;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool e4m3 = cache->dtype == SD_E4M3;
  if (x->dtype == SD_F32) sd::launch_kv_rows<float>(s, a, cache->d_head, e4m3, append);
  else sd::launch_kv_rows<sd::bf16>(s, a, cache->d_head, e4m3, append);
  return hipGetLastError() == hipSuccess ? SD_OK : kv_fail(SD_EHIP, "kernel launch");
}

// The checks that the scratch's size depends on.
sd_status kv_attention_plan(const sd_kv_cache* c, int32_t n_heads, int32_t rows, int32_t max_len, int32_t dtype, sd::KvPlan& p) {
  if (n_heads < 1 || n_heads % c->n_kv_heads) return kv_fail(SD_EINVAL, "n_heads must be a multiple of n_kv_heads");
  if (rows < 1) return kv_fail(SD_EINVAL, "rows must be positive");
  if (max_len < 1 || max_len > SD_KV_MAX_LEN) return kv_fail(SD_ERANGE, "max_len outside 1 .. SD_KV_MAX_LEN");
  if (c->n_seq > 65535) return kv_fail(SD_ERANGE, "more than 65535 sequences");
  const int64_t pairs = (int64_t)rows * (n_heads / c->n_kv_heads);
  if (pairs > 65535 || (int64_t)c->n_seq * rows * n_heads > 0x7fffffff / 128) return kv_fail(SD_ERANGE, "too many rows");
  p = sd::kv_plan(c->n_seq, c->n_kv_heads, (int)pairs, max_len, c->d_head, c->dtype == SD_E4M3, dtype == SD_F32);
  if ((int64_t)c->n_seq * c->n_kv_heads * p.groups > SD_KV_MAX_GROUPS)
    return kv_fail(SD_ERANGE, "more than SD_KV_MAX_GROUPS (sequence, 16 rows, kv head)s");
  return SD_OK;
}
}  // namespace

extern "C" sd_status sd_kv_append(const sd_kv_cache* cache, const sd_kv_rows* rows_in, const int32_t* seq, const int32_t* pos, int32_t rows, void* stream) {
  return kv_rows(cache, rows_in, seq, pos, rows, stream, true);
}

extern "C" sd_status sd_kv_read(const sd_kv_cache* cache, const sd_kv_rows* rows_out, const int32_t* seq, const int32_t* pos, int32_t rows, void* stream) {
  return kv_rows(cache, rows_out, seq, pos, rows, stream, false);
}

extern "C" size_t sd_kv_attention_scratch_bytes(const sd_kv_cache* cache, int32_t n_heads, int32_t rows, int32_t max_len) {
  sd::KvCacheArgs a{};
  size_t most = 0;
  for (int32_t dtype : {SD_F32, SD_BF16}) {          // (they are cut differently)
    sd::KvPlan p{};
    if (kv_cache_args(cache, a) != SD_OK || kv_attention_plan(cache, n_heads, rows, max_len, dtype, p) != SD_OK) return 0;
    const size_t n = sd::kv_scratch_bytes(cache->n_seq, cache->n_kv_heads, cache->d_head, p);
    if (n > most) most = n;
  }
  return most;
}

extern "C" sd_status sd_kv_attention(const sd_kv_cache* cache, const void* q, int64_t q_row_stride, int64_t q_head_stride, int32_t dtype, const int32_t* pos,
                                     int32_t n_heads, int32_t rows, int32_t max_len, float scale, void* out, float* lse,
                                     void* scratch, size_t scratch_bytes, void* stream) {
  sd::KvAttnArgs a{};
  sd::KvPlan p{};
  sd_status st = kv_cache_args(cache, a.c);
  if (st == SD_OK && dtype != SD_F32 && dtype != SD_BF16) st = kv_fail(SD_EINVAL, "queries are SD_F32 or SD_BF16");
  if (st == SD_OK) st = kv_attention_plan(cache, n_heads, rows, max_len, dtype, p);
  if (st != SD_OK) return st;
  if (!q || !pos || !out || !scratch) return kv_fail(SD_EINVAL, "null pointer");
  if (!aligned16(q) || !aligned16(out) || !aligned16(scratch)) return kv_fail(SD_EINVAL, "q, out and scratch must be 16-byte aligned");
  if ((q_row_stride | q_head_stride) & 7) return kv_fail(SD_EINVAL, "strides must be multiples of 8 elements");
  a.c_log2 = scale * 1.44269504088896340736f;
  if (!(scale > 0.0f) || !std::isfinite(a.c_log2)) return kv_fail(SD_EINVAL, "scale must be positive");
  if (scratch_bytes < sd::kv_scratch_bytes(cache->n_seq, cache->n_kv_heads, cache->d_head, p)) return kv_fail(SD_ENOMEM, "scratch too small: see sd_kv_attention_scratch_bytes");
  a.q = q; a.q_row = q_row_stride; a.q_head = q_head_stride; a.out = out; a.lse = lse; a.pos = pos;
  a.R = rows; a.H = n_heads; a.G = n_heads / cache->n_kv_heads;
  a.n_seq = cache->n_seq; a.max_len = max_len;
  sd::kv_set_plan(a, p);
  a.tickets = static_cast<unsigned*>(scratch);
  a.partial = reinterpret_cast<float*>(static_cast<char*>(scratch) + sd::KV_TICKET_BYTES);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == SD_F32) sd::launch_kv_attention<float>(s, a, cache->d_head, cache->dtype == SD_E4M3, cache->n_seq, p);
  else sd::launch_kv_attention<sd::bf16>(s, a, cache->d_head, cache->dtype == SD_E4M3, cache->n_seq, p);
  return hipGetLastError() == hipSuccess ? SD_OK : kv_fail(SD_EHIP, "kernel launch");
}
