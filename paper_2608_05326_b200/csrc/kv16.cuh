// Shared pieces of the 16-bit paged cache: argument checks, the view as the kernels take it, sequence of a row.
#pragma once

#include "kv8.cuh"

namespace qevict {

struct Kv16View {
  int n_seqs, Hkv, D, block_log2, max_blocks, n_pages;
  void* pages[2];          // keys, values
  long long stride[2][3];  // elements: page, head, token
  const int32_t* table;    // [n_seqs][max_blocks]
  int32_t* status;         // or nullptr
};

// Strides that a vector of 16 bytes can follow; a dimension of one element has none that matters.
inline bool bad_stride(int64_t stride, long long extent) { return extent > 1 && (stride <= 0 || stride % 8 || stride >= (1ll << 38)); }

// nullptr if the view is usable, else the reason (and its status).
inline const char* kv16_check(const qevict_kv16_cache* c, qevict_status* st, Kv16View* v) {
  *st = QEVICT_ERR_INVALID_ARG;
  if (!c) return "cache is NULL";
  if (c->struct_size != sizeof(qevict_kv16_cache)) return "struct_size does not match this library's qevict_kv16_cache";
  if (c->device < 0) return "device must be >= 0";
  if (c->dtype != QEVICT_DTYPE_FP16 && c->dtype != QEVICT_DTYPE_BF16) return "dtype must be fp16 or bf16";
  if (c->reserved != 0) return "reserved must be 0";
  if (c->n_seqs < 0 || c->n_kv_heads < 1 || c->max_blocks < 1 || c->n_pages < 1)
    return "n_seqs must be >= 0, n_kv_heads, max_blocks and n_pages >= 1";
  *st = QEVICT_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128) return "block must be 16, 32, 64 or 128 tokens";
  if (c->n_kv_heads > 1024 || c->n_seqs > 65535) return "more than 1024 KV heads or 65535 sequences";
  if (c->n_pages > 0x7fffffff - 1) return "more than 2^31 - 2 pages";
  if ((long long)c->max_blocks * c->block > (1ll << 30)) return "max_blocks * block exceeds 2^30 tokens";
  *st = QEVICT_ERR_INVALID_ARG;
  if (!c->k_pages || !c->v_pages) return "pages must not be NULL";
  if (c->n_seqs > 0 && !c->block_table) return "block_table must not be NULL";
  if (misaligned16(c->k_pages) || misaligned16(c->v_pages)) return "pages must be 16-byte aligned";
  if (misaligned4(c->block_table) || misaligned4(c->status)) return "block_table and status must be 4-byte aligned";
  const long long extent[3] = {c->n_pages, c->n_kv_heads, c->block};
  for (int i = 0; i < 3; ++i)
    if (bad_stride(c->k_stride[i], extent[i]) || bad_stride(c->v_stride[i], extent[i]))
      return "strides of the pages must be positive multiples of 16 bytes";
  v->n_seqs = c->n_seqs; v->Hkv = c->n_kv_heads; v->D = c->head_dim;
  v->block_log2 = c->block == 16 ? 4 : c->block == 32 ? 5 : c->block == 64 ? 6 : 7;
  v->max_blocks = c->max_blocks; v->n_pages = c->n_pages;
  v->pages[0] = c->k_pages; v->pages[1] = c->v_pages;
  for (int i = 0; i < 3; ++i) { v->stride[0][i] = c->k_stride[i]; v->stride[1][i] = c->v_stride[i]; }
  v->table = c->block_table; v->status = c->status;
  return nullptr;
}

// The sequence whose rows hold `row`, for a whole warp: the last one that starts at or before it, 32 bounds at a look.  -1 if
// its bounds do not hold the row or reach outside the `total` rows.  Ascending bounds give every row its sequence; others may
// leave rows without one.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int n_seqs, long long row, long long total, int lane, int* first) {
  if (!cu) {
    *first = (int)row;
    return row < n_seqs ? (int)row : -1;
  }
  int lo = 0;
  for (int len = n_seqs; len > 0;) {
    const int step = (len + 31) >> 5, at = lane * step;
    const int c = __popc(__ballot_sync(0xffffffffu, at < len && cu[lo + at] <= row));
    if (c == 0) return -1;
    lo += (c - 1) * step;
    if (step == 1) break;
    len = min(step, len - (c - 1) * step);
  }
  if (n_seqs < 1) return -1;
  const int a = cu[lo], b = cu[lo + 1];
  *first = a;
  return a >= 0 && a <= row && row < b && b <= total ? lo : -1;
}

}  // namespace qevict
