// Shared pieces of the 8-bit block-scaled cache: argument checks, code conversions.
#pragma once

#include <atomic>

#include "ctx.h"

namespace qevict {

// The view as the kernels take it.
struct Kv8View {
  int n_seqs, Hkv, D, block, max_blocks, n_pages;
  uint8_t* codes[2];   // keys, values: [n_pages][Hkv][block][D]
  float* scale[2];     // [n_pages][Hkv]
  void* tail[2];       // [n_seqs][Hkv][block][D]
  const int32_t* table;  // [n_seqs][max_blocks]
  int32_t* status;     // or nullptr
};

__device__ __forceinline__ void kv8_record(int32_t* status, int code) {
  if (status) record_check(status, code);
}

// Packed pairs of float32: one instruction for two fused multiply-adds or additions.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;\n" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Runs `set` (function attributes of a kernel) once for each device; `done` has a bit per device and is the kernel's own.
template <class F> inline cudaError_t once_per_device(std::atomic<uint64_t>& done, int device, F set) {
  const uint64_t bit = device < 64 ? 1ull << device : 0ull;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  const cudaError_t e = set();
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

// 0, or a scale that is a float32 times log2 e too and leaves logits their bits.
inline bool usable_scale(float s) { return s == 0.f || (s >= 1e-30f && s <= 2e38f); }

inline bool misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

// nullptr if the view is usable, else the reason (and its status).
inline const char* kv8_check(const qevict_kv8_cache* c, qevict_status* st, Kv8View* v) {
  *st = QEVICT_ERR_INVALID_ARG;
  if (!c) return "cache is NULL";
  if (c->struct_size != sizeof(qevict_kv8_cache)) return "struct_size does not match this library's qevict_kv8_cache";
  if (c->device < 0) return "device must be >= 0";
  if (c->dtype != QEVICT_DTYPE_FP16 && c->dtype != QEVICT_DTYPE_BF16) return "dtype must be fp16 or bf16";
  if (c->code != QEVICT_CODE_INT8 && c->code != QEVICT_CODE_E4M3) return "code must be a QEVICT_CODE_* value";
  if (c->n_seqs < 0 || c->n_kv_heads < 1 || c->max_blocks < 1 || c->n_pages < 0)
    return "n_seqs and n_pages must be >= 0, n_kv_heads and max_blocks >= 1";
  *st = QEVICT_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128) return "block must be 16, 32, 64 or 128 tokens";
  if (c->n_kv_heads > 1024 || c->n_seqs > 8192) return "more than 1024 KV heads or 8192 sequences";
  if ((long long)c->n_pages * c->n_kv_heads > 0x7fffffffll) return "n_pages * n_kv_heads exceeds 2^31 - 1";
  if ((long long)c->max_blocks * c->block > (1ll << 30)) return "max_blocks * block exceeds 2^30 tokens";
  *st = QEVICT_ERR_INVALID_ARG;
  if (c->n_pages > 0 && (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale)) return "code pools and scales must not be NULL";
  if (c->n_seqs > 0 && (!c->k_tail || !c->v_tail || !c->block_table)) return "tails and block_table must not be NULL";
  if (misaligned16(c->k_codes) || misaligned16(c->v_codes) || misaligned16(c->k_tail) || misaligned16(c->v_tail))
    return "code pools and tails must be 16-byte aligned";
  if (misaligned4(c->k_scale) || misaligned4(c->v_scale) || misaligned4(c->block_table) || misaligned4(c->status))
    return "scales, block_table and status must be 4-byte aligned";
  v->n_seqs = c->n_seqs; v->Hkv = c->n_kv_heads; v->D = c->head_dim; v->block = c->block;
  v->max_blocks = c->max_blocks; v->n_pages = c->n_pages;
  v->codes[0] = (uint8_t*)c->k_codes; v->codes[1] = (uint8_t*)c->v_codes;
  v->scale[0] = c->k_scale; v->scale[1] = c->v_scale;
  v->tail[0] = c->k_tail; v->tail[1] = c->v_tail;
  v->table = c->block_table; v->status = c->status;
  return nullptr;
}

}  // namespace qevict
