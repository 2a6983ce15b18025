// Attention over whole prompts: checks of the arguments, key parts, launch (the kernels: prompt_attn.cuh).
#include "prompt_attn.cuh"

namespace qevict {

namespace {

const char* prompt_check(const qevict_prompt_args* p, qevict_status* st) {
  *st = QEVICT_ERR_INVALID_ARG;
  if (!p) return "args is NULL";
  if (p->struct_size != sizeof(qevict_prompt_args)) return "struct_size does not match this library's qevict_prompt_args";
  if (p->device < 0) return "device must be >= 0";
  if (p->dtype != QEVICT_DTYPE_FP16 && p->dtype != QEVICT_DTYPE_BF16) return "dtype must be fp16 or bf16";
  if (p->layout != QEVICT_LAYOUT_PACKED && p->layout != QEVICT_LAYOUT_PADDED) return "layout must be a QEVICT_LAYOUT_* value";
  if (p->causal != 0 && p->causal != 1) return "causal must be 0 or 1";
  if (p->n_seqs < 0 || p->max_q < 0 || p->max_k < 0 || p->total_q < 0 || p->total_k < 0) return "sizes must be >= 0";
  if (p->n_kv_heads < 1 || p->n_q_heads < 1 || p->n_q_heads % p->n_kv_heads) return "n_q_heads must be a multiple of n_kv_heads";
  if (!usable_scale(p->softmax_scale)) return "softmax_scale must be 0 or between 1e-30 and 2e38";
  *st = QEVICT_ERR_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return "head_dim must be 64 or 128";
  if (p->n_seqs > 65535 || p->n_q_heads > 1024) return "more than 65535 sequences or 1024 heads";
  if (p->total_q > 0x7fffffff - 1024 || p->total_k > 0x7fffffff - 1024 || p->max_q > 0x7fffffff - 1024 || p->max_k > 0x7fffffff - 1024)
    return "more than 2^31 - 1024 tokens";
  int P, T;
  prompt_tile(p->n_q_heads / p->n_kv_heads, &P, &T);
  if (prompt_tiles(p->layout == QEVICT_LAYOUT_PADDED, p->n_seqs, p->max_q, p->total_q, T) * (p->n_q_heads / P) > (1ll << 24))
    return "more than 2^24 query tiles in one call";
  *st = QEVICT_ERR_INVALID_ARG;
  if (p->n_seqs > 0 && p->layout == QEVICT_LAYOUT_PACKED && (!p->q_bounds || !p->k_bounds)) return "the packed layout needs q_bounds and k_bounds";
  return nullptr;
}

// The arguments with bounds that do not pass the rows there are: a packed sequence has no more than all of them, and the plan
// and the merge's grid (at most 2^29 CTAs with the limit on query tiles) go by the bounds.
qevict_prompt_args prompt_cut(const qevict_prompt_args& p) {
  qevict_prompt_args c = p;
  if (p.layout == QEVICT_LAYOUT_PACKED) {
    if (c.max_q > c.total_q) c.max_q = (int32_t)c.total_q;
    if (c.max_k > c.total_k) c.max_k = (int32_t)c.total_k;
  }
  return c;
}

const char* prompt_check_pointers(const qevict_prompt_args* p) {
  const bool keys = p->max_k > 0 && (p->layout == QEVICT_LAYOUT_PADDED || p->total_k > 0);
  if (!p->q || !p->out) return "q and out must not be NULL";
  if (keys && (!p->k || !p->v)) return "k and v must not be NULL";
  if (misaligned16(p->q) || misaligned16(p->out) || misaligned16(p->k) || misaligned16(p->v)) return "q, k, v and out must be 16-byte aligned";
  if (misaligned4(p->lse) || misaligned4(p->q_bounds) || misaligned4(p->k_bounds) || misaligned4(p->status))
    return "lse, bounds and status must be 4-byte aligned";
  // a dimension of one element has no stride that matters
  const bool padded = p->layout == QEVICT_LAYOUT_PADDED;
  auto bad = [&](const int64_t* s, int heads, long long tokens) {
    const long long size[3] = {padded ? p->n_seqs : 1, heads, tokens};
    for (int i = 0; i < 3; ++i)
      if (size[i] > 1 && (s[i] <= 0 || s[i] % 8 || s[i] >= (1ll << 38))) return true;
    return false;
  };
  const long long nq = padded ? p->max_q : p->total_q, nk = padded ? p->max_k : p->total_k;
  if (bad(p->q_stride, p->n_q_heads, nq) || bad(p->out_stride, p->n_q_heads, nq) || bad(p->k_stride, p->n_kv_heads, nk) ||
      bad(p->v_stride, p->n_kv_heads, nk))
    return "strides must be positive multiples of 16 bytes";
  return nullptr;
}

long long prompt_rows(const qevict_prompt_args* p) {
  return p->layout == QEVICT_LAYOUT_PADDED ? (long long)p->n_seqs * p->max_q : p->total_q;
}
// Work items that share a query tile's keys: the number that makes the call shortest by a model in key tiles (about 2 us).
// An item costs its key tiles and some three more; items go to the SMs as these fall free, so the call takes the work of all
// items over the SMs and about half an item for the uneven end, at least one item; and every part of the keys writes and reads
// its rows' results in float32 once more.  (28 heads, a piece of 500 tokens behind 16000 next to one of 166 behind 3714: 237,
// 174, 190, 157 us with one, two, three, five items for each tile; the model takes five, 152 to 169 us with the present merge.)
int prompt_splits(const qevict_prompt_args* p) {
  int P, T;
  prompt_tile(p->n_q_heads / p->n_kv_heads, &P, &T);
  const double tiles = (double)prompt_tiles(p->layout == QEVICT_LAYOUT_PADDED, p->n_seqs, p->max_q, p->total_q, T) * (p->n_q_heads / P);
  const double keys = (double)(((long long)p->max_k + TILE - 1) / TILE), sms = prompt_sms(p->device);
  const double merge = (double)prompt_rows(p) * p->n_q_heads * p->head_dim * 8.0 / 8e6 / 2.0;  // bytes at 8 MB a us: they stay in the L2
  int best = 1;
  double least = 0.0;
  for (int s = 1; s <= 64 && (s == 1 || keys / s >= 4.0); ++s) {
    const double item = keys / s + 3.0, spread = tiles * s * item / sms + item / 2;
    const double cost = (spread > item ? spread : item) + (s > 1 ? merge * s + 4.0 : 0.0);
    if (s == 1 || cost < least) {
      least = cost;
      best = s;
    }
  }
  return best;
}

size_t prompt_o_bytes(const qevict_prompt_args* p, int splits) {
  return ((size_t)splits * prompt_rows(p) * p->n_q_heads * p->head_dim * sizeof(float) + 255) & ~(size_t)255;
}
size_t prompt_bytes(const qevict_prompt_args* p, int splits) {
  return splits > 1 ? prompt_o_bytes(p, splits) + (size_t)splits * prompt_rows(p) * p->n_q_heads * sizeof(float) : 0;
}

template <class T, int D>
cudaError_t launch_prompt(const PromptArgs& a, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, int device, cudaStream_t s) {
  auto kernel = prompt_attn_kernel<T, D, false>;
  static std::atomic<uint64_t> done{0};
  cudaError_t e = once_per_device(done, device, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PromptSmem<D>::BYTES); });
  const long long tiles = prompt_tiles(a.padded, a.n_seqs, a.max_q, a.total_q, a.T);
  if (e == cudaSuccess)
    e = launch_pdl(kernel, dim3((unsigned)(tiles * (a.Hq / a.P) * a.splits)), dim3(PROMPT_THREADS), PromptSmem<D>::BYTES, s, a, mq, mk, mv);
  if (e == cudaSuccess && a.splits > 1) {
    const unsigned ctas = (unsigned)(((long long)a.max_q * a.Hq + 7) / 8);
    e = launch_pdl(prompt_merge_kernel<T, D>, dim3(ctas, a.n_seqs), dim3(256), 0, s, a);
  }
  return e;
}

}  // namespace

}  // namespace qevict

using namespace qevict;

extern "C" {

QEVICT_API qevict_status qevict_prompt_attn_scratch_bytes(const qevict_prompt_args* args, uint64_t* bytes) {
  qevict_status st;
  const char* why = prompt_check(args, &st);
  if (!why && !bytes) { why = "bytes is NULL"; st = QEVICT_ERR_INVALID_ARG; }
  if (why) return stateless_fail(st, why);
  const qevict_prompt_args cut = prompt_cut(*args);
  *bytes = prompt_bytes(&cut, prompt_splits(&cut));
  return QEVICT_OK;
}

QEVICT_API qevict_status qevict_prompt_attn(const qevict_prompt_args* given, void* scratch, uint64_t scratch_bytes, void* stream) {
  qevict_status st;
  const char* why = prompt_check(given, &st);
  if (why) return stateless_fail(st, why);
  const qevict_prompt_args cut = prompt_cut(*given), *args = &cut;
  const bool padded = args->layout == QEVICT_LAYOUT_PADDED;
  if (args->n_seqs == 0 || args->max_q == 0 || (!padded && args->total_q == 0)) return QEVICT_OK;
  why = prompt_check_pointers(args);
  if (why) return stateless_fail(QEVICT_ERR_INVALID_ARG, why);
  PromptArgs a = {};
  a.padded = padded; a.n_seqs = args->n_seqs; a.Hq = args->n_q_heads; a.Hkv = args->n_kv_heads; a.D = args->head_dim;
  a.max_q = args->max_q; a.max_k = args->max_k; a.causal = args->causal;
  prompt_tile(a.Hq / a.Hkv, &a.P, &a.T);
  a.splits = prompt_splits(args);
  const size_t need = prompt_bytes(args, a.splits);
  if (need > 0 && (!scratch || scratch_bytes < need))
    return stateless_fail(QEVICT_ERR_NO_MEMORY, "scratch too small: see qevict_prompt_attn_scratch_bytes");
  if (need > 0 && misaligned16(scratch)) return stateless_fail(QEVICT_ERR_INVALID_ARG, "scratch must be 16-byte aligned");
  a.total_q = args->total_q; a.total_k = args->total_k;
  a.scale_log2 = (float)((args->softmax_scale > 0.f ? (double)args->softmax_scale : 1.0 / sqrt((double)args->head_dim)) * 1.4426950408889634);
  a.out = args->out; a.lse = args->lse; a.q_bounds = args->q_bounds; a.k_bounds = args->k_bounds;
  for (int i = 0; i < 3; ++i) a.out_stride[i] = args->out_stride[i];
  a.rows = prompt_rows(args);
  a.part_o = static_cast<float*>(scratch);
  a.part_lse = reinterpret_cast<float*>(static_cast<char*>(scratch) + prompt_o_bytes(args, a.splits));
  a.status = args->status;
#ifdef QEVICT_DEBUG_BOUNDS
  a.give_up_warp = -1;
  a.give_up_at = 0;
  if (const char* e = getenv("QEVICT_CHECK_GIVE_UP")) sscanf(e, "%d:%d", &a.give_up_warp, &a.give_up_at);
#endif
  DeviceGuard guard(args->device);
  cudaError_t e = guard.err;
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  CUtensorMap mq, mk, mv;
  const long long nq = padded ? args->max_q : args->total_q, nk = padded ? args->max_k : args->total_k;
  const long long seqs = padded ? args->n_seqs : 1;
  if (!make_map(&mq, args->dtype, args->q, a.D, nq, a.Hq, seqs, args->q_stride, a.T, a.P) ||
      !make_map(&mk, args->dtype, args->k, a.D, args->max_k > 0 ? nk : 0, a.Hkv, seqs, args->k_stride, TILE, 1) ||
      !make_map(&mv, args->dtype, args->v, a.D, args->max_k > 0 ? nk : 0, a.Hkv, seqs, args->v_stride, TILE, 1))
    return stateless_fail(QEVICT_ERR_CUDA, "a tensor map could not be made for q, k or v");
  cudaStream_t s = (cudaStream_t)stream;
  if (args->dtype == QEVICT_DTYPE_FP16)
    e = a.D == 128 ? launch_prompt<__half, 128>(a, mq, mk, mv, args->device, s) : launch_prompt<__half, 64>(a, mq, mk, mv, args->device, s);
  else
    e = a.D == 128 ? launch_prompt<__nv_bfloat16, 128>(a, mq, mk, mv, args->device, s) : launch_prompt<__nv_bfloat16, 64>(a, mq, mk, mv, args->device, s);
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  return QEVICT_OK;
}

}  // extern "C"
