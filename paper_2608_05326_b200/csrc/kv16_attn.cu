// Attention of new tokens over the 16-bit paged cache: checks of the arguments, plan, launch.
//
// The kernel is the prompt attention's (prompt_attn.cuh) with keys and values by page: a tile of 128 keys is 1 to 8
// pages, each copied by TMA from where the table says, page after page into the rows that they have in the tile.
#include "prompt_attn.cuh"

namespace qevict {

namespace {

struct Plan {
  int P, T;           // rows of a query tile: heads, tokens
  int per_part;       // key tiles of a part
  int pieces;         // parts of the longest sequence
  bool pairs;         // whether there can be sequences with few queries and more than one key tile
  bool compact;
  long long pair_rows, rows;  // of the partial results
  long long positions;        // of the grid
  size_t o_bytes, bytes;
};

const char* attn_check(const qevict_kv16_attn_args* p, Kv16View* view, qevict_status* st) {
  *st = QEVICT_ERR_INVALID_ARG;
  if (!p) return "args is NULL";
  if (p->struct_size != sizeof(qevict_kv16_attn_args)) return "struct_size does not match this library's qevict_kv16_attn_args";
  if (const char* why = kv16_check(p->cache, st, view)) return why;
  *st = QEVICT_ERR_INVALID_ARG;
  if (p->causal != 0 && p->causal != 1) return "causal must be 0 or 1";
  if (p->max_q < 0 || p->max_len < 0 || p->total_q < 0) return "sizes must be >= 0";
  if (p->n_q_heads < 1 || p->n_q_heads % view->Hkv) return "n_q_heads must be a multiple of n_kv_heads";
  if (!usable_scale(p->softmax_scale)) return "softmax_scale must be 0 or between 1e-30 and 2e38";
  if (!p->cu_q && p->max_q > 1) return "without cu_q every sequence has one token: max_q must be 0 or 1";
  if (!p->cu_q && p->max_q == 1 && p->total_q < view->n_seqs) return "without cu_q total_q must be at least n_seqs";
  *st = QEVICT_ERR_UNSUPPORTED;
  if (p->n_q_heads > 1024) return "more than 1024 heads";
  if (p->total_q > 0x7fffffff - 1024 || p->max_q > 0x7fffffff - 1024) return "more than 2^31 - 1024 tokens";
  return nullptr;
}

// Parts of the keys: the number that makes the call shortest by a model in steps (two tiles' products, about 2 us).  An item
// costs its steps and some three more; items go to the SMs as these fall free, so the call takes the work of all items over the
// SMs and about half an item for the uneven end, at least one item; and every part of the keys writes and reads its rows'
// results in float32 once more.
Plan attn_plan(const qevict_kv16_attn_args* p, const Kv16View& c) {
  Plan l = {};
  prompt_tile(p->n_q_heads / c.Hkv, &l.P, &l.T);
  long long longest = (long long)c.max_blocks << c.block_log2;
  if (p->max_len < longest) longest = p->max_len;
  const long long max_q = p->max_q < p->total_q ? p->max_q : p->total_q;
  const long long rows = p->cu_q ? p->total_q : (p->total_q < c.n_seqs ? p->total_q : c.n_seqs);
  const long long keys = (longest + TILE - 1) / TILE, groups = p->n_q_heads / l.P;
  const long long tiles = prompt_tiles(false, c.n_seqs, max_q, rows, l.T) * groups;
  const bool few = max_q <= l.T;  // every sequence has one tile of rows: a step takes two key tiles
  l.pairs = keys > 1;
  const double steps = few ? (keys + 1) / 2 : keys, sms = prompt_sms(p->cache->device);
  const double merge = (double)rows * p->n_q_heads * c.D * 8.0 / 8e6 / 2.0;
  double least = 0.0;
  long long best = 1;
  for (int s = 1; s <= 32 && (s == 1 || steps / s >= (few ? 1.0 : 4.0)); ++s) {
    const double item = steps / s + 3.0, spread = tiles * s * item / sms + item / 2;
    const double cost = (spread > item ? spread : item) + (s > 1 ? merge * s + 4.0 : 0.0);
    if (s == 1 || cost < least) {
      least = cost;
      best = s;
    }
  }
  l.per_part = (int)(keys > 0 ? (keys + best - 1) / best : 1);
  l.pieces = (int)(keys > 0 ? (keys + l.per_part - 1) / l.per_part : 1);
  l.rows = l.pieces > 1 && !few ? rows : 0;
  l.compact = (long long)c.n_seqs * l.T < rows;
  l.pair_rows = !l.pairs ? 0 : l.compact ? (long long)c.n_seqs * l.T : rows;
  l.positions = tiles * l.pieces;
  const long long partial = 2 * l.pieces * l.pair_rows + l.pieces * l.rows;
  l.o_bytes = ((size_t)partial * p->n_q_heads * c.D * sizeof(float) + 255) & ~(size_t)255;
  l.bytes = partial ? l.o_bytes + (size_t)partial * p->n_q_heads * sizeof(float) : 0;
  return l;
}

const char* attn_check_pointers(const qevict_kv16_attn_args* p) {
  if (!p->q || !p->out || !p->lens) return "q, out and lens must not be NULL";
  if (misaligned16(p->q) || misaligned16(p->out)) return "q and out must be 16-byte aligned";
  if (misaligned4(p->lse) || misaligned4(p->lens) || misaligned4(p->cu_q)) return "lse, lens and cu_q must be 4-byte aligned";
  if (bad_stride(p->q_stride[0], p->total_q) || bad_stride(p->q_stride[1], p->n_q_heads) || bad_stride(p->out_stride[0], p->total_q) ||
      bad_stride(p->out_stride[1], p->n_q_heads))
    return "strides must be positive multiples of 16 bytes";
  return nullptr;
}

template <class T, int D>
cudaError_t launch_paged(const PromptArgs& a, const Plan& l, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, int device, cudaStream_t s) {
  auto kernel = prompt_attn_kernel<T, D, true>;
  static std::atomic<uint64_t> done{0};
  cudaError_t e = once_per_device(done, device, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PromptSmem<D>::BYTES); });
  if (e == cudaSuccess) e = launch_pdl(kernel, dim3((unsigned)l.positions), dim3(PROMPT_THREADS), PromptSmem<D>::BYTES, s, a, mq, mk, mv);
  if (e == cudaSuccess && l.bytes > 0) {
    // pairs alone: their rows, sequence by sequence; else all rows
    const bool by_seq = l.rows == 0 && l.compact;
    const long long rows = by_seq ? l.T : a.total_q;
    e = launch_pdl(prompt_merge_kernel<T, D, true>, dim3((unsigned)((rows * a.Hq + 7) / 8), by_seq ? a.n_seqs : 1), dim3(256), 0, s, a, by_seq);
  }
  return e;
}

}  // namespace

}  // namespace qevict

using namespace qevict;

extern "C" {

QEVICT_API qevict_status qevict_kv16_attn_scratch_bytes(const qevict_kv16_attn_args* p, uint64_t* bytes) {
  qevict_status st;
  Kv16View view;
  const char* why = attn_check(p, &view, &st);
  if (!why && !bytes) { why = "bytes is NULL"; st = QEVICT_ERR_INVALID_ARG; }
  if (why) return stateless_fail(st, why);
  *bytes = view.n_seqs > 0 ? attn_plan(p, view).bytes : 0;
  return QEVICT_OK;
}

QEVICT_API qevict_status qevict_kv16_attn(const qevict_kv16_attn_args* p, void* scratch, uint64_t scratch_bytes, void* stream) {
  qevict_status st;
  Kv16View view;
  const char* why = attn_check(p, &view, &st);
  if (why) return stateless_fail(st, why);
  if (view.n_seqs == 0 || p->max_q == 0 || p->total_q == 0) return QEVICT_OK;
  why = attn_check_pointers(p);
  if (why) return stateless_fail(QEVICT_ERR_INVALID_ARG, why);
  const Plan l = attn_plan(p, view);
  if (l.positions > (1ll << 28)) return stateless_fail(QEVICT_ERR_UNSUPPORTED, "more than 2^28 work items in one call");
  if (l.bytes > 0 && (!scratch || scratch_bytes < l.bytes))
    return stateless_fail(QEVICT_ERR_NO_MEMORY, "scratch too small: see qevict_kv16_attn_scratch_bytes");
  if (l.bytes > 0 && misaligned16(scratch)) return stateless_fail(QEVICT_ERR_INVALID_ARG, "scratch must be 16-byte aligned");
  const qevict_kv16_cache* c = p->cache;
  PromptArgs a = {};
  const long long capacity = (long long)view.max_blocks << view.block_log2;
  a.n_seqs = view.n_seqs; a.Hq = p->n_q_heads; a.Hkv = view.Hkv; a.D = view.D;
  a.max_q = (int)(p->max_q < p->total_q ? p->max_q : p->total_q);
  a.max_k = (int)(p->max_len < capacity ? p->max_len : capacity);
  a.causal = p->causal;
  a.P = l.P; a.T = l.T; a.splits = l.pieces;
  a.total_q = p->cu_q ? p->total_q : view.n_seqs;
  a.scale_log2 = (float)((p->softmax_scale > 0.f ? (double)p->softmax_scale : 1.0 / sqrt((double)view.D)) * 1.4426950408889634);
  a.out = p->out; a.lse = p->lse; a.q_bounds = p->cu_q; a.k_bounds = p->lens;
  a.lse_rows = p->total_q;
  a.out_stride[1] = p->out_stride[1]; a.out_stride[2] = p->out_stride[0];
  a.part_o = static_cast<float*>(scratch);
  a.part_lse = reinterpret_cast<float*>(static_cast<char*>(scratch) + l.o_bytes);
  a.rows = l.rows; a.pair_rows = l.pair_rows; a.compact = l.compact;
  a.status = view.status;
  a.table = view.table; a.max_blocks = view.max_blocks; a.block_log2 = view.block_log2; a.n_pages = view.n_pages;
  a.per_part = l.per_part;
#ifdef QEVICT_DEBUG_BOUNDS
  a.give_up_warp = -1;
  if (const char* e = getenv("QEVICT_CHECK_GIVE_UP")) sscanf(e, "%d:%d", &a.give_up_warp, &a.give_up_at);
#endif
  DeviceGuard guard(c->device);
  cudaError_t e = guard.err;
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  CUtensorMap mq, mk, mv;
  const int64_t q_stride[3] = {0, p->q_stride[1], p->q_stride[0]};
  if (!make_map(&mq, c->dtype, p->q, a.D, p->total_q, a.Hq, 1, q_stride, a.T, a.P) ||
      !make_map(&mk, c->dtype, c->k_pages, a.D, c->block, a.Hkv, c->n_pages, c->k_stride, c->block, 1) ||
      !make_map(&mv, c->dtype, c->v_pages, a.D, c->block, a.Hkv, c->n_pages, c->v_stride, c->block, 1))
    return stateless_fail(QEVICT_ERR_CUDA, "a tensor map could not be made for q or the pages");
  cudaStream_t s = (cudaStream_t)stream;
  if (c->dtype == QEVICT_DTYPE_FP16)
    e = a.D == 128 ? launch_paged<__half, 128>(a, l, mq, mk, mv, c->device, s) : launch_paged<__half, 64>(a, l, mq, mk, mv, c->device, s);
  else
    e = a.D == 128 ? launch_paged<__nv_bfloat16, 128>(a, l, mq, mk, mv, c->device, s) : launch_paged<__nv_bfloat16, 64>(a, l, mq, mk, mv, c->device, s);
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  return QEVICT_OK;
}

}  // extern "C"
