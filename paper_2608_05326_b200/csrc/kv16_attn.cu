// Attention of new tokens over the 16-bit paged cache: checks of the arguments, plan, launch.
//
// Up to 16 rows for a KV head (a token or a draft for the heads that share it): kv16_few.cuh.  More: the prompt attention's kernel
// (prompt_attn.cuh) with keys and values by page: a tile of 128 keys is 1 to 8 pages, each copied by TMA from where the
// table says, page after page into the rows that they have in the tile.
#include "kv16_few.cuh"

namespace qevict {

namespace {

constexpr int FEW_CLUSTER_KEYS = 1024;  // of a CTA
// Whole items: item_of adds up those of 32 sequences in 32 bits, each of which may have all rows of the call where bounds fall and rise.
constexpr long long MOST_ITEMS = 1ll << 24;

struct Plan {
  int P, T;       // rows of a query tile: heads, tokens
  bool few;       // few_attn_kernel has the call
  int ranks;      // with clusters of as many CTAs, else 0
  bool by_range;  // equal ranges, else whole items
  bool cuts;      // an item may be shared
  int slot_rows;
  unsigned ctas;
  size_t cut_bytes, o_bytes, bytes;
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

Plan with_scratch(Plan l, const qevict_kv16_attn_args* p, const Kv16View& c) {
  if (!l.cuts) return l;
  const size_t slots = 2 * (size_t)l.ctas * l.slot_rows;
  l.cut_bytes = ((size_t)l.ctas * sizeof(PagedCut) + 255) & ~(size_t)255;
  l.o_bytes = slots * c.D * sizeof(float);
  l.bytes = l.cut_bytes + l.o_bytes + slots * sizeof(float);
  return l;
}

template <class K> cudaError_t few_attributes(K kernel, int smem) {
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, 45);  // FEW_CTAS fit; the rest is L1
  return e;
}
template <class T, int D> cudaError_t few_cluster_attributes(int device) {
  static std::atomic<uint64_t> done{0};
  return once_per_device(done, device, [] {
    auto kernel = few_attn_kernel<T, D, true>;
    const cudaError_t e = few_attributes(kernel, few_smem(D));
    return e != cudaSuccess ? e : cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  });
}
void few_cluster_config(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* attr, int D, int ranks, dim3 grid, cudaStream_t s) {
  cfg->gridDim = grid;
  cfg->blockDim = dim3(32 * FEW_WARPS);
  cfg->dynamicSmemBytes = few_smem(D);
  cfg->stream = s;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ranks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg->attrs = attr;
  cfg->numAttrs = 2;
}

// The largest cluster that the device holds, asked once for the instance that takes most of it: 16 thread blocks on a whole one; a part
// of one may have fewer SMs side by side, and a launch of more is an error.
int few_most_ranks(int device) {
#ifdef QEVICT_DEBUG_BOUNDS
  if (const char* e = getenv("QEVICT_CHECK_CLUSTER")) return atoi(e);  // the checking build can be told of a smaller one
#endif
  static std::atomic<int> known[64];
  if (device >= 64) return 1;
  int most = known[device].load(std::memory_order_relaxed);
  if (most > 0) return most;
  DeviceGuard guard(device);
  if (guard.err != cudaSuccess || few_cluster_attributes<__nv_bfloat16, 128>(device) != cudaSuccess) {
    (void)cudaGetLastError();
    return 16;  // (no device: the size of the scratch is asked for elsewhere; the launch says so)
  }
  for (most = 16; most > 1; most /= 2) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    few_cluster_config(&cfg, attr, 128, most, dim3(most), nullptr);
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, few_attn_kernel<__nv_bfloat16, 128, true>, &cfg) == cudaSuccess && n > 0) break;
    (void)cudaGetLastError();
  }
  known[device].store(most, std::memory_order_relaxed);
  return most;
}

// Equal ranges of the work for all SMs; a call of many items (six for each SM, by its rows) hands out whole ones as SMs fall free,
// longest first: CTAs that work on one head then walk its keys together, and the L2 serves most of them.  Both sides, best graph replays,
// 32 / 8 heads of 128: 4 prompts of 2048 (7 items for each SM) whole 179 us, ranges 215; 8192 behind 57344 (7) 6.6 and 7.2 ms; 16384 alone
// (14) 1.83 and 1.99 ms; 4096 behind 57344 (3.5) 3.57 and 3.43 ms; 2048 (1.7) 1.75 and 1.63 ms.  The rows do not say how unlike the
// items are: a prompt of 8192 beside one token with 131072 takes 1.39 ms in whole items, 8 of which last beyond all others, 0.67 in ranges.
Plan attn_plan(const qevict_kv16_attn_args* p, const Kv16View& c) {
  Plan l = {};
  prompt_tile(p->n_q_heads / c.Hkv, &l.P, &l.T);
  long long longest = (long long)c.max_blocks << c.block_log2;
  if (p->max_len < longest) longest = p->max_len;
  const long long max_q = p->max_q < p->total_q ? p->max_q : p->total_q;
  const long long rows = p->cu_q ? p->total_q : (p->total_q < c.n_seqs ? p->total_q : c.n_seqs);
  const long long groups = p->n_q_heads / l.P, items = prompt_tiles(false, c.n_seqs, max_q, rows, l.T) * groups;
  const int sms = prompt_sms(p->cache->device), group = p->n_q_heads / c.Hkv;
  const long long units = c.n_seqs * (long long)c.Hkv, steps = (longest + FEW_KEYS - 1) / FEW_KEYS + FEW_ITEM_COST;
  if (group * max_q <= FEW_ROWS && units * steps < (1ll << 30)) {
    l.few = true;
    l.P = group;
    l.T = max_q > 0 ? (int)max_q : 1;
    // clusters as large as one wave holds, four steps of keys for each CTA at least
    const long long room = (long long)sms * FEW_CTAS;
    const int most_ranks = few_most_ranks(p->cache->device);
    int ranks = 1;
    while (ranks < most_ranks && units * ranks * 2 <= room && ranks * 2 * FEW_WARPS * FEW_KEYS <= longest) ranks *= 2;
    if (longest <= (long long)ranks * FEW_CLUSTER_KEYS && units * longest <= room * FEW_CLUSTER_KEYS) {
      l.ranks = ranks;
      return l;
    }
    const long long most = units * steps / FEW_RANGE_LEAST + 1;
    l.by_range = true;
    l.ctas = (unsigned)(most < room ? most : room);
    l.cuts = longest > FEW_KEYS && l.ctas > 1;
    l.slot_rows = FEW_SLOT_ROWS;
    return with_scratch(l, p, c);
  }
  l.by_range = rows / (2 * l.T) * groups < 6 * sms;
  if (!l.by_range) {
    l.ctas = items <= MOST_ITEMS ? (unsigned)items : 0u;
    return l;
  }
  const long long most = items * (KEY_COST * longest + ITEM_COST_PAIR) / RANGE_LEAST + 1;
  l.ctas = (unsigned)(most < sms ? most : sms);
  l.cuts = longest > TILE && l.ctas > 1;
  l.slot_rows = max_q <= l.T ? TILE : 2 * TILE;
  return with_scratch(l, p, c);
}

// A page's rows of a head by one copy of {64 channels, 8 tokens, d / 64 pieces, block / 8 groups}, which lands group by group with
// a group's pieces side by side; heads are reached in pieces too.  Where a head's stride is no number of pieces, by a
// copy for each 64 channels, which lands group by group.
bool whole_pages(const qevict_kv16_cache* c) {
  return c->n_kv_heads == 1 || (c->k_stride[1] % 64 == 0 && c->v_stride[1] % 64 == 0);
}
bool make_page_map(CUtensorMap* map, const qevict_kv16_cache* c, const void* base, const int64_t* stride, bool whole, int* head_step) {
  const cuuint64_t d = c->head_dim, heads = c->n_kv_heads;
  const int64_t head = heads > 1 ? stride[1] : (int64_t)d;
  *head_step = whole ? (int)(head / 64) : 1;
  if (head / 64 > 0x7fffffff / c->n_kv_heads) return false;
  const cuuint64_t dims[5] = {whole ? 64 : d, 8, whole ? (heads - 1) * (head / 64) + d / 64 : heads, (cuuint64_t)c->block / 8, (cuuint64_t)c->n_pages};
  const cuuint64_t st[4] = {(cuuint64_t)stride[2] * 2, (cuuint64_t)(whole ? 64 : head) * 2, (cuuint64_t)stride[2] * 16,
                            (cuuint64_t)(c->n_pages > 1 ? stride[0] : (int64_t)d) * 2};
  const cuuint32_t box[5] = {64, 8, whole ? (cuuint32_t)d / 64 : 1, (cuuint32_t)c->block / 8, 1}, el[5] = {1, 1, 1, 1, 1};
  EncodeFn fn = encode_fn();
  return fn && fn(map, c->dtype == QEVICT_DTYPE_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base),
                  dims, st, box, el, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

const char* attn_check_pointers(const qevict_kv16_attn_args* p) {
  if (!p->q || !p->out || !p->lens) return "q, out and lens must not be NULL";
  if (misaligned16(p->q) || misaligned16(p->out)) return "q and out must be 16-byte aligned";
  if (misaligned4(p->lse) || misaligned4(p->lens) || misaligned4(p->cu_q)) return "lse, lens and cu_q must be 4-byte aligned";
  if (bad_stride(p->q_stride[0], p->total_q) || bad_stride(p->q_stride[1], p->n_q_heads) || bad_stride(p->out_stride[0], p->total_q) ||
      bad_stride(p->out_stride[1], p->n_q_heads))
    return "strides must be positive multiples of 16 bytes";
  if (p->q == p->out && ((p->total_q > 1 && p->q_stride[0] != p->out_stride[0]) || (p->n_q_heads > 1 && p->q_stride[1] != p->out_stride[1])))
    return "an output in its input's place must have its strides";
  return nullptr;
}

template <class T, int D>
cudaError_t launch_few(const PromptArgs& a, const Plan& l, const FewPages& g, int device, cudaStream_t s) {
  if (!l.ranks) {
    auto kernel = few_attn_kernel<T, D, false>;
    static std::atomic<uint64_t> done{0};
    cudaError_t e = once_per_device(done, device, [&] { return few_attributes(kernel, few_smem(D)); });
    if (e == cudaSuccess) e = launch_pdl(kernel, dim3(l.ctas), dim3(32 * FEW_WARPS), few_smem(D), s, a, g);
    if (e == cudaSuccess && l.cuts) e = launch_pdl(paged_merge_kernel<T, D>, dim3(l.slot_rows / 32, l.ctas, D / 64), dim3(32 * MERGE_WARPS), 0, s, a);
    return e;
  }
  const cudaError_t e = few_cluster_attributes<T, D>(device);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  few_cluster_config(&cfg, attr, D, l.ranks, dim3(l.ranks * a.Hkv, a.n_seqs), s);
  return cudaLaunchKernelEx(&cfg, few_attn_kernel<T, D, true>, a, g);
}

template <class T, int D>
cudaError_t launch_paged(const PromptArgs& a, const Plan& l, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, int device, cudaStream_t s) {
  auto kernel = prompt_attn_kernel<T, D, true>;
  static std::atomic<uint64_t> done{0};
  cudaError_t e = once_per_device(done, device, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PromptSmem<D>::BYTES); });
  if (e == cudaSuccess) e = launch_pdl(kernel, dim3(l.ctas), dim3(PROMPT_THREADS), PromptSmem<D>::BYTES, s, a, mq, mk, mv);
  if (e == cudaSuccess && l.cuts) e = launch_pdl(paged_merge_kernel<T, D>, dim3(l.slot_rows / 32, l.ctas, D / 64), dim3(32 * MERGE_WARPS), 0, s, a);
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
  if (l.ctas == 0 && !l.few) return stateless_fail(QEVICT_ERR_UNSUPPORTED, "more than 2^24 work items in one call");
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
  a.P = l.P; a.T = l.T; a.splits = 1;
  a.groups = a.Hq / a.P; a.inv_step = 1.0 / (2 * a.T);
  a.total_q = p->cu_q ? p->total_q : view.n_seqs;
  a.scale_log2 = (float)((p->softmax_scale > 0.f ? (double)p->softmax_scale : 1.0 / sqrt((double)view.D)) * 1.4426950408889634);
  a.out = p->out; a.lse = p->lse; a.q_bounds = p->cu_q; a.k_bounds = p->lens;
  a.lse_rows = p->total_q;
  a.out_stride[1] = p->out_stride[1]; a.out_stride[2] = p->out_stride[0];
  if (l.cuts) {
    char* base = static_cast<char*>(scratch);
    a.cuts = reinterpret_cast<PagedCut*>(base);
    a.part_o = reinterpret_cast<float*>(base + l.cut_bytes);
    a.part_lse = reinterpret_cast<float*>(base + l.cut_bytes + l.o_bytes);
  }
  a.by_range = l.by_range; a.slot_rows = l.slot_rows;
  a.status = view.status;
  a.table = view.table; a.max_blocks = view.max_blocks; a.block_log2 = view.block_log2; a.n_pages = view.n_pages;
  const bool whole = whole_pages(c);
  a.boxes = whole ? 1 : a.D / 64;
  a.group_bytes = whole ? 16 * a.D : 1024;
  a.half_bytes = whole ? 1024 : TILE * 128;
#ifdef QEVICT_DEBUG_BOUNDS
  a.give_up_warp = -1;
  if (const char* e = getenv("QEVICT_CHECK_GIVE_UP")) sscanf(e, "%d:%d", &a.give_up_warp, &a.give_up_at);
#endif
  DeviceGuard guard(c->device);
  cudaError_t e = guard.err;
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  cudaStream_t s = (cudaStream_t)stream;
  if (l.few) {
    FewPages g = {};
    for (int w = 0; w < 2; ++w) {
      g.pages[w] = view.pages[w];
      for (int i = 0; i < 3; ++i) g.stride[w][i] = view.stride[w][i];
      g.q_stride[w] = p->q_stride[w];
    }
    g.q = p->q;
    if (c->dtype == QEVICT_DTYPE_FP16)
      e = a.D == 128 ? launch_few<__half, 128>(a, l, g, c->device, s) : launch_few<__half, 64>(a, l, g, c->device, s);
    else
      e = a.D == 128 ? launch_few<__nv_bfloat16, 128>(a, l, g, c->device, s) : launch_few<__nv_bfloat16, 64>(a, l, g, c->device, s);
    if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
    return QEVICT_OK;
  }
  CUtensorMap mq, mk, mv;
  const int64_t q_stride[3] = {0, p->q_stride[1], p->q_stride[0]};
  if (!make_map(&mq, c->dtype, p->q, a.D, p->total_q, a.Hq, 1, q_stride, a.T, a.P) ||
      !make_page_map(&mk, c, c->k_pages, c->k_stride, whole, &a.head_step[0]) ||
      !make_page_map(&mv, c, c->v_pages, c->v_stride, whole, &a.head_step[1]))
    return stateless_fail(QEVICT_ERR_CUDA, "a tensor map could not be made for q or the pages");
  if (c->dtype == QEVICT_DTYPE_FP16)
    e = a.D == 128 ? launch_paged<__half, 128>(a, l, mq, mk, mv, c->device, s) : launch_paged<__half, 64>(a, l, mq, mk, mv, c->device, s);
  else
    e = a.D == 128 ? launch_paged<__nv_bfloat16, 128>(a, l, mq, mk, mv, c->device, s) : launch_paged<__nv_bfloat16, 64>(a, l, mq, mk, mv, c->device, s);
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  return QEVICT_OK;
}

}  // extern "C"
