// Attention over whole prompts on the 5th-generation tensor cores.
//
//     S = Q K^T,  P = 2^(S * scale * log2 e - m),  O += P V,  out = O / sum P,  lse = ln sum exp(scale * S)
//
// A work item is two tiles of 128 query rows (the heads that share a KV head, some tokens of each: see prompt_tile) against
// the keys in tiles of 128, last tile first.  A CTA
// stays on its SM and takes over grid positions that have not started (the hardware hands them out), so that one item's
// start and results run beside another's products.  Twenty warps: eight for each query tile's softmax (two threads to a
// row), one that issues the products, one that issues the copies, one that fetches work items.
//   - Q, K, V tiles come by TMA (boxes of 64 channels x 128 tokens, 128-byte swizzle); K and V share a ring.
//   - S (128 x 128 fp32) and O (128 x d fp32) of both tiles fill the 512 columns of tensor memory.  P goes back over S
//     in 16 bits and is the A operand of the second product from there.
//   - While one tile's warps are in their softmax, the tensor cores work on the other tile's products.
//   - The reference exponent m of a row moves only when a logit exceeds it by 2^8 (then O is rescaled in tensor
//     memory); P is at most 2^8, sums are float32.
// What bounds it: at d = 128 a key tile costs both query tiles 2048 tensor-core cycles at best; with both operands of S in
// shared memory the products alone take about 2750 (8 KB of operands for 64 cycles of products, at 128 bytes a cycle, and
// the copies write through the same port), and a step takes about 3600 with the softmax behind it.  Measured, call after
// call: causal 32768 tokens x 32 heads 7.97 ms (1103 TFLOP/s, 0.78 of the measured sustained rate; the power limit holds it there:
// single calls of a cool card take 6.9 to 7.4 ms); 12 packed prompts of up to 4001 tokens 594 us (849 TFLOP/s), the best of graph
// replays 497 to 512 us; d = 64: 16384 tokens x 32 heads 1.57 ms (702 TFLOP/s: half the products for the same exponentials).
// Shares of the
// exponentials as polynomials on the FMA units were slower at every share (1/2 to 1/16): what the softmax waits for is
// issue and hand-over, not the exponential unit.
//
// Few query rows (one token, a short piece behind a long prefix): the keys are split over several CTAs whose partial
// outputs prompt_merge_kernel joins.
//
// Keys past the sequence's end are masked by selection, so what lies there (another sequence, padding, NaN) never
// enters; value rows past the end are zeroed in shared memory before the product reads them, since 0 * NaN is NaN.
// Every wait is bounded; one that runs out records CHECK_COPY_TIMEOUT and the CTA leaves after its copies have landed and its
// unfinished rows have become not-a-number.
#include <cuda.h>
#ifdef QEVICT_DEBUG_BOUNDS
#include <stdio.h>
#include <stdlib.h>
#endif

#include "kv8.cuh"

namespace qevict {

namespace {

constexpr int PROMPT_THREADS = 640;  // four softmax warpgroups, one for products, copies and work items (a warp idle)
constexpr int MMA_WARP = 16, LOAD_WARP = 17, ITEM_WARP = 18;
constexpr int TILE = 128;           // query rows of a tile, keys of a tile
constexpr float PROMPT_LAZY = 8.f;  // log2

struct PromptArgs {
  int padded, n_seqs, Hq, Hkv, D, max_q, max_k, causal, splits;
  int P, T;  // a tile's rows: P query heads of one KV head, T tokens each
  long long total_q, total_k;
  float scale_log2;
  void* out;
  float* lse;
  const int32_t* q_bounds;
  const int32_t* k_bounds;
  long long out_stride[3];
  float* part_o;    // [split][row][Hq][D]
  float* part_lse;  // [split][row][Hq] (log2)
  long long rows;   // rows of the partial results
  int32_t* status;
#ifdef QEVICT_DEBUG_BOUNDS
  int give_up_warp, give_up_at;  // in every CTA this warp gives up at this wait of its (QEVICT_CHECK_GIVE_UP=warp:wait)
#endif
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ float ex2p(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}\n" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Looks at a barrier until its phase is over, a number of times (a look that finds nothing takes about 1.5 us: the hardware waits).
// ITEM: what is waited for may take as long as a whole work item; such a wait also ends when another of the CTA has given up
// (*failed).  (A look at that word in the short waits too: 1 % slower.)
#ifdef QEVICT_DEBUG_BOUNDS
constexpr uint32_t LOOKS = 1u << 14, LOOKS_ITEM = 1u << 20;  // 25 ms, 1.6 s: the checking build has waits give up on purpose
#else
constexpr uint32_t LOOKS = 1u << 20, LOOKS_ITEM = 1u << 26;
#endif
template <bool ITEM = false> __device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, const volatile uint32_t* failed = nullptr) {
  for (uint32_t it = 0; it < (ITEM ? LOOKS_ITEM : LOOKS); ++it) {
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}\n"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    if (done) return true;
    if (ITEM && *failed) return false;
  }
  return false;
}
__device__ __forceinline__ bool bar_peek(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}\n"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
// the same for a whole warp, with one answer; says so where it gives up
template <bool ITEM> __device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t* failed) {
  const bool yes = __all_sync(0xffffffffu, bar_wait<ITEM>(bar, parity, failed));
  if (!yes) *failed = 1;
  return yes;
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int tok, int head, int seq) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(tok), "r"(head), "r"(seq) : "memory");
}
__device__ __forceinline__ void commit_to(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Descriptor of a shared-memory operand with the 128-byte swizzle: the low word holds the address and the leading byte
// offset, the high word (constant) the stride of 1024 bytes between groups of eight rows, version 1 and the swizzle.
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo) { return ((addr >> 4) & 0x3FFFu) | ((lbo >> 4) << 16); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}\n" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(acc), "r"(DESC_HI)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 db, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}\n" ::"r"(d), "r"(a), "r"(b_lo), "r"(idesc), "r"(acc), "r"(DESC_HI)
      : "memory");
}
__device__ __forceinline__ void tm_ld32(uint32_t addr, float* v) {
  uint32_t* u = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
      "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
        "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]),
        "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]),
        "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_ld8(uint32_t addr, float* v) {
  uint32_t* u = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_st8(uint32_t addr, const uint32_t* u) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};\n" ::"r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]),
               "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_ld16(uint32_t addr, float* v) {
  uint32_t* u = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
        "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

template <class T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) { return as_u32(__floats2half2_rn(a, b)); }
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) { return as_u32(__floats2bfloat162_rn(a, b)); }

// Rows of a sequence: first row, count, sequence coordinate of the tensor map.
__device__ __forceinline__ void span_of(const int32_t* bounds, int padded, int s, int most, long long total, int* first, int* n) {
  if (padded) {
    *first = 0;
    *n = bounds ? max(0, min(bounds[s], most)) : most;
  } else {
    const long long b0 = max(0ll, min((long long)bounds[s], total)), b1 = max(b0, min((long long)bounds[s + 1], total));
    *first = (int)b0;
    *n = (int)min(b1 - b0, (long long)most);
  }
}

// Whether span_of has to cut sequence s: outside the rows there are, longer than the bound, falling.
__device__ __forceinline__ bool span_cut(const int32_t* bounds, int padded, int s, int most, long long total) {
  if (padded) return bounds && (bounds[s] < 0 || bounds[s] > most);
  const long long b0 = bounds[s], b1 = bounds[s + 1];
  return b0 < 0 || b1 < b0 || b1 > total || b1 - b0 > most;
}

// Column of the 16 keys `k` (0 .. 3) of half `half` of a tile's P, over the S of the same half: the thread that writes it
// has read what it overwrites.
__device__ __forceinline__ constexpr int P_COL(int half, int k) { return half * 64 + k * 8; }

template <int D> struct PromptSmem {
  static constexpr int STAGES = D == 128 ? 5 : 8;
  static constexpr int HALF = TILE * 128;             // 64 channels of 128 rows
  static constexpr int TILE_BYTES = HALF * (D / 64);
  static constexpr int Q_OFF = 0, KV_OFF = 2 * TILE_BYTES, BAR_OFF = KV_OFF + STAGES * TILE_BYTES;
  static constexpr int WORDS = 256, ITEMS = 320, ROWS = 544;  // behind the barriers: words, work items, row maxima
  static constexpr int BYTES = BAR_OFF + ROWS + 2048;
};

// A work item: two tiles of T tokens of P heads of one sequence, or a part of their keys.
struct PromptItem {
  int valid, h0, s, split, r0, q0, nq, k0, nk;  // h0: first query head, r0: first token
  int lo, n;       // key tiles of this item
  int nt0, nt1;    // end of the two query tiles' key tiles
  __device__ __forceinline__ int cnt(int w) const { return max(0, (w ? nt1 : nt0) - lo); }
  __device__ __forceinline__ bool dirty() const { return n > lo && n * TILE > nk; }  // the first tile reaches past the sequence
};

// The item of grid position x, for a whole warp; not valid where x lies past the last sequence's.  Positions go by the
// sequences' own lengths, so a batch of very different lengths has next to no empty positions, and by falling cost, so that the
// SMs end together: sequences in groups of 32; in a group the tiles by falling number of keys, level by level (a level: the rows
// of one tile more or less; a sequence's tiles have one each, from its prefix on); on a level the sequences that have it; then
// the heads, then the parts of the keys.  *at, *before: where the last search ended (first sequence of the group, items before
// it), which is where the next one starts; positions mostly grow, but nothing promises it: a smaller one starts at the front.
__device__ __forceinline__ PromptItem item_of(const PromptArgs& a, int x, int lane, int* at, int* before) {
  PromptItem it;
  const int t = x / a.splits, step = 2 * a.T, groups = a.Hq / a.P;
  it.split = x - t * a.splits;
  it.h0 = 0;
  it.valid = 0;
  it.s = 0;
  int mt = 0;
  if (t < *before) {
    *at = 0;
    *before = 0;
  }
  for (; *at < a.n_seqs; *at += 32) {
    const int s = *at + lane;
    int first, n = 0, keys = 0;
    if (s < a.n_seqs) {
      span_of(a.q_bounds, a.padded, s, a.max_q, a.total_q, &first, &n);
      span_of(a.k_bounds, a.padded, s, a.max_k, a.total_k, &first, &keys);
    }
    const int tiles = (n + step - 1) / step, base = (keys - n) / step, top = base + tiles;  // its levels: base .. top - 1
    const int all = __reduce_add_sync(0xffffffffu, tiles) * groups, in = t - *before;
    if (in < all) {
      // the level: the largest L with more than `in` items on the levels from L on
      auto from = [&](int level) { return __reduce_add_sync(0xffffffffu, min(tiles, max(0, top - level))) * groups; };
      int lo = __reduce_min_sync(0xffffffffu, tiles ? base : 0x7fffffff), hi = __reduce_max_sync(0xffffffffu, tiles ? top - 1 : -0x7fffffff);
      while (lo < hi) {
        const int mid = lo + ((hi - lo + 1) >> 1);
        if (from(mid) > in) lo = mid; else hi = mid - 1;
      }
      const int k = in - from(lo + 1), nth = k / groups;
      uint32_t have = __ballot_sync(0xffffffffu, tiles > 0 && base <= lo && lo < top);
      for (int i = 0; i < nth; ++i) have &= have - 1;
      const int who = __ffs(have) - 1;
      it.valid = 1;
      it.s = *at + who;
      it.h0 = (k - nth * groups) * a.P;
      mt = lo - __shfl_sync(0xffffffffu, base, who);
      break;
    }
    *before += all;
  }
  it.r0 = mt * step;
  if (!it.valid) return it;
  span_of(a.q_bounds, a.padded, it.s, a.max_q, a.total_q, &it.q0, &it.nq);
  span_of(a.k_bounds, a.padded, it.s, a.max_k, a.total_k, &it.k0, &it.nk);
  int nt[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int rw = it.r0 + w * a.T, last = min(rw + a.T, it.nq) - 1;
    const int lim = rw >= it.nq ? 0 : (a.causal ? min(it.nk, last + it.nk - it.nq + 1) : it.nk);
    nt[w] = lim > 0 ? (lim + TILE - 1) / TILE : 0;
  }
  it.lo = 0;
  it.n = max(nt[0], nt[1]);
  if (a.splits > 1) {
    const int per = (it.n + a.splits - 1) / a.splits;
    it.lo = min(it.n, it.split * per);
    it.n = min(it.n, it.lo + per);
  }
  it.nt0 = min(nt[0], it.n);
  it.nt1 = min(nt[1], it.n);
  return it;
}

template <class T, int D>
__global__ void __launch_bounds__(PROMPT_THREADS, 1)
    prompt_attn_kernel(const PromptArgs a, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                       const __grid_constant__ CUtensorMap mv) {
  using SM = PromptSmem<D>;
  constexpr int NS = SM::STAGES;
  extern __shared__ __align__(1024) unsigned char sm[];  // the swizzle counts from multiples of 1024 bytes
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const uint32_t smb = smem_u32(sm), bars = smb + SM::BAR_OFF;
  // barriers: Q full / empty; ring full / empty; S ready, P ready, O ready of both tiles; value tail zeroed; work items
  // full / empty (two places); answer to the request for the next one; products done after a failure
  const uint32_t b_q = bars, b_full = bars + 8, b_empty = b_full + 8 * NS, b_s = b_empty + 8 * NS, b_p = b_s + 16, b_o = b_p + 16,
                 b_clean = b_o + 16, b_qe = b_clean + 8, b_item = b_qe + 8, b_taken = b_item + 16, b_next = b_taken + 16,
                 b_done = b_next + 8;
  // words: 0 .. 3 the answer; 4 tensor memory; 5 loads of K and V issued; 6 a wait has given up; 7 loads of Q; 8 requests for items
  volatile uint32_t* words = reinterpret_cast<volatile uint32_t*>(sm + SM::BAR_OFF + SM::WORDS);
  PromptItem* items = reinterpret_cast<PromptItem*>(sm + SM::BAR_OFF + SM::ITEMS);
  static_assert(SM::ITEMS + sizeof(PromptItem) * 4 <= SM::ROWS, "two work items, and two that could not be handed out");
  if (smb & 1023u) {  // no tile would be where the products look for it
    kv8_record(a.status, CHECK_ALIGNMENT);
    return;
  }
  if (wid == MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((void*)(words + 4))), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 0) {
    bar_init(b_q, 1);
    bar_init(b_qe, 1);
    for (int i = 0; i < NS; ++i) { bar_init(b_full + 8 * i, 1); bar_init(b_empty + 8 * i, 1); }
    for (int w = 0; w < 2; ++w) {
      bar_init(b_s + 8 * w, 1);
      bar_init(b_p + 8 * w, 8);
      bar_init(b_o + 8 * w, 1);
      bar_init(b_item + 8 * w, 1);
      bar_init(b_taken + 8 * w, 18);
    }
    bar_init(b_clean, 1);
    bar_init(b_next, 1);
    bar_init(b_done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    for (int i = 5; i < 9; ++i) words[i] = 0;
    for (int i = 0; i < 4; ++i) items[i].valid = 0;
  }
  tm_before();
  __syncthreads();
  tm_after();
  const uint32_t tmem = words[4];
  pdl_prologue();
  bool ok = true, leader = false;  // leader: the lane that issues the products
#ifdef QEVICT_DEBUG_BOUNDS
  int waits = 0;
  auto gives_up = [&] {
    if (a.give_up_warp != wid || ++waits != a.give_up_at) return false;
    words[6] = 1;
    return true;
  };
#else
  auto gives_up = [] { return false; };
#endif
  auto wait = [&](uint32_t bar, uint32_t parity) { return !gives_up() && warp_wait<false>(bar, parity, words + 6); };
  auto wait_item = [&](uint32_t bar, uint32_t parity) { return !gives_up() && warp_wait<true>(bar, parity, words + 6); };

  // The next item, in the place that the item warp fills; the one before is given back.  No item on failure.
  int taken = 0;
  auto next_item = [&]() -> const PromptItem* {
    if (taken > 0) {
      __syncwarp();
      if (lane == 0) bar_arrive(b_taken + 8 * ((taken - 1) & 1));
    }
    const int place = taken & 1;
    ok = ok && wait(b_item + 8 * place, (uint32_t)(taken >> 1) & 1u);
    ++taken;
    return ok && items[place].valid ? &items[place] : nullptr;
  };

  // registers: 640 x 96 at launch = 512 x 112 + 128 x 32
  if (wid >= MMA_WARP) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
    if (wid == ITEM_WARP) {
      // Work items: the CTA's own grid position first, then positions that have not started, taken over one at a time
      // while the item before is in work.  (A grid of single-item CTAs pays for start, first loads and results of every
      // item with idle tensor cores: 12 packed prompts of up to 4001 tokens took 620 us.)
      int x = blockIdx.x, y, z, put = 0, at = 0, before = 0;
      bool checks = false;  // whoever has position 0 (of its own or taken over) looks at the bounds
      auto item_at = [&] {
#ifdef QEVICT_DEBUG_BOUNDS  // the checking build has its positions fall
        return item_of(a, (int)gridDim.x - 1 - x, lane, &at, &before);
#else
        return item_of(a, x, lane, &at, &before);
#endif
      };
      for (uint32_t ask = 0;; ++ask) {
        if (lane == 0) {
          words[8] = ask + 1;
          bar_expect(b_next, 16);
          asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                           smem_u32((void*)words)), "r"(b_next) : "memory");
        }
        checks = checks || x == 0;
        const PromptItem it = item_at();
        if (it.valid) {
          if (put >= 2) ok = wait_item(b_taken + 8 * (put & 1), (uint32_t)((put >> 1) - 1) & 1u);
          if (ok && lane == 0) {
            items[put & 1] = it;
            bar_arrive(b_item + 8 * (put & 1));
          } else if (!ok && lane == 0) {
            items[2] = it;
          }
          ++put;
        }
        __syncwarp();
        // (whatever has happened meanwhile: the answer is written to this CTA's memory)
        if (!warp_wait<false>(b_next, ask & 1u, words + 6)) {
          ok = false;
          break;
        }
        uint32_t got;
        asm volatile(
            "{\n\t.reg .b128 c;\n\t.reg .pred q;\n\tld.shared.b128 c, [%4];\n\t"
            "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 q, c;\n\tselp.u32 %0, 1, 0, q;\n\t"
            "mov.u32 %1, 0;\n\tmov.u32 %2, 0;\n\tmov.u32 %3, 0;\n\t"
            "@q clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, %2, %3, _}, c;\n\t}\n"
            : "=r"(got), "=r"(x), "=r"(y), "=r"(z) : "r"(smem_u32((void*)words)) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the answer is read before the next one is written
        __syncwarp();
        if (!got) break;
        if (!ok) {  // taken over, and nobody else's now
          checks = checks || x == 0;
          const PromptItem lost = item_at();
          if (lane == 0) items[3] = lost;
          break;
        }
      }
      // no more items
      if (ok && put >= 2) ok = wait_item(b_taken + 8 * (put & 1), (uint32_t)((put >> 1) - 1) & 1u);
      if (ok && lane == 0) {
        items[put & 1].valid = 0;
        bar_arrive(b_item + 8 * (put & 1));
      }
      if (checks && a.status) {
        for (int s = lane; s < a.n_seqs; s += 32)
          if (span_cut(a.q_bounds, a.padded, s, a.max_q, a.total_q) || span_cut(a.k_bounds, a.padded, s, a.max_k, a.total_k))
            kv8_record(a.status, CHECK_LENGTH);
      }
    } else if (wid == LOAD_WARP) {
      int slot = 0, q_turn = 0, issued = 0;
      uint32_t phase = 0;
      while (const PromptItem* item = next_item()) {
        const PromptItem& it = *item;
        const int cs = a.padded ? it.s : 0, loads = 2 * (it.n - it.lo), hk = it.h0 / (a.Hq / a.Hkv);
        if (loads == 0) continue;
        if (q_turn > 0) ok = wait_item(b_qe, (uint32_t)(q_turn - 1) & 1u);
        ++q_turn;
        if (ok && lane == 0) {
          bar_expect(b_q, (uint32_t)((it.cnt(0) > 0) + (it.cnt(1) > 0)) * (uint32_t)(a.T * a.P * D * 2));
#pragma unroll
          for (int w = 0; w < 2; ++w)
            if (it.cnt(w) > 0)
              for (int x = 0; x < D / 64; ++x)
                tma_load(smb + SM::Q_OFF + w * SM::TILE_BYTES + x * SM::HALF, &mq, b_q, x * 64, it.q0 + it.r0 + w * a.T, it.h0, cs);
          words[7] = (uint32_t)q_turn;
        }
        int v_slot = 0;
        uint32_t v_phase = 0;
        for (int i = 0; i < loads && ok; ++i) {  // K, V of the last tile, K, V of the one before, ...
          const int j = it.n - 1 - (i >> 1);
          if (issued >= NS) ok = wait_item(b_empty + 8 * slot, phase ^ 1u);
          if (ok && lane == 0) {
            bar_expect(b_full + 8 * slot, SM::TILE_BYTES);
            for (int x = 0; x < D / 64; ++x)
              tma_load(smb + SM::KV_OFF + slot * SM::TILE_BYTES + x * SM::HALF, (i & 1) ? &mv : &mk, b_full + 8 * slot, x * 64, it.k0 + j * TILE, hk, cs);
            words[5] = issued + 1;
          }
          ++issued;
          if (i == 1) { v_slot = slot; v_phase = phase; }
          if (++slot == NS) { slot = 0; phase ^= 1u; }
          if (ok && i == min(3, loads) - 1 && it.dirty()) {  // zero the value rows past the end
            ok = wait(b_full + 8 * v_slot, v_phase);
            const int from = it.nk - (it.n - 1) * TILE, per = (TILE - from) * 8;
            if (ok) {
              unsigned char* v0 = sm + SM::KV_OFF + v_slot * SM::TILE_BYTES + from * 128;
              for (int k = lane; k < per * (D / 64); k += 32) {
                const int x = k / per;
                *reinterpret_cast<uint4*>(v0 + x * SM::HALF + (k - x * per) * 16) = make_uint4(0u, 0u, 0u, 0u);
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) bar_arrive(b_clean);
            }
          }
          __syncwarp();
        }
      }
    } else if (wid == MMA_WARP) {
      // One thread issues every product, in the order S0 S1 | PV0 S0 PV1 S1 | ...: while one tile's softmax runs, the tensor
      // cores have the other tile's products.  S of the next tile overwrites P: one thread's products run in the order of
      // their issue.  (Two threads, one per tile, were slower, 9.8 against 8.4 ms on 32k tokens x 32 heads: their products
      // interleave, and both tiles wait for the slower.)
      // The whole warp walks the loop and one elected lane issues: what the products take (addresses, descriptors) is then
      // the same for all lanes and stays in uniform registers, which is where the instruction wants it.
      const uint32_t u_tm = (uint32_t)uniform((int)tmem), u_sm = (uint32_t)uniform((int)smb);
      const uint32_t fmt = Tr<T>::MAGIC == 0x64006400u ? 0u : 1u;  // 0 = fp16, 1 = bf16
      const uint32_t base = (1u << 4) | (fmt << 7) | (fmt << 10) | ((128u >> 4) << 24);
      const uint32_t id_s = base | ((128u >> 3) << 17);                           // both operands K-major
      const uint32_t id_o = base | (1u << 16) | ((uint32_t)(D >> 3) << 17);       // V: channels contiguous (N-major)
      const uint32_t q_lo = desc_lo(u_sm + SM::Q_OFF, 16), k_lo = desc_lo(u_sm + SM::KV_OFF, 16), v_lo = desc_lo(u_sm + SM::KV_OFF, SM::HALF);
      const uint32_t ub = u_sm + SM::BAR_OFF, u_full = ub + 8, u_empty = u_full + 8 * NS, u_s = u_empty + 8 * NS, u_p = u_s + 16, u_o = u_p + 16;
      leader = elect_one();
      // Half of the products of S, a look at the other tile's P, the other half: the look's latency passes while the tensor
      // cores have work.  (A wait costs this warp some 90 cycles even when there is nothing to wait for, and the queue
      // of products is short: with the waits between the products the call took 7 % longer.)
      bool seen = false;
      auto issue_s = [&](int w, int slot, uint32_t other_phase) {
        const uint32_t qa = q_lo + w * (SM::TILE_BYTES >> 4), ka = k_lo + slot * (SM::TILE_BYTES >> 4);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          if (leader) {
#pragma unroll
            for (int ks = part * (D / 32); ks < (part + 1) * (D / 32); ++ks) {
              const uint32_t o = ((uint32_t)(ks >> 2) * SM::HALF + (ks & 3) * 32) >> 4;
              mma_ss(u_tm + w * 128, qa + o, ka + o, id_s, ks > 0);
            }
            if (part == 1) commit_to(u_s + 8 * w);
          }
          __syncwarp();
          if (part == 0) seen = bar_peek(u_p + 8 * (w ^ 1), other_phase);
        }
      };
      auto p_ready = [&](int w, uint32_t phase) {
        const bool yes = __all_sync(0xffffffffu, seen) || wait(u_p + 8 * w, phase);
        seen = false;
        return yes;
      };
      auto issue_o = [&](int w, int slot, uint32_t acc) {
        const uint32_t va = v_lo + slot * (SM::TILE_BYTES >> 4);
        if (leader) {
#pragma unroll
          for (int ks = 0; ks < TILE / 16; ++ks)
            mma_ts(u_tm + 256 + w * 128, u_tm + w * 128 + P_COL(ks >> 2, ks & 3), va + ks * (2048 >> 4), id_o, ks > 0 ? 1u : acc);
        }
        __syncwarp();
      };
      int slot = 0;  // ring position and phase
      uint32_t phase = 0, phase0 = 0, phase1 = 0, q_phase = 0, clean_phase = 0;
      while (const PromptItem* item = next_item()) {
        const PromptItem& it = *item;
        const int u_n = uniform(it.n), u_lo = uniform(it.lo), u_n0 = uniform(it.nt0), u_n1 = uniform(it.nt1);
        if (u_n <= u_lo) continue;
        const bool dirty = it.dirty();
        if (!(ok = wait(ub, q_phase) && wait(u_full + 8 * slot, phase))) break;
        q_phase ^= 1u;
        if (u_n - 1 < u_n0) issue_s(0, slot, phase1);
        if (u_n - 1 < u_n1) issue_s(1, slot, phase0);
        seen = false;
        if (leader) {
          commit_to(u_empty + 8 * slot);
          if (u_n - 1 == u_lo) commit_to(b_qe);
        }
        __syncwarp();
        if (++slot == NS) { slot = 0; phase ^= 1u; }
        uint32_t acc0 = 0, acc1 = 0;
        for (int j = u_n - 1; j >= u_lo; --j) {
          const int sv = slot;
          ok = wait(u_full + 8 * sv, phase);  // V(j)
          if (++slot == NS) { slot = 0; phase ^= 1u; }
          if (ok && j == u_n - 1 && dirty) {
            ok = wait(b_clean, clean_phase);
            clean_phase ^= 1u;
          }
          const bool more = j > u_lo;
          if (more) ok = ok && wait(u_full + 8 * slot, phase);  // K(j - 1)
          if (!ok) break;
          if (j < u_n0) {
            if (!(ok = p_ready(0, phase0))) break;
            tm_after();
            issue_o(0, sv, acc0);
            acc0 = 1u;
            phase0 ^= 1u;
            if (!more && leader) commit_to(u_o);
          }
          if (more && j - 1 < u_n0) issue_s(0, slot, phase1);
          if (j < u_n1) {
            if (!(ok = p_ready(1, phase1))) break;
            tm_after();
            issue_o(1, sv, acc1);
            acc1 = 1u;
            phase1 ^= 1u;
            if (!more && leader) commit_to(u_o + 8);
          }
          if (more && j - 1 < u_n1) issue_s(1, slot, phase0);
          if (leader) {
            commit_to(u_empty + 8 * sv);
            if (more) commit_to(u_empty + 8 * slot);
            if (j - 1 == u_lo) commit_to(b_qe);  // the last S
          }
          __syncwarp();
          if (more && ++slot == NS) { slot = 0; phase ^= 1u; }
        }
        seen = false;
        if (!ok) break;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
    // Two threads to a row: 64 keys of every tile each.  The two warps that share rows meet at a barrier of their own, which
    // also gives both the same answer to whether a wait of either's has run out, so that both leave at the same point.
    const int w = wid >> 3, half = (wid >> 2) & 1, r = (wid & 3) * 32 + lane;
    const int hl = r / a.T, tok = w * a.T + r - hl * a.T;  // head and token of this row; rows past P heads are not used
    const uint32_t lane_base = (uint32_t)((wid & 3) * 32) << 16;
    const uint32_t ts = tmem + lane_base + w * 128, to = tmem + lane_base + 256 + w * 128 + half * (D / 2);
    float* xch = reinterpret_cast<float*>(sm + SM::BAR_OFF + SM::ROWS) + w * 2 * TILE + r;  // the two halves' values of a row
    auto meet = [&] {
      uint32_t both;
      asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}\n"
                   : "=r"(both) : "r"((uint32_t)ok), "r"(1 + w * 4 + (wid & 3)) : "memory");
      ok = both != 0;
    };
    uint32_t s_phase = 0, o_phase = 0;
    while (true) {
      const PromptItem* item = next_item();
      meet();
      if (!ok || !item) break;
      const PromptItem& it = *item;
      const int cnt = it.cnt(w);
      // keys that this row still sees from the tile's (this half's) first on; grows by a tile each time
      int left = (a.causal ? min(it.nk, it.r0 + tok + it.nk - it.nq + 1) : it.nk) - ((w ? it.nt1 : it.nt0) - 1) * TILE - half * (TILE / 2);
      const bool mine = it.r0 + tok < it.nq && hl < a.P;  // rows of nobody hold anything, and have no say below
      float m = -INFINITY, l = 0.f;
      for (int i = cnt; i > 0; --i, left += TILE) {
        // S(j) stands for P V of the tile before too: a commit waits for everything its thread has issued before
        ok = wait(b_s + 8 * w, s_phase);
        s_phase ^= 1u;
        float x[TILE / 2];
        if (ok) {
          tm_after();
          tm_ld32(ts + half * 64, x);
          tm_ld32(ts + half * 64 + 32, x + 32);
          tm_wait_ld();
          if (__any_sync(0xffffffffu, left < TILE / 2)) {
#pragma unroll
            for (int c = 0; c < TILE / 2; ++c) x[c] = c < left ? x[c] : -INFINITY;
          }
          float mx[4] = {max3(x[0], x[1], x[2]), max3(x[3], x[4], x[5]), max3(x[6], x[7], x[8]), max3(x[9], x[10], x[11])};
#pragma unroll
          for (int c = 12; c < TILE / 2 - 4; c += 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], x[c + 2 * k], x[c + 2 * k + 1]);
          mx[0] = max3(mx[0], x[TILE / 2 - 4], x[TILE / 2 - 3]);
          mx[1] = max3(mx[1], x[TILE / 2 - 2], x[TILE / 2 - 1]);
          xch[half * TILE] = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
        }
        meet();
        if (!ok) break;
        const float top_x = fmaxf(xch[0], xch[TILE]) * a.scale_log2;
        if (__any_sync(0xffffffffu, mine && top_x > m + PROMPT_LAZY)) {
          const float m_new = fmaxf(m, top_x);
          const float f = m_new == m ? 1.f : ex2p(m - m_new);
          m = m_new;
          l *= f;
          if (i < cnt) {
#pragma unroll 1
            for (int c = 0; c < D / 2; c += 8) {  // few at a time: the logits stay in registers
              float o[8];
              tm_ld8(to + c, o);
              tm_wait_ld();
#pragma unroll
              for (int k = 0; k < 8; ++k) o[k] *= f;
              tm_st8(to + c, reinterpret_cast<const uint32_t*>(o));
            }
          }
        }
        const float ms = m == -INFINITY ? 0.f : -m;
        uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
        for (int q = 0; q < 4; ++q) {  // P of 16 keys at a time: what else is live fits the registers (a spill here costs 30 to 60 %)
          uint32_t p[8];
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            float p0, p1;
            unpair(fma2(pair(x[q * 16 + 2 * c], x[q * 16 + 2 * c + 1]), pair(a.scale_log2, a.scale_log2), pair(ms, ms)), p0, p1);
            p0 = ex2p(p0);
            p1 = ex2p(p1);
            sum[c & 1] = add2(sum[c & 1], pair(p0, p1));
            p[c] = pack2<T>(p0, p1);
          }
          tm_st8(ts + P_COL(half, q), p);
        }
        tm_wait_st();
        tm_before();
        __syncwarp();
        if (lane == 0) bar_arrive(b_p + 8 * w);
        float s0, s1;
        unpair(add2(sum[0], sum[1]), s0, s1);
        l += s0 + s1;
      }
      if (!ok) break;
      // results: the two halves' sums, half of the channels each
      if (cnt > 0) {
        ok = wait(b_o + 8 * w, o_phase);
        o_phase ^= 1u;
      }
      tm_after();
      xch[half * TILE] = l;
      meet();
      if (!ok) break;
      l = xch[0] + xch[TILE];
      const int row = it.r0 + tok, hq = it.h0 + hl;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const long long prow = a.padded ? (long long)it.s * a.max_q + row : (long long)it.q0 + row;
      const float lse2 = l == 0.f ? -INFINITY : m + log2f(l);
      if (mine && half == 0) {
        if (a.splits > 1)
          a.part_lse[((long long)it.split * a.rows + prow) * a.Hq + hq] = lse2;
        else if (a.lse)
          a.lse[a.padded ? ((long long)it.s * a.Hq + hq) * a.max_q + row : hq * a.total_q + prow] = lse2 * 0.6931471805599453f;
      }
      T* out = static_cast<T*>(a.out) + (a.padded ? it.s * a.out_stride[0] + row * a.out_stride[2] : prow * a.out_stride[2]) +
               hq * a.out_stride[1] + half * (D / 2);
      float* po = a.part_o + (((long long)it.split * a.rows + prow) * a.Hq + hq) * D + half * (D / 2);
#pragma unroll 1
      for (int c = 0; c < D / 2; c += 16) {
        float o[16];
        if (cnt > 0) {  // warp-uniform
          tm_ld16(to + c, o);
          tm_wait_ld();
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) o[k] = l == 0.f ? 0.f : o[k] * inv;
        if (!mine) continue;
        if (a.splits > 1) {
#pragma unroll
          for (int k = 0; k < 16; k += 4) *reinterpret_cast<float4*>(po + c + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
        } else {
#pragma unroll
          for (int k = 0; k < 16; k += 8)
            *reinterpret_cast<uint4*>(out + c + k) =
                make_uint4(pack2<T>(o[k], o[k + 1]), pack2<T>(o[k + 2], o[k + 3]), pack2<T>(o[k + 4], o[k + 5]), pack2<T>(o[k + 6], o[k + 7]));
        }
      }
      __syncwarp();
    }
  }
  tm_before();
  __syncthreads();
  tm_after();
  if (words[6]) {  // a wait has given up: nothing may be under way when tensor and shared memory are given back
    if (wid == MMA_WARP) {
      if (leader) commit_to(b_done);
      __syncwarp();
      bar_wait(b_done, 0);
    }
    if (tid == 0) {
      const int issued = (int)words[5], queries = (int)words[7], asked = (int)words[8];
      for (int i = max(0, issued - NS); i < issued; ++i) bar_wait(b_full + 8 * (i % NS), (uint32_t)(i / NS) & 1u);
      if (queries) bar_wait(b_q, (uint32_t)(queries - 1) & 1u);
      if (asked) bar_wait(b_next, (uint32_t)(asked - 1) & 1u);
      kv8_record(a.status, CHECK_COPY_TIMEOUT);
    }
    // The rows of the items that may not be finished become not-a-number, for callers who do not read the status: the two that
    // were handed out last and the two that were not.
    for (int n = 0; n < 4; ++n) {
      const PromptItem& it = items[n];
      for (int i = tid; it.valid && i < 2 * a.T * a.P; i += PROMPT_THREADS) {
        const int row = it.r0 + i / a.P, hq = it.h0 + i % a.P;
        if (row >= it.nq) break;
        const long long prow = a.padded ? (long long)it.s * a.max_q + row : (long long)it.q0 + row;
        if (a.splits > 1) {
          a.part_lse[((long long)it.split * a.rows + prow) * a.Hq + hq] = NAN;  // as a weight, it makes the merged row that
          continue;
        }
        if (a.lse) a.lse[a.padded ? ((long long)it.s * a.Hq + hq) * a.max_q + row : hq * a.total_q + prow] = NAN;
        T* out = static_cast<T*>(a.out) + (a.padded ? it.s * a.out_stride[0] + row * a.out_stride[2] : prow * a.out_stride[2]) + hq * a.out_stride[1];
        for (int c = 0; c < D; ++c) out[c] = Tr<T>::from_float(NAN);
      }
    }
  }
  __syncthreads();
  if (wid == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// Joins the partial results of a split call: one warp per (row, head), a lane per part for the weights (at most 64 parts), then
// per 2 or 4 channels.
template <class T, int D>
__global__ void __launch_bounds__(256) prompt_merge_kernel(const PromptArgs a) {
  constexpr int PER = D / 32;
  const int lane = threadIdx.x & 31, s = blockIdx.y;
  pdl_prologue();
  int q0, nq;
  span_of(a.q_bounds, a.padded, s, a.max_q, a.total_q, &q0, &nq);
  const long long at = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int row = (int)(at / a.Hq), hq = (int)(at - (long long)row * a.Hq);
  if (row >= nq) return;
  const long long prow = a.padded ? (long long)s * a.max_q + row : (long long)q0 + row;
  const long long first = prow * a.Hq + hq, next = a.rows * a.Hq;  // of part 0; from part to part
  float w0 = lane < a.splits ? a.part_lse[first + lane * next] : -INFINITY;
  float w1 = lane + 32 < a.splits ? a.part_lse[first + (lane + 32) * next] : -INFINITY;
  float M = fmaxf(w0, w1);
#pragma unroll
  for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  const float Ms = M == -INFINITY ? 0.f : M;
  w0 = ex2p(w0 - Ms);
  w1 = ex2p(w1 - Ms);
  float L = w0 + w1;
#pragma unroll
  for (int o = 16; o; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
  float sum[PER] = {};
#pragma unroll 4
  for (int i = 0; i < a.splits; ++i) {
    const float f = __shfl_sync(0xffffffffu, i < 32 ? w0 : w1, i & 31);
    const float* src = a.part_o + (first + i * next) * D + lane * PER;
    float v[PER];
    if (PER == 4) {
      const float4 x = *reinterpret_cast<const float4*>(src);
      v[0] = x.x; v[1] = x.y; v[2 % PER] = x.z; v[3 % PER] = x.w;
    } else {
      const float2 x = *reinterpret_cast<const float2*>(src);
      v[0] = x.x; v[1] = x.y;
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) sum[k] += f * v[k];
  }
  T* out = static_cast<T*>(a.out) + (a.padded ? s * a.out_stride[0] + row * a.out_stride[2] : prow * a.out_stride[2]) + hq * a.out_stride[1] + lane * PER;
#pragma unroll
  for (int k = 0; k < PER; k += 2)
    *reinterpret_cast<uint32_t*>(out + k) = L == 0.f ? 0u : pack2<T>(sum[k] / L, sum[k + 1] / L);
  if (lane == 0 && a.lse)
    a.lse[a.padded ? ((long long)s * a.Hq + hq) * a.max_q + row : hq * a.total_q + prow] =
        L == 0.f ? -INFINITY : (Ms + log2f(L)) * 0.6931471805599453f;
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
  static EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}

// {channel, token, head, sequence} map of boxes of 64 channels x some tokens x some heads
bool make_map(CUtensorMap* map, int dtype, const void* base, int D, long long tokens, int heads, long long seqs, const int64_t* stride,
              int box_tokens, int box_heads) {
  memset(map, 0, sizeof(*map));
  if (tokens < 1) return true;  // no rows: no copy is made
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)tokens, (cuuint64_t)heads, (cuuint64_t)seqs};
  // a dimension of one element has no stride that matters
  const cuuint64_t st[3] = {(cuuint64_t)(tokens > 1 ? stride[2] : D) * 2, (cuuint64_t)(heads > 1 ? stride[1] : D) * 2,
                            (cuuint64_t)(seqs > 1 ? stride[0] : D) * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)box_tokens, (cuuint32_t)box_heads, 1}, el[4] = {1, 1, 1, 1};
  EncodeFn fn = encode_fn();
  return fn && fn(map, dtype == QEVICT_DTYPE_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base),
                  dims, st, box, el, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Rows of a query tile: the heads that share a KV head side by side (P of them, the largest divisor of the group up to 32),
// as many tokens of each as fit 128 rows.  Never more tiles than one head at a time, fewer for few tokens, and the
// triangle at the causal edge is P times narrower.
void prompt_tile(const qevict_prompt_args* p, int* P, int* T) {
  const int G = p->n_q_heads / p->n_kv_heads;
  *P = G < 32 ? G : 32;
  while (G % *P) --*P;
  *T = TILE / *P;
}

// Most tile pairs that the sequences can have, for one group of heads: with max_q rows each, or total_q rows cut anywhere.
long long prompt_tiles(bool padded, int n_seqs, long long max_q, long long total_q, int T) {
  const long long each = n_seqs * ((max_q + 2 * T - 1) / (2 * T)), all = total_q / (2 * T) + n_seqs;
  return padded || each < all ? each : all;
}

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
  prompt_tile(p, &P, &T);
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

int prompt_sms(int device) {
  int n = 0;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) {
    (void)cudaGetLastError();
    n = SM_COUNT_FALLBACK;
  }
  return n;
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
  prompt_tile(p, &P, &T);
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
  auto kernel = prompt_attn_kernel<T, D>;
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
  PromptArgs a;
  a.padded = padded; a.n_seqs = args->n_seqs; a.Hq = args->n_q_heads; a.Hkv = args->n_kv_heads; a.D = args->head_dim;
  a.max_q = args->max_q; a.max_k = args->max_k; a.causal = args->causal;
  prompt_tile(args, &a.P, &a.T);
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
