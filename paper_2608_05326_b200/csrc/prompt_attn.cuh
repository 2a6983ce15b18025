// Attention over whole prompts, and of new tokens over a paged cache (PAGED), on the 5th-generation tensor cores.
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
//   - The reference exponent m of a row moves only when a logit exceeds by 2^8 the largest one that it was set by (then O is
//     rescaled in tensor memory); sums are float32.  P is rounded to the type of the values, with which it enters the product:
//     half a step each.  In fp16 m stands 2^7 below the largest logit (P_UP), so that P fills the type's range up to 2^15 and is
//     lost below 2^-32 of the largest probability: with m at the largest logit 65536 keys at 2^-25 of it stayed in the sum and
//     vanished from the product, 0.2 % of the row.
// What bounds it: at d = 128 a key tile costs both query tiles 2048 tensor-core cycles at best; with both operands of S in
// shared memory the products alone take about 2750 (8 KB of operands for 64 cycles of products, at 128 bytes a cycle, and
// the copies write through the same port), and a step takes about 3600 with the softmax behind it.  Measured, call after
// call: causal 32768 tokens x 32 heads 7.82 to 7.97 ms (1103 to 1125 TFLOP/s, 0.8 of the measured sustained rate; the power limit holds
// it there: single calls of a cool card take 6.8 to 7.4 ms); 12 packed prompts of up to 4001 tokens 572 to 594 us (849 to 882 TFLOP/s),
// the best of graph replays 494 to 512 us; d = 64: 16384 tokens x 32 heads 1.57 ms (702 TFLOP/s: half the products for the same
// exponentials).  Shares of the exponentials as polynomials on the FMA units were slower at every share (1/2 to 1/16): what the
// softmax waits for is issue and hand-over, not the exponential unit.
//
// Few query rows (one token, a short piece behind a long prefix): the keys are split over several CTAs whose partial
// outputs prompt_merge_kernel joins.
//
// PAGED: keys and values come by page, one copy for each page of a head (a box of {64 channels, 8 tokens, d / 64 pieces, groups}: the
// pieces of eight keys land side by side, which the products' descriptors follow); copies of 64 channels of a page took 276 us
// where these took 214, pages of 16 tokens, 8 x 65536 tokens.  Calls with fewer than six items for each SM give every CTA an
// equal range of the work (PagedRange) and join what ranges share in paged_merge_kernel; others hand out whole items as above.
// A sequence with one tile of rows has both query tiles take the same rows and half of the keys each.  Measured, 32 / 8 heads of
// 128, call after call on several cards (single calls of a cool one): 8192 tokens behind 57344 7.70 to 7.79 ms, 1060 to 1071 TFLOP/s (6.6);
// pieces of up to 701 tokens behind up to 24000 of four prompts 480 to 490 us, 888 to 906 TFLOP/s (415); drafts of up to 5 tokens of 16
// users with up to 32768 178 to 188 us, 5.0 to 5.3 TB/s (165).  Registers: of the 476 bytes that the compiler reports
// as spilled at d = 128 (832 loaded) 290 (530) go with the item warp's search for its range, which runs beside the products in 32
// registers: without that search it reports 184 (300), and 28 (24) for the kernel without pages.
//
// Keys past the sequence's end are masked by selection, so what lies there (another sequence, padding, NaN) never
// enters; value rows past the end are zeroed in shared memory before the product reads them, since 0 * NaN is NaN.
// Every wait is bounded; one that runs out records CHECK_COPY_TIMEOUT and the CTA leaves after its copies have landed and its
// unfinished rows have become not-a-number.
#pragma once

#include <cuda.h>
#ifdef QEVICT_DEBUG_BOUNDS
#include <stdio.h>
#include <stdlib.h>
#endif

#include "kv16.cuh"

namespace qevict {

namespace {

constexpr int PROMPT_THREADS = 640;  // four softmax warpgroups, one for products, copies and work items (a warp idle)
constexpr int MMA_WARP = 16, LOAD_WARP = 17, ITEM_WARP = 18;
constexpr int TILE = 128;           // query rows of a tile, keys of a tile
constexpr float PROMPT_LAZY = 8.f;  // log2
// How far below a row's largest logit its reference is set (log2); P is at most 2^(P_UP + PROMPT_LAZY).
template <class T> constexpr float P_UP = 0.f;  // bf16 has the range of float32
template <> constexpr float P_UP<__half> = 7.f;

// An item whose keys the ranges of several CTAs share: it starts in the CTA that has this record and ends in the range of CTA `last`.
struct PagedCut {
  int valid, s, h0, r0, q0, nq, last, pair;
};

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
  // keys and values in pages (PAGED): a sequence's length is k_bounds[s], its rows of q are q_bounds' or, without them, row s
  const int32_t* table;  // [n_seqs][max_blocks]
  int max_blocks, block_log2, n_pages;
  long long lse_rows;    // rows of lse
  double inv_step;       // 1 / (2 T)
  int groups;            // Hq / P
  int by_range;          // each CTA has an equal range of the call's work, else whole items as they fall free
  int slot_rows;         // rows of a partial result: [slot][D / 4][slot_rows][4], a warp's rows side by side
  PagedCut* cuts;        // [CTAs]
  int group_bytes, half_bytes;  // of K and V tiles in shared memory: from 8 keys to the next 8, from 64 channels to the next 64
  int boxes;             // copies for each page: one, or one for each 64 channels
  int head_step[2];      // keys, values: from head to head in the third coordinate
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
// a page's rows of a head: {channels, 8 tokens, 64-channel pieces of heads, groups of 8 tokens, pages}
__device__ __forceinline__ void tma_page(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int piece, int page) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %4, %6}], [%2];"
               ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(0), "r"(piece), "r"(page) : "memory");
}
__device__ __forceinline__ void commit_to(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Descriptor of a shared-memory operand with the 128-byte swizzle: the low word holds the address and the leading byte
// offset, the high word (constant) the stride of 1024 bytes between groups of eight rows, version 1 and the swizzle.
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo) { return ((addr >> 4) & 0x3FFFu) | ((lbo >> 4) << 16); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t acc, uint32_t b_hi = DESC_HI) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %6};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}\n" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(acc), "r"(DESC_HI), "r"(b_hi)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t acc, uint32_t b_hi = DESC_HI) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 db, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}\n" ::"r"(d), "r"(a), "r"(b_lo), "r"(idesc), "r"(acc), "r"(b_hi)
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
  static constexpr int WORDS = 320, ITEMS = 384, ROWS = 656;  // behind the barriers: words, work items, row maxima
  static constexpr int BYTES = BAR_OFF + ROWS + 2048;
};

// The rows of sequence s among the queries, its keys.
template <bool PAGED> __device__ __forceinline__ void q_span(const PromptArgs& a, int s, int* first, int* n) {
  if (PAGED && !a.q_bounds) {
    *first = s;
    *n = min(1, a.max_q);
  } else {
    span_of(a.q_bounds, a.padded, s, a.max_q, a.total_q, first, n);
  }
}
template <bool PAGED> __device__ __forceinline__ void k_span(const PromptArgs& a, int s, int* first, int* n) {
  span_of(a.k_bounds, PAGED || a.padded, s, a.max_k, a.total_k, first, n);
}
template <bool PAGED> __device__ __forceinline__ bool seq_cut(const PromptArgs& a, int s) {
  return (!(PAGED && !a.q_bounds) && span_cut(a.q_bounds, a.padded, s, a.max_q, a.total_q)) ||
         span_cut(a.k_bounds, PAGED || a.padded, s, a.max_k, a.total_k);
}

// Few queries (one tile of rows) have both query tiles of a CTA take the same rows, each one half of the key tiles: one's softmax
// then runs beside the other's products as it does for two tiles of rows.
__device__ __forceinline__ bool paged_pair(const PromptArgs& a, int nq, int keys) { return nq <= a.T && keys > TILE; }

// A work item: two tiles of T tokens of P heads of one sequence, or a part of their keys.
struct PromptItem {
  int valid, h0, s, split, r0, q0, nq, k0, nk;  // h0: first query head, r0: first token
  int lo, n;       // key tiles of this item
  int nt0, nt1;    // end of the two query tiles' key tiles
  // paged: both tiles have the same rows, the second one the key tiles lo .. mid - 1; where the results go, -1: to the output; key
  // tiles of the CTA's items before
  int pair, mid, slot, before;
  __device__ __forceinline__ int cnt(int w) const { return pair ? (w ? mid - lo : n - mid) : max(0, (w ? nt1 : nt0) - lo); }
  __device__ __forceinline__ bool dirty() const { return n > lo && n * TILE > nk; }  // the first tile reaches past the sequence
};

// Key tiles that an item's two query tiles see.
__device__ __forceinline__ void item_tiles(const PromptArgs& a, PromptItem* it) {
  int nt[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int rw = it->r0 + w * a.T, last = min(rw + a.T, it->nq) - 1;
    const int lim = rw >= it->nq ? 0 : (a.causal ? min(it->nk, last + it->nk - it->nq + 1) : it->nk);
    nt[w] = lim > 0 ? (lim + TILE - 1) / TILE : 0;
  }
  it->lo = 0;
  it->n = max(nt[0], nt[1]);
  it->nt0 = nt[0];
  it->nt1 = nt[1];
}
// What each query tile does of the item's key tiles lo .. n - 1.
template <bool PAGED> __device__ __forceinline__ void item_streams(const PromptArgs& a, PromptItem* it) {
  it->nt0 = min(it->nt0, it->n);
  it->nt1 = min(it->nt1, it->n);
  it->pair = PAGED && paged_pair(a, it->nq, it->nk);
  it->mid = it->lo;
  if (it->pair) {
    it->mid = it->lo + (it->n - it->lo) / 2;
    it->nt0 = it->n;
    it->nt1 = it->mid;
  }
}

// The item of grid position x, for a whole warp; not valid where x lies past the last sequence's.  Positions go by the
// sequences' own lengths, so a batch of very different lengths has next to no empty positions, and by falling cost, so that the
// SMs end together: sequences in groups of 32; in a group the tiles by falling number of keys, level by level (a level: the rows
// of one tile more or less; a sequence's tiles have one each, from its prefix on); on a level the sequences that have it; then
// the heads, then the parts of the keys.  *at, *before: where the last search ended (first sequence of the group, items before
// it), which is where the next one starts; positions mostly grow, but nothing promises it: a smaller one starts at the front.
template <bool PAGED> __device__ __forceinline__ PromptItem item_of(const PromptArgs& a, int x, int lane, int* at, int* before) {
  PromptItem it;
  const int t = x / a.splits, step = 2 * a.T, groups = a.Hq / a.P;
  it.split = x - t * a.splits;
  it.h0 = 0;
  it.valid = 0;
  it.slot = -1;
  it.before = 0;
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
      q_span<PAGED>(a, s, &first, &n);
      k_span<PAGED>(a, s, &first, &keys);
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
  q_span<PAGED>(a, it.s, &it.q0, &it.nq);
  k_span<PAGED>(a, it.s, &it.k0, &it.nk);
  item_tiles(a, &it);
  if (a.splits > 1) {
    const int per = (it.n + a.splits - 1) / a.splits;
    it.lo = min(it.n, it.split * per);
    it.n = min(it.n, it.lo + per);
  }
  item_streams<PAGED>(a, &it);
  return it;
}

// Paged calls with few items for the SMs: each CTA has an equal range of the call's work, whatever the lengths.
//
// The items stand in a row: sequence by sequence, heads in it, tiles of rows in these.  An item costs its visible keys (three
// quarters for pairs, whose two tiles a step bandwidth bounds) and a constant (8200 cycles of 3800 for a tile of keys; pairs,
// which drain the copies, 16500 of 2000).  Pairs' keys at two, three and four quarters, graph replays: a piece of 2048 tokens between 31
// single ones 707, 703, 731 us (heads of 64: 636, 609, 653); drafts of 16 users 245, 241, 269; of 64 users with 2048 tokens each 122,
// 121, 120; a piece of 300 between 8 single ones 193, 235, 287.  CTA c has what lies in [c, c + 1) * W of the sum.  An end inside an
// item is moved to a key tile: an item has the CTAs that have tiles of it, and where these are several, each writes a partial result.
// The ranges are a function of the lengths alone.  The sum is held in 64 bits: bounds that fall and rise give many sequences the same
// rows, so no bound on the rows keeps it within 32 (an item that crossed the end of a sum that had wrapped named a CTA behind the
// last, whose results the join then read behind the scratch).
constexpr int ITEM_COST = 1024, KEY_COST = 4, ITEM_COST_PAIR = 3200, KEY_COST_PAIR = 3, RANGE_LEAST = 1024;

// (What runs before the first copy runs once, from instructions that are fetched as they come: some 50 cycles for each, so its
// divisions are worth replacing.)
// x / y where that is below 2^20: the float quotient is off by less than one
template <class U> __device__ __forceinline__ uint32_t small_quotient(U x, U y) {
  uint32_t q = (uint32_t)__fdividef((float)x, (float)y);
  if (q * y > x) --q;
  if (x - q * y >= y) ++q;
  return q;
}
struct PagedSeq {
  int q0, nq, nk, tiles, key_cost;
  // visible keys of row tile t, and of all before it
  __device__ __forceinline__ int keys(const PromptArgs& a, int t) const {
    return !a.causal || t == tiles - 1 ? nk : max(0, nk - nq + (t + 1) * 2 * a.T);
  }
  __device__ __forceinline__ long long before(const PromptArgs& a, int t) const {
    if (!a.causal) return (long long)t * nk;
    // full tiles of rows, of which the first u see nothing (fewer than 2^10 in a call of ranges)
    const int step = 2 * a.T, full = t < tiles ? t : tiles - 1, u = nk < nq ? min(full, (nq - nk) / step) : 0;
    return (long long)(full - u) * (nk - nq) + a.T * (full * (full + 1) - u * (u + 1)) + (t < tiles ? 0 : nk);
  }
  __device__ __forceinline__ uint32_t item_cost() const { return key_cost == KEY_COST ? ITEM_COST : ITEM_COST_PAIR; }
  __device__ __forceinline__ uint64_t cost(const PromptArgs& a, int t) const { return (uint64_t)key_cost * (uint32_t)keys(a, t) + item_cost(); }
  __device__ __forceinline__ uint64_t cost_before(const PromptArgs& a, int t) const { return t > 0 ? key_cost * (uint64_t)before(a, t) + t * item_cost() : 0ull; }
};

__device__ __forceinline__ PagedSeq paged_seq(const PromptArgs& a, int q0, int nq, int nk) {
  // (x + 1/2) / step is at least 1 / (2 step) from a whole number, far more than it is rounded by
  return {q0, nq, nk, (int)((nq + 2 * a.T - 0.5) * a.inv_step), paged_pair(a, nq, nk) ? KEY_COST_PAIR : KEY_COST};
}

struct PagedRange {
  uint64_t width, lo, hi, at;  // this CTA's part of the sum; start of the current item
  int s, h, t;
  bool begun;  // the current item has been given
  PagedSeq seq;
  int lane_q0, lane_nq, lane_nk, first;  // the lane's sequence of 32, of which `first` is the first

  __device__ __forceinline__ PagedSeq look(const PromptArgs& a, int s0, int lane) {
    int k0;
    lane_q0 = lane_nq = lane_nk = 0;
    first = s0;
    if (s0 + lane < a.n_seqs) {
      q_span<true>(a, s0 + lane, &lane_q0, &lane_nq);
      k_span<true>(a, s0 + lane, &k0, &lane_nk);
    }
    return paged_seq(a, lane_q0, lane_nq, lane_nk);
  }
  __device__ __forceinline__ PagedSeq sequence(const PromptArgs& a, int s, int lane) {  // of the whole warp
    if (s >= first + 32) look(a, s & ~31, lane);
    return paged_seq(a, __shfl_sync(0xffffffffu, lane_q0, s & 31), __shfl_sync(0xffffffffu, lane_nq, s & 31),
                     __shfl_sync(0xffffffffu, lane_nk, s & 31));
  }

  __device__ __forceinline__ PagedRange(const PromptArgs& a, int lane) {
    const int groups = a.groups;
    uint64_t sum = 0, mine = 0;
#pragma unroll 1
    for (int i = 0; i < a.n_seqs; i += 32) {
      const PagedSeq q = look(a, i, lane);
      mine = q.cost_before(a, q.tiles) * groups;
      // (a sequence's work is below 2^44: in a call of ranges fewer than 2^11 items of 2^33 at most)
      sum += __reduce_add_sync(0xffffffffu, (uint32_t)mine & 0xffffffu) + ((uint64_t)__reduce_add_sync(0xffffffffu, (uint32_t)(mine >> 24)) << 24);
    }
    width = sum >> 31 ? (sum + gridDim.x - 1) / gridDim.x : ((uint32_t)sum + gridDim.x - 1) / gridDim.x;
    begun = false;
    if (width < RANGE_LEAST) width = RANGE_LEAST;
    lo = blockIdx.x * width;
    hi = min(lo + width, sum);
    s = a.n_seqs;
    if (lo >= sum) return;
    uint64_t front = 0;  // cost of the sequences before
#pragma unroll 1
    for (int i = 0; i < a.n_seqs; i += 32) {
      if (a.n_seqs > 32) {
        const PagedSeq q = look(a, i, lane);
        mine = q.cost_before(a, q.tiles) * groups;
      }
      uint64_t upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint64_t x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, front + upto > lo);
      if (past) {
        const int who = __ffs(past) - 1;
        s = i + who;
        front += __shfl_sync(0xffffffffu, upto - mine, who);
        break;
      }
      front += __shfl_sync(0xffffffffu, upto, 31);
    }
    seq = sequence(a, s, lane);
    const uint64_t head = seq.cost_before(a, seq.tiles);
    h = small_quotient(lo - front, head);
    front += h * head;
    int t0 = 0, t1 = seq.tiles - 1;  // the last tile that starts at or before lo
#pragma unroll 1
    while (t0 < t1) {
      const int mid = (t0 + t1 + 1) >> 1;
      if (front + seq.cost_before(a, mid) <= lo) t0 = mid; else t1 = mid - 1;
    }
    t = t0;
    at = front + seq.cost_before(a, t);
  }

  // The next item of the range, its key tiles in it; false behind the last one.
  __device__ __forceinline__ bool next(const PromptArgs& a, int lane, bool writes, PromptItem* it) {
#pragma unroll 1
    while (true) {
      if (begun) {
        at += seq.cost(a, t);
        if (++t == seq.tiles) {
          t = 0;
          if (++h == a.groups) {
            h = 0;
            do {
              if (++s < a.n_seqs) seq = sequence(a, s, lane);
            } while (s < a.n_seqs && seq.tiles == 0);
          }
        }
      }
      begun = true;
      if (s >= a.n_seqs || at >= hi) return false;
      const uint64_t end = at + seq.cost(a, t);
      it->valid = 1;
      it->s = s; it->h0 = h * a.P; it->r0 = t * 2 * a.T;
      it->q0 = seq.q0; it->nq = seq.nq; it->k0 = 0; it->nk = seq.nk;
      it->split = 0;
      item_tiles(a, it);
      const int all = it->n;
      auto tiles_upto = [&](uint64_t x) {
        if (x <= at + seq.item_cost()) return 0;
        const uint32_t rows = (uint32_t)((x - at - seq.item_cost()) / TILE);
        return (int)(seq.key_cost == KEY_COST ? rows / KEY_COST : rows / KEY_COST_PAIR);
      };
      const bool ends = end <= hi;
      it->lo = lo > at ? tiles_upto(lo) : 0;
      it->n = ends ? all : tiles_upto(hi);
      it->slot = it->lo == 0 && ends ? -1 : 2 * (int)blockIdx.x + (it->lo == 0);
      if (it->lo == 0 && it->n > 0 && !ends && writes) {
        const PagedCut c = {1, s, it->h0, it->r0, seq.q0, seq.nq, (int)small_quotient(end - 1, width), seq.key_cost == KEY_COST_PAIR};
        a.cuts[blockIdx.x] = c;
      }
      if (it->n > it->lo || (all == 0 && ends)) {
        item_streams<true>(a, it);
        return true;
      }
    }
  }
};

// Four channels from c on of row r of a partial result.  (Rows of D channels side by side had a warp write 32 pieces of 16 bytes at a
// time: 25 to 33 thousand cycles for the results of an item.)
template <int D> __device__ __forceinline__ float4* part_at(const PromptArgs& a, int slot, int c, int r) {
  return reinterpret_cast<float4*>(a.part_o) + ((long long)slot * (D / 4) + (c >> 2)) * a.slot_rows + r;
}

template <class T, int D, bool PAGED>
__global__ void __launch_bounds__(PROMPT_THREADS, 1)
    prompt_attn_kernel(const PromptArgs a, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                       const __grid_constant__ CUtensorMap mv) {
  using SM = PromptSmem<D>;
  constexpr int NS = SM::STAGES;
  extern __shared__ __align__(1024) unsigned char sm[];  // the swizzle counts from multiples of 1024 bytes
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const uint32_t smb = smem_u32(sm), bars = smb + SM::BAR_OFF;
  // barriers: Q full / empty; ring full / empty; S ready, P ready, O ready of both tiles; value tail zeroed; work items
  // full / empty (two places); answer to the request for the next one; products done after a failure; (paged) the four warps
  // that share rows of a pair
  const uint32_t b_q = bars, b_full = bars + 8, b_empty = b_full + 8 * NS, b_s = b_empty + 8 * NS, b_p = b_s + 16, b_o = b_p + 16,
                 b_clean = b_o + 16, b_qe = b_clean + 8, b_item = b_qe + 8, b_taken = b_item + 16, b_next = b_taken + 16,
                 b_done = b_next + 8, b_quad = b_done + 8;
  // (paged) words 9 .. 12: a byte for each of the last 16 key tiles, bit i: its i-th block is absent
  // words: 0 .. 3 the answer; 4 tensor memory; 5 loads of K and V issued; 6 a wait has given up; 7 loads of Q; 8 requests for items
  volatile uint32_t* words = reinterpret_cast<volatile uint32_t*>(sm + SM::BAR_OFF + SM::WORDS);
  volatile uint8_t* masks = reinterpret_cast<volatile uint8_t*>(words + 9);
  PromptItem* items = reinterpret_cast<PromptItem*>(sm + SM::BAR_OFF + SM::ITEMS);
  static_assert(SM::ITEMS + sizeof(PromptItem) * 4 <= SM::ROWS, "two work items, and two that could not be handed out");
  if (smb & 1023u) {  // no tile would be where the products look for it
    if (PAGED) pdl_prologue();
    if (PAGED && a.cuts && tid == 0) a.cuts[blockIdx.x].valid = 0;
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
    for (int i = 0; i < 4; ++i) bar_init(b_quad + 8 * i, 4);
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
      int x = blockIdx.x, y, z, put = 0, at = 0, before = 0, k_tiles = 0;
      bool checks = false;  // whoever has position 0 (of its own or taken over) looks at the bounds
      auto item_at = [&] {
#ifdef QEVICT_DEBUG_BOUNDS  // the checking build has its positions fall
        return item_of<PAGED>(a, (int)gridDim.x - 1 - x, lane, &at, &before);
#else
        return item_of<PAGED>(a, x, lane, &at, &before);
#endif
      };
      auto hand_out = [&](const PromptItem& it) {
        if (put >= 2) ok = wait_item(b_taken + 8 * (put & 1), (uint32_t)((put >> 1) - 1) & 1u);
        if (ok && lane == 0) {
          items[put & 1] = it;
          bar_arrive(b_item + 8 * (put & 1));
        } else if (!ok && lane == 0) {
          items[2] = it;
        }
        ++put;
      };
      if (PAGED && a.by_range) {
        checks = blockIdx.x == 0;
        if (a.cuts && lane == 0) a.cuts[blockIdx.x].valid = 0;
        PagedRange range(a, lane);
        PromptItem it;
        while (ok && range.next(a, lane, lane == 0, &it)) {
          it.before = k_tiles;
          k_tiles += it.n - it.lo;
          hand_out(it);
          __syncwarp();
        }
      } else
      for (uint32_t ask = 0;; ++ask) {
        if (lane == 0) {
          words[8] = ask + 1;
          bar_expect(b_next, 16);
          asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                           smem_u32((void*)words)), "r"(b_next) : "memory");
        }
        checks = checks || x == 0;
        PromptItem it = item_at();
        if (it.valid) {
          if (PAGED) {
            it.before = k_tiles;
            k_tiles += it.n - it.lo;
          }
          hand_out(it);
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
          if (seq_cut<PAGED>(a, s)) kv8_record(a.status, CHECK_LENGTH);
      }
    } else if (wid == LOAD_WARP) {
      int slot = 0, q_turn = 0, issued = 0;
      uint32_t phase = 0;
      while (const PromptItem* item = next_item()) {
        const PromptItem& it = *item;
        const int cs = a.padded ? it.s : 0, hk = it.h0 / (a.Hq / a.Hkv);
        const bool pair = PAGED && it.pair;
        const int c0 = pair ? it.cnt(0) : it.n - it.lo, c1 = pair ? it.cnt(1) : 0;  // key tiles of the (two) streams
        if (c0 == 0) continue;
        auto load_q = [&] {
          if (q_turn > 0) ok = wait_item(b_qe, (uint32_t)(q_turn - 1) & 1u);
          ++q_turn;
          if (ok && lane == 0) {
            const int two = (it.cnt(0) > 0) + (!pair && it.cnt(1) > 0);
            bar_expect(b_q, (uint32_t)two * (uint32_t)(a.T * a.P * D * 2));
#pragma unroll
            for (int w = 0; w < 2; ++w)
              if (it.cnt(w) > 0 && !(pair && w))
                for (int x = 0; x < D / 64; ++x)
                  tma_load(smb + SM::Q_OFF + w * SM::TILE_BYTES + x * SM::HALF, &mq, b_q, x * 64, it.q0 + it.r0 + w * a.T, it.h0, cs);
            words[7] = (uint32_t)q_turn;
          }
        };
        if (!PAGED) load_q();
        int k_tiles = it.before;
        int v_slot = 0;
        uint32_t v_phase = 0;
        bool clean = it.dirty(), v_seen = false;
        // Paged: 32 page ids of each stream, one per lane, and the 32 below them on their way.  A block that is not there has a
        // page behind the last one: the copy then writes zeros.
        const int per_log2 = 7 - a.block_log2;  // blocks of a tile
        const int blocks = PAGED ? (it.nk + (1 << a.block_log2) - 1) >> a.block_log2 : 0;
        int window[2] = {0, 0}, id[2] = {0, 0}, ahead[2] = {0, 0};
        auto fetch = [&](int win) {
          const int b = win * 32 + lane;
          return win >= 0 && b < blocks ? a.table[(size_t)it.s * a.max_blocks + b] : -1;
        };
        auto look = [&](int p) {  // a page id, or the place of none
          if (p >= 0 && p < a.n_pages) return p;
          if (p != -1) kv8_record(a.status, CHECK_PAGE_ID);
          return a.n_pages;
        };
        if (PAGED) {
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            window[w] = (((w ? it.mid : it.n) - 1) << per_log2) >> 5;
            if (w == 0 || c1 > 0) {
              id[w] = fetch(window[w]);
              ahead[w] = fetch(window[w] - 1);
            }
          }
          id[0] = look(id[0]);
          if (c1 > 0) id[1] = look(id[1]);
        }
        auto issue = [&](int w, bool value, int j) {  // the next slot of the ring: K or V of key tile j (of stream w)
          if (!ok) return;
          if (issued >= NS) ok = wait_item(b_empty + 8 * slot, phase ^ 1u);
          const uint32_t dst = smb + SM::KV_OFF + slot * SM::TILE_BYTES, bar = b_full + 8 * slot;
          if constexpr (PAGED) {
            const int first = j << per_log2;
            if ((first >> 5) != window[w]) {
              window[w] = first >> 5;
              id[w] = look(ahead[w]);
              ahead[w] = fetch(window[w] - 1);
            }
            const uint32_t none = __ballot_sync(0xffffffffu, id[w] == a.n_pages && window[w] * 32 + lane < blocks);
            const int i = lane & ((1 << per_log2) - 1), x = lane >> per_log2;
            const int page = __shfl_sync(0xffffffffu, id[w], (first & 31) + i);
            if (ok && lane == 0) {
              if (!value) masks[k_tiles & 15] = (uint8_t)((none >> (first & 31)) & ((1u << (1 << per_log2)) - 1u));
              bar_expect(bar, SM::TILE_BYTES);
              words[5] = issued + 1;
            }
            __syncwarp();
            if (ok && x < a.boxes)
              tma_page(dst + x * SM::HALF + i * (a.group_bytes << (a.block_log2 - 3)), value ? &mv : &mk, bar, x * 64,
                       hk * (value ? a.head_step[1] : a.head_step[0]), page);
            k_tiles += !value;
          } else if (ok && lane == 0) {
            bar_expect(bar, SM::TILE_BYTES);
            for (int x = 0; x < D / 64; ++x)
              tma_load(dst + x * SM::HALF, value ? &mv : &mk, bar, x * 64, it.k0 + j * TILE, hk, cs);
            words[5] = issued + 1;
          }
          ++issued;
          if (value && !v_seen) { v_slot = slot; v_phase = phase; v_seen = true; }
          if (++slot == NS) { slot = 0; phase ^= 1u; }
          __syncwarp();
        };
        auto zero_tail = [&] {  // zero the value rows past the end
          clean = false;
          ok = ok && wait(b_full + 8 * v_slot, v_phase);
          const int from = it.nk - (it.n - 1) * TILE, per = (TILE - from) * 8;
          if (ok) {
            unsigned char* v0 = sm + SM::KV_OFF + v_slot * SM::TILE_BYTES;
            for (int k = lane; k < per * (D / 64); k += 32) {
              const int x = k / per, row = from + ((k - x * per) >> 3), at = (k - x * per) & 7;
              const int to = PAGED ? (row >> 3) * a.group_bytes + x * a.half_bytes + (row & 7) * 128 : row * 128 + x * SM::HALF;
              *reinterpret_cast<uint4*>(v0 + to + at * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(b_clean);
          }
          __syncwarp();
        };
        // K, V of the last tile, K, V of the one before, ...; those of two streams in turn, in the order of their products.  (The
        // queries' place is free when the last item's last S is done: its first keys need not wait for that.)
        issue(0, false, it.n - 1);
        if (PAGED) load_q();
        if (c1 > 0) issue(1, false, it.mid - 1);
        for (int i = 0; i < c0 && ok; ++i) {
          issue(0, true, it.n - 1 - i);
          if (i + 1 < c0) issue(0, false, it.n - 2 - i);
          if (clean) zero_tail();
          if (i < c1) issue(1, true, it.mid - 1 - i);
          if (i + 1 < c1) issue(1, false, it.mid - 2 - i);
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
      const uint32_t q_lo = desc_lo(u_sm + SM::Q_OFF, 16), k_lo = desc_lo(u_sm + SM::KV_OFF, 16), v_lo = desc_lo(u_sm + SM::KV_OFF, PAGED ? (uint32_t)a.half_bytes : SM::HALF);
      const uint32_t kv_hi = PAGED ? ((uint32_t)a.group_bytes >> 4) | (DESC_HI & ~0x3fffu) : DESC_HI;
      const uint32_t k_half = PAGED ? (uint32_t)a.half_bytes : SM::HALF, v_step = PAGED ? (uint32_t)a.group_bytes * 2 : 2048u;
      const uint32_t ub = u_sm + SM::BAR_OFF, u_full = ub + 8, u_empty = u_full + 8 * NS, u_s = u_empty + 8 * NS, u_p = u_s + 16, u_o = u_p + 16;
      leader = elect_one();
      // Half of the products of S, a look at the other tile's P, the other half: the look's latency passes while the tensor
      // cores have work.  (A wait costs this warp some 90 cycles even when there is nothing to wait for, and the queue
      // of products is short: with the waits between the products the call took 7 % longer.)
      bool seen = false;
      auto issue_s = [&](int w, int slot, uint32_t other_phase, int rows) {
        const uint32_t qa = q_lo + rows * (SM::TILE_BYTES >> 4), ka = k_lo + slot * (SM::TILE_BYTES >> 4);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          if (leader) {
#pragma unroll
            for (int ks = part * (D / 32); ks < (part + 1) * (D / 32); ++ks) {
              const uint32_t o = ((uint32_t)(ks >> 2) * SM::HALF + (ks & 3) * 32) >> 4;
              if constexpr (PAGED)
                mma_ss(u_tm + w * 128, qa + o, ka + (((uint32_t)(ks >> 2) * k_half + (ks & 3) * 32) >> 4), id_s, ks > 0, kv_hi);
              else
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
            mma_ts(u_tm + 256 + w * 128, u_tm + w * 128 + P_COL(ks >> 2, ks & 3), va + ks * (v_step >> 4), id_o, ks > 0 ? 1u : acc, kv_hi);
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
        if constexpr (PAGED) {
          if (uniform(it.pair)) {
            // two streams of key tiles against the same rows: S0 S1 | PV0 S0 PV1 S1 | ..., a slot of the ring for each product
            const int u_mid = uniform(it.mid), c[2] = {u_n - u_mid, u_mid - u_lo};
            uint32_t acc[2] = {0u, 0u};
            seen = false;
            auto step_s = [&](int w) {  // S of stream w from the next slot, which holds its keys
              issue_s(w, slot, w ? phase0 : phase1, 0);
              if (leader) commit_to(u_empty + 8 * slot);
              __syncwarp();
              if (++slot == NS) { slot = 0; phase ^= 1u; }
            };
            step_s(0);
            if (c[1] > 0) {
              if (!(ok = wait(u_full + 8 * slot, phase))) break;
              step_s(1);
            }
            seen = false;
            if (c[0] == 1 && leader) commit_to(b_qe);
            __syncwarp();
            for (int i = 0; i < c[0] && ok; ++i) {
#pragma unroll
              for (int w = 0; w < 2; ++w) {
                if (i >= c[w]) {
                  seen = false;
                  continue;
                }
                const int sv = slot;
                ok = wait(u_full + 8 * sv, phase);
                if (++slot == NS) { slot = 0; phase ^= 1u; }
                if (ok && w == 0 && i == 0 && dirty) {
                  ok = wait(b_clean, clean_phase);
                  clean_phase ^= 1u;
                }
                const bool more = i + 1 < c[w];
                if (more) ok = ok && wait(u_full + 8 * slot, phase);
                ok = ok && p_ready(w, w ? phase1 : phase0);
                if (!ok) break;
                tm_after();
                issue_o(w, sv, acc[w]);
                acc[w] = 1u;
                if (w) phase1 ^= 1u; else phase0 ^= 1u;
                if (leader) {
                  commit_to(u_empty + 8 * sv);
                  if (!more) commit_to(u_o + 8 * w);
                }
                __syncwarp();
                if (more) step_s(w);
              }
              if (ok && i + 2 == c[0]) {  // the last S
                if (leader) commit_to(b_qe);
                __syncwarp();
              }
            }
            seen = false;
            if (!ok) break;
            continue;
          }
        }
        if (u_n - 1 < u_n0) issue_s(0, slot, phase1, 0);
        if (u_n - 1 < u_n1) issue_s(1, slot, phase0, 1);
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
          if (more && j - 1 < u_n0) issue_s(0, slot, phase1, 0);
          if (j < u_n1) {
            if (!(ok = p_ready(1, phase1))) break;
            tm_after();
            issue_o(1, sv, acc1);
            acc1 = 1u;
            phase1 ^= 1u;
            if (!more && leader) commit_to(u_o + 8);
          }
          if (more && j - 1 < u_n1) issue_s(1, slot, phase0, 1);
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
    const uint32_t lane_base = (uint32_t)((wid & 3) * 32) << 16;
    const uint32_t ts = tmem + lane_base + w * 128, to = tmem + lane_base + 256 + w * 128 + half * (D / 2);
    // What a row needs once for each item is made anew each time, from a thread index that the compiler cannot keep: the registers are
    // the logits', and what waits for its turn in local memory comes from the L2 (shared memory leaves the L1 little).
    struct Row {
      int w, half, r, hl, row;  // tile, half of the keys and channels, row of the tile, head and token
      bool mine;                // rows of nobody hold anything, and have no say below
    };
    auto row_of = [&](const PromptItem& it) {
      uint32_t t;
      asm volatile("mov.u32 %0, %%tid.x;" : "=r"(t));
      Row x;
      x.w = t >> 8;
      x.half = (t >> 7) & 1;
      x.r = t & 127;
      x.hl = x.r / a.T;
      x.row = it.r0 + (PAGED && it.pair ? 0 : x.w * a.T) + x.r - x.hl * a.T;
      x.mine = x.row < it.nq && x.hl < a.P;
      return x;
    };
    float* xch = reinterpret_cast<float*>(sm + SM::BAR_OFF + SM::ROWS) + w * 2 * TILE + r;  // the two halves' values of a row
    auto meet = [&] {
      uint32_t both;
      asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}\n"
                   : "=r"(both) : "r"((uint32_t)ok), "r"(1 + w * 4 + (wid & 3)) : "memory");
      ok = both != 0;
    };
    uint32_t s_phase = 0, o_phase = 0, quad_phase = 0;
    // The four warps that share a pair's rows meet at a barrier with a bounded wait, which ends too when another tile's warps have given
    // up; the two that share a tile then agree.
    auto meet4 = [&] {
      tm_before();
      __syncwarp();
      if (lane == 0) bar_arrive(b_quad + 8 * (wid & 3));
      ok = ok && wait_item(b_quad + 8 * (wid & 3), quad_phase);
      quad_phase ^= 1u;
      tm_after();
      meet();
      return ok;
    };
    while (true) {
      const PromptItem* item = next_item();
      meet();
      if (!ok || !item) break;
      const PromptItem& it = *item;
      const int cnt = it.cnt(w);
      int left;  // keys that this row still sees from the tile's (this half's) first on; grows by a tile each time
      bool mine;
      {
        const Row x = row_of(it);
        left = (a.causal ? min(it.nk, x.row + it.nk - it.nq + 1) : it.nk) - ((w ? it.nt1 : it.nt0) - 1) * TILE - half * (TILE / 2);
        mine = x.mine;
      }
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
          if constexpr (PAGED) {
            // (read from the item each time: the registers are the logits')
            const volatile PromptItem& v = it;
            const uint32_t none = masks[(v.pair ? v.before + w + 2 * (cnt - i) : v.before + v.n - i - (w ? v.nt1 : v.nt0) + cnt) & 15];
            if (none) {  // blocks that are not there, 16 keys at a time
#pragma unroll
              for (int c = 0; c < TILE / 2; ++c)
                if ((none >> ((half * (TILE / 2) + (c & ~15)) >> a.block_log2)) & 1u) x[c] = -INFINITY;
            }
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
        const float top_x = fmaxf(xch[0], xch[TILE]) * a.scale_log2 - P_UP<T>;
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
      float f0 = 1.f, f1 = 0.f;  // factors of the outputs
      if constexpr (PAGED) {
        if (it.pair) {
          // both tiles' sums of the same rows: four warps share them, a quarter of the channels each
          if (!(ok = meet4())) break;
          xch[half * TILE] = half ? l : m;
          if (!(ok = meet4())) break;
          const float* both = xch - w * 2 * TILE;
          const float m0 = both[0], m1 = both[2 * TILE];
          m = fmaxf(m0, m1);
          f0 = m == -INFINITY ? 0.f : ex2p(m0 - m);
          f1 = m == -INFINITY ? 0.f : ex2p(m1 - m);
          l = both[TILE] * f0 + both[3 * TILE] * f1;
        }
      }
      {
        const Row x = row_of(it);
        const bool pair = PAGED && it.pair, partial = PAGED ? it.slot >= 0 : a.splits > 1, none = l == 0.f;
        const int hq = it.h0 + x.hl, c0 = pair ? (2 * x.w + x.half) * (D / 4) : x.half * (D / 2);
        const long long prow = a.padded ? (long long)it.s * a.max_q + x.row : (long long)it.q0 + x.row;
        const long long place = PAGED ? (long long)it.slot * a.slot_rows + (pair ? 0 : x.w * TILE) + x.r : ((long long)it.split * a.rows + prow) * a.Hq + hq;
        const float lse2 = none ? -INFINITY : m + log2f(l), inv = none ? 0.f : 1.f / l;
        if (x.mine && c0 == 0) {
          if (partial)
            a.part_lse[place] = lse2;
          else if (a.lse)
            a.lse[a.padded ? ((long long)it.s * a.Hq + hq) * a.max_q + x.row : hq * (PAGED ? a.lse_rows : a.total_q) + prow] = lse2 * 0.6931471805599453f;
        }
        f0 *= inv;
        f1 *= inv;
        const bool first = pair || cnt > 0, second = pair && it.cnt(1) > 0;  // tiles with products (warp-uniform)
        const uint32_t from = words[4] + (uint32_t)((x.r & 96) << 16) + 256 + (pair ? 0 : x.w * 128) + c0;
        // where 16 bytes of the row go, and from one such piece to the next
        unsigned char* to_row;
        long long step = 16;
        if (!partial) {
          to_row = reinterpret_cast<unsigned char*>(static_cast<T*>(a.out) + (a.padded ? it.s * a.out_stride[0] + x.row * a.out_stride[2] : prow * a.out_stride[2]) +
                                                    hq * a.out_stride[1] + c0);
        } else if (PAGED) {
          to_row = reinterpret_cast<unsigned char*>(part_at<D>(a, it.slot, c0, (pair ? 0 : x.w * TILE) + x.r));
          step = 16ll * a.slot_rows;
        } else {
          to_row = reinterpret_cast<unsigned char*>(a.part_o + place * D + c0);
        }
#pragma unroll 1
        for (int c = 0; c < (pair ? D / 4 : D / 2); c += 16) {
          float o[16];
          if (first) {
            tm_ld16(from + c, o);
            if (PAGED && second) {
              float o1[16];
              tm_ld16(from + 128 + c, o1);
              tm_wait_ld();
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] = o[k] * f0 + o1[k] * f1;
            } else {
              tm_wait_ld();
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] *= f0;
            }
          }
          if (x.mine) {
#pragma unroll
            for (int k = 0; k < 16; ++k) o[k] = none ? 0.f : o[k];
            if (partial) {
#pragma unroll
              for (int k = 0; k < 16; k += 4) *reinterpret_cast<float4*>(to_row + (k >> 2) * step) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
              to_row += 4 * step;
            } else {
#pragma unroll
              for (int k = 0; k < 16; k += 8)
                *reinterpret_cast<uint4*>(to_row + 2 * k) = make_uint4(pack2<T>(o[k], o[k + 1]), pack2<T>(o[k + 2], o[k + 3]), pack2<T>(o[k + 4], o[k + 5]), pack2<T>(o[k + 6], o[k + 7]));
              to_row += 32;
            }
          }
          __syncwarp();
        }
        if constexpr (PAGED) {
          if (pair && !(ok = meet4())) break;  // the next item's first products overwrite both
        }
      }
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
    // were handed out last and the two that were not.  Of a range, all.
    auto lose = [&](const PromptItem& it, int first, int step) {
      for (int i = first; it.valid && i < 2 * a.T * a.P; i += step) {
        const int row = it.r0 + i / a.P, hl = i % a.P, hq = it.h0 + hl;
        if (row >= it.nq) break;
        const long long prow = a.padded ? (long long)it.s * a.max_q + row : (long long)it.q0 + row;
        if (PAGED ? it.slot >= 0 : a.splits > 1) {  // as a weight, it makes the merged row that
          const int w = (row - it.r0) / a.T;
          a.part_lse[PAGED ? (long long)it.slot * a.slot_rows + w * TILE + hl * a.T + row - it.r0 - w * a.T
                           : ((long long)it.split * a.rows + prow) * a.Hq + hq] = NAN;
          continue;
        }
        if (a.lse) a.lse[a.padded ? ((long long)it.s * a.Hq + hq) * a.max_q + row : hq * (PAGED ? a.lse_rows : a.total_q) + prow] = NAN;
        T* out = static_cast<T*>(a.out) + (a.padded ? it.s * a.out_stride[0] + row * a.out_stride[2] : prow * a.out_stride[2]) + hq * a.out_stride[1];
        for (int c = 0; c < D; ++c) out[c] = Tr<T>::from_float(NAN);
      }
    };
    if (PAGED && a.by_range) {
      if (wid == ITEM_WARP) {
        PagedRange range(a, lane);
        PromptItem it;
        while (range.next(a, lane, lane == 0, &it)) lose(it, lane, 32);
      }
    } else {
      for (int n = 0; n < 4; ++n) lose(items[n], tid, PROMPT_THREADS);
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

// Paged: joins the partial results of the items that ranges share: blockIdx.y is the CTA in whose range such an item starts, a lane
// per row of 32, a warp per four channels of 64.  The warps look for the largest reference together, and many parts' rows are
// requested at a time (one long sequence may have 60 parts: one after the other they took 13 us).
constexpr int MERGE_WARPS = 16;
template <class T, int D>
__global__ void __launch_bounds__(32 * MERGE_WARPS) paged_merge_kernel(const PromptArgs a) {
  __shared__ float red[MERGE_WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane, c4 = blockIdx.z * 64 + warp * 4, cta = blockIdx.y;
  pdl_prologue();
  const PagedCut c = a.cuts[cta];
  if (!c.valid) return;  // the whole CTA leaves
  const int w = i / TILE, r = i - w * TILE, hl = r / a.T, tok = w * a.T + r - hl * a.T;
  const bool mine = hl < a.P && c.r0 + tok < c.nq && !(c.pair && w);
  const int parts = c.last - cta + 1;
  // part 0 ends its CTA's range, the others begin theirs
  auto slot = [&](int p) { return 2 * (cta + p) + (p == 0); };
  auto lse_of = [&](int p) { return a.part_lse[(long long)slot(p) * a.slot_rows + i]; };
  float top = -INFINITY;
  if (mine)
    for (int p = warp; p < parts; p += MERGE_WARPS) {
      const float x = lse_of(p);
      top = x != x || top != top ? NAN : fmaxf(top, x);  // not a number: the part was given up
    }
  red[warp][lane] = top;
  __syncthreads();
  if (!mine) return;
#pragma unroll
  for (int k = 0; k < MERGE_WARPS; ++k) {
    const float x = red[k][lane];
    top = x != x || top != top ? NAN : fmaxf(top, x);
  }
  const float ref = top == -INFINITY ? 0.f : top;
  float sum = 0.f, y[4] = {};
#pragma unroll 8
  for (int p = 0; p < parts; ++p) {
    const float f = ex2p(lse_of(p) - ref);
    const float4 v = *part_at<D>(a, slot(p), c4, i);
    sum += f;
    y[0] += f * v.x;
    y[1] += f * v.y;
    y[2] += f * v.z;
    y[3] += f * v.w;
  }
  const bool none = sum == 0.f;
  const float inv = none ? 0.f : 1.f / sum;
#pragma unroll
  for (int k = 0; k < 4; ++k) y[k] = none ? 0.f : y[k] * inv;
  const long long prow = (long long)c.q0 + c.r0 + tok;
  const int hq = c.h0 + hl;
  *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + prow * a.out_stride[2] + hq * a.out_stride[1] + c4) =
      make_uint2(pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3]));
  if (c4 == 0 && a.lse) a.lse[hq * a.lse_rows + prow] = none ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeFn encode_fn() {
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
inline bool make_map(CUtensorMap* map, int dtype, const void* base, int D, long long tokens, int heads, long long seqs, const int64_t* stride,
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
inline void prompt_tile(int G, int* P, int* T) {
  *P = G < 32 ? G : 32;
  while (G % *P) --*P;
  *T = TILE / *P;
}

// Most tile pairs that the sequences can have, for one group of heads: with max_q rows each, or total_q rows cut anywhere.
inline long long prompt_tiles(bool padded, int n_seqs, long long max_q, long long total_q, int T) {
  const long long each = n_seqs * ((max_q + 2 * T - 1) / (2 * T)), all = total_q / (2 * T) + n_seqs;
  return padded || each < all ? each : all;
}

inline int prompt_sms(int device) {
  int n = 0;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) {
    (void)cudaGetLastError();
    n = SM_COUNT_FALLBACK;
  }
  return n;
}

}  // namespace

}  // namespace qevict
