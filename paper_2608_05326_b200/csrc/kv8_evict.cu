// One-way eviction from the 8-bit cache by accumulated attention mass.
//
// One CTA per sequence.  Scores become 32-bit keys that order like them (NaN lowest, -0 equal to 0); the key of the
// last block that is kept among the candidates comes from a radix selection (four 8-bit digits, histograms in shared
// memory); blocks above it stay, and of those equal to it the first ones in block order do.  A scan over the CTA for each
// 1024 blocks turns the decisions into places (a second one where only some of the equal ones stay).  The data are a few
// tens of KB per sequence: the launch, the dependent steps and fetching code that runs once are all the time there is, so the
// loops stay rolled.  (16 sequences of 8192 blocks: 17 us; keys in registers with unrolled rounds and counts against
// thresholds in place of the histograms took 23 us, a run of consecutive blocks per thread 25 us: its stores scatter.)
#include "kv8.cuh"

namespace qevict {

namespace {

constexpr int EVICT_THREADS = 1024;
constexpr int EVICT_MAX_BLOCKS = 16384;

__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);  // -0 + 0 = +0
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Exclusive prefix sums over the CTA of two counts packed in one word (16 bits each: at most 1024 of each), and their
// totals.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* s_warp, uint32_t* total) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  uint32_t v = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += y;
  }
  if (lane == 31) s_warp[wid] = v;
  __syncthreads();
  const int nw = blockDim.x >> 5;
  uint32_t w = lane < nw ? s_warp[lane] : 0u;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  *total = __shfl_sync(0xffffffffu, w, 31);
  const uint32_t before = wid ? __shfl_sync(0xffffffffu, w, wid - 1) : 0u;
  __syncthreads();
  return before + v - x;
}

__global__ void __launch_bounds__(EVICT_THREADS) kv8_evict_kernel(const qevict_kv8_evict_args a) {
  extern __shared__ uint32_t s_key[];  // [max_blocks] keys, then [max_blocks] page ids, then [max_blocks] scores
  const int mb = a.max_blocks, s = blockIdx.x, tid = threadIdx.x, nt = blockDim.x, lane = tid & 31;
  int32_t* s_page = reinterpret_cast<int32_t*>(s_key + mb);
  float* s_score = reinterpret_cast<float*>(s_page + mb);
  __shared__ uint32_t hist[256], s_warp[32], s_pick[3];
  pdl_prologue();
  const size_t row = (size_t)s * mb;
  const int len = a.lens[s];
#pragma unroll 4
  for (int i = tid; i < mb; i += nt) {  // everything is read before anything is written: the outputs may be the inputs
    const float x = a.scores[row + i];
    s_score[i] = x;
    s_key[i] = order_key(x);
    s_page[i] = a.table[row + i];
  }
  const int full = min(max(len, 0) / a.block, mb);
  const bool over = full > a.budget;
  const int c0 = a.sink, c1 = full - a.recent;                // candidates
  const int want = a.budget - a.sink - a.recent;              // of them stay
  uint32_t cut = 0xffffffffu;  // candidates with a larger key stay,
  int ties = 0;                // and the first `ties` with this key,
  bool all_ties = true;        // which may be all of them
  __syncthreads();
  if (over && want > 0) {
    uint32_t prefix = 0, mask = 0;
    int left = want;
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += nt) hist[i] = 0;
      __syncthreads();
      for (int i = c0 + tid; i < c1; i += nt) {
        const uint32_t k = s_key[i];
        if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (tid < 32) {  // lane l takes the digits 255 - 8 l .. 248 - 8 l
        uint32_t mine[8], sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) { mine[j] = hist[255 - 8 * lane - j]; sum += mine[j]; }
        uint32_t inc = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += y;
        }
        uint32_t run = inc - sum;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (run < (uint32_t)left && run + mine[j] >= (uint32_t)left) {
            s_pick[0] = 255 - 8 * lane - j;
            s_pick[1] = run;
            s_pick[2] = mine[j];
          }
          run += mine[j];
        }
      }
      __syncthreads();
      prefix |= s_pick[0] << shift;
      mask |= 255u << shift;
      left -= (int)s_pick[1];
      all_ties = left == (int)s_pick[2];
      __syncthreads();
    }
    cut = prefix;
    ties = left;
  }
  // places, `nt` entries at a time
  int n_keep = 0, n_free = 0, n_tie = 0;
#pragma unroll 1
  for (int base = 0; base < mb; base += nt) {
    const int i = base + tid;
    const bool in = i < mb, cand = in && over && i >= c0 && i < c1;
    const uint32_t k = cand ? s_key[i] : 0u;
    const bool tie = cand && want > 0 && k == cut;
    uint32_t total;
    bool keep = in && (!cand || (want > 0 && k > cut) || (tie && all_ties));
    if (!all_ties) {
      const uint32_t tb = block_scan(tie ? 1u : 0u, s_warp, &total);
      keep = keep || (tie && n_tie + (int)tb < ties);
      n_tie += (int)total;
    }
    const int page = in ? s_page[i] : -1;
    const bool gone = in && !keep, listed = gone && page >= 0 && page < a.n_pages;
    const uint32_t at = block_scan((keep ? 1u : 0u) | (listed ? 0x10000u : 0u), s_warp, &total);
    if (keep) {
      const size_t to = row + n_keep + (at & 0xffffu);
      a.table_out[to] = page;
      a.scores_out[to] = s_score[i];
      if (a.kept) a.kept[to] = i;
    }
    if (listed && a.freed) a.freed[row + n_free + (at >> 16)] = page;
    n_keep += (int)(total & 0xffffu);
    n_free += (int)(total >> 16);
  }
  for (int i = n_keep + tid; i < mb; i += nt) {
    a.table_out[row + i] = -1;
    a.scores_out[row + i] = 0.f;
    if (a.kept) a.kept[row + i] = -1;
  }
  if (a.freed)
    for (int i = n_free + tid; i < mb; i += nt) a.freed[row + i] = -1;
  if (tid == 0) {
    a.lens_out[s] = len - (mb - n_keep) * a.block;
    if (a.n_freed) a.n_freed[s] = n_free;
  }
}

}  // namespace

}  // namespace qevict

using namespace qevict;

extern "C" QEVICT_API qevict_status qevict_kv8_evict(const qevict_kv8_evict_args* p, void* stream) {
  auto bad = [](const char* msg) { return stateless_fail(QEVICT_ERR_INVALID_ARG, msg); };
  if (!p) return bad("args is NULL");
  if (p->struct_size != sizeof(qevict_kv8_evict_args)) return bad("struct_size does not match this library's qevict_kv8_evict_args");
  if (p->device < 0) return bad("device must be >= 0");
  if (p->n_seqs < 0 || p->max_blocks < 1 || p->block < 1 || p->n_pages < 0)
    return bad("n_seqs and n_pages must be >= 0, max_blocks and block >= 1");
  if (p->budget < 0 || p->sink < 0 || p->recent < 0 || (long long)p->sink + p->recent > p->budget)
    return bad("sink and recent must be >= 0 and their sum at most budget");
  if (p->max_blocks > EVICT_MAX_BLOCKS) return stateless_fail(QEVICT_ERR_UNSUPPORTED, "more than 16384 blocks per sequence");
  if (p->n_seqs == 0) return QEVICT_OK;
  if (!p->table || !p->lens || !p->scores || !p->table_out || !p->lens_out || !p->scores_out)
    return bad("table, lens, scores and their outputs must not be NULL");
  if ((p->freed == nullptr) != (p->n_freed == nullptr)) return bad("freed and n_freed go together");
  if (misaligned4(p->table) || misaligned4(p->lens) || misaligned4(p->scores) || misaligned4(p->table_out) || misaligned4(p->lens_out) ||
      misaligned4(p->scores_out) || misaligned4(p->kept) || misaligned4(p->freed) || misaligned4(p->n_freed))
    return bad("arrays must be 4-byte aligned");
  DeviceGuard guard(p->device);
  cudaError_t e = guard.err;
  const size_t smem = (size_t)p->max_blocks * 12;
  static std::atomic<uint64_t> done{0};
  if (e == cudaSuccess && smem > 40 * 1024)
    e = once_per_device(done, p->device, [] { return cudaFuncSetAttribute(kv8_evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, EVICT_MAX_BLOCKS * 12); });
  int nt = 128;  // a thread per entry up to 1024 threads
  while (nt < p->max_blocks && nt < EVICT_THREADS) nt <<= 1;
  if (e == cudaSuccess) e = launch_pdl(kv8_evict_kernel, dim3(p->n_seqs), dim3(nt), smem, (cudaStream_t)stream, *p);
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  return QEVICT_OK;
}
