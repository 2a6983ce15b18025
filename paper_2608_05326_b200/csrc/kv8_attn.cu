// Attention of one token per sequence over the 8-bit block-scaled cache.
//
//     x_i = scale * q . (s_b c_i) * log2 e,  out = sum_i 2^(x_i - M) s'_b c'_i / L,  L = sum_i 2^(x_i - M)
//     mass_b = sum_heads sum_{i in b} 2^(x_i - M) / L
// The codes are read once (one byte per element, keys and values); everything else is small, so HBM bounds the call.
//
// Work.  The cache of a call is a sequence of units of UT tokens (32, or 16 where a block has 16), ordered by
// (sequence, KV head, token).  Every warp of the grid takes one contiguous run of them, equal to within one unit, so
// ragged lengths balance without a plan on the host: each CTA sums the lengths itself.  A warp's part of a
// (sequence, KV head) is one partial result; run w's part of row r is slot w + r of the scratch (both only grow along
// the order, so slots are distinct); where a row's slots lie is written down for kv8_merge_kernel.
//
// Tile.  Both products put the cache on the A side of mma.m16n8k16 (tokens, then channels on M; the G heads that
// share the KV head on N).  Codes become fp16 operands in registers, exactly, and the block's scale multiplies the logits /
// the block's output in float32.  The contraction index may be permuted as long as both sides agree, so a lane takes whole
// 4-byte words of its key row, and the token pairs of the values come out of byte permutes.  The query goes to fp16 after a division by a power of two per head, which brings its largest
// element into [1, 2): exact but for elements 2^-14 below the largest, which lose at most 2^-25 of it.
// Probabilities enter the second product as fp16 (2^-11); the sums of the softmax, the block masses and the output
// are float32.
//
// Measured: 16 ragged contexts of up to 32768 tokens, 32 / 8 heads of 128, int8 (472 MB): 103 us, of which this kernel 90 us
// (5.2 TB/s; the copies without arithmetic 82 us), merge and masses the rest; 8 contexts of 65536, 28 / 4 heads, e4m3 (538 MB):
// 108 us; one of 2048 tokens: 9.2 us, two dependent launches.  At 6.45 TB/s the bytes alone would take 73, 83 and 0.7 us.
#include <cuda.h>

#include "kv8.cuh"

namespace qevict {

namespace {

constexpr int WARPS = 4;                  // warps per CTA
constexpr int ATTN_THREADS = WARPS * 32;
constexpr int RING_BYTES = 16384;         // of a warp (d = 128): stages of one unit's keys or values
constexpr float LAZY = 8.f;               // the reference exponent moves only when a logit exceeds it by this (log2)

struct Kv8AttnArgs {
  Kv8View c;
  int Hq, G;
  float scale_log2;
  const void* q;
  const int32_t* lens;
  int max_len;     // already cut to max_blocks * block
  int n_warps;     // warps of the attention grid
  int max_units;   // units of a sequence of max_len tokens
  int least_run;   // units of a run, where there are runs enough
  void* out;
  float* lse;
  const float* score_in;
  float* score_out;
  float* part_o;   // [slot][G][D]
  float2* part_ml; // [slot][G] {reference, sum}
  int2* rows;      // [seq][Hkv] first slot and number of the row's partial results
  float2* rec;     // [seq][max_units][Hq] {reference, sum} of every unit, or nullptr
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}

// Codes as fp16 operands.  int8: code + 128 as a subnormal fp16, 2^-24 per unit (exact, and the tensor cores take
// subnormals): one masking instruction for two codes, against three for code values proper.  The 128 comes off in the
// accumulator's start value: -128 sum q for the logits, -128 sum p (a product with ones, over the same rounded p) for the
// output.  The sums have terms of at most 255 instead of 127 units, which doubles their rounding errors (2^-24 of the
// largest partial sum) and no more.  e4m3: the conversion instruction.
template <int CODE> struct Unit { static constexpr float value = CODE == QEVICT_CODE_INT8 ? 0x1p24f : 1.f; };
// a word of four codes c0 c1 c2 c3 -> operand registers for the pairs {c0, c2}, {c1, c3} (int8) or {c0, c1}, {c2, c3} (e4m3)
template <int CODE> __device__ __forceinline__ void codes_to_h2(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (CODE == QEVICT_CODE_INT8) {
    asm("lop3.b32 %0, %1, 0x00ff00ff, 0x00800080, 0x6A;\n" : "=r"(lo) : "r"(w));  // (w & mask) ^ sign bits
    asm("lop3.b32 %0, %1, 0x00ff00ff, 0x00800080, 0x6A;\n" : "=r"(hi) : "r"(w >> 8));
  } else {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}\n"
        : "=r"(lo), "=r"(hi) : "r"(w));
  }
}
// which code of a lane's word meets element j of its k-step's operand (0, 1 in the first register, 2, 3 in the second)
template <int CODE> __device__ __forceinline__ constexpr int code_at(int j) {
  return CODE == QEVICT_CODE_INT8 ? (j & 1) * 2 + (j >> 1) : j;
}

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
  return y;
}

// Tokens of a sequence that the call sees: a length beyond the bound is cut to the whole blocks within it (a partial
// one would be in the tail, and the tail holds later tokens).
__device__ __forceinline__ int clamp_len(const Kv8AttnArgs& a, int len) {
  return len <= a.max_len ? max(0, len) : a.max_len / a.c.block * a.c.block;
}

// The kernels of a call follow one another by programmatic launch.  The attention kernel lets the next one start only when
// a warp has nothing left to read: its own CTAs fill the SMs, and CTAs of the next kernel that slipped in between cost a
// second wave (16 ragged contexts: 104 us, 117 with the release at the start).  The merge releases nothing early for the same
// reason.
__device__ __forceinline__ void wait_prior() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }
__device__ __forceinline__ void release_next() { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); }

// Prefix sums of the sequences' units per KV head, in shared memory.
__device__ void unit_prefix(const Kv8AttnArgs& a, int ut, int* pre, int* s_w) {
  const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, wid = tid >> 5;
  int base = 0;
  for (int s0 = 0; s0 < a.c.n_seqs; s0 += nt) {
    const int s = s0 + tid;
    int x = s < a.c.n_seqs ? (clamp_len(a, a.lens[s]) + ut - 1) / ut : 0;
    int v = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += y;
    }
    if (lane == 31) s_w[wid] = v;
    __syncthreads();
    int before = base, all = base;
    for (int i = 0; i < (nt >> 5); ++i) {
      if (i < wid) before += s_w[i];
      all += s_w[i];
    }
    if (s < a.c.n_seqs) pre[s] = before + v - x;
    base = all;
    __syncthreads();
  }
  if (tid == 0) pre[a.c.n_seqs] = base;
  __syncthreads();
}

// First unit of run w of n over `total` units; the run that holds unit u.  There are never more runs than units, so
// that no run is empty and every slot between a row's first and last is written; and where warps are plenty a run has
// least_run units, since every run's partial result has to be merged.
__device__ __forceinline__ int runs_of(long long total, int n_warps, int least_run) {
  return (int)min((long long)n_warps, (total + least_run - 1) / least_run);
}
__device__ __forceinline__ long long run_start(long long total, int n, int w) { return total * w / n; }
__device__ __forceinline__ int run_of(long long total, int n, long long u) { return (int)(((u + 1) * n - 1) / total); }

// sequence of unit u: the last s with pre[s] * Hkv <= u and units of its own
__device__ __forceinline__ int seq_of(const int* pre, int n_seqs, int u_per_head) {
  int lo = 0, hi = n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pre[mid] <= u_per_head) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Shared-memory byte offset of 16-byte chunk `c` of token row `r` of a tile, so that the 8 lanes of a load phase
// fall into different banks (rows of 128 bytes: chunk ^ row; rows of 64 bytes: two rows share a 128-byte line).
template <int D> __device__ __forceinline__ uint32_t swz(int r, int c) {
  if (D == 128) return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4));
  const int line = r >> 1, c8 = ((r & 1) << 2) | c;
  return (uint32_t)(line * 128 + ((c8 ^ ((line & 3) << 1)) << 4));
}

// One warp's running state for one (sequence, KV head).
template <int D, int NT> struct Acc {
  float o[NT][D / 16][4];  // output, channels x heads
  float m[NT][2], l[NT][2];  // reference (log2), lane's share of the sum; heads 2 t, 2 t + 1 of head tile nt
};

__host__ __device__ constexpr int ring_of(int ut) { return RING_BYTES / (ut * 128); }  // 4 stages for units of 32 tokens, 8 for 16

template <class T, int CODE, int D, int NT, int UT>
__global__ void __launch_bounds__(ATTN_THREADS, NT == 1 ? 3 : 2) kv8_attn_kernel(const Kv8AttnArgs a) {
  constexpr int KS = D / 16, MT = UT / 16, STAGE = UT * D, RING = ring_of(UT);
  extern __shared__ __align__(128) unsigned char sm[];
  const Kv8View& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
  int* pre = reinterpret_cast<int*>(sm + WARPS * RING * STAGE);
  __shared__ int s_w[WARPS];
  wait_prior();
  unit_prefix(a, UT, pre, s_w);
  const long long total = (long long)pre[c.n_seqs] * c.Hkv;
  const int w = blockIdx.x * WARPS + wid, n_runs = runs_of(total, a.n_warps, a.least_run);
  // where the rows' partial results will lie, for the merge: a few rows for each thread of the grid
  for (int r = blockIdx.x * ATTN_THREADS + tid; r < c.n_seqs * c.Hkv; r += gridDim.x * ATTN_THREADS) {
    const int s = r / c.Hkv, h = r - s * c.Hkv, nu = pre[s + 1] - pre[s];
    int2 v = make_int2(0, 0);
    if (nu > 0) {
      const long long u0 = (long long)pre[s] * c.Hkv + (long long)h * nu;
      const int w0 = run_of(total, n_runs, u0);
      v = make_int2(w0 + r, run_of(total, n_runs, u0 + nu - 1) - w0 + 1);
    }
    a.rows[r] = v;
  }
  if (w >= n_runs) return;
  long long u = run_start(total, n_runs, w);
  const long long u_end = run_start(total, n_runs, w + 1);
  unsigned char* ring = sm + wid * RING * STAGE;
  const uint32_t ring_a = (uint32_t)__cvta_generic_to_shared(ring);
  const int upb_log2 = __ffs(c.block / UT) - 1, block_log2 = __ffs(c.block) - 1;  // units of a block; both are powers of two

  while (u < u_end) {
    const int s = seq_of(pre, c.n_seqs, (int)(u / c.Hkv));
    const int nu = pre[s + 1] - pre[s];
    const long long in_seq = u - (long long)pre[s] * c.Hkv;
    const int h = (int)(in_seq / nu);
    const int i0 = (int)(in_seq - (long long)h * nu), i1 = (int)min((long long)nu, i0 + (u_end - u));
    const int row = s * c.Hkv + h;
    const int len = clamp_len(a, a.lens[s]);
    const int n_code = len >> block_log2 << upb_log2;  // units that lie in full blocks
    u += i1 - i0;

    // queries of this KV head: B fragments in fp16, divided by a power of two per head
    uint32_t qf[NT][KS][2];
    float qs[NT][2];     // of heads 2 t, 2 t + 1: that power of two times the softmax scale
    float q_off[NT][2];  // and where their logits start
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int hl = nt * 8 + g;
      float x[KS][4], mx = 0.f;
      const T* qp = static_cast<const T*>(a.q) + ((size_t)s * a.Hq + h * a.G + hl) * D + t * (D / 4);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[ks][j] = hl < a.G ? Tr<T>::to_float(qp[ks * 4 + j]) : 0.f;
          mx = fmaxf(mx, fabsf(x[ks][j]));
        }
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      // 2^-e with e the exponent of the largest element (kept where both it and its inverse are normal)
      const int e = min(max((int)(__float_as_uint(mx) >> 23), 2), 252);
      const float down = __uint_as_float((uint32_t)(254 - e) << 23), up = __uint_as_float((uint32_t)e << 23);
      float sum = 0.f;  // of the rounded elements
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const __half2 p0 = __floats2half2_rn(x[ks][code_at<CODE>(0)] * down, x[ks][code_at<CODE>(1)] * down);
        const __half2 p1 = __floats2half2_rn(x[ks][code_at<CODE>(2)] * down, x[ks][code_at<CODE>(3)] * down);
        qf[nt][ks][0] = as_u32(p0);
        qf[nt][ks][1] = as_u32(p1);
        const float2 f0 = __half22float2(p0), f1 = __half22float2(p1);
        sum += (f0.x + f0.y) + (f1.x + f1.y);
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      const float off = CODE == QEVICT_CODE_INT8 ? -128.f * 0x1p-24f * sum : 0.f;
      q_off[nt][0] = __shfl_sync(0xffffffffu, off, 8 * t);
      q_off[nt][1] = __shfl_sync(0xffffffffu, off, 8 * t + 4);
      qs[nt][0] = __shfl_sync(0xffffffffu, up, 8 * t) * a.scale_log2;
      qs[nt][1] = __shfl_sync(0xffffffffu, up, 8 * t + 4) * a.scale_log2;
    }

    Acc<D, NT> acc;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      acc.m[nt][0] = acc.m[nt][1] = -INFINITY;
      acc.l[nt][0] = acc.l[nt][1] = 0.f;
#pragma unroll
      for (int mt = 0; mt < KS; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc.o[nt][mt][j] = 0.f;
    }

    // Softmax of one unit's logits x (log2 domain, -inf where masked): moves the reference if it must, turns x into
    // probabilities, adds the sums, writes the unit's record.
    auto softmax = [&](float (&x)[NT][MT][4], int unit) {
      bool over = false;
      float mx[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float v = -INFINITY;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) v = fmaxf(v, fmaxf(x[nt][mt][j], x[nt][mt][j + 2]));
          mx[nt][j] = v;
          over |= v > acc.m[nt][j] + LAZY;  // -inf + LAZY = -inf: the first finite logit counts
        }
      if (__any_sync(0xffffffffu, over)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float v = mx[nt][j];
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
            const float old = acc.m[nt][j], m = fmaxf(old, v);
            const float f = m == old ? 1.f : ex2(old - m);
            acc.m[nt][j] = m;
            acc.l[nt][j] *= f;
#pragma unroll
            for (int mt = 0; mt < KS; ++mt) {
              acc.o[nt][mt][j] *= f;
              acc.o[nt][mt][j + 2] *= f;
            }
          }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float m = acc.m[nt][j] == -INFINITY ? 0.f : acc.m[nt][j];
          float sum = 0.f;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            x[nt][mt][j] = ex2(x[nt][mt][j] - m);
            x[nt][mt][j + 2] = ex2(x[nt][mt][j + 2] - m);
            sum += x[nt][mt][j] + x[nt][mt][j + 2];
          }
          acc.l[nt][j] += sum;
          if (a.rec) {
            sum += __shfl_xor_sync(0xffffffffu, sum, 4);
            sum += __shfl_xor_sync(0xffffffffu, sum, 8);
            sum += __shfl_xor_sync(0xffffffffu, sum, 16);
            const int hl = nt * 8 + 2 * t + j;
            if (g == 0 && hl < a.G) a.rec[((size_t)s * a.max_units + unit) * a.Hq + h * a.G + hl] = make_float2(acc.m[nt][j], sum);
          }
        }
    };

    // ---- units in full blocks: ring of asynchronous copies -----------------------------------------------------
    const int e1 = min(i1, n_code);
    if (i0 < e1) {
      // page and scales of 32 blocks at a time, one per lane; the copies run RING - 1 stages ahead
      auto fetch = [&](int blk0, int& page) {
        page = -1;
        const int b = blk0 + lane;
        if (b < n_code >> upb_log2) {
          page = c.table[(size_t)s * c.max_blocks + b];
          if (page < 0 || page >= c.n_pages) {
            if (page != -1) kv8_record(c.status, CHECK_PAGE_ID);
            page = -1;
          }
        }
      };
      int f_blk0 = i0 >> upb_log2, f_page;  // producer's window of 32 blocks
      fetch(f_blk0, f_page);
      const int e_end = 2 * (e1 - i0);
      auto issue = [&](int e) {  // stage e: keys (even) or values of unit i0 + e / 2
        if (e < e_end) {
          const int i = i0 + (e >> 1), kv = e & 1, b = i >> upb_log2;
          if (b >= f_blk0 + 32) {
            f_blk0 += 32;
            fetch(f_blk0, f_page);
          }
          const int page = __shfl_sync(0xffffffffu, f_page, b - f_blk0);
          if (page >= 0) {
            const uint8_t* src = (kv ? c.codes[1] : c.codes[0]) +
                                 (((size_t)((unsigned)page * (unsigned)c.Hkv + (unsigned)h) << block_log2) + (unsigned)((i - (b << upb_log2)) * UT)) * D;
            const uint32_t dst = ring_a + (uint32_t)(e % RING) * STAGE;
#pragma unroll
            for (int n = 0; n < UT * D / 512; ++n) {
              const int ch = n * 32 + lane, r = ch / (D / 16), cc = ch - r * (D / 16);
              cp16(dst + swz<D>(r, cc), src + ch * 16);
            }
          }
        }
        asm volatile("cp.async.commit_group;\n" ::: "memory");
      };
      auto arrived = [&] {  // the oldest stage that has not been used
        asm volatile("cp.async.wait_group %0;\n" ::"n"(RING - 2) : "memory");
        __syncwarp();
      };
      for (int e = 0; e < RING - 1; ++e) issue(e);
      int s_blk0 = (i0 >> upb_log2) - 32, s_page = -1;
      float s_k = 0.f, s_v = 0.f;
      for (int i = i0; i < e1; ++i) {
        const int b = i >> upb_log2;
        if (b >= s_blk0 + 32) {  // consumer's window: scales too
          s_blk0 = s_blk0 + 32 > b ? s_blk0 + 32 : b;
          fetch(s_blk0, s_page);
          s_k = s_page >= 0 ? c.scale[0][(size_t)s_page * c.Hkv + h] : 0.f;
          s_v = s_page >= 0 ? c.scale[1][(size_t)s_page * c.Hkv + h] : 0.f;
        }
        const int page = __shfl_sync(0xffffffffu, s_page, b - s_blk0);
        const float ksc = __shfl_sync(0xffffffffu, s_k, b - s_blk0), vsc = __shfl_sync(0xffffffffu, s_v, b - s_blk0);
        const int e = 2 * (i - i0);
        const unsigned char* kt = ring + (e % RING) * STAGE;
        const unsigned char* vt = ring + ((e + 1) % RING) * STAGE;
        arrived();
        if (page < 0) {  // absent block: nothing was copied
          if (a.rec)
            for (int hl = lane; hl < a.G; hl += 32) a.rec[((size_t)s * a.max_units + i) * a.Hq + h * a.G + hl] = make_float2(-INFINITY, 0.f);
          issue(e + RING - 1);
          arrived();
        } else {
          float x[NT][MT][4];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            uint32_t k0[KS], k1[KS];  // this lane's words of token rows g and g + 8: channels t D/4 ..
#pragma unroll
            for (int v = 0; v < D / 64; ++v) {
              const uint4 p = *reinterpret_cast<const uint4*>(kt + swz<D>(mt * 16 + g, t * (D / 64) + v));
              const uint4 r = *reinterpret_cast<const uint4*>(kt + swz<D>(mt * 16 + g + 8, t * (D / 64) + v));
              k0[v * 4] = p.x; k0[v * 4 + 1] = p.y; k0[v * 4 + 2] = p.z; k0[v * 4 + 3] = p.w;
              k1[v * 4] = r.x; k1[v * 4 + 1] = r.y; k1[v * 4 + 2] = r.z; k1[v * 4 + 3] = r.w;
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int j = 0; j < 4; ++j) x[nt][mt][j] = q_off[nt][j & 1];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
              uint32_t a0, a1, a2, a3;
              codes_to_h2<CODE>(k0[ks], a0, a2);
              codes_to_h2<CODE>(k1[ks], a1, a3);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma16816<__half>(x[nt][mt], a0, a1, a2, a3, qf[nt][ks][0], qf[nt][ks][1]);
            }
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float f = qs[nt][j] * ksc;
              // 2^24 f has to be a float32: from 2^100 on the logits take the unit first
              if (Unit<CODE>::value != 1.f && f > 0x1p100f) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                  x[nt][mt][j] *= Unit<CODE>::value;
                  x[nt][mt][j + 2] *= Unit<CODE>::value;
                }
              } else {
                f *= Unit<CODE>::value;
              }
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                x[nt][mt][j] *= f;
                x[nt][mt][j + 2] *= f;
              }
            }
          __syncwarp();  // every lane has read the keys: the next copy may go there
          issue(e + RING - 1);
          softmax(x, i);
          arrived();
          uint32_t p0[NT][MT], p1[NT][MT];
          float o[NT][KS][4];  // this unit's output before the block's scale
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float start[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              p0[nt][mt] = transpose8(as_u32(__floats2half2_rn(x[nt][mt][0], x[nt][mt][1])));
              p1[nt][mt] = transpose8(as_u32(__floats2half2_rn(x[nt][mt][2], x[nt][mt][3])));
              // -128 units for every p: the product with a matrix of -2^-17
              if (CODE == QEVICT_CODE_INT8) mma16816<__half>(start, 0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u, p0[nt][mt], p1[nt][mt]);
            }
#pragma unroll
            for (int mt = 0; mt < KS; ++mt)
#pragma unroll
              for (int j = 0; j < 4; ++j) o[nt][mt][j] = start[j & 1];
          }
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            // this lane's tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9, channels g D/8 ..
            uint32_t v[4][D / 32];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              const int r = mt * 16 + 2 * t + (n & 1) + (n >> 1) * 8;
              if (D == 128) {
                const uint4 p = *reinterpret_cast<const uint4*>(vt + swz<D>(r, g));
                v[n][0] = p.x; v[n][1] = p.y; v[n][2 % (D / 32)] = p.z; v[n][3 % (D / 32)] = p.w;
              } else {
                const uint2 p = *reinterpret_cast<const uint2*>(vt + swz<D>(r, g >> 1) + (g & 1) * 8);
                v[n][0] = p.x; v[n][1] = p.y;
              }
            }
#pragma unroll
            for (int q4 = 0; q4 < D / 32; ++q4) {
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                // two channels of two tokens in one word, in the order that codes_to_h2 takes apart into pairs of tokens
                constexpr int lo = CODE == QEVICT_CODE_INT8 ? 0x5410 : 0x5140, hi = CODE == QEVICT_CODE_INT8 ? 0x7632 : 0x7362;
                const uint32_t ab = __byte_perm(v[0][q4], v[1][q4], half ? hi : lo), cd = __byte_perm(v[2][q4], v[3][q4], half ? hi : lo);
                uint32_t a0, a1, a2, a3;
                codes_to_h2<CODE>(ab, a0, a1);
                codes_to_h2<CODE>(cd, a2, a3);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma16816<__half>(o[nt][q4 * 2 + half], a0, a1, a2, a3, p0[nt][mt], p1[nt][mt]);
              }
            }
          }
          float vs = vsc * Unit<CODE>::value;
          if (Unit<CODE>::value != 1.f && vsc > 0x1p100f) {  // the same for the block's output
            vs = vsc;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int mt = 0; mt < KS; ++mt)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[nt][mt][j] *= Unit<CODE>::value;
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < KS; ++mt)
#pragma unroll
              for (int j = 0; j < 4; ++j) acc.o[nt][mt][j] = fmaf(o[nt][mt][j], vs, acc.o[nt][mt][j]);
        }
        __syncwarp();
        issue(e + RING);
      }
      asm volatile("cp.async.wait_group 0;\n" ::: "memory");
      __syncwarp();
    }

    // ---- units of the open block: 16-bit rows -----------------------------------------------------------------
    for (int i = max(i0, n_code); i < i1; ++i) {
      const int r0 = (i - n_code) * UT, rows = len - n_code * UT - r0;  // valid tokens from r0 on
      const T* kp = static_cast<const T*>(c.tail[0]) + ((size_t)row * c.block + r0) * D;
      const T* vp = static_cast<const T*>(c.tail[1]) + ((size_t)row * c.block + r0) * D;
      float x[NT][MT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[nt][mt][j] = 0.f;
#pragma unroll 2
      for (int ks = 0; ks < KS; ++ks) {
        uint2 qv[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int hl = nt * 8 + g;
          qv[nt] = hl < a.G ? *reinterpret_cast<const uint2*>(static_cast<const T*>(a.q) + ((size_t)s * a.Hq + h * a.G + hl) * D + t * (D / 4) + ks * 4)
                            : make_uint2(0u, 0u);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint2 ka = make_uint2(0u, 0u), kb = ka;
          const int ra = mt * 16 + g, rb = ra + 8;
          if (ra < rows) ka = *reinterpret_cast<const uint2*>(kp + (size_t)ra * D + t * (D / 4) + ks * 4);
          if (rb < rows) kb = *reinterpret_cast<const uint2*>(kp + (size_t)rb * D + t * (D / 4) + ks * 4);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma16816<T>(x[nt][mt], ka.x, kb.x, ka.y, kb.y, qv[nt].x, qv[nt].y);
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            x[nt][mt][j] = mt * 16 + g + (j >> 1) * 8 < rows ? x[nt][mt][j] * a.scale_log2 : -INFINITY;
      softmax(x, i);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        // probabilities in T, and (bf16) what the rounding left, so that the open block is as exact as the others
        uint32_t p0[NT], p1[NT], d0[NT], d1[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          T hi[4], lo[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            hi[j] = Tr<T>::from_float(x[nt][mt][j]);
            lo[j] = Tr<T>::from_float(x[nt][mt][j] - Tr<T>::to_float(hi[j]));
          }
          p0[nt] = transpose8(*reinterpret_cast<uint32_t*>(&hi[0]));
          p1[nt] = transpose8(*reinterpret_cast<uint32_t*>(&hi[2]));
          d0[nt] = transpose8(*reinterpret_cast<uint32_t*>(&lo[0]));
          d1[nt] = transpose8(*reinterpret_cast<uint32_t*>(&lo[2]));
        }
#pragma unroll 2
        for (int o2 = 0; o2 < KS; ++o2) {  // channels g D/8 + 2 o2, + 1
          uint32_t v[4];
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const int r = mt * 16 + 2 * t + (n & 1) + (n >> 1) * 8;
            v[n] = r < rows ? *reinterpret_cast<const uint32_t*>(vp + (size_t)r * D + g * (D / 8) + 2 * o2) : 0u;
          }
          const uint32_t a0 = __byte_perm(v[0], v[1], 0x5410), a1 = __byte_perm(v[0], v[1], 0x7632);
          const uint32_t a2 = __byte_perm(v[2], v[3], 0x5410), a3 = __byte_perm(v[2], v[3], 0x7632);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int z = 0; z < KS; ++z)
              if (z == o2) {  // keeps the accumulators in registers under the partial unroll
                mma16816<T>(acc.o[nt][z], a0, a1, a2, a3, p0[nt], p1[nt]);
                mma16816<T>(acc.o[nt][z], a0, a1, a2, a3, d0[nt], d1[nt]);
              }
          }
        }
      }
    }

    if (u >= u_end) release_next();
    // ---- partial result of this run's part of the row -----------------------------------------------------------
    const size_t slot = (size_t)w + row;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float l = acc.l[nt][j];
        l += __shfl_xor_sync(0xffffffffu, l, 4);
        l += __shfl_xor_sync(0xffffffffu, l, 8);
        l += __shfl_xor_sync(0xffffffffu, l, 16);
        const int hl = nt * 8 + 2 * t + j;
        if (hl < a.G) {
          if (g == 0) a.part_ml[slot * a.G + hl] = make_float2(acc.m[nt][j], l);
          float4* dst = reinterpret_cast<float4*>(a.part_o + (slot * a.G + hl) * D + g * (D / 8));
#pragma unroll
          for (int mt = 0; mt < KS; mt += 2)
            dst[mt >> 1] = make_float4(acc.o[nt][mt][j], acc.o[nt][mt][j + 2], acc.o[nt][mt + 1][j], acc.o[nt][mt + 1][j + 2]);
        }
      }
  }
}

// Merges the partial results and adds up the block masses, side by side in one launch: a CTA has a (query head, sequence) or
// some blocks of a sequence.  The masses need every head's maximum and denominator; their CTAs work those out for themselves
// from the {reference, sum} pairs, 8 to 32 threads to a head.
// (As a kernel of their own behind the merge the masses cost 0.4 to 3 us more and a launch; as a second task of the merge's CTAs,
// each of which then goes through both tasks' code and statistics, 2 to 4 us more.)
constexpr int MERGE_THREADS = 256, MERGE_WARPS = MERGE_THREADS / 32;

// One (query head, sequence).  A warp takes partials wid, wid + 8, ... with a running maximum of its own, so that everything
// it needs is requested at once; the eight warps' results meet in shared memory.
template <class T> __device__ void merge_head(const Kv8AttnArgs& a, int s, int hq) {
  __shared__ float s_m[MERGE_WARPS], s_l[MERGE_WARPS], s_o[MERGE_WARPS][128];
  const int h = hq / a.G, hl = hq - h * a.G, D = a.c.D, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int2 where = a.rows[s * a.c.Hkv + h];
  const int n = where.y;
  if (tid == 0 && a.c.status && hq == 0 && a.lens[s] > a.max_len) kv8_record(a.c.status, CHECK_LENGTH);
  const float2* ml0 = a.part_ml + (size_t)where.x * a.G + hl;
  const float* o0 = a.part_o + ((size_t)where.x * a.G + hl) * D;
  // lanes hold 4 channels each (d = 64: half the lanes, twice as many partials at a time)
  const int per = D / 4, sub = lane / per, subs = 32 / per, c4 = lane - sub * per;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int AT_ONCE = 8;
  for (int i0 = wid * subs + sub; i0 < n; i0 += AT_ONCE * MERGE_WARPS * subs) {
    float2 ml[AT_ONCE];
    float4 v[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const int i = i0 + k * MERGE_WARPS * subs;
      ml[k] = i < n ? ml0[(size_t)i * a.G] : make_float2(-INFINITY, 0.f);
      v[k] = i < n ? *reinterpret_cast<const float4*>(o0 + (size_t)i * a.G * D + c4 * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) top = fmaxf(top, ml[k].x);
    const float ref = top == -INFINITY ? 0.f : top, f0 = ex2(m - ref);  // m = -inf: 0
    l *= f0;
    o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
    m = top;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const float f = ex2(ml[k].x - ref);
      l += ml[k].y * f;
      o.x += v[k].x * f; o.y += v[k].y * f; o.z += v[k].z * f; o.w += v[k].w * f;
    }
  }
  if (subs == 2) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, 16), top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
    const float f = ex2(m - ref);
    l *= f;
    l += __shfl_xor_sync(0xffffffffu, l, 16);
    o.x *= f; o.y *= f; o.z *= f; o.w *= f;
    o.x += __shfl_xor_sync(0xffffffffu, o.x, 16);
    o.y += __shfl_xor_sync(0xffffffffu, o.y, 16);
    o.z += __shfl_xor_sync(0xffffffffu, o.z, 16);
    o.w += __shfl_xor_sync(0xffffffffu, o.w, 16);
    m = top;
  }
  if (lane == 0) {
    s_m[wid] = m;
    s_l[wid] = l;
  }
  if (sub == 0) *reinterpret_cast<float4*>(&s_o[wid][c4 * 4]) = o;
  __syncthreads();
  if (tid < D) {
    float M = s_m[0];
#pragma unroll
    for (int i = 1; i < MERGE_WARPS; ++i) M = fmaxf(M, s_m[i]);
    const float Ms = M == -INFINITY ? 0.f : M;
    float L = 0.f, v = 0.f;
#pragma unroll
    for (int i = 0; i < MERGE_WARPS; ++i) {
      const float f = ex2(s_m[i] - Ms);
      L += s_l[i] * f;
      v += s_o[i][tid] * f;
    }
    static_cast<T*>(a.out)[((size_t)s * a.Hq + hq) * D + tid] = Tr<T>::from_float(L > 0.f ? v / L : (L == 0.f ? 0.f : v));
    if (tid == 0 && a.lse) a.lse[(size_t)s * a.Hq + hq] = L == 0.f ? -INFINITY : (Ms + log2f(L)) * 0.6931471805599453f;
  }
}

// Blocks b0 .. b1 - 1 of a sequence.  One warp per block, a lane per head, fixed shuffle trees.
__device__ void block_masses(const Kv8AttnArgs& a, int s, int b0, int b1, int ut, float2* s_stat) {
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int nu = (clamp_len(a, a.lens[s]) + ut - 1) / ut, upb = a.c.block / ut;
  if (b0 * upb < nu) {
    const int per_log2 = a.Hq <= 8 ? 5 : a.Hq <= 16 ? 4 : 3, per = 1 << per_log2;  // threads to a head
#pragma unroll 1
    for (int h0 = 0; h0 < a.Hq; h0 += MERGE_THREADS >> per_log2) {
      const int hq = h0 + (tid >> per_log2), part = tid & (per - 1);
      float m = -INFINITY, l = 0.f;
      if (hq < a.Hq) {
        const int h = hq / a.G;
        const int2 where = a.rows[s * a.c.Hkv + h];
        const float2* ml = a.part_ml + (size_t)where.x * a.G + hq - h * a.G;
        for (int i0 = part; i0 < where.y; i0 += 8 * per) {
          float2 v[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = i0 + k * per < where.y ? ml[(size_t)(i0 + k * per) * a.G] : make_float2(-INFINITY, 0.f);
          float top = m;
#pragma unroll
          for (int k = 0; k < 8; ++k) top = fmaxf(top, v[k].x);
          const float ref = top == -INFINITY ? 0.f : top;
          l *= ex2(m - ref);
#pragma unroll
          for (int k = 0; k < 8; ++k) l += v[k].y * ex2(v[k].x - ref);
          m = top;
        }
      }
      float M = m;
      for (int o = per >> 1; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      const float Ms = M == -INFINITY ? 0.f : M;
      l *= ex2(m - Ms);
      for (int o = per >> 1; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
      if (hq < a.Hq && part == 0) s_stat[hq] = make_float2(Ms, l == 0.f ? 0.f : 1.f / l);
    }
  }
  __syncthreads();
#pragma unroll 1
  for (int b = b0 + wid; b < b1; b += MERGE_WARPS) {
    const size_t at = (size_t)s * a.c.max_blocks + b;
    const float before = a.score_in ? a.score_in[at] : 0.f;
    const int have = min(upb, nu - b * upb);  // units of this block that were read
    float mass = 0.f;
    for (int h = lane; h < a.Hq && have > 0; h += 32) {
      const float2* rec = a.rec + ((size_t)s * a.max_units + (size_t)b * upb) * a.Hq + h;
      float2 r[4];  // a block has at most four units
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = i < have ? rec[(size_t)i * a.Hq] : make_float2(-INFINITY, 0.f);
      const float2 st = s_stat[h];
#pragma unroll
      for (int i = 0; i < 4; ++i) mass += r[i].y * ex2(r[i].x - st.x) * st.y;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, o);
    if (lane == 0) a.score_out[at] = before + mass;
  }
}

template <class T> __global__ void __launch_bounds__(MERGE_THREADS) kv8_merge_kernel(const Kv8AttnArgs a, int ut, int mass_blocks) {
  extern __shared__ float2 s_stat[];  // [Hq] {maximum, 1 / denominator}
  wait_prior();
  const int b0 = ((int)blockIdx.x - a.Hq) * mass_blocks;
  if (b0 < 0) merge_head<T>(a, blockIdx.y, blockIdx.x);
  else block_masses(a, blockIdx.y, b0, min(b0 + mass_blocks, a.c.max_blocks), ut, s_stat);
}

struct Plan {
  int ut, n_warps, max_units, max_len, least_run;
  size_t off_ml, off_rec, off_rows, bytes;
};

int sm_count(int device) {
  int n = 0;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) {
    (void)cudaGetLastError();
    n = SM_COUNT_FALLBACK;
  }
  return n;
}

const char* plan_of(const Kv8View& c, int Hq, int max_len, bool scores, int sms, qevict_status* st, Plan* p) {
  *st = QEVICT_ERR_INVALID_ARG;
  if (Hq < 1 || Hq % c.Hkv) return "n_q_heads must be a multiple of n_kv_heads";
  if (max_len < 0) return "max_len must be >= 0";
  *st = QEVICT_ERR_UNSUPPORTED;
  if (Hq / c.Hkv > 16) return "more than 16 query heads per KV head";
  const long long cap = (long long)c.max_blocks * c.block;
  p->max_len = (int)(max_len < cap ? max_len : cap);
  p->ut = c.block >= 32 ? 32 : 16;
  p->max_units = (p->max_len + p->ut - 1) / p->ut;
  if ((long long)c.n_seqs * p->max_units > 0x7fffffffll) return "n_seqs * max_len is too large for one call";
  const int G = Hq / c.Hkv;
  const int ctas_per_sm = G <= 8 ? 3 : 2;
  // A unit costs a warp about 1.3 us, and the merge about 1 us for every 64 partial results of a row: r units a run take
  // 1.3 r + units / (64 r) us on one long row, least at sqrt(units / 80) (one sequence of 29660 tokens with one KV head for 16
  // heads: 29 us, 34 with a unit a run; one of 60000 with two KV heads for four: 18 and 22; a sequence with eight KV heads
  // loses 1 to 2 %).
  p->least_run = (int)(sqrt(p->max_units / 80.0) + 0.5);
  if (p->least_run < 1) p->least_run = 1;
  const long long units = ((long long)c.n_seqs * c.Hkv * p->max_units + p->least_run - 1) / p->least_run;
  long long ctas = (units + WARPS - 1) / WARPS;
  if (ctas > (long long)sms * ctas_per_sm) ctas = (long long)sms * ctas_per_sm;
  if (ctas < 1) ctas = 1;
  p->n_warps = (int)ctas * WARPS;
  const size_t slots = (size_t)p->n_warps + (size_t)c.n_seqs * c.Hkv;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  p->off_ml = up(slots * G * c.D * sizeof(float));
  p->off_rows = p->off_ml + up(slots * G * sizeof(float2));
  p->off_rec = p->off_rows + up((size_t)c.n_seqs * c.Hkv * sizeof(int2));
  p->bytes = p->off_rec + (scores ? up((size_t)c.n_seqs * p->max_units * Hq * sizeof(float2)) : 0);
  return nullptr;
}

template <class T, int CODE, int D, int NT, int UT> cudaError_t launch_attn(const Kv8AttnArgs& a, int device, cudaStream_t s) {
  constexpr int RING = ring_of(UT);
  const size_t smem = (size_t)WARPS * RING * UT * D + (size_t)(a.c.n_seqs + 1) * sizeof(int);
  auto kernel = kv8_attn_kernel<T, CODE, D, NT, UT>;
  static std::atomic<uint64_t> done{0};
  cudaError_t e = once_per_device(done, device, [&] {  // the largest batch that is taken
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, WARPS * RING * UT * D + 8193 * (int)sizeof(int));
  });
  if (e == cudaSuccess) e = launch_pdl(kernel, dim3(a.n_warps / WARPS), dim3(ATTN_THREADS), smem, s, a);
  return e;
}

template <class T, int CODE, int D, int NT> cudaError_t launch_attn_ut(const Kv8AttnArgs& a, int ut, int device, cudaStream_t s) {
  return ut == 32 ? launch_attn<T, CODE, D, NT, 32>(a, device, s) : launch_attn<T, CODE, D, NT, 16>(a, device, s);
}
template <class T, int CODE> cudaError_t launch_attn_shape(const Kv8AttnArgs& a, int ut, int device, cudaStream_t s) {
  const bool wide = a.G > 8;
  if (a.c.D == 128) return wide ? launch_attn_ut<T, CODE, 128, 2>(a, ut, device, s) : launch_attn_ut<T, CODE, 128, 1>(a, ut, device, s);
  return wide ? launch_attn_ut<T, CODE, 64, 2>(a, ut, device, s) : launch_attn_ut<T, CODE, 64, 1>(a, ut, device, s);
}
template <class T> cudaError_t launch_all(const Kv8AttnArgs& a, int code, int ut, int sms, int device, cudaStream_t s) {
  cudaError_t e = code == QEVICT_CODE_INT8 ? launch_attn_shape<T, QEVICT_CODE_INT8>(a, ut, device, s) : launch_attn_shape<T, QEVICT_CODE_E4M3>(a, ut, device, s);
  // the same split of the SM's memory as the attention kernel's: an SM has to drain before it changes it
  static std::atomic<uint64_t> done{0};
  if (e == cudaSuccess)
    e = once_per_device(done, device, [] {
      const cudaError_t x = cudaFuncSetAttribute(kv8_merge_kernel<T>, cudaFuncAttributePreferredSharedMemoryCarveout, 100);
      return x != cudaSuccess ? x : cudaFuncSetAttribute(kv8_merge_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 16384 * (int)sizeof(float2));
    });
  // Blocks of a mass CTA: one to four for each of its warps, so that they about fill the SMs (one context of 2048 tokens 10.8 us
  // with four, 9.0 with one; two of 8000 tokens 14.7 and 12.3, with the statistics' threads by the number of heads).
  int mass_blocks = MERGE_WARPS;
  while (mass_blocks < 4 * MERGE_WARPS && (long long)a.c.max_blocks * a.c.n_seqs > (long long)sms * mass_blocks) mass_blocks += MERGE_WARPS;
  const int mass_ctas = a.score_out ? (a.c.max_blocks + mass_blocks - 1) / mass_blocks : 0;
  if (e == cudaSuccess)
    e = launch_pdl(kv8_merge_kernel<T>, dim3(a.Hq + mass_ctas, a.c.n_seqs), dim3(MERGE_THREADS), a.score_out ? (size_t)a.Hq * sizeof(float2) : 0, s, a, ut, mass_blocks);
  return e;
}

}  // namespace

}  // namespace qevict

using namespace qevict;

extern "C" {

QEVICT_API qevict_status qevict_kv8_attn_scratch_bytes(const qevict_kv8_cache* cache, int32_t n_q_heads, int32_t max_len,
                                                       int32_t with_scores, uint64_t* bytes) {
  Kv8View v;
  qevict_status st;
  Plan p;
  const char* why = kv8_check(cache, &st, &v);
  if (!why && !bytes) { why = "bytes is NULL"; st = QEVICT_ERR_INVALID_ARG; }
  if (!why) why = plan_of(v, n_q_heads, max_len, with_scores != 0, sm_count(cache->device), &st, &p);
  if (why) return stateless_fail(st, why);
  *bytes = p.bytes;
  return QEVICT_OK;
}

QEVICT_API qevict_status qevict_kv8_attn(const qevict_kv8_cache* cache, int32_t n_q_heads, float softmax_scale, const void* q,
                                         const int32_t* lens, int32_t max_len, void* out, float* lse, const float* score_in,
                                         float* score_out, void* scratch, uint64_t scratch_bytes, void* stream) {
  Kv8AttnArgs a;
  qevict_status st;
  Plan p;
  auto bad = [](const char* msg) { return stateless_fail(QEVICT_ERR_INVALID_ARG, msg); };
  const char* why = kv8_check(cache, &st, &a.c);
  const int sms = why ? 0 : sm_count(cache->device);
  if (!why) why = plan_of(a.c, n_q_heads, max_len, score_out != nullptr, sms, &st, &p);
  if (why) return stateless_fail(st, why);
  if (!usable_scale(softmax_scale)) return bad("softmax_scale must be 0 or between 1e-30 and 2e38");
  if (score_in && !score_out) return bad("score_in needs score_out");
  if (a.c.n_seqs == 0) return QEVICT_OK;
  if (!q || !lens || !out || !scratch) return bad("q, lens, out and scratch must not be NULL");
  if (misaligned16(q) || misaligned16(out) || (reinterpret_cast<uintptr_t>(scratch) & 15u)) return bad("q, out and scratch must be 16-byte aligned");
  if (misaligned4(lens) || misaligned4(lse) || misaligned4(score_in) || misaligned4(score_out)) return bad("lens, lse and scores must be 4-byte aligned");
  if (scratch_bytes < p.bytes) return stateless_fail(QEVICT_ERR_NO_MEMORY, "scratch too small: see qevict_kv8_attn_scratch_bytes");
  a.Hq = n_q_heads; a.G = n_q_heads / a.c.Hkv;
  a.scale_log2 = (float)((softmax_scale > 0.f ? (double)softmax_scale : 1.0 / sqrt((double)a.c.D)) * 1.4426950408889634);
  a.q = q; a.lens = lens; a.max_len = p.max_len; a.n_warps = p.n_warps; a.max_units = p.max_units; a.least_run = p.least_run;
  a.out = out; a.lse = lse; a.score_in = score_in; a.score_out = score_out;
  char* base = static_cast<char*>(scratch);
  a.part_o = reinterpret_cast<float*>(base);
  a.part_ml = reinterpret_cast<float2*>(base + p.off_ml);
  a.rows = reinterpret_cast<int2*>(base + p.off_rows);
  a.rec = score_out ? reinterpret_cast<float2*>(base + p.off_rec) : nullptr;
  DeviceGuard guard(cache->device);
  cudaError_t e = guard.err;
  cudaStream_t s = (cudaStream_t)stream;
  if (e == cudaSuccess)
    e = cache->dtype == QEVICT_DTYPE_FP16 ? launch_all<__half>(a, cache->code, p.ut, sms, cache->device, s) : launch_all<__nv_bfloat16>(a, cache->code, p.ut, sms, cache->device, s);
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  return QEVICT_OK;
}

}  // extern "C"
