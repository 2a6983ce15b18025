// Attention of few new tokens (a step of decoding, drafts) over the 16-bit paged cache.
//
//     S = Q K^T,  P = 2^(S * scale * log2 e - m),  O += P V
//
// The rows are the tokens of all heads that share a KV head, at most 16 of them, so keys and values are read once and
// bandwidth bounds it, or the latency of a short call.  The four warps of a CTA take 16 keys in turn, straight from global memory
// into the registers that the products want them in, the next ones on their way while these are in work, and join their sums
// through shared memory in the end.
//   - mma.m16n8k16 contracts over channels in any order, so a lane takes 16 bytes of a key as the operands of two steps (elements
//     0, 1 | 2, 3 and 4, 5 | 6, 7), and the queries are laid out to match.
//   - A lane has 16 bytes of two neighbouring keys' values; byte permutes pair them, and the output's columns come in the order
//     that this gives (channel 8 n + e is column n of step e).
//   - Keys past the end and blocks that are not there are not read; their operands are zero and their logits masked.
// How the keys are shared: a call with up to FEW_CLUSTER_KEYS keys for each CTA of one wave gives a (sequence, KV head) a cluster of
// up to 16 CTAs, which join their sums through each other's shared memory (one launch, no scratch); any other gives each CTA an equal
// range of its work (FewRange) and joins what ranges share in a second launch.
// Measured (32 / 8 heads of 128, one token for each of n sequences, graph replays; beside it the kernel for tiles of rows, which takes
// 16 rows as 128): n = 1, 128 tokens 5.5 us (14.1), 2048 tokens 9.2 us (17.8), 8000: 17.5 to 18.4 us (22.9); n = 16, 2000: 34.3 us (40.7).
// Ranges, call after call: n = 64, 2048 tokens 109 us (124), 8 x 65536 tokens of 28 / 4 heads 195 to 205 us (5.2 to 5.5 TB/s; 230): short
// runs take 193 us either way, but here the power limit leaves 1.75 GHz where tensor memory products of 128 rows leave 1.57.
// The rest of P behind its rounding as a second product takes the error against 64 bits from 2.0e-3 to 1.6e-3 in bf16 (the output's own
// rounding) and costs 5 to 6 % (8 x 65536 193 -> 204 us): left out, as in the kernel for tiles.
// Loads on their way have their place in the L1, so shared memory is kept small: with all of it 8 x 65536 tokens took 270 us; through a
// ring in shared memory (cp.async) 231 us.
#pragma once

#include "prompt_attn.cuh"

namespace qevict {

namespace {

constexpr int FEW_WARPS = 4, FEW_KEYS = 16;
constexpr int FEW_ITEM_COST = 5, FEW_RANGE_LEAST = 8;  // steps of 16 keys
constexpr int FEW_ROWS = 16, FEW_SLOT_ROWS = 32, FEW_CTAS = 3;  // of an SM: 168 registers a thread
constexpr int few_smem(int D) { return (FEW_WARPS * 72 + D) * FEW_ROWS * 4 + D / 32 * 1024 + (FEW_WARPS + 1) * FEW_ROWS * 8; }

__device__ __forceinline__ uint4 ld_page16(const void* p) {
  uint4 r;
  asm("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
  return r;
}
__device__ __forceinline__ float peer_float(uint32_t addr, int rank) {
  uint32_t p;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(p) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(p) : "memory");
  return v;
}
__device__ __forceinline__ float4 peer_float4(uint32_t addr, int rank) {
  uint32_t p;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(p) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(p) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

struct FewPages {
  const void* pages[2];
  long long stride[2][3];
  const void* q;
  long long q_stride[2];  // token, head
};

// A CTA's equal range of the work: the sequences' KV heads stand in a row, each of its steps and FEW_ITEM_COST more.  An end inside a
// KV head's constant is moved to its first step.  (The host sees to it that the sum fits 31 bits.)
struct FewRange {
  uint32_t width, lo, hi, at;  // this CTA's part of the sum; start of the current item
  int s, h, q0, nq, nk;
  int lane_q0, lane_nq, lane_nk, first;  // the lane's sequence of 32, of which `first` is the first

  static __device__ __forceinline__ uint32_t cost(int nq, int nk) { return nq > 0 ? (nk + FEW_KEYS - 1) / FEW_KEYS + FEW_ITEM_COST : 0; }
  __device__ __forceinline__ uint32_t look(const PromptArgs& a, int s0, int lane) {  // work of the lane's sequence
    int k0;
    lane_q0 = lane_nq = lane_nk = 0;
    first = s0;
    if (s0 + lane < a.n_seqs) {
      q_span<true>(a, s0 + lane, &lane_q0, &lane_nq);
      k_span<true>(a, s0 + lane, &k0, &lane_nk);
    }
    return cost(lane_nq, lane_nk) * a.Hkv;
  }
  __device__ __forceinline__ void sequence(const PromptArgs& a, int lane) {
    if (s >= first + 32) look(a, s & ~31, lane);
    q0 = __shfl_sync(0xffffffffu, lane_q0, s & 31);
    nq = __shfl_sync(0xffffffffu, lane_nq, s & 31);
    nk = __shfl_sync(0xffffffffu, lane_nk, s & 31);
  }
  __device__ __forceinline__ FewRange(const PromptArgs& a, int lane) {
    uint32_t sum = 0, mine = 0;
    for (int i = 0; i < a.n_seqs; i += 32) {
      mine = look(a, i, lane);
      sum += __reduce_add_sync(0xffffffffu, mine);
    }
    width = (sum + gridDim.x - 1) / gridDim.x;
    if (width < FEW_RANGE_LEAST) width = FEW_RANGE_LEAST;
    lo = blockIdx.x * width;
    hi = min(lo + width, sum);
    s = a.n_seqs;
    if (lo >= sum) return;
    uint32_t front = 0;  // work of the sequences before
#pragma unroll 1
    for (int i = 0; i < a.n_seqs; i += 32) {
      if (a.n_seqs > 32) mine = look(a, i, lane);
      uint32_t upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
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
    sequence(a, lane);
    h = small_quotient(lo - front, cost(nq, nk));
    at = front + h * cost(nq, nk);
  }
  // The next item, its steps in the range; false behind the last one.
  __device__ __forceinline__ bool next(const PromptArgs& a, int lane, bool writes, PromptItem* it) {
#pragma unroll 1
    while (s < a.n_seqs && at < hi) {
      const uint32_t end = at + cost(nq, nk);
      const int all = (nk + FEW_KEYS - 1) / FEW_KEYS;
      auto steps_upto = [&](uint32_t x) { return x <= at + FEW_ITEM_COST ? 0 : (int)(x - at - FEW_ITEM_COST); };
      const bool ends = end <= hi;
      it->s = s; it->h0 = h * a.P; it->q0 = q0; it->nq = nq; it->nk = nk;
      it->lo = lo > at ? steps_upto(lo) : 0;
      it->n = ends ? all : steps_upto(hi);
      it->slot = it->lo == 0 && ends ? -1 : 2 * (int)blockIdx.x + (it->lo == 0);
      if (it->lo == 0 && it->n > 0 && !ends && writes) {
        const PagedCut c = {1, s, it->h0, 0, q0, nq, (int)small_quotient(end - 1, width), 0};
        a.cuts[blockIdx.x] = c;
      }
      at = end;
      if (++h == a.Hkv) {
        h = 0;
        do {
          if (++s < a.n_seqs) sequence(a, lane);
        } while (s < a.n_seqs && nq == 0);
      }
      if (it->n > it->lo || (all == 0 && ends)) return true;
    }
    return false;
  }
};

// CLUSTER: blockIdx is (KV head * ranks + rank, sequence)
template <class T, int D, bool CLUSTER>
__global__ void __launch_bounds__(32 * FEW_WARPS, FEW_CTAS) few_attn_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ FewPages g) {
  constexpr int J = D / 32;       // 16-byte pieces of a key in a lane
  constexpr int H = D / 64;       // of a value
  constexpr int N = D / 8;        // column steps of the output
  constexpr int LINE = 64 + 8;    // floats from row to row of a warp's output, 64 channels at a time
  extern __shared__ __align__(16) unsigned char few_sm[];
  auto os = reinterpret_cast<float (*)[FEW_ROWS][LINE]>(few_sm);                    // outputs: the warps', [FEW_WARPS]
  auto mine = reinterpret_cast<float (*)[D]>(os + FEW_WARPS);                       // the CTA's, [FEW_ROWS]
  auto qf = reinterpret_cast<uint4 (*)[32]>(mine + FEW_ROWS);                       // queries, [2 J]
  auto ms = reinterpret_cast<float (*)[FEW_ROWS]>(qf + 2 * J), ls = ms + FEW_WARPS + 1;  // references and sums: the warps', the CTA's
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = lane >> 2, c = lane & 3;
  pdl_prologue();
  if (!CLUSTER && a.cuts && tid == 0) a.cuts[blockIdx.x].valid = 0;

  // keys f0 * 16 .. f1 * 16 - 1 for the rows of one KV head
  auto attend = [&](const PromptItem& it, int f0, int f1, auto take) {
    const int hk = it.h0 / a.P;
    // pages of this warp's next 32 steps, one per lane
    const int blocks = (it.nk + (1 << a.block_log2) - 1) >> a.block_log2;
    auto fetch = [&](int k0) {
      const int step = f0 + warp + (k0 + lane) * FEW_WARPS, b = step >> (a.block_log2 - 4);
      int p = -1;
      if (step < f1 && b < blocks) {
        p = a.table[(size_t)it.s * a.max_blocks + b];
        if (p < 0 || p >= a.n_pages) {
          if (p != -1) kv8_record(a.status, CHECK_PAGE_ID);
          p = -1;
        }
      }
      return p;
    };
    int ids = fetch(0);
    // queries, in the order of the operands; requested before the pages' rows, behind which they would wait
    uint2 q[J / 2][2];
#pragma unroll
    for (int u = 0; u < J / 2; ++u) {
      const int ju = warp + u * FEW_WARPS, ch = (c + 4 * (ju >> 1)) * 8 + (ju & 1) * 4;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = row + 8 * i, hl = r / a.T, tok = r - hl * a.T;
        q[u][i] = make_uint2(0u, 0u);
        if (hl < a.P && tok < it.nq)
          q[u][i] = *reinterpret_cast<const uint2*>(static_cast<const T*>(g.q) + (long long)(it.q0 + tok) * g.q_stride[0] + (long long)(it.h0 + hl) * g.q_stride[1] + ch);
      }
    }
    // this lane's parts of the keys and values of a step; rows past the end are zero
    uint4 k[2][J], v[4][H];
    auto load_k = [&](int step, int page) {
      const int t = (step * FEW_KEYS) & ((1 << a.block_log2) - 1), left = it.nk - step * FEW_KEYS;
      const T* p = static_cast<const T*>(g.pages[0]) + page * g.stride[0][0] + hk * g.stride[0][1] + (t + row) * g.stride[0][2] + c * 8;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int j = 0; j < J; ++j)
          k[n][j] = n * 8 + row < left ? ld_page16(p + n * 8 * g.stride[0][2] + j * 32) : make_uint4(0u, 0u, 0u, 0u);
    };
    auto load_v = [&](int step, int page) {
      const int t = (step * FEW_KEYS) & ((1 << a.block_log2) - 1), left = it.nk - step * FEW_KEYS;
      const T* p = static_cast<const T*>(g.pages[1]) + page * g.stride[1][0] + hk * g.stride[1][1] + (t + 2 * c) * g.stride[1][2] + row * 8;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = (i & 1) + (i >> 1) * 8;
#pragma unroll
        for (int h = 0; h < H; ++h)
          v[i][h] = 2 * c + key < left ? ld_page16(p + key * g.stride[1][2] + h * 64) : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    int step = f0 + warp, at = 0, page = __shfl_sync(0xffffffffu, ids, 0);
    if (step < f1 && page >= 0) {
      load_k(step, page);
      load_v(step, page);
    }
#pragma unroll
    for (int u = 0; u < J / 2; ++u) qf[warp + u * FEW_WARPS][lane] = make_uint4(q[u][0].x, q[u][1].x, q[u][0].y, q[u][1].y);
    // keys that the rows of this lane see, that every row sees
    const int all_see = a.causal ? it.nk - it.nq + 1 : it.nk;
    int sees[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) sees[i] = a.causal ? min(it.nk, all_see + (row + 8 * i) % a.T) : it.nk;
    float o[N][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < N; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    __syncthreads();
    for (; step < f1; step += FEW_WARPS) {
      int next = -1;
      if (step + FEW_WARPS < f1) {
        if (((++at) & 31) == 0) ids = fetch(at);
        next = __shfl_sync(0xffffffffu, ids, at & 31);
      }
      if (page >= 0) {
        float x[2][4] = {};
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const uint4 q0 = qf[2 * j][lane], q1 = qf[2 * j + 1][lane];
          mma16816<T>(x[0], q0.x, q0.y, q0.z, q0.w, k[0][j].x, k[0][j].y);
          mma16816<T>(x[1], q0.x, q0.y, q0.z, q0.w, k[1][j].x, k[1][j].y);
          mma16816<T>(x[0], q1.x, q1.y, q1.z, q1.w, k[0][j].z, k[0][j].w);
          mma16816<T>(x[1], q1.x, q1.y, q1.z, q1.w, k[1][j].z, k[1][j].w);
        }
        if (next >= 0) load_k(step + FEW_WARPS, next);
        const int key0 = step * FEW_KEYS;
        if (key0 + FEW_KEYS > all_see) {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + n * 8 + 2 * c + (i & 1) >= sees[i >> 1]) x[n][i] = -INFINITY;
        }
        bool moves = false;
        float top[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float t = fmaxf(fmaxf(x[0][2 * i], x[0][2 * i + 1]), fmaxf(x[1][2 * i], x[1][2 * i + 1]));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
          top[i] = t * a.scale_log2 - P_UP<T>;
          moves = moves || top[i] > m[i] + PROMPT_LAZY;
        }
        if (__any_sync(0xffffffffu, moves)) {  // each row by its own logits: what else is in the tile has no say
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (!(top[i] > m[i] + PROMPT_LAZY)) continue;
            const float f = ex2p(m[i] - top[i]);
            m[i] = top[i];
            l[i] *= f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
              o[n][2 * i] *= f;
              o[n][2 * i + 1] *= f;
            }
          }
        }
        // P enters the product in the type of the values, half a step off each (prompt_attn.cuh says why m is where it is)
        uint32_t p[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float sub = m[i] == -INFINITY ? 0.f : -m[i];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const float e0 = ex2p(fmaf(x[n][2 * i], a.scale_log2, sub)), e1 = ex2p(fmaf(x[n][2 * i + 1], a.scale_log2, sub));
            l[i] += e0 + e1;
            p[2 * n + i] = pack2<T>(e0, e1);
          }
        }
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int sel = e & 1 ? 0x7632 : 0x5410;
            auto word = [&](const uint4& u) { return e < 2 ? u.x : e < 4 ? u.y : e < 6 ? u.z : u.w; };
            mma16816<T>(o[h * 8 + e], p[0], p[1], p[2], p[3], __byte_perm(word(v[0][h]), word(v[1][h]), sel), __byte_perm(word(v[2][h]), word(v[3][h]), sel));
          }
        if (next >= 0) load_v(step + FEW_WARPS, next);
      } else if (next >= 0) {
        load_k(step + FEW_WARPS, next);
        load_v(step + FEW_WARPS, next);
      }
      page = next;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float t = l[i];
      t += __shfl_xor_sync(0xffffffffu, t, 1);
      t += __shfl_xor_sync(0xffffffffu, t, 2);
      if (c == 0) {
        ms[warp][row + 8 * i] = m[i];
        ls[warp][row + 8 * i] = t;
      }
    }
    // the warps' sums, 64 channels at a time: eight of row r to `take`, with the reference and the sum, before the division
#pragma unroll
    for (int h = 0; h < H; ++h) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          *reinterpret_cast<float2*>(&os[warp][row + 8 * i][e * 8 + 2 * c]) = make_float2(o[h * 8 + e][2 * i], o[h * 8 + e][2 * i + 1]);
      __syncthreads();
      const int r = tid >> 3, n = tid & 7;
      if (r / a.T < a.P && r % a.T < it.nq) {
        float top = ms[0][r], sum = 0.f, y[8] = {};
#pragma unroll
        for (int w = 1; w < FEW_WARPS; ++w) top = fmaxf(top, ms[w][r]);
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) {
          const float f = top == -INFINITY ? 0.f : ex2p(ms[w][r] - top);
          sum += f * ls[w][r];
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] += f * os[w][r][i * 8 + n];
        }
        take(r, h * 8 + n, top, sum, y);
      }
      __syncthreads();
    }
  };
  auto result = [&](const PromptItem& it, int r, int n, float top, float sum, float (&y)[8]) {
    const int hl = r / a.T, tok = r - hl * a.T, hq = it.h0 + hl;
    const float inv = sum == 0.f ? 0.f : 1.f / sum, lse2 = sum == 0.f ? -INFINITY : top + log2f(sum);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = sum == 0.f ? 0.f : y[i] * inv;
    const long long prow = it.q0 + tok;
    if (!CLUSTER && it.slot >= 0) {
      *part_at<D>(a, it.slot, n * 8, r) = make_float4(y[0], y[1], y[2], y[3]);
      *part_at<D>(a, it.slot, n * 8 + 4, r) = make_float4(y[4], y[5], y[6], y[7]);
      if (n == 0) a.part_lse[(long long)it.slot * a.slot_rows + r] = lse2;
      return;
    }
    *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + prow * a.out_stride[2] + hq * a.out_stride[1] + n * 8) =
        make_uint4(pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3]), pack2<T>(y[4], y[5]), pack2<T>(y[6], y[7]));
    if (n == 0 && a.lse) a.lse[hq * a.lse_rows + prow] = lse2 * 0.6931471805599453f;
  };

  if constexpr (!CLUSTER) {
    if (blockIdx.x == 0 && a.status)
      for (int s = tid; s < a.n_seqs; s += 32 * FEW_WARPS)
        if (seq_cut<true>(a, s)) kv8_record(a.status, CHECK_LENGTH);
    FewRange range(a, lane);
    PromptItem it;
    while (range.next(a, lane, tid == 0, &it))
      attend(it, it.lo, it.n, [&](int r, int n, float top, float sum, float (&y)[8]) { result(it, r, n, top, sum, y); });
    return;
  }
  uint32_t rank, ranks;
  asm("mov.u32 %0, %%cluster_ctarank;\nmov.u32 %1, %%cluster_nctarank;" : "=r"(rank), "=r"(ranks));
  PromptItem it;
  it.s = blockIdx.y;
  it.h0 = blockIdx.x / ranks * a.P;
  int k0;
  q_span<true>(a, it.s, &it.q0, &it.nq);
  k_span<true>(a, it.s, &k0, &it.nk);
  if (blockIdx.x == 0 && tid == 0 && a.status && seq_cut<true>(a, it.s)) kv8_record(a.status, CHECK_LENGTH);
  const int steps = (it.nk + FEW_KEYS - 1) / FEW_KEYS, per = (steps + ranks - 1) / ranks;
  attend(it, min(steps, (int)rank * per), min(steps, (int)(rank + 1) * per), [&](int r, int n, float top, float sum, float (&y)[8]) {
    float4* po = reinterpret_cast<float4*>(&mine[r][n * 8]);
    po[0] = make_float4(y[0], y[1], y[2], y[3]);
    po[1] = make_float4(y[4], y[5], y[6], y[7]);
    if (n == 0) {
      ms[FEW_WARPS][r] = top;
      ls[FEW_WARPS][r] = sum;
    }
  });
  cluster_meet();
  for (int e = tid * (int)ranks + (int)rank; e < FEW_ROWS * N; e += 32 * FEW_WARPS * (int)ranks) {
    const int r = e / N, n = e - r * N;
    if (r / a.T >= a.P || r % a.T >= it.nq) continue;
    const uint32_t at_m = smem_u32(&ms[FEW_WARPS][r]), at_l = smem_u32(&ls[FEW_WARPS][r]), at_o = smem_u32(&mine[r][n * 8]);
    float top = -INFINITY, sum = 0.f, y[8] = {};
    for (int k = 0; k < (int)ranks; ++k) {
      const float mk = peer_float(at_m, k), lk = peer_float(at_l, k);
      const float4 y0 = peer_float4(at_o, k), y1 = peer_float4(at_o + 16, k);
      const float t = fmaxf(top, mk), f0 = t == -INFINITY ? 0.f : ex2p(top - t), f1 = t == -INFINITY ? 0.f : ex2p(mk - t);
      const float z[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
      sum = sum * f0 + lk * f1;
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = y[i] * f0 + z[i] * f1;
      top = t;
    }
    result(it, r, n, top, sum, y);
  }
  cluster_meet();  // the others have read this CTA's
}

}  // namespace

}  // namespace qevict
