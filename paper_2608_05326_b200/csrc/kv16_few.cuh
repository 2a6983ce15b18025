// Attention of few new tokens (a step of decoding, drafts) over the 16-bit paged cache.
//
//     S = Q K^T,  P = 2^(S * scale * log2 e - m),  O += P V
//
// The rows are the tokens of all heads that share a KV head, at most 16 MT of them, so keys and values are read once and
// bandwidth bounds it.  A CTA has an equal range of the call's work (PagedRange, 16 keys at a time); its four warps
// take 16 keys in turn, straight from global memory into the registers that the products want them in, the next ones on their way
// while these are in work, and join their sums through shared memory when the sequence or the range ends.
//   - mma.m16n8k16 contracts over channels in any order, so a lane takes 16 bytes of a key as the operands of two steps (elements
//     0, 1 | 2, 3 and 4, 5 | 6, 7), and the queries are laid out to match.
//   - A lane has 16 bytes of two neighbouring keys' values; byte permutes pair them, and the output's columns come in the order
//     that this gives (channel 8 n + e is column n of step e).
//   - Keys past the end and blocks that are not there are not read; their operands are zero and their logits masked.
#pragma once

#include "prompt_attn.cuh"

namespace qevict {

namespace {

constexpr int FEW_WARPS = 4, FEW_KEYS = 16;
constexpr int FEW_ITEM_COST = 256, FEW_RANGE_LEAST = 512;
template <int D, int MT> constexpr int few_ctas() { return MT == 1 ? 3 : 2; }  // of an SM: 168 or 255 registers a thread
template <int D, int MT> constexpr int few_smem() { return MT * D / 32 * 1024 + FEW_WARPS * MT * 16 * (D + 8 + 2) * 4; }

__device__ __forceinline__ uint4 ld_page16(const void* p) {
  uint4 r;
  asm("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
  return r;
}

struct FewPages {
  const void* pages[2];
  long long stride[2][3];
  const void* q;
  long long q_stride[2];  // token, head
};

template <class T, int D, int MT>
__global__ void __launch_bounds__(32 * FEW_WARPS, few_ctas<D, MT>()) few_attn_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ FewPages g) {
  constexpr int J = D / 32;       // 16-byte pieces of a key in a lane
  constexpr int N = D / 8;        // column steps of the output
  constexpr int LINE = D + 8;     // floats from row to row in shared memory
  constexpr int ROWS = MT * 16;
  extern __shared__ __align__(16) unsigned char few_sm[];
  auto qf = reinterpret_cast<uint4 (*)[2 * J][32]>(few_sm);                         // queries, [MT]
  auto os = reinterpret_cast<float (*)[ROWS][LINE]>(few_sm + MT * J * 1024);         // the warps' outputs, [FEW_WARPS]
  auto ms = reinterpret_cast<float (*)[ROWS]>(os + FEW_WARPS), ls = ms + FEW_WARPS;  // their references and sums
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = lane >> 2, c = lane & 3;
  pdl_prologue();
  if (a.cuts && tid == 0) a.cuts[blockIdx.x].valid = 0;
  if (blockIdx.x == 0 && a.status)
    for (int s = tid; s < a.n_seqs; s += 32 * FEW_WARPS)
      if (seq_cut<true>(a, s)) kv8_record(a.status, CHECK_LENGTH);
  PagedRange<FEW_KEYS, FEW_ITEM_COST, FEW_RANGE_LEAST> range(a, lane);
  PromptItem it;
  while (range.next(a, warp == 0 ? lane : 1, &it)) {
    const int hk = it.h0 / a.P, f0 = it.lo, f1 = it.n;
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
    // queries, in the order of the operands
    for (int e = tid; e < MT * 2 * J * 32; e += 32 * FEW_WARPS) {
      const int l = e & 31, ju = (e >> 5) % (2 * J), mt = (e >> 5) / (2 * J);
      const int ch = ((l & 3) + 4 * (ju >> 1)) * 8 + (ju & 1) * 4;
      uint2 v[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = mt * 16 + (l >> 2) + 8 * i, hl = r / a.T, tok = r - hl * a.T;
        v[i] = make_uint2(0u, 0u);
        if (hl < a.P && tok < it.nq)
          v[i] = *reinterpret_cast<const uint2*>(static_cast<const T*>(g.q) + (long long)(it.q0 + tok) * g.q_stride[0] + (long long)(it.h0 + hl) * g.q_stride[1] + ch);
      }
      qf[mt][ju][l] = make_uint4(v[0].x, v[1].x, v[0].y, v[1].y);
    }
    // keys that the rows of this lane see
    int sees[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = mt * 16 + row + 8 * i, tok = r - r / a.T * a.T;
        sees[mt][i] = a.causal ? min(it.nk, it.nk - it.nq + tok + 1) : it.nk;
      }
    const int all_see = a.causal ? it.nk - it.nq + 1 : it.nk;  // keys that every row sees
    float o[MT][N][4], m[MT][2], l[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int n = 0; n < N; ++n) o[mt][n][0] = o[mt][n][1] = o[mt][n][2] = o[mt][n][3] = 0.f;
      m[mt][0] = m[mt][1] = -INFINITY;
      l[mt][0] = l[mt][1] = 0.f;
    }
    uint4 k[2][J], v[4][D / 64];
    // this lane's parts of the keys and values of a step; rows past the end are zero
    auto base = [&](int w, int step, int page) {
      const int t = (step * FEW_KEYS) & ((1 << a.block_log2) - 1);
      return static_cast<const T*>(g.pages[w]) + page * g.stride[w][0] + hk * g.stride[w][1] + t * g.stride[w][2];
    };
    auto load_k = [&](int step, int page) {
      const T* p = base(0, step, page) + c * 8;
      const int left = it.nk - step * FEW_KEYS;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int j = 0; j < J; ++j)
          k[n][j] = n * 8 + row < left ? ld_page16(p + (n * 8 + row) * g.stride[0][2] + j * 32) : make_uint4(0u, 0u, 0u, 0u);
    };
    auto load_v = [&](int step, int page) {
      const T* p = base(1, step, page) + row * 8;
      const int left = it.nk - step * FEW_KEYS;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = 2 * c + (i & 1) + (i >> 1) * 8;
#pragma unroll
        for (int h = 0; h < D / 64; ++h)
          v[i][h] = key < left ? ld_page16(p + key * g.stride[1][2] + h * 64) : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    int step = f0 + warp, at = 0;
    int page = __shfl_sync(0xffffffffu, ids, 0);
    if (step < f1 && page >= 0) {
      load_k(step, page);
      load_v(step, page);
    }
    __syncthreads();
    for (; step < f1; step += FEW_WARPS) {
      int next = -1;
      if (step + FEW_WARPS < f1) {
        if (((++at) & 31) == 0) ids = fetch(at);
        next = __shfl_sync(0xffffffffu, ids, at & 31);
      }
      if (page < 0) {  // not there
        page = next;
        if (page >= 0) {
          load_k(step + FEW_WARPS, page);
          load_v(step + FEW_WARPS, page);
        }
        continue;
      }
      float x[MT][2][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int n = 0; n < 2; ++n) x[mt][n][0] = x[mt][n][1] = x[mt][n][2] = x[mt][n][3] = 0.f;
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const uint4 q0 = qf[mt][2 * j][lane], q1 = qf[mt][2 * j + 1][lane];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            mma16816<T>(x[mt][n], q0.x, q0.y, q0.z, q0.w, k[n][j].x, k[n][j].y);
            mma16816<T>(x[mt][n], q1.x, q1.y, q1.z, q1.w, k[n][j].z, k[n][j].w);
          }
        }
      if (next >= 0) load_k(step + FEW_WARPS, next);
      const int key0 = step * FEW_KEYS;
      if (key0 + FEW_KEYS > all_see) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + n * 8 + 2 * c + (i & 1) >= sees[mt][i >> 1]) x[mt][n][i] = -INFINITY;
      }
      uint32_t p[MT][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        bool moves = false;
        float top[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float t = fmaxf(fmaxf(x[mt][0][2 * i], x[mt][0][2 * i + 1]), fmaxf(x[mt][1][2 * i], x[mt][1][2 * i + 1]));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
          top[i] = t * a.scale_log2;
          moves = moves || top[i] > m[mt][i] + PROMPT_LAZY;
        }
        if (__any_sync(0xffffffffu, moves)) {  // each row by its own logits: what else is in the tile has no say
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (!(top[i] > m[mt][i] + PROMPT_LAZY)) continue;
            const float f = ex2p(m[mt][i] - top[i]);
            m[mt][i] = top[i];
            l[mt][i] *= f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
              o[mt][n][2 * i] *= f;
              o[mt][n][2 * i + 1] *= f;
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float sub = m[mt][i] == -INFINITY ? 0.f : -m[mt][i];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const float e0 = ex2p(fmaf(x[mt][n][2 * i], a.scale_log2, sub)), e1 = ex2p(fmaf(x[mt][n][2 * i + 1], a.scale_log2, sub));
            l[mt][i] += e0 + e1;
            p[mt][2 * n + i] = pack2<T>(e0, e1);
          }
        }
      }
#pragma unroll
      for (int h = 0; h < D / 64; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int sel = e & 1 ? 0x7632 : 0x5410;
          auto word = [&](const uint4& u) { return e < 2 ? u.x : e < 4 ? u.y : e < 6 ? u.z : u.w; };
          const uint32_t b0 = __byte_perm(word(v[0][h]), word(v[1][h]), sel), b1 = __byte_perm(word(v[2][h]), word(v[3][h]), sel);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) mma16816<T>(o[mt][h * 8 + e], p[mt][0], p[mt][1], p[mt][2], p[mt][3], b0, b1);
        }
      if (next >= 0) load_v(step + FEW_WARPS, next);
      page = next;
    }
    // the warps' sums
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = mt * 16 + row + 8 * i;
        float t = l[mt][i];
        t += __shfl_xor_sync(0xffffffffu, t, 1);
        t += __shfl_xor_sync(0xffffffffu, t, 2);
        if (c == 0) {
          ms[warp][r] = m[mt][i];
          ls[warp][r] = t;
        }
#pragma unroll
        for (int n = 0; n < N; ++n) *reinterpret_cast<float2*>(&os[warp][r][n * 8 + 2 * c]) = make_float2(o[mt][n][2 * i], o[mt][n][2 * i + 1]);
      }
    __syncthreads();
    for (int e = tid; e < MT * 16 * N; e += 32 * FEW_WARPS) {  // eight channels of a row
      const int r = e / N, n = e - r * N, hl = r / a.T, tok = r - hl * a.T;
      if (hl >= a.P) break;
      if (tok >= it.nq) continue;
      float top = ms[0][r];
#pragma unroll
      for (int w = 1; w < FEW_WARPS; ++w) top = fmaxf(top, ms[w][r]);
      float sum = 0.f, y[8] = {};
#pragma unroll
      for (int w = 0; w < FEW_WARPS; ++w) {
        const float f = top == -INFINITY ? 0.f : ex2p(ms[w][r] - top);
        sum += f * ls[w][r];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] += f * os[w][r][(n >> 3) * 64 + i * 8 + (n & 7)];
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum, lse2 = sum == 0.f ? -INFINITY : top + log2f(sum);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = sum == 0.f ? 0.f : y[i] * inv;
      const long long prow = it.q0 + tok, slot = (long long)it.slot * a.slot_rows + r;
      const int hq = it.h0 + hl;
      if (it.slot >= 0) {
        float4* po = reinterpret_cast<float4*>(a.part_o + slot * D + n * 8);
        po[0] = make_float4(y[0], y[1], y[2], y[3]);
        po[1] = make_float4(y[4], y[5], y[6], y[7]);
        if (n == 0) a.part_lse[slot] = lse2;
      } else {
        *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + prow * a.out_stride[2] + hq * a.out_stride[1] + n * 8) =
            make_uint4(pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3]), pack2<T>(y[4], y[5]), pack2<T>(y[6], y[7]));
        if (n == 0 && a.lse) a.lse[hq * a.lse_rows + prow] = lse2 * 0.6931471805599453f;
      }
    }
    __syncthreads();
  }
}

}  // namespace

}  // namespace qevict
