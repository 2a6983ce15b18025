// Append to the 8-bit block-scaled cache.
//
// A sequence's new tokens touch the blocks start / B .. (start + n - 1) / B.  A block that is full afterwards is
// quantised from its rows -- the old ones from the 16-bit tail, the new ones from the call's input -- the tokens of
// the block that stays open go to the tail.
//     scale = RN(amax / M), code = nearest(RN(x / scale)),  M = 127 (int8) or 448 (e4m3)
// with IEEE float32 divisions, so the codes are a function of the values alone (a zero of either sign has code 0).
//
// One CTA per (block of the call, KV head and K or V, sequence): the block's rows are read once, into registers, the
// maximum is taken over the CTA and the codes are written from the same registers.  Bandwidth bounds prompts (3 bytes
// an element), latency single tokens (four prompts of up to 16001 tokens x 8 heads of 128: 49 us, 0.81 of the bandwidth; 16 single
// tokens: 2.3 us).  The divisions are what could cost more than the traffic; all of a block's have the
// same divisor, so its reciprocal is taken once and each quotient costs five multiply-adds (see `quotients`).
// The tail has room for one block, and the CTA of the call's first block is the only one that reads it; it also writes
// the rows of the block that stays open, after it has read the old ones.
#include "kv8.cuh"

namespace qevict {

namespace {

constexpr int APPEND_CTAS = 4096;  // a CTA takes several (head, K or V) pairs where there are more than these

struct Kv8AppendArgs {
  Kv8View c;
  const void* src[2];
  long long token_stride, head_stride, total_new;
  const int32_t* start;
  const int32_t* cu_new;
  int max_new;
  int per_cta;  // (head, K or V) pairs that a CTA takes one after the other
};

// x / b rounded to nearest, for b in [2^-60, 2^60] and r = 1 / b rounded to nearest: the product x r is within 2 ulp; one
// correction by the exact remainder brings it within 1 ulp, and from there one more gives the correctly rounded quotient
// (Markstein 1990).  Where x is so small that a remainder is not exact, the quotient is far below half a code.
// Two at a time: packed float32 instructions halve what has to be issued.
__device__ __forceinline__ uint64_t quotient2(uint64_t x, uint64_t nb, uint64_t r) {  // nb: -b twice
  uint64_t q = fma2(x, r, 0ull);
  q = fma2(fma2(nb, q, x), r, q);
  return fma2(fma2(nb, q, x), r, q);
}

// Four pairs of quotients -> eight codes.
template <int CODE> __device__ __forceinline__ uint2 encode8(const uint64_t (&y)[4]) {
  uint2 r;
  if (CODE == QEVICT_CODE_INT8) {
    // 1.5 * 2^23 + y rounds y to the nearest integer, ties to even, and leaves it in the low byte; |y| <= 127 (1 + 2^-23)
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      unpair(add2(y[i], pair(12582912.f, 12582912.f)), a, b);
      h[i] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040);
    }
    r.x = __byte_perm(h[0], h[1], 0x5410);
    r.y = __byte_perm(h[2], h[3], 0x5410);
  } else {
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      unpair(y[i], a, b);
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(h[i]) : "f"(b), "f"(a));
    }
    r.x = (uint32_t)h[0] | ((uint32_t)h[1] << 16);
    r.y = (uint32_t)h[2] | ((uint32_t)h[3] << 16);
  }
  return r;
}

template <class T> __device__ __forceinline__ uint64_t floats_of(uint32_t w);
template <> __device__ __forceinline__ uint64_t floats_of<__nv_bfloat16>(uint32_t w) {
  return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ uint64_t floats_of<__half>(uint32_t w) {
  const float2 f = __half22float2(as_t2<__half2>(w));
  return pair(f.x, f.y);
}

// Rows of a sequence that are not stored: beyond the bound, outside the input, of falling bounds.
__device__ __noinline__ void check_rows(const int32_t* cu_new, int32_t* status, int s, int max_new, long long total_new) {
  const long long c0 = cu_new[s], c1 = cu_new[s + 1];
  if (c1 < c0 || c1 - c0 > max_new || (c1 > c0 && (c0 < 0 || c1 > total_new))) kv8_record(status, CHECK_LENGTH);
}

// NT threads, NV 16-byte vectors of the block in each: NT * NV = block * D / 8.
template <class T, int CODE, int D, int NT, int NV>
__global__ void __launch_bounds__(NT, NV <= 4 ? 10 : 640 / NT) kv8_append_kernel(const Kv8AppendArgs a) {
  const Kv8View& c = a.c;
  constexpr int nt = NT;
  const int tid = threadIdx.x;
  const int n_hw = 2 * c.Hkv, chunks = (n_hw + a.per_cta - 1) / a.per_cta;
  const int s = blockIdx.y, bx = blockIdx.x / chunks, hw0 = (blockIdx.x - bx * chunks) * a.per_cta, hw1 = min(n_hw, hw0 + a.per_cta);
  constexpr int VR = D / 8;  // vectors per row
  const int B = c.block;
  __shared__ __align__(16) uint32_t red[2][NT / 32];
  pdl_prologue();
  // a CTA of its own for each sequence: in the others these comparisons change the schedule of everything behind them (4 to 10 %)
  if (a.cu_new && blockIdx.x == gridDim.x - 1) {
    if (tid == 0 && a.start[s] >= 0) check_rows(a.cu_new, c.status, s, a.max_new, a.total_new);
    return;
  }
  const int st = a.start[s];
  long long row0 = s;
  int n = 1;
  if (a.cu_new) {
    const int c0 = a.cu_new[s], c1 = a.cu_new[s + 1];
    row0 = c0;
    n = c1 > c0 ? (int)min((long long)a.max_new, (long long)c1 - c0) : 0;
  }
  if (st < 0 || n <= 0 || row0 < 0 || row0 + n > a.total_new) return;  // the whole CTA leaves
  const long long cap = (long long)c.max_blocks * B;
  if ((long long)st + n > cap) {
    if (tid == 0 && blockIdx.x == 0) kv8_record(c.status, CHECK_LENGTH);
    n = (int)(cap - st);
    if (n <= 0) return;
  }
  const int first = st / B, end = st + n, last_open = end / B;  // last_open: block that stays open (rows 0 .. end % B)
  const int blk = first + bx, pos0 = blk * B;
  const bool full = blk < last_open;  // full after this call
  if (!full && bx > 0) return;
  const int page = full ? c.table[(size_t)s * c.max_blocks + blk] : -1;
  const bool there = page >= 0 && page < c.n_pages;
  if (full && !there && page != -1 && tid == 0) kv8_record(c.status, CHECK_PAGE_ID);
  auto input = [&](int hw) {  // head hw % Hkv of K (hw < Hkv) or V, this sequence's first new row
    const int w = hw >= c.Hkv;
    return static_cast<const T*>(w ? a.src[1] : a.src[0]) + row0 * a.token_stride + (long long)(hw - w * c.Hkv) * a.head_stride;
  };
  auto tail_of = [&](int hw) {
    const int w = hw >= c.Hkv;
    return static_cast<T*>(w ? c.tail[1] : c.tail[0]) + ((size_t)s * c.Hkv + (hw - w * c.Hkv)) * B * D;
  };
  // this thread's vectors lie nt / VR rows apart
  const int r0 = tid / VR, step = nt / VR;
  auto load = [&](int hw, uint4 (&x)[NV]) {
    const T* src = input(hw) + (tid & (VR - 1)) * 8;
    if (pos0 >= st) {  // all of the block is new
      const T* p = src + (long long)(pos0 + r0 - st) * a.token_stride;
      const long long d = (long long)step * a.token_stride;
#pragma unroll
      for (int i = 0; i < NV; ++i, p += d) x[i] = *reinterpret_cast<const uint4*>(p);
    } else {
      const T* tail = tail_of(hw) + (tid & (VR - 1)) * 8;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int r = r0 + i * step, pos = pos0 + r;
        x[i] = *reinterpret_cast<const uint4*>(pos < st ? tail + (size_t)r * D : src + (long long)(pos - st) * a.token_stride);
      }
    }
  };
  // one (head, K or V) after the other; the next one's rows are on their way while this one's codes are made
  uint4 x[NV], ahead[NV];
  if (full && there) load(hw0, x);
  for (int hw = hw0; hw < hw1; ++hw) {
    if (full && there) {
      if (hw + 1 < hw1) load(hw + 1, ahead);
      uint32_t m2 = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i) {  // magnitudes of 16-bit floats order like their bits (NaN above infinity)
        m2 = __vmaxu2(m2, __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu),
                                   __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu)));
      }
      uint32_t m = max(m2 & 0xffffu, m2 >> 16);
      m = __reduce_max_sync(0xffffffffu, m);
      uint32_t* mine = red[(hw - hw0) & 1];
      if ((tid & 31) == 0) mine[tid >> 5] = m;
      __syncthreads();
      m = 0;
#pragma unroll
      for (int i = 0; i < NT / 128; ++i) {
        const uint4 p = reinterpret_cast<const uint4*>(mine)[i];
        m = max(m, max(max(p.x, p.y), max(p.z, p.w)));
      }
      const uint16_t mb = (uint16_t)m;
      const float amax = Tr<T>::to_float(*reinterpret_cast<const T*>(&mb));
      float scale = __fdiv_rn(amax, CODE == QEVICT_CODE_INT8 ? 127.f : 448.f);
      const bool finite = isfinite(amax);
      if (!finite || !(scale > 0.f)) scale = 1.f;
      const int w = hw >= c.Hkv;
      const size_t ph = (size_t)page * c.Hkv + (hw - w * c.Hkv);
      uint2* dst = reinterpret_cast<uint2*>((w ? c.codes[1] : c.codes[0]) + ph * B * D) + tid;
      if (!finite) {
#pragma unroll
        for (int i = 0; i < NV; ++i) dst[i * nt] = make_uint2(0u, 0u);
      } else if (scale >= 0x1p-60f && scale <= 0x1p60f) {
        const float r = __frcp_rn(scale);
        const uint64_t nb2 = pair(-scale, -scale), r2 = pair(r, r);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          uint64_t y[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) y[k] = quotient2(floats_of<T>(k == 0 ? x[i].x : k == 1 ? x[i].y : k == 2 ? x[i].z : x[i].w), nb2, r2);
          dst[i * nt] = encode8<CODE>(y);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          uint64_t y[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float f0, f1;
            unpair(floats_of<T>(k == 0 ? x[i].x : k == 1 ? x[i].y : k == 2 ? x[i].z : x[i].w), f0, f1);
            y[k] = pair(__fdiv_rn(f0 + 0.f, scale), __fdiv_rn(f1 + 0.f, scale));  // (-0 becomes 0, as in `quotient2`)
          }
          dst[i * nt] = encode8<CODE>(y);
        }
      }
      if (tid == 0) {
        (w ? c.scale[1] : c.scale[0])[ph] = scale;
        if (!finite) kv8_record(c.status, CHECK_NOT_FINITE);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) x[i] = ahead[i];
    }
    if (bx == 0) {  // rows of the open block (behind the reads of the old ones above: one block, one CTA)
      if (!(full && there)) __syncthreads();
      const T* src = input(hw);
      T* tail = tail_of(hw);
      const int from = max(st, last_open * B), rows = end - from;
      for (int v = tid; v < rows * VR; v += nt) {
        const int r = v / VR, cv = v - r * VR;
        reinterpret_cast<uint4*>(tail + (size_t)(from + r - last_open * B) * D)[cv] =
            *(reinterpret_cast<const uint4*>(src + (long long)(from + r - st) * a.token_stride) + cv);
      }
    }
  }
}

template <class T, int CODE, int D> cudaError_t launch_append(const Kv8AppendArgs& a, dim3 grid, cudaStream_t s) {
  switch (a.c.block * D / 8) {  // 16 tokens of 64 channels: 128 vectors, 128 of 128: 2048
    case 128: return launch_pdl(kv8_append_kernel<T, CODE, D, 128, 1>, grid, dim3(128), 0, s, a);
    case 256: return launch_pdl(kv8_append_kernel<T, CODE, D, 128, 2>, grid, dim3(128), 0, s, a);
    case 512: return launch_pdl(kv8_append_kernel<T, CODE, D, 128, 4>, grid, dim3(128), 0, s, a);
    case 1024: return launch_pdl(kv8_append_kernel<T, CODE, D, 128, 8>, grid, dim3(128), 0, s, a);
    default: return launch_pdl(kv8_append_kernel<T, CODE, D, 256, 8>, grid, dim3(256), 0, s, a);  // (the registers of a thread end at 8)
  }
}
template <class T, int CODE> cudaError_t launch_append_d(const Kv8AppendArgs& a, dim3 grid, cudaStream_t s) {
  return a.c.D == 128 ? launch_append<T, CODE, 128>(a, grid, s) : launch_append<T, CODE, 64>(a, grid, s);
}

}  // namespace

}  // namespace qevict

using namespace qevict;

extern "C" QEVICT_API qevict_status qevict_kv8_append(const qevict_kv8_cache* cache, const void* k, const void* v,
                                                      int64_t token_stride, int64_t head_stride, int64_t total_new,
                                                      const int32_t* start, const int32_t* cu_new, int32_t max_new, void* stream) {
  Kv8AppendArgs a;
  qevict_status st;
  const char* why = kv8_check(cache, &st, &a.c);
  if (why) return stateless_fail(st, why);
  if (total_new < 0 || max_new < 0) return stateless_fail(QEVICT_ERR_INVALID_ARG, "total_new and max_new must be >= 0");
  if (!cu_new && max_new > 1) return stateless_fail(QEVICT_ERR_INVALID_ARG, "without cu_new every sequence has one token: max_new must be 0 or 1");
  if (!cu_new && max_new == 1 && total_new < a.c.n_seqs) return stateless_fail(QEVICT_ERR_INVALID_ARG, "without cu_new total_new must be at least n_seqs");
  if (a.c.n_seqs == 0 || max_new == 0 || total_new == 0) return QEVICT_OK;
  if (!k || !v || !start) return stateless_fail(QEVICT_ERR_INVALID_ARG, "k, v and start must not be NULL");
  if (misaligned16(k) || misaligned16(v) || token_stride % 8 || head_stride % 8)
    return stateless_fail(QEVICT_ERR_INVALID_ARG, "k, v and their strides must be multiples of 16 bytes");
  if (misaligned4(start) || misaligned4(cu_new)) return stateless_fail(QEVICT_ERR_INVALID_ARG, "start and cu_new must be 4-byte aligned");
  if (token_stride < 0 || head_stride < 0) return stateless_fail(QEVICT_ERR_INVALID_ARG, "strides must be >= 0");
  if (max_new > total_new) max_new = (int32_t)total_new;
  if (max_new > (1 << 30)) return stateless_fail(QEVICT_ERR_UNSUPPORTED, "more than 2^30 tokens in one call");
  a.src[0] = k; a.src[1] = v;
  a.token_stride = token_stride; a.head_stride = head_stride; a.total_new = total_new;
  a.start = start; a.cu_new = cu_new; a.max_new = max_new;
  // blocks that max_new tokens can touch, wherever they start
  const long long touched = ((long long)max_new + a.c.block - 2) / a.c.block + 1;
  const long long blocks = touched < a.c.max_blocks ? touched : a.c.max_blocks;
  if (blocks * 2 * a.c.Hkv >= 0x7fffffffll) return stateless_fail(QEVICT_ERR_UNSUPPORTED, "max_new * n_kv_heads is too large for one call");
  // Few blocks: one pair per CTA, for the latency.  Many: several, so that the start of a CTA (lengths, page, first rows: three
  // dependent reads) is paid less often (measured when it was chosen, with the code of then: 39k tokens x 8 heads of 128 53 us with at most 4096 CTAs, 68 us
  // with half of that, 84 us with one pair per CTA; 12 pieces of up to 2k tokens x 4 heads: 13, 17 and 23 us.  CTAs of 256
  // threads: 56 and 15 us; of 512: 75 and 23 us).
  a.per_cta = 1;
  while (a.per_cta < 8 && a.per_cta < 2 * a.c.Hkv && blocks * a.c.n_seqs * 2 * a.c.Hkv > (long long)a.per_cta * APPEND_CTAS) a.per_cta *= 2;
  const long long chunks = (2 * a.c.Hkv + a.per_cta - 1) / a.per_cta;
  DeviceGuard guard(cache->device);
  cudaError_t e = guard.err;
  cudaStream_t s = (cudaStream_t)stream;
  dim3 grid((unsigned)(blocks * chunks) + (cu_new ? 1 : 0), a.c.n_seqs);
  if (e == cudaSuccess) {
    const bool i8 = cache->code == QEVICT_CODE_INT8;
    if (cache->dtype == QEVICT_DTYPE_FP16)
      e = i8 ? launch_append_d<__half, QEVICT_CODE_INT8>(a, grid, s) : launch_append_d<__half, QEVICT_CODE_E4M3>(a, grid, s);
    else
      e = i8 ? launch_append_d<__nv_bfloat16, QEVICT_CODE_INT8>(a, grid, s) : launch_append_d<__nv_bfloat16, QEVICT_CODE_E4M3>(a, grid, s);
  }
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  return QEVICT_OK;
}
