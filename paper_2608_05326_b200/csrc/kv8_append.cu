// Append to the 8-bit block-scaled cache.
//
// A sequence's new tokens touch the blocks start / B .. (start + n - 1) / B.  A block that is full afterwards is
// quantised from its rows -- the old ones from the 16-bit tail, the new ones from the call's input -- the tokens of
// the block that stays open go to the tail.
//     scale = RN(amax / M), code = nearest(RN(x / scale)),  M = 127 (int8) or 448 (e4m3)
// with IEEE float32 divisions, so the codes are a function of the values alone.
//
// One CTA per (block of the call, KV head and K or V, sequence): the block's rows are read once, into registers, the
// maximum is taken over the CTA and the codes are written from the same registers.  The work per element is a few
// dozen instructions against 3 bytes of traffic: bandwidth for prompts, latency for single tokens.
// The tail has room for one block, and the CTA of the call's first block is the only one that reads it; it also writes
// the rows of the block that stays open, after it has read the old ones.
#include "kv8.cuh"

namespace qevict {

namespace {

constexpr int APPEND_THREADS = 256;

struct Kv8AppendArgs {
  Kv8View c;
  const void* src[2];
  long long token_stride, head_stride, total_new;
  const int32_t* start;
  const int32_t* cu_new;
  int max_new;
};

template <int CODE> __device__ __forceinline__ uint2 encode8(const float (&y)[8]) {
  uint2 r;
  if (CODE == QEVICT_CODE_INT8) {
    // 1.5 * 2^23 + y rounds y to the nearest integer, ties to even, and leaves it in the low byte
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(fminf(fmaxf(y[i], -127.f), 127.f) + 12582912.f);
    r.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    r.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
  } else {
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(h[i]) : "f"(y[2 * i + 1]), "f"(y[2 * i]));
    r.x = (uint32_t)h[0] | ((uint32_t)h[1] << 16);
    r.y = (uint32_t)h[2] | ((uint32_t)h[3] << 16);
  }
  return r;
}

// NV: 16-byte vectors a thread holds of the block (block * D / 8 / threads).
template <class T, int CODE, int NV>
__global__ void __launch_bounds__(APPEND_THREADS) kv8_append_kernel(const Kv8AppendArgs a) {
  const Kv8View& c = a.c;
  const int s = blockIdx.z, h = blockIdx.y >> 1, w = blockIdx.y & 1, tid = threadIdx.x, nt = blockDim.x;
  const int B = c.block, D = c.D, VR = D >> 3;  // vectors per row
  __shared__ uint32_t red[APPEND_THREADS / 32];
  pdl_prologue();
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
    if (tid == 0 && blockIdx.x == 0 && blockIdx.y == 0) kv8_record(c.status, CHECK_LENGTH);
    n = (int)(cap - st);
    if (n <= 0) return;
  }
  const int first = st / B, end = st + n, last_open = end / B;  // last_open: block that stays open (rows 0 .. end % B)
  const int blk = first + blockIdx.x;
  const T* src = static_cast<const T*>(a.src[w]) + row0 * a.token_stride + (long long)h * a.head_stride;
  T* tail = static_cast<T*>(c.tail[w]) + ((size_t)s * c.Hkv + h) * B * D;

  if (blk < last_open) {  // a block that is full now
    const int pos0 = blk * B;
    uint4 x[NV];
    uint32_t m2 = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = tid + i * nt, r = v / VR, cv = v - r * VR, pos = pos0 + r;
      const T* p = pos < st ? tail + (size_t)r * D : src + (long long)(pos - st) * a.token_stride;
      x[i] = *(reinterpret_cast<const uint4*>(p) + cv);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {  // magnitudes of 16-bit floats order like their bits (NaN above infinity)
      m2 = __vmaxu2(m2, __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu),
                                 __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu)));
    }
    uint32_t m = max(m2 & 0xffffu, m2 >> 16);
    m = __reduce_max_sync(0xffffffffu, m);
    if ((tid & 31) == 0) red[tid >> 5] = m;
    __syncthreads();
    m = 0;
    for (int i = 0; i < (nt >> 5); ++i) m = max(m, red[i]);
    const uint16_t mb = (uint16_t)m;
    const float amax = Tr<T>::to_float(*reinterpret_cast<const T*>(&mb));
    float scale = __fdiv_rn(amax, CODE == QEVICT_CODE_INT8 ? 127.f : 448.f);
    const bool finite = isfinite(amax);
    if (!finite || !(scale > 0.f)) scale = 1.f;
    const int page = c.table[(size_t)s * c.max_blocks + blk];
    if (page >= 0 && page < c.n_pages) {
      uint2* dst = reinterpret_cast<uint2*>(c.codes[w] + ((size_t)page * c.Hkv + h) * B * D);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const T* e = reinterpret_cast<const T*>(&x[i]);
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = finite ? __fdiv_rn(Tr<T>::to_float(e[j]), scale) : 0.f;
        dst[tid + i * nt] = encode8<CODE>(y);
      }
      if (tid == 0) c.scale[w][(size_t)page * c.Hkv + h] = scale;
    } else if (tid == 0 && page != -1) {
      kv8_record(c.status, CHECK_PAGE_ID);
    }
  }
  if (blockIdx.x == 0) {  // rows of the open block (behind the reads of the old ones above: one block, one CTA)
    __syncthreads();
    const int from = max(st, last_open * B), rows = end - from;
    for (int v = tid; v < rows * VR; v += nt) {
      const int r = v / VR, cv = v - r * VR;
      reinterpret_cast<uint4*>(tail + (size_t)(from + r - last_open * B) * D)[cv] =
          *(reinterpret_cast<const uint4*>(src + (long long)(from + r - st) * a.token_stride) + cv);
    }
  }
}

template <class T, int CODE> cudaError_t launch_append(const Kv8AppendArgs& a, dim3 grid, cudaStream_t s) {
  const int nvec = a.c.block * a.c.D / 8;
  const int nt = nvec < APPEND_THREADS ? nvec : APPEND_THREADS;
  switch (nvec / nt) {
    case 1: return launch_pdl(kv8_append_kernel<T, CODE, 1>, grid, dim3(nt), 0, s, a);
    case 2: return launch_pdl(kv8_append_kernel<T, CODE, 2>, grid, dim3(nt), 0, s, a);
    case 4: return launch_pdl(kv8_append_kernel<T, CODE, 4>, grid, dim3(nt), 0, s, a);
    default: return launch_pdl(kv8_append_kernel<T, CODE, 8>, grid, dim3(nt), 0, s, a);
  }
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
  const int blocks = (int)(touched < a.c.max_blocks ? touched : a.c.max_blocks);
  DeviceGuard guard(cache->device);
  cudaError_t e = guard.err;
  cudaStream_t s = (cudaStream_t)stream;
  dim3 grid(blocks, 2 * a.c.Hkv, a.c.n_seqs);
  if (e == cudaSuccess) {
    const bool i8 = cache->code == QEVICT_CODE_INT8;
    if (cache->dtype == QEVICT_DTYPE_FP16)
      e = i8 ? launch_append<__half, QEVICT_CODE_INT8>(a, grid, s) : launch_append<__half, QEVICT_CODE_E4M3>(a, grid, s);
    else
      e = i8 ? launch_append<__nv_bfloat16, QEVICT_CODE_INT8>(a, grid, s) : launch_append<__nv_bfloat16, QEVICT_CODE_E4M3>(a, grid, s);
  }
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  return QEVICT_OK;
}
