// Rotary positions by themselves, and on the way into the 16-bit paged cache.
//
//     theta = position[axis[p]] * inv_freq[p],   (x, y) -> scale * (x cos theta - y sin theta, y cos theta + x sin theta)
//
// Bandwidth bounds it: an element is read once and written once.  The angle is the same for all heads of a token, so a CTA takes a
// few tokens and goes over their heads: cosines and sines are computed once per CTA (the angle in turns in 64 bits, its
// fraction in float32, then sincospif) and each thread keeps those of its pairs in registers from head to head.  Rows
// are requested before the angles are computed and, for the cache, before the place of the token is looked up (bounds,
// start, page: three dependent reads), the next heads' before the present ones are turned.  Measured: 16384 tokens x 32 heads
// of 128, three axes 46 us (5.8 TB/s, 0.89 of the copy bandwidth); four prompts of up to 16001 tokens x 48 heads into the cache 168 us
// (6.1 TB/s); 16 tokens 2.8 and 3.9 us.
#include "kv16.cuh"

namespace qevict {

namespace {

constexpr int ROTARY_THREADS = 256;
constexpr int MAX_TOKENS = 8;  // of a CTA

struct RotaryArgs {
  double turns[128];  // inv_freq / 2 pi
  uint8_t axis[128];
  int n_pairs, interleaved;
  float scale, sin_scale;  // sin_scale: negative for the inverse
  int D, U;                // channels; units of 2 V channels in a head
  int heads[3];            // queries, keys (both rotated), values
  int T, HL;               // tokens of a CTA, heads side by side
  const void* src[3];
  long long src_token[3], src_head[3];
  void* dst[2];            // queries, keys (without a cache)
  long long dst_token[2], dst_head[2];
  const int32_t* positions;
  long long axis_stride, rows;
  // cache
  Kv16View c;
  const int32_t* start;
  const int32_t* cu;
};

template <int V> struct Vec;
template <> struct Vec<8> { using type = uint4; };
template <> struct Vec<4> { using type = uint2; };

template <int V> __device__ __forceinline__ typename Vec<V>::type load_row(const void* p) {
  typename Vec<V>::type r;
  if constexpr (V == 8) {
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
  } else {
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];\n" : "=r"(r.x), "=r"(r.y) : "l"(p) : "memory");
  }
  return r;
}

// Rows of the sequences that are not stored although the call has them: falling bounds, rows outside the input.
__device__ __noinline__ void check_bounds(const RotaryArgs& a) {
  for (int s = threadIdx.x; s < a.c.n_seqs; s += ROTARY_THREADS) {
    const long long c0 = a.cu[s], c1 = a.cu[s + 1];
    if (a.start[s] >= 0 && (c1 < c0 || (c1 > c0 && (c0 < 0 || c1 > a.rows)))) kv8_record(a.c.status, CHECK_LENGTH);
  }
}

// V: channels of a vector; a unit is two vectors, V pairs.  NB: units that a thread has in flight.
template <class T, int V, int NB, bool CACHE>
__global__ void __launch_bounds__(ROTARY_THREADS) rotary_kernel(const __grid_constant__ RotaryArgs a) {
  using Vec = typename Vec<V>::type;
  using T2 = typename Tr<T>::T2;
  __shared__ __align__(16) float2 angle[MAX_TOKENS * 128];
  __shared__ long long place[MAX_TOKENS];  // of the token in its sequence, -1: a row of nobody
  __shared__ int page[MAX_TOKENS];         // -1: not stored
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row0 = (long long)blockIdx.x * a.T;
  pdl_prologue();
  if (CACHE && a.cu && blockIdx.x == gridDim.x - 1) {  // a CTA of its own for each
    if (blockIdx.y == 0) check_bounds(a);
    return;
  }
  const int u = tid % a.U, hl = (tid / a.U) % a.HL, t = tid / (a.U * a.HL);
  const long long row = row0 + t;
  const bool active = t < a.T && row < a.rows;
  const int nq = a.heads[0], nk = nq + a.heads[1], all = nk + a.heads[2];
  // channels of this thread's two vectors: in a rotated head, in one that is not
  const int units = a.n_pairs / V;
  int c0, c1;
  if (u >= units) {
    c0 = 2 * a.n_pairs + (u - units) * 2 * V;
    c1 = c0 + V;
  } else if (a.interleaved) {
    c0 = u * 2 * V;
    c1 = c0 + V;
  } else {
    c0 = u * V;
    c1 = c0 + a.n_pairs;
  }
  auto source = [&](int h, const T** p0, const T** p1) {
    const int w = h < nq ? 0 : h < nk ? 1 : 2;
    const T* p = static_cast<const T*>(a.src[w]) + row * a.src_token[w] + (long long)(h - (w == 0 ? 0 : w == 1 ? nq : nk)) * a.src_head[w];
    *p0 = p + c0;
    *p1 = p + c1;
  };
  Vec x[NB][2], ahead[NB][2];
  auto load = [&](int h0, Vec (&x)[NB][2]) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int h = h0 + i * a.HL;
      if (active && h < all) {
        const T *p0, *p1;
        source(h, &p0, &p1);
        x[i][0] = load_row<V>(p0);
        x[i][1] = load_row<V>(p1);
      }
    }
  };
  const int stride = a.HL * NB * gridDim.y;
  int h0 = blockIdx.y * a.HL * NB + hl;
  load(h0, x);
  if (CACHE) {
    for (int k = warp; k < a.T; k += ROTARY_THREADS / 32) {
      const long long r = row0 + k;
      int first = 0, s = -1;
      if (r < a.rows) s = sequence_of(a.cu, a.c.n_seqs, r, a.rows, lane, &first);
      if (lane == 0) {
        long long at = -1;
        int id = -1;
        const int from = s >= 0 ? a.start[s] : -1;
        if (from >= 0) {
          at = from + (r - first);
          const long long b = at >> a.c.block_log2;
          if (b >= a.c.max_blocks) {
            kv8_record(a.c.status, CHECK_LENGTH);
          } else {
            id = a.c.table[(size_t)s * a.c.max_blocks + b];
            if (id < 0 || id >= a.c.n_pages) {
              if (id != -1) kv8_record(a.c.status, CHECK_PAGE_ID);
              id = -1;
            }
          }
        }
        place[k] = at;
        page[k] = id;
      }
    }
    if (!a.positions) __syncthreads();
  }
  // (tokens side by side: lanes that read different frequencies from the arguments wait for one another)
  for (int e = tid; e < a.T * a.n_pairs; e += ROTARY_THREADS) {
    const int p = e / a.T, k = e - p * a.T;
    const long long r = row0 + k;
    double at = 0.0;
    if (a.positions) {
      if (r < a.rows) at = a.positions[a.axis[p] * a.axis_stride + r];
    } else if (CACHE) {
      at = (double)place[k];
    }
    const double turns = at * a.turns[p];
    float sn, cs;
    sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
    angle[k * a.n_pairs + p] = make_float2(cs * a.scale, sn * a.sin_scale);
  }
  __syncthreads();
  if (!active) return;
  const long long at = CACHE ? place[t] : 0;
  if (at < 0) return;
  const int id = CACHE ? page[t] : 0;
  float2 cs[V];
  if (u < units) {
#pragma unroll
    for (int i = 0; i < V; ++i) cs[i] = angle[t * a.n_pairs + u * V + i];
  }
  for (; h0 < all; h0 += stride) {
    load(h0 + stride, ahead);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int h = h0 + i * a.HL;
      if (h >= all) break;
      const int w = h < nq ? 0 : h < nk ? 1 : 2;
      Vec y0 = x[i][0], y1 = x[i][1];
      if (w < 2 && u < units) {
        uint32_t* v0 = reinterpret_cast<uint32_t*>(&y0);
        uint32_t* v1 = reinterpret_cast<uint32_t*>(&y1);
        if (a.interleaved) {
#pragma unroll
          for (int k = 0; k < V; ++k) {
            uint32_t& v = k < V / 2 ? v0[k] : v1[k - V / 2];
            const T2 p = as_t2<T2>(v);
            const float f = Tr<T>::to_float(p.x), g = Tr<T>::to_float(p.y);
            T2 r;
            r.x = Tr<T>::from_float(f * cs[k].x - g * cs[k].y);
            r.y = Tr<T>::from_float(g * cs[k].x + f * cs[k].y);
            v = as_u32(r);
          }
        } else {
#pragma unroll
          for (int k = 0; k < V / 2; ++k) {
            const T2 p = as_t2<T2>(v0[k]), q = as_t2<T2>(v1[k]);
            T2 r, s;
            const float f0 = Tr<T>::to_float(p.x), g0 = Tr<T>::to_float(q.x), f1 = Tr<T>::to_float(p.y), g1 = Tr<T>::to_float(q.y);
            const float2 a0 = cs[2 * k], a1 = cs[2 * k + 1];
            r.x = Tr<T>::from_float(f0 * a0.x - g0 * a0.y);
            s.x = Tr<T>::from_float(g0 * a0.x + f0 * a0.y);
            r.y = Tr<T>::from_float(f1 * a1.x - g1 * a1.y);
            s.y = Tr<T>::from_float(g1 * a1.x + f1 * a1.y);
            v0[k] = as_u32(r);
            v1[k] = as_u32(s);
          }
        }
      }
      T* out;
      if (CACHE && w > 0) {
        if (id < 0) continue;
        const int kv = w - 1;
        out = static_cast<T*>(a.c.pages[kv]) + id * a.c.stride[kv][0] + (long long)(h - (w == 1 ? nq : nk)) * a.c.stride[kv][1] +
              (at & ((1 << a.c.block_log2) - 1)) * a.c.stride[kv][2];
      } else {
        out = static_cast<T*>(w == 0 ? a.dst[0] : a.dst[1]) + row * (w == 0 ? a.dst_token[0] : a.dst_token[1]) +
              (long long)(h - (w == 0 ? 0 : nq)) * (w == 0 ? a.dst_head[0] : a.dst_head[1]);
      }
      *reinterpret_cast<Vec*>(out + c0) = y0;
      *reinterpret_cast<Vec*>(out + c1) = y1;
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      x[i][0] = ahead[i][0];
      x[i][1] = ahead[i][1];
    }
  }
}

const char* rotation_check(const qevict_rotation* r, int head_dim, qevict_status* st) {
  *st = QEVICT_ERR_INVALID_ARG;
  if (r->struct_size != sizeof(qevict_rotation)) return "struct_size does not match this library's qevict_rotation";
  if (r->interleaved != 0 && r->interleaved != 1) return "interleaved must be 0 or 1";
  if (r->n_axes < 1 || r->n_axes > 8) return "n_axes must be 1 to 8";
  if (r->n_pairs < 4 || r->n_pairs > 128 || r->n_pairs % 4) return "n_pairs must be a multiple of 4, 4 to 128";
  if (2 * r->n_pairs > head_dim) return "the rotation has more channels than a head";
  if (!(fabs(r->scale) <= 65536.0)) return "scale of the rotation must be at most 65536 in magnitude";
  for (int p = 0; p < r->n_pairs; ++p) {
    if (!(fabs(r->inv_freq[p]) <= 16.0)) return "inv_freq must be at most 16 in magnitude";
    if (r->axis[p] >= r->n_axes) return "axis of a pair is not below n_axes";
  }
  return nullptr;
}

void set_rotation(RotaryArgs* a, const qevict_rotation* r, bool inverse) {
  a->n_pairs = r ? r->n_pairs : 0;
  a->interleaved = r ? r->interleaved : 0;
  a->scale = r ? (float)r->scale : 1.f;
  a->sin_scale = inverse ? -a->scale : a->scale;
  for (int p = 0; p < a->n_pairs; ++p) {
    a->turns[p] = r->inv_freq[p] / 6.283185307179586476925287;
    a->axis[p] = r->axis[p];
  }
}

int rotary_sms(int device) {
  int n = 0;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) {
    (void)cudaGetLastError();
    n = SM_COUNT_FALLBACK;
  }
  return n;
}

// Few rows (a step of decoding): a unit for each thread, spread over the SMs.  Many: eight tokens for each CTA, whose angles then cost
// little beside their heads (16384 tokens x 32 heads of 128: 4 tokens 59 us, 8 46 us, 16 50 us).  NB, units in work and as many on
// their way: 4 for queries and keys (2: 52 us, 1: 49 us), 2 into the cache (the places take registers: four prompts of up to 16001
// tokens x 48 heads 168 us, 4: 172 us, 1: 181 us) and where a CTA has lanes for half the heads.
template <class T, int V, bool CACHE> cudaError_t launch_v(RotaryArgs& a, int device, cudaStream_t s) {
  a.U = a.D / (2 * V);
  const int all = a.heads[0] + a.heads[1] + a.heads[2], lanes = ROTARY_THREADS / a.U;
  const bool few = a.rows * all * a.U <= (long long)rotary_sms(device) * 4 * ROTARY_THREADS;
  a.T = few ? (all < lanes ? lanes / all : 1) : MAX_TOKENS;
  if (a.T > MAX_TOKENS) a.T = MAX_TOKENS;
  if (a.T > lanes) a.T = lanes;
  a.HL = lanes / a.T;
  const dim3 grid((unsigned)((a.rows + a.T - 1) / a.T) + (CACHE && a.cu ? 1 : 0), few ? (unsigned)((all + a.HL - 1) / a.HL) : 1u);
  auto kernel = few ? rotary_kernel<T, V, 1, CACHE> : rotary_kernel<T, V, 2, CACHE>;
  if constexpr (!CACHE) {
    if (!few && all > 2 * a.HL) kernel = rotary_kernel<T, V, 4, CACHE>;
  }
  return launch_pdl(kernel, grid, dim3(ROTARY_THREADS), 0, s, a);
}

template <bool CACHE> cudaError_t launch_rotary(RotaryArgs& a, int dtype, int device, void* stream) {
  DeviceGuard guard(device);
  if (guard.err != cudaSuccess) return guard.err;
  cudaStream_t s = (cudaStream_t)stream;
  const bool wide = a.D % 16 == 0 && a.n_pairs % 8 == 0;  // else vectors of 8 bytes
  if (dtype == QEVICT_DTYPE_FP16) return wide ? launch_v<__half, 8, CACHE>(a, device, s) : launch_v<__half, 4, CACHE>(a, device, s);
  return wide ? launch_v<__nv_bfloat16, 8, CACHE>(a, device, s) : launch_v<__nv_bfloat16, 4, CACHE>(a, device, s);
}

bool bad_rows(const int64_t* stride, long long tokens, int heads) { return bad_stride(stride[0], tokens) || bad_stride(stride[1], heads); }

// Strides and addresses of a tensor of rows, `out` of the same where it is given.
const char* rows_check(const void* p, const int64_t* stride, long long tokens, int heads) {
  if (!p) return "q, k, v and outputs that the call has must not be NULL";
  if (misaligned16(p)) return "q, k, v and outputs must be 16-byte aligned";
  if (bad_rows(stride, tokens, heads)) return "strides must be positive multiples of 16 bytes";
  return nullptr;
}
const char* out_check(const void* p, const int64_t* stride, const void* out, const int64_t* out_stride, long long tokens, int heads) {
  if (const char* why = rows_check(p, stride, tokens, heads)) return why;
  if (const char* why = rows_check(out, out_stride, tokens, heads)) return why;
  if (p == out && ((tokens > 1 && stride[0] != out_stride[0]) || (heads > 1 && stride[1] != out_stride[1])))
    return "an output in its input's place must have its strides";
  return nullptr;
}

}  // namespace

}  // namespace qevict

using namespace qevict;

extern "C" {

QEVICT_API qevict_status qevict_rope(const qevict_rope_args* p, void* stream) {
  auto bad = [](const char* why) { return stateless_fail(QEVICT_ERR_INVALID_ARG, why); };
  auto unsupported = [](const char* why) { return stateless_fail(QEVICT_ERR_UNSUPPORTED, why); };
  if (!p) return bad("args is NULL");
  if (p->struct_size != sizeof(qevict_rope_args)) return bad("struct_size does not match this library's qevict_rope_args");
  if (p->device < 0) return bad("device must be >= 0");
  if (p->dtype != QEVICT_DTYPE_FP16 && p->dtype != QEVICT_DTYPE_BF16) return bad("dtype must be fp16 or bf16");
  if (p->inverse != 0 && p->inverse != 1) return bad("inverse must be 0 or 1");
  if (p->reserved != 0) return bad("reserved must be 0");
  if (p->n_q_heads < 1 || p->n_k_heads < 0 || p->tokens < 0) return bad("n_q_heads must be >= 1, n_k_heads and tokens >= 0");
  if (p->head_dim < 8 || p->head_dim > 256 || p->head_dim % 8) return unsupported("head_dim must be a multiple of 8, 8 to 256");
  if (p->n_q_heads > 1024 || p->n_k_heads > 1024) return unsupported("more than 1024 heads");
  if (p->tokens > 0x7fffffff - 1024) return unsupported("more than 2^31 - 1024 tokens");
  if (!p->rotation) return bad("rotation is NULL");
  qevict_status st;
  if (const char* why = rotation_check(p->rotation, p->head_dim, &st)) return stateless_fail(st, why);
  if (p->tokens == 0) return QEVICT_OK;
  if (const char* why = out_check(p->q, p->q_stride, p->q_out, p->q_out_stride, p->tokens, p->n_q_heads)) return bad(why);
  if (p->n_k_heads)
    if (const char* why = out_check(p->k, p->k_stride, p->k_out, p->k_out_stride, p->tokens, p->n_k_heads)) return bad(why);
  if (!p->positions || misaligned4(p->positions)) return bad("positions must be given, 4-byte aligned");
  if (p->rotation->n_axes > 1 && (p->axis_stride < 0 || p->axis_stride >= (1ll << 38))) return bad("axis_stride must be >= 0");
  RotaryArgs a = {};
  set_rotation(&a, p->rotation, p->inverse != 0);
  a.D = p->head_dim;
  a.heads[0] = p->n_q_heads; a.heads[1] = p->n_k_heads;
  a.src[0] = p->q; a.src[1] = p->k;
  a.dst[0] = p->q_out; a.dst[1] = p->k_out;
  a.src_token[0] = p->q_stride[0]; a.src_head[0] = p->q_stride[1];
  a.src_token[1] = p->k_stride[0]; a.src_head[1] = p->k_stride[1];
  a.dst_token[0] = p->q_out_stride[0]; a.dst_head[0] = p->q_out_stride[1];
  a.dst_token[1] = p->k_out_stride[0]; a.dst_head[1] = p->k_out_stride[1];
  a.positions = p->positions; a.axis_stride = p->axis_stride; a.rows = p->tokens;
  const cudaError_t e = launch_rotary<false>(a, p->dtype, p->device, stream);
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  return QEVICT_OK;
}

QEVICT_API qevict_status qevict_kv16_append(const qevict_kv16_append_args* p, void* stream) {
  auto bad = [](const char* why) { return stateless_fail(QEVICT_ERR_INVALID_ARG, why); };
  if (!p) return bad("args is NULL");
  if (p->struct_size != sizeof(qevict_kv16_append_args)) return bad("struct_size does not match this library's qevict_kv16_append_args");
  RotaryArgs a = {};
  qevict_status st;
  if (const char* why = kv16_check(p->cache, &st, &a.c)) return stateless_fail(st, why);
  if (p->rotation)
    if (const char* why = rotation_check(p->rotation, a.c.D, &st)) return stateless_fail(st, why);
  if (p->total_new < 0 || p->n_q_heads < 0) return bad("total_new and n_q_heads must be >= 0");
  if (p->n_q_heads > 1024) return stateless_fail(QEVICT_ERR_UNSUPPORTED, "more than 1024 heads");
  if (p->total_new > 0x7fffffff - 1024) return stateless_fail(QEVICT_ERR_UNSUPPORTED, "more than 2^31 - 1024 tokens");
  if (p->positions && !p->rotation) return bad("positions without a rotation");
  if (!p->cu_new && p->total_new > 0 && p->total_new < a.c.n_seqs) return bad("without cu_new total_new must be at least n_seqs");
  if (a.c.n_seqs == 0 || p->total_new == 0) return QEVICT_OK;
  if (const char* why = rows_check(p->k, p->k_stride, p->total_new, a.c.Hkv)) return bad(why);
  if (const char* why = rows_check(p->v, p->v_stride, p->total_new, a.c.Hkv)) return bad(why);
  if (p->n_q_heads)
    if (const char* why = out_check(p->q, p->q_stride, p->q_out, p->q_out_stride, p->total_new, p->n_q_heads)) return bad(why);
  if (!p->start) return bad("start must not be NULL");
  if (misaligned4(p->start) || misaligned4(p->cu_new) || misaligned4(p->positions)) return bad("start, cu_new and positions must be 4-byte aligned");
  if (p->positions && p->rotation->n_axes > 1 && (p->axis_stride < 0 || p->axis_stride >= (1ll << 38))) return bad("axis_stride must be >= 0");
  set_rotation(&a, p->rotation, false);
  a.D = a.c.D;
  a.heads[0] = p->n_q_heads; a.heads[1] = a.heads[2] = a.c.Hkv;
  a.src[0] = p->q; a.src[1] = p->k; a.src[2] = p->v;
  a.dst[0] = p->q_out;
  a.src_token[0] = p->q_stride[0]; a.src_head[0] = p->q_stride[1];
  a.src_token[1] = p->k_stride[0]; a.src_head[1] = p->k_stride[1];
  a.src_token[2] = p->v_stride[0]; a.src_head[2] = p->v_stride[1];
  a.dst_token[0] = p->q_out_stride[0]; a.dst_head[0] = p->q_out_stride[1];
  a.positions = p->positions; a.axis_stride = p->axis_stride;
  a.rows = p->cu_new ? p->total_new : a.c.n_seqs;  // (without bounds the rows behind the sequences are nobody's)
  a.start = p->start; a.cu = p->cu_new;
  const cudaError_t e = launch_rotary<true>(a, p->cache->dtype, p->cache->device, stream);
  if (e != cudaSuccess) return stateless_fail(QEVICT_ERR_CUDA, cudaGetErrorString(e));
  return QEVICT_OK;
}

}  // extern "C"
