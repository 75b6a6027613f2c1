// Rows into a cache of 4 bits (format: hack.h) and back.
//
// A thread owns a block of 16 elements of K and the same block of V: 32 (bf16) or 64 (fp32) bytes in, eight bytes of codes and
// one of scale out, so that a warp reads and writes consecutive bytes, and nothing is exchanged.  Bound:
// bytes; the rounding to the nearest code, exact in spite of an inexact reciprocal, stays under them.
#include <string>

#include "entry_checks.h"
#include "kv4.cuh"

namespace hack {
namespace {

using namespace kv4;

constexpr int kThreads = 256;

struct RowsParams {
  Planes planes;
  int n_tokens, blocks;               // rows of a head at most; blocks per row
  int kv_heads;
  long long threads;                  // heads * n_tokens * blocks
  hack_strides_t ks, vs;
  const void *k, *v;                  // append; the outputs of a read
  const int32_t* lens;
  const int32_t* new_lens;
  // rows of a layer's planes instead of [batch, heads, tokens, head_dim] tensors
  const int32_t* src_row;             // [heads] first row, or NULL
  const uint8_t* is_ctx;              // [kv_heads] type of a head
  int src_len[2];                     // rows of a head of each type
};

template <typename T> struct Sixteen;           // 16 elements of a row
template <> struct Sixteen<float> {
  uint4 u[4];
  __device__ __forceinline__ void load(const void* p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = static_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void values(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[4 * i] = __uint_as_float(u[i].x); x[4 * i + 1] = __uint_as_float(u[i].y);
      x[4 * i + 2] = __uint_as_float(u[i].z); x[4 * i + 3] = __uint_as_float(u[i].w);
    }
  }
  static __device__ __forceinline__ void store(void* p, const float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) static_cast<float4*>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  }
};
template <> struct Sixteen<__nv_bfloat16> {
  uint4 u[2];
  __device__ __forceinline__ void load(const void* p) {
#pragma unroll
    for (int i = 0; i < 2; ++i) u[i] = static_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void values(float* x) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t w[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
        x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      }
    }
  }
  static __device__ __forceinline__ void store(void* p, const float* x) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[8 * i + 2 * j], x[8 * i + 2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&h);
      }
      static_cast<uint4*>(p)[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
};

// Scale byte and codes of a block.
__device__ __forceinline__ uint2 quantise(float* x, uint32_t& byte) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < kBlock; ++i) {
    x[i] = x[i] == x[i] ? x[i] : 0.f;
    top = fmaxf(top, fabsf(x[i]));
  }
  // The smallest s with 7 s >= top: the rounded quotient, to three mantissa bits upwards, is it or a neighbour (7 s is exact)
  const uint32_t up = (__float_as_uint(fminf(top * (1.f / 7.f), 3840.f)) + 0xfffffu) >> 20;
  int e = min(max((int)up - (int)((127 - 20) << 3), 0), 255);
  if (e < 255 && 7.f * scale_value(e) < top) ++e;
  if (e > 0 && 7.f * scale_value(e - 1) >= top) --e;
  byte = e;
  const float s = scale_value(e), inv = 1.f / s, half = 0.5f * s;
  uint32_t code[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < kBlock; ++i) {
    // x * inv may fall on the wrong side of the middle between two codes, or on it; what is left of x beside the code is exact
    float t = rintf(fminf(fmaxf(x[i] * inv, -7.f), 7.f));
    const float left = fmaf(-t, s, x[i]);
    const bool odd = (int)t & 1;
    if (left > half || (odd && left == half)) t += 1.f;
    if (left < -half || (odd && left == -half)) t -= 1.f;
    t = fminf(fmaxf(t, -7.f), 7.f);
    code[i >> 3] |= (uint32_t)((int)t + 8) << (4 * (i & 7));
  }
  return make_uint2(code[0], code[1]);
}

// Head, token and block of a thread; false past the end.
__device__ __forceinline__ bool place(const RowsParams& p, int& head, int& token, int& block) {
  const long long at = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (at >= p.threads) return false;
  block = (int)(at % p.blocks);
  const long long row = at / p.blocks;
  head = (int)(row / p.n_tokens);
  token = (int)(row - (long long)head * p.n_tokens);
  return true;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) kv4_append_kernel(const __grid_constant__ RowsParams p) {
  pdl_wait();
  int head, token, block;
  if (!place(p, head, token, block)) return;
  const int b = head / p.kv_heads, h = head - b * p.kv_heads;
  const T *k = static_cast<const T*>(p.k) + block * kBlock, *v = static_cast<const T*>(p.v) + block * kBlock;
  if (p.src_row) {
    if (token >= p.src_len[p.is_ctx[h] ? 1 : 0]) return;
    const long long at = ((long long)p.src_row[head] + token) * p.blocks * kBlock;
    k += at;
    v += at;
  } else {
    if (p.new_lens && token >= p.new_lens[b]) return;
    k += b * p.ks.batch + h * p.ks.head + token * p.ks.token;
    v += b * p.vs.batch + h * p.vs.head + token * p.vs.token;
  }
  const long long slot = (long long)max(p.lens[head], 0) + token;
  if (slot >= p.planes.cap) return;
  Sixteen<T> rk, rv;
  rk.load(k);
  rv.load(v);
  const long long at = (first_row(p.planes, head) + slot) * p.blocks + block;
  float x[kBlock];
  uint32_t byte;
  rk.values(x);
  uint2 code = quantise(x, byte);
  reinterpret_cast<uint2*>(p.planes.k_codes)[at] = code;
  p.planes.k_scales[at] = (unsigned char)byte;
  rv.values(x);
  code = quantise(x, byte);
  reinterpret_cast<uint2*>(p.planes.v_codes)[at] = code;
  p.planes.v_scales[at] = (unsigned char)byte;
}

__device__ __forceinline__ void block_values(const uint2& code, uint32_t byte, float* x) {
  const float s = scale_value(byte);
#pragma unroll
  for (int i = 0; i < kBlock; ++i) x[i] = (float)((int)(((i < 8 ? code.x : code.y) >> (4 * (i & 7))) & 15) - 8) * s;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) kv4_read_kernel(const __grid_constant__ RowsParams p) {
  pdl_wait();
  int head, token, block;
  if (!place(p, head, token, block)) return;
  const int b = head / p.kv_heads, h = head - b * p.kv_heads;
  T* k = static_cast<T*>(const_cast<void*>(p.k)) + b * p.ks.batch + h * p.ks.head + token * p.ks.token + block * kBlock;
  T* v = static_cast<T*>(const_cast<void*>(p.v)) + b * p.vs.batch + h * p.vs.head + token * p.vs.token + block * kBlock;
  const long long slot = (long long)p.lens[head] + token;
  uint2 kc = make_uint2(0x88888888u, 0x88888888u), vc = kc;      // code 8 stands for 0
  uint32_t kb = 0, vb = 0;
  if (slot >= 0 && slot < p.planes.cap) {
    const long long at = (first_row(p.planes, head) + slot) * p.blocks + block;
    kc = reinterpret_cast<const uint2*>(p.planes.k_codes)[at];
    vc = reinterpret_cast<const uint2*>(p.planes.v_codes)[at];
    kb = p.planes.k_scales[at];
    vb = p.planes.v_scales[at];
  }
  float x[kBlock];
  block_values(kc, kb, x);
  Sixteen<T>::store(k, x);
  block_values(vc, vb, x);
  Sixteen<T>::store(v, x);
}

template <typename F>
hack_status_t launch_rows(F* kern, RowsParams& p, int heads, cudaStream_t st) {
  p.threads = (long long)heads * p.n_tokens * p.blocks;
  const long long grid = (p.threads + kThreads - 1) / kThreads;
  if (grid > 0x7fffffffll) {
    set_error("more rows than a launch has places for");
    return HACK_ERR_UNSUPPORTED;
  }
  launch_k(kern, dim3((unsigned)grid), dim3(kThreads), 0, st, p);
  return launched(1) < 0 ? HACK_ERR_CUDA : HACK_OK;
}

hack_status_t invalid(const char* text) {
  set_error(text);
  return HACK_ERR_INVALID_ARG;
}

hack_status_t check_rows(const hack_kv4_t* kv, const hack_kv4_rows_t* r, const void* k, const void* v, const int32_t* at, bool written) {
  const hack_status_t s = kv4_check(kv);
  if (s != HACK_OK) return s;
  if (!r) return invalid("rows is NULL");
  if (r->dtype != HACK_F32 && r->dtype != HACK_BF16) { set_error("dtype must be HACK_F32 or HACK_BF16"); return HACK_ERR_UNSUPPORTED; }
  if (r->n_tokens < 0) return invalid("n_tokens is negative");
  if (r->n_tokens == 0) return HACK_OK;
  if (!k || !v || !at) return invalid("a tensor is NULL");
  const int elt = r->dtype == HACK_F32 ? 4 : 2;
  const char* text = view_error(k, r->k, kv->batch, kv->n_kv_heads, r->n_tokens, kv->head_dim, elt, written);
  if (!text) text = view_error(v, r->v, kv->batch, kv->n_kv_heads, r->n_tokens, kv->head_dim, elt, written);
  return text ? invalid(text) : HACK_OK;
}

RowsParams rows_params(const hack_kv4_t* kv) {
  RowsParams p{};
  p.planes = kv4_planes(kv);
  p.blocks = kv->head_dim / kBlock;
  p.kv_heads = kv->n_kv_heads;
  return p;
}

}  // namespace

hack_status_t kv4_check(const hack_kv4_t* kv) {
  if (!kv) return invalid("kv is NULL");
  if (kv->head_dim != 64 && kv->head_dim != 128) { set_error("head_dim must be 64 or 128"); return HACK_ERR_UNSUPPORTED; }
  if (kv->device < 0 || kv->batch < 1 || kv->n_kv_heads < 1 || kv->cap < 1 || (long long)kv->batch * kv->n_kv_heads > 0x7fffffffll)
    return invalid("batch, n_kv_heads and cap must be positive, device not negative");
  const void* planes[4] = {kv->k_codes, kv->v_codes, kv->k_scales, kv->v_scales};
  for (const void* q : planes)
    if (!q || (reinterpret_cast<uintptr_t>(q) & 15)) return invalid("a plane is NULL or not 16-byte aligned");
  return HACK_OK;
}

kv4::Planes kv4_planes(const hack_kv4_t* kv) {
  return {static_cast<unsigned char*>(kv->k_codes), static_cast<unsigned char*>(kv->v_codes),
          static_cast<unsigned char*>(kv->k_scales), static_cast<unsigned char*>(kv->v_scales), kv->row_off, kv->cap};
}

hack_status_t launch_store_kv4(const StepArgs& a, int dtype, const hack_kv4_t* kv, const int32_t* lens, cudaStream_t st) {
  RowsParams p = rows_params(kv);
  p.k = a.k_plane;
  p.v = a.v_plane;
  p.lens = lens;
  p.src_row = a.row_off;
  p.is_ctx = a.is_ctx;
  int longest = 0;
  for (int t = 0; t < 2; ++t) {
    p.src_len[t] = a.kept[t];
    if (a.heads_of[t] > 0 && a.kept[t] > longest) longest = a.kept[t];
  }
  p.n_tokens = longest;
  if (longest == 0) return HACK_OK;
  return dtype == HACK_F32 ? launch_rows(kv4_append_kernel<float>, p, a.batch * a.n_heads, st)
                           : launch_rows(kv4_append_kernel<__nv_bfloat16>, p, a.batch * a.n_heads, st);
}

}  // namespace hack

extern "C" hack_status_t hack_kv4_append(const hack_kv4_t* kv, const hack_kv4_rows_t* rows, const void* k, const void* v,
                                         const int32_t* lens, const int32_t* new_lens, void* stream) {
  using namespace hack;
  const hack_status_t s = check_rows(kv, rows, k, v, lens, false);
  if (s != HACK_OK || rows->n_tokens == 0) return s;
  HACK_ON_DEVICE_OF(kv->device);
  RowsParams p = rows_params(kv);
  p.n_tokens = rows->n_tokens;
  p.ks = rows->k;
  p.vs = rows->v;
  p.k = k;
  p.v = v;
  p.lens = lens;
  p.new_lens = new_lens;
  const int heads = kv->batch * kv->n_kv_heads;
  return rows->dtype == HACK_F32 ? launch_rows(kv4_append_kernel<float>, p, heads, (cudaStream_t)stream)
                                 : launch_rows(kv4_append_kernel<__nv_bfloat16>, p, heads, (cudaStream_t)stream);
}

extern "C" hack_status_t hack_kv4_read(const hack_kv4_t* kv, const hack_kv4_rows_t* rows, void* k_out, void* v_out,
                                       const int32_t* first, void* stream) {
  using namespace hack;
  const hack_status_t s = check_rows(kv, rows, k_out, v_out, first, true);
  if (s != HACK_OK || rows->n_tokens == 0) return s;
  HACK_ON_DEVICE_OF(kv->device);
  RowsParams p = rows_params(kv);
  p.n_tokens = rows->n_tokens;
  p.ks = rows->k;
  p.vs = rows->v;
  p.k = k_out;
  p.v = v_out;
  p.lens = first;
  const int heads = kv->batch * kv->n_kv_heads;
  return rows->dtype == HACK_F32 ? launch_rows(kv4_read_kernel<float>, p, heads, (cudaStream_t)stream)
                                 : launch_rows(kv4_read_kernel<__nv_bfloat16>, p, heads, (cudaStream_t)stream);
}
