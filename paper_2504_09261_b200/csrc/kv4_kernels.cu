// Rows into a cache of 4 bits (format: hack.h) and back.
//
// A thread owns a block of 16 elements of K and the same block of V: 32 (bf16) or 64 (fp32) bytes in, eight bytes of codes and
// one of scale out, so that a warp reads and writes consecutive bytes, and nothing is exchanged.  Bound: bytes, if the
// arithmetic stays under them: five instructions an element in for bf16 (largest of a block on the bits, a quotient
// rounded into the low bits of a number), about a dozen for fp32, two an element out (codes to bf16 as in the
// attention; a conversion of integers an element took 30 us of the special-function unit's time where the bytes take 26).
#include <string>

#include "entry_checks.h"
#include "kv4.cuh"
#include "tc_ptx.cuh"

namespace hack {
namespace {

using namespace kv4;

constexpr int kThreads = 256;
constexpr int kMaxCap = 0x7fffffff - 511;

struct RowsParams {
  Planes planes;
  int n_tokens;                       // rows of a head at most
  int kv_heads;
  int whole;                          // the blocks of k and v start on 32-byte boundaries
  long long threads;                  // heads * n_tokens * blocks
  hack_strides_t ks, vs;
  const void *k, *v;                  // append; the outputs of a read
  const int32_t* lens;
  const int32_t* new_lens;
  // rows of a layer's planes instead of [batch, heads, tokens, head_dim] tensors
  const int32_t* src_row;             // [heads] first row, or NULL
  const uint8_t* is_ctx;              // [kv_heads] type of a head
  int src_len[2];                     // rows of a head of each type
  int src_cap[2];                     // and those it has room for (checked build)
  int* status;
};

// 16 elements of a row as words; `whole`: they start on a 32-byte boundary.
__device__ __forceinline__ void load_32b(const void* p, uint32_t* w, bool whole) {
  if (whole) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 u = static_cast<const uint4*>(p)[i];
      w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
    }
  }
}
template <typename T> struct Sixteen;
template <> struct Sixteen<float> {
  uint32_t w[16];
  __device__ __forceinline__ void load(const void* p, bool whole) {
    load_32b(p, w, whole);
    load_32b(static_cast<const float*>(p) + 8, w + 8, whole);
  }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(w[i]); }
  // bits of the largest magnitude; any NaN is above infinity
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, w[i] & 0x7fffffffu);
    return m;
  }
  __device__ __forceinline__ void limit(float most) {
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(fminf(fmaxf(at(i), -most), most));
  }
  __device__ __forceinline__ void no_nans() {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if ((w[i] & 0x7fffffffu) > 0x7f800000u) w[i] = 0;
  }
};
template <> struct Sixteen<__nv_bfloat16> {
  uint32_t w[8];
  __device__ __forceinline__ void load(const void* p, bool whole) { load_32b(p, w, whole); }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
    return max(m & 0xffff0000u, m << 16);
  }
  // (seven times the largest scale is a bf16 number)
  __device__ __forceinline__ void limit(float most) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = fminf(fmaxf(at(2 * i), -most), most), y = fminf(fmaxf(at(2 * i + 1), -most), most);
      w[i] = __float_as_uint(x) >> 16 | (__float_as_uint(y) & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void no_nans() {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if ((w[i] & 0x7fffu) > 0x7f80u) w[i] &= 0xffff0000u;
      if ((w[i] & 0x7fff0000u) > 0x7f800000u) w[i] &= 0xffffu;
    }
  }
};

// Scale byte and codes of a block.
template <typename T> __device__ __forceinline__ uint2 quantise(Sixteen<T>& x, uint32_t& byte) {
  uint32_t top_bits = x.top();
  if (top_bits > 0x7f800000u) {
    x.no_nans();
    top_bits = x.top();
  }
  const float top = __uint_as_float(top_bits);
  // The smallest s with 7 s >= top: the rounded quotient, to three mantissa bits upwards, is it or a neighbour (7 s is exact)
  const uint32_t up = (__float_as_uint(fminf(top * (1.f / 7.f), 3840.f)) + 0xfffffu) >> 20;
  int e = min(max((int)up - (int)((127 - 20) << 3), 0), 255);
  if (e < 255 && 7.f * scale_value(e) < top) ++e;
  if (e > 0 && 7.f * scale_value(e - 1) >= top) --e;
  byte = e;
  const float s = scale_value(e), inv = 1.f / s;
  if (top > 7.f * s) x.limit(7.f * s);         // the largest scale of all, and beyond seven of it
  // A quotient + kMagic has c + 8 in its low bits, ties to even.
  constexpr float kMagic = 12582912.f + 8.f;
  uint32_t code[2] = {0, 0};
  if constexpr (sizeof(T) == 2) {
    // x (inv + rest) is within 2^-48 of x / s, so that its product is the quotient correctly rounded: exactly the middle between two
    // codes where x / s is (eight significant bits over four do not come nearer to one without being it).
    const float rest = fmaf(-s, inv, 1.f) * inv;
#pragma unroll
    for (int i = 0; i < kBlock; ++i) {
      const float v = x.at(i);
      code[i >> 3] += __float_as_uint(fmaf(v, inv, v * rest) + kMagic) << (4 * (i & 7));
    }
  } else {
    // The quotient may fall on the wrong side of a middle, or on it: what is left of x beside the code, which is exact, tells.
    const int half = __float_as_int(0.5f * s);
#pragma unroll
    for (int i = 0; i < kBlock; ++i) {
      const float v = x.at(i), r = fmaf(v, inv, kMagic);
      int n = __float_as_int(r);
      const float left = fmaf(kMagic - r, s, v);
      // on the middle, an odd code gives way: the float below one half of s
      if (fabsf(left) > __int_as_float(half - (n & 1))) n += (__float_as_int(left) >> 31) | 1;
      code[i >> 3] += (uint32_t)n << (4 * (i & 7));
    }
  }
  // (the bits of kMagic without its 8, once for each of the eight codes)
  constexpr uint32_t kBase = 0x4b400000u;
  uint32_t extra = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) extra += kBase << (4 * i);
  return make_uint2(code[0] - extra, code[1] - extra);
}

// Head, token and block of a thread; false past the end.
template <int BLOCKS> __device__ __forceinline__ bool place(const RowsParams& p, int& head, int& token, int& block) {
  const long long at = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (at >= p.threads) return false;
  block = (int)(at % BLOCKS);
  if (p.threads <= 0x7fffffffll) {
    const uint32_t row = (uint32_t)at / BLOCKS;
    head = row / (uint32_t)p.n_tokens;
    token = row - (uint32_t)head * (uint32_t)p.n_tokens;
  } else {
    const long long row = at / BLOCKS;
    head = (int)(row / p.n_tokens);
    token = (int)(row - (long long)head * p.n_tokens);
  }
  return true;
}

template <typename T, int BLOCKS>
__global__ void __launch_bounds__(kThreads) kv4_append_kernel(const __grid_constant__ RowsParams p) {
  pdl_wait();
  int head, token, block;
  if (!place<BLOCKS>(p, head, token, block)) return;
  const int b = head / p.kv_heads, h = head - b * p.kv_heads;
  const T *k = static_cast<const T*>(p.k) + block * kBlock, *v = static_cast<const T*>(p.v) + block * kBlock;
  if (p.src_row) {
    const int type = p.is_ctx[h] ? 1 : 0;
    if (token >= p.src_len[type] || !dbg_ok(p.src_row[head] >= 0 && token < p.src_cap[type], p.status, 15)) return;
    const long long at = ((long long)p.src_row[head] + token) * (BLOCKS * kBlock);
    k += at;
    v += at;
  } else {
    if (p.new_lens && token >= p.new_lens[b]) return;
    k += b * p.ks.batch + h * p.ks.head + token * p.ks.token;
    v += b * p.vs.batch + h * p.vs.head + token * p.vs.token;
  }
  // (read whether or not it has a place: the length is on its way meanwhile)
  Sixteen<T> rk, rv;
  rk.load(k, p.whole);
  rv.load(v, p.whole);
  const long long slot = (long long)max(p.lens[head], 0) + token;
  const long long first = first_row(p.planes, head);
  if (slot >= p.planes.cap || !inside(p.planes, first)) return;
  const long long at = (first + slot) * BLOCKS + block;
  uint32_t byte;
  uint2 code = quantise(rk, byte);
  reinterpret_cast<uint2*>(p.planes.k_codes)[at] = code;
  p.planes.k_scales[at] = (unsigned char)byte;
  code = quantise(rv, byte);
  reinterpret_cast<uint2*>(p.planes.v_codes)[at] = code;
  p.planes.v_scales[at] = (unsigned char)byte;
}

// A block's values, in bf16 pairs.
__device__ __forceinline__ void block_values(const uint2& code, uint32_t byte, uint32_t* w) {
  const Scale2 s = scale2(byte * 0x10001u);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t c = i ? code.y : code.x;
    const uint32_t a = values2(c, 0, s), b = values2(c, 4, s), d = values2(c, 8, s), e = values2(c, 12, s);   // (0,4) (1,5) (2,6) (3,7)
    w[4 * i] = __byte_perm(a, b, 0x5410);
    w[4 * i + 1] = __byte_perm(d, e, 0x5410);
    w[4 * i + 2] = __byte_perm(a, b, 0x7632);
    w[4 * i + 3] = __byte_perm(d, e, 0x7632);
  }
}
template <typename T> __device__ __forceinline__ void store_block(T* dst, const uint32_t* w, bool whole) {
  if constexpr (sizeof(T) == 2) {
    ptx::st_global_32b(dst, w, whole);
  } else {
    uint32_t x[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[2 * i] = w[i] << 16;
      x[2 * i + 1] = w[i] & 0xffff0000u;
    }
    ptx::st_global_32b(dst, x, whole);
    ptx::st_global_32b(dst + 8, x + 8, whole);
  }
}

template <typename T, int BLOCKS>
__global__ void __launch_bounds__(kThreads) kv4_read_kernel(const __grid_constant__ RowsParams p) {
  pdl_wait();
  int head, token, block;
  if (!place<BLOCKS>(p, head, token, block)) return;
  const int b = head / p.kv_heads, h = head - b * p.kv_heads;
  T* k = static_cast<T*>(const_cast<void*>(p.k)) + b * p.ks.batch + h * p.ks.head + token * p.ks.token + block * kBlock;
  T* v = static_cast<T*>(const_cast<void*>(p.v)) + b * p.vs.batch + h * p.vs.head + token * p.vs.token + block * kBlock;
  const long long slot = (long long)p.lens[head] + token;
  uint2 kc = make_uint2(0x88888888u, 0x88888888u), vc = kc;      // code 8 stands for 0
  uint32_t kb = 0, vb = 0;
  const long long first = first_row(p.planes, head);
  if (slot >= 0 && slot < p.planes.cap && inside(p.planes, first)) {
    const long long at = (first + slot) * BLOCKS + block;
    kc = reinterpret_cast<const uint2*>(p.planes.k_codes)[at];
    vc = reinterpret_cast<const uint2*>(p.planes.v_codes)[at];
    kb = p.planes.k_scales[at];
    vb = p.planes.v_scales[at];
  }
  uint32_t w[8];
  block_values(kc, kb, w);
  store_block(k, w, p.whole);
  block_values(vc, vb, w);
  store_block(v, w, p.whole);
}

bool on_sectors(const void* ptr, const hack_strides_t& s, int elt) {
  const int unit = 32 / elt;
  return reinterpret_cast<uintptr_t>(ptr) % 32 == 0 && s.batch % unit == 0 && s.head % unit == 0 && s.token % unit == 0;
}

// A row's blocks are consecutive threads'.
hack_status_t launch_rows(bool read, RowsParams& p, int dtype, int head_dim, int heads, cudaStream_t st) {
  const int blocks = head_dim / kBlock, elt = dtype == HACK_F32 ? 4 : 2;
  p.threads = (long long)heads * p.n_tokens * blocks;
  p.whole = on_sectors(p.k, p.ks, elt) && on_sectors(p.v, p.vs, elt);
  const long long grid = (p.threads + kThreads - 1) / kThreads;
  if (grid > 0x7fffffffll) {
    set_error("more rows than a launch has places for");
    return HACK_ERR_UNSUPPORTED;
  }
  auto go = [&](auto* append, auto* back) { launch_k(read ? back : append, dim3((unsigned)grid), dim3(kThreads), 0, st, p); };
  if (dtype == HACK_F32) {
    if (blocks == 4) go(kv4_append_kernel<float, 4>, kv4_read_kernel<float, 4>);
    else go(kv4_append_kernel<float, 8>, kv4_read_kernel<float, 8>);
  } else {
    if (blocks == 4) go(kv4_append_kernel<__nv_bfloat16, 4>, kv4_read_kernel<__nv_bfloat16, 4>);
    else go(kv4_append_kernel<__nv_bfloat16, 8>, kv4_read_kernel<__nv_bfloat16, 8>);
  }
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
  if (off_its_size(at, 4)) return invalid("lengths or first rows are not on a multiple of 4 bytes");
  const int elt = r->dtype == HACK_F32 ? 4 : 2;
  const char* text = view_error(k, r->k, kv->batch, kv->n_kv_heads, r->n_tokens, kv->head_dim, elt, written);
  if (!text) text = view_error(v, r->v, kv->batch, kv->n_kv_heads, r->n_tokens, kv->head_dim, elt, written);
  return text ? invalid(text) : HACK_OK;
}

RowsParams rows_params(const hack_kv4_t* kv) {
  RowsParams p{};
  p.planes = kv4_planes(kv);
  p.kv_heads = kv->n_kv_heads;
  return p;
}

}  // namespace

hack_status_t kv4_check(const hack_kv4_t* kv) {
  if (!kv) return invalid("kv is NULL");
  if (kv->head_dim != 64 && kv->head_dim != 128) { set_error("head_dim must be 64 or 128"); return HACK_ERR_UNSUPPORTED; }
  if (kv->device < 0 || kv->batch < 1 || kv->n_kv_heads < 1 || kv->cap < 1 || (long long)kv->batch * kv->n_kv_heads > 0x7fffffffll)
    return invalid("batch, n_kv_heads and cap must be positive, device not negative");
  // (a tile of 128 rows that starts among a head's last ones must end within 32 bits)
  if (kv->cap > kMaxCap) return invalid("cap is beyond 2^31 - 512 rows");
  if (kv->rows < kv->cap || (!kv->row_off && kv->rows < (long long)kv->batch * kv->n_kv_heads * kv->cap)) return invalid("the planes have too few rows");
  const void* planes[4] = {kv->k_codes, kv->v_codes, kv->k_scales, kv->v_scales};
  for (const void* q : planes)
    if (!q || (reinterpret_cast<uintptr_t>(q) & 15)) return invalid("a plane is NULL or not 16-byte aligned");
  if (off_its_size(kv->row_off, 8)) return invalid("row_off is not on a multiple of 8 bytes");
  return HACK_OK;
}

kv4::Planes kv4_planes(const hack_kv4_t* kv) {
  return {static_cast<unsigned char*>(kv->k_codes), static_cast<unsigned char*>(kv->v_codes),
          static_cast<unsigned char*>(kv->k_scales), static_cast<unsigned char*>(kv->v_scales), kv->row_off, (long long)kv->rows, kv->cap};
}

hack_status_t launch_store_kv4(const StepArgs& a, int dtype, const hack_kv4_t* kv, const int32_t* lens, uint64_t& launches, cudaStream_t st) {
  RowsParams p = rows_params(kv);
  p.k = a.k_plane;
  p.v = a.v_plane;
  p.lens = lens;
  p.src_row = a.row_off;
  p.is_ctx = a.is_ctx;
  p.status = a.status;
  int longest = 0;
  for (int t = 0; t < 2; ++t) {
    p.src_len[t] = a.kept[t];
    p.src_cap[t] = a.cap[t];
    if (a.heads_of[t] > 0 && a.kept[t] > longest) longest = a.kept[t];
  }
  p.n_tokens = longest;
  if (longest == 0) return HACK_OK;
  const hack_status_t s = launch_rows(false, p, dtype, a.head_dim, a.batch * a.n_heads, st);
  launches += s == HACK_OK;
  return s;
}

}  // namespace hack

extern "C" hack_status_t hack_kv4_append(const hack_kv4_t* kv, const hack_kv4_rows_t* rows, const void* k, const void* v,
                                         const int32_t* lens, const int32_t* new_lens, void* stream) {
  using namespace hack;
  const hack_status_t s = check_rows(kv, rows, k, v, lens, false);
  if (s != HACK_OK || rows->n_tokens == 0) return s;
  if (off_its_size(new_lens, 4)) return invalid("new_lens is not on a multiple of 4 bytes");
  HACK_ON_DEVICE_OF(kv->device);
  RowsParams p = rows_params(kv);
  p.n_tokens = rows->n_tokens;
  p.ks = rows->k;
  p.vs = rows->v;
  p.k = k;
  p.v = v;
  p.lens = lens;
  p.new_lens = new_lens;
  return launch_rows(false, p, rows->dtype, kv->head_dim, kv->batch * kv->n_kv_heads, (cudaStream_t)stream);
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
  return launch_rows(true, p, rows->dtype, kv->head_dim, kv->batch * kv->n_kv_heads, (cudaStream_t)stream);
}
