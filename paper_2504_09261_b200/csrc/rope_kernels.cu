// Rotary positions, and norms of queries and keys with the rotation in the same pass.
//
// Pair i of a token at position p turns by p * freq[i].  The angle is formed in 64 bits as a number of turns, of
// which only the fraction is kept (positions of millions would leave 32 bits no digits behind the point), and the
// fraction goes through sincospif.  A group of lanes owns a row of head_dim elements, 16 bytes a lane: the sum of
// squares is a few shuffles, and in the half layout the partner of a lane's elements sits rotary_dim / 2 elements on,
// in the same slots of another lane of the group (or, where rotary_dim / 2 is no multiple of a lane's elements, anywhere in
// the row, which then goes through shared memory).
//
// Bound: bytes, each read and written once.  So that they are all the kernel does, a group keeps the cosines, sines
// and weights of its lanes in registers and walks over the heads of its token, kUnroll rows in flight; the
// cosines of a CTA's tokens are formed once, by all its threads, in shared memory.
#include <algorithm>
#include <cmath>
#include <string>

#include "entry_checks.h"
#include "hack_internal.h"

namespace hack {
namespace {

constexpr int kThreads = 128;
constexpr int kUnroll = 4;          // rows of a group in flight

struct RopeParams {
  // rows of three kinds, walked by CTAs of their own: [0] queries (or the only tensor), [1] keys, [2] values (copied)
  const void* in[3];
  void* out[3];
  hack_strides_t is[3], os[3];
  int heads[3];
  int chunks[3];                    // CTAs over a kind's heads
  const float* weight[2];
  const float* gain[2];
  int batch, n_tokens;
  int tiles;                        // CTAs over the tokens
  int tile_tokens;                  // tokens of a CTA, a power of two no larger than its groups
  int chunk_heads;                  // heads of a CTA
  int norm;
  float eps, inv_eps;
  const void* positions;
  int positions_f32;
  long long positions_stride;
  int pairs, axes, layout;          // pairs == 0: no rotation
  float gain_cs, sin_sign;
  double turns[HACK_ROPE_MAX_PAIRS];   // freq / 2 pi
};

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& u, float* x) {
    x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 pack(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// LANED: in the half layout, a lane's elements have their partners in one other lane (rotary_dim / 2 a multiple of them).
template <typename T, int D, bool LANED>
__global__ void __launch_bounds__(kThreads, 6) rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int N = Vec<T>::N, LANES = D / N, GROUPS = kThreads / LANES;
  extern __shared__ float2 cs[];                       // [tile_tokens][pairs] cosine, sine
  __shared__ float staged[LANED ? 1 : GROUPS][LANED ? 1 : D + 4];   // whole rows, where partners are anywhere
  pdl_wait();
  // the CTA's place: kind and chunk of heads, tokens, batch element
  int at = blockIdx.x;
  const int tile = at % p.tiles;
  at /= p.tiles;
  const int chunks = p.chunks[0] + p.chunks[1] + p.chunks[2];
  int chunk = at % chunks;
  const int b = at / chunks;
  int kind = 0;
  while (chunk >= p.chunks[kind]) chunk -= p.chunks[kind++];
  const int t0 = tile * p.tile_tokens;
  const bool rotate = p.pairs > 0 && kind < 2;
  const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int token_of = group & (p.tile_tokens - 1), head_lanes = GROUPS / p.tile_tokens, head_of = group / p.tile_tokens;
  const int token = t0 + token_of;
  const bool live = token < p.n_tokens;
  const int e0 = lane * N, half = p.pairs;
  const int h_first = chunk * p.chunk_heads, h_end = min(p.heads[kind], h_first + p.chunk_heads);
  const T* in = static_cast<const T*>(p.in[kind]) + b * p.is[kind].batch + (long long)token * p.is[kind].token + e0;
  T* out = static_cast<T*>(p.out[kind]) + b * p.os[kind].batch + (long long)token * p.os[kind].token + e0;
  const long long in_head = p.is[kind].head, out_head = p.os[kind].head;
  uint4 raw[kUnroll];
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + u * head_lanes + head_of;
      raw[u] = make_uint4(0, 0, 0, 0);
      if (live && h < h_end) raw[u] = *reinterpret_cast<const uint4*>(in + h * in_head);
    }
  };
  load(h_first);                                       // under the forming of the cosines

  if (kind == 2) {                                     // values are copied
    for (int h0 = h_first; h0 < h_end; h0 += head_lanes * kUnroll) {
      if (h0 > h_first) load(h0);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int h = h0 + u * head_lanes + head_of;
        if (live && h < h_end) *reinterpret_cast<uint4*>(out + h * out_head) = raw[u];
      }
    }
    return;
  }
  if (rotate) {
    const int tokens = min(p.tile_tokens, p.n_tokens - t0), per_axis = p.pairs / p.axes;
    for (int i = threadIdx.x; i < tokens * p.pairs; i += kThreads) {
      const int t = i / p.pairs, pair = i - t * p.pairs;
      const long long where = b * p.positions_stride + (long long)(t0 + t) * p.axes + pair / per_axis;
      const double pos = p.positions_f32 ? (double)static_cast<const float*>(p.positions)[where]
                                         : (double)static_cast<const int32_t*>(p.positions)[where];
      const double turns = pos * p.turns[pair];
      float s, c;
      sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
      cs[i] = make_float2(p.gain_cs * c, p.gain_cs * p.sin_sign * s);
    }
    __syncthreads();
  }
  // What the lane keeps: y = f (x * own + partner * other), f the row's norm and gain.  The weights are in the factors.
  float own[N], other[N];
  int from = lane;                                     // half layout: the lane with the partners
  const bool halves = p.layout == HACK_ROPE_HALF;
  const float* weight = p.weight[kind];
  const float* gain = p.gain[kind];
#pragma unroll
  for (int e = 0; e < N; ++e) { own[e] = weight ? weight[e0 + e] : 1.f; other[e] = 0.f; }
  if (rotate) {
    const float2* row = cs + (live ? token_of : 0) * p.pairs;
    if (halves && e0 < 2 * half) from = e0 < half ? lane + half / N : lane - half / N;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int d = e0 + e;
      if (d >= 2 * half) continue;
      const bool first = halves ? d < half : (e & 1) == 0;
      const int partner = halves ? (first ? d + half : d - half) : d ^ 1;
      const float2 v = row[halves ? (first ? d : partner) : d >> 1];
      other[e] = (first ? -v.y : v.y) * (weight ? weight[partner] : 1.f);
      own[e] *= v.x;
    }
  }
  // what neither turns nor is scaled leaves as it came
  const bool as_is = p.norm == HACK_NORM_NONE && !weight && !gain && (!rotate || e0 >= 2 * half);

  // All groups of a warp take the same number of turns: the shuffles need every lane.  The rows in flight go through each
  // step together (row by row, a chain of shuffles each, the bf16 form took 89 us where this takes less).
  for (int h0 = h_first; h0 < h_end; h0 += head_lanes * kUnroll) {
    if (h0 > h_first) load(h0);
    float f[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + u * head_lanes + head_of;
      f[u] = gain && h < h_end ? gain[h] : 1.f;
    }
    if (p.norm != HACK_NORM_NONE) {
      float sum[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        float x[N];
        Vec<T>::unpack(raw[u], x);
        sum[u] = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) sum[u] = fmaf(x[e], x[e], sum[u]);
      }
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1)
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], o, LANES);
      // (L2: a comparison, not fminf, which would turn the NaN of a row with one into 1 / eps)
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const float r = rsqrtf(p.norm == HACK_NORM_RMS ? fmaf(sum[u], 1.f / D, p.eps) : sum[u]);
        f[u] *= p.norm == HACK_NORM_L2 && r > p.inv_eps ? p.inv_eps : r;
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + u * head_lanes + head_of;
      float x[N], y[N];
      Vec<T>::unpack(raw[u], x);
      if (rotate) {
        float xp[N];                                   // the partners
        if (!halves) {
#pragma unroll
          for (int e = 0; e < N; ++e) xp[e] = x[e ^ 1];
        } else if (LANED) {
          uint4 o;
          o.x = __shfl_sync(0xffffffffu, raw[u].x, from, LANES);
          o.y = __shfl_sync(0xffffffffu, raw[u].y, from, LANES);
          o.z = __shfl_sync(0xffffffffu, raw[u].z, from, LANES);
          o.w = __shfl_sync(0xffffffffu, raw[u].w, from, LANES);
          Vec<T>::unpack(o, xp);
        } else {
          float* row = staged[group];
#pragma unroll
          for (int e = 0; e < N; ++e) row[e0 + e] = x[e];
          __syncwarp();
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const int d = e0 + e;
            xp[e] = d < 2 * half ? row[d < half ? d + half : d - half] : 0.f;
          }
          __syncwarp();
        }
        // (an element that does not turn has factor 0 for a partner that may be infinite)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          y[e] = f[u] * (e0 + e < 2 * half ? fmaf(x[e], own[e], xp[e] * other[e]) : x[e] * own[e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = x[e] * (f[u] * own[e]);
      }
      if (live && h < h_end) *reinterpret_cast<uint4*>(out + h * out_head) = as_is ? raw[u] : Vec<T>::pack(y);
    }
  }
}

template <typename T, int D, bool LANED>
int launch(RopeParams& p, cudaStream_t st) {
  constexpr int GROUPS = kThreads / (D / Vec<T>::N);
  p.tile_tokens = 1;
  while (p.tile_tokens < GROUPS && p.tile_tokens < p.n_tokens) p.tile_tokens *= 2;
  p.tiles = (p.n_tokens + p.tile_tokens - 1) / p.tile_tokens;
  // Heads of a CTA: as many as leave two CTAs for every SM, so that cosines, weights and the launch of a CTA are shared,
  // but no more than eight turns (four: 85 us where eight take 77, sixteen 77).
  const int head_lanes = GROUPS / p.tile_tokens, most = std::max({p.heads[0], p.heads[1], p.heads[2]});
  p.chunk_heads = head_lanes;
  auto count = [&](int per) {
    long long n = 0;
    for (int k = 0; k < 3; ++k) n += (p.heads[k] + per - 1) / per;
    return n * p.tiles * p.batch;
  };
  while (p.chunk_heads < most && p.chunk_heads < 8 * kUnroll * head_lanes && count(2 * p.chunk_heads) >= 2ll * sm_count()) p.chunk_heads *= 2;
  const long long grid = count(p.chunk_heads);
  if (grid > 0x7fffffffll) {
    set_error("rotation: more rows than a launch has places for");
    return -2;
  }
  for (int k = 0; k < 3; ++k) p.chunks[k] = (p.heads[k] + p.chunk_heads - 1) / p.chunk_heads;
  launch_k(rope_kernel<T, D, LANED>, dim3((unsigned)grid), dim3(kThreads), (size_t)p.tile_tokens * p.pairs * sizeof(float2), st, p);
  return launched(1);
}

int launch_any(RopeParams& p, int dtype, int head_dim, cudaStream_t st) {
  const int n = dtype == HACK_F32 ? 4 : 8;
  const bool laned = p.layout != HACK_ROPE_HALF || p.pairs % n == 0;
  if (dtype == HACK_F32) {
    if (head_dim == 64) return laned ? launch<float, 64, true>(p, st) : launch<float, 64, false>(p, st);
    return laned ? launch<float, 128, true>(p, st) : launch<float, 128, false>(p, st);
  }
  if (head_dim == 64) return laned ? launch<__nv_bfloat16, 64, true>(p, st) : launch<__nv_bfloat16, 64, false>(p, st);
  return laned ? launch<__nv_bfloat16, 128, true>(p, st) : launch<__nv_bfloat16, 128, false>(p, st);
}

bool bad(const char* text) {
  set_error(text);
  return true;
}

bool bad_view(const void* ptr, const hack_strides_t& s, int batch, int heads, int tokens, int head_dim, int elt, bool written) {
  const char* text = view_error(ptr, s, batch, heads, tokens, head_dim, elt, written);
  return text ? bad(text) : false;
}

bool bad_plan(const hack_rope_plan_t* plan, int head_dim) {
  if (plan->head_dim != head_dim) return bad("the plan is for another head_dim");
  if ((plan->layout != HACK_ROPE_HALF && plan->layout != HACK_ROPE_PAIRS) || (plan->axes != 1 && plan->axes != 2) ||
      plan->rotary_dim < 2 || plan->rotary_dim > head_dim || plan->rotary_dim % (2 * plan->axes))
    return bad("the plan was not made by hack_rope_plan");
  return false;
}

void set_rotation(RopeParams& p, const hack_rope_plan_t* plan, const void* positions, int f32, long long stride, bool transpose) {
  p.positions = positions;
  p.positions_f32 = f32;
  p.positions_stride = stride;
  p.pairs = plan->rotary_dim / 2;
  p.axes = plan->axes;
  p.layout = plan->layout;
  p.gain_cs = plan->gain;
  p.sin_sign = transpose ? -1.f : 1.f;
  for (int i = 0; i < p.pairs; ++i) p.turns[i] = plan->freq[i] * 0.15915494309189533577;
}

hack_status_t done(int n) { return n >= 0 ? HACK_OK : n == -2 ? HACK_ERR_UNSUPPORTED : HACK_ERR_CUDA; }

// What both entry points ask of sizes and types; HACK_OK, or the error with its text.
hack_status_t check_sizes(int device, int dtype, int batch, int heads, int tokens, int head_dim) {
  if (dtype != HACK_F32 && dtype != HACK_BF16) { set_error("dtype must be HACK_F32 or HACK_BF16"); return HACK_ERR_UNSUPPORTED; }
  if (head_dim != 64 && head_dim != 128) { set_error("head_dim must be 64 or 128"); return HACK_ERR_UNSUPPORTED; }
  if (device < 0 || batch < 1 || heads < 1 || tokens < 0) {
    set_error("batch and heads must be positive, device and tokens not negative");
    return HACK_ERR_INVALID_ARG;
  }
  return HACK_OK;
}

}  // namespace
}  // namespace hack

extern "C" hack_status_t hack_rope_plan(int32_t head_dim, int32_t rotary_dim, int32_t layout, int32_t axes, double base,
                                        int32_t scaling, double factor, int64_t trained_length, double turns_fast,
                                        double turns_slow, hack_rope_plan_t* out) {
  using hack::set_error;
  auto invalid = [](const char* text) { set_error(text); return HACK_ERR_INVALID_ARG; };
  if (!out) return invalid("out is NULL");
  if (head_dim != 64 && head_dim != 128) { set_error("head_dim must be 64 or 128"); return HACK_ERR_UNSUPPORTED; }
  if (axes != 1 && axes != 2) return invalid("axes must be 1 or 2");
  if (rotary_dim < 2 || rotary_dim > head_dim || rotary_dim % (2 * axes)) return invalid("rotary_dim must be a multiple of 2 * axes in 2..head_dim");
  if (layout != HACK_ROPE_HALF && layout != HACK_ROPE_PAIRS) return invalid("unknown layout");
  if (scaling < HACK_ROPE_PLAIN || scaling > HACK_ROPE_BANDS) return invalid("unknown scaling");
  if (!(base > 1.0) || !std::isfinite(base)) return invalid("base must be finite and greater than 1");
  if (scaling != HACK_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return invalid("factor must be finite and at least 1");
  if (turns_fast == 0.0) turns_fast = 32.0;
  if (turns_slow == 0.0) turns_slow = 1.0;
  if (scaling == HACK_ROPE_BANDS && (trained_length < 1 || !(turns_slow > 0.0) || !(turns_fast > turns_slow) || !std::isfinite(turns_fast)))
    return invalid("bands need trained_length >= 1 and turns_fast > turns_slow > 0");
  hack_rope_plan_t p{};
  p.head_dim = head_dim;
  p.rotary_dim = rotary_dim;
  p.layout = layout;
  p.axes = axes;
  p.gain = 1.f;
  const int pairs = rotary_dim / 2 / axes, dim = 2 * pairs;    // of one axis
  const double b = scaling == HACK_ROPE_BASE ? base * std::pow(factor, (double)dim / std::max(dim - 2, 1)) : base;
  double low = 0, high = 0;
  if (scaling == HACK_ROPE_BANDS) {
    auto pair_of = [&](double turns) { return dim * std::log((double)trained_length / (turns * 6.283185307179586477)) / (2 * std::log(base)); };
    low = std::max(std::floor(pair_of(turns_fast)), 0.0);
    high = std::min(std::ceil(pair_of(turns_slow)), dim - 1.0);
    p.gain = (float)(1.0 + 0.1 * std::log(factor));
  }
  for (int i = 0; i < pairs; ++i) {
    double f = std::pow(b, -2.0 * i / dim);
    if (scaling == HACK_ROPE_LINEAR) f /= factor;
    if (scaling == HACK_ROPE_BANDS) {
      // (from `high` on by itself: where every pair turns less than turns_slow times, high is 0 or below and there is no ramp)
      const double ramp = i >= high ? 1.0 : std::min(1.0, std::max(0.0, (i - low) / std::max(high - low, 0.001)));
      f = f * (1.0 - ramp) + f / factor * ramp;
    }
    for (int a = 0; a < axes; ++a) p.freq[a * pairs + i] = f;
  }
  *out = p;
  return HACK_OK;
}

extern "C" hack_status_t hack_rope(const hack_rope_plan_t* plan, const hack_rope_args_t* args, const void* x, void* y,
                                   const void* positions, void* stream) {
  using namespace hack;
  if (!plan || !args) { set_error("plan or args is NULL"); return HACK_ERR_INVALID_ARG; }
  const hack_rope_args_t& a = *args;
  const hack_status_t st = check_sizes(a.device, a.dtype, a.batch, a.n_heads, a.n_tokens, plan->head_dim);
  if (st != HACK_OK) return st;
  if (bad_plan(plan, plan->head_dim)) return HACK_ERR_INVALID_ARG;
  if (a.n_tokens == 0) return HACK_OK;
  if (!positions || off_its_size(positions, 4)) { set_error("positions is NULL or not on a multiple of 4 bytes"); return HACK_ERR_INVALID_ARG; }
  const int elt = a.dtype == HACK_F32 ? 4 : 2;
  if (bad_view(x, a.x, a.batch, a.n_heads, a.n_tokens, plan->head_dim, elt, false) ||
      bad_view(y, a.y, a.batch, a.n_heads, a.n_tokens, plan->head_dim, elt, true))
    return HACK_ERR_INVALID_ARG;
  HACK_ON_DEVICE_OF(a.device);
  RopeParams p{};
  p.in[0] = x;
  p.out[0] = y;
  p.is[0] = a.x;
  p.os[0] = a.y;
  p.heads[0] = a.n_heads;
  p.batch = a.batch;
  p.n_tokens = a.n_tokens;
  set_rotation(p, plan, positions, a.positions_f32 != 0, a.positions_stride, a.transpose != 0);
  return done(launch_any(p, a.dtype, plan->head_dim, (cudaStream_t)stream));
}

extern "C" hack_status_t hack_qk_norm_rope(const hack_rope_plan_t* plan, const hack_qkv_args_t* args, const void* q, const void* k,
                                           const void* v, void* q_out, void* k_out, void* v_out, const void* positions,
                                           const float* q_weight, const float* k_weight, const float* q_gain,
                                           const float* k_gain, void* stream) {
  using namespace hack;
  if (!args) { set_error("args is NULL"); return HACK_ERR_INVALID_ARG; }
  const hack_qkv_args_t& a = *args;
  hack_status_t st = check_sizes(a.device, a.dtype, a.batch, a.n_heads, a.n_tokens, a.head_dim);
  if (st != HACK_OK) return st;
  if ((!k != !k_out) || (!v != !v_out)) { set_error("k and k_out, v and v_out: both or neither"); return HACK_ERR_INVALID_ARG; }
  if ((k || v) && a.n_kv_heads < 1) { set_error("n_kv_heads must be positive"); return HACK_ERR_INVALID_ARG; }
  if (a.norm < HACK_NORM_NONE || a.norm > HACK_NORM_L2) { set_error("unknown norm"); return HACK_ERR_INVALID_ARG; }
  if (a.norm != HACK_NORM_NONE && !(a.eps > 0.f && std::isfinite(a.eps))) { set_error("eps must be finite and positive"); return HACK_ERR_INVALID_ARG; }
  // (a row without length is multiplied by it)
  if (a.norm == HACK_NORM_L2 && !std::isfinite(1.f / a.eps)) { set_error("the L2 norm needs an eps whose reciprocal is finite"); return HACK_ERR_INVALID_ARG; }
  if (!plan != !positions) { set_error("plan and positions: both or neither"); return HACK_ERR_INVALID_ARG; }
  if (plan && bad_plan(plan, a.head_dim)) return HACK_ERR_INVALID_ARG;
  if (a.n_tokens == 0) return HACK_OK;
  for (const void* x : {positions, (const void*)q_weight, (const void*)k_weight, (const void*)q_gain, (const void*)k_gain})
    if (off_its_size(x, 4)) { set_error("positions, weights or gains are not on a multiple of 4 bytes"); return HACK_ERR_INVALID_ARG; }
  const int elt = a.dtype == HACK_F32 ? 4 : 2;
  const void* in[3] = {q, k, v};
  void* out[3] = {q_out, k_out, v_out};
  const hack_strides_t is[3] = {a.q, a.k, a.v}, os[3] = {a.q_out, a.k_out, a.v_out};
  RopeParams p{};
  for (int i = 0; i < 3; ++i) {
    if (i > 0 && !in[i]) continue;
    const int heads = i == 0 ? a.n_heads : a.n_kv_heads;
    if (bad_view(in[i], is[i], a.batch, heads, a.n_tokens, a.head_dim, elt, false) ||
        bad_view(out[i], os[i], a.batch, heads, a.n_tokens, a.head_dim, elt, true))
      return HACK_ERR_INVALID_ARG;
    p.in[i] = in[i];
    p.out[i] = out[i];
    p.is[i] = is[i];
    p.os[i] = os[i];
    p.heads[i] = heads;
  }
  HACK_ON_DEVICE_OF(a.device);
  p.weight[0] = q_weight;
  p.weight[1] = k_weight;
  p.gain[0] = q_gain;
  p.gain[1] = k_gain;
  p.batch = a.batch;
  p.n_tokens = a.n_tokens;
  p.norm = a.norm;
  p.eps = a.eps;
  p.inv_eps = 1.f / a.eps;
  if (plan) set_rotation(p, plan, positions, a.positions_f32 != 0, a.positions_stride, false);
  return done(launch_any(p, a.dtype, a.head_dim, (cudaStream_t)stream));
}
