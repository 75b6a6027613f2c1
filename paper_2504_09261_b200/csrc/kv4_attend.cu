// Attention over a cache of 4 bits (format and masks: hack.h).
//
// A stored element is c * s with c of four bits and s of four significant bits, which bf16 holds exactly: the matrix
// instructions see what is stored, not a rounding of it.  The query rows of the heads that share a stored head are the rows
// of one product: m = token * group + head, in tiles of 16.
//
// kv4_attend_kernel: few rows, or fp32.  A warp takes chunks of 32 stored rows through a ring of its own in shared memory
// (cp.async, so that neither their place nor the end of a head has to be aligned); its lanes read the codes there in the
// order of the matrix fragments - the order of the elements inside a product is free as long as both operands
// have it - so that a value costs a shift, a mask and an FMA for two.  Softmax with a running maximum that is raised only when
// a logit exceeds it by 2^16; a CTA's warps are merged in shared memory, CTAs that share the rows of a head (`splits`)
// through partial results in the workspace, which kv4_combine_kernel adds up.
// fp32: queries and probabilities as sums of three bf16 numbers, which is all of their 24 bits.
#include <algorithm>
#include <cmath>
#include <string>

#include "entry_checks.h"
#include "kv4.cuh"
#include "kv4_attend.h"
#include "tc_ptx.cuh"

namespace hack {
namespace {

using namespace kv4;
using ptx::ex2;
using ptx::mma16816;
using ptx::smem_u32;

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kRows = 16;                    // query rows of a CTA
constexpr int kChunk = 32;                   // stored rows of a turn of a warp
constexpr int kStages = 3;
constexpr float kRaise = 16.f;               // log2 by which a logit may exceed the reference maximum
constexpr int kTcRows = 48;                  // bf16: from so many query rows of a stored head on, tiles of 128 on the tensor cores
constexpr uint32_t kWaitPolls = 1u << 24;    // of a wait in that kernel: a large part of a second at least

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
template <int BYTES> __device__ __forceinline__ void cp_async_small(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(live ? BYTES : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

template <int D> struct Ring {
  static constexpr int kCodes = kChunk * D / 2, kScales = kChunk * D / 16;   // bytes of a chunk, of K or V
  static constexpr int kStage = 2 * (kCodes + kScales);
  static constexpr int kWarp = kStages * kStage;
};
// The ring, later the warps' outputs; fp32: the query's fragments behind it.
template <int D, bool F32> constexpr size_t smem_bytes() {
  constexpr size_t ring = (size_t)kWarps * Ring<D>::kWarp, merge = (size_t)kWarps * kRows * D * 4;
  return (ring > merge ? ring : merge) + (F32 ? 3 * (D / 16) * 32 * 16 : 0);
}

template <int D, bool F32>
__global__ void __launch_bounds__(kThreads) kv4_attend_kernel(const __grid_constant__ Kv4AttendParams p) {
  constexpr int KS = D / 16;                 // k-steps of Q K^T, and a lane's 4 codes each
  constexpr int NT = D / 8;                  // column tiles of the output
  constexpr int CODES = Ring<D>::kCodes, SCALES = Ring<D>::kScales;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float merge_m[kWarps][kRows], merge_l[kWarps][kRows];
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, t = lane & 3;
  const int split = blockIdx.x, unit = blockIdx.y + blockIdx.z * gridDim.y;
  if (unit >= p.units) return;
  const int head = unit / p.tiles, tile = unit - head * p.tiles;          // stored head, tile of query rows
  const int b = head / p.kv_heads, kvh = head - b * p.kv_heads;
  const int nq = p.new_lens ? min(max(p.new_lens[b], 0), p.n_queries) : p.n_queries;
  const int len = kv4_length(p, head, nq);
  const int rows = nq * p.group, m0 = tile * kRows;
  const Kv4Range range = kv4_range(p, len, nq, m0, min(m0 + kRows, rows) - 1);
  const int chunks1 = (range.sink_end + kChunk - 1) / kChunk, chunks = m0 < rows ? chunks1 + (range.hi - range.lo + kChunk - 1) / kChunk : 0;
  const int c_begin = (int)((long long)chunks * split / p.splits), c_end = (int)((long long)chunks * (split + 1) / p.splits);

  const long long row0 = first_row(p.planes, head);
  const uint32_t ring = smem_u32(smem) + warp * Ring<D>::kWarp;
  // Chunk c: its first stored row and the end of the rows that count
  auto chunk_at = [&](int c, int& first, int& end) {
    first = c < chunks1 ? c * kChunk : range.lo + (c - chunks1) * kChunk;
    end = c < chunks1 ? range.sink_end : range.hi;
  };
  auto fetch = [&](int c, int stage) {
    if (c < c_end) {
      int first, end;
      chunk_at(c, first, end);
      const uint32_t at = ring + stage * Ring<D>::kStage;
      constexpr int PIECES = D / 32;         // 16-byte pieces of a row's codes
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int piece = i * 32 + lane, row = piece / PIECES;
        const bool live = first + row < end;
        const long long src = (row0 + (live ? first + row : 0)) * (D / 2) + (piece % PIECES) * 16;
        cp_async16(at + piece * 16, p.planes.k_codes + src, live);
        cp_async16(at + CODES + piece * 16, p.planes.v_codes + src, live);
      }
      const bool live = first + lane < end;
      const long long src = (row0 + (live ? first + lane : 0)) * (D / 16);
      cp_async_small<D / 16>(at + 2 * CODES + lane * (D / 16), p.planes.k_scales + src, live);
      cp_async_small<D / 16>(at + 2 * CODES + SCALES + lane * (D / 16), p.planes.v_scales + src, live);
    }
    cp_async_commit();
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) fetch(c_begin + warp + s * kWarps, s);

  // Query fragments.  Lane t of a row holds its elements [t D/4, (t+1) D/4): code word w of them is two k-steps, of which step
  // 2w + u takes elements 2u and 2u + 4 as its columns 2t and 2t + 1, and 2u + 1 and 2u + 5 as 2t + 8 and 2t + 9.
  uint32_t qf[F32 ? 1 : KS][4];
  uint4* const q_smem = reinterpret_cast<uint4*>(smem + smem_bytes<D, false>());   // fp32: [3][KS][32]
  const int row_token[2] = {(m0 + r) / p.group, (m0 + r + 8) / p.group};
  const int row_head[2] = {(m0 + r) % p.group, (m0 + r + 8) % p.group};
  const bool row_live[2] = {m0 + r < rows, m0 + r + 8 < rows};
#pragma unroll
  for (int w = 0; w < KS / 2; ++w) {
    if (F32 && w % kWarps != warp) continue;           // the warps share the fragments
    uint32_t part[F32 ? 3 : 1][2][4];                  // per row: pairs (0,4) (1,5) (2,6) (3,7)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const long long at = b * p.q_stride.batch + (long long)(kvh * p.group + row_head[i]) * p.q_stride.head + row_token[i] * p.q_stride.token +
                           t * (D / 4) + w * 8;
      if constexpr (F32) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float4 v = row_live[i] ? *reinterpret_cast<const float4*>(static_cast<const float*>(p.q) + at + 4 * e) : make_float4(0.f, 0.f, 0.f, 0.f);
          x[4 * e] = v.x; x[4 * e + 1] = v.y; x[4 * e + 2] = v.z; x[4 * e + 3] = v.w;
        }
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t h = pack2(x[e], x[e + 4]);
            part[k][i][e] = h;
            x[e] -= low(h);
            x[e + 4] -= high(h);
          }
      } else {
        const uint4 v = row_live[i] ? *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + at) : make_uint4(0, 0, 0, 0);
        part[0][i][0] = __byte_perm(v.x, v.z, 0x5410);
        part[0][i][1] = __byte_perm(v.x, v.z, 0x7632);
        part[0][i][2] = __byte_perm(v.y, v.w, 0x5410);
        part[0][i][3] = __byte_perm(v.y, v.w, 0x7632);
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (F32) {
#pragma unroll
        for (int k = 0; k < 3; ++k)
          q_smem[(k * KS + 2 * w + u) * 32 + lane] = make_uint4(part[k][0][2 * u], part[k][1][2 * u], part[k][0][2 * u + 1], part[k][1][2 * u + 1]);
      } else {
        qf[2 * w + u][0] = part[0][0][2 * u];
        qf[2 * w + u][1] = part[0][1][2 * u];
        qf[2 * w + u][2] = part[0][0][2 * u + 1];
        qf[2 * w + u][3] = part[0][1][2 * u + 1];
      }
    }
  }
  if (F32) __syncthreads();

  float o[NT][4];
#pragma unroll
  for (int j = 0; j < NT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
  float m[2] = {kNoLogit, kNoLogit}, l[2] = {0.f, 0.f};
  const float c = p.scale_log2;
  const int at_row[2] = {len - nq + row_token[0], len - nq + row_token[1]};

  int stage = 0;
  for (int ch = c_begin + warp; ch < c_end; ch += kWarps) {
    cp_async_wait<kStages - 2>();
    __syncwarp();
    int first, end;
    chunk_at(ch, first, end);
    const unsigned char* at = smem + warp * Ring<D>::kWarp + stage * Ring<D>::kStage;
    // ---- logits: four tiles of eight stored rows
    float s[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
      const int row = 8 * j + r;
      uint32_t w[KS / 2];
      if constexpr (D == 128) {
        const uint4 v = *reinterpret_cast<const uint4*>(at + row * 64 + t * 16);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(at + row * 32 + t * 8);
        w[0] = v.x; w[1] = v.y;
      }
#pragma unroll
      for (int blk = 0; blk < D / 64; ++blk) {
        const uint32_t byte = at[2 * CODES + row * (D / 16) + t * (D / 64) + blk];
        const Scale2 sc = scale2(byte | byte << 16);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t word = w[2 * blk + i];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t b0 = values2(word, 8 * u, sc), b1 = values2(word, 8 * u + 4, sc);
            const int ks = 2 * (2 * blk + i) + u;
            if constexpr (F32) {
#pragma unroll
              for (int k = 2; k >= 0; --k) {
                const uint4 a = q_smem[(k * KS + ks) * 32 + lane];
                mma16816(s[j], reinterpret_cast<const uint32_t*>(&a), b0, b1);
              }
            } else {
              mma16816(s[j], qf[ks], b0, b1);
            }
          }
        }
      }
    }
    // ---- softmax.  Stored rows of this lane: first + 8 j + 2 t + (0, 1)
    if (first + kChunk > end || !kv4_all_see(p, range, first)) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = first + 8 * j + 2 * t + (e & 1);
          if (row >= end || !kv4_sees(p, at_row[e >> 1], row)) s[j][e] = -INFINITY;
        }
    }
    float top[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      top[i] = fmaxf(fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1])),
                     fmaxf(fmaxf(s[2][2 * i], s[2][2 * i + 1]), fmaxf(s[3][2 * i], s[3][2 * i + 1])));
    }
    if (__any_sync(0xffffffffu, (top[0] - m[0]) * c > kRaise || (top[1] - m[1]) * c > kRaise)) {
      float f[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float mx = fmaxf(m[i], top[i]);
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        f[i] = ex2((m[i] - mx) * c);
        m[i] = mx;
        l[i] *= f[i];
      }
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        o[j][0] *= f[0]; o[j][1] *= f[0];
        o[j][2] *= f[1]; o[j][3] *= f[1];
      }
    }
    // (a row that has seen nothing yet has a reference of -3.4e38, whose product may overflow)
    const float nmc[2] = {m[0] == kNoLogit ? 0.f : -m[0] * c, m[1] == kNoLogit ? 0.f : -m[1] * c};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] = ex2(fmaf(s[j][e], c, nmc[e >> 1]));
    // ---- values: two steps of sixteen stored rows; the sums are of the probabilities as the products see them
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t pf[F32 ? 3 : 1][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x = s[2 * k + (i >> 1)][2 * (i & 1)], y = s[2 * k + (i >> 1)][2 * (i & 1) + 1];
        if constexpr (F32) {
          l[i & 1] += x + y;
#pragma unroll
          for (int q = 0; q < 3; ++q) {
            const uint32_t h = pack2(x, y);
            pf[q][i] = h;
            x -= low(h);
            y -= high(h);
          }
        } else {
          pf[0][i] = pack2(x, y);
          l[i & 1] += low(pf[0][i]) + high(pf[0][i]);
        }
      }
      const unsigned char* codes = at + CODES + r * (D / 16);
      const unsigned char* scales = at + 2 * CODES + SCALES + (r * (D / 8)) / kBlock;
      uint32_t w[4][D / 64];
      uint32_t byte[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {          // rows 2t, 2t + 1, 2t + 8, 2t + 9
        const int row = 16 * k + 2 * t + (i & 1) + 8 * (i >> 1);
        if constexpr (D == 128) {
          const uint2 v = *reinterpret_cast<const uint2*>(codes + row * 64);
          w[i][0] = v.x; w[i][1] = v.y;
        } else {
          w[i][0] = *reinterpret_cast<const uint32_t*>(codes + row * 32);
        }
        byte[i] = scales[row * (D / 16)];
      }
      const Scale2 s0 = scale2(byte[0] | byte[1] << 16), s1 = scale2(byte[2] | byte[3] << 16);
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t sel = half ? 0x7632 : 0x5410;
          const uint32_t w0 = __byte_perm(w[0][x], w[1][x], sel), w1 = __byte_perm(w[2][x], w[3][x], sel);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t b0 = values2(w0, 4 * i, s0), b1 = values2(w1, 4 * i, s1);
#pragma unroll
            for (int q = F32 ? 2 : 0; q >= 0; --q) mma16816(o[8 * x + 4 * half + i], pf[q], b0, b1);
          }
        }
    }
    __syncwarp();
    fetch(ch + (kStages - 1) * kWarps, stage == 0 ? kStages - 1 : stage - 1);
    stage = stage == kStages - 1 ? 0 : stage + 1;
  }
  cp_async_wait<0>();

  // ---- the warps' shares
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    if (t == 0) merge_m[warp][r + 8 * i] = m[i];
  }
  __syncthreads();                           // (and every warp is done with its ring)
  float f[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float mx = merge_m[0][r + 8 * i];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) mx = fmaxf(mx, merge_m[w][r + 8 * i]);
    f[i] = ex2((m[i] - mx) * c);
    if (t == 0) merge_l[warp][r + 8 * i] = l[i] * f[i];
  }
  float* const mine = reinterpret_cast<float*>(smem) + warp * kRows * D;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < NT; j += 4)
        *reinterpret_cast<float4*>(mine + (r + 8 * i) * D + (2 * t + e) * NT + j) =
            make_float4(o[j][2 * i + e] * f[i], o[j + 1][2 * i + e] * f[i], o[j + 2][2 * i + e] * f[i], o[j + 3][2 * i + e] * f[i]);
  __syncthreads();
  for (int x = threadIdx.x; x < kRows * D / 4; x += kThreads) {
    const int row = x / (D / 4), d = (x - row * (D / 4)) * 4;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    float total = 0.f, mx = kNoLogit;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem) + (w * kRows + row) * D + d);
      sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
      total += merge_l[w][row];
      mx = fmaxf(mx, merge_m[w][row]);
    }
    if (m0 + row >= rows) continue;
    if (p.splits > 1) {
      float* part = p.partial + ((long long)unit * p.splits + split) * (kRows * (D + 2));
      *reinterpret_cast<float4*>(part + row * D + d) = sum;
      if (d == 0) {
        part[kRows * D + 2 * row] = mx;
        part[kRows * D + 2 * row + 1] = total;
      }
    } else {
      kv4_store<F32>(p, b, kvh, m0 + row, d, sum, total);
    }
  }
}

// Partial results of the splits added up: D / 4 threads for a query row.
template <int D, bool F32>
__global__ void __launch_bounds__(256) kv4_combine_kernel(const __grid_constant__ Kv4AttendParams p) {
  pdl_wait();
  constexpr int LANES = D / 4, PER = 256 / LANES;
  const long long index = (long long)blockIdx.x * PER + threadIdx.x / LANES;
  const int unit = (int)(index / p.tile_rows), row = (int)(index - (long long)unit * p.tile_rows), d = (threadIdx.x % LANES) * 4;
  if (unit >= p.units) return;
  const int head = unit / p.tiles, tile = unit - head * p.tiles;
  const int b = head / p.kv_heads, kvh = head - b * p.kv_heads;
  const int nq = p.new_lens ? min(max(p.new_lens[b], 0), p.n_queries) : p.n_queries;
  const int m = tile * p.tile_rows + row;
  if (m >= nq * p.group) return;
  const long long step = (long long)p.tile_rows * (D + 2);
  const float* part = p.partial + (long long)unit * p.splits * step;
  const float* stats = part + (long long)p.tile_rows * D + 2 * row;
  float mx = kNoLogit;
  for (int s = 0; s < p.splits; ++s) mx = fmaxf(mx, stats[s * step]);
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  float total = 0.f;
  for (int s = 0; s < p.splits; ++s) {
    const float f = ex2((stats[s * step] - mx) * p.scale_log2);
    const float4 v = *reinterpret_cast<const float4*>(part + s * step + (long long)row * D + d);
    total += f * stats[s * step + 1];
    sum.x = fmaf(f, v.x, sum.x); sum.y = fmaf(f, v.y, sum.y); sum.z = fmaf(f, v.z, sum.z); sum.w = fmaf(f, v.w, sum.w);
  }
  kv4_store<F32>(p, b, kvh, m, d, sum, total);
}

template <int D, bool F32>
int launch_attend(const Kv4AttendParams& p, cudaStream_t st) {
  if (p.tile_rows == kRows) {
    constexpr size_t smem = smem_bytes<D, F32>();
    if (!allow_dynamic_smem(kv4_attend_kernel<D, F32>, smem)) return -1;
    const int y = std::min(p.units, 32768);
    launch_k(kv4_attend_kernel<D, F32>, dim3(p.splits, y, (p.units + y - 1) / y), dim3(kThreads), smem, st, p);
  } else if (launch_kv4_attend_tc(p, D, st) < 0) {
    return -1;
  }
  if (p.splits > 1) {
    constexpr int PER = 256 / (D / 4);
    launch_k(kv4_combine_kernel<D, F32>, dim3((unsigned)(((long long)p.units * p.tile_rows + PER - 1) / PER)), dim3(256), 0, st, p);
  }
  return launched(1);
}

hack_status_t invalid(const char* text) {
  set_error(text);
  return HACK_ERR_INVALID_ARG;
}

hack_status_t check_attend(const hack_kv4_t* kv, const hack_kv4_attend_t* a) {
  const hack_status_t s = kv4_check(kv);
  if (s != HACK_OK) return s;
  if (!a) return invalid("args is NULL");
  if (a->dtype != HACK_F32 && a->dtype != HACK_BF16) { set_error("dtype must be HACK_F32 or HACK_BF16"); return HACK_ERR_UNSUPPORTED; }
  if (a->n_heads < 1 || a->n_heads % kv->n_kv_heads) return invalid("n_heads must be a multiple of n_kv_heads");
  if (a->n_queries < 0 || a->max_len < 0) return invalid("n_queries and max_len must not be negative");
  if (a->window < 0 || a->n_sink < 0) return invalid("window and n_sink must not be negative");
  if (a->wait_polls < 0) return invalid("wait_polls must not be negative");
  if (!(a->sm_scale >= 0.f) || !std::isfinite(a->sm_scale)) return invalid("sm_scale must be finite and non-negative");
  if ((long long)a->n_queries * (a->n_heads / kv->n_kv_heads) > 0x3fffffffll) return invalid("too many queries");
  return HACK_OK;
}

// Sizes of the launches, from those of the call alone.
hack_status_t plan(const hack_kv4_t* kv, const hack_kv4_attend_t* a, Kv4AttendParams& p, size_t& workspace) {
  p.kv_heads = kv->n_kv_heads;
  p.group = a->n_heads / kv->n_kv_heads;
  p.n_queries = a->n_queries;
  p.max_len = std::min(a->max_len, kv->cap);
  p.causal = a->causal != 0;
  p.window = a->window;
  p.n_sink = a->window > 0 ? a->n_sink : 0;
  p.appended = a->appended != 0;
  const int heads = kv->batch * kv->n_kv_heads, rows = a->n_queries * p.group;
  const bool tc = a->dtype == HACK_BF16 && rows >= kTcRows;
  p.tile_rows = tc ? 128 : kRows;
  p.tiles = (rows + p.tile_rows - 1) / p.tile_rows;
  const long long units = (long long)heads * p.tiles;
  if (units > 0x3fffffffll) { set_error("more query rows than a launch has places for"); return HACK_ERR_UNSUPPORTED; }
  p.units = (int)units;
  // rows that a tile of queries walks at most
  long long walked = p.max_len;
  if (p.window > 0) walked = std::min<long long>(walked, (long long)p.window + p.n_sink + p.n_queries);
  const int sms = sm_count();
  if (tc) {
    p.tiles_per_cta = units <= sms ? 1 : 2;
    const long long ctas = (long long)heads * ((p.tiles + p.tiles_per_cta - 1) / p.tiles_per_cta);
    p.splits = (int)std::max<long long>(1, std::min<long long>((walked + 127) / 128 / 4, sms / ctas));
  } else {
    const long long turns = (walked + kChunk * kWarps - 1) / (kChunk * kWarps);
    p.splits = (int)std::max<long long>(1, std::min<long long>(turns / 2, 4ll * sms / units));
  }
  p.wait_polls = a->wait_polls > 0 ? (uint32_t)a->wait_polls : kWaitPolls;
  workspace = p.splits > 1 ? (size_t)p.units * p.splits * p.tile_rows * (kv->head_dim + 2) * 4 : 0;
  return HACK_OK;
}

}  // namespace
}  // namespace hack

extern "C" hack_status_t hack_kv4_workspace(const hack_kv4_t* kv, const hack_kv4_attend_t* args, size_t* bytes) {
  using namespace hack;
  const hack_status_t s = check_attend(kv, args);
  if (s != HACK_OK) return s;
  if (!bytes) return invalid("bytes is NULL");
  HACK_ON_DEVICE_OF(kv->device);
  Kv4AttendParams p{};
  return plan(kv, args, p, *bytes);
}

extern "C" hack_status_t hack_kv4_attend(const hack_kv4_t* kv, const hack_kv4_attend_t* args, const void* q, void* out,
                                         const int32_t* lens, const int32_t* new_lens, void* workspace, void* stream) {
  using namespace hack;
  hack_status_t s = check_attend(kv, args);
  if (s != HACK_OK) return s;
  const hack_kv4_attend_t& a = *args;
  if (a.n_queries == 0) return HACK_OK;
  if (!lens) return invalid("lens is NULL");
  const int elt = a.dtype == HACK_F32 ? 4 : 2;
  const char* text = view_error(q, a.q, kv->batch, a.n_heads, a.n_queries, kv->head_dim, elt, false);
  if (!text) text = view_error(out, a.out, kv->batch, a.n_heads, a.n_queries, kv->head_dim, elt, true);
  if (text) return invalid(text);
  HACK_ON_DEVICE_OF(kv->device);
  Kv4AttendParams p{};
  size_t need = 0;
  s = plan(kv, args, p, need);
  if (s != HACK_OK) return s;
  if (need > 0 && (!workspace || a.workspace_bytes < 0 || (size_t)a.workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15)))
    return invalid("the workspace is smaller than hack_kv4_workspace asks for, or not 16-byte aligned");
  p.planes = kv4_planes(kv);
  p.lens = lens;
  p.new_lens = new_lens;
  p.q = q;
  p.out = out;
  p.q_stride = a.q;
  p.out_stride = a.out;
  p.scale_log2 = (a.sm_scale > 0.f ? a.sm_scale : 1.f / std::sqrt((float)kv->head_dim)) * 1.4426950408889634f;
  p.out_sectors = reinterpret_cast<uintptr_t>(out) % 32 == 0 && a.out.batch * elt % 32 == 0 && a.out.head * elt % 32 == 0 && a.out.token * elt % 32 == 0;
  p.partial = static_cast<float*>(workspace);
  cudaStream_t st = (cudaStream_t)stream;
  int n;
  if (kv->head_dim == 64) n = a.dtype == HACK_F32 ? launch_attend<64, true>(p, st) : launch_attend<64, false>(p, st);
  else n = a.dtype == HACK_F32 ? launch_attend<128, true>(p, st) : launch_attend<128, false>(p, st);
  return n < 0 ? HACK_ERR_CUDA : HACK_OK;
}
