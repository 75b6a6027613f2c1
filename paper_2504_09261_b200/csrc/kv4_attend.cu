// Attention over a cache of 4 bits (format and masks: hack.h).
//
// A stored element is c * s with c of four bits and s of four significant bits, which bf16 holds exactly: the matrix
// instructions see what is stored, not a rounding of it.  The query rows of the heads that share a stored head are the rows
// of one product: m = token * group + head, in tiles of 8, 16 or 128.
//
// kv4_attend_kernel: few rows, or fp32.  A warp takes chunks of 32 stored rows through a ring of its own in shared memory
// (cp.async, so that neither their place nor the end of a head has to be aligned); its lanes read the codes there in the
// order of the matrix fragments - the order of the elements inside a product is free as long as both operands
// have it - so that a value costs a shift, a mask and an FMA for two.  The stored rows are the 16 rows of a product
// and the queries its eight columns (K Q^T, then V^T P^T): one query, or the few that share a stored head, leave as little of it
// empty as can be, and hold half the registers of the other way round.  Softmax with a running maximum that is
// raised only when a logit exceeds it by 2^16; a CTA's warps are merged in shared memory, CTAs that share the rows of a head
// (`splits`) as a cluster, through each other's shared memory, or through partial results in the workspace, which kv4_combine_kernel
// adds up.
// bf16: a probability is rounded once for the product with the values, which costs as much accuracy again as the rounding of the
// result; as the sum of two bf16 numbers it costs a tenth of the time instead (32 heads of up to 65 536 rows 63 and 70 us).  fp32:
// queries and probabilities as sums of three bf16 numbers, which is all of their 24 bits.
// kv4_attend_tc_kernel (kv4_attend_tc.cu): bf16, many query rows.
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
using ptx::smem_u32;

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kCombineThreads = 256, kMaxSplits = 64, kMaxCluster = 8;
constexpr int kChunk = 32;                   // stored rows of a turn of a warp
constexpr int kStages = 3;
constexpr float kRaise = 16.f;               // log2 by which a logit may exceed the reference maximum
constexpr uint32_t kWaitPolls = 1u << 24;    // of a wait in that kernel: a large part of a second at least

template <int BYTES> __device__ __forceinline__ void cp_async(uint32_t dst, const void* src, int bytes) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// D += A B, 16 x 8 x 16.  (Not volatile: the chains of independent products may be interleaved.)
__device__ __forceinline__ void mma(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit numbers in fragment order, transposed
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Shared memory of a cluster's CTAs
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, int rank) {
  uint32_t x;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(x) : "r"(addr), "r"(rank));
  return x;
}
__device__ __forceinline__ float4 load_shared4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float2 load_shared2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
// (of every thread; the loops ahead of it are left by part of a warp at a time, and an aligned instruction is for whole ones)
__device__ __forceinline__ void cluster_barrier() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int D> struct Ring {
  static constexpr int kCodes = kChunk * D / 2, kScales = kChunk * D / 16;   // bytes of a chunk, of K or V
  static constexpr int kStage = 2 * (kCodes + kScales);
  static constexpr int kWarp = kStages * kStage;
};
// The ring, later the warps' outputs; fp32: the query's fragments behind it.
template <int D, bool F32, int NQ> constexpr size_t smem_bytes() {
  constexpr size_t ring = (size_t)kWarps * Ring<D>::kWarp, merge = (size_t)(kWarps + 1) * 8 * NQ * D * 4;
  return (ring > merge ? ring : merge) + (F32 ? 3 * NQ * (D / 16) * 32 * 8 : 0);
}

// CTAs that an SM holds: of 128, 168 or 255 registers a thread
constexpr int ctas_per_sm(bool f32, int nq) { return 5 - nq - (f32 ? 1 : 0); }

// NQ: groups of eight query rows of a CTA
template <int D, bool F32, int NQ>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(F32, NQ)) kv4_attend_kernel(const __grid_constant__ Kv4AttendParams p) {
  constexpr int ROWS = 8 * NQ;
  constexpr int KS = D / 16;                 // k-steps of K Q^T; tiles of 16 elements of the output
  constexpr int NP = F32 ? 3 : 1;            // bf16 numbers that a query element, and a probability, is the sum of
  constexpr int CODES = Ring<D>::kCodes, SCALES = Ring<D>::kScales;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float merge_m[kWarps][ROWS], merge_l[kWarps][ROWS];
  __shared__ float2 cta_stats[ROWS];         // clusters: the CTA's reference maximum and sum of every row
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, t = lane & 3;
  const int split = blockIdx.x, unit = blockIdx.y + blockIdx.z * gridDim.y;
  if (unit >= p.units) return;
  const int head = unit / p.tiles, tile = unit - head * p.tiles;          // stored head, tile of query rows
  const int b = head / p.kv_heads, kvh = head - b * p.kv_heads;
  const int nq = p.new_lens ? min(max(p.new_lens[b], 0), p.n_queries) : p.n_queries;
  const int len = kv4_length(p, head, nq);
  const int rows = nq * p.group, m0 = tile * ROWS;
  const Kv4Range range = kv4_range(p, len, nq, m0, min(m0 + ROWS, rows) - 1);
  const int chunks1 = (range.sink_end + kChunk - 1) / kChunk, chunks = m0 < rows ? kv4_chunks(range, kChunk) : 0;
  const int c_begin = (int)((long long)chunks * split / p.splits), c_end = (int)((long long)chunks * (split + 1) / p.splits);

  const uint32_t ring = smem_u32(smem) + warp * Ring<D>::kWarp;
  const long long row0 = first_row(p.planes, head);
  // the lane's place in a chunk's codes and scales, which are runs of bytes
  const unsigned char* const kc = p.planes.k_codes + row0 * (D / 2) + lane * 16;
  const unsigned char* const vc = p.planes.v_codes + row0 * (D / 2) + lane * 16;
  const unsigned char* const ks_ = p.planes.k_scales + (row0 + lane) * (D / 16);
  const unsigned char* const vs_ = p.planes.v_scales + (row0 + lane) * (D / 16);
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
      constexpr int PIECES = CODES / 512;    // of a lane
      const long long off = (long long)first * (D / 2), off_s = (long long)first * (D / 16);
      if (first + kChunk <= end) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          cp_async<16>(at + i * 512 + lane * 16, kc + off + i * 512, 16);
          cp_async<16>(at + CODES + i * 512 + lane * 16, vc + off + i * 512, 16);
        }
        cp_async<D / 16>(at + 2 * CODES + lane * (D / 16), ks_ + off_s, D / 16);
        cp_async<D / 16>(at + 2 * CODES + SCALES + lane * (D / 16), vs_ + off_s, D / 16);
      } else {                               // rows behind the end are filled with zeros and not read
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          const int bytes = (i * 512 + lane * 16) / (D / 2) < end - first ? 16 : 0;
          cp_async<16>(at + i * 512 + lane * 16, bytes ? kc + off + i * 512 : kc, bytes);
          cp_async<16>(at + CODES + i * 512 + lane * 16, bytes ? vc + off + i * 512 : vc, bytes);
        }
        const int bytes = lane < end - first ? D / 16 : 0;
        cp_async<D / 16>(at + 2 * CODES + lane * (D / 16), bytes ? ks_ + off_s : p.planes.k_scales, bytes);
        cp_async<D / 16>(at + 2 * CODES + SCALES + lane * (D / 16), bytes ? vs_ + off_s : p.planes.v_scales, bytes);
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) fetch(c_begin + warp + s * kWarps, s);

  // Query fragments (the second operand: 16 elements x 8 query rows).  Lane t of row r holds its elements [t D/4, (t+1) D/4): code
  // word w of them is two k-steps, of which step 2w + u takes elements 2u and 2u + 4 as its 2t and 2t + 1, and 2u + 1 and 2u + 5
  // as 2t + 8 and 2t + 9.
  uint2 qf[F32 ? 1 : NQ][F32 ? 1 : KS];
  uint2* const q_smem = reinterpret_cast<uint2*>(smem + smem_bytes<D, false, NQ>());   // fp32: [3][NQ][KS][32]
#pragma unroll
  for (int g = 0; g < NQ; ++g) {
    const int m = m0 + 8 * g + r, token = m / p.group;
    const bool live = m < rows;
    const long long at = b * p.q_stride.batch + (long long)(kvh * p.group + m - token * p.group) * p.q_stride.head + token * p.q_stride.token + t * (D / 4);
#pragma unroll
    for (int w = 0; w < KS / 2; ++w) {
      if constexpr (F32) {
        if (w % kWarps != warp) continue;                // the warps share the fragments
        float x[8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float4 v = live ? *reinterpret_cast<const float4*>(static_cast<const float*>(p.q) + at + w * 8 + 4 * e) : make_float4(0.f, 0.f, 0.f, 0.f);
          x[4 * e] = v.x; x[4 * e + 1] = v.y; x[4 * e + 2] = v.z; x[4 * e + 3] = v.w;
        }
#pragma unroll
        for (int k = 0; k < NP; ++k) {
          uint32_t h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            h[e] = pack2(x[e], x[e + 4]);
            x[e] -= low(h[e]);
            x[e + 4] -= high(h[e]);
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) q_smem[((k * NQ + g) * KS + 2 * w + u) * 32 + lane] = make_uint2(h[2 * u], h[2 * u + 1]);
        }
      } else {
        const uint4 v = live ? *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + at + w * 8) : make_uint4(0, 0, 0, 0);
        qf[g][2 * w] = make_uint2(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632));
        qf[g][2 * w + 1] = make_uint2(__byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
      }
    }
  }
  if (F32) __syncthreads();

  // Of group g the lane has query rows 8 g + 2 t and + 1: logits of stored rows r and r + 8 of a tile of 16, outputs of elements
  // r D/8 + 2 i and + 1.
  float o[NQ][KS][4], m[NQ][2], l[NQ][2];
  int at_row[NQ][2];                           // positions
#pragma unroll
  for (int g = 0; g < NQ; ++g) {
#pragma unroll
    for (int i = 0; i < KS; ++i) o[g][i][0] = o[g][i][1] = o[g][i][2] = o[g][i][3] = 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      m[g][e] = kNoLogit;
      l[g][e] = 0.f;
      at_row[g][e] = len - nq + (m0 + 8 * g + 2 * t + e) / p.group;
    }
  }
  const float c = p.scale_log2;

  int stage = 0;
#pragma unroll 1
  for (int ch = c_begin + warp; ch < c_end; ch += kWarps) {
    cp_async_wait<kStages - 2>();
    __syncwarp();
    int first, end;
    chunk_at(ch, first, end);
    const unsigned char* at = smem + warp * Ring<D>::kWarp + stage * Ring<D>::kStage;
    // ---- logits: two tiles of 16 stored rows
    float s[NQ][2][4];
#pragma unroll
    for (int T = 0; T < 2; ++T) {
      float small[F32 ? NQ : 1][4];          // fp32: what the queries' second and third parts give
#pragma unroll
      for (int g = 0; g < NQ; ++g) {
        s[g][T][0] = s[g][T][1] = s[g][T][2] = s[g][T][3] = 0.f;
        if constexpr (F32) small[g][0] = small[g][1] = small[g][2] = small[g][3] = 0.f;
      }
      uint32_t w[2][KS / 2];
      Scale2 sc[2][D / 64];
#pragma unroll
      for (int i = 0; i < 2; ++i) {            // stored rows r and r + 8 of the tile
        const int row = 16 * T + 8 * i + r;
        if constexpr (D == 128) {
          const uint4 v = *reinterpret_cast<const uint4*>(at + row * 64 + t * 16);
          w[i][0] = v.x; w[i][1] = v.y; w[i][2] = v.z; w[i][3] = v.w;
          const uint32_t bytes = *reinterpret_cast<const uint16_t*>(at + 2 * CODES + row * 8 + t * 2);
          sc[i][0] = scale2(__byte_perm(bytes, 0, 0x4040));
          sc[i][1] = scale2(__byte_perm(bytes, 0, 0x4141));
        } else {
          const uint2 v = *reinterpret_cast<const uint2*>(at + row * 32 + t * 8);
          w[i][0] = v.x; w[i][1] = v.y;
          sc[i][0] = scale2(at[2 * CODES + row * 4 + t] * 0x10001u);
        }
      }
#pragma unroll
      for (int x = 0; x < KS / 2; ++x)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const Scale2 &s0 = sc[0][x / 2], &s1 = sc[1][x / 2];
          const uint32_t a0 = values2(w[0][x], 8 * u, s0), a1 = values2(w[1][x], 8 * u, s1);
          const uint32_t a2 = values2(w[0][x], 8 * u + 4, s0), a3 = values2(w[1][x], 8 * u + 4, s1);
#pragma unroll
          for (int g = 0; g < NQ; ++g) {
            if constexpr (F32) {
#pragma unroll
              for (int k = NP - 1; k >= 0; --k) {
                const uint2 q = q_smem[((k * NQ + g) * KS + 2 * x + u) * 32 + lane];
                mma(k ? small[g] : s[g][T], a0, a1, a2, a3, q.x, q.y);
              }
            } else {
              mma(s[g][T], a0, a1, a2, a3, qf[g][2 * x + u].x, qf[g][2 * x + u].y);
            }
          }
        }
      if constexpr (F32) {
#pragma unroll
        for (int g = 0; g < NQ; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[g][T][e] += small[g][e];
      }
    }
    // ---- softmax
    if (first + kChunk > end || !kv4_all_see(range, first)) {
#pragma unroll
      for (int g = 0; g < NQ; ++g)
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int row = first + 16 * T + 8 * (e >> 1) + r;
            if (row >= end || !kv4_sees(p, at_row[g][e & 1], row)) s[g][T][e] = -INFINITY;
          }
    }
    float top[NQ][2];
    bool raise = false;
#pragma unroll
    for (int g = 0; g < NQ; ++g)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        top[g][e] = fmaxf(fmaxf(s[g][0][e], s[g][0][2 + e]), fmaxf(s[g][1][e], s[g][1][2 + e]));
        raise |= (top[g][e] - m[g][e]) * c > kRaise;
      }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int g = 0; g < NQ; ++g)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mx = fmaxf(m[g][e], top[g][e]);
#pragma unroll
          for (int x = 4; x < 32; x *= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
          const float f = ex2((m[g][e] - mx) * c);
          m[g][e] = mx;
          l[g][e] *= f;
#pragma unroll
          for (int i = 0; i < KS; ++i) { o[g][i][e] *= f; o[g][i][2 + e] *= f; }
        }
    }
    // the probabilities as the second operand of the products with the values: 16 stored rows x 8 query rows
    uint32_t pf[NP][NQ][2][2];
#pragma unroll
    for (int g = 0; g < NQ; ++g) {
      // (a row that has seen nothing yet has a reference of -3.4e38, whose product may overflow)
      const float n0 = m[g][0] == kNoLogit ? 0.f : -m[g][0] * c, n1 = m[g][1] == kNoLogit ? 0.f : -m[g][1] * c;
#pragma unroll
      for (int T = 0; T < 2; ++T)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float x = ex2(fmaf(s[g][T][2 * i], c, n0)), y = ex2(fmaf(s[g][T][2 * i + 1], c, n1));
          if constexpr (F32) { l[g][0] += x; l[g][1] += y; }
#pragma unroll
          for (int k = 0; k < NP; ++k) {
            const uint32_t h = pack2(x, y);
            if constexpr (F32) { x -= low(h); y -= high(h); }
            else add_bf162(l[g][0], l[g][1], h);       // the sums are of what the products see
            pf[k][g][T][i] = transposed(h);
          }
        }
    }
    // ---- values
#pragma unroll
    for (int T = 0; T < 2; ++T) {
      const unsigned char* codes = at + CODES + r * (D / 16);
      const unsigned char* scales = at + 2 * CODES + SCALES + (r * (D / 8)) / kBlock;
      uint32_t w[4][D / 64], byte[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {          // stored rows 2t, 2t + 1, 2t + 8, 2t + 9
        const int row = 16 * T + 2 * t + (i & 1) + 8 * (i >> 1);
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
          for (int i = 0; i < 2; ++i) {      // elements 8 x + 4 half + 2 i and + 1 of the lane's
            const uint32_t a0 = values2(w0, 8 * i, s0), a1 = values2(w0, 8 * i + 4, s0), a2 = values2(w1, 8 * i, s1), a3 = values2(w1, 8 * i + 4, s1);
#pragma unroll
            for (int g = 0; g < NQ; ++g) {
              float* const to = o[g][4 * x + 2 * half + i];
              if constexpr (F32) {
                // matrix instructions cut off what a sum does not hold: a long chain of them drifts by half a step each, so that
                // fp32 adds their results to the outputs by itself
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = NP - 1; k >= 0; --k) mma(sum, a0, a1, a2, a3, pf[k][g][T][0], pf[k][g][T][1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) to[e] += sum[e];
              } else {
                mma(to, a0, a1, a2, a3, pf[0][g][T][0], pf[0][g][T][1]);
              }
            }
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
  for (int g = 0; g < NQ; ++g)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int x = 4; x < 32; x *= 2) l[g][e] += __shfl_xor_sync(0xffffffffu, l[g][e], x);
      if (r == 0) merge_m[warp][8 * g + 2 * t + e] = m[g][e];
    }
  __syncthreads();                           // (and every warp is done with its ring)
  float* const mine = reinterpret_cast<float*>(smem) + warp * ROWS * D;
#pragma unroll
  for (int g = 0; g < NQ; ++g)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = 8 * g + 2 * t + e;
      float mx = merge_m[0][row];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) mx = fmaxf(mx, merge_m[w][row]);
      const float f = ex2((m[g][e] - mx) * c);
      if (r == 0) merge_l[warp][row] = l[g][e] * f;
#pragma unroll
      for (int i = 0; i < KS; i += 2)
        *reinterpret_cast<float4*>(mine + row * D + r * (D / 8) + 2 * i) =
            make_float4(o[g][i][e] * f, o[g][i][2 + e] * f, o[g][i + 1][e] * f, o[g][i + 1][2 + e] * f);
    }
  __syncthreads();
  float* const cta_out = reinterpret_cast<float*>(smem) + kWarps * ROWS * D;   // clusters: the CTA's outputs, behind the warps'
#pragma unroll 1
  for (int x = threadIdx.x; x < ROWS * D / 4; x += kThreads) {
    const int row = x / (D / 4), d = (x - row * (D / 4)) * 4;
    if (m0 + row >= rows) break;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    float total = 0.f, mx = kNoLogit;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem) + (w * ROWS + row) * D + d);
      sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
      total += merge_l[w][row];
      mx = fmaxf(mx, merge_m[w][row]);
    }
    if (p.splits == 1) {
      kv4_store<F32>(p, b, kvh, m0 + row, d, sum, total);
    } else if (p.clustered) {
      *reinterpret_cast<float4*>(cta_out + row * D + d) = sum;
      if (d == 0) cta_stats[row] = make_float2(mx, total);
    } else {
      float* part = p.partial + ((long long)unit * p.splits + split) * (ROWS * (D + 2));
      *reinterpret_cast<float4*>(part + row * D + d) = sum;
      if (d == 0) {
        part[ROWS * D + 2 * row] = mx;
        part[ROWS * D + 2 * row + 1] = total;
      }
    }
  }
  if (!p.clustered) return;
  // ---- the cluster's shares: every CTA adds up a part of the outputs from all of them
  cluster_barrier();
  const int per = (ROWS * D / 4 + p.splits - 1) / p.splits;
#pragma unroll 1
  for (int i = threadIdx.x; i < per; i += kThreads) {
    const int x = split * per + i, row = x / (D / 4), d = (x - row * (D / 4)) * 4;
    if (row >= ROWS || m0 + row >= rows) break;
    const uint32_t out_at = smem_u32(cta_out + row * D + d), stats_at = smem_u32(&cta_stats[row]);
    float2 stats[kMaxCluster];
    float4 v[kMaxCluster];
    float mx = kNoLogit, total = 0.f;
#pragma unroll
    for (int s = 0; s < kMaxCluster; ++s) {
      if (s >= p.splits) break;
      stats[s] = load_shared2(at_rank(stats_at, s));
      v[s] = load_shared4(at_rank(out_at, s));
    }
#pragma unroll
    for (int s = 0; s < kMaxCluster; ++s)
      if (s < p.splits) mx = fmaxf(mx, stats[s].x);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int s = 0; s < kMaxCluster; ++s) {
      if (s >= p.splits) break;
      const float f = ex2((stats[s].x - mx) * c);
      total += f * stats[s].y;
      sum.x = fmaf(f, v[s].x, sum.x); sum.y = fmaf(f, v[s].y, sum.y); sum.z = fmaf(f, v[s].z, sum.z); sum.w = fmaf(f, v[s].w, sum.w);
    }
    kv4_store<F32>(p, b, kvh, m0 + row, d, sum, total);
  }
  cluster_barrier();                         // (the others may still read this CTA's)
}

// Partial results of the splits (at most 64) added up: a CTA for a query row, its groups of D / 4 threads share the splits.  (One
// group for all of them, one after the other, took 0.3 us a split.)
template <int D, bool F32>
__global__ void __launch_bounds__(kCombineThreads) kv4_combine_kernel(const __grid_constant__ Kv4AttendParams p) {
  constexpr int LANES = D / 4, GROUPS = kCombineThreads / LANES;
  __shared__ float weight[kMaxSplits];
  __shared__ float4 sums[GROUPS][LANES];
  pdl_wait();
  const int rows = p.n_queries * p.group, head = blockIdx.x / rows, m = blockIdx.x - head * rows;
  const int tile = m / p.tile_rows, row = m - tile * p.tile_rows, unit = head * p.tiles + tile;
  const int b = head / p.kv_heads, kvh = head - b * p.kv_heads;
  if (p.new_lens && m >= p.new_lens[b] * (long long)p.group) return;
  const long long step = (long long)p.tile_rows * (D + 2);
  const float* part = p.partial + (long long)unit * p.splits * step;
  const int lane = threadIdx.x & 31, group = threadIdx.x / LANES, d = (threadIdx.x % LANES) * 4;
  // the first outputs are on their way while the weights are formed
  constexpr int AHEAD = 4;
  float4 v[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (group + i * GROUPS < p.splits) v[i] = *reinterpret_cast<const float4*>(part + (group + i * GROUPS) * step + (long long)row * D + d);
  float total = 0.f;
  {
    // every warp for itself: reference maximum and sum of splits lane and lane + 32
    const float* stats = part + (long long)p.tile_rows * D + 2 * row;
    float2 x[2];
    float mx = kNoLogit;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int s = lane + 32 * i;
      x[i] = s < p.splits ? *reinterpret_cast<const float2*>(stats + s * step) : make_float2(kNoLogit, 0.f);
      mx = fmaxf(mx, x[i].x);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float f = ex2((x[i].x - mx) * p.scale_log2);
      total += f * x[i].y;
      if (threadIdx.x < 32) weight[lane + 32 * i] = f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  }
  __syncthreads();
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4& x, float f) {
    sum.x = fmaf(f, x.x, sum.x); sum.y = fmaf(f, x.y, sum.y); sum.z = fmaf(f, x.z, sum.z); sum.w = fmaf(f, x.w, sum.w);
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (group + i * GROUPS < p.splits) add(v[i], weight[group + i * GROUPS]);
  for (int s = group + AHEAD * GROUPS; s < p.splits; s += GROUPS)
    add(*reinterpret_cast<const float4*>(part + s * step + (long long)row * D + d), weight[s]);
  sums[group][threadIdx.x % LANES] = sum;
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int g = 1; g < GROUPS; ++g) add(sums[g][threadIdx.x], 1.f);
  kv4_store<F32>(p, b, kvh, m, d, sum, total);
}

template <int D, bool F32, int NQ>
int launch_few(const Kv4AttendParams& p, cudaStream_t st) {
  constexpr size_t smem = smem_bytes<D, F32, NQ>();
  if (!allow_dynamic_smem(kv4_attend_kernel<D, F32, NQ>, smem)) return -1;
  const int y = std::min(p.units, 32768);
  const dim3 grid(p.splits, y, (p.units + y - 1) / y);
  if (!p.clustered) {
    launch_k(kv4_attend_kernel<D, F32, NQ>, grid, dim3(kThreads), smem, st, p);
    return 1;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cudaLaunchKernelEx(&cfg, kv4_attend_kernel<D, F32, NQ>, p);
  return 1;
}

template <int D, bool F32>
int launch_attend(const Kv4AttendParams& p, cudaStream_t st) {
  const int r = p.tile_rows == 8 ? launch_few<D, F32, 1>(p, st) : p.tile_rows == 16 ? launch_few<D, F32, 2>(p, st) : launch_kv4_attend_tc(p, D, st);
  if (r < 0) return -1;
  if (p.splits > 1 && !p.clustered) {
    launch_k(kv4_combine_kernel<D, F32>, dim3((unsigned)(p.units / p.tiles) * p.n_queries * p.group), dim3(kCombineThreads), 0, st, p);
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
  if (a->form < 0 || a->form > HACK_KV4_MANY) return invalid("unknown form");
  if (a->form == HACK_KV4_MANY && a->dtype != HACK_BF16) { set_error("HACK_KV4_MANY serves bf16"); return HACK_ERR_UNSUPPORTED; }
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
  // (positions are above -2^30: a window or a number of first rows that reaches past all of them must not wrap)
  p.window = std::min(a->window, 1 << 30);
  p.n_sink = a->window > 0 ? std::min(a->n_sink, 1 << 30) : 0;
  p.appended = a->appended != 0;
  const int heads = kv->batch * kv->n_kv_heads, rows = a->n_queries * p.group;
  // rows that a unit's queries, 256 rows of them at most, walk at most (us with those of all queries counted, and of a unit's:
  // 8 query heads of 1 024 tokens on 2 stored ones x 128, a window of 256, 31.6 and 19.4; 2 heads, a window of 1 024, 19.4 and 14.7)
  long long walked = p.max_len;
  if (p.window > 0)
    walked = std::min<long long>(walked, (long long)p.window + p.n_sink + (p.causal ? std::min(p.n_queries, 256 / p.group + 2) : p.n_queries));
  // Which kernel: estimated us of a launch in one wave or more, fitted to both forms (us, few-rows form and tensor cores: 16 heads of
  // 10 521 rows x 128, 32 queries 22.1 and 25.8, 48 26.8 and 26.6, 64 35.3 and 27.3; 64 heads of 2 240 rows, 48 queries 31.9 and 34.4,
  // 64 38.9 and 35.9; 4 heads of 700 rows x 64, 64 queries 6.3 and 12.9; 128 heads of 680 rows 14.9 and 14.1).
  const bool wide = kv->head_dim == 128;
  // (16 heads, 1 024 queries: 64 and 128 rows 20.5 and 9.8 us: what a CTA costs at least)
  const double few_tiles = (double)heads * ((rows + 15) / 16);
  const double few_us = std::max(5.0 + (wide ? 1.45e-3 : 0.9e-3) * few_tiles * ((walked + 31) / 32),
                                 8.0 * few_tiles / (sm_count() * ctas_per_sm(false, 2)));
  const double tc_us = (wide ? 13.0 : 12.0) + (wide ? 10.7e-3 : 6.6e-3) * heads * ((rows + 127) / 128) * ((walked + 127) / 128);
  const bool tc = a->form == 0 ? a->dtype == HACK_BF16 && rows > 16 && tc_us < few_us : a->form == HACK_KV4_MANY;
  p.tile_rows = tc ? 128 : rows <= 8 ? 8 : 16;
  p.tiles = (rows + p.tile_rows - 1) / p.tile_rows;
  const long long units = (long long)heads * p.tiles;
  if (units * p.tile_rows > 0x3fffffffll) { set_error("more query rows than a launch has places for"); return HACK_ERR_UNSUPPORTED; }
  p.units = (int)units;
  const int sms = sm_count();
  if (tc) {
    p.tiles_per_cta = units <= sms ? 1 : 2;
    const long long ctas = (long long)heads * ((p.tiles + p.tiles_per_cta - 1) / p.tiles_per_cta);
    p.splits = (int)std::max<long long>(1, std::min<long long>({(walked + 127) / 128 / 4, sms / ctas, kMaxSplits}));
  } else {
    // CTAs that share a unit's rows, in a cluster or with a second launch: the least of estimated us, fitted to both.  A turn
    // (a chunk a warp) takes the longer the more CTAs an SM has, what follows the turns 2 or 2.7 us and more.  (us in a cluster and
    // with a second launch: 128 heads of 2 240 rows x 64, two CTAs 9.8 and 10.9, four 9.9 and 10.7; 32 heads of 4 096 rows x 128,
    // eight CTAs 9.5 and 10.0.  Clusters of other sizes may, and more than fit at once do find their places late: 128 heads, three
    // and five CTAs 11.3 and 13.3; 32 heads, sixteen 13.4 where a second launch takes 10.3.)
    const long long turns = std::max<long long>(1, (walked + kChunk * kWarps - 1) / (kChunk * kWarps));
    const int per_sm = ctas_per_sm(a->dtype == HACK_F32, p.tile_rows / 8);
    const double turn_us = (wide ? 1.0 : 0.6) * (a->dtype == HACK_F32 ? 0.8 * (p.tile_rows / 8) + 0.7 : p.tile_rows == 16 ? 1.4 : 1.0);
    double best = 0;
    p.splits = 1;
    for (int n = 1; n <= kMaxSplits && n <= turns; ++n) {
      const long long ctas = units * n, places = (long long)sms * per_sm;
      const int on_sm = (int)std::min<long long>(per_sm, (ctas + sms - 1) / sms);
      const double waves = n == 1 ? std::max(1.0, (double)ctas / places) : (double)((ctas + places - 1) / places);
      const double work = waves * ((double)((turns + n - 1) / n) * turn_us * (0.55 + 0.38 * on_sm) + 2.2);
      const bool cluster = n > 1 && n <= kMaxCluster && ctas <= places;
      const double cost = work + (n == 1 ? 0.0 : cluster ? 2.0 + ((n & (n - 1)) ? 1.0 : 0.0) : 2.7 + 0.03 * n);
      if (n == 1 || cost < best) {
        best = cost;
        p.splits = n;
        p.clustered = cluster;
      }
    }
  }
  // (a role may wait for a whole unit of work: some sixty polls a block)
  p.wait_polls = a->wait_polls > 0 ? (uint32_t)a->wait_polls : kWaitPolls + (uint32_t)std::min<long long>(walked, 1 << 30);
  workspace = p.splits > 1 && !p.clustered ? (size_t)p.units * p.splits * p.tile_rows * (kv->head_dim + 2) * 4 : 0;
  return HACK_OK;
}

}  // namespace
}  // namespace hack

extern "C" hack_status_t hack_kv4_workspace(const hack_kv4_t* kv, const hack_kv4_attend_t* args, size_t* bytes) {
  using namespace hack;
  const hack_status_t s = check_attend(kv, args);
  if (s != HACK_OK) return s;
  if (!bytes) return invalid("bytes is NULL");
  *bytes = 0;
  if (args->n_queries == 0) return HACK_OK;      // (there is nothing to plan a launch for)
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
  if (!lens || off_its_size(lens, 4) || off_its_size(new_lens, 4)) return invalid("lens is NULL, or lens or new_lens not on a multiple of 4 bytes");
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
