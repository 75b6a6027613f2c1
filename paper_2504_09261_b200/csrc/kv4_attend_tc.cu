// Attention over a cache of 4 bits on the 5th-generation tensor cores: bf16 queries, many of them to a stored head.
//
// A CTA takes one or two tiles of 128 query rows (token * group + head of the group) of a stored head and walks over the
// blocks of 128 stored rows that they see.  What is multiplied is the stored values themselves, exact in bf16:
//   warps 0, 2   : issue the products Q K^T and P V (a thread each)
//   warps 4-11   : softmax of the two tiles, one thread per query row; they also put the queries into shared memory
//   warps 12-15  : read codes and scales, a tile of K or V ahead in registers, and write the values as the operand tiles
// A word of eight codes becomes the elements 0 4 1 5 2 6 3 7 of its eight (a shift, a mask and an FMA for two): the order of
// the elements inside Q K^T is free as long as both sides have it, so the queries are written in it as well, and
// the columns of P V are put right when the output is written.
// Tensor memory (512 columns): logits [0,128), one buffer which the tiles take in turn; probabilities [128,192) and [192,256);
// outputs from 256 on.  A softmax thread reads its logit row into registers and gives the buffer back at once, so that the
// next Q K^T runs under it; the output is rescaled only when a row's maximum grows by more than 2^32.
// Every wait is bounded; a CTA that gives up lets its products end, frees its tensor memory and raises the status word.
#include <algorithm>

#include "entry_checks.h"
#include "kv4_attend.h"
#include "tc_ptx.cuh"

namespace hack {

__device__ int g_kv4_status = 0;

namespace {

using namespace kv4;
using namespace ptx;

constexpr int kBM = 128, kBN = 128;
constexpr int kQkWarp = 0, kPvWarp = 2, kSoftmaxWarps = 4, kValueWarps = 12;    // first of each role
constexpr int kThreads = 512;
// 256 * 200 + 128 * 72 + 128 * 40 registers = 512 * 128
constexpr int kSoftmaxRegs = 200, kValueRegs = 72, kIssueRegs = 40;
constexpr int kStages = 2;
constexpr float kRaise = 32.f;               // log2 by which a logit may exceed the reference maximum
constexpr uint32_t kDrainPolls = 1u << 22;

struct Bars {
  uint64_t q_full[2];
  uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
  uint64_t s_full[2], s_free, p_full[2], p_free[2];
  uint64_t drain[2];
  uint32_t tmem_base;
  int gave_up;
};

__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity, Bars* b, uint32_t polls) {
  const uint32_t addr = smem_u32(bar);
  if (__builtin_expect(mbar_try_wait(addr, parity), 1)) return true;
  volatile int* const flag = &b->gave_up;
#pragma unroll 1
  for (; !mbar_try_wait(addr, parity); --polls) {
    if (*flag) return false;
    if (polls == 0) { *flag = 1; return false; }
  }
  return true;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) kv4_attend_tc_kernel(const __grid_constant__ Kv4AttendParams p) {
  constexpr uint32_t SUB_BYTES = kBN * 128, TILE_BYTES = D / 64 * SUB_BYTES;      // tiles of 64 columns: 128 rows x 128 bytes
  constexpr uint32_t S_COL = 0, P_COL = 128, O_COL = 256;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t raw = smem_u32(smem_dyn), base = (raw + 1023u) & ~1023u;         // the swizzle needs 1024-byte alignment
  const uint32_t q_sm = base, k_sm = q_sm + 2 * TILE_BYTES, v_sm = k_sm + kStages * TILE_BYTES;
  unsigned char* const sm = smem_dyn + (base - raw);
  Bars* const bars = reinterpret_cast<Bars*>(sm + (2 + 2 * kStages) * TILE_BYTES);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t polls = p.wait_polls;

  pdl_grid_wait();
  // Heads inside units of the same place: the last tiles, of a causal call the longest, come first
  const int split = blockIdx.x % p.splits, at = blockIdx.x / p.splits;
  const int heads = p.units / p.tiles, per = p.tiles_per_cta, cta_units = (p.tiles + per - 1) / per;
  const int head = at % heads, cta_unit = cta_units - 1 - at / heads;
  const int b = head / p.kv_heads, kvh = head - b * p.kv_heads;
  const int nq = p.new_lens ? min(max(p.new_lens[b], 0), p.n_queries) : p.n_queries;
  const int rows = nq * p.group, m0 = cta_unit * per * kBM;
  if (m0 >= rows) return;                    // (the queries of a padded batch that it does not have)
  const int ntile = per == 2 && m0 + kBM < rows ? 2 : 1;
  const int len = kv4_length(p, head, nq);
  const Kv4Range range = kv4_range(p, len, nq, m0, min(m0 + per * kBM, rows) - 1);
  const int blocks1 = (range.sink_end + kBN - 1) / kBN, blocks = blocks1 + (range.hi - range.lo + kBN - 1) / kBN;
  const int j_begin = (int)((long long)blocks * split / p.splits), j_end = (int)((long long)blocks * (split + 1) / p.splits);
  const int nblk = j_end - j_begin;
  auto block_at = [&](int j, int& first, int& end) {
    first = j < blocks1 ? j * kBN : range.lo + (j - blocks1) * kBN;
    end = j < blocks1 ? range.sink_end : range.hi;
  };

  if (tid == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&bars->q_full[t]), 4);          // an arrival of each warp of the tile
      mbar_init(smem_u32(&bars->s_full[t]), 1);
      mbar_init(smem_u32(&bars->p_full[t]), 4);
      mbar_init(smem_u32(&bars->p_free[t]), 1);
      mbar_init(smem_u32(&bars->drain[t]), 1);
    }
    mbar_init(smem_u32(&bars->s_free), 4);
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&bars->k_full[s]), 4);
      mbar_init(smem_u32(&bars->k_empty[s]), 1);
      mbar_init(smem_u32(&bars->v_full[s]), 4);
      mbar_init(smem_u32(&bars->v_empty[s]), 1);
    }
    bars->gave_up = 0;
    fence_barrier_init();
    fence_proxy_async();
  }
  if (warp == kQkWarp) {
    __syncwarp();
    tmem_alloc(smem_u32(&bars->tmem_base), 512);
    tmem_relinquish();
    // the next launch may start once every CTA of this one holds its tensor memory
    pdl_launch_dependents();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&bars->tmem_base);

  if (warp >= kValueWarps) {
    // ------------------------------------------------------------------ codes to values
    reg_dec<kValueRegs>();
    constexpr int LPR = D / 32, RPW = 32 / LPR, PASSES = kBN / (4 * RPW);   // lanes of a row (16 bytes of codes each), rows of a warp
    const int t = lane % LPR, row_in = (warp - kValueWarps) * RPW + lane / LPR;
    const long long row0 = first_row(p.planes, head);
    uint4 codes[2][PASSES];
    uint32_t scales[2][PASSES];
    auto load = [&](int item, int set) {       // item 2 j: keys of block j, 2 j + 1: its values
      int first, end;
      block_at(j_begin + (item >> 1), first, end);
      const unsigned char* c = item & 1 ? p.planes.v_codes : p.planes.k_codes;
      const unsigned char* s = item & 1 ? p.planes.v_scales : p.planes.k_scales;
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        // (a row past the end: any finite values, its logits do not count)
        const long long row = row0 + min(first + i * 4 * RPW + row_in, end - 1);
        codes[set][i] = *reinterpret_cast<const uint4*>(c + row * (D / 2) + t * 16);
        scales[set][i] = *reinterpret_cast<const uint16_t*>(s + row * (D / 16) + t * 2);
      }
    };
    auto write = [&](int item, int set) {
      const int j = item >> 1, slot = j % kStages;
      const uint32_t tile = (item & 1 ? v_sm : k_sm) + slot * TILE_BYTES;
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        const int row = i * 4 * RPW + row_in;
        const uint4 u = codes[set][i];
        // eight lanes write eight different 16-byte columns: those of the second 64 elements take their words in another order
        const bool other = D == 128 && (t & 2);
        const uint32_t w[4] = {other ? u.z : u.x, other ? u.w : u.y, other ? u.x : u.z, other ? u.y : u.w};
        const uint32_t lo = scales[set][i] & 0xff, hi = scales[set][i] >> 8;
        const Scale2 s0 = scale2((other ? hi : lo) * 0x10001u), s1 = scale2((other ? lo : hi) * 0x10001u);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const Scale2& s = k < 2 ? s0 : s1;
          const int chunk = 4 * t + (other ? k ^ 2 : k);
          const uint32_t dst = tile + (chunk >> 3) * SUB_BYTES + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
          const uint32_t x = values2(w[k], 0, s), y = values2(w[k], 4, s), z = values2(w[k], 8, s), q = values2(w[k], 12, s);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(x), "r"(y), "r"(z), "r"(q) : "memory");
        }
      }
    };
    auto turn = [&](int item, int set) {
      if (item + 1 < 2 * nblk) load(item + 1, set ^ 1);
      const int j = item >> 1, slot = j % kStages;
      if (j >= kStages &&
          !__all_sync(0xffffffffu, wait_bar(item & 1 ? &bars->v_empty[slot] : &bars->k_empty[slot], (j / kStages - 1) & 1, bars, polls)))
        return false;
      write(item, set);
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(item & 1 ? &bars->v_full[slot] : &bars->k_full[slot]));
      return true;
    };
    if (nblk > 0) load(0, 0);
#pragma unroll 1
    for (int j = 0; j < nblk; ++j)
      if (!turn(2 * j, 0) || !turn(2 * j + 1, 1)) break;
  } else if (warp >= kSoftmaxWarps) {
    // ------------------------------------------------------------------ queries, softmax, output
    reg_inc<kSoftmaxRegs>();
    const int t = (warp - kSoftmaxWarps) >> 2, row = tid & 127;
    if (t < ntile) {
      const int m = m0 + t * kBM + row, token = m / p.group;
      const bool live = m < rows;
      const long long q_at = b * p.q_stride.batch + (long long)(kvh * p.group + m - token * p.group) * p.q_stride.head +
                             (long long)token * p.q_stride.token;
#pragma unroll 4
      for (int chunk = 0; chunk < D / 8; ++chunk) {
        const uint4 v = live ? reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + q_at)[chunk] : make_uint4(0, 0, 0, 0);
        const uint32_t dst = q_sm + t * TILE_BYTES + (chunk >> 3) * SUB_BYTES + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(__byte_perm(v.x, v.z, 0x5410)), "r"(__byte_perm(v.x, v.z, 0x7632)),
                     "r"(__byte_perm(v.y, v.w, 0x5410)), "r"(__byte_perm(v.y, v.w, 0x7632)) : "memory");
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars->q_full[t]));

      const uint32_t lane_addr = static_cast<uint32_t>((warp & 3) * 32) << 16;
      const uint32_t s_addr = tmem + lane_addr + S_COL, p_addr = tmem + lane_addr + P_COL + t * 64, o_addr = tmem + lane_addr + O_COL + t * D;
      const float c = p.scale_log2;
      float m_used = kNoLogit, l = 0.f;
      bool ok = true;
      auto bar_all = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bar(bar, parity, bars, polls)) != 0; };
      const int pos = len - nq + token;
      const int see_hi = p.causal ? min(len, pos + 1) : len, see_lo = p.window > 0 ? pos - p.window + 1 : 0;
#pragma unroll 1
      for (int j = 0; j < nblk; ++j) {
        int first, end;
        block_at(j_begin + j, first, end);
        ok = bar_all(&bars->s_full[t], j & 1);
        if (!ok) break;
        tc_fence_after();
        uint32_t sr[kBN];
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) tmem_ld32(s_addr + ch * 32, sr + ch * 32);
        tmem_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->s_free));       // the logits are in registers
        if (__builtin_expect(first + kBN > min(end, range.all_hi) || !(first >= range.all_lo || first + kBN <= range.all_sink), 0)) {
          const int hi = min(end, see_hi) - first, lo = see_lo - first, sink = (p.window > 0 ? p.n_sink : 0) - first;
#pragma unroll
          for (int i = 0; i < kBN; ++i)
            if (i >= hi || (i < lo && i >= sink)) sr[i] = 0xff800000u;   // -inf
        }
        float mx4[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          mx4[u] = -INFINITY;
#pragma unroll
          for (int i = 0; i < 16; ++i) mx4[u] = max3(mx4[u], __uint_as_float(sr[u * 32 + 2 * i]), __uint_as_float(sr[u * 32 + 2 * i + 1]));
        }
        const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
        const bool grow = (mx - m_used) * c > kRaise;              // in the first block that the row sees anything of
        const bool any = __any_sync(0xffffffffu, grow);
        float alpha = 1.f;
        if (any) {
          const float m_new = grow ? mx : m_used;
          alpha = grow ? ex2((m_used - m_new) * c) : 1.f;
          l *= alpha;
          m_used = m_new;
        }
        const float nmc = m_used == kNoLogit ? 0.f : -m_used * c;  // (nothing seen: the product may overflow)
        const float2 c2 = make_float2(c, c), nmc2 = make_float2(nmc, nmc);
        // the sums are of the probabilities as the products see them
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        uint32_t pk[kBN / 2];
#pragma unroll
        for (int i = 0; i < kBN / 2; ++i) {
          const float2 x = fma2(make_float2(__uint_as_float(sr[2 * i]), __uint_as_float(sr[2 * i + 1])), c2, nmc2);
          float2 pr;
          pr.x = ex2(x.x);
          pr.y = ex2(x.y);
          const __nv_bfloat162 hh = __floats2bfloat162_rn(pr.x, pr.y);
          pk[i] = *reinterpret_cast<const uint32_t*>(&hh);
          add_bf162(sum[2 * (i & 1)], sum[2 * (i & 1) + 1], pk[i]);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        if (j > 0) {
          // the product of the block before still reads P_t and adds to O_t
          ok = bar_all(&bars->p_free[t], (j - 1) & 1);
          if (!ok) break;
          tc_fence_after();
          if (any) {
#pragma unroll 1
            for (int ch = 0; ch < D / 8; ++ch) {
              uint32_t orr[8];
              tmem_ld8(o_addr + ch * 8, orr);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 8; ++i) orr[i] = __float_as_uint(__uint_as_float(orr[i]) * alpha);
              tmem_st8(o_addr + ch * 8, orr);
            }
          }
        }
        tmem_st32(p_addr, pk);
        tmem_st32(p_addr + 32, pk + 32);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->p_full[t]));
      }
      if (ok && nblk > 0) {
        ok = bar_all(&bars->p_free[t], (nblk - 1) & 1);
        tc_fence_after();
      }
      if (ok) {
        const int g = m - token * p.group;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        unsigned char* dst = nullptr;
        float* part = nullptr;
        if (p.splits > 1) {
          const long long unit = (long long)head * p.tiles + cta_unit * per + t;
          float* const at_split = p.partial + (unit * p.splits + split) * (kBM * (D + 2));
          part = at_split + row * D;
          if (live) *reinterpret_cast<float2*>(at_split + kBM * D + 2 * row) = make_float2(m_used, l);
        } else {
          dst = reinterpret_cast<unsigned char*>(static_cast<__nv_bfloat16*>(p.out) + b * p.out_stride.batch +
                                                 (long long)(kvh * p.group + g) * p.out_stride.head + (long long)token * p.out_stride.token);
        }
#pragma unroll 1
        for (int ch = 0; ch < D / 16; ++ch) {
          uint32_t o[16];
          if (nblk > 0) {
            tmem_ld16(o_addr + ch * 16, o);
            tmem_wait_ld();
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = 0;
          }
          // columns 0 4 1 5 2 6 3 7 of every eight
          float x[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(o[(i & 8) + 2 * (i & 3) + ((i >> 2) & 1)]);
          if (!live) continue;
          if (part) {
#pragma unroll
            for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(part + ch * 16)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
          } else {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const __nv_bfloat162 hh = __floats2bfloat162_rn(x[2 * i] * inv, x[2 * i + 1] * inv);
              w[i] = *reinterpret_cast<const uint32_t*>(&hh);
            }
            st_global_32b(dst + ch * 32, w, p.out_sectors != 0);
          }
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ issuers of the products
    reg_dec<kIssueRegs>();
    // An issuer leaves when its last product has ended, or after a while
    auto drained = [&](uint64_t* bar) {
      mma_commit(smem_u32(bar));
#pragma unroll 1
      for (uint32_t it = 0; it < kDrainPolls && !mbar_try_wait(smem_u32(bar), 0); ++it) {}
    };
    if (warp == kQkWarp && lane == 0) {
      constexpr uint32_t IDESC = idesc_bf16_f32(kBM, kBN, 0);
      const uint64_t q_desc = smem_desc_sw128(q_sm, 16, 1024), k_desc = smem_desc_sw128(k_sm, 16, 1024);
      bool ok = true;
      uint32_t use = 0;                                  // products issued
#pragma unroll 1
      for (int j = 0; j < nblk && ok; ++j) {
        const uint32_t slot = j % kStages;
        const uint64_t kd = k_desc + (uint64_t)((slot * TILE_BYTES) >> 4);
#pragma unroll 1
        for (int t = 0; t < ntile; ++t) {
          if (j == 0) ok = wait_bar(&bars->q_full[t], 0, bars, polls);
          if (ok && t == 0) ok = wait_bar(&bars->k_full[slot], (j / kStages) & 1, bars, polls);
          if (!ok || !wait_bar(&bars->s_free, (use - 1) & 1, bars, polls)) { ok = false; break; }   // (a fresh barrier passes for odd)
          tc_fence_after();
          const uint64_t qd = q_desc + (uint64_t)((t * TILE_BYTES) >> 4);
          if constexpr (D == 128) mma_ss_chain8(tmem + S_COL, qd, kd, IDESC, 0);
          else mma_ss_chain4(tmem + S_COL, qd, kd, IDESC, 0);
          mma_commit(smem_u32(&bars->s_full[t]));
          ++use;
        }
        if (ok) mma_commit(smem_u32(&bars->k_empty[slot]));
      }
      drained(&bars->drain[0]);
    } else if (warp == kPvWarp && lane == 0) {
      constexpr uint32_t IDESC = idesc_bf16_f32(kBM, D, 1);          // V: rows of the tile are the summed index
      const uint64_t v_desc = smem_desc_sw128(v_sm, SUB_BYTES, 1024);
      bool ok = true;
#pragma unroll 1
      for (int j = 0; j < nblk && ok; ++j) {
        const uint32_t slot = j % kStages;
        const uint64_t vd = v_desc + (uint64_t)((slot * TILE_BYTES) >> 4);
#pragma unroll 1
        for (int t = 0; t < ntile; ++t) {
          if (t == 0) ok = wait_bar(&bars->v_full[slot], (j / kStages) & 1, bars, polls);
          if (!ok || !wait_bar(&bars->p_full[t], j & 1, bars, polls)) { ok = false; break; }
          tc_fence_after();
          const uint32_t o = tmem + O_COL + t * D, pa = tmem + P_COL + t * 64;
          mma_ts_chain4(o, pa, vd, IDESC, j > 0);
          mma_ts_chain4(o, pa + 32, vd + 4 * 128, IDESC, 1);
          mma_commit(smem_u32(&bars->p_free[t]));
        }
        if (ok) mma_commit(smem_u32(&bars->v_empty[slot]));
      }
      drained(&bars->drain[1]);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kQkWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (tid == 0 && bars->gave_up) atomicExch(&g_kv4_status, 1);
}

template <int D> constexpr size_t smem_bytes() { return 1024 + (2 + 2 * kStages) * (size_t)(D / 64) * kBN * 128 + sizeof(Bars) + 64; }

template <int D>
int launch(const Kv4AttendParams& p, cudaStream_t st) {
  // (more than half of an SM's shared memory at head_dim 64 as well: a CTA owns the SM's tensor memory)
  constexpr size_t smem = smem_bytes<128>();
  static_assert(smem_bytes<D>() <= smem, "");
  if (!allow_dynamic_smem(kv4_attend_tc_kernel<D>, smem)) return -1;
  const int heads = p.units / p.tiles, cta_units = (p.tiles + p.tiles_per_cta - 1) / p.tiles_per_cta;
  launch_k(kv4_attend_tc_kernel<D>, dim3((unsigned)((long long)heads * cta_units * p.splits)), dim3(kThreads), smem, st, p);
  return launched(1);
}

}  // namespace

int launch_kv4_attend_tc(const Kv4AttendParams& p, int head_dim, cudaStream_t st) {
  return head_dim == 64 ? launch<64>(p, st) : launch<128>(p, st);
}

}  // namespace hack

extern "C" hack_status_t hack_kv4_poll_status(int32_t device, void* stream) {
  using namespace hack;
  DeviceScope scope(device);
  cudaError_t e = scope.err;
  int status = 0;
  const int zero = 0;
  if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&status, g_kv4_status, sizeof(int));
  if (e == cudaSuccess && status) e = cudaMemcpyToSymbol(g_kv4_status, &zero, sizeof(int));
  if (e != cudaSuccess) {
    set_error(std::string("hack_kv4_poll_status: ") + cudaGetErrorString(e));
    return HACK_ERR_CUDA;
  }
  if (status) {
    set_error("hack_kv4_attend: a bounded device-side wait expired");
    return HACK_ERR_TIMEOUT;
  }
  return HACK_OK;
}
