// Attention over a cache of 4 bits on the 5th-generation tensor cores: bf16 queries, many of them to a stored head.
//
// A unit of work is one or two tiles of 128 query rows (token * group + head of the group) of a stored head, and the blocks of
// 128 stored rows that they see (or a share of them: `splits`).  What is multiplied is the stored values themselves, exact
// in bf16:
//   warps 0, 2   : issue the products Q K^T and P V (a thread each)
//   warp  1      : finds the CTA's next unit
//   warps 4-11   : softmax of the two tiles, one thread per query row, and their output
//   warps 12-15  : queries into shared memory; codes and scales, a tile of K or V ahead in registers, into operand tiles of values
// A word of eight codes becomes the elements 0 4 1 5 2 6 3 7 of its eight (a shift, a mask and an FMA for two): the order of
// the elements inside Q K^T is free as long as both sides have it, so the queries are written in it as well, and
// the columns of P V are put right when the output is written.
// Tensor memory (512 columns): logits [0,128), one buffer which the tiles take in turn; probabilities [128,192) and [192,256);
// outputs from 256 on.  A softmax thread reads its logit row into registers and gives the buffer back at once, so that the
// next Q K^T runs under it; the output is rescaled only when a row's maximum grows by more than 2^32.
// A CTA that is through with a unit takes over one that has not been launched yet (cluster launch control): its queries and
// first tiles are on their way under the last softmax and the output of the unit before.
// A probability is rounded to bf16 once, for the product with the values and the row's sum alike: the product takes bf16, and a
// second one for the rest would be half as much work again for the tensor pipe, one of the three resources that bound it.
// Every wait is bounded; a CTA that gives up lets its products end, frees its tensor memory and raises the status word.
#include <algorithm>
#include <type_traits>

#include "entry_checks.h"
#include "kv4_attend.h"
#include "tc_ptx.cuh"

namespace hack {

__device__ int g_kv4_status = 0;

namespace {

using namespace kv4;
using namespace ptx;

constexpr int kBM = 128, kBN = 128;
constexpr int kQkWarp = 0, kUnitWarp = 1, kPvWarp = 2, kSoftmaxWarps = 4, kValueWarps = 12;    // first of each role
constexpr int kThreads = 512;
// 256 * 184 + 128 * 96 + 128 * 48 registers = 512 * 128
constexpr int kSoftmaxRegs = 184, kValueRegs = 96, kIssueRegs = 48;
constexpr int kStages = 2;
constexpr float kRaise = 32.f;               // log2 by which a logit may exceed the reference maximum
constexpr uint32_t kDrainPolls = 1u << 22;
constexpr int kShortUnit = 16;               // blocks below which the next unit is asked for at the start of one

// A unit of work, in shared memory.  (Worked out by one thread for all roles: the same code in each of them was 10 % of the largest
// launch's time, in waits for instructions.)
struct Unit {
  long long row0;                            // first row of the stored head
  int more;                                  // 0: there is no unit any more
  int b, kvh, head;                          // the stored head
  int len, nq, rows, m0, ntile;              // its length, tokens and query rows; first row and tiles of the unit (0: nothing to do)
  int tile, split;                           // number of its first tile in the head; share of the blocks
  int j_begin, nblk;                         // its blocks
  // The rows that its queries may see, [0, seam) and [seam + skip, seam + skip + ...), as one list of `total`: place v of it is row v, or
  // v + skip from the seam on.  Blocks are 128 places.
  int seam, skip, total;
  int all_lo, all_hi, all_sink;              // Kv4Range
};

struct Bars {
  uint4 answer;                              // of cluster launch control
  Unit unit[2];                              // units of even and odd count
  uint64_t u_full[2], u_empty[2], asked;
  uint64_t q_full[2], q_free[2];
  uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
  uint64_t s_full[2], s_free, p_full[2], p_free[2];
  uint64_t drain[2];
  uint32_t tmem_base;
  int gave_up;
};

// Unit number x of the launch; x < 0: there is no more.
__device__ __forceinline__ void make_unit(const Kv4AttendParams& p, int x, volatile Unit& u) {
  u.more = x >= 0;
  u.ntile = u.nblk = 0;
  if (x < 0) return;
  const int heads = p.units / p.tiles, per = p.tiles_per_cta, cta_units = (p.tiles + per - 1) / per;
  const int split = x % p.splits;
  x /= p.splits;
  const int head = x % heads, tile = (cta_units - 1 - x / heads) * per;   // the last tiles, of a causal call the longest, come first
  const int b = head / p.kv_heads;
  const int nq = p.new_lens ? min(max(p.new_lens[b], 0), p.n_queries) : p.n_queries;
  const int rows = nq * p.group, m0 = tile * kBM;
  if (m0 >= rows) return;                    // queries of a padded batch that it does not have
  const int len = kv4_length(p, head, nq);
  const Kv4Range r = kv4_range(p, len, nq, m0, min(m0 + per * kBM, rows) - 1);
  const int total = r.sink_end + r.hi - r.lo;
  const uint32_t blocks = (total + kBN - 1) / kBN, begin = blocks * split / p.splits;
  u.row0 = first_row(p.planes, head);
  u.b = b;
  u.kvh = head - b * p.kv_heads;
  u.head = head;
  u.len = len;
  u.nq = nq;
  u.rows = rows;
  u.m0 = m0;
  u.ntile = per == 2 && m0 + kBM < rows ? 2 : 1;
  u.tile = tile;
  u.split = split;
  u.j_begin = begin;
  u.nblk = blocks * (split + 1) / p.splits - begin;
  u.seam = r.sink_end;
  u.skip = r.lo - r.sink_end;
  u.total = total;
  u.all_lo = r.all_lo;
  u.all_hi = r.all_hi;
  u.all_sink = r.all_sink;
}
// Bits below n
__device__ __forceinline__ uint32_t bits_below(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

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

// Logits of places that a query does not see become -inf where they are.  It sees those below `head` (of the first run), and from the
// seam on those below hi that are not below lo or are below sink.  32 at a time, as bits.  (On all 128 in registers, with three
// comparisons for each, it took 4 us a block.)
__device__ __forceinline__ void hide(uint32_t s_addr, int head, int seam, int hi, int lo, int sink) {
#pragma unroll 1
  for (int ch = 0; ch < kBN / 32; ++ch) {
    const int at = 32 * ch;
    const uint32_t keep = bits_below(head - at) | (bits_below(hi - at) & ~bits_below(seam - at) & (~bits_below(lo - at) | bits_below(sink - at)));
    if (__all_sync(0xffffffffu, keep == ~0u)) continue;
    uint32_t z[32];
    tmem_ld32(s_addr + ch * 32, z);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 32; ++i) z[i] = keep & (1u << i) ? z[i] : 0xff800000u;
    tmem_st32(s_addr + ch * 32, z);
  }
  tmem_wait_st();
}

// A tile of queries into shared memory by 128 threads, AHEAD loads of each in flight; elements in the order 0 4 1 5 2 6 3 7 of every
// eight.  (A row a thread, 16 bytes of 32 rows an instruction, took 4 us.)
template <int D, int AHEAD>
__device__ __forceinline__ void load_queries(const Kv4AttendParams& p, const volatile Unit& u, int tile, int thread, uint32_t q_sm) {
  constexpr int LPR = D / 8, RPT = 128 / LPR;            // threads of a row, rows of a turn
  const int chunk = thread % LPR, rows = u.rows;
  int m = u.m0 + tile * kBM + thread / LPR, token = m / p.group, g = m - token * p.group;
  const int dt = RPT / p.group, dg = RPT - dt * p.group;
  const __nv_bfloat16* const q = static_cast<const __nv_bfloat16*>(p.q) + u.b * p.q_stride.batch + (long long)(u.kvh * p.group) * p.q_stride.head + chunk * 8;
  const uint32_t to = q_sm + (chunk >> 3) * (kBN * 128);
#pragma unroll 1
  for (int first = thread / LPR; first < kBM; first += AHEAD * RPT) {
    uint4 v[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      v[i] = make_uint4(0, 0, 0, 0);
      if (m < rows) v[i] = *reinterpret_cast<const uint4*>(q + (long long)g * p.q_stride.head + (long long)token * p.q_stride.token);
      m += RPT;
      token += dt;
      g += dg;
      if (g >= p.group) { g -= p.group; ++token; }
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int row = first + i * RPT;
      const uint32_t dst = to + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(__byte_perm(v[i].x, v[i].z, 0x5410)),
                   "r"(__byte_perm(v[i].x, v[i].z, 0x7632)), "r"(__byte_perm(v[i].y, v[i].w, 0x5410)), "r"(__byte_perm(v[i].y, v[i].w, 0x7632)) : "memory");
    }
  }
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
  if (tid == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&bars->u_full[t]), 1);
      mbar_init(smem_u32(&bars->u_empty[t]), 14);
      mbar_init(smem_u32(&bars->q_full[t]), 4);
      mbar_init(smem_u32(&bars->q_free[t]), 1);
      mbar_init(smem_u32(&bars->s_full[t]), 1);
      mbar_init(smem_u32(&bars->p_full[t]), 4);
      mbar_init(smem_u32(&bars->p_free[t]), 1);
      mbar_init(smem_u32(&bars->drain[t]), 1);
    }
    mbar_init(smem_u32(&bars->asked), 1);
    mbar_init(smem_u32(&bars->s_free), 4);               // the warps of the tile whose logits were in the buffer
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
  if (tid == kUnitWarp * 32) make_unit(p, blockIdx.x, bars->unit[0]);
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

  // A role takes unit number n of the CTA (the first is ready, the others warp 1 makes), and gives it back.  False: a wait gave up.
  auto take_unit = [&](int n) { return n == 0 || wait_bar(&bars->u_full[n & 1], ((n - 1) >> 1) & 1, bars, polls); };
  auto give_unit = [&](int n) { mbar_arrive(smem_u32(&bars->u_empty[n & 1])); };

  if (warp >= kValueWarps) {
    // ------------------------------------------------------------------ codes to values
    reg_dec<kValueRegs>();
    constexpr int LPR = D / 32, RPW = 32 / LPR, PASSES = kBN / (4 * RPW);   // lanes of a row (16 bytes of codes each), rows of a warp
    const int t = lane % LPR, row_in = (warp - kValueWarps) * RPW + lane / LPR;
    uint4 codes[2][PASSES];
    uint32_t scales[2][PASSES];
    uint32_t g = 0;                            // blocks of the units before
    const volatile Unit* unit = bars->unit;
    long long row0 = 0;
    int j_begin = 0, seam = 0, skip = 0, last = 0;        // of the unit
    auto load = [&](int item, int set) {       // item 2 j: keys of block j, 2 j + 1: its values
      const int first = (j_begin + (item >> 1)) * kBN;
      const unsigned char* c = item & 1 ? p.planes.v_codes : p.planes.k_codes;
      const unsigned char* s = item & 1 ? p.planes.v_scales : p.planes.k_scales;
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        // (a place past the end: any finite values, its logits do not count)
        const int v = min(first + i * 4 * RPW + row_in, last);
        const long long row = row0 + (v < seam ? v : v + skip);
        codes[set][i] = *reinterpret_cast<const uint4*>(c + row * (D / 2) + t * 16);
        scales[set][i] = *reinterpret_cast<const uint16_t*>(s + row * (D / 16) + t * 2);
      }
    };
    auto write = [&](uint32_t tile, int set) {
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        const int row = i * 4 * RPW + row_in;
        const uint4 c = codes[set][i];
        // eight lanes write eight different 16-byte columns: those of the second 64 elements take their words in another order
        const bool other = D == 128 && (t & 2);
        const uint32_t w[4] = {other ? c.z : c.x, other ? c.w : c.y, other ? c.x : c.z, other ? c.y : c.w};
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
    uint32_t q_loads[2] = {0, 0};
    // a tile of queries; those of the first unit come through the softmax warps, which have nothing else to do then
    auto queries = [&](int tile, int n) {
      if (n > 0) {
        if (q_loads[tile] > 0 && !__all_sync(0xffffffffu, wait_bar(&bars->q_free[tile], (q_loads[tile] - 1) & 1, bars, polls))) return false;
        load_queries<D, 8>(p, *unit, tile, tid & 127, q_sm + tile * TILE_BYTES);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->q_full[tile]));
      }
      ++q_loads[tile];
      return true;
    };
    auto turn = [&](auto keys, int j, int set, int nblk) {
      constexpr bool K = decltype(keys)::value;
      const int item = 2 * j + (K ? 0 : 1);
      if (item + 1 < 2 * nblk) load(item + 1, set ^ 1);
      const uint32_t n = g + j, slot = n % kStages;
      if (n >= kStages &&
          !__all_sync(0xffffffffu, wait_bar(K ? &bars->k_empty[slot] : &bars->v_empty[slot], (n / kStages - 1) & 1, bars, polls)))
        return false;
      write((K ? k_sm : v_sm) + slot * TILE_BYTES, set);
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(K ? &bars->k_full[slot] : &bars->v_full[slot]));
      return true;
    };
    bool ok = true;
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      ok = __all_sync(0xffffffffu, take_unit(n));
      if (!ok) break;
      unit = &bars->unit[n & 1];
      const int nblk = unit->nblk;
      if (!unit->more) break;
      if (nblk > 0) {
        row0 = unit->row0;
        j_begin = unit->j_begin;
        seam = unit->seam;
        skip = unit->skip;
        last = unit->total - 1;
        load(0, 0);
        ok = queries(0, n) && (unit->ntile == 1 || queries(1, n));
#pragma unroll 1
        for (int j = 0; j < nblk && ok; ++j) ok = turn(std::true_type(), j, 0, nblk) && turn(std::false_type(), j, 1, nblk);
        g += nblk;
      }
      __syncwarp();
      if (lane == 0) give_unit(n);
    }
  } else if (warp >= kSoftmaxWarps) {
    // ------------------------------------------------------------------ softmax, output
    reg_inc<kSoftmaxRegs>();
    const int t = (warp - kSoftmaxWarps) >> 2, row = tid & 127;
    const uint32_t lane_addr = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lane_addr + S_COL, p_addr = tmem + lane_addr + P_COL + t * 64, o_addr = tmem + lane_addr + O_COL + t * D;
    const float c = p.scale_log2;
    uint32_t cnt = 0;                          // blocks of this tile so far
    bool ok = true;
    auto bar_all = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bar(bar, parity, bars, polls)) != 0; };
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      ok = __all_sync(0xffffffffu, take_unit(n));
      if (!ok) break;
      const volatile Unit& u = bars->unit[n & 1];                  // (registers that live through a block are scarce)
      if (!u.more) break;
      if (t >= u.ntile) {
        __syncwarp();
        if (lane == 0) give_unit(n);
        continue;
      }
      const int nblk = u.nblk, j_begin = u.j_begin, seam = u.seam, skip = u.skip, total = u.total;
      const int all_lo = u.all_lo, all_hi = u.all_hi, all_sink = u.all_sink;
      if (n == 0 && nblk > 0) {
        load_queries<D, D / 8>(p, u, t, row, q_sm + t * TILE_BYTES);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->q_full[t]));
      }
      float m_used = kNoLogit, l = 0.f;
#pragma unroll 1
      for (int j = 0; j < nblk; ++j) {
        const int first = (j_begin + j) * kBN, next = first + kBN;
        // whether every query of the unit sees all of the block: up to its last row, and from its first row behind the seam on
        const bool hides = next > total || (next > seam ? next + skip : next) > all_hi ||
                           !(next <= seam || max(first, seam) + skip >= all_lo || next + skip <= all_sink);
        ok = bar_all(&bars->s_full[t], cnt & 1);
        if (!ok) break;
        tc_fence_after();
        if (__builtin_expect(hides, 0)) {
          const int pos = u.len - u.nq + (u.m0 + t * kBM + row) / p.group;
          const int hi = p.causal ? pos + 1 : u.len, lo = p.window > 0 ? pos - p.window + 1 : 0;
          hide(s_addr, min(seam, hi) - first, seam - first, min(total, hi - skip) - first, lo - skip - first, all_sink - skip - first);
        }
        uint32_t sr[kBN];
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) tmem_ld32(s_addr + ch * 32, sr + ch * 32);
        tmem_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->s_free));       // the logits are in registers
        float mx4[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          mx4[v] = -INFINITY;
#pragma unroll
          for (int i = 0; i < 16; ++i) mx4[v] = max3(mx4[v], __uint_as_float(sr[v * 32 + 2 * i]), __uint_as_float(sr[v * 32 + 2 * i + 1]));
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
          const float2 z = fma2(make_float2(__uint_as_float(sr[2 * i]), __uint_as_float(sr[2 * i + 1])), c2, nmc2);
          const __nv_bfloat162 hh = __floats2bfloat162_rn(ex2(z.x), ex2(z.y));
          pk[i] = *reinterpret_cast<const uint32_t*>(&hh);
          add_bf162(sum[2 * (i & 1)], sum[2 * (i & 1) + 1], pk[i]);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        if (cnt > 0) {
          // the product of the block before still reads P_t and adds to O_t
          ok = bar_all(&bars->p_free[t], (cnt - 1) & 1);
          if (!ok) break;
          tc_fence_after();
          if (any && j > 0) {
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
        ++cnt;
      }
      if (ok && nblk > 0) {
        ok = bar_all(&bars->p_free[t], (cnt - 1) & 1);             // the unit's last product
        tc_fence_after();
      }
      if (!ok) break;
      const float inv = l > 0.f ? 1.f / l : 0.f;
      const int tile = u.tile + t, m = tile * kBM + row, token = m / p.group;
      const bool live = m < u.rows;
      unsigned char* dst = nullptr;
      float* part = nullptr;
      if (p.splits > 1) {
        float* const at_split = p.partial + (((long long)u.head * p.tiles + tile) * p.splits + u.split) * (kBM * (D + 2));
        part = at_split + row * D;
        if (live) *reinterpret_cast<float2*>(at_split + kBM * D + 2 * row) = make_float2(m_used, l);
      } else {
        dst = reinterpret_cast<unsigned char*>(static_cast<__nv_bfloat16*>(p.out) + u.b * p.out_stride.batch +
                                               (long long)(u.kvh * p.group + m - token * p.group) * p.out_stride.head +
                                               (long long)token * p.out_stride.token);
      }
#pragma unroll 1
      for (int half = 0; half < D / 64; ++half) {
        uint32_t o[64];
        __syncwarp();                                              // (threads without a row of their own left the half before early)
        if (nblk > 0) {
          tmem_ld32(o_addr + half * 64, o);
          tmem_ld32(o_addr + half * 64 + 32, o + 32);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int i = 0; i < 64; ++i) o[i] = 0;
        }
        if (!live) continue;
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) {
          // columns 0 4 1 5 2 6 3 7 of every eight
          float y[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) y[i] = __uint_as_float(o[16 * ch + (i & 8) + 2 * (i & 3) + ((i >> 2) & 1)]);
          if (part) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              reinterpret_cast<float4*>(part + half * 64 + ch * 16)[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
          } else {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const __nv_bfloat162 hh = __floats2bfloat162_rn(y[2 * i] * inv, y[2 * i + 1] * inv);
              w[i] = *reinterpret_cast<const uint32_t*>(&hh);
            }
            st_global_32b(dst + half * 128 + ch * 32, w, p.out_sectors != 0);
          }
        }
      }
      tc_fence_before();                                           // (the next unit's products write there)
      __syncwarp();
      if (lane == 0) give_unit(n);
    }
  } else {
    reg_dec<kIssueRegs>();
    // An issuer leaves when its last product has ended, or after a while
    auto drained = [&](uint64_t* bar) {
      mma_commit(smem_u32(bar));
#pragma unroll 1
      for (uint32_t it = 0; it < kDrainPolls && !mbar_try_wait(smem_u32(bar), 0); ++it) {}
    };
    bool ok = true;
    if (warp == kUnitWarp && lane == 0) {
      // ---------------------------------------------------------------- the CTA's next unit
      uint32_t q_loads = 0, answers = 0;                           // units with products, of this CTA; answers
      bool asked = false;
#pragma unroll 1
      for (int n = 0; ok; ++n) {
        int next = -1;
        if (p.steal) {
          // asked for at the start of a short unit, of a long one behind its last product with the first tile's queries
          // (asked for earlier, it would be kept from CTAs that are idle by then)
          const int nblk = bars->unit[n & 1].nblk;
          if (nblk >= kShortUnit) ok = wait_bar(&bars->q_free[0], q_loads & 1, bars, polls);
          if (nblk > 0) ++q_loads;
          if (!ok) break;
          mbar_expect_tx(smem_u32(&bars->asked), 16);
          clc_ask(smem_u32(&bars->answer), smem_u32(&bars->asked));
          asked = true;
          ok = wait_bar(&bars->asked, answers & 1, bars, polls);
          if (!ok) break;
          asked = false;
          ++answers;
          next = clc_answer(smem_u32(&bars->answer));
          fence_proxy_async();                                     // the next answer overwrites what was just read
        }
        const int slot = (n + 1) & 1;
        // (unit n - 1 has been given back)
        if (n >= 1) ok = wait_bar(&bars->u_empty[slot], ((n - 1) >> 1) & 1, bars, polls);
        if (!ok) break;
        make_unit(p, next, bars->unit[slot]);
        mbar_arrive(smem_u32(&bars->u_full[slot]));
        if (next < 0) break;
      }
      if (asked) {                                                 // an answer on its way gets a bounded chance to land
#pragma unroll 1
        for (uint32_t it = 0; it < kDrainPolls && !mbar_try_wait(smem_u32(&bars->asked), answers & 1); ++it) {}
      }
    } else if (warp == kQkWarp && lane == 0) {
      // ---------------------------------------------------------------- issuer of Q K^T
      constexpr uint32_t IDESC = idesc_bf16_f32(kBM, kBN, 0);
      const uint64_t q_desc = smem_desc_sw128(q_sm, 16, 1024), k_desc = smem_desc_sw128(k_sm, 16, 1024);
      uint32_t use = 0, g = 0, q_odd = 0;                          // products issued; blocks of the units before; parity of the tiles' queries
#pragma unroll 1
      for (int n = 0; ok; ++n) {
        ok = take_unit(n);
        if (!ok) break;
        const int nblk = bars->unit[n & 1].nblk, ntile = bars->unit[n & 1].ntile, more = bars->unit[n & 1].more;
        give_unit(n);
        if (!more) break;
#pragma unroll 1
        for (int j = 0; j < nblk && ok; ++j) {
          const uint32_t slot = (g + j) % kStages;
          const uint64_t kd = k_desc + (uint64_t)((slot * TILE_BYTES) >> 4);
#pragma unroll 1
          for (int t = 0; t < ntile; ++t) {
            if (j == 0) {
              ok = wait_bar(&bars->q_full[t], (q_odd >> t) & 1, bars, polls);
              q_odd ^= 1u << t;
            }
            if (ok && t == 0) ok = wait_bar(&bars->k_full[slot], ((g + j) / kStages) & 1, bars, polls);
            if (!ok || !wait_bar(&bars->s_free, (use - 1) & 1, bars, polls)) { ok = false; break; }   // (a fresh barrier passes for odd)
            tc_fence_after();
            const uint64_t qd = q_desc + (uint64_t)((t * TILE_BYTES) >> 4);
            if constexpr (D == 128) mma_ss_chain8(tmem + S_COL, qd, kd, IDESC, 0);
            else mma_ss_chain4(tmem + S_COL, qd, kd, IDESC, 0);
            mma_commit(smem_u32(&bars->s_full[t]));
            ++use;
            if (j == nblk - 1) mma_commit(smem_u32(&bars->q_free[t]));
          }
          if (ok) mma_commit(smem_u32(&bars->k_empty[slot]));
        }
        g += nblk;
      }
      drained(&bars->drain[0]);
    } else if (warp == kPvWarp && lane == 0) {
      // ---------------------------------------------------------------- issuer of P V
      constexpr uint32_t IDESC = idesc_bf16_f32(kBM, D, 1);        // V: rows of the tile are the summed index
      const uint64_t v_desc = smem_desc_sw128(v_sm, SUB_BYTES, 1024);
      uint32_t g = 0, odd = 0;                                     // blocks of the units before; parity of the tiles' products
#pragma unroll 1
      for (int n = 0; ok; ++n) {
        ok = take_unit(n);
        if (!ok) break;
        const int nblk = bars->unit[n & 1].nblk, ntile = bars->unit[n & 1].ntile, more = bars->unit[n & 1].more;
        give_unit(n);
        if (!more) break;
#pragma unroll 1
        for (int j = 0; j < nblk && ok; ++j) {
          const uint32_t slot = (g + j) % kStages;
          const uint64_t vd = v_desc + (uint64_t)((slot * TILE_BYTES) >> 4);
#pragma unroll 1
          for (int t = 0; t < ntile; ++t) {
            if (t == 0) ok = wait_bar(&bars->v_full[slot], ((g + j) / kStages) & 1, bars, polls);
            if (!ok || !wait_bar(&bars->p_full[t], (odd >> t) & 1, bars, polls)) { ok = false; break; }
            odd ^= 1u << t;
            tc_fence_after();
            const uint32_t o = tmem + O_COL + t * D, pa = tmem + P_COL + t * 64;
            mma_ts_chain4(o, pa, vd, IDESC, j > 0);
            mma_ts_chain4(o, pa + 32, vd + 4 * 128, IDESC, 1);
            mma_commit(smem_u32(&bars->p_free[t]));
          }
          if (ok) mma_commit(smem_u32(&bars->v_empty[slot]));
        }
        g += nblk;
      }
      drained(&bars->drain[1]);
    }
  }
  __syncwarp();                              // (an issuer is one thread of its warp)
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
int launch(Kv4AttendParams p, cudaStream_t st) {
  // (more than half of an SM's shared memory at head_dim 64 as well: a CTA owns the SM's tensor memory)
  constexpr size_t smem = smem_bytes<128>();
  static_assert(smem_bytes<D>() <= smem, "");
  if (!allow_dynamic_smem(kv4_attend_tc_kernel<D>, smem)) return -1;
  const int heads = p.units / p.tiles, cta_units = (p.tiles + p.tiles_per_cta - 1) / p.tiles_per_cta;
  const int grid = heads * cta_units * p.splits;
  p.steal = grid > sm_count();               // more units than CTAs run at once
  launch_k(kv4_attend_tc_kernel<D>, dim3(grid), dim3(kThreads), smem, st, p);
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
