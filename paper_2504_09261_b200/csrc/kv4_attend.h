// Attention over a cache of 4 bits: what its kernels share.
#pragma once

#include "kv4.cuh"

namespace hack {

struct Kv4AttendParams {
  kv4::Planes planes;
  int kv_heads, group;              // group: query heads of a stored head
  int n_queries, max_len;
  int causal, window, n_sink, appended;
  int tile_rows;                    // query rows of a tile: 8 or 16, or 128 on the tensor cores
  int tiles, units, splits;         // tiles of query rows of a stored head, all of them, CTAs that share the rows of one
  int clustered;                    // few rows: they are a cluster
  int tiles_per_cta;                // tensor cores: 1 or 2
  int steal;                        // tensor cores: more units than CTAs run at once, a CTA goes on with another one
  int out_sectors;                  // rows of the output start on 32-byte boundaries
  uint32_t wait_polls;              // limit of a wait
  float scale_log2;                 // sm_scale * log2(e)
  const int32_t* lens;
  const int32_t* new_lens;
  const void* q;
  void* out;
  hack_strides_t q_stride, out_stride;
  float* partial;                   // [units][splits]: [tile_rows][D] outputs, [tile_rows][2] reference maximum and sum
};

// The tensor-core kernel (bf16); partial results where splits > 1.
int launch_kv4_attend_tc(const Kv4AttendParams& p, int head_dim, cudaStream_t st);

// Rows of a head that its queries may see: [0, sink_end) and [lo, hi).  Every row of a tile sees all of [all_lo, all_hi), and those of
// [0, all_sink).
struct Kv4Range { int sink_end, lo, hi, all_lo, all_hi, all_sink; };

#if defined(__CUDACC__)
__device__ __forceinline__ int kv4_length(const Kv4AttendParams& p, int head, int nq) {
  // (64 bits: a length next to the end of 32 must not wrap)
  const long long len = (long long)max(p.lens[head], 0) + (p.appended ? nq : 0);
  if (p.planes.row_off && !kv4::inside(p.planes, (long long)p.planes.row_off[head])) return 0;
  return (int)min(len, (long long)min(p.max_len, p.planes.cap));
}
// Of the query rows first .. last of a head (row = token * group + head of the group)
__device__ __forceinline__ Kv4Range kv4_range(const Kv4AttendParams& p, int len, int nq, int first, int last) {
  Kv4Range r;
  const int at0 = len - nq + first / p.group, at1 = len - nq + last / p.group;   // positions of the first and last token
  r.hi = p.causal ? max(min(len, at1 + 1), 0) : len;
  r.all_hi = p.causal ? min(len, at0 + 1) : len;
  r.lo = p.window > 0 ? min(max(at0 - p.window + 1, 0), r.hi) : 0;
  r.all_lo = p.window > 0 ? max(at1 - p.window + 1, 0) : 0;
  r.sink_end = p.window > 0 ? min(p.n_sink, r.lo) : 0;
  r.all_sink = p.window > 0 ? p.n_sink : 0;
  return r;
}
// Runs of `size` rows that cover it
__device__ __forceinline__ int kv4_chunks(const Kv4Range& r, int size) { return (r.sink_end + size - 1) / size + (r.hi - r.lo + size - 1) / size; }
// Whether every query row of the tile sees the 32 rows from `first` on
__device__ __forceinline__ bool kv4_all_see(const Kv4Range& r, int first) {
  return first + 32 <= r.all_hi && (first >= r.all_lo || first + 32 <= r.all_sink);
}
// Whether a query at position `at` sees `row` (below the length)
__device__ __forceinline__ bool kv4_sees(const Kv4AttendParams& p, int at, int row) {
  return (!p.causal || row <= at) && (p.window == 0 || row < p.n_sink || row > at - p.window);
}
// Four elements of output row m of a stored head; total: the sum they are divided by, 0 where nothing was seen
template <bool F32>
__device__ __forceinline__ void kv4_store(const Kv4AttendParams& p, int b, int kvh, int m, int d, float4 sum, float total) {
  const float inv = total > 0.f ? 1.f / total : 0.f;
  sum.x *= inv; sum.y *= inv; sum.z *= inv; sum.w *= inv;
  const int token = m / p.group, g = m - token * p.group;
  const long long at = b * p.out_stride.batch + (long long)(kvh * p.group + g) * p.out_stride.head + (long long)token * p.out_stride.token + d;
  if (F32) {
    *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = sum;
  } else {
    const __nv_bfloat162 x = __floats2bfloat162_rn(sum.x, sum.y), y = __floats2bfloat162_rn(sum.z, sum.w);
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
  }
}
#endif

}  // namespace hack
