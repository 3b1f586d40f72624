// Exact attention: what its kernels share (not part of the ABI) - arguments, the 4-bit rows of a paged cache, which
// piece of a packed batch a CTA works on, and how cached sequences are split over CTAs and joined again.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "avq_internal.h"

namespace avq {
namespace exact {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct PromptArgs {
  const void *Q, *K, *V;
  void* Y;
  float* lse;
  const int32_t *cu_q, *cu_k;
  int64_t q_stride, k_stride, v_stride, y_stride;
  int32_t H, Hk, d, S, Tq, Tk;
  int32_t causal;
  float scale;
  int32_t* status;
  float* parts;                  // room for the partial results of split pieces, or null
};

struct CachedArgs {
  const void *Q, *keys, *values;
  void* Y;
  float* lse;
  float* partial;                // slots of partial results
  int2* records;                 // of each segment: the first and last CTA that left a part of it, or (-1, ..): one had it all
  const int32_t *table, *lens;
  int64_t q_stride, y_stride;
  int32_t H, Hk, d, B, nq, pages, page, table_pages;
  float scale;
  int32_t* status;
};

struct AppendArgs {
  const void *K, *V, *Q;
  void *keys, *values, *Q_out;
  const int32_t* slots;
  const float *cos, *sin;
  const int32_t* pos;
  int64_t k_stride, v_stride, q_stride, q_out_stride;
  int32_t T, H, Hk, d, page, pages, angles, rot, adjacent;
  int32_t* status;
};

struct ReadArgs {
  const void *keys, *values;
  void *K, *V;
  const int32_t* slots;
  int64_t k_stride, v_stride;
  int32_t T, Hk, d, page, pages;
  int32_t* status;
};

__device__ __forceinline__ void report(int32_t* status, int32_t code) {
  if (status) atomicCAS(status, 0, code);
}

// ---------------------------------------------------------------- element types
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// 8 consecutive elements, 16-byte aligned
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
  const uint4 a = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// ---------------------------------------------------------------- rows of a 4-bit cache
// Bytes of one head's share of a page, and the places in it (the layout is the header's).
__host__ __device__ __forceinline__ int64_t q4_page_bytes(int page, int d) { return (int64_t)page * (5 * d / 8); }
__device__ __forceinline__ int q4_code_at(int row, int d, int dim8) {      // the word of dimensions 8 dim8 .. + 7
  return row * (d >> 1) + (dim8 & 3) * (d >> 3) + 4 * (dim8 >> 2);
}
__device__ __forceinline__ int q4_pair_at(int row, int d, int page, int group) {
  return page * (d >> 1) + row * (d >> 3) + 4 * group;
}
__device__ __forceinline__ void q4_decode8(uint32_t word, uint32_t pair, float (&v)[8]) {
  const float lo = __uint_as_float(pair << 16), step = __uint_as_float(pair & 0xffff0000u);
  // a code in the low bits of 2^23 is the float 2^23 + code (cheaper than a conversion)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = __fadd_rn(__uint_as_float(((word >> (4 * i)) & 15u) | 0x4b000000u), -8388608.f);
    v[i] = __fadd_rn(lo, __fmul_rn(c, step));
  }
}

// ---------------------------------------------------------------- packed batches
// One tile of `rows` queries of one sequence.
struct Piece {
  int32_t q0, nq, k0, nk;        // the sequence's queries and keys
  int32_t first;                 // the tile's first query within the sequence
};
// Whether sequence s is usable, and its bounds.
__device__ __forceinline__ bool sequence(const PromptArgs& a, int s, Piece& p) {
  p.q0 = a.cu_q[s];
  const int q1 = a.cu_q[s + 1];
  int k1 = q1;
  p.k0 = p.q0;
  if (a.cu_k) { p.k0 = a.cu_k[s]; k1 = a.cu_k[s + 1]; }
  const bool ok = p.q0 >= 0 && q1 >= p.q0 && q1 <= a.Tq && p.k0 >= 0 && k1 >= p.k0 && k1 <= a.Tk;
  p.nq = ok ? q1 - p.q0 : 0;
  p.nk = ok ? k1 - p.k0 : 0;
  return ok;
}
// The tile number `index`, counted from the last tile of the last sequence down: of one causal sequence the tiles with
// the most keys come first, so that no long one is left for the end.  Called by all lanes of a warp; false: there are
// not so many tiles.  One pass over the bounds of at most S sequences, 32 at a time.
__device__ __forceinline__ bool find_piece(const PromptArgs& a, int rows, int index, Piece& out) {
  const int lane = threadIdx.x & 31;
  int left = index;
  for (int top = a.S; top > 0; top -= 32) {
    const int s = top - 1 - lane;
    Piece p = {0, 0, 0, 0, 0};
    if (s >= 0 && !sequence(a, s, p)) report(a.status, DEV_BAD_INDEX);
    const int tiles = (p.nq + rows - 1) / rows;
    int sum = tiles;                                       // inclusive over the lanes
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += up;
    }
    const uint32_t in = __ballot_sync(0xffffffffu, sum > left);
    if (in) {
      const int who = __ffs(in) - 1;
      const int before = __shfl_sync(0xffffffffu, sum - tiles, who);
      const int n = __shfl_sync(0xffffffffu, tiles, who);
      out.q0 = __shfl_sync(0xffffffffu, p.q0, who);
      out.nq = __shfl_sync(0xffffffffu, p.nq, who);
      out.k0 = __shfl_sync(0xffffffffu, p.k0, who);
      out.nk = __shfl_sync(0xffffffffu, p.nk, who);
      out.first = (n - 1 - (left - before)) * rows;
      return true;
    }
    left -= __shfl_sync(0xffffffffu, sum, 31);
  }
  return false;
}
// Tiles that S sequences of together T queries can have, and one more, whose CTA passes over every sequence and so
// reports unusable ones.  (sum of ceil(n/rows) < T/rows + S.)
inline int64_t most_pieces(int64_t T, int64_t S, int64_t rows) { return T / rows + S + 1; }

// ---------------------------------------------------------------- cached sequences over CTAs
// Queries of one sequence that share a key head, nq * H/Hk rows, are taken in blocks of kRows.  A segment is one such
// block of one key head of one sequence; its tokens are units of kUnit.  The units of all segments, in the order
// (sequence, key head, block, unit), are dealt out in equal runs to the CTAs, whatever the lengths: a CTA finishes the
// segments that lie inside its run and leaves partial results of the at most two that do not, its first in slot 2 c,
// its last in slot 2 c + 1.  join_kernel merges those in the order of the CTAs, by the records that the CTAs with the
// segments' first units leave.
// A segment also costs a CTA its queries, the start of its copies and the end of its sums, whatever its length: about as much
// as kSetup units, which stand before its own (six sequences of which one has 4 tokens, float32: 52.6 us
// without, 41.4 with 8, 30.5 with 16, 29.3 with 32, which costs a step of 64 sequences 2 %).
constexpr int kRows = 16, kUnit = 16, kSetup = 16;
constexpr int kMaxCtas = 148 * 4;                          // (more SMs than that are not asked for)
__host__ __device__ constexpr int64_t slot_floats(int d) { return (int64_t)kRows * (d + 2); }

__device__ __forceinline__ int clipped_len(const CachedArgs& a, int b, bool tell) {
  const int n = a.lens[b];
  const int64_t most = (int64_t)a.table_pages * a.page;
  if (tell && (n < 0 || n > most)) report(a.status, DEV_BAD_INDEX);
  return n < 0 ? 0 : (int64_t)n > most ? (int)most : n;
}
__device__ __forceinline__ int units_of(int len) { return (len + kUnit - 1) / kUnit; }
__device__ __forceinline__ int weight_of(int units) { return units > 0 ? units + kSetup : 0; }
__device__ __forceinline__ int segments_per_sequence(const CachedArgs& a) {
  return a.Hk * ((a.nq * (a.H / a.Hk) + kRows - 1) / kRows);
}
// Sum over the block of one value per thread (scratch: 33 words of shared memory); every thread gets it.
__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  int64_t s = 0;
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) s += scratch[w];
  return s;
}

// The physical page of a sequence's token, or -1 (reported) if the table holds no usable one.
__device__ __forceinline__ int page_of(const CachedArgs& a, int b, int token) {
  const int p = a.table[(int64_t)b * a.table_pages + token / a.page];
  if (p >= 0 && p < a.pages) return p;
  report(a.status, DEV_BAD_INDEX);
  return -1;
}
// A CTA's share of one segment: units unit .. unit + n - 1 of its `units`.
struct Segment {
  int32_t b, hk, block, len;
  int32_t unit, n, units;
};
struct Place {                   // of the first unit not yet handed out
  int64_t at, before;            // its number, the number of the first unit of sequence b
  int32_t b;
};
struct Walk {                    // shared: every thread reads one place and the first writes the next beside it
  int64_t scratch[34], end, run; // end of the CTA's run, length of every CTA's
  Place place[2];
};
// (64-bit divisions are long; nearly all are of numbers that fit 32 bits.)
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
  return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}
__device__ __forceinline__ int64_t run_of(int64_t total, int ctas, int least) {
  const int64_t run = quotient(total + ctas - 1, ctas);
  return run < least ? least : run;
}
// Every thread of the block calls these two and gets the same segment; false: the run is over.  `turn`: 0, 1, ... of the
// calls.  Between two calls the block meets at a barrier.
__device__ __forceinline__ bool walk_next(const CachedArgs& a, Walk& w, Segment& sg, int turn) {
  const int per = segments_per_sequence(a), blocks = per / a.Hk;
  const Place p = w.place[turn & 1];
  const int64_t end = w.end;
  int64_t at = p.at, before = p.before;
  int b = p.b, len = clipped_len(a, b, false), U = units_of(len), W = weight_of(U);
  while (at < end) {                                       // (a run's last bit may be a setup alone: that segment is the next CTA's)
    while (at >= before + (int64_t)W * per) {              // (ends: at < end <= the weight of all)
      before += (int64_t)W * per;
      len = clipped_len(a, ++b, false);
      U = units_of(len);
      W = weight_of(U);
    }
    const int64_t rel = at - before;
    const int seg = (int)quotient(rel, W), x = (int)(rel - (int64_t)seg * W), take = (int)min((int64_t)(W - x), end - at);
    at += take;
    sg.unit = max(0, x - kSetup);
    sg.n = x + take - kSetup - sg.unit;
    if (sg.n <= 0) continue;
    sg.b = b; sg.hk = seg / blocks; sg.block = seg % blocks; sg.len = len;
    sg.units = U;
    if (threadIdx.x == 0) {
      w.place[(turn + 1) & 1] = {at, before, b};
      if (sg.unit == 0) {                                  // (the CTA with a segment's first unit tells of it)
        const int64_t last = before + (int64_t)(seg + 1) * W - 1;
        a.records[(int64_t)b * per + seg] = sg.n == U ? make_int2(-1, 0) : make_int2(blockIdx.x, (int)quotient(last, w.run));
      }
    }
    return true;
  }
  return false;
}
// Sum of `v` over the threads before this one; `total`: over all of them.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* scratch, int64_t& total) {
  int64_t sum = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t up = __shfl_up_sync(0xffffffffu, sum, o);
    if ((int)(threadIdx.x & 31) >= o) sum += up;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 31) scratch[threadIdx.x >> 5] = sum;
  __syncthreads();
  total = 0;
  for (int k = 0; k < (int)(blockDim.x >> 5); ++k) {
    if (k < (int)(threadIdx.x >> 5)) sum += scratch[k];
    total += scratch[k];
  }
  return sum - v;
}
__device__ __forceinline__ bool walk_begin(const CachedArgs& a, int least, Walk& w, Segment& sg) {
  const int per = segments_per_sequence(a);
  int64_t total = 0;
  if (a.B > (int)blockDim.x) {                             // more than one scan: all lengths once for their sum
    int64_t mine = 0;
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) mine += weight_of(units_of(clipped_len(a, b, false)));
    total = block_sum(mine, w.scratch) * per;
  }
  int64_t before = 0;
  for (int b0 = 0; b0 < a.B; b0 += blockDim.x) {           // the sequence that holds the run's first unit
    const int b = b0 + threadIdx.x;
    const int64_t u = b < a.B ? (int64_t)weight_of(units_of(clipped_len(a, b, blockIdx.x == 0))) * per : 0;
    int64_t all;
    const int64_t base = before + block_scan(u, w.scratch, all);
    if (a.B <= (int)blockDim.x) total = all;
    const int64_t run = run_of(total, gridDim.x, least), at = (int64_t)blockIdx.x * run;
    if (blockIdx.x > 0 && at >= total) return false;
    if (u > 0 && at >= base && at < base + u) {
      w.place[0] = {at, base, b};
      w.end = min(at + run, total);
      w.run = run;
    }
    before += all;
    if (at < before && blockIdx.x > 0) break;              // (the first CTA looks at every length, to report bad ones)
  }
  __syncthreads();
  return total > 0 && walk_next(a, w, sg, 0);
}
// Where a share of a segment leaves its partial result, or null: the share is all of it.
__device__ __forceinline__ float* segment_slot(const CachedArgs& a, const Segment& sg) {
  if (sg.n == sg.units) return nullptr;
  return a.partial + (int64_t)(2 * blockIdx.x + (sg.unit == 0)) * slot_floats(a.d);
}

// ---------------------------------------------------------------- kernels' host sides
avq_status cache_append(const AppendArgs& a, int dtype, int bits, cudaStream_t st);
avq_status cache_read(const ReadArgs& a, int dtype, int bits, cudaStream_t st);
avq_status simt_prompt(const PromptArgs& a, int dtype, cudaStream_t st);
avq_status simt_cached(const CachedArgs& a, int dtype, int bits, cudaStream_t st);
avq_status tc_prompt(const PromptArgs& a, cudaStream_t st);
avq_status tc_prompt_f32(const PromptArgs& a, cudaStream_t st);
constexpr int kPromptCtas = 148;                           // (more SMs than that are not asked for)
size_t tc_prompt_part_bytes(int d);
avq_status tc_cached(const CachedArgs& a, int dtype, int bits, cudaStream_t st);
avq_status join(const CachedArgs& a, int dtype, cudaStream_t st);

}  // namespace exact
}  // namespace avq
