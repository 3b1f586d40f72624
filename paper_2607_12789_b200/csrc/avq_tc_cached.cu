// Attention over a paged cache on the tensor cores (d 64 or 128): rows of bfloat16, rows of float32, or 4 bits.
//
// One query has a product of d multiply-adds with every cached token, so the call is bound by reading the cache once; the
// arithmetic has to keep out of the way.  Query heads that share a key head, and the nq queries of a sequence, are the
// rows of one product: S^T = K Q^T with 16 tokens by 8 (NT = 1) or 16 (NT = 2) rows, O^T += V^T P^T, by warp-level
// mma.sync (the rows are too few for tcgen05's 128 x N tiles, and both operands of the second product come from where
// they are: values from shared memory, weights from registers).
//
// The units of all segments are dealt out evenly (avq_exact.cuh).  Each warp of a CTA takes every kWarps-th unit of 16
// tokens through a ring of its own in shared memory, filled by 16-byte cp.async STAGES - 1 units ahead, with running
// maxima, sums and output of its own: no barrier between warps until a segment's end, when they are added in the order
// of the warps.  Chunks of 16 bytes are swizzled so that every fragment load is free of bank conflicts.
//
// 4 bits: the codes enter the products as integers and are never turned into the values they stand for.
//   keys    s = sum_g step_g <q_g, c_g> + lo_g sum(q_g):  one accumulator per group of 32 dimensions.
//   values  o_g += (p step_g) c + (p lo_g):  the weight is multiplied by each group's step before it is rounded to
//           bfloat16; p lo_g is summed per row and group in float32.
//   Keys: a code in the low bits of a 16-bit half is a subnormal number of half precision, c 2^-24, one place further up
//   c 2^-20; the tensor cores take those exactly, and the queries (brought to 2^14 by a power of two for their row, and
//   by 2^-4 where the code stands higher) lose nothing that a float32 sum would keep.  An AND makes a pair of codes.
//   Values: o_g += (p step_g) (c - 8) + p (lo_g + 8 step_g), the second sum small where values lie about zero, so that the
//   rounding of the weights meets c - 8 and not c.  The weights p step_g have a range of their own and stay bfloat16; an
//   AND-OR makes 0x4300 | c, which is 128 + c, of a code, and a product of the same rounded weights with a constant -136
//   takes the 136 out again.  (With three parts the 136 is taken off the codes: 143 times a part would cost the sum bits.)
// bfloat16 queries: weights are rounded to bfloat16 for the value product (their sums are of the float32 ones), which is 1.8e-3
// to 2.3e-3 of the result off where float32 weights are 1.6e-3 to 1.7e-3, the outputs' own rounding; parts would double it.
// float32: rows by tf32 products of two parts each (the lowest product left out: 2^-22 of a term; a unit's values and 32
// dimensions of its logits are summed from zero and added in registers, the low parts' products apart, since the tensor cores
// cut sums off; logits that the parts of an infinity make a NaN are taken again from the operands); 4 bits with float32
// queries by three parts of the query (half precision) and of the weight (bfloat16), which are all of their 24 bits, with the
// keys' codes about their middle too.
//
// Measured (B200, several calls one after another): 64 sequences of 1 .. 4096 tokens, 8 key heads, d 128, bfloat16 rows 78.5 us
// for 467 MB, 5.95 TB/s, 91 % of the measured copy rate, the joining kernel in it; the same in 4 bits, lengths to 8192, with the
// rows' way into the cache 91.7 us for 268 MB (2.9 TB/s), two sequences of 131072 and 28076 39 us for 102 MB: there the
// instructions that take codes apart and scale (450 for 16 tokens of one head, half of the issue slots) and the start of the
// CTAs are the time; float32 rows 29.5 us for 105 MB, a captured call; 4 bits with float32 queries, 64 sequences of up to 4096
// tokens, 8 key heads, d 128, 79 us.
//
// The running maximum of a row is raised only when a logit exceeds it by 2^8 (weights stay below 2^8, sums far inside
// float32): most units need a vote instead of shuffles and rescaling.
#include "avq_exact_mma.cuh"

namespace avq {
namespace exact {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr float kRaise = 8.f;
enum Rows { kBf16 = 0, kQ4 = 1, kF32 = 2 };

template <int MODE, int D> __host__ __device__ constexpr int unit_bytes() {
  return MODE == kQ4 ? 2 * kUnit * (D / 2 + D / 8) : 2 * kUnit * D * (MODE == kF32 ? 4 : 2);
}
// (4 bits: two CTAs to an SM, units in pairs and eight of them in a warp's ring 39.1 us for two long sequences; three CTAs with
// six 41.9, which leave the pairs too few registers, with seven 47.3.)
template <int MODE, int D> __host__ __device__ constexpr int stages() { return MODE == kQ4 ? 8 : MODE == kBf16 && D == 64 ? 5 : 3; }
template <int MODE, int D, int NT> __host__ __device__ constexpr int ctas_per_sm() { return MODE == kF32 && D == 128 ? 1 : 2; }
// Query fragments in shared memory: float32 queries only (their parts would take too many registers).
template <int MODE, int D, int NT, int PARTS> __host__ __device__ constexpr int query_bytes() {
  return MODE == kF32 ? (D / 8) * NT * 32 * 16 : MODE == kQ4 && PARTS == 3 ? (D / 16) * NT * 32 * 24 : 0;
}
template <int MODE, int D, int NT, int PARTS> __host__ __device__ constexpr size_t cached_smem() {
  return (size_t)kWarps * stages<MODE, D>() * unit_bytes<MODE, D>() + query_bytes<MODE, D, NT, PARTS>();
}

template <int MODE, int D, int NT, int PARTS>
struct Warp {
  [[maybe_unused]] static constexpr int kChunks = D * (MODE == kF32 ? 4 : 2) / 16;          // of a raw row
  static constexpr int kGroups = D / 32;
  static constexpr int kUnitBytes = unit_bytes<MODE, D>();
  static constexpr int kV = MODE == kQ4 ? kUnit * D / 2 : kUnitBytes / 2;  // offsets within a unit
  [[maybe_unused]] static constexpr int kKPairs = kUnit * D, kVPairs = kKPairs + kUnit * D / 8;

  float O[D / 16][NT][4];        // C fragments of O^T: columns (rows of the product) 8 nt + 2 t, + 1
  float m[NT][2], l[NT][2];      // maximum (the same in the 8 lanes of a column), this lane's share of the sum
  float limit[NT][2], sub[NT][2];   // the logit that raises the maximum, what is taken off scale * logit (powers of two)
  float off[NT][2][MODE == kQ4 ? kGroups : 1];   // sum p lo_g, this lane's share
  uint32_t q[MODE == kBf16 || (MODE == kQ4 && PARTS == 1) ? D / 16 : 1][NT][2];
  float qsum[MODE == kQ4 ? kGroups : 1][NT][2];
  float qback[NT][2];            // (4 bits) what the products with the codes are multiplied by: 2^24 and the row's power of two
  int lim[NT][2];                // tokens that the column's query sees

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) O[i][n][e] = 0.f;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[n][e] = limit[n][e] = -INFINITY;
        l[n][e] = sub[n][e] = 0.f;
#pragma unroll
        for (int w = 0; w < (MODE == kQ4 ? kGroups : 1); ++w) off[n][e][w] = 0.f;
      }
  }

  // Where a key head's rows are: this lane's first copy of the first page, bytes from page to page.
  struct Source {
    const char *k, *v, *pairs;
    int64_t page_bytes;
  };
  static __device__ __forceinline__ Source source_of(const CachedArgs& a, int hk, int lane) {
    Source r;
    constexpr int row = MODE == kQ4 ? D / 2 + D / 8 : D * (MODE == kF32 ? 4 : 2);
    const int64_t head = (int64_t)a.page * row;
    r.page_bytes = head * a.Hk;
    r.k = static_cast<const char*>(a.keys) + hk * head + 16 * lane;
    r.v = static_cast<const char*>(a.values) + hk * head + 16 * lane;
    if constexpr (MODE == kQ4) {
      constexpr int pairs = kUnit * D / 8 / 16;            // 16-byte chunks of a unit's (lo, step) pairs: 16 or 8
      r.pairs = (lane < pairs ? r.k : r.v) + a.page * (D / 2) + 16 * (lane % pairs) - 16 * lane;
    }
    return r;
  }
  // Copies of one unit, the `in_page`-th 16 rows of a page, into `dst` (shared).  Rows behind a sequence's last come along:
  // what they hold is kept out of the products.
  static __device__ __forceinline__ void fetch(uint32_t dst, const Source& src, int page, int in_page, int lane) {
    const int64_t at_page = (int64_t)page * src.page_bytes;
    if constexpr (MODE == kQ4) {
      constexpr int per = D / 32, count = kUnit * per;     // 16-byte chunks of a code row, of the unit
      const char *k = src.k + at_page + in_page * (kUnit * D / 2), *v = src.v + at_page + in_page * (kUnit * D / 2);
#pragma unroll
      for (int i0 = 0; i0 < count; i0 += 32) {
        const int i = i0 + lane, r = i / per, c = i % per;
        const uint32_t at = dst + 16 * (r * per + (D == 128 ? c ^ ((r >> 1) & 3) : c ^ ((r >> 2) & 1)));
        cp_async16(at, k + 16 * i0);
        cp_async16(at + kV, v + 16 * i0);
      }
      constexpr int pairs = kUnit * D / 8 / 16;
      if (2 * pairs == 32 || lane < 2 * pairs)
        cp_async16(dst + (lane < pairs ? kKPairs : kVPairs) + 16 * (lane % pairs), src.pairs + at_page + in_page * (kUnit * D / 8));
    } else {
      constexpr int row = kChunks * 16;
      const char *k = src.k + at_page + in_page * (kUnit * row), *v = src.v + at_page + in_page * (kUnit * row);
#pragma unroll
      for (int i0 = 0; i0 < kUnit * kChunks; i0 += 32) {
        const int i = i0 + lane, r = i / kChunks, c = i % kChunks;
        const uint32_t at = dst + r * row + 16 * (c ^ swizzle(r));
        cp_async16(at, k + 16 * i0);
        cp_async16(at + kV, v + 16 * i0);
      }
    }
  }

  // The queries of a segment: fragments in registers, or (float32) written to shared memory by one warp for all.
  template <typename T>
  __device__ __forceinline__ void load_queries(const CachedArgs& a, const Segment& sg, uint4* shared, bool write, int lane) {
    const int g = lane >> 2, t = lane & 3, G = a.H / a.Hk, rows = min(kRows, a.nq * G - sg.block * kRows);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = 8 * n + g, qi = sg.block * kRows + r;
      const bool ok = r < rows;
      const T* src = static_cast<const T*>(a.Q) + ((int64_t)sg.b * a.nq + (ok ? qi / G : 0)) * a.q_stride +
                     ((int64_t)sg.hk * G + (ok ? qi % G : 0)) * D;
      auto at = [&](int k) { return ok ? to_f32(src[k]) : 0.f; };
      if constexpr (MODE == kBf16) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          q[k][n][0] = ok ? *reinterpret_cast<const uint32_t*>(src + 16 * k + 2 * t) : 0u;
          q[k][n][1] = ok ? *reinterpret_cast<const uint32_t*>(src + 16 * k + 2 * t + 8) : 0u;
        }
      } else if constexpr (MODE == kQ4) {
        float part[kGroups], x[kGroups][8], most = 0.f;
#pragma unroll
        for (int w = 0; w < kGroups; ++w) {
          if (ok) load8(src + 32 * w + 8 * t, x[w]);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (!ok) x[w][i] = 0.f;
            most = fmaxf(most, fabsf(x[w][i]));
          }
          part[w] = ((x[w][0] + x[w][1]) + (x[w][2] + x[w][3])) + ((x[w][4] + x[w][5]) + (x[w][6] + x[w][7]));
        }
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        // the power of two that brings the row's largest element to 2^14 .. 2^15 (an infinity stays one)
        const int e = min(max((int)(__float_as_uint(most) >> 23), 27), 244);
        const float up = __uint_as_float((uint32_t)(268 - e) << 23);          // 2^(141 - e), e biased
        const float back = __uint_as_float((uint32_t)(e + (PARTS == 1 ? 10 : -14)) << 23);   // 2^(e - 141), with 2^24 where codes are c 2^-24
#pragma unroll
        for (int w = 0; w < kGroups; ++w)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const float u0 = x[w][2 * s] * up, u1 = x[w][2 * s + 4] * up, v0 = x[w][2 * s + 1] * up * 0.0625f, v1 = x[w][2 * s + 5] * up * 0.0625f;
            if constexpr (PARTS == 1) {
              q[2 * w + s][n][0] = pack_f16(u0, u1);
              q[2 * w + s][n][1] = pack_f16(v0, v1);
            } else if (write) {
              uint32_t p0[3], p1[3];
              three_f16_parts(u0, u1, p0);
              three_f16_parts(v0, v1, p1);
              uint2* to = reinterpret_cast<uint2*>(shared) + ((2 * w + s) * NT + n) * 3 * 32 + lane;
#pragma unroll
              for (int i = 0; i < 3; ++i) to[32 * i] = make_uint2(p0[i], p1[i]);
            }
          }
        qback[n][0] = __shfl_sync(0xffffffffu, back, 8 * t);
        qback[n][1] = __shfl_sync(0xffffffffu, back, 8 * t + 4);
#pragma unroll
        for (int w = 0; w < kGroups; ++w) {              // sums of groups, moved to the lanes of their columns
          part[w] *= 1.f / back;                           // (a power of two)
          part[w] += __shfl_xor_sync(0xffffffffu, part[w], 1);
          part[w] += __shfl_xor_sync(0xffffffffu, part[w], 2);
          qsum[w][n][0] = __shfl_sync(0xffffffffu, part[w], 8 * t);
          qsum[w][n][1] = __shfl_sync(0xffffffffu, part[w], 8 * t + 4);
        }
      } else if (write) {
#pragma unroll 4
        for (int k = 0; k < D / 8; ++k) {                // steps 2 c, 2 c + 1: dimensions 16 c + 4 t + (0, 1) and (2, 3)
          const int dim = 16 * (k / 2) + 4 * t + 2 * (k % 2);
          const float x = at(dim), y = at(dim + 1), xh = tf32_high(x), yh = tf32_high(y);
          shared[(k * NT + n) * 32 + lane] =
              make_uint4(__float_as_uint(xh), __float_as_uint(yh), tf32_low(x, xh), tf32_low(y, yh));
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int c = 8 * n + 2 * t + e;
        lim[n][e] = c < rows ? sg.len - a.nq + 1 + (sg.block * kRows + c) / G : 0;
      }
    }
  }

  __device__ __forceinline__ void logits(uint32_t at, const uint4* shared, float (&s)[NT][4], int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
    if constexpr (MODE == kBf16) {
      const int r = lane & 15;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        uint32_t x[4];
        ldmatrix4(x, at + r * (2 * D) + 16 * ((2 * k + (lane >> 4)) ^ swizzle(r)));
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_bf16(s[n], x, q[k][n][0], q[k][n][1]);
      }
    } else if constexpr (MODE == kQ4) {
      uint32_t x[kGroups], y[kGroups], px[kGroups], py[kGroups];   // tokens g and g + 8
      if constexpr (D == 128) {
        lds_words(x, at + g * 64 + 16 * (t ^ ((g >> 1) & 3)));
        lds_words(y, at + (g + 8) * 64 + 16 * (t ^ ((g >> 1) & 3)));
      } else {
        lds_words(x, at + g * 32 + (8 * t ^ (16 * ((g >> 2) & 1))));
        lds_words(y, at + (g + 8) * 32 + (8 * t ^ (16 * ((g >> 2) & 1))));
      }
      lds_words(px, at + kKPairs + g * (D / 8));
      lds_words(py, at + kKPairs + (g + 8) * (D / 8));
#pragma unroll
      for (int w = 0; w < kGroups; ++w) {
        float c[NT][4];
        if constexpr (PARTS == 1) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t f[4] = {subnormal_codes(x[w], 2 * k), subnormal_codes(y[w], 2 * k), subnormal_codes(x[w], 2 * k + 1),
                                   subnormal_codes(y[w], 2 * k + 1)};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              if (k == 0) mma_f16_first(c[n], f, q[2 * w][n][0], q[2 * w][n][1]);
              else mma_f16(c[n], f, q[2 * w + 1][n][0], q[2 * w + 1][n][1]);
            }
          }
        } else {
          // (codes about their middle, the high parts' products from zero, the others in a sum of their own: what the tensor cores
          // cut off is little.  All in one chain, of codes from 0: up to 3e-6 of the result instead of 5e-7.)
          float low[NT][4];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t f[4] = {centred_codes(x[w], 2 * k), centred_codes(y[w], 2 * k), centred_codes(x[w], 2 * k + 1),
                                   centred_codes(y[w], 2 * k + 1)};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint2* from = reinterpret_cast<const uint2*>(shared) + ((2 * w + k) * NT + n) * 3 * 32 + lane;
              float high[4];
              if (k == 0) mma_f16_first(low[n], f, from[64].x, from[64].y);
              else mma_f16(low[n], f, from[64].x, from[64].y);
              mma_f16(low[n], f, from[32].x, from[32].y);
              mma_f16_first(high, f, from[0].x, from[0].y);
#pragma unroll
              for (int e = 0; e < 4; ++e) c[n][e] = k == 0 ? high[e] : c[n][e] + high[e];
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) c[n][e] += low[n][e];
        }
        const float sx = high_f(px[w]), sy = high_f(py[w]);
        // (of a code's middle, where it is left out of the codes)
        const float lx = PARTS == 1 ? low_f(px[w]) : fmaf(8.f, sx, low_f(px[w])), ly = PARTS == 1 ? low_f(py[w]) : fmaf(8.f, sy, low_f(py[w]));
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            // (the query's power of two is in qsum too: taken back at the end)
            s[n][e] = fmaf(sx, c[n][e], w == 0 ? lx * qsum[w][n][e] : fmaf(lx, qsum[w][n][e], s[n][e]));
            s[n][2 + e] = fmaf(sy, c[n][2 + e], w == 0 ? ly * qsum[w][n][e] : fmaf(ly, qsum[w][n][e], s[n][2 + e]));
          }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][e] *= qback[n][e & 1];
    } else {
      // (sums of the products with a low part apart, those of the high parts from zero every 32 dimensions and added in
      // registers: the tensor cores cut sums off)
      float low[NT][4] = {};
#pragma unroll 2
      for (int c2 = 0; c2 < D / 32; ++c2) {
        float high[NT][4];
#pragma unroll
        for (int c1 = 0; c1 < 2; ++c1) {
          const int c = 2 * c2 + c1;
          const uint4 u = lds128(at + g * (4 * D) + 16 * ((4 * c + t) ^ swizzle(g)));
          const uint4 v = lds128(at + (g + 8) * (4 * D) + 16 * ((4 * c + t) ^ swizzle(g)));
          const uint32_t xs[4] = {u.x, u.y, u.z, u.w}, ys[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint32_t hi[4] = {xs[2 * k], ys[2 * k], xs[2 * k + 1], ys[2 * k + 1]}, lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float x = __uint_as_float(hi[i]), h = tf32_high(x);
              hi[i] = __float_as_uint(h);
              lo[i] = tf32_low(x, h);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint4 f = shared[((2 * c + k) * NT + n) * 32 + lane];
              mma_tf32(low[n], lo, f.x, f.y);
              mma_tf32(low[n], hi, f.z, f.w);
              if (c1 == 0 && k == 0) mma_tf32_first(high[n], hi, f.x, f.y);
              else mma_tf32(high[n], hi, f.x, f.y);
            }
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n][e] += high[n][e];
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][e] += low[n][e];
    }
  }

  // (float32 rows) The parts of an infinity can make a NaN of a logit that is none: such logits once more, from the rows
  // themselves.  (A row that has had a NaN keeps it.)
  __device__ __forceinline__ void mend_logits(uint32_t at, const CachedArgs& a, const Segment& sg, float (&s)[NT][4], int lane) {
    const int g = lane >> 2, t = lane & 3, G = a.H / a.Hk, rows = min(kRows, a.nq * G - sg.block * kRows);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = 8 * n + 2 * t + (e & 1), r = g + 8 * (e >> 1), q = sg.block * kRows + c;
        if (s[n][e] == s[n][e] || l[n][e & 1] != l[n][e & 1] || c >= rows) continue;
        const float* src = static_cast<const float*>(a.Q) + ((int64_t)sg.b * a.nq + q / G) * a.q_stride + ((int64_t)sg.hk * G + q % G) * D;
        float sum = 0.f;
#pragma unroll 1
        for (int k = 0; k < D / 4; ++k) {
          const float4 x = reinterpret_cast<const float4*>(src)[k];
          const uint4 y = lds128(at + r * (4 * D) + 16 * (k ^ swizzle(r)));
          sum = fmaf(x.x, __uint_as_float(y.x), sum);
          sum = fmaf(x.y, __uint_as_float(y.y), sum);
          sum = fmaf(x.z, __uint_as_float(y.z), sum);
          sum = fmaf(x.w, __uint_as_float(y.w), sum);
        }
        s[n][e] = sum;
      }
  }

  // O^T += V^T P^T for one unit.  p: weights in the layout of the logits.
  // SKIP: tokens from `seen` on do not exist for this product (raw rows: their values are made zero).
  template <bool SKIP>
  __device__ __forceinline__ void values(uint32_t at, const float (&p)[NT][4], int seen, int lane) {
    const int g = lane >> 2, t = lane & 3;
    if constexpr (MODE == kBf16) {
      uint32_t b[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        b[n][0] = transpose8(pack_bf16(p[n][0], p[n][1]));
        b[n][1] = transpose8(pack_bf16(p[n][2], p[n][3]));
      }
      const int r = (lane & 7) + 8 * (lane >> 4), c = (lane >> 3) & 1;
      const uint32_t keep[2] = {(2 * t < seen ? 0xffffu : 0u) | (2 * t + 1 < seen ? 0xffff0000u : 0u),
                                (2 * t + 8 < seen ? 0xffffu : 0u) | (2 * t + 9 < seen ? 0xffff0000u : 0u)};
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        uint32_t v[4];
        ldmatrix4_trans(v, at + kV + r * (2 * D) + 16 * ((2 * i + c) ^ swizzle(r)));
        if (SKIP) { v[0] &= keep[0]; v[1] &= keep[0]; v[2] &= keep[1]; v[3] &= keep[1]; }
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_bf16(O[i][n], v, b[n][0], b[n][1]);
      }
    } else if constexpr (MODE == kQ4) {
      uint32_t px[kGroups], py[kGroups], cw[4][kGroups];
      lds_words(px, at + kVPairs + g * (D / 8));
      lds_words(py, at + kVPairs + (g + 8) * (D / 8));
#pragma unroll
      for (int j = 0; j < 4; ++j) {                      // tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
        const int r = 2 * t + (j & 1) + 8 * (j >> 1);
        if constexpr (D == 128) lds_words(cw[j], at + kV + r * 64 + 16 * ((g >> 1) ^ ((r >> 1) & 3)));
        else lds_words(cw[j], at + kV + r * 32 + (8 * (g >> 1) ^ (16 * ((r >> 2) & 1))));
      }
      const uint32_t half = (g & 1) ? 0x7632u : 0x5410u; // upper or lower halves of two words
      constexpr uint32_t minus[4] = {0xc308c308u, 0xc308c308u, 0xc308c308u, 0xc308c308u};   // -136
#pragma unroll
      for (int w = 0; w < kGroups; ++w) {
        const float sx = high_f(px[w]), sy = high_f(py[w]), lx = fmaf(8.f, sx, low_f(px[w])), ly = fmaf(8.f, sy, low_f(py[w]));
        uint32_t b[NT][PARTS][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            x[e] = p[n][e] * sx;
            x[2 + e] = p[n][2 + e] * sy;
            if (!SKIP) {
              off[n][e][w] = fmaf(p[n][e], lx, fmaf(p[n][2 + e], ly, off[n][e][w]));
            } else {                                     // (a token that is not seen may have any step and lo)
              if (p[n][e] == 0.f) x[e] = 0.f;
              else off[n][e][w] = fmaf(p[n][e], lx, off[n][e][w]);
              if (p[n][2 + e] == 0.f) x[2 + e] = 0.f;
              else off[n][e][w] = fmaf(p[n][2 + e], ly, off[n][e][w]);
            }
          }
          if constexpr (PARTS == 1) {
            b[n][0][0] = transpose8(pack_bf16(x[0], x[1]));
            b[n][0][1] = transpose8(pack_bf16(x[2], x[3]));
          } else {
            uint32_t u[3], v[3];
            three_parts(x[0], x[1], u);
            three_parts(x[2], x[3], v);
#pragma unroll
            for (int i = 0; i < 3; ++i) { b[n][i][0] = transpose8(u[i]); b[n][i][1] = transpose8(v[i]); }
          }
        }
        const uint32_t u = __byte_perm(cw[0][w], cw[1][w], half), v = __byte_perm(cw[2][w], cw[3][w], half);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t f[4] = {codes_at(u, 2 * j), codes_at(u, 2 * j + 1), codes_at(v, 2 * j), codes_at(v, 2 * j + 1)};
          if constexpr (PARTS == 3) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = centred(f[i]);
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            if constexpr (PARTS == 3) {
              float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int i = PARTS - 1; i >= 0; --i) mma_bf16(part, f, b[n][i][0], b[n][i][1]);
#pragma unroll
              for (int e = 0; e < 4; ++e) O[2 * w + j][n][e] += part[e];
            } else {
              mma_bf16(O[2 * w + j][n], f, b[n][0][0], b[n][0][1]);
              mma_bf16(O[2 * w + j][n], minus, b[n][0][0], b[n][0][1]);
            }
          }
        }
      }
    } else {
      // weights as B fragments: lane (g, t) needs row g's weights of tokens t + 4 j, which lanes 4 (t + 4 j) + g / 2 hold
      uint32_t hi[NT][4], lo[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int from = 4 * (t + 4 * (j & 1)) + (g >> 1);
          const float x = __shfl_sync(0xffffffffu, p[n][2 * (j >> 1)], from), y = __shfl_sync(0xffffffffu, p[n][2 * (j >> 1) + 1], from);
          const float w = (g & 1) ? y : x, h = tf32_high(w);
          hi[n][j] = __float_as_uint(h);
          lo[n][j] = tf32_low_weight(w, h);
        }
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        uint32_t v[4][4];                                // tokens t + 4 j, dimensions 32 c + 4 g ..
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = t + 4 * j;
          const uint4 u = lds128(at + kV + r * (4 * D) + 16 * ((8 * c + g) ^ swizzle(r)));
          const bool keep = !SKIP || r < seen;
          v[j][0] = keep ? u.x : 0u; v[j][1] = keep ? u.y : 0u; v[j][2] = keep ? u.z : 0u; v[j][3] = keep ? u.w : 0u;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float part[NT][4];
#pragma unroll
          for (int k = 0; k < 2; ++k) {                    // tokens 8 k ..
            uint32_t h[4] = {v[2 * k][2 * i], v[2 * k][2 * i + 1], v[2 * k + 1][2 * i], v[2 * k + 1][2 * i + 1]}, x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float f = __uint_as_float(h[e]), fh = tf32_high(f);
              h[e] = __float_as_uint(fh);
              // (weights go up to 2^8: two of an infinity's stand-ins can overflow, and then have to have its sign)
              x[e] = tf32_low(f, fh) | (__float_as_uint(f) & 0x80000000u);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              if (k == 0) mma_tf32_first(part[n], x, hi[n][0], hi[n][1]);
              else mma_tf32(part[n], x, hi[n][2], hi[n][3]);
              mma_tf32(part[n], h, lo[n][2 * k], lo[n][2 * k + 1]);
              mma_tf32(part[n], h, hi[n][2 * k], hi[n][2 * k + 1]);
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) O[2 * c + i][n][e] += part[n][e];
        }
      }
    }
  }

  // The columns' largest logits of this lane; the maxima raised where one is too far above; weights in the logits' place.
  static __device__ __forceinline__ void tops(const float (&s)[NT][4], float (&top)[NT][2]) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) top[n][e] = fmaxf(s[n][e], s[n][2 + e]);
  }
  __device__ __forceinline__ void raise_to(const float (&top)[NT][2], float c) {
    bool raise = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) raise |= top[n][e] > limit[n][e];
    if (!__any_sync(0xffffffffu, raise)) return;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = top[n][e];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
        if (!(x > limit[n][e])) continue;                  // (each column by its own logits alone: roundings too)
        const float f = x == -INFINITY ? 1.f : ex2((m[n][e] - x) * c);
        m[n][e] = x;
        limit[n][e] = x + kRaise / c;
        sub[n][e] = x == -INFINITY ? 0.f : x * c;
        l[n][e] *= f;
#pragma unroll
        for (int w = 0; w < (MODE == kQ4 ? kGroups : 1); ++w) off[n][e][w] *= f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) { O[i][n][e] *= f; O[i][n][2 + e] *= f; }
      }
  }
  __device__ __forceinline__ void weigh(float (&s)[NT][4], float c) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        s[n][e] = ex2(fmaf(s[n][e], c, -sub[n][e]));
        s[n][2 + e] = ex2(fmaf(s[n][2 + e], c, -sub[n][e]));
        l[n][e] += s[n][e] + s[n][2 + e];
      }
  }

  // Two units that every query sees whole, at `at` and `then`: one vote for both, and two chains of products.
  __device__ __forceinline__ void pair(uint32_t at, uint32_t then, const uint4* shared, float c, int lane) {
    float s[2][NT][4], top[2][NT][2];
    logits(at, shared, s[0], lane);
    logits(then, shared, s[1], lane);
    tops(s[0], top[0]);
    tops(s[1], top[1]);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) top[0][n][e] = fmaxf(top[0][n][e], top[1][n][e]);
    raise_to(top[0], c);
    weigh(s[0], c);
    weigh(s[1], c);
    values<false>(at, s[0], kUnit, lane);
    values<false>(then, s[1], kUnit, lane);
  }

  // One unit: tokens from `token` on, of which the first `rows` count, in shared memory at `at`.
  __device__ __forceinline__ void unit(uint32_t at, const uint4* shared, const CachedArgs& a, const Segment& sg, int token, int rows, float c,
                                       int lane) {
    const int g = lane >> 2, len = sg.len, nq = a.nq;
    float s[NT][4];
    logits(at, shared, s, lane);
    const bool edge = rows < kUnit || token + kUnit > len - nq + 1;
    if (edge) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = g + 8 * (e >> 1);
          if (r >= rows || token + r >= lim[n][e & 1]) s[n][e] = -INFINITY;
        }
    }
    if constexpr (MODE == kF32) {
      float all = s[0][0];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) all = max_nan(all, s[n][e]);
      if (all != all) mend_logits(at, a, sg, s, lane);
    }
    float top[NT][2];
    tops(s, top);
    raise_to(top, c);
    weigh(s, c);
    if (!edge) {
      values<false>(at, s, kUnit, lane);
      return;
    }

    if (MODE == kQ4 || nq == 1) {
      values<true>(at, s, rows, lane);
      return;
    }
    // Some queries see fewer of these tokens than others: one product per distinct number, from values that are zero
    // beyond it, and of each only the columns that it is for (a weight of zero times an infinity would be NaN).
    int done = -1;
    while (true) {
      int next = kUnit + 1;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int v = min(max(lim[n][e] - token, 0), rows);
          if (v > done) next = min(next, v);
        }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) next = min(next, __shfl_xor_sync(0xffffffffu, next, o));
      if (next > kUnit) break;
      done = next;
      if (next == 0) continue;
      float keep[D / 16][NT][4];
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) keep[i][n][e] = O[i][n][e];
      values<true>(at, s, next, lane);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (min(max(lim[n][e & 1] - token, 0), rows) != next) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i) O[i][n][e] = keep[i][n][e];
          }
    }
  }

  // Dimension of element e of O[i] in this lane.
  static __device__ __forceinline__ int dim_of(int i, int e, int g) {
    if constexpr (MODE == kBf16) return 16 * i + g + 8 * (e >> 1);
    return 32 * (i >> 1) + 4 * g + 2 * (i & 1) + (e >> 1);
  }
};

template <typename T, int MODE, int D, int NT>
__global__ void __launch_bounds__(kThreads, ctas_per_sm<MODE, D, NT>()) cached_kernel(const CachedArgs a, int least) {
  constexpr int PARTS = sizeof(T) == 4 && MODE == kQ4 ? 3 : 1, S = stages<MODE, D>();
  using W = Warp<MODE, D, NT, PARTS>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Walk walk;
  __shared__ float ms[kWarps][8 * NT], ls[kWarps][8 * NT];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint4* queries = reinterpret_cast<uint4*>(smem + (size_t)kWarps * S * W::kUnitBytes);
  const uint32_t ring = tc::smem_u32(smem) + warp * S * W::kUnitBytes;
  const float c = a.scale * kLog2e;
  const int G = a.H / a.Hk, per_page = a.page / kUnit, shift = per_page > 1 ? 32 - __clz(per_page - 1) : 0;
  W w;
  Segment sg;
  int turn = 0;
  for (bool more = walk_begin(a, least, walk, sg); more; more = walk_next(a, walk, sg, ++turn)) {
    const int first = sg.unit + warp, end = sg.unit + sg.n;
    const int mine = first < end ? (end - first + kWarps - 1) / kWarps : 0;
    // Where this warp's units are, 32 of them at a time, one in each lane: physical page and place in it in one word (fewer
    // than 2^28 of them), the next 32 read ahead.  A page that is not there is read as the first one: none of its rows count.
    const typename W::Source src = W::source_of(a, sg.hk, lane);
    const int32_t* table = a.table + (int64_t)sg.b * a.table_pages;
    auto place_of = [&](int k) {
      if (k >= mine) return 0;
      const int u = first + k * kWarps, entry = u / per_page, page = table[entry];
      return page < 0 || page >= a.pages ? -1 : page << shift | (u - entry * per_page);
    };
    int places = place_of(lane), then_places = 0, fetched = 0;
    uint32_t bad = 0;                                      // of the units in flight, those whose page is not there
    auto fetch = [&](int slot) {
      bad <<= 1;
      if (fetched < mine) {
        if ((fetched & 31) == 0) {
          if (fetched > 0) places = then_places;
          then_places = place_of(fetched + 32 + lane);
        }
        int place = __shfl_sync(0xffffffffu, places, fetched & 31);
        if (place < 0) {
          bad |= 1;
          place = 0;
          if (lane == 0) report(a.status, DEV_BAD_INDEX);
        }
        W::fetch(ring + slot * W::kUnitBytes, src, place >> shift, place & ((1 << shift) - 1), lane);
        ++fetched;
      }
      cp_async_commit();
    };
    auto take_queries = [&] {
      if (MODE == kF32 || PARTS == 3) __syncthreads();     // (the segment before is done with the shared queries)
      w.template load_queries<T>(a, sg, queries, warp == 0, lane);
      if (MODE == kF32 || PARTS == 3) __syncthreads();
    };
    // 4 bits: the queries first, or they would wait behind the ring's first copies, which the arithmetic is behind anyway (two
    // long sequences 45.1 -> 43.4 us).  Rows: the copies first, the cache is all that is waited for (53.3 against 57.3 us).
    if constexpr (MODE == kQ4) take_queries();
    // (units in pairs where the ring holds two of them and as many again in flight)
    constexpr bool kPairs = MODE == kQ4 && NT == 1;
    constexpr int kAhead = kPairs ? S - 2 : S - 1;         // units fetched ahead
#pragma unroll
    for (int k = 0; k < kAhead; ++k) fetch(k);
    if constexpr (MODE != kQ4) take_queries();
    w.clear();
    int now = 0, next = kAhead, token = first * kUnit;
    auto after = [](int slot) { return slot + 1 == S ? 0 : slot + 1; };
    for (int k = 0; k < mine; k += kPairs ? 2 : 1) {
      cp_async_wait<kPairs ? S - 4 : S - 2>();
      __syncwarp();
      fetch(next);
      next = after(next);
      if constexpr (kPairs) {
        fetch(next);
        next = after(next);
        const int then = after(now), last = token + kWarps * kUnit;
        if (k + 1 < mine && last + kUnit <= sg.len - a.nq + 1 && (bad >> (S - 2) & 3) == 0) {
          w.pair(ring + now * W::kUnitBytes, ring + then * W::kUnitBytes, queries, c, lane);
        } else {
          w.unit(ring + now * W::kUnitBytes, queries, a, sg, token, bad >> (S - 1) & 1 ? 0 : min(kUnit, sg.len - token), c, lane);
          if (k + 1 < mine)
            w.unit(ring + then * W::kUnitBytes, queries, a, sg, last, bad >> (S - 2) & 1 ? 0 : min(kUnit, sg.len - last), c, lane);
        }
        token += 2 * kWarps * kUnit;
        now = after(then);
      } else {
        w.unit(ring + now * W::kUnitBytes, queries, a, sg, token, bad >> (S - 1) & 1 ? 0 : min(kUnit, sg.len - token), c, lane);
        token += kWarps * kUnit;
        now = after(now);
      }
      __syncwarp();
    }
    cp_async_wait<0>();
    // ---- the warps' results added: maxima, sums and outputs through shared memory, in the order of the warps
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          w.l[n][e] += __shfl_xor_sync(0xffffffffu, w.l[n][e], o);
#pragma unroll
          for (int x = 0; x < (MODE == kQ4 ? W::kGroups : 1); ++x)
            if (MODE == kQ4) w.off[n][e][x] += __shfl_xor_sync(0xffffffffu, w.off[n][e][x], o);
        }
        // (a warp that met nothing but NaN has raised no maximum: it must not pass for one that saw no token)
        if (w.l[n][e] != w.l[n][e]) w.m[n][e] = w.l[n][e];
        if (g == 0) { ms[warp][8 * n + 2 * t + e] = w.m[n][e]; ls[warp][8 * n + 2 * t + e] = w.l[n][e]; }
      }
    __syncthreads();                                       // (every warp is done with its ring: it holds the outputs now)
    float* out = reinterpret_cast<float*>(smem);           // [kWarps][8 NT][D + 4]
    constexpr int kPitch = D + 4;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * n + 2 * t + e;
        float top = ms[0][r];
#pragma unroll
        for (int x = 1; x < kWarps; ++x) top = fmaxf(top, ms[x][r]);
        const float f = w.m[n][e] == -INFINITY ? 0.f : ex2((w.m[n][e] - top) * c);
        float* row = out + (warp * 8 * NT + r) * kPitch;
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float v = w.O[i][n][2 * h + e];
            if constexpr (MODE == kQ4) v += w.off[n][e][i >> 1];
            row[W::dim_of(i, 2 * h, g)] = f == 0.f ? 0.f : v * f;
          }
      }
    __syncthreads();
    const int rows = min(kRows, a.nq * G - sg.block * kRows);
    float* slot = segment_slot(a, sg);
    for (int r = warp; r < rows; r += kWarps) {
      float top = ms[0][r], sum = 0.f;
#pragma unroll
      for (int x = 1; x < kWarps; ++x) top = fmaxf(top, ms[x][r]);
#pragma unroll
      for (int x = 0; x < kWarps; ++x) sum += ms[x][r] == -INFINITY ? 0.f : ls[x][r] * ex2((ms[x][r] - top) * c);
      const int q = sg.block * kRows + r;
      const int64_t token = (int64_t)sg.b * a.nq + q / G;
      const int h = sg.hk * G + q % G;
      constexpr int kPer = D / 32;
      float y[kPer] = {};
#pragma unroll
      for (int x = 0; x < kWarps; ++x)
#pragma unroll
        for (int i = 0; i < kPer; ++i) y[i] += out[(x * 8 * NT + r) * kPitch + kPer * lane + i];
      if (slot) {
        if (lane == 0) { slot[r] = sum != sum ? sum : top == -INFINITY ? -INFINITY : top * c; slot[kRows + r] = sum; }
#pragma unroll
        for (int i = 0; i < kPer; ++i) slot[2 * kRows + r * D + kPer * lane + i] = y[i];
      } else {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        T* Y = static_cast<T*>(a.Y) + token * a.y_stride + (int64_t)h * D + kPer * lane;
#pragma unroll
        for (int i = 0; i < kPer; ++i) Y[i] = from_f32<T>(y[i] * inv);
        if (a.lse && lane == 0) a.lse[token * a.H + h] = sum == 0.f ? -INFINITY : (top * c + log2f(sum)) * kLn2;
      }
    }
    __syncthreads();                                       // (the ring may be filled again)
  }
}

template <typename T, int MODE, int D, int NT>
avq_status launch(const CachedArgs& a, int dtype, cudaStream_t st) {
  constexpr int PARTS = sizeof(T) == 4 && MODE == kQ4 ? 3 : 1;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return AVQ_ERR_CUDA;
  avq_status s = open_shared_memory<cached_kernel<T, MODE, D, NT>>(dev);
  if (s != AVQ_OK) return s;
  const int ctas = min(sms * ctas_per_sm<MODE, D, NT>(), kMaxCtas), least = 2 * kWarps;
  cached_kernel<T, MODE, D, NT><<<ctas, kThreads, cached_smem<MODE, D, NT, PARTS>(), st>>>(a, least);
  s = cuda_ok(cudaGetLastError());
  return s == AVQ_OK ? join(a, dtype, st) : s;
}
template <typename T, int MODE>
avq_status launch_rows(const CachedArgs& a, int dtype, cudaStream_t st) {
  const bool few = a.nq * (a.H / a.Hk) <= 8;
  if (a.d == 64) return few ? launch<T, MODE, 64, 1>(a, dtype, st) : launch<T, MODE, 64, 2>(a, dtype, st);
  return few ? launch<T, MODE, 128, 1>(a, dtype, st) : launch<T, MODE, 128, 2>(a, dtype, st);
}

}  // namespace

avq_status tc_cached(const CachedArgs& a, int dtype, int bits, cudaStream_t st) {
  if (dtype == AVQ_F32) return bits == 4 ? launch_rows<float, kQ4>(a, dtype, st) : launch_rows<float, kF32>(a, dtype, st);
  return bits == 4 ? launch_rows<__nv_bfloat16, kQ4>(a, dtype, st) : launch_rows<__nv_bfloat16, kBf16>(a, dtype, st);
}

}  // namespace exact
}  // namespace avq
