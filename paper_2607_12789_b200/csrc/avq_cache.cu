// Paged cache of keys and values: rows in (rotated by their positions, stored in the tensors' type or in 4 bits) and
// rows out.  Both kernels are copies with a little arithmetic: a lane takes 8 dimensions (16 or 32
// bytes) of a row, d/8 neighbouring lanes a row, so that a row's partner dimensions of the rotation and the groups of 32
// of the 4-bit form are within a warp, and every lane has loaded its part before any stores (queries may be rotated in
// place).  16384 tokens, 16 query and 8 key heads, d 128, bfloat16: into 4 bits with the rotation 60 us (231 MB, 3.8 TB/s, two
// thirds of the issue slots: the rotation's products and the codes are what is left), back 20 us (88 MB, 4.4 TB/s).
#include "avq_exact.cuh"

namespace avq {
namespace exact {
namespace {

__device__ __forceinline__ float min_nan(float a, float b) {   // NaN if either is
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ float min3_nan(float a, float b, float c) {
  float r;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Eight elements as they are in memory, and as float32.
template <typename T> struct Raw;
template <> struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  __device__ __forceinline__ Raw from_lane(int lane) const {
    Raw r;
    r.a = make_float4(__shfl_sync(0xffffffffu, a.x, lane), __shfl_sync(0xffffffffu, a.y, lane), __shfl_sync(0xffffffffu, a.z, lane),
                      __shfl_sync(0xffffffffu, a.w, lane));
    r.b = make_float4(__shfl_sync(0xffffffffu, b.x, lane), __shfl_sync(0xffffffffu, b.y, lane), __shfl_sync(0xffffffffu, b.z, lane),
                      __shfl_sync(0xffffffffu, b.w, lane));
    return r;
  }
};
template <> struct Raw<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ Raw from_lane(int lane) const {
    Raw r;
    r.a = make_uint4(__shfl_sync(0xffffffffu, a.x, lane), __shfl_sync(0xffffffffu, a.y, lane), __shfl_sync(0xffffffffu, a.z, lane),
                     __shfl_sync(0xffffffffu, a.w, lane));
    return r;
  }
};
// Rounded to T and back.
__device__ __forceinline__ void round_to(float (&)[8], const float*) {}
__device__ __forceinline__ void round_to(float (&v)[8], const __nv_bfloat16*) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint32_t w = pack_bf16(v[i], v[i + 1]);
    v[i] = __uint_as_float(w << 16);
    v[i + 1] = __uint_as_float(w & 0xffff0000u);
  }
}

constexpr uint32_t magic_sum() {                           // of 1.5 * 2^23 at the places of 8 codes
  uint32_t n = 0;
  for (int i = 0; i < 8; ++i) n += 0x4b400000u << (4 * i);
  return n;
}
constexpr uint32_t kMagicSum = magic_sum();

// Four lanes hold a group of 32 values, 8 each: their codes, and (lo, step) for the group's first lane to store.
// lo and step are rounded to bfloat16 as they are stored, so that codes refer to what a reader will see; products and
// differences are rounded one by one (no fused multiply-add): the result is the same wherever it is computed.
__device__ __forceinline__ uint32_t q4_encode8(const float (&v)[8], uint32_t& pair) {
  float lo = min_nan(min3_nan(v[0], v[1], v[2]), min3_nan(v[3], v[4], v[5])), hi = max_nan(max3_nan(v[0], v[1], v[2]), max3_nan(v[3], v[4], v[5]));
  lo = min3_nan(lo, v[6], v[7]);
  hi = max3_nan(hi, v[6], v[7]);
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const __nv_bfloat16 lob = __float2bfloat16_rn(lo);
  lo = __bfloat162float(lob);
  const __nv_bfloat16 stepb = __float2bfloat16_rn(__fmul_rn(__fsub_rn(hi, lo), (float)(1.0 / 15.0)));
  const float step = __bfloat162float(stepb);
  pair = (uint32_t)__bfloat16_as_ushort(lob) | (uint32_t)__bfloat16_as_ushort(stepb) << 16;
  if (!(step > 0.f)) return 0;                             // (a NaN too: the group reads as NaN whatever its codes)
  // Quotients as correctly rounded divisions have them, by Markstein's two steps from the reciprocal (ties of codes are
  // common among bfloat16 values: a division for each that is next to one was three quarters of this kernel's
  // instructions).  Adding 1.5 * 2^23 rounds to the nearest integer, ties to even, and leaves it in the low bits.
  constexpr float kMagic = 12582912.f;
  uint32_t word = 0;
  if (step >= 1e-30f) {
    const float by = __frcp_rn(step);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = __fsub_rn(v[i], lo), q = __fmul_rn(x, by), c = __fmaf_rn(__fmaf_rn(-q, step, x), by, q);
      word += __float_as_uint(fminf(fmaxf(__fadd_rn(c, kMagic), kMagic), kMagic + 15.f)) << (4 * i);   // (the magic number's own low bits are zero)
    }
    word -= kMagicSum;
  } else {                                                 // (the reciprocal may be beyond the largest number)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = fminf(fmaxf(__fdiv_rn(__fsub_rn(v[i], lo), step), 0.f), 15.f);
      word |= (__float_as_uint(__fadd_rn(c, kMagic)) & 15u) << (4 * i);
    }
  }
  return word;
}

constexpr int kThreads = 256;

// Heads of a token that a lane takes one after the other: their loads are in flight together, and the angles of its
// dimensions are read once for all of them.
constexpr int kHeads = 4;

// The row that a lane works on and its place in it.  (The number of lanes of a row, d / 8, divides 32 or nearly so; a
// division of numbers up to 32 by a float reciprocal is exact.)
struct Lane {
  int lanes, sub, j;             // lanes of a row, this lane's row within the warp, its place in the row
  int token;                     // (beyond the last one for lanes without a row)
};
__device__ __forceinline__ Lane lane_of(int d) {
  Lane r;
  const int lane = threadIdx.x & 31;
  r.lanes = d >> 3;
  const float by = __frcp_ru((float)r.lanes);
  const int per = (int)(32.f * by);
  r.sub = (int)((float)lane * by);
  r.j = lane - r.sub * r.lanes;
  r.token = r.sub < per ? (blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * per + r.sub : 0x7fffffff;
  return r;
}

// kHeads heads of one token: `src` and `dst` are this lane's 8 dimensions of the first of them, `heads` of which exist.
// TURN: 0 as they are, 1 pairs of halves, 2 pairs of neighbours.  BITS: 4 for codes (dst: a page's share of the head),
// otherwise rows of T, `next` elements apart.
template <typename T, int BITS, int TURN>
__device__ __forceinline__ void append_heads(const AppendArgs& a, const Lane& at, int heads, const T* src, int slot, int pos, bool ok,
                                             char* dst, int64_t next) {
  const int j = at.j;
  Raw<T> x[kHeads];
#pragma unroll
  for (int u = 0; u < kHeads; ++u) x[u].load(src + (u < heads ? u : 0) * a.d);
  const int half = a.rot >> 4;                             // lanes of the first halves of the pairs
  const bool first = j < half, turned = 8 * j < a.rot;
  float cs[8], sn[8];
  if constexpr (TURN == 1) {
    if (turned && ok) {
      const int64_t row = (int64_t)pos * (a.rot >> 1) + 8 * (first ? j : j - half);
      load8(a.cos + row, cs);
      load8(a.sin + row, sn);
      if (first) {                                         // x1 cos - x2 sin, x2 cos + x1 sin: one form, the sine's sign
#pragma unroll
        for (int i = 0; i < 8; ++i) sn[i] = -sn[i];
      }
    }
  } else if constexpr (TURN == 2) {
    if (turned && ok) {
      const int64_t row = (int64_t)pos * (a.rot >> 1) + 4 * j;
      const float4 c = *reinterpret_cast<const float4*>(a.cos + row), s = *reinterpret_cast<const float4*>(a.sin + row);
      cs[0] = c.x; cs[1] = c.y; cs[2] = c.z; cs[3] = c.w;
      sn[0] = s.x; sn[1] = s.y; sn[2] = s.z; sn[3] = s.w;
    }
  }
  const int from = (at.sub * at.lanes + (turned ? (first ? j + half : j - half) : j)) & 31;
  const int row = BITS == 4 ? (ok ? slot : 0) % a.page : 0;
  char* pair_at = dst + q4_pair_at(row, a.d, a.page, j >> 2);
  char* code_at = dst + q4_code_at(row, a.d, j);
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    if (u >= heads) break;
    float v[8];
    x[u].values(v);
    if constexpr (TURN == 1) {
      float w[8];
      x[u].from_lane(from).values(w);
      if (turned) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fadd_rn(__fmul_rn(v[i], cs[i]), __fmul_rn(w[i], sn[i]));
      }
    } else if constexpr (TURN == 2) {
      if (turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = v[2 * i], f = v[2 * i + 1];
          v[2 * i] = __fsub_rn(__fmul_rn(e, cs[i]), __fmul_rn(f, sn[i]));
          v[2 * i + 1] = __fadd_rn(__fmul_rn(f, cs[i]), __fmul_rn(e, sn[i]));
        }
      }
    }
    if constexpr (BITS == 4) {                             // d % 32 == 0: a group's four lanes are neighbours
      if constexpr (TURN != 0) round_to(v, (const T*)nullptr);
      uint32_t pair;
      const uint32_t word = q4_encode8(v, pair);
      if (ok) {
        *reinterpret_cast<uint32_t*>(code_at + u * next) = word;
        if ((j & 3) == 0) *reinterpret_cast<uint32_t*>(pair_at + u * next) = pair;
      }
    } else if (ok) {
      store8(reinterpret_cast<T*>(dst) + u * next, v);
    }
  }
}

// A lane takes kHeads heads of keys, of values or of queries (blockIdx.y) of one token; a block does one kind of work.
template <typename T, int BITS, int TURN>
__global__ void __launch_bounds__(kThreads) append_kernel(const AppendArgs a) {
  const Lane at = lane_of(a.d);
  const int parts = (a.Hk + kHeads - 1) / kHeads, group = blockIdx.y;
  const bool in = at.token < a.T;
  const int token = in ? at.token : 0;                     // (a lane without a row goes along: the shuffles are the warp's)
  const int slot = a.slots[token], pos = TURN ? a.pos[token] : 0;
  bool ok = in && slot != -1;
  if (ok && (slot < 0 || slot >= a.pages * a.page || (TURN && (pos < 0 || pos >= a.angles)))) {
    report(a.status, DEV_BAD_INDEX);
    ok = false;
  }
  const int col = 8 * min(at.j, at.lanes - 1);
  if (group >= 2 * parts) {
    const int h = (group - 2 * parts) * kHeads;
    append_heads<T, 0, TURN>(a, at, min(kHeads, a.H - h), static_cast<const T*>(a.Q) + token * a.q_stride + (int64_t)h * a.d + col, slot, pos, ok,
                             reinterpret_cast<char*>(static_cast<T*>(a.Q_out) + token * a.q_out_stride + (int64_t)h * a.d + col), a.d);
    return;
  }
  const bool key = group < parts;
  const int h = (key ? group : group - parts) * kHeads, heads = min(kHeads, a.Hk - h);
  const int p = ok ? slot / a.page : 0;
  const T* src = key ? static_cast<const T*>(a.K) + token * a.k_stride : static_cast<const T*>(a.V) + token * a.v_stride;
  src += (int64_t)h * a.d + col;
  char* dst = static_cast<char*>(key ? a.keys : a.values);
  int64_t next;
  if constexpr (BITS == 4) {
    next = q4_page_bytes(a.page, a.d);
    dst += ((int64_t)p * a.Hk + h) * next;
  } else {
    next = (int64_t)a.page * a.d;
    dst = reinterpret_cast<char*>(reinterpret_cast<T*>(dst) + ((int64_t)p * a.Hk + h) * next + (int64_t)(ok ? slot - p * a.page : 0) * a.d + col);
  }
  if (key) append_heads<T, BITS, TURN>(a, at, heads, src, slot, pos, ok, dst, next);
  else append_heads<T, BITS, 0>(a, at, heads, src, slot, pos, ok, dst, next);
}

template <typename T, int BITS>
__global__ void __launch_bounds__(kThreads) read_kernel(const ReadArgs a) {
  const Lane at = lane_of(a.d);
  if (at.token >= a.T) return;
  const int token = at.token, j = at.j, head0 = blockIdx.y * kHeads;
  const int slot = a.slots[token];
  if (slot == -1) return;
  if (slot < 0 || slot >= a.pages * a.page) { report(a.status, DEV_BAD_INDEX); return; }
  const int p = slot / a.page, r = slot - p * a.page;
  float v[kHeads][8];
  uint32_t word[kHeads], pair[kHeads];
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const int head = head0 + u;
    if (head >= 2 * a.Hk) break;
    const bool key = head < a.Hk;
    const void* base = key ? a.keys : a.values;
    const int64_t at_head = (int64_t)p * a.Hk + (key ? head : head - a.Hk);
    if (BITS == 4) {
      const char* at = static_cast<const char*>(base) + at_head * q4_page_bytes(a.page, a.d);
      word[u] = *reinterpret_cast<const uint32_t*>(at + q4_code_at(r, a.d, j));
      pair[u] = *reinterpret_cast<const uint32_t*>(at + q4_pair_at(r, a.d, a.page, j >> 2));
    } else {
      load8(static_cast<const T*>(base) + (at_head * a.page + r) * a.d + 8 * j, v[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const int head = head0 + u;
    if (head >= 2 * a.Hk) break;
    const bool key = head < a.Hk;
    if (BITS == 4) q4_decode8(word[u], pair[u], v[u]);
    T* out = static_cast<T*>(key ? a.K : a.V) + token * (key ? a.k_stride : a.v_stride) + (int64_t)(key ? head : head - a.Hk) * a.d;
    store8(out + 8 * j, v[u]);
  }
}

template <typename Kernel, typename Args>
avq_status launch_rows(Kernel kernel, const Args& a, int groups, cudaStream_t st) {
  const int per = (kThreads / 32) * (32 / (a.d >> 3));
  kernel<<<dim3((unsigned)(((int64_t)a.T + per - 1) / per), (unsigned)groups), kThreads, 0, st>>>(a);
  return cuda_ok(cudaGetLastError());
}

}  // namespace

namespace {
template <typename T, int BITS>
avq_status append(const AppendArgs& a, cudaStream_t st) {
  const int groups = 2 * ((a.Hk + kHeads - 1) / kHeads) + (a.H + kHeads - 1) / kHeads;
  if (a.rot == 0) return launch_rows(append_kernel<T, BITS, 0>, a, groups, st);
  return a.adjacent ? launch_rows(append_kernel<T, BITS, 2>, a, groups, st) : launch_rows(append_kernel<T, BITS, 1>, a, groups, st);
}
}  // namespace

avq_status cache_append(const AppendArgs& a, int dtype, int bits, cudaStream_t st) {
  if (dtype == AVQ_F32) return bits == 4 ? append<float, 4>(a, st) : append<float, 32>(a, st);
  return bits == 4 ? append<__nv_bfloat16, 4>(a, st) : append<__nv_bfloat16, 16>(a, st);
}
avq_status cache_read(const ReadArgs& a, int dtype, int bits, cudaStream_t st) {
  const int groups = (2 * a.Hk + kHeads - 1) / kHeads;
  if (dtype == AVQ_F32) return bits == 4 ? launch_rows(read_kernel<float, 4>, a, groups, st) : launch_rows(read_kernel<float, 32>, a, groups, st);
  return bits == 4 ? launch_rows(read_kernel<__nv_bfloat16, 4>, a, groups, st) : launch_rows(read_kernel<__nv_bfloat16, 16>, a, groups, st);
}

}  // namespace exact
}  // namespace avq
