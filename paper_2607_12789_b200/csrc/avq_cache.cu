// Paged cache of keys and values: rows in (rotated by their positions, stored in the tensors' type or in 4 bits) and
// rows out.  Both kernels are copies with a little arithmetic, bound by memory: a lane takes 8 dimensions (16 or 32
// bytes) of a row, d/8 neighbouring lanes a row, so that a row's partner dimensions of the rotation and the groups of 32
// of the 4-bit form are within a warp, and every lane has loaded its part before any stores (queries may be rotated in
// place).
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

// Four lanes hold a group of 32 values, 8 each: their codes, and (lo, step) for the group's first lane to store.
// lo and step are rounded to bfloat16 as they are stored, so that codes refer to what a reader will see; products and
// differences are rounded one by one (no fused multiply-add): the result is the same wherever it is computed.
__device__ __forceinline__ uint32_t q4_encode8(const float (&v)[8], uint32_t mask, uint32_t& pair) {
  float lo = v[0], hi = v[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) { lo = min_nan(lo, v[i]); hi = max_nan(hi, v[i]); }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    lo = min_nan(lo, __shfl_xor_sync(mask, lo, o));
    hi = max_nan(hi, __shfl_xor_sync(mask, hi, o));
  }
  const __nv_bfloat16 lob = __float2bfloat16_rn(lo);
  lo = __bfloat162float(lob);
  const __nv_bfloat16 stepb = __float2bfloat16_rn(__fmul_rn(__fsub_rn(hi, lo), (float)(1.0 / 15.0)));
  const float step = __bfloat162float(stepb);
  pair = (uint32_t)__bfloat16_as_ushort(lob) | (uint32_t)__bfloat16_as_ushort(stepb) << 16;
  uint32_t word = 0;
  if (step > 0.f) {                                        // (not for a NaN: the group reads as NaN whatever its codes)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = rintf(__fdiv_rn(__fsub_rn(v[i], lo), step));
      word |= (uint32_t)fminf(fmaxf(c, 0.f), 15.f) << (4 * i);
    }
  }
  return word;
}

constexpr int kThreads = 256;

// One row is one head of one token: Hk of keys, Hk of values, then H of queries (if any), token by token.
template <typename T, int BITS>
__global__ void __launch_bounds__(kThreads) append_kernel(const AppendArgs a) {
  const int lanes = a.d >> 3, per = 32 / lanes, lane = threadIdx.x & 31;
  const int sub = lane / lanes, j = lane - sub * lanes;
  const int64_t row = ((int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * per + sub;
  const bool in = sub < per && row < a.rows;
  const int heads = a.H + 2 * a.Hk;
  const int64_t token = in ? row / heads : 0;
  const int head = in ? (int)(row - token * heads) : 0;
  const bool key = head < a.Hk, value = !key && head < 2 * a.Hk, turn = !value && a.rot > 0;
  const int slot = in ? a.slots[token] : -1;
  const int pos = in && a.rot > 0 ? a.pos[token] : 0;
  bool ok = in && slot != -1;
  if (ok && (slot < 0 || slot >= a.pages * a.page || pos < 0 || (a.rot > 0 && pos >= a.angles))) {
    report(a.status, DEV_BAD_INDEX);
    ok = false;
  }
  float v[8] = {};
  if (ok) {
    const T* src = key ? static_cast<const T*>(a.K) + token * a.k_stride + (int64_t)head * a.d
                 : value ? static_cast<const T*>(a.V) + token * a.v_stride + (int64_t)(head - a.Hk) * a.d
                         : static_cast<const T*>(a.Q) + token * a.q_stride + (int64_t)(head - 2 * a.Hk) * a.d;
    load8(src + 8 * j, v);
  }
  if (a.rot > 0) {                                         // the same for the whole grid: shuffles by all lanes
    const int half = a.rot >> 4;                           // lanes of the first halves of the pairs
    const bool turned = turn && ok && 8 * j < a.rot;
    if (a.adjacent) {
      if (turned) {
        const float4 c = *reinterpret_cast<const float4*>(a.cos + (int64_t)pos * (a.rot >> 1) + 4 * j);
        const float4 s = *reinterpret_cast<const float4*>(a.sin + (int64_t)pos * (a.rot >> 1) + 4 * j);
        const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = v[2 * i], y = v[2 * i + 1];
          v[2 * i] = to_f32(from_f32<T>(__fsub_rn(__fmul_rn(x, cs[i]), __fmul_rn(y, sn[i]))));
          v[2 * i + 1] = to_f32(from_f32<T>(__fadd_rn(__fmul_rn(y, cs[i]), __fmul_rn(x, sn[i]))));
        }
      }
    } else {
      const bool first = j < half;
      const int from = sub * lanes + (8 * j < a.rot ? (first ? j + half : j - half) : j);
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __shfl_sync(0xffffffffu, v[i], from & 31);
      if (turned) {
        float cs[8], sn[8];
        const int64_t at = (int64_t)pos * (a.rot >> 1) + 8 * (first ? j : j - half);
        load8(a.cos + at, cs);
        load8(a.sin + at, sn);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = __fmul_rn(v[i], cs[i]), y = __fmul_rn(w[i], sn[i]);
          v[i] = to_f32(from_f32<T>(first ? __fsub_rn(x, y) : __fadd_rn(x, y)));
        }
      }
    }
  }
  if (BITS == 4) {                                         // d % 32 == 0: a group's four lanes are neighbours
    uint32_t pair;
    const uint32_t word = q4_encode8(v, 0xffffffffu, pair);
    if (ok && (key || value)) {
      const int p = slot / a.page, r = slot - p * a.page;
      char* at = static_cast<char*>(key ? a.keys : a.values) +
                 ((int64_t)p * a.Hk + (key ? head : head - a.Hk)) * q4_page_bytes(a.page, a.d);
      *reinterpret_cast<uint32_t*>(at + q4_code_at(r, a.d, j)) = word;
      if ((j & 3) == 0) *reinterpret_cast<uint32_t*>(at + q4_pair_at(r, a.d, a.page, j >> 2)) = pair;
    }
  } else if (ok && (key || value)) {
    const int p = slot / a.page, r = slot - p * a.page;
    store8(static_cast<T*>(key ? a.keys : a.values) +
               (((int64_t)p * a.Hk + (key ? head : head - a.Hk)) * a.page + r) * a.d + 8 * j, v);
  }
  if (ok && !key && !value)
    store8(static_cast<T*>(a.Q_out) + token * a.q_out_stride + (int64_t)(head - 2 * a.Hk) * a.d + 8 * j, v);
}

template <typename T, int BITS>
__global__ void __launch_bounds__(kThreads) read_kernel(const ReadArgs a) {
  const int lanes = a.d >> 3, per = 32 / lanes, lane = threadIdx.x & 31;
  const int sub = lane / lanes, j = lane - sub * lanes;
  const int64_t row = ((int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * per + sub;
  if (sub >= per || row >= a.rows) return;
  const int64_t token = row / (2 * a.Hk);
  const int head = (int)(row - token * (2 * a.Hk));
  const bool key = head < a.Hk;
  const int hk = key ? head : head - a.Hk, slot = a.slots[token];
  if (slot == -1) return;
  if (slot < 0 || slot >= a.pages * a.page) { report(a.status, DEV_BAD_INDEX); return; }
  const int p = slot / a.page, r = slot - p * a.page;
  const void* base = key ? a.keys : a.values;
  float v[8];
  if (BITS == 4) {
    const char* at = static_cast<const char*>(base) + ((int64_t)p * a.Hk + hk) * q4_page_bytes(a.page, a.d);
    q4_decode8(*reinterpret_cast<const uint32_t*>(at + q4_code_at(r, a.d, j)),
               *reinterpret_cast<const uint32_t*>(at + q4_pair_at(r, a.d, a.page, j >> 2)), v);
  } else {
    load8(static_cast<const T*>(base) + (((int64_t)p * a.Hk + hk) * a.page + r) * a.d + 8 * j, v);
  }
  T* out = static_cast<T*>(key ? a.K : a.V) + token * (key ? a.k_stride : a.v_stride) + (int64_t)hk * a.d;
  store8(out + 8 * j, v);
}

template <typename Kernel, typename Args>
avq_status launch_rows(Kernel kernel, const Args& a, cudaStream_t st) {
  const int64_t per = (int64_t)(kThreads / 32) * (32 / (a.d >> 3));
  kernel<<<(unsigned)((a.rows + per - 1) / per), kThreads, 0, st>>>(a);
  return cuda_ok(cudaGetLastError());
}

}  // namespace

avq_status cache_append(const AppendArgs& a, int dtype, int bits, cudaStream_t st) {
  if (dtype == AVQ_F32) return bits == 4 ? launch_rows(append_kernel<float, 4>, a, st) : launch_rows(append_kernel<float, 32>, a, st);
  return bits == 4 ? launch_rows(append_kernel<__nv_bfloat16, 4>, a, st) : launch_rows(append_kernel<__nv_bfloat16, 16>, a, st);
}
avq_status cache_read(const ReadArgs& a, int dtype, int bits, cudaStream_t st) {
  if (dtype == AVQ_F32) return bits == 4 ? launch_rows(read_kernel<float, 4>, a, st) : launch_rows(read_kernel<float, 32>, a, st);
  return bits == 4 ? launch_rows(read_kernel<__nv_bfloat16, 4>, a, st) : launch_rows(read_kernel<__nv_bfloat16, 16>, a, st);
}

}  // namespace exact
}  // namespace avq
