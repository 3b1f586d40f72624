// Exact attention of packed float32 sequences on the tensor cores (d 64 or 128): every product as three tf32 products of
// the operands' high and low parts (the product of the two low parts, 2^-22 of a term, is left out), float32 sums.
//
// 4 warps, 16 MT rows of one head each, over tiles of 32 keys.  Queries, keys and values lie in shared memory as they are,
// swizzled, and are taken apart in registers: a 16-byte load gives a lane 4 dimensions, which serve as the k indices of two
// steps of Q K^T (the order of dimensions within a sum is free, as long as both operands have the same) or as the columns
// of four tiles of P V.  The weights stay in the registers that the logits came in: key 2 t of a tile of 8 is index t of
// the next product's sum, key 2 t + 1 index t + 4.  The next tile's copies (cp.async) run under the products.
// Bound by the products, three of each, whose sums the tensor cores cut off instead of rounding: the low parts' products have
// sums of their own in Q K^T, a tile's P V is summed from zero and added in registers (all in one chain: 6.7e-6 of the result
// off instead of 5.9e-7; only the first of the two left out: 1.1e-6).  Eight images of 785 tokens, 12 heads, d 64: 372 us, of
// the CUDA cores 540; with one row tile to a warp as much, with three CTAs to an SM, whose registers do not hold the sums, 20 more.
// 5 of it are for infinities: logits that their parts make a NaN are taken again from the rows (one branch for a tile: one for each
// row of it cost 29), and the low part of a weight is never zero.
#include "avq_exact_mma.cuh"

namespace avq {
namespace exact {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps, kKeys = 32;
template <int D> __host__ __device__ constexpr int row_tiles() { return D == 64 ? 2 : 1; }
template <int D> __host__ __device__ constexpr int tile_rows() { return 16 * kWarps * row_tiles<D>(); }
template <int D> __host__ __device__ constexpr size_t f32_smem() { return sizeof(float) * D * (tile_rows<D>() + 4 * kKeys); }

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
// High and low parts of four values.
__device__ __forceinline__ void apart(const uint4& x, uint32_t (&hi)[4], uint32_t (&lo)[4]) {
  const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float f = __uint_as_float(v[i]), h = tf32_high(f);
    hi[i] = __float_as_uint(h);
    lo[i] = tf32_low(f, h);
  }
}

// The product of rows qr and kr as they lie in shared memory, in float32.
template <int D>
__device__ __forceinline__ float plain_product(uint32_t qs, int qr, uint32_t kt, int kr) {
  float s = 0.f;
#pragma unroll 1
  for (int c = 0; c < D / 4; ++c) {
    const uint4 x = lds128(qs + qr * 4 * D + 16 * (c ^ swizzle(qr))), y = lds128(kt + kr * 4 * D + 16 * (c ^ swizzle(kr)));
    s = fmaf(__uint_as_float(x.x), __uint_as_float(y.x), s);
    s = fmaf(__uint_as_float(x.y), __uint_as_float(y.y), s);
    s = fmaf(__uint_as_float(x.z), __uint_as_float(y.z), s);
    s = fmaf(__uint_as_float(x.w), __uint_as_float(y.w), s);
  }
  return s;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2) prompt_f32_kernel(const PromptArgs a) {
  constexpr int MT = row_tiles<D>(), R = tile_rows<D>(), kChunks = D / 4, kRow = 4 * D;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ Piece shared_piece;
  __shared__ int found;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  if (warp == 0) {
    Piece p;
    const bool ok = find_piece(a, R, blockIdx.x, p);
    if (lane == 0) { found = ok; shared_piece = p; }
  }
  __syncthreads();
  if (!found) return;
  const Piece pc = shared_piece;
  const int h = blockIdx.y, hk = h / (a.H / a.Hk), rows = min(R, pc.nq - pc.first);
  const uint32_t qs = tc::smem_u32(smem), ks = qs + R * kRow, vs = ks + 2 * kKeys * kRow;
  const float* Q = static_cast<const float*>(a.Q) + (int64_t)(pc.q0 + pc.first) * a.q_stride + (int64_t)h * D;
  const float* K = static_cast<const float*>(a.K) + (int64_t)pc.k0 * a.k_stride + (int64_t)hk * D;
  const float* V = static_cast<const float*>(a.V) + (int64_t)pc.k0 * a.v_stride + (int64_t)hk * D;
  // query i of the tile sees the keys below nk, and with `causal` those up to i + shift
  const int shift = a.causal ? pc.first + pc.nk - pc.nq : pc.nk;
  const int last = a.causal ? min(pc.nk, rows + shift) : pc.nk, tiles = last > 0 ? (last + kKeys - 1) / kKeys : 0;
  auto fetch = [&](int j) {
    const uint32_t at = (j & 1) * kKeys * kRow;
#pragma unroll
    for (int i0 = 0; i0 < kKeys * kChunks; i0 += kThreads) {
      const int i = i0 + threadIdx.x, r = i / kChunks, c = i % kChunks, key = j * kKeys + r;
      const bool there = key < pc.nk;
      const uint32_t dst = at + r * kRow + 16 * (c ^ swizzle(r));
      cp_async16_or_zero(ks + dst, K + (there ? (int64_t)key * a.k_stride + 4 * c : 0), there);
      cp_async16_or_zero(vs + dst, V + (there ? (int64_t)key * a.v_stride + 4 * c : 0), there);
    }
  };
  if (tiles > 0) {
    for (int i = threadIdx.x; i < R * kChunks; i += kThreads) {
      const int r = i / kChunks, c = i % kChunks;
      cp_async16_or_zero(qs + r * kRow + 16 * (c ^ swizzle(r)), Q + (r < rows ? (int64_t)r * a.q_stride + 4 * c : 0), r < rows);
    }
    fetch(0);
  }
  cp_async_commit();
  float O[MT][D / 8][4], m[MT][2], l[MT][2];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) O[i][n][e] = 0.f;
    m[i][0] = m[i][1] = -INFINITY;
    l[i][0] = l[i][1] = 0.f;
  }
  const float to_log2 = a.scale * kLog2e;
  int wide_from = 0x7fffffff;                              // first key of the first tile with such values
  for (int j = 0; j < tiles; ++j) {
    cp_async_wait<0>();
    __syncthreads();
    if (j + 1 < tiles) fetch(j + 1);
    cp_async_commit();
    const uint32_t kt = ks + (j & 1) * kKeys * kRow, vt = vs + (j & 1) * kKeys * kRow;
    float s[MT][kKeys / 8][4], low[MT][kKeys / 8][4];      // sums of the high parts' products, of the others
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int n = 0; n < kKeys / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][n][e] = low[i][n][e] = 0.f;
#pragma unroll 2
    for (int c = 0; c < D / 16; ++c) {
      uint32_t qh[MT][2][4], ql[MT][2][4];                 // [row tile][row g, g + 8][dimension]
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int r = 16 * (MT * warp + i) + g + 8 * x;
          apart(lds128(qs + r * kRow + 16 * ((4 * c + t) ^ swizzle(r))), qh[i][x], ql[i][x]);
        }
#pragma unroll
      for (int n = 0; n < kKeys / 8; ++n) {
        const int r = 8 * n + g;
        uint32_t kh[4], kl[4];
        apart(lds128(kt + r * kRow + 16 * ((4 * c + t) ^ swizzle(r))), kh, kl);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            const uint32_t ah[4] = {qh[i][0][2 * k], qh[i][1][2 * k], qh[i][0][2 * k + 1], qh[i][1][2 * k + 1]};
            const uint32_t al[4] = {ql[i][0][2 * k], ql[i][1][2 * k], ql[i][0][2 * k + 1], ql[i][1][2 * k + 1]};
            mma_tf32(low[i][n], al, kh[2 * k], kh[2 * k + 1]);
            mma_tf32(low[i][n], ah, kl[2 * k], kl[2 * k + 1]);
            mma_tf32(s[i][n], ah, kh[2 * k], kh[2 * k + 1]);
          }
      }
    }
    const int k0 = j * kKeys;
    const bool edge = k0 + kKeys > pc.nk || (a.causal && k0 + kKeys > shift + 1);
    float tops[MT][2], all = -INFINITY;                    // NaN if any logit of the row, of this lane is
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int row = 16 * (MT * warp + i) + g + 8 * x;
        tops[i][x] = -INFINITY;
#pragma unroll
        for (int n = 0; n < kKeys / 8; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float& v = s[i][n][2 * x + e];
            v = (v + low[i][n][2 * x + e]) * to_log2;
            if (edge) {
              const int key = k0 + 8 * n + 2 * t + e;
              if (key >= pc.nk || (a.causal && key > row + shift)) v = -INFINITY;
            }
            tops[i][x] = max_nan(tops[i][x], v);
          }
        all = max_nan(all, tops[i][x]);
      }
    if (all != all) {
      // The parts of an infinity can make a NaN of a logit that is none: such logits once more, from the rows themselves.
      // (A row that has had a NaN keeps it.)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          tops[i][x] = -INFINITY;
#pragma unroll
          for (int n = 0; n < kKeys / 8; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& v = s[i][n][2 * x + e];
              if (v != v && l[i][x] == l[i][x])
                v = plain_product<D>(qs, 16 * (MT * warp + i) + g + 8 * x, kt, 8 * n + 2 * t + e) * to_log2;
              tops[i][x] = fmaxf(tops[i][x], v);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float top = tops[i][x];
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        top = fmaxf(top, m[i][x]);
        const float use = top == -INFINITY ? 0.f : top, f = ex2(m[i][x] - use);
        m[i][x] = top;
        float z = 0.f;
#pragma unroll
        for (int n = 0; n < kKeys / 8; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float& v = s[i][n][2 * x + e];
            v = ex2(v - use);
            z += v;
          }
        l[i][x] = l[i][x] * f + z;                         // this lane's keys; the four lanes are added at the end
#pragma unroll
        for (int n = 0; n < D / 8; ++n) { O[i][n][2 * x] *= f; O[i][n][2 * x + 1] *= f; }
      }
    if (edge) {
      // Not every row sees every key: an infinity or a NaN among the values must not meet a weight of zero.  It becomes zero
      // here, and is added at the end to the rows that do see it.
      bool wide = false;
      for (int i = threadIdx.x; i < kKeys * kChunks; i += kThreads) {
        const uint4 v = lds128(vt + 16 * i);
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
        bool odd = false;
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (!isfinite(__uint_as_float(w[q]))) { odd = true; w[q] = 0u; }
        if (odd) asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(vt + 16 * i), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
        wide |= odd;
      }
      if (__syncthreads_or(wide)) wide_from = min(wide_from, k0);
    }
    // A tile's values are summed from zero, 32 columns at a time, and added to the output in registers: the tensor cores cut
    // sums off, which over all tiles was 6.7e-6 of the result.
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      float part[MT][4][4];
#pragma unroll
      for (int n = 0; n < kKeys / 8; ++n) {
        uint32_t ph[MT][4], pl[MT][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float p = s[i][n][(q & 1) * 2 + (q >> 1)], hi = tf32_high(p);   // rows g, g + 8 of key r, then of key r + 1
            ph[i][q] = __float_as_uint(hi);
            pl[i][q] = tf32_low_weight(p, hi);
          }
        const int r = 8 * n + 2 * t;                       // keys r and r + 1
        uint32_t xh[4], xl[4], yh[4], yl[4];
        apart(lds128(vt + r * kRow + 16 * ((8 * c + g) ^ swizzle(r))), xh, xl);
        apart(lds128(vt + (r + 1) * kRow + 16 * ((8 * c + g) ^ swizzle(r + 1))), yh, yl);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            if (n == 0) mma_tf32_first(part[i][q], pl[i], xh[q], yh[q]);
            else mma_tf32(part[i][q], pl[i], xh[q], yh[q]);
            mma_tf32(part[i][q], ph[i], xl[q], yl[q]);
            mma_tf32(part[i][q], ph[i], xh[q], yh[q]);
          }
      }
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) O[i][4 * c + q][e] += part[i][q][e];
    }
  }
  cp_async_wait<0>();
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float z = l[i][x];
      z += __shfl_xor_sync(0xffffffffu, z, 1);
      z += __shfl_xor_sync(0xffffffffu, z, 2);
      const int row = 16 * (MT * warp + i) + g + 8 * x;
      if (row >= rows) continue;
      const int64_t token = pc.q0 + pc.first + row;
      const float inv = z == 0.f ? 0.f : 1.f / z;
#pragma unroll
      for (int n = 0; n < D / 8; ++n) { O[i][n][2 * x] *= inv; O[i][n][2 * x + 1] *= inv; }
      const int sees = a.causal ? min(pc.nk, row + shift + 1) : pc.nk;
      for (int key = wide_from; key < sees; ++key) {
        const float* v = V + (int64_t)key * a.v_stride + 8 * t;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
          for (int q = 0; q < 8; ++q)
            if (!isfinite(v[32 * c + q])) O[i][4 * c + (q & 3)][2 * x + (q >> 2)] += v[32 * c + q];
      }
      float* Y = static_cast<float*>(a.Y) + token * a.y_stride + (int64_t)h * D + 8 * t;
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          *reinterpret_cast<float4*>(Y + 32 * c + 4 * e) = make_float4(O[i][4 * c][2 * x + e], O[i][4 * c + 1][2 * x + e],
                                                                     O[i][4 * c + 2][2 * x + e], O[i][4 * c + 3][2 * x + e]);
      if (a.lse && t == 0) a.lse[token * a.H + h] = z == 0.f ? -INFINITY : (m[i][x] + log2f(z)) * kLn2;
    }
}

template <int D>
avq_status launch(const PromptArgs& a, cudaStream_t st) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return AVQ_ERR_CUDA;
  const avq_status s = open_shared_memory<prompt_f32_kernel<D>>(dev);
  if (s != AVQ_OK) return s;
  prompt_f32_kernel<D><<<dim3((unsigned)most_pieces(a.Tq, a.S, tile_rows<D>()), a.H), kThreads, f32_smem<D>(), st>>>(a);
  return cuda_ok(cudaGetLastError());
}

}  // namespace

avq_status tc_prompt_f32(const PromptArgs& a, cudaStream_t st) { return a.d == 64 ? launch<64>(a, st) : launch<128>(a, st); }

}  // namespace exact
}  // namespace avq
