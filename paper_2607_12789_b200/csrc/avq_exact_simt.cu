// Exact attention on the CUDA cores: head dimensions that the tensor-core kernels do not take, and AVQ_FLAG_SIMT; and the
// kernel that joins the partial results of split sequences, whichever kernel left them.
#include <algorithm>

#include "avq_exact.cuh"
#include "avq_tc_common.cuh"

namespace avq {
namespace exact {
namespace {

using tc::f32x2;
using tc::fma2;
using tc::mul2;
using tc::pack2;
using tc::unpack2;

// ---------------------------------------------------------------- packed prompts
// A CTA takes 16 RT queries of one head over tiles of 64 keys with the running maximum and sum of the softmax.  256
// threads as 16 x 16: thread (ty, tx) owns rows ty RT.. and, of the logits, keys 4 tx.. + 3; of the output, columns
// 4 tx + 64 j.. + 3.  Q and K lie transposed in shared memory ([dimension][row]), so that each step of a product is
// two or three 16-byte loads for 4 RT multiply-adds, taken in pairs of rows (fma.rn.f32x2).  Bound by the multiply-adds and
// the loads that feed them: eight images of 785 tokens, 12 heads, d 64, float32, 540 us, 28 of the 75 TFLOP/s.
// DM: head dimensions up to DM, the rest filled with zeros.
constexpr int kPromptThreads = 256, kPromptKeys = 64;
template <int DM, int RT>
constexpr size_t prompt_smem() {
  return sizeof(float) * ((size_t)DM * 16 * RT + (size_t)DM * kPromptKeys * 2 + (size_t)kPromptKeys * 16 * RT);
}

template <typename T, int DM, int RT>
__global__ void __launch_bounds__(kPromptThreads) prompt_simt_kernel(const PromptArgs a) {
  constexpr int R = 16 * RT, KT = kPromptKeys, CJ = DM / 64;
  extern __shared__ __align__(16) float smem[];
  float* Qs = smem;                                       // [DM][R]
  float* Ks = Qs + DM * R;                                // [DM][KT]
  float* Vs = Ks + DM * KT;                               // [KT][DM]
  float* Ps = Vs + KT * DM;                               // [KT][R]
  __shared__ Piece shared_piece;
  __shared__ int found;
  if (threadIdx.x < 32) {
    Piece p;
    const bool ok = find_piece(a, R, blockIdx.x, p);
    if (threadIdx.x == 0) { found = ok; shared_piece = p; }
  }
  __syncthreads();
  if (!found) return;
  const Piece pc = shared_piece;
  const int h = blockIdx.y, hk = h / (a.H / a.Hk), d = a.d;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int rows = min(R, pc.nq - pc.first);
  const T* Q = static_cast<const T*>(a.Q) + (int64_t)(pc.q0 + pc.first) * a.q_stride + (int64_t)h * d;
  const T* K = static_cast<const T*>(a.K) + (int64_t)pc.k0 * a.k_stride + (int64_t)hk * d;
  const T* V = static_cast<const T*>(a.V) + (int64_t)pc.k0 * a.v_stride + (int64_t)hk * d;
  const float to_log2 = a.scale * kLog2e;
  for (int i = threadIdx.x; i < R * (DM / 8); i += kPromptThreads) {
    const int r = i % R, c = 8 * (i / R);
    float v[8] = {};
    if (r < rows && c < d) load8(Q + (int64_t)r * a.q_stride + c, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) Qs[(c + k) * R + r] = v[k] * to_log2;
  }
  f32x2 O[RT / 2][4 * CJ];
  float m[RT], l[RT];
#pragma unroll
  for (int r = 0; r < RT / 2; ++r)
#pragma unroll
    for (int j = 0; j < 4 * CJ; ++j) O[r][j] = 0ull;
#pragma unroll
  for (int r = 0; r < RT; ++r) { m[r] = -INFINITY; l[r] = 0.f; }
  // query i of the tile sees the keys below nk, and with `causal` those up to i + shift
  const int shift = a.causal ? pc.first + pc.nk - pc.nq : pc.nk;
  const int last = a.causal ? min(pc.nk, rows + shift) : pc.nk;
  for (int k0 = 0; k0 < last; k0 += KT) {
    __syncthreads();
    for (int i = threadIdx.x; i < KT * (DM / 8); i += kPromptThreads) {
      const int r = i % KT, c = 8 * (i / KT);
      float v[8] = {};
      if (k0 + r < pc.nk && c < d) load8(K + (int64_t)(k0 + r) * a.k_stride + c, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) Ks[(c + k) * KT + r] = v[k];
    }
    for (int i = threadIdx.x; i < KT * (DM / 8); i += kPromptThreads) {
      const int r = i / (DM / 8), c = 8 * (i % (DM / 8));
      float v[8] = {};
      if (k0 + r < pc.nk && c < d) load8(V + (int64_t)(k0 + r) * a.v_stride + c, v);
      store8(Vs + r * DM + c, v);
    }
    __syncthreads();
    f32x2 s2[RT / 2][4];
#pragma unroll
    for (int r = 0; r < RT / 2; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c) s2[r][c] = 0ull;
#pragma unroll 4
    for (int k = 0; k < DM; ++k) {
      const float4 kv = *reinterpret_cast<const float4*>(Ks + k * KT + 4 * tx);
      const f32x2 kk[4] = {pack2(kv.x, kv.x), pack2(kv.y, kv.y), pack2(kv.z, kv.z), pack2(kv.w, kv.w)};
#pragma unroll
      for (int r = 0; r < RT / 2; r += 2) {
        const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(Qs + k * R + ty * RT + 2 * r);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s2[r][c] = fma2(q.x, kk[c], s2[r][c]);
          s2[r + 1][c] = fma2(q.y, kk[c], s2[r + 1][c]);
        }
      }
    }
    const bool edge = k0 + KT > pc.nk || (a.causal && k0 + KT > shift + 1);
    float s[RT][4];
#pragma unroll
    for (int r = 0; r < RT / 2; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c) unpack2(s2[r][c], s[2 * r][c], s[2 * r + 1][c]);
    if (edge) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int j = k0 + 4 * tx + c;
          if (j >= pc.nk || (a.causal && j > ty * RT + r + shift)) s[r][c] = -INFINITY;
        }
    }
    float f[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float t = fmaxf(fmaxf(s[r][0], s[r][1]), fmaxf(s[r][2], s[r][3]));
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
      t = fmaxf(t, m[r]);
      const float use = t == -INFINITY ? 0.f : t;
      f[r] = exp2f(m[r] - use);
      m[r] = t;
      float z = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) { s[r][c] = exp2f(s[r][c] - use); z += s[r][c]; }
      l[r] = l[r] * f[r] + z;                              // this thread's columns; the 16 are added at the end
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int r = 0; r < RT; r += 4)
        *reinterpret_cast<float4*>(Ps + (4 * tx + c) * R + ty * RT + r) = make_float4(s[r][c], s[r + 1][c], s[r + 2][c], s[r + 3][c]);
#pragma unroll
    for (int r = 0; r < RT / 2; ++r) {
      const f32x2 ff = pack2(f[2 * r], f[2 * r + 1]);
#pragma unroll
      for (int j = 0; j < 4 * CJ; ++j) O[r][j] = mul2(O[r][j], ff);
    }
    __syncwarp();                                          // a row's weights come from the 16 lanes that read them
    const int keys = min(KT, last - k0);
    if (!edge) {
#pragma unroll 2
      for (int k = 0; k < KT; ++k) {
        ulonglong2 p[RT / 4];
#pragma unroll
        for (int r = 0; r < RT / 4; ++r) p[r] = *reinterpret_cast<const ulonglong2*>(Ps + k * R + ty * RT + 4 * r);
#pragma unroll
        for (int j = 0; j < CJ; ++j) {
          const float4 v = *reinterpret_cast<const float4*>(Vs + k * DM + 4 * tx + 64 * j);
          const f32x2 vv[4] = {pack2(v.x, v.x), pack2(v.y, v.y), pack2(v.z, v.z), pack2(v.w, v.w)};
#pragma unroll
          for (int r = 0; r < RT / 4; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              O[2 * r][4 * j + c] = fma2(p[r].x, vv[c], O[2 * r][4 * j + c]);
              O[2 * r + 1][4 * j + c] = fma2(p[r].y, vv[c], O[2 * r + 1][4 * j + c]);
            }
        }
      }
    } else {
      // a weight of zero takes no value, so that what a masked key holds (an infinity, a NaN) stays out of the row
      for (int k = 0; k < keys; ++k)
#pragma unroll
        for (int r = 0; r < RT / 2; ++r) {
          const float2 p = *reinterpret_cast<const float2*>(Ps + k * R + ty * RT + 2 * r);
          const f32x2 pp = pack2(p.x, p.y);
#pragma unroll
          for (int j = 0; j < 4 * CJ; ++j) {
            const float v = Vs[k * DM + 4 * tx + 64 * (j >> 2) + (j & 3)];
            O[r][j] = fma2(pp, pack2(p.x == 0.f ? 0.f : v, p.y == 0.f ? 0.f : v), O[r][j]);
          }
        }
    }
  }
#pragma unroll
  for (int r = 0; r < RT; ++r) {
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], o);
    const int row = ty * RT + r;
    if (row >= rows) continue;
    const int64_t token = pc.q0 + pc.first + row;
    const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
    T* Y = static_cast<T*>(a.Y) + token * a.y_stride + (int64_t)h * d;
#pragma unroll
    for (int j = 0; j < CJ; ++j) {
      const int c = 4 * tx + 64 * j;
      if (c >= d) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float lo, hi;
        unpack2(O[r >> 1][4 * j + i], lo, hi);
        Y[c + i] = from_f32<T>(((r & 1) ? hi : lo) * inv);
      }
    }
    if (a.lse && tx == 0) a.lse[token * a.H + h] = l[r] == 0.f ? -INFINITY : (m[r] + log2f(l[r])) * kLn2;
  }
}

template <typename T, int DM, int RT>
avq_status launch_prompt(const PromptArgs& a, int dev, cudaStream_t st) {
  avq_status s = open_shared_memory<prompt_simt_kernel<T, DM, RT>>(dev);
  if (s != AVQ_OK) return s;
  const dim3 grid((unsigned)most_pieces(a.Tq, a.S, 16 * RT), a.H);
  prompt_simt_kernel<T, DM, RT><<<grid, kPromptThreads, prompt_smem<DM, RT>(), st>>>(a);
  return cuda_ok(cudaGetLastError());
}

// ---------------------------------------------------------------- cached sequences
// A CTA walks its run of units (avq_exact.cuh), 32 tokens of a segment at a time: their keys and values go to shared
// memory as float32, every (row, token) pair's logit is one thread's, weights and running maxima are a warp's per row,
// and a thread owns output columns.  The kernel for the shapes that no other takes: 64 sequences over a bfloat16 cache at
// d 128 1454 us, where the tensor-core kernel takes 78.5.
constexpr int kCachedThreads = 128, kCachedTokens = 32;
inline size_t cached_smem(int d) {
  return sizeof(float) * ((size_t)kRows * d + (size_t)kCachedTokens * (2 * d + 4) + kRows * kCachedTokens + 3 * kRows);
}

template <typename T, int BITS>
__global__ void __launch_bounds__(kCachedThreads) cached_simt_kernel(const CachedArgs a, int least) {
  extern __shared__ __align__(16) float smem[];
  const int d = a.d, kd = d + 4, G = a.H / a.Hk;
  float* Qs = smem;                                        // [kRows][d]
  float* Ks = Qs + kRows * d;                              // [tokens][d + 4]
  float* Vs = Ks + kCachedTokens * kd;                     // [tokens][d]
  float* Ps = Vs + kCachedTokens * d;                      // [kRows][tokens]
  float* ms = Ps + kRows * kCachedTokens;
  float* ls = ms + kRows;
  float* fs = ls + kRows;
  __shared__ Walk walk;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  Segment sg;
  int turn = 0;
  for (bool more = walk_begin(a, least, walk, sg); more; more = walk_next(a, walk, sg, ++turn)) {
    const int rows = min(kRows, a.nq * G - sg.block * kRows);
    __syncthreads();
    for (int i = tid; i < rows * (d / 8); i += kCachedThreads) {
      const int r = i / (d / 8), c = 8 * (i % (d / 8)), q = sg.block * kRows + r;
      float v[8];
      load8(static_cast<const T*>(a.Q) + ((int64_t)sg.b * a.nq + q / G) * a.q_stride + ((int64_t)sg.hk * G + q % G) * d + c, v);
      store8(Qs + r * d + c, v);
    }
    if (tid < kRows) { ms[tid] = -INFINITY; ls[tid] = 0.f; }
    float O[kRows][2] = {};
    const int end = min(sg.len, (sg.unit + sg.n) * kUnit);
    for (int t0 = sg.unit * kUnit; t0 < end; t0 += kCachedTokens) {
      __syncthreads();
      for (int i = tid; i < 2 * kCachedTokens * (d / 8); i += kCachedThreads) {
        const bool value = i >= kCachedTokens * (d / 8);
        const int e = value ? i - kCachedTokens * (d / 8) : i;
        const int r = e / (d / 8), c = e % (d / 8), t = t0 + r;
        float v[8] = {};
        const int page = t < end ? page_of(a, sg.b, t) : -1;
        if (page >= 0) {
          const void* base = value ? a.values : a.keys;
          const int row = t % a.page;
          if (BITS == 4) {
            const char* at = static_cast<const char*>(base) + ((int64_t)page * a.Hk + sg.hk) * q4_page_bytes(a.page, d);
            q4_decode8(*reinterpret_cast<const uint32_t*>(at + q4_code_at(row, d, c)),
                       *reinterpret_cast<const uint32_t*>(at + q4_pair_at(row, d, a.page, c >> 2)), v);
          } else {
            load8(static_cast<const T*>(base) + (((int64_t)page * a.Hk + sg.hk) * a.page + row) * d + 8 * c, v);
          }
        }
        store8((value ? Vs + r * d : Ks + r * kd) + 8 * c, v);
      }
      __syncthreads();
      for (int i = tid; i < rows * kCachedTokens; i += kCachedThreads) {
        const int r = i / kCachedTokens, t = i % kCachedTokens;
        float s = 0.f;
        for (int c = 0; c < d; c += 4) {
          const float4 q = *reinterpret_cast<const float4*>(Qs + r * d + c);
          const float4 k = *reinterpret_cast<const float4*>(Ks + t * kd + c);
          s = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, s))));
        }
        const int seen = sg.len - a.nq + (sg.block * kRows + r) / G + 1;
        const bool ok = t0 + t < min(seen, end) && page_of(a, sg.b, t0 + t) >= 0;
        Ps[r * kCachedTokens + t] = ok ? s * (a.scale * kLog2e) : -INFINITY;
      }
      __syncthreads();
      for (int r = warp; r < rows; r += kCachedThreads / 32) {
        const float s = Ps[r * kCachedTokens + lane], old = ms[r];
        float t = s;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
        t = fmaxf(t, old);
        const float use = t == -INFINITY ? 0.f : t;
        const float p = exp2f(s - use);
        float z = p;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        Ps[r * kCachedTokens + lane] = p;
        if (lane == 0) {
          fs[r] = exp2f(old - use);
          ms[r] = t;
          ls[r] = ls[r] * fs[r] + z;
        }
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int c = tid + kCachedThreads * j;
        if (c >= d) continue;
#pragma unroll
        for (int r = 0; r < kRows; ++r)
          if (r < rows) O[r][j] *= fs[r];
        for (int t = 0; t < kCachedTokens; ++t) {
          const float v = Vs[t * d + c];
#pragma unroll
          for (int r = 0; r < kRows; ++r)
            if (r < rows) {
              const float p = Ps[r * kCachedTokens + t];
              if (p != 0.f) O[r][j] = fmaf(p, v, O[r][j]);   // (a masked token's value may be anything)
            }
        }
      }
    }
    __syncthreads();
    float* slot = segment_slot(a, sg);
    for (int r = 0; r < rows; ++r) {
      const int q = sg.block * kRows + r;
      const int64_t token = (int64_t)sg.b * a.nq + q / G;
      const int h = sg.hk * G + q % G;
      float o[2];
#pragma unroll
      for (int k = 0; k < kRows; ++k)                      // (a register array has no run-time index)
        if (k == r) { o[0] = O[k][0]; o[1] = O[k][1]; }
      if (slot) {
        // (a share that met nothing but NaN has raised no maximum: it must not pass for one that saw no token)
        if (tid == 0) { slot[r] = ls[r] == ls[r] ? ms[r] : ls[r]; slot[kRows + r] = ls[r]; }
      } else if (a.lse && tid == 0) {
        a.lse[token * a.H + h] = ls[r] == 0.f ? -INFINITY : (ms[r] + log2f(ls[r])) * kLn2;
      }
      const float inv = ls[r] == 0.f ? 0.f : 1.f / ls[r];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int c = tid + kCachedThreads * j;
        if (c >= d) continue;
        if (slot) slot[2 * kRows + r * d + c] = o[j];
        else static_cast<T*>(a.Y)[token * a.y_stride + (int64_t)h * d + c] = from_f32<T>(o[j] * inv);
      }
    }
  }
}

// ---------------------------------------------------------------- joining partial results
// One CTA per row of a segment: nothing to do if one CTA held the whole segment; zeros if the sequence is empty;
// otherwise the partial rows of CTAs c0 .. c1 are brought to their common maximum and added, each warp a share of them in
// ascending order, the warps' sums in the order of the warps.
// Threads of a row's CTA: two warps where segments are many (and parts of each few), eight where they are few (their parts
// many).  64 and 256 threads, with the kernel before, 4096 tokens of bfloat16 a segment: 8 segments 12.3 and 10.2 us, 24 13.6
// and 13.0, 48 17.5 and 17.4, 64 28.6 and 28.8, 96 38.8 and 38.7, 128 49.9 and 51.4, 512 167 and 171; in 4 bits 13.1 and 11.1,
// 15.7 and 15.0, 19.2 and 19.1, 21.5 and 21.5, 26.5 and 26.7, 31.8 and 34.1, 96 and 102.
constexpr int kJoinMost = 256, kJoinFew = 64, kJoinMany = 128;
template <typename T>
__global__ void __launch_bounds__(kJoinMost) join_kernel(const CachedArgs a) {
  const int threads = blockDim.x, warps = threads >> 5;
  __shared__ float sums[kJoinMost / 32][256 + 1];
  tc::pdl_wait();                                          // records and slots come from the kernel before
  const int G = a.H / a.Hk, per = segments_per_sequence(a), blocks = per / a.Hk;
  const int b = blockIdx.x / per, seg = blockIdx.x % per;
  const int hk = seg / blocks, block = seg % blocks, r = blockIdx.y;
  const int q = block * kRows + r;
  if (q >= a.nq * G) return;
  const int32_t* record = reinterpret_cast<const int32_t*>(a.records + blockIdx.x);
  const int c0 = tc::ld_after_wait(record), c1 = tc::ld_after_wait(record + 1);   // (of an empty sequence: anything)
  const int U = units_of(clipped_len(a, b, false));
  const int64_t token = (int64_t)b * a.nq + q / G;
  const int h = hk * G + q % G, d = a.d;
  T* Y = static_cast<T*>(a.Y) + token * a.y_stride + (int64_t)h * d;
  if (U == 0) {
    for (int c = threadIdx.x; c < d; c += threads) Y[c] = from_f32<T>(0.f);
    if (a.lse && threadIdx.x == 0) a.lse[token * a.H + h] = -INFINITY;
    return;
  }
  if (c0 < 0) return;
  const int64_t size = slot_floats(d);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = c1 - c0 + 1;
  auto slot = [&](int i) { return a.partial + (int64_t)(2 * (c0 + i) + (i == 0)) * size; };
  float m = -INFINITY;
  for (int i = lane; i < n; i += 32) m = fmaxf(m, tc::ld_after_wait(slot(i) + r));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float use = m == -INFINITY ? 0.f : m;
  float l = 0.f, x[8] = {};                                // columns lane + 32 j
  // a batch of partial rows per turn, all its loads in flight together
  constexpr int kBatch = 4;
  for (int i0 = warp; i0 < n; i0 += kBatch * warps) {
    float top[kBatch], sum[kBatch], part[kBatch][8];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int i = i0 + k * warps;
      top[k] = -INFINITY;
      sum[k] = 0.f;
      if (i >= n) continue;
      const float* s = slot(i);
      top[k] = tc::ld_after_wait(s + r);
      sum[k] = tc::ld_after_wait(s + kRows + r);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (lane + 32 * j < d) part[k][j] = tc::ld_after_wait(s + 2 * kRows + r * d + lane + 32 * j);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const float w = exp2f(top[k] - use);
      if (w == 0.f) continue;
      l = fmaf(w, sum[k], l);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (lane + 32 * j < d) x[j] = fmaf(w, part[k][j], x[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) sums[warp][lane + 32 * j] = x[j];
  if (lane == 0) sums[warp][256] = l;
  __syncthreads();
  l = 0.f;
  for (int w = 0; w < warps; ++w) l += sums[w][256];
  const float inv = l == 0.f ? 0.f : 1.f / l;
  for (int c = threadIdx.x; c < d; c += threads) {
    float y = 0.f;
    for (int w = 0; w < warps; ++w) y += sums[w][c];
    Y[c] = from_f32<T>(y * inv);
  }
  if (a.lse && threadIdx.x == 0) a.lse[token * a.H + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace

avq_status simt_prompt(const PromptArgs& a, int dtype, cudaStream_t st) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return AVQ_ERR_CUDA;
  if (dtype == AVQ_F32)
    return a.d <= 64 ? launch_prompt<float, 64, 8>(a, dev, st)
         : a.d <= 128 ? launch_prompt<float, 128, 8>(a, dev, st) : launch_prompt<float, 256, 4>(a, dev, st);
  return a.d <= 64 ? launch_prompt<__nv_bfloat16, 64, 8>(a, dev, st)
       : a.d <= 128 ? launch_prompt<__nv_bfloat16, 128, 8>(a, dev, st) : launch_prompt<__nv_bfloat16, 256, 4>(a, dev, st);
}

avq_status join(const CachedArgs& a, int dtype, cudaStream_t st) {
  const int G = a.H / a.Hk;
  const dim3 grid((unsigned)((int64_t)a.B * a.Hk * ((a.nq * G + kRows - 1) / kRows)), (unsigned)std::min(kRows, a.nq * G));
  const dim3 block(grid.x >= kJoinMany ? kJoinFew : kJoinMost);
  return cuda_ok(dtype == AVQ_F32 ? tc::launch_pdl(join_kernel<float>, grid, block, 0, st, true, a)
                                  : tc::launch_pdl(join_kernel<__nv_bfloat16>, grid, block, 0, st, true, a));
}

namespace {
template <typename T, int BITS>
avq_status launch_cached(const CachedArgs& a, int dtype, cudaStream_t st) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return AVQ_ERR_CUDA;
  avq_status s = open_shared_memory<cached_simt_kernel<T, BITS>>(dev);
  if (s != AVQ_OK) return s;
  constexpr int ctas = 148 * 2, least = 4;
  cached_simt_kernel<T, BITS><<<ctas, kCachedThreads, cached_smem(a.d), st>>>(a, least);
  s = cuda_ok(cudaGetLastError());
  return s == AVQ_OK ? join(a, dtype, st) : s;
}
}  // namespace

avq_status simt_cached(const CachedArgs& a, int dtype, int bits, cudaStream_t st) {
  if (dtype == AVQ_F32) return bits == 4 ? launch_cached<float, 4>(a, dtype, st) : launch_cached<float, 32>(a, dtype, st);
  return bits == 4 ? launch_cached<__nv_bfloat16, 4>(a, dtype, st) : launch_cached<__nv_bfloat16, 16>(a, dtype, st);
}

}  // namespace exact
}  // namespace avq
