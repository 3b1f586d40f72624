// Exact attention of packed bfloat16 sequences on the tensor cores (d 64 or 128).
//
//   S = Q K^T,  P = exp(scale (S - m)),  O += P V,  l += sum P,  Y = O / l     over tiles of 128 keys
//
// A CTA takes two tiles of 128 rows of one key head: the H/Hk query heads that share it are rows of one tile, (query,
// head) with the head fastest, so that a tile of keys and values is read once for all of them and a short sequence fills
// the rows that it can.  Roles by warp:
//   0-3, 4-7  one tile each, a thread per row: logits out of tensor memory, maximum, weights back as bfloat16 in their
//             place, sum; at the end the outputs out of tensor memory
//   8         loads (TMA): the two tiles of queries, then keys and values in turn through a ring
//   9         issues every tcgen05.mma: S of one tile while the other tile's weights are being computed
//   10, 11    clean the value tiles that not every row sees whole: rows behind the last key become zero (they are
//             another sequence's), infinities and NaN too (a weight of zero times one of them would be NaN); the
//             latter are added back at the end to the rows that do see them
// Bound: per pair of tiles of 128 keys (d = 128) the products take 2048 cycles of the tensor pipe, the 32768
// exponentials as many of the MUFU pipe; so a share of them is computed by a polynomial on the FMA pipe (kPolyOf8).
// The maximum that weights refer to is raised only when a row exceeds it by 2^8, which spares nearly every rescaling of
// O: weights stay below 2^8, and what they are relative to cancels in O / l.
#include "avq_exact.cuh"
#include "avq_tc_common.cuh"

namespace avq {
namespace exact {
namespace {

using namespace tc;

constexpr int kTile = 128, kThreads = 384, kLoader = 8, kIssuer = 9, kGuards = 64;
constexpr int kMost = 96;                                  // weights of a tile that the product starts with
constexpr int kReady = 8;                                  // value tiles that the guards can be ahead by, at least
constexpr float kRaise = 8.f;
constexpr int kFewRegs = 80, kManyRegs = 208;              // per thread of warps 8-11, of warps 0-7
template <int D> __host__ __device__ constexpr int ring_slots() { return D == 128 ? 5 : 10; }
template <int D> __host__ __device__ constexpr int tile_bytes() { return kTile * D * 2; }
template <int D> __host__ __device__ constexpr size_t prompt_smem() { return 1024 + (size_t)(2 + ring_slots<D>()) * tile_bytes<D>(); }

struct Shared {
  uint64_t q_full, full[10], empty[10], raw[kReady], cleaned[kReady], s_full[2], p_most[2], p_ready[2], done[2], drained;
  Piece piece;
  uint32_t tmem;
  int found, abort_flag, wide;
};

__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// 32 columns of this thread's row; the registers are not valid before tmem_wait.
__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, "
      "%25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]),
                      "+r"(r[i + 7])::"memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t at, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, "
      "%25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]),
      "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
      "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
      "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
      "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
      "r"(r[14]), "r"(r[15]), "r"(at)
      : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// NaN if any of the three is.
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// 2^x of two values up to 2^8 on the FMA pipe: the nearest integer n by adding 1.5 * 2^23, 2^(x - n) on [-1/2, 1/2] by a
// polynomial of degree 3 fitted for the smallest largest relative error (7.5e-5; the weights are rounded to bfloat16,
// 3.9e-3, next), n added to the exponent.  Below -126: 2^-126.  A NaN gives anything: its row's maximum is NaN too.
__device__ __forceinline__ void poly_ex2(f32x2 x, float& lo, float& hi) {
  float a, b;
  unpack2(x, a, b);
  x = pack2(fmaxf(a, -126.f), fmaxf(b, -126.f));
  const f32x2 magic = pack2(12582912.f, 12582912.f), minus = pack2(-12582912.f, -12582912.f), neg = pack2(-1.f, -1.f);
  const f32x2 n = add2(x, magic), f = fma2(add2(n, minus), neg, x);
  f32x2 y = fma2(f, pack2(0.0551716685f, 0.0551716685f), pack2(0.242611125f, 0.242611125f));
  y = fma2(y, f, pack2(0.693260968f, 0.693260968f));
  y = fma2(y, f, pack2(0.999928057f, 0.999928057f));
  float n0, n1, y0, y1;
  unpack2(n, n0, n1);
  unpack2(y, y0, y1);
  lo = __uint_as_float(__float_as_uint(y0) + (__float_as_uint(n0) << 23));
  hi = __uint_as_float(__float_as_uint(y1) + (__float_as_uint(n1) << 23));
}
constexpr int kPolyOf8 = 2;                                // pairs of 8 whose exponentials the polynomial computes

// What is added to scale * logit, in powers of two: an infinite or NaN maximum makes every weight of the row NaN.
__device__ __forceinline__ float reference(float m, float c) {
  return m == -INFINITY ? 0.f : isfinite(m) ? -m * c : __int_as_float(0x7fffffff);
}
__device__ __forceinline__ float row_max(const uint32_t (&s)[4][32]) {
  float top[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    top[q] = max3_nan(__uint_as_float(s[q][0]), __uint_as_float(s[q][1]), __uint_as_float(s[q][31]));
#pragma unroll
    for (int k = 2; k + 1 < 31; k += 2) top[q] = max3_nan(top[q], __uint_as_float(s[q][k]), __uint_as_float(s[q][k + 1]));
    top[q] = max3_nan(top[q], __uint_as_float(s[q][30]), __uint_as_float(s[q][30]));
  }
  return max3_nan(max3_nan(top[0], top[1], top[2]), top[3], top[3]);
}
// Weights of the 32-column quarters FROM .. TO - 1 of a row, as bfloat16 over the row's logits in tensor memory; returns
// their sum.  EDGE: the tile holds masked logits, whose weights have to be exactly zero (no polynomial).  mx: gets the
// maximum of the whole row.
template <bool EDGE, int FROM, int TO>
__device__ __forceinline__ float weights(const uint32_t (&s)[4][32], float c, float sub, uint32_t at, float* mx) {
  const f32x2 c2 = pack2(c, c), sub2 = pack2(sub, sub);
  f32x2 sum[2] = {0ull, 0ull};
  if (mx) *mx = row_max(s);
#pragma unroll
  for (int q = FROM; q < TO; ++q) {
    uint32_t p[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const f32x2 x = fma2(pack2u(s[q][2 * k], s[q][2 * k + 1]), c2, sub2);
      float lo, hi;
      if (!EDGE && (k & 7) >= 8 - kPolyOf8) {
        poly_ex2(x, lo, hi);
      } else {
        unpack2(x, lo, hi);
        lo = ex2(lo);
        hi = ex2(hi);
      }
      sum[k & 1] = add2(sum[k & 1], pack2(lo, hi));
      p[k] = pack_bf16(lo, hi);
    }
    tmem_st16(at + 16 * q, p);
  }
  float lo, hi;
  unpack2(add2(sum[0], sum[1]), lo, hi);
  return lo + hi;
}

// What of a tile of rows a CTA needs to know.
struct Rows {
  int count;       // tokens of the tile that exist
  int first;       // its first token within the sequence
  int all, most;   // keys that every row sees, that any row sees
  int tiles;       // tiles of keys
};
__device__ __forceinline__ Rows rows_of(const Piece& p, int tile, int per, int causal) {
  Rows r;
  r.first = p.first + tile * per;
  r.count = min(per, p.nq - r.first);
  if (r.count <= 0) return {0, r.first, 0, 0, 0};
  r.all = causal ? max(0, min(p.nk, r.first + 1 + p.nk - p.nq)) : p.nk;
  r.most = causal ? max(0, min(p.nk, r.first + r.count + p.nk - p.nq)) : p.nk;
  r.tiles = (r.most + kTile - 1) / kTile;
  return r;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
prompt_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV, const PromptArgs a) {
  constexpr int kSlots = ring_slots<D>(), kSub = D / 64, kSubBytes = kTile * 128;
  constexpr uint32_t kColO = 256;
  extern __shared__ uint8_t raw[];
  __shared__ Shared sh;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = smem + 2 * tile_bytes<D>();
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int G = a.H / a.Hk, per = kTile / G, used = per * G;
  const int hk = blockIdx.x % a.Hk;
  if (warp == 0) {
    Piece p;
    const bool ok = find_piece(a, 2 * per, blockIdx.x / a.Hk, p);
    if (lane == 0) { sh.found = ok; sh.piece = p; }
  } else if (warp == kLoader && lane == 0) {
    prefetch_tmap(&tmQ); prefetch_tmap(&tmK); prefetch_tmap(&tmV);
    mbar_init(&sh.q_full, 1);
    for (int i = 0; i < kSlots; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
    for (int i = 0; i < kReady; ++i) { mbar_init(&sh.raw[i], 1); mbar_init(&sh.cleaned[i], kGuards); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.s_full[i], 1); mbar_init(&sh.p_most[i], kTile); mbar_init(&sh.p_ready[i], kTile); mbar_init(&sh.done[i], 1); }
    mbar_init(&sh.drained, 1);
    sh.abort_flag = 0;
    sh.wide = 0;
    mbar_fence_init();
  }
  __syncthreads();
  if (!sh.found) return;
  const Piece pc = sh.piece;
  if (warp == kIssuer) {                                   // (only CTAs with work hold tensor memory)
    tmem_alloc(&sh.tmem, 512);
    tmem_relinquish();
  }
  // rows of a tile that hold no query: whatever was in shared memory might be NaN and slow the softmax down
  for (int i = threadIdx.x; i < 2 * kSub * (kTile - used) * 8; i += kThreads) {
    const int c = i & 7, r = (i >> 3) % (kTile - used), s = (i >> 3) / (kTile - used);
    *reinterpret_cast<uint4*>(smem + s * kSubBytes + (used + r) * 128 + 16 * c) = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  volatile int* abort_flag = &sh.abort_flag;
  auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, abort_flag, a.status, DEV_TIMEOUT_ATTEND); };
  auto wait_warp = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
  const Rows row0 = rows_of(pc, 0, per, a.causal), row1 = rows_of(pc, 1, per, a.causal);
  const int tiles = max(row0.tiles, row1.tiles);
  const int guarded = row0.all / kTile;                    // from here on, not every row sees a whole tile of keys

  // Where an entry of the ring (K 0, V 0, K 1, V 1, ...) lands: its slot's barrier, or for value tiles that the guards have
  // first a barrier of theirs (they look at no other turn of a slot, and a barrier's phases must not be missed).
  auto turn_of = [&](int e) { return (e & 1) && (e >> 1) >= guarded ? ((e >> 1) - guarded) / kReady : e / kSlots; };
  auto landing = [&](int e) { return (e & 1) && (e >> 1) >= guarded ? &sh.raw[((e >> 1) - guarded) % kReady] : &sh.full[e % kSlots]; };

  // The softmax needs the registers: a row of logits is 128 of them.  (What the block was launched with covers the shares:
  // the host checks it.)  Each warp of a group of four moves its share in its own branch.
  if (warp >= kLoader) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegs));
  if (warp == kLoader) {
    int e = 0;
    bool ok = true;
    if (elect_one() && tiles > 0) {
      mbar_expect_tx(&sh.q_full, (row1.tiles ? 2 : 1) * kSub * used * 128);
      for (int i = 0; i < (row1.tiles ? 2 : 1); ++i)
        for (int s = 0; s < kSub; ++s)
          tma_load_3d(smem + (i * kSub + s) * kSubBytes, &tmQ, 64 * s, hk * G, pc.q0 + pc.first + i * per, &sh.q_full);
    }
    __syncwarp();
    for (; e < 2 * tiles; ++e) {
      const int slot = e % kSlots;
      if (e >= kSlots && !(ok = wait_warp(&sh.empty[slot], ((e / kSlots) - 1) & 1))) break;
      if (elect_one()) {
        uint64_t* bar = landing(e);
        if (bar != &sh.full[slot]) mbar_arrive(&sh.full[slot]);   // (nobody waits for this turn of the slot: it only passes)
        mbar_expect_tx(bar, tile_bytes<D>());
        for (int s = 0; s < kSub; ++s)
          tma_load_3d(ring + slot * tile_bytes<D>() + s * kSubBytes, (e & 1) ? &tmV : &tmK, 64 * s, hk, pc.k0 + (e >> 1) * kTile, bar);
      }
      __syncwarp();
    }
    if (!ok) {                                             // no copy is left in flight when the CTA ends
      int none = 0;
      mbar_wait(&sh.q_full, 0, &none, a.status, DEV_TIMEOUT_ATTEND);
      for (int i = max(0, e - kSlots); i < e; ++i) mbar_wait(landing(i), turn_of(i) & 1, &none, a.status, DEV_TIMEOUT_ATTEND);
    }
  } else if (warp == kIssuer) {
    const uint32_t q_at = smem_u32(smem), r_at = smem_u32(ring);
    constexpr uint32_t kIdS = umma_idesc_bf16(kTile, kTile), kIdO = umma_idesc_bf16(kTile, D) | (1u << 16);
    auto issue_s = [&](int i, int slot) {
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint32_t o = (k >> 2) * kSubBytes + (k & 3) * 32;
        umma_bf16(tmem + 128 * i, umma_desc_sw128(q_at + i * tile_bytes<D>() + o), umma_desc_sw128(r_at + slot * tile_bytes<D>() + o), kIdS,
                  k > 0);
      }
      umma_commit(&sh.s_full[i]);
    };
    auto issue_o = [&](int i, int slot, int from, int to, bool more) {
#pragma unroll
      for (int k = from; k < to; ++k)
        umma_bf16_ts(tmem + kColO + 128 * i, tmem + 128 * i + 8 * k,
                     umma_desc_sw128_mn(r_at + slot * tile_bytes<D>() + k * 2048, kSubBytes), kIdO, more || k > 0);
    };
    auto full = [&](int e) { return wait_warp(&sh.full[e % kSlots], (e / kSlots) & 1); };
    bool ok = tiles == 0 || (wait_warp(&sh.q_full, 0) && full(0));
    tc_fence_after();
    if (ok && tiles > 0) {
      if (elect_one()) {
        if (row0.tiles > 0) issue_s(0, 0);
        if (row1.tiles > 0) issue_s(1, 0);
        umma_commit(&sh.empty[0]);
      }
      __syncwarp();
    }
    for (int j = 0; ok && j < tiles; ++j) {
      const int ev = 2 * j + 1, ek = 2 * j + 2;
      ok = j < guarded ? full(ev) : wait_warp(&sh.cleaned[(j - guarded) % kReady], ((j - guarded) / kReady) & 1);
      if (ok && j + 1 < tiles) ok = full(ek);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int n = i ? row1.tiles : row0.tiles;
        if (j < n) {
          ok = ok && wait_warp(&sh.p_most[i], j & 1);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) issue_o(i, ev % kSlots, 0, kMost / 16, j > 0);
          __syncwarp();
          if (!(ok = wait_warp(&sh.p_ready[i], j & 1))) break;
          tc_fence_after();
          if (elect_one()) {
            issue_o(i, ev % kSlots, kMost / 16, kTile / 16, true);
            if (j + 1 < n) issue_s(i, ek % kSlots);
            else umma_commit(&sh.done[i]);
          }
          __syncwarp();
        }
      }
      if (ok && elect_one()) {
        umma_commit(&sh.empty[ev % kSlots]);
        if (j + 1 < tiles) umma_commit(&sh.empty[ek % kSlots]);
      }
      __syncwarp();
    }
    if (!ok) {                                             // products in flight end before tensor memory is given back
      if (elect_one()) umma_commit(&sh.drained);
      __syncwarp();
      int none = 0;
      mbar_wait(&sh.drained, 0, &none, a.status, DEV_TIMEOUT_ATTEND);
    }
  } else if (warp > kIssuer) {
    const int id = threadIdx.x - 32 * (kIssuer + 1);
    bool wide = false;
    for (int j = guarded; j < tiles; ++j) {
      const int e = 2 * j + 1, slot = e % kSlots;
      if (!wait_warp(landing(e), turn_of(e) & 1)) break;
      const int keys = pc.nk - j * kTile;
      uint4* v = reinterpret_cast<uint4*>(ring + slot * tile_bytes<D>());
      for (int i = id; i < tile_bytes<D>() / 16; i += kGuards) {
        const int r = (i >> 3) & (kTile - 1);
        if (r >= keys) {
          v[i] = make_uint4(0, 0, 0, 0);
          continue;
        }
        const uint4 x = v[i];
        uint32_t w[4] = {x.x, x.y, x.z, x.w};
        // an exponent of all ones in either half: with the low bits masked off the sum carries out of it
        uint32_t odd = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) odd |= ((w[q] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
        if (odd) {
          wide = true;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t bits = ((w[q] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
            if (bits & 0x8000u) w[q] &= 0xffff0000u;
            if (bits & 0x80000000u) w[q] &= 0x0000ffffu;
          }
          v[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      if (wide) *reinterpret_cast<volatile int*>(&sh.wide) = 1;
      fence_proxy_async();
      mbar_arrive(&sh.cleaned[(j - guarded) % kReady]);
    }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegs));
    const int i = warp >> 2, r = threadIdx.x & 127;
    const Rows rows = i ? row1 : row0;
    const uint32_t at = tmem + ((uint32_t)(32 * (warp & 3)) << 16), at_s = at + 128 * i, at_o = at + kColO + 128 * i;
    const int token = rows.first + r / G;                  // within the sequence
    const int sees = a.causal ? max(0, min(pc.nk, token + 1 + pc.nk - pc.nq)) : pc.nk;
    const float c = a.scale * kLog2e;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int j = 0; j < rows.tiles; ++j) {
      if (!(ok = wait_warp(&sh.s_full[i], j & 1))) break;
      tc_fence_after();
      uint32_t s[4][32];
#pragma unroll
      for (int q = 0; q < 4; ++q) tmem_ld32(at_s + 32 * q, s[q]);
#pragma unroll
      for (int q = 0; q < 4; ++q) tmem_wait(s[q]);
      const bool edge = (j + 1) * kTile > rows.all;
      if (edge) {
        const int n = sees - j * kTile;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int k = 0; k < 32; ++k)
            if (32 * q + k >= n) s[q][k] = 0xff800000u;
      }
      // The weights of all but the last quarter are taken with the maximum of the tiles before; the tile's own is found on
      // the side.  Only where it is higher by 2^8 (or there is none before, or a NaN) they are taken again.
      float mx = -INFINITY, sum = 0.f;
      if (j == 0) mx = row_max(s);
      else sum = edge ? weights<true, 0, kMost / 32>(s, c, reference(m, c), at_s, &mx) : weights<false, 0, kMost / 32>(s, c, reference(m, c), at_s, &mx);
      if (__any_sync(0xffffffffu, !((mx - m) * c <= kRaise))) {
        const float up = max3_nan(m, mx, mx);
        const float f = up == m || up == -INFINITY ? 1.f : ex2((m - up) * c);
        m = up;
        l *= f;
        if (j > 0) {
          // S of this tile was issued behind O of the tile before, so O is complete
#pragma unroll
          for (int q = 0; q < D / 32; ++q) {
            uint32_t o[32];
            tmem_ld32(at_o + 32 * q, o);
            tmem_wait(o);
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
            tmem_st32(at_o + 32 * q, o);
          }
        }
        sum = weights<true, 0, kMost / 32>(s, c, reference(m, c), at_s, nullptr);
      }
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(&sh.p_most[i]);
      sum += edge ? weights<true, kMost / 32, 4>(s, c, reference(m, c), at_s, nullptr) : weights<false, kMost / 32, 4>(s, c, reference(m, c), at_s, nullptr);
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(&sh.p_ready[i]);
      l += sum;
    }
    if (ok && rows.tiles > 0) ok = wait_warp(&sh.done[i], 0);
    if (ok && rows.tiles > guarded && rows.tiles > 0) {    // (whether a value was set to zero)
      const int g = tiles - 1 - guarded;
      ok = g < 0 || wait_warp(&sh.cleaned[g % kReady], (g / kReady) & 1);
    }
    tc_fence_after();
    if (ok) {
      const bool mine = r < used && token < pc.nq && rows.count > 0;
      const bool wide = *reinterpret_cast<volatile int*>(&sh.wide) != 0;
      const int64_t t = (int64_t)pc.q0 + token;
      const int h = hk * G + r % G;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      __nv_bfloat16* Y = static_cast<__nv_bfloat16*>(a.Y) + t * a.y_stride + (int64_t)h * D;
#pragma unroll
      for (int q = 0; q < D / 32; ++q) {
        uint32_t o[32];
        if (rows.tiles > 0) {
          tmem_ld32(at_o + 32 * q, o);
          tmem_wait(o);
        }
        float y[32];
#pragma unroll
        for (int k = 0; k < 32; ++k) y[k] = l == 0.f ? 0.f : __uint_as_float(o[k]) * inv;
        if (wide && mine) {                                // rare: infinities and NaN of the cleaned tiles, where seen
          for (int k = guarded * kTile; k < sees; ++k) {
            const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.V) + (int64_t)(pc.k0 + k) * a.v_stride + (int64_t)hk * D + 32 * q;
#pragma unroll
            for (int x = 0; x < 32; ++x) {
              const float f = __bfloat162float(v[x]);
              if (!isfinite(f)) y[x] += f;
            }
          }
        }
        if (mine) {
#pragma unroll
          for (int k = 0; k < 32; k += 8)
            *reinterpret_cast<uint4*>(Y + 32 * q + k) = make_uint4(pack_bf16(y[k], y[k + 1]), pack_bf16(y[k + 2], y[k + 3]),
                                                                   pack_bf16(y[k + 4], y[k + 5]), pack_bf16(y[k + 6], y[k + 7]));
        }
      }
      if (mine && a.lse) a.lse[t * a.H + h] = l == 0.f ? -INFINITY : (m * c + log2f(l)) * kLn2;
    }
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  if (warp == kIssuer) tmem_dealloc(tmem, 512);
}

// Whether the block's registers at launch cover the shares that its warps ask for (or they would wait for good).
template <int D>
bool registers_cover() {
  static const bool ok = [] {
    cudaFuncAttributes fa;
    return cudaFuncGetAttributes(&fa, prompt_tc_kernel<D>) == cudaSuccess &&
           fa.numRegs * kThreads >= 32 * (kLoader * kManyRegs + (kThreads / 32 - kLoader) * kFewRegs);
  }();
  return ok;
}

template <int D>
avq_status launch(const PromptArgs& a, cudaStream_t st) {
  const int G = a.H / a.Hk, per = kTile / G;
  CUtensorMap tmQ, tmK, tmV;
  const uint64_t dq[3] = {(uint64_t)D, (uint64_t)a.H, (uint64_t)a.Tq}, dk[3] = {(uint64_t)D, (uint64_t)a.Hk, (uint64_t)a.Tk};
  const uint32_t bq[3] = {64, (uint32_t)G, (uint32_t)per}, bk[3] = {64, 1, (uint32_t)kTile};
  avq_status s = make_tmap_rows(&tmQ, a.Q, dq, a.q_stride, bq);
  if (s != AVQ_OK) return s;
  // (without keys no CTA loads any: the maps only have to exist)
  s = a.Tk ? make_tmap_rows(&tmK, a.K, dk, a.k_stride, bk) : make_tmap_rows(&tmK, a.Q, dq, a.q_stride, bk);
  if (s != AVQ_OK) return s;
  s = a.Tk ? make_tmap_rows(&tmV, a.V, dk, a.v_stride, bk) : make_tmap_rows(&tmV, a.Q, dq, a.q_stride, bk);
  if (s != AVQ_OK) return s;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return AVQ_ERR_CUDA;
  s = open_shared_memory<prompt_tc_kernel<D>>(dev);
  if (s != AVQ_OK) return s;
  if (!registers_cover<D>()) return AVQ_ERR_CUDA;
  const int64_t grid = most_pieces(a.Tq, a.S, 2 * per) * a.Hk;
  if (grid >= (int64_t)1 << 31) return AVQ_ERR_UNSUPPORTED;
  prompt_tc_kernel<D><<<(unsigned)grid, kThreads, prompt_smem<D>(), st>>>(tmQ, tmK, tmV, a);
  return cuda_ok(cudaGetLastError());
}

}  // namespace

avq_status tc_prompt(const PromptArgs& a, cudaStream_t st) { return a.d == 64 ? launch<64>(a, st) : launch<128>(a, st); }

}  // namespace exact
}  // namespace avq
