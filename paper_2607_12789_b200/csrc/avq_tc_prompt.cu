// Exact attention of packed bfloat16 sequences on the tensor cores (d 64 or 128).
//
//   S = Q K^T,  P = exp(scale (S - m)),  O += P V,  l += sum P,  Y = O / l     over tiles of 128 keys
//
// A CTA takes two tiles of 128 rows of one key head: the H/Hk query heads that share it are rows of one tile, (query,
// head) with the head fastest, so that a tile of keys and values is read once for all of them and a short sequence fills
// the rows that it can.  Roles by warp:
//   0-3, 4-7  one tile each, a thread per row: logits out of tensor memory, maximum, weights back as bfloat16 in their
//             place, sum; at the end the outputs out of tensor memory
//   8         loads (TMA): the two tiles of queries, then keys and values in turn through a ring; the next task's while the
//             last one's outputs are being written
//   9         issues every tcgen05.mma: S of one tile while the other tile's weights are being computed
//   10, 11    clean the value tiles that not every row sees whole: rows behind the last key become zero (they are
//             another sequence's), infinities and NaN too (a weight of zero times one of them would be NaN); the
//             latter are added back at the end to the rows that do see them; warp 10 also hands out the tasks
// Bound at d = 128: per pair of tiles of 128 keys the products take 2048 cycles of the tensor pipe and the 32768
// exponentials as many of the MUFU pipe, in turn for each tile of rows; what keeps them from overlapping fully is the way
// from logits to weights and back.  A quarter of the exponentials by a polynomial on the FMA pipe was 4 % slower than
// none (16384 tokens of 16 heads: 949 and 906 us): a second form of the code costs more than the pipe gains.
// Measured: 16384 tokens, 16 heads on 4, d 128, causal 886 us (1241 TFLOP/s, 75 % of the measured burst rate; 1035 us and 1062
// TFLOP/s when it runs on and on at the power limit), 16 prompts of up to 2048 tokens, 32 heads on 8, 187 us (691 TFLOP/s: a third
// of the time is the first logits and the outputs of each of 1704 short pieces).  d 64: half the products for as many exponentials,
// which alone would allow 1190 TFLOP/s; 16384 tokens of 16 heads 706 (the way from logits to weights and back, again).
// The maximum that weights refer to is raised only when a row exceeds it by 2^8, which spares nearly every rescaling of
// O: weights stay below 2^8, and what they are relative to cancels in O / l.
// Weights are rounded to bfloat16 for the value product (2^-8 of each at most; their sum l is of the float32
// ones): two parts would double it.  Against 64 bits 2.0e-3 of the result, where float32 weights have 1.6e-3, the outputs' own
// rounding.
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
constexpr int kSplitBelow = 148, kSplitKeys = AVQ_PROMPT_SPLIT_KEYS, kLeastTiles = 4, kSetupTiles = 2;   // when pieces are split, and into parts of what size at least
constexpr int kFewRegs = 80, kManyRegs = 208;              // per thread of warps 8-11, of warps 0-7
template <int D> __host__ __device__ constexpr int ring_slots() { return D == 128 ? 5 : 10; }
template <int D> __host__ __device__ constexpr int tile_bytes() { return kTile * D * 2; }
template <int D> __host__ __device__ constexpr size_t prompt_smem() { return 1024 + (size_t)(2 + ring_slots<D>()) * tile_bytes<D>(); }

// What a CTA works on next: a pair of tiles of rows, and of which tiles of keys.
struct Task {
  Piece piece;
  int32_t hk, from, to;          // key head; tiles of keys from .. to - 1
  int32_t slot;                  // where a part of a piece leaves its partial result, or -1: the rows' outputs
  int32_t index;                 // number of the piece, or -1: there is nothing more to do
};
constexpr int kTasks = 4;        // handed out ahead: a task's loads and first products do not wait for the end of the one before
constexpr int kMostSplit = 160;  // pieces of a call whose pieces are split
struct Shared {
  uint64_t q_full, q_free, full[10], empty[10], raw[kReady], cleaned[kReady], s_full[2], p_most[2], p_ready[2], done[2], o_free[2];
  uint64_t task_full[kTasks], task_free[kTasks], drained;
  Task task[kTasks];
  uint32_t tmem;
  int progress;                  // tiles that have been asked for
  int abort_flag, wide[kTasks];
  int32_t before[kMostSplit + 1];   // split calls: tiles of keys, with the setups, of the pieces before each
};

__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// As mbar_wait, but the limit is on the time without progress: some waits last a whole task (value tiles that the guards see
// first, room for the next task), which may be millions of tiles.  Ends all the same: there are only so many tiles.
__device__ __forceinline__ bool mbar_wait_or_progress(uint64_t* bar, uint32_t parity, volatile int* abort_flag, const volatile int* progress,
                                                      int32_t* status_word, int32_t code) {
  if (mbar_test_wait(bar, parity)) return true;
  while (true) {
    const int seen = *progress;
    const unsigned long long t0 = global_timer_ns();
    for (uint32_t polls = 0; polls < kWaitLimitPolls; ++polls) {
      if (mbar_try_wait(bar, parity, kWaitTryNs)) return true;
      if (*abort_flag) return false;
      if (global_timer_ns() - t0 > kWaitLimitNs) break;
    }
    if (*progress == seen) break;
  }
  *abort_flag = 1;
  if (status_word) atomicCAS(status_word, 0, code);
  return false;
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
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
      "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
      "r"(r[14]), "r"(r[15]), "r"(at)
      : "memory");
}
__device__ __forceinline__ void store32(void* to, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f, uint32_t g, uint32_t h) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e), "r"(f), "r"(g), "r"(h)
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
// their sum.  mx: gets the maximum of the whole row.
template <int FROM, int TO>
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
      unpack2(x, lo, hi);
      lo = ex2(lo);
      hi = ex2(hi);
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

// ---- which CTA does what
// Many pieces: CTA c of n takes the pieces' (key head fastest) numbers c, 2 n - 1 - c, 2 n + c, ...: of one causal sequence the
// sizes fall with the number, and going back and forth evens them out.
// Few pieces (`run` > 0): all tiles of keys of all pieces and key heads, in that order, are dealt out in runs of `run`; a CTA
// finishes what lies inside its run and leaves partial results of the at most two pieces that do not, its first in slot
// 2 c, its last in slot 2 c + 1; prompt_join_kernel adds them in the order of the CTAs.  What a piece costs whatever its
// tiles (its first logits, its outputs) counts as kSetupTiles more, ahead of its own.
__device__ __forceinline__ int tiles_of(const Piece& p, int per, int causal) {
  const Rows a = rows_of(p, 0, per, causal), b = rows_of(p, 1, per, causal);
  return max(a.tiles, b.tiles);
}
// before[k]: tiles of keys, with the setups, of the pieces 0 .. k - 1; returns those of all `pieces`.  By one warp; bounds:
// scratch of S words.
__device__ __forceinline__ int sum_tiles(const PromptArgs& a, int per, int pieces, int4* bounds, int32_t* before) {
  const int lane = threadIdx.x & 31;
  for (int s = lane; s < a.S; s += 32) {
    Piece p;
    if (!sequence(a, s, p)) report(a.status, DEV_BAD_INDEX);
    bounds[s] = make_int4(p.q0, p.nq, p.k0, p.nk);
  }
  __syncwarp();
  int sum = 0;
  for (int k0 = 0; k0 < pieces; k0 += 32) {
    const int k = k0 + lane;
    int n = 0, left = k;
    for (int s = a.S - 1; s >= 0 && k < pieces; --s) {     // (the order is find_piece's)
      const int4 q = bounds[s];
      const int tiles = (q.y + 2 * per - 1) / (2 * per);
      if (left < tiles) {
        n = tiles_of({q.x, q.y, q.z, q.w, (tiles - 1 - left) * 2 * per}, per, a.causal);
        n += n > 0 ? kSetupTiles : 0;
        break;
      }
      left -= tiles;
    }
    int x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += up;
    }
    if (k < pieces) before[k] = sum + x - n;
    sum += __shfl_sync(0xffffffffu, x, 31);
  }
  if (lane == 0) before[pieces] = sum;
  __syncwarp();
  return sum;
}
// A part: for each 4 columns the values of its 256 rows, then the rows' maxima, then their sums (neighbouring rows are
// neighbouring lanes of the kernels).
__host__ __device__ constexpr int64_t part_floats(int d) { return (int64_t)2 * kTile * (d + 2); }

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
prompt_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV, const PromptArgs a, int pieces, int least, float* parts) {
  constexpr int kSlots = ring_slots<D>(), kSub = D / 64, kSubBytes = kTile * 128;
  constexpr uint32_t kColO = 256;
  extern __shared__ uint8_t raw[];
  __shared__ Shared sh;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = smem + 2 * tile_bytes<D>();
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int G = a.H / a.Hk, per = kTile / G, used = per * G;
  if (warp == kIssuer) {
    tmem_alloc(&sh.tmem, 512);
    tmem_relinquish();
  } else if (warp == kLoader && lane == 0) {
    prefetch_tmap(&tmQ); prefetch_tmap(&tmK); prefetch_tmap(&tmV);
    mbar_init(&sh.q_full, 1);
    mbar_init(&sh.q_free, 1);
    for (int i = 0; i < kSlots; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
    for (int i = 0; i < kReady; ++i) { mbar_init(&sh.raw[i], 1); mbar_init(&sh.cleaned[i], kGuards); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.s_full[i], 1); mbar_init(&sh.p_most[i], kTile); mbar_init(&sh.p_ready[i], kTile);
      mbar_init(&sh.done[i], 1); mbar_init(&sh.o_free[i], kTile);
    }
    for (int i = 0; i < kTasks; ++i) { mbar_init(&sh.task_full[i], 1); mbar_init(&sh.task_free[i], kThreads / 32 - 1); }
    mbar_init(&sh.drained, 1);
    sh.abort_flag = sh.progress = 0;
    mbar_fence_init();
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
  volatile int* progress = &sh.progress;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    return mbar_wait_or_progress(bar, parity, abort_flag, progress, a.status, DEV_TIMEOUT_ATTEND);
  };
  auto wait_warp = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
  // The task number t, for all roles but the one that hands them out; false: no more (or the CTA gave up).
  auto next_task = [&](int t, Task& task) {
    if (!wait_warp(&sh.task_full[t % kTasks], (t / kTasks) & 1)) { task.index = -1; return false; }
    task = sh.task[t % kTasks];
    return task.index >= 0;
  };
  auto end_task = [&](int t) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.task_free[t % kTasks]);
  };
  // Tiles of keys of a task that a tile of rows takes, and the first of them (absolute) that not every row sees whole.
  auto share = [&](const Task& k, const Rows& r) { return max(0, min(k.to, r.tiles) - k.from); };

  // The softmax needs the registers: a row of logits is 128 of them.  (What the block was launched with covers the shares:
  // the host checks it.)  Each warp of a group of four moves its share in its own branch.
  if (warp >= kLoader) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegs));

  if (warp == kLoader) {
    int e = 0, g = 0, t = 0;                               // entries of the ring, value tiles that the guards have first, tasks
    bool ok = true;
    uint32_t last = 0;                                     // (giving up: whether the last entries landed at their slot's barrier)
    Task task;
    for (; ok && next_task(t, task); ++t) {
      const Rows row0 = rows_of(task.piece, 0, per, a.causal), row1 = rows_of(task.piece, 1, per, a.causal);
      const int guarded = row0.all / kTile, both = share(task, row1) > 0 ? 2 : 1;
      // (every task is one turn of q_full and of q_free, also one without keys: no turn may be missed)
      if (t > 0 && !(ok = wait_warp(&sh.q_free, (t - 1) & 1))) break;
      if (task.to > task.from) {
        if (elect_one()) {
          // (a tile that takes no part is not loaded; whichever of the two it is, the other's place stays its own)
          const int lo = share(task, row0) > 0 ? 0 : 1;
          mbar_expect_tx(&sh.q_full, (both - lo) * kSub * used * 128);
          for (int i = lo; i < both; ++i)
            for (int s = 0; s < kSub; ++s)
              tma_load_3d(smem + (i * kSub + s) * kSubBytes, &tmQ, 64 * s, task.hk * G, task.piece.q0 + task.piece.first + i * per, &sh.q_full);
        }
        __syncwarp();
      } else if (lane == 0) {
        mbar_arrive(&sh.q_full);
      }
      for (int x = 2 * task.from; x < 2 * task.to; ++x, ++e) {
        const int slot = e % kSlots, j = x >> 1;
        if (e >= kSlots && !(ok = wait_warp(&sh.empty[slot], ((e / kSlots) - 1) & 1))) break;
        // Value tiles that the guards have first land at a barrier of theirs (they look at no other turn of a slot, and a
        // barrier's phases must not be missed); the slot's own barrier only passes.
        const bool guard = (x & 1) && j >= guarded;
        if (elect_one()) {
          uint64_t* bar = guard ? &sh.raw[g % kReady] : &sh.full[slot];
          if (guard) mbar_arrive(&sh.full[slot]);
          mbar_expect_tx(bar, tile_bytes<D>());
          *progress = e;
          for (int s = 0; s < kSub; ++s)
            tma_load_3d(ring + slot * tile_bytes<D>() + s * kSubBytes, (x & 1) ? &tmV : &tmK, 64 * s, task.hk, task.piece.k0 + j * kTile, bar);
        }
        __syncwarp();
        last = last << 1 | (guard ? 1u : 0u);
        g += guard;
      }
      end_task(t);
    }
    if (!ok || *abort_flag) {                              // no copy is left in flight when the CTA ends
      int none = 0;
      if (t > 0 || e > 0) mbar_wait(&sh.q_full, t & 1, &none, a.status, DEV_TIMEOUT_ATTEND);
      for (int i = 0; i < min(e, kSlots); ++i) {
        const int x = e - 1 - i;
        if (last >> i & 1) { --g; mbar_wait(&sh.raw[g % kReady], (g / kReady) & 1, &none, a.status, DEV_TIMEOUT_ATTEND); }
        else mbar_wait(&sh.full[x % kSlots], (x / kSlots) & 1, &none, a.status, DEV_TIMEOUT_ATTEND);
      }
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
    bool ok = true;
    int e0 = 0, g = 0;                                     // entries and guarded value tiles of the tasks before
    int turn[2] = {0, 0}, took[2] = {0, 0};                // tiles of keys, tasks that each tile of rows has taken
    Task task;
    for (int t = 0; ok && next_task(t, task); ++t) {
      const Rows row0 = rows_of(task.piece, 0, per, a.causal), row1 = rows_of(task.piece, 1, per, a.causal);
      const int guarded = row0.all / kTile, tiles = task.to - task.from;
      const int n[2] = {share(task, row0), share(task, row1)};
      if (!(ok = wait_warp(&sh.q_full, t & 1))) break;
      if (tiles > 0) {
        if (!(ok = full(e0))) break;
        tc_fence_after();
        if (elect_one()) {
          if (n[0] > 0) issue_s(0, e0 % kSlots);
          if (n[1] > 0) issue_s(1, e0 % kSlots);
          umma_commit(&sh.empty[e0 % kSlots]);
          if (tiles == 1) umma_commit(&sh.q_free);
        }
        __syncwarp();
      }
      for (int j = 0; ok && j < tiles; ++j) {
        const int ev = e0 + 2 * j + 1, ek = ev + 1;
        if (task.from + j < guarded) ok = full(ev);
        else { ok = wait_warp(&sh.cleaned[g % kReady], (g / kReady) & 1); ++g; }
        if (ok && j + 1 < tiles) ok = full(ek);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (j < n[i]) {
            // (the outputs of this tile's last task have been read before they are overwritten)
            if (j == 0 && took[i] > 0) ok = ok && wait_warp(&sh.o_free[i], (took[i] - 1) & 1);
            ok = ok && wait_warp(&sh.p_most[i], (turn[i] + j) & 1);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) issue_o(i, ev % kSlots, 0, kMost / 16, j > 0);
            __syncwarp();
            if (!(ok = wait_warp(&sh.p_ready[i], (turn[i] + j) & 1))) break;
            tc_fence_after();
            if (elect_one()) {
              issue_o(i, ev % kSlots, kMost / 16, kTile / 16, true);
              if (j + 1 < n[i]) issue_s(i, ek % kSlots);
              else umma_commit(&sh.done[i]);
            }
            __syncwarp();
          }
        }
        if (ok && elect_one()) {
          umma_commit(&sh.empty[ev % kSlots]);
          if (j + 1 < tiles) umma_commit(&sh.empty[ek % kSlots]);
          if (j + 2 == tiles) umma_commit(&sh.q_free);     // the task's last logits have been issued
        }
        __syncwarp();
      }
      if (tiles == 0 && lane == 0) mbar_arrive(&sh.q_free);
      e0 += 2 * tiles;
#pragma unroll
      for (int i = 0; i < 2; ++i) { turn[i] += n[i]; took[i] += n[i] > 0; }
      end_task(t);
    }
    if (!ok || *abort_flag) {                              // products in flight end before tensor memory is given back
      if (elect_one()) umma_commit(&sh.drained);
      __syncwarp();
      int none = 0;
      mbar_wait(&sh.drained, 0, &none, a.status, DEV_TIMEOUT_ATTEND);
    }
  } else {
    // The guards; the first of their warps hands out the tasks too.
    const bool chief = warp == kIssuer + 1;
    const int id = threadIdx.x - 32 * (kIssuer + 1);
    int e0 = 0, g = 0, number = blockIdx.x, round = 0;
    int64_t at = 0, end = 0;
    if (chief && least > 0) {
      const int64_t total = (int64_t)sum_tiles(a, per, pieces, reinterpret_cast<int4*>(ring), sh.before) * a.Hk, run = run_of(total, gridDim.x, least);
      fence_proxy_async();                                 // (the ring's place, which the copies get with the first task)
      at = (int64_t)blockIdx.x * run;
      end = min(at + run, total);
    }
    auto hand_out = [&](int t) {                           // false: the CTA gave up
      Task task = {};
      task.index = -1;
      task.slot = -1;
      if (least > 0) {
        while (at < end && task.index < 0) {
          int k = 0;                                       // the last piece that begins at or before `at` and has tiles
          for (int x = lane; x < pieces; x += 32)
            if ((int64_t)sh.before[x] * a.Hk <= at && sh.before[x + 1] > sh.before[x]) k = max(k, x);
          k = __reduce_max_sync(0xffffffffu, k);
          const int W = sh.before[k + 1] - sh.before[k], U = W - kSetupTiles;
          const int rel = (int)(at - (int64_t)sh.before[k] * a.Hk), x = rel % W, take = (int)min((int64_t)(W - x), end - at);
          at += take;
          if (x + take <= kSetupTiles) continue;           // (the setup alone: the piece is the next CTA's)
          find_piece(a, 2 * per, k, task.piece);
          task.index = k;
          task.hk = rel / W;
          task.from = max(0, x - kSetupTiles);
          task.to = x + take - kSetupTiles;
          if (task.from > 0 || task.to < U) task.slot = 2 * blockIdx.x + (task.from == 0);
        }
      } else {
        if (find_piece(a, 2 * per, number / a.Hk, task.piece)) {
          task.index = number / a.Hk;
          task.hk = number % a.Hk;
          task.to = tiles_of(task.piece, per, a.causal);
        }
        number = ++round & 1 ? (round + 1) * (int)gridDim.x - 1 - blockIdx.x : round * (int)gridDim.x + blockIdx.x;
      }
      if (t >= kTasks && !wait_warp(&sh.task_free[t % kTasks], ((t / kTasks) - 1) & 1)) return false;
      if (lane == 0) {
        sh.task[t % kTasks] = task;
        sh.wide[t % kTasks] = 0;
        mbar_arrive(&sh.task_full[t % kTasks]);
      }
      __syncwarp();
      return true;
    };
    bool ok = !chief || hand_out(0);
    Task task;
    for (int t = 0; ok && next_task(t, task); ++t) {
      if (chief) ok = hand_out(t + 1);
      const int guarded = rows_of(task.piece, 0, per, a.causal).all / kTile;
      bool wide = false;
      for (int j = max(guarded, task.from); ok && j < task.to; ++j, ++g) {
        const int slot = (e0 + 2 * (j - task.from) + 1) % kSlots;
        if (!(ok = wait_warp(&sh.raw[g % kReady], (g / kReady) & 1))) break;
        const int keys = task.piece.nk - j * kTile;
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
        if (wide) *reinterpret_cast<volatile int*>(&sh.wide[t % kTasks]) = 1;
        fence_proxy_async();
        mbar_arrive(&sh.cleaned[g % kReady]);
      }
      e0 += 2 * (task.to - task.from);
      if (!chief) end_task(t);
    }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegs));
    const int i = warp >> 2, r = threadIdx.x & 127;
    const uint32_t at = tmem + ((uint32_t)(32 * (warp & 3)) << 16), at_s = at + 128 * i, at_o = at + kColO + 128 * i;
    const float c = a.scale * kLog2e;
    // (whole sectors where rows are aligned to them: half as many stores of a row per lane)
    const bool wide_stores = ((reinterpret_cast<uintptr_t>(a.Y) | (uintptr_t)(2 * a.y_stride)) & 31) == 0;
    bool ok = true;
    int turn = 0, took = 0, guards = 0;                    // tiles of keys and tasks of this tile of rows, guarded value tiles
    for (int t = 0; ok; ++t) {
      // (the task's fields are read where they are needed: the registers are the logits')
      const volatile Task& task = sh.task[t % kTasks];
      if (!wait_warp(&sh.task_full[t % kTasks], (t / kTasks) & 1) || task.index < 0) break;
      int n, from, all, sees;
      {
        const Piece pc = {task.piece.q0, task.piece.nq, task.piece.k0, task.piece.nk, task.piece.first};
        const Rows rows = rows_of(pc, i, per, a.causal);
        const int token = rows.first + r / G;              // within the sequence
        from = task.from;
        n = max(0, min(task.to, rows.tiles) - from);
        all = rows.all;
        sees = a.causal ? max(0, min(pc.nk, token + 1 + pc.nk - pc.nq)) : pc.nk;
      }
      float m = -INFINITY, l = 0.f, limit = -INFINITY;
      for (int jj = 0; jj < n; ++jj) {
        const int j = from + jj;
        if (!(ok = wait_warp(&sh.s_full[i], (turn + jj) & 1))) break;
        tc_fence_after();
        uint32_t s[4][32];
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld32(at_s + 32 * q, s[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_wait(s[q]);
        const bool edge = (j + 1) * kTile > all;
        if (edge) {
          const int most = sees - j * kTile;
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (32 * q + k >= most) s[q][k] = 0xff800000u;
        }
        // The weights of all but the last quarter are taken with the maximum of the tiles before; the tile's own is found on
        // the side.  Only where it is higher by 2^8 (or a NaN, or there is none before) they are taken again.
        float mx = -INFINITY, sum = 0.f;
        bool first = jj == 0;
        while (true) {
          if (first) mx = row_max(s);
          else sum = weights<0, kMost / 32>(s, c, reference(m, c), at_s, &mx);
          // (each row by its own logits alone: what others hold, and whether they are raised, does not change its roundings)
          const bool raise = first || mx > limit || (mx != mx && m == m);
          if (!__any_sync(0xffffffffu, raise)) break;
          first = false;
          const float up = raise ? max3_nan(m, mx, mx) : m;
          const float f = up == m || up == -INFINITY ? 1.f : ex2((m - up) * c);
          m = up;
          limit = m == m ? m + kRaise / c : INFINITY;
          l *= f;
          if (jj > 0) {
            // (S of this tile was issued behind O of the tile before, so O is complete)
#pragma unroll
            for (int q = 0; q < D / 16; ++q) {
              float o[16];
              uint32_t w[16];
              tmem_ld16(at_o + 16 * q, o);
#pragma unroll
              for (int k = 0; k < 16; ++k) w[k] = __float_as_uint(o[k] * f);
              tmem_st16(at_o + 16 * q, w);
            }
          }
        }
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(&sh.p_most[i]);
        sum += weights<kMost / 32, 4>(s, c, reference(m, c), at_s, nullptr);
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(&sh.p_ready[i]);
        l += sum;
      }
      turn += n;
      const Piece pc = {task.piece.q0, task.piece.nq, task.piece.k0, task.piece.nk, task.piece.first};
      const int first = max(rows_of(pc, 0, per, a.causal).all / kTile, from);   // of the value tiles of this task that the guards had
      const int cleaned = max(0, task.to - first), token = pc.first + i * per + r / G;
      if (ok && n > 0) ok = wait_warp(&sh.done[i], took & 1);
      // (whether a value was set to zero: the last of the task's cleaned tiles tells for all, and the product with it is over)
      if (ok && cleaned > 0) ok = wait_warp(&sh.cleaned[(guards + cleaned - 1) % kReady], ((guards + cleaned - 1) / kReady) & 1);
      guards += cleaned;
      took += n > 0;
      tc_fence_after();
      if (ok) {
        const bool mine = r < used && token < pc.nq;
        const int slot = task.slot, hk = task.hk, to = task.to;
        const bool wide = *reinterpret_cast<volatile int*>(&sh.wide[t % kTasks]) != 0;
        const int64_t row = (int64_t)pc.q0 + token;
        const int h = hk * G + r % G;
        const float inv = slot >= 0 ? 1.f : l == 0.f ? 0.f : 1.f / l;
        __nv_bfloat16* Y = static_cast<__nv_bfloat16*>(a.Y) + row * a.y_stride + (int64_t)h * D;
        float* part = parts + (int64_t)max(slot, 0) * part_floats(D) + 4 * (i * kTile + r);
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
          uint32_t o[32];
          if (n > 0) {
            tmem_ld32(at_o + 32 * q, o);
            tmem_wait(o);
          }
          if (q == D / 32 - 1 && n > 0) {                  // the next task may have the outputs' place
            tc_fence_before();
            mbar_arrive(&sh.o_free[i]);
          }
          float y[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) y[k] = l == 0.f ? 0.f : __uint_as_float(o[k]) * inv;
          if (wide && mine) {                              // rare: infinities and NaN of the cleaned tiles, where seen
            for (int k = first * kTile; k < min(sees, to * kTile); ++k) {
              const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.V) + (int64_t)(pc.k0 + k) * a.v_stride + (int64_t)hk * D + 32 * q;
#pragma unroll
              for (int x = 0; x < 32; ++x) {
                const float f = __bfloat162float(v[x]);
                if (!isfinite(f)) y[x] += f;
              }
            }
          }
          if (slot >= 0) {
#pragma unroll
            for (int k = 0; k < 32; k += 4)
              *reinterpret_cast<float4*>(part + (32 * q + k) * 2 * kTile) = make_float4(y[k], y[k + 1], y[k + 2], y[k + 3]);
          } else if (mine && wide_stores) {
#pragma unroll
            for (int k = 0; k < 32; k += 16)
              store32(Y + 32 * q + k, pack_bf16(y[k], y[k + 1]), pack_bf16(y[k + 2], y[k + 3]), pack_bf16(y[k + 4], y[k + 5]),
                      pack_bf16(y[k + 6], y[k + 7]), pack_bf16(y[k + 8], y[k + 9]), pack_bf16(y[k + 10], y[k + 11]),
                      pack_bf16(y[k + 12], y[k + 13]), pack_bf16(y[k + 14], y[k + 15]));
          } else if (mine) {
#pragma unroll
            for (int k = 0; k < 32; k += 8)
              *reinterpret_cast<uint4*>(Y + 32 * q + k) = make_uint4(pack_bf16(y[k], y[k + 1]), pack_bf16(y[k + 2], y[k + 3]),
                                                                     pack_bf16(y[k + 4], y[k + 5]), pack_bf16(y[k + 6], y[k + 7]));
          }
        }
        if (slot >= 0) {
          float* stat = parts + (int64_t)slot * part_floats(D) + 2 * kTile * D + i * kTile + r;
          stat[0] = m == -INFINITY ? -INFINITY : m * c;
          stat[2 * kTile] = l;
        } else if (mine && a.lse) {
          a.lse[row * a.H + h] = l == 0.f ? -INFINITY : (m * c + log2f(l)) * kLn2;
        }
      }
      end_task(t);
    }
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  if (warp == kIssuer) tmem_dealloc(tmem, 512);
}

// ---- partial results of split pieces: 32 rows to a CTA, a row per lane, a share of the columns per warp.  Nothing to do if one
// CTA had the whole piece, zeros if its rows see no key; else the parts are brought to their common maximum and added in the
// order of the CTAs.
constexpr int kJoinRows = 32, kJoinWarps = 8;
template <int D>
__global__ void __launch_bounds__(32 * kJoinWarps) prompt_join_kernel(const PromptArgs a, int pieces, int least, int ctas, const float* parts) {
  __shared__ int4 bounds[kMostSplit];
  __shared__ int32_t before[kMostSplit + 1];
  __shared__ Piece shared_piece;
  __shared__ int found;
  pdl_wait();                                              // (every CTA: the grid's end is to mean the end of the kernel before, too)
  const int G = a.H / a.Hk, per = kTile / G, k = blockIdx.x / a.Hk, hk = blockIdx.x % a.Hk;
  if (threadIdx.x < 32) {
    sum_tiles(a, per, pieces, bounds, before);
    Piece p;
    const bool ok = find_piece(a, 2 * per, k, p);
    if (threadIdx.x == 0) { found = ok; shared_piece = p; }
  }
  __syncthreads();
  if (!found) return;
  const Piece pc = shared_piece;
  const int W = before[k + 1] - before[k], U = max(0, W - kSetupTiles);
  const int64_t run = run_of((int64_t)before[pieces] * a.Hk, ctas, least), g0 = (int64_t)before[k] * a.Hk + (int64_t)hk * W + kSetupTiles;
  const int c0 = (int)quotient(g0, run), c1 = U > 0 ? (int)quotient(g0 + U - 1, run) : c0;
  if (U > 0 && c0 == c1) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = blockIdx.y * kJoinRows + lane, i = r / kTile, x = r % kTile, token = pc.first + i * per + x / G;
  if (x >= per * G || token >= pc.nq) return;
  constexpr int kPer = D / kJoinWarps, kBatch = 4;         // columns of a lane, parts in flight together
  const int n = U > 0 ? c1 - c0 + 1 : 0;
  auto slot = [&](int p) { return parts + (int64_t)(2 * (c0 + p) + (p == 0)) * part_floats(D); };
  float m = -INFINITY, l = 0.f, y[kPer] = {};
#pragma unroll 8
  for (int p = 0; p < n; ++p) m = fmaxf(m, ld_after_wait(slot(p) + 2 * kTile * D + r));
  const float use = m == -INFINITY ? 0.f : m;
  for (int p0 = 0; p0 < n; p0 += kBatch) {
    float top[kBatch], sum[kBatch];
    float4 v[kBatch][kPer / 4];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      top[b] = -INFINITY;
      if (p0 + b >= n) continue;
      const float* s = slot(p0 + b);
      top[b] = ld_after_wait(s + 2 * kTile * D + r);
      sum[b] = ld_after_wait(s + 2 * kTile * D + 2 * kTile + r);
#pragma unroll
      for (int q = 0; q < kPer / 4; ++q) v[b][q] = ld_after_wait(reinterpret_cast<const float4*>(s + (warp * kPer + 4 * q) * 2 * kTile + 4 * r));
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const float w = exp2f(top[b] - use);
      if (w == 0.f) continue;
      l = fmaf(w, sum[b], l);
#pragma unroll
      for (int q = 0; q < kPer / 4; ++q) {
        y[4 * q] = fmaf(w, v[b][q].x, y[4 * q]);
        y[4 * q + 1] = fmaf(w, v[b][q].y, y[4 * q + 1]);
        y[4 * q + 2] = fmaf(w, v[b][q].z, y[4 * q + 2]);
        y[4 * q + 3] = fmaf(w, v[b][q].w, y[4 * q + 3]);
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int64_t row = (int64_t)pc.q0 + token;
  const int h = hk * G + x % G;
  __nv_bfloat16* Y = static_cast<__nv_bfloat16*>(a.Y) + row * a.y_stride + (int64_t)h * D + warp * kPer;
#pragma unroll
  for (int q = 0; q < kPer; q += 8)
    *reinterpret_cast<uint4*>(Y + q) = make_uint4(pack_bf16(y[q] * inv, y[q + 1] * inv), pack_bf16(y[q + 2] * inv, y[q + 3] * inv),
                                                  pack_bf16(y[q + 4] * inv, y[q + 5] * inv), pack_bf16(y[q + 6] * inv, y[q + 7] * inv));
  if (a.lse && warp == 0) a.lse[row * a.H + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
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
  int sms = 0;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return AVQ_ERR_CUDA;
  sms = sms < kPromptCtas ? sms : kPromptCtas;
  const int64_t pieces = most_pieces(a.Tq, a.S, 2 * per), all = pieces * a.Hk;
  if (all >= (int64_t)1 << 30) return AVQ_ERR_UNSUPPORTED;
  // Pieces that cannot fill the GPU, over keys that can be long, are split, if the caller's workspace holds the parts.  The host
  // knows how many keys there are, not how they are spread.  64 queries a sequence, 4 heads to a key head, d 128, whole and split:
  // one sequence of 1024, 2048, 16384 keys, 4 key heads 23.6 and 23.6, 37.9 and 25.1, 237 and 32.5 us; 4 sequences (36 pieces) of
  // 512, 1024, 4096 keys 16.4 and 24.6, 23.6 and 26.4, 66.6 and 28.6; 8 key heads and 8 sequences (136 pieces) of 512, 2048, 8192
  // keys 17.9 and 35.8, 39.7 and 51.3, 129 and 97; 16 sequences (264 pieces, not split) of 4096 keys 75.8 and 128.  So even
  // short sequences lose up to some 30 us by the rule, and one long one among them gains hundreds.
  const bool split = a.parts && all <= kSplitBelow && pieces <= kMostSplit && a.S <= kMostSplit && a.Tk >= kSplitKeys;
  const int grid = split ? sms : (int)(all < sms ? all : sms), least = split ? kLeastTiles : 0;
  prompt_tc_kernel<D><<<grid, kThreads, prompt_smem<D>(), st>>>(tmQ, tmK, tmV, a, (int)pieces, least, a.parts);
  if (cudaGetLastError() != cudaSuccess) return AVQ_ERR_CUDA;
  if (!split) return AVQ_OK;
  return cuda_ok(launch_pdl(prompt_join_kernel<D>, dim3((unsigned)all, 2 * kTile / kJoinRows), dim3(32 * kJoinWarps), 0, st, true, a, (int)pieces,
                            least, grid, (const float*)a.parts));
}

}  // namespace

size_t tc_prompt_part_bytes(int d) { return sizeof(float) * 2 * kPromptCtas * (size_t)part_floats(d); }
avq_status tc_prompt(const PromptArgs& a, cudaStream_t st) { return a.d == 64 ? launch<64>(a, st) : launch<128>(a, st); }

}  // namespace exact
}  // namespace avq
