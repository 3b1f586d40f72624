// C ABI of the exact operators: argument validation and dispatch.  The kernels live in avq_exact_simt.cu (CUDA cores,
// and the joining of split sequences), avq_tc_prompt.cu, avq_tc_prompt_f32.cu and avq_tc_cached.cu (tensor cores) and avq_cache.cu (rows into and out of a cache).
#include "avq_exact.cuh"

namespace avq {
namespace exact {
namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

avq_status validate_cache(const avq_cache* c) {
  if (!c) return AVQ_ERR_NULL;
  if (c->pages <= 0 || c->page <= 0 || c->Hk <= 0 || c->d <= 0) return AVQ_ERR_SHAPE;
  if (c->dtype != AVQ_F32 && c->dtype != AVQ_BF16) return AVQ_ERR_SHAPE;
  if (c->bits != 4 && c->bits != (c->dtype == AVQ_F32 ? 32 : 16)) return AVQ_ERR_SHAPE;
  if (c->d % 8 != 0 || c->d > 256 || (c->bits == 4 && c->d % 32 != 0)) return AVQ_ERR_UNSUPPORTED;
  if (c->page % 16 != 0 || c->page > 1024 || c->Hk > 65535) return AVQ_ERR_UNSUPPORTED;
  if ((int64_t)c->pages * c->page >= (int64_t)1 << 31) return AVQ_ERR_UNSUPPORTED;
  return AVQ_OK;
}
avq_status validate_heads(const avq_heads* h) {
  if (!h) return AVQ_ERR_NULL;
  if (h->H <= 0 || h->Hk <= 0 || h->d <= 0 || h->H % h->Hk != 0) return AVQ_ERR_SHAPE;
  if (h->dtype != AVQ_F32 && h->dtype != AVQ_BF16) return AVQ_ERR_SHAPE;
  if (!isfinite(h->scale)) return AVQ_ERR_SHAPE;
  if (h->flags & ~(uint32_t)(AVQ_FLAG_SIMT | AVQ_FLAG_CAUSAL)) return AVQ_ERR_SHAPE;
  if (h->d % 8 != 0 || h->d > 256 || h->H > 65535) return AVQ_ERR_UNSUPPORTED;
  return AVQ_OK;
}
// Rows of a call, tokens of a sequence: beyond, sums of row numbers and tiles would pass 32 bits.
bool too_many(int64_t rows) { return rows >= (int64_t)1 << 30; }
size_t es(int dtype) { return dtype == AVQ_F32 ? 4 : 2; }
// Rows of n heads, `stride` elements apart.
avq_status validate_rows(const void* p, int64_t stride, int64_t n, int d, int dtype) {
  if (!p) return AVQ_ERR_NULL;
  if (stride < n * d) return AVQ_ERR_SHAPE;
  if (stride >= (int64_t)1 << 31) return AVQ_ERR_UNSUPPORTED;
  if (!aligned16(p) || stride * (int64_t)es(dtype) % 16 != 0) return AVQ_ERR_ALIGN;
  return AVQ_OK;
}
avq_status validate_header(const void* header) {
  return reinterpret_cast<uintptr_t>(header) & 255u ? AVQ_ERR_ALIGN : AVQ_OK;
}
bool tensor_path(const avq_heads& h) { return !(h.flags & AVQ_FLAG_SIMT); }

avq_status validate_prompt(const avq_heads* h) {
  avq_status s = validate_heads(h);
  if (s != AVQ_OK) return s;
  if (h->dtype == AVQ_BF16 && tensor_path(*h) &&
      ((h->d != 64 && h->d != 128) || !(h->scale > 0.f) || h->H / h->Hk > 128))
    return AVQ_ERR_UNSUPPORTED;
  return AVQ_OK;
}
avq_status validate_cached(const avq_heads* h, int32_t B, int32_t nq) {
  avq_status s = validate_heads(h);
  if (s != AVQ_OK) return s;
  if (B < 0 || nq <= 0 || (h->flags & AVQ_FLAG_CAUSAL)) return AVQ_ERR_SHAPE;
  if (tensor_path(*h) && ((h->d != 64 && h->d != 128) || !(h->scale > 0.f))) return AVQ_ERR_UNSUPPORTED;
  if ((int64_t)B * nq * h->H >= (int64_t)1 << 31 || (int64_t)nq * (h->H / h->Hk) >= 1 << 20) return AVQ_ERR_UNSUPPORTED;
  return AVQ_OK;
}

size_t records_bytes(const avq_heads& h, int32_t B, int32_t nq) {   // a record for each segment, and up to 256 bytes
  const size_t segments = (size_t)B * h.Hk * (((size_t)nq * (h.H / h.Hk) + kRows - 1) / kRows);
  return (segments * sizeof(int2) + 255) / 256 * 256;
}

#define AVQ_TRY(call)                   \
  do {                                  \
    const avq_status s_ = (call);       \
    if (s_ != AVQ_OK) return s_;        \
  } while (0)

// The checks and dispatch of avq_prompt_attend and avq_prompt_attend_scratch; header and room are checked behind the rows.
avq_status prompt(const avq_heads* heads, const void* Q, int64_t q_stride, const void* K, int64_t k_stride, const void* V,
                  int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k, int32_t S, int32_t Tq, int32_t Tk, void* Y,
                  int64_t y_stride, float* lse_out, void* header, void* parts, size_t parts_bytes, void* stream) {
  AVQ_TRY(validate_prompt(heads));
  if (S < 0 || Tq < 0 || Tk < 0 || (!cu_k && Tk != Tq)) return AVQ_ERR_SHAPE;
  if (S == 0 || Tq == 0) return AVQ_OK;
  if (!cu_q) return AVQ_ERR_NULL;
  const avq_heads& h = *heads;
  AVQ_TRY(validate_rows(Q, q_stride, h.H, h.d, h.dtype));
  AVQ_TRY(validate_rows(Y, y_stride, h.H, h.d, h.dtype));
  if (Tk > 0) {
    AVQ_TRY(validate_rows(K, k_stride, h.Hk, h.d, h.dtype));
    AVQ_TRY(validate_rows(V, v_stride, h.Hk, h.d, h.dtype));
  }
  if (!header) return AVQ_ERR_WORKSPACE;
  AVQ_TRY(validate_header(header));
  AVQ_TRY(validate_header(parts));
  if (too_many(Tq) || too_many(Tk)) return AVQ_ERR_UNSUPPORTED;
  if (S > (1 << 16)) return AVQ_ERR_UNSUPPORTED;         // (every CTA passes over the sequences behind its own)
  const size_t room = avq_prompt_split_bytes(heads) - 256;
  const PromptArgs a = {Q, K, V, Y, lse_out, cu_q, cu_k, q_stride, k_stride, v_stride, y_stride, h.H, h.Hk, h.d, S, Tq, Tk,
                        (h.flags & AVQ_FLAG_CAUSAL) ? 1 : 0, h.scale, static_cast<int32_t*>(header),
                        room > 0 && parts_bytes >= room ? static_cast<float*>(parts) : nullptr};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!tensor_path(h) || (h.dtype == AVQ_F32 && h.d != 64 && h.d != 128)) return simt_prompt(a, h.dtype, st);
  return h.dtype == AVQ_F32 ? tc_prompt_f32(a, st) : tc_prompt(a, st);
}

// The same of avq_cache_attend and avq_cache_attend_scratch.
avq_status cached(const avq_heads* heads, const avq_cache* cache, const void* Q, int64_t q_stride, const int32_t* table,
                  int32_t table_pages, const int32_t* lens, int32_t B, int32_t nq, void* Y, int64_t y_stride, float* lse_out,
                  void* header, void* scratch, size_t scratch_bytes, void* stream) {
  AVQ_TRY(validate_cached(heads, B, nq));
  AVQ_TRY(validate_cache(cache));
  const avq_heads& h = *heads;
  const avq_cache& c = *cache;
  if (c.Hk != h.Hk || c.d != h.d || c.dtype != h.dtype || table_pages < 0) return AVQ_ERR_SHAPE;
  if (too_many((int64_t)table_pages * c.page)) return AVQ_ERR_UNSUPPORTED;
  if (B == 0) return AVQ_OK;
  if (!c.keys || !c.values || !lens || (table_pages > 0 && !table)) return AVQ_ERR_NULL;
  if (!aligned16(c.keys) || !aligned16(c.values)) return AVQ_ERR_ALIGN;
  AVQ_TRY(validate_rows(Q, q_stride, h.H, h.d, h.dtype));
  AVQ_TRY(validate_rows(Y, y_stride, h.H, h.d, h.dtype));
  if (!header || !scratch || scratch_bytes < avq_cache_attend_workspace_bytes(heads, B, nq) - 256) return AVQ_ERR_WORKSPACE;
  AVQ_TRY(validate_header(header));
  AVQ_TRY(validate_header(scratch));
  const CachedArgs a = {Q, c.keys, c.values, Y, lse_out, reinterpret_cast<float*>(static_cast<char*>(scratch) + records_bytes(h, B, nq)),
                        static_cast<int2*>(scratch),
                        table, lens, q_stride, y_stride, h.H, h.Hk, h.d, B, nq, c.pages, c.page, table_pages, h.scale,
                        static_cast<int32_t*>(header)};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return tensor_path(h) ? tc_cached(a, h.dtype, c.bits, st) : simt_cached(a, h.dtype, c.bits, st);
}

// What follows the header of a workspace of `bytes` bytes, its size in `rest` (0 and null if it does not even hold a header).
void* behind_header(void* workspace, size_t bytes, size_t* rest) {
  *rest = workspace && bytes >= 256 ? bytes - 256 : 0;
  return *rest ? static_cast<char*>(workspace) + 256 : nullptr;
}

}  // namespace
}  // namespace exact
}  // namespace avq

using namespace avq;
using namespace avq::exact;

extern "C" {

size_t avq_prompt_workspace_bytes(const avq_heads* heads) { return validate_prompt(heads) == AVQ_OK ? 256 : 0; }

size_t avq_prompt_split_bytes(const avq_heads* heads) {
  if (validate_prompt(heads) != AVQ_OK) return 0;
  return 256 + (heads->dtype == AVQ_BF16 && tensor_path(*heads) ? tc_prompt_part_bytes(heads->d) : 0);
}

avq_status avq_prompt_attend(const avq_heads* heads, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                             const void* V, int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k, int32_t S,
                             int32_t Tq, int32_t Tk, void* Y, int64_t y_stride, float* lse_out, void* workspace,
                             size_t workspace_bytes, void* stream) {
  size_t rest;
  void* parts = behind_header(workspace, workspace_bytes, &rest);
  return prompt(heads, Q, q_stride, K, k_stride, V, v_stride, cu_q, cu_k, S, Tq, Tk, Y, y_stride, lse_out,
                workspace_bytes >= 256 ? workspace : nullptr, parts, rest, stream);
}

avq_status avq_prompt_attend_scratch(const avq_heads* heads, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                             const void* V, int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k, int32_t S,
                             int32_t Tq, int32_t Tk, void* Y, int64_t y_stride, float* lse_out, void* header, void* scratch,
                             size_t scratch_bytes, void* stream) {
  return prompt(heads, Q, q_stride, K, k_stride, V, v_stride, cu_q, cu_k, S, Tq, Tk, Y, y_stride, lse_out, header, scratch,
                scratch_bytes, stream);
}

size_t avq_cache_bytes(const avq_cache* cache) {
  if (validate_cache(cache) != AVQ_OK) return 0;
  const size_t rows = (size_t)cache->pages * cache->Hk * cache->page;
  return rows * (cache->bits == 4 ? 5 * (size_t)cache->d / 8 : (size_t)cache->d * es(cache->dtype));
}

avq_status avq_cache_append(const avq_cache* cache, const void* K, int64_t k_stride, const void* V, int64_t v_stride,
                            const int32_t* slots, int32_t T, const avq_rotation* rot, const void* Q, int64_t q_stride,
                            int32_t H, void* Q_out, int64_t q_out_stride, void* header, void* stream) {
  AVQ_TRY(validate_cache(cache));
  const avq_cache& c = *cache;
  if (T < 0 || (Q && H <= 0)) return AVQ_ERR_SHAPE;
  if (rot) {
    if (rot->dims < 0 || rot->dims > c.d || rot->dims % 16 != 0 || rot->rows < 0) return AVQ_ERR_SHAPE;
    if (rot->dims > 0 && (!aligned16(rot->cos) || !aligned16(rot->sin))) return AVQ_ERR_ALIGN;
  }
  if (T == 0) return AVQ_OK;
  if (!c.keys || !c.values || !slots) return AVQ_ERR_NULL;
  if (!aligned16(c.keys) || !aligned16(c.values)) return AVQ_ERR_ALIGN;
  AVQ_TRY(validate_rows(K, k_stride, c.Hk, c.d, c.dtype));
  AVQ_TRY(validate_rows(V, v_stride, c.Hk, c.d, c.dtype));
  if (Q) {
    if (H > 65535) return AVQ_ERR_UNSUPPORTED;
    AVQ_TRY(validate_rows(Q, q_stride, H, c.d, c.dtype));
    AVQ_TRY(validate_rows(Q_out, q_out_stride, H, c.d, c.dtype));
  }
  AVQ_TRY(validate_header(header));
  const bool turn = rot && rot->dims > 0;
  if (turn && (!rot->cos || !rot->sin || !rot->pos)) return AVQ_ERR_NULL;
  const int heads = (Q ? H : 0) + 2 * c.Hk;
  const AppendArgs a = {K, V, Q, c.keys, c.values, Q_out, slots, turn ? rot->cos : nullptr, turn ? rot->sin : nullptr,
                        turn ? rot->pos : nullptr, k_stride, v_stride, q_stride, q_out_stride, T,
                        Q ? H : 0, c.Hk, c.d, c.page, c.pages, turn ? rot->rows : 0, turn ? rot->dims : 0,
                        turn ? rot->adjacent : 0, static_cast<int32_t*>(header)};
  if (too_many(T) || (int64_t)T * heads >= (int64_t)1 << 34) return AVQ_ERR_UNSUPPORTED;
  return cache_append(a, c.dtype, c.bits, static_cast<cudaStream_t>(stream));
}

avq_status avq_cache_read(const avq_cache* cache, const int32_t* slots, int32_t T, void* K, int64_t k_stride, void* V,
                          int64_t v_stride, void* header, void* stream) {
  AVQ_TRY(validate_cache(cache));
  const avq_cache& c = *cache;
  if (T < 0) return AVQ_ERR_SHAPE;
  if (T == 0) return AVQ_OK;
  if (!c.keys || !c.values || !slots) return AVQ_ERR_NULL;
  if (!aligned16(c.keys) || !aligned16(c.values)) return AVQ_ERR_ALIGN;
  AVQ_TRY(validate_rows(K, k_stride, c.Hk, c.d, c.dtype));
  AVQ_TRY(validate_rows(V, v_stride, c.Hk, c.d, c.dtype));
  AVQ_TRY(validate_header(header));
  const ReadArgs a = {c.keys, c.values, K, V, slots, k_stride, v_stride, T, c.Hk, c.d, c.page, c.pages,
                      static_cast<int32_t*>(header)};
  if (too_many(T) || (int64_t)T * 2 * c.Hk >= (int64_t)1 << 34) return AVQ_ERR_UNSUPPORTED;
  return cache_read(a, c.dtype, c.bits, static_cast<cudaStream_t>(stream));
}

size_t avq_cache_attend_workspace_bytes(const avq_heads* heads, int32_t B, int32_t nq) {
  if (validate_cached(heads, B, nq) != AVQ_OK) return 0;
  return 256 + records_bytes(*heads, B, nq) + sizeof(float) * 2 * kMaxCtas * (size_t)slot_floats(heads->d);
}

avq_status avq_cache_attend(const avq_heads* heads, const avq_cache* cache, const void* Q, int64_t q_stride,
                            const int32_t* table, int32_t table_pages, const int32_t* lens, int32_t B, int32_t nq, void* Y,
                            int64_t y_stride, float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  size_t rest;
  void* scratch = behind_header(workspace, workspace_bytes, &rest);
  return cached(heads, cache, Q, q_stride, table, table_pages, lens, B, nq, Y, y_stride, lse_out, workspace, scratch, rest, stream);
}

avq_status avq_cache_attend_scratch(const avq_heads* heads, const avq_cache* cache, const void* Q, int64_t q_stride,
                            const int32_t* table, int32_t table_pages, const int32_t* lens, int32_t B, int32_t nq, void* Y,
                            int64_t y_stride, float* lse_out, void* header, void* scratch, size_t scratch_bytes, void* stream) {
  return cached(heads, cache, Q, q_stride, table, table_pages, lens, B, nq, Y, y_stride, lse_out, header, scratch, scratch_bytes, stream);
}

}  // extern "C"
