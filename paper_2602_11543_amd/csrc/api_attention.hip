// C ABI of the attention half of a block: argument checks ahead of any launch.
#include "kernels.h"

using namespace spes;

namespace {

bool dtype_ok(int dtype) { return dtype == SPES_F32 || dtype == SPES_BF16; }

constexpr int kMaxRopeDim = 256, kMaxHeadDim = 128, kMaxHeads = 1024;
constexpr long kMaxRopeHeads = 1l << 22;         // a token's elements, and the number of a head some rounds behind the last one, fit 32 bits
constexpr long kMaxRow = 1l << 20, kMaxGroup = 1l << 28;          // in elements: 32-bit byte offsets from a tile's first row

constexpr long kMaxRows = (1l << 31) - (1l << 16);               // the number of a row a few tiles behind the last one still fits 32 bits
// A launch has fewer than 2^32 threads: blocks of 256 for 128 rows of queries, or in the backward for 64 keys, and one more for each sequence
constexpr long kMaxQueryRows = 1l << 30, kMaxKeyRows = 1l << 29, kMaxSeqs = 1l << 22;

// A score is the scale times a sum of up to 128 products, each off by as much as 2^-126 where it is denormal: under a larger scale by more than 2^-24 in all
constexpr float kMostScale = 0x1p95f;
// The bf16 gradients of keys sum scores on top of -lse / scale, and ln of 2^31 keys over this is 2^124.4 (behind it lse / scale is a score's own sum of products)
constexpr float kLeastScale = 0x1p-120f;

bool stride_ok(int64_t stride, int dtype) { return stride % (dtype == SPES_F32 ? 4 : 8) == 0; }

int qk_supported(const spes_qk_shape* p) {
  if (p == nullptr) return SPES_EINVAL;
  if (p->T < 0 || p->heads < 1 || p->kv_heads < 1 || p->head_dim < 1 || p->rot_dim < 0 || p->rot_dim > p->head_dim || p->n_pos < 0 ||
      !dtype_ok(p->dtype) || !(p->eps >= 0.f))
    return SPES_EINVAL;
  if (p->head_dim % 8 != 0 || p->head_dim > kMaxRopeDim || p->rot_dim % 16 != 0) return SPES_ESHAPE;
  const long heads = (long)p->heads + p->kv_heads;
  if (heads > kMaxRopeHeads || heads * p->T >= 1l << 31) return SPES_ESHAPE;
  if (p->q_row < (long)p->heads * p->head_dim || p->k_row < (long)p->kv_heads * p->head_dim) return SPES_EINVAL;
  return SPES_OK;
}
QkShape shape_of(const spes_qk_shape& p) {
  return {p.q_row, p.k_row, p.T, p.heads, p.kv_heads, p.head_dim, p.rot_dim, p.interleaved != 0, p.n_pos, p.eps};
}
// table and positions
bool angles_ok(const spes_qk_shape& p, const float* table, const int32_t* pos) {
  if (p.rot_dim == 0) return table == nullptr && pos == nullptr;
  return table != nullptr && p.n_pos >= 1 && (pos != nullptr || p.n_pos >= p.T);
}

int attn_supported(const spes_attn_shape* p) {
  if (p == nullptr) return SPES_EINVAL;
  if (p->n_seq < 0 || p->q_rows < 0 || p->k_rows < 0 || p->heads < 1 || p->kv_heads < 1 || p->head_dim < 1 || !dtype_ok(p->dtype) || p->window < 0 ||
      !(p->scale > 0.f && p->scale <= kMostScale))
    return SPES_EINVAL;
  if (p->heads % p->kv_heads != 0 || (p->window > 0 && !p->causal)) return SPES_EINVAL;
  if (p->head_dim % 8 != 0 || p->head_dim > kMaxHeadDim || p->heads > kMaxHeads) return SPES_ESHAPE;
  for (const int64_t stride : {p->q_row, p->q_head, p->k_row, p->k_head, p->v_row, p->v_head})
    if (stride < p->head_dim) return SPES_EINVAL;
  if (p->q_row > kMaxRow || p->k_row > kMaxRow || p->v_row > kMaxRow) return SPES_ESHAPE;
  if (p->q_head > kMaxGroup / (p->heads / p->kv_heads)) return SPES_ESHAPE;
  if ((long)p->q_rows * p->heads > kMaxQueryRows || p->k_rows > kMaxRows || (long)p->n_seq * p->kv_heads > kMaxSeqs) return SPES_ESHAPE;
  for (const int64_t stride : {p->q_row, p->q_head, p->k_row, p->k_head, p->v_row, p->v_head})
    if (!stride_ok(stride, p->dtype)) return SPES_EALIGN;
  return SPES_OK;
}
// The backward writes tensors that are laid out as q, k and v are: no two of their elements in one place
bool apart(int64_t row, int64_t head, long rows, long heads, long dim) { return row >= (heads - 1) * head + dim || head >= (rows - 1) * row + dim; }
int attn_bwd_supported(const spes_attn_shape* p) {
  const int rc = attn_supported(p);
  if (rc != SPES_OK) return rc;
  if (!apart(p->q_row, p->q_head, p->q_rows, p->heads, p->head_dim) || !apart(p->k_row, p->k_head, p->k_rows, p->kv_heads, p->head_dim) ||
      !apart(p->v_row, p->v_head, p->k_rows, p->kv_heads, p->head_dim))
    return SPES_EINVAL;
  if (p->dtype == SPES_BF16 && p->scale < kLeastScale) return SPES_EINVAL;
  return (long)p->k_rows * p->kv_heads > kMaxKeyRows ? SPES_ESHAPE : SPES_OK;
}
AttnShape shape_of(const spes_attn_shape& p, const int32_t* q_start, const int32_t* k_start, const int32_t* k_len) {
  return {q_start, k_start, k_len, p.q_row, p.q_head, p.k_row, p.k_head, p.v_row, p.v_head, p.n_seq, p.q_rows, p.k_rows, p.heads, p.kv_heads,
          p.heads / p.kv_heads, p.head_dim, p.causal != 0, p.window, p.scale};
}
bool element_aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

extern "C" {

SPES_API int spes_qk_rope_fwd(const spes_qk_shape* shape, const void* q, const void* k, const void* q_weight, const void* k_weight, const float* table,
                              const int32_t* pos, void* q_out, void* k_out, void* stream) {
  const int rc = qk_supported(shape);
  if (rc != SPES_OK) return rc;
  if ((q_weight == nullptr) != (k_weight == nullptr) || !angles_ok(*shape, table, pos)) return SPES_EINVAL;
  if (!stride_ok(shape->q_row, shape->dtype) || !stride_ok(shape->k_row, shape->dtype)) return SPES_EALIGN;
  if (shape->T == 0) return SPES_OK;
  if (!q || !k || !q_out || !k_out) return SPES_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_weight) || !aligned16(k_weight) || !aligned16(table) || !aligned16(pos) || !aligned16(q_out) ||
      !aligned16(k_out))
    return SPES_EALIGN;
  return launch_qk_rope_fwd(shape->dtype, shape_of(*shape), q, k, q_weight, k_weight, table, pos, q_out, k_out, static_cast<hipStream_t>(stream));
}

SPES_API size_t spes_qk_rope_scratch_bytes(const spes_qk_shape* shape) {
  return qk_supported(shape) == SPES_OK ? qk_rope_scratch_bytes(shape_of(*shape)) : 0;
}

SPES_API int spes_qk_rope_bwd(const spes_qk_shape* shape, const void* dq, const void* dk, const void* q, const void* k, const void* q_weight,
                              const void* k_weight, const float* table, const int32_t* pos, void* dq_in, void* dk_in, float* d_q_weight,
                              float* d_k_weight, int32_t accumulate, void* scratch, void* stream) {
  const int rc = qk_supported(shape);
  if (rc != SPES_OK) return rc;
  if ((q_weight == nullptr) != (k_weight == nullptr) || (d_q_weight == nullptr) != (d_k_weight == nullptr) || !angles_ok(*shape, table, pos))
    return SPES_EINVAL;
  if (d_q_weight && (!q_weight || !scratch)) return SPES_EINVAL;
  if (!stride_ok(shape->q_row, shape->dtype) || !stride_ok(shape->k_row, shape->dtype)) return SPES_EALIGN;
  if (shape->T == 0 && !d_q_weight) return SPES_OK;
  if (shape->T > 0 && (!dq || !dk || !dq_in || !dk_in || (q_weight && (!q || !k)))) return SPES_EINVAL;
  for (const void* p : {dq, dk, q, k, q_weight, k_weight, static_cast<const void*>(table), static_cast<const void*>(pos), static_cast<const void*>(dq_in),
                        static_cast<const void*>(dk_in), static_cast<const void*>(d_q_weight), static_cast<const void*>(d_k_weight),
                        static_cast<const void*>(scratch)})
    if (!aligned16(p)) return SPES_EALIGN;
  return launch_qk_rope_bwd(shape->dtype, shape_of(*shape), dq, dk, q, k, q_weight, k_weight, table, pos, dq_in, dk_in, d_q_weight, d_k_weight,
                            accumulate != 0, static_cast<float*>(scratch), static_cast<hipStream_t>(stream));
}

SPES_API size_t spes_attn_scratch_bytes(const spes_attn_shape* shape, int32_t backward) {
  if ((backward ? attn_bwd_supported(shape) : attn_supported(shape)) != SPES_OK) return 0;
  const AttnShape a = shape_of(*shape, nullptr, nullptr, nullptr);
  return backward ? attn_bwd_scratch_bytes(shape->dtype, a) : attn_fwd_scratch_bytes(shape->dtype, a);
}

SPES_API int spes_attn_fwd(const spes_attn_shape* shape, const void* q, const void* k, const void* v, const int32_t* q_start, const int32_t* k_start,
                           const int32_t* k_len, void* o, float* lse, void* scratch, void* stream) {
  const int rc = attn_supported(shape);
  if (rc != SPES_OK) return rc;
  if (shape->n_seq == 0 || shape->q_rows == 0) return SPES_OK;
  if (!q || !q_start || !k_start || !o || !lse || !scratch || (shape->k_rows > 0 && (!k || !v))) return SPES_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !element_aligned4(q_start) || !element_aligned4(k_start) || !element_aligned4(k_len) ||
      !aligned16(o) || !aligned16(lse) || !aligned16(scratch))
    return SPES_EALIGN;
  return launch_attn_fwd(shape->dtype, shape_of(*shape, q_start, k_start, k_len), q, k, v, o, lse, scratch, static_cast<hipStream_t>(stream));
}

SPES_API int spes_attn_bwd(const spes_attn_shape* shape, const void* d_o, const void* q, const void* k, const void* v, const int32_t* q_start,
                           const int32_t* k_start, const int32_t* k_len, const void* o, const float* lse, void* dq, void* dk, void* dv, void* scratch,
                           void* stream) {
  const int rc = attn_bwd_supported(shape);
  if (rc != SPES_OK) return rc;
  if (shape->n_seq == 0 || (shape->q_rows == 0 && shape->k_rows == 0)) return SPES_OK;
  if (!q_start || !k_start || !scratch || (shape->q_rows > 0 && (!d_o || !q || !o || !lse || !dq)) || (shape->k_rows > 0 && (!k || !v || !dk || !dv)))
    return SPES_EINVAL;
  for (const void* p : {d_o, q, k, v, o, static_cast<const void*>(lse), static_cast<const void*>(dq), static_cast<const void*>(dk),
                        static_cast<const void*>(dv), static_cast<const void*>(scratch)})
    if (!aligned16(p)) return SPES_EALIGN;
  if (!element_aligned4(q_start) || !element_aligned4(k_start) || !element_aligned4(k_len)) return SPES_EALIGN;
  return launch_attn_bwd(shape->dtype, shape_of(*shape, q_start, k_start, k_len), d_o, q, k, v, o, lse, dq, dk, dv, scratch,
                         static_cast<hipStream_t>(stream));
}

}  // extern "C"
