// C entry points of the token operators: argument checks, then one launcher.
// Every check is made on the host before anything is enqueued.
#include <string>

#include "../../include/ncodec.h"
#include "areas.hpp"
#include "tokens.hpp"

namespace {

using nc::all_apart;
using nc::Area;

// Records the message; nothing is thrown across the C entry.
ncodec_status set_error(ncodec_status st, const char* where, const char* why, size_t bytes = 0) noexcept {
  try {
    return nc::set_error(st, std::string(where) + ": " + why + (bytes ? std::to_string(bytes) + " bytes" : ""));
  } catch (...) {
    return st;
  }
}

constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr int64_t kMaxPositions = (int64_t)1 << 30;  // of a sequence that softmax attention sees: 32-bit counts past its end

bool dtype_ok(int32_t d) { return d == NCODEC_DTYPE_FP16 || d == NCODEC_DTYPE_BF16; }
bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }
bool stride_ok(int64_t s) { return s >= 0 && s <= kMaxStride; }

ncodec_status finish(hipError_t e, const char* where) {
  if (e == hipSuccess) return NCODEC_OK;
  return set_error(NCODEC_EHIP, where, hipGetErrorString(e));
}

// Why a shape is refused, or NULL.
const char* linear_fault(const ncodec_linear_shape& s, ncodec_status* st) {
  *st = NCODEC_EINVAL;
  if (!dtype_ok(s.dtype)) return "dtype is not an ncodec_dtype";
  if (s.act < NCODEC_ACT_NONE || s.act > NCODEC_ACT_GELU) return "act is not an ncodec_act";
  if (s.gated != 0 && s.gated != 1) return "gated must be 0 or 1";
  if (s.reserved) return "reserved must be 0";
  *st = NCODEC_ESHAPE;
  if (s.m < 0 || s.m >= kMaxRows) return "m must be in [0, 2^31)";
  if (s.n < 1 || s.n > (1 << 20) || s.k < 1 || s.k > (1 << 20)) return "n and k must be in [1, 2^20]";
  if (s.ldx < s.k || s.ldw < s.k || s.ldy < s.n) return "a row stride is below its row";
  if (!stride_ok(s.ldx) || !stride_ok(s.ldw) || !stride_ok(s.ldy)) return "a row stride is above 2^40";
  return nullptr;
}

const char* qk_fault(const ncodec_qk_shape& s, ncodec_status* st) {
  *st = NCODEC_EINVAL;
  if (!dtype_ok(s.dtype)) return "dtype is not an ncodec_dtype";
  if (s.norm != 0 && s.norm != 1) return "norm must be 0 or 1";
  if (s.interleaved != 0 && s.interleaved != 1) return "interleaved must be 0 or 1";
  if (s.reserved) return "reserved must be 0";
  if (s.norm && !(s.eps >= 0.f && s.eps < __builtin_huge_valf())) return "eps must be finite and not negative";
  *st = NCODEC_ESHAPE;
  if (s.tokens < 0 || s.tokens >= kMaxRows) return "tokens must be in [0, 2^31)";
  if (s.q_heads < 0 || s.q_heads > 4096 || s.k_heads < 0 || s.k_heads > 4096) return "heads must be in [0, 4096]";
  if (s.head_dim < 1 || s.head_dim > 256) return "head_dim must be in [1, 256]";
  if (s.axes < 0 || s.axes > 3) return "axes must be in [0, 3]";
  int64_t pairs = 0;
  for (int a = 0; a < 3; ++a) {
    if (s.section[a] < 0 || (a >= s.axes && s.section[a])) return "a section is negative, or given to no axis";
    pairs += s.section[a];
  }
  if (2 * pairs > s.head_dim) return "the sections hold more pairs than head_dim / 2";
  const int64_t strides[8] = {s.q_token_stride,  s.q_head_stride,  s.k_token_stride,  s.k_head_stride,
                              s.qo_token_stride, s.qo_head_stride, s.ko_token_stride, s.ko_head_stride};
  for (int64_t v : strides)
    if (!stride_ok(v)) return "a stride is negative or above 2^40";
  if ((s.tokens > 1 && s.q_heads && s.qo_token_stride < s.head_dim) || (s.q_heads > 1 && s.qo_head_stride < s.head_dim) ||
      (s.tokens > 1 && s.k_heads && s.ko_token_stride < s.head_dim) || (s.k_heads > 1 && s.ko_head_stride < s.head_dim))
    return "an output stride is below head_dim";
  return nullptr;
}

const char* decay_fault(const ncodec_decay_shape& s, ncodec_status* st) {
  *st = NCODEC_EINVAL;
  if (!dtype_ok(s.dtype)) return "dtype is not an ncodec_dtype";
  if (!(s.scale > -__builtin_huge_valf() && s.scale < __builtin_huge_valf())) return "scale must be finite";
  *st = NCODEC_ESHAPE;
  if (s.tokens < 0 || s.tokens >= kMaxRows) return "tokens must be in [0, 2^31)";
  if (s.heads < 1 || s.heads > 4096 || s.kv_heads < 1 || s.kv_heads > 4096) return "heads must be in [1, 4096]";
  if (s.heads % s.kv_heads) return "heads must be a multiple of kv_heads";
  if (s.head_dim < 1 || s.head_dim > 128 || s.value_dim < 1 || s.value_dim > 128)
    return "head_dim and value_dim must be in [1, 128]";
  if (s.batch < 0 || s.batch >= (1 << 24) || s.batch * s.heads >= (1 << 24)) return "batch * heads must be below 2^24";
  const int64_t strides[12] = {s.q_batch_stride, s.q_token_stride, s.q_head_stride, s.k_batch_stride,
                               s.k_token_stride, s.k_head_stride,  s.v_batch_stride, s.v_token_stride,
                               s.v_head_stride,  s.o_batch_stride, s.o_token_stride, s.o_head_stride};
  for (int64_t v : strides)
    if (!stride_ok(v)) return "a stride is negative or above 2^40";
  if ((s.batch > 1 && s.o_batch_stride < s.value_dim) || (s.tokens > 1 && s.o_token_stride < s.value_dim) ||
      (s.heads > 1 && s.o_head_stride < s.value_dim))
    return "an output stride is below value_dim";
  return nullptr;
}

const char* heads_fault(int64_t heads, int64_t kv_heads, int64_t head_dim, int64_t value_dim) {
  if (heads < 1 || heads > 4096 || kv_heads < 1 || kv_heads > 4096) return "heads must be in [1, 4096]";
  if (heads % kv_heads) return "heads must be a multiple of kv_heads";
  if (head_dim < 1 || head_dim > 128 || value_dim < 1 || value_dim > 128)
    return "head_dim and value_dim must be in [1, 128]";
  return nullptr;
}

// Softmax attention takes the scale times log2(e): room for that.
bool scale_ok(float f) { return f >= -0x1p100f && f <= 0x1p100f; }

const char* window_fault(const ncodec_window_shape& s, ncodec_status* st) {
  *st = NCODEC_EINVAL;
  if (!dtype_ok(s.dtype)) return "dtype is not an ncodec_dtype";
  if (!scale_ok(s.scale)) return "scale must be in [-2^100, 2^100]";
  *st = NCODEC_ESHAPE;
  if (s.tokens < 0 || s.tokens > kMaxPositions) return "tokens must be in [0, 2^30]";
  if (s.window < 0 || s.window >= kMaxRows || s.sinks < 0 || s.sinks >= kMaxRows)
    return "window and sinks must be in [0, 2^31)";
  if (const char* why = heads_fault(s.heads, s.kv_heads, s.head_dim, s.value_dim)) return why;
  if (s.batch < 0 || s.batch >= (1 << 24) || s.batch * s.heads >= (1 << 24)) return "batch * heads must be below 2^24";
  const int64_t strides[12] = {s.q_batch_stride, s.q_token_stride, s.q_head_stride, s.k_batch_stride,
                               s.k_token_stride, s.k_head_stride,  s.v_batch_stride, s.v_token_stride,
                               s.v_head_stride,  s.o_batch_stride, s.o_token_stride, s.o_head_stride};
  for (int64_t v : strides)
    if (!stride_ok(v)) return "a stride is negative or above 2^40";
  if ((s.batch > 1 && s.o_batch_stride < s.value_dim) || (s.tokens > 1 && s.o_token_stride < s.value_dim) ||
      (s.heads > 1 && s.o_head_stride < s.value_dim))
    return "an output stride is below value_dim";
  return nullptr;
}

// `written`: rows of the cache have to be different ones.
const char* cache_fault(const ncodec_cache_shape& c, bool written, ncodec_status* st) {
  *st = NCODEC_EINVAL;
  if (!dtype_ok(c.dtype)) return "dtype is not an ncodec_dtype";
  if (c.reserved) return "reserved must be 0";
  *st = NCODEC_ESHAPE;
  if (const char* why = heads_fault(c.kv_heads, c.kv_heads, c.head_dim, c.value_dim)) return why;
  if (c.page_size < 1 || c.page_size > 4096 || (c.page_size & (c.page_size - 1)))
    return "page_size must be a power of two up to 4096";
  if (c.pages < 0 || c.pages >= kMaxRows) return "pages must be in [0, 2^31)";
  const int64_t strides[6] = {c.k_page_stride, c.k_token_stride, c.k_head_stride,
                              c.v_page_stride, c.v_token_stride, c.v_head_stride};
  for (int64_t v : strides)
    if (!stride_ok(v)) return "a stride is negative or above 2^40";
  for (int i = 0; written && i < 6; ++i) {
    const int64_t count = i % 3 == 0 ? c.pages : i % 3 == 1 ? c.page_size : c.kv_heads;
    if (count > 1 && strides[i] < (i < 3 ? c.head_dim : c.value_dim)) return "a stride of the cache is below its row";
  }
  return nullptr;
}

const char* table_fault(const ncodec_cache_shape& c, int64_t batch, int64_t columns, int64_t stride) {
  if (batch < 0 || batch >= (1 << 24) || batch * c.kv_heads >= (1 << 24)) return "batch * heads must be below 2^24";
  if (columns < 0 || columns > kMaxPositions || columns * c.page_size > kMaxPositions)
    return "columns * page_size must be in [0, 2^30]";
  if (!stride_ok(stride)) return "a stride is negative or above 2^40";
  return nullptr;
}

const char* paged_fault(const ncodec_cache_shape& c, const ncodec_paged_shape& s, ncodec_status* st) {
  if (const char* why = cache_fault(c, false, st)) return why;
  *st = NCODEC_EINVAL;
  if (!scale_ok(s.scale)) return "scale must be in [-2^100, 2^100]";
  *st = NCODEC_ESHAPE;
  if (const char* why = heads_fault(s.heads, c.kv_heads, c.head_dim, c.value_dim)) return why;
  if (s.window < 0 || s.window >= kMaxRows || s.sinks < 0 || s.sinks >= kMaxRows)
    return "window and sinks must be in [0, 2^31)";
  if (const char* why = table_fault(c, s.batch, s.columns, s.table_stride)) return why;
  if (s.batch * s.heads >= (1 << 24)) return "batch * heads must be below 2^24";
  if (!stride_ok(s.q_batch_stride) || !stride_ok(s.q_head_stride) || !stride_ok(s.o_batch_stride) || !stride_ok(s.o_head_stride))
    return "a stride is negative or above 2^40";
  if ((s.batch > 1 && s.o_batch_stride < c.value_dim) || (s.heads > 1 && s.o_head_stride < c.value_dim))
    return "an output stride is below value_dim";
  return nullptr;
}

const char* append_fault(const ncodec_cache_shape& c, const ncodec_append_shape& s, ncodec_status* st) {
  if (const char* why = cache_fault(c, true, st)) return why;
  if (const char* why = table_fault(c, s.batch, s.columns, s.table_stride)) return why;
  if (s.tokens < 0 || s.tokens >= kMaxRows) return "tokens must be in [0, 2^31)";
  const int64_t strides[6] = {s.k_batch_stride, s.k_token_stride, s.k_head_stride,
                              s.v_batch_stride, s.v_token_stride, s.v_head_stride};
  for (int64_t v : strides)
    if (!stride_ok(v)) return "a stride is negative or above 2^40";
  return nullptr;
}

const char* evict_fault(const ncodec_cache_shape& c, const ncodec_evict_shape& s, ncodec_status* st) {
  if (const char* why = cache_fault(c, true, st)) return why;
  if (const char* why = table_fault(c, s.batch, s.columns, s.table_stride)) return why;
  if (const char* why = table_fault(c, s.batch, s.new_columns, s.new_table_stride)) return why;
  if (s.keep < 1 || s.keep > s.new_columns * c.page_size) return "keep must be in [1, new_columns * page_size]";
  if (s.sinks < 0 || s.recent < 0 || s.sinks > s.keep || s.recent > s.keep - s.sinks)
    return "sinks + recent must be in [0, keep]";
  return nullptr;
}

Area table_area(const int32_t* d, int64_t batch, int64_t columns, int64_t stride) {
  return Area(d, 2 * columns, {batch, 2 * stride});  // in 16-bit units, as all strided operands
}
Area k_area(const ncodec_cache_shape& c, const void* d) {
  return Area(d, c.head_dim, {c.pages, c.k_page_stride, c.page_size, c.k_token_stride, c.kv_heads, c.k_head_stride});
}
Area v_area(const ncodec_cache_shape& c, const void* d) {
  return Area(d, c.value_dim, {c.pages, c.v_page_stride, c.page_size, c.v_token_stride, c.kv_heads, c.v_head_stride});
}

}  // namespace

extern "C" ncodec_status ncodec_linear(const ncodec_linear_shape* shape, const void* d_x, const void* d_w,
                                       const void* d_b, const void* d_r, void* d_y, void* hip_stream) {
  if (!shape) return set_error(NCODEC_EINVAL, "linear", "shape is NULL");
  ncodec_status st;
  if (const char* why = linear_fault(*shape, &st)) return set_error(st, "linear", why);
  if (d_r && (shape->ldr < shape->n || !stride_ok(shape->ldr)))
    return set_error(NCODEC_ESHAPE, "linear", "ldr is below n or above 2^40");
  if (shape->m == 0) return NCODEC_OK;
  if (!d_x || !d_w || !d_y) return set_error(NCODEC_EINVAL, "linear", "d_x, d_w and d_y must be non-NULL");
  if (!aligned(d_x, 2) || !aligned(d_w, 2) || !aligned(d_y, 2) || !aligned(d_b, 2) || !aligned(d_r, 2))
    return set_error(NCODEC_EINVAL, "linear", "a pointer is not aligned to an element");
  if (d_r == d_y && d_r && shape->ldr != shape->ldy)
    return set_error(NCODEC_EINVAL, "linear", "d_y is d_r, but ldy is not ldr");
  {
    const ncodec_linear_shape& s = *shape;
    const int64_t nw = s.n * (s.gated ? 2 : 1);
    const Area y(d_y, s.n, {s.m, s.ldy}), r(d_r == d_y ? nullptr : d_r, s.n, {s.m, s.ldr});
    if (!all_apart(y, {Area(d_x, s.k, {s.m, s.ldx}), Area(d_w, s.k, {nw, s.ldw}), Area(d_b, nw, 2), r}))
      return set_error(NCODEC_EINVAL, "linear", "d_y overlaps an input");
  }
  return finish(nc::launch_linear({*shape, d_x, d_w, d_b, d_r, d_y}, (hipStream_t)hip_stream), "linear");
}

extern "C" ncodec_status ncodec_qk_norm_rope(const ncodec_qk_shape* shape, const void* d_q, const void* d_k,
                                             const void* d_wq, const void* d_wk, const int32_t* d_pos,
                                             const float* d_freq, void* d_qo, void* d_ko, void* hip_stream) {
  if (!shape) return set_error(NCODEC_EINVAL, "qk_norm_rope", "shape is NULL");
  ncodec_status st;
  if (const char* why = qk_fault(*shape, &st)) return set_error(st, "qk_norm_rope", why);
  if (shape->tokens == 0 || shape->q_heads + shape->k_heads == 0) return NCODEC_OK;
  if (shape->q_heads && (!d_q || !d_qo)) return set_error(NCODEC_EINVAL, "qk_norm_rope", "d_q and d_qo must be non-NULL");
  if (shape->k_heads && (!d_k || !d_ko)) return set_error(NCODEC_EINVAL, "qk_norm_rope", "d_k and d_ko must be non-NULL");
  const bool rot = shape->section[0] + shape->section[1] + shape->section[2] > 0;
  if (rot && (!d_pos || !d_freq)) return set_error(NCODEC_EINVAL, "qk_norm_rope", "d_pos and d_freq must be non-NULL");
  if (!aligned(d_q, 2) || !aligned(d_k, 2) || !aligned(d_qo, 2) || !aligned(d_ko, 2) || !aligned(d_wq, 2) ||
      !aligned(d_wk, 2) || (rot && (!aligned(d_pos, 4) || !aligned(d_freq, 4))))
    return set_error(NCODEC_EINVAL, "qk_norm_rope", "a pointer is not aligned to an element");
  {
    const ncodec_qk_shape& s = *shape;
    const Area q(d_q, s.head_dim, {s.tokens, s.q_token_stride, s.q_heads, s.q_head_stride}),
        k(d_k, s.head_dim, {s.tokens, s.k_token_stride, s.k_heads, s.k_head_stride}),
        qo(d_qo, s.head_dim, {s.tokens, s.qo_token_stride, s.q_heads, s.qo_head_stride}),
        ko(d_ko, s.head_dim, {s.tokens, s.ko_token_stride, s.k_heads, s.ko_head_stride});
    const Area wq(s.norm ? d_wq : nullptr, s.head_dim, 2), wk(s.norm ? d_wk : nullptr, s.head_dim, 2),
        pos(rot ? d_pos : nullptr, s.tokens * s.axes, 4),
        freq(rot ? d_freq : nullptr, s.section[0] + s.section[1] + s.section[2], 4);
    const auto same = [&](const void* a, const void* b, int64_t heads, int64_t ta, int64_t tb, int64_t ha, int64_t hb) {
      return a == b && (s.tokens == 1 || ta == tb) && (heads == 1 || ha == hb);
    };
    const Area none(nullptr, 0, 2);
    const bool q_in_place = same(d_q, d_qo, s.q_heads, s.q_token_stride, s.qo_token_stride, s.q_head_stride, s.qo_head_stride),
               k_in_place = same(d_k, d_ko, s.k_heads, s.k_token_stride, s.ko_token_stride, s.k_head_stride, s.ko_head_stride);
    if (!all_apart(qo, {q_in_place ? none : q, k, ko, wq, wk, pos, freq}) ||
        !all_apart(ko, {k_in_place ? none : k, q, wq, wk, pos, freq}))
      return set_error(NCODEC_EINVAL, "qk_norm_rope", "an output overlaps an input that it is not, or the other output");
  }
  return finish(nc::launch_qk_norm_rope({*shape, d_q, d_k, d_wq, d_wk, d_pos, d_freq, d_qo, d_ko},
                                        (hipStream_t)hip_stream),
                "qk_norm_rope");
}

extern "C" size_t ncodec_decay_attention_workspace_bytes(const ncodec_decay_shape* shape) {
  ncodec_status st;
  if (!shape || decay_fault(*shape, &st)) return 0;
  return nc::decay_workspace_bytes(*shape);
}

extern "C" ncodec_status ncodec_decay_attention(const ncodec_decay_shape* shape, const void* d_q, const void* d_k,
                                                const void* d_v, const float* d_log_decay, const int32_t* d_lengths,
                                                const float* d_state_in, float* d_state_out, void* d_o,
                                                void* d_workspace, size_t ws_bytes, void* hip_stream) {
  if (!shape) return set_error(NCODEC_EINVAL, "decay_attention", "shape is NULL");
  ncodec_status st;
  if (const char* why = decay_fault(*shape, &st)) return set_error(st, "decay_attention", why);
  if (shape->batch == 0) return NCODEC_OK;
  if (!d_log_decay) return set_error(NCODEC_EINVAL, "decay_attention", "d_log_decay is NULL");
  if (shape->tokens > 0 && (!d_q || !d_k || !d_v || !d_o))
    return set_error(NCODEC_EINVAL, "decay_attention", "d_q, d_k, d_v and d_o must be non-NULL");
  if (!aligned(d_q, 2) || !aligned(d_k, 2) || !aligned(d_v, 2) || !aligned(d_o, 2) || !aligned(d_log_decay, 4) ||
      !aligned(d_lengths, 4) || !aligned(d_state_in, 4) || !aligned(d_state_out, 4))
    return set_error(NCODEC_EINVAL, "decay_attention", "a pointer is not aligned to an element");
  const size_t need = nc::decay_workspace_bytes(*shape);
  if (need && (!d_workspace || ws_bytes < need || !aligned(d_workspace, 256)))
    return set_error(NCODEC_ENOMEM, "decay_attention", "the workspace must be 256-byte aligned and hold ", need);
  {
    const ncodec_decay_shape& s = *shape;
    const Area q(d_q, s.head_dim, {s.batch, s.q_batch_stride, s.tokens, s.q_token_stride, s.heads, s.q_head_stride}),
        k(d_k, s.head_dim, {s.batch, s.k_batch_stride, s.tokens, s.k_token_stride, s.kv_heads, s.k_head_stride}),
        v(d_v, s.value_dim, {s.batch, s.v_batch_stride, s.tokens, s.v_token_stride, s.kv_heads, s.v_head_stride}),
        o(d_o, s.value_dim, {s.batch, s.o_batch_stride, s.tokens, s.o_token_stride, s.heads, s.o_head_stride});
    const int64_t elements = s.batch * s.heads * s.head_dim * s.value_dim;
    const Area decay(d_log_decay, s.heads, 4), lengths(d_lengths, s.batch, 4), si(d_state_in, elements, 4),
        so(d_state_out, elements, 4);
    if (!all_apart(o, {q, k, v, decay, lengths, si, so}) ||
        !all_apart(so, {q, k, v, decay, lengths, d_state_out == d_state_in ? Area(nullptr, 0, 4) : si}))
      return set_error(NCODEC_EINVAL, "decay_attention", "an output overlaps an input that it is not, or the other output");
  }
  return finish(nc::launch_decay_attention({*shape, d_q, d_k, d_v, d_log_decay, d_lengths, d_state_in, d_state_out,
                                            d_o, d_workspace},
                                           (hipStream_t)hip_stream),
                "decay_attention");
}

extern "C" ncodec_status ncodec_window_attention(const ncodec_window_shape* shape, const void* d_q, const void* d_k,
                                                 const void* d_v, const int32_t* d_lengths, void* d_o,
                                                 void* hip_stream) {
  if (!shape) return set_error(NCODEC_EINVAL, "window_attention", "shape is NULL");
  ncodec_status st;
  if (const char* why = window_fault(*shape, &st)) return set_error(st, "window_attention", why);
  if (shape->batch == 0 || shape->tokens == 0) return NCODEC_OK;
  if (!d_q || !d_k || !d_v || !d_o)
    return set_error(NCODEC_EINVAL, "window_attention", "d_q, d_k, d_v and d_o must be non-NULL");
  if (!aligned(d_q, 2) || !aligned(d_k, 2) || !aligned(d_v, 2) || !aligned(d_o, 2) || !aligned(d_lengths, 4))
    return set_error(NCODEC_EINVAL, "window_attention", "a pointer is not aligned to an element");
  {
    const ncodec_window_shape& s = *shape;
    const Area q(d_q, s.head_dim, {s.batch, s.q_batch_stride, s.tokens, s.q_token_stride, s.heads, s.q_head_stride}),
        k(d_k, s.head_dim, {s.batch, s.k_batch_stride, s.tokens, s.k_token_stride, s.kv_heads, s.k_head_stride}),
        v(d_v, s.value_dim, {s.batch, s.v_batch_stride, s.tokens, s.v_token_stride, s.kv_heads, s.v_head_stride}),
        o(d_o, s.value_dim, {s.batch, s.o_batch_stride, s.tokens, s.o_token_stride, s.heads, s.o_head_stride});
    if (!all_apart(o, {q, k, v, Area(d_lengths, s.batch, 4)}))
      return set_error(NCODEC_EINVAL, "window_attention", "d_o overlaps an input");
  }
  return finish(nc::launch_window_attention({*shape, d_q, d_k, d_v, d_lengths, d_o}, (hipStream_t)hip_stream),
                "window_attention");
}

extern "C" size_t ncodec_paged_attention_workspace_bytes(const ncodec_cache_shape* cache,
                                                         const ncodec_paged_shape* shape, int32_t mass) {
  ncodec_status st;
  if (!cache || !shape || paged_fault(*cache, *shape, &st)) return 0;
  return nc::paged_workspace_bytes(*cache, *shape, mass != 0);
}

extern "C" ncodec_status ncodec_paged_attention(const ncodec_cache_shape* cache, const ncodec_paged_shape* shape,
                                                const void* d_q, const void* d_k_cache, const void* d_v_cache,
                                                const int32_t* d_table, const int32_t* d_lengths, float* d_mass,
                                                void* d_o, void* d_workspace, size_t ws_bytes, void* hip_stream) {
  if (!cache || !shape) return set_error(NCODEC_EINVAL, "paged_attention", "a shape is NULL");
  ncodec_status st;
  if (const char* why = paged_fault(*cache, *shape, &st)) return set_error(st, "paged_attention", why);
  if (shape->batch == 0) return NCODEC_OK;
  const ncodec_cache_shape& c = *cache;
  const ncodec_paged_shape& s = *shape;
  if (!d_q || !d_o || !d_lengths || (s.columns && !d_table) || (c.pages && (!d_k_cache || !d_v_cache)))
    return set_error(NCODEC_EINVAL, "paged_attention", "d_q, the cache, d_table, d_lengths and d_o must be non-NULL");
  if (!aligned(d_q, 2) || !aligned(d_k_cache, 2) || !aligned(d_v_cache, 2) || !aligned(d_o, 2) || !aligned(d_table, 4) ||
      !aligned(d_lengths, 4) || !aligned(d_mass, 4))
    return set_error(NCODEC_EINVAL, "paged_attention", "a pointer is not aligned to an element");
  const size_t need = nc::paged_workspace_bytes(c, s, d_mass != nullptr);
  if (need && (!d_workspace || ws_bytes < need || !aligned(d_workspace, 256)))
    return set_error(NCODEC_ENOMEM, "paged_attention", "the workspace must be 256-byte aligned and hold ", need);
  const Area q(d_q, c.head_dim, {s.batch, s.q_batch_stride, s.heads, s.q_head_stride}),
      o(d_o, c.value_dim, {s.batch, s.o_batch_stride, s.heads, s.o_head_stride}), k = k_area(c, d_k_cache),
      v = v_area(c, d_v_cache), table = table_area(d_table, s.batch, s.columns, s.table_stride),
      lengths(d_lengths, s.batch, 4), mass(d_mass, s.batch * c.kv_heads * s.columns * c.page_size, 4);
  if (!all_apart(o, {q, k, v, table, lengths, mass}) || !all_apart(mass, {q, k, v, table, lengths}))
    return set_error(NCODEC_EINVAL, "paged_attention", "an output overlaps an input or the other output");
  return finish(nc::launch_paged_attention({c, s, d_q, d_k_cache, d_v_cache, d_table, d_lengths, d_mass, d_o, d_workspace},
                                           (hipStream_t)hip_stream),
                "paged_attention");
}

extern "C" ncodec_status ncodec_cache_append(const ncodec_cache_shape* cache, const ncodec_append_shape* shape,
                                             const void* d_k, const void* d_v, void* d_k_cache, void* d_v_cache,
                                             const int32_t* d_table, const int32_t* d_starts, const int32_t* d_counts,
                                             float* d_mass, void* hip_stream) {
  if (!cache || !shape) return set_error(NCODEC_EINVAL, "cache_append", "a shape is NULL");
  ncodec_status st;
  if (const char* why = append_fault(*cache, *shape, &st)) return set_error(st, "cache_append", why);
  const ncodec_cache_shape& c = *cache;
  const ncodec_append_shape& s = *shape;
  if (s.batch == 0 || s.tokens == 0 || s.columns == 0 || c.pages == 0) return NCODEC_OK;
  if (!d_k || !d_v || !d_k_cache || !d_v_cache || !d_table || !d_starts)
    return set_error(NCODEC_EINVAL, "cache_append", "d_k, d_v, the cache, d_table and d_starts must be non-NULL");
  if (!aligned(d_k, 2) || !aligned(d_v, 2) || !aligned(d_k_cache, 2) || !aligned(d_v_cache, 2) || !aligned(d_table, 4) ||
      !aligned(d_starts, 4) || !aligned(d_counts, 4) || !aligned(d_mass, 4))
    return set_error(NCODEC_EINVAL, "cache_append", "a pointer is not aligned to an element");
  const Area k(d_k, c.head_dim, {s.batch, s.k_batch_stride, s.tokens, s.k_token_stride, c.kv_heads, s.k_head_stride}),
      v(d_v, c.value_dim, {s.batch, s.v_batch_stride, s.tokens, s.v_token_stride, c.kv_heads, s.v_head_stride}),
      kc = k_area(c, d_k_cache), vc = v_area(c, d_v_cache),
      table = table_area(d_table, s.batch, s.columns, s.table_stride), starts(d_starts, s.batch, 4),
      counts(d_counts, s.batch, 4), mass(d_mass, s.batch * c.kv_heads * s.columns * c.page_size, 4);
  if (!all_apart(kc, {k, v, vc, table, starts, counts, mass}) || !all_apart(vc, {k, v, table, starts, counts, mass}) ||
      !all_apart(mass, {k, v, table, starts, counts}))
    return set_error(NCODEC_EINVAL, "cache_append", "an output overlaps an input or another output");
  return finish(nc::launch_cache_append({c, s, d_k, d_v, d_k_cache, d_v_cache, d_table, d_starts, d_counts, d_mass},
                                        (hipStream_t)hip_stream),
                "cache_append");
}

extern "C" size_t ncodec_cache_evict_workspace_bytes(const ncodec_cache_shape* cache, const ncodec_evict_shape* shape) {
  ncodec_status st;
  if (!cache || !shape || evict_fault(*cache, *shape, &st)) return 0;
  return nc::evict_workspace_bytes(*cache, *shape);
}

extern "C" ncodec_status ncodec_cache_evict(const ncodec_cache_shape* cache, const ncodec_evict_shape* shape,
                                            void* d_k_cache, void* d_v_cache, const int32_t* d_table,
                                            const int32_t* d_lengths, const float* d_mass, const int32_t* d_new_table,
                                            int32_t* d_new_lengths, float* d_new_mass, int32_t* d_kept,
                                            void* d_workspace, size_t ws_bytes, void* hip_stream) {
  if (!cache || !shape) return set_error(NCODEC_EINVAL, "cache_evict", "a shape is NULL");
  ncodec_status st;
  if (const char* why = evict_fault(*cache, *shape, &st)) return set_error(st, "cache_evict", why);
  const ncodec_cache_shape& c = *cache;
  const ncodec_evict_shape& s = *shape;
  if (s.batch == 0) return NCODEC_OK;
  if ((c.pages && (!d_k_cache || !d_v_cache)) || (s.columns && (!d_table || !d_mass)) || !d_lengths || !d_new_table ||
      !d_new_lengths || !d_new_mass || !d_kept)
    return set_error(NCODEC_EINVAL, "cache_evict", "the cache, the tables, d_lengths, d_mass and the outputs must be non-NULL");
  if (!aligned(d_k_cache, 2) || !aligned(d_v_cache, 2) || !aligned(d_table, 4) || !aligned(d_lengths, 4) ||
      !aligned(d_mass, 4) || !aligned(d_new_table, 4) || !aligned(d_new_lengths, 4) || !aligned(d_new_mass, 4) ||
      !aligned(d_kept, 4))
    return set_error(NCODEC_EINVAL, "cache_evict", "a pointer is not aligned to an element");
  const size_t need = nc::evict_workspace_bytes(c, s);
  if (need && (!d_workspace || ws_bytes < need || !aligned(d_workspace, 256)))
    return set_error(NCODEC_ENOMEM, "cache_evict", "the workspace must be 256-byte aligned and hold ", need);
  const int64_t bk = s.batch * c.kv_heads;
  const Area kc = k_area(c, d_k_cache), vc = v_area(c, d_v_cache),
             table = table_area(d_table, s.batch, s.columns, s.table_stride),
             new_table = table_area(d_new_table, s.batch, s.new_columns, s.new_table_stride),
             lengths(d_lengths, s.batch, 4), mass(d_mass, bk * s.columns * c.page_size, 4),
             new_lengths(d_new_lengths, s.batch, 4), new_mass(d_new_mass, bk * s.new_columns * c.page_size, 4),
             kept(d_kept, bk * s.keep, 4);
  if (!all_apart(kc, {vc, table, new_table, lengths, mass, new_lengths, new_mass, kept}) ||
      !all_apart(vc, {table, new_table, lengths, mass, new_lengths, new_mass, kept}) ||
      !all_apart(new_lengths, {table, new_table, lengths, mass, new_mass, kept}) ||
      !all_apart(new_mass, {table, new_table, lengths, mass, kept}) ||
      !all_apart(kept, {table, new_table, lengths, mass}))
    return set_error(NCODEC_EINVAL, "cache_evict", "an output overlaps an input or another output");
  return finish(nc::launch_cache_evict({c, s, d_k_cache, d_v_cache, d_table, d_lengths, d_mass, d_new_table,
                                        d_new_lengths, d_new_mass, d_kept, d_workspace},
                                       (hipStream_t)hip_stream),
                "cache_evict");
}
