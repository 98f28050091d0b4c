// C-ABI layer of the layer calls: argument checks, and from the ABI's structs to the launch interface.
#include "../../include/tng.h"

#include "tng_layer_kernels.hpp"

#include <cfloat>
#include <cmath>

namespace {

constexpr uint64_t kMaxDrawn = 1ull << 33, kMaxSide = 1ull << 22, kMaxRows = 1ull << 23;
constexpr uint64_t kMaxStride = 1ull << 40;  // (products of strides and indexes stay far inside 64 bits)

inline size_t round_up(size_t v) { return (v + 255) / 256 * 256; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t size_of(int32_t type) {
  return type == TNG_TYPE_I8 ? 1 : type == TNG_TYPE_I64 ? 8 : type == TNG_TYPE_F32 || type == TNG_TYPE_I32 ? 4 : 2;
}
inline bool is_ids(int32_t type) { return type == TNG_TYPE_I32 || type == TNG_TYPE_I64; }
inline bool is_float(int32_t type) { return type == TNG_TYPE_F32 || type == TNG_TYPE_BF16 || type == TNG_TYPE_F16; }
inline bool empty(const tng_matrix& a) { return a.rows == 0 || a.cols == 0; }

// Whether the matrix can be worked on: sizes, strides, address.
bool sound(const tng_matrix* a, bool output) {
  if (a == nullptr || a->workers == 0 || a->workers > 65535u) return false;
  if (a->type < TNG_TYPE_F32 || a->type > TNG_TYPE_I64) return false;
  if (a->rows > kMaxDrawn || a->cols > kMaxDrawn || a->ld > kMaxStride || a->pitch > kMaxStride) return false;
  if (empty(*a)) return true;
  if (a->rows > kMaxDrawn / a->cols) return false;
  if (a->data == nullptr || !aligned(a->data, size_of(a->type))) return false;
  if (a->rows > 1 && a->ld < a->cols && (output || a->ld != 0)) return false;
  const uint64_t extent = (a->rows > 1 ? (a->rows - 1) * a->ld : 0) + a->cols;
  return a->workers == 1 || a->pitch >= extent || (!output && a->pitch == 0);
}

bool same_size(const tng_matrix* a, const tng_matrix* b) {
  return a->workers == b->workers && a->rows == b->rows && a->cols == b->cols;
}

bool sides_ok(const tng_matrix* a) { return a->rows <= kMaxSide && a->cols <= kMaxSide && a->workers * a->rows <= kMaxRows; }

bool drop_ok(const tng_drop* d) {
  return d != nullptr && d->site < (1u << 24) && d->p >= 0.f && d->p < 1.f && (d->relu == 0 || d->relu == 1);
}

tng::DropArgs drop_args(const tng_drop& d, uint32_t stream) {
  tng::DropArgs a;
  a.k0 = (uint32_t)d.seed;
  a.k1 = (uint32_t)(d.seed >> 32);
  a.iter = d.iter;
  a.word = stream | d.site << 8;
  a.threshold = (uint32_t)std::ceil((double)d.p * 0x1p24) << 8;  // (below 2^24: p is below 1)
  a.scale = (float)(1.0 / (1.0 - (double)d.p));
  a.relu = d.relu;
  return a;
}

tng::View view(const tng_matrix* a) {
  if (a == nullptr) return tng::View{nullptr, 0, 0};
  // Strides that no index reaches are made what suits the products: single rows of several workers lie as one worker's rows do, and one row
  // by itself begins aligned as its address does.
  // (The products' fast kernels then read its last codes as a whole aligned piece of 16 bytes, as they do every last row's; a page that holds
  // one of them holds the piece.)
  uint64_t ld = a->ld;
  if (a->rows <= 1) ld = a->workers > 1 && a->pitch < (1u << 23) ? a->pitch : (a->cols + 15) / 16 * 16;
  return tng::View{a->data, ld, a->workers > 1 ? a->pitch : a->rows * ld};
}

tng::Extent extent(const tng_matrix* a) { return tng::Extent{a->workers, a->rows, a->cols}; }

inline tng_status hip_status(hipError_t e) { return e == hipSuccess ? TNG_OK : TNG_ERR_HIP; }

// a, b, y of a product and what goes with them, or false.
bool product_of(const tng_matrix* a, const tng_matrix* b, const tng_matrix* y, tng::Product* p) {
  if (!sound(a, false) || !sound(b, false) || !sound(y, true)) return false;
  if (a->type != TNG_TYPE_I8 || b->type != TNG_TYPE_I8 || !is_float(y->type)) return false;
  if (a->cols != b->cols || y->rows != a->rows || y->cols != b->rows || y->workers != a->workers) return false;
  if (b->workers != 1 && b->workers != a->workers) return false;
  if (!sides_ok(a) || !sides_ok(b)) return false;
  *p = tng::Product{};
  p->workers = a->workers;
  p->rows = a->rows;
  p->channels = b->rows;
  p->depth = a->cols;
  p->a = view(a);
  p->b = view(b);
  if (b->workers == 1) p->b.pitch = 0;
  p->b_scale_pitch = b->workers == 1 ? 0 : b->rows;
  p->y = view(y);
  p->type = (tng_type)y->type;
  return true;
}

// Where tng_linear_i8 keeps the codes of x: rows 16 bytes apart, their scales, and what the product needs.
struct LinearScratch {
  tng_matrix q;  // (data: set where the workspace is known)
  tng::Product product;
  size_t scale_at, rest_at, bytes;
};

bool linear_scratch(const tng_matrix* x, const tng_matrix* b, const tng_matrix* y, LinearScratch* l) {
  if (!sound(x, false) || !is_float(x->type) || !sides_ok(x) || y == nullptr || y->type != x->type) return false;
  const uint64_t ld = (x->cols + 15) / 16 * 16;
  l->q = tng_matrix{reinterpret_cast<void*>((uintptr_t)256), TNG_TYPE_I8, x->workers, x->rows, x->cols, ld, x->rows * ld};
  if (!product_of(&l->q, b, y, &l->product)) return false;
  l->scale_at = round_up(x->workers * x->rows * ld);
  l->rest_at = l->scale_at + round_up(x->workers * x->rows * sizeof(float));
  l->bytes = l->rest_at + 256 + tng::product_scratch_bytes(l->product);
  return true;
}

bool norm_ok(const tng_rms* n) {
  return n != nullptr && n->eps >= FLT_MIN && n->eps <= 0x1p64f && aligned(n->weight, 4);
}

tng::NormArgs norm_args(const tng_rms& n) { return tng::NormArgs{n.weight, n.eps}; }

// Whether two matrices begin at one place.
bool same_place(const tng_matrix* a, const tng_matrix* b) { return a != nullptr && b != nullptr && !empty(*a) && !empty(*b) && a->data == b->data; }

// Whether a result that may be an input is that, or begins elsewhere: of another type or other strides at its place, what one row's work writes is what
// another's still reads.
bool is_or_apart(const tng_matrix* in, const tng_matrix* out) {
  if (!same_place(in, out)) return true;
  return in->type == out->type && (in->rows <= 1 || in->ld == out->ld) && (in->workers == 1 || in->pitch == out->pitch);
}

// x and what goes with it in front of a norm; the matrices that may be absent are of x's type and size where they are there.
bool normed_ok(const tng_matrix* x, const tng_matrix* residual, const tng_rms* norm, const tng_matrix* h) {
  if (!norm_ok(norm) || !sound(x, false) || !is_float(x->type) || !sides_ok(x)) return false;
  if (residual != nullptr && (!sound(residual, false) || residual->type != x->type || !same_size(x, residual))) return false;
  return h == nullptr || (sound(h, true) && h->type == x->type && same_size(x, h) && is_or_apart(x, h) && is_or_apart(residual, h));
}

// Tokens and the matrix with a row for each of them.
bool tokens_ok(const tng_matrix* ids, const tng_matrix* rows, bool output) {
  if (!sound(ids, false) || !is_ids(ids->type) || ids->cols != 1) return false;
  if (!sound(rows, output) || !is_float(rows->type) || !sides_ok(rows)) return false;
  return rows->workers == ids->workers && rows->rows == ids->rows;
}

bool embed_grad_ok(const tng_matrix* ids, const tng_matrix* dy, const tng_matrix* dtable) {
  if (!tokens_ok(ids, dy, false) || !sound(dtable, true) || dtable->type != TNG_TYPE_F32) return false;
  return dtable->workers == dy->workers && dtable->cols == dy->cols && dtable->rows <= kMaxSide;
}

// Matrices that are orthogonalised, apart from where they lie.
bool update_ok(const tng_matrix* x) {
  return x != nullptr && is_float(x->type) && x->workers != 0 && x->workers <= 65535u && x->rows <= 65536 && x->cols <= 65536 &&
         x->workers * x->rows <= kMaxRows;
}

bool scale_ok(const float* scale) { return scale == nullptr || std::isfinite(*scale); }

}  // namespace

extern "C" {

tng_status tng_dropout(void* hip_stream, const tng_drop* drop, const tng_matrix* x, const tng_matrix* residual, const tng_matrix* y) {
  if (!drop_ok(drop) || !sound(x, false) || !sound(y, true) || (residual != nullptr && !sound(residual, false)))
    return TNG_ERR_INVALID_ARG;
  if (!is_float(x->type) || y->type != x->type || !same_size(x, y)) return TNG_ERR_INVALID_ARG;
  if (residual != nullptr && (residual->type != x->type || !same_size(x, residual))) return TNG_ERR_INVALID_ARG;
  if (empty(*x)) return TNG_OK;
  return hip_status(tng::launch_dropout((tng_type)x->type, extent(x), drop_args(*drop, tng::kStreamDropout), view(x), view(residual),
                                        view(y), static_cast<hipStream_t>(hip_stream)));
}

tng_status tng_dropout_grad(void* hip_stream, const tng_drop* drop, const tng_matrix* x, const tng_matrix* dy, const tng_matrix* dx) {
  if (!drop_ok(drop) || !sound(dy, false) || !sound(dx, true)) return TNG_ERR_INVALID_ARG;
  if (!is_float(dy->type) || dx->type != dy->type || !same_size(dy, dx)) return TNG_ERR_INVALID_ARG;
  if (drop->relu && (!sound(x, false) || x->type != dy->type || !same_size(x, dy))) return TNG_ERR_INVALID_ARG;
  if (empty(*dy)) return TNG_OK;
  return hip_status(tng::launch_dropout_grad((tng_type)dy->type, extent(dy), drop_args(*drop, tng::kStreamDropout),
                                             view(drop->relu ? x : nullptr), view(dy), view(dx), static_cast<hipStream_t>(hip_stream)));
}

tng_status tng_quantize_rows(void* hip_stream, const tng_drop* drop, const tng_matrix* x, const tng_matrix* q, float* scale,
                             const tng_matrix* qt) {
  if ((drop != nullptr && !drop_ok(drop)) || !sound(x, false) || !sound(q, true) || (qt != nullptr && !sound(qt, true)))
    return TNG_ERR_INVALID_ARG;
  if (!is_float(x->type) || q->type != TNG_TYPE_I8 || !same_size(x, q) || !sides_ok(x)) return TNG_ERR_INVALID_ARG;
  if (qt != nullptr && (qt->type != TNG_TYPE_I8 || qt->workers != x->workers || qt->rows != x->cols || qt->cols != x->rows))
    return TNG_ERR_INVALID_ARG;
  if (x->rows == 0) return TNG_OK;
  if (scale == nullptr || !aligned(scale, 4)) return TNG_ERR_INVALID_ARG;
  // (rows without elements: their scales are 0)
  const tng::DropArgs d = drop != nullptr ? drop_args(*drop, tng::kStreamDropout) : tng::DropArgs{};
  return hip_status(tng::launch_quantize_rows((tng_type)x->type, extent(x), drop != nullptr ? &d : nullptr, view(x), view(q), scale,
                                              x->cols == 0 ? tng::View{nullptr, 0, 0} : view(qt), static_cast<hipStream_t>(hip_stream)));
}

size_t tng_quantize_grad_bytes(const tng_matrix* dy) {
  if (dy == nullptr || dy->rows > kMaxSide || dy->cols > kMaxSide || dy->workers == 0 || dy->workers > 65535u || !sides_ok(dy)) return 0;
  return 256 + tng::quantize_grad_floats(extent(dy)) * sizeof(float);
}

tng_status tng_quantize_grad(void* hip_stream, const tng_drop* key, const tng_matrix* dy, const float* col_scale, const float* row_scale,
                             const tng_matrix* q, float* q_scale, const tng_matrix* qt, float* qt_scale, float* col_sum, void* workspace,
                             size_t workspace_bytes) {
  if (!drop_ok(key) || !sound(dy, false) || !sound(q, true) || !sound(qt, true)) return TNG_ERR_INVALID_ARG;
  if (!is_float(dy->type) || q->type != TNG_TYPE_I8 || qt->type != TNG_TYPE_I8 || !same_size(dy, q) || !sides_ok(dy))
    return TNG_ERR_INVALID_ARG;
  if (qt->workers != dy->workers || qt->rows != dy->cols || qt->cols != dy->rows) return TNG_ERR_INVALID_ARG;
  if ((dy->rows != 0 && q_scale == nullptr) || (dy->cols != 0 && qt_scale == nullptr)) return TNG_ERR_INVALID_ARG;
  if (!aligned(col_scale, 4) || !aligned(row_scale, 4) || !aligned(q_scale, 4) || !aligned(qt_scale, 4) || !aligned(col_sum, 4))
    return TNG_ERR_INVALID_ARG;
  if (dy->rows == 0 && dy->cols == 0) return TNG_OK;
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < tng_quantize_grad_bytes(dy)) return TNG_ERR_WORKSPACE;
  return hip_status(tng::launch_quantize_grad((tng_type)dy->type, extent(dy), drop_args(*key, tng::kStreamRounding), view(dy), col_scale,
                                              row_scale, view(q), q_scale, view(qt), qt_scale, col_sum, static_cast<float*>(workspace),
                                              static_cast<hipStream_t>(hip_stream)));
}

size_t tng_matmul_i8_bytes(const tng_matrix* a, const tng_matrix* b, const tng_matrix* y) {
  tng::Product p;
  if (!product_of(a, b, y, &p)) return 0;
  return 256 + tng::product_scratch_bytes(p);
}

tng_status tng_matmul_i8(void* hip_stream, const tng_matrix* a, const float* a_scale, const tng_matrix* b, const float* b_scale,
                         const float* bias, const tng_drop* drop, const tng_matrix* x, const tng_matrix* y, void* workspace,
                         size_t workspace_bytes) {
  tng::Product p;
  if (!product_of(a, b, y, &p)) return TNG_ERR_INVALID_ARG;
  if (!aligned(a_scale, 4) || !aligned(b_scale, 4) || !aligned(bias, 4)) return TNG_ERR_INVALID_ARG;
  if (drop != nullptr) {
    if (!drop_ok(drop)) return TNG_ERR_INVALID_ARG;
    if (drop->relu && (!sound(x, false) || x->type != y->type || !same_size(x, y))) return TNG_ERR_INVALID_ARG;
  }
  if (empty(*y)) return TNG_OK;
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < 256 + tng::product_scratch_bytes(p)) return TNG_ERR_WORKSPACE;
  p.a_scale = a_scale;
  p.b_scale = b_scale;
  p.bias = bias;
  tng::DropArgs d{};
  if (drop != nullptr) {
    d = drop_args(*drop, tng::kStreamDropout);
    p.drop = &d;
    if (drop->relu) p.x = view(x);
  }
  return hip_status(tng::launch_product(p, workspace, static_cast<hipStream_t>(hip_stream)));
}

size_t tng_linear_i8_bytes(const tng_matrix* x, const tng_matrix* b, const tng_matrix* y) {
  LinearScratch l;
  return linear_scratch(x, b, y, &l) ? l.bytes : 0;
}

tng_status tng_linear_i8(void* hip_stream, const tng_drop* drop, const tng_matrix* x, const tng_matrix* b, const float* b_scale,
                         const float* bias, const tng_matrix* y, void* workspace, size_t workspace_bytes) {
  LinearScratch l;
  if ((drop != nullptr && !drop_ok(drop)) || !linear_scratch(x, b, y, &l)) return TNG_ERR_INVALID_ARG;
  if (!aligned(b_scale, 4) || !aligned(bias, 4)) return TNG_ERR_INVALID_ARG;
  if (empty(*y)) return TNG_OK;
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < l.bytes) return TNG_ERR_WORKSPACE;
  if (drop == nullptr && tng::coded_product_applies(l.product, view(x))) {
    l.product.b_scale = b_scale;
    l.product.bias = bias;
    return hip_status(tng::launch_coded_product(l.product, view(x), static_cast<hipStream_t>(hip_stream)));
  }
  char* at = static_cast<char*>(workspace);
  l.q.data = at;
  float* scale = reinterpret_cast<float*>(at + l.scale_at);
  const tng_status s = tng_quantize_rows(hip_stream, drop, x, &l.q, scale, nullptr);
  if (s != TNG_OK) return s;
  return tng_matmul_i8(hip_stream, &l.q, scale, b, b_scale, bias, nullptr, nullptr, y, at + l.rest_at, workspace_bytes - l.rest_at);
}

tng_status tng_rms_norm(void* hip_stream, const tng_matrix* x, const tng_matrix* residual, const tng_rms* norm, const tng_matrix* h,
                        const tng_matrix* y) {
  if (!normed_ok(x, residual, norm, h) || !sound(y, true) || y->type != x->type || !same_size(x, y) || same_place(h, y))
    return TNG_ERR_INVALID_ARG;
  if (!is_or_apart(x, y) || !is_or_apart(residual, y)) return TNG_ERR_INVALID_ARG;
  if (empty(*x)) return TNG_OK;
  return hip_status(tng::launch_rms_norm((tng_type)x->type, extent(x), view(x), view(residual), norm_args(*norm), view(h), view(y), nullptr,
                                         static_cast<hipStream_t>(hip_stream)));
}

tng_status tng_rms_norm_codes(void* hip_stream, const tng_matrix* x, const tng_matrix* residual, const tng_rms* norm, const tng_matrix* h,
                              const tng_matrix* q, float* scale, const tng_matrix* qt) {
  if (!normed_ok(x, residual, norm, h) || !sound(q, true) || q->type != TNG_TYPE_I8 || !same_size(x, q)) return TNG_ERR_INVALID_ARG;
  if (qt != nullptr && (!sound(qt, true) || qt->type != TNG_TYPE_I8 || qt->workers != x->workers || qt->rows != x->cols || qt->cols != x->rows))
    return TNG_ERR_INVALID_ARG;
  for (const tng_matrix* codes : {q, qt})
    if (same_place(x, codes) || same_place(residual, codes) || same_place(h, codes)) return TNG_ERR_INVALID_ARG;
  if (same_place(q, qt)) return TNG_ERR_INVALID_ARG;
  if (x->rows == 0) return TNG_OK;
  if (scale == nullptr || !aligned(scale, 4)) return TNG_ERR_INVALID_ARG;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (x->cols == 0)  // (rows without elements: their scales are 0)
    return hip_status(tng::launch_quantize_rows((tng_type)x->type, extent(x), nullptr, view(x), view(q), scale, tng::View{nullptr, 0, 0}, s));
  const hipError_t e =
      tng::launch_rms_norm((tng_type)x->type, extent(x), view(x), view(residual), norm_args(*norm), view(h), view(q), scale, s);
  return hip_status(e != hipSuccess || qt == nullptr ? e : tng::launch_turn_codes(extent(x), view(q), view(qt), s));
}

size_t tng_rms_norm_grad_bytes(const tng_matrix* dy) {
  if (dy == nullptr || !is_float(dy->type) || dy->workers == 0 || dy->workers > 65535u || !sides_ok(dy)) return 0;
  return 256 + tng::rms_norm_grad_floats(extent(dy)) * sizeof(float);
}

tng_status tng_rms_norm_grad(void* hip_stream, const tng_matrix* dy, const tng_matrix* h, const tng_matrix* dresidual, const tng_rms* norm,
                             const tng_matrix* dx, float* dw, void* workspace, size_t workspace_bytes) {
  if (!normed_ok(dy, h, norm, dx) || h == nullptr || dx == nullptr || !aligned(dw, 4)) return TNG_ERR_INVALID_ARG;
  if (dresidual != nullptr && (!sound(dresidual, false) || dresidual->type != dy->type || !same_size(dy, dresidual))) return TNG_ERR_INVALID_ARG;
  if (!is_or_apart(dresidual, dx)) return TNG_ERR_INVALID_ARG;
  if (dy->cols == 0 || (dy->rows == 0 && dw == nullptr)) return TNG_OK;
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < tng_rms_norm_grad_bytes(dy)) return TNG_ERR_WORKSPACE;
  return hip_status(tng::launch_rms_norm_grad((tng_type)dy->type, extent(dy), view(dy), view(h), view(dresidual), norm_args(*norm), view(dx), dw,
                                              static_cast<float*>(workspace), static_cast<hipStream_t>(hip_stream)));
}

tng_status tng_embed(void* hip_stream, const tng_matrix* ids, const tng_matrix* table, const float* scale, const tng_matrix* y) {
  if (!tokens_ok(ids, y, true) || !scale_ok(scale) || !sound(table, false) || !is_float(table->type)) return TNG_ERR_INVALID_ARG;
  if (table->rows > kMaxSide || table->cols != y->cols || (table->workers != 1 && table->workers != y->workers)) return TNG_ERR_INVALID_ARG;
  if (same_place(table, y) || same_place(ids, y)) return TNG_ERR_INVALID_ARG;
  if (empty(*y)) return TNG_OK;
  tng::View rows = view(table);
  if (table->workers == 1) rows.pitch = 0;
  return hip_status(tng::launch_embed((tng_type)ids->type, (tng_type)table->type, (tng_type)y->type, y->workers, y->rows, y->cols, table->rows,
                                      view(ids), rows, scale != nullptr ? *scale : 1.f, view(y), static_cast<hipStream_t>(hip_stream)));
}

size_t tng_embed_grad_bytes(const tng_matrix* ids, const tng_matrix* dy, const tng_matrix* dtable) {
  if (!embed_grad_ok(ids, dy, dtable)) return 0;
  return 256 + tng::embed_grad_words(dy->workers, dy->rows, dy->cols, dtable->rows) * sizeof(uint32_t);
}

tng_status tng_embed_grad(void* hip_stream, const tng_matrix* ids, const tng_matrix* dy, const float* scale, const tng_matrix* dtable, void* workspace,
                          size_t workspace_bytes) {
  if (!embed_grad_ok(ids, dy, dtable) || !scale_ok(scale)) return TNG_ERR_INVALID_ARG;
  if (empty(*dtable)) return TNG_OK;
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < tng_embed_grad_bytes(ids, dy, dtable)) return TNG_ERR_WORKSPACE;
  return hip_status(tng::launch_embed_grad((tng_type)ids->type, (tng_type)dy->type, dy->workers, dy->rows, dy->cols, dtable->rows, view(ids),
                                           view(dy), scale != nullptr ? *scale : 1.f, view(dtable), static_cast<uint32_t*>(workspace),
                                           static_cast<hipStream_t>(hip_stream)));
}

size_t tng_orthogonalize_bytes(const tng_matrix* x) { return update_ok(x) ? 256 + tng::orthogonal_bytes(extent(x)) : 0; }

tng_status tng_orthogonalize(void* hip_stream, const tng_matrix* x, const tng_orthogonal* plan, const tng_matrix* y, void* workspace,
                             size_t workspace_bytes) {
  if (!sound(x, false) || !sound(y, true) || !update_ok(x) || !is_float(y->type) || !same_size(x, y) || !is_or_apart(x, y)) return TNG_ERR_INVALID_ARG;
  if (plan == nullptr || plan->coefficients == nullptr || plan->steps < 1 || plan->steps > 64) return TNG_ERR_INVALID_ARG;
  if (!(plan->eps >= FLT_MIN && plan->eps <= FLT_MAX) || !std::isfinite(plan->scale)) return TNG_ERR_INVALID_ARG;
  for (uint32_t k = 0; k < 3 * plan->steps; ++k)
    if (!std::isfinite(plan->coefficients[k])) return TNG_ERR_INVALID_ARG;
  if (!tng::orthogonal_in_range(plan->coefficients, plan->steps)) return TNG_ERR_UNSUPPORTED;
  if (empty(*x)) return TNG_OK;
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < tng_orthogonalize_bytes(x)) return TNG_ERR_WORKSPACE;
  return hip_status(tng::launch_orthogonalize((tng_type)x->type, (tng_type)y->type, extent(x), view(x), plan->coefficients, plan->steps, plan->eps,
                                              plan->scale, view(y), static_cast<char*>(workspace), static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
