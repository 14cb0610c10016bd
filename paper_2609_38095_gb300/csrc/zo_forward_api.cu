// zo_forward_api.cu -- the extern "C" entry points declared in
// include/zo_forward.h: argument validation and the choice of kernel.
// Everything here runs on the host and only enqueues kernels.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <utility>

#include "zo_forward.cuh"
#include "zo_forward.h"
#include "zo_launch.h"

namespace {

constexpr int64_t kMaxIndex = INT64_C(0x7FFFFFFF);  // rows, keys and launch grids count in 32 bits

int element_size(int32_t dtype) { return dtype == ZO_F32 ? 4 : 2; }

bool known(int32_t dtype) { return dtype == ZO_F32 || dtype == ZO_BF16 || dtype == ZO_F16; }

bool misaligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

bool bad_strides(int64_t a, int64_t b, int64_t c = 0) { return a < 0 || b < 0 || c < 0; }

int check_heads(int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t dtype) {
  if (head_dim < 1 || head_dim > ZO_MAX_HEAD_DIM || heads < 1 || heads > ZO_MAX_HEADS || kv_heads < 1 ||
      heads % kv_heads != 0)
    return ZO_ERR_ARG;
  return known(dtype) ? ZO_OK : ZO_ERR_DTYPE;
}

int check_scores(float scale, float softcap) {
  return std::isfinite(scale) && std::isfinite(softcap) && softcap >= 0.0f ? ZO_OK : ZO_ERR_ARG;
}

// A tensor's elements as its arguments give them: up to three dimensions of runs of contiguous bytes.
struct Dimension {
  int64_t count, stride;  // in elements
};
struct Tensor {
  const void* ptr;
  Dimension d[3];  // the outermost first, as the argument names them
  int64_t run;
  size_t size;
  double bytes;  // from the first to the last, 0 where there are none
};

Tensor tensor(const void* p, int64_t run, size_t size, Dimension a, Dimension b, Dimension c) {
  Tensor t = {p, {a, b, c}, run, size, 0.0};
  if (p != nullptr && a.count > 0 && b.count > 0 && c.count > 0)
    t.bytes = size * (static_cast<double>(a.count - 1) * a.stride + static_cast<double>(b.count - 1) * b.stride +
                      static_cast<double>(c.count - 1) * c.stride + run);
  return t;
}
Tensor tensor(const zo_rows& x, int64_t tokens, int64_t heads, int64_t run, size_t size) {
  return tensor(x.ptr, run, size, {1, 0}, {tokens, x.token}, {heads, x.head});
}
Tensor tensor(const zo_pages& x, int64_t pages, int64_t page_size, int64_t heads, int64_t run, size_t size) {
  return tensor(x.ptr, run, size, {pages, x.page}, {page_size, x.token}, {heads, x.head});
}

// The same in bytes: dimensions from the widest step down, what is contiguous together as one, the last a run.
using Wide = __int128;  // any 64-bit strides and counts
struct Places {
  int n;
  Wide count[4], step[4], extent[5];  // extent[i]: bytes from the first to the last of dimensions i ..
};

Places places(const Tensor& t) {
  Dimension d[3] = {t.d[0], t.d[1], t.d[2]};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (d[i].stride < d[j].stride) std::swap(d[i], d[j]);
  Wide count[4], step[4];
  int n = 0;
  count[n] = static_cast<Wide>(t.run) * t.size, step[n++] = 1;
  for (int i = 2; i >= 0; --i) {  // from the innermost out
    const Wide s = static_cast<Wide>(d[i].stride) * t.size;
    if (d[i].count == 1) continue;
    if (s == count[n - 1] * step[n - 1]) {
      count[n - 1] *= d[i].count;
    } else {
      count[n] = d[i].count, step[n++] = s;
    }
  }
  Places r;
  r.n = n;
  r.extent[n] = 1;
  for (int i = n - 1; i >= 0; --i) {
    r.count[i] = count[n - 1 - i], r.step[i] = step[n - 1 - i];
    r.extent[i] = r.extent[i + 1] + (r.count[i] - 1) * r.step[i];
  }
  return r;
}

// Whether elements of an output lie over one another (rows or heads with a stride of less than what they hold).
bool folds(const Tensor& t) {
  double inner = static_cast<double>(t.run);
  bool nested = true;  // each dimension's stride passes the ones behind it: mostly, and nothing more is to be looked at
  for (int i = 2; i >= 0 && nested; --i) {
    nested = t.d[i].count == 1 || t.d[i].stride >= inner;
    inner += static_cast<double>(t.d[i].count - 1) * t.d[i].stride;
  }
  if (nested || t.bytes == 0.0) return false;
  const Places a = places(t);
  for (int i = 0; i + 1 < a.n; ++i)
    if (a.step[i] < a.count[a.n - 1]) return true;
  return false;
}

Wide floor_div(Wide a, Wide b) { return a / b - (a % b < 0); }

// Whether dimensions i.. of a and j.. of b, which starts `delta` bytes behind a, share a byte. Exact where steps are equal,
// or one step holds few of the other's; false where neither is so, since what cannot be shown is not refused.
bool meet(Wide delta, const Places& a, int i, const Places& b, int j) {
  const Wide ea = a.extent[i], eb = b.extent[j];
  if (delta >= ea || -delta >= eb) return false;
  const bool run_a = i == a.n - 1, run_b = j == b.n - 1;
  if (run_a && run_b) return true;
  if (run_a || (!run_b && a.step[i] < b.step[j])) return meet(-delta, b, j, a, i);  // a has the wider step
  const Wide step = a.step[i], inner = a.extent[i + 1];
  if (step == 0) return meet(delta, a, i + 1, b, j);
  if (!run_b && b.step[j] == step && inner <= step && b.extent[j + 1] <= step) {  // rows k apart: at most two k matter
    const Wide k0 = floor_div(-delta, step);
    for (Wide k = k0; k <= k0 + 1; ++k)
      if (k > -a.count[i] && k < b.count[j] && meet(delta + k * step, a, i + 1, b, j + 1)) return true;
    return false;
  }
  const Wide from = std::max<Wide>(0, floor_div(delta - inner, step) + 1);
  const Wide to = std::min<Wide>(a.count[i] - 1, floor_div(delta + eb - 1, step));
  if (run_b && to - from > 1) return true;  // one between the first and the last starts within the run
  if (to - from > 3) return false;
  for (Wide x = from; x <= to; ++x)
    if (meet(delta - x * step, a, i + 1, b, j)) return true;
  return false;
}

bool meet(const Tensor& a, const Tensor& b) {
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.ptr), pb = reinterpret_cast<uintptr_t>(b.ptr);
  // apart, or empty, mostly (a double's rounding aside, which the exact form settles)
  if (a.bytes == 0.0 || b.bytes == 0.0 ||
      (pa < pb ? static_cast<double>(pb - pa) > a.bytes * 1.000001 : static_cast<double>(pa - pb) > b.bytes * 1.000001))
    return false;
  return meet(static_cast<Wide>(pb) - static_cast<Wide>(pa), places(a), 0, places(b), 0);
}

// Each element of one at the other's own place.
bool same_rows(const zo_rows& a, const void* ptr, int64_t token, int64_t head, int64_t tokens, int64_t heads) {
  return a.ptr == ptr && (tokens <= 1 || a.token == token) && (heads <= 1 || a.head == head);
}

Tensor vector(const void* p, int64_t n, size_t size) { return tensor(p, n, size, {1, 0}, {1, 0}, {n > 0, 0}); }

// Attention of `nodes` rows per sequence over a paged cache: checks of the arguments, and from them the kernels' (but the masks).
int check_paged(const zo_pages* q, const zo_pages* k, const zo_pages* v, const zo_pages* out, int64_t batch, int32_t nodes,
                int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t dtype, const int32_t* pages, int64_t pages_stride,
                int64_t max_pages, int64_t n_pages, int32_t page_size, const int32_t* lengths, const void* masks, float scale,
                float softcap, const float* slopes, float* lse, zo::DraftParams* params, int* sms) {
  if (k == nullptr || v == nullptr) return ZO_ERR_ARG;
  int rc = check_heads(heads, kv_heads, head_dim, dtype);
  if (rc == ZO_OK) rc = check_scores(scale, softcap);
  if (rc != ZO_OK) return rc;
  // a launch has at most 16 CTAs per row and query head
  if (batch < 0 || batch > kMaxIndex / 16 / heads / nodes || max_pages < 0 || n_pages < 0 || n_pages > kMaxIndex ||
      page_size < 1 || pages_stride < 0 || max_pages > kMaxIndex)
    return ZO_ERR_ARG;
  for (const zo_pages* x : {q, k, v, out})
    if (bad_strides(x->page, x->token, x->head)) return ZO_ERR_ARG;
  if (batch == 0) return ZO_OK;
  if (q->ptr == nullptr || out->ptr == nullptr || lengths == nullptr || masks == nullptr) return ZO_ERR_ARG;
  if ((max_pages > 0 && pages == nullptr) || (n_pages > 0 && (k->ptr == nullptr || v->ptr == nullptr))) return ZO_ERR_ARG;
  const size_t size = element_size(dtype);
  if (misaligned(q->ptr, size) || misaligned(k->ptr, size) || misaligned(v->ptr, size) || misaligned(out->ptr, size) ||
      misaligned(pages, 4) || misaligned(lengths, 4) || misaligned(slopes, 4) || misaligned(lse, 4))
    return ZO_ERR_ALIGN;
  const Tensor to = tensor(*out, batch, nodes, heads, head_dim, size);
  const bool in_place = q->ptr == out->ptr && (batch <= 1 || q->page == out->page) && (nodes <= 1 || q->token == out->token) &&
                        (heads <= 1 || q->head == out->head);
  if (folds(to) || meet(to, tensor(*k, n_pages, page_size, kv_heads, head_dim, size)) ||
      meet(to, tensor(*v, n_pages, page_size, kv_heads, head_dim, size)) ||
      (!in_place && meet(to, tensor(*q, batch, nodes, heads, head_dim, size))))
    return ZO_ERR_ARG;
  rc = zo::device_sms(sms);
  if (rc != ZO_OK) return rc;
  const auto lone = [](int64_t stride, int64_t n) { return n > 1 ? stride : 0; };  // one element has no stride
  zo::DraftParams& p = *params;
  p.q = q->ptr, p.k = k->ptr, p.v = v->ptr, p.out = out->ptr;
  p.q_token = q->page, p.q_head = q->head, p.out_token = out->page, p.out_head = out->head;
  p.q_node = q->token, p.out_node = out->token;
  p.k_page = lone(k->page, n_pages), p.k_token = lone(k->token, page_size), p.k_head = lone(k->head, kv_heads);
  p.v_page = lone(v->page, n_pages), p.v_token = lone(v->token, page_size), p.v_head = lone(v->head, kv_heads);
  p.pages_stride = pages_stride, p.max_pages = max_pages, p.n_pages = n_pages;
  p.pages = pages, p.lengths = lengths;
  p.heads = heads, p.kv_heads = kv_heads, p.group = heads / kv_heads, p.dim = head_dim, p.page_size = page_size;
  p.page_shift = (page_size & (page_size - 1)) == 0 ? __builtin_ctz(page_size) : -1;
  p.scale = scale, p.softcap = softcap;
  p.slopes = slopes;
  p.lse = lse;
  p.drafts = nodes;
  return ZO_OK;
}

// What the losses over rows of logits share.
int check_rows(const void* logits, int64_t row, int64_t tokens, int64_t vocab, int32_t dtype, const void* targets,
               int32_t target_bytes, int32_t flags, int32_t known_flags, const void* loss) {
  if (tokens < 0 || tokens > kMaxIndex / 8 || vocab < 1 || vocab > kMaxIndex || row < 0 ||
      (target_bytes != 4 && target_bytes != 8) || (flags & ~known_flags) != 0)
    return ZO_ERR_ARG;
  if (!known(dtype)) return ZO_ERR_DTYPE;
  if (loss == nullptr || (tokens > 0 && (logits == nullptr || targets == nullptr))) return ZO_ERR_ARG;
  if (misaligned(logits, element_size(dtype)) || misaligned(targets, target_bytes) ||
      misaligned(loss, flags & ZO_LOSS_F32 ? 4 : 8))
    return ZO_ERR_ALIGN;
  return ZO_OK;
}

// A loss's outputs, over none of its inputs (vectors) nor one another; the gradient may be the logits.
int check_outputs(const void* logits, int64_t row, const void* grad, int64_t grad_row, float grad_scale, int64_t tokens,
                  int64_t vocab, int32_t dtype, Tensor loss, Tensor logp, std::initializer_list<Tensor> inputs) {
  const size_t size = element_size(dtype);
  if (!std::isfinite(grad_scale) || (grad != nullptr && grad_row < 0)) return ZO_ERR_ARG;
  if (misaligned(grad, size) || misaligned(logp.ptr, 4)) return ZO_ERR_ALIGN;
  const Tensor in = tensor(logits, vocab, size, {1, 0}, {1, 0}, {tokens, row});
  const Tensor out = tensor(grad, vocab, size, {1, 0}, {1, 0}, {grad != nullptr ? tokens : 0, grad_row});
  const bool in_place = grad == logits && (tokens <= 1 || grad_row == row);
  bool over = folds(out) || (!in_place && meet(out, in)) || meet(loss, in) || meet(logp, in) || meet(loss, out) ||
              meet(logp, out) || meet(loss, logp);
  for (const Tensor& t : inputs) {
    if (misaligned(t.ptr, t.size)) return ZO_ERR_ALIGN;
    over = over || meet(out, t) || meet(loss, t) || meet(logp, t);
  }
  return over ? ZO_ERR_ARG : ZO_OK;
}

// A workspace's parts, each on 8 bytes: the rows' log-probabilities and log-sums, the sequences' sums (or a mean's weight) and counts, the
// rows' slopes.
struct LossWork {
  float2 *logp, *lse, *sums;
  float *counts, *slopes;
};
int64_t loss_work_size(int64_t tokens, int64_t sequences) {
  const int64_t t = tokens > 0 ? tokens : 1;
  return 16 * t + 8 * sequences + (4 * (sequences + t) + 7) / 8 * 8;
}
LossWork loss_work(void* p, int64_t tokens, int64_t sequences) {
  char* at = static_cast<char*>(p);
  const int64_t t = tokens > 0 ? tokens : 1;
  return {reinterpret_cast<float2*>(at), reinterpret_cast<float2*>(at + 8 * t), reinterpret_cast<float2*>(at + 16 * t),
          reinterpret_cast<float*>(at + 16 * t + 8 * sequences), reinterpret_cast<float*>(at + 16 * t + 12 * sequences)};
}

int finish(cudaError_t e, const char* what) { return e == cudaSuccess ? ZO_OK : zo::report_cuda_error(e, what); }

}  // namespace

extern "C" {

int zo_rotary_table(float* table, int64_t rows, int32_t rotary_dim, double base, double scale, int64_t original,
                    double low, double high, double magnitude, void* stream) {
  if (rows < 0 || rotary_dim < 2 || rotary_dim > ZO_MAX_HEAD_DIM || rotary_dim % 2 != 0) return ZO_ERR_ARG;
  if (!(std::isfinite(base) && base > 0.0 && std::isfinite(scale) && scale > 0.0 && original >= 0)) return ZO_ERR_ARG;
  if (!(std::isfinite(low) && std::isfinite(high) && low <= high && std::isfinite(magnitude))) return ZO_ERR_ARG;
  if (rows == 0) return ZO_OK;
  if (table == nullptr) return ZO_ERR_ARG;
  if (misaligned(table, 4)) return ZO_ERR_ALIGN;
  return finish(zo::launch_rotary_table(table, rows, rotary_dim, base, scale, original, low, high, magnitude,
                                        static_cast<cudaStream_t>(stream)),
                "rotary_table_kernel");
}

int zo_document_spans(const int32_t* q_starts, const int32_t* k_starts, const int32_t* prefix, int32_t docs,
                      int32_t* spans, int64_t tokens, void* stream) {
  if (docs < 0 || tokens < 0 || tokens > kMaxIndex) return ZO_ERR_ARG;
  if (tokens == 0) return ZO_OK;
  if (spans == nullptr || (docs > 0 && (q_starts == nullptr || k_starts == nullptr))) return ZO_ERR_ARG;
  if (misaligned(q_starts, 4) || misaligned(k_starts, 4) || misaligned(prefix, 4) || misaligned(spans, 4))
    return ZO_ERR_ALIGN;
  return finish(zo::launch_document_spans(q_starts, k_starts, prefix, docs, spans, tokens,
                                          static_cast<cudaStream_t>(stream)),
                "document_spans_kernel");
}

int zo_rotate_heads(const zo_head_part* parts, int32_t n_parts, int64_t tokens, int32_t head_dim, int32_t dtype,
                    const float* table, int64_t table_rows, int32_t rotary_dim, int32_t layout, const void* positions,
                    const void* slots, int32_t index_bytes, int64_t n_slots, int64_t page_size, float eps,
                    void* stream) {
  if (n_parts < 0 || n_parts > 3 || (n_parts > 0 && parts == nullptr)) return ZO_ERR_ARG;
  if (tokens < 0 || tokens > kMaxIndex || head_dim < 1 || head_dim > ZO_MAX_HEAD_DIM) return ZO_ERR_ARG;
  if (!known(dtype)) return ZO_ERR_DTYPE;
  if (!(std::isfinite(eps) && eps >= 0.0f) || (index_bytes != 4 && index_bytes != 8)) return ZO_ERR_ARG;
  zo::RotateParams r = {};
  bool rotate = false, slotted = false;
  const size_t size = element_size(dtype);
  for (int i = 0; i < n_parts; ++i) {
    const zo_head_part& in = parts[i];
    if (in.heads < 1 || in.heads > ZO_MAX_HEADS || (in.flags & ~(ZO_HEADS_ROTATE | ZO_HEADS_SLOTTED)) != 0 ||
        in.reserved != 0 || bad_strides(in.in.token, in.in.head) || bad_strides(in.out.token, in.out.head, in.out.page))
      return ZO_ERR_ARG;
    if (in.weight != nullptr && !known(in.weight_dtype)) return ZO_ERR_DTYPE;
    if (tokens > 0 && (in.in.ptr == nullptr || in.out.ptr == nullptr)) return ZO_ERR_ARG;
    if (misaligned(in.in.ptr, size) || misaligned(in.out.ptr, size) ||
        (in.weight != nullptr && misaligned(in.weight, element_size(in.weight_dtype))))
      return ZO_ERR_ALIGN;
    zo::RotatePart& out = r.part[i];
    const int64_t one = in.heads > 1;  // one head has no stride, nor has one token
    out = {in.in.ptr,         in.out.ptr,  in.weight,    tokens > 1 ? in.in.token : 0,
           in.in.head * one,  in.out.page, in.out.token, in.out.head * one,
           in.weight_dtype, in.heads, (in.flags & ZO_HEADS_ROTATE) != 0, (in.flags & ZO_HEADS_SLOTTED) != 0, 0};
    rotate = rotate || out.rotate;
    slotted = slotted || out.slotted;
  }
  if (rotate) {
    if (rotary_dim < 2 || rotary_dim % 2 != 0 || rotary_dim > head_dim || table_rows < 0 ||
        (layout != ZO_ROTARY_HALF && layout != ZO_ROTARY_INTERLEAVED))
      return ZO_ERR_ARG;
    if (tokens > 0 && (positions == nullptr || (table == nullptr && table_rows > 0))) return ZO_ERR_ARG;
    if (misaligned(table, 4) || misaligned(positions, index_bytes)) return ZO_ERR_ALIGN;
  }
  if (slotted) {
    if (n_slots < 0 || page_size < 1 || (tokens > 0 && slots == nullptr)) return ZO_ERR_ARG;
    if (misaligned(slots, index_bytes)) return ZO_ERR_ALIGN;
  }
  if (n_parts == 0 || tokens == 0) return ZO_OK;
  Tensor in[3], out[3];
  for (int i = 0; i < n_parts; ++i) {
    const zo_head_part& x = parts[i];
    in[i] = tensor(x.in, tokens, x.heads, head_dim, size);
    const zo_rows rows = {x.out.ptr, x.out.token, x.out.head};
    out[i] = (x.flags & ZO_HEADS_SLOTTED) == 0
                 ? tensor(rows, tokens, x.heads, head_dim, size)
                 : tensor(x.out, n_slots > 0 ? (n_slots - 1) / page_size + 1 : 0, std::min(n_slots, page_size), x.heads, head_dim, size);
  }
  for (int i = 0; i < n_parts; ++i) {
    const zo_head_part& x = parts[i];
    const bool in_place = same_rows(x.in, x.out.ptr, x.out.token, x.out.head, tokens, x.heads);
    if (folds(out[i])) return ZO_ERR_ARG;
    for (int j = 0; j < n_parts; ++j)
      if ((meet(out[i], in[j]) && !(i == j && in_place)) || (i < j && meet(out[i], out[j]))) return ZO_ERR_ARG;
  }
  r.n_parts = n_parts;
  r.dim = head_dim;
  r.rotary = rotate ? rotary_dim : 0;
  r.interleaved = layout == ZO_ROTARY_INTERLEAVED;
  r.index64 = index_bytes == 8;
  r.tokens = tokens;
  r.table = table;
  r.table_rows = table_rows;
  r.positions = positions;
  r.slots = slots;
  r.n_slots = n_slots;
  r.page_size = page_size;
  r.eps = eps;
  return finish(zo::launch_rotate_heads(r, dtype, static_cast<cudaStream_t>(stream)), "rotate_heads_kernel");
}

int zo_attention(const zo_rows* q, const zo_rows* k, const zo_rows* v, const zo_rows* out, int64_t q_tokens,
                 int64_t k_tokens, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t dtype,
                 const int32_t* spans, float scale, float softcap, const float* slopes, float* lse, void* stream) {
  if (q == nullptr || k == nullptr || v == nullptr || out == nullptr) return ZO_ERR_ARG;
  if (q_tokens < 0 || q_tokens > kMaxIndex || k_tokens < 0 || k_tokens > kMaxIndex) return ZO_ERR_ARG;
  int rc = check_heads(heads, kv_heads, head_dim, dtype);
  if (rc == ZO_OK) rc = check_scores(scale, softcap);
  if (rc != ZO_OK) return rc;
  if (bad_strides(q->token, q->head, k->token) || bad_strides(k->head, v->token, v->head) ||
      bad_strides(out->token, out->head))
    return ZO_ERR_ARG;
  if (q_tokens == 0) return ZO_OK;
  if (q->ptr == nullptr || out->ptr == nullptr || spans == nullptr) return ZO_ERR_ARG;
  if (k_tokens > 0 && (k->ptr == nullptr || v->ptr == nullptr)) return ZO_ERR_ARG;
  const size_t size = element_size(dtype);
  if (misaligned(q->ptr, size) || misaligned(k->ptr, size) || misaligned(v->ptr, size) || misaligned(out->ptr, size) ||
      misaligned(spans, 4) || misaligned(slopes, 4) || misaligned(lse, 4))
    return ZO_ERR_ALIGN;
  const Tensor to = tensor(*out, q_tokens, heads, head_dim, size);
  if (folds(to) || meet(to, tensor(*q, q_tokens, heads, head_dim, size)) ||
      meet(to, tensor(*k, k_tokens, kv_heads, head_dim, size)) || meet(to, tensor(*v, k_tokens, kv_heads, head_dim, size)))
    return ZO_ERR_ARG;
  const auto lone = [](int64_t stride, int64_t n) { return n > 1 ? stride : 0; };  // one element has no stride
  zo::AttentionParams p = {};
  p.q = q->ptr, p.k = k->ptr, p.v = v->ptr, p.out = out->ptr;
  p.q_token = lone(q->token, q_tokens), p.q_head = lone(q->head, heads);
  p.k_token = lone(k->token, k_tokens), p.k_head = lone(k->head, kv_heads);
  p.v_token = lone(v->token, k_tokens), p.v_head = lone(v->head, kv_heads);
  p.out_token = lone(out->token, q_tokens), p.out_head = lone(out->head, heads);
  p.q_tokens = q_tokens, p.k_tokens = k_tokens;
  p.heads = heads, p.group = heads / kv_heads, p.dim = head_dim;
  p.spans = spans;
  p.scale = scale, p.softcap = softcap;
  p.slopes = slopes;
  p.lse = lse;
  cudaError_t e = cudaSuccess;
  if (zo::launch_attention_mma(p, dtype, static_cast<cudaStream_t>(stream), &e)) return finish(e, "attention_mma_kernel");
  int sms = 0;
  rc = zo::device_sms(&sms);
  if (rc != ZO_OK) return rc;
  return finish(zo::launch_attention_tiles(p, dtype, sms, static_cast<cudaStream_t>(stream)), "attention_tiles_kernel");
}

int zo_attention_decode(const zo_rows* q, const zo_pages* k, const zo_pages* v, const zo_rows* out, int64_t batch,
                        int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t dtype, const int32_t* pages,
                        int64_t pages_stride, int64_t max_pages, int64_t n_pages, int32_t page_size,
                        const int32_t* lengths, float scale, float softcap, const float* slopes, float* lse,
                        void* stream) {
  if (q == nullptr || out == nullptr) return ZO_ERR_ARG;
  const zo_pages qs = {q->ptr, q->token, 0, q->head}, outs = {out->ptr, out->token, 0, out->head};
  zo::DraftParams p = {};
  int sms = 0;
  const int rc = check_paged(&qs, k, v, &outs, batch, 1, heads, kv_heads, head_dim, dtype, pages, pages_stride, max_pages,
                             n_pages, page_size, lengths, lengths, scale, softcap, slopes, lse, &p, &sms);
  if (rc != ZO_OK || batch == 0) return rc;
  cudaError_t e = cudaSuccess;
  if (zo::launch_decode_mma(p, batch, dtype, sms, static_cast<cudaStream_t>(stream), &e))
    return finish(e, "decode_mma_kernel");
  return finish(zo::launch_decode_scalar(p, batch, dtype, sms, static_cast<cudaStream_t>(stream)),
                "decode_scalar_kernel");
}

int zo_draft_masks(const int32_t* parents, int64_t batch, int32_t drafts, int64_t* masks, void* stream) {
  if (batch < 0 || batch > kMaxIndex / ZO_MAX_DRAFTS || drafts < 1 || drafts > ZO_MAX_DRAFTS) return ZO_ERR_ARG;
  if (batch == 0) return ZO_OK;
  if (parents == nullptr || masks == nullptr) return ZO_ERR_ARG;
  if (misaligned(parents, 4) || misaligned(masks, 8)) return ZO_ERR_ALIGN;
  if (meet(vector(masks, batch * drafts, 8), vector(parents, batch * drafts, 4))) return ZO_ERR_ARG;
  return finish(zo::launch_draft_masks(parents, batch, drafts, masks, static_cast<cudaStream_t>(stream)),
                "draft_masks_kernel");
}

int64_t zo_attention_draft_workspace_size(int64_t batch, int32_t drafts, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                          int32_t dtype) {
  if (batch < 0 || batch > kMaxIndex || drafts < 1 || drafts > ZO_MAX_DRAFTS || check_heads(heads, kv_heads, head_dim, dtype) != ZO_OK)
    return 0;
  return zo::draft_wide_work(batch, static_cast<int64_t>(drafts) * (heads / kv_heads), head_dim, dtype);
}

int zo_attention_draft(const zo_pages* q, const zo_pages* k, const zo_pages* v, const zo_pages* out, int64_t batch,
                       int32_t drafts, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t dtype,
                       const int32_t* pages, int64_t pages_stride, int64_t max_pages, int64_t n_pages,
                       int32_t page_size, const int32_t* lengths, const int64_t* masks, float scale, float softcap,
                       const float* slopes, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  if (q == nullptr || out == nullptr || drafts < 1 || drafts > ZO_MAX_DRAFTS) return ZO_ERR_ARG;
  zo::DraftParams p = {};
  int sms = 0;
  const int rc = check_paged(q, k, v, out, batch, drafts, heads, kv_heads, head_dim, dtype, pages, pages_stride, max_pages,
                             n_pages, page_size, lengths, masks, scale, softcap, slopes, lse, &p, &sms);
  if (rc != ZO_OK || batch == 0) return rc;
  if (misaligned(masks, 8) || misaligned(workspace, 16)) return ZO_ERR_ALIGN;
  const int64_t work = zo_attention_draft_workspace_size(batch, drafts, heads, kv_heads, head_dim, dtype);
  if (work > 0 && (workspace == nullptr || workspace_bytes < work)) return ZO_ERR_WORKSPACE;
  p.masks = masks;
  cudaError_t e = cudaSuccess;
  if (zo::launch_draft_wide(p, batch, dtype, sms, workspace, static_cast<cudaStream_t>(stream), &e))
    return finish(e, "draft_wide_kernel");
  if (zo::launch_draft_mma(p, batch, dtype, sms, static_cast<cudaStream_t>(stream), &e))
    return finish(e, "draft_mma_kernel");
  return finish(zo::launch_draft_scalar(p, batch, dtype, sms, static_cast<cudaStream_t>(stream)),
                "decode_scalar_kernel");
}

int64_t zo_token_loss_workspace_size(int64_t tokens) { return 8 * (tokens > 0 ? tokens : 1); }

int zo_token_loss(const void* logits, int64_t row, int64_t tokens, int64_t vocab, int32_t dtype, const void* targets,
                  int32_t target_bytes, int32_t flags, void* loss, float* nll, void* workspace,
                  int64_t workspace_bytes, void* stream) {
  int rc = check_rows(logits, row, tokens, vocab, dtype, targets, target_bytes, flags,
                      ZO_LOSS_MEAN | ZO_LOSS_ADD | ZO_LOSS_F32, loss);
  if (rc != ZO_OK) return rc;
  if (misaligned(nll, 4) || misaligned(workspace, 8)) return ZO_ERR_ALIGN;
  if (workspace == nullptr || workspace_bytes < zo_token_loss_workspace_size(tokens)) return ZO_ERR_WORKSPACE;
  int sms = 0;
  rc = zo::device_sms(&sms);
  if (rc != ZO_OK) return rc;
  zo::TokenLossParams p = {};
  p.logits = logits;
  p.row = row, p.tokens = tokens, p.vocab = vocab;
  p.targets = targets;
  p.target64 = target_bytes == 8, p.flags = flags;
  p.loss = loss, p.nll = nll;
  p.rows = static_cast<double*>(workspace);
  return finish(zo::launch_token_loss(p, dtype, sms, static_cast<cudaStream_t>(stream)), "token_loss_kernel");
}

int64_t zo_policy_loss_workspace_size(int64_t tokens) { return loss_work_size(tokens, 1); }

int zo_policy_loss(const void* logits, int64_t row, int64_t tokens, int64_t vocab, int32_t dtype, const void* targets,
                   int32_t target_bytes, const float* old_logp, const float* advantages, const float* ref_logp,
                   const float* weights, float clip_low, float clip_high, float kl, int32_t flags, void* loss,
                   void* grad, int64_t grad_row, float grad_scale, float* logp, void* workspace,
                   int64_t workspace_bytes, void* stream) {
  int rc = check_rows(logits, row, tokens, vocab, dtype, targets, target_bytes, flags,
                      ZO_LOSS_MEAN | ZO_LOSS_ADD | ZO_LOSS_F32, loss);
  if (rc != ZO_OK) return rc;
  if (!(clip_low >= 0.0f && clip_low <= 1.0f) || !(std::isfinite(clip_high) && clip_high >= 0.0f) || !(std::isfinite(kl) && kl >= 0.0f) ||
      (kl != 0.0f && ref_logp == nullptr && tokens > 0) || (tokens > 0 && (old_logp == nullptr || advantages == nullptr)))
    return ZO_ERR_ARG;
  rc = check_outputs(logits, row, grad, grad_row, grad_scale, tokens, vocab, dtype, vector(loss, 1, flags & ZO_LOSS_F32 ? 4 : 8),
                     vector(logp, tokens, 4),
                     {vector(targets, tokens, target_bytes), vector(old_logp, tokens, 4), vector(advantages, tokens, 4),
                      vector(ref_logp, tokens, 4), vector(weights, tokens, 4)});
  if (rc != ZO_OK) return rc;
  if (misaligned(workspace, 8)) return ZO_ERR_ALIGN;
  if (workspace == nullptr || workspace_bytes < zo_policy_loss_workspace_size(tokens)) return ZO_ERR_WORKSPACE;
  int sms = 0;
  rc = zo::device_sms(&sms);
  if (rc != ZO_OK) return rc;
  const LossWork work = loss_work(workspace, tokens, 1);
  zo::PolicyLossParams p = {};
  p.rows = {logits, row, tokens, vocab, targets, target_bytes == 8, flags, loss, work.logp, work.lse};
  p.old_logp = old_logp, p.advantages = advantages, p.weights = weights;
  p.ref_logp = kl != 0.0f ? ref_logp : nullptr;
  p.clip_low = clip_low, p.clip_high = clip_high, p.kl = kl;
  p.logp = logp;
  p.unit = flags & ZO_LOSS_MEAN ? reinterpret_cast<float*>(work.sums) : nullptr;
  p.slopes = grad != nullptr ? work.slopes : nullptr;
  const zo::LogitsGradParams g = {logits, grad, row, grad_row, tokens, vocab, targets, target_bytes == 8, work.slopes,
                                  work.lse, grad_scale};
  return finish(zo::launch_policy_loss(p, grad != nullptr ? &g : nullptr, dtype, sms, static_cast<cudaStream_t>(stream)),
                "zo_policy_loss");
}

int64_t zo_preference_loss_workspace_size(int64_t tokens, int64_t pairs) {
  return loss_work_size(tokens, 2 * (pairs > 0 ? pairs : 0));
}

int zo_preference_loss(const void* logits, int64_t row, int64_t tokens, int64_t vocab, int32_t dtype,
                       const void* targets, int32_t target_bytes, const int32_t* starts, int64_t pairs,
                       const float* ref_logp, float beta, float margin, float smoothing, int32_t flags, void* loss,
                       void* grad, int64_t grad_row, float grad_scale, float* logp, void* workspace,
                       int64_t workspace_bytes, void* stream) {
  int rc = check_rows(logits, row, tokens, vocab, dtype, targets, target_bytes, flags,
                      ZO_LOSS_MEAN | ZO_LOSS_ADD | ZO_LOSS_F32 | ZO_LOSS_BY_LENGTH, loss);
  if (rc != ZO_OK) return rc;
  if (pairs < 0 || pairs > kMaxIndex / 8 || starts == nullptr || !(std::isfinite(beta) && beta >= 0.0f) ||
      !std::isfinite(margin) || !(smoothing >= 0.0f && smoothing <= 1.0f))
    return ZO_ERR_ARG;
  rc = check_outputs(logits, row, grad, grad_row, grad_scale, tokens, vocab, dtype, vector(loss, 1, flags & ZO_LOSS_F32 ? 4 : 8),
                     vector(logp, 2 * pairs, 4),
                     {vector(targets, tokens, target_bytes), vector(starts, 2 * pairs + 1, 4), vector(ref_logp, 2 * pairs, 4)});
  if (rc != ZO_OK) return rc;
  if (misaligned(workspace, 8)) return ZO_ERR_ALIGN;
  if (workspace == nullptr || workspace_bytes < zo_preference_loss_workspace_size(tokens, pairs)) return ZO_ERR_WORKSPACE;
  int sms = 0;
  rc = zo::device_sms(&sms);
  if (rc != ZO_OK) return rc;
  const LossWork work = loss_work(workspace, tokens, 2 * pairs);
  zo::PreferenceLossParams p = {};
  p.rows = {logits, row, tokens, vocab, targets, target_bytes == 8, flags & ~ZO_LOSS_BY_LENGTH, loss, work.logp, work.lse};
  p.starts = starts;
  p.pairs = pairs;
  p.ref_logp = ref_logp;
  p.beta = beta, p.margin = margin, p.smoothing = smoothing;
  p.by_length = (flags & ZO_LOSS_BY_LENGTH) != 0;
  p.logp = logp;
  p.sums = work.sums, p.counts = work.counts;
  p.slopes = grad != nullptr ? work.slopes : nullptr;
  const zo::LogitsGradParams g = {logits, grad, row, grad_row, tokens, vocab, targets, target_bytes == 8, work.slopes,
                                  work.lse, grad_scale};
  return finish(zo::launch_preference_loss(p, grad != nullptr ? &g : nullptr, dtype, sms, static_cast<cudaStream_t>(stream)),
                "zo_preference_loss");
}

}  // extern "C"
