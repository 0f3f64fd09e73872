// Argument marshalling of the calls that a decode step makes for every layer and
// token: the checks of the tensors and the call of the C ABI, as a Python extension.
// In Python the same checks cost more than the launches (paged_append of 23 rows 11.4
// us a call, of which 2 us the launch and 1.6 us on the GPU). Each function takes
// tensors (or None) by position and returns the call's status; a tensor that does not
// fit raises ValueError or TypeError before anything is called.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <string>

#include "../../include/decomoe.h"

namespace {

struct Refused {
  PyObject* type;
  std::string what;
};
[[noreturn]] void refuse(PyObject* type, const std::string& what) { throw Refused{type, what}; }
void need(bool ok, const char* what) {
  if (!ok) refuse(PyExc_ValueError, what);
}

// The device of the tensors of the call that is being marshalled; -1: none seen yet.
thread_local int device_seen = -1;

// A strided device tensor argument; null for None where that is allowed.
const at::Tensor* tensor(PyObject* o, const char* what, bool none_ok = false) {
  if (o == Py_None && none_ok) return nullptr;
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, std::string(what) + ": a tensor expected");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.layout() != at::kStrided || !t.is_cuda()) refuse(PyExc_ValueError, std::string(what) + ": device tensors expected");
  const int at = static_cast<int>(t.get_device());
  if (device_seen >= 0 && at != device_seen) refuse(PyExc_ValueError, std::string(what) + ": all tensors must be on one device");
  device_seen = at;
  return &t;
}
// Launches, streams and the number of SMs go by the current device.
void on_current(const char* what) {
  if (device_seen >= 0 && device_seen != static_cast<int>(c10::cuda::current_device()))
    refuse(PyExc_ValueError, std::string(what) + ": the tensors are not on the current device");
}
const at::Tensor* whole(PyObject* o, const char* what, bool none_ok = false) {
  const at::Tensor* t = tensor(o, what, none_ok);
  if (t != nullptr && !t->is_contiguous()) refuse(PyExc_ValueError, std::string(what) + ": contiguous tensors expected");
  return t;
}
const at::Tensor* index(PyObject* o, const char* what, bool none_ok = false) {
  const at::Tensor* t = whole(o, what, none_ok);
  if (t != nullptr && t->scalar_type() != at::kInt)
    refuse(PyExc_ValueError, std::string(what) + ": index arrays must be contiguous int32 device tensors");
  return t;
}
template <typename T = void>
T* ptr(const at::Tensor* t) {
  return t == nullptr ? nullptr : static_cast<T*>(t->data_ptr());
}
int dtype(const at::Tensor& t, const char* what) {
  if (t.scalar_type() == at::kBFloat16) return DECOMOE_BF16;
  if (t.scalar_type() == at::kFloat) return DECOMOE_F32;
  refuse(PyExc_TypeError, std::string(what) + ": unsupported dtype");
}
bool shaped(const at::Tensor* t, std::initializer_list<int64_t> s) { return t->sizes() == at::IntArrayRef(s); }

// The stride (elements) between the rows of a tensor [N, ...] whose rows are
// contiguous; the rows may lie apart (slices of wider ones).
int64_t row_stride(const at::Tensor& t, const char* what) {
  int64_t inner = 1;
  for (int64_t i = t.dim() - 1; i >= 1; --i) {
    if (t.size(i) != 1 && t.stride(i) != inner) refuse(PyExc_ValueError, std::string(what) + ": rows must be contiguous");
    inner *= t.size(i);
  }
  return t.size(0) > 1 ? t.stride(0) : inner;
}

// The key and value pools [num_pages, page_size, Hkv, D].
struct Pool {
  const at::Tensor *k, *v;
  int64_t pages, ps, hkv, d, stride;
};
Pool pool(PyObject* k, PyObject* v, const char* what) {
  Pool p = {};
  p.k = tensor(k, what);
  p.v = tensor(v, what);
  if (p.k->dim() != 4 || p.k->sizes() != p.v->sizes() || p.k->scalar_type() != p.v->scalar_type())
    refuse(PyExc_ValueError, std::string(what) + ": two pools [num_pages, page_size, Hkv, D] of one shape and type expected");
  p.pages = p.k->size(0);
  p.ps = p.k->size(1);
  p.hkv = p.k->size(2);
  p.d = p.k->size(3);
  p.stride = row_stride(*p.k, what);
  if (row_stride(*p.v, what) != p.stride)
    refuse(PyExc_ValueError, std::string(what) + ": the two pools must have the same page stride");
  need(p.ps <= INT32_MAX && p.hkv <= INT32_MAX && p.d <= INT32_MAX && p.hkv * p.d <= INT32_MAX, "pool: sizes out of range");
  return p;
}

// The pool of a cache in 4 bits, [num_pages, Hkv, page_size / 8, tile bytes], for heads of d.
struct Pool4 {
  const at::Tensor* t;
  int64_t pages, ps, hkv, group, stride;
};
Pool4 pool4(PyObject* o, int64_t d, const char* what) {
  Pool4 p = {};
  p.t = tensor(o, what);
  if (p.t->dim() != 4 || p.t->scalar_type() != at::kByte)
    refuse(PyExc_ValueError, std::string(what) + ": a pool [num_pages, Hkv, page_size / 8, tile bytes] uint8 expected");
  p.pages = p.t->size(0);
  p.hkv = p.t->size(1);
  p.ps = 8 * p.t->size(2);
  const int64_t groups = d > 0 && d <= 128 ? (p.t->size(3) - 8 * d) / 64 : 0;
  if (groups < 1 || groups > d || d % groups != 0 || p.t->size(3) != 8 * d + 64 * groups)
    refuse(PyExc_ValueError, std::string(what) + ": a tile of the pool has 16 * (D / 2 + 4 * D / group) bytes");
  p.group = d / groups;
  p.stride = row_stride(*p.t, what);
  need(p.hkv <= INT32_MAX && p.t->size(2) <= INT32_MAX / 8, "pool: sizes out of range");
  return p;
}

int to_int(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{nullptr, ""};
  need(v >= INT32_MIN && v <= INT32_MAX, "an integer is out of range");
  return static_cast<int>(v);
}
float to_float(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{nullptr, ""};
  return static_cast<float>(v);
}
// The stream handle given, or (None) the current stream of the current device.
decomoe_stream_t stream(PyObject* o) {
  if (o == Py_None) return reinterpret_cast<decomoe_stream_t>(c10::cuda::getCurrentCUDAStream().stream());
  void* p = PyLong_AsVoidPtr(o);
  if (p == nullptr && PyErr_Occurred()) throw Refused{nullptr, ""};
  return reinterpret_cast<decomoe_stream_t>(p);
}

// cached, fresh, page_size, free_pages, block_table, seq_len, row_start, slot_map,
// positions, free_head, free_head_out, status, stream
int paged_plan(PyObject* const* a) {
  const char* n = "paged_plan";
  const at::Tensor *cached = index(a[0], n), *fresh = index(a[1], n), *pages = index(a[3], n), *table = index(a[4], n),
                   *len = index(a[5], n), *start = index(a[6], n), *slots = index(a[7], n), *pos = index(a[8], n, true),
                   *head = index(a[9], n, true), *head_out = index(a[10], n, true), *status = index(a[11], n, true);
  const int64_t B = cached->numel(), N = slots->numel();
  need(cached->dim() == 1 && slots->dim() == 1 && pages->dim() == 1 && shaped(fresh, {B}) && shaped(len, {B}) &&
           shaped(start, {B + 1}) && table->dim() == 2 && table->size(0) == B && (pos == nullptr || shaped(pos, {N})) &&
           (head == nullptr || head->numel() == 1) && (head_out == nullptr || head_out->numel() == 1) &&
           (status == nullptr || status->numel() >= 1),
       "paged_plan: cached, fresh, seq_len [B], row_start [B + 1], block_table [B, max_pages], free_pages [n], slot_map "
       "and positions [N], free_head and free_head_out [1] expected");
  on_current(n);
  return decomoe_paged_plan(ptr<int32_t>(cached), ptr<int32_t>(fresh), B, to_int(a[2]), ptr<int32_t>(pages), pages->numel(),
                            ptr<int32_t>(head), ptr<int32_t>(head_out), ptr<int32_t>(table), table->size(1),
                            ptr<int32_t>(len), ptr<int32_t>(start), ptr<int32_t>(slots), ptr<int32_t>(pos), N,
                            ptr<int32_t>(status), stream(a[12]));
}

// cached, fresh, page_size, free_pages, block_table, seq_len, slot_map, positions,
// free_head, free_head_out, status, stream
int paged_plan_step(PyObject* const* a) {
  const char* n = "paged_plan_step";
  const at::Tensor *cached = index(a[0], n), *fresh = index(a[1], n), *pages = index(a[3], n), *table = index(a[4], n),
                   *len = index(a[5], n), *slots = index(a[6], n), *pos = index(a[7], n, true), *head = index(a[8], n, true),
                   *head_out = index(a[9], n, true), *status = index(a[10], n, true);
  const int64_t B = cached->numel();
  need(cached->dim() == 1 && pages->dim() == 1 && shaped(fresh, {B}) && shaped(len, {B}) && shaped(slots, {B}) &&
           table->dim() == 2 && table->size(0) == B && (pos == nullptr || shaped(pos, {B})) &&
           (head == nullptr || head->numel() == 1) && (head_out == nullptr || head_out->numel() == 1) &&
           (status == nullptr || status->numel() >= 1),
       "paged_plan_step: cached, fresh, seq_len, slot_map and positions [B], block_table [B, max_pages], free_pages [n], "
       "free_head and free_head_out [1] expected");
  on_current(n);
  return decomoe_paged_plan_step(ptr<int32_t>(cached), ptr<int32_t>(fresh), B, to_int(a[2]), ptr<int32_t>(pages),
                                 pages->numel(), ptr<int32_t>(head), ptr<int32_t>(head_out), ptr<int32_t>(table),
                                 table->size(1), ptr<int32_t>(len), ptr<int32_t>(slots), ptr<int32_t>(pos),
                                 ptr<int32_t>(status), stream(a[11]));
}

// cached, seq_len, block_table, page_size, free_head, free_head_out, stream
int paged_advance(PyObject* const* a) {
  const char* n = "paged_advance";
  const at::Tensor *cached = index(a[0], n), *len = index(a[1], n), *table = index(a[2], n), *head = index(a[4], n, true),
                   *head_out = index(a[5], n, true);
  const int64_t B = cached->numel();
  need(cached->dim() == 1 && shaped(len, {B}) && table->dim() == 2 && table->size(0) == B &&
           (head == nullptr || head->numel() == 1) && (head_out == nullptr || head_out->numel() == 1),
       "paged_advance: cached and seq_len [B], block_table [B, max_pages], free_head and free_head_out [1] expected");
  on_current(n);
  return decomoe_paged_advance(ptr<int32_t>(cached), ptr<int32_t>(len), ptr<int32_t>(table), B, table->size(1),
                               to_int(a[3]), ptr<int32_t>(head), ptr<int32_t>(head_out), stream(a[6]));
}

// k_new, v_new, slot_map, k_pages, v_pages, status, stream
int paged_append(PyObject* const* a) {
  const char* n = "paged_append";
  const Pool p = pool(a[3], a[4], n);
  const at::Tensor *k = tensor(a[0], n), *v = tensor(a[1], n), *slots = index(a[2], n), *status = index(a[5], n, true);
  const int64_t N = slots->numel();
  need(slots->dim() == 1 && shaped(k, {N, p.hkv, p.d}) && shaped(v, {N, p.hkv, p.d}) &&
           (status == nullptr || status->numel() >= 1),
       "paged_append: k_new, v_new [N, Hkv, D] and slot_map [N] expected");
  if (k->scalar_type() != p.k->scalar_type() || v->scalar_type() != p.k->scalar_type())
    refuse(PyExc_TypeError, "paged_append: rows and pools must have one type");
  on_current(n);
  return decomoe_paged_append(ptr(k), row_stride(*k, n), ptr(v), row_stride(*v, n), N, static_cast<int>(p.hkv * p.d),
                              dtype(*p.k, n), ptr<int32_t>(slots), ptr(p.k), ptr(p.v), p.pages, static_cast<int>(p.ps),
                              p.stride, ptr<int32_t>(status), stream(a[6]));
}

// q, k_pages, v_pages, block_table, seq_len, out, ws, hide_begin, hide_count, scale, status, stream
int paged_attention(PyObject* const* a) {
  const char* n = "paged_attention";
  const Pool p = pool(a[1], a[2], n);
  const at::Tensor *q = tensor(a[0], n), *table = index(a[3], n), *len = index(a[4], n), *out = whole(a[5], n),
                   *ws = whole(a[6], n), *hb = index(a[7], n, true), *hc = index(a[8], n, true),
                   *status = index(a[10], n, true);
  need(q->dim() == 3 && q->size(2) == p.d && out->sizes() == q->sizes(),
       "paged_attention: q and out [B, Hq, D] expected, D as the pools have it");
  const int64_t B = q->size(0), hq = q->size(1);
  need(shaped(len, {B}) && table->dim() == 2 && table->size(0) == B && (hb == nullptr || shaped(hb, {B})) &&
           (hc == nullptr || shaped(hc, {B})) && (status == nullptr || status->numel() >= 1) && hq <= INT32_MAX,
       "paged_attention: block_table [B, max_pages], seq_len, hide_begin and hide_count [B] expected");
  if (q->scalar_type() != at::kBFloat16 || p.k->scalar_type() != at::kBFloat16 || out->scalar_type() != at::kBFloat16)
    refuse(PyExc_TypeError, "paged_attention: q, pools and out must be bf16");
  on_current(n);
  return decomoe_paged_attention(ptr(q), row_stride(*q, n), B, ptr(p.k), ptr(p.v), p.pages, static_cast<int>(p.ps), p.stride,
                                 ptr<int32_t>(table), table->size(1), ptr<int32_t>(len), ptr<int32_t>(hb), ptr<int32_t>(hc),
                                 static_cast<int>(hq), static_cast<int>(p.hkv), static_cast<int>(p.d), to_float(a[9]),
                                 ptr(out), ptr(ws), ws->nbytes(), ptr<int32_t>(status), stream(a[11]));
}

// k_new, v_new, slot_map, pages, status, stream
int paged_append_q4(PyObject* const* a) {
  const char* n = "paged_append_q4";
  const at::Tensor *k = tensor(a[0], n), *v = tensor(a[1], n), *slots = index(a[2], n), *status = index(a[4], n, true);
  need(k->dim() == 3, "paged_append_q4: k_new [N, Hkv, D] expected");
  const Pool4 p = pool4(a[3], k->size(2), n);
  const int64_t N = slots->numel(), d = k->size(2);
  need(slots->dim() == 1 && shaped(k, {N, p.hkv, d}) && shaped(v, {N, p.hkv, d}) && (status == nullptr || status->numel() >= 1),
       "paged_append_q4: k_new, v_new [N, Hkv, D] and slot_map [N] expected");
  if (k->scalar_type() != at::kBFloat16 || v->scalar_type() != at::kBFloat16)
    refuse(PyExc_TypeError, "paged_append_q4: rows must be bf16");
  on_current(n);
  return decomoe_paged_append_q4(ptr(k), row_stride(*k, n), ptr(v), row_stride(*v, n), N, static_cast<int>(p.hkv),
                                 static_cast<int>(d), static_cast<int>(p.group), ptr<int32_t>(slots), ptr(p.t), p.pages,
                                 static_cast<int>(p.ps), p.stride, ptr<int32_t>(status), stream(a[5]));
}

// slot_map, pages, k_out, v_out, status, stream
int paged_read_q4(PyObject* const* a) {
  const char* n = "paged_read_q4";
  const at::Tensor *slots = index(a[0], n), *k = tensor(a[2], n), *v = tensor(a[3], n), *status = index(a[4], n, true);
  need(k->dim() == 3, "paged_read_q4: k_out [N, Hkv, D] expected");
  const Pool4 p = pool4(a[1], k->size(2), n);
  const int64_t N = slots->numel(), d = k->size(2);
  need(slots->dim() == 1 && shaped(k, {N, p.hkv, d}) && shaped(v, {N, p.hkv, d}) && (status == nullptr || status->numel() >= 1),
       "paged_read_q4: k_out, v_out [N, Hkv, D] and slot_map [N] expected");
  if (k->scalar_type() != at::kBFloat16 || v->scalar_type() != at::kBFloat16)
    refuse(PyExc_TypeError, "paged_read_q4: rows must be bf16");
  on_current(n);
  return decomoe_paged_read_q4(ptr<int32_t>(slots), N, ptr(p.t), p.pages, static_cast<int>(p.ps), p.stride,
                               static_cast<int>(p.hkv), static_cast<int>(d), static_cast<int>(p.group), ptr(k),
                               row_stride(*k, n), ptr(v), row_stride(*v, n), ptr<int32_t>(status), stream(a[5]));
}

// q, pages, block_table, seq_len, out, ws, hide_begin, hide_count, scale, status, stream
int paged_attention_q4(PyObject* const* a) {
  const char* n = "paged_attention_q4";
  const at::Tensor *q = tensor(a[0], n), *table = index(a[2], n), *len = index(a[3], n), *out = whole(a[4], n),
                   *ws = whole(a[5], n), *hb = index(a[6], n, true), *hc = index(a[7], n, true),
                   *status = index(a[9], n, true);
  need(q->dim() == 3 && out->sizes() == q->sizes(), "paged_attention_q4: q and out [B, Hq, D] expected");
  const int64_t B = q->size(0), hq = q->size(1), d = q->size(2);
  const Pool4 p = pool4(a[1], d, n);
  need(shaped(len, {B}) && table->dim() == 2 && table->size(0) == B && (hb == nullptr || shaped(hb, {B})) &&
           (hc == nullptr || shaped(hc, {B})) && (status == nullptr || status->numel() >= 1) && hq <= INT32_MAX,
       "paged_attention_q4: block_table [B, max_pages], seq_len, hide_begin and hide_count [B] expected");
  if (q->scalar_type() != at::kBFloat16 || out->scalar_type() != at::kBFloat16)
    refuse(PyExc_TypeError, "paged_attention_q4: q and out must be bf16");
  on_current(n);
  return decomoe_paged_attention_q4(ptr(q), row_stride(*q, n), B, ptr(p.t), p.pages, static_cast<int>(p.ps), p.stride,
                                    static_cast<int>(p.group), ptr<int32_t>(table), table->size(1), ptr<int32_t>(len),
                                    ptr<int32_t>(hb), ptr<int32_t>(hc), static_cast<int>(hq), static_cast<int>(p.hkv),
                                    static_cast<int>(d), to_float(a[8]), ptr(out), ptr(ws), ws->nbytes(),
                                    ptr<int32_t>(status), stream(a[10]));
}

// logits, tokens, logprob, entropy, top_id, top_logprob, scale, status, stream
int token_logprobs(PyObject* const* a) {
  const char* n = "token_logprobs";
  const at::Tensor *x = tensor(a[0], n), *tokens = index(a[1], n, true), *logprob = whole(a[2], n, true),
                   *entropy = whole(a[3], n, true), *id = index(a[4], n, true), *top = whole(a[5], n, true),
                   *status = index(a[7], n, true);
  need(x->dim() == 2, "token_logprobs: logits [T, V] expected");
  const int64_t T = x->size(0), V = x->size(1);
  need((tokens == nullptr || shaped(tokens, {T})) && (logprob == nullptr || shaped(logprob, {T})) &&
           (entropy == nullptr || shaped(entropy, {T})) && (status == nullptr || status->numel() >= 1),
       "token_logprobs: tokens, logprob and entropy [T] expected");
  const at::Tensor* best = id != nullptr ? id : top;
  int64_t k = 0;
  if (best != nullptr) {
    need(best->dim() == 2 && best->size(0) == T, "token_logprobs: top_id and top_logprob [T, n] expected");
    k = best->size(1);
    need((id == nullptr || shaped(id, {T, k})) && (top == nullptr || shaped(top, {T, k})) && k <= INT32_MAX,
         "token_logprobs: top_id and top_logprob must have one shape");
  }
  for (const at::Tensor* t : {logprob, entropy, top})
    if (t != nullptr && t->scalar_type() != at::kFloat)
      refuse(PyExc_TypeError, "token_logprobs: logprob, entropy and top_logprob must be float32");
  on_current(n);
  return decomoe_token_logprobs(ptr(x), T, V, row_stride(*x, n), dtype(*x, n), ptr<int32_t>(tokens), to_float(a[6]),
                                static_cast<int>(k), ptr<float>(logprob), ptr<float>(entropy), k > 0 ? ptr<int32_t>(id) : nullptr,
                                k > 0 ? ptr<float>(top) : nullptr, ptr<int32_t>(status), stream(a[8]));
}

// x, residual, weight, sum_out, y, y8, y8_scale, eps, stream
int add_rmsnorm_q8(PyObject* const* a) {
  const char* n = "add_rmsnorm_q8";
  const at::Tensor *x = whole(a[0], n), *res = whole(a[1], n, true), *w = whole(a[2], n, true), *sum = whole(a[3], n, true),
                   *y = whole(a[4], n, true), *y8 = whole(a[5], n, true), *scale = whole(a[6], n, true);
  need(x->dim() == 2 && x->size(1) <= INT32_MAX, "add_rmsnorm_q8: x [T, d] expected");
  const int64_t T = x->size(0), d = x->size(1);
  for (const at::Tensor* t : {res, sum, y})
    need(t == nullptr || (t->sizes() == x->sizes() && t->scalar_type() == x->scalar_type()),
         "add_rmsnorm_q8: residual, sum_out and y must have x's shape and type");
  need(w == nullptr || (shaped(w, {d}) && w->scalar_type() == x->scalar_type()),
       "add_rmsnorm_q8: weight [d] of x's type expected");
  need(y8 == nullptr || (y8->sizes() == x->sizes() && y8->scalar_type() == at::kFloat8_e4m3fn),
       "add_rmsnorm_q8: y8 [T, d] float8_e4m3fn expected");
  need(scale == nullptr || (scale->numel() == T && scale->scalar_type() == at::kFloat),
       "add_rmsnorm_q8: y8_scale [T] float32 expected");
  on_current(n);
  return decomoe_add_rmsnorm_q8(ptr(x), ptr(res), ptr(w), T, static_cast<int>(d), to_float(a[7]), dtype(*x, n), ptr(sum),
                                ptr(y), ptr(y8), ptr<float>(scale), stream(a[8]));
}

// x, w, w_scale, out, x_scale, stream
int w4_linear(PyObject* const* a) {
  const char* n = "w4_linear";
  const at::Tensor *x = tensor(a[0], n), *w = whole(a[1], n), *ws = whole(a[2], n), *out = whole(a[3], n),
                   *xs = whole(a[4], n, true);
  need(x->dim() == 2 && x->size(1) <= INT32_MAX && w->dim() == 2, "w4_linear: x [T, K] and w [N, K / 2] expected");
  const int64_t T = x->size(0), K = x->size(1), N = w->size(0);
  need(K % 2 == 0 && shaped(w, {N, K / 2}) && w->scalar_type() == at::kByte && ws->dim() == 2 && ws->size(0) == N &&
           ws->scalar_type() == at::kBFloat16,
       "w4_linear: w [N, K / 2] uint8 and w_scale [N, K / group] bf16 expected");
  need(shaped(out, {T, N}), "w4_linear: out [T, N] expected");
  const int64_t groups = ws->size(1);
  need(groups > 0 && K % groups == 0, "w4_linear: K must be groups * group");
  int xt = DECOMOE_E4M3;
  if (x->scalar_type() == at::kFloat8_e4m3fn)
    need(xs != nullptr && xs->scalar_type() == at::kFloat && xs->numel() == T, "w4_linear: e4m3 rows need x_scale [T] float32");
  else
    xt = dtype(*x, n);
  on_current(n);
  return decomoe_w4_linear(ptr(x), xt, row_stride(*x, n), ptr<float>(xs), T, static_cast<int>(K), ptr(w), ptr(ws),
                           static_cast<int>(K / groups), N, ptr(out), dtype(*out, n), stream(a[5]));
}

template <int (*F)(PyObject* const*), int ARGS>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    device_seen = -1;
    if (n != ARGS) refuse(PyExc_TypeError, "wrong number of arguments");
    return PyLong_FromLong(F(args));
  } catch (const Refused& e) {
    if (e.type != nullptr) PyErr_SetString(e.type, e.what.c_str());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

#define DM_ENTRY(name, args) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<name, args>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {DM_ENTRY(paged_plan, 13),   DM_ENTRY(paged_plan_step, 12),  DM_ENTRY(paged_advance, 7),
                         DM_ENTRY(paged_append, 7),  DM_ENTRY(paged_attention, 12), DM_ENTRY(paged_append_q4, 6),
                         DM_ENTRY(paged_read_q4, 6), DM_ENTRY(paged_attention_q4, 11), DM_ENTRY(token_logprobs, 9),
                         DM_ENTRY(add_rmsnorm_q8, 9), DM_ENTRY(w4_linear, 6),     {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
