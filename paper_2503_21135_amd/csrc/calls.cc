// calls.cc -- the Python module _calls: marshals torch tensors into the entry points of the
// normed append, the cache in 8 bits and the verification of drafts.
//
// These calls take a few microseconds on the device.  Checking their dozen tensors (type, shape,
// strides, device) in Python takes seven; here it takes a fraction of one.  Nothing else happens
// here: the entry points check what they can see, and everything else runs in their kernels.
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <stdexcept>
#include <string>

#include "moe_quant.h"

namespace {

PyObject* g_error = nullptr;   // MoEError

struct Entries {
  decltype(&moe_cache_append_norm) append_norm;
  decltype(&moe_qcache_append) append;
  decltype(&moe_qcache_read) read;
  decltype(&moe_qcache_attention) attention;
  decltype(&moe_qcache_keep) keep;
  decltype(&moe_draft_verify) verify;
} g_entry{};

std::string text(const char* format, ...) {
  char buf[512];
  va_list args;
  va_start(args, format);
  vsnprintf(buf, sizeof buf, format, args);
  va_end(args);
  return buf;
}
[[noreturn]] void refuse(const std::string& what) { throw std::runtime_error(what); }

const at::Tensor* tensor(PyObject* o, const char* what, bool optional = false) {
  if (o == Py_None && optional) return nullptr;
  if (!THPVariable_Check(o)) refuse(text("%s must be a tensor", what));
  return &THPVariable_Unpack(o);
}
int64_t number(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw std::invalid_argument("");   // the Python error stands
  return v;
}
int32_t small(PyObject* o, const char* what) {
  const int64_t v = number(o);
  if (v < INT32_MIN || v > INT32_MAX) refuse(text("%s = %lld is out of range", what, static_cast<long long>(v)));
  return static_cast<int32_t>(v);
}
int32_t size32(int64_t n, const char* what) {
  if (n > INT32_MAX) refuse(text("%s: too many", what));
  return static_cast<int32_t>(n);
}

std::string described(const at::Tensor& t) {
  std::string s = std::string(at::toString(t.scalar_type())) + " (";
  for (int64_t i = 0; i < t.dim(); i++) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + ") on " + t.device().str();
}

// the device that a call works on: where `t` is, and its other tensors have to be
int device_of(const at::Tensor& t, const char* what) {
  if (!t.is_cuda()) refuse(text("%s must be a device tensor", what));
  return t.get_device();
}
void* array(const at::Tensor* t, int64_t n, at::ScalarType type, int dev, const char* what) {
  if (!t) return nullptr;
  if (t->scalar_type() != type || t->numel() != n || !t->is_cuda() || t->get_device() != dev || !t->is_contiguous())
    refuse(text("%s must be %lld contiguous values of %s on device %d, not %s", what, static_cast<long long>(n), at::toString(type), dev,
                described(*t).c_str()));
  return t->data_ptr();
}
void* array(PyObject* o, int64_t n, at::ScalarType type, int dev, const char* what, bool optional = true) {
  return array(tensor(o, what, optional), n, type, dev, what);
}
// a [N][H][D] tensor whose heads lie side by side: data, and the stride of a token
struct Heads { void* at = nullptr; int64_t ld = 0; };
Heads heads(const at::Tensor* t, int64_t N, int64_t H, int64_t D, at::ScalarType type, int dev, const char* what) {
  if (!t) return {};
  if (t->scalar_type() != type || t->dim() != 3 || t->size(0) != N || t->size(1) != H || t->size(2) != D || !t->is_cuda() ||
      t->get_device() != dev || t->stride(2) != 1 || (t->stride(1) != D && H > 1))
    refuse(text("%s must be a %s tensor of shape (%lld, %lld, %lld) on device %d, the heads of a token side by side, not %s", what,
                at::toString(type), static_cast<long long>(N), static_cast<long long>(H), static_cast<long long>(D), dev, described(*t).c_str()));
  return {t->data_ptr(), N > 1 ? t->stride(0) : H * D};
}
// a [T][n] tensor whose rows are contiguous
Heads rows(const at::Tensor* t, int64_t T, int64_t n, int dev, const char* what) {
  if (!t) return {};
  if (t->dim() != 2 || t->size(0) != T || t->size(1) != n || !t->is_cuda() || t->get_device() != dev || (t->stride(1) != 1 && n > 1))
    refuse(text("%s must be a tensor of shape (%lld, %lld) on device %d with contiguous rows, not %s", what, static_cast<long long>(T),
                static_cast<long long>(n), dev, described(*t).c_str()));
  return {t->data_ptr(), T > 1 ? t->stride(0) : n};
}
int type_of(const at::Tensor& t, const char* what) {
  switch (t.scalar_type()) {
    case at::kBFloat16: return MOE_TYPE_BF16;
    case at::kHalf: return MOE_TYPE_FP16;
    case at::kFloat: return MOE_TYPE_FP32;
    default: refuse(text("%s must be bfloat16, float16 or float32, not %s", what, at::toString(t.scalar_type())));
  }
}
at::ScalarType type16(int type) { return type == MOE_TYPE_BF16 ? at::kBFloat16 : at::kHalf; }

// table, lengths and row offsets of a batch
struct Batch { const int32_t *table, *len, *off; int32_t pages, n_seqs; };
Batch batch(PyObject* const* a, int dev) {
  const at::Tensor &table = *tensor(a[0], "table"), &len = *tensor(a[1], "cache_len");
  if (table.dim() != 2) refuse("table must be [sequences][pages]");
  const int64_t B = len.numel();
  return {static_cast<int32_t*>(array(&table, B * table.size(1), at::kInt, dev, "table")), static_cast<int32_t*>(array(&len, B, at::kInt, dev, "cache_len")),
          static_cast<int32_t*>(array(a[2], B + 1, at::kInt, dev, "new_off", false)), size32(table.size(1), "pages"), size32(B, "sequences")};
}

void count(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) refuse(text("%lld arguments, not %lld", static_cast<long long>(n), static_cast<long long>(want)));
}
template <class T>
T* address(PyObject* o) { return reinterpret_cast<T*>(number(o)); }

// C++ exceptions end here
template <int (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    return PyLong_FromLong(F(a, n));
  } catch (const std::invalid_argument&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(g_error ? g_error : PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

// desc, table, lens, new_off, max_new, q, k, v, q_out, w_q, w_k, eps, positions, cos, sin, interleaved, status, stream
template <class CACHE, class CALL>
int append_to(CALL call, PyObject* const* a, Py_ssize_t n) {
  count(n, 18);
  const CACHE* C = address<CACHE>(a[0]);
  const at::Tensor &k = *tensor(a[6], "k"), *q = tensor(a[5], "q", true), *q_out = tensor(a[8], "q_out", true), *cos = tensor(a[13], "cos", true);
  const int dev = device_of(k, "k");
  if (!q != !q_out || !cos != (a[14] == Py_None)) refuse("q and q_out, cos and sin come in pairs");
  if (k.dim() != 3 || (q && q->dim() != 3)) refuse("q, k and v must be [tokens][heads][head_dim]");
  if (cos && (cos->dim() != 2 || cos->numel() == 0)) refuse("cos and sin must be [positions][half], and not empty");
  const int64_t N = k.size(0), D = C->head_dim, Hq = q ? q->size(1) : 0, max_pos = cos ? cos->size(0) : 1, half = cos ? cos->size(1) : 0;
  const at::ScalarType t = type16(C->type);
  const Batch b = batch(a + 1, dev);
  const Heads qh = heads(q, N, Hq, D, t, dev, "q"), kh = heads(&k, N, C->n_heads, D, t, dev, "k"),
              vh = heads(tensor(a[7], "v"), N, C->n_heads, D, t, dev, "v"), oh = heads(q_out, N, Hq, D, t, dev, "q_out");
  const double eps = PyFloat_AsDouble(a[11]);
  if (eps == -1. && PyErr_Occurred()) throw std::invalid_argument("");
  const int interleaved = PyObject_IsTrue(a[15]);
  if (interleaved < 0) throw std::invalid_argument("");
  return call(C, b.table, b.pages, b.len, b.n_seqs, b.off, size32(N, "tokens"), small(a[4], "max_new"), qh.at, qh.ld, size32(Hq, "heads"), kh.at,
              kh.ld, vh.at, vh.ld, static_cast<float*>(array(a[9], D, at::kFloat, dev, "w_q")),
              static_cast<float*>(array(a[10], D, at::kFloat, dev, "w_k")), static_cast<float>(eps),
              static_cast<int32_t*>(array(a[12], N, at::kInt, dev, "positions")), static_cast<float*>(array(cos, max_pos * half, at::kFloat, dev, "cos")),
              static_cast<float*>(array(a[14], max_pos * half, at::kFloat, dev, "sin")), size32(2 * half, "rotated channels"),
              size32(max_pos, "positions"), interleaved, oh.at, oh.ld, static_cast<int32_t*>(array(a[16], 1, at::kInt, dev, "status")),
              address<void>(a[17]));
}
int append_norm(PyObject* const* a, Py_ssize_t n) { return append_to<moe_cache_t>(g_entry.append_norm, a, n); }
int append(PyObject* const* a, Py_ssize_t n) { return append_to<moe_qcache_t>(g_entry.append, a, n); }

// desc, table, first, row_off, max_rows, k_out, v_out, status, stream
int read(PyObject* const* a, Py_ssize_t n) {
  count(n, 9);
  const moe_qcache_t* C = address<moe_qcache_t>(a[0]);
  const at::Tensor *k = tensor(a[5], "k_out", true), *v = tensor(a[6], "v_out", true), *any = k ? k : v;
  if (!any) refuse("k_out or v_out must be given");
  const int dev = device_of(*any, "k_out and v_out");
  if (any->dim() != 3) refuse("k_out and v_out must be [rows][heads][head_dim]");
  const int64_t N = any->size(0);
  const at::ScalarType t = type16(C->type);
  const Batch b = batch(a + 1, dev);
  const Heads kh = heads(k, N, C->n_heads, C->head_dim, t, dev, "k_out"), vh = heads(v, N, C->n_heads, C->head_dim, t, dev, "v_out");
  return g_entry.read(C, b.table, b.pages, b.len, b.n_seqs, b.off, size32(N, "rows"), small(a[4], "max_rows"), kh.at, kh.ld, vh.at, vh.ld,
                      static_cast<int32_t*>(array(a[7], 1, at::kInt, dev, "status")), address<void>(a[8]));
}

// desc, table, lens, new_off, max_new, max_len, q, out, scale, mask, ws, status, stream
int attention(PyObject* const* a, Py_ssize_t n) {
  count(n, 13);
  const moe_qcache_t* C = address<moe_qcache_t>(a[0]);
  const at::Tensor &q = *tensor(a[6], "q"), *mask = tensor(a[9], "mask", true), *ws = tensor(a[10], "ws", true);
  const int dev = device_of(q, "q");
  if (q.dim() != 3 || q.size(2) != C->head_dim) refuse(text("q must be [tokens][heads][%d], not %s", C->head_dim, described(q).c_str()));
  const int64_t N = q.size(0), Hq = q.size(1), words = mask ? (mask->dim() ? mask->size(-1) : 0) : 0, bytes = ws ? ws->numel() : 0;
  if (mask && words < 1) refuse("mask must be [tokens][words], a word at least");   // an empty one has no address, as none
  const at::ScalarType t = type16(C->type);
  const Batch b = batch(a + 1, dev);
  const Heads qh = heads(&q, N, Hq, C->head_dim, t, dev, "q"), oh = heads(tensor(a[7], "out"), N, Hq, C->head_dim, t, dev, "out");
  const double scale = PyFloat_AsDouble(a[8]);
  if (scale == -1. && PyErr_Occurred()) throw std::invalid_argument("");
  return g_entry.attention(C, b.table, b.pages, b.len, b.n_seqs, b.off, size32(N, "tokens"), small(a[4], "max_new"), small(a[5], "max_len"), qh.at, qh.ld,
                           size32(Hq, "heads"), static_cast<uint64_t*>(array(mask, N * words, at::kLong, dev, "mask")), size32(words, "mask words"),
                           static_cast<float>(scale), oh.at, oh.ld, static_cast<int32_t*>(array(a[11], 1, at::kInt, dev, "status")),
                           array(ws, bytes, at::kByte, dev, "ws"), static_cast<size_t>(bytes), address<void>(a[12]));
}

// desc, table, lens, new_off, keep, n_keep, len_out, status, stream
int keep(PyObject* const* a, Py_ssize_t n) {
  count(n, 9);
  const at::Tensor &len = *tensor(a[2], "cache_len"), &list = *tensor(a[4], "keep");
  const int dev = device_of(len, "cache_len");
  const Batch b = batch(a + 1, dev);
  const int64_t most = list.dim() ? list.size(-1) : 0;
  return g_entry.keep(address<moe_qcache_t>(a[0]), b.table, b.pages, b.len, b.n_seqs, b.off,
                      static_cast<int32_t*>(array(&list, b.n_seqs * most, at::kInt, dev, "keep")), size32(most, "kept tokens"),
                      static_cast<int32_t*>(array(a[5], b.n_seqs, at::kInt, dev, "n_keep", false)),
                      static_cast<int32_t*>(array(a[6], b.n_seqs, at::kInt, dev, "len_out")),
                      static_cast<int32_t*>(array(a[7], 1, at::kInt, dev, "status")), address<void>(a[8]));
}

// logits, tokens, new_off, max_new, keep, n_keep, next, ws, parents, draft, u, u_next, temperature, status, stream
int verify(PyObject* const* a, Py_ssize_t n) {
  count(n, 15);
  const at::Tensor &logits = *tensor(a[0], "logits"), &kept = *tensor(a[5], "n_keep"), *draft = tensor(a[9], "draft_probs", true), &ws = *tensor(a[7], "ws");
  const int dev = device_of(logits, "logits");
  if (logits.dim() != 2) refuse("logits must be [rows][vocabulary]");
  const int64_t N = logits.size(0), V = logits.size(1), B = kept.numel();
  const int32_t most = small(a[3], "max_new");
  const Heads l = rows(&logits, N, V, dev, "logits"), d = rows(draft, N, V, dev, "draft_probs");
  auto ints = [&](int i, int64_t k, const char* what, bool optional) { return static_cast<int32_t*>(array(a[i], k, at::kInt, dev, what, optional)); };
  auto floats = [&](int i, int64_t k, const char* what) { return static_cast<float*>(array(a[i], k, at::kFloat, dev, what)); };
  return g_entry.verify(l.at, type_of(logits, "logits"), l.ld, size32(N, "rows"), size32(V, "vocabulary"), ints(1, N, "tokens", false), ints(8, N, "parents", true),
                        ints(2, B + 1, "new_off", false), size32(B, "sequences"), most, d.at, draft ? type_of(*draft, "draft_probs") : 0, d.ld,
                        floats(12, B, "temperature"), floats(10, N, "u"), floats(11, B, "u_next"), ints(4, B * std::max(most, 0), "keep", false),
                        ints(5, B, "n_keep", false), ints(6, B, "next_token", false), ints(13, 1, "status", true),
                        array(&ws, ws.numel(), at::kByte, dev, "ws"), static_cast<size_t>(ws.numel()), address<void>(a[14]));
}

// bind(MoEError, addresses of the six entry points)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "bind takes the error class and six addresses");
    return nullptr;
  }
  long long at[6];
  for (int i = 0; i < 6; i++) {
    at[i] = PyLong_AsLongLong(a[i + 1]);
    if (PyErr_Occurred()) return nullptr;
  }
  Py_INCREF(a[0]);
  Py_XSETREF(g_error, a[0]);
  g_entry = {reinterpret_cast<decltype(g_entry.append_norm)>(at[0]), reinterpret_cast<decltype(g_entry.append)>(at[1]),
             reinterpret_cast<decltype(g_entry.read)>(at[2]), reinterpret_cast<decltype(g_entry.attention)>(at[3]),
             reinterpret_cast<decltype(g_entry.keep)>(at[4]), reinterpret_cast<decltype(g_entry.verify)>(at[5])};
  Py_RETURN_NONE;
}

#define FAST(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {FAST("bind", bind),
                          FAST("append_norm", (entry<append_norm>)),
                          FAST("append", (entry<append>)),
                          FAST("read", (entry<read>)),
                          FAST("attention", (entry<attention>)),
                          FAST("keep", (entry<keep>)),
                          FAST("verify", (entry<verify>)),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&kModule); }
