// The Python side of h2o_rotate, h2o_pages_append and h2o_pages_attend: checks of tensors and packing of arguments.  A decoding
// step is a few microseconds on the GPU; the same checks in Python take longer than that (append of 64 tokens: 8.1 us a call
// with them there, 5 with them here).  Calls the C ABI through addresses that binding.py passes in, so it belongs to whichever
// build of the library is loaded.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "h2o.h"

namespace {

decltype(&h2o_rotate) rotate_fn = nullptr;
decltype(&h2o_pages_append) append_fn = nullptr;
decltype(&h2o_pages_scratch_bytes) scratch_fn = nullptr;
decltype(&h2o_pages_attend) attend_fn = nullptr;

// A refused argument: becomes a ValueError.
struct Refused {
  const char* why;
};
void need(bool ok, const char* why) {
  if (!ok) throw Refused{why};
}

const at::Tensor& tensor(PyObject* o, const char* why) {
  need(THPVariable_Check(o), why);
  return THPVariable_Unpack(o);
}
const at::Tensor* maybe_tensor(PyObject* o, const char* why) { return o == Py_None ? nullptr : &tensor(o, why); }
int64_t integer(PyObject* o) {
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw python_error();
  return x;
}
int32_t integer32(PyObject* o, const char* why) {
  const int64_t x = integer(o);
  need(x >= INT32_MIN && x <= INT32_MAX, why);
  return (int32_t)x;
}
void* address(PyObject* o) { return reinterpret_cast<void*>(static_cast<uintptr_t>(integer(o))); }

bool of_format(const at::Tensor& t, int64_t format) { return t.scalar_type() == (format == H2O_F32 ? at::kFloat : at::kBFloat16); }

// The stride between the tokens of [tokens, heads, dim] with dense heads, 0 where there is one token at most.
int64_t token_stride(const at::Tensor& t, const char* dense, const char* broadcast) {
  const auto n = t.sizes();
  const auto s = t.strides();
  need(n[0] == 0 || (s[2] == 1 && (n[1] <= 1 || s[1] == n[2])), dense);
  if (n[0] <= 1) return 0;
  need(s[0] != 0, broadcast);  // (0 means dense to the library)
  return s[0];
}

// positions: int64 [axes, tokens], or [tokens] for one axis; its address and the stride from axis to axis.
const int64_t* positions_of(const at::Tensor& p, int64_t axes, int64_t tokens, int64_t index, int64_t& stride) {
  need(p.scalar_type() == at::kLong && p.get_device() == index, "positions must be int64 on the rotary's device");
  const bool two = p.dim() == 2;
  need((two && p.size(0) == axes && p.size(1) == tokens) || (axes == 1 && p.dim() == 1 && p.size(0) == tokens), "positions must be [axes, tokens]");
  need(tokens <= 1 || p.stride(two ? 1 : 0) == 1, "positions must lie token after token");
  stride = axes > 1 ? p.stride(0) : 0;
  need(axes == 1 || tokens == 0 || stride >= tokens, "positions must not be broadcast over the axes");
  return static_cast<const int64_t*>(p.data_ptr());
}

h2o_sequences_t sequences_of(const at::Tensor& table, const at::Tensor& length, int32_t max_length, int64_t index, int64_t& batch) {
  need(length.scalar_type() == at::kInt && length.dim() == 1 && length.get_device() == index && length.is_contiguous(),
       "length must be a contiguous int32 [batch] on the pages' device");
  batch = length.size(0);
  need(table.scalar_type() == at::kInt && table.dim() == 2 && table.size(0) == batch && table.get_device() == index,
       "table must be int32 [batch, pages] on the pages' device");
  const int64_t pages = table.size(1), stride = table.stride(0);
  need((pages <= 1 || table.stride(1) == 1) && (batch <= 1 || pages == 0 || stride >= pages), "a sequence's entries of the table must be dense, and its own");
  need(pages <= INT32_MAX && batch <= INT32_MAX, "table is too large");
  return {static_cast<const int32_t*>(table.data_ptr()), static_cast<const int32_t*>(length.data_ptr()), batch > 1 ? stride : 0, (int32_t)pages, max_length};
}

const int32_t* cu_of(const at::Tensor* cu, int64_t batch, int64_t tokens, int64_t index) {
  if (!cu) {
    need(tokens >= batch, "without cu there is one token per sequence");
    return nullptr;
  }
  need(cu->scalar_type() == at::kInt && cu->dim() == 1 && cu->size(0) == batch + 1 && cu->get_device() == index && cu->is_contiguous(),
       "cu must be a contiguous int32 [batch + 1] on the pages' device");
  return static_cast<const int32_t*>(cu->data_ptr());
}

// q and what becomes of it: query heads per K/V head.
int32_t group_of(const at::Tensor& q, const at::Tensor& out, int64_t heads, int64_t dim, int64_t format, int64_t index) {
  need(q.dim() == 3 && q.size(2) == dim && q.size(1) >= heads && q.size(1) % heads == 0, "q must be [tokens, a multiple of the heads, head_dim]");
  need(of_format(q, format) && out.scalar_type() == q.scalar_type() && out.sizes() == q.sizes(), "q and its output must have the pages' dtype and one shape");
  need(q.get_device() == index && out.get_device() == index, "q and its output must be on the pages' device");
  need(q.size(1) <= INT32_MAX, "q has too many heads");
  return (int32_t)(q.size(1) / heads);
}

// Runs f, which returns an H2O code; a refusal becomes a ValueError.
template <typename F>
PyObject* guarded(const char* who, F f) {
  HANDLE_TH_ERRORS
  try {
    return PyLong_FromLong(f());
  } catch (const Refused& r) {
    return PyErr_Format(PyExc_ValueError, "%s: %s", who, r.why);
  }
  END_HANDLE_TH_ERRORS
}
bool count_is(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return false;
}
template <typename F>
int without_gil(F f) {
  pybind11::gil_scoped_release release;
  return f();
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count_is(n, 4)) return nullptr;
  return guarded("bind", [&] {
    rotate_fn = reinterpret_cast<decltype(rotate_fn)>(address(a[0]));
    append_fn = reinterpret_cast<decltype(append_fn)>(address(a[1]));
    scratch_fn = reinterpret_cast<decltype(scratch_fn)>(address(a[2]));
    attend_fn = reinterpret_cast<decltype(attend_fn)>(address(a[3]));
    return 0;
  });
}

// rotate(rotary, device, head_dim, axes, x, positions, out, inverse, stream)
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count_is(n, 9)) return nullptr;
  return guarded("H2ORotary", [&] {
    const int64_t index = integer(a[1]), dim = integer(a[2]);
    const at::Tensor &x = tensor(a[4], "x must be a tensor"), &out = tensor(a[6], "out must be a tensor");
    need(x.dim() == 3 && x.size(2) == dim && out.sizes() == x.sizes(), "x and out must be [tokens, heads, head_dim]");
    const auto type = x.scalar_type();
    need((type == at::kFloat || type == at::kBFloat16) && out.scalar_type() == type, "x and out must both be float32 or bfloat16");
    need(x.get_device() == index && out.get_device() == index, "x and out must be on the rotary's device");
    need(x.size(1) <= INT32_MAX, "x has too many heads");
    int64_t stride;
    const int64_t* at = positions_of(tensor(a[5], "positions must be a tensor"), integer(a[3]), x.size(0), index, stride);
    const int64_t xs = token_stride(x, "x must have dense heads", "x must not be broadcast over the tokens");
    const int64_t os = token_stride(out, "out must have dense heads", "out must not be broadcast over the tokens");
    const auto* rotary = static_cast<const h2o_rotary_t*>(address(a[0]));
    const int inverse = PyObject_IsTrue(a[7]);
    if (inverse < 0) throw python_error();
    void* stream = address(a[8]);
    return without_gil([&] {
      return rotate_fn(rotary, x.data_ptr(), out.data_ptr(), type == at::kFloat ? H2O_F32 : H2O_BF16, x.size(0), (int32_t)x.size(1), (int32_t)dim, xs, os, at,
                       stride, inverse, stream);
    });
  });
}

// append(handle, device, heads, head_dim, format, k, v, table, length, cu, rotary, rotary's device, head_dim and axes, positions, q,
// q_out, stream); rotary 0: none
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count_is(n, 18)) return nullptr;
  return guarded("H2OPages", [&] {
    const int64_t index = integer(a[1]), heads = integer(a[2]), dim = integer(a[3]), format = integer(a[4]);
    const at::Tensor &k = tensor(a[5], "k must be a tensor"), &v = tensor(a[6], "v must be a tensor");
    need(k.dim() == 3 && v.sizes() == k.sizes() && k.size(1) == heads && k.size(2) == dim, "k and v must be [tokens, heads, head_dim]");
    need(of_format(k, format) && of_format(v, format) && k.get_device() == index && v.get_device() == index,
         "k and v must have the pages' dtype and be on the pages' device");
    h2o_tokens_t t = {};
    t.n_tokens = k.size(0);
    t.kv_stride = token_stride(k, "k must have dense heads", "k must not be broadcast over the tokens");
    need(token_stride(v, "v must have dense heads", "v must not be broadcast over the tokens") == t.kv_stride, "k and v must have one token stride");
    int64_t batch;
    const h2o_sequences_t s =
        sequences_of(tensor(a[7], "table must be a tensor"), tensor(a[8], "length must be a tensor"), INT32_MAX, index, batch);
    t.k = k.data_ptr();
    t.v = v.data_ptr();
    t.cu = cu_of(maybe_tensor(a[9], "cu must be a tensor"), batch, t.n_tokens, index);
    t.batch = (int32_t)batch;
    t.query_group = 1;
    const auto* rotary = static_cast<const h2o_rotary_t*>(address(a[10]));
    const at::Tensor* positions = maybe_tensor(a[14], "positions must be a tensor");
    need(rotary || !positions, "positions belong to a rotary");
    if (rotary) {
      need(integer(a[11]) == index && integer(a[12]) == dim, "rotary must be for the pages' head_dim and device");
      if (positions) t.positions = positions_of(*positions, integer(a[13]), t.n_tokens, index, t.position_stride);
    }
    const at::Tensor *q = maybe_tensor(a[15], "q must be a tensor"), *q_out = maybe_tensor(a[16], "q_out must be a tensor");
    need(!q == !q_out, "q and q_out go together");
    if (q) {
      t.query_group = group_of(*q, *q_out, heads, dim, format, index);
      need(q->size(0) == t.n_tokens, "q must have as many tokens as k");
      t.q = q->data_ptr();
      t.q_out = q_out->data_ptr();
      t.q_stride = token_stride(*q, "q must have dense heads", "q must not be broadcast over the tokens");
      t.q_out_stride = token_stride(*q_out, "q_out must have dense heads", "q_out must not be broadcast over the tokens");
    }
    auto* pages = static_cast<h2o_pages_t*>(address(a[0]));
    void* stream = address(a[17]);
    return without_gil([&] { return append_fn(pages, &t, &s, rotary, stream); });
  });
}

// attend(handle, device, heads, head_dim, format, q, table, length, out, max_len, window, sinks, cu, max_q, lse, softmax_scale, stream)
// Scratch comes from torch's allocator on the current stream.
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count_is(n, 17)) return nullptr;
  return guarded("H2OPages", [&] {
    const int64_t index = integer(a[1]), heads = integer(a[2]), dim = integer(a[3]), format = integer(a[4]);
    const at::Tensor &q = tensor(a[5], "q must be a tensor"), &out = tensor(a[8], "out must be a tensor");
    h2o_queries_t t = {};
    t.query_group = group_of(q, out, heads, dim, format, index);
    t.q_rows = q.size(0);
    t.q_stride = token_stride(q, "q must have dense heads", "q must not be broadcast over the tokens");
    t.out_stride = token_stride(out, "out must have dense heads", "out must not be broadcast over the tokens");
    int64_t batch;
    const h2o_sequences_t s = sequences_of(tensor(a[6], "table must be a tensor"), tensor(a[7], "length must be a tensor"),
                                           integer32(a[9], "max_len is out of range"), index, batch);
    const at::Tensor *cu = maybe_tensor(a[12], "cu must be a tensor"), *lse = maybe_tensor(a[14], "lse must be a tensor");
    t.max_q = integer32(a[13], "max_q is out of range");
    need(cu || t.max_q == 1, "without cu there is one token per sequence");
    t.cu_q = cu_of(cu, batch, t.q_rows, index);
    if (lse) {
      need(lse->scalar_type() == at::kFloat && lse->dim() == 2 && lse->size(0) == t.q_rows && lse->size(1) == q.size(1) && lse->get_device() == index &&
               lse->is_contiguous(),
           "lse must be a contiguous float32 [tokens, query heads] on the pages' device");
      t.lse = static_cast<float*>(lse->data_ptr());
    }
    const double scale = PyFloat_AsDouble(a[15]);
    if (scale == -1.0 && PyErr_Occurred()) throw python_error();
    t.q = q.data_ptr();
    t.out = out.data_ptr();
    t.softmax_scale = (float)scale;
    t.dtype = (int32_t)format;
    t.batch = (int32_t)batch;
    auto* pages = static_cast<h2o_pages_t*>(address(a[0]));
    const int32_t window = integer32(a[10], "window is out of range"), sinks = integer32(a[11], "sinks is out of range");
    const size_t bytes = scratch_fn(pages, &t, &s, window, sinks);
    at::Tensor scratch;
    if (bytes) scratch = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));  // (torch's blocks are 512-byte aligned)
    void* stream = address(a[16]);
    return without_gil([&] { return attend_fn(pages, &t, &s, window, sinks, bytes ? scratch.data_ptr() : nullptr, bytes, stream); });
  });
}

#define H2O_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {H2O_METHOD(bind), H2O_METHOD(rotate), H2O_METHOD(append), H2O_METHOD(attend), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pages", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__pages() { return PyModule_Create(&module); }
