// Argument marshalling of the linear-layer, row-quantisation and cache entry points, for the calls
// whose own time is a few microseconds: tensors are looked at and outputs allocated here instead of
// attribute by attribute from Python (11 us of a 7 us single-token linear layer were spent there,
// 4 of them in the library).  No arithmetic, no CUDA: the C entry points are called by address.
//
// Every function returns its result, or the negative GEMM_ERR_* code of the entry point as an int.
#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/b200kv.h"

namespace {

struct Refused {
  PyObject* type;
  std::string text;
};

struct Raised {};  // a Python error is set already

struct Entries {
  decltype(&gemm_fp16_linear) fp16_linear;
  decltype(&gemm_s8_linear) s8_linear;
  decltype(&gemm_s4_linear) s4_linear;
  decltype(&gemm_quantize_rows) quantize_rows;
  decltype(&kv_append_s8_rows) kv_append;
  decltype(&kv_read_s8_rows) kv_read;
  decltype(&kv_attention_s8_rows) kv_attention;
} g_entry = {};

// The current device, asked for once a call (with the first CUDA tensor).  Per thread: kv_read lets other threads run
// while it waits for a count.
thread_local int g_device = -1;
int device() {
  if (g_device < 0) g_device = c10::cuda::current_device();
  return g_device;
}

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) throw Refused{PyExc_TypeError, std::string(what) + " must be a CUDA tensor"};
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) throw Refused{PyExc_TypeError, std::string(what) + " must be a CUDA tensor"};
  if (t.get_device() != device())
    throw Refused{PyExc_ValueError, std::string(what) + " is not on the current CUDA device"};
  return t;
}

const at::Tensor& typed(PyObject* o, at::ScalarType type, const char* what) {
  const at::Tensor& t = tensor(o, what);
  if (t.scalar_type() != type)
    throw Refused{PyExc_TypeError, std::string(what) + " must have dtype " + c10::toString(type) + ", got " +
                                       c10::toString(t.scalar_type())};
  return t;
}

void* dense(PyObject* o, at::ScalarType type, const char* what) {
  const at::Tensor& t = typed(o, type, what);
  if (!t.is_contiguous()) throw Refused{PyExc_ValueError, std::string(what) + " must be contiguous"};
  return t.data_ptr();
}

int narrow(int64_t v, const char* what) {
  if (v < -0x7fffffffll || v > 0x7fffffffll) throw Refused{PyExc_ValueError, std::string(what) + " does not fit 32 bits"};
  return static_cast<int>(v);
}

// Python numbers.  What is no integer (or number) raises Python's own TypeError.
int integer(PyObject* o, const char* what) {
  int overflow = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
  if (v == -1 && !overflow && PyErr_Occurred()) throw Raised{};
  return narrow(overflow ? INT64_MAX : v, what);
}
float number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return static_cast<float>(v);
}

// A matrix whose rows are contiguous: pointer and row pitch.
void* rows_of(const at::Tensor& t, int64_t rows, int64_t cols, const char* what, long long* pitch) {
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols)
    throw Refused{PyExc_ValueError, std::string(what) + " must have shape (" + std::to_string(rows) + ", " +
                                        std::to_string(cols) + ")"};
  if (cols > 1 && t.stride(1) != 1) throw Refused{PyExc_ValueError, std::string(what) + " must have contiguous rows"};
  // (a pitch of 0, a broadcast row, would read as "dense" in the entry points)
  if (rows > 1 && t.stride(0) < cols) throw Refused{PyExc_ValueError, std::string(what) + " must have rows that do not overlap"};
  *pitch = rows > 1 ? t.stride(0) : cols;
  return t.data_ptr();
}

// The stream to launch on: None = the current one.
struct Launch {
  gemm_stream_t handle;
  bool foreign;
};
Launch stream_of(PyObject* o) {
  const cudaStream_t current = c10::cuda::getCurrentCUDAStream().stream();
  if (o == Py_None) return {reinterpret_cast<gemm_stream_t>(current), false};
  const auto s = reinterpret_cast<cudaStream_t>(PyLong_AsVoidPtr(o));
  return {reinterpret_cast<gemm_stream_t>(s), s != current};
}

c10::cuda::CUDAStream torch_stream(const Launch& s) {
  return c10::cuda::getStreamFromExternal(reinterpret_cast<cudaStream_t>(s.handle), device());
}

// An output of our own: if the work runs on another stream than the current one, the allocator must
// not hand its memory on before that stream is done with it.
at::Tensor new_out(at::IntArrayRef shape, at::ScalarType type, const Launch& s) {
  at::Tensor t = at::empty(shape, at::TensorOptions().dtype(type).device(at::kCUDA, device()));
  if (s.foreign) t.record_stream(torch_stream(s).unwrap());
  return t;
}

// Runs f with C++ exceptions turned into Python ones.
template <class F>
PyObject* guarded(F&& f) {
  try {
    g_device = -1;
    return f();
  } catch (const Raised&) {
  } catch (const Refused& r) {
    PyErr_SetString(r.type, r.text.c_str());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

PyObject* code(int rc) { return PyLong_FromLong(rc); }

bool arity(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return false;
}

// linear(precision, A, B, row_scale, col_scale, bias, activation, residual, C, half, stream)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 11)) return nullptr;
  return guarded([&]() -> PyObject* {
    const int precision = integer(a[0], "precision");
    const at::ScalarType in = precision == GEMM_PREC_FP16 ? at::kHalf : precision == GEMM_PREC_S8 ? at::kChar : at::kByte;
    const at::Tensor &A = typed(a[1], in, "A"), &B = typed(a[2], in, "B");
    if (A.dim() != 2 || B.dim() != 2 || A.size(1) != B.size(1))
      throw Refused{PyExc_ValueError, "A and B disagree on K"};
    const int M = narrow(A.size(0), "M"), N = narrow(B.size(0), "N");
    const int K = narrow(A.size(1) * (precision == GEMM_PREC_S4 ? 2 : 1), "K");
    gemm_epilogue_t e = {};
    e.activation = integer(a[6], "activation");
    const Launch s = stream_of(a[10]);
    at::ScalarType out = PyObject_IsTrue(a[9]) ? at::kHalf : at::kFloat;
    at::Tensor C;
    if (a[8] != Py_None) {
      C = tensor(a[8], "C");
      out = C.scalar_type();
      if (out != at::kHalf && out != at::kFloat) throw Refused{PyExc_TypeError, "the result is float32 or float16"};
    }
    e.c_is_fp16 = out == at::kHalf;
    void* const pa = dense(a[1], in, "A");
    void* const pb = dense(a[2], in, "B");
    if (a[5] != Py_None) {
      e.bias = static_cast<const float*>(dense(a[5], at::kFloat, "bias"));
      if (THPVariable_Unpack(a[5]).numel() != N) throw Refused{PyExc_ValueError, "bias needs N entries"};
    }
    if (a[7] != Py_None) e.residual = rows_of(typed(a[7], out, "residual"), M, N, "residual", &e.ldr);
    const float *rs = nullptr, *cs = nullptr;
    if (precision != GEMM_PREC_FP16) {
      rs = static_cast<const float*>(dense(a[3], at::kFloat, "row_scale"));
      cs = static_cast<const float*>(dense(a[4], at::kFloat, "col_scale"));
      if (THPVariable_Unpack(a[3]).numel() != M || THPVariable_Unpack(a[4]).numel() != N)
        throw Refused{PyExc_ValueError, "row_scale needs M entries, col_scale N"};
    }
    if (!C.defined()) C = new_out({M, N}, out, s);
    void* const pc = rows_of(C, M, N, "C", &e.ldc);
    int rc;
    if (precision == GEMM_PREC_FP16)
      rc = g_entry.fp16_linear(M, N, K, pa, pb, pc, &e, s.handle);
    else if (precision == GEMM_PREC_S8)
      rc = g_entry.s8_linear(M, N, K, static_cast<const int8_t*>(pa), static_cast<const int8_t*>(pb), rs, cs, pc, &e, s.handle);
    else
      rc = g_entry.s4_linear(M, N, K, static_cast<const uint8_t*>(pa), static_cast<const uint8_t*>(pb), rs, cs, pc, &e, s.handle);
    return rc ? code(rc) : THPVariable_Wrap(C);
  });
}

// quantize_rows(precision, X, Q, row_scale, stream)
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 5)) return nullptr;
  return guarded([&]() -> PyObject* {
    const int precision = integer(a[0], "precision");
    const at::Tensor& X = tensor(a[1], "X");
    if (X.dim() != 2 || (X.scalar_type() != at::kHalf && X.scalar_type() != at::kFloat))
      throw Refused{PyExc_TypeError, "X must be a float16 or float32 matrix"};
    const int64_t rows = X.size(0), K = X.size(1), width = precision == GEMM_PREC_S4 ? K / 2 : K;
    const at::ScalarType type = precision == GEMM_PREC_S4 ? at::kByte : at::kChar;
    long long ldx;
    void* const px = rows_of(X, rows, K, "X", &ldx);
    const Launch s = stream_of(a[4]);
    at::Tensor Q, scale;
    if (a[2] != Py_None) {
      dense(a[2], type, "Q");
      Q = THPVariable_Unpack(a[2]);
      if (Q.dim() != 2 || Q.size(0) != rows || Q.size(1) != width)
        throw Refused{PyExc_ValueError, "Q must have shape (" + std::to_string(rows) + ", " + std::to_string(width) + ")"};
    } else {
      Q = new_out({rows, width}, type, s);
    }
    if (a[3] != Py_None) {
      dense(a[3], at::kFloat, "row_scale");
      scale = THPVariable_Unpack(a[3]);
      if (scale.numel() != rows) throw Refused{PyExc_ValueError, "row_scale needs one entry per row"};
    } else {
      scale = new_out({rows}, at::kFloat, s);
    }
    const int rc = g_entry.quantize_rows(precision, narrow(rows, "rows"), narrow(K, "K"), px, ldx, X.scalar_type() == at::kHalf,
                                         Q.data_ptr(), static_cast<float*>(scale.data_ptr()), s.handle);
    if (rc) return code(rc);
    PyObject* const q = THPVariable_Wrap(Q);
    PyObject* const sc = THPVariable_Wrap(scale);
    PyObject* const both = PyTuple_Pack(2, q, sc);
    Py_XDECREF(q);
    Py_XDECREF(sc);
    return both;
  });
}

kv_cache_s8_t cache_of(PyObject* o) {
  if (!PyTuple_Check(o) && !PyList_Check(o))
    throw Refused{PyExc_TypeError, "cache is (k, v, k_scale, v_scale)"};
  if (PySequence_Fast_GET_SIZE(o) != 4) throw Refused{PyExc_ValueError, "cache is (k, v, k_scale, v_scale)"};
  PyObject** const i = PySequence_Fast_ITEMS(o);
  kv_cache_s8_t c = {};
  c.k = static_cast<int8_t*>(dense(i[0], at::kChar, "k"));
  c.v = static_cast<int8_t*>(dense(i[1], at::kChar, "v"));
  c.k_scale = static_cast<float*>(dense(i[2], at::kFloat, "k_scale"));
  c.v_scale = static_cast<float*>(dense(i[3], at::kFloat, "v_scale"));
  const auto shape = THPVariable_Unpack(i[0]).sizes();
  const auto ks = THPVariable_Unpack(i[2]).sizes();
  if (shape.size() != 4 || THPVariable_Unpack(i[1]).sizes() != shape || ks != shape.slice(0, 2) ||
      THPVariable_Unpack(i[3]).sizes() != ks)
    throw Refused{PyExc_ValueError, "cache is (k, v, k_scale, v_scale): two (pages, heads, page, dim), two (pages, heads)"};
  c.num_pages = narrow(shape[0], "pages");
  c.kv_heads = narrow(shape[1], "heads");
  c.page_size = narrow(shape[2], "page");
  c.head_dim = narrow(shape[3], "dim");
  return c;
}

struct Batch {
  int batch, width;
  const int *cu, *start, *table;
};
Batch batch_of(PyObject* cu, PyObject* start, PyObject* table, const char* what) {
  Batch b;
  b.cu = static_cast<const int*>(dense(cu, at::kInt, "cu"));
  b.start = static_cast<const int*>(dense(start, at::kInt, what));
  b.table = static_cast<const int*>(dense(table, at::kInt, "block_table"));
  const at::Tensor& t = THPVariable_Unpack(table);
  b.batch = narrow(THPVariable_Unpack(start).numel(), "batch");
  if (THPVariable_Unpack(cu).numel() != b.batch + 1ll)
    throw Refused{PyExc_ValueError, std::string("cu needs one entry more than ") + what};
  if (t.dim() != 2 || t.size(0) != b.batch) throw Refused{PyExc_ValueError, "block_table needs one row per sequence"};
  b.width = narrow(t.size(1), "block_table");
  return b;
}

struct Rows {
  void* ptr;
  int64_t tokens, heads;
  long long token, head;  // strides
};
Rows heads_of(const at::Tensor& t, int heads, int dim, const char* what) {
  if (t.dim() != 3 || t.size(2) != dim || (heads && t.size(1) != heads) || t.stride(2) != 1)
    throw Refused{PyExc_ValueError, std::string(what) + " must be (tokens, heads, " + std::to_string(dim) + ") with contiguous heads"};
  Rows r;
  r.ptr = t.data_ptr();
  r.tokens = t.size(0);
  r.heads = t.size(1);
  r.head = r.heads > 1 ? t.stride(1) : dim;
  r.token = r.tokens > 1 ? t.stride(0) : r.heads * dim;
  return r;
}

// kv_append(cache, k, v, cu, past, table, max_new, stream)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 8)) return nullptr;
  return guarded([&]() -> PyObject* {
    const kv_cache_s8_t c = cache_of(a[0]);
    const Rows k = heads_of(typed(a[1], at::kHalf, "k"), c.kv_heads, c.head_dim, "k");
    const Rows v = heads_of(typed(a[2], at::kHalf, "v"), c.kv_heads, c.head_dim, "v");
    if (k.tokens != v.tokens || k.token != v.token || k.head != v.head)
      throw Refused{PyExc_ValueError, "k and v must have the same shape and strides"};
    const Batch b = batch_of(a[3], a[4], a[5], "past");
    const int max_new = integer(a[6], "max_new");
    if (k.tokens == 0) Py_RETURN_NONE;
    const int rc = g_entry.kv_append(&c, b.batch, b.cu, b.start, b.table, b.width, max_new,
                                     k.ptr, v.ptr, k.token, k.head, narrow(k.tokens, "tokens"), stream_of(a[7]).handle);
    if (rc) return code(rc);
    Py_RETURN_NONE;
  });
}

// kv_read(cache, cu, first, table, max_read, tokens, out, stream)
PyObject* kv_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 8)) return nullptr;
  return guarded([&]() -> PyObject* {
    const kv_cache_s8_t c = cache_of(a[0]);
    const Batch b = batch_of(a[1], a[2], a[3], "first");
    const int max_read = integer(a[4], "max_read");
    const Launch s = stream_of(a[7]);
    at::Tensor out[2];
    if (a[6] != Py_None) {
      if (!PyTuple_Check(a[6]) || PyTuple_GET_SIZE(a[6]) != 2) throw Refused{PyExc_TypeError, "out is a tuple of two tensors"};
      for (int i = 0; i < 2; ++i) {
        dense(PyTuple_GET_ITEM(a[6], i), at::kHalf, i ? "v" : "k");
        out[i] = THPVariable_Unpack(PyTuple_GET_ITEM(a[6], i));
        if (out[i].dim() != 3 || out[i].size(1) != c.kv_heads || out[i].size(2) != c.head_dim || out[i].sizes() != out[0].sizes())
          throw Refused{PyExc_ValueError, "outputs are two (tokens, kv_heads, head_dim)"};
      }
    } else {
      int64_t tokens;
      if (a[5] == Py_None) {  // cu[-1], in the order of the stream, which is waited for
        c10::cuda::OptionalCUDAStreamGuard on;
        if (s.foreign) on.reset_stream(torch_stream(s));
        tokens = THPVariable_Unpack(a[1]).reshape(-1).select(0, b.batch).item<int>();
      } else {
        tokens = integer(a[5], "tokens");
      }
      if (tokens < 0) throw Refused{PyExc_ValueError, "tokens must not be negative"};
      for (auto& t : out) t = new_out({tokens, c.kv_heads, c.head_dim}, at::kHalf, s);
    }
    if (out[0].size(0) > 0) {
      const int rc = g_entry.kv_read(&c, b.batch, b.cu, b.start, b.table, b.width, max_read,
                                     out[0].data_ptr(), out[1].data_ptr(), narrow(out[0].size(0), "tokens"), s.handle);
      if (rc) return code(rc);
    }
    PyObject* const k = THPVariable_Wrap(out[0]);
    PyObject* const v = THPVariable_Wrap(out[1]);
    PyObject* const both = PyTuple_Pack(2, k, v);
    Py_XDECREF(k);
    Py_XDECREF(v);
    return both;
  });
}

// kv_attention(q, cache, cu, kv_len, table, max_q, softmax_scale, window, out, stream)
PyObject* kv_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 10)) return nullptr;
  return guarded([&]() -> PyObject* {
    const kv_cache_s8_t c = cache_of(a[1]);
    const at::Tensor& qt = typed(a[0], at::kHalf, "q");
    const Rows q = heads_of(qt, 0, c.head_dim, "q");
    const Batch b = batch_of(a[2], a[3], a[4], "kv_len");
    const int max_q = integer(a[5], "max_q"), window = integer(a[7], "window");
    const float scale = number(a[6]);
    const Launch s = stream_of(a[9]);
    at::Tensor out;
    if (a[8] != Py_None) {
      out = typed(a[8], at::kHalf, "out");
      if (out.sizes() != qt.sizes()) throw Refused{PyExc_ValueError, "out must have the shape of q"};
    } else {
      out = new_out(qt.sizes(), at::kHalf, s);
    }
    const Rows o = heads_of(out, 0, c.head_dim, "out");
    if (o.head != c.head_dim) throw Refused{PyExc_ValueError, "the heads of a row of out must be contiguous"};
    if (q.tokens > 0) {
      const int rc = g_entry.kv_attention(&c, b.batch, b.cu, b.start, b.table, b.width, max_q, narrow(q.heads, "heads"), q.ptr,
                                          q.token, q.head, scale, window, out.data_ptr(), o.token,
                                          narrow(q.tokens, "tokens"), s.handle);
      if (rc) return code(rc);
    }
    return THPVariable_Wrap(out);
  });
}

// entries(address, ...): in the order of the struct above
PyObject* entries(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 7)) return nullptr;
  void* p[7];
  for (int i = 0; i < 7; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an entry point is missing");
      return nullptr;
    }
  }
  g_entry.fp16_linear = reinterpret_cast<decltype(g_entry.fp16_linear)>(p[0]);
  g_entry.s8_linear = reinterpret_cast<decltype(g_entry.s8_linear)>(p[1]);
  g_entry.s4_linear = reinterpret_cast<decltype(g_entry.s4_linear)>(p[2]);
  g_entry.quantize_rows = reinterpret_cast<decltype(g_entry.quantize_rows)>(p[3]);
  g_entry.kv_append = reinterpret_cast<decltype(g_entry.kv_append)>(p[4]);
  g_entry.kv_read = reinterpret_cast<decltype(g_entry.kv_read)>(p[5]);
  g_entry.kv_attention = reinterpret_cast<decltype(g_entry.kv_attention)>(p[6]);
  Py_RETURN_NONE;
}

#define METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(entries),   METHOD(linear),  METHOD(quantize_rows), METHOD(kv_append),
                         METHOD(kv_read),   METHOD(kv_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
