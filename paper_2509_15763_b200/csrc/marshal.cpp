// Argument marshalling of the Python binding: takes torch tensors, checks that they are contiguous CUDA tensors, and
// calls the C entry point of the same name (include/unigist.h).  Nothing is kept between calls.  Every tensor is read
// under the interpreter lock; what runs without it sees plain pointers and numbers.
// A generation loop makes two of these calls per token and is bound by them: through ctypes, with a Python-level
// check and a pointer object per tensor, a decode call took 14 us of host time against 6 this way.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include <string>
#include <vector>

#include "unigist.h"

namespace {

[[noreturn]] void raise(PyObject* type, const char* msg) {
  PyErr_SetString(type, msg);
  throw python_error();  // "a Python exception is set"
}

// A tensor argument as the C call takes it: its address (null for None), and what is needed of its sizes.
struct Arg {
  const at::Tensor* t;
  void* p;
  size_t bytes;
  operator void*() const { return p; }
  operator float*() const { return static_cast<float*>(p); }
  operator int32_t*() const { return static_cast<int32_t*>(p); }
};

// A problem's fields by name.  The names are made once, when the module is loaded (ten strings a call took 0.75 us).
enum { kBatch, kRawLen, kNumSinks, kRatio, kWindow, kNumQHeads, kNumKvHeads, kHeadDim, kSoftmaxScale, kFlags, kFields };
constexpr const char* kFieldName[kFields] = {"batch",        "raw_len",  "num_sinks",     "ratio", "window", "num_q_heads",
                                             "num_kv_heads", "head_dim", "softmax_scale", "flags"};
PyObject* g_field[kFields];

// The arguments of one call, read left to right (the caller holds a reference to each for the length of the call).
struct Args {
  PyObject* const* a;
  Py_ssize_t n, at = 0;

  PyObject* next() {
    if (at >= n) raise(PyExc_TypeError, "too few arguments");
    return a[at++];
  }
  const at::Tensor* contiguous() {  // null for None
    PyObject* o = next();
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, "expected a torch.Tensor");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) raise(PyExc_ValueError, "tensors must be contiguous CUDA tensors");
    return &t;
  }
  static Arg arg(const at::Tensor* t) {  // (data_ptr() throws for a tensor without storage: a transform's or a tracer's)
    return t ? Arg{t, t->data_ptr(), (size_t)t->numel() * t->element_size()} : Arg{nullptr, nullptr, 0};
  }
  Arg tensor() { return arg(contiguous()); }
  // The calls on chunks say what they take: on the current device, of an element type (a workspace of any).
  Arg tensor(at::ScalarType type, const char* name) {
    const at::Tensor* t = contiguous();
    if (t) check(*t, type, name);
    return arg(t);
  }
  Arg workspace() {
    const at::Tensor* t = contiguous();
    if (t) check_device(*t, "workspace");
    return arg(t);
  }
  // A [rows, heads, head_dim] tensor whose heads lie together; the rows may be any distance apart (part of a projection's output).
  Arg rows(const char* name, int64_t* stride) {
    PyObject* o = next();
    *stride = 0;
    if (o == Py_None) return {nullptr, nullptr, 0};
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, "expected a torch.Tensor");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.dim() != 3) raise(PyExc_ValueError, (std::string(name) + " must be a [rows, heads, head_dim] CUDA tensor").c_str());
    check(t, at::kBFloat16, name);
    const int64_t row = t.size(1) * t.size(2);
    if ((t.size(2) > 1 && t.stride(2) != 1) || (t.size(1) > 1 && t.stride(1) != t.size(2)))
      raise(PyExc_ValueError, (std::string("the heads of a row of ") + name + " must be contiguous").c_str());
    *stride = t.size(0) > 1 ? t.stride(0) : row;
    return {&t, t.data_ptr(), (size_t)t.numel() * 2};
  }
  static void check(const at::Tensor& t, at::ScalarType type, const char* name) {
    if (t.scalar_type() != type) raise(PyExc_ValueError, (std::string(name) + " must be " + c10::toString(type)).c_str());
    check_device(t, name);
  }
  static void check_device(const at::Tensor& t, const char* name) {
    if (t.device().index() != c10::cuda::current_device()) raise(PyExc_ValueError, (std::string(name) + " is not on the current device").c_str());
  }
  std::vector<uint8_t> byte_list(const char* what) {
    PyObject* seq = PySequence_Fast(next(), what);
    if (!seq) throw python_error();
    std::vector<uint8_t> v;
    for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(seq); ++i) {
      const long x = PyLong_AsLong(PySequence_Fast_GET_ITEM(seq, i));
      if ((x == -1 && PyErr_Occurred()) || x < 0 || x > 255) {
        Py_DECREF(seq);
        if (PyErr_Occurred()) throw python_error();
        raise(PyExc_ValueError, what);
      }
      v.push_back((uint8_t)x);
    }
    Py_DECREF(seq);
    return v;
  }
  long long integer() {
    const long long v = PyLong_AsLongLong(next());
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
  }
  double real() {
    const double v = PyFloat_AsDouble(next());
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
  }
  void* stream() {  // None: torch's current stream
    PyObject* o = next();
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    if (!h) throw python_error();
    void* p = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    if (!p && PyErr_Occurred()) throw python_error();
    return p;
  }
  unigist_problem problem() {
    PyObject* o = next();
    auto field = [&](int name) {
      PyObject* v = PyObject_GetAttr(o, g_field[name]);
      if (!v) throw python_error();
      if (!PyLong_CheckExact(v)) {
        PyObject* i = PyNumber_Index(v);  // whatever counts as an integer (numpy's too), as ctypes takes it; no float
        Py_DECREF(v);
        if (!i) throw python_error();
        v = i;
      }
      const unsigned long long x = PyLong_AsUnsignedLongLongMask(v);
      Py_DECREF(v);
      if (PyErr_Occurred()) throw python_error();
      return x;
    };
    unigist_problem p;
    p.batch = (int32_t)field(kBatch);
    p.raw_len = (int32_t)field(kRawLen);
    p.num_sinks = (int32_t)field(kNumSinks);
    p.ratio = (int32_t)field(kRatio);
    p.window = (int32_t)field(kWindow);
    p.num_q_heads = (int32_t)field(kNumQHeads);
    p.num_kv_heads = (int32_t)field(kNumKvHeads);
    p.head_dim = (int32_t)field(kHeadDim);
    PyObject* s = PyObject_GetAttr(o, g_field[kSoftmaxScale]);
    if (!s) throw python_error();
    p.softmax_scale = (float)PyFloat_AsDouble(s);
    Py_DECREF(s);
    if (PyErr_Occurred()) throw python_error();
    p.flags = (uint32_t)field(kFlags);
    return p;
  }
  std::vector<int32_t> int_list() {
    PyObject* seq = PySequence_Fast(next(), "expected a sequence of document lengths");
    if (!seq) throw python_error();
    std::vector<int32_t> v;
    for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(seq); ++i) {
      PyObject* x = PyNumber_Long(PySequence_Fast_GET_ITEM(seq, i));
      v.push_back(x ? (int32_t)PyLong_AsUnsignedLongLongMask(x) : 0);
      Py_XDECREF(x);
      if (PyErr_Occurred()) {
        Py_DECREF(seq);
        throw python_error();
      }
    }
    Py_DECREF(seq);
    return v;
  }
};

int32_t dim(const Arg& a, int64_t i) {
  if (!a.t) raise(PyExc_TypeError, "a tensor is missing");
  if (i >= a.t->dim()) raise(PyExc_IndexError, "a tensor has too few dimensions");
  return (int32_t)a.t->size(i);
}

// Runs a call with the interpreter lock released and hands its status back.
template <typename Fn>
int32_t unlocked(Fn fn) {
  struct Released {
    PyThreadState* state = PyEval_SaveThread();
    ~Released() { PyEval_RestoreThread(state); }  // also when the call throws (out of memory)
  } released;
  return fn();
}

// A METH_FASTCALL function around `body(Args&) -> status`.
template <int32_t (*kBody)(Args&)>
PyObject* call(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args args{a, n};
  return PyLong_FromLong(kBody(args));
  END_HANDLE_TH_ERRORS
}

template <decltype(unigist_gist_shift)* kFn>
int32_t shift(Args& a) {
  const unigist_problem p = a.problem();
  const Arg src = a.tensor(), dst = a.tensor();
  void* st = a.stream();
  const int32_t heads = dim(src, 2), eb = (int32_t)src.t->element_size();
  return unlocked([&] { return kFn(&p, src, dst, heads, eb, st); });
}

int32_t rope(Args& a) {
  const unigist_problem p = a.problem();
  const Arg src = a.tensor(), dst = a.tensor();
  const float base = (float)a.real();
  const uint32_t flags = (uint32_t)a.integer();
  void* st = a.stream();
  const int32_t heads = dim(src, 2);
  return unlocked([&] { return unigist_rope(&p, src, dst, heads, base, flags, st); });
}

int32_t attn_fwd(Args& a) {
  const unigist_problem p = a.problem();
  const Arg q = a.tensor(), k = a.tensor(), v = a.tensor(), o = a.tensor(), lse = a.tensor(), ws = a.tensor();
  void* st = a.stream();
  return unlocked([&] { return unigist_attn_fwd(&p, q, k, v, o, lse, ws, ws.bytes, st); });
}

int32_t attn_bwd(Args& a) {
  const unigist_problem p = a.problem();
  const Arg q = a.tensor(), k = a.tensor(), v = a.tensor(), o = a.tensor(), lse = a.tensor(), d_o = a.tensor(),
            dq = a.tensor(), dk = a.tensor(), dv = a.tensor(), ws = a.tensor();
  void* st = a.stream();
  return unlocked([&] { return unigist_attn_bwd(&p, q, k, v, o, lse, d_o, dq, dk, dv, ws, ws.bytes, st); });
}

int32_t attn_fwd_docs(Args& a) {
  const unigist_problem p = a.problem();
  const std::vector<int32_t> docs = a.int_list();
  const Arg q = a.tensor(), k = a.tensor(), v = a.tensor(), o = a.tensor(), lse = a.tensor(), ws = a.tensor();
  void* st = a.stream();
  return unlocked([&] {
    return unigist_attn_fwd_docs(&p, (int32_t)docs.size(), docs.data(), q, k, v, o, lse, ws, ws.bytes, st);
  });
}

int32_t attn_bwd_docs(Args& a) {
  const unigist_problem p = a.problem();
  const std::vector<int32_t> docs = a.int_list();
  const Arg q = a.tensor(), k = a.tensor(), v = a.tensor(), o = a.tensor(), lse = a.tensor(), d_o = a.tensor(),
            dq = a.tensor(), dk = a.tensor(), dv = a.tensor(), ws = a.tensor();
  void* st = a.stream();
  return unlocked([&] {
    return unigist_attn_bwd_docs(&p, (int32_t)docs.size(), docs.data(), q, k, v, o, lse, d_o, dq, dk, dv, ws,
                                 ws.bytes, st);
  });
}

int32_t kv_compact(Args& a) {
  const unigist_problem p = a.problem();
  const Arg k = a.tensor(), v = a.tensor(), kc = a.tensor(), vc = a.tensor(), table = a.tensor(), lens = a.tensor(),
            kept = a.tensor(), ws = a.tensor();
  void* st = a.stream();
  const int32_t blocks = dim(kc, 0), width = dim(table, 1);
  return unlocked([&] {
    return unigist_kv_compact(&p, k, v, kc, vc, blocks, table, width, lens, kept, ws, ws.bytes, st);
  });
}

int32_t prefill_chunk(Args& a) {
  const unigist_problem p = a.problem();
  const int32_t u0 = (int32_t)a.integer(), c = (int32_t)a.integer();
  const Arg q = a.tensor(), k = a.tensor(), v = a.tensor(), kc = a.tensor(), vc = a.tensor(), table = a.tensor(),
            lens = a.tensor(), o = a.tensor(), lse = a.tensor(), ws = a.tensor();
  void* st = a.stream();
  const int32_t blocks = dim(kc, 0), width = dim(table, 1);
  return unlocked([&] {
    return unigist_prefill_chunk(&p, u0, c, q, k, v, kc, vc, blocks, table, width, lens, o, lse, ws, ws.bytes, st);
  });
}

int32_t cache_state_init(Args& a) {
  const unigist_problem p = a.problem();
  const int32_t units = (int32_t)a.integer();
  const Arg state = a.tensor();
  void* st = a.stream();
  return unlocked([&] { return unigist_cache_state_init(&p, units, state, st); });
}

int32_t cache_append(Args& a) {
  const unigist_problem p = a.problem();
  const Arg k = a.tensor(), v = a.tensor();
  const int32_t is_gist = (int32_t)a.integer();
  const Arg kc = a.tensor(), vc = a.tensor(), table = a.tensor(), lens = a.tensor(), state = a.tensor();
  void* st = a.stream();
  const int32_t blocks = dim(kc, 0), width = dim(table, 1);
  return unlocked([&] {
    return unigist_cache_append(&p, k, v, is_gist, kc, vc, blocks, table, width, lens, state, st);
  });
}

int32_t decode_step(Args& a) {
  const unigist_problem p = a.problem();
  const Arg q = a.tensor(), kc = a.tensor(), vc = a.tensor(), table = a.tensor(), lens = a.tensor(),
            state = a.tensor(), o = a.tensor(), lse = a.tensor(), ws = a.tensor();
  void* st = a.stream();
  const int32_t blocks = dim(kc, 0), width = dim(table, 1);
  return unlocked([&] {
    return unigist_decode_step(&p, q, kc, vc, blocks, table, width, lens, state, o, lse, ws, ws.bytes, st);
  });
}

template <bool kStatic>
int32_t decode(Args& a) {
  const Arg q = a.tensor(), kc = a.tensor(), vc = a.tensor(), table = a.tensor(), lens = a.tensor(), o = a.tensor(),
            lse = a.tensor(), ws = kStatic ? Arg{} : a.tensor();
  const float scale = (float)a.real();
  void* st = a.stream();
  if (!q.t || q.t->dim() != 3) raise(PyExc_ValueError, "q must be [num_seqs, num_q_heads, head_dim]");
  const int32_t S = dim(q, 0), Hq = dim(q, 1), D = dim(q, 2), Hkv = dim(kc, 1), blocks = dim(kc, 0), width = dim(table, 1);
  return unlocked([&] {
    return kStatic
               ? unigist_decode_static(S, Hq, Hkv, D, scale, q, kc, vc, blocks, table, width, lens, o, lse, st)
               : unigist_decode(S, Hq, Hkv, D, scale, q, kc, vc, blocks, table, width, lens, o, lse, ws, ws.bytes, st);
  });
}

// What every call on chunks takes its sizes from; a tensor that does not fit them is an error here (the C call sees addresses).
void expect(bool fits, const char* what) {
  if (!fits) raise(PyExc_ValueError, what);
}
int64_t size_of(const Arg& a, int64_t i) { return a.t && i < a.t->dim() ? a.t->size(i) : -1; }
void expect_cache(const Arg& c, int32_t Hkv, int32_t D, int32_t blocks, const char* what) {
  expect(c.t && c.t->dim() == 4 && size_of(c, 0) == blocks && size_of(c, 1) == Hkv && size_of(c, 2) == UNIGIST_PAGE_TOKENS && size_of(c, 3) == D, what);
}
void expect_weights(const Arg& w, const Arg& kc, const char* what) {
  expect(!w.t || (w.t->dim() == 3 && size_of(w, 0) == size_of(kc, 0) && size_of(w, 1) == size_of(kc, 1) && size_of(w, 2) == UNIGIST_PAGE_TOKENS), what);
}
struct Batch {  // cu_rows, block_table, seq_lens
  Arg cu, table, lens;
  int32_t seqs, width;
  void expect_fits() {
    expect(table.t && table.t->dim() == 2, "block_table must be [num_seqs, max_blocks_per_seq]");
    seqs = dim(table, 0), width = dim(table, 1);
    expect(lens.t && (size_t)seqs * 4 == lens.bytes, "seq_lens must be [num_seqs]");
    expect(!cu.t || (size_t)(seqs + 1) * 4 == cu.bytes, "cu_rows must be [num_seqs + 1]");
  }
};
// Positions [axes, rows] and the axis of every pair, or None for both.
struct Rotation {
  Arg pos;
  std::vector<uint8_t> freq_axis;
  int32_t axes;
  void expect_fits(int64_t rows, int64_t head_dim) {
    expect(pos.t && pos.t->dim() == 2 && size_of(pos, 1) == rows, "pos_ids must be [num_axes, rows]");
    expect((int64_t)freq_axis.size() == head_dim / 2, "freq_axis must name an axis for each of the head_dim / 2 pairs");
    axes = dim(pos, 0);
  }
};

int32_t rope_axes(Args& a) {
  int64_t ss, ds;
  const Arg src = a.rows("src", &ss), dst = a.rows("dst", &ds);
  Rotation r{a.tensor(at::kInt, "pos_ids"), a.byte_list("freq_axis must be a sequence of small numbers"), 0};
  const float theta = (float)a.real();
  const uint32_t flags = (uint32_t)a.integer();
  void* st = a.stream();
  expect(src.t && dst.t && src.t->sizes() == dst.t->sizes(), "src and dst must have the same shape");
  r.expect_fits(src.t->size(0), src.t->size(2));
  const int32_t n = dim(src, 0), heads = dim(src, 1), D = dim(src, 2);
  return unlocked([&] { return unigist_rope_axes(n, heads, D, src, ss, dst, ds, r.pos, r.axes, r.freq_axis.data(), theta, flags, st); });
}

int32_t chunk_append(Args& a) {
  int64_t ks, vs;
  const Arg k = a.rows("k_new", &ks), v = a.rows("v_new", &vs);
  Batch b;
  b.cu = a.tensor(at::kInt, "cu_rows");
  const Arg kc = a.tensor(at::kBFloat16, "k_cache"), vc = a.tensor(at::kBFloat16, "v_cache");
  b.table = a.tensor(at::kInt, "block_table");
  b.lens = a.tensor(at::kInt, "seq_lens");
  const Arg new_lens = a.tensor(at::kInt, "new_lens"), w = a.tensor(at::kFloat, "weights");
  Rotation r{a.tensor(at::kInt, "pos_ids"), {}, 0};
  if (r.pos.t)
    r.freq_axis = a.byte_list("freq_axis must be a sequence of small numbers");
  else
    a.next();
  const float theta = (float)a.real();
  void* st = a.stream();
  b.expect_fits();
  expect(k.t && v.t && k.t->sizes() == v.t->sizes(), "k_new and v_new must have the same shape");
  const int32_t n = dim(k, 0), Hkv = dim(k, 1), D = dim(k, 2), blocks = dim(kc, 0);
  expect_cache(kc, Hkv, D, blocks, "k_cache must be [num_blocks, heads of k_new, 64, head_dim]");
  expect_cache(vc, Hkv, D, blocks, "v_cache must have the shape of k_cache");
  expect_weights(w, kc, "weights must be [num_blocks, num_kv_heads, 64]");
  expect(b.cu.t, "cu_rows is missing");
  expect(new_lens.t && new_lens.bytes == b.lens.bytes, "new_lens must be [num_seqs]");
  if (r.pos.t) r.expect_fits(n, D);
  return unlocked([&] {
    return unigist_chunk_append(b.seqs, Hkv, D, n, k, ks, v, vs, b.cu, r.pos, r.axes, r.freq_axis.data(), theta, kc, vc, w, blocks, b.table,
                                b.width, b.lens, new_lens, st);
  });
}

int32_t chunk_attn(Args& a) {
  int64_t qs;
  const Arg q = a.rows("q", &qs);
  Batch b;
  b.cu = a.tensor(at::kInt, "cu_rows");
  const Arg kc = a.tensor(at::kBFloat16, "k_cache"), vc = a.tensor(at::kBFloat16, "v_cache");
  b.table = a.tensor(at::kInt, "block_table");
  b.lens = a.tensor(at::kInt, "seq_lens");
  const Arg o = a.tensor(at::kBFloat16, "o"), lse = a.tensor(at::kFloat, "lse"), ws = a.workspace();
  const float scale = (float)a.real();
  void* st = a.stream();
  b.expect_fits();
  expect(q.t && o.t && q.t->sizes() == o.t->sizes(), "q and o must have the same shape");
  const int32_t n = dim(q, 0), Hq = dim(q, 1), D = dim(q, 2), blocks = dim(kc, 0), Hkv = dim(kc, 1);
  expect_cache(kc, Hkv, D, blocks, "k_cache must be [num_blocks, num_kv_heads, 64, head_dim of q]");
  expect_cache(vc, Hkv, D, blocks, "v_cache must have the shape of k_cache");
  expect(b.cu.t, "cu_rows is missing");
  expect(!lse.t || (lse.t->dim() == 2 && size_of(lse, 0) == n && size_of(lse, 1) == Hq), "lse must be [rows, num_q_heads]");
  return unlocked([&] {
    return unigist_chunk_attn(b.seqs, Hq, Hkv, D, scale, n, q, qs, b.cu, kc, vc, blocks, b.table, b.width, b.lens, o, lse, ws, ws.bytes, st);
  });
}

int32_t cache_weigh(Args& a) {
  int64_t qs;
  const Arg q = a.rows("q", &qs);
  Batch b;
  b.cu = a.tensor(at::kInt, "cu_rows");
  const Arg lse = a.tensor(at::kFloat, "lse"), kc = a.tensor(at::kBFloat16, "k_cache");
  b.table = a.tensor(at::kInt, "block_table");
  b.lens = a.tensor(at::kInt, "seq_lens");
  const Arg w_in = a.tensor(at::kFloat, "weights_in"), w_out = a.tensor(at::kFloat, "weights_out");
  const float decay = (float)a.real(), scale = (float)a.real();
  void* st = a.stream();
  b.expect_fits();
  expect(q.t && b.cu.t && w_out.t, "a tensor is missing");
  const int32_t n = dim(q, 0), Hq = dim(q, 1), D = dim(q, 2), blocks = dim(kc, 0), Hkv = dim(kc, 1);
  expect_cache(kc, Hkv, D, blocks, "k_cache must be [num_blocks, num_kv_heads, 64, head_dim of q]");
  expect(lse.t && lse.t->dim() == 2 && size_of(lse, 0) == n && size_of(lse, 1) == Hq, "lse must be [rows, num_q_heads]");
  expect_weights(w_in, kc, "weights_in must be [num_blocks, num_kv_heads, 64]");
  expect_weights(w_out, kc, "weights_out must be [num_blocks, num_kv_heads, 64]");
  return unlocked([&] {
    return unigist_cache_weigh(b.seqs, Hq, Hkv, D, scale, n, q, qs, b.cu, lse, kc, blocks, b.table, b.width, b.lens, w_in, decay, w_out, st);
  });
}

int32_t cache_evict(Args& a) {
  const Arg kc = a.tensor(at::kBFloat16, "k_cache"), vc = a.tensor(at::kBFloat16, "v_cache"), w = a.tensor(at::kFloat, "weights");
  Batch b;
  b.cu = {nullptr, nullptr, 0};
  b.table = a.tensor(at::kInt, "block_table");
  b.lens = a.tensor(at::kInt, "seq_lens");
  const Arg to = a.tensor(at::kInt, "new_table"), new_lens = a.tensor(at::kInt, "new_lens"), kept = a.tensor(at::kInt, "kept_idx");
  const int32_t keep = (int32_t)a.integer(), first = (int32_t)a.integer(), last = (int32_t)a.integer();
  void* st = a.stream();
  b.expect_fits();
  const int32_t blocks = dim(kc, 0), Hkv = dim(kc, 1), D = dim(kc, 3);
  expect_cache(kc, Hkv, D, blocks, "k_cache must be [num_blocks, num_kv_heads, 64, head_dim]");
  expect_cache(vc, Hkv, D, blocks, "v_cache must have the shape of k_cache");
  expect(w.t, "weights is missing");
  expect_weights(w, kc, "weights must be [num_blocks, num_kv_heads, 64]");
  expect(to.t && to.t->dim() == 2 && size_of(to, 0) == b.seqs, "new_table must be [num_seqs, new_max_blocks_per_seq]");
  expect(new_lens.t && new_lens.bytes == b.lens.bytes, "new_lens must be [num_seqs]");
  expect(kept.t && kept.t->dim() == 3 && size_of(kept, 0) == b.seqs && size_of(kept, 1) == Hkv && size_of(kept, 2) == keep,
         "kept_idx must be [num_seqs, num_kv_heads, keep]");
  const int32_t to_width = dim(to, 1);
  return unlocked([&] {
    return unigist_cache_evict(b.seqs, Hkv, D, keep, first, last, kc, vc, w, blocks, b.table, b.width, b.lens, to, to_width, new_lens, kept, st);
  });
}

#define FN(name, ...) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<__VA_ARGS__>)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {FN("gist_shift", shift<unigist_gist_shift>),
                          FN("gist_unshift", shift<unigist_gist_unshift>),
                          FN("rope", rope),
                          FN("attn_fwd", attn_fwd),
                          FN("attn_bwd", attn_bwd),
                          FN("attn_fwd_docs", attn_fwd_docs),
                          FN("attn_bwd_docs", attn_bwd_docs),
                          FN("kv_compact", kv_compact),
                          FN("prefill_chunk", prefill_chunk),
                          FN("cache_state_init", cache_state_init),
                          FN("cache_append", cache_append),
                          FN("decode_step", decode_step),
                          FN("decode", decode<false>),
                          FN("decode_static", decode<true>),
                          FN("rope_axes", rope_axes),
                          FN("chunk_append", chunk_append),
                          FN("chunk_attn", chunk_attn),
                          FN("cache_weigh", cache_weigh),
                          FN("cache_evict", cache_evict),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
  for (int i = 0; i < kFields; ++i)
    if (!g_field[i] && !(g_field[i] = PyUnicode_InternFromString(kFieldName[i]))) return nullptr;
  return PyModule_Create(&kModule);
}
