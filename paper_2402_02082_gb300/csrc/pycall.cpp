// Argument marshalling of the Python binding in C++: tensors to pointers and sizes, then the C call.
//
// What bounds it: a call's launches cost 2-4 us of host time, and marshalling the same arguments in
// Python (shape tuples, a ctypes structure, the current stream) cost another 9 us, more than most
// of the kernels take.  With it here a whole cross-attention call costs 2.3 us (11.3 before) and a
// verification call of two launches 3.8 us (13.6).
//
// Each function takes the arguments of binding.py's function of the same name by position and
// returns the C function's status, or -1 for a call that it does not take.  It takes plain CUDA
// tensors of the documented shapes and types, plain int and float values, and a stream that is
// None, an int or a torch.cuda.Stream; everything else, and everything wrong, goes to the Python
// code, which accepts or refuses it.  Nothing is kept from one call to the next.
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cstdint>

#include "glide.h"

namespace {

PyObject* g_stream_type = nullptr;  // torch.cuda.Stream

struct NotTaken {};

// One call's arguments, read from left to right; the first unusual one throws NotTaken.
class Args {
 public:
  Args(PyObject* const* v, Py_ssize_t n, Py_ssize_t want) : v_(v) {
    if (n != want) throw NotTaken{};
  }

  const at::Tensor& tensor(at::ScalarType type) {
    const at::Tensor& t = any_tensor();
    if (t.scalar_type() != type) throw NotTaken{};
    return t;
  }
  // contiguous, of this shape
  const at::Tensor& tensor(at::ScalarType type, std::initializer_list<int64_t> shape) {
    const at::Tensor& t = tensor(type);
    if (t.sizes() != at::IntArrayRef(shape) || !t.is_contiguous()) throw NotTaken{};
    return t;
  }
  // a cache or the queries: bf16 or fp32, contiguous, no size beyond 32 bits
  const at::Tensor& data() {
    const at::Tensor& t = any_tensor();
    if ((t.scalar_type() != at::kBFloat16 && t.scalar_type() != at::kFloat) || !t.is_contiguous()) throw NotTaken{};
    for (int64_t s : t.sizes())
      if (s > INT_MAX) throw NotTaken{};
    return t;
  }
  // an 8-bit cache's codes, contiguous, no size beyond 32 bits
  const at::Tensor& codes() {
    const at::Tensor& t = any_tensor();
    if ((t.scalar_type() != at::kFloat8_e4m3fn && t.scalar_type() != at::kByte) || !t.is_contiguous()) throw NotTaken{};
    for (int64_t s : t.sizes())
      if (s > INT_MAX) throw NotTaken{};
    return t;
  }
  const at::Tensor& any_tensor() {
    PyObject* o = *v_++;
    if (!THPVariable_CheckExact(o)) throw NotTaken{};
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage()) throw NotTaken{};
    return t;
  }
  bool none() {
    if (*v_ != Py_None) return false;
    ++v_;
    return true;
  }
  int32_t i32() { return static_cast<int32_t>(integer(INT_MIN, INT_MAX)); }
  uint32_t u32() { return static_cast<uint32_t>(integer(0, UINT_MAX)); }
  float f32() {
    PyObject* o = *v_;
    if (!PyFloat_CheckExact(o)) return static_cast<float>(integer(-(1 << 24), 1 << 24));
    ++v_;
    return static_cast<float>(PyFloat_AS_DOUBLE(o));
  }
  glide_stream_t stream() {
    PyObject* o = *v_++;
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    if (PyLong_CheckExact(o)) return handle(o);
    if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != g_stream_type) throw NotTaken{};
    struct Ref {
      PyObject* o;
      ~Ref() { Py_XDECREF(o); }
    } h{PyObject_GetAttrString(o, "cuda_stream")};
    if (h.o == nullptr || !PyLong_CheckExact(h.o)) throw NotTaken{};
    return handle(h.o);
  }

 private:
  long long integer(long long lo, long long hi) {
    PyObject* o = *v_++;
    if (!PyLong_CheckExact(o)) throw NotTaken{};
    int over = 0;
    const long long x = PyLong_AsLongLongAndOverflow(o, &over);
    if (over != 0 || x < lo || x > hi) throw NotTaken{};
    return x;
  }
  static glide_stream_t handle(PyObject* o) {
    void* p = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) throw NotTaken{};
    return static_cast<glide_stream_t>(p);
  }
  PyObject* const* v_;
};

template <class T>
T* ptr(const at::Tensor& t) {
  return static_cast<T*>(t.data_ptr());
}
int32_t* ints(const at::Tensor& t) { return ptr<int32_t>(t); }

// Runs `body`, which throws before its C call or returns that call's status; the GIL is given up
// around the C call alone, as ctypes does.
template <class F>
PyObject* call(F body) {
  long status = -1;
  try {
    status = body();
  } catch (...) {
    PyErr_Clear();
  }
  return PyLong_FromLong(status);
}
template <class F>
long without_gil(F f) {
  PyThreadState* s = PyEval_SaveThread();
  const long status = f();
  PyEval_RestoreThread(s);
  return status;
}

int32_t dim(const at::Tensor& t, int i) { return static_cast<int32_t>(t.size(i)); }

// queries [B, rows, H, D] and caches [B, H_kv, S_cap, D]
glide_attn_desc describe(const at::Tensor& q, const at::Tensor& K, const at::Tensor& V) {
  if (K.dim() != 4 || q.dim() != 4 || V.sizes() != K.sizes() || K.scalar_type() != V.scalar_type() ||
      q.scalar_type() != K.scalar_type() || q.size(0) != K.size(0) || q.size(3) != K.size(3))
    throw NotTaken{};
  glide_attn_desc d{};
  d.B = dim(K, 0);
  d.H = dim(q, 2);
  d.D = dim(K, 3);
  d.S_cap = dim(K, 2);
  d.dtype = K.scalar_type() == at::kBFloat16 ? GLIDE_BF16 : GLIDE_F32;
  d.H_kv = dim(K, 1) == d.H ? 0 : dim(K, 1);
  return d;
}
// What the kernels read and write as dense rows behind the pointer: the result, of the queries'
// shape, and the lengths of d.B sequences.
void check_dense(const at::Tensor& out, const at::Tensor& q, const at::Tensor& len, const glide_attn_desc& d) {
  if (out.sizes() != q.sizes() || !out.is_contiguous() || len.numel() < d.B || !len.is_contiguous()) throw NotTaken{};
}
void options(glide_attn_desc& d, Args& a) {
  d.scale = a.f32();
  d.flags = a.u32();
  d.max_ctas = a.i32();
}

// q, K, V, kv_len, max_kv_len, out, workspace (not where kNoAlloc), scale, flags, max_ctas, stream
template <bool kNoAlloc>
PyObject* cross_attn(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, kNoAlloc ? 10 : 11);
    const at::Tensor &q = a.data(), &K = a.data(), &V = a.data(), &len = a.tensor(at::kInt);
    glide_attn_desc d = describe(q, K, V);
    const int32_t most = a.i32();
    const at::Tensor& out = a.tensor(at::kFloat);
    if (q.size(1) != 1) throw NotTaken{};
    check_dense(out, q, len, d);
    void* ws = nullptr;
    size_t bytes = 0;
    if constexpr (!kNoAlloc) {
      const at::Tensor& w = a.any_tensor();
      ws = w.data_ptr();
      bytes = w.nbytes();
    }
    options(d, a);
    const glide_stream_t stream = a.stream();
    const void *pq = q.data_ptr(), *pk = K.data_ptr(), *pv = V.data_ptr();
    const int32_t* pl = ints(len);
    float* po = ptr<float>(out);
    return without_gil([&] {
      return long(kNoAlloc ? glide_cross_attn_noalloc(&d, pq, pk, pv, pl, most, po, stream)
                           : glide_cross_attn(&d, pq, pk, pv, pl, most, po, ws, bytes, stream));
    });
  });
}

// q, parent_idx, K, V, kv_len, max_kv_len, out, workspace, scale, flags, max_ctas, stream
PyObject* verify_attn(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 12);
    const at::Tensor &q = a.data(), &parent = a.tensor(at::kInt), &K = a.data(), &V = a.data();
    const at::Tensor& len = a.tensor(at::kInt);
    glide_attn_desc d = describe(q, K, V);
    const int32_t most = a.i32(), nodes = dim(q, 1);
    const at::Tensor &out = a.tensor(at::kFloat), &w = a.any_tensor();
    if (parent.dim() != 2 || parent.size(0) != d.B || parent.size(1) != nodes || !parent.is_contiguous())
      throw NotTaken{};
    check_dense(out, q, len, d);
    options(d, a);
    const glide_stream_t stream = a.stream();
    const void *pq = q.data_ptr(), *pk = K.data_ptr(), *pv = V.data_ptr();
    const int32_t *pp = ints(parent), *pl = ints(len);
    float* po = ptr<float>(out);
    void* ws = w.data_ptr();
    const size_t bytes = w.nbytes();
    return without_gil(
        [&] { return long(tree_verify_attn(&d, pq, nodes, pp, pk, pv, pl, most, po, ws, bytes, stream)); });
  });
}

// q, K, V, seq_len, L, out, workspace, scale, max_ctas, stream
PyObject* block_attn(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 10);
    const at::Tensor &q = a.data(), &K = a.data(), &V = a.data(), &len = a.tensor(at::kInt);
    glide_attn_desc d = describe(q, K, V);
    const int32_t L = a.i32(), T = dim(q, 1);
    const at::Tensor &out = a.tensor(at::kFloat), &w = a.any_tensor();
    if (len.dim() != 1 || len.size(0) != d.B) throw NotTaken{};
    check_dense(out, q, len, d);
    d.scale = a.f32();
    d.max_ctas = a.i32();
    const glide_stream_t stream = a.stream();
    const void *pq = q.data_ptr(), *pk = K.data_ptr(), *pv = V.data_ptr();
    const int32_t* pl = ints(len);
    float* po = ptr<float>(out);
    void* ws = w.data_ptr();
    const size_t bytes = w.nbytes();
    return without_gil(
        [&] { return long(glide_block_cross_attn(&d, pq, T, L, pk, pv, pl, po, ws, bytes, stream)); });
  });
}

// draft_tokens, parent_idx, target_logits, path, length, bonus, workspace, stream
PyObject* accept(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 8);
    const at::Tensor &tok = a.tensor(at::kInt), &parent = a.tensor(at::kInt), &logits = a.data();
    if (logits.dim() != 3 || logits.scalar_type() != at::kFloat) throw NotTaken{};
    const int32_t B = dim(logits, 0), nodes = dim(logits, 1), V = dim(logits, 2);
    const at::IntArrayRef rows = logits.sizes().slice(0, 2);
    const at::Tensor &path = a.tensor(at::kInt, {B, nodes}), &length = a.tensor(at::kInt, {B}),
                     &bonus = a.tensor(at::kInt, {B}), &w = a.any_tensor();
    if (tok.sizes() != rows || parent.sizes() != rows || !tok.is_contiguous() || !parent.is_contiguous())
      throw NotTaken{};
    const glide_stream_t stream = a.stream();
    const int32_t *pt = ints(tok), *pp = ints(parent);
    const float* pg = ptr<float>(logits);
    int32_t *pa = ints(path), *pl = ints(length), *pb = ints(bonus);
    void* ws = w.data_ptr();
    const size_t bytes = w.nbytes();
    return without_gil([&] { return long(tree_accept(pt, pp, pg, B, nodes, V, pa, pl, pb, ws, bytes, stream)); });
  });
}

// probs, root_token, max_tokens, draft_tokens, parent_idx, n_nodes, workspace, conf, fixed_k, stream
PyObject* expand(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 10);
    const at::Tensor& probs = a.data();
    if (probs.dim() != 3 || probs.scalar_type() != at::kFloat) throw NotTaken{};
    const int32_t B = dim(probs, 0), gamma = dim(probs, 1), V = dim(probs, 2);
    const at::Tensor& root = a.tensor(at::kInt, {B});
    const int32_t most = a.i32();
    const int64_t nodes = int64_t(most) + 1;
    const at::Tensor &tok = a.tensor(at::kInt, {B, nodes}), &parent = a.tensor(at::kInt, {B, nodes}),
                     &count = a.tensor(at::kInt, {B}), &w = a.any_tensor();
    float* conf = a.none() ? nullptr : ptr<float>(a.tensor(at::kFloat, {B, gamma}));
    const int32_t k = a.i32();
    const glide_stream_t stream = a.stream();
    const float* pp = ptr<float>(probs);
    const int32_t* pr = ints(root);
    int32_t *pt = ints(tok), *pa = ints(parent), *pn = ints(count);
    void* ws = w.data_ptr();
    const size_t bytes = w.nbytes();
    return without_gil(
        [&] { return long(cape_expand(pp, pr, B, gamma, V, most, k, pt, pa, pn, conf, ws, bytes, stream)); });
  });
}

// K, V, kv_len, path, length, new_kv_len, stream
PyObject* compact(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 7);
    const at::Tensor &K = a.data(), &V = a.data();
    const int64_t rank = K.dim();
    if ((rank != 4 && rank != 5) || K.sizes() != V.sizes() || K.scalar_type() != V.scalar_type()) throw NotTaken{};
    const int o = static_cast<int>(rank) - 4;
    glide_attn_desc d{};
    d.B = dim(K, o);
    d.H = dim(K, o + 1);
    d.S_cap = dim(K, o + 2);
    d.D = dim(K, o + 3);
    d.dtype = K.scalar_type() == at::kBFloat16 ? GLIDE_BF16 : GLIDE_F32;
    const int32_t layers = o ? dim(K, 0) : 1;
    const int64_t stride = int64_t(d.B) * d.H * d.S_cap * d.D;
    const at::Tensor &len = a.tensor(at::kInt, {d.B}), &path = a.tensor(at::kInt);
    if (path.dim() != 2 || path.size(0) != d.B || path.size(1) > INT_MAX || !path.is_contiguous()) throw NotTaken{};
    const int32_t nodes = dim(path, 1);
    const at::Tensor &length = a.tensor(at::kInt, {d.B}), &fresh = a.tensor(at::kInt, {d.B});
    const glide_stream_t stream = a.stream();
    void *pk = K.data_ptr(), *pv = V.data_ptr();
    const int32_t *pl = ints(len), *pp = ints(path), *pn = ints(length);
    int32_t* po = ints(fresh);
    return without_gil(
        [&] { return long(glide_kv_compact(&d, layers, stride, pk, pv, pl, nodes, pp, pn, po, stream)); });
  });
}

// draft_tokens, draft_probs, target_logits, uniforms, n_accepted, next_token, workspace, stream
PyObject* sample(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 8);
    const at::Tensor& tok = a.tensor(at::kInt);
    if (tok.dim() != 2 || tok.size(0) > INT_MAX || tok.size(1) >= INT_MAX || !tok.is_contiguous()) throw NotTaken{};
    const int32_t B = dim(tok, 0), gamma = dim(tok, 1);
    const at::Tensor &probs = a.data(), &logits = a.data();
    if (probs.dim() != 3 || logits.dim() != 3 || probs.scalar_type() != at::kFloat ||
        logits.scalar_type() != at::kFloat)
      throw NotTaken{};
    const int32_t V = dim(logits, 2);
    if (probs.sizes() != at::IntArrayRef({B, gamma, V}) || logits.sizes() != at::IntArrayRef({B, int64_t(gamma) + 1, V}))
      throw NotTaken{};
    const at::Tensor &u = a.tensor(at::kFloat, {B, int64_t(gamma) + 1}), &acc = a.tensor(at::kInt, {B}),
                     &next = a.tensor(at::kInt, {B}), &w = a.any_tensor();
    const glide_stream_t stream = a.stream();
    const int32_t* pt = ints(tok);
    const float *pp = ptr<float>(probs), *pg = ptr<float>(logits), *pu = ptr<float>(u);
    int32_t *pa = ints(acc), *pn = ints(next);
    void* ws = w.data_ptr();
    const size_t bytes = w.nbytes();
    return without_gil([&] { return long(spec_sample_accept(pt, pp, pg, pu, B, gamma, V, pa, pn, ws, bytes, stream)); });
  });
}

// An 8-bit cache: K, V codes (float8 or their bytes) and K_exp, V_exp, contiguous, of `rank` dimensions
// ([B, H_kv, S_cap, D], and [layers, ...] before them where rank is 5).
struct Cache8 {
  glide_kv8_cache c;
  at::IntArrayRef sizes;
  int device;
};
Cache8 cache8(Args& a) {
  const at::Tensor &K = a.codes(), &V = a.codes(), &Ke = a.tensor(at::kChar), &Ve = a.tensor(at::kChar);
  const int64_t rank = K.dim();
  if ((rank != 4 && rank != 5) || K.sizes() != V.sizes()) throw NotTaken{};
  for (const at::Tensor* e : {&Ke, &Ve}) {
    if (e->dim() != rank - 1 || !e->is_contiguous() || e->sizes().slice(0, rank - 2) != K.sizes().slice(0, rank - 2) ||
        e->size(rank - 2) != (K.size(rank - 2) + GLIDE_KV8_BLOCK - 1) / GLIDE_KV8_BLOCK || e->device() != K.device())
      throw NotTaken{};
  }
  if (V.device() != K.device()) throw NotTaken{};
  return {{K.data_ptr(), V.data_ptr(), static_cast<int8_t*>(Ke.data_ptr()), static_cast<int8_t*>(Ve.data_ptr())},
          K.sizes(), K.get_device()};
}
// Sizes of a cache's layer, and of the rows [.., B, rows, H_kv, D] or slabs [.., B, H_kv, rows, D] beside it.
glide_attn_desc describe8(const Cache8& k, at::ScalarType type) {
  const size_t o = k.sizes.size() - 4;
  glide_attn_desc d{};
  d.B = static_cast<int32_t>(k.sizes[o]);
  d.H = static_cast<int32_t>(k.sizes[o + 1]);
  d.S_cap = static_cast<int32_t>(k.sizes[o + 2]);
  d.D = static_cast<int32_t>(k.sizes[o + 3]);
  d.dtype = type == at::kBFloat16 ? GLIDE_BF16 : GLIDE_F32;
  return d;
}
int32_t layers8(const Cache8& k) { return k.sizes.size() == 5 ? static_cast<int32_t>(k.sizes[0]) : 1; }
void on(int device, std::initializer_list<const at::Tensor*> ts) {
  for (const at::Tensor* t : ts)
    if (t->get_device() != device) throw NotTaken{};
}

// k_new, v_new, K, V, K_exp, V_exp, kv_len, new_kv_len, path, length, stream
PyObject* kv8_append(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 11);
    const at::Tensor &kn = a.data(), &vn = a.data();
    const Cache8 k = cache8(a);
    const glide_attn_desc d = describe8(k, kn.scalar_type());
    const size_t o = k.sizes.size() - 4;
    if (kn.sizes() != vn.sizes() || kn.scalar_type() != vn.scalar_type() || kn.dim() != int64_t(o) + 4 ||
        (o && kn.size(0) != k.sizes[0]) || kn.size(o) != d.B || kn.size(o + 2) != d.H || kn.size(o + 3) != d.D)
      throw NotTaken{};
    const int32_t rows = dim(kn, static_cast<int>(o) + 1);
    const at::Tensor &len = a.tensor(at::kInt, {d.B}), &fresh = a.tensor(at::kInt, {d.B});
    on(k.device, {&kn, &vn, &len, &fresh});
    const int32_t *path = nullptr, *m = nullptr;
    if (!a.none()) {
      const at::Tensor& t = a.tensor(at::kInt, {d.B, rows});
      on(k.device, {&t});
      path = ints(t);
    }
    if (!a.none()) {
      const at::Tensor& t = a.tensor(at::kInt, {d.B});
      on(k.device, {&t});
      m = ints(t);
    }
    const glide_stream_t stream = a.stream();
    const int32_t layers = layers8(k);
    const void *pk = kn.data_ptr(), *pv = vn.data_ptr();
    const int32_t* pl = ints(len);
    int32_t* po = ints(fresh);
    return without_gil(
        [&] { return long(glide_kv8_append(&d, layers, &k.c, pk, pv, pl, rows, path, m, po, stream)); });
  });
}

// K, V, K_exp, V_exp, kv_len, K_out, V_out, stream
PyObject* kv8_read(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 8);
    const Cache8 k = cache8(a);
    const at::Tensor& len = a.tensor(at::kInt);
    const at::Tensor &K = a.data(), &V = a.data();
    const glide_attn_desc d = describe8(k, K.scalar_type());
    const size_t o = k.sizes.size() - 4;
    if (len.dim() != 1 || len.size(0) != d.B || !len.is_contiguous() || K.sizes() != V.sizes() ||
        K.scalar_type() != V.scalar_type() || K.dim() != int64_t(o) + 4 ||
        K.sizes().slice(0, o + 2) != k.sizes.slice(0, o + 2) || K.size(o + 3) != d.D)
      throw NotTaken{};
    on(k.device, {&len, &K, &V});
    const glide_stream_t stream = a.stream();
    const int32_t layers = layers8(k), rows = dim(K, static_cast<int>(o) + 2);
    const int32_t* pl = ints(len);
    void *pk = K.data_ptr(), *pv = V.data_ptr();
    return without_gil([&] { return long(glide_kv8_read(&d, layers, &k.c, pl, rows, pk, pv, stream)); });
  });
}

// q, (parent, k_tree, v_tree where kTree,) K, V, K_exp, V_exp, kv_len, max_kv_len, out, workspace, scale, max_ctas, stream
template <bool kTree>
PyObject* kv8_attn(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, kTree ? 15 : 12);
    const at::Tensor& q = a.data();
    if (q.dim() != 4) throw NotTaken{};
    const int32_t nodes = dim(q, 1);
    const at::Tensor *parent = nullptr, *kt = nullptr, *vt = nullptr;
    if constexpr (kTree) {
      parent = &a.tensor(at::kInt, {q.size(0), nodes});
      kt = &a.data();
      vt = &a.data();
    } else if (nodes != 1) {
      throw NotTaken{};
    }
    const Cache8 k = cache8(a);
    if (k.sizes.size() != 4) throw NotTaken{};
    glide_attn_desc d = describe8(k, q.scalar_type());
    if (q.size(0) != d.B || q.size(3) != d.D) throw NotTaken{};
    if constexpr (kTree) {
      for (const at::Tensor* t : {kt, vt})
        if (t->scalar_type() != q.scalar_type() || t->sizes() != at::IntArrayRef({d.B, nodes, d.H, d.D})) throw NotTaken{};
      on(k.device, {parent, kt, vt});
    }
    const int32_t heads = dim(q, 2);
    if (heads != d.H) {
      d.H_kv = d.H;
      d.H = heads;
    }
    const at::Tensor& len = a.tensor(at::kInt, {d.B});
    const int32_t most = a.i32();
    const at::Tensor &out = a.data(), &w = a.any_tensor();
    if (out.sizes() != q.sizes() || out.scalar_type() != q.scalar_type() || !w.is_contiguous()) throw NotTaken{};
    on(k.device, {&q, &len, &out, &w});
    d.scale = a.f32();
    d.max_ctas = a.i32();
    const glide_stream_t stream = a.stream();
    const void* pq = q.data_ptr();
    const int32_t* pl = ints(len);
    void *po = out.data_ptr(), *ws = w.data_ptr();
    const size_t bytes = w.nbytes();
    if constexpr (kTree) {
      const int32_t* pp = ints(*parent);
      const void *pk = kt->data_ptr(), *pv = vt->data_ptr();
      return without_gil(
          [&] { return long(glide_kv8_verify_attn(&d, pq, nodes, pp, pk, pv, &k.c, pl, most, po, ws, bytes, stream)); });
    } else {
      return without_gil([&] { return long(glide_kv8_cross_attn(&d, pq, &k.c, pl, most, po, ws, bytes, stream)); });
    }
  });
}

// ------------------------------------------------------------------ cache in pages
// The calls launch on the current device.
void on_current(std::initializer_list<const at::Tensor*> ts) { on(c10::cuda::current_device(), ts); }

// Rows of new tokens [T, heads, D], heads and elements dense; the elements from token to token.
struct TokenRows {
  const at::Tensor* t;
  int64_t stride;
};
TokenRows token_rows(Args& a) {
  const at::Tensor& t = a.any_tensor();
  if ((t.scalar_type() != at::kBFloat16 && t.scalar_type() != at::kFloat) || t.dim() != 3) throw NotTaken{};
  for (int64_t s : t.sizes())
    if (s < 1 || s > INT_MAX) throw NotTaken{};
  if (t.stride(2) != 1 || (t.size(1) > 1 && t.stride(1) != t.size(2))) throw NotTaken{};
  return {&t, t.size(0) > 1 ? t.stride(0) : t.size(1) * t.size(2)};
}
struct Pool {
  glide_page_pool c;
  const at::Tensor* K;
};
Pool page_pool(Args& a) {
  const at::Tensor &K = a.data(), &V = a.data();
  if (K.dim() != 4 || V.sizes() != K.sizes() || V.scalar_type() != K.scalar_type()) throw NotTaken{};
  on_current({&K, &V});
  return {{K.data_ptr(), V.data_ptr(), dim(K, 0), dim(K, 2)}, &K};
}
glide_attn_desc describe_rows(int32_t B, const at::Tensor& q, int32_t H_kv) {
  glide_attn_desc d{};
  d.B = B;
  d.H = dim(q, 1);
  d.D = dim(q, 2);
  d.S_cap = 1;
  d.dtype = q.scalar_type() == at::kBFloat16 ? GLIDE_BF16 : GLIDE_F32;
  d.H_kv = H_kv == d.H ? 0 : H_kv;
  return d;
}

// q_len, kv_len, held, block_table, free_pages, n_free, page_size, cu_q, slots, new_kv_len, new_held, new_n_free,
// positions, stream
PyObject* page_plan(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 14);
    const at::Tensor &q = a.tensor(at::kInt), &kv = a.tensor(at::kInt), &held = a.tensor(at::kInt),
                     &table = a.tensor(at::kInt), &free = a.tensor(at::kInt), &n_free = a.tensor(at::kInt, {1});
    const int32_t P = a.i32();
    if (table.dim() != 2 || !table.is_contiguous() || free.dim() != 1 || !free.is_contiguous()) throw NotTaken{};
    const int64_t B = table.size(0);
    if (B > INT_MAX - 1 || table.size(1) > INT_MAX || free.size(0) > INT_MAX) throw NotTaken{};
    for (const at::Tensor* t : {&q, &kv, &held})
      if (t->sizes() != at::IntArrayRef({B}) || !t->is_contiguous()) throw NotTaken{};
    const at::Tensor &cu = a.tensor(at::kInt, {B + 1}), &slots = a.tensor(at::kInt);
    if (slots.dim() != 1 || slots.size(0) > INT_MAX || !slots.is_contiguous()) throw NotTaken{};
    const at::Tensor &nkv = a.tensor(at::kInt, {B}), &nheld = a.tensor(at::kInt, {B}), &nn = a.tensor(at::kInt, {1});
    on_current({&q, &kv, &held, &table, &free, &n_free, &cu, &slots, &nkv, &nheld, &nn});
    int32_t* pos = nullptr;
    if (!a.none()) {
      const at::Tensor& t = a.tensor(at::kInt, {slots.size(0)});
      on_current({&t});
      pos = ints(t);
    }
    const glide_stream_t stream = a.stream();
    const int32_t b = static_cast<int32_t>(B), T = dim(slots, 0), W = dim(table, 1), cap = dim(free, 0);
    const int32_t *pq = ints(q), *pk = ints(kv), *ph = ints(held), *pf = ints(n_free);
    int32_t *pt = ints(table), *pfree = ints(free), *pc = ints(cu), *ps = ints(slots), *a1 = ints(nkv), *a2 = ints(nheld),
            *a3 = ints(nn);
    return without_gil(
        [&] { return long(glide_page_plan(b, T, P, W, pq, pk, ph, pt, pfree, cap, pf, pc, ps, pos, a1, a2, a3, stream)); });
  });
}

// k_new, v_new, K, V, slots, stream
PyObject* paged_append(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 6);
    const TokenRows k = token_rows(a), w = token_rows(a);
    const Pool pool = page_pool(a);
    const at::Tensor& K = *pool.K;
    const at::Tensor& slots = a.tensor(at::kInt, {k.t->size(0)});
    for (const at::Tensor* t : {k.t, w.t})
      if (t->scalar_type() != K.scalar_type() || t->sizes() != at::IntArrayRef({slots.size(0), K.size(1), K.size(3)}))
        throw NotTaken{};
    on_current({k.t, w.t, &slots});
    const glide_stream_t stream = a.stream();
    const glide_attn_desc d = describe_rows(1, *k.t, dim(K, 1));
    const int32_t T = dim(slots, 0);
    const void *pk = k.t->data_ptr(), *pv = w.t->data_ptr();
    const int32_t* ps = ints(slots);
    return without_gil([&] { return long(glide_paged_append(&d, &pool.c, pk, pv, k.stride, w.stride, T, ps, stream)); });
  });
}

// What both attention calls end with: out, workspace, scale, flags, stream.
struct RowsTail {
  void *out, *ws;
  size_t bytes;
  glide_stream_t stream;
};
RowsTail rows_tail(Args& a, const at::Tensor& q, glide_attn_desc& d) {
  const at::Tensor &out = a.data(), &w = a.any_tensor();
  if (out.sizes() != q.sizes() || out.scalar_type() != q.scalar_type() || !w.is_contiguous()) throw NotTaken{};
  on_current({&q, &out, &w});
  d.scale = a.f32();
  d.flags = a.u32();
  return {out.data_ptr(), w.data_ptr(), w.nbytes(), a.stream()};
}

// q, K, V, block_table, cu_q, max_q, kv_len, max_kv_len, out, workspace, scale, flags, stream
PyObject* paged_attn(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 13);
    const TokenRows q = token_rows(a);
    const Pool pool = page_pool(a);
    const at::Tensor& K = *pool.K;
    const at::Tensor& table = a.tensor(at::kInt);
    if (q.t->scalar_type() != K.scalar_type() || q.t->size(2) != K.size(3) || table.dim() != 2 || !table.is_contiguous() ||
        table.size(0) > INT_MAX - 1 || table.size(1) > INT_MAX)
      throw NotTaken{};
    const int64_t B = table.size(0);
    const at::Tensor& cu = a.tensor(at::kInt, {B + 1});
    const int32_t max_q = a.i32();
    const at::Tensor& len = a.tensor(at::kInt, {B});
    const int32_t most = a.i32();
    glide_attn_desc d = describe_rows(static_cast<int32_t>(B), *q.t, dim(K, 1));
    on_current({&table, &cu, &len});
    const RowsTail e = rows_tail(a, *q.t, d);
    const int32_t T = dim(*q.t, 0), W = dim(table, 1);
    const void* pq = q.t->data_ptr();
    const int32_t *pc = ints(cu), *pt = ints(table), *pl = ints(len);
    return without_gil([&] {
      return long(glide_paged_attn(&d, pq, q.stride, T, pc, max_q, &pool.c, pt, W, pl, most, e.out, e.ws, e.bytes, e.stream));
    });
  });
}

// q, k, v, cu, max_len, out, workspace, scale, flags, stream
PyObject* prompt_attn(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call([&] {
    Args a(v, n, 10);
    const TokenRows q = token_rows(a), k = token_rows(a), w = token_rows(a);
    for (const at::Tensor* t : {k.t, w.t})
      if (t->scalar_type() != q.t->scalar_type() || t->sizes() != at::IntArrayRef({q.t->size(0), k.t->size(1), q.t->size(2)}))
        throw NotTaken{};
    const at::Tensor& cu = a.tensor(at::kInt);
    if (cu.dim() != 1 || cu.size(0) < 2 || cu.size(0) > INT_MAX || !cu.is_contiguous()) throw NotTaken{};
    const int32_t max_len = a.i32();
    glide_attn_desc d = describe_rows(dim(cu, 0) - 1, *q.t, dim(*k.t, 1));
    on_current({k.t, w.t, &cu});
    const RowsTail e = rows_tail(a, *q.t, d);
    const int32_t T = dim(*q.t, 0);
    const void *pq = q.t->data_ptr(), *pk = k.t->data_ptr(), *pv = w.t->data_ptr();
    const int32_t* pc = ints(cu);
    return without_gil([&] {
      return long(glide_prompt_attn(&d, pq, q.stride, pk, k.stride, pv, w.stride, T, pc, max_len, e.out, e.ws, e.bytes,
                                    e.stream));
    });
  });
}

#define FN(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {FN("cross_attn", cross_attn<false>),
                          FN("cross_attn_noalloc", cross_attn<true>),
                          FN("verify_attn", verify_attn),
                          FN("block_attn", block_attn),
                          FN("accept", accept),
                          FN("expand", expand),
                          FN("compact", compact),
                          FN("sample", sample),
                          FN("kv8_append", kv8_append),
                          FN("kv8_read", kv8_read),
                          FN("kv8_cross", kv8_attn<false>),
                          FN("kv8_verify", kv8_attn<true>),
                          FN("page_plan", page_plan),
                          FN("paged_append", paged_append),
                          FN("paged_attn", paged_attn),
                          FN("prompt_attn", prompt_attn),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_glidecall", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__glidecall() {
  PyObject* m = PyImport_ImportModule("torch.cuda");
  if (m == nullptr) return nullptr;
  g_stream_type = PyObject_GetAttrString(m, "Stream");  // held for the process's life, as the module is
  Py_DECREF(m);
  return g_stream_type == nullptr ? nullptr : PyModule_Create(&kModule);
}
