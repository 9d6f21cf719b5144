// Argument marshalling of the Python binding in native code (host code only): checks of the tensors,
// output tensors and the call of the C entry point, for the calls that a decoding loop makes once
// or several times per step.  Their kernels take 5 to 15 us on small inputs, the same work in Python
// 5 to 20 us per call: a whole step of 1 sequence, 1 head, fp32 took 98 us, most of it here.
//
// Nothing is decided here that binding.py does not say: a function returns None, with nothing enqueued,
// whenever an argument is not what the entry point wants, and binding.py then goes through its own
// checks, which name the argument.  Tensors of other classes than torch.Tensor and Parameter are left to it
// too.  What can fail stands in front of the C call, the Python objects of its results among it: a call
// that has been enqueued returns them and is never made again.  A call that the library refuses returns its
// status.  The interpreter is left to other threads during allocations and the C call, as torch and ctypes
// do.  No state is kept but the addresses of the entry points.
#include <ATen/ATen.h>
#include <Python.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <memory>
#include <vector>

#include "../../include/propd.h"

namespace {

struct Entries {
  decltype(&propd_tree_mask) tree_mask = nullptr;
  decltype(&propd_tree_attention) tree_attention = nullptr;
  decltype(&propd_early_prune) early_prune = nullptr;
  decltype(&propd_early_prune_prob) early_prune_prob = nullptr;
  decltype(&propd_accept_path) accept_path = nullptr;
  decltype(&propd_commit_path) commit_path = nullptr;
  decltype(&propd_workspace_bytes) workspace_bytes = nullptr;
  decltype(&propd_grouped_attention) grouped_attention = nullptr;
  decltype(&propd_cache_observe) cache_observe = nullptr;
  decltype(&propd_cache_evict) cache_evict = nullptr;
  decltype(&propd_rotary) rotary = nullptr;
  decltype(&propd_paged_attention) paged_attention = nullptr;
  decltype(&propd_paged_commit) paged_commit = nullptr;
  decltype(&propd_paged_prompt) paged_prompt = nullptr;
  decltype(&propd_paged_read) paged_read = nullptr;
  decltype(&propd_accept_sampled) accept_sampled = nullptr;
};

struct NotThis {};  // the Python code takes over
struct Raised {};   // a Python error is set
struct Refused {
  propd_status status;
};

const at::Tensor &tensor(PyObject *o) {
  if (!THPVariable_CheckExact(o)) throw NotThis{};
  return THPVariable_Unpack(o);
}

void need(bool ok) {
  if (!ok) throw NotThis{};
}

// Other threads may run Python meanwhile: a launch waits where the queue is full, an allocation where memory has to be
// given back first, and what they wait for may need the interpreter.
struct Unlocked {
  PyThreadState *const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

template <class F>
auto unlocked(F &&f) {
  const Unlocked u;
  return f();
}

template <class Entry, class... Args>
void call(Entry entry, Args... args) {
  const propd_status status = unlocked([&] { return entry(args...); });
  if (status != PROPD_OK) throw Refused{status};
}

// a contiguous tensor of this type in GPU memory
const at::Tensor &dev(PyObject *o, at::ScalarType type) {
  const at::Tensor &t = tensor(o);
  need(t.is_cuda() && t.scalar_type() == type && t.is_contiguous());
  return t;
}

propd_dtype type_of(const at::Tensor &t) {
  if (t.scalar_type() == at::kBFloat16) return PROPD_BF16;
  need(t.scalar_type() == at::kFloat);
  return PROPD_F32;
}

void *ptr(PyObject *o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }

long long whole(PyObject *o) {
  need(PyLong_Check(o));
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    throw NotThis{};
  }
  return v;
}

int32_t whole32(PyObject *o) {
  const long long v = whole(o);
  need(v >= INT32_MIN && v <= INT32_MAX);
  return (int32_t)v;
}

int32_t size32(int64_t n) {
  need(n <= INT32_MAX);
  return (int32_t)n;
}

float real(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    throw NotThis{};
  }
  return (float)v;
}

bool truth(PyObject *o) {
  const int t = PyObject_IsTrue(o);
  if (t < 0) throw Raised{};
  return t == 1;
}

// binding._stream, called once the arguments have passed
void *stream_of(PyObject *current) {
  PyObject *o = PyObject_CallNoArgs(current);
  void *p = o ? PyLong_AsVoidPtr(o) : nullptr;
  Py_XDECREF(o);
  if (PyErr_Occurred()) throw Raised{};
  return p;
}

// the fields of binding.Tree: n_nodes, parent, token, depth, anc
propd_tree tree_of(PyObject *const *f) {
  const at::Tensor &parent = tensor(f[1]);
  need(parent.dim() >= 2);
  propd_tree t;
  t.B = size32(parent.size(0));
  t.T_max = size32(parent.size(1));
  t.n_nodes = (const int32_t *)ptr(f[0]);
  t.parent = (const int32_t *)parent.data_ptr();
  t.token = (const int32_t *)ptr(f[2]);
  t.depth = (const int32_t *)ptr(f[3]);
  t.anc = (const uint64_t *)ptr(f[4]);
  return t;
}

struct Workspace {
  at::Tensor own;
  void *ptr;
  size_t bytes;
};

Workspace workspace(PyObject *o, size_t need_bytes, const at::Tensor &like) {
  Workspace w;
  if (o != Py_None) {
    const at::Tensor &t = tensor(o);
    w.bytes = t.nbytes();
    need(w.bytes >= need_bytes && t.numel() * t.element_size() == (int64_t)w.bytes && t.device() == like.device() && t.is_contiguous());
    w.ptr = t.data_ptr();
  } else {
    w.own = unlocked([&] { return at::empty({(int64_t)(need_bytes > 256 ? need_bytes : 256)}, like.options().dtype(at::kByte)); });
    w.ptr = w.own.data_ptr();
    w.bytes = (size_t)w.own.numel();
  }
  return w;
}

struct Release {
  void operator()(PyObject *o) const { Py_DECREF(o); }
};
using Owned = std::unique_ptr<PyObject, Release>;

Owned owned(PyObject *o) {
  if (!o) throw Raised{};
  return Owned(o);
}

Owned object(const at::Tensor &t) {
  if (t.defined()) return owned(THPVariable_Wrap(t));
  Py_INCREF(Py_None);
  return Owned(Py_None);
}

Owned object(PyObject *o) {
  Py_INCREF(o);
  return Owned(o);
}

template <class... Items>
Owned tuple_of(Items... items) {
  Owned r = owned(PyTuple_New((Py_ssize_t)sizeof...(items)));
  Py_ssize_t n = 0;
  (PyTuple_SET_ITEM(r.get(), n++, items.release()), ...);
  return r;
}

Entries entries;

template <class F>
PyObject *guarded(F &&f) {
  try {
    return f().release();
  } catch (const NotThis &) {
  } catch (const Raised &) {
    return nullptr;
  } catch (const Refused &r) {
    return PyLong_FromLong((long)r.status);
  } catch (const std::exception &e) {  // for instance out of memory: the Python code meets the same and says so
    PyErr_Clear();
  }
  Py_RETURN_NONE;
}

template <class E>
void take(PyObject *o, E &entry) {
  entry = reinterpret_cast<E>(PyLong_AsVoidPtr(o));
}

PyObject *py_init(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "init: seven addresses");
    return nullptr;
  }
  take(a[0], entries.tree_mask);
  take(a[1], entries.tree_attention);
  take(a[2], entries.early_prune);
  take(a[3], entries.early_prune_prob);
  take(a[4], entries.accept_path);
  take(a[5], entries.commit_path);
  take(a[6], entries.workspace_bytes);
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

PyObject *py_init_cache(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 4) {
    PyErr_SetString(PyExc_TypeError, "init_cache: four addresses");
    return nullptr;
  }
  take(a[0], entries.grouped_attention);
  take(a[1], entries.cache_observe);
  take(a[2], entries.cache_evict);
  take(a[3], entries.rotary);
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

PyObject *py_init_paged(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "init_paged: five addresses");
    return nullptr;
  }
  take(a[0], entries.paged_attention);
  take(a[1], entries.paged_commit);
  take(a[2], entries.paged_prompt);
  take(a[3], entries.paged_read);
  take(a[4], entries.accept_sampled);
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

// tree_mask(n_nodes, parent, stream) -> (depth, anc)
PyObject *py_tree_mask(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 3);
    const at::Tensor &nodes = dev(a[0], at::kInt), &parent = dev(a[1], at::kInt);
    need(parent.dim() == 2);
    const int64_t B = parent.size(0), T = parent.size(1);
    at::Tensor depth, anc;
    {
      const Unlocked u;
      depth = at::empty({B, T}, parent.options());
      anc = at::empty({B, T, 2}, parent.options().dtype(at::kLong));
    }
    Owned result = tuple_of(object(depth), object(anc));
    call(entries.tree_mask, size32(B), size32(T), (const int32_t *)nodes.data_ptr(), (const int32_t *)parent.data_ptr(),
         (int32_t *)depth.data_ptr(), (uint64_t *)anc.data_ptr(), stream_of(a[2]));
    return result;
  });
}

// tree_attention(*tree, q, k_cache, v_cache, k_tree, v_tree, seq_lens, scale, out, workspace, stream) -> out
PyObject *py_tree_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 15);
    const propd_tree tree = tree_of(a);
    const at::Tensor &q = tensor(a[5]);
    const propd_dtype dt = type_of(q);
    need(q.dim() == 4);
    const int64_t B = q.size(0), H = q.size(1), T = q.size(2), d = q.size(3);
    const at::Tensor &kc = dev(a[6], q.scalar_type()), &vc = dev(a[7], q.scalar_type());
    const at::Tensor &kt = dev(a[8], q.scalar_type()), &vt = dev(a[9], q.scalar_type()), &seq = dev(a[10], at::kInt);
    need(q.is_cuda() && q.is_contiguous() && kc.dim() == 4);
    const int64_t L = kc.size(2);
    need(kc.sizes() == at::IntArrayRef({B, H, L, d}) && vc.sizes() == kc.sizes() && kt.sizes() == q.sizes() && vt.sizes() == q.sizes());
    need(tree.B == B && tree.T_max == T);
    const at::Tensor out = a[12] == Py_None ? unlocked([&] { return at::empty_like(q); }) : tensor(a[12]);
    const Workspace w = workspace(a[13], entries.workspace_bytes(PROPD_WS_TREE_ATTENTION, tree.B, tree.T_max, size32(H), size32(d),
                                                                 size32(L), 0, 0), q);
    Owned result = a[12] != Py_None ? object(a[12]) : object(out);
    call(entries.tree_attention, &tree, dt, size32(H), size32(d), real(a[11]), q.data_ptr(), L ? kc.data_ptr() : nullptr,
         L ? vc.data_ptr() : nullptr, kt.data_ptr(), vt.data_ptr(), (const int32_t *)seq.data_ptr(),
         size32(L), out.data_ptr(), w.ptr, w.bytes, stream_of(a[14]));
    return result;
  });
}

// early_prune(*tree, hidden, head, mode, value, payloads, payload_out, want_extra, workspace, stream) -> (keep_bits, new_index, orig_index,
// n_kept, cu_nodes, n_nodes, parent, token, depth, anc, rank or log_marginal or None, [payloads]); mode -1: top-k, else propd_prob_mode
PyObject *py_early_prune(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 14);
    const propd_tree tree = tree_of(a);
    const at::Tensor &hid = tensor(a[5]);
    const propd_dtype dt = type_of(hid);
    need(hid.dim() == 3 && hid.is_cuda() && hid.is_contiguous());
    const at::Tensor &head = dev(a[6], hid.scalar_type());
    const int64_t B = hid.size(0), T = hid.size(1), hidden = hid.size(2);
    need(head.dim() == 2 && head.size(1) == hidden && tree.B == B && tree.T_max == T);
    const int64_t vocab = head.size(0);
    const long long mode = whole(a[7]);
    const bool top_k = mode < 0, extra = truth(a[11]);
    const int32_t count = top_k || mode == PROPD_PROB_RANK ? whole32(a[8]) : 0;
    const float threshold = mode == PROPD_PROB_THRESHOLD ? real(a[8]) : 0.f;
    need(PyList_Check(a[9]) || PyTuple_Check(a[9]));
    const Py_ssize_t n_pay = PySequence_Fast_GET_SIZE(a[9]);
    const bool given = a[10] != Py_None;
    need(n_pay <= PROPD_MAX_PAYLOADS);
    need(!given || ((PyList_Check(a[10]) || PyTuple_Check(a[10])) && PySequence_Fast_GET_SIZE(a[10]) >= n_pay));
    // held here: the lists are not looked at again, other threads may change them
    at::Tensor src[PROPD_MAX_PAYLOADS], dst[PROPD_MAX_PAYLOADS];
    Owned dst_object[PROPD_MAX_PAYLOADS];
    for (Py_ssize_t i = 0; i < n_pay; ++i) {
      src[i] = tensor(PySequence_Fast_GET_ITEM(a[9], i));
      need(src[i].is_cuda() && src[i].is_contiguous() && (src[i].dim() == 3 || src[i].dim() == 4));
      need(src[i].size(0) == B && src[i].size(-2) == T);
      if (!given) continue;
      PyObject *const o = PySequence_Fast_GET_ITEM(a[10], i);
      dst[i] = tensor(o);
      need(dst[i].sizes() == src[i].sizes() && dst[i].scalar_type() == src[i].scalar_type() && dst[i].is_contiguous());
      dst_object[i] = object(o);
    }
    // per-node and per-sequence outputs in one allocation each, every one of them on a multiple of 16 bytes
    const bool rank = top_k && extra;
    std::vector<at::Tensor> nodes, counts;
    at::Tensor keep, cu, anc, more;
    {
      const Unlocked u;
      const auto i32 = hid.options().dtype(at::kInt), i64 = hid.options().dtype(at::kLong);
      nodes = at::empty_strided({rank ? 6 : 5, B, T}, {(B * T + 3) / 4 * 4, T, 1}, i32).unbind(0);
      counts = at::empty_strided({2, B}, {(B + 3) / 4 * 4, 1}, i32).unbind(0);
      keep = at::empty({B, 2}, i64);
      cu = at::empty({B + 1}, i32);
      anc = at::empty({B, T, 2}, i64);
      if (rank) more = nodes[5];
      if (!top_k && extra) more = at::empty({B, T}, hid.options().dtype(at::kFloat));
      for (Py_ssize_t i = 0; i < n_pay && !given; ++i) dst[i] = at::empty_like(src[i]);
    }
    propd_payload pay[PROPD_MAX_PAYLOADS];
    for (Py_ssize_t i = 0; i < n_pay; ++i) {
      const int64_t outer = src[i].dim() == 3 ? 1 : src[i].size(1), row = src[i].size(-1) * src[i].element_size();
      pay[i] = propd_payload{src[i].data_ptr(), dst[i].data_ptr(), (size_t)row, outer, outer * T * row, T * row, row};
      if (!given) dst_object[i] = object(dst[i]);
    }
    int32_t *node[5];
    for (int i = 0; i < 5; ++i) node[i] = (int32_t *)nodes[i].data_ptr();
    propd_tree_out out;
    out.n_nodes = (int32_t *)counts[1].data_ptr();
    out.parent = node[2];
    out.token = node[3];
    out.depth = node[4];
    out.anc = (uint64_t *)anc.data_ptr();
    const Workspace w = workspace(a[12], entries.workspace_bytes(PROPD_WS_EARLY_PRUNE, tree.B, tree.T_max, 0, 0, 0, size32(hidden),
                                                                 size32(vocab)), hid);
    uint64_t *keep_p = (uint64_t *)keep.data_ptr();
    int32_t *kept_p = (int32_t *)counts[0].data_ptr(), *cu_p = (int32_t *)cu.data_ptr();
    Owned moved = owned(PyList_New(n_pay));
    for (Py_ssize_t i = 0; i < n_pay; ++i) PyList_SET_ITEM(moved.get(), i, dst_object[i].release());
    Owned result = tuple_of(object(keep), object(nodes[0]), object(nodes[1]), object(counts[0]), object(cu), object(counts[1]),
                            object(nodes[2]), object(nodes[3]), object(nodes[4]), object(anc), object(more), std::move(moved));
    void *st = stream_of(a[13]);
    if (top_k)
      call(entries.early_prune, &tree, dt, size32(hidden), size32(vocab), count, hid.data_ptr(), head.data_ptr(), keep_p, node[0], node[1],
           kept_p, cu_p, &out, rank ? (int32_t *)more.data_ptr() : nullptr, (int32_t)n_pay, pay, w.ptr, w.bytes, st);
    else
      call(entries.early_prune_prob, &tree, dt, size32(hidden), size32(vocab), (propd_prob_mode)mode, threshold, count, hid.data_ptr(),
           head.data_ptr(), keep_p, node[0], node[1], kept_p, cu_p, &out, more.defined() ? (float *)more.data_ptr() : nullptr,
           (int32_t)n_pay, pay, w.ptr, w.bytes, st);
    return result;
  });
}

// accept_path(*tree, logits, path_stride or None, workspace, stream) -> (accept_len, path, next_token)
PyObject *py_accept_path(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 9);
    const propd_tree tree = tree_of(a);
    const at::Tensor &logits = tensor(a[5]);
    const propd_dtype dt = type_of(logits);
    need(logits.dim() == 3 && logits.is_cuda() && logits.is_contiguous() && tree.B == logits.size(0) && tree.T_max == logits.size(1));
    const int32_t vocab = size32(logits.size(2)), stride = a[6] == Py_None ? tree.T_max : whole32(a[6]);
    need(stride >= 0);
    at::Tensor len, path, next;
    {
      const Unlocked u;
      const auto i32 = logits.options().dtype(at::kInt);
      len = at::empty({tree.B}, i32);
      path = at::empty({tree.B, stride}, i32);
      next = at::empty({tree.B}, i32);
    }
    const Workspace w = workspace(a[7], entries.workspace_bytes(PROPD_WS_ACCEPT_PATH, tree.B, tree.T_max, 0, 0, 0, 0, vocab), logits);
    Owned result = tuple_of(object(len), object(path), object(next));
    call(entries.accept_path, &tree, dt, vocab, logits.data_ptr(), (int32_t *)len.data_ptr(), (int32_t *)path.data_ptr(), stride,
         (int32_t *)next.data_ptr(), w.ptr, w.bytes, stream_of(a[8]));
    return result;
  });
}

// commit_path(*tree, accept_len, path, next_token, k_tree, v_tree, k_cache, v_cache, seq_lens, out_stride or None, stream) -> tokens
PyObject *py_commit_path(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 15);
    const propd_tree tree = tree_of(a);
    const at::Tensor &len = dev(a[5], at::kInt), &path = dev(a[6], at::kInt), &next = dev(a[7], at::kInt), &seq = dev(a[12], at::kInt);
    const at::Tensor &kt = tensor(a[8]);
    const propd_dtype dt = type_of(kt);
    need(kt.dim() == 4 && kt.is_cuda() && kt.is_contiguous() && path.dim() >= 2);
    const at::Tensor &vt = dev(a[9], kt.scalar_type()), &kc = dev(a[10], kt.scalar_type()), &vc = dev(a[11], kt.scalar_type());
    const int64_t B = kt.size(0), H = kt.size(1), T = kt.size(2), d = kt.size(3);
    need(kc.dim() == 4);
    const int64_t L = kc.size(2);
    need(vt.sizes() == kt.sizes() && kc.sizes() == at::IntArrayRef({B, H, L, d}) && vc.sizes() == kc.sizes() && tree.B == B && tree.T_max == T);
    const int32_t stride = size32(path.size(1)), out_stride = a[13] == Py_None ? stride : whole32(a[13]);
    need(out_stride >= 0);
    const at::Tensor out = unlocked([&] { return at::empty({B, out_stride}, kt.options().dtype(at::kInt)); });
    Owned result = object(out);
    call(entries.commit_path, &tree, dt, size32(H), size32(d), (const int32_t *)len.data_ptr(), (const int32_t *)path.data_ptr(), stride,
         (const int32_t *)next.data_ptr(), kt.data_ptr(), vt.data_ptr(), kc.data_ptr(), vc.data_ptr(), size32(L),
         (int32_t *)seq.data_ptr(), (int32_t *)out.data_ptr(), out_stride, stream_of(a[14]));
    return result;
  });
}

// ---- a bounded cache with shared heads: all tensors contiguous on one GPU, the current one (binding._all_dev)
struct Device {
  c10::Device device;
  explicit Device(const at::Tensor &t) : device(t.device()) {
    need(device.is_cuda() && c10::impl::VirtualGuardImpl(device.type()).getDevice() == device);
  }
  const at::Tensor &operator()(PyObject *o, at::ScalarType type, at::IntArrayRef shape) const {
    const at::Tensor &t = tensor(o);
    need(t.device() == device && t.scalar_type() == type && t.is_contiguous() && t.sizes() == shape);
    return t;
  }
  // None where the argument may be left out
  template <class T>
  T *optional(PyObject *o, at::ScalarType type, at::IntArrayRef shape) const {
    return o == Py_None ? nullptr : (T *)(*this)(o, type, shape).data_ptr();
  }
};

bool overlap(const at::Tensor &x, const at::Tensor &y) {
  const char *a = (const char *)x.data_ptr(), *b = (const char *)y.data_ptr();
  return x.nbytes() && y.nbytes() && a < b + y.nbytes() && b < a + x.nbytes();
}

// from arguments that may be None
void apart(const at::Tensor &out, std::initializer_list<PyObject *> others) {
  for (PyObject *o : others) need(o == Py_None || !overlap(out, tensor(o)));
}

void same_or_apart(const at::Tensor &out, const at::Tensor &in) { need(out.data_ptr() == in.data_ptr() || !overlap(out, in)); }

// grouped_attention(*tree, q, k_cache, v_cache, k_tree, v_tree, seq_lens, scale, cap, window, slopes, position, dropped, want_lse, out, lse,
// workspace, stream) -> out or (out, lse)
PyObject *py_grouped_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 22);
    const at::Tensor &q = tensor(a[5]), &kt0 = tensor(a[8]), &kc0 = tensor(a[6]);
    const propd_dtype dt = type_of(q);
    const at::ScalarType type = q.scalar_type();
    need(q.dim() == 4 && kt0.dim() == 4 && kc0.dim() == 4 && q.is_contiguous());
    const Device on(q);
    const int64_t B = q.size(0), H = q.size(1), T = q.size(2), d = q.size(3), Hk = kt0.size(1), L = kc0.size(2);
    need(Hk >= 1 && H % Hk == 0);
    const at::Tensor &kc = on(a[6], type, {B, Hk, L, d}), &vc = on(a[7], type, {B, Hk, L, d});
    const at::Tensor &kt = on(a[8], type, {B, Hk, T, d}), &vt = on(a[9], type, {B, Hk, T, d}), &seq = on(a[10], at::kInt, {B});
    on(a[0], at::kInt, {B});
    on(a[4], at::kLong, {B, T, 2});
    const propd_tree tree = tree_of(a);
    need(tree.B == B && tree.T_max == T);
    propd_score_rule rule;
    rule.scale = real(a[11]);
    rule.cap = real(a[12]);
    rule.window = whole32(a[13]);
    rule.slopes = on.optional<float>(a[14], at::kFloat, {H});
    int32_t *position = on.optional<int32_t>(a[15], at::kInt, {B, Hk, L}), *dropped = on.optional<int32_t>(a[16], at::kInt, {B});
    const bool want = truth(a[17]) || a[19] != Py_None;
    at::Tensor out, lse;
    {
      const Unlocked u;
      if (a[18] == Py_None) out = at::empty_like(q);
      if (want && a[19] == Py_None) lse = at::empty({B, H, T}, q.options().dtype(at::kFloat));
    }
    if (a[18] != Py_None) out = on(a[18], type, q.sizes());
    if (a[19] != Py_None) lse = on(a[19], at::kFloat, {B, H, T});
    const std::initializer_list<PyObject *> read = {a[0], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[14], a[15], a[16]};
    if (a[18] != Py_None) apart(out, read);
    if (a[19] != Py_None) apart(lse, read);
    need(!want || !overlap(out, lse));
    if (a[20] != Py_None) {
      apart(tensor(a[20]), read);
      need(!overlap(tensor(a[20]), out) && (!want || !overlap(tensor(a[20]), lse)));
    }
    const Workspace w = workspace(a[20], entries.workspace_bytes(PROPD_WS_GROUPED_ATTENTION, tree.B, tree.T_max, size32(H), size32(d),
                                                                 size32(L), 0, 0), q);
    Owned o = a[18] != Py_None ? object(a[18]) : object(out);
    Owned result = want ? tuple_of(std::move(o), a[19] != Py_None ? object(a[19]) : object(lse)) : std::move(o);
    call(entries.grouped_attention, &tree, dt, size32(H), size32(Hk), size32(d), &rule, q.data_ptr(), L ? kc.data_ptr() : nullptr,
         L ? vc.data_ptr() : nullptr, kt.data_ptr(), vt.data_ptr(), (const int32_t *)seq.data_ptr(), L ? position : nullptr, dropped, size32(L),
         out.data_ptr(), want ? (float *)lse.data_ptr() : nullptr, w.ptr, w.bytes, stream_of(a[21]));
    return result;
  });
}

// cache_observe(*tree, accept_len, accept_path, q, lse, k_cache, k_tree, seq_lens, dropped, position, weight, scale, cap, window, slopes, decay,
// weight_out, position_out, stream) -> True
PyObject *py_cache_observe(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 23);
    const at::Tensor &q = tensor(a[7]), &kc0 = tensor(a[9]), &kt0 = tensor(a[10]), &path0 = tensor(a[6]);
    const propd_dtype dt = type_of(q);
    const at::ScalarType type = q.scalar_type();
    need(q.dim() == 4 && kt0.dim() == 4 && kc0.dim() == 4 && path0.dim() == 2 && q.is_contiguous());
    const Device on(q);
    const int64_t B = q.size(0), H = q.size(1), T = q.size(2), d = q.size(3), Hk = kt0.size(1), L = kc0.size(2), P = path0.size(1);
    need(Hk >= 1 && H % Hk == 0);
    on(a[0], at::kInt, {B});
    const propd_tree tree = tree_of(a);
    need(tree.B == B && tree.T_max == T);
    const at::Tensor &len = on(a[5], at::kInt, {B}), &path = on(a[6], at::kInt, {B, P}), &lse = on(a[8], at::kFloat, {B, H, T});
    const at::Tensor &kc = on(a[9], type, {B, Hk, L, d}), &kt = on(a[10], type, {B, Hk, T, d}), &seq = on(a[11], at::kInt, {B});
    int32_t *dropped = on.optional<int32_t>(a[12], at::kInt, {B}), *position = on.optional<int32_t>(a[13], at::kInt, {B, Hk, L});
    const at::Tensor &weight = on(a[14], at::kFloat, {B, Hk, L});
    propd_score_rule rule;
    rule.scale = real(a[15]);
    rule.cap = real(a[16]);
    rule.window = whole32(a[17]);
    rule.slopes = on.optional<float>(a[18], at::kFloat, {H});
    const float decay = real(a[19]);
    const at::Tensor &weight_out = a[20] == Py_None ? weight : on(a[20], at::kFloat, {B, Hk, L});
    int32_t *position_out = a[21] == Py_None ? position : on.optional<int32_t>(a[21], at::kInt, {B, Hk, L});
    same_or_apart(weight_out, weight);
    if (position && a[21] != Py_None) same_or_apart(tensor(a[21]), tensor(a[13]));
    PyObject *const at_out = a[21] != Py_None ? a[21] : a[13];
    const std::initializer_list<PyObject *> read = {a[0], a[5], a[6], a[7], a[8], a[9], a[10], a[11], a[12], a[18]};
    apart(weight_out, read);
    apart(weight_out, {a[13], at_out});
    if (at_out != Py_None) {
      apart(tensor(at_out), read);
      apart(tensor(at_out), {a[14]});
    }
    Owned result = object(Py_True);
    call(entries.cache_observe, &tree, dt, size32(H), size32(Hk), size32(d), &rule, decay, (const int32_t *)len.data_ptr(),
         (const int32_t *)path.data_ptr(), size32(P), q.data_ptr(), (const float *)lse.data_ptr(), kc.data_ptr(), kt.data_ptr(),
         (const int32_t *)seq.data_ptr(), dropped, position, (const float *)weight.data_ptr(), size32(L), position_out,
         (float *)weight_out.data_ptr(), stream_of(a[22]));
    return result;
  });
}

// cache_evict(k_cache, v_cache, seq_lens, dropped, position, weight, the same four for the results, budget, recent, sinks, workspace, stream) -> True
PyObject *py_cache_evict(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 15);
    const at::Tensor &k = tensor(a[0]);
    const propd_dtype dt = type_of(k);
    need(k.dim() == 4 && k.is_contiguous());
    const Device on(k);
    const at::Tensor &v = on(a[1], k.scalar_type(), k.sizes());
    need(!overlap(k, v));
    const int64_t B = k.size(0), Hk = k.size(1), L = k.size(2), d = k.size(3);
    propd_cache_rows rows[2];
    for (int i = 0; i < 2; ++i) {
      rows[i].seq_lens = (int32_t *)on(a[2 + 4 * i], at::kInt, {B}).data_ptr();
      rows[i].dropped = (int32_t *)on(a[3 + 4 * i], at::kInt, {B}).data_ptr();
      rows[i].position = (int32_t *)on(a[4 + 4 * i], at::kInt, {B, Hk, L}).data_ptr();
      rows[i].weight = (float *)on(a[5 + 4 * i], at::kFloat, {B, Hk, L}).data_ptr();
    }
    for (int i = 2; i < 6; ++i) same_or_apart(tensor(a[4 + i]), tensor(a[i]));
    for (int i = 2; i < 10; ++i) {
      apart(tensor(a[i]), {a[0], a[1]});
      for (int j = 6; j < 10; ++j) need(i % 4 == j % 4 || !overlap(tensor(a[j]), tensor(a[i])));
    }
    if (a[13] != Py_None)
      for (int i = 0; i < 10; ++i) need(!overlap(tensor(a[13]), tensor(a[i])));
    const int32_t budget = whole32(a[10]), recent = whole32(a[11]), sinks = whole32(a[12]);
    const Workspace w = workspace(a[13], entries.workspace_bytes(PROPD_WS_CACHE_EVICT, size32(B), 0, size32(Hk), 0, size32(L), 0, 0), k);
    Owned result = object(Py_True);
    call(entries.cache_evict, size32(B), dt, size32(Hk), size32(d), size32(L), budget, recent, sinks, k.data_ptr(), v.data_ptr(),
         (const propd_cache_rows *)&rows[0], (const propd_cache_rows *)&rows[1], w.ptr, w.bytes, stream_of(a[14]));
    return result;
  });
}

// rotary(q, k, inv_freq, offset, start, axis_of, n_rows, adjacent, q_out, k_out, stream) -> (q_out, k_out)
PyObject *py_rotary(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 11);
    const at::Tensor &q = tensor(a[0]), &inv = tensor(a[2]), &off = tensor(a[3]);
    const propd_dtype dt = type_of(q);
    const at::ScalarType type = q.scalar_type();
    need(q.dim() == 4 && q.is_contiguous() && inv.dim() == 1 && (off.dim() == 2 || off.dim() == 3));
    const Device on(q);
    const int64_t B = q.size(0), H = q.size(1), S = q.size(2), d = q.size(3), pairs = inv.size(0);
    const bool keys = a[1] != Py_None, each = off.dim() == 3;
    need(keys ? tensor(a[1]).dim() == 4 : a[9] == Py_None);
    const int64_t Hk = keys ? tensor(a[1]).size(1) : 0, offset_axes = each ? off.size(1) : 1;
    need(a[4] == Py_None || tensor(a[4]).dim() == 2);
    const int64_t axes = a[4] != Py_None ? tensor(a[4]).size(1) : offset_axes;
    on(a[2], at::kFloat, {pairs});
    if (each) on(a[3], at::kInt, {B, offset_axes, S});
    else on(a[3], at::kInt, {B, S});
    const int32_t *start = on.optional<int32_t>(a[4], at::kInt, {B, axes}), *axis_of = on.optional<int32_t>(a[5], at::kInt, {pairs});
    const int32_t *n_rows = on.optional<int32_t>(a[6], at::kInt, {B});
    const bool adjacent = truth(a[7]);
    at::Tensor k, q_out, k_out;
    if (keys) k = on(a[1], type, {B, Hk, S, d});
    {
      const Unlocked u;
      if (a[8] == Py_None) q_out = at::empty_like(q);
      if (keys && a[9] == Py_None) k_out = at::empty_like(k);
    }
    if (a[8] != Py_None) q_out = on(a[8], type, q.sizes());
    if (a[9] != Py_None) k_out = on(a[9], type, k.sizes());
    same_or_apart(q_out, q);
    if (a[8] != Py_None) apart(q_out, {a[2], a[3], a[4], a[5], a[6]});
    if (a[9] != Py_None) apart(k_out, {a[2], a[3], a[4], a[5], a[6]});
    if (keys) {
      same_or_apart(k_out, k);
      need(!overlap(q_out, k) && !overlap(q_out, k_out) && !overlap(k_out, q));
    }
    Owned result = tuple_of(a[8] != Py_None ? object(a[8]) : object(q_out), a[9] != Py_None ? object(a[9]) : object(k_out));
    call(entries.rotary, dt, size32(B), size32(S), size32(H), size32(Hk), size32(d), size32(2 * pairs), (int32_t)adjacent, size32(axes), axis_of,
         (const float *)inv.data_ptr(), start, (const int32_t *)off.data_ptr(), size32(offset_axes), n_rows, q.data_ptr(),
         keys ? k.data_ptr() : nullptr, q_out.data_ptr(), keys ? k_out.data_ptr() : nullptr, stream_of(a[10]));
    return result;
  });
}

// ---- a paged cache and acceptance by sampling

// the fields of binding.PagedCache: k_pages, v_pages, page_table, k_scale, v_scale
struct Paged {
  propd_paged_cache c;
  int64_t capacity;
};
Paged paged_of(PyObject *const *f, const Device &on, at::ScalarType type, int64_t B, int64_t Hk, int64_t d) {
  const at::Tensor &k = tensor(f[0]), &table0 = tensor(f[2]);
  need(k.dim() == 4 && table0.dim() == 2);
  const bool codes = k.scalar_type() == at::kFloat8_e4m3fn;
  const at::ScalarType kind = codes ? at::kFloat8_e4m3fn : type;
  const int64_t n = k.size(0), rows = k.size(2);
  on(f[0], kind, {n, Hk, rows, d});
  const at::Tensor &v = on(f[1], kind, {n, Hk, rows, d}), &table = on(f[2], at::kInt, {B, table0.size(1)});
  Paged p;
  p.c.k_pages = k.data_ptr();
  p.c.v_pages = v.data_ptr();
  p.c.k_scale = codes ? (uint8_t *)on(f[3], at::kByte, {n, Hk, rows}).data_ptr() : nullptr;
  p.c.v_scale = codes ? (uint8_t *)on(f[4], at::kByte, {n, Hk, rows}).data_ptr() : nullptr;
  if (!codes) need(f[3] == Py_None && f[4] == Py_None);
  p.c.page_table = (const int32_t *)table.data_ptr();
  p.c.dt = codes ? PROPD_E4M3 : type_of(k);
  p.c.n_pages = size32(n);
  p.c.table_pages = size32(table.size(1));
  p.c.page_rows = size32(rows);
  p.capacity = table.size(1) * rows;
  return p;
}

// a cache that is written to: its tensors lie apart from each other and from what is read
void written_apart(PyObject *const *f, std::initializer_list<PyObject *> read, PyObject *lens, PyObject *lens_out) {
  for (int i : {0, 1, 3, 4}) {
    if (f[i] == Py_None) continue;
    const at::Tensor &t = tensor(f[i]);
    for (int j = 0; j < 5; ++j) need(j == i || f[j] == Py_None || !overlap(t, tensor(f[j])));
    apart(t, read);
    apart(t, {lens, lens_out});
  }
  same_or_apart(tensor(lens_out), tensor(lens));
  apart(tensor(lens_out), read);
  apart(tensor(lens_out), {f[2]});
}

// paged_attention(*tree, *cache, q, k_tree, v_tree, seq_lens, scale, cap, window, slopes, want_lse, out, lse, workspace, stream) -> out or (out, lse)
PyObject *py_paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 23);
    PyObject *const *f = a + 5, *const *x = a + 10;
    const at::Tensor &q = tensor(x[0]), &kt0 = tensor(x[1]);
    const propd_dtype dt = type_of(q);
    const at::ScalarType type = q.scalar_type();
    need(q.dim() == 4 && kt0.dim() == 4 && q.is_contiguous());
    const Device on(q);
    const int64_t B = q.size(0), H = q.size(1), T = q.size(2), d = q.size(3), Hk = kt0.size(1);
    need(Hk >= 1 && H % Hk == 0);
    const at::Tensor &kt = on(x[1], type, {B, Hk, T, d}), &vt = on(x[2], type, {B, Hk, T, d}), &seq = on(x[3], at::kInt, {B});
    on(a[0], at::kInt, {B});
    on(a[4], at::kLong, {B, T, 2});
    const propd_tree tree = tree_of(a);
    need(tree.B == B && tree.T_max == T);
    const Paged cache = paged_of(f, on, type, B, Hk, d);
    propd_score_rule rule;
    rule.scale = real(x[4]);
    rule.cap = real(x[5]);
    rule.window = whole32(x[6]);
    rule.slopes = on.optional<float>(x[7], at::kFloat, {H});
    const bool want = truth(x[8]) || x[10] != Py_None;
    at::Tensor out, lse;
    {
      const Unlocked u;
      if (x[9] == Py_None) out = at::empty_like(q);
      if (want && x[10] == Py_None) lse = at::empty({B, H, T}, q.options().dtype(at::kFloat));
    }
    if (x[9] != Py_None) out = on(x[9], type, q.sizes());
    if (x[10] != Py_None) lse = on(x[10], at::kFloat, {B, H, T});
    const std::initializer_list<PyObject *> read = {a[0], a[4], f[0], f[1], f[2], f[3], f[4], x[0], x[1], x[2], x[3], x[7]};
    if (x[9] != Py_None) apart(out, read);
    if (x[10] != Py_None) apart(lse, read);
    need(!want || !overlap(out, lse));
    if (x[11] != Py_None) {
      apart(tensor(x[11]), read);
      need(!overlap(tensor(x[11]), out) && (!want || !overlap(tensor(x[11]), lse)));
    }
    const Workspace w = workspace(x[11], entries.workspace_bytes(PROPD_WS_PAGED_ATTENTION, tree.B, tree.T_max, size32(H), size32(d), size32(cache.capacity), 0, 0), q);
    Owned o = x[9] != Py_None ? object(x[9]) : object(out);
    Owned result = want ? tuple_of(std::move(o), x[10] != Py_None ? object(x[10]) : object(lse)) : std::move(o);
    call(entries.paged_attention, &tree, dt, size32(H), size32(Hk), size32(d), &rule, q.data_ptr(), &cache.c, kt.data_ptr(), vt.data_ptr(),
         (const int32_t *)seq.data_ptr(), out.data_ptr(), want ? (float *)lse.data_ptr() : nullptr, w.ptr, w.bytes, stream_of(x[12]));
    return result;
  });
}

// paged_commit(*tree, *cache, accept_len, path, next_token, k_tree, v_tree, seq_lens, seq_lens_out or None, out_stride or None, stream) -> tokens
PyObject *py_paged_commit(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 19);
    PyObject *const *f = a + 5, *const *x = a + 10;
    const at::Tensor &kt = tensor(x[3]), &path0 = tensor(x[1]);
    const propd_dtype dt = type_of(kt);
    need(kt.dim() == 4 && kt.is_contiguous() && path0.dim() == 2);
    const Device on(kt);
    const int64_t B = kt.size(0), Hk = kt.size(1), T = kt.size(2), d = kt.size(3), P = path0.size(1);
    const at::Tensor &vt = on(x[4], kt.scalar_type(), kt.sizes());
    const at::Tensor &len = on(x[0], at::kInt, {B}), &path = on(x[1], at::kInt, {B, P}), &next = on(x[2], at::kInt, {B}), &seq = on(x[5], at::kInt, {B});
    on(a[0], at::kInt, {B});
    on(a[2], at::kInt, {B, T});
    const propd_tree tree = tree_of(a);
    need(tree.B == B && tree.T_max == T);
    PyObject *const lens_out = x[6] == Py_None ? x[5] : x[6];
    const at::Tensor &seq_out = on(lens_out, at::kInt, {B});
    const Paged cache = paged_of(f, on, kt.scalar_type(), B, Hk, d);
    written_apart(f, {a[0], a[2], x[0], x[1], x[2], x[3], x[4]}, x[5], lens_out);
    const int32_t stride = size32(P), out_stride = x[7] == Py_None ? stride : whole32(x[7]);
    need(out_stride >= 0);
    const at::Tensor out = unlocked([&] { return at::empty({B, out_stride}, kt.options().dtype(at::kInt)); });
    Owned result = object(out);
    call(entries.paged_commit, &tree, dt, size32(Hk), size32(d), (const int32_t *)len.data_ptr(), (const int32_t *)path.data_ptr(), stride,
         (const int32_t *)next.data_ptr(), kt.data_ptr(), vt.data_ptr(), &cache.c, (const int32_t *)seq.data_ptr(), (int32_t *)seq_out.data_ptr(),
         (int32_t *)out.data_ptr(), out_stride, stream_of(x[8]));
    return result;
  });
}

// paged_prompt(*cache, k, v, seq_lens, n_rows or None, seq_lens_out or None, stream) -> True
PyObject *py_paged_prompt(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 11);
    PyObject *const *x = a + 5;
    const at::Tensor &k = tensor(x[0]);
    const propd_dtype dt = type_of(k);
    need(k.dim() == 4 && k.is_contiguous());
    const Device on(k);
    const int64_t B = k.size(0), Hk = k.size(1), S = k.size(2), d = k.size(3);
    const at::Tensor &v = on(x[1], k.scalar_type(), k.sizes()), &seq = on(x[2], at::kInt, {B});
    const int32_t *rows = on.optional<int32_t>(x[3], at::kInt, {B});
    PyObject *const lens_out = x[4] == Py_None ? x[2] : x[4];
    const at::Tensor &seq_out = on(lens_out, at::kInt, {B});
    const Paged cache = paged_of(a, on, k.scalar_type(), B, Hk, d);
    written_apart(a, {x[0], x[1], x[3]}, x[2], lens_out);
    Owned result = object(Py_True);
    call(entries.paged_prompt, dt, size32(B), size32(S), size32(Hk), size32(d), rows, k.data_ptr(), v.data_ptr(), &cache.c, (const int32_t *)seq.data_ptr(),
         (int32_t *)seq_out.data_ptr(), stream_of(x[5]));
    return result;
  });
}

// paged_read(*cache, seq_lens, k_out, v_out, first or None, stream) -> True
PyObject *py_paged_read(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 10);
    PyObject *const *x = a + 5;
    const at::Tensor &k = tensor(x[1]);
    const propd_dtype dt = type_of(k);
    need(k.dim() == 4 && k.is_contiguous());
    const Device on(k);
    const int64_t B = k.size(0), Hk = k.size(1), S = k.size(2), d = k.size(3);
    const at::Tensor &v = on(x[2], k.scalar_type(), k.sizes()), &seq = on(x[0], at::kInt, {B});
    const int32_t *first = on.optional<int32_t>(x[3], at::kInt, {B});
    const Paged cache = paged_of(a, on, k.scalar_type(), B, Hk, d);
    for (const at::Tensor *out : {&k, &v}) apart(*out, {x[0], x[3], a[0], a[1], a[2], a[3], a[4]});
    need(!overlap(k, v));
    Owned result = object(Py_True);
    call(entries.paged_read, dt, size32(B), size32(S), size32(Hk), size32(d), &cache.c, (const int32_t *)seq.data_ptr(), first, k.data_ptr(), v.data_ptr(),
         stream_of(x[4]));
    return result;
  });
}

// accept_sampled(*tree, logits, u, u_next, inv_temperature, draft_logits or None, draft_inv_temperature, path_stride or None, workspace, stream)
// -> (length, path, next)
PyObject *py_accept_sampled(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> Owned {
    need(n == 14);
    PyObject *const *x = a + 5;
    const at::Tensor &logits = tensor(x[0]);
    const propd_dtype dt = type_of(logits);
    need(logits.dim() == 3 && logits.is_contiguous());
    const Device on(logits);
    const int64_t B = logits.size(0), T = logits.size(1), V = logits.size(2);
    const at::Tensor &u = on(x[1], at::kFloat, {B, T}), &u_next = on(x[2], at::kFloat, {B});
    on(a[0], at::kInt, {B});
    on(a[1], at::kInt, {B, T});
    on(a[2], at::kInt, {B, T});
    const propd_tree tree = tree_of(a);
    need(tree.B == B && tree.T_max == T);
    const float inv = real(x[3]), draft_inv = real(x[5]);
    const void *draft = on.optional<void>(x[4], logits.scalar_type(), logits.sizes());
    const int32_t stride = x[6] == Py_None ? size32(T) : whole32(x[6]), vocab = size32(V);
    need(stride >= 0);
    const auto i32 = logits.options().dtype(at::kInt);
    at::Tensor len, path, next;
    {
      const Unlocked unlock;
      len = at::empty({B}, i32);
      path = at::empty({B, stride}, i32);
      next = at::empty({B}, i32);
    }
    if (x[7] != Py_None) apart(tensor(x[7]), {a[0], a[1], a[2], x[0], x[1], x[2], x[4]});
    const Workspace w = workspace(x[7], entries.workspace_bytes(PROPD_WS_ACCEPT_SAMPLED, tree.B, tree.T_max, 0, 0, 0, 0, vocab), logits);
    Owned result = tuple_of(object(len), object(path), object(next));
    call(entries.accept_sampled, &tree, dt, vocab, logits.data_ptr(), inv, draft, draft_inv, (const float *)u.data_ptr(), (const float *)u_next.data_ptr(),
         (int32_t *)len.data_ptr(), (int32_t *)path.data_ptr(), stride, (int32_t *)next.data_ptr(), w.ptr, w.bytes, stream_of(x[8]));
    return result;
  });
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(init),        METHOD(tree_mask),   METHOD(tree_attention), METHOD(early_prune),
                         METHOD(accept_path), METHOD(commit_path), METHOD(grouped_attention), METHOD(cache_observe),
                         METHOD(cache_evict), METHOD(rotary),      METHOD(init_cache),  METHOD(init_paged),  METHOD(paged_attention),
                         METHOD(paged_commit), METHOD(paged_prompt), METHOD(paged_read),   METHOD(accept_sampled),    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__marshal() { return PyModule_Create(&module); }
