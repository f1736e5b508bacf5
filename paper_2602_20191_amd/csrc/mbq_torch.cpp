// The stage call of the Python binding, and the calls beside a frozen blob, in native code: allocates what the caller left to the binding, checks the tensors,
// hands their addresses to the C ABI.  The same work in Python (six allocations, nine argument arrays, two size queries, the
// stream's handle) took 22.6 us a call of one 2048 x 2048 linear, twice what its two launches take on the GPU.
// Nothing is kept from one call for the next.
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdint.h>

#include <array>
#include <string>

namespace {

constexpr int kMaxGroup = 16;  // more than the C ABI takes: it refuses those itself

// addresses of the library's calls and what the binding raises, handed over once by bind()
typedef int (*StageFn)(const void*, int64_t, int64_t, int, const void* const*, const void* const*, int, const void* const*,
                       const int64_t*, void* const*, void* const*, void* const*, void* const*, void*, size_t, void*, size_t, int,
                       void*);
typedef int (*StageCfgFn)(const void*, int64_t, int64_t, int, const void* const*, const void* const*, const void*,
                          const void* const*, const int64_t*, void* const*, void* const*, void* const*, void* const*, void*,
                          size_t, void*, size_t, int, void*);
struct Library {
  StageFn stage = nullptr;
  StageCfgFn stage_cfg = nullptr;
  size_t (*route_bytes)(int64_t, int64_t) = nullptr;
  size_t (*linear_bytes)(int64_t, int64_t, int64_t) = nullptr;
  const char* (*last_error)() = nullptr;
  PyObject *error = nullptr, *device = nullptr, *stream = nullptr;  // MbqError; current device, its stream's handle
};
Library lib;

struct PythonError {};  // a Python exception is set

[[noreturn]] void fail(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw PythonError{};
}
const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a tensor");
  return THPVariable_Unpack(o);
}
void* pointer(const at::Tensor& t) {
  if (!t.is_cuda() || !t.is_contiguous()) fail(lib.error, "tensors handed to libmbq must be contiguous device tensors");
  return t.data_ptr();
}

struct Owned {  // a reference of one's own
  PyObject* o;
  explicit Owned(PyObject* p) : o(p) {
    if (!p) throw PythonError{};
  }
  Owned(const Owned&) = delete;
  Owned& operator=(const Owned&) = delete;
  ~Owned() { Py_XDECREF(o); }
  PyObject* take() {
    PyObject* p = o;
    o = nullptr;
    return p;
  }
};
// the elements of any sequence (borrowed for as long as the object lives)
struct Items {
  Owned fast;
  explicit Items(PyObject* o) : fast(PySequence_Fast(o, "expected a sequence")) {}
  Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(fast.o); }
  PyObject* operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(fast.o, i); }
};
int64_t whole(PyObject* o) {
  Owned v(PyNumber_Long(o));
  const long long r = PyLong_AsLongLong(v.o);
  if (r == -1 && PyErr_Occurred()) throw PythonError{};
  return r;
}

// stage(X, Wr, br, blobs, Ns, routing, Y, ws_route, ws_linear, algo, cfg): routing, Y and the workspaces may be None; cfg: the
// address of an mbq_config, or 0 for the default slices
PyObject* stage_call(PyObject* const* args) {
  const at::Tensor& X = tensor(args[0]);
  const int64_t cfg = whole(args[10]);
  if (X.dim() != 2 || X.scalar_type() != at::kBFloat16) fail(PyExc_AssertionError, "X must be a bf16 matrix");
  const int64_t T = X.size(0), K = X.size(1);
  const Items Wr(args[1]), br(args[2]), blobs(args[3]), Ns(args[4]);
  const Py_ssize_t n = Ns.size();
  const auto fits = [&](const Items& items) { return cfg ? items.size() >= n : items.size() == n; };
  if (n < 1 || !fits(Wr) || !fits(br) || !fits(blobs))
    fail(PyExc_AssertionError, "Wr, br, blobs and Ns must have the same length of at least 1");
  if (n > kMaxGroup) fail(lib.error, "too many matrices for one call");
  const int P = (int)tensor(Wr[0]).size(0);
  const auto of = [&](at::ScalarType type) { return at::TensorOptions().dtype(type).device(X.device()); };

  const void *w[kMaxGroup], *b[kMaxGroup], *blob[kMaxGroup];
  void *prec[kMaxGroup], *perm[kMaxGroup], *offsets[kMaxGroup], *y[kMaxGroup];
  int64_t rows[kMaxGroup], most = 0;
  for (Py_ssize_t i = 0; i < n; ++i) {
    w[i] = pointer(tensor(Wr[i]));
    b[i] = pointer(tensor(br[i]));
    blob[i] = pointer(tensor(blobs[i]));
    rows[i] = whole(Ns[i]);
    if (rows[i] > most) most = rows[i];
  }
  // what the caller gave comes back as it is, also beyond the n that are used
  const auto given = [&](PyObject* o, const char* what) {
    Owned all(PySequence_List(o));
    if (PyList_GET_SIZE(all.o) < n) fail(PyExc_AssertionError, what);
    return all.take();
  };
  Owned routing(args[5] != Py_None ? given(args[5], "one routing per matrix") : PyList_New(n));
  if (args[5] != Py_None) {
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(routing.o); ++i) {
      Owned r(PySequence_Tuple(PyList_GET_ITEM(routing.o, i)));
      if (PyTuple_GET_SIZE(r.o) < 3) fail(PyExc_IndexError, "a routing has precisions, order and offsets");
      if (i < n) {
        prec[i] = pointer(tensor(PyTuple_GET_ITEM(r.o, 0)));
        perm[i] = pointer(tensor(PyTuple_GET_ITEM(r.o, 1)));
        offsets[i] = pointer(tensor(PyTuple_GET_ITEM(r.o, 2)));
      }
      PyList_SetItem(routing.o, i, r.take());
    }
  } else {
    for (Py_ssize_t i = 0; i < n; ++i) {
      Owned r(PyTuple_New(3));
      void** const to[3] = {&prec[i], &perm[i], &offsets[i]};
      // (the tokens of a configuration are still sorted into the default's four buckets)
      const int64_t size[3] = {T, T, cfg ? 5 : P + 1};
      for (int k = 0; k < 3; ++k) {
        at::Tensor t = at::empty({size[k]}, of(at::kInt));
        *to[k] = t.data_ptr();
        Owned o(THPVariable_Wrap(std::move(t)));
        PyTuple_SET_ITEM(r.o, k, o.take());
      }
      PyList_SET_ITEM(routing.o, i, r.take());
    }
  }
  Owned Y(args[6] != Py_None ? given(args[6], "one output per matrix") : PyList_New(n));
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (args[6] != Py_None) {
      y[i] = pointer(tensor(PyList_GET_ITEM(Y.o, i)));
    } else {
      at::Tensor t = at::empty({T, rows[i]}, of(at::kFloat));
      y[i] = t.data_ptr();
      Owned o(THPVariable_Wrap(std::move(t)));
      PyList_SET_ITEM(Y.o, i, o.take());
    }
  }
  // workspaces: of the caller, or one allocation for what is missing (in use until the stream has passed the call, which is
  // as long as the allocator keeps it from others)
  void *ws_route = nullptr, *ws_linear = nullptr;
  size_t route_bytes = 0, linear_bytes = 0;
  at::Tensor own;
  if (args[7] != Py_None) {
    const at::Tensor& t = tensor(args[7]);
    ws_route = pointer(t);
    route_bytes = (size_t)t.numel();
  }
  if (args[8] != Py_None) {
    const at::Tensor& t = tensor(args[8]);
    ws_linear = pointer(t);
    linear_bytes = (size_t)t.numel();
  }
  if (!ws_route || !ws_linear) {
    size_t at_linear = 0;
    if (args[7] == Py_None) {
      route_bytes = lib.route_bytes(T, K);
      at_linear = (route_bytes + 255) / 256 * 256;
    }
    if (args[8] == Py_None) linear_bytes = lib.linear_bytes(T, most, K);
    own = at::empty({(int64_t)(at_linear + (args[8] == Py_None ? linear_bytes : 0))}, of(at::kByte));
    char* const base = static_cast<char*>(own.data_ptr());
    if (args[7] == Py_None) ws_route = base;
    if (args[8] == Py_None) ws_linear = base + at_linear;
  }
  Owned device(PyObject_CallNoArgs(lib.device));
  Owned handle(PyObject_CallFunctionObjArgs(lib.stream, device.o, nullptr));
  void* const stream = PyLong_AsVoidPtr(handle.o);
  if (!stream && PyErr_Occurred()) throw PythonError{};
  const int algo = (int)whole(args[9]);
  void* const x = pointer(X);
  int status;
  Py_BEGIN_ALLOW_THREADS;
  status = cfg ? lib.stage_cfg(x, T, K, (int)n, w, b, reinterpret_cast<const void*>((intptr_t)cfg), blob, rows, prec, perm, offsets,
                               y, ws_route, route_bytes, ws_linear, linear_bytes, algo, stream)
               : lib.stage(x, T, K, (int)n, w, b, P, blob, rows, prec, perm, offsets, y, ws_route, route_bytes, ws_linear,
                           linear_bytes, algo, stream);
  Py_END_ALLOW_THREADS;
  if (status != 0) {
    const std::string text = std::string(cfg ? "mbq_routed_linear_group_cfg" : "mbq_routed_linear_group") +
                             " failed with status " + std::to_string(status) + ": " + lib.last_error();
    fail(lib.error, text.c_str());
  }
  return PyTuple_Pack(2, routing.o, Y.o);
}

PyObject* stage(PyObject*, PyObject* const* args, Py_ssize_t count) {
  HANDLE_TH_ERRORS  // torch's errors as the Python exceptions that they are elsewhere (torch.OutOfMemoryError among them)
  try {
    if (!lib.stage) fail(PyExc_RuntimeError, "bind() comes first");
    if (count != 11) fail(PyExc_TypeError, "stage() takes 11 arguments");
    return stage_call(args);
  } catch (const PythonError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// bind(stage, stage_cfg, route_bytes, linear_bytes, last_error, MbqError, current_device, raw_stream)
PyObject* bind(PyObject*, PyObject* args) {
  Py_ssize_t a[5];
  PyObject* o[3];
  if (!PyArg_ParseTuple(args, "nnnnnOOO", &a[0], &a[1], &a[2], &a[3], &a[4], &o[0], &o[1], &o[2])) return nullptr;
  lib.stage = reinterpret_cast<StageFn>(a[0]);
  lib.stage_cfg = reinterpret_cast<StageCfgFn>(a[1]);
  lib.route_bytes = reinterpret_cast<decltype(lib.route_bytes)>(a[2]);
  lib.linear_bytes = reinterpret_cast<decltype(lib.linear_bytes)>(a[3]);
  lib.last_error = reinterpret_cast<decltype(lib.last_error)>(a[4]);
  PyObject** const to[3] = {&lib.error, &lib.device, &lib.stream};
  for (int i = 0; i < 3; ++i) {
    Py_INCREF(o[i]);
    Py_XSETREF(*to[i], o[i]);
  }
  Py_RETURN_NONE;
}

// ---- what stands beside a frozen blob: adapters, the balance loss, the routers' gradients ----------------------------
// The same work in Python took 17 to 27 us a call, two to six times what the launches take on the GPU for small batches.
typedef int (*LoraFn)(const void*, int64_t, int64_t, int, const void* const*, const void* const*, const int64_t*, int64_t, int,
                      const void*, const void*, const void*, const void*, const void*, const void* const*, void* const*,
                      void* const*, void*, size_t, void*);
typedef int (*LoraBackwardFn)(const void*, int64_t, int64_t, int, const void* const*, const void* const*, const int64_t*, int64_t,
                              int, const void*, const void*, const void*, const void*, const void*, const void* const*,
                              const void* const*, const void*, void*, void* const*, void* const*, void*, size_t, void*);
typedef int (*BalanceFn)(int, const void* const*, int64_t, int, const void*, const double*, double, void* const*, void* const*,
                         void* const*, void*, size_t, void*);
typedef int (*RouteBackwardFn)(const void*, int64_t, int64_t, int, const void* const*, int, const void* const*, const void*,
                               const void*, void*, void* const*, void* const*, void*, size_t, void*);
struct Beside {
  LoraFn lora = nullptr;
  size_t (*lora_bytes)(int64_t, int64_t, int, int) = nullptr;
  LoraBackwardFn lora_backward = nullptr;
  size_t (*lora_backward_bytes)(int64_t, int64_t, int, const int64_t*, int64_t, int) = nullptr;
  BalanceFn balance = nullptr;
  size_t (*balance_bytes)(int64_t, int) = nullptr;
  RouteBackwardFn route_backward = nullptr;
  size_t (*route_backward_bytes)(int64_t, int64_t, int, int) = nullptr;
};
Beside beside;

void assert_that(bool holds, const char* text) {
  if (!holds) fail(PyExc_AssertionError, text);
}
std::string shown(at::ScalarType type, at::IntArrayRef shape) {
  std::string s = std::string(c10::toString(type)) + " [";
  for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
  return s + "]";
}
// Where the call runs: the device of its first tensor, which has to be the current one, whose current stream it goes to.
struct Place {
  at::Device device;
  void* stream;
  explicit Place(const at::Tensor& t) : device(t.device()), stream(nullptr) {
    if (!t.is_cuda()) fail(lib.error, "tensors handed to libmbq must be contiguous device tensors");
    Owned current(PyObject_CallNoArgs(lib.device));
    if (whole(current.o) != device.index()) {
      const std::string text = "the tensors are on " + device.str() + ", the current device is " + std::to_string(whole(current.o));
      fail(lib.error, text.c_str());
    }
    Owned handle(PyObject_CallFunctionObjArgs(lib.stream, current.o, nullptr));
    stream = PyLong_AsVoidPtr(handle.o);
    if (!stream && PyErr_Occurred()) throw PythonError{};
  }
  // the address of a contiguous tensor of this type and shape on this device
  void* of(const at::Tensor& t, at::ScalarType type, at::IntArrayRef shape, const char* what) const {
    if (t.scalar_type() != type || t.sizes() != shape) {
      const std::string text = std::string(what) + " must be " + shown(type, shape) + ", got " + shown(t.scalar_type(), t.sizes());
      fail(PyExc_AssertionError, text.c_str());
    }
    if (t.device() != device) {
      const std::string text = std::string(what) + " is on " + t.device().str() + ", the call on " + device.str();
      fail(lib.error, text.c_str());
    }
    return pointer(t);
  }
  void* of(PyObject* o, at::ScalarType type, at::IntArrayRef shape, const char* what) const {
    return of(tensor(o), type, shape, what);
  }
  void* maybe(PyObject* o, at::ScalarType type, at::IntArrayRef shape, const char* what) const {
    return o == Py_None ? nullptr : of(o, type, shape, what);
  }
  at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type) const {
    return at::empty(shape, at::TensorOptions().dtype(type).device(device));
  }
};
// An output: the caller's, or a new one.
PyObject* output(const Place& place, PyObject* given, at::ScalarType type, at::IntArrayRef shape, const char* what, void** to) {
  if (given && given != Py_None) {
    *to = place.of(given, type, shape, what);
    Py_INCREF(given);
    return given;
  }
  at::Tensor t = place.fresh(shape, type);
  *to = t.data_ptr();
  return Owned(THPVariable_Wrap(std::move(t))).take();
}
// One output per projection, as a list; given: None or a sequence of n.
struct Outputs {
  Owned list;
  void* address[kMaxGroup] = {};
  template <typename Shape>
  Outputs(const Place& place, PyObject* given, Py_ssize_t n, at::ScalarType type, const Shape& shape, const char* what)
      : list(PyList_New(n)) {
    if (given == Py_None) {
      for (Py_ssize_t i = 0; i < n; ++i) PyList_SET_ITEM(list.o, i, output(place, nullptr, type, shape(i), what, &address[i]));
      return;
    }
    const Items items(given);
    if (items.size() != n) {
      const std::string text = std::string("one ") + what + " per projection";
      fail(PyExc_AssertionError, text.c_str());
    }
    for (Py_ssize_t i = 0; i < n; ++i) PyList_SET_ITEM(list.o, i, output(place, items[i], type, shape(i), what, &address[i]));
  }
};
// The workspace of a call: the caller's, or a new one, in use until the stream has passed the call.
struct Workspace {
  at::Tensor own;
  void* address;
  size_t bytes;
  Workspace(const Place& place, PyObject* given, size_t need) {
    if (given != Py_None) {
      const at::Tensor& t = tensor(given);
      if (t.device() != place.device) fail(lib.error, "the workspace is on another device");
      address = pointer(t);
      bytes = (size_t)t.numel() * t.element_size();
    } else {
      bytes = need < 256 ? 256 : need;
      own = place.fresh({(int64_t)bytes}, at::kByte);
      address = own.data_ptr();
    }
  }
};
void check(int status, const char* what) {
  if (status == 0) return;
  const std::string text = std::string(what) + " failed with status " + std::to_string(status) + ": " + lib.last_error();
  fail(lib.error, text.c_str());
}
Py_ssize_t group(Py_ssize_t n) {
  assert_that(n >= 1, "at least one projection");
  if (n > kMaxGroup) fail(lib.error, "too many projections for one call");
  return n;
}

// What both directions of the adapters read: X, A, B, (adapter, perm, offsets), scale, ranks.
struct LoraInputs {
  Place place;
  int64_t T, K, adapters, r, N[kMaxGroup];
  Py_ssize_t n;
  void *x, *a[kMaxGroup], *b[kMaxGroup], *scale, *ranks, *token[3];
  LoraInputs(PyObject* X, PyObject* A, PyObject* B, PyObject* tokens, PyObject* scales, PyObject* own_ranks) : place(tensor(X)) {
    const at::Tensor& xt = tensor(X);
    const Items as(A), bs(B), ts(tokens);
    assert_that(xt.dim() == 2 && as.size() >= 1 && as.size() == bs.size() && tensor(as[0]).dim() == 3,
                "X must be a matrix, A and B as many pools [adapters, r, columns] as there are projections");
    assert_that(ts.size() == 3, "tokens are (adapter, perm, offsets)");
    n = group(as.size());
    T = xt.size(0), K = xt.size(1), adapters = tensor(as[0]).size(0), r = tensor(as[0]).size(1);
    x = place.of(xt, at::kBFloat16, {T, K}, "X");
    for (Py_ssize_t i = 0; i < n; ++i) {
      const at::Tensor& bt = tensor(bs[i]);
      N[i] = bt.dim() == 3 ? bt.size(2) : 0;
      a[i] = place.of(as[i], at::kBFloat16, {adapters, r, K}, "A");
      b[i] = place.of(bt, at::kBFloat16, {adapters, r, N[i]}, "B");
    }
    token[0] = place.of(ts[0], at::kInt, {T}, "adapter");
    token[1] = place.of(ts[1], at::kInt, {T}, "perm");
    token[2] = place.of(ts[2], at::kInt, {adapters + 1}, "offsets");
    scale = place.of(scales, at::kFloat, {adapters}, "scale");
    ranks = place.maybe(own_ranks, at::kInt, {adapters}, "ranks");
  }
};

// lora(X, A, B, tokens, scale, ranks, base, Y, H, ws)
PyObject* lora_call(PyObject* const* args) {
  const LoraInputs in(args[0], args[1], args[2], args[3], args[4], args[5]);
  const auto wide = [&](Py_ssize_t i) { return std::array<int64_t, 2>{in.T, in.N[i]}; };
  const void* base[kMaxGroup] = {};
  if (args[6] != Py_None) {
    const Items items(args[6]);
    assert_that(items.size() == in.n, "one base per projection");
    for (Py_ssize_t i = 0; i < in.n; ++i) base[i] = in.place.maybe(items[i], at::kFloat, wide(i), "base");
  }
  void* h[kMaxGroup] = {};
  if (args[8] != Py_None) {
    const Items items(args[8]);
    assert_that(items.size() == in.n, "one H per projection");
    for (Py_ssize_t i = 0; i < in.n; ++i) h[i] = in.place.of(items[i], at::kFloat, {in.T, in.r}, "H");
  }
  Outputs y(in.place, args[7], in.n, at::kFloat, wide, "Y");
  const Workspace ws(in.place, args[9], args[9] == Py_None ? beside.lora_bytes(in.T, in.K, (int)in.n, (int)in.r) : 0);
  int status;
  Py_BEGIN_ALLOW_THREADS;
  status = beside.lora(in.x, in.T, in.K, (int)in.n, in.a, in.b, in.N, in.adapters, (int)in.r, in.ranks, in.scale, in.token[0],
                       in.token[1], in.token[2], base, y.address, args[8] != Py_None ? h : nullptr, ws.address, ws.bytes,
                       in.place.stream);
  Py_END_ALLOW_THREADS;
  check(status, "mbq_lora_group");
  return y.list.take();
}

// lora_backward(X, A, B, tokens, scale, dY, H, ranks, base, dX, dA, dB, ws)
PyObject* lora_backward_call(PyObject* const* args) {
  const LoraInputs in(args[0], args[1], args[2], args[3], args[4], args[7]);
  const Items dys(args[5]), hs(args[6]);
  assert_that(dys.size() == in.n && hs.size() == in.n, "one dY and H per projection");
  const void *dy[kMaxGroup], *h[kMaxGroup];
  for (Py_ssize_t i = 0; i < in.n; ++i) {
    dy[i] = in.place.of(dys[i], at::kFloat, {in.T, in.N[i]}, "dY");
    h[i] = in.place.of(hs[i], at::kFloat, {in.T, in.r}, "H");
  }
  const void* base = in.place.maybe(args[8], at::kFloat, {in.T, in.K}, "base");
  void* dx = nullptr;
  Owned dX(output(in.place, args[9], at::kFloat, {in.T, in.K}, "dX", &dx));
  Outputs da(in.place, args[10], in.n, at::kFloat, [&](Py_ssize_t) { return std::array<int64_t, 3>{in.adapters, in.r, in.K}; }, "dA");
  Outputs db(in.place, args[11], in.n, at::kFloat, [&](Py_ssize_t i) { return std::array<int64_t, 3>{in.adapters, in.r, in.N[i]}; },
             "dB");
  const Workspace ws(in.place, args[12],
                     args[12] == Py_None ? beside.lora_backward_bytes(in.T, in.K, (int)in.n, in.N, in.adapters, (int)in.r) : 0);
  int status;
  Py_BEGIN_ALLOW_THREADS;
  status = beside.lora_backward(in.x, in.T, in.K, (int)in.n, in.a, in.b, in.N, in.adapters, (int)in.r, in.ranks, in.scale,
                                in.token[0], in.token[1], in.token[2], dy, h, base, dx, da.address, db.address, ws.address, ws.bytes,
                                in.place.stream);
  Py_END_ALLOW_THREADS;
  check(status, "mbq_lora_backward_group");
  return PyTuple_Pack(3, dX.o, da.list.o, db.list.o);
}

void* mask_of(const Place& place, PyObject* o, int64_t T) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  assert_that(t.scalar_type() == at::kBool || t.scalar_type() == at::kByte, "mask must be bool or uint8");
  return place.of(t, t.scalar_type(), {T}, "mask");
}

// balance(logits, coef, mask, target, want_grad, out, ws)
PyObject* balance_call(PyObject* const* args) {
  const Items logits(args[0]);
  const Py_ssize_t n = group(logits.size());
  const at::Tensor& first = tensor(logits[0]);
  const Place place(first);
  assert_that(first.dim() == 2, "logits must be one matrix [T, P] per router");
  const int64_t T = first.size(0), P = first.size(1);
  const double coef = PyFloat_AsDouble(args[1]);
  if (coef == -1.0 && PyErr_Occurred()) throw PythonError{};
  const void* s[kMaxGroup];
  for (Py_ssize_t i = 0; i < n; ++i) s[i] = place.of(logits[i], at::kDouble, {T, P}, "logits");
  const void* mask = mask_of(place, args[2], T);
  double target[kMaxGroup] = {};
  if (args[3] != Py_None) {
    const Items items(args[3]);
    assert_that(items.size() == P && P <= kMaxGroup, "target must have one share per precision");
    for (int64_t e = 0; e < P; ++e) {
      target[e] = PyFloat_AsDouble(items[e]);
      if (target[e] == -1.0 && PyErr_Occurred()) throw PythonError{};
    }
  }
  const int want = PyObject_IsTrue(args[4]);
  if (want < 0) throw PythonError{};
  void *counts[kMaxGroup], *loss[kMaxGroup], *grad[kMaxGroup] = {};
  Owned list(PyList_New(n));
  Owned given(args[5] == Py_None ? PyTuple_New(0) : PySequence_Tuple(args[5]));
  assert_that(args[5] == Py_None || PyTuple_GET_SIZE(given.o) == n, "one (counts, loss, dlogits) per router");
  for (Py_ssize_t i = 0; i < n; ++i) {
    Owned of(args[5] == Py_None ? PyTuple_New(0) : PySequence_Tuple(PyTuple_GET_ITEM(given.o, i)));
    const bool has = args[5] != Py_None;
    assert_that(!has || PyTuple_GET_SIZE(of.o) == 3, "one (counts, loss, dlogits) per router");
    if (has) {
      assert_that(PyTuple_GET_ITEM(of.o, 0) != Py_None && PyTuple_GET_ITEM(of.o, 1) != Py_None &&
                      (!want || PyTuple_GET_ITEM(of.o, 2) != Py_None),
                  "one (counts, loss, dlogits) per router");
    }
    Owned c(output(place, has ? PyTuple_GET_ITEM(of.o, 0) : nullptr, at::kInt, {P}, "counts", &counts[i]));
    Owned l(output(place, has ? PyTuple_GET_ITEM(of.o, 1) : nullptr, at::kFloat, {1}, "loss", &loss[i]));
    if (want) {
      Owned d(output(place, has ? PyTuple_GET_ITEM(of.o, 2) : nullptr, at::kFloat, {T, P}, "dlogits", &grad[i]));
      PyList_SET_ITEM(list.o, i, Owned(PyTuple_Pack(3, c.o, l.o, d.o)).take());
    } else {
      PyList_SET_ITEM(list.o, i, Owned(PyTuple_Pack(3, c.o, l.o, has ? PyTuple_GET_ITEM(of.o, 2) : Py_None)).take());
    }
  }
  const Workspace ws(place, args[6], args[6] == Py_None ? beside.balance_bytes(T, (int)n) : 0);
  int status;
  Py_BEGIN_ALLOW_THREADS;
  status = beside.balance((int)n, s, T, (int)P, mask, args[3] != Py_None ? target : nullptr, coef, counts, loss,
                          want ? grad : nullptr, ws.address, ws.bytes, place.stream);
  Py_END_ALLOW_THREADS;
  check(status, "mbq_balance_loss_group");
  return list.take();
}

// route_backward(X, Wr, dlogits, mask, base, dX, dWr, dbr, ws)
PyObject* route_backward_call(PyObject* const* args) {
  const at::Tensor& X = tensor(args[0]);
  const Place place(X);
  const Items wr(args[1]), ds(args[2]);
  assert_that(X.dim() == 2 && wr.size() >= 1 && wr.size() == ds.size() && tensor(wr[0]).dim() == 2,
              "X must be a matrix, Wr and dlogits one matrix per router");
  const Py_ssize_t n = group(wr.size());
  const int64_t T = X.size(0), K = X.size(1), P = tensor(wr[0]).size(0);
  void* const x = place.of(X, at::kBFloat16, {T, K}, "X");
  const void *w[kMaxGroup], *d[kMaxGroup];
  for (Py_ssize_t i = 0; i < n; ++i) {
    w[i] = place.of(wr[i], at::kFloat, {P, K}, "Wr");
    d[i] = place.of(ds[i], at::kFloat, {T, P}, "dlogits");
  }
  const void* mask = mask_of(place, args[3], T);
  const void* base = place.maybe(args[4], at::kFloat, {T, K}, "base");
  void* dx = nullptr;
  Owned dX(output(place, args[5], at::kFloat, {T, K}, "dX", &dx));
  Outputs dw(place, args[6], n, at::kFloat, [&](Py_ssize_t) { return std::array<int64_t, 2>{P, K}; }, "dWr");
  Outputs db(place, args[7], n, at::kFloat, [&](Py_ssize_t) { return std::array<int64_t, 1>{P}; }, "dbr");
  const Workspace ws(place, args[8], args[8] == Py_None ? beside.route_backward_bytes(T, K, (int)n, (int)P) : 0);
  int status;
  Py_BEGIN_ALLOW_THREADS;
  status = beside.route_backward(x, T, K, (int)n, w, (int)P, d, mask, base, dx, dw.address, db.address, ws.address, ws.bytes,
                                 place.stream);
  Py_END_ALLOW_THREADS;
  check(status, "mbq_route_backward_group");
  return PyTuple_Pack(3, dX.o, dw.list.o, db.list.o);
}

template <PyObject* (*call)(PyObject* const*), int kArgs>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  try {
    if (!beside.lora) fail(PyExc_RuntimeError, "bind_beside() comes first");
    if (count != kArgs) fail(PyExc_TypeError, "wrong number of arguments");
    return call(args);
  } catch (const PythonError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
template <PyObject* (*call)(PyObject* const*), int kArgs>
PyCFunction fast() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<call, kArgs>));
}

// bind_beside(the calls and their workspace queries, in the order of Beside), after bind()
PyObject* bind_beside(PyObject*, PyObject* args) {
  Py_ssize_t a[8];
  if (!PyArg_ParseTuple(args, "nnnnnnnn", &a[0], &a[1], &a[2], &a[3], &a[4], &a[5], &a[6], &a[7])) return nullptr;
  beside.lora = reinterpret_cast<LoraFn>(a[0]);
  beside.lora_bytes = reinterpret_cast<decltype(beside.lora_bytes)>(a[1]);
  beside.lora_backward = reinterpret_cast<LoraBackwardFn>(a[2]);
  beside.lora_backward_bytes = reinterpret_cast<decltype(beside.lora_backward_bytes)>(a[3]);
  beside.balance = reinterpret_cast<BalanceFn>(a[4]);
  beside.balance_bytes = reinterpret_cast<decltype(beside.balance_bytes)>(a[5]);
  beside.route_backward = reinterpret_cast<RouteBackwardFn>(a[6]);
  beside.route_backward_bytes = reinterpret_cast<decltype(beside.route_backward_bytes)>(a[7]);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"stage", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(stage)), METH_FASTCALL, nullptr},
                         {"bind", bind, METH_VARARGS, nullptr},
                         {"lora", fast<lora_call, 10>(), METH_FASTCALL, nullptr},
                         {"lora_backward", fast<lora_backward_call, 13>(), METH_FASTCALL, nullptr},
                         {"balance", fast<balance_call, 7>(), METH_FASTCALL, nullptr},
                         {"route_backward", fast<route_backward_call, 9>(), METH_FASTCALL, nullptr},
                         {"bind_beside", bind_beside, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mbq_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mbq_torch(void) { return PyModule_Create(&module); }
