// What binding.py's entry points do per call, in native code: reads the arguments, allocates the outputs and the workspace with
// torch's allocator and calls the C ABI of umas.h.  The entry points themselves (names, defaults, errors, results) are
// binding.py's; a call here returns its outputs, or the status (an int) when the library refuses.
// In Python most of a small call went into this: 27 tensors at 1.3 us, a pointer at 0.5 to 1 us each, structs of pointers and the
// current stream (2.9 us): routing, advantages, KL, whitening and the ready batch of 40 000 tokens took 139 us to issue, 54 of them
// in the library.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/TensorOptions.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <initializer_list>
#include <vector>

#include "../../include/umas.h"

namespace {

struct Failed {};   // a Python error is set

// ------------------------------------------------------------------ arguments
[[noreturn]] void type_error(const char* what, PyObject* got) {
  PyErr_Format(PyExc_TypeError, "%s expected, got %s", what, Py_TYPE(got)->tp_name);
  throw Failed();
}
// anything with __index__ (Python's and numpy's integers), no floats; more bits than fit are cut off
int64_t integer(PyObject* o) {
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
  if (v == static_cast<unsigned long long>(-1) && PyErr_Occurred()) throw Failed();
  return static_cast<int64_t>(v);
}
int32_t integer32(PyObject* o) { return static_cast<int32_t>(integer(o)); }
int64_t as_int(PyObject* o) {                             // int(o)
  PyObject* n = PyNumber_Long(o);
  if (!n) throw Failed();
  const int64_t v = integer(n);
  Py_DECREF(n);
  return v;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Failed();
  return static_cast<float>(v);
}
int truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Failed();
  return v;
}
void* stream_of(PyObject* o) { return reinterpret_cast<void*>(static_cast<uintptr_t>(integer(o))); }

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) type_error("tensor", o);
  return THPVariable_Unpack(o);
}
template <class T>
T* ptr(const at::Tensor& t) { return static_cast<T*>(t.data_ptr()); }
template <class T>
T* ptr_or_null(PyObject* o) { return o == Py_None ? nullptr : ptr<T>(tensor(o)); }
// pointers of arrays that may be empty: an empty tensor has no storage, the ABI wants non-NULL pointers even for size 0
template <class T>
T* ptr_or(const at::Tensor& t, void* otherwise) {
  T* p = ptr<T>(t);
  return p ? p : static_cast<T*>(otherwise);
}
// A kernel gets addresses: an array in host memory would fault the GPU.  `dev` is where the call's first array lies (H, the mask, the streams); pinned host memory is in
// reach of a kernel as well.
void in_reach(const at::Tensor& t, const at::Device& dev, const char* name) {
  if (t.device() == dev || t.numel() == 0 || (t.is_cpu() && t.is_pinned())) return;
  PyErr_Format(PyExc_ValueError, "%s is not on the device of the other arrays", name);
  throw Failed();
}
struct Named {
  PyObject* o;                                            // a tensor or None
  const char* name;
};
void in_reach(std::initializer_list<Named> arrays, const at::Device& dev) {
  for (const Named& a : arrays)
    if (a.o != Py_None) in_reach(tensor(a.o), dev, a.name);
}
void on_gpu(const at::Device& dev) {
  if (dev.is_cuda()) return;
  PyErr_SetString(PyExc_ValueError, "H and what goes with it must be on a GPU");
  throw Failed();
}
// (H on the host goes with a workspace there; an empty one the library refuses itself, behind its own checks)
void on_gpu(const at::Tensor& ws, const at::Device& dev) {
  in_reach(ws, dev, "workspace");
  if (ws.numel() != 0) on_gpu(ws.device());
}
// Bytes of a workspace that the binding has made: none on the host, so that the library, whose checks of the call's host arrays come first, refuses.
size_t bytes_of(const at::Tensor& ws) { return ws.is_cuda() ? static_cast<size_t>(ws.numel()) : 0; }
int dtype_code(PyObject* o) {
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() == at::kFloat) return UMAS_F32;
  if (t.scalar_type() == at::kBFloat16) return UMAS_BF16;
  PyObject* dt = PyObject_GetAttrString(o, "dtype");
  if (dt) PyErr_Format(PyExc_TypeError, "unsupported dtype %S", dt);
  Py_XDECREF(dt);
  throw Failed();
}
struct Rows {                                             // [n, d] hidden states
  const at::Tensor& t;
  int dt;
  int64_t n;
  int32_t d;
  explicit Rows(PyObject* o) : t(tensor(o)) {
    if (t.dim() != 2) {
      PyErr_Format(PyExc_ValueError, "H must have two dimensions, not %d", static_cast<int>(t.dim()));
      throw Failed();
    }
    n = t.size(0);
    d = static_cast<int32_t>(t.size(1));
    dt = dtype_code(o);
  }
};
struct Selection {                                        // None: all rows; an empty one still needs a pointer
  const int32_t* p = nullptr;
  int64_t n;
  Selection(PyObject* o, int64_t all, void* otherwise = nullptr) : n(all) {
    if (o == Py_None) return;
    const at::Tensor& t = tensor(o);
    n = t.numel();
    p = ptr_or<const int32_t>(t, otherwise);
  }
  void point(void* otherwise, PyObject* o) { if (o != Py_None && !p) p = static_cast<const int32_t*>(otherwise); }
};

// The calls that list logits and teach targets read and write [n, k] arrays: types, shapes, layout and device are looked at here, where a wrong one would be read
// out of bounds.
void same_head(const Rows& H, const at::Tensor& W) {
  in_reach(W, H.t.device(), "W");
  if (W.dim() == 2 && W.size(1) == H.d && W.scalar_type() == H.t.scalar_type() && H.t.is_contiguous() && W.is_contiguous()) return;
  PyErr_SetString(PyExc_ValueError, "H [n, d] and W [V, d] must be contiguous and of one type and width");
  throw Failed();
}
const at::Tensor& targets(PyObject* o, at::ScalarType type, int64_t n, int64_t k, const at::Device& dev, const char* name) {
  const at::Tensor& t = tensor(o);
  in_reach(t, dev, name);
  if (t.scalar_type() != type) {
    PyErr_Format(PyExc_TypeError, "%s must be %s", name, type == at::kInt ? "int32" : "float32");
    throw Failed();
  }
  if (t.numel() != n * k || t.dim() == 0 || t.size(0) != n || !t.is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s must be contiguous and hold %lld values for each of the %lld rows of H", name, static_cast<long long>(k), static_cast<long long>(n));
    throw Failed();
  }
  return t;
}

PyObject* ascontiguousarray = nullptr;                    // numpy's
// A host array of the ABI's type: the object's own memory where it has that type, is contiguous and lies at a multiple of the type's
// size, else numpy's copy.
struct HostArray {
  Py_buffer view{};
  bool held = false;
  int64_t len = 0;                                        // of the first dimension
  HostArray() = default;
  HostArray(const HostArray&) = delete;
  ~HostArray() { if (held) PyBuffer_Release(&view); }
  void get(PyObject* o, char kind, int size, const char* np_type) {
    if (o == Py_None) return;
    if (PyBytes_Check(o) || !(PyObject_CheckBuffer(o) && take(o, kind, size))) {   // bytes: text to numpy
      PyErr_Clear();
      PyObject* a = PyObject_CallFunction(ascontiguousarray, "Os", o, np_type);
      if (!a) throw Failed();
      bool ok = take(a, kind, size);                      // the view holds the array
      if (!ok) {                                          // the right type and contiguous, but not aligned
        PyErr_Clear();
        PyObject* const c = PyObject_CallMethod(a, "copy", nullptr);
        Py_DECREF(a);
        if (!(a = c)) throw Failed();
        ok = take(a, kind, size);
      }
      Py_DECREF(a);
      if (!ok) {
        if (!PyErr_Occurred()) PyErr_Format(PyExc_TypeError, "array of %s expected", np_type);
        throw Failed();
      }
    }
    len = view.ndim > 0 ? view.shape[0] : 1;                // a single number: one entry
  }
  template <class T>
  const T* as() const { return held ? static_cast<const T*>(view.buf) : nullptr; }

 private:
  bool take(PyObject* o, char kind, int size) {           // kind: i(nteger), u(nsigned), f(loat)
    if (PyObject_GetBuffer(o, &view, PyBUF_FORMAT | PyBUF_C_CONTIGUOUS) != 0) return false;
    const char* f = view.format;
    bool ok = f && f[0] && !f[1] && view.itemsize == size && reinterpret_cast<uintptr_t>(view.buf) % size == 0;
    if (ok) ok = kind == 'i' ? f[0] == 'i' || f[0] == 'l' || f[0] == 'q' : kind == 'u' ? f[0] == 'B' : f[0] == 'f';
    if (!ok) PyBuffer_Release(&view);
    held = ok;
    return ok;
  }
};
#define I32_ARRAY(name, obj) HostArray name; name.get(obj, 'i', 4, "int32")
#define I64_ARRAY(name, obj) HostArray name; name.get(obj, 'i', 8, "int64")
#define F32_ARRAY(name, obj) HostArray name; name.get(obj, 'f', 4, "float32")
#define U8_ARRAY(name, obj) HostArray name; name.get(obj, 'u', 1, "uint8")

// ------------------------------------------------------------------ outputs
at::Tensor fresh(at::IntArrayRef size, at::ScalarType type, const at::Device& dev) {
  return at::empty(size, at::TensorOptions().dtype(type).device(dev));
}
at::Tensor workspace(size_t bytes, const at::Device& dev) {
  return fresh({static_cast<int64_t>(std::max<size_t>(bytes, 256))}, at::kByte, dev);
}
struct Output {                                           // what the caller passed, or a new tensor
  at::Tensor t;
  PyObject* given;
  template <class Make>
  Output(PyObject* o, Make make) : given(o == Py_None ? nullptr : o) { t = given ? tensor(o) : make(); }
  PyObject* object() const {
    if (!given) return THPVariable_Wrap(t);
    Py_INCREF(given);
    return given;
  }
};
PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* pack(std::initializer_list<PyObject*> items) {  // takes the references
  bool ok = true;
  for (PyObject* o : items) ok = ok && o;
  PyObject* r = ok ? PyTuple_New(static_cast<Py_ssize_t>(items.size())) : nullptr;
  if (!r) {
    for (PyObject* o : items) Py_XDECREF(o);
    return nullptr;
  }
  Py_ssize_t i = 0;
  for (PyObject* o : items) PyTuple_SET_ITEM(r, i++, o);
  return r;
}
struct Unlocked {                                         // the interpreter lock is taken again also when the call throws
  PyThreadState* const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <class Call>
umas_status unlocked(Call call) {                         // the library needs no Python
  const Unlocked without_lock;
  return call();
}
#define UMAS_CALL(...)                                                        \
  do {                                                                        \
    const umas_status s__ = unlocked([&] { return __VA_ARGS__; });            \
    if (s__ != UMAS_OK) return PyLong_FromLong(static_cast<long>(s__));       \
  } while (0)

constexpr int kStreamTensors = 16;
const char* const kStreamNames[kStreamTensors] = {"model_tok_off", "perm", "tok_turn", "tok_role", "tok_mask", "tok_reward", "turn_seg_off",
                                                  "seg_turn", "model_turn_off", "traj_seg_off", "model_trajrun_off", "rowsel",
                                                  "model_rowsel_off", "turn_scalar", "turn_step", "tok_flags"};
static_assert(sizeof(umas_streams) == kStreamTensors * sizeof(void*), "one pointer per name");
PyObject* g_stream_names[kStreamTensors];
PyObject *g_n_tokens, *g_n_turns, *g_n_models;

struct Ref {                                              // an owned reference
  PyObject* o;
  explicit Ref(PyObject* p) : o(p) { if (!p) throw Failed(); }
  Ref(const Ref&) = delete;
  ~Ref() { Py_DECREF(o); }
};
// the ABI's struct of a Streams object; the object keeps its tensors
umas_streams streams_of(PyObject* o, const at::Device& dev, void* otherwise) {
  umas_streams s;
  void** p = reinterpret_cast<void**>(&s);
  for (int i = 0; i < kStreamTensors; ++i) {
    const Ref t(PyObject_GetAttr(o, g_stream_names[i]));
    in_reach(tensor(t.o), dev, kStreamNames[i]);
    p[i] = ptr_or<void>(tensor(t.o), otherwise);
  }
  return s;
}
int64_t int_attr(PyObject* o, PyObject* name) { const Ref v(PyObject_GetAttr(o, name)); return integer(v.o); }
at::Device device_of(PyObject* streams, int field) { const Ref t(PyObject_GetAttr(streams, g_stream_names[field])); return tensor(t.o).device(); }
constexpr int kTokReward = 5, kRowsel = 11;

// ------------------------------------------------------------------ entry points
PyObject* assign(PyObject* const* a) {
  umas_graph g;
  umas_rewards r;
  g.n_roles = integer32(a[0]);
  g.n_models = integer32(a[1]);
  for (int i : {3, 5})                                    // offsets have a length
    if (a[i] != Py_None && PyObject_Size(a[i]) < 0) throw Failed();
  I32_ARRAY(role_to_model, a[2]);
  I32_ARRAY(traj_turn_off, a[3]);
  I32_ARRAY(turn_role, a[4]);
  I64_ARRAY(turn_tok_off, a[5]);
  const at::Tensor& mask = tensor(a[6]);
  I32_ARRAY(turn_pred_off, a[7]);
  I32_ARRAY(turn_pred, a[8]);
  I32_ARRAY(traj_group, a[9]);
  F32_ARRAY(role_reward, a[10]);
  F32_ARRAY(turn_reward, a[11]);
  F32_ARRAY(traj_reward, a[12]);
  F32_ARRAY(w_role, a[13]);
  F32_ARRAY(w_turn, a[14]);
  F32_ARRAY(w_traj, a[15]);
  r.place_mode = integer32(a[16]);
  r.norm_eps = real(a[17]);
  void* const st = stream_of(a[18]);
  const int64_t N = mask.numel(), U = turn_tok_off.len - 1, M = g.n_models;
  g.n_traj = static_cast<int32_t>(traj_turn_off.len - 1);
  g.n_turns = static_cast<int32_t>(U);
  g.n_tokens = N;
  g.role_to_model = role_to_model.as<int32_t>();
  g.traj_turn_off = traj_turn_off.as<int32_t>();
  g.turn_role = turn_role.as<int32_t>();
  g.turn_tok_off = turn_tok_off.as<int64_t>();
  g.turn_pred_off = turn_pred_off.as<int32_t>();
  g.turn_pred = turn_pred.as<int32_t>();
  g.traj_group = traj_group.as<int32_t>();
  r.role_reward = role_reward.as<float>();
  r.turn_reward = turn_reward.as<float>();
  r.traj_reward = traj_reward.as<float>();
  r.w_role = w_role.as<float>();
  r.w_turn = w_turn.as<float>();
  r.w_traj = w_traj.as<float>();
  const at::Device dev = mask.device();
  const int64_t U1 = std::max<int64_t>(U, 1), N1 = std::max<int64_t>(N, 1);
  const auto i64 = at::kLong, i32 = at::kInt, f32 = at::kFloat, u8 = at::kByte;
  const at::Tensor out[kStreamTensors] = {
      fresh({M + 1}, i64, dev), fresh({N}, i64, dev), fresh({N}, i32, dev), fresh({N}, i32, dev), fresh({N}, u8, dev), fresh({N}, f32, dev),
      fresh({U + 1}, i64, dev), fresh({U1}, i32, dev), fresh({M + 1}, i32, dev), fresh({U + 1}, i64, dev), fresh({M + 1}, i32, dev),
      fresh({N1}, i32, dev), fresh({M + 1}, i64, dev), fresh({U1}, f32, dev), fresh({U1}, i32, dev), fresh({N}, u8, dev)};
  const at::Tensor ws = workspace(umas_assign_workspace_bytes(&g), dev);
  umas_streams s;
  for (int i = 0; i < kStreamTensors; ++i) reinterpret_cast<void**>(&s)[i] = ptr_or<void>(out[i], ws.data_ptr());
  UMAS_CALL(umas_assign_token_rewards(&g, &r, ptr_or<uint8_t>(mask, ws.data_ptr()), &s, ws.data_ptr(), bytes_of(ws), st));
  PyObject* res = PyTuple_New(3 + kStreamTensors);
  if (!res) return nullptr;
  PyTuple_SET_ITEM(res, 0, PyLong_FromLongLong(N));
  PyTuple_SET_ITEM(res, 1, PyLong_FromLongLong(U));
  PyTuple_SET_ITEM(res, 2, PyLong_FromLongLong(M));
  for (int i = 0; i < kStreamTensors; ++i) PyTuple_SET_ITEM(res, 3 + i, wrap(out[i]));
  return res;
}

PyObject* advantages(PyObject* const* a) {                // streams, value, gamma, lam, gamma_turn, seg_mode, stream
  const at::Device dev = device_of(a[0], kTokReward);
  const int64_t N = int_attr(a[0], g_n_tokens);
  const int32_t U = static_cast<int32_t>(int_attr(a[0], g_n_turns));
  const float gamma = real(a[2]), lam = real(a[3]), gamma_turn = real(a[4]);
  const int32_t seg = integer32(a[5]);
  const at::Tensor adv = fresh({N}, at::kFloat, dev), ret = fresh({N}, at::kFloat, dev), ws = workspace(umas_advantages_workspace_bytes(N), dev);
  const umas_streams s = streams_of(a[0], dev, ws.data_ptr());
  in_reach({{a[1], "value"}}, dev);
  const float* value = ptr_or_null<const float>(a[1]);
  void* const st = stream_of(a[6]);
  UMAS_CALL(umas_advantages(&s, N, U, value, gamma, lam, gamma_turn, seg, ptr<float>(adv), ptr<float>(ret), ws.data_ptr(), bytes_of(ws), st));
  return pack({wrap(adv), wrap(ret)});
}

PyObject* policy_logprobs(PyObject* const* a) {           // H, W, ids, rowsel, want_entropy, workspace, stream
  const Rows H(a[0]);
  const at::Tensor &W = tensor(a[1]), &ids = tensor(a[2]);
  const int32_t V = static_cast<int32_t>(W.size(0));
  Selection sel(a[3], H.n);
  const at::Device dev = H.t.device();
  on_gpu(dev);
  in_reach({{a[1], "W"}, {a[2], "ids"}, {a[3], "rowsel"}, {a[5], "workspace"}}, dev);
  const at::Tensor logp = fresh({H.n}, at::kFloat, dev), lse = fresh({H.n}, at::kFloat, dev);
  const bool want = truth(a[4]);
  const at::Tensor entropy = want ? fresh({H.n}, at::kFloat, dev) : at::Tensor();
  const umas_dtype dt = static_cast<umas_dtype>(H.dt);
  const Output ws(a[5], [&] { return workspace(umas_policy_logprobs_workspace_bytes(sel.n, H.d, V, dt), dev); });
  sel.point(ws.t.data_ptr(), a[3]);
  void* const st = stream_of(a[6]);
  float* const e = want ? ptr<float>(entropy) : nullptr;
  UMAS_CALL(umas_policy_logprobs(H.t.data_ptr(), W.data_ptr(), dt, H.n, H.d, V, ptr<int32_t>(ids), sel.p, sel.n, ptr<float>(logp), ptr<float>(lse), e,
                                 ws.t.data_ptr(), ws.t.numel(), st));
  if (!want) Py_INCREF(Py_None);
  return pack({wrap(logp), wrap(lse), want ? wrap(entropy) : Py_None});
}

PyObject* policy_logprobs_static(PyObject* const* a) {    // H, W, ids, rowsel, logp, lse, entropy, stream
  const Rows H(a[0]);
  const at::Tensor &W = tensor(a[1]), &ids = tensor(a[2]);
  const at::Device dev = H.t.device();
  on_gpu(dev);
  in_reach({{a[1], "W"}, {a[2], "ids"}, {a[3], "rowsel"}, {a[4], "logp"}, {a[5], "lse"}, {a[6], "entropy"}}, dev);
  auto row = [&] { return fresh({H.n}, at::kFloat, dev); };
  const Output logp(a[4], row), lse(a[5], row), entropy(a[6], row);
  Selection sel(a[3], H.n);
  sel.point(W.data_ptr(), a[3]);
  void* const st = stream_of(a[7]);
  UMAS_CALL(umas_policy_logprobs_static(H.t.data_ptr(), W.data_ptr(), static_cast<umas_dtype>(H.dt), H.n, H.d, static_cast<int32_t>(W.size(0)),
                                        ptr<int32_t>(ids), sel.p, sel.n, ptr<float>(logp.t), ptr<float>(lse.t), ptr<float>(entropy.t), st));
  return pack({logp.object(), lse.object(), entropy.object()});
}

PyObject* ppo_loss(PyObject* const* a) {
  // H, W, ids, rowsel, logp_old, adv, tok_role, n_roles, clip_eps, entropy_coef, dual_clip, accumulate_dW, norm_rows, logp_ref, kl_coef,
  // dW, dH, logp_new, stats, workspace, stream
  const Rows H(a[0]);
  const at::Tensor &W = tensor(a[1]), &ids = tensor(a[2]), &adv = tensor(a[5]);
  const int32_t V = static_cast<int32_t>(W.size(0)), n_roles = integer32(a[7]);
  Selection sel(a[3], H.n);
  const at::Device dev = H.t.device();
  on_gpu(dev);
  in_reach({{a[1], "W"}, {a[2], "ids"}, {a[3], "rowsel"}, {a[4], "logp_old"}, {a[5], "adv"}, {a[6], "tok_role"}, {a[13], "logp_ref"}, {a[15], "dW"}, {a[16], "dH"},
            {a[17], "logp_new"}, {a[18], "stats"}, {a[19], "workspace"}}, dev);
  const umas_dtype dt = static_cast<umas_dtype>(H.dt);
  const Output dW(a[15], [&] { return fresh({W.size(0), H.d}, at::kFloat, dev); });
  const Output dH(a[16], [&] { return at::empty_like(H.t); });
  const Output logp_new(a[17], [&] { return fresh({H.n}, at::kFloat, dev); });
  const Output stats(a[18], [&] { return fresh({(1 + static_cast<int64_t>(n_roles)) * static_cast<int64_t>(sizeof(umas_loss_stats))}, at::kByte, dev); });
  const float clip_eps = real(a[8]), entropy_coef = real(a[9]), dual_clip = real(a[10]), kl_coef = real(a[14]);
  const Output ws(a[19], [&] {
    const auto bytes = entropy_coef > 0.f ? umas_ppo_loss_workspace_bytes_entropy : umas_ppo_loss_workspace_bytes;
    return workspace(bytes(sel.n, H.d, V, dt, n_roles), dev);
  });
  sel.point(ws.t.data_ptr(), a[3]);
  const float* const logp_old = ptr_or_null<const float>(a[4]);
  const int32_t* const role = ptr_or_null<const int32_t>(a[6]);
  const int32_t accumulate = truth(a[11]);
  const int64_t norm_rows = as_int(a[12]);
  const float* const logp_ref = ptr_or_null<const float>(a[13]);
  void* const st = stream_of(a[20]);
  UMAS_CALL(umas_ppo_loss_fwd_bwd(H.t.data_ptr(), W.data_ptr(), dt, H.n, H.d, V, ptr<int32_t>(ids), sel.p, sel.n, logp_old, ptr<float>(adv), role,
                                  n_roles, clip_eps, entropy_coef, dual_clip, accumulate, norm_rows, logp_ref, kl_coef,
                                  ptr<umas_loss_stats>(stats.t), ptr<float>(logp_new.t), dH.t.data_ptr(), ptr<float>(dW.t), ws.t.data_ptr(),
                                  ws.t.numel(), st));
  return pack({stats.object(), logp_new.object(), dH.object(), dW.object()});
}

// (the checks of the two calls below and their kin, see same_head)
const at::Tensor* targets_or_null(PyObject* o, at::ScalarType type, int64_t n, const at::Device& dev, const char* name) {
  return o == Py_None ? nullptr : &targets(o, type, n, 1, dev, name);
}
void whole_selection(PyObject* o, const at::Device& dev) {
  if (o == Py_None) return;
  const at::Tensor& t = tensor(o);
  in_reach(t, dev, "rowsel");
  if (t.scalar_type() == at::kInt && t.is_contiguous()) return;
  PyErr_SetString(PyExc_TypeError, "rowsel must be contiguous and int32");
  throw Failed();
}
void room(const Output& out, at::ScalarType type, int64_t n, const at::Device& dev, const char* name) {
  in_reach(out.t, dev, name);
  if (!out.given || (out.t.scalar_type() == type && out.t.numel() == n && out.t.is_contiguous())) return;
  PyErr_Format(PyExc_ValueError, "%s must be contiguous, %s and hold %lld values", name, c10::toString(type), static_cast<long long>(n));
  throw Failed();
}

PyObject* top_logits(PyObject* const* a) {                // H, W, k, rowsel, ids, logits, lse, workspace, stream
  const Rows H(a[0]);
  const at::Tensor& W = tensor(a[1]);
  const int32_t V = static_cast<int32_t>(W.size(0)), k = integer32(a[2]);
  Selection sel(a[3], H.n);
  const at::Device dev = H.t.device();
  const umas_dtype dt = static_cast<umas_dtype>(H.dt);
  const int64_t places = std::max(k, 0);
  const Output ids(a[4], [&] { return fresh({H.n, places}, at::kInt, dev); });
  const Output logits(a[5], [&] { return fresh({H.n, places}, at::kFloat, dev); });
  const Output lse(a[6], [&] { return fresh({H.n}, at::kFloat, dev); });
  const Output ws(a[7], [&] { return workspace(umas_top_logits_workspace_bytes(sel.n, H.d, V, k, dt), dev); });
  sel.point(ws.t.data_ptr(), a[3]);
  void* const st = stream_of(a[8]);
  same_head(H, W);
  whole_selection(a[3], dev);
  room(ids, at::kInt, H.n * places, dev, "ids");
  room(logits, at::kFloat, H.n * places, dev, "logits");
  room(lse, at::kFloat, H.n, dev, "lse");
  on_gpu(ws.t, dev);
  UMAS_CALL(umas_top_logits(H.t.data_ptr(), W.data_ptr(), dt, H.n, H.d, V, sel.p, sel.n, k, ptr<int32_t>(ids.t), ptr<float>(logits.t), ptr<float>(lse.t),
                            ws.t.data_ptr(), ws.t.numel(), st));
  return pack({ids.object(), logits.object(), lse.object()});
}

// What cross entropy and distillation have in common; `o` from weight on: weight, tok_role, n_roles, train_head, accumulate_dW, norm_rows, dW, dH, row_out,
// stats, workspace, stream.
struct Taught {
  const Rows H;
  const at::Tensor& W;
  const int32_t V;
  Selection sel;
  const at::Device dev;
  const umas_dtype dt;
  const float* weight;
  const int32_t *role, n_roles;
  const bool head;
  const int32_t accumulate;
  const int64_t norm_rows;
  at::Tensor dW;
  PyObject* dW_given;
  const Output dH, row_out, stats;
  int32_t dW_type;
  void* const st;
  Taught(PyObject* h, PyObject* w, PyObject* rowsel, PyObject* const* o)
      : H(h), W(tensor(w)), V(static_cast<int32_t>(W.size(0))), sel(rowsel, H.n), dev(H.t.device()), dt(static_cast<umas_dtype>(H.dt)),
        weight(ptr_or_null<const float>(o[0])), role(ptr_or_null<const int32_t>(o[1])), n_roles(integer32(o[2])), head(truth(o[3])), accumulate(truth(o[4])),
        norm_rows(as_int(o[5])), dW_given(o[6] == Py_None ? nullptr : o[6]), dH(o[7], [&] { return at::empty_like(H.t); }),
        row_out(o[8], [&] { return fresh({H.n}, at::kFloat, dev); }),
        stats(o[9], [&] { return fresh({(1 + static_cast<int64_t>(std::max(n_roles, 0))) * static_cast<int64_t>(sizeof(umas_target_stats))}, at::kByte, dev); }),
        dW_type(UMAS_NO_DW), st(stream_of(o[11])) {
    same_head(H, W);
    whole_selection(rowsel, dev);
    targets_or_null(o[0], at::kFloat, H.n, dev, "weight");
    targets_or_null(o[1], at::kInt, H.n, dev, "tok_role");
    room(dH, H.t.scalar_type(), H.t.numel(), dev, "dH");
    room(row_out, at::kFloat, H.n, dev, "the output of every row");
    room(stats, at::kByte, (1 + static_cast<int64_t>(std::max(n_roles, 0))) * static_cast<int64_t>(sizeof(umas_target_stats)), dev, "stats");
    if (head && accumulate && !dW_given) {
      PyErr_SetString(PyExc_ValueError, "accumulate_dW needs the dW to add to");
      throw Failed();
    }
    if (!head) return;
    dW = dW_given ? tensor(dW_given) : at::empty_like(W);
    in_reach(dW, dev, "dW");
    if (dW.scalar_type() != at::kFloat && dW.scalar_type() != W.scalar_type()) {
      PyErr_SetString(PyExc_TypeError, "dW must be float32 or of the type of W");
      throw Failed();
    }
    if (dW.numel() != W.numel() || !dW.is_contiguous()) {
      PyErr_SetString(PyExc_ValueError, "dW must be contiguous and of the shape of W");
      throw Failed();
    }
    dW_type = dW.scalar_type() == at::kFloat ? UMAS_F32 : UMAS_BF16;
  }
  PyObject* results() const {
    PyObject* w = Py_None;
    if (head && !dW_given) w = wrap(dW);
    else {
      if (head) w = dW_given;
      Py_INCREF(w);
    }
    return pack({stats.object(), row_out.object(), dH.object(), w});
  }
};

PyObject* cross_entropy(PyObject* const* a) {
  // H, W, ids, rowsel, z_coef, weight, tok_role, n_roles, train_head, accumulate_dW, norm_rows, dW, dH, logp, stats, workspace, stream
  Taught T(a[0], a[1], a[3], a + 5);
  const at::Tensor& ids = targets(a[2], at::kInt, T.H.n, 1, T.dev, "ids");
  const float z_coef = real(a[4]);
  const Output ws(a[15], [&] { return workspace(umas_cross_entropy_workspace_bytes(T.sel.n, T.H.d, T.V, T.dt, T.dW_type), T.dev); });
  on_gpu(ws.t, T.dev);
  T.sel.point(ws.t.data_ptr(), a[3]);
  UMAS_CALL(umas_cross_entropy_fwd_bwd(T.H.t.data_ptr(), T.W.data_ptr(), T.dt, T.H.n, T.H.d, T.V, ptr<int32_t>(ids), T.sel.p, T.sel.n, T.weight, T.role,
                                       T.n_roles, z_coef, T.accumulate, T.norm_rows, ptr<umas_target_stats>(T.stats.t), ptr<float>(T.row_out.t),
                                       T.dH.t.data_ptr(), T.head ? T.dW.data_ptr() : nullptr, T.dW_type, ws.t.data_ptr(), ws.t.numel(), T.st));
  return T.results();
}

PyObject* distill(PyObject* const* a) {
  // H, W, top_ids, top_logits, teacher_lse, rowsel, weight, tok_role, n_roles, train_head, accumulate_dW, norm_rows, dW, dH, kl, stats, workspace, stream
  Taught T(a[0], a[1], a[5], a + 6);
  const int64_t k = tensor(a[2]).dim() == 2 ? tensor(a[2]).size(1) : 0;
  const at::Tensor &ids = targets(a[2], at::kInt, T.H.n, k, T.dev, "top_ids"), &logits = targets(a[3], at::kFloat, T.H.n, k, T.dev, "top_logits");
  const float* const lse = a[4] == Py_None ? nullptr : ptr<const float>(targets(a[4], at::kFloat, T.H.n, 1, T.dev, "teacher_lse"));
  const int32_t places = static_cast<int32_t>(std::min<int64_t>(k, 1 << 30));
  const Output ws(a[16], [&] { return workspace(umas_distill_workspace_bytes(T.sel.n, T.H.d, T.V, places, T.dt, T.dW_type), T.dev); });
  on_gpu(ws.t, T.dev);
  T.sel.point(ws.t.data_ptr(), a[5]);
  UMAS_CALL(umas_distill_fwd_bwd(T.H.t.data_ptr(), T.W.data_ptr(), T.dt, T.H.n, T.H.d, T.V, ptr<int32_t>(ids), ptr<float>(logits), places, lse, T.sel.p,
                                 T.sel.n, T.weight, T.role, T.n_roles, T.accumulate, T.norm_rows, ptr<umas_target_stats>(T.stats.t), ptr<float>(T.row_out.t),
                                 T.dH.t.data_ptr(), T.head ? T.dW.data_ptr() : nullptr, T.dW_type, ws.t.data_ptr(), ws.t.numel(), T.st));
  return T.results();
}

// ------------------------------------------------------------------ around a head
// An array that a call reads or writes: its type, length, layout and device are looked at before any address is taken.
const at::Tensor& whole(const at::Tensor& t, at::ScalarType type, int64_t n, const at::Device& dev, const char* name) {
  in_reach(t, dev, name);
  if (t.scalar_type() == type && t.numel() == n && t.is_contiguous()) return t;
  PyErr_Format(PyExc_ValueError, "%s must be contiguous, %s and hold %lld values", name, c10::toString(type), static_cast<long long>(n));
  throw Failed();
}
const at::Tensor& whole(PyObject* o, at::ScalarType type, int64_t n, const at::Device& dev, const char* name) { return whole(tensor(o), type, n, dev, name); }
void* whole_or_null(PyObject* o, at::ScalarType type, int64_t n, const at::Device& dev, const char* name) {
  return o == Py_None ? nullptr : whole(o, type, n, dev, name).data_ptr();
}
void on_a_gpu(const at::Tensor& t, const char* name) {     // the one that the launches go to: their stream is of the current device
  if (t.is_cuda() && t.device() == c10::impl::getDeviceGuardImpl(at::kCUDA)->getDevice()) return;
  PyErr_Format(PyExc_ValueError, t.is_cuda() ? "%s and what goes with it must be on the current GPU" : "%s and what goes with it must be on a GPU", name);
  throw Failed();
}
void same_address(const char* a, const at::Tensor& x, const char* b, const at::Tensor& y) {   // two outputs of a call
  if (x.data_ptr() != y.data_ptr() || x.numel() == 0) return;
  PyErr_Format(PyExc_ValueError, "%s and %s must be different arrays", a, b);
  throw Failed();
}
// x, gain, residual, eps, hidden, then the output (y, or q and scale), inv_rms, stream
template <bool QUANT>
PyObject* norm(PyObject* const* a) {
  const Rows x(a[0]);
  const at::Device dev = x.t.device();
  const at::ScalarType type = x.t.scalar_type(), out_type = QUANT ? at::kFloat8_e4m3fn : type;
  const at::Tensor& gain = whole(a[1], type, x.d, dev, "gain");
  whole(x.t, type, x.n * x.d, dev, "x");
  const bool sum = a[2] != Py_None;
  void* const residual = whole_or_null(a[2], type, x.n * x.d, dev, "residual");
  const float eps = real(a[3]);
  if (!sum && a[4] != Py_None) {
    PyErr_SetString(PyExc_ValueError, "hidden is x itself where there is no residual");
    throw Failed();
  }
  PyObject* const* const o = a + 5;                        // the output
  const Output hidden(a[4], [&] { return sum ? at::empty_like(x.t) : at::Tensor(); });
  const Output y(o[0], [&] { return fresh({x.n, x.d}, out_type, dev); });
  const Output scale(QUANT ? o[1] : Py_None, [&] { return QUANT ? fresh({x.n}, at::kFloat, dev) : at::Tensor(); });
  const Output inv_rms(o[QUANT ? 2 : 1], [&] { return fresh({x.n}, at::kFloat, dev); });
  if (sum) whole(hidden.t, type, x.n * x.d, dev, "hidden");
  whole(y.t, out_type, x.n * x.d, dev, QUANT ? "q" : "y");
  whole(inv_rms.t, at::kFloat, x.n, dev, "inv_rms");
  if (sum) same_address("hidden", hidden.t, "the output", y.t);
  if constexpr (QUANT) whole(scale.t, at::kFloat, x.n, dev, "scale");
  on_a_gpu(x.t, "x");
  void* const st = stream_of(o[QUANT ? 3 : 2]);
  const umas_dtype dt = static_cast<umas_dtype>(x.dt);
  void* const h = sum ? hidden.t.data_ptr() : nullptr;
  if constexpr (QUANT) {
    UMAS_CALL(umas_rms_norm_quantized(x.t.data_ptr(), residual, gain.data_ptr(), dt, x.n, x.d, eps, h, static_cast<uint8_t*>(y.t.data_ptr()), ptr<float>(scale.t),
                                      ptr<float>(inv_rms.t), st));
  } else {
    UMAS_CALL(umas_rms_norm(x.t.data_ptr(), residual, gain.data_ptr(), dt, x.n, x.d, eps, h, y.t.data_ptr(), ptr<float>(inv_rms.t), st));
  }
  PyObject* same = nullptr;
  if (!sum) Py_INCREF(same = a[0]);
  if constexpr (QUANT) return pack({y.object(), scale.object(), sum ? hidden.object() : same, inv_rms.object()});
  else return pack({y.object(), sum ? hidden.object() : same, inv_rms.object()});
}
PyObject* rms_norm(PyObject* const* a) { return norm<false>(a); }
PyObject* rms_norm_quantized(PyObject* const* a) { return norm<true>(a); }

PyObject* rms_norm_bwd(PyObject* const* a) {              // dy, hidden, gain, inv_rms, dhidden, accumulate_dgain, dx, dgain, workspace, stream
  const Rows dy(a[0]);
  const at::Device dev = dy.t.device();
  const at::ScalarType type = dy.t.scalar_type();
  const int64_t all = dy.n * dy.d;
  whole(dy.t, type, all, dev, "dy");
  const at::Tensor &hidden = whole(a[1], type, all, dev, "hidden"), &gain = whole(a[2], type, dy.d, dev, "gain"), &inv_rms = whole(a[3], at::kFloat, dy.n, dev, "inv_rms");
  void* const dhidden = whole_or_null(a[4], type, all, dev, "dhidden");
  const int32_t accumulate = truth(a[5]);
  if (accumulate && a[7] == Py_None) {
    PyErr_SetString(PyExc_ValueError, "accumulate_dgain needs the dgain to add to");
    throw Failed();
  }
  const Output dx(a[6], [&] { return at::empty_like(dy.t); });
  const Output dgain(a[7], [&] { return fresh({dy.d}, at::kFloat, dev); });
  const Output ws(a[8], [&] { return workspace(umas_rms_norm_workspace_bytes(dy.n, dy.d), dev); });
  whole(dx.t, type, all, dev, "dx");
  whole(dgain.t, at::kFloat, dy.d, dev, "dgain");
  in_reach(ws.t, dev, "workspace");
  on_a_gpu(dy.t, "dy");
  void* const st = stream_of(a[9]);
  UMAS_CALL(umas_rms_norm_bwd(dy.t.data_ptr(), hidden.data_ptr(), gain.data_ptr(), ptr<float>(inv_rms), dhidden, static_cast<umas_dtype>(dy.dt), dy.n, dy.d, accumulate,
                              dx.t.data_ptr(), ptr<float>(dgain.t), ws.t.data_ptr(), ws.t.nbytes(), st));
  return pack({dx.object(), dgain.object()});
}

// temperature, top_k, top_p, min_p: each a number or a tensor with one for each of n rows
umas_sampling sampling_of(PyObject* const* a, int64_t n, const at::Device& dev) {
  umas_sampling s{1.0, 1.0, 0.0, 0, nullptr, nullptr, nullptr, nullptr};
  auto number = [&](PyObject* o, double* one, const float** each, const char* name) {
    if (THPVariable_Check(o)) {
      *each = ptr<const float>(whole(o, at::kFloat, n, dev, name));
      return;
    }
    *one = PyFloat_AsDouble(o);
    if (*one == -1.0 && PyErr_Occurred()) throw Failed();
  };
  number(a[0], &s.temperature, &s.temperature_of, "temperature");
  number(a[2], &s.top_p, &s.top_p_of, "top_p");
  number(a[3], &s.min_p, &s.min_p_of, "min_p");
  if (THPVariable_Check(a[1])) s.top_k_of = ptr<const int32_t>(whole(a[1], at::kInt, n, dev, "top_k"));
  else s.top_k = static_cast<int32_t>(std::max<int64_t>(std::min<int64_t>(as_int(a[1]), INT32_MAX), INT32_MIN));
  return s;
}
struct DrawnOutputs {                                     // ids, logp, logq
  const Output ids, logp, logq;
  DrawnOutputs(PyObject* const* a, int64_t n, const at::Device& dev)
      : ids(a[0], [&] { return fresh({n}, at::kInt, dev); }), logp(a[1], [&] { return fresh({n}, at::kFloat, dev); }), logq(a[2], [&] { return fresh({n}, at::kFloat, dev); }) {
    whole(ids.t, at::kInt, n, dev, "ids");
    whole(logp.t, at::kFloat, n, dev, "logp");
    whole(logq.t, at::kFloat, n, dev, "logq");
    same_address("logp", logp.t, "logq", logq.t);
  }
  void apart_from(const at::Tensor& u, PyObject* const* settings) const {   // temperature, top_k, top_p, min_p
    for (const at::Tensor& o : {logp.t, logq.t}) {
      same_address("u", u, "an output", o);
      for (int i : {0, 2, 3})
        if (THPVariable_Check(settings[i])) same_address("a setting", tensor(settings[i]), "an output", o);
    }
    if (THPVariable_Check(settings[1])) same_address("top_k", tensor(settings[1]), "ids", ids.t);
  }
};
PyObject* sample_logits(PyObject* const* a) {             // logits, u, temperature, top_k, top_p, min_p, ids, logp, logq, workspace, stream
  const Rows z(a[0]);
  const at::Device dev = z.t.device();
  if (z.n > 0 && z.d > 0 && ((z.d > 1 && z.t.stride(1) != 1) || (z.n > 1 && z.t.stride(0) < z.d))) {
    PyErr_SetString(PyExc_ValueError, "logits [n, V]: the numbers of a row must lie next to each other, the rows one behind the other");
    throw Failed();
  }
  const at::Tensor& u = whole(a[1], at::kFloat, z.n, dev, "u");
  const umas_sampling s = sampling_of(a + 2, z.n, dev);
  const DrawnOutputs out(a + 6, z.n, dev);
  out.apart_from(u, a + 2);
  const Output ws(a[9], [&] { return workspace(umas_sample_logits_workspace_bytes(z.n, z.d), dev); });
  in_reach(ws.t, dev, "workspace");
  on_a_gpu(z.t, "logits");
  void* const st = stream_of(a[10]);
  UMAS_CALL(umas_sample_logits(z.t.data_ptr(), static_cast<umas_dtype>(z.dt), z.n, z.d, z.n > 1 ? z.t.stride(0) : z.d, ptr<float>(u), &s, ptr<int32_t>(out.ids.t),
                               ptr<float>(out.logp.t), ptr<float>(out.logq.t), ws.t.data_ptr(), ws.t.nbytes(), st));
  return pack({out.ids.object(), out.logp.object(), out.logq.object()});
}
PyObject* sample_tokens(PyObject* const* a) {             // H, W, u, rowsel, temperature, top_k, top_p, min_p, ids, logp, logq, workspace, stream
  const Rows H(a[0]);
  const at::Tensor& W = tensor(a[1]);
  const at::Device dev = H.t.device();
  same_head(H, W);
  const int32_t V = static_cast<int32_t>(W.size(0));
  whole_selection(a[3], dev);
  Selection sel(a[3], H.n);
  const at::Tensor& u = whole(a[2], at::kFloat, H.n, dev, "u");
  const umas_sampling s = sampling_of(a + 4, H.n, dev);
  const DrawnOutputs out(a + 8, H.n, dev);
  out.apart_from(u, a + 4);
  const umas_dtype dt = static_cast<umas_dtype>(H.dt);
  const Output ws(a[11], [&] { return workspace(umas_sample_tokens_workspace_bytes(sel.n, H.d, V, dt), dev); });
  in_reach(ws.t, dev, "workspace");
  on_a_gpu(H.t, "H");
  sel.point(ws.t.data_ptr(), a[3]);
  void* const st = stream_of(a[12]);
  UMAS_CALL(umas_sample_tokens(H.t.data_ptr(), W.data_ptr(), dt, H.n, H.d, V, sel.p, sel.n, ptr<float>(u), &s, ptr<int32_t>(out.ids.t), ptr<float>(out.logp.t),
                               ptr<float>(out.logq.t), ws.t.data_ptr(), ws.t.nbytes(), st));
  return pack({out.ids.object(), out.logp.object(), out.logq.object()});
}

PyObject* clip_gradients(PyObject* const* a) {            // gradients, max_norm, out, stats, workspace, stream
  const Ref list(PySequence_Fast(a[0], "gradients must be a list of tensors"));
  const Ref to(a[2] == Py_None ? (Py_INCREF(list.o), list.o) : PySequence_Fast(a[2], "out must be a list of tensors"));
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(list.o);
  if (PySequence_Fast_GET_SIZE(to.o) != n) {
    PyErr_SetString(PyExc_ValueError, "out must hold a tensor for every gradient");
    throw Failed();
  }
  if (n == 0) {
    PyErr_SetString(PyExc_ValueError, "gradients must hold a tensor");
    throw Failed();
  }
  const at::Device dev = tensor(PySequence_Fast_GET_ITEM(list.o, 0)).device();
  std::vector<umas_gradient> g(static_cast<size_t>(n));
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* const o = PySequence_Fast_GET_ITEM(list.o, i);
    const int dt = dtype_code(o);
    const at::Tensor &x = tensor(o), &y = tensor(PySequence_Fast_GET_ITEM(to.o, i));
    whole(x, x.scalar_type(), x.numel(), dev, "a gradient");
    whole(y, x.scalar_type(), x.numel(), dev, "an output of a gradient");
    g[static_cast<size_t>(i)] = umas_gradient{x.data_ptr(), y.data_ptr(), x.numel(), dt};
  }
  const double max_norm = PyFloat_AsDouble(a[1]);
  if (max_norm == -1.0 && PyErr_Occurred()) throw Failed();
  const Output stats(a[3], [&] { return fresh({static_cast<int64_t>(sizeof(umas_clip_stats))}, at::kByte, dev); });
  const Output ws(a[4], [&] { return workspace(umas_clip_workspace_bytes(static_cast<int32_t>(std::min<Py_ssize_t>(n, INT32_MAX))), dev); });
  whole(stats.t, at::kByte, static_cast<int64_t>(sizeof(umas_clip_stats)), dev, "stats");
  in_reach(ws.t, dev, "workspace");
  on_a_gpu(tensor(PySequence_Fast_GET_ITEM(list.o, 0)), "gradients");
  void* const st = stream_of(a[5]);
  UMAS_CALL(umas_clip_gradients(g.data(), static_cast<int32_t>(n), max_norm, ptr<umas_clip_stats>(stats.t), ws.t.data_ptr(), ws.t.nbytes(), st));
  PyObject* const written = PySequence_List(to.o);
  return pack({stats.object(), written});
}

PyObject* values(PyObject* const* a) {                    // H, w, bias, rowsel, value, stream
  const Rows H(a[0]);
  const at::Tensor& w = tensor(a[1]);
  on_gpu(H.t.device());
  in_reach({{a[1], "w"}, {a[3], "rowsel"}, {a[4], "value"}}, H.t.device());
  const Output value(a[4], [&] { return fresh({H.n}, at::kFloat, H.t.device()); });
  Selection sel(a[3], H.n);
  sel.point(w.data_ptr(), a[3]);
  const float bias = real(a[2]);
  void* const st = stream_of(a[5]);
  UMAS_CALL(umas_values(H.t.data_ptr(), w.data_ptr(), bias, static_cast<umas_dtype>(H.dt), H.n, H.d, sel.p, sel.n, ptr<float>(value.t), st));
  return value.object();
}

PyObject* value_loss(PyObject* const* a) {
  // H, w, bias, rowsel, value_old, ret, tok_role, n_roles, clip_eps_v, accumulate_dH, accumulate_dw, norm_rows, dH, dw, db, value_new,
  // stats, workspace, stream
  const Rows H(a[0]);
  const at::Tensor& w = tensor(a[1]);
  const at::Device dev = H.t.device();
  on_gpu(dev);
  in_reach({{a[1], "w"}, {a[3], "rowsel"}, {a[4], "value_old"}, {a[5], "ret"}, {a[6], "tok_role"}, {a[12], "dH"}, {a[13], "dw"}, {a[14], "db"}, {a[15], "value_new"}, {a[16], "stats"},
            {a[17], "workspace"}}, dev);
  const umas_dtype dt = static_cast<umas_dtype>(H.dt);
  const int32_t n_roles = integer32(a[7]);
  Selection sel(a[3], H.n);
  const Output dH(a[12], [&] { return at::empty_like(H.t); });
  const Output dw(a[13], [&] { return fresh({H.d}, at::kFloat, dev); });
  const Output db(a[14], [&] { return fresh({1}, at::kFloat, dev); });
  const Output value_new(a[15], [&] { return fresh({H.n}, at::kFloat, dev); });
  const Output stats(a[16], [&] { return fresh({(1 + static_cast<int64_t>(n_roles)) * static_cast<int64_t>(sizeof(umas_value_stats))}, at::kByte, dev); });
  const Output ws(a[17], [&] { return workspace(umas_value_workspace_bytes(sel.n, H.d, dt, n_roles), dev); });
  sel.point(ws.t.data_ptr(), a[3]);
  const float bias = real(a[2]), clip_eps = real(a[8]);
  const float *const value_old = ptr_or_null<const float>(a[4]), *const ret = ptr_or_null<const float>(a[5]);
  const int32_t* const role = ptr_or_null<const int32_t>(a[6]);
  const int32_t acc_dH = truth(a[9]), acc_dw = truth(a[10]);
  const int64_t norm_rows = as_int(a[11]);
  void* const st = stream_of(a[18]);
  UMAS_CALL(umas_value_loss_fwd_bwd(H.t.data_ptr(), w.data_ptr(), bias, dt, H.n, H.d, sel.p, sel.n, value_old, ret, role, n_roles, clip_eps, acc_dH,
                                    acc_dw, norm_rows, ptr<umas_value_stats>(stats.t), ptr<float>(value_new.t), dH.t.data_ptr(),
                                    ptr<float>(dw.t), ptr<float>(db.t), ws.t.data_ptr(), ws.t.numel(), st));
  return pack({stats.object(), value_new.object(), dH.object(), dw.object(), db.object()});
}

PyObject* kl_rewards(PyObject* const* a) {                // tok_reward, logp, logp_ref, tok_mask, beta, out, stream
  const at::Tensor& r = tensor(a[0]);
  const int64_t n = r.numel();
  const at::Device dev = r.device();
  in_reach({{a[1], "logp"}, {a[2], "logp_ref"}, {a[3], "tok_mask"}, {a[5], "out"}}, dev);
  const Output out(a[5], [&] { return at::empty_like(r); });
  const at::Tensor kl = fresh({1}, at::kFloat, dev), ws = workspace(umas_kl_rewards_workspace_bytes(n), dev);
  auto at_ = [&](const at::Tensor& t) { return n ? t.data_ptr() : ws.data_ptr(); };
  const at::Tensor &logp = tensor(a[1]), &ref = tensor(a[2]), &mask = tensor(a[3]);
  const float beta = real(a[4]);
  void* const st = stream_of(a[6]);
  UMAS_CALL(umas_kl_rewards(static_cast<float*>(at_(r)), static_cast<float*>(at_(logp)), static_cast<float*>(at_(ref)), static_cast<uint8_t*>(at_(mask)), n,
                            beta, static_cast<float*>(at_(out.t)), ptr<float>(kl), ws.data_ptr(), bytes_of(ws), st));
  return pack({out.object(), wrap(kl)});
}

PyObject* whiten(PyObject* const* a) {                    // adv, tok_mask, tok_role, model_tok_off, n_roles, scope, eps, out, stream
  const at::Tensor& adv = tensor(a[0]);
  const int64_t n = adv.numel();
  const at::Device dev = adv.device();
  in_reach({{a[1], "tok_mask"}, {a[2], "tok_role"}, {a[7], "out"}}, dev);
  I64_ARRAY(off, a[3]);
  const int32_t n_models = static_cast<int32_t>(off.len - 1), n_roles = integer32(a[4]), scope = integer32(a[5]);
  const Output out(a[7], [&] { return at::empty_like(adv); });
  const at::Tensor ws = workspace(umas_whiten_workspace_bytes(n, n_models, n_roles), dev);
  auto at_ = [&](PyObject* o) -> void* { return o == Py_None ? nullptr : n ? tensor(o).data_ptr() : ws.data_ptr(); };
  const float eps = real(a[6]);
  const float* const x = static_cast<float*>(at_(a[0]));
  const uint8_t* const mask = static_cast<uint8_t*>(at_(a[1]));
  const int32_t* const role = static_cast<int32_t*>(at_(a[2]));
  float* const y = static_cast<float*>(n ? out.t.data_ptr() : ws.data_ptr());
  void* const st = stream_of(a[8]);
  UMAS_CALL(umas_whiten_advantages(x, mask, role, off.as<int64_t>(), n_models, n_roles, n, scope, eps, y, ws.data_ptr(), bytes_of(ws), st));
  return out.object();
}

PyObject* ready_batch(PyObject* const* a) {               // streams, traj_turn_off, cut, parts or rows, keep, order, stream
  const at::Device dev = device_of(a[0], kRowsel);
  I32_ARRAY(tto, a[1]);
  const int32_t cut = integer32(a[2]);                    // 0: by trajectories, 1: by rows, 2: packed
  U8_ARRAY(keep, a[4]);
  I32_ARRAY(order, a[5]);
  const int32_t B = static_cast<int32_t>(tto.len - 1), U = static_cast<int32_t>(int_attr(a[0], g_n_turns)), M = static_cast<int32_t>(int_attr(a[0], g_n_models));
  int64_t n_rowsel;
  {
    const Ref t(PyObject_GetAttr(a[0], g_stream_names[kRowsel]));
    n_rowsel = tensor(t.o).numel();
  }
  const int64_t arg = cut == 2 ? as_int(a[3]) : integer32(a[3]);
  const at::Tensor rows = fresh({std::max<int64_t>(n_rowsel, 1)}, at::kInt, dev);
  const at::Tensor off = fresh({M, (cut == 2 ? B : arg) + 1}, at::kLong, dev);
  const at::Tensor parts = cut == 2 ? fresh({M}, at::kInt, dev) : at::Tensor();
  const at::Tensor ws = workspace(umas_ready_batch_workspace_bytes(B, M), dev);
  const umas_streams s = streams_of(a[0], dev, ws.data_ptr());
  const int32_t* const t = tto.as<int32_t>();
  const uint8_t* const k = keep.as<uint8_t>();
  const int32_t* const o = order.as<int32_t>();
  void* const st = stream_of(a[6]);
  if (cut == 2) {
    UMAS_CALL(umas_ready_batch_packed(&s, M, U, t, B, k, o, arg, ptr<int32_t>(rows), ptr<int64_t>(off), ptr<int32_t>(parts), ws.data_ptr(), bytes_of(ws), st));
    return pack({wrap(rows), wrap(off), wrap(parts)});
  }
  const auto fn = cut == 1 ? umas_ready_batch_balanced : umas_ready_batch;
  UMAS_CALL(fn(&s, M, U, t, B, k, o, static_cast<int32_t>(arg), ptr<int32_t>(rows), ptr<int64_t>(off), ws.data_ptr(), bytes_of(ws), st));
  return pack({wrap(rows), wrap(off)});
}

// ------------------------------------------------------------------ module
template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", N, n);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Failed&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
#define ENTRY(name, f, n) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&entry<f, n>)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {ENTRY("assign", assign, 19), ENTRY("advantages", advantages, 7), ENTRY("policy_logprobs", policy_logprobs, 7),
                           ENTRY("policy_logprobs_static", policy_logprobs_static, 8), ENTRY("ppo_loss", ppo_loss, 21), ENTRY("top_logits", top_logits, 9),
                           ENTRY("cross_entropy", cross_entropy, 17), ENTRY("distill", distill, 18), ENTRY("rms_norm", rms_norm, 8),
                           ENTRY("rms_norm_quantized", rms_norm_quantized, 9), ENTRY("rms_norm_bwd", rms_norm_bwd, 10), ENTRY("sample_logits", sample_logits, 11),
                           ENTRY("sample_tokens", sample_tokens, 13), ENTRY("clip_gradients", clip_gradients, 6), ENTRY("values", values, 6),
                           ENTRY("value_loss", value_loss, 19), ENTRY("kl_rewards", kl_rewards, 7), ENTRY("whiten", whiten, 9),
                           ENTRY("ready_batch", ready_batch, 7), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_umas_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__umas_torch() {
  PyObject* np = PyImport_ImportModule("numpy");
  if (!np) return nullptr;
  ascontiguousarray = PyObject_GetAttrString(np, "ascontiguousarray");
  Py_DECREF(np);
  if (!ascontiguousarray) return nullptr;
  for (int i = 0; i < kStreamTensors; ++i) g_stream_names[i] = PyUnicode_InternFromString(kStreamNames[i]);
  g_n_tokens = PyUnicode_InternFromString("n_tokens");
  g_n_turns = PyUnicode_InternFromString("n_turns");
  g_n_models = PyUnicode_InternFromString("n_models");
  return PyModule_Create(&g_module);
}
