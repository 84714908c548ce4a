// The part of the Python binding that runs on every call: argument checks on torch tensors, the
// current stream, and the call into the C ABI (include/pcgrl.h), without a Python frame, a ctypes
// conversion or a Python-level attribute lookup per argument.  A pcgrl_step from Python is bound by
// this path for every batch whose kernel takes less than it: 9 us a call when the same checks were
// made in Python and the call through ctypes (3 us of it the library and the launch), against a
// kernel of 4.5 us for 64 levels of 16x16.
//
// Only what is plainly right is handled here.  Anything else -- a wrong type, shape, device or
// layout, an argument that is missing, a tensor that torch itself refuses to look into (one without
// storage, say) -- makes the call return kLook, and the Python method then goes through the arguments
// one by one and says what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "../../include/pcgrl.h"

namespace {

constexpr long kLook = 1000;  // "look at the arguments": no library code is positive

struct Env {
  PyObject_HEAD pcgrl_ctx* ctx;
  int device;
  int64_t B, M, Hm, Wm;
  int64_t obs[4], onehot[4];  // the shape of an observation buffer, and of its one-hot cells
  int obs_dims;
};

// A tensor argument as a device pointer: contiguous, of this element type and on this device, with
// the `nd` sizes of `dims` behind `lead` leading ones (lead < 0: none, else the size of the one
// there is).
bool tensor(PyObject* o, const Env* e, c10::ScalarType type, int64_t lead, const int64_t* dims, int nd, void** out) {
  if (!THPVariable_Check(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  const int extra = lead >= 0 ? 1 : 0;
  if (!t.is_cuda() || t.get_device() != e->device || t.scalar_type() != type || t.dim() != nd + extra) return false;
  if (extra && t.size(0) != lead) return false;
  for (int i = 0; i < nd; ++i)
    if (t.size(i + extra) != dims[i]) return false;
  if (!t.is_contiguous()) return false;
  *out = t.data_ptr();
  return true;
}
bool optional(PyObject* o, const Env* e, c10::ScalarType type, int64_t lead, const int64_t* dims, int nd, void** out) {
  *out = nullptr;
  return o == Py_None || tensor(o, e, type, lead, dims, nd, out);
}

void* stream_of(const Env* e) { return c10::hip::getCurrentHIPStream((c10::DeviceIndex)e->device).stream(); }

PyObject* look() { return PyLong_FromLong(kLook); }
template <typename F> PyObject* call(F&& f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// step(actions, obs, reward, done)
PyObject* env_step(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Env* e = reinterpret_cast<Env*>(self);
  void *act, *obs, *rew, *done;
  if (n != 4 || !e->ctx || !tensor(a[0], e, at::kInt, -1, &e->B, 1, &act) ||
      !optional(a[1], e, at::kByte, -1, e->obs, e->obs_dims, &obs) || !optional(a[2], e, at::kFloat, -1, &e->B, 1, &rew) ||
      !optional(a[3], e, at::kByte, -1, &e->B, 1, &done))
    return look();
  void* st = stream_of(e);
  return call([&] {
    return pcgrl_step(e->ctx, static_cast<const int32_t*>(act), static_cast<uint8_t*>(obs), static_cast<float*>(rew),
                      static_cast<uint8_t*>(done), st);
  });
}

// rollout(actions, obs, reward, done)
PyObject* env_rollout(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Env* e = reinterpret_cast<Env*>(self);
  if (n != 4 || !e->ctx || !THPVariable_Check(a[0]) || THPVariable_Unpack(a[0]).dim() != 2) return look();
  const int64_t T = THPVariable_Unpack(a[0]).size(0);
  int64_t slots = 1;
  if (a[1] != Py_None) {
    if (!THPVariable_Check(a[1]) || THPVariable_Unpack(a[1]).dim() != e->obs_dims + 1) return look();
    slots = THPVariable_Unpack(a[1]).size(0);
  }
  void *act, *obs, *rew, *done;
  if (T > (1 << 20) || slots > (1 << 20) || !tensor(a[0], e, at::kInt, T, &e->B, 1, &act) ||
      !optional(a[1], e, at::kByte, slots, e->obs, e->obs_dims, &obs) || !optional(a[2], e, at::kFloat, T, &e->B, 1, &rew) ||
      !optional(a[3], e, at::kByte, T, &e->B, 1, &done))
    return look();
  void* st = stream_of(e);
  return call([&] {
    return pcgrl_rollout(e->ctx, static_cast<const int32_t*>(act), (int32_t)T, static_cast<uint8_t*>(obs), (int32_t)slots,
                         static_cast<float*>(rew), static_cast<uint8_t*>(done), st);
  });
}

// reset(seed, obs): the seed as ctypes takes it, any Python integer modulo 2^64
PyObject* env_reset(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Env* e = reinterpret_cast<Env*>(self);
  void* obs;
  if (n != 2 || !e->ctx || !PyLong_Check(a[0]) || !optional(a[1], e, at::kByte, -1, e->obs, e->obs_dims, &obs)) return look();
  const unsigned long long seed = PyLong_AsUnsignedLongLongMask(a[0]);
  if (PyErr_Occurred()) return nullptr;
  void* st = stream_of(e);
  return call([&] { return pcgrl_reset(e->ctx, (uint64_t)seed, static_cast<uint8_t*>(obs), st); });
}

at::TensorOptions on_device(const Env* e, c10::ScalarType type) {
  return at::TensorOptions().dtype(type).device(at::Device(at::kCUDA, (c10::DeviceIndex)e->device));
}

// metrics(out) / exact_diameter(out) / observe(obs)
PyObject* env_metrics(PyObject* self, PyObject* o) {
  Env* e = reinterpret_cast<Env*>(self);
  const int64_t dims[2] = {e->B, e->M};
  void* out;
  if (!e->ctx || !tensor(o, e, at::kInt, -1, dims, 2, &out)) return look();
  void* st = stream_of(e);
  return call([&] { return pcgrl_metrics(e->ctx, static_cast<int32_t*>(out), st); });
}
PyObject* env_exact_diameter(PyObject* self, PyObject* o) {
  Env* e = reinterpret_cast<Env*>(self);
  void* out;
  if (!e->ctx || !tensor(o, e, at::kInt, -1, &e->B, 1, &out)) return look();
  void* st = stream_of(e);
  return call([&] { return pcgrl_exact_diameter(e->ctx, static_cast<int32_t*>(out), st); });
}
PyObject* env_observe(PyObject* self, PyObject* o) {
  Env* e = reinterpret_cast<Env*>(self);
  void* obs;
  if (!e->ctx || !tensor(o, e, at::kByte, -1, e->obs, e->obs_dims, &obs)) return look();
  void* st = stream_of(e);
  return call([&] { return pcgrl_observe(e->ctx, static_cast<uint8_t*>(obs), st); });
}

// unpack_obs(packed, out): the element type is that of `out`
PyObject* env_unpack_obs(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Env* e = reinterpret_cast<Env*>(self);
  void *packed, *out;
  if (n != 2 || !e->ctx || !tensor(a[0], e, at::kByte, -1, e->obs, e->obs_dims, &packed) || !THPVariable_Check(a[1])) return look();
  const c10::ScalarType type = THPVariable_Unpack(a[1]).scalar_type();
  const int code = type == at::kByte ? PCGRL_UNPACK_U8 : type == at::kHalf ? PCGRL_UNPACK_F16
                   : type == at::kBFloat16 ? PCGRL_UNPACK_BF16 : type == at::kFloat ? PCGRL_UNPACK_F32 : -1;
  if (code < 0 || !tensor(a[1], e, type, -1, e->onehot, 4, &out)) return look();
  void* st = stream_of(e);
  return call([&] { return pcgrl_unpack_obs(e->ctx, static_cast<const uint8_t*>(packed), out, code, st); });
}

// set_state(tiles, frozen, hw, pos)
PyObject* env_set_state(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Env* e = reinterpret_cast<Env*>(self);
  const int64_t grid[3] = {e->B, e->Hm, e->Wm}, pair[2] = {e->B, 2};
  void *tiles, *frozen, *hw, *pos;
  if (n != 4 || !e->ctx || !tensor(a[0], e, at::kChar, -1, grid, 3, &tiles) ||
      !optional(a[1], e, at::kByte, -1, grid, 3, &frozen) || !tensor(a[2], e, at::kShort, -1, pair, 2, &hw) ||
      !tensor(a[3], e, at::kShort, -1, pair, 2, &pos))
    return look();
  void* st = stream_of(e);
  return call([&] {
    return pcgrl_set_state(e->ctx, static_cast<const int8_t*>(tiles), static_cast<const uint8_t*>(frozen),
                           static_cast<const int16_t*>(hw), static_cast<const int16_t*>(pos), st);
  });
}

// get_state() -> (rc, tiles, frozen, hw, pos, counters), new tensors
PyObject* env_get_state(PyObject* self, PyObject*) {
  Env* e = reinterpret_cast<Env*>(self);
  if (!e->ctx) return look();
  HANDLE_TH_ERRORS
  at::Tensor tiles = at::empty({e->B, e->Hm, e->Wm}, on_device(e, at::kChar));
  at::Tensor frozen = at::empty({e->B, e->Hm, e->Wm}, on_device(e, at::kByte));
  at::Tensor hw = at::empty({e->B, 2}, on_device(e, at::kShort));
  at::Tensor pos = at::empty({e->B, 2}, on_device(e, at::kShort));
  at::Tensor counters = at::empty({e->B, 3}, on_device(e, at::kInt));
  void* st = stream_of(e);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = pcgrl_get_state(e->ctx, static_cast<int8_t*>(tiles.data_ptr()), static_cast<uint8_t*>(frozen.data_ptr()),
                       static_cast<int16_t*>(hw.data_ptr()), static_cast<int16_t*>(pos.data_ptr()),
                       static_cast<int32_t*>(counters.data_ptr()), st);
  Py_END_ALLOW_THREADS
  return Py_BuildValue("(iNNNNN)", rc, THPVariable_Wrap(tiles), THPVariable_Wrap(frozen), THPVariable_Wrap(hw),
                       THPVariable_Wrap(pos), THPVariable_Wrap(counters));
  END_HANDLE_TH_ERRORS
}

// ---- the policy's side

int logit_type(const at::Tensor& t) {
  const c10::ScalarType s = t.scalar_type();
  return s == at::kHalf ? PCGRL_UNPACK_F16 : s == at::kBFloat16 ? PCGRL_UNPACK_BF16 : s == at::kFloat ? PCGRL_UNPACK_F32 : -1;
}

// A matrix whose rows are contiguous and may lie apart (one_for_all: or be one and the same); n and V < 0: any size.
bool rows(PyObject* o, const Env* e, bool one_for_all, int64_t n, int64_t V, void** out, int64_t* stride) {
  if (!THPVariable_Check(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.get_device() != e->device) return false;
  const bool one = one_for_all && t.dim() == 1;
  if (!one && t.dim() != 2) return false;
  const int64_t tn = one ? n : t.size(0), tV = one ? t.size(0) : t.size(1), across = one ? 0 : t.stride(0), along = one ? t.stride(0) : t.stride(1);
  if ((n >= 0 && tn != n) || (V >= 0 && tV != V) || (tV > 1 && along != 1)) return false;
  if (tn > 1 && across < tV && !(one_for_all && across == 0)) return false;
  *stride = tn > 1 ? across : tV;
  *out = t.data_ptr();
  return true;
}
bool mask_rows(PyObject* o, const Env* e, int64_t n, int64_t V, void** out, int64_t* stride) {
  *out = nullptr;
  *stride = 0;
  if (o == Py_None) return true;
  if (!THPVariable_Check(o)) return false;
  const c10::ScalarType s = THPVariable_Unpack(o).scalar_type();
  return (s == at::kByte || s == at::kBool) && rows(o, e, true, n, V, out, stride);
}
bool number(PyObject* o, double* out) {
  if (!PyFloat_Check(o) && !PyLong_Check(o)) return false;
  *out = PyFloat_AsDouble(o);
  if (*out != -1. || !PyErr_Occurred()) return true;
  PyErr_Clear();  // (a whole number that no double holds)
  return false;
}
// An output: the caller's tensor, or a new one where there is none.
bool output(PyObject* o, const Env* e, c10::ScalarType type, const int64_t* dims, int nd, at::Tensor* t, void** out) {
  if (o != Py_None) {
    if (!tensor(o, e, type, -1, dims, nd, out)) return false;
    *t = THPVariable_Unpack(o);
    return true;
  }
  *t = at::empty(at::IntArrayRef(dims, (size_t)nd), on_device(e, type));
  *out = t->data_ptr();
  return true;
}

// What a call has written through a pointer has changed for autograd too: a backward pass that has kept it then says so.  (New tensors
// have not been seen by anybody, and tensors of inference mode have no version.)
void written(PyObject* o) {
  if (o == Py_None) return;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

struct Draw {
  pcgrl_sampling how;
  void *logits, *mask, *uniform, *actions, *log_probs;
  int64_t n;
  at::Tensor a, lp;
};
// logits, uniform, mask, temperature, top_k, top_p, min_p, actions, log_probs
bool drawing(PyObject* const* a, const Env* e, int64_t n, Draw* d) {
  std::memset(&d->how, 0, sizeof(d->how));
  if (!rows(a[0], e, false, n, -1, &d->logits, &d->how.logits_stride)) return false;
  const at::Tensor& x = THPVariable_Unpack(a[0]);
  d->n = x.size(0);
  d->how.type = logit_type(x);
  if (d->how.type < 0 || x.size(1) < 1 || x.size(1) > PCGRL_MAX_CLASSES) return false;
  d->how.n_classes = (int32_t)x.size(1);
  double k;
  if (!mask_rows(a[2], e, d->n, x.size(1), &d->mask, &d->how.mask_stride) || !number(a[3], &d->how.temperature) || !PyLong_Check(a[4]) ||
      !number(a[4], &k) || !(k >= 0. && k <= 2147483647.) || !number(a[5], &d->how.top_p) || !number(a[6], &d->how.min_p))
    return false;
  d->how.top_k = (int32_t)k;
  if (d->how.temperature == 0. ? !optional(a[1], e, at::kFloat, -1, &d->n, 1, &d->uniform) : !tensor(a[1], e, at::kFloat, -1, &d->n, 1, &d->uniform))
    return false;
  return output(a[7], e, at::kInt, &d->n, 1, &d->a, &d->actions) && output(a[8], e, at::kFloat, &d->n, 1, &d->lp, &d->log_probs);
}

PyObject* env_sample(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Env* e = reinterpret_cast<Env*>(self);
  Draw d;
  if (n != 9 || !e->ctx || !drawing(a, e, -1, &d)) return look();
  void* st = stream_of(e);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = pcgrl_sample(e->ctx, &d.how, d.logits, static_cast<const uint8_t*>(d.mask), static_cast<const float*>(d.uniform), d.n,
                    static_cast<int32_t*>(d.actions), static_cast<float*>(d.log_probs), st);
  Py_END_ALLOW_THREADS
  if (rc == PCGRL_OK)
    for (int i : {7, 8}) written(a[i]);
  return Py_BuildValue("(iNN)", rc, THPVariable_Wrap(d.a), THPVariable_Wrap(d.lp));
}

// ... and obs, reward, done
PyObject* env_step_logits(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Env* e = reinterpret_cast<Env*>(self);
  Draw d;
  void *obs, *rew, *done;
  if (n != 12 || !e->ctx || !optional(a[9], e, at::kByte, -1, e->obs, e->obs_dims, &obs) || !optional(a[10], e, at::kFloat, -1, &e->B, 1, &rew) ||
      !optional(a[11], e, at::kByte, -1, &e->B, 1, &done) || !drawing(a, e, e->B, &d))
    return look();
  void* st = stream_of(e);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = pcgrl_step_logits(e->ctx, &d.how, d.logits, static_cast<const uint8_t*>(d.mask), static_cast<const float*>(d.uniform),
                         static_cast<int32_t*>(d.actions), static_cast<float*>(d.log_probs), static_cast<uint8_t*>(obs),
                         static_cast<float*>(rew), static_cast<uint8_t*>(done), st);
  Py_END_ALLOW_THREADS
  if (rc == PCGRL_OK)
    for (int i : {7, 8, 9, 10, 11}) written(a[i]);
  return Py_BuildValue("(iNN)", rc, THPVariable_Wrap(d.a), THPVariable_Wrap(d.lp));
}

// advantages(reward, done, values, discount, trace, advantages, returns)
PyObject* env_advantages(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Env* e = reinterpret_cast<Env*>(self);
  if (n != 7 || !e->ctx || !THPVariable_Check(a[0]) || !THPVariable_Check(a[1]) || !THPVariable_Check(a[2])) return look();
  const at::Tensor& r = THPVariable_Unpack(a[0]);
  if (r.dim() != 2 || r.size(0) > (1 << 20) || r.size(1) > (1 << 24)) return look();
  const int64_t shape[2] = {r.size(0), r.size(1)}, longer[2] = {shape[0] + 1, shape[1]};
  const at::Tensor &d = THPVariable_Unpack(a[1]), &v = THPVariable_Unpack(a[2]);
  const int type = logit_type(v);
  void *rew, *done, *val, *adv, *ret;
  double discount, trace;
  at::Tensor ta, tr;
  if (type < 0 || !tensor(a[0], e, at::kFloat, -1, shape, 2, &rew) ||
      !tensor(a[1], e, d.scalar_type() == at::kBool ? at::kBool : at::kByte, -1, shape, 2, &done) || !tensor(a[2], e, v.scalar_type(), -1, longer, 2, &val) ||
      !number(a[3], &discount) || !number(a[4], &trace) || !output(a[5], e, at::kFloat, shape, 2, &ta, &adv) || !output(a[6], e, at::kFloat, shape, 2, &tr, &ret))
    return look();
  void* st = stream_of(e);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = pcgrl_advantages(e->ctx, static_cast<const float*>(rew), static_cast<const uint8_t*>(done), val, type, (int32_t)shape[0], (int32_t)shape[1],
                        discount, trace, static_cast<float*>(adv), static_cast<float*>(ret), st);
  Py_END_ALLOW_THREADS
  if (rc == PCGRL_OK)
    for (int i : {5, 6}) written(a[i]);
  return Py_BuildValue("(iNN)", rc, THPVariable_Wrap(ta), THPVariable_Wrap(tr));
}

// policy_loss(logits, actions, advantages, old_log_probs, mask, values, returns, temperature, clip_low, clip_high, entropy_coef,
//             value_coef, scale, grad_logits, grad_values, log_probs, entropies, stats, workspace)
PyObject* env_policy_loss(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Env* e = reinterpret_cast<Env*>(self);
  if (n != 19 || !e->ctx) return look();
  pcgrl_loss l;
  std::memset(&l, 0, sizeof(l));
  void *x, *m, *act, *adv, *old, *val, *ret, *gx, *gv = nullptr, *lp, *h, *stats, *room;
  if (!rows(a[0], e, false, -1, -1, &x, &l.logits_stride)) return look();
  const at::Tensor& t = THPVariable_Unpack(a[0]);
  const int64_t N = t.size(0), V = t.size(1), dims[2] = {N, V}, n_stats = PCGRL_LOSS_STATS;
  l.type = logit_type(t);
  if (l.type < 0 || V < 1 || V > PCGRL_MAX_CLASSES) return look();
  const c10::ScalarType type = t.scalar_type();
  at::Tensor tg, tv, ts, tw;
  if (!tensor(a[1], e, at::kInt, -1, &N, 1, &act) || !tensor(a[2], e, at::kFloat, -1, &N, 1, &adv) || !optional(a[3], e, at::kFloat, -1, &N, 1, &old) ||
      !mask_rows(a[4], e, N, V, &m, &l.mask_stride) || !optional(a[5], e, type, -1, &N, 1, &val) || !optional(a[6], e, at::kFloat, -1, &N, 1, &ret) ||
      (val && !ret) || !number(a[7], &l.temperature) || !number(a[8], &l.clip_low) || !number(a[9], &l.clip_high) || !number(a[10], &l.entropy_coef) ||
      !number(a[11], &l.value_coef))
    return look();
  if (a[12] == Py_None) l.scale = 1. / (double)(N > 1 ? N : 1);
  else if (!number(a[12], &l.scale)) return look();
  if (!optional(a[15], e, at::kFloat, -1, &N, 1, &lp) || !optional(a[16], e, at::kFloat, -1, &N, 1, &h)) return look();
  if (a[13] == Py_None) {
    if (!output(a[13], e, type, dims, 2, &tg, &gx)) return look();
    l.grad_stride = V;
  } else {
    if (!THPVariable_Check(a[13]) || THPVariable_Unpack(a[13]).scalar_type() != type || !rows(a[13], e, false, N, V, &gx, &l.grad_stride)) return look();
    tg = THPVariable_Unpack(a[13]);
  }
  if (val ? !output(a[14], e, type, &N, 1, &tv, &gv) : a[14] != Py_None) return look();
  const int64_t size = pcgrl_policy_loss_workspace();
  if (!output(a[17], e, at::kFloat, &n_stats, 1, &ts, &stats)) return look();
  if (a[18] != Py_None) {
    if (!THPVariable_Check(a[18]) || THPVariable_Unpack(a[18]).numel() < size) return look();
    const int64_t all = THPVariable_Unpack(a[18]).numel();
    if (!tensor(a[18], e, at::kByte, -1, &all, 1, &room)) return look();
  } else if (!output(a[18], e, at::kByte, &size, 1, &tw, &room)) {
    return look();
  }
  l.n_classes = (int32_t)V;
  l.n_rows = N;
  l.logits = x;
  l.mask = static_cast<const uint8_t*>(m);
  l.actions = static_cast<const int32_t*>(act);
  l.advantages = static_cast<const float*>(adv);
  l.old_log_probs = static_cast<const float*>(old);
  l.values = val;
  l.returns = static_cast<const float*>(ret);
  l.grad_logits = gx;
  l.grad_values = gv;
  l.log_probs = static_cast<float*>(lp);
  l.entropies = static_cast<float*>(h);
  l.stats = static_cast<float*>(stats);
  l.workspace = room;
  void* st = stream_of(e);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = pcgrl_policy_loss(e->ctx, &l, st);
  Py_END_ALLOW_THREADS
  if (rc == PCGRL_OK)
    for (int i : {13, 14, 15, 16, 17, 18}) written(a[i]);
  PyObject* values = val ? THPVariable_Wrap(tv) : Py_NewRef(Py_None);
  return Py_BuildValue("(iNNN)", rc, THPVariable_Wrap(ts), THPVariable_Wrap(tg), values);
}

PyObject* env_close(PyObject* self, PyObject*) {
  reinterpret_cast<Env*>(self)->ctx = nullptr;
  Py_RETURN_NONE;
}

// Env(ctx, device, M, max_h, max_w, obs_shape, onehot_shape)
PyObject* env_new(PyTypeObject* type, PyObject* args, PyObject*) {
  unsigned long long ctx;
  int device;
  long long M, Hm, Wm, h[4];
  PyObject* shape;
  if (!PyArg_ParseTuple(args, "KiLLLO!(LLLL)", &ctx, &device, &M, &Hm, &Wm, &PyTuple_Type, &shape, &h[0], &h[1], &h[2], &h[3]))
    return nullptr;
  const Py_ssize_t nd = PyTuple_Size(shape);
  if (nd < 1 || nd > 4) {
    PyErr_SetString(PyExc_ValueError, "an observation buffer has one to four dimensions");
    return nullptr;
  }
  Env* e = reinterpret_cast<Env*>(type->tp_alloc(type, 0));
  if (!e) return nullptr;
  e->ctx = reinterpret_cast<pcgrl_ctx*>((uintptr_t)ctx);
  e->device = device;
  e->M = M;
  e->Hm = Hm;
  e->Wm = Wm;
  e->obs_dims = (int)nd;
  for (int i = 0; i < 4; ++i) e->onehot[i] = h[i];
  for (Py_ssize_t i = 0; i < nd; ++i) e->obs[i] = PyLong_AsLongLong(PyTuple_GetItem(shape, i));
  e->B = e->obs[0];
  if (PyErr_Occurred()) {
    Py_DECREF(e);
    return nullptr;
  }
  return reinterpret_cast<PyObject*>(e);
}

// The tensor accessors and the stream lookup throw, and no C++ exception may reach the interpreter's
// frames: the process would end.  The Python checks make the same accesses and raise what torch says.
// (Nothing throws while the interpreter lock is released: the library's C entry points do not.)
template <auto F, typename... A> PyObject* guarded(PyObject* self, A... args) noexcept {
  try {
    return F(self, args...);
  } catch (...) {
    PyErr_Clear();  // (a tensor type written in Python leaves its exception behind)
    return look();
  }
}

template <auto F> PyCFunction one() { return guarded<F, PyObject*>; }
template <auto F> PyCFunction fast() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<F, PyObject* const*, Py_ssize_t>));
}
PyMethodDef env_methods[] = {
    {"step", fast<env_step>(), METH_FASTCALL, nullptr}, {"rollout", fast<env_rollout>(), METH_FASTCALL, nullptr},
    {"reset", fast<env_reset>(), METH_FASTCALL, nullptr}, {"unpack_obs", fast<env_unpack_obs>(), METH_FASTCALL, nullptr},
    {"set_state", fast<env_set_state>(), METH_FASTCALL, nullptr},
    {"sample", fast<env_sample>(), METH_FASTCALL, nullptr}, {"step_logits", fast<env_step_logits>(), METH_FASTCALL, nullptr},
    {"advantages", fast<env_advantages>(), METH_FASTCALL, nullptr}, {"policy_loss", fast<env_policy_loss>(), METH_FASTCALL, nullptr},
    {"metrics", one<env_metrics>(), METH_O, nullptr}, {"exact_diameter", one<env_exact_diameter>(), METH_O, nullptr},
    {"observe", one<env_observe>(), METH_O, nullptr}, {"get_state", env_get_state, METH_NOARGS, nullptr},
    {"close", env_close, METH_NOARGS, nullptr}, {nullptr, nullptr, 0, nullptr},
};

PyTypeObject EnvType = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "pcgrl_py", "Call path of the Python binding.", -1, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_pcgrl_py() {
  EnvType.tp_name = "pcgrl_py.Env";
  EnvType.tp_basicsize = sizeof(Env);
  EnvType.tp_flags = Py_TPFLAGS_DEFAULT;
  EnvType.tp_new = env_new;
  EnvType.tp_methods = env_methods;
  if (PyType_Ready(&EnvType) < 0) return nullptr;
  PyObject* m = PyModule_Create(&module_def);
  if (!m) return nullptr;
  Py_INCREF(&EnvType);
  if (PyModule_AddObject(m, "Env", reinterpret_cast<PyObject*>(&EnvType)) < 0 || PyModule_AddIntConstant(m, "LOOK", kLook) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
