// The Python calls of a serving loop without ctypes: parameters read from the tensors, outputs allocated and the C
// function called in one step.  A call costs what its launch costs, and ctypes, the attribute reads and four
// torch.empty cost more than that: 14.8 us for a compress call whose kernel takes 9 us, 6.2 us for a token in
// decode whose kernel takes 3 us.  An attend call takes the host 5.7 us here with one kernel and 9 with two.
//
// It takes the plain forms only (exact tensors of one device, four dimensions, integers and floats as such).  Anything
// else - and what lagkv_plan refuses or an allocator throws - it leaves alone and says so (None, or -1): lagkv.py
// then goes through its own steps, which raise what they raise.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cmath>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include "compress_ws.h"
#include "lagkv.h"

namespace {

decltype(&lagkv_plan) plan_fn;
decltype(&lagkv_workspace_bytes) workspace_fn;
decltype(&lagkv_compress) compress_fn;
decltype(&lagkv_append_and_compress) append_fn;
decltype(&lagkv_attend_workspace_bytes) attend_ws_fn;
decltype(&lagkv_attend) attend_fn;
decltype(&lagkv_attend_blocks) attend_blocks_fn;
decltype(&lagkv_block_bounds) bounds_fn;
decltype(&lagkv_select_blocks) select_fn;
PyObject* raw_stream_fn;  // device index -> handle of the current stream

bool to_int(PyObject* o, int32_t* v) {
  if (!PyLong_Check(o)) return false;
  int over = 0;
  const long x = PyLong_AsLongAndOverflow(o, &over);
  if (over || x < INT32_MIN || x > INT32_MAX) return false;
  *v = (int32_t)x;
  return true;
}

bool to_double(PyObject* o, double* v) {
  if (!PyFloat_CheckExact(o)) return false;
  *v = PyFloat_AS_DOUBLE(o);
  return true;
}

// A [B,H,T,D] device tensor of one of the element types.
const at::Tensor* rows_of(PyObject* o, int32_t* dtype) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.layout() != at::kStrided || t.dim() != 4 || t.stride(3) != 1) return nullptr;
  switch (t.scalar_type()) {
    case at::kFloat: *dtype = LAGKV_F32; break;
    case at::kBFloat16: *dtype = LAGKV_BF16; break;
    case at::kHalf: *dtype = LAGKV_F16; break;
    default: return nullptr;
  }
  return &t;
}

bool alike(const at::Tensor& a, const at::Tensor& b) {
  return a.sizes() == b.sizes() && a.strides() == b.strides() && a.device() == b.device();
}

// S, L, r, variant, std_ddof, launch from args[0 .. 6)
bool params_of(PyObject* const* args, const at::Tensor& K, int32_t dtype, lagkv_params* p) {
  if (K.size(0) > INT32_MAX || K.size(1) > INT32_MAX || K.size(3) > INT32_MAX) return false;
  p->B = (int32_t)K.size(0);
  p->H = (int32_t)K.size(1);
  p->D = (int32_t)K.size(3);
  p->dtype = dtype;
  p->stride_b = K.stride(0);
  p->stride_h = K.stride(1);
  p->stride_t = K.stride(2);
  return to_int(args[0], &p->S) && to_int(args[1], &p->L) && to_double(args[2], &p->r) && to_int(args[3], &p->variant) &&
         to_int(args[4], &p->std_ddof) && to_int(args[5], &p->launch);
}

bool stream_of(const at::Tensor& t, void** s) {
  PyObject* i = PyLong_FromLong(t.device().index());
  PyObject* h = i ? PyObject_CallFunctionObjArgs(raw_stream_fn, i, nullptr) : nullptr;
  Py_XDECREF(i);
  if (!h) return false;
  *s = (void*)PyLong_AsSize_t(h);
  Py_DECREF(h);
  return !PyErr_Occurred();
}

PyObject* none() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

// compress(K, V, S, L, r, variant, std_ddof, launch, want_idx, want_scores)
//   -> (K_out, V_out, idx or None, scores or None, bytes of the plan), the status that lagkv_compress refused with (it is
//      not called a second time), or None: not called
PyObject* compress(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 10 || !PyBool_Check(args[8]) || !PyBool_Check(args[9])) return none();
  try {
    int32_t dt, dv;
    const at::Tensor *K = rows_of(args[0], &dt), *V = rows_of(args[1], &dv);
    lagkv_params p;
    void* stream;
    if (!K || !V || dt != dv || !alike(*K, *V) || !params_of(args + 2, *K, dt, &p)) return none();
    const int64_t T = K->size(2);
    lagkv_plan_t pl;
    if (plan_fn(&p, T, -1, &pl) != LAGKV_OK || !stream_of(*K, &stream)) return none();
    const auto opt = K->options().requires_grad(false);
    const int64_t B = p.B, H = p.H, D = p.D;
    at::Tensor Ko = at::empty({B, H, pl.T_out, D}, opt), Vo = at::empty({B, H, pl.T_out, D}, opt), idx, scores, ws;
    if (args[8] == Py_True) idx = at::empty({B, H, pl.T_out}, opt.dtype(at::kInt));
    if (args[9] == Py_True) scores = at::empty({B, H, pl.n_scored * p.L}, opt.dtype(at::kFloat));
    size_t need = 0;
    if (workspace_fn(&p, T)) {
      need = lagkv::compress_ws(B * H, pl.n_scored, p.L, pl.k, true).total;
      ws = at::empty({(int64_t)need}, opt.dtype(at::kByte));
    }
    const void *k = K->data_ptr(), *v = V->data_ptr();
    void *ko = Ko.data_ptr(), *vo = Vo.data_ptr(), *w = need ? ws.data_ptr() : nullptr;
    int32_t* ip = idx.defined() ? (int32_t*)idx.data_ptr() : nullptr;
    float* sp = scores.defined() ? (float*)scores.data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = compress_fn(&p, k, v, T, ko, vo, ip, sp, w, need, stream);
    Py_END_ALLOW_THREADS
    if (rc != LAGKV_OK) return PyLong_FromLong(rc);
    PyObject* out = PyTuple_New(5);
    if (!out) return nullptr;
    auto put = [&](int i, const at::Tensor& t) {
      PyObject* o = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
      PyTuple_SET_ITEM(out, i, o);
      return o != nullptr;
    };
    bool ok = put(0, Ko);
    ok = put(1, Vo) && ok;
    ok = put(2, idx) && ok;
    ok = put(3, scores) && ok;
    PyObject* b = PyBytes_FromStringAndSize((const char*)&pl, sizeof(pl));
    PyTuple_SET_ITEM(out, 4, b);
    if (ok && b) return out;
    Py_DECREF(out);
    return nullptr;
  } catch (...) {
    return none();
  }
}

// append(counters, K of the cache, S, L, r, variant, std_ddof, launch, workspace or None, K_new, V_new)
//   -> the status of lagkv_append_and_compress, or -1: not called
PyObject* append(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  auto status = [](long v) {
    PyErr_Clear();
    return PyLong_FromLong(v);
  };
  if (nargs != 11) return status(-1);
  try {
    int32_t dc, dk, dv;
    const at::Tensor *C = rows_of(args[1], &dc), *K = rows_of(args[9], &dk), *V = rows_of(args[10], &dv);
    lagkv_params p;
    void* stream;
    if (!C || !K || !V || dk != dc || dv != dc || !alike(*K, *V) || K->device() != C->device() ||
        K->size(0) != C->size(0) || K->size(1) != C->size(1) || K->size(3) != C->size(3) ||
        !params_of(args + 2, *K, dk, &p))
      return status(-1);
    const size_t need = workspace_fn(&p, C->size(2));
    void* w = nullptr;
    size_t ws_bytes = 0;
    if (args[8] != Py_None) {
      if (!THPVariable_CheckExact(args[8])) return status(-1);
      const at::Tensor& ws = THPVariable_Unpack(args[8]);
      w = ws.data_ptr();
      ws_bytes = (size_t)ws.numel();
    }
    if (ws_bytes < need || !stream_of(*C, &stream)) return status(-1);
    const void *k = K->data_ptr(), *v = V->data_ptr();
    const int64_t n_new = K->size(2);
    Py_buffer view;
    if (PyObject_GetBuffer(args[0], &view, PyBUF_WRITABLE) != 0) return status(-1);
    int rc = -1;
    if (view.len == (Py_ssize_t)sizeof(lagkv_cache)) {
      Py_BEGIN_ALLOW_THREADS
      rc = append_fn(&p, (lagkv_cache*)view.buf, k, v, n_new, w, ws_bytes, stream);
      Py_END_ALLOW_THREADS
    }
    PyBuffer_Release(&view);
    return status(rc);
  } catch (...) {
    return status(-1);
  }
}

// ---- the operators that read a cache ----

// An optional dense int32 tensor on `device`: false where it is there and is none.
bool ints_of(PyObject* o, const at::Tensor& like, const at::Tensor** t) {
  *t = nullptr;
  if (o == Py_None) return true;
  if (!THPVariable_CheckExact(o)) return false;
  *t = &THPVariable_Unpack(o);
  return (*t)->scalar_type() == at::kInt && (*t)->device() == like.device() && (*t)->layout() == at::kStrided && (*t)->is_contiguous();
}
bool small(const at::Tensor& t) {
  for (int64_t n : t.sizes())
    if (n > INT32_MAX) return false;
  return true;
}
// A backward pass or, of a dual tensor, a tangent that the operators do not give.
template <typename... Ts>
bool needs_grad(const Ts*... t) {
  return (c10::GradMode::is_enabled() && ((t && t->requires_grad()) || ...)) || ((t && t->_fw_grad(0).defined()) || ...);
}
bool device_is_current(const at::Tensor& t) {
  return c10::impl::VirtualGuardImpl(at::DeviceType::CUDA).getDevice() == t.device();
}
const void* at_of(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

// attend(q, K, V, K_new, V_new, parents, lengths, scale or None, out or None, want_lse, ws or None, blocks or None, block)
//   -> (out, lse or None), the status that the C function refused with, or None: not called
PyObject* attend(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 13 || !PyBool_Check(args[9])) return none();
  try {
    int32_t dq, dk, dv;
    const at::Tensor *q = rows_of(args[0], &dq), *K = rows_of(args[1], &dk), *V = rows_of(args[2], &dv);
    if (!q || !K || !V || dq != dk || dq != dv || q->device() != K->device() || !alike(*K, *V) || !small(*q) || !small(*K)) return none();
    lagkv_attend_params p = {};
    p.B = (int32_t)K->size(0);
    p.H = (int32_t)K->size(1);
    p.T = K->size(2);
    p.D = (int32_t)K->size(3);
    p.N = (int32_t)q->size(2);
    p.dtype = dq;
    if (q->size(0) != p.B || q->size(3) != p.D || p.H == 0 || q->size(1) % p.H != 0) return none();
    p.G = (int32_t)(q->size(1) / p.H);
    const at::Tensor *Kn = nullptr, *Vn = nullptr, *parents, *lengths, *blocks;
    if (args[3] != Py_None || args[4] != Py_None) {
      Kn = rows_of(args[3], &dk);
      Vn = rows_of(args[4], &dv);
      if (!Kn || !Vn || dk != dq || dv != dq || !alike(*Kn, *Vn) || Kn->device() != q->device() || Kn->size(0) != p.B ||
          Kn->size(1) != p.H || Kn->size(2) != p.N || Kn->size(3) != p.D)
        return none();
      p.new_stride_b = Kn->stride(0);
      p.new_stride_h = Kn->stride(1);
      p.new_stride_n = Kn->stride(2);
    }
    if (!ints_of(args[5], *q, &parents) || !ints_of(args[6], *q, &lengths) || !ints_of(args[11], *q, &blocks)) return none();
    if (parents) {
      if (!Kn || parents->dim() < 1 || parents->dim() > 2 || parents->size(-1) != p.N || (parents->dim() == 2 && parents->size(0) != p.B))
        return none();
      p.parents_stride_b = parents->dim() == 2 ? p.N : 0;
    }
    if (lengths && (lengths->dim() != 1 || lengths->size(0) != p.B)) return none();
    if (blocks) {
      if (blocks->dim() != 4 || blocks->size(0) != p.B || blocks->size(1) != p.H || blocks->size(2) != p.N ||
          blocks->size(3) > INT32_MAX || !to_int(args[12], &p.block))
        return none();
      p.n_blocks = (int32_t)blocks->size(3);
    }
    if (args[7] == Py_None) p.scale = 1.0 / std::sqrt((double)p.D);
    else if (!to_double(args[7], &p.scale)) return none();
    if (needs_grad(q, K, V, Kn, Vn) || !device_is_current(*q)) return none();
    p.q_stride_b = q->stride(0);
    p.q_stride_h = q->stride(1);
    p.q_stride_n = q->stride(2);
    p.kv_stride_b = K->stride(0);
    p.kv_stride_h = K->stride(1);
    p.kv_stride_t = K->stride(2);
    void* stream;
    if (!stream_of(*q, &stream)) return none();
    const auto opt = q->options().requires_grad(false);
    at::Tensor out, lse, ws;
    if (args[8] == Py_None) {
      out = at::empty_like(*q, opt);
      if (out.stride(3) != 1) return none();
    } else {
      int32_t d;
      const at::Tensor* given = rows_of(args[8], &d);
      if (!given || d != dq || given->device() != q->device() || given->sizes() != q->sizes()) return none();
      out = *given;
    }
    p.out_stride_b = out.stride(0);
    p.out_stride_h = out.stride(1);
    p.out_stride_n = out.stride(2);
    if (args[9] == Py_True) lse = at::empty({q->size(0), q->size(1), q->size(2)}, opt.dtype(at::kFloat));
    size_t need = attend_ws_fn(&p);
    if (args[10] != Py_None) {
      if (!THPVariable_CheckExact(args[10])) return none();
      ws = THPVariable_Unpack(args[10]);
      if (ws.scalar_type() != at::kByte || !ws.is_contiguous() || ws.device() != q->device()) return none();
      need = (size_t)ws.numel();
    } else if (need) {
      ws = at::empty({(int64_t)need}, opt.dtype(at::kByte));
    }
    const void *qp = q->data_ptr(), *kp = K->data_ptr(), *vp = V->data_ptr(), *knp = at_of(Kn), *vnp = at_of(Vn);
    const int32_t *pp = (const int32_t*)at_of(parents), *lp = (const int32_t*)at_of(lengths), *bp = (const int32_t*)at_of(blocks);
    void *op = out.data_ptr(), *wp = ws.defined() ? ws.data_ptr() : nullptr;
    float* ep = lse.defined() ? (float*)lse.data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = blocks ? attend_blocks_fn(&p, qp, kp, vp, lp, bp, knp, vnp, pp, op, ep, wp, need, stream)
                : attend_fn(&p, qp, kp, vp, lp, knp, vnp, pp, op, ep, wp, need, stream);
    Py_END_ALLOW_THREADS
    if (rc != LAGKV_OK) return PyLong_FromLong(rc);
    PyObject* o = args[8] == Py_None ? THPVariable_Wrap(out) : Py_NewRef(args[8]);
    PyObject* e = o ? (lse.defined() ? THPVariable_Wrap(lse) : Py_NewRef(Py_None)) : nullptr;
    PyObject* both = e ? PyTuple_Pack(2, o, e) : nullptr;
    Py_XDECREF(o);
    Py_XDECREF(e);
    return both;
  } catch (...) {
    return none();
  }
}

// select_blocks(q, lo, hi, T, block, k, first, last, lengths or None) -> blocks, a status, or None: not called
PyObject* select_blocks(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 9) return none();
  try {
    int32_t dq, dl, dh, first, last, T;
    const at::Tensor *q = rows_of(args[0], &dq), *lo = rows_of(args[1], &dl), *hi = rows_of(args[2], &dh), *lengths;
    if (!q || !lo || !hi || dq != dl || dq != dh || q->device() != lo->device() || !alike(*lo, *hi) || !small(*q) ||
        !small(*lo))
      return none();
    lagkv_attend_params p = {};
    if (!to_int(args[3], &T) || !to_int(args[4], &p.block) || !to_int(args[5], &p.n_blocks) || !to_int(args[6], &first) ||
        !to_int(args[7], &last) || !ints_of(args[8], *q, &lengths) || T < 0 || p.block < 1 || p.n_blocks < 1)
      return none();
    p.B = (int32_t)lo->size(0);
    p.H = (int32_t)lo->size(1);
    p.D = (int32_t)lo->size(3);
    p.N = (int32_t)q->size(2);
    p.dtype = dq;
    p.T = T;
    if (q->size(0) != p.B || q->size(3) != p.D || p.H == 0 || q->size(1) % p.H != 0 || lo->size(2) != ((int64_t)T + p.block - 1) / p.block ||
        (lengths && (lengths->dim() != 1 || lengths->size(0) != p.B)) || needs_grad(q, lo, hi) || !device_is_current(*q))
      return none();
    p.G = (int32_t)(q->size(1) / p.H);
    p.q_stride_b = q->stride(0);
    p.q_stride_h = q->stride(1);
    p.q_stride_n = q->stride(2);
    p.kv_stride_b = lo->stride(0);
    p.kv_stride_h = lo->stride(1);
    p.kv_stride_t = lo->stride(2);
    void* stream;
    if (!stream_of(*q, &stream)) return none();
    const auto opt = q->options().requires_grad(false);
    at::Tensor out = at::empty({p.B, p.H, p.N, p.n_blocks}, opt.dtype(at::kInt));
    const int64_t need = lo->size(0) * lo->size(1) * lo->size(2) * p.N * 8;
    at::Tensor ws = at::empty({need}, opt.dtype(at::kByte));
    const void *qp = q->data_ptr(), *lp = lo->data_ptr(), *hp = hi->data_ptr();
    const int32_t* np = (const int32_t*)at_of(lengths);
    int32_t* op = (int32_t*)out.data_ptr();
    void* wp = ws.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = select_fn(&p, qp, lp, hp, np, first, last, op, wp, (size_t)need, stream);
    Py_END_ALLOW_THREADS
    return rc == LAGKV_OK ? THPVariable_Wrap(out) : PyLong_FromLong(rc);
  } catch (...) {
    return none();
  }
}

// block_bounds(K, block, lengths or None, start, lo or None, hi or None) -> (lo, hi), a status, or None: not called
PyObject* block_bounds(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 6) return none();
  try {
    int32_t dk, dl, dh, start;
    const at::Tensor *K = rows_of(args[0], &dk), *lengths;
    lagkv_attend_params p = {};
    if (!K || !small(*K) || !to_int(args[1], &p.block) || !ints_of(args[2], *K, &lengths) || !to_int(args[3], &start) || p.block < 1) return none();
    p.B = (int32_t)K->size(0);
    p.H = (int32_t)K->size(1);
    p.D = (int32_t)K->size(3);
    p.T = K->size(2);
    p.dtype = dk;
    p.kv_stride_b = K->stride(0);
    p.kv_stride_h = K->stride(1);
    p.kv_stride_t = K->stride(2);
    if ((lengths && (lengths->dim() != 1 || lengths->size(0) != p.B)) || needs_grad(K) || !device_is_current(*K)) return none();
    const int64_t nb = (p.T + p.block - 1) / p.block;
    at::Tensor lo, hi;
    if (args[4] == Py_None && args[5] == Py_None) {
      if (start > 0) return none();
      const auto opt = K->options().requires_grad(false);
      lo = at::empty({p.B, p.H, nb, p.D}, opt);
      hi = at::empty({p.B, p.H, nb, p.D}, opt);
    } else {
      const at::Tensor *l = rows_of(args[4], &dl), *u = rows_of(args[5], &dh);
      if (!l || !u || dl != dk || dh != dk || l->device() != K->device() || !alike(*l, *u) || l->size(0) != p.B || l->size(1) != p.H || l->size(2) != nb || l->size(3) != p.D)
        return none();
      lo = *l;
      hi = *u;
    }
    p.out_stride_b = lo.stride(0);
    p.out_stride_h = lo.stride(1);
    p.out_stride_n = lo.stride(2);
    void* stream;
    if (!stream_of(*K, &stream)) return none();
    const void* kp = K->data_ptr();
    const int32_t* np = (const int32_t*)at_of(lengths);
    void *lp = lo.data_ptr(), *hp = hi.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = bounds_fn(&p, kp, np, start, lp, hp, stream);
    Py_END_ALLOW_THREADS
    if (rc != LAGKV_OK) return PyLong_FromLong(rc);
    if (args[4] != Py_None) return PyTuple_Pack(2, args[4], args[5]);
    PyObject* l = THPVariable_Wrap(lo);
    PyObject* u = l ? THPVariable_Wrap(hi) : nullptr;
    PyObject* both = u ? PyTuple_Pack(2, l, u) : nullptr;
    Py_XDECREF(l);
    Py_XDECREF(u);
    return both;
  } catch (...) {
    return none();
  }
}

// init(plan, workspace_bytes, compress, append_and_compress, attend_workspace_bytes, attend, attend_blocks, block_bounds,
//      select_blocks: addresses; raw stream function)
PyObject* init(PyObject*, PyObject* args) {
  size_t a[9];
  PyObject* f;
  static_assert(sizeof(size_t) == sizeof(unsigned long), "");
  if (!PyArg_ParseTuple(args, "kkkkkkkkkO", &a[0], &a[1], &a[2], &a[3], &a[4], &a[5], &a[6], &a[7], &a[8], &f)) return nullptr;
  plan_fn = (decltype(plan_fn))a[0];
  workspace_fn = (decltype(workspace_fn))a[1];
  compress_fn = (decltype(compress_fn))a[2];
  append_fn = (decltype(append_fn))a[3];
  attend_ws_fn = (decltype(attend_ws_fn))a[4];
  attend_fn = (decltype(attend_fn))a[5];
  attend_blocks_fn = (decltype(attend_blocks_fn))a[6];
  bounds_fn = (decltype(bounds_fn))a[7];
  select_fn = (decltype(select_fn))a[8];
  Py_INCREF(f);
  Py_XSETREF(raw_stream_fn, f);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"init", init, METH_VARARGS, nullptr},
    {"compress", (PyCFunction)(void (*)(void))compress, METH_FASTCALL, nullptr},
    {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, nullptr},
    {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
    {"select_blocks", (PyCFunction)(void (*)(void))select_blocks, METH_FASTCALL, nullptr},
    {"block_bounds", (PyCFunction)(void (*)(void))block_bounds, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lagkv_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lagkv_native(void) { return PyModule_Create(&module); }
