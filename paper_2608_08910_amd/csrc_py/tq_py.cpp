// Native half of the Python binding (tq.py): the argument checks and the C-ABI call of the
// entry points that a serving loop makes, in one C call. The checks through Python
// attributes and the ctypes conversion cost about 7 us a call, more than the smaller kernels
// take (2048 x 4096, one token: 4.4 us a call, 9.8 through Python).
//
// Every function returns the C status, or None if an argument is not exactly what the call
// needs: the caller then takes the Python path, which names the fault. Nothing is cached:
// each call checks its own arguments.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include "../../include/tq.h"

namespace {

struct Api {
  decltype(&tq_quantize_act) quantize_act;
  decltype(&tq_gemv) gemv;
  decltype(&tq_gemv_f32) gemv_f32;
  decltype(&tq_gemv2) gemv2;
  decltype(&tq_gemv_mx) gemv_mx;
  decltype(&tq_moe_grouped) moe_grouped;
  decltype(&tq_route) route;
  decltype(&tq_route_balance) route_balance;
  decltype(&tq_route_bwd) route_bwd;
  decltype(&tq_moe_weight_grad) weight_grad;
  decltype(&tq_block_norm) block_norm;
  decltype(&tq_block_norm_bwd) block_norm_bwd;
  decltype(&tq_lora) lora;
  decltype(&tq_lora_bwd) lora_bwd;
  decltype(&tq_quantize_mx) quantize_mx;
  decltype(&tq_gemm_mx) gemm_mx;
  decltype(&tq_gemm_mx_bwd) gemm_mx_bwd;
  decltype(&tq_gated_mx) gated_mx;
  decltype(&tq_gated_mx_bwd) gated_mx_bwd;
} api;

// A plain contiguous device tensor of this type and shape (dims: its nd sizes; dev_any: of any).
struct Arg {
  void* ptr = nullptr;
  bool ok = false;
};

Arg dev_sizes(PyObject* o, at::ScalarType dt, int nd, const int64_t* dims) {
  Arg a;
  if (!THPVariable_CheckExact(o)) return a;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.scalar_type() != dt || !t.is_contiguous()) return a;
  if (nd >= 0) {
    if (t.dim() != nd) return a;
    for (int i = 0; i < nd; ++i)
      if (t.size(i) != dims[i]) return a;
  }
  a.ptr = t.data_ptr();
  a.ok = true;
  return a;
}

template <typename... D>
Arg dev(PyObject* o, at::ScalarType dt, D... d) {
  const int64_t dims[] = {(int64_t)d...};
  return dev_sizes(o, dt, (int)sizeof...(d), dims);
}

Arg dev_any(PyObject* o, at::ScalarType dt) { return dev_sizes(o, dt, -1, nullptr); }

bool to_i64(PyObject* o, int64_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  *v = PyLong_AsLongLongAndOverflow(o, &over);
  return over == 0;
}
bool to_i32(PyObject* o, int64_t* v) { return to_i64(o, v) && *v >= INT32_MIN && *v <= INT32_MAX; }

// sizes of a plain 2-D tensor
bool sizes2(PyObject* o, int64_t* a, int64_t* b) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.dim() != 2) return false;
  *a = t.size(0);
  *b = t.size(1);
  return true;
}

// C++ exceptions (a tensor without storage, say) also mean the Python path.
template <typename F>
PyObject* call(F f) {
  int64_t st = 0;
  bool ok = false;
  try {
    ok = f(&st);
  } catch (...) {
    ok = false;
  }
  if (PyErr_Occurred()) PyErr_Clear();
  if (!ok) Py_RETURN_NONE;
  return PyLong_FromLongLong(st);
}

template <typename F>
int64_t unlocked(F f) {
  PyThreadState* s = PyEval_SaveThread();
  const int64_t st = f();
  PyEval_RestoreThread(s);
  return st;
}

constexpr auto kF32 = at::kFloat, kI8 = at::kChar, kU8 = at::kByte, kI16 = at::kShort, kI32 = at::kInt;

// (x, q, d, bsum, stream)
PyObject* py_quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call([&](int64_t* st) {
    int64_t t, k, stream;
    if (n != 5 || !sizes2(a[0], &t, &k) || k > INT32_MAX || !to_i64(a[4], &stream)) return false;
    const Arg x = dev(a[0], kF32, t, k), q = dev(a[1], kI8, t, k), d = dev(a[2], kF32, t, k / 256),
              b = dev(a[3], kI32, t, k / 256);
    if (!x.ok || !q.ok || !d.ok || !b.ok) return false;
    *st = unlocked([&] {
      return api.quantize_act((const float*)x.ptr, t, (int32_t)k, (int8_t*)q.ptr, (float*)d.ptr, (int32_t*)b.ptr, (void*)stream);
    });
    return true;
  });
}

// (n, k, codes, scales, x, y, q, d, bsum, stream)
PyObject* py_gemv_f32(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return call([&](int64_t* st) {
    int64_t n, k, t, kx, stream;
    if (nargs != 10 || !to_i32(a[0], &n) || !to_i32(a[1], &k) || k < 0 || !sizes2(a[4], &t, &kx) || !to_i64(a[9], &stream))
      return false;
    const int64_t kb = k / 256;
    const Arg c = dev(a[2], kU8, n, kb, 128), s = dev(a[3], kI16, n, kb), x = dev(a[4], kF32, t, k), y = dev(a[5], kF32, t, n),
              q = dev(a[6], kI8, t, k), d = dev(a[7], kF32, t, kb), b = dev(a[8], kI32, t, kb);
    if (!c.ok || !s.ok || !x.ok || !y.ok || !q.ok || !d.ok || !b.ok) return false;
    const tq_mat m = {(int32_t)n, (int32_t)k, (uint8_t*)c.ptr, (uint16_t*)s.ptr};
    *st = unlocked([&] {
      return api.gemv_f32(&m, (const float*)x.ptr, t, (float*)y.ptr, (int8_t*)q.ptr, (float*)d.ptr, (int32_t*)b.ptr, nullptr,
                          (void*)stream);
    });
    return true;
  });
}

// (n, k, codes, scales, q, d, bsum, y, stream)
PyObject* py_gemv(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return call([&](int64_t* st) {
    int64_t n, k, t, kq, stream;
    if (nargs != 9 || !to_i32(a[0], &n) || !to_i32(a[1], &k) || k < 0 || !sizes2(a[4], &t, &kq) || !to_i64(a[8], &stream))
      return false;
    const int64_t kb = k / 256;
    const Arg c = dev(a[2], kU8, n, kb, 128), s = dev(a[3], kI16, n, kb), q = dev(a[4], kI8, t, k), d = dev(a[5], kF32, t, kb),
              b = dev(a[6], kI32, t, kb), y = dev(a[7], kF32, t, n);
    if (!c.ok || !s.ok || !q.ok || !d.ok || !b.ok || !y.ok) return false;
    const tq_mat m = {(int32_t)n, (int32_t)k, (uint8_t*)c.ptr, (uint16_t*)s.ptr};
    *st = unlocked([&] {
      return api.gemv(&m, (const int8_t*)q.ptr, (const float*)d.ptr, (const int32_t*)b.ptr, t, (float*)y.ptr, nullptr,
                      (void*)stream);
    });
    return true;
  });
}

// (n, k, codes, scales, q, d, y, stream)
template <typename Mat, typename Scale>
PyObject* gemv_planes(PyObject* const* a, Py_ssize_t nargs, tq_status (*fn)(const Mat*, const int8_t*, const float*, int64_t, float*, int32_t*, void*),
                      Arg (*scales)(PyObject*, int64_t, int64_t)) {
  return call([&](int64_t* st) {
    int64_t n, k, t, kq, stream;
    if (nargs != 8 || !to_i32(a[0], &n) || !to_i32(a[1], &k) || k < 0 || !sizes2(a[4], &t, &kq) || !to_i64(a[7], &stream))
      return false;
    const int64_t kb = k / 256;
    const Arg c = dev(a[2], kU8, n, kb, 128), s = scales(a[3], n, k), q = dev(a[4], kI8, t, k), d = dev(a[5], kF32, t, kb),
              y = dev(a[6], kF32, t, n);
    if (!c.ok || !s.ok || !q.ok || !d.ok || !y.ok) return false;
    const Mat m = {(int32_t)n, (int32_t)k, (uint8_t*)c.ptr, (Scale*)s.ptr};
    *st = unlocked([&] {
      return fn(&m, (const int8_t*)q.ptr, (const float*)d.ptr, t, (float*)y.ptr, nullptr, (void*)stream);
    });
    return true;
  });
}
PyObject* py_gemv2(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return gemv_planes<tq_mat2, uint16_t>(a, n, api.gemv2,
                                        [](PyObject* o, int64_t r, int64_t k) { return dev(o, kI16, r, k / 256, (int64_t)2); });
}
PyObject* py_gemv_mx(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return gemv_planes<tq_mat_mx, uint8_t>(a, n, api.gemv_mx,
                                         [](PyObject* o, int64_t r, int64_t k) { return dev(o, kU8, r, k / 32); });
}

// (n_experts, hidden, inter, codes tuple, scales tuple, x, topk_idx, topk_w, out, ws, flags, stream)
PyObject* py_moe_grouped(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return call([&](int64_t* st) {
    int64_t E, H, I, t, h, t2, topk, flags, stream;
    if (nargs != 12 || !to_i32(a[0], &E) || !to_i32(a[1], &H) || !to_i32(a[2], &I) || H < 0 || I < 0 || !sizes2(a[5], &t, &h) ||
        h != H || !sizes2(a[6], &t2, &topk) || t2 != t || topk > INT32_MAX || !to_i32(a[10], &flags) || !to_i64(a[11], &stream))
      return false;
    if (!PyTuple_CheckExact(a[3]) || !PyTuple_CheckExact(a[4]) || PyTuple_GET_SIZE(a[3]) != 3 || PyTuple_GET_SIZE(a[4]) != 3)
      return false;
    const int64_t rows[3] = {I, I, H}, kbs[3] = {H / 256, H / 256, I / 256};
    Arg c[3], s[3];
    for (int p = 0; p < 3; ++p) {
      c[p] = dev(PyTuple_GET_ITEM(a[3], p), kU8, E, rows[p], kbs[p], (int64_t)128);
      s[p] = dev(PyTuple_GET_ITEM(a[4], p), kI16, E, rows[p], kbs[p]);
      if (!c[p].ok || !s[p].ok) return false;
    }
    const Arg x = dev(a[5], kF32, t, H), idx = dev(a[6], kI32, t, topk), w = dev(a[7], kF32, t, topk), out = dev(a[8], kF32, t, H),
              ws = dev_any(a[9], kU8);
    if (!x.ok || !idx.ok || !w.ok || !out.ok || !ws.ok) return false;
    tq_experts ex{};
    ex.n_experts = (int32_t)E;
    ex.hidden = (int32_t)H;
    ex.inter = (int32_t)I;
    ex.gate_codes = (uint8_t*)c[0].ptr;
    ex.gate_scales = (uint16_t*)s[0].ptr;
    ex.up_codes = (uint8_t*)c[1].ptr;
    ex.up_scales = (uint16_t*)s[1].ptr;
    ex.down_codes = (uint8_t*)c[2].ptr;
    ex.down_scales = (uint16_t*)s[2].ptr;
    for (int p = 0; p < 3; ++p) {
      ex.stride_codes[p] = rows[p] * kbs[p] * 128;
      ex.stride_scales[p] = rows[p] * kbs[p];
    }
    const size_t wsn = (size_t)THPVariable_Unpack(a[9]).numel();
    *st = unlocked([&] {
      return api.moe_grouped(&ex, (const float*)x.ptr, t, (const int32_t*)idx.ptr, (const float*)w.ptr, (int32_t)topk,
                             (float*)out.ptr, ws.ptr, wsn, (int32_t)flags, (void*)stream);
    });
    return true;
  });
}

// ---- around the frozen passes. Their tensors may be fp32, bfloat16 or fp16, some may be None, and all
// of a call's lie on the current device.

struct Call {
  int64_t device;
  bool ok = true;

  void* take(PyObject* o, at::ScalarType dt, int nd, const int64_t* dims) {
    const Arg a = dev_sizes(o, dt, nd, dims);
    if (!a.ok || THPVariable_Unpack(o).get_device() != device) ok = false;
    return a.ptr;
  }
  template <typename T = void, typename... D>
  T* need(PyObject* o, at::ScalarType dt, D... d) {
    const int64_t dims[] = {(int64_t)d...};
    return (T*)take(o, dt, (int)sizeof...(d), dims);
  }
  template <typename T = void, typename... D>
  T* maybe(PyObject* o, at::ScalarType dt, D... d) {
    return o == Py_None ? nullptr : need<T>(o, dt, d...);
  }
  void* workspace(PyObject* o, size_t* n) {
    void* p = take(o, kU8, -1, nullptr);
    if (ok) *n = (size_t)THPVariable_Unpack(o).numel();
    return p;
  }
};

// fp32, bfloat16 or fp16 as the library names it
bool elem_type(PyObject* o, at::ScalarType* dt, int32_t* ty) {
  if (!THPVariable_CheckExact(o)) return false;
  *dt = THPVariable_Unpack(o).scalar_type();
  if (*dt == kF32) *ty = TQ_F32;
  else if (*dt == at::kBFloat16) *ty = TQ_BF16;
  else if (*dt == at::kHalf) *ty = TQ_F16;
  else return false;
  return true;
}

bool to_f32(PyObject* o, float* v) {
  if (!PyFloat_CheckExact(o)) return false;
  *v = (float)PyFloat_AS_DOUBLE(o);
  return true;
}

struct RouteArgs {
  Call c;
  int64_t t, e, k, flags, stream;
  at::ScalarType dt;
  int32_t ty;
  const void* logits;
  int32_t* idx;
  float* w;
  const uint8_t* mask;
};
// (logits, topk_idx, topk_w, token_mask, flags, ..., device, stream), nargs of them
bool route_args(PyObject* const* a, Py_ssize_t n, Py_ssize_t nargs, RouteArgs* r) {
  int64_t t2;
  if (n != nargs || !sizes2(a[0], &r->t, &r->e) || !sizes2(a[1], &t2, &r->k) || t2 != r->t || r->e > INT32_MAX || r->k > INT32_MAX ||
      !to_i32(a[4], &r->flags) || !elem_type(a[0], &r->dt, &r->ty) || !to_i64(a[nargs - 2], &r->c.device) ||
      !to_i64(a[nargs - 1], &r->stream))
    return false;
  r->logits = r->c.need(a[0], r->dt, r->t, r->e);
  r->idx = r->c.need<int32_t>(a[1], kI32, r->t, r->k);
  r->w = r->c.need<float>(a[2], kF32, r->t, r->k);
  r->mask = r->c.maybe<uint8_t>(a[3], kU8, r->t);
  return r->c.ok;
}

PyObject* py_route(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call([&](int64_t* st) {
    RouteArgs r;
    if (!route_args(a, n, 7, &r)) return false;
    *st = unlocked([&] {
      return api.route(r.logits, r.ty, r.t, (int32_t)r.e, r.mask, (int32_t)r.k, (int32_t)r.flags, r.idx, r.w, (void*)r.stream);
    });
    return true;
  });
}

// (logits, topk_idx, topk_w, token_mask, flags, counts, p_mean, coef, loss, ws, alpha, device, stream)
PyObject* py_route_balance(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call([&](int64_t* st) {
    RouteArgs r;
    float alpha;
    size_t wsn = 0;
    if (!route_args(a, n, 13, &r) || !to_f32(a[10], &alpha)) return false;
    int32_t* counts = r.c.need<int32_t>(a[5], kI32, r.e);
    float *mean = r.c.need<float>(a[6], kF32, r.e), *coef = r.c.need<float>(a[7], kF32, r.e), *loss = r.c.need<float>(a[8], kF32, 1);
    void* ws = r.c.workspace(a[9], &wsn);
    if (!r.c.ok) return false;
    *st = unlocked([&] {
      return api.route_balance(r.logits, r.ty, r.t, (int32_t)r.e, r.mask, (int32_t)r.k, (int32_t)r.flags, alpha, r.idx, r.w, counts,
                               mean, coef, loss, ws, wsn, (void*)r.stream);
    });
    return true;
  });
}

// (logits, topk_idx, topk_w, token_mask, flags, dlogits, dw, coef, dloss, device, stream)
PyObject* py_route_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call([&](int64_t* st) {
    RouteArgs r;
    if (!route_args(a, n, 11, &r)) return false;
    void* dl = r.c.need(a[5], r.dt, r.t, r.e);
    const float *dw = r.c.maybe<float>(a[6], kF32, r.t, r.k), *coef = r.c.maybe<float>(a[7], kF32, r.e),
                *dloss = r.c.maybe<float>(a[8], kF32, 1);
    if (!r.c.ok) return false;
    *st = unlocked([&] {
      return api.route_bwd(r.logits, r.ty, r.t, (int32_t)r.e, r.mask, (int32_t)r.k, (int32_t)r.flags, r.idx, r.w, dw, coef, dloss, dl,
                           (void*)r.stream);
    });
    return true;
  });
}

// (yd, dout, topk_idx, dw, n_experts, device, stream)
PyObject* py_weight_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call([&](int64_t* st) {
    Call c;
    int64_t t, h, t2, k, e, stream;
    if (n != 7 || !sizes2(a[1], &t, &h) || !sizes2(a[2], &t2, &k) || t2 != t || h > INT32_MAX || k > INT32_MAX || !to_i32(a[4], &e) ||
        !to_i64(a[5], &c.device) || !to_i64(a[6], &stream))
      return false;
    const float *yd = c.need<float>(a[0], kF32, t * k, h), *dout = c.need<float>(a[1], kF32, t, h);
    const int32_t* idx = c.need<int32_t>(a[2], kI32, t, k);
    float* dw = c.need<float>(a[3], kF32, t, k);
    if (!c.ok) return false;
    *st = unlocked([&] { return api.weight_grad(yd, dout, t, (int32_t)h, idx, (int32_t)k, (int32_t)e, dw, (void*)stream); });
    return true;
  });
}

struct NormArgs {
  Call c;
  int64_t t, h, stream;
  at::ScalarType xdt, ydt;
  int32_t xt, yt, kind = TQ_GATE_NONE;
  const float *g_post, *gate, *g_pre;
  float rs, eps;
};
// the stream tensor and one of the block's; (g_post, gate, res_scale, g_pre, eps) at a + 4, (device, stream) last
bool norm_args(PyObject* const* a, Py_ssize_t n, Py_ssize_t nargs, PyObject* x, PyObject* y, NormArgs* r) {
  if (!sizes2(x, &r->t, &r->h) || r->h > INT32_MAX || !elem_type(x, &r->xdt, &r->xt) || !elem_type(y, &r->ydt, &r->yt) ||
      !to_f32(a[6], &r->rs) || !to_f32(a[8], &r->eps) || !to_i64(a[nargs - 2], &r->c.device) || !to_i64(a[nargs - 1], &r->stream))
    return false;
  r->g_post = r->c.maybe<float>(a[4], kF32, r->h);
  r->g_pre = r->c.maybe<float>(a[7], kF32, r->h);
  r->gate = nullptr;
  if (a[5] != Py_None) {
    if (!THPVariable_CheckExact(a[5])) return false;
    const bool channel = THPVariable_Unpack(a[5]).dim() == 1;
    r->kind = channel ? TQ_GATE_CHANNEL : TQ_GATE_TOKEN;
    r->gate = channel ? r->c.need<float>(a[5], kF32, r->h) : r->c.need<float>(a[5], kF32, r->t, 1);
  }
  return r->c.ok;
}

// (x, y, x_out, h, g_post, gate, res_scale, g_pre, eps, device, stream)
PyObject* py_block_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call([&](int64_t* st) {
    NormArgs r;
    if (n != 11 || !norm_args(a, n, 11, a[0], a[1] != Py_None ? a[1] : a[3], &r)) return false;
    const void *x = r.c.need(a[0], r.xdt, r.t, r.h), *y = r.c.maybe(a[1], r.ydt, r.t, r.h);
    void *xo = r.c.maybe(a[2], r.xdt, r.t, r.h), *h = r.c.maybe(a[3], r.ydt, r.t, r.h);
    if (!r.c.ok) return false;
    *st = unlocked([&] {
      return api.block_norm(x, r.xt, y, r.yt, r.t, (int32_t)r.h, r.g_post, r.gate, r.kind, r.rs, r.g_pre, r.eps, xo, h, (void*)r.stream);
    });
    return true;
  });
}

// (x_out, y, dx, dy, g_post, gate, res_scale, g_pre, eps, dx_out, dh, dg_post, dgate, dg_pre, ws, device, stream)
PyObject* py_block_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call([&](int64_t* st) {
    NormArgs r;
    size_t wsn = 0;
    if (n != 17 || !norm_args(a, n, 17, a[2], a[3] != Py_None ? a[3] : a[10], &r)) return false;
    const void *xo = r.c.maybe(a[0], r.xdt, r.t, r.h), *y = r.c.maybe(a[1], r.ydt, r.t, r.h), *dxo = r.c.maybe(a[9], r.xdt, r.t, r.h),
               *dh = r.c.maybe(a[10], r.ydt, r.t, r.h);
    void *dx = r.c.need(a[2], r.xdt, r.t, r.h), *dy = r.c.maybe(a[3], r.ydt, r.t, r.h);
    float *dgp = r.c.maybe<float>(a[11], kF32, r.h), *dpre = r.c.maybe<float>(a[13], kF32, r.h);
    if (a[12] != Py_None && r.kind == TQ_GATE_NONE) return false;
    float* dgate = r.kind == TQ_GATE_TOKEN ? r.c.maybe<float>(a[12], kF32, r.t, 1) : r.c.maybe<float>(a[12], kF32, r.h);
    void* ws = r.c.workspace(a[14], &wsn);
    if (!r.c.ok) return false;
    *st = unlocked([&] {
      return api.block_norm_bwd(xo, r.xt, y, r.yt, r.t, (int32_t)r.h, r.g_post, r.gate, r.kind, r.rs, r.g_pre, r.eps, dxo, dh, dx, dy,
                                dgp, dgate, dpre, ws, wsn, (void*)r.stream);
    });
    return true;
  });
}

// (a, b, scale, ranks, x, ids, ..., ws, device, stream): the descriptor, x and ids
bool lora_args(PyObject* const* a, Py_ssize_t n, Py_ssize_t nargs, Call* c, tq_adapters* ad, int64_t* t, const float** x,
               const int32_t** ids, void** ws, size_t* wsn, int64_t* stream) {
  int64_t kx;
  at::ScalarType dt;
  if (n != nargs || !THPVariable_CheckExact(a[0]) || !THPVariable_CheckExact(a[1]) || !elem_type(a[0], &dt, &ad->type) ||
      !sizes2(a[4], t, &kx) || !to_i64(a[nargs - 2], &c->device) || !to_i64(a[nargs - 1], stream))
    return false;
  const at::Tensor &ta = THPVariable_Unpack(a[0]), &tb = THPVariable_Unpack(a[1]);
  if (ta.dim() != 3 || tb.dim() != 3 || ta.numel() == 0 || tb.numel() == 0) return false;
  const int64_t na = ta.size(0), r = ta.size(1), k = ta.size(2), nn = tb.size(1);
  if (na > INT32_MAX || r > INT32_MAX || k > INT32_MAX || nn > INT32_MAX) return false;
  ad->n_adapters = (int32_t)na;
  ad->rank = (int32_t)r;
  ad->n = (int32_t)nn;
  ad->k = (int32_t)k;
  ad->a = c->need(a[0], dt, na, r, k);
  ad->b = c->need(a[1], dt, na, nn, r);
  ad->scale = c->maybe<float>(a[2], kF32, na);
  ad->ranks = c->maybe<int32_t>(a[3], kI32, na);
  *x = c->need<float>(a[4], kF32, *t, k);
  *ids = c->need<int32_t>(a[5], kI32, *t);
  *ws = c->workspace(a[nargs - 3], wsn);
  return c->ok;
}

// (a, b, scale, ranks, x, ids, y, out, v, ws, device, stream)
PyObject* py_lora(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call([&](int64_t* st) {
    Call c;
    tq_adapters ad{};
    int64_t t, stream;
    const float* x;
    const int32_t* ids;
    void* ws;
    size_t wsn = 0;
    if (!lora_args(a, n, 12, &c, &ad, &t, &x, &ids, &ws, &wsn, &stream)) return false;
    const float* y = c.maybe<float>(a[6], kF32, t, ad.n);
    float *out = c.need<float>(a[7], kF32, t, ad.n), *v = c.maybe<float>(a[8], kF32, t, ad.rank);
    if (!c.ok) return false;
    *st = unlocked([&] { return api.lora(&ad, x, t, ids, y, out, v, ws, wsn, (void*)stream); });
    return true;
  });
}

// (a, b, scale, ranks, x, ids, v, dy, da, db, dx, out, ws, device, stream)
PyObject* py_lora_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call([&](int64_t* st) {
    Call c;
    tq_adapters ad{};
    int64_t t, stream;
    const float* x;
    const int32_t* ids;
    void* ws;
    size_t wsn = 0;
    if (!lora_args(a, n, 15, &c, &ad, &t, &x, &ids, &ws, &wsn, &stream)) return false;
    const float *v = c.need<float>(a[6], kF32, t, ad.rank), *dy = c.need<float>(a[7], kF32, t, ad.n),
                *dx = c.maybe<float>(a[10], kF32, t, ad.k);
    float *da = c.need<float>(a[8], kF32, ad.n_adapters, ad.rank, ad.k), *db = c.need<float>(a[9], kF32, ad.n_adapters, ad.n, ad.rank),
          *out = c.maybe<float>(a[11], kF32, t, ad.k);
    if (!c.ok) return false;
    *st = unlocked([&] { return api.lora_bwd(&ad, x, v, dy, t, ids, dx, out, da, db, ws, wsn, (void*)stream); });
    return true;
  });
}

// ---- MXFP4 feed-forward block

// A matrix of n rows: its four arguments from a[0] (n, k, codes, scales).
bool mat_mx(PyObject* const* a, Call* c, tq_mat_mx* m) {
  int64_t n, k;
  if (!to_i32(a[0], &n) || !to_i32(a[1], &k) || n < 0 || k < 0) return false;
  m->n = (int32_t)n;
  m->k = (int32_t)k;
  m->codes = c->need<uint8_t>(a[2], kU8, n, k / 256, (int64_t)128);
  m->scales = c->need<uint8_t>(a[3], kU8, n, k / 32);
  return c->ok;
}

// (x, codes, scales, values, flags, device, stream)
PyObject* py_quantize_mx(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return call([&](int64_t* st) {
    Call c;
    int64_t t, k, flags, stream;
    at::ScalarType dt;
    int32_t ty;
    if (nargs != 7 || !sizes2(a[0], &t, &k) || k > INT32_MAX || !elem_type(a[0], &dt, &ty) || !to_i32(a[4], &flags) ||
        !to_i64(a[5], &c.device) || !to_i64(a[6], &stream))
      return false;
    const void* x = c.need(a[0], dt, t, k);
    uint8_t *codes = c.maybe<uint8_t>(a[1], kU8, t, k / 256, (int64_t)128), *scales = c.maybe<uint8_t>(a[2], kU8, t, k / 32);
    void* values = c.maybe(a[3], dt, t, k);
    if (!c.ok) return false;
    *st = unlocked([&] { return api.quantize_mx(x, ty, t, (int32_t)k, (int32_t)flags, codes, scales, values, (void*)stream); });
    return true;
  });
}

// (w: n, k, codes, scales, x: the same, y, device, stream)
PyObject* py_gemm_mx(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return call([&](int64_t* st) {
    Call c;
    int64_t stream;
    at::ScalarType dt;
    int32_t ty;
    tq_mat_mx w, x;
    if (nargs != 11 || !elem_type(a[8], &dt, &ty) || !to_i64(a[9], &c.device) || !to_i64(a[10], &stream) || !mat_mx(a, &c, &w) ||
        !mat_mx(a + 4, &c, &x))
      return false;
    void* y = c.need(a[8], dt, x.n, w.n);
    if (!c.ok) return false;
    *st = unlocked([&] { return api.gemm_mx(&w, &x, ty, y, (void*)stream); });
    return true;
  });
}

// (w: n, k, codes, scales, dy, dx, ws, device, stream)
PyObject* py_gemm_mx_bwd(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return call([&](int64_t* st) {
    Call c;
    int64_t t, n, stream;
    at::ScalarType dt;
    int32_t ty;
    size_t wsn = 0;
    tq_mat_mx w;
    if (nargs != 9 || !sizes2(a[4], &t, &n) || !elem_type(a[4], &dt, &ty) || !to_i64(a[7], &c.device) || !to_i64(a[8], &stream) ||
        !mat_mx(a, &c, &w))
      return false;
    const void* dy = c.need(a[4], dt, t, w.n);
    void *dx = c.need(a[5], dt, t, w.k), *ws = c.workspace(a[6], &wsn);
    if (!c.ok) return false;
    *st = unlocked([&] { return api.gemm_mx_bwd(&w, dy, ty, t, dx, ws, wsn, (void*)stream); });
    return true;
  });
}

// (gate: n, k, codes, scales, up, x: the same, h, act, g_add, u_add, g, u, device, stream)
PyObject* py_gated_mx(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return call([&](int64_t* st) {
    Call c;
    int64_t act, stream;
    at::ScalarType dt;
    int32_t ty;
    tq_mat_mx gate, up, x;
    if (nargs != 20 || !elem_type(a[12], &dt, &ty) || !to_i32(a[13], &act) || !to_i64(a[18], &c.device) || !to_i64(a[19], &stream) ||
        !mat_mx(a, &c, &gate) || !mat_mx(a + 4, &c, &up) || !mat_mx(a + 8, &c, &x))
      return false;
    const int64_t t = x.n, n = gate.n;
    void* h = c.need(a[12], dt, t, n);
    const float *ga = c.maybe<float>(a[14], kF32, t, n), *ua = c.maybe<float>(a[15], kF32, t, n);
    void *g = c.maybe(a[16], dt, t, n), *u = c.maybe(a[17], dt, t, n);
    if (!c.ok) return false;
    *st = unlocked([&] { return api.gated_mx(&gate, &up, &x, (int32_t)act, ga, ua, ty, h, g, u, (void*)stream); });
    return true;
  });
}

// (gate: n, k, codes, scales, up: the same, g, u, dh, dg, du, dx, ws, act, device, stream)
PyObject* py_gated_mx_bwd(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return call([&](int64_t* st) {
    Call c;
    int64_t t, n, act, stream;
    at::ScalarType dt;
    int32_t ty;
    size_t wsn = 0;
    tq_mat_mx gate, up;
    if (nargs != 18 || !sizes2(a[10], &t, &n) || !elem_type(a[10], &dt, &ty) || !to_i32(a[15], &act) || !to_i64(a[16], &c.device) ||
        !to_i64(a[17], &stream) || !mat_mx(a, &c, &gate) || !mat_mx(a + 4, &c, &up) || n != gate.n)
      return false;
    const void *g = c.need(a[8], dt, t, n), *u = c.need(a[9], dt, t, n), *dh = c.need(a[10], dt, t, n);
    void *dg = c.need(a[11], dt, t, n), *du = c.need(a[12], dt, t, n), *dx = c.maybe(a[13], dt, t, gate.k);
    void* ws = a[14] == Py_None ? nullptr : c.workspace(a[14], &wsn);
    if (!c.ok) return false;
    *st = unlocked([&] {
      return api.gated_mx_bwd(&gate, &up, (int32_t)act, ty, t, g, u, dh, dg, du, dx, ws, wsn, (void*)stream);
    });
    return true;
  });
}

// bind(addresses of the C entry points, in the order of Api)
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr int kEntries = sizeof(Api) / sizeof(void*);
  int64_t v[kEntries];
  if (n != kEntries) {
    PyErr_Format(PyExc_TypeError, "bind: %d addresses", kEntries);
    return nullptr;
  }
  for (int i = 0; i < kEntries; ++i)
    if (!to_i64(a[i], &v[i])) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "bind: an address is not an int");
      return nullptr;
    }
  api.quantize_act = reinterpret_cast<decltype(api.quantize_act)>(v[0]);
  api.gemv = reinterpret_cast<decltype(api.gemv)>(v[1]);
  api.gemv_f32 = reinterpret_cast<decltype(api.gemv_f32)>(v[2]);
  api.gemv2 = reinterpret_cast<decltype(api.gemv2)>(v[3]);
  api.gemv_mx = reinterpret_cast<decltype(api.gemv_mx)>(v[4]);
  api.moe_grouped = reinterpret_cast<decltype(api.moe_grouped)>(v[5]);
  api.route = reinterpret_cast<decltype(api.route)>(v[6]);
  api.route_balance = reinterpret_cast<decltype(api.route_balance)>(v[7]);
  api.route_bwd = reinterpret_cast<decltype(api.route_bwd)>(v[8]);
  api.weight_grad = reinterpret_cast<decltype(api.weight_grad)>(v[9]);
  api.block_norm = reinterpret_cast<decltype(api.block_norm)>(v[10]);
  api.block_norm_bwd = reinterpret_cast<decltype(api.block_norm_bwd)>(v[11]);
  api.lora = reinterpret_cast<decltype(api.lora)>(v[12]);
  api.lora_bwd = reinterpret_cast<decltype(api.lora_bwd)>(v[13]);
  api.quantize_mx = reinterpret_cast<decltype(api.quantize_mx)>(v[14]);
  api.gemm_mx = reinterpret_cast<decltype(api.gemm_mx)>(v[15]);
  api.gemm_mx_bwd = reinterpret_cast<decltype(api.gemm_mx_bwd)>(v[16]);
  api.gated_mx = reinterpret_cast<decltype(api.gated_mx)>(v[17]);
  api.gated_mx_bwd = reinterpret_cast<decltype(api.gated_mx_bwd)>(v[18]);
  Py_RETURN_NONE;
}

#define TQ_PY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {TQ_PY(bind),  TQ_PY(quantize_act), TQ_PY(gemv),        TQ_PY(gemv_f32),
                         TQ_PY(gemv2), TQ_PY(gemv_mx),      TQ_PY(moe_grouped), TQ_PY(route),
                         TQ_PY(route_balance), TQ_PY(route_bwd), TQ_PY(weight_grad), TQ_PY(block_norm),
                         TQ_PY(block_norm_bwd), TQ_PY(lora), TQ_PY(lora_bwd), TQ_PY(quantize_mx), TQ_PY(gemm_mx),
                         TQ_PY(gemm_mx_bwd), TQ_PY(gated_mx), TQ_PY(gated_mx_bwd), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tqpy", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tqpy() { return PyModule_Create(&module); }
