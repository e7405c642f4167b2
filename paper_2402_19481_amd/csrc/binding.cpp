// The operations of __init__.py that a caller issues one by one, bound natively: a few kernels of some microseconds each are waited for
// less than they take to issue.  Marshalling only: checks that a tensor is one the library can take, allocates the result with torch,
// and calls the C entry point on the current stream, with the interpreter released.  Per call ctypes and Python took 7 - 8 us of the host
// beside the launch, this 2; three calls of a small float32 block 30 -> 20 us.  The entry points are addresses that __init__.py hands over
// (of the library that it has loaded).
#include <Python.h>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

enum { kF32 = 0, kBF16 = 1 };
PyObject *g_error = nullptr, *g_torch_memory = nullptr, *g_torch_device = nullptr;   // DfError, torch.OutOfMemoryError, torch.AcceleratorError
const char* (*g_strerror)(int) = nullptr;

struct Failed {};                                      // a Python exception is set

[[noreturn]] void fail(PyObject* kind, const char* text) {
  PyErr_SetString(kind, text);
  throw Failed{};
}
const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a tensor");
  return THPVariable_Unpack(o);
}
// Device pointer of a tensor, nullptr for None
void* ptr(PyObject* o) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (!t.is_cuda() || !t.is_contiguous()) fail(g_error, "tensors must be contiguous and on the GPU");
  return t.data_ptr();
}
int dtype(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return kF32;
  if (t.scalar_type() == at::kBFloat16) return kBF16;
  PyErr_Format(g_error, "unsupported dtype torch.%s", t.scalar_type() == at::kHalf ? "float16" : c10::toString(t.scalar_type()));
  throw Failed{};
}
long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Failed{};
  return v;
}
int int32(PyObject* o) {
  const long long v = integer(o);
  if (v != (int)v) fail(PyExc_OverflowError, "integer out of range");
  return (int)v;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Failed{};
  return (float)v;
}
void dims(const at::Tensor& t, int64_t n, const char* text) {
  if (t.dim() != n) fail(PyExc_ValueError, text);
}
// `what` divided by a caller's number, as Python's // and with its exception
long long over(long long what, long long by) {
  if (by == 0) fail(PyExc_ZeroDivisionError, "integer division or modulo by zero");
  const long long q = what / by;
  return q * by != what && (what < 0) != (by < 0) ? q - 1 : q;
}
int small(long long v) {                               // (the C entry points refuse what is not positive)
  return v > 0x7fffffffLL ? fail(PyExc_OverflowError, "size out of range"), 0 : (int)v;
}
void* stream() { return (void*)c10::hip::getCurrentHIPStream().stream(); }
void check(int rc) {
  if (rc == 0) return;
  PyErr_Format(g_error, "libdistrifusion: %s (%d)", g_strerror(rc), rc);
  throw Failed{};
}
template <typename F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const Failed&) {
    return nullptr;
  } catch (python_error& e) {
    e.restore();
  } catch (const c10::OutOfMemoryError& e) {           // (as torch raises them: its own translation is not exported)
    PyErr_SetString(g_torch_memory, e.what_without_backtrace());
  } catch (const c10::AcceleratorError& e) {
    PyErr_SetString(g_torch_device, e.what_without_backtrace());
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
#define DF_ARGS(n) \
  if (na != (n)) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }
// The interpreter is released while torch allocates (its allocator may have to wait for others) and the library launches
struct Released {
  PyThreadState* state = PyEval_SaveThread();
  ~Released() { PyEval_RestoreThread(state); }
};

using GnFn = int (*)(const void*, void*, const float*, float*, const float*, const float*, int, int, int, int, int, int, int, float, int, int,
                     int, void*);
using ConvFn = int (*)(const void*, const void*, const void*, const float*, void*, int, int, int, int, int, int, int, int, int, int, int, void*);
using AttnFn = int (*)(const void*, const void*, const void*, const void*, const void*, void*, int, int, int, int, int, int, float, int, void*);
using AttnAxisFn = int (*)(const void*, const void*, const void*, const void*, const void*, void*, int, int, int, int, int, int, int, float, int,
                           int, void*);
using LinearFn = int (*)(const void*, const void*, const float*, const float*, void*, int, int, int, int, void*);
using RefreshFn = int (*)(void*, const void*, int, long long, int, int, int, void*);
GnFn g_gn;
ConvFn g_conv;
AttnFn g_attn;
AttnAxisFn g_attn_axis;
LinearFn g_linear;
RefreshFn g_refresh;

using RopeFn = int (*)(const void*, long long, long long, const void*, long long, long long, void*, long long, long long, void*, long long, long long,
                       const float*, const float*, const float*, const int*, int, int, int, int, int, int, int, int, float, int, int, void*);
using Kv4BytesFn = size_t (*)(int, int, int, int);
using Kv4RefreshFn = int (*)(void*, const void*, long long, long long, const void*, long long, long long, int, int, int, int, int, int, int, int, int,
                             void*);
using Kv4ReadFn = int (*)(const void*, void*, void*, int, int, int, int, int, void*);
using AttnKv4Fn = int (*)(const void*, long long, long long, const void*, const int*, void*, int, int, int, int, int, int, float, int, void*, size_t,
                          void*);
using AttnKv4BytesFn = size_t (*)(int, int, int, int, int, int, int);
using DisplacedKv4Fn = int (*)(const void*, long long, long long, const void*, long long, long long, const void*, long long, long long, const void*,
                               void*, int, int, int, int, int, int, int, int, float, int, int, void*, size_t, void*);
using DisplacedKv4BytesFn = size_t (*)(int, int, int, int, int, int, int, int, int, int);
using CrossFn = int (*)(const void*, long long, long long, const void*, long long, long long, const void*, long long, long long,
                        const unsigned char*, const int*, void*, int, int, int, int, int, int, float, int, void*, size_t, void*);
using CrossBytesFn = size_t (*)(int, int, int, int, int, int, int, int);
RopeFn g_rope;
Kv4BytesFn g_kv4_bytes;
Kv4RefreshFn g_kv4_refresh;
Kv4ReadFn g_kv4_read;
AttnKv4Fn g_attn_kv4;
AttnKv4BytesFn g_attn_kv4_bytes;
DisplacedKv4Fn g_displaced_kv4;
DisplacedKv4BytesFn g_displaced_kv4_bytes;
CrossFn g_cross;
CrossBytesFn g_cross_bytes;

// A tensor [B, tokens, heads, d] whose heads lie side by side: its address and the elements between tokens and batch items
struct Heads {
  void* p = nullptr;
  long long ld = 0, bs = 0;
  int B = 0, T = 0, H = 0, d = 0, dt = 0;
};
Heads heads(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o);
  if (t.dim() != 4) {
    PyErr_Format(PyExc_ValueError, "%s: expected [B, tokens, heads, d]", name);
    throw Failed{};
  }
  if (!t.is_cuda() || (t.size(3) > 1 && t.stride(3) != 1) || (t.size(2) > 1 && t.stride(2) != t.size(3))) {
    PyErr_Format(g_error, "%s must be on the GPU, the heads of a token side by side", name);
    throw Failed{};
  }
  Heads h;
  h.p = t.data_ptr();
  h.ld = t.size(1) > 1 ? t.stride(1) : 0;
  h.bs = t.size(0) > 1 ? t.stride(0) : 0;
  h.B = small(t.size(0)); h.T = small(t.size(1)); h.H = small(t.size(2)); h.d = small(t.size(3));
  h.dt = dtype(t);
  return h;
}
void same(const Heads& a, const Heads& b, bool tokens, bool nheads, const char* text) {
  if (a.B != b.B || a.d != b.d || (tokens && a.T != b.T) || (nheads && a.H != b.H)) fail(PyExc_ValueError, text);
  if (a.dt != b.dt) fail(g_error, "tensors must have the same type");
}
// A contiguous tensor of the given type and sizes on the device of `like`, nullptr for None
void* given(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> sizes, const at::Tensor& like, const char* name) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != type) {
    PyErr_Format(g_error, "%s: expected a tensor of torch.%s", name, c10::toString(type));
    throw Failed{};
  }
  if (t.sizes() != at::IntArrayRef(sizes)) {
    PyErr_Format(PyExc_ValueError, "%s: wrong shape", name);
    throw Failed{};
  }
  if (t.device() != like.device() || !t.is_contiguous()) fail(g_error, "tensors must be contiguous and on the same GPU");
  return t.data_ptr();
}
void together(const at::Tensor& a, PyObject* o) {
  if (o != Py_None && tensor(o).device() != a.device()) fail(g_error, "tensors must be on the same GPU");
}
// A 4-bit cache of these sizes.  kv4_cache makes it [d + 4, B, kv_heads, rows], so that sizes of as many bytes are told apart (and a slice along
// any of them is not contiguous or has other sizes); memory of a caller's own in another form goes by its bytes.
void* cache_of(PyObject* o, const at::Tensor& like, int B, long long L, int kv_heads, int d) {
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != at::kByte || !t.is_contiguous() || !t.is_cuda() || t.device() != like.device())
    fail(g_error, "cache: expected a tensor of kv4_cache on the same GPU");
  const size_t bytes = L > 0x7fffffffLL ? 0 : g_kv4_bytes(B, (int)L, kv_heads, d);
  const bool made = t.dim() == 4;
  if (bytes == 0 || (size_t)t.numel() != bytes || (made && (t.size(0) != d + 4 || t.size(1) != B || t.size(2) != kv_heads)))
    fail(PyExc_ValueError, "cache: not one of these sizes");
  return t.data_ptr();
}
at::Tensor result(const at::Tensor& q, PyObject* out, bool& made) {
  made = out == Py_None;
  if (made) return at::empty(q.sizes(), q.options());
  const at::Tensor& t = tensor(out);
  if (t.sizes() != q.sizes()) fail(PyExc_ValueError, "out: expected the shape of q");
  if (t.scalar_type() != q.scalar_type() || t.device() != q.device() || !t.is_contiguous())
    fail(g_error, "out must be contiguous, of q's type and on its GPU");
  return t;
}
at::Tensor workspace(const at::Tensor& q, size_t bytes) {
  return bytes ? at::empty({(int64_t)bytes}, q.options().dtype(at::kByte)) : at::Tensor();
}
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
float scale_of(PyObject* o, int d) { return o == Py_None ? (float)std::pow((double)d, -0.5) : real(o); }

// setup(DfError, torch.OutOfMemoryError, torch.AcceleratorError, addresses of df_strerror, df_groupnorm_stale, df_conv3x3_halo_axis,
// df_attn_displaced, df_attn_displaced_axis, df_linear, df_buffer_refresh, df_qk_norm_rope, df_kv4_bytes, df_kv4_refresh, df_kv4_read, df_attn_kv4,
// df_attn_kv4_workspace_bytes, df_attn_displaced_kv4, df_attn_displaced_kv4_workspace_bytes, df_cross_attn, df_cross_attn_workspace_bytes)
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(20)
  return guarded([&]() -> PyObject* {
    void* f[17];
    for (int i = 0; i < 17; ++i) f[i] = (void*)integer(a[i + 3]);
    PyObject** const kinds[] = {&g_error, &g_torch_memory, &g_torch_device};
    for (int i = 0; i < 3; ++i) {
      Py_INCREF(a[i]);
      Py_XDECREF(*kinds[i]);
      *kinds[i] = a[i];
    }
    g_strerror = (const char* (*)(int))f[0];
    g_gn = (GnFn)f[1]; g_conv = (ConvFn)f[2]; g_attn = (AttnFn)f[3]; g_attn_axis = (AttnAxisFn)f[4]; g_linear = (LinearFn)f[5];
    g_refresh = (RefreshFn)f[6];
    g_rope = (RopeFn)f[7]; g_kv4_bytes = (Kv4BytesFn)f[8]; g_kv4_refresh = (Kv4RefreshFn)f[9]; g_kv4_read = (Kv4ReadFn)f[10];
    g_attn_kv4 = (AttnKv4Fn)f[11]; g_attn_kv4_bytes = (AttnKv4BytesFn)f[12]; g_displaced_kv4 = (DisplacedKv4Fn)f[13];
    g_displaced_kv4_bytes = (DisplacedKv4BytesFn)f[14]; g_cross = (CrossFn)f[15]; g_cross_bytes = (CrossBytesFn)f[16];
    Py_RETURN_NONE;
  });
}

// x_fresh, stale_stats, gamma, beta, G, patch_idx, N, eps, stat_mode, fuse_silu, fresh_stats_out or None -> (y, fresh_stats)
PyObject* groupnorm_stale(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(11)
  return guarded([&] {
    const at::Tensor& x = tensor(a[0]);
    dims(x, 4, "x_fresh: expected [B, R, W, C]");
    const int G = int32(a[4]), patch = int32(a[5]), N = int32(a[6]), mode = int32(a[8]), silu = int32(a[9]);
    const float eps = real(a[7]);
    const void *xp = ptr(a[0]), *st = ptr(a[1]), *gm = ptr(a[2]), *bt = ptr(a[3]);
    void* fp = ptr(a[10]);
    const int dt = dtype(x), B = small(x.size(0)), R = small(x.size(1)), W = small(x.size(2)), C = small(x.size(3));
    at::Tensor y, fs;
    int rc;
    {
      Released r;
      y = at::empty_like(x);
      if (a[10] == Py_None) {
        fs = at::empty({B, G, 2}, x.options().dtype(at::kFloat));
        fp = fs.data_ptr();
      }
      rc = g_gn(xp, y.data_ptr(), (const float*)st, (float*)fp, (const float*)gm, (const float*)bt, B, R, W, C, G, patch, N, eps, mode, silu, dt,
                stream());
    }
    check(rc);
    PyObject* fo = a[10] == Py_None ? THPVariable_Wrap(std::move(fs)) : Py_NewRef(a[10]);
    PyObject* yo = THPVariable_Wrap(std::move(y));
    PyObject* t = PyTuple_Pack(2, yo, fo);
    Py_XDECREF(yo);
    Py_XDECREF(fo);
    return t;
  });
}

// x_fresh, stale_full, w, bias, patch_idx, N, stride, act, axis -> y
PyObject* conv3x3_halo(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(9)
  return guarded([&] {
    const at::Tensor &x = tensor(a[0]), &w = tensor(a[2]);
    dims(x, 4, "x_fresh: expected [B, R, W, Cin]");
    if (w.dim() < 1) fail(PyExc_ValueError, "w: expected [Cout, 3, 3, Cin]");
    const int patch = int32(a[4]), N = int32(a[5]), stride = int32(a[6]), act = int32(a[7]), axis = int32(a[8]);
    const long long Ro = over(x.size(1), stride), Wo = over(x.size(2), stride);
    const void *xp = ptr(a[0]), *sp = ptr(a[1]), *wp = ptr(a[2]), *bp = ptr(a[3]);
    const int dt = dtype(x), B = small(x.size(0)), Cin = small(x.size(3)), Cout = small(w.size(0));
    const int H = small(x.size(1) * (axis == 0 ? N : 1)), W = small(x.size(2) * (axis == 0 ? 1 : N));
    at::Tensor y;
    int rc;
    {
      Released r;
      y = at::empty({B, Ro, Wo, Cout}, x.options());
      rc = g_conv(xp, sp, wp, (const float*)bp, y.data_ptr(), B, H, W, Cin, Cout, patch, N, stride, act, dt, axis, stream());
    }
    check(rc);
    return THPVariable_Wrap(std::move(y));
  });
}

// q, k_fresh, v_fresh, k_stale, v_stale, heads, patch_idx, N, scale or None, out or None -> out
PyObject* attn_displaced(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(10)
  return guarded([&] {
    const at::Tensor& q = tensor(a[0]);
    dims(q, 3, "q: expected [B, Lq, C]");
    const int heads = int32(a[5]), patch = int32(a[6]), N = int32(a[7]);
    const long long d = over(q.size(2), heads);
    const float scale = a[8] == Py_None ? (float)std::pow((double)d, -0.5) : real(a[8]);
    const void *qp = ptr(a[0]), *kf = ptr(a[1]), *vf = ptr(a[2]), *ks = ptr(a[3]), *vs = ptr(a[4]);
    void* op = ptr(a[9]);
    const int dt = dtype(q), B = small(q.size(0)), L = small(q.size(1) * N), hd = small(d);
    at::Tensor out;
    int rc;
    {
      Released r;
      if (a[9] == Py_None) {
        out = at::empty_like(q);
        op = out.data_ptr();
      }
      rc = g_attn(qp, kf, vf, ks, vs, op, B, L, heads, hd, patch, N, scale, dt, stream());
    }
    check(rc);
    return a[9] == Py_None ? THPVariable_Wrap(std::move(out)) : Py_NewRef(a[9]);
  });
}

// q, k_fresh, v_fresh, k_stale, v_stale, heads, H, W, patch_idx, N, scale or None, axis -> out
PyObject* attn_displaced_axis(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(12)
  return guarded([&] {
    const at::Tensor& q = tensor(a[0]);
    dims(q, 3, "q: expected [B, Lq, C]");
    const int heads = int32(a[5]), H = int32(a[6]), W = int32(a[7]), patch = int32(a[8]), N = int32(a[9]), axis = int32(a[11]);
    const long long d = over(q.size(2), heads);
    const float scale = a[10] == Py_None ? (float)std::pow((double)d, -0.5) : real(a[10]);
    const void *qp = ptr(a[0]), *kf = ptr(a[1]), *vf = ptr(a[2]), *ks = ptr(a[3]), *vs = ptr(a[4]);
    const int dt = dtype(q), B = small(q.size(0)), hd = small(d);
    at::Tensor out;
    int rc;
    {
      Released r;
      out = at::empty_like(q);
      rc = g_attn_axis(qp, kf, vf, ks, vs, out.data_ptr(), B, H, W, heads, hd, patch, N, scale, dt, axis, stream());
    }
    check(rc);
    return THPVariable_Wrap(std::move(out));
  });
}

// x, w, bias, residual, out or None, dtype of a new out (0 float32, 1 bf16) -> out
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(6)
  return guarded([&] {
    const at::Tensor &x = tensor(a[0]), &w = tensor(a[1]);
    dims(x, 2, "x: expected [M, K]");
    if (w.dim() < 1) fail(PyExc_ValueError, "w: expected [N, K]");
    const void *xp = ptr(a[0]), *wp = ptr(a[1]), *bp = ptr(a[2]), *rp = ptr(a[3]);
    void* op = ptr(a[4]);
    const int dt = a[4] != Py_None ? dtype(tensor(a[4])) : int32(a[5]), M = small(x.size(0)), Nn = small(w.size(0)), K = small(x.size(1));
    at::Tensor out;
    int rc;
    {
      Released r;
      if (a[4] == Py_None) {
        out = at::empty({M, Nn}, x.options().dtype(dt == kF32 ? at::kFloat : at::kBFloat16));
        op = out.data_ptr();
      }
      rc = g_linear(xp, wp, (const float*)bp, (const float*)rp, op, M, Nn, K, dt, stream());
    }
    check(rc);
    return a[4] == Py_None ? THPVariable_Wrap(std::move(out)) : Py_NewRef(a[4]);
  });
}

// dst_full, src_patch, patch_idx, N -> dst_full
PyObject* buffer_refresh(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(4)
  return guarded([&] {
    const at::Tensor& t = tensor(a[0]);
    if (t.dim() < 1) fail(PyExc_ValueError, "dst_full: expected [B, ...]");
    const int patch = int32(a[2]), N = int32(a[3]), B = small(t.size(0));
    void *dp = ptr(a[0]), *sp = ptr(a[1]);
    const long long per = over(t.numel(), B);
    const int dt = dtype(t);
    int rc;
    {
      Released r;
      rc = g_refresh(dp, sp, B, per, patch, N, dt, stream());
    }
    check(rc);
    return Py_NewRef(a[0]);
  });
}

// q, k or None, q_gamma, k_gamma, rot, pos (None or tensors), eps, norm, interleaved, q_out, k_out (None or tensors) -> (q_out, k_out)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(11)
  return guarded([&] {
    const at::Tensor& q = tensor(a[0]);
    const Heads hq = heads(a[0], "q");
    Heads hk, oq, ok;
    if (a[1] != Py_None) {
      hk = heads(a[1], "k");
      same(hq, hk, true, false, "k: expected [B, T, kv_heads, d] like q");
      if (hk.H == 0) fail(PyExc_ValueError, "k: no heads");
      together(q, a[1]);
    } else if (a[10] != Py_None) {
      fail(PyExc_ValueError, "k_out without k");
    }
    const float eps = real(a[6]);
    const int norm = int32(a[7]), inter = int32(a[8]);
    const void *qg = given(a[2], at::kFloat, {hq.d}, q, "q_gamma"), *kg = given(a[3], at::kFloat, {hq.d}, q, "k_gamma");
    const void *rot = nullptr, *pos = given(a[5], at::kInt, {hq.B, hq.T}, q, "pos");
    int rot_dim = 0, rot_len = 0;
    if (a[4] != Py_None) {
      const at::Tensor& t = tensor(a[4]);
      dims(t, 3, "rot: expected [rows, rot_dim / 2, 2]");
      rot = given(a[4], at::kFloat, {t.size(0), t.size(1), 2}, q, "rot");
      rot_len = small(t.size(0));
      rot_dim = small(2 * t.size(1));
    }
    for (int i = 9; i < 11; ++i) {
      if (a[i] == Py_None) continue;
      Heads& o = i == 9 ? oq : ok;
      o = heads(a[i], i == 9 ? "q_out" : "k_out");
      same(i == 9 ? hq : hk, o, true, true, i == 9 ? "q_out: expected the shape of q" : "k_out: expected the shape of k");
      together(q, a[i]);
    }
    c10::OptionalDeviceGuard guard(q.device());
    at::Tensor qn, kn;
    int rc;
    {
      Released r;
      const auto fresh = [&](at::Tensor& t, Heads& o, const Heads& in) {
        t = at::empty({in.B, in.T, in.H, in.d}, q.options());
        o = in;
        o.p = t.data_ptr();
        o.ld = (long long)in.H * in.d;
        o.bs = o.ld * in.T;
      };
      if (!oq.p) fresh(qn, oq, hq);
      if (hk.p && !ok.p) fresh(kn, ok, hk);
      rc = g_rope(hq.p, hq.ld, hq.bs, hk.p, hk.ld, hk.bs, oq.p, oq.ld, oq.bs, ok.p, ok.ld, ok.bs, (const float*)qg, (const float*)kg,
                  (const float*)rot, (const int*)pos, hq.B, hq.T, hq.H, hk.H, hq.d, rot_dim, rot_len, norm, eps, inter, hq.dt, stream());
    }
    check(rc);
    PyObject* qo = qn.defined() ? THPVariable_Wrap(std::move(qn)) : Py_NewRef(a[9]);
    PyObject* ko = kn.defined() ? THPVariable_Wrap(std::move(kn)) : Py_NewRef(a[10]);
    PyObject* t = PyTuple_Pack(2, qo, ko);
    Py_XDECREF(qo);
    Py_XDECREF(ko);
    return t;
  });
}

// cache, k, v, H, W, patch_idx, N, axis -> cache.  H 0: W is ignored, the patch is k's tokens of N times as many
PyObject* kv4_refresh(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(8)
  return guarded([&] {
    const at::Tensor& k = tensor(a[1]);
    const Heads hk = heads(a[1], "k"), hv = heads(a[2], "v");
    same(hk, hv, true, true, "v: expected the shape of k");
    together(k, a[2]);
    int H = int32(a[3]), W = int32(a[4]);
    const int patch = int32(a[5]), N = int32(a[6]), axis = int32(a[7]);
    if (H == 0) { H = 1; W = small((long long)hk.T * N); }
    if (N > 0 && (long long)H * W != (long long)hk.T * N) fail(PyExc_ValueError, "k: expected the tokens of one patch");
    void* c = cache_of(a[0], k, hk.B, (long long)H * W, hk.H, hk.d);
    c10::OptionalDeviceGuard guard(k.device());
    int rc;
    {
      Released r;
      rc = g_kv4_refresh(c, hk.p, hk.ld, hk.bs, hv.p, hv.ld, hv.bs, hk.B, H, W, hk.H, hk.d, patch, N, hk.dt, axis, stream());
    }
    check(rc);
    return Py_NewRef(a[0]);
  });
}

// cache, B, L, kv_heads, d, dtype (0 float32, 1 bf16) -> (k, v)
PyObject* kv4_read(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(6)
  return guarded([&] {
    const at::Tensor& t = tensor(a[0]);
    const int B = int32(a[1]), L = int32(a[2]), H = int32(a[3]), d = int32(a[4]), dt = int32(a[5]);
    const void* c = cache_of(a[0], t, B, L, H, d);
    c10::OptionalDeviceGuard guard(t.device());
    at::Tensor k, v;
    int rc;
    {
      Released r;
      k = at::empty({B, L, H, d}, t.options().dtype(dt == kF32 ? at::kFloat : at::kBFloat16));
      v = at::empty_like(k);
      rc = g_kv4_read(c, k.data_ptr(), v.data_ptr(), B, L, H, d, dt, stream());
    }
    check(rc);
    PyObject* ko = THPVariable_Wrap(std::move(k));
    PyObject* vo = THPVariable_Wrap(std::move(v));
    PyObject* r = PyTuple_Pack(2, ko, vo);
    Py_XDECREF(ko);
    Py_XDECREF(vo);
    return r;
  });
}

// q, cache, L, kv_heads, lens or None, scale or None, out or None -> out
PyObject* attn_kv4(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(7)
  return guarded([&] {
    const at::Tensor& q = tensor(a[0]);
    const Heads h = heads(a[0], "q");
    const int L = int32(a[2]), kv = int32(a[3]);
    const void* c = cache_of(a[1], q, h.B, L, kv, h.d);
    const void* lens = given(a[4], at::kInt, {h.B}, q, "lens");
    const float scale = scale_of(a[5], h.d);
    c10::OptionalDeviceGuard guard(q.device());
    bool made;
    at::Tensor out = result(q, a[6], made);
    int rc;
    {
      Released r;
      const size_t bytes = g_attn_kv4_bytes(h.B, h.T, L, h.H, kv, h.d, h.dt);
      const at::Tensor w = workspace(q, bytes);
      rc = g_attn_kv4(h.p, h.ld, h.bs, c, (const int*)lens, out.data_ptr(), h.B, h.T, L, h.H, kv, h.d, scale, h.dt, address(w), bytes, stream());
    }
    check(rc);
    return made ? THPVariable_Wrap(std::move(out)) : Py_NewRef(a[6]);
  });
}

// q, k_fresh, v_fresh, cache, H (0: as kv4_refresh), W, patch_idx, N, scale or None, axis, out or None -> out
PyObject* attn_displaced_kv4(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(11)
  return guarded([&] {
    const at::Tensor& q = tensor(a[0]);
    const Heads h = heads(a[0], "q"), hk = heads(a[1], "k_fresh"), hv = heads(a[2], "v_fresh");
    same(h, hk, true, false, "k_fresh: expected [B, Lq, kv_heads, d] like q");
    same(hk, hv, true, true, "v_fresh: expected the shape of k_fresh");
    together(q, a[1]);
    together(q, a[2]);
    int H = int32(a[4]), W = int32(a[5]);
    const int patch = int32(a[6]), N = int32(a[7]), axis = int32(a[9]);
    if (H == 0) { H = 1; W = small((long long)h.T * N); }
    if (N > 0 && (long long)H * W != (long long)h.T * N) fail(PyExc_ValueError, "q: expected the tokens of one patch");
    const void* c = cache_of(a[3], q, h.B, (long long)H * W, hk.H, h.d);
    const float scale = scale_of(a[8], h.d);
    c10::OptionalDeviceGuard guard(q.device());
    bool made;
    at::Tensor out = result(q, a[10], made);
    int rc;
    {
      Released r;
      const size_t bytes = g_displaced_kv4_bytes(h.B, H, W, h.H, hk.H, h.d, patch, N, h.dt, axis);
      const at::Tensor w = workspace(q, bytes);
      rc = g_displaced_kv4(h.p, h.ld, h.bs, hk.p, hk.ld, hk.bs, hv.p, hv.ld, hv.bs, c, out.data_ptr(), h.B, H, W, h.H, hk.H, h.d, patch, N, scale, h.dt,
                           axis, address(w), bytes, stream());
    }
    check(rc);
    return made ? THPVariable_Wrap(std::move(out)) : Py_NewRef(a[10]);
  });
}

// q, k, v, key_mask, lens, scale, out (None or values) -> out
PyObject* cross_attn(PyObject*, PyObject* const* a, Py_ssize_t na) {
  DF_ARGS(7)
  return guarded([&] {
    const at::Tensor& q = tensor(a[0]);
    const Heads h = heads(a[0], "q"), hk = heads(a[1], "k"), hv = heads(a[2], "v");
    same(h, hk, false, false, "k: expected [B, Lk, kv_heads, d] like q");
    same(hk, hv, true, true, "v: expected the shape of k");
    together(q, a[1]);
    together(q, a[2]);
    const bool bytes_mask = a[3] != Py_None && tensor(a[3]).scalar_type() == at::kByte;
    const void* mask = given(a[3], bytes_mask ? at::kByte : at::kBool, {hk.B, hk.T}, q, "key_mask");
    const void* lens = given(a[4], at::kInt, {h.B}, q, "lens");
    const float scale = scale_of(a[5], h.d);
    c10::OptionalDeviceGuard guard(q.device());
    bool made;
    at::Tensor out = result(q, a[6], made);
    int rc;
    {
      Released r;
      const size_t bytes = g_cross_bytes(h.B, h.T, hk.T, h.H, hk.H, h.d, mask != nullptr, h.dt);
      const at::Tensor w = workspace(q, bytes);
      rc = g_cross(h.p, h.ld, h.bs, hk.p, hk.ld, hk.bs, hv.p, hv.ld, hv.bs, (const unsigned char*)mask, (const int*)lens, out.data_ptr(), h.B, h.T,
                   hk.T, h.H, hk.H, h.d, scale, h.dt, address(w), bytes, stream());
    }
    check(rc);
    return made ? THPVariable_Wrap(std::move(out)) : Py_NewRef(a[6]);
  });
}

#define DF_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {DF_METHOD(setup),  DF_METHOD(groupnorm_stale), DF_METHOD(conv3x3_halo), DF_METHOD(attn_displaced), DF_METHOD(attn_displaced_axis),
                         DF_METHOD(linear), DF_METHOD(buffer_refresh), DF_METHOD(qk_norm_rope), DF_METHOD(kv4_refresh), DF_METHOD(kv4_read),
                         DF_METHOD(attn_kv4), DF_METHOD(attn_displaced_kv4), DF_METHOD(cross_attn), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
