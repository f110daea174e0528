// The entry points' usual case in native code: what binding.py does with the tensors of a call (their sizes, strides, types and
// addresses, the current stream) took 3.5 of the 7.3 us of a small one, as much as the library and the runtime; here 0.4.
// A function looks at its arguments as binding.py passes them on. Where they are plain tensors on the current GPU of the shapes and types that
// the entry point takes, with an output tensor given and no stream, it makes the call and returns the output, or raises what
// the library's status stands for: the call is made once (a second one could succeed after a launch error that an
// earlier call had left, and an accumulating GEMM would have added twice). Everything else returns None: binding.py then goes
// through it step by step, allocates, or raises.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/mlt.h"

namespace {

// the library's functions, as binding.py has loaded them
decltype(&mlt_gemm) call_gemm;
decltype(&mlt_gemm_bias_act) call_gemm_bias_act;
decltype(&mlt_gemm_acc) call_gemm_acc;
decltype(&mlt_mha_fwd) call_mha_fwd;
decltype(&mlt_paged_attn_decode) call_paged;
decltype(&mlt_quant_fp8) call_quant_fp8;
decltype(&mlt_gemm_fp8) call_gemm_fp8;
decltype(&mlt_paged_append) call_append;
decltype(&mlt_paged_append_fp8) call_append_fp8;
decltype(&mlt_paged_attn_decode_fp8) call_paged_fp8;
PyObject* error_class;      // binding.MltError(status, where)

// A plain tensor with memory of its own kind on GPU `device` (-1: the first one sets it), or null
const at::Tensor* plain(PyObject* o, int& device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || !t.has_storage() || t.layout() != at::kStrided) return nullptr;
  if (device < 0) device = t.device().index();
  return t.device().index() == device ? &t : nullptr;
}

int dtype_code(const at::Tensor& t) {
  const auto s = t.scalar_type();
  return s == at::kBFloat16 ? MLT_BF16 : s == at::kHalf ? MLT_FP16 : -1;
}

// leading dimension of a matrix with contiguous rows, or -1
int64_t row_stride(const at::Tensor& t) {
  if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) return -1;
  return t.size(0) > 1 ? t.stride(0) : t.size(1) > 1 ? t.size(1) : 1;
}

struct Gemm {
  int64_t M, N, K, lda, ldb, ldc;
  int dtype, device = -1;
  void *a, *b, *c, *stream;
};

bool on_current_device(int device, void** stream) {
  if (c10::hip::current_device() != device) return false;
  *stream = c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream();
  return true;
}

bool gemm_operands(PyObject* A, PyObject* B, PyObject* C, bool transB, bool c_is_fp32, Gemm& g) {
  const at::Tensor *a = plain(A, g.device), *b = a ? plain(B, g.device) : nullptr, *c = b ? plain(C, g.device) : nullptr;
  if (!c) return false;
  g.dtype = dtype_code(*a);
  if (g.dtype < 0 || b->scalar_type() != a->scalar_type()) return false;
  if (c->scalar_type() != (c_is_fp32 ? at::kFloat : a->scalar_type())) return false;
  g.lda = row_stride(*a);
  g.ldb = row_stride(*b);
  g.ldc = row_stride(*c);
  if (g.lda < 0 || g.ldb < 0 || g.ldc < 0) return false;
  g.M = a->size(0);
  g.K = a->size(1);
  g.N = transB ? b->size(0) : b->size(1);
  if ((transB ? b->size(1) : b->size(0)) != g.K || c->size(0) != g.M || c->size(1) != g.N) return false;
  if (!on_current_device(g.device, &g.stream)) return false;
  g.a = a->data_ptr();
  g.b = b->data_ptr();
  g.c = c->data_ptr();
  return true;
}

PyObject* result(int rc, PyObject* out, const char* where) {
  if (rc != MLT_OK) {
    if (PyObject* e = PyObject_CallFunction(error_class, "is", rc, where)) {
      PyErr_SetObject(error_class, e);
      Py_DECREF(e);
    }
    return nullptr;
  }
  Py_INCREF(out);
  return out;
}

// gemm(A, B, C, transB, stream)
PyObject* py_gemm(PyObject*, PyObject* const* v, Py_ssize_t n) {
  Gemm g;
  if (n != 5 || v[4] != Py_None || !PyBool_Check(v[3]) || !gemm_operands(v[0], v[1], v[2], v[3] == Py_True, false, g)) Py_RETURN_NONE;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call_gemm(g.M, g.N, g.K, g.a, g.lda, g.b, g.ldb, v[3] == Py_True, g.c, g.ldc, g.dtype, g.stream);
  Py_END_ALLOW_THREADS
  return result(rc, v[2], "mlt_gemm");
}

// gemm_acc(A, B, C, transB, stream)
PyObject* py_gemm_acc(PyObject*, PyObject* const* v, Py_ssize_t n) {
  Gemm g;
  if (n != 5 || v[4] != Py_None || !PyBool_Check(v[3]) || !gemm_operands(v[0], v[1], v[2], v[3] == Py_True, true, g)) Py_RETURN_NONE;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call_gemm_acc(g.M, g.N, g.K, g.a, g.lda, g.b, g.ldb, v[3] == Py_True, (float*)g.c, g.ldc, g.dtype, g.stream);
  Py_END_ALLOW_THREADS
  return result(rc, v[2], "mlt_gemm_acc");
}

// gemm_bias_act(A, B, bias, act, C, transB, stream)
PyObject* py_gemm_bias_act(PyObject*, PyObject* const* v, Py_ssize_t n) {
  Gemm g;
  if (n != 7 || v[6] != Py_None || !PyBool_Check(v[5]) || !PyLong_CheckExact(v[3])) Py_RETURN_NONE;
  int overflow = 0;
  const long act = PyLong_AsLongAndOverflow(v[3], &overflow);
  if (overflow || act < 0 || act > 2 || !gemm_operands(v[0], v[1], v[4], v[5] == Py_True, false, g)) Py_RETURN_NONE;
  void* bias = nullptr;
  if (v[2] != Py_None) {
    const at::Tensor* t = plain(v[2], g.device);
    if (!t || dtype_code(*t) != g.dtype || t->dim() != 1 || t->size(0) != g.N || !t->is_contiguous()) Py_RETURN_NONE;
    bias = t->data_ptr();
  }
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call_gemm_bias_act(g.M, g.N, g.K, g.a, g.lda, g.b, g.ldb, v[5] == Py_True, bias, (int)act, g.c, g.ldc, g.dtype, g.stream);
  Py_END_ALLOW_THREADS
  return result(rc, v[4], "mlt_gemm_bias_act");
}

// mha_fwd(Q, K, V, scale, causal, O, stream)
PyObject* py_mha_fwd(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 7 || v[6] != Py_None || !PyFloat_CheckExact(v[3]) || !PyBool_Check(v[4])) Py_RETURN_NONE;
  int device = -1;
  const at::Tensor* t[4];
  PyObject* const o[4] = {v[0], v[1], v[2], v[5]};
  for (int i = 0; i < 4; ++i) {
    t[i] = plain(o[i], device);
    if (!t[i] || t[i]->dim() != 4 || !t[i]->is_contiguous() || t[i]->scalar_type() != t[0]->scalar_type()) Py_RETURN_NONE;
  }
  const at::Tensor &q = *t[0], &k = *t[1];
  const int dtype = dtype_code(q);
  if (dtype < 0 || k.size(0) != q.size(0) || k.size(1) != q.size(1) || k.size(3) != q.size(3)) Py_RETURN_NONE;
  if (t[2]->sizes() != k.sizes() || t[3]->sizes() != q.sizes()) Py_RETURN_NONE;
  void* stream;
  if (!on_current_device(device, &stream)) Py_RETURN_NONE;
  const int64_t B = q.size(0), H = q.size(1), Sq = q.size(2), Sk = k.size(2), D = q.size(3);
  void* p[4];
  for (int i = 0; i < 4; ++i) p[i] = t[i]->data_ptr();
  const float scale = (float)PyFloat_AS_DOUBLE(v[3]);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call_mha_fwd(B, H, Sq, Sk, D, p[0], p[1], p[2], p[3], scale, v[4] == Py_True, dtype, stream);
  Py_END_ALLOW_THREADS
  return result(rc, v[5], "mlt_mha_fwd");
}

// paged_attn_decode(Q, Kc, Vc, block_table, seq_lens, scale, O)
PyObject* py_paged(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 7 || !PyFloat_CheckExact(v[5])) Py_RETURN_NONE;
  int device = -1;
  const at::Tensor* t[6];
  PyObject* const o[6] = {v[0], v[1], v[2], v[3], v[4], v[6]};
  for (int i = 0; i < 6; ++i) {
    t[i] = plain(o[i], device);
    if (!t[i] || !t[i]->is_contiguous()) Py_RETURN_NONE;
  }
  const at::Tensor &q = *t[0], &kc = *t[1], &vc = *t[2], &table = *t[3], &lens = *t[4], &out = *t[5];
  const int dtype = dtype_code(q);
  if (dtype < 0 || q.dim() != 3 || kc.dim() != 4 || kc.size(1) != q.size(1) || kc.size(3) != q.size(2)) Py_RETURN_NONE;
  if (vc.sizes() != kc.sizes() || kc.scalar_type() != q.scalar_type() || vc.scalar_type() != q.scalar_type()) Py_RETURN_NONE;
  if (table.scalar_type() != at::kInt || lens.scalar_type() != at::kInt || table.dim() != 2 || lens.dim() != 1) Py_RETURN_NONE;
  if (table.size(0) != q.size(0) || lens.size(0) != q.size(0)) Py_RETURN_NONE;
  if (out.scalar_type() != q.scalar_type() || out.sizes() != q.sizes()) Py_RETURN_NONE;
  void* stream;
  if (!on_current_device(device, &stream)) Py_RETURN_NONE;
  const int64_t B = q.size(0), H = q.size(1), D = q.size(2), block = kc.size(2), blocks = table.size(1), num = kc.size(0);
  void* p[6];
  for (int i = 0; i < 6; ++i) p[i] = t[i]->data_ptr();
  const float scale = (float)PyFloat_AS_DOUBLE(v[5]);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call_paged(B, H, D, block, blocks, num, p[0], p[1], p[2], (const int32_t*)p[3], (const int32_t*)p[4], p[5], scale, dtype, stream);
  Py_END_ALLOW_THREADS
  return result(rc, v[6], "mlt_paged_attn_decode");
}

// ---- the 8-bit operators

bool is(const at::Tensor& t, at::ScalarType type) { return t.scalar_type() == type; }
bool sized(const at::Tensor& t, int64_t a, int64_t b) { return t.dim() == 2 && t.size(0) == a && t.size(1) == b; }

// quant_fp8(X, block_rows, Xq, S, stream)
PyObject* py_quant_fp8(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 5 || v[4] != Py_None || !PyLong_CheckExact(v[1])) Py_RETURN_NONE;
  int overflow = 0, device = -1;
  const long rows = PyLong_AsLongAndOverflow(v[1], &overflow);
  if (overflow || rows < 1) Py_RETURN_NONE;
  const at::Tensor *x = plain(v[0], device), *q = x ? plain(v[2], device) : nullptr, *s = q ? plain(v[3], device) : nullptr;
  if (!s) Py_RETURN_NONE;
  const int dtype = dtype_code(*x);
  const int64_t ldx = row_stride(*x), ldq = row_stride(*q), lds = row_stride(*s);
  if (dtype < 0 || ldx < 0 || ldq < 0 || lds < 0 || !is(*q, at::kFloat8_e4m3fn) || !is(*s, at::kFloat) || q->sizes() != x->sizes()) Py_RETURN_NONE;
  const int64_t M = x->size(0), K = x->size(1);
  if (!sized(*s, (K + 127) / 128, (M + rows - 1) / rows)) Py_RETURN_NONE;
  void* stream;
  if (!on_current_device(device, &stream)) Py_RETURN_NONE;
  void *px = x->data_ptr(), *pq = q->data_ptr(), *ps = s->data_ptr();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call_quant_fp8(M, K, px, ldx, rows, pq, ldq, (float*)ps, lds, dtype, stream);
  Py_END_ALLOW_THREADS
  PyObject* out = PyTuple_Pack(2, v[2], v[3]);
  if (!out) return nullptr;
  PyObject* r = result(rc, out, "mlt_quant_fp8");
  Py_DECREF(out);
  return r;
}

// gemm_fp8(A, Sa, B, Sb, C, stream)
PyObject* py_gemm_fp8(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 6 || v[5] != Py_None) Py_RETURN_NONE;
  int device = -1;
  const at::Tensor* t[5];
  int64_t ld[5];
  for (int i = 0; i < 5; ++i) {
    t[i] = plain(v[i], device);
    if (!t[i] || (ld[i] = row_stride(*t[i])) < 0) Py_RETURN_NONE;
  }
  const at::Tensor &a = *t[0], &sa = *t[1], &b = *t[2], &sb = *t[3], &c = *t[4];
  const int dtype = dtype_code(c);
  if (dtype < 0 || !is(a, at::kFloat8_e4m3fn) || !is(b, at::kFloat8_e4m3fn) || !is(sa, at::kFloat) || !is(sb, at::kFloat)) Py_RETURN_NONE;
  const int64_t M = a.size(0), K = a.size(1), N = b.size(0), kb = (K + 127) / 128;
  if (b.size(1) != K || !sized(sa, kb, M) || !sized(sb, kb, (N + 127) / 128) || !sized(c, M, N)) Py_RETURN_NONE;
  void* stream;
  if (!on_current_device(device, &stream)) Py_RETURN_NONE;
  void* p[5];
  for (int i = 0; i < 5; ++i) p[i] = t[i]->data_ptr();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call_gemm_fp8(M, N, K, p[0], ld[0], (const float*)p[1], ld[1], p[2], ld[2], (const float*)p[3], ld[3], p[4], ld[4], dtype, stream);
  Py_END_ALLOW_THREADS
  return result(rc, v[4], "mlt_gemm_fp8");
}

// Row stride of [T, heads, D] whose heads lie side by side, or -1
int64_t head_rows(const at::Tensor& t, int64_t T, int64_t D) {
  if (t.dim() != 3 || t.size(0) != T || t.size(2) != D || (D > 1 && t.stride(2) != 1) || (t.size(1) > 1 && t.stride(1) != D)) return -1;
  return T > 1 ? t.stride(0) : t.size(1) * D;
}

// paged_append(Q, K, V, offsets, seq_lens, block_table, cos, sin, Kc, Vc, Ks, Vs, Qo, interleaved, stream): with queries, angles and a
// Qo; without Ks and Vs (None): the 16-bit cache
PyObject* py_append(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 15 || v[14] != Py_None || !PyBool_Check(v[13])) Py_RETURN_NONE;
  const bool fp8 = v[10] != Py_None;
  int device = -1;
  const at::Tensor* t[13];
  for (int i = 0; i < 13; ++i) {
    t[i] = nullptr;
    if (!fp8 && (i == 10 || i == 11)) continue;
    t[i] = plain(v[i], device);
    if (!t[i] || (i > 2 && !t[i]->is_contiguous())) Py_RETURN_NONE;
  }
  const at::Tensor &q = *t[0], &k = *t[1], &vv = *t[2], &offsets = *t[3], &lens = *t[4], &table = *t[5], &cs = *t[6], &sn = *t[7], &kc = *t[8], &vc = *t[9], &qo = *t[12];
  const int dtype = dtype_code(k);
  if (dtype < 0 || k.dim() != 3 || q.dim() != 3 || !is(q, k.scalar_type()) || !is(vv, k.scalar_type()) || !is(qo, k.scalar_type())) Py_RETURN_NONE;
  const int64_t T = k.size(0), H = k.size(1), D = k.size(2), Hq = q.size(1);
  const int64_t ldq = head_rows(q, T, D), ldk = head_rows(k, T, D), ldv = head_rows(vv, T, D);
  if (ldq < 0 || ldk < 0 || ldv < 0 || vv.size(1) != H || qo.sizes() != q.sizes()) Py_RETURN_NONE;
  if (!is(offsets, at::kInt) || !is(lens, at::kInt) || !is(table, at::kInt) || offsets.dim() != 1 || lens.dim() != 1 || table.dim() != 2) Py_RETURN_NONE;
  const int64_t B = lens.size(0);
  if (offsets.size(0) != B + 1 || table.size(0) != B) Py_RETURN_NONE;
  if (!is(cs, at::kFloat) || !is(sn, at::kFloat) || cs.dim() != 2 || cs.sizes() != sn.sizes()) Py_RETURN_NONE;
  const at::ScalarType want = fp8 ? at::kFloat8_e4m3fn : k.scalar_type();
  if (!is(kc, want) || !is(vc, want) || kc.dim() != 4 || kc.size(1) != H || kc.size(3) != D || vc.sizes() != kc.sizes()) Py_RETURN_NONE;
  const int64_t nb = kc.size(0);
  for (int i = 10; fp8 && i < 12; ++i)
    if (!is(*t[i], at::kFloat) || !sized(*t[i], nb, H)) Py_RETURN_NONE;
  void* stream;
  if (!on_current_device(device, &stream)) Py_RETURN_NONE;
  void* p[13];
  for (int i = 0; i < 13; ++i) p[i] = t[i] ? t[i]->data_ptr() : nullptr;
  const int64_t bs = kc.size(2), per = table.size(1), rot = 2 * cs.size(1), positions = cs.size(0);
  const int pairs = v[13] == Py_True;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  if (fp8)
    rc = call_append_fp8(T, B, Hq, H, D, bs, per, nb, p[0], ldq, p[1], ldk, p[2], ldv, (const int32_t*)p[3], (const int32_t*)p[4], (const int32_t*)p[5], (const float*)p[6],
                         (const float*)p[7], rot, positions, pairs, p[12], p[8], p[9], (float*)p[10], (float*)p[11], dtype, stream);
  else
    rc = call_append(T, B, Hq, H, D, bs, per, nb, p[0], ldq, p[1], ldk, p[2], ldv, (const int32_t*)p[3], (const int32_t*)p[4], (const int32_t*)p[5], (const float*)p[6],
                     (const float*)p[7], rot, positions, pairs, p[12], p[8], p[9], dtype, stream);
  Py_END_ALLOW_THREADS
  return result(rc, v[12], fp8 ? "mlt_paged_append_fp8" : "mlt_paged_append");
}

// paged_attn_decode_fp8(Q, Kc, Vc, Ks, Vs, block_table, seq_lens, scale, O, stream)
PyObject* py_paged_fp8(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 10 || v[9] != Py_None || !PyFloat_CheckExact(v[7])) Py_RETURN_NONE;
  int device = -1;
  const at::Tensor* t[8];
  PyObject* const o[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[8]};
  for (int i = 0; i < 8; ++i) {
    t[i] = plain(o[i], device);
    if (!t[i] || !t[i]->is_contiguous()) Py_RETURN_NONE;
  }
  const at::Tensor &q = *t[0], &kc = *t[1], &vc = *t[2], &table = *t[5], &lens = *t[6], &out = *t[7];
  const int dtype = dtype_code(q);
  if (dtype < 0 || q.dim() != 3 || kc.dim() != 4 || kc.size(3) != q.size(2) || vc.sizes() != kc.sizes()) Py_RETURN_NONE;
  if (!is(kc, at::kFloat8_e4m3fn) || !is(vc, at::kFloat8_e4m3fn)) Py_RETURN_NONE;
  const int64_t nb = kc.size(0), H = kc.size(1), B = q.size(0);
  for (int i = 3; i < 5; ++i)
    if (!is(*t[i], at::kFloat) || !sized(*t[i], nb, H)) Py_RETURN_NONE;
  if (!is(table, at::kInt) || !is(lens, at::kInt) || table.dim() != 2 || lens.dim() != 1 || table.size(0) != B || lens.size(0) != B) Py_RETURN_NONE;
  if (!is(out, q.scalar_type()) || out.sizes() != q.sizes()) Py_RETURN_NONE;
  void* stream;
  if (!on_current_device(device, &stream)) Py_RETURN_NONE;
  void* p[8];
  for (int i = 0; i < 8; ++i) p[i] = t[i]->data_ptr();
  const int64_t Hq = q.size(1), D = q.size(2), bs = kc.size(2), per = table.size(1);
  const float scale = (float)PyFloat_AS_DOUBLE(v[7]);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call_paged_fp8(B, Hq, H, D, bs, per, nb, p[0], p[1], p[2], (const float*)p[3], (const float*)p[4], (const int32_t*)p[5], (const int32_t*)p[6], p[7], scale, dtype, stream);
  Py_END_ALLOW_THREADS
  return result(rc, v[8], "mlt_paged_attn_decode_fp8");
}

// A torch error in here (a tensor without memory behind it, say) is binding.py's to meet again
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* v, Py_ssize_t n) {
  try {
    return F(self, v, n);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// bind(error class, gemm, gemm_bias_act, gemm_acc, mha_fwd, paged_attn_decode[, quant_fp8, gemm_fp8, paged_append, paged_append_fp8,
// paged_attn_decode_fp8]): the library functions' addresses; those that are left out stay as they are
PyObject* py_bind(PyObject*, PyObject* args) {
  Py_ssize_t a[10] = {};
  PyObject* err;
  if (!PyArg_ParseTuple(args, "Onnnnn|nnnnn", &err, &a[0], &a[1], &a[2], &a[3], &a[4], &a[5], &a[6], &a[7], &a[8], &a[9])) return nullptr;
  Py_INCREF(err);
  error_class = err;
  call_gemm = reinterpret_cast<decltype(call_gemm)>(a[0]);
  call_gemm_bias_act = reinterpret_cast<decltype(call_gemm_bias_act)>(a[1]);
  call_gemm_acc = reinterpret_cast<decltype(call_gemm_acc)>(a[2]);
  call_mha_fwd = reinterpret_cast<decltype(call_mha_fwd)>(a[3]);
  call_paged = reinterpret_cast<decltype(call_paged)>(a[4]);
  if (a[5]) call_quant_fp8 = reinterpret_cast<decltype(call_quant_fp8)>(a[5]);
  if (a[6]) call_gemm_fp8 = reinterpret_cast<decltype(call_gemm_fp8)>(a[6]);
  if (a[7]) call_append = reinterpret_cast<decltype(call_append)>(a[7]);
  if (a[8]) call_append_fp8 = reinterpret_cast<decltype(call_append_fp8)>(a[8]);
  if (a[9]) call_paged_fp8 = reinterpret_cast<decltype(call_paged_fp8)>(a[9]);
  Py_RETURN_NONE;
}

#define MLT_FAST(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(guarded<f>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {MLT_FAST("gemm", py_gemm),
                         MLT_FAST("gemm_acc", py_gemm_acc),
                         MLT_FAST("gemm_bias_act", py_gemm_bias_act),
                         MLT_FAST("mha_fwd", py_mha_fwd),
                         MLT_FAST("paged_attn_decode", py_paged),
                         MLT_FAST("quant_fp8", py_quant_fp8),
                         MLT_FAST("gemm_fp8", py_gemm_fp8),
                         MLT_FAST("paged_append", py_append),
                         MLT_FAST("paged_attn_decode_fp8", py_paged_fp8),
                         {"bind", py_bind, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", MLT_TORCH_VERSION) != 0) Py_CLEAR(m);   // whose tensors it knows
  return m;
}
