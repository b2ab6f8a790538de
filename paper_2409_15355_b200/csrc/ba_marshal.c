/*
 * Argument marshalling of the hot calls for Python: tensors to addresses, numbers to C types, one call of the library.
 * A request of 32 layers makes 64 of these calls, and a small request takes the GPU less time than ctypes took to issue it:
 * ba_final_attend 6.6 -> 4.0 us, ba_reencode_k 4.6 -> 2.8 us a call (a kernel launch included), a small request 33.4 -> 27.5 us.
 * Nothing else happens here; the functions are those of the library that bind() is given (the handle ctypes opened), their
 * prototypes the header's.  Only the usual arguments are taken: None, an int that fits, a contiguous torch tensor, the ctypes
 * class of a structure.  With any other the whole call goes to the function bind() was given, which makes it through ctypes: what
 * is accepted, and what is raised, is decided there alone.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>
#include <stdint.h>

#include "ba.h"

static PyObject *s_data_ptr, *s_is_contiguous, *s_stride, *s_shape, *s_dtype, *s_is_cuda, *int32_type;
static PyObject *other_way, *t_handle, *t_segments, *t_pages, *t_shared;
/* bind()'s: the ctypes way, c_void_p, ba_segments, ba_page_table, ba_shared_batch */

/* The converters return 1, 0 (an exception is set) or this: not an argument this file takes. */
#define UNUSUAL (-1)

static int unusual_if(PyObject *exception) {
  if (!PyErr_ExceptionMatches(exception)) return 0;
  PyErr_Clear();
  return UNUSUAL;
}
static int from_int(PyObject *o, void **out) {
  *out = PyLong_AsVoidPtr(o);
  return *out == NULL && PyErr_Occurred() ? unusual_if(PyExc_OverflowError) : 1;
}
/* None -> NULL, an int -> that address, an object with is_contiguous() and data_ptr() (a torch tensor) -> its data. */
static int to_address(PyObject *o, void **out) {
  if (o == Py_None) { *out = NULL; return 1; }
  if (PyLong_Check(o)) return from_int(o, out);
  PyObject *r = PyObject_CallMethodNoArgs(o, s_is_contiguous);
  if (!r) return unusual_if(PyExc_AttributeError);
  const int yes = PyObject_IsTrue(r);
  Py_DECREF(r);
  if (yes < 0) return 0;
  if (!yes) { PyErr_SetString(PyExc_ValueError, "tensor must be contiguous"); return 0; }
  r = PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (!r) return unusual_if(PyExc_AttributeError);
  const int k = PyLong_Check(r) ? from_int(r, out) : UNUSUAL;
  Py_DECREF(r);
  return k;
}
/* The memory of an instance of ctypes class `type`, at least `bytes` of it. */
static int to_memory(PyObject *o, PyObject *type, size_t bytes, void **out) {
  const int is = PyObject_IsInstance(o, type);
  if (is < 0) return 0;
  if (!is) return UNUSUAL;
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return 0;
  const int fits = (size_t)b.len >= bytes;
  *out = b.buf;
  PyBuffer_Release(&b);
  return fits ? 1 : UNUSUAL;
}
static int to_context(PyObject *o, ba_ctx **out) {
  void *at;
  if (o == Py_None || PyLong_Check(o)) return to_address(o, (void **)out);
  const int k = to_memory(o, t_handle, sizeof(void *), &at);
  if (k == 1) *out = *(ba_ctx **)at;
  return k;
}
static int to_int(PyObject *o, int32_t *out) {
  if (!PyLong_Check(o)) return UNUSUAL;
  int overflow;
  const long v = PyLong_AsLongAndOverflow(o, &overflow);
  if (overflow || v < INT32_MIN || v > INT32_MAX) return UNUSUAL;
  *out = (int32_t)v;
  return 1;
}
static int to_size(PyObject *o, size_t *out) {
  if (!PyLong_Check(o)) return UNUSUAL;
  *out = PyLong_AsSize_t(o);
  return *out == (size_t)-1 && PyErr_Occurred() ? unusual_if(PyExc_OverflowError) : 1;
}
/* A [rows, heads, head_dim] tensor whose rows may lie apart, a whole row or more: its data and row stride (0: packed).  Anything else -- rows that
 * share memory, whose stride would be taken for packed rows -- is the other way's. */
static int to_rows(PyObject *o, void **out, int64_t *stride) {
  *stride = 0;
  if (o == Py_None || PyLong_Check(o)) return to_address(o, out);
  PyObject *r = PyObject_CallMethodNoArgs(o, s_is_contiguous);
  if (!r) return unusual_if(PyExc_AttributeError);
  const int packed = PyObject_IsTrue(r);
  Py_DECREF(r);
  if (packed < 0) return 0;
  if (!packed) {
    PyObject *st = PyObject_CallMethodNoArgs(o, s_stride), *sh = st ? PyObject_GetAttr(o, s_shape) : NULL;
    int k = UNUSUAL;
    if (st && sh && PyTuple_Check(st) && PyTuple_Check(sh) && PyTuple_GET_SIZE(st) == 3 && PyTuple_GET_SIZE(sh) == 3) {
      const long long s0 = PyLong_AsLongLong(PyTuple_GET_ITEM(st, 0)), s1 = PyLong_AsLongLong(PyTuple_GET_ITEM(st, 1));
      const long long heads = PyLong_AsLongLong(PyTuple_GET_ITEM(sh, 1)), d = PyLong_AsLongLong(PyTuple_GET_ITEM(sh, 2));
      if (PyLong_AsLongLong(PyTuple_GET_ITEM(st, 2)) == 1 && s1 == d && d > 0 && s0 / d >= heads && !PyErr_Occurred()) { *stride = s0; k = 1; }
    }
    Py_XDECREF(st); Py_XDECREF(sh);
    PyErr_Clear();
    if (k != 1) return k;
  }
  r = PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (!r) return unusual_if(PyExc_AttributeError);
  const int k = PyLong_Check(r) ? from_int(r, out) : UNUSUAL;
  Py_DECREF(r);
  return k;
}
/* An int32 tensor on the device, by its contents' address.  Anything else -- other types, the host's -- is the other way's, which refuses it. */
static int to_table(PyObject *o, void **out) {
  if (o != Py_None && !PyLong_Check(o)) {
    PyObject *t = PyObject_GetAttr(o, s_dtype);
    if (!t) return unusual_if(PyExc_AttributeError);
    if (!int32_type) {                             /* (torch has one object for a type; this file does not import torch) */
      PyObject *name = PyObject_Str(t);
      if (name && PyUnicode_Check(name) && PyUnicode_CompareWithASCIIString(name, "torch.int32") == 0) int32_type = Py_NewRef(t);
      Py_XDECREF(name);
      PyErr_Clear();
    }
    const int is = t == int32_type;
    Py_DECREF(t);
    PyObject *there = is ? PyObject_GetAttr(o, s_is_cuda) : NULL;
    const int cuda = there == Py_True;
    Py_XDECREF(there);
    PyErr_Clear();
    if (!cuda) return UNUSUAL;
  }
  return to_address(o, out);
}
static int to_float(PyObject *o, float *out) {
  if (!PyFloat_Check(o)) return UNUSUAL;
  *out = (float)PyFloat_AS_DOUBLE(o);
  return 1;
}
/* other_way(name, arguments ...) */
static PyObject *go_other_way(const char *name, PyObject *const *args, Py_ssize_t nargs) {
  PyObject *all = PyTuple_New(nargs + 1), *n = PyUnicode_FromString(name);
  if (!all || !n) { Py_XDECREF(all); Py_XDECREF(n); return NULL; }
  PyTuple_SET_ITEM(all, 0, n);
  for (Py_ssize_t i = 0; i < nargs; ++i) PyTuple_SET_ITEM(all, i + 1, Py_NewRef(args[i]));
  PyObject *r = PyObject_Call(other_way, all, NULL);
  Py_DECREF(all);
  return r;
}

#define ARGS(name, n)                                                                                   \
  static const char function[] = #name;                                                                 \
  if (!other_way) return PyErr_Format(PyExc_RuntimeError, "no library bound");                          \
  if (nargs != (n)) return PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", (n), nargs)
#define TAKE(convert)                                                                     \
  do {                                                                                    \
    const int taken = (convert);                                                          \
    if (taken != 1) return taken == UNUSUAL ? go_other_way(function, args, nargs) : NULL; \
  } while (0)
#define P(i, v) void *v; TAKE(to_address(args[i], &v))
#define I(i, v) int32_t v; TAKE(to_int(args[i], &v))
#define CTX ba_ctx *ctx; TAKE(to_context(args[0], &ctx))
#define SEG(i, v) void *v; TAKE(to_memory(args[i], t_segments, sizeof(ba_segments), &v))
#define PAGES(i, v) void *v; TAKE(to_memory(args[i], t_pages, sizeof(ba_page_table), &v))
#define R(i, v) void *v; int64_t v##_stride; TAKE(to_rows(args[i], &v, &v##_stride))
#define T(i, v) void *v; TAKE(to_table(args[i], &v))
#define F(i, v) float v; TAKE(to_float(args[i], &v))
#define SHARED(i, v) void *v; TAKE(to_memory(args[i], t_shared, sizeof(ba_shared_batch), &v))
#define CALL(expr)                                   \
  do {                                               \
    ba_status st;                                    \
    Py_BEGIN_ALLOW_THREADS st = (expr);              \
    Py_END_ALLOW_THREADS return PyLong_FromLong(st); \
  } while (0)
#define FUNCTIONS(X) X(ba_segment) X(ba_reencode_k) X(ba_reencode_k_paged) X(ba_block_prefill) X(ba_block_prefill_bwd) \
  X(ba_final_attend) X(ba_final_attend_fused) X(ba_final_attend_paged) X(ba_final_attend_fused_paged)
/* (a library without these is taken as well: calls of them go the ctypes way) */
#define MORE_FUNCTIONS(X) X(ba_qk_norm_rope) X(ba_qk_norm_rope_bwd) X(ba_append_paged) X(ba_shared_prefix_attend)
#define DECLARE(f) static __typeof__(&f) p_##f;
FUNCTIONS(DECLARE)
MORE_FUNCTIONS(DECLARE)

static PyObject *m_segment(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_segment, 11); CTX; P(1, lens); P(2, nblocks); I(3, batch); I(4, n_blocks); I(5, n_tokens); I(6, mode); P(7, buf);
  size_t bytes; TAKE(to_size(args[8], &bytes));
  SEG(9, out); P(10, stream);
  CALL(p_ba_segment(ctx, lens, nblocks, batch, n_blocks, n_tokens, mode, buf, bytes, out, stream));
}
static PyObject *m_reencode_k(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_reencode_k, 10); CTX; P(1, src); P(2, off); I(3, n_src); P(4, dst); P(5, cu); P(6, delta); I(7, n_blocks); I(8, n_rows); P(9, stream);
  CALL(p_ba_reencode_k(ctx, src, off, n_src, dst, cu, delta, n_blocks, n_rows, stream));
}
static PyObject *m_reencode_k_paged(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_reencode_k_paged, 9); CTX; P(1, pool); PAGES(2, pages); P(3, dst); P(4, cu); P(5, delta); I(6, n_blocks); I(7, n_rows); P(8, stream);
  CALL(p_ba_reencode_k_paged(ctx, pool, pages, dst, cu, delta, n_blocks, n_rows, stream));
}
static PyObject *m_block_prefill(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_block_prefill, 10); CTX; P(1, q); P(2, k); P(3, v); P(4, o); P(5, lse); SEG(6, seg); I(7, mode); I(8, out); P(9, stream);
  CALL(p_ba_block_prefill(ctx, q, k, v, o, lse, seg, mode, out, stream));
}
static PyObject *m_block_prefill_bwd(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_block_prefill_bwd, 14); CTX; P(1, q); P(2, k); P(3, v); P(4, o); P(5, lse); P(6, d_o); P(7, dq); P(8, dk); P(9, dv); SEG(10, seg); I(11, mode);
  I(12, out); P(13, stream);
  CALL(p_ba_block_prefill_bwd(ctx, q, k, v, o, lse, d_o, dq, dk, dv, seg, mode, out, stream));
}
static PyObject *m_final_attend(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_final_attend, 16); CTX; P(1, q); P(2, k); P(3, v); I(4, n_final); P(5, kc); P(6, vc); I(7, n_cache); P(8, voff); I(9, n_v); P(10, o);
  P(11, lse); SEG(12, seg); I(13, mode); I(14, out); P(15, stream);
  CALL(p_ba_final_attend(ctx, q, k, v, n_final, kc, vc, n_cache, voff, n_v, o, lse, seg, mode, out, stream));
}
static PyObject *m_final_attend_fused(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_final_attend_fused, 17); CTX; P(1, q); P(2, k); P(3, v); I(4, n_final); P(5, ks); P(6, vs); I(7, n_src); P(8, off); I(9, n_cache); P(10, k_out);
  P(11, o); P(12, lse); SEG(13, seg); I(14, mode); I(15, out); P(16, stream);
  CALL(p_ba_final_attend_fused(ctx, q, k, v, n_final, ks, vs, n_src, off, n_cache, k_out, o, lse, seg, mode, out, stream));
}
static PyObject *m_final_attend_paged(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_final_attend_paged, 15); CTX; P(1, q); P(2, k); P(3, v); I(4, n_final); P(5, kc); I(6, n_cache); P(7, pool); PAGES(8, pages); P(9, o); P(10, lse);
  SEG(11, seg); I(12, mode); I(13, out); P(14, stream);
  CALL(p_ba_final_attend_paged(ctx, q, k, v, n_final, kc, n_cache, pool, pages, o, lse, seg, mode, out, stream));
}
static PyObject *m_final_attend_fused_paged(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_final_attend_fused_paged, 16); CTX; P(1, q); P(2, k); P(3, v); I(4, n_final); P(5, kp); P(6, vp); PAGES(7, pages); I(8, n_cache); P(9, k_out); P(10, o);
  P(11, lse); SEG(12, seg); I(13, mode); I(14, out); P(15, stream);
  CALL(p_ba_final_attend_fused_paged(ctx, q, k, v, n_final, kp, vp, pages, n_cache, k_out, o, lse, seg, mode, out, stream));
}

#define PRESENT(f) if (!p_##f || !t_shared) return go_other_way(function, args, nargs)
static PyObject *m_qk_norm_rope(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_qk_norm_rope, 11); PRESENT(ba_qk_norm_rope); CTX; R(1, q); R(2, k); I(3, n); T(4, pos); P(5, wq); P(6, wk); F(7, eps); P(8, q_out); P(9, k_out);
  P(10, stream);
  CALL(p_ba_qk_norm_rope(ctx, q, q_stride, k, k_stride, n, pos, wq, wk, eps, q_out, k_out, stream));
}
static PyObject *m_qk_norm_rope_bwd(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_qk_norm_rope_bwd, 16); PRESENT(ba_qk_norm_rope_bwd); CTX; R(1, q); R(2, k); I(3, n); T(4, pos); P(5, wq); P(6, wk); F(7, eps); P(8, dyq); P(9, dyk);
  R(10, dq); R(11, dk); P(12, dwq); P(13, dwk); I(14, type); P(15, stream);
  CALL(p_ba_qk_norm_rope_bwd(ctx, q, q_stride, k, k_stride, n, pos, wq, wk, eps, dyq, dyk, dq, dq_stride, dk, dk_stride, dwq, dwk, type, stream));
}
static PyObject *m_append_paged(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_append_paged, 17); PRESENT(ba_append_paged); CTX; R(1, q); R(2, k); R(3, v); I(4, n); T(5, pos); P(6, wq); P(7, wk); F(8, eps); T(9, cu);
  T(10, start); I(11, n_seqs); P(12, q_out); P(13, kp); P(14, vp); PAGES(15, pages); P(16, stream);
  CALL(p_ba_append_paged(ctx, q, q_stride, k, k_stride, v, v_stride, n, pos, wq, wk, eps, cu, start, n_seqs, q_out, kp, vp, pages, stream));
}
static PyObject *m_shared_prefix_attend(PyObject *self, PyObject *const *args, Py_ssize_t nargs) {
  ARGS(ba_shared_prefix_attend, 15); PRESENT(ba_shared_prefix_attend); CTX; P(1, q); I(2, n); P(3, kx); P(4, vx); I(5, nx);
  void *px = NULL;
  if (args[6] != Py_None) TAKE(to_memory(args[6], t_pages, sizeof(ba_page_table), &px));
  P(7, kp); P(8, vp); PAGES(9, pages); SHARED(10, shared); P(11, o); P(12, lse); I(13, out); P(14, stream);
  CALL(p_ba_shared_prefix_attend(ctx, q, n, kx, vx, nx, px, kp, vp, pages, shared, o, lse, out, stream));
}

/* bind(handle, other_way, c_void_p, ba_segments, ba_page_table[, ba_shared_batch]): take the library's functions from the shared object a dlopen
 * handle names. */
static PyObject *m_bind(PyObject *self, PyObject *args) {
  PyObject *handle, *way, *handle_type, *segments, *pages, *shared = NULL;
  if (!PyArg_ParseTuple(args, "OOOOO|O", &handle, &way, &handle_type, &segments, &pages, &shared)) return NULL;
  void *h = PyLong_AsVoidPtr(handle);
  if (!h && PyErr_Occurred()) return NULL;
#define RESOLVE(f) \
  if (!(p_##f = (__typeof__(&f))dlsym(h, #f))) return PyErr_Format(PyExc_RuntimeError, "%s is not in the library", #f);
  FUNCTIONS(RESOLVE)
#define RESOLVE_IF_THERE(f) p_##f = (__typeof__(&f))dlsym(h, #f);
  MORE_FUNCTIONS(RESOLVE_IF_THERE)
  Py_XSETREF(t_handle, Py_NewRef(handle_type));
  Py_XSETREF(t_segments, Py_NewRef(segments));
  Py_XSETREF(t_pages, Py_NewRef(pages));
  if (shared) Py_XSETREF(t_shared, Py_NewRef(shared));
  Py_XSETREF(other_way, Py_NewRef(way));
  Py_RETURN_NONE;
}

#define METHOD(n) {#n, (PyCFunction)(void (*)(void))m_##n, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {{"bind", m_bind, METH_VARARGS, NULL}, METHOD(segment), METHOD(reencode_k), METHOD(reencode_k_paged),
                                METHOD(block_prefill), METHOD(block_prefill_bwd), METHOD(final_attend), METHOD(final_attend_fused),
                                METHOD(final_attend_paged), METHOD(final_attend_fused_paged),
                                METHOD(qk_norm_rope), METHOD(qk_norm_rope_bwd), METHOD(append_paged), METHOD(shared_prefix_attend), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "ba_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit_ba_marshal(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_stride = PyUnicode_InternFromString("stride");
  s_shape = PyUnicode_InternFromString("shape");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  return s_data_ptr && s_is_contiguous && s_stride && s_shape && s_dtype && s_is_cuda ? PyModule_Create(&module) : NULL;
}
