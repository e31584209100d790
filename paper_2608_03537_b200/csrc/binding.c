// Argument marshalling of the Python entry points, as a CPython extension (_binding.<tag>.so).
//
// A call of a small problem is bound by the time its Python caller spends on it: building the descriptor field by field
// through ctypes, wrapping every pointer and asking for the current stream took 9 of the 13.5 us that a 16 x 256 x 64
// post-norm call cost the host (4.0 us of it inside the library).  This module reads the tensors' shapes, strides and
// addresses through their Python interface (no dependence on the tensor library's binary interface), fills the C structures
// and calls the entry point with the interpreter lock released.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "comfuse.h"

typedef comfuse_status_t (*gemm_epilogue_fn)(const comfuse_gemm_desc_t*, const void*, const void*, void*, const comfuse_epilogue_args_t*, void*, size_t, void*);
typedef comfuse_status_t (*b2b_gemm_fn)(const comfuse_b2b_desc_t*, const void*, const void*, const void*, const void*, const void*, const void*,
                                        const void*, void*, void*, size_t, void*);
typedef comfuse_status_t (*gemm_spec_fn)(const comfuse_fusion_spec_t*, const comfuse_gemm_shape_t*, const void*, const void*, void*, const void* const*,
                                         const int64_t*, void* const*, int32_t, void*, size_t, void*);
typedef comfuse_status_t (*quantize_rows_fn)(const comfuse_quantize_desc_t*, const void*, const void*, const void*, void*, int8_t*, float*, void*, void*);
typedef comfuse_status_t (*gemm_q8_fn)(const comfuse_gemm_q8_desc_t*, const int8_t*, const float*, const int8_t*, const float*, const void*, const void*, void*,
                                       void*);
static quantize_rows_fn f_quantize_rows;
static gemm_q8_fn f_gemm_q8;
static PyObject *t_bf16, *t_f16, *t_f32, *t_i8, *s_dtype, *s_get_device;  // the tensor library's element types (bind_q8)
static gemm_epilogue_fn f_gemm_epilogue;
static b2b_gemm_fn f_b2b_gemm;
static gemm_spec_fn f_gemm_spec;
static PyObject *s_data_ptr, *s_shape, *s_stride, *s_dim, *s_is_contiguous, *s_numel, *s_element_size, *s_cuda_stream;

#define MAX_DIMS 64  // (tensors have no more)
typedef struct {
  int n;
  int64_t size[MAX_DIMS], stride[MAX_DIMS];
} Geometry;

static int to_i64(PyObject* o, int64_t* out) {  // int(o); wraps like a C integer
  PyObject* v = PyLong_Check(o) ? Py_NewRef(o) : PyNumber_Long(o);
  if (!v) return 0;
  *out = (int64_t)PyLong_AsUnsignedLongLongMask(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}
static int to_f64(PyObject* o, double* out) {  // float(o): numbers, tensors of one element, texts
  if (PyFloat_CheckExact(o)) {
    *out = PyFloat_AS_DOUBLE(o);
    return 1;
  }
  PyObject* v = PyNumber_Float(o);
  if (!v) return 0;
  *out = PyFloat_AS_DOUBLE(v);
  Py_DECREF(v);
  return 1;
}
static int tuple_i64(PyObject* t, int64_t* out, int* n) {
  PyObject* seq = t ? PySequence_Fast(t, "a shape or stride") : NULL;
  Py_XDECREF(t);
  if (!seq) return 0;
  const Py_ssize_t len = PySequence_Fast_GET_SIZE(seq);
  if (len > MAX_DIMS) {
    Py_DECREF(seq);
    PyErr_SetString(PyExc_AssertionError, "too many dimensions");
    return 0;
  }
  for (Py_ssize_t i = 0; i < len; ++i)
    if (!to_i64(PySequence_Fast_GET_ITEM(seq, i), out + i)) {
      Py_DECREF(seq);
      return 0;
    }
  *n = (int)len;
  Py_DECREF(seq);
  return 1;
}
static int shape_of(PyObject* t, Geometry* g) { return tuple_i64(PyObject_GetAttr(t, s_shape), g->size, &g->n); }
static int geometry(PyObject* t, Geometry* g) {
  int n = 0;
  if (!shape_of(t, g) || !tuple_i64(PyObject_CallMethodNoArgs(t, s_stride), g->stride, &n)) return 0;
  if (n != g->n || n < 2) {
    PyErr_SetString(PyExc_IndexError, "Dimension out of range (a matrix or a batch of matrices is expected)");
    return 0;
  }
  return 1;
}
static int method_i64(PyObject* t, PyObject* name, int64_t* out) {
  PyObject* v = PyObject_CallMethodNoArgs(t, name);
  if (!v) return 0;
  const int ok = to_i64(v, out);
  Py_DECREF(v);
  return ok;
}
static int pointer(PyObject* t, const void** out) {  // None: a null pointer
  int64_t v = 0;
  if (t != Py_None && !method_i64(t, s_data_ptr, &v)) return 0;
  *out = (const void*)(uintptr_t)v;
  return 1;
}
static int workspace_of(PyObject* t, void** ptr, size_t* bytes) {
  int64_t n = 0, size = 0;
  *bytes = 0;
  if (!pointer(t, (const void**)ptr)) return 0;
  if (t == Py_None) return 1;
  if (!method_i64(t, s_numel, &n) || !method_i64(t, s_element_size, &size)) return 0;
  *bytes = (size_t)(n * size);
  return 1;
}
static int contiguous(PyObject* t) {
  PyObject* v = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  if (!v) return 0;
  const int yes = PyObject_IsTrue(v);
  Py_DECREF(v);
  if (yes == 0) PyErr_SetString(PyExc_AssertionError, "a dense tensor is expected");
  return yes == 1;
}
static int require(int cond, const char* what) {
  if (!cond) PyErr_SetString(PyExc_AssertionError, what);
  return cond;
}
// a stream object (which may be callable), or the function that returns the current stream's handle
static int stream_of(PyObject* s, void** out) {
  PyObject* v = PyFunction_Check(s) ? PyObject_CallNoArgs(s) : PyObject_GetAttr(s, s_cuda_stream);
  int64_t h = 0;
  if (!v) return 0;
  const int ok = to_i64(v, &h);
  Py_DECREF(v);
  *out = (void*)(uintptr_t)h;
  return ok;
}
static int fixed_args(Py_ssize_t got, Py_ssize_t want, const char* name) {
  if (got != want) PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", name, want, got);
  return got == want;
}

// a = (A, B, Y, kind, residual, alpha, eps, mask, fused, flags, softcap)
static int fill_desc(PyObject* const* a, comfuse_gemm_desc_t* d) {
  Geometry A, B, Y, R;
  int64_t kind, mask, flags;
  if (!geometry(a[0], &A) || !geometry(a[1], &B) || !geometry(a[2], &Y)) return 0;
  if (!to_i64(a[9], &flags)) return 0;
  const int batched = A.n == 3, b_nk = (flags & COMFUSE_FLAG_B_ROW_MAJOR_NK) != 0;
  const int64_t M = A.size[A.n - 2], K = A.size[A.n - 1], N = B.size[B.n - (b_nk ? 2 : 1)];
  if (!require(B.size[B.n - (b_nk ? 1 : 2)] == K && Y.size[Y.n - 2] == M && Y.size[Y.n - 1] == N, "shapes of A, B and Y do not match")) return 0;
  if (!require(A.stride[A.n - 1] == 1 && B.stride[B.n - 1] == 1 && Y.stride[Y.n - 1] == 1, "the last dimension of A, B and Y must be dense")) return 0;
  memset(d, 0, sizeof(*d));
  d->batch = (int32_t)(batched ? A.size[0] : 1);
  d->M = (int32_t)M;
  d->N = (int32_t)N;
  d->K = (int32_t)K;
  d->lda = A.stride[A.n - 2];
  d->ldb = B.stride[B.n - 2];
  d->ldy = Y.stride[Y.n - 2];
  d->batch_stride_a = batched ? A.stride[0] : M * d->lda;
  d->batch_stride_b = batched ? B.stride[0] : (b_nk ? N : K) * d->ldb;
  d->batch_stride_y = batched ? Y.stride[0] : M * d->ldy;
  d->ldr = N;
  d->batch_stride_r = M * N;
  if (a[4] != Py_None) {
    if (!geometry(a[4], &R)) return 0;
    d->ldr = R.stride[R.n - 2];
    d->batch_stride_r = batched ? R.stride[0] : M * d->ldr;
  }
  if (!to_i64(a[3], &kind) || !to_i64(a[7], &mask)) return 0;
  double alpha, eps, softcap;
  if (!to_f64(a[5], &alpha) || !to_f64(a[6], &eps) || !to_f64(a[10], &softcap)) return 0;
  const int fused = PyObject_IsTrue(a[8]);
  if (fused < 0) return 0;
  d->kind = (int32_t)kind;
  d->mask = (int32_t)mask;
  d->alpha = (float)alpha;
  d->eps = (float)eps;
  d->fused = fused;
  d->flags = (uint32_t)flags;
  d->softcap = (float)softcap;
  return 1;
}

// gemm_desc(A, B, Y, kind, residual, alpha, eps, mask, fused, flags, softcap) -> bytes of a comfuse_gemm_desc_t
static PyObject* py_gemm_desc(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  comfuse_gemm_desc_t d;
  if (!fixed_args(n, 11, "gemm_desc") || !fill_desc(a, &d)) return NULL;
  return PyBytes_FromStringAndSize((const char*)&d, sizeof(d));
}

// gemm_epilogue(<the arguments of gemm_desc>, bias, gamma, beta, mask_tensor, row_max, row_argmax, workspace, stream) -> status
static PyObject* py_gemm_epilogue(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  comfuse_gemm_desc_t d;
  comfuse_epilogue_args_t e;
  const void *A, *B, *Y;
  void *ws, *stream;
  size_t ws_bytes;
  if (!fixed_args(n, 19, "gemm_epilogue") || !fill_desc(a, &d)) return NULL;
  memset(&e, 0, sizeof(e));
  if (!pointer(a[11], &e.bias) || !pointer(a[4], &e.residual) || !pointer(a[12], &e.gamma) || !pointer(a[13], &e.beta) || !pointer(a[14], &e.mask) ||
      !pointer(a[15], (const void**)&e.row_max) || !pointer(a[16], (const void**)&e.row_argmax) || !workspace_of(a[17], &ws, &ws_bytes) ||
      !pointer(a[0], &A) || !pointer(a[1], &B) || !pointer(a[2], &Y) || !stream_of(a[18], &stream))
    return NULL;
  comfuse_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = f_gemm_epilogue(&d, A, B, (void*)Y, &e, ws, ws_bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

// b2b(kind, X, W1, b1, W2, b2, gamma, beta, O, eps, alpha, fused, flags, workspace, stream) -> status
static PyObject* py_b2b(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  comfuse_b2b_desc_t d;
  Geometry X, W1, W2, O;
  int64_t kind, flags;
  if (!fixed_args(n, 15, "b2b") || !to_i64(a[0], &kind) || !to_i64(a[12], &flags)) return NULL;
  const int attention = kind == COMFUSE_B2B_SOFTMAX_ATTENTION;
  if (!shape_of(a[1], &X) || !shape_of(a[2], &W1) || !shape_of(a[4], &W2)) return NULL;
  if (X.n != (attention ? 3 : 2)) {
    PyErr_Format(PyExc_ValueError, "a tensor of %d dimensions is expected, got %d", attention ? 3 : 2, X.n);
    return NULL;
  }
  if (W2.n <= (attention ? 2 : 1) || (!attention && W1.n < 2)) {
    PyErr_SetString(PyExc_IndexError, "tuple index out of range");
    return NULL;
  }
  memset(&d, 0, sizeof(d));
  const int64_t nb = attention ? X.size[0] : 1, M = X.size[X.n - 2], K = X.size[X.n - 1];
  const int64_t N1 = attention ? W2.size[1] : W1.size[1], N2 = attention ? W2.size[2] : W2.size[1];
  if (attention) {
    const int rm = (flags & COMFUSE_B2B_FLAG_KEYS_ROW_MAJOR) != 0;
    if (!shape_of(a[8], &O)) return NULL;
    if (!require(W1.n == 3 && W1.size[0] == nb && W1.size[1] == (rm ? N1 : K) && W1.size[2] == (rm ? K : N1) && W2.n == 3 && W2.size[0] == nb && O.n == 3 &&
                     O.size[0] == nb && O.size[1] == M && O.size[2] == N2,
                 "shapes of Q, keys, V and O do not match"))
      return NULL;
  } else if (kind == COMFUSE_B2B_MLP_RELU) {
    if (!shape_of(a[8], &O)) return NULL;
    if (!require(W1.n == 2 && W1.size[0] == K && W2.n == 2 && W2.size[0] == N1 && O.n == 2 && O.size[0] == M && O.size[1] == N2, "shapes of X, W1, W2 and O do not match"))
      return NULL;
  }
  if (!contiguous(a[1]) || !contiguous(a[2]) || !contiguous(a[4]) || !contiguous(a[8])) return NULL;
  double eps, alpha;
  if (!to_f64(a[9], &eps) || !to_f64(a[10], &alpha)) return NULL;
  const int fused = PyObject_IsTrue(a[11]);
  if (fused < 0) return NULL;
  d.M = (int32_t)M;
  d.K = (int32_t)K;
  d.N1 = (int32_t)N1;
  d.N2 = (int32_t)N2;
  d.eps = (float)eps;
  d.fused = fused;
  d.kind = (int32_t)kind;
  d.batch = (int32_t)nb;
  d.alpha = (float)alpha;
  d.flags = (int32_t)flags;
  const void* p[8];
  void *ws, *stream;
  size_t ws_bytes;
  for (int i = 0; i < 8; ++i)
    if (!pointer(a[1 + i], p + i)) return NULL;
  if (!workspace_of(a[13], &ws, &ws_bytes) || !stream_of(a[14], &stream)) return NULL;
  comfuse_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = f_b2b_gemm(&d, p[0], p[1], p[2], p[3], p[4], p[5], p[6], (void*)p[7], ws, ws_bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

// A sequence of tensors (something with a length: a generator's tensors would be gone before the launch is enqueued), held for the
// length of a call, and zeroed room for `arrays` 8-byte values of each.  The library reads as many entries as the program
// names, so there is room for the most that a program can name, however few were given.
#define MIN_ROOM (COMFUSE_SPEC_MAX_PARAMS > COMFUSE_SPEC_MAX_ROW_OUTPUTS ? COMFUSE_SPEC_MAX_PARAMS : COMFUSE_SPEC_MAX_ROW_OUTPUTS)
typedef struct {
  PyObject* seq;
  Py_ssize_t n, room;
  int64_t* values;
} Held;
static int hold(PyObject* o, int arrays, Held* h) {
  if (PyObject_Size(o) < 0) return 0;
  h->seq = PySequence_Fast(o, "a sequence of tensors is expected");
  if (!h->seq) return 0;
  h->n = PySequence_Fast_GET_SIZE(h->seq);
  h->room = h->n > MIN_ROOM ? h->n : MIN_ROOM;
  h->values = PyMem_Calloc((size_t)(h->room * arrays), sizeof(int64_t));
  if (!h->values) PyErr_NoMemory();
  return h->values != NULL;
}
static void let_go(Held* h) {
  PyMem_Free(h->values);
  Py_XDECREF(h->seq);
}

// gemm_spec(A, B, Y, address of the comfuse_fusion_spec_t, params, row_out, fused, b_nk, workspace, stream) -> status
static int gemm_spec_call(PyObject* const* a, Held* params, Held* rows, comfuse_status_t* st) {
  Geometry A, B, Y;
  comfuse_gemm_shape_t s;
  int64_t spec, fused;
  if (!geometry(a[0], &A) || !geometry(a[1], &B) || !geometry(a[2], &Y) || !to_i64(a[3], &spec) || !to_i64(a[6], &fused)) return 0;
  const int b_nk = PyObject_IsTrue(a[7]);
  if (b_nk < 0) return 0;
  const int batched = A.n == 3;
  memset(&s, 0, sizeof(s));
  const int64_t M = A.size[A.n - 2], K = A.size[A.n - 1], N = B.size[B.n - (b_nk ? 2 : 1)];
  s.batch = (int32_t)(batched ? A.size[0] : 1);
  s.M = (int32_t)M;
  s.N = (int32_t)N;
  s.K = (int32_t)K;
  s.lda = A.stride[A.n - 2] ? A.stride[A.n - 2] : K;
  s.ldb = B.stride[B.n - 2] ? B.stride[B.n - 2] : (b_nk ? K : N);
  s.ldy = Y.stride[Y.n - 2] ? Y.stride[Y.n - 2] : N;
  s.batch_stride_a = batched && A.stride[0] ? A.stride[0] : M * s.lda;
  s.batch_stride_b = batched && B.stride[0] ? B.stride[0] : (b_nk ? N : K) * s.ldb;
  s.batch_stride_y = batched && Y.stride[0] ? Y.stride[0] : M * s.ldy;
  s.flags = b_nk ? COMFUSE_FLAG_B_ROW_MAJOR_NK : 0;
  if (!hold(a[4], 2, params) || !hold(a[5], 1, rows)) return 0;
  int64_t* ld = params->values + params->room;
  for (Py_ssize_t i = 0; i < params->n; ++i) {
    PyObject* t = PySequence_Fast_GET_ITEM(params->seq, i);
    int64_t dims = 0;
    Geometry g;
    if (t == Py_None) continue;
    if (!method_i64(t, s_data_ptr, params->values + i) || !method_i64(t, s_dim, &dims)) return 0;
    if (dims < 2) continue;
    if (!geometry(t, &g)) return 0;
    ld[i] = g.stride[g.n - 2];
  }
  for (Py_ssize_t i = 0; i < rows->n; ++i)
    if (!method_i64(PySequence_Fast_GET_ITEM(rows->seq, i), s_data_ptr, rows->values + i)) return 0;
  const void *pA, *pB, *pY;
  void *ws, *stream;
  size_t ws_bytes;
  if (!workspace_of(a[8], &ws, &ws_bytes) || !pointer(a[0], &pA) || !pointer(a[1], &pB) || !pointer(a[2], &pY) || !stream_of(a[9], &stream)) return 0;
  Py_BEGIN_ALLOW_THREADS
  *st = f_gemm_spec((const comfuse_fusion_spec_t*)(uintptr_t)spec, &s, pA, pB, (void*)pY, (const void* const*)params->values, ld, (void* const*)rows->values,
                    (int32_t)fused, ws, ws_bytes, stream);
  Py_END_ALLOW_THREADS
  return 1;
}
static PyObject* py_gemm_spec(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Held params = {0}, rows = {0};
  comfuse_status_t st;
  if (!fixed_args(n, 10, "gemm_spec")) return NULL;
  const int ok = gemm_spec_call(a, &params, &rows, &st);
  let_go(&params);
  let_go(&rows);
  return ok ? PyLong_FromLong((long)st) : NULL;
}

// ---- the 8-bit integer layers.  Their tensors have more than one element type, so types, shapes and devices are looked at one by one.
//
// Asking a tensor for these through its Python interface takes 0.5 us a tensor, 3.5 of the 7 us that a norm of one token cost its caller.
// Where the tensor's class offers the DLPack exchange interface (a public, versioned C structure behind a capsule), one call fills in all of
// them; the Python interface remains for whatever does not.
typedef struct { uint32_t major, minor; } DlVersion;
typedef struct {
  void* data;
  struct { int32_t type, id; } device;  // type: 1 = host, 2 = CUDA
  int32_t ndim;
  struct { uint8_t code, bits; uint16_t lanes; } dtype;  // code: 0 = int, 2 = IEEE float, 4 = bfloat
  int64_t* shape;
  int64_t* strides;  // elements; NULL = dense
  uint64_t byte_offset;
} DlTensor;
typedef struct {
  DlVersion version;
  void* previous;
  void *allocate, *managed_from_object, *managed_to_object;
  int (*tensor_from_object)(void* object, DlTensor* out);  // a view for the length of the call; 0 = filled in, -1 = a Python error is set
  int (*current_stream)(int32_t device_type, int32_t device_id, void** out);
} DlExchange;
static const DlExchange* dl_exchange;
static PyTypeObject* dl_type;  // the class whose tensors it takes

enum { TYPE_BF16 = COMFUSE_DTYPE_BF16, TYPE_F16 = COMFUSE_DTYPE_F16, TYPE_F32 = COMFUSE_DTYPE_F32, TYPE_I8 = 3, TYPE_OTHER = -1 };
// types that only the key-value cache's calls take (`type` is TYPE_OTHER)
enum { WIDE_NONE, WIDE_I32, WIDE_I64, WIDE_F64 };
typedef struct {
  Geometry g;
  int type, wide;
  int bytes;       // of an element; 0 = not asked for
  int64_t device;  // -1 = host
  const void* p;
} Described;
static PyObject *t_i32, *t_i64, *t_f64;  // (bind_kv)

static int describe(PyObject* t, Described* d) {
  if (dl_exchange && PyObject_TypeCheck(t, dl_type)) {
    DlTensor v;
    if (dl_exchange->tensor_from_object(t, &v) == 0 && v.ndim <= MAX_DIMS) {
      d->g.n = v.ndim;
      int64_t dense = 1;
      for (int i = v.ndim - 1; i >= 0; --i) {
        d->g.size[i] = v.shape[i];
        d->g.stride[i] = v.strides ? v.strides[i] : dense;
        dense *= v.shape[i];
      }
      const int code = v.dtype.code, bits = v.dtype.bits;
      d->type = v.dtype.lanes != 1 ? TYPE_OTHER
                : code == 4 && bits == 16 ? TYPE_BF16
                : code == 2 && bits == 16 ? TYPE_F16
                : code == 2 && bits == 32 ? TYPE_F32
                : code == 0 && bits == 8  ? TYPE_I8
                                          : TYPE_OTHER;
      d->wide = v.dtype.lanes != 1 ? WIDE_NONE : code == 0 && bits == 32 ? WIDE_I32 : code == 0 && bits == 64 ? WIDE_I64 : code == 2 && bits == 64 ? WIDE_F64 : WIDE_NONE;
      d->bytes = (bits * v.dtype.lanes + 7) / 8;
      d->device = v.device.type == 2 ? v.device.id : v.device.type == 1 ? -1 : -2;
      d->p = (const char*)v.data + v.byte_offset;
      return 1;
    }
    PyErr_Clear();
  }
  int n = 0;
  PyObject* type = PyObject_GetAttr(t, s_dtype);
  if (!type) return 0;
  Py_DECREF(type);  // (a tensor's type outlives it)
  d->type = type == t_bf16 ? TYPE_BF16 : type == t_f16 ? TYPE_F16 : type == t_f32 ? TYPE_F32 : type == t_i8 ? TYPE_I8 : TYPE_OTHER;
  d->bytes = 0;
  d->wide = type == t_i32 ? WIDE_I32 : type == t_i64 ? WIDE_I64 : type == t_f64 ? WIDE_F64 : WIDE_NONE;
  return shape_of(t, &d->g) && tuple_i64(PyObject_CallMethodNoArgs(t, s_stride), d->g.stride, &n) && method_i64(t, s_get_device, &d->device) && pointer(t, &d->p);
}
static int refuse(const char* what, const char* why) {
  PyErr_Format(PyExc_AssertionError, "%s %s", what, why);
  return 0;
}
static int fits(const Described* d, int type, int64_t device, int64_t dims, int64_t batch, int64_t rows, int64_t cols, const char* what) {
  if (d->type != type) return refuse(what, "has another element type than the call takes");
  if (d->g.n != dims || (batch >= 0 && d->g.size[0] != batch) || (rows >= 0 && d->g.size[d->g.n - 2] != rows) || (cols >= 0 && d->g.size[d->g.n - 1] != cols))
    return refuse(what, "has a shape that does not match the call");
  if (d->device != device) return refuse(what, "is not on the current device");
  return 1;
}
// A matrix, or a batch of them (batch >= 0), with the given element type and, where they are given (>= 0), sizes, and a dense last dimension.
// None, where that may be: a null pointer.
static int matrix(PyObject* t, int type, int64_t device, int64_t batch, int64_t rows, int64_t cols, const char* what, Described* d) {
  if (!describe(t, d) || !fits(d, type, device, batch >= 0 ? 3 : 2, batch, rows, cols, what)) return 0;
  Geometry* g = &d->g;
  if (g->stride[g->n - 1] != 1 && g->size[g->n - 1] != 1) return refuse(what, "must be dense in its last dimension");
  if (g->size[g->n - 2] == 1) g->stride[g->n - 2] = (g->size[g->n - 1] + 15) / 16 * 16;  // (one row: nothing is addressed by its stride)
  return 1;
}
static int optional_matrix(PyObject* t, int type, int64_t device, int64_t batch, int64_t rows, int64_t cols, const char* what, Described* d) {
  if (t != Py_None) return matrix(t, type, device, batch, rows, cols, what, d);
  memset(d->g.stride, 0, 3 * sizeof(int64_t));
  d->g.n = 3;
  d->p = NULL;
  return 1;
}
// A dense vector of n elements (or [batch, n]).  None: a null pointer.
static int vector(PyObject* t, int type, int64_t device, int64_t batch, int64_t n, const char* what, const void** p) {
  Described d;
  *p = NULL;
  if (t == Py_None) return 1;
  if (!describe(t, &d) || !fits(&d, type, device, batch >= 0 ? 2 : 1, batch, -1, n, what)) return 0;
  if ((d.g.stride[d.g.n - 1] != 1 && n != 1) || (batch > 1 && d.g.stride[0] != n)) return refuse(what, "must be dense");
  *p = d.p;
  return 1;
}
// The element type of an operand that may have several, looked at first.
static int float_type(const Described* d, const char* what, int* type) {
  *type = d->type;
  return d->type == TYPE_BF16 || d->type == TYPE_F16 || d->type == TYPE_F32 ? 1 : refuse(what, "has another element type than the call takes");
}

// The stream of a call: as in stream_of, or, for the function that returns the current stream's handle, through the exchange interface.
static int stream_on(PyObject* s, int64_t device, void** out) {
  if (dl_exchange && dl_exchange->current_stream && PyFunction_Check(s)) {
    if (dl_exchange->current_stream(2, (int32_t)device, out) == 0) return 1;
    PyErr_Clear();
  }
  return stream_of(s, out);
}

// quantize_rows(kind, x, residual, gamma, h, q, scale, values, eps, device, stream) -> status
static PyObject* py_quantize_rows(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  comfuse_quantize_desc_t d;
  Described x, r, h, q, v;
  const void *gamma, *scale;
  int64_t kind, device;
  double eps;
  void* stream;
  int type;
  if (!fixed_args(n, 11, "quantize_rows") || !to_i64(a[0], &kind) || !to_i64(a[9], &device) || !to_f64(a[8], &eps)) return NULL;
  if (!describe(a[1], &x) || !float_type(&x, "x", &type) || !matrix(a[1], type, device, -1, -1, -1, "x", &x)) return NULL;
  const int64_t M = x.g.size[0], N = x.g.size[1];
  if (!optional_matrix(a[2], type, device, -1, M, N, "residual", &r) || !vector(a[3], type, device, -1, N, "gamma", &gamma) ||
      !optional_matrix(a[4], type, device, -1, M, N, "h", &h) || !matrix(a[5], TYPE_I8, device, -1, M, N, "q", &q) ||
      !vector(a[6], TYPE_F32, device, -1, M, "scale", &scale) || !optional_matrix(a[7], TYPE_BF16, device, -1, M, N, "values", &v) || !stream_on(a[10], device, &stream))
    return NULL;
  if (!require(M <= INT32_MAX && N <= INT32_MAX, "sizes are 32-bit numbers")) return NULL;
  memset(&d, 0, sizeof(d));
  d.kind = (int32_t)kind;
  d.dtype = type;
  d.rows = (int32_t)M;
  d.N = (int32_t)N;
  d.ldx = x.g.stride[0];
  d.ldr = r.g.stride[0];
  d.ldh = h.g.stride[0];
  d.ldq = q.g.stride[0];
  d.ldv = v.g.stride[0];
  d.eps = (float)eps;
  comfuse_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = f_quantize_rows(&d, x.p, r.p, gamma, (void*)h.p, (int8_t*)q.p, (float*)scale, (void*)v.p, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

// gemm_q8(A, scale_a, B, scale_b, Y, bias, residual, activation, device, stream) -> status
static PyObject* py_gemm_q8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  comfuse_gemm_q8_desc_t d;
  Described A, B, Y, r;
  const void *sa, *sb, *bias;
  int64_t activation, device;
  void* stream;
  int type;
  if (!fixed_args(n, 10, "gemm_q8") || !to_i64(a[7], &activation) || !to_i64(a[8], &device)) return NULL;
  if (!describe(a[0], &A) || !describe(a[4], &Y) || !float_type(&Y, "Y", &type)) return NULL;
  const int64_t batch = A.g.n == 3 ? A.g.size[0] : -1;
  if (!matrix(a[0], TYPE_I8, device, batch, -1, -1, "A", &A)) return NULL;
  const int64_t M = A.g.size[A.g.n - 2], K = A.g.size[A.g.n - 1];
  if (!matrix(a[2], TYPE_I8, device, batch, -1, K, "B", &B)) return NULL;
  const int64_t N = B.g.size[B.g.n - 2];
  if (!vector(a[1], TYPE_F32, device, batch, M, "scale_a", &sa) || !vector(a[3], TYPE_F32, device, batch, N, "scale_b", &sb) ||
      !matrix(a[4], type, device, batch, M, N, "Y", &Y) || !vector(a[5], type, device, -1, N, "bias", &bias) ||
      !optional_matrix(a[6], type, device, batch, M, N, "residual", &r) || !stream_on(a[9], device, &stream))
    return NULL;
  if (!require(batch <= INT32_MAX && M <= INT32_MAX && N <= INT32_MAX && K <= INT32_MAX, "sizes are 32-bit numbers")) return NULL;
  memset(&d, 0, sizeof(d));
  d.batch = (int32_t)(batch < 0 ? 1 : batch);
  d.M = (int32_t)M;
  d.N = (int32_t)N;
  d.K = (int32_t)K;
  d.lda = A.g.stride[A.g.n - 2];
  d.ldb = B.g.stride[B.g.n - 2];
  d.ldy = Y.g.stride[Y.g.n - 2];
  d.ldr = r.g.stride[r.g.n - 2];
  if (batch >= 0) {
    d.batch_stride_a = A.g.stride[0];
    d.batch_stride_b = B.g.stride[0];
    d.batch_stride_y = Y.g.stride[0];
    d.batch_stride_r = r.g.stride[0];
  }
  d.dtype = type;
  d.activation = (int32_t)activation;
  comfuse_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = f_gemm_q8(&d, (const int8_t*)A.p, (const float*)sa, (const int8_t*)B.p, (const float*)sb, bias, r.p, (void*)Y.p, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

// ---- the key-value cache
typedef comfuse_status_t (*rotary_fn)(const comfuse_rotary_desc_t*, const comfuse_rotary_t*, const void*, void*, void*);
typedef comfuse_status_t (*cache_write_fn)(const comfuse_cache_write_desc_t*, const comfuse_kv_cache_t*, const comfuse_rotary_t*, const void*, const void*, const void*, void*, const int64_t*,
                                           void*);
typedef comfuse_status_t (*cache_read_fn)(const comfuse_cache_read_desc_t*, const comfuse_kv_cache_t*, const int64_t*, void*, void*, void*);
typedef comfuse_status_t (*paged_attention_fn)(const comfuse_paged_attention_desc_t*, const comfuse_kv_cache_t*, const void*, const int32_t*, const int32_t*, const float*, void*, float*, void*,
                                               size_t, void*);
typedef comfuse_status_t (*paged_attention_size_fn)(const comfuse_paged_attention_desc_t*, const comfuse_kv_cache_t*, size_t*);
static rotary_fn f_rotary;
static cache_write_fn f_cache_write;
static cache_read_fn f_cache_read;
static paged_attention_fn f_paged_attention;
static paged_attention_size_fn f_paged_attention_size;

// A tensor of n dimensions with the given element type (or, type < 0, wide type) and, where they are given (>= 0), sizes; its last dimension is dense.
static int shaped(Described* d, int type, int wide, int64_t device, int n, const int64_t* sizes, const char* what) {
  if (type >= 0 ? d->type != type : d->wide != wide) return refuse(what, "has another element type than the call takes");
  int same = d->g.n == n;
  for (int i = 0; same && i < n; ++i) same = sizes[i] < 0 ? d->g.size[i] <= INT32_MAX : d->g.size[i] == sizes[i];
  if (!same) return refuse(what, "has a shape that does not match the call");
  if (d->device != device) return refuse(what, "is not on the current device");
  if (n > 0 && d->g.stride[n - 1] != 1 && d->g.size[n - 1] != 1) return refuse(what, "must be dense in its last dimension");
  return 1;
}
static int tensor(PyObject* t, int type, int wide, int64_t device, int n, const int64_t* sizes, const char* what, Described* d) {
  return describe(t, d) && shaped(d, type, wide, device, n, sizes, what);
}
static int dense(const Described* d, const char* what) {
  int64_t want = 1;
  for (int i = d->g.n - 1; i >= 0; --i) {
    if (d->g.size[i] != 1 && d->g.stride[i] != want) return refuse(what, "must be dense");
    want *= d->g.size[i];
  }
  return 1;
}
static int type_16(PyObject* t, const char* what, Described* d, int* type) {
  if (!describe(t, d)) return 0;
  *type = d->type;
  return d->type == TYPE_BF16 || d->type == TYPE_F16 ? 1 : refuse(what, "has another element type than the call takes");
}
static int no_negative_strides(const Described* d, const char* what) {
  for (int i = 0; i < d->g.n; ++i)
    if (d->g.stride[i] < 0) return refuse(what, "has a negative stride");
  return 1;
}

// a = (positions, freqs, sections, adjacent, inverse), for `tokens` rows
static int fill_rotary(PyObject* const* a, int64_t device, int64_t tokens, comfuse_rotary_t* r) {
  Described pos, freqs;
  memset(r, 0, sizeof(*r));
  const int64_t any[1] = {-1};
  if (!tensor(a[1], -1, WIDE_F64, device, 1, any, "freqs", &freqs) || !describe(a[0], &pos)) return 0;
  const int axes = pos.g.n == 2 ? (int)(pos.g.size[0] <= 4 ? pos.g.size[0] : 5) : 1;
  const int64_t one[1] = {tokens}, more[2] = {-1, tokens};
  if (!shaped(&pos, -1, WIDE_I32, device, pos.g.n == 2 ? 2 : 1, pos.g.n == 2 ? more : one, "positions") || !no_negative_strides(&pos, "positions")) return 0;
  if (!require(axes <= 4, "positions has more than 4 axes")) return 0;
  r->positions = pos.p;
  r->axis_stride = axes > 1 ? pos.g.stride[0] : 0;
  r->axes = axes;
  r->freqs = freqs.p;
  r->pairs = (int32_t)freqs.g.size[0];
  if (a[2] == Py_None) {
    if (!require(axes == 1, "sections has to say how many pairs belong to each axis")) return 0;
    r->sections[0] = r->pairs;
  } else {
    int64_t s[MAX_DIMS], sum = 0;
    int n = 0;
    if (!tuple_i64(Py_NewRef(a[2]), s, &n)) return 0;
    if (!require(n == axes, "sections and positions name different numbers of axes")) return 0;
    for (int i = 0; i < n; ++i) {
      if (!require(s[i] >= 0 && s[i] <= r->pairs, "sections does not add up to the pairs")) return 0;
      r->sections[i] = (int32_t)s[i];
      sum += s[i];
    }
    if (!require(sum == r->pairs, "sections does not add up to the pairs")) return 0;
  }
  r->adjacent = PyObject_IsTrue(a[3]);
  r->inverse = PyObject_IsTrue(a[4]);
  return r->adjacent >= 0 && r->inverse >= 0;
}

// a = (k_cache, v_cache, k_scale, v_scale), `type` of the rows around
static int fill_cache(PyObject* const* a, int type, int64_t device, comfuse_kv_cache_t* c) {
  Described k, v, ks, vs;
  const int64_t any[4] = {-1, -1, -1, -1};
  memset(c, 0, sizeof(*c));
  if (!describe(a[0], &k)) return 0;
  const int held = k.type == TYPE_I8 ? TYPE_I8 : type;
  if (!shaped(&k, held, 0, device, 4, any, "k_cache") || !tensor(a[1], held, 0, device, 4, k.g.size, "v_cache", &v) || !no_negative_strides(&k, "k_cache") ||
      !no_negative_strides(&v, "v_cache"))
    return 0;
  c->k = (void*)k.p;
  c->v = (void*)v.p;
  c->pages = (int32_t)k.g.size[0];
  c->heads = (int32_t)k.g.size[1];
  c->page_size = (int32_t)k.g.size[2];
  c->D = (int32_t)k.g.size[3];
  c->dtype = type;
  c->quantized = held == TYPE_I8;
  memcpy(c->k_strides, k.g.stride, sizeof(c->k_strides));
  memcpy(c->v_strides, v.g.stride, sizeof(c->v_strides));
  if (!c->quantized) return require(a[2] == Py_None && a[3] == Py_None, "k_scale and v_scale belong to a cache of int8 codes");
  if (!require(a[2] != Py_None && a[3] != Py_None, "a cache of int8 codes has k_scale and v_scale")) return 0;
  if (!describe(a[2], &ks) || !describe(a[3], &vs)) return 0;
  const Described* const both[2] = {&ks, &vs};
  for (int i = 0; i < 2; ++i) {  // (any strides, the last one too)
    const char* what = i ? "v_scale" : "k_scale";
    const Described* d = both[i];
    if (d->type != TYPE_F32) return refuse(what, "has another element type than the call takes");
    if (d->g.n != 3 || memcmp(d->g.size, k.g.size, 3 * sizeof(int64_t)) != 0) return refuse(what, "has a shape that does not match the call");
    if (d->device != device) return refuse(what, "is not on the current device");
    if (!no_negative_strides(d, what)) return 0;
  }
  c->k_scale = (float*)ks.p;
  c->v_scale = (float*)vs.p;
  memcpy(c->k_scale_strides, ks.g.stride, sizeof(c->k_scale_strides));
  memcpy(c->v_scale_strides, vs.g.stride, sizeof(c->v_scale_strides));
  return 1;
}
// Rows [tokens, heads, D]
static int rows_described(Described* d, int type, int64_t device, int64_t tokens, int64_t heads, int64_t D, const char* what, int64_t* strides) {
  const int64_t sizes[3] = {tokens, heads, D};
  if (!shaped(d, type, 0, device, 3, sizes, what) || !no_negative_strides(d, what)) return 0;
  strides[0] = d->g.stride[0];
  strides[1] = d->g.stride[1];
  return 1;
}
static int rows_of(PyObject* t, int type, int64_t device, int64_t tokens, int64_t heads, int64_t D, const char* what, int64_t* strides, Described* d) {
  return describe(t, d) && rows_described(d, type, device, tokens, heads, D, what, strides);
}
static int slots_of(PyObject* t, int64_t device, int64_t tokens, Described* d) {
  const int64_t sizes[1] = {tokens};
  return tensor(t, -1, WIDE_I64, device, 1, sizes, "slots", d);
}

// rotary(x, positions, freqs, sections, adjacent, inverse, out, device, stream) -> status
static PyObject* py_rotary(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  comfuse_rotary_desc_t d;
  comfuse_rotary_t r;
  Described x, out;
  int64_t device;
  void* stream;
  int type;
  memset(&d, 0, sizeof(d));
  if (!fixed_args(n, 9, "rotary") || !to_i64(a[7], &device) || !describe(a[0], &x) || !float_type(&x, "x", &type)) return NULL;
  if (!rows_described(&x, type, device, -1, -1, -1, "x", d.x_strides) || !fill_rotary(a + 1, device, x.g.size[0], &r) ||
      !rows_of(a[6], type, device, x.g.size[0], x.g.size[1], x.g.size[2], "out", d.out_strides, &out) || !stream_on(a[8], device, &stream))
    return NULL;
  d.tokens = (int32_t)x.g.size[0];
  d.heads = (int32_t)x.g.size[1];
  d.D = (int32_t)x.g.size[2];
  d.dtype = type;
  comfuse_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = f_rotary(&d, &r, x.p, (void*)out.p, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

// cache_write(k, v, k_cache, v_cache, k_scale, v_scale, slots, q, q_out, positions, freqs, sections, adjacent, inverse, device, stream) -> status
static PyObject* py_cache_write(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  comfuse_cache_write_desc_t d;
  comfuse_kv_cache_t c;
  comfuse_rotary_t r;
  Described k, v, q, q_out, slots;
  int64_t device;
  void* stream;
  int type;
  memset(&d, 0, sizeof(d));
  q.p = q_out.p = NULL;
  if (!fixed_args(n, 16, "cache_write") || !to_i64(a[14], &device) || !type_16(a[0], "k", &k, &type) || !fill_cache(a + 2, type, device, &c)) return NULL;
  if (!rows_described(&k, type, device, -1, c.heads, c.D, "k", d.k_strides)) return NULL;
  const int64_t tokens = k.g.size[0];
  if (!rows_of(a[1], type, device, tokens, c.heads, c.D, "v", d.v_strides, &v) || !slots_of(a[6], device, tokens, &slots)) return NULL;
  if (!require((a[7] == Py_None) == (a[8] == Py_None), "q and q_out come together") || !require((a[9] == Py_None) == (a[10] == Py_None), "positions and freqs come together") ||
      !require(a[7] == Py_None || a[9] != Py_None, "q is there to be turned: positions and freqs are missing"))
    return NULL;
  const int turned = a[9] != Py_None;
  if (turned && !fill_rotary(a + 9, device, tokens, &r)) return NULL;
  if (a[7] != Py_None) {
    if (!rows_of(a[7], type, device, tokens, -1, c.D, "q", d.q_strides, &q) || !rows_of(a[8], type, device, tokens, q.g.size[1], c.D, "q_out", d.q_out_strides, &q_out)) return NULL;
    if (!require(q.g.size[1] > 0, "q has no heads")) return NULL;
    d.q_heads = (int32_t)q.g.size[1];
  }
  if (!stream_on(a[15], device, &stream)) return NULL;
  d.tokens = (int32_t)tokens;
  comfuse_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = f_cache_write(&d, &c, turned ? &r : NULL, k.p, v.p, q.p, (void*)q_out.p, (const int64_t*)slots.p, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

// cache_read(k_cache, v_cache, k_scale, v_scale, slots, k, v, device, stream) -> status
static PyObject* py_cache_read(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  comfuse_cache_read_desc_t d;
  comfuse_kv_cache_t c;
  Described k, v, slots;
  int64_t device;
  void* stream;
  int type;
  memset(&d, 0, sizeof(d));
  if (!fixed_args(n, 9, "cache_read") || !to_i64(a[7], &device) || !type_16(a[5], "k", &k, &type) || !fill_cache(a, type, device, &c)) return NULL;
  if (!rows_described(&k, type, device, -1, c.heads, c.D, "k", d.k_strides)) return NULL;
  const int64_t tokens = k.g.size[0];
  if (!rows_of(a[6], type, device, tokens, c.heads, c.D, "v", d.v_strides, &v) || !slots_of(a[4], device, tokens, &slots) || !stream_on(a[8], device, &stream)) return NULL;
  d.tokens = (int32_t)tokens;
  comfuse_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = f_cache_read(&d, &c, (const int64_t*)slots.p, (void*)k.p, (void*)v.p, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

// a = (q, k_cache, v_cache, k_scale, v_scale, table, alpha, softcap, window, max_length): what the workspace's size depends on
static int fill_attention(PyObject* const* a, int64_t device, comfuse_paged_attention_desc_t* d, comfuse_kv_cache_t* c, Described* q, Described* table, int* type) {
  int64_t window, max_length;
  double alpha, softcap;
  memset(d, 0, sizeof(*d));
  if (!type_16(a[0], "q", q, type) || !fill_cache(a + 1, *type, device, c)) return 0;
  const int dims = q->g.n == 3 ? 3 : 4;  // [sequences, heads, D]: one new token each
  const int64_t three[3] = {-1, -1, c->D}, four[4] = {-1, -1, -1, c->D};
  if (!shaped(q, *type, 0, device, dims, dims == 3 ? three : four, "q") || !no_negative_strides(q, "q")) return 0;
  const int64_t batch = q->g.size[0], width[2] = {batch, -1};
  if (!tensor(a[5], -1, WIDE_I32, device, 2, width, "page_table", table) || !no_negative_strides(table, "page_table")) return 0;
  if (a[6] == Py_None) alpha = 0.;
  else if (!to_f64(a[6], &alpha)) return 0;
  if (!to_f64(a[7], &softcap) || !to_i64(a[8], &window)) return 0;
  if (a[9] == Py_None) max_length = 0;
  else if (!to_i64(a[9], &max_length) || !require(max_length >= 1, "max_length is at least 1")) return 0;
  if (!require(window >= 0, "window is not negative")) return 0;
  d->batch = (int32_t)batch;
  d->tokens = dims == 3 ? 1 : (int32_t)q->g.size[1];
  d->q_heads = (int32_t)q->g.size[dims - 2];
  d->table_width = (int32_t)table->g.size[1];
  d->table_stride = table->g.stride[0];
  d->q_strides[0] = q->g.stride[0];
  d->q_strides[1] = dims == 3 ? 0 : q->g.stride[1];
  d->q_strides[2] = q->g.stride[dims - 2];
  d->max_length = (int32_t)(max_length > INT32_MAX ? INT32_MAX : max_length);
  d->window = (int32_t)(window > INT32_MAX ? INT32_MAX : window);
  d->alpha = (float)alpha;
  d->softcap = (float)softcap;
  return 1;
}

// paged_attention(<the arguments of fill_attention>, lengths, slopes, out, lse, workspace, device, stream) -> status
static PyObject* py_paged_attention(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  comfuse_paged_attention_desc_t d;
  comfuse_kv_cache_t c;
  Described q, table, lengths, slopes, out, lse, ws;
  int64_t device;
  void* stream;
  int type;
  size_t ws_bytes = 0;
  slopes.p = lse.p = ws.p = NULL;
  if (!fixed_args(n, 17, "paged_attention") || !to_i64(a[15], &device) || !fill_attention(a, device, &d, &c, &q, &table, &type)) return NULL;
  const int dims = q.g.n;
  const int64_t batch[1] = {d.batch}, heads[1] = {d.q_heads};
  if (!tensor(a[10], -1, WIDE_I32, device, 1, batch, "lengths", &lengths) || !tensor(a[12], type, 0, device, dims, q.g.size, "out", &out) || !no_negative_strides(&out, "out")) return NULL;
  if (a[11] != Py_None && !tensor(a[11], TYPE_F32, 0, device, 1, heads, "slopes", &slopes)) return NULL;
  if (a[13] != Py_None && (!tensor(a[13], TYPE_F32, 0, device, dims - 1, q.g.size, "lse", &lse) || !dense(&lse, "lse"))) return NULL;
  if (a[14] != Py_None) {
    void* p;
    if (!describe(a[14], &ws)) return NULL;
    if (ws.device != device) return refuse("workspace", "is not on the current device"), NULL;
    if (!dense(&ws, "workspace")) return NULL;
    ws_bytes = (size_t)ws.bytes;
    for (int i = 0; i < ws.g.n; ++i) ws_bytes *= (size_t)ws.g.size[i];
    if (!ws.bytes && !workspace_of(a[14], &p, &ws_bytes)) return NULL;
  }
  if (!stream_on(a[16], device, &stream)) return NULL;
  d.out_strides[0] = out.g.stride[0];
  d.out_strides[1] = dims == 3 ? 0 : out.g.stride[1];
  d.out_strides[2] = out.g.stride[dims - 2];
  comfuse_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = f_paged_attention(&d, &c, q.p, table.p, lengths.p, slopes.p, (void*)out.p, (float*)lse.p, (void*)ws.p, ws_bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

// paged_attention_size(<the arguments of fill_attention>, device) -> (status, bytes)
static PyObject* py_paged_attention_size(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  comfuse_paged_attention_desc_t d;
  comfuse_kv_cache_t c;
  Described q, table;
  int64_t device;
  int type;
  size_t bytes = 0;
  if (!fixed_args(n, 11, "paged_attention_size") || !to_i64(a[10], &device) || !fill_attention(a, device, &d, &c, &q, &table, &type)) return NULL;
  const comfuse_status_t st = f_paged_attention_size(&d, &c, &bytes);
  return Py_BuildValue("iK", (int)st, (unsigned long long)bytes);
}

// bind_kv(addresses of comfuse_rotary, _cache_write, _cache_read, _paged_attention, _paged_attention_workspace_size, the tensor library's int32, int64 and fp64 types)
static PyObject* py_bind_kv(PyObject* self, PyObject* args) {
  unsigned long long f[5];
  PyObject* t[3];
  if (!PyArg_ParseTuple(args, "KKKKKOOO", f, f + 1, f + 2, f + 3, f + 4, t, t + 1, t + 2)) return NULL;
  f_rotary = (rotary_fn)(uintptr_t)f[0];
  f_cache_write = (cache_write_fn)(uintptr_t)f[1];
  f_cache_read = (cache_read_fn)(uintptr_t)f[2];
  f_paged_attention = (paged_attention_fn)(uintptr_t)f[3];
  f_paged_attention_size = (paged_attention_size_fn)(uintptr_t)f[4];
  t_i32 = Py_NewRef(t[0]);
  t_i64 = Py_NewRef(t[1]);
  t_f64 = Py_NewRef(t[2]);
  Py_RETURN_NONE;
}

// stream(function or stream object, device) -> the handle that a call would use
static PyObject* py_stream(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t device;
  void* out;
  if (!fixed_args(n, 2, "stream") || !to_i64(a[1], &device) || !stream_on(a[0], device, &out)) return NULL;
  return PyLong_FromUnsignedLongLong((unsigned long long)(uintptr_t)out);
}

// describe(tensor) -> (element type, device, address, shape, strides), as the 8-bit entry points see it
static PyObject* py_describe(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Described d;
  if (!fixed_args(n, 1, "describe") || !describe(a[0], &d)) return NULL;
  PyObject *size = PyTuple_New(d.g.n), *stride = PyTuple_New(d.g.n);
  for (int i = 0; size && stride && i < d.g.n; ++i) {
    PyTuple_SET_ITEM(size, i, PyLong_FromLongLong(d.g.size[i]));
    PyTuple_SET_ITEM(stride, i, PyLong_FromLongLong(d.g.stride[i]));
  }
  return Py_BuildValue("iLKNN", d.type, (long long)d.device, (unsigned long long)(uintptr_t)d.p, size, stride);
}

// bind_q8(address of comfuse_quantize_rows, of comfuse_gemm_q8, the tensor library's bf16, fp16, fp32 and int8 types, its tensor class, the class's
// DLPack exchange capsule or None)
static PyObject* py_bind_q8(PyObject* self, PyObject* args) {
  unsigned long long r, g;
  PyObject *t[4], *type, *capsule;
  if (!PyArg_ParseTuple(args, "KKOOOOO!O", &r, &g, t, t + 1, t + 2, t + 3, &PyType_Type, &type, &capsule)) return NULL;
  f_quantize_rows = (quantize_rows_fn)(uintptr_t)r;
  f_gemm_q8 = (gemm_q8_fn)(uintptr_t)g;
  t_bf16 = Py_NewRef(t[0]);
  t_f16 = Py_NewRef(t[1]);
  t_f32 = Py_NewRef(t[2]);
  t_i8 = Py_NewRef(t[3]);
  dl_exchange = NULL;
  if (capsule != Py_None) {
    const DlExchange* e = PyCapsule_GetPointer(capsule, "dlpack_exchange_api");
    if (!e) return NULL;
    if (e->version.major == 1 && e->tensor_from_object) {  // (a minor version only adds to the end)
      dl_type = (PyTypeObject*)Py_NewRef(type);
      dl_exchange = e;
    }
  }
  Py_RETURN_NONE;
}

// bind(address of comfuse_gemm_epilogue, of comfuse_b2b_gemm, of comfuse_gemm_spec): the loaded library's entry points
static PyObject* py_bind(PyObject* self, PyObject* args) {
  unsigned long long e, b, s;
  if (!PyArg_ParseTuple(args, "KKK", &e, &b, &s)) return NULL;
  f_gemm_epilogue = (gemm_epilogue_fn)(uintptr_t)e;
  f_b2b_gemm = (b2b_gemm_fn)(uintptr_t)b;
  f_gemm_spec = (gemm_spec_fn)(uintptr_t)s;
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", py_bind, METH_VARARGS, NULL},
    {"gemm_desc", (PyCFunction)(void (*)(void))py_gemm_desc, METH_FASTCALL, NULL},
    {"gemm_epilogue", (PyCFunction)(void (*)(void))py_gemm_epilogue, METH_FASTCALL, NULL},
    {"b2b", (PyCFunction)(void (*)(void))py_b2b, METH_FASTCALL, NULL},
    {"gemm_spec", (PyCFunction)(void (*)(void))py_gemm_spec, METH_FASTCALL, NULL},
    {"bind_q8", py_bind_q8, METH_VARARGS, NULL},
    {"stream", (PyCFunction)(void (*)(void))py_stream, METH_FASTCALL, NULL},
    {"describe", (PyCFunction)(void (*)(void))py_describe, METH_FASTCALL, NULL},
    {"bind_kv", py_bind_kv, METH_VARARGS, NULL},
    {"rotary", (PyCFunction)(void (*)(void))py_rotary, METH_FASTCALL, NULL},
    {"cache_write", (PyCFunction)(void (*)(void))py_cache_write, METH_FASTCALL, NULL},
    {"cache_read", (PyCFunction)(void (*)(void))py_cache_read, METH_FASTCALL, NULL},
    {"paged_attention", (PyCFunction)(void (*)(void))py_paged_attention, METH_FASTCALL, NULL},
    {"paged_attention_size", (PyCFunction)(void (*)(void))py_paged_attention_size, METH_FASTCALL, NULL},
    {"quantize_rows", (PyCFunction)(void (*)(void))py_quantize_rows, METH_FASTCALL, NULL},
    {"gemm_q8", (PyCFunction)(void (*)(void))py_gemm_q8, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__binding(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_dim = PyUnicode_InternFromString("dim");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_numel = PyUnicode_InternFromString("numel");
  s_element_size = PyUnicode_InternFromString("element_size");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_get_device = PyUnicode_InternFromString("get_device");
  return PyModule_Create(&module);
}
