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
typedef struct {
  Geometry g;
  int type;
  int64_t device;  // -1 = host
  const void* p;
} Described;

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
