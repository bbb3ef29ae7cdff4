// Argument marshalling of the entry points on 4-bit data and on pages for Python, natively: at a decode step's sizes a call is bound by what the host
// does for it, and checking a dozen tensors and filling the C structs takes longer in Python than the launches do.  Nothing is kept
// between calls.  Every check that fails raises the package's CcaError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>

#include "../../include/cca.h"

namespace {

struct Handle {                      // what the methods need of a CCA object
  cca_handle* h;
  int64_t E, hq, hk, dh, k_seq, k_ch;
  int device;
};

// The Python and the torch that this was compiled against, for the build to compare.
__attribute__((used)) const char built_for[] = CCA_BUILT_FOR;

PyObject* cca_error = nullptr;       // the package's CcaError once it has been set
struct Raised {};                    // a Python exception is set

[[noreturn]] void refuse(const std::string& msg) {
  PyErr_SetString(cca_error ? cca_error : PyExc_RuntimeError, msg.c_str());
  throw Raised();
}
Handle* handle_of(PyObject* o) {
  auto* p = static_cast<Handle*>(PyCapsule_GetPointer(o, "cca_handle"));
  if (!p) throw Raised();
  return p;
}
const at::Tensor& tensor_of(PyObject* o, const char* name) {
  if (!o || !THPVariable_Check(o)) refuse(std::string(name) + ": wants a tensor");
  return THPVariable_Unpack(o);
}
// A contiguous tensor of this type and shape on the handle's device.
void* need(const at::Tensor& t, const char* name, at::ScalarType type, std::initializer_list<int64_t> shape, const Handle* h) {
  if (t.scalar_type() == type && t.get_device() == h->device && t.is_contiguous() &&
      t.sizes() == at::IntArrayRef(shape.begin(), shape.size()))
    return t.data_ptr();
  auto dims = [](at::IntArrayRef d) {
    std::string r = "(";
    for (size_t i = 0; i < d.size(); ++i) r += (i ? ", " : "") + std::to_string(d[i]);
    return r + ")";
  };
  refuse(std::string(name) + ": wants a contiguous " + c10::toString(type) + " tensor of shape " +
         dims(at::IntArrayRef(shape.begin(), shape.size())) + " on cuda:" + std::to_string(h->device) + ", got " +
         c10::toString(t.scalar_type()) + " " + dims(t.sizes()) + " on " + t.device().str() + (t.is_contiguous() ? "" : ", not contiguous"));
}
void* need(PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> shape, const Handle* h) {
  return need(tensor_of(o, name), name, type, shape, h);
}
bool absent(PyObject* o) { return !o || o == Py_None; }
PyObject* item_of(PyObject* dict, PyObject* key, const char* name) {       // borrowed, null if there is none
  if (!PyDict_Check(dict)) refuse(std::string("wants a dict that holds \"") + name + "\"");
  PyObject* o = PyDict_GetItemWithError(dict, key);
  if (!o && PyErr_Occurred()) throw Raised();
  return o;
}
// The key is made once, with its hash.
#define ITEM(dict, name) item_of(dict, [] { static PyObject* k = PyUnicode_InternFromString(name); return k; }(), name)
int64_t whole(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}
void check(int code, const Handle* h, const char* what) {
  if (code == CCA_OK) return;
  refuse(std::string(what) + ": " + cca_status_string(code) +
         (code == CCA_ERR_CUDA ? " (cudaError " + std::to_string(cca_last_cuda_error(h->h)) + ")" : ""));
}
void* stream(const Handle* h) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)h->device).stream(); }
at::Tensor fresh(std::initializer_list<int64_t> shape, at::ScalarType type, const Handle* h) {
  return at::detail::empty_cuda(at::IntArrayRef(shape.begin(), shape.size()), type, at::Device(at::kCUDA, (c10::DeviceIndex)h->device),
                                c10::nullopt);
}
struct Workspace { void* p; size_t n; };
Workspace workspace_of(PyObject* o, const Handle* h) {
  const at::Tensor& t = tensor_of(o, "workspace");
  if (t.scalar_type() != at::kByte || t.get_device() != h->device || !t.is_contiguous())
    refuse("workspace: wants a contiguous uint8 tensor on the handle's device");
  const uintptr_t p = reinterpret_cast<uintptr_t>(t.data_ptr()), a = (p + 255) / 256 * 256;
  const size_t n = (size_t)t.numel();
  return {reinterpret_cast<void*>(a), n > a - p ? n - (a - p) : 0};
}

// The dict of tensors that new_qcache makes; "weight" and "position" may be absent.
cca_qcache qcache_of(PyObject* d, const Handle* h, int64_t* B) {
  cca_qcache c;
  const at::Tensor &len = tensor_of(ITEM(d, "len"), "len"), &codes = tensor_of(ITEM(d, "k_codes"), "k_codes");
  if (len.dim() != 1 || codes.dim() != 4) refuse("len: wants one dimension, k_codes: four");
  const int64_t b = len.size(0), S = codes.size(2), hk = h->hk, dh = h->dh;
  c.k_codes = need(codes, "k_codes", at::kByte, {b, hk, S, dh / 2}, h);
  c.v_codes = need(ITEM(d, "v_codes"), "v_codes", at::kByte, {b, hk, S, dh / 2}, h);
  c.k_scales = need(ITEM(d, "k_scales"), "k_scales", at::kBFloat16, {b, hk, S, dh / 32}, h);
  c.v_scales = need(ITEM(d, "v_scales"), "v_scales", at::kBFloat16, {b, hk, S, dh / 32}, h);
  PyObject *w = ITEM(d, "weight"), *p = ITEM(d, "position");
  c.weight = absent(w) ? nullptr : static_cast<float*>(need(w, "weight", at::kFloat, {b, hk, S}, h));
  c.position = absent(p) ? nullptr : static_cast<int32_t*>(need(p, "position", at::kInt, {b, hk, S}, h));
  c.len = static_cast<int32_t*>(need(len, "len", at::kInt, {b}, h));
  c.S_max = S;
  *B = b;
  return c;
}
cca_qlinear_weights qlinear_of(PyObject* d, const Handle* h) {
  PyObject *n = ITEM(d, "N"), *k = ITEM(d, "K");
  if (!n || !k) refuse("wants a dict that holds \"N\" and \"K\"");
  const int64_t N = whole(n), K = whole(k), n16 = (N + 15) / 16, k128 = (K + 127) / 128;
  return {need(ITEM(d, "codes"), "codes", at::kByte, {n16, k128, 16, 64}, h),
          need(ITEM(d, "scales"), "scales", at::kBFloat16, {n16, k128, 16, 4}, h), N, K};
}
cca_q_decode_state state_of(PyObject* d, const Handle* h, int64_t* B) {
  cca_q_decode_state s;
  PyObject* cache = ITEM(d, "cache");
  if (!cache) refuse("state: wants \"cache\"");
  s.cache = qcache_of(cache, h, B);
  const int64_t pad = h->k_seq + h->k_ch - 2, L = (h->hq + h->hk) * h->dh;
  s.qk0_hist = pad > 0 ? need(ITEM(d, "qk0_hist"), "qk0_hist", at::kFloat, {*B, pad, L}, h) : nullptr;
  s.x_prev = need(ITEM(d, "x_prev"), "x_prev", at::kBFloat16, {*B, h->E}, h);
  s.pos = static_cast<int32_t*>(need(ITEM(d, "pos"), "pos", at::kInt, {*B}, h));
  return s;
}

// The dict of tensors that new_pages makes.
cca_pages pages_of(PyObject* d, const Handle* h, int64_t* B) {
  cca_pages c;
  const at::Tensor &k = tensor_of(ITEM(d, "k"), "k"), &table = tensor_of(ITEM(d, "table"), "table");
  if (k.dim() != 4 || table.dim() != 2) refuse("k: wants four dimensions, table: two");
  const int64_t n = k.size(0), P = k.size(2), b = table.size(0), wide = table.size(1);
  c.k = need(k, "k", at::kBFloat16, {n, h->hk, P, h->dh}, h);
  c.v = need(ITEM(d, "v"), "v", at::kBFloat16, {n, h->hk, P, h->dh}, h);
  c.refs = static_cast<int32_t*>(need(ITEM(d, "refs"), "refs", at::kInt, {n}, h));
  c.table = static_cast<int32_t*>(need(table, "table", at::kInt, {b, wide}, h));
  c.len = static_cast<int32_t*>(need(ITEM(d, "len"), "len", at::kInt, {b}, h));
  c.n_pages = n;
  c.page_size = P;
  c.max_pages = wide;
  *B = b;
  return c;
}
int32_t* optional_ints(PyObject* o, const char* name, std::initializer_list<int64_t> shape, const Handle* h) {
  return absent(o) ? nullptr : static_cast<int32_t*>(need(o, name, at::kInt, shape, h));
}

// A method: refuses the wrong number of arguments, turns C++ exceptions into Python's.
template <int N, typename F>
PyObject* method(PyObject* const* a, Py_ssize_t n, F f) {
  if (n != N) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  try {
    return f();
  } catch (const Raised&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
PyObject* none() { Py_RETURN_NONE; }

PyObject* new_handle(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<8>(a, n, [&] {
    auto* h = new Handle{reinterpret_cast<cca_handle*>(PyLong_AsVoidPtr(a[0])), whole(a[1]), whole(a[2]), whole(a[3]), whole(a[4]),
                         whole(a[5]), whole(a[6]), (int)whole(a[7])};
    return PyCapsule_New(h, "cca_handle", [](PyObject* o) { delete static_cast<Handle*>(PyCapsule_GetPointer(o, "cca_handle")); });
  });
}
PyObject* close_handle(PyObject*, PyObject* const* a, Py_ssize_t n) {       // every later call is refused
  return method<1>(a, n, [&] { handle_of(a[0])->h = nullptr; return none(); });
}
PyObject* set_error(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<1>(a, n, [&] { Py_INCREF(a[0]); cca_error = a[0]; return none(); });
}

// (handle, cache, k, v, position | None, count | None)
PyObject* qcache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<6>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_qcache c = qcache_of(a[1], h, &B);
    const at::Tensor& k = tensor_of(a[2], "k");
    const int64_t rows = k.dim() == 4 ? k.size(1) : 0;
    const void* kp = need(k, "k", at::kBFloat16, {B, rows, h->hk, h->dh}, h);
    const void* vp = need(a[3], "v", at::kBFloat16, {B, rows, h->hk, h->dh}, h);
    auto* pos = absent(a[4]) ? nullptr : static_cast<int32_t*>(need(a[4], "position", at::kInt, {B}, h));
    auto* cnt = absent(a[5]) ? nullptr : static_cast<int32_t*>(need(a[5], "count", at::kInt, {B}, h));
    check(cca_qcache_append(h->h, kp, vp, pos, cnt, &c, B, rows, stream(h)), h, "cca_qcache_append");
    return none();
  });
}
// (handle, cache, n, first | None) -> (k, v)
PyObject* qcache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<4>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_qcache c = qcache_of(a[1], h, &B);
    const int64_t rows = whole(a[2]);
    if (rows < 0) refuse("cca_qcache_read: invalid argument");
    auto* first = absent(a[3]) ? nullptr : static_cast<int32_t*>(need(a[3], "first", at::kInt, {B}, h));
    at::Tensor k = fresh({B, rows, h->hk, h->dh}, at::kFloat, h), v = fresh({B, rows, h->hk, h->dh}, at::kFloat, h);
    check(cca_qcache_read(h->h, &c, first, static_cast<float*>(k.data_ptr()), static_cast<float*>(v.data_ptr()), B, rows, stream(h)), h,
          "cca_qcache_read");
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(k)), THPVariable_Wrap(std::move(v)));
  });
}
// (handle, q, cache, max_len, workspace, out | None, accumulate | None) -> out
PyObject* qcache_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<7>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_qcache c = qcache_of(a[2], h, &B);
    const void* q = need(a[1], "q", at::kBFloat16, {B, h->hq, h->dh}, h);
    const Workspace ws = workspace_of(a[4], h);
    const int64_t max_len = whole(a[3]);
    const int acc = absent(a[6]) ? c.weight != nullptr : PyObject_IsTrue(a[6]);
    if (acc < 0) throw Raised();
    at::Tensor made;
    void* out;
    if (absent(a[5])) {
      made = fresh({B, h->hq, h->dh}, at::kBFloat16, h);
      out = made.data_ptr();
    } else {
      out = need(a[5], "out", at::kBFloat16, {B, h->hq, h->dh}, h);
    }
    check(cca_qcache_attention(h->h, q, out, &c, max_len, acc, ws.p, ws.n, B, stream(h)), h, "cca_qcache_attention");
    if (made.defined()) return THPVariable_Wrap(std::move(made));
    Py_INCREF(a[5]);
    return a[5];
  });
}
// (handle, cache, keep, recent, next_position, max_len, workspace)
PyObject* qcache_evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<7>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_qcache c = qcache_of(a[1], h, &B);
    const int64_t keep = whole(a[2]), recent = whole(a[3]), max_len = whole(a[5]);
    auto* next = static_cast<int32_t*>(need(a[4], "next_position", at::kInt, {B}, h));
    const Workspace ws = workspace_of(a[6], h);
    check(cca_qcache_evict(h->h, &c, keep, recent, next, max_len, ws.p, ws.n, B, stream(h)), h, "cca_qcache_evict");
    return none();
  });
}
// (handle, weights, x, out | None, dtype) -> out
PyObject* qlinear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<5>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    const cca_qlinear_weights w = qlinear_of(a[1], h);
    const at::Tensor& x = tensor_of(a[2], "x");
    const int64_t M = x.dim() > 0 ? x.size(0) : 0;
    const void* xp = need(x, "x", at::kBFloat16, {M, w.K}, h);
    if (!THPDtype_Check(a[4])) refuse("cca_qlinear: out_dtype is no torch.dtype");
    const at::ScalarType type = absent(a[3]) ? reinterpret_cast<THPDtype*>(a[4])->scalar_type : tensor_of(a[3], "out").scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) refuse(std::string("cca_qlinear: output type ") + c10::toString(type));
    at::Tensor made;
    void* out;
    if (absent(a[3])) {
      made = fresh({M, w.N}, type, h);
      out = made.data_ptr();
    } else {
      out = need(a[3], "out", type, {M, w.N}, h);
    }
    check(cca_qlinear(h->h, &w, xp, out, type == at::kFloat, M, stream(h)), h, "cca_qlinear");
    if (made.defined()) return THPVariable_Wrap(std::move(made));
    Py_INCREF(a[3]);
    return a[3];
  });
}
// (handle, w)  w: bf16 [N, K] -> (codes, scales)
PyObject* qlinear_pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<2>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    const at::Tensor& w = tensor_of(a[1], "w");
    if (w.dim() != 2) refuse("w: wants two dimensions");
    const int64_t N = w.size(0), K = w.size(1);
    const void* wp = need(w, "w", at::kBFloat16, {N, K}, h);
    size_t cb, sb;
    check(cca_qlinear_sizes(N, K, &cb, &sb), h, "cca_qlinear_sizes");
    at::Tensor codes = fresh({(N + 15) / 16, (K + 127) / 128, 16, 64}, at::kByte, h);
    at::Tensor scales = fresh({(N + 15) / 16, (K + 127) / 128, 16, 4}, at::kBFloat16, h);
    const cca_qlinear_weights out{codes.data_ptr(), scales.data_ptr(), N, K};
    check(cca_qlinear_pack(h->h, wp, &out, stream(h)), h, "cca_qlinear_pack");
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(codes)), THPVariable_Wrap(std::move(scales)));
  });
}
// (handle, weights, x, state, max_len, workspace, out | None) -> out
PyObject* decode_step_q(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<7>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_q_decode_state s = state_of(a[3], h, &B);
    cca_q_weights w;
    PyObject *qkv = ITEM(a[1], "w_qkv"), *vp = ITEM(a[1], "w_vp"), *up = ITEM(a[1], "w_o");
    if (!qkv || !vp || !up) refuse("weights: wants \"w_qkv\", \"w_vp\" and \"w_o\"");
    w.w_qkv = qlinear_of(qkv, h);
    w.w_vp = qlinear_of(vp, h);
    w.w_o = qlinear_of(up, h);
    const int64_t L = (h->hq + h->hk) * h->dh;
    PyObject *c0 = ITEM(a[1], "conv0_w"), *c1 = ITEM(a[1], "conv1_w"), *t = ITEM(a[1], "temp");
    w.conv0_w = absent(c0) ? nullptr : need(c0, "conv0_w", at::kBFloat16, {L, h->k_seq}, h);
    w.conv1_w = absent(c1) ? nullptr : need(c1, "conv1_w", at::kBFloat16, {L, h->dh, h->k_ch}, h);
    w.temp = absent(t) ? nullptr : static_cast<float*>(need(t, "temp", at::kFloat, {h->hk}, h));
    const void* x = need(a[2], "x", at::kBFloat16, {B, h->E}, h);
    const int64_t max_len = whole(a[4]);
    const Workspace ws = workspace_of(a[5], h);
    at::Tensor made;
    void* out;
    if (absent(a[6])) {
      made = fresh({B, h->E}, at::kBFloat16, h);
      out = made.data_ptr();
    } else {
      out = need(a[6], "out", at::kBFloat16, {B, h->E}, h);
    }
    check(cca_decode_step_q(h->h, &w, x, out, &s, max_len, ws.p, ws.n, B, stream(h)), h, "cca_decode_step_q");
    if (made.defined()) return THPVariable_Wrap(std::move(made));
    Py_INCREF(a[6]);
    return a[6];
  });
}
// (handle, x, workspace, state)
PyObject* decode_state_from_prefill_q(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<4>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_q_decode_state s = state_of(a[3], h, &B);
    const at::Tensor& x = tensor_of(a[1], "x");
    const int64_t S = x.dim() == 3 ? x.size(1) : 0;
    const void* xp = need(x, "x", at::kBFloat16, {B, S, h->E}, h);
    const Workspace ws = workspace_of(a[2], h);
    check(cca_decode_state_from_prefill_q(h->h, xp, ws.p, ws.n, B, S, &s, stream(h)), h, "cca_decode_state_from_prefill_q");
    return none();
  });
}

// (handle, pages, n, workspace, count | None, first | None)
PyObject* pages_reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<6>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_pages c = pages_of(a[1], h, &B);
    const Workspace ws = workspace_of(a[3], h);
    const int32_t *count = optional_ints(a[4], "count", {B}, h), *first = optional_ints(a[5], "first", {B}, h);
    check(cca_pages_reserve(h->h, &c, whole(a[2]), count, first, ws.p, ws.n, B, stream(h)), h, "cca_pages_reserve");
    return none();
  });
}
// (handle, pages, parent, child, workspace)
PyObject* pages_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<5>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_pages c = pages_of(a[1], h, &B);
    const at::Tensor& child = tensor_of(a[3], "child");
    const int64_t pairs = child.dim() == 1 ? child.size(0) : 0;
    auto* cp = static_cast<int32_t*>(need(child, "child", at::kInt, {pairs}, h));
    auto* pp = static_cast<int32_t*>(need(a[2], "parent", at::kInt, {pairs}, h));
    const Workspace ws = workspace_of(a[4], h);
    check(cca_pages_fork(h->h, &c, pp, cp, pairs, ws.p, ws.n, B, stream(h)), h, "cca_pages_fork");
    return none();
  });
}
// (handle, pages, keep)
PyObject* pages_free(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<3>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_pages c = pages_of(a[1], h, &B);
    auto* keep = static_cast<int32_t*>(need(a[2], "keep", at::kInt, {B}, h));
    check(cca_pages_free(h->h, &c, keep, B, stream(h)), h, "cca_pages_free");
    return none();
  });
}
// (handle, pages, workspace, used | None) -> used
PyObject* pages_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<4>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_pages c = pages_of(a[1], h, &B);
    const Workspace ws = workspace_of(a[2], h);
    at::Tensor made;
    int32_t* used = optional_ints(a[3], "used", {1}, h);
    if (!used) {
      made = fresh({1}, at::kInt, h);
      used = static_cast<int32_t*>(made.data_ptr());
    }
    check(cca_pages_compact(h->h, &c, used, ws.p, ws.n, B, stream(h)), h, "cca_pages_compact");
    if (made.defined()) return THPVariable_Wrap(std::move(made));
    Py_INCREF(a[3]);
    return a[3];
  });
}
// (handle, pages, k, v, count | None)
PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<5>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_pages c = pages_of(a[1], h, &B);
    const at::Tensor& k = tensor_of(a[2], "k");
    const int64_t rows = k.dim() == 4 ? k.size(1) : 0;
    const void* kp = need(k, "k", at::kBFloat16, {B, rows, h->hk, h->dh}, h);
    const void* vp = need(a[3], "v", at::kBFloat16, {B, rows, h->hk, h->dh}, h);
    const int32_t* count = optional_ints(a[4], "count", {B}, h);
    check(cca_paged_append(h->h, kp, vp, count, &c, B, rows, stream(h)), h, "cca_paged_append");
    return none();
  });
}
// (handle, pages, n, first | None) -> (k, v)
PyObject* paged_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<4>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_pages c = pages_of(a[1], h, &B);
    const int64_t rows = whole(a[2]);
    if (rows < 0) refuse("cca_paged_read: invalid argument");
    if (rows > (int64_t)1 << 24 || B * rows > (int64_t)1 << 30) check(CCA_ERR_UNSUPPORTED, h, "cca_paged_read");      // (before memory is asked for)
    const int32_t* first = optional_ints(a[3], "first", {B}, h);
    at::Tensor k = fresh({B, rows, h->hk, h->dh}, at::kBFloat16, h), v = fresh({B, rows, h->hk, h->dh}, at::kBFloat16, h);
    check(cca_paged_read(h->h, &c, first, k.data_ptr(), v.data_ptr(), B, rows, stream(h)), h, "cca_paged_read");
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(k)), THPVariable_Wrap(std::move(v)));
  });
}
// (handle, q, pages, max_len, workspace, out | None, lse | None) -> out
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<7>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_pages c = pages_of(a[2], h, &B);
    const void* q = need(a[1], "q", at::kBFloat16, {B, h->hq, h->dh}, h);
    const Workspace ws = workspace_of(a[4], h);
    const int64_t max_len = whole(a[3]);
    auto* lse = absent(a[6]) ? nullptr : static_cast<float*>(need(a[6], "lse", at::kFloat, {B, h->hq}, h));
    at::Tensor made;
    void* out;
    if (absent(a[5])) {
      made = fresh({B, h->hq, h->dh}, at::kBFloat16, h);
      out = made.data_ptr();
    } else {
      out = need(a[5], "out", at::kBFloat16, {B, h->hq, h->dh}, h);
    }
    check(cca_paged_attention(h->h, q, out, lse, &c, max_len, ws.p, ws.n, B, stream(h)), h, "cca_paged_attention");
    if (made.defined()) return THPVariable_Wrap(std::move(made));
    Py_INCREF(a[5]);
    return a[5];
  });
}
cca_paged_decode_state paged_state_of(PyObject* d, const Handle* h, int64_t* B) {
  cca_paged_decode_state s;
  PyObject* pages = ITEM(d, "pages");
  if (!pages) refuse("state: wants \"pages\"");
  s.pages = pages_of(pages, h, B);
  const int64_t pad = h->k_seq + h->k_ch - 2, L = (h->hq + h->hk) * h->dh;
  s.qk0_hist = pad > 0 ? need(ITEM(d, "qk0_hist"), "qk0_hist", at::kFloat, {*B, pad, L}, h) : nullptr;
  s.x_prev = need(ITEM(d, "x_prev"), "x_prev", at::kBFloat16, {*B, h->E}, h);
  return s;
}
// (handle, weights, x, state, max_len, workspace, out | None) -> out
PyObject* decode_step_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<7>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_paged_decode_state s = paged_state_of(a[3], h, &B);
    const int64_t Lq = h->hq * h->dh, Lk = h->hk * h->dh, L = Lq + Lk;
    cca_weights w;
    w.w_qk = need(ITEM(a[1], "w_qk"), "w_qk", at::kBFloat16, {L, h->E}, h);
    w.w_v1 = need(ITEM(a[1], "w_v1"), "w_v1", at::kBFloat16, {Lk / 2, h->E}, h);
    w.w_v2 = need(ITEM(a[1], "w_v2"), "w_v2", at::kBFloat16, {Lk / 2, h->E}, h);
    w.w_o = need(ITEM(a[1], "w_o"), "w_o", at::kBFloat16, {h->E, Lq}, h);
    PyObject *c0 = ITEM(a[1], "conv0_w"), *c1 = ITEM(a[1], "conv1_w"), *t = ITEM(a[1], "temp");
    w.conv0_w = absent(c0) ? nullptr : need(c0, "conv0_w", at::kBFloat16, {L, h->k_seq}, h);
    w.conv1_w = absent(c1) ? nullptr : need(c1, "conv1_w", at::kBFloat16, {L, h->dh, h->k_ch}, h);
    w.temp = absent(t) ? nullptr : static_cast<float*>(need(t, "temp", at::kFloat, {h->hk}, h));
    const void* x = need(a[2], "x", at::kBFloat16, {B, h->E}, h);
    const int64_t max_len = whole(a[4]);
    const Workspace ws = workspace_of(a[5], h);
    at::Tensor made;
    void* out;
    if (absent(a[6])) {
      made = fresh({B, h->E}, at::kBFloat16, h);
      out = made.data_ptr();
    } else {
      out = need(a[6], "out", at::kBFloat16, {B, h->E}, h);
    }
    check(cca_decode_step_paged(h->h, &w, x, out, &s, max_len, ws.p, ws.n, B, stream(h)), h, "cca_decode_step_paged");
    if (made.defined()) return THPVariable_Wrap(std::move(made));
    Py_INCREF(a[6]);
    return a[6];
  });
}
// (handle, x, workspace, state)
PyObject* decode_state_from_prefill_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return method<4>(a, n, [&] {
    const Handle* h = handle_of(a[0]);
    int64_t B;
    const cca_paged_decode_state s = paged_state_of(a[3], h, &B);
    const at::Tensor& x = tensor_of(a[1], "x");
    const int64_t S = x.dim() == 3 ? x.size(1) : 0;
    const void* xp = need(x, "x", at::kBFloat16, {B, S, h->E}, h);
    const Workspace ws = workspace_of(a[2], h);
    check(cca_decode_state_from_prefill_paged(h->h, xp, ws.p, ws.n, B, S, &s, stream(h)), h, "cca_decode_state_from_prefill_paged");
    return none();
  });
}

#define M(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {M(new_handle), M(close_handle), M(set_error), M(qcache_append), M(qcache_read), M(qcache_attention),
                         M(qcache_evict), M(qlinear), M(qlinear_pack), M(decode_step_q), M(decode_state_from_prefill_q),
                         M(pages_reserve), M(pages_fork), M(pages_free), M(pages_compact), M(paged_append), M(paged_read),
                         M(paged_attention), M(decode_step_paged), M(decode_state_from_prefill_paged),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bind() { return PyModule_Create(&module); }
