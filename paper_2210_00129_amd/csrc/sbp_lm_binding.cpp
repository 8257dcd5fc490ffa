// The language-model steps (sbp_lm.h) between Python and the C ABI, in native code as the calls of sbp_binding.cpp are: checks of the
// tensors, allocation of the outputs and the workspace, the current stream of the tensors' device, the call.
#include "sbp_binding.h"

#include <c10/core/DeviceGuard.h>

#include "sbp_lm.h"

namespace {

decltype(&sbp_forward_attention_masked) f_attn = nullptr;
decltype(&sbp_backward_attention_masked_workspace) f_attn_bwd_ws = nullptr;
decltype(&sbp_backward_attention_masked) f_attn_bwd = nullptr;
decltype(&sbp_forward_residual_norm) f_norm = nullptr;
decltype(&sbp_backward_residual_norm_workspace) f_norm_bwd_ws = nullptr;
decltype(&sbp_backward_residual_norm) f_norm_bwd = nullptr;
decltype(&sbp_forward_embedding) f_emb = nullptr;
decltype(&sbp_backward_embedding_workspace) f_emb_bwd_ws = nullptr;
decltype(&sbp_backward_embedding) f_emb_bwd = nullptr;

float number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PyFail{};
  return (float)v;
}
// a number of a C int field: whole, and refused where it does not fit
int32_t number32(PyObject* o) {
  const int64_t v = integer(o, true);
  if (v != (int32_t)v) fail(PyExc_ValueError, "%s", "a size is beyond 32 bits");
  return (int32_t)v;
}
// flags: 32 bits, and refused where one is set beyond them
uint32_t flags32(PyObject* o) {
  const uint64_t v = bits64(o, true);
  if (v >> 32) fail(PyExc_ValueError, "%s", "unknown flags beyond 32 bits");
  return (uint32_t)v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw PyFail{};
  return v;
}

// address of a tensor (nullptr: NULL) that has to be contiguous, on the device, of this shape and type
template <typename P = void>
P* address(const at::Tensor* t, const char* name, at::IntArrayRef sizes, at::ScalarType type, c10::Device device) {
  if (!t) return nullptr;
  if (!t->is_cuda()) fail(PyExc_ValueError, "%s must live in GPU memory", name);
  if (t->device() != device) fail(PyExc_ValueError, "%s is on another device", name);
  if (t->scalar_type() != type) {
    PyErr_Format(PyExc_TypeError, "%s must be %s, got %s", name, c10::toString(type), c10::toString(t->scalar_type()));
    throw PyFail{};
  }
  if (t->sizes() != sizes) {
    std::string want, got;
    for (int64_t v : sizes) want += (want.empty() ? "" : ", ") + std::to_string(v);
    for (int64_t v : t->sizes()) got += (got.empty() ? "" : ", ") + std::to_string(v);
    PyErr_Format(PyExc_ValueError, "%s must have shape (%s), got (%s)", name, want.c_str(), got.c_str());
    throw PyFail{};
  }
  if (!t->is_contiguous()) fail(PyExc_ValueError, "%s must be contiguous", name);
  return static_cast<P*>(t->data_ptr());
}

const at::Tensor& matrix(PyObject* o, const char* name) {
  const at::Tensor& t = needed(o, name);
  if (!t.is_cuda()) fail(PyExc_ValueError, "%s must live in GPU memory", name);
  if (t.dim() != 2) fail(PyExc_ValueError, "%s must have 2 dimensions", name);
  return t;
}

// the given tensor or a new one, kept in `made`
const at::Tensor* or_new(const at::Tensor* given, at::Tensor& made, at::IntArrayRef sizes, at::ScalarType type, c10::Device device) {
  if (given) return given;
  made = empty(sizes, type, device);
  return &made;
}
struct Workspace {
  at::Tensor made;
  void* p = nullptr;
  size_t bytes = 0;
  Workspace(PyObject* o, size_t need, c10::Device device) {
    const at::Tensor* t = tensor(o, "workspace");
    if (t && (!t->is_cuda() || t->device() != device || !t->is_contiguous())) fail(PyExc_ValueError, "%s", "workspace must be a contiguous tensor on the tensors' device");
    if (!t && need) { made = empty({(int64_t)need}, at::kByte, device); t = &made; }
    if (!t) return;
    p = t->data_ptr();
    bytes = t->nbytes();
  }
};
// the work goes to the current stream of the tensors' device, which is the current device meanwhile
template <class F>
void run(c10::Device device, F&& f) {
  void* const stream = stream_of(device);
  check(enqueue([&] {
    c10::DeviceGuard guard(device);
    return f(stream);
  }));
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    count(n, 11);
    f_attn = reinterpret_cast<decltype(f_attn)>(bits64(a[0]));
    f_attn_bwd_ws = reinterpret_cast<decltype(f_attn_bwd_ws)>(bits64(a[1]));
    f_attn_bwd = reinterpret_cast<decltype(f_attn_bwd)>(bits64(a[2]));
    f_norm = reinterpret_cast<decltype(f_norm)>(bits64(a[3]));
    f_norm_bwd_ws = reinterpret_cast<decltype(f_norm_bwd_ws)>(bits64(a[4]));
    f_norm_bwd = reinterpret_cast<decltype(f_norm_bwd)>(bits64(a[5]));
    f_emb = reinterpret_cast<decltype(f_emb)>(bits64(a[6]));
    f_emb_bwd_ws = reinterpret_cast<decltype(f_emb_bwd_ws)>(bits64(a[7]));
    f_emb_bwd = reinterpret_cast<decltype(f_emb_bwd)>(bits64(a[8]));
    Py_INCREF(a[9]);
    Py_XDECREF(f_check);
    f_check = a[9];
    Py_INCREF(a[10]);
    Py_XDECREF(f_stream);
    f_stream = a[10];
    Py_RETURN_NONE;
  } catch (const PyFail&) { return nullptr; }
}

// a: h, d, scale, h_kv, cap, causal, slopes, doc, prefix
sbp_attention_desc attention_desc(PyObject* const* a, int32_t B, int32_t n, c10::Device device) {
  sbp_attention_desc d{};
  d.B = B; d.n = n;
  d.h = number32(a[0]); d.d = number32(a[1]); d.scale = number(a[2]);
  d.h_kv = a[3] == Py_None ? d.h : number32(a[3]);
  d.cap = number(a[4]); d.causal = truth(a[5]);
  d.slopes = address<const float>(tensor(a[6], "slopes"), "slopes", {d.h}, at::kFloat, device);
  d.doc = address<const int32_t>(tensor(a[7], "doc"), "doc", {(int64_t)B * n}, at::kInt, device);
  d.prefix = address<const int32_t>(tensor(a[8], "prefix"), "prefix", {B}, at::kInt, device);
  return d;
}
int32_t tokens_per_sample(int64_t rows, int32_t B, const char* what) {
  if (B < 1 || rows % B) fail(PyExc_ValueError, "%s", what);
  const int64_t n = rows / B;
  if (n != (int32_t)n) fail(PyExc_ValueError, "%s", "too many tokens");
  return (int32_t)n;
}

// (qkv, B, h, d, scale, h_kv, cap, causal, slopes, doc, prefix, out, lse_out) -> (A, lse)
PyObject* attention_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    count(n, 13);
    const at::Tensor& qkv = matrix(a[0], "qkv");
    const int32_t code = dtype_code(qkv), B = number32(a[1]);
    const int64_t rows = qkv.size(0);
    const c10::Device device = qkv.device();
    const at::ScalarType type = qkv.scalar_type();
    const sbp_attention_desc d = attention_desc(a + 2, B, tokens_per_sample(rows, B, "rows of qkv must be B * n"), device);
    const int64_t width = (int64_t)d.h * d.d;
    const void* qkv_p = address(&qkv, "qkv", {rows, width + 2 * (int64_t)d.h_kv * d.d}, type, device);
    at::Tensor made_A, made_lse;
    void* A = address(or_new(tensor(a[11], "out"), made_A, {rows, width}, type, device), "out", {rows, width}, type, device);
    float* lse = address<float>(or_new(tensor(a[12], "lse_out"), made_lse, {rows, d.h}, at::kFloat, device), "lse_out", {rows, d.h}, at::kFloat, device);
    run(device, [&](void* s) { return f_attn(&d, qkv_p, code, A, lse, s); });
    return pack({keep_or_wrap(a[11], made_A), keep_or_wrap(a[12], made_lse)});
  } catch (const PyFail&) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// (qkv_k, A_k, dA_k, lse_k, B, h, d, scale, h_kv, cap, causal, slopes, doc, prefix, n, idx, out, workspace) -> dqkv_k
PyObject* attention_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    count(n, 18);
    const at::Tensor& qkv = matrix(a[0], "qkv_k");
    const int32_t code = dtype_code(qkv), B = number32(a[4]);
    const int64_t rows = qkv.size(0);
    const c10::Device device = qkv.device();
    const at::ScalarType type = qkv.scalar_type();
    const int32_t n_k = tokens_per_sample(rows, B, "rows of qkv_k must be B * n_k");
    const at::Tensor* idx = tensor(a[15], "idx");
    if (a[14] == Py_None && idx) fail(PyExc_ValueError, "%s", "n (tokens per sample) is needed with idx");
    const sbp_attention_desc d = attention_desc(a + 5, B, a[14] == Py_None ? n_k : number32(a[14]), device);
    const int64_t width = (int64_t)d.h * d.d, all = width + 2 * (int64_t)d.h_kv * d.d;
    const void* qkv_p = address(&qkv, "qkv_k", {rows, all}, type, device);
    const void* A = address(&needed(a[1], "A_k"), "A_k", {rows, width}, type, device);
    const void* dA = address(&needed(a[2], "dA_k"), "dA_k", {rows, width}, type, device);
    const float* lse = address<const float>(&needed(a[3], "lse_k"), "lse_k", {rows, d.h}, at::kFloat, device);
    const int32_t* ip = address<const int32_t>(idx, "idx", {rows}, at::kInt, device);
    at::Tensor made;
    void* out = address(or_new(tensor(a[16], "out"), made, {rows, all}, type, device), "out", {rows, all}, type, device);
    const Workspace ws(a[17], f_attn_bwd_ws(&d, n_k, code), device);
    run(device, [&](void* s) { return f_attn_bwd(&d, qkv_p, A, dA, lse, ip, n_k, code, out, ws.p, ws.bytes, s); });
    return keep_or_wrap(a[16], made);
  } catch (const PyFail&) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

int32_t channels(int64_t C) {
  if (C != (int32_t)C) fail(PyExc_ValueError, "%s", "too many channels");
  return (int32_t)C;
}

// a: gate, alpha, gamma_post, beta_post, gamma_pre, beta_pre, kind, eps
sbp_residual_norm_desc norm_desc(PyObject* const* a, int64_t M, int64_t C, c10::Device device) {
  sbp_residual_norm_desc d{};
  d.M = M; d.C = channels(C); d.G = 1;
  const at::Tensor* gate = tensor(a[0], "gate");
  if (gate && gate->dim() == 1) {
    d.gate = address<const float>(gate, "gate", {C}, at::kFloat, device);
  } else if (gate) {
    if (gate->dim() != 2) fail(PyExc_ValueError, "%s", "gate must be [C] or [G, C]");
    if (gate->size(0) != (int32_t)gate->size(0)) fail(PyExc_ValueError, "%s", "too many gates");
    d.G = (int32_t)gate->size(0);
    d.gate = address<const float>(gate, "gate", {d.G, C}, at::kFloat, device);
  }
  d.alpha = number(a[1]);
  d.gamma_post = address<const float>(tensor(a[2], "gamma_post"), "gamma_post", {C}, at::kFloat, device);
  d.beta_post = address<const float>(tensor(a[3], "beta_post"), "beta_post", {C}, at::kFloat, device);
  d.gamma_pre = address<const float>(tensor(a[4], "gamma_pre"), "gamma_pre", {C}, at::kFloat, device);
  d.beta_pre = address<const float>(tensor(a[5], "beta_pre"), "beta_pre", {C}, at::kFloat, device);
  d.kind = number32(a[6]); d.eps = number(a[7]);
  return d;
}

// (x, y, gate, alpha, gamma_post, beta_post, gamma_pre, beta_pre, kind, eps, x_out, z) -> (x_out, z)
PyObject* norm_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    count(n, 12);
    const at::Tensor& x = matrix(a[0], "x");
    const int32_t code = dtype_code(x);
    const int64_t M = x.size(0), C = x.size(1);
    const c10::Device device = x.device();
    const at::ScalarType type = x.scalar_type();
    const sbp_residual_norm_desc d = norm_desc(a + 2, M, C, device);
    const void *xp = address(&x, "x", {M, C}, type, device), *yp = address(tensor(a[1], "y"), "y", {M, C}, type, device);
    at::Tensor made_x, made_z;
    const at::Tensor* z = tensor(a[11], "z");
    if (!z && d.gamma_pre) z = or_new(nullptr, made_z, {M, C}, type, device);
    void* x_out = address(or_new(tensor(a[10], "x_out"), made_x, {M, C}, type, device), "x_out", {M, C}, type, device);
    void* zp = address(z, "z", {M, C}, type, device);
    run(device, [&](void* s) { return f_norm(&d, xp, yp, code, x_out, zp, s); });
    return pack({keep_or_wrap(a[10], made_x), keep_or_wrap(a[11], made_z)});
  } catch (const PyFail&) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// what a caller's container lent: it may lose the object while a lookup runs Python code or other threads run
struct Held {
  PyObject* o[7] = {};
  ~Held() { for (PyObject* p : o) Py_XDECREF(p); }
};

const char* const kOutputs[7] = {"dx", "dy_k", "dgate", "dgamma_post", "dbeta_post", "dgamma_pre", "dbeta_pre"};

// (dx_out, dz_k, x_out_k, y_k, idx, M, gate, alpha, gamma_post, beta_post, gamma_pre, None, kind, eps, inv, flags, want, dx, dy_k, grads,
//  workspace) -> dict
PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    count(n, 21);
    const at::Tensor *dx_out = tensor(a[0], "dx_out"), *dz = tensor(a[1], "dz_k"), *x_out = tensor(a[2], "x_out_k"), *y = tensor(a[3], "y_k");
    const at::Tensor *idx = tensor(a[4], "idx"), *inv = tensor(a[14], "inv");
    PyObject* first = y ? a[3] : dz ? a[1] : a[0];
    if (first == Py_None) fail(PyExc_ValueError, "%s", "one of dx_out, dz_k and y_k is needed");
    const at::Tensor& some = matrix(first, "dx_out, dz_k or y_k");
    const int32_t code = dtype_code(some);
    const int64_t C = some.size(1), M = integer(a[5], true);
    const c10::Device device = some.device();
    const at::ScalarType type = some.scalar_type();
    const uint32_t flags = flags32(a[15]);
    const bool compact = flags & SBP_FLAG_DX_COMPACT;
    const int64_t K = idx ? idx->numel() : some.size(0), rows = compact ? K : M;
    const sbp_residual_norm_desc d = norm_desc(a + 6, M, C, device);
    // what is wanted, one bit per output
    unsigned want = 3u | (d.gate ? 4u : 0u) | (d.gamma_post ? 8u : 0u) | (d.beta_post ? 16u : 0u) | (dz ? 32u : 0u);
    if (a[16] != Py_None) {
      want = 0;
      PyObject* list = PySequence_Fast(a[16], "want must be a sequence of names");
      if (!list) throw PyFail{};
      for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(list); ++i) {
        PyObject* name = PySequence_Fast_GET_ITEM(list, i);
        int at = -1;
        for (int q = 0; q < 7; ++q)
          if (PyUnicode_Check(name) && PyUnicode_CompareWithASCIIString(name, kOutputs[q]) == 0) at = q;
        if (at < 0) {
          PyErr_Format(PyExc_ValueError, "unknown output %S", name);
          Py_DECREF(list);
          throw PyFail{};
        }
        want |= 1u << at;
      }
      Py_DECREF(list);
    }
    const void* dx_out_p = address(dx_out, "dx_out", {rows, C}, type, device);
    const void* dz_p = address(dz, "dz_k", {K, C}, type, device);
    const void* x_out_p = address(x_out, "x_out_k", {K, C}, type, device);
    const void* y_p = address(y, "y_k", {K, C}, type, device);
    const int32_t* idx_p = address<const int32_t>(idx, "idx", {K}, at::kInt, device);
    const int32_t* inv_p = address<const int32_t>(inv, "inv", {M}, at::kInt, device);
    PyObject* given[7] = {a[17], a[18], Py_None, Py_None, Py_None, Py_None, Py_None};
    Held held;
    if (a[19] != Py_None) {
      if (!PyDict_Check(a[19])) fail(PyExc_TypeError, "%s", "grads must be a dict");
      for (int q = 2; q < 7; ++q) {
        PyObject* g = PyDict_GetItemString(a[19], kOutputs[q]);
        if (!g) continue;
        Py_INCREF(g);
        given[q] = held.o[q] = g;
      }
    }
    at::Tensor made[7];
    void* p[7] = {};
    for (int q = 0; q < 7; ++q) {
      if (!(want >> q & 1)) continue;
      if (q >= 2 && given[q] == Py_None && (flags & SBP_FLAG_ACCUMULATE_DW)) fail(PyExc_ValueError, "%s has to be given in grads to be accumulated into", kOutputs[q]);
      const at::Tensor* gate = tensor(a[6], "gate");
      const std::vector<int64_t> shape = q == 0 ? std::vector<int64_t>{rows, C} : q == 1 ? std::vector<int64_t>{K, C}
                                         : q == 2 && gate ? gate->sizes().vec() : std::vector<int64_t>{C};
      const at::ScalarType t = q < 2 ? type : at::kFloat;
      p[q] = address(or_new(tensor(given[q], kOutputs[q]), made[q], shape, t, device), kOutputs[q], shape, t, device);
    }
    const sbp_residual_norm_grads g{(float*)p[2], (float*)p[3], (float*)p[4], (float*)p[5], (float*)p[6]};
    const Workspace ws(a[20], f_norm_bwd_ws(&d, K, code, flags), device);
    run(device, [&](void* s) { return f_norm_bwd(&d, dx_out_p, dz_p, x_out_p, y_p, idx_p, inv_p, K, code, p[0], p[1], &g, ws.p, ws.bytes, flags, s); });
    PyObject* out = PyDict_New();
    for (int q = 0; out && q < 7; ++q) {
      if (!(want >> q & 1)) continue;
      PyObject* o = keep_or_wrap(given[q], made[q]);
      if (!o || PyDict_SetItemString(out, kOutputs[q], o) < 0) { Py_XDECREF(o); Py_DECREF(out); return nullptr; }
      Py_DECREF(o);
    }
    return out;
  } catch (const PyFail&) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

const void* token_address(const at::Tensor& t, c10::Device device, int32_t* bytes) {
  if (t.scalar_type() != at::kInt && t.scalar_type() != at::kLong) fail(PyExc_TypeError, "tokens must be int32 or int64, got %s", c10::toString(t.scalar_type()));
  *bytes = t.scalar_type() == at::kInt ? 4 : 8;
  return address(&t, "tokens", t.sizes(), t.scalar_type(), device);
}

// (tokens, table, scale, out) -> E
PyObject* embedding_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    count(n, 4);
    const at::Tensor &tokens = needed(a[0], "tokens"), &table = matrix(a[1], "table");
    const int32_t code = dtype_code(table);
    const c10::Device device = table.device();
    const int64_t V = table.size(0);
    const int32_t C = channels(table.size(1));
    int32_t bytes;
    const void* tp = token_address(tokens, device, &bytes);
    const void* p = address(&table, "table", {V, C}, table.scalar_type(), device);
    std::vector<int64_t> shape = tokens.sizes().vec();
    shape.push_back(C);
    at::Tensor made;
    void* out = address(or_new(tensor(a[3], "out"), made, shape, table.scalar_type(), device), "out", shape, table.scalar_type(), device);
    const float scale = number(a[2]);
    const int64_t M = tokens.numel();
    run(device, [&](void* s) { return f_emb(tp, bytes, p, M, V, C, scale, code, out, s); });
    return keep_or_wrap(a[3], made);
  } catch (const PyFail&) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// (dE, tokens, V, idx, scale, flags, dtable, workspace) -> dtable
PyObject* embedding_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    count(n, 8);
    const at::Tensor &dE = matrix(a[0], "dE"), &tokens = needed(a[1], "tokens");
    const at::Tensor* idx = tensor(a[3], "idx");
    const int32_t code = dtype_code(dE);
    const c10::Device device = dE.device();
    const int64_t V = integer(a[2], true), M = tokens.numel(), K = idx ? idx->numel() : M;
    const int32_t C = channels(dE.size(1));
    const uint32_t flags = flags32(a[5]);
    if (V < 0) fail(PyExc_ValueError, "%s", "V must not be negative");
    int32_t bytes;
    const void* tp = token_address(tokens, device, &bytes);
    const void* p = address(&dE, "dE", {flags & SBP_FLAG_DY_COMPACT ? K : M, C}, dE.scalar_type(), device);
    const int32_t* ip = address<const int32_t>(idx, "idx", {K}, at::kInt, device);
    const at::ScalarType type = flags & SBP_FLAG_DW_OUT_BF16 ? at::kBFloat16 : at::kFloat;
    const at::Tensor* given = tensor(a[6], "dtable");
    if (!given && (flags & SBP_FLAG_ACCUMULATE_DW)) fail(PyExc_ValueError, "%s", "dtable has to be given to be accumulated into");
    at::Tensor made;
    void* out = address(or_new(given, made, {V, C}, type, device), "dtable", {V, C}, type, device);
    const float scale = number(a[4]);
    const Workspace ws(a[7], f_emb_bwd_ws(M, K, V, C, code, flags), device);
    run(device, [&](void* s) { return f_emb_bwd(p, tp, bytes, ip, M, K, V, C, scale, code, out, ws.p, ws.bytes, flags, s); });
    return keep_or_wrap(a[6], made);
  } catch (const PyFail&) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

template <class F>
PyCFunction method(F* f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)); }

PyMethodDef methods[] = {{"bind", method(bind), METH_FASTCALL, nullptr},
                         {"attention_forward", method(attention_forward), METH_FASTCALL, nullptr},
                         {"attention_backward", method(attention_backward), METH_FASTCALL, nullptr},
                         {"norm_forward", method(norm_forward), METH_FASTCALL, nullptr},
                         {"norm_backward", method(norm_backward), METH_FASTCALL, nullptr},
                         {"embedding_forward", method(embedding_forward), METH_FASTCALL, nullptr},
                         {"embedding_backward", method(embedding_backward), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native_lm", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native_lm(void) { return PyModule_Create(&module); }
