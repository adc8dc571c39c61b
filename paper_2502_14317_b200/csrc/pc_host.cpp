// Host side of hot_path() in binding.py as one call: output and workspace tensors, descriptor, launches; and of the calls on 8-bit
// caches and of cache_attn, whose kernels take a few us where ctypes and the checks took 10 to 15 in Python.
//
// What bounds a short prompt through the whole path is the time between its launches: of 54 us a pass over four chunks of 256 tokens
// that keeps nothing between calls, thirteen new tensors made one by one in Python took 26 and the arguments some 6 more,
// beside 22 for the six launches and their tensor maps; the kernels need 36.  Here a new tensor takes a third of that.
//
// The library's entry points come as addresses with each call: this module holds no state.
#include <Python.h>
#include <ATen/ATen.h>
#include <climits>
#include <string>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <pybind11/pybind11.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/pc.h"

namespace {

// outputs and workspaces, in the order of binding.py's _HOT_PATH_BUFFERS
enum { O, K_ROT, WIN_SCORE, WIN_LSE, SCORE, KEPT, IDX, KC, VC, POS, FG, STATUS, WS_PREFILL, WS_PAR, N_BUFFERS };
// result codes beside the library's own; with BAD_BUFFER the stage is the buffer's place
enum { NOT_INNERMOST = 1, NOT_CONTIGUOUS = 2, BAD_INPUT = 3, BAD_BUFFER = 4 };

using ws_bytes_fn = size_t (*)(const pc_prefill_desc*, int32_t, int32_t, size_t*);
using hot_path_fn = int32_t (*)(const pc_prefill_desc*, const pc_hot_path_args*, int32_t*, void*);

struct Call {
  ws_bytes_fn ws_bytes;
  hot_path_fn run;
  at::Tensor q, k, v, given, t[N_BUFFERS];
  bool has_given, made[N_BUFFERS] = {};
  int64_t C, L, Hq, Hkv, d, w, m, k_keep;
  double theta, scale;
  void* stream;
  int32_t rc, stage = 0;

  // Whether buffer i can be written as contiguous elements of that type (any type for a workspace, whose bytes are counted).
  bool writable(int i, at::ScalarType type) {
    if (t[i].scalar_type() == type && t[i].device() == q.device() && t[i].is_contiguous()) return true;
    rc = BAD_BUFFER; stage = i;
    return false;
  }
  // Buffer i is about to be dropped.  Its memory belongs to the stream it was made on; the calls that used it may have been on the present
  // one, and it is not given out again before that has come here.
  void let_go(int i) {
    if (t[i].is_cuda()) t[i].record_stream(c10::impl::VirtualGuardImpl(t[i].device().type()).getStream(t[i].device()));
  }
  // Buffer i of these sizes.  One that is there may be of an earlier call with other sizes: it serves as it is, or through a view of its
  // first elements where it has enough, and is replaced where it has not.  False: one that cannot be written.
  bool make(int i, at::IntArrayRef sizes, at::ScalarType type) {
    if (t[i].defined()) {
      if (i == O && t[i].sizes().equals(sizes) && t[i].scalar_type() == type && t[i].device() == q.device()) return true;   // any strides
      if (!writable(i, type)) return false;
      if (t[i].sizes().equals(sizes)) return true;
      int64_t n = 1;
      for (int64_t s : sizes) n *= s;
      if (n >= 0 && t[i].numel() >= n) {
        t[i] = t[i].view(-1).narrow(0, 0, n).view(sizes);
        made[i] = true;
        return true;
      }
      let_go(i);
    }
    t[i] = at::empty(sizes, at::TensorOptions().dtype(type).device(q.device()));
    return made[i] = true;
  }
  void operator()();
};

void Call::operator()() {
  // The launches go by q's sizes alone: keys and values of others would be read out of range.
  for (const at::Tensor* x : {&q, &k, &v})
    if (x->scalar_type() != at::kBFloat16 || x->device() != q.device()) { rc = BAD_INPUT; return; }
  for (const at::Tensor* x : {&k, &v})                             // (chunks beyond the queries' are not looked at)
    if (x->dim() != 4 || x->size(0) < C || x->size(1) != L || x->size(2) != Hkv || x->size(3) != d) { rc = BAD_INPUT; return; }
  if (has_given && given.device() != q.device()) { rc = BAD_INPUT; return; }
  const int64_t mk = m * k_keep;
  if (has_given) t[SCORE] = given;
  if (!(make(O, q.sizes(), at::kBFloat16) && make(K_ROT, k.sizes(), at::kBFloat16) && make(WIN_SCORE, {C, Hkv, L}, at::kFloat) &&
        make(WIN_LSE, {C, Hq, w}, at::kFloat) && (has_given || make(SCORE, {C}, at::kFloat)) && make(KEPT, {m}, at::kInt) &&
        make(IDX, {m, Hkv, k_keep}, at::kInt) && make(KC, {Hkv, mk, d}, at::kBFloat16) && make(VC, {Hkv, mk, d}, at::kBFloat16) &&
        make(POS, {Hkv, mk}, at::kInt) && make(FG, {1, w, Hq, d}, at::kBFloat16)))
    return;
  const bool clear = !t[STATUS].defined() || t[STATUS].numel() < 1;
  if (!make(STATUS, {1}, at::kInt)) return;

  pc_prefill_desc desc;
  desc.C = (int32_t)C; desc.L = (int32_t)L; desc.w = (int32_t)w; desc.Hq = (int32_t)Hq; desc.Hkv = (int32_t)Hkv; desc.d = (int32_t)d;
  desc.rope_theta = (float)theta;
  desc.softmax_scale = (float)scale;
  const at::Tensor* const in[4] = {&q, &k, &v, &t[O]};
  int64_t* const strides[4] = {desc.q_stride, desc.k_stride, desc.v_stride, desc.o_stride};
  for (int i = 0; i < 4; ++i) {
    TORCH_CHECK_INDEX(in[i]->dim() == 4, "tuple index out of range");
    if (in[i]->stride(3) != 1) { rc = NOT_INNERMOST; return; }
    for (int j = 0; j < 3; ++j) strides[i][j] = in[i]->stride(j);
  }
  for (int i : {WS_PREFILL, WS_PAR})
    if (t[i].defined() && !writable(i, t[i].scalar_type())) return;
  size_t need_par = 0;
  const size_t need = ws_bytes(&desc, (int32_t)m, (int32_t)k_keep, &need_par);
  auto scratch = [&](size_t bytes) { return at::empty({(int64_t)std::max<size_t>(bytes, 16)}, at::TensorOptions().dtype(at::kByte).device(q.device())); };
  if (!t[WS_PREFILL].defined() || (size_t)t[WS_PREFILL].numel() < need) {      // 0: a bad argument, which the call below names
    if (t[WS_PREFILL].defined()) let_go(WS_PREFILL);
    t[WS_PREFILL] = scratch(std::max(need, need_par));
    made[WS_PREFILL] = true;
  }
  if (!t[WS_PAR].defined() || (size_t)t[WS_PAR].numel() < need_par) {          // (the prefill is done with its own by then)
    if (t[WS_PAR].defined()) let_go(WS_PAR);
    t[WS_PAR] = (size_t)t[WS_PREFILL].numel() >= need_par ? t[WS_PREFILL] : scratch(need_par);
    made[WS_PAR] = true;
  }
  if (!t[K_ROT].is_contiguous() || !v.is_contiguous()) { rc = NOT_CONTIGUOUS; return; }
  // the window is the same in every chunk: take it from chunk 0
  at::Tensor window;
  const char* q_win = static_cast<const char*>(q.data_ptr()) + (L - w) * Hq * d * 2;
  if (!q.is_contiguous()) {
    window = q.as_strided({1, w, Hq, d}, q.strides(), q.storage_offset() + (L - w) * q.stride(1)).contiguous();
    q_win = static_cast<const char*>(window.data_ptr());
  }
  pc_hot_path_args a;
  a.q = q.data_ptr(); a.k = k.data_ptr(); a.v = v.data_ptr(); a.q_win = q_win;
  a.o = t[O].data_ptr(); a.k_rot = t[K_ROT].data_ptr();
  a.win_score = static_cast<float*>(t[WIN_SCORE].data_ptr()); a.win_lse = static_cast<float*>(t[WIN_LSE].data_ptr());
  a.given_score = has_given ? static_cast<const float*>(given.data_ptr()) : nullptr;
  a.chunk_score = static_cast<float*>(t[SCORE].data_ptr());
  a.kept = static_cast<int32_t*>(t[KEPT].data_ptr()); a.idx = static_cast<int32_t*>(t[IDX].data_ptr());
  a.kc = t[KC].data_ptr(); a.vc = t[VC].data_ptr(); a.pos = static_cast<int32_t*>(t[POS].data_ptr()); a.fg = t[FG].data_ptr();
  a.status_word = static_cast<int32_t*>(t[STATUS].data_ptr());
  a.ws_prefill = t[WS_PREFILL].data_ptr(); a.ws_prefill_bytes = (size_t)t[WS_PREFILL].numel();
  a.ws_parallel = t[WS_PAR].data_ptr(); a.ws_parallel_bytes = (size_t)t[WS_PAR].numel();
  a.m = (int32_t)m; a.k_keep = (int32_t)k_keep; a.n_score = (int32_t)t[SCORE].numel(); a.clear_status = clear;
  rc = run(&desc, &a, &stage, stream);
}

// hot_path(ws_bytes, run, stream, q, k, v, chunk_score or None, buffers, (C, L, Hq, Hkv, d, w, m, k_keep), rope_theta, softmax_scale)
// -> (result code, stage, buffers): those given, or new ones in the place of None and of those that are too small
PyObject* hot_path(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  unsigned long long ws_bytes, run, stream;
  PyObject *in[3], *given, *buffers;
  Call c;
  if (!PyArg_ParseTuple(args, "KKKOOOOO!(LLLLLLLL)dd", &ws_bytes, &run, &stream, &in[0], &in[1], &in[2], &given, &PyTuple_Type, &buffers, &c.C,
                        &c.L, &c.Hq, &c.Hkv, &c.d, &c.w, &c.m, &c.k_keep, &c.theta, &c.scale))
    return nullptr;
  if (PyTuple_GET_SIZE(buffers) != N_BUFFERS) { PyErr_SetString(PyExc_TypeError, "hot_path: wrong number of buffers"); return nullptr; }
  c.ws_bytes = reinterpret_cast<ws_bytes_fn>(static_cast<uintptr_t>(ws_bytes));
  c.run = reinterpret_cast<hot_path_fn>(static_cast<uintptr_t>(run));
  c.stream = reinterpret_cast<void*>(static_cast<uintptr_t>(stream));
  auto tensor = [](PyObject* p, at::Tensor& t) {
    if (p == Py_None) return true;
    if (!THPVariable_Check(p)) { PyErr_SetString(PyExc_TypeError, "hot_path: expected a tensor"); return false; }
    t = THPVariable_Unpack(p);
    return true;
  };
  if (!tensor(in[0], c.q) || !tensor(in[1], c.k) || !tensor(in[2], c.v) || !tensor(given, c.given)) return nullptr;
  c.has_given = given != Py_None;
  for (int i = 0; i < N_BUFFERS; ++i)
    if (!tensor(PyTuple_GET_ITEM(buffers, i), c.t[i])) return nullptr;
  {
    pybind11::gil_scoped_release release;
    c();
  }
  PyObject* const out = PyTuple_New(N_BUFFERS);
  if (out == nullptr) return nullptr;
  PyObject* ws_prefill = nullptr;
  for (int i = 0; i < N_BUFFERS; ++i) {
    PyObject* p = PyTuple_GET_ITEM(buffers, i);
    if (i == SCORE && c.has_given) p = given;
    else if (i == WS_PAR && c.made[i] && c.t[i].is_same(c.t[WS_PREFILL])) p = ws_prefill;
    else if (c.made[i]) p = nullptr;
    if (p != nullptr) Py_INCREF(p);
    else p = c.t[i].defined() ? THPVariable_Wrap(c.t[i]) : (Py_INCREF(Py_None), Py_None);
    if (p == nullptr) { Py_DECREF(out); return nullptr; }
    if (i == WS_PREFILL) ws_prefill = p;
    PyTuple_SET_ITEM(out, i, p);
  }
  return Py_BuildValue("iiN", (int)c.rc, (int)c.stage, out);
  END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------------------------ 8-bit caches, attention over shared and own caches
// An argument that does not fit: its text goes to binding.py, which raises it as a PcError.
struct Refused { const char* why; };
void need(bool ok, const char* why) { if (!ok) throw Refused{why}; }

bool is_tensor(PyObject* p, at::Tensor& t, const char* why) {       // false: None
  if (p == nullptr || p == Py_None) return false;
  need(THPVariable_Check(p), why);
  t = THPVariable_Unpack(p);
  return true;
}

// a cache's dict -> descriptor; its tensors are held by the dict
struct Cache {
  pc_kv_cache c = {};
  at::Device device = at::kCPU;
  explicit Cache(PyObject* dict) {
    need(PyDict_Check(dict), "a cache is a dict with format, k, v, k_scale and v_scale");
    PyObject* const f = PyDict_GetItemString(dict, "format");
    const char* const name = f != nullptr && PyUnicode_Check(f) ? PyUnicode_AsUTF8(f) : nullptr;
    const std::string format = name ? name : "";
    at::ScalarType type = at::kBFloat16;
    if (format == "int8") { c.format = PC_KV_INT8; type = at::kChar; }
    else if (format == "e4m3") { c.format = PC_KV_E4M3; type = at::kFloat8_e4m3fn; }
    else { need(format == "bf16", "the format of a cache must be bf16, int8 or e4m3"); c.format = PC_KV_BF16; }
    const char* const bad = "k and v of a cache must be contiguous [B, Hkv, capacity, d] of its format, on one device";
    const char* const bad_scale = "k_scale and v_scale of a cache must be contiguous float32 [B, Hkv, capacity] on its device";
    at::Tensor k, v, s[2];
    need(is_tensor(PyDict_GetItemString(dict, "k"), k, bad) && is_tensor(PyDict_GetItemString(dict, "v"), v, bad), bad);
    need(k.dim() == 4 && k.sizes().equals(v.sizes()) && k.scalar_type() == type && v.scalar_type() == type && k.is_contiguous() &&
         v.is_contiguous() && k.device() == v.device(), bad);
    need(k.size(0) <= INT32_MAX && k.size(1) <= INT32_MAX && k.size(3) <= INT32_MAX, bad);
    device = k.device();
    c.B = (int32_t)k.size(0); c.Hkv = (int32_t)k.size(1); c.capacity = k.size(2); c.d = (int32_t)k.size(3);
    c.k = k.data_ptr(); c.v = v.data_ptr();
    if (c.format == PC_KV_BF16) return;
    for (int i = 0; i < 2; ++i) {
      need(is_tensor(PyDict_GetItemString(dict, i ? "v_scale" : "k_scale"), s[i], bad_scale), bad_scale);
      need(s[i].dim() == 3 && s[i].sizes().equals(k.sizes().slice(0, 3)) && s[i].scalar_type() == at::kFloat && s[i].is_contiguous() &&
           s[i].device() == device, bad_scale);
    }
    c.k_scale = static_cast<float*>(s[0].data_ptr()); c.v_scale = static_cast<float*>(s[1].data_ptr());
  }
};

// bf16 rows [B,n,H,d] with a contiguous head dimension -> strides
const void* rows_of(const at::Tensor& t, at::IntArrayRef sizes, at::Device device, int64_t (&stride)[3], const char* why) {
  need(t.dim() == 4 && t.sizes().equals(sizes) && t.scalar_type() == at::kBFloat16 && t.device() == device && t.stride(3) == 1, why);
  for (int i = 0; i < 3; ++i) stride[i] = t.size(i) > 1 ? t.stride(i) : sizes[3];     // (of one entry any stride will do)
  need(stride[0] != 0 || stride[1] != 0 || stride[2] != 0, why);                      // (three zeros would stand for contiguous rows)
  return t.data_ptr();
}
const int32_t* per_sequence(PyObject* p, int64_t B, at::Device device, const char* why) {
  at::Tensor t;
  if (!is_tensor(p, t, why)) return nullptr;
  need(t.dim() == 1 && t.size(0) == B && t.scalar_type() == at::kInt && t.is_contiguous() && t.device() == device, why);
  return static_cast<const int32_t*>(t.data_ptr());
}
// at: a number or an int32 tensor [B]
const int32_t* start_of(PyObject* at, int64_t B, at::Device device, int32_t& at0) {
  const char* const why = "at must be a number or a contiguous int32 tensor with one entry per sequence";
  at0 = 0;
  if (THPVariable_Check(at)) return per_sequence(at, B, device, why);
  const long long x = PyLong_AsLongLong(at);
  if (x == -1 && PyErr_Occurred()) { PyErr_Clear(); throw Refused{why}; }
  need(x >= INT32_MIN && x <= INT32_MAX, why);
  at0 = (int32_t)x;
  return nullptr;
}

template <class F>
F entry(unsigned long long address) { return reinterpret_cast<F>(static_cast<uintptr_t>(address)); }
template <class F>
PyObject* refusing(F f) {
  try { return f(); }
  catch (const Refused& r) { return Py_BuildValue("s", r.why); }
}

// kv_quantize(run, stream, need_cuda, cache, k, v, at, status or None) -> result code, or the reason of a refusal
PyObject* kv_quantize(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  unsigned long long run, stream;
  int cuda;
  PyObject *dict, *pk, *pv, *at, *status;
  if (!PyArg_ParseTuple(args, "KKpOOOOO", &run, &stream, &cuda, &dict, &pk, &pv, &at, &status)) return nullptr;
  return refusing([&]() {
    const char* const bad = "k and v must be bfloat16 [B, n, Hkv, d] with the B, Hkv and d of the cache and a contiguous head dimension, on its device";
    const Cache c(dict);
    at::Tensor k, v, st;
    need(is_tensor(pk, k, bad) && is_tensor(pv, v, bad) && k.dim() == 4 && k.size(1) <= INT32_MAX, bad);
    need(!cuda || k.is_cuda(), "tensors must live on a CUDA device");
    int64_t ks[3], vs[3];
    const int64_t sizes[4] = {c.c.B, k.size(1), c.c.Hkv, c.c.d};
    const void* const kp = rows_of(k, sizes, c.device, ks, bad);
    const void* const vp = rows_of(v, sizes, c.device, vs, bad);
    int32_t at0;
    const int32_t* const each = start_of(at, c.c.B, c.device, at0);
    const char* const bad_status = "status must be an int32 tensor on the cache's device";
    const bool has = is_tensor(status, st, bad_status);
    need(!has || (st.scalar_type() == at::kInt && st.numel() >= 1 && st.device() == c.device), bad_status);
    using fn = int32_t (*)(const pc_kv_cache*, const void*, const int64_t*, const void*, const int64_t*, int32_t, int32_t, const int32_t*, int32_t*, void*);
    return PyLong_FromLong(entry<fn>(run)(&c.c, kp, ks, vp, vs, (int32_t)k.size(1), at0, each,
                                          has ? static_cast<int32_t*>(st.data_ptr()) : nullptr, entry<void*>(stream)));
  });
  END_HANDLE_TH_ERRORS
}

// gather_kv_quantize(run, stream, need_cuda, k_src, v_src, kept, idx, cache, pos_out or None, want_pos) -> (result code, pos or None), or the
// reason of a refusal
PyObject* gather_kv_quantize(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  unsigned long long run, stream;
  int cuda, want_pos;
  PyObject *src[2], *which[2], *dict, *pos_out;
  if (!PyArg_ParseTuple(args, "KKpOOOOOOp", &run, &stream, &cuda, &src[0], &src[1], &which[0], &which[1], &dict, &pos_out, &want_pos)) return nullptr;
  return refusing([&]() -> PyObject* {
    const char* const bad = "k_src and v_src must be bfloat16 [C, L, Hkv, d] and share strides with a contiguous head dimension, on one device";
    const char* const bad_idx = "idx must be contiguous int32 [m, Hkv, k], kept contiguous int32 [m], on the device of k_src";
    at::Tensor k, v, kept, idx, pos;
    need(is_tensor(src[0], k, bad) && is_tensor(src[1], v, bad) && k.dim() == 4 && k.sizes().equals(v.sizes()) && k.strides().equals(v.strides()) &&
         k.stride(3) == 1 && k.scalar_type() == at::kBFloat16 && v.scalar_type() == at::kBFloat16 && k.device() == v.device(), bad);
    need(!cuda || k.is_cuda(), "tensors must live on a CUDA device");
    need(is_tensor(which[0], kept, bad_idx) && is_tensor(which[1], idx, bad_idx) && idx.dim() == 3 && kept.dim() == 1 && kept.size(0) == idx.size(0) &&
         idx.size(1) == k.size(2) && idx.size(0) <= INT32_MAX && idx.size(2) <= INT32_MAX, bad_idx);
    for (const at::Tensor* t : {&kept, &idx}) need(t->scalar_type() == at::kInt && t->is_contiguous() && t->device() == k.device(), bad_idx);
    const int64_t m = idx.size(0), Hkv = idx.size(1), n = idx.size(2);
    const Cache c(dict);
    need(c.c.format != PC_KV_BF16 && c.c.B == 1 && c.c.Hkv == Hkv && c.c.capacity >= m * n && c.c.d == k.size(3) && c.device == k.device(),
         "the cache must be an 8-bit one that holds m * k entries of one sequence, with the Hkv and d of k_src, on its device");
    const char* const bad_pos = "pos_out must be contiguous int32 [Hkv, m*k] on the device of k_src";
    const int64_t sizes[2] = {Hkv, m * n};
    const bool given = is_tensor(pos_out, pos, bad_pos);
    if (given)
      need(pos.sizes().equals(sizes) && pos.scalar_type() == at::kInt && pos.is_contiguous() && pos.device() == k.device(), bad_pos);
    else if (want_pos)
      pos = at::empty(sizes, at::TensorOptions().dtype(at::kInt).device(k.device()));
    const int64_t stride[3] = {k.stride(0), k.stride(1), k.stride(2)};
    using fn = int32_t (*)(const void*, const void*, const int64_t*, const int32_t*, const int32_t*, int32_t, int32_t, const pc_kv_cache*, int32_t*, void*);
    const int32_t rc = entry<fn>(run)(k.data_ptr(), v.data_ptr(), stride, static_cast<const int32_t*>(kept.data_ptr()),
                                      static_cast<const int32_t*>(idx.data_ptr()), (int32_t)m, (int32_t)n, &c.c,
                                      pos.defined() ? static_cast<int32_t*>(pos.data_ptr()) : nullptr, entry<void*>(stream));
    PyObject* const x = given ? (Py_INCREF(pos_out), pos_out) : pos.defined() ? THPVariable_Wrap(pos) : (Py_INCREF(Py_None), Py_None);
    return Py_BuildValue("iN", (int)rc, x);
  });
  END_HANDLE_TH_ERRORS
}

// kv_dequantize(run, stream, need_cuda, cache, n or None, at, k_out or None, v_out or None) -> (result code, k, v), or the reason of a refusal
PyObject* kv_dequantize(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  unsigned long long run, stream;
  int cuda;
  PyObject *dict, *pn, *at, *out[2];
  if (!PyArg_ParseTuple(args, "KKpOOOOO", &run, &stream, &cuda, &dict, &pn, &at, &out[0], &out[1])) return nullptr;
  return refusing([&]() -> PyObject* {
    const Cache c(dict);
    need(!cuda || c.device.is_cuda(), "tensors must live on a CUDA device");
    long long n = c.c.capacity;
    if (pn != Py_None) n = PyLong_AsLongLong(pn);
    if (n == -1 && PyErr_Occurred()) return nullptr;
    need(n >= 1 && n <= INT32_MAX, "n must be at least 1");
    int32_t at0;
    const int32_t* const each = start_of(at, c.c.B, c.device, at0);
    at::Tensor t[2];
    const int64_t sizes[4] = {c.c.B, c.c.Hkv, n, c.c.d};
    for (int i = 0; i < 2; ++i) {
      const char* const bad = "k_out and v_out must be contiguous bfloat16 [B, Hkv, n, d] on the cache's device";
      if (is_tensor(out[i], t[i], bad))
        need(t[i].dim() == 4 && t[i].sizes().equals(sizes) && t[i].scalar_type() == at::kBFloat16 && t[i].is_contiguous() && t[i].device() == c.device, bad);
      else
        t[i] = at::empty(sizes, at::TensorOptions().dtype(at::kBFloat16).device(c.device));
    }
    using fn = int32_t (*)(const pc_kv_cache*, int32_t, int32_t, const int32_t*, void*, void*, void*);
    const int32_t rc = entry<fn>(run)(&c.c, (int32_t)n, at0, each, t[0].data_ptr(), t[1].data_ptr(), entry<void*>(stream));
    return Py_BuildValue("iNN", (int)rc, THPVariable_Wrap(t[0]), THPVariable_Wrap(t[1]));
  });
  END_HANDLE_TH_ERRORS
}

// Outputs and workspace of an attention call (out, lse, status, workspace): given, kept from an earlier call (through a view where that had other
// sizes), or new.
struct AttnOut {
  static constexpr const char* names[4] = {"out", "lse", "status", "workspace"};
  static constexpr at::ScalarType types[4] = {at::kBFloat16, at::kFloat, at::kInt, at::kByte};
  at::Device device;
  PyObject *const *given, *buffers;
  const bool keeps;
  at::Tensor t[4];
  PyObject* same[4] = {};                                            // objects that are returned as they came
  bool serves[4] = {};                                               // what is kept stays, though this call may have a view of its first elements alone
  int32_t clear_status = 0;

  void fits(int i, const char* why) const { need(t[i].scalar_type() == types[i] && t[i].device() == device && t[i].is_contiguous(), why); }
  PyObject* kept(int i) const { return keeps ? PyDict_GetItemString(buffers, names[i]) : nullptr; }
  static void let_go(at::Tensor& x) {
    if (x.is_cuda()) x.record_stream(c10::impl::VirtualGuardImpl(x.device().type()).getStream(x.device()));
  }
  AttnOut(at::Device dev, PyObject* const (&g)[4], PyObject* b, bool want_lse, int64_t B, int64_t w, int64_t Hq, int64_t d)
      : device(dev), given(g), buffers(b), keeps(b != Py_None) {
    need(!keeps || PyDict_Check(buffers), "buffers must be a dict");
    const int64_t s_out[4] = {B, w, Hq, d}, s_lse[3] = {B, Hq, w}, s_one[1] = {1};
    const at::IntArrayRef sizes[3] = {s_out, s_lse, s_one};
    for (int i = 0; i < 3; ++i) {
      if (i == 1 && !want_lse && given[1] == Py_None) continue;
      if (is_tensor(given[i], t[i], "out, lse_out and status must be tensors")) {
        static const char* const bad[3] = {"out must be contiguous bfloat16 [B, w, Hq, d]", "lse_out must be contiguous float32 [B, Hq, w]",
                                           "status must be a contiguous int32 tensor"};
        fits(i, bad[i]);
        need(i == 2 ? t[i].numel() >= 1 : t[i].sizes().equals(sizes[i]), bad[i]);
        same[i] = given[i];
        continue;
      }
      PyObject* const p = kept(i);
      if (is_tensor(p, t[i], "buffers must hold tensors")) {
        fits(i, "a kept buffer is of another type or device, or not contiguous");
        if (t[i].sizes().equals(sizes[i])) { same[i] = p; continue; }
        int64_t count = 1;
        for (int64_t x : sizes[i]) count *= x;
        if (t[i].numel() >= count) { t[i] = t[i].view(-1).narrow(0, 0, count).view(sizes[i]); serves[i] = true; continue; }
        let_go(t[i]);
      }
      t[i] = at::empty(sizes[i], at::TensorOptions().dtype(types[i]).device(device));
      if (i == 2) clear_status = 1;
    }
  }
  void workspace(size_t bytes) {                                     // 0: a bad argument, which the call names
    PyObject* const p = given[3] != Py_None ? given[3] : kept(3);
    const bool has = is_tensor(p, t[3], "workspace must be a tensor");
    if (has) fits(3, "workspace must be a contiguous uint8 tensor on the queries' device");
    if (has && (size_t)t[3].numel() >= bytes) {
      same[3] = p;
    } else {
      if (has) let_go(t[3]);
      t[3] = at::empty({(int64_t)std::max<size_t>(bytes, 16)}, at::TensorOptions().dtype(at::kByte).device(device));
    }
  }
  template <class A>
  void put(A& a) const {
    a.out = t[0].data_ptr();
    a.lse = t[1].defined() ? static_cast<float*>(t[1].data_ptr()) : nullptr;
    a.status_word = static_cast<int32_t*>(t[2].data_ptr());
    a.workspace = t[3].data_ptr();
    a.workspace_bytes = (size_t)t[3].numel();
  }
  PyObject* result(int32_t rc) const {                               // (result code, dict of out, lse, status, workspace)
    PyObject* const r = PyDict_New();
    if (r == nullptr) return nullptr;
    for (int i = 0; i < 4; ++i) {
      PyObject* const x = same[i] ? (Py_INCREF(same[i]), same[i]) : t[i].defined() ? THPVariable_Wrap(t[i]) : (Py_INCREF(Py_None), Py_None);
      const bool ok = x != nullptr && PyDict_SetItemString(r, names[i], x) == 0 &&
                      (rc != PC_OK || !keeps || !t[i].defined() || serves[i] || PyDict_SetItemString(buffers, names[i], x) == 0);
      Py_XDECREF(x);
      if (!ok) { Py_DECREF(r); return nullptr; }
    }
    return Py_BuildValue("iN", (int)rc, r);
  }
};

// cache_attn(ws_bytes, run, stream, need_cuda, q, k_win, v_win, prefix, own, own_len, q_pos, (out, lse, status, workspace), buffers,
//            n_prefix, n_own, q_pos0, want_lse, rope_theta, softmax_scale)
// -> (result code, dict of out, lse, status, workspace), or the reason of a refusal.  Every object may be None but q; n = ALL: the capacity.
constexpr long long ALL = LLONG_MIN;
PyObject* cache_attn(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  unsigned long long ws_bytes, run, stream;
  int cuda, want_lse;
  long long n[2], q_pos0;
  double theta, scale;
  PyObject *pq, *pk, *pv, *dict[2], *own_len, *q_pos, *given[4], *buffers;
  if (!PyArg_ParseTuple(args, "KKKpOOOOOOO(OOOO)OLLLpdd", &ws_bytes, &run, &stream, &cuda, &pq, &pk, &pv, &dict[0], &dict[1], &own_len, &q_pos,
                        &given[0], &given[1], &given[2], &given[3], &buffers, &n[0], &n[1], &q_pos0, &want_lse, &theta, &scale))
    return nullptr;
  return refusing([&]() -> PyObject* {
    const char* const bad_q = "q must be bfloat16 [B, w, Hq, d] with a contiguous head dimension";
    at::Tensor q, kw, vw;
    need(is_tensor(pq, q, bad_q) && q.dim() == 4, bad_q);
    need(!cuda || q.is_cuda(), "tensors must live on a CUDA device");
    const at::Device device = q.device();
    const int64_t B = q.size(0), w = q.size(1), Hq = q.size(2), d = q.size(3);
    need(B <= INT32_MAX && w <= INT32_MAX && Hq <= INT32_MAX && d <= INT32_MAX && q_pos0 >= INT32_MIN && q_pos0 <= INT32_MAX, bad_q);
    pc_cache_attn_args a = {};
    a.B = (int32_t)B; a.w = (int32_t)w; a.Hq = (int32_t)Hq; a.d = (int32_t)d; a.q_pos0 = (int32_t)q_pos0;
    a.rope_theta = (float)theta; a.softmax_scale = (float)scale;
    a.q = rows_of(q, q.sizes(), device, a.q_stride, bad_q);
    pc_kv_cache c[2];
    for (int i = 0; i < 2; ++i) {
      if (dict[i] == Py_None) { need(n[i] == 0 || n[i] == ALL, i ? "n_own without a cache" : "n_prefix without a cache"); continue; }
      const Cache cache(dict[i]);
      need(cache.device == device, "the caches and the queries must be on one device");
      c[i] = cache.c;
      (i ? a.own : a.prefix) = &c[i];
      const long long entries = n[i] == ALL ? c[i].capacity : n[i];
      need(entries >= 0 && entries <= c[i].capacity, i ? "n_own is negative or more than the cache holds" : "n_prefix is negative or more than the cache holds");
      need(entries <= INT32_MAX, "a cache of more entries than can be counted");
      (i ? a.n_own : a.n_prefix) = (int32_t)entries;
      a.Hkv = c[i].Hkv;
    }
    const char* const bad_win = "k_win and v_win must be bfloat16 [B, w, Hkv, d] with a contiguous head dimension, on the queries' device";
    const bool has_k = is_tensor(pk, kw, bad_win), has_v = is_tensor(pv, vw, bad_win);
    need(has_k == has_v, "k_win and v_win go together");
    if (has_k) {
      need(kw.dim() == 4, bad_win);
      if (a.Hkv == 0) a.Hkv = (int32_t)kw.size(2);
      const int64_t sizes[4] = {B, w, a.Hkv, d};
      a.k_win = rows_of(kw, sizes, device, a.k_win_stride, bad_win);
      a.v_win = rows_of(vw, sizes, device, a.v_win_stride, bad_win);
    }
    a.q_pos = per_sequence(q_pos, B, device, "q_pos must be a contiguous int32 tensor with one entry per sequence");
    a.own_len = per_sequence(own_len, B, device, "own_len must be a contiguous int32 tensor with one entry per sequence");
    AttnOut o(device, given, buffers, want_lse != 0, B, w, Hq, d);
    a.clear_status = o.clear_status;
    o.workspace(entry<size_t (*)(const pc_cache_attn_args*)>(ws_bytes)(&a));
    o.put(a);
    return o.result(entry<int32_t (*)(const pc_cache_attn_args*, void*)>(run)(&a, entry<void*>(stream)));
  });
  END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------------------------ paged caches, drafted tokens, log probabilities
// The launches go to the current device's stream.
void need_current(at::Device device) {
  need(device.is_cuda(), "tensors must live on a CUDA device");
  need(c10::impl::VirtualGuardImpl(device.type()).getDevice() == device, "tensors must live on the current CUDA device");
}
// int32 [B,n] with a contiguous last dimension -> address and stride; null: None
const int32_t* table_of(PyObject* p, int64_t B, int64_t n, at::Device device, int64_t& stride, const char* why) {
  at::Tensor t;
  stride = 0;
  if (!is_tensor(p, t, why)) return nullptr;
  need(t.dim() == 2 && t.size(0) == B && (n < 0 || t.size(1) == n) && t.size(1) >= 1 && t.size(1) <= INT32_MAX && t.scalar_type() == at::kInt &&
       t.device() == device && (t.stride(1) == 1 || t.size(1) == 1), why);
  stride = B > 1 ? t.stride(0) : 0;
  return static_cast<const int32_t*>(t.data_ptr());
}

// drafted tokens' parents: int32 [B,n], or [n] for all sequences (stride 0); null: None
const int32_t* parents_of(PyObject* p, int64_t B, int64_t n, at::Device device, int64_t& stride, const char* why) {
  at::Tensor t;
  stride = 0;
  if (!is_tensor(p, t, why) || t.dim() != 1) return table_of(p, B, n, device, stride, why);
  need(t.size(0) == n && t.scalar_type() == at::kInt && t.device() == device && (t.stride(0) == 1 || n == 1), why);
  return static_cast<const int32_t*>(t.data_ptr());
}

// page_append(run, stream, need_cuda, cache, k, v, table, at, pos, count, pick, parents, status, pos0, rope_theta) -> result code, or the reason of a refusal
PyObject* page_append(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  unsigned long long run, stream;
  int cuda;
  long long pos0;
  double theta;
  PyObject *dict, *pk, *pv, *table, *at, *pos, *count, *pick, *parents, *status;
  if (!PyArg_ParseTuple(args, "KKpOOOOOOOOOOLd", &run, &stream, &cuda, &dict, &pk, &pv, &table, &at, &pos, &count, &pick, &parents, &status, &pos0, &theta))
    return nullptr;
  return refusing([&]() {
    const char* const bad = "k and v must be bfloat16 [B, n, Hkv, d] with the Hkv and d of the pages and a contiguous head dimension, on their device";
    const Cache c(dict);
    if (cuda) need_current(c.device);
    at::Tensor k, v, st, t;
    need(is_tensor(pk, k, bad) && is_tensor(pv, v, bad) && k.dim() == 4 && k.size(0) >= 1 && k.size(0) <= INT32_MAX && k.size(1) <= INT32_MAX, bad);
    const int64_t B = k.size(0), sizes[4] = {B, k.size(1), c.c.Hkv, c.c.d};
    pc_page_append_args a = {};
    a.k = rows_of(k, sizes, c.device, a.k_stride, bad);
    a.v = rows_of(v, sizes, c.device, a.v_stride, bad);
    a.pages = &c.c;
    a.B = (int32_t)B;
    a.n = a.n_src = (int32_t)k.size(1);
    const char* const bad_table = "table must be int32 [B, pages of a sequence] with a contiguous last dimension, on the pages' device";
    need(is_tensor(table, t, bad_table) && t.dim() == 2, bad_table);
    a.table = table_of(table, B, -1, c.device, a.table_stride, bad_table);
    a.n_table = (int32_t)t.size(1);
    const char* const bad_pick = "pick must be int32 [B, tokens to be written] with a contiguous last dimension, on the pages' device";
    if (is_tensor(pick, t, bad_pick)) {
      need(t.dim() == 2, bad_pick);
      a.n = (int32_t)t.size(1);
      a.pick = table_of(pick, B, -1, c.device, a.pick_stride, bad_pick);
    }
    a.parents = parents_of(parents, B, a.n, c.device, a.parents_stride, "parents must be int32 [B, n] or [n] with a contiguous last dimension, on the pages' device");
    need(a.parents == nullptr || a.pick == nullptr, "pick and parents do not go together");
    a.at = start_of(at, B, c.device, a.at0);
    a.pos = per_sequence(pos, B, c.device, "pos must be a contiguous int32 tensor with one entry per sequence");
    a.count = per_sequence(count, B, c.device, "count must be a contiguous int32 tensor with one entry per sequence");
    const char* const bad_status = "status must be an int32 tensor on the pages' device";
    const bool has = is_tensor(status, st, bad_status);
    need(!has || (st.scalar_type() == at::kInt && st.numel() >= 1 && st.device() == c.device), bad_status);
    a.status_word = has ? static_cast<int32_t*>(st.data_ptr()) : nullptr;
    need(pos0 >= INT32_MIN && pos0 <= INT32_MAX, "pos0 must be a number of 32 bits");
    a.pos0 = (int32_t)pos0;
    a.rope_theta = (float)theta;
    return PyLong_FromLong(entry<int32_t (*)(const pc_page_append_args*, void*)>(run)(&a, entry<void*>(stream)));
  });
  END_HANDLE_TH_ERRORS
}

// tree_attn(ws_bytes, run, stream, need_cuda, q, cache, table, lens, pos, parents, (out, lse, status, workspace), buffers, max_len, pos0, want_lse, rope_theta,
//           softmax_scale) -> (result code, dict of out, lse, status, workspace), or the reason of a refusal.  max_len = ALL: as many as the table holds.
PyObject* tree_attn(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  unsigned long long ws_bytes, run, stream;
  int cuda, want_lse;
  long long max_len, pos0;
  double theta, scale;
  PyObject *pq, *dict, *table, *lens, *pos, *parents, *given[4], *buffers;
  if (!PyArg_ParseTuple(args, "KKKpOOOOOO(OOOO)OLLpdd", &ws_bytes, &run, &stream, &cuda, &pq, &dict, &table, &lens, &pos, &parents, &given[0], &given[1],
                        &given[2], &given[3], &buffers, &max_len, &pos0, &want_lse, &theta, &scale))
    return nullptr;
  return refusing([&]() -> PyObject* {
    const char* const bad_q = "q must be bfloat16 [B, w, Hq, d] with the d of the pages and a contiguous head dimension";
    const Cache c(dict);
    at::Tensor q, t;
    need(is_tensor(pq, q, bad_q) && q.dim() == 4 && q.size(3) == c.c.d, bad_q);
    if (cuda) need_current(q.device());
    need(c.device == q.device(), "the pages and the queries must be on one device");
    const int64_t B = q.size(0), w = q.size(1), Hq = q.size(2);
    need(B <= INT32_MAX && w <= INT32_MAX && Hq <= INT32_MAX, bad_q);
    pc_tree_attn_args a = {};
    a.B = (int32_t)B; a.w = (int32_t)w; a.Hq = (int32_t)Hq;
    a.q = rows_of(q, q.sizes(), c.device, a.q_stride, bad_q);
    a.pages = &c.c;
    const char* const bad_table = "table must be int32 [B, pages of a sequence] with a contiguous last dimension, on the queries' device";
    need(is_tensor(table, t, bad_table) && t.dim() == 2, bad_table);
    a.table = table_of(table, B, -1, c.device, a.table_stride, bad_table);
    a.n_table = (int32_t)t.size(1);
    const char* const bad_lens = "lens must be a contiguous int32 tensor with one entry per sequence";
    a.lens = per_sequence(lens, B, c.device, bad_lens);
    need(a.lens != nullptr, bad_lens);
    a.pos = per_sequence(pos, B, c.device, "pos must be a contiguous int32 tensor with one entry per sequence");
    a.parents = parents_of(parents, B, w, c.device, a.parents_stride, "parents must be int32 [B, w] or [w] with a contiguous last dimension, on the queries' device");
    const long long room = c.c.capacity * a.n_table - w;             // entries that a sequence can have before its new tokens
    need(room >= 0, "the table has no room for the new tokens");
    need(max_len == ALL || (max_len >= 0 && max_len <= room), "max_len is negative or more than the table holds beside the new tokens");
    const long long most = max_len == ALL ? room : max_len;
    need(most <= INT32_MAX, "a table of more entries than can be counted");
    need(pos0 >= INT32_MIN && pos0 <= INT32_MAX, "pos0 must be a number of 32 bits");
    a.max_len = (int32_t)most; a.pos0 = (int32_t)pos0;
    a.rope_theta = (float)theta; a.softmax_scale = (float)scale;
    AttnOut o(c.device, given, buffers, want_lse != 0, B, w, Hq, c.c.d);
    a.clear_status = o.clear_status;
    o.workspace(entry<size_t (*)(const pc_tree_attn_args*)>(ws_bytes)(&a));
    o.put(a);
    return o.result(entry<int32_t (*)(const pc_tree_attn_args*, void*)>(run)(&a, entry<void*>(stream)));
  });
  END_HANDLE_TH_ERRORS
}

// token_logprobs(run, stream, need_cuda, logits, tokens or None, top, group, want_entropy, scale) -> (result code, dict of logprob, entropy, top_id, top_logprob,
// nll), or the reason of a refusal
PyObject* token_logprobs(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  unsigned long long run, stream;
  int cuda, want_entropy;
  long long top, group;
  double scale;
  PyObject *pl, *pt;
  if (!PyArg_ParseTuple(args, "KKpOOLLpd", &run, &stream, &cuda, &pl, &pt, &top, &group, &want_entropy, &scale)) return nullptr;
  return refusing([&]() -> PyObject* {
    const char* const bad = "logits must be float32, bfloat16 or float16 [N, V] with a contiguous last dimension";
    at::Tensor x, t;
    need(is_tensor(pl, x, bad) && x.dim() == 2 && (x.stride(1) == 1 || x.size(1) == 1) && x.size(0) <= INT32_MAX && x.size(1) <= INT32_MAX, bad);
    if (cuda) need_current(x.device());
    pc_token_logprobs_args a = {};
    const int64_t N = x.size(0);
    if (x.scalar_type() == at::kFloat) a.type = PC_LOGITS_F32;
    else if (x.scalar_type() == at::kBFloat16) a.type = PC_LOGITS_BF16;
    else { need(x.scalar_type() == at::kHalf, bad); a.type = PC_LOGITS_F16; }
    a.N = (int32_t)N; a.V = (int32_t)x.size(1);
    a.stride = N > 1 ? x.stride(0) : 0;
    a.logits = x.data_ptr();
    a.tokens = per_sequence(pt, N, x.device(), "tokens must be a contiguous int32 tensor with one entry per row");
    need(top >= 0 && top <= PC_MOST_ALTERNATIVES && top <= x.size(1), "top must be between 0 and 32 and no more than the logits of a row");
    need(group >= 0 && (group == 0 || (a.tokens != nullptr && N % group == 0)), "group must divide the rows, and needs tokens");
    a.top = (int32_t)top; a.group = (int32_t)group; a.scale = (float)scale;
    at::Tensor o[5];
    const auto f32 = at::TensorOptions().dtype(at::kFloat).device(x.device());
    if (a.tokens) { o[0] = at::empty({N}, f32); a.logprob = static_cast<float*>(o[0].data_ptr()); }
    if (want_entropy) { o[1] = at::empty({N}, f32); a.entropy = static_cast<float*>(o[1].data_ptr()); }
    if (top) {
      o[2] = at::empty({N, (int64_t)top}, f32.dtype(at::kInt));
      o[3] = at::empty({N, (int64_t)top}, f32);
      a.top_id = static_cast<int32_t*>(o[2].data_ptr());
      a.top_logprob = static_cast<float*>(o[3].data_ptr());
    }
    if (group) { o[4] = at::empty({N / group}, f32); a.nll = static_cast<float*>(o[4].data_ptr()); }
    const int32_t rc = entry<int32_t (*)(const pc_token_logprobs_args*, void*)>(run)(&a, entry<void*>(stream));
    static const char* const names[5] = {"logprob", "entropy", "top_id", "top_logprob", "nll"};
    PyObject* const r = PyDict_New();
    if (r == nullptr) return nullptr;
    for (int i = 0; i < 5; ++i) {
      PyObject* const y = o[i].defined() ? THPVariable_Wrap(o[i]) : (Py_INCREF(Py_None), Py_None);
      const bool ok = y != nullptr && PyDict_SetItemString(r, names[i], y) == 0;
      Py_XDECREF(y);
      if (!ok) { Py_DECREF(r); return nullptr; }
    }
    return Py_BuildValue("iN", (int)rc, r);
  });
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"hot_path", hot_path, METH_VARARGS, "See binding.py."},
                         {"kv_quantize", kv_quantize, METH_VARARGS, "See binding.py."},
                         {"gather_kv_quantize", gather_kv_quantize, METH_VARARGS, "See binding.py."},
                         {"kv_dequantize", kv_dequantize, METH_VARARGS, "See binding.py."},
                         {"cache_attn", cache_attn, METH_VARARGS, "See binding.py."},
                         {"page_append", page_append, METH_VARARGS, "See binding.py."},
                         {"tree_attn", tree_attn, METH_VARARGS, "See binding.py."},
                         {"token_logprobs", token_logprobs, METH_VARARGS, "See binding.py."},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_pc_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pc_host() { return PyModule_Create(&module_def); }
