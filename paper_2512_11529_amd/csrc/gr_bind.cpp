// Argument marshalling of the Python binding for the calls of the decode loop: tensors are checked, the parameter structs of
// the C ABI are filled and the calls made here.  In Python (per-attribute checks, ctypes structs) this took 8 to 13 us a call, longer
// than the kernels of a small batch; here it is about one.  Host code only; the library is reached through the addresses that
// bind() is given, so whatever libgr.so the package has loaded is the one that runs.
#include <Python.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <optional>
#include <string>

#include "gr.h"

namespace {

decltype(&gr_beam_attn) p_attn = nullptr;
decltype(&gr_beam_attn_slots) p_attn_slots = nullptr;
decltype(&gr_beam_attn_fp8kv) p_attn_fp8kv = nullptr;
decltype(&gr_beam_attn_workspace_bytes) p_attn_ws = nullptr;
decltype(&gr_prefill_attn) p_prefill = nullptr;
decltype(&gr_beam_select) p_select = nullptr;
decltype(&gr_beam_select_noalloc) p_select_noalloc = nullptr;
decltype(&gr_beam_select_workspace_bytes) p_select_ws = nullptr;
decltype(&gr_beam_reorder) p_reorder = nullptr;
decltype(&gr_beam_slot_update) p_slot_update = nullptr;
decltype(&gr_page_map) p_page_map = nullptr;
decltype(&gr_page_write) p_page_write = nullptr;
decltype(&gr_beam_attn_paged) p_attn_paged = nullptr;
decltype(&gr_beam_attn_paged_workspace_bytes) p_attn_paged_ws = nullptr;
decltype(&gr_logits_adjust) p_adjust = nullptr;

struct Error {};        // a Python exception is set

std::string shape_text(c10::IntArrayRef s) {
  std::string t = "(";
  for (size_t i = 0; i < s.size(); i++) t += (i ? ", " : "") + std::to_string(s[i]);
  return t + (s.size() == 1 ? ",)" : ")");
}
const char* dtype_text(at::ScalarType t) {
  return t == at::kBFloat16 ? "torch.bfloat16" : t == at::kFloat ? "torch.float32" : t == at::kInt ? "torch.int32" : t == at::kByte ? "torch.uint8" : "another type";
}

// A contiguous GPU tensor of the type; of so many dimensions, or of the shape.
const at::Tensor& tensor_nd(PyObject* o, at::ScalarType dt, const char* name, int dims) {
  const at::Tensor* t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
  if (!t || !t->is_cuda() || !t->is_contiguous()) {
    PyErr_Format(PyExc_TypeError, "%s: expected a contiguous CUDA tensor", name);
    throw Error();
  }
  if (t->scalar_type() != dt) {
    PyErr_Format(PyExc_TypeError, "%s: expected %s, got %s", name, dtype_text(dt), dtype_text(t->scalar_type()));
    throw Error();
  }
  if (t->dim() != dims) {
    PyErr_Format(PyExc_ValueError, "%s: expected %d dimensions, got shape %s", name, dims, shape_text(t->sizes()).c_str());
    throw Error();
  }
  return *t;
}
const at::Tensor& tensor(PyObject* o, at::ScalarType dt, const char* name, c10::IntArrayRef shape) {
  const at::Tensor* t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
  if (t && t->is_cuda() && t->is_contiguous() && t->scalar_type() == dt && t->sizes() != shape) {
    PyErr_Format(PyExc_ValueError, "%s: expected shape %s, got %s", name, shape_text(shape).c_str(), shape_text(t->sizes()).c_str());
    throw Error();
  }
  return tensor_nd(o, dt, name, (int)shape.size());
}
const void* any_tensor(PyObject* o, size_t* bytes) {        // None or a tensor of any kind
  if (o == Py_None) { *bytes = 0; return nullptr; }
  if (!THPVariable_Check(o)) { PyErr_SetString(PyExc_TypeError, "expected a tensor or None"); throw Error(); }
  const at::Tensor& t = THPVariable_Unpack(o);
  *bytes = (size_t)t.numel() * t.element_size();
  return t.data_ptr();
}
long long integer(PyObject* o) {                            // int(o)
  if (PyLong_CheckExact(o)) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Error();
    return v;
  }
  PyObject* i = PyNumber_Long(o);
  if (!i) throw Error();
  const long long v = PyLong_AsLongLong(i);
  Py_DECREF(i);
  if (v == -1 && PyErr_Occurred()) throw Error();
  return v;
}
double real(PyObject* o) {                                  // float(o)
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Error();
  return v;
}
PyObject* current_stream = nullptr;                         // callable: the current stream's handle
void* stream_of(PyObject* o) {                              // a torch stream, or None for the current one
  PyObject* h = o == Py_None ? PyObject_CallNoArgs(current_stream) : PyObject_GetAttrString(o, "cuda_stream");
  if (!h) throw Error();
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(h);
  Py_DECREF(h);
  if (PyErr_Occurred()) throw Error();
  return (void*)(uintptr_t)v;
}
void* pointer(PyObject* o) { return (void*)(uintptr_t)(unsigned long long)integer(o); }
void count(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); throw Error(); }
}

// The tensors' common GPU, which becomes the current one until the end of the call (whatever was current), and the stream: the given one, which has to be of
// that GPU, or its current one.
struct OnDevice {
  std::optional<c10::DeviceGuard> guard;
  c10::Device device{c10::kCPU};
  void add(const char* name, const at::Tensor& t) {
    if (!guard) { device = t.device(); guard.emplace(device); return; }
    if (t.device() == device) return;
    PyErr_Format(PyExc_ValueError, "%s: expected a tensor on %s, got one on %s", name, device.str().c_str(), t.device().str().c_str());
    throw Error();
  }
  void* stream(PyObject* o) const {
    if (o != Py_None) {
      PyObject* at = PyObject_GetAttrString(o, "device_index");
      if (!at) throw Error();
      const long long index = integer(at);
      Py_DECREF(at);
      if (index != device.index()) {
        PyErr_Format(PyExc_ValueError, "stream: expected one of %s", device.str().c_str());
        throw Error();
      }
    }
    return stream_of(o);
  }
};

template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const Error&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
// the call itself, without the interpreter lock (a full launch queue makes it wait)
template <class F>
PyObject* status_of(F&& call) {
  gr_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
PyObject* workspace_wanted(size_t need) { return PyLong_FromUnsignedLongLong(need); }

// attn(q, k, v, cu_seqlens, k_own, v_own, slot | None, u, sm_scale, max_L, total_L, out, lse | None, workspace | None, stream, fp8, k_scale, v_scale)
//   -> status (<= 0), or the workspace bytes that the call needs when none was given
PyObject* attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    count(n, 18);
    const bool fp8 = a[15] == Py_True;
    const at::ScalarType kv = fp8 ? at::kByte : at::kBFloat16;
    const at::Tensor& q = tensor_nd(a[0], at::kBFloat16, "q", 4);
    const int64_t B = q.size(0), W = q.size(1), Hq = q.size(2), d = q.size(3);
    const at::Tensor& k = tensor_nd(a[1], kv, fp8 ? "k_shared_fp8" : "k_shared", 3);
    const int64_t rows = k.size(0), Hkv = k.size(1);
    tensor(a[1], kv, fp8 ? "k_shared_fp8" : "k_shared", {rows, Hkv, d});
    const at::Tensor& v = tensor(a[2], kv, fp8 ? "v_shared_fp8" : "v_shared", {rows, Hkv, d});
    const at::Tensor& cu = tensor(a[3], at::kInt, "cu_seqlens", {B + 1});
    const at::Tensor& ku = tensor_nd(a[4], at::kBFloat16, "k_unshared", 5);
    const int64_t ND = ku.size(2);
    tensor(a[4], at::kBFloat16, "k_unshared", {B, W, ND, Hkv, d});
    const at::Tensor& vu = tensor(a[5], at::kBFloat16, "v_unshared", {B, W, ND, Hkv, d});
    const long long total_L = integer(a[10]);
    if (rows < total_L) {
      PyErr_Format(PyExc_ValueError, "%s has fewer rows than total_L", fp8 ? "k_shared_fp8" : "k_shared");
      throw Error();
    }
    const at::Tensor& out = tensor(a[11], at::kBFloat16, "out", {B, W, Hq, d});
    gr_attn_fp8kv_params p;
    p.attn.B = (int32_t)B; p.attn.W = (int32_t)W; p.attn.Hq = (int32_t)Hq; p.attn.Hkv = (int32_t)Hkv; p.attn.d = (int32_t)d;
    p.attn.ND = (int32_t)ND; p.attn.u = (int32_t)integer(a[7]);
    p.attn.max_L = (int32_t)integer(a[9]); p.attn.total_L = total_L; p.attn.sm_scale = (float)real(a[8]);
    p.attn.q = q.data_ptr(); p.attn.k_shared = k.data_ptr(); p.attn.v_shared = v.data_ptr(); p.attn.cu_seqlens = (const int32_t*)cu.data_ptr();
    p.attn.k_unshared = ku.data_ptr(); p.attn.v_unshared = vu.data_ptr(); p.attn.out = out.data_ptr();
    p.attn.lse_out = a[12] == Py_None ? nullptr : (float*)tensor(a[12], at::kFloat, "lse_out", {B, W, Hq}).data_ptr();
    p.k_scale = (float)real(a[16]); p.v_scale = (float)real(a[17]);
    const int32_t* slot = a[6] == Py_None ? nullptr : (const int32_t*)tensor(a[6], at::kInt, "slot", {B, W, ND}).data_ptr();
    size_t ws_bytes;
    void* ws = const_cast<void*>(any_tensor(a[13], &ws_bytes));
    void* stream = stream_of(a[14]);
    if (a[13] == Py_None) {
      const size_t need = p_attn_ws(&p.attn);
      if (need > 0) return workspace_wanted(need);
    }
    return status_of([&] {
      return fp8 ? p_attn_fp8kv(&p, ws, ws_bytes, stream) : slot ? p_attn_slots(&p.attn, slot, ws, ws_bytes, stream) : p_attn(&p.attn, ws, ws_bytes, stream);
    });
  });
}

// prefill(q, k, v, cu_seqlens, sm_scale, max_L, total_L, out, lse | None, stream) -> status
PyObject* prefill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    count(n, 10);
    const at::Tensor& q = tensor_nd(a[0], at::kBFloat16, "q", 3);
    const int64_t T = q.size(0), Hq = q.size(1), d = q.size(2);
    const at::Tensor& k = tensor_nd(a[1], at::kBFloat16, "k", 3);
    const int64_t Hkv = k.size(1);
    tensor(a[1], at::kBFloat16, "k", {T, Hkv, d});
    const at::Tensor& v = tensor(a[2], at::kBFloat16, "v", {T, Hkv, d});
    const at::Tensor& cu = tensor_nd(a[3], at::kInt, "cu_seqlens", 1);
    const long long total_L = integer(a[6]);
    if (T < total_L) { PyErr_SetString(PyExc_ValueError, "q has fewer rows than total_L"); throw Error(); }
    const at::Tensor& out = tensor(a[7], at::kBFloat16, "out", {T, Hq, d});
    gr_prefill_params p;
    p.B = (int32_t)(cu.size(0) - 1); p.Hq = (int32_t)Hq; p.Hkv = (int32_t)Hkv; p.d = (int32_t)d;
    p.max_L = (int32_t)integer(a[5]); p.total_L = total_L; p.sm_scale = (float)real(a[4]);
    p.q = q.data_ptr(); p.k = k.data_ptr(); p.v = v.data_ptr(); p.cu_seqlens = (const int32_t*)cu.data_ptr(); p.out = out.data_ptr();
    p.lse_out = a[8] == Py_None ? nullptr : (float*)tensor(a[8], at::kFloat, "lse_out", {T, Hq}).data_ptr();
    void* stream = stream_of(a[9]);
    return status_of([&] { return p_prefill(&p, stream); });
  });
}

// select(mask | None, logits, scores_in, prefix_in, range_in, step, flags, parent, token, scores, prefix, range, item_index,
//        workspace | None, noalloc, stream) -> status, or the workspace bytes that the call needs
PyObject* select(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    count(n, 16);
    const at::Tensor& logits = tensor_nd(a[1], at::kFloat, "logits", 3);
    const int64_t B = logits.size(0), W = logits.size(1), V = logits.size(2);
    gr_select_params p;
    p.logits = (const float*)logits.data_ptr();
    p.scores_in = (const float*)tensor(a[2], at::kFloat, "scores_in", {B, W}).data_ptr();
    const at::Tensor& prefix = tensor_nd(a[3], at::kInt, "prefix_in", 3);
    const int64_t depth = prefix.size(2);
    p.prefix_in = (const int32_t*)tensor(a[3], at::kInt, "prefix_in", {B, W, depth}).data_ptr();
    p.range_in = (const int32_t*)tensor(a[4], at::kInt, "range_in", {B, W, 2}).data_ptr();
    p.parent_out = (int32_t*)tensor(a[7], at::kInt, "parent", {B, W}).data_ptr();
    p.token_out = (int32_t*)tensor(a[8], at::kInt, "token", {B, W}).data_ptr();
    p.scores_out = (float*)tensor(a[9], at::kFloat, "scores", {B, W}).data_ptr();
    p.prefix_out = (int32_t*)tensor(a[10], at::kInt, "prefix", {B, W, depth}).data_ptr();
    p.range_out = (int32_t*)tensor(a[11], at::kInt, "range", {B, W, 2}).data_ptr();
    p.item_index_out = (int32_t*)tensor(a[12], at::kInt, "item_index", {B, W}).data_ptr();
    p.B = (int32_t)B; p.W = (int32_t)W; p.V = (int32_t)V; p.depth = (int32_t)depth;
    p.step = (int32_t)integer(a[5]); p.flags = (int32_t)integer(a[6]);
    size_t bytes;
    p.mask = any_tensor(a[0], &bytes);
    void* ws = const_cast<void*>(any_tensor(a[13], &bytes));
    const bool noalloc = a[14] == Py_True;
    void* stream = stream_of(a[15]);
    if (!noalloc && a[13] == Py_None) return workspace_wanted(p_select_ws(p.B, p.W, p.V, p.depth));
    return status_of([&] { return noalloc ? p_select_noalloc(&p, stream) : p_select(&p, ws, bytes, stream); });
  });
}

// reorder(parent, k_own, v_own, u, stream) -> status
PyObject* reorder(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    count(n, 5);
    const at::Tensor& k = tensor_nd(a[1], at::kBFloat16, "k_unshared", 5);
    const at::Tensor& parent = tensor(a[0], at::kInt, "parent", {k.size(0), k.size(1)});
    const at::Tensor& v = tensor(a[2], at::kBFloat16, "v_unshared", k.sizes());
    const int32_t u = (int32_t)integer(a[3]);
    void* stream = stream_of(a[4]);
    return status_of([&] {
      return p_reorder((int32_t)k.size(0), (int32_t)k.size(1), (int32_t)k.size(2), (int32_t)k.size(3), (int32_t)k.size(4), u, (const int32_t*)parent.data_ptr(),
                       k.data_ptr(), v.data_ptr(), stream);
    });
  });
}

// slot_update(parent, slot_in | None, u, ND, out, stream) -> status
PyObject* slot_update(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    count(n, 6);
    const at::Tensor& parent = tensor_nd(a[0], at::kInt, "parent", 2);
    const int64_t B = parent.size(0), W = parent.size(1), ND = integer(a[3]);
    const int32_t* slot_in = a[1] == Py_None ? nullptr : (const int32_t*)tensor(a[1], at::kInt, "slot_in", {B, W, ND}).data_ptr();
    int32_t* out = (int32_t*)tensor(a[4], at::kInt, "out", {B, W, ND}).data_ptr();
    const int32_t u = (int32_t)integer(a[2]);
    void* stream = stream_of(a[5]);
    return status_of([&] { return p_slot_update((int32_t)B, (int32_t)W, (int32_t)ND, u, (const int32_t*)parent.data_ptr(), slot_in, out, stream); });
  });
}

// a number of the C ABI's structs
int32_t int32_of(int64_t v, const char* name) {
  if (v == (int32_t)v) return (int32_t)v;
  PyErr_Format(PyExc_ValueError, "%s: %lld does not fit 32 bits", name, (long long)v);
  throw Error();
}

// page_map(seq_lens, new_lens, free_pages, block_table, page_size, n_pages, total_new, lens, cu_new, slot, taken, stream) -> status
PyObject* page_map(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    count(n, 12);
    OnDevice on;
    auto ints = [&](PyObject* o, const char* name, c10::IntArrayRef shape) {
      const at::Tensor& t = tensor(o, at::kInt, name, shape);
      on.add(name, t);
      return (int32_t*)t.data_ptr();
    };
    const at::Tensor& table = tensor_nd(a[3], at::kInt, "block_table", 2);
    on.add("block_table", table);
    const int64_t B = table.size(0), free_pages = tensor_nd(a[2], at::kInt, "free_pages", 1).size(0);
    gr_page_map_params p{};
    p.B = (int32_t)B; p.max_pages = int32_of(table.size(1), "block_table"); p.page_size = int32_of(integer(a[4]), "page_size"); p.n_pages = int32_of(integer(a[5]), "n_pages");
    p.n_free = int32_of(free_pages, "free_pages"); p.total_new = integer(a[6]);
    p.seq_lens = ints(a[0], "seq_lens", {B}); p.new_lens = ints(a[1], "new_lens", {B}); p.free_pages = ints(a[2], "free_pages", {free_pages});
    p.block_table = (int32_t*)table.data_ptr();
    p.lens_out = ints(a[7], "lens", {B}); p.cu_new = ints(a[8], "cu_new", {B + 1}); p.slot = ints(a[9], "slot", {p.total_new}); p.taken = ints(a[10], "taken", {2});
    void* stream = on.stream(a[11]);
    return status_of([&] { return p_page_map(&p, stream); });
  });
}

// Rows [T, Hkv, d] that are whole in memory and one stride apart; -> that stride
int64_t rows_of(PyObject* o, const char* name, const at::Tensor** t) {
  *t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
  const bool dense = *t && (*t)->is_cuda() && (*t)->dim() == 3 && ((*t)->numel() == 0 || (((*t)->size(2) == 1 || (*t)->stride(2) == 1) && ((*t)->size(1) == 1 || (*t)->stride(1) == (*t)->size(2))));
  if (!dense) {
    PyErr_Format(PyExc_TypeError, "%s: expected a CUDA tensor [rows, KV heads, head size] of contiguous rows", name);
    throw Error();
  }
  if ((*t)->scalar_type() != at::kBFloat16) {
    PyErr_Format(PyExc_TypeError, "%s: expected torch.bfloat16, got %s", name, dtype_text((*t)->scalar_type()));
    throw Error();
  }
  return (*t)->size(0) > 1 ? (*t)->stride(0) : (*t)->size(1) * (*t)->size(2);
}
const at::Tensor& pool(PyObject* o, const char* name, bool* fp8) {
  *fp8 = THPVariable_Check(o) && THPVariable_Unpack(o).scalar_type() == at::kByte;
  return tensor_nd(o, *fp8 ? at::kByte : at::kBFloat16, name, 4);
}

// page_write(k, v, slot, k_pages, v_pages, k_scale, v_scale, stream) -> status
PyObject* page_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    count(n, 8);
    OnDevice on;
    const at::Tensor *k, *v;
    gr_page_write_params p{};
    p.k_stride = rows_of(a[0], "k", &k);
    p.v_stride = rows_of(a[1], "v", &v);
    on.add("k", *k);
    on.add("v", *v);
    if (v->sizes() != k->sizes()) {
      PyErr_Format(PyExc_ValueError, "v: expected shape %s, got %s", shape_text(k->sizes()).c_str(), shape_text(v->sizes()).c_str());
      throw Error();
    }
    bool fp8;
    const at::Tensor& kp = pool(a[3], "k_pages", &fp8);
    const at::ScalarType type = fp8 ? at::kByte : at::kBFloat16;
    tensor(a[3], type, "k_pages", {kp.size(0), kp.size(1), k->size(1), k->size(2)});
    const at::Tensor& vp = tensor(a[4], type, "v_pages", kp.sizes());
    const at::Tensor& slot = tensor(a[2], at::kInt, "slot", {k->size(0)});
    on.add("slot", slot);
    on.add("k_pages", kp);
    on.add("v_pages", vp);
    p.T = k->size(0); p.Hkv = (int32_t)k->size(1); p.d = (int32_t)k->size(2); p.n_pages = (int32_t)kp.size(0); p.page_size = (int32_t)kp.size(1);
    p.kv_type = fp8 ? GR_KV_FP8 : GR_KV_BF16;
    p.k_scale = (float)real(a[5]); p.v_scale = (float)real(a[6]);
    p.k = k->data_ptr(); p.v = v->data_ptr(); p.slot = (const int32_t*)slot.data_ptr(); p.k_pages = kp.data_ptr(); p.v_pages = vp.data_ptr();
    void* stream = on.stream(a[7]);
    return status_of([&] { return p_page_write(&p, stream); });
  });
}

// attn_paged(q, k_pages, v_pages, block_table, seq_lens, k_own | None, v_own | None, u, sm_scale, max_L, prefix_pages | None, prefix_L, k_scale, v_scale,
//            slot | None, out, lse | None, workspace | None, stream) -> status (<= 0), or the workspace bytes that the call needs when none was given
PyObject* attn_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    count(n, 19);
    OnDevice on;
    const at::Tensor& q = tensor_nd(a[0], at::kBFloat16, "q", 4);
    on.add("q", q);
    const int64_t B = q.size(0), W = q.size(1), Hq = q.size(2), d = q.size(3);
    auto given = [&](PyObject* o, at::ScalarType type, const char* name, c10::IntArrayRef shape) -> void* {
      if (o == Py_None) return nullptr;
      const at::Tensor& t = tensor(o, type, name, shape);
      on.add(name, t);
      return t.data_ptr();
    };
    bool fp8;
    const at::Tensor& kp = pool(a[1], "k_pages", &fp8);
    const at::ScalarType type = fp8 ? at::kByte : at::kBFloat16;
    const int64_t pages = kp.size(0), page = kp.size(1), Hkv = kp.size(2);
    gr_attn_paged_params p{};
    p.k_pages = given(a[1], type, "k_pages", {pages, page, Hkv, d});
    p.v_pages = given(a[2], type, "v_pages", {pages, page, Hkv, d});
    const at::Tensor& table = tensor_nd(a[3], at::kInt, "block_table", 2);
    p.block_table = (const int32_t*)given(a[3], at::kInt, "block_table", {B, table.size(1)});
    p.seq_lens = (const int32_t*)given(a[4], at::kInt, "seq_lens", {B});
    const long long prefix_L = integer(a[11]), max_L = integer(a[9]);
    if (prefix_L < 0 || prefix_L >= (1ll << 31) || max_L < 0 || max_L >= (1ll << 31)) { PyErr_SetString(PyExc_ValueError, "prefix_L and max_L: expected numbers of tokens"); throw Error(); }
    p.prefix_pages = page > 0 && prefix_L % page == 0 ? (const int32_t*)given(a[10], at::kInt, "prefix_pages", {prefix_L / page}) : nullptr;
    const int64_t ND = a[5] == Py_None ? 0 : tensor_nd(a[5], at::kBFloat16, "k_unshared", 5).size(2);
    p.k_unshared = given(a[5], at::kBFloat16, "k_unshared", {B, W, ND, Hkv, d});
    p.v_unshared = given(a[6], at::kBFloat16, "v_unshared", {B, W, ND, Hkv, d});
    p.slot = (const int32_t*)given(a[14], at::kInt, "slot", {B, W, ND});
    p.out = given(a[15], at::kBFloat16, "out", {B, W, Hq, d});
    p.lse_out = (float*)given(a[16], at::kFloat, "lse_out", {B, W, Hq});
    p.B = (int32_t)B; p.W = (int32_t)W; p.Hq = (int32_t)Hq; p.Hkv = (int32_t)Hkv; p.d = (int32_t)d; p.ND = (int32_t)ND; p.u = int32_of(integer(a[7]), "u");
    p.page_size = (int32_t)page; p.max_pages = int32_of(table.size(1), "block_table"); p.n_pages = (int32_t)pages; p.prefix_L = (int32_t)prefix_L; p.max_L = (int32_t)max_L;
    p.kv_type = fp8 ? GR_KV_FP8 : GR_KV_BF16;
    p.sm_scale = (float)real(a[8]); p.k_scale = (float)real(a[12]); p.v_scale = (float)real(a[13]);
    p.q = q.data_ptr();
    size_t ws_bytes;
    void* ws = const_cast<void*>(any_tensor(a[17], &ws_bytes));
    if (a[17] != Py_None) on.add("workspace", THPVariable_Unpack(a[17]));
    void* stream = on.stream(a[18]);
    if (a[17] == Py_None) {
      const size_t need = p_attn_paged_ws(&p);
      if (need > 0) return workspace_wanted(need);
    }
    return status_of([&] { return p_attn_paged(&p, ws, ws_bytes, stream); });
  });
}

// adjust(logits, step, prefix | None, scores | None, history | None, cu_history | None, repetition | None, frequency | None, presence | None, bias | None,
//        allowed | None, allowed_row | None, out, stream) -> status
PyObject* adjust(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    count(n, 14);
    OnDevice on;
    const at::Tensor& logits = tensor_nd(a[0], at::kFloat, "logits", 3);
    on.add("logits", logits);
    const int64_t B = logits.size(0), W = logits.size(1), V = logits.size(2);
    auto given = [&](PyObject* o, at::ScalarType type, const char* name, c10::IntArrayRef shape) -> void* {
      if (o == Py_None) return nullptr;
      const at::Tensor& t = tensor(o, type, name, shape);
      on.add(name, t);
      return t.data_ptr();
    };
    gr_logits_adjust_params p{};
    const int64_t rows = a[4] == Py_None ? 0 : tensor_nd(a[4], at::kInt, "history", 2).size(0);
    const int64_t depth = a[4] != Py_None ? tensor_nd(a[4], at::kInt, "history", 2).size(1) : a[2] != Py_None ? tensor_nd(a[2], at::kInt, "prefix", 3).size(2) : integer(a[1]) + 1;
    p.logits = (const float*)logits.data_ptr();
    p.prefix = (const int32_t*)given(a[2], at::kInt, "prefix", {B, W, depth});
    p.scores = (const float*)given(a[3], at::kFloat, "scores", {B, W});
    p.history = (const int32_t*)given(a[4], at::kInt, "history", {rows, depth});
    p.cu_history = (const int32_t*)given(a[5], at::kInt, "cu_history", {B + 1});
    p.repetition = (const float*)given(a[6], at::kFloat, "repetition", {B});
    p.frequency = (const float*)given(a[7], at::kFloat, "frequency", {B});
    p.presence = (const float*)given(a[8], at::kFloat, "presence", {B});
    const bool of_request = a[9] != Py_None && THPVariable_Check(a[9]) && THPVariable_Unpack(a[9]).dim() == 2;
    p.bias = (const float*)(of_request ? given(a[9], at::kFloat, "bias", {B, V}) : given(a[9], at::kFloat, "bias", {V}));
    p.bias_rows = of_request ? (int32_t)B : 1;
    const int64_t masks = a[10] == Py_None ? 0 : tensor_nd(a[10], at::kInt, "allowed", 2).size(0);
    p.allowed = (const uint32_t*)given(a[10], at::kInt, "allowed", {masks, (V + 31) / 32});
    p.allowed_row = (const int32_t*)given(a[11], at::kInt, "allowed_row", {B, W});
    p.out = (float*)given(a[12], at::kFloat, "out", {B, W, V});
    p.B = (int32_t)B; p.W = (int32_t)W; p.V = (int32_t)V; p.depth = (int32_t)depth; p.step = int32_of(integer(a[1]), "step");
    p.n_history = int32_of(rows, "history"); p.n_allowed = int32_of(masks, "allowed");
    void* stream = on.stream(a[13]);
    return status_of([&] { return p_adjust(&p, stream); });
  });
}

// bind(addresses of the fifteen entry points in the order of their declaration above, callable that returns the current stream's handle)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    count(n, 16);
    p_attn = (decltype(p_attn))pointer(a[0]);
    p_attn_slots = (decltype(p_attn_slots))pointer(a[1]);
    p_attn_fp8kv = (decltype(p_attn_fp8kv))pointer(a[2]);
    p_attn_ws = (decltype(p_attn_ws))pointer(a[3]);
    p_prefill = (decltype(p_prefill))pointer(a[4]);
    p_select = (decltype(p_select))pointer(a[5]);
    p_select_noalloc = (decltype(p_select_noalloc))pointer(a[6]);
    p_select_ws = (decltype(p_select_ws))pointer(a[7]);
    p_reorder = (decltype(p_reorder))pointer(a[8]);
    p_slot_update = (decltype(p_slot_update))pointer(a[9]);
    p_page_map = (decltype(p_page_map))pointer(a[10]);
    p_page_write = (decltype(p_page_write))pointer(a[11]);
    p_attn_paged = (decltype(p_attn_paged))pointer(a[12]);
    p_attn_paged_ws = (decltype(p_attn_paged_ws))pointer(a[13]);
    p_adjust = (decltype(p_adjust))pointer(a[14]);
    Py_INCREF(a[15]);
    Py_XSETREF(current_stream, a[15]);
    Py_RETURN_NONE;
  });
}

PyMethodDef methods[] = {{"attn", (PyCFunction)(void*)attn, METH_FASTCALL, nullptr},
                         {"prefill", (PyCFunction)(void*)prefill, METH_FASTCALL, nullptr},
                         {"select", (PyCFunction)(void*)select, METH_FASTCALL, nullptr},
                         {"reorder", (PyCFunction)(void*)reorder, METH_FASTCALL, nullptr},
                         {"slot_update", (PyCFunction)(void*)slot_update, METH_FASTCALL, nullptr},
                         {"page_map", (PyCFunction)(void*)page_map, METH_FASTCALL, nullptr},
                         {"page_write", (PyCFunction)(void*)page_write, METH_FASTCALL, nullptr},
                         {"attn_paged", (PyCFunction)(void*)attn_paged, METH_FASTCALL, nullptr},
                         {"adjust", (PyCFunction)(void*)adjust, METH_FASTCALL, nullptr},
                         {"bind", (PyCFunction)(void*)bind, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "gr_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_gr_bind(void) { return PyModule_Create(&module); }
