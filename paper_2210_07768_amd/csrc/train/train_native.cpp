// The part of the trainer's Python binding that runs once per call: checks of tensors, results and scratch from
// torch's allocator, the lists of slots and tensors as the C ABI takes them.  In Python this took 9 us for a gated block,
// 20 for 24 slots and 90 for 48 tensors, more than the GPU needs for small ones.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>
#include <vector>

#include "fbx_train.h"

namespace {

struct {
  decltype(&fbx_train_last_error) last_error;
  decltype(&fbx_embed_forward) embed_forward;
  decltype(&fbx_embed_backward_scratch) embed_backward_scratch;
  decltype(&fbx_embed_backward) embed_backward;
  decltype(&fbx_gated_scratch) gated_scratch;
  decltype(&fbx_gated_forward) gated_forward;
  decltype(&fbx_gated_backward) gated_backward;
  decltype(&fbx_adamw_step) adamw_step;
} g;
PyObject *g_error = nullptr, *g_stream = nullptr;  // FbxError; torch's function from a device to its current stream
PyObject* g_memory = nullptr;  // torch.OutOfMemoryError
PyObject *g_values, *g_offsets, *g_arity, *g_ends;

struct Refused {
  fbx_status status;
  std::string why;
};
[[noreturn]] void bad(std::string why) { throw Refused{FBX_E_ARG, std::move(why)}; }
void check(fbx_status s) {
  if (s != FBX_OK) throw Refused{s, g.last_error()};
}
struct PythonError {};

// Runs a call; its exceptions become Python's.
template <class F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const Refused& r) {
    PyObject* e = PyObject_CallFunction(g_error, "is", static_cast<int>(r.status), r.why.c_str());
    if (e) {
      PyErr_SetObject(g_error, e);
      Py_DECREF(e);
    }
  } catch (const PythonError&) {
  } catch (const std::bad_alloc&) {
    PyErr_NoMemory();
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(g_memory ? g_memory : PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) bad(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}
// A tensor whose gradient a call may take part in.  A tangent (forward mode) would be lost without a word.
const at::Tensor& input(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t._fw_grad(0).defined()) bad(std::string(name) + ": derivatives in forward mode are not supported");
  return t;
}
fbx_dtype code(const at::Tensor& t) {
  const auto s = t.scalar_type();
  if (s == at::kFloat) return FBX_F32;
  if (s == at::kHalf) return FBX_F16;
  if (s == at::kBFloat16) return FBX_BF16;
  bad(std::string(c10::toString(s)) + ": float32, float16 and bfloat16 are supported");
}
void* on_gpu(const at::Tensor& t) {
  if (!t.is_cuda()) bad("tensors must be on the GPU");
  return t.data_ptr();
}
void* stream_of(const at::Tensor& t) {
  PyObject* i = PyLong_FromLong(t.get_device());
  PyObject* s = i ? PyObject_CallOneArg(g_stream, i) : nullptr;
  Py_XDECREF(i);
  if (!s) throw PythonError{};
  void* p = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return p;
}

// A matrix whose rows are contiguous; the distance between them.
uint64_t matrix(const at::Tensor& t, const char* name, const at::Tensor* like = nullptr, int64_t rows = -1, int64_t cols = -1) {
  if (t.dim() != 2) bad(std::string(name) + " must have two dimensions");
  if (like && (t.scalar_type() != like->scalar_type() || t.device() != like->device())) bad(std::string(name) + " must have the type and device of the others");
  if (rows >= 0 && (t.size(0) != rows || t.size(1) != cols))
    bad(std::string(name) + " must be of shape (" + std::to_string(rows) + ", " + std::to_string(cols) + ")");
  if (t.size(1) > 1 && t.stride(1) != 1) bad(std::string(name) + ": elements of a row must be adjacent");
  if (t.size(0) <= 1) return t.size(1);
  if (t.stride(0) < t.size(1)) bad(std::string(name) + ": rows may not overlap");
  return t.stride(0);
}

// A tensor given for a result, like torch's own `out`: it has no history of its own.
const at::Tensor& result(PyObject* o) {
  const at::Tensor& t = tensor(o, "out");
  if (t.requires_grad() && c10::GradMode::is_enabled()) bad("out cannot take part in autograd");
  return t;
}
// Autograd then knows that it changed.
void changed(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

at::Tensor scratch(uint64_t bytes, const at::Tensor& like) {
  return bytes ? at::empty({static_cast<int64_t>(bytes)}, like.options().dtype(at::kByte).memory_format(c10::nullopt)) : at::Tensor();
}
void* pointer(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
PyObject* wrap(at::Tensor t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(std::move(t));
}

struct Held {
  PyObject* o;
  ~Held() { Py_XDECREF(o); }
};
// A slot's k-th part (a new reference): an attribute, or an entry of a tuple.
PyObject* part_of(PyObject* slot, int k) {
  PyObject* const names[4] = {g_values, g_offsets, g_arity, g_ends};
  const bool tuple = PyTuple_Check(slot) && PyTuple_GET_SIZE(slot) == 4;
  PyObject* o = tuple ? PyTuple_GET_ITEM(slot, k) : PyObject_GetAttr(slot, names[k]);
  if (!o) throw PythonError{};
  if (tuple) Py_INCREF(o);
  return o;
}

// The slots of a call: the library's own table as bytes, or a sequence of objects with values, offsets, fixed_arity and
// tile_ends (a tuple has them in this order).
struct Slots {
  std::vector<fbx_slot_view> own;
  const fbx_slot_view* views = nullptr;
  uint32_t n = 0;

  Slots(PyObject* o, int64_t n_records, const at::Device& device) {
    if (PyBytes_Check(o)) {
      views = reinterpret_cast<const fbx_slot_view*>(PyBytes_AS_STRING(o));
      n = static_cast<uint32_t>(PyBytes_GET_SIZE(o) / sizeof(fbx_slot_view));
      return;
    }
    PyObject* seq = PySequence_Fast(o, "slots must be an ExtractResult or a sequence");
    if (!seq) throw PythonError{};
    const Held held{seq};
    own.resize(PySequence_Fast_GET_SIZE(seq));
    for (size_t i = 0; i < own.size(); ++i) {
      PyObject* s = PySequence_Fast_GET_ITEM(seq, i);
      const Held part[4] = {{part_of(s, 0)}, {part_of(s, 1)}, {part_of(s, 2)}, {part_of(s, 3)}};
      if (part[3].o != Py_None) bad("slots in arrival order are taken as a whole ExtractResult");
      fbx_slot_view& v = own[i] = fbx_slot_view{};
      const at::Tensor& values = whole(part[0].o, device, "a slot's values must be contiguous 64-bit integers on the table's device");
      v.n_values = values.numel();
      v.values = static_cast<const uint64_t*>(values.data_ptr());
      if (part[1].o == Py_None) {
        const long long arity = PyLong_AsLongLong(part[2].o);
        if (arity == -1 && PyErr_Occurred()) throw PythonError{};
        if (arity < 1 || arity > 0xffffffffll) bad("a slot without offsets has a fixed_arity of at least 1");
        v.fixed_arity = static_cast<uint32_t>(arity);
      } else {
        const char* why = "a slot's offsets must be n_records + 1 contiguous 64-bit integers on the table's device";
        const at::Tensor& offsets = whole(part[1].o, device, why);
        if (offsets.numel() != n_records + 1) bad(why);
        v.offsets = static_cast<const uint64_t*>(offsets.data_ptr());
      }
    }
    views = own.data();
    n = static_cast<uint32_t>(own.size());
  }
  static const at::Tensor& whole(PyObject* o, const at::Device& device, const char* why) {
    const at::Tensor& t = tensor(o, "a slot's array");
    if (t.device() != device || (t.scalar_type() != at::kLong && t.scalar_type() != at::kUInt64) || !t.is_contiguous()) bad(why);
    return t;
  }
};

// versions(tensor, or a sequence of slots): grows whenever torch, or a call of this library's binding, has written to what was given.
PyObject* versions(PyObject*, PyObject* o) {
  return guarded([&]() -> PyObject* {
    auto version = [](PyObject* t) -> unsigned long long {
      if (!THPVariable_Check(t) || THPVariable_Unpack(t).is_inference()) return 0;
      return THPVariable_Unpack(t).unsafeGetTensorImpl()->version_counter().current_version();
    };
    if (THPVariable_Check(o)) return PyLong_FromUnsignedLongLong(version(o));
    const Held seq{PySequence_Fast(o, "slots must be an ExtractResult or a sequence")};
    if (!seq.o) throw PythonError{};
    unsigned long long sum = 0;
    for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(seq.o); ++i)
      for (int k = 0; k < 2; ++k) {
        const Held array{part_of(PySequence_Fast_GET_ITEM(seq.o, i), k)};
        sum += version(array.o);
      }
    return PyLong_FromUnsignedLongLong(sum);
  });
}

// embed(slots, table, n_records, tile, mean, out)
PyObject* embed(PyObject*, PyObject* args) {
  PyObject *slots_o, *table_o, *out_o;
  long long n_records;
  unsigned int tile;
  int mean;
  if (!PyArg_ParseTuple(args, "OOLIpO", &slots_o, &table_o, &n_records, &tile, &mean, &out_o)) return nullptr;
  return guarded([&] {
    const at::Tensor& table = input(table_o, "table");
    const fbx_dtype dtype = code(table);
    const int64_t rows = table.dim() == 2 ? table.size(0) : 0, dim = table.dim() == 2 ? table.size(1) : 0;
    const uint64_t stride = matrix(table, "table");
    if (n_records < 0) bad("n_records is negative");
    const Slots slots(slots_o, n_records, table.device());
    on_gpu(table);
    const c10::DeviceGuard guard(table.device());
    at::Tensor out;
    if (out_o == Py_None) {
      out = at::empty({n_records, slots.n, dim}, table.options());
    } else {
      out = result(out_o);
      if (out.dim() != 3 || out.size(0) != n_records || out.size(1) != slots.n || out.size(2) != dim || out.scalar_type() != table.scalar_type() || out.device() != table.device())
        bad("out must be n_records x slots x dim with the table's type and device");
      if ((dim > 1 && out.stride(2) != 1) || (slots.n > 1 && out.stride(1) != dim)) bad("out: a record's rows must be adjacent");
    }
    const uint64_t record_stride = n_records > 1 ? out.stride(0) : slots.n * dim;
    check(g.embed_forward(slots.views, slots.n, n_records, tile, table.data_ptr(), rows, static_cast<uint32_t>(dim), stride, dtype, mean, out.data_ptr(), record_stride,
                          stream_of(table)));
    if (out_o != Py_None) changed(out);
    return wrap(std::move(out));
  });
}

// embed_backward(dout, slots, tile, rows, mean, out)
PyObject* embed_backward(PyObject*, PyObject* args) {
  PyObject *dout_o, *slots_o, *out_o;
  unsigned int tile;
  long long rows;
  int mean;
  if (!PyArg_ParseTuple(args, "OOILpO", &dout_o, &slots_o, &tile, &rows, &mean, &out_o)) return nullptr;
  return guarded([&] {
    at::Tensor dout = input(dout_o, "dout");
    const fbx_dtype dtype = code(dout);
    const int64_t n_records = dout.size(0), n_slots = dout.size(1), dim = dout.size(2);
    const Slots slots(slots_o, n_records, dout.device());
    if (slots.n != n_slots) bad("dout must have as many slots as there are");
    if (rows < 1) bad("rows must be at least 1");
    on_gpu(dout);
    const c10::DeviceGuard guard(dout.device());
    if ((dim > 1 && dout.stride(2) != 1) || (n_slots > 1 && dout.stride(1) != dim) || (n_records > 1 && dout.stride(0) < n_slots * dim)) dout = dout.contiguous();
    at::Tensor out = out_o == Py_None ? at::empty({rows, dim}, dout.options()) : result(out_o);
    const uint64_t stride = matrix(out, "out", &dout, rows, dim);
    uint64_t need = 0;
    check(g.embed_backward_scratch(slots.views, slots.n, n_records, rows, static_cast<uint32_t>(dim), mean, &need));
    const at::Tensor s = scratch(need, dout);
    check(g.embed_backward(slots.views, slots.n, n_records, tile, dout.data_ptr(), n_records > 1 ? dout.stride(0) : n_slots * dim, rows, static_cast<uint32_t>(dim), stride,
                           dtype, mean, out.data_ptr(), pointer(s), need, stream_of(dout)));
    if (out_o != Py_None) changed(out);
    return wrap(std::move(out));
  });
}

struct Block {
  fbx_gated a{};
  const at::Tensor &x, &w_gate, &w_up;

  Block(PyObject* x_o, PyObject* gate_o, PyObject* up_o, int act) : x(input(x_o, "x")), w_gate(input(gate_o, "w_gate")), w_up(input(up_o, "w_up")) {
    a.dtype = code(x);
    a.ld_x = matrix(x, "x");
    const int64_t hidden = w_gate.dim() == 2 ? w_gate.size(0) : 0;
    a.ld_w_gate = matrix(w_gate, "w_gate", &x, hidden, x.size(1));
    a.ld_w_up = matrix(w_up, "w_up", &x, hidden, x.size(1));
    if (hidden >> 32 || x.size(1) >> 32) bad("inputs and hidden must be 1 .. 2^20");
    a.records = x.size(0);
    a.inputs = static_cast<uint32_t>(x.size(1));
    a.hidden = static_cast<uint32_t>(hidden);
    a.act = static_cast<fbx_act>(act);
    a.d_x = x.data_ptr();
    a.d_w_gate = w_gate.data_ptr();
    a.d_w_up = w_up.data_ptr();
  }
};

// gated(x, w_gate, w_up, act, out)
PyObject* gated(PyObject*, PyObject* args) {
  PyObject *x, *gate, *up, *out_o;
  int act;
  if (!PyArg_ParseTuple(args, "OOOiO", &x, &gate, &up, &act, &out_o)) return nullptr;
  return guarded([&] {
    const Block b(x, gate, up, act);
    if (out_o != Py_None) matrix(result(out_o), "out", &b.x, b.a.records, b.a.hidden);
    on_gpu(b.x);
    const c10::DeviceGuard guard(b.x.device());
    at::Tensor out = out_o == Py_None ? at::empty({static_cast<int64_t>(b.a.records), b.a.hidden}, b.x.options()) : tensor(out_o, "out");
    const uint64_t ld = matrix(out, "out");
    uint64_t need = 0;
    check(g.gated_scratch(&b.a, 0, &need));
    const at::Tensor s = scratch(need, b.x);
    check(g.gated_forward(&b.a, out.data_ptr(), ld, pointer(s), need, stream_of(b.x)));
    if (out_o != Py_None) changed(out);
    return wrap(std::move(out));
  });
}

// gated_backward(dh, x, w_gate, w_up, act, need_dx, need_dw)
PyObject* gated_backward(PyObject*, PyObject* args) {
  PyObject *dh_o, *x, *gate, *up;
  int act, need_dx, need_dw;
  if (!PyArg_ParseTuple(args, "OOOOipp", &dh_o, &x, &gate, &up, &act, &need_dx, &need_dw)) return nullptr;
  return guarded([&]() -> PyObject* {
    const Block b(x, gate, up, act);
    const at::Tensor& dh = input(dh_o, "dh");
    const uint64_t ld_dh = matrix(dh, "dh", &b.x, b.a.records, b.a.hidden), k = b.a.inputs;
    on_gpu(b.x);
    const c10::DeviceGuard guard(b.x.device());
    at::Tensor dx, dw_gate, dw_up;
    if (need_dx) dx = at::empty({static_cast<int64_t>(b.a.records), static_cast<int64_t>(k)}, b.x.options());
    if (need_dw) {
      dw_gate = at::empty({b.a.hidden, static_cast<int64_t>(k)}, b.x.options());
      dw_up = at::empty({b.a.hidden, static_cast<int64_t>(k)}, b.x.options());
    }
    uint64_t need = 0;
    check(g.gated_scratch(&b.a, 1, &need));
    const at::Tensor s = scratch(need, b.x);
    check(g.gated_backward(&b.a, dh.data_ptr(), ld_dh, pointer(dx), k, pointer(dw_gate), k, pointer(dw_up), k, pointer(s), need, stream_of(b.x)));
    PyObject* out = PyTuple_New(3);
    if (!out) throw PythonError{};
    PyTuple_SET_ITEM(out, 0, wrap(std::move(dx)));
    PyTuple_SET_ITEM(out, 1, wrap(std::move(dw_gate)));
    PyTuple_SET_ITEM(out, 2, wrap(std::move(dw_up)));
    return out;
  });
}

// A list of tensors; none where it is None.
struct List {
  PyObject* seq = nullptr;
  explicit List(PyObject* o) {
    if (o == Py_None) return;
    seq = PySequence_Fast(o, "params, grads, states and copies must be lists");
    if (!seq) throw PythonError{};
  }
  ~List() { Py_XDECREF(seq); }
  List(const List&) = delete;
  Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(seq); }
  const at::Tensor& operator[](Py_ssize_t i) const { return tensor(PySequence_Fast_GET_ITEM(seq, i), "an entry of a list"); }
};

// adamw(params, grads, m, v, m_scale, v_scale, copies, step, lr, beta1, beta2, eps, weight_decay, grad_scale, seed, keep_roots, check_only)
PyObject* adamw(PyObject*, PyObject* args) {
  PyObject* lists[7];
  fbx_adamw h{};
  unsigned long long step, seed;
  int keep_roots, check_only;
  if (!PyArg_ParseTuple(args, "OOOOOOOKddddddKpp", &lists[0], &lists[1], &lists[2], &lists[3], &lists[4], &lists[5], &lists[6], &step, &h.lr, &h.beta1, &h.beta2, &h.eps,
                        &h.weight_decay, &h.grad_scale, &seed, &keep_roots, &check_only))
    return nullptr;
  return guarded([&]() -> PyObject* {
    const List p(lists[0]), grad(lists[1]), m(lists[2]), v(lists[3]), m_scale(lists[4]), v_scale(lists[5]), copy(lists[6]);
    if (!p.seq || !grad.seq || !m.seq || !v.seq || !m_scale.seq != !v_scale.seq) bad("params, grads and states must be lists, and m_scale and v_scale both or neither");
    const Py_ssize_t n = p.size();
    for (const List* l : {&grad, &m, &v, &m_scale, &v_scale, &copy})
      if (l->seq && l->size() != n) bad("params, grads, states and copies must be lists of one length");
    if (!n) Py_RETURN_NONE;
    const bool eight = m_scale.seq;
    h.state_bits = !eight ? 32 : keep_roots ? 8 | FBX_ADAMW_KEEP_ROOTS : 8;
    h.step = step;
    h.seed = seed;
    h.param_dtype = code(p[0]);
    h.grad_dtype = code(grad[0]);
    h.copy_dtype = copy.seq ? code(copy[0]) : FBX_F32;
    const at::Device where = p[0].device();
    auto same = [&](const at::Tensor& t) {
      if (t.device() != where || !t.is_contiguous()) bad("all tensors must be contiguous and on one device");
      return t.data_ptr();
    };
    std::vector<fbx_adamw_tensor> all(n);
    for (Py_ssize_t i = 0; i < n; ++i) {
      fbx_adamw_tensor& t = all[i];
      const int64_t size = p[i].numel(), blocks = (size + 31) / 32;
      if (p[i].scalar_type() != p[0].scalar_type() || grad[i].scalar_type() != grad[0].scalar_type() || (copy.seq && copy[i].scalar_type() != copy[0].scalar_type()))
        bad("all weights are of one type, and so are all gradients and all copies");
      if (grad[i].sizes() != p[i].sizes() || m[i].numel() != size || v[i].numel() != size || (eight && (m_scale[i].numel() != blocks || v_scale[i].numel() != blocks)) ||
          (copy.seq && copy[i].numel() != size))
        bad("a gradient, state or copy is not of its weights' size");
      if (eight) {
        if (m[i].itemsize() != 1 || v[i].itemsize() != 1 || m_scale[i].itemsize() != 1 || v_scale[i].itemsize() != 1) bad("8-bit states are held in bytes");
      } else if (m[i].scalar_type() != at::kFloat || v[i].scalar_type() != at::kFloat) {
        bad("32-bit states are float32");
      }
      t.d_param = same(p[i]);
      t.d_grad = same(grad[i]);
      t.d_m = same(m[i]);
      t.d_v = same(v[i]);
      if (eight) {
        t.d_m_scale = static_cast<uint8_t*>(same(m_scale[i]));
        t.d_v_scale = static_cast<uint8_t*>(same(v_scale[i]));
      }
      if (copy.seq) t.d_copy = same(copy[i]);
      // (what the library refuses too, but of one list at a time)
      if (size && copy.seq && (h.copy_dtype == FBX_F32 || h.param_dtype != FBX_F32)) bad("a copy is in float16 or bfloat16, of weights in float32");
      if (static_cast<uint64_t>(size) > FBX_ADAMW_MOST) bad("a tensor has more than 2^35 - 2048 elements");
      t.n = size;
    }
    on_gpu(p[0]);
    if (check_only) Py_RETURN_NONE;
    const c10::DeviceGuard guard(where);
    check(g.adamw_step(&h, all.data(), static_cast<uint32_t>(n), stream_of(p[0])));
    for (Py_ssize_t i = 0; i < n; ++i)
      for (const List* l : {&p, &m, &v, &m_scale, &v_scale, &copy})
        if (l->seq) changed((*l)[i]);
    Py_RETURN_NONE;
  });
}

// bind(FbxError, torch.OutOfMemoryError, stream function, addresses of the library's functions in the order of `g`)
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *error, *memory, *stream;
  unsigned long long at[8];
  if (!PyArg_ParseTuple(args, "OOOKKKKKKKK", &error, &memory, &stream, &at[0], &at[1], &at[2], &at[3], &at[4], &at[5], &at[6], &at[7])) return nullptr;
  static_assert(sizeof g == sizeof at, "eight pointers");
  memcpy(&g, at, sizeof g);
  Py_INCREF(error);
  Py_INCREF(memory);
  Py_INCREF(stream);
  g_error = error;
  g_memory = memory;
  g_stream = stream;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         {"embed", embed, METH_VARARGS, nullptr},
                         {"versions", versions, METH_O, nullptr},
                         {"embed_backward", embed_backward, METH_VARARGS, nullptr},
                         {"gated", gated, METH_VARARGS, nullptr},
                         {"gated_backward", gated_backward, METH_VARARGS, nullptr},
                         {"adamw", adamw, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_train", "The native part of the trainer's binding.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__train(void) {
  g_values = PyUnicode_InternFromString("values");
  g_offsets = PyUnicode_InternFromString("offsets");
  g_arity = PyUnicode_InternFromString("fixed_arity");
  g_ends = PyUnicode_InternFromString("tile_ends");
  return PyModule_Create(&module);
}
