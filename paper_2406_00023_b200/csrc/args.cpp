// Argument marshalling of the row operators (tokens sorted by a given choice, norms around a block) and of the calls composed of
// them for Python: a call of a few microseconds on the GPU should not wait for as many of attribute look-ups.  Checks what
// addresses alone do not show (type, place, order and size of every tensor, what buffers were made for), takes the current
// stream, and calls the C function with plain pointers.
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <utility>

#include "../../include/etr.h"

namespace {

enum Config { SORT, NORM, LAYER };               // of an operator's first argument
// ACT_*: rows of activations (R: rows of the sorted buffers); W_EHD, G_EHD: an expert weight, its gradient; the rest are handles
enum Kind { ACT_TD, ACT_RD, F32_D, F32_T, F32_TK, F32_EM, I32_TK, W_EHD, G_EHD, SCRATCH, PLAN, LAYER_BUF, BLOCK_BUF, NORM_CFG };

// Buffers, the configuration that their memory was carved for, and the device that it is on (-1: not a GPU).
struct PlanFor {
  etr_sort_plan plan;
  etr_sort_config made;
  int32_t device;
  bool fits(const etr_sort_config& c) const {      // d and dtype do not matter to it
    return made.T == c.T && made.k == c.k && made.E == c.E && made.align == c.align && made.capacity == c.capacity;
  }
};
struct LayerFor {
  etr_buffers buf;
  etr_config made;
  int32_t device;
  // Buffers of a larger layer serve a smaller one.  The scratch has a size of its own, which the C call checks.  router: the layer's
  // own router runs too, whose members are as long as the batch; the experts alone need the rows.
  bool fits(const etr_config& c, bool router) const {
    const auto rows = [](const etr_config& q) { return (int64_t)q.E * ((q.capacity + 127ll) / 128 * 128); };
    const auto bytes = [](const etr_config& q) { return q.dtype == ETR_BF16 ? 2 : 4; };
    const __int128 has = rows(made) * bytes(made), wants = rows(c) * bytes(c);
    if (wants * c.d > has * made.d || wants * c.h > has * made.h) return false;
    return !router || (rows(c) <= rows(made) && c.T <= made.T && c.E <= made.E && (int64_t)c.T * c.k <= (int64_t)made.T * made.k &&
                       (int64_t)c.T * c.E <= (int64_t)made.T * made.E && (int64_t)c.T * (c.d / c.D) <= (int64_t)made.T * (made.d / made.D));
  }
};
struct BlockFor {
  etr_block_buffers buf;
  etr_norm_config made;
  int32_t device;
  bool fits(const etr_norm_config& n) const { return made.T == n.T && made.d == n.d && made.dtype == n.dtype; }
};

constexpr int MOST = 20;
struct Arg { const char* name; Kind kind; bool optional; };
struct Op { const char* name; Config config; int n; Arg arg[MOST]; };

constexpr bool OPT = true, NEED = false;
const Op OPS[] = {
    {"etr_sort", SORT, 2, {{"topk_idx", I32_TK, NEED}, {"plan", PLAN, NEED}}},
    {"etr_sort_rows", SORT, 3, {{"X", ACT_TD, NEED}, {"plan", PLAN, NEED}, {"Xs", ACT_RD, NEED}}},
    {"etr_sort_rows_bwd", SORT, 3, {{"dXs", ACT_RD, NEED}, {"plan", PLAN, NEED}, {"dX", ACT_TD, NEED}}},
    {"etr_unsort_rows", SORT, 4, {{"O", ACT_RD, NEED}, {"weights", F32_TK, NEED}, {"plan", PLAN, NEED}, {"Y", ACT_TD, NEED}}},
    {"etr_unsort_rows_bwd", SORT, 6, {{"dY", ACT_TD, NEED}, {"O", ACT_RD, NEED}, {"weights", F32_TK, NEED}, {"plan", PLAN, NEED},
                                      {"dO", ACT_RD, NEED}, {"dweights", F32_TK, NEED}}},
    {"etr_prenorm", NORM, 4, {{"X", ACT_TD, NEED}, {"w", F32_D, OPT}, {"N", ACT_TD, NEED}, {"rstd", F32_T, OPT}}},
    {"etr_prenorm_bwd", NORM, 8, {{"dN", ACT_TD, NEED}, {"X", ACT_TD, NEED}, {"w", F32_D, OPT}, {"rstd", F32_T, NEED}, {"dres", ACT_TD, OPT},
                                   {"dX", ACT_TD, NEED}, {"dw", F32_D, OPT}, {"ws", SCRATCH, OPT}}},
    {"etr_join", NORM, 9, {{"X", ACT_TD, NEED}, {"Y", ACT_TD, NEED}, {"w_post", F32_D, OPT}, {"gate", F32_T, OPT}, {"w_next", F32_D, OPT},
                            {"Xo", ACT_TD, NEED}, {"N", ACT_TD, OPT}, {"rstd_y", F32_T, OPT}, {"rstd_o", F32_T, OPT}}},
    {"etr_join_bwd", NORM, 15, {{"dXo", ACT_TD, OPT}, {"dN", ACT_TD, OPT}, {"Y", ACT_TD, NEED}, {"Xo", ACT_TD, OPT}, {"w_post", F32_D, OPT},
                                 {"gate", F32_T, OPT}, {"w_next", F32_D, OPT}, {"rstd_y", F32_T, OPT}, {"rstd_o", F32_T, OPT},
                                 {"dX", ACT_TD, NEED}, {"dY", ACT_TD, NEED}, {"dw_post", F32_D, OPT}, {"dgate", F32_T, OPT},
                                 {"dw_next", F32_D, OPT}, {"ws", SCRATCH, OPT}}},
    {"etr_routed_forward", LAYER, 9, {{"X", ACT_TD, NEED}, {"topk_idx", I32_TK, NEED}, {"weights", F32_TK, NEED}, {"W1g", W_EHD, NEED},
                                      {"W1u", W_EHD, NEED}, {"W2", W_EHD, NEED}, {"buf", LAYER_BUF, NEED}, {"plan", PLAN, NEED},
                                      {"Y", ACT_TD, NEED}}},
    {"etr_routed_backward", LAYER, 12, {{"weights", F32_TK, NEED}, {"W1g", W_EHD, NEED}, {"W1u", W_EHD, NEED}, {"W2", W_EHD, NEED},
                                        {"dY", ACT_TD, NEED}, {"buf", LAYER_BUF, NEED}, {"plan", PLAN, NEED}, {"dX", ACT_TD, NEED},
                                        {"dweights", F32_TK, NEED}, {"dW1g", G_EHD, NEED}, {"dW1u", G_EHD, NEED}, {"dW2", G_EHD, NEED}}},
    {"etr_block_forward", LAYER, 12, {{"ncfg", NORM_CFG, NEED}, {"X", ACT_TD, NEED}, {"w_pre", F32_D, OPT}, {"w_post", F32_D, OPT},
                                      {"gate", F32_T, OPT}, {"R", F32_EM, NEED}, {"W1g", W_EHD, NEED}, {"W1u", W_EHD, NEED},
                                      {"W2", W_EHD, NEED}, {"buf", LAYER_BUF, NEED}, {"bb", BLOCK_BUF, NEED}, {"Xo", ACT_TD, NEED}}},
    {"etr_block_backward", LAYER, 20, {{"ncfg", NORM_CFG, NEED}, {"X", ACT_TD, NEED}, {"w_pre", F32_D, OPT}, {"w_post", F32_D, OPT},
                                       {"gate", F32_T, OPT}, {"R", F32_EM, NEED}, {"W1g", W_EHD, NEED}, {"W1u", W_EHD, NEED},
                                       {"W2", W_EHD, NEED}, {"dXo", ACT_TD, NEED}, {"buf", LAYER_BUF, NEED}, {"bb", BLOCK_BUF, NEED},
                                       {"dX", ACT_TD, NEED}, {"dw_pre", F32_D, OPT}, {"dw_post", F32_D, OPT}, {"dgate", F32_T, OPT},
                                       {"dR", F32_EM, NEED}, {"dW1g", G_EHD, NEED}, {"dW1u", G_EHD, NEED}, {"dW2", G_EHD, NEED}}},
};
constexpr int N_OPS = sizeof(OPS) / sizeof(OPS[0]);

void* g_fn[N_OPS];
int64_t (*g_n_rows)(const etr_sort_config*);
etr_status (*g_ws_bytes)(const etr_norm_config*, size_t*);
etr_status (*g_validate)(const etr_config*);

PyObject* refuse(int code, const Op& op, const Arg& a, const char* what) {
  PyObject* said = PyUnicode_FromFormat("%s: %s: %s", op.name, a.name, what);
  return said ? Py_BuildValue("(iN)", code, said) : nullptr;
}

template <size_t>
using Ptr = void*;
template <size_t... I>
etr_status with(void* fn, const void* cfg, void* const* a, void* st, std::index_sequence<I...>) {
  return reinterpret_cast<etr_status (*)(const void*, Ptr<I>..., void*)>(fn)(cfg, a[I]..., st);
}
template <size_t N>
etr_status with(void* fn, const void* cfg, void* const* a, void* st) { return with(fn, cfg, a, st, std::make_index_sequence<N>()); }
etr_status call(void* fn, int n, const void* c, void* const* a, void* st) {
  switch (n) {
    case 2: return with<2>(fn, c, a, st);
    case 3: return with<3>(fn, c, a, st);
    case 4: return with<4>(fn, c, a, st);
    case 6: return with<6>(fn, c, a, st);
    case 8: return with<8>(fn, c, a, st);
    case 9: return with<9>(fn, c, a, st);
    case 12: return with<12>(fn, c, a, st);
    case 15: return with<15>(fn, c, a, st);
    case 20: return with<20>(fn, c, a, st);
  }
  return ETR_ERR_ARG;
}

// What a call's configuration says of its tensors.
struct Sizes {
  int64_t T, d, k, weight, pooled;                 // weight: E h d; pooled: E m
  at::ScalarType act, weights, grads;
  etr_sort_config sort;                            // of the plan
};
at::ScalarType type_of(int dtype) { return dtype == ETR_BF16 ? at::kBFloat16 : at::kFloat; }
Sizes sizes_of(Config kind, const void* cfg) {
  Sizes z = {};
  if (kind == SORT) {
    z.sort = *static_cast<const etr_sort_config*>(cfg);
    z.T = z.sort.T; z.d = z.sort.d; z.k = z.sort.k; z.act = type_of(z.sort.dtype);
  } else if (kind == NORM) {
    const auto& m = *static_cast<const etr_norm_config*>(cfg);
    z.T = m.T; z.d = m.d; z.act = type_of(m.dtype);
  } else {
    const auto& c = *static_cast<const etr_config*>(cfg);
    z.T = c.T; z.d = c.d; z.k = c.k;
    z.weight = (int64_t)c.E * c.h * c.d;
    z.pooled = (int64_t)c.E * (c.d / c.D);
    z.act = type_of(c.dtype);
    z.weights = type_of(c.weight_dtype);
    z.grads = c.grad_fp32 || c.weight_dtype != c.dtype ? at::kFloat : z.act;
    z.sort = etr_sort_config{c.T, c.k, c.E, c.d, c.dtype, 128, c.capacity, 0};
  }
  return z;
}
int64_t count_of(Kind kind, const Sizes& z) {
  switch (kind) {
    case ACT_TD: return z.T * z.d;
    case ACT_RD: return g_n_rows(&z.sort) * z.d;
    case F32_D: return z.d;
    case F32_T: return z.T;
    case F32_EM: return z.pooled;
    case W_EHD:
    case G_EHD: return z.weight;
    default: return z.T * z.k;
  }
}
at::ScalarType type_of(Kind kind, const Sizes& z) {
  switch (kind) {
    case ACT_TD:
    case ACT_RD: return z.act;
    case W_EHD: return z.weights;
    case G_EHD: return z.grads;
    case I32_TK: return at::kInt;
    default: return at::kFloat;
  }
}

// Other Python threads run during a call, as they do under ctypes: a launch can wait for a full queue or for a module to load.
struct Unlocked {
  PyThreadState* const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

// run(op, config address, arguments...): 0, or (status, what was wrong).  Handles are addresses of PlanFor, LayerFor, BlockFor and of a
// norm's configuration; they are looked over before the tensors, since the kernels write through their addresses.  Nothing
// here allocates or waits.
PyObject* run(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  try {
    const long i = nargs >= 2 ? PyLong_AsLong(args[0]) : -1;
    if (i < 0 || i >= N_OPS || nargs != 2 + OPS[i].n) {
      PyErr_SetString(PyExc_TypeError, "run(op, config, arguments...)");
      return nullptr;
    }
    const Op& op = OPS[i];
    const void* cfg = PyLong_AsVoidPtr(args[1]);
    if (PyErr_Occurred()) return nullptr;
    args += 2;
    if (op.config == LAYER) {
      const etr_status code = g_validate(static_cast<const etr_config*>(cfg));
      if (code != ETR_OK) return Py_BuildValue("(is)", code, op.name);
    }
    const Sizes z = sizes_of(op.config, cfg);
    void* a[MOST];
    int on[MOST];                                  // a handle's device
    for (int j = 0; j < op.n; ++j) {
      const Arg& w = op.arg[j];
      if (w.kind < PLAN) continue;
      void* p = a[j] = PyLong_AsVoidPtr(args[j]);      // each For starts with the struct that the C function takes
      if (PyErr_Occurred()) return nullptr;
      bool fits = true;
      if (w.kind == PLAN) {
        fits = static_cast<PlanFor*>(p)->fits(z.sort);
        on[j] = static_cast<PlanFor*>(p)->device;
      } else if (w.kind == LAYER_BUF) {
        fits = static_cast<LayerFor*>(p)->fits(*static_cast<const etr_config*>(cfg), op.arg[0].kind == NORM_CFG);
        on[j] = static_cast<LayerFor*>(p)->device;
      } else if (w.kind == BLOCK_BUF) {
        fits = static_cast<BlockFor*>(p)->fits(*static_cast<const etr_norm_config*>(a[0]));
        on[j] = static_cast<BlockFor*>(p)->device;
      }
      if (!fits) return refuse(ETR_ERR_WORKSPACE, op, w, "made for another configuration");
    }
    int device = -1;
    for (int j = 0; j < op.n; ++j) {
      const Arg& w = op.arg[j];
      if (w.kind < PLAN || w.kind == NORM_CFG) continue;
      if (on[j] < 0) return refuse(ETR_ERR_ARG, op, w, "not on a CUDA device");
      if (device < 0) device = on[j];
      if (on[j] != device) return refuse(ETR_ERR_ARG, op, w, "on another device than the buffers before it");
    }
    for (int j = 0; j < op.n; ++j) {
      PyObject* o = args[j];
      const Arg& w = op.arg[j];
      if (w.kind >= PLAN) continue;
      if (o == Py_None) {
        if (!w.optional) return refuse(ETR_ERR_ARG, op, w, "a tensor is wanted");
        a[j] = nullptr;
        continue;
      }
      if (!THPVariable_Check(o)) return refuse(ETR_ERR_ARG, op, w, "a tensor is wanted");
      const at::Tensor& t = THPVariable_Unpack(o);
      if (!t.is_cuda()) return refuse(ETR_ERR_ARG, op, w, "not on a CUDA device");
      if (device < 0) device = t.get_device();
      if (t.get_device() != device) return refuse(ETR_ERR_ARG, op, w, "on another device than the tensors before it");
      if (!t.is_contiguous()) return refuse(ETR_ERR_SHAPE, op, w, "not contiguous");
      if (w.kind == SCRATCH) {
        size_t need = 0;
        const etr_status code = g_ws_bytes(static_cast<const etr_norm_config*>(cfg), &need);
        if (code != ETR_OK) return refuse(code, op, w, "configuration");
        if (t.nbytes() < need) return refuse(ETR_ERR_WORKSPACE, op, w, "too small");
      } else {
        if (t.scalar_type() != type_of(w.kind, z)) return refuse(ETR_ERR_ARG, op, w, "of another type");
        if (t.numel() != count_of(w.kind, z)) return refuse(ETR_ERR_SHAPE, op, w, "of another size");
      }
      a[j] = t.data_ptr();
    }
    if (device < 0) return Py_BuildValue("(is)", ETR_ERR_ARG, op.name);
    if (device != c10::cuda::current_device()) return Py_BuildValue("(is)", ETR_ERR_ARG, "tensors on another than the current device");
    void* const stream = c10::cuda::getCurrentCUDAStream(device).stream();
    etr_status code;
    {
      const Unlocked meanwhile;
      code = call(g_fn[i], op.n, cfg, a, stream);
    }
    return code == ETR_OK ? PyLong_FromLong(0) : Py_BuildValue("(is)", code, op.name);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// bind(addresses of the functions in `names`, of etr_sort_n_rows, etr_norm_workspace_bytes and etr_validate)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != N_OPS + 3) {
    PyErr_SetString(PyExc_TypeError, "bind(addresses...)");
    return nullptr;
  }
  for (int i = 0; i < N_OPS; ++i) g_fn[i] = PyLong_AsVoidPtr(args[i]);
  g_n_rows = reinterpret_cast<decltype(g_n_rows)>(PyLong_AsVoidPtr(args[N_OPS]));
  g_ws_bytes = reinterpret_cast<decltype(g_ws_bytes)>(PyLong_AsVoidPtr(args[N_OPS + 1]));
  g_validate = reinterpret_cast<decltype(g_validate)>(PyLong_AsVoidPtr(args[N_OPS + 2]));
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

PyMethodDef METHODS[] = {{"run", (PyCFunction)(void*)run, METH_FASTCALL, nullptr}, {"bind", (PyCFunction)(void*)bind, METH_FASTCALL, nullptr}, {}};
PyModuleDef MODULE = {PyModuleDef_HEAD_INIT, "_args", nullptr, -1, METHODS};

}  // namespace

PyMODINIT_FUNC PyInit__args() {
  PyObject* m = PyModule_Create(&MODULE);
  if (m == nullptr) return nullptr;
  PyObject* names = PyTuple_New(N_OPS);
  for (int i = 0; names && i < N_OPS; ++i) PyTuple_SET_ITEM(names, i, PyUnicode_FromString(OPS[i].name));
  if (names == nullptr || PyModule_AddObject(m, "names", names) < 0) return nullptr;
  return m;
}
