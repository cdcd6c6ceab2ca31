// Argument marshalling of the row operators (tokens sorted by a given choice, norms around a block) for Python: a call of a few
// microseconds on the GPU should not wait for as many of attribute look-ups.  Checks what addresses alone do not show
// (type, place, order and size of every tensor), takes the current stream, and calls the C function with plain pointers.
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/etr.h"

namespace {

enum Kind { ACT_TD, ACT_RD, F32_D, F32_T, F32_TK, I32_TK, PLAN, SCRATCH };     // R: rows of the sorted buffers
// A plan and the configuration that its memory was carved for (d and dtype do not matter to it).
struct PlanFor {
  etr_sort_plan plan;
  etr_sort_config made;
  bool fits(const etr_sort_config& c) const {
    return made.T == c.T && made.k == c.k && made.E == c.E && made.align == c.align && made.capacity == c.capacity;
  }
};
struct Arg { const char* name; Kind kind; bool optional; };
struct Op { const char* name; bool sort; int n; Arg arg[15]; };

constexpr bool OPT = true, NEED = false;
const Op OPS[] = {
    {"etr_sort", true, 2, {{"topk_idx", I32_TK, NEED}, {"plan", PLAN, NEED}}},
    {"etr_sort_rows", true, 3, {{"X", ACT_TD, NEED}, {"plan", PLAN, NEED}, {"Xs", ACT_RD, NEED}}},
    {"etr_sort_rows_bwd", true, 3, {{"dXs", ACT_RD, NEED}, {"plan", PLAN, NEED}, {"dX", ACT_TD, NEED}}},
    {"etr_unsort_rows", true, 4, {{"O", ACT_RD, NEED}, {"weights", F32_TK, NEED}, {"plan", PLAN, NEED}, {"Y", ACT_TD, NEED}}},
    {"etr_unsort_rows_bwd", true, 6, {{"dY", ACT_TD, NEED}, {"O", ACT_RD, NEED}, {"weights", F32_TK, NEED}, {"plan", PLAN, NEED},
                                      {"dO", ACT_RD, NEED}, {"dweights", F32_TK, NEED}}},
    {"etr_prenorm", false, 4, {{"X", ACT_TD, NEED}, {"w", F32_D, OPT}, {"N", ACT_TD, NEED}, {"rstd", F32_T, OPT}}},
    {"etr_prenorm_bwd", false, 8, {{"dN", ACT_TD, NEED}, {"X", ACT_TD, NEED}, {"w", F32_D, OPT}, {"rstd", F32_T, NEED}, {"dres", ACT_TD, OPT},
                                   {"dX", ACT_TD, NEED}, {"dw", F32_D, OPT}, {"ws", SCRATCH, OPT}}},
    {"etr_join", false, 9, {{"X", ACT_TD, NEED}, {"Y", ACT_TD, NEED}, {"w_post", F32_D, OPT}, {"gate", F32_T, OPT}, {"w_next", F32_D, OPT},
                            {"Xo", ACT_TD, NEED}, {"N", ACT_TD, OPT}, {"rstd_y", F32_T, OPT}, {"rstd_o", F32_T, OPT}}},
    {"etr_join_bwd", false, 15, {{"dXo", ACT_TD, OPT}, {"dN", ACT_TD, OPT}, {"Y", ACT_TD, NEED}, {"Xo", ACT_TD, OPT}, {"w_post", F32_D, OPT},
                                 {"gate", F32_T, OPT}, {"w_next", F32_D, OPT}, {"rstd_y", F32_T, OPT}, {"rstd_o", F32_T, OPT},
                                 {"dX", ACT_TD, NEED}, {"dY", ACT_TD, NEED}, {"dw_post", F32_D, OPT}, {"dgate", F32_T, OPT},
                                 {"dw_next", F32_D, OPT}, {"ws", SCRATCH, OPT}}},
};
constexpr int N_OPS = sizeof(OPS) / sizeof(OPS[0]);

void* g_fn[N_OPS];
int64_t (*g_n_rows)(const etr_sort_config*);
etr_status (*g_ws_bytes)(const etr_norm_config*, size_t*);

PyObject* refuse(int code, const Op& op, const Arg& a, const char* what) {
  PyObject* said = PyUnicode_FromFormat("%s: %s: %s", op.name, a.name, what);
  return said ? Py_BuildValue("(iN)", code, said) : nullptr;
}

template <class... P>
etr_status with(void* fn, const void* cfg, void* st, P... p) {
  return reinterpret_cast<etr_status (*)(const void*, P..., void*)>(fn)(cfg, p..., st);
}
etr_status call(void* fn, int n, const void* c, void* const* a, void* st) {
  switch (n) {
    case 2: return with(fn, c, st, a[0], a[1]);
    case 3: return with(fn, c, st, a[0], a[1], a[2]);
    case 4: return with(fn, c, st, a[0], a[1], a[2], a[3]);
    case 6: return with(fn, c, st, a[0], a[1], a[2], a[3], a[4], a[5]);
    case 8: return with(fn, c, st, a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]);
    case 9: return with(fn, c, st, a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8]);
    case 15: return with(fn, c, st, a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11], a[12], a[13], a[14]);
  }
  return ETR_ERR_ARG;
}

// run(op, config address, device, arguments...): 0, or (status, what was wrong).  Plans are addresses of PlanFor; `device` is
// the one that the plan's memory is on (-1: not a GPU), and -1 where the operator takes no plan.  The plan is looked over
// before the tensors: the kernels write through its addresses.  Nothing here allocates or waits.
PyObject* run(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  try {
    const long i = nargs >= 3 ? PyLong_AsLong(args[0]) : -1;
    if (i < 0 || i >= N_OPS || nargs != 3 + OPS[i].n) {
      PyErr_SetString(PyExc_TypeError, "run(op, config, device, arguments...)");
      return nullptr;
    }
    const Op& op = OPS[i];
    const void* cfg = PyLong_AsVoidPtr(args[1]);
    int device = (int)PyLong_AsLong(args[2]);
    if (PyErr_Occurred()) return nullptr;
    const auto* s = static_cast<const etr_sort_config*>(cfg);
    const auto* m = static_cast<const etr_norm_config*>(cfg);
    const int64_t T = op.sort ? s->T : m->T, d = op.sort ? s->d : m->d;
    const auto act = (op.sort ? s->dtype : m->dtype) == ETR_BF16 ? at::kBFloat16 : at::kFloat;
    void* a[15];
    for (int j = 0; j < op.n; ++j) {
      const Arg& w = op.arg[j];
      if (w.kind != PLAN) continue;
      auto* p = static_cast<PlanFor*>(PyLong_AsVoidPtr(args[3 + j]));
      if (PyErr_Occurred()) return nullptr;
      if (p == nullptr || !p->fits(*s)) return refuse(ETR_ERR_WORKSPACE, op, w, "made for another configuration");
      if (device < 0) return refuse(ETR_ERR_ARG, op, w, "not on a CUDA device");
      a[j] = &p->plan;
    }
    for (int j = 0; j < op.n; ++j) {
      PyObject* o = args[3 + j];
      const Arg& w = op.arg[j];
      if (w.kind == PLAN) continue;
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
        const etr_status code = g_ws_bytes(m, &need);
        if (code != ETR_OK) return refuse(code, op, w, "configuration");
        if (t.nbytes() < need) return refuse(ETR_ERR_WORKSPACE, op, w, "too small");
      } else {
        const bool is_act = w.kind == ACT_TD || w.kind == ACT_RD;
        if (t.scalar_type() != (is_act ? act : w.kind == I32_TK ? at::kInt : at::kFloat)) return refuse(ETR_ERR_ARG, op, w, "of another type");
        int64_t n = 0;
        switch (w.kind) {
          case ACT_TD: n = T * d; break;
          case ACT_RD: n = g_n_rows(s) * d; break;
          case F32_D: n = d; break;
          case F32_T: n = T; break;
          default: n = T * s->k;
        }
        if (t.numel() != n) return refuse(ETR_ERR_SHAPE, op, w, "of another size");
      }
      a[j] = t.data_ptr();
    }
    if (device < 0) return Py_BuildValue("(is)", ETR_ERR_ARG, op.name);
    if (device != c10::cuda::current_device()) return Py_BuildValue("(is)", ETR_ERR_ARG, "tensors on another than the current device");
    const etr_status code = call(g_fn[i], op.n, cfg, a, c10::cuda::getCurrentCUDAStream(device).stream());
    return code == ETR_OK ? PyLong_FromLong(0) : Py_BuildValue("(is)", code, op.name);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// bind(addresses of the functions in `names`, of etr_sort_n_rows, of etr_norm_workspace_bytes)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != N_OPS + 2) {
    PyErr_SetString(PyExc_TypeError, "bind(addresses...)");
    return nullptr;
  }
  for (int i = 0; i < N_OPS; ++i) g_fn[i] = PyLong_AsVoidPtr(args[i]);
  g_n_rows = reinterpret_cast<decltype(g_n_rows)>(PyLong_AsVoidPtr(args[N_OPS]));
  g_ws_bytes = reinterpret_cast<decltype(g_ws_bytes)>(PyLong_AsVoidPtr(args[N_OPS + 1]));
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
