// Argument marshalling of the operators around the head, for the Python binding: checks tensors, fills the C ABI's
// argument tables and allocates the outputs.  A decoding step calls several of these for every token, and a
// list of some hundred gradients or caches costs the interpreter more time than the GPU needs for them.
// Nothing is computed here; the entry points of libprunedctc are handed in by address (bind).
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <vector>

#include "../../include/prunedctc.h"

namespace {

struct {
  decltype(&pctc_clip_workspace_bytes) clip_workspace_bytes;
  decltype(&pctc_clip_grad_norm) clip_grad_norm;
  decltype(&pctc_grad_sqsum) grad_sqsum;
  decltype(&pctc_grad_scale) grad_scale;
  decltype(&pctc_beam_workspace_bytes) beam_workspace_bytes;
  decltype(&pctc_beam_select) beam_select;
  decltype(&pctc_beam_reorder) beam_reorder;
  decltype(&pctc_prefix_state_bytes) prefix_state_bytes;
  decltype(&pctc_prefix_advance) prefix_advance;
  decltype(&pctc_prefix_read) prefix_read;
  decltype(&pctc_prefix_decode) prefix_decode;
} api;
PyObject* error_type = nullptr;       // PctcError(status, what)

// The Python error is set already.
struct Failed {};

template <typename... Args>
[[noreturn]] void fail(PyObject* type, const char* format, Args... args) {
  PyErr_Format(type, format, args...);
  throw Failed{};
}

void check(pctc_status_t st, const char* what) {
  if (st == PCTC_OK) return;
  PyObject* e = PyObject_CallFunction(error_type, "is", (int)st, what);
  if (e) {
    PyErr_SetObject(error_type, e);
    Py_DECREF(e);
  }
  throw Failed{};
}

#define MARSHAL_BEGIN HANDLE_TH_ERRORS try {
#define MARSHAL_END                          \
  }                                          \
  catch (const Failed&) {                    \
    return nullptr;                          \
  }                                          \
  END_HANDLE_TH_ERRORS

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s must be a tensor", what);
  const at::Tensor& t = THPVariable_Unpack(o);
  // the memory of such a view holds other values than the view
  if (t.is_conj() || t.is_neg())
    fail(PyExc_ValueError, "%s must not be a lazily conjugated or negated view (resolve_conj, resolve_neg)", what);
  return t;
}
at::Tensor optional_tensor(PyObject* o, const char* what) { return o == Py_None ? at::Tensor() : tensor(o, what); }

void want(Py_ssize_t got, Py_ssize_t n) {
  if (got != n) fail(PyExc_TypeError, "%d arguments expected, got %d", (int)n, (int)got);
}
long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Failed{};
  return v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Failed{};
  return v;
}

at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, at::Device dev) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
}
// Contiguous tensors that share one allocation: a decoding step's outputs cost the allocator one visit.
class Shared {
 public:
  explicit Shared(at::Device dev) : dev_(dev) {}
  size_t add(at::IntArrayRef shape, at::ScalarType type) {
    int64_t n = 1;
    for (const int64_t s : shape) n *= s;
    parts_.push_back(Part{shape.vec(), type, bytes_});
    bytes_ += ((int64_t)(n * c10::elementSize(type)) + 15) / 16 * 16;
    return parts_.size() - 1;
  }
  void allocate() { base_ = empty({std::max<int64_t>(bytes_, 1)}, at::kByte, dev_); }
  at::Tensor get(size_t i) const {
    const Part& p = parts_[i];
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(base_.storage()), base_.key_set(),
                                                            c10::scalarTypeToTypeMeta(p.type));
    t.unsafeGetTensorImpl()->set_storage_offset(base_.storage_offset() + p.at / (int64_t)c10::elementSize(p.type));
    t.unsafeGetTensorImpl()->set_sizes_contiguous(p.shape);
    return t;
  }

 private:
  struct Part {
    std::vector<int64_t> shape;
    at::ScalarType type;
    int64_t at;
  };
  at::Device dev_;
  std::vector<Part> parts_;
  int64_t bytes_ = 0;
  at::Tensor base_;
};

void* stream_of(at::Device dev) { return c10::cuda::getCurrentCUDAStream(dev.index()).stream(); }
void* ptr(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
// A tensor of the caller's that has been written to counts up, as by torch's own in-place operations, so that a backward
// pass that has saved it does not go on with other values.
void written(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void written(PyObject* list) {
  for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) written(THPVariable_Unpack(PyList_GET_ITEM(list, i)));
}

// ---- gradients ----

struct Grads {
  at::Device dev = at::Device(at::kCPU);
  std::vector<void*> ptrs;
  std::vector<int64_t> numels;
  std::vector<int32_t> kinds;
  int n() const { return (int)ptrs.size(); }
};
Grads read_grads(PyObject* list, const char* what) {
  const Py_ssize_t n = PyList_GET_SIZE(list);
  if (n == 0) fail(PyExc_ValueError, "%s must hold at least one tensor", what);
  Grads g;
  g.ptrs.reserve(n);
  g.numels.reserve(n);
  g.kinds.reserve(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor& t = tensor(PyList_GET_ITEM(list, i), what);
    if (i == 0) g.dev = t.device();
    if (!t.is_cuda() || t.device() != g.dev) fail(PyExc_ValueError, "%s must be CUDA tensors of one device", what);
    if (t.scalar_type() != at::kBFloat16 && t.scalar_type() != at::kFloat)
      fail(PyExc_ValueError, "%s must be bf16 or fp32", what);
    if (!t.is_contiguous()) fail(PyExc_ValueError, "%s must be contiguous", what);
    g.ptrs.push_back(t.data_ptr());
    g.numels.push_back(t.numel());
    g.kinds.push_back(t.scalar_type() == at::kFloat ? PCTC_FP32 : PCTC_BF16);
  }
  return g;
}
// out: None (in place) or one tensor of the same shape for every gradient
Grads read_outs(PyObject* out, PyObject* grads, const Grads& g) {
  if (out == Py_None) return Grads();
  if (PyList_GET_SIZE(out) != g.n()) fail(PyExc_ValueError, "out must hold one tensor of the same shape for every gradient");
  Grads o = read_grads(out, "out");
  for (int i = 0; i < g.n(); ++i)
    if (!tensor(PyList_GET_ITEM(out, i), "out").sizes().equals(tensor(PyList_GET_ITEM(grads, i), "grads").sizes()))
      fail(PyExc_ValueError, "out must hold one tensor of the same shape for every gradient");
  if (o.dev != g.dev) fail(PyExc_ValueError, "out must be on the gradients' device");
  return o;
}
at::Tensor workspace_for(const Grads& g, PyObject* given) {
  size_t need = 0;
  check(api.clip_workspace_bytes(g.n(), &need), "pctc_clip_workspace_bytes");
  at::Tensor w = optional_tensor(given, "workspace");
  if (w.defined() && (w.device() != g.dev || w.scalar_type() != at::kByte || !w.is_contiguous()))
    fail(PyExc_ValueError, "workspace must be contiguous bytes on the gradients' device");
  return w.defined() && (size_t)w.numel() >= need ? w : empty({(int64_t)need}, at::kByte, g.dev);
}

PyObject* pair(const at::Tensor& a, const at::Tensor& b) {
  PyObject* t = PyTuple_New(2);
  if (!t) return nullptr;
  PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(a));
  PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(b));
  return t;
}

// clip_grad_norm(grads, out, max_norm, eps, workspace) -> (norm, workspace)
PyObject* clip_grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 5);
  const Grads g = read_grads(a[0], "grads"), o = read_outs(a[1], a[0], g);
  const double max_norm = real(a[2]), eps = real(a[3]);
  const c10::cuda::CUDAGuard guard(g.dev);
  const at::Tensor ws = workspace_for(g, a[4]), norm = empty({1}, at::kFloat, g.dev);
  check(api.clip_grad_norm(g.n(), g.ptrs.data(), o.n() ? o.ptrs.data() : nullptr, g.numels.data(), g.kinds.data(),
                           o.n() ? o.kinds.data() : nullptr, (float)max_norm, (float)eps, (float*)ptr(norm), ptr(ws),
                           (size_t)ws.numel(), stream_of(g.dev)),
        "pctc_clip_grad_norm");
  written(a[1] == Py_None ? a[0] : a[1]);
  return pair(norm, ws);
  MARSHAL_END
}
// grad_sqsum(grads, workspace) -> (sqsum, workspace)
PyObject* grad_sqsum(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 2);
  const Grads g = read_grads(a[0], "grads");
  const c10::cuda::CUDAGuard guard(g.dev);
  const at::Tensor ws = workspace_for(g, a[1]), sq = empty({1}, at::kDouble, g.dev);
  check(api.grad_sqsum(g.n(), g.ptrs.data(), g.numels.data(), g.kinds.data(), (double*)ptr(sq), ptr(ws),
                       (size_t)ws.numel(), stream_of(g.dev)),
        "pctc_grad_sqsum");
  return pair(sq, ws);
  MARSHAL_END
}
// grad_scale(grads, out, sqsum, max_norm, eps) -> norm
PyObject* grad_scale(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 5);
  const Grads g = read_grads(a[0], "grads"), o = read_outs(a[1], a[0], g);
  const at::Tensor& sq = tensor(a[2], "sqsum");
  if (sq.scalar_type() != at::kDouble || sq.numel() != 1 || sq.device() != g.dev)
    fail(PyExc_ValueError, "sqsum must be one fp64 value on the gradients' device");
  const double max_norm = real(a[3]), eps = real(a[4]);
  const c10::cuda::CUDAGuard guard(g.dev);
  const at::Tensor norm = empty({1}, at::kFloat, g.dev);
  check(api.grad_scale(g.n(), g.ptrs.data(), o.n() ? o.ptrs.data() : nullptr, g.numels.data(), g.kinds.data(),
                       o.n() ? o.kinds.data() : nullptr, (const double*)ptr(sq), (float)max_norm, (float)eps,
                       (float*)ptr(norm), stream_of(g.dev)),
        "pctc_grad_scale");
  written(a[1] == Py_None ? a[0] : a[1]);
  return THPVariable_Wrap(norm);
  MARSHAL_END
}

// ---- beams ----

void put(PyObject* dict, const char* key, const at::Tensor& t) {
  PyObject* v = THPVariable_Wrap(t);
  if (!v || PyDict_SetItemString(dict, key, v) != 0) {
    Py_XDECREF(v);
    Py_DECREF(dict);
    throw Failed{};
  }
  Py_DECREF(v);
}

// beam_select(logits, scores, beams, finished, eos_id or None) -> dict
PyObject* beam_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 5);
  const at::Tensor& x = tensor(a[0], "logits");
  const at::Tensor& s = tensor(a[1], "scores");
  if (x.dim() != 3 || (x.scalar_type() != at::kBFloat16 && x.scalar_type() != at::kFloat))
    fail(PyExc_ValueError, "logits must be [N, B, V], bf16 or fp32");
  const int64_t N = x.size(0), B = x.size(1), V = x.size(2), K = integer(a[2]);
  if (!x.is_cuda() || (V > 1 && x.stride(2) != 1)) fail(PyExc_ValueError, "logits must be a CUDA tensor with contiguous rows");
  const at::Device dev = x.device();
  if (s.scalar_type() != at::kFloat || s.dim() != 2 || s.size(0) != N || s.size(1) != B || !s.is_contiguous() || s.device() != dev)
    fail(PyExc_ValueError, "scores must be contiguous fp32 [N, B] on the device of the logits");
  const at::Tensor f = optional_tensor(a[3], "finished");
  const int64_t eos = a[4] == Py_None ? -1 : integer(a[4]);
  if (f.defined()) {
    if (f.scalar_type() != at::kBool || f.dim() != 2 || f.size(0) != N || f.size(1) != B || !f.is_contiguous() || f.device() != dev)
      fail(PyExc_ValueError, "finished must be contiguous bool [N, B] on the device of the logits");
    if (a[4] == Py_None) fail(PyExc_ValueError, "finished needs an eos_id");
  }
  if (a[4] != Py_None && !(0 <= eos && eos < V)) fail(PyExc_ValueError, "eos_id must be a token");
  if (K < 1) fail(PyExc_ValueError, "beams must be at least 1");
  if (B > 1 && x.stride(1) < V) fail(PyExc_ValueError, "rows of logits overlap");
  pctc_beam_t p;                        // a dimension of size 1 has no stride that counts
  if (N > INT32_MAX || B > INT32_MAX || K > INT32_MAX) check(PCTC_ERR_UNSUPPORTED, "pctc_beam_select");
  p.N = (int32_t)N; p.B = (int32_t)B; p.K = (int32_t)K; p.V = V;
  p.stride_n = N > 1 ? x.stride(0) : 0;
  p.stride_b = B > 1 ? x.stride(1) : V;
  p.dtype = x.scalar_type() == at::kFloat ? PCTC_FP32 : PCTC_BF16;
  p.eos_id = (int32_t)eos;
  const c10::cuda::CUDAGuard guard(dev);
  size_t need = 0;
  check(api.beam_workspace_bytes(&p, &need), "pctc_beam_workspace_bytes");
  Shared out(dev);
  for (const at::ScalarType type : {at::kFloat, at::kInt, at::kInt, at::kBool}) out.add({N, K}, type);
  out.add({N}, at::kInt);
  out.allocate();
  const at::Tensor scores = out.get(0), parents = out.get(1), tokens = out.get(2), finished = out.get(3), flags = out.get(4);
  const at::Tensor ws = empty({(int64_t)need}, at::kByte, dev);
  check(api.beam_select(&p, ptr(x), (const float*)ptr(s), (const uint8_t*)ptr(f), (float*)ptr(scores),
                        (int32_t*)ptr(parents), (int32_t*)ptr(tokens), (uint8_t*)ptr(finished), (int32_t*)ptr(flags),
                        ptr(ws), need, stream_of(dev)),
        "pctc_beam_select");
  PyObject* d = PyDict_New();
  if (!d) return nullptr;
  put(d, "scores", scores);
  put(d, "parents", parents);
  put(d, "tokens", tokens);
  put(d, "finished", finished);
  put(d, "flags", flags);
  return d;
  MARSHAL_END
}

struct Layout {
  int64_t n, b, segments, segment_stride, units, unit;
};
// Layout in bytes of a state [N, B, ...] whose dimensions behind the beams are contiguous.
Layout layout_of(const at::Tensor& x, int64_t axis, const char* what) {
  const int64_t size = (int64_t)x.element_size();
  int64_t inner = 1;
  for (int64_t d = x.dim() - 1; d > 1; --d) {
    if (x.size(d) != 1 && x.stride(d) != inner) fail(PyExc_ValueError, "%s must be contiguous behind the beam dimension", what);
    inner *= x.size(d);
  }
  Layout l{x.stride(0) * size, x.stride(1) * size, 1, 0, 1, inner * size};
  if (axis < 0) return l;
  if (axis < 2 || axis >= x.dim()) fail(PyExc_ValueError, "a time axis lies behind the beam dimension");
  l.unit = size;
  for (int64_t d = axis + 1; d < x.dim(); ++d) l.unit *= x.size(d);
  for (int64_t d = 2; d < axis; ++d) l.segments *= x.size(d);
  l.units = x.size(axis);
  l.segment_stride = l.units * l.unit;
  return l;
}

// beam_reorder(states, parents, lengths, time_axes, out): lists, the last two or None
PyObject* beam_reorder(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 5);
  const Py_ssize_t m = PyList_GET_SIZE(a[0]);
  if (m == 0) fail(PyExc_ValueError, "states must hold at least one tensor");
  const at::Tensor& first = tensor(PyList_GET_ITEM(a[0], 0), "states");
  const at::Device dev = first.device();
  if (!first.is_cuda()) fail(PyExc_ValueError, "states must be CUDA tensors");
  const at::Tensor& parents = tensor(a[1], "parents");
  if (parents.scalar_type() != at::kInt || parents.dim() != 2 || !parents.is_contiguous() || parents.device() != dev)
    fail(PyExc_ValueError, "parents must be contiguous int32 [N, K] on the states' device");
  const int64_t N = parents.size(0), K = parents.size(1), B = first.dim() > 1 ? first.size(1) : 0;
  const bool in_place = a[4] == Py_None;
  if ((!in_place && PyList_GET_SIZE(a[4]) != m) || (a[3] != Py_None && PyList_GET_SIZE(a[3]) != m))
    fail(PyExc_ValueError, "out and time_axes must have one entry for every state");
  const at::Tensor lengths = optional_tensor(a[2], "lengths");
  if (lengths.defined() && (lengths.scalar_type() != at::kInt || lengths.dim() != 1 || lengths.size(0) != N ||
                            !lengths.is_contiguous() || lengths.device() != dev))
    fail(PyExc_ValueError, "lengths must be contiguous int32 [N] on the states' device");
  if (N > INT32_MAX || B > INT32_MAX || K > INT32_MAX) check(PCTC_ERR_UNSUPPORTED, "pctc_beam_reorder");
  std::vector<pctc_beam_state_t> table;
  table.reserve(m);
  for (Py_ssize_t i = 0; i < m; ++i) {
    const at::Tensor& x = tensor(PyList_GET_ITEM(a[0], i), "states");
    const at::Tensor& o = in_place ? x : tensor(PyList_GET_ITEM(a[4], i), "out");
    PyObject* ax = a[3] == Py_None ? Py_None : PyList_GET_ITEM(a[3], i);
    const bool timed = ax != Py_None;
    const int64_t axis = timed ? integer(ax) : -1;
    if (timed && !lengths.defined()) fail(PyExc_ValueError, "a time axis needs lengths");
    if (timed && axis < 0) fail(PyExc_ValueError, "a time axis lies behind the beam dimension");
    if (x.dim() < 2 || x.size(0) != N || x.size(1) != B || x.device() != dev)
      fail(PyExc_ValueError, "states must be [N, B, ...] on one device");
    bool fits = o.dim() == x.dim() && o.size(0) == N && o.size(1) == K && o.scalar_type() == x.scalar_type() && o.device() == dev;
    for (int64_t d = 2; fits && d < x.dim(); ++d) fits = o.size(d) == x.size(d);
    if (!fits)
      fail(PyExc_ValueError, "%s", in_place ? "in place, parents must have as many columns as the states have beams"
                                       : "out must be [N, K, ...] tensors of the states' types");
    if (x.numel() == 0) continue;
    const Layout l = layout_of(x, axis, "states");
    Layout lo = l;
    if (!in_place) lo = layout_of(o, axis, "out");
    table.push_back(pctc_beam_state_t{ptr(x), ptr(o), l.n, l.b, lo.n, lo.b, l.segments, l.segment_stride, l.units, l.unit,
                                      timed ? 1 : 0, 0});
  }
  const c10::cuda::CUDAGuard guard(dev);
  check(api.beam_reorder((int32_t)table.size(), table.data(), (int32_t)N, (int32_t)B, (int32_t)K, (const int32_t*)ptr(parents),
                         (const int32_t*)ptr(lengths), stream_of(dev)),
        "pctc_beam_reorder");
  written(in_place ? a[0] : a[4]);
  Py_RETURN_NONE;
  MARSHAL_END
}

// ---- prefix search ----

pctc_prefix_t prefix_problem(int64_t N, int64_t T, int64_t k, PyObject* beams, PyObject* blank, PyObject* max_frames) {
  const int64_t b = integer(beams), bl = integer(blank), m = integer(max_frames);
  for (const int64_t v : {N, T, k, b, bl, m})
    if (v > INT32_MAX || v < INT32_MIN) check(PCTC_ERR_UNSUPPORTED, "prefix search");
  return pctc_prefix_t{(int32_t)N, (int32_t)T, (int32_t)k, (int32_t)b, (int32_t)bl, (int32_t)m};
}
// The checks of a portion of frames.
void prefix_inputs(const at::Tensor& c, const at::Tensor& l, int64_t N, int64_t index) {
  if (c.scalar_type() != at::kInt || l.scalar_type() != at::kFloat) fail(PyExc_ValueError, "classes must be int32 and logprobs fp32");
  if (c.dim() != 3 || c.size(0) != N || !l.sizes().equals(c.sizes())) fail(PyExc_ValueError, "classes and logprobs must be [N, frames, k]");
  const bool there = index < 0 ? !c.is_cuda() && !l.is_cuda()
                               : c.is_cuda() && l.is_cuda() && c.get_device() == index && l.get_device() == index;
  if (!there) fail(PyExc_ValueError, "classes and logprobs must be on the state's device");
  if (!c.is_contiguous() || !l.is_contiguous()) fail(PyExc_ValueError, "classes and logprobs must be contiguous");
}
// Lengths that are none of 0 .. T become -1, which the C entry points refuse.
std::vector<int32_t> prefix_lengths(PyObject* list, int64_t N, int64_t T) {
  if (PyList_GET_SIZE(list) != N) fail(PyExc_ValueError, "one length per utterance is required");
  std::vector<int32_t> lengths(N);
  for (int64_t i = 0; i < N; ++i) {
    const int64_t v = integer(PyList_GET_ITEM(list, i));
    lengths[i] = (int32_t)(v < 0 || v > T ? -1 : v);
  }
  return lengths;
}
// The frames of a portion; one without any (which the C ABI has no form for) becomes one frame of which nothing is read.
struct Frames {
  at::Tensor none;
  const int32_t* classes;
  const float* logprobs;
  Frames(const at::Tensor& c, const at::Tensor& l, at::Device dev) {
    if (c.numel() == 0) none = empty({std::max<int64_t>(1, c.size(0) * c.size(2))}, at::kInt, dev);
    classes = (const int32_t*)ptr(none.defined() ? none : c);
    logprobs = (const float*)ptr(none.defined() ? none : l);
  }
};
at::Tensor prefix_state(const pctc_prefix_t& p, at::Device dev) {
  size_t need = 0;
  check(api.prefix_state_bytes(&p, &need), "pctc_prefix_state_bytes");
  return empty({(int64_t)need}, at::kByte, dev);
}

// What a read writes, in one allocation.
struct PrefixOut {
  Shared shared;
  at::Tensor tokens, sizes, scores, flags;
  PrefixOut(const pctc_prefix_t& p, int64_t width, at::Device dev) : shared(dev) {
    if (width < 1 || width > INT32_MAX) fail(PyExc_ValueError, "max_tokens must be at least 1");
    shared.add({p.N, p.beams, width}, at::kInt);
    shared.add({p.N, p.beams}, at::kInt);
    shared.add({p.N, p.beams}, at::kFloat);
    shared.add({p.N}, at::kInt);
    shared.allocate();
    tokens = shared.get(0);
    sizes = shared.get(1);
    scores = shared.get(2);
    flags = shared.get(3);
  }
  PyObject* dict() const {
    PyObject* d = PyDict_New();
    if (!d) throw Failed{};
    put(d, "tokens", tokens);
    put(d, "token_lengths", sizes);
    put(d, "scores", scores);
    put(d, "flags", flags);
    return d;
  }
};

// prefix_check(classes, logprobs, N, device index): the checks of a portion of frames
PyObject* prefix_check(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 4);
  prefix_inputs(tensor(a[0], "classes"), tensor(a[1], "logprobs"), integer(a[2]), integer(a[3]));
  Py_RETURN_NONE;
  MARSHAL_END
}
// prefix_start(N, beams, blank, max_frames, device index) -> state
PyObject* prefix_start(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 5);
  const pctc_prefix_t p = prefix_problem(integer(a[0]), 1, 1, a[1], a[2], a[3]);
  const at::Device dev(at::kCUDA, (c10::DeviceIndex)integer(a[4]));
  const c10::cuda::CUDAGuard guard(dev);
  return THPVariable_Wrap(prefix_state(p, dev));
  MARSHAL_END
}
// prefix_advance(state, classes, logprobs, lengths list, N, beams, blank, max_frames, fresh)
PyObject* prefix_advance(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 9);
  const at::Tensor& state = tensor(a[0], "state");
  const at::Tensor& c = tensor(a[1], "classes");
  const at::Tensor& l = tensor(a[2], "logprobs");
  const at::Device dev = state.device();
  prefix_inputs(c, l, integer(a[4]), dev.index());
  const pctc_prefix_t p = prefix_problem(c.size(0), std::max<int64_t>(1, c.size(1)), c.size(2), a[5], a[6], a[7]);
  const std::vector<int32_t> lengths = prefix_lengths(a[3], p.N, c.size(1));
  const c10::cuda::CUDAGuard guard(dev);
  const Frames in(c, l, dev);
  check(api.prefix_advance(&p, in.classes, in.logprobs, lengths.data(), (int32_t)integer(a[8]),
                           ptr(state), (size_t)state.numel(), stream_of(dev)),
        "pctc_prefix_advance");
  Py_RETURN_NONE;
  MARSHAL_END
}
// prefix_read(state, N, beams, blank, max_frames, width) -> dict
PyObject* prefix_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 6);
  const at::Tensor& state = tensor(a[0], "state");
  const pctc_prefix_t p = prefix_problem(integer(a[1]), 1, 1, a[2], a[3], a[4]);
  const at::Device dev = state.device();
  const c10::cuda::CUDAGuard guard(dev);
  const PrefixOut o(p, integer(a[5]), dev);
  check(api.prefix_read(&p, ptr(state), (size_t)state.numel(), (int32_t*)ptr(o.tokens), (int32_t)o.tokens.size(2),
                        (int32_t*)ptr(o.sizes), (float*)ptr(o.scores), (int32_t*)ptr(o.flags), stream_of(dev)),
        "pctc_prefix_read");
  return o.dict();
  MARSHAL_END
}
// prefix_decode(classes, logprobs, lengths list, beams, blank) -> (dict, state)
PyObject* prefix_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 5);
  const at::Tensor& c = tensor(a[0], "classes");
  const at::Tensor& l = tensor(a[1], "logprobs");
  if (!c.is_cuda()) fail(PyExc_ValueError, "the state of a prefix search lives on a CUDA device");
  const at::Device dev = c.device();
  prefix_inputs(c, l, c.dim() ? c.size(0) : 0, dev.index());
  PyObject* frames = PyLong_FromLongLong(std::max<int64_t>(1, c.size(1)));
  if (!frames) throw Failed{};
  pctc_prefix_t p;
  try {
    p = prefix_problem(c.size(0), std::max<int64_t>(1, c.size(1)), c.size(2), a[3], a[4], frames);
  } catch (...) {
    Py_DECREF(frames);
    throw;
  }
  Py_DECREF(frames);
  for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[2]); ++i)
    if (integer(PyList_GET_ITEM(a[2], i)) > c.size(1)) fail(PyExc_ValueError, "more frames than the state has room for");
  const std::vector<int32_t> lengths = prefix_lengths(a[2], p.N, c.size(1));
  const c10::cuda::CUDAGuard guard(dev);
  const at::Tensor state = prefix_state(p, dev);
  const PrefixOut o(p, p.max_frames, dev);
  const Frames in(c, l, dev);
  check(api.prefix_decode(&p, in.classes, in.logprobs, lengths.data(), ptr(state), (size_t)state.numel(),
                          (int32_t*)ptr(o.tokens), p.max_frames, (int32_t*)ptr(o.sizes), (float*)ptr(o.scores),
                          (int32_t*)ptr(o.flags), stream_of(dev)),
        "pctc_prefix_decode");
  PyObject* d = o.dict();
  PyObject* s = THPVariable_Wrap(state);
  PyObject* both = s ? PyTuple_Pack(2, d, s) : nullptr;
  Py_DECREF(d);
  Py_XDECREF(s);
  return both;
  MARSHAL_END
}

// bind(addresses of the C entry points in the order of `api`, PctcError)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 2);
  void** slots = (void**)&api;
  const Py_ssize_t m = sizeof(api) / sizeof(void*);
  if (!PyList_Check(a[0]) || PyList_GET_SIZE(a[0]) != m) fail(PyExc_TypeError, "%d addresses expected", (int)m);
  for (Py_ssize_t i = 0; i < m; ++i) slots[i] = (void*)(uintptr_t)integer(PyList_GET_ITEM(a[0], i));
  Py_INCREF(a[1]);
  Py_XSETREF(error_type, a[1]);
  Py_RETURN_NONE;
  MARSHAL_END
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(bind), FAST(clip_grad_norm), FAST(grad_sqsum), FAST(grad_scale), FAST(beam_select),
                         FAST(beam_reorder), FAST(prefix_check), FAST(prefix_start), FAST(prefix_advance),
                         FAST(prefix_read), FAST(prefix_decode),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
