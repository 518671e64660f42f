// Argument marshalling of the operators around the head, for the Python binding: checks tensors, fills the C ABI's
// argument tables and allocates the outputs.  A decoding step calls several of these for every token, and a
// list of some hundred gradients or caches costs the interpreter more time than the GPU needs for them.
// Nothing is computed here; the entry points of libprunedctc are handed in by address (bind).
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
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
  decltype(&pctc_embed) embed;
  decltype(&pctc_embed_grad_workspace_bytes) embed_grad_workspace_bytes;
  decltype(&pctc_embed_grad) embed_grad;
  decltype(&pctc_dropout) dropout;
  decltype(&pctc_policy_workspace_bytes) policy_workspace_bytes;
  decltype(&pctc_policy_loss) policy_loss;
  decltype(&pctc_i8_quantize) i8_quantize;
  decltype(&pctc_i8_matmul) i8_matmul;
  decltype(&pctc_i8_logits_workspace_bytes) i8_logits_workspace_bytes;
  decltype(&pctc_i8_logits) i8_logits;
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
  // What at::empty does, on the current stream, without its way through the dispatcher (0.5 us).
  void allocate() {
    const c10::cuda::CUDAGuard guard(dev_);
    base_ = c10::Storage(c10::Storage::use_byte_size_t(), (size_t)std::max<int64_t>(bytes_, 1), c10::cuda::CUDACachingAllocator::get(), true);
  }
  at::Tensor get(size_t i) const { return view(i, 0, parts_[i].shape); }
  // `shape` values of part i from the first one on.
  at::Tensor view(size_t i, int64_t first, at::IntArrayRef shape) const {
    const Part& p = parts_[i];
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(base_), c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                                            c10::scalarTypeToTypeMeta(p.type));
    t.unsafeGetTensorImpl()->set_storage_offset(p.at / (int64_t)c10::elementSize(p.type) + first);
    t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
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
  c10::Storage base_;
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

// ---- the head's matrix and the loss ----

bool is_float(at::ScalarType t) { return t == at::kBFloat16 || t == at::kFloat; }
int32_t kind_of(at::ScalarType t) { return t == at::kFloat ? PCTC_FP32 : t == at::kBFloat16 ? PCTC_BF16 : PCTC_INT8; }
at::ScalarType dtype_or(PyObject* o, at::ScalarType other) {
  if (o == Py_None) return other;
  if (!THPDtype_Check(o)) fail(PyExc_TypeError, "dtype must be a torch.dtype");
  const at::ScalarType t = ((THPDtype*)o)->scalar_type;
  if (!is_float(t)) fail(PyExc_ValueError, "dtype must be bf16 or fp32");
  return t;
}
// A tensor [..., cols] as rows with one stride.
struct RowView {
  int64_t rows = 1, cols = 1, ld = 1;
};
RowView rows_of(const at::Tensor& t, const char* what) {
  if (t.dim() < 1) fail(PyExc_ValueError, "%s must have a dimension", what);
  RowView v;
  v.cols = t.size(-1);
  v.ld = std::max<int64_t>(1, v.cols);
  if (t.numel() == 0) {
    for (int64_t d = 0; d + 1 < t.dim(); ++d) v.rows *= t.size(d);
    return v;
  }
  if (v.cols > 1 && t.stride(-1) != 1) fail(PyExc_ValueError, "%s must be contiguous in its last dimension", what);
  int64_t next = 0;                       // the stride that the next dimension outwards has to have, behind the innermost one
  for (int64_t d = t.dim() - 2; d >= 0; --d) {
    if (t.size(d) == 1) continue;
    if (v.rows == 1) v.ld = t.stride(d);
    else if (t.stride(d) != next) fail(PyExc_ValueError, "the rows of %s must lie one stride apart", what);
    if (v.ld < v.cols) fail(PyExc_ValueError, "rows of %s overlap", what);   // (an expanded dimension has the stride 0)
    next = t.stride(d) * t.size(d);
    v.rows *= t.size(d);
  }
  return v;
}
std::vector<int64_t> with_last(const at::Tensor& t, int64_t last, bool replace) {
  std::vector<int64_t> s = t.sizes().vec();
  if (replace) s.pop_back();
  s.push_back(last);
  return s;
}
bool has_shape(const at::Tensor& t, const std::vector<int64_t>& s) { return t.sizes().equals(s); }
// The given bytes; new ones where there are none or, if they come back to the caller (`back`), too few.
at::Tensor bytes_or(PyObject* given, size_t need, at::Device dev, bool back = true) {
  const at::Tensor w = optional_tensor(given, "workspace");
  if (w.defined() && (w.device() != dev || w.scalar_type() != at::kByte || !w.is_contiguous()))
    fail(PyExc_ValueError, "workspace must be contiguous bytes on the device of the call");
  return w.defined() && (!back || (size_t)w.numel() >= need) ? w : empty({(int64_t)need}, at::kByte, dev);
}
uint64_t word(PyObject* o, const char* what) {
  if (!PyLong_Check(o)) fail(PyExc_TypeError, "%s must be an integer", what);
  return PyLong_AsUnsignedLongLongMask(o);
}
bool truth(PyObject* o) {
  const int t = PyObject_IsTrue(o);
  if (t < 0) throw Failed{};
  return t != 0;
}
const at::Tensor& token_ids(PyObject* o) {
  const at::Tensor& t = tensor(o, "tokens");
  if (!t.is_cuda() || t.scalar_type() != at::kInt || !t.is_contiguous()) fail(PyExc_ValueError, "tokens must be a contiguous int32 CUDA tensor");
  return t;
}
// An 8-bit matrix [rows, cols] with a scale a row.
void check_i8(const at::Tensor& q, const at::Tensor& s, at::Device dev, const char* what) {
  if (q.scalar_type() != at::kChar || q.dim() != 2 || q.device() != dev || s.device() != dev || s.scalar_type() != at::kFloat ||
      s.dim() != 1 || s.size(0) != q.size(0) || !s.is_contiguous())
    fail(PyExc_ValueError, "%s must be int8 [rows, D] with contiguous fp32 scales [rows], on one device", what);
}
// The pitch of its rows for the product (of a single row, any that will do).
int64_t i8_pitch(const RowView& v) { return v.rows > 1 ? v.ld : (v.cols + 15) / 16 * 16; }

// embed(tokens, W, row_scales or None, scale, dtype or None, out or None) -> out
PyObject* embed(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 6);
  const at::Tensor& t = token_ids(a[0]);
  const at::Tensor& W = tensor(a[1], "W");
  const at::Tensor s = optional_tensor(a[2], "row_scales");
  const at::Device dev = t.device();
  if (W.dim() != 2 || W.device() != dev) fail(PyExc_ValueError, "W must be [V, D] on the tokens' device");
  if (s.defined()) check_i8(W, s, dev, "a quantized head");
  else if (!is_float(W.scalar_type())) fail(PyExc_ValueError, "W must be bf16 or fp32, or a quantized head");
  const RowView w = rows_of(W, "W");
  const at::Tensor given = optional_tensor(a[5], "out");
  const at::ScalarType type = dtype_or(a[4], given.defined() ? given.scalar_type() : s.defined() ? at::kBFloat16 : W.scalar_type());
  const std::vector<int64_t> shape = with_last(t, W.size(1), false);
  if (given.defined() && (given.device() != dev || given.scalar_type() != type || !is_float(type) || !has_shape(given, shape)))
    fail(PyExc_ValueError, "out must be [*tokens.shape, D] of the asked type (bf16 or fp32) on the tokens' device");
  const int64_t ld_out = given.defined() ? rows_of(given, "out").ld : W.size(1);
  const c10::cuda::CUDAGuard guard(dev);
  const at::Tensor out = given.defined() ? given : empty(shape, type, dev);
  const pctc_embed_t p{t.numel(), W.size(0), W.size(1), w.ld, ld_out, kind_of(W.scalar_type()), kind_of(type), (float)real(a[3]), 0};
  check(api.embed(&p, (const int32_t*)ptr(t), ptr(W), (const float*)ptr(s), ptr(out), stream_of(dev)), "pctc_embed");
  if (given.defined()) written(given);
  return THPVariable_Wrap(out);
  MARSHAL_END
}
// embed_grad(tokens, grad, V or None, dW or None, scale, accumulate, dtype or None, workspace) -> (dW, workspace)
PyObject* embed_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 8);
  const at::Tensor& t = token_ids(a[0]);
  const at::Tensor& g = tensor(a[1], "grad");
  const at::Device dev = t.device();
  if (g.device() != dev || !is_float(g.scalar_type()) || g.dim() != t.dim() + 1 || !g.sizes().slice(0, t.dim()).equals(t.sizes()))
    fail(PyExc_ValueError, "grad must be [*tokens.shape, D], bf16 or fp32, on the tokens' device");
  const int64_t D = g.size(-1);
  const at::Tensor given = optional_tensor(a[3], "dW");
  const bool accumulate = truth(a[5]);
  if (!given.defined() && (accumulate || a[2] == Py_None)) fail(PyExc_ValueError, "%s", accumulate ? "accumulating needs a dW" : "vocab or dW must be given");
  const at::ScalarType type = dtype_or(a[6], given.defined() ? given.scalar_type() : g.scalar_type());
  const int64_t V = given.defined() && given.dim() == 2 ? given.size(0) : a[2] == Py_None ? 0 : integer(a[2]);
  if (given.defined() && (given.dim() != 2 || given.size(1) != D || given.device() != dev || given.scalar_type() != type ||
                          !is_float(type) || (a[2] != Py_None && integer(a[2]) != V)))
    fail(PyExc_ValueError, "dW must be [V, D], bf16 or fp32, on the tokens' device");
  if (V < 1 || D < 1) fail(PyExc_ValueError, "vocab and D must be at least 1");
  const RowView x = rows_of(g, "grad");
  const int64_t ld_w = given.defined() ? rows_of(given, "dW").ld : D;
  const c10::cuda::CUDAGuard guard(dev);
  const pctc_embed_t p{t.numel(), V, D, ld_w, x.ld, kind_of(type), kind_of(g.scalar_type()), (float)real(a[4]), accumulate ? 1 : 0};
  size_t need = 0;
  check(api.embed_grad_workspace_bytes(&p, &need), "pctc_embed_grad_workspace_bytes");
  const at::Tensor dW = given.defined() ? given : empty({V, D}, type, dev), ws = bytes_or(a[7], need, dev);
  check(api.embed_grad(&p, (const int32_t*)ptr(t), ptr(g), ptr(dW), ptr(ws), (size_t)ws.numel(), stream_of(dev)), "pctc_embed_grad");
  if (given.defined()) written(given);
  return pair(dW, ws);
  MARSHAL_END
}
// dropout(x, p, seed, offset, step or None, residual or None, out or None) -> out
PyObject* dropout(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 7);
  const at::Tensor& x = tensor(a[0], "x");
  if (!x.is_cuda() || !is_float(x.scalar_type())) fail(PyExc_ValueError, "x must be a bf16 or fp32 CUDA tensor");
  const at::Device dev = x.device();
  const at::Tensor step = optional_tensor(a[4], "step"), res = optional_tensor(a[5], "residual"), given = optional_tensor(a[6], "out");
  if (step.defined() && (step.scalar_type() != at::kLong || step.numel() != 1 || step.device() != dev))
    fail(PyExc_ValueError, "step must be one int64 value on the device of x");
  for (const at::Tensor* t : {&res, &given})
    if (t->defined() && (t->device() != dev || t->scalar_type() != x.scalar_type() || !t->sizes().equals(x.sizes())))
      fail(PyExc_ValueError, "residual and out must be of x's shape, type and device");
  const RowView v = rows_of(x, "x");
  const int64_t ld_res = res.defined() ? rows_of(res, "residual").ld : 1;
  const int64_t ld_out = given.defined() ? rows_of(given, "out").ld : std::max<int64_t>(1, v.cols);
  const c10::cuda::CUDAGuard guard(dev);
  const at::Tensor out = given.defined() ? given : empty(x.sizes(), x.scalar_type(), dev);
  pctc_dropout_t p{v.rows, v.cols, v.ld, ld_res, ld_out, kind_of(x.scalar_type()), 0, real(a[1]), word(a[2], "seed"), word(a[3], "offset")};
  check(api.dropout(&p, ptr(x), ptr(res), (const int64_t*)ptr(step), ptr(out), stream_of(dev)), "pctc_dropout");
  if (given.defined()) written(given);
  return THPVariable_Wrap(out);
  MARSHAL_END
}
// policy_loss(logp, old_logp, advantages, ref_logp, mask, lengths (each or None), low, high, kl_weight, reduction, negated,
//             want_grad, workspace or None) -> dict
PyObject* policy_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 13);
  const at::Tensor& x = tensor(a[0], "logp");
  if (!x.is_cuda() || x.scalar_type() != at::kFloat || x.dim() < 1 || x.dim() > 2) fail(PyExc_ValueError, "logp must be an fp32 CUDA tensor [N, T] or [N]");
  const at::Device dev = x.device();
  const int64_t N = x.size(0), T = x.dim() == 2 ? x.size(1) : 1;
  const auto same = [&](PyObject* o, at::ScalarType type, const char* what) {
    const at::Tensor t = optional_tensor(o, what);
    if (t.defined() && (t.scalar_type() != type || !t.sizes().equals(x.sizes()) || t.device() != dev))
      fail(PyExc_ValueError, "%s must be %s of logp's shape on its device", what, type == at::kBool ? "bool" : "fp32");
    return t;
  };
  const auto stride = [&](const at::Tensor& t, const char* what) -> int64_t {
    if (!t.defined() || t.numel() == 0) return T;
    if (T > 1 && t.stride(1) != 1) fail(PyExc_ValueError, "%s must be contiguous in its last dimension", what);
    if (N > 1 && t.stride(0) < T) fail(PyExc_ValueError, "rows of %s overlap", what);
    return N > 1 ? t.stride(0) : T;
  };
  tensor(a[1], "old_logp");
  const at::Tensor old = same(a[1], at::kFloat, "old_logp"), ref = same(a[3], at::kFloat, "ref_logp"), mask = same(a[4], at::kBool, "mask");
  const at::Tensor& adv = tensor(a[2], "advantages");
  const bool each = adv.sizes().equals(x.sizes());
  if (adv.scalar_type() != at::kFloat || adv.device() != dev ||
      (!each && (adv.dim() != 1 || adv.size(0) != N || !adv.is_contiguous())))
    fail(PyExc_ValueError, "advantages must be fp32, contiguous [N] or of logp's shape, on its device");
  const at::Tensor lengths = optional_tensor(a[5], "lengths");
  if (lengths.defined() && (lengths.scalar_type() != at::kInt || lengths.dim() != 1 || lengths.size(0) != N || !lengths.is_contiguous() || lengths.device() != dev))
    fail(PyExc_ValueError, "lengths must be contiguous int32 [N] on the device of logp");
  pctc_policy_t p = {};
  p.N = N;
  p.T = T;
  p.ld_logp = stride(x, "logp");
  p.ld_old = stride(old, "old_logp");
  p.ld_ref = stride(ref, "ref_logp");
  p.ld_adv = each ? stride(adv, "advantages") : 0;
  p.ld_mask = stride(mask, "mask");
  p.ld_grad = T;
  p.clip_low = real(a[6]);
  p.clip_high = real(a[7]);
  p.kl_weight = real(a[8]);
  p.reduction = (int32_t)integer(a[9]);
  p.negated = truth(a[10]) ? 1 : 0;
  const c10::cuda::CUDAGuard guard(dev);
  size_t need = 0;
  check(api.policy_workspace_bytes(&p, &need), "pctc_policy_workspace_bytes");
  const bool want_grad = truth(a[11]), own = a[12] == Py_None;
  Shared out(dev), scalars(dev);            // apart, so that whoever keeps the loss does not keep the gradient and the workspace
  const size_t work = out.add({own ? (int64_t)(need + 255) / 256 * 256 : 0}, at::kByte);      // first: its alignment is the allocation's
  const size_t grad = want_grad ? out.add(x.sizes(), at::kFloat) : 0;
  const size_t stats = scalars.add({3}, at::kFloat), count = scalars.add({1}, at::kInt);
  if (own || want_grad) out.allocate();
  scalars.allocate();
  const at::Tensor ws = own ? out.get(work) : bytes_or(a[12], need, dev), g = want_grad ? out.get(grad) : at::Tensor();
  const at::Tensor loss = scalars.view(stats, 0, {1}), kl = scalars.view(stats, 1, {1}), clipped = scalars.view(stats, 2, {1});
  const at::Tensor counted = scalars.get(count);
  check(api.policy_loss(&p, (const float*)ptr(x), (const float*)ptr(old), (const float*)ptr(ref), (const float*)ptr(adv),
                        (const uint8_t*)ptr(mask), (const int32_t*)ptr(lengths), (float*)ptr(g), (float*)ptr(loss),
                        (int32_t*)ptr(counted), ptr(ws), (size_t)ws.numel(), stream_of(dev)),
        "pctc_policy_loss");
  PyObject* d = PyDict_New();
  if (!d) return nullptr;
  put(d, "loss", loss);
  put(d, "kl", kl);
  put(d, "clipped", clipped);
  put(d, "count", counted);
  if (want_grad) put(d, "grad", g);
  put(d, "workspace", ws);
  return d;
  MARSHAL_END
}
// quantize_rows(x) -> (q, scales)
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 1);
  const at::Tensor& x = tensor(a[0], "x");
  if (!x.is_cuda() || !is_float(x.scalar_type()) || x.dim() != 2 || x.size(1) < 1) fail(PyExc_ValueError, "x must be a bf16 or fp32 CUDA tensor [rows, D]");
  const at::Device dev = x.device();
  const RowView v = rows_of(x, "x");
  const int64_t line = v.cols < 512 ? 16 : 128, ld = (v.cols + line - 1) / line * line;   // long rows start on whole lines
  const c10::cuda::CUDAGuard guard(dev);
  const at::Tensor whole = empty({v.rows, ld}, at::kChar, dev), scales = empty({v.rows}, at::kFloat, dev);
  check(api.i8_quantize(v.rows, v.cols, kind_of(x.scalar_type()), ptr(x), v.ld, (int8_t*)ptr(whole), ld, (float*)ptr(scales), stream_of(dev)),
        "pctc_i8_quantize");
  return pair(ld == v.cols ? whole : whole.narrow(1, 0, v.cols), scales);
  MARSHAL_END
}
at::Tensor bias_of(PyObject* o, int64_t n, at::Device dev) {
  const at::Tensor b = optional_tensor(o, "bias");
  if (b.defined() && (!is_float(b.scalar_type()) || b.dim() != 1 || b.size(0) != n || !b.is_contiguous() || b.device() != dev))
    fail(PyExc_ValueError, "bias must be contiguous [channels], bf16 or fp32, on the operands' device");
  return b;
}
pctc_i8_t i8_problem(int64_t m, int64_t n, int64_t k, at::ScalarType type, int64_t lda, int64_t ldb, const at::Tensor& bias) {
  for (const int64_t v : {m, n, k})
    if (v > INT32_MAX) check(PCTC_ERR_UNSUPPORTED, "8-bit product");
  return pctc_i8_t{(int32_t)m, (int32_t)n, (int32_t)k, kind_of(type), lda, ldb, n, bias.defined() ? kind_of(bias.scalar_type()) : 0, 0};
}
// matmul_i8(a, a_scales, b, b_scales, bias or None, dtype or None, status or None) -> [m, n]
PyObject* matmul_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 7);
  const at::Tensor& A = tensor(a[0], "a");
  const at::Tensor& as = tensor(a[1], "a_scales");
  const at::Tensor& B = tensor(a[2], "b");
  const at::Tensor& bs = tensor(a[3], "b_scales");
  const at::Device dev = A.device();
  if (!A.is_cuda()) fail(PyExc_ValueError, "the operands must be CUDA tensors");
  check_i8(A, as, dev, "a");
  check_i8(B, bs, dev, "b");
  if (A.size(1) != B.size(1)) fail(PyExc_ValueError, "the operands must have rows of one length");
  const at::Tensor bias = bias_of(a[4], B.size(0), dev), status = optional_tensor(a[6], "status");
  if (status.defined() && (status.scalar_type() != at::kInt || status.numel() < 1 || status.device() != dev || !status.is_contiguous()))
    fail(PyExc_ValueError, "status must be an int32 tensor on the operands' device");
  const at::ScalarType type = dtype_or(a[5], at::kFloat);
  const pctc_i8_t p = i8_problem(A.size(0), B.size(0), A.size(1), type, i8_pitch(rows_of(A, "a")), i8_pitch(rows_of(B, "b")), bias);
  const c10::cuda::CUDAGuard guard(dev);
  const at::Tensor C = empty({A.size(0), B.size(0)}, type, dev);
  check(api.i8_matmul(&p, (const int8_t*)ptr(A), (const float*)ptr(as), (const int8_t*)ptr(B), (const float*)ptr(bs), ptr(bias), ptr(C),
                      (int32_t*)ptr(status), stream_of(dev)),
        "pctc_i8_matmul");
  if (status.defined()) written(status);
  return THPVariable_Wrap(C);
  MARSHAL_END
}
// quantized_logits(x, q, scales, bias or None, dtype or None, workspace) -> (logits, workspace)
PyObject* quantized_logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MARSHAL_BEGIN
  want(n, 6);
  const at::Tensor& x = tensor(a[0], "hidden");
  const at::Tensor& q = tensor(a[1], "q");
  const at::Tensor& s = tensor(a[2], "scales");
  const at::Device dev = x.device();
  if (!x.is_cuda() || !is_float(x.scalar_type())) fail(PyExc_ValueError, "hidden must be a bf16 or fp32 CUDA tensor");
  check_i8(q, s, dev, "the head");
  const RowView v = rows_of(x, "hidden");
  if (v.cols != q.size(1)) fail(PyExc_ValueError, "hidden must be [..., D] for a head [V, D]");
  const at::Tensor bias = bias_of(a[3], q.size(0), dev);
  const at::ScalarType type = dtype_or(a[4], x.scalar_type());
  const pctc_i8_t p = i8_problem(v.rows, q.size(0), v.cols, type, v.ld, i8_pitch(rows_of(q, "the head")), bias);
  const c10::cuda::CUDAGuard guard(dev);
  size_t need = 0;
  check(api.i8_logits_workspace_bytes(&p, &need), "pctc_i8_logits_workspace_bytes");
  const at::Tensor C = empty(with_last(x, q.size(0), true), type, dev), ws = bytes_or(a[5], need, dev, false);
  check(api.i8_logits(&p, ptr(x), kind_of(x.scalar_type()), (const int8_t*)ptr(q), (const float*)ptr(s), ptr(bias), ptr(C), ptr(ws),
                      (size_t)ws.numel(), stream_of(dev)),
        "pctc_i8_logits");
  return pair(C, ws);
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
                         FAST(prefix_read), FAST(prefix_decode), FAST(embed), FAST(embed_grad), FAST(dropout),
                         FAST(policy_loss), FAST(quantize_rows), FAST(matmul_i8), FAST(quantized_logits),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
