// The decoding model's calls for PyTorch: tensors in, tensors out.  These come
// once a layer and token, so their host time counts; marshalling them from
// Python through ctypes took 18 to 28 us a call, this takes 5 to 7.  Checks of
// arguments and allocation of results only: the work is behind the C ABI
// (include/coverprune.h), whose entry points are called here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <cmath>
#include <string>

#include "coverprune.h"

namespace {

using at::Tensor;

struct Refusal {
  PyObject* type;
  std::string what;
};
[[noreturn]] void bad_value(const std::string& what) { throw Refusal{PyExc_ValueError, what}; }
[[noreturn]] void bad_type(const std::string& what) { throw Refusal{PyExc_TypeError, what}; }

std::string text(at::IntArrayRef s) {
  std::string x = "(";
  for (size_t i = 0; i < s.size(); ++i) x += (i ? ", " : "") + std::to_string(s[i]);
  return x + (s.size() == 1 ? ",)" : ")");
}

// Every tensor of a call is on one device: the first one's.  None may require a gradient
// where autograd records, as the results carry no history, but those read while
// `differentiable` is set: `history` tells whether one did.
struct Call {
  int device = -1;
  bool differentiable = false, history = false;

  const Tensor& tensor(const char* name, PyObject* o) {
    if (!THPVariable_Check(o)) bad_type(std::string(name) + " must be a tensor");
    const Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) bad_value(std::string(name) + " must be a CUDA tensor");
    const int at = (int)t.get_device();
    if (device < 0) device = at;
    if (at != device) bad_value(std::string(name) + " is on another device than the tensors before it");
    if (t.requires_grad() && at::GradMode::is_enabled()) {
      if (!differentiable)
        bad_value(std::string(name) + " requires a gradient, which this call does not give: detach it or call under torch.no_grad()");
      history = true;
    }
    return t;
  }
  // A dense tensor of a type (and, where it is given, a shape).
  const Tensor& dense(const char* name, PyObject* o, at::ScalarType type, at::IntArrayRef shape = {}, bool any = true) {
    const Tensor& t = of_type(name, o, type);
    if (!any && t.sizes() != shape) bad_value(std::string(name) + " must have shape " + text(shape) + ", got " + text(t.sizes()));
    if (!t.is_contiguous()) bad_value(std::string(name) + " must be contiguous");
    return t;
  }
  const Tensor& of_type(const char* name, PyObject* o, at::ScalarType type) {
    const Tensor& t = tensor(name, o);
    if (t.scalar_type() != type)
      bad_type(std::string(name) + " must be " + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
    return t;
  }
  template <typename T>
  T* optional(const char* name, PyObject* o, at::ScalarType type, at::IntArrayRef shape = {}, bool any = true) {
    return o == Py_None ? nullptr : (T*)dense(name, o, type, shape, any).data_ptr();
  }
  // The status word; a tensor without one would pass for none given.
  int32_t* word(const char* name, PyObject* o) {
    int32_t* p = optional<int32_t>(name, o, at::kInt);
    if (o != Py_None && !p) bad_value(std::string(name) + " must have an element");
    return p;
  }
  // Rows of heads: only the last dimension has to be dense.
  const Tensor& rows(const char* name, PyObject* o, int dims) {
    if (!THPVariable_Check(o)) bad_type(std::string(name) + " must be a tensor");
    const int64_t n = THPVariable_Unpack(o).dim();
    if (n != dims) bad_value(std::string(name) + " must have " + std::to_string(dims) + " dimensions, got " + std::to_string(n));
    const Tensor& t = tensor(name, o);
    if (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1) bad_value(std::string(name) + " must be dense in its last dimension");
    return t;
  }
  const Tensor& result(const char* name, PyObject* o, const Tensor& like) {
    const Tensor& t = written(name, rows(name, o, (int)like.dim()));
    if (t.sizes() != like.sizes() || t.scalar_type() != like.scalar_type())
      bad_value(std::string(name) + " must be " + text(like.sizes()) + " of " + c10::toString(like.scalar_type()));
    return t;
  }
  // What is written must not share elements (an expanded tensor does).
  static const Tensor& written(const char* name, const Tensor& t) {
    for (int64_t i = 0; i < t.dim(); ++i)
      if (t.size(i) > 1 && t.stride(i) == 0) bad_value(std::string(name) + " is written and must not be expanded");
    return t;
  }
  // A new tensor, dense; allocated straight from CUDA's allocator, past the dispatch
  // of torch.empty (1 us a tensor).
  Tensor made(at::IntArrayRef sizes, at::ScalarType type) const {
    return Tensor(at::detail::empty_cuda(sizes, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)device), std::nullopt));
  }
  // One like `t`, in the order of its strides where they leave no gaps.
  Tensor like(const Tensor& t) const {
    if (t.is_contiguous() || !t.is_non_overlapping_and_dense()) return made(t.sizes(), t.scalar_type());
    return Tensor(at::detail::empty_strided_cuda(t.sizes(), t.strides(), t.scalar_type(),
                                                 c10::Device(c10::kCUDA, (c10::DeviceIndex)device)));
  }
  cp_stream_t stream() const { return (cp_stream_t)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
};

int row_type(const Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return CP_BF16;
  if (t.scalar_type() == at::kFloat) return CP_F32;
  bad_type(std::string("features must be bfloat16 or float32, got ") + c10::toString(t.scalar_type()));
}

int64_t integer(PyObject* o) {
  const int64_t x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw python_error();
  return x;
}
double real(PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw python_error();
  return x;
}

cp_rope rope_of(Call& c, PyObject* inv_freq, int64_t D, int layout, float scale) {
  const Tensor& f = c.dense("inv_freq", inv_freq, at::kDouble);
  if (f.dim() != 1 || 2 * f.size(0) > D)
    bad_value("inv_freq must hold one frequency for each rotated pair, at most " + std::to_string(D / 2));
  return cp_rope{(const double*)f.data_ptr(), (int32_t)(2 * f.size(0)), layout, scale};
}

cp_rows rows_of(const Tensor& in, const Tensor& out) {
  const int b = (int)in.dim() - 3;  // 1 if there is a batch dimension
  cp_rows r{};
  r.in = in.data_ptr();
  r.out = out.data_ptr();
  r.heads = in.size(1 + b);
  for (int i = 0; i < 2 + b; ++i) {
    r.in_stride[i + 1 - b] = in.stride(i);
    r.out_stride[i + 1 - b] = out.stride(i);
  }
  return r;
}

// The scales of a 4-bit cache's rows; 1 for a row's components each 16, to a multiple of 4.
const Tensor& blocks_of(Call& c, const char* name, PyObject* o, const cp_cache& x) {
  const Tensor& t = c.rows(name, o, 4);
  if (t.scalar_type() != at::kFloat8_e4m3fn)
    bad_type(std::string(name) + " must be float8_e4m3fn, got " + c10::toString(t.scalar_type()));
  const int64_t shape[4] = {x.pages, x.page_size, x.heads, (x.D / 16 + 3) / 4 * 4};
  if (t.sizes() != at::IntArrayRef(shape, 4))
    bad_value(std::string(name) + " must have shape " + text(at::IntArrayRef(shape, 4)) + ", got " + text(t.sizes()));
  return t;
}

cp_cache cache_of(Call& c, PyObject* k_cache, PyObject* v_cache, PyObject* table, PyObject* k_scale, PyObject* v_scale,
                  PyObject* k_block, PyObject* v_block) {
  const Tensor& k = c.rows("k_cache", k_cache, 4);
  const Tensor& v = c.tensor("v_cache", v_cache);
  cp_cache x{};
  x.struct_size = sizeof(x);
  switch (k.scalar_type()) {
    case at::kFloat: x.dtype = CP_F32; break;
    case at::kBFloat16: x.dtype = CP_BF16; break;
    case at::kFloat8_e4m3fn: x.dtype = CP_E4M3; break;
    case at::kByte:
      if (k_block != Py_None && v_block != Py_None) {
        x.dtype = CP_I4;
        break;
      }
      bad_type("a cache of uint8 holds 4 bits an element and needs k_block and v_block");
    default:
      bad_type(std::string("the cache must be float32, bfloat16 or float8_e4m3fn, got ") + c10::toString(k.scalar_type()));
  }
  if (v.sizes() != k.sizes() || v.strides() != k.strides() || v.scalar_type() != k.scalar_type())
    bad_value("k_cache and v_cache must share shape, strides and dtype");
  const Tensor& t = c.of_type("table", table, at::kInt);
  if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) bad_value("table must be [B, width], dense in its last dimension");
  const int64_t each = x.dtype == CP_I4 ? 2 : 1;  // elements of the cache in one of the tensor
  x.k = k.data_ptr();
  x.v = v.data_ptr();
  x.pages = k.size(0);
  x.page_size = k.size(1);
  x.heads = k.size(2);
  x.D = k.size(3) * each;
  // strides of dimensions of one do not matter, whatever the tensor says
  x.page_stride = x.pages > 1 ? k.stride(0) * each : 0;
  x.slot_stride = x.page_size > 1 ? k.stride(1) * each : 0;
  x.head_stride = x.heads > 1 ? k.stride(2) * each : 0;
  if (x.dtype == CP_I4) {
    const Tensor& kb = blocks_of(c, "k_block", k_block, x);
    const Tensor& vb = blocks_of(c, "v_block", v_block, x);
    if (vb.strides() != kb.strides()) bad_value("k_block and v_block must share strides");
    x.k_block = kb.data_ptr();
    x.v_block = vb.data_ptr();
    x.block_page_stride = x.pages > 1 ? kb.stride(0) : 0;
    x.block_slot_stride = x.page_size > 1 ? kb.stride(1) : 0;
    x.block_head_stride = x.heads > 1 ? kb.stride(2) : 0;
  } else if (k_block != Py_None || v_block != Py_None) {
    bad_value("k_block and v_block go with a cache of uint8");
  }
  x.k_scale = c.optional<const float>("k_scale", k_scale, at::kFloat, {x.heads}, false);
  x.v_scale = c.optional<const float>("v_scale", v_scale, at::kFloat, {x.heads}, false);
  x.table = (const int32_t*)t.data_ptr();
  x.table_width = t.size(0) ? t.size(1) : 0;  // nothing, at no address
  x.table_stride = t.stride(0);
  return x;
}

// A cache that a call writes.
void written_cache(const cp_cache& x, PyObject* k_cache, PyObject* v_cache, PyObject* k_block, PyObject* v_block) {
  Call::written("k_cache", THPVariable_Unpack(k_cache));
  Call::written("v_cache", THPVariable_Unpack(v_cache));
  if (x.dtype != CP_I4) return;
  Call::written("k_block", THPVariable_Unpack(k_block));
  Call::written("v_block", THPVariable_Unpack(v_block));
}

// Weights of the keys, a row a sequence.
const Tensor& weights_of(Call& c, const char* name, PyObject* o, int64_t B, int64_t keys) {
  const Tensor& t = c.of_type(name, o, at::kFloat);
  if (t.dim() != 2 || t.size(0) != B || t.size(1) < keys || (t.size(1) > 1 && t.stride(1) != 1))
    bad_value(std::string(name) + " must be [" + std::to_string(B) + ", at least " + std::to_string(keys) +
              "], dense in its last dimension");
  return t;
}

// Autograd learns that a tensor of the caller's was written, and so notices where it had
// saved it.
void changed(PyObject* o) {
  if (o == Py_None) return;
  const Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// The call itself, with other threads let run: a full queue makes it wait.
template <typename F>
int launch(F f) {
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = f();
  Py_END_ALLOW_THREADS;
  return st;
}

PyObject* own(PyObject* o) {
  Py_INCREF(o);
  return o;
}

// A refused argument raises; a status other than CP_OK comes back as a number.
template <typename F>
PyObject* entry(F f) {
  HANDLE_TH_ERRORS
  try {
    return f();
  } catch (const Refusal& r) {
    PyErr_SetString(r.type, r.what.c_str());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

bool counted(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
  return false;
}

// (x or a sequence of them, pos, inv_freq, layout, scale, inverse, out or None); None comes
// back, and nothing is done, where an x requires a gradient
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (!counted(n_args, 7)) return nullptr;
  return entry([&]() -> PyObject* {
    const bool many = PyList_Check(a[0]) || PyTuple_Check(a[0]);
    // tuples of our own: a list may change while other threads run
    const THPObjectPtr x_list(many ? PySequence_Tuple(a[0]) : nullptr);
    const Py_ssize_t n = many ? PyTuple_GET_SIZE(x_list.get()) : 1;
    if (n < 1 || n > 4) bad_value("x must be a tensor or a list of one to four");
    PyObject* const* xs = many ? PySequence_Fast_ITEMS(x_list.get()) : a;
    Call c;
    c.differentiable = true;
    if (!THPVariable_Check(xs[0])) bad_type("x must be a tensor");
    const int dims = (int)THPVariable_Unpack(xs[0]).dim();
    if (dims != 3 && dims != 4) bad_value("x must be [T, heads, D] or [B, T, heads, D]");
    const Tensor& first = c.rows("x", xs[0], dims);
    const int64_t D = first.size(dims - 1), T = first.size(dims - 3), B = dims == 4 ? first.size(0) : 1;
    const int dtype = row_type(first);
    for (Py_ssize_t i = 1; i < n; ++i) {
      const Tensor& x = c.rows("x", xs[i], dims);
      if (x.size(dims - 1) != D || x.size(dims - 3) != T || (dims == 4 && x.size(0) != B) ||
          x.scalar_type() != first.scalar_type())
        bad_value("tensors turned together must share tokens, width and dtype");
    }
    c.differentiable = false;
    const Tensor& pos = c.dense("pos", a[1], at::kLong);
    int64_t pos_stride = 0;
    if (dims == 4 && pos.dim() == 2 && pos.size(0) == B && pos.size(1) == T)
      pos_stride = T;
    else if (pos.dim() != 1 || pos.size(0) != T)
      bad_value("pos must be [" + std::to_string(T) + "]" + (dims == 4 ? " or " + text({B, T}) : std::string()) + ", got " +
                text(pos.sizes()));
    const cp_rope rope = rope_of(c, a[2], D, (int)integer(a[3]), (float)real(a[4]));
    const int inverse = (int)integer(a[5]);
    const bool given = a[6] != Py_None, given_many = PyList_Check(a[6]) || PyTuple_Check(a[6]);
    const THPObjectPtr out_list(given_many ? PySequence_Tuple(a[6]) : nullptr);
    if (given && (given_many != many || (many && PyTuple_GET_SIZE(out_list.get()) != n))) bad_value("out must match x");
    PyObject* const* outs = given_many ? PySequence_Fast_ITEMS(out_list.get()) : a + 6;
    if (c.history) {
      if (given) bad_value("out cannot be given where x requires a gradient");
      return own(Py_None);
    }

    c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.device);
    cp_rows rows[4];
    Tensor made[4];
    for (Py_ssize_t i = 0; i < n; ++i) {
      const Tensor& x = THPVariable_Unpack(xs[i]);
      if (!given) made[i] = c.like(x);
      rows[i] = rows_of(x, given ? c.result("out", outs[i], x) : made[i]);
      if (B == 0 || T == 0) rows[i].heads = 0;  // nothing, at no address
    }
    const int st = launch([&] {
      return coverprune_rotary(rows, (int)n, dtype, B, T, D, (const int64_t*)pos.data_ptr(), pos_stride, &rope, inverse,
                               c.stream());
    });
    if (st != CP_OK) return PyLong_FromLong(st);
    for (Py_ssize_t i = 0; given && i < n; ++i) changed(outs[i]);
    if (!many) return given ? own(a[6]) : THPVariable_Wrap(made[0]);
    PyObject* list = PyList_New(n);
    for (Py_ssize_t i = 0; list && i < n; ++i) PyList_SET_ITEM(list, i, given ? own(outs[i]) : THPVariable_Wrap(made[i]));
    return list;
  });
}

// (k, v, k_cache, v_cache, table, lens, starts, pos, inv_freq, layout, scale, q, k_scale,
// v_scale, new_lens, q_out, status, k_block, v_block) -> (new_lens, q_out)
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (!counted(n_args, 19)) return nullptr;
  return entry([&]() -> PyObject* {
    Call c;
    const cp_cache cache = cache_of(c, a[2], a[3], a[4], a[12], a[13], a[17], a[18]);
    written_cache(cache, a[2], a[3], a[17], a[18]);
    const Tensor& k = c.rows("k", a[0], 3);
    const Tensor& v = c.rows("v", a[1], 3);
    const int64_t T = k.size(0), B = THPVariable_Unpack(a[4]).size(0);
    if (k.size(1) != cache.heads || k.size(2) != cache.D || v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type())
      bad_value("k and v must be [T, " + std::to_string(cache.heads) + ", " + std::to_string(cache.D) + "] of one dtype");
    const int dtype = row_type(k);
    const Tensor& lens = c.dense("lens", a[5], at::kInt, {B}, false);
    if (a[6] == Py_None && T != B)
      bad_value("without starts there is one row a sequence: " + std::to_string(T) + " rows, " + std::to_string(B) + " sequences");
    const int32_t* starts = c.optional<const int32_t>("starts", a[6], at::kInt, {B + 1}, false);
    const int64_t* pos = c.optional<const int64_t>("pos", a[7], at::kLong, {T}, false);
    cp_rope rope{};
    if (a[8] != Py_None) rope = rope_of(c, a[8], cache.D, (int)integer(a[9]), (float)real(a[10]));
    const bool queries = a[11] != Py_None;
    if (queries) {
      const Tensor& q = c.rows("q", a[11], 3);
      if (q.size(0) != T || q.size(2) != cache.D || q.scalar_type() != k.scalar_type())
        bad_value("q must be [" + std::to_string(T) + ", heads, " + std::to_string(cache.D) + "] of k's dtype");
    }
    int32_t* status = c.word("status", a[16]);
    int32_t* given_lens = c.optional<int32_t>("new_lens", a[14], at::kInt, {B}, false);

    c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.device);
    Tensor lens_out, q_out;
    if (!given_lens) lens_out = c.like(lens);
    cp_rows rows{};
    if (queries) {
      const Tensor& q = THPVariable_Unpack(a[11]);
      if (a[15] == Py_None) q_out = c.like(q);
      rows = rows_of(q, a[15] == Py_None ? q_out : c.result("q_out", a[15], q));
    }
    const int64_t ks[2] = {k.stride(0), k.stride(1)}, vs[2] = {v.stride(0), v.stride(1)};
    const int st = launch([&] {
      return coverprune_cache_append(&cache, k.data_ptr(), ks, v.data_ptr(), vs, dtype, T, starts,
                                     (const int32_t*)lens.data_ptr(), B, pos, a[8] == Py_None ? nullptr : &rope,
                                     queries ? &rows : nullptr, given_lens ? given_lens : (int32_t*)lens_out.data_ptr(), status,
                                     c.stream());
    });
    if (st != CP_OK) return PyLong_FromLong(st);
    for (const int i : {2, 3, 14, 16, 17, 18}) changed(a[i]);  // the caches, new_lens, status, the caches' scales
    if (queries) changed(a[15]);
    PyObject* first = given_lens ? own(a[14]) : THPVariable_Wrap(lens_out);
    PyObject* second = !queries || a[15] != Py_None ? own(a[15]) : THPVariable_Wrap(q_out);
    PyObject* both = first && second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_XDECREF(first);
    Py_XDECREF(second);
    return both;
  });
}

// (q, k_cache, v_cache, table, lens, scale or None, window, keep, k_scale, v_scale, lse, out, ws,
// status, k_block, v_block, weight) -> (out, lse or None, ws)
PyObject* decode_attention(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (!counted(n_args, 17)) return nullptr;
  return entry([&]() -> PyObject* {
    Call c;
    const cp_cache cache = cache_of(c, a[1], a[2], a[3], a[8], a[9], a[14], a[15]);
    const Tensor& q = c.rows("q", a[0], 3);
    const int64_t B = THPVariable_Unpack(a[3]).size(0), Hq = q.size(1), keys = cache.table_width * cache.page_size;
    if (q.size(2) != cache.D || q.size(0) != B)
      bad_value("q must be [" + std::to_string(B) + ", heads, " + std::to_string(cache.D) + "], got " + text(q.sizes()));
    const int dtype = row_type(q);
    const Tensor& lens = c.dense("lens", a[4], at::kInt, {B}, false);
    const uint8_t* keep = nullptr;
    int64_t keep_stride = 0;
    if (a[7] != Py_None) {
      const Tensor& m = c.of_type("keep", a[7], at::kBool);
      if (m.dim() != 2 || m.size(0) != B || m.size(1) < keys || (m.size(1) > 1 && m.stride(1) != 1))
        bad_value("keep must be [" + std::to_string(B) + ", at least " + std::to_string(keys) + "], dense in its last dimension");
      keep = (const uint8_t*)m.data_ptr();
      keep_stride = m.stride(0);
    }
    const float scale = a[5] == Py_None ? (float)(1.0 / std::sqrt((double)(cache.D > 0 ? cache.D : 1))) : (float)real(a[5]);
    const int64_t window = integer(a[6]);
    int32_t* status = c.word("status", a[13]);
    const bool weigh = a[16] != Py_None;
    if (weigh) Call::written("weight", weights_of(c, "weight", a[16], B, keys));
    const int with_lse = PyObject_IsTrue(a[10]);
    if (with_lse < 0) throw python_error();

    c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.device);
    Tensor out, lse, ws;
    if (a[12] == Py_None) {
      size_t bytes = 0;
      const int st = weigh ? coverprune_decode_weigh_workspace_size(B, Hq, &cache, &bytes)
                           : coverprune_decode_workspace_size(B, Hq, &cache, &bytes);
      if (st != CP_OK) return PyLong_FromLong(st);
      ws = c.made({(int64_t)bytes}, at::kByte);
    }
    const Tensor& work = a[12] == Py_None ? ws : c.tensor("ws", a[12]);
    if (!work.is_contiguous()) bad_value("ws must be contiguous");  // all its bytes are written to, in a row
    if (a[11] == Py_None) out = c.made(q.sizes(), q.scalar_type());
    const Tensor& to = a[11] == Py_None ? out : c.result("out", a[11], q);
    if (with_lse) lse = c.made({B, Hq}, at::kFloat);
    const int64_t qs[2] = {q.stride(0), q.stride(1)}, os[2] = {to.stride(0), to.stride(1)};
    const int st = launch([&] {
      float* to_lse = with_lse ? (float*)lse.data_ptr() : nullptr;
      const size_t room = (size_t)work.numel() * work.element_size();
      if (weigh) {
        const Tensor& w = THPVariable_Unpack(a[16]);
        return coverprune_decode_attention_weigh(q.data_ptr(), qs, dtype, B, Hq, &cache, (const int32_t*)lens.data_ptr(), keep,
                                                 keep_stride, scale, window, to.data_ptr(), os, to_lse, (float*)w.data_ptr(),
                                                 w.stride(0), work.data_ptr(), room, status, c.stream());
      }
      return coverprune_decode_attention(q.data_ptr(), qs, dtype, B, Hq, &cache, (const int32_t*)lens.data_ptr(), keep,
                                         keep_stride, scale, window, to.data_ptr(), os, to_lse, work.data_ptr(), room, status,
                                         c.stream());
    });
    if (st != CP_OK) return PyLong_FromLong(st);
    for (const int i : {11, 12, 13, 16}) changed(a[i]);  // out, ws, status, weight
    PyObject* x = a[11] == Py_None ? THPVariable_Wrap(out) : own(a[11]);
    PyObject* y = with_lse ? THPVariable_Wrap(lse) : own(Py_None);
    PyObject* z = a[12] == Py_None ? THPVariable_Wrap(ws) : own(a[12]);
    PyObject* all = x && y && z ? PyTuple_Pack(3, x, y, z) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    Py_XDECREF(z);
    return all;
  });
}

// (k_cache, v_cache, table, lens, starts, tokens or None, k_scale, v_scale, k_block, v_block, float32 or
// None, k_out, v_out, status) -> (k, v)
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (!counted(n_args, 14)) return nullptr;
  return entry([&]() -> PyObject* {
    Call c;
    const cp_cache cache = cache_of(c, a[0], a[1], a[2], a[6], a[7], a[8], a[9]);
    const int64_t B = THPVariable_Unpack(a[2]).size(0);
    const Tensor& lens = c.dense("lens", a[3], at::kInt, {B}, false);
    const int32_t* starts = c.optional<const int32_t>("starts", a[4], at::kInt, {B + 1}, false);
    int64_t T = B;
    if (a[5] != Py_None)
      T = integer(a[5]);
    else if (a[11] != Py_None)
      T = c.rows("k_out", a[11], 3).size(0);
    else if (a[4] != Py_None)
      bad_value("with starts, tokens says how many rows there are");
    if (T < 0) bad_value("tokens must not be negative, got " + std::to_string(T));
    if (a[4] == Py_None && T != B)
      bad_value("without starts there is one row a sequence: " + std::to_string(T) + " rows, " + std::to_string(B) + " sequences");
    at::ScalarType type = cache.dtype == CP_F32 ? at::kFloat : at::kBFloat16;
    if (a[10] != Py_None) {
      const int wide = PyObject_IsTrue(a[10]);
      if (wide < 0) throw python_error();
      type = wide ? at::kFloat : at::kBFloat16;
    } else if (a[11] != Py_None) {
      type = c.rows("k_out", a[11], 3).scalar_type();
    }
    int32_t* status = c.word("status", a[13]);

    c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.device);
    Tensor made[2];
    const int64_t shape[3] = {T, cache.heads, cache.D};
    const char* const name[2] = {"k_out", "v_out"};
    for (int i = 0; i < 2; ++i) {
      if (a[11 + i] == Py_None) {
        made[i] = c.made(at::IntArrayRef(shape, 3), type);
        continue;
      }
      const Tensor& t = Call::written(name[i], c.rows(name[i], a[11 + i], 3));
      if (t.sizes() != at::IntArrayRef(shape, 3) || t.scalar_type() != type)
        bad_value(std::string(name[i]) + " must be " + text(at::IntArrayRef(shape, 3)) + " of " + c10::toString(type));
    }
    const Tensor& k = a[11] == Py_None ? made[0] : THPVariable_Unpack(a[11]);
    const Tensor& v = a[12] == Py_None ? made[1] : THPVariable_Unpack(a[12]);
    const int dtype = row_type(k);
    const int64_t ks[2] = {k.stride(0), k.stride(1)}, vs[2] = {v.stride(0), v.stride(1)};
    const int st = launch([&] {
      return coverprune_cache_read(&cache, T, starts, (const int32_t*)lens.data_ptr(), B, k.data_ptr(), ks, v.data_ptr(), vs,
                                   dtype, status, c.stream());
    });
    if (st != CP_OK) return PyLong_FromLong(st);
    for (const int i : {11, 12, 13}) changed(a[i]);
    PyObject* x = a[11] == Py_None ? THPVariable_Wrap(made[0]) : own(a[11]);
    PyObject* y = a[12] == Py_None ? THPVariable_Wrap(made[1]) : own(a[12]);
    PyObject* both = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return both;
  });
}

// (k_cache, v_cache, table, lens, weight, left, first, recent, k_block, v_block, new_lens, new_weight, kept, status)
// -> (new_lens, new_weight, kept)
PyObject* cache_evict(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (!counted(n_args, 14)) return nullptr;
  return entry([&]() -> PyObject* {
    Call c;
    const cp_cache cache = cache_of(c, a[0], a[1], a[2], Py_None, Py_None, a[8], a[9]);
    written_cache(cache, a[0], a[1], a[8], a[9]);
    const int64_t B = THPVariable_Unpack(a[2]).size(0), keys = cache.table_width * cache.page_size;
    const Tensor& lens = c.dense("lens", a[3], at::kInt, {B}, false);
    const Tensor& weight = weights_of(c, "weight", a[4], B, keys);
    const int64_t left = integer(a[5]), first = integer(a[6]), recent = integer(a[7]);
    if (left < 0 || first < 0 || recent < 0 || first > left || recent > left - first)
      bad_value("of the keys that are left, " + std::to_string(left) + ", the first " + std::to_string(first) + " and the last " +
                std::to_string(recent) + " must be parts");
    int32_t* given_lens = c.optional<int32_t>("new_lens", a[10], at::kInt, {B}, false);
    if (a[11] != Py_None && Call::written("new_weight", weights_of(c, "new_weight", a[11], B, keys)).sizes() != weight.sizes())
      bad_value("new_weight must have weight's shape");
    int32_t* given_kept = c.optional<int32_t>("kept", a[12], at::kInt, {B, left}, false);
    int32_t* status = c.word("status", a[13]);

    c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.device);
    Tensor made_lens, made_weight, made_kept;
    if (!given_lens) made_lens = c.like(lens);
    if (a[11] == Py_None) made_weight = c.made(weight.sizes(), at::kFloat);
    if (!given_kept) made_kept = c.made({B, left}, at::kInt);
    const Tensor& to = a[11] == Py_None ? made_weight : THPVariable_Unpack(a[11]);
    const int st = launch([&] {
      return coverprune_cache_evict(&cache, (const int32_t*)lens.data_ptr(), B, (const float*)weight.data_ptr(), weight.stride(0),
                                    left, first, recent, given_lens ? given_lens : (int32_t*)made_lens.data_ptr(),
                                    (float*)to.data_ptr(), to.stride(0), to.size(1),
                                    given_kept ? given_kept : (int32_t*)made_kept.data_ptr(), status, c.stream());
    });
    if (st != CP_OK) return PyLong_FromLong(st);
    for (const int i : {0, 1, 8, 9, 10, 11, 12, 13}) changed(a[i]);
    PyObject* x = given_lens ? own(a[10]) : THPVariable_Wrap(made_lens);
    PyObject* y = a[11] == Py_None ? THPVariable_Wrap(made_weight) : own(a[11]);
    PyObject* z = given_kept ? own(a[12]) : THPVariable_Wrap(made_kept);
    PyObject* all = x && y && z ? PyTuple_Pack(3, x, y, z) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    Py_XDECREF(z);
    return all;
  });
}

PyMethodDef methods[] = {
    {"rotary", (PyCFunction)(void (*)(void))rotary, METH_FASTCALL, nullptr},
    {"cache_append", (PyCFunction)(void (*)(void))cache_append, METH_FASTCALL, nullptr},
    {"decode_attention", (PyCFunction)(void (*)(void))decode_attention, METH_FASTCALL, nullptr},
    {"cache_read", (PyCFunction)(void (*)(void))cache_read, METH_FASTCALL, nullptr},
    {"cache_evict", (PyCFunction)(void (*)(void))cache_evict, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "coverprune_torch", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit_coverprune_torch() { return PyModule_Create(&module); }
