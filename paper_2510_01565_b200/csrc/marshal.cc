// Marshalling of the context-free operators (include/dit_ops.h) from Python: checks the tensors, allocates results that the caller did
// not bring, and calls libdit.  The small shapes of these operators take the GPU 2 to 10 us; the same steps written in Python over
// ctypes took 8 of a call's 12 us, here they take 1.  Nothing is computed here.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>
#include <vector>

#include "../../include/dit_ops.h"
#include "prompt_call.h"

namespace {

PyObject* g_error = nullptr;                     // binding.DitError(status, detail)

struct Refused { int status; std::string what; };
[[noreturn]] void refuse(std::string what, int status = DIT_ERR_INVALID_ARG) { throw Refused{status, std::move(what)}; }
struct PythonError {};                           // a Python exception is set

// Runs one entry point; C++ exceptions end here.
template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const Refused& r) {
    PyObject* e = PyObject_CallFunction(g_error, "is", r.status, r.what.c_str());
    if (e) { PyErr_SetObject(g_error, e); Py_DECREF(e); }
  } catch (const PythonError&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

void check(dit_status s) {
  if (s != DIT_OK) refuse(dit_status_string(s), s);
}

bool given(PyObject* o) { return o != Py_None; }

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) refuse(std::string(what) + " must be a tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.is_neg()) refuse(std::string(what) + " is a lazily negated view, whose memory holds the other sign (resolve_neg)");
  return t;
}

// Row stride in elements of a CUDA matrix whose rows are contiguous (the rows themselves may lie apart).
int64_t matrix(const at::Tensor& t, const char* what) {
  if (!t.is_cuda() || t.dim() != 2) refuse(std::string(what) + " must be a CUDA matrix");
  if (t.size(1) > 1 && t.stride(1) != 1) refuse(std::string(what) + " must be contiguous along its columns");
  return t.size(0) > 1 ? t.stride(0) : t.size(1);
}

bool shaped(const at::Tensor& t, int64_t rows, int64_t cols) { return t.dim() == 2 && t.size(0) == rows && t.size(1) == cols; }

dit_type type_of(at::ScalarType t) {
  if (t == at::kHalf) return DIT_TYPE_F16;
  if (t == at::kBFloat16) return DIT_TYPE_BF16;
  if (t == at::kFloat) return DIT_TYPE_F32;
  refuse(std::string(c10::toString(t)) + " is not one of float16, bfloat16, float32");
}

// Row stride of codes: a single row has none of its own, and any multiple of 16 describes it.
int64_t pitch(int64_t ld, int64_t rows) { return rows > 1 ? ld : (ld + 15) / 16 * 16; }

// Uninitialised memory of the current stream (see OnStream) on the device of `like`, which is current.  Straight from the allocator: by way of the
// dispatcher the three results of a small quantisation took 3 of its 6.8 us.
at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
  const c10::cuda::CUDAGuard on(like.device());
  return at::detail::empty_generic(sizes, c10::cuda::CUDACachingAllocator::get(), c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt);
}

// Uninitialised e4m3 codes [rows, cols] whose rows start on 16-byte boundaries.
at::Tensor codes_for(int64_t rows, int64_t cols, const at::Tensor& like) {
  const int64_t wide = (cols + 15) / 16 * 16;
  at::Tensor t = empty({rows, wide}, at::kFloat8_e4m3fn, like);
  return wide == cols ? t : t.narrow(1, 0, cols);
}

void same_device(const at::Tensor& first, std::initializer_list<const at::Tensor*> others) {
  for (const at::Tensor* t : others)
    if (t && t->defined() && t->device() != first.device()) refuse("tensors lie on different devices");
}

// The stream of a call on `device`: the given torch.cuda.Stream, or the current one.  While it lives, device and stream are
// current, so that what the call allocates belongs to the stream that uses it: memory of another stream could be
// handed out again, or still be in use, while the kernels run.
struct OnStream {
  c10::cuda::OptionalCUDAGuard device;
  c10::cuda::OptionalCUDAStreamGuard stream;
  void* raw;
  OnStream(PyObject* given_stream, c10::Device on);
};

cudaStream_t given_stream_on(PyObject* stream, c10::Device device) {
  PyObject* index = PyObject_GetAttrString(stream, "device_index");
  if (!index) throw PythonError{};
  const long at = PyLong_AsLong(index);
  Py_DECREF(index);
  PyObject* raw = PyObject_GetAttrString(stream, "cuda_stream");
  if (!raw) throw PythonError{};
  void* s = PyLong_AsVoidPtr(raw);
  Py_DECREF(raw);
  if (PyErr_Occurred()) throw PythonError{};
  if (at != device.index()) refuse("the stream belongs to another device than the tensors");
  return static_cast<cudaStream_t>(s);
}

OnStream::OnStream(PyObject* given_stream, c10::Device on) {
  if (!given(given_stream)) {
    device.set_device(on);
    raw = c10::cuda::getCurrentCUDAStream(on.index()).stream();
  } else {
    raw = given_stream_on(given_stream, on);
    stream.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(raw), on.index()));
  }
}

int64_t number(PyObject* o, const char* what) {
  PyObject* n = PyNumber_Index(o);
  if (!n) { PyErr_Clear(); refuse(std::string(what) + " must be whole numbers"); }
  const long long v = PyLong_AsLongLong(n);
  Py_DECREF(n);
  if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); refuse(std::string(what) + " is out of range"); }
  return v;
}

std::vector<int32_t> numbers(PyObject* o, const char* what) {
  PyObject* seq = PySequence_Tuple(o);           // a copy: an item's __index__ may change a list
  if (!seq) { PyErr_Clear(); refuse(std::string(what) + " must be a sequence of whole numbers"); }
  std::vector<int32_t> v;
  try {
    const Py_ssize_t n = PyTuple_GET_SIZE(seq);
    v.reserve(n);
    for (Py_ssize_t i = 0; i < n; ++i) {
      const int64_t x = number(PyTuple_GET_ITEM(seq, i), what);
      if (x < INT32_MIN || x > INT32_MAX) refuse(std::string(what) + " is out of range", DIT_ERR_SHAPE);
      v.push_back(static_cast<int32_t>(x));
    }
  } catch (...) { Py_DECREF(seq); throw; }
  Py_DECREF(seq);
  return v;
}

void arity(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); throw PythonError{}; }
}

PyObject* pair(const at::Tensor& a, const at::Tensor& b) {
  PyObject* t = PyTuple_New(2);
  if (!t) throw PythonError{};
  PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(a));
  PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(b));
  return t;
}

// x, codes, scales, stream
PyObject* quantize_block128(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    arity(n, 4);
    const at::Tensor& x = tensor(a[0], "x");
    const int64_t ld = matrix(x, "x"), rows = x.size(0), cols = x.size(1), groups = (cols + DIT_BLOCK - 1) / DIT_BLOCK;
    const dit_type type = type_of(x.scalar_type());
    const OnStream on(a[3], x.device());
    const at::Tensor codes = given(a[1]) ? tensor(a[1], "codes") : codes_for(rows, cols, x);
    const at::Tensor scales = given(a[2]) ? tensor(a[2], "scales") : empty({groups, rows}, at::kFloat, x);
    if (codes.scalar_type() != at::kFloat8_e4m3fn || !shaped(codes, rows, cols)) refuse("codes must be float8_e4m3fn, shaped like x");
    if (scales.scalar_type() != at::kFloat || !shaped(scales, groups, rows)) refuse("scales must be fp32 [ceil(cols / 128), rows]");
    same_device(x, {&codes, &scales});
    const int64_t ld_codes = pitch(matrix(codes, "codes"), rows), ld_scales = matrix(scales, "scales");
    check(dit_quantize_block128(x.data_ptr(), type, ld, rows, cols, codes.data_ptr(), ld_codes, static_cast<float*>(scales.data_ptr()), ld_scales,
                                on.raw));
    return pair(codes, scales);
  });
}

// w, codes, scales, stream
PyObject* quantize_weight_block128(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    arity(n, 4);
    const at::Tensor& w = tensor(a[0], "w");
    const int64_t ld = matrix(w, "w"), n_in = w.size(0), n_out = w.size(1);
    const int64_t gn = (n_out + DIT_BLOCK - 1) / DIT_BLOCK, gk = (n_in + DIT_BLOCK - 1) / DIT_BLOCK;
    const dit_type type = type_of(w.scalar_type());
    const OnStream on(a[3], w.device());
    const at::Tensor codes = given(a[1]) ? tensor(a[1], "codes") : codes_for(n_out, n_in, w);
    const at::Tensor scales = given(a[2]) ? tensor(a[2], "scales") : empty({gn, gk}, at::kFloat, w);
    if (codes.scalar_type() != at::kFloat8_e4m3fn || !shaped(codes, n_out, n_in)) refuse("codes must be float8_e4m3fn [out, in]");
    if (scales.scalar_type() != at::kFloat || !shaped(scales, gn, gk) || !scales.is_contiguous())
      refuse("scales must be contiguous fp32 [ceil(out / 128), ceil(in / 128)]");
    same_device(w, {&codes, &scales});
    const int64_t ld_codes = pitch(matrix(codes, "codes"), n_out);
    check(dit_quantize_weight_block128(w.data_ptr(), type, ld, n_in, n_out, codes.data_ptr(), ld_codes, static_cast<float*>(scales.data_ptr()),
                                       on.raw));
    return pair(codes, scales);
  });
}

// a, a_scales, b, b_scales, bias, out, out_dtype, stream
PyObject* gemm_block128(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    arity(n, 8);
    const at::Tensor &x = tensor(a[0], "a"), &sx = tensor(a[1], "a_scales"), &y = tensor(a[2], "b"), &sy = tensor(a[3], "b_scales");
    dit_gemm_block128_args g{};
    const int64_t lda = matrix(x, "a"), ldb = matrix(y, "b"), ld_sa = matrix(sx, "a_scales");
    g.m = x.size(0); g.k = x.size(1); g.n = y.size(0);
    const int64_t groups = (g.k + DIT_BLOCK - 1) / DIT_BLOCK;
    if (x.scalar_type() != at::kFloat8_e4m3fn || y.scalar_type() != at::kFloat8_e4m3fn) refuse("a and b must be float8_e4m3fn codes");
    if (y.size(1) != g.k) refuse("a and b differ in k");
    if (sx.scalar_type() != at::kFloat || !shaped(sx, groups, g.m)) refuse("a_scales must be fp32 [ceil(k / 128), m]");
    if (sy.scalar_type() != at::kFloat || !sy.is_contiguous() || !shaped(sy, (g.n + DIT_BLOCK - 1) / DIT_BLOCK, groups))
      refuse("b_scales must be contiguous fp32 [ceil(n / 128), ceil(k / 128)]");
    at::Tensor bias;
    if (given(a[4])) {
      bias = tensor(a[4], "bias");
      if (!bias.is_cuda() || bias.scalar_type() != at::kFloat || bias.dim() != 1 || bias.size(0) != g.n || !bias.is_contiguous()) refuse("bias must be contiguous fp32 [n]");
    }
    if (given(a[6]) && !THPDtype_Check(a[6])) refuse("out_dtype must be a dtype");
    const at::ScalarType wanted = given(a[6]) ? reinterpret_cast<THPDtype*>(a[6])->scalar_type : at::kHalf;
    type_of(wanted);
    const OnStream on(a[7], x.device());
    const at::Tensor out = given(a[5]) ? tensor(a[5], "out") : empty({g.m, g.n}, wanted, x);
    if (!shaped(out, g.m, g.n) || (given(a[6]) && out.scalar_type() != wanted)) refuse("out must be [m, n] of out_dtype");
    same_device(x, {&sx, &y, &sy, &bias, &out});
    g.a = x.data_ptr(); g.a_scales = static_cast<const float*>(sx.data_ptr()); g.b = y.data_ptr(); g.b_scales = static_cast<const float*>(sy.data_ptr());
    g.bias = bias.defined() ? static_cast<const float*>(bias.data_ptr()) : nullptr;
    g.out = out.data_ptr();
    g.lda = pitch(lda, g.m); g.ldb = pitch(ldb, g.n); g.ld_a_scales = ld_sa; g.ld_out = matrix(out, "out");
    g.out_type = type_of(out.scalar_type());
    check(dit_gemm_block128(&g, on.raw));
    return THPVariable_Wrap(out);
  });
}

struct Batch {
  dit_attention_batch b{};
  std::vector<int32_t> q_lens, kv_lens;
  int64_t q_blocks = 0;
  at::Tensor q, k, v;
};

// q, k, v (None for the selector), q_lens, kv_lens, n_heads
void fill(Batch& t, PyObject* q, PyObject* k, PyObject* v, PyObject* q_lens, PyObject* kv_lens, PyObject* n_heads) {
  t.q = tensor(q, "q"); t.k = tensor(k, "k");
  if (v) t.v = tensor(v, "v");
  t.q_lens = numbers(q_lens, "q_lens"); t.kv_lens = numbers(kv_lens, "kv_lens");
  if (t.q_lens.size() != t.kv_lens.size()) refuse("q_lens and kv_lens differ in length");
  if (t.q_lens.size() > DIT_MAX_REQUESTS) refuse("too many requests", DIT_ERR_CAPACITY);
  const int64_t heads = number(n_heads, "n_heads");
  dit_attention_batch& b = t.b;
  b.ld_q = matrix(t.q, "q"); b.ld_k = matrix(t.k, "k");
  if (v) b.ld_v = matrix(t.v, "v");
  const int64_t width = t.q.size(1);
  if (heads < 1 || width % heads) refuse("the columns of q do not divide into n_heads");
  int64_t rows = 0, kv_rows = 0;
  for (size_t r = 0; r < t.q_lens.size(); ++r) {
    if (t.q_lens[r] < 0 || t.kv_lens[r] < 0) refuse("a length is negative");
    rows += t.q_lens[r]; kv_rows += t.kv_lens[r];
    t.q_blocks += (static_cast<int64_t>(t.q_lens[r]) + DIT_BLOCK - 1) / DIT_BLOCK;
  }
  if (t.q.size(0) != rows || !shaped(t.k, kv_rows, width) || (v && !shaped(t.v, kv_rows, width))) refuse("q, k and v must be [sum of lengths, width]");
  if (t.k.scalar_type() != t.q.scalar_type() || (v && t.v.scalar_type() != t.q.scalar_type())) refuse("q, k and v differ in type");
  b.type = type_of(t.q.scalar_type());
  b.q = t.q.data_ptr(); b.k = t.k.data_ptr(); b.v = v ? t.v.data_ptr() : nullptr;
  b.n_heads = static_cast<int32_t>(heads); b.head_dim = static_cast<int32_t>(width / heads);
  b.n_requests = static_cast<int32_t>(t.q_lens.size()); b.q_lens = t.q_lens.data(); b.kv_lens = t.kv_lens.data();
}

void check_lists(const at::Tensor& index, const at::Tensor& count, const Batch& t) {
  if (!index.is_cuda() || index.scalar_type() != at::kInt || !index.is_contiguous() || index.dim() != 3 || index.size(0) != t.b.n_heads || index.size(1) != t.q_blocks)
    refuse("block_index must be contiguous int32 [n_heads, query blocks, entries]");
  if (!count.is_cuda() || count.scalar_type() != at::kInt || !count.is_contiguous() || !shaped(count, t.b.n_heads, t.q_blocks))
    refuse("block_count must be contiguous int32 [n_heads, query blocks]");
}

// q, k, q_lens, kv_lens, n_heads, keep, tail_rows, index, count, workspace, stream
PyObject* select_blocks(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    arity(n, 11);
    Batch t;
    fill(t, a[0], a[1], nullptr, a[2], a[3], a[4]);
    const std::vector<int32_t> keep = numbers(a[5], "keep"), tail = given(a[6]) ? numbers(a[6], "tail_rows") : std::vector<int32_t>();
    if (keep.size() != t.q_lens.size() || (given(a[6]) && tail.size() != keep.size())) refuse("keep and tail_rows need one number per request");
    int64_t widest = 1;
    for (const int32_t x : keep) {
      if (x < 1) refuse("keep must be at least 1");
      widest = std::max<int64_t>(widest, x);
    }
    const OnStream on(a[10], t.q.device());
    const at::Tensor index = given(a[7]) ? tensor(a[7], "block_index") : empty({t.b.n_heads, t.q_blocks, widest}, at::kInt, t.q);
    const at::Tensor count = given(a[8]) ? tensor(a[8], "block_count") : empty({t.b.n_heads, t.q_blocks}, at::kInt, t.q);
    check_lists(index, count, t);
    const at::Tensor workspace = given(a[9]) ? tensor(a[9], "workspace") : empty({static_cast<int64_t>(std::max<size_t>(16, dit_select_blocks_workspace(&t.b)))}, at::kByte, t.q);
    if (!workspace.is_cuda() || !workspace.is_contiguous()) refuse("workspace must be a contiguous CUDA tensor");
    same_device(t.q, {&t.k, &index, &count, &workspace});
    check(dit_select_blocks(&t.b, keep.data(), given(a[6]) ? tail.data() : nullptr, static_cast<int32_t*>(index.data_ptr()), static_cast<int32_t*>(count.data_ptr()),
                            index.size(2), workspace.data_ptr(), workspace.nbytes(), on.raw));
    return pair(index, count);
  });
}

// q, k, v, q_lens, kv_lens, n_heads, index, count, scale, out, stream
PyObject* block_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    arity(n, 11);
    Batch t;
    fill(t, a[0], a[1], a[2], a[3], a[4], a[5]);
    const at::Tensor &index = tensor(a[6], "block_index"), &count = tensor(a[7], "block_count");
    check_lists(index, count, t);
    const double scale = PyFloat_AsDouble(a[8]);
    if (scale == -1.0 && PyErr_Occurred()) throw PythonError{};
    if (scale != 0.0 && static_cast<float>(scale) == 0.f) refuse("scale rounds to zero, which stands for 1 / sqrt(head_dim)");
    const OnStream on(a[10], t.q.device());
    const at::Tensor out = given(a[9]) ? tensor(a[9], "out") : empty({t.q.size(0), t.q.size(1)}, t.q.scalar_type(), t.q);
    if (!shaped(out, t.q.size(0), t.q.size(1)) || out.scalar_type() != t.q.scalar_type()) refuse("out must be shaped and typed like q");
    same_device(t.q, {&t.k, &t.v, &index, &count, &out});
    const int64_t ld_out = matrix(out, "out");
    check(dit_block_attention(&t.b, static_cast<const int32_t*>(index.data_ptr()), static_cast<const int32_t*>(count.data_ptr()), std::max<int64_t>(index.size(2), 1),
                              static_cast<float>(scale), out.data_ptr(), ld_out, on.raw));
    return THPVariable_Wrap(out);
  });
}

// ------------------------------------------------------------------------------------------------ 4-bit floating point
PyObject* triple(const at::Tensor& a, const at::Tensor& b, const at::Tensor& c) {
  PyObject* t = PyTuple_New(3);
  if (!t) throw PythonError{};
  PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(a));
  PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(b));
  if (c.defined()) PyTuple_SET_ITEM(t, 2, THPVariable_Wrap(c));
  else { Py_INCREF(Py_None); PyTuple_SET_ITEM(t, 2, Py_None); }
  return t;
}

int32_t group_of(PyObject* o) {
  const int64_t g = number(o, "group");
  if (g != 16 && g != 32) refuse("group must be 16 or 32");
  return static_cast<int32_t>(g);
}

int64_t pitch16(const at::Tensor& codes) {       // row stride of codes in bytes; a single row has none of its own
  return pitch(matrix(codes, "codes"), codes.size(0));
}
void check_fp4(const at::Tensor& codes, const at::Tensor& scales, const at::Tensor& row_scales, int64_t rows, int64_t cols, int32_t group, const char* of) {
  if (codes.scalar_type() != at::kByte || !shaped(codes, rows, (cols + 1) / 2)) refuse(std::string(of) + " must be uint8 codes [rows, ceil(columns / 2)]");
  if (!scales.is_cuda() || scales.scalar_type() != at::kByte || !scales.is_contiguous() || scales.dim() != 3 || scales.size(0) != (rows + 127) / 128 ||
      scales.size(1) != (cols + 4 * group - 1) / (4 * group) || scales.size(2) != 512)
    refuse(std::string("the scales of ") + of + " must be contiguous uint8 [ceil(rows / 128), ceil(columns / (4 group)), 512]");
  if (row_scales.defined() && (!row_scales.is_cuda() || row_scales.scalar_type() != at::kFloat || row_scales.dim() != 1 || row_scales.size(0) != rows || !row_scales.is_contiguous()))
    refuse(std::string("the row scales of ") + of + " must be contiguous fp32 [rows]");
}
at::Tensor optional(PyObject* o, const char* what) { return given(o) ? tensor(o, what) : at::Tensor(); }
float* floats(const at::Tensor& t) { return t.defined() ? static_cast<float*>(t.data_ptr()) : nullptr; }

// x, group, codes, scales, row_scales, stream
template <bool kWeight>
PyObject* quantize_to_fp4(PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    arity(n, 6);
    const char* name = kWeight ? "w" : "x";
    const at::Tensor& x = tensor(a[0], name);
    const int64_t ld = matrix(x, name);
    const int32_t group = group_of(a[1]);
    const int64_t rows = x.size(kWeight ? 1 : 0), cols = x.size(kWeight ? 0 : 1);    // of the quantised matrix
    const dit_type type = type_of(x.scalar_type());
    if (cols < 1 || (kWeight && rows < 1)) refuse("an empty row has no scales", DIT_ERR_SHAPE);
    const OnStream on(a[5], x.device());
    at::Tensor codes = optional(a[2], "codes"), scales = optional(a[3], "scales"), row_scales = optional(a[4], "row_scales");
    if (!codes.defined()) {
      const int64_t half = (cols + 1) / 2, wide = (half + 15) / 16 * 16;
      codes = empty({rows, wide}, at::kByte, x);
      if (wide != half) codes = codes.narrow(1, 0, half);
    }
    if (!scales.defined()) scales = empty({(rows + 127) / 128, (cols + 4 * group - 1) / (4 * group), 512}, at::kByte, x);
    if (group == 32 && row_scales.defined()) refuse("groups of 32 have no row scales");
    if (group == 16 && !row_scales.defined()) row_scales = empty({rows}, at::kFloat, x);
    check_fp4(codes, scales, row_scales, rows, cols, group, "the result");
    same_device(x, {&codes, &scales, &row_scales});
    check((kWeight ? dit_quantize_weight_fp4 : dit_quantize_fp4)(x.data_ptr(), type, ld, x.size(0), x.size(1), group, codes.data_ptr(), pitch16(codes), scales.data_ptr(),
                                                                 floats(row_scales), on.raw));
    return triple(codes, scales, row_scales);
  });
}
PyObject* quantize_fp4(PyObject*, PyObject* const* a, Py_ssize_t n) { return quantize_to_fp4<false>(a, n); }
PyObject* quantize_weight_fp4(PyObject*, PyObject* const* a, Py_ssize_t n) { return quantize_to_fp4<true>(a, n); }

at::ScalarType wanted_type(PyObject* dtype, PyObject* out) {
  if (given(dtype) && !THPDtype_Check(dtype)) refuse("out_dtype must be a dtype");
  const at::ScalarType t = given(dtype) ? reinterpret_cast<THPDtype*>(dtype)->scalar_type : (given(out) ? tensor(out, "out").scalar_type() : at::kHalf);
  type_of(t);
  return t;
}

// codes, scales, cols, group, row_scales, out, out_dtype, stream
PyObject* dequantize_fp4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    arity(n, 8);
    const at::Tensor &codes = tensor(a[0], "codes"), &scales = tensor(a[1], "scales");
    const int64_t cols = number(a[2], "cols");
    const int32_t group = group_of(a[3]);
    const int64_t ld = pitch16(codes), rows = codes.size(0);
    const at::Tensor row_scales = optional(a[4], "row_scales");
    if (cols < 1) refuse("cols must be at least 1", DIT_ERR_SHAPE);
    check_fp4(codes, scales, row_scales, rows, cols, group, "codes");
    const at::ScalarType wanted = wanted_type(a[6], a[5]);
    const OnStream on(a[7], codes.device());
    const at::Tensor out = given(a[5]) ? tensor(a[5], "out") : empty({rows, cols}, wanted, codes);
    if (!shaped(out, rows, cols) || out.scalar_type() != wanted) refuse("out must be [rows, cols] of out_dtype");
    same_device(codes, {&scales, &row_scales, &out});
    const int64_t ld_out = matrix(out, "out");
    check(dit_dequantize_fp4(codes.data_ptr(), ld, scales.data_ptr(), floats(row_scales), rows, cols, group, out.data_ptr(), type_of(wanted), ld_out, on.raw));
    return THPVariable_Wrap(out);
  });
}

// a, a_scales, b, b_scales, k, group, a_row_scales, b_row_scales, bias, out, out_dtype, stream
PyObject* gemm_fp4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    arity(n, 12);
    const at::Tensor &x = tensor(a[0], "a"), &sx = tensor(a[1], "a_scales"), &y = tensor(a[2], "b"), &sy = tensor(a[3], "b_scales");
    dit_gemm_fp4_args g{};
    g.k = number(a[4], "k");
    g.group = group_of(a[5]);
    if (g.k < 1) refuse("k must be at least 1", DIT_ERR_SHAPE);
    g.lda = pitch16(x); g.ldb = pitch16(y);
    g.m = x.size(0); g.n = y.size(0);
    const at::Tensor rx = optional(a[6], "a_row_scales"), ry = optional(a[7], "b_row_scales"), bias = optional(a[8], "bias");
    check_fp4(x, sx, rx, g.m, g.k, g.group, "a");
    check_fp4(y, sy, ry, g.n, g.k, g.group, "b");
    if (bias.defined() && (!bias.is_cuda() || bias.scalar_type() != at::kFloat || bias.dim() != 1 || bias.size(0) != g.n || !bias.is_contiguous()))
      refuse("bias must be contiguous fp32 [n]");
    const at::ScalarType wanted = wanted_type(a[10], a[9]);
    const OnStream on(a[11], x.device());
    const at::Tensor out = given(a[9]) ? tensor(a[9], "out") : empty({g.m, g.n}, wanted, x);
    if (!shaped(out, g.m, g.n) || out.scalar_type() != wanted) refuse("out must be [m, n] of out_dtype");
    same_device(x, {&sx, &rx, &y, &sy, &ry, &bias, &out});
    g.ld_out = matrix(out, "out");
    g.a = x.data_ptr(); g.a_scales = sx.data_ptr(); g.a_rows = floats(rx);
    g.b = y.data_ptr(); g.b_scales = sy.data_ptr(); g.b_rows = floats(ry);
    g.bias = floats(bias); g.out = out.data_ptr(); g.out_type = type_of(wanted);
    check(dit_gemm_fp4(&g, on.raw));
    return THPVariable_Wrap(out);
  });
}

// ------------------------------------------------------------------------------------------------ prompts
double real(PyObject* o, const char* what) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); refuse(std::string(what) + " must be a number"); }
  return v;
}
bool truth(PyObject* o) {
  const int t = PyObject_IsTrue(o);
  if (t < 0) throw PythonError{};
  return t != 0;
}

// x, n_heads, lens, first, positions, rotary_dim, interleaved, base, factor, ramp, magnitude, inverse, out, stream
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    arity(n, 14);
    const at::Tensor& x = tensor(a[0], "x");
    dit_rotary_args r{};
    r.ld_x = matrix(x, "x"); r.rows = x.size(0); r.type = type_of(x.scalar_type());
    const int64_t heads = number(a[1], "n_heads"), width = x.size(1);
    if (heads < 1 || heads > INT32_MAX || width < 1 || width % heads) refuse("the columns of x do not divide into n_heads");
    if (width / heads > INT32_MAX) refuse("head_dim is out of range", DIT_ERR_SHAPE);
    r.n_heads = static_cast<int32_t>(heads); r.head_dim = static_cast<int32_t>(width / heads);
    if (given(a[2]) == given(a[4])) refuse("either lens or positions");
    if (given(a[4]) && given(a[3])) refuse("first goes with lens");
    std::vector<int32_t> lens, first;
    at::Tensor positions;
    if (given(a[2])) {
      lens = numbers(a[2], "lens");
      if (given(a[3])) first = numbers(a[3], "first");
      if (given(a[3]) && first.size() != lens.size()) refuse("lens and first differ in length");
      if (lens.size() > DIT_MAX_REQUESTS) refuse("too many requests", DIT_ERR_CAPACITY);
      r.n_requests = static_cast<int32_t>(lens.size()); r.lens = lens.data(); r.first = given(a[3]) ? first.data() : nullptr;
      if (lens.empty()) r.lens = r.first = nullptr;
    } else {
      positions = tensor(a[4], "positions");
      if (!positions.is_cuda() || positions.scalar_type() != at::kInt || positions.dim() != 1 || positions.size(0) != r.rows || !positions.is_contiguous())
        refuse("positions must be contiguous int32 [rows]");
      r.positions = static_cast<const int32_t*>(positions.data_ptr());
    }
    const int64_t rotary_dim = given(a[5]) ? number(a[5], "rotary_dim") : r.head_dim;
    if (rotary_dim < 2 || rotary_dim > r.head_dim) refuse("rotary_dim must lie between 2 and head_dim", DIT_ERR_SHAPE);
    r.rotary_dim = static_cast<int32_t>(rotary_dim);
    r.interleaved = truth(a[6]); r.base = real(a[7], "base"); r.factor = real(a[8], "factor");
    if (given(a[9])) {
      PyObject* ramp = PySequence_Tuple(a[9]);
      if (!ramp) { PyErr_Clear(); refuse("ramp must be (low, high, trained length)"); }
      double v[3] = {};
      const bool three = PyTuple_GET_SIZE(ramp) == 3;
      try {
        for (int i = 0; three && i < 3; ++i) v[i] = real(PyTuple_GET_ITEM(ramp, i), "ramp");
      } catch (...) { Py_DECREF(ramp); throw; }
      Py_DECREF(ramp);
      if (!three || !(v[2] > 0.0)) refuse("ramp must be (low, high, trained length), the length positive");
      r.low = v[0]; r.high = v[1]; r.trained_len = v[2];
    }
    const double magnitude = real(a[10], "magnitude");
    r.magnitude = static_cast<float>(magnitude);
    r.inverse = truth(a[11]);
    const OnStream on(a[13], x.device());
    const at::Tensor out = given(a[12]) ? tensor(a[12], "out") : empty({x.size(0), x.size(1)}, x.scalar_type(), x);
    if (!shaped(out, x.size(0), x.size(1)) || out.scalar_type() != x.scalar_type()) refuse("out must be shaped and typed like x");
    same_device(x, {&positions, &out});
    r.ld_out = matrix(out, "out");
    r.x = x.data_ptr(); r.out = out.data_ptr();
    check(dit_rotary(&r, on.raw));
    return THPVariable_Wrap(out);
  });
}

// q, k, v, q_lens, kv_lens, n_heads, n_kv_heads, causal, scale, out, workspace, stream
PyObject* prompt_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    arity(n, 12);
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
    const std::vector<int32_t> q_lens = numbers(a[3], "q_lens"), kv_lens = numbers(a[4], "kv_lens");
    if (q_lens.size() != kv_lens.size()) refuse("q_lens and kv_lens differ in length");
    if (q_lens.size() > DIT_MAX_REQUESTS) refuse("too many requests", DIT_ERR_CAPACITY);
    const int64_t heads = number(a[5], "n_heads"), kv_heads = given(a[6]) ? number(a[6], "n_kv_heads") : heads;
    dit_prompt_attention_args p{};
    p.ld_q = matrix(q, "q"); p.ld_k = matrix(k, "k"); p.ld_v = matrix(v, "v");
    const int64_t width = q.size(1);
    if (heads < 1 || width < 1 || width % heads) refuse("the columns of q do not divide into n_heads");
    if (kv_heads < 1 || heads % kv_heads) refuse("n_kv_heads must divide n_heads");
    if (heads > INT32_MAX || width / heads > INT32_MAX) refuse("n_heads is out of range", DIT_ERR_SHAPE);
    const int64_t kv_width = width / heads * kv_heads;
    int64_t rows = 0, kv_rows = 0;
    for (size_t r = 0; r < q_lens.size(); ++r) {
      if (q_lens[r] < 0 || kv_lens[r] < 0) refuse("a length is negative");
      rows += q_lens[r]; kv_rows += kv_lens[r];
    }
    if (q.size(0) != rows || !shaped(k, kv_rows, kv_width) || !shaped(v, kv_rows, kv_width)) refuse("q must be [sum of q_lens, n_heads * d], k and v [sum of kv_lens, n_kv_heads * d]");
    if (k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type()) refuse("q, k and v differ in type");
    p.type = type_of(q.scalar_type());
    p.n_heads = static_cast<int32_t>(heads); p.n_kv_heads = static_cast<int32_t>(kv_heads); p.head_dim = static_cast<int32_t>(width / heads);
    p.causal = truth(a[7]);
    const double scale = real(a[8], "scale");
    if (scale != 0.0 && static_cast<float>(scale) == 0.f) refuse("scale rounds to zero, which stands for 1 / sqrt(head_dim)");
    p.scale = static_cast<float>(scale);
    p.n_requests = static_cast<int32_t>(q_lens.size()); p.q_lens = q_lens.data(); p.kv_lens = kv_lens.data();
    const OnStream on(a[11], q.device());
    const at::Tensor out = given(a[9]) ? tensor(a[9], "out") : empty({rows, width}, q.scalar_type(), q);
    if (!shaped(out, rows, width) || out.scalar_type() != q.scalar_type()) refuse("out must be shaped and typed like q");
    const at::Tensor workspace = optional(a[10], "workspace");
    if (workspace.defined() && (!workspace.is_cuda() || !workspace.is_contiguous())) refuse("workspace must be a contiguous CUDA tensor");
    same_device(q, {&k, &v, &out, &workspace});
    p.ld_out = matrix(out, "out");
    p.q = q.data_ptr(); p.k = k.data_ptr(); p.v = v.data_ptr(); p.out = out.data_ptr();
    if (workspace.defined()) {
      p.workspace = workspace.data_ptr(); p.workspace_bytes = workspace.nbytes();
      check(dit_prompt_attention(&p, on.raw));
    } else {
      struct Room { const at::Tensor& like; at::Tensor memory; } room{q, {}};
      check(dit::prompt_attention_in(p, [](void* context, size_t bytes) {
        Room& r = *static_cast<Room*>(context);
        r.memory = empty({static_cast<int64_t>(bytes)}, at::kByte, r.like);
        return r.memory.data_ptr();
      }, &room, on.raw));
    }
    return THPVariable_Wrap(out);
  });
}

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XDECREF(g_error);
  g_error = cls;
  Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {FAST(quantize_block128), FAST(quantize_weight_block128), FAST(gemm_block128), FAST(select_blocks), FAST(block_attention),
                          FAST(quantize_fp4), FAST(quantize_weight_fp4), FAST(dequantize_fp4), FAST(gemm_fp4), FAST(rotary), FAST(prompt_attention),
                          {"set_error", &set_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&kModule); }
