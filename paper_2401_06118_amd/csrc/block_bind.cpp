// Python binding of the operators in block.py and ends.py: shapes, types and strides are read
// from the tensors, output tensors are made, and the C ABI (include/aqlm.h) is
// called.  A decode step makes several such calls per layer, each a few
// microseconds long on the GPU: marshalled in Python they took 12 to 18 us of
// host time, here about half.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <hip/hip_runtime_api.h>

#include <stdexcept>
#include <string>

#include "../../include/aqlm.h"

namespace {

struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};
[[noreturn]] void refuse(const std::string& what) { throw Refused(what); }

// check(status, name) of the package: raises for a status that is not AQLM_OK.
PyObject* g_check = nullptr;
struct PyRaised {};

void done(int status, const char* name) {
  if (status == AQLM_OK) return;
  PyObject* r = g_check ? PyObject_CallFunction(g_check, "is", status, name) : nullptr;
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_Format(PyExc_RuntimeError, "%s: status %d", name, status);
  throw PyRaised();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}
bool given(PyObject* o) { return o != Py_None; }

int dtype_of(const at::Tensor& t, const char* name) {
  switch (t.scalar_type()) {
    case at::kHalf: return AQLM_F16;
    case at::kBFloat16: return AQLM_BF16;
    case at::kFloat: return AQLM_F32;
    default: refuse(std::string(name) + " must be fp16, bf16 or fp32");
  }
}

// A [tokens, heads, head_dim] activation; `like`: one whose type, head size and
// device it must have; tokens and heads of -1: any.
aqlm_heads heads(const at::Tensor& t, const char* name, const at::Tensor* like = nullptr, int64_t tokens = -1,
                 int64_t n = -1) {
  if (!t.is_cuda() || t.dim() != 3) refuse(std::string(name) + " must be a GPU tensor [tokens, heads, head_dim]");
  if (t.size(2) > 1 && t.stride(2) != 1) refuse(std::string("the elements of a head of ") + name + " must be contiguous");
  if ((tokens >= 0 && t.size(0) != tokens) || (n >= 0 && t.size(1) != n))
    refuse(std::string(name) + " does not have the tokens and heads of the other activations");
  if (like && (t.scalar_type() != like->scalar_type() || t.size(2) != like->size(2) || t.device() != like->device()))
    refuse(std::string(name) + " must have the type, head size and device of the other activations");
  dtype_of(t, name);
  if (t.size(1) > INT32_MAX) refuse(std::string(name) + " has too many heads");
  // (the stride of a dimension of one is never used, whatever it says)
  return aqlm_heads{t.data_ptr(), t.size(0) > 1 ? t.stride(0) : 0, t.size(1) > 1 ? t.stride(1) : 0, (int32_t)t.size(1)};
}

// A contiguous vector of n elements of a type on a device.
void* vector(const at::Tensor& t, const char* name, const at::Tensor& like, int64_t n, at::ScalarType type) {
  if (t.scalar_type() != type || t.numel() != n || !t.is_cuda() || t.device() != like.device() || !t.is_contiguous())
    refuse(std::string(name) + " must be a contiguous GPU tensor of " + std::to_string(n) + " elements of type " +
           c10::toString(type));
  return t.data_ptr();
}

// An [rows, n] table whose rows are contiguous.
void* table2(const at::Tensor& t, const char* name, const at::Tensor& like, int64_t rows, at::ScalarType type) {
  if (t.scalar_type() != type || t.dim() != 2 || t.size(0) != rows || !t.is_cuda() || t.device() != like.device() ||
      (t.size(1) > 1 && t.stride(1) != 1))
    refuse(std::string(name) + " must be a GPU tensor [" + std::to_string(rows) + ", n] of type " +
           c10::toString(type) + ", its rows contiguous");
  return t.data_ptr();
}

aqlm_rotation rotation(const at::Tensor& like, PyObject* table, PyObject* qw, PyObject* kw, double eps, bool inter) {
  aqlm_rotation r{};
  const int64_t dim = like.size(2);
  if (given(table)) {
    const at::Tensor& t = tensor(table, "table");
    if (t.scalar_type() != at::kFloat || t.dim() != 3 || t.size(2) != 2 || !t.is_cuda() || t.device() != like.device() ||
        !t.is_contiguous())
      refuse("table must be a contiguous fp32 GPU tensor [positions, rot / 2, 2]");
    if (2 * t.size(1) > dim)
      refuse("the table rotates " + std::to_string(2 * t.size(1)) + " elements of heads of " + std::to_string(dim));
    r.rot = (int32_t)(2 * t.size(1));
    if (r.rot > 0) {
      r.table = t.data_ptr<float>();
      r.rows = t.size(0);
    }
  }
  r.interleaved = inter;
  r.eps = (float)eps;
  if (given(qw)) r.q_weight = vector(tensor(qw, "q_weight"), "q_weight", like, dim, like.scalar_type());
  if (given(kw)) r.k_weight = vector(tensor(kw, "k_weight"), "k_weight", like, dim, like.scalar_type());
  return r;
}

// A caller's output, checked, or a new contiguous one of t's shape.
at::Tensor output(PyObject* out, const at::Tensor& t) {
  if (!given(out)) return at::empty(t.sizes(), t.options());
  const at::Tensor& o = tensor(out, "out");
  if (o.sizes() != t.sizes() || o.scalar_type() != t.scalar_type() || o.device() != t.device())
    refuse("out must have the shape, type and device of its input");
  return o;
}

// A tensor of the caller's that a call has written: autograd's check of saved tensors
// goes by their version.
void written(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void written(PyObject* out) {
  if (given(out)) written(tensor(out, "out"));
}

aqlm_paged_cache cache(const at::Tensor& k, const at::Tensor& v, const at::Tensor& table, const at::Tensor& lens,
                       const at::Tensor& cu) {
  aqlm_paged_cache c{};
  if (k.dim() != 4 || !k.is_cuda() || v.dim() != 4 || !v.is_cuda())
    refuse("k_cache and v_cache must be GPU tensors [pages, page_size, kv heads, head_dim]");
  if (k.sizes() != v.sizes() || k.scalar_type() != v.scalar_type() || k.device() != v.device())
    refuse("k_cache and v_cache must have one shape, type and device");
  if (k.size(3) > 1 && (k.stride(3) != 1 || v.stride(3) != 1))
    refuse("the elements of a head of k_cache and v_cache must be contiguous");
  if (table.scalar_type() != at::kInt || table.dim() != 2 || table.device() != k.device() ||
      (table.size(1) > 1 && table.stride(1) != 1))
    refuse("block_table must be an int32 tensor [sequences, pages] on the cache's device");
  for (int i = 1; i < 4; ++i)
    if (k.size(i) > INT32_MAX) refuse("k_cache is too large");
  if (table.size(0) > INT32_MAX || table.size(1) > INT32_MAX) refuse("block_table is too large");
  c.k = k.data_ptr();
  c.v = v.data_ptr();
  c.pages = k.size(0);
  c.page_size = (int32_t)k.size(1);
  c.kv_heads = (int32_t)k.size(2);
  c.head_dim = (int32_t)k.size(3);
  // (the stride of a dimension of one is never used, whatever it says)
  c.k_page_stride = c.pages > 1 ? k.stride(0) : 0;
  c.v_page_stride = c.pages > 1 ? v.stride(0) : 0;
  c.k_slot_stride = c.page_size > 1 ? k.stride(1) : 0;
  c.v_slot_stride = c.page_size > 1 ? v.stride(1) : 0;
  c.k_head_stride = c.kv_heads > 1 ? k.stride(2) : 0;
  c.v_head_stride = c.kv_heads > 1 ? v.stride(2) : 0;
  c.seqs = (int32_t)table.size(0);
  c.table_width = (int32_t)table.size(1);
  c.block_table = table.data_ptr<int32_t>();
  c.table_stride = c.seqs > 1 ? table.stride(0) : 0;
  c.kv_lens = (const int32_t*)vector(lens, "kv_lens", k, c.seqs, at::kInt);
  c.cu_new = (const int32_t*)vector(cu, "cu_new", k, c.seqs + 1, at::kInt);
  c.dtype = dtype_of(k, "k_cache");
  return c;
}

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PyRaised();
  return v;
}
int64_t integer(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PyRaised();
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw PyRaised();
  return v != 0;
}
void* stream_of(PyObject* o) { return (void*)(uintptr_t)integer(o); }
int32_t int32_or(int64_t v, const char* name) {
  if (v > INT32_MAX || v < INT32_MIN) refuse(std::string(name) + " is out of range");
  return (int32_t)v;
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", N, n);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const PyRaised&) {
  } catch (const Refused& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* none() { Py_RETURN_NONE; }

// q, k, table, positions, q_weight, k_weight, eps, interleaved, out q, out k, stream
PyObject* rope(PyObject* const* a) {
  const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k");
  const aqlm_heads hq = heads(q, "q"), hk = heads(k, "k", &q, q.size(0));
  const aqlm_rotation r = rotation(q, a[2], a[4], a[5], number(a[6]), truth(a[7]));
  const void* pos = vector(tensor(a[3], "positions"), "positions", q, q.size(0), at::kInt);
  const at::Tensor oq = output(a[8], q), ok = output(a[9], k);
  const aqlm_heads hoq = heads(oq, "out"), hok = heads(ok, "out");
  done(aqlm_rope(&hq, &hk, &hoq, &hok, dtype_of(q, "q"), q.size(0), int32_or(q.size(2), "head_dim"),
                 (const int32_t*)pos, &r, stream_of(a[10])),
       "aqlm_rope");
  written(a[8]);
  written(a[9]);
  return Py_BuildValue("NN", wrap(oq), wrap(ok));
}

// dq, dk, table, positions, q, k, q_weight, k_weight, eps, interleaved, out q, out k, stream;
// the last of the results is the workspace
PyObject* rope_backward(PyObject* const* a) {
  const at::Tensor &dq = tensor(a[0], "dq"), &dk = tensor(a[1], "dk");
  const aqlm_heads hdq = heads(dq, "dq"), hdk = heads(dk, "dk", &dq, dq.size(0));
  const int64_t tokens = dq.size(0), dim = dq.size(2);
  const aqlm_rotation r = rotation(dq, a[2], a[6], a[7], number(a[8]), truth(a[9]));
  const void* pos = vector(tensor(a[3], "positions"), "positions", dq, tokens, at::kInt);
  const bool nq = given(a[6]), nk = given(a[7]);
  if ((nq && !given(a[4])) || (nk && !given(a[5]))) refuse("q and k are needed where their norm has a weight");
  aqlm_heads hq{}, hk{};
  if (nq) hq = heads(tensor(a[4], "q"), "q", &dq, tokens, dq.size(1));
  if (nk) hk = heads(tensor(a[5], "k"), "k", &dq, tokens, dk.size(1));
  const at::Tensor gq = output(a[10], dq), gk = output(a[11], dk);
  const aqlm_heads hgq = heads(gq, "out"), hgk = heads(gk, "out");
  at::Tensor ws, wq, wk;
  size_t bytes = 0;
  if (nq || nk) {
    bytes = aqlm_rope_backward_workspace_bytes(int32_or(dim, "head_dim"));
    ws = at::empty({(int64_t)bytes}, dq.options().dtype(at::kByte));
    if (nq) wq = at::empty({dim}, dq.options().dtype(at::kFloat));
    if (nk) wk = at::empty({dim}, dq.options().dtype(at::kFloat));
  }
  if (tokens > 0) {
    done(aqlm_rope_backward(&hdq, &hdk, nq ? &hq : nullptr, nk ? &hk : nullptr, &hgq, &hgk,
                            nq ? wq.data_ptr<float>() : nullptr, nk ? wk.data_ptr<float>() : nullptr,
                            dtype_of(dq, "dq"), tokens, int32_or(dim, "head_dim"), (const int32_t*)pos, &r,
                            bytes ? ws.data_ptr() : nullptr, bytes, stream_of(a[12])),
         "aqlm_rope_backward");
  } else {  // (nothing to sum over)
    if (nq) wq.zero_();
    if (nk) wk.zero_();
  }
  written(a[10]);
  written(a[11]);
  return Py_BuildValue("NNNNN", wrap(gq), wrap(gk), nq ? wrap(wq) : none(), nk ? wrap(wk) : none(),
                       bytes ? wrap(ws) : none());
}

// q, k, v, k_cache, v_cache, block_table, kv_lens, cu_new, table, q_weight, k_weight, eps, interleaved, out, stream
PyObject* paged_append(PyObject* const* a) {
  const at::Tensor &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &kc = tensor(a[3], "k_cache");
  const aqlm_paged_cache c = cache(kc, tensor(a[4], "v_cache"), tensor(a[5], "block_table"), tensor(a[6], "kv_lens"),
                                   tensor(a[7], "cu_new"));
  const aqlm_heads hk = heads(k, "k", nullptr, -1, c.kv_heads), hv = heads(v, "v", &k, k.size(0), c.kv_heads);
  if (k.scalar_type() != kc.scalar_type() || k.size(2) != c.head_dim || k.device() != kc.device())
    refuse("the activations must have the cache's type, head size and device");
  const aqlm_rotation r = rotation(k, a[8], a[9], a[10], number(a[11]), truth(a[12]));
  aqlm_heads hq{}, ho{};
  at::Tensor out;
  if (given(a[0])) {
    const at::Tensor& q = tensor(a[0], "q");
    hq = heads(q, "q", &k, k.size(0));
    out = output(a[13], q);
    ho = heads(out, "out");
  }
  done(aqlm_paged_append(given(a[0]) ? &hq : nullptr, &hk, &hv, given(a[0]) ? &ho : nullptr, &c, k.size(0), &r,
                         stream_of(a[14])),
       "aqlm_paged_append");
  written(kc);
  written(tensor(a[4], "v_cache"));
  if (given(a[0])) written(a[13]);
  return given(a[0]) ? wrap(out) : none();
}

// q, k_cache, v_cache, block_table, kv_lens, cu_new, scale, causal, window, max_new, return_lse, out, workspace, stream
PyObject* paged_attention(PyObject* const* a) {
  const at::Tensor &q = tensor(a[0], "q"), &kc = tensor(a[1], "k_cache");
  const aqlm_paged_cache c = cache(kc, tensor(a[2], "v_cache"), tensor(a[3], "block_table"), tensor(a[4], "kv_lens"),
                                   tensor(a[5], "cu_new"));
  const aqlm_heads hq = heads(q, "q");
  if (q.scalar_type() != kc.scalar_type() || q.size(2) != c.head_dim || q.device() != kc.device())
    refuse("q must have the cache's type, head size and device");
  if (c.kv_heads <= 0 || q.size(1) % c.kv_heads != 0) refuse("the query heads must be a multiple of the kv heads");
  const at::Tensor& ws = tensor(a[12], "workspace");
  if (!ws.is_cuda() || ws.device() != q.device() || !ws.is_contiguous())
    refuse("workspace must be a contiguous GPU tensor on q's device");
  const float scale = given(a[6]) ? (float)number(a[6]) : (float)(1.0 / std::sqrt((double)q.size(2)));
  const at::Tensor out = output(a[11], q);
  const aqlm_heads ho = heads(out, "out");
  at::Tensor lse;
  if (truth(a[10])) lse = at::empty({q.size(0), q.size(1)}, q.options().dtype(at::kFloat));
  done(aqlm_paged_attention(&hq, &ho, lse.defined() ? lse.data_ptr<float>() : nullptr, &c, q.size(0), integer(a[9]),
                            scale, truth(a[7]), int32_or(integer(a[8]), "window"), ws.data_ptr(), ws.nbytes(),
                            stream_of(a[13])),
       "aqlm_paged_attention");
  written(a[11]);
  return lse.defined() ? Py_BuildValue("NN", wrap(out), wrap(lse)) : wrap(out);
}

// logits, tokens, token_lens, prompt_lens, repetition, frequency, presence, bias_ids, bias_values, mask, out, stream
PyObject* process_logits(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0], "logits");
  if (x.dim() != 2 || !x.is_cuda() || (x.size(1) > 1 && x.stride(1) != 1))
    refuse("logits must be a GPU tensor [rows, vocab], its rows contiguous");
  const int dtype = dtype_of(x, "logits");
  const int64_t rows = x.size(0), vocab = x.size(1);
  aqlm_logit_rules r{};
  const bool penalties = given(a[4]) || given(a[5]) || given(a[6]);
  if (given(a[1])) {
    const at::Tensor& t = tensor(a[1], "tokens");
    if (!given(a[2])) refuse("tokens need token_lens");
    const void* ids = table2(t, "tokens", x, rows, at::kInt);
    const void* lens = vector(tensor(a[2], "token_lens"), "token_lens", x, rows, at::kInt);
    const void* prompts = given(a[3]) ? vector(tensor(a[3], "prompt_lens"), "prompt_lens", x, rows, at::kInt) : nullptr;
    const float* p[3];
    const char* names[3] = {"repetition", "frequency", "presence"};
    for (int i = 0; i < 3; ++i)
      p[i] = given(a[4 + i]) ? (const float*)vector(tensor(a[4 + i], names[i]), names[i], x, rows, at::kFloat) : nullptr;
    if (t.size(1) > 0) {  // (otherwise there is nothing to penalise)
      r.tokens = (const int32_t*)ids;
      r.token_lens = (const int32_t*)lens;
      r.prompt_lens = (const int32_t*)prompts;
      r.repetition = p[0];
      r.frequency = p[1];
      r.presence = p[2];
      r.history = int32_or(t.size(1), "tokens");
      r.token_stride = rows > 1 ? t.stride(0) : 0;
    }
  } else if (penalties) {
    refuse("penalties need tokens");
  }
  if (given(a[7]) != given(a[8])) refuse("bias_ids and bias_values go together");
  if (given(a[7])) {
    const at::Tensor &ids = tensor(a[7], "bias_ids"), &values = tensor(a[8], "bias_values");
    if (ids.sizes() != values.sizes() || ids.strides() != values.strides())
      refuse("bias_ids and bias_values must have one shape and layout");
    const void* pi = table2(ids, "bias_ids", x, rows, at::kInt);
    const void* pv = table2(values, "bias_values", x, rows, at::kFloat);
    if (ids.size(1) > 0) {
      r.bias_ids = (const int32_t*)pi;
      r.bias_values = (const float*)pv;
      r.biases = int32_or(ids.size(1), "bias_ids");
      r.bias_stride = rows > 1 ? ids.stride(0) : 0;
    }
  }
  if (given(a[9])) {
    const at::Tensor& m = tensor(a[9], "mask");
    r.mask = (const uint32_t*)table2(m, "mask", x, rows, at::kInt);
    r.mask_stride = rows > 1 ? m.stride(0) : 0;
    if (m.size(1) < (vocab + 31) / 32) refuse("mask must have " + std::to_string((vocab + 31) / 32) + " words per row");
  }
  const at::Tensor out = output(a[10], x);
  if (out.size(1) > 1 && out.stride(1) != 1) refuse("the rows of out must be contiguous");
  done(aqlm_process_logits(x.data_ptr(), rows > 1 ? x.stride(0) : 0, out.data_ptr(), rows > 1 ? out.stride(0) : 0,
                           dtype, rows, vocab, &r, stream_of(a[11])),
       "aqlm_process_logits");
  written(a[10]);
  return wrap(out);
}

// ---------------------------------------------------------------------------
// ends.py

// A call's launches go to the tensors' device, whichever is the current one.
struct OnDevice {
  int before = 0;
  bool changed = false;
  explicit OnDevice(const at::Tensor& t) {
    if (hipGetDevice(&before) == hipSuccess && t.get_device() != before)
      changed = hipSetDevice(t.get_device()) == hipSuccess;
  }
  ~OnDevice() {
    if (changed) (void)hipSetDevice(before);
  }
};

// A [rows, n] activation with contiguous rows; `like`: one whose type and device it has;
// rows, n of -1: any.
const at::Tensor& rows2(PyObject* o, const char* name, const at::Tensor* like = nullptr, int64_t rows = -1,
                        int64_t n = -1) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda() || t.dim() != 2 || (t.size(1) > 1 && t.size(0) > 0 && t.stride(1) != 1))
    refuse(std::string(name) + " must be a GPU tensor with two dimensions, its rows contiguous");
  if ((rows >= 0 && t.size(0) != rows) || (n >= 0 && t.size(1) != n))
    refuse(std::string(name) + " does not have the shape of the other tensors");
  if (like && (t.scalar_type() != like->scalar_type() || t.device() != like->device()))
    refuse(std::string(name) + " must have the type and device of the other tensors");
  dtype_of(t, name);
  return t;
}
// (the stride of a dimension of one is never used, whatever it says)
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : 0; }

// A caller's output of a shape and type, checked, or a new one.
at::Tensor output2(PyObject* out, const char* name, const at::Tensor& like, int64_t rows, int64_t n, at::ScalarType type) {
  if (!given(out)) return at::empty({rows, n}, like.options().dtype(type));
  const at::Tensor& o = rows2(out, name, nullptr, rows, n);
  if (o.scalar_type() != type || o.device() != like.device())
    refuse(std::string(name) + " must have the type and device of the result");
  return o;
}

aqlm_norm norm_of(PyObject* weight, PyObject* bias, double eps, bool rms, const at::Tensor& like) {
  aqlm_norm n{};
  if (given(weight)) n.weight = vector(tensor(weight, "weight"), "weight", like, like.size(1), like.scalar_type());
  if (given(bias)) n.bias = vector(tensor(bias, "bias"), "bias", like, like.size(1), like.scalar_type());
  n.eps = (float)eps;
  n.rms = rms;
  return n;
}

// table, tokens, scale, out, stream
PyObject* embed(PyObject* const* a) {
  const at::Tensor &table = rows2(a[0], "table"), &tokens = tensor(a[1], "tokens");
  if (tokens.dim() != 1) refuse("tokens must be an int32 tensor [tokens]");
  const int64_t count = tokens.numel();
  const void* ids = vector(tokens, "tokens", table, count, at::kInt);
  const at::Tensor out = output2(a[3], "out", table, count, table.size(1), table.scalar_type());
  const OnDevice on(table);
  done(aqlm_embed(table.data_ptr(), row_stride(table), (const int32_t*)ids, out.data_ptr(), row_stride(out),
                  dtype_of(table, "table"), count, table.size(0), table.size(1), (float)number(a[2]), stream_of(a[4])),
       "aqlm_embed");
  written(a[3]);
  return wrap(out);
}

// dout, tokens, vocab, scale, fp32, out, stream; the last of the results is the workspace
PyObject* embed_backward(PyObject* const* a) {
  const at::Tensor &dout = rows2(a[0], "dout"), &tokens = tensor(a[1], "tokens");
  const int64_t count = dout.size(0), vocab = integer(a[2]);
  if (tokens.dim() != 1) refuse("tokens must be an int32 tensor [tokens]");
  const void* ids = vector(tokens, "tokens", dout, count, at::kInt);
  if (vocab <= 0) refuse("vocab must be positive");
  at::ScalarType type = truth(a[4]) ? at::kFloat : dout.scalar_type();
  if (given(a[5]) && tensor(a[5], "out").scalar_type() == at::kFloat) type = at::kFloat;
  const size_t bytes = aqlm_embed_backward_workspace_bytes(count, vocab, dout.size(1), dtype_of(dout, "dout"));
  if (bytes == 0) done(AQLM_ERR_SHAPE, "aqlm_embed_backward");
  const at::Tensor out = output2(a[5], "out", dout, vocab, dout.size(1), type);
  const at::Tensor ws = at::empty({(int64_t)bytes}, dout.options().dtype(at::kByte));
  const OnDevice on(dout);
  done(aqlm_embed_backward(dout.data_ptr(), row_stride(dout), (const int32_t*)ids, out.data_ptr(), row_stride(out),
                           dtype_of(dout, "dout"), dtype_of(out, "out"), count, vocab, dout.size(1), (float)number(a[3]),
                           ws.data_ptr(), bytes, stream_of(a[6])),
       "aqlm_embed_backward");
  written(a[5]);
  return Py_BuildValue("NN", wrap(out), wrap(ws));
}

// x, weight, bias, residual, eps, rms, out, sum_out, stream
PyObject* layer_norm(PyObject* const* a) {
  const at::Tensor& x = rows2(a[0], "x");
  const int64_t rows = x.size(0), dim = x.size(1);
  const aqlm_norm n = norm_of(a[1], a[2], number(a[4]), truth(a[5]), x);
  const at::Tensor out = output2(a[6], "out", x, rows, dim, x.scalar_type());
  const bool both = given(a[3]);
  if (!both && given(a[7])) refuse("sum_out goes with residual");
  at::Tensor r, sum;
  if (both) {
    r = rows2(a[3], "residual", &x, rows, dim);
    sum = output2(a[7], "sum_out", x, rows, dim, x.scalar_type());
  }
  const OnDevice on(x);
  done(aqlm_layer_norm(x.data_ptr(), row_stride(x), both ? r.data_ptr() : nullptr, both ? row_stride(r) : 0,
                       out.data_ptr(), row_stride(out), both ? sum.data_ptr() : nullptr, both ? row_stride(sum) : 0,
                       dtype_of(x, "x"), rows, dim, &n, stream_of(a[8])),
       "aqlm_layer_norm");
  written(a[6]);
  written(a[7]);
  return both ? Py_BuildValue("NN", wrap(out), wrap(sum)) : wrap(out);
}

// dy, x, weight, dsum, eps, rms, bias, out, stream; the last of the results is the workspace
PyObject* layer_norm_backward(PyObject* const* a) {
  const at::Tensor& dy = rows2(a[0], "dy");
  const int64_t rows = dy.size(0), dim = dy.size(1);
  const at::Tensor& x = rows2(a[1], "x", &dy, rows, dim);
  const aqlm_norm n = norm_of(a[2], Py_None, number(a[4]), truth(a[5]), dy);
  at::Tensor dsum, ws, dw, db;
  if (given(a[3])) dsum = rows2(a[3], "dsum", &dy, rows, dim);
  const at::Tensor out = output2(a[7], "out", dy, rows, dim, dy.scalar_type());
  const bool bias = truth(a[6]);
  size_t bytes = 0;
  if (n.weight || bias) {
    bytes = aqlm_layer_norm_backward_workspace_bytes(dim);
    ws = at::empty({(int64_t)bytes}, dy.options().dtype(at::kByte));
    if (n.weight) dw = at::empty({dim}, dy.options().dtype(at::kFloat));
    if (bias) db = at::empty({dim}, dy.options().dtype(at::kFloat));
  }
  const OnDevice on(dy);
  done(aqlm_layer_norm_backward(dy.data_ptr(), row_stride(dy), x.data_ptr(), row_stride(x),
                                dsum.defined() ? dsum.data_ptr() : nullptr, dsum.defined() ? row_stride(dsum) : 0,
                                out.data_ptr(), row_stride(out), dw.defined() ? dw.data_ptr<float>() : nullptr,
                                bias ? db.data_ptr<float>() : nullptr, dtype_of(dy, "dy"), rows, dim, &n,
                                bytes ? ws.data_ptr() : nullptr, bytes, stream_of(a[8])),
       "aqlm_layer_norm_backward");
  written(a[7]);
  return Py_BuildValue("NNNN", wrap(out), dw.defined() ? wrap(dw) : none(), bias ? wrap(db) : none(),
                       bytes ? wrap(ws) : none());
}

// logits, teacher, ids, teacher_lse, weights, temperature, grad, out, stream; the last of the results is the workspace
PyObject* distill_loss(PyObject* const* a) {
  const at::Tensor& x = rows2(a[0], "logits");
  const int64_t rows = x.size(0), vocab = x.size(1);
  const at::Tensor &t = rows2(a[1], "teacher_logits", nullptr, rows), &ids = tensor(a[2], "teacher_ids");
  if (t.device() != x.device()) refuse("teacher_logits must be on the device of logits");
  const void* pi = table2(ids, "teacher_ids", x, rows, at::kInt);
  if (ids.size(1) != t.size(1)) refuse("teacher_logits and teacher_ids must have one shape");
  const void* lse = given(a[3]) ? vector(tensor(a[3], "teacher_lse"), "teacher_lse", x, rows, at::kFloat) : nullptr;
  const void* w = given(a[4]) ? vector(tensor(a[4], "weights"), "weights", x, rows, at::kFloat) : nullptr;
  const bool want = truth(a[6]);
  if (!want && given(a[7])) refuse("out is the gradient's, which is not asked for");
  at::Tensor grad;
  if (want) grad = output2(a[7], "out", x, rows, vocab, x.scalar_type());
  const at::Tensor loss = at::empty({rows}, x.options().dtype(at::kFloat));
  const OnDevice on(x);
  const size_t bytes = aqlm_distill_loss_workspace_bytes(rows, vocab, ids.size(1), dtype_of(x, "logits"));
  at::Tensor ws;
  if (bytes) ws = at::empty({(int64_t)bytes}, x.options().dtype(at::kByte));
  done(aqlm_distill_loss(x.data_ptr(), row_stride(x), dtype_of(x, "logits"), t.data_ptr(), row_stride(t),
                         dtype_of(t, "teacher_logits"), (const int32_t*)pi, row_stride(ids), (const float*)lse,
                         (const float*)w, (float)number(a[5]), loss.data_ptr<float>(), want ? grad.data_ptr() : nullptr,
                         want ? row_stride(grad) : 0, rows, vocab, ids.size(1), bytes ? ws.data_ptr() : nullptr, bytes,
                         stream_of(a[8])),
       "aqlm_distill_loss");
  written(a[7]);
  return Py_BuildValue("NNN", wrap(loss), want ? wrap(grad) : none(), bytes ? wrap(ws) : none());
}

// logits, uniform, temperature, top_k, top_p, min_p, return_logprob, stream; the last of the results is the workspace
PyObject* sample(PyObject* const* a) {
  const at::Tensor& x = rows2(a[0], "logits");
  const int64_t rows = x.size(0);
  const void* u = vector(tensor(a[1], "uniform"), "uniform", x, rows, at::kFloat);
  auto rule = [&](int i, const char* name, at::ScalarType type) -> const void* {
    return given(a[i]) ? vector(tensor(a[i], name), name, x, rows, type) : nullptr;
  };
  aqlm_sampling r{};
  r.temperature = (const float*)rule(2, "temperature", at::kFloat);
  r.top_k = (const int32_t*)rule(3, "top_k", at::kInt);
  r.top_p = (const float*)rule(4, "top_p", at::kFloat);
  r.min_p = (const float*)rule(5, "min_p", at::kFloat);
  const bool want = truth(a[6]);
  const at::Tensor tokens = at::empty({rows}, x.options().dtype(at::kInt));
  at::Tensor logprob;
  if (want) logprob = at::empty({rows}, x.options().dtype(at::kFloat));
  const size_t bytes = aqlm_sample_workspace_bytes(rows, x.size(1), &r);
  at::Tensor ws;
  if (bytes) ws = at::empty({(int64_t)bytes}, x.options().dtype(at::kByte));
  const OnDevice on(x);
  done(aqlm_sample(x.data_ptr(), row_stride(x), dtype_of(x, "logits"), rows, x.size(1), (const float*)u, &r,
                   tokens.data_ptr<int32_t>(), want ? logprob.data_ptr<float>() : nullptr, bytes ? ws.data_ptr() : nullptr,
                   bytes, stream_of(a[7])),
       "aqlm_sample");
  return Py_BuildValue("NNN", wrap(tokens), want ? wrap(logprob) : none(), bytes ? wrap(ws) : none());
}

// Whether a stream (its handle) is recording a graph.
PyObject* capturing(PyObject* const* a) {
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  const hipError_t e = hipStreamIsCapturing((hipStream_t)stream_of(a[0]), &status);
  if (e != hipSuccess) throw std::runtime_error(std::string("hipStreamIsCapturing: ") + hipGetErrorString(e));
  return PyBool_FromLong(status != hipStreamCaptureStatusNone);
}

PyObject* set_check(PyObject* const* a) {
  Py_INCREF(a[0]);
  Py_XDECREF(g_check);
  g_check = a[0];
  return none();
}

#define AQLM_ENTRY(F, N) \
  { #F, (PyCFunction)(void (*)(void))entry<F, N>, METH_FASTCALL, nullptr }
PyMethodDef methods[] = {AQLM_ENTRY(rope, 11),           AQLM_ENTRY(rope_backward, 13),   AQLM_ENTRY(paged_append, 15),
                         AQLM_ENTRY(paged_attention, 14), AQLM_ENTRY(process_logits, 12), AQLM_ENTRY(capturing, 1),
                         AQLM_ENTRY(set_check, 1),      AQLM_ENTRY(embed, 5),            AQLM_ENTRY(embed_backward, 7),
                         AQLM_ENTRY(layer_norm, 9),     AQLM_ENTRY(layer_norm_backward, 9),
                         AQLM_ENTRY(distill_loss, 9),   AQLM_ENTRY(sample, 8),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_block", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__block(void) { return PyModule_Create(&module); }
