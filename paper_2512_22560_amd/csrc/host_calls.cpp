// What the binding checks and unpacks of its tensors in front of the calls that an engine makes every step, as a Python module of its
// own: the smallest of these calls are shorter on the GPU than that was in Python.  A write of five tokens (2.6 us on the GPU): 9.8 us
// with 5.8 of Python, 5.1 with this module; of 512 single tokens (7.2 on the GPU) 10.5 -> 7.2; a decode step over 37 short contexts
// (two launches) 10.6 -> 8.4.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>
#include <initializer_list>

#include "rollattn.h"

namespace {

decltype(&kv_write_rope) call_kv_write_rope = nullptr;      // the library's, as `bind` was given them
decltype(&attn_decode) call_attn_decode = nullptr;
decltype(&attn_append) call_attn_append = nullptr;
decltype(&kv_write_norm_rope) call_kv_write_norm_rope = nullptr;
decltype(&attn_tree_mask) call_attn_tree_mask = nullptr;
decltype(&attn_tree) call_attn_tree = nullptr;
decltype(&kv_accept) call_kv_accept = nullptr;

struct Refusal {
  PyObject* kind;
  const char* what;
};
struct Raised {};                                           // a Python error is set already

struct Unlocked {                                           // without the interpreter's lock
  PyThreadState* const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) throw Refusal{PyExc_TypeError, "librollattn takes torch tensors"};
  return THPVariable_Unpack(o);
}

const at::Tensor* maybe(PyObject* o) { return o == Py_None ? nullptr : &tensor(o); }

const at::Tensor& dense(const at::Tensor& t) {
  if (!t.is_contiguous()) throw Refusal{PyExc_ValueError, "librollattn takes dense row-major arrays"};
  return t;
}

const at::Tensor* dense(const at::Tensor* t) { return t ? &dense(*t) : nullptr; }

void* address(const at::Tensor& t) { return t.data_ptr(); }
void* address(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

int32_t whole(int64_t n) {
  if (n < INT32_MIN || n > INT32_MAX) throw Refusal{PyExc_ValueError, "librollattn counts in 32 bits"};
  return (int32_t)n;
}

int64_t number(PyObject* o) {
  PyObject* n = PyNumber_Long(o);
  if (!n) throw Raised{};
  const long long v = PyLong_AsLongLong(n);
  Py_DECREF(n);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}

int dtype_code(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return ROLLATTN_F32;
    case at::kBFloat16: return ROLLATTN_BF16;
    case at::kByte:
    case at::kFloat8_e4m3fn: return ROLLATTN_FP8_E4M3;
    case at::kChar: return ROLLATTN_INT8_HEAD;
    default:
      PyErr_Format(PyExc_TypeError, "unsupported element type torch.%s", c10::toString(t.scalar_type()));
      throw Raised{};
  }
}

// E4M3 codes have a scale for each page, or with scales [num_pages, Hkv] one for each page and KV head, as int8 ones always do.
int kv_code(const at::Tensor& pages, const at::Tensor* k_scale, const at::Tensor* v_scale) {
  const int code = dtype_code(pages);
  if (code < ROLLATTN_FP8_E4M3 || !k_scale || !v_scale) return code;
  if (k_scale->scalar_type() != at::kFloat || v_scale->scalar_type() != at::kFloat) throw Refusal{PyExc_TypeError, "scales are float32"};
  const int64_t held[] = {pages.size(0), pages.size(1)}, n = held[0];
  if (k_scale->sizes() == at::IntArrayRef(held, 2) && v_scale->sizes() == at::IntArrayRef(held, 2))
    return code == ROLLATTN_INT8_HEAD ? ROLLATTN_INT8_HEAD : ROLLATTN_FP8_E4M3_HEAD;
  if (code == ROLLATTN_INT8_HEAD) throw Refusal{PyExc_ValueError, "scales of each page and KV head are [num_pages, Hkv]"};
  const int64_t nk = k_scale->numel(), nv = v_scale->numel();
  if (!(k_scale->dim() == 1 && v_scale->dim() == 1 && nk >= n && nv >= n) && !(nk == n && nv == n))
    throw Refusal{PyExc_ValueError, "scales of both pools are [num_pages], or of each page and KV head [num_pages, Hkv]"};
  return code;
}

void dims(const at::Tensor& t, int n, const char* what) {
  if (t.dim() != n) throw Refusal{PyExc_ValueError, what};
}

// int32 arrays of at least so many entries
void ints(const at::Tensor& t, int64_t least, const char* what) {
  if (t.scalar_type() != at::kInt) throw Refusal{PyExc_TypeError, what};
  if (t.numel() < least) throw Refusal{PyExc_ValueError, what};
}

// Elements between the rows of consecutive tokens; a token's heads lie side by side.
int64_t row_stride(const at::Tensor& t) {
  const int64_t heads = t.size(1), d = t.size(2);
  if ((t.stride(1) == d || heads == 1) && t.stride(2) == 1) {
    if (t.size(0) <= 1) return heads * d;
    // (one row for all of them, say: a step of 0 means dense rows to the library)
    if (t.stride(0) < heads * d) throw Refusal{PyExc_ValueError, "the rows of tokens do not overlap"};
    return t.stride(0);
  }
  if (t.numel()) throw Refusal{PyExc_ValueError, "the heads of a token lie side by side"};
  return heads * d;
}

// (the kernels would read host addresses, or another GPU's, as this one's)
void one_gpu(std::initializer_list<const at::Tensor*> all) {
  int64_t device = -1;
  for (const at::Tensor* t : all) {
    if (!t) continue;
    if (!t->is_cuda() || (device >= 0 && t->get_device() != device)) throw Refusal{PyExc_ValueError, "tensors are on one GPU"};
    device = t->get_device();
  }
}

// the chunks of B trajectories
void chunks(const at::Tensor& q_lens, const at::Tensor& q_offsets, const at::Tensor& table) {
  ints(q_lens, table.size(0), "q_lens is [B] int32");
  ints(q_offsets, table.size(0) + 1, "q_offsets is [B + 1] int32");
}

rollattn_desc descriptor(const at::Tensor& rows, int64_t hq, const at::Tensor& k_pages, const at::Tensor& table, float sm_scale, const at::Tensor* k_scale,
                         const at::Tensor* v_scale) {
  dims(k_pages, 4, "pools are [num_pages, Hkv, page_size, D]");
  dims(table, 2, "page_table is [B, max_pages] int32");
  ints(table, 0, "page_table is [B, max_pages] int32");
  rollattn_desc d{};
  d.batch = whole(table.size(0));
  d.num_q_heads = whole(hq);
  d.num_kv_heads = whole(k_pages.size(1));
  d.head_dim = whole(k_pages.size(3));
  d.page_size = whole(k_pages.size(2));
  d.max_pages_per_seq = whole(table.size(1));
  d.num_pages = k_pages.size(0);
  d.q_dtype = dtype_code(rows);
  d.kv_dtype = kv_code(k_pages, k_scale, v_scale);
  d.sm_scale = sm_scale;
  return d;
}

template <class F>
PyObject* guarded(Py_ssize_t nargs, Py_ssize_t want, F&& f) {
  if (nargs != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments instead of %zd", nargs, want);
    return nullptr;
  }
  try {
    return f();
  } catch (const Refusal& r) {
    PyErr_SetString(r.kind, r.what);
  } catch (const Raised&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "host_calls");
  }
  return nullptr;
}

// q, k_new, v_new, q_lens, q_offsets, k_pages, v_pages, page_table, ctx_lens, cos_sin, max_q_len, positions, pair_axes, interleaved, k_scale,
// v_scale, q_out, stream; with norms: q_weight, k_weight, eps
PyObject* write_rope(PyObject* const* args, Py_ssize_t nargs, bool norms) {
  return guarded(nargs, norms ? 21 : 18, [&]() -> PyObject* {
    const at::Tensor *q = maybe(args[0]), &k_new = tensor(args[1]), &v_new = tensor(args[2]);
    const at::Tensor &q_lens = dense(tensor(args[3])), &q_offsets = dense(tensor(args[4])), &k_pages = dense(tensor(args[5])), &v_pages = dense(tensor(args[6]));
    const at::Tensor &page_table = dense(tensor(args[7])), &ctx_lens = dense(tensor(args[8])), &cos_sin = dense(tensor(args[9]));
    const at::Tensor *positions = dense(maybe(args[11])), *k_scale = dense(maybe(args[14])), *v_scale = dense(maybe(args[15])), *q_out = dense(maybe(args[16]));
    dims(k_new, 3, "k_new and v_new are [total_q, Hkv, D] rows of the pools");
    dims(k_pages, 4, "pools are [num_pages, Hkv, page_size, D]");
    const int64_t total_q = k_new.size(0), hkv = k_new.size(1), d = k_new.size(2);
    if (v_new.sizes() != k_new.sizes() || v_pages.sizes() != k_pages.sizes() || hkv != k_pages.size(1) || d != k_pages.size(3))
      throw Refusal{PyExc_ValueError, "k_new and v_new are [total_q, Hkv, D] rows of the pools"};
    if (v_new.scalar_type() != k_new.scalar_type() || v_pages.scalar_type() != k_pages.scalar_type() || (q && q->scalar_type() != k_new.scalar_type()))
      throw Refusal{PyExc_TypeError, "q, k_new and v_new are of one type, and so are the pools"};
    dims(cos_sin, 2, "cos_sin is [num_positions, rot_dim] float32");
    if (cos_sin.scalar_type() != at::kFloat) throw Refusal{PyExc_TypeError, "cos_sin is [num_positions, rot_dim] float32"};
    rollattn_rope rope{};
    int64_t hq = hkv;
    if (q) {
      dims(*q, 3, "q is [total_q, Hq, D]");
      hq = q->size(1);
      if (q->size(0) != total_q || q->size(2) != d) throw Refusal{PyExc_ValueError, "q is [total_q, Hq, D]"};
      rope.q_stride = row_stride(*q);
      if (!q_out || q_out->sizes() != q->sizes() || q_out->scalar_type() != q->scalar_type()) throw Refusal{PyExc_ValueError, "q_out takes the rotated q"};
    } else if (q_out) {
      throw Refusal{PyExc_ValueError, "q_out takes the rotated q"};
    }
    int64_t axes = 1;
    if (positions) {
      if (positions->dim() == 2) axes = positions->size(0);
      if (positions->scalar_type() != at::kInt || positions->numel() != axes * total_q || positions->dim() > 2)
        throw Refusal{PyExc_ValueError, "positions is [axes, total_q] int32"};
    }
    if (args[12] != Py_None) {
      char* bytes;
      Py_ssize_t n;
      if (PyBytes_AsStringAndSize(args[12], &bytes, &n)) throw Raised{};
      if (2 * n != cos_sin.size(1)) throw Refusal{PyExc_ValueError, "pair_axes has an axis for each pair"};
      rope.pair_axes = (const uint8_t*)bytes;
    } else if (axes > 1) {
      throw Refusal{PyExc_ValueError, "several axes need pair_axes"};
    }
    const int turned = PyObject_IsTrue(args[13]);
    if (turned < 0) throw Raised{};
    rope.cos_sin = (const float*)address(cos_sin);
    rope.positions = (const int32_t*)address(positions);
    rope.num_positions = whole(cos_sin.size(0));
    rope.rot_dim = whole(cos_sin.size(1));
    rope.num_axes = whole(axes);
    rope.interleaved = turned;
    rope.k_stride = row_stride(k_new);
    rope.v_stride = row_stride(v_new);
    rollattn_norm norm{};
    if (norms) {
      const at::Tensor *q_weight = dense(maybe(args[18])), &k_weight = dense(tensor(args[19]));
      if (k_weight.scalar_type() != at::kFloat || (q_weight && q_weight->scalar_type() != at::kFloat)) throw Refusal{PyExc_TypeError, "weights of norms are [D] float32"};
      if (k_weight.numel() != d || (q && !q_weight) || (q_weight && q_weight->numel() != d)) throw Refusal{PyExc_ValueError, "weights of norms are [D] float32"};
      norm.q_weight = (const float*)address(q_weight);
      norm.k_weight = (const float*)address(k_weight);
      norm.eps = (float)PyFloat_AsDouble(args[20]);
      if (PyErr_Occurred()) throw Raised{};
    }
    const rollattn_desc desc = descriptor(k_new, hq, k_pages, page_table, 1.f, k_scale, v_scale);
    ints(ctx_lens, page_table.size(0), "ctx_lens is [B] int32");
    chunks(q_lens, q_offsets, page_table);
    if (norms) one_gpu({q, &k_new, &v_new, &q_lens, &q_offsets, &k_pages, &v_pages, &page_table, &ctx_lens, &cos_sin, positions, k_scale, v_scale, q_out, maybe(args[18]), &tensor(args[19])});
    const int32_t total = whole(total_q), longest = whole(number(args[10]));
    void* const stream = (void*)(uintptr_t)number(args[17]);
    void *const p_q = address(q), *const p_k = address(k_new), *const p_v = address(v_new), *const p_out = address(q_out), *const p_kp = address(k_pages), *const p_vp = address(v_pages);
    const int32_t *const p_lens = (int32_t*)address(q_lens), *const p_off = (int32_t*)address(q_offsets), *const p_table = (int32_t*)address(page_table), *const p_ctx = (int32_t*)address(ctx_lens);
    float *const p_ks = (float*)address(k_scale), *const p_vs = (float*)address(v_scale);
    int rc;
    {
      const Unlocked other_threads_run;
      if (norms) rc = call_kv_write_norm_rope(&desc, &rope, &norm, p_q, p_k, p_v, p_lens, p_off, total, longest, p_out, p_kp, p_vp, p_table, p_ctx, p_ks, p_vs, stream);
      else rc = call_kv_write_rope(&desc, &rope, p_q, p_k, p_v, p_lens, p_off, total, longest, p_out, p_kp, p_vp, p_table, p_ctx, p_ks, p_vs, stream);
    }
    return PyLong_FromLong(rc);
  });
}

PyObject* host_kv_write_rope(PyObject*, PyObject* const* args, Py_ssize_t nargs) { return write_rope(args, nargs, false); }
PyObject* host_kv_write_norm_rope(PyObject*, PyObject* const* args, Py_ssize_t nargs) { return write_rope(args, nargs, true); }

// The descriptor of an attention call.
rollattn_desc attention(const at::Tensor& q, const at::Tensor& out, const at::Tensor& k_pages, const at::Tensor& v_pages, const at::Tensor& table, const at::Tensor& ctx_lens,
                        PyObject* scale, const at::Tensor* k_scale, const at::Tensor* v_scale) {
  if (q.dim() < 2) throw Refusal{PyExc_ValueError, "query rows are [rows, Hq, D]"};
  if (v_pages.sizes() != k_pages.sizes() || dtype_code(v_pages) != dtype_code(k_pages)) throw Refusal{PyExc_ValueError, "both pools are of one size and type"};
  if (out.numel() < q.numel() || out.scalar_type() != q.scalar_type()) throw Refusal{PyExc_ValueError, "out takes a row for each of q's, of its type"};
  const double sm_scale = PyFloat_AsDouble(scale);
  if (sm_scale == -1. && PyErr_Occurred()) throw Raised{};
  rollattn_desc desc = descriptor(q, q.size(1), k_pages, table, (float)sm_scale, k_scale, v_scale);
  if (q.numel() != q.size(0) * q.size(1) * k_pages.size(3)) throw Refusal{PyExc_ValueError, "query rows are [rows, Hq, D]"};
  ints(ctx_lens, table.size(0), "ctx_lens is [B] int32");
  desc.k_scale = (const float*)address(k_scale);
  desc.v_scale = (const float*)address(v_scale);
  return desc;
}

// q, k_pages, v_pages, page_table, ctx_lens, sm_scale, k_scale, v_scale, out, workspace, stream
PyObject* host_attn_decode(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded(nargs, 11, [&]() -> PyObject* {
    const at::Tensor &q = dense(tensor(args[0])), &k_pages = dense(tensor(args[1])), &v_pages = dense(tensor(args[2])), &page_table = dense(tensor(args[3]));
    const at::Tensor &ctx_lens = dense(tensor(args[4])), *k_scale = dense(maybe(args[6])), *v_scale = dense(maybe(args[7])), &out = dense(tensor(args[8]));
    const at::Tensor& workspace = tensor(args[9]);
    const rollattn_desc desc = attention(q, out, k_pages, v_pages, page_table, ctx_lens, args[5], k_scale, v_scale);
    if (q.size(0) < page_table.size(0)) throw Refusal{PyExc_ValueError, "a decode step has a query row for each trajectory"};
    void* const stream = (void*)(uintptr_t)number(args[10]);
    void *const p_q = address(q), *const p_kp = address(k_pages), *const p_vp = address(v_pages), *const p_out = address(out), *const p_ws = address(workspace);
    const int32_t *const p_table = (int32_t*)address(page_table), *const p_ctx = (int32_t*)address(ctx_lens);
    const size_t room = (size_t)workspace.nbytes();
    int rc;
    {
      const Unlocked other_threads_run;
      rc = call_attn_decode(&desc, p_q, p_kp, p_vp, p_table, p_ctx, p_out, p_ws, room, stream);
    }
    return PyLong_FromLong(rc);
  });
}

// q_chunk, q_lens, q_offsets, k_pages, v_pages, page_table, ctx_lens, sm_scale, max_q_len, k_scale, v_scale, out, workspace, stream
PyObject* host_attn_append(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded(nargs, 14, [&]() -> PyObject* {
    const at::Tensor &q = dense(tensor(args[0])), &q_lens = dense(tensor(args[1])), &q_offsets = dense(tensor(args[2])), &k_pages = dense(tensor(args[3]));
    const at::Tensor &v_pages = dense(tensor(args[4])), &page_table = dense(tensor(args[5])), &ctx_lens = dense(tensor(args[6]));
    const at::Tensor *k_scale = dense(maybe(args[9])), *v_scale = dense(maybe(args[10])), &out = dense(tensor(args[11])), &workspace = tensor(args[12]);
    const rollattn_desc desc = attention(q, out, k_pages, v_pages, page_table, ctx_lens, args[7], k_scale, v_scale);
    chunks(q_lens, q_offsets, page_table);
    const int32_t total = whole(q.size(0)), longest = whole(number(args[8]));
    void* const stream = (void*)(uintptr_t)number(args[13]);
    void *const p_q = address(q), *const p_kp = address(k_pages), *const p_vp = address(v_pages), *const p_out = address(out), *const p_ws = address(workspace);
    const int32_t *const p_lens = (int32_t*)address(q_lens), *const p_off = (int32_t*)address(q_offsets), *const p_table = (int32_t*)address(page_table), *const p_ctx = (int32_t*)address(ctx_lens);
    const size_t room = (size_t)workspace.nbytes();
    int rc;
    {
      const Unlocked other_threads_run;
      rc = call_attn_append(&desc, p_q, p_lens, p_off, total, longest, p_kp, p_vp, p_table, p_ctx, p_out, p_ws, room, stream);
    }
    return PyLong_FromLong(rc);
  });
}

// parents, q_lens, q_offsets, ctx_lens, max_q_len, tree_mask, positions, stream
PyObject* host_attn_tree_mask(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded(nargs, 8, [&]() -> PyObject* {
    const at::Tensor &parents = dense(tensor(args[0])), &q_lens = dense(tensor(args[1])), &q_offsets = dense(tensor(args[2])), &ctx_lens = dense(tensor(args[3]));
    const at::Tensor &mask = dense(tensor(args[5])), *positions = dense(maybe(args[6]));
    dims(parents, 1, "parents is [total_q] int32");
    ints(parents, 0, "parents is [total_q] int32");
    dims(q_lens, 1, "q_lens is [B] int32");
    const int64_t total_q = parents.size(0), batch = q_lens.size(0);
    ints(q_lens, batch, "q_lens is [B] int32");
    ints(q_offsets, batch + 1, "q_offsets is [B + 1] int32");
    ints(ctx_lens, batch, "ctx_lens is [B] int32");
    if (mask.scalar_type() != at::kLong) throw Refusal{PyExc_TypeError, "tree_mask is [total_q, mask_words] int64"};
    if (mask.dim() != 2 || mask.size(0) != total_q) throw Refusal{PyExc_ValueError, "tree_mask is [total_q, mask_words] int64"};
    if (positions) {
      ints(*positions, 0, "positions is [total_q] int32");
      if (positions->numel() != total_q) throw Refusal{PyExc_ValueError, "positions is [total_q] int32"};
    }
    one_gpu({&parents, &q_lens, &q_offsets, &ctx_lens, &mask, positions});
    const int32_t b = whole(batch), total = whole(total_q), longest = whole(number(args[4])), words = whole(mask.size(1));
    void* const stream = (void*)(uintptr_t)number(args[7]);
    const int32_t *const p_par = (int32_t*)address(parents), *const p_lens = (int32_t*)address(q_lens), *const p_off = (int32_t*)address(q_offsets), *const p_ctx = (int32_t*)address(ctx_lens);
    uint64_t* const p_mask = (uint64_t*)address(mask);
    int32_t* const p_pos = (int32_t*)address(positions);
    int rc;
    {
      const Unlocked other_threads_run;
      rc = call_attn_tree_mask(p_par, p_lens, p_off, p_ctx, b, total, longest, p_mask, words, p_pos, stream);
    }
    return PyLong_FromLong(rc);
  });
}

// q, q_lens, q_offsets, tree_mask, k_pages, v_pages, page_table, ctx_lens, sm_scale, max_q_len, k_scale, v_scale, out, lse, workspace, stream
PyObject* host_attn_tree(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded(nargs, 16, [&]() -> PyObject* {
    const at::Tensor &q = dense(tensor(args[0])), &q_lens = dense(tensor(args[1])), &q_offsets = dense(tensor(args[2])), &mask = dense(tensor(args[3]));
    const at::Tensor &k_pages = dense(tensor(args[4])), &v_pages = dense(tensor(args[5])), &page_table = dense(tensor(args[6])), &ctx_lens = dense(tensor(args[7]));
    const at::Tensor *k_scale = dense(maybe(args[10])), *v_scale = dense(maybe(args[11])), &out = dense(tensor(args[12])), *lse = dense(maybe(args[13])), &workspace = dense(tensor(args[14]));
    const rollattn_desc desc = attention(q, out, k_pages, v_pages, page_table, ctx_lens, args[8], k_scale, v_scale);
    chunks(q_lens, q_offsets, page_table);
    if (mask.scalar_type() != at::kLong) throw Refusal{PyExc_TypeError, "tree_mask is [total_q, mask_words] int64"};
    if (mask.dim() != 2 || mask.size(0) != q.size(0)) throw Refusal{PyExc_ValueError, "tree_mask is [total_q, mask_words] int64"};
    if (lse && (lse->scalar_type() != at::kFloat || lse->numel() != q.size(0) * q.size(1))) throw Refusal{PyExc_ValueError, "lse is [total_q, Hq] float32"};
    one_gpu({&q, &q_lens, &q_offsets, &mask, &k_pages, &v_pages, &page_table, &ctx_lens, k_scale, v_scale, &out, lse, &workspace});
    const int32_t total = whole(q.size(0)), longest = whole(number(args[9])), words = whole(mask.size(1));
    void* const stream = (void*)(uintptr_t)number(args[15]);
    void *const p_q = address(q), *const p_kp = address(k_pages), *const p_vp = address(v_pages), *const p_out = address(out), *const p_ws = address(workspace);
    const int32_t *const p_lens = (int32_t*)address(q_lens), *const p_off = (int32_t*)address(q_offsets), *const p_table = (int32_t*)address(page_table), *const p_ctx = (int32_t*)address(ctx_lens);
    const uint64_t* const p_mask = (uint64_t*)address(mask);
    float* const p_lse = (float*)address(lse);
    const size_t room = (size_t)workspace.nbytes();
    int rc;
    {
      const Unlocked other_threads_run;
      rc = call_attn_tree(&desc, p_q, p_lens, p_off, total, longest, p_mask, words, p_kp, p_vp, p_table, p_ctx, p_out, p_lse, p_ws, room, stream);
    }
    return PyLong_FromLong(rc);
  });
}

// accepted, accept_lens, q_lens, q_offsets, k_pages, v_pages, page_table, ctx_lens, max_q_len, k_scale, v_scale, stream
PyObject* host_kv_accept(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded(nargs, 12, [&]() -> PyObject* {
    const at::Tensor &accepted = dense(tensor(args[0])), &accept_lens = dense(tensor(args[1])), &q_lens = dense(tensor(args[2])), &q_offsets = dense(tensor(args[3]));
    const at::Tensor &k_pages = dense(tensor(args[4])), &v_pages = dense(tensor(args[5])), &page_table = dense(tensor(args[6])), &ctx_lens = dense(tensor(args[7]));
    const at::Tensor *k_scale = dense(maybe(args[9])), *v_scale = dense(maybe(args[10]));
    dims(k_pages, 4, "pools are [num_pages, Hkv, page_size, D]");
    if (v_pages.sizes() != k_pages.sizes() || dtype_code(v_pages) != dtype_code(k_pages)) throw Refusal{PyExc_ValueError, "both pools are of one size and type"};
    rollattn_desc desc = descriptor(k_pages, k_pages.size(1), k_pages, page_table, 1.f, k_scale, v_scale);
    desc.q_dtype = desc.kv_dtype == ROLLATTN_F32 ? ROLLATTN_F32 : ROLLATTN_BF16;
    dims(accepted, 1, "accepted is [total_q] int32");
    ints(accepted, 0, "accepted is [total_q] int32");
    ints(accept_lens, page_table.size(0), "accept_lens is [B] int32");
    ints(ctx_lens, page_table.size(0), "ctx_lens is [B] int32");
    chunks(q_lens, q_offsets, page_table);
    one_gpu({&accepted, &accept_lens, &q_lens, &q_offsets, &k_pages, &v_pages, &page_table, &ctx_lens, k_scale, v_scale});
    const int32_t total = whole(accepted.size(0)), longest = whole(number(args[8]));
    void* const stream = (void*)(uintptr_t)number(args[11]);
    void *const p_kp = address(k_pages), *const p_vp = address(v_pages);
    const int32_t *const p_acc = (int32_t*)address(accepted), *const p_alen = (int32_t*)address(accept_lens), *const p_lens = (int32_t*)address(q_lens), *const p_off = (int32_t*)address(q_offsets);
    const int32_t *const p_table = (int32_t*)address(page_table), *const p_ctx = (int32_t*)address(ctx_lens);
    float *const p_ks = (float*)address(k_scale), *const p_vs = (float*)address(v_scale);
    int rc;
    {
      const Unlocked other_threads_run;
      rc = call_kv_accept(&desc, p_acc, p_alen, p_lens, p_off, total, longest, p_kp, p_vp, p_table, p_ctx, p_ks, p_vs, stream);
    }
    return PyLong_FromLong(rc);
  });
}

// addresses of the library's calls
PyObject* host_bind(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded(nargs, 7, [&]() -> PyObject* {
    call_kv_write_rope = (decltype(call_kv_write_rope))(uintptr_t)number(args[0]);
    call_attn_decode = (decltype(call_attn_decode))(uintptr_t)number(args[1]);
    call_attn_append = (decltype(call_attn_append))(uintptr_t)number(args[2]);
    call_kv_write_norm_rope = (decltype(call_kv_write_norm_rope))(uintptr_t)number(args[3]);
    call_attn_tree_mask = (decltype(call_attn_tree_mask))(uintptr_t)number(args[4]);
    call_attn_tree = (decltype(call_attn_tree))(uintptr_t)number(args[5]);
    call_kv_accept = (decltype(call_kv_accept))(uintptr_t)number(args[6]);
    Py_RETURN_NONE;
  });
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))host_bind, METH_FASTCALL, nullptr},
    {"kv_write_rope", (PyCFunction)(void (*)(void))host_kv_write_rope, METH_FASTCALL, nullptr},
    {"attn_decode", (PyCFunction)(void (*)(void))host_attn_decode, METH_FASTCALL, nullptr},
    {"attn_append", (PyCFunction)(void (*)(void))host_attn_append, METH_FASTCALL, nullptr},
    {"kv_write_norm_rope", (PyCFunction)(void (*)(void))host_kv_write_norm_rope, METH_FASTCALL, nullptr},
    {"attn_tree_mask", (PyCFunction)(void (*)(void))host_attn_tree_mask, METH_FASTCALL, nullptr},
    {"attn_tree", (PyCFunction)(void (*)(void))host_attn_tree, METH_FASTCALL, nullptr},
    {"kv_accept", (PyCFunction)(void (*)(void))host_kv_accept, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host_calls() { return PyModule_Create(&module); }
