// Python binding of the entry points whose calls are as short as their launches
// (the paged cache, its attention, the adapters): the arguments' checks, the
// results' memory on the current stream, and the library call, in one step
// each.  ops.py gives them their names, defaults and documentation.
//
// The same work in Python with ctypes takes 15 to 20 us a call, this 3 to 9 (13
// for the attention of drafted trees, which sets up TMA and launches two kernels);
// the kernels of a small call take 3 to 14.  A wrong argument raises ValueError
// before the library is reached; a status other than 0 is returned as an int.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>

#include <cmath>

#include "kvcache.cuh"

namespace {

using at::ScalarType;
using at::Tensor;

struct BadArgument {};  // a Python error has been set

[[noreturn]] void refuse(const char* format, const char* what = "", int64_t a = 0, int64_t b = 0, int64_t c = 0) {
  PyErr_Format(PyExc_ValueError, format, what, (long long)a, (long long)b, (long long)c);
  throw BadArgument{};
}

int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw BadArgument{};
  return v;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw BadArgument{};
  return v != 0;
}

bool given(PyObject* o) { return o != Py_None; }

const Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

bool on(const Tensor* t, int64_t index) { return t && t->is_cuda() && t->get_device() == index; }

// [tokens, heads, D], dense along D; heads < 0: any number.
const Tensor& heads(PyObject* o, ScalarType type, int64_t H, int64_t D, int64_t index, const char* what) {
  const Tensor* t = tensor(o);
  if (!on(t, index) || t->scalar_type() != type || t->dim() != 3 || t->size(2) != D || (H >= 0 && t->size(1) != H) ||
      t->stride(2) != 1)
    refuse(type == ScalarType::BFloat16
               ? "%s must be a bfloat16 CUDA tensor [tokens, heads, %lld] (heads as the call needs them) on device "
                 "%lld with unit last stride"
               : "%s must be a float32 CUDA tensor [tokens, heads, %lld] (heads as the call needs them) on device "
                 "%lld with unit last stride",
           what, D, index);
  return *t;
}

// The stride of an axis; 0 where it has one element, whose stride leads nowhere and may be anything.
int64_t step(const Tensor& t, int axis) { return t.size(axis) == 1 ? 0 : t.stride(axis); }

const Tensor& vector(PyObject* o, ScalarType type, int64_t n, int64_t index, const char* what) {
  const Tensor* t = tensor(o);
  if (!on(t, index) || t->scalar_type() != type || t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1))
    refuse(type == ScalarType::Long ? "%s must be a dense int64 CUDA tensor of %lld elements on device %lld"
                                    : "%s must be a dense int32 CUDA tensor of %lld elements on device %lld",
           what, n, index);
  return *t;
}

// [rows, cols], dense along a row; its row stride, at least cols, goes to ld (cols where there is one row).
const Tensor& rows(PyObject* o, ScalarType type, int64_t n, int64_t cols, int64_t index, const char* what,
                   int64_t* ld) {
  const Tensor* t = tensor(o);
  bool ok = on(t, index) && t->scalar_type() == type && t->dim() == 2 && t->size(0) == n && t->size(1) == cols &&
            (t->stride(1) == 1 || cols <= 1);
  if (ok) {
    *ld = n <= 1 ? cols : t->stride(0);
    ok = *ld >= cols;
  }
  if (!ok)
    refuse(type == ScalarType::BFloat16
               ? "%s must be a bfloat16 CUDA tensor [%lld, %lld] on device %lld with unit column stride"
               : "%s must be a float32 CUDA tensor [%lld, %lld] on device %lld with unit column stride",
           what, n, cols, index);
  return *t;
}

void dense(const Tensor& t, const char* what) {
  if (!t.is_contiguous()) refuse("%s must be dense", what);
}

Tensor fresh(at::IntArrayRef shape, ScalarType type, const Tensor& like) {
  return at::empty(shape, like.options().dtype(type));
}

struct Unlocked {  // other Python threads run while a launch waits for room in the stream's queue
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

PyObject* status_of(int st) { return PyLong_FromLong(st); }

template <typename... T>
PyObject* tuple_of(T&&... t) {
  PyObject* r = PyTuple_New(sizeof...(t));
  if (!r) throw BadArgument{};
  Py_ssize_t i = 0;
  ((PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(std::move(t)))), ...);  // it takes the references over
  return r;
}

template <typename F>
PyObject* guarded(F body) {
  HANDLE_TH_ERRORS
  try {
    return body();
  } catch (const BadArgument&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

void* stream_of(PyObject* o) { return reinterpret_cast<void*>(static_cast<intptr_t>(integer(o))); }

const mixfp4_kv_cache* cache_of(PyObject* o) {
  return reinterpret_cast<const mixfp4_kv_cache*>(static_cast<intptr_t>(integer(o)));
}

bool counted(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return false;
}

// (cache, index, k, v, slots, q, positions, cos_sin, interleaved, mode, out, stream)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!counted(n, 12)) return nullptr;
  return guarded([&]() -> PyObject* {
    const mixfp4_kv_cache* c = cache_of(a[0]);
    const int64_t index = integer(a[1]), D = c->head_dim;
    const Tensor* k0 = tensor(a[2]);
    if (!k0 || (k0->scalar_type() != ScalarType::BFloat16 && k0->scalar_type() != ScalarType::Float))
      refuse("%s must be a bfloat16 or float32 CUDA tensor", "k");
    const ScalarType type = k0->scalar_type();
    const Tensor& k = heads(a[2], type, c->heads, D, index, "k");
    const Tensor& v = heads(a[3], type, c->heads, D, index, "v");
    const int64_t T = k.size(0);
    if (v.size(0) != T) refuse("k and %s must have as many tokens", "v");
    const Tensor& slots = vector(a[4], ScalarType::Long, T, index, "slots");
    const int64_t* positions = nullptr;
    const float* angles = nullptr;
    int64_t table = 0, rot = 0;
    if (given(a[7])) {
      positions = vector(a[6], ScalarType::Long, T, index, "positions").const_data_ptr<int64_t>();
      const Tensor* cs = tensor(a[7]);
      if (!on(cs, index) || cs->scalar_type() != ScalarType::Float || cs->dim() != 2 || !cs->is_contiguous())
        refuse("%s must be a dense float32 CUDA tensor [positions, rot_dim]", "cos_sin");
      table = cs->size(0), rot = cs->size(1);
      if (rot % 2 != 0 || rot > D) refuse("%s must be even and at most head_dim", "rot_dim");
      angles = cs->const_data_ptr<float>();
    }
    Tensor out;
    const void* qp = nullptr;
    int64_t H = 0, qt = 0, qh = 0;
    if (given(a[5])) {
      const Tensor& q = heads(a[5], type, -1, D, index, "q");
      if (q.size(0) != T) refuse("%s must have as many tokens as k", "q");
      H = q.size(1), qt = step(q, 0), qh = step(q, 1), qp = q.const_data_ptr();
      if (given(a[10])) {
        out = heads(a[10], ScalarType::BFloat16, H, D, index, "out");
        if (out.size(0) != T) refuse("%s must have as many tokens as q", "out");
        dense(out, "out");
      } else {
        out = fresh({T, H, D}, ScalarType::BFloat16, k);
      }
    }
    const bool interleaved = truth(a[8]);
    if (given(a[10]) && qp &&
        mixfp4::append_overlaps(qp, qt, qh, H, k.const_data_ptr(), step(k, 0), step(k, 1), v.const_data_ptr(),
                                step(v, 0), step(v, 1),
                                type == ScalarType::Float ? MIXFP4_DTYPE_F32 : MIXFP4_DTYPE_BF16, T, rot, interleaved,
                                c->heads, D, out.const_data_ptr()))
      refuse("%s must not overlap k, v or q (it may be q itself, bf16 and dense, if the rotation is interleaved or over "
             "a multiple of 32 elements)", "out");
    const int mode = (int)integer(a[9]);
    void* stream = stream_of(a[11]);
    int st;
    {
      Unlocked unlocked;
      st = mixfp4_kv_append(qp, qt, qh, H, k.const_data_ptr(), step(k, 0), step(k, 1), v.const_data_ptr(), step(v, 0),
                            step(v, 1),
                            type == ScalarType::Float ? MIXFP4_DTYPE_F32 : MIXFP4_DTYPE_BF16, T, positions, angles,
                            table, rot, interleaved, c, slots.const_data_ptr<int64_t>(),
                            out.defined() ? out.mutable_data_ptr() : nullptr, mode, stream);
    }
    if (st) return status_of(st);
    if (!out.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(out));
  });
}

// (cache, index, slots, float32, k_out, v_out, stream)
PyObject* kv_gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!counted(n, 7)) return nullptr;
  return guarded([&]() -> PyObject* {
    const mixfp4_kv_cache* c = cache_of(a[0]);
    const int64_t index = integer(a[1]);
    const Tensor* s = tensor(a[2]);
    if (!s || s->dim() != 1) refuse("%s must be 1-D", "slots");
    const int64_t T = s->size(0);
    const Tensor& slots = vector(a[2], ScalarType::Long, T, index, "slots");
    const bool f32 = truth(a[3]);
    const ScalarType type = f32 ? ScalarType::Float : ScalarType::BFloat16;
    Tensor out[2];
    for (int i = 0; i < 2; ++i) {
      if (given(a[4 + i])) {
        out[i] = heads(a[4 + i], type, c->heads, c->head_dim, index, "out");
        if (out[i].size(0) != T) refuse("%s must have a row per slot", "out");
        dense(out[i], "out");
      } else {
        out[i] = fresh({T, c->heads, c->head_dim}, type, slots);
      }
    }
    void* stream = stream_of(a[6]);
    int st;
    {
      Unlocked unlocked;
      st = mixfp4_kv_gather(c, slots.const_data_ptr<int64_t>(), T, out[0].mutable_data_ptr(),
                            out[1].mutable_data_ptr(), f32 ? MIXFP4_DTYPE_F32 : MIXFP4_DTYPE_BF16, stream);
    }
    if (st) return status_of(st);
    return tuple_of(out[0], out[1]);
  });
}

const Tensor& table_of(PyObject* o, int64_t B, int64_t index) {
  const Tensor* table = tensor(o);
  if (!on(table, index) || table->scalar_type() != ScalarType::Int || table->dim() != 2 ||
      (B >= 0 && table->size(0) != B) || (table->stride(1) != 1 && table->size(1) > 1))
    refuse("%s must be an int32 CUDA tensor [%lld, pages] on device %lld with unit column stride", "block_table", B,
           index);
  return *table;
}
// A table's stride from row to row, at least its width.
int64_t table_step(const Tensor& table) {
  const int64_t pages = table.size(1);
  if (table.size(0) > 1 && table.stride(0) < pages) refuse("%s must not have overlapping rows", "block_table");
  return std::max(step(table, 0), pages);
}

// (cache, index, q, block_table, lengths, scale, window, out, lse, want_lse, workspace, stream)
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!counted(n, 12)) return nullptr;
  return guarded([&]() -> PyObject* {
    const mixfp4_kv_cache* c = cache_of(a[0]);
    const int64_t index = integer(a[1]), D = c->head_dim;
    const Tensor& q = heads(a[2], ScalarType::BFloat16, -1, D, index, "q");
    const int64_t B = q.size(0), H = q.size(1);
    if (H % c->heads != 0) refuse("%s must be a multiple of the cache's heads", "q_heads");
    const Tensor& table = table_of(a[3], B, index);
    const int64_t ts = table_step(table);
    const Tensor& lengths = vector(a[4], ScalarType::Int, B, index, "lengths");
    float scale = (float)std::pow((double)D, -0.5);
    if (given(a[5])) {
      const double v = PyFloat_AsDouble(a[5]);
      if (v == -1.0 && PyErr_Occurred()) throw BadArgument{};
      scale = (float)v;
    }
    const int64_t window = integer(a[6]);
    if (window < 0) refuse("%s must not be negative", "window");
    Tensor out, lse, workspace;
    if (given(a[7])) {
      out = heads(a[7], ScalarType::BFloat16, H, D, index, "out");
      if (out.size(0) != B) refuse("%s must have a row per sequence", "out");
      dense(out, "out");
    }
    if (given(a[8])) {
      const Tensor* t = tensor(a[8]);
      if (!on(t, index) || t->scalar_type() != ScalarType::Float || t->dim() != 2 || t->size(0) != B ||
          t->size(1) != H || !t->is_contiguous())
        refuse("%s must be a dense float32 CUDA tensor [%lld, %lld] on device %lld", "lse", B, H, index);
      lse = *t;
    }
    int64_t need = 0;
    if (given(a[10])) {
      const Tensor* t = tensor(a[10]);
      if (!on(t, index) || !t->is_contiguous())
        refuse("%s must be a dense CUDA tensor on device %lld", "workspace", index);
      workspace = *t;
      need = t->numel() * t->element_size();
    } else {
      if (const int st = mixfp4_paged_attention_workspace(c, B, H, &need)) return status_of(st);
      workspace = fresh({need}, ScalarType::Byte, q);
    }
    if (!out.defined()) out = fresh({B, H, D}, ScalarType::BFloat16, q);
    if (!lse.defined() && truth(a[9])) lse = fresh({B, H}, ScalarType::Float, q);
    void* stream = stream_of(a[11]);
    int st;
    {
      Unlocked unlocked;
      st = mixfp4_paged_attention(q.const_data_ptr(), step(q, 0), step(q, 1), B, H, c,
                                  table.const_data_ptr<int32_t>(), ts, table.size(1),
                                  lengths.const_data_ptr<int32_t>(), scale, window, out.mutable_data_ptr(),
                                  lse.defined() ? lse.mutable_data_ptr<float>() : nullptr,
                                  workspace.mutable_data_ptr(), need, stream);
    }
    if (st) return status_of(st);
    if (!lse.defined()) return THPVariable_Wrap(std::move(out));
    return tuple_of(out, lse);
  });
}

// Masks of drafts, int64: none, [t] for all sequences (`stride` 0), or [B, t].
const int64_t* masks(PyObject* o, int64_t B, int64_t t, int64_t index, int64_t* stride) {
  *stride = 0;
  if (!given(o)) return nullptr;
  const Tensor* m = tensor(o);
  const int64_t d = m ? m->dim() : 0;
  if (!on(m, index) || m->scalar_type() != ScalarType::Long || d < 1 || d > 2 || m->size(d - 1) != t ||
      (m->stride(d - 1) != 1 && t > 1) || (d == 2 && m->size(0) != B))
    refuse("%s must be an int64 CUDA tensor [%lld, %lld] or [%lld] with unit last stride", "mask", B, t, t);
  if (d == 2 && B > 1) *stride = m->stride(0);
  if (*stride != 0 && *stride < t) refuse("%s must not have overlapping rows", "mask");
  return m->const_data_ptr<int64_t>();
}

int64_t length_of(PyObject* o, const char* what) {
  const Tensor* t = tensor(o);
  if (!t || t->dim() != 1) refuse("%s must be a 1-D int32 CUDA tensor", what);
  return t->size(0);
}

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw BadArgument{};
  return v;
}

// (cache, index, q, block_table, lengths, mask, counts, scale, window, softcap, slopes, out, lse, want_lse, workspace,
// status_word, stream)
PyObject* tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!counted(n, 17)) return nullptr;
  return guarded([&]() -> PyObject* {
    const mixfp4_kv_cache* c = cache_of(a[0]);
    const int64_t index = integer(a[1]), D = c->head_dim;
    const Tensor* qp = tensor(a[2]);
    if (!on(qp, index) || qp->scalar_type() != ScalarType::BFloat16 || qp->dim() != 4 || qp->size(3) != D ||
        qp->stride(3) != 1)
      refuse("%s must be a bfloat16 CUDA tensor [sequences, drafts, heads, %lld] on device %lld with unit last stride", "q",
             D, index);
    const Tensor& q = *qp;
    const int64_t B = q.size(0), t = q.size(1), H = q.size(2);
    if (t > 64) refuse("%s must have at most 64 drafts of a sequence", "q");
    if (H % c->heads != 0) refuse("%s must be a multiple of the cache's heads", "q_heads");
    const Tensor& table = table_of(a[3], B, index);
    const Tensor& lengths = vector(a[4], ScalarType::Int, B, index, "lengths");
    int64_t mask_stride;
    const int64_t* mask = masks(a[5], B, t, index, &mask_stride);
    const int32_t* counts = nullptr;
    if (given(a[6])) counts = vector(a[6], ScalarType::Int, B, index, "counts").const_data_ptr<int32_t>();
    const float scale = given(a[7]) ? (float)number(a[7]) : (float)std::pow((double)D, -0.5);
    const int64_t window = integer(a[8]);
    if (window < 0) refuse("%s must not be negative", "window");
    const float softcap = (float)number(a[9]);
    if (!(softcap == 0.0f || (softcap >= 1e-6f && softcap <= 1e6f))) refuse("%s must be 0 or 1e-6 to 1e6", "softcap");
    const float* slopes = nullptr;
    if (given(a[10])) {
      const Tensor* s = tensor(a[10]);
      if (!on(s, index) || s->scalar_type() != ScalarType::Float || s->dim() != 1 || s->size(0) != H ||
          !s->is_contiguous())
        refuse("%s must be a dense float32 CUDA tensor of %lld elements on device %lld", "slopes", H, index);
      slopes = s->const_data_ptr<float>();
    }
    Tensor out, lse, workspace;
    if (given(a[11])) {
      const Tensor* o = tensor(a[11]);
      if (!on(o, index) || o->scalar_type() != ScalarType::BFloat16 || o->sizes() != q.sizes() || !o->is_contiguous())
        refuse("%s must be a dense bfloat16 CUDA tensor of q's shape", "out");
      out = *o;
    }
    if (given(a[12])) {
      const Tensor* s = tensor(a[12]);
      if (!on(s, index) || s->scalar_type() != ScalarType::Float || s->dim() != 3 || s->size(0) != B ||
          s->size(1) != t || s->size(2) != H || !s->is_contiguous())
        refuse("%s must be a dense float32 CUDA tensor [%lld, %lld, %lld]", "lse", B, t, H);
      lse = *s;
    }
    int64_t need = 0;
    if (given(a[14])) {
      const Tensor* w = tensor(a[14]);
      if (!on(w, index) || !w->is_contiguous())
        refuse("%s must be a dense CUDA tensor on device %lld", "workspace", index);
      workspace = *w;
      need = w->numel() * w->element_size();
    } else {
      if (const int st = mixfp4_tree_attention_workspace(c, B, t, H, &need)) return status_of(st);
      workspace = fresh({need}, ScalarType::Byte, q);
    }
    if (!out.defined()) out = fresh(q.sizes(), ScalarType::BFloat16, q);
    if (!lse.defined() && truth(a[13])) lse = fresh({B, t, H}, ScalarType::Float, q);
    uint32_t* status = reinterpret_cast<uint32_t*>(given(a[15]) ? static_cast<intptr_t>(integer(a[15])) : 0);
    void* stream = stream_of(a[16]);
    const int64_t ts = table_step(table);
    int st;
    {
      Unlocked unlocked;
      st = mixfp4_tree_attention(q.const_data_ptr(), step(q, 0), step(q, 1), step(q, 2), B, t, H, c,
                                 table.const_data_ptr<int32_t>(), ts, table.size(1),
                                 lengths.const_data_ptr<int32_t>(), mask, mask_stride, counts, scale, window, softcap,
                                 slopes, out.mutable_data_ptr(), lse.defined() ? lse.mutable_data_ptr<float>() : nullptr,
                                 workspace.mutable_data_ptr(), need, status, stream);
    }
    if (st) return status_of(st);
    if (!lse.defined()) return THPVariable_Wrap(std::move(out));
    return tuple_of(out, lse);
  });
}

// (cache, index, block_table, lengths, path, counts, out, stream)
PyObject* kv_accept(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!counted(n, 8)) return nullptr;
  return guarded([&]() -> PyObject* {
    const mixfp4_kv_cache* c = cache_of(a[0]);
    const int64_t index = integer(a[1]), B = length_of(a[3], "lengths");
    const Tensor& table = table_of(a[2], B, index);
    const Tensor& lengths = vector(a[3], ScalarType::Int, B, index, "lengths");
    const Tensor* path = tensor(a[4]);
    if (!on(path, index) || path->scalar_type() != ScalarType::Int || path->dim() != 2 || path->size(0) != B ||
        path->size(1) > 64 || (path->stride(1) != 1 && path->size(1) > 1) ||
        (B > 1 && path->stride(0) < path->size(1)))
      refuse("%s must be an int32 CUDA tensor [%lld, at most 64] on device %lld with unit column stride", "path", B, index);
    const Tensor& counts = vector(a[5], ScalarType::Int, B, index, "counts");
    Tensor out = given(a[6]) ? vector(a[6], ScalarType::Int, B, index, "out") : fresh({B}, ScalarType::Int, lengths);
    void* stream = stream_of(a[7]);
    const int64_t ts = table_step(table);
    int st;
    {
      Unlocked unlocked;
      st = mixfp4_kv_accept(c, table.const_data_ptr<int32_t>(), ts, table.size(1), lengths.const_data_ptr<int32_t>(),
                            counts.const_data_ptr<int32_t>(), B, path->const_data_ptr<int32_t>(), step(*path, 0),
                            path->size(1), out.mutable_data_ptr<int32_t>(), stream);
    }
    if (st) return status_of(st);
    return THPVariable_Wrap(std::move(out));
  });
}

// (cache, index, block_table, lengths, parents, fresh, table_out, lengths_out, stream)
PyObject* kv_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!counted(n, 9)) return nullptr;
  return guarded([&]() -> PyObject* {
    const mixfp4_kv_cache* c = cache_of(a[0]);
    const int64_t index = integer(a[1]), B = length_of(a[3], "lengths"), N = length_of(a[4], "parents");
    const Tensor& table = table_of(a[2], B, index);
    const Tensor& lengths = vector(a[3], ScalarType::Int, B, index, "lengths");
    const Tensor& parents = vector(a[4], ScalarType::Int, N, index, "parents");
    const Tensor& own = vector(a[5], ScalarType::Int, N, index, "fresh");
    const int64_t pages = table.size(1);
    Tensor out;
    if (given(a[6])) {
      out = table_of(a[6], N, index);
      if (out.size(1) != pages) refuse("%s must be as wide as block_table", "out");
      dense(out, "out");
    } else {
      out = fresh({N, pages}, ScalarType::Int, parents);
    }
    Tensor lens = given(a[7]) ? vector(a[7], ScalarType::Int, N, index, "out") : fresh({N}, ScalarType::Int, parents);
    void* stream = stream_of(a[8]);
    const int64_t ts = table_step(table);
    int st;
    {
      Unlocked unlocked;
      st = mixfp4_kv_fork(c, table.const_data_ptr<int32_t>(), ts, pages, lengths.const_data_ptr<int32_t>(), B,
                          parents.const_data_ptr<int32_t>(), own.const_data_ptr<int32_t>(), N,
                          out.mutable_data_ptr<int32_t>(), lens.mutable_data_ptr<int32_t>(), stream);
    }
    if (st) return status_of(st);
    return tuple_of(out, lens);
  });
}

// (cache, index, src, dst, stream)
PyObject* kv_copy_pages(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!counted(n, 5)) return nullptr;
  return guarded([&]() -> PyObject* {
    const mixfp4_kv_cache* c = cache_of(a[0]);
    const int64_t index = integer(a[1]), N = length_of(a[2], "src");
    const Tensor& src = vector(a[2], ScalarType::Int, N, index, "src");
    const Tensor& dst = vector(a[3], ScalarType::Int, N, index, "dst");
    void* stream = stream_of(a[4]);
    int st;
    {
      Unlocked unlocked;
      st = mixfp4_kv_copy_pages(c, src.const_data_ptr<int32_t>(), dst.const_data_ptr<int32_t>(), N, stream);
    }
    return status_of(st);
  });
}

struct Adapters {
  const Tensor *a, *b, *scaling;
  int64_t count, R, K, N;
};

Adapters adapters_of(PyObject* a, PyObject* b, PyObject* scaling, int64_t index) {
  Adapters ad{tensor(a), tensor(b), tensor(scaling), 0, 0, 0, 0};
  for (const Tensor* t : {ad.a, ad.b})
    if (!on(t, index) || t->scalar_type() != ScalarType::BFloat16 || t->dim() != 3 || !t->is_contiguous())
      refuse("%s must be dense 3-D bf16 CUDA tensors", "the adapters' a and b");
  ad.count = ad.a->size(0), ad.R = ad.a->size(1), ad.K = ad.a->size(2), ad.N = ad.b->size(1);
  if (ad.b->size(0) != ad.count || ad.b->size(2) != ad.R || !on(ad.scaling, index) ||
      ad.scaling->scalar_type() != ScalarType::Float || ad.scaling->dim() != 1 ||
      ad.scaling->size(0) != ad.count || !ad.scaling->is_contiguous())
    refuse("%s must fit together", "the adapters' tensors");
  return ad;
}

int64_t segments_of(PyObject* starts, PyObject* ids, int64_t T, int64_t index, const int32_t** s, const int32_t** i) {
  const Tensor* t = tensor(ids);
  if (!t || t->dim() != 1) refuse("%s must be a 1-D int32 CUDA tensor", "ids");
  const int64_t count = t->size(0);
  *i = vector(ids, ScalarType::Int, count, index, "ids").const_data_ptr<int32_t>();
  *s = vector(starts, ScalarType::Int, count + 1, index, "starts").const_data_ptr<int32_t>();
  if (count == 0 && T > 0) refuse("%s without a segment", "tokens");
  return count;
}

int64_t tokens_of(PyObject* x) {
  const Tensor* t = tensor(x);
  if (!t || t->dim() != 2) refuse("%s must be a 2-D bf16 CUDA tensor", "x");
  return t->size(0);
}

// A float32 [n, cols] result or base: the caller's (dense ones where `whole`), or new memory.
Tensor result(PyObject* o, int64_t n, int64_t cols, int64_t index, const char* what, int64_t* ld, bool whole,
              const Tensor& like) {
  if (!given(o)) {
    *ld = cols;
    return fresh({n, cols}, ScalarType::Float, like);
  }
  Tensor t = rows(o, ScalarType::Float, n, cols, index, what, ld);
  if (whole) dense(t, what);
  return t;
}

// (a, b, scaling, index, x, starts, ids, base, out, u, stream)
PyObject* lora(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!counted(n, 11)) return nullptr;
  return guarded([&]() -> PyObject* {
    const int64_t index = integer(a[3]);
    const Adapters ad = adapters_of(a[0], a[1], a[2], index);
    const int64_t T = tokens_of(a[4]);
    int64_t ldx, ldb = 0, ldo, ldu;
    const Tensor& x = rows(a[4], ScalarType::BFloat16, T, ad.K, index, "x", &ldx);
    const int32_t *starts, *ids;
    const int64_t S = segments_of(a[5], a[6], T, index, &starts, &ids);
    const float* base = nullptr;
    if (given(a[7])) base = rows(a[7], ScalarType::Float, T, ad.N, index, "base", &ldb).const_data_ptr<float>();
    Tensor out = result(a[8], T, ad.N, index, "out", &ldo, false, x);
    Tensor u = result(a[9], T, ad.R, index, "u", &ldu, true, x);
    void* stream = stream_of(a[10]);
    int st;
    {
      Unlocked unlocked;
      st = mixfp4_lora(x.const_data_ptr(), MIXFP4_DTYPE_BF16, T, ad.K, ldx, ad.a->const_data_ptr(),
                       ad.b->const_data_ptr(), ad.scaling->const_data_ptr<float>(), ad.count, ad.R, ad.N, starts, ids,
                       S, base, ldb, out.mutable_data_ptr<float>(), ldo, u.mutable_data_ptr<float>(), stream);
    }
    if (st) return status_of(st);
    return tuple_of(out, u);
  });
}

// (a, b, scaling, index, dy, x, u, starts, ids, base, out, da, db, workspace, stream)
PyObject* lora_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!counted(n, 15)) return nullptr;
  return guarded([&]() -> PyObject* {
    const int64_t index = integer(a[3]);
    const Adapters ad = adapters_of(a[0], a[1], a[2], index);
    const int64_t T = tokens_of(a[5]);
    int64_t ldx, ldy, ldb = 0, ldo, ldu;
    const Tensor& x = rows(a[5], ScalarType::BFloat16, T, ad.K, index, "x", &ldx);
    const Tensor& dy = rows(a[4], ScalarType::BFloat16, T, ad.N, index, "dy", &ldy);
    if (ad.N % 16 != 0) refuse("%s must be a multiple of 16", "N");
    const int32_t *starts, *ids;
    const int64_t S = segments_of(a[7], a[8], T, index, &starts, &ids);
    if (!given(a[6])) refuse("%s is what the forward pass returned", "u");
    const Tensor& u = rows(a[6], ScalarType::Float, T, ad.R, index, "u", &ldu);
    dense(u, "u");
    const float* base = nullptr;
    if (given(a[9])) base = rows(a[9], ScalarType::Float, T, ad.K, index, "base", &ldb).const_data_ptr<float>();
    Tensor grads[2];
    for (int i = 0; i < 2; ++i) {
      const Tensor& like = i == 0 ? *ad.a : *ad.b;
      if (given(a[11 + i])) {
        const Tensor* t = tensor(a[11 + i]);
        if (!on(t, index) || t->scalar_type() != ScalarType::Float || t->sizes() != like.sizes() ||
            !t->is_contiguous())
          refuse("%s must be a dense float32 tensor of the adapters' shape", i == 0 ? "da" : "db");
        grads[i] = *t;
      }
    }
    Tensor v = result(a[13], T, ad.R, index, "workspace", &ldu, true, x);
    Tensor out = result(a[10], T, ad.K, index, "out", &ldo, false, x);
    for (int i = 0; i < 2; ++i)
      if (!grads[i].defined()) grads[i] = fresh((i == 0 ? ad.a : ad.b)->sizes(), ScalarType::Float, x);
    void* stream = stream_of(a[14]);
    int st;
    {
      Unlocked unlocked;
      st = mixfp4_lora_backward(dy.const_data_ptr(), ldy, x.const_data_ptr(), ldx, MIXFP4_DTYPE_BF16, T, ad.K,
                                u.const_data_ptr<float>(), ad.a->const_data_ptr(), ad.b->const_data_ptr(),
                                ad.scaling->const_data_ptr<float>(), ad.count, ad.R, ad.N, starts, ids, S, base, ldb,
                                out.mutable_data_ptr<float>(), ldo, grads[0].mutable_data_ptr<float>(),
                                grads[1].mutable_data_ptr<float>(), v.mutable_data_ptr<float>(), stream);
    }
    if (st) return status_of(st);
    return tuple_of(out, grads[0], grads[1]);
  });
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(kv_append), METHOD(kv_gather),     METHOD(paged_attention),
                         METHOD(lora),      METHOD(lora_backward), METHOD(tree_attention),
                         METHOD(kv_accept), METHOD(kv_fork),       METHOD(kv_copy_pages),  {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
