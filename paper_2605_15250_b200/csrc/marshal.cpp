// Argument checks of the append calls and of the attention over E4M3 pages, for the Python binding: one function per C entry point that
// looks at the tensors, raises GqlaError for what the entry point does not take, and calls it on the current stream.
//
// These calls are made once per layer and step with a dozen tensors each.  Asking a tensor for its shape, type, strides, device and
// address from Python costs half a microsecond, and the calls took 14 to 20 us of host time for kernels of 3 to 13 us; from here the
// same questions cost nanoseconds.  The entry points come in as addresses (bind), so this module links no part of the CUDA library.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <algorithm>
#include <cstring>
#include <initializer_list>
#include <stdexcept>
#include <string>

#include "../../include/gqla.h"

namespace {

struct Refusal : std::runtime_error {
    using std::runtime_error::runtime_error;
};
struct PythonError {};  // an exception of the interpreter is set

PyObject* g_error = nullptr;  // GqlaError
struct Entries {
    decltype(&gqla_append_rope) append_rope;
    decltype(&gqla_append_rope_fp8) append_rope_fp8;
    decltype(&gqla_append_planes_fp8) append_planes_fp8;
    decltype(&gqla_decode_absorb_fp8_paged) decode_absorb;
    decltype(&gqla_decode_gqa_fp8_paged) decode_gqa;
    decltype(&gqla_status_str) status_str;
} g{};

// The arguments of a call, taken one after another, and what all of its tensors have in common: the current device.
class Args {
public:
    Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t expected) : args_(args) {
        if (n != expected) throw Refusal("wrong number of arguments");
    }
    gqla_dims dims() {
        gqla_dims d;
        Py_buffer b;
        if (PyObject_GetBuffer(next(), &b, PyBUF_SIMPLE) != 0) throw PythonError();
        const bool ok = b.len == (Py_ssize_t)sizeof(d);
        if (ok) memcpy(&d, b.buf, sizeof(d));
        PyBuffer_Release(&b);
        if (!ok) throw Refusal("dims: expected a GqlaDims");
        return d;
    }
    const at::Tensor& tensor(const char* what) {
        const at::Tensor* t = optional(what);
        if (t == nullptr) throw Refusal(std::string(what) + ": expected a tensor, got None");
        return *t;
    }
    const at::Tensor* optional(const char* what) {
        PyObject* o = next();
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) throw Refusal(std::string(what) + ": expected a tensor, got " + Py_TYPE(o)->tp_name);
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda()) throw Refusal(std::string(what) + ": expected a CUDA tensor, got one on " + t.device().str());
        if (device_ < 0) device_ = c10::cuda::current_device();
        if (t.get_device() != device_)
            throw Refusal(std::string(what) + ": expected a tensor on cuda:" + std::to_string(device_) + ", got one on " + t.device().str());
        return &t;
    }
    int32_t i32(const char* what) {
        const long long v = PyLong_AsLongLong(next());
        if (v == -1 && PyErr_Occurred()) throw PythonError();
        if (v < INT32_MIN || v > INT32_MAX) throw Refusal(std::string(what) + ": " + std::to_string(v) + " does not fit 32 bits");
        return (int32_t)v;
    }
    float f32() {
        const double v = PyFloat_AsDouble(next());
        if (v == -1.0 && PyErr_Occurred()) throw PythonError();
        return (float)v;
    }
    int32_t* status_word() {
        const at::Tensor* t = optional("status_word");
        if (t == nullptr) return nullptr;
        if (t->scalar_type() != at::kInt || t->numel() < 1) throw Refusal("status_word: expected int32");
        return static_cast<int32_t*>(t->data_ptr());
    }
    void* stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device_).stream(); }

private:
    PyObject* next() { return *args_++; }
    PyObject* const* args_;
    int device_ = -1;
};

using Shape = std::initializer_list<int64_t>;

// (By hand: no iostreams here.  Where the linker takes the C++ runtime from its archive, this module has a copy of its own, and a stream's
// facets, looked up by ids that the process shared, belonged to another one.)
std::string text(c10::IntArrayRef shape) {
    std::string s = "[";
    for (size_t i = 0; i < shape.size(); ++i) s += (i > 0 ? ", " : "") + std::to_string(shape[i]);
    return s + "]";
}
std::string text(at::ScalarType type, c10::IntArrayRef shape) { return std::string(c10::toString(type)) + " " + text(shape); }

void expect(const char* what, const at::Tensor& t, Shape shape, at::ScalarType type) {
    if (t.scalar_type() == type && t.sizes() == c10::IntArrayRef(shape.begin(), shape.size())) return;
    throw Refusal(std::string(what) + ": expected " + text(type, c10::IntArrayRef(shape.begin(), shape.size())) + ", got " +
                  text(t.scalar_type(), t.sizes()));
}
// A contiguous tensor; its address.
template <typename T = void>
T* dense(const char* what, const at::Tensor& t, Shape shape, at::ScalarType type) {
    expect(what, t, shape, type);
    if (!t.is_contiguous()) throw Refusal(std::string(what) + ": expected a contiguous tensor");
    return static_cast<T*>(t.data_ptr());
}
// A tensor of rows, whose last dimension is contiguous; its address.
template <typename T = void>
T* rows(const char* what, const at::Tensor& t, Shape shape, at::ScalarType type) {
    expect(what, t, shape, type);
    if (t.stride(-1) != 1 && t.size(-1) > 1) throw Refusal(std::string(what) + ": the last dimension has to be contiguous");
    return static_cast<T*>(t.data_ptr());
}
// The elements between steps of `dim`; the stride of a dimension of one element is arbitrary and never stepped by.
int64_t step(const at::Tensor& t, int64_t dim) {
    if (t.size(dim) > 1) return t.stride(dim);
    int64_t n = 1;
    for (int64_t i = dim + 1; i < t.dim(); ++i) n *= t.size(i);
    return std::max(t.stride(dim), n);
}
int64_t length(const char* what, const at::Tensor& t, int64_t dim) {
    if (t.dim() <= dim) throw Refusal(std::string(what) + ": too few dimensions");
    return t.size(dim);
}
int32_t size32(const char* what, int64_t n) {
    if (n > INT32_MAX) throw Refusal(std::string(what) + ": " + std::to_string(n) + " does not fit 32 bits");
    return (int32_t)n;
}
gqla_dtype dtype_of(const char* what, const at::Tensor& t) {
    if (t.scalar_type() == at::kBFloat16) return GQLA_BF16;
    if (t.scalar_type() == at::kFloat) return GQLA_F32;
    throw Refusal(std::string(what) + ": unsupported dtype " + c10::toString(t.scalar_type()));
}

// What the append calls share: new_start, seqlens, rope, style, k_r, q_r, q_out (in this order; the new rows' type and number given).
struct Append {
    int32_t B;
    const int32_t *new_start, *seqlens;
    const void* k_r;
    int64_t k_r_stride;
    const float* rope;
    int32_t rope_rows;
    gqla_rope_style style;
    const void* q_r = nullptr;
    int64_t q_tok = 0, q_head = 0;
    void* q_out = nullptr;
    int64_t o_tok = 0, o_head = 0;
    Append(Args& a, const gqla_dims& d, int64_t n, at::ScalarType type) {
        const at::Tensor &start = a.tensor("new_start"), &lens = a.tensor("seqlens"), &table = a.tensor("rope");
        B = size32("seqlens", length("seqlens", lens, 0));
        new_start = dense<int32_t>("new_start", start, {B + (int64_t)1}, at::kInt);
        seqlens = dense<int32_t>("seqlens", lens, {B}, at::kInt);
        rope_rows = size32("rope", length("rope", table, 0));
        rope = dense<float>("rope", table, {rope_rows, d.d_r}, at::kFloat);
        style = (gqla_rope_style)a.i32("style");
        const at::Tensor& k = a.tensor("k_r");
        k_r = rows("k_r", k, {n, d.d_r}, type);
        k_r_stride = step(k, 0);
        const at::Tensor *q = a.optional("q_r"), *o = a.optional("q_out");
        if ((q == nullptr) != (o == nullptr)) throw Refusal("q_r and q_out come together");
        if (q != nullptr) {
            q_r = rows("q_r", *q, {n, d.h_q, d.d_r}, type);
            q_out = rows("q_out", *o, {n, d.h_q, d.d_r}, type);
            q_tok = step(*q, 0); q_head = step(*q, 1);
            o_tok = step(*o, 0); o_head = step(*o, 1);
        }
    }
};

struct Pages {
    const int32_t* table = nullptr;
    int32_t max_pages = 0, page_size = 0;
    int64_t n = 0;
    Pages() = default;
    Pages(const at::Tensor& t, int32_t size, int64_t n_rows, int64_t B) : page_size(size) {
        if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(0) != B || !t.is_contiguous() || t.size(1) > INT32_MAX) {
            throw Refusal("block_table: expected contiguous int32 [" + std::to_string(B) + ", max_pages], got " + text(t.scalar_type(), t.sizes()));
        }
        if (size < 1 || n_rows % size != 0)
            throw Refusal("a cache of " + std::to_string(n_rows) + " rows is not made of pages of " + std::to_string(size));
        table = static_cast<const int32_t*>(t.data_ptr());
        max_pages = (int32_t)t.size(1);
        n = n_rows / size;
    }
};

// The E4M3 planes and their scales: k_c8, v8, k_r8, k_scale, v_scale, r_scale, block_table, page_size.
struct Planes {
    uint8_t *k_c, *v, *k_r;
    int64_t k_r_stride, n_rows;
    float *k_scale, *v_scale, *r_scale;
    Pages pages;
    Planes(Args& a, const gqla_dims& d, int64_t B) {
        const at::Tensor &kt = a.tensor("k_c8"), &vt = a.tensor("v8"), &rt = a.tensor("k_r8");
        const at::Tensor &ks = a.tensor("k_scale"), &vs = a.tensor("v_scale"), &rs = a.tensor("r_scale"), &table = a.tensor("block_table");
        n_rows = length("k_c8", kt, 0);
        pages = Pages(table, a.i32("page_size"), n_rows, B);
        k_c = dense<uint8_t>("k_c8", kt, {n_rows, d.g, d.d_h}, at::kByte);
        v = dense<uint8_t>("v8", vt, {n_rows, d.g, d.d_h}, at::kByte);
        k_r = rows<uint8_t>("k_r8", rt, {n_rows, d.d_r}, at::kByte);
        k_r_stride = step(rt, 0);
        k_scale = dense<float>("k_scale", ks, {pages.n, d.g}, at::kFloat);
        v_scale = dense<float>("v_scale", vs, {pages.n, d.g}, at::kFloat);
        r_scale = dense<float>("r_scale", rs, {pages.n}, at::kFloat);
    }
};

// Partials and the merged output of an attention call: num_splits (in front), o_part, lse_part, out, lse.
struct Partials {
    int32_t splits;
    float *o_part, *lse_part, *lse = nullptr;
    void* out = nullptr;
    Partials(Args& a, const gqla_dims& d, int64_t B, int64_t s_q, int64_t width, at::ScalarType type) {
        splits = a.i32("num_splits");
        const int64_t slots = splits < 0 ? -(int64_t)splits : splits;
        o_part = dense<float>("o_part", a.tensor("o_part"), {B, slots, s_q, d.h_q, width}, at::kFloat);
        lse_part = dense<float>("lse_part", a.tensor("lse_part"), {B, slots, s_q, d.h_q}, at::kFloat);
        if (const at::Tensor* t = a.optional("out")) out = dense("out", *t, {B, s_q, d.h_q, width}, type);
        if (const at::Tensor* t = a.optional("lse")) lse = dense<float>("lse", *t, {B, s_q, d.h_q}, at::kFloat);
    }
};

// dims, c, new_start, seqlens, rope, style, k_r, q_r, q_out, cache, seq_start, block_table, page_size, status_word
gqla_status append_rope(Args& a) {
    const gqla_dims d = a.dims();
    const at::Tensor& c = a.tensor("c");
    const int64_t n = length("c", c, 0);
    const gqla_dtype dtype = dtype_of("c", c);
    const Append s(a, d, n, c.scalar_type());
    const at::Tensor& cache = a.tensor("cache");
    const at::Tensor *start = a.optional("seq_start"), *table = a.optional("block_table");
    const int32_t page_size = a.i32("page_size");
    int32_t* status = a.status_word();
    const void* c_rows = rows("c", c, {n, d.r_kv}, c.scalar_type());
    const int64_t n_rows = length("cache", cache, 0);
    void* dst = rows("cache", cache, {n_rows, (int64_t)d.r_kv + d.d_r}, c.scalar_type());
    if ((start == nullptr) == (table == nullptr)) throw Refusal("either seq_start (packed) or block_table (paged)");
    const int64_t* starts = start != nullptr ? dense<int64_t>("seq_start", *start, {s.B}, at::kLong) : nullptr;
    const Pages pages = table != nullptr ? Pages(*table, page_size, n_rows, s.B) : Pages();
    return g.append_rope(&d, dtype, s.B, n, s.new_start, s.seqlens, c_rows, step(c, 0), s.k_r, s.k_r_stride, s.rope, s.rope_rows, s.style,
                         s.q_r, s.q_tok, s.q_head, s.q_out, s.o_tok, s.o_head, dst, step(cache, 0), n_rows, starts, pages.table,
                         pages.max_pages, pages.page_size, status, a.stream());
}

// dims, c, new_start, seqlens, rope, style, k_r, q_r, q_out, cache8, page_scale, block_table, page_size, status_word
gqla_status append_rope_fp8(Args& a) {
    const gqla_dims d = a.dims();
    const at::Tensor& c = a.tensor("c");
    const int64_t n = length("c", c, 0);
    const gqla_dtype dtype = dtype_of("c", c);
    const Append s(a, d, n, c.scalar_type());
    const at::Tensor &cache = a.tensor("cache8"), &scale = a.tensor("page_scale"), &table = a.tensor("block_table");
    const int64_t n_rows = length("cache8", cache, 0);
    const Pages pages(table, a.i32("page_size"), n_rows, s.B);
    int32_t* status = a.status_word();
    const void* c_rows = rows("c", c, {n, d.r_kv}, c.scalar_type());
    uint8_t* dst = rows<uint8_t>("cache8", cache, {n_rows, (int64_t)d.r_kv + d.d_r}, at::kByte);
    float* scales = dense<float>("page_scale", scale, {pages.n}, at::kFloat);
    return g.append_rope_fp8(&d, dtype, s.B, n, s.new_start, s.seqlens, c_rows, step(c, 0), s.k_r, s.k_r_stride, s.rope, s.rope_rows,
                             s.style, s.q_r, s.q_tok, s.q_head, s.q_out, s.o_tok, s.o_head, dst, step(cache, 0), n_rows, scales,
                             pages.table, pages.max_pages, pages.page_size, status, a.stream());
}

// dims, k_c, v, new_start, seqlens, rope, style, k_r, q_r, q_out, k_c8, v8, k_r8, k_scale, v_scale, r_scale, block_table, page_size,
// status_word
gqla_status append_planes_fp8(Args& a) {
    const gqla_dims d = a.dims();
    const at::Tensor &kt = a.tensor("k_c"), &vt = a.tensor("v");
    const int64_t n = length("k_c", kt, 0);
    const gqla_dtype dtype = dtype_of("k_c", kt);
    const Append s(a, d, n, kt.scalar_type());
    const void* k_c = dense("k_c", kt, {n, d.g, d.d_h}, kt.scalar_type());
    const void* v = dense("v", vt, {n, d.g, d.d_h}, kt.scalar_type());
    const Planes p(a, d, s.B);
    int32_t* status = a.status_word();
    return g.append_planes_fp8(&d, dtype, s.B, n, s.new_start, s.seqlens, k_c, v, s.k_r, s.k_r_stride, s.rope, s.rope_rows, s.style, s.q_r,
                               s.q_tok, s.q_head, s.q_out, s.o_tok, s.o_head, p.k_c, p.v, p.k_r, p.k_r_stride, p.n_rows, p.k_scale,
                               p.v_scale, p.r_scale, p.pages.table, p.pages.max_pages, p.pages.page_size, status, a.stream());
}

// dims, q_hat, cache8, page_scale, block_table, page_size, seqlens, scale, num_splits, o_part, lse_part, out, lse, status_word
gqla_status decode_absorb(Args& a) {
    const gqla_dims d = a.dims();
    const at::Tensor &q = a.tensor("q_hat"), &cache = a.tensor("cache8"), &scale = a.tensor("page_scale"), &table = a.tensor("block_table");
    const int64_t B = length("q_hat", q, 0), s_q = length("q_hat", q, 1), n_rows = length("cache8", cache, 0);
    const int64_t width = (int64_t)d.r_kv + d.d_r;
    const gqla_dtype dtype = dtype_of("q_hat", q);
    const Pages pages(table, a.i32("page_size"), n_rows, B);
    const int32_t* lens = dense<int32_t>("seqlens", a.tensor("seqlens"), {B}, at::kInt);
    const float factor = a.f32();
    const Partials out(a, d, B, s_q, d.r_kv, q.scalar_type());
    int32_t* status = a.status_word();
    const void* queries = dense("q_hat", q, {B, s_q, d.h_q, width}, q.scalar_type());
    const uint8_t* codes = rows<uint8_t>("cache8", cache, {n_rows, width}, at::kByte);
    const float* scales = dense<float>("page_scale", scale, {pages.n}, at::kFloat);
    return g.decode_absorb(&d, dtype, size32("q_hat", B), size32("q_hat", s_q), factor, out.splits, queries, codes, step(cache, 0), n_rows,
                           scales, pages.table, pages.max_pages, pages.page_size, lens, out.o_part, out.lse_part, out.out, out.lse, status,
                           a.stream());
}

// dims, q, k_c8, v8, k_r8, k_scale, v_scale, r_scale, block_table, page_size, seqlens, scale, num_splits, o_part, lse_part, out, lse,
// status_word
gqla_status decode_gqa(Args& a) {
    const gqla_dims d = a.dims();
    const at::Tensor& q = a.tensor("q");
    const int64_t B = length("q", q, 0), s_q = length("q", q, 1);
    const gqla_dtype dtype = dtype_of("q", q);
    const Planes p(a, d, B);
    const int32_t* lens = dense<int32_t>("seqlens", a.tensor("seqlens"), {B}, at::kInt);
    const float factor = a.f32();
    const Partials out(a, d, B, s_q, d.d_h, q.scalar_type());
    int32_t* status = a.status_word();
    const void* queries = dense("q", q, {B, s_q, d.h_q, (int64_t)d.d_h + d.d_r}, q.scalar_type());
    return g.decode_gqa(&d, dtype, size32("q", B), size32("q", s_q), factor, out.splits, queries, p.k_c, p.v, p.k_r, p.k_r_stride, p.n_rows,
                        p.k_scale, p.v_scale, p.r_scale, p.pages.table, p.pages.max_pages, p.pages.page_size, lens, out.o_part,
                        out.lse_part, out.out, out.lse, status, a.stream());
}

constexpr char kAppendRope[] = "gqla_append_rope", kAppendRopeFp8[] = "gqla_append_rope_fp8", kAppendPlanesFp8[] = "gqla_append_planes_fp8",
               kDecodeAbsorb[] = "gqla_decode_absorb_fp8_paged", kDecodeGqa[] = "gqla_decode_gqa_fp8_paged";

template <gqla_status (*CALL)(Args&), int N, const char* NAME>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (g.status_str == nullptr) {
        PyErr_SetString(PyExc_RuntimeError, "bind() comes first");
        return nullptr;
    }
    try {
        Args a(args, n, N);
        const gqla_status s = CALL(a);
        if (s != GQLA_OK) throw Refusal(std::string(g.status_str(s)) + " (status " + std::to_string((int)s) + ")");
        Py_RETURN_NONE;
    } catch (const PythonError&) {
        return nullptr;
    } catch (const Refusal& e) {
        PyErr_Format(g_error, "%s: %s", NAME, e.what());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// bind(GqlaError, addresses of the five entry points and of gqla_status_str)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "bind takes an exception and six addresses");
        return nullptr;
    }
    void* at[6];
    for (int i = 0; i < 6; ++i) {
        at[i] = PyLong_AsVoidPtr(args[i + 1]);
        if (at[i] == nullptr && PyErr_Occurred()) return nullptr;
    }
    Py_INCREF(args[0]);
    Py_XDECREF(g_error);
    g_error = args[0];
    g = Entries{(decltype(Entries::append_rope))at[0],   (decltype(Entries::append_rope_fp8))at[1], (decltype(Entries::append_planes_fp8))at[2],
                (decltype(Entries::decode_absorb))at[3], (decltype(Entries::decode_gqa))at[4],      (decltype(Entries::status_str))at[5]};
    Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f))
PyMethodDef kMethods[] = {
    {"bind", FAST(bind), METH_FASTCALL, nullptr},
    {kAppendRope, FAST((entry<append_rope, 14, kAppendRope>)), METH_FASTCALL, nullptr},
    {kAppendRopeFp8, FAST((entry<append_rope_fp8, 14, kAppendRopeFp8>)), METH_FASTCALL, nullptr},
    {kAppendPlanesFp8, FAST((entry<append_planes_fp8, 19, kAppendPlanesFp8>)), METH_FASTCALL, nullptr},
    {kDecodeAbsorb, FAST((entry<decode_absorb, 14, kDecodeAbsorb>)), METH_FASTCALL, nullptr},
    {kDecodeGqa, FAST((entry<decode_gqa, 18, kDecodeGqa>)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#define TEXT_OF(x) #x
#define TEXT(x) TEXT_OF(x)
// (build.py and the binding look for this in the file)
constexpr char kStamp[] = "built for torch " TORCH_VERSION ", Python " TEXT(PY_MAJOR_VERSION) "." TEXT(PY_MINOR_VERSION) ";";

PyMODINIT_FUNC PyInit__marshal() {
    PyObject* m = PyModule_Create(&kModule);
    if (m != nullptr && PyModule_AddStringConstant(m, "stamp", kStamp) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
