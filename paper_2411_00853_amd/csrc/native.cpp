// Marshalling of tensors for the calls of spec_q8.h and spec_prompt.h, as an extension module: these calls last a few microseconds on the GPU, and
// reading a tensor's type, shape and address from Python took as long again for every call.  Checks of arguments only -- no arithmetic,
// no allocation, and the functions called are the library's, whose addresses bind() receives.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>

#include "../../include/spec_prompt.h"
#include "../../include/spec_q8.h"

namespace {

struct Bad : std::runtime_error {
    using std::runtime_error::runtime_error;
};

constexpr auto F8 = at::kFloat8_e4m3fn, F32 = at::kFloat, BF16 = at::kBFloat16, I32 = at::kInt;

struct Library {
    decltype(&spec_q8_quantize) quantize;
    decltype(&spec_q8_add_rmsnorm) add_rmsnorm;
    decltype(&spec_q8_swiglu) swiglu;
    decltype(&spec_q8_gemm) gemm;
    decltype(&spec_kv8_append) append;
    decltype(&spec_kv8_attention) attention;
    decltype(&spec_filter_sample) sample;
    decltype(&spec_prompt_rmsnorm) prompt_rmsnorm;
    decltype(&spec_prompt_gemm) prompt_gemm;
    decltype(&spec_prompt_append) prompt_append;
    decltype(&spec_prompt_attention) prompt_attention;
} lib{};

std::string text(at::IntArrayRef s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + ")";
}

const at::Tensor& tensor(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o)) throw Bad(std::string(name) + ": expected a tensor");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) throw Bad(std::string(name) + ": expected a device tensor");
    return t;
}

void* whole(const at::Tensor& t, const char* name)
{
    if (!t.is_contiguous()) throw Bad(std::string(name) + ": expected a contiguous tensor");
    return t.data_ptr();
}

void* shaped(const at::Tensor& t, at::IntArrayRef shape, at::ScalarType type, const char* name)
{
    if (t.scalar_type() != type) throw Bad(std::string(name) + ": expected " + at::toString(type) + ", got " + at::toString(t.scalar_type()));
    if (t.sizes() != shape) throw Bad(std::string(name) + ": expected shape " + text(shape) + ", got " + text(t.sizes()));
    return whole(t, name);
}

void* shaped(PyObject* o, at::IntArrayRef shape, at::ScalarType type, const char* name) { return shaped(tensor(o, name), shape, type, name); }

void* optional(PyObject* o, at::IntArrayRef shape, at::ScalarType type, const char* name)
{
    return o == Py_None ? nullptr : shaped(o, shape, type, name);
}

int code(const at::Tensor& t, const char* name)
{
    if (t.scalar_type() == F32) return SPEC_DTYPE_FP32;
    if (t.scalar_type() == BF16) return SPEC_DTYPE_BF16;
    throw Bad(std::string(name) + ": expected Float or BFloat16, got " + at::toString(t.scalar_type()));
}

int32_t narrow(int64_t v, const char* name)
{
    if (v < INT32_MIN || v > INT32_MAX) throw Bad(std::string(name) + ": " + std::to_string(v) + " does not fit 32 bits");
    return (int32_t)v;
}

int32_t integer(PyObject* o, const char* name)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Bad(std::string(name) + ": expected a whole number");
    }
    return narrow(v, name);
}

float real(PyObject* o, const char* name)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Bad(std::string(name) + ": expected a number");
    }
    return (float)v;
}

void* stream_of(PyObject* o) { return o == Py_None ? nullptr : PyLong_AsVoidPtr(o); }

// Rows of contiguous elements, any distance apart
struct Rows {
    void* p;
    int64_t ld;
    int32_t rows, cols;
};
Rows rows_of(const at::Tensor& t, const char* name)
{
    if (t.dim() != 2) throw Bad(std::string(name) + ": expected two dimensions");
    const int64_t rows = t.size(0), cols = t.size(1);
    if (cols > 1 && t.stride(1) != 1) throw Bad(std::string(name) + ": expected rows of contiguous elements");
    return {t.data_ptr(), rows > 1 ? t.stride(0) : cols, narrow(rows, name), narrow(cols, name)};
}

int64_t padded(int64_t cols) { return (cols + SPEC_Q8_BLOCK - 1) / SPEC_Q8_BLOCK * SPEC_Q8_BLOCK; }

struct Q8Out {
    void* q;
    float* scales;
};
Q8Out q8_out(PyObject* q, PyObject* scales, int64_t rows, int64_t cols)
{
    const int64_t kp = padded(cols);
    return {shaped(q, {rows, kp}, F8, "q"), (float*)shaped(scales, {kp / SPEC_Q8_BLOCK, rows}, F32, "scales")};
}

int quantize(PyObject* const* a)   // x, q, scales, stream
{
    const at::Tensor& x = tensor(a[0], "x");
    const Rows r = rows_of(x, "x");
    const Q8Out o = q8_out(a[1], a[2], r.rows, r.cols);
    return lib.quantize(r.p, code(x, "x"), r.ld, r.rows, r.cols, o.q, o.scales, stream_of(a[3]));
}

int add_rmsnorm(PyObject* const* a)   // x, delta, gain, eps, x_out, q, scales, stream
{
    const at::Tensor& x = tensor(a[0], "x");
    const Rows r = rows_of(x, "x");
    void* xp = whole(x, "x");
    int delta_code = SPEC_DTYPE_FP32;
    void* delta = nullptr;
    if (a[1] != Py_None) {
        const at::Tensor& d = tensor(a[1], "delta");
        delta_code = code(d, "delta");
        delta = shaped(d, x.sizes(), d.scalar_type(), "delta");
    }
    const Q8Out o = q8_out(a[5], a[6], r.rows, r.cols);
    return lib.add_rmsnorm(xp, code(x, "x"), delta, delta_code, (float*)shaped(a[2], {r.cols}, F32, "gain"), real(a[3], "eps"), r.rows, r.cols,
                           optional(a[4], x.sizes(), x.scalar_type(), "x_out"), o.q, o.scales, stream_of(a[7]));
}

int swiglu(PyObject* const* a)   // gate_up, q, scales, stream
{
    const at::Tensor& x = tensor(a[0], "gate_up");
    const Rows r = rows_of(x, "gate_up");
    if (r.cols % 2) throw Bad("gate_up: expected as many up columns as gate columns");
    const Q8Out o = q8_out(a[1], a[2], r.rows, r.cols / 2);
    return lib.swiglu(whole(x, "gate_up"), code(x, "gate_up"), r.rows, r.cols / 2, o.q, o.scales, stream_of(a[3]));
}

int gemm(PyObject* const* a)   // q, scales, w_packed, w_scales, y, stream
{
    const at::Tensor &q = tensor(a[0], "q"), &w = tensor(a[2], "w_packed"), &y = tensor(a[4], "y");
    if (q.dim() != 2 || y.dim() != 2) throw Bad("q, y: expected two dimensions");
    const int64_t M = q.size(0), kp = q.size(1), N = y.size(1), blocks = kp / SPEC_Q8_BLOCK;
    if (kp % SPEC_Q8_BLOCK || w.numel() != (N + 15) / 16 * 16 * kp) throw Bad("w_packed: expected a packed matrix of " + std::to_string(N) + " x " + std::to_string(kp));
    const int yc = code(y, "y");
    return lib.gemm(shaped(q, {M, kp}, F8, "q"), (float*)shaped(a[1], {blocks, M}, F32, "scales"), shaped(w, w.sizes(), F8, "w_packed"),
                    (float*)shaped(a[3], {(N + 127) / 128, blocks}, F32, "w_scales"), shaped(y, {M, N}, y.scalar_type(), "y"), yc, narrow(M, "q"),
                    narrow(N, "y"), narrow(kp, "q"), stream_of(a[5]));
}

spec_kv8_cache cache_of(PyObject* const* a)   // data, scales, table, head_dim
{
    const at::Tensor &data = tensor(a[0], "data"), &table = tensor(a[2], "table");
    const int32_t hd = integer(a[3], "head_dim");
    if (data.dim() != 4 || table.dim() != 2) throw Bad("data, table: expected four and two dimensions");
    const int64_t pages = data.size(0), heads = data.size(1);
    return {shaped(data, {pages, heads, 2, (int64_t)SPEC_KV8_PAGE * hd}, F8, "data"), (float*)shaped(a[1], {pages, heads, 2}, F32, "scales"),
            (const int32_t*)shaped(table, table.sizes(), I32, "table"), narrow(pages, "data"), narrow(heads, "data"), hd, narrow(table.size(0), "table"),
            narrow(table.size(1), "table")};
}

int append(PyObject* const* a)   // cache (4), qkv, row0, kv_len, n_q_heads, max_window, cos_sin, q_out, stream
{
    const spec_kv8_cache c = cache_of(a);
    const at::Tensor& qkv = tensor(a[4], "qkv");
    if (qkv.dim() != 2) throw Bad("qkv: expected two dimensions");
    const int64_t rows = qkv.size(0);
    const int32_t hq = integer(a[7], "n_q_heads");
    int64_t max_pos = 0;
    const float* cos_sin = nullptr;
    if (a[9] != Py_None) {
        const at::Tensor& t = tensor(a[9], "cos_sin");
        max_pos = t.dim() ? t.size(0) : 0;
        cos_sin = (const float*)shaped(t, {max_pos, c.head_dim / 2, 2}, F32, "cos_sin");
    }
    return lib.append(&c, shaped(qkv, {rows, ((int64_t)hq + 2 * c.n_kv_heads) * c.head_dim}, BF16, "qkv"), hq,
                      (const int32_t*)shaped(a[5], {c.batch + 1}, I32, "row0"), (const int32_t*)shaped(a[6], {c.batch}, I32, "kv_len"),
                      narrow(rows, "qkv"), integer(a[8], "max_window"), cos_sin, narrow(max_pos, "cos_sin"),
                      optional(a[10], {rows, (int64_t)hq * c.head_dim}, BF16, "q_out"), stream_of(a[11]));
}

int attention(PyObject* const* a)   // cache (4), q, row0, kv_len, n_q_heads, max_window, max_len, scale, out, workspace, stream
{
    const spec_kv8_cache c = cache_of(a);
    const at::Tensor &q = tensor(a[4], "q"), &out = tensor(a[11], "out");
    const int32_t hq = integer(a[7], "n_q_heads");
    const Rows r = rows_of(q, "q");
    const int64_t cols = (int64_t)hq * c.head_dim;
    if (q.scalar_type() != BF16 || r.cols != cols) throw Bad("q: expected BFloat16 rows of " + std::to_string(cols));
    void* ws = nullptr;
    size_t bytes = 0;
    if (a[12] != Py_None) {
        const at::Tensor& t = tensor(a[12], "workspace");
        ws = whole(t, "workspace");
        bytes = t.nbytes();
    }
    return lib.attention(&c, r.p, r.ld, hq, (const int32_t*)shaped(a[5], {c.batch + 1}, I32, "row0"),
                         (const int32_t*)shaped(a[6], {c.batch}, I32, "kv_len"), r.rows, integer(a[8], "max_window"), integer(a[9], "max_len"),
                         real(a[10], "scale"), shaped(out, {r.rows, cols}, BF16, "out"), ws, bytes, stream_of(a[13]));
}

int sample(PyObject* const* a)   // logits, uniforms, temperature, tokens, top_k, top_p, min_p, logprob, n_kept, logits_out, workspace, stream
{
    const at::Tensor& x = tensor(a[0], "logits");
    const Rows r = rows_of(x, "logits");
    const at::IntArrayRef row(x.sizes().data(), 1);
    spec_filter_args args{};
    args.logits = r.p;
    args.dtype = code(x, "logits");
    args.rows = r.rows;
    args.vocab = r.cols;
    args.ld = r.ld;
    args.uniforms = (const float*)shaped(a[1], row, F32, "uniforms");
    args.temperature = (const float*)optional(a[2], row, F32, "temperature");
    args.top_k = (const int32_t*)optional(a[4], row, I32, "top_k");
    args.top_p = (const float*)optional(a[5], row, F32, "top_p");
    args.min_p = (const float*)optional(a[6], row, F32, "min_p");
    spec_filter_out out{};
    out.tokens = (int32_t*)shaped(a[3], row, I32, "tokens");
    out.logprob = (float*)optional(a[7], row, F32, "logprob");
    out.n_kept = (int32_t*)optional(a[8], row, I32, "n_kept");
    out.logits_out = (float*)optional(a[9], x.sizes(), F32, "logits_out");
    void* ws = nullptr;
    size_t bytes = 0;
    if (a[10] != Py_None) {
        const at::Tensor& t = tensor(a[10], "workspace");
        ws = whole(t, "workspace");
        bytes = t.nbytes();
    }
    return lib.sample(&args, &out, ws, bytes, stream_of(a[11]));
}

// The calls on prompts take tensors of the device that is current (their last argument)
const at::Tensor& here(PyObject* o, const char* name, PyObject* device)
{
    const at::Tensor& t = tensor(o, name);
    if (t.get_device() != integer(device, "device"))
        throw Bad(std::string(name) + ": of device " + std::to_string(t.get_device()) + ", the current one is " + std::to_string(integer(device, "device")));
    return t;
}
void* optional_here(PyObject* o, at::IntArrayRef shape, at::ScalarType type, const char* name, PyObject* device)
{
    return o == Py_None ? nullptr : shaped(here(o, name, device), shape, type, name);
}

struct Scratch {
    void* p;
    size_t bytes;
};
Scratch scratch(PyObject* o, PyObject* device)
{
    if (o == Py_None) return {nullptr, 0};
    const at::Tensor& t = here(o, "workspace", device);
    return {whole(t, "workspace"), t.nbytes()};
}

// Rows of bf16 numbers, `cols` of them (less than 0: any number)
Rows bf16_rows(const at::Tensor& t, int64_t cols, const char* name)
{
    const Rows r = rows_of(t, name);
    if (t.scalar_type() != BF16 || (cols >= 0 && r.cols != cols))
        throw Bad(std::string(name) + ": expected BFloat16 rows" + (cols < 0 ? "" : " of " + std::to_string(cols)) + ", got " +
                  at::toString(t.scalar_type()) + " " + text(t.sizes()));
    return r;
}

int prompt_rmsnorm(PyObject* const* a)   // x, gain, eps, y, stream, device
{
    const at::Tensor& x = here(a[0], "x", a[5]);
    const Rows r = rows_of(x, "x");
    return lib.prompt_rmsnorm(r.p, code(x, "x"), r.ld, (float*)shaped(here(a[1], "gain", a[5]), {r.cols}, F32, "gain"), real(a[2], "eps"), r.rows, r.cols,
                              shaped(here(a[3], "y", a[5]), x.sizes(), BF16, "y"), stream_of(a[4]));
}

int prompt_gemm(PyObject* const* a)   // x, w_packed, y, bias, activation, residual, workspace, stream, device
{
    const at::Tensor &w = here(a[1], "w_packed", a[8]), &y = here(a[2], "y", a[8]);
    const Rows x = bf16_rows(here(a[0], "x", a[8]), -1, "x"), o = rows_of(y, "y");
    spec_prompt_epilogue e{};
    e.activation = integer(a[4], "activation");
    const int64_t n_out = (int64_t)o.cols * (e.activation == SPEC_ACT_SWIGLU ? 2 : 1), kp = ((int64_t)x.cols + 127) / 128 * 128;
    if (o.rows != x.rows) throw Bad("y: expected " + std::to_string(x.rows) + " rows, got " + std::to_string(o.rows));
    if (w.scalar_type() != BF16 || w.numel() != (n_out + 15) / 16 * 16 * kp)
        throw Bad("w_packed: expected a packed BFloat16 matrix of " + std::to_string(n_out) + " x " + std::to_string(x.cols));
    e.bias = (const float*)optional_here(a[3], {n_out}, F32, "bias", a[8]);
    if (a[5] != Py_None) {
        const at::Tensor& t = here(a[5], "residual", a[8]);
        const Rows r = rows_of(t, "residual");
        if (t.sizes() != y.sizes()) throw Bad("residual: expected shape " + text(y.sizes()) + ", got " + text(t.sizes()));
        e.residual = r.p;
        e.ld_residual = r.ld;
        e.residual_dtype = code(t, "residual");
    }
    const Scratch s = scratch(a[6], a[8]);
    return lib.prompt_gemm(x.p, x.ld, whole(w, "w_packed"), &e, o.p, code(y, "y"), o.ld, x.rows, o.cols, x.cols, s.p, s.bytes, stream_of(a[7]));
}

int prompt_append(PyObject* const* a)   // handle, layer, qkv, rotated, row0, seq_slot, pos0, rotated columns, qkv columns, stream, device
{
    const at::Tensor& row0 = here(a[4], "row0", a[10]);
    const Rows x = bf16_rows(here(a[2], "qkv", a[10]), integer(a[8], "columns"), "qkv"), o = bf16_rows(here(a[3], "rotated", a[10]), integer(a[7], "columns"), "rotated");
    if (o.rows != x.rows) throw Bad("rotated: expected " + std::to_string(x.rows) + " rows, got " + std::to_string(o.rows));
    if (row0.dim() != 1 || !row0.size(0)) throw Bad("row0: expected the sequences' first rows and one number more");
    const int64_t batch = row0.size(0) - 1;
    return lib.prompt_append(a[0] == Py_None ? nullptr : (spec_handle*)PyLong_AsVoidPtr(a[0]), integer(a[1], "layer"), x.p, x.ld, o.p, o.ld,
                             (const int32_t*)shaped(row0, {batch + 1}, I32, "row0"), (const int32_t*)shaped(here(a[5], "seq_slot", a[10]), {batch}, I32, "seq_slot"),
                             (const int32_t*)optional_here(a[6], {batch}, I32, "pos0", a[10]), narrow(batch, "row0"), x.rows, stream_of(a[9]));
}

int prompt_attention(PyObject* const* a)   // q, k, v, n_q_heads, n_kv_heads, q_row0, k_row0, out, scale, max_q_len, max_k_len, workspace, stream, device
{
    const at::Tensor& row0 = here(a[5], "q_row0", a[13]);
    spec_prompt_attn_args p{};
    p.n_q_heads = integer(a[3], "n_q_heads");
    p.n_kv_heads = integer(a[4], "n_kv_heads");
    if (p.n_q_heads <= 0 || p.n_kv_heads <= 0) throw Bad("n_q_heads, n_kv_heads: expected positive numbers");
    const Rows q = bf16_rows(here(a[0], "q", a[13]), -1, "q");
    if (q.cols % p.n_q_heads) throw Bad("q: " + std::to_string(q.cols) + " columns are not those of " + std::to_string(p.n_q_heads) + " heads");
    p.head_dim = q.cols / p.n_q_heads;
    const Rows k = bf16_rows(here(a[1], "k", a[13]), (int64_t)p.n_kv_heads * p.head_dim, "k"), v = bf16_rows(here(a[2], "v", a[13]), k.cols, "v"),
               out = bf16_rows(here(a[7], "out", a[13]), q.cols, "out");
    if (v.rows != k.rows) throw Bad("v: expected " + std::to_string(k.rows) + " rows, got " + std::to_string(v.rows));
    if (out.rows != q.rows) throw Bad("out: expected " + std::to_string(q.rows) + " rows, got " + std::to_string(out.rows));
    if (row0.dim() != 1 || !row0.size(0)) throw Bad("q_row0: expected the sequences' first rows and one number more");
    if (a[6] == Py_None && k.rows != q.rows) throw Bad("k_row0: sequences of " + std::to_string(k.rows) + " key rows need their own");
    p.q = q.p, p.k = k.p, p.v = v.p, p.out = out.p;
    p.ld_q = q.ld, p.ld_k = k.ld, p.ld_v = v.ld, p.ld_out = out.ld;
    p.q_row0 = (const int32_t*)shaped(row0, {row0.size(0)}, I32, "q_row0");
    p.k_row0 = (const int32_t*)optional_here(a[6], {row0.size(0)}, I32, "k_row0", a[13]);
    p.batch = narrow(row0.size(0) - 1, "q_row0");
    p.q_rows = q.rows;
    p.k_rows = k.rows;
    p.scale = real(a[8], "scale");
    p.max_q_len = integer(a[9], "max_q_len");
    p.max_k_len = integer(a[10], "max_k_len");
    const Scratch s = scratch(a[11], a[13]);
    return lib.prompt_attention(&p, s.p, s.bytes, stream_of(a[12]));
}

template <int (*F)(PyObject* const*), Py_ssize_t COUNT>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    try {
        if (n != COUNT) throw Bad("expected " + std::to_string(COUNT) + " arguments, got " + std::to_string(n));
        if (!lib.quantize) throw Bad("the library is not bound");
        return PyLong_FromLong(F(args));
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
        return nullptr;
    }
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    constexpr Py_ssize_t COUNT = sizeof(Library) / sizeof(void*);
    if (n != COUNT) {
        PyErr_SetString(PyExc_ValueError, "expected the addresses of as many functions as there are calls");
        return nullptr;
    }
    void* p[COUNT];
    for (int i = 0; i < COUNT; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a function's address is null");
            return nullptr;
        }
    }
    lib = {(decltype(lib.quantize))p[0], (decltype(lib.add_rmsnorm))p[1], (decltype(lib.swiglu))p[2], (decltype(lib.gemm))p[3],
           (decltype(lib.append))p[4], (decltype(lib.attention))p[5], (decltype(lib.sample))p[6], (decltype(lib.prompt_rmsnorm))p[7],
           (decltype(lib.prompt_gemm))p[8], (decltype(lib.prompt_append))p[9], (decltype(lib.prompt_attention))p[10]};
    Py_RETURN_NONE;
}

#define ENTRY(name, fn) {name, (PyCFunction)(void (*)(void))(fn), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY("bind", bind),
                         ENTRY("quantize", (call<quantize, 4>)),
                         ENTRY("add_rmsnorm", (call<add_rmsnorm, 8>)),
                         ENTRY("swiglu", (call<swiglu, 4>)),
                         ENTRY("gemm", (call<gemm, 6>)),
                         ENTRY("append", (call<append, 12>)),
                         ENTRY("attention", (call<attention, 14>)),
                         ENTRY("sample", (call<sample, 12>)),
                         ENTRY("prompt_rmsnorm", (call<prompt_rmsnorm, 6>)),
                         ENTRY("prompt_gemm", (call<prompt_gemm, 9>)),
                         ENTRY("prompt_append", (call<prompt_append, 11>)),
                         ENTRY("prompt_attention", (call<prompt_attention, 14>)),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
