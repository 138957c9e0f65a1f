// Compiled half of the decoding tensor helpers (decoding.py): checks tensors,
// allocates outputs and temporary workspaces with torch's allocator, and calls
// the C entry points on the current stream of the tensors' device.  A call on
// a few tokens is host work first: the kernels of a decoding step take 3 to 5
// us each, and the same marshalling in Python with ctypes took 7 to 15.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>

#include "quartz.h"

namespace {

using at::Tensor;

#define NEED(ok, ...) TORCH_CHECK_VALUE(ok, __VA_ARGS__)

const Tensor& tensor(PyObject* o, const char* what)
{
    TORCH_CHECK_TYPE(THPVariable_Check(o), what, " must be a tensor");
    return THPVariable_Unpack(o);
}

// a tensor, or undefined for None
Tensor optional(PyObject* o, const char* what) { return o == Py_None ? Tensor() : tensor(o, what); }

int64_t integer(PyObject* o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred())
        throw python_error();
    return v;
}

int32_t small(PyObject* o, const char* what)
{
    const int64_t v = integer(o);
    NEED(v >= INT32_MIN && v <= INT32_MAX, what, " is out of range");
    return (int32_t)v;
}

double real(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred())
        throw python_error();
    return v;
}

int32_t layout_of(PyObject* o)
{
    if (PyUnicode_Check(o)) {
        if (PyUnicode_CompareWithASCIIString(o, "half") == 0)
            return QUARTZ_ROTARY_HALF;
        if (PyUnicode_CompareWithASCIIString(o, "interleaved") == 0)
            return QUARTZ_ROTARY_INTERLEAVED;
    }
    NEED(false, "layout must be \"half\" or \"interleaved\"");
    return 0;
}

// strides count where more than one element is reached
bool strided(const Tensor& t, int64_t dim) { return t.size(dim) > 1 && t.numel() > 0; }
bool unit(const Tensor& t, int64_t dim) { return !strided(t, dim) || t.stride(dim) == 1; }
int64_t stride_of(const Tensor& t, int64_t dim) { return strided(t, dim) ? t.stride(dim) : 0; }

// Whether sum c_k w_k = target has a solution with 0 <= c_k <= most_k: the places
// that a strided tensor reaches, or the differences of two tensors' places.  The
// largest weight goes first: what the others reach in all leaves it few values, one
// or two where strides nest as they do in views of one tensor.
class Combination {
public:
    void add(int64_t weight, int64_t most)
    {
        if (most <= 0)
            return;
        int i = 0;
        while (i < count_ && weight_[i] > weight)
            ++i;
        if (i < count_ && weight_[i] == weight) {
            most_[i] += most;
            return;
        }
        NEED(count_ < kTerms, "tensors of that many dimensions cannot be told apart");
        for (int j = count_++; j > i; --j) {
            weight_[j] = weight_[j - 1];
            most_[j] = most_[j - 1];
        }
        weight_[i] = weight;
        most_[i] = most;
    }

    bool reaches(int64_t target)
    {
        reach_[count_] = 0;
        dense_[count_] = true;
        for (int k = count_ - 1; k >= 0; --k) {
            reach_[k] = reach_[k + 1] + weight_[k] * most_[k];
            dense_[k] = dense_[k + 1] && weight_[k] <= reach_[k + 1] + 1;
        }
        tries_ = 0;
        return search(0, target);
    }

private:
    bool search(int k, int64_t target)
    {
        if (target < 0 || target > reach_[k])
            return false;
        if (dense_[k])                             // every number up to there
            return true;
        NEED(++tries_ <= kTries, "tensors of these strides cannot be told apart");
        const int64_t rest = target - reach_[k + 1];
        int64_t c = rest > 0 ? (rest + weight_[k] - 1) / weight_[k] : 0;
        for (const int64_t last = std::min(most_[k], target / weight_[k]); c <= last; ++c)
            if (search(k + 1, target - c * weight_[k]))
                return true;
        return false;
    }

    static constexpr int kTerms = 16, kTries = 100000;
    int64_t weight_[kTerms], most_[kTerms], reach_[kTerms + 1];
    bool dense_[kTerms + 1];
    int count_ = 0, tries_ = 0;
};

// bytes from a tensor's first element to the end of its last
int64_t extent(const Tensor& t)
{
    int64_t elements = 1;
    for (int64_t i = 0; i < t.dim(); ++i)
        elements += (t.size(i) - 1) * t.stride(i);
    return elements * t.element_size();
}

// two tensors with a byte in common
bool share(const Tensor& a, const Tensor& b)
{
    if (!a.defined() || !b.defined() || a.numel() == 0 || b.numel() == 0 || a.device() != b.device())
        return false;
    const int64_t a0 = reinterpret_cast<int64_t>(a.data_ptr()), b0 = reinterpret_cast<int64_t>(b.data_ptr());
    const int64_t b_extent = extent(b);
    if (a0 + extent(a) <= b0 || b0 + b_extent <= a0)
        return false;
    // a0 + i = b0 + j for places i of a and j of b: i + (b's extent - 1 - j) = b0 - a0 + b's extent - 1
    Combination c;
    c.add(1, a.element_size() - 1 + b.element_size() - 1);
    for (const Tensor* t : {&a, &b})
        for (int64_t i = 0; i < t->dim(); ++i)
            if (t->stride(i) != 0)
                c.add(t->stride(i) * t->element_size(), t->size(i) - 1);
    return c.reaches(b0 - a0 + b_extent - 1);
}

// a tensor that reaches one element twice
bool repeats(const Tensor& t)
{
    if (t.numel() == 0 || t.is_contiguous())
        return false;
    for (int64_t k = 0; k < t.dim(); ++k) {
        if (t.size(k) == 1)
            continue;
        if (t.stride(k) == 0)
            return true;
        // two places apart by one step of k or more, and by any of the others' steps either way: none
        Combination c;
        c.add(t.stride(k), t.size(k) - 2);
        int64_t target = -t.stride(k);
        for (int64_t i = 0; i < t.dim(); ++i) {
            if (i == k || t.size(i) == 1)
                continue;
            if (t.stride(i) != 0)
                c.add(t.stride(i), 2 * (t.size(i) - 1));
            target += (t.size(i) - 1) * t.stride(i);
        }
        if (c.reaches(target))
            return true;
    }
    return false;
}

// an output whose elements are distinct, and none of them an input's
template <typename... T>
void fresh(const Tensor& out, const T&... inputs)
{
    if (!out.defined())
        return;
    NEED(!repeats(out), "out must not hold one element twice");
    NEED(!(share(out, inputs) || ...), "out must not share memory with an input");
}

// a caller's workspace
template <typename... T>
void scratch(const Tensor& workspace, const T&... inputs)
{
    if (!workspace.defined())
        return;
    NEED(workspace.is_contiguous(), "the workspace must be contiguous");
    NEED(!(share(workspace, inputs) || ...), "the workspace must not share memory with an input");
}

bool in_place(const Tensor& out, const Tensor& x)
{
    if (!out.defined() || out.data_ptr() != x.data_ptr() || out.sizes() != x.sizes())
        return false;
    for (int64_t i = 0; i < x.dim(); ++i)
        if (stride_of(out, i) != stride_of(x, i))
            return false;
    return true;
}

void* address(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

template <typename... T>
void same_device(const Tensor& a, const T&... others)
{
    [[maybe_unused]] auto check = [&](const Tensor& t) {
        NEED(!t.defined() || t.device() == a.device(), "all tensors must be on one device: ", t.device(), " beside ",
             a.device());
    };
    (check(others), ...);
    NEED(a.is_cuda(), "the tensors must be on a GPU, not on ", a.device());
}

// `call` with the raw current stream of the tensors' device, that device being current
template <typename F>
void launch(const char* name, const Tensor& on, F&& call)
{
    const c10::hip::OptionalHIPGuard guard(on.device().index());
    const hipStream_t stream = c10::hip::getCurrentHIPStream(on.device().index()).stream();
    quartz_status status;
    Py_BEGIN_ALLOW_THREADS
    status = call(stream);
    Py_END_ALLOW_THREADS
    if (status == QUARTZ_OK)
        return;
    PyObject* module = PyImport_ImportModule("paper_2509_26436_amd");
    PyObject* type = module ? PyObject_GetAttrString(module, "QuartzError") : nullptr;
    PyObject* error = type ? PyObject_CallFunction(type, "is", (int)status, name) : nullptr;
    if (error)
        PyErr_SetObject(type, error);
    Py_XDECREF(error);
    Py_XDECREF(type);
    Py_XDECREF(module);
    throw python_error();
}

// leading dimension of a bf16 matrix with unit column stride
int64_t rows_of(const Tensor& t, const char* what)
{
    NEED(t.scalar_type() == at::kBFloat16 && t.dim() == 2 && unit(t, 1), what,
         " must be a 2-D bf16 tensor with unit column stride");
    return strided(t, 0) ? t.stride(0) : (t.size(1) + 7) / 8 * 8;
}

struct Mx {
    Tensor codes, scales;
    int64_t rows, K;
};

Mx mx_of(PyObject* codes, PyObject* scales, PyObject* rows, PyObject* K)
{
    Mx t{tensor(codes, "codes"), tensor(scales, "scales"), integer(rows), integer(K)};
    NEED(t.K >= 0 && t.K % 64 == 0 && t.rows >= 0, "rows must not be negative, K must be a multiple of 64");
    NEED(t.codes.scalar_type() == at::kByte && t.scales.scalar_type() == at::kByte && t.codes.dim() == 3 &&
             t.scales.dim() == 3 && t.codes.size(0) == t.K / 32 && t.codes.size(1) == t.rows &&
             t.codes.size(2) == 16 && t.scales.size(0) == (t.K + 127) / 128 && t.scales.size(1) == t.rows &&
             t.scales.size(2) == 4 && t.codes.is_contiguous() && t.scales.is_contiguous(),
         "codes must be contiguous uint8 [K/32, rows, 16], scales contiguous uint8 [ceil(K/128), rows, 4]");
    NEED(t.codes.device() == t.scales.device(), "codes and scales must be on one device");
    return t;
}

const uint8_t* bytes(const Tensor& t) { return static_cast<const uint8_t*>(t.data_ptr()); }

#define ARGUMENTS(count)                                                                   \
    if (n != count) {                                                                      \
        PyErr_Format(PyExc_TypeError, "%d arguments are wanted, got %zd", count, n);       \
        return nullptr;                                                                    \
    }

// (codes, scales, rows, K)
PyObject* check_mx(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(4)
    mx_of(a[0], a[1], a[2], a[3]);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// (x) -> codes, scales
PyObject* quantize_new(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(1)
    const Tensor& x = tensor(a[0], "x");
    const int64_t ldx = rows_of(x, "x"), M = x.size(0), K = x.size(1);
    NEED(K % 64 == 0, "K must be a multiple of 64");
    same_device(x);
    const auto options = x.options().dtype(at::kByte).requires_grad(false);
    Tensor codes = at::empty({K / 32, M, 16}, options), scales = at::empty({(K + 127) / 128, M, 4}, options);
    launch("quartz_mxfp4_quantize", x, [&](hipStream_t s) {
        return quartz_mxfp4_quantize(x.data_ptr(), M, K, ldx, static_cast<uint8_t*>(codes.data_ptr()),
                                     static_cast<uint8_t*>(scales.data_ptr()), s);
    });
    PyObject* both = PyTuple_New(2);
    PyTuple_SET_ITEM(both, 0, THPVariable_Wrap(std::move(codes)));
    PyTuple_SET_ITEM(both, 1, THPVariable_Wrap(std::move(scales)));
    return both;
    END_HANDLE_TH_ERRORS
}

// (x, codes, scales, rows, K)
PyObject* quantize_into(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(5)
    const Tensor& x = tensor(a[0], "x");
    const int64_t ldx = rows_of(x, "x"), M = x.size(0), K = x.size(1);
    const Mx t = mx_of(a[1], a[2], a[3], a[4]);
    NEED(t.rows == M && t.K == K, "out must have x's rows and K");
    fresh(t.codes, x, t.scales);
    fresh(t.scales, x);
    same_device(x, t.codes);
    launch("quartz_mxfp4_quantize", x, [&](hipStream_t s) {
        return quartz_mxfp4_quantize(x.data_ptr(), M, K, ldx, static_cast<uint8_t*>(t.codes.data_ptr()),
                                     static_cast<uint8_t*>(t.scales.data_ptr()), s);
    });
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// (codes, scales, rows, K, out) -> out
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(5)
    const Mx t = mx_of(a[0], a[1], a[2], a[3]);
    Tensor out = optional(a[4], "out");
    fresh(out, t.codes, t.scales);
    same_device(t.codes, out);
    if (!out.defined())
        out = at::empty({t.rows, t.K}, t.codes.options().dtype(at::kBFloat16));
    const int64_t ldy = rows_of(out, "out");
    NEED(out.size(0) == t.rows && out.size(1) == t.K, "out must be bf16 [rows, K]");
    launch("quartz_mxfp4_dequantize", out, [&](hipStream_t s) {
        return quartz_mxfp4_dequantize(bytes(t.codes), bytes(t.scales), t.rows, t.K, out.data_ptr(), ldy, s);
    });
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// the columns of a layer's output that it writes
Tensor written(const Tensor& out, int64_t N)
{
    return out.defined() && out.dim() == 2 && out.size(1) > N ? out.narrow(1, 0, N) : out;
}

// checks bias and out of a layer [M, N]; returns ldy
int64_t layer_out(const Tensor& on, int64_t M, int64_t N, const Tensor& bias, Tensor& out)
{
    NEED(!bias.defined() || (bias.scalar_type() == at::kBFloat16 && bias.dim() == 1 && bias.size(0) == N && unit(bias, 0)),
         "bias must be bf16 [N], contiguous");
    if (!out.defined()) {
        out = at::empty({M, N}, on.options().dtype(at::kBFloat16).requires_grad(false));
        return N;
    }
    const int64_t ldy = rows_of(out, "out");
    NEED(out.size(0) == M && out.size(1) >= N, "out must be bf16 [M, >= N]");
    return ldy;
}

// (x codes, scales, rows, K, w codes, scales, rows, K, bias, epilogue, out) -> out
PyObject* linear_mx(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(11)
    const Mx x = mx_of(a[0], a[1], a[2], a[3]), w = mx_of(a[4], a[5], a[6], a[7]);
    const Tensor bias = optional(a[8], "bias");
    const int32_t epilogue = small(a[9], "epilogue");
    Tensor out = optional(a[10], "out");
    NEED(x.K == w.K, "K mismatch between activations and weights");
    fresh(written(out, w.rows), x.codes, x.scales, w.codes, w.scales, bias);
    same_device(w.codes, x.codes, bias, out);
    const int64_t ldy = layer_out(w.codes, x.rows, w.rows, bias, out);
    launch("quartz_mxfp4_linear", out, [&](hipStream_t s) {
        return quartz_mxfp4_linear(bytes(x.codes), bytes(x.scales), bytes(w.codes), bytes(w.scales), address(bias),
                                   out.data_ptr(), x.rows, w.rows, w.K, ldy, epilogue, s);
    });
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// bytes of a caller's workspace, or of a temporary one of `need`
size_t workspace_of(Tensor& workspace, size_t need, const Tensor& on)
{
    if (workspace.defined())
        return workspace.nbytes();
    if (need > 0)
        workspace = at::empty({(int64_t)need}, on.options().dtype(at::kByte).requires_grad(false));
    return need;
}

// (x, w codes, scales, rows, K, bias, epilogue, out, workspace) -> out
PyObject* linear_bf16(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(9)
    const Tensor& x = tensor(a[0], "x");
    const Mx w = mx_of(a[1], a[2], a[3], a[4]);
    const Tensor bias = optional(a[5], "bias");
    const int32_t epilogue = small(a[6], "epilogue");
    Tensor out = optional(a[7], "out"), workspace = optional(a[8], "workspace");
    const int64_t ldx = rows_of(x, "x"), M = x.size(0);
    NEED(x.size(1) == w.K, "K mismatch between activations and weights");
    fresh(written(out, w.rows), x, w.codes, w.scales, bias, workspace);
    scratch(workspace, x, w.codes, w.scales, bias);
    same_device(x, w.codes, bias, out, workspace);
    const int64_t ldy = layer_out(x, M, w.rows, bias, out);
    const size_t size = workspace_of(workspace, quartz_mxfp4_linear_workspace_bytes(M, w.K), x);
    launch("quartz_mxfp4_linear_bf16", x, [&](hipStream_t s) {
        return quartz_mxfp4_linear_bf16(x.data_ptr(), ldx, bytes(w.codes), bytes(w.scales), address(bias),
                                        out.data_ptr(), M, w.rows, w.K, ldy, epilogue, address(workspace), size, s);
    });
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

void heads_of(const Tensor& t, const char* what)
{
    NEED(t.scalar_type() == at::kBFloat16 && t.dim() == 3 && unit(t, 2), what,
         " must be a bf16 [tokens, heads, d] tensor with unit stride along d");
}

const int32_t* int32_of(const Tensor& t, int64_t count, const char* what)
{
    NEED(t.scalar_type() == at::kInt && t.dim() == 1 && t.size(0) == count && unit(t, 0), what,
         " must be a contiguous int32 tensor of ", count);
    return static_cast<const int32_t*>(t.data_ptr());
}

int64_t rotated(const Tensor& freqs, int64_t d)
{
    NEED(freqs.scalar_type() == at::kLong && freqs.dim() == 1 && freqs.is_contiguous() && 2 * freqs.size(0) <= d,
         "freqs must be a contiguous int64 tensor of at most d / 2 (rotary_frequencies)");
    return 2 * freqs.size(0);
}

// (x, positions, freqs, layout, inverse, magnitude, out) -> out
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(7)
    const Tensor& x = tensor(a[0], "x");
    const Tensor &positions = tensor(a[1], "positions"), &freqs = tensor(a[2], "freqs");
    heads_of(x, "x");
    const int64_t tokens = x.size(0), heads = x.size(1), d = x.size(2), rot = rotated(freqs, d);
    const int32_t* p = int32_of(positions, tokens, "positions");
    const int32_t layout = layout_of(a[3]);
    const int inverse = PyObject_IsTrue(a[4]);
    if (inverse < 0)
        throw python_error();
    const float magnitude = (float)real(a[5]);
    Tensor out = optional(a[6], "out");
    fresh(out, in_place(out, x) ? Tensor() : x, positions, freqs);
    same_device(x, positions, freqs, out);
    if (!out.defined())
        out = at::empty_like(x, x.options().requires_grad(false));
    heads_of(out, "out");
    NEED(out.sizes() == x.sizes(), "out must have x's shape");
    launch("quartz_rotary", x, [&](hipStream_t s) {
        return quartz_rotary(x.data_ptr(), out.data_ptr(), tokens, heads, d, rot, stride_of(x, 0), stride_of(x, 1),
                             stride_of(out, 0), stride_of(out, 1), p,
                             static_cast<const int64_t*>(freqs.data_ptr()), layout, inverse, magnitude, s);
    });
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

struct Cache {
    Tensor k, v, table;
    float k_scale, v_scale;
    int32_t type;
    int64_t pages, heads, page, d, stride;
};

// a page of [heads][page][d] is contiguous
bool page_contiguous(const Tensor& t)
{
    return t.is_contiguous() || (t.stride(3) == 1 && (t.stride(2) == t.size(3) || t.size(2) == 1) &&
                                 (t.stride(1) == t.size(2) * t.size(3) || t.size(1) == 1));
}

Cache cache_of(PyObject* k, PyObject* v, PyObject* table, PyObject* k_scale, PyObject* v_scale)
{
    Cache c{tensor(k, "k"), tensor(v, "v"), tensor(table, "table"), (float)real(k_scale), (float)real(v_scale),
            0, 0, 0, 0, 0, 0};
    const auto type = c.k.scalar_type();
    NEED((type == at::kBFloat16 || type == at::kFloat8_e4m3fn) && c.v.scalar_type() == type,
         "k and v must both be bf16 or both float8_e4m3fn");
    NEED(c.k.dim() == 4 && c.k.sizes() == c.v.sizes(), "k and v must be [pages, heads, page_size, d], both alike");
    NEED(page_contiguous(c.k) && page_contiguous(c.v) && (!strided(c.k, 0) || c.k.stride(0) == c.v.stride(0)),
         "a page must be contiguous, and k and v must have one page stride");
    NEED(c.table.scalar_type() == at::kInt && c.table.dim() == 2 && unit(c.table, 1),
         "table must be an int32 [sequences, pages] tensor with unit column stride");
    NEED(c.k.device() == c.v.device() && c.k.device() == c.table.device(), "k, v and table must be on one device");
    c.type = type == at::kBFloat16 ? QUARTZ_CACHE_BF16 : QUARTZ_CACHE_E4M3;
    c.pages = c.k.size(0);
    c.heads = c.k.size(1);
    c.page = c.k.size(2);
    c.d = c.k.size(3);
    c.stride = strided(c.k, 0) ? c.k.stride(0) : c.heads * c.page * c.d;
    return c;
}

const int32_t* table_at(const Cache& c) { return static_cast<const int32_t*>(c.table.data_ptr()); }
int64_t table_stride(const Cache& c) { return strided(c.table, 0) ? c.table.stride(0) : c.table.size(1); }

// (k, v, table, k_scale, v_scale)
PyObject* check_cache(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(5)
    cache_of(a[0], a[1], a[2], a[3], a[4]);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// (the cache's five, k, v, positions, sequences, freqs, layout, magnitude)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(12)
    const Cache c = cache_of(a[0], a[1], a[2], a[3], a[4]);
    const Tensor &k = tensor(a[5], "k"), &v = tensor(a[6], "v"), &positions = tensor(a[7], "positions");
    const Tensor sequences = optional(a[8], "sequences"), freqs = optional(a[9], "freqs");
    heads_of(k, "k");
    heads_of(v, "v");
    NEED(k.sizes() == v.sizes() && k.size(1) == c.heads && k.size(2) == c.d,
         "k and v must be [tokens, heads, d] with the cache's heads and d");
    const int64_t tokens = k.size(0);
    const int32_t* p = int32_of(positions, tokens, "positions");
    const int32_t* s = sequences.defined() ? int32_of(sequences, tokens, "sequences") : nullptr;
    const int64_t rot = freqs.defined() ? rotated(freqs, c.d) : 0;
    const int32_t layout = layout_of(a[10]);
    const float magnitude = (float)real(a[11]);
    NEED(!share(c.k, c.v), "the cache's keys and values must not share memory");
    for (const Tensor* pages : {&c.k, &c.v})
        NEED(!share(*pages, k) && !share(*pages, v) && !share(*pages, positions) && !share(*pages, sequences) &&
                 !share(*pages, freqs) && !share(*pages, c.table),
             "the cache must not share memory with an input");
    same_device(c.k, k, v, positions, sequences, freqs);
    launch("quartz_paged_append", k, [&](hipStream_t stream) {
        return quartz_paged_append(k.data_ptr(), v.data_ptr(), tokens, c.heads, c.d, stride_of(k, 0),
                                   stride_of(k, 1), stride_of(v, 0), stride_of(v, 1), p, s,
                                   static_cast<const int64_t*>(address(freqs)), rot, layout, magnitude,
                                   c.k.data_ptr(), c.v.data_ptr(), c.type, c.k_scale, c.v_scale, c.pages, c.page,
                                   c.stride, table_at(c), c.table.size(0), c.table.size(1), table_stride(c), stream);
    });
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// (the cache's five, q, lengths, scale, window, out, workspace) -> out
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(11)
    const Cache c = cache_of(a[0], a[1], a[2], a[3], a[4]);
    const Tensor &q = tensor(a[5], "q"), &lengths = tensor(a[6], "lengths");
    heads_of(q, "q");
    const int64_t sequences = q.size(0), heads = q.size(1), d = q.size(2), window = integer(a[8]);
    NEED(d == c.d && c.table.size(0) == sequences && c.heads > 0 && heads % c.heads == 0,
         "q must be [sequences, heads, d] with the cache's d, a row of the table a sequence, and heads a multiple of "
         "the cache's");
    const int32_t* len = int32_of(lengths, sequences, "lengths");
    const float scale = a[7] == Py_None ? (float)(1.0 / std::sqrt((double)d)) : (float)real(a[7]);
    Tensor out = optional(a[9], "out"), workspace = optional(a[10], "workspace");
    fresh(out, q, c.k, c.v, c.table, lengths, workspace);
    scratch(workspace, q, c.k, c.v, c.table, lengths);
    same_device(c.k, q, lengths, out, workspace);
    const c10::hip::OptionalHIPGuard guard(q.device().index());    // the workspace is sized for its compute units
    if (!out.defined())
        out = at::empty({sequences, heads, d}, q.options().requires_grad(false));
    heads_of(out, "out");
    NEED(out.sizes() == q.sizes(), "out must have q's shape");
    const size_t size = workspace_of(
        workspace, quartz_paged_attention_workspace_bytes(sequences, heads, c.heads, d, c.page, c.table.size(1), window),
        q);
    launch("quartz_paged_attention", q, [&](hipStream_t s) {
        return quartz_paged_attention(q.data_ptr(), out.data_ptr(), sequences, heads, c.heads, d, stride_of(q, 0),
                                      stride_of(q, 1), stride_of(out, 0), stride_of(out, 1), c.k.data_ptr(),
                                      c.v.data_ptr(), c.type, c.k_scale, c.v_scale, c.pages, c.page, c.stride, table_at(c),
                                      c.table.size(1), table_stride(c), len, scale, window, address(workspace), size,
                                      s);
    });
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// (q, k, positions, freqs, q_weight, k_weight, eps, axes, layout, magnitude, q_out, k_out) -> q_out, k_out
PyObject* head_norm_rotary(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(12)
    const Tensor& q = tensor(a[0], "q");
    const Tensor k = optional(a[1], "k"), &positions = tensor(a[2], "positions"), &freqs = tensor(a[3], "freqs");
    const Tensor weight[2] = {optional(a[4], "q_weight"), optional(a[5], "k_weight")}, axes = optional(a[7], "axes");
    heads_of(q, "q");
    const int64_t tokens = q.size(0), d = q.size(2), rot = rotated(freqs, d);
    if (k.defined()) {
        heads_of(k, "k");
        NEED(k.size(0) == tokens && k.size(2) == d, "k must be [tokens, heads, d] with q's tokens and d");
    }
    NEED(positions.scalar_type() == at::kInt && (positions.dim() == 1 || positions.dim() == 2) &&
             positions.size(-1) == tokens && unit(positions, -1),
         "positions must be int32 [tokens] or [axes, tokens] with unit stride along the tokens");
    const int64_t axis_count = positions.dim() == 2 ? positions.size(0) : 1;
    const int64_t axis_stride = positions.dim() == 2 ? stride_of(positions, 0) : 0;
    NEED(axis_count > 0, "positions must have an axis");
    const int32_t* axis = axes.defined() ? int32_of(axes, rot / 2, "axes") : nullptr;
    const bool norm = a[6] != Py_None;
    const float eps = norm ? (float)real(a[6]) : 0.0f, magnitude = (float)real(a[9]);
    for (const Tensor& w : weight)
        NEED(!w.defined() || (w.scalar_type() == at::kBFloat16 && w.dim() == 1 && w.size(0) == d && unit(w, 0)),
             "weights must be bf16 [d], contiguous");
    NEED(norm || (!weight[0].defined() && !weight[1].defined()), "weights belong to a norm (eps is None)");
    NEED(k.defined() || !weight[1].defined(), "k_weight without k");
    const int32_t layout = layout_of(a[8]);
    const Tensor* x[2] = {&q, &k};
    Tensor out[2] = {optional(a[10], "q_out"), optional(a[11], "k_out")};
    NEED(k.defined() || !out[1].defined(), "k_out without k");
    for (int i = 0; i < 2; ++i)
        fresh(out[i], in_place(out[i], *x[i]) ? Tensor() : *x[i], *x[1 - i], positions, freqs, weight[0], weight[1], axes);
    NEED(!share(out[0], out[1]), "the outputs must not share memory");
    same_device(q, k, positions, freqs, weight[0], weight[1], axes, out[0], out[1]);
    for (int i = 0; i < 2; ++i) {
        if (!x[i]->defined())
            continue;
        if (!out[i].defined())
            out[i] = at::empty(x[i]->sizes(), x[i]->options().requires_grad(false));
        heads_of(out[i], "out");
        NEED(out[i].sizes() == x[i]->sizes(), "outputs must have the inputs' shapes");
    }
    const auto stride = [](const Tensor& t, int64_t dim) { return t.defined() ? stride_of(t, dim) : 0; };
    launch("quartz_head_norm_rotary", q, [&](hipStream_t s) {
        return quartz_head_norm_rotary(
            q.data_ptr(), out[0].data_ptr(), q.size(1), stride(q, 0), stride(q, 1), stride(out[0], 0), stride(out[0], 1),
            address(weight[0]), address(k), address(out[1]), k.defined() ? k.size(1) : 0, stride(k, 0), stride(k, 1),
            stride(out[1], 0), stride(out[1], 1), address(weight[1]), tokens, d, rot,
            static_cast<const int32_t*>(positions.data_ptr()), axis_count, axis_stride, axis,
            static_cast<const int64_t*>(freqs.data_ptr()), layout, norm, eps, magnitude, s);
    });
    PyObject* both = PyTuple_New(2);
    for (int i = 0; i < 2; ++i) {
        if (!x[i]->defined())
            Py_INCREF(Py_None);
        PyTuple_SET_ITEM(both, i, x[i]->defined() ? THPVariable_Wrap(std::move(out[i])) : Py_None);
    }
    return both;
    END_HANDLE_TH_ERRORS
}

// (the cache's five, q, starts, lengths, tree, scale, window, cap, slopes, prefix, out, workspace) -> out
PyObject* prompt_attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(16)
    const Cache c = cache_of(a[0], a[1], a[2], a[3], a[4]);
    const Tensor &q = tensor(a[5], "q"), &starts = tensor(a[6], "starts"), &lengths = tensor(a[7], "lengths");
    const Tensor tree = optional(a[8], "tree"), slopes = optional(a[12], "slopes"), prefix = optional(a[13], "prefix");
    heads_of(q, "q");
    const int64_t tokens = q.size(0), heads = q.size(1), d = q.size(2), sequences = c.table.size(0), window = integer(a[10]);
    NEED(d == c.d && c.heads > 0 && heads % c.heads == 0,
         "q must be [tokens, heads, d] with the cache's d and heads a multiple of the cache's");
    const int32_t* first = int32_of(starts, sequences + 1, "starts");
    const int32_t* len = int32_of(lengths, sequences, "lengths");
    const int32_t* before = prefix.defined() ? int32_of(prefix, sequences, "prefix") : nullptr;
    NEED(!slopes.defined() || (slopes.scalar_type() == at::kFloat && slopes.dim() == 1 && slopes.size(0) == heads && unit(slopes, 0)),
         "slopes must be a contiguous fp32 tensor of ", heads);
    NEED(!tree.defined() || (tree.scalar_type() == at::kLong && tree.dim() == 2 && tree.size(0) == tokens && tree.size(1) > 0 && unit(tree, 1)),
         "tree must be an int64 [tokens, words] tensor with unit column stride");
    const float scale = a[9] == Py_None ? (float)(1.0 / std::sqrt((double)d)) : (float)real(a[9]);
    const float cap = (float)real(a[11]);
    Tensor out = optional(a[14], "out"), workspace = optional(a[15], "workspace");
    fresh(out, q, c.k, c.v, c.table, starts, lengths, tree, slopes, prefix, workspace);
    scratch(workspace, q, c.k, c.v, c.table, starts, lengths, tree, slopes, prefix);
    same_device(c.k, q, starts, lengths, tree, slopes, prefix, out, workspace);
    const c10::hip::OptionalHIPGuard guard(q.device().index());    // the workspace is sized for its compute units
    if (!out.defined())
        out = at::empty({tokens, heads, d}, q.options().requires_grad(false));
    heads_of(out, "out");
    NEED(out.sizes() == q.sizes(), "out must have q's shape");
    const size_t size = workspace_of(
        workspace, quartz_paged_prompt_workspace_bytes(tokens, sequences, heads, c.heads, d, c.page, c.table.size(1)), q);
    const auto call = [&](auto entry, auto... own) {
        return [&, entry, own...](hipStream_t s) {
            return entry(q.data_ptr(), out.data_ptr(), tokens, sequences, heads, c.heads, d, stride_of(q, 0),
                         stride_of(q, 1), stride_of(out, 0), stride_of(out, 1), c.k.data_ptr(), c.v.data_ptr(), c.type,
                         c.k_scale, c.v_scale, c.pages, c.page, c.stride, table_at(c), c.table.size(1), table_stride(c),
                         first, len, own..., address(workspace), size, s);
        };
    };
    if (tree.defined())
        launch("quartz_paged_tree_attention", q,
               call(quartz_paged_tree_attention, static_cast<const uint64_t*>(tree.data_ptr()), tree.size(1),
                    stride_of(tree, 0), scale, cap));
    else
        launch("quartz_paged_prompt_attention", q,
               call(quartz_paged_prompt_attention, scale, window, cap, static_cast<const float*>(address(slopes)), before));
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// (the cache's five, first, kept)
PyObject* keep(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(7)
    const Cache c = cache_of(a[0], a[1], a[2], a[3], a[4]);
    const Tensor &first = tensor(a[5], "first"), &kept = tensor(a[6], "kept");
    const int64_t sequences = c.table.size(0);
    const int32_t* begin = int32_of(first, sequences, "first");
    NEED(kept.scalar_type() == at::kInt && kept.dim() == 2 && kept.size(0) == sequences && unit(kept, 1),
         "kept must be an int32 [sequences, most] tensor with unit column stride, a row of the table a sequence");
    NEED(!strided(kept, 0) || kept.stride(0) >= kept.size(1), "the rows of kept must not overlap");
    NEED(!share(c.k, c.v), "the cache's keys and values must not share memory");
    for (const Tensor* pages : {&c.k, &c.v})
        NEED(!share(*pages, first) && !share(*pages, kept) && !share(*pages, c.table),
             "the cache must not share memory with an input");
    same_device(c.k, first, kept);
    launch("quartz_paged_keep", c.k, [&](hipStream_t s) {
        return quartz_paged_keep(begin, static_cast<const int32_t*>(kept.data_ptr()), sequences, kept.size(1),
                                 strided(kept, 0) ? kept.stride(0) : kept.size(1), c.k.data_ptr(), c.v.data_ptr(), c.type,
                                 c.heads, c.d, c.pages, c.page, c.stride, table_at(c), c.table.size(1), table_stride(c), s);
    });
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction fast() { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)); }

PyMethodDef kMethods[] = {
    {"check_mx", fast<check_mx>(), METH_FASTCALL, nullptr},
    {"quantize_new", fast<quantize_new>(), METH_FASTCALL, nullptr},
    {"quantize_into", fast<quantize_into>(), METH_FASTCALL, nullptr},
    {"dequantize", fast<dequantize>(), METH_FASTCALL, nullptr},
    {"linear_mx", fast<linear_mx>(), METH_FASTCALL, nullptr},
    {"linear_bf16", fast<linear_bf16>(), METH_FASTCALL, nullptr},
    {"rotary", fast<rotary>(), METH_FASTCALL, nullptr},
    {"check_cache", fast<check_cache>(), METH_FASTCALL, nullptr},
    {"append", fast<append>(), METH_FASTCALL, nullptr},
    {"attention", fast<attention>(), METH_FASTCALL, nullptr},
    {"head_norm_rotary", fast<head_norm_rotary>(), METH_FASTCALL, nullptr},
    {"prompt_attention", fast<prompt_attention>(), METH_FASTCALL, nullptr},
    {"keep", fast<keep>(), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_decoding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__decoding() { return PyModule_Create(&kModule); }
