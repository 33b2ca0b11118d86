// The part of paper_1902_01064_b200/nn.py between its Python signatures and the C ABI: checks of torch tensors, outputs and
// workspaces from torch's allocator, the current stream.  A small call costs what its host side costs (a product of 4
// groups of 32 rows: 12 us from Python, of which the GPU needs 5), so this part is native.  It computes nothing; the
// entries of the loaded library (its ordinary or its bounds-checked build) are handed over by address.
#include <ATen/ATen.h>
#include <ATen/MemoryOverlap.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <optional>
#include <sstream>
#include <string>

#include "hop.h"

namespace {

PyObject* g_error = nullptr;            // hop.HopError
struct {
    decltype(&hop_linear_workspace) linear_workspace;
    decltype(&hop_linear) linear;
    decltype(&hop_norm_workspace) norm_workspace;
    decltype(&hop_norm_forward) norm_forward;
    decltype(&hop_norm_backward) norm_backward;
    decltype(&hop_dropout) dropout;
} g_api;

template <typename... A>
[[noreturn]] void refuse(int code, const A&... a) {
    std::ostringstream s;
    (s << ... << a);
    PyObject* args = Py_BuildValue("(is)", code, s.str().c_str());
    if (args) {
        PyErr_SetObject(g_error, args);
        Py_DECREF(args);
    }
    throw python_error();
}
template <typename... A> [[noreturn]] void bad(const A&... a) { refuse(HOP_E_ARG, a...); }

int code_of(at::ScalarType t) { return t == at::kFloat ? HOP_DT_F32 : t == at::kHalf ? HOP_DT_F16 : t == at::kBFloat16 ? HOP_DT_BF16 : -1; }

const at::Tensor& tensor(const char* name, PyObject* o) {
    if (!THPVariable_Check(o)) bad(name, ": not a tensor");
    return THPVariable_Unpack(o);
}
// A row array: 2-D (leading dimensions joined when they can be viewed as one), unit stride along the columns
at::Tensor rows_of(const char* name, const at::Tensor& given, const at::Tensor* like = nullptr, int64_t r = -1, int64_t c = -1,
                   std::optional<at::ScalarType> dtype = std::nullopt) {
    at::Tensor t = given;
    if (t.dim() != 2) {
        if (t.dim() == 0) bad(name, ": a scalar");
        if (t.numel() == 0) {
            int64_t lead = 1;
            for (int64_t i = 0; i + 1 < t.dim(); ++i) lead *= t.size(i);
            t = t.reshape({lead, t.size(-1)});
        } else {
            try {
                t = t.view({-1, t.size(-1)});
            } catch (const c10::Error&) {
                bad(name, ": leading dimensions of strides ", given.strides(), " do not join into rows");
            }
        }
    }
    if (!t.is_cuda()) bad(name, ": on ", t.device(), ", not on a CUDA device");
    if (like) {
        const at::ScalarType want = dtype.value_or(like->scalar_type());
        if (t.device() != like->device() || t.scalar_type() != want) bad(name, ": ", t.scalar_type(), " on ", t.device(), ", expected ", want, " on ", like->device());
    }
    if ((r >= 0 && t.size(0) != r) || (c >= 0 && t.size(1) != c)) bad(name, ": shape ", t.sizes(), ", expected [", r, ", ", c, "]");
    if (t.stride(1) != 1 && t.size(1) > 1 && t.size(0)) bad(name, ": columns of stride ", t.stride(1));     // (without rows there is nothing to stride over)
    return t;
}
// A caller's tensor that is written: autograd records no such write, so it is refused where one would be expected ...
void writable(const char* name, const at::Tensor& t) {
    if (t.requires_grad() && c10::GradMode::is_enabled()) bad(name, ": requires a gradient, and what is written into it would have none (detach it, or write under no_grad)");
}
// ... and made known to what saved the tensor, as an in-place operator of torch does
void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// A destination in an operand's memory is written while the operand is read.  Views side by side in one buffer pass: of strided
// ones only a common first element is known without walking them.
void apart(const char* name, const at::Tensor& out, const at::Tensor& operand) {
    if (!out.numel() || !operand.numel() || !out.is_alias_of(operand)) return;
    const at::MemOverlapStatus s = at::get_overlap_status(out, operand);
    if (s == at::MemOverlapStatus::Full || s == at::MemOverlapStatus::Partial || out.const_data_ptr() == operand.const_data_ptr())
        bad(name, ": shares memory with an operand of the call");
}
at::Tensor row_out(const char* name, PyObject* out, const at::Tensor& like, int64_t r, int64_t c, at::ScalarType dtype) {
    if (out == Py_None) return at::empty({r, c}, like.options().dtype(dtype));
    writable(name, tensor(name, out));
    at::Tensor t = rows_of(name, tensor(name, out), &like, r, c, dtype);
    if (r > 1 && t.stride(0) < c) bad(name, ": rows of stride ", t.stride(0), " overlap");
    return t;
}
// A new row array in the shape of `given`, and its rows
struct Fresh { at::Tensor whole, rows; };
Fresh fresh_like(const at::Tensor& given, const at::Tensor& rows) {
    if (given.dim() == 2) { const at::Tensor t = at::empty({rows.size(0), rows.size(1)}, rows.options()); return {t, t}; }
    const at::Tensor t = at::empty(given.sizes(), rows.options());
    return {t, t.view({rows.size(0), rows.size(1)})};
}
struct Groups { const int32_t* at = nullptr; int32_t n = 1; };
Groups groups_of(PyObject* o, const at::Tensor& like) {
    if (o == Py_None) return {};
    const at::Tensor& t = tensor("offsets", o);
    if (t.scalar_type() != at::kInt || t.dim() != 1 || !t.is_contiguous() || t.device() != like.device() || t.numel() < 2)
        bad("offsets: a contiguous int32 vector of groups + 1 entries on the operands' device is expected");
    if (t.numel() - 1 > HOP_MAX_GROUPS) bad("offsets: ", t.numel() - 1, " groups, at most ", HOP_MAX_GROUPS);
    return {t.const_data_ptr<int32_t>(), (int32_t)(t.numel() - 1)};
}
std::optional<at::ScalarType> dtype_of(PyObject* o) {
    if (o == Py_None) return std::nullopt;
    if (!THPDtype_Check(o)) bad("out_dtype: not a torch dtype");
    return reinterpret_cast<THPDtype*>(o)->scalar_type;
}
int32_t narrow(const char* what, int64_t v) {
    if (v < 0 || v > 0x7fffffff) bad(what, ": ", v, " does not fit 32 bits");
    return (int32_t)v;
}
bool truth(const char* name, PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) { PyErr_Clear(); bad(name, ": neither true nor false"); }
    return v == 1;
}

// The device of a call made current, and its stream
struct On {
    c10::cuda::OptionalCUDAGuard guard;
    void* stream;
    explicit On(const at::Tensor& t) {
        if (t.get_device() != c10::cuda::current_device()) guard.set_device(t.device());
        stream = c10::cuda::getCurrentCUDAStream(t.get_device()).stream();
    }
};
void check(int rc, const char* msg) {
    if (rc != HOP_OK) refuse(rc, msg);
}
at::Tensor work(int64_t bytes, const at::Tensor& like) { return at::empty({bytes}, like.options().dtype(at::kByte)); }

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* wrap_or_none(const at::Tensor& t) {
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}

// ------------------------------------------------------------------------------------------------ grouped products
at::Tensor weights_of(const char* name, PyObject* o, int64_t groups, const at::Tensor& like, bool same_type) {
    at::Tensor w = tensor(name, o);
    if (w.dim() == 2) w = w.unsqueeze(0);
    if (w.dim() != 3 || w.size(0) != groups || w.device() != like.device() || (same_type && w.scalar_type() != like.scalar_type()))
        bad(name, ": shape ", w.sizes(), ", ", w.scalar_type(), " on ", w.device(), "; expected (", groups, ", n, k) of ", like.scalar_type(), " on ", like.device());
    if (w.stride(2) != 1 && w.size(2) > 1) bad(name, ": last dimension of stride ", w.stride(2));
    return w;
}
void run_linear(hop_linear_args& g, const at::Tensor& a, const at::Tensor& out, const Groups& gr) {
    char msg[512];
    msg[0] = 0;
    g.dtype = code_of(a.scalar_type());
    g.out_dtype = code_of(out.scalar_type());
    g.offsets = gr.at;
    g.groups = gr.n;
    g.rows = a.size(0);
    g.a = a.const_data_ptr();
    g.a_stride = a.stride(0);
    g.out = out.mutable_data_ptr();
    if (out.dim() == 3) { g.out_group_stride = out.stride(0); g.out_stride = out.stride(1); }
    else g.out_stride = out.stride(0);
    int64_t bytes = 0;
    check(g_api.linear_workspace(&g, &bytes, msg, sizeof(msg)), msg);
    On on(a);
    at::Tensor hold;
    if (bytes) {
        hold = work(bytes, a);
        g.workspace = hold.mutable_data_ptr();
        g.workspace_bytes = bytes;
    }
    check(g_api.linear(&g, on.stream, msg, sizeof(msg)), msg);
}

// (way, x or dy, w, offsets, out, out_dtype)
PyObject* linear_rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 6) bad("linear_rows: 6 arguments");
    const long way = PyLong_AsLong(args[0]);
    const bool fwd = way == HOP_LINEAR_FORWARD;
    const char* name = fwd ? "x" : "dy";
    const at::Tensor a = rows_of(name, tensor(name, args[1]));
    const Groups gr = groups_of(args[3], a);
    const at::Tensor w = weights_of("w", args[2], gr.n, a, true);
    const int64_t in = w.size(fwd ? 2 : 1), cols = w.size(fwd ? 1 : 2);
    if (in != a.size(1)) bad("w: ", in, fwd ? " input" : " output", " columns, ", name, " has ", a.size(1));
    const at::ScalarType type = dtype_of(args[5]).value_or(args[4] == Py_None ? a.scalar_type() : tensor("out", args[4]).scalar_type());
    const at::Tensor out = row_out("out", args[4], a, a.size(0), cols, type);
    if (args[4] != Py_None) { apart("out", out, a); apart("out", out, w); }
    hop_linear_args g = {};
    g.way = (int32_t)way;
    g.n = narrow("n", w.size(1));
    g.k = narrow("k", w.size(2));
    g.w = w.const_data_ptr();
    g.w_group_stride = w.stride(0);
    g.w_stride = w.stride(1);
    run_linear(g, a, out, gr);
    if (args[4] != Py_None) { written(tensor("out", args[4])); return Py_NewRef(args[4]); }
    return wrap(out);
    END_HANDLE_TH_ERRORS
}
// (dy, x, offsets, out, out_dtype, accumulate)
PyObject* linear_dw(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 6) bad("linear_dw: 6 arguments");
    const at::Tensor dy = rows_of("dy", tensor("dy", args[0]));
    const at::Tensor x = rows_of("x", tensor("x", args[1]), &dy, dy.size(0));
    const Groups gr = groups_of(args[2], dy);
    const bool accumulate = truth("accumulate", args[5]);
    const int64_t N = dy.size(1), K = x.size(1);
    at::Tensor out;
    if (args[3] == Py_None) {
        if (accumulate) bad("accumulate without out");
        out = at::empty({gr.n, N, K}, dy.options().dtype(dtype_of(args[4]).value_or(at::kFloat)));
    } else {
        writable("out", tensor("out", args[3]));
        out = weights_of("out", args[3], gr.n, dy, false);
        if (out.size(1) != N || out.size(2) != K || (N > 1 && out.stride(1) < K) || (gr.n > 1 && out.stride(0) < (N - 1) * out.stride(1) + K))
            bad("out: shape ", out.sizes(), " of strides ", out.strides(), ", expected (", gr.n, ", ", N, ", ", K, ") without overlap");
        apart("out", out, dy);
        apart("out", out, x);
    }
    hop_linear_args g = {};
    g.way = HOP_LINEAR_DW;
    g.accumulate = accumulate;
    g.n = narrow("n", N);
    g.k = narrow("k", K);
    g.b = x.const_data_ptr();
    g.b_stride = x.stride(0);
    run_linear(g, dy, out, gr);
    if (args[3] != Py_None) { written(tensor("out", args[3])); return Py_NewRef(args[3]); }
    return wrap(out);
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------------------------------------ the end of a block
uint64_t u64(const char* name, PyObject* o, uint64_t most) {
    const uint64_t v = PyLong_AsUnsignedLongLong(o);
    if (PyErr_Occurred()) { PyErr_Clear(); bad("seed: 64 bits, step and site: 32 bits, unsigned (", name, ")"); }
    if (v > most) bad("seed: 64 bits, step and site: 32 bits, unsigned (", name, ")");
    return v;
}
double number(const char* name, PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) { PyErr_Clear(); bad(name, ": not a number"); }
    return v;
}
const char* const kVectors[5] = {"w_post", "c_post", "gate", "w_pre", "c_pre"};
struct NormCall {
    hop_norm_args a = {};
    at::Tensor first, b, token_gate, vec[5];
};
// args: b, token_gate, the five vectors, offsets, kind, post, pre, eps, scale, skip, p, seed, step, site
constexpr int kNormArgs = 18;
void norm_args(NormCall& c, PyObject* const* v) {
    const at::Tensor& first = c.first;
    hop_norm_args& a = c.a;
    a.dtype = code_of(first.scalar_type());
    if (a.dtype < 0) refuse(HOP_E_UNSUPPORTED, "rows of ", first.scalar_type());
    const char* kind = PyUnicode_Check(v[8]) ? PyUnicode_AsUTF8(v[8]) : "";
    if (!std::strcmp(kind, "rms")) a.kind = HOP_NORM_RMS;
    else if (!std::strcmp(kind, "layer")) a.kind = HOP_NORM_LAYER;
    else bad("kind: '", kind, "' (rms or layer)");
    const int64_t rows = first.size(0), cols = first.size(1);
    const Groups gr = groups_of(v[7], first);
    a.rows = rows;
    a.cols = narrow("columns", cols);
    a.groups = gr.n;
    a.offsets = gr.at;
    a.post_norm = v[9] != Py_None ? truth("post", v[9]) : v[2] != Py_None || v[3] != Py_None;
    a.pre_norm = v[10] != Py_None ? truth("pre", v[10]) : v[5] != Py_None || v[6] != Py_None;
    a.eps = (float)number("eps", v[11]);
    a.scale = (float)number("scale", v[12]);
    a.skip = (float)number("skip", v[13]);
    a.p = number("p", v[14]);
    a.seed = u64("seed", v[15], ~0ull);
    a.step = (uint32_t)u64("step", v[16], 0xffffffffull);
    a.site = (uint32_t)u64("site", v[17], 0xffffffffull);
    if (v[0] != Py_None) { c.b = rows_of("b", tensor("b", v[0]), &first, rows, cols); a.b = c.b.const_data_ptr(); a.b_stride = c.b.stride(0); }
    if (v[1] != Py_None) {
        c.token_gate = rows_of("token_gate", tensor("token_gate", v[1]), &first, rows, cols);
        a.token_gate = c.token_gate.const_data_ptr();
        a.token_gate_stride = c.token_gate.stride(0);
    }
    const float** ptr[5] = {&a.w_post, &a.c_post, &a.gate, &a.w_pre, &a.c_pre};
    int64_t* stride[5] = {&a.w_post_stride, &a.c_post_stride, &a.gate_stride, &a.w_pre_stride, &a.c_pre_stride};
    for (int i = 0; i < 5; ++i) {
        if (v[2 + i] == Py_None) continue;
        at::Tensor t = tensor(kVectors[i], v[2 + i]);
        if (t.dim() == 1 && gr.n == 1) t = t.unsqueeze(0);
        if (t.scalar_type() != at::kFloat || t.device() != first.device() || t.dim() != 2 || t.size(0) != gr.n || t.size(1) != cols || (t.stride(1) != 1 && cols > 1))
            bad(kVectors[i], ": float32 (", gr.n, ", ", cols, ") with unit stride along the columns expected on ", first.device());
        *ptr[i] = t.const_data_ptr<float>();
        *stride[i] = t.stride(0);
        c.vec[i] = t;
    }
}

// (x, norm arguments...)
PyObject* norm_forward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 1 + kNormArgs) bad("norm_forward: ", 1 + kNormArgs, " arguments");
    char msg[512];
    NormCall c;
    c.first = rows_of("x", tensor("x", args[0]));
    norm_args(c, args + 1);
    c.a.x = c.first.const_data_ptr();
    c.a.x_stride = c.first.stride(0);
    const at::Tensor& x = THPVariable_Unpack(args[0]);
    Fresh r, h;
    if (c.b.defined()) {
        r = fresh_like(x, c.first);
        c.a.r = r.rows.mutable_data_ptr();
        c.a.r_stride = r.rows.stride(0);
    }
    if (c.a.pre_norm) {
        h = fresh_like(x, c.first);
        c.a.h = h.rows.mutable_data_ptr();
        c.a.h_stride = h.rows.stride(0);
    }
    On on(c.first);
    check(g_api.norm_forward(&c.a, on.stream, msg, sizeof(msg)), msg);
    PyObject* first = c.b.defined() ? wrap(r.whole) : Py_NewRef(args[0]);
    PyObject* second = wrap_or_none(h.whole);
    PyObject* both = first && second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_XDECREF(first);
    Py_XDECREF(second);
    return both;
    END_HANDLE_TH_ERRORS
}
// (dr, dh, r, norm arguments..., out or None: a dict of destinations by name)
PyObject* norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 4 + kNormArgs) bad("norm_backward: ", 4 + kNormArgs, " arguments");
    char msg[512];
    msg[0] = 0;
    NormCall c;
    c.first = rows_of("r", tensor("r", args[2]));
    norm_args(c, args + 3);
    hop_norm_args& a = c.a;
    const int64_t rows = c.first.size(0), cols = c.first.size(1);
    a.r = const_cast<void*>(c.first.const_data_ptr());
    a.r_stride = c.first.stride(0);
    at::Tensor dr, dh;
    if (args[0] != Py_None) { dr = rows_of("dr", tensor("dr", args[0]), &c.first, rows, cols); a.dr = dr.const_data_ptr(); a.dr_stride = dr.stride(0); }
    if (args[1] != Py_None) { dh = rows_of("dh", tensor("dh", args[1]), &c.first, rows, cols); a.dh = dh.const_data_ptr(); a.dh_stride = dh.stride(0); }
    bool given[8] = {};
    at::Tensor got[8];              // dx, db, dw_post, dc_post, dgate, dw_pre, dc_pre, dtoken_gate
    PyObject* dest = args[3 + kNormArgs];
    if (dest != Py_None && PyDict_Check(dest)) {
        PyObject *key, *value;
        for (Py_ssize_t at = 0; PyDict_Next(dest, &at, &key, &value);) {
            const char* name = PyUnicode_Check(key) ? PyUnicode_AsUTF8(key) : "";
            int i = 0;
            while (i < 5 && !(name[0] == 'd' && !std::strcmp(name + 1, kVectors[i]))) ++i;
            if (i == 5 || !c.vec[i].defined()) bad("out: ", name, " is the gradient of nothing that was given");
            const at::Tensor& t = tensor(name, value);
            writable(name, t);
            if (t.dim() != 2 || t.size(0) != a.groups || t.size(1) != cols || t.scalar_type() != at::kFloat || t.device() != c.first.device() ||
                (cols > 1 && t.stride(1) != 1) || (a.groups > 1 && t.stride(0) < cols))
                bad("out: ", name, " is not a float32 (", a.groups, ", ", cols, ") without overlap");
            for (const at::Tensor& v : c.vec)
                if (v.defined()) apart(name, t, v);
            for (int k = 2; k < 7; ++k)
                if (given[k]) apart(name, t, got[k]);
            got[2 + i] = t;
            given[2 + i] = true;
        }
    } else if (dest != Py_None) {
        bad("out: not a dict");
    }
    auto row_gradient = [&](int i, PyObject* of, void*& p, int64_t& stride) {       // in the shape of what it is the gradient of
        const Fresh t = fresh_like(THPVariable_Unpack(of), c.first);
        got[i] = t.whole;
        p = t.rows.mutable_data_ptr();
        stride = t.rows.stride(0);
    };
    row_gradient(0, args[2], a.dx, a.dx_stride);
    if (c.b.defined()) row_gradient(1, args[3], a.db, a.db_stride);
    if (c.token_gate.defined()) row_gradient(7, args[4], a.dtoken_gate, a.dtoken_gate_stride);
    float** ptr[5] = {&a.dw_post, &a.dc_post, &a.dgate, &a.dw_pre, &a.dc_pre};
    int64_t* stride[5] = {&a.dw_post_stride, &a.dc_post_stride, &a.dgate_stride, &a.dw_pre_stride, &a.dc_pre_stride};
    for (int i = 0; i < 5; ++i) {
        if (!c.vec[i].defined()) continue;
        if (!got[2 + i].defined()) got[2 + i] = at::empty({a.groups, cols}, c.first.options().dtype(at::kFloat));
        *ptr[i] = got[2 + i].mutable_data_ptr<float>();
        *stride[i] = got[2 + i].stride(0);
    }
    int64_t bytes = 0;
    check(g_api.norm_workspace(&a, &bytes, msg, sizeof(msg)), msg);
    On on(c.first);
    at::Tensor hold;
    if (bytes) {
        hold = work(bytes, c.first);
        a.workspace = hold.mutable_data_ptr();
        a.workspace_bytes = bytes;
    }
    check(g_api.norm_backward(&a, on.stream, msg, sizeof(msg)), msg);
    for (int i = 2; i < 7; ++i)
        if (given[i]) written(got[i]);
    PyObject* out = PyTuple_New(8);
    for (int i = 0; out && i < 8; ++i) PyTuple_SET_ITEM(out, i, wrap_or_none(got[i]));
    return out;
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------------------------------------ dropout
// (x, p, seed, step, site, out)
PyObject* dropout(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 6) bad("dropout: 6 arguments");
    char msg[512];
    const at::Tensor& x = tensor("x", args[0]);
    const at::Tensor v = rows_of("x", x);
    const int dtype = code_of(v.scalar_type());
    if (dtype < 0) refuse(HOP_E_UNSUPPORTED, "rows of ", v.scalar_type());
    const double p = number("p", args[1]);
    const uint64_t seed = u64("seed", args[2], ~0ull), step = u64("step", args[3], 0xffffffffull), site = u64("site", args[4], 0xffffffffull);
    const at::Tensor res = args[5] == Py_None ? at::empty(x.sizes(), x.options()) : tensor("out", args[5]);
    if (args[5] != Py_None) writable("out", res);
    at::Tensor y = rows_of("out", res, &v, v.size(0), v.size(1));
    if (v.size(0) > 1 && y.stride(0) < v.size(1)) bad("out: rows of stride ", y.stride(0), " overlap");
    // (in place: each element is read before it is written, by the same thread or warp)
    if (args[5] != Py_None && !(y.const_data_ptr() == v.const_data_ptr() && (v.size(0) <= 1 || y.stride(0) == v.stride(0)))) apart("out", y, v);
    On on(v);
    check(g_api.dropout(v.const_data_ptr(), v.stride(0), y.mutable_data_ptr(), y.stride(0), v.size(0), v.size(1), dtype, p, seed, (uint32_t)step, (uint32_t)site,
                        on.stream, msg, sizeof(msg)), msg);
    if (args[5] != Py_None) { written(res); return Py_NewRef(args[5]); }
    return wrap(res);
    END_HANDLE_TH_ERRORS
}

// (HopError, addresses of the six entries)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "bind: 7 arguments"); return nullptr; }
    uintptr_t at[6];
    for (int i = 0; i < 6; ++i) {
        at[i] = (uintptr_t)PyLong_AsUnsignedLongLong(args[1 + i]);
        if (PyErr_Occurred()) return nullptr;
    }
    g_api = {reinterpret_cast<decltype(&hop_linear_workspace)>(at[0]), reinterpret_cast<decltype(&hop_linear)>(at[1]),
             reinterpret_cast<decltype(&hop_norm_workspace)>(at[2]), reinterpret_cast<decltype(&hop_norm_forward)>(at[3]),
             reinterpret_cast<decltype(&hop_norm_backward)>(at[4]), reinterpret_cast<decltype(&hop_dropout)>(at[5])};
    Py_XDECREF(g_error);
    g_error = Py_NewRef(args[0]);
    Py_RETURN_NONE;
}

#define HOP_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {HOP_METHOD(bind), HOP_METHOD(linear_rows), HOP_METHOD(linear_dw), HOP_METHOD(norm_forward), HOP_METHOD(norm_backward),
                          HOP_METHOD(dropout), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_hop_nn", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__hop_nn() { return PyModule_Create(&kModule); }
