// The block operators' Python entry points: checks of tensors, outputs and workspaces, and the call into the C ABI.
// Native because a small call is bound by the host: marshalled in Python, a feed-forward call took 31 us of the host's time
// and a checkpoint call 13 us, of which 11 and 4.6 us were the library's.  (paper_2504_18454_b200/block.py documents them.)
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <dlfcn.h>

#include <optional>
#include <string>

#include "../../include/palsgd_block.h"

namespace {

// The library that the package has loaded (bind), and the package's exception.
struct Library {
    decltype(&palsgd_act8_pack) act8_pack;
    decltype(&palsgd_act8_unpack) act8_unpack;
    decltype(&palsgd_ffn_forward) ffn_forward;
    decltype(&palsgd_ffn_backward) ffn_backward;
    decltype(&palsgd_qk_norm_rope_forward) qk_forward;
    decltype(&palsgd_qk_norm_rope_backward) qk_backward;
    decltype(&palsgd_linear_forward) linear_forward;
    decltype(&palsgd_linear_backward) linear_backward;
    decltype(&palsgd_layer_norm_forward) norm_forward;
    decltype(&palsgd_layer_norm_backward) norm_backward;
    decltype(&palsgd_cross_entropy_forward) loss_forward;
    decltype(&palsgd_cross_entropy_backward) loss_backward;
    decltype(&palsgd_last_cuda_error) last_cuda_error;
} g_lib;
PyObject* g_error = nullptr;

struct Refusal { int status; const char* where; std::string why; };

[[noreturn]] void refuse(const char* where, std::string why) { throw Refusal{PALSGD_EINVAL, where, std::move(why)}; }

void check(int rc, const char* where)
{
    if (rc) throw Refusal{rc, where, rc == PALSGD_ECUDA ? g_lib.last_cuda_error(nullptr) : ""};
}

template <typename F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t expected, F&& f)
{
    HANDLE_TH_ERRORS
    if (given != expected || !g_error) { PyErr_SetString(PyExc_TypeError, "called by paper_2504_18454_b200/block.py only"); return nullptr; }
    try {
        return f();
    } catch (const Refusal& r) {
        PyObject* e = PyObject_CallFunction(g_error, "iss", r.status, r.where, r.why.c_str());
        if (e) { PyErr_SetObject(g_error, e); Py_DECREF(e); }
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

const at::Tensor& tensor(PyObject* o, const char* where, const char* name)
{
    if (!THPVariable_Check(o)) refuse(where, std::string(name) + " must be a tensor");
    return THPVariable_Unpack(o);
}
std::optional<at::Tensor> maybe(PyObject* o, const char* where, const char* name)
{
    if (o == Py_None) return std::nullopt;
    return tensor(o, where, name);
}

std::string text(at::IntArrayRef s)
{
    std::string t = "(";
    for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
    return t + ")";
}

void fit(const at::Tensor& t, const char* where, const char* name, at::IntArrayRef shape, at::ScalarType type, at::Device device)
{
    if (t.sizes() != shape) refuse(where, std::string(name) + " must have shape " + text(shape) + ", not " + text(t.sizes()));
    if (t.scalar_type() != type) refuse(where, std::string(name) + " must be " + at::toString(type) + ", not " + at::toString(t.scalar_type()));
    if (t.device() != device) refuse(where, std::string(name) + " must be on " + device.str() + ", not " + t.device().str());
    if (shape.back() > 1 && t.stride(-1) != 1 && t.numel()) refuse(where, "the last axis of " + std::string(name) + " must be contiguous");
}

at::Device on_cuda(const at::Tensor& t, const char* where, const char* name, int64_t dims)
{
    if (!t.is_cuda()) refuse(where, std::string(name) + " must be a CUDA tensor");
    if (t.dim() != dims) refuse(where, std::string(name) + " must have " + std::to_string(dims) + " axes, not " + std::to_string(t.dim()));
    return t.device();
}

int precision(at::ScalarType t, const char* where, const char* name)
{
    if (t == at::kBFloat16) return PALSGD_PREC_BF16_MASTER;
    if (t == at::kFloat) return PALSGD_PREC_FP32;
    refuse(where, std::string(name) + " must be float32 or bfloat16, not " + at::toString(t));
}

palsgd_mat mat(const at::Tensor& t)                      // (K, rows, cols), (K, cols) of one row, or (rows, cols) of one worker
{
    return t.dim() == 3 ? palsgd_mat{t.data_ptr(), t.stride(0), t.stride(1)} : palsgd_mat{t.data_ptr(), t.stride(0), 0};
}
palsgd_heads heads(const at::Tensor& t) { return palsgd_heads{t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)}; }

int64_t groups(int64_t cols) { return (cols + PALSGD_ACT8_GROUP - 1) / PALSGD_ACT8_GROUP; }

// The device and the stream of a call (None: torch's current one); allocations meanwhile belong to them.
struct On {
    c10::cuda::CUDAGuard device;
    std::optional<c10::cuda::CUDAStreamGuard> other;
    void* raw;
    On(at::Device d, PyObject* stream) : device(d)
    {
        const c10::cuda::CUDAStream now = c10::cuda::getCurrentCUDAStream(d.index());
        raw = now.stream();
        if (stream == Py_None) return;
        void* want = PyLong_AsVoidPtr(stream);
        if (!want && PyErr_Occurred()) throw python_error();
        if (want == raw) return;
        raw = want;
        // stream 0 is the legacy default stream, which torch knows as its default stream
        other.emplace(want ? c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(want), d.index()) : c10::cuda::getDefaultCUDAStream(d.index()));
    }
};

// (as at::empty, without its way through the dispatcher: 0.5 us less a tensor)
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, at::Device d) { return at::detail::empty_cuda(shape, type, d, std::nullopt); }

// The library wrote to these tensors: autograd is to see that, as of an in-place operation, where it has saved one of them.
template <typename... T>
void written(const T&... t)
{
    auto note = [](const at::Tensor& x) { if (!x.is_inference()) x.unsafeGetTensorImpl()->bump_version(); };
    (note(t), ...);
}

// (beyond 32 bits, where the C call's arguments end: a value that none of them accepts)
int64_t integer(PyObject* o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v == (int32_t)v ? v : INT32_MIN;
}

PyObject* wrap(const std::optional<at::Tensor>& t)
{
    if (t) return THPVariable_Wrap(*t);
    Py_RETURN_NONE;
}
template <typename... T>
PyObject* pack(const T&... t)
{
    PyObject* r = PyTuple_New(sizeof...(T));
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(r, i++, wrap(t)), ...);
    return r;
}

struct NoGil {
    PyThreadState* s = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(s); }
};

// call(workspace, its bytes): for the size, then with the memory (the caller's, or fresh)
template <typename F>
void with_workspace(F&& call, PyObject* given, at::Device d, const char* where)
{
    size_t n = 0;
    check(call(nullptr, &n), where);
    at::Tensor ws;
    if (given != Py_None) {
        ws = tensor(given, where, "workspace");
        if (ws.scalar_type() != at::kByte || ws.device() != d || !ws.is_contiguous()) refuse(where, "workspace must be a contiguous uint8 tensor on " + d.str());
        // (an empty tensor's address is NULL, which would ask for the size once more and do nothing)
        if ((size_t)ws.numel() < n) refuse(where, "workspace must have " + std::to_string(n) + " bytes, not " + std::to_string(ws.numel()));
    } else {
        ws = fresh({(int64_t)n}, at::kByte, d);
    }
    n = (size_t)ws.numel();
    int rc;
    {
        NoGil release;
        rc = call(ws.data_ptr(), &n);
    }
    check(rc, where);
}

// ---------------------------------------------------------------------------------------------- 8-bit checkpoints

// (x, q or None, exponent or None, stream) -> (q, exponent)
PyObject* act8_pack(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 4, [&] {
        const char* where = "palsgd_act8_pack";
        const at::Tensor& x = tensor(a[0], where, "x");
        const at::Device d = on_cuda(x, where, "x", x.dim() == 2 ? 2 : 3);
        const int prec = precision(x.scalar_type(), where, "x");
        fit(x, where, "x", x.sizes(), x.scalar_type(), d);
        c10::SmallVector<int64_t, 3> gs(x.sizes().begin(), x.sizes().end());
        gs.back() = groups(gs.back());
        const On on(d, a[3]);
        const at::Tensor q = a[1] == Py_None ? fresh(x.sizes(), at::kChar, d) : tensor(a[1], where, "out.q");
        const at::Tensor e = a[2] == Py_None ? fresh(gs, at::kByte, d) : tensor(a[2], where, "out.exponent");
        fit(q, where, "out.q", x.sizes(), at::kChar, d);
        fit(e, where, "out.exponent", gs, at::kByte, d);
        const bool one = x.dim() == 2;
        auto m = [&](const at::Tensor& t) { return one ? palsgd_mat{t.data_ptr(), 0, t.stride(0)} : mat(t); };
        const palsgd_mat mx = m(x), mq = m(q), me = m(e);
        check(g_lib.act8_pack(prec, one ? 1u : (uint32_t)std::min<int64_t>(x.size(0), 65), x.size(-2), x.size(-1), &mx, &mq, &me, on.raw), where);
        written(q, e);
        return pack(std::optional<at::Tensor>(q), std::optional<at::Tensor>(e));
    });
}

// (q, exponent, dtype, out or None, stream) -> x
PyObject* act8_unpack(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 5, [&] {
        const char* where = "palsgd_act8_unpack";
        const at::Tensor &q = tensor(a[0], where, "q"), &e = tensor(a[1], where, "exponent");
        const at::Device d = on_cuda(q, where, "q", q.dim() == 2 ? 2 : 3);
        if (!THPDtype_Check(a[2])) refuse(where, "dtype must be a torch dtype");
        const at::ScalarType type = reinterpret_cast<THPDtype*>(a[2])->scalar_type;
        const int prec = precision(type, where, "dtype");
        c10::SmallVector<int64_t, 3> gs(q.sizes().begin(), q.sizes().end());
        gs.back() = groups(gs.back());
        fit(q, where, "q", q.sizes(), at::kChar, d);
        fit(e, where, "exponent", gs, at::kByte, d);
        const On on(d, a[4]);
        const at::Tensor x = a[3] == Py_None ? fresh(q.sizes(), type, d) : tensor(a[3], where, "out");
        fit(x, where, "out", q.sizes(), type, d);
        const bool one = q.dim() == 2;
        auto m = [&](const at::Tensor& t) { return one ? palsgd_mat{t.data_ptr(), 0, t.stride(0)} : mat(t); };
        const palsgd_mat mx = m(x), mq = m(q), me = m(e);
        check(g_lib.act8_unpack(prec, one ? 1u : (uint32_t)std::min<int64_t>(q.size(0), 65), q.size(-2), q.size(-1), &mq, &me, &mx, on.raw), where);
        written(x);
        return wrap(x);
    });
}

// ---------------------------------------------------------------------------------------------- gated feed-forward

struct Ffn {
    int64_t K, M, D, F;
    at::ScalarType type;
    at::Device d;
    palsgd_ffn_shape shape;
    palsgd_mat w_gate, w_up, w_down;
};

// x or dy, and the weights
Ffn ffn(const char* where, const at::Tensor& x, const char* name, PyObject* wg, PyObject* wu, PyObject* wd, int64_t act, int64_t save)
{
    const at::Device d = on_cuda(x, where, name, 3);
    Ffn f{x.size(0), x.size(1), x.size(2), 0, x.scalar_type(), d, {}, {}, {}, {}};
    const int prec = precision(f.type, where, name);
    fit(x, where, name, x.sizes(), f.type, d);
    const at::Tensor &g = tensor(wg, where, "w_gate"), &u = tensor(wu, where, "w_up"), &w = tensor(wd, where, "w_down");
    f.F = g.dim() == 3 ? g.size(1) : 0;
    fit(g, where, "w_gate", {f.K, f.F, f.D}, f.type, d);
    fit(u, where, "w_up", {f.K, f.F, f.D}, f.type, d);
    fit(w, where, "w_down", {f.K, f.D, f.F}, f.type, d);
    f.w_gate = mat(g); f.w_up = mat(u); f.w_down = mat(w);
    f.shape = palsgd_ffn_shape{(uint32_t)std::min<int64_t>(f.K, 65), prec, (int32_t)act, (int32_t)save, (uint64_t)f.M, (uint64_t)f.D, (uint64_t)f.F};
    return f;
}

// The 8-bit or plain saved matrices: tensors given (or fresh where `make`), checked.
struct SavedMats {
    std::optional<at::Tensor> t[4];                      // gate, up, gate_e, up_e
    palsgd_mat m[4];
    const palsgd_mat* at(int i) const { return t[i] ? &m[i] : nullptr; }
};
SavedMats saved(const char* where, const Ffn& f, PyObject* const* given, bool make)
{
    static const char* names[4] = {"gate", "up", "gate.exponent", "up.exponent"};
    SavedMats s;
    const bool eight = f.shape.save == PALSGD_SAVE_8BIT;
    const int64_t full[3] = {f.K, f.M, f.F}, per[3] = {f.K, f.M, groups(f.F)};
    for (int i = 0; i < (f.shape.save == PALSGD_SAVE_NONE ? 0 : eight ? 4 : 2); ++i) {
        const at::IntArrayRef shape = i < 2 ? full : per;
        const at::ScalarType type = i >= 2 ? at::kByte : eight ? at::kChar : f.type;
        s.t[i] = given[i] == Py_None && make ? fresh(shape, type, f.d) : tensor(given[i], where, names[i]);
        fit(*s.t[i], where, names[i], shape, type, f.d);
        s.m[i] = mat(*s.t[i]);
    }
    return s;
}

// (x, w_gate, w_up, w_down, activation, save, out, gate, up, gate_e, up_e, workspace, stream) -> (y, gate, up, gate_e, up_e)
PyObject* ffn_forward(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 13, [&] {
        const char* where = "palsgd_ffn_forward";
        const at::Tensor& x = tensor(a[0], where, "x");
        const Ffn f = ffn(where, x, "x", a[1], a[2], a[3], integer(a[4]), integer(a[5]));
        const On on(f.d, a[12]);
        const at::Tensor y = a[6] == Py_None ? fresh(x.sizes(), f.type, f.d) : tensor(a[6], where, "out");
        fit(y, where, "out", x.sizes(), f.type, f.d);
        const SavedMats s = saved(where, f, a + 7, true);
        const palsgd_mat mx = mat(x), my = mat(y);
        with_workspace([&](void* ws, size_t* n) {
            return g_lib.ffn_forward(&f.shape, &mx, &f.w_gate, &f.w_up, &f.w_down, &my, s.at(0), s.at(1), s.at(2), s.at(3), ws, n, on.raw);
        }, a[11], f.d, where);
        written(y);
        for (const auto& t : s.t) if (t) written(*t);
        return pack(std::optional<at::Tensor>(y), s.t[0], s.t[1], s.t[2], s.t[3]);
    });
}

// (dy, x, x_e, w_gate, w_up, w_down, activation, save, gate, up, gate_e, up_e, need_dx, dx, dw_gate, dw_up, dw_down, workspace, stream)
PyObject* ffn_backward(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 19, [&] {
        const char* where = "palsgd_ffn_backward";
        const at::Tensor& dy = tensor(a[0], where, "dy");
        const Ffn f = ffn(where, dy, "dy", a[3], a[4], a[5], integer(a[6]), integer(a[7]));
        const at::Tensor& x = tensor(a[1], where, "x");
        const std::optional<at::Tensor> xe = maybe(a[2], where, "x.exponent");
        fit(x, where, xe ? "x.q" : "x", dy.sizes(), xe ? at::kChar : f.type, f.d);
        if (xe) fit(*xe, where, "x.exponent", {f.K, f.M, groups(f.D)}, at::kByte, f.d);
        const SavedMats s = saved(where, f, a + 8, false);
        const On on(f.d, a[18]);
        static const char* names[4] = {"dx", "dw_gate", "dw_up", "dw_down"};
        const int64_t want[4][3] = {{f.K, f.M, f.D}, {f.K, f.F, f.D}, {f.K, f.F, f.D}, {f.K, f.D, f.F}};
        std::optional<at::Tensor> out[4];
        palsgd_mat m[4];
        for (int i = integer(a[12]) ? 0 : 1; i < 4; ++i) {
            out[i] = a[13 + i] == Py_None ? fresh(want[i], f.type, f.d) : tensor(a[13 + i], where, names[i]);
            fit(*out[i], where, names[i], want[i], f.type, f.d);
            m[i] = mat(*out[i]);
        }
        const palsgd_mat mdy = mat(dy), mx = mat(x), me = xe ? mat(*xe) : palsgd_mat{};
        with_workspace([&](void* ws, size_t* n) {
            return g_lib.ffn_backward(&f.shape, &mdy, &mx, xe ? &me : nullptr, &f.w_gate, &f.w_up, &f.w_down, s.at(0), s.at(1), s.at(2), s.at(3),
                                      out[0] ? &m[0] : nullptr, &m[1], &m[2], &m[3], ws, n, on.raw);
        }, a[17], f.d, where);
        for (const auto& t : out) if (t) written(*t);
        return pack(out[0], out[1], out[2], out[3]);
    });
}

// ---------------------------------------------------------------------------------------------- q/k norm + rotation

struct Qk {
    at::Tensor q, k, wq, wk, cos, sin, pos;
    at::ScalarType type;
    at::Device d;
    palsgd_qk_shape shape;
    palsgd_heads hq, hk;
    palsgd_mat mq, mk;
    const float *c, *s;
    const int32_t* p;
};

// q, k, w_q, w_k, cos, sin, positions, eps, interleaved
Qk qk(const char* where, PyObject* const* a)
{
    const at::Tensor &q = tensor(a[0], where, "q"), &k = tensor(a[1], where, "k"), &wq = tensor(a[2], where, "w_q"), &wk = tensor(a[3], where, "w_k");
    const at::Tensor &cos = tensor(a[4], where, "cos"), &sin = tensor(a[5], where, "sin"), &pos = tensor(a[6], where, "positions");
    const at::Device d = on_cuda(q, where, "q", 4);
    const at::ScalarType type = q.scalar_type();
    const int prec = precision(type, where, "q");
    const int64_t K = q.size(0), M = q.size(1), HQ = q.size(2), DH = q.size(3), HK = k.dim() == 4 ? k.size(2) : -1;
    fit(q, where, "q", q.sizes(), type, d);
    fit(k, where, "k", {K, M, HK, DH}, type, d);
    fit(wq, where, "w_q", {K, DH}, type, d);
    fit(wk, where, "w_k", {K, DH}, type, d);
    if (cos.dim() != 2) refuse(where, "cos must be a (rows, rotary_dim / 2) tensor");
    fit(cos, where, "cos", cos.sizes(), at::kFloat, d);
    fit(sin, where, "sin", cos.sizes(), at::kFloat, d);
    if (!cos.is_contiguous() || !sin.is_contiguous()) refuse(where, "cos and sin must be contiguous");
    fit(pos, where, "positions", {K, M}, at::kInt, d);
    const double eps = PyFloat_AsDouble(a[7]);
    if (eps == -1.0 && PyErr_Occurred()) throw python_error();
    auto small = [](int64_t v) { return (uint32_t)std::min<int64_t>(v, 0x7FFFFFFF); };
    palsgd_qk_shape s{(uint32_t)std::min<int64_t>(K, 65), prec, (uint64_t)M, small(HQ), small(HK), small(DH), small(2 * cos.size(1)), integer(a[8]) ? 1 : 0, 0,
                      (uint64_t)cos.size(0), K > 1 ? pos.stride(0) : 0, eps};
    return Qk{q, k, wq, wk, cos, sin, pos, type, d, s, heads(q), heads(k), mat(wq), mat(wk), cos.data_ptr<float>(), sin.data_ptr<float>(), pos.data_ptr<int32_t>()};
}

// (..., q_out, k_out, stream) -> (q_out, k_out)
PyObject* qk_forward(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 12, [&] {
        const char* where = "palsgd_qk_norm_rope_forward";
        const Qk t = qk(where, a);
        const On on(t.d, a[11]);
        const at::Tensor oq = a[9] == Py_None ? fresh(t.q.sizes(), t.type, t.d) : tensor(a[9], where, "q_out");
        const at::Tensor ok = a[10] == Py_None ? fresh(t.k.sizes(), t.type, t.d) : tensor(a[10], where, "k_out");
        fit(oq, where, "q_out", t.q.sizes(), t.type, t.d);
        fit(ok, where, "k_out", t.k.sizes(), t.type, t.d);
        const palsgd_heads hoq = heads(oq), hok = heads(ok);
        check(g_lib.qk_forward(&t.shape, &t.hq, &t.hk, &t.mq, &t.mk, t.c, t.s, t.p, &hoq, &hok, on.raw), where);
        written(oq, ok);
        return pack(std::optional<at::Tensor>(oq), std::optional<at::Tensor>(ok));
    });
}

// (..., dq_out, dk_out, dq, dk, dw_q, dw_k, workspace, stream) -> (dq, dk, dw_q, dw_k)
PyObject* qk_backward(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 17, [&] {
        const char* where = "palsgd_qk_norm_rope_backward";
        const Qk t = qk(where, a);
        const at::Tensor &gq = tensor(a[9], where, "dq_out"), &gk = tensor(a[10], where, "dk_out");
        fit(gq, where, "dq_out", t.q.sizes(), t.type, t.d);
        fit(gk, where, "dk_out", t.k.sizes(), t.type, t.d);
        const On on(t.d, a[16]);
        static const char* names[4] = {"dq", "dk", "dw_q", "dw_k"};
        const at::Tensor* like[4] = {&t.q, &t.k, &t.wq, &t.wk};
        std::optional<at::Tensor> out[4];
        for (int i = 0; i < 4; ++i) {
            out[i] = a[11 + i] == Py_None ? fresh(like[i]->sizes(), t.type, t.d) : tensor(a[11 + i], where, names[i]);
            fit(*out[i], where, names[i], like[i]->sizes(), t.type, t.d);
        }
        const palsgd_heads hgq = heads(gq), hgk = heads(gk), hdq = heads(*out[0]), hdk = heads(*out[1]);
        const palsgd_mat mdq = mat(*out[2]), mdk = mat(*out[3]);
        with_workspace([&](void* ws, size_t* n) {
            return g_lib.qk_backward(&t.shape, &hgq, &hgk, &t.hq, &t.hk, &t.mq, &t.mk, t.c, t.s, t.p, &hdq, &hdk, &mdq, &mdk, ws, n, on.raw);
        }, a[15], t.d, where);
        for (const auto& t : out) if (t) written(*t);
        return pack(out[0], out[1], out[2], out[3]);
    });
}

// ---------------------------------------------------------------------------------------------- linear

uint32_t workers(int64_t K) { return (uint32_t)std::min<int64_t>(K, 65); }       // (more than there may be are as good as 65)
const palsgd_mat* at(const std::optional<at::Tensor>& t, const palsgd_mat& m) { return t ? &m : nullptr; }
palsgd_mat mat(const std::optional<at::Tensor>& t) { return t ? mat(*t) : palsgd_mat{}; }

struct Linear {
    int64_t K, M, D, N;
    at::ScalarType type;
    at::Device d;
    palsgd_linear_shape shape;
    palsgd_mat w;
};

// x (its last axis: d_in) or dy (d_out), and the weights
Linear linear(const char* where, const at::Tensor& t, const char* name, bool back, PyObject* weight, int64_t act, int64_t save)
{
    const at::Device d = on_cuda(t, where, name, 3);
    const at::Tensor& w = tensor(weight, where, "w");
    Linear f{t.size(0), t.size(1), 0, 0, t.scalar_type(), d, {}, {}};
    const int prec = precision(f.type, where, name);
    fit(t, where, name, t.sizes(), f.type, d);
    f.D = back ? (w.dim() == 3 ? w.size(2) : 0) : t.size(2);
    f.N = back ? t.size(2) : (w.dim() == 3 ? w.size(1) : 0);
    fit(w, where, "w", {f.K, f.N, f.D}, f.type, d);
    f.w = mat(w);
    f.shape = palsgd_linear_shape{workers(f.K), prec, (int32_t)act, (int32_t)save, (uint64_t)f.M, (uint64_t)f.D, (uint64_t)f.N};
    return f;
}

// (x, w, bias, residual, activation, save, out, pre, pre_e, workspace, stream) -> (y, pre, pre_e)
PyObject* linear_forward(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 11, [&] {
        const char* where = "palsgd_linear_forward";
        const at::Tensor& x = tensor(a[0], where, "x");
        const Linear f = linear(where, x, "x", false, a[1], integer(a[4]), integer(a[5]));
        const int64_t ys[3] = {f.K, f.M, f.N}, es[3] = {f.K, f.M, groups(f.N)};
        const std::optional<at::Tensor> bias = maybe(a[2], where, "bias"), residual = maybe(a[3], where, "residual");
        if (bias) fit(*bias, where, "bias", {f.K, f.N}, f.type, f.d);
        if (residual) fit(*residual, where, "residual", ys, f.type, f.d);
        const On on(f.d, a[10]);
        const at::Tensor y = a[6] == Py_None ? fresh(ys, f.type, f.d) : tensor(a[6], where, "out");
        fit(y, where, "out", ys, f.type, f.d);
        std::optional<at::Tensor> pre, pre_e;
        const bool eight = f.shape.save == PALSGD_SAVE_8BIT;
        if (f.shape.save == PALSGD_SAVE_FULL || eight) {
            const at::ScalarType type = eight ? at::kChar : f.type;
            pre = a[7] == Py_None ? fresh(ys, type, f.d) : tensor(a[7], where, eight ? "saved.q" : "saved");
            fit(*pre, where, eight ? "saved.q" : "saved", ys, type, f.d);
        }
        if (eight) {
            pre_e = a[8] == Py_None ? fresh(es, at::kByte, f.d) : tensor(a[8], where, "saved.exponent");
            fit(*pre_e, where, "saved.exponent", es, at::kByte, f.d);
        }
        const palsgd_mat mx = mat(x), my = mat(y), mb = mat(bias), mr = mat(residual), mp = mat(pre), me = mat(pre_e);
        with_workspace([&](void* ws, size_t* n) {
            return g_lib.linear_forward(&f.shape, &mx, &f.w, at(bias, mb), at(residual, mr), &my, at(pre, mp), at(pre_e, me), ws, n, on.raw);
        }, a[9], f.d, where);
        written(y);
        if (pre) written(*pre);
        if (pre_e) written(*pre_e);
        return pack(std::optional<at::Tensor>(y), pre, pre_e);
    });
}

// (dy, x, x_e, w, pre, pre_e, activation, save, need_dx, need_db, dx, dw, db, workspace, stream) -> (dx, dw, db)
PyObject* linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 15, [&] {
        const char* where = "palsgd_linear_backward";
        const at::Tensor& dy = tensor(a[0], where, "dy");
        const Linear f = linear(where, dy, "dy", true, a[3], integer(a[6]), integer(a[7]));
        const at::Tensor& x = tensor(a[1], where, "x");
        const std::optional<at::Tensor> xe = maybe(a[2], where, "x.exponent"), pre = maybe(a[4], where, "saved"), pre_e = maybe(a[5], where, "saved.exponent");
        const int64_t xs[3] = {f.K, f.M, f.D}, ys[3] = {f.K, f.M, f.N};
        const bool eight = f.shape.save == PALSGD_SAVE_8BIT;
        fit(x, where, xe ? "x.q" : "x", xs, xe ? at::kChar : f.type, f.d);
        if (xe) fit(*xe, where, "x.exponent", {f.K, f.M, groups(f.D)}, at::kByte, f.d);
        if (pre) fit(*pre, where, eight ? "saved.q" : "saved", ys, eight ? at::kChar : f.type, f.d);
        if (pre_e) fit(*pre_e, where, "saved.exponent", {f.K, f.M, groups(f.N)}, at::kByte, f.d);
        const On on(f.d, a[14]);
        static const char* names[3] = {"dx", "dw", "db"};
        const int64_t ws3[3] = {f.K, f.N, f.D}, bs[2] = {f.K, f.N};
        const at::IntArrayRef want[3] = {xs, ws3, bs};
        const bool need[3] = {integer(a[8]) != 0, true, integer(a[9]) != 0};
        std::optional<at::Tensor> out[3];
        palsgd_mat m[3];
        for (int i = 0; i < 3; ++i) {
            if (!need[i]) continue;
            out[i] = a[10 + i] == Py_None ? fresh(want[i], f.type, f.d) : tensor(a[10 + i], where, names[i]);
            fit(*out[i], where, names[i], want[i], f.type, f.d);
            m[i] = mat(*out[i]);
        }
        const palsgd_mat mdy = mat(dy), mx = mat(x), me = mat(xe), mp = mat(pre), mpe = mat(pre_e);
        with_workspace([&](void* ws, size_t* n) {
            return g_lib.linear_backward(&f.shape, &mdy, &mx, at(xe, me), &f.w, at(pre, mp), at(pre_e, mpe), at(out[0], m[0]), &m[1], at(out[2], m[2]), ws, n, on.raw);
        }, a[13], f.d, where);
        for (const auto& t : out) if (t) written(*t);
        return pack(out[0], out[1], out[2]);
    });
}

// ---------------------------------------------------------------------------------------------- layer norm

struct Norm {
    int64_t K, M, D;
    at::ScalarType type;
    at::Device d;
    palsgd_norm_shape shape;
    palsgd_mat w;
};
Norm norm(const char* where, const at::Tensor& x, const char* name, PyObject* weight, double eps)
{
    const at::Device d = on_cuda(x, where, name, 3);
    Norm f{x.size(0), x.size(1), x.size(2), x.scalar_type(), d, {}, {}};
    const int prec = precision(f.type, where, name);
    fit(x, where, name, x.sizes(), f.type, d);
    const at::Tensor& w = tensor(weight, where, "w");
    fit(w, where, "w", {f.K, f.D}, f.type, d);
    f.w = mat(w);
    f.shape = palsgd_norm_shape{workers(f.K), prec, (uint64_t)f.M, (uint64_t)f.D, eps};
    return f;
}

// (x, w, b, residual, eps, need_stats, y, total, mean, rstd, stream) -> (y, total, mean, rstd)
PyObject* norm_forward(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 11, [&] {
        const char* where = "palsgd_layer_norm_forward";
        const double eps = PyFloat_AsDouble(a[4]);
        if (eps == -1.0 && PyErr_Occurred()) throw python_error();
        const at::Tensor& x = tensor(a[0], where, "x");
        const Norm f = norm(where, x, "x", a[1], eps);
        const at::Tensor& b = tensor(a[2], where, "b");
        fit(b, where, "b", {f.K, f.D}, f.type, f.d);
        const std::optional<at::Tensor> residual = maybe(a[3], where, "residual");
        if (residual) fit(*residual, where, "residual", x.sizes(), f.type, f.d);
        const On on(f.d, a[10]);
        const at::Tensor y = a[6] == Py_None ? fresh(x.sizes(), f.type, f.d) : tensor(a[6], where, "y");
        fit(y, where, "y", x.sizes(), f.type, f.d);
        std::optional<at::Tensor> total, mean, rstd;
        if (residual) {
            total = a[7] == Py_None ? fresh(x.sizes(), f.type, f.d) : tensor(a[7], where, "total");
            fit(*total, where, "total", x.sizes(), f.type, f.d);
        }
        const int64_t rows[2] = {f.K, f.M};
        if (integer(a[5])) {
            mean = a[8] == Py_None ? fresh(rows, at::kFloat, f.d) : tensor(a[8], where, "mean");
            rstd = a[9] == Py_None ? fresh(rows, at::kFloat, f.d) : tensor(a[9], where, "rstd");
            fit(*mean, where, "mean", rows, at::kFloat, f.d);
            fit(*rstd, where, "rstd", rows, at::kFloat, f.d);
        }
        const palsgd_mat mx = mat(x), mb = mat(b), my = mat(y), mr = mat(residual), mt = mat(total), mm = mat(mean), ms = mat(rstd);
        check(g_lib.norm_forward(&f.shape, &mx, at(residual, mr), &f.w, &mb, &my, at(total, mt), at(mean, mm), at(rstd, ms), on.raw), where);
        written(y);
        for (const auto* t : {&total, &mean, &rstd}) if (*t) written(**t);
        return pack(std::optional<at::Tensor>(y), total, mean, rstd);
    });
}

// (dy, x, w, mean, rstd, dtotal, dx, dw, db, workspace, stream) -> (dx, dw, db)
PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 11, [&] {
        const char* where = "palsgd_layer_norm_backward";
        const at::Tensor& dy = tensor(a[0], where, "dy");
        const Norm f = norm(where, dy, "dy", a[2], 0.0);
        const at::Tensor &x = tensor(a[1], where, "x"), &mean = tensor(a[3], where, "mean"), &rstd = tensor(a[4], where, "rstd");
        const int64_t rows[2] = {f.K, f.M}, cols[2] = {f.K, f.D};
        fit(x, where, "x", dy.sizes(), f.type, f.d);
        fit(mean, where, "mean", rows, at::kFloat, f.d);
        fit(rstd, where, "rstd", rows, at::kFloat, f.d);
        const std::optional<at::Tensor> past = maybe(a[5], where, "dtotal");
        if (past) fit(*past, where, "dtotal", dy.sizes(), f.type, f.d);
        const On on(f.d, a[10]);
        static const char* names[3] = {"dx", "dw", "db"};
        const at::IntArrayRef want[3] = {dy.sizes(), cols, cols};
        std::optional<at::Tensor> out[3];
        palsgd_mat m[3];
        for (int i = 0; i < 3; ++i) {
            out[i] = a[6 + i] == Py_None ? fresh(want[i], f.type, f.d) : tensor(a[6 + i], where, names[i]);
            fit(*out[i], where, names[i], want[i], f.type, f.d);
            m[i] = mat(*out[i]);
        }
        const palsgd_mat mdy = mat(dy), mx = mat(x), mm = mat(mean), ms = mat(rstd), mp = mat(past);
        with_workspace([&](void* ws, size_t* n) {
            return g_lib.norm_backward(&f.shape, &mdy, &mx, &f.w, &mm, &ms, at(past, mp), &m[0], &m[1], &m[2], ws, n, on.raw);
        }, a[9], f.d, where);
        for (const auto& t : out) written(*t);
        return pack(out[0], out[1], out[2]);
    });
}

// ---------------------------------------------------------------------------------------------- cross entropy

struct Loss {
    int64_t rows[2];
    at::Device d;
    palsgd_loss_shape shape;
    palsgd_mat logits;
    const int32_t* targets;
};
Loss loss(const char* where, const at::Tensor& z, PyObject* targets)
{
    const at::Device d = on_cuda(z, where, "logits", 3);
    const int prec = precision(z.scalar_type(), where, "logits");
    fit(z, where, "logits", z.sizes(), z.scalar_type(), d);
    const at::Tensor& t = tensor(targets, where, "targets");
    fit(t, where, "targets", {z.size(0), z.size(1)}, at::kInt, d);
    return Loss{{z.size(0), z.size(1)}, d, palsgd_loss_shape{workers(z.size(0)), prec, (uint64_t)z.size(1), (uint64_t)z.size(2), z.size(0) > 1 ? t.stride(0) : 0},
                mat(z), t.data_ptr<int32_t>()};
}

// (logits, targets, loss, lse, stream) -> (loss, lse)
PyObject* loss_forward(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 5, [&] {
        const char* where = "palsgd_cross_entropy_forward";
        const Loss f = loss(where, tensor(a[0], where, "logits"), a[1]);
        const On on(f.d, a[4]);
        const at::Tensor out = a[2] == Py_None ? fresh(f.rows, at::kFloat, f.d) : tensor(a[2], where, "loss");
        const at::Tensor lse = a[3] == Py_None ? fresh(f.rows, at::kFloat, f.d) : tensor(a[3], where, "lse");
        fit(out, where, "loss", f.rows, at::kFloat, f.d);
        fit(lse, where, "lse", f.rows, at::kFloat, f.d);
        const palsgd_mat mo = mat(out), ml = mat(lse);
        check(g_lib.loss_forward(&f.shape, &f.logits, f.targets, &mo, &ml, on.raw), where);
        written(out, lse);
        return pack(std::optional<at::Tensor>(out), std::optional<at::Tensor>(lse));
    });
}

// (dloss, logits, targets, lse, out, stream) -> dlogits
PyObject* loss_backward(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 6, [&] {
        const char* where = "palsgd_cross_entropy_backward";
        const at::Tensor &dloss = tensor(a[0], where, "dloss"), &z = tensor(a[1], where, "logits"), &lse = tensor(a[3], where, "lse");
        const Loss f = loss(where, z, a[2]);
        fit(dloss, where, "dloss", f.rows, at::kFloat, f.d);
        fit(lse, where, "lse", f.rows, at::kFloat, f.d);
        const On on(f.d, a[5]);
        const at::Tensor dz = a[4] == Py_None ? fresh(z.sizes(), z.scalar_type(), f.d) : tensor(a[4], where, "out");
        fit(dz, where, "out", z.sizes(), z.scalar_type(), f.d);
        const palsgd_mat md = mat(dloss), ml = mat(lse), mz = mat(dz);
        check(g_lib.loss_backward(&f.shape, &md, &f.logits, f.targets, &ml, &mz, on.raw), where);
        written(dz);
        return wrap(dz);
    });
}

// (handle of the loaded library, exception class)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 2) { PyErr_SetString(PyExc_TypeError, "bind(handle, error)"); return nullptr; }
    void* lib = PyLong_AsVoidPtr(a[0]);
    if (PyErr_Occurred()) return nullptr;
    const struct { const char* name; void** to; } all[] = {
        {"palsgd_act8_pack", (void**)&g_lib.act8_pack}, {"palsgd_act8_unpack", (void**)&g_lib.act8_unpack},
        {"palsgd_ffn_forward", (void**)&g_lib.ffn_forward}, {"palsgd_ffn_backward", (void**)&g_lib.ffn_backward},
        {"palsgd_qk_norm_rope_forward", (void**)&g_lib.qk_forward}, {"palsgd_qk_norm_rope_backward", (void**)&g_lib.qk_backward},
        {"palsgd_linear_forward", (void**)&g_lib.linear_forward}, {"palsgd_linear_backward", (void**)&g_lib.linear_backward},
        {"palsgd_layer_norm_forward", (void**)&g_lib.norm_forward}, {"palsgd_layer_norm_backward", (void**)&g_lib.norm_backward},
        {"palsgd_cross_entropy_forward", (void**)&g_lib.loss_forward}, {"palsgd_cross_entropy_backward", (void**)&g_lib.loss_backward},
        {"palsgd_last_cuda_error", (void**)&g_lib.last_cuda_error}};
    for (const auto& f : all)
        if (!(*f.to = dlsym(lib, f.name))) { PyErr_Format(PyExc_ImportError, "the library has no %s", f.name); return nullptr; }
    Py_INCREF(a[1]);
    Py_XSETREF(g_error, a[1]);
    Py_RETURN_NONE;
}

#define ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(act8_pack), ENTRY(act8_unpack), ENTRY(ffn_forward), ENTRY(ffn_backward), ENTRY(qk_forward), ENTRY(qk_backward),
                         ENTRY(linear_forward), ENTRY(linear_backward), ENTRY(norm_forward), ENTRY(norm_backward), ENTRY(loss_forward), ENTRY(loss_backward), ENTRY(bind),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_block", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__block() { return PyModule_Create(&module); }
