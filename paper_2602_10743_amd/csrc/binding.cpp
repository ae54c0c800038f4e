// Native part of the Python binding: argument checks, output and workspace allocation and
// the C ABI call of the filter layer's entry points (include/kla.h), for
// paper_2602_10743_amd/__init__.py.
//
// A training step of a few sequences is bound by the host: through ctypes and torch.empty the
// forward took 21 us and the backward 33 us of it, more than their kernels.  Functions return the
// output tensors; where the library refuses the call, those of the layer return its status code and
// those of the operators around it raise KLAError.  Past the checks they give
// up the interpreter lock, as ctypes does: allocations and a full launch queue can block, and under
// KLA_CHECK=1 the library waits for the stream.
#include <array>
#include <initializer_list>
#include <stdexcept>
#include <string>
#include <vector>

#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/extension.h>

#include "kla.h"

namespace py = pybind11;
using at::Tensor;
using Opt = c10::optional<Tensor>;

namespace {

const char* kNames[6] = {"q", "k", "v", "a", "p", "r"};

[[noreturn]] void value_error(const std::string& s) { throw py::value_error(s); }

std::string shape_str(at::IntArrayRef s) {
    std::string o = "(";
    for (size_t i = 0; i < s.size(); ++i) o += (i ? ", " : "") + std::to_string(s[i]);
    return o + (s.size() == 1 ? ",)" : ")");
}

int dtype_of(const Tensor& q) {
    if (q.scalar_type() == at::kFloat) return KLA_F32;
    if (q.scalar_type() == at::kBFloat16) return KLA_BF16;
    throw py::type_error("unsupported dtype " + std::string(py::str(py::cast(q).attr("dtype"))) +
                         "; use float32 or bfloat16");
}

void* ptr(const Tensor& t) { return t.data_ptr(); }
void* ptr(const Opt& t) { return t ? t->data_ptr() : nullptr; }
float* fptr(const Opt& t) { return static_cast<float*>(ptr(t)); }

hipStream_t stream_of(const Tensor& t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

// q [B, T, H, dk] and the other per-token tensors (a, p absent with OU gates)
kla_desc check_inputs(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor* a, const Tensor* p,
                      const Tensor& r) {
    if (!q.is_cuda()) value_error("KLA tensors must live on a GPU; the layer has no CPU path");
    const int dt = dtype_of(q);
    if (q.dim() != 4) value_error("q must be [B, T, H, dk]");
    const int64_t B = q.size(0), T = q.size(1), H = q.size(2), dk = q.size(3), dv = v.size(-1);
    const std::array<int64_t, 4> ks{B, T, H, dk}, vs{B, T, H, dv};
    const std::array<int64_t, 3> rs{B, T, H};
    const Tensor* t[6] = {&q, &k, &v, a, p, &r};
    for (int i : {1, 3, 4, 2, 5}) {
        if (!t[i]) continue;
        const at::IntArrayRef want = i == 2 ? at::IntArrayRef(vs) : i == 5 ? at::IntArrayRef(rs) : at::IntArrayRef(ks);
        if (t[i]->sizes() != want)
            value_error(std::string(kNames[i]) + " has shape " + shape_str(t[i]->sizes()) + ", expected " + shape_str(want));
        if (t[i]->scalar_type() != q.scalar_type() || t[i]->device() != q.device())
            value_error(std::string(kNames[i]) + " must share q's dtype and device");
    }
    for (int i = 0; i < 6; ++i)
        if (t[i] && !t[i]->is_contiguous()) value_error(std::string(kNames[i]) + " must be contiguous");
    return kla_desc{(int32_t)B, (int32_t)T, (int32_t)H, (int32_t)dk, (int32_t)dv, (kla_dtype)dt};
}

void check_f32(const Opt& t, at::IntArrayRef shape, const Tensor& q, const char* name) {
    if (!t) return;
    if (t->scalar_type() != at::kFloat || t->sizes() != shape || t->device() != q.device() || !t->is_contiguous())
        value_error(std::string(name) + " must be a contiguous float32 tensor of shape " + shape_str(shape) + " on " +
                    q.device().str());
}

void check_belief(const kla_desc& d, const Opt& lam, const Opt& eta, const Tensor& q, const char* ln, const char* en) {
    check_f32(lam, {d.B, d.H, d.dk}, q, ln);
    check_f32(eta, {d.B, d.H, d.dk, d.dv}, q, en);
}

void check_ou(const Opt& a, const Opt& p, const Opt& delta, int64_t H, int64_t dk, const Tensor& q) {
    check_f32(a, {H, dk}, q, "a");
    check_f32(p, {H, dk}, q, "p");
    check_f32(delta, {H, dk}, q, "delta");
}

// a per-token gate tensor, which has to be there (none with OU gates)
const Tensor* per_token(const Opt& t, bool ou, const char* name) {
    if (ou) return nullptr;
    if (!t) throw py::type_error(std::string(name) + " must be a tensor");
    return &*t;
}

Tensor bytes(size_t n, const Tensor& q) {
    return at::empty({(int64_t)(n > 1 ? n : 1)}, q.options().dtype(at::kByte));
}

py::object obj(const Opt& t) { return t ? py::cast(*t) : py::none(); }

// (y, yvar, lamT, etaT, saved) or a status.  ou: OU gates, a, p, delta [H, dk] fp32 (the library
// refuses the call when one is absent).
py::object forward(const Tensor& q, const Tensor& k, const Tensor& v, const Opt& a, const Opt& p, const Opt& delta,
                   const Tensor& r, const Opt& lam0, const Opt& eta0, const Opt& y_in, bool want_var, bool want_state,
                   bool save, bool ou) {
    const kla_desc d = check_inputs(q, k, v, per_token(a, ou, "a"), per_token(p, ou, "p"), r);
    if (ou) check_ou(a, p, delta, d.H, d.dk, q);
    check_belief(d, lam0, eta0, q, "lam0", "eta0");
    Tensor y;
    Opt yvar, lamT, etaT, saved;
    kla_status st;
    {
        py::gil_scoped_release unlocked;
        const auto f32 = q.options().dtype(at::kFloat);
        y = y_in ? *y_in : at::empty({d.B, d.T, d.H, d.dv}, q.options());
        if (want_var) yvar = at::empty({d.B, d.T, d.H}, f32);
        if (want_state) {
            lamT = at::empty({d.B, d.H, d.dk}, f32);
            etaT = at::empty({d.B, d.H, d.dk, d.dv}, f32);
        }
        const size_t ns = save ? kla_saved_bytes(&d) : 0, nw = kla_forward_workspace(&d);
        if (ns) saved = bytes(ns, q);
        const Tensor ws = bytes(nw, q);
        st = ou ? kla_forward_ou(&d, ptr(q), ptr(k), ptr(v), (const float*)ptr(a), (const float*)ptr(p), fptr(delta),
                                 ptr(r), fptr(lam0), fptr(eta0), ptr(y), fptr(yvar), fptr(lamT), fptr(etaT), ptr(saved),
                                 ptr(ws), nw, stream_of(q))
                : kla_forward(&d, ptr(q), ptr(k), ptr(v), ptr(a), ptr(p), ptr(r), fptr(lam0), fptr(eta0), ptr(y),
                              fptr(yvar), fptr(lamT), fptr(etaT), ptr(saved), ptr(ws), nw, stream_of(q));
    }
    if (st != KLA_OK) return py::int_((int)st);
    return py::make_tuple(y, obj(yvar), obj(lamT), obj(etaT), obj(saved));
}

// (dq, dk, dv, da, dp, dr, dlam0, deta0[, ddelta]) or a status
py::object backward(const Tensor& q, const Tensor& k, const Tensor& v, const Opt& a, const Opt& p, const Opt& delta,
                    const Tensor& r, const Opt& lam0, const Opt& eta0, const Tensor& dy, const Opt& dlamT,
                    const Opt& detaT, const Opt& saved, bool want_init, const Opt& dyvar, bool noalloc, bool ou) {
    const kla_desc d = check_inputs(q, k, v, per_token(a, ou, "a"), per_token(p, ou, "p"), r);
    if (ou) check_ou(a, p, delta, d.H, d.dk, q);
    check_belief(d, lam0, eta0, q, "lam0", "eta0");
    check_belief(d, dlamT, detaT, q, "dlamT", "detaT");
    check_f32(dyvar, {d.B, d.T, d.H}, q, "dyvar");
    if (dy.sizes() != at::IntArrayRef({d.B, d.T, d.H, d.dv}) || dy.scalar_type() != q.scalar_type() || !dy.is_contiguous())
        value_error("dy must be a contiguous [B, T, H, dv] tensor in the input dtype");
    Tensor dq, dk, dv, da, dp, dr;
    Opt ddelta, dlam0, deta0;
    kla_status st;
    {
        py::gil_scoped_release unlocked;
        const auto f32 = q.options().dtype(at::kFloat);
        dq = at::empty_like(q), dk = at::empty_like(k), dv = at::empty_like(v), dr = at::empty_like(r);
        da = ou ? at::empty({d.H, d.dk}, f32) : at::empty_like(*a);
        dp = ou ? at::empty({d.H, d.dk}, f32) : at::empty_like(*p);
        if (ou) ddelta = at::empty({d.H, d.dk}, f32);
        if (want_init) {
            dlam0 = at::empty({d.B, d.H, d.dk}, f32);
            deta0 = at::empty({d.B, d.H, d.dk, d.dv}, f32);
        }
        if (noalloc) {
            st = kla_backward_noalloc(&d, ptr(q), ptr(k), ptr(v), ptr(a), ptr(p), ptr(r), fptr(lam0), fptr(eta0), ptr(saved),
                                      ptr(dy), fptr(dyvar), fptr(dlamT), fptr(detaT), ptr(dq), ptr(dk), ptr(dv), ptr(da),
                                      ptr(dp), ptr(dr), fptr(dlam0), fptr(deta0), stream_of(q));
        } else if (ou) {
            const size_t nw = kla_backward_ou_workspace(&d, saved.has_value());
            const Tensor ws = bytes(nw, q);
            st = kla_backward_ou(&d, ptr(q), ptr(k), ptr(v), (const float*)ptr(a), (const float*)ptr(p), fptr(delta), ptr(r),
                                 fptr(lam0), fptr(eta0), ptr(saved), ptr(dy), fptr(dyvar), fptr(dlamT), fptr(detaT), ptr(dq),
                                 ptr(dk), ptr(dv), (float*)ptr(da), (float*)ptr(dp), fptr(ddelta), ptr(dr), fptr(dlam0),
                                 fptr(deta0), ptr(ws), nw, stream_of(q));
        } else {
            const size_t nw = kla_backward_workspace(&d, saved.has_value());
            const Tensor ws = bytes(nw, q);
            st = kla_backward(&d, ptr(q), ptr(k), ptr(v), ptr(a), ptr(p), ptr(r), fptr(lam0), fptr(eta0), ptr(saved), ptr(dy),
                              fptr(dyvar), fptr(dlamT), fptr(detaT), ptr(dq), ptr(dk), ptr(dv), ptr(da), ptr(dp), ptr(dr),
                              fptr(dlam0), fptr(deta0), ptr(ws), nw, stream_of(q));
        }
    }
    if (st != KLA_OK) return py::int_((int)st);
    if (ou) return py::make_tuple(dq, dk, dv, da, dp, dr, obj(dlam0), obj(deta0), *ddelta);
    return py::make_tuple(dq, dk, dv, da, dp, dr, obj(dlam0), obj(deta0));
}

// (y, yvar) or a status; lam, eta updated in place
py::object decode_step(const Tensor& q, const Tensor& k, const Tensor& v, const Opt& a, const Opt& p,
                       const Opt& delta, const Tensor& r, const Opt& lam, const Opt& eta, const Opt& y_in,
                       bool want_var, bool ou) {
    if (!q.is_cuda() || (q.scalar_type() != at::kFloat && q.scalar_type() != at::kBFloat16))
        value_error("decode inputs must be fp32/bf16 GPU tensors");
    if (q.dim() != 3) value_error("q must be [S, H, dk]");
    const int64_t S = q.size(0), H = q.size(1), dk = q.size(2), dv = v.size(-1);
    const std::array<int64_t, 3> ks{S, H, dk}, vs{S, H, dv};
    const std::array<int64_t, 2> rs{S, H};
    const Tensor* t[6] = {&q, &k, &v, per_token(a, ou, "a"), per_token(p, ou, "p"), &r};
    for (int i : {1, 3, 4, 2, 5}) {
        if (!t[i]) continue;
        const at::IntArrayRef want = i == 2 ? at::IntArrayRef(vs) : i == 5 ? at::IntArrayRef(rs) : at::IntArrayRef(ks);
        if (t[i]->sizes() != want || t[i]->scalar_type() != q.scalar_type() || !t[i]->is_contiguous())
            value_error(std::string(kNames[i]) + " must be a contiguous " + shape_str(want) + " tensor in q's dtype");
    }
    if (ou) check_ou(a, p, delta, H, dk, q);
    check_f32(lam, {S, H, dk}, q, "lam");
    check_f32(eta, {S, H, dk, dv}, q, "eta");
    const kla_dtype dt = (kla_dtype)dtype_of(q);
    Tensor y;
    Opt yvar;
    kla_status st;
    {
        py::gil_scoped_release unlocked;
        y = y_in ? *y_in : at::empty({S, H, dv}, q.options());
        if (want_var) yvar = at::empty({S, H}, q.options().dtype(at::kFloat));
        st = ou ? kla_decode_step_ou(S, H, dk, dv, dt, ptr(q), ptr(k), ptr(v), (const float*)ptr(a),
                                     (const float*)ptr(p), fptr(delta), ptr(r), fptr(lam), fptr(eta),
                                     ptr(y), fptr(yvar), stream_of(q))
                : kla_decode_step(S, H, dk, dv, dt, ptr(q), ptr(k), ptr(v), ptr(a), ptr(p), ptr(r), fptr(lam),
                                  fptr(eta), ptr(y), fptr(yvar), stream_of(q));
    }
    if (st != KLA_OK) return py::int_((int)st);
    return py::make_tuple(y, obj(yvar));
}

// ---- the operators around the layer: each call runs on its tensors' device, whichever is current

// strided: any strides will do, the caller makes the tensor dense
void check_gpu(const Tensor& t, const char* name, bool strided = false) {
    if (!t.is_cuda()) value_error(std::string(name) + " must live on a GPU; there is no CPU path");
    if (!strided && !t.is_contiguous()) value_error(std::string(name) + " must be contiguous");
}

void check_like(const Tensor& t, at::IntArrayRef shape, const Tensor& q, const char* name, bool strided = false) {
    if (t.sizes() != shape) value_error(std::string(name) + " has shape " + shape_str(t.sizes()) + ", expected " + shape_str(shape));
    if (t.scalar_type() != q.scalar_type() || t.device() != q.device())
        value_error(std::string(name) + " must share the inputs' dtype and device");
    if (!strided && !t.is_contiguous()) value_error(std::string(name) + " must be contiguous");
}

void check_int(const Opt& t, at::ScalarType type, at::IntArrayRef shape, const Tensor& q, const char* name) {
    if (!t) return;
    if (t->scalar_type() != type || t->sizes() != shape || t->device() != q.device() || !t->is_contiguous())
        value_error(std::string(name) + " must be a contiguous " + (type == at::kInt ? "int32" : "int64") +
                    " tensor of shape " + shape_str(shape) + " on " + q.device().str());
}

// Outputs given by the caller: workgroups read inputs while others write, so the two must not overlap; and
// autograd is told that their values change, so that a node that saved one refuses its backward.
void check_apart(const Tensor& out, const char* name, std::initializer_list<const Tensor*> ins) {
    const char* a = (const char*)out.data_ptr();
    for (const Tensor* t : ins) {
        const char* b = (const char*)t->data_ptr();
        if (a < b + t->nbytes() && b < a + out.nbytes()) value_error(std::string(name) + " must not overlap an input");
    }
}

void changed(const Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

int32_t int32_of(int64_t n, const char* what) {
    if (n > INT32_MAX) value_error(std::string(what) + " does not fit 32 bits");
    return (int32_t)n;
}

kla_desc check_lin(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& g, const Opt& s, const Opt& len,
                   bool strided = false) {
    check_gpu(q, "q", strided);
    const int dt = dtype_of(q);
    if (q.dim() != 4 || v.dim() != 4) value_error("q must be [B, T, H, dk] and v [B, T, H, dv]");
    const int64_t B = q.size(0), T = q.size(1), H = q.size(2), dk = q.size(3), dv = v.size(3);
    check_like(k, {B, T, H, dk}, q, "k", strided);
    check_like(v, {B, T, H, dv}, q, "v", strided);
    check_f32(g, {H}, q, "g");
    check_f32(s, {B, H, dk, dv}, q, "s0");
    check_int(len, at::kInt, {B}, q, "lengths");
    return kla_desc{int32_of(B, "B"), int32_of(T, "T"), int32_of(H, "H"), int32_of(dk, "dk"), int32_of(dv, "dv"), (kla_dtype)dt};
}

// A call the library refused: KLAError in Python (the translator below).
struct Refused : std::runtime_error {
    kla_status status;
    const char* where;
    Refused(kla_status s, const char* w) : std::runtime_error(std::string(w) + ": " + kla_status_string(s)), status(s), where(w) {}
};

void ok(kla_status s, const char* where) {
    if (s != KLA_OK) throw Refused(s, where);
}

using Tensors = torch::autograd::variable_list;
using Ctx = torch::autograd::AutogradContext;
Opt some(const Tensor& t) { return t.defined() ? Opt(t) : Opt(); }
Tensor or_undefined(const Opt& t) { return t ? *t : Tensor(); }
// An input as the library takes it, on 16 bytes: a slice of a larger one, such as one layer's row of stacked
// weights, need not be and is copied.
Tensor aligned(const Tensor& t) {
    return t.defined() && reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 ? t.clone() : t;
}
Opt aligned(const Opt& t) { return t ? Opt(aligned(*t)) : Opt(); }
Tensor dense(const Tensor& t) { return t.defined() ? t.contiguous() : t; }
// The nodes' backward passes are not differentiable themselves.
void once() {
    TORCH_CHECK_NOT_IMPLEMENTED(!at::GradMode::is_enabled(), "second derivatives (create_graph=True) are not available");
}
// Where a backward is captured, no node that takes its gradients may belong to the default stream, as a leaf's
// does that an eager graph made which still lives: autograd would have that stream, which cannot be captured, wait
// for the capture, and so end it and the process.
void check_capture(const Tensor& t) {
    const auto stream = c10::hip::getCurrentHIPStream(t.device().index());
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    if (!stream.stream() || hipStreamIsCapturing(stream.stream(), &status) != hipSuccess || status == hipStreamCaptureStatusNone)
        return;
    const auto node = torch::autograd::get_current_node();
    if (!node) return;
    for (const auto& edge : node->next_edges()) {
        if (!edge.function) continue;
        const auto other = edge.function->stream();
        TORCH_CHECK(!other || other->id() != 0,
                    "a backward pass is captured while a graph of the same leaves, made on the default stream, still "
                    "lives: drop its outputs first");
    }
}

// The raw calls take checked tensors and need no interpreter lock.
Tensors lin_forward(const kla_desc& d, const Tensor& q_in, const Tensor& k_in, const Tensor& v_in, const Tensor& g_in,
                    const Opt& s0_in, const Opt& len_in, const Opt& y_in, bool want_state) {
    const c10::hip::HIPGuard on(q_in.device().index());
    const Tensor q = aligned(q_in), k = aligned(k_in), v = aligned(v_in), g = aligned(g_in);
    const Opt s0 = aligned(s0_in), len = aligned(len_in);
    const Tensor y = y_in ? *y_in : at::empty({d.B, d.T, d.H, d.dv}, q.options());
    Opt sT, ws;
    if (want_state) sT = at::empty({d.B, d.H, d.dk, d.dv}, q.options().dtype(at::kFloat));
    const size_t nw = kla_linear_attn_workspace(&d);
    if (nw) ws = bytes(nw, q);
    ok(kla_linear_attn_forward(&d, ptr(q), ptr(k), ptr(v), (const float*)ptr(g), fptr(s0), (const int32_t*)ptr(len), ptr(y),
                               fptr(sT), ptr(ws), nw, stream_of(q)),
       "kla_linear_attn_forward");
    return {y, or_undefined(sT)};
}

Tensors lin_backward(const kla_desc& d, const Tensor& q_in, const Tensor& k_in, const Tensor& v_in, const Tensor& g_in,
                     const Opt& s0_in, const Opt& len_in, const Tensor& dy_in, const Opt& dsT_in, bool want_init) {
    const c10::hip::HIPGuard on(q_in.device().index());
    const Tensor q = aligned(q_in), k = aligned(k_in), v = aligned(v_in), g = aligned(g_in), dy = aligned(dy_in);
    const Opt s0 = aligned(s0_in), len = aligned(len_in), dsT = aligned(dsT_in);
    const Tensor dq = at::empty_like(q), dk = at::empty_like(k), dv = at::empty_like(v);
    Opt ds0, ws;
    if (want_init) ds0 = at::empty({d.B, d.H, d.dk, d.dv}, q.options().dtype(at::kFloat));
    const size_t nw = kla_linear_attn_backward_workspace(&d);
    if (nw) ws = bytes(nw, q);
    ok(kla_linear_attn_backward(&d, ptr(q), ptr(k), ptr(v), (const float*)ptr(g), fptr(s0), (const int32_t*)ptr(len), ptr(dy),
                                fptr(dsT), ptr(dq), ptr(dk), ptr(dv), fptr(ds0), ptr(ws), nw, stream_of(q)),
       "kla_linear_attn_backward");
    return {dq, dk, dv, or_undefined(ds0)};
}

// (y, sT)
py::object linear_attn_forward(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& g, const Opt& s0,
                               const Opt& len, const Opt& y_in, bool want_state) {
    const kla_desc d = check_lin(q, k, v, g, s0, len);
    if (y_in) {
        check_like(*y_in, {d.B, d.T, d.H, d.dv}, q, "y");
        check_apart(*y_in, "y", {&q, &k, &v, &g});
        if (s0) check_apart(*y_in, "y", {&*s0});
        if (len) check_apart(*y_in, "y", {&*len});
    }
    Tensors out;
    {
        py::gil_scoped_release unlocked;
        out = lin_forward(d, q, k, v, g, s0, len, y_in, want_state);
    }
    if (y_in) changed(*y_in);
    return py::make_tuple(out[0], obj(some(out[1])));
}

// (dq, dk, dv, ds0)
py::object linear_attn_backward(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& g, const Opt& s0,
                                const Opt& len, const Tensor& dy, const Opt& dsT, bool want_init) {
    const kla_desc d = check_lin(q, k, v, g, s0, len);
    check_like(dy, {d.B, d.T, d.H, d.dv}, q, "dy");
    check_f32(dsT, {d.B, d.H, d.dk, d.dv}, q, "dsT");
    Tensors out;
    {
        py::gil_scoped_release unlocked;
        out = lin_backward(d, q, k, v, g, s0, len, dy, dsT, want_init);
    }
    return py::make_tuple(out[0], out[1], out[2], obj(some(out[3])));
}

// y, sT with their gradients.  Nodes in C++: through Python's they took most of a small training step.
struct LinearAttn : torch::autograd::Function<LinearAttn> {
    static Tensors forward(Ctx* ctx, const Tensor& q_in, const Tensor& k_in, const Tensor& v_in, const Tensor& g, const Opt& s0,
                           const Opt& len, const kla_desc& d) {
        const Tensor q = dense(q_in), k = dense(k_in), v = dense(v_in);   // parts of a fused projection
        ctx->save_for_backward({q, k, v, g, or_undefined(s0), or_undefined(len)});
        ctx->set_materialize_grads(false);   // an unused output's gradient stays undefined: nothing to fill or read
        ctx->saved_data["init"] = s0 && s0->requires_grad();
        return lin_forward(d, q, k, v, g, s0, len, c10::nullopt, true);
    }
    static Tensors backward(Ctx* ctx, Tensors up) {
        once();
        const Tensors x = ctx->get_saved_variables();
        const Tensor &q = x[0], &v = x[2];
        check_capture(q);
        const kla_desc d{(int32_t)q.size(0), (int32_t)q.size(1), (int32_t)q.size(2), (int32_t)q.size(3), (int32_t)v.size(3),
                         q.scalar_type() == at::kFloat ? KLA_F32 : KLA_BF16};
        const Tensor dy = up[0].defined() ? dense(up[0]) : at::zeros_like(v);
        const Tensors out = lin_backward(d, q, x[1], v, x[3], some(x[4]), some(x[5]), dy, some(dense(up[1])),
                                         ctx->saved_data["init"].toBool());
        return {out[0], out[1], out[2], Tensor(), out[3], Tensor(), Tensor()};
    }
};

py::object linear_attn(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& g, const Opt& s0, const Opt& len) {
    const kla_desc d = check_lin(q, k, v, g, s0, len, true);
    if (g.requires_grad()) value_error("g holds constants: the decays take no gradient");
    Tensors out;
    {
        py::gil_scoped_release unlocked;
        out = LinearAttn::apply(q, k, v, g, s0, len, d);
    }
    return py::make_tuple(out[0], out[1]);
}

// y; state updated in place
py::object linear_attn_step(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& g, const Tensor& state,
                            const Opt& y_in) {
    check_gpu(q, "q");
    const int dt = dtype_of(q);
    if (q.dim() != 3 || v.dim() != 3) value_error("q must be [S, H, dk] and v [S, H, dv]");
    const int64_t S = q.size(0), H = q.size(1), dk = q.size(2), dv = v.size(2);
    check_like(k, {S, H, dk}, q, "k");
    check_like(v, {S, H, dv}, q, "v");
    check_f32(g, {H}, q, "g");
    check_f32(state, {S, H, dk, dv}, q, "state");
    if (y_in) {
        check_like(*y_in, {S, H, dv}, q, "y");
        check_apart(*y_in, "y", {&q, &k, &v, &g, &state});
    }
    check_apart(state, "state", {&q, &k, &v, &g});
    const int32_t s32 = int32_of(S, "S"), h32 = int32_of(H, "H"), dk32 = int32_of(dk, "dk"), dv32 = int32_of(dv, "dv");
    Tensor y;
    {
        py::gil_scoped_release unlocked;
        const c10::hip::HIPGuard on(q.device().index());
        y = y_in ? *y_in : at::empty({S, H, dv}, q.options());
        const Tensor qa = aligned(q), ka = aligned(k), va = aligned(v), ga = aligned(g);
        ok(kla_linear_attn_step(s32, h32, dk32, dv32, dt, ptr(qa), ptr(ka), ptr(va), (const float*)ptr(ga), (float*)ptr(state),
                                ptr(y), stream_of(q)),
           "kla_linear_attn_step");
    }
    changed(state);
    if (y_in) changed(*y_in);
    return py::cast(y);
}

struct Rows {
    int64_t rows;
    int32_t n;
    int dtype;
    std::vector<int64_t> lead;
};

Rows rows_of(const Tensor& x, const char* name) {
    if (!x.is_cuda()) value_error(std::string(name) + " must live on a GPU; there is no CPU path");
    const int dt = dtype_of(x);
    if (x.dim() < 1) value_error(std::string(name) + " must have a last dimension");
    const int64_t n = x.size(-1);
    std::vector<int64_t> lead(x.sizes().begin(), x.sizes().end() - 1);
    int64_t rows = 1;
    for (int64_t s : lead) rows *= s;
    return {rows, int32_of(n, "the row length"), dt, lead};
}

Rows check_rows(const Tensor& x, const char* name) {
    const Rows r = rows_of(x, name);
    check_gpu(x, name);
    return r;
}

Tensors norm_forward(const Rows& r, const Tensor& x_in, const Tensor& w_in, const Opt& bias_in, double eps) {
    const c10::hip::HIPGuard on(x_in.device().index());
    const Tensor x = aligned(x_in), w = aligned(w_in);
    const Opt bias = aligned(bias_in);
    const Tensor out = at::empty_like(x), mean = at::empty(r.lead, x.options().dtype(at::kFloat)), rstd = at::empty_like(mean);
    ok(kla_layer_norm_forward(r.rows, r.n, r.dtype, ptr(x), (const float*)ptr(w), fptr(bias), (float)eps, ptr(out),
                              (float*)ptr(mean), (float*)ptr(rstd), stream_of(x)),
       "kla_layer_norm_forward");
    return {out, mean, rstd};
}

Tensors norm_backward(const Rows& r, const Tensor& x_in, const Tensor& w_in, const Tensor& mean_in, const Tensor& rstd_in,
                      const Tensor& dout_in, bool want_bias) {
    const c10::hip::HIPGuard on(x_in.device().index());
    const Tensor x = aligned(x_in), w = aligned(w_in), mean = aligned(mean_in), rstd = aligned(rstd_in), dout = aligned(dout_in);
    const Tensor dx = at::empty_like(x), dw = at::empty_like(w);
    Opt db;
    if (want_bias) db = at::empty_like(w);
    const size_t nw = kla_layer_norm_workspace(r.n);
    const Tensor ws = bytes(nw, x);
    ok(kla_layer_norm_backward(r.rows, r.n, r.dtype, ptr(x), (const float*)ptr(w), (const float*)ptr(mean),
                               (const float*)ptr(rstd), ptr(dout), ptr(dx), (float*)ptr(dw), fptr(db), ptr(ws), nw, stream_of(x)),
       "kla_layer_norm_backward");
    return {dx, dw, or_undefined(db)};
}

// (out, mean, rstd)
py::object layer_norm_forward(const Tensor& x, const Tensor& w, const Opt& bias, double eps) {
    const Rows r = check_rows(x, "x");
    check_f32(w, {r.n}, x, "w");
    check_f32(bias, {r.n}, x, "bias");
    Tensors out;
    {
        py::gil_scoped_release unlocked;
        out = norm_forward(r, x, w, bias, eps);
    }
    return py::make_tuple(out[0], out[1], out[2]);
}

// (dx, dw, dbias)
py::object layer_norm_backward(const Tensor& x, const Tensor& w, const Tensor& mean, const Tensor& rstd, const Tensor& dout,
                               bool want_bias) {
    const Rows r = check_rows(x, "x");
    check_f32(w, {r.n}, x, "w");
    check_f32(mean, r.lead, x, "mean");
    check_f32(rstd, r.lead, x, "rstd");
    check_like(dout, x.sizes(), x, "dout");
    Tensors out;
    {
        py::gil_scoped_release unlocked;
        out = norm_backward(r, x, w, mean, rstd, dout, want_bias);
    }
    return py::make_tuple(out[0], out[1], obj(some(out[2])));
}

struct LayerNorm : torch::autograd::Function<LayerNorm> {
    static Tensor forward(Ctx* ctx, const Tensor& x_in, const Tensor& w, const Opt& bias, double eps) {
        const Tensor x = aligned(dense(x_in));
        const Tensors out = norm_forward(rows_of(x, "x"), x, w, bias, eps);
        ctx->save_for_backward({x, w, out[1], out[2]});
        ctx->saved_data["bias"] = bias && bias->requires_grad();
        return out[0];
    }
    static Tensors backward(Ctx* ctx, Tensors up) {
        once();
        const Tensors s = ctx->get_saved_variables();
        check_capture(s[0]);
        const Tensors out = norm_backward(rows_of(s[0], "x"), s[0], s[1], s[2], s[3], dense(up[0]),
                                          ctx->saved_data["bias"].toBool());
        return {out[0], out[1], out[2], Tensor()};
    }
};

Tensor layer_norm(const Tensor& x, const Tensor& w, const Opt& bias, double eps) {
    const Rows r = rows_of(x, "x");
    check_f32(w, {r.n}, x, "w");
    check_f32(bias, {r.n}, x, "bias");
    py::gil_scoped_release unlocked;
    return LayerNorm::apply(x, w, bias, eps);
}

struct Logits {
    int32_t S, V;
    int64_t n;
    int dtype;
    std::vector<int64_t> lead;
};

// logits [*lead, V], target [*tail] with lead ending in tail: the dimensions before it are draws
Logits logits_of(const Tensor& x, const Tensor& target) {
    const Rows r = rows_of(x, "logits");
    const at::IntArrayRef lead(r.lead), t = target.sizes();
    if (t.size() > lead.size() || lead.slice(lead.size() - t.size()) != t)
        value_error("target has shape " + shape_str(t) + ", expected the last dimensions of " + shape_str(lead));
    int64_t S = 1;
    for (size_t i = 0; i < lead.size() - t.size(); ++i) S *= lead[i];
    return {int32_of(S, "the number of draws"), r.n, target.numel(), r.dtype, r.lead};
}

Logits check_logits(const Tensor& x, const Tensor& target) {
    const Logits l = logits_of(x, target);
    check_gpu(x, "logits");
    check_int(target, at::kLong, target.sizes(), x, "target");
    return l;
}

std::vector<int64_t> with(std::vector<int64_t> lead, int64_t n) {
    lead.push_back(n);
    return lead;
}

// logp, entropy, stat, top_logp, top_index.  No rows, or no draws of them: nothing to do.
Tensors logp_forward(const Logits& l, const Tensor& x_in, const Tensor& target_in, bool want_entropy, int32_t top,
                     bool want_stat) {
    const c10::hip::HIPGuard on(x_in.device().index());
    const Tensor x = aligned(x_in), target = aligned(target_in);
    const auto f32 = x.options().dtype(at::kFloat);
    const Tensor logp = at::empty(l.lead, f32);
    Opt entropy, stat, top_logp, top_index, ws;
    if (want_entropy) entropy = at::empty(l.lead, f32);
    if (want_stat) stat = at::empty(with(l.lead, 2), f32);
    if (top > 0) {
        top_logp = at::empty(with(l.lead, top), f32);
        top_index = at::empty(with(l.lead, top), x.options().dtype(at::kLong));
    }
    const size_t nw = kla_token_logp_workspace(l.S, l.n, l.V, top);
    if (nw) ws = bytes(nw, x);
    if (logp.numel() > 0)
        ok(kla_token_logp_forward(l.S, l.n, l.V, top, l.dtype, ptr(x), (const int64_t*)ptr(target), (float*)ptr(logp),
                                  fptr(entropy), fptr(stat), fptr(top_logp), (int64_t*)ptr(top_index), ptr(ws), nw, stream_of(x)),
           "kla_token_logp_forward");
    return {logp, or_undefined(entropy), or_undefined(stat), or_undefined(top_logp), or_undefined(top_index)};
}

Tensor logp_backward(const Logits& l, const Tensor& x_in, const Tensor& target_in, const Tensor& stat_in,
                     const Opt& entropy_in, const Opt& dlogp_in, const Opt& dentropy_in) {
    const c10::hip::HIPGuard on(x_in.device().index());
    const Tensor x = aligned(x_in), target = aligned(target_in), stat = aligned(stat_in);
    const Opt entropy = aligned(entropy_in), dlogp = aligned(dlogp_in), dentropy = aligned(dentropy_in);
    const Tensor dx = at::empty_like(x);
    if (x.numel() > 0)
        ok(kla_token_logp_backward(l.S, l.n, l.V, l.dtype, ptr(x), (const int64_t*)ptr(target), (const float*)ptr(stat),
                                   fptr(entropy), fptr(dlogp), fptr(dentropy), ptr(dx), stream_of(x)),
           "kla_token_logp_backward");
    return dx;
}

// (logp, entropy, stat, top_logp, top_index)
py::object token_logp_forward(const Tensor& x, const Tensor& target, bool want_entropy, int64_t top, bool want_stat) {
    const Logits l = check_logits(x, target);
    if (top < 0) value_error("top must not be negative");
    const int32_t top32 = int32_of(top, "top");
    Tensors out;
    {
        py::gil_scoped_release unlocked;
        out = logp_forward(l, x, target, want_entropy, top32, want_stat);
    }
    return py::make_tuple(out[0], obj(some(out[1])), obj(some(out[2])), obj(some(out[3])), obj(some(out[4])));
}

// dlogits
Tensor token_logp_backward(const Tensor& x, const Tensor& target, const Tensor& stat, const Opt& entropy,
                           const Opt& dlogp, const Opt& dentropy) {
    const Logits l = check_logits(x, target);
    check_f32(stat, with(l.lead, 2), x, "stat");
    check_f32(entropy, l.lead, x, "entropy");
    check_f32(dlogp, l.lead, x, "dlogp");
    check_f32(dentropy, l.lead, x, "dentropy");
    py::gil_scoped_release unlocked;
    return logp_backward(l, x, target, stat, entropy, dlogp, dentropy);
}

struct TokenLogp : torch::autograd::Function<TokenLogp> {
    static Tensors forward(Ctx* ctx, const Tensor& x_in, const Tensor& target_in, bool want_entropy) {
        const Tensor x = aligned(dense(x_in)), target = aligned(dense(target_in));
        const Tensors out = logp_forward(logits_of(x, target), x, target, want_entropy, 0, true);
        ctx->save_for_backward({x, target, out[2], out[1]});
        ctx->set_materialize_grads(false);
        return want_entropy ? Tensors{out[0], out[1]} : Tensors{out[0]};
    }
    static Tensors backward(Ctx* ctx, Tensors up) {
        once();
        const Tensors s = ctx->get_saved_variables();
        check_capture(s[0]);
        const Tensor dentropy = up.size() > 1 ? dense(up[1]) : Tensor();
        return {logp_backward(logits_of(s[0], s[1]), s[0], s[1], s[2], some(s[3]), some(dense(up[0])), some(dentropy)), Tensor(),
                Tensor()};
    }
};

py::object token_logp(const Tensor& x, const Tensor& target, bool want_entropy) {
    logits_of(x, target);
    if (target.scalar_type() != at::kLong || target.device() != x.device())
        value_error("target must be an int64 tensor on " + x.device().str());
    Tensors out;
    {
        py::gil_scoped_release unlocked;
        out = TokenLogp::apply(x, target, want_entropy);
    }
    if (!want_entropy) return py::cast(out[0]);
    return py::make_tuple(out[0], out[1]);
}

}  // namespace

PYBIND11_MODULE(_kla_torch, m) {
    py::register_exception_translator([](std::exception_ptr p) {
        try {
            if (p) std::rethrow_exception(p);
        } catch (const Refused& e) {
            const py::object type = py::module_::import("paper_2602_10743_amd").attr("KLAError");
            PyErr_SetObject(type.ptr(), type((int)e.status, e.where).ptr());
        }
    });
    m.def("linear_attn", &linear_attn);
    m.def("layer_norm", &layer_norm);
    m.def("token_logp", &token_logp);
    m.def("linear_attn_forward", &linear_attn_forward);
    m.def("linear_attn_backward", &linear_attn_backward);
    m.def("linear_attn_step", &linear_attn_step);
    m.def("layer_norm_forward", &layer_norm_forward);
    m.def("layer_norm_backward", &layer_norm_backward);
    m.def("token_logp_forward", &token_logp_forward);
    m.def("token_logp_backward", &token_logp_backward);
    m.def("forward", &forward);
    m.def("backward", &backward);
    m.def("decode_step", &decode_step);
}
