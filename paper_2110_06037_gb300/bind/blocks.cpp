// Tensor front end of the state-space block's operators: checks tensors, allocates
// outputs and scratch on PyTorch's current stream and calls the C ABI (include/sn.h).
//
// A token's operators run for a few microseconds each on the GPU, as long as their
// arguments take to be marshalled from Python (ctypes and tensor attributes: 9 us for
// a dense layer of one row, 14 for a norm with two outputs, on the GB300's Arm host);
// here the same takes the launch and the allocations.
#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <pybind11/stl.h>
#include <torch/csrc/utils/pybind.h>

#include <algorithm>
#include <optional>
#include <string>

#include "sn.h"

namespace py = pybind11;

namespace {

using at::Tensor;
using Opt = std::optional<Tensor>;

struct Fail {
    int status;
    std::string msg;
};
[[noreturn]] void refuse(const std::string &msg) { throw Fail{SN_EINVAL, msg}; }
void check(sn_status rc) {
    if (rc != SN_OK) throw Fail{(int)rc, sn_last_error()};
}

std::string shape_of(const Tensor &t) {
    std::string s = "(";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + ")";
}
int dtype_of(at::ScalarType t, const char *what) {
    if (t == at::kFloat) return SN_F32;
    if (t == at::kHalf) return SN_F16;
    if (t == at::kBFloat16) return SN_BF16;
    refuse(std::string(what) + " must be fp32, fp16 or bf16, not " + at::toString(t));
}

// rows of a tensor [..., width] whose leading axes collapse to evenly spaced rows
struct Rows {
    void *p = nullptr;
    int64_t ld = 0, n = 0;
};
Rows rows_of(const Tensor &t, int64_t width, const char *what, std::optional<at::ScalarType> like = {}) {
    if (!t.is_cuda()) refuse(std::string(what) + " must be a CUDA tensor");
    if (like && t.scalar_type() != *like)
        refuse(std::string(what) + " must be " + at::toString(*like) + ", not " + at::toString(t.scalar_type()));
    const int64_t d = t.dim();
    if (d == 0 || t.size(d - 1) != width)
        refuse(std::string(what) + " must have rows of " + std::to_string(width) + ", not shape " + shape_of(t));
    if (width > 1 && t.numel() && t.stride(d - 1) != 1) refuse(std::string("the values of a row of ") + what + " must be contiguous");
    Rows r;
    r.p = t.data_ptr();
    r.n = 1;
    // leading axes of more than one entry, from the last: each a multiple of the one behind it
    // (an expanded axis, of stride 0, is none: its rows are not apart)
    int64_t expect = 0;
    bool seen = false;
    for (int64_t i = d - 2; i >= 0; --i) {
        const int64_t n = t.size(i), stride = t.stride(i);
        r.n *= n;
        if (n == 1 || t.numel() == 0) continue;
        if (stride == 0) refuse(std::string("the rows of ") + what + " lie on one another (an expanded axis)");
        if (!seen) r.ld = stride;
        else if (stride != expect) refuse(std::string("the leading axes of ") + what + " do not collapse to evenly spaced rows");
        seen = true;
        expect = stride * n;
    }
    if (r.n <= 1) r.ld = std::max(r.ld, width);
    return r;
}
// pointer of a contiguous CUDA tensor of exactly this shape and type
void *whole(const Tensor &t, at::IntArrayRef shape, at::ScalarType dtype, const char *what) {
    if (t.is_cuda() && t.scalar_type() == dtype && t.sizes() == shape && t.is_contiguous()) return t.data_ptr();
    std::string s = "(";
    for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
    refuse(std::string(what) + " must be a contiguous CUDA " + at::toString(dtype) + " tensor of shape " + s + "), not " +
           at::toString(t.scalar_type()) + " " + shape_of(t) + " on " + t.device().str());
}
void *whole(const Opt &t, at::IntArrayRef shape, at::ScalarType dtype, const char *what) {
    return t ? whole(*t, shape, dtype, what) : nullptr;
}
// entries of a buffer of them
int64_t entries_of(const Tensor &t, const char *what) {
    if (t.dim() == 0) refuse(std::string(what) + " has no axis of entries");
    return t.size(0);
}
const int32_t *index_of(const Opt &t, int64_t n, const char *what) {
    return static_cast<const int32_t *>(whole(t, {n}, at::kInt, what));
}
// what a call takes beside its first tensor: on the same device (a handle's weights are on
// `handle`, -1 where it has none)
struct Device {
    int index;
    Device(const Tensor &first, int handle) : index(first.is_cuda() ? first.get_device() : -1) {
        if (handle >= 0 && index >= 0 && handle != index)
            refuse("the handle's weights are on device " + std::to_string(handle) + ", the call's tensors on " + std::to_string(index));
    }
    void same(const Tensor &t, const char *what) const {
        if (index >= 0 && (!t.is_cuda() || t.get_device() != index))
            refuse(std::string(what) + " is on " + t.device().str() + ", the call's first tensor on device " + std::to_string(index));
    }
    void same(const Opt &t, const char *what) const {
        if (t) same(*t, what);
    }
};
// an output: the caller's, or a new one
Tensor output(const Opt &out, at::IntArrayRef shape, at::ScalarType dtype, const Tensor &like, const char *what) {
    if (!out) return at::empty(shape, like.options().dtype(dtype));
    if (out->sizes() != shape || out->scalar_type() != dtype) refuse(std::string(what) + " has another shape or type than the result");
    return *out;
}
at::DimVector shape_with(const Tensor &t, int64_t last) {
    at::DimVector s(t.sizes().begin(), t.sizes().end());
    s.back() = last;
    return s;
}
void *stream_of(const Tensor &t) { return c10::cuda::getCurrentCUDAStream(t.get_device()).stream(); }
Tensor scratch(int64_t bytes, const Tensor &like) { return at::empty({bytes}, like.options().dtype(at::kByte)); }

Tensor dense_q4(intptr_t handle, int device, const Tensor &x, const Opt &out) {
    const auto *w = reinterpret_cast<const sn_q4_weights *>(handle);
    const int dt = dtype_of(x.scalar_type(), "x");
    const Rows r = rows_of(x, w->k, "x");
    Device(x, device).same(out, "out");
    const c10::cuda::CUDAGuard guard(x.device());
    Tensor y = output(out, shape_with(x, w->n), x.scalar_type(), x, "out");
    const Rows o = rows_of(y, w->n, "out");
    int64_t bytes = 0;
    check(sn_q4_workspace(w, dt, r.n, r.p, r.ld, &bytes));
    Tensor work;
    if (bytes) work = scratch(bytes, x);
    check(sn_q4_dense(w, dt, r.n, r.p, r.ld, o.p, o.ld, bytes ? work.data_ptr() : nullptr, bytes, stream_of(x)));
    return y;
}

py::tuple block_norm(intptr_t handle, int device, const Opt &y, const Opt &residual, const Opt &gate, int64_t per, const Opt &out,
                     const Opt &out_normed, const std::optional<at::ScalarType> &dtype) {
    const auto *p = reinterpret_cast<const sn_norm_params *>(handle);
    if (!y && !residual) refuse("neither y nor residual");
    const Tensor &first = y ? *y : *residual;
    const at::ScalarType type = y || !dtype ? first.scalar_type() : *dtype;
    const int64_t d = p->dim;
    const int dt = dtype_of(type, "rows");
    const Device on(first, device);
    on.same(residual, "residual"), on.same(gate, "gate"), on.same(out, "out"), on.same(out_normed, "out_normed");
    Rows ry, rr, rg, rs, rn;
    int rdt = dt;
    int64_t rows = 0;
    if (y) {
        ry = rows_of(*y, d, "y");
        rows = ry.n;
    }
    if (residual) {
        rdt = dtype_of(residual->scalar_type(), "residual");
        rr = rows_of(*residual, d, "residual");
        if (y && rr.n != rows) refuse("residual and y have different rows");
        rows = rr.n;
    }
    if (gate) {
        rg = rows_of(*gate, d, "gate", type);
        if (per < 1 || rg.n < (rows + per - 1) / per) refuse("too few gate rows");
    }
    const c10::cuda::CUDAGuard guard(first.device());
    Opt total, normed;
    if (y || out) {
        total = output(out, first.sizes(), residual ? residual->scalar_type() : type, first, "out");
        rs = rows_of(*total, d, "out");
    }
    if (p->pre) {
        normed = output(out_normed, first.sizes(), type, first, "out_normed");
        rn = rows_of(*normed, d, "out_normed");
    }
    check(sn_block_norm(p, dt, rows, ry.p, ry.ld, rg.p, rg.ld, per, rdt, rr.p, rr.ld, rs.p, rs.ld, rn.p, rn.ld, stream_of(first)));
    return py::make_tuple(total ? *total : *residual, normed);
}

struct Batch {
    int64_t tokens, max_len;
    int32_t n;
    const int32_t *offsets;
};
Batch batch_of(const Tensor &t, const Opt &offsets, const std::optional<int64_t> &max_len) {
    if (!offsets) {
        if (t.dim() != 3) refuse("without offsets the input is [batch, tokens, channels]");
        return Batch{t.size(0) * t.size(1), t.size(1), (int32_t)t.size(0), nullptr};
    }
    if (t.dim() != 2 || !max_len) refuse("with offsets the input is [tokens, channels], and max_len is needed");
    const int64_t n = offsets->numel() - 1;
    if (n < 0) refuse("offsets are empty");
    return Batch{t.size(0), std::min(*max_len, t.size(0)), (int32_t)n, index_of(offsets, n + 1, "offsets")};
}

Tensor causal_conv(const Tensor &x, const Tensor &weight, const Opt &bias, bool silu, const Opt &offsets,
                   const std::optional<int64_t> &max_len, const Opt &kept, const Opt &slots, const Opt &pos, const Opt &out) {
    if (weight.dim() != 2) refuse("weight must be [channels, width]");
    const int64_t c = weight.size(0), width = weight.size(1);
    const int dt = dtype_of(x.scalar_type(), "x");
    const Device on(x, -1);
    on.same(weight, "weight"), on.same(bias, "bias"), on.same(offsets, "offsets"), on.same(kept, "kept");
    on.same(slots, "slots"), on.same(pos, "pos"), on.same(out, "out");
    const Batch b = batch_of(x, offsets, max_len);
    const Rows r = rows_of(x, c, "x");
    const int64_t n = kept ? entries_of(*kept, "kept") : b.n;
    void *kp = kept ? whole(*kept, {n, width, c}, x.scalar_type(), "kept") : nullptr;
    if (kept && !slots && n < b.n) refuse("kept has fewer entries than there are sequences");
    const auto *w = static_cast<const float *>(whole(weight, {c, width}, at::kFloat, "weight"));
    const auto *wb = static_cast<const float *>(whole(bias, {c}, at::kFloat, "bias"));
    const c10::cuda::CUDAGuard guard(x.device());
    Tensor y = output(out, x.sizes(), x.scalar_type(), x, "out");
    const Rows o = rows_of(y, c, "out");
    check(sn_causal_conv(dt, (int32_t)c, (int32_t)width, silu, w, wb, b.tokens, b.n, b.max_len, b.offsets, r.p, r.ld, o.p, o.ld, kp, (int32_t)n,
                         index_of(slots, b.n, "slots"), index_of(pos, b.n, "pos"), stream_of(x)));
    return y;
}

struct States {
    int64_t n;
    float *in, *out;
};
States states_of(const sn_ssm_params *p, const Opt &in, const Opt &out, int64_t batch, bool slots) {
    const int64_t n = in ? entries_of(*in, "state_in") : out ? entries_of(*out, "state_out") : batch;
    const int64_t shape[4] = {n, p->heads, p->head_dim, p->state};
    States s{n, static_cast<float *>(whole(in, shape, at::kFloat, "state_in")), static_cast<float *>(whole(out, shape, at::kFloat, "state_out"))};
    if (!slots && (in || out) && n < batch) refuse("fewer states than sequences");
    return s;
}
int64_t channels_of(const sn_ssm_params *p) { return (int64_t)p->heads * p->head_dim + 2LL * p->groups * p->state; }

Tensor scan(intptr_t handle, int device, const Tensor &xbc, const Tensor &dt, const Opt &offsets, const std::optional<int64_t> &max_len,
            const Opt &state_in, const Opt &state_out, const Opt &slots, const Opt &out) {
    const auto *p = reinterpret_cast<const sn_ssm_params *>(handle);
    const int code = dtype_of(xbc.scalar_type(), "xbc");
    const Device on(xbc, device);
    on.same(dt, "dt"), on.same(offsets, "offsets"), on.same(state_in, "state_in"), on.same(state_out, "state_out");
    on.same(slots, "slots"), on.same(out, "out");
    const Batch b = batch_of(xbc, offsets, max_len);
    const Rows r = rows_of(xbc, channels_of(p), "xbc"), rd = rows_of(dt, p->heads, "dt", xbc.scalar_type());
    if (rd.n != b.tokens) refuse("dt and xbc have different tokens");
    const States s = states_of(p, state_in, state_out, b.n, slots.has_value());
    const c10::cuda::CUDAGuard guard(xbc.device());
    const int64_t inner = (int64_t)p->heads * p->head_dim;
    Tensor y = output(out, shape_with(xbc, inner), xbc.scalar_type(), xbc, "out");
    const Rows o = rows_of(y, inner, "out");
    int64_t bytes = 0;
    check(sn_ssm_workspace(p, code, b.tokens, b.n, b.max_len, &bytes));
    Tensor work;
    if (bytes) work = scratch(bytes, xbc);
    check(sn_ssm_scan(p, code, b.tokens, b.n, b.max_len, b.offsets, r.p, r.ld, rd.p, rd.ld, s.in, s.out, (int32_t)s.n,
                      index_of(slots, b.n, "slots"), o.p, o.ld, bytes ? work.data_ptr() : nullptr, bytes, stream_of(xbc)));
    return y;
}

Tensor step(intptr_t handle, int device, const Tensor &xbc, const Tensor &dt, const Tensor &kept, const Tensor &state, const Opt &pos, const Opt &state_out,
            const Opt &slots, const Opt &out) {
    const auto *p = reinterpret_cast<const sn_ssm_params *>(handle);
    const int code = dtype_of(xbc.scalar_type(), "xbc");
    const Device on(xbc, device);
    on.same(dt, "dt"), on.same(kept, "kept"), on.same(state, "state"), on.same(pos, "pos"), on.same(state_out, "state_out");
    on.same(slots, "slots"), on.same(out, "out");
    const Rows r = rows_of(xbc, channels_of(p), "xbc"), rd = rows_of(dt, p->heads, "dt", xbc.scalar_type());
    if (rd.n != r.n) refuse("dt and xbc have different rows");
    const States s = states_of(p, state, state_out ? state_out : Opt(state), r.n, slots.has_value());
    void *kp = whole(kept, {s.n, p->width, channels_of(p)}, xbc.scalar_type(), "kept");
    const c10::cuda::CUDAGuard guard(xbc.device());
    const int64_t inner = (int64_t)p->heads * p->head_dim;
    Tensor y = output(out, shape_with(xbc, inner), xbc.scalar_type(), xbc, "out");
    const Rows o = rows_of(y, inner, "out");
    check(sn_ssm_step(p, code, (int32_t)r.n, r.p, r.ld, rd.p, rd.ld, kp, s.in, s.out, (int32_t)s.n, index_of(slots, r.n, "slots"),
                      index_of(pos, r.n, "pos"), o.p, o.ld, stream_of(xbc)));
    return y;
}

}  // namespace

PYBIND11_MODULE(_blocks, m) {
    m.doc() = "Tensor front end of the state-space block's operators (see blocks.py)";
    py::register_exception_translator([](std::exception_ptr e) {
        try {
            if (e) std::rethrow_exception(e);
        } catch (const Fail &f) {
            py::object type = py::module_::import("paper_2110_06037_gb300._sn").attr("SnError");
            PyErr_SetObject(type.ptr(), py::make_tuple(f.status, f.msg).ptr());
        }
    });
    m.def("dense_q4", &dense_q4);
    m.def("block_norm", &block_norm);
    m.def("causal_conv", &causal_conv);
    m.def("scan", &scan);
    m.def("step", &step);
}
