// Tensor front end of the state-space block's operators: checks tensors, allocates
// outputs and scratch on PyTorch's current stream and calls the C ABI (include/sn.h).
//
// A token's operators run for a few microseconds each on the GPU, as long as their
// arguments take to be marshalled from Python (ctypes and tensor attributes: 9 us for
// a dense layer of one row, 14 for a norm with two outputs, on the GB300's Arm host);
// here the same takes the launch and the allocations.
#include "tensors.h"

void bind_attention(py::module_ &m);  // attention.cpp

namespace {

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
    m.doc() = "Tensor front end of the block and attention operators (see blocks.py, attention.py)";
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
    bind_attention(m);
}
