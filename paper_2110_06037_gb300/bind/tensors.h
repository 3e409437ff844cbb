// What the tensor front ends of the operators share: checks of tensors, outputs, scratch, errors.
#pragma once

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

struct Fail {  // (one type for all files: the module turns it into SnError)
    int status;
    std::string msg;
};

namespace {  // (of each file that includes it)

using at::Tensor;
using Opt = std::optional<Tensor>;

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

}  // namespace
