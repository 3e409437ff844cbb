// Tensor front end of the attention layer's operators (see attention.py): checks tensors, allocates
// outputs and scratch on PyTorch's current stream and calls the C ABI (include/sn.h).
#include <cmath>

#include "tensors.h"

namespace {

// the heads of a tensor [..., heads, dim] whose leading axes collapse to evenly spaced tokens
struct Heads {
    void *p = nullptr;
    int64_t ld = 0, hd = 0, n = 0, heads = 0;
};
Heads heads_of(const Tensor &t, int64_t dim, const char *what, std::optional<at::ScalarType> like = {}) {
    if (!t.is_cuda()) refuse(std::string(what) + " must be a CUDA tensor");
    if (like && t.scalar_type() != *like)
        refuse(std::string(what) + " must be " + at::toString(*like) + ", not " + at::toString(t.scalar_type()));
    const int64_t d = t.dim();
    if (d < 2 || t.size(d - 1) != dim)
        refuse(std::string(what) + " must have heads of " + std::to_string(dim) + ", not shape " + shape_of(t));
    Heads r;
    r.p = t.data_ptr();
    r.heads = t.size(d - 2);
    r.n = 1;
    for (int64_t i = 0; i < d - 2; ++i) r.n *= t.size(i);
    if (t.numel() == 0) return r;
    if (dim > 1 && t.stride(d - 1) != 1) refuse(std::string("the values of a head of ") + what + " must be contiguous");
    auto apart = [&](int64_t i) {
        if (t.size(i) > 1 && t.stride(i) <= 0) refuse(std::string("the heads of ") + what + " lie on one another (an expanded axis)");
    };
    apart(d - 2);
    r.hd = r.heads > 1 ? t.stride(d - 2) : dim;
    bool seen = false;
    int64_t expect = 0;
    for (int64_t i = d - 3; i >= 0; --i) {
        if (t.size(i) == 1) continue;
        apart(i);
        if (!seen) r.ld = t.stride(i);
        else if (t.stride(i) != expect) refuse(std::string("the leading axes of ") + what + " do not collapse to evenly spaced tokens");
        seen = true;
        expect = t.stride(i) * t.size(i);
    }
    if (!seen) r.ld = std::max(dim, r.heads * r.hd);
    return r;
}
Tensor output_like(const Opt &out, const Tensor &t, const char *what) { return output(out, t.sizes(), t.scalar_type(), t, what); }

// the tokens of a batch: [batch, tokens, heads, dim], or [tokens, heads, dim] with offsets
Batch tokens_of(const Tensor &t, const Opt &offsets, const std::optional<int64_t> &max_len, const char *what) {
    if (!offsets) {
        if (t.dim() != 4) refuse(std::string("without offsets ") + what + " is [batch, tokens, heads, dim]");
        if (t.size(0) > 65535) throw Fail{SN_EUNSUPPORTED, "more than 65535 sequences"};
        return Batch{t.size(0) * t.size(1), t.size(1), (int32_t)t.size(0), nullptr};
    }
    if (t.dim() != 3 || !max_len) refuse(std::string("with offsets ") + what + " is [tokens, heads, dim], and max_len is needed");
    const int64_t n = offsets->numel() - 1;
    if (n < 0) refuse("offsets are empty");
    if (n > 65535) throw Fail{SN_EUNSUPPORTED, "more than 65535 sequences"};
    return Batch{t.size(0), std::min(*max_len, t.size(0)), (int32_t)n, index_of(offsets, n + 1, "offsets")};
}
struct Table {
    const int32_t *p;
    int32_t n, width;
};
Table table_of(const Tensor &t, int64_t batch, const Opt &slots) {
    if (t.dim() != 2) refuse("table must be [entries, pages], not shape " + shape_of(t));
    if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX) refuse("table is too large");
    const auto *p = static_cast<const int32_t *>(whole(t, t.sizes(), at::kInt, "table"));
    if (!slots && t.size(0) < batch) refuse("table has fewer entries than there are sequences");
    return Table{p, (int32_t)t.size(0), (int32_t)t.size(1)};
}
bool same_dtype(const sn_kv_cache *c, int dt) { return c->dtype == SN_QI8 || c->dtype == dt; }

py::tuple head_rope(intptr_t handle, int device, const Opt &q, const Opt &k, const Opt &pos, const Opt &q_out, const Opt &k_out) {
    sn_rope_params p = *reinterpret_cast<const sn_rope_params *>(handle);
    if (!q && !k) refuse("neither q nor k");
    if ((!q && q_out) || (!k && k_out)) refuse("an output without its input");
    const Tensor &first = q ? *q : *k;
    const int dt = dtype_of(first.scalar_type(), "q and k");
    const Device on(first, device);
    on.same(k, "k"), on.same(pos, "pos"), on.same(q_out, "q_out"), on.same(k_out, "k_out");
    Heads hq, hk;
    if (q) hq = heads_of(*q, p.head_dim, "q");
    if (k) hk = heads_of(*k, p.head_dim, "k", first.scalar_type());
    const int64_t tokens = q ? hq.n : hk.n;
    if (q && k && hq.n != hk.n) refuse("q and k have different tokens");
    const int32_t *at = nullptr;
    if (pos) {
        // [tokens], or [tokens, axes]; leading axes as those of q and k
        const int64_t n = pos->numel();
        int64_t axes = 1;
        if (pos->dim() && !(n == tokens && pos->dim() == first.dim() - 2)) axes = pos->size(pos->dim() - 1);
        if (axes < 1 || n != tokens * axes) refuse("pos must have a position (or one an axis) of each token, not shape " + shape_of(*pos));
        if (axes < p.axes) refuse("pos has " + std::to_string(axes) + " axes, the pairs' are " + std::to_string(p.axes));
        at = static_cast<const int32_t *>(whole(*pos, pos->sizes(), at::kInt, "pos"));
        if (axes > 65536) refuse("pos has too many axes");
        p.axes = (int32_t)axes;
    } else if (p.pairs && tokens) {
        refuse("pos is needed");
    }
    const c10::cuda::CUDAGuard guard(first.device());
    Opt yq, yk;
    Heads oq, ok;
    if (q) yq = output_like(q_out, *q, "q_out"), oq = heads_of(*yq, p.head_dim, "q_out");
    if (k) yk = output_like(k_out, *k, "k_out"), ok = heads_of(*yk, p.head_dim, "k_out");
    check(sn_head_rope(&p, dt, tokens, (int32_t)hq.heads, hq.p, hq.ld, hq.hd, oq.p, oq.ld, oq.hd, (int32_t)hk.heads, hk.p, hk.ld, hk.hd,
                       ok.p, ok.ld, ok.hd, at, stream_of(first)));
    return py::make_tuple(yq, yk);
}

void kv_write(intptr_t handle, int device, const Tensor &k, const Tensor &v, const Tensor &table, const Opt &offsets,
              const std::optional<int64_t> &max_len, const Opt &pos, const Opt &slots) {
    const auto *c = reinterpret_cast<const sn_kv_cache *>(handle);
    const int dt = dtype_of(k.scalar_type(), "k and v");
    const Device on(k, device);
    on.same(v, "v"), on.same(table, "table"), on.same(offsets, "offsets"), on.same(pos, "pos"), on.same(slots, "slots");
    const Batch b = tokens_of(k, offsets, max_len, "k");
    const Heads hk = heads_of(k, c->head_dim, "k"), hv = heads_of(v, c->head_dim, "v", k.scalar_type());
    if (v.sizes() != k.sizes()) refuse("k and v have different shapes");
    if (hk.heads != c->heads) refuse("the cache has " + std::to_string(c->heads) + " heads, k " + std::to_string(hk.heads));
    if (!same_dtype(c, dt)) refuse("k and v have another type than the cache");
    const Table t = table_of(table, b.n, slots);
    const c10::cuda::CUDAGuard guard(k.device());
    check(sn_kv_write(c, dt, b.tokens, b.n, b.max_len, b.offsets, index_of(pos, b.n, "pos"), t.p, t.n, t.width,
                      index_of(slots, b.n, "slots"), hk.p, hk.ld, hk.hd, hv.p, hv.ld, hv.hd, stream_of(k)));
}

py::tuple kv_read(intptr_t handle, int device, const Tensor &table, const Opt &offsets, const std::optional<int64_t> &max_len,
                  const Opt &pos, const std::optional<int64_t> &tokens, const std::optional<at::ScalarType> &dtype, const Opt &slots,
                  const Opt &k_out, const Opt &v_out) {
    const auto *c = reinterpret_cast<const sn_kv_cache *>(handle);
    const Device on(table, device);
    on.same(offsets, "offsets"), on.same(pos, "pos"), on.same(slots, "slots"), on.same(k_out, "k_out"), on.same(v_out, "v_out");
    at::ScalarType type = c->dtype == SN_F32 ? at::kFloat : c->dtype == SN_F16 ? at::kHalf : at::kBFloat16;
    if (c->dtype == SN_QI8) {
        if (!dtype && !k_out) refuse("dtype is needed for a cache of codes");
        type = dtype ? *dtype : k_out->scalar_type();
    } else if (dtype && *dtype != type) {
        refuse("dtype is another than the cache's");
    }
    const int dt = dtype_of(type, "dtype");
    int64_t n, batch, longest;
    at::DimVector shape;
    if (offsets) {
        if (!max_len || !tokens) refuse("with offsets, max_len and tokens are needed");
        batch = offsets->numel() - 1, n = *tokens, longest = std::min(*max_len, n);
        if (batch < 0) refuse("offsets are empty");
        shape = {n, c->heads, c->head_dim};
    } else {
        if (!max_len) refuse("max_len, the tokens of every sequence, is needed");
        batch = pos ? pos->numel() : slots ? slots->numel() : table.dim() ? table.size(0) : 0;
        longest = *max_len, n = batch * longest;
        if (tokens && *tokens != n) refuse("without offsets there are sequences * max_len tokens");
        shape = {batch, longest, c->heads, c->head_dim};
    }
    if (batch > 65535) throw Fail{SN_EUNSUPPORTED, "more than 65535 sequences"};
    if (n < 0 || longest < 0) refuse("negative size");
    const int32_t *off = offsets ? index_of(offsets, batch + 1, "offsets") : nullptr;
    const Table t = table_of(table, batch, slots);
    const c10::cuda::CUDAGuard guard(table.device());
    Tensor k = output(k_out, shape, type, table, "k_out"), v = output(v_out, shape, type, table, "v_out");
    const Heads hk = heads_of(k, c->head_dim, "k_out"), hv = heads_of(v, c->head_dim, "v_out");
    check(sn_kv_read(c, dt, n, (int32_t)batch, longest, off, index_of(pos, batch, "pos"), t.p, t.n, t.width, index_of(slots, batch, "slots"),
                     hk.p, hk.ld, hk.hd, hv.p, hv.ld, hv.hd, stream_of(table)));
    return py::make_tuple(k, v);
}

Tensor attend(intptr_t handle, int device, const Tensor &q, const Tensor &table, const Opt &offsets, const std::optional<int64_t> &max_len,
              const Opt &pos, const std::optional<int64_t> &max_context, const std::optional<double> &scale, const Opt &slots, const Opt &out) {
    const auto *c = reinterpret_cast<const sn_kv_cache *>(handle);
    const int dt = dtype_of(q.scalar_type(), "q");
    const Device on(q, device);
    on.same(table, "table"), on.same(offsets, "offsets"), on.same(pos, "pos"), on.same(slots, "slots"), on.same(out, "out");
    const Batch b = tokens_of(q, offsets, max_len, "q");
    const Heads h = heads_of(q, c->head_dim, "q");
    if (h.heads > 65535) throw Fail{SN_EUNSUPPORTED, "more than 65535 heads"};
    if (!same_dtype(c, dt)) refuse("q has another type than the cache");
    const Table t = table_of(table, b.n, slots);
    const int64_t room = (int64_t)t.width * c->page;
    const int64_t context = max_context ? std::min(*max_context, room) : room;
    const float f = (float)(scale ? *scale : 1.0 / std::sqrt((double)c->head_dim));
    const c10::cuda::CUDAGuard guard(q.device());
    Tensor y = output_like(out, q, "out");
    const Heads o = heads_of(y, c->head_dim, "out");
    int64_t bytes = 0;
    check(sn_attend_workspace(c, dt, (int32_t)h.heads, b.tokens, b.n, b.max_len, context, &bytes));
    Tensor work;
    if (bytes) work = scratch(bytes, q);
    check(sn_attend(c, dt, (int32_t)h.heads, f, b.tokens, b.n, b.max_len, context, b.offsets, index_of(pos, b.n, "pos"), t.p, t.n, t.width,
                    index_of(slots, b.n, "slots"), h.p, h.ld, h.hd, o.p, o.ld, o.hd, bytes ? work.data_ptr() : nullptr, bytes, stream_of(q)));
    return y;
}

py::tuple verify_draft(const Tensor &target, const Opt &draft, const Opt &tokens, const Opt &accept, const Tensor &sample, const Opt &offsets,
                       const std::optional<int64_t> &max_len, const Opt &out, const Opt &count) {
    const int dt = dtype_of(target.scalar_type(), "target and draft");
    const Device on(target, -1);
    on.same(draft, "draft"), on.same(tokens, "tokens"), on.same(accept, "accept"), on.same(sample, "sample");
    on.same(offsets, "offsets"), on.same(out, "out"), on.same(count, "count");
    const int64_t batch = sample.numel(), drafts = tokens ? tokens->numel() : 0;
    if (batch > 65535) throw Fail{SN_EUNSUPPORTED, "more than 65535 sequences"};
    if (target.dim() < 2) refuse("target must be rows of probabilities, not shape " + shape_of(target));
    const int64_t vocab = target.size(target.dim() - 1);
    if (vocab > INT32_MAX) throw Fail{SN_EUNSUPPORTED, "vocab beyond 2^24"};
    int64_t longest;
    const int32_t *off = nullptr;
    if (offsets) {
        if (!max_len) refuse("with offsets, max_len is needed");
        longest = *max_len;
        off = index_of(offsets, batch + 1, "offsets");
    } else {
        longest = batch ? drafts / batch : 0;
        if (longest * batch != drafts || (max_len && *max_len != longest)) refuse("without offsets every sequence has max_len tokens");
    }
    if (longest < 0) refuse("negative max_len");
    const Rows rt = rows_of(target, vocab, "target");
    if (rt.n != drafts + batch) refuse("target must have a row more a sequence than there are tokens");
    Rows rd;
    const int32_t *x = nullptr;
    const float *u = nullptr;
    if (drafts) {
        if (!draft || !accept) refuse("draft and accept are needed");
        rd = rows_of(*draft, vocab, "draft", target.scalar_type());
        if (rd.n != drafts) refuse("draft must have a row of each token");
        if (accept->numel() != drafts) refuse("accept must have a number of each token");
        x = static_cast<const int32_t *>(whole(*tokens, tokens->sizes(), at::kInt, "tokens"));
        u = static_cast<const float *>(whole(*accept, accept->sizes(), at::kFloat, "accept"));
    }
    const auto *s = static_cast<const float *>(whole(sample, sample.sizes(), at::kFloat, "sample"));
    const c10::cuda::CUDAGuard guard(target.device());
    Tensor y = output(out, {batch, longest + 1}, at::kInt, target, "out"), n = output(count, {batch}, at::kInt, target, "count");
    check(sn_verify_draft(dt, (int32_t)vocab, drafts, (int32_t)batch, longest, off, rt.p, rt.ld, rd.p, rd.ld, x, u, s,
                          static_cast<int32_t *>(whole(y, y.sizes(), at::kInt, "out")),
                          static_cast<int32_t *>(whole(n, n.sizes(), at::kInt, "count")), stream_of(target)));
    return py::make_tuple(y, n);
}

}  // namespace

void bind_attention(py::module_ &m) {
    m.def("head_rope", &head_rope);
    m.def("kv_write", &kv_write);
    m.def("kv_read", &kv_read);
    m.def("attend", &attend);
    m.def("verify_draft", &verify_draft);
}
