// extern "C" boundary of the attention layer's operators (declared in include/sn.h):
// every argument is checked here, before anything is launched.
#include <cmath>

#include "abi_checks.h"

using namespace sn;

namespace {

// the heads of a tensor's tokens: apart from one another
sn_status heads_of(const char *name, const void *p, int64_t tokens, int64_t heads, int64_t stride, int64_t head_stride, int64_t dim,
                   int32_t dt, const char *what) {
    SN_NEED(p, std::string("NULL ") + what);
    SN_NEED(aligned(p, dtype_size(dt)), std::string("misaligned ") + what);
    const int64_t most = int64_t{1} << 40;
    SN_NEED(stride >= 0 && head_stride >= 0 && stride <= most && head_stride <= most, std::string("bad strides of ") + what);
    const bool t = tokens > 1, h = heads > 1;
    SN_NEED((!t || stride >= dim) && (!h || head_stride >= dim) &&
                (!t || !h || stride >= (heads - 1) * head_stride + dim || head_stride >= (tokens - 1) * stride + dim),
            std::string("the heads of ") + what + " lie on one another");
    return SN_OK;
}
sn_status cache_of(const char *name, const sn_kv_cache *c) {
    SN_NEED(c, "NULL cache");
    SN_NEED(float_type(c->dtype) || c->dtype == SN_QI8, "bad dtype of the cache");
    SN_NEED(c->pages >= 1 && c->heads >= 1 && c->head_dim >= 1, "sizes must be positive");
    SN_NEED(c->page == 16 || c->page == 32 || c->page == 64 || c->page == 128 || c->page == 256,
            "a page has 16, 32, 64, 128 or 256 tokens");
    if (c->head_dim % 16 || c->head_dim > 256)
        return fail(SN_EUNSUPPORTED, std::string(name) + ": head_dim must be a multiple of 16 up to 256");
    if (c->heads > 65535) return fail(SN_EUNSUPPORTED, std::string(name) + ": more than 65535 heads");
    SN_NEED(c->k && c->v && aligned(c->k, 16) && aligned(c->v, 16), "NULL or misaligned keys or values");
    if (c->dtype == SN_QI8) {
        SN_NEED(c->k_scale && c->v_scale && aligned(c->k_scale, 16) && aligned(c->v_scale, 16), "NULL or misaligned scales");
    } else {
        SN_NEED(!c->k_scale && !c->v_scale, "scales without codes");
    }
    return SN_OK;
}

sn_status table_of(const char *name, const int32_t *table, int32_t n_slots, int32_t width, int32_t batch, const int32_t *slots) {
    SN_NEED(width >= 0 && n_slots >= 0, "negative size");
    SN_NEED(aligned(table, 4), "misaligned table");
    SN_NEED(table || width == 0 || n_slots == 0, "NULL table");
    SN_NEED(slots || n_slots >= batch, "fewer entries of the table than sequences");
    return SN_OK;
}

sn_status kv(const char *name, bool write, const sn_kv_cache *c, int32_t dtype, int64_t tokens, int32_t batch, int64_t max_len,
             const int32_t *offsets, const int32_t *pos, const int32_t *table, int32_t n_slots, int32_t width, const int32_t *slots,
             const void *k, int64_t k_stride, int64_t k_head_stride, const void *v, int64_t v_stride, int64_t v_head_stride,
             void *stream) {
    if (sn_status rc = cache_of(name, c)) return rc;
    SN_NEED(float_type(dtype) && (c->dtype == SN_QI8 || c->dtype == dtype), "the tokens' dtype is the cache's, or any where it holds codes");
    if (sn_status rc = sequences(name, tokens, batch, max_len, offsets, n_slots, slots, pos)) return rc;
    if (sn_status rc = table_of(name, table, n_slots, width, batch, slots)) return rc;
    if (tokens == 0 || batch == 0) return SN_OK;
    const int64_t d = c->head_dim;
    if (sn_status rc = heads_of(name, k, tokens, c->heads, k_stride, k_head_stride, d, dtype, "k")) return rc;
    if (sn_status rc = heads_of(name, v, tokens, c->heads, v_stride, v_head_stride, d, dtype, "v")) return rc;
    if (!write) SN_NEED(k != v, "v over k");
    const k::SeqArgs q{tokens, max_len, batch, n_slots, offsets, slots, pos};
    const k::TableArgs t{table, table ? width : 0};
    const k::HeadsArgs hk{c->heads, k, k_stride, k_head_stride, const_cast<void *>(k), k_stride, k_head_stride, nullptr};
    const k::HeadsArgs hv{c->heads, v, v_stride, v_head_stride, const_cast<void *>(v), v_stride, v_head_stride, nullptr};
    const auto st = static_cast<cudaStream_t>(stream);
    if (write) SN_CUDA_TRY(k::kv_write(*c, dtype, q, t, hk, hv, st));
    else SN_CUDA_TRY(k::kv_read(*c, dtype, q, t, hk, hv, st));
    return SN_OK;
}

sn_status attend_sizes(const char *name, const sn_kv_cache *c, int32_t dtype, int32_t q_heads, int64_t max_context) {
    if (sn_status rc = cache_of(name, c)) return rc;
    SN_NEED(float_type(dtype) && (c->dtype == SN_QI8 || c->dtype == dtype), "the queries' dtype is the cache's, or any where it holds codes");
    SN_NEED(q_heads >= 1 && q_heads % c->heads == 0, "q_heads must be a multiple of the cache's heads");
    if (q_heads > 65535) return fail(SN_EUNSUPPORTED, std::string(name) + ": more than 65535 heads");
    SN_NEED(max_context >= 0, "negative max_context");
    return SN_OK;
}
int64_t context_of(int64_t max_context) { return max_context < INT32_MAX ? max_context : INT32_MAX; }

}  // namespace

extern "C" {

sn_status sn_rope_turns(const double *radians, int32_t n, uint64_t *turns) {
    SN_GUARD({
        const char *name = "sn_rope_turns";
        SN_NEED(n >= 0 && (n == 0 || (radians && turns)), "NULL argument or negative size");
        for (int32_t i = 0; i < n; ++i)
            SN_NEED(std::isfinite(radians[i]) && std::fabs(radians[i]) <= 1048576.0, "an angle beyond 2^20 or not finite");
        for (int32_t i = 0; i < n; ++i) {
            // 1 / 2 pi in two parts (off by less than 2^-108 of it), so that a turn's fraction is good to 64 bits
            // for angles of up to a few turns
            constexpr double hi = 0.15915494309189535, lo = -9.839338337591243e-18;
            const double a = std::fabs(radians[i]);
            const volatile double rounded = a * hi;  // (never part of a fused operation)
            const double p = rounded, e = std::fma(a, hi, -p) + a * lo;
            const double whole = std::floor(p), f = p - whole;  // exact
            const double top = std::floor(f * 4294967296.0), rest = (f * 4294967296.0 - top) * 4294967296.0 + e * 18446744073709551616.0;
            const double carry = std::floor(rest / 4294967296.0);
            const uint64_t t = ((uint64_t)(int64_t)(top + carry) << 32) + (uint64_t)(rest - carry * 4294967296.0);
            turns[i] = radians[i] < 0.0 ? 0 - t : t;
        }
        return SN_OK;
    })
}

sn_status sn_head_rope(const sn_rope_params *p, int32_t dtype, int64_t tokens, int32_t q_heads, const void *q, int64_t q_stride,
                       int64_t q_head_stride, void *q_out, int64_t q_out_stride, int64_t q_out_head_stride, int32_t k_heads,
                       const void *k, int64_t k_stride, int64_t k_head_stride, void *k_out, int64_t k_out_stride,
                       int64_t k_out_head_stride, const int32_t *pos, void *stream) {
    SN_GUARD({
        const char *name = "sn_head_rope";
        SN_NEED(p, "NULL parameters");
        SN_NEED(p->head_dim >= 2 && p->head_dim % 2 == 0, "head_dim must be even and positive");
        if (p->head_dim > 256) return fail(SN_EUNSUPPORTED, "sn_head_rope: head_dim beyond 256");
        SN_NEED(p->pairs >= 0 && p->pairs <= p->head_dim / 2, "pairs must be at most half of head_dim");
        SN_NEED(p->axes >= 1 && p->axes <= 65536, "bad number of axes");
        SN_NEED(p->norm == SN_HEADS_RMS || p->norm == SN_HEADS_LAYER || p->norm == SN_HEADS_NONE, "bad norm");
        SN_NEED(p->interleaved == 0 || p->interleaved == 1, "interleaved is 0 or 1");
        SN_NEED(p->eps >= 0.0f && p->eps < 1e30f, "bad eps");
        SN_NEED(p->pairs == 0 || p->turns, "NULL turns");
        SN_NEED(aligned(p->turns, 8) && aligned(p->axis, 4) && aligned(pos, 4) && aligned(p->q_weight, 4) && aligned(p->k_weight, 4),
                "misaligned turns, axis, pos or weights");
        SN_NEED(p->norm != SN_HEADS_NONE || (!p->q_weight && !p->k_weight), "weights without a norm");
        SN_NEED(float_type(dtype), "bad dtype");
        SN_NEED(tokens >= 0 && q_heads >= 0 && k_heads >= 0, "negative size");
        if (tokens == 0 || (q_heads == 0 && k_heads == 0)) return SN_OK;
        SN_NEED(p->pairs == 0 || pos, "NULL pos");
        if (tokens > kMaxRows) return fail(SN_EUNSUPPORTED, "sn_head_rope: more than 2^31 - 1 tokens");
        if (q_heads > 65535 || k_heads > 65535) return fail(SN_EUNSUPPORTED, "sn_head_rope: more than 65535 heads");
        const int64_t d = p->head_dim;
        k::HeadsArgs h[2] = {{q_heads, q, q_stride, q_head_stride, q_out, q_out_stride, q_out_head_stride, p->q_weight},
                             {k_heads, k, k_stride, k_head_stride, k_out, k_out_stride, k_out_head_stride, p->k_weight}};
        const char *in[2] = {"q", "k"}, *out[2] = {"q_out", "k_out"};
        for (int i = 0; i < 2; ++i) {
            if (h[i].heads == 0) continue;
            if (sn_status rc = heads_of(name, h[i].x, tokens, h[i].heads, h[i].ldx, h[i].hx, d, dtype, in[i])) return rc;
            if (sn_status rc = heads_of(name, h[i].y, tokens, h[i].heads, h[i].ldy, h[i].hy, d, dtype, out[i])) return rc;
            SN_NEED(h[i].y != h[i].x || ((tokens == 1 || h[i].ldx == h[i].ldy) && (h[i].heads == 1 || h[i].hx == h[i].hy)),
                    std::string(out[i]) + " over " + in[i] + " needs its strides");
        }
        if (q_heads && k_heads) {
            SN_NEED(q_out != k_out, "k_out over q_out");
            SN_NEED(q_out != k && k_out != q, "an output over the other input");
        }
        SN_CUDA_TRY(k::head_rope(*p, dtype, tokens, h[0], h[1], pos, static_cast<cudaStream_t>(stream)));
        return SN_OK;
    })
}

sn_status sn_kv_write(const sn_kv_cache *c, int32_t dtype, int64_t tokens, int32_t batch, int64_t max_len, const int32_t *offsets,
                      const int32_t *pos, const int32_t *table, int32_t n_slots, int32_t width, const int32_t *slots, const void *k,
                      int64_t k_stride, int64_t k_head_stride, const void *v, int64_t v_stride, int64_t v_head_stride, void *stream) {
    SN_GUARD({
        return kv("sn_kv_write", true, c, dtype, tokens, batch, max_len, offsets, pos, table, n_slots, width, slots, k, k_stride,
                  k_head_stride, v, v_stride, v_head_stride, stream);
    })
}

sn_status sn_kv_read(const sn_kv_cache *c, int32_t dtype, int64_t tokens, int32_t batch, int64_t max_len, const int32_t *offsets,
                     const int32_t *pos, const int32_t *table, int32_t n_slots, int32_t width, const int32_t *slots, void *k,
                     int64_t k_stride, int64_t k_head_stride, void *v, int64_t v_stride, int64_t v_head_stride, void *stream) {
    SN_GUARD({
        return kv("sn_kv_read", false, c, dtype, tokens, batch, max_len, offsets, pos, table, n_slots, width, slots, k, k_stride,
                  k_head_stride, v, v_stride, v_head_stride, stream);
    })
}

sn_status sn_attend_workspace(const sn_kv_cache *c, int32_t dtype, int32_t q_heads, int64_t tokens, int32_t batch, int64_t max_len,
                              int64_t max_context, int64_t *bytes) {
    SN_GUARD({
        const char *name = "sn_attend_workspace";
        if (sn_status rc = attend_sizes(name, c, dtype, q_heads, max_context)) return rc;
        SN_NEED(bytes, "NULL bytes");
        SN_NEED(tokens >= 0 && batch >= 0 && max_len >= 0, "negative size");
        if (batch > 65535) return fail(SN_EUNSUPPORTED, "sn_attend_workspace: more than 65535 sequences");
        if (tokens > kMaxRows || max_len > kMaxRows) return fail(SN_EUNSUPPORTED, "sn_attend_workspace: more than 2^31 - 1 tokens");
        k::AttendArgs a{};
        a.q.tokens = tokens, a.q.batch = batch, a.q.max_len = max_len;
        a.max_context = context_of(max_context);
        a.h.heads = q_heads;
        *bytes = tokens && batch ? (int64_t)k::attend_workspace(*c, dtype, a) : 0;
        return SN_OK;
    })
}

sn_status sn_attend(const sn_kv_cache *c, int32_t dtype, int32_t q_heads, float scale, int64_t tokens, int32_t batch, int64_t max_len,
                    int64_t max_context, const int32_t *offsets, const int32_t *pos, const int32_t *table, int32_t n_slots,
                    int32_t width, const int32_t *slots, const void *q, int64_t q_stride, int64_t q_head_stride, void *y,
                    int64_t y_stride, int64_t y_head_stride, void *work, int64_t work_bytes, void *stream) {
    SN_GUARD({
        const char *name = "sn_attend";
        if (sn_status rc = attend_sizes(name, c, dtype, q_heads, max_context)) return rc;
        SN_NEED(std::isfinite(scale), "scale is not finite");
        if (sn_status rc = sequences(name, tokens, batch, max_len, offsets, n_slots, slots, pos)) return rc;
        if (sn_status rc = table_of(name, table, n_slots, width, batch, slots)) return rc;
        if (tokens == 0 || batch == 0) return SN_OK;
        const int64_t d = c->head_dim;
        if (sn_status rc = heads_of(name, q, tokens, q_heads, q_stride, q_head_stride, d, dtype, "q")) return rc;
        if (sn_status rc = heads_of(name, y, tokens, q_heads, y_stride, y_head_stride, d, dtype, "y")) return rc;
        SN_NEED(y != q, "y over q");
        const k::AttendArgs a{{tokens, max_len, batch, n_slots, offsets, slots, pos}, {table, table ? width : 0}, context_of(max_context),
                              scale, {q_heads, q, q_stride, q_head_stride, y, y_stride, y_head_stride, nullptr}};
        const int64_t need = (int64_t)k::attend_workspace(*c, dtype, a);
        SN_NEED(need == 0 || (work && aligned(work, 256) && work_bytes >= need),
                "needs " + std::to_string(need) + " bytes of scratch aligned to 256 (sn_attend_workspace)");
        SN_CUDA_TRY(k::attend(*c, dtype, a, work, static_cast<cudaStream_t>(stream)));
        return SN_OK;
    })
}

sn_status sn_verify_draft(int32_t dtype, int32_t vocab, int64_t tokens, int32_t batch, int64_t max_len, const int32_t *offsets,
                          const void *target, int64_t target_stride, const void *draft, int64_t draft_stride, const int32_t *drafted,
                          const float *accept, const float *sample, int32_t *out, int32_t *count, void *stream) {
    SN_GUARD({
        const char *name = "sn_verify_draft";
        SN_NEED(float_type(dtype), "bad dtype");
        SN_NEED(vocab >= 1, "vocab must be positive");
        if (vocab > (1 << 24)) return fail(SN_EUNSUPPORTED, "sn_verify_draft: vocab beyond 2^24");
        SN_NEED(tokens >= 0 && batch >= 0 && max_len >= 0, "negative size");
        if (batch > 65535) return fail(SN_EUNSUPPORTED, "sn_verify_draft: more than 65535 sequences");
        if (tokens > kMaxRows - 65536 || max_len > kMaxRows - 65536) return fail(SN_EUNSUPPORTED, "sn_verify_draft: more than 2^31 - 2^16 - 1 tokens");
        if (!offsets) SN_NEED((int64_t)batch * max_len == tokens, "without offsets there are batch * max_len tokens");
        if (batch == 0) return SN_OK;
        if (sn_status rc = rows_of(name, target, target_stride, vocab, dtype, "target")) return rc;
        if (tokens) {
            if (sn_status rc = rows_of(name, draft, draft_stride, vocab, dtype, "draft")) return rc;
            SN_NEED(drafted && accept && aligned(drafted, 4) && aligned(accept, 4), "NULL or misaligned drafted tokens or accept");
        }
        SN_NEED(sample && out && count, "NULL sample, out or count");
        SN_NEED(aligned(offsets, 4) && aligned(sample, 4) && aligned(out, 4) && aligned(count, 4), "misaligned argument");
        SN_NEED(out != count && (!drafted || (out != drafted && count != drafted)), "outputs over one another or over the drafted tokens");
        const k::VerifyArgs a{{tokens, max_len, batch, 0, offsets, nullptr, nullptr}, target, tokens ? draft : nullptr, target_stride,
                              tokens ? draft_stride : 0, drafted, accept, sample, out, count};
        SN_CUDA_TRY(k::verify_draft(dtype, vocab, a, static_cast<cudaStream_t>(stream)));
        return SN_OK;
    })
}

}  // extern "C"
