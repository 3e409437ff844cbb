// extern "C" boundary of the state-space block's operators (declared in
// include/sn.h): every argument is checked here, before anything is launched.
#include <new>
#include <string>

#include "sn_internal.h"

using namespace sn;

#define SN_GUARD(...)                                                    \
    try {                                                                \
        __VA_ARGS__                                                      \
    } catch (const std::bad_alloc &) {                                   \
        return fail(SN_ENOMEM, "host allocation failed");                \
    } catch (const std::exception &ex) {                                 \
        return fail(SN_EINVAL, std::string("internal error: ") + ex.what()); \
    } catch (...) {                                                      \
        return fail(SN_EINVAL, "internal error");                        \
    }
#define SN_NEED(cond, what) \
    if (!(cond)) return fail(SN_EINVAL, std::string(name) + ": " + what)

namespace {

constexpr int64_t kMaxRows = INT32_MAX;

bool float_type(int32_t dt) { return dt == SN_F32 || dt == SN_F16 || dt == SN_BF16; }
bool aligned(const void *p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

sn_status q4_sizes(const char *name, int64_t n, int64_t k, int32_t group) {
    SN_NEED(n >= 1 && k >= 1, "n and k must be positive");
    SN_NEED(group == 32 || group == 64 || group == 128, "group must be 32, 64 or 128");
    if (k > (1 << 24) || n > (1 << 26)) return fail(SN_EUNSUPPORTED, std::string(name) + ": k beyond 2^24 or n beyond 2^26");
    return SN_OK;
}

sn_status q4_weights(const char *name, const sn_q4_weights *w) {
    SN_NEED(w, "NULL weights");
    if (sn_status rc = q4_sizes(name, w->n, w->k, w->group)) return rc;
    SN_NEED(w->scale_dtype == SN_F16 || w->scale_dtype == SN_BF16, "scales must be fp16 or bf16");
    SN_NEED(w->act >= SN_ACT_NONE && w->act <= SN_ACT_HSIGMOID, "bad act");
    SN_NEED(w->packed && aligned(w->packed, 256), "packed must be device memory aligned to 256 bytes");
    SN_NEED(aligned(w->bias, 4), "misaligned bias");
    return SN_OK;
}

sn_status rows_of(const char *name, const void *p, int64_t stride, int64_t len, int32_t dt, const char *what) {
    SN_NEED(p, std::string("NULL ") + what);
    SN_NEED(stride >= len, std::string("the stride of ") + what + " is shorter than its rows");
    SN_NEED(aligned(p, dtype_size(dt)), std::string("misaligned ") + what);
    return SN_OK;
}

sn_status sequences(const char *name, int64_t tokens, int32_t batch, int64_t max_len, const int32_t *offsets,
                    int32_t n_slots, const int32_t *slots, const int32_t *pos) {
    SN_NEED(tokens >= 0 && batch >= 0 && max_len >= 0 && n_slots >= 0, "negative size");
    if (batch > 65535) return fail(SN_EUNSUPPORTED, std::string(name) + ": more than 65535 sequences");
    if (tokens > kMaxRows || max_len > kMaxRows) return fail(SN_EUNSUPPORTED, std::string(name) + ": more than 2^31 - 1 tokens");
    SN_NEED(max_len <= tokens || batch == 0 || tokens == 0, "max_len beyond the tokens there are");
    if (!offsets) SN_NEED((int64_t)batch * max_len == tokens, "without offsets there are batch * max_len tokens");
    SN_NEED(aligned(offsets, 4) && aligned(slots, 4) && aligned(pos, 4), "misaligned offsets, slots or pos");
    return SN_OK;
}

sn_status ssm(const char *name, const sn_ssm_params *p) {
    SN_NEED(p, "NULL parameters");
    SN_NEED(p->heads >= 1 && p->head_dim >= 1 && p->groups >= 1 && p->state >= 1, "sizes must be positive");
    SN_NEED(p->heads % p->groups == 0, "heads must be a multiple of groups");
    if (p->head_dim > 256 || p->state > 256 || p->heads > 65535)
        return fail(SN_EUNSUPPORTED, std::string(name) + ": head_dim and state go up to 256, heads up to 65535");
    SN_NEED(p->a, "NULL a");
    SN_NEED(aligned(p->a, 4) && aligned(p->d, 4) && aligned(p->dt_bias, 4), "misaligned weights");
    return SN_OK;
}
int64_t ssm_channels(const sn_ssm_params *p) {
    return (int64_t)p->heads * p->head_dim + 2LL * p->groups * p->state;
}

}  // namespace

extern "C" {

sn_status sn_q4_bytes(int32_t n, int32_t k, int32_t group, int64_t *bytes) {
    SN_GUARD({
        const char *name = "sn_q4_bytes";
        SN_NEED(bytes, "NULL argument");
        if (sn_status rc = q4_sizes(name, n, k, group)) return rc;
        *bytes = (int64_t)k::q4_bytes(n, k, group);
        return SN_OK;
    })
}

sn_status sn_q4_quantize(const void *w_dev, int32_t dtype, int32_t n, int32_t k, int32_t group, int32_t scale_dtype,
                         uint8_t *codes, void *scales, void *stream) {
    SN_GUARD({
        const char *name = "sn_q4_quantize";
        if (sn_status rc = q4_sizes(name, n, k, group)) return rc;
        SN_NEED(float_type(dtype), "bad dtype");
        SN_NEED(scale_dtype == SN_F16 || scale_dtype == SN_BF16, "scales must be fp16 or bf16");
        SN_NEED(w_dev && codes && scales, "NULL argument");
        SN_NEED(aligned(w_dev, dtype_size(dtype)) && aligned(scales, 2), "misaligned argument");
        SN_CUDA_TRY(k::q4_quantize(w_dev, dtype, n, k, group, scale_dtype, codes, scales, static_cast<cudaStream_t>(stream)));
        return SN_OK;
    })
}

sn_status sn_q4_pack(const uint8_t *codes, const void *scales, const sn_q4_weights *w, void *stream) {
    SN_GUARD({
        const char *name = "sn_q4_pack";
        if (sn_status rc = q4_weights(name, w)) return rc;
        SN_NEED(codes && scales && aligned(scales, 2), "NULL or misaligned codes or scales");
        SN_CUDA_TRY(k::q4_pack(codes, scales, *w, static_cast<cudaStream_t>(stream)));
        return SN_OK;
    })
}

sn_status sn_q4_workspace(const sn_q4_weights *w, int32_t dtype, int64_t rows, const void *x, int64_t x_stride,
                          int64_t *bytes) {
    SN_GUARD({
        const char *name = "sn_q4_workspace";
        if (sn_status rc = q4_weights(name, w)) return rc;
        SN_NEED(bytes && rows >= 0 && float_type(dtype), "bad argument");
        *bytes = rows ? (int64_t)k::q4_workspace(*w, dtype, rows, x, x_stride) : 0;
        return SN_OK;
    })
}

sn_status sn_q4_dense(const sn_q4_weights *w, int32_t dtype, int64_t rows, const void *x, int64_t x_stride, void *y,
                      int64_t y_stride, void *work, int64_t work_bytes, void *stream) {
    SN_GUARD({
        const char *name = "sn_q4_dense";
        if (sn_status rc = q4_weights(name, w)) return rc;
        SN_NEED(float_type(dtype), "bad dtype");
        SN_NEED(rows >= 0, "negative rows");
        if (rows == 0) return SN_OK;
        if (rows > kMaxRows) return fail(SN_EUNSUPPORTED, "sn_q4_dense: more than 2^31 - 1 rows");
        if (sn_status rc = rows_of(name, x, x_stride, w->k, dtype, "x")) return rc;
        if (sn_status rc = rows_of(name, y, y_stride, w->n, dtype, "y")) return rc;
        SN_NEED(y != x, "y over x");
        const int64_t need = (int64_t)k::q4_workspace(*w, dtype, rows, x, x_stride);
        SN_NEED(need == 0 || (work && aligned(work, 256) && work_bytes >= need),
                "needs " + std::to_string(need) + " bytes of scratch aligned to 256 (sn_q4_workspace)");
        SN_CUDA_TRY(k::q4_dense(*w, dtype, rows, x, x_stride, y, y_stride, work, static_cast<cudaStream_t>(stream)));
        return SN_OK;
    })
}

sn_status sn_block_norm(const sn_norm_params *p, int32_t dtype, int64_t rows, const void *y, int64_t y_stride,
                        const void *gate, int64_t gate_stride, int64_t rows_per_gate, int32_t res_dtype,
                        const void *residual, int64_t residual_stride, void *sum_out, int64_t sum_stride, void *normed,
                        int64_t normed_stride, void *stream) {
    SN_GUARD({
        const char *name = "sn_block_norm";
        SN_NEED(p, "NULL parameters");
        SN_NEED(p->dim >= 1, "dim must be positive");
        if (p->dim > (1 << 28)) return fail(SN_EUNSUPPORTED, "sn_block_norm: dim beyond 2^28");
        SN_NEED(p->kind == SN_NORM_RMS || p->kind == SN_NORM_LAYER, "bad kind");
        SN_NEED(p->gate >= SN_GATE_NONE && p->gate <= SN_GATE_SILU, "bad gate");
        SN_NEED(p->gate_after == 0 || p->gate_after == 1, "gate_after is 0 or 1");
        SN_NEED(p->eps >= 0.0f && p->eps < 1e30f, "bad eps");
        SN_NEED(aligned(p->post, 4) && aligned(p->post_bias, 4) && aligned(p->pre, 4) && aligned(p->pre_bias, 4) &&
                    aligned(p->scale, 4), "misaligned weights");
        SN_NEED((p->post || !p->post_bias) && (p->pre || !p->pre_bias), "a norm's bias without its weight");
        SN_NEED(float_type(dtype), "bad dtype");
        SN_NEED(rows >= 0, "negative rows");
        if (rows == 0) return SN_OK;
        SN_NEED(!residual || res_dtype == dtype || res_dtype == SN_F32, "the residual has the rows' dtype or fp32");
        SN_NEED((p->gate != SN_GATE_NONE) == (gate != nullptr), "a gate tensor goes with a gate option");
        SN_NEED(y || !gate, "a gate without y");
        SN_NEED(!gate || rows_per_gate >= 1, "rows_per_gate must be positive");
        SN_NEED((p->pre != nullptr) == (normed != nullptr), "normed goes with pre weights");
        SN_NEED(y || residual, "neither y nor residual");
        SN_NEED(sum_out || normed, "no output");
        if (rows > kMaxRows) return fail(SN_EUNSUPPORTED, "sn_block_norm: more than 2^31 - 1 rows");
        const int32_t sum_dt = residual ? res_dtype : dtype;
        if (y) if (sn_status rc = rows_of(name, y, y_stride, p->dim, dtype, "y")) return rc;
        if (gate) if (sn_status rc = rows_of(name, gate, gate_stride, p->dim, dtype, "gate")) return rc;
        if (residual) if (sn_status rc = rows_of(name, residual, residual_stride, p->dim, res_dtype, "residual")) return rc;
        if (sum_out) if (sn_status rc = rows_of(name, sum_out, sum_stride, p->dim, sum_dt, "sum_out")) return rc;
        if (normed) if (sn_status rc = rows_of(name, normed, normed_stride, p->dim, dtype, "normed")) return rc;
        SN_NEED(sum_out != normed, "sum_out and normed are the same");
        SN_NEED(!sum_out || sum_out != y || (sum_dt == dtype && sum_stride == y_stride), "sum_out over y needs its type and stride");
        SN_NEED(!sum_out || sum_out != residual || sum_stride == residual_stride, "sum_out over residual needs its stride");
        SN_NEED(!normed || normed != y || normed_stride == y_stride, "normed over y needs its stride");
        SN_NEED(!normed || (normed != residual && normed != gate), "normed over residual or gate");
        SN_NEED(!sum_out || sum_out != gate, "sum_out over gate");
        k::NormArgs a{y, gate, residual, sum_out, normed, rows, y_stride, gate_stride, gate ? rows_per_gate : 1,
                      residual_stride, sum_stride, normed_stride};
        SN_CUDA_TRY(k::block_norm(*p, dtype, res_dtype, a, static_cast<cudaStream_t>(stream)));
        return SN_OK;
    })
}

sn_status sn_causal_conv(int32_t dtype, int32_t channels, int32_t width, int32_t silu, const float *weight,
                         const float *bias, int64_t tokens, int32_t batch, int64_t max_len, const int32_t *offsets,
                         const void *x, int64_t x_stride, void *y, int64_t y_stride, void *kept, int32_t n_slots,
                         const int32_t *slots, const int32_t *pos, void *stream) {
    SN_GUARD({
        const char *name = "sn_causal_conv";
        SN_NEED(float_type(dtype), "bad dtype");
        SN_NEED(channels >= 1 && width >= 1, "channels and width must be positive");
        if (width > 8 || channels > (1 << 28)) return fail(SN_EUNSUPPORTED, "sn_causal_conv: width goes up to 8, channels to 2^28");
        SN_NEED(silu == 0 || silu == 1, "silu is 0 or 1");
        if (sn_status rc = sequences(name, tokens, batch, max_len, offsets, n_slots, slots, pos)) return rc;
        SN_NEED(weight && aligned(weight, 4) && aligned(bias, 4), "NULL or misaligned weights");
        SN_NEED(!kept || n_slots >= 1 || batch == 0, "kept without entries");
        SN_NEED(aligned(kept, dtype_size(dtype)), "misaligned kept");
        if (batch == 0 || max_len == 0) return SN_OK;
        if (sn_status rc = rows_of(name, x, x_stride, channels, dtype, "x")) return rc;
        if (sn_status rc = rows_of(name, y, y_stride, channels, dtype, "y")) return rc;
        SN_NEED(x != y, "y over x");
        const k::SeqArgs q{tokens, max_len, batch, n_slots, offsets, slots, pos};
        SN_CUDA_TRY(k::causal_conv(dtype, channels, width, silu, weight, bias, q, x, x_stride, y, y_stride, kept,
                                   static_cast<cudaStream_t>(stream)));
        return SN_OK;
    })
}

sn_status sn_ssm_workspace(const sn_ssm_params *p, int32_t dtype, int64_t tokens, int32_t batch, int64_t max_len,
                           int64_t *bytes) {
    SN_GUARD({
        const char *name = "sn_ssm_workspace";
        if (sn_status rc = ssm(name, p)) return rc;
        SN_NEED(bytes && float_type(dtype) && tokens >= 0 && batch >= 0 && max_len >= 0, "bad argument");
        const k::SeqArgs q{tokens, max_len, batch, 0, nullptr, nullptr, nullptr};
        *bytes = tokens && batch ? (int64_t)k::ssm_workspace(*p, dtype, q) : 0;
        return SN_OK;
    })
}

sn_status sn_ssm_scan(const sn_ssm_params *p, int32_t dtype, int64_t tokens, int32_t batch, int64_t max_len,
                      const int32_t *offsets, const void *xbc, int64_t xbc_stride, const void *dt, int64_t dt_stride,
                      const float *state_in, float *state_out, int32_t n_slots, const int32_t *slots, void *y,
                      int64_t y_stride, void *work, int64_t work_bytes, void *stream) {
    SN_GUARD({
        const char *name = "sn_ssm_scan";
        if (sn_status rc = ssm(name, p)) return rc;
        SN_NEED(float_type(dtype), "bad dtype");
        if (sn_status rc = sequences(name, tokens, batch, max_len, offsets, n_slots, slots, nullptr)) return rc;
        SN_NEED((!state_in && !state_out) || n_slots >= 1 || batch == 0, "states without entries");
        SN_NEED(aligned(state_in, 4) && aligned(state_out, 4), "misaligned states");
        if (batch == 0) return SN_OK;
        if (tokens > 0) {
            if (sn_status rc = rows_of(name, xbc, xbc_stride, ssm_channels(p), dtype, "xbc")) return rc;
            if (sn_status rc = rows_of(name, dt, dt_stride, p->heads, dtype, "dt")) return rc;
            if (sn_status rc = rows_of(name, y, y_stride, (int64_t)p->heads * p->head_dim, dtype, "y")) return rc;
            SN_NEED(y != xbc && y != dt, "y over an input");
        }
        const k::SeqArgs q{tokens, max_len, batch, n_slots, offsets, slots, nullptr};
        const int64_t need = tokens ? (int64_t)k::ssm_workspace(*p, dtype, q) : 0;
        SN_NEED(need == 0 || (work && aligned(work, 256) && work_bytes >= need),
                "needs " + std::to_string(need) + " bytes of scratch aligned to 256 (sn_ssm_workspace)");
        SN_CUDA_TRY(k::ssm_scan(*p, dtype, q, xbc, xbc_stride, dt, dt_stride, state_in, state_out, y, y_stride, work,
                                static_cast<cudaStream_t>(stream)));
        return SN_OK;
    })
}

sn_status sn_ssm_step(const sn_ssm_params *p, int32_t dtype, int32_t batch, const void *xbc, int64_t xbc_stride,
                      const void *dt, int64_t dt_stride, void *kept, const float *state_in, float *state_out,
                      int32_t n_slots, const int32_t *slots, const int32_t *pos, void *y, int64_t y_stride, void *stream) {
    SN_GUARD({
        const char *name = "sn_ssm_step";
        if (sn_status rc = ssm(name, p)) return rc;
        SN_NEED(float_type(dtype), "bad dtype");
        SN_NEED(p->width >= 1, "width must be positive");
        if (p->width > 8) return fail(SN_EUNSUPPORTED, "sn_ssm_step: width goes up to 8");
        SN_NEED(p->conv_w && aligned(p->conv_w, 4) && aligned(p->conv_b, 4), "NULL or misaligned convolution weights");
        if (sn_status rc = sequences(name, batch, batch, 1, nullptr, n_slots, slots, pos)) return rc;
        if (batch == 0) return SN_OK;
        if (sn_status rc = rows_of(name, xbc, xbc_stride, ssm_channels(p), dtype, "xbc")) return rc;
        if (sn_status rc = rows_of(name, dt, dt_stride, p->heads, dtype, "dt")) return rc;
        if (sn_status rc = rows_of(name, y, y_stride, (int64_t)p->heads * p->head_dim, dtype, "y")) return rc;
        SN_NEED(y != xbc && y != dt, "y over an input");
        SN_NEED(kept && state_out && n_slots >= 1, "kept and state_out are needed");
        SN_NEED(aligned(kept, dtype_size(dtype)) && aligned(state_in, 4) && aligned(state_out, 4), "misaligned kept or states");
        const k::SeqArgs q{batch, 1, batch, n_slots, nullptr, slots, pos};
        SN_CUDA_TRY(k::ssm_step(*p, dtype, q, xbc, xbc_stride, dt, dt_stride, kept, state_in, state_out, y, y_stride,
                                static_cast<cudaStream_t>(stream)));
        return SN_OK;
    })
}

sn_status sn_check_device(void *stream) {
    SN_GUARD({
        SN_CUDA_TRY(cudaStreamSynchronize(static_cast<cudaStream_t>(stream)));
        int word = 0;
        SN_CUDA_TRY(cudaMemcpy(&word, k::device_error_word(), sizeof(int), cudaMemcpyDeviceToHost));
        if (!word) return SN_OK;
        const int zero = 0;
        SN_CUDA_TRY(cudaMemcpy(k::device_error_word(), &zero, sizeof(int), cudaMemcpyHostToDevice));
        return fail(SN_ETIMEOUT, "device error word set: " + std::to_string(word) + " (a bounded wait in a kernel gave up)");
    })
}

}  // extern "C"
