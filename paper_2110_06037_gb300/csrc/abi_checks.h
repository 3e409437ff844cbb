// Checks that the C entries of the block and attention operators share.
#pragma once

#include <new>
#include <string>

#include "sn_internal.h"

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

namespace sn {

constexpr int64_t kMaxRows = INT32_MAX;

inline bool float_type(int32_t dt) { return dt == SN_F32 || dt == SN_F16 || dt == SN_BF16; }
inline bool aligned(const void *p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

inline sn_status rows_of(const char *name, const void *p, int64_t stride, int64_t len, int32_t dt, const char *what) {
    SN_NEED(p, std::string("NULL ") + what);
    SN_NEED(stride >= len, std::string("the stride of ") + what + " is shorter than its rows");
    SN_NEED(aligned(p, dtype_size(dt)), std::string("misaligned ") + what);
    return SN_OK;
}

inline sn_status sequences(const char *name, int64_t tokens, int32_t batch, int64_t max_len, const int32_t *offsets,
                    int32_t n_slots, const int32_t *slots, const int32_t *pos) {
    SN_NEED(tokens >= 0 && batch >= 0 && max_len >= 0 && n_slots >= 0, "negative size");
    if (batch > 65535) return fail(SN_EUNSUPPORTED, std::string(name) + ": more than 65535 sequences");
    if (tokens > kMaxRows || max_len > kMaxRows) return fail(SN_EUNSUPPORTED, std::string(name) + ": more than 2^31 - 1 tokens");
    SN_NEED(max_len <= tokens || batch == 0 || tokens == 0, "max_len beyond the tokens there are");
    if (!offsets) SN_NEED((int64_t)batch * max_len == tokens, "without offsets there are batch * max_len tokens");
    SN_NEED(aligned(offsets, 4) && aligned(slots, 4) && aligned(pos, 4), "misaligned offsets, slots or pos");
    return SN_OK;
}

}  // namespace sn
