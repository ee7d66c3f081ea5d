// Argument checks of the replica operators.
#include <exception>
#include <new>

#include "replica.hpp"

namespace arp {

ar_status check_dtype(const char* what, int32_t dtype, int32_t* esize) {
    switch (dtype) {
        case AR_F32: *esize = 4; return AR_OK;
        case AR_BF16: *esize = 2; return AR_OK;
        case AR_I32:
            return fail(AR_ERR_UNSUPPORTED, std::string(what) + " is AR_F32 or AR_BF16");
        default: return fail(AR_ERR_INVALID_ARG, std::string("unknown ") + what);
    }
}

ar_status check_extent(const char* what, int64_t v) {
    if (v < 0) return fail(AR_ERR_INVALID_ARG, std::string(what) + " must be >= 0");
    if (v > kMaxExtent)
        return fail(AR_ERR_UNSUPPORTED, std::string(what) + " exceeds 2^31 - 1");
    return AR_OK;
}

ar_status check_matrix(const MatArg& m) {
    if (m.rows == 0 || m.cols == 0) return AR_OK;
    const std::string name = m.name;
    if (!m.ptr) return fail(AR_ERR_INVALID_ARG, name + " is NULL");
    if (reinterpret_cast<uintptr_t>(m.ptr) % uintptr_t(m.esize))
        return fail(AR_ERR_INVALID_ARG, name + " is not aligned to its elements");
    if (m.stride < m.cols)
        return fail(AR_ERR_INVALID_ARG, name + ": the row stride is below the row's width");
    // the last byte's offset has to fit
    if (m.stride > (INT64_MAX / m.esize - m.cols) / m.rows)
        return fail(AR_ERR_INVALID_ARG, name + ": stride * rows overflows");
    return AR_OK;
}

ar_status check_apart(const MatArg& a, const MatArg& b) {
    if (!a.ptr || !b.ptr || a.rows == 0 || a.cols == 0 || b.rows == 0 || b.cols == 0)
        return AR_OK;
    const uint64_t pa = reinterpret_cast<uint64_t>(a.ptr), pb = reinterpret_cast<uint64_t>(b.ptr);
    const uint64_t sa = uint64_t(a.stride) * uint64_t(a.esize),
                   sb = uint64_t(b.stride) * uint64_t(b.esize);
    const uint64_t wa = uint64_t(a.cols) * uint64_t(a.esize),
                   wb = uint64_t(b.cols) * uint64_t(b.esize);
    const uint64_t ea = pa + uint64_t(a.rows - 1) * sa + wa,
                   eb = pb + uint64_t(b.rows - 1) * sb + wb;
    if (ea <= pb || eb <= pa) return AR_OK;
    // Columns of one wider matrix: with a common row stride the rows lie side
    // by side where the second begins behind the first's width and ends
    // before its next row.  One row has any stride.
    if (sa == sb || a.rows == 1 || b.rows == 1) {
        const uint64_t s = a.rows == 1 ? sb : sa;
        const uint64_t d = pb >= pa ? (pb - pa) % s : (s - (pa - pb) % s) % s;
        if (d >= wa && d + wb <= s) return AR_OK;
    }
    return fail(AR_ERR_INVALID_ARG, std::string(a.name) + " overlaps " + b.name);
}

ar_status check_workspace(const void* ws, int64_t have, int64_t need) {
    if (need == 0) return AR_OK;
    if (!ws || have < need)
        return fail(AR_ERR_INVALID_ARG,
                    "the call needs a workspace of " + std::to_string(need) + " bytes");
    if (reinterpret_cast<uintptr_t>(ws) % 16)
        return fail(AR_ERR_INVALID_ARG, "the workspace is not aligned to 16 bytes");
    return AR_OK;
}

ar_status launch_status(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return AR_OK;
    return fail(AR_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

ar_status thrown() noexcept {
    try {
        try {
            throw;
        } catch (const std::bad_alloc&) {
            return fail(AR_ERR_OOM, "host allocation failed");
        } catch (const std::exception& e) {
            return fail(AR_ERR_INTERNAL, e.what());
        }
    } catch (...) {
        return AR_ERR_OOM;  // nor is there memory for the text
    }
}

}  // namespace arp
