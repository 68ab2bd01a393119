// abi_checks.h -- checks of arguments that the entry points of sequence operators
// share; each raises the error that the call returns.
#pragma once
#include <climits>

#include "../../include/tq_seq.h"
#include "abi_util.h"

namespace tq {

constexpr int64_t kMaxIndex = INT32_MAX;
constexpr int64_t kMaxWidth = 1 << 20;

inline std::string text(const char *call, const char *what) { return std::string(call) + ": " + what; }

inline void check_type(const char *call, int type)
{
    if (type != TQ_F32 && type != TQ_BF16 && type != TQ_F16) fail(TQ_E_INVALID, text(call, "unknown type"));
}

inline size_t size_of(int type) { return type == TQ_F32 ? 4 : 2; }

inline void check_size(const char *call, const char *name, int64_t n)
{
    if (n < 0) fail(TQ_E_INVALID, text(call, name) + " must not be negative");
    if (n > kMaxIndex) fail(TQ_E_UNSUPPORTED, text(call, name) + " must be below 2^31");
}

inline void check_array(const char *call, const char *name, const void *p, size_t align)
{
    if (!p) fail(TQ_E_INVALID, text(call, name) + " is NULL");
    check_align(p, align, name);
}

inline void check_maybe(const char *name, const void *p, size_t align)
{
    if (p) check_align(p, align, name);
}

inline void check_ld(const char *call, const char *name, int64_t ld, int64_t D)
{
    if (ld < D) fail(TQ_E_INVALID, text(call, name) + " is shorter than a row");
}

// Rows of an output must not fall on one another: step and batch strides that
// keep B x T rows of D elements apart.
inline void check_strides(const char *call, const char *name, int64_t B, int64_t T, int64_t D, int64_t batch, int64_t step,
                          bool out)
{
    if (batch < 0 || step < 0) fail(TQ_E_INVALID, text(call, name) + " strides must not be negative");
    if (!out) return;
    const bool steps_inside = (T <= 1 || step >= D) && (B <= 1 || batch >= (T > 1 ? (T - 1) * step : 0) + D);
    const bool batch_inside = (B <= 1 || batch >= D) && (T <= 1 || step >= (B > 1 ? (B - 1) * batch : 0) + D);
    if (!steps_inside && !batch_inside) fail(TQ_E_INVALID, text(call, name) + " strides make rows overlap");
}

inline void check_space(const char *call, const void *ws, size_t have, size_t need)
{
    if (need == 0) return;
    if (!ws) fail(TQ_E_INVALID, text(call, "workspace is NULL"));
    check_align(ws, 256, "workspace");
    if (have < need)
        fail(TQ_E_INVALID, text(call, "workspace of ") + std::to_string(have) + " bytes, " + std::to_string(need) +
                               " are needed");
}

inline void give(size_t *bytes, size_t n)
{
    if (!bytes) fail(TQ_E_INVALID, "bytes is NULL");
    *bytes = n;
}

} // namespace tq
