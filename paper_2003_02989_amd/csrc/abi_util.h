// abi_util.h -- what the extern "C" entry points share: errors raised inside a
// call, their text for tq_last_error, and the checks of pointer arguments.
#pragma once
#include <hip/hip_runtime.h>

#include <new>
#include <string>

#include "../../include/tq.h"
#include "program.h"

namespace tq {

// The calling thread's text of tq_last_error.
std::string &error_text();

[[noreturn]] inline void fail(int status, const std::string &m) { throw Error{status, m}; }

inline void hip_check(hipError_t e, const char *what)
{
    if (e != hipSuccess) fail(TQ_E_DEVICE, std::string(what) + ": " + hipGetErrorString(e));
}

inline void check_align(const void *p, size_t a, const char *name)
{
    if (reinterpret_cast<uintptr_t>(p) % a != 0)
        fail(TQ_E_INVALID, std::string(name) + " must be " + std::to_string(a) + "-byte aligned");
}

inline hipStream_t as_stream(void *s) { return static_cast<hipStream_t>(s); }

// Runs f and turns what it throws into a status: no exception leaves the call.
template <class F> tq_status guarded(F &&f)
{
    try {
        f();
        error_text().clear();
        return TQ_OK;
    } catch (const Error &e) {
        error_text() = e.msg;
        return (tq_status)e.status;
    } catch (const std::bad_alloc &) {
        error_text() = "host allocation failed";
        return TQ_E_NOMEM;
    } catch (...) {
        error_text() = "internal error";
        return TQ_E_DEVICE;
    }
}

} // namespace tq
