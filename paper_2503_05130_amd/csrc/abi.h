// What every C entry point is wrapped in: argument errors as exceptions of this
// library, none of which crosses the ABI, and the calling thread's message.
#pragma once

#include <hip/hip_runtime.h>

#include <new>
#include <string>

#include "iefwd.h"

namespace iefwd {

// The message iefwd_last_error returns, of the calling thread.
std::string &last_error_text();

struct Error {
    int status;
    std::string msg;
};

[[noreturn]] inline void fail(int status, const std::string &msg) { throw Error{status, msg}; }

inline void hip_check(hipError_t e, const char *what) {
    if (e != hipSuccess) fail(IEFWD_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

template <class F>
int guarded(F &&f) {
    last_error_text().clear();
    try {
        f();
        return IEFWD_OK;
    } catch (const Error &e) {
        last_error_text() = e.msg;
        return e.status;
    } catch (const std::bad_alloc &) {
        last_error_text() = "host allocation failed";
        return IEFWD_ENOMEM;
    } catch (...) {
        last_error_text() = "unexpected internal error";
        return IEFWD_EHIP;
    }
}

}  // namespace iefwd
