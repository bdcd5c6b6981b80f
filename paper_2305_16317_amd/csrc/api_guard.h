// What every C entry point shares: exceptions end at the entry point as a
// pd_status and the calling thread's error message.
#pragma once

#include <exception>
#include <new>
#include <string>

#include "pd_internal.h"

namespace pd {

// the calling thread's message behind pd_last_error()
std::string& last_error();

template <class F>
pd_status guard(F&& f) {
    try {
        f();
        last_error().clear();
        return PD_OK;
    } catch (const Error& e) {
        last_error() = e.msg;
        return e.code;
    } catch (const std::bad_alloc&) {
        last_error() = "host allocation failed";
        return PD_ERR_OOM;
    } catch (const std::exception& e) {
        last_error() = e.what();
        return PD_ERR_DEVICE;
    } catch (...) {
        last_error() = "unknown error";
        return PD_ERR_DEVICE;
    }
}

inline void require(bool ok, const std::string& msg) {
    if (!ok) fail(PD_ERR_INVALID_ARG, msg);
}
inline void require(bool ok, const char* msg) {
    if (!ok) fail(PD_ERR_INVALID_ARG, msg);
}

}  // namespace pd
