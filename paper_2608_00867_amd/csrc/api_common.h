// api_common.h -- what the host sources of the C ABI share: the calling
// thread's error text and launch record, which nuna_api.cpp owns.
#pragma once

#include <stdint.h>

#include "nuna.h"

namespace nuna {

// Sets the calling thread's error text and returns `st`.
nuna_status_t api_fail(nuna_status_t st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// NUNA_OK, with the error text cleared.
nuna_status_t api_ok();
// From a catch handler: the exception in flight as a status.
nuna_status_t api_exception();
// NUNA_OK, or NUNA_ERR_HIP naming the call that failed.
nuna_status_t api_hip(hipError_t e, const char* what);
// Starts the record of a call's launches (nuna_last_launch).
void api_begin_launches();

}  // namespace nuna
