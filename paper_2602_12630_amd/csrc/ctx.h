/*
 * What the sources of the library beside tc_lib.cpp need of a context, which is defined there.
 */
#pragma once
#include "../../include/tc.h"
#include "rt.h"

namespace tc {
rt::stream_t ctx_stream(const tc_ctx* ctx);
int ctx_device(const tc_ctx* ctx);
int ctx_use_device(tc_ctx* ctx);                                   /* makes the context's GPU the current one */
int ctx_fail(tc_ctx* ctx, int code, const char* msg);              /* keeps the message for tc_last_error, returns code */
int ctx_fail_hip(tc_ctx* ctx, int e, const char* where);           /* the same for a runtime error: TC_ERR_HIP */
}  // namespace tc
