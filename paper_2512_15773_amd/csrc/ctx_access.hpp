// What the attention and cache entry points use of a context (defined in tsdp.hip beside it).
#pragma once
#include <stdint.h>
#include "../../include/tsdp.h"

namespace tsdp {

int ctx_fail(tsdp_ctx* c, int code, const char* msg) noexcept;    // keeps the message, returns the code
int ctx_device(const tsdp_ctx* c) noexcept;                       // the device that was current in tsdp_create
int32_t* ctx_status(tsdp_ctx* c) noexcept;                        // device status word of tsdp_status

}  // namespace tsdp
