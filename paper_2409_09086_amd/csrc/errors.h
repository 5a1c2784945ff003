// The calling thread's last failure (infmllm_last_error): every entry point returns through these.
#pragma once
#include <hip/hip_runtime.h>

namespace infmllm {

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int fail_hip(hipError_t e, const char* what);

}  // namespace infmllm
