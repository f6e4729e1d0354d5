// What the single-operator entry points share: error returns, the check for a device, and the end of a call.
#pragma once
#include <cuda_runtime.h>
#include <stdarg.h>
#include <stdio.h>

#include <exception>

#include "../../include/mslt.h"

namespace mslt {
void set_last_error(const char* msg);  // defined with the C ABI (mslt.cu)
namespace {

inline int op_refuse(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  set_last_error(buf);
  return code;
}

inline int op_need_device() {
  int ndev = 0;
  if (cudaGetDeviceCount(&ndev) != cudaSuccess || ndev < 1)
    return op_refuse(MSLT_ERR_CUDA, "no CUDA device: this library has no CPU path");
  return 0;
}

inline int op_end(const char* what, cudaStream_t st, int sync) {
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess && sync) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return op_refuse(MSLT_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
  return 0;
}

// Nothing throws across the C boundary: what the standard library throws becomes a status.
template <typename F>
inline int op_nothrow(const char* what, F&& body) {
  try {
    return body();
  } catch (const std::exception& e) {
    return op_refuse(MSLT_ERR_CUDA, "%s: %s", what, e.what());
  } catch (...) {
    return op_refuse(MSLT_ERR_CUDA, "%s: unknown exception", what);
  }
}

}  // namespace
}  // namespace mslt
