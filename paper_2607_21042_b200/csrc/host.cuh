// Host-side pieces that every entry point shares: the error text of a failed call without a handle, the device's SM count.
#pragma once
#include <cuda_runtime.h>
#include "../../include/tts_gpt.h"

namespace ttsgpt {

// records the text that tts_gpt_last_error(NULL) returns on this thread, and returns `code`
int fail_op(int code, const char *fmt, ...);

// SMs of the current device
inline int device_sms() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && sms > 0) return sms;
  return 148;
}

}  // namespace ttsgpt
