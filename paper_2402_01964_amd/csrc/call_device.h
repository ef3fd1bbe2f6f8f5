// call_device.h -- the device of a call that no table belongs to, and its
// launches.  Private to libnlb.so.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/nlb.h"

namespace {

// Makes `device` (-1: the current one) the current device for as long as it
// lives.  rc: NLB_OK, or why it could not.
class CallDevice {
  public:
    explicit CallDevice(int32_t device) {
        int n = 0;
        rc = NLB_EDEVICE;
        if (hipGetDevice(&prev_) != hipSuccess || hipGetDeviceCount(&n) != hipSuccess || n < 1) return;
        if (device >= n) rc = NLB_EINVAL;
        else if (device < 0 || device == prev_) rc = NLB_OK;
        else if (hipSetDevice(device) == hipSuccess) {
            set_ = true;
            rc = NLB_OK;
        }
    }
    ~CallDevice() {
        if (set_) (void)hipSetDevice(prev_);
    }
    int rc;

  private:
    int prev_ = -1;
    bool set_ = false;
};

// Starts a kernel.  What it returns is this launch's own: kernels that read
// what it leaves are not started after a failure, and an error that an earlier
// call of the program left is not taken for one.
template <typename T> struct Given { typedef T type; };
template <typename... P>
int enqueue(void (*kernel)(P...), dim3 blocks, uint32_t threads, uint32_t lds, hipStream_t stream,
            typename Given<P>::type... args) {
    void *p[] = {(void *)&args...};
    if (hipLaunchKernel((const void *)kernel, blocks, dim3(threads), p, lds, stream) == hipSuccess) return NLB_OK;
    (void)hipGetLastError();
    return NLB_EDEVICE;
}

}  // namespace
