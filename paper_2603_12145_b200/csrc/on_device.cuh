// on_device.cuh -- a call's device: what a handle enqueues goes to the device that it was created on,
// whichever is current in the calling thread.  (The default stream's value is the same on every
// device: a launch on it goes to the current one, with another one's pointers.)
#pragma once

#include <cuda_runtime.h>

namespace {

class OnDevice {
public:
    explicit OnDevice(int device)
    {
        int current = 0;
        ok_ = cudaGetDevice(&current) == cudaSuccess;
        if (ok_ && current != device) {
            ok_ = cudaSetDevice(device) == cudaSuccess;
            if (ok_) back_ = current;
        }
        if (!ok_) cudaGetLastError();
    }
    ~OnDevice()
    {
        if (back_ >= 0) cudaSetDevice(back_);
    }
    OnDevice(const OnDevice &) = delete;
    OnDevice &operator=(const OnDevice &) = delete;
    bool ok() const { return ok_; }

private:
    bool ok_ = false;
    int back_ = -1;        // the device to make current again
};

}  // namespace
