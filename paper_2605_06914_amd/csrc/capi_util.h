// What the C-ABI layers of the operators beside the decode step share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>
#include <string>

#include "taper_attn.h"

namespace taper {

int set_error(int code, const std::string& msg);  // (of the calling thread: taper_last_error)

inline int hip_error(hipError_t e, const char* what) { return set_error(TAPER_EHIP, std::string(what) + ": " + hipGetErrorString(e)); }
#define HIP_TRY(expr)                                             \
    do {                                                          \
        hipError_t e_ = (expr);                                   \
        if (e_ != hipSuccess) return taper::hip_error(e_, #expr); \
    } while (0)

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// The calls of an object run on its device whatever the calling thread's current one is.
class OnDevice {
  public:
    explicit OnDevice(int device) {
        error = hipGetDevice(&before_);
        if (error == hipSuccess && before_ != device) {
            error = hipSetDevice(device);
            changed_ = error == hipSuccess;
        }
    }
    ~OnDevice() {
        if (changed_) (void)hipSetDevice(before_);
    }
    OnDevice(const OnDevice&) = delete;
    hipError_t error;

  private:
    int before_ = 0;
    bool changed_ = false;
};

// No C++ exception leaves a C entry point.
template <typename F>
int guarded(F&& f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return set_error(TAPER_ENOMEM, "host allocation failed");
    } catch (...) {
        return set_error(TAPER_EINVAL, "unexpected error");
    }
}

}  // namespace taper
