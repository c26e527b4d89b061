// What the C-ABI layers of the operators beside the decode step share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>
#include <string>

#include "taper_attn.h"
#include "taper_plan.h"

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

// Whether what is enqueued on `s` is recorded into a graph.
inline bool recording(hipStream_t s) {
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(s, &status) != hipSuccess) (void)hipGetLastError();  // (the launch itself will say what is wrong)
    return status != hipStreamCaptureStatusNone;
}

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

// What a batch's arrays say, checked as taper_plan_build_segments checks them: block table, lengths, page counts, segments and request
// CSR of `out`.  (Its shares are for a single workgroup, which is the quickest; they are not used.)
inline int resolve_batch(int page_size, int n_seqs, const int32_t* block_table, int bt_row_stride, const int32_t* branch_group,
                         const int32_t* prefix_len, const int32_t* seg_start, const int32_t* seg_len, int64_t n_pool_pages, HostPlan* out) {
    taper_attn_config one_head = {1, 1, 64, page_size, 1.0f, -1, TAPER_PARTIAL_F16_SCALED};
    taper_plan_options o = {};
    o.target_workgroups = 1;
    o.share_prefix = 1;
    o.pool_pct = o.solo_item_tokens = o.small_step_grid = -1;
    std::string err;
    const int st = build_host_plan_segments(one_head, n_seqs, block_table, bt_row_stride, branch_group, prefix_len, seg_start, seg_len,
                                            n_pool_pages, &o, out, &err);
    return st == TAPER_OK ? st : set_error(st, err);
}

}  // namespace taper
