// What the C boundary's calls on logits share: refusals, the device that they launch on, exceptions that stay inside.
#pragma once
#include <new>
#include <string>
#include "zf_internal.h"
#include "zf_ops.h"

namespace zf {
namespace {

int refuse(const char *why) { set_error(why); return ZF_ERR_INVALID_ARG; }
template <class F>
int on_device(int32_t device, F launch) {     // launches on `device`, and leaves the thread's current device as it was
    int before = -1;
    hipError_t e = hipGetDevice(&before);
    const bool other = e == hipSuccess && before != device;
    if (e == hipSuccess && other) e = hipSetDevice(device);
    if (e == hipSuccess) {
        e = launch();
        if (other) { const hipError_t back = hipSetDevice(before); if (e == hipSuccess) e = back; }
    }
    if (e == hipSuccess) return ZF_OK;
    set_error(std::string("HIP: ") + hipGetErrorString(e));
    return ZF_ERR_DEVICE;
}
template <class F>
auto guarded(F f) -> decltype(f()) {          // nothing is thrown across the boundary (an error's text may find no memory)
    try { return f(); } catch (const std::bad_alloc &) { return ZF_ERR_OOM; }
}
bool element_aligned(const void *p, int32_t dtype) { return (uintptr_t)p % (dtype == 0 ? 4 : 2) == 0; }


}  // namespace
}  // namespace zf
