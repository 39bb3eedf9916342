// The library's second stream and its events (mdn_api.hip).  Host only.
#pragma once
#include <hip/hip_runtime.h>

#include <mutex>
#include <vector>

namespace mdn {

// One set per device, shared by every call on that device.  A call that uses them holds the device's mutex while it ENQUEUES (the kernels
// themselves run after it has returned): an event is recorded and waited for inside one such section, so calls from several host threads
// cannot interleave their record / wait pairs; their work on the second stream is simply ordered one call after the other.
struct Side {
    hipStream_t stream = nullptr;
    std::vector<hipEvent_t> ev;
    std::mutex mutex;
};

// the current device's, or null
Side *side_device();
// the same with its stream and n events created (once, default priority), or null; call with the lock held
Side *side(int n);

// what mdn_set_segments() asked for; 0: automatic
int requested_segments();

} // namespace mdn
