// Scratch memory of the calls that split their work over workgroups: one buffer
// per (device, stream), so that calls on different streams never share one; calls
// on one stream are ordered by the stream.  It grows on demand outside capture
// (allocation is not capturable).  A buffer that a call under capture was given
// lies in that call's graph, so it is kept for good: only buffers that no capture
// has seen are freed when they are outgrown.
//
// `Device` makes the calls, so that the host's side can run without one:
// stream, error (0 is success), alloc, free, capturing.
#pragma once

#include <cstddef>
#include <map>
#include <mutex>
#include <utility>

namespace neo {

enum class WorkspaceError { kNone, kCapturing, kStatus, kFree, kAlloc };

template <typename Device>
class Workspaces {
public:
    // At least `bytes` for a call on `st`, in *ws; `e`: the device's error of the
    // call that failed.
    WorkspaceError get(int dev, typename Device::stream st, size_t bytes, float** ws, typename Device::error* e) {
        std::lock_guard<std::mutex> lk(mu_);
        Buffer& b = buffers_[{dev, st}];
        if (b.bytes < bytes) {
            bool capturing = false;
            *e = Device::capturing(st, &capturing);
            if (*e) return WorkspaceError::kStatus;
            if (capturing) return WorkspaceError::kCapturing;
            float* old = b.captured ? nullptr : b.ws;
            b = Buffer{};
            if (old && (*e = Device::free(old))) return WorkspaceError::kFree;
            if ((*e = Device::alloc(bytes, &b.ws))) {
                b.ws = nullptr;
                return WorkspaceError::kAlloc;
            }
            b.bytes = bytes;
        } else if (!b.captured) {
            // (a status that cannot be told counts as capture: the buffer is kept)
            if (Device::capturing(st, &b.captured)) b.captured = true;
        }
        *ws = b.ws;
        return WorkspaceError::kNone;
    }

private:
    struct Buffer {
        float* ws = nullptr;
        size_t bytes = 0;
        bool captured = false;  // a graph may hold it
    };
    std::mutex mu_;
    std::map<std::pair<int, typename Device::stream>, Buffer> buffers_;
};

}  // namespace neo
