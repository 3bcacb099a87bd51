// Scratch memory of the calls that split their work over workgroups: one buffer
// per (device, stream), so that calls on different streams never share one; calls
// on one stream are ordered by the stream.  It grows on demand outside capture
// (allocation is not capturable).  A buffer that a call under capture was given
// lies in that call's graph, so it is kept for good: only buffers that no capture
// has seen are freed when they are outgrown.
//
// A call holds its buffer until its last launch is queued: no other thread's call
// on that stream can queue launches in between, which would find the one's parts
// where they look for their own, or free the buffer before the launch.
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

struct Workspace {
    float* ptr = nullptr;
    std::unique_lock<std::mutex> held;  // let go with the object
};

template <typename Device>
class Workspaces {
public:
    // At least `bytes` for a call on `st`, which holds them until *ws goes; `e`: the
    // device's error of the call that failed.
    WorkspaceError get(int dev, typename Device::stream st, size_t bytes, Workspace* ws, typename Device::error* e) {
        Buffer* buffer;
        {
            std::lock_guard<std::mutex> lk(mu_);
            buffer = &buffers_[{dev, st}];  // (stays where it is)
        }
        std::unique_lock<std::mutex> held(buffer->mu);
        State& b = buffer->state;
        if (b.bytes < bytes) {
            bool capturing = false;
            *e = Device::capturing(st, &capturing);
            if (*e) return WorkspaceError::kStatus;
            if (capturing) return WorkspaceError::kCapturing;
            float* old = b.captured ? nullptr : b.ws;
            b = State{};
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
        ws->ptr = b.ws;
        ws->held = std::move(held);
        return WorkspaceError::kNone;
    }

private:
    struct State {
        float* ws = nullptr;
        size_t bytes = 0;
        bool captured = false;  // a graph may hold it
    };
    struct Buffer {
        std::mutex mu;
        State state;
    };
    std::mutex mu_;  // of the table
    std::map<std::pair<int, typename Device::stream>, Buffer> buffers_;
};

}  // namespace neo
