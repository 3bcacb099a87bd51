"""The table of scratch buffers (csrc/workspace.h), compiled for the host over a
device of pretence: what is kept, freed, refused and shared."""
import ctypes
import os
import subprocess
import threading

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1809_02697_amd", "csrc")
SHIM = r"""
#include <cstdlib>
#include <set>

#include "workspace.h"

struct Pretence {
    typedef long stream;
    typedef int error;
    static std::set<float*> freed;
    static std::set<long> under_capture;
    static int status, room;
    static int alloc(size_t bytes, float** p) {
        if ((int)bytes > room) return 2;
        *p = static_cast<float*>(malloc(bytes));
        return 0;
    }
    static int free(float* p) {  // (its address stays taken, so that no later buffer has it)
        freed.insert(p);
        return 0;
    }
    static int capturing(long st, bool* yes) {
        *yes = under_capture.count(st);
        return status;
    }
};
std::set<float*> Pretence::freed;
std::set<long> Pretence::under_capture;
int Pretence::status = 0, Pretence::room = 1 << 30;
neo::Workspaces<Pretence> table;

extern "C" {
// the buffer, or minus the error
long get(int dev, long st, long bytes) {
    neo::Workspace ws;
    int e = 0;
    const neo::WorkspaceError r = table.get(dev, st, bytes, &ws, &e);
    return r == neo::WorkspaceError::kNone ? (long)ws.ptr : -(long)r;
}
// the same, held until let_go on the same thread
static thread_local neo::Workspace mine;
long hold(int dev, long st, long bytes) {
    int e = 0;
    return table.get(dev, st, bytes, &mine, &e) == neo::WorkspaceError::kNone ? (long)mine.ptr : 0;
}
void let_go() { mine = neo::Workspace(); }
void capture(long st, int on) {
    if (on) Pretence::under_capture.insert(st);
    else Pretence::under_capture.erase(st);
}
int is_freed(long p) { return Pretence::freed.count((float*)p); }
void set_status(int v) { Pretence::status = v; }
void set_room(int v) { Pretence::room = v; }
}
"""


@pytest.fixture()
def host(tmp_path):
    (tmp_path / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-pthread", "-I", CSRC, "-o", str(tmp_path / "shim.so"),
                    str(tmp_path / "shim.cpp")], check=True, timeout=100)
    L = ctypes.CDLL(str(tmp_path / "shim.so"))
    L.get.restype, L.get.argtypes = ctypes.c_long, [ctypes.c_int, ctypes.c_long, ctypes.c_long]
    L.hold.restype, L.hold.argtypes = L.get.restype, L.get.argtypes
    L.is_freed.argtypes = [ctypes.c_long]
    return L


def test_one_buffer_a_stream_grown_and_freed(host):
    a = host.get(0, 7, 100)
    assert a > 0 and host.get(0, 7, 40) == a == host.get(0, 7, 100)
    assert len({a, host.get(0, 8, 100), host.get(1, 7, 100)}) == 3
    b = host.get(0, 7, 101)
    assert b not in (a, 0) and host.is_freed(a) and not host.is_freed(b) and host.get(0, 7, 100) == b


def test_a_captured_buffer_is_never_freed(host):
    """Graphs captured from small to large, with larger calls outside between them."""
    held = []
    for n in (100, 1000, 10000):
        warm = host.get(0, 7, n)
        host.capture(7, 1)
        assert host.get(0, 7, n) == warm
        host.capture(7, 0)
        held.append(warm)
        host.get(0, 7, 5 * n)
    assert len(set(held)) == 3 and not any(host.is_freed(p) for p in held)
    # a buffer that no capture saw goes when it is outgrown
    last = host.get(0, 7, 50000)
    host.get(0, 7, 60000)
    assert host.is_freed(last)


def test_growth_under_capture_is_refused(host):
    a = host.get(0, 7, 100)
    host.capture(7, 1)
    assert host.get(0, 7, 101) == -1 and host.get(0, 9, 8) > 0
    assert host.get(0, 7, 100) == a and not host.is_freed(a)
    host.capture(7, 0)
    assert host.get(0, 7, 101) > 0 and not host.is_freed(a)


def test_errors(host):
    a = host.get(0, 7, 100)
    host.set_status(3)
    assert host.get(0, 7, 101) == -2 and host.get(0, 7, 100) == a      # unknown: as if captured
    host.set_status(0)
    host.set_room(50)
    assert host.get(0, 7, 101) == -4 and not host.is_freed(a)
    assert host.get(0, 7, 40) > 0                                       # the next call that fits
    host.set_room(1 << 30)
    assert host.get(0, 7, 101) > 0


def test_a_call_holds_its_buffer_until_its_launches_are_queued(host):
    """Calls of two threads on one stream come one after the other, and the second,
    larger one does not free what the first still launches with; other streams go on."""
    queue, taken, go = [], threading.Event(), threading.Event()

    def first():
        p = host.hold(0, 7, 100)
        queue.append("first main")
        taken.set()
        go.wait(20)
        queue.append("first join" if not host.is_freed(p) else "freed")
        host.let_go()

    def second():
        taken.wait(20)
        p = host.hold(0, 7, 200)
        queue.extend(["second main", "second join"])
        host.let_go()
        assert p > 0

    threads = [threading.Thread(target=f) for f in (first, second)]
    for t in threads:
        t.start()
    assert taken.wait(20)
    threads[1].join(0.3)
    assert threads[1].is_alive() and host.get(0, 8, 100) > 0 and host.get(1, 7, 100) > 0
    go.set()
    for t in threads:
        t.join(20)
    assert queue == ["first main", "first join", "second main", "second join"]
