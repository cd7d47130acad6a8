"""A kernel's shared-memory limit after first calls on two threads (shared_limit.cuh,
compiled for the host, against a made-up driver): in every order of their steps the
limit holds what each of them needs, and still does for later calls."""

import subprocess

from paper_1601_04033_gb300 import build

SRC = r"""
#include <condition_variable>
#include <cstdio>
#include <mutex>
#include <thread>
#include <vector>
#include "shared_limit.cuh"

static const int64_t kMost = 200;
struct Driver {                        // limits of devices; gates that hold a call up
    std::mutex m;
    std::condition_variable cv;
    int64_t limit[70] = {};
    int calls = 0;
    int set(int dev, int64_t bytes) {
        ++calls;
        if (bytes > kMost) return 1;
        limit[dev] = bytes;
        return 0;
    }
};

// Two first calls that both find nothing raised.  One is slow: it sets its size after
// the other has returned, or (early) before the other sets its own, and goes on only
// when that one has returned.
static int run(int64_t need_a, int64_t need_b, bool a_slow, bool early, int dev) {
    fasgd::SharedLimit s;
    Driver d;
    int in = 0;
    bool fast_done = false, slow_set = false;
    const auto call = [&](int64_t need, bool slow) {
        s.ensure(dev, need, kMost, [&](int64_t bytes) {
            std::unique_lock<std::mutex> lock(d.m);
            ++in;
            d.cv.notify_all();
            d.cv.wait(lock, [&] { return in == 2; });
            if (slow && !early) d.cv.wait(lock, [&] { return fast_done; });
            if (!slow && early) d.cv.wait(lock, [&] { return slow_set; });
            const int error = d.set(dev, bytes);
            slow_set = slow_set || slow;
            d.cv.notify_all();
            if (slow && early) d.cv.wait(lock, [&] { return fast_done; });
            return error;
        });
        if (!slow) {
            std::lock_guard<std::mutex> lock(d.m);
            fast_done = true;
            d.cv.notify_all();
        }
    };
    std::thread a(call, need_a, a_slow), b(call, need_b, !a_slow);
    a.join();
    b.join();
    int bad = 0;
    for (const int64_t need : {need_a, need_b, kMost}) {
        const int e = s.ensure(dev, need, kMost, [&](int64_t bytes) { return d.set(dev, bytes); });
        if (e != 0 || d.limit[dev] < need) {
            std::printf("needs %d and %d, %s slow%s: limit %d, then %d\n", (int)need_a, (int)need_b, a_slow ? "a" : "b",
                        early ? " and early" : "", (int)d.limit[dev], (int)need);
            ++bad;
        }
    }
    return bad;
}
int main() {
    int bad = 0;
    for (const int64_t a : {60, 100, 200})
        for (const int64_t b : {60, 100, 200})
            for (int order = 0; order < 4; ++order)
                for (const int dev : {0, 3, 63, 64, 69}) bad += run(a, b, order & 1, order & 2, dev);
    // One call a device where nobody is in the way; an error is not taken for success.
    fasgd::SharedLimit s;
    Driver d;
    for (int i = 0; i < 5; ++i) s.ensure(1, 50 + i, kMost, [&](int64_t n) { return d.set(1, n); });
    if (d.calls != 1) std::printf("%d calls\n", d.calls), ++bad;
    if (s.ensure(1, kMost + 1, kMost, [&](int64_t n) { return d.set(1, n); }) == 0) std::printf("too much\n"), ++bad;
    if (s.ensure(2, 50, kMost, [&](int64_t) { return 7; }) != 7) std::printf("error\n"), ++bad;
    if (s.ensure(2, 50, kMost, [&](int64_t n) { return d.set(2, n); }) != 0 || d.limit[2] < 50) std::printf("again\n"), ++bad;
    return bad != 0;
}
"""


def test_first_calls_on_two_threads(tmp_path):
    src, exe = tmp_path / "limit.cpp", tmp_path / "limit"
    src.write_text(SRC)
    r = subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-pthread", f"-I{build.CSRC}", "-x", "c++", str(src),
                        "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
