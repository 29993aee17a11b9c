"""Runs device functions that are control flow above all (waits, hand-overs) on the host: their text is taken from the source,
put between definitions that stand in for what a GPU has, and compiled with g++.  A lane is a thread; a vote or a __syncwarp that a
lane of the warp never reaches is an error, as is a lane that does not return in time."""
import os
import re
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_19578_b200", "csrc")


def text(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def definition(source, start):
    """A template function or struct from its first line, which `start` (a regular expression) finds, to its closing brace."""
    m = re.search(start, source, re.M)
    assert m, start
    at = source.index("{", m.end() - 1 if source[m.end() - 1] == "{" else m.end())
    depth = 0
    for i in range(at, len(source)):
        depth += {"{": 1, "}": -1}.get(source[i], 0)
        if depth == 0:
            return source[m.start():i + 1] + (";" if source[i + 1] == ";" else "")
    raise AssertionError(start)


PRELUDE = r'''
#include <algorithm>
#include <chrono>
#include <condition_variable>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <mutex>
#include <thread>
#include <vector>
#define __device__
#define __host__
#define __noinline__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __align__(n) alignas(n)
using std::max;
using std::min;
struct uint4 { uint32_t x, y, z, w; };
struct uint2 { uint32_t x, y; };
struct Dim { unsigned x; };
thread_local Dim threadIdx{0}, blockIdx{0};
[[noreturn]] void fail(const char* what) { std::printf("FAILED: %s\n", what); std::fflush(stdout); std::_Exit(1); }

// The lanes that run, meeting at votes.
struct Warp {
  std::mutex m;
  std::condition_variable cv;
  int lanes = 1, at = 0, gone = 0;
  bool all = true, any = false, was_all = true, was_any = false;
  long round = 0;
  void meet(bool p) {
    std::unique_lock<std::mutex> l(m);
    if (gone > 0) fail("a vote that a lane which has returned does not reach");
    all = all && p;
    any = any || p;
    if (++at == lanes) {
      was_all = all; was_any = any;
      all = true; any = false; at = 0;
      ++round;
      cv.notify_all();
      return;
    }
    const long mine = round;
    if (!cv.wait_for(l, std::chrono::seconds(20), [&] { return round != mine || gone > 0; })) fail("a vote that not all lanes reach");
    if (round == mine) fail("a vote that a lane which has returned does not reach");
  }
  void leave() {
    std::unique_lock<std::mutex> l(m);
    ++gone;
    cv.notify_all();
  }
} warp;
inline bool __all_sync(uint32_t, bool p) { warp.meet(p); return warp.was_all; }
inline bool __any_sync(uint32_t, bool p) { warp.meet(p); return warp.was_any; }
inline void __syncwarp() { warp.meet(true); }
inline void __threadfence_block() {}
inline void __nanosleep(unsigned) {}
std::atomic<long long> now{0}, tick{100000000};     // the clock moves when it is looked at
inline long long clock64() { return now += tick; }
inline int atomicCAS(int* p, int expected, int x) { const int old = *p; if (old == expected) *p = x; return old; }
enum { SP_ERR_RANGE = -6, SP_ERR_TIMEOUT = -5 };
struct Abort { volatile int* flag; int* status; };
inline void report_range(int* status, int where) { if (atomicCAS(status, 0, SP_ERR_RANGE) == 0) status[1] = where; }
inline void report_timeout(int* status, int where) { if (atomicCAS(status, 0, SP_ERR_TIMEOUT) == 0) status[1] = where; }
constexpr long long kWaitCycles = 1000000000ll;

// Every lane's part of `body(lane)`, in threads of their own.
inline void run_lanes(int lanes, std::function<void(int)> body) {
  warp.lanes = lanes; warp.at = warp.gone = 0; warp.all = true; warp.any = false;
  std::vector<std::thread> t;
  for (int i = 0; i < lanes; ++i) t.emplace_back([&, i] { body(i); warp.leave(); });
  for (auto& x : t) x.join();
}
'''


def run(tmp_path, program, seconds=60):
    """Compiles and runs; what it printed."""
    cxx = os.environ.get("CXX") or shutil.which("g++")
    src, exe = tmp_path / "emulated.cpp", tmp_path / "emulated"
    src.write_text("#include <atomic>\n" + PRELUDE + program)
    r = subprocess.run([cxx, "-O1", "-std=c++17", "-w", "-pthread", str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[:4000]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=seconds)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout + r.stderr
    return r.stdout
