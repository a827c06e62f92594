"""The bounded waits of the block-scaled 8-bit product (csrc/matmul_wait.h),
compiled for the host with a barrier and a cycle counter of the test's own: no
GPU, and no wait that really lasts."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_02438_gb300", "csrc")

HARNESS = r"""
#include <cstdint>
#include <cstdio>
#define __device__
#define __forceinline__ inline
// a clock that steps on every reading, and a barrier that completes at cycle `done_at`
static long long now, step = 1000000, done_at;
static long long clock64() { return now += step; }
static bool mbar_try_wait(uint64_t *, uint32_t) { return now >= done_at; }
#include "matmul_wait.h"
using namespace xp;
static int failed;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); failed = 1; } } while (0)

int main()
{
    uint64_t bar = 0;
    volatile int abort = 0;
    const long long SEC = MM_WAIT_CYCLES / 2;

    // a phase that completes in time, one that does not, and another role's abort
    now = 5; done_at = SEC;
    CHECK(mm_wait(&bar, 0, &abort) && abort == 0 && now < SEC + 2 * step);
    now = 5; done_at = 100 * SEC;
    CHECK(!mm_wait(&bar, 0, &abort) && abort == 1 && now > MM_WAIT_CYCLES && now < MM_WAIT_CYCLES + 4 * step);
    now = 5; abort = 1;
    CHECK(!mm_wait(&bar, 0, &abort) && now < 5 + 2 * step);

    // waits that name one start end together, however many of them had to wait
    volatile long long since = 0;
    abort = 0; now = 5; done_at = 0;
    CHECK(mm_wait(&bar, 0, &abort, MM_WAIT_CYCLES, &since) && since == 0);       // no wait: no start
    long long first = now;
    bool ok = true;
    for (int i = 0; i < 8 && ok; ++i) {
        done_at = now + SEC * 9 / 10 * 2;                                        // each 0.9 of the limit
        ok = mm_wait(&bar, 0, &abort, MM_WAIT_CYCLES, &since);
    }
    const long long sender_ends = now;
    CHECK(!ok && abort == 1 && sender_ends - first < MM_WAIT_CYCLES + 8 * step);

    // the receiver: its own work was given up at once, and the sender, whose waits
    // began with its own, sends as late as it can; the receiver has to be there
    abort = 1; now = first; done_at = sender_ends + 1;
    CHECK(mm_wait_joined(&bar, &abort));
    CHECK(now >= sender_ends);
    // with nothing set, the same
    abort = 0; now = first;
    CHECK(mm_wait_joined(&bar, &abort) && abort == 0 && now >= sender_ends);
    // a sender that never comes: bounded, and reported
    abort = 0; now = first; done_at = 1000 * SEC;
    CHECK(!mm_wait_joined(&bar, &abort) && abort == 1 && now - first < 4 * MM_WAIT_CYCLES);
    return failed;
}
"""


def test_receiver_of_a_split_outlasts_its_senders(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "wait.cpp", tmp_path / "wait"
    src.write_text(HARNESS)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I" + CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout


@pytest.mark.parametrize("name", ["matmul_fp8.cu", "matmul_fp8_wide.cu"])
def test_both_kernels_wait_for_their_sums_this_way(name):
    with open(os.path.join(CSRC, name)) as f:
        src = f.read()
    waits = re.findall(r"(mm_wait\w*)\(\s*&?(?:sh\.)?joined\b", src)
    assert waits == ["mm_wait_joined"]
