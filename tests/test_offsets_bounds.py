"""CPU run of the device's search for a token's request (csrc/pk_device.cuh: warp_find_request, lane_request_window), the
header itself, compiled for the host with 32 threads as the lanes of a warp and every load checked: whatever the offsets
hold, no load lies outside them and the request is one of the call's; with good offsets it is the right one."""
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HOST = r"""
#include <barrier>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <thread>
#include <type_traits>
#include <vector>
#define __device__
#define __forceinline__ inline
#define asm
#define volatile(...)
static thread_local struct { unsigned x; } threadIdx;
static std::barrier<> sync_point(32);
static int64_t shared_word[32];
static const int64_t *first_word, *last_word;
static long stray;
template <typename T> T exchange(T v, int from) {
    shared_word[threadIdx.x] = (int64_t)v;
    sync_point.arrive_and_wait();
    const T r = (T)shared_word[from & 31];
    sync_point.arrive_and_wait();
    return r;
}
template <typename T> T __shfl_sync(unsigned, T v, int from) { return exchange(v, from); }
static unsigned __ballot_sync(unsigned, bool p) {
    shared_word[threadIdx.x] = p;
    sync_point.arrive_and_wait();
    unsigned r = 0;
    for (int i = 0; i < 32; ++i) r |= (unsigned)shared_word[i] << i;
    sync_point.arrive_and_wait();
    return r;
}
static bool __all_sync(unsigned m, bool p) { return __ballot_sync(m, p) == 0xffffffffu; }
static int __clz(int x) { return x ? __builtin_clz((unsigned)x) : 32; }
static int min(int a, int b) { return a < b ? a : b; }
static uint32_t min(uint32_t a, uint32_t b) { return a < b ? a : b; }
static int64_t max(int64_t a, int64_t b) { return a > b ? a : b; }
static int atomicCAS(int32_t *, int, int) { return 0; }
static int64_t __ldcg(const int64_t *p) {
    if (p < first_word || p > last_word) {
        __atomic_add_fetch(&stray, 1, __ATOMIC_RELAXED);
        return 0;
    }
    return *p;
}
#include "pk_device.cuh"
// cases on stdin: R, first item, R + 1 offsets; on stdout: stray loads, then every lane's request
int main() {
    long R, g0;
    while (scanf("%ld %ld", &R, &g0) == 2) {
        std::vector<int64_t> off(R + 1);
        for (auto &o : off) {
            long x;
            if (scanf("%ld", &x) != 1) return 1;
            o = x;
        }
        first_word = off.data(), last_word = off.data() + R, stray = 0;
        std::vector<uint32_t> got(32);
        std::vector<std::thread> lanes;
        for (unsigned l = 0; l < 32; ++l)
            lanes.emplace_back([&, l] {
                threadIdx.x = l;
                got[l] = pk::lane_request_window(off.data(), (uint32_t)R, g0, off[R], g0 + l);
            });
        for (auto &t : lanes) t.join();
        printf("%ld", stray);
        for (uint32_t r : got) printf(" %u", r);
        printf("\n");
    }
}
"""


@pytest.fixture(scope="module")
def search(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("search")
    (d / "host.cpp").write_text(HOST)
    csrc = os.path.join(ROOT, "paper_2609_38706_gb300", "csrc")
    subprocess.run([cxx, "-std=c++20", "-O1", "-fwrapv", "-w", "-pthread", f"-I{csrc}", str(d / "host.cpp"), "-o", str(d / "host")],
                   check=True)

    def run(cases):
        text = "\n".join(f"{len(o) - 1} {g0} " + " ".join(str(int(x)) for x in o) for o, g0 in cases)
        out = subprocess.run([str(d / "host")], input=text, capture_output=True, text=True, timeout=300, check=True).stdout
        rows = [[int(x) for x in line.split()] for line in out.splitlines()]
        assert len(rows) == len(cases)
        return rows

    return run


LOW, HIGH = -(1 << 63), (1 << 63) - 1


def test_no_load_outside_the_offsets(search):
    rng = np.random.default_rng(3)
    cases = []
    for R in (1, 2, 31, 32, 33, 40, 100):
        good = np.arange(R + 1) * 3
        for last in (LOW, LOW + 1, -5, 0, 1, HIGH):
            for g0 in (0, 32):
                for o in (good.copy(), np.full(R + 1, last, object), np.full(R + 1, LOW, object)):
                    o = [int(x) for x in o]
                    o[R] = last
                    cases.append((o, g0))
        for _ in range(4):
            cases.append(([int(x) for x in rng.choice([LOW, -7, 0, 5, 40, HIGH], R + 1)], 32 * int(rng.integers(0, 3))))
    for (o, g0), (stray, *got) in zip(cases, search(cases)):
        assert stray == 0 and max(got) < len(o) - 1, (o[:3], o[-1], g0, got)


def test_good_offsets_find_their_request(search):
    rng = np.random.default_rng(4)
    cases = []
    for R in (1, 3, 33, 120):
        for most in (1, 3, 40):
            o = np.concatenate(([0], np.cumsum(rng.integers(0, most + 1, R))))
            o[-1] += 1
            cases += [(o, g0) for g0 in range(0, int(o[-1]), max(32, int(o[-1]) // 3 // 32 * 32))]
    for (o, g0), (stray, *got) in zip(cases, search(cases)):
        n = min(32, int(o[-1]) - g0)
        assert stray == 0 and got[:n] == (np.searchsorted(o, np.arange(g0, g0 + n), side="right") - 1).tolist()
