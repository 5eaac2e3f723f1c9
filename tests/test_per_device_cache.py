"""The host's per-device caches under threads that all make a first call: a reader never sees a part of the value,
the fill runs once, a failed one is tried again.  Compiled alone with the thread sanitizer where it works, since a
race on the flag seldom shows in the values."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <cstdio>
#include <thread>
#include <vector>
#include "per_device.h"
struct Pair { long a, b; };
int main()
{
    static stmoe_host::PerDevice<Pair> kept[64];
    std::atomic<int> fills{0}, bad{0}, failed{0};
    for (auto &cache : kept) {
        std::atomic<bool> go{false};
        std::vector<std::thread> threads;
        for (int t = 0; t < 8; ++t)
            threads.emplace_back([&, t] {
                while (!go.load()) {}
                for (int i = 0; i < 20; ++i) {
                    Pair p{0, 0};
                    const int dev = (t + i) % 2 ? 63 : 0;
                    const int rc = cache.get(dev, &p, [&](Pair &q) {
                        if (fills.fetch_add(1) % 3 == 0) return -3;
                        q.a = 7, q.b = dev + 1;
                        return 0;
                    });
                    if (rc == -3) failed.fetch_add(1);
                    else if (rc != 0 || p.a != 7 || p.b != dev + 1) bad.fetch_add(1);
                }
            });
        go.store(true);
        for (auto &t : threads) t.join();
    }
    const int good = fills.load() - failed.load();
    std::printf("fills %d failed %d bad %d\n", good, failed.load(), bad.load());
    return bad.load() != 0 || good != 2 * 64;
}
"""


def _build(tmp_path, name, source, *flags):
    src, exe = tmp_path / f"{name}.cpp", tmp_path / name
    src.write_text(source)
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-g", "-pthread", *flags,
                           "-I", os.path.join(ROOT, "paper_2606_15453_b200", "csrc"), "-o", str(exe), str(src)])
    return str(exe)


def test_threads_that_make_the_first_call_together(tmp_path):
    exe = _build(tmp_path, "plain", SOURCE)
    for _ in range(5):
        r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stdout + r.stderr


def test_no_race_under_the_thread_sanitizer(tmp_path):
    try:
        probe = _build(tmp_path, "probe", "int main() { return 0; }", "-fsanitize=thread")
        works = subprocess.run([probe], capture_output=True, timeout=60).returncode == 0
    except subprocess.CalledProcessError:
        works = False
    if not works:
        pytest.skip("no thread sanitizer on this machine")
    r = subprocess.run([_build(tmp_path, "race", SOURCE, "-fsanitize=thread")], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "data race" not in r.stderr, r.stdout + r.stderr[-3000:]
