"""The host's bookkeeping of static counter slots (csrc/slot_table.h), compiled here by the C++ compiler: a slot whose last
runs may still be queued is not handed on before something has waited for them, a captured one never."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_13764_b200", "csrc")

PROGRAM = r"""
#include "slot_table.h"
#include <cstdio>
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
using nk::SlotTable;
int main() {
    static SlotTable t;
    int waits = 0;
    bool can_wait = true;
    auto wait = [&] { ++waits; return can_wait; };
    const int a = t.take(wait), b = t.take(wait);
    CHECK(a >= 0 && b >= 0 && a != b);
    t.give(-1, true, true);                        // a plan without a slot
    t.give(a, false, false);
    CHECK(t.take(wait) == a);                      // no run of it is left: straight on
    t.give(a, true, false);                        // destroyed with runs queued
    t.give(b, true, true);                         // and held by a graph
    for (int i = 0; i < SlotTable::SLOTS - 2; ++i) {
        const int s = t.take(wait);
        CHECK(s >= 0 && s != a && s != b);
    }
    CHECK(waits == 0);                             // every other slot went first, without a wait
    can_wait = false;
    CHECK(t.take(wait) == -1 && waits == 1);       // the wait failed: none
    can_wait = true;
    CHECK(t.take(wait) == a && waits == 2);
    CHECK(t.take(wait) == -1 && waits == 2);       // nothing in flight is left to wait for; the captured one stays out
    t.give(a, false, false);
    CHECK(t.take(wait) == a);
    return 0;
}
"""


def test_a_slot_is_not_handed_on_while_its_runs_may_be_queued(tmp_path):
    compiler = shutil.which("g++") or shutil.which("c++")
    if not compiler:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "slots.cpp", tmp_path / "slots"
    src.write_text(PROGRAM)
    subprocess.check_call([compiler, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe), "-pthread"])
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0, out.stdout
