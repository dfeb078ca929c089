"""The debug build's table of the callers' buffers (csrc/debug_kept.h, host arithmetic): a range is never larger than the
buffer that was last handed over at its place."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "debug_kept.h"
using namespace hadfl;
extern "C" {
DebugKept *kept_new() { return new DebugKept; }
void kept_delete(DebugKept *k) { delete k; }
int kept_keep(DebugKept *k, uint64_t owner, const uint64_t *lo_hi, int n) {
  DebugKept::Range r[8];
  for (int i = 0; i < n; ++i) r[i] = {lo_hi[2 * i], lo_hi[2 * i + 1]};
  return k->keep((const void *)(uintptr_t)owner, r, n);
}
void kept_forget(DebugKept *k, uint64_t owner) { k->forget((const void *)(uintptr_t)owner); }
int kept_all(DebugKept *k, uint64_t *lo_hi) {
  int n = 0;
  k->each([&](const DebugKept::Range &r) { lo_hi[2 * n] = r.lo; lo_hi[2 * n++ + 1] = r.hi; });
  return n;
}
int kept_room() { return DebugKept::kRoom; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    at = tmp_path_factory.mktemp("kept")
    (at / "kept.cpp").write_text(SOURCE)
    out = at / "libkept.so"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2111_08274_b200", "csrc"), "-o", str(out), str(at / "kept.cpp")], check=True)
    lib = C.CDLL(str(out))
    lib.kept_new.restype = C.c_void_p
    return lib


class Table:
    def __init__(self, lib):
        self.lib, self.k = lib, C.c_void_p(lib.kept_new())

    def keep(self, owner, *ranges):
        flat = [x for r in ranges for x in r]
        return bool(self.lib.kept_keep(self.k, C.c_uint64(owner), (C.c_uint64 * len(flat))(*flat), len(ranges)))

    def forget(self, owner):
        self.lib.kept_forget(self.k, C.c_uint64(owner))

    def all(self):
        buf = (C.c_uint64 * (2 * self.lib.kept_room()))()
        n = self.lib.kept_all(self.k, buf)
        return sorted((buf[2 * i], buf[2 * i + 1]) for i in range(n))

    def holds(self, lo, hi):
        return any(a <= lo and hi <= b for a, b in self.all())

    def __del__(self):
        self.lib.kept_delete(self.k)


@pytest.fixture
def table(lib):
    return Table(lib)


def test_same_buffers_again_change_nothing(table):
    assert table.keep(1, (100, 200), (300, 400)) and not table.keep(1, (100, 200), (300, 400)) and not table.keep(1, (300, 400))
    assert table.all() == [(100, 200), (300, 400)]


def test_a_smaller_buffer_at_the_place_of_a_larger_one_ends_where_it_ends(table):
    table.keep(1, (1000, 9000))
    assert table.keep(1, (1000, 2000)) and table.all() == [(1000, 2000)] and not table.holds(1000, 2016)
    assert table.keep(1, (1500, 1600)) and table.all() == [(1500, 1600)]
    assert table.keep(1, (1000, 9000)) and table.all() == [(1000, 9000)]


def test_buffers_of_other_handles_give_way_too(table):
    table.keep(1, (1000, 9000), (20000, 30000))
    table.keep(2, (8000, 8500))
    assert table.all() == [(8000, 8500), (20000, 30000)]


def test_neighbours_stay(table):
    table.keep(1, (1000, 2000))
    table.keep(1, (2000, 3000))
    assert table.all() == [(1000, 2000), (2000, 3000)] and not table.holds(1990, 2010)


def test_overlapping_buffers_of_one_call(table):
    """Two sets of messages may be two windows of one buffer."""
    for _ in range(2):
        table.keep(1, (0x1000, 0x5000), (0x2000, 0x6000))
        assert table.all() == [(0x1000, 0x5000), (0x2000, 0x6000)]
    assert not table.keep(1, (0x1000, 0x5000), (0x2000, 0x6000), (0x1000, 0x5000))


def test_a_destroyed_handle_leaves_nothing(table):
    table.keep(1, (1000, 2000), (3000, 4000))
    table.keep(2, (1000, 2000))                      # the same buffer, used by both
    table.forget(1)
    assert table.all() == [(1000, 2000)]
    table.forget(2)
    assert table.all() == []
    assert table.keep(3, (1500, 1600)) and table.all() == [(1500, 1600)]


def test_the_one_not_used_for_the_longest_time_makes_room(table, lib):
    room = lib.kept_room()
    for i in range(room):
        table.keep(1, (1000 * (i + 1), 1000 * (i + 1) + 10))
    table.keep(1, (1000, 1010))                      # used again
    table.keep(1, (500, 510), (700, 710))
    gone = {(2000, 2010), (3000, 3010)}
    assert set(table.all()) == {(1000 * (i + 1), 1000 * (i + 1) + 10) for i in range(room)} - gone | {(500, 510), (700, 710)}


def test_empty_buffers_are_no_ranges(table):
    assert not table.keep(1, (1000, 1000)) and table.all() == []
