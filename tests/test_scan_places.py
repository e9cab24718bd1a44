"""The order in which a scan's workgroups take their tasks (csrc/scan_places.h):
every task is taken once, a place after its runners and the places below it, and
with few workgroups running at once, one call or several, all of them end."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = """
#include "scan_places.h"
using namespace tgm;
extern "C" int32_t runners() { return kMaxRunners; }
extern "C" int32_t narrow(int32_t blocks, int32_t V) { return ScanTasks{blocks, 1, V, 8}.narrow(); }
extern "C" int64_t all(int32_t blocks, int32_t groups, int32_t V, int32_t W)
{
    return ScanTasks{blocks, groups, V, W}.all();
}
extern "C" int32_t slice(int32_t V, int32_t W) { return ScanTasks{1, 1, V, W}.deep(); }
extern "C" void task(uint32_t t, int32_t blocks, int32_t groups, int32_t V, int32_t W, int32_t *out)
{
    const ScanTask s = wide_task(ScanTasks{blocks, groups, V, W}, t);
    out[0] = s.block, out[1] = s.place;
}
"""


@pytest.fixture(scope="module")
def places(tmp_path_factory):
    d = tmp_path_factory.mktemp("places")
    src, so = d / "shim.cpp", d / "shim.so"
    src.write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2402_15113_amd", "csrc"), str(src), "-o", str(so)],
                   check=True)
    lib = C.CDLL(str(so))
    lib.all.restype = C.c_int64
    return lib


def tasks(lib, blocks, groups, V, W):
    """The tasks of a wide call in order: ("run", the chains of a runner, each of a block)
    or ("place", block, place)."""
    out, found, deep = (C.c_int32 * 2)(), [], lib.slice(V, W)
    for t in range(lib.all(blocks, groups, V, W)):
        lib.task(C.c_uint32(t), blocks, groups, V, W, out)
        b, p = out[0], out[1]
        if p >= 0:
            found.append(("place", b, p))
        else:
            chains = [((-1 - p) * W + w) for w in range(W)]
            end = min(blocks, b + deep)
            found.append(("run", [(b + c // V, c % V) for c in chains if b + c // V < end]))
    return found


# channel blocks, places of each, runners of each, wavefronts of a workgroup: widths of up
# to 65,536 channels
SHAPES = [(9, 4, 1, 8), (5, 2, 2, 4), (16, 3, 2, 8), (17, 3, 2, 4), (32, 5, 1, 4), (33, 5, 1, 4),
          (63, 3, 2, 8), (64, 7, 1, 8), (65, 7, 1, 8), (512, 3, 2, 8), (1024, 2, 1, 8),
          (1024, 5, 1, 4)]


@pytest.mark.parametrize("blocks,groups,V,W", SHAPES)
def test_each_task_once_and_in_order(places, blocks, groups, V, W):
    chains, done, runners = set(), [0] * blocks, 0
    for t in tasks(places, blocks, groups, V, W):
        if t[0] == "run":
            assert t[1] and not chains & set(t[1])
            chains |= set(t[1])
            runners += 1
        else:
            _, b, p = t
            assert p == done[b] and all((b, v) in chains for v in range(V))
            done[b] += 1
    assert done == [groups] * blocks
    assert chains == {(b, v) for b in range(blocks) for v in range(V)}
    assert runners + groups * blocks <= (groups + V) * blocks


def run(calls, slots):
    """Workgroups in the calls' orders as slots come free.  A place ends once it has
    started (all that it waits for has), a runner once all places of its blocks have.
    Whether all of them end."""
    most = [{t[1]: t[2] for t in c if t[0] == "place"} for c in calls]
    state = [dict(next=0, seen={}, running=[]) for _ in calls]
    moved = True
    while moved:
        moved = False
        for c, s in zip(calls, state):
            while slots and s["next"] < len(c):
                t = c[s["next"]]
                s["next"] += 1
                if t[0] == "place":
                    s["seen"][t[1]] = t[2]
                s["running"].append(t)
                slots -= 1
                moved = True
        for s, top in zip(state, most):
            stay = [t for t in s["running"]
                    if t[0] == "run" and any(s["seen"].get(b, -1) < top[b] for b, _ in t[1])]
            if len(stay) < len(s["running"]):
                slots += len(s["running"]) - len(stay)
                s["running"], moved = stay, True
    return all(s["next"] == len(c) and not s["running"] for c, s in zip(calls, state))


@pytest.mark.parametrize("blocks,groups,V,W", SHAPES)
def test_every_workgroup_ends(places, blocks, groups, V, W):
    most = places.runners()
    c = tasks(places, blocks, groups, V, W)
    assert run([c], most + 1)
    for n in (2, 4, 16):
        assert run([c] * n, n * most + 1)


@pytest.mark.parametrize("V", [1, 2])
def test_narrow_calls_bound_the_runners(places, V):
    """Each block's tasks in order, the blocks' in any (here the last block's first)."""
    most = places.runners()
    for blocks in range(1, 2 * most):
        assert places.narrow(blocks, V) == (blocks * V <= most)
        if places.narrow(blocks, V):
            assert places.all(blocks, 5, V, 8) == blocks * (V + 5)
            of = lambda b: [("run", [(b, v)]) for v in range(V)] + [("place", b, p)
                                                                    for p in range(5)]
            c = [t for b in range(blocks)[::-1] for t in of(b)]
            d = [t for row in zip(*(of(b) for b in range(blocks))) for t in row]
            assert run([c, d, d], 3 * most + 1)


def test_the_model_sees_a_call_that_hangs():
    """All blocks' runners before any place: they hold every slot."""
    c = [("run", [(b, 0)]) for b in range(1024)] + [("place", b, p) for p in range(3)
                                                   for b in range(1024)]
    assert not run([c], 512) and run([c], 1025)


def test_many_calls_at_once_on_the_chip(places):
    """Two workgroups a CU at least: 63 calls of 8,192 channels at a time."""
    assert 63 * places.runners() < 512
    assert run([tasks(places, 64, 2, 2, 8)] * 63, 512)
