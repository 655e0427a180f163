"""How the layers' launches are cut (layer_plan.h), checked on the host for sizes that no test could hold on a GPU."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Resident(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int) for k in ("sv", "log_tx", "log_block", "log_cluster", "slots", "fold", "log_sub")] + \
               [("group_magic", ctypes.c_uint32), ("per", ctypes.c_int), ("slices", ctypes.c_uint32), ("units", ctypes.c_uint32)]


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("plan") / "plan.so")
    res = subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wno-unused-function", "-shared", "-fPIC", "-I",
                          os.path.join(ROOT, "paper_2007_13221_b200", "csrc"), os.path.join(ROOT, "tests", "layer_plan_check.cpp"), "-o", out],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    lib = ctypes.CDLL(out)
    i64, i32 = ctypes.c_int64, ctypes.c_int
    lib.drop_sums.restype, lib.drop_sums.argtypes = i64, [i64, i64, i32, i32]
    lib.drop_used.restype, lib.drop_used.argtypes = i64, [i64, i64, i32, i32, i32]
    return lib


def plan(rules, size, n, samples, pixels, channels, groups, drop, v, two, preset=0):
    """(plan, bytes of shared memory) or None."""
    r, shared = Resident(), ctypes.c_uint64()
    found = rules.plan_norm((ctypes.c_int64 * 7)(size, n, samples, pixels, channels, groups, drop), v, int(two), ctypes.c_uint64(preset),
                            ctypes.byref(shared), ctypes.byref(r))
    return (r, shared.value) if found else None


@pytest.mark.parametrize("preset", [0, 1000, 2 ** 64 - 1])
@pytest.mark.parametrize("size,pixels,channels,groups", [(4, 4_300_000, 64, 1), (2, 640_000, 1024, 1), (2, 25_000_000, 32, 1), (4, 2 ** 31 - 1, 4, 1)])
def test_samples_of_too_many_pixels_are_refused_whatever_memory_held_before(rules, size, pixels, channels, groups, preset):
    for two in (False, True):
        for drop in (False, True):
            assert plan(rules, size, 1, 1, pixels, channels, groups, drop, 16 // size, two, preset) is None


def test_a_plan_holds_what_it_is_for(rules):
    """Slots for every pixel of a block, blocks for every pixel of a sample, slices of whole groups for every channel."""
    for size, v in ((2, 8), (2, 4), (2, 2), (4, 4), (4, 2), (4, 1)):
        for channels, groups in ((64, 32), (64, 1), (96, 3), (1000, 125), (2048, 64), (120, 120), (24, 24)):
            if channels % v:
                continue
            for pixels in (1, 2, 31, 64, 100, 784, 3136, 12544, 70000, 10 ** 7):
                for n, samples, two, drop in ((1, 1, True, True), (8, 16, False, False), (8, 16, True, False), (2, 700, True, True)):
                    got = plan(rules, size, n, samples, pixels, channels, groups, drop, v, two)
                    if got is None:
                        continue
                    r, _ = got
                    assert r.log_block in (7, 8) and 0 <= r.log_cluster <= 3 and r.sv <= 1 << r.log_tx <= 128
                    assert r.per << r.log_cluster >= pixels and r.slots << (r.log_block - r.log_tx) >= r.per
                    assert r.slices * r.sv * v >= channels and r.units == n * samples * r.slices
                    assert r.sv * v % (channels // groups) == 0


def test_no_plan_needs_more_shared_memory_than_a_block_has(rules):
    """220 KB, which is what the kernels are allowed; few units of wide slices are spread over more blocks, whose exchanged sums take more."""
    for size in (2, 4):
        for v in [k for k in (1, 2, 4, 8) if 4 <= k * size <= 16]:
            for drop in (False, True):
                for two in (False, True):
                    for per_group in (1, 3, 8, 12, 64, 100, 128, 256, 300, 512, 1000, 1024):
                        for groups in (1, 2, 4, 32):
                            if per_group * groups % v:
                                continue
                            for samples in (1, 8, 74, 1000):
                                for pixels in (1, 7, 20, 49, 64, 97, 100, 104, 108, 112, 120, 196, 400, 784, 1000, 3136):
                                    got = plan(rules, size, 1, samples, pixels, per_group * groups, groups, drop, v, two)
                                    assert got is None or got[1] <= 220 * 1024, (size, v, drop, two, per_group, groups, samples, pixels)


SUMS = [(1, 1), (1, 1001), (1, 2 ** 20 + 1), (1, 2 ** 30 + 1), (2, 1001), (7, 10001), (8, 10001), (9, 1001), (100, 10001), (33, 64), (1000, 1), (65536, 3),
        (10 ** 6, 7), (4096, 1024), (8192, 4096), (77, 201), (9999, 1111), (2 ** 20, 16384), (2 ** 34, 1), (5, 2 ** 31 + 5)]


@pytest.mark.parametrize("n", [1, 8, 300])
@pytest.mark.parametrize("v", [4, 8])
def test_a_dropout_s_workspace_is_as_small_as_stated(rules, n, v):
    """4 bytes for every 128 elements, 1.3 MB at most where there are few, and a walked row (v rows, or 32 vectors and a row of them) a worker."""
    for rows, cols in SUMS:
        if rows * cols * n > 2 ** 34:
            continue
        got, folded = 4 * n * rules.drop_sums(rows, cols, n, v), v * cols if rows >= v else cols
        assert got <= 4 * n * rows * cols / 128 + 1.3e6 + 4 * n * (folded + 32 * v + cols), (rows, cols, got)
        if rows == 1:
            assert got == 0


@pytest.mark.parametrize("v", [4, 8])
def test_a_dropout_s_workspace_holds_any_call(rules, v):
    for n in (1, 3, 64):
        for most, cols in SUMS:
            room = rules.drop_sums(most, cols, n, v)
            for rows in {1, 2, 3, 7, 8, 9, 31, 32, 33, 100, 129, most // 3, most // 2, most - 1, most}:
                if 1 <= rows <= most:
                    for dense in (0, 1):
                        assert rules.drop_used(rows, cols, n, v, dense) <= room, (n, most, cols, rows, dense)


def places(a):
    at, run, sizes, strides = a
    got = set()
    for i in range(sizes[0]):
        for j in range(sizes[1]):
            for k in range(sizes[2]):
                first = at + i * strides[0] + j * strides[1] + k * strides[2]
                got.update(range(first, first + run))
    return got


def test_whether_arrays_share_memory_is_known(rules):
    """Against every element: exact where arrays are alike or one has no gaps, and never wrong where it says that they share."""
    import random
    rng = random.Random(5)
    counts = {}
    for _ in range(20000):
        sizes, run = [rng.choice([1, 1, 2, 3, 5]) for _ in range(3)], rng.choice([1, 2, 4, 7])
        arrays = []
        for written in (True, False):
            strides, inner = [0, 0, 0], run
            for k in rng.sample(range(3), 3):
                pad = rng.choice([0, 0, 1, run, 9])
                strides[k] = inner + pad
                inner = strides[k] * (sizes[k] - 1) + inner
                if not written and rng.random() < 0.1:
                    strides[k] = rng.choice([0, 1])
            arrays.append((rng.randrange(0, 60), run, sizes, strides))
        if rng.random() < 0.5:
            arrays[1] = (arrays[1][0], run, sizes, arrays[0][3])
        one, other = (places(a) for a in arrays)
        raw = [(ctypes.c_int64 * 8)(a[0], a[1], *[v for pair in zip(a[2], a[3]) for v in pair]) for a in arrays]
        is_same = ctypes.c_int()
        got, share = bool(rules.arrays_share(*raw, ctypes.byref(is_same))), bool(one & other)
        like = all(s == 1 or p == q for s, p, q in zip(sizes, arrays[0][3], arrays[1][3]))
        gapless = any(max(p) - min(p) + 1 == len(p) for p in (one, other))
        nested = len(other) == run * sizes[0] * sizes[1] * sizes[2]
        if like or gapless and nested:
            assert got == share, arrays
        assert share or not got, arrays
        assert not is_same.value or one == other
        counts[like, gapless, share] = counts.get((like, gapless, share), 0) + 1
    assert all(counts.get((a, b, c), 0) > 100 for a in (False, True) for b in (False, True) for c in (False, True)), counts
