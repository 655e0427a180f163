"""CPU-side checks of cser_layers.h: plain C, every declared function exported, exercised and bound, structs laid out alike."""
import ctypes
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "cser_layers.h")).read(), flags=re.S)


def test_header_is_plain_c_and_every_function_is_exported_and_used(tmp_path):
    import __graft_entry__
    __graft_entry__.build()
    pkg = os.path.join(ROOT, "paper_2007_13221_b200")
    exe = str(tmp_path / "abi_layers_c_check")
    src = os.path.join(ROOT, "tests", "abi_layers_c_check.c")
    res = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), src, "-o",
                          exe, "-L", pkg, "-l:libcser.so", "-Wl,-rpath," + pkg], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0, (run.returncode, run.stdout, run.stderr)
    names = set(re.findall(r"\b(cser_[a-z0-9_]+)\s*\(", HEADER))
    assert len(names) >= 10 and names <= set(re.findall(r"\b(cser_[a-z0-9_]+)\b", open(src).read()))
    lib = ctypes.CDLL(os.path.join(pkg, "libcser.so"))
    from paper_2007_13221_b200 import layers
    bound = layers.lib()
    for name in names:
        assert hasattr(lib, name), name
        assert getattr(bound, name).argtypes is not None, name


def test_the_structs_have_the_header_s_layout():
    """Fields of 8 bytes (or structs of those) in the header's order."""
    from paper_2007_13221_b200 import layers
    for name, struct, size in (("cser_rows", layers._Rows, 24), ("cser_pixels", layers._Pixels, 32), ("cser_norm_inputs", layers._NormInputs, 96)):
        body = re.search(r"typedef struct %s \{(.*?)\}" % name, HEADER, flags=re.S).group(1)
        names = [n for line in body.split(";") for n in re.findall(r"(\w+)\s*(?:,|$)", line.replace("*", " ").strip())]
        assert names == [f[0] for f in struct._fields_]
        assert ctypes.sizeof(struct) == size


def test_stamp_covers_the_layers_sources(tmp_path):
    """Their device and host code are headers of cser.cu: a changed one gives another id."""
    import shutil
    import __graft_entry__ as g
    src = os.path.join(ROOT, "paper_2007_13221_b200", "csrc")
    copy = shutil.copytree(src, tmp_path / "csrc")
    before = g.source_id(str(copy / "cser.cu"))
    for name in ("layers.cuh", "layer_common.cuh", "drop_kernels.cuh", "norm_kernels.cuh"):
        with open(copy / name, "a") as f:
            f.write("\n")
        after = g.source_id(str(copy / "cser.cu"))
        assert after != before, name
        before = after


def test_norms_of_too_many_groups_are_refused():
    """Before anything is allocated: the groups of all samples are numbered with 31 bits."""
    import pytest
    from paper_2007_13221_b200 import layers
    from paper_2007_13221_b200.binding import CSERError
    with pytest.raises(CSERError, match="2\\^31"):
        layers.GroupNorm(2, 2 ** 23, 256, 128)


def test_a_norm_with_a_dropout_needs_the_step():
    """Refused before anything else of a call is looked at; a norm without a dropout goes on to its arrays."""
    import pytest
    import torch
    from paper_2007_13221_b200 import layers
    from paper_2007_13221_b200.binding import CSERError
    op = object.__new__(layers.GroupNorm)
    op.h, op.n, op.max_samples, op.channels, op.groups, op.dtype = None, 1, 2, 8, 2, torch.float32
    x = torch.zeros((1, 2, 3, 8))
    for drops, match in ((True, "step"), (False, "CUDA")):
        op.drops = drops
        with pytest.raises(CSERError, match=match):
            op.apply(x)
        with pytest.raises(CSERError, match=match):
            op.grad(x, x, torch.zeros((2, 1, 2, 2)))


def test_numbers_that_the_c_types_would_cut_are_refused():
    """2^32 as an int32 is 0: another worker's mask, silently."""
    import pytest
    from paper_2007_13221_b200 import layers
    from paper_2007_13221_b200.binding import CSERError
    for kw in (dict(n_workers=2 ** 32 + 1), dict(max_rows=2 ** 64 + 1), dict(cols=2 ** 64 + 1), dict(first_worker=2 ** 32), dict(first_worker=-2 ** 32)):
        with pytest.raises(CSERError, match=next(iter(kw))):
            layers.Dropout(**{**dict(n_workers=1, max_rows=1, cols=1, p=0.5, seed=0, site=1), **kw})
    for kw in (dict(n_workers=2 ** 32 + 1), dict(max_samples=2 ** 64 + 1), dict(channels=2 ** 64 + 8), dict(groups=2 ** 64 + 2)):
        with pytest.raises(CSERError, match=next(iter(kw))):
            layers.GroupNorm(**{**dict(n_workers=1, max_samples=1, channels=8, groups=2), **kw})
