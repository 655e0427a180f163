"""CPU-side checks of cser_train.h: plain C, every declared function exported, exercised and bound."""
import ctypes
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "cser_train.h")).read(), flags=re.S)
    return set(re.findall(r"\b(cser_[a-z0-9_]+)\s*\(", text))


def test_header_is_plain_c_and_every_function_is_exported_and_used(tmp_path):
    import __graft_entry__
    __graft_entry__.build()
    pkg = os.path.join(ROOT, "paper_2007_13221_b200")
    exe = str(tmp_path / "abi_train_c_check")
    src = os.path.join(ROOT, "tests", "abi_train_c_check.c")
    res = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), src, "-o",
                          exe, "-L", pkg, "-l:libcser.so", "-Wl,-rpath," + pkg], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0, (run.returncode, run.stdout, run.stderr)
    names = declared()
    assert len(names) >= 10 and names <= set(re.findall(r"\b(cser_[a-z0-9_]+)\b", open(src).read()))
    lib = ctypes.CDLL(os.path.join(pkg, "libcser.so"))
    from paper_2007_13221_b200 import train
    bound = train.lib()
    for name in names:
        assert hasattr(lib, name), name
        assert getattr(bound, name).argtypes is not None, name


def test_the_struct_of_inputs_has_the_header_s_layout():
    """Nine 8-byte fields in the header's order."""
    from paper_2007_13221_b200 import train
    text = open(os.path.join(ROOT, "include", "cser_train.h")).read()
    body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct cser_xent_inputs \{(.*?)\}", text, flags=re.S).group(1), flags=re.S)
    names = [n for line in body.split(";") for n in re.findall(r"(\w+)\s*(?:,|$)", line.replace("*", " ").strip())]
    assert names == [f[0] for f in train._XentInputs._fields_]
    assert ctypes.sizeof(train._XentInputs) == 8 * len(names)


def test_stamp_covers_all_sources_of_the_library():
    import __graft_entry__ as g
    src = os.path.join(ROOT, "paper_2007_13221_b200", "csrc", "cser.cu")
    assert {os.path.basename(f) for f in g.sources_of(src)} == {"cser.cu", "orth.cu", "xent.cu"}
