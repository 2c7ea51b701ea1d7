"""Host plan of the adapters (CPU): a C++ program compiled against the built library
(tests/native/adapter_plan_check.cpp) checks that every row is done once, by its
adapter, and that a tile's buffers keep apart, aligned and within a CTA's memory."""
import os
import random
import shutil
import subprocess

import pytest

from test_boundary_cpu import ppas  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2608_15171_gb300")


@pytest.fixture(scope="module")
def checker(ppas, tmp_path_factory):  # noqa: F811
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path_factory.mktemp("aplan") / "adapter_plan_check")
    cmd = [gxx, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"),
           "-I", "/usr/local/cuda/include", os.path.join(ROOT, "tests", "native", "adapter_plan_check.cpp"),
           "-o", exe, "-L", PKG, "-lppas", f"-Wl,-rpath,{PKG}", "-L/usr/local/cuda/lib64", "-lcudart"]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    return exe


def _run(exe, cases):
    text = "".join(f"plan {int(copies)} {rows} {total} {len(lens)} " + " ".join(f"{n} {a}" for n, a in zip(lens, ids)) + "\n"
                   for copies, rows, total, lens, ids in cases)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(cases)
    for line, case in zip(out, cases):
        assert line.startswith("ok "), (line, case)
    return [[int(x) for x in line.split()[1:]] for line in out]


def test_shapes(checker):
    out = subprocess.run([checker], input="shapes\n", capture_output=True, text=True, check=True).stdout
    assert out.startswith("ok "), out


def test_known_plans(checker):
    never = 2 ** 31 - 1
    got = _run(checker, [
        (True, 48, 513, [1], [0]),
        (True, 48, 513, [1, 1, 1, 1], [0, 1, 0, 1]),       # two units of listed rows
        (False, 48, 513, [5, 3], [-1, -1]),                # nothing to do
        (True, 48, 513, [40, 30], [-1, -1]),               # one run, copied 32 rows at a time
        (True, 48, 513, [300, 300], [2, 2]),               # one run: 4 tiles of 128, one of 88
        (True, 48, 513, [512], [0]),                       # too few rows for tiles
        (True, 48, 513, [513], [0]),
        (True, never, 513, [600], [0]),
        (True, 48, 513, [600, 1, 1, 47], [0, 1, 0, 1]),    # short runs beside tiles
    ])
    assert got == [[1, 0, 0], [2, 2, 0], [0, 0, 0], [3, 0, 0], [0, 0, 5], [32, 0, 0], [0, 0, 5], [38, 0, 0], [4, 1, 5]]


def test_random_plans(checker):
    rng = random.Random(5)
    cases = []
    for _ in range(400):
        n = rng.choice([1, 2, 5, 30, 200])
        lens = [rng.choice([1, 1, 1, 2, 7, 15, 16, 17, 47, 48, 49, 128, 200, 700]) for _ in range(n)]
        ids = [rng.randrange(-1, rng.choice([1, 3, 50])) for _ in range(n)]
        cases.append((rng.random() < 0.5, rng.choice([48, 48, 128, 2 ** 31 - 1]), rng.choice([1, 513, 2000]), lens, ids))
    _run(checker, cases)
