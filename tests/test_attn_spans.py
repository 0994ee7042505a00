"""The search for a token's document, run on the CPU (tests/host/spans.cpp),
where a signed overflow ends the program."""

import bisect
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


@pytest.fixture(scope="module")
def search(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("spans") / "spans")
    r = subprocess.run([HIPCC, "-std=c++17", "-O1", "-ftrapv", "--offload-host-only", "-I",
                        os.path.join(ROOT, "paper_2607_14530_amd", "csrc"),
                        os.path.join(ROOT, "tests", "host", "spans.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(cases):
        text = "".join(f"{n} {t} {len(p)} " + " ".join(f"{i} {s}" for i, s in p) + "\n" for n, t, p in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True)
        assert out.returncode == 0, (out.returncode, out.stderr)
        return [int(x) for x in out.stdout.split()]
    return run


def test_small(search):
    r = random.Random(1)
    cases, want = [], []
    for _ in range(300):
        n = r.randrange(0, 20)
        starts = sorted(r.randrange(-3, 30) for _ in range(n + 1))
        t = r.randrange(0, 32)
        cases.append((n, t, list(enumerate(starts))))
        want.append(max(0, bisect.bisect_right(starts, t) - 1))
    assert search(cases) == want


def test_as_many_documents_as_their_number_holds(search):
    """Nearly all of them empty: the indices' sum passes 31 bits on the way."""
    cases, want = [], []
    for n in (2 ** 30 - 1, 2 ** 30, 2 ** 30 + 7, 2 ** 31 - 2, 2 ** 31 - 1):
        cases += [(n, 5, [(n, 9)]), (n, 5, [(n - 2, 5), (n - 1, 6)]), (n, 9, [(n, 9)]), (n, 5, [(n, 5)])]
        want += [n - 1, n - 2, n, n]
    assert search(cases) == want
