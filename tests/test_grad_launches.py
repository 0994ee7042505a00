"""The launches of the gradient norm and clip, recorded on the CPU
(tests/host/grad_launches.cpp): every chunk's sum has a place in the workspace
and every tensor its chunks, in the norm's pass and in the clip's."""

import os
import shutil
import subprocess

import pytest

from paper_2607_14530_amd import xhc as X

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
CHUNKS = 16384


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("grad") / "grad_launches")
    r = subprocess.run([HIPCC, "-std=c++17", "-O1", "--offload-host-only",
                        "-I", os.path.join(ROOT, "paper_2607_14530_amd", "csrc"), "-I", os.path.join(ROOT, "include"),
                        os.path.join(ROOT, "tests", "host", "grad_launches.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(counts, clip=True):
        line = " ".join(map(str, [int(clip), len(counts), *counts]))
        out = subprocess.run([exe], input=line, capture_output=True, text=True)
        assert out.returncode == 0, out.stderr
        return [line.split() for line in out.stdout.splitlines()]
    return run


def tensors(words):
    """(index, elements, first chunk) of a launch's tensors"""
    v = list(map(int, words))
    return list(zip(v[::3], v[1::3], v[2::3]))


def check(record, counts, clip=True):
    lines = record(counts, clip)
    assert lines[0][0] == "places" and lines[-1] == ["end", "0"]
    places, chunk = int(lines[0][1]), int(lines[0][3])
    assert X.xhc_grad_workspace_bytes(len(counts)) == 16 + 8 * places
    assert chunk % 2048 == 0 and chunk >= 8192
    wanted = [(i, c) for i, c in enumerate(counts) if c]

    def walk(launches, at):
        """The tensors of the launches in turn; each launch has a chunk, and each tensor all of its own."""
        seen = []
        for grid, table in launches:
            assert 1 <= grid
            first = 0
            for i, c, f in table:
                assert f == first
                first += -(-c // chunk)
                seen.append((i, c))
            assert first == grid
            at += grid
        return seen, at

    squares = [(int(w[2]), tensors(w[3:])) for w in lines if w[0] == "squares"]
    starts = [int(w[1]) for w in lines if w[0] == "squares"]
    seen, total = walk(squares, 0)
    assert seen == wanted
    assert starts == [sum(g for g, _ in squares[:k]) for k in range(len(squares))]
    assert total <= places, (total, places)                     # every sum has a place
    norms = [w for w in lines if w[0] == "norm"]
    scales = [w for w in lines if w[0] == "scale"]
    if not clip:
        assert norms == [["norm", str(total), "0"]] and not scales
        return
    assert all(int(w[3]) == total for w in scales)
    own = [w[2] for w in scales]
    assert (norms == [["norm", str(total), "1"]] and set(own) <= {"0"}) or (not norms and own == ["1"])
    seen, _ = walk([(int(w[1]), tensors(w[4:])) for w in reversed(scales)], 0)
    assert seen == wanted


@pytest.mark.parametrize("q", [8192, 10240, 12288, 14336, 1 << 20])
@pytest.mark.parametrize("more", [-1, 0, 1, 8190, 16383, 16384])
def test_every_sum_has_a_place(record, q, more):
    """Totals around a multiple of the number of chunks, in one tensor and in
    several whose last chunks are short."""
    total = CHUNKS * q + more
    for counts in ([total], [1, total - 1], [total - 1, 1], [q + 1] * 50 + [total - 50 * (q + 1)], [total // 3] * 3):
        check(record, counts)
        check(record, counts, clip=False)


def test_the_largest_total(record):
    check(record, [1 << 40])
    check(record, [(1 << 40) - 4095] + [1] * 4095)


@pytest.mark.parametrize("full", [0, 1, 127, 128, 129, 256, 384])
@pytest.mark.parametrize("empty", [0, 1, 127, 128, 300])
def test_empty_tensors_at_any_place(record, full, empty):
    """Empty tensors before, behind and between the others: no launch without
    a chunk, none left out."""
    some = [5 + 9000 * (i % 3) for i in range(full)]
    mixed = [c for i in range(max(full, empty)) for c in some[i:i + 1] + [0] * (i < empty)]
    for counts in (some + [0] * empty, [0] * empty + some, mixed):
        check(record, counts)
        check(record, counts, clip=False)
