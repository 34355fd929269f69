"""The joining of a paged decode's partial sums where a cluster goes through several units: blocks hand each other slices segment after segment, and one
of them may be late."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2603_14303_b200 import binding, build

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HERE = os.path.dirname(os.path.abspath(__file__))
MS = 1_000_000
HEADS, D, PART = 3, 64, 8 * 64 + 16     # of the probe; floats of a partial sum


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("join") / "probe.so")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, *build.NVCC_FLAGS, "-Xcompiler", "-fvisibility=default", "-shared", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                    os.path.join(HERE, "paged_join_probe.cu"), "-o", lib], check=True)
    run = ctypes.CDLL(lib).run_probe
    run.argtypes = [ctypes.c_void_p] + [ctypes.c_int] * 5 + [ctypes.c_longlong, ctypes.c_ulonglong] + [ctypes.c_void_p] * 6

    def call(rows, parties, cluster, late=0, segment=0, delay_ms=0.0, limit_ms=500.0):
        out = torch.full((len(rows), HEADS, D), -1.0, device=DEV)
        tickets = torch.zeros(1024, dtype=torch.int32, device=DEV)
        part = torch.full((2 * parties * PART,), float("inf"), device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        left = torch.zeros(parties * cluster, dtype=torch.int64, device=DEV)
        lens = torch.tensor(rows, dtype=torch.int32, device=DEV)
        assert run(lens.data_ptr(), len(rows), parties, cluster, late, segment, int(delay_ms * MS), int(limit_ms * MS), out.data_ptr(), tickets.data_ptr(),
                   part.data_ptr(), status.data_ptr(), left.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert int(tickets.count_nonzero()) == 0          # left as they were, whatever happened
        return out.double().cpu().numpy(), int(status), left.cpu().numpy()
    return call


def segments(rows, parties, cluster):
    """The units of each party's stretch, in order."""
    tiles = [((n - 1) // 64 + 1) * 4 for n in rows]
    ends = np.cumsum(tiles)
    stretch = max(-(-int(ends[-1]) // parties), cluster * 8)
    assert not (stretch < 64 * cluster and len(rows) <= parties)      # (a line cut at the units' ends has one segment per party)
    return [[u for u, e in enumerate(ends) if e > p * stretch and e - tiles[u] < (p + 1) * stretch] for p in range(parties)]


def expected(rows, parties, cluster):
    out = np.zeros((len(rows), HEADS, D))
    seg = segments(rows, parties, cluster)
    column = np.arange(D)
    for u in range(len(rows)):
        for h in range(HEADS):
            num, den = np.zeros(D), 0.0
            for p in range(parties):
                if u in seg[p]:
                    for r in range(cluster):
                        w = 2.0 ** ((u + p * 3 + r * 2 + h) % 5 - 2)
                        num, den = num + w * ((u * 7 + p * 13 + r * 29 + h * 3 + column) % 97) / 16.0, den + w * (1 + r)
            out[u, h] = num / den
    return out


LINES = [([300] * 5, 1, 2), ([64, 900, 1, 130, 700, 64, 64], 1, 4), ([500, 70, 64, 900, 640, 200, 1000], 2, 4), ([2000, 64, 64, 64, 64, 64, 2000, 130, 130], 2, 8),
         ([100] * 12, 3, 3)]


@pytest.mark.parametrize("rows,parties,cluster", LINES)
def test_segment_after_segment(probe, rows, parties, cluster):
    """At least three in a row: the receiving places and the barriers' phases come round again."""
    assert max(len(s) for s in segments(rows, parties, cluster)) >= 3
    out, status, _ = probe(rows, parties, cluster)
    assert status == binding.SC_OK
    np.testing.assert_allclose(out, expected(rows, parties, cluster), rtol=1e-5)   # (fp32 sums of at most 16 parts)


@pytest.mark.parametrize("rows,parties,cluster", LINES)
@pytest.mark.parametrize("segment", [0, 1, 2])
def test_a_block_later_than_one_limit(probe, rows, parties, cluster, segment):
    """The clock of a wait runs on while a context is switched off: a wait is given a second turn."""
    out, status, _ = probe(rows, parties, cluster, late=1, segment=segment, delay_ms=75, limit_ms=50)
    assert status == binding.SC_OK
    np.testing.assert_allclose(out, expected(rows, parties, cluster), rtol=1e-5)


def _late_by_too_much(probe, rows, parties, cluster, segment, late):
    """`late` (of the first cluster) is later than both limits.  What is a number is right, the rest is what it has to be."""
    want, seg = expected(rows, parties, cluster), segments(rows, parties, cluster)
    out, status, left = probe(rows, parties, cluster, late=late, segment=segment, delay_ms=150, limit_ms=30)
    assert status == binding.SC_ERR_TIMEOUT
    fine = np.isfinite(out)
    np.testing.assert_allclose(out[fine], want[fine], rtol=1e-5)
    mine = seg[0]
    for p in range(1, parties):                                     # the other clusters' own units
        for u in seg[p]:
            assert u in mine or fine[u].all()
    for u in mine[:segment]:                                        # before it was late
        assert fine[u].all()
    n4 = HEADS * D // 4
    size = -(-n4 // cluster)
    own = np.zeros(n4, bool)
    own[late * size:(late + 1) * size] = True                       # the late block's slice, for which it had everybody's sums
    own = np.repeat(own, 4).reshape(HEADS, D)
    for i, u in enumerate(mine[segment:]):
        shared = any(u in seg[p] for p in range(1, parties))
        if i > 0:
            assert not fine[u].any()
        else:
            assert not fine[u][~own].any() and (shared or fine[u][own].all())
    if segment == len(mine) - 1:                                    # those that gave up leave after the one that did not
        assert (left[:cluster] >= left[late] - 5 * MS).all()
    return out


@pytest.mark.parametrize("rows,parties,cluster", LINES)
@pytest.mark.parametrize("segment", [0, 1, 2, -1])
def test_a_block_later_than_both_limits(probe, rows, parties, cluster, segment):
    """From the segment on that it was late for nothing is handed on: no sum is made of two segments' slices."""
    _late_by_too_much(probe, rows, parties, cluster, segment % len(segments(rows, parties, cluster)[0]), late=1)


def test_any_block_may_be_late(probe):
    rows, parties, cluster = LINES[3]
    for late in range(cluster):
        _late_by_too_much(probe, rows, parties, cluster, 3, late)
        out, status, _ = probe(rows, parties, cluster)              # and the next launch is as if nothing had been
        assert status == binding.SC_OK
        np.testing.assert_allclose(out, expected(rows, parties, cluster), rtol=1e-5)


def test_a_shared_unit_one_of_whose_parts_is_not_complete(probe):
    """The unit that two clusters share, with the first one late for it: whoever joins the parts, they give NaN."""
    rows, parties, cluster = LINES[2]
    seg = segments(rows, parties, cluster)
    shared = seg[0][-1]
    assert shared in seg[1]
    out = _late_by_too_much(probe, rows, parties, cluster, len(seg[0]) - 2, late=2)   # late for the one before: nothing of the shared one is handed on
    assert np.isnan(out[shared]).all()
