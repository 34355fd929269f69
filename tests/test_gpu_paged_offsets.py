"""sc_paged_append over batches some of whose offsets break the rules: a sequence is appended whole, or left as it is with its length where it was;
a sequence whose tokens start before an offset that stands in front of its own is left too, so no token is two sequences'."""
import pytest
import torch

import paged_plain as pp
from paper_2603_14303_b200 import binding

pytestmark = pytest.mark.gpu
DEV = pp.DEV


def _check(off, have, ps, W, bounds=False, seq_len=None):
    """Offsets and lengths as lists; every page, every query and every length is compared."""
    B, T = len(off) - 1, max(max(off), 1)
    P, d = B * W, 8
    gen = torch.Generator().manual_seed(B * 1000 + T)
    table = torch.randperm(P, generator=gen).to(torch.int32).view(B, W)
    k = torch.zeros((P, 1, ps, d), device=DEV)
    mn, mx = (torch.full((P, 1, d), 5.0, device=DEV) for _ in range(2)) if bounds else (None, None)
    cache = binding.PagedCache(k, k.clone(), table.to(DEV), None, mn, mx)
    new = 1.0 + torch.rand((T, 1, d), generator=gen)
    q_out = torch.full((T, 1, d), -1.0, device=DEV)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    status = pp.status_word()
    lens, _ = binding.paged_append(cache, new.to(DEV), new.to(DEV), i32(off), i32(have), seq_len=None if seq_len is None else i32(seq_len),
                                   q=new.to(DEV), q_out=q_out, status=status)
    want_k, want_q, want_len = torch.zeros((P, 1, ps, d)), torch.full((T, 1, d), -1.0), list(have)
    at_fault, top = 0, off[0]
    for b in range(B):
        top = max(top, off[b])
        n = off[b + 1] - off[b] if seq_len is None else seq_len[b]
        if off[b] < top or off[b] < 0 or not 0 <= n <= off[b + 1] - off[b]:
            at_fault += 1
            continue
        want_len[b] += n
        for i in range(n):
            row = have[b] + i
            want_k[int(table[b, row // ps]), 0, row % ps] = new[off[b] + i, 0]
            want_q[off[b] + i] = new[off[b] + i]
    assert lens.tolist() == want_len
    assert torch.equal(k.cpu(), want_k) and torch.equal(cache.v.cpu(), want_k) and torch.equal(q_out.cpu(), want_q)
    assert int(status) == (binding.SC_ERR_INVALID_ARG if at_fault else binding.SC_OK)


@pytest.mark.parametrize("ps", [1, 4, 80])
@pytest.mark.parametrize("off", [(0, 6, 0, 6), (0, 100, 0, 100, 0, 100), (0, 100, 50, 100, 130), (0, 9, -3, 9, 20), (40, 3, 3, 41, 44), (5, 0, 2, 5, 9), (0, 7, 7, 9, 9)])
def test_sequences_behind_a_fall(off, ps):
    _check(list(off), [3 * b for b in range(len(off) - 1)], ps, 120 // ps + 1)


@pytest.mark.parametrize("bounds", [False, True])
@pytest.mark.parametrize("falls", [(3,), (255,), (256,), (257,), (100, 300), (511, 512), (599,), ()])
def test_falls_in_batches_of_several_rounds(falls, bounds):
    """Single tokens; at a fall the offsets go back by twenty, so the sequences that follow are at fault until the offsets are back."""
    off = [0]
    for b in range(600):
        off.append(off[-1] + 1 if b not in falls else max(off[-1] - 20, 0))
    _check(off, [b % 5 for b in range(600)], 4, 2, bounds)


def test_sequences_without_tokens_in_between():
    """Many sequences, few of which have tokens: every length is told."""
    n = [2 if b % 97 == 0 else 0 for b in range(1500)]
    off = [0]
    for m in n:
        off.append(off[-1] + m)
    _check(off, [1] * 1500, 4, 1)
    _check([0] * 1501, [2] * 1500, 4, 1)
    _check([0, *([0] * 1499), 3], [1] * 1500, 4, 1)


def test_shorter_than_their_ranges_behind_a_fall():
    _check([0, 10, 4, 12, 20], [0] * 4, 4, 5, seq_len=[5, 0, 2, 3])
