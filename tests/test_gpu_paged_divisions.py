"""sc_paged_decode_attn over lines that are divided in every way the launch has, with one row that rules the softmax, at the edges of every tile by turns:
a row that is lost, or read twice from another place, changes an output from one row's values to another's.  And the same divisions against
Eq. 4 in 64 bits."""
import math

import pytest
import torch

import paged_plain as pp
from helpers import TOL, assert_close_vectors
from paper_2603_14303_b200 import binding

pytestmark = pytest.mark.gpu
DEV = pp.DEV
BF, F32 = torch.bfloat16, torch.float32
GENERIC = binding.SC_FLAG_GENERIC

# name: type, KV heads, queries of each, d, page size, lengths, flags, entries per table beyond the longest sequence
CASES = {
    # more than 64 units, of more than 192 tiles on the average: one block per SM (17 x 8 units on 148 blocks: several segments each)
    "one block per SM": (BF, 8, 4, 128, 16, [5000 - 111 * b for b in range(17)], 0, 2),
    "one block per SM, d = 64, eight queries": (BF, 6, 8, 64, 32, [4000 + 77 * b for b in range(12)], 0, 2),
    "one block per SM, uneven": (BF, 4, 4, 128, 16, [30000, 1, 17000, 64, 9000, 65, 8000, 0, 20000, 500, 700, 9001, 13, 4000, 4000, 4001, 12000], 0, 2),
    # 17 to 64 units of more than 512 tiles: clusters of four, a segment or a few each
    "clusters, 32 long units": (BF, 8, 4, 128, 16, [9000, 12345, 8500, 9001], 0, 2),
    "clusters, 20 long units": (BF, 4, 7, 128, 64, [10007, 9000, 16000, 8200, 11111], 0, 2),
    "clusters, cut at the units' ends": (BF, 2, 4, 128, 16, [82500, 7, 7, 130, 7, 64, 65, 1, 7, 9000], 0, 2),
    "clusters, cut, pages that split tiles": (BF, 2, 4, 64, 24, [82500, 7, 7, 130, 7, 64, 65, 1, 7, 9000], 0, 2),
    "clusters, 20 long units, generic kernel": (F32, 4, 2, 64, 24, [10007, 9000, 16000, 8200, 11111], 0, 2),
    # clusters whose stretches go through many units: receiving places and barriers' phases come round again
    "clusters through many units": (BF, 2, 4, 128, 16, [82400, 7, 7, 130, 7, 64, 65, 1, 9000, 42000, 0, 64, 500], 0, 2),
    "clusters through many units, 64 units": (BF, 4, 8, 128, 16, [40000, 7, 64, 1, 20000, 130, 30000, 5, 65, 12000, 700, 20000, 3, 9000, 64, 500], 0, 2),
    "clusters through many units, d = 256": (BF, 4, 4, 256, 16, [20000, 5, 64, 16000, 1, 130, 20000, 9000, 700, 18000], 0, 2),
    "clusters through many units, float32": (F32, 1, 4, 256, 24, [60000, 5, 300, 65, 0, 130, 1, 40000, 700, 40, 33000, 2000], 0, 2),
    "clusters through many units, generic kernel": (BF, 2, 8, 256, 16, [60000, 5, 300, 7000, 1, 40000, 700, 33000], GENERIC, 2),
    # up to 16 units: clusters too, cut at the units' ends
    "16 units, one of them long": (BF, 2, 4, 128, 16, [20000] + [5] * 7, 0, 2),
    "16 units, the last one long": (BF, 2, 8, 128, 16, [5, 64, 65, 0, 130, 1, 700, 20000], 0, 2),
    "16 units, d = 256": (BF, 1, 4, 256, 16, [5, 300, 65, 0, 130, 1, 9000, 700, 40, 40, 40, 2000], 0, 2),
    "16 units, float32": (F32, 2, 4, 128, 16, [9000, 5, 700, 3000, 64, 1, 333, 20], 0, 2),
    "16 units, generic kernel": (BF, 2, 8, 96, 24, [333, 5, 700, 6000, 64, 1, 9000, 20], 0, 2),
    "16 units, generic kernel forced": (BF, 2, 4, 128, 16, [20000] + [5] * 7, GENERIC, 2),
    # the same short sequences in narrow tables (clusters of eight) and in tables for 128 K rows (of four)
    "short, narrow tables": (BF, 8, 4, 128, 16, [2047], 0, 1),
    "short, wide tables": (BF, 8, 4, 128, 16, [2047], 0, 8192),
    "16 short units, narrow tables": (BF, 8, 4, 128, 16, [2300, 1700], 0, 1),
    "16 short units, wide tables": (BF, 8, 4, 128, 16, [2300, 1700], 0, 8192),
    "short, wide tables, float32": (F32, 4, 2, 64, 24, [2000, 1, 700], 0, 5000),
    # many units: spare rounds
    "many short units": (BF, 8, 4, 128, 16, [20 + 3 * b for b in range(80)], 0, 2),
    "short units, cut at their ends": (BF, 8, 4, 128, 16, [100 + 31 * b for b in range(20)], 0, 2),
}


def _cache(dtype, H, d, ps, lens, extra, spread):
    gen = torch.Generator(device=DEV).manual_seed(7)
    need = [-(-n // ps) for n in lens]
    W, P = max(need) + extra, sum(need) + 1
    perm = torch.randperm(P, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(lens), W), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = perm[at:at + m]
        at += m
    k, v = ((torch.randn((P, ps, H, d), generator=gen, device=DEV) * s).to(dtype).transpose(1, 2) for s in (spread, 1.0))
    return binding.PagedCache(k, v, table), torch.tensor(lens, dtype=torch.int32, device=DEV), int(perm[at])   # (and a page that no table names)


@pytest.mark.parametrize("name", CASES)
def test_a_row_that_rules(name):
    """Query g of a head looks along axis g, where the row it is to find has a key of its own: the output is that row's value, to the last bit
    but where that is zero.  By arithmetic: the row scores strong^2 / sqrt(d) > 59.7 (strong rounded to bf16: 21.875, 24.25, 26, 31), the others at
    most strong * 0.05 * 6 / sqrt(d) < 0.9, so each of at most 82500 adds less than e^-58.8 of |v| <= 6.5: 2e-20 together.  Half a step of a value
    that is not zero (above 1e-8 here) is more than 1e-16; a value of zero may become that sum."""
    dtype, H, G, d, ps, lens, flags, extra = CASES[name]
    cache, ln, spare = _cache(dtype, H, d, ps, lens, extra, 0.05)
    B, strong = len(lens), float(torch.tensor(math.sqrt(60 * math.sqrt(d))).to(dtype))
    q = torch.zeros((B, H, G, d), dtype=dtype, device=DEV)
    for g in range(G):
        q[:, :, g, g] = strong
    q = q.view(B, H * G, d)
    ws, status, out = binding.paged_decode_workspace(B, H * G, H, d, DEV), pp.status_word(), torch.empty_like(q)
    tiles = ((ln.long() + 15) // 16).view(B, 1, 1)
    bi, hi, gi = (torch.arange(n, device=DEV).view(s) for n, s in ((B, (B, 1, 1)), (H, (1, H, 1)), (G, (1, 1, G))))
    live = (ln > 0).view(B, 1, 1, 1).expand(B, H, G, d)
    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    for i in range(-(-2 * max(-(-n // 16) for n in lens) // G)):
        at = i * G + gi + 5 * hi                                          # edge by edge: first and last row of each tile, heads apart
        row = torch.minimum(at // 2 % tiles.clamp(min=1) * 16 + at % 2 * 15, (ln.long() - 1).view(B, 1, 1)).clamp(min=0)
        page = torch.where(live[..., 0], cache.table[bi, row // ps].long(), spare)
        r = row % ps
        old = cache.k[page, hi, r, gi]
        cache.k[page, hi, r, gi] = torch.where(live[..., 0], strong, old)
        binding.paged_decode_attn(q, cache, ln, out=out, workspace=ws, status=status, flags=flags)
        want = torch.where(live, cache.v[page, hi, r], 0.0)
        wrong += ((out.view(B, H, G, d).double() - want.double()).abs() > 2e-20).sum()
        cache.k[page, hi, r, gi] = old
    pp.ok(status)
    assert int(wrong) == 0
    assert int(ws[:4096].count_nonzero()) == 0


@pytest.mark.parametrize("name", CASES)
def test_against_the_formula(name):
    dtype, H, G, d, ps, lens, flags, extra = CASES[name]
    cache, ln, _ = _cache(dtype, H, d, ps, lens, extra, 1.0)
    B = len(lens)
    q = torch.randn((B, H * G, d), generator=torch.Generator().manual_seed(1)).to(dtype).to(DEV)
    runs = [binding.paged_decode_attn(q, cache, ln, flags=flags) for _ in range(2)]
    assert pp.same_bits(*runs)
    want = torch.zeros((B, H, G, d), dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        ids = cache.table[b, :-(-n // ps)].long()
        for h in range(H if n else 0):
            k, v = (t[ids, h].reshape(-1, d)[:n].double() for t in (cache.k, cache.v))
            want[b, h] = torch.softmax(q[b, h * G:(h + 1) * G].double() @ k.T / math.sqrt(d), 1) @ v
    assert_close_vectors(runs[0].double().cpu().numpy(), want.view(B, H * G, d).cpu().numpy(), TOL[dtype], name)
