"""sc_paged_select against bounds in 64 bits, and sparse attention as it is used: append with bounds, select, attention over the choice."""
import pytest
import torch

import paged_plain as pp
from helpers import TOL, assert_close_vectors
from paper_2603_14303_b200 import binding

pytestmark = pytest.mark.gpu
DEV = pp.DEV
BF, F32 = torch.bfloat16, torch.float32


def _pages(dtype, B, Hkv, d, ps, lens, own_pages=False, seed=0, spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    flat = [n for row in lens for n in row]
    W = max([-(-n // ps) for n in flat] + [0]) + 2
    P = sum(-(-n // ps) for n in flat) + 3
    heads = 1 if own_pages else Hkv
    table = pp.tables(flat, ps, P, W, gen).view(B, -1, W)
    mid = torch.randn((P, heads, d), generator=gen) * spread
    half = torch.rand((P, heads, d), generator=gen) * 2
    return table, (mid - half).to(dtype), (mid + half).to(dtype)


def _cache(dtype, table, mn, mx, ps):
    k = torch.zeros((mn.shape[0], mn.shape[1], ps, mn.shape[2]), dtype=dtype, device=DEV)   # (not read)
    return binding.PagedCache(k, k, table.to(DEV), None, mn.to(DEV), mx.to(DEV))


def _check(dtype, q, table, mn, mx, lens, ps, keep, n_first, n_last):
    status = pp.status_word()
    got, ln = binding.paged_select(q.to(DEV), _cache(dtype, table, mn, mx, ps), lens.to(DEV), keep, n_first, n_last, status=status)
    pp.ok(status)
    want, wl = pp.select(q, mn, mx, table, lens, ps, keep, n_first, n_last)
    assert torch.equal(ln.cpu(), wl)
    assert torch.equal(got.cpu(), want)


def _random(dtype, B, Hkv, G, d, ps, lens, keep, n_first=0, n_last=1, own_pages=False, seed=0, spread=1.0):
    lens = [[n] if not isinstance(n, (list, tuple)) else list(n) for n in lens]
    table, mn, mx = _pages(dtype, B, Hkv, d, ps, lens, own_pages, seed, spread)
    q = torch.randn((B, Hkv * G, d), generator=torch.Generator().manual_seed(seed + 1)).to(dtype)
    _check(dtype, q, table, mn, mx, torch.tensor(lens, dtype=torch.int32), ps, keep, n_first, n_last)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("keep,n_first,n_last", [(1, 0, 1), (4, 1, 2), (7, 0, 7), (8, 8 - 1, 1), (16, 1, 1), (63, 2, 3)])
def test_ragged_batch(dtype, keep, n_first, n_last):
    _random(dtype, 8, 2, 4, 128, 16, [0, 1, 16 * keep, 16 * keep + 1, 1000, 16 * keep - 1, 1024, 777], keep, n_first, n_last)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [8, 40, 64, 96, 128, 256])
@pytest.mark.parametrize("G", [1, 4, 7, 16])
def test_heads(dtype, d, G):
    _random(dtype, 2, 3, G, d, 16, [2000, 900], 20)


@pytest.mark.parametrize("ps", [1, 5, 64])
def test_page_sizes(ps):
    _random(BF, 3, 2, 4, 128, ps, [ps * 300 - ps // 2, ps * 40, ps * 41 - ps + 1], 40)


@pytest.mark.parametrize("pages", [500, 513, 2000, 8192, 20000])
def test_many_pages(pages):
    _random(BF, 1, 2, 4, 64, 4, [pages * 4 - 1], 128, 1, 2)
    _random(F32, 2, 1, 2, 32, 4, [pages * 4, pages * 2], 17)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_widest_tables(dtype):
    """As many pages as a call takes, more of them kept than are ranked in shared memory; few of them in use under wide tables."""
    W = binding.SC_SELECT_MAX_PAGES
    for n, keep in ((W * 2 - 1, 3000), (40000, 17), (300, 100)):
        table, mn, mx = _pages(dtype, 1, 1, 16, 2, [[n]])
        table = torch.cat([table, torch.full((1, 1, W - table.shape[2]), -1, dtype=torch.int32)], 2) if table.shape[2] < W else table[:, :, :W].contiguous()
        q = torch.randn((1, 2, 16), generator=torch.Generator().manual_seed(1)).to(dtype)
        _check(dtype, q, table, mn, mx, torch.tensor([[n]], dtype=torch.int32), 2, keep, 1, 2)


def test_tables_per_head():
    _random(BF, 2, 3, 4, 128, 16, [(50, 700, 0), (1000, 333, 16)], 9, own_pages=True)
    _random(F32, 2, 3, 4, 128, 16, [(50, 700, 0), (1000, 333, 16)], 9)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_equal_bounds_go_to_the_earlier_page(dtype):
    """All pages alike, all but some alike, and groups of equal ones: the tie is at the border."""
    n, keep = 300, 40
    table, mn, mx = _pages(dtype, 1, 2, 64, 16, [[n * 16]])
    q = torch.randn((1, 8, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    lens = torch.tensor([[n * 16]], dtype=torch.int32)
    flat_mn, flat_mx = torch.full_like(mn, -1.0), torch.full_like(mx, 1.0)
    _check(dtype, q, table, flat_mn, flat_mx, lens, 16, keep, 0, 1)
    _check(dtype, q, table, torch.zeros_like(mn), torch.zeros_like(mx), lens, 16, keep, 1, 1)
    some = flat_mx.clone()
    some[table[0, 0, 100:120].long()] = 2.0
    _check(dtype, q, table, flat_mn, some, lens, 16, keep, 0, 1)
    few = torch.randint(0, 6, (n,), generator=torch.Generator().manual_seed(2)).float()
    steps = flat_mx.clone()
    steps[table[0, 0, :n].long()] = (1 + few / 8)[:, None, None].to(dtype).expand(-1, 2, 64)
    _check(dtype, q, table, flat_mn, steps, lens, 16, keep, 0, 1)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_bounds_closer_than_32_bits_tell(dtype):
    """Bounds that differ in the tenth digit: one large term common to all pages, small ones that order them."""
    n, keep, d = 400, 64, 64
    table, mn, mx = _pages(dtype, 1, 1, d, 16, [[n * 16]])
    q = torch.ones((1, 2, d)).to(dtype)
    q[:, :, 0] = 2.0 ** 20
    q[:, :, 1] = 2.0 ** -14
    mn, mx = torch.zeros_like(mn), torch.zeros_like(mx)
    mx[:, :, 0] = 1.5
    mx[:, :, 1] = torch.randint(0, 256, (mx.shape[0], 1), generator=torch.Generator().manual_seed(3)).float().to(dtype)
    lens = torch.tensor([[n * 16]], dtype=torch.int32)
    _check(dtype, q, table, mn, mx, lens, 16, keep, 0, 1)
    # large terms that cancel
    mn[:, :, 2] = mx[:, :, 2] = -1.5
    q[:, :, 2] = 2.0 ** 20
    _check(dtype, q, table, mn, mx, lens, 16, keep, 0, 1)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_bounds_that_are_not_finite(dtype):
    n, keep, d = 300, 20, 64
    table, mn, mx = _pages(dtype, 1, 1, d, 16, [[n * 16]])
    q = torch.randn((1, 4, d), generator=torch.Generator().manual_seed(1)).to(dtype)
    q = torch.where(q == 0, torch.ones_like(q), q)
    lens = torch.tensor([[n * 16]], dtype=torch.int32)
    ids = table[0, 0].long()
    mx[ids[10], 0, 3], mn[ids[200], 0, 5], mx[ids[77]], mn[ids[78]] = float("nan"), float("nan"), float("inf"), -float("inf")
    _check(dtype, q, table, mn, mx, lens, 16, keep, 0, 1)
    _check(dtype, q, table, mn, mx, lens, 16, 2, 0, 1)
    big = 3.0e38
    _check(dtype, (q * 0 + big).to(dtype), table, mn.nan_to_num(0, 1, -1), mx.nan_to_num(0, 1, -1) * 1.0, lens, 16, keep, 0, 1)


def test_a_page_that_does_not_exist():
    """Its bound ranks below all others; where all pages are kept it is handed on."""
    table, mn, mx = _pages(BF, 1, 1, 64, 16, [[1600]])
    q = torch.randn((1, 4, 64), generator=torch.Generator().manual_seed(1)).to(BF)
    lens = torch.tensor([[1600]], dtype=torch.int32)
    broken = table.clone()
    broken[0, 0, 3], broken[0, 0, 50] = -1, 2 ** 31 - 1
    status = pp.status_word()
    got, _ = binding.paged_select(q.to(DEV), _cache(BF, broken, mn, mx, 16), lens.to(DEV), 98, status=status)
    assert int(status) == binding.SC_ERR_INVALID_ARG
    want = torch.cat([table[0, 0, :3], table[0, 0, 4:50], table[0, 0, 51:100]])
    assert got[0, 0].tolist() == want.tolist()
    got, _ = binding.paged_select(q.to(DEV), _cache(BF, broken, mn, mx, 16), lens.to(DEV), 100)
    assert got[0, 0].tolist() == broken[0, 0, :100].tolist()


def test_deterministic_and_captured():
    table, mn, mx = _pages(BF, 4, 2, 128, 16, [[9000], [5000], [100], [3000]])
    cache = _cache(BF, table, mn, mx, 16)
    q = torch.randn((4, 8, 128), generator=torch.Generator().manual_seed(1)).to(BF).to(DEV)
    lens = torch.tensor([9000, 5000, 100, 3000], dtype=torch.int32, device=DEV)
    want = binding.paged_select(q, cache, lens, 32)
    out, ln = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.sc_paged_select(q, cache, lens, 32, 0, 1, out, ln)
    for _ in range(3):
        out.zero_(), ln.zero_()
        g.replay()
        assert torch.equal(out, want[0]) and torch.equal(ln, want[1])


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_sparse_attention_from_append_to_output(dtype, layout):
    """A prompt and some tokens are appended with bounds, then each step's query attends to the pages picked for it: what attention over
    those pages says; and with all pages kept, what attention over the whole cache says."""
    gen = torch.Generator().manual_seed(7)
    B, H, G, d, ps, W, keep = 2, 2, 4, 128, 16, 40, 6
    P = B * W
    k = pp.on_device(torch.zeros((P, H, ps, d), dtype=dtype), layout)
    v = pp.on_device(torch.zeros((P, H, ps, d), dtype=dtype), layout)
    mn, mx = torch.zeros((P, H, d), dtype=dtype, device=DEV), torch.zeros((P, H, d), dtype=dtype, device=DEV)
    table = torch.randperm(P, generator=gen).to(torch.int32).view(B, W)
    cache = binding.PagedCache(k, v, table.to(DEV), None, mn, mx)
    inv = (10000.0 ** (-torch.arange(0, d, 2).float() / d)).to(DEV)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    status = pp.status_word()
    for news in ([300, 41], [1, 1], [1, 1], [0, 200], [16, 1], [1, 1]):
        T = sum(news)
        off = torch.tensor([0, news[0], T], dtype=torch.int32, device=DEV)
        kn, vn = (torch.randn((T, H, d), generator=gen).to(dtype).to(DEV) for _ in range(2))
        lens, _ = binding.paged_append(cache, kn, vn, off, lens, inv_freq=inv, status=status)
        q = torch.randn((B, H * G, d), generator=gen).to(dtype)
        sel, ln = binding.paged_select(q.to(DEV), cache, lens, keep, 1, 1, status=status)
        want_sel, want_ln = pp.select(q, mn.cpu(), mx.cpu(), table.view(B, 1, W), lens.cpu().view(B, 1), ps, keep, 1, 1)
        assert torch.equal(sel.cpu(), want_sel) and torch.equal(ln.cpu(), want_ln)
        got = binding.paged_decode_attn(q.to(DEV), cache.over(sel), ln, status=status)
        want = pp.attention(q, k.cpu(), v.cpu(), want_sel, want_ln)
        assert_close_vectors(got.double().cpu().numpy(), want.numpy(), TOL[dtype], "sparse")
        sel, ln = binding.paged_select(q.to(DEV), cache, lens, W, status=status)
        whole = binding.paged_decode_attn(q.to(DEV), cache.over(sel), ln, status=status)
        want = pp.attention(q, k.cpu(), v.cpu(), table.view(B, 1, W), lens.cpu().view(B, 1))
        assert_close_vectors(whole.double().cpu().numpy(), want.numpy(), TOL[dtype], "all pages")
    pp.ok(status)
    # the bounds bound: every key of a page lies between its page's
    for b in range(B):
        for j in range(int(lens[b]) // ps):
            p = int(table[b, j])
            assert bool((k[p] >= mn[p].unsqueeze(1)).all()) and bool((k[p] <= mx[p].unsqueeze(1)).all())
