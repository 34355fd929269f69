"""sc_paged_append against its formulas in 64 bits: what is written, what is left alone, the pages' bounds, the rotation at far
positions, ragged batches, and the calls that it answers through the status word."""
import pytest
import torch

import paged_plain as pp
from paper_2603_14303_b200 import binding

pytestmark = pytest.mark.gpu
DEV = pp.DEV
BF, F32 = torch.bfloat16, torch.float32


def _run(dtype, Hkv, Hq, d, ps, lens, news, layout="hnd", rot=None, pairs=False, bounds=False, count=False, pad=0, gap=0, fused=False,
         positions=None, with_q=True, seed=0):
    """Appends news[b] rows behind lens[b], and compares everything that the call may or may not touch."""
    gen = torch.Generator().manual_seed(seed)
    B, rot = len(lens), d if rot is None else rot
    W = max(-(-(a + m) // ps) for a, m in zip(lens, news)) + 1
    P = sum(-(-(a + m) // ps) for a, m in zip(lens, news)) + 2
    table = pp.tables([a + m for a, m in zip(lens, news)], ps, P, W, gen)
    k, v = (pp.pool(P, Hkv, ps, d, dtype, layout, gen) for _ in range(2))
    off, slots = [0], []
    for m in news:
        slots.append(m)
        off.append(off[-1] + m + gap)     # gap: tokens of no sequence, behind each
    T = off[-1] + pad
    seq_len = torch.tensor(slots, dtype=torch.int32) if gap else None
    kn, vn, q = (torch.randn((T, h, d), generator=gen).to(dtype) for h in (Hkv, Hkv, Hq))
    inv = (10000.0 ** (-torch.arange(0, rot, 2).float() / max(rot, 1))) if rot else None
    pos = None if positions is None else torch.randint(0, positions, (T,), generator=gen, dtype=torch.int32)
    cnt = torch.randint(1, 9, (P, Hkv, ps), generator=gen, dtype=torch.int32) if count else None
    cnt_new = torch.randint(1, 9, (T, Hkv), generator=gen, dtype=torch.int32) if count == "given" else None
    mn, mx = k.amin(2), k.amax(2)
    # on the device
    dk, dv = pp.on_device(k, layout), pp.on_device(v, layout)
    dev = lambda t: None if t is None else t.to(DEV)
    dmn, dmx = (dev(mn), dev(mx)) if bounds else (None, None)
    cache = binding.PagedCache(dk, dv, dev(table), dev(cnt), dmn, dmx)
    if fused:   # one projection's output: queries, keys, values side by side; queries rotated in place
        x = torch.cat([q, kn, vn], 1).to(DEV)
        dq, dkn, dvn = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        q_out = dq
    else:
        dq, dkn, dvn = dev(q), dev(kn), dev(vn)
        q_out = torch.full_like(dq, 3.0)
    status = pp.status_word()
    len_out = torch.full((B,), -1, dtype=torch.int32, device=DEV)
    binding.sc_paged_append(cache, dkn, dvn, dev(torch.tensor(off, dtype=torch.int32)), dev(torch.tensor(lens, dtype=torch.int32)),
                            dev(seq_len), dev(cnt_new), len_out, dq if with_q else None, q_out if with_q else None, dev(inv), dev(pos), status,
                            binding.SC_FLAG_ROPE_PAIRS if pairs else 0)
    pp.ok(status)
    assert len_out.tolist() == [a + m for a, m in zip(lens, news)]
    # what should be there
    got_k, got_v, got_q = dk.cpu(), dv.cpu(), q_out.cpu()
    wk, wv, wcnt = k.clone(), v.clone(), cnt.clone() if count else None
    live = torch.zeros(T, dtype=torch.bool)
    for b in range(B):
        for i in range(news[b]):
            t, row = off[b] + i, lens[b] + i
            page, r = int(table[b, row // ps]), row % ps
            live[t] = True
            at = torch.tensor([row if pos is None else int(pos[t])])
            want, mass = pp.rotate(kn[t:t + 1], at, inv, pairs) if rot else (kn[t:t + 1].double(), torch.zeros(1, Hkv, d))
            pp.assert_rotated(got_k[page, :, r], want[0], mass[0], f"k of token {t}")
            if with_q:
                want, mass = pp.rotate(q[t:t + 1], at, inv, pairs) if rot else (q[t:t + 1].double(), torch.zeros(1, Hq, d))
                pp.assert_rotated(got_q[t], want[0], mass[0], f"q of token {t}")
            if r == 0:
                mn[page], mx[page] = got_k[page, :, 0], got_k[page, :, 0]
            mn[page], mx[page] = torch.minimum(mn[page], got_k[page, :, r]), torch.maximum(mx[page], got_k[page, :, r])
            wk[page, :, r], wv[page, :, r] = got_k[page, :, r], vn[t]
            if count:
                wcnt[page, :, r] = cnt_new[t] if cnt_new is not None else 1
    assert pp.same_bits(got_k, wk) and pp.same_bits(got_v, wv)      # values copied, every other row as it was
    if with_q:
        rest = q[~live] if fused else torch.full_like(q[~live], 3.0)
        assert pp.same_bits(got_q[~live], rest)
    if layout == "gaps":
        whole = dk.as_strided((P, Hkv + 1, ps + 1, d + 16), ((Hkv + 1) * (ps + 1) * (d + 16), (ps + 1) * (d + 16), d + 16, 1))
        assert bool((whole[:, Hkv] == 7).all()) and bool((whole[:, :, ps] == 7).all()) and bool((whole[..., d:] == 7).all())
    if bounds:
        assert torch.equal(dmn.cpu(), mn) and torch.equal(dmx.cpu(), mx)
    if count:
        assert torch.equal(cache.count.cpu(), wcnt)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", ["hnd", "nhd", "gaps"])
def test_ragged_batch(dtype, layout):
    _run(dtype, 4, 12, 128, 16, [0, 5, 16, 31, 100, 7], [3, 1, 40, 2, 0, 17], layout, bounds=True)


@pytest.mark.parametrize("d,rot,pairs", [(128, 64, False), (128, 64, True), (64, 0, False), (96, 96, False), (96, 20, False), (256, 256, True),
                                         (8, 8, False), (8, 2, True), (24, 24, False), (256, 250, False), (40, 6, True), (32, 16, False)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_head_sizes_and_rotated_parts(dtype, d, rot, pairs):
    _run(dtype, 2, 6, d, 8, [3, 0, 9], [11, 1, 20], rot=rot, pairs=pairs, bounds=True)


@pytest.mark.parametrize("ps", [1, 2, 5, 16, 17, 48, 256])
@pytest.mark.parametrize("bounds", [False, True])
def test_page_sizes(ps, bounds):
    _run(BF, 2, 2, 64, ps, [0, 1, 15, 16, 300], [33, 1, 2, 16, 270], "nhd", bounds=bounds)


@pytest.mark.parametrize("ps", [63, 64, 65, 100, 128, 1000, 100000])
def test_long_pages_are_shared_out(ps):
    """Without bounds a page's rows may be several blocks' work."""
    _run(BF, 2, 4, 64, ps, [0, 1, 64, 150, 63], [300, 65, 128, 1, 2], "nhd", gap=3)


@pytest.mark.parametrize("Hkv,Hq", [(1, 1), (1, 32), (8, 8), (3, 21), (32, 64), (70, 70)])
def test_heads(Hkv, Hq):
    _run(BF, Hkv, Hq, 32, 16, [2, 30], [1, 20], bounds=True)


@pytest.mark.parametrize("B", [1, 2, 255, 256, 257, 700])
def test_single_tokens(B):
    _run(BF, 2, 4, 128, 16, [(7 * b) % 50 for b in range(B)], [1] * B, "nhd", bounds=True)


def test_tokens_of_no_sequence_are_left_alone():
    _run(BF, 2, 4, 64, 16, [0, 3, 20], [4, 0, 30], pad=5, gap=3)
    _run(F32, 2, 4, 64, 16, [0, 3, 20], [4, 0, 30], pad=5, gap=0)


@pytest.mark.parametrize("count", [True, "given"])
def test_counts(count):
    _run(BF, 4, 4, 64, 16, [0, 3, 20], [4, 1, 30], count=count, gap=2, with_q=False, rot=0)


def test_one_projection_output_rotated_in_place():
    _run(BF, 4, 16, 128, 16, [0, 13], [40, 1], fused=True)
    _run(F32, 4, 16, 128, 16, [0, 13], [40, 1], fused=True, pairs=True)


def test_positions_of_their_own():
    _run(BF, 2, 4, 128, 16, [4, 0], [9, 30], positions=2 ** 31 - 1)
    _run(F32, 2, 4, 128, 16, [4, 0], [9, 30], positions=131072)


def test_far_rows():
    """Rows far behind in a cache: positions past 2^17, and a pool whose offsets pass 2^32 bytes."""
    d, ps, Hkv, n = 128, 16, 8, 200000
    P = 140000                                             # 140000 pages x 32 KB: 4.6 GB
    k = torch.zeros((P, Hkv, ps, d), dtype=BF, device=DEV)
    v = torch.zeros((P, Hkv, ps, d), dtype=BF, device=DEV)
    table = torch.full((1, 15000), -1, dtype=torch.int32, device=DEV)
    first = n // ps
    table[0, first] = P - 1
    gen = torch.Generator().manual_seed(3)
    kn, vn = (torch.randn((5, Hkv, d), generator=gen).to(BF) for _ in range(2))
    inv = 500000.0 ** (-torch.arange(0, d, 2).float() / d)
    status = pp.status_word()
    cache = binding.PagedCache(k, v, table)
    lens, _ = binding.paged_append(cache, kn.to(DEV), vn.to(DEV), torch.tensor([0, 5], dtype=torch.int32, device=DEV),
                                   torch.tensor([n], dtype=torch.int32, device=DEV), inv_freq=inv.to(DEV), status=status)
    pp.ok(status)
    want, mass = pp.rotate(kn, torch.arange(n, n + 5), inv, False)
    pp.assert_rotated(k[P - 1, :, :5].transpose(0, 1).cpu(), want, mass, "k")
    assert pp.same_bits(v[P - 1, :, :5].transpose(0, 1), vn)
    assert int(k[:P - 1].count_nonzero()) == 0 and int(k[P - 1, :, 5:].count_nonzero()) == 0


def test_bounds_with_keys_that_are_not_numbers():
    k = torch.zeros((2, 1, 4, 8), dtype=F32, device=DEV)
    mn, mx = torch.full((2, 1, 8), 9.0, device=DEV), torch.full((2, 1, 8), 9.0, device=DEV)
    cache = binding.PagedCache(k, k.clone(), torch.tensor([[1, 0]], dtype=torch.int32, device=DEV), None, mn, mx)
    new = torch.arange(24, dtype=F32, device=DEV).view(3, 1, 8) - 10
    new[1, 0, 2], new[0, 0, 3], new[2, 0, 4] = float("nan"), float("inf"), -float("inf")
    binding.paged_append(cache, new, new, torch.tensor([0, 3], dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV))
    assert torch.equal(mn[1].isnan(), new.isnan().any(0)) and torch.equal(mx[1].isnan(), new.isnan().any(0))
    good = ~new.isnan().any(0)
    assert torch.equal(mn[1][good], new.amin(0)[good]) and torch.equal(mx[1][good], new.amax(0)[good])
    assert bool((mn[0] == 9).all())


def _small(B=2, W=2, ps=4):
    k = torch.zeros((8, 1, ps, 8), dtype=F32, device=DEV)
    table = torch.arange(B * W, dtype=torch.int32, device=DEV).view(B, W)
    return binding.PagedCache(k, k.clone(), table)


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def test_a_sequence_without_room_is_left_as_it_is():
    c, status = _small(), pp.status_word()
    new = torch.ones((6, 1, 8), device=DEV)
    q_out = torch.zeros_like(new)
    lens, _ = binding.paged_append(c, new, new, _i32(0, 3, 6), _i32(6, 5), q=new, q_out=q_out, status=status)
    assert int(status) == binding.SC_ERR_CAPACITY
    assert lens.tolist() == [6, 8]
    assert int(c.k[:2].count_nonzero()) == 0 and int(c.k[2].count_nonzero()) == 0 and bool((c.k[3, 0, 1:] == 1).all())
    assert bool((q_out == 1).all())


def test_lengths_near_the_largest_integer():
    c, status = _small(), pp.status_word()
    new = torch.ones((2, 1, 8), device=DEV)
    lens, _ = binding.paged_append(c, new, new, _i32(0, 1, 2), _i32(2 ** 31 - 1, 0), status=status)
    assert int(status) == binding.SC_ERR_CAPACITY and lens.tolist() == [2 ** 31 - 1, 1]
    assert int(c.k.count_nonzero()) == 8


@pytest.mark.parametrize("bad", [-1, 8, 2 ** 31 - 1, -2 ** 31])
def test_a_page_that_does_not_exist(bad):
    c, status = _small(), pp.status_word()
    c.table[0, 1] = bad
    new = torch.ones((6, 1, 8), device=DEV)
    binding.paged_append(c, new, new, _i32(0, 6, 6), _i32(0, 0), status=status)
    assert int(status) == binding.SC_ERR_INVALID_ARG
    assert bool((c.k[0] == 1).all()) and int(c.k[1:].count_nonzero()) == 0


@pytest.mark.parametrize("off,length,have", [((0, 7, 7), None, (0, 0)), ((3, 1, 2), None, (0, 0)), ((-1, 1, 2), None, (0, 0)),
                                             ((0, 2, 4), (3, 1), (0, 0)), ((0, 2, 4), (-1, 1), (0, 0)), ((0, 2, 4), None, (-1, 0))])
def test_offsets_and_lengths_that_break_the_rules(off, length, have):
    c, status = _small(), pp.status_word()
    new = torch.ones((6, 1, 8), device=DEV)
    binding.paged_append(c, new, new, _i32(*off), _i32(*have), seq_len=None if length is None else _i32(*length), status=status)
    assert int(status) == binding.SC_ERR_INVALID_ARG
    assert int(c.k[:2].count_nonzero()) == 0        # the sequence at fault


def test_no_tokens():
    c, status = _small(), pp.status_word()
    none = torch.zeros((0, 1, 8), device=DEV)
    lens, _ = binding.paged_append(c, none, none, _i32(0, 0, 0), _i32(3, 8), status=status)
    pp.ok(status)
    assert lens.tolist() == [3, 8] and int(c.k.count_nonzero()) == 0


def test_captured_and_replayed():
    """One capture serves a growing cache: lengths are read on the device."""
    gen = torch.Generator().manual_seed(5)
    B, H, d, ps = 3, 2, 64, 4
    k = torch.zeros((40, H, ps, d), dtype=BF, device=DEV)
    table = torch.randperm(36, generator=gen)[:36].to(torch.int32).view(3, 12).to(DEV)
    cache = binding.PagedCache(k, torch.zeros_like(k), table)
    new = torch.zeros((B, H, d), dtype=BF, device=DEV)
    off, lens, nxt = _i32(0, 1, 2, 3), torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    status = pp.status_word()

    def step():
        binding.paged_append(cache, new, new, off, lens, len_out=nxt, status=status)
        lens.copy_(nxt)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    lens.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    rows = torch.randn((20, B, H, d), generator=gen).to(BF).to(DEV)
    for r in rows:
        new.copy_(r)
        g.replay()
    pp.ok(status)
    assert lens.tolist() == [20] * B
    for b in range(B):
        got = k[table[b, :5].long()].transpose(1, 2).reshape(20, H, d)
        assert pp.same_bits(got, rows[:, b])
