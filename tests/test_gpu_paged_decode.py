"""sc_paged_decode_attn against Eq. 4 in 64 bits: types, head layouts, lengths from none to long ones, page sizes and layouts, counts and
tables per head; what it leaves alone; and the calls that it answers through the status word."""
import numpy as np
import pytest
import torch

import paged_plain as pp
from helpers import TOL, assert_close_vectors
from paper_2603_14303_b200 import binding

pytestmark = pytest.mark.gpu
DEV = pp.DEV
BF, F32 = torch.bfloat16, torch.float32


def _cache(dtype, B, Hkv, d, ps, lens, layout="hnd", own_pages=False, count=False, seed=0, extra=2, dirty=True):
    """A cache on the CPU and on the device; rows behind a sequence's last are not numbers where `dirty`."""
    gen = torch.Generator().manual_seed(seed)
    flat = [n for row in lens for n in row]
    W = max([-(-n // ps) for n in flat] + [0]) + extra
    P = sum(-(-n // ps) for n in flat) + 3
    heads = 1 if own_pages else Hkv
    k, v = (pp.pool(P, heads, ps, d, dtype, layout, gen) for _ in range(2))
    table = pp.tables(flat, ps, P, W, gen).view(B, -1, W)
    cnt = torch.randint(1, 40, (P, heads, ps), generator=gen, dtype=torch.int32) if count else None
    if dirty:
        for n, t in zip(flat, table.view(len(flat), W)):
            if n % ps:
                for x in (k, v):
                    x[int(t[n // ps]), :, n % ps:] = float("nan")
                if count:
                    cnt[int(t[n // ps]), :, n % ps:] = -7
        used = torch.zeros(P, dtype=torch.bool)
        for n, t in zip(flat, table.view(len(flat), W)):
            used[t[:-(-n // ps)].long()] = True
        k[~used] = float("inf")
        v[~used] = float("nan")
    return k, v, table, cnt


def _device(k, v, table, cnt, layout):
    return binding.PagedCache(pp.on_device(k, layout), pp.on_device(v, layout), table.to(DEV), None if cnt is None else cnt.to(DEV))


def _check(dtype, B, Hkv, G, d, ps, lens, layout="hnd", own_pages=False, count=False, scale=0.0, flags=0, seed=0, q_scale=1.0):
    lens = [[n] if not isinstance(n, (list, tuple)) else list(n) for n in lens]
    k, v, table, cnt = _cache(dtype, B, Hkv, d, ps, lens, layout, own_pages, count, seed)
    gen = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn((B, Hkv * G, d), generator=gen) * q_scale).to(dtype)
    ln = torch.tensor(lens, dtype=torch.int32)
    # large scores: what fp32 sums of that size can be off by is allowed beside the usual tolerance (see pp.attention)
    want, bound = pp.attention(q, k, v, table, ln, scale, cnt, rounding=True) if q_scale != 1.0 else (pp.attention(q, k, v, table, ln, scale, cnt), 0.0)
    status = pp.status_word()
    ws = binding.paged_decode_workspace(B, Hkv * G, Hkv, d, DEV)
    cache = _device(k, v, table, cnt, layout)
    runs = [binding.paged_decode_attn(q.to(DEV), cache, ln.to(DEV), workspace=ws, scale=scale, status=status, flags=flags) for _ in range(2)]
    pp.ok(status)
    assert pp.same_bits(*runs)                                   # a fixed order
    assert int(ws[:4096].count_nonzero()) == 0                   # its counters are left as they were
    got = runs[0].double().cpu()
    got = want + torch.sign(got - want) * ((got - want).abs() - bound).clamp(min=0.0)
    assert_close_vectors(got.numpy(), want.numpy(), TOL[dtype], "attention")
    empty = [(b, h) for b in range(B) for h in range(Hkv) if lens[b][h if len(lens[b]) > 1 else 0] == 0]
    for b, h in empty:
        assert int(runs[0][b, h * G:(h + 1) * G].count_nonzero()) == 0


EDGES = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 129]


@pytest.mark.parametrize("flags", [0, binding.SC_FLAG_GENERIC])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", ["hnd", "nhd", "gaps"])
def test_lengths_at_the_edges_of_tiles(dtype, layout, flags):
    _check(dtype, len(EDGES), 2, 4, 128, 16, EDGES, layout, flags=flags)


@pytest.mark.parametrize("ps", [1, 3, 8, 16, 24, 32, 100, 128, 1000])
@pytest.mark.parametrize("flags", [0, binding.SC_FLAG_GENERIC])
def test_page_sizes(ps, flags):
    _check(BF, 3, 2, 4, 128, ps, [1000, 77, 130], "nhd", flags=flags, count=True)


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8, 9, 16, 20])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_query_groups(dtype, G):
    _check(dtype, 2, 3, G, 128, 16, [333, 40])


@pytest.mark.parametrize("d", [8, 40, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_head_sizes(dtype, d):
    _check(dtype, 3, 2, 3, d, 16, [200, 1, 90], count=True)


@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("G", [4, 8])
def test_generic_kernels_of_the_other_head_sizes(G, d):
    _check(BF, 3, 2, G, d, 16, [700, 15, 0], "nhd", flags=binding.SC_FLAG_GENERIC)
    _check(BF, 1, 2, G, d, 24, [5000], flags=binding.SC_FLAG_GENERIC)


@pytest.mark.parametrize("B,n", [(1500, 20), (2200, 3)])
def test_more_sequences_than_blocks(B, n):
    _check(BF, B, 1, 4, 64, 16, [(b * 7) % n for b in range(B)])


@pytest.mark.parametrize("G,d", [(4, 64), (8, 64), (16, 64), (4, 256), (8, 256), (5, 256)])
@pytest.mark.parametrize("ps", [16, 24])
def test_head_sizes_and_groups(G, d, ps):
    _check(BF, 3, 2, G, d, ps, [700, 15, 0], "nhd")


@pytest.mark.parametrize("flags", [0, binding.SC_FLAG_GENERIC])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_tables_and_lengths_per_head(dtype, flags):
    _check(dtype, 2, 3, 4, 128, 16, [(50, 700, 0), (1, 333, 16)], own_pages=True, count=True, flags=flags)


@pytest.mark.parametrize("flags", [0, binding.SC_FLAG_GENERIC])
def test_tables_per_head_of_shared_pages(flags):
    _check(BF, 2, 3, 4, 128, 16, [(50, 700, 0), (1, 333, 16)], count=True, flags=flags)


@pytest.mark.parametrize("B,n", [(1, 5000), (1, 40000), (2, 9001)])
@pytest.mark.parametrize("Hkv,G,d", [(8, 4, 128), (1, 8, 128), (1, 16, 64), (4, 7, 128)])
def test_long_sequences(B, n, Hkv, G, d):
    _check(BF, B, Hkv, G, d, 64, [n - 13 * b for b in range(B)])


def test_long_float32():
    _check(F32, 1, 2, 4, 128, 16, [9001])
    _check(F32, 2, 2, 4, 64, 24, [9001, 3])


@pytest.mark.parametrize("lens", [[20000] + [5] * 15, [5] * 15 + [20000], [0] * 7 + [3000] + [0] * 8, [0] * 16, list(range(0, 1600, 100))])
@pytest.mark.parametrize("flags", [0, binding.SC_FLAG_GENERIC])
def test_uneven_batches(lens, flags):
    _check(BF, 16, 2, 4, 128, 32, lens, flags=flags)


@pytest.mark.parametrize("B", [33, 64, 257])
def test_many_sequences(B):
    _check(BF, B, 2, 4, 128, 16, [(37 * b) % 300 for b in range(B)], "nhd")
    _check(F32, B, 2, 2, 64, 16, [(37 * b) % 100 for b in range(B)])


def test_scale_and_large_scores():
    _check(BF, 2, 2, 4, 128, 16, [300, 41], scale=0.3)
    _check(BF, 2, 2, 4, 128, 16, [300, 41], q_scale=30.0, count=True)   # a softmax that one row rules
    _check(F32, 2, 2, 4, 64, 16, [300, 41], scale=1.0, q_scale=20.0)


def test_pages_that_sequences_share():
    """A common prefix: tables of several sequences that name the same pages."""
    k, v, table, _ = _cache(BF, 3, 2, 128, 16, [[320], [64], [64]])
    table[1, 0, :4], table[2, 0, :4] = table[0, 0, :4], table[0, 0, :4]
    q = torch.randn((3, 8, 128), generator=torch.Generator().manual_seed(1)).to(BF)
    ln = torch.tensor([[320], [64], [64]], dtype=torch.int32)
    got = binding.paged_decode_attn(q.to(DEV), _device(k, v, table, None, "hnd"), ln.to(DEV))
    assert_close_vectors(got.double().cpu().numpy(), pp.attention(q, k, v, table, ln).numpy(), TOL[BF], "attention")


def test_lengths_beyond_the_table_and_below_zero():
    k, v, table, _ = _cache(BF, 2, 2, 128, 16, [[64], [48]], extra=0)
    q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(1)).to(BF)
    cache = _device(k, v, table, None, "hnd")
    for lens in ([[2 ** 31 - 1], [-3]], [[65], [-2 ** 31]]):
        got = binding.paged_decode_attn(q.to(DEV), cache, torch.tensor(lens, dtype=torch.int32, device=DEV))
        want = pp.attention(q, k, v, table, torch.tensor([[64], [0]]))
        assert_close_vectors(got.double().cpu().numpy(), want.numpy(), TOL[BF], "attention")


@pytest.mark.parametrize("flags", [0, binding.SC_FLAG_GENERIC])
@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1, -2 ** 31])
def test_a_page_that_does_not_exist(bad, flags):
    """Its rows are left out of the sums, the others' result stands, the status word tells."""
    k, v, table, _ = _cache(BF, 2, 2, 128, 16, [[300], [16]])
    q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(1)).to(BF)
    broken = table.clone()
    broken[0, 0, 5] = bad
    broken[1, 0, 0] = k.shape[0]
    status = pp.status_word()
    got = binding.paged_decode_attn(q.to(DEV), _device(k, v, broken, None, "hnd"), torch.tensor([[300], [16]], dtype=torch.int32, device=DEV),
                                    status=status, flags=flags)
    assert int(status) == binding.SC_ERR_INVALID_ARG
    left = torch.cat([table[:, :, :5], table[:, :, 6:]], 2)
    want = pp.attention(q, k, v, left, torch.tensor([[284], [0]]))
    assert_close_vectors(got.double().cpu().numpy(), want.numpy(), TOL[BF], "attention")


@pytest.mark.parametrize("flags", [0, binding.SC_FLAG_GENERIC])
def test_values_that_are_not_finite_stay_in_their_head(flags):
    k, v, table, _ = _cache(BF, 2, 2, 128, 16, [[100], [100]])
    v[int(table[0, 0, 1]), 1, 3, 7] = float("inf")
    k[int(table[1, 0, 2]), 0, 5, 9] = float("nan")
    q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(1)).to(BF)
    ln = torch.tensor([[100], [100]], dtype=torch.int32)
    got = binding.paged_decode_attn(q.to(DEV), _device(k, v, table, None, "hnd"), ln.to(DEV), flags=flags).double().cpu()
    want = pp.attention(q, k, v, table, ln)
    assert not bool(got[0, 4:, 7].isfinite().any()) and bool(got[1, :4].isnan().all())
    fine = want.isfinite()
    assert torch.equal(got.isfinite(), fine)
    assert_close_vectors(torch.where(fine, got, 0.0).numpy(), torch.where(fine, want, 0.0).numpy(), TOL[BF], "attention")


@pytest.mark.parametrize("dtype,flags", [(BF, 0), (BF, binding.SC_FLAG_GENERIC), (torch.float32, 0)])
@pytest.mark.parametrize("lens", [(5, 100), (3000, 700), (40000, 9)])
def test_scores_none_of_which_is_a_number(dtype, flags, lens):
    """A query head of NaN, and keys of NaN in every row of a stretch: the outputs are not numbers, the other heads' are untouched."""
    k, v, table, _ = _cache(dtype, 2, 2, 128, 16, [[n] for n in lens])
    for page in table[1, 0, : -(-lens[1] // 16)].tolist():
        k[page, 1, :, 3] = float("nan")
    q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(3)).to(dtype)
    q[0, 2, 17] = float("nan")
    ln = torch.tensor([[n] for n in lens], dtype=torch.int32)
    got = binding.paged_decode_attn(q.to(DEV), _device(k, v, table, None, "hnd"), ln.to(DEV), flags=flags).double().cpu()
    assert bool(got[0, 2].isnan().all()) and bool(got[1, 4:].isnan().all())
    want = pp.attention(q, k, v, table, ln)
    fine = want.isfinite()
    assert int(fine.sum()) == (7 + 4) * 128 and torch.equal(got.isfinite(), fine)
    assert_close_vectors(torch.where(fine, got, 0.0).numpy(), torch.where(fine, want, 0.0).numpy(), TOL[dtype], "attention")


@pytest.mark.parametrize("dtype,d,Hkv,G", [(BF, 128, 8, 4), (BF, 64, 4, 8), (F32, 64, 8, 2), (BF, 96, 8, 1)])
@pytest.mark.parametrize("B", [40, 170])
def test_many_short_sequences(dtype, d, Hkv, G, B):
    """More heads than blocks, of no row, one, a round of a block's warps and one more."""
    gen = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 150, (B,), generator=gen).tolist()
    lens[:6] = [64, 65, 0, 1, 16, 63]
    lens[-2:] = [129, 0]
    _check(dtype, B, Hkv, G, d, 16, lens)


def test_a_pool_past_32_bits():
    """Pages whose offsets pass 2^32 bytes and 2^31 elements."""
    P, ps, H, d = 140000, 16, 8, 128
    k = torch.zeros((P, H, ps, d), dtype=BF, device=DEV)
    v = torch.zeros((P, H, ps, d), dtype=BF, device=DEV)
    gen = torch.Generator().manual_seed(2)
    ids = torch.tensor([[P - 1, 3, P - 2, 139000]], dtype=torch.int32)
    for i in ids[0].tolist():
        k[i] = torch.randn((H, ps, d), generator=gen).to(BF).to(DEV)
        v[i] = torch.randn((H, ps, d), generator=gen).to(BF).to(DEV)
    q = torch.randn((1, 32, d), generator=gen).to(BF)
    n = 61
    small = torch.arange(4, dtype=torch.int32).view(1, 1, 4)
    kk, vv = k[ids[0].long().to(DEV)].cpu(), v[ids[0].long().to(DEV)].cpu()
    want = pp.attention(q, kk, vv, small, torch.tensor([[n]]))
    for flags in (0, binding.SC_FLAG_GENERIC):
        got = binding.paged_decode_attn(q.to(DEV), binding.PagedCache(k, v, ids.to(DEV)), torch.tensor([n], dtype=torch.int32, device=DEV),
                                        flags=flags)
        assert_close_vectors(got.double().cpu().numpy(), want.numpy(), TOL[BF], "attention")


def test_one_workspace_for_calls_of_all_shapes():
    """Sized for any of them, used by turns by batches, head sizes and types that leave partial sums in different places."""
    calls = []
    for i, (dtype, B, Hkv, G, d, lens) in enumerate([(BF, 16, 4, 4, 128, [[3000 - 100 * b] for b in range(16)]), (F32, 1, 2, 8, 256, [[4000]]),
                                                     (BF, 1, 8, 4, 128, [[20000]]), (BF, 2, 2, 16, 64, [[900], [5000]]), (F32, 9, 2, 2, 64, [[700]] * 9)]):
        k, v, table, _ = _cache(dtype, B, Hkv, d, 16, lens, seed=i, dirty=False)
        q = torch.randn((B, Hkv * G, d), generator=torch.Generator().manual_seed(i)).to(dtype).to(DEV)
        calls.append((q, _device(k, v, table, None, "hnd"), torch.tensor(lens, dtype=torch.int32, device=DEV)))
    ws = binding.paged_decode_workspace(1, 1, 1, 256, DEV)
    alone = [binding.paged_decode_attn(*c) for c in calls]
    for turn in range(3):
        for order in (calls, calls[::-1]):
            for c in order:
                i = next(j for j, o in enumerate(calls) if o is c)
                assert pp.same_bits(binding.paged_decode_attn(*c, workspace=ws, flags=0), alone[i])
            binding.paged_decode_attn(*calls[0], workspace=ws, flags=binding.SC_FLAG_GENERIC)


def test_captured_and_replayed_while_the_cache_grows():
    """Append and attention of a step in one graph: lengths and tables are read on the device."""
    gen = torch.Generator().manual_seed(4)
    B, H, G, d, ps, W = 3, 2, 4, 128, 16, 12
    P = B * W
    k, v = (torch.full((P, H, ps, d), float("nan"), dtype=BF, device=DEV) for _ in range(2))
    table = torch.randperm(P, generator=gen).to(torch.int32).view(B, 1, W)
    cache = binding.PagedCache(k, v, table.to(DEV))
    x = torch.zeros((B, H * (G + 2), d), dtype=BF, device=DEV)
    off = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    lens, nxt = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(2))
    inv = (10000.0 ** (-torch.arange(0, d, 2).float() / d)).to(DEV)
    q_out, out = torch.zeros((B, H * G, d), dtype=BF, device=DEV), torch.zeros((B, H * G, d), dtype=BF, device=DEV)
    ws, status = binding.paged_decode_workspace(B, H * G, H, d, DEV), pp.status_word()

    def step():
        binding.paged_append(cache, x[:, H * G:H * G + H], x[:, H * G + H:], off, lens, inv_freq=inv, q=x[:, :H * G], q_out=q_out, len_out=nxt,
                             status=status)
        lens.copy_(nxt)
        binding.paged_decode_attn(q_out, cache, lens, out=out, workspace=ws, status=status)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    lens.copy_(torch.tensor([0, 5, 100], dtype=torch.int32))
    first = torch.randn((P, H, ps, d), generator=gen).to(BF)
    k.copy_(first), v.copy_(first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(40):
        x.copy_(torch.randn(x.shape, generator=gen).to(BF))
        g.replay()
        if i % 13 == 0 or i == 39:
            want = pp.attention(q_out.cpu(), k.cpu(), v.cpu(), table, lens.cpu().view(B, 1))
            assert_close_vectors(out.double().cpu().numpy(), want.numpy(), TOL[BF], f"step {i}")
    pp.ok(status)
    assert lens.tolist() == [40, 45, 140]


def test_on_another_stream():
    k, v, table, _ = _cache(BF, 2, 2, 128, 16, [[900], [100]])
    q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(1)).to(BF).to(DEV)
    cache, ln = _device(k, v, table, None, "hnd"), torch.tensor([[900], [100]], dtype=torch.int32, device=DEV)
    want = binding.paged_decode_attn(q, cache, ln)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = binding.paged_decode_attn(q, cache, ln)
    torch.cuda.current_stream().wait_stream(s)
    assert pp.same_bits(got, want)


def test_compressed_cache_in_pages():
    """The cores of sc_compress, put into pages with their counts, give what sc_decode_attn gives over the contiguous cores; tokens that
    follow are appended to the pages."""
    from paper_2603_14303_b200 import synth
    w = synth.Workload("paged", B=2, n=1500, L=1, Hkv=4, Hq=16, d=128, gap=("poisson", 20.0), centroids=("uniform", 4), seed=11)
    ids, run_id, run_lens = synth.token_ids(w)
    K, V = (t.to(DEV) for t in synth.layer_kv(w, 0, run_id, run_lens))
    layer = binding.compress(K, V, binding.chunk(ids.to(DEV), w.delims), w.tau)
    ps = 16
    need = (layer.core_len.cpu() + 40 + ps - 1) // ps
    W, P = int(need.max()), int(need.sum())
    gen = torch.Generator().manual_seed(0)
    table = pp.tables([int(x) * ps for x in need.view(-1)], ps, P, W, gen).view(2, 4, W).to(DEV)
    pages = torch.full((P, 1, ps, 128), float("nan"), dtype=BF, device=DEV)
    cache = binding.PagedCache(pages, pages.clone(), table, torch.zeros((P, 1, ps), dtype=torch.int32, device=DEV))
    status = pp.status_word()
    lens = binding.paged_store(layer, cache, status=status)
    assert torch.equal(lens, layer.core_len)
    q = synth.queries(w, 0, 0).to(DEV)
    want = binding.decode_attn(q, layer).double().cpu().numpy()
    assert_close_vectors(binding.paged_decode_attn(q, cache, lens, status=status).double().cpu().numpy(), want, TOL[BF], "cores")
    # 40 generated tokens behind them, one step at a time, every head a sequence of its own
    new = torch.randn((40, 2, 2, 4, 128), generator=gen).to(BF).to(DEV)   # [step, K or V, B, Hkv, d]
    off = torch.arange(9, dtype=torch.int32, device=DEV)
    for x in new:
        lens, _ = binding.paged_append(cache.one_head_sequences(), x[0].reshape(8, 1, 128), x[1].reshape(8, 1, 128), off, lens.view(8), status=status)
    pp.ok(status)
    lens = lens.view(2, 4)
    assert torch.equal(lens, layer.core_len + 40)
    want = pp.attention(q.cpu(), cache.k.cpu(), cache.v.cpu(), table.cpu(), lens.cpu(), count=cache.count.cpu())
    assert_close_vectors(binding.paged_decode_attn(q, cache, lens).double().cpu().numpy(), want.numpy(), TOL[BF], "cores and tokens")
    assert bool((cache.count[cache.count > 0] >= 1).all()) and np.all(np.isfinite(want.numpy()))
