"""The binding of the calls on a paged cache: what it refuses before anything is enqueued, what it allocates, and a whole step as a model makes it."""
import pytest
import torch

import paged_plain as pp
from helpers import TOL, assert_close_vectors
from paper_2603_14303_b200 import binding

pytestmark = pytest.mark.gpu
DEV = pp.DEV
BF, F32 = torch.bfloat16, torch.float32


def _cache(P=6, H=2, ps=4, d=16, B=2, W=3, dtype=BF, **kw):
    k = torch.zeros((P, H, ps, d), dtype=dtype, device=DEV)
    table = torch.arange(B * W, dtype=torch.int32, device=DEV).view(B, W)
    parts = dict(k=k, v=k.clone(), table=table)
    parts.update(kw)
    return binding.PagedCache(**parts)


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


K = torch.zeros((6, 2, 4, 16), dtype=BF)


@pytest.mark.parametrize("kw", [dict(v=torch.zeros((6, 2, 4, 8), dtype=BF, device="cpu")), dict(k=K), dict(v=K[:, :, ::2]),
                                dict(table=torch.zeros((2, 3), dtype=torch.int64)), dict(table=torch.zeros(3, dtype=torch.int32)),
                                dict(count=torch.zeros((6, 2, 4), dtype=torch.int64)), dict(count=torch.zeros((6, 4, 2), dtype=torch.int32)),
                                dict(k_min=torch.zeros((6, 2, 16), dtype=BF)), dict(k_min=torch.zeros((6, 2, 16)), k_max=torch.zeros((6, 2, 16))),
                                dict(k_min=torch.zeros((6, 16, 2), dtype=BF).transpose(1, 2), k_max=torch.zeros((6, 2, 16), dtype=BF))])
def test_caches_refused(kw):
    on_device = "v" in kw and kw["v"].shape[-1] == 8 or "k" in kw
    with pytest.raises((ValueError, TypeError)):
        _cache(**{n: t if on_device else t.to(DEV) for n, t in kw.items()})


def test_layouts_refused_and_taken():
    wide = torch.zeros((6, 2, 4, 32), dtype=BF, device=DEV)
    assert _cache(k=wide[..., :16], v=wide[..., 16:]).d == 16
    with pytest.raises(ValueError):
        _cache(k=wide[..., ::2], v=wide[..., ::2])                       # d not contiguous
    with pytest.raises(ValueError):
        _cache(k=wide[..., :16])                                          # v laid out in another way
    with pytest.raises(TypeError):
        _cache(k=wide[..., :16].half(), v=wide[..., :16].half())
    many = torch.zeros((4, 5, 9), dtype=torch.int32, device=DEV)
    assert _cache(table=many[:2, 0, :3]).table_heads == 1                 # rows far apart
    with pytest.raises(ValueError):
        _cache(table=many[:2, :2, :3])                                    # a sequence's tables are not evenly spaced
    with pytest.raises(ValueError):
        _cache(table=many[:2, :3, 0].t())                                 # entries apart


def _z(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype, device=DEV)


INT = dict(dtype=torch.int32)


@pytest.mark.parametrize("name,make", [("k_new", lambda: _z(3, 2, 8)), ("k_new", lambda: _z(3, 1, 16)), ("k_new", lambda: _z(3, 2, 16, dtype=F32)),
                                       ("k_new", lambda: _z(3, 16, 2).transpose(1, 2)), ("v_new", lambda: _z(4, 2, 16)),
                                       ("v_new", lambda: _z(3, 2, 32)[..., ::2]), ("v_new", lambda: _z(3, 2, 32)[..., :16]),
                                       ("seq_off", lambda: _z(3, dtype=torch.int64)), ("seq_off", lambda: _z(2, **INT)), ("cache_len", lambda: _z(3, **INT)),
                                       ("cache_len", lambda: _z(4, **INT)[::2]), ("seq_len", lambda: _z(1, **INT)), ("len_out", lambda: _z(2, dtype=F32)),
                                       ("positions", lambda: _z(2, **INT)), ("count_new", lambda: _z(3, **INT)), ("q", lambda: _z(3, 4, 16)),
                                       ("q_out", lambda: _z(3, 4, 16)), ("inv_freq", lambda: _z(8, dtype=torch.float64)), ("inv_freq", lambda: _z(16, dtype=F32)[::2])])
def test_appends_refused(name, make):
    args = dict(k_new=_z(3, 2, 16), v_new=_z(3, 2, 16), seq_off=_i32(0, 1, 3), cache_len=_i32(0, 0))
    args[name] = make()
    c, before = _cache(), binding.launch_counter()
    with pytest.raises((ValueError, TypeError)):
        binding.sc_paged_append(c, **args)
    assert binding.launch_counter() == before


def test_host_tensors_refused():
    c = _cache()
    new = torch.zeros((3, 2, 16), dtype=BF)
    with pytest.raises(ValueError):
        binding.paged_append(c, new, new, _i32(0, 1, 3), _i32(0, 0))
    with pytest.raises(ValueError):
        binding.paged_append(c, new.to(DEV), new.to(DEV), torch.tensor([0, 1, 3], dtype=torch.int32), _i32(0, 0))
    q = torch.zeros((2, 4, 16), dtype=BF)
    with pytest.raises(ValueError):
        binding.paged_decode_attn(q, c, _i32(1, 1))
    with pytest.raises(ValueError):
        binding.paged_decode_attn(q.to(DEV), c, torch.tensor([1, 1], dtype=torch.int32))


def test_attention_and_selection_refused():
    c = _cache()
    q = torch.zeros((2, 4, 16), dtype=BF, device=DEV)
    ws = binding.paged_decode_workspace(2, 4, 2, 16, DEV)
    before = binding.launch_counter()
    for bad in (q[:1], q.float(), torch.zeros((2, 4, 32), dtype=BF, device=DEV), torch.zeros((2, 16, 4), dtype=BF, device=DEV).transpose(1, 2)):
        with pytest.raises(ValueError):
            binding.paged_decode_attn(bad, c, _i32(1, 1), workspace=ws)
    for lens in (_i32(1), _i32(1, 1, 1, 1), torch.ones(2, device=DEV)):
        with pytest.raises(ValueError):
            binding.paged_decode_attn(q, c, lens, workspace=ws)
    with pytest.raises(ValueError):
        binding.paged_decode_attn(q, c, _i32(1, 1), out=torch.zeros((2, 2, 16), dtype=BF, device=DEV), workspace=ws)
    with pytest.raises(binding.ScError):
        binding.paged_decode_attn(q, c, _i32(1, 1), workspace=ws[:100])
    with pytest.raises(binding.ScError):
        binding.paged_decode_attn(q[:, :3].contiguous(), c, _i32(1, 1), workspace=ws)      # three query heads on two
    with pytest.raises(ValueError):
        binding.paged_select(q, c, _i32(1, 1), 2)                                          # no bounds
    bounds = torch.zeros((6, 2, 16), dtype=BF, device=DEV)
    full = _cache(k_min=bounds, k_max=bounds.clone())
    for keep, first, last in ((0, 0, 1), (2, 2, 1), (2, 0, 0), (2, -1, 1)):
        with pytest.raises((binding.ScError, RuntimeError)):
            binding.paged_select(q, full, _i32(1, 1), keep, first, last)
    with pytest.raises(ValueError):
        c.one_head_sequences()
    assert binding.launch_counter() == before


@pytest.mark.parametrize("status", [lambda: torch.zeros(1, dtype=torch.int32), lambda: _z(1, dtype=torch.int64), lambda: _z(0, **INT)],
                         ids=["host", "long", "empty"])
def test_status_words_refused(status):
    c, q, lens = _cache(k_min=_z(6, 2, 16), k_max=_z(6, 2, 16)), _z(2, 2, 16), _i32(0, 0)
    calls = [lambda s: binding.paged_append(c, _z(3, 2, 16), _z(3, 2, 16), _i32(0, 1, 3), _i32(0, 0), status=s),
             lambda s: binding.paged_decode_attn(q, c, lens, status=s), lambda s: binding.paged_select(q, c, lens, 2, status=s)]
    before = binding.launch_counter()
    for call in calls:
        with pytest.raises(ValueError, match="status"):
            call(status())
    assert binding.launch_counter() == before


def test_workspaces_refused():
    c, q, lens = _cache(), _z(2, 2, 16), _i32(0, 0)
    size = binding.paged_decode_workspace(2, 2, 2, 16, DEV).numel()
    before = binding.launch_counter()
    for ws in (_z(1, dtype=torch.uint8).expand(size), torch.zeros(size, dtype=torch.uint8)):   # one byte shown many times; on the host
        with pytest.raises(ValueError, match="workspace"):
            binding.paged_decode_attn(q, c, lens, workspace=ws)
    with pytest.raises(binding.ScError):
        binding.paged_decode_attn(q, c, lens, workspace=_z(size - 16, dtype=torch.uint8))
    assert binding.launch_counter() == before


def test_one_launch_per_call():
    bounds = torch.zeros((6, 2, 16), dtype=BF, device=DEV)
    c = _cache(k_min=bounds, k_max=bounds.clone())
    new = torch.ones((3, 2, 16), dtype=BF, device=DEV)
    before = binding.launch_counter()
    lens, _ = binding.paged_append(c, new, new, _i32(0, 1, 3), _i32(0, 0))
    sel, ln = binding.paged_select(torch.ones((2, 4, 16), dtype=BF, device=DEV), c, lens, 1)
    out = binding.paged_decode_attn(torch.ones((2, 4, 16), dtype=BF, device=DEV), c.over(sel), ln)
    assert binding.launch_counter() == before + 3
    assert bool((out == 1).all())


@pytest.mark.parametrize("name,H,Hq,d", [("gqa", 4, 16, 128), ("mqa", 1, 8, 64)])
def test_layers_of_a_model(name, H, Hq, d):
    """Three layers with a table of their own over one pool each, a ragged batch: a prompt chunk, then single tokens.  All layers append at the
    same lengths, which move on once per step; workspace and status word are shared."""
    gen = torch.Generator().manual_seed(3)
    B, L, ps, W = 3, 3, 16, 9
    table = torch.randperm(B * W, generator=gen).to(torch.int32).view(B, W).to(DEV)
    caches = [binding.PagedCache(*(torch.full((B * W, ps, H, d), float("nan"), dtype=BF, device=DEV).transpose(1, 2) for _ in range(2)), table) for _ in range(L)]
    inv = (10000.0 ** (-torch.arange(0, d, 2).float() / d)).to(DEV)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    ws, status = binding.paged_decode_workspace(B, Hq, H, d, DEV), pp.status_word()
    for news in ([70, 1, 33], [1, 1, 1], [1, 1, 1], [1, 16, 15]):
        off = torch.tensor([0, *torch.tensor(news).cumsum(0).tolist()], dtype=torch.int32, device=DEV)
        nxt = torch.empty_like(lens)
        for c in caches:
            x = torch.randn((sum(news), Hq + 2 * H, d), generator=gen).to(BF).to(DEV)
            _, q = binding.paged_append(c, x[:, Hq:Hq + H], x[:, Hq + H:], off, lens, inv_freq=inv, q=x[:, :Hq], len_out=nxt, status=status)
            last = q[(off[1:] - 1).long()]                              # the last token of each sequence attends to its whole cache
            got = binding.paged_decode_attn(last, c, nxt, workspace=ws, status=status)
            want = pp.attention(last.cpu(), c.k.cpu(), c.v.cpu(), table.cpu().view(B, 1, W), nxt.cpu().view(B, 1))
            assert_close_vectors(got.double().cpu().numpy(), want.numpy(), TOL[BF], "layer")
        lens = nxt
    pp.ok(status)
    assert lens.tolist() == [73, 19, 50]


def test_two_graphs_that_share_a_workspace_by_turns():
    """Replayed one after the other in one stream, over caches of different shapes."""
    gen = torch.Generator().manual_seed(8)
    ws = binding.paged_decode_workspace(1, 1, 1, 128, DEV)
    graphs = []
    for B, H, G, n in ((1, 4, 4, 9000), (6, 2, 4, 2500)):
        need = -(-n // 16)
        k, v = (torch.randn((B * need, H, 16, 128), generator=gen).to(BF).to(DEV) for _ in range(2))
        c = binding.PagedCache(k, v, torch.arange(B * need, dtype=torch.int32, device=DEV).view(B, need))
        q, lens = torch.randn((B, H * G, 128), generator=gen).to(BF).to(DEV), torch.full((B,), n, dtype=torch.int32, device=DEV)
        want, out = binding.paged_decode_attn(q, c, lens), torch.empty_like(q)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(3):
                binding.paged_decode_attn(q, c, lens, out=out, workspace=ws)
        graphs.append((g, out, want, c, q, lens))     # (a graph does not keep its inputs)
    for _ in range(5):
        for g, out, *_ in graphs:
            out.zero_()
            g.replay()
    torch.cuda.synchronize()
    for _, out, want, *_ in graphs:
        assert pp.same_bits(out, want)
    assert int(ws[:4096].count_nonzero()) == 0
