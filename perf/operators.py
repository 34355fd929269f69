"""What is timed of the paged cache: rows appended to pages with the position rotation on the way, attention of one new
token over the pages, and the choice of pages for sparse attention.

A case is one dict of plain values; its ``kind`` says which call one pass makes:

  append   new tokens' keys and values are rotated and join the cache, their queries are rotated beside them
  decode   one new token per sequence attends to its whole paged cache
  select   each (sequence, KV head) picks the pages that its queries bound highest
  sparse   select, then attention over the pages picked

``run`` computes them with elementary torch operations where ``own`` is false and calls the library where it is true.
Sizes are those of the repository's own workloads (``synth.config``) and tests, with odd ones beside them; ``draw`` covers
the ranges between.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

# the parameters that each kind reads, with what they are when a case does not say
_COMMON = dict(B=1, Hkv=8, G=4, d=128, dtype="bf16", ps=16, layout="hnd", spread=0.0)
_KINDS = {
    # n rows are in the cache, `new` tokens per sequence join it (ragged where spread > 0); rot columns are rotated;
    # bounds: the pages' smallest and largest keys are kept up to date
    "append": dict(_COMMON, n=2048, new=1, rot=128, interleaved=False, bounds=False),
    # own_pages: a table and pages per head, as for a compressed cache whose heads differ in length; count: rows are cores
    "decode": dict(_COMMON, n=2048, own_pages=False, count=False),
    "select": dict(_COMMON, n=32768, keep=128, first=1, last=2),
    "sparse": dict(_COMMON, n=32768, keep=128, first=1, last=2),
}
_MAX_BYTES = {"append": 8.6e8, "decode": 8.1e8, "select": 1.8e8, "sparse": 1.8e8}   # of a drawn case


def _case(kind, **kw):
    assert set(kw) <= set(_KINDS[kind]) | {"name"}, set(kw)
    return {"kind": kind, **_KINDS[kind], **kw}


def listed():
    return [
        # a decode step's append at batch 1, 32K context: pure latency
        _case("append", name="append_1", n=32767),
        # a decode step of 64 sequences, token-major pages, the pages' bounds kept for sparse attention
        _case("append", name="append_64", B=64, n=8192, spread=0.5, layout="nhd", bounds=True),
        # chunked prefill: a ragged batch of prompts of up to 8K tokens joins caches that hold some already
        _case("append", name="append_prompts", B=6, n=1000, new=8192, spread=0.6, ps=64, bounds=True),
        # float32, 64 columns of which half are rotated as neighbouring pairs, pages of an odd size, ragged
        _case("append", name="append_f32", B=7, n=100, new=300, spread=0.9, d=64, dtype="f32", ps=24, rot=32, interleaved=True),
        # a short chat: latency
        _case("decode", name="decode_2k", n=2047),
        # one sequence of 32K tokens: split over the length
        _case("decode", name="decode_32k", n=32768),
        # seven query heads on each of four KV heads, 128K tokens
        _case("decode", name="decode_128k_g7", n=131071, Hkv=4, G=7, ps=64),
        # batched serving: 16 sequences of 8K to 16K tokens, token-major pages
        _case("decode", name="decode_16x16k", B=16, n=16384, spread=0.5, ps=32, layout="nhd"),
        # a compressed cache in pages: a table per head, heads of different lengths, counts
        _case("decode", name="decode_cores", B=4, n=17039, spread=0.3, own_pages=True, count=True),
        # float32, 64 columns, pages of an odd size, lengths from none to all
        _case("decode", name="decode_f32", B=5, n=4099, spread=1.0, Hkv=4, G=2, d=64, dtype="f32", ps=24),
        # 8192 pages a head, 128 of them kept: the largest single context
        _case("select", name="select_128k", n=131072),
        # sparse attention of a batch: 64 pages of 32 tokens out of up to 1024
        _case("sparse", name="sparse_16x32k", B=16, spread=0.5, ps=32, keep=64),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """One more case: sizes log-uniform over the ranges, odd ones included, within the largest listed cost of its kind."""
    while True:
        kind = rng.choice(["append", "append", "decode", "decode", "decode", "decode", "select", "sparse"])
        Hkv, G = rng.choice([(8, 4), (8, 4), (4, 7), (8, 1), (1, 8), (2, 5), (4, 16)])
        f32 = rng.random() < 0.2
        d = rng.choice([64, 128, 96]) if f32 else rng.choice([128, 128, 128, 64, 256])
        kw = dict(B=_log(rng, 1, 64), Hkv=Hkv, G=G, d=d, dtype="f32" if f32 else "bf16", ps=rng.choice([16, 16, 32, 64, 128, 8, 24, 5]),
                  layout=rng.choice(["hnd", "nhd"]), spread=rng.choice([0.0, 0.3, 0.6, 1.0]))
        if kind == "append":
            inter = rng.random() < 0.3
            kw.update(n=_log(rng, 1, 32768), new=1 if rng.random() < 0.5 else _log(rng, 2, 8192), bounds=rng.random() < 0.5,
                      interleaved=inter, rot=rng.choice([d, d, d // 2, 0]))
        elif kind == "decode":
            kw.update(n=_log(rng, 1, 131072))
            if rng.random() < 0.3:
                kw.update(own_pages=True, count=True)
        else:
            kw.update(n=_log(rng, 256, 131072), keep=_log(rng, 4, 256))
        c = _case(kind, **kw)
        held = c["B"] * (c["n"] + c.get("new", 0)) * c["Hkv"] * d * 2 * (4 if f32 else 2)
        if work(c)["bytes"] <= _MAX_BYTES[kind] and held <= 3e9:
            return c


# ------------------------------------------------------------------------------------------ sizes


def _parts(c, salt):
    """Numbers in [1 - spread, 1], one per sequence, the same for every seed; the first is 1."""
    r = random.Random("%s %d" % (sorted((k, v) for k, v in c.items() if k != "name"), salt))
    return [1.0 if b == 0 else 1.0 - c["spread"] * r.random() for b in range(c["B"])]


def _lens(c):
    """Rows in the cache: [B] (before the call, for an append), or [B][Hkv] where every head has its own."""
    rows = [int(round(c["n"] * p)) for p in _parts(c, 0)]
    if not c.get("own_pages"):
        return rows
    r = random.Random(c["n"])
    return [[min(c["n"], int(ln * (0.9 + 0.2 * r.random()))) for _ in range(c["Hkv"])] for ln in rows]


def _news(c):
    return [max(1, int(round(c["new"] * p))) for p in _parts(c, 1)]


def _esz(c):
    return 2 if c["dtype"] == "bf16" else 4


def _flat(rows):
    return [x for r in rows for x in (r if isinstance(r, list) else [r])]


def _kept_rows(c):
    """Rows per KV head that a sparse step attends to, over all sequences."""
    total = 0
    for ln in _lens(c):
        pages = -(-ln // c["ps"])
        total += ln if pages <= c["keep"] else (c["keep"] - 1) * c["ps"] + ln - (pages - 1) * c["ps"]
    return total


def work(case):
    c, kind, e = case, case["kind"], _esz(case)
    H, G, d, ps = c["Hkv"], c["G"], c["d"], c["ps"]
    if kind == "append":
        news, lens = _news(c), _lens(c)
        T = sum(news)
        b = T * (2 * H + H * G) * d * e * 2 + 8 * c["B"]
        if c["bounds"]:   # written for every page touched, read for those that had rows
            touched = sum((ln + m - 1) // ps - ln // ps + 1 for ln, m in zip(lens, news))
            old = sum(ln % ps != 0 for ln in lens)
            b += (touched + old) * 2 * H * d * e
        return {"bytes": b, "flops": 3 * T * (H + H * G) * c["rot"]}
    rows = _flat(_lens(c)) if not c.get("own_pages") else []
    q_out = 2 * c["B"] * H * G * d * e
    if kind == "decode":
        head_rows = sum(_flat(_lens(c))) * (1 if c["own_pages"] else H)
        pages = sum(-(-x // ps) for x in _flat(_lens(c)))
        return {"bytes": head_rows * (2 * d * e + (4 if c["count"] else 0)) + 4 * pages + q_out, "flops": 4 * head_rows * G * d}
    # a sequence whose pages are all kept needs no score
    scored = sum(max(-(-x // ps) - c["first"] - c["last"], 0) for x in rows if -(-x // ps) > c["keep"])
    b = scored * H * 2 * d * e + q_out // 2 + 4 * sum(-(-x // ps) for x in rows) + 4 * c["B"] * H * (c["keep"] + 1)
    f = 4 * scored * H * G * d
    if kind == "sparse":
        b += _kept_rows(c) * H * 2 * d * e + q_out // 2
        f += 4 * _kept_rows(c) * H * G * d
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------------------------------ inputs


def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + salt * 7919 + 11) & 0x7FFFFFFFFFFFFFFF)
    return g


def _pool(c, pages, heads, g, fill):
    """Page storage seen as [pages, heads, ps, d]; token-major storage is the same view of [pages, ps, heads, d]."""
    shape = (pages, heads, c["ps"], c["d"]) if c["layout"] == "hnd" else (pages, c["ps"], heads, c["d"])
    t = torch.empty(shape, dtype=_DTYPES[c["dtype"]], device=DEV)
    if fill:
        t.normal_(generator=g)
    else:
        t.zero_()
    return t if c["layout"] == "hnd" else t.transpose(1, 2)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _norm(shape, g, c):
    return torch.randn(shape, generator=g, device=DEV).to(_DTYPES[c["dtype"]])


def prepare(case, seed):
    """Pages in random order in a pool a little larger than they need, keys and values N(0, 1) (in a cache that pages are
    picked from, keys that also drift from page to page, so that pages differ), queries N(0, 1)."""
    c, kind = case, case["kind"]
    B, H, G, d, ps = c["B"], c["Hkv"], c["G"], c["d"], c["ps"]
    g = _gen(seed, 1)
    s = {"case": c}
    lens = _lens(c)
    own_pages = bool(c.get("own_pages"))
    flat = _flat(lens)
    news = _news(c) if kind == "append" else [0] * len(flat)
    need = [-(-(a + m) // ps) for a, m in zip(flat, news)]
    used = sum(need)
    pages = used + 3
    width = max(max(need), 1) + 1
    perm = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros((len(flat), width), dtype=torch.int32, device=DEV)
    col = torch.arange(width, device=DEV)
    have = col.view(1, width) < torch.tensor(need, device=DEV).view(-1, 1)
    table[have] = perm[:used]
    s["table"] = table.view(B, -1, width)
    heads = 1 if own_pages else H
    s["k"], s["v"] = _pool(c, pages, heads, g, kind != "append"), _pool(c, pages, heads, g, kind != "append")
    s["lens"] = _i32(flat).view(B, -1)
    if kind in ("select", "sparse"):
        drift = torch.randn((pages, heads, 1, d), generator=g, device=DEV) * 0.7
        s["k"].copy_(s["k"].float() + drift)
    if kind in ("select", "sparse") or c.get("bounds"):
        s["k_min"] = s["k"].amin(2).contiguous()
        s["k_max"] = s["k"].amax(2).contiguous()
    if c.get("count"):
        s["count"] = 1 + torch.floor(-3.0 * torch.log(torch.rand((pages, heads, ps), generator=g, device=DEV).clamp_(min=1e-7))).int()
    if kind != "append":
        s["q"] = _norm((B, H * G, d), g, c)
        return s
    # the projections' output as one row per token: queries, keys, values
    T = sum(news)
    s["T"] = T
    s["qkv"] = _norm((T, H * G + 2 * H, d), g, c)
    off = [0]
    for m in news:
        off.append(off[-1] + m)
    s["seq_off"] = _i32(off)
    s["q_out"] = torch.zeros((T, H * G, d), dtype=_DTYPES[c["dtype"]], device=DEV)
    s["len_out"] = torch.zeros((B,), dtype=torch.int32, device=DEV)
    s["inv_freq"] = 500000.0 ** (-torch.arange(0, c["rot"], 2, device=DEV).float() / max(c["rot"], 1))
    if c["bounds"]:   # what the rows already there would have left: zeros
        s["k_min"].zero_()
        s["k_max"].zero_()
    return s


# ------------------------------------------------------------------------------------------ the plain form


def _rows_of(s, name):
    """Every row of every table, [B, Hkv, pages * ps, ...], in float32 (counts as they are)."""
    c, t = s["case"], s["table"].long().clamp(min=0)
    B, H = c["B"], c["Hkv"]
    pool = s[name]
    h = torch.arange(H, device=DEV) if pool.shape[1] == H else torch.zeros(H, dtype=torch.long, device=DEV)
    got = pool[t.expand(B, H, t.shape[2]), h.view(1, H, 1)]
    got = got.reshape(B, H, -1, *got.shape[4:])
    return got if got.dtype == torch.int32 else got.float()


def _plain_attn(s):
    c = s["case"]
    B, H, G, d = c["B"], c["Hkv"], c["G"], c["d"]
    k, v = _rows_of(s, "k"), _rows_of(s, "v")
    q = s["q"].float().view(B, H, G, d)
    x = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(d)
    if c.get("count"):
        x = x + torch.log(_rows_of(s, "count").float()).unsqueeze(2)
    live = torch.arange(x.shape[3], device=DEV).view(1, 1, 1, -1) < s["lens"].view(B, -1, 1, 1)
    x = torch.where(live, x, -math.inf)
    m = torch.amax(x, 3, keepdim=True).clamp(min=-1e30)
    w = torch.exp(x - m)
    total = w.sum(3, keepdim=True)
    out = torch.matmul(w, torch.where(live.transpose(2, 3), v, 0.0)) / total
    return torch.where(total > 0, out, 0.0).view(B, H * G, d).to(s["q"].dtype)


def _plain_select(s):
    """Page bounds and their order in 64 bits: the last page kept and the first one left out can be close."""
    c = s["case"]
    B, H, G, d, ps, keep = c["B"], c["Hkv"], c["G"], c["d"], c["ps"], c["keep"]
    t = s["table"].long()
    W = t.shape[2]
    n_pages = ((s["lens"] + ps - 1) // ps).view(B, 1, 1).long()
    h = torch.arange(H, device=DEV).view(1, H, 1)
    q = s["q"].double().view(B, H, G, d)
    at = t.expand(B, H, W)
    score = torch.matmul(q.clamp(min=0), s["k_max"][at, h].double().transpose(2, 3))
    score += torch.matmul(q.clamp(max=0), s["k_min"][at, h].double().transpose(2, 3))
    score = score.amax(2)
    p = torch.arange(W, device=DEV).view(1, 1, W)
    score = torch.where((p < c["first"]) | (p >= n_pages - c["last"]), math.inf, score)
    score = torch.where(p < n_pages, score, -math.inf)
    order = torch.sort(score, dim=2, descending=True, stable=True)[1][:, :, :keep]
    kept = torch.where(order < n_pages, order, W)
    kept = torch.sort(kept, dim=2)[0]
    if kept.shape[2] < keep:
        kept = torch.cat([kept, kept.new_full((B, H, keep - kept.shape[2]), W)], 2)
    table = torch.where(kept < W, torch.gather(at, 2, kept.clamp(max=W - 1)), -1).int()
    n_kept = torch.minimum(n_pages, torch.tensor(keep, device=DEV)).view(B, 1)
    lens = s["lens"] - (n_pages.view(B, 1) - n_kept).int() * ps
    return table, lens.int().expand(B, H).contiguous()


def _rotate(x, cos, sin, rot, interleaved):
    """x [T, heads, d] in float32; cos, sin [T, rot / 2]."""
    c, s = cos.unsqueeze(1), sin.unsqueeze(1)
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * c - b * s, b * c + a * s], 3).flatten(2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * c - b * s, b * c + a * s], 2)
    return torch.cat([y, x[..., rot:]], 2)


def _plain_append(s):
    c = s["case"]
    H, HG, ps, rot = c["Hkv"], c["Hkv"] * c["G"], c["ps"], c["rot"]
    tok = torch.arange(s["T"], device=DEV)
    seq = torch.bucketize(tok, s["seq_off"][1:].long(), right=True)
    lens = s["lens"].view(-1)
    row = lens[seq] + tok - s["seq_off"][seq]
    page = s["table"][seq, 0, (row // ps).long()].long()
    x = s["qkv"].float()
    if rot:
        angle = row.double().unsqueeze(1) * s["inv_freq"].double()   # in 64 bits: far positions
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        x = torch.cat([_rotate(x[:, :HG + H], cos, sin, rot, c["interleaved"]), x[:, HG + H:]], 1)
    x = x.to(s["qkv"].dtype)
    k = x[:, HG:HG + H]
    s["q_out"].copy_(x[:, :HG])
    s["k"][page, :, (row % ps).long()] = k
    s["v"][page, :, (row % ps).long()] = x[:, HG + H:]
    s["len_out"].copy_(lens + (s["seq_off"][1:] - s["seq_off"][:-1]))
    out = {"q": s["q_out"], "k": s["k"], "v": s["v"], "len": s["len_out"]}
    if c["bounds"]:
        fresh = torch.zeros(s["k_min"].shape[0], dtype=torch.int32, device=DEV)   # pages whose first row is new
        fresh.scatter_reduce_(0, page, (row % ps == 0).int(), "amax")
        at = page.view(-1, 1, 1).expand(-1, H, c["d"])
        for name, way, far in (("k_min", "amin", math.inf), ("k_max", "amax", -math.inf)):
            b = torch.where(fresh.view(-1, 1, 1) > 0, far, s[name].float())
            b.scatter_reduce_(0, at, k.float(), way)
            s[name].copy_(b)
            out[name] = s[name]
    return out


# ------------------------------------------------------------------------------------------ one pass


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if own:
        return _own(s, c, kind)
    if kind == "append":
        return _plain_append(s)
    if kind == "decode":
        return _plain_attn(s)
    table, lens = _plain_select(s)
    if kind == "select":
        return {"table": table, "len": lens}
    return {"table": table, "len": lens, "out": _plain_attn(dict(s, table=table, lens=lens))}


def _own(s, c, kind):
    from paper_2603_14303_b200 import binding as sc
    if "cache" not in s:   # what a program keeps with its cache
        s["cache"] = sc.PagedCache(s["k"], s["v"], s["table"], s.get("count"), s.get("k_min"), s.get("k_max"))
        if kind != "append":
            s["ws"] = sc.paged_decode_workspace(c["B"], c["Hkv"] * c["G"], c["Hkv"], c["d"], DEV)
    cache = s["cache"]
    if kind == "append":
        H, HG = c["Hkv"], c["Hkv"] * c["G"]
        x = s["qkv"]
        sc.paged_append(cache, x[:, HG:HG + H], x[:, HG + H:], s["seq_off"], s["lens"], inv_freq=s["inv_freq"] if c["rot"] else None,
                        interleaved=c["interleaved"], q=x[:, :HG], q_out=s["q_out"], len_out=s["len_out"])
        out = {"q": s["q_out"], "k": s["k"], "v": s["v"], "len": s["len_out"]}
        if c["bounds"]:
            out.update(k_min=s["k_min"], k_max=s["k_max"])
        return out
    if kind == "decode":
        return sc.paged_decode_attn(s["q"], cache, s["lens"], workspace=s["ws"])
    table, lens = sc.paged_select(s["q"], cache, s["lens"], c["keep"], c["first"], c["last"])
    if kind == "select":
        return {"table": table, "len": lens}
    out = sc.paged_decode_attn(s["q"], cache.over(table), lens, workspace=s["ws"])
    return {"table": table, "len": lens, "out": out}


# ------------------------------------------------------------------------------------------ from the definitions, in 64 bits


def _attend(s, c, b, h, pages, length):
    """Eq. 4 for the query group of one head over the first `length` rows of `pages`."""
    hp = h if s["k"].shape[1] > 1 or c["Hkv"] == 1 else 0
    q = s["q"][b, h * c["G"]:(h + 1) * c["G"]].double()
    if length == 0:
        return torch.zeros_like(q)
    pages = pages[:-(-length // c["ps"])].long()
    k = s["k"][pages, hp].reshape(-1, c["d"])[:length].double()
    v = s["v"][pages, hp].reshape(-1, c["d"])[:length].double()
    x = q @ k.T * c["d"] ** -0.5
    if c.get("count"):
        x += s["count"][pages, hp].reshape(-1)[:length].double().log()
    return torch.softmax(x, 1) @ v


def _exact_rows(c, x, pos, freq):
    """The rotation of x [T, heads, d] as a complex product, positions [T]."""
    x = x.double()
    r = c["rot"]
    if not r:
        return x
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos.double()[:, None] * freq.double()[None])[:, None]
    if c["interleaved"]:
        z = torch.view_as_complex(x[..., :r].unflatten(-1, (r // 2, 2)).contiguous()) * turn
        return torch.cat([torch.view_as_real(z).flatten(-2), x[..., r:]], -1)
    z = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * turn
    return torch.cat([z.real, z.imag, x[..., r:]], -1)


def exact(case, seed):
    c, kind = case, case["kind"]
    if kind == "select":   # whole numbers only
        return None
    s = prepare(case, seed)
    B, H, G, ps = c["B"], c["Hkv"], c["G"], c["ps"]
    lens = s["lens"].tolist()
    if kind == "append":
        HG = H * G
        out = {n: s[n].double().contiguous() for n in ("k", "v", "k_min", "k_max") if n in s}
        out["q"] = s["q_out"].double()
        off, table = s["seq_off"].tolist(), s["table"].tolist()
        for b in range(B):
            a, e, n0 = off[b], off[b + 1], lens[b][0]
            pos = torch.arange(n0, n0 + e - a, device=DEV)
            qk = _exact_rows(c, s["qkv"][a:e, :HG + H], pos, s["inv_freq"])
            out["q"][a:e] = qk[:, :HG]
            page = s["table"][b, 0, pos // ps].long()
            out["k"][page, :, pos % ps] = qk[:, HG:]
            out["v"][page, :, pos % ps] = s["qkv"][a:e, HG + H:].double()
            if c["bounds"]:
                for j in range(n0 // ps, (n0 + e - a - 1) // ps + 1):
                    rows = qk[max(j * ps - n0, 0):(j + 1) * ps - n0, HG:]
                    lo, hi = rows.amin(0), rows.amax(0)
                    pg = table[b][0][j]
                    if j * ps < n0:
                        lo, hi = torch.minimum(lo, out["k_min"][pg]), torch.maximum(hi, out["k_max"][pg])
                    out["k_min"][pg], out["k_max"][pg] = lo, hi
        out["len"] = None
        return out
    if kind == "decode":
        out = [torch.cat([_attend(s, c, b, h, s["table"][b, h if c["own_pages"] else 0], lens[b][h if c["own_pages"] else 0])
                          for h in range(H)]) for b in range(B)]
        return torch.stack(out)
    out = torch.empty_like(s["q"], dtype=torch.float64)
    for b in range(B):
        n = -(-lens[b][0] // ps)
        ids = s["table"][b, 0, :n].long()
        tail = lens[b][0] - (n - 1) * ps
        for h in range(H):
            chosen, length = ids, lens[b][0]
            if n > c["keep"]:
                q = s["q"][b, h * G:(h + 1) * G].double()[:, None]
                bound = torch.maximum(q * s["k_min"][ids, h].double(), q * s["k_max"][ids, h].double()).sum(2).amax(0)
                bound[:c["first"]] = math.inf
                bound[n - c["last"]:] = math.inf
                chosen = ids[bound.argsort(descending=True, stable=True)[:c["keep"]].sort()[0]]
                length = (c["keep"] - 1) * ps + tail
            out[b, h * G:(h + 1) * G] = _attend(s, c, b, h, chosen, length)
    return {"table": None, "len": None, "out": out}
