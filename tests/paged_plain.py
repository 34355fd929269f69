"""Plain forms of the calls on a paged cache, in 64 bits on the CPU, and random caches for their tests."""
import math

import torch

from paper_2603_14303_b200 import binding

DEV = "cuda:0"


def pool(P, heads, ps, d, dtype, layout, gen, fill=True):
    """[P, heads, ps, d] on the CPU: head-major, token-major, or with gaps between rows, heads and pages."""
    t = torch.randn((P, heads, ps, d), generator=gen).to(dtype) if fill else torch.zeros((P, heads, ps, d), dtype=dtype)
    return t


def on_device(t, layout):
    """A CPU pool [P, heads, ps, d] on the device in the storage that `layout` names, seen as [P, heads, ps, d]."""
    P, H, ps, d = t.shape
    if layout == "hnd":
        return t.to(DEV)
    if layout == "nhd":
        return t.transpose(1, 2).contiguous().to(DEV).transpose(1, 2)
    assert layout == "gaps"   # wider rows, a spare head and a spare row per page
    big = torch.full((P, H + 1, ps + 1, d + 16), 7.0, dtype=t.dtype, device=DEV)
    view = big[:, :H, :ps, :d]
    view.copy_(t.to(DEV))
    return view


def tables(lens, ps, P, width, gen):
    """Random distinct pages for tables of the given lengths; entries behind a table's end name no page."""
    need = [-(-n // ps) for n in lens]
    assert sum(need) <= P and max(need, default=0) <= width
    perm = torch.randperm(P, generator=gen).tolist()
    out, at = [], 0
    for k in need:
        out.append(perm[at:at + k] + [-5 if i % 2 else 2 ** 30 for i in range(width - k)])
        at += k
    return torch.tensor(out, dtype=torch.int32).view(len(lens), width)


def rows_of(t, table, n, h, ps):
    """The first n rows of a table, [n, ...] in 64 bits; h: the head inside the pages."""
    ids = table[:-(-n // ps)].long()
    return t[ids, h].reshape(-1, *t.shape[3:])[:n].double()


def attention(q, k, v, table, lens, scale=0.0, count=None, rounding=False):
    """q [B, Hq, d]; k, v [P, heads, ps, d]; table [B, th, W]; lens [B, th].  Eq. 4 row by row of the batch, in 64 bits.

    ``rounding``: also what scores in fp32 can be off by, as a bound on each output's error.  A sum of d products in any order, each of them
    in at most d roundings, is off by at most d 2^-24 sum |q_c k_tc|; the score made of it is rounded twice more: delta_t.  Weights
    w_t exp(e_t) with |e_t| <= delta_t move sum w v / sum w by sum p_t |e_t| |v_t - out| to first order (p = w / sum w); doubled for what
    is left of the series (delta < 1/2 here)."""
    B, Hq, d = q.shape
    bound = torch.zeros((B, Hq, d), dtype=torch.float64)
    heads, ps, th = k.shape[1], k.shape[2], table.shape[1]
    Hkv = max(heads, th)
    G = Hq // Hkv
    out = torch.zeros((B, Hq, d), dtype=torch.float64)
    for b in range(B):
        for h in range(Hkv):
            t = h if th > 1 else 0
            n = min(max(int(lens[b, t]), 0), table.shape[2] * ps)
            if n == 0:
                continue
            hp = h if heads > 1 else 0
            kk, vv = (rows_of(x, table[b, t], n, hp, ps) for x in (k, v))
            x = q[b, h * G:(h + 1) * G].double() @ kk.T * (scale if scale else 1.0 / math.sqrt(d))
            if count is not None:
                x = x + rows_of(count, table[b, t], n, hp, ps).log()
            w = torch.exp(x - x.amax(1, keepdim=True))
            o = w @ vv / w.sum(1, keepdim=True)
            out[b, h * G:(h + 1) * G] = o
            if rounding:
                qq, sc = q[b, h * G:(h + 1) * G].double(), scale if scale else 1.0 / math.sqrt(d)
                delta = d * 2.0 ** -24 * sc * (qq.abs() @ kk.abs().T) + 2.0 ** -23 * x.abs()
                assert float((delta * (w > 1e-12)).max()) < 0.5
                p = w / w.sum(1, keepdim=True) * delta
                bound[b, h * G:(h + 1) * G] = 2 * torch.einsum("gt,gtc->gc", p, (vv.unsqueeze(0) - o.unsqueeze(1)).abs())
    return (out, bound) if rounding else out


def select(q, k_min, k_max, table, lens, ps, keep, n_first, n_last):
    """The pages picked, from bounds in 64 bits; ties to the earlier page."""
    B, Hq, d = q.shape
    th, heads = table.shape[1], k_min.shape[1]
    Hkv = max(heads, th)
    G = Hq // Hkv
    out = torch.full((B, Hkv, keep), -1, dtype=torch.int32)
    ln = torch.zeros((B, Hkv), dtype=torch.int32)
    for b in range(B):
        for h in range(Hkv):
            t, hp = (h if th > 1 else 0), (h if heads > 1 else 0)
            n_rows = min(max(int(lens[b, t]), 0), table.shape[2] * ps)
            n = -(-n_rows // ps)
            ids = table[b, t, :n].long()
            if n <= keep:
                out[b, h, :n] = ids.int()
                ln[b, h] = n_rows
                continue
            qq = q[b, h * G:(h + 1) * G].double().unsqueeze(1)
            bound = torch.maximum(qq * k_min[ids, hp].double(), qq * k_max[ids, hp].double()).sum(2)
            bound = torch.where(bound.isnan().any(0), math.inf, bound.amax(0))   # (not a number: above all)
            order = sorted(range(n), key=lambda p: (0 if p < n_first or p >= n - n_last else 1, -float(bound[p]), p))
            out[b, h] = ids[sorted(order[:keep])].int()
            ln[b, h] = n_rows - (n - keep) * ps
    return out, ln


def rotate(x, pos, inv_freq, pairs):
    """x [T, H, d] and positions [T], in 64 bits: the rotated rows, and |x1| + |x2| of each element's pair (0 where it is only copied)."""
    x = x.double()
    r = 2 * inv_freq.numel()
    a = pos.double()[:, None] * inv_freq.double()[None]
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    y, mass = x.clone(), torch.zeros_like(x)
    i1 = torch.arange(0, r, 2) if pairs else torch.arange(r // 2)
    i2 = i1 + 1 if pairs else i1 + r // 2
    y[..., i1] = x[..., i1] * c - x[..., i2] * s
    y[..., i2] = x[..., i2] * c + x[..., i1] * s
    mass[..., i1] = mass[..., i2] = x[..., i1].abs() + x[..., i2].abs()
    return y, mass


def assert_rotated(got, want, mass, what):
    """One rounding to the storage type (half a step), and in fp32: sine and cosine off by at most 2.2e-7 (the angle, at most half a
    turn, rounded to 24 bits: pi 2^-25; the functions' two last places: 1.2e-7), three roundings of the products and their sum: 2^-24
    each of |x1| + |x2| at most.  A value that is only copied keeps its bits."""
    eps = torch.finfo(got.dtype).eps / 2
    err = (got.double().cpu() - want).abs()
    tol = eps * want.abs() * (1 + 2.0 ** -8) + mass * (2.2e-7 + 3 * 2.0 ** -24) * (1 + 2.0 ** -6)
    assert bool((err <= tol).all()), (what, float((err - tol).max()))


def same_bits(a, b):
    kind = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.cpu().contiguous().view(kind), b.cpu().contiguous().view(kind))


def status_word():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def ok(status):
    binding.check_status(status)
