"""Every kernel of the attention over a quantised cache, a CTA per unit and in
equal runs of tiles, at the contents and lengths where each can go wrong.

Every test asserts which kernel its sizes run (quant_ways.py), so that a change
of the choice does not empty it.  Tolerances as derived in test_gpu_quant.py;
those of single tests stand beside them."""
import math

import numpy as np
import pytest

from paper_2401_16757_gb300 import capi

from quant_ways import WAYS, tiling
from test_gpu_quant import SENT, Attend, _dt, _stream, _torch

pytestmark = pytest.mark.gpu

EPS = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
way_of_call = pytest.mark.parametrize("way", sorted(WAYS))


def _lengths(n, tokens, cap):
    """None, one, a tile's edges, all, and many short ones, so that a run of tiles holds pieces of several sequences."""
    lens = [cap, 0, 1, 127, 128, 129, cap - 1, cap // 2 + 5, tokens, max(0, tokens - 2)] + [cap // 3 + 77 * i for i in range(5)]
    lens = [min(cap, x) for x in lens]
    lens = lens[:n] + [(i * 37) % 131 if i % 4 else (i * 613) % (cap + 1) for i in range(n - len(lens[:n]))]
    counts = [tokens - i % (tokens + 1) if i % 3 == 2 else tokens for i in range(n)]
    return lens, counts


class Wide(Attend):
    """Attend's inputs, made on the GPU (some of these caches are large): of a way's sizes."""

    def __init__(self, way, dtype="bf16", fmt="e4m3", block=32, lens=None, counts=None, seed=0, kv_stride=0, seq_stride=0):
        torch = _torch()
        (n, t, h, kv, d, cap), self.route = WAYS[way]
        usual = _lengths(n, t, cap)
        lens, counts = usual[0] if lens is None else lens, usual[1] if counts is None else counts
        self.__dict__.update(dtype=dtype, fmt=fmt, n=n, t=t, h=h, kv=kv, d=d, max_seq=cap, block=block, scale=0.0, pad=0, kd=kv * d)
        self.lens, self.counts = np.asarray(lens, dtype=np.int32), None if counts == "all" else np.asarray(counts, dtype=np.int32)
        g = torch.Generator(device="cuda").manual_seed(seed)
        top, blocks = {"i8": 127.0, "e4m3": 448.0}[fmt], -(-cap // block)
        self.q = (torch.randn(n, t, h * d, generator=g, device="cuda") * 1.5).to(_dt(dtype))
        row = torch.arange(cap, device="cuda")
        used = torch.from_numpy(np.clip(self.lens, 0, cap)).cuda()
        hidden = row >= used[:, None]

        def codes():
            x = (torch.randn(n, cap, kv * d, generator=g, device="cuda") * (top / 4)).clamp_(-top, top)
            x = (x.round_() if fmt == "i8" else x).to(_dt(fmt))
            raw = torch.randint(0, 256, (997, kv * d), generator=g, device="cuda").to(torch.uint8)  # codes behind the rows in use: anything
            x.view(torch.uint8)[hidden] = raw[torch.arange(int(hidden.sum()), device="cuda") % 997]
            return x

        def scales():
            s = torch.exp2(torch.rand(n, kv, blocks, generator=g, device="cuda") * 2 - 1) * (4 / top)
            behind = (torch.arange(blocks, device="cuda") >= -(-used[:, None] // block))[:, None].expand_as(s)
            return torch.where(behind, torch.tensor([math.nan, math.inf, -1.0], device="cuda")[torch.arange(blocks, device="cuda") % 3], s)

        self.k, self.v, self.ks, self.vs = codes(), codes(), scales(), scales()
        self.out = torch.full((n, t, h * d), SENT, dtype=_dt(dtype), device="cuda")
        self.lse = torch.full((n, h, t), SENT, device="cuda")

    def args(self, **kw):
        a = super().args(**kw)
        assert tiling(a) == self.route
        return a

    def lost(self):
        """Of a query's largest product of a probability and its value scale, what every such product may be off by."""
        rows = self.t * (self.h // self.kv)
        return 2.0 ** (-39 if rows <= 16 or (rows <= 32 and self.d == 64) else -32)

    def check(self, skip=()):
        """As Attend's, with two terms of its own: the promised bound of small products for these sizes, and for fp16
        results half of its least step, 2^-25 (below 2^-14 a rounding is no longer relative)."""
        torch = _torch()
        t, h, kv, d, B = self.t, self.h, self.kv, self.d, self.block
        grp, floor = h // kv, 2.0 ** -25 if self.dtype == "f16" else 0.0
        for b in range(self.n):
            ln, c = int(self.lens[b]), t if self.counts is None else int(self.counts[b])
            if b in skip:
                ln = c = 0
            assert (self.out[b, c:] == SENT).all() and (self.lse[b, :, c:] == SENT).all()
            if c == 0:
                continue
            got = self.out[b, :c].double().view(c, kv, grp, d).permute(1, 2, 0, 3)  # [kv, grp, c, d]
            lse = self.lse[b, :, :c].double().view(kv, grp, c)
            if ln == 0:
                assert (got == 0).all() and (lse == -math.inf).all()
                continue
            row = torch.arange(ln, device="cuda")
            seen = row <= (ln - c + torch.arange(c, device="cuda"))[:, None]
            vs = self.vs[b][:, row // B].double()
            code = self.v[b, :ln].double().view(ln, kv, d).transpose(0, 1)
            k = self.k[b, :ln].double().view(ln, kv, d).transpose(0, 1) * self.ks[b][:, row // B].double()[..., None]
            q = self.q[b, :c].double().view(c, kv, grp, d).permute(1, 2, 0, 3).reshape(kv, grp * c, d)
            s = (q @ k.transpose(1, 2) / math.sqrt(d)).view(kv, grp, c, ln)
            size = (q.abs() @ k.abs().transpose(1, 2) / math.sqrt(d)).view(kv, grp, c, ln)
            off = size.masked_fill(~seen, 0).amax(-1) * (d + 8) * 2.0 ** -23
            s = s.masked_fill(~seen, -math.inf)
            true = torch.logsumexp(s, -1)
            p = torch.exp(s - true.masked_fill(true == -math.inf, 0)[..., None])
            pv = p * vs[:, None, None]
            want, size = ((pv.view(kv, grp * c, ln) @ x).view(kv, grp, c, d) for x in (code, code.abs()))
            most = pv.amax(-1)[..., None] * code.abs().sum(1)[:, None, None]
            rel = (2 * off + 2.0 ** -21 + (ln / 16 + 40) * 2.0 ** -23 + 2.0 ** -22)[..., None]
            tol = EPS[self.dtype] * want.abs() + floor + rel * size + self.lost() * most
            assert ((got - want).abs() <= tol * (1 + 2.0 ** -10)).all(), (b, ((got - want).abs() / tol).max().item())
            hit = torch.isfinite(true)
            assert (lse[~hit] == -math.inf).all() and (got[~hit] == 0).all()
            tol = off + 2.0 ** -20 + (ln / 16 + 40) * 2.0 ** -23 + 2.0 ** -22 * true.abs()
            assert ((lse - true).abs() <= tol)[hit].all(), b


def _bits(*tensors):
    return [x.clone().view(_torch().uint8) for x in tensors]


@way_of_call
@pytest.mark.parametrize("dtype,fmt,block", [("bf16", "e4m3", 64), ("bf16", "i8", 16), ("f16", "e4m3", 32), ("f16", "i8", 128)])
def test_definition_and_the_same_bits(way, dtype, fmt, block):
    torch = _torch()
    c = Wide(way, dtype, fmt, block, seed=21)
    c.call()
    capi.device_sync()
    c.check()
    want = _bits(c.out, c.lse)
    for _ in range(3):
        c.out.fill_(SENT), c.lse.fill_(SENT)
        c.call()
    capi.device_sync()
    assert all(torch.equal(x, y) for x, y in zip(want, _bits(c.out, c.lse)))


@way_of_call
def test_bad_sequences_are_left_alone(way):
    (n, t, h, kv, d, cap), _ = WAYS[way]
    for i, (length, count) in enumerate(((cap + 1, t), (-1, t), (cap, t + 1), (cap, -1))):
        lens, counts = _lengths(n, t, cap)
        lens[-1], counts[-1] = length, count
        lens[1], counts[1] = (-2 ** 31, t) if i % 2 else (5, 2 ** 31 - 1)
        c = Wide(way, lens=lens, counts=counts, seed=22)
        c.call()
        with pytest.raises(capi.SwapnetError) as e:
            capi.device_sync()
        assert e.value.code == capi.ERR_INVALID_ARG
        c.check(skip=(1, n - 1))
    capi.device_sync()


@way_of_call
def test_graphs_and_streams(way):
    """Captured, replayed on other inputs of other lengths; two calls at once with workspaces of their own."""
    torch = _torch()
    (n, t, h, kv, d, cap), _ = WAYS[way]
    lens, counts = _lengths(n, t, cap)
    a, b = Wide(way, seed=23), Wide(way, lens=lens[::-1], counts=counts[::-1], seed=24)
    a.call(), b.call()
    capi.device_sync()
    want = [_bits(x.out, x.lse) for x in (a, b)]
    keep = a._keep
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.call(lens=keep[0].data_ptr(), space=a.space)
    a.out.fill_(SENT), a.lse.fill_(SENT)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want[0], _bits(a.out, a.lse)))
    kept = [getattr(a, name).clone() for name in ("q", "k", "v", "ks", "vs")] + [x.clone() for x in keep]
    for name in ("q", "k", "v", "ks", "vs"):
        getattr(a, name).copy_(getattr(b, name))
    for x, y in zip(keep, b._keep):
        x.copy_(y)
    a.out.fill_(SENT), a.lse.fill_(SENT)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want[1], _bits(a.out, a.lse)))
    for x, y in zip([getattr(a, name) for name in ("q", "k", "v", "ks", "vs")] + list(keep), kept):
        x.copy_(y)
    for x in (a, b):
        x.out.fill_(SENT), x.lse.fill_(SENT)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for x, s in ((a, streams[0]), (b, streams[1])):
            x.call(stream=s.cuda_stream, space=x.space, lens=x._keep[0].data_ptr())
    torch.cuda.synchronize()
    for w, x in zip(want, (a, b)):
        assert all(torch.equal(u, v) for u, v in zip(w, _bits(x.out, x.lse)))


@way_of_call
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_scales_that_are_no_numbers(way, fmt):
    """A block of one sequence and head with such a scale and any codes: the queries that see one of its rows get no number,
    all others the same bits."""
    torch = _torch()
    (n, t, h, kv, d, cap), _ = WAYS[way]
    B, at, group = 16, n - 1, h // kv
    lens, counts = _lengths(n, t, cap)
    lens[at], counts[at] = min(cap, t + 180), t
    good = Wide(way, fmt=fmt, block=B, lens=lens, counts=counts, seed=25)
    good.call()
    capi.device_sync()
    ref = good.out.view(n, t, kv, group, d).clone()
    for which, value in (("ks", math.nan), ("vs", math.nan), ("vs", math.inf)):
        c = Wide(way, fmt=fmt, block=B, lens=lens, counts=counts, seed=25)
        ln = lens[at]
        block = (ln - 2) // B  # the last rows but one, seen by the last queries
        getattr(c, which)[at, kv - 1, block] = value
        for x in (c.k, c.v):
            x.view(torch.uint8)[at, block * B:(block + 1) * B, (kv - 1) * d:] = 0x7f
        c.call()
        capi.device_sync()
        first = max(0, block * B - (ln - t))  # the first query that sees the block
        out = c.out.view(n, t, kv, group, d)
        hit = out[at, first:, kv - 1]
        assert not torch.isfinite(hit).any() if value == math.inf else torch.isnan(hit).all()
        same = torch.ones_like(out, dtype=torch.bool)
        same[at, first:, kv - 1] = False
        assert torch.equal(out[same], ref[same])


def _full(way, dtype, fmt, block, seed=0):
    """A call whose sequences are all full; rows seen by each query."""
    (n, t, h, kv, d, cap), _ = WAYS[way]
    c = Wide(way, dtype, fmt, block, lens=[cap] * n, counts="all", seed=seed)
    return c, (cap - t + _torch().arange(1, t + 1, device="cuda"))


@way_of_call
@pytest.mark.parametrize("least", [2.0 ** -100, 2.0 ** -48])
def test_zeros_beside_large_values(way, least):
    """All scores equal; every other block of 16 rows has small values, the others large ones: the mean of what is seen."""
    torch = _torch()
    c, n = _full(way, "bf16", "i8", 16)
    c.q.zero_(), c.v.fill_(64)
    if least < 2.0 ** -48:
        c.v[:, torch.arange(c.max_seq, device="cuda") % 32 < 16] = 0
    for large in (1.0, 2.0 ** 40, 2.0 ** 64):
        c.vs[:, :, 0::2], c.vs[:, :, 1::2] = least, large
        c.call()
        capi.device_sync()
        big = (n // 32 * 16 + (n % 32 - 16).clamp(min=0)).double()
        want = (64 * large * big + (64 * least if least == 2.0 ** -48 else 0.0) * (n - big)) / n
        # half a step of bf16; sums of n equal terms, two parts of p and the division: (n / 16 + 40) 2^-23
        tol = want * (2.0 ** -8 + (c.max_seq / 16 + 40) * 2.0 ** -23)
        assert ((c.out.double() - want[:, None]).abs() <= tol[:, None]).all(), large
        assert ((c.lse.double() - torch.log(n.double())).abs() <= (c.max_seq / 16 + 40) * 2.0 ** -22).all()


@way_of_call
@pytest.mark.parametrize("score", [-3000.0, 3000.0])
def test_scores_far_from_zero(way, score):
    """All scores equal and far from what exponentials hold: the mean of the values seen; then one key above all others."""
    torch = _torch()
    c, n = _full(way, "f16", "i8", 32)
    ln, d = c.max_seq, c.d
    c.k.fill_(64 if score > 0 else -64), c.ks.fill_(1.0), c.vs.fill_(2.0 ** -6)
    c.q.fill_(4.0)
    c.scale = 3000 / (4.0 * 64 * d)
    c.v.zero_()
    c.v[:, ::2] = 64
    c.call()
    capi.device_sync()
    want = ((n + 1) // 2).double() / n
    # half a step of fp16; the scores are exact but for one rounding each: 2^-22 of 3000 / ln 2 bits, for all the same
    assert ((c.out.double() - want[:, None]).abs() <= (want * (2.0 ** -11 + (ln / 16 + 40) * 2.0 ** -23))[:, None]).all()
    assert ((c.lse.double() - score - torch.log(n.double())).abs() <= 3000 * 2.0 ** -21 + (ln / 16 + 40) * 2.0 ** -22).all()
    at = ln - c.t - 30
    c.k[:, at] = 127 if score > 0 else -1
    c.call()
    capi.device_sync()
    assert (c.out == (1.0 if at % 2 == 0 else 0.0)).all()


@way_of_call
def test_scores_that_climb(way):
    """Each tile's scores far above all before it, the last tile's far below: every reference, sum and output of what came
    before is brought up to date, tile after tile and across runs."""
    torch = _torch()
    c, n = _full(way, "f16", "i8", 16)
    ln, d, t = c.max_seq, c.d, c.t
    tile = torch.arange(ln, device="cuda") // 128
    c.q.fill_(1.0), c.ks.fill_(1.0), c.vs.fill_(2.0 ** -6)
    climb = torch.where(tile < tile[-1], tile, 0).to(torch.int8)
    c.k.copy_(climb[None, :, None].expand_as(c.k))
    c.scale = 20.0 / d  # 20 a tile: e^20 times the weight of the tile before
    c.v.copy_(((torch.arange(ln, device="cuda") % 5) * 16)[None, :, None].expand_as(c.v))
    c.call()
    capi.device_sync()
    s, v = 20.0 * climb.double(), (torch.arange(ln, device="cuda") % 5).double() / 4
    seen = torch.arange(ln, device="cuda") < n[:, None]
    p = torch.where(seen, torch.exp(s - s.max()), torch.zeros(1, dtype=torch.float64, device="cuda"))
    want, lse = (p * v).sum(1) / p.sum(1), s.max() + torch.log(p.sum(1))
    # scores of up to 20 a tile, in bits 1.5 times that, are rounded twice, by 2^-24 each; then as everywhere
    rel = 2 * 1.5 * 20 * (ln / 128) * 2.0 ** -23 + 2.0 ** -20 + (ln / 16 + 40) * 2.0 ** -23
    assert ((c.out.double() - want[:, None]).abs() <= (want * (2.0 ** -11 + rel))[:, None]).all()
    assert ((c.lse.double() - lse).abs() <= rel + 2.0 ** -22 * lse).all()


@way_of_call
def test_a_dominant_key_hides_nothing(way):
    """Beside a key that gets nearly everything and has the value 0, the others decide the output."""
    torch = _torch()
    c, n = _full(way, "f16", "i8", 16)
    c.k.zero_(), c.v.fill_(64), c.ks.fill_(1.0), c.vs.fill_(2.0 ** -6)
    c.q.fill_(0.5)
    c.scale = 16.0 / (0.5 * 4 * c.d)
    c.k[:, 5] = 4  # score 16: e^16 = 8.9e6 times the others
    c.v[:, 5] = 0
    c.call()
    capi.device_sync()
    want = (n - 1).double() / ((n - 1).double() + math.exp(16.0))
    # fp16 results of 2e-5 to 8e-4 (below 2^-14 in steps of 2^-24: half of one is 2^-25); p: 2^-21 of the sums, and of every
    # key up to 2^-39 or 2^-32 of the largest product
    tol = want * (2.0 ** -11 + 2.0 ** -13) + 2.0 ** -25 + n.double() * c.lost()
    assert ((c.out.double() - want[:, None]).abs() <= tol[:, None]).all()


@way_of_call
@pytest.mark.parametrize("dtype,fmt,block", [("bf16", "e4m3", 64), ("f16", "i8", 16)])
def test_sequence_strides(way, dtype, fmt, block):
    """A sequence's rows a padded number of codes apart, no multiple of a row's, and the sequences' rows in turn: the bits of the
    packed call, whatever lies between."""
    torch = _torch()
    c = Wide(way, dtype, fmt, block, seed=26)
    c.call()
    capi.device_sync()
    want, (n, cap, kd) = _bits(c.out, c.lse), c.k.shape
    for kv_stride, seq_stride in ((kd, kd * cap + 48), (kd + 16, (kd + 16) * cap + 16), (n * kd, kd), (n * kd + 16, kd)):
        total = (n - 1) * seq_stride + (cap - 1) * kv_stride + kd
        flat = [torch.full((total,), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(2)]
        for x, of in zip(flat, (c.k, c.v)):
            torch.as_strided(x, (n, cap, kd), (seq_stride, kv_stride, 1)).copy_(of.view(torch.uint8))
        c.out.fill_(SENT), c.lse.fill_(SENT)
        c.call(k=flat[0].data_ptr(), v=flat[1].data_ptr(), kv_stride=kv_stride, seq_stride=seq_stride)
        capi.device_sync()
        assert all(torch.equal(x, y) for x, y in zip(want, _bits(c.out, c.lse))), (kv_stride, seq_stride)


@way_of_call
def test_small_products_beside_large_ones(way):
    """One key in 32 has nearly all of the weight and the value 0 in every dim but the first; the others' products are 2^-30 of
    its own, or 2^-36 where a call promises 2^-39 of the largest: what they add up to is the output of the other dims."""
    torch = _torch()
    c, n = _full(way, "bf16", "i8", 16)
    exact = c.lost() == 2.0 ** -39
    below = 35.63 if exact else 29.63  # bits, no whole number of them: a lost low part shows
    c.k.zero_(), c.ks.fill_(1.0), c.vs.fill_(2.0 ** 20)
    c.q.fill_(0.5)
    heavy = torch.arange(c.max_seq, device="cuda") % 32 == 9
    c.k[:, heavy] = 4
    c.scale = below * math.log(2) / (0.5 * 4 * c.d)  # of the heavy keys' scores
    c.v.fill_(64)
    first = torch.arange(c.kv, device="cuda") * c.d
    c.v[:, heavy] = 0
    for e in first.tolist():
        c.v[:, heavy, e] = 64
    c.call()
    capi.device_sync()
    many = ((n - 1 - 9) // 32 + 1).clamp(min=0).double()  # heavy keys seen
    light, w = n.double() - many, 2.0 ** -below
    want = light * w / (many + light * w) * 64 * 2.0 ** 20
    # a score of up to 36 bits, rounded three times by 2^-24: 36 2^-22 of p; sums; half a step of bf16; what is promised of
    # every light key's product, as a share of the heavy keys' sum
    tol = want * (2.0 ** -8 + 36 * 2.0 ** -22 + (c.max_seq / 16 + 40) * 2.0 ** -23) + light / many * c.lost() * 64 * 2.0 ** 20
    assert (tol < want / 3).all()
    got = c.out.double().view(c.n, c.t, c.h, c.d)
    assert ((got[..., 1:] - want[:, None, None]).abs() <= tol[:, None, None] * (1 + 2.0 ** -10)).all(), ((got[..., 1:] / want[:, None, None] - 1).abs().max().item())
    near = 64 * 2.0 ** 20
    assert ((got[..., 0] - near).abs() <= near * (2.0 ** -8 + 2.0 ** -12)).all()


@way_of_call
def test_weights_of_zeros_far_below(way):
    """One key above all others, whose weights are 2^-20 of its own; every other block of 16 rows holds zeros beside value scales
    of 2^64.  Their keys' weights still count, in lse and in what is divided by the sum."""
    torch = _torch()
    c, n = _full(way, "bf16", "i8", 16)
    c.k.zero_(), c.ks.fill_(1.0), c.q.fill_(0.5)
    c.k[:, 19] = 4
    c.scale = 20 * math.log(2) / (0.5 * 4 * c.d)
    c.v.fill_(64)
    c.v[:, torch.arange(c.max_seq, device="cuda") % 32 < 16] = 0
    c.vs[:, :, 0::2], c.vs[:, :, 1::2] = 2.0 ** -100, 2.0 ** 64
    c.call()
    capi.device_sync()
    n, top = n.double(), 2.0 ** 20
    lse = torch.log(top + n - 1)
    big = (n // 32 * 16 + (n % 32 - 16).clamp(min=0))
    want = 64 * 2.0 ** 64 * (top + big - 1) / (top + n - 1)
    # a score of 20 bits, whose factors round by 2^-24 twice, with the scale's exponent 84: 2^-24 of all that; sums of n terms.
    # What n / 2 lost weights would change is more
    rel = 128 * 2.0 ** -24 + (c.max_seq / 16 + 40) * 2.0 ** -23
    assert rel < (n / 4 / top).min()
    assert ((c.lse.double() - lse).abs() <= rel + 2.0 ** -22 * lse).all()
    assert ((c.out.double() - want[:, None]).abs() <= (want * (2.0 ** -8 + rel))[:, None]).all()
