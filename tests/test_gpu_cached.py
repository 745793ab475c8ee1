"""The cached-attention calls (swapnet_attention_tree, swapnet_attention_weights,
swapnet_cache_evict, swapnet_tree_accept) against plain float64 restatements of
their definitions, at the sizes, masks and contents where they can go wrong.

Tolerances, derived before any run.  A score is a sum of D products, each exact
in fp32, accumulated in fp32: off by at most D 2^-23 sum|q_i k_i| (the tensor
cores' sums are allowed a whole step each), which is p's relative error; p goes
to the product with V in two parts (bf16: 2^-18 of p left; fp16: 2^-22, or
2^-25 where p is below the normal range); 2^x is off by 2^-22, the sums over n
keys by (n / 16 + 40) 2^-23 of sum p |v|.  The quotient doubles what p carries,
and the result is rounded once, by half a step of its type."""
import numpy as np
import pytest

from paper_2401_16757_gb300 import capi

pytestmark = pytest.mark.gpu

SENT = 7.0  # what outputs hold before a call


def _torch():
    import torch
    return torch


def _dt(dtype):
    torch = _torch()
    return {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def _tree(rng, n, t):
    par = np.full((n, t), -1, dtype=np.int32)
    for b in range(n):
        for i in range(1, t):
            par[b, i] = rng.integers(max(-1, i - 9), i)
    return par


def _ancestors(par, count):
    see = np.zeros((count, count), dtype=bool)
    for i in range(count):
        j = i
        while j >= 0:
            see[i, j] = True
            j = par[j] if par is not None else j - 1
    return see


class Case:
    """Inputs of one attention call, their float64 results and bounds."""

    def __init__(self, dtype, n_seq, tokens, heads, kv_heads, dim, max_seq, lens, counts=None, draft=True, chain=False,
                 weigh=False, seed=0, scale=0.0, poison=True, pad=0):
        torch = _torch()
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.shape = (n_seq, tokens, heads, kv_heads, dim, max_seq)
        self.dtype, self.draft, self.weigh, self.scale = dtype, draft, weigh, scale
        dt = _dt(dtype)
        self.lens = np.asarray(lens, dtype=np.int32)
        self.counts = None if counts is None else np.asarray(counts, dtype=np.int32)

        def normal(*shape, std=1.0):
            return (torch.randn(*shape, generator=g, dtype=torch.float32) * std).to(dt)

        # `pad` elements behind every row: strides that are not the widths
        self.q = normal(n_seq * tokens, heads * dim + pad, std=1.5)
        self.k, self.v = normal(n_seq, max_seq, kv_heads * dim + pad), normal(n_seq, max_seq, kv_heads * dim + pad)
        self.kn = self.vn = self.par = None
        if draft:
            self.kn, self.vn = (normal(n_seq * tokens, kv_heads * dim + pad) for _ in range(2))
            self.par = None if chain else _tree(rng, n_seq, tokens)
        self.win = torch.rand(n_seq, kv_heads, max_seq, generator=g) * 3 if weigh else None
        if poison:  # hidden rows hold anything
            bad = torch.tensor([float("nan"), float("inf"), -float("inf")], dtype=dt)
            for b in range(n_seq):
                for x in (self.k, self.v):
                    x[b, self.lens[b]:] = bad[rng.integers(0, 3)]
                if draft and self.counts is not None:
                    c = int(self.counts[b])
                    for x in (self.kn, self.vn):
                        x.view(n_seq, tokens, -1)[b, c:] = float("nan")
        self.pad = pad

    def count(self, b):
        return self.shape[1] if self.counts is None else int(self.counts[b])

    def run(self, lse=True, stream=None, workspace=None):
        torch = _torch()
        n, t, h, kv, d, cap = self.shape
        dev = {x: (None if getattr(self, x) is None else getattr(self, x).cuda()) for x in ("q", "k", "v", "kn", "vn", "win")}
        ints = {x: (None if getattr(self, x) is None else torch.from_numpy(getattr(self, x)).cuda())
                for x in ("lens", "counts", "par")}
        self.out = torch.full((n * t, h * d + self.pad), SENT, dtype=_dt(self.dtype), device="cuda")
        self.lse = torch.full((n, h, t), SENT, device="cuda") if lse else None
        self.w = torch.full((n, kv, cap), SENT, device="cuda") if self.weigh else None
        p = lambda x: 0 if x is None else x.data_ptr()  # noqa: E731
        wide, kvw = h * d + self.pad, kv * d + self.pad
        args = capi.cached_attention(
            self.dtype, n, t, h, kv, d, cap, q=p(dev["q"]), k=p(dev["k"]), v=p(dev["v"]), lens=p(ints["lens"]),
            counts=p(ints["counts"]), parents=p(ints["par"]), k_new=p(dev["kn"]), v_new=p(dev["vn"]), out=p(self.out),
            lse=p(self.lse), weights_in=p(dev["win"]), weights=p(self.w), scale=self.scale, q_stride=wide, kv_stride=kvw,
            new_stride=kvw, out_stride=wide)
        need = capi.attention_tree_workspace(args)
        ws = torch.full((max(need, 256) // 4,), float("nan"), device="cuda")  # nothing is expected in it
        s = stream or torch.cuda.current_stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            capi.attention_tree(args, ws.data_ptr(), need, s.cuda_stream)
        self.keep = (dev, ints, ws, args)
        torch.cuda.synchronize()
        return self

    def reference(self, b, rows=None):
        """(seen, scores, p, values, |q||k| sums, lse) of sequence b in float64; keys: cached rows, then drafted nodes."""
        torch = _torch()
        n, t, h, kv, d, _ = self.shape
        m, c = int(self.lens[b]), self.count(b)
        k, v = self.k[b, :m, :kv * d].double(), self.v[b, :m, :kv * d].double()
        if self.draft:
            k = torch.cat([k, self.kn.view(n, t, -1)[b, :c, :kv * d].double()])
            v = torch.cat([v, self.vn.view(n, t, -1)[b, :c, :kv * d].double()])
            seen = np.ones((c, m + c), dtype=bool)
            seen[:, m:] = _ancestors(None if self.par is None else self.par[b], c)
        else:
            seen = np.arange(m)[None, :] <= (m - c + np.arange(c))[:, None]
        at = np.arange(c) if rows is None else rows
        q = self.q.view(n, t, -1)[b, at, :h * d].double().view(c, h, d)
        k, v = k.view(-1, kv, d), v.view(-1, kv, d)
        own = torch.arange(h) // (h // kv)
        sc = self.scale or d ** -0.5
        z = torch.einsum("ihd,jhd->hij", q, k[:, own]) * sc
        zabs = torch.einsum("ihd,jhd->hij", q.abs(), torch.nan_to_num(k[:, own].abs(), 0, 0, 0)) * sc
        see = torch.from_numpy(seen)
        z = torch.where(see, z, torch.tensor(-float("inf"), dtype=torch.float64))
        zabs = torch.where(see, zabs, torch.zeros((), dtype=torch.float64))
        return see, z, zabs, v, own

    def check(self):
        torch = _torch()
        n, t, h, kv, d, cap = self.shape
        out = self.out.cpu().double()[:, :h * d].view(n, t, h, d)
        if self.pad:
            assert torch.all(self.out[:, h * d:] == SENT)
        lse = None if self.lse is None else self.lse.cpu().double()
        half = torch.finfo(_dt(self.dtype)).eps / 2
        for b in range(n):
            c, m = self.count(b), int(self.lens[b])
            assert torch.all(out[b, c:] == SENT) and (lse is None or torch.all(lse[b, :, c:] == SENT))
            if c == 0:
                continue
            see, z, zabs, v, own = self.reference(b)
            keys = z.shape[-1]
            if keys == 0:
                assert torch.all(out[b, :c] == 0) and (lse is None or torch.all(lse[b, :, :c] == -float("inf")))
                continue
            ref_lse = torch.logsumexp(z, -1)
            empty = ~see.any(-1)
            p = torch.exp(z - torch.where(torch.isinf(ref_lse), torch.zeros_like(ref_lse), ref_lse)[..., None])
            vz = torch.nan_to_num(v[:, own], 0, 0, 0)
            ref = torch.einsum("hij,jhd->ihd", p, vz)
            mass = torch.einsum("hij,jhd->ihd", p, vz.abs())
            es = (d * 2.0 ** -23 * zabs.amax(-1) + 2.0 ** -21 * (1 + z.masked_fill(~see, 0).abs().amax(-1))).T  # [i, h]
            sums = (keys / 16 + 40) * 2.0 ** -23
            parts = 2.0 ** -18
            tiny = keys * 2.0 ** -25 * vz.abs().amax(0)[None] if self.dtype == "f16" else 0.0
            tol = half * ref.abs() + (2 * es[..., None] + parts + 2 * sums) * mass + tiny + 1e-30
            if self.dtype == "f16":
                tol = tol + 2.0 ** -25  # the least step of the type, halved
            err = (out[b, :c] - ref).abs()
            assert torch.all(err <= tol), (b, float((err / tol).max()), float(err.max()))
            if lse is not None:
                e = (lse[b, :, :c] - ref_lse).abs()
                lt = es.T + sums + 2.0 ** -22 * ref_lse.abs()
                ok = torch.where(empty[None], lse[b, :, :c] == -float("inf"), e <= lt)
                assert torch.all(ok), (b, float(torch.nan_to_num(e / lt, 0).max()))
            assert torch.all(out[b, :c][empty] == 0)
            if self.weigh:
                self.check_weights(self.w.cpu().double()[b], b, p, es, m, sums)
        return self

    def check_weights(self, w, b, p, es, m, sums):
        torch = _torch()
        n, t, h, kv, d, cap = self.shape
        add = p.view(kv, h // kv, -1, p.shape[-1]).sum(dim=(1, 2))[:, :m]
        slack = (p * (2 * es.T[..., None] + 2 * sums)).view(kv, h // kv, -1, p.shape[-1]).sum(dim=(1, 2))[:, :m]
        ref = self.win[b, :, :m].double() + add
        tol = slack + ref.abs() * (p.shape[1] * h // kv + 4) * 2.0 ** -24
        err = (w[:, :m] - ref).abs()
        assert torch.all(err <= tol), float((err / tol).max())
        assert torch.all(w[:, m:] == SENT)


LAYOUTS = [(8, 8, 128), (8, 2, 64), (6, 2, 128), (12, 1, 64), (5, 5, 64)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv,dim", LAYOUTS)
@pytest.mark.parametrize("tokens", [1, 2, 5, 16, 17, 33, 64, 127, 128])
def test_tree(dtype, heads, kv, dim, tokens):
    """Drafted trees of every size on ragged caches, among them empty ones, ends inside and on every tile border."""
    lens = [0, 1, 15, 16, 17, 127, 128, 129, 300]
    counts = [max(0, tokens - i % 4) if i else tokens for i in range(len(lens))]
    Case(dtype, len(lens), tokens, heads, kv, dim, 301, lens, counts, seed=tokens).run().check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,counts", [(1, None), (3, None), (16, [16, 3, 0, 1, 16]), (40, [40, 39, 1, 17, 33])])
def test_drafted_chain_and_scale(dtype, tokens, counts):
    Case(dtype, 5, tokens, 4, 2, 128, 700, [700, 3, 650, 0, 64], counts, chain=True, scale=0.3, seed=3).run().check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv,dim", LAYOUTS)
@pytest.mark.parametrize("tokens", [1, 2, 7, 30, 100, 200])
@pytest.mark.parametrize("weigh", [False, True])
def test_last_rows_of_the_cache(dtype, heads, kv, dim, tokens, weigh):
    """Causal runs and single tokens, with and without the cached rows' weights; rows that see nothing give zeros."""
    lens = [tokens, max(tokens - 1, 0), 0, tokens + 1, 128 + tokens, 311]
    Case(dtype, len(lens), tokens, heads, kv, dim, 333, lens, draft=False, weigh=weigh, seed=tokens + 50).run().check()


@pytest.mark.parametrize("tokens", [1, 20])
def test_long_cache_is_split(tokens):
    """One sequence on many SMs: the splits' join, and a cache that is nearly empty in the same plan."""
    Case("bf16", 2, tokens, 8, 2, 128, 9000, [8999, 7], seed=9).run().check()
    Case("f16", 2, tokens, 8, 2, 128, 9000, [8999, 30], draft=False, weigh=True, seed=9).run().check()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens", [12, 20])
def test_many_sequences_with_many_tiles_each(dim, tokens):
    """Enough sequences that each CTA passes dozens of key tiles, of caches that DRAM has to deliver."""
    torch = _torch()
    rng = np.random.default_rng(1)
    n, cap = 40, 4224
    lens = rng.integers(3900, cap + 1, size=n)
    eng = _any_engine()
    for draft in (True, False):
        c = Case("bf16", n, tokens, 32, 8, dim, cap, lens, draft=draft, weigh=not draft, seed=5, poison=False).run()
        eng.sync()  # no wait gave up
        full, t = c.lens.copy(), tokens
        for b in (0, 17, n - 1):
            one = Case.__new__(Case)
            one.__dict__.update(c.__dict__)
            one.shape = (1,) + c.shape[1:]
            one.lens = full[b:b + 1]
            for x in ("k", "v", "win"):
                setattr(one, x, None if getattr(c, x) is None else getattr(c, x)[b:b + 1])
            for x in ("q", "kn", "vn", "out"):
                setattr(one, x, None if getattr(c, x) is None else getattr(c, x)[b * t:(b + 1) * t])
            one.par = None if c.par is None else c.par[b:b + 1]
            one.lse = c.lse[b:b + 1]
            one.w = None if c.w is None else c.w[b:b + 1]
            one.check()
    torch.cuda.synchronize()


@pytest.mark.parametrize("draft", [False, True])
def test_strides_and_streams(draft):
    torch = _torch()
    s = torch.cuda.Stream()
    Case("bf16", 3, 9, 6, 3, 128, 200, [200, 64, 150], draft=draft, weigh=not draft, pad=24, seed=4).run(stream=s).check()
    Case("f16", 3, 70, 8, 8, 64, 200, [200, 80, 150], draft=draft, weigh=not draft, pad=8, seed=5).run(stream=s).check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens", [6, 40, 100])
def test_hidden_rows_that_are_not_numbers(dtype, tokens):
    """A drafted node whose key or value is not finite reaches only those who see it."""
    torch = _torch()
    c = Case(dtype, 1, tokens, 4, 2, 64, 150, [133], seed=12)
    clean = Case(dtype, 1, tokens, 4, 2, 64, 150, [133], seed=12)
    bad = tokens // 2
    c.vn[bad, 3] = float("nan")
    c.vn[bad, 70] = float("inf")
    c.kn[bad + 1, 5] = float("nan")
    c.run()
    clean.run()
    see = _ancestors(c.par[0], tokens)
    touched = see[:, bad] | see[:, bad + 1]
    assert 0 < touched.sum() < tokens
    a, b = c.out.cpu(), clean.out.cpu()
    assert torch.equal(a[~touched], b[~touched])
    assert torch.equal(c.lse.cpu()[..., ~touched], clean.lse.cpu()[..., ~touched])
    v = see[:, bad] & ~see[:, bad + 1]
    x = a[v].view(int(v.sum()), 4, 64)
    assert v.any() and torch.all(torch.isnan(x[:, :2, 3])) and torch.all(torch.isinf(x[:, 2:, 6]))
    rest = x.clone()
    rest[:, :2, 3] = 0
    rest[:, 2:, 6] = 0
    assert torch.all(torch.isfinite(rest))
    assert torch.all(torch.isnan(a[see[:, bad + 1]].view(-1, 4, 64)[:, :2]))


def test_later_rows_that_are_not_numbers():
    """Causal runs: a later row's infinite value does not reach the rows before it."""
    torch = _torch()
    for tokens in (10, 90):
        c = Case("bf16", 1, tokens, 4, 4, 128, 200, [180], draft=False, seed=2)
        clean = Case("bf16", 1, tokens, 4, 4, 128, 200, [180], draft=False, seed=2)
        c.v[0, 180 - tokens // 2] = float("inf")
        c.run()
        clean.run()
        before = tokens - tokens // 2
        assert torch.equal(c.out[:before], clean.out[:before])
        assert not torch.any(torch.isfinite(c.out[before:]))


@pytest.mark.parametrize("draft,tokens,cap", [(False, 300, 700), (False, 300, 5000), (False, 12, 700), (True, 128, 700), (True, 100, 5000)])
def test_values_that_are_not_numbers_in_many_tiles(draft, tokens, cap):
    """Several such rows, in both halves of neighbouring key tiles: the elements and the queries that none of them reaches keep
    their bits or their value, the others are not finite, on every one of many runs."""
    torch = _torch()
    n, h, kv, d = 3, 8, 2, 128
    g = torch.Generator().manual_seed(tokens)
    lens = [cap - 1, cap // 2, tokens + 3]
    k, v = (torch.randn(n, cap, kv * d, generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn(n * tokens, h * d, generator=g).bfloat16().cuda()
    kn, vn = (torch.randn(n * tokens, kv * d, generator=g).bfloat16().cuda() for _ in range(2))
    par = np.tile(np.arange(-1, tokens - 1, dtype=np.int32), (n, 1))  # a chain, so that what is seen is a range
    par, dl = torch.from_numpy(par).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    x = (kn, vn, par) if draft else (None, None, None)
    clean = _attend(q, k.data_ptr(), v.data_ptr(), *x, dl, n, tokens, h, kv, d, cap)
    bad = sorted({min(tokens - 1, i) for i in (3, 5, 60, 70, 71, 99, 127, 130, 200, 290)})
    for b in range(n):
        for i, at in enumerate(bad):
            (vn[b * tokens + at] if draft else v[b, lens[b] - tokens + at])[7 + 128 * (i % 2)] = float("nan") if i % 3 else float("inf")
    first = [min((at for i, at in enumerate(bad) if i % 2 == s), default=tokens) for s in range(2)]
    want = clean[0].view(n, tokens, kv, h // kv, d)
    got = None
    for _ in range(20):
        run = _attend(q, k.data_ptr(), v.data_ptr(), *x, dl, n, tokens, h, kv, d, cap)
        assert got is None or all(torch.equal(torch.nan_to_num(a, 77.0), torch.nan_to_num(b, 77.0)) for a, b in zip(run, got))
        got = run
    out = got[0].view(n, tokens, kv, h // kv, d)
    assert torch.equal(got[1], clean[1])  # scores have nothing to do with it
    assert torch.equal(out[:, :bad[0]], want[:, :bad[0]])
    for s in range(2):
        assert not torch.any(torch.isfinite(out[:, first[s]:, s, :, 7])) and torch.all(torch.isfinite(out[:, :first[s], s]))
    keep = torch.ones(d, dtype=torch.bool, device="cuda")
    keep[7] = False
    # a row added by hand in fp32 in place of two products: a rounding of the result to either side, and 2^-13 of values of up to 4
    a, b = out[..., keep].double(), want[..., keep].double()
    assert torch.all((a - b).abs() <= 2.0 ** -7 * b.abs() + 2.0 ** -11)


def test_sequences_out_of_range_are_left_alone():
    """Bad lengths, counts and parents: that sequence's outputs stay, the others are right, and the next sync reports it."""
    torch = _torch()
    eng = _any_engine()
    for what in ("len", "negative", "count", "parent", "self"):
        c = Case("bf16", 3, 8, 4, 2, 128, 100, [40, 50, 60], [8, 8, 8], seed=6, poison=False)
        if what == "len":
            c.lens[1] = 101
        elif what == "negative":
            c.lens[1] = -1
        elif what == "count":
            c.counts[1] = 9
        elif what == "parent":
            c.par[1, 3] = -2
        else:
            c.par[1, 3] = 3
        c.run()
        out, lse = c.out.clone().view(3, 8, -1), c.lse.clone()
        assert torch.all(out[1] == SENT) and torch.all(lse[1] == SENT)
        with pytest.raises(capi.SwapnetError) as e:
            eng.sync()
        assert e.value.code == capi.ERR_INVALID_ARG
        eng.sync()
        c.lens[1], c.counts[1] = 50, 8
        c.par[1, 3] = 0
        c.run().check()
        got = c.out.view(3, 8, -1)
        assert torch.equal(got[0], out[0]) and torch.equal(got[2], out[2])
    eng.sync()


def _any_engine():
    import synth
    m = dict(name="yolov3", model_id=61, dtype="f16", input=(1, 1, 1, 64),
             layers=[dict(op="linear", src=[-1], k=64, n=64, act="relu", res=None, res_post=False)], outputs=[0])
    return capi.Engine(capi.Plan.resident(capi.Desc(m)), capi.HostWeights(synth.gen.model_weights(m)))


def test_same_bits_every_time_and_in_a_graph():
    torch = _torch()
    for kw in (dict(tokens=4, draft=True), dict(tokens=1, draft=False, weigh=True), dict(tokens=60, draft=True),
               dict(tokens=60, draft=False, weigh=True)):
        t = kw.pop("tokens")
        c = Case("bf16", 4, t, 8, 2, 128, 2000, [2000, 333, 1900, 64], seed=8, **kw).run().check()
        first = [x.clone() for x in (c.out, c.lse, c.w) if x is not None]
        dev, ints, ws, args = c.keep
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            capi.attention_tree(args, ws.data_ptr(), ws.numel() * 4, torch.cuda.current_stream().cuda_stream)
        for x in (c.out, c.lse, c.w):
            if x is not None:
                x.fill_(SENT)
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(first, [x for x in (c.out, c.lse, c.w) if x is not None]):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv,dim", LAYOUTS)
@pytest.mark.parametrize("tokens", [1, 3, 16, 40, 150])
@pytest.mark.parametrize("pick", [False, True])
def test_weights_from_lse(dtype, heads, kv, dim, tokens, pick):
    """The weights call on its own: all queries, or a list of them in any order."""
    torch = _torch()
    rng = np.random.default_rng(tokens)
    lens = [tokens, tokens + 1, 129 + tokens, 333, max(0, tokens - 1)]
    counts = [min(tokens, x) for x in (tokens, 1, max(1, tokens // 2), 0, 2)]
    if not pick:
        counts = [tokens] * 5
    c = Case(dtype, 5, tokens, heads, kv, dim, 340, lens, counts, draft=False, weigh=True, seed=tokens + 7)
    rows = np.stack([rng.permutation(tokens) for _ in range(5)]).astype(np.int32) if pick else None
    n, t, h, kvh, d, cap = c.shape
    lse = torch.full((n, h, t), float("nan"))
    refs = []
    for b in range(n):
        x = c.count(b)
        see, z, zabs, v, own = c.reference(b, None if rows is None else rows[b, :x])
        l = torch.logsumexp(z, -1).float() if x and z.shape[-1] else torch.full((h, x), -float("inf"))
        lse[b][:, np.arange(x) if rows is None else rows[b, :x]] = l
        refs.append((see, z, zabs, l))
    dev = [x.cuda() for x in (c.q, c.k, lse, c.win)]
    ints = [torch.from_numpy(c.lens).cuda(), torch.from_numpy(c.counts).cuda(),
            None if rows is None else torch.from_numpy(np.ascontiguousarray(rows)).cuda()]
    w = torch.full((n, kvh, cap), SENT, device="cuda")
    args = capi.cached_attention(dtype, n, t, h, kvh, d, cap, q=dev[0].data_ptr(), k=dev[1].data_ptr(),
                                 lens=ints[0].data_ptr(), counts=ints[1].data_ptr(),
                                 rows=0 if rows is None else ints[2].data_ptr(), lse=dev[2].data_ptr(),
                                 weights_in=dev[3].data_ptr(), weights=w.data_ptr())
    capi.attention_weights(args, torch.cuda.current_stream().cuda_stream)
    got = w.cpu().double()
    for b, (see, z, zabs, l) in enumerate(refs):
        m = int(c.lens[b])
        if z.shape[-1] == 0 or z.shape[1] == 0:
            assert torch.equal(got[b, :, :m], c.win[b, :, :m].double()) and torch.all(got[b, :, m:] == SENT)
            continue
        p = torch.where(see, torch.exp(z - l.double()[..., None]), torch.zeros((), dtype=torch.float64))
        # lse itself was rounded to 32 bits: half a step of it
        es = (d * 2.0 ** -23 * zabs.amax(-1) + 2.0 ** -21 * (1 + z.masked_fill(~see, 0).abs().amax(-1))).T
        c.check_weights(got[b], b, p, es, m, 2.0 ** -22)
    # in place
    args.weights = args.weights_in
    capi.attention_weights(args, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for b in range(n):
        m = int(c.lens[b])
        assert torch.equal(dev[3][b, :, :m], w[b, :, :m]) and torch.equal(dev[3][b, :, m:].cpu(), c.win[b, :, m:])


def test_a_query_listed_twice_counts_twice():
    torch = _torch()
    c = Case("f16", 1, 6, 4, 2, 64, 90, [70], draft=False, seed=21)
    rows = torch.tensor([[3, 3, 0, 3]], dtype=torch.int32)
    z = [torch.einsum("hd,jhd->hj", c.q[r].double().view(4, 64), c.k[0, :67 + i].double().view(-1, 2, 64).repeat_interleave(2, 1)) / 8
         for i, r in enumerate(rows[0].tolist())]
    lse = torch.randn(1, 4, 6)
    lse[0, :, 3], lse[0, :, 0] = z[3].logsumexp(-1).float(), z[2].logsumexp(-1).float()
    want = torch.zeros(2, 70, dtype=torch.float64)
    for i, r in enumerate(rows[0].tolist()):
        want[:, :67 + i] += torch.exp(z[i] - lse[0, :, r, None].double()).view(2, 2, -1).sum(1)
    dev = [x.cuda() for x in (c.q, c.k, lse, rows, torch.tensor([70], dtype=torch.int32), torch.tensor([4], dtype=torch.int32))]
    listed = torch.zeros(1, 6, dtype=torch.int32, device="cuda")
    listed[:, :4] = dev[3]
    w = torch.full((1, 2, 90), SENT, device="cuda")
    capi.attention_weights(capi.cached_attention("f16", 1, 6, 4, 2, 64, 90, q=dev[0].data_ptr(), k=dev[1].data_ptr(),
                                                 lens=dev[4].data_ptr(), counts=dev[5].data_ptr(), rows=listed.data_ptr(),
                                                 lse=dev[2].data_ptr(), weights=w.data_ptr()),
                           torch.cuda.current_stream().cuda_stream)
    # scores of at most about 20 in fp32, 64 products each: 64 2^-23 * 40 of the weight
    assert torch.all((w[0, :, :70].cpu().double() - want).abs() <= 4e-4 * want + 1e-9) and torch.all(w[..., 70:] == SENT)


# ------------------------------------------- layouts, numbers and neighbours
def _attend(q, k, v, kn, vn, par, lens, n, t, h, kv, d, cap, kv_stride=0, seq_stride=0, weigh=False):
    """out, lse and weights of a call on device tensors (k, v: addresses)."""
    torch = _torch()
    out, lse = torch.full_like(q, SENT), torch.full((n, h, t), SENT, device="cuda")
    w = torch.full((n, kv, cap), SENT, device="cuda") if weigh else None
    p = lambda x: 0 if x is None else x.data_ptr()  # noqa: E731
    a = capi.cached_attention("bf16", n, t, h, kv, d, cap, q=p(q), k=k, v=v, lens=p(lens), k_new=p(kn), v_new=p(vn), parents=p(par),
                              out=p(out), lse=p(lse), weights=p(w), kv_stride=kv_stride, seq_stride=seq_stride)
    ws = torch.empty(max(256, capi.attention_tree_workspace(a)), dtype=torch.uint8, device="cuda")
    capi.attention_tree(a, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    return [x for x in (out, lse, w) if x is not None]


def test_offsets_past_32_bits_and_interleaved_sequences():
    """Rows millions of elements apart, the sequences' rows side by side: the same bits as on packed caches, in every call."""
    torch = _torch()
    n, h, kv, d, cap, stride = 2, 8, 2, 128, 200, 12_000_000
    width = kv * d
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(n, cap, width, generator=g).bfloat16().cuda() for _ in range(2))
    lens = torch.tensor([200, 190], dtype=torch.int32, device="cuda")
    big = torch.zeros(cap, stride, dtype=torch.bfloat16, device="cuda")
    assert (cap - 1) * stride > 2 ** 31
    wide = big[:, :4 * width].view(cap, n, 2, width)  # row, sequence, keys and values

    def fill():
        wide[:, :, 0], wide[:, :, 1] = k.transpose(0, 1), v.transpose(0, 1)

    fill()
    at = dict(k=big.data_ptr(), v=big.data_ptr() + 2 * width, kv_stride=stride, seq_stride=2 * width)
    for t in (1, 3, 30):
        q = torch.randn(n * t, h * d, generator=g).bfloat16().cuda()
        kn, vn = (torch.randn(n * t, width, generator=g).bfloat16().cuda() for _ in range(2))
        par = torch.from_numpy(_tree(np.random.default_rng(t), n, t)).cuda()
        for draft in (False, True):
            x = (kn, vn, par) if draft else (None, None, None)
            a = _attend(q, k.data_ptr(), v.data_ptr(), *x, lens, n, t, h, kv, d, cap, weigh=not draft)
            b = _attend(q, at["k"], at["v"], *x, lens, n, t, h, kv, d, cap, stride, 2 * width, weigh=not draft)
            assert all(torch.equal(y, z) for y, z in zip(a, b)), (t, draft)
            ws = []
            for kk, st, sq in ((k.data_ptr(), 0, 0), (at["k"], stride, 2 * width)):
                w = torch.full((n, kv, cap), SENT, device="cuda")
                capi.attention_weights(capi.cached_attention("bf16", n, t, h, kv, d, cap, q=q.data_ptr(), k=kk, lens=lens.data_ptr(),
                                                             lse=a[1].data_ptr(), weights=w.data_ptr(), kv_stride=st, seq_stride=sq),
                                       torch.cuda.current_stream().cuda_stream)
                ws.append(w)
            assert torch.equal(*ws)
    # acceptance appends at rows behind 2^31 elements
    t = 8
    draft = torch.randn(n * t, width, generator=g).bfloat16().cuda()
    ids = torch.zeros(n, t, dtype=torch.int32, device="cuda")
    path = torch.empty_like(ids)
    acc, nxt, lo = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(3))
    few = torch.tensor([185, 181], dtype=torch.int32, device="cuda")
    capi.tree_accept("bf16", n, t, width, cap, ids=ids.data_ptr(), targets=torch.zeros_like(ids).data_ptr(), lens=few.data_ptr(),
                     caches=[at["k"], at["v"]], drafts=[draft.data_ptr()] * 2, path=path.data_ptr(), accepted=acc.data_ptr(),
                     next=nxt.data_ptr(), lens_out=lo.data_ptr(), cache_stride=stride, seq_stride=2 * width,
                     stream=torch.cuda.current_stream().cuda_stream)
    assert lo.tolist() == [193, 189]
    for b, m in enumerate(few.tolist()):
        for i, old in enumerate((k, v)):
            want = old[b].clone()
            want[m:m + t] = draft.view(n, t, width)[b]
            assert torch.equal(wide[:, b, i], want)
    # eviction, to another cache and in place
    w = torch.rand(n, kv, cap, generator=g).cuda()
    kept, lo = torch.zeros(n, kv, 150, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    ref = [torch.zeros(n, cap, width, dtype=torch.bfloat16, device="cuda") for _ in range(2)] + [torch.zeros_like(w)]
    fill()
    common = dict(lens=lens.data_ptr(), kept=kept.data_ptr(), lens_out=lo.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
    capi.cache_evict("bf16", n, kv, d, cap, 150, 9, 2, k=k.data_ptr(), v=v.data_ptr(), weights=w.data_ptr(), k_out=ref[0].data_ptr(),
                     v_out=ref[1].data_ptr(), weights_out=ref[2].data_ptr(), **common)
    got = [torch.zeros_like(x) for x in ref]
    src = dict(k=at["k"], v=at["v"], kv_stride=stride, seq_stride=2 * width)
    capi.cache_evict("bf16", n, kv, d, cap, 150, 9, 2, weights=w.data_ptr(), k_out=got[0].data_ptr(), v_out=got[1].data_ptr(),
                     weights_out=got[2].data_ptr(), **src, **common)
    assert all(torch.equal(x, y) for x, y in zip(ref, got)) and kept.max() > 180
    capi.cache_evict("bf16", n, kv, d, cap, 150, 9, 2, weights=w.data_ptr(), k_out=at["k"], v_out=at["v"], out_stride=stride,
                     out_seq_stride=2 * width, weights_out=w.data_ptr(), **src, **common)
    for b in range(n):
        for i in range(2):
            assert torch.equal(wide[:150, b, i], ref[i][b, :150])
    for b, m in enumerate(lens.tolist()):  # (weights behind the sequence's end stay as they were)
        assert torch.equal(w[b, :, :m], ref[2][b, :, :m])
    assert torch.all(big[:, 4 * width:4 * width + 64] == 0)


@pytest.mark.parametrize("heads,kv,tokens", [(160, 160, 20), (160, 160, 2), (256, 2, 1), (100, 1, 3)])
def test_more_heads_than_sms_and_wide_groups(heads, kv, tokens):
    Case("bf16", 2, tokens, heads, kv, 64, 300, [300, 5 + tokens], draft=True, seed=31).run().check()
    Case("f16", 2, tokens, heads, kv, 64, 300, [300, 5 + tokens], draft=False, weigh=True, seed=32).run().check()


@pytest.mark.parametrize("draft", [False, True])
def test_runs_over_many_idle_sequences(draft):
    """A run of key tiles that passes more than a hundred sequences without a query, and ends in others of a tile each."""
    n = 200
    lens = [130] * n
    lens[0], lens[-1] = 4000, 2500
    counts = [20] * n
    for b in range(1, 140):
        counts[b], lens[b] = 0, b
    Case("bf16", n, 20, 1, 1, 64, 4096, lens, counts, draft=draft, weigh=not draft, seed=33, poison=False).run().check()


@pytest.mark.parametrize("tokens", [2, 20])
def test_replays_follow_the_lengths_and_calls_run_side_by_side(tokens):
    """A captured call reads the lengths of the moment; calls on two streams at once, with workspaces of their own, give the
    bits that they give alone."""
    torch = _torch()
    n, h, kv, d, cap = 3, 8, 2, 128, 3000
    g = torch.Generator().manual_seed(8)
    k, v = (torch.randn(n, cap, kv * d, generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn(n * tokens, h * d, generator=g).bfloat16().cuda()
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([3000, 20, 777], [64, 2999, 25], [0, 3000, 3000])]
    alone = [_attend(q, k.data_ptr(), v.data_ptr(), None, None, None, x, n, tokens, h, kv, d, cap, weigh=True) for x in lens]
    now = lens[0].clone()
    s = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _attend(q, k.data_ptr(), v.data_ptr(), None, None, None, now, n, tokens, h, kv, d, cap, weigh=True)
    for x, want in zip(lens, alone):
        now.copy_(x)
        for y in got:
            y.fill_(SENT)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, z) for y, z in zip(got, want))
    res = [[], []]
    for _ in range(8):
        for i in range(2):
            with torch.cuda.stream(s[i]):
                res[i].append(_attend(q, k.data_ptr(), v.data_ptr(), None, None, None, lens[i], n, tokens, h, kv, d, cap, weigh=True))
    torch.cuda.synchronize()
    for i in range(2):
        for r in res[i]:
            assert all(torch.equal(y, z) for y, z in zip(r, alone[i]))


# ------------------------------------------------------------------ eviction
def _keep_rows(w, m, keep, recent, sink):
    if m <= keep:
        return np.arange(m)
    key = np.where(np.isnan(w[:m]), np.inf, w[:m].astype(np.float64) + 0.0)
    key[np.isnan(w[:m])] = np.finfo(np.float64).max  # above every fp32, below the protected rows
    inf = np.isposinf(w[:m])
    key[inf] = 1e300
    key[:sink] = np.inf
    if recent:
        key[m - recent:] = np.inf
    return np.sort(np.argsort(-key, kind="stable")[:keep])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("kv,dim", [(1, 128), (3, 64), (8, 128), (2, 24), (2, 200)])
@pytest.mark.parametrize("keep,recent,sink", [(1, 0, 0), (7, 3, 4), (64, 10, 1), (100, 99, 0), (4097, 500, 4)])
@pytest.mark.parametrize("in_place", [False, True])
def test_eviction(dtype, kv, dim, keep, recent, sink, in_place):
    torch = _torch()
    cap = max(300, keep + 4500 if keep > 1000 else 0)
    lens = np.array([cap, 0, 1, keep, min(cap, keep + 1), cap - 37], dtype=np.int32)
    n, pad = len(lens), 8
    g = torch.Generator().manual_seed(keep + dim)
    k, v = ((torch.randn(n, cap, kv * dim + pad, generator=g)).to(_dt(dtype)) for _ in range(2))
    w = torch.rand(n, kv, cap, generator=g) ** 4
    w = torch.where(w < 0.05, torch.zeros(()), w)  # many equal ones
    w[0, 0, 5:90:3] = -0.0
    w[0, -1, 11], w[0, -1, 20], w[0, -1, 33] = float("nan"), float("inf"), -1.0
    w[-1, 0, :] = 0.25  # nothing but ties
    dk, dv, dw, dl = k.cuda(), v.cuda(), w.cuda(), torch.from_numpy(lens).cuda()
    ocap = cap if in_place else keep + 3
    if in_place:
        ok, ov, ow = dk, dv, dw
    else:
        ok, ov = (torch.full((n, ocap, kv * dim + pad), SENT, dtype=_dt(dtype), device="cuda") for _ in range(2))
        ow = torch.full((n, kv, ocap), SENT, device="cuda")
    kept = torch.full((n, kv, keep), -5, dtype=torch.int32, device="cuda")
    lo = torch.full((n,), -5, dtype=torch.int32, device="cuda")
    stride = kv * dim + pad
    capi.cache_evict(dtype, n, kv, dim, cap, keep, recent, sink, k=dk.data_ptr(), v=dv.data_ptr(), weights=dw.data_ptr(),
                     lens=dl.data_ptr(), k_out=ok.data_ptr(), v_out=ov.data_ptr(), weights_out=ow.data_ptr(),
                     kept=kept.data_ptr(), lens_out=lo.data_ptr(), out_capacity=ocap, kv_stride=stride, out_stride=stride,
                     stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    before = dict(k=k, v=v, w=w)
    gk, gv, gw = (x.cpu() for x in (ok, ov, ow))
    for b in range(n):
        m = int(lens[b])
        x = min(m, keep)
        assert int(lo[b]) == x
        for h in range(kv):
            rows = _keep_rows(w[b, h].numpy(), m, keep, recent, sink)
            assert np.array_equal(kept[b, h, :x].cpu().numpy(), rows), (b, h)
            assert torch.all(kept[b, h, x:] == -5)
            cols = slice(h * dim, (h + 1) * dim)
            for got, name in ((gk, "k"), (gv, "v")):
                assert torch.equal(got[b, :x, cols], before[name][b, rows, cols])
                rest = got[b, x:, cols]
                assert torch.equal(rest, before[name][b, x:, cols]) if in_place else torch.all(rest == SENT)
            assert torch.equal(torch.nan_to_num(gw[b, h, :x], -9), torch.nan_to_num(w[b, h, rows], -9))
            assert torch.all(gw[b, h, x:min(m, ocap)] == 0)  # where later rows start from
            rest = gw[b, h, min(m, ocap):]
            assert torch.equal(torch.nan_to_num(rest, -9), torch.nan_to_num(w[b, h, min(m, ocap):], -9)) if in_place else torch.all(rest == SENT)
        assert torch.all(gk[b, :, kv * dim:] == SENT) if not in_place else torch.equal(gk[b, :, kv * dim:], k[b, :, kv * dim:])


# ---------------------------------------------------------------- acceptance
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,width,caches,chain", [(1, 64, 1, False), (2, 1024, 3, True), (24, 136, 5, False),
                                                       (128, 4096, 2, False), (128, 64, 256, True), (9, 8, 0, False)])
def test_acceptance(dtype, tokens, width, caches, chain):
    torch = _torch()
    rng = np.random.default_rng(tokens + width)
    n, cap, pad = 6, 200, 8
    par = _tree(rng, n, tokens)
    counts = np.array([tokens, 1, max(1, tokens // 2), tokens, max(1, tokens - 1), tokens], dtype=np.int32)
    lens = np.array([0, 5, 40, cap - tokens, 17, 60], dtype=np.int32)
    targets = rng.integers(0, 5, size=(n, tokens)).astype(np.int32)  # few tokens: many siblings fit
    ids = rng.integers(0, 5, size=(n, tokens)).astype(np.int32)
    if chain:
        ids[0, 1:] = targets[0, :-1]  # the whole chain
    g = torch.Generator().manual_seed(1)
    cs = [(torch.randn(n, cap, width + pad, generator=g)).to(_dt(dtype)) for _ in range(min(caches, 8))]
    cs = [cs[i % 8].clone() for i in range(caches)]
    ds = [(torch.randn(n * tokens, width, generator=g)).to(_dt(dtype)) for _ in range(min(caches, 8))]
    ds = [ds[i % 8] for i in range(caches)]
    dc, dd = [x.cuda() for x in cs], [x.cuda() for x in ds]
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    dev = {k: i32(v) for k, v in dict(ids=ids, targets=targets, par=par, counts=counts, lens=lens).items()}
    path = torch.full((n, tokens), -7, dtype=torch.int32, device="cuda")
    acc, nxt, lo = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(3))
    capi.tree_accept(dtype, n, tokens, width, cap, ids=dev["ids"].data_ptr(), targets=dev["targets"].data_ptr(),
                     parents=0 if chain else dev["par"].data_ptr(), counts=dev["counts"].data_ptr(), lens=dev["lens"].data_ptr(),
                     caches=np.array([x.data_ptr() for x in dc], dtype=np.uint64),
                     drafts=np.array([x.data_ptr() for x in dd], dtype=np.uint64), path=path.data_ptr(),
                     accepted=acc.data_ptr(), next=nxt.data_ptr(), lens_out=lo.data_ptr(), cache_stride=width + pad,
                     stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for b in range(n):
        p = np.arange(-1, tokens - 1) if chain else par[b]
        at, want = 0, [0]
        while True:
            nx = next((i for i in range(1, counts[b]) if p[i] == at and ids[b, i] == targets[b, at]), None)
            if nx is None:
                break
            want.append(nx)
            at = nx
        x, m = len(want), int(lens[b])
        assert int(acc[b]) == x and int(nxt[b]) == targets[b, at] and int(lo[b]) == m + x
        assert path[b].tolist() == want + [-1] * (tokens - x)
        for c in range(caches):
            ref = cs[c][b].clone()
            ref[m:m + x, :width] = ds[c].view(n, tokens, width)[b, want]
            assert torch.equal(dc[c][b].cpu(), ref), (b, c)
    assert not chain or tokens == 1 or int(acc[0]) == tokens


def test_acceptance_without_room_is_left_alone():
    torch = _torch()
    eng = _any_engine()
    lens = torch.tensor([10, 8, -1], dtype=torch.int32, device="cuda")
    ids = torch.tensor([[1, 2], [1, 2], [1, 2]], dtype=torch.int32, device="cuda")
    tgt = torch.tensor([[2, 3], [2, 3], [2, 3]], dtype=torch.int32, device="cuda")
    cache = torch.zeros(3, 10, 64, dtype=torch.bfloat16, device="cuda")
    new = torch.ones(6, 64, dtype=torch.bfloat16, device="cuda")
    path = torch.full((3, 2), -7, dtype=torch.int32, device="cuda")
    acc, nxt, lo = (torch.full((3,), -7, dtype=torch.int32, device="cuda") for _ in range(3))
    capi.tree_accept("bf16", 3, 2, 64, 10, ids=ids.data_ptr(), targets=tgt.data_ptr(), lens=lens.data_ptr(),
                     caches=[cache.data_ptr()], drafts=[new.data_ptr()], path=path.data_ptr(), accepted=acc.data_ptr(),
                     next=nxt.data_ptr(), lens_out=lo.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
    with pytest.raises(capi.SwapnetError) as e:
        eng.sync()
    assert e.value.code == capi.ERR_INVALID_ARG
    assert acc.tolist() == [-7, 2, -7] and lo.tolist() == [-7, 10, -7] and path.tolist() == [[-7, -7], [0, 1], [-7, -7]]
    assert torch.all(cache[0] == 0) and torch.all(cache[2] == 0) and torch.all(cache[1, :8] == 0) and torch.all(cache[1, 8:] == 1)


# ------------------------------------------------------------------ together
def test_a_draft_is_verified_accepted_weighed_and_evicted():
    """The calls as a program chains them, on one stream without waiting: the cache after acceptance gives a next token's
    attention equal to the one over the whole history, and after eviction over the rows kept."""
    torch = _torch()
    torch.manual_seed(0)
    n, t, h, kv, d, cap, vocab = 3, 6, 8, 2, 128, 96, 50
    dt = torch.bfloat16
    lens = torch.tensor([30, 64, 7], dtype=torch.int32, device="cuda")
    k, v = (torch.randn(n, cap, kv * d, device="cuda").to(dt) for _ in range(2))
    kn, vn = (torch.randn(n * t, kv * d, device="cuda").to(dt) for _ in range(2))
    q = torch.randn(n * t, h * d, device="cuda").to(dt)
    par = torch.tensor([[-1, 0, 0, 2, 2, 4]] * n, dtype=torch.int32, device="cuda")
    ids = torch.tensor([[9, 1, 2, 3, 4, 5]] * n, dtype=torch.int32, device="cuda")
    tgt = torch.tensor([[2, 0, 4, 0, 7, 0], [1, 11, 0, 0, 0, 0], [8, 0, 0, 0, 0, 0]], dtype=torch.int32, device="cuda")
    out, lse = torch.zeros(n * t, h * d, dtype=dt, device="cuda"), torch.zeros(n, h, t, device="cuda")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    path, acc, nxt, lens2, lens3 = i32(n, t), i32(n), i32(n), i32(n), i32(n)
    w = torch.zeros(n, kv, cap, device="cuda")
    kept = i32(n, kv, 20)
    s = torch.cuda.current_stream().cuda_stream
    a = capi.cached_attention("bf16", n, t, h, kv, d, cap, q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(),
                              lens=lens.data_ptr(), parents=par.data_ptr(), k_new=kn.data_ptr(), v_new=vn.data_ptr(),
                              out=out.data_ptr(), lse=lse.data_ptr())
    ws = torch.empty(max(256, capi.attention_tree_workspace(a)), dtype=torch.uint8, device="cuda")
    k0, v0 = k.clone(), v.clone()
    capi.attention_tree(a, ws.data_ptr(), ws.numel(), s)
    capi.tree_accept("bf16", n, t, kv * d, cap, ids=ids.data_ptr(), targets=tgt.data_ptr(), parents=par.data_ptr(),
                     lens=lens.data_ptr(), caches=[k.data_ptr(), v.data_ptr()], drafts=[kn.data_ptr(), vn.data_ptr()],
                     path=path.data_ptr(), accepted=acc.data_ptr(), next=nxt.data_ptr(), lens_out=lens2.data_ptr(), stream=s)
    b_ = capi.cached_attention("bf16", n, t, h, kv, d, cap, q=q.data_ptr(), k=k.data_ptr(), lens=lens2.data_ptr(),
                               counts=acc.data_ptr(), rows=path.data_ptr(), lse=lse.data_ptr(), weights=w.data_ptr())
    capi.attention_weights(b_, s)
    k1, v1, w1 = k.clone(), v.clone(), w.clone()
    capi.cache_evict("bf16", n, kv, d, cap, 20, 4, 1, k=k.data_ptr(), v=v.data_ptr(), weights=w.data_ptr(),
                     lens=lens2.data_ptr(), k_out=k.data_ptr(), v_out=v.data_ptr(), weights_out=w.data_ptr(),
                     kept=kept.data_ptr(), lens_out=lens3.data_ptr(), stream=s)
    torch.cuda.synchronize()
    assert acc.tolist() == [3, 2, 1] and nxt.tolist() == [7, 11, 8]
    assert path.tolist() == [[0, 2, 4, -1, -1, -1], [0, 1, -1, -1, -1, -1], [0, -1, -1, -1, -1, -1]]
    assert lens3.tolist() == [20, 20, 8]
    group = h // kv
    for b in range(n):
        rows = [x for x in path[b].tolist() if x >= 0]
        m = int(lens[b])
        full_k = torch.cat([k0[b, :m], kn.view(n, t, -1)[b, rows]]).double().view(-1, kv, d)
        full_v = torch.cat([v0[b, :m], vn.view(n, t, -1)[b, rows]]).double().view(-1, kv, d)
        assert torch.equal(k1[b, :m + len(rows)].double().view(-1, kv, d), full_k)
        assert torch.equal(v1[b, :m + len(rows)].double().view(-1, kv, d), full_v)
        want = torch.zeros(kv, m + len(rows), dtype=torch.float64, device="cuda")
        for i, r in enumerate(rows):
            x = q.view(n, t, h, d)[b, r].double()
            z = torch.einsum("hd,jhd->hj", x, full_k[:m + i + 1].repeat_interleave(group, 1)) / d ** 0.5
            p = torch.softmax(z, -1)
            want[:, :m + i + 1] += p.view(kv, group, -1).sum(1)
            o = torch.einsum("hj,jhd->hd", p, full_v[:m + i + 1].repeat_interleave(group, 1)).view(-1)
            got = out.view(n, t, -1)[b, r].double()
            # bf16 rounding of values of about one, and the bounds above
            assert torch.all((got - o).abs() <= 2.0 ** -8 * o.abs() + 1e-3)
        assert torch.all((w1[b, :, :want.shape[1]].double() - want).abs() <= 1e-3 * want + 1e-6)
        for hd in range(kv):
            keep = _keep_rows(w1[b, hd].cpu().numpy(), m + len(rows), 20, 4, 1)
            x = len(keep)
            assert kept[b, hd, :x].tolist() == keep.tolist()
            assert torch.equal(k[b, :x, hd * d:(hd + 1) * d], k1[b, keep, hd * d:(hd + 1) * d])
            assert torch.equal(w[b, hd, :x], w1[b, hd, keep])
