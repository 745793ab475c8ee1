"""The quantised-cache calls (swapnet_cache_append, swapnet_attention_quantized)
against plain float64 restatements of their definitions, at the sizes, masks
and contents where they can go wrong.

Tolerances, derived before any run.  A prepared row: the norm's sum of D
squares, quotient and root carry (D / 2 + 8) 2^-24, an angle 2^-23, a product
and a sum 2^-23 of their operands: 2^-16 of the row's largest element in all;
then one rounding, by half a step of its type.  A code is off by half a step of
its own (I8: scale / 2; E4M3: 2^-4 of the value, at least 2^-10 of the scale)
from the row's 16-bit value.  A score is a sum of D products accumulated in
fp32: off by at most (D + 8) 2^-23 sum|q_i k_i| scale (the tensor cores' sums
are allowed a whole step each, and a score is scaled and shifted three times),
which is p's relative error; 2^x is off by 2^-22, two fp16 parts leave 2^-22 of
p and 2^-32 of the largest; the sums over n keys by (n / 16 + 40) 2^-23 of sum p
|v|.  The quotient doubles what p carries."""
import math

import numpy as np
import pytest

from paper_2401_16757_gb300 import capi

pytestmark = pytest.mark.gpu

SENT = 7.0  # what outputs hold before a call
LEAST = 2.0 ** -100


def _torch():
    import torch
    return torch


def _dt(dtype):
    torch = _torch()
    return {"f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}[dtype]


def _eps(dtype):
    return {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]


def _stream():
    return _torch().cuda.current_stream().cuda_stream


# ------------------------------------------------------------------- append
def _scale(fmt, m):
    """The scale of blocks with largest magnitudes m (float64 array of 16-bit values)."""
    if fmt == "i8":
        s = m.astype(np.float32) / np.float32(127)
    else:
        f, e = np.frexp(m / 448.0)
        s = np.ldexp(1.0, np.where(f == 0.5, e - 1, e)) * (m > 0)
    s = np.maximum(s.astype(np.float64), LEAST)
    return np.where(np.isfinite(m), s, np.nan)


def _code(fmt, x, scale):
    """Values (float64) of the codes of finite x."""
    torch = _torch()
    y = x / scale
    if fmt == "i8":
        return np.rint((x.astype(np.float32) / scale.astype(np.float32)).astype(np.float64))
    return torch.from_numpy(y).float().to(torch.float8_e4m3fn).double().numpy()


def _prepared(x, gain, eps, theta, rope, halves, sections, pos):
    """float64 rows [t, heads, d], pos [axes, t]."""
    y = x.copy()
    if gain is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * gain
    if theta:
        n = rope // 2
        axis = np.repeat([0, 1, 2], sections) if any(sections[1:]) else np.zeros(n, dtype=int)
        ang = np.stack([pos[a].astype(np.float64) * float(np.float32(theta)) ** (-2.0 * i / rope) for i, a in enumerate(axis)], -1)[:, None]
        at = np.arange(n)
        at, by = (at, at + n) if halves else (2 * at, 2 * at + 1)
        a, b = y[..., at].copy(), y[..., by].copy()
        y[..., at], y[..., by] = a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)
    return y


class Append:
    """Inputs of one append call on a cache whose first rows came by an earlier one."""

    def __init__(self, dtype, fmt, n_seq, tokens, heads, kv_heads, dim, max_seq, block, lens, counts=None, norm=False, halves=False,
                 theta=10000.0, rope_dim=0, sections=(0, 0, 0), far=None, seed=0, pad=0, std=1.0):
        torch = _torch()
        g = torch.Generator().manual_seed(seed)
        self.__dict__.update(dtype=dtype, fmt=fmt, n=n_seq, t=tokens, heads=heads, kv=kv_heads, d=dim, max_seq=max_seq, block=block,
                             theta=theta, rope=rope_dim or dim, halves=halves, sections=sections, pad=pad)
        self.rope_arg = rope_dim
        self.lens, self.counts = np.asarray(lens, dtype=np.int32), None if counts is None else np.asarray(counts, dtype=np.int32)
        dt = _dt(dtype)

        def normal(*shape, std=1.0):
            return (torch.randn(*shape, generator=g, dtype=torch.float32) * std).to(dt).cuda()

        self.q = normal(n_seq, tokens, heads * dim + pad, std=2.0) if heads else None
        self.k_new, self.v_new = normal(n_seq, tokens, kv_heads * dim + pad, std=std), normal(n_seq, tokens, kv_heads * dim + pad, std=std)
        self.gains = (normal(dim), normal(dim)) if norm else None
        self.pos = None
        if far is not None:
            axes = 3 if any(sections[1:]) else 1
            self.pos = torch.randint(0, far, (axes, n_seq, tokens), generator=g, dtype=torch.int32).cuda()
        kd = kv_heads * dim + (2 * pad if fmt in ("i8", "e4m3") else pad)
        self.kd = kd
        self.coded = fmt in ("i8", "e4m3")
        ct = _dt(fmt)
        self.k, self.v = (torch.full((n_seq, max_seq, kd), SENT, device="cuda").to(ct) for _ in range(2))
        self.blocks = -(-max_seq // block) if self.coded else 0
        self.ks = self.vs = self.ko = self.vo = self.ko2 = self.vo2 = None
        if self.coded:
            self.ks, self.vs = (torch.full((n_seq, kv_heads, self.blocks), SENT, device="cuda") for _ in range(2))
            self.ko, self.vo = normal(n_seq, block, kv_heads, dim), normal(n_seq, block, kv_heads, dim)
            self.ko2, self.vo2 = (torch.full_like(self.ko, SENT) for _ in range(2))
        self.q_out = torch.full_like(self.q, SENT) if heads else None
        self.lens_out = torch.full((n_seq,), -9, dtype=torch.int32, device="cuda")

    def dev(self, x):
        return None if x is None else _torch().from_numpy(np.ascontiguousarray(x)).cuda()

    def call(self, in_place=False, stream=0, **kw):
        p = lambda x: 0 if x is None else x.data_ptr()  # noqa: E731
        if "lens" not in kw:  # (a capture takes no copies from the host)
            self._keep = self.dev(self.lens), self.dev(self.counts)
        lens, counts = self._keep
        gq, gk = self.gains or (None, None)
        args = dict(
            q=p(self.q), k_new=p(self.k_new), v_new=p(self.v_new), q_gain=p(gq) if self.heads else 0, k_gain=p(gk), lens=p(lens),
            counts=p(counts), positions=p(self.pos), q_out=p(self.q_out), k=p(self.k), v=p(self.v), k_scale=p(self.ks),
            v_scale=p(self.vs), k_open=p(self.ko), v_open=p(self.vo), k_open_out=0 if in_place else p(self.ko2),
            v_open_out=0 if in_place else p(self.vo2), lens_out=p(self.lens_out), block=self.block if self.coded else 0,
            rope_dim=self.rope_arg, theta=self.theta, halves=self.halves, sections=self.sections, eps=1e-5,
            q_stride=self.heads * self.d + self.pad if self.heads else 0, out_stride=self.heads * self.d + self.pad if self.heads else 0,
            new_stride=self.kv * self.d + self.pad, kv_stride=self.kd, seq_stride=self.kd * self.max_seq)
        args.update(kw)
        capi.cache_append(self.dtype, self.fmt, self.n, self.t, self.heads, self.kv, self.d, self.max_seq,
                          stream=stream or _stream(), **args)

    def check(self, open_rows=None):
        """Results of the call with other open buffers against the definition."""
        f64 = lambda x: x.double().cpu().numpy()  # noqa: E731
        n, t, h, kv, d, B = self.n, self.t, self.heads, self.kv, self.d, self.block
        eps = _eps(self.dtype)
        gq, gk = [None if self.gains is None else f64(x) for x in (self.gains or (0, 0))]
        k, v = f64(self.k)[..., :kv * d].reshape(n, -1, kv, d), f64(self.v)[..., :kv * d].reshape(n, -1, kv, d)
        assert (f64(self.k)[..., kv * d:] == SENT).all() and (f64(self.v)[..., kv * d:] == SENT).all()
        for b in range(n):
            ln, c = int(self.lens[b]), t if self.counts is None else int(self.counts[b])
            assert int(self.lens_out[b]) == ln + c
            pos = np.broadcast_to(ln + np.arange(c), (3, c)) if self.pos is None else self.pos[:, b, :c].cpu().numpy()
            rows = []
            for x, gain, heads in ((self.q, gq, h), (self.k_new, gk, kv), (self.v_new, None, kv)):
                if not heads:
                    rows.append(None)
                    continue
                y = f64(x)[b, :c, :heads * d].reshape(c, heads, d)
                if x is not self.v_new:
                    y = _prepared(y, gain, 1e-5, self.theta, self.rope, self.halves, self.sections, pos)
                rows.append(y)
            if h:
                got, want = f64(self.q_out)[b], rows[0]
                assert (got[c:] == SENT).all() and (got[:, h * d:] == SENT).all()
                got = got[:c, :h * d].reshape(c, h, d)
                assert (np.abs(got - want) <= eps * np.abs(want) + 2.0 ** -16 * np.abs(want).max(-1, keepdims=True)).all()
            if not self.coded:
                for cache, want, exact in ((k, rows[1], False), (v, rows[2], True)):
                    got = cache[b, ln:ln + c]
                    tol = 0 if exact else eps * np.abs(want) + 2.0 ** -16 * np.abs(want).max(-1, keepdims=True)
                    assert (np.abs(got - want) <= tol).all()
                    assert (cache[b, :ln] == SENT).all() and (cache[b, ln + c:] == SENT).all()
                continue
            for cache, scales, was, now, new, exact in ((k, f64(self.ks), f64(self.ko), f64(self.ko2), rows[1], False),
                                                        (v, f64(self.vs), f64(self.vo), f64(self.vo2), rows[2], True)):
                first, end = ln // B, ln + c
                assert (cache[b, :first * B] == SENT).all()
                assert (cache[b, end if c else 0:] == SENT).all()
                whole = np.concatenate([was[b, :ln % B], new])
                # rows that stay open: the earlier ones as they are, new ones rounded
                rest = end % B
                assert (now[b, rest:] == SENT).all()
                got, want = now[b, :rest], whole[len(whole) - rest:]
                fresh = np.arange(len(whole) - rest, len(whole)) >= ln % B
                tol = (eps * np.abs(want) + 2.0 ** -16 * np.abs(want).max(-1, keepdims=True)) * (0 if exact else fresh[:, None, None])
                assert (np.abs(got - want) <= tol).all()
                touched = -(-end // B) - first if c else 0
                keep = np.ones(scales.shape[2], dtype=bool)
                keep[first:first + touched] = False
                assert (scales[b][:, keep] == SENT).all()
                for i in range(touched):
                    x = whole[i * B:(i + 1) * B]
                    s = scales[b, :, first + i]
                    m = np.abs(x).max((0, 2))
                    code = cache[b, (first + i) * B:(first + i) * B + len(x)]
                    if exact:
                        assert (s == _scale(self.fmt, m)).all()
                        assert (code == _code(self.fmt, x, s[None, :, None])).all()
                        continue
                    off = (eps * m + 2.0 ** -16 * m) * 1.001
                    assert (s >= _scale(self.fmt, m - off) * (1 - 2.0 ** -22)).all() and (s <= _scale(self.fmt, m + off) * (1 + 2.0 ** -22)).all()
                    s = s[None, :, None]
                    step = s / 2 if self.fmt == "i8" else np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * s)
                    tol = step * (1 + 2.0 ** -4) + eps * np.abs(x) + 2.0 ** -16 * m[None, :, None]
                    assert (np.abs(code * s - x) <= tol).all()


@pytest.mark.parametrize("kw", [
    dict(dtype="bf16", fmt="e4m3", n_seq=1, tokens=1, heads=8, kv_heads=8, dim=128, max_seq=40, block=16, lens=[0]),
    dict(dtype="bf16", fmt="i8", n_seq=3, tokens=1, heads=6, kv_heads=2, dim=64, max_seq=64, block=16, lens=[15, 16, 63], norm=True, halves=True),
    dict(dtype="f16", fmt="e4m3", n_seq=4, tokens=5, heads=5, kv_heads=5, dim=64, max_seq=70, block=32, lens=[30, 0, 65, 31],
         counts=[5, 0, 5, 1], rope_dim=32, norm=True),
    dict(dtype="f16", fmt="i8", n_seq=2, tokens=130, heads=4, kv_heads=1, dim=128, max_seq=200, block=64, lens=[63, 70], counts=[129, 130],
         halves=True, rope_dim=64, pad=8),
    dict(dtype="bf16", fmt="e4m3", n_seq=2, tokens=300, heads=3, kv_heads=3, dim=128, max_seq=512, block=128, lens=[127, 1], norm=True,
         sections=(16, 24, 24), halves=True, far=5000),
    dict(dtype="bf16", fmt="e4m3", n_seq=1, tokens=33, heads=2, kv_heads=1, dim=64, max_seq=33, block=16, lens=[0], sections=(8, 12, 12), far=1 << 24),
    dict(dtype="f16", fmt="i8", n_seq=5, tokens=2, heads=0, kv_heads=7, dim=64, max_seq=9, block=16, lens=[7, 0, 3, 1, 5], theta=0.0, pad=16),
    dict(dtype="bf16", fmt="i8", n_seq=1, tokens=3, heads=1, kv_heads=1, dim=128, max_seq=3, block=128, lens=[0], far=1 << 24, halves=True, std=1e4),
    dict(dtype="bf16", fmt="e4m3", n_seq=2, tokens=20, heads=2, kv_heads=2, dim=128, max_seq=64, block=32, lens=[12, 31], std=1e-34, theta=0.0),
    dict(dtype="f16", fmt="f16", n_seq=3, tokens=37, heads=12, kv_heads=4, dim=64, max_seq=64, block=0, lens=[0, 27, 20], counts=[37, 37, 0],
         norm=True, pad=8),
    dict(dtype="bf16", fmt="bf16", n_seq=2, tokens=600, heads=14, kv_heads=6, dim=128, max_seq=700, block=0, lens=[100, 0], counts=[600, 599],
         halves=True, rope_dim=16),
    dict(dtype="bf16", fmt="bf16", n_seq=1, tokens=4, heads=0, kv_heads=3, dim=128, max_seq=4, block=0, lens=[0], norm=True, theta=500000.0, far=1 << 24),
    # many rows, eight heads of a token in the same lanes (the last ones fewer)
    dict(dtype="f16", fmt="e4m3", n_seq=1, tokens=1100, heads=19, kv_heads=2, dim=128, max_seq=1200, block=128, lens=[77], norm=True, halves=True,
         sections=(24, 20, 20), far=100000, pad=8),
    dict(dtype="bf16", fmt="i8", n_seq=2, tokens=1030, heads=9, kv_heads=1, dim=64, max_seq=1030, block=64, lens=[0, 0], counts=[1030, 1001],
         rope_dim=48),
])
def test_append_against_the_definition(kw):
    c = Append(seed=3, **kw)
    c.call()
    capi.device_sync()
    c.check()
    first = [x.clone() for x in (c.k, c.lens_out) + ((c.ko2, c.ks) if c.coded else ())]
    c.call()  # with the open rows elsewhere the call may be repeated
    capi.device_sync()
    for x, y in zip(first, [c.k, c.lens_out] + ([c.ko2, c.ks] if c.coded else [])):
        assert x.cpu().view(_torch().uint8).numpy().tobytes() == y.cpu().view(_torch().uint8).numpy().tobytes()


@pytest.mark.parametrize("fmt,block,dim,steps", [("e4m3", 16, 128, [1] * 40), ("i8", 32, 64, [5, 1, 26, 1, 64, 3]), ("e4m3", 64, 128, [70, 58, 1, 200]),
                                                ("i8", 128, 128, [100, 28, 129])])
def test_a_cache_is_a_function_of_its_rows(fmt, block, dim, steps):
    """Rows appended in one call or in many, in place: the same codes, scales and open rows, bit for bit."""
    torch = _torch()
    total = sum(steps)
    one = Append("bf16", fmt, 2, total, 4, 2, dim, total + 3, block, [0, 0], norm=True, halves=True, seed=5)
    one.call(in_place=True)
    many = Append("bf16", fmt, 2, total, 4, 2, dim, total + 3, block, [0, 0], norm=True, halves=True, seed=5)
    at, q = 0, []
    for t in steps:
        part = Append("bf16", fmt, 2, t, 4, 2, dim, total + 3, block, [at, at], norm=True, halves=True, seed=5)
        part.gains = many.gains
        for name in ("k", "v", "ks", "vs", "ko", "vo"):
            setattr(part, name, getattr(many, name))
        part.q, part.k_new, part.v_new = (x[:, at:at + t].contiguous() for x in (many.q, many.k_new, many.v_new))
        part.call(in_place=True)
        q.append(part.q_out)
        at += t
    capi.device_sync()
    rest = total % block
    same = [(one.k, many.k), (one.v, many.v), (one.ks, many.ks), (one.vs, many.vs), (one.ko[:, :rest], many.ko[:, :rest]),
            (one.vo[:, :rest], many.vo[:, :rest]), (one.q_out, torch.cat(q, dim=1))]
    for x, y in same:
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


def test_append_leaves_a_sequence_without_room_alone():
    for change in (dict(lens=[30, 5, 3]), dict(lens=[-1, 5, 3]), dict(lens=[41, 5, 3]), dict(lens=[3, 5, 3], counts=[12, 11, 11]),
                   dict(lens=[3, 5, 3], counts=[-1, 11, 11])):
        for fmt in ("i8", "f16"):
            kw = dict(change)
            c = Append("f16", fmt, 3, 11, 2, 2, 64, 40, 16 if fmt == "i8" else 0, seed=1, **kw)
            c.call()
            with pytest.raises(capi.SwapnetError) as e:
                capi.device_sync()
            assert e.value.code == capi.ERR_INVALID_ARG
            assert (c.k[0].double() == SENT).all() and (c.q_out[0] == SENT).all() and int(c.lens_out[0]) == -9
            if c.coded:
                assert (c.ks[0] == SENT).all() and (c.ko2[0] == SENT).all()
            # the others are done
            assert c.lens_out.tolist()[1:] == [16, 14] and not (c.q_out[1:] == SENT).all()
    capi.device_sync()


def test_rows_taken_back():
    """A sequence whose last rows are taken back, within the open block: what is appended then is as if they had never been."""
    torch = _torch()
    kw = dict(dtype="bf16", fmt="i8", n_seq=1, heads=2, kv_heads=2, dim=64, max_seq=64, block=32, norm=True)
    a, b = (Append(tokens=10, lens=[0], seed=1, **kw) for _ in range(2))
    a.call(in_place=True), b.call(in_place=True)
    gone = Append(tokens=9, lens=[10], seed=2, std=50.0, **kw)  # larger values: other scales and codes
    last = Append(tokens=5, lens=[10], seed=3, **kw)
    again = Append(tokens=5, lens=[10], seed=3, **kw)
    for x, of in ((gone, a), (last, a), (again, b)):
        for name in ("k", "v", "ks", "vs", "ko", "vo"):
            setattr(x, name, getattr(of, name))
        x.gains = a.gains
        x.call(in_place=True)
    capi.device_sync()
    for name in ("k", "v", "ko", "vo"):
        assert torch.equal(getattr(a, name)[:, :15], getattr(b, name)[:, :15])
    assert torch.equal(a.ks[:, :, :1], b.ks[:, :, :1]) and torch.equal(a.vs[:, :, :1], b.vs[:, :, :1])


def test_append_reports_positions_out_of_range():
    torch = _torch()
    for bad in (-1, 1 << 24, -2 ** 31):
        c = Append("bf16", "e4m3", 1, 4, 2, 2, 128, 40, 16, [0], far=100, seed=2)
        c.pos[0, 0, 2] = bad
        c.call()
        with pytest.raises(capi.SwapnetError) as e:
            capi.device_sync()
        assert e.value.code == capi.ERR_INVALID_ARG
        c.pos[0, 0, 2] = 0  # what it counts as
        c.check()
    assert torch.cuda.is_available()


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_append_of_values_that_are_no_numbers(fmt):
    """The scale of such a block is no number, of that head alone; others are as ever."""
    for bad in (float("inf"), -float("inf"), float("nan")):
        c = Append("bf16", fmt, 1, 40, 2, 3, 64, 64, 16, [0], theta=0.0, seed=4)
        good = Append("bf16", fmt, 1, 40, 2, 3, 64, 64, 16, [0], theta=0.0, seed=4)
        c.v_new[0, 20, 64 + 5] = bad  # head 1, block 1
        c.call()
        good.call()
        capi.device_sync()
        vs = c.vs.cpu().numpy()
        assert np.isnan(vs[0, 1, 1]) and np.isfinite(np.delete(vs.reshape(-1), 1 * 4 + 1)).all()
        a, b = c.v.view(_torch().uint8).cpu().numpy().copy(), good.v.view(_torch().uint8).cpu().numpy().copy()
        if fmt == "i8":
            assert (a[0, 16:32, 64:128] == 0).all()
        a[0, 16:32, 64:128] = b[0, 16:32, 64:128] = 0
        assert (a == b).all()


@pytest.mark.parametrize("dtype,bits", [("f16", 10), ("bf16", 7)])
def test_i8_codes_are_the_rounded_quotients(dtype, bits):
    """Every fraction of a largest magnitude against every fraction of a value, at each distance of their exponents that a
    code tells apart: the code is the quotient by the scale as fp32 rounds it, rounded to the nearest, ties to even."""
    torch = _torch()
    n, dt = 1 << bits, _dt(dtype)
    most = torch.arange(n, 2 * n, device="cuda", dtype=torch.float32)  # a head each
    x = most[None].repeat(n, 1)
    for shift in range(9):
        y = (x * 2.0 ** -shift).clamp(max=most[:, None]).to(dt)
        rows = torch.zeros(n, 1024, dtype=dt, device="cuda")  # 16 rows of 64 elements a head
        rows[:, :n] = y
        rows[:, 0] = most
        rows[:, 1::2] *= -1
        k = rows.view(n, 16, 64).transpose(0, 1).contiguous().view(1, 16, n * 64)
        codes, scale = torch.zeros(2, 16, n * 64, dtype=torch.int8, device="cuda"), torch.zeros(2, n, device="cuda")
        room, lens = torch.zeros_like(k), torch.zeros(1, dtype=torch.int32, device="cuda")
        capi.cache_append(dtype, "i8", 1, 16, 0, n, 64, 16, k_new=k.data_ptr(), v_new=k.data_ptr(), lens=lens.data_ptr(),
                          k=codes[0].data_ptr(), v=codes[1].data_ptr(), k_scale=scale[0].data_ptr(), v_scale=scale[1].data_ptr(),
                          k_open=room.data_ptr(), v_open=room.data_ptr() + 32 * n, block=16, stream=_stream())
        capi.device_sync()
        want = most.cpu().numpy() / np.float32(127)
        assert (scale[0].cpu().numpy() == want).all() and (scale[1].cpu().numpy() == want).all()
        want = np.rint(rows.float().cpu().numpy() / want[:, None])
        for c in codes:
            assert (c.view(16, n, 64).transpose(0, 1).reshape(n, 1024).cpu().numpy() == want).all()


def test_queries_in_place_on_a_stream_of_their_own_and_in_a_graph():
    torch = _torch()
    kw = dict(dtype="bf16", fmt="e4m3", n_seq=3, tokens=2, heads=8, kv_heads=2, dim=128, max_seq=64, block=16, lens=[15, 3, 40], norm=True)
    want = Append(seed=8, **kw)
    want.call()
    got, side = Append(seed=8, **kw), torch.cuda.Stream()
    torch.cuda.synchronize()
    got.call(q_out=got.q.data_ptr(), stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got.q, want.q_out) and torch.equal(got.ks, want.ks) and torch.equal(got.k.view(torch.uint8), want.k.view(torch.uint8))
    c = Append(seed=8, **kw)
    c.call()
    capi.device_sync()
    lens, _ = c._keep
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(lens=lens.data_ptr())
    other = Append(seed=9, **dict(kw, lens=[0, 31, 17]))
    c.q.copy_(other.q), c.k_new.copy_(other.k_new), c.v_new.copy_(other.v_new), lens.copy_(other.dev(other.lens))
    for name in ("k", "v", "ks", "vs", "ko2", "vo2", "q_out", "ko", "vo"):
        getattr(c, name).copy_(getattr(other, name))
    c.gains[0].copy_(other.gains[0]), c.gains[1].copy_(other.gains[1])
    graph.replay()
    torch.cuda.synchronize()
    c.lens = other.lens
    c.check()


# ---------------------------------------------------------------- attention
class Attend:
    """Inputs of one attention call, their float64 results and bounds."""

    def __init__(self, dtype, fmt, n_seq, tokens, heads, kv_heads, dim, max_seq, block, lens, counts=None, seed=0, scale=0.0, pad=0,
                 spread=1.0, std=1.5):
        torch = _torch()
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.__dict__.update(dtype=dtype, fmt=fmt, n=n_seq, t=tokens, h=heads, kv=kv_heads, d=dim, max_seq=max_seq, block=block,
                             scale=scale, pad=pad)
        self.lens, self.counts = np.asarray(lens, dtype=np.int32), None if counts is None else np.asarray(counts, dtype=np.int32)
        self.q = (torch.randn(n_seq, tokens, heads * dim + pad, generator=g) * std).to(_dt(dtype)).cuda()
        top = {"i8": 127.0, "e4m3": 448.0}[fmt]
        self.kd = kv_heads * dim + 2 * pad

        def codes():
            x = (torch.randn(n_seq, max_seq, self.kd, generator=g) * top / 4).clamp(-top, top)
            x = x.round() if fmt == "i8" else x
            return x.to(_dt(fmt)).cuda()

        self.k, self.v = codes(), codes()
        blocks = -(-max_seq // block)
        self.ks = torch.from_numpy((np.exp2(rng.uniform(-1, 1, (n_seq, kv_heads, blocks))) * 4 / top).astype(np.float32))
        self.vs = torch.from_numpy((np.exp2(rng.uniform(-1, 1, (n_seq, kv_heads, blocks)) * spread) * 4 / top).astype(np.float32))
        for b in range(n_seq):  # codes behind the rows in use, and scales of blocks behind them, hold anything
            used = min(max_seq, max(0, int(self.lens[b])))
            raw = torch.randint(0, 256, (max_seq - used, self.kd), generator=g).to(torch.uint8).cuda()
            for x in (self.k, self.v):
                x.view(torch.uint8)[b, used:] = raw
            for x in (self.ks, self.vs):
                x[b, :, -(-used // block):] = float(rng.choice([np.nan, np.inf, -1.0]))
        self.ks, self.vs = self.ks.cuda(), self.vs.cuda()
        self.out = torch.full((n_seq, tokens, heads * dim + pad), SENT, dtype=_dt(dtype), device="cuda")
        self.lse = torch.full((n_seq, heads, tokens), SENT, device="cuda")

    def args(self, **kw):
        torch = _torch()
        if "lens" not in kw or not hasattr(self, "_keep"):  # (a capture takes no copies from the host)
            self._keep = torch.from_numpy(self.lens).cuda(), None if self.counts is None else torch.from_numpy(self.counts).cuda()
        lens, counts = self._keep
        a = dict(q=self.q.data_ptr(), k=self.k.data_ptr(), v=self.v.data_ptr(), k_scale=self.ks.data_ptr(), v_scale=self.vs.data_ptr(),
                 lens=lens.data_ptr(), counts=0 if counts is None else counts.data_ptr(), out=self.out.data_ptr(), lse=self.lse.data_ptr(),
                 scale=self.scale, q_stride=self.q.shape[2], out_stride=self.out.shape[2], kv_stride=self.kd, seq_stride=self.kd * self.max_seq)
        a.update(kw)
        return capi.quantized_attention(self.dtype, self.fmt, self.n, self.t, self.h, self.kv, self.d, self.max_seq, self.block, **a)

    def call(self, stream=0, space=None, **kw):
        torch = _torch()
        a = self.args(**kw)
        need = capi.attention_quantized_workspace(a)
        self.space = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda") if space is None else space
        assert self.space.numel() >= need
        capi.attention_quantized(a, self.space.data_ptr() if need else 0, self.space.numel(), stream or _stream())

    def check(self, skip=()):
        torch = _torch()
        n, t, h, kv, d, B = self.n, self.t, self.h, self.kv, self.d, self.block
        grp, scale, eps = h // kv, self.scale or 1 / math.sqrt(d), _eps(self.dtype)
        for b in range(n):
            ln, c = int(self.lens[b]), t if self.counts is None else int(self.counts[b])
            if b in skip:
                ln = c = 0
            assert (self.out[b, c:] == SENT).all() and (self.out[b, :, h * d:] == SENT).all() and (self.lse[b, :, c:] == SENT).all()
            if c == 0:
                continue
            row = torch.arange(ln, device="cuda")
            seen = (row <= (ln - c + torch.arange(c, device="cuda"))[:, None])[None]
            for e in range(kv):
                k, v = (x[b, :ln, e * d:(e + 1) * d].double() * s[b, e][row // B].double()[:, None]
                        for x, s in ((self.k, self.ks), (self.v, self.vs)))
                q = self.q[b, :c, e * grp * d:(e + 1) * grp * d].double().view(c, grp, d).transpose(0, 1)
                if ln == 0:
                    assert (self.out[b, :c, e * grp * d:(e + 1) * grp * d] == 0).all()
                    assert (self.lse[b, e * grp:(e + 1) * grp, :c] == -math.inf).all()
                    continue
                s = torch.where(seen, q @ k.T * scale, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
                off = torch.where(seen, (q.abs() @ k.abs().T) * scale, torch.zeros_like(s)).amax(-1) * (d + 8) * 2.0 ** -23
                m = s.amax(-1, keepdim=True)
                p = torch.where(seen, torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m)), torch.zeros_like(s))
                l = p.sum(-1, keepdim=True)
                lse = (m + torch.log(l))[..., 0]
                p = p / torch.where(l > 0, l, torch.ones_like(l))
                want, size = p @ v, p @ v.abs()
                # p times a value scale, 2^7 or more where it is largest, is off by up to half of fp16's least step, 2^-25:
                # by 2^-32 of the largest, times the row's code
                vs = self.vs[b, e][row // B].double()
                part = (p * vs).amax(-1)[..., None] * self.v[b, :ln, e * d:(e + 1) * d].double().abs().sum(0)
                rel = 2 * off + 2.0 ** -21 + (ln / 16 + 40) * 2.0 ** -23 + 2.0 ** -22
                tol = eps * want.abs() + rel[..., None] * size + 2.0 ** -32 * part
                got = self.out[b, :c, e * grp * d:(e + 1) * grp * d].double().view(c, grp, d).transpose(0, 1)
                ok = (got - want).abs() <= tol * (1 + 2.0 ** -10)
                if self.dtype == "f16":  # from half a step behind its largest number on, 65520, the nearest fp16 is infinite
                    ok |= torch.isinf(got) & (got.sign() == want.sign()) & (want.abs() + tol >= 65520)
                assert ok.all(), (b, e, ((got - want).abs() / tol).max().item())
                gl = self.lse[b, e * grp:(e + 1) * grp, :c].double()
                hit = torch.isfinite(lse)
                assert (gl[~hit] == -math.inf).all()
                tol = off + 2.0 ** -20 + (ln / 16 + 40) * 2.0 ** -23 + 2.0 ** -22 * lse.abs()
                assert ((gl - lse).abs() <= tol)[hit].all(), (b, e)


@pytest.mark.parametrize("kw", [
    dict(dtype="bf16", fmt="i8", n_seq=1, tokens=1, heads=8, kv_heads=8, dim=128, max_seq=160, block=16, lens=[100]),
    dict(dtype="bf16", fmt="e4m3", n_seq=1, tokens=1, heads=4, kv_heads=4, dim=128, max_seq=544, block=32, lens=[543]),
    dict(dtype="f16", fmt="i8", n_seq=6, tokens=1, heads=8, kv_heads=2, dim=64, max_seq=65, block=32, lens=[0, 1, 31, 32, 33, 65]),
    dict(dtype="f16", fmt="e4m3", n_seq=6, tokens=2, heads=10, kv_heads=2, dim=128, max_seq=200, block=64, lens=[0, 1, 2, 64, 129, 200]),
    dict(dtype="bf16", fmt="i8", n_seq=3, tokens=7, heads=6, kv_heads=3, dim=128, max_seq=300, block=128, lens=[5, 300, 128], counts=[7, 3, 0], pad=16),
    dict(dtype="f16", fmt="e4m3", n_seq=1, tokens=3, heads=16, kv_heads=4, dim=64, max_seq=5000, block=128, lens=[4999]),
    dict(dtype="bf16", fmt="e4m3", n_seq=2, tokens=8, heads=8, kv_heads=2, dim=128, max_seq=1000, block=64, lens=[1000, 517]),
    dict(dtype="bf16", fmt="i8", n_seq=2, tokens=40, heads=4, kv_heads=4, dim=64, max_seq=333, block=16, lens=[333, 12], counts=[40, 39]),
    dict(dtype="f16", fmt="i8", n_seq=2, tokens=200, heads=8, kv_heads=2, dim=128, max_seq=400, block=64, lens=[400, 200], counts=[199, 200]),
    dict(dtype="bf16", fmt="e4m3", n_seq=1, tokens=150, heads=3, kv_heads=1, dim=64, max_seq=700, block=32, lens=[700], scale=0.3),
    dict(dtype="f16", fmt="e4m3", n_seq=1, tokens=1, heads=100, kv_heads=1, dim=128, max_seq=90, block=16, lens=[77]),
    dict(dtype="bf16", fmt="i8", n_seq=1, tokens=2, heads=128, kv_heads=1, dim=128, max_seq=1500, block=16, lens=[1500]),
    dict(dtype="bf16", fmt="i8", n_seq=20, tokens=1, heads=16, kv_heads=16, dim=128, max_seq=700, block=32, lens=list(range(0, 700, 35))),
    dict(dtype="bf16", fmt="i8", n_seq=2, tokens=5, heads=8, kv_heads=4, dim=64, max_seq=2100, block=16, lens=[2100, 2063], spread=20.0),
    dict(dtype="f16", fmt="e4m3", n_seq=2, tokens=70, heads=4, kv_heads=2, dim=128, max_seq=600, block=16, lens=[600, 64], spread=20.0),
    dict(dtype="bf16", fmt="e4m3", n_seq=2, tokens=1, heads=4, kv_heads=1, dim=128, max_seq=300, block=32, lens=[300, 299], std=1e-30),
    dict(dtype="bf16", fmt="i8", n_seq=2, tokens=33, heads=4, kv_heads=1, dim=128, max_seq=300, block=32, lens=[300, 299], std=1e4, scale=1e-5),
    # rows of other strides on the tensor cores, one and two rows a lane
    dict(dtype="f16", fmt="i8", n_seq=2, tokens=50, heads=4, kv_heads=2, dim=64, max_seq=400, block=16, lens=[399, 50], pad=24),
    dict(dtype="bf16", fmt="e4m3", n_seq=2, tokens=11, heads=8, kv_heads=2, dim=128, max_seq=400, block=128, lens=[399, 250], pad=8),
    # runs of tiles over more sequences than a CTA keeps sizes of, some of them empty
    dict(dtype="bf16", fmt="i8", n_seq=70, tokens=2, heads=2, kv_heads=1, dim=64, max_seq=9000, block=64,
         lens=[(i * 1237) % 3000 * (i % 5 > 0) for i in range(69)] + [9000], counts=[2 - i % 3 % 2 for i in range(70)]),
    dict(dtype="f16", fmt="e4m3", n_seq=66, tokens=40, heads=1, kv_heads=1, dim=64, max_seq=6000, block=16,
         lens=[(i * 1237) % 1000 * (i % 4 > 0) for i in range(65)] + [6000], counts=[40 - i % 41 for i in range(66)]),
    # a unit over many runs: tails of one tile, rows that see nothing of them
    dict(dtype="f16", fmt="i8", n_seq=1, tokens=30, heads=1, kv_heads=1, dim=128, max_seq=20000, block=32, lens=[19970]),
    dict(dtype="bf16", fmt="e4m3", n_seq=1, tokens=300, heads=1, kv_heads=1, dim=128, max_seq=9000, block=64, lens=[8833]),
    # many units of more rows
    dict(dtype="bf16", fmt="i8", n_seq=20, tokens=100, heads=8, kv_heads=8, dim=128, max_seq=300, block=16,
         lens=[(i * 97) % 201 + 100 for i in range(20)], counts=[100 - i * 5 for i in range(20)]),
    dict(dtype="f16", fmt="e4m3", n_seq=30, tokens=50, heads=8, kv_heads=8, dim=128, max_seq=2000, block=64,
         lens=[(i * 1237) % 2001 for i in range(30)], counts=[min(50 - i, (i * 1237) % 2001) for i in range(30)]),
    # units of 17 to 32 rows of 128
    dict(dtype="f16", fmt="i8", n_seq=1, tokens=17, heads=1, kv_heads=1, dim=128, max_seq=128, block=16, lens=[128]),
    dict(dtype="bf16", fmt="e4m3", n_seq=5, tokens=8, heads=16, kv_heads=4, dim=128, max_seq=700, block=64, lens=[0, 3, 128, 129, 700],
         counts=[8, 5, 8, 0, 7], pad=16),
    dict(dtype="bf16", fmt="i8", n_seq=3, tokens=3, heads=20, kv_heads=2, dim=128, max_seq=400, block=16, lens=[1, 257, 400], pad=8),
    dict(dtype="f16", fmt="e4m3", n_seq=2, tokens=1, heads=31, kv_heads=1, dim=128, max_seq=3000, block=128, lens=[2999, 640]),
    dict(dtype="f16", fmt="i8", n_seq=70, tokens=25, heads=2, kv_heads=2, dim=128, max_seq=1500, block=32,
         lens=[(i * 1237) % 1400 * (i % 4 > 0) for i in range(69)] + [1500], counts=[25 - i % 26 for i in range(70)]),
    dict(dtype="bf16", fmt="e4m3", n_seq=2, tokens=8, heads=8, kv_heads=2, dim=128, max_seq=40000, block=16, lens=[39999, 9], spread=20.0),
    dict(dtype="bf16", fmt="i8", n_seq=40, tokens=4, heads=32, kv_heads=4, dim=128, max_seq=600, block=32,
         lens=[(i * 731) % 600 + 1 for i in range(40)], std=4.0),
])
def test_attention_against_the_definition(kw):
    c = Attend(seed=6, **kw)
    c.call()
    capi.device_sync()
    c.check()


@pytest.mark.parametrize("tokens,heads,max_seq", [(1, 4, 300), (6, 4, 300), (12, 4, 300), (50, 4, 300), (150, 2, 300), (1, 4, 9000), (12, 4, 9000), (50, 2, 9000)])
def test_attention_leaves_bad_sequences_alone(tokens, heads, max_seq):
    """A CTA per unit (short caches) or equal runs (long ones)."""
    for lens, counts in (([max_seq + 1, 300], None), ([-1, 300], None), ([200, 300], [tokens + 1, tokens]), ([200, 300], [-1, tokens])):
        c = Attend("bf16", "i8", 2, tokens, heads, 2, 128, max_seq, 32, lens, counts, seed=2)
        c.call()
        with pytest.raises(capi.SwapnetError) as e:
            capi.device_sync()
        assert e.value.code == capi.ERR_INVALID_ARG
        c.check(skip=(0,))
    capi.device_sync()


@pytest.mark.parametrize("dim,tokens", [(128, 2), (128, 12), (128, 70), (128, 200), (64, 12), (64, 70), (64, 200)])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_scales_that_are_no_numbers_reach_only_the_queries_that_see_them(dim, tokens, fmt):
    """A block whose scale is no number: queries that see one of its rows get no number, the others are untouched by it,
    also where they share a tile with the block's rows; codes there may be any bytes."""
    torch = _torch()
    ln, B = 300, 16
    good = Attend("bf16", fmt, 1, tokens, 4, 2, dim, 320, B, [ln], seed=11)
    good.call()
    capi.device_sync()
    for which, value in (("ks", math.nan), ("vs", math.nan), ("vs", math.inf)):
        c = Attend("bf16", fmt, 1, tokens, 4, 2, dim, 320, B, [ln], seed=11)
        block = (ln - 2) // B  # the last rows but one, seen by the last queries
        getattr(c, which)[0, 1, block] = value
        for x in (c.k, c.v):
            x.view(torch.uint8)[0, block * B:(block + 1) * B, dim:2 * dim] = 0x7f
        c.call()
        capi.device_sync()
        first = max(0, block * B - (ln - tokens))  # the first query that sees the block
        out, ref = c.out.view(1, tokens, 4, dim), good.out.view(1, tokens, 4, dim)
        assert torch.equal(out[:, :, :2], ref[:, :, :2])  # the other key head
        assert torch.equal(out[:, :first], ref[:, :first])
        if value == math.inf:
            assert not torch.isfinite(out[:, first:, 2:]).any()
        else:
            assert torch.isnan(out[:, first:, 2:]).all()


@pytest.mark.parametrize("tokens", [1, 40, 150])
def test_a_dominant_key_hides_nothing(tokens):
    """Beside a key that gets nearly everything and has the value 0, the others decide the output."""
    torch = _torch()
    c = Attend("f16", "i8", 1, tokens, 2, 1, 64, 4000, 16, [4000], seed=3)
    c.k.zero_(), c.v.fill_(64), c.ks.fill_(1.0), c.vs.fill_(2.0 ** -6)
    c.q.fill_(0.5)
    c.k[0, 5] = 4  # score 0.5 * 4 * 64 / 8 = 16: e^16 = 8.9e6 times the others
    c.v[0, 5] = 0
    c.call()
    capi.device_sync()
    n = 4000 - tokens + torch.arange(1, tokens + 1, dtype=torch.float64)  # rows seen
    want = (n - 1) / (n - 1 + math.exp(16.0))
    got = c.out.double().cpu()[0]
    # fp16 results of about 4e-4: half a step is 2^-11 of them; p: 2^-21 of the sums
    assert ((got - want[:, None]).abs() <= want[:, None] * (2.0 ** -11 + 2.0 ** -10 * 2.0 ** -3)).all()


@pytest.mark.parametrize("dim,tokens,max_seq", [(128, 1, 900), (128, 1, 9000), (128, 12, 900), (128, 40, 900), (64, 40, 900), (64, 150, 900)])
@pytest.mark.parametrize("least", [2.0 ** -100, 2.0 ** -48])
def test_zeros_beside_large_values_keep_their_weights(dim, tokens, max_seq, least):
    """All scores equal; every other block of 16 rows has small values, the others large ones: the mean of what is seen."""
    torch = _torch()
    for large in (1.0, 2.0 ** 40, 2.0 ** 64):
        c = Attend("bf16", "i8", 1, tokens, 2, 1, dim, max_seq, 16, [max_seq], seed=5)
        c.q.zero_(), c.v.fill_(64)
        c.vs[0, 0, 0::2], c.vs[0, 0, 1::2] = least, large
        if least < 2.0 ** -48:
            for i in range(0, max_seq, 32):
                c.v[0, i:i + 16] = 0
        c.call()
        capi.device_sync()
        n = max_seq - tokens + torch.arange(1, tokens + 1)
        big = n // 32 * 16 + (n % 32 - 16).clamp(min=0)
        want = (64 * large * big + (64 * least if least == 2.0 ** -48 else 0.0) * (n - big)).double() / n
        got = c.out.double().cpu()[0]
        # half a step of bf16; sums of n equal terms, two parts of p and the division: (n / 16 + 40) 2^-23
        tol = want * (2.0 ** -8 + (max_seq / 16 + 40) * 2.0 ** -23)
        assert ((got - want[:, None]).abs() <= tol[:, None]).all(), (large, ((got / want[:, None]) - 1).abs().max().item())
        lse = c.lse.double().cpu()[0]
        assert ((lse - torch.log(n.double())).abs() <= (max_seq / 16 + 40) * 2.0 ** -22).all()


def test_values_below_the_least_exponent():
    """Scales under 2^-48 lose bits from below: 2^-39 of 2^-48, whatever the scale."""
    torch = _torch()
    for tokens in (1, 40, 150):
        for small in (2.0 ** -60, 2.0 ** -70):
            c = Attend("bf16", "e4m3", 1, tokens, 2, 1, 64, 700, 32, [700], seed=7)
            c.q.zero_(), c.v.fill_(64), c.vs.fill_(small)
            c.call()
            capi.device_sync()
            want = torch.full((tokens, 128), 64 * small, dtype=torch.float64)
            # p is at least 2^7 (more rows: where the first keys put it), so that half of 2^-24 is 2^-32 of 2^-48 / scale
            tol = want * (2.0 ** -8 + (700 / 16 + 40) * 2.0 ** -23 + 2.0 ** -32 * 2.0 ** -48 / small)
            assert ((c.out.double().cpu()[0] - want).abs() <= tol).all(), (tokens, small)


@pytest.mark.parametrize("dim,tokens", [(128, 1), (128, 12), (128, 40), (64, 12), (64, 40), (64, 150)])
@pytest.mark.parametrize("score", [-3000.0, 3000.0])
def test_scores_far_from_zero(dim, tokens, score):
    """All scores equal and far from what exponentials hold: the mean of the values seen; then one key above all others."""
    torch = _torch()
    ln = 1400
    c = Attend("f16", "i8", 1, tokens, 2, 1, dim, ln, 32, [ln], seed=13)
    c.k.fill_(64 if score > 0 else -64), c.ks.fill_(1.0), c.vs.fill_(2.0 ** -6)
    c.q.fill_(4.0)
    c.scale = 3000 / (4.0 * 64 * dim)
    c.v.zero_()
    c.v[0, ::2] = 64
    c.call()
    capi.device_sync()
    n = ln - tokens + torch.arange(1, tokens + 1)
    want = ((n + 1) // 2).double() / n
    got, lse = c.out.double().cpu()[0], c.lse.double().cpu()[0]
    # half a step of fp16; the scores are exact (powers of two and 3000 / 2^15, one rounding each: 2^-22 of 3000 / ln 2 bits, for all the same)
    assert ((got - want[:, None]).abs() <= want[:, None] * (2.0 ** -11 + (ln / 16 + 40) * 2.0 ** -23)).all()
    assert ((lse - score - torch.log(n.double())).abs() <= 3000 * 2.0 ** -21 + (ln / 16 + 40) * 2.0 ** -22).all()
    c.k[0, ln - tokens - 30] = 127 if score > 0 else -1
    c.call()
    capi.device_sync()
    assert (c.out[0] == (1.0 if (ln - tokens - 30) % 2 == 0 else 0.0)).all()


def test_large_offsets():
    """Rows of a cache beyond 2^32 bytes."""
    torch = _torch()
    n, stride, d = 4100, 1 << 20, 64
    kv = torch.zeros(n * stride, dtype=torch.int8, device="cuda")
    small = Attend("bf16", "i8", 1, 5, 4, 2, d, n, 32, [n], seed=1)
    rows = torch.arange(n, device="cuda")
    for h in range(2 * d):
        kv[rows * stride + h] = small.k[0, :, h]
        kv[rows * stride + 2 * d + h] = small.v[0, :, h]
    small.call()
    want = small.out.clone()
    small.call(k=kv.data_ptr(), v=kv.data_ptr() + 2 * d, kv_stride=stride, seq_stride=0)
    capi.device_sync()
    assert torch.equal(small.out, want)
    far = Append("bf16", "i8", 1, 3, 0, 2, d, n, 32, [n - 3], theta=0.0, seed=2)
    near = Append("bf16", "i8", 1, 3, 0, 2, d, n, 32, [n - 3], theta=0.0, seed=2)
    far.call(k=kv.data_ptr(), v=kv.data_ptr() + 2 * d, kv_stride=stride, seq_stride=0)
    near.call()
    capi.device_sync()
    for r in range(n - 3, n):
        assert torch.equal(kv[r * stride:r * stride + 2 * d], near.k[0, r]) and torch.equal(kv[r * stride + 2 * d:r * stride + 4 * d], near.v[0, r])
    del kv


@pytest.mark.parametrize("tokens", [1, 7, 9, 150])
def test_attention_in_graphs_and_on_streams(tokens):
    """Captured and replayed on other inputs; two calls at once with workspaces of their own; the same bits every time."""
    torch = _torch()
    kw = dict(dtype="bf16", fmt="e4m3", n_seq=2, tokens=tokens, heads=8, kv_heads=2, dim=128, max_seq=3000, block=64)
    a, b = Attend(lens=[2999, 1500], seed=1, **kw), Attend(lens=[700, 3000], seed=2, **kw)
    a.call()
    b.call()
    capi.device_sync()
    want = [a.out.clone(), b.out.clone()]
    lens = a._keep[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.call(lens=lens.data_ptr(), space=a.space)
    a.out.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.out, want[0])
    for name in ("q", "k", "v", "ks", "vs"):
        getattr(a, name).copy_(getattr(b, name))
    lens.copy_(torch.from_numpy(b.lens))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.out, want[1])
    c = Attend(lens=[2999, 1500], seed=1, **kw)
    streams = [torch.cuda.Stream() for _ in range(2)]
    c.call()
    torch.cuda.synchronize()
    for x in (b, c):
        x.out.fill_(0)
    torch.cuda.synchronize()
    for _ in range(4):
        for x, s in ((c, streams[0]), (b, streams[1])):
            x.call(stream=s.cuda_stream, space=x.space, lens=x._keep[0].data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(c.out, want[0]) and torch.equal(b.out, want[1])


@pytest.mark.parametrize("dtype,fmt,block", [("bf16", "e4m3", 16), ("f16", "i8", 32)])
def test_append_and_attend_together(dtype, fmt, block):
    """A prompt, then decode steps and a run of tokens: attention over what the appends left, step by step against the float64 attention of
    the cache's values."""
    torch = _torch()
    n, h, kv, d, cap = 2, 8, 2, 128, 120
    store, lens = None, np.array([0, 0], dtype=np.int32)
    for i, (t, counts) in enumerate([(50, [50, 33]), (1, [1, 1]), (1, [1, 0]), (9, [9, 4]), (1, [1, 1])]):
        c = Append(dtype, fmt, n, t, h, kv, d, cap, block, lens, counts, norm=True, seed=20 + i)
        if store:
            for name in ("k", "v", "ks", "vs", "ko", "vo"):
                setattr(c, name, getattr(store, name))
        c.call(in_place=True)
        lens = lens + c.counts
        a = Attend(dtype, fmt, n, t, h, kv, d, cap, block, lens, counts, seed=1)
        a.q, a.k, a.v, a.ks, a.vs = c.q_out, c.k, c.v, c.ks, c.vs
        a.call(lens=c.lens_out.data_ptr())
        capi.device_sync()
        a.check()
        store = c
