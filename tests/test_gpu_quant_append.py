"""swapnet_cache_append where its users' calls go beyond the sizes of
test_gpu_quant.py."""
import decimal

import numpy as np
import pytest

from paper_2401_16757_gb300 import capi

from test_gpu_quant import Append, _stream, _torch

pytestmark = pytest.mark.gpu


def _angles(theta, rope, positions):
    """position * theta^(-2 i / rope) less whole turns, as exact as float64 holds it, and the angles as they are: [t][pairs]."""
    decimal.getcontext().prec = 60
    D = decimal.Decimal
    pi = D("3.14159265358979323846264338327950288419716939937510582097494459")
    log = D(float(np.float32(theta))).ln()
    freq = [(log * (-2 * i) / rope).exp() for i in range(rope // 2)]
    rest = np.empty((len(positions), rope // 2))
    for t, p in enumerate(positions):
        for i, f in enumerate(freq):
            x = int(p) * f
            rest[t, i] = float(x - (x / (2 * pi)).to_integral_value() * 2 * pi)
    return rest, np.outer(positions, [float(f) for f in freq])


@pytest.mark.parametrize("theta,rope", [(10000.0, 128), (1e6, 48), (1.0, 128), (0.5, 128), (0.01, 128), (1e-4, 48), (1e-6, 128)])
def test_angles_of_far_positions(theta, rope):
    """Pairs (a, b) of large numbers chosen for each angle x so that a cos x - b sin x nearly vanishes: what is left shows the
    angle's error, |(a, b)| times it.

    Promised: 2^-21, and 2^-49 of position * frequency.  Sine and cosine as functions of the angle: 2^-23 (series 2^-25, their last step
    2^-24).  The product b sin x: 2^-24 of itself; the sum and the result: half a step of fp16."""
    torch = _torch()
    rng = np.random.default_rng(int(theta * 8) + rope)
    pos = np.concatenate([[0, 1, 2, 4095, (1 << 24) - 1, (1 << 23) + 1], rng.integers(1 << 22, 1 << 24, 26)])
    rest, full = _angles(theta, rope, pos)
    c, s = np.cos(rest), np.sin(rest)
    n, pairs = rest.shape
    # of the larger of cos and sin the partner is the quotient, rounded; the best of many
    swap = np.abs(s) < np.abs(c)
    big, small = np.where(swap, c, s), np.where(swap, s, c)
    tries = rng.uniform(20000, 60000, (400, n, pairs)).astype(np.float16).astype(np.float64)
    other = (tries * small / big).astype(np.float16).astype(np.float64)
    best = np.abs(other * big - tries * small).argmin(0)[None]
    lead, follow = (np.take_along_axis(x, best, 0)[0] for x in (tries, other))
    a, b = np.where(swap, follow, lead), np.where(swap, lead, follow)
    q = np.zeros((n, 2, 128))
    q[:, 0, 0:rope:2], q[:, 0, 1:rope:2] = a, b          # u = a cos - b sin is small
    q[:, 1, 0:rope:2], q[:, 1, 1:rope:2] = b, -a         # v = -a cos + b sin is small
    dev = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(t).cuda()  # noqa: E731
    q, rows = dev(q, torch.float16), torch.zeros(n, 128, dtype=torch.float16, device="cuda")
    out, k, v = torch.zeros_like(q), torch.zeros_like(rows), torch.zeros_like(rows)
    lens, at = dev(np.zeros(1), torch.int32), dev(pos, torch.int32)
    capi.cache_append("f16", "f16", 1, n, 2, 1, 128, n, k_new=rows.data_ptr(), v_new=rows.data_ptr(), lens=lens.data_ptr(), k=k.data_ptr(),
                      v=v.data_ptr(), q=q.data_ptr(), q_out=out.data_ptr(), positions=at.data_ptr(), theta=theta, rope_dim=rope, stream=_stream())
    capi.device_sync()
    got = out.double().cpu().numpy()
    want = a * c - b * s
    size = np.hypot(a, b)
    tol = size * (2.0 ** -21 + 2.0 ** -49 * full) + (np.abs(a) + np.abs(b)) * 2.0 ** -23 + np.abs(b) * 2.0 ** -24 + 2.0 ** -11 * np.abs(want) + 2.0 ** -25
    assert 2.0 ** -11 * np.abs(want).max() < 2.0 ** -3 * (size * 2.0 ** -21).max()  # (what fp16's step hides)
    for x in (got[:, 0, 0:rope:2] - want, got[:, 1, 1:rope:2] + want):
        worst = np.abs(x) / tol
        assert (worst <= 1).all(), (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


def _bytes(x):
    return x.contiguous().view(_torch().uint8)


@pytest.mark.parametrize("fmt,dtype,dim", [("i8", "bf16", 128), ("e4m3", "f16", 64), ("bf16", "bf16", 128)])
@pytest.mark.parametrize("tokens,lens,counts", [(5, [30, 0, 65], [5, 0, 4]), (150, [31, 32, 1], [150, 97, 130])])
def test_sequence_strides(fmt, dtype, dim, tokens, lens, counts):
    """A sequence's rows a padded number of elements apart, and rows of all sequences in turn: the rows of the packed call, bit
    for bit, and nothing written beside them."""
    torch = _torch()
    n, kv, cap, block = 3, 2, 200, 32 if fmt in ("i8", "e4m3") else 0
    kw = dict(dtype=dtype, fmt=fmt, n_seq=n, tokens=tokens, heads=4, kv_heads=kv, dim=dim, max_seq=cap, block=block, lens=lens, counts=counts,
              norm=True, halves=True, seed=31)
    want = Append(**kw)
    want.call()
    capi.device_sync()
    kd = kv * dim
    for kv_stride, seq_stride in ((kd, kd * cap + 48), (kd + 16, (kd + 16) * cap + 16), (n * kd, kd), (n * kd + 32, kd)):
        total = (n - 1) * seq_stride + (cap - 1) * kv_stride + kd
        c = Append(**kw)
        k, v = (torch.full((total,), 7.0, device="cuda").to(want.k.dtype) for _ in range(2))
        c.call(k=k.data_ptr(), v=v.data_ptr(), kv_stride=kv_stride, seq_stride=seq_stride)
        capi.device_sync()
        for flat, ref, scales, ref_scales in ((k, want.k, c.ks, want.ks), (v, want.v, c.vs, want.vs)):
            left = _bytes(flat).clone().view(total, -1)
            for b in range(n):
                rows = torch.as_strided(flat, (cap, kd), (kv_stride, 1), b * seq_stride)
                assert torch.equal(_bytes(rows), _bytes(ref[b]))
                at = (b * seq_stride + torch.arange(cap, device="cuda")[:, None] * kv_stride + torch.arange(kd, device="cuda")).flatten()
                left[at] = _bytes(torch.full((1,), 7.0, device="cuda").to(flat.dtype))
            assert (left == left[:1]).all()
            if block:
                assert torch.equal(scales, ref_scales)
        assert torch.equal(c.q_out, want.q_out)
        if block:
            assert torch.equal(c.ko2, want.ko2) and torch.equal(c.vo2, want.vo2)


@pytest.mark.parametrize("fmt,dtype", [("i8", "bf16"), ("e4m3", "f16")])
@pytest.mark.parametrize("tokens,lens,counts", [(5, [30, 7, 65, 31, 64, 0], [5, 0, 5, 0, 0, 0]), (1, [127, 33], [0, 0]), (40, [1, 95, 32], [0, 0, 40])])
def test_requests_that_bring_nothing(fmt, dtype, tokens, lens, counts):
    """Open rows elsewhere: those of a sequence without new tokens are passed on, its codes and scales left as they were."""
    c = Append(dtype, fmt, len(lens), tokens, 4, 2, 64, 150, 32, lens, counts, norm=True, halves=True, seed=32)
    c.call()
    capi.device_sync()
    c.check()
    for b, (ln, count) in enumerate(zip(lens, counts)):
        if count == 0:
            assert (_bytes(c.ko2[b, :ln % 32]) == _bytes(c.ko[b, :ln % 32])).all() and (_bytes(c.vo2[b, :ln % 32]) == _bytes(c.vo[b, :ln % 32])).all()
            assert (c.ks[b] == 7.0).all() and (c.k[b].double() == 7.0).all() and (c.vs[b] == 7.0).all() and (c.v[b].double() == 7.0).all()


@pytest.mark.parametrize("fmt,dtype,block", [("i8", "bf16", 16), ("e4m3", "bf16", 32), ("e4m3", "f16", 64)])
def test_a_draft_taken_back_across_a_block(fmt, dtype, block):
    """A drafted run appended with its open rows elsewhere, then appended again from the open rows of before with the counts
    that were accepted: the cache of those rows alone, bit for bit, whatever blocks the draft had begun."""
    torch = _torch()
    n, tokens, cap, dim = 5, 24, 160, 64
    lens = [block - 3, block - 3, 2 * block - 1, block, 5]
    accepted = [2, 9, 1, 24, 0]
    kw = dict(dtype=dtype, fmt=fmt, n_seq=n, heads=4, kv_heads=2, dim=dim, max_seq=cap, block=block, norm=True, halves=True)

    def prompt():
        a = Append(tokens=max(lens), lens=[0] * n, counts=lens, seed=41, **kw)
        a.call(in_place=True)
        return a

    def then(a, counts, **call):
        c = Append(tokens=tokens, lens=lens, counts=counts, seed=42, **kw)
        for name in ("k", "v", "ks", "vs", "ko", "vo"):
            setattr(c, name, getattr(a, name))
        c.gains = a.gains
        c.v_new[:, 3:] *= 30  # (rejected rows that would enlarge the scales)
        c.call(**call)
        return c

    a, b = prompt(), prompt()
    then(a, [tokens] * n)                 # the draft: its open rows go elsewhere
    x = then(a, accepted, in_place=True)  # what was accepted, from the state of before
    y = then(b, accepted, in_place=True)  # as if there had been no draft
    capi.device_sync()
    assert x.lens_out.tolist() == y.lens_out.tolist() == [u + v for u, v in zip(lens, accepted)]
    for s in range(n):
        end = lens[s] + accepted[s]
        for name in ("ko", "vo"):
            assert torch.equal(_bytes(getattr(x, name)[s, :end % block]), _bytes(getattr(y, name)[s, :end % block]))
        if accepted[s] == 0:
            continue
        for name in ("k", "v"):
            assert torch.equal(_bytes(getattr(x, name)[s, :end]), _bytes(getattr(y, name)[s, :end]))
        for name in ("ks", "vs"):
            assert torch.equal(getattr(x, name)[s, :, :-(-end // block)], getattr(y, name)[s, :, :-(-end // block)])
