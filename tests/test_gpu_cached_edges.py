"""Cached-attention calls where an order of events, a range of numbers or a
limit of the machine decides the result: late value tiles beside values that
are not numbers, and what else the layouts of test_gpu_cached.py do not reach."""
import numpy as np
import pytest

from paper_2401_16757_gb300 import capi
from test_gpu_cached import SENT, _any_engine, _torch

pytestmark = pytest.mark.gpu


def _stream():
    return _torch().cuda.current_stream().cuda_stream


def _call(dtype, n, t, h, kv, d, cap, q, k, v, lens, lse=True, weights=None, **ptrs):
    """out and lse of one attention call on device tensors, beside a workspace of its own."""
    torch = _torch()
    out = torch.full((n * t, h * d), SENT, dtype=q.dtype, device="cuda")
    sums = torch.full((n, h, t), SENT, device="cuda") if lse else None
    a = capi.cached_attention(dtype, n, t, h, kv, d, cap, q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), lens=lens.data_ptr(),
                              out=out.data_ptr(), lse=sums.data_ptr() if lse else 0,
                              weights=0 if weights is None else weights.data_ptr(), **{x: y.data_ptr() for x, y in ptrs.items()})
    ws = torch.empty(max(256, capi.attention_tree_workspace(a)), dtype=torch.uint8, device="cuda")
    capi.attention_tree(a, ws.data_ptr(), ws.numel(), _stream())
    return out, sums


@pytest.mark.parametrize("tokens", [8, 24])
def test_values_that_are_not_numbers_beside_late_value_tiles(tokens):
    """Drafted values in L2, cached ones in DRAM (1 GB of them): the draft's tile is at hand while the product of the tile
    before still waits for its values.  What no infinite value reaches has the bits of a call without one, what one reaches
    is right in its other columns, on every one of many runs."""
    torch = _torch()
    n, h, kv, d, cap = 32, 32, 8, 128, 8192
    g = torch.Generator(device="cuda").manual_seed(tokens)
    k, v = (torch.empty(n, cap, kv * d, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    q = torch.empty(n * tokens, h * d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    kn, vn = (torch.empty(n * tokens, kv * d, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    lens = torch.tensor([129 + 251 * b for b in range(n)], dtype=torch.int32, device="cuda")
    par = torch.full((n, tokens), 0, dtype=torch.int32, device="cuda")  # all nodes below node 0
    par[:, 0] = -1
    clean = _call("bf16", n, tokens, h, kv, d, cap, q, k, v, lens, k_new=kn, v_new=vn, parents=par)
    bad = [tokens // 3, tokens - 1]
    for at in bad:
        vn.view(n, tokens, kv, d)[:, at, :, 5] = float("inf")
    rest = torch.ones(d, dtype=torch.bool, device="cuda")
    rest[5] = False
    want = clean[0].view(n, tokens, h, d)
    others = [i for i in range(tokens) if i not in bad]
    for _ in range(20):
        kn.mul_(1), vn.mul_(1)  # the draft is in L2
        out, lse = _call("bf16", n, tokens, h, kv, d, cap, q, k, v, lens, k_new=kn, v_new=vn, parents=par)
        out = out.view(n, tokens, h, d)
        assert torch.equal(lse, clean[1])
        assert torch.equal(out[:, others], want[:, others])
        assert not torch.any(torch.isfinite(out[:, bad][..., 5]))
        # a row added by hand in fp32 in place of two products: a rounding of the result to either side, and 2^-13 of values of up to 4
        a, b = out[:, bad][..., rest].double(), want[:, bad][..., rest].double()
        assert torch.all((a - b).abs() <= 2.0 ** -7 * b.abs() + 2.0 ** -11)
    _any_engine().sync()  # no wait gave up


@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 64), (6, 2, 128), (40, 1, 64)])
@pytest.mark.parametrize("tokens", [6, 70, 200])
@pytest.mark.parametrize("unused", [float("nan"), float("inf"), -float("inf"), 1.0])
def test_listed_rows_out_of_range_add_nothing(heads, kv, dim, tokens, unused):
    """Entries below 0 and from `tokens` on, among right ones, whatever the first and the last query row hold: the weights are
    those of the list's other entries at their places, and the entry is reported."""
    torch = _torch()
    eng = _any_engine()
    n, cap, count = 2, 300, tokens - 2
    g = torch.Generator(device="cuda").manual_seed(tokens)
    q = torch.empty(n, tokens, heads * dim, dtype=torch.float16, device="cuda").normal_(generator=g)
    k = torch.empty(n, cap, kv * dim, dtype=torch.float16, device="cuda").normal_(generator=g)
    q[:, 0], q[:, -1] = unused, unused  # in use for no entry
    lens = torch.tensor([cap, max(tokens, 130)], dtype=torch.int32, device="cuda")
    counts = torch.full((n,), count, dtype=torch.int32, device="cuda")
    rows = (torch.arange(tokens, device="cuda") + 1).clamp(max=tokens - 2).int().expand(n, tokens).contiguous()
    wrong = sorted({1, count // 2, count - 1})
    for b in range(n):
        for i, at in enumerate(wrong):
            rows[b, at] = (-1, tokens, -2 ** 31, 2 ** 31 - 1)[(i + b) % 4]
    group = heads // kv
    own = torch.arange(heads, device="cuda") // group
    lse = torch.full((n, heads, tokens), float("nan"), device="cuda")
    want = torch.zeros(n, kv, cap, dtype=torch.float64, device="cuda")
    slack = torch.zeros_like(want)
    for b in range(n):
        m = int(lens[b])
        keys = k[b, :m].double().view(m, kv, dim)[:, own]
        z0 = torch.einsum("ihd,jhd->hij", q[b, 1:-1].double().view(-1, heads, dim), keys) / dim ** 0.5
        lse[b, :, 1:-1] = torch.logsumexp(z0, -1).float()
        for i in range(count):
            r = int(rows[b, i])
            if i in wrong:
                continue
            z = z0[:, r - 1]
            seen = torch.arange(m, device="cuda") <= m - count + i
            p = torch.where(seen, torch.exp(z - lse[b, :, r, None].double()), torch.zeros((), dtype=torch.float64, device="cuda"))
            # a score's sum of dim products in fp32, a step each, and 2^x of it
            e = dim * 2.0 ** -23 * torch.einsum("hd,jhd->hj", q[b, r].double().abs().view(heads, dim), keys.abs()) / dim ** 0.5
            want[b, :, :m] += p.view(kv, group, m).sum(1)
            slack[b, :, :m] += (p * (e + 2.0 ** -20 * (1 + z.abs()))).view(kv, group, m).sum(1)
    w = torch.full((n, kv, cap), SENT, device="cuda")
    capi.attention_weights(capi.cached_attention("f16", n, tokens, heads, kv, dim, cap, q=q.data_ptr(), k=k.data_ptr(),
                                                 lens=lens.data_ptr(), counts=counts.data_ptr(), rows=rows.data_ptr(),
                                                 lse=lse.data_ptr(), weights=w.data_ptr()), _stream())
    with pytest.raises(capi.SwapnetError) as x:
        eng.sync()
    assert x.value.code == capi.ERR_INVALID_ARG
    eng.sync()
    for b in range(n):
        m = int(lens[b])
        err = (w[b, :, :m].double() - want[b, :, :m]).abs()
        assert torch.all(err <= slack[b, :, :m] + (count * group + 4) * 2.0 ** -24 * want[b, :, :m] + 2.0 ** -126)
        assert torch.all(w[b, :, m:] == SENT)


@pytest.mark.parametrize("tokens,group", [(1, 128), (3, 100)])
def test_weights_of_a_cache_whose_rows_times_heads_pass_32_bits(tokens, group):
    """Rows times the heads of a group beyond 2^31: every row gets its attention, from the first to the last."""
    torch = _torch()
    dim, length = 64, 2 ** 31 // group + 300_001
    cap = length + 5
    g = torch.Generator(device="cuda").manual_seed(group)
    k = torch.empty(cap, dim, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    q = torch.empty(tokens, group * dim, dtype=torch.bfloat16, device="cuda").normal_(0, 0.5, generator=g)
    rows = q.double().view(tokens * group, dim)
    step = 1 << 18
    last = torch.arange(tokens, device="cuda").repeat_interleave(group) + length - tokens  # a row's own cache row

    def scores(j0):
        z = rows @ k[j0:min(j0 + step, length)].double().T / dim ** 0.5
        return z.masked_fill(torch.arange(j0, j0 + z.shape[1], device="cuda") > last[:, None], -float("inf"))

    parts = torch.stack([torch.logsumexp(scores(j0), -1) for j0 in range(0, length, step)])
    lse = torch.logsumexp(parts, 0).float()  # [query, head]
    lens = torch.tensor([length], dtype=torch.int32, device="cuda")
    stats = lse.view(tokens, group).T.contiguous()
    w = torch.full((cap,), SENT, device="cuda")
    capi.attention_weights(capi.cached_attention("bf16", 1, tokens, group, 1, dim, cap, q=q.data_ptr(), k=k.data_ptr(),
                                                 lens=lens.data_ptr(), lse=stats.data_ptr(), weights=w.data_ptr()), _stream())
    assert torch.all(w[length:] == SENT)
    norm = float(rows.abs().sum(1).max()) * float(k.abs().max()) / dim ** 0.5  # of any score's products
    for j0 in range(0, length, step):
        p = torch.exp(scores(j0) - lse[:, None].double())
        want = p.sum(0)
        # a score's sum of dim products in fp32, a step each; 2^x of numbers of up to 64; the sum over the rows
        e = dim * 2.0 ** -23 * norm + 2.0 ** -16 + tokens * group * 2.0 ** -24
        assert torch.all((w[j0:j0 + p.shape[1]].double() - want).abs() <= e * want), j0


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,kv,dim,length,draft", [
    (1, 8, 128, 300, False), (1, 8, 128, 8000, False), (1, 1, 64, 131000, False), (16, 2, 64, 5000, True), (7, 8, 128, 100, True),
    (24, 8, 128, 700, True), (20, 2, 64, 3900, False), (64, 4, 64, 131000, True), (100, 2, 128, 9000, True), (128, 8, 128, 9000, False)])
@pytest.mark.parametrize("below", [12, 20, 24, 26, 28, 30])
@pytest.mark.parametrize("first", [True, False])
def test_a_dominant_key_without_a_value_leaves_the_rest(dtype, tokens, kv, dim, length, draft, below, first):
    """One key takes all but 2^-below of a row's attention per other key, and its values are 0: the output is the other keys',
    to the type's rounding, whether the dominant key comes first or among the last."""
    torch = _torch()
    n, h, cap = 1, kv, length + 9
    g = torch.Generator(device="cuda").manual_seed(length + below)
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    # scores: the first element's product alone
    q, k = torch.zeros(tokens, h, dim, dtype=dt, device="cuda"), torch.zeros(n, cap, kv, dim, dtype=dt, device="cuda")
    q[..., 0] = 1.0
    k[..., 0] = torch.empty(n, cap, kv, device="cuda").uniform_(-0.5, 0.5, generator=g).to(dt)
    at = 0 if first else length - tokens - 1
    k[:, at, :, 0] = below * np.log(2.0)
    v = torch.empty(n, cap, kv, dim, device="cuda").uniform_(0.5, 1.5, generator=g).to(dt)
    v[:, at] = 0
    kn = torch.zeros(tokens, kv, dim, dtype=dt, device="cuda")
    vn = torch.empty(tokens, kv, dim, device="cuda").uniform_(0.5, 1.5, generator=g).to(dt)
    a = dict(k_new=kn, v_new=vn) if draft else {}
    lens = torch.tensor([length], dtype=torch.int32, device="cuda")
    out = torch.empty(tokens, h, dim, dtype=dt, device="cuda")
    lse = torch.empty(1, h, tokens, device="cuda")
    c = capi.cached_attention(dtype, n, tokens, h, kv, dim, cap, q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), lens=lens.data_ptr(),
                              out=out.data_ptr(), lse=lse.data_ptr(), scale=1.0, **{x: y.data_ptr() for x, y in a.items()})
    ws = torch.empty(max(256, capi.attention_tree_workspace(c)), dtype=torch.uint8, device="cuda")
    capi.attention_tree(c, ws.data_ptr(), ws.numel(), _stream())
    z = k[0, :length, :, 0].double()  # [row, head]
    e = torch.exp(z)
    sums, vals = torch.cumsum(e, 0), torch.cumsum(e[..., None] * v[0, :length].double(), 0)
    if draft:  # a chain
        sums, vals = sums[-1:].expand(tokens, -1), vals[-1:].expand(tokens, -1, -1)
        sums = sums + torch.cumsum(torch.ones(tokens, kv, dtype=torch.float64, device="cuda"), 0)
        vals = vals + torch.cumsum(vn.double(), 0)
    else:
        sums, vals = sums[length - tokens:], vals[length - tokens:]
    ref = vals / sums[..., None]
    # 2^x of numbers of up to 31 (fp32 scores: exact products of a single element); the sums over the keys, as they
    # are added in tiles of 16 and more; the parts of p; a rounding of the output, half a step at least
    keys = length + tokens
    half = torch.finfo(dt).eps / 2
    rel = 2 * (32 * 2.0 ** -23 + 2.0 ** -21) + 2 * (keys / 16 + 40) * 2.0 ** -23 + 2.0 ** -17
    tol = (half + rel) * ref
    if dtype == "f16":
        few = tokens * h // kv <= 16
        # half of fp16's least step for every key's p, which ends at 2^15, 2^7 or 2^12; values of up to 1.5
        lost = keys * 2.0 ** -40 if few else min(keys, 31 * 128 + 128) * 2.0 ** -32 + keys * 2.0 ** -37
        tol = tol + 1.5 * lost + 2.0 ** -25
    err = (out.double() - ref).abs()
    assert torch.all(err <= tol), float((err / tol).max())
    assert torch.all((lse[0].T.double() - torch.log(sums)).abs() <= rel + 2.0 ** -23 * torch.log(sums).abs())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,length,dim", [(1, 16, 128), (1, 300, 64), (1, 9000, 128), (16, 300, 64), (5, 9000, 64)])
def test_probabilities_of_few_rows_keep_their_bits(dtype, tokens, length, dim):
    """Two keys whose probabilities differ by 2^-12 and whose values cancel: the difference is right to fp32's steps."""
    torch = _torch()
    h, cap = 64, length + 16
    g = torch.Generator(device="cuda").manual_seed(length + tokens)
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    q, k = torch.zeros(tokens, h, dim, dtype=dt, device="cuda"), torch.zeros(1, cap, h, dim, dtype=dt, device="cuda")
    v = torch.zeros(1, cap, h, dim, dtype=dt, device="cuda")
    q[..., 0], q[..., 1], q[..., 2] = 1.0, 2.0 ** -12, 1.0
    k[:, :, :, 2] = -64.0  # nothing
    k[:, 0, :, 2] = 0.0    # the largest score, 0
    a, b = (3, 9) if length == 16 else (3, length - tokens - 2)
    c = -torch.empty(h, device="cuda").uniform_(0.3, 0.9, generator=g).to(dt)
    for at, more, value in ((a, 0.0, 1.0), (b, 1.0, -1.0)):
        k[0, at, :, 0], k[0, at, :, 1], k[0, at, :, 2] = c, more, 0.0
        v[0, at] = value
    v[0, a, :, 1::2] = -v[0, a, :, 1::2]
    v[0, b, :, 1::2] = -v[0, b, :, 1::2]
    lens = torch.tensor([length], dtype=torch.int32, device="cuda")
    out = torch.empty(tokens, h, dim, dtype=dt, device="cuda")
    args = capi.cached_attention(dtype, 1, tokens, h, h, dim, cap, q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(),
                                 lens=lens.data_ptr(), out=out.data_ptr(), scale=1.0)
    ws = torch.empty(max(256, capi.attention_tree_workspace(args)), dtype=torch.uint8, device="cuda")
    capi.attention_tree(args, ws.data_ptr(), ws.numel(), _stream())
    pa, pb = torch.exp(c.double()), torch.exp(c.double() + 2.0 ** -12)
    ref = ((pa - pb) / (1 + pa + pb))[None, :, None] * torch.tensor([1.0, -1.0], dtype=torch.float64, device="cuda").repeat(dim // 2)
    # 2^x to 2^-22 and its argument to 2^-24 of at most 1.3; eight steps of the sums of products; the quotient; the rounding
    half = torch.finfo(dt).eps / 2
    tol = half * ref.abs() + (((pa + pb) * (2.0 ** -22 + 1.3 * 2.0 ** -24) + 8 * 2.0 ** -23 * pb) / (1 + pa + pb))[None, :, None]
    if dtype == "f16":  # 22 bits of each p, and half of the type's least step
        tol = tol + ((pa + pb) * 2.0 ** -23 / (1 + pa + pb))[None, :, None] + 2.0 ** -25
    err = (out.double() - ref).abs()
    assert torch.all(err <= tol), float((err / tol).max())


def test_errors_are_reported_without_an_engine():
    """Each call's value out of range is reported once by the device, without an engine; an engine's next sync is clean."""
    torch = _torch()
    capi.device_sync()
    n, t, h, d, cap = 2, 3, 2, 64, 20
    q, k = torch.zeros(n * t, h * d, dtype=torch.float16, device="cuda"), torch.zeros(n, cap, h * d, dtype=torch.float16, device="cuda")
    out, lse, w = torch.zeros_like(q), torch.zeros(n, h, t, device="cuda"), torch.zeros(n, h, cap, device="cuda")
    bad = torch.tensor([5, cap + 1], dtype=torch.int32, device="cuda")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    ids, tgt, path, acc, nxt, lo, kept = i32(n, t), i32(n, t), i32(n, t), i32(n), i32(n), i32(n), i32(n, h, 4)
    args = capi.cached_attention("f16", n, t, h, h, d, cap, q=q.data_ptr(), k=k.data_ptr(), v=k.data_ptr(), lens=bad.data_ptr(),
                                 out=out.data_ptr(), lse=lse.data_ptr(), weights=w.data_ptr())
    ws = torch.empty(max(256, capi.attention_tree_workspace(args)), dtype=torch.uint8, device="cuda")
    to = [torch.zeros(n, cap, h * d, dtype=torch.float16, device="cuda") for _ in range(2)] + [torch.zeros_like(w)]
    calls = [
        lambda: capi.attention_tree(args, ws.data_ptr(), ws.numel(), _stream()),
        lambda: capi.attention_weights(args, _stream()),
        lambda: capi.tree_accept("f16", n, t, h * d, cap, ids=ids.data_ptr(), targets=tgt.data_ptr(), lens=bad.data_ptr(),
                                 caches=[to[0].data_ptr()], drafts=[q.data_ptr()], path=path.data_ptr(), accepted=acc.data_ptr(),
                                 next=nxt.data_ptr(), lens_out=lo.data_ptr(), stream=_stream()),
        lambda: capi.cache_evict("f16", n, h, d, cap, 4, 1, 1, k=k.data_ptr(), v=k.data_ptr(), weights=w.data_ptr(), lens=bad.data_ptr(),
                                 k_out=to[0].data_ptr(), v_out=to[1].data_ptr(), weights_out=to[2].data_ptr(), kept=kept.data_ptr(),
                                 lens_out=lo.data_ptr(), stream=_stream()),
    ]
    eng = _any_engine()
    for call in calls:
        call()
        with pytest.raises(capi.SwapnetError) as x:
            capi.device_sync()
        assert x.value.code == capi.ERR_INVALID_ARG and "length" in str(x.value)
        capi.device_sync()
        eng.sync()


@pytest.mark.parametrize("weights", [False, True])
def test_a_decoder_accepts_what_the_cache_has_room_for(weights):
    """Two rows free: a child that the model chose is accepted behind its parent. One row free: the same path changes
    nothing and is reported, a path of one node is accepted."""
    import synth
    from test_gpu_decode_cache import CFG, Engines
    e = Engines({"prefill": (30, False), "tree": (4, True)}, weights=weights)
    e.run("prefill", synth.gen.model_input(synth.arch.llm(tokens=30, **CFG)).reshape(-1))
    rows, parents = CFG["max_seq"], [-1, 0, 0, 0]

    def choice():
        """The model's choice at node 0, which sees the cache and itself."""
        return int(e.run("tree", [1, 2, 3, 4], parents)[1][0])

    def state():
        return e.caches("tree").copy(), e.weights("tree").copy() if weights else np.zeros(0)

    e.header[0] = rows - 2
    t = choice()
    child = 5 if t != 5 else 6
    _, tok = e.run("tree", [1, child, t, 7], parents)
    assert int(tok[0]) == t
    before = state()
    path, n, nxt = e.accept("tree")
    assert path == [0, 2] and n == 2 and nxt == int(tok[2]) and int(e.header[0]) == rows
    after = state()
    assert np.array_equal(after[0][:, :, :rows - 2], before[0][:, :, :rows - 2]) and not np.array_equal(after[0], before[0])
    if weights:  # two queries' attention in every layer and head
        assert np.all(np.abs(after[1].sum(-1) - before[1].sum(-1) - 2) <= 1e-3)
    e.header[0] = rows - 1
    t = choice()
    e.run("tree", [1, child if child != t else 9, t, 7], parents)
    before = state()
    with pytest.raises(capi.SwapnetError) as x:
        e.accept("tree")
    assert x.value.code == capi.ERR_INVALID_ARG
    assert int(e.header[0]) == rows - 1 and int(e.header[3]) == 0
    assert all(np.array_equal(a, b) for a, b in zip(state(), before))
    others = [i for i in range(20, 30) if i != t][:3]
    _, tok = e.run("tree", [1] + others, parents)
    path, n, nxt = e.accept("tree")
    assert path == [0] and n == 1 and nxt == t == int(tok[0]) and int(e.header[0]) == rows


def test_token_ids_off_their_four_bytes_are_refused():
    from test_gpu_decode_cache import Engines
    eng = Engines({"tree": (4, True)}).e["tree"][2]
    for ids, targets in ((18, 16), (16, 17)):
        with pytest.raises(capi.SwapnetError) as x:
            eng.tree_accept(ids, targets)
        assert x.value.code == capi.ERR_MISALIGNED


@pytest.mark.parametrize("dtype,tokens,heads,kv,dim", [("bf16", 6, 8, 2, 128), ("f16", 40, 8, 8, 64), ("bf16", 100, 4, 2, 128)])
def test_a_captured_chain_of_the_calls_follows_its_inputs(dtype, tokens, heads, kv, dim):
    """Verification, acceptance, weighing and eviction captured into one graph: replays on other lengths, trees and tokens give
    the bits of the same calls made one by one."""
    torch = _torch()
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    n, cap, keep = 5, 700, 150
    g = torch.Generator(device="cuda").manual_seed(tokens)
    rng = np.random.default_rng(tokens)

    def normal(*shape):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(generator=g)

    def inputs():
        par = np.full((n, tokens), -1, dtype=np.int32)
        for i in range(1, tokens):
            par[:, i] = rng.integers(max(0, i - 4), i, size=n)
        i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()  # noqa: E731
        return dict(k=normal(n, cap, kv * dim), v=normal(n, cap, kv * dim), q=normal(n * tokens, heads * dim),
                    kn=normal(n * tokens, kv * dim), vn=normal(n * tokens, kv * dim),
                    w=torch.empty(n, kv, cap, device="cuda").uniform_(0, 2, generator=g), par=i32(par),
                    lens=i32(rng.integers(0, cap - tokens, size=n)), counts=i32(rng.integers(1, tokens + 1, size=n)),
                    ids=i32(rng.integers(0, 3, size=(n, tokens))), tgt=i32(rng.integers(0, 3, size=(n, tokens))))

    sets = [inputs() for _ in range(3)]
    s = {x: y.clone() for x, y in sets[0].items()}  # the buffers that the calls use
    out, lse = torch.empty(n * tokens, heads * dim, dtype=dt, device="cuda"), torch.empty(n, heads, tokens, device="cuda")
    i32 = lambda *shape: torch.empty(*shape, dtype=torch.int32, device="cuda")  # noqa: E731
    path, acc, nxt, lens2, lens3, kept = i32(n, tokens), i32(n), i32(n), i32(n), i32(n), i32(n, kv, keep)
    p = {x: y.data_ptr() for x, y in s.items()}
    a = capi.cached_attention(dtype, n, tokens, heads, kv, dim, cap, q=p["q"], k=p["k"], v=p["v"], lens=p["lens"], counts=p["counts"],
                              parents=p["par"], k_new=p["kn"], v_new=p["vn"], out=out.data_ptr(), lse=lse.data_ptr())
    w = capi.cached_attention(dtype, n, tokens, heads, kv, dim, cap, q=p["q"], k=p["k"], lens=lens2.data_ptr(), counts=acc.data_ptr(),
                              rows=path.data_ptr(), lse=lse.data_ptr(), weights_in=p["w"], weights=p["w"])
    ws = torch.empty(max(256, capi.attention_tree_workspace(a)), dtype=torch.uint8, device="cuda")
    results = [out, lse, path, acc, nxt, lens2, lens3, kept, s["k"], s["v"], s["w"]]

    def chain():
        capi.attention_tree(a, ws.data_ptr(), ws.numel(), _stream())
        capi.tree_accept(dtype, n, tokens, kv * dim, cap, ids=p["ids"], targets=p["tgt"], parents=p["par"], counts=p["counts"],
                         lens=p["lens"], caches=[p["k"], p["v"]], drafts=[p["kn"], p["vn"]], path=path.data_ptr(),
                         accepted=acc.data_ptr(), next=nxt.data_ptr(), lens_out=lens2.data_ptr(), stream=_stream())
        capi.attention_weights(w, _stream())
        capi.cache_evict(dtype, n, kv, dim, cap, keep, 20, 2, k=p["k"], v=p["v"], weights=p["w"], lens=lens2.data_ptr(), k_out=p["k"],
                         v_out=p["v"], weights_out=p["w"], kept=kept.data_ptr(), lens_out=lens3.data_ptr(), stream=_stream())

    def reset(i):
        for x, y in sets[i].items():
            s[x].copy_(y)
        for x in results[:8]:
            x.fill_(7)

    alone = []
    for i in range(3):
        reset(i)
        chain()
        alone.append([x.clone() for x in results])
    graph = torch.cuda.CUDAGraph()
    reset(0)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        chain()
    for i in (2, 0, 1, 2):
        reset(i)
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(results, alone[i])), i
    capi.device_sync()
    assert max(int(x[3].max()) for x in alone) > 1 and min(int(x[6].min()) for x in alone) < keep
