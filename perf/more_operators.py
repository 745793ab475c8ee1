"""A decoder's key-value cache held in 8 bits: rows appended to it (with the
norms of queries and keys and the position rotation in the same pass) and the
attention that reads it.

The cache competes with the swapped weights' arena for a memory budget; in 8
bits, with a scale for each block of rows and head, it takes half the bytes.

A case names an operator and its sizes; prepare() gives what a program has in
hand before the call, run() is one call through the C ABI's Python binding
(own) or the same from elementary torch operations, exact() the same result in
64 bits.
"""
import math

import numpy as np
import torch

own = False

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
TOP = {"i8": 127.0, "e4m3": 448.0}  # the largest code


def listed():
    return [
        # the smallest call: a decode step of one request, a small block of rows (latency)
        dict(name="append_small", kind="append", dtype="bf16", cache="e4m3", n_seq=1, tokens=1, heads=8, kv_heads=8,
             dim=128, length=100, capacity=160, block=16, norm=False, halves=False, rope_dim=128, axes=1, far=0),
        # a decode step of many requests of a model with norms of queries and keys
        dict(name="append_decode", kind="append", dtype="bf16", cache="e4m3", n_seq=64, tokens=1, heads=32, kv_heads=8,
             dim=128, length=2000, capacity=2048, block=64, norm=True, halves=True, rope_dim=128, axes=1, far=0),
        # the 512-token prompt of the 7B-shaped decoder into an empty cache
        dict(name="append_prompt", kind="append", dtype="bf16", cache="e4m3", n_seq=1, tokens=512, heads=32, kv_heads=32,
             dim=128, length=0, capacity=544, block=32, norm=False, halves=False, rope_dim=128, axes=1, far=0),
        # prompts with images or video: positions of three axes, behind what is cached
        dict(name="append_video", kind="append", dtype="f16", cache="e4m3", n_seq=4, tokens=3001, heads=16, kv_heads=2,
             dim=128, length=77, capacity=4000, block=128, norm=True, halves=True, rope_dim=128, axes=3, far=0),
        # a cache that stays in 16 bits, half of a narrow head rotated, far positions
        dict(name="append_rows16", kind="append", dtype="f16", cache="f16", n_seq=16, tokens=700, heads=12, kv_heads=4,
             dim=64, length=100, capacity=1024, block=0, norm=True, halves=False, rope_dim=32, axes=1, far=1000000),
        # a batch's 16-bit cache (keys rotated before) put into 8 bits
        dict(name="append_convert", kind="append", dtype="bf16", cache="i8", n_seq=8, tokens=4096, heads=0, kv_heads=8,
             dim=128, length=0, capacity=4200, block=64, norm=False, halves=False, rope_dim=0, axes=1, far=0),
        # the smallest call: a decode step of one request on a hundred rows (latency)
        dict(name="attend_small", kind="attend", dtype="bf16", cache="i8", n_seq=1, tokens=1, heads=8, kv_heads=8,
             dim=128, length=100, capacity=160, block=16),
        # a decode step of the 7B-shaped decoder, its cache of 544 rows nearly full
        dict(name="attend_7b", kind="attend", dtype="bf16", cache="e4m3", n_seq=1, tokens=1, heads=32, kv_heads=32,
             dim=128, length=543, capacity=544, block=32),
        # single tokens of many requests with long histories: the largest call
        dict(name="attend_decode", kind="attend", dtype="bf16", cache="i8", n_seq=64, tokens=1, heads=32, kv_heads=8,
             dim=128, length=16384, capacity=16400, block=64),
        # one request with a very long history, three tokens, 64-wide heads
        dict(name="attend_long", kind="attend", dtype="f16", cache="e4m3", n_seq=1, tokens=3, heads=16, kv_heads=4,
             dim=64, length=131001, capacity=131072, block=128),
        # drafted runs of many requests verified
        dict(name="attend_draft", kind="attend", dtype="bf16", cache="e4m3", n_seq=32, tokens=8, heads=32, kv_heads=8,
             dim=128, length=8000, capacity=8192, block=64),
        # a chunk of a long prompt behind what is cached
        dict(name="attend_chunk", kind="attend", dtype="f16", cache="i8", n_seq=2, tokens=1000, heads=32, kv_heads=8,
             dim=128, length=4096, capacity=4100, block=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend"])
    heads, kv = rng.choice([(8, 8), (32, 32), (32, 8), (16, 2), (12, 4), (6, 1)])
    c = dict(kind=kind, dtype=rng.choice(["f16", "bf16"]), n_seq=_log(rng, 1, 64), heads=heads, kv_heads=kv,
             dim=rng.choice([64, 128]), block=rng.choice([16, 32, 64, 128]))
    if kind == "append":
        c["cache"] = rng.choice(["e4m3", "e4m3", "e4m3", "i8", c["dtype"]])
        most = max(1, (1 << 26) // (c["n_seq"] * (heads + 2 * kv) * c["dim"]))
        c["tokens"] = min(most, rng.choice([1, _log(rng, 2, 4096)]))
        c["length"] = _log(rng, 1, max(2, min(4096, (1 << 18) // (c["n_seq"] * kv)))) - 1
        c["capacity"] = c["length"] + c["tokens"] + rng.choice([0, 1, 13, 64])
        c.update(norm=rng.random() < 0.5, halves=rng.random() < 0.5, rope_dim=rng.choice([c["dim"], c["dim"] // 2]),
                 axes=rng.choice([1, 1, 3]), far=rng.choice([0, 0, _log(rng, 1000, 4000000)]))
        if c["cache"] == "i8":  # rows of another cache, rotated before
            c.update(heads=0, norm=False, halves=False, rope_dim=0, axes=1, far=0)
        if c["cache"] == c["dtype"]:
            c["block"] = 0
        return c
    c["cache"] = rng.choice(["e4m3", "i8"])
    c["tokens"] = rng.choice([1, _log(rng, 2, 8), _log(rng, 9, 1000)])
    most = max(64, (1 << 22) // (c["n_seq"] * kv))
    if c["tokens"] > 8:  # products within the largest listed case's
        c["n_seq"] = min(c["n_seq"], max(1, (1 << 27) // (heads * c["tokens"] ** 2)))
        most = min(most, max(64, (1 << 27) // (c["n_seq"] * heads * c["tokens"])))
    c["length"] = max(c["tokens"], _log(rng, 17, min(most, 131000)))
    c["capacity"] = c["length"] + rng.choice([0, 1, 13, 64, 300])
    return c


# ------------------------------------------------------------------ inputs
def _lens(c):
    """Cached rows of each request: the longest first, the others down to half of that; in a batch the last one's
    place is not in use."""
    n, low = c["length"], (c["length"] + 1) // 2
    lens = [n - b * 7919 % (n - low + 1) for b in range(c["n_seq"])]
    if c["kind"] == "attend" and c["n_seq"] >= 6:
        lens[-1] = 0
    return lens


def _counts(c):
    """Tokens of each request."""
    t = c["tokens"]
    counts = [t - b * 3 % (t // 2 + 1) for b in range(c["n_seq"])]
    if c["kind"] == "append" and c["n_seq"] >= 6:
        counts[-1] = 0
    return counts


def _sections(c):
    """Pairs that each position axis turns: time, height, width."""
    pairs = c["rope_dim"] // 2
    return (pairs, 0, 0) if c["axes"] == 1 else (pairs - 2 * (3 * pairs // 8), 3 * pairs // 8, 3 * pairs // 8)


def _blocks(c):
    return -(-c["capacity"] // c["block"])


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TORCH[c["dtype"]]
    n, t, kv, d, cap = c["n_seq"], c["tokens"], c["kv_heads"], c["dim"], c["capacity"]

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(0, std, generator=g)

    def whole(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    def uniform(*shape):
        return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(0, 1, generator=g)

    def codes():
        x = torch.empty(n, cap, kv, d, dtype=torch.float16, device="cuda").normal_(0, TOP[c["cache"]] / 4.2, generator=g)
        return x.clamp_(-TOP[c["cache"]], TOP[c["cache"]]).round_().to(TORCH[c["cache"]])

    def scales(std):  # standard deviations around `std`
        return torch.exp(0.5 * (2 * uniform(n, kv, _blocks(c)) - 1)) * (std * 4.2 / TOP[c["cache"]])

    s = dict(case=c, lens=whole(_lens(c)), counts=whole(_counts(c)))
    if c["kind"] == "attend":
        s["q"] = normal(n, t, c["heads"], d, std=2.0)
        s["k"], s["v"] = codes(), codes()
        s["k_scale"], s["v_scale"] = scales(1.0), scales(1.0)
        s["out"] = torch.zeros(n, t, c["heads"], d, dtype=dt, device="cuda")
        s["lse"] = torch.zeros(n, c["heads"], t, device="cuda")
        return s
    # projections: a key's channels differ in size, as trained ones' do
    s["k_new"] = normal(n, t, kv, d) * torch.exp(uniform(d) * 2 - 1).to(dt)
    s["v_new"] = normal(n, t, kv, d)
    s["k"], s["v"] = (torch.zeros(n, cap, kv, d, dtype=dt, device="cuda").to(TORCH[c["cache"]]) for _ in range(2))
    s["lens_out"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    if c["heads"]:
        s["q"] = normal(n, t, c["heads"], d, std=2.0)
        s["q_out"] = torch.zeros(n, t, c["heads"], d, dtype=dt, device="cuda")
    if c["norm"]:
        s["q_gain"], s["k_gain"] = (1 + 0.2 * normal(d)), (1 + 0.2 * normal(d))
    if c["axes"] == 3:  # frames of an image or a video: time, row, column
        at = s["lens"][:, None] + torch.arange(t, device="cuda", dtype=torch.int32) + c["far"]
        s["positions"] = torch.stack([at // 64, at // 8 % 64, at % 64 * 3]).contiguous()
    elif c["far"]:
        s["positions"] = (s["lens"][:, None] + torch.arange(t, device="cuda", dtype=torch.int32) + c["far"])[None].contiguous()
    if c["block"]:
        s["k_scale"], s["v_scale"] = torch.zeros(n, kv, _blocks(c), device="cuda"), torch.zeros(n, kv, _blocks(c), device="cuda")
        # the last block's rows so far, in 16 bits
        s["k_open"], s["v_open"] = normal(n, c["block"], kv, d), normal(n, c["block"], kv, d)
        s["k_open_out"], s["v_open_out"] = torch.zeros_like(s["k_open"]), torch.zeros_like(s["v_open"])
    return s


# -------------------------------------------------------------- plain forms
EPS, THETA = 1e-6, 10000.0


def _ready(s, x, gain):
    """Rows [n, t, heads, d] of queries or keys: norm of each head, then the rotation, rounded to the storage type."""
    c = s["case"]
    y = x.float()
    if c["norm"]:
        y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + EPS) * gain.float()
    r = c["rope_dim"]
    if r:
        t = c["tokens"]
        pos = s["positions"] if "positions" in s else (s["lens"][:, None] + torch.arange(t, device="cuda"))[None]
        axis = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(_sections(c), device="cuda"), output_size=r // 2)
        freq = THETA ** (-2.0 * torch.arange(r // 2, device="cuda", dtype=torch.float64) / r)
        angle = pos[axis].permute(1, 2, 0).double() * freq  # [n, t, pairs]
        cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
        a, b = (y[..., : r // 2], y[..., r // 2: r]) if c["halves"] else (y[..., 0:r:2], y[..., 1:r:2])
        u, w = a * cos - b * sin, b * cos + a * sin
        turned = torch.cat([u, w], dim=-1) if c["halves"] else torch.stack([u, w], dim=-1).flatten(-2)
        y = torch.cat([turned, y[..., r:]], dim=-1)
    return y.to(x.dtype)


def _quantise(c, rows, valid):
    """Codes (as bytes) and scales of rows [n, blocks, block, kv, d]; valid [n, blocks, block]."""
    x = rows.float().masked_fill(~valid[..., None, None], 0)
    most = x.abs().amax(dim=(2, 4))  # [n, blocks, kv]
    top = torch.full_like(most, TOP[c["cache"]])  # (a tensor: a quotient by a number is a product with its reciprocal)
    if c["cache"] == "i8":
        scale = (most / top).clamp(min=2.0 ** -100)
        code = torch.round(x / scale[:, :, None, :, None]).to(torch.int8)
    else:  # the least power of two that keeps the largest value within the codes
        m, e = torch.frexp(most / top)
        scale = torch.ldexp(torch.ones_like(most), torch.where(m > 0.5, e, e - 1)).clamp(min=2.0 ** -100)
        scale = torch.where(most > 0, scale, torch.full_like(scale, 2.0 ** -100))
        code = (x / scale[:, :, None, :, None]).to(torch.float8_e4m3fn)
    return code.view(torch.uint8), scale.permute(0, 2, 1)


def _plain_append(s):
    c = s["case"]
    n, t, b, d, kv = c["n_seq"], c["tokens"], c["block"], c["dim"], c["kv_heads"]
    lens, counts = s["lens"].long(), s["counts"].long()
    used = torch.arange(t, device="cuda") < counts[:, None]
    got = []
    if c["heads"]:
        got.append(torch.where(used[:, :, None, None], _ready(s, s["q"], s.get("q_gain")), s["q_out"]))
    seq = torch.arange(n, device="cuda")[:, None]
    new = [_ready(s, s["k_new"], s.get("k_gain")), s["v_new"]]
    if not b:
        at = (lens[:, None] + torch.arange(t, device="cuda"))[used]
        for cache, rows in zip((s["k"], s["v"]), new):
            cache[seq.expand(-1, t)[used], at] = rows[used]
        return got + [s["k"], s["v"], s["lens_out"].copy_(s["lens"] + s["counts"])]
    first, end = lens // b, lens + counts  # the blocks from the one that is open on
    nb = (t + 2 * b - 2) // b
    row = first[:, None] * b + torch.arange(nb * b, device="cuda")  # [n, rows]
    held = row < end[:, None]
    valid = held & (counts > 0)[:, None]
    old = row < lens[:, None]
    tail = (end // b)[:, None]  # the block that stays open
    staged = held & (row // b == tail)
    for rows, cache, scales, opened, opened_out in (
            (new[0], s["k"], s["k_scale"], s["k_open"], s["k_open_out"]),
            (new[1], s["v"], s["v_scale"], s["v_open"], s["v_open_out"])):
        whole = torch.where(old[:, :, None, None], opened[seq, row % b], rows[seq, (row - lens[:, None]).clamp(0, t - 1)])
        code, scale = _quantise(c, whole.view(n, nb, b, kv, d), valid.view(n, nb, b))
        at, of = row[valid], seq.expand_as(row)[valid]
        cache.view(torch.uint8)[of, at] = code.reshape(n, nb * b, kv, d)[valid]
        has = valid.view(n, nb, b)[:, :, 0]
        which = (first[:, None] + torch.arange(nb, device="cuda"))[has]
        scales[seq.expand(-1, nb)[has], :, which] = scale.permute(0, 2, 1)[has]
        opened_out[seq.expand_as(row)[staged], (row % b)[staged]] = whole[staged]
    return got + [s["k"], s["v"], s["k_scale"], s["v_scale"], s["k_open_out"], s["v_open_out"],
                  s["lens_out"].copy_(s["lens"] + s["counts"])]


def _plain_attend(s):
    c = s["case"]
    n, t, h, kv, d, cap, b = (c[x] for x in ("n_seq", "tokens", "heads", "kv_heads", "dim", "capacity", "block"))

    def values(code, scale):  # [n, kv, cap, d] in 32 bits
        rows = torch.repeat_interleave(scale, b, dim=2)[:, :, :cap, None]
        return code.permute(0, 2, 1, 3).float() * rows

    lens, counts = s["lens"].long(), s["counts"].long()
    j, i = torch.arange(cap, device="cuda"), torch.arange(t, device="cuda")
    last = lens[:, None] - counts[:, None] + i
    seen = (j <= last[:, :, None]) & (j < lens[:, None, None])
    q = s["q"].float().view(n, t, kv, h // kv, d).permute(0, 2, 3, 1, 4).reshape(n, kv, h // kv * t, d)
    x = torch.matmul(q, values(s["k"], s["k_scale"]).transpose(2, 3)).view(n, kv, h // kv, t, cap) / math.sqrt(d)
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    del x
    l = p.sum(dim=-1, keepdim=True)
    lse = (m + torch.log(l)).view(n, h, t)
    p = p / torch.where(l > 0, l, torch.ones_like(l))
    o = torch.matmul(p.view(n, kv, -1, cap), values(s["v"], s["v_scale"]))
    out = o.view(n, kv, h // kv, t, d).permute(0, 3, 1, 2, 4).reshape(n, t, h, d).to(s["q"].dtype)
    used = i < counts[:, None]
    return [out.masked_fill(~used[:, :, None, None], 0), lse.masked_fill(~used[:, None, :], 0)]


def run(state):
    s = state
    c = s["case"]
    if not own:
        return _plain_append(s) if c["kind"] == "append" else _plain_attend(s)
    from paper_2401_16757_gb300 import capi

    stream = torch.cuda.current_stream().cuda_stream

    def at(name):
        return s[name].data_ptr() if name in s else 0

    if c["kind"] == "append":
        capi.cache_append(
            c["dtype"], c["cache"], c["n_seq"], c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["capacity"],
            k_new=at("k_new"), v_new=at("v_new"), lens=at("lens"), k=at("k"), v=at("v"), q=at("q"), q_out=at("q_out"),
            counts=at("counts"), positions=at("positions"), q_gain=at("q_gain"), k_gain=at("k_gain"), k_scale=at("k_scale"),
            v_scale=at("v_scale"), k_open=at("k_open"), v_open=at("v_open"), k_open_out=at("k_open_out"),
            v_open_out=at("v_open_out"), lens_out=at("lens_out"), block=c["block"], rope_dim=c["rope_dim"],
            theta=THETA if c["rope_dim"] else 0.0, halves=c["halves"], sections=_sections(c), eps=EPS, stream=stream)
        got = [s["q_out"]] if c["heads"] else []
        if c["block"]:
            return got + [s[x] for x in ("k", "v", "k_scale", "v_scale", "k_open_out", "v_open_out", "lens_out")]
        return got + [s["k"], s["v"], s["lens_out"]]
    args = capi.quantized_attention(
        c["dtype"], c["cache"], c["n_seq"], c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["capacity"], c["block"],
        q=at("q"), k=at("k"), v=at("v"), k_scale=at("k_scale"), v_scale=at("v_scale"), lens=at("lens"), counts=at("counts"),
        out=at("out"), lse=at("lse"))
    space = torch.empty(capi.attention_quantized_workspace(args), dtype=torch.uint8, device="cuda")
    capi.attention_quantized(args, space.data_ptr(), space.numel(), stream)
    return [s["out"], s["lse"]]


# ------------------------------------------------------------ what it takes
def work(case):
    """Bytes: the rows and scales in use, queries, outputs, once each. Operations: two per product and sum of every
    (query, visible row) pair, for the scores and for the values."""
    c = case
    lens, counts = _lens(c), _counts(c)
    d, kv, h, b = c["dim"], c["kv_heads"], c["heads"], c["block"]
    if c["kind"] == "attend":
        pairs = sum(max(0, x * (y - (x - 1) / 2)) for x, y in zip(counts, lens))
        rows = sum(lens)
        return dict(bytes=rows * kv * 2 * d + 8 * kv * sum(-(-x // b) for x in lens) + sum(counts) * h * (4 * d + 4) + 8 * len(lens),
                    flops=4 * d * h * pairs)
    new = sum(counts)
    byte = new * (4 * h * d + 4 * kv * d) + 12 * len(lens) + (4 * c["axes"] * new if c["far"] or c["axes"] == 3 else 0)
    if not b:
        return dict(bytes=byte + new * 4 * kv * d, flops=0)
    opened = sum(y % b for x, y in zip(counts, lens) if x)  # rows of the open blocks, read again
    left = sum((x + y) % b for x, y in zip(counts, lens))
    touched = sum(-(-(x + y) // b) - y // b for x, y in zip(counts, lens) if x)
    return dict(bytes=byte + 2 * kv * d * (2 * opened + new + opened + 2 * left) + 8 * kv * touched, flops=0)


# --------------------------------------------------------------- in 64 bits
def exact(case, seed):
    return (_exact_append if case["kind"] == "append" else _exact_attend)(case, prepare(case, seed))


def _exact_attend(c, s):
    n, t, h, kv, d, b = (c[x] for x in ("n_seq", "tokens", "heads", "kv_heads", "dim", "block"))
    group = h // kv
    out = torch.zeros(n, t, h, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(n, h, t, dtype=torch.float64, device="cuda")
    for i, (m, x) in enumerate(zip(_lens(c), _counts(c))):
        row = torch.arange(m, device="cuda")
        seen = row <= (m - x + torch.arange(x, device="cuda"))[:, None]
        for e in range(kv):
            at = slice(e * group, (e + 1) * group)
            k = s["k"][i, :m, e].double() * s["k_scale"][i, e][row // b].double()[:, None]
            v = s["v"][i, :m, e].double() * s["v_scale"][i, e][row // b].double()[:, None]
            z = torch.einsum("ihd,jd->hij", s["q"][i, :x, at].double(), k) / d ** 0.5
            z = torch.where(seen, z, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
            if m == 0:
                lse[i, at, :x] = -math.inf
                continue
            lse[i, at, :x] = torch.logsumexp(z, dim=-1)
            p = torch.where(seen, torch.exp(z - lse[i, at, :x, None]), torch.zeros_like(z))
            out[i, :x, at] = torch.einsum("hij,jd->ihd", p, v)
    return [out, lse]


def _exact_append(c, s):
    n, t, kv, d, b, r = (c[x] for x in ("n_seq", "tokens", "kv_heads", "dim", "block", "rope_dim"))
    lens, counts = _lens(c), _counts(c)
    of_pair = [a for a, pairs in enumerate(_sections(c)) for _ in range(pairs)]
    freq = torch.tensor([math.pow(THETA, -2.0 * i / r) for i in range(r // 2)], dtype=torch.float64, device="cuda") if r else None

    def ready(x, gain, i, m):  # one request's rows [m, heads, d]
        y = x[i, :m].double().clone()
        if c["norm"]:
            y = y / torch.sqrt(torch.sum(y ** 2, dim=-1, keepdim=True) / d + EPS) * gain.double()
        if r and m:
            if "positions" in s:
                pos = torch.stack([s["positions"][a, i, :m] for a in of_pair], dim=1).double()
            else:
                pos = (lens[i] + torch.arange(m, device="cuda", dtype=torch.float64))[:, None]
            turn = torch.polar(torch.ones_like(pos * freq), pos * freq)[:, None]
            at = torch.arange(r // 2, device="cuda")
            at, by = (at, at + r // 2) if c["halves"] else (2 * at, 2 * at + 1)
            z = torch.complex(y[..., at], y[..., by]) * turn
            y[..., at], y[..., by] = z.real, z.imag
        return y

    got = []
    if c["heads"]:
        q = s["q_out"].double()
        for i, m in enumerate(counts):
            q[i, :m] = ready(s["q"], s.get("q_gain"), i, m)
        got.append(q)
    new = [lambda i, m: ready(s["k_new"], s.get("k_gain"), i, m), lambda i, m: s["v_new"][i, :m].double()]
    caches = [s["k"].double(), s["v"].double()]
    ends = np.array([x + y for x, y in zip(lens, counts)], dtype=np.int32)
    if not b:
        for cache, rows in zip(caches, new):
            for i, m in enumerate(counts):
                cache[i, lens[i]:lens[i] + m] = rows(i, m)
        return got + caches + [ends]
    scales = [s["k_scale"].double(), s["v_scale"].double()]
    opened = [s["k_open_out"].double(), s["v_open_out"].double()]
    for cache, scale, left, rows, before in zip(caches, scales, opened, new, (s["k_open"], s["v_open"])):
        for i, m in enumerate(counts):
            rest = int(ends[i]) % b
            if m == 0:
                left[i, :rest] = before[i, :rest].double()
                continue
            first = lens[i] // b
            x = torch.cat([before[i, :lens[i] % b].double(), rows(i, m)])
            nb = -(-x.shape[0] // b)
            whole = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, nb * b - x.shape[0])).view(nb, b, kv, d)
            held = whole.to(TORCH[c["dtype"]]).double()  # what is quantised is the row as 16 bits hold it
            most = held.abs().amax(dim=(1, 3)).clamp(min=1e-30)
            if c["cache"] == "i8":
                step = most.cpu().numpy().astype(np.float32) / np.float32(127)
            else:
                m, e = np.frexp(most.cpu().numpy() / 448)
                step = np.ldexp(1.0, np.where(m == 0.5, e - 1, e))
            step = torch.from_numpy(step.astype(np.float64)).cuda()
            code = held / step[:, None, :, None]
            if c["cache"] == "i8":
                code = torch.round(code)
            cache[i, first * b:first * b + x.shape[0]] = code.view(nb * b, kv, d)[:x.shape[0]]
            scale[i, :, first:first + nb] = step.T
            if rest:
                left[i, :rest] = x[x.shape[0] - rest:]
    if c["cache"] == "i8":
        caches = [x.to(torch.int8) for x in caches]
    return got + caches + scales + opened + [ends]
