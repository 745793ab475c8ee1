"""Attention over a decoder's key-value cache as a program under a memory
budget uses it: verifying a tree of drafted tokens in one pass over the
weights, weighing the cached rows by the attention they get, evicting the rows
that get least, and accepting the drafted path.

A case names an operator and its sizes; prepare() gives what a program has in
hand before the call, run() is one call through the C ABI's Python binding
(own) or the same from elementary torch operations, exact() the same result in
64 bits.
"""
import math

import numpy as np
import torch

own = False

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # the smallest call: a short tree of drafted tokens of one request on
        # a prompt of a hundred tokens, 8 heads (latency)
        dict(name="tree_small", kind="attend", dtype="bf16", n_seq=1, tokens=7, heads=8, kv_heads=8, dim=128,
             length=100, capacity=160, draft=True, weigh=False),
        # the 7B-shaped decoder's heads and its cache of 544 rows: a wide tree
        # verified while one pass of the weights crosses the host link
        dict(name="tree_7b", kind="attend", dtype="bf16", n_seq=1, tokens=64, heads=32, kv_heads=32, dim=128,
             length=511, capacity=544, draft=True, weigh=False),
        # many requests of ragged lengths, shared key heads, a tree each
        dict(name="tree_batch", kind="attend", dtype="bf16", n_seq=32, tokens=24, heads=32, kv_heads=8, dim=128,
             length=8000, capacity=8192, draft=True, weigh=False),
        # one request with a very long history, a small tree, 64-wide heads
        dict(name="tree_long", kind="attend", dtype="f16", n_seq=1, tokens=13, heads=16, kv_heads=4, dim=64,
             length=131001, capacity=131072, draft=True, weigh=False),
        # single tokens of many requests, with the attention that each cached
        # row got: the largest call
        dict(name="decode_weighed", kind="attend", dtype="bf16", n_seq=64, tokens=1, heads=32, kv_heads=8, dim=128,
             length=16384, capacity=16400, draft=False, weigh=True),
        # a chunk of a long prompt behind what is cached, with the weights of
        # the cached rows
        dict(name="chunk_weighed", kind="attend", dtype="f16", n_seq=2, tokens=1000, heads=32, kv_heads=8, dim=128,
             length=4096, capacity=4100, draft=False, weigh=True),
        # the weights of a 512-token prompt of the 7B-shaped decoder
        dict(name="weigh_prompt", kind="weigh", dtype="bf16", n_seq=1, tokens=512, pick=False, heads=32, kv_heads=32,
             dim=128, length=512, capacity=544),
        # the weights that the accepted tokens of many requests give
        dict(name="weigh_accepted", kind="weigh", dtype="bf16", n_seq=32, tokens=24, pick=True, heads=32, kv_heads=8,
             dim=128, length=8000, capacity=8192),
        # the 7B-shaped decoder's cache, full, halved (all heads of one layer)
        dict(name="evict_small", kind="evict", dtype="bf16", n_seq=1, kv_heads=32, dim=128, length=544, capacity=544,
             keep=272, recent=64, sink=4),
        # the caches of many requests
        dict(name="evict_batch", kind="evict", dtype="f16", n_seq=32, kv_heads=8, dim=128, length=8001, capacity=8192,
             keep=4000, recent=512, sink=4),
        # one request of the 7B-shaped decoder: keys and values of 32 layers
        dict(name="accept_7b", kind="accept", dtype="bf16", n_seq=1, tokens=64, caches=64, kv_heads=32, dim=128,
             length=480, capacity=544),
        # many requests, shared key heads, 16 layers
        dict(name="accept_batch", kind="accept", dtype="f16", n_seq=32, tokens=24, caches=32, kv_heads=8, dim=128,
             length=1000, capacity=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "weigh", "evict", "accept"])
    heads, kv = rng.choice([(8, 8), (32, 32), (32, 8), (16, 2), (12, 4), (6, 1)])
    c = dict(kind=kind, dtype=rng.choice(["f16", "bf16"]), n_seq=_log(rng, 1, 64), kv_heads=kv, dim=rng.choice([64, 128]))
    if kind == "attend":
        c["draft"] = rng.random() < 0.6
        c["tokens"] = _log(rng, 1, 128) if c["draft"] else rng.choice([1, _log(rng, 2, 1000)])
        c["weigh"] = not c["draft"] and rng.random() < 0.6
        c["heads"] = heads
    elif kind == "weigh":
        c.update(heads=heads, tokens=_log(rng, 1, 512), pick=rng.random() < 0.5)
    elif kind == "accept":
        c.update(tokens=_log(rng, 2, 128), caches=2 * _log(rng, 1, 40))
        c["n_seq"] = min(c["n_seq"], max(1, 8192 // (kv * c["caches"])))
    room = 1 << 20 if kind == "accept" else 2 << 20
    most = max(64, room // (c["n_seq"] * kv))
    if kind == "accept":
        most = min(4096, max(16, most // c["caches"]))
    elif kind == "weigh" or (kind == "attend" and c["tokens"] > 8):  # products within the largest listed case's
        c["n_seq"] = min(c["n_seq"], max(1, (1 << 27) // (heads * c["tokens"] ** 2)))
        most = min(most, max(64, (1 << 27) // (c["n_seq"] * heads * c["tokens"])))
    c["length"] = _log(rng, 17, min(most, 131000))
    if not c.get("draft", True) or kind == "weigh":
        c["length"] = max(c["length"], c["tokens"])
    c["capacity"] = c["length"] + rng.choice([0, 1, 13, 64, 300])
    if kind == "accept":
        c["capacity"] += c["tokens"]
    if kind == "evict":
        c["keep"] = max(2, int(c["length"] * rng.uniform(0.2, 0.95)))
        c["recent"] = int(c["keep"] * rng.uniform(0, 0.5))
        c["sink"] = min(rng.choice([0, 1, 4]), c["keep"] - c["recent"])
    return c


# ------------------------------------------------------------------ inputs
def _lens(c):
    """Cached rows of each request: the longest first, the others down to half of that."""
    n, low = c["length"], (c["length"] + 1) // 2
    if c["kind"] == "weigh" or not c.get("draft", True):
        low = max(low, c["tokens"])
    return [n - b * 7919 % (n - low + 1) for b in range(c["n_seq"])]


def _counts(c):
    """Nodes in use of each request's tree (or accepted rows, where rows are picked)."""
    t = c["tokens"]
    if c.get("pick"):
        return [1 + b * 5 % max(1, t // 3) for b in range(c["n_seq"])]
    return [t - b * 3 % (t // 2 + 1) for b in range(c["n_seq"])]


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TORCH[c["dtype"]]
    n, kv, d, cap = c["n_seq"], c["kv_heads"], c["dim"], c["capacity"]

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(0, std, generator=g)

    def whole(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    def uniform(*shape):
        return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(0, 1, generator=g)

    s = dict(case=c, lens=whole(_lens(c)))
    if c["kind"] != "accept":
        s["k"], s["v"] = normal(n, cap, kv, d), normal(n, cap, kv, d)
    if c["kind"] in ("attend", "weigh"):
        t, h = c["tokens"], c["heads"]
        s["q"] = normal(n, t, h, d, std=2.0)
        s["weights_in"] = uniform(n, kv, cap) * 3
        s["weights"] = torch.zeros(n, kv, cap, device="cuda")
    if c["kind"] == "attend":
        s["out"] = torch.zeros(n, t, h, d, dtype=dt, device="cuda")
        s["lse"] = torch.zeros(n, h, t, device="cuda")
        if c["draft"]:
            s["k_new"], s["v_new"] = normal(n, t, kv, d), normal(n, t, kv, d)
            s["counts"] = whole(_counts(c))
            s["parents"] = _tree(n, t, uniform)
    if c["kind"] == "weigh":
        if c["pick"]:  # the accepted rows, in the order of the path
            s["counts"] = whole(_counts(c))
            s["rows"] = torch.argsort(uniform(n, t), dim=1)
            s["rows"] = torch.sort(s["rows"][:, : max(_counts(c))], dim=1)[0]
            s["rows"] = torch.nn.functional.pad(s["rows"], (0, t - s["rows"].shape[1])).to(torch.int32).contiguous()
        s["lse"] = _plain_lse(s)
    if c["kind"] == "evict":
        # most rows get little, a few a lot, some nothing that 32 bits hold
        w = uniform(n, kv, cap) ** 4 * 5
        s["weights_in"] = torch.where(w < 1e-6, torch.zeros_like(w), w)
        keep = c["keep"]
        s["k_out"], s["v_out"] = torch.zeros(n, keep, kv, d, dtype=dt, device="cuda"), torch.zeros(n, keep, kv, d, dtype=dt, device="cuda")
        s["weights"] = torch.zeros(n, kv, keep, device="cuda")
        s["kept"] = torch.full((n, kv, keep), -1, dtype=torch.int32, device="cuda")
        s["lens_out"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    if c["kind"] == "accept":
        t, k = c["tokens"], c["caches"]
        s["caches"], s["drafts"] = normal(k, n, cap, kv, d), normal(k, n, t, kv, d)
        s["cache_ptrs"] = np.array([x.data_ptr() for x in s["caches"]], dtype=np.uint64)
        s["draft_ptrs"] = np.array([x.data_ptr() for x in s["drafts"]], dtype=np.uint64)
        s["counts"] = whole(_counts(c))
        s["parents"] = _tree(n, t, uniform)
        s["targets"] = (uniform(n, t) * 32000).to(torch.int32)
        of_parent = torch.gather(s["targets"], 1, s["parents"].clamp(min=0).long())
        s["ids"] = torch.where(uniform(n, t) < 0.7, of_parent, (uniform(n, t) * 32000).to(torch.int32))
        s["path"] = torch.full((n, t), -1, dtype=torch.int32, device="cuda")
        for name in ("accepted", "next", "lens_out"):
            s[name] = torch.zeros(n, dtype=torch.int32, device="cuda")
    return s


def _tree(n, t, uniform):
    """Parents of drafted nodes: node 0 is the root, the others hang below an earlier one of the last eight."""
    i = torch.arange(t, device="cuda", dtype=torch.float32)
    back = (uniform(n, t) * torch.clamp(i, max=8)).floor()
    parent = (i - 1 - back).clamp(min=0).to(torch.int32)
    parent[:, 0] = -1
    return parent.contiguous()


# -------------------------------------------------------------- plain forms
def _seen(s, t, keys, draft):
    """[n, t, keys (+ t drafted)]: what each query sees."""
    lens = s["lens"].long()
    j = torch.arange(keys, device="cuda")
    i = torch.arange(t, device="cuda")
    n = lens.numel()
    if not draft:  # the queries are the last rows of the cache
        count = s["counts"].long() if "counts" in s else torch.full((n,), t, device="cuda")
        last = lens[:, None] - count[:, None] + i
        return (j <= last[:, :, None]) & (j < lens[:, None, None]) & (i < count[:, None])[:, :, None]
    old = (j < lens[:, None, None]).expand(n, t, keys)
    parents = s["parents"].long()
    above = torch.nn.functional.one_hot(parents.clamp(min=0), t) * (parents >= 0)[:, :, None]
    reach = torch.eye(t, device="cuda").expand(n, t, t)
    steps = max(1, math.ceil(math.log2(t + 1)))
    up = (reach + above.float()).clamp(max=1)
    for _ in range(steps):  # reached in 2^k steps
        up = (up @ up).clamp(max=1)
    used = i < s["counts"].long()[:, None]
    return torch.cat([old, up > 0.5], dim=2) & used[:, :, None]


def _scores(q, k, seen):
    """[n, kv, group, t, keys] in 32 bits, -inf where a key is not seen."""
    n, t, h, d = q.shape
    kv = k.shape[2]
    a = q.float().view(n, t, kv, h // kv, d).permute(0, 2, 3, 1, 4).reshape(n, kv, h // kv * t, d)
    x = torch.matmul(a, k.float().permute(0, 2, 3, 1)).view(n, kv, h // kv, t, -1) / math.sqrt(d)
    return x.masked_fill(~seen[:, None, None], -math.inf)


def _plain_lse(s):
    """[n, heads, t] of the queries over the cache (an earlier attention call's output)."""
    c = s["case"]
    n, t, h = c["n_seq"], c["tokens"], c["heads"]
    got = torch.zeros(n, h, t, device="cuda")
    if not c["pick"]:
        x = _scores(s["q"], s["k"], _seen(s, t, c["capacity"], False))
        got.copy_(torch.logsumexp(x, dim=-1).view(n, h, t))
        return got
    at = s["rows"].long()
    q = torch.gather(s["q"], 1, at[:, :, None, None].expand(-1, -1, h, c["dim"]))
    x = _scores(q, s["k"], _seen(s, t, c["capacity"], False))
    used = (torch.arange(t, device="cuda") < s["counts"][:, None])[:, None, :]
    lse = torch.logsumexp(x, dim=-1).view(n, h, t)
    # rows of the list's unused end are not looked at
    spare = torch.zeros(n, h, t + 1, device="cuda")
    spare.scatter_(2, torch.where(used, at[:, None, :], t).expand(n, h, t), lse)
    return spare[:, :, :t].contiguous()


def _plain_attend(s):
    c = s["case"]
    n, t, h, kv, d, cap = (c[x] for x in ("n_seq", "tokens", "heads", "kv_heads", "dim", "capacity"))
    seen = _seen(s, t, cap, c["draft"])
    k, v = s["k"], s["v"]
    if c["draft"]:
        k, v = torch.cat([k, s["k_new"]], dim=1), torch.cat([v, s["v_new"]], dim=1)
    x = _scores(s["q"], k, seen)
    m = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    l = p.sum(dim=-1, keepdim=True)
    lse = (m + torch.log(l)).view(n, h, t)
    p = p / torch.where(l > 0, l, torch.ones_like(l))
    o = torch.matmul(p.view(n, kv, -1, p.shape[-1]), v.float().permute(0, 2, 1, 3))
    out = o.view(n, kv, h // kv, t, d).permute(0, 3, 1, 2, 4).reshape(n, t, h, d).to(s["q"].dtype)
    used = torch.ones(n, t, dtype=torch.bool, device="cuda")
    if c["draft"]:
        used = torch.arange(t, device="cuda") < s["counts"][:, None]
    got = [out.masked_fill(~used[:, :, None, None], 0), lse.masked_fill(~used[:, None, :], 0)]
    if c["weigh"]:
        w = s["weights_in"] + p.sum(dim=(2, 3))
        got.append(w.masked_fill(~(torch.arange(cap, device="cuda") < s["lens"][:, None])[:, None], 0))
    return got


def _plain_weigh(s):
    c = s["case"]
    n, t, h, kv, d, cap = (c[x] for x in ("n_seq", "tokens", "heads", "kv_heads", "dim", "capacity"))
    q, lse = s["q"], s["lse"]
    if c["pick"]:
        at = s["rows"].long()
        q = torch.gather(q, 1, at[:, :, None, None].expand(-1, -1, h, d))
        lse = torch.gather(lse, 2, at[:, None, :].expand(-1, h, -1))
    x = _scores(q, s["k"], _seen(s, t, cap, False))
    p = torch.exp(x - lse.view(n, kv, h // kv, t, 1))
    w = s["weights_in"] + p.sum(dim=(2, 3))
    return [w.masked_fill(~(torch.arange(cap, device="cuda") < s["lens"][:, None])[:, None], 0)]


def _plain_evict(s):
    c = s["case"]
    cap, keep = c["capacity"], c["keep"]
    lens = s["lens"].long()[:, None, None]
    j = torch.arange(cap, device="cuda")
    w = s["weights_in"]
    rank = torch.where((j < c["sink"]) | (j >= lens - c["recent"]), torch.full_like(w, math.inf), w)
    rank = torch.where(j < lens, rank, torch.full_like(w, -math.inf))
    order = torch.sort(rank, dim=-1, descending=True, stable=True)[1][..., :keep]
    valid = torch.arange(keep, device="cuda") < lens.clamp(max=keep)
    at = torch.sort(torch.where(valid, order, torch.full_like(order, cap)), dim=-1)[0]
    from_row = at.clamp(max=cap - 1)
    wide = from_row.permute(0, 2, 1)[..., None].expand(-1, -1, -1, c["dim"])
    gone = ~valid.permute(0, 2, 1)[..., None]
    return [torch.gather(s["k"], 1, wide).masked_fill(gone, 0), torch.gather(s["v"], 1, wide).masked_fill(gone, 0),
            torch.gather(w, 2, from_row).masked_fill(~valid, 0), at.masked_fill(~valid, -1).to(torch.int32),
            s["lens"].clamp(max=keep)]


def _path(ids, targets, parents, counts):
    """(path, accepted, next) of the greedy walk; path is -1 behind the accepted nodes."""
    n, t = ids.shape
    i = torch.arange(t, device=ids.device)
    fits = (parents >= 0) & (i < counts[:, None]) & (ids == torch.gather(targets, 1, parents.clamp(min=0).long()))
    after = torch.full((n, t + 1), t, dtype=torch.long, device=ids.device)  # the lowest child that fits; t: none
    after.scatter_reduce_(1, torch.where(fits, parents.long(), t), torch.where(fits, i, t).expand(n, t), "amin")
    after[:, t] = t
    at = torch.zeros(n, dtype=torch.long, device=ids.device)
    steps = []
    for _ in range(t):
        steps.append(at)
        at = torch.gather(after, 1, at[:, None])[:, 0]
    path = torch.stack(steps, dim=1)
    accepted = (path < t).sum(dim=1)
    last = torch.gather(path, 1, accepted[:, None] - 1)
    return path.masked_fill(path == t, -1).int(), accepted.int(), torch.gather(targets, 1, last)[:, 0]


def _plain_accept(s):
    c = s["case"]
    t = c["tokens"]
    path, accepted, following = _path(s["ids"], s["targets"], s["parents"], s["counts"])
    to = s["lens"].long()[:, None] + torch.arange(t, device="cuda")
    used = path >= 0
    seq = torch.arange(c["n_seq"], device="cuda")[:, None].expand(-1, t)[used]
    to, at = to[used], path[used].long()
    for cache, new in zip(s["caches"], s["drafts"]):
        cache[seq, to] = new[seq, at]
    return [path, accepted, following, s["lens"] + accepted, s["caches"]]


def run(state):
    s = state
    c = s["case"]
    if not own:
        return {"attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict, "accept": _plain_accept}[c["kind"]](s)
    from paper_2401_16757_gb300 import capi

    stream = torch.cuda.current_stream().cuda_stream
    if c["kind"] in ("attend", "weigh"):
        args = capi.cached_attention(
            c["dtype"], c["n_seq"], c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["capacity"],
            q=s["q"].data_ptr(), k=s["k"].data_ptr(), v=s["v"].data_ptr(), lens=s["lens"].data_ptr(),
            counts=s["counts"].data_ptr() if "counts" in s else 0,
            parents=s["parents"].data_ptr() if "parents" in s else 0,
            rows=s["rows"].data_ptr() if "rows" in s else 0,
            k_new=s["k_new"].data_ptr() if "k_new" in s else 0, v_new=s["v_new"].data_ptr() if "v_new" in s else 0,
            out=s["out"].data_ptr() if "out" in s else 0, lse=s["lse"].data_ptr(),
            weights_in=s["weights_in"].data_ptr() if c.get("weigh", True) else 0,
            weights=s["weights"].data_ptr() if c.get("weigh", True) else 0)
        if c["kind"] == "weigh":
            capi.attention_weights(args, stream)
            return [s["weights"]]
        space = torch.empty(capi.attention_tree_workspace(args), dtype=torch.uint8, device="cuda")
        capi.attention_tree(args, space.data_ptr(), space.numel(), stream)
        return [s["out"], s["lse"]] + ([s["weights"]] if c["weigh"] else [])
    if c["kind"] == "evict":
        capi.cache_evict(
            c["dtype"], c["n_seq"], c["kv_heads"], c["dim"], c["capacity"], c["keep"], c["recent"], c["sink"],
            k=s["k"].data_ptr(), v=s["v"].data_ptr(), weights=s["weights_in"].data_ptr(), lens=s["lens"].data_ptr(),
            k_out=s["k_out"].data_ptr(), v_out=s["v_out"].data_ptr(), out_capacity=c["keep"],
            weights_out=s["weights"].data_ptr(), kept=s["kept"].data_ptr(), lens_out=s["lens_out"].data_ptr(),
            stream=stream)
        return [s["k_out"], s["v_out"], s["weights"], s["kept"], s["lens_out"]]
    capi.tree_accept(
        c["dtype"], c["n_seq"], c["tokens"], c["kv_heads"] * c["dim"], c["capacity"], ids=s["ids"].data_ptr(),
        targets=s["targets"].data_ptr(), parents=s["parents"].data_ptr(), counts=s["counts"].data_ptr(),
        lens=s["lens"].data_ptr(), caches=s["cache_ptrs"], drafts=s["draft_ptrs"], path=s["path"].data_ptr(),
        accepted=s["accepted"].data_ptr(), next=s["next"].data_ptr(), lens_out=s["lens_out"].data_ptr(), stream=stream)
    return [s["path"], s["accepted"], s["next"], s["lens_out"], s["caches"]]


# ------------------------------------------------------------ what it takes
def work(case):
    """Bytes: the cached rows in use, the queries, the outputs, the tree, once each. Operations: two per product
    and sum of every (query, visible row) pair, for the scores and for the values."""
    c = case
    lens, d, kv, n = _lens(c), c["dim"], c["kv_heads"], c["n_seq"]
    row = kv * d * 2
    if c["kind"] in ("attend", "weigh"):
        t, h = c["tokens"], c["heads"]
        if c["kind"] == "weigh":
            counts = _counts(c) if c["pick"] else [t] * n
            pairs = sum(x * (y - (x - 1) / 2) for x, y in zip(counts, lens))
            return dict(bytes=sum(lens) * (row + 8 * kv) + sum(counts) * h * (2 * d + 4) + 4 * n, flops=2 * d * h * pairs)
        counts = _counts(c) if c["draft"] else [t] * n
        pairs = sum(x * y if c["draft"] else x * (y - (x - 1) / 2) for x, y in zip(counts, lens))
        b = sum(lens) * 2 * row + sum(counts) * h * (4 * d + 4) + 4 * n
        if c["draft"]:
            b += sum(counts) * (2 * row + 4)
            pairs += sum(min(x, 1 + x // 4) * x for x in counts)  # a node's ancestors
        if c["weigh"]:
            b += sum(lens) * 8 * kv
        return dict(bytes=b, flops=4 * d * h * pairs)
    if c["kind"] == "evict":
        kept = sum(min(x, c["keep"]) for x in lens)
        return dict(bytes=kept * (4 * row + 8 * kv) + sum(lens) * 4 * kv, flops=0)
    # about four rows of a request are accepted
    return dict(bytes=n * (min(4, c["tokens"]) * 2 * row * c["caches"] + 16 * c["tokens"]), flops=0)


# --------------------------------------------------------------- in 64 bits
def exact(case, seed):
    c = case
    s = prepare(c, seed)
    n, cap, kv, d = c["n_seq"], c["capacity"], c["kv_heads"], c["dim"]
    lens = _lens(c)
    if c["kind"] in ("attend", "weigh"):
        return _exact_attend(c, s, lens)
    if c["kind"] == "evict":
        keep = c["keep"]
        k, v = (torch.zeros(n, keep, kv, d, dtype=torch.float64) for _ in range(2))
        w, kept = torch.zeros(n, kv, keep, dtype=torch.float64), np.full((n, kv, keep), -1, dtype=np.int32)
        score = s["weights_in"].double().cpu().numpy()
        host_k, host_v = s["k"].cpu(), s["v"].cpu()
        for b in range(n):
            for h in range(kv):
                r = [math.inf if j < c["sink"] or j >= lens[b] - c["recent"] else x for j, x in enumerate(score[b, h, :lens[b]])]
                at = np.sort(np.argsort(-np.array(r), kind="stable")[:keep])
                kept[b, h, :len(at)] = at
                k[b, :len(at), h], v[b, :len(at), h] = host_k[b, at, h].double(), host_v[b, at, h].double()
                w[b, h, :len(at)] = torch.from_numpy(score[b, h, at])
        return [k, v, w, kept, np.array([min(x, keep) for x in lens], dtype=np.int32)]
    ids, targets, parents, counts = (s[x].tolist() for x in ("ids", "targets", "parents", "counts"))
    path = np.full((n, c["tokens"]), -1, dtype=np.int32)
    caches = s["caches"].double()
    accepted, following = [], []
    for b in range(n):
        at, row = 0, lens[b]
        while at is not None:
            path[b, row - lens[b]] = at
            for x, y in zip(caches, s["drafts"]):
                x[b, row] = y[b, at].double()
            row += 1
            last = at
            at = next((i for i in range(1, counts[b]) if parents[b][i] == last and ids[b][i] == targets[b][last]), None)
        accepted.append(row - lens[b])
        following.append(targets[b][last])
    whole = [np.array(x, dtype=np.int32) for x in (accepted, following, [x + y for x, y in zip(lens, accepted)])]
    return [path, *whole, caches]


def _exact_attend(c, s, lens):
    n, t, h, kv, d, cap = (c[x] for x in ("n_seq", "tokens", "heads", "kv_heads", "dim", "capacity"))
    out, lse = torch.zeros(n, t, h, d, dtype=torch.float64, device="cuda"), torch.zeros(n, h, t, dtype=torch.float64, device="cuda")
    weights = torch.zeros(n, kv, cap, dtype=torch.float64, device="cuda")
    counts = s["counts"].tolist() if "counts" in s else [t] * n
    group = h // kv
    for b in range(n):
        x, m = counts[b], lens[b]
        rows = s["rows"][b, :x].long() if "rows" in s else torch.arange(x, device="cuda")
        seen = torch.zeros(x, m + (x if c.get("draft") else 0), dtype=torch.bool, device="cuda")
        if c.get("draft"):
            above = s["parents"][b].tolist()
            host = torch.zeros(x, x, dtype=torch.bool)
            for i in range(x):
                j = i
                while j >= 0:
                    host[i, j] = True
                    j = above[j]
            seen[:, :m], seen[:, m:] = True, host.cuda()
        else:
            seen = torch.arange(m, device="cuda") <= (m - x + torch.arange(x, device="cuda"))[:, None]
        for g in range(kv):
            k, v = s["k"][b, :m, g].double(), s["v"][b, :m, g].double()
            if c.get("draft"):
                k, v = torch.cat([k, s["k_new"][b, :x, g].double()]), torch.cat([v, s["v_new"][b, :x, g].double()])
            q = s["q"][b, rows][:, g * group:(g + 1) * group].double()
            z = torch.einsum("ihd,jd->hij", q, k) / d ** 0.5
            z = torch.where(seen, z, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
            at = slice(g * group, (g + 1) * group)
            if c["kind"] == "weigh":  # the softmax of the statistics that were handed in
                p = torch.exp(z - s["lse"][b, at][:, rows].double()[..., None])
            else:
                lse[b, at, :x] = torch.logsumexp(z, dim=-1)
                p = torch.exp(z - lse[b, at, :x, None])
                out[b, :x, at] = torch.einsum("hij,jd->ihd", p, v)
            if not c.get("draft"):
                weights[b, g, :m] = s["weights_in"][b, g, :m].double() + p.sum(dim=(0, 1))
    if c["kind"] == "weigh":
        return [weights]
    return [out, lse] + ([weights] if c["weigh"] else [])
