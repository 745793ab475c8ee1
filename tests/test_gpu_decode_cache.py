"""Decoders whose attention layers carry flags: drafted trees verified and
accepted in a pass, the weights of the cached rows, eviction; through the
engine, swapped and resident, against the oracle and against plain decoding."""
import numpy as np
import pytest

import synth
from oracle import forward as F
from oracle import plan as OP
from paper_2401_16757_gb300 import capi
from helpers import rel_l2

pytestmark = pytest.mark.gpu

CFG = dict(layers=2, d=256, heads=2, ffn=688, vocab=1000, max_seq=96)
CHAIN_TOL = 2.0 ** -7  # whole bf16 decoders: one step of the type at 1.0 (tests/test_gpu_llm.py)


class Engines:
    """Engines over one set of weights and one state: name -> (tokens, layer flags)."""

    def __init__(self, kinds, weights=False, resident=False, cfg=CFG):
        import torch
        self.torch = torch
        self.cfg = cfg
        self.e = {}
        self.w = self.host = None
        size = 0
        for name, (tokens, tree) in kinds.items():
            m = synth.arch.llm(tokens=tokens, tree=tree, weights=weights, **cfg)
            if self.w is None:
                self.w = synth.gen.model_weights(m)
                self.host = capi.HostWeights(self.w)
            d = capi.Desc(m)
            plan = capi.Plan.resident(d) if resident else capi.Plan.partition(d, OP.weight_bytes(m) // 2 // 256 * 256)
            eng = capi.Engine(plan, self.host)
            info = plan.info()
            din = torch.zeros(max(16, info["input_bytes"]), dtype=torch.uint8, device="cuda")
            dout = torch.zeros(info["output_bytes"], dtype=torch.uint8, device="cuda")
            self.e[name] = (m, plan, eng, din, dout, plan.output_offsets(), plan.state_layout(), tokens)
            size = max(size, info["state_bytes"])
        self.state = torch.zeros(size, dtype=torch.uint8, device="cuda")
        for x in self.e.values():
            x[2].bind_state(self.state.data_ptr(), size)

    def words(self, name, off, n=1):
        return self.state[off:off + 4 * n].view(self.torch.int32)

    @property
    def header(self):
        return self.state[:32].view(self.torch.int32)

    def set_tree(self, name, parents):
        lay = self.e[name][6]
        self.words(name, lay["tree_count"])[0] = len(parents)
        self.words(name, lay["tree_parents"], len(parents)).copy_(self.torch.tensor(parents, dtype=self.torch.int32))

    def run(self, name, ids, parents=None, sync=True):
        m, plan, eng, din, dout, offs, lay, tokens = self.e[name]
        ids = np.ascontiguousarray(ids, dtype=np.int32)
        if parents is not None:
            self.set_tree(name, parents)
        din[:ids.nbytes].copy_(self.torch.from_numpy(ids.view(np.uint8).reshape(-1)))
        eng.infer(din.data_ptr(), dout.data_ptr(), self.torch.cuda.current_stream().cuda_stream)
        if sync:
            eng.sync()
        host = dout.cpu().numpy()
        v, n = self.cfg["vocab"], ids.size
        logits = host[offs[0]:offs[0] + n * v * 2].view(np.uint16).reshape(n, v).copy()
        return logits, host[offs[1]:offs[1] + n * 4].view(np.int32).copy()

    def accept(self, name):
        m, plan, eng, din, dout, offs, lay, tokens = self.e[name]
        eng.tree_accept(din.data_ptr(), dout.data_ptr() + offs[1], self.torch.cuda.current_stream().cuda_stream)
        eng.sync()
        n = int(self.header[3])
        return self.words(name, lay["tree_path"], tokens).tolist()[:n], n, int(self.header[4])

    def caches(self, name):
        """[layers, 2, max_seq, d] as float64."""
        lay, c = self.e[name][6], self.cfg
        raw = self.state[lay["caches"]:lay["caches"] + 2 * c["layers"] * lay["cache_bytes"]].cpu().numpy()
        raw = raw.reshape(c["layers"], 2, -1)[:, :, :c["max_seq"] * c["d"] * 2].copy()
        return raw.view(np.uint16).reshape(c["layers"], 2, c["max_seq"], c["d"])

    def weights(self, name):
        lay, c = self.e[name][6], self.cfg
        n = c["layers"] * c["heads"] * c["max_seq"]
        return self.state[lay["weights"]:lay["weights"] + 4 * n].view(self.torch.float32).cpu().numpy().reshape(c["layers"], c["heads"], -1)


PARENTS = [-1, 0, 0, 1, 1, 2, 4, 6, 0, 8, 9]


def _paths(parents):
    out = []
    for i in range(len(parents)):
        p, j = [], i
        while j >= 0:
            p.insert(0, j)
            j = parents[j]
        out.append(p)
    return out


@pytest.mark.parametrize("resident", [False, True])
def test_tree_nodes_equal_their_paths(resident):
    """Every node's logits are those of the oracle after the prompt and the node's path."""
    ids = synth.gen.model_input(synth.arch.llm(tokens=37, **CFG)).reshape(-1)
    e = Engines({"prefill": (37, False), "tree": (len(PARENTS), True)}, resident=resident)
    e.run("prefill", ids)
    before = e.caches("tree").copy()
    tree = np.array([7, 99, 500, 1, 999, 320, 64, 65, 12, 0, 402], dtype=np.int32)
    logits, tok = e.run("tree", tree, PARENTS)
    assert e.header[:2].tolist() == [37, 0] and np.array_equal(before, e.caches("tree"))  # nothing is in the caches yet
    got = F.decode(logits, "bf16")
    for path in _paths(PARENTS):
        st = F.new_state()
        x = np.concatenate([ids, tree[path]]).astype(np.int32)
        mp = synth.arch.llm(tokens=x.size, **CFG)
        ref = F.forward(mp, e.w, x.reshape(-1, 1, 1, 1), state=st)[0].reshape(x.size, -1)[-1]
        assert rel_l2(got[path[-1]], ref) <= CHAIN_TOL, path
        assert np.argmax(got[path[-1]]) == tok[path[-1]]


def test_swapped_equals_resident():
    ids = synth.gen.model_input(synth.arch.llm(tokens=20, **CFG)).reshape(-1)
    out = []
    for resident in (False, True):
        e = Engines({"prefill": (20, False), "tree": (40, True)}, weights=True, resident=resident)
        a = e.run("prefill", ids)
        parents = [-1] + [max(0, i - 1 - i % 5) for i in range(1, 40)]
        b = e.run("tree", np.arange(40) * 7 % 1000, parents)
        acc = e.accept("tree")
        e.e["tree"][2].evict(18, 6, 2, e.torch.cuda.current_stream().cuda_stream)
        e.e["tree"][2].sync()
        out.append((a, b, acc, e.caches("tree").copy(), e.weights("tree").copy(), e.header[:2].tolist()))
    (a, b) = out
    assert all(np.array_equal(x, y) for x, y in zip(a[0] + a[1], b[0] + b[1]))
    assert a[2] == b[2] and np.array_equal(a[3], b[3]) and np.array_equal(a[4], b[4]) and a[5] == b[5]


def test_speculative_decoding_gives_the_greedy_tokens():
    """Trees that hold the greedy continuation beside wrong guesses: the accepted path is the walk of the pass's own choices,
    the choices are those of one token at a time (but for ties within the rounding), passes are saved, and the caches hold
    the same rows up to the rounding of other sums.  The greedy tokens are fed either way."""
    steps = 24
    ids = synth.gen.model_input(synth.arch.llm(tokens=30, **CFG)).reshape(-1)
    plain = Engines({"prefill": (30, False), "decode": (1, False)})
    want, margin = [int(plain.run("prefill", ids)[1][-1])], [1.0]
    for _ in range(steps + 8):
        logits, t = plain.run("decode", [want[-1]])
        x = np.sort(F.decode(logits, "bf16")[0])
        margin.append((x[-1] - x[-2]) / np.abs(x).max())
        want.append(int(t[0]))
    e = Engines({"prefill": (30, False), "tree": (7, True)})
    e.run("prefill", ids)
    passes = done = 0  # done: greedy tokens in the caches
    # node 0: the last token; a wrong and a right child; the right one's children: wrong, right; then a right one and a dead end
    parents, right = [-1, 0, 0, 2, 2, 4, 3], {0: 0, 2: 1, 4: 2, 5: 3}
    while done < steps:
        n = [want[done], (want[done + 1] + 1) % 1000, want[done + 1], (want[done + 2] + 3) % 1000, want[done + 2], want[done + 3], 5]
        if passes % 3 == 1:
            n[4] = (want[done + 2] + 9) % 1000  # no right grandchild this time
        _, tok = e.run("tree", n, parents)
        for i, k in right.items():
            if passes % 3 != 1 or i < 4:
                assert tok[i] == want[done + k + 1] or margin[done + k + 1] <= 6 * CHAIN_TOL, (passes, i)
        path, acc, nxt = e.accept("tree")
        walk = [0]
        while True:
            c = [i for i in range(1, 7) if parents[i] == walk[-1] and n[i] == tok[walk[-1]]]
            if not c:
                break
            walk.append(c[0])
        assert path == walk and acc == len(walk) and nxt == tok[walk[-1]]
        if any(i not in right for i in walk):  # a tie went to a wrong guess: its rows are not the greedy ones
            walk = [i for i in walk if i in right]
            e.header[0] = 30 + done + len(walk)
        done += len(walk)
        passes += 1
        assert int(e.header[0]) == 30 + done
    assert passes < steps
    rows = 30 + steps
    a, b = F.decode(plain.caches("decode"), "bf16")[:, :, :rows], F.decode(e.caches("tree"), "bf16")[:, :, :rows]
    assert rel_l2(b, a) <= CHAIN_TOL


def _oracle_weights(e, ids):
    """Attention per (layer, head, row) summed over the run's tokens, from the oracle's own forward pass."""
    import numpy as np
    m = synth.arch.llm(tokens=len(ids), **CFG)
    st = F.new_state()
    acts = F.forward_range(m, e.w, {}, F._model_input(m, np.asarray(ids, dtype=np.int32).reshape(-1, 1, 1, 1)), 0, len(m["layers"]), st)
    out = np.zeros((CFG["layers"], CFG["heads"], CFG["max_seq"]))
    li = 0
    n, dh = len(ids), CFG["d"] // CFG["heads"]
    for i, L in enumerate(m["layers"]):
        if L["op"] != "attention":
            continue
        q = F.round_as(F.rope(F._as2d(acts[L["src"][0]]), np.arange(n), L["heads"], L["theta"]), "bf16")
        k = st["kv"][i][0][:n]
        for h in range(CFG["heads"]):
            z = q[:, h * dh:(h + 1) * dh] @ k[:, h * dh:(h + 1) * dh].T / dh ** 0.5
            z = np.where(np.tril(np.ones((n, n), dtype=bool)), z, -np.inf)
            p = np.exp(z - z.max(1, keepdims=True))
            out[li, h, :n] = (p / p.sum(1, keepdims=True)).sum(0)
        li += 1
    return out


@pytest.mark.parametrize("prefill", [5, 41, 64])
def test_weights_of_prefill_decode_and_trees(prefill):
    """The weights after a prompt, single tokens and accepted nodes are the column sums of the oracle's attention."""
    ids = synth.gen.model_input(synth.arch.llm(tokens=prefill, **CFG)).reshape(-1)
    e = Engines({"prefill": (prefill, False), "decode": (1, False), "tree": (5, True)}, weights=True)
    plain = Engines({"prefill": (prefill, False)})
    a, b = e.run("prefill", ids), plain.run("prefill", ids)
    assert rel_l2(F.decode(a[0], "bf16"), F.decode(b[0], "bf16")) <= CHAIN_TOL
    text = list(ids)
    t = int(a[1][-1])
    for _ in range(3):
        text.append(t)
        t = int(e.run("decode", [t])[1][0])
    _, tok = e.run("tree", [t, 3, 4, 5, 6], [-1, 0, 0, 1, 2])
    path, n, nxt = e.accept("tree")
    text += [[t, 3, 4, 5, 6][i] for i in path]
    got, want = e.weights("tree"), _oracle_weights(e, text)
    m = len(text)
    assert int(e.header[0]) == m and n >= 1
    # every query's attention adds up to one
    assert np.all(np.abs(got[:, :, :m].sum(-1) - m) <= 1e-4 * m)
    assert np.all(got[:, :, m:] == 0)
    assert rel_l2(got[0], want[0]) <= 2e-3 and rel_l2(got, want) <= CHAIN_TOL


def test_eviction_keeps_rotation_and_rows():
    """After an eviction the caches hold the rows kept, later tokens are rotated as at their true position, and attention
    runs over the rows that are left."""
    torch = __import__("torch")
    n, keep = 50, 20
    ids = synth.gen.model_input(synth.arch.llm(tokens=n, **CFG)).reshape(-1)
    e = Engines({"prefill": (n, False), "decode": (1, False)}, weights=True)
    ref = Engines({"prefill": (n, False), "decode": (1, False)}, weights=True)
    e.run("prefill", ids)
    ref.run("prefill", ids)
    before, w = e.caches("decode").copy(), e.weights("decode").copy()
    eng = e.e["decode"][2]
    eng.evict(keep, 6, 1, torch.cuda.current_stream().cuda_stream)
    eng.sync()
    assert e.header[:2].tolist() == [keep, n - keep]
    after, w2 = e.caches("decode"), e.weights("decode")
    dh = CFG["d"] // CFG["heads"]
    for l in range(CFG["layers"]):
        for h in range(CFG["heads"]):
            key = w[l, h, :n].astype(np.float64)
            key[0] = np.inf
            key[n - 6:] = np.inf
            rows = np.sort(np.argsort(-key, kind="stable")[:keep])
            cols = slice(h * dh, (h + 1) * dh)
            assert np.array_equal(after[l, :, :keep, cols], before[l, :, rows, cols].transpose(1, 0, 2))
            assert np.array_equal(w2[l, h, :keep], w[l, h, rows]) and np.all(w2[l, h, keep:] == 0)
            assert np.array_equal(after[l, :, keep:, cols], before[l, :, keep:, cols])
    eng.evict(keep + 5, 6, 1, torch.cuda.current_stream().cuda_stream)  # more than there are: nothing changes
    eng.sync()
    assert e.header[:2].tolist() == [keep, n - keep]
    e.run("decode", [123])
    ref.run("decode", [123])
    assert e.header[:2].tolist() == [keep + 1, n - keep] and ref.header[:2].tolist() == [n + 1, 0]
    # the first layer's key and value depend on the token and its position alone
    assert np.array_equal(e.caches("decode")[0, :, keep], ref.caches("decode")[0, :, n])
    # and the first layer's weights grow by one in all, on the rows that are left
    grown = e.weights("decode")[0, :, :keep + 1].sum(-1) - np.concatenate([w2[0, :, :keep], np.zeros((2, 1))], 1).sum(-1)
    assert np.all(np.abs(grown - 1) <= 1e-4)


def test_tree_errors_are_reported():
    e = Engines({"prefill": (30, False), "tree": (4, True)})
    ids = synth.gen.model_input(synth.arch.llm(tokens=30, **CFG)).reshape(-1)
    e.run("prefill", ids)
    for bad in ([-1, 1, 0, 0], [-1, 0, -2, 0]):
        with pytest.raises(capi.SwapnetError) as x:
            e.run("tree", [1, 2, 3, 4], bad)
        assert x.value.code == capi.ERR_INVALID_ARG
    # the cache's last rows: a path of two fits, then no more
    e.header[0] = 95
    e.run("tree", [1, 2, 3, 4], [-1, 0, 0, 0])
    tok = e.run("tree", [1, 2, 3, 4], [-1, 0, 0, 0])[1]
    path, n, _ = e.accept("tree") if tok[0] not in (2, 3, 4) else ([0], 1, 0)
    assert n == 1
    e.header[0] = 96
    e.run("tree", [1, 2, 3, 4], [-1, 0, 0, 0])
    with pytest.raises(capi.SwapnetError) as x:
        e.accept("tree")
    assert x.value.code == capi.ERR_INVALID_ARG
    assert e.header[0].item() == 96 and e.header[3].item() == 0


def test_cnn_and_plain_decoders_have_no_such_calls():
    e = Engines({"decode": (1, False)})
    eng = e.e["decode"][2]
    for call in (lambda: eng.evict(10), lambda: eng.tree_accept(16, 16)):
        with pytest.raises(capi.SwapnetError) as x:
            call()
        assert x.value.code == capi.ERR_INVALID_ARG
    w = Engines({"decode": (1, False)}, weights=True).e["decode"][2]
    for kw in (dict(keep=0), dict(keep=97), dict(keep=10, recent=8, sink=3), dict(keep=5, recent=-1)):
        with pytest.raises(capi.SwapnetError) as x:
            w.evict(**kw)
        assert x.value.code == capi.ERR_INVALID_ARG
