"""Refusals and workspace sizes of the cached-attention calls: decided on the
host, before anything is launched, so they need no GPU."""
import numpy as np
import pytest

from paper_2401_16757_gb300 import capi

A = 1 << 20  # an aligned address; nothing is read from it


def _attn(**kw):
    base = dict(dtype="bf16", n_seq=2, tokens=4, heads=8, kv_heads=2, head_dim=128, max_seq=100, q=A, k=A, v=A, lens=A,
                out=A, lse=A)
    base.update(kw)
    return capi.cached_attention(base.pop("dtype"), *[base.pop(x) for x in ("n_seq", "tokens", "heads", "kv_heads", "head_dim",
                                                                            "max_seq")], **base)


def _code(call, *a, **kw):
    with pytest.raises(capi.SwapnetError) as e:
        call(*a, **kw)
    assert str(e.value)
    return e.value.code


@pytest.mark.parametrize("change,code", [
    (dict(dtype="f32"), capi.ERR_UNSUPPORTED), (dict(dtype=9), capi.ERR_UNSUPPORTED),
    (dict(n_seq=0), capi.ERR_INVALID_ARG), (dict(tokens=0), capi.ERR_INVALID_ARG), (dict(max_seq=0), capi.ERR_INVALID_ARG),
    (dict(heads=7), capi.ERR_INVALID_ARG), (dict(head_dim=96), capi.ERR_UNSUPPORTED),
    (dict(n_seq=70000), capi.ERR_UNSUPPORTED), (dict(n_seq=40000, tokens=30000), capi.ERR_UNSUPPORTED), (dict(heads=258, kv_heads=2), capi.ERR_UNSUPPORTED),
    (dict(q=0), capi.ERR_INVALID_ARG), (dict(k=0), capi.ERR_INVALID_ARG), (dict(v=0), capi.ERR_INVALID_ARG),
    (dict(lens=0), capi.ERR_INVALID_ARG), (dict(out=0), capi.ERR_INVALID_ARG),
    (dict(q=A + 8), capi.ERR_MISALIGNED), (dict(k=A + 2), capi.ERR_MISALIGNED), (dict(out=A + 4), capi.ERR_MISALIGNED),
    (dict(q_stride=1023), capi.ERR_INVALID_ARG), (dict(q_stride=1028), capi.ERR_MISALIGNED),
    (dict(kv_stride=128), capi.ERR_INVALID_ARG), (dict(out_stride=-8), capi.ERR_INVALID_ARG),
    (dict(seq_stride=-8), capi.ERR_INVALID_ARG), (dict(seq_stride=12), capi.ERR_MISALIGNED),
    (dict(scale=-1.0), capi.ERR_INVALID_ARG), (dict(scale=float("nan")), capi.ERR_INVALID_ARG),
    (dict(scale=float("inf")), capi.ERR_INVALID_ARG),
    (dict(rows=A), capi.ERR_INVALID_ARG), (dict(k_new=A), capi.ERR_INVALID_ARG), (dict(parents=A), capi.ERR_INVALID_ARG),
    (dict(k_new=A, v_new=A, tokens=129), capi.ERR_UNSUPPORTED), (dict(k_new=A, v_new=A, weights=A), capi.ERR_INVALID_ARG),
    (dict(weights_in=A), capi.ERR_INVALID_ARG), (dict(weights=A, lse=0, tokens=9), capi.ERR_INVALID_ARG),
])
def test_attention_refuses(change, code):
    a = _attn(**change)
    assert _code(capi.attention_tree_workspace, a) == code
    assert _code(capi.attention_tree, a, A, 1 << 40) == code


def test_attention_workspace():
    """A function of the sizes: nothing for one split, more with splits and stored scores; too little of it is refused."""
    assert capi.attention_tree_workspace(_attn(max_seq=200)) == 0
    long = _attn(max_seq=8192)
    need = capi.attention_tree_workspace(long)
    assert need > 0 and need == capi.attention_tree_workspace(_attn(max_seq=8192, q=2 * A))
    assert capi.attention_tree_workspace(_attn(max_seq=8192, tokens=1, weights=A)) > \
        capi.attention_tree_workspace(_attn(max_seq=8192, tokens=1))
    assert _code(capi.attention_tree, long, A, need - 1) == capi.ERR_INVALID_ARG
    assert _code(capi.attention_tree, long, 0, need) == capi.ERR_INVALID_ARG
    assert _code(capi.attention_tree, long, A + 16, need) == capi.ERR_MISALIGNED
    assert capi.lib().swapnet_attention_tree_workspace(None, None) == capi.ERR_INVALID_ARG
    assert capi.lib().swapnet_attention_tree(None, None, 0, None) == capi.ERR_INVALID_ARG
    assert capi.lib().swapnet_attention_weights(None, None) == capi.ERR_INVALID_ARG
    assert capi.lib().swapnet_cache_evict(None, None) == capi.ERR_INVALID_ARG
    assert capi.lib().swapnet_tree_accept(None, None) == capi.ERR_INVALID_ARG


@pytest.mark.parametrize("change,code", [
    (dict(lse=0), capi.ERR_INVALID_ARG), (dict(weights=0), capi.ERR_INVALID_ARG), (dict(k_new=A, v_new=A), capi.ERR_INVALID_ARG),
    (dict(parents=A), capi.ERR_INVALID_ARG), (dict(dtype="f32"), capi.ERR_UNSUPPORTED), (dict(q=A + 8), capi.ERR_MISALIGNED),
])
def test_weights_refuse(change, code):
    assert _code(capi.attention_weights, _attn(**{"weights": A, **change})) == code


def _evict(**kw):
    base = dict(dtype="f16", n_seq=2, kv_heads=2, head_dim=64, max_seq=100, keep=50, recent=10, sink=4, k=A, v=2 * A,
                weights=3 * A, lens=4 * A, k_out=5 * A, v_out=6 * A, weights_out=7 * A, kept=8 * A, lens_out=9 * A)
    base.update(kw)
    return capi.cache_evict(**base)


@pytest.mark.parametrize("change,code", [
    (dict(dtype="f32"), capi.ERR_UNSUPPORTED), (dict(keep=0), capi.ERR_INVALID_ARG), (dict(head_dim=60), capi.ERR_UNSUPPORTED),
    (dict(recent=47), capi.ERR_INVALID_ARG), (dict(recent=-1), capi.ERR_INVALID_ARG), (dict(sink=-1), capi.ERR_INVALID_ARG),
    (dict(kept=0), capi.ERR_INVALID_ARG), (dict(weights=0), capi.ERR_INVALID_ARG), (dict(lens_out=4 * A), capi.ERR_INVALID_ARG),
    (dict(out_capacity=49), capi.ERR_INVALID_ARG), (dict(k_out=A), capi.ERR_INVALID_ARG),
    (dict(k_out=A, v_out=2 * A, weights_out=3 * A, out_capacity=50), capi.ERR_INVALID_ARG),
    (dict(v_out=5 * A), capi.ERR_INVALID_ARG), (dict(k=A + 8), capi.ERR_MISALIGNED), (dict(kv_stride=132), capi.ERR_MISALIGNED),
    (dict(kv_stride=120), capi.ERR_INVALID_ARG), (dict(out_seq_stride=-8), capi.ERR_INVALID_ARG),
    (dict(max_seq=1 << 28, keep=1 << 28), capi.ERR_UNSUPPORTED),
])
def test_eviction_refuses(change, code):
    assert _code(_evict, **change) == code


def _accept(**kw):
    base = dict(dtype="f16", n_seq=2, tokens=8, width=64, max_seq=100, ids=A, targets=A, lens=A, caches=np.array([A]),
                drafts=np.array([A]), path=A, accepted=A, next=A, lens_out=2 * A)
    base.update(kw)
    return capi.tree_accept(**base)


@pytest.mark.parametrize("change,code", [
    (dict(dtype="f32"), capi.ERR_UNSUPPORTED), (dict(tokens=0), capi.ERR_INVALID_ARG), (dict(tokens=129), capi.ERR_UNSUPPORTED),
    (dict(width=60), capi.ERR_UNSUPPORTED), (dict(ids=0), capi.ERR_INVALID_ARG), (dict(next=0), capi.ERR_INVALID_ARG),
    (dict(lens_out=A), capi.ERR_INVALID_ARG), (dict(width=1 << 25), capi.ERR_UNSUPPORTED), (dict(caches=np.array([0])), capi.ERR_INVALID_ARG),
    (dict(caches=np.array([A + 8])), capi.ERR_MISALIGNED), (dict(cache_stride=32), capi.ERR_INVALID_ARG),
    (dict(new_stride=68), capi.ERR_MISALIGNED),
    (dict(caches=np.full(257, A), drafts=np.full(257, A)), capi.ERR_UNSUPPORTED),
])
def test_acceptance_refuses(change, code):
    assert _code(_accept, **change) == code


@pytest.mark.parametrize("change", [{}, dict(path=2 * A), dict(path=2 * A, accepted=3 * A),
                                    dict(path=2 * A, accepted=3 * A, next=4 * A, lens_out=5 * A, counts=3 * A),
                                    dict(path=2 * A, accepted=3 * A, next=4 * A, lens_out=5 * A, parents=2 * A)])
def test_acceptance_refuses_results_over_inputs(change):
    assert _code(_accept, **change) == capi.ERR_INVALID_ARG


def test_acceptance_needs_a_draft_per_cache():
    with pytest.raises(ValueError):
        _accept(caches=np.array([A, A]))


# --------------------------------------------------- decoders with the flags
def _llm(**kw):
    import synth
    return synth.arch.llm(layers=2, d=256, heads=2, ffn=688, vocab=1000, max_seq=90, **kw)


def test_state_layout():
    """The caches stay where they were; what the flags add lies behind them and nothing overlaps."""
    base = capi.Plan.resident(capi.Desc(_llm(tokens=4)))
    tree = capi.Plan.resident(capi.Desc(_llm(tokens=4, tree=True)))
    both = capi.Plan.resident(capi.Desc(_llm(tokens=4, tree=True, weights=True)))
    weigh = capi.Plan.resident(capi.Desc(_llm(tokens=9, weights=True)))
    cache = (90 * 256 * 2 + 255) // 256 * 256
    assert base.info()["state_bytes"] == 256 + 4 * cache
    l0, l1, l2, l3 = (p.state_layout() for p in (base, tree, both, weigh))
    assert l0 == dict(caches=256, cache_bytes=cache, weights=0, tree_count=0, tree_parents=0, tree_path=0, layers=2)
    for lay, p in ((l1, tree), (l2, both), (l3, weigh)):
        assert lay["caches"] == 256 and lay["cache_bytes"] == cache and lay["layers"] == 2
        assert p.info()["state_bytes"] > 256 + 4 * cache
    assert l1["weights"] == 0 and l2["weights"] == l3["weights"] == 256 + 4 * cache
    assert l3["tree_count"] == 0 and l2["tree_count"] >= l2["weights"] + 2 * 2 * 2 * 90 * 4
    assert l1["tree_count"] < l1["tree_parents"] < l1["tree_path"] and (l1["tree_parents"] - l1["tree_count"]) % 256 == 0


@pytest.mark.parametrize("change,code", [
    (dict(tokens=129, tree=True), capi.ERR_UNSUPPORTED),
    (dict(tokens=4, tree=True, heads=4), capi.ERR_UNSUPPORTED),  # head width 64
    (dict(tokens=4, weights=True, heads=1), capi.ERR_UNSUPPORTED),
])
def test_flags_that_no_kernel_takes(change, code):
    import synth
    cfg = dict(layers=2, d=256, heads=2, ffn=688, vocab=1000, max_seq=90)
    cfg.update(change)
    assert _code(capi.Plan.resident, capi.Desc(synth.arch.llm(**cfg))) == code


def test_flags_are_the_same_on_every_layer():
    m = _llm(tokens=4)
    att = [L for L in m["layers"] if L["op"] == "attention"]
    att[0]["weights"] = True
    assert _code(capi.Plan.resident, capi.Desc(m)) == capi.ERR_INVALID_ARG
    att[1]["weights"] = True
    att[1]["max_seq"] = 91
    assert _code(capi.Plan.resident, capi.Desc(m)) == capi.ERR_INVALID_ARG
    att[1]["max_seq"] = 90
    assert capi.Plan.resident(capi.Desc(m)).state_layout()["weights"] > 0
    assert capi.lib().swapnet_plan_state_layout(None, None) == capi.ERR_INVALID_ARG
    assert capi.lib().swapnet_engine_tree_accept(None, None, None, None) == capi.ERR_INVALID_ARG
    assert capi.lib().swapnet_engine_evict(None, 1, 0, 0, None) == capi.ERR_INVALID_ARG


def test_argument_blocks_have_the_header_layout():
    """The blocks are packed in one step: every value lands in the field of its name."""
    import ctypes as C

    from paper_2401_16757_gb300 import _capi

    for form, block in ((_capi._ATTENTION, _capi.CachedAttention), (_capi._EVICTION, _capi.CacheEviction),
                        (_capi._ACCEPTANCE, _capi.TreeAcceptance)):
        assert form.size == C.sizeof(block)
    names = [n for n, _ in _capi.CachedAttention._fields_]
    a = capi.cached_attention(**{n: i + 1 for i, n in enumerate(names)})
    assert [getattr(a, n) for n in names] == [i + 1 for i in range(len(names))]


@pytest.mark.parametrize("scale", [2.5e38, 3.4e38])
def test_a_scale_beyond_the_base_two_scores_is_refused(scale):
    """The kernels scale by log2(e) times as much: beyond fp32 a score of 0 would become NaN."""
    assert _code(capi.attention_tree, _attn(scale=scale), A, 1 << 40) == capi.ERR_INVALID_ARG
    assert _code(capi.attention_weights, _attn(scale=scale, weights=A)) == capi.ERR_INVALID_ARG
    assert capi.attention_tree_workspace(_attn(scale=2.3e38)) == 0


@pytest.mark.parametrize("off", [1, 2, 3])
def test_index_and_float_arrays_off_their_four_bytes_are_refused(off):
    """Single elements of them are loaded: an address between two would fault on the device."""
    for name in ("lens", "counts", "lse"):
        assert _code(capi.attention_tree, _attn(**{name: A + off}), A, 1 << 40) == capi.ERR_MISALIGNED, name
    assert _code(capi.attention_tree, _attn(k_new=A, v_new=A, parents=A + off), A, 1 << 40) == capi.ERR_MISALIGNED
    for name in ("weights", "weights_in"):
        assert _code(capi.attention_tree, _attn(**{"weights": A, name: A + off}), A, 1 << 40) == capi.ERR_MISALIGNED, name
    for name in ("lens", "counts", "lse", "rows", "weights", "weights_in"):
        assert _code(capi.attention_weights, _attn(**{"weights": A, name: A + off})) == capi.ERR_MISALIGNED, name
    for name in ("weights", "lens", "weights_out", "kept", "lens_out"):
        assert _code(_evict, **{name: 16 * A + off}) == capi.ERR_MISALIGNED, name
    good = dict(path=2 * A, accepted=3 * A, next=4 * A, lens_out=5 * A)
    for name in ("ids", "targets", "lens", "parents", "counts", "path", "accepted", "next", "lens_out"):
        assert _code(_accept, **{**good, name: 16 * A + off}) == capi.ERR_MISALIGNED, name


def _apart(**kw):
    """An attention call whose operands all lie apart."""
    base = dict(q=1 * A, k=2 * A, v=3 * A, lens=4 * A, out=5 * A, lse=6 * A, max_seq=200)
    base.update(kw)
    return _attn(**base)


@pytest.mark.parametrize("change", [dict(out=1 * A), dict(out=2 * A), dict(out=3 * A), dict(out=4 * A), dict(lse=1 * A), dict(lse=5 * A),
                                    dict(k_new=5 * A, v_new=8 * A), dict(k_new=8 * A, v_new=9 * A, parents=6 * A), dict(counts=5 * A),
                                    dict(weights=1 * A), dict(weights=6 * A), dict(weights=8 * A, weights_in=5 * A)])
def test_attention_refuses_results_over_inputs(change):
    """CTAs read the inputs while others write the results."""
    assert _code(capi.attention_tree, _apart(**change), 20 * A, 1 << 40) == capi.ERR_INVALID_ARG


def test_attention_refuses_a_workspace_that_is_an_operand():
    long = dict(max_seq=8192)
    assert capi.attention_tree_workspace(_apart(**long)) > 0
    for at in (1, 2, 3, 4, 5, 6):
        assert _code(capi.attention_tree, _apart(**long), at * A, 1 << 40) == capi.ERR_INVALID_ARG


@pytest.mark.parametrize("at", [1, 2, 4, 6, 8])
def test_weights_refuse_results_over_inputs(at):
    assert _code(capi.attention_weights, _apart(weights=at * A, rows=8 * A)) == capi.ERR_INVALID_ARG


@pytest.mark.parametrize("change", [dict(k_out=2 * A), dict(v_out=1 * A), dict(k_out=3 * A), dict(weights_out=1 * A), dict(kept=4 * A),
                                    dict(kept=9 * A), dict(kept=3 * A), dict(lens_out=5 * A), dict(kept=7 * A)])
def test_eviction_refuses_results_over_other_operands(change):
    assert _code(_evict, **change) == capi.ERR_INVALID_ARG


@pytest.mark.parametrize("change", [dict(path=3 * A), dict(accepted=4 * A), dict(next=5 * A), dict(lens_out=2 * A)])
def test_acceptance_refuses_results_over_results(change):
    assert _code(_accept, **{**dict(path=2 * A, accepted=3 * A, next=4 * A, lens_out=5 * A), **change}) == capi.ERR_INVALID_ARG
