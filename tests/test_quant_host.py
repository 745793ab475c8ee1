"""Refusals and workspace sizes of the quantised-cache calls: decided on the
host, before anything is launched, so they need no GPU."""
import ctypes as C

import pytest

from paper_2401_16757_gb300 import capi

from quant_ways import WAYS, tiling

A = 1 << 20  # an aligned address; nothing is read from it


def _at(i):
    return A + 4096 * i


def _rows(**kw):
    """Arguments of cache_append that are in order (addresses that differ), with changes."""
    base = dict(dtype="bf16", cache_dtype="e4m3", n_seq=2, tokens=4, heads=8, kv_heads=2, head_dim=128, max_seq=100,
                k_new=_at(1), v_new=_at(2), lens=_at(3), k=_at(4), v=_at(5), q=_at(6), q_out=_at(7), k_scale=_at(8), v_scale=_at(9),
                k_open=_at(10), v_open=_at(11), block=32, theta=10000.0, eps=1e-6)
    base.update(kw)
    return base


def _attn(**kw):
    base = dict(dtype="bf16", cache_dtype="i8", n_seq=2, tokens=4, heads=8, kv_heads=2, head_dim=128, max_seq=100, block=32,
                q=_at(1), k=_at(2), v=_at(3), k_scale=_at(4), v_scale=_at(5), lens=_at(6), out=_at(7), lse=_at(8))
    base.update(kw)
    return capi.quantized_attention(**base)


def _code(call, *a, **kw):
    with pytest.raises(capi.SwapnetError) as e:
        call(*a, **kw)
    assert str(e.value)
    return e.value.code


INVALID, UNSUPPORTED, MISALIGNED = capi.ERR_INVALID_ARG, capi.ERR_UNSUPPORTED, capi.ERR_MISALIGNED
PLAIN = dict(cache_dtype="bf16", block=0, k_scale=0, v_scale=0, k_open=0, v_open=0)  # a 16-bit cache


@pytest.mark.parametrize("change,code", [
    (dict(dtype="f32"), UNSUPPORTED), (dict(cache_dtype="f16"), UNSUPPORTED), (dict(cache_dtype="f32"), UNSUPPORTED),
    (dict(cache_dtype="i32"), UNSUPPORTED), (dict(n_seq=0), INVALID), (dict(tokens=0), INVALID), (dict(kv_heads=0), INVALID),
    (dict(heads=-1), INVALID), (dict(max_seq=0), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(block=0), UNSUPPORTED),
    (dict(block=24), UNSUPPORTED), (dict(block=256), UNSUPPORTED), (dict(n_seq=70000), UNSUPPORTED),
    (dict(max_seq=(1 << 24) + 1), UNSUPPORTED), (dict(n_seq=60000, tokens=30000), UNSUPPORTED),
    (dict(k_new=0), INVALID), (dict(v_new=0), INVALID), (dict(lens=0), INVALID), (dict(k=0), INVALID), (dict(v=0), INVALID),
    (dict(q=0), INVALID), (dict(q_out=0), INVALID), (dict(heads=0), INVALID), (dict(heads=0, q=0, q_out=0, q_gain=_at(12)), INVALID),
    (dict(k_scale=0), INVALID), (dict(v_scale=0), INVALID), (dict(k_open=0), INVALID), (dict(v_open=0), INVALID),
    (dict(k_open_out=_at(12)), INVALID), (dict(v_open_out=_at(12)), INVALID),
    (dict(k_open_out=_at(10), v_open_out=_at(12)), INVALID), (dict(k_open_out=_at(11), v_open_out=_at(10)), INVALID),
    (dict(theta=-1.0), INVALID), (dict(theta=float("inf")), INVALID), (dict(theta=float("nan")), INVALID),
    (dict(theta=1e-30), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(rope_dim=8), UNSUPPORTED), (dict(rope_dim=144), UNSUPPORTED), (dict(rope_dim=40), UNSUPPORTED),
    (dict(rope_dim=-16), UNSUPPORTED), (dict(sections=(16, 24, 23)), INVALID), (dict(sections=(-1, 33, 32)), INVALID),
    (dict(theta=0.0, positions=_at(12)), INVALID),
    (dict(q_stride=1016), INVALID), (dict(q_stride=1028), MISALIGNED), (dict(out_stride=512), INVALID),
    (dict(new_stride=128), INVALID), (dict(new_stride=260), MISALIGNED), (dict(kv_stride=240), INVALID),
    (dict(kv_stride=264), MISALIGNED), (dict(seq_stride=-16), INVALID), (dict(seq_stride=24), MISALIGNED),
    (dict(q=_at(6) + 8), MISALIGNED), (dict(k=_at(4) + 8), MISALIGNED), (dict(v_new=_at(2) + 2), MISALIGNED),
    (dict(q_gain=_at(12) + 4), MISALIGNED), (dict(k_open=_at(10) + 8), MISALIGNED), (dict(lens=_at(3) + 2), MISALIGNED),
    (dict(k_scale=_at(8) + 1), MISALIGNED), (dict(positions=_at(12) + 2), MISALIGNED), (dict(lens_out=_at(12) + 2), MISALIGNED),
    (dict(k=_at(5)), INVALID), (dict(k=_at(1)), INVALID), (dict(q_out=_at(1)), INVALID), (dict(lens_out=_at(3)), INVALID),
    (dict(k_scale=_at(9)), INVALID), (dict(k=_at(6)), INVALID), (dict(k_open=_at(1)), INVALID), (dict(k_open=_at(4)), INVALID),
    (dict(q_out=_at(6), out_stride=2048), INVALID),
    (dict(PLAIN, block=32), UNSUPPORTED), (dict(PLAIN, k_scale=_at(8)), INVALID), (dict(PLAIN, k_open=_at(8)), INVALID),
    (dict(PLAIN, kv_stride=260), MISALIGNED),
])
def test_append_refuses(change, code):
    assert _code(capi.cache_append, **_rows(**change)) == code


@pytest.mark.parametrize("change,code", [
    (dict(dtype="f32"), UNSUPPORTED), (dict(cache_dtype="bf16"), UNSUPPORTED), (dict(cache_dtype=9), UNSUPPORTED),
    (dict(n_seq=0), INVALID), (dict(tokens=0), INVALID), (dict(heads=0), INVALID), (dict(max_seq=0), INVALID),
    (dict(heads=7), INVALID), (dict(head_dim=80), UNSUPPORTED), (dict(block=0), UNSUPPORTED), (dict(block=48), UNSUPPORTED),
    (dict(n_seq=70000), UNSUPPORTED), (dict(n_seq=40000, tokens=30000), UNSUPPORTED), (dict(heads=258), UNSUPPORTED),
    (dict(tokens=(1 << 18) + 1), UNSUPPORTED), (dict(q=0), INVALID), (dict(k=0), INVALID), (dict(v=0), INVALID),
    (dict(k_scale=0), INVALID), (dict(v_scale=0), INVALID), (dict(lens=0), INVALID), (dict(out=0), INVALID),
    (dict(q=_at(1) + 8), MISALIGNED), (dict(k=_at(2) + 8), MISALIGNED), (dict(out=_at(7) + 4), MISALIGNED),
    (dict(k_scale=_at(4) + 2), MISALIGNED), (dict(lens=_at(6) + 1), MISALIGNED), (dict(lse=_at(8) + 2), MISALIGNED),
    (dict(q_stride=1016), INVALID), (dict(q_stride=1028), MISALIGNED), (dict(kv_stride=128), INVALID),
    (dict(kv_stride=264), MISALIGNED), (dict(seq_stride=-16), INVALID), (dict(seq_stride=40), MISALIGNED),
    (dict(out_stride=-8), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=3e38), INVALID),
])
def test_attention_refuses(change, code):
    a = _attn(**change)
    assert _code(capi.attention_quantized_workspace, a) == code
    assert _code(capi.attention_quantized, a, A, 1 << 40) == code


def test_attention_refuses_results_over_operands():
    for change in (dict(out=_at(1)), dict(out=_at(2)), dict(lse=_at(5)), dict(lse=_at(6)), dict(lse=_at(7))):
        assert _code(capi.attention_quantized, _attn(**change), A, 1 << 40) == INVALID
    long = _attn(max_seq=100000)
    assert _code(capi.attention_quantized, long, _at(2), 1 << 40) == INVALID


def test_attention_workspace():
    """A function of the sizes; too little of it is refused."""
    assert capi.attention_quantized_workspace(_attn(max_seq=100)) == 0
    long = _attn(max_seq=100000)
    need = capi.attention_quantized_workspace(long)
    assert need > 0 and need == capi.attention_quantized_workspace(_attn(max_seq=100000, q=2 * A, lse=0))
    assert _code(capi.attention_quantized, long, A, need - 1) == INVALID
    assert _code(capi.attention_quantized, long, 0, need) == INVALID
    assert _code(capi.attention_quantized, long, A + 16, need) == MISALIGNED
    lib = capi.lib()
    assert lib.swapnet_attention_quantized_workspace(None, None) == INVALID
    assert lib.swapnet_attention_quantized(None, None, 0, None) == INVALID
    assert lib.swapnet_cache_append(None, None) == INVALID


def test_argument_blocks_are_the_structs():
    assert C.sizeof(capi.CacheRows) == capi._ROWS.size and C.sizeof(capi.QuantizedAttention) == capi._QUANTIZED.size
    a = _attn(scale=0.5, out_stride=2048)
    assert (a.cache_dtype, a.block, a.scale, a.lse, a.out_stride) == (capi.I8, 32, 0.5, _at(8), 2048)


@pytest.mark.parametrize("way", sorted(WAYS))
@pytest.mark.parametrize("dtype,fmt,block", [("bf16", "i8", 16), ("f16", "e4m3", 128)])
def test_sizes_that_run_each_kernel(way, dtype, fmt, block):
    """What the tests of the kernels' edges rely on: a changed choice shows here."""
    (n, t, h, kv, d, cap), want = WAYS[way]
    a = _attn(dtype=dtype, cache_dtype=fmt, n_seq=n, tokens=t, heads=h, kv_heads=kv, head_dim=d, max_seq=cap, block=block)
    assert tiling(a) == want
    assert (capi.attention_quantized_workspace(a) > 0) == want[2]
    assert capi.attention_quantized_tiling(a)["ctas"] >= 1


def test_tiling_refuses():
    lib, t = capi.lib(), capi.QuantizedTiling()
    assert lib.swapnet_attention_quantized_tiling(None, C.byref(t)) == INVALID
    assert lib.swapnet_attention_quantized_tiling(C.byref(_attn()), None) == INVALID
    assert _code(capi.attention_quantized_tiling, _attn(block=24)) == UNSUPPORTED
