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
