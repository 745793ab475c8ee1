"""Sizes of quantised-attention calls that run each of its kernels, with a CTA
per unit and in equal runs of tiles, far from where the choice changes."""
from paper_2401_16757_gb300 import capi

# name: (n_seq, tokens, heads, kv_heads, head_dim, max_seq), (kernel, rows of a unit, shared)
WAYS = {
    "warp 8, 128": ((3, 1, 8, 2, 128, 300), ("warp", 8, False)),
    "warp 8, 128, runs": ((3, 2, 8, 2, 128, 4000), ("warp", 8, True)),
    "warp 8, 64": ((3, 4, 2, 1, 64, 300), ("warp", 8, False)),
    "warp 8, 64, runs": ((3, 1, 8, 2, 64, 4000), ("warp", 8, True)),
    "warp 16, 128": ((3, 12, 1, 1, 128, 300), ("warp", 16, False)),
    "warp 16, 128, runs": ((3, 4, 8, 2, 128, 4000), ("warp", 16, True)),
    "warp 16, 64": ((3, 5, 6, 2, 64, 300), ("warp", 16, False)),
    "warp 16, 64, runs": ((3, 12, 1, 1, 64, 4000), ("warp", 16, True)),
    "warp 32, 128": ((40, 100, 1, 1, 128, 200), ("warp", 32, False)),
    "warp 32, 128, runs": ((3, 7, 8, 2, 128, 4000), ("warp", 32, True)),
    "warp 32, 64": ((3, 25, 2, 2, 64, 300), ("warp", 32, False)),
    "warp 32, 64, runs": ((3, 5, 5, 1, 64, 4000), ("warp", 32, True)),
    "keys": ((40, 25, 1, 1, 128, 700), ("keys", 32, False)),
    "keys, two units": ((3, 50, 2, 2, 128, 400), ("keys", 32, False)),
    "keys, runs": ((200, 8, 4, 1, 128, 4500), ("keys", 32, True)),
    "keys, runs, odd rows": ((100, 3, 14, 2, 128, 4500), ("keys", 32, True)),
    "rows 64, 128": ((100, 50, 1, 1, 128, 1500), ("rows", 64, False)),
    "rows 64, 128, runs": ((100, 13, 4, 1, 128, 7000), ("rows", 64, True)),
    "rows 64, 64": ((100, 13, 4, 1, 64, 1500), ("rows", 64, False)),
    "rows 64, 64, runs": ((100, 50, 1, 1, 64, 7000), ("rows", 64, True)),
    "rows 128, 128": ((100, 150, 1, 1, 128, 500), ("rows", 128, False)),
    "rows 128, 128, runs": ((40, 50, 4, 1, 128, 6000), ("rows", 128, True)),
    "rows 128, 64": ((100, 37, 4, 1, 64, 500), ("rows", 128, False)),
    "rows 128, 64, runs": ((40, 200, 1, 1, 64, 6000), ("rows", 128, True)),
}


def tiling(args):
    t = capi.attention_quantized_tiling(args)
    return t["kernel"], t["rows"], t["shared"]
