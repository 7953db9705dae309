"""Attention over pages where the call may expect much work: long tables (of which the sequences fill little) and many rows of the query, which
workgroups of eight wavefronts and of two tiles of columns have. The bounds are those of the other shapes."""
import math

import numpy as np
import pytest
import torch

from oracle import paged
from test_gpu_paged import check, dev, filled, host, yoco  # noqa: F401

pytestmark = pytest.mark.gpu

SHAPES = [                        # B, T, N, Hq, Hkv, d, lens, columns of the table
    (3, 1, 3000, 32, 8, 128, [3000, 64, 1999], 200),
    (3, 1, 3000, 32, 8, 128, [0, 1, 2999], 200),
    (2, 2, 2500, 8, 2, 128, [2500, 1], 1100),              # 8 columns
    (2, 4, 2500, 8, 2, 64, [2011, 65], 1100),              # 16
    (1, 1, 20000, 12, 4, 64, [20000], 1100),
    (2, 6, 700, 8, 2, 128, [700, 65], 9000),               # 24 columns: a tile and a half
    (3, 10, 300, 8, 2, 128, [300, 0, 9], 3000),            # 40, and rows before the first position
    (2, 20, 1000, 4, 1, 64, [1000, 63], 6000),             # 80
    (1, 1, 5000, 32, 1, 128, [5000], 33000),               # 32: one row
    (1, 17, 20000, 2, 1, 128, [20000], 20000),             # 34, in many parts
    (2, 33, 64, 1, 1, 64, [64, 33], 17000),                # 33: a row in the second of two tiles
    (1, 32, 20000, 64, 8, 64, [20000], 20000),             # ranges of pages of equal length, over several tiles
]


@pytest.mark.parametrize("cache", ["int4", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(x) for x in s[:6]))
def test_attention_with_long_tables(yoco, shape, cache):  # noqa: F811
    B, T, N, Hq, Hkv, d, lens, cols = shape
    rng = np.random.default_rng(B + N + Hq + T)
    c, table, k, v = filled(yoco, rng, cache, B, N, Hkv, d)
    long = np.full((B, cols), -1, np.int32)
    long[:, :table.shape[1]] = table
    q = paged.bf16(rng.standard_normal((B, T, Hq, d)).astype(np.float32))
    scale, t, n = 1.0 / math.sqrt(d), dev(long), dev(np.array(lens))
    ws = torch.full((max(yoco.paged_attn_workspace(c, B, cols, T, Hq), 16) // 4,), float("nan"), device="cuda")
    o = yoco.paged_attn(c, t, dev(q, torch.bfloat16), n, scale, workspace=ws)
    for b in range(B):
        check(host(o[b]), q[b], k[b], v[b], lens[b], scale, "%s sequence %d" % (cache, b))
    for _ in range(3):                                       # the same bits again
        assert torch.equal(yoco.paged_attn(c, t, dev(q, torch.bfloat16), n, scale, workspace=ws), o)


@pytest.mark.parametrize("cache", ["int4", "bf16"])
def test_many_rows_where_pages_are_missing(yoco, cache):  # noqa: F811
    rng = np.random.default_rng(8)
    c, table, k, v = filled(yoco, rng, cache, 1, 900, 2, 128)
    table[0, [0, 5, 14]] = [-1, c.n_pages, -7]
    k[0][:, np.isin(np.arange(900) // 64, [0, 5, 14])] = np.nan
    long = np.full((1, 20000), 1 << 30, np.int32)
    long[:, :table.shape[1]] = table
    q = paged.bf16(rng.standard_normal((1, 12, 8, 128)).astype(np.float32))
    o = yoco.paged_attn(c, dev(long), dev(q, torch.bfloat16), dev(np.array([900])), 0.09)
    check(host(o[0]), q[0], k[0], v[0], 900, 0.09, cache)
