"""The coding of rows into pages bit for bit where it takes other ways: keys that turn over a part or all of a head (by nothing, which leaves every
finite number as it is), rows that share a workgroup in odd numbers, and magnitudes at both ends of float32."""
import numpy as np
import pytest
import torch

from oracle import paged
from test_gpu_paged import TD, dev, make, rows_of, tables, yoco  # noqa: F401

pytestmark = pytest.mark.gpu


def coded(c, n, Hkv, d):
    return paged.read_pool(c.mem.cpu().numpy(), n, Hkv, d, True)


@pytest.mark.parametrize("src", ["bf16", "f32"])
@pytest.mark.parametrize("d,dims,neighbours", [(128, 128, False), (128, 112, False), (128, 96, False), (128, 80, False), (128, 64, False), (128, 16, False), (128, 128, True), (128, 96, True),
                                               (64, 64, False), (64, 48, False), (64, 64, True)])
@pytest.mark.parametrize("Hkv,B,T,pos", [(3, 2, 1, [5, 64]), (1, 2, 7, [0, 61]), (5, 1, 150, [3]), (2, 3, 13, [16, 3, 120])])
def test_rows_that_turn_by_nothing_keep_their_codes(yoco, d, dims, neighbours, Hkv, B, T, pos, src):  # noqa: F811
    rng = np.random.default_rng(d + dims + T)
    table, n = tables(rng, B, 4)
    c = make(yoco, "int4", n, Hkv, d)
    k, v = rows_of(rng, (B, T, Hkv, d), src), rows_of(rng, (B, T, Hkv, d), src)
    size = np.exp2(rng.integers(-148, 120, (B, T, Hkv, 1)).astype(np.float64))          # down to where all of a group is one value, up to where ranges overflow
    k[..., : d // 2] = np.clip(k[..., : d // 2] * size, -3.3e38, 3.3e38).astype(np.float32)
    k = paged.bf16(k) if src == "bf16" else k
    yoco.paged_append(c, dev(table), dev(np.array(pos)), dev(k, TD[src]), dev(v, TD[src]), turns=torch.zeros(dims // 2, dtype=torch.int64, device="cuda"), neighbours=neighbours)
    for x, got in zip((k, v), coded(c, n, Hkv, d)):
        codes, scale, base = paged.code(x)
        for b in range(B):
            for t in range(T):
                at = pos[b] + t
                page, r = table[b, at // 64], at % 64
                for a, w in zip(got, (codes[b, t], scale[b, t], base[b, t])):
                    assert np.array_equal(a[page, :, r], w, equal_nan=a.dtype.kind == "f"), (b, t)
