"""The cache in pages on the GPU: rows as they are coded and placed, read back, and attended over, against plain numpy
definitions (float64, and float32 where a rounding decides a code).

Bounds. Rotation: the angle is the upper 32 bits of an exact one (2^-32 turns, then a float32 rounding of at most pi: 2.4e-7),
cosine and sine are good to an ulp, and a result is two products and a sum: |x| + |y| times 1e-6 holds with room. A code decides by
float32 arithmetic that is compared bit for bit where nothing is rotated. Attention: the output is rounded to bf16 (half an ulp, 2^-9 of it),
softmax weights times scales are rounded to fp16 or kept to 16 bits (2^-11 of a term, whose sizes add up to no more than twice
the largest |v|), sums are float32 (far below both)."""
import math

import numpy as np
import pytest
import torch

from oracle import paged

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def yoco():
    import paper_2405_05254_amd as y
    y.lib()                       # fails loudly if libyoco.so is not built
    assert torch.cuda.is_available()
    return y


def kind(yoco, cache):
    return yoco.INT4 if cache == "int4" else torch.bfloat16


def host(t):
    return t.detach().float().cpu().numpy()


def make(yoco, cache, n_pages, Hkv, d, fill=0xAB):
    c = yoco.PagedCache(n_pages, Hkv, d, kind(yoco, cache))
    c.mem.fill_(fill)
    return c


def tables(rng, B, cols, spare=2):
    n = B * cols + spare
    return rng.permutation(n)[:B * cols].reshape(B, cols).astype(np.int32), n


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def rows_of(rng, shape, src):
    x = (rng.standard_normal(shape) * np.exp2(rng.integers(-6, 6, shape[:-1]))[..., None]).astype(np.float32)
    x.reshape(-1, shape[-1])[0] = 0.0
    return paged.bf16(x) if src == "bf16" else x


# ------------------------------------------------------------ rows into pages
@pytest.mark.parametrize("cache", ["int4", "bf16"])
@pytest.mark.parametrize("src", ["bf16", "f32"])
@pytest.mark.parametrize("d,Hkv,B,T,pos", [(128, 2, 1, 1, [0]), (128, 3, 3, 1, [63, 64, 200]), (64, 5, 2, 1, [127, 7]), (128, 1, 2, 70, [0, 33]), (64, 2, 2, 130, [65, 1]), (128, 8, 1, 256, [64])])
def test_rows_are_placed_and_coded_exactly(yoco, cache, src, d, Hkv, B, T, pos):
    rng = np.random.default_rng(d + Hkv + T)
    cols = 7
    table, n = tables(rng, B, cols)
    c = make(yoco, cache, n, Hkv, d)
    before = paged.read_pool(c.mem.cpu().numpy(), n, Hkv, d, cache == "int4")
    k, v = rows_of(rng, (B, T, Hkv, d), src), rows_of(rng, (B, T, Hkv, d), src)
    rows = [T - 3 * b if T > 3 * b else T for b in range(B)]
    yoco.paged_append(c, dev(table), dev(np.array(pos)), dev(k, TD[src]), dev(v, TD[src]), rows=dev(np.array(rows)))
    after = paged.read_pool(c.mem.cpu().numpy(), n, Hkv, d, cache == "int4")
    for x, old, new in zip((k, v), before, after):
        want = [a.copy() for a in old] if cache == "int4" else old.copy()
        codes, scale, base = paged.code(x)
        for b in range(B):
            for t in range(rows[b]):
                at = pos[b] + t
                page, r = table[b, at // 64], at % 64
                if cache == "int4":
                    want[0][page, :, r], want[1][page, :, r], want[2][page, :, r] = codes[b, t], scale[b, t], base[b, t]
                else:
                    want[page, :, r] = paged.bf16(x[b, t])
        for a, w in zip(new if cache == "int4" else (new,), want if cache == "int4" else (want,)):
            assert np.array_equal(a, w, equal_nan=a.dtype.kind == "f")          # bytes of other rows stay as they were
    # and the values that a program reads back
    gk, gv = yoco.paged_read(c, dev(table), dev(np.array(pos)), T, dtype=torch.float32)
    for x, got in ((k, host(gk)), (v, host(gv))):
        want = paged.stands_for(*paged.code(x)) if cache == "int4" else paged.bf16(x)
        for b in range(B):
            assert np.array_equal(got[b, :rows[b]], want[b, :rows[b]].astype(np.float32))
    bk, _ = yoco.paged_read(c, dev(table), dev(np.array(pos)), T)
    assert torch.equal(bk, gk.bfloat16())


@pytest.mark.parametrize("cache", ["int4", "bf16"])
def test_groups_that_are_not_finite(yoco, cache):
    c = make(yoco, cache, 1, 1, 128)
    x = np.ones((1, 6, 1, 128), np.float32)
    x[0, 0, 0, 5], x[0, 1, 0, 70], x[0, 2, 0, 0], x[0, 2, 0, 1], x[0, 4, 0, 127] = np.inf, np.nan, 3e38, -3e38, -np.inf
    x[0, 5, 0, :64] = np.linspace(1e-39, 2e-39, 64)                             # a range below the normal numbers
    table, pos = dev(np.zeros((1, 1), np.int32)), dev(np.zeros(1, np.int64))
    yoco.paged_append(c, table, pos, dev(x), dev(x))
    for got in yoco.paged_read(c, table, pos, 6, dtype=torch.float32):
        got = host(got)
        if cache == "int4":
            want = paged.stands_for(*paged.code(x))
            assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(got).sum() == 4 * 64
            assert np.allclose(got, want, atol=1e-38, rtol=0, equal_nan=True)
        else:
            assert np.array_equal(got[:, :5], paged.bf16(x)[:, :5], equal_nan=True)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("src", ["bf16", "f32"])
@pytest.mark.parametrize("cache", ["int4", "bf16"])
@pytest.mark.parametrize("d,dims,Hq,Hkv,pos,T", [(128, 128, 6, 2, [0, 1000003], 1), (128, 64, 3, 3, [5, 700], 67), (64, 64, 8, 1, [524287 - 40, 0], 33), (64, 16, 1, 1, [3, 9], 2)])
def test_rotation(yoco, d, dims, Hq, Hkv, pos, T, cache, src, neighbours):
    rng = np.random.default_rng(d + dims + T)
    B, cols = 2, max((p + T + 63) // 64 for p in pos)
    table = np.full((B, cols), -1, np.int32)                                    # only the pages that are met exist
    used = sorted({(b, (pos[b] + t) // 64) for b in range(B) for t in range(T)})
    for i, (b, col) in enumerate(used):
        table[b, col] = i
    c = make(yoco, cache, len(used), Hkv, d)
    # views of one joined product, as a program has them
    joined = dev(rng.standard_normal((B, T, Hq + 2 * Hkv, d)).astype(np.float32), TD[src])
    q, k, v = joined.split([Hq, Hkv, Hkv], 2)
    got = yoco.paged_append(c, dev(table), dev(np.array(pos)), k, v, q=q, turns=yoco.rotation_turns(dims, 10000.0), neighbours=neighbours)
    gk, gv = (host(x) for x in yoco.paged_read(c, dev(table), dev(np.array(pos)), T, dtype=torch.float32))
    units = paged.turns([10000.0 ** (-2.0 * p / dims) for p in range(dims // 2)])
    q, k, v, got = host(q), host(k), host(v), host(got)
    round_off = 2.0 ** -8 if src == "bf16" else 0.0
    for b in range(B):
        for t in range(T):
            want = paged.rotate(q[b, t], pos[b] + t, units, neighbours)
            assert (np.abs(got[b, t] - want) <= round_off * np.abs(want) + 1e-6 * 2 * np.abs(q[b, t]).max()).all()
            want = paged.rotate(k[b, t], pos[b] + t, units, neighbours)
            if cache == "bf16":
                bound = 2.0 ** -8 * np.abs(want)
            else:
                g = want.reshape(Hkv, -1, 64)
                step = (g.max(-1) - g.min(-1)) / 15
                bound = np.broadcast_to((0.5 * step + 15 * 2.0 ** -9 * step + 2.0 ** -8 * np.abs(g.min(-1)))[..., None], g.shape).reshape(want.shape)
            assert (np.abs(gk[b, t] - want) <= bound + 1e-5).all()
    assert np.array_equal(gv, (paged.stands_for(*paged.code(v)) if cache == "int4" else paged.bf16(v)).astype(np.float32))


def test_queries_are_turned_in_place(yoco):
    c = make(yoco, "int4", 4, 2, 128)
    table, pos = dev(np.arange(4, dtype=np.int32).reshape(2, 2)), dev(np.array([3, 70]))
    k = torch.randn(2, 5, 2, 128, device="cuda", dtype=torch.bfloat16)
    q = torch.randn(2, 5, 6, 128, device="cuda", dtype=torch.bfloat16)
    want = yoco.paged_append(c, table, pos, k, k, q=q, turns=yoco.rotation_turns(128))
    again = q.clone()
    assert yoco.paged_append(c, table, pos, k, k, q=again, turns=yoco.rotation_turns(128), q_out=again) is again
    assert torch.equal(again, want) and not torch.equal(q, want)
    assert torch.equal(yoco.paged_append(c, table, pos, k, k, q=q), q)          # no rotation: a copy


@pytest.mark.parametrize("cache", ["int4", "bf16"])
def test_rows_without_a_page_are_left_out(yoco, cache):
    c = make(yoco, cache, 2, 1, 64)
    table = dev(np.array([[0, -1, 7], [1, 2, 1 << 30]], np.int32))              # two pages exist
    k = torch.randn(2, 192, 1, 64, device="cuda", dtype=torch.bfloat16)
    yoco.paged_append(c, table, dev(np.array([0, 0])), k, k)
    untouched = c.mem.clone()
    yoco.paged_append(c, table, dev(np.array([64, -130])), k[:, :128].contiguous(), k[:, :128].contiguous())      # no page, and before the first row
    yoco.paged_append(c, table, dev(np.array([192, 1 << 40])), k, k)                                              # behind the table
    assert torch.equal(c.mem, untouched)
    got, _ = yoco.paged_read(c, table, dev(np.array([-3, 60])), 8)
    own, _ = yoco.paged_read(c, table, dev(np.array([0, 60])), 5)
    assert (got[0, :3] == 0).all() and torch.equal(got[0, 3:], own[0]) and torch.equal(got[1, :4], own[1, :4]) and (got[1, 4:] == 0).all()


def test_nothing_to_append(yoco):
    c = make(yoco, "int4", 1, 1, 128)
    before = c.mem.clone()
    table, pos = dev(np.zeros((1, 1), np.int32)), dev(np.zeros(1, np.int64))
    k = torch.randn(1, 3, 1, 128, device="cuda")
    yoco.paged_append(c, table, pos, k[:, :0], k[:, :0])
    yoco.paged_append(c, table, pos, k, k, rows=dev(np.zeros(1, np.int64)))
    assert torch.equal(c.mem, before)
    assert yoco.paged_read(c, table, pos, 0)[0].shape == (1, 0, 1, 128)
    q = torch.empty(1, 0, 4, 128, device="cuda", dtype=torch.bfloat16)
    assert yoco.paged_attn(c, table, q, pos, 1.0).shape == q.shape


# ------------------------------------------------------------ attention over the pages
def filled(yoco, rng, cache, B, N, Hkv, d, std=1.0, offset=0.0, poison=True):
    """A pool whose rows 0 .. N - 1 of every sequence are written, the rest and other pages full of NaN; and its values."""
    cols = -(-N // 64)
    table, n = tables(rng, B, cols, spare=3)
    c = make(yoco, cache, n, Hkv, d, 0xFF if poison else 0)
    k = (rng.standard_normal((B, N, Hkv, d)) * std + offset).astype(np.float32)
    v = (rng.standard_normal((B, N, Hkv, d)) * std + offset).astype(np.float32)
    t, zero = dev(table), torch.zeros(B, dtype=torch.int64, device="cuda")
    yoco.paged_append(c, t, zero, dev(k), dev(v))
    k, v = (host(x).transpose(0, 2, 1, 3) for x in yoco.paged_read(c, t, zero, N, dtype=torch.float32))
    return c, table, k, v


def check(got, q, k, v, n, scale, what):
    want = paged.attend(q, k, v, n, scale)
    most = np.abs(v[:, :max(n, 1)]).max() if n > 0 else 0.0
    err, bound = np.abs(got - want), 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * most
    print("%s: max error %.2e of at most %.2e" % (what, err.max(), bound.flat[err.argmax()]), flush=True)
    assert np.isfinite(got).all() and (err <= bound).all(), what


SHAPES = [  # B, T, N, Hq, Hkv, d, lens
    (1, 1, 1, 1, 1, 128, [1]), (2, 1, 64, 3, 1, 128, [64, 63]), (3, 1, 200, 24, 8, 128, [200, 65, 0]), (2, 1, 1000, 16, 16, 128, [1000, 129]),
    (1, 1, 5000, 6, 2, 128, [4999]), (2, 1, 700, 32, 4, 128, [700, 1]), (1, 1, 3000, 16, 1, 128, [2500]), (2, 1, 333, 40, 2, 128, [333, 300]),
    (2, 1, 777, 24, 8, 64, [777, 100]), (1, 1, 4096, 17, 1, 64, [4096]), (2, 3, 300, 24, 8, 128, [300, 2]), (1, 6, 2049, 32, 8, 128, [2049]),
    (2, 5, 130, 4, 4, 64, [130, 64]), (1, 65, 500, 6, 2, 128, [400]), (1, 40, 40, 8, 8, 64, [40]), (70, 1, 150, 4, 2, 128, list(range(81, 151))),
    (5, 2, 1300, 12, 4, 128, [1300, 7, 640, 0, 1000])]


@pytest.mark.parametrize("cache", ["int4", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(x) for x in s[:6]))
def test_attention(yoco, shape, cache):
    B, T, N, Hq, Hkv, d, lens = shape
    rng = np.random.default_rng(B + N + Hq)
    c, table, k, v = filled(yoco, rng, cache, B, N, Hkv, d)
    q = paged.bf16(rng.standard_normal((B, T, Hq, d)).astype(np.float32))
    scale, t, n = 1.0 / math.sqrt(d), dev(table), dev(np.array(lens))
    ws = torch.full((max(yoco.paged_attn_workspace(c, B, table.shape[1], T, Hq), 16) // 4,), float("nan"), device="cuda")
    o = yoco.paged_attn(c, t, dev(q, torch.bfloat16), n, scale, workspace=ws)
    for b in range(B):
        check(host(o[b]), q[b], k[b], v[b], lens[b], scale, "%s sequence %d" % (cache, b))
    for _ in range(3):                                                          # the same bits again, and with scratch from torch
        assert torch.equal(yoco.paged_attn(c, t, dev(q, torch.bfloat16), n, scale), o)


@pytest.mark.parametrize("cache", ["int4", "bf16"])
@pytest.mark.parametrize("std,offset,qstd,scale", [(1.0, 0.0, 8.0, 0.3), (1e-3, 0.0, 1.0, 0.1), (50.0, 0.0, 0.05, 0.09), (0.1, 20.0, 1.0, 0.088), (1e-12, 0.0, 1e12, 0.1), (1.0, 0.0, 1.0, 0.0), (1.0, 0.0, 1.0, -0.1)])
def test_attention_over_other_magnitudes(yoco, cache, std, offset, qstd, scale):
    rng = np.random.default_rng(int(abs(math.log(std)) * 10))
    c, table, k, v = filled(yoco, rng, cache, 1, 1500, 2, 128, std, offset)
    q = paged.bf16((rng.standard_normal((1, 1, 6, 128)) * qstd).astype(np.float32))
    o = yoco.paged_attn(c, dev(table), dev(q, torch.bfloat16), dev(np.array([1500])), scale)
    want = paged.attend(q[0], k[0], v[0], 1500, scale)
    most = np.abs(v[0]).max()
    # scores in float32: products of |q| |k| summed over 128 dimensions, off by up to 2^-20 of that sum, move a weight by as much
    moved = abs(scale) * np.abs(q).max() * np.abs(k).max() * 128 * 2.0 ** -20
    assert (np.abs(host(o[0]) - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -9 + 2 * moved) * most).all()


@pytest.mark.parametrize("cache", ["int4", "bf16"])
def test_attention_where_pages_are_missing(yoco, cache):
    rng = np.random.default_rng(5)
    c, table, k, v = filled(yoco, rng, cache, 2, 640, 2, 128)
    table[0, [0, 3, 9]] = [-1, c.n_pages, 1 << 30]
    table[1, :] = -1
    k[0][:, np.isin(np.arange(640) // 64, [0, 3, 9])] = np.nan
    k[1][:] = np.nan
    q = paged.bf16(rng.standard_normal((2, 1, 4, 128)).astype(np.float32))
    o = yoco.paged_attn(c, dev(table), dev(q, torch.bfloat16), dev(np.array([640, 640])), 0.09)
    check(host(o[0]), q[0], k[0], v[0], 640, 0.09, cache)
    assert (o[1] == 0).all()


def test_lengths_are_clamped_to_the_table(yoco):
    rng = np.random.default_rng(6)
    c, table, k, v = filled(yoco, rng, "int4", 2, 128, 1, 128)
    q = paged.bf16(rng.standard_normal((2, 1, 2, 128)).astype(np.float32))
    o = yoco.paged_attn(c, dev(table), dev(q, torch.bfloat16), dev(np.array([1 << 40, -5])), 0.09)
    check(host(o[0]), q[0], k[0], v[0], 128, 0.09, "clamped")
    assert (o[1] == 0).all()


@pytest.mark.parametrize("cache", ["int4", "bf16"])
def test_visible_values_that_are_not_finite_stay_in_their_sequence(yoco, cache):
    rng = np.random.default_rng(7)
    c, table, k, v = filled(yoco, rng, cache, 3, 200, 1, 128)
    bad = torch.full((1, 1, 1, 128), float("nan"), device="cuda")
    yoco.paged_append(c, dev(table[1:2]), dev(np.array([130])), bad, bad)
    q = paged.bf16(rng.standard_normal((3, 1, 3, 128)).astype(np.float32))
    o = host(yoco.paged_attn(c, dev(table), dev(q, torch.bfloat16), dev(np.array([200, 200, 130])), 0.09))
    assert np.isnan(o[1]).all()
    for b, n in ((0, 200), (2, 130)):
        check(o[b], q[b], k[b], v[b], n, 0.09, cache)
    o = yoco.paged_attn(c, dev(table[1:2]), dev(q[1:2], torch.bfloat16), dev(np.array([130])), 0.09)       # the row is not seen
    check(host(o[0]), q[1], k[1], v[1], 130, 0.09, cache)


@pytest.mark.parametrize("cache", ["int4", "bf16"])
def test_pools_beyond_32_bits(yoco, cache):
    rng = np.random.default_rng(8)
    page = 16 * (4608 if cache == "int4" else 16384)
    n = (1 << 32) // page + 40                                                  # each plane passes 4 GiB
    c = yoco.PagedCache(n, 16, 128, kind(yoco, cache))
    table = np.array([[n - 1, 3, n - 2, n - 30]], np.int32)
    k = rng.standard_normal((1, 256, 16, 128)).astype(np.float32)
    v = rng.standard_normal((1, 256, 16, 128)).astype(np.float32)
    zero = dev(np.zeros(1, np.int64))
    yoco.paged_append(c, dev(table), zero, dev(k), dev(v))
    k, v = (host(x).transpose(0, 2, 1, 3) for x in yoco.paged_read(c, dev(table), zero, 256, dtype=torch.float32))
    q = paged.bf16(rng.standard_normal((1, 1, 16, 128)).astype(np.float32))
    o = yoco.paged_attn(c, dev(table), dev(q, torch.bfloat16), dev(np.array([256])), 0.088)
    check(host(o[0]), q[0], k[0], v[0], 256, 0.088, cache)


def test_many_splits_of_one_long_sequence(yoco):
    rng = np.random.default_rng(9)
    c, table, k, v = filled(yoco, rng, "int4", 1, 70000, 1, 128)
    q = paged.bf16(rng.standard_normal((1, 1, 3, 128)).astype(np.float32))
    for n in (70000, 65537, 64, 4097):
        o = yoco.paged_attn(c, dev(table), dev(q, torch.bfloat16), dev(np.array([n])), 0.088)
        check(host(o[0]), q[0], k[0], v[0], n, 0.088, "%d rows" % n)


def test_on_another_stream(yoco):
    rng = np.random.default_rng(10)
    c, table, k, v = filled(yoco, rng, "int4", 2, 3000, 2, 128)
    q = paged.bf16(rng.standard_normal((2, 1, 6, 128)).astype(np.float32))
    t, n, qd = dev(table), dev(np.array([3000, 2999])), dev(q, torch.bfloat16)
    want = yoco.paged_attn(c, t, qd, n, 0.088)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        late = torch.empty_like(qd)
        late.copy_(qd)
        o = yoco.paged_attn(c, t, late, n, 0.088)
    s.synchronize()
    assert torch.equal(o, want)


@pytest.mark.parametrize("cache", ["int4", "bf16"])
def test_a_step_replays_from_a_graph(yoco, cache):
    """Append and attend, captured once, replayed over advancing positions with eager work between."""
    rng = np.random.default_rng(11)
    B, N, Hq, Hkv, d = 3, 900, 6, 2, 128
    c, table, k, v = filled(yoco, rng, cache, B, N, Hkv, d)
    eager, _, _, _ = filled(yoco, np.random.default_rng(11), cache, B, N, Hkv, d)
    t, pos, turns = dev(table), dev(np.array([500, 100, 777])), yoco.rotation_turns(d)
    lens = pos + 1
    q, kn, vn = (torch.randn(B, 1, h, d, device="cuda", dtype=torch.bfloat16) for h in (Hq, Hkv, Hkv))
    ws = torch.empty(max(16, yoco.paged_attn_workspace(c, B, t.shape[1], 1, Hq)), dtype=torch.uint8, device="cuda")
    qr, o = torch.empty_like(q), torch.empty_like(q)

    def step(cache):
        yoco.paged_append(cache, t, pos, kn, vn, q=q, turns=turns, q_out=qr)
        yoco.paged_attn(cache, t, qr, lens, 0.088, workspace=ws, out=o)

    step(c)
    step(eager)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(c)
    for i in range(5):
        pos += 1
        lens += 1
        for x in (q, kn, vn):
            x.copy_(torch.randn_like(x))
        g.replay()
        torch.cuda.synchronize()
        got = o.clone()
        step(eager)
        assert torch.equal(o, got), i
    assert torch.equal(c.mem, eager.mem)
