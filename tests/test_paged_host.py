"""The cache in pages and beam search, without a GPU: the order inside a page, the definitions that the GPU tests compare with,
and what the calls refuse before they launch anything."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2405_05254_amd as yoco
from oracle import paged
from paper_2405_05254_amd import binding as yb

P = 0x7F0000000000          # never dereferenced: every call below fails on the host


# ------------------------------------------------------------ definitions
@pytest.mark.parametrize("d", [64, 128])
def test_every_value_has_a_place_of_its_own(d):
    for at in paged.places(d, False):
        assert sorted(at.ravel()) == list(range(ROWS_D(d)))
    for byte, nibble in paged.places(d, True):
        assert sorted((2 * byte + nibble).ravel()) == list(range(ROWS_D(d)))
        rows_of_byte = [set(np.nonzero(byte == x)[0]) for x in range(0, 32 * d, 37)]
        assert all(len(r) == 1 for r in rows_of_byte)          # a row is written without reading its neighbours


def ROWS_D(d):
    return 64 * d


def test_pool_bytes():
    n = C.c_size_t()
    for d, dtype, page in ((128, yoco.BF16, 16384), (64, yoco.BF16, 8192), (128, yoco.INT4, 4608), (64, yoco.INT4, 2304)):
        assert yoco.lib().yoco_paged_cache_bytes(7, 3, d, dtype, C.byref(n)) == 0 and n.value == 2 * 7 * 3 * page
        assert page == paged.page_bytes(d, dtype == yoco.INT4)


def test_codes_are_within_half_a_step():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((500, 128)) * np.exp2(rng.integers(-30, 30, (500, 1))) + rng.standard_normal((500, 1))).astype(np.float32)
    x[3] = 0.0
    x[4] = 7.25
    c, scale, base = paged.code(x)
    y = paged.stands_for(c, scale, base)
    g = x.reshape(500, 2, 64).astype(np.float64)
    step = (g.max(-1) - g.min(-1)) / 15
    # half a step, what bf16 rounds off the scale (15 times 2^-9 of it) and off the minimum (2^-9)
    bound = 0.5 * step + 15 * 2.0 ** -9 * step + 2.0 ** -8 * np.abs(g.min(-1)) + 1e-30
    assert (np.abs(y.reshape(g.shape) - g) <= bound[..., None]).all()
    assert (y[3] == 0).all() and (y[4] == 7.25).all() and c.max() == 15


def test_a_group_that_is_not_finite_reads_as_nan():
    x = np.ones((4, 128), np.float32)
    x[0, 5], x[1, 70], x[2, 0], x[2, 1] = np.inf, np.nan, 3e38, -3e38
    y = paged.stands_for(*paged.code(x))
    assert np.isnan(y[0, :64]).all() and (y[0, 64:] == 1).all() and np.isnan(y[1, 64:]).all() and np.isnan(y[2, :64]).all() and (y[3] == 1).all()


def test_rotation_keeps_products_of_distances():
    rng = np.random.default_rng(2)
    units = paged.turns([10000.0 ** (-p / 32) for p in range(32)])
    q, k = rng.standard_normal((1, 64)), rng.standard_normal((1, 64))
    for neighbours in (False, True):
        near = paged.rotate(q, 9, units, neighbours) @ paged.rotate(k, 4, units, neighbours).T
        far = paged.rotate(q, 1000005, units, neighbours) @ paged.rotate(k, 1000000, units, neighbours).T
        assert abs(near - far) < 1e-9 and np.allclose(paged.rotate(q, 0, units, neighbours), q)
        assert abs(np.linalg.norm(paged.rotate(q, 77, units, neighbours)) - np.linalg.norm(q)) < 1e-12


def test_turn_units_match_the_definition():
    got = yoco.rotation_turns(128, 10000.0, device="cpu")
    want = paged.turns([10000.0 ** (-2.0 * p / 128) for p in range(64)])
    assert got.dtype == torch.int64 and [int(x) % 2 ** 64 for x in got] == want
    assert int(yoco.turn_units([math.pi], device="cpu")[0]) == -2 ** 63


def test_select_by_hand():
    logits = np.log(np.array([[0.1, 0.6, 0.3, 0.0], [0.25, 0.25, 0.25, 0.25]], np.float32) + 1e-30)
    parent, token, score, done = paged.select(logits, np.array([-1.0, -1.0]), None, 2)
    assert (parent, token, done) == ([0, 0], [1, 2], [False, True]) and abs(score[0] - (-1 + math.log(0.6))) < 1e-6
    parent, token, score, done = paged.select(logits, np.array([-3.0, -1.0]), np.array([False, True]), 2)
    assert (parent, token, done) == ([1, 0], [2, 1], [True, False]) and score[0] == -1.0
    parent, token, score, done = paged.select(logits, np.array([-np.inf, -1.0]), None, -1)
    assert (parent, token) == ([1, 1], [0, 1])                                   # equal logits: the lower tokens
    assert paged.select(logits, np.array([-np.inf, np.nan]), None, -1) == ([0, 1], [0, 0], [-math.inf, -math.inf], [False, False])


# ------------------------------------------------------------ refusals
def pool(d=128, dtype=None, n_pages=4, Hkv=2):
    return yb._Paged(P, P + 4096, n_pages, Hkv, d, yoco.INT4 if dtype is None else dtype)


@pytest.mark.parametrize("args,code", [((0, 8, 128, 3), -1), ((4, 0, 128, 3), -1), ((4, 8, 96, 3), -2), ((4, 8, 128, 0), -2), ((4, 8, 128, 2), -2), ((4, 8, 128, 9), -2)])
def test_pool_sizes_that_are_refused(args, code):
    n = C.c_size_t()
    assert yoco.lib().yoco_paged_cache_bytes(*args, C.byref(n)) == code


def test_pool_memory_is_checked():
    L, out = yoco.lib(), yb._Paged()
    need = 2 * 5 * 2 * 4608
    assert L.yoco_paged_cache_init(P, need, 5, 2, 128, yoco.INT4, C.byref(out)) == 0 and out.v == P + need // 2
    assert L.yoco_paged_cache_init(P, need - 1, 5, 2, 128, yoco.INT4, C.byref(out)) == -4
    assert L.yoco_paged_cache_init(P + 16, need, 5, 2, 128, yoco.INT4, C.byref(out)) == -3
    assert L.yoco_paged_cache_init(None, need, 5, 2, 128, yoco.INT4, C.byref(out)) == -1


APPEND = dict(c=pool(), table=P, B=2, cols=3, pos=P, rows=None, T=5, k=P, ks=256, v=P, vs=256, q=None, qs=0, q_out=None, Hq=0, rot=None, dtype=1)


@pytest.mark.parametrize("change,code", [
    (dict(c=None), -1), (dict(c=pool(96)), -2), (dict(c=pool(dtype=2)), -2), (dict(c=pool(n_pages=0)), -1), (dict(table=None), -1), (dict(B=0), -1), (dict(cols=0), -1),
    (dict(cols=1 << 25), -2), (dict(pos=None), -1), (dict(pos=P + 4), -3), (dict(rows=P + 4), -3), (dict(T=-1), -1), (dict(T=1 << 31), -2), (dict(k=None), -1), (dict(k=P + 8), -3),
    (dict(ks=248), -1), (dict(vs=260), -3), (dict(q=P, qs=512, Hq=4), -1), (dict(q=P, qs=512, q_out=P + 4, Hq=4), -3), (dict(q=P, qs=512, q_out=P, Hq=0), -1),
    (dict(q=P, qs=520, q_out=P, Hq=4), -1), (dict(q=P, qs=504, q_out=P + 64, Hq=4), -1), (dict(rot=yb._Rotation(P, 24, 0)), -1), (dict(rot=yb._Rotation(P, 144, 0)), -1),
    (dict(rot=yb._Rotation(None, 64, 0)), -1), (dict(rot=yb._Rotation(P + 4, 64, 0)), -3), (dict(dtype=2), -2), (dict(dtype=3), -2)])
def test_append_refuses(change, code):
    a = dict(APPEND, **change)
    ref = lambda x: None if x is None else C.byref(x)                            # noqa: E731
    rc = yoco.lib().yoco_paged_append(ref(a["c"]), a["table"], a["B"], a["cols"], a["pos"], a["rows"], a["T"], a["k"], a["ks"], a["v"], a["vs"], a["q"], a["qs"], a["q_out"],
                                      a["Hq"], ref(a["rot"]), a["dtype"], None)
    assert rc == code and yoco.lib().yoco_last_error_string()


def test_nothing_to_append_read_or_attend_is_no_error():
    L, c = yoco.lib(), pool()
    assert L.yoco_paged_append(C.byref(c), P, 2, 3, None, None, 0, None, 0, None, 0, None, 0, None, 0, None, 1, None) == 0
    assert L.yoco_paged_read(C.byref(c), P, 2, 3, None, 0, None, None, 1, None) == 0
    assert L.yoco_paged_attn(C.byref(c), P, 2, 3, None, None, None, 0, 4, 1.0, None, 0, None) == 0
    assert L.yoco_beam_reorder_rows(None, None, 0, 1, 4, None, None) == 0


@pytest.mark.parametrize("change,code", [(dict(c=pool(96)), -2), (dict(table=None), -1), (dict(pos=None), -1), (dict(T=-1), -1), (dict(k=P + 8), -3), (dict(v=None), -1), (dict(dtype=3), -2),
                                         (dict(T=1 << 30), -2)])
def test_read_refuses(change, code):
    a = dict(dict(c=pool(), table=P, pos=P, T=4, k=P, v=P, dtype=1), **change)
    assert yoco.lib().yoco_paged_read(C.byref(a["c"]), a["table"], 2, 3, a["pos"], a["T"], a["k"], a["v"], a["dtype"], None) == code


@pytest.mark.parametrize("change,code", [(dict(c=pool(96)), -2), (dict(table=None), -1), (dict(lens=None), -1), (dict(lens=P + 4), -3), (dict(q=None), -1), (dict(o=P + 8), -3), (dict(T=-1), -1),
                                         (dict(Hq=3), -1), (dict(Hq=0), -1), (dict(T=1 << 23), -2), (dict(B=70000), -2)])
def test_attn_refuses(change, code):
    a = dict(dict(c=pool(), table=P, B=2, q=P, o=P, lens=P, T=1, Hq=4), **change)
    assert yoco.lib().yoco_paged_attn(C.byref(a["c"]), a["table"], a["B"], 3, a["q"], a["o"], a["lens"], a["T"], a["Hq"], 1.0, P, 1 << 40, None) == code


@pytest.mark.parametrize("change,code", [(dict(B=0), -1), (dict(W=17), -2), (dict(W=0), -1), (dict(V=0), -1), (dict(V=524289), -2), (dict(stride=99), -1), (dict(dtype=2), -2), (dict(logits=None), -1),
                                         (dict(logits=P + 4), -3), (dict(scores=None), -1), (dict(parent=None), -1), (dict(token=P + 2), -3), (dict(ws=0), -4), (dict(eos=100), -1), (dict(B=9000, W=8), -2)])
def test_select_refuses(change, code):
    a = dict(dict(logits=P, stride=100, scores=P, done=P, eos=2, B=2, W=4, V=100, dtype=0, parent=P, token=P, ws=1 << 40), **change)
    a["stride"] = max(a["stride"], a["V"]) if "stride" not in change else a["stride"]
    assert yoco.lib().yoco_beam_select(a["logits"], a["stride"], a["scores"], a["done"], a["eos"], a["B"], a["W"], a["V"], a["dtype"], a["parent"], a["token"], P, P, P, a["ws"], None) == code


@pytest.mark.parametrize("change,code", [(dict(W=17), -2), (dict(home=P), -1), (dict(home=None), -1), (dict(parent=None), -1), (dict(lens=P + 4), -3), (dict(table=None), -1), (dict(cols=0), -1)])
def test_reorder_pages_refuses(change, code):
    c = pool()
    a = dict(dict(table=P, home=P + 4096, W=4, cols=3, parent=P, lens=P), **change)
    assert yoco.lib().yoco_beam_reorder_pages(C.byref(c), a["table"], a["home"], 1, a["W"], a["cols"], a["parent"], a["lens"], None) == code


def test_reorder_rows_refuses():
    L = yoco.lib()
    mem, size = (C.c_void_p * 2)(P, P + 4096), (C.c_int64 * 2)(64, 64)
    assert L.yoco_beam_reorder_rows(mem, size, 2, 1, 17, P, None) == -2
    assert L.yoco_beam_reorder_rows(mem, size, 2, 1, 4, None, None) == -1
    assert L.yoco_beam_reorder_rows(mem, size, -1, 1, 4, P, None) == -1
    assert L.yoco_beam_reorder_rows(mem, (C.c_int64 * 2)(64, 24), 2, 1, 4, P, None) == -3
    assert L.yoco_beam_reorder_rows((C.c_void_p * 2)(P, P + 8), size, 2, 1, 4, P, None) == -3
    assert L.yoco_beam_reorder_rows((C.c_void_p * 2)(P, None), size, 2, 1, 4, P, None) == -1


def test_the_binding_refuses_what_does_not_fit():
    with pytest.raises(yoco.YocoError):
        yoco.PagedCache(4, 2, 128, torch.int8, device="cpu")
    with pytest.raises(yoco.YocoError, match="device tensor"):
        yoco.PagedCache(4, 2, 128, yoco.INT4, device="cpu")
