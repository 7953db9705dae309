"""Beam search on the GPU: selection against float64 scores over sorted candidates, and states in the order of their parents.

Scores: base + (x - lse) in float32, with lse good to a few ulp of its size: 2e-6 times the largest of |base|, |x|, |lse| and 1. Beams and
tokens have to be the definition's wherever its scores are further apart than that."""
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
    y.lib()
    assert torch.cuda.is_available()
    return y


def check(yoco, logits, scores, done, eos, x):
    """logits: numpy values of the device tensor x."""
    before = x.clone()
    d = None if done is None else torch.from_numpy(done).cuda()
    got = yoco.beam_select(x, torch.from_numpy(scores).cuda(), done=d, eos=eos)
    again = yoco.beam_select(x, torch.from_numpy(scores).cuda(), done=d, eos=eos,
                             workspace=torch.full((yoco.beam_select_workspace(*x.shape),), 255, dtype=torch.uint8, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(got, again)) and torch.equal(x.view(torch.uint8), before.view(torch.uint8))
    parent, token, score, ended = (t.cpu().numpy() for t in got)
    for b in range(x.shape[0]):
        wp, wt, ws, wd = paged.select(logits[b], scores[b], None if done is None else done[b], eos)
        finite = np.isfinite(ws)
        size = max(1.0, np.max(np.abs(scores[b][np.isfinite(scores[b])]), initial=0.0), np.max(np.abs(logits[b][np.isfinite(logits[b])]), initial=0.0))
        tol = 2e-6 * size
        assert np.array_equal(np.isfinite(score[b]), finite)
        assert (np.abs(score[b][finite] - np.array(ws)[finite]) <= tol + 1e-6 * np.abs(np.array(ws)[finite])).all()
        assert (parent[b].tolist(), token[b].tolist(), ended[b].tolist()) == (wp, wt, wd), (b, score[b], ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,W,V", [(1, 1, 1), (1, 4, 7), (2, 3, 100), (1, 16, 5), (3, 8, 1000), (1, 4, 32000), (2, 5, 2047), (1, 8, 2049), (1, 2, 100003), (5, 16, 16385), (1, 1, 524288), (20, 8, 4096)])
def test_selection(yoco, B, W, V, dtype):
    rng = np.random.default_rng(B + W + V)
    x = torch.from_numpy((rng.standard_normal((B, W, V)) * 3).astype(np.float32)).cuda().to(TD[dtype])
    scores = -(rng.random((B, W)) * 3).astype(np.float32)
    check(yoco, x.float().cpu().numpy(), scores, None, -1, x)
    done = rng.random((B, W)) < 0.4
    check(yoco, x.float().cpu().numpy(), scores, done, min(2, V - 1), x)


def test_rows_that_start_anywhere(yoco):
    rng = np.random.default_rng(3)
    joined = torch.from_numpy(rng.standard_normal((2, 3, 1013)).astype(np.float32)).cuda()
    for dtype in TD:
        wide = joined.to(TD[dtype])
        x = wide[:, :, :1000]
        check(yoco, x.float().cpu().numpy(), np.zeros((2, 3), np.float32) - np.arange(3, dtype=np.float32) / 7, None, 5, x)
    with pytest.raises(yoco.YocoError):
        yoco.beam_select(wide[:, :, ::2], torch.zeros(2, 3, device="cuda"))


def test_equal_logits_go_to_the_lowest_token(yoco):
    for V in (3, 5000, 70000):
        x = torch.zeros(1, 8, V, device="cuda", dtype=torch.bfloat16)
        scores = np.array([[0, -1, -2, -3, -4, -5, -6, -7]], np.float32)
        check(yoco, np.zeros((1, 8, V), np.float32), scores, None, -1, x)
    x = torch.zeros(1, 4, 6000, device="cuda")
    x[0, 1, 4999], x[0, 1, 17], x[0, 1, 5999] = 9.0, 9.0, 9.0
    check(yoco, x.cpu().numpy(), np.array([[-50, 0, -50, -50]], np.float32), None, -1, x)


def test_equal_scores_go_to_the_lowest_beam(yoco):
    row = torch.randn(5000, device="cuda")
    x = row.expand(4, 5000).contiguous().view(1, 4, 5000)
    parent, token, score, _ = yoco.beam_select(x, torch.zeros(1, 4, device="cuda"))
    assert parent.tolist() == [[0, 1, 2, 3]] and (token == int(row.argmax())).all() and (score == score[0, 0]).all()


def test_logits_that_are_not_finite(yoco):
    rng = np.random.default_rng(4)
    for V in (50, 9000):
        x = rng.standard_normal((1, 4, V)).astype(np.float32)
        x[0, 0, ::2] = -np.inf
        x[0, 1, :] = -np.inf
        x[0, 2, 7] = np.nan
        x[0, 3, [5, 8]] = np.inf
        check(yoco, x, np.array([[-1, 0, -2, -3]], np.float32), None, -1, torch.from_numpy(x).cuda())
        x[:] = -np.inf
        x[0, 2, 11] = 0.5
        check(yoco, x, np.array([[-1, 0, -2, -3]], np.float32), None, 3, torch.from_numpy(x).cuda())
        x[:] = np.nan
        check(yoco, x, np.array([[-1, 0, -2, -3]], np.float32), None, -1, torch.from_numpy(x).cuda())


def test_beams_that_are_dead_or_finished(yoco):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((3, 4, 300)).astype(np.float32)
    scores = np.array([[0, -np.inf, -np.inf, -np.inf], [-1, np.nan, -2, -np.inf], [-9, -0.01, -9, -0.02]], np.float32)
    check(yoco, x, scores, None, 2, torch.from_numpy(x).cuda())                  # a first step: one beam is alive
    done = np.array([[1, 0, 0, 0], [1, 1, 1, 1], [0, 1, 0, 1]], bool)
    check(yoco, x, scores, done, 2, torch.from_numpy(x).cuda())


def test_selection_refuses(yoco):
    x, s = torch.zeros(2, 4, 100, device="cuda"), torch.zeros(2, 4, device="cuda")
    for bad in (lambda: yoco.beam_select(x[0], s), lambda: yoco.beam_select(x, s[:1]), lambda: yoco.beam_select(x, s.double()), lambda: yoco.beam_select(x.half(), s),
                lambda: yoco.beam_select(x, s, done=s), lambda: yoco.beam_select(torch.zeros(1, 17, 10, device="cuda"), torch.zeros(1, 17, device="cuda")),
                lambda: yoco.beam_select(x, s, done=s > 0, eos=100), lambda: yoco.beam_select(x, s, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), lambda: yoco.beam_select(x.cpu(), s)):
        with pytest.raises(yoco.YocoError):
            bad()


# ------------------------------------------------------------ states in the order of their parents
@pytest.mark.parametrize("B,W,n,size", [(1, 1, 1, 4), (1, 4, 3, 1000), (3, 8, 2, 64), (2, 16, 40, 4), (2, 5, 1, 300000), (1, 2, 33, 128)])
def test_rows_follow_their_parents(yoco, B, W, n, size):
    rng = np.random.default_rng(B + W + n)
    parent = rng.integers(0, W, (B, W)).astype(np.int32)
    if W >= 5:
        parent[0, 1], parent[0, 3] = -1, W                                      # none of the beams: stays
    states = [torch.randn(B * W, size + 4 * i, device="cuda") for i in range(n)]
    p = np.where((parent < 0) | (parent >= W), np.arange(W), parent)
    at = torch.from_numpy((p + W * np.arange(B)[:, None]).ravel()).cuda()
    want = [s[at].clone() for s in states]
    yoco.beam_reorder_rows(states, torch.from_numpy(parent).cuda())
    assert all(torch.equal(a, b) for a, b in zip(states, want))


def test_rows_of_any_type_and_refusals(yoco):
    parent = torch.tensor([[1, 0, 2]], dtype=torch.int32, device="cuda")
    ring, code = torch.randn(3, 2, 5, 8, device="cuda", dtype=torch.bfloat16), torch.arange(48, dtype=torch.uint8, device="cuda").view(3, 16)
    want = [x[[1, 0, 2]].clone() for x in (ring, code)]
    yoco.beam_reorder_rows([ring, code], parent)
    assert torch.equal(ring, want[0]) and torch.equal(code, want[1])
    yoco.beam_reorder_rows([], parent)
    yoco.beam_reorder_rows([torch.empty(3, 0, device="cuda")], parent)
    for bad in ([torch.zeros(4, 8, device="cuda")], [torch.zeros(3, 3, device="cuda")], [torch.zeros(3, 16, device="cuda")[:, :8]], [torch.zeros(3, 8)]):
        with pytest.raises(yoco.YocoError):
            yoco.beam_reorder_rows(bad, parent)
    with pytest.raises(TypeError):
        yoco.beam_reorder_rows([1], parent)


@pytest.mark.parametrize("dtype", ["int4", "bf16"])
@pytest.mark.parametrize("B,W,cols,Hkv,d,lens", [(1, 1, 2, 1, 128, [70]), (2, 4, 5, 2, 128, [130, 128]), (3, 8, 300, 1, 64, [0, 19199, 19200]), (1, 16, 3, 3, 64, [1]), (2, 5, 4, 2, 128, [255, 256])])
def test_page_tables_follow_their_parents(yoco, dtype, B, W, cols, Hkv, d, lens):
    rng = np.random.default_rng(B + W + cols)
    n = B * W * cols + B * cols                                                  # every beam's own pages, and the prompts'
    order = rng.permutation(n).astype(np.int32)
    home, prompt = order[:B * W * cols].reshape(B, W, cols), order[B * W * cols:].reshape(B, 1, cols)
    table = np.where(rng.random((B, W, cols)) < 0.5, home, prompt)
    c = yoco.PagedCache(n, Hkv, d, yoco.INT4 if dtype == "int4" else torch.bfloat16)
    c.mem.copy_(torch.randint(0, 256, c.mem.shape, dtype=torch.uint8, device="cuda"))
    td, hd = torch.from_numpy(table.reshape(B * W, cols)).cuda(), torch.from_numpy(home.reshape(B * W, cols).copy()).cuda()
    ld = torch.tensor([x for x in lens for _ in range(W)], dtype=torch.int64, device="cuda")
    k, v = c.mem.cpu().numpy().reshape(2, n, -1)
    for step in range(3):
        parent = rng.integers(0, W, (B, W)).astype(np.int32) if step else np.broadcast_to(np.arange(W, dtype=np.int32), (B, W)).copy()
        if W > 3 and step:
            parent[0, 2] = W + 7
        k, v, table = paged.reorder_pages(k, v, table, home, parent, lens)
        yoco.beam_reorder_pages(c, td, hd, torch.from_numpy(parent).cuda(), ld)
        assert np.array_equal(td.cpu().numpy().reshape(B, W, cols), table)
        assert np.array_equal(c.mem.cpu().numpy().reshape(2, n, -1), np.stack([k, v]))
        assert np.array_equal(hd.cpu().numpy().reshape(home.shape), home)


def test_page_table_refusals(yoco):
    c = yoco.PagedCache(8, 1, 64, yoco.INT4)
    t, parent, lens = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    for bad in (lambda: yoco.beam_reorder_pages(c, t, t, parent, lens), lambda: yoco.beam_reorder_pages(c, t, t[:2].clone(), parent, lens), lambda: yoco.beam_reorder_pages(c, t, t.clone(), parent[:1], lens),
                lambda: yoco.beam_reorder_pages(c, t, t.clone(), parent, lens[:2]), lambda: yoco.beam_reorder_pages(c, t.long(), t.clone(), parent, lens)):
        with pytest.raises(yoco.YocoError):
            bad()


def test_a_step_replays_from_a_graph(yoco):
    B, W, V = 2, 4, 9000
    x, scores = torch.randn(B, W, V, device="cuda"), torch.zeros(B, W, device="cuda")
    ws = torch.empty(yoco.beam_select_workspace(B, W, V), dtype=torch.uint8, device="cuda")
    state, start = torch.randn(B * W, 512, device="cuda"), torch.randn(B * W, 512, device="cuda")
    yoco.beam_select(x, scores, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        parent, token, best, _ = yoco.beam_select(x, scores, workspace=ws)
        yoco.beam_reorder_rows([state], parent)
    for i in range(4):
        x.copy_(torch.randn_like(x))
        scores.copy_(-torch.rand(B, W, device="cuda"))
        state.copy_(start)
        g.replay()
        torch.cuda.synchronize()
        p, t, s, _ = yoco.beam_select(x, scores)
        assert torch.equal(p, parent) and torch.equal(t, token) and torch.equal(s, best)
        at = (p.long() + W * torch.arange(B, device="cuda")[:, None]).view(-1)
        assert torch.equal(state, start[at])
