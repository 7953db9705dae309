"""Beam search through a whole stack: every returned score against its sequence scored all at once by the float64 oracle (bf16 pages), and
against the same tokens run again without a change of beams (4-bit pages, rotation), where every number is formed alike.

Against the oracle: the attention operands q, k, v and o are rounded to bf16 in each of 4 layers, 16 independent roundings of
2^-9 / sqrt(3) each, 4.5e-3 of the logits' size in the mean square; a score is a sum of n of them. Six times that.
Against the run without changes: the float32 scores of n selections, each good to 2e-6 of the largest number in it."""
import numpy as np
import pytest
import torch

import oracle
import yoco_synth as ys

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def yoco():
    import paper_2405_05254_amd as y
    y.lib()
    assert torch.cuda.is_available()
    return y


def stack_of(kind, d=64):
    from paper_2405_05254_amd.stack import YocoStack
    s = dict(ys.CONFIGS["tiny_fp32"]["stack"], window=24, d=d, self_kind=kind)
    w = ys.stack_weights(7, s, "bf16")
    return YocoStack(w, torch.bfloat16), w


def prompts_of(lengths, vocab=1000):
    return [torch.from_numpy(ys.tokens(40 + n, n, vocab)).cuda() for n in lengths]


def log_probs(logits, tokens):
    x = logits.astype(np.float64)
    top = x.max(-1, keepdims=True)
    lse = top[..., 0] + np.log(np.exp(x - top).sum(-1))
    return np.take_along_axis(x, tokens[..., None], -1)[..., 0] - lse


@pytest.mark.parametrize("kind", ["swa", "gret"])
@pytest.mark.parametrize("lengths,W,steps", [((5,), 4, 70), ((63, 64, 130), 3, 6), ((1, 40), 1, 30), ((127, 128), 16, 3)])
def test_a_score_is_its_sequence_s(yoco, kind, lengths, W, steps):
    st, w = stack_of(kind)
    prompts = prompts_of(lengths)
    tokens, scores = yoco.BeamSearch(st, W, max(lengths) + steps - 1, cache_dtype=torch.bfloat16).generate(prompts, steps)
    assert tokens.shape == (len(lengths), W, steps) and scores.shape == (len(lengths), W)
    tokens, scores = tokens.cpu().numpy(), scores.cpu().numpy()
    for b, p in enumerate(prompts):
        p = p.cpu().numpy()
        assert (np.diff(scores[b]) <= 0).all() and len({tuple(t) for t in tokens[b]}) == W
        for i in range(W):
            ref = oracle.yoco_stack(np.concatenate([p, tokens[b, i, :-1]]), w, "full")[len(p) - 1:]
            want = log_probs(ref, tokens[b, i].astype(np.int64)).sum()
            tol = 6 * np.sqrt(steps) * 4.5e-3 * np.std(ref) + 2e-6 * steps * max(1.0, abs(want))
            print("request %d beam %d: %.4f, oracle %.4f, within %.4f" % (b, i, scores[b, i], want, tol), flush=True)
            assert abs(scores[b, i] - want) <= tol


@pytest.mark.parametrize("kind,d,base", [("swa", 128, 10000.0), ("gret", 64, 10000.0), ("swa", 64, None)])
def test_beams_that_changed_places_are_what_they_would_be(yoco, kind, d, base):
    """The final sequences once more, each beam fed its own tokens from the prompt on."""
    W, steps, lengths = 4, 40, (3, 50, 64)
    st, _ = stack_of(kind, d)
    prompts = prompts_of(lengths)
    search = yoco.BeamSearch(st, W, max(lengths) + steps, rotation_base=base)
    moved = []
    plain = search.reorder
    search.reorder = lambda parent: (moved.append(parent.cpu()), plain(parent))
    tokens, scores = search.generate(prompts, steps)
    assert any((p != torch.arange(W)).any() for p in moved[1:])            # behind the prompt all come from beam 0
    search.reorder = plain
    logits = [search.start(prompts)[:, None].expand(-1, W, -1)]
    for n in range(steps - 1):
        search.reorder(torch.zeros(len(lengths), W, dtype=torch.int32, device="cuda") if n == 0 else torch.arange(W, dtype=torch.int32, device="cuda").repeat(len(lengths), 1))
        logits.append(search.advance(tokens[:, :, n]).view(len(lengths), W, -1))
    x = torch.stack(logits, 2).cpu().numpy()
    want = log_probs(x, tokens.cpu().numpy().astype(np.int64)).sum(-1)
    assert (np.abs(scores.cpu().numpy() - want) <= 2e-6 * steps * np.maximum(1.0, np.abs(want))).all()


def test_ended_beams_stay_ended(yoco):
    st, w = stack_of("swa")
    prompts = prompts_of((9, 20))
    tokens, _ = yoco.BeamSearch(st, 4, 64, cache_dtype=torch.bfloat16).generate(prompts, 12)
    eos = int(tokens[0, 0, 3])
    tokens, scores = yoco.BeamSearch(st, 4, 64, eos=eos, cache_dtype=torch.bfloat16).generate(prompts, 12)
    tokens, scores = tokens.cpu().numpy(), scores.cpu().numpy()
    ended = 0
    for b, p in enumerate(prompts):
        for i in range(4):
            t = tokens[b, i]
            n = int(np.argmax(t == eos)) + 1 if (t == eos).any() else len(t)
            ended += n < len(t)
            assert (t[n:] == eos).all()
            ref = oracle.yoco_stack(np.concatenate([p.cpu().numpy(), t[:n - 1]]), w, "full")[len(p) - 1:]
            want = log_probs(ref, t[:n].astype(np.int64)).sum()
            assert abs(scores[b, i] - want) <= 6 * np.sqrt(n) * 4.5e-3 * np.std(ref) + 2e-6 * n * max(1.0, abs(want))
    assert ended


def test_one_object_serves_one_batch_after_another(yoco):
    st, _ = stack_of("gret")
    search = yoco.BeamSearch(st, 3, 200, cache_dtype=torch.bfloat16)
    first = search.generate(prompts_of((70, 3)), 5)
    search.generate(prompts_of((150,)), 9)
    again = search.generate(prompts_of((70, 3)), 5)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
