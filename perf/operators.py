"""Generation over a paged cache, as cases that can be timed and whose outputs can be compared: rows are rotated to their
positions and appended to pages of 64 rows (bf16, or 4-bit codes), queries attend over the pages, beam search selects its
continuations and reorders page tables and other states after them.

A case is a dict of plain values. `listed()` gives the fixed ones, `draw(rng)` one more of the same ranges, `prepare`
makes what a program has in hand before the call, `run` is one pass (`own` false: elementary torch operations in float32;
true: the library's calls), `exact` the same from the definition in float64, `work` what a pass cannot do without.

Heads, dimensions, windows, layers and cache lengths are this repository's (24 query and 8 KV heads of 128, 13 layers,
windows of 1024, caches of up to 512K rows, a vocabulary of 32000); batches, beams and larger vocabularies are generic.
"""
import math

import torch

own = False

DEV = "cuda"
ROWS = 64                       # rows of a page
GROUP = 64                      # dimensions of a row that share a 4-bit scale and minimum
ROT_BASE = 10000.0


def listed():
    return [
        # One generation step of 16 sequences far into their caches: a row each, rotated and coded; latency counts.
        dict(name="append_step", op="append", cache="int4", src="bf16", B=16, T=1, N=32768, Hq=24, Hkv=8, d=128, rot=128, pairs="halves", ragged=False),
        # The rows of one long prompt, early exit: everything the cross-decoder will ever read, and its rotated queries.
        dict(name="append_prompt", op="append", cache="int4", src="bf16", B=1, T=32768, N=32768, Hq=24, Hkv=8, d=128, rot=128, pairs="halves", ragged=False),
        # Ordinary prompts of different lengths behind a shared prefix, float32 projections, smaller heads, half of each rotated.
        dict(name="append_ragged_f32", op="append", cache="bf16", src="f32", B=4, T=1500, N=2011, Hq=16, Hkv=4, d=64, rot=32, pairs="neighbours", ragged=True),
        # Short conversations of different lengths, one new token each: latency and launches count.
        dict(name="attend_short", op="attend", cache="int4", B=8, T=1, N=3000, Hq=24, Hkv=8, d=128, ragged=True),
        # One layer's step over 16 caches of 32K rows.
        dict(name="attend_16x32k", op="attend", cache="int4", B=16, T=1, N=32768, Hq=24, Hkv=8, d=128, ragged=False),
        # One layer's step over a single cache of 512K rows.
        dict(name="attend_1x512k", op="attend", cache="int4", B=1, T=1, N=524288, Hq=24, Hkv=8, d=128, ragged=False),
        # A batch over bf16 pages, ragged, an odd number of sequences.
        dict(name="attend_bf16", op="attend", cache="bf16", B=13, T=1, N=9001, Hq=24, Hkv=8, d=128, ragged=True),
        # Several proposed tokens checked at once: six causal rows a sequence.
        dict(name="attend_rows", op="attend", cache="int4", B=3, T=6, N=20000, Hq=32, Hkv=8, d=128, ragged=True),
        # One request's selection: 4 beams of a 32000-word vocabulary in bf16.
        dict(name="select_one", op="select", dtype="bf16", B=1, W=4, V=32000, done=False),
        # A batch of requests, 8 beams, a large vocabulary in float32, some beams finished.
        dict(name="select_batch", op="select", dtype="f32", B=16, W=8, V=128000, done=True),
        # After it: one request with gated-retention states, whose beams share most pages.
        dict(name="reorder_states", op="reorder", cache="int4", kind="states", B=1, W=4, layers=13, N=1500, Hkv=8, d=128, H=24, window=0),
        # A batch of requests with the rolling windows of 13 layers.
        dict(name="reorder_rings", op="reorder", cache="bf16", kind="rings", B=2, W=8, layers=13, N=3000, Hkv=8, d=128, H=24, window=1024),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "select", "reorder"])
    cache = rng.choice(["int4", "int4", "bf16"])
    d = rng.choice([128, 128, 64])
    Hq, Hkv = rng.choice([(24, 8), (24, 8), (16, 16), (16, 4), (32, 8), (64, 4), (24, 1)])
    if op == "append":
        T = rng.choice([1, 1, rng.randint(2, 9), _log(rng, 10, 32768)])
        B = _log(rng, 1, max(1, min(64, 32768 * 40 // (T * max(Hq + 2 * Hkv, 40)))))
        rot = rng.choice([d, d, d // 2, 0])
        return dict(op=op, cache=cache, src=rng.choice(["bf16", "bf16", "f32"]) if T * B < 16384 else "bf16", B=B, T=T,
                    N=T + _log(rng, 1, 65536 // B), Hq=Hq, Hkv=Hkv, d=d, rot=rot, pairs=rng.choice(["halves", "halves", "neighbours"]),
                    ragged=T > 1 and rng.random() < 0.5)
    if op == "attend":
        T = rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 9, 64)])
        B = _log(rng, 1, 64 if T == 1 else 8)
        most = 524288 * 8 // max(Hkv, 8) // B // (1 if cache == "int4" else 4) // (1 if T * Hq <= 64 else 4)
        return dict(op=op, cache=cache, B=B, T=T, N=_log(rng, 64 + T, max(most // (8 if T > 8 else 1), 200)), Hq=Hq, Hkv=Hkv, d=d, ragged=rng.random() < 0.6)
    if op == "select":
        return dict(op=op, dtype=rng.choice(["bf16", "f32"]), B=_log(rng, 1, 16), W=rng.choice([1, 2, 3, 4, 5, 8]), V=_log(rng, 1000, 128000), done=rng.random() < 0.5)
    kind = rng.choice(["states", "rings"])
    return dict(op=op, cache=cache, kind=kind, B=rng.choice([1, 1, 2]), W=rng.choice([2, 3, 4, 5, 8]), layers=rng.choice([4, 12, 13]),
                N=_log(rng, 70, 4000), Hkv=Hkv, d=d, H=rng.choice([16, 24]), window=rng.choice([512, 1024]) if kind == "rings" else 0)


# ---------------------------------------------------------------- the cache
# mem: uint8 [2, pages, Hkv, page bytes], K pages and then V pages; table: int32 [B, columns], the page of rows 64 c .. of each
# sequence. Inside a page (row r, dimension e):
#   bf16  K element ((r/16 * d/32 + e/32) * 64 + (e/8 % 4) * 16 + r%16) * 8 + e%8
#         V element ((e/16 * 2 + r/32) * 64 + (r%16 / 4) * 16 + e%16) * 8 + (r/16 % 2) * 4 + r%4
#   int4  K byte ((i/4) * 64 + (e/8 % 4) * 16 + r%16) * 16 + (i%4) * 4 + (e%8) / 2 with i = r/16 * d/32 + e/32, nibble e%2
#         V byte (e/32 * 64 + (r%16 / 4) * 16 + e%16) * 16 + r/16 * 4 + r%4, nibble e/16 % 2
#         then, from byte 32 d on, [64 rows][d/64 groups] of two bf16, scale and minimum
def _page_bytes(cache, d):
    return 36 * d if cache == "int4" else 128 * d


def _places(cache, d, dev):
    """Where the values of a page are: (row [64,1], dimension [1,d]) -> byte and nibble of K and V (int4), or element (bf16)."""
    r, e = torch.arange(ROWS, device=dev)[:, None], torch.arange(d, device=dev)[None, :]
    i, part = r // 16 * (d // 32) + e // 32, r % 16 // 4
    if cache == "bf16":
        return ((i * 64 + e // 8 % 4 * 16 + r % 16) * 8 + e % 8, ((e // 16 * 2 + r // 32) * 64 + part * 16 + e % 16) * 8 + r // 16 % 2 * 4 + r % 4)
    k = (i // 4 * 64 + e // 8 % 4 * 16 + r % 16) * 16 + i % 4 * 4 + e % 8 // 2
    v = (e // 32 * 64 + part * 16 + e % 16) * 16 + r // 16 * 4 + r % 4
    return k, (e % 2).expand_as(k), v, (e // 16 % 2).expand_as(v)


def _code(x):
    """float32 [..., d] -> codes (uint8 [..., d]) and bf16 scale and minimum [..., d/64, 2]."""
    g = x.unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1), g.amax(-1)
    scale, base = ((hi - lo) / 15.0).bfloat16(), lo.bfloat16()
    s = scale.float()
    inv = torch.where(s >= 2.0 ** -126, 1.0 / s, 0.0)
    scale = torch.where(s >= 2.0 ** -126, scale, 0.0)
    c = torch.round((g - base.float()[..., None]) * inv[..., None]).clamp(0.0, 15.0)
    return c.flatten(-2).to(torch.uint8), torch.stack([scale, base], -1)


def _nibbles(codes, which):
    """Codes [..., d] -> the bytes they fill [..., d/2]: K pairs neighbouring dimensions, V dimensions 16 apart."""
    c = codes.unflatten(-1, (-1, 2)) if which == 0 else codes.unflatten(-1, (-1, 2, 16)).transpose(-1, -2).flatten(-3, -2)
    return c[..., 0] | c[..., 1] << 4


def _values(plane, cache, d, which, pages):
    """The rows of the given pages (long [B, columns]) of one plane, float32 [B, Hkv, 64 columns, d]."""
    x = plane[pages].transpose(1, 2)                                           # [B, Hkv, columns, bytes]
    lead = x.shape[:3]
    if cache == "bf16":
        x = x.contiguous().view(torch.bfloat16)
        if which == 0:
            x = x.view(*lead, 4, d // 32, 4, 16, 8).permute(0, 1, 2, 3, 6, 4, 5, 7)
        else:
            x = x.view(*lead, d // 16, 2, 4, 16, 2, 4).permute(0, 1, 2, 4, 7, 5, 8, 3, 6)
        return x.reshape(*lead[:2], lead[2] * ROWS, d).float()
    param = x[..., 32 * d:].contiguous().view(torch.bfloat16).view(*lead, ROWS, d // GROUP, 2).float()
    x = x[..., :32 * d]
    x = torch.stack([x & 15, x >> 4], -1)
    if which == 0:                                                             # load, part, row, tile of the load, step, byte, nibble
        x = x.reshape(*lead, d // 32, 4, 16, 128 // d, d // 32, 4, 2).permute(0, 1, 2, 3, 6, 5, 7, 4, 8, 9)
    else:                                                                      # pair of tiles, part, dimension, tile of rows, row, nibble
        x = x.reshape(*lead, d // 32, 4, 16, 4, 4, 2).permute(0, 1, 2, 6, 4, 7, 3, 8, 5)
    x = x.reshape(*lead, ROWS, d // GROUP, GROUP).float()
    x = x * param[..., :1] + param[..., 1:]
    return x.reshape(*lead[:2], lead[2] * ROWS, d)


def _turns(rot, dev):
    """The rotation of each pair by one position, in 2^-64 of a full turn (wrapped to the signed range)."""
    t = [int(round(ROT_BASE ** (-2.0 * p / rot) / (2.0 * math.pi) * 2.0 ** 64)) for p in range(rot // 2)]
    return torch.tensor([x - 2 ** 64 if x >= 2 ** 63 else x for x in t], dtype=torch.int64, device=dev)


def _rotated(x, pos, turns, rot, pairs):
    """float32 [B, T, H, d], pos long [B, T]."""
    if not rot:
        return x
    a = (pos[..., None] * turns >> 32).float() * (2.0 * math.pi / 2.0 ** 32)   # the product wraps at full turns
    c, s = a.cos()[:, :, None], a.sin()[:, :, None]
    r = x[..., :rot]
    x1, x2 = (r[..., :rot // 2], r[..., rot // 2:]) if pairs == "halves" else (r[..., 0::2], r[..., 1::2])
    y1, y2 = x1 * c - x2 * s, x2 * c + x1 * s
    y = torch.cat([y1, y2], -1) if pairs == "halves" else torch.stack([y1, y2], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


# ---------------------------------------------------------------- inputs
class _Draws:
    """Random tensors on the GPU from one seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=self.g).to(dtype)

    def whole(self, lo, hi, shape, dtype=torch.int64):
        return torch.randint(lo, hi + 1, shape, dtype=dtype, device=DEV, generator=self.g)

    def tables(self, B, columns, spare=3):
        """Pages scattered over a pool with a few to spare, and how many there are."""
        n = B * columns + spare
        order = torch.randperm(n, generator=self.g, device=DEV)
        return order[:B * columns].to(torch.int32).view(B, columns).contiguous(), n


def _fill(r, mem, cache, Hkv, d):
    """Rows of normal numbers in every page."""
    at = _places(cache, d, DEV)
    step = max(1, (1 << 27) // (Hkv * ROWS * d))
    for which in range(2):
        for p in range(0, mem.shape[1], step):
            out = mem[which, p:p + step]
            x = r.normal((out.shape[0], Hkv, ROWS, d))
            if cache == "bf16":
                inverse = torch.argsort(at[which].flatten())
                out.copy_(x.bfloat16().flatten(-2)[..., inverse].view(torch.uint8))
                continue
            codes, param = _code(x)
            byte = at[2 * which]
            byte = byte[:, 0::2] if which == 0 else byte.unflatten(-1, (-1, 2, 16))[:, :, 0].flatten(-2)
            inverse = torch.argsort(byte.flatten())
            out[..., :32 * d] = _nibbles(codes, which).flatten(-2)[..., inverse]
            out[..., 32 * d:] = param.flatten(-3).view(torch.uint8)


def _cache(r, case, n, filled):
    mem = torch.zeros((2, n, case["Hkv"], _page_bytes(case["cache"], case["d"])), dtype=torch.uint8, device=DEV)
    if filled:
        _fill(r, mem, case["cache"], case["Hkv"], case["d"])
    return mem


def _handle(s):
    """The library's cache over the same memory."""
    import paper_2405_05254_amd as yoco
    return yoco.PagedCache(s["mem"].shape[1], s["Hkv"], s["d"], yoco.INT4 if s["cache"] == "int4" else torch.bfloat16, mem=s["mem"])


def prepare(case, seed):
    r, s = _Draws(seed), dict(case)
    op = case["op"]
    if op == "append":
        B, T, N, Hq, Hkv, d = (case[x] for x in ("B", "T", "N", "Hq", "Hkv", "d"))
        s["table"], n = r.tables(B, -(-N // ROWS))
        s["mem"] = _cache(r, case, n, False)
        s["pos"] = torch.full((B,), N - T, dtype=torch.int64, device=DEV) if T == N or not case["ragged"] else r.whole(0, N - T, (B,))
        s["rows"] = r.whole(T // 2, T, (B,)) if case["ragged"] else None
        # one product of the projections: the rows of q, k and v lie side by side in it
        qkv = r.normal((B, T, Hq + 2 * Hkv, d), 1.0, torch.float32 if case["src"] == "f32" else torch.bfloat16)
        s["q"], s["k"], s["v"] = qkv.split([Hq, Hkv, Hkv], 2)
        s["turns"] = _turns(case["rot"], DEV) if case["rot"] else None
    elif op == "attend":
        B, T, N = case["B"], case["T"], case["N"]
        s["table"], n = r.tables(B, -(-N // ROWS))
        s["mem"] = _cache(r, case, n, True)
        s["lens"] = r.whole(max(T, N // 8), N, (B,)) if case["ragged"] else torch.full((B,), N, dtype=torch.int64, device=DEV)
        s["q"] = r.normal((B, T, case["Hq"], case["d"]), 1.0, torch.bfloat16)
        s["scale"] = 1.0 / math.sqrt(case["d"])
    elif op == "select":
        B, W, V = case["B"], case["W"], case["V"]
        s["logits"] = r.normal((B, W, V), 2.5, torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
        s["scores"] = -r.normal((B, W), 4.0).abs()
        s["done"] = r.whole(0, 3, (B, W)) == 0 if case["done"] else torch.zeros((B, W), dtype=torch.bool, device=DEV)
        s["eos"] = 2
    else:
        B, W, N = case["B"], case["W"], case["N"]
        columns = -(-N // ROWS) + 1
        s["home"], n = r.tables(B * W, columns)
        s["mem"] = _cache(r, case, n, True)
        # the prompt's pages are the first beam's, and so is what the beams have shared since
        s["table"] = s["home"].view(B, W, columns)[:, :1].expand(B, W, columns).reshape(B * W, columns).contiguous()
        tail = N // ROWS
        s["table"][:, tail] = s["home"][:, tail]
        s["lens"] = torch.full((B * W,), N, dtype=torch.int64, device=DEV)
        s["parent"] = r.whole(0, W - 1, (B, W), torch.int32)
        if case["kind"] == "states":
            s["states"] = [r.normal((B * W, case["H"], 128, 128)) for _ in range(case["layers"])]
        else:
            s["states"] = [r.normal((B * W, case["H"], case["window"], 128), 1.0, torch.bfloat16) for _ in range(2 * case["layers"])]
    if own and "mem" in s:
        s["handle"] = _handle(s)
    return s


# ---------------------------------------------------------------- one pass, in plain operations
def _append(s):
    B, T, Hkv, d, cache = (s[x] for x in ("B", "T", "Hkv", "d", "cache"))
    pos = s["pos"][:, None] + torch.arange(T, device=DEV)
    q = _rotated(s["q"].float(), pos, s["turns"], s["rot"], s["pairs"]).to(s["q"].dtype)
    k, v = _rotated(s["k"].float(), pos, s["turns"], s["rot"], s["pairs"]), s["v"].float()
    page = s["table"].long().gather(1, pos // ROWS)
    new = (torch.arange(T, device=DEV) < (s["rows"][:, None] if s["rows"] is not None else T)).expand(B, T)
    head = (page[..., None] * Hkv + torch.arange(Hkv, device=DEV))[new]                # page and head of every row that is new
    row, size, at = (pos % ROWS)[new], _page_bytes(cache, d), _places(cache, d, DEV)
    for which, x in enumerate((k, v)):
        plane = s["mem"][which].view(-1)
        if cache == "bf16":
            plane.view(torch.bfloat16)[head[..., None] * (size // 2) + at[which][row][:, None]] = x[new].bfloat16()
            continue
        codes, param = _code(x[new])
        byte = at[2 * which][row]
        byte = byte[:, 0::2] if which == 0 else byte.unflatten(-1, (-1, 2, 16))[:, :, 0].flatten(-2)
        plane[head[..., None] * size + byte[:, None]] = _nibbles(codes, which)
        n = 4 * (d // GROUP)
        plane[head[..., None] * size + 32 * d + (row * n)[:, None, None] + torch.arange(n, device=DEV)] = param.flatten(-2).view(torch.uint8)
    if cache == "bf16":
        return {"q": q, "mem": s["mem"].view(torch.bfloat16)}
    first = s["pos"][:, None] // ROWS + torch.arange((T + ROWS - 2) // ROWS + 1, device=DEV)      # the pages that hold the rows
    pages = s["table"].long().gather(1, first.clamp(max=s["table"].shape[1] - 1))
    at = (pos - s["pos"][:, None] // ROWS * ROWS)[:, None, :, None].expand(B, Hkv, T, d)
    k, v = (_values(s["mem"][which], cache, d, which, pages).gather(2, at).transpose(1, 2).bfloat16() for which in range(2))
    return {"q": q, "k": k.contiguous(), "v": v.contiguous()}


def _attend(s):
    B, T, Hq, Hkv, d = (s[x] for x in ("B", "T", "Hq", "Hkv", "d"))
    pages = s["table"].long()
    k = _values(s["mem"][0], s["cache"], d, 0, pages)
    G, N = Hq // Hkv, k.shape[2]
    q = s["q"].float().view(B, T, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, d)
    p = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    del k
    seen = (s["lens"][:, None] - T + 1 + torch.arange(T, device=DEV))[:, None, :, None, None]                   # rows that each query row sees
    p = p.view(B, Hkv, T, G, N).masked_fill_(torch.arange(N, device=DEV) >= seen, float("-inf"))
    p = torch.exp(p - p.amax(-1, keepdim=True))
    p = (p / p.sum(-1, keepdim=True)).view(B, Hkv, T * G, N)
    o = torch.matmul(p, _values(s["mem"][1], s["cache"], d, 1, pages))
    return o.view(B, Hkv, T, G, d).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, d).bfloat16()


def _select(s):
    B, W, V = s["B"], s["W"], s["V"]
    x = s["logits"].float()
    most = x.amax(-1, keepdim=True)
    lse = most + torch.log(torch.exp(x - most).sum(-1, keepdim=True))
    best, token = torch.sort(x, dim=-1, descending=True, stable=True)          # a beam's candidates, equal ones by their index
    best, token = best[..., :W], token[..., :W]
    score = s["scores"][..., None] + (best - lse)
    done = s["done"][..., None]                                                # a finished beam stays as it is
    first = torch.arange(W, device=DEV) == 0
    score = torch.where(done, torch.where(first, s["scores"][..., None], float("-inf")), score)
    token = torch.where(done, s["eos"], token)
    score, at = torch.sort(score.view(B, W * W), dim=-1, descending=True, stable=True)
    score, at = score[:, :W], at[:, :W]
    token = token.reshape(B, W * W).gather(1, at)
    parent = at // W
    return {"parent": parent.int(), "token": token.int(), "scores": score, "done": s["done"].gather(1, parent) | (token == s["eos"])}


def _reorder(s):
    B, W = s["B"], s["W"]
    parent = (s["parent"].long() + torch.arange(B, device=DEV)[:, None] * W).view(-1)
    tail = (s["lens"] // ROWS)[:, None]
    table = s["table"][parent]
    into = s["home"].gather(1, tail)
    source = torch.where((s["lens"] % ROWS)[:, None] > 0, table.gather(1, tail), into)
    s["mem"][:, into.view(-1).long()] = s["mem"][:, source.view(-1).long()]
    s["table"].copy_(table.scatter(1, tail, into))
    [x.copy_(x[parent]) for x in s["states"]]
    return {"table": s["table"], "mem": s["mem"], "states": s["states"]}


# ---------------------------------------------------------------- the same through the library
def _library(s):
    import paper_2405_05254_amd as yoco
    op = s["op"]
    if op == "append":
        q = yoco.paged_append(s["handle"], s["table"], s["pos"], s["k"], s["v"], rows=s["rows"], q=s["q"], turns=s["turns"], neighbours=s["pairs"] == "neighbours")
        if s["cache"] == "bf16":
            return {"q": q, "mem": s["mem"].view(torch.bfloat16)}
        k, v = yoco.paged_read(s["handle"], s["table"], s["pos"], s["T"])
        return {"q": q, "k": k, "v": v}
    if op == "attend":
        return yoco.paged_attn(s["handle"], s["table"], s["q"], s["lens"], s["scale"])
    if op == "select":
        parent, token, scores, done = yoco.beam_select(s["logits"], s["scores"], done=s["done"], eos=s["eos"])
        return {"parent": parent, "token": token, "scores": scores, "done": done}
    yoco.beam_reorder_pages(s["handle"], s["table"], s["home"], s["parent"], s["lens"])
    yoco.beam_reorder_rows(s["states"], s["parent"])
    return {"table": s["table"], "mem": s["mem"], "states": s["states"]}


def run(s):
    return _library(s) if own else {"append": _append, "attend": _attend, "select": _select, "reorder": _reorder}[s["op"]](s)


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_turn(x, pos, case):
    """x float64 [T, H, d] at positions pos [T]."""
    rot, y = case["rot"], x.clone()
    for p in range(rot // 2):
        i, j = (p, p + rot // 2) if case["pairs"] == "halves" else (2 * p, 2 * p + 1)
        a = pos.double() * ROT_BASE ** (-2.0 * p / rot)
        c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
        y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y


def _exact_rows(s, which, b, g, n):
    """The first n rows of a sequence and KV head, from the layout's definition, float64 [n, d]."""
    d, at = s["d"], _places(s["cache"], s["d"], DEV)
    r = torch.arange(n, device=DEV)
    raw = s["mem"][which, :, g][s["table"][b].long()][r // ROWS]                # the page of every row
    if s["cache"] == "bf16":
        return raw.view(torch.bfloat16).gather(1, at[which][r % ROWS]).double()
    byte, nibble = at[2 * which][r % ROWS], at[2 * which + 1][r % ROWS]
    code = raw.gather(1, byte) >> 4 * nibble & 15
    param = raw[:, 32 * d:].contiguous().view(torch.bfloat16).view(n, ROWS, d // GROUP, 2)[r, r % ROWS].double()
    group = torch.arange(d, device=DEV) // GROUP
    return param[:, group, 1] + param[:, group, 0] * code.double()


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "append":
        q = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
        for b in range(case["B"]):
            pos = s["pos"][b] + torch.arange(case["T"], device=DEV)
            q[b] = _exact_turn(s["q"][b].double(), pos, case)
        return {"q": q, "mem": None} if case["cache"] == "bf16" else {"q": q, "k": None, "v": None}
    if op == "attend":
        T, G = case["T"], case["Hq"] // case["Hkv"]
        if case["B"] * case["Hkv"] * case["N"] > 1 << 23:
            return None
        o = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
        for b, n in enumerate(s["lens"].tolist()):
            for g in range(case["Hkv"]):
                k, v = _exact_rows(s, 0, b, g, n), _exact_rows(s, 1, b, g, n)
                for i in range(T):
                    m = n - T + 1 + i
                    w = torch.softmax(s["q"][b, i, g * G:(g + 1) * G].double() @ k[:m].t() * s["scale"], -1)
                    o[b, i, g * G:(g + 1) * G] = w @ v[:m]
        return o
    if op == "select":
        scores = torch.empty((case["B"], case["W"]), dtype=torch.float64, device=DEV)
        for b in range(case["B"]):
            x = torch.log_softmax(s["logits"][b].double(), -1) + s["scores"][b].double()[:, None]
            x[s["done"][b]] = float("-inf")
            x[s["done"][b], s["eos"]] = s["scores"][b][s["done"][b]].double()
            scores[b] = torch.topk(x.view(-1), case["W"]).values
        return {"parent": None, "token": None, "scores": scores, "done": None}
    beams = [b * case["W"] + p for b, chosen in enumerate(s["parent"].tolist()) for p in chosen]
    return {"table": None, "mem": None, "states": [torch.stack([x[i] for i in beams]).double() for x in s["states"]]}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    op = case["op"]
    if op == "append":
        rows, Hq, Hkv, d = case["B"] * case["T"], case["Hq"], case["Hkv"], case["d"]
        new = rows * 3 // 4 if case["ragged"] else rows
        size = 4 if case["src"] == "f32" else 2
        cached = 2 * Hkv * _page_bytes(case["cache"], d) // ROWS
        back = new * cached + rows * 2 * Hkv * d * 2 if case["cache"] == "int4" else 0      # read again as the values they stand for
        return {"bytes": rows * 2 * Hq * d * size + new * (2 * Hkv * d * size + cached) + back,
                "flops": 3 * rows * (Hq + Hkv) * case["rot"] + new * 2 * Hkv * d * (5 if case["cache"] == "int4" else 0)}
    if op == "attend":
        B, T, Hq, Hkv, d = (case[x] for x in ("B", "T", "Hq", "Hkv", "d"))
        n = case["N"] * 9 // 16 if case["ragged"] else case["N"]
        return {"bytes": B * (2 * n * Hkv * _page_bytes(case["cache"], d) // ROWS + 2 * T * Hq * d * 2), "flops": 4 * d * B * T * Hq * n}
    if op == "select":
        n = case["B"] * case["W"] * case["V"]
        return {"bytes": n * (4 if case["dtype"] == "f32" else 2), "flops": 4 * n}
    beams, moved = case["B"] * case["W"], (case["W"] - 1) / case["W"]                        # a beam's parent is another one, as drawn
    state = case["layers"] * case["H"] * 128 * (128 * 4 if case["kind"] == "states" else 2 * case["window"] * 2)
    page = 2 * case["Hkv"] * _page_bytes(case["cache"], case["d"]) if case["N"] % ROWS else 0
    table = 4 * (case["N"] // ROWS + 1)
    return {"bytes": int(beams * 2 * (moved * (state + page) + table)), "flops": 0}
