"""The cache in pages and beam search, from their definitions: the place of every value in a page, the float32 rule that
decides a 4-bit code, rotation by positions and attention in float64, selection over sorted candidates, reordering one beam at a
time. Plain numpy, nothing shared with the library."""
import math

import numpy as np

ROWS, GROUP = 64, 64


def bf16(x):
    """float32 -> bfloat16 values (round to nearest even), as float32."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    r = (u + (((u >> 16) & 1) + np.uint32(0x7FFF))) & np.uint32(0xFFFF0000)
    return np.where(np.isnan(x), np.float32(np.nan), r.view(np.float32))


def page_bytes(d, coded):
    return 36 * d if coded else 128 * d


def places(d, coded):
    """For row r and dimension e of a page (index arrays [64,d]): K and V as element (bf16), or as byte and nibble (4 bits)."""
    r, e = np.meshgrid(np.arange(ROWS), np.arange(d), indexing="ij")
    i = r // 16 * (d // 32) + e // 32
    if not coded:
        return (((i * 64 + e // 8 % 4 * 16 + r % 16) * 8 + e % 8), ((e // 16 * 2 + r // 32) * 64 + r % 16 // 4 * 16 + e % 16) * 8 + r // 16 % 2 * 4 + r % 4)
    k = (i // 4 * 64 + e // 8 % 4 * 16 + r % 16) * 16 + i % 4 * 4 + e % 8 // 2
    v = (e // 32 * 64 + r % 16 // 4 * 16 + e % 16) * 16 + r // 16 * 4 + r % 4
    return (k, e % 2), (v, e // 16 % 2)


def code(x):
    """float32 [..., d] -> codes [..., d] (uint8), scale and minimum [..., d/64] (bf16 values). Every step rounds to float32."""
    f = np.float32
    g = np.ascontiguousarray(x, dtype=f).reshape(x.shape[:-1] + (-1, GROUP))
    with np.errstate(all="ignore"):
        lo, hi = g.min(-1), g.max(-1)
        span = (hi - lo).astype(f)
        scale, base = bf16((span * f(1.0 / 15.0)).astype(f)), bf16(lo)
        scale = np.where(scale < f(2.0 ** -126), f(0), scale)
        bad = ~(np.isfinite(g).all(-1) & np.isfinite(span) & np.isfinite(scale) & np.isfinite(base))
        inv = np.where(scale > 0, (f(1) / np.where(scale > 0, scale, f(1))).astype(f), f(0))
        y = ((g - base[..., None]).astype(f) * inv[..., None]).astype(f)
        c = np.clip(np.rint(np.where(np.isfinite(y), y, f(0))), 0, 15)
    c = np.where(bad[..., None], 0, c).astype(np.uint8).reshape(x.shape)
    return c, np.where(bad, f(0), scale), np.where(bad, f(np.nan), base)


def stands_for(codes, scale, base):
    """float64 values of codes [..., d]."""
    c = codes.reshape(codes.shape[:-1] + (-1, GROUP)).astype(np.float64)
    return (base[..., None].astype(np.float64) + scale[..., None].astype(np.float64) * c).reshape(codes.shape)


def read_pool(mem, n_pages, Hkv, d, coded):
    """uint8 memory of a pool -> K and V [n_pages,Hkv,64,d]: bf16 values, or (codes, scale, minimum)."""
    raw = np.asarray(mem).reshape(2, n_pages, Hkv, page_bytes(d, coded))
    out = []
    for which, at in enumerate(places(d, coded)):
        x = raw[which]
        if not coded:
            bits = np.ascontiguousarray(x).view(np.uint16)[..., at].astype(np.uint32) << 16
            out.append(bits.view(np.float32))
            continue
        byte, nibble = at
        c = (x[..., byte] >> (4 * nibble)) & 15
        param = np.ascontiguousarray(x[..., 32 * d:]).view(np.uint16).reshape(n_pages, Hkv, ROWS, d // GROUP, 2).astype(np.uint32) << 16
        param = param.view(np.float32)
        out.append((c.astype(np.uint8), param[..., 0], param[..., 1]))
    return out


def turns(angles):
    """Whole 2^-64 turns of angles in radians, in exact arithmetic of their float64 quotient."""
    return [int(round(a / (2 * math.pi) * 2 ** 64)) % 2 ** 64 for a in angles]


def rotate(x, pos, units, neighbours):
    """float64 [H,d] at position pos: the first 2 len(units) dimensions turned by pos * units 2^-64 turns."""
    y, half = np.array(x, dtype=np.float64), len(units)
    for p, u in enumerate(units):
        i, j = (2 * p, 2 * p + 1) if neighbours else (p, p + half)
        a = 2 * math.pi * ((pos * u) % 2 ** 64) / 2 ** 64
        y[:, i] = x[:, i] * math.cos(a) - x[:, j] * math.sin(a)
        y[:, j] = x[:, j] * math.cos(a) + x[:, i] * math.sin(a)
    return y


def attend(q, k, v, n, scale):
    """q [T,Hq,d], the last T of n rows; k, v [Hkv,N,d] with a row of NaN in k where no page is; float64 [T,Hq,d]."""
    T, Hq, d = q.shape
    G, o = Hq // k.shape[0], np.zeros(q.shape)
    for i in range(T):
        m = n - T + 1 + i
        for h in range(Hq):
            if m <= 0:
                continue
            K, V = k[h // G, :m].astype(np.float64), v[h // G, :m].astype(np.float64)
            there = ~np.isnan(K[:, 0])
            if not there.any():
                continue
            s = scale * (K[there] @ q[i, h].astype(np.float64))
            w = np.exp(s - s.max())
            o[i, h] = (w / w.sum()) @ V[there]
    return o


def select(logits, scores, done, eos):
    """One request: logits [W,V] float32 values, scores [W], done [W] -> lists of parent, token, score (float64), done."""
    W, V = logits.shape
    found = []
    for w in range(W):
        base = float(scores[w])
        if math.isnan(base) or base == -math.inf:
            continue
        if done is not None and done[w]:
            found.append((base, w, 0.0, eos))
            continue
        x = logits[w].astype(np.float64)
        x = np.where(np.isnan(x), -np.inf, np.minimum(x, float(np.finfo(np.float32).max)))
        if not (x > -np.inf).any():
            continue
        top = x.max()
        lse = top + math.log(np.exp(x - top).sum())
        order = np.lexsort((np.arange(V), -x))[:W]
        found += [(base + (x[t] - lse), w, x[t], int(t)) for t in order if x[t] > -np.inf]
    found.sort(key=lambda c: (-c[0], c[1], -c[2], c[3]))
    word = eos if eos >= 0 else 0
    out = [(c[1], c[3], c[0]) for c in found[:W]]
    out += [(w, word, -math.inf) for w in range(len(out), W)]
    ended = [bool(done is not None and done[p]) or (eos >= 0 and t == eos) for p, t, _ in out]
    return [p for p, _, _ in out], [t for _, t, _ in out], [s for _, _, s in out], ended


def reorder_pages(k, v, table, home, parent, lens):
    """k, v: pools [n_pages, ...]; table, home [B,W,cols]; parent [B,W]; lens [B]. New copies of (k, v, table)."""
    k2, v2, table2 = k.copy(), v.copy(), table.copy()
    B, W, cols = table.shape
    for b in range(B):
        n = int(lens[b])
        tail = max(n, 0) // ROWS
        for w in range(W):
            p = int(parent[b, w])
            p = p if 0 <= p < W else w
            table2[b, w] = table[b, p]
            if tail >= cols:
                continue
            src, dst = int(table[b, p, tail]), int(home[b, w, tail])
            table2[b, w, tail] = dst
            if n > 0 and n % ROWS and 0 <= src < len(k) and 0 <= dst < len(k):
                k2[dst], v2[dst] = k[src], v[src]
    return k2, v2, table2
