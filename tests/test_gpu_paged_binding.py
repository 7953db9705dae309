"""What the calls over a cache in pages refuse when they are given tensors: shapes, types, strides, devices and workspaces that do not fit."""
import pytest
import torch

pytestmark = pytest.mark.gpu

B, T, Hq, Hkv, d, cols = 2, 3, 4, 2, 128, 2


@pytest.fixture(scope="module")
def yoco():
    import paper_2405_05254_amd as y
    y.lib()
    assert torch.cuda.is_available()
    return y


def good(yoco):
    cache = yoco.PagedCache(B * cols, Hkv, d, yoco.INT4)
    cache.mem.zero_()
    bf = dict(device="cuda", dtype=torch.bfloat16)
    return dict(cache=cache, table=torch.arange(B * cols, device="cuda", dtype=torch.int32).view(B, cols), pos=torch.zeros(B, dtype=torch.int64, device="cuda"),
                k=torch.ones(B, T, Hkv, d, **bf), v=torch.ones(B, T, Hkv, d, **bf), q=torch.ones(B, T, Hq, d, **bf), turns=yoco.rotation_turns(d),
                rows=torch.full((B,), T, dtype=torch.int64, device="cuda"), lens=torch.full((B,), T, dtype=torch.int64, device="cuda"))


APPEND = [
    ("k of another batch", lambda g: g.update(k=g["k"][:1], v=g["v"][:1])),
    ("heads that the cache does not have", lambda g: g.update(k=g["q"], v=g["q"])),
    ("another head size", lambda g: g.update(k=g["k"][..., :64].contiguous(), v=g["v"][..., :64].contiguous())),
    ("k and v of two types", lambda g: g.update(v=g["v"].float())),
    ("a type that is no source", lambda g: g.update(k=g["k"].half(), v=g["v"].half(), q=None)),
    ("elements that are apart", lambda g: g.update(k=torch.ones(B, T, Hkv, 2 * d, device="cuda", dtype=torch.bfloat16)[..., ::2])),
    ("rows that are unevenly apart", lambda g: g.update(k=torch.ones(B, T + 1, Hkv, d, device="cuda", dtype=torch.bfloat16)[:, :T])),
    ("q of another type", lambda g: g.update(q=g["q"].float())),
    ("q of another length", lambda g: g.update(q=g["q"][:, :2].contiguous())),
    ("a table of another type", lambda g: g.update(table=g["table"].long())),
    ("a table of one dimension", lambda g: g.update(table=g["table"].view(-1))),
    ("a table that is no dense matrix", lambda g: g.update(table=torch.zeros(cols, B, dtype=torch.int32, device="cuda").t())),
    ("positions of another type", lambda g: g.update(pos=g["pos"].int())),
    ("positions of another batch", lambda g: g.update(pos=g["pos"][:1])),
    ("rows of another batch", lambda g: g.update(rows=g["rows"][:1])),
    ("turns of another type", lambda g: g.update(turns=g["turns"].double())),
    ("turns of more than a head", lambda g: g.update(turns=yoco_turns(256))),
    ("turns of 12 dimensions", lambda g: g.update(turns=g["turns"][:6])),
    ("k on the host", lambda g: g.update(k=g["k"].cpu())),
    ("a table on the host", lambda g: g.update(table=g["table"].cpu())),
]


def yoco_turns(dims):
    import paper_2405_05254_amd as y
    return y.rotation_turns(dims)


@pytest.mark.parametrize("what,change", APPEND, ids=[x[0] for x in APPEND])
def test_append_refuses(yoco, what, change):
    g = good(yoco)
    yoco.paged_append(g["cache"], g["table"], g["pos"], g["k"], g["v"], rows=g["rows"], q=g["q"], turns=g["turns"])
    torch.cuda.synchronize()
    before = g["cache"].mem.clone()
    change(g)
    with pytest.raises(yoco.YocoError):
        yoco.paged_append(g["cache"], g["table"], g["pos"], g["k"], g["v"], rows=g["rows"], q=g["q"], turns=g["turns"])
    torch.cuda.synchronize()
    assert torch.equal(before, g["cache"].mem)


ATTEND = [
    ("q of float32", lambda g: g.update(q=g["q"].float())),
    ("q of another batch", lambda g: g.update(q=g["q"][:1])),
    ("q of another head size", lambda g: g.update(q=g["q"][..., :64].contiguous())),
    ("query heads that do not divide", lambda g: g.update(q=g["q"][:, :, :3].contiguous())),
    ("q that is not dense", lambda g: g.update(q=g["q"].transpose(1, 2).contiguous().transpose(1, 2))),
    ("lens of another type", lambda g: g.update(lens=g["lens"].int())),
    ("lens of another batch", lambda g: g.update(lens=g["lens"][:1])),
    ("an output of another shape", lambda g: g.update(out=g["q"][:1])),
    ("an output of another type", lambda g: g.update(out=g["q"].float())),
    ("a workspace that is too small", lambda g: g.update(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))),
    ("a workspace on the host", lambda g: g.update(workspace=torch.empty(1 << 24, dtype=torch.uint8))),
    ("q on the host", lambda g: g.update(q=g["q"].cpu())),
]


@pytest.mark.parametrize("what,change", ATTEND, ids=[x[0] for x in ATTEND])
def test_attention_refuses(yoco, what, change):
    g = dict(good(yoco), out=None, workspace=None)
    change(g)
    with pytest.raises(yoco.YocoError):
        yoco.paged_attn(g["cache"], g["table"], g["q"], g["lens"], 0.1, workspace=g["workspace"], out=g["out"])


def test_read_refuses(yoco):
    g = good(yoco)
    for args, kw in (((g["table"], g["pos"], -1), {}), ((g["table"], g["pos"][:1], 2), {}), ((g["table"].cpu(), g["pos"], 2), {}), ((g["table"], g["pos"], 2), dict(dtype=torch.float16))):
        with pytest.raises(yoco.YocoError):
            yoco.paged_read(g["cache"], *args, **kw)
    with pytest.raises(TypeError):
        yoco.paged_read(g["cache"], g["table"], [0, 0], 2)
