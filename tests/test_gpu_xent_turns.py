"""The softmax cross-entropy over so many rows that its blocks take them in several
turns, labels and logits of later turns being loaded ahead: row by row against the
formulas in 64 bits."""
import pytest
import torch

import paper_2010_07565_amd as bg
import rowops as ro

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    bg.load()


def reference(z, labels, weight):
    """rowops.xent over whole arrays of finite logits: row losses, gradient and their
    bounds (float64, on the GPU)."""
    rows, cols = z.shape
    has = (labels >= 0) & (labels < cols)
    y = torch.where(has, labels, 0).long()[:, None]
    m = z.amax(1, keepdim=True)
    t = z - m
    e = t.exp()
    s = e.sum(1, keepdim=True)
    p, at = e / s, z.gather(1, y)
    rel = ro.U * (8 * t.abs() + 64)
    hot = torch.zeros_like(z).scatter_(1, y, 1.0)
    own = (e * rel).sum(1, keepdim=True) / s
    g = weight * (p - hot)
    dg = abs(weight) * (p * (rel + own) + 4 * ro.U * hot) + 4 * ro.U * g.abs() + 2.0 ** -125
    l = m + s.log() - at
    dl = own + 4 * ro.U * (m.abs() + s.log().abs() + at.abs())
    on = has[:, None]
    return [torch.where(on, v, 0) for v in (l, dl, g, dg)]


def inside(got, want, bound, dtype, what):
    """|got - want| within the bound and the rounding to dtype."""
    rel, least = ro.STORED[dtype]
    over = ~((got.double() - want).abs() <= bound + rel * (want.abs() + bound) + least)
    assert not bool(over.any()), "%s: %d of %d outside" % (what, int(over.sum()), over.numel())


# 1, 16 and 64 lanes a row and 4 waves a row, at least three turns of every block and a
# last one that is not whole
@pytest.mark.parametrize("cols,rows,dtype", [
    (3, 800001, torch.float32), (4, 1400003, torch.float16), (7, 700001, torch.bfloat16),
    (32, 400001, torch.bfloat16), (47, 200003, torch.float32), (47, 200003, torch.bfloat16),
    (100, 50001, torch.float32), (200, 50001, torch.float16), (300, 13001, torch.float32),
    (1000, 13001, torch.bfloat16), (2000, 3501, torch.float32), (5000, 3301, torch.float16)])
@pytest.mark.parametrize("labelled", [0.02, 0.5, 1.0])
@pytest.mark.parametrize("layout", ["dense", "gaps", "in place"])
def test_several_turns(cols, rows, dtype, labelled, layout):
    gen = torch.Generator("cuda").manual_seed(cols)
    pad = 3 if layout == "gaps" else 0
    y = torch.randint(0, cols, (rows,), device="cuda", generator=gen, dtype=torch.int32)
    off = torch.rand(rows, device="cuda", generator=gen) >= labelled
    y[off] = torch.randint(-3, 0, (int(off.sum()),), device="cuda", generator=gen, dtype=torch.int32)
    y[off & (y == -3)] = cols
    flat = torch.full((rows, cols + pad), float("nan"), dtype=dtype, device="cuda")
    z = flat[:, :cols]
    z.copy_((3 * torch.randn(rows, cols, device="cuda", generator=gen)).to(dtype))
    l, dl, g, dg = reference(z.double(), y, 0.25)
    z[off] = float("nan")                              # not read
    out = z if layout == "in place" else torch.full_like(flat, 9.0)[:, :cols]
    loss, row = torch.empty(1, device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    ws = torch.full((bg.softmax_xent_workspace_bytes(rows, cols),), 255, dtype=torch.uint8, device="cuda")
    bg.bigcn_softmax_xent(z, y, 0.25, loss=loss, row_loss=row, dlogits=out, workspace=ws)
    inside(row[:, None], l, dl, torch.float32, "row losses")
    total = 0.25 * l.sum()
    inside(loss, total, 0.25 * dl.sum() + 2 * ro.U * total.abs(), torch.float32, "loss")
    inside(out, g, dg, dtype, "gradient")
    if pad:
        assert bool((out.as_strided((rows - 1, pad), (cols + pad, 1), cols) == 9.0).all())
