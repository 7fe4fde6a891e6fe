"""Layer norm over so many rows that its blocks take them in several turns and, for the
gradients of gamma and beta, in several runs of turns: element by element against the
formulas in 64 bits, which are evaluated in pieces on the GPU."""
import numpy as np
import pytest
import torch

import paper_2010_07565_amd as bg
import rowops as ro

pytestmark = pytest.mark.gpu

GUARD = 4096     # bytes behind a workspace that have to stay as they were


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    bg.load()


def inside(got, want, bound, dtype, what):
    """|got - want| within the bound and the rounding to dtype (float64 on the GPU)."""
    rel, least = ro.STORED[dtype]
    bound = bound + rel * (want.abs() + bound) + least
    over = ~((got.double() - want).abs() <= bound)
    assert not bool(over.any()), "%s: %d of %d outside" % (what, int(over.sum()), over.numel())


def gradients(dy, mean, rstd, gamma, x=None, codes=None, qscale=None, act="none"):
    """One call over poisoned outputs and workspace; nothing behind the workspace moves."""
    rows, cols = dy.shape
    need = bg.layernorm_backward_workspace_bytes(rows, cols)
    flat = torch.full((need + GUARD,), 255, dtype=torch.uint8, device="cuda")
    dx = torch.full_like(dy, float("nan"))
    dg, db = (torch.full((cols,), float("nan"), device="cuda") for _ in range(2))
    bg.bigcn_layernorm_backward(dy, mean, rstd, x=x, codes=codes, qscale=qscale, gamma=gamma, act=act,
                                dx=dx, dgamma=dg, dbeta=db, workspace=flat[:need])
    assert bool((flat[need:] == 255).all())
    return dx, dg, db


# (columns, rows): 16, 8 and 4 rows of a block in a wave's lanes, a row a block of 2, 4
# and 8 waves; rows are for two runs and a part of a third with as many blocks as the
# narrowest types get, with a last turn that is not whole
LONG = [(1, 2500003), (5, 2500003), (64, 2300003), (256, 1100003), (513, 560003), (1433, 280003),
        (1537, 260003), (2049, 210003), (5000, 70001)]


@pytest.mark.parametrize("cols,rows", LONG)
@pytest.mark.parametrize("source", ["x", "q8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_gradients_over_several_runs(cols, rows, source, dtype):
    gen = torch.Generator("cuda").manual_seed(cols)
    x = torch.randn(rows, cols, device="cuda", generator=gen).to(dtype)
    x.add_(0.5).clamp_(min=0)                       # a ReLU's output
    dy = torch.randn(rows, cols, device="cuda", generator=gen).add_(0.25).to(dtype)
    gamma = torch.rand(cols, device="cuda", generator=gen).add_(0.5)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    codes = torch.empty(rows, cols, dtype=torch.int8, device="cuda")
    qscale = torch.empty(rows, bg.checkpoint_groups(cols), device="cuda")
    bg.bigcn_layernorm(x, eps=ro.EPS, mean=mean, rstd=rstd, codes=codes, qscale=qscale)
    if source == "x":
        dx, dg, db = gradients(dy, mean, rstd, gamma, x=x, act="relu")
    else:
        dx, dg, db = gradients(dy, mean, rstd, gamma, codes=codes, qscale=qscale, act="relu")
    again = gradients(dy, mean, rstd, gamma, **(dict(x=x) if source == "x" else dict(
        codes=codes, qscale=qscale)), act="relu")
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dg, db)))
    del again
    want = [torch.zeros(cols, dtype=torch.float64, device="cuda") for _ in range(2)]
    bound = [torch.zeros(cols, dtype=torch.float64, device="cuda") for _ in range(2)]
    step = max(1, 40_000_000 // cols)
    for a in range(0, rows, step):
        b = min(rows, a + step)
        xs = x[a:b].double()
        if source == "q8":
            xs = codes[a:b].double() * qscale[a:b].double().repeat_interleave(64, 1)[:, :cols]
        ds, m, r = dy[a:b].double(), mean[a:b, None].double(), rstd[a:b, None].double()
        xh, g = (xs - m) * r, ds * gamma.double()
        # (the bounds of rowops.norm_grad)
        dxh = r * 2 * ro.U * (xs.abs() + m.abs())
        c1, c2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
        a1, a2 = g.abs().mean(1, keepdim=True), (g * xh).abs().mean(1, keepdim=True)
        ref = r * (g - c1 - xh * c2)
        lim = r * (4 * ro.U * g.abs() + (ro.ROW + 4 * ro.U) * a1 + (ro.ROW + 10 * ro.U) * xh.abs() * a2
                   + dxh * c2.abs() + xh.abs() * (g.abs() * dxh).mean(1, keepdim=True)) \
            + 4 * ro.U * ref.abs() + 4 * ro.TINY
        on = xs > 0
        inside(dx[a:b], torch.where(on, ref, 0), torch.where(on, lim, 0), dtype, "dx")
        want[0] += (ds * xh).sum(0)
        want[1] += ds.sum(0)
        bound[0] += (ro.COLUMN + 6 * ro.U) * (ds * xh).abs().sum(0) + (ds.abs() * dxh).sum(0)
        bound[1] += ro.COLUMN * ds.abs().sum(0)
    inside(dg, want[0], bound[0], torch.float32, "dgamma")
    inside(db, want[1], bound[1], torch.float32, "dbeta")


def test_error_of_column_sums_does_not_grow_with_the_rows():
    """One row in 256 of a column has the gradient 2^23 + 127, two million rows in all.
    Sums of 511 of them in 32 bits lose 127 units an addition from the 256th on, more
    than the bound of 100 roundings allows: runs are short and joined in 64 bits."""
    rows, each = 511 * (1 << 20), 1 << 14
    value = float((1 << 23) + 127)
    dy = torch.zeros(rows, 1, device="cuda")
    # (of each run of 64 turns of the blocks the first turn, and a wave's first row in it)
    dy.view(-1, 64, each)[:, 0, ::4] = value
    x, mean, rstd = torch.ones_like(dy), torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    dg, db = (torch.full((1,), float("nan"), device="cuda") for _ in range(2))
    ws = torch.full((bg.layernorm_backward_workspace_bytes(rows, 1),), 255, dtype=torch.uint8, device="cuda")
    bg.bigcn_layernorm_backward(dy, mean, rstd, x=x, dgamma=dg, dbeta=db, workspace=ws)
    want = value * (rows // 64 // 4)
    assert abs(float(db) - want) <= ro.COLUMN * want
    assert abs(float(dg) - want) <= (ro.COLUMN + 8 * ro.U) * want      # (xhat = 1: two roundings)


@pytest.mark.parametrize("cols,rows", [(3, 300001), (64, 80003), (100, 60001), (300, 40001),
                                       (602, 20003), (1433, 9001), (1537, 7001), (2049, 5003),
                                       (5000, 5003), (8192, 4099)])
@pytest.mark.parametrize("dtype", ro.TYPES, ids=["f32", "f16", "bf16"])
def test_forward_over_several_turns(cols, rows, dtype):
    """Every output of each row against its formula, where a block takes rows in turn."""
    gen = torch.Generator("cuda").manual_seed(cols)
    x = torch.randn(rows, cols, device="cuda", generator=gen)
    x = (x * torch.randn(rows, 1, device="cuda", generator=gen).exp()
         + torch.randn(rows, 1, device="cuda", generator=gen)).to(dtype)
    gamma = torch.rand(cols, device="cuda", generator=gen).mul_(3).sub_(1.5)
    beta = torch.rand(cols, device="cuda", generator=gen).sub_(0.5)
    q = bg.checkpoint_groups(cols)
    y, mean, rstd = torch.full_like(x, float("nan")), *(torch.full((rows,), float("nan"), device="cuda")
                                                        for _ in range(2))
    codes = torch.full((rows, cols), 77, dtype=torch.int8, device="cuda")
    qscale = torch.full((rows, q), float("nan"), device="cuda")
    bits, scale = torch.zeros(rows, q, dtype=torch.int64, device="cuda"), torch.empty(rows, device="cuda")
    bg.bigcn_layernorm(x, gamma, beta, eps=ro.EPS, y=y, mean=mean, rstd=rstd, codes=codes, qscale=qscale,
                       bits=bits, scale=scale)
    over = x.clone()
    bg.bigcn_layernorm(over, gamma, beta, eps=ro.EPS, y=over)
    assert torch.equal(over, y)
    alone = torch.empty_like(codes), torch.empty_like(qscale)
    bg.bigcn_checkpoint_q8(x, *alone)
    assert torch.equal(alone[0], codes) and torch.equal(alone[1], qscale)
    back = torch.empty_like(x, dtype=torch.float32)
    bg.bigcn_restore_q8(codes, qscale, back)
    assert torch.equal(torch.sign(back), torch.sign(x).float())
    step = qscale.repeat_interleave(64, 1)[:, :cols]
    assert bool(((back - x.float()).abs() <= step * 1.00001).all())
    # (the formulas and bounds of rowops.norm)
    x64, g64, b64 = x.double(), gamma.double(), beta.double()
    m = x64.mean(1, keepdim=True)
    c = x64 - m
    r = 1 / ((c * c).mean(1, keepdim=True) + float(np.float32(ro.EPS))).sqrt()
    ref = g64 * c * r + b64
    dm = ro.ROW * x64.abs().mean(1, keepdim=True) + ro.U * m.abs() + ro.TINY
    own = ro.U * (x64.abs() + m.abs())
    dv = ro.ROW * (c * c).mean(1, keepdim=True) + dm ** 2 + (2 * c.abs() * own).mean(1, keepdim=True)
    dr = r * (0.5 * dv * r * r + 6 * ro.U)
    lim = g64.abs() * ((dm + own + ro.TINY) * r + c.abs() * dr + 2 * ro.U * (c * r).abs()) \
        + 3 * ro.U * ((g64 * c * r).abs() + b64.abs()) + 4 * ro.TINY
    inside(mean[:, None], m, dm, torch.float32, "mean")
    inside(rstd[:, None], r, dr, torch.float32, "rstd")
    inside(y, ref, lim, dtype, "y")
    s = ref.abs().mean(1)
    inside(scale, s, lim.mean(1) + (ro.ROW + 4 * ro.U) * s, torch.float32, "scale")
    at = torch.arange(cols, device="cuda")
    on = (bits[:, at // 64] >> (at % 64)) & 1
    sure = ref.abs() > lim
    assert bool(((on == 1) == (ref >= 0))[sure].all())


def test_the_current_stream_is_the_calls():
    """Without a stream a call is on the current one: in order with what is enqueued there."""
    import paper_2010_07565_amd._lib as lib
    side = torch.cuda.Stream()
    assert lib._stream(None) == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(side):
        assert lib._stream(None) == side.cuda_stream == torch.cuda.current_stream().cuda_stream
    x = torch.empty(300001, 256, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for k in range(3):
            x.normal_()
            bg.bigcn_layernorm(x, eps=ro.EPS, y=y)
        z.copy_(y)
    side.synchronize()
    bg.bigcn_layernorm(x, eps=ro.EPS, y=y)
    assert torch.equal(y, z)
