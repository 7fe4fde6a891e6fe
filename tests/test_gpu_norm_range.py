"""Layer norm at the ends of its types' range: finite rows whose sums or squares pass it,
and the signs of what is no number."""
import numpy as np
import pytest
import torch

import paper_2010_07565_amd as bg
import rowops as ro

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    bg.load()


def every_output(x, gamma=None, beta=None, eps=ro.EPS):
    rows, cols = x.shape
    q = bg.checkpoint_groups(cols)
    o = dict(y=torch.full_like(x, float("nan")), mean=torch.empty(rows, device="cuda"),
             rstd=torch.empty(rows, device="cuda"),
             codes=torch.empty(rows, cols, dtype=torch.int8, device="cuda"),
             qscale=torch.empty(rows, q, device="cuda"),
             bits=torch.empty(rows, q, dtype=torch.int64, device="cuda"),
             scale=torch.empty(rows, device="cuda"))
    bg.bigcn_layernorm(x, gamma, beta, eps=eps, **o)
    return o


def wide_rows(rng, cols, dtype):
    """Finite rows of every size from 1 to the type's largest value, among them."""
    top = float(torch.finfo(dtype).max)
    v = rng.standard_normal((40, cols)) / 5
    v = np.clip(v, -1, 1)
    k = np.arange(cols)
    rows = [v[i] * s for i, s in enumerate((1, 1e15, 1e17, 1e18, 1e19, 3e19, 1e25, 1e30, 1e37, top))]
    rows += [np.where(k == cols // 2, top, 0), np.where(k == 0, -top, v[11]),   # one large element
             np.full(cols, 2.0 ** 127), np.full(cols, -2.0 ** 100), np.full(cols, 3 * 2.0 ** 120),  # constant
             np.where(k % 2 == 0, top, -top),
             np.where(k == cols - 1, top, -top), np.where(k == 0, -top, top),   # x - mean passes top
             np.where(k < cols // 2, top, top * 0.5),                           # the sum passes top
             1e38 + 1e36 * v[19], v[20], -2e38 + 1e30 * v[21], np.linspace(-1, 1, cols) * top]
    return torch.from_numpy(np.array(rows)).to(dtype)


@pytest.mark.parametrize("cols", [1, 2, 3, 5, 64, 100, 300, 400, 602, 1433, 2049, 5000, 8192])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_finite_rows(cols, dtype):
    rng = np.random.default_rng(cols)
    x = wide_rows(rng, cols, dtype)
    assert bool(torch.isfinite(x).all())
    g = torch.from_numpy(rng.uniform(-1.5, 1.5, cols).astype(np.float32))
    b = torch.from_numpy(rng.uniform(-0.5, 0.5, cols).astype(np.float32))
    got = every_output(x.cuda(), g.cuda(), b.cuda())
    x64 = ro.f64(x)
    ref = ro.norm(x64, ro.f64(g), ro.f64(b))
    ro.within(ro.f64(got["mean"]), ref["mean"], ref["dmean"], "mean")
    # (1 / deviation is subnormal where the deviation is above 2^126)
    ro.within(ro.f64(got["rstd"]), ref["rstd"], ref["drstd"] + ro.TINY, "rstd")
    ro.within(ro.f64(got["y"]), ref["y"], ref["dy"] + ro.store_bound(np.abs(ref["y"]) + ref["dy"], dtype), "y")
    s = np.abs(ref["y"]).mean(1)
    ro.within(ro.f64(got["scale"]), s, ref["dy"].mean(1) + (ro.ROW + 4 * ro.U) * s, "scale")
    have = np.unpackbits(got["bits"].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :cols] == 1
    sure = np.abs(ref["y"]) > ref["dy"]
    assert np.array_equal(have[sure], (ref["y"] >= 0)[sure])
    for i in (12, 13, 14):      # a constant row is its mean
        assert torch.equal(got["y"][i].cpu(), b.to(dtype)) and float(got["mean"][i]) == float(x[i, 0])
    # rows beside such ones are what they are alone
    alone = every_output(x[[0, 20]].cuda(), g.cuda(), b.cuda())
    for k in got:
        assert torch.equal(got[k][[0, 20]], alone[k]), k
    over = x.cuda()
    bg.bigcn_layernorm(over, g.cuda(), b.cuda(), eps=ro.EPS, y=over)
    assert torch.equal(over, got["y"])


@pytest.mark.parametrize("eps", [1.2e-38, 1e30, 3.4e38])
def test_eps_at_the_ends_of_its_range(eps):
    rng = np.random.default_rng(6)
    x = wide_rows(rng, 100, torch.float32)
    got = every_output(x.cuda(), eps=eps)
    ref = ro.norm(ro.f64(x), np.ones(100), np.zeros(100), eps)
    ro.within(ro.f64(got["rstd"]), ref["rstd"], ref["drstd"] + ro.TINY, "rstd")
    # (a deviation within the rounding of the mean is all that a constant row has)
    ro.within(ro.f64(got["y"]), ref["y"], ref["dy"] + ro.store_bound(np.abs(ref["y"]), torch.float32), "y")


@pytest.mark.parametrize("cols", [2, 64, 300, 1433, 2049])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("source", ["x", "q8"])
def test_gradients_of_finite_rows(cols, dtype, source):
    rng = np.random.default_rng(cols)
    x = wide_rows(rng, cols, dtype).cuda()
    if source == "q8":
        # rows whose spread is below their checkpoint's steps: of the restored row (x - mean)
        # rstd and the gradient by the formula pass fp32's range
        f = every_output(x)
        far = np.abs(ro.values(f["codes"].cpu().numpy(), f["qscale"].cpu().numpy())).max(1) \
            * ro.f64(f["rstd"])
        assert (far < 1e30).sum() >= 15
        x = x[torch.from_numpy(far < 1e30).cuda()]
    rows = x.shape[0]
    g = torch.from_numpy(rng.uniform(-1.5, 1.5, cols).astype(np.float32)).cuda()
    dy = torch.from_numpy(rng.standard_normal((rows, cols))).to(dtype).cuda()
    f = every_output(x)
    dx, dg, db = torch.empty_like(dy), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(bg.layernorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    kept = dict(x=x) if source == "x" else dict(codes=f["codes"], qscale=f["qscale"])
    bg.bigcn_layernorm_backward(dy, f["mean"], f["rstd"], gamma=g, dx=dx, dgamma=dg, dbeta=db,
                                workspace=ws, **kept)
    x64 = ro.f64(x) if source == "x" else ro.values(f["codes"].cpu().numpy(), f["qscale"].cpu().numpy())
    ref = ro.norm_grad(ro.f64(dy), x64, ro.f64(f["mean"]), ro.f64(f["rstd"]), ro.f64(g))
    ro.within(ro.f64(dx), ref["dx"], ref["ddx"] + ro.store_bound(np.abs(ref["dx"]) + ref["ddx"], dtype), "dx")
    ro.within(ro.f64(dg), ref["dgamma"], ref["ddgamma"], "dgamma")
    ro.within(ro.f64(db), ref["dbeta"], ref["ddbeta"], "dbeta")


@pytest.mark.parametrize("cols", [1, 3, 64, 100, 300, 602, 1433, 2049, 5000])
def test_bits_of_what_is_no_number(cols):
    """The packed signs are those of the pack of the fp32 y, which sets no bit for a NaN and
    sets the bit of -0."""
    rng = np.random.default_rng(cols)
    x = torch.from_numpy(rng.standard_normal((24, cols)).astype(np.float32)).cuda()
    nan = np.array([0x7FC00000, 0xFFC00000], np.uint32).view(np.float32)     # of either sign
    x[3, 0], x[4, cols - 1] = float(nan[0]), float("inf")
    x[5].view(torch.int32)[cols // 2] = -0x400000
    x[6] = float("-inf")
    assert int(torch.isnan(x).sum()) == 2
    gamma = torch.from_numpy(rng.uniform(-1.5, 1.5, cols).astype(np.float32)).cuda()
    beta = torch.from_numpy(rng.uniform(-0.5, 0.5, cols).astype(np.float32)).cuda()
    gamma[cols // 3], beta[cols // 3] = 0.0, -0.0
    for bad in (False, True):
        if bad:
            gamma[cols // 2] = float("nan")
        got = every_output(x, gamma, beta)
        bits, scale = torch.empty_like(got["bits"]), torch.empty_like(got["scale"])
        bg.bigcn_binarize_pack(got["y"], bits, scale)
        assert torch.equal(bits, got["bits"])
        assert int(got["bits"][3:7].abs().sum()) == 0
        assert torch.equal(torch.isnan(scale), torch.isnan(got["scale"]))
