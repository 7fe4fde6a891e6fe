"""Outputs of the packed layer backward that lie over an input: dzeta over the packed signs."""
import numpy as np
import pytest
import torch

import workloads
import paper_2010_07565_amd as bg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", ["sym", "mean"])
@pytest.mark.parametrize("d_in,d_out", [(130, 4), (500, 7)])
def test_dzeta_over_the_signs(norm, d_in, d_out):
    """The signs are read before dzeta is written: every gradient as with dzeta beside them."""
    dev = torch.device("cuda:0")
    bg.load()
    rng = np.random.default_rng(d_in)
    g = workloads.random_small_graph(700, 3000, rng, isolated=3)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
    rowptr, colidx = t(g.rowptr), t(g.colidx)
    wt = t(rng.standard_normal((d_out, d_in)).astype(np.float32))
    wbits, alpha = bg.pack_weights(wt)
    gout = t(rng.standard_normal((g.n, d_out)).astype(np.float32))
    words = bg.words(d_in)
    res = []
    for over in (False, True):
        # 32-bit words of the rows of signs, a row of dzeta in the first of each row's
        flat = torch.empty(g.n, 2 * words + 2, dtype=torch.float32, device=dev)
        hbits = flat.view(torch.int64)[:, :words]
        hscale = torch.empty(g.n, device=dev)
        bg.bigcn_binarize_pack(t(np.random.default_rng(3).standard_normal((g.n, d_in)).astype(np.float32)),
                               hbits, hscale, rowptr=rowptr, norm=norm)
        dzeta = flat[:, :d_out] if over else torch.empty(g.n, d_out, device=dev)
        r = dict(dwt=torch.empty_like(wt), dwt_tilde=torch.empty_like(wt),
                 dh=torch.empty(g.n, d_in, device=dev), db=torch.empty(d_out, device=dev))
        ws = torch.empty(bg.layer_backward_workspace_bytes(g.n, g.nnz, d_in, d_out), dtype=torch.uint8,
                         device=dev)
        bg.bigcn_layer_backward_packed(rowptr, colidx, hbits, hscale, wt, wbits, alpha, gout, r["dwt"],
                                       ws, norm=norm, dh=r["dh"], dwt_tilde=r["dwt_tilde"], db=r["db"],
                                       dzeta=dzeta)
        torch.cuda.synchronize()
        res.append(dict(r, dzeta=dzeta.clone()))
    for k in res[0]:
        assert torch.equal(res[0][k], res[1][k]), k
