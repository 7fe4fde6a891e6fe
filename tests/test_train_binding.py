"""The training operators' workspace sizes at their largest, and the binding's checks.
No GPU is needed."""
import paper_2010_07565_amd as bg


def test_workspace_of_the_norm_gradients():
    """Up to 1536 columns no more than 8 KB a column, however many rows there are; wider
    rows leave a set of sums every 64 of them, and no more than one a row."""
    most = (1 << 31) - 1
    for cols in (1, 3, 64, 256, 602, 1433, 1536):
        sizes = [bg.layernorm_backward_workspace_bytes(rows, cols) for rows in
                 (1, 1000, 20000, 1000000, 20000000, most)]
        assert all(0 < s <= 8192 * cols + 256 for s in sizes), (cols, sizes)
        assert sizes == sorted(sizes)
    for cols in (1537, 2048, 4096, 8192):
        for rows in (1, 100, 1000, 20000, 1000000, most):
            sets = min(rows, rows // 64 + 1536)
            assert 0 < bg.layernorm_backward_workspace_bytes(rows, cols) <= sets * 2 * cols * 4 + 256
    assert bg.layernorm_backward_workspace_bytes(0, 64) == 0
    assert bg.layernorm_backward_workspace_bytes(most + 1, 8192) == 0    # (refused)
