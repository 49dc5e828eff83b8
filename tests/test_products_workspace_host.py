"""The workspace of the products by element (no GPU): a program that asks once, for its largest batch, may use it for every smaller one."""
import pytest

gp = pytest.importorskip("paper_2504_10700_amd.gp_binding")


@pytest.mark.parametrize("shape", [(89, 128, 128, 64, 0), (1024, 1, 1, 1, 0), (3, 2048, 1024, 7, 2), (8, 64, 64, 3, 1), (8, 512, 700, 1, 0), (2, 300, 200, 1, 2), (5, 128, 384, 5, 1)], ids=str)
def test_the_workspace_of_a_larger_batch_serves(shape):
    elements, k_in, k_out, components, dtype = shape
    cfg = gp.make_config(elements, k_in, k_out, components, dtype)
    bytes_of = [gp.gp_workspace_bytes(cfg, n) for n in list(range(6000)) + [10_000, 100_000, 1_000_000]]
    assert bytes_of[0] >= 256
    most = 0
    for n, b in enumerate(bytes_of):
        if n > gp.GP_UNGROUPED:
            assert b >= most, n
        most = max(most, b)
