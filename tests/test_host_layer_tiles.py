"""That the shapes of test_gpu_layers_many_tiles.py are launched as that file needs them, seen through the stand-in of test_host_launches.py."""
import pytest

import test_gpu_layers_many_tiles as shapes
from test_host_launches import calls, host_library, pytestmark  # noqa: F401  (fixture)
from test_host_layers import GOES, gated, gated_grad, loss_grad


def ceil(a, b):
    return -(-a // b)


@pytest.mark.parametrize("rows,K1,K2,F", shapes.WIDE)
def test_wide_tiles(host_library, rows, K1, K2, F):  # noqa: F811
    (s, fwd), (s2, bwd) = calls(host_library, gated(rows, K1, K2, F) + [GOES], gated_grad(rows, K1, K2, F) + [GOES])
    assert s == s2 == 0
    for line in (fwd[0], bwd[0]):
        assert line.startswith("grid 148 cluster 2 ") and "ModeE1" in line
    assert ceil(rows, 256) * ceil(F, 256) > 74


@pytest.mark.parametrize("rows,K1,K2,F", shapes.FEW_GATE)
def test_gates_of_few_rows(host_library, rows, K1, K2, F):  # noqa: F811
    (s, log), = calls(host_library, gated_grad(rows, K1, K1 if K2 == 0 else max(K2, 0), F, x2=K2 > 0, w2=K2 >= 0) + [GOES])
    assert s == 0 and log[0].startswith("grid 148 cluster 1 ") and "EpilogueE5" in log[0]
    assert ceil(F, 128 if K2 < 0 else 64) > 148


@pytest.mark.parametrize("rows,D,V", shapes.FEW_LOSS)
def test_losses_of_few_rows(host_library, rows, D, V):  # noqa: F811
    (s, log), = calls(host_library, loss_grad(rows, D, V) + [GOES])
    assert s == 0 and log[0].startswith("grid 148 cluster 1 ") and "EpilogueE6" in log[0]
    assert ceil(V, 128) > 148


def test_pieces_whose_sum_is_not_cut(host_library):  # noqa: F811
    (s, log), = calls(host_library, loss_grad(16384, 1024, 8200) + [GOES])
    assert s == 0 and [("EpilogueE4" in line, "EpilogueE0" in line) for line in log] == [(True, False), (False, True)] * 2


@pytest.mark.parametrize("dtype,H,N", shapes.NORM)
def test_norm_gradients_stages(dtype, H, N):
    """A stage holds at most 64 KB of both tensors for all CTAs of an SM, so these rows fill five of them for each of 148 SMs."""
    row = H * N * (2 if dtype == shapes.BF else 4)
    rows = shapes.norm_rows(dtype, H, N)
    assert rows % 2 == 1 and rows * 2 * row > 5 * 148 * 65536
