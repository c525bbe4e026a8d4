"""What the host code of the operators around the recurrence asks of the CUDA runtime, seen through the stand-in of test_host_launches.py: the
shapes of its launches, and that a device which places no clusters gets launches without any."""
import pytest

from test_host_launches import calls, host_library, pytestmark  # noqa: F401  (fixture)

BIG = [1 << 40]
LL = lambda n: {"ll": n}  # noqa: E731


def gated(rows, K1, K2, F, x2=True, w2=True, act=0):
    return ["gf_gated_linear", ["p", "p", "p" if x2 else None, "p" if w2 else None, act, "p", LL(rows), K1, K2, F, None]]


def gated_grad(rows, K1, K2, F, x2=True, w2=True, act=0):
    return ["gf_gated_linear_backward", ["p", "p", "p" if x2 else None, "p" if w2 else None, act, "p", "p", "p", "p" if x2 else None, "p" if w2 else None,
                                         LL(rows), K1, K2, F, "ws", BIG, None]]


def loss(rows, D, V):
    return ["gf_vocab_loss", ["p"] * 5 + [LL(rows), D, LL(V), "ws", BIG, None]]


def loss_grad(rows, D, V):
    return ["gf_vocab_loss_backward", ["p"] * 7 + [LL(rows), D, LL(V), "ws", BIG, None]]


GOES, NONE = [0, 0], [9, 0]          # clusters are placed, or refused (invalid configuration)


def test_gated_linear_launches(host_library):  # noqa: F811
    decode, train, few = gated(4, 2048, 7168, 2048), gated(16384, 2048, 7168, 2048), gated(333, 768, 768, 2688, x2=False)
    got = calls(host_library, decode + [GOES], train + [GOES], few + [GOES], decode + [NONE], train + [NONE])
    assert all(s == 0 for s, _ in got)
    logs = [log for _, log in got]
    assert logs[0][0].startswith("grid 96 cluster 6 ") and "ModeE2" in logs[0][0] and len(logs[0]) == 1      # a cluster per 128 columns
    assert logs[1][0].startswith("grid 148 cluster 2 ") and "ModeE1" in logs[1][0] and len(logs[1]) == 1     # whole accumulators
    assert logs[2][0].startswith("grid 126 cluster 1 ") and len(logs[2]) == 1
    for log, grid in ((logs[3], 32), (logs[4], 148)):
        assert len(log) == 2 and "refused" in log[0] and log[1].startswith(f"grid {grid} cluster 1 ") and "ModeE0" in log[1]


@pytest.mark.parametrize("refused", [GOES, NONE])
def test_gradients_launches(host_library, refused):  # noqa: F811
    todo = [gated_grad(8192, 2048, 2048, 7168, x2=False), gated_grad(2500, 520, 1000, 4008), loss(8192, 2048, 65536), loss_grad(8192, 2048, 65536), loss_grad(7, 768, 40011)]
    for s, log in calls(host_library, *[c + [refused] for c in todo]):
        assert s == 0
        went = [line for line in log if "refused" not in line]
        if refused == NONE:
            assert all(" cluster 1 " in line for line in went)
        else:
            assert went == log
        kernels = [line.split()[-1] for line in went]
        assert all("pair_gemm" in k or "sum_slices" in k or "join" in k for k in kernels)
    # the vocabulary in four pieces of 16384: logits again, then both products; fp32 sums are added up once, behind the last
    s, log = calls(host_library, todo[3] + [GOES])[0]
    assert sum("EpilogueE4" in line for line in log) == 4 and sum("EpilogueE0" in line for line in log) == 4 and sum("sum_slices" in line for line in log) <= 1


def test_calls_of_nothing_clear_what_they_owe(host_library):  # noqa: F811
    got = calls(host_library, gated(0, 64, 72, 136) + [GOES], gated_grad(0, 64, 72, 136) + [GOES], loss(0, 64, 100) + [GOES], loss_grad(0, 64, 100) + [GOES])
    assert [s for s, _ in got] == [0] * 4
    assert got[0][1] == [] and got[2][1] == []
    assert sorted(int(line.split()[3]) for line in got[1][1]) == [0, 0, 64 * 136 * 2, 72 * 136 * 2]
    assert [int(line.split()[3]) for line in got[3][1]] == [100 * 64 * 2]
