"""qm_linear_fp8's kernel for many rows where waits run out: NaN in what it could not compute, other outputs as ever."""
import pytest
import torch

import paper_2408_02897_b200 as qm
from test_gpu_linear_fp8 import codes

pytestmark = pytest.mark.gpu


@pytest.fixture
def starved_producer():
    L = qm.lib()
    L.qm_debug_set_wait_limit_ns(2_000_000)                            # 2 ms instead of 1 s
    yield L
    L.qm_debug_stop_producer_after(0xffffffff)
    L.qm_debug_set_wait_limit_ns(0)


# (on 148 SMs) a tile of 16 k-blocks for each of 64 pairs; 160 tiles of nine for 74
@pytest.mark.parametrize("M,N,K", [(2048, 2048, 2048), (2560, 4096, 1152)])
@pytest.mark.parametrize("side", [128, 1])
@pytest.mark.parametrize("stop", [0, 1, 2, 6, 13])
def test_pairs_that_give_up(starved_producer, M, N, K, side, stop):
    """Many calls that give up one after the other, on two streams: each returns, and a full one behind them is right."""
    _, _, x, dx = codes(M, K, "e4m3", 12, 1, 0.01)
    _, _, w, dw = codes(N, K, "e4m3", 13, side, 0.01)

    def call(stream=None):
        return qm.qm_linear_fp8(x, dx, w, dw, K, side_w=side, stream=stream)
    sound = call()
    torch.cuda.synchronize()
    starved_producer.qm_debug_stop_producer_after(stop)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [call(streams[i % 2]) for i in range(6)]
    torch.cuda.synchronize()
    for y in got:
        bad = y.isnan()
        assert torch.equal(y[~bad], sound[~bad]) and bad.any()
        if stop < -(-K // 128):
            assert bad.all()                                           # no tile is complete
    starved_producer.qm_debug_stop_producer_after(0xffffffff)
    assert torch.equal(call(), sound)
