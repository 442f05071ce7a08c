"""Widths of adapters that the kernels' 32-bit arithmetic does not hold are refused.  No GPU."""
import pytest

from paper_1904_04956_amd import binding as bl


@pytest.mark.parametrize("change", [dict(K=2 ** 31 - 1), dict(N=2 ** 31 - 1), dict(K=2 ** 31 - 20), dict(N=2 ** 31 - 20), dict(K=2 ** 30), dict(N=2 ** 30), dict(K=2 ** 31 - 1, N=2 ** 31 - 1)])
@pytest.mark.parametrize("mode", [0, 1])
def test_widths_near_the_largest_int_are_refused(change, mode):
    cfg = bl.adapter_config(*{**dict(T=1, B=1, K=8, N=8, rank=1, count=1, mode=mode, scale=1.0), **change}.values())
    P = 4096
    for call in (lambda: bl.adapter_scratch_bytes(cfg, bl.ADAPTER_FORWARD), lambda: bl.adapter_scratch_bytes(cfg, bl.ADAPTER_BACKWARD),
                 lambda: bl.adapter_forward(cfg, P, P, P, P, P, P, P, P, P, 1 << 62, 0), lambda: bl.adapter_backward(cfg, P, P, P, P, P, P, P, P, P, P, P, P, P, 1 << 62, 0)):
        with pytest.raises(bl.BlstmError) as e:
            call()
        assert e.value.code == -2
