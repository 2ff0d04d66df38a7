"""What counts as a change of the position bias between a training call's forward and backward pass (a fake CUDA runtime, no
GPU)."""
import pytest

from test_host_train import BF16, FP32, INVALID, UNSUPPORTED, Layer, lib  # noqa: F401  (lib: the fixture)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_calls_that_change_no_position_bias_leave_the_pass(lib, dtype):  # noqa: F811
    lay = Layer(lib, dtype)
    detach = lambda: lay.is_(lib.eigen_attn_bias_attach(lay.h, 0, 0, None, 0, None), None)
    lay.train_attach()
    lay.forward()
    lay.is_(lay.alibi(None), None)                           # none to none
    lay.backward()
    lay.is_(lay.alibi([0.0, 0.0]), None)
    lay.backward()
    detach()                                                 # none there
    lay.backward()
    for bad in ([0.5, -1.0], [float("nan"), 0.5], [0.5, float("inf")]):
        lay.is_(lay.alibi(bad), INVALID)                     # refused
        lay.backward()
    lay.is_(lay.alibi([0.5, 0.25]), None)
    lay.backward(want=INVALID)
    lay.forward()
    lay.is_(lay.alibi([0.25, -1.0]), INVALID)
    lay.backward()
    lay.bias_attach(want=INVALID)                            # the layer has an ALiBi bias
    lay.backward()
    lay.is_(lay.alibi(None), None)
    lay.backward(want=INVALID)
    lay.bias_attach()
    lay.forward()
    lay.is_(lay.alibi([0.5, 0.25]), INVALID)
    lay.is_(lay.alibi(None), None)
    lay.is_(lib.eigen_attn_bias_set(lay.h, None, None), INVALID)
    lay.backward()
    lay.backward(table=True)
    detach()
    lay.backward(want=INVALID)


def test_a_refused_slope_leaves_the_bias_that_was_there(lib):  # noqa: F811
    lay = Layer(lib)
    lay.train_attach(group=2)
    lay.is_(lay.alibi([0.5, 0.25]), None)
    before = lay.ws.copy()
    lay.is_(lay.alibi([0.125, -1.0]), INVALID)
    lay.forward(group=2, want=UNSUPPORTED)                   # still there
    assert (lay.ws == before).all()
    lay.is_(lay.alibi(None), None)
    lay.forward(group=2)
