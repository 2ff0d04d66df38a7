"""Uses of the training calls that lie between their parts: scratch of another size than the pass, buffers replaced under work
that is still to run, waits that run out.  (Guard regions lie around every buffer, see conftest.py.)"""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_train import BF, F32
from test_gpu_train_use import Step, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("attached", [2, 16])
def test_scratch_for_more_query_heads_than_the_pass_has(dtype, attached):
    """The table's gradient of a pass with one query head per K/V head, in scratch for several: the same bits."""
    a, b = (Step(2, 300, [32, 40], [40, 32], 64, dtype, bias=True, seed=4, lens=[300, 129]) for _ in range(2))
    b.lay.train_attach(300, attached)
    assert same(a.run(), b.run())
    b.lay.poll_status()
