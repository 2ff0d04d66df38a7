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


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("how", ["replaced", "detached"])
def test_scratch_that_is_replaced_while_another_stream_has_a_pass_to_run(dtype, how, monkeypatch):
    """Its memory is not handed out before that pass is over."""
    from paper_2408_05646_b200 import binding
    monkeypatch.setattr(binding, "device_alloc", binding._default_alloc)     # (the guards' keeps every buffer alive)
    want = Step(2, 300, [32, 40], [40, 32], 64, dtype, seed=8).run()
    a = Step(2, 300, [32, 40], [40, 32], 64, dtype, seed=8, attach=8000)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(400_000_000)                       # some 0.2 s in front of the passes
    got = a.run(stream=s)
    at, n = a.lay.train_buf.data_ptr(), a.lay.train_buf.numel()
    if how == "replaced":
        a.lay.train_attach(16)
    else:
        a.lay.train_detach()
    others = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    assert not s.query()                                     # it has not begun
    assert all(x.data_ptr() + n <= at or at + n <= x.data_ptr() for x in others)
    for x in others:
        x.fill_(0xff)
    s.synchronize()
    assert same(got, want)
    a.lay.poll_status()


@pytest.mark.parametrize("group,bias", [(1, True), (4, False)])
@pytest.mark.parametrize("r", [40, 112])
@pytest.mark.parametrize("call", ["forward", "backward", "both"])
def test_a_wait_that_runs_out_is_reported_once_and_the_layer_recovers(call, r, group, bias):
    """One softmax warp reports its first wait as run out (the library's own hook): every other wait of its CTA then gives up, with
    products and copies of other warps under way.  The launch ends, the timeout is reported once, and the next step is right."""
    from paper_2408_05646_b200 import binding
    s = Step(4, 1200, [r] * 4, [r] * 4, 128, BF, group, bias, seed=6, lens=[1200, 700, 1, 1199])
    want = s.run()
    s.lay.poll_status()
    for _ in range(3):
        if call != "backward":
            s.lay.set_option(binding.EA_OPT_TEST_WAIT_GIVES_UP, 1)
        s.lay.train_forward(*s.x[:3], lens=s.lens, group=group)
        if call != "forward":
            s.lay.set_option(binding.EA_OPT_TEST_WAIT_GIVES_UP, 1)
            s.lay.train_backward(s.x[3], bias_grad=bias)
        with pytest.raises(binding.EigenAttnError) as e:
            s.lay.poll_status()
        assert e.value.status == binding.EA_ERR_TIMEOUT
        s.lay.poll_status()
        assert same(s.run(), want)                           # the hook was armed for one launch
        s.lay.poll_status()
