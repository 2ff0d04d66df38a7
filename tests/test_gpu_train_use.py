"""Training calls as they are used: many items per block, captured and replayed, on other streams, again and again, next to
decode; gradients against differences; a few steps of descent."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import training as oracle
from test_gpu_train import BF, F32, close, layer, rows, run_case

pytestmark = pytest.mark.gpu
BUCKETS = (16, 64)


class Step:
    """A layer with inputs of its own: forward and backward pass, with a learned bias where `bias` is set."""

    def __init__(self, B, T, r_k, r_v, d_head, dtype, group=1, bias=False, seed=0, lens=None, attach=None):
        gen = torch.Generator().manual_seed(seed)
        self.lay, self.group, self.bias = layer(B, r_k, r_v, d_head, dtype), group, bias
        self.x = [rows(gen, B, T, r_k, group, dtype, 1.5, 0.0).cuda(), rows(gen, B, T, r_k, 1, dtype, 1.0, 0.0).cuda(),
                  rows(gen, B, T, r_v, 1, dtype, 1.0, 0.0).cuda(), rows(gen, B, T, r_v, group, dtype, 1.0, 0.0).cuda()]
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
        if bias:
            self.lay.bias_attach(*BUCKETS)
            self.table = torch.randn(len(r_k), BUCKETS[0], generator=gen).to(dtype).cuda()
            self.lay.set_bias(self.table)
        self.lay.train_attach(attach or T, group)

    def run(self, stream=None):
        q, k, v, g = self.x
        out = self.lay.train_forward(q, k, v, lens=self.lens, group=self.group, stream=stream)
        return (out,) + tuple(self.lay.train_backward(g, bias_grad=self.bias, stream=stream))


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,T,H,group,lens", [(4, 700, 8, 1, [700, 0, 333, 1]), (2, 500, 3, 8, [500, 129]), (1, 1500, 12, 1, None)])
def test_many_items_for_every_block(dtype, B, T, H, group, lens):
    run_case(B, T, [24] * H, [16] * H, 32, dtype, group=group, lens=lens, seed=T)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_widest_heads_over_many_tiles(dtype):
    run_case(1, 1100, [128, 128], [128, 128], 128, dtype, lens=[1090])


def test_tiles_of_very_different_sizes():
    """Blocks of 128 tokens scaled by powers of two, one of them zero: each has a scale of its own.  Errors are relative to the
    terms (close) down to where fp16 runs out of range; its smallest half step is 2^-25.  P enters the forward products times
    2^7 and, by the tile's deviation from the largest v', up to 2 max|v'| / |v'_j| less: 2^-31 max|v'| for every key.  dv': P
    times 2^14, in the same way 2^-38 max|do'| for every query.  dS is scaled so that 2^24 2^(-e-e') becomes 2^15, and the
    smallest exponents have 2^-e <= 2^-7 max|do'|, 2^-e' <= 2^-7 max|v'|: a half step is 2^-16 2^-14 max|do'| max|v'|, and with
    the tile's deviation dq' is off by 2^-29 max|do'| max|v'| max|k'| scale for every key, dk' by the same with q'."""
    T, r = 640, [32, 48]
    gen = torch.Generator().manual_seed(1)
    x = [rows(gen, 2, T, r, 1, BF, 1.0, 0.0) for _ in range(4)]
    for a, powers in zip(x, ((0, 0, 2, -3, 0), (0, 2, -9, 0, 1), (0, -8, 6, None, 0), (-7, 0, 8, None, -2))):
        for t, e in enumerate(powers):
            a[:, 128 * t:128 * t + 128] *= 0.0 if e is None else 2.0 ** e
    lay = layer(2, r, r, 64, BF)
    lay.train_attach(T)
    out = lay.train_forward(*[a.cuda() for a in x[:3]])
    got = (out,) + tuple(lay.train_backward(x[3].cuda()))
    want = oracle.train(*[a.double().numpy() for a in x], r, r, 64)
    mq, mk, mv, mg = (a.abs().max().item() for a in x)
    floor = {"out": 2.0 ** -31 * mv, "dv": 2.0 ** -38 * mg, "dq": 2.0 ** -29 / 8 * mg * mv * mk, "dk": 2.0 ** -29 / 8 * mg * mv * mq}
    for name, y in zip(("out", "dq", "dk", "dv"), got):
        over = np.abs(y.double().cpu().numpy() - want[name]) - 2.0 ** -8 * np.abs(want[name]) - 2.0 ** -11 * want[name + "_size"]
        assert over.max() <= T * floor[name], (name, over.max(), T * floor[name])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_sequence_that_is_not_finite_stays_alone(dtype, bad):
    a, b = (Step(3, 200, [32, 24], [24, 32], 64, dtype, seed=2) for _ in range(2))
    for i in range(4):
        b.x[i][1, 150:160] = bad
    for x, y in zip(a.run(), b.run()):
        assert torch.equal(x[0], y[0]) and torch.equal(x[2], y[2])
        assert torch.isfinite(x.float()).all() and not torch.isfinite(y[1].float()).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("group,bias", [(1, True), (4, False)])
def test_the_same_bits_every_time(dtype, group, bias):
    s = Step(4, 600, [40] * 6, [32] * 6, 64, dtype, group, bias, lens=[600, 70, 350, 599])
    first = s.run()
    for _ in range(4):
        assert same(first, s.run())
    other = Step(4, 600, [40] * 6, [32] * 6, 64, dtype, group, bias, lens=[600, 70, 350, 599], attach=2000)
    assert same(first, other.run())                          # a larger scratch


@pytest.mark.parametrize("dtype", [BF, F32])
def test_back_again_with_another_gradient(dtype):
    a, b = (Step(2, 300, [32, 40], [40, 32], 64, dtype, bias=True, seed=5) for _ in range(2))
    first = a.run()
    b.lay.train_forward(*b.x[:3])
    b.lay.train_backward(torch.randn_like(b.x[3].float()).to(dtype), bias_grad=True)
    assert same(first[1:], b.lay.train_backward(b.x[3], bias_grad=True))
    double = a.lay.train_backward(2 * a.x[3], bias_grad=True)            # linear, and exactly so in a power of two
    for x, y in zip(first[1:], double):
        assert torch.equal(2 * x, y)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("group,bias", [(1, True), (4, False)])
def test_captured_and_replayed(dtype, group, bias):
    """A captured step follows the tensors' contents, the lengths among them, with uncaptured steps of other sizes between."""
    args = (3, 333, [32, 24], [24, 40], 64, dtype, group, bias)
    s, ref = Step(*args, seed=1, lens=[333, 100, 0]), Step(*args, seed=1, lens=[333, 100, 0])
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = s.run(stream=torch.cuda.current_stream())
    gen = torch.Generator().manual_seed(9)
    for lens in ([333, 100, 0], [1, 333, 257], [0, 0, 0], [64, 65, 128]):
        for x, y in zip(s.x, ref.x):
            new = torch.randn(x.shape, generator=gen).to(dtype).cuda()
            x.copy_(new)
            y.copy_(new)
        s.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        ref.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        for x in captured:
            x.fill_(float("nan"))
        graph.replay()
        want = ref.run()
        assert same(captured, want), lens
        small = [x[:, :50].contiguous() for x in s.x]        # an uncaptured step on the same scratch
        s.lay.train_forward(*small[:3], group=group)
        s.lay.train_backward(small[3])
    s.lay.poll_status()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_whole_captured_step_with_its_table(dtype):
    """bias_set, both passes and the table's update in one graph: every replay is an uncaptured step."""
    s, ref = (Step(2, 150, [32, 24], [24, 40], 64, dtype, bias=True, seed=3) for _ in range(2))

    def step(s, stream=None):
        s.lay.set_bias(s.table, stream=stream)
        got = s.run(stream=stream)
        s.table.sub_(got[4], alpha=0.5)
        return got

    step(s)
    step(ref)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(s, torch.cuda.current_stream())
    for _ in range(3):
        graph.replay()
        assert same(captured, step(ref)) and torch.equal(s.table, ref.table)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_long_text(dtype):
    """20000 tokens, two heads, the formulas in 64 bits on the device, 1000 queries at a time.  Tolerances as in close, with
    sqrt(20000 / 64) - sqrt(300 / 64) = 15 half steps more for the longer sums of fp32 layers."""
    T, r, d, chunk = 20000, [16, 24], 32, 1000
    s = Step(1, T, r, r, d, dtype, bias=True, seed=11)
    out, dq, dk, dv, dtable = s.run()
    s.lay.poll_status()
    starts = torch.tensor(s.lay.bias_starts(), device="cuda")
    half = torch.finfo(dtype).eps / 2
    cols, _ = oracle.packed_columns(r)
    at = torch.arange(T, device="cuda")
    by, by_size = torch.zeros(2, BUCKETS[0], dtype=torch.float64, device="cuda"), torch.zeros(2, BUCKETS[0], dtype=torch.float64, device="cuda")
    for h, c in enumerate(cols):
        c = torch.as_tensor(c, device="cuda")
        q, k, v, g = (x[0][:, c].double() for x in s.x)
        table = s.table[h].double()
        want = {n: torch.zeros_like(q) for n in ("out", "dq", "dk", "dv")}
        size = {n: torch.zeros_like(q) for n in want}
        for i in range(0, T, chunk):
            n = i + chunk
            dist = at[i:n, None] - at[None, :n]
            bucket = torch.bucketize(dist.clamp(min=0), starts, right=True) - 1
            S = q[i:n] @ k[:n].T / np.sqrt(d) + table[bucket]
            P = torch.softmax(S.masked_fill(dist < 0, float("-inf")), dim=1)
            o = P @ v[:n]
            delta = (o * g[i:n]).sum(1, keepdim=True)
            dS = P * (g[i:n] @ v[:n].T - delta)
            A = P * (g[i:n].abs() @ v[:n].abs().T + (o * g[i:n]).abs().sum(1, keepdim=True))
            want["out"][i:n], size["out"][i:n] = o, P @ v[:n].abs()
            want["dq"][i:n], size["dq"][i:n] = dS @ k[:n] / np.sqrt(d), A @ k[:n].abs() / np.sqrt(d)
            want["dk"][:n] += dS.T @ q[i:n] / np.sqrt(d)
            size["dk"][:n] += A.T @ q[i:n].abs() / np.sqrt(d)
            want["dv"][:n] += P.T @ g[i:n]
            size["dv"][:n] += P.T @ g[i:n].abs()
            by[h] += torch.bincount(bucket.flatten(), dS.flatten(), BUCKETS[0])
            by_size[h] += torch.bincount(bucket.flatten(), A.flatten(), BUCKETS[0])
        for name, x in zip(want, (out, dq, dk, dv)):
            over = (x[0][:, c].double() - want[name]).abs() - half * want[name].abs() - (2.0 ** -11 if dtype == BF else 60 * half) * size[name]
            assert over.max() <= 0, (h, name, over.max().item())
    over = (dtable.double() - by).abs() - half * by.abs() - (2.0 ** -12 if dtype == BF else 60 * half) * by_size
    assert over.max() <= 0


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_backward_pass_before_the_captured_forward_pass_has_run(dtype):
    """Its results are of no use, but it reads and writes nothing outside."""
    s = Step(2, 200, [32, 24], [24, 40], 64, dtype)
    s.lay.train_buf.fill_(0x7f)                              # lengths of 2^31 and so on
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = s.lay.train_forward(*s.x[:3], stream=torch.cuda.current_stream())
    s.lay.train_backward(s.x[3])
    torch.cuda.synchronize()
    s.lay.poll_status()
    graph.replay()
    got = (out,) + tuple(s.lay.train_backward(s.x[3]))
    assert same(got, Step(2, 200, [32, 24], [24, 40], 64, dtype).run())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_two_layers_on_two_streams(dtype):
    want = [Step(2, 400, [40] * 4, [40] * 4, 64, dtype, bias=True, seed=i).run() for i in range(2)]
    steps = [Step(2, 400, [40] * 4, [40] * 4, 64, dtype, bias=True, seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [s.run(stream=st) for s, st in zip(steps, streams)]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert same(a, b)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_tensors_off_the_16_byte_boundaries(dtype):
    """Inputs and outputs one element behind a boundary: the same bits, and nothing written beside them."""
    a, b = (Step(2, 150, [32, 20], [20, 32], 64, dtype, seed=3) for _ in range(2))

    def shifted(x, fill=0.0):
        buf = torch.full((x.numel() + 33,), fill, dtype=x.dtype, device=x.device)
        y = buf[1:1 + x.numel()].view(x.shape)
        y.copy_(x)
        return buf, y

    x = [shifted(t)[1] for t in b.x]
    want = a.run()
    outs = [shifted(t, 7.0) for t in want]
    for _, y in outs:
        y.fill_(float("nan"))
    b.lay.train_forward(*x[:3], out=outs[0][1])
    b.lay.train_backward(x[3], dq=outs[1][1], dk=outs[2][1], dv=outs[3][1])
    assert same(want, [y for _, y in outs])
    for buf, y in outs:
        assert buf[0] == 7.0 and (buf[1 + y.numel():] == 7.0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_training_leaves_the_cache_alone_and_agrees_with_decode(dtype):
    """The last row of the forward pass is what decode gives for the same query, rows and bias; and a decode between the two
    passes changes neither.  16-bit layers: two roundings and P at 2^-8 of the terms in decode, below four times 2^-8; fp32
    layers: 45 half steps (close) on either side."""
    B, T, r, d = 2, 150, [32, 24], 64
    s = Step(B, T, r, r, d, dtype, bias=True, seed=4)
    want = s.run()
    lay = layer(B, r, r, d, dtype, n_max=T)
    lay.bias_attach(*BUCKETS)
    lay.set_bias(s.table)
    lay.train_attach(T)
    lay.append_kv(s.x[1], s.x[2], preprojected=True)
    last = s.x[0][:, -1:].contiguous()

    def decode():
        return lay.decode(last, q_preprojected=True, out_lowrank=True).clone()

    before = decode()
    out = lay.train_forward(*s.x[:3])
    between = decode()
    got = (out,) + tuple(lay.train_backward(s.x[3], bias_grad=True))
    assert torch.equal(before, between) and torch.equal(before, decode()) and same(want, got)
    size = s.x[2].float().abs().amax(dim=1)                  # the terms are averages of these
    error = (out[:, -1].float() - before.float().view(B, -1)).abs()
    assert (error <= (2.0 ** -6 if dtype == BF else 2.0 ** -17) * size).all()


@pytest.mark.parametrize("group,bias", [(1, True), (3, False)])
def test_gradients_against_differences_of_the_forward_pass(group, bias):
    """fp32: (L(x + e u) - L(x - e u)) / 2e with L = sum(out g) against the gradients' product with u.  An output and a gradient
    are off by less than 45 * 2^-24 of their terms (close): the sums of these, the outputs' over e, are what is allowed, and
    the formula's own error at this e, which is worked out in 64 bits."""
    B, T, r, d = 2, 90, [16, 24], 32
    s = Step(B, T, r, r, d, F32, group, bias, seed=6)
    got = s.run()
    gen = torch.Generator().manual_seed(7)
    e = 2.0 ** -6

    def loss64(x, table):
        b = None if table is None else oracle.bias_by_distance(table, BUCKETS[1], T)
        return oracle.train(*[y.double().cpu().numpy() for y in x], r, r, d, group, None, b)

    base64 = loss64(s.x, s.table.double().cpu().numpy() if bias else None)
    noise = 45 * 2.0 ** -24 * np.sum(base64["out_size"] * np.abs(s.x[3].double().cpu().numpy())) / e
    for which in range(4 if bias else 3):
        name = ("dq", "dk", "dv", "table")[which]
        base = s.table if which == 3 else s.x[which]
        u = torch.randn(base.shape, generator=gen).cuda() * (base != 0)
        values, exact = [], []
        for sign in (1, -1):
            x = list(s.x)
            table = s.table if bias else None
            moved = base + sign * e * u
            if which == 3:
                table = moved
            else:
                x[which] = moved
            if bias:
                s.lay.set_bias(table)
            out = s.lay.train_forward(*x[:3], group=group)
            values.append((out.double() * x[3].double()).sum().item())
            exact.append(np.sum(loss64(x, table.double().cpu().numpy() if bias else None)["out"] * x[3].double().cpu().numpy()))
        if bias:
            s.lay.set_bias(s.table)
        by_hand = (got[1 + which].double() * u.double()).sum().item()
        difference, exact_difference = (values[0] - values[1]) / (2 * e), (exact[0] - exact[1]) / (2 * e)
        # the formula's truncation, from a step an eighth as long (its own is a 64th of it)
        fine = []
        for sign in (1, -1):
            x, table = [y.double() for y in s.x], s.table.double().cpu().numpy() if bias else None
            step = sign * e / 8 * u.double()
            if which == 3:
                table = table + step.cpu().numpy()
            else:
                x[which] = x[which] + step
            fine.append(np.sum(loss64(x, table)["out"] * x[3].cpu().numpy()))
        truncation = abs(exact_difference - (fine[0] - fine[1]) * 4 / e) * 64 / 63
        abs_u = u.abs().double().cpu().numpy()
        terms = np.sum(base64["by_distance_size"]) * abs_u.max() if which == 3 else np.sum(base64[name + "_size"] * abs_u)
        gradient_noise = 45 * 2.0 ** -24 * terms
        assert abs(difference - by_hand) <= noise + truncation * 1.01 + gradient_noise, (name, difference, by_hand, noise, truncation)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_steps_of_descent(dtype):
    """Forward pass, gradient of a loss on the outputs, backward pass, update of the rows and of the bias table: runs, with
    finite gradients that are those of the 64-bit formulas at the first and at the last step."""
    B, T, r, d = 2, 140, [24, 32], 64
    s = Step(B, T, r, r, d, dtype, bias=True, seed=8, lens=[140, 61])
    target = s.x[3]
    cols, width = oracle.packed_columns(r)
    master = [x.float() for x in s.x[:3]] + [s.table.float()]
    for step in range(5):
        x, table = [m.to(dtype) for m in master[:3]], master[3].to(dtype)
        s.lay.set_bias(table)
        out = s.lay.train_forward(*x, lens=s.lens)
        g = (out.float() - target.float()).to(dtype)
        grads = s.lay.train_backward(g, bias_grad=True)
        if step in (0, 4):
            want = oracle.train(*[y.double().cpu().numpy() for y in x], g.double().cpu().numpy(), r, r, d, 1, [140, 61],
                                oracle.bias_by_distance(table.double().cpu().numpy(), BUCKETS[1], T))
            for name, y in zip(("out", "dq", "dk", "dv"), (out,) + grads[:3]):
                close(y, want[name], want[name + "_size"], dtype, name)
        for m, y in zip(master, grads):
            assert torch.isfinite(y.float()).all()
            m -= 0.05 * y.float()
    s.lay.poll_status()


def test_refusals_that_need_a_device():
    from paper_2408_05646_b200 import binding
    s = Step(1, 64, [32], [32], 64, BF, bias=True)
    with pytest.raises(binding.EigenAttnError):
        s.lay.set_rope(10000.0)
    s.lay.bias_detach()
    s.lay.set_rope(10000.0)
    with pytest.raises(binding.EigenAttnError):
        s.lay.train_forward(*s.x[:3])
    with pytest.raises(binding.EigenAttnError):
        s.lay.bias_attach(*BUCKETS)
    s.lay.set_rope(0.0)
    s.lay.train_forward(*s.x[:3])
    with pytest.raises(binding.EigenAttnError):
        s.lay.train_backward(s.x[3], bias_grad=True)
    s.lay.train_backward(s.x[3])
    s.lay.train_detach()
    with pytest.raises(binding.EigenAttnError):
        s.lay.train_backward(s.x[3])


def test_tensors_that_the_binding_refuses():
    s = Step(2, 64, [32, 16], [16, 32], 64, BF, bias=True)
    q, k, v, g = s.x
    wide = torch.zeros(2, 64, 2 * q.shape[2], dtype=BF, device="cuda")
    lens = torch.tensor([64, 3], dtype=torch.int32, device="cuda")
    for bad in (q.float(), q.cpu(), q[:, :, :-8].contiguous(), wide[:, :, ::2], wide, q[:1]):
        with pytest.raises(AssertionError):
            s.lay.train_forward(bad, k, v)
        with pytest.raises(AssertionError):
            s.lay.train_forward(q, bad, v)
    for bad in (lens.cpu(), lens.long(), lens[:1], torch.zeros(4, dtype=torch.int32, device="cuda")[::2]):
        with pytest.raises(AssertionError):
            s.lay.train_forward(q, k, v, lens=bad)
    with pytest.raises(AssertionError):
        s.lay.train_forward(q, k, v, group=2)
    with pytest.raises(AssertionError):
        s.lay.train_forward(q[:, :63].contiguous(), k, v)
    want = Step(2, 64, [32, 16], [16, 32], 64, BF, bias=True).run()
    out = s.lay.train_forward(q, k, v)
    for bad in (g.float(), g.cpu(), g[:, :63].contiguous()):
        with pytest.raises(AssertionError):
            s.lay.train_backward(bad)
    for bad in (s.table.float(), s.table.cpu(), s.table[:, :-1].contiguous(), s.table[:1]):
        with pytest.raises(AssertionError):
            s.lay.set_bias(bad)
    assert same((out,) + tuple(s.lay.train_backward(g, bias_grad=True)), want)       # none of them changed anything
