"""Training in the rank-r space, and a learned bias of relative positions: what is measured, and the operators in their plain form.

Three operators over one layer's rows of rank r (q', k', v' as merged weights hand them over, Eq. 8 of the paper):

  train      causal attention of T tokens that keeps what its gradient needs, and the backward pass behind it
  backward   the backward pass alone, which recomputes the probabilities: gradients of q', k', v', and of the bias table
  decode     one new token per sequence over the cached rows, with the bias of each row's distance

The bias is one number per head and bucket of distances: the first half of the buckets hold one distance each, the others
grow in a geometric series up to a largest distance, and what lies behind it shares the last bucket.

`run` computes them with elementary torch operations, or, where `own` is true, through the layer's public calls.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
SEG = 64          # tokens that share a component: neighbouring tokens of a text have similar keys


def _case(name, op, dtype="bf16", batch=1, heads=32, group=1, d_head=128, ranks="80", tokens=0, context=0, ragged=False,
          page=0, alibi=False, buckets=0, far=0):
    return dict(name=name, op=op, dtype=dtype, batch=batch, heads=heads, group=group, d_head=d_head, ranks=ranks,
                tokens=tokens, context=context, ragged=ragged, page=page, alibi=alibi, buckets=buckets, far=far)


def listed():
    return [
        # the smallest layer (single precision, four heads) and a sentence: pure latency
        _case("backward_fp32_tiny", "backward", dtype="fp32", heads=4, d_head=64, ranks="32", tokens=77),
        # one short text through a 7B-class layer: latency at full width
        _case("backward_b1_t129", "backward", tokens=129),
        # the prompt workload the prefill is quoted on, as a fine-tuning batch
        _case("backward_7b_4k", "backward", batch=4, tokens=4096),
        # one long text of an ALiBi layer
        _case("backward_alibi_8k", "backward", ranks="64", tokens=8192, alibi=True),
        # grouped queries, texts of unequal lengths padded to a common one
        _case("backward_gqa_ragged", "backward", batch=8, heads=8, group=4, tokens=1500, ragged=True),
        # ranks that differ by head, as the compression picks them; a whole training step
        _case("train_ranks_1k", "train", batch=2, ranks="48,64,80,96,112", tokens=1111),
        # a small encoder-sized layer with a learned bias: a whole training step
        _case("train_bias_small", "train", batch=4, heads=8, d_head=64, ranks="40", tokens=200, buckets=32, far=128),
        # the same at single precision
        _case("train_bias_fp32", "train", dtype="fp32", batch=2, heads=8, d_head=64, ranks="40", tokens=500, buckets=32, far=128),
        # a 7B-class layer with a learned bias, long texts of unequal lengths
        _case("train_bias_7b_2k", "train", batch=4, tokens=2048, ragged=True, buckets=32, far=128),
        # one user, a short conversation: latency
        _case("decode_bias_b1", "decode", context=1000, buckets=32, far=128),
        # many conversations of unequal lengths in pages
        _case("decode_bias_paged", "decode", batch=16, context=8192, ragged=True, page=128, buckets=32, far=128),
        # the long-context batch the decode benchmark is quoted on
        _case("decode_bias_32k", "decode", batch=16, context=32768, buckets=64, far=1024),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    op = rng.choice(["backward", "backward", "train", "train", "decode"])
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    d_head = rng.choice([64, 96, 128, 128]) if dtype == "bf16" else rng.choice([64, 80])
    choices = [r for r in (20, 24, 32, 40, 48, 64, 80, 96, 112, 128) if r <= d_head]
    ranks = ",".join(str(r) for r in rng.sample(choices, 2)) if rng.random() < 0.3 else str(rng.choice(choices))
    widest = max(int(r) for r in ranks.split(","))
    heads = _log_int(rng, 2, 32)
    buckets = rng.choice([8, 21, 32, 64]) if op == "decode" or rng.random() < 0.4 else 0
    far = rng.choice([64, 128, 200, 1024]) if buckets else 0
    ragged = rng.random() < 0.4
    if op == "decode":
        batch = _log_int(rng, 1, 64)
        room = 1.3e9 / (batch * heads * 2 * widest) / (4 if dtype == "fp32" else 1)
        context = _log_int(rng, 40, int(max(41, min(131072, room))))
        drawn = _case("", op, dtype, batch, heads, 1, d_head, ranks, 0, context, ragged, 128 if rng.random() < 0.25 else 0,
                      False, buckets, far)
    else:
        group = rng.choice([1, 1, 2, 4]) if not buckets else 1
        alibi = group == 1 and not buckets and rng.random() < 0.3
        if heads * group > 32:
            heads = 32 // group
        batch = _log_int(rng, 1, 16)
        # (scores of a pass: those of the largest listed case of the type)
        room = math.sqrt((8e6 if dtype == "fp32" else 2e9) / (batch * heads * group))
        tokens = _log_int(rng, 17, int(max(18, min(8192, room))))
        drawn = _case("", op, dtype, batch, heads, group, d_head, ranks, tokens, 0, ragged, 0, alibi, buckets, far)
    return {k: v for k, v in drawn.items() if k != "name"}


# ---------------------------------------------------------------- what a case stands for

def _ranks(case):
    r = [int(x) for x in case["ranks"].split(",")]
    return [r[h % len(r)] for h in range(case["heads"])]


def _pad8(r):
    return (r + 7) // 8 * 8


def _lens(case):
    n, B = case["tokens"] or case["context"], case["batch"]
    return [max(1, n * (b + 1) // B - b % 3) for b in range(B)] if case["ragged"] else [n] * B


def _slopes(case):
    return [2.0 ** (-8.0 * (h + 1) / case["heads"]) for h in range(case["heads"])] if case["alibi"] else None


def _starts(n_buckets, far):
    """First distance of every bucket: single ones below half = n_buckets // 2, from there a geometric series up to `far`:
    distance d lies in bucket half + k, k the largest with (d / half)^rest >= (far / half)^k, or in the last one."""
    half = n_buckets // 2
    rest = n_buckets - half
    starts, d = list(range(half)), half
    for k in range(rest):
        while d ** rest * half ** k < far ** k * half ** rest:
            d += 1
        starts.append(d)
    return starts


def _bucket_of(case, count):
    """Bucket of the distances 0 .. count - 1."""
    starts = _starts(case["buckets"], case["far"])
    out, k = [], 0
    for d in range(count):
        while k + 1 < len(starts) and starts[k + 1] <= d:
            k += 1
        out.append(k)
    return out


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    B, H, g, d = case["batch"], case["heads"], case["group"], case["d_head"]
    rs, lens = sum(_ranks(case)), _lens(case)
    table = H * case["buckets"] * es
    if case["op"] == "decode":
        return {"bytes": 2 * rs * es * sum(lens) + 2 * B * H * d * es + 2 * d * rs * 4 + table, "flops": 4 * rs * sum(lens)}
    pairs = sum(n * (n + 1) // 2 for n in lens) * g
    rows = sum(lens)
    # q', k', v' and the gradient of o' in, the gradients of q', k', v' out; a whole step also writes o'
    moved = rs * es * rows * (g + 2 + g) + rs * es * rows * (g + 2) + 2 * table
    flops = 2 * pairs * rs * 5
    if case["op"] == "train":
        moved += rs * es * rows * g
        flops += 2 * pairs * rs * 2
    else:
        moved += rs * es * rows * g + 4 * rows * H * g          # o' and the log-sum-exp of the forward pass
    return {"bytes": moved, "flops": flops}


# ---------------------------------------------------------------- inputs

def _basis(d, r, gen):
    q, _ = torch.linalg.qr(torch.randn(d, r, generator=gen, dtype=torch.float64))
    return q.float()


def _columns(case, group):
    """Where the packed rows keep head h * group + i: [H * group][R] columns, the packed width where a head has none."""
    ranks = _ranks(case)
    R = max(_pad8(r) for r in ranks)
    width = group * sum(_pad8(r) for r in ranks)
    at, base = [], 0
    for r in ranks:
        for _ in range(group):
            at.append([base + c if c < r else width for c in range(R)])
            base += _pad8(r)
    return torch.tensor(at), width


def prepare(case, seed):
    dev = torch.device("cuda")
    dt = DTYPES[case["dtype"]]
    B, H, g, T, n = (case[k] for k in ("batch", "heads", "group", "tokens", "context"))
    gen = torch.Generator(device=dev).manual_seed(seed)
    s = {"case": case, "lens": torch.tensor(_lens(case), device=dev)}
    s["slopes"] = torch.tensor(_slopes(case), device=dev, dtype=torch.float64) if case["alibi"] else None
    rows = T or n

    def packed(group, scale, shared):
        at, width = _columns(case, group)
        pad = -(-rows // SEG) * SEG
        x = torch.randn(B, pad, width, generator=gen, device=dev, dtype=dt)
        if shared:
            part = torch.randn(B, pad // SEG, 1, width, generator=gen, device=dev, dtype=dt)
            x.view(B, pad // SEG, SEG, width).mul_(0.8).add_(part, alpha=0.6)
        live = torch.zeros(width + 1, device=dev)
        live[at.to(dev).flatten()] = scale
        x.mul_(live[:width].to(dt))
        return x[:, :rows].contiguous()

    s["k"], s["v"] = packed(1, 1.0, True), packed(1, 1.0, True)
    if case["buckets"]:
        s["table"] = torch.randn(H, case["buckets"], generator=gen, device=dev).to(dt)
        s["bucket"] = torch.tensor(_bucket_of(case, rows), device=dev)
    s["col_k"], s["wide_k"] = _columns(case, g)
    s["col_1"], s["wide_1"] = _columns(case, 1)
    s["col_k"], s["col_1"] = s["col_k"].to(dev), s["col_1"].to(dev)
    if T:
        s["q"] = packed(g, 1.5, False)
        # the gradient a loss sends back: small numbers, and none for padded tokens
        s["d_out"] = packed(g, 2.0 ** -10, False)
        s["d_out"].masked_fill_((torch.arange(T, device=dev) >= s["lens"][:, None])[:, :, None], 0)
    else:
        s["q"] = (torch.randn(B, 1, H, case["d_head"], generator=gen, device=dev) * 2.0).to(dt)
    cpu = torch.Generator().manual_seed(seed)
    bases = {}
    for side in "kv":
        bases[side] = torch.zeros(H, case["d_head"], s["col_1"].shape[1])
        for h, r in enumerate(_ranks(case)):
            bases[side][h, :, :r] = _basis(case["d_head"], r, cpu)
    s["U_k"], s["U_v"] = bases["k"].to(dev), bases["v"].to(dev)
    if own:
        s["layer"] = _layer(s, bases)
    return s


def _layer(s, bases):
    """The layer a user's program holds: its bias set, its scratch attached, its cache filled."""
    from paper_2408_05646_b200 import binding
    case, ranks = s["case"], _ranks(s["case"])
    B, H, T, n = (case[k] for k in ("batch", "heads", "tokens", "context"))
    n_max = -(-n // 128) * 128 if n else 8
    lay = binding.EigenAttnLayer(B, H, case["d_head"], n_max, DTYPES[case["dtype"]],
                                 [bases["k"][h, :, :r].numpy() for h, r in enumerate(ranks)],
                                 [bases["v"][h, :, :r].numpy() for h, r in enumerate(ranks)])
    if case["alibi"]:
        lay.set_alibi(_slopes(case))
    if case["buckets"]:
        lay.bias_attach(case["buckets"], case["far"])
        lay.set_bias(s["table"])
    if T:
        lay.train_attach(T, case["group"])
        s["lens32"] = s["lens"].to(torch.int32) if case["ragged"] else None
        if case["op"] == "backward":
            lay.train_forward(s["q"], s["k"], s["v"], lens=s["lens32"], group=case["group"])
        return lay
    if case["page"]:
        pages = list(range(B * n_max // case["page"]))
        random.Random(5).shuffle(pages)
        width = len(pages) // B
        lay.set_page_table([pages[b * width:(b + 1) * width] for b in range(B)], case["page"])
    for x in range(0, n, 8192):          # a prompt arrives in chunks
        lay.append_kv(s["k"][:, x:x + 8192].contiguous(), s["v"][:, x:x + 8192].contiguous(), preprojected=True)
    if case["ragged"]:
        lay.set_lens(_lens(case))
    return lay


# ---------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    if case["op"] == "decode":
        return _decode_own(s) if own else _decode_plain(s)
    return _train_own(s) if own else _train_plain(s)


def _train_own(s):
    case, lay = s["case"], s["layer"]
    result = {}
    if case["op"] == "train":
        if case["buckets"]:
            lay.set_bias(s["table"])      # the optimiser has changed it since the step before
        result["out"] = lay.train_forward(s["q"], s["k"], s["v"], lens=s["lens32"], group=case["group"])
    if case["buckets"]:
        result["dq"], result["dk"], result["dv"], result["dtable"] = lay.train_backward(s["d_out"], bias_grad=True)
    else:
        result["dq"], result["dk"], result["dv"] = lay.train_backward(s["d_out"])
    return result


def _heads(x, at):
    """Packed rows [T][width] as [heads][T][R], zeros where a head has no such column."""
    return torch.nn.functional.pad(x, (0, 1))[:, at].permute(1, 0, 2)


def _pack(x, at, width):
    """[heads][T][R] back to packed rows."""
    out = torch.zeros(x.shape[1], width + 1, dtype=x.dtype, device=x.device)
    out[:, at.flatten()] = x.permute(1, 0, 2).flatten(1)
    return out[:, :width]


def _by_distance(x):
    """[heads][T][T] summed over what has the same distance i - j >= 0: [heads][T], in 64 bits."""
    H, T, _ = x.shape
    # row i moved so that its column T - 1 - i + j holds entry j: distance d stands in column T - 1 - d throughout
    y = torch.nn.functional.pad(x.flip(1), (0, T)).flatten(1)
    return y[:, :T * (2 * T - 1)].view(H, T, 2 * T - 1)[:, :, :T].sum(1, dtype=torch.float64).flip(1)


def _train_plain(s):
    case = s["case"]
    B, H, g, d, T = (case[k] for k in ("batch", "heads", "group", "d_head", "tokens"))
    dt, dev = DTYPES[case["dtype"]], s["q"].device
    scale = 1.0 / math.sqrt(d)
    parts = {k: [] for k in ("out", "dq", "dk", "dv")}
    sums = torch.zeros(H, T, dtype=torch.float64, device=dev)
    place = torch.arange(T, device=dev)
    far = place[:, None] - place
    for b in range(B):
        q, do = _heads(s["q"][b].float(), s["col_k"]), _heads(s["d_out"][b].float(), s["col_k"])
        k, v = (_heads(s[x][b].float(), s["col_1"]).repeat_interleave(g, 0) for x in "kv")
        x = (q @ k.transpose(1, 2)).mul_(scale)
        if s["slopes"] is not None:
            x -= (s["slopes"][:, None, None] * far).float()
        if case["buckets"]:
            x += s["table"].float()[:, s["bucket"][far.clamp_min(0)]]
        shut = (far < 0) | (place[:, None] >= s["lens"][b])
        x.masked_fill_(shut, -math.inf)
        p = torch.exp_(x.sub_(x.amax(2, keepdim=True).clamp_min(-1e30)))
        p /= p.sum(2, keepdim=True).clamp_min(1e-30)
        if case["op"] == "train":
            parts["out"].append(_pack(p @ v, s["col_k"], s["wide_k"]).to(dt))
        parts["dv"].append(_pack((p.transpose(1, 2) @ do).view(H, g, T, -1).sum(1), s["col_1"], s["wide_1"]).to(dt))
        dx = do @ v.transpose(1, 2)
        dx.sub_((p * dx).sum(2, keepdim=True)).mul_(p)
        del p, x
        parts["dq"].append(_pack((dx @ k).mul_(scale), s["col_k"], s["wide_k"]).to(dt))
        parts["dk"].append(_pack((dx.transpose(1, 2) @ q).mul_(scale).view(H, g, T, -1).sum(1), s["col_1"], s["wide_1"]).to(dt))
        if case["buckets"]:
            sums += _by_distance(dx)
        del dx
    result = {k: torch.stack(x) for k, x in parts.items() if x}
    if case["buckets"]:
        into = torch.nn.functional.one_hot(s["bucket"], case["buckets"]).double()
        result["dtable"] = (sums @ into).to(dt)
    return result


def _decode_own(s):
    return {"out": s["layer"].decode(s["q"])}


def _decode_plain(s):
    case = s["case"]
    B, H, d, n = (case[k] for k in ("batch", "heads", "d_head", "context"))
    out = []
    place = torch.arange(n, device=s["q"].device)
    for b in range(B):
        k, v = (_heads(s[x][b], s["col_1"]).float() for x in "kv")
        q = torch.einsum("hd,hdr->hr", s["q"][b, 0].float(), s["U_k"]) / math.sqrt(d)
        x = torch.einsum("hr,hnr->hn", q, k)
        x += s["table"].float()[:, s["bucket"][(s["lens"][b] - 1 - place).clamp_min(0)]]
        x.masked_fill_(place >= s["lens"][b], -math.inf)
        p = torch.exp(x - x.amax(1, keepdim=True))
        o = torch.einsum("hn,hnr->hr", p, v) / p.sum(1, keepdim=True)
        out.append(torch.einsum("hr,hdr->hd", o, s["U_v"]))
    return {"out": torch.stack(out)[:, None].to(DTYPES[case["dtype"]])}


# ---------------------------------------------------------------- the definitions in 64 bits, one sequence and head at a time

def exact(case, seed):
    s = prepare(case, seed)
    B, H, g, d, T = (case[k] for k in ("batch", "heads", "group", "d_head", "tokens"))
    lens, ranks, slopes, dev = _lens(case), _ranks(case), _slopes(case), s["q"].device
    starts = torch.tensor(_starts(case["buckets"], case["far"]), device=dev) if case["buckets"] else None
    rows = max(lens)
    bucket = torch.searchsorted(starts, torch.arange(rows, device=dev), right=True) - 1 if case["buckets"] else None
    if case["op"] == "decode":
        out = torch.zeros(B, 1, H, d, dtype=torch.float64, device=dev)
        base = 0
        for h, r in enumerate(ranks):
            Uk, Uv = s["U_k"][h, :, :r].double(), s["U_v"][h, :, :r].double()
            for b, n in enumerate(lens):
                K, V = (s[x][b, :n, base:base + r].double() for x in "kv")
                x = K @ (s["q"][b, 0, h].double() @ Uk) / math.sqrt(d) + s["table"][h].double()[bucket[:n].flip(0)]
                out[b, 0, h] = (torch.softmax(x, 0) @ V) @ Uv.T
            base += _pad8(r)
        return {"out": out}
    if B * H * g * T * T > 3e9:
        return None
    got = {"out": torch.zeros(B, T, s["wide_k"], dtype=torch.float64, device=dev)}
    got["dq"] = torch.zeros_like(got["out"])
    got["dk"] = torch.zeros(B, T, s["wide_1"], dtype=torch.float64, device=dev)
    got["dv"] = torch.zeros_like(got["dk"])
    if case["buckets"]:
        got["dtable"] = torch.zeros(H, case["buckets"], dtype=torch.float64, device=dev)
    base = 0
    for h, r in enumerate(ranks):
        for b, n in enumerate(lens):
            far = torch.arange(n, device=dev)[:, None] - torch.arange(n, device=dev)
            keys = [s[x][b, :n, base:base + r].double().requires_grad_() for x in "kv"]
            biases = s["table"][h].double()[bucket[:n]].requires_grad_() if case["buckets"] else None
            for i in range(g):
                at = slice(g * base + i * _pad8(r), g * base + i * _pad8(r) + r)
                q = s["q"][b, :n, at].double().requires_grad_()
                x = q @ keys[0].T / math.sqrt(d)
                if slopes:
                    x = x - slopes[h] * far
                if biases is not None:
                    x = x + biases.index_select(0, far.clamp_min(0).flatten()).view(n, n)
                o = torch.softmax(x.masked_fill(far < 0, -math.inf), 1) @ keys[1]
                o.backward(s["d_out"][b, :n, at].double())
                got["out"][b, :n, at], got["dq"][b, :n, at] = o.detach(), q.grad
                del o, x
            got["dk"][b, :n, base:base + r], got["dv"][b, :n, base:base + r] = keys[0].grad, keys[1].grad
            if biases is not None:
                got["dtable"][h].index_add_(0, bucket[:n], biases.grad)
        base += _pad8(r)
    if case["op"] != "train":
        del got["out"]
    return got
