"""Speculative and block-sparse decoding over the rank-r cache: what is measured, and the operators in their plain form.

Four operators over one layer's cache (K' and V' rows of rank r per K/V head, Section 4 of the paper):

  tree     attention of T drafted tokens per sequence, arranged as a tree, over the cached rows and their own ancestors;
           the drafted rows are projected and stored behind the sequence's rows
  step     the same followed by the acceptance of one path: its rows move together, the sequence grows by them
  blocks   per-channel minima and maxima of the keys of every complete block of cached rows
  sparse   decode over the blocks whose bound on the scores is highest for the token's query, besides the first and
           the newest ones

`run` computes them with elementary torch operations, or, where `own` is true, through the layer's public calls.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
SEG = 64          # rows that share a component: neighbouring tokens of a text have similar keys


def _case(name, op, dtype="bf16", batch=1, heads=32, group=1, d_head=128, ranks="80", context=2048, ragged=False,
          page=0, alibi=False, tokens=0, chain=False, block=0, budget=0):
    return dict(name=name, op=op, dtype=dtype, batch=batch, heads=heads, group=group, d_head=d_head, ranks=ranks,
                context=context, ragged=ragged, page=page, alibi=alibi, tokens=tokens, chain=chain, block=block,
                budget=budget)


def listed():
    return [
        # the smallest layer (single precision, four heads): a handful of drafted tokens, pure latency
        _case("tree_fp32_tiny", "tree", dtype="fp32", heads=4, d_head=64, ranks="32", context=512, tokens=5),
        # one user of a 7B-class layer, a short chain from a draft model: latency again, at full width
        _case("tree_chain_b1", "tree", context=2048, tokens=4, chain=True),
        # grouped queries, sequences of unequal lengths, a wide tree: 128 query rows for every K/V head
        _case("tree_gqa_ragged", "tree", batch=16, heads=8, group=4, context=8192, ragged=True, tokens=32),
        # the long-context batch the decode benchmark is quoted on, a tree of 16 tokens per sequence
        _case("tree_7b_32k", "tree", batch=16, context=32768, tokens=16),
        # one whole speculative step on a paged cache: the widest odd tree, a context that ends inside a tile
        _case("step_paged", "step", batch=8, context=4097, page=128, tokens=63),
        # many short conversations of an ALiBi layer, small trees
        _case("step_b64_short", "step", batch=64, ranks="64", context=777, alibi=True, tokens=8),
        # block bounds after one prompt
        _case("blocks_b1_8k", "blocks", context=8192, block=64),
        # block bounds of a whole long-context batch
        _case("blocks_7b_32k", "blocks", batch=16, context=32768, block=32),
        # the smallest layer, single precision
        _case("sparse_fp32_tiny", "sparse", dtype="fp32", heads=4, d_head=64, ranks="32", context=500, block=16, budget=8),
        # one very long conversation of an ALiBi layer
        _case("sparse_b1_131k", "sparse", ranks="64", context=131072, alibi=True, block=64, budget=64),
        # ranks that differ by head, grouped queries, unequal lengths (some shorter than the budget)
        _case("sparse_gqa_ragged", "sparse", batch=16, heads=8, group=4, ranks="48,64,80,96,112", context=32768, ragged=True,
              block=128, budget=32),
        # the long-context batch: an eighth of the rows
        _case("sparse_7b_32k", "sparse", batch=16, context=32768, block=32, budget=128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    op = rng.choice(["tree", "tree", "step", "blocks", "sparse", "sparse"])
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    group = rng.choice([1, 1, 1, 2, 4, 8]) if op != "blocks" else 1
    heads = _log_int(rng, 2, 32)
    if heads * group > 64:
        heads = 64 // group
    d_head = rng.choice([64, 96, 128, 128]) if dtype == "bf16" else rng.choice([64, 80])
    choices = [r for r in (24, 32, 48, 64, 80, 96, 112, 128) if r <= d_head]
    ranks = ",".join(str(r) for r in rng.sample(choices, 2)) if op == "sparse" and rng.random() < 0.3 else str(rng.choice(choices))
    batch = _log_int(rng, 1, 64)
    tokens = _log_int(rng, 1, 64) if op in ("tree", "step") else 0
    block = rng.choice([16, 32, 64, 128]) if op in ("blocks", "sparse") else 0
    widest = max(int(r) for r in ranks.split(","))
    # rows of a sequence: bounded by the cache of the largest listed case, and by its scores in the plain form
    room = 1.3e9 / (batch * heads * 2 * widest) / (4 if dtype == "fp32" else 1)
    room = min(room, 2.6e8 / (batch * heads * group * max(1, tokens)))
    context = _log_int(rng, max(block, 40), int(max(max(block, 40) + 1, min(131072, room))))
    budget = _log_int(rng, 3, max(4, min(256, 8192 // block))) if op == "sparse" else 0
    return {k: v for k, v in _case("", op, dtype, batch, heads, group, d_head, ranks, context, ragged=rng.random() < 0.4,
                                   page=128 if rng.random() < 0.25 else 0, alibi=group == 1 and rng.random() < 0.25,
                                   tokens=tokens, chain=rng.random() < 0.3, block=block, budget=budget).items() if k != "name"}


# ---------------------------------------------------------------- what a case stands for

def _ranks(case):
    r = [int(x) for x in case["ranks"].split(",")]
    return [r[h % len(r)] for h in range(case["heads"])]


def _lens(case):
    n, B = case["context"], case["batch"]
    return [max(1, n * (b + 1) // B - b % 3) for b in range(B)] if case["ragged"] else [n] * B


def _slopes(case):
    return [2.0 ** (-8.0 * (h + 1) / case["heads"]) for h in range(case["heads"])] if case["alibi"] else None


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    B, H, g, d, T = case["batch"], case["heads"], case["group"], case["d_head"], case["tokens"]
    lens, rs = _lens(case), sum(_ranks(case))
    if case["op"] == "blocks":
        rows = sum(n // case["block"] for n in lens) * case["block"]
        return {"bytes": rs * es * (rows + 2 * rows // case["block"]), "flops": 2 * rs * rows}
    bases = 2 * d * rs * 4
    if case["op"] == "sparse":
        nb = [-(-n // case["block"]) for n in lens]
        rows = sum(min(n, case["budget"] * case["block"]) for n in lens)
        scored = sum(n for n in nb if n > case["budget"])
        io = 2 * B * H * g * d * es + 4 * B * H * case["budget"]
        flops = 2 * g * (rs * 2 * rows + rs * scored + B * 2 * d * rs)
        return {"bytes": 2 * rs * es * rows + 2 * rs * es * scored + io + bases, "flops": flops}
    io = (2 * g + 2) * B * T * H * d * es + 2 * B * T * rs * es + 8 * B * T
    if case["op"] == "step":
        io += 2 * B * (T // 2) * rs * es * 2          # an accepted path of about half the depth is read and written
    flops = 2 * g * T * 2 * rs * (sum(lens) + B * T) + 2 * B * T * d * rs * (2 * g + 2)
    return {"bytes": 2 * rs * es * sum(lens) + io + bases, "flops": flops}


# ---------------------------------------------------------------- inputs

def _basis(d, r, gen):
    q, _ = torch.linalg.qr(torch.randn(d, r, generator=gen, dtype=torch.float64))
    return q.float()


def _trees(case, seed):
    """Parent of every drafted token (-1: the last cached token), ancestor masks and one accepted path per sequence."""
    rng = random.Random(seed * 7919 + 1)
    B, T = case["batch"], case["tokens"]
    masks, paths = [], []
    for b in range(B):
        parent, bits = [], []
        for t in range(T):
            p = t - 1 if case["chain"] else max(rng.randint(-1, t - 1), rng.randint(-1, t - 1))
            parent.append(p)
            bits.append((1 << t) | (bits[p] if p >= 0 else 0))
        masks.append([x - (1 << 64) if x >> 63 else x for x in bits])
        path, t = [], rng.randint(0, T - 1)
        while t >= 0:
            path.append(t)
            t = parent[t]
        path.reverse()
        paths.append(path[:rng.randint(0 if b % 4 == 3 else 1, len(path))])
    return masks, paths


def prepare(case, seed):
    dev = torch.device("cuda")
    dt = DTYPES[case["dtype"]]
    B, H, g, d, T, n = (case[k] for k in ("batch", "heads", "group", "d_head", "tokens", "context"))
    ranks = _ranks(case)
    R = max(ranks)
    cpu = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device=dev).manual_seed(seed)
    live = torch.zeros(H, R)
    for h, r in enumerate(ranks):
        live[h, :r] = 1.0
    bases = {}
    for side in "kv":
        bases[side] = torch.zeros(H, d, R)
        for h, r in enumerate(ranks):
            bases[side][h, :, :r] = _basis(d, r, cpu)

    def rows(scale):
        pad = -(-n // SEG) * SEG
        x = torch.randn(B, pad, H, R, generator=gen, device=dev, dtype=dt)
        shared = torch.randn(B, pad // SEG, 1, H, R, generator=gen, device=dev, dtype=dt)
        x.view(B, pad // SEG, SEG, H, R).mul_(0.8).add_(shared, alpha=0.6)
        return (x.mul_(live.to(dev, dt) * scale))[:, :n]

    def tokens(count, heads, scale):
        return (torch.randn(B, count, heads, d, generator=gen, device=dev) * scale).to(dt)

    s = {"case": case, "lens": torch.tensor(_lens(case), device=dev), "K": rows(1.0), "V": rows(1.0),
         "U_k": bases["k"].to(dev), "U_v": bases["v"].to(dev), "ranks": ranks}
    s["slopes"] = torch.tensor(_slopes(case), device=dev, dtype=torch.float64) if case["alibi"] else None
    if T:
        masks, paths = _trees(case, seed)
        s["mask"] = torch.tensor(masks, dtype=torch.int64, device=dev)
        s["paths"] = paths
        s["moved"] = torch.tensor([p + list(range(len(p), T)) for p in paths], device=dev)
        s["q"], s["k"], s["v"] = tokens(T, H * g, 2.0), tokens(T, H, 1.0), tokens(T, H, 1.0)
    elif case["op"] == "sparse":
        s["q"] = tokens(1, H * g, 2.0)
        s["lo"], s["hi"] = _block_bounds(s["K"], case["block"])
    if own:
        s["layer"] = _layer(s, bases)
    return s


def _block_bounds(K, block):
    B, n, H, R = K.shape
    x = K[:, :n // block * block].view(B, n // block, block, H, R)
    return x.amin(2), x.amax(2)


def _layer(s, bases):
    """The layer a user's program holds: the cache filled, its lengths set, the block bounds up to date."""
    from paper_2408_05646_b200 import binding
    case, ranks = s["case"], s["ranks"]
    B, H, d, T, n = (case[k] for k in ("batch", "heads", "d_head", "tokens", "context"))
    n_max = -(-(n + T) // 128) * 128
    lay = binding.EigenAttnLayer(B, H, d, n_max, DTYPES[case["dtype"]],
                                 [bases["k"][h, :, :r].numpy() for h, r in enumerate(ranks)],
                                 [bases["v"][h, :, :r].numpy() for h, r in enumerate(ranks)])
    if case["page"]:
        pages = list(range(B * n_max // case["page"]))
        random.Random(5).shuffle(pages)
        width = len(pages) // B
        s["pages"] = torch.tensor(pages, device="cuda").view(B, width)
        lay.set_page_table(s["pages"].tolist(), case["page"])
    R = max(ranks)
    cols = torch.tensor([h * R + c for h, r in enumerate(ranks) for c in range(r)], device="cuda")
    for x in range(0, n, 8192):          # a prompt arrives in chunks
        part = [s[side][:, x:x + 8192].reshape(B, -1, H * R).contiguous() for side in "KV"]
        lay.append_kv(*[p if len(cols) == H * R else p[:, :, cols] for p in part], preprojected=True)
    if case["ragged"]:
        lay.set_lens(_lens(case))
    if case["alibi"]:
        lay.set_alibi(_slopes(case))
    if T:
        lay.tree_attach(T, case["group"])
        s["pools"] = [_pool(lay, i, H, B * n_max, R) for i in (0, 1)]
        at = s["lens"][:, None] + torch.arange(T, device="cuda")
        if case["page"]:
            s["at"] = s["pages"].gather(1, at // case["page"]) * case["page"] + at % case["page"]
        else:
            s["at"] = at + n_max * torch.arange(B, device="cuda")[:, None]
    else:
        lay.sparse_attach(case["block"])
        lay.sparse_sync()
    return lay


def _pool(lay, side, H, rows, r):
    """All heads' K' (or V') slabs as one [H][rows][r] view of the cache."""
    first = lay.cache_layout(0)[side]
    step = lay.cache_layout(1)[side] - first
    flat = lay.cache.view(lay.torch_dtype)
    es = flat.element_size()
    return flat.as_strided((H, rows, r), (step // es, r, 1), flat.storage_offset() + first // es)


# ---------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if op == "blocks":
        return _blocks_own(s) if own else _blocks_plain(s)
    if op == "sparse":
        return _sparse_own(s) if own else _sparse_plain(s)
    return _tree_own(s) if own else _tree_plain(s)


def _rewind(s):
    case = s["case"]
    if case["ragged"]:
        s["layer"].set_lens(_lens(case))
    else:
        s["layer"].set_len(case["context"])


def _tree_own(s):
    case, lay = s["case"], s["layer"]
    if case["op"] == "step":
        _rewind(s)                        # the pass before this one has grown the sequences
    out = lay.decode_tree(s["q"], s["k"], s["v"], s["mask"], group=case["group"])
    if case["op"] == "step":
        lay.tree_commit(s["paths"], case["tokens"])
    B, H, T = case["batch"], case["heads"], case["tokens"]
    if not case["ragged"] and not case["page"]:
        n = case["context"]
        k, v = (p.view(H, B, -1, p.shape[-1])[:, :, n:n + T] for p in s["pools"])
    else:
        k, v = (p[:, s["at"]] for p in s["pools"])
    return {"out": out, "k": k, "v": v}


def _tree_plain(s):
    case = s["case"]
    B, H, g, d, T, n = (case[k] for k in ("batch", "heads", "group", "d_head", "tokens", "context"))
    dt = DTYPES[case["dtype"]]
    # the drafted rows as the cache keeps them, and the queries, in the rank-r space
    kn = torch.einsum("bthd,hdr->bhtr", s["k"].float(), s["U_k"]).to(dt)
    vn = torch.einsum("bthd,hdr->bhtr", s["v"].float(), s["U_v"]).to(dt)
    q = torch.einsum("bthgd,hdr->bhgtr", s["q"].float().view(B, T, H, g, d), s["U_k"]).reshape(B, H, g * T, -1)
    q = q * (1.0 / math.sqrt(d))
    seen = (s["mask"][:, :, None] >> torch.arange(T, device=q.device)) & 1 > 0                   # [B][T][T]
    old = q @ s["K"].permute(0, 2, 3, 1).float()                                                 # [B][H][gT][n]
    new = q @ kn.float().transpose(2, 3)
    if s["slopes"] is not None:
        depth = (seen & ~torch.eye(T, device=q.device, dtype=torch.bool)).sum(2)                 # [B][T]: ancestors
        pos = s["lens"][:, None] + depth
        far = pos[:, :, None] - torch.arange(n, device=q.device)
        old -= (s["slopes"][:, None, None] * far[:, None]).float()
        new -= (s["slopes"][:, None, None] * (pos[:, :, None] - pos[:, None, :])[:, None]).float()
    old.masked_fill_((torch.arange(n, device=q.device) >= s["lens"][:, None])[:, None, None], -math.inf)
    new = new.view(B, H, g, T, T).masked_fill(~seen[:, None, None], -math.inf).view(B, H, g * T, T)
    top = torch.maximum(old.amax(3, keepdim=True), new.amax(3, keepdim=True)).clamp_min(-1e30)
    old, new = torch.exp_(old.sub_(top)), torch.exp(new - top)
    o = old @ s["V"].permute(0, 2, 1, 3).float() + new @ vn.float()
    o = o / (old.sum(3, keepdim=True) + new.sum(3, keepdim=True)).clamp_min(1e-30)
    out = torch.einsum("bhgtr,hdr->bthgd", o.view(B, H, g, T, -1), s["U_v"]).reshape(B, T, H * g, d).to(dt)
    if case["op"] == "step":
        at = s["moved"][:, None, :, None].expand(-1, H, -1, kn.shape[3])
        kn, vn = kn.gather(2, at), vn.gather(2, at)
    return {"out": out, "k": kn.transpose(0, 1), "v": vn.transpose(0, 1)}


def _complete(s):
    """[B][blocks]: the blocks whose rows are all there."""
    nb = s["K"].shape[1] // s["case"]["block"]
    return torch.arange(nb, device=s["K"].device) < (s["lens"] // s["case"]["block"])[:, None]


def _blocks_own(s):
    lay = s["layer"]
    lay.set_len(0)                        # forget the bounds of the pass before this one
    _rewind(s)
    lay.sparse_sync()
    return _bounds_of(s)


def _bounds_of(s):
    """The bounds as [B][blocks][H][r], zeros where a sequence has no such block (a view where all have)."""
    case, lay = s["case"], s["layer"]
    nb = case["context"] // case["block"]
    x = lay.sparse_bounds()               # [H][B][blocks of n_max][2][r]
    if case["page"]:
        per = case["page"] // case["block"]
        blk = torch.arange(nb, device=x.device)
        at = s["pages"][:, blk // per] * per + blk % per
        x = x.reshape(case["heads"], -1, 2, x.shape[-1])[:, at]
    x = x[:, :, :nb].permute(1, 2, 0, 3, 4)
    if case["ragged"]:
        x = x.masked_fill(~_complete(s)[:, :, None, None, None], 0)          # (nothing has been written there)
    return {"lo": x[..., 0, :], "hi": x[..., 1, :]}


def _blocks_plain(s):
    lo, hi = _block_bounds(s["K"], s["case"]["block"])
    if s["case"]["ragged"]:
        there = _complete(s)[:, :, None, None]
        lo, hi = lo * there, hi * there
    return {"lo": lo, "hi": hi}


def _sparse_own(s):
    out, index = s["layer"].decode_sparse(s["q"], s["case"]["budget"], group=s["case"]["group"], return_index=True)
    return {"out": out, "index": index}


def _sparse_plain(s):
    case = s["case"]
    B, H, g, d, n, G, M = (case[k] for k in ("batch", "heads", "group", "d_head", "context", "block", "budget"))
    dev = s["K"].device
    # the choice in 64 bits: two bounds may be close
    q64 = torch.einsum("bhgd,hdr->bhgr", s["q"].double().view(B, H, g, d), s["U_k"].double()) / math.sqrt(d)
    lo, hi = s["lo"].double(), s["hi"].double()                                                  # [B][blocks][H][R]
    bound = (torch.einsum("bhgr,bnhr->bhgn", q64.clamp_min(0), hi) +
             torch.einsum("bhgr,bnhr->bhgn", q64.clamp_max(0), lo)).amax(2)                      # [B][H][blocks]
    nb = -(-n // G)
    bound = torch.nn.functional.pad(bound, (0, nb - bound.shape[2]))
    blk = torch.arange(nb, device=dev)
    if s["slopes"] is not None:
        bound = bound - s["slopes"][:, None] * (s["lens"][:, None] - 1 - (blk * G + G - 1))[:, None]
    have = -(-s["lens"] // G)                                                                    # blocks of a sequence
    bound = torch.where(((blk < 1) | (blk == have[:, None] - 1))[:, None], math.inf, bound)
    bound = torch.where((blk >= have[:, None])[:, None], -math.inf, bound)
    pick = bound.sort(dim=2, descending=True, stable=True).indices[:, :, :M]
    pick = torch.where(pick < have[:, None, None], pick, nb).sort(dim=2).values
    pick = torch.nn.functional.pad(pick, (0, M - pick.shape[2]), value=nb)
    row = (pick[..., None] * G + torch.arange(G, device=dev)).view(B, H, M * G)
    dead = (row >= s["lens"][:, None, None]) | (pick == nb).repeat_interleave(G, 2)
    at = (torch.arange(B, device=dev)[:, None, None], row.clamp_max(n - 1), torch.arange(H, device=dev)[:, None])
    q = q64.float()
    p = q @ s["K"][at].float().transpose(2, 3)                                                   # [B][H][g][rows]
    if s["slopes"] is not None:
        p -= (s["slopes"][:, None] * (s["lens"][:, None, None] - 1 - row))[:, :, None].float()
    p = torch.softmax(p.masked_fill(dead[:, :, None], -math.inf), 3)
    o = p @ s["V"][at].float()
    out = torch.einsum("bhgr,hdr->bhgd", o, s["U_v"]).reshape(B, 1, H * g, d).to(DTYPES[case["dtype"]])
    return {"out": out, "index": torch.where(pick == nb, -1, pick).to(torch.int32)}


# ---------------------------------------------------------------- the definitions in 64 bits, one sequence and head at a time

def exact(case, seed):
    B, H, g, d, T = (case[k] for k in ("batch", "heads", "group", "d_head", "tokens"))
    if B * H * g * max(1, T) * case["context"] > 6e8 or B * H > 4096:
        return None
    s = prepare(case, seed)
    if case["op"] == "blocks":
        G, nb = case["block"], case["context"] // case["block"]
        ends = torch.zeros(2, B, nb, H, max(s["ranks"]), dtype=torch.float64, device=s["K"].device)
        for b, n in enumerate(_lens(case)):
            for j in range(n // G if B * nb <= 20000 else 0):
                part = s["K"][b, j * G:(j + 1) * G].double().sort(0).values
                ends[0, b, j], ends[1, b, j] = part[0], part[-1]
        return {"lo": ends[0], "hi": ends[1]} if B * nb <= 20000 else None
    lens, dt, slopes = _lens(case), DTYPES[case["dtype"]], _slopes(case)
    dev = s["K"].device
    out = torch.zeros(B, max(1, T), H, g, d, dtype=torch.float64, device=dev)
    rows = [torch.zeros(H, B, T, max(s["ranks"]), dtype=torch.float64, device=dev) for _ in "kv"]
    for b in range(B):
        n = lens[b]
        seen = (s["mask"][b][:, None] >> torch.arange(T, device=dev)).bitwise_and(1).bool() if T else None
        for h in range(H):
            Uk, Uv = s["U_k"][h].double(), s["U_v"][h].double()
            K, V = s["K"][b, :n, h].double(), s["V"][b, :n, h].double()
            place = torch.arange(n, device=dev, dtype=torch.float64)
            if T:
                kn, vn = s["k"][b, :, h].double() @ Uk, s["v"][b, :, h].double() @ Uv
                rows[0][h, b], rows[1][h, b] = kn, vn
                K, V = torch.cat([K, kn.to(dt).double()]), torch.cat([V, vn.to(dt).double()])
                here = n + seen.sum(1).double() - seen.diagonal().double()
                place = torch.cat([place, here])
                open_ = torch.cat([torch.ones(T, n, dtype=torch.bool, device=dev), seen], 1)
            else:
                chosen = _chosen(s, b, h, n, slopes)
                here = torch.full((1,), n - 1.0, device=dev, dtype=torch.float64)
                open_ = torch.zeros(1, n, dtype=torch.bool, device=dev)
                for c in chosen:
                    open_[0, c * case["block"]:(c + 1) * case["block"]] = True
            Q = s["q"][b].view(-1, H, g, d)[:, h].double() @ Uk                                  # [T][g][R]
            for i in range(g):
                x = Q[:, i] @ K.T / math.sqrt(d)
                if slopes:
                    x = x - slopes[h] * (here[:, None] - place)
                x = x.masked_fill(~open_, -math.inf)
                w = torch.exp(x - torch.logsumexp(x, 1, keepdim=True))
                out[b, :, h, i] = (w @ V) @ Uv.T
    out = out.view(B, -1, H * g, d)
    if not T:
        return {"out": out, "index": None}
    if case["op"] == "step":
        for b, path in enumerate(s["paths"]):
            for r in rows:
                r[:, b, :len(path)] = r[:, b, path].clone()
    return {"out": out, "k": rows[0], "v": rows[1]}


def _chosen(s, b, h, n, slopes):
    case = s["case"]
    G, M, g, d = case["block"], case["budget"], case["group"], case["d_head"]
    nb = -(-n // G)
    if nb <= M:
        return list(range(nb))
    Q = s["q"][b, 0].view(-1, g, d)[h].double() @ s["U_k"][h].double()
    mid = s["K"][b, G:(nb - 1) * G, h].double().view(nb - 2, G, -1)
    lo, hi = mid.min(1).values, mid.max(1).values
    top = torch.maximum(Q[:, None] * lo, Q[:, None] * hi).sum(2).max(0).values / math.sqrt(d)
    if slopes:
        top = top - slopes[h] * (n - 1 - (torch.arange(1, nb - 1, device=top.device) * G + G - 1)).double()
    best = sorted(range(nb - 2), key=lambda j, v=top.tolist(): (-v[j], j))[:M - 2]
    return sorted([0] + [j + 1 for j in best] + [nb - 1])
