"""Performance cases of the operators that read a KV cache, through the entry points a program calls:

  attend         attention of one or more new tokens (a single token, a tree of drafted tokens, a chunk of a
                 prompt) over a cache and over themselves
  block_bounds   the smallest and largest key of every block of rows, channel by channel
  select_blocks  the blocks that each query reads, by an upper bound on their attention logits
  attend_blocks  `attend` over the selected blocks alone

A case is a dict of plain values.  `B` holds the batch (layers folded in), `H` the KV heads, `G` the query
heads that share one, `N` the new tokens, `D` the channels and `T` the rows of the cache.  `ragged` gives each
batch entry a length of its own.  `new` says what the tokens see of each other: "none" (only the cache is
read), "chain" (each the ones before it and itself), "tree" (each its ancestors and itself).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _case(name, op, **kw):
    c = dict(name=name, op=op, B=1, H=8, G=4, N=1, D=128, T=0, dtype="bf16", new="none", ragged=False,
             block=0, k=0, first=0, last=0, start=0)
    c.update(kw)
    return c


def listed():
    return [
        # One token over a short fp32 cache (the repository's tiny configuration, compressed): a call's own latency.
        _case("token_tiny_f32", "attend", H=2, G=2, D=64, T=640, dtype="f32", new="chain"),
        # One layer of one request in decode, its 16K prompt compressed to a quarter: few streams.
        _case("token_16k", "attend", T=4288, new="chain"),
        # One layer of 32 requests in decode, compressed from up to 32K, each with a length of its own.
        _case("token_b32", "attend", B=32, T=8384, new="chain", ragged=True),
        # 64 drafted tokens of four requests, verified over caches compressed from 128K.
        _case("tree64_128k", "attend", B=4, N=64, T=33536, new="tree"),
        # A small tree, a head of 80 channels in fp16, seven query heads a KV head, odd lengths.
        _case("tree21_head80_f16", "attend", B=2, H=4, G=7, N=21, D=80, T=2999, dtype="f16", new="tree", ragged=True),
        # A chunk of 512 prompt tokens over what a 64K prompt left of itself: bound by the products.
        _case("chunk512_64k", "attend", N=512, T=8640, new="chain"),
        # Bounds of a whole prompt's keys, one layer of four 128K requests.
        _case("bounds_128k", "block_bounds", B=4, T=131072, block=64),
        # Bounds behind the last 200 rows of a cache in decode, the others being up to date.
        _case("bounds_decode_f32", "block_bounds", B=8, H=4, D=96, T=8384 + 77, dtype="f32", block=32, start=8261),
        # The 64 blocks of 64 rows that one token of each of four 128K requests reads.
        _case("select_128k", "select_blocks", B=4, T=131072, block=64, k=64, first=1, last=4),
        # Blocks of 16 rows for 16 drafted tokens, fp32, six query heads a KV head.
        _case("select_tree16_f32", "select_blocks", B=2, H=4, G=6, N=16, D=96, T=20011, dtype="f32", block=16, k=100,
              first=1, last=2, ragged=True),
        # One token of each of four 128K requests over 4096 of their rows.
        _case("blocks_128k", "attend_blocks", B=4, T=131072, block=64, k=64, new="chain"),
        # 24 drafted tokens, each over 32 blocks of its own, fp16.
        _case("blocks_tree24_f16", "attend_blocks", N=24, T=32768 - 5, dtype="f16", block=32, k=32, new="tree", ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    op = rng.choice(["attend"] * 5 + ["block_bounds", "select_blocks"] + ["attend_blocks"] * 3)
    c = _case("", op, B=_log(rng, 1, 32), H=rng.choice([1, 2, 4, 8]), G=rng.choice([1, 2, 4, 4, 5, 7, 8]),
              D=rng.choice([128, 128, 128, 64, 80, 96, 256, 100]), T=_log(rng, 16, 131072),
              dtype=rng.choice(["bf16", "bf16", "bf16", "f16", "f32"]), ragged=rng.random() < 0.4)
    kind = rng.choice(["token", "token", "tree", "tree", "chunk"])
    c["N"] = 1 if kind == "token" else _log(rng, 2, 64) if kind == "tree" else _log(rng, 16, 512)
    c["new"] = "none" if kind == "token" and rng.random() < 0.3 else "tree" if kind == "tree" else "chain"
    if op != "attend":
        c["block"] = rng.choice([16, 32, 64, 128])
        c["k"] = min(_log(rng, 4, 128), -(-c["T"] // c["block"]))
        c["first"], c["last"] = min(1, c["k"] // 2), min(rng.choice([0, 1, 3]), c["k"] // 2)
        if kind == "chunk":
            c["N"] = _log(rng, 2, 64)
    if op == "block_bounds":
        c.update(N=1, G=1, new="none", ragged=False, start=0 if rng.random() < 0.6 else rng.randrange(c["T"]))
    if op == "select_blocks":
        c["new"] = "none"
    return c


def draw(rng):
    """One more case: the sizes spread over what the listed ones span."""
    most = {o: max(work(x)["bytes"] for x in listed() if x["op"] == o) for o in {x["op"] for x in listed()}}
    flops = max(work(x)["flops"] for x in listed())
    while True:
        c = _draw(rng)
        # the logits, or gathered rows, that the plain forms hold, and the products
        held = c["B"] * c["H"] * c["N"] * (c["k"] * c["block"] * c["D"] if c["op"] == "attend_blocks" else c["G"] * (c["T"] + c["N"]))
        w = work(c)
        if w["bytes"] <= most[c["op"]] and w["flops"] <= flops and held <= 2.8e8:
            del c["name"]
            return c


def _lengths(case):
    B, T = case["B"], case["T"]
    return [T - (b * T) // (2 * B) if case["ragged"] else T for b in range(B)]


def work(case):
    """What one pass cannot do without: each input read once, each output written once."""
    B, H, G, N, D = (case[x] for x in ("B", "H", "G", "N", "D"))
    e = BYTES[case["dtype"]]
    block, k, rows = case["block"], case["k"], sum(_lengths(case))
    if case["op"] == "block_bounds":
        lo = case["start"] // block * block
        return {"bytes": B * H * D * e * ((case["T"] - lo) + 2 * -(-(case["T"] - lo) // block)), "flops": 0}
    if case["op"] == "select_blocks":
        nb = sum(-(-x // block) for x in _lengths(case))
        return {"bytes": H * nb * 2 * D * e + B * H * G * N * D * e + B * H * N * k * 4, "flops": 4 * H * N * D * nb}
    tokens = B * H * N
    new = 0 if case["new"] == "none" else N
    pairs = 0 if new == 0 else B * H * G * (N * (N + 1) // 2 if case["new"] == "chain" else N)
    io = 2 * tokens * G * D * e + tokens * G * 4 + 2 * B * H * new * D * e
    if case["op"] == "attend":
        return {"bytes": io + 2 * H * rows * D * e, "flops": 4 * D * (H * G * N * rows + pairs)}
    picked = sum(min(N * k * block, x) for x in _lengths(case))  # rows that can be shared are read once
    return {"bytes": io + 2 * H * picked * D * e + tokens * k * 4,
            "flops": 4 * D * (G * H * N * sum(min(k * block, x) for x in _lengths(case)) + pairs)}


def prepare(case, seed):
    """A cache as a model leaves it: keys with a scale for each channel and a few strong channels, values with a
    scale for each row; queries, drafted tokens and their tree, lists of blocks."""
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + 17)
    rng = random.Random(seed)
    B, H, G, N, D, T = (case[x] for x in ("B", "H", "G", "N", "D", "T"))
    dt = DTYPES[case["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=g, device=dev, dtype=dtype)

    channel = torch.exp(0.5 * normal(1, H, 1, D, dtype=torch.float32))
    channel[..., torch.randperm(D, generator=g, device=dev)[:max(1, D // 32)]] *= 6.0

    def keys(rows):
        return normal(B, H, rows, D).mul_(channel.to(dt))

    def values(rows):
        return normal(B, H, rows, D).mul_(torch.exp(0.3 * normal(B, H, rows, 1, dtype=torch.float32)).to(dt))

    lengths = torch.tensor(_lengths(case), dtype=torch.int32, device=dev) if case["ragged"] else None
    s = dict(case=dict(case), lengths=lengths, scale=1.0 / math.sqrt(D))
    if case["op"] == "block_bounds":
        s["K"] = keys(T)
        nb = -(-T // case["block"])
        # (what a program has: the bounds of the rows before `start`, up to date, and room for the others)
        s["lo"], s["hi"] = (torch.zeros(B, H, nb, D, dtype=dt, device=dev) for _ in range(2))
        return s
    # queries come from a projection as [B, N, heads, D]
    s["q"] = normal(B, N, H * G, D).transpose(1, 2)
    if case["op"] == "select_blocks":
        K, pad = keys(T), -T % case["block"]
        last = K[:, :, T - 1:]
        K = torch.cat([K, last.expand(B, H, pad, D)], 2).unflatten(2, (-1, case["block"]))
        s["lo"], s["hi"] = K.amin(3), K.amax(3)
        return s
    s["K"], s["V"] = keys(T), values(T)
    s["K_new"] = s["V_new"] = s["parents"] = None
    if case["new"] != "none":
        s["K_new"], s["V_new"] = keys(N), values(N)
    if case["new"] == "tree":
        # each token drafted behind one of the eight before it, or behind the cache
        s["parents"] = torch.tensor([[rng.randrange(max(-1, n - 8), n) for n in range(N)] for _ in range(B)],
                                    dtype=torch.int32, device=dev)
    if case["op"] == "attend_blocks":
        k, lists = case["k"], []
        for x in _lengths(case):
            nb = -(-x // case["block"])
            pick = torch.rand(H, N, nb, generator=g, device=dev).argsort(-1)[..., :min(k, nb)].sort(-1).values
            lists.append(torch.nn.functional.pad(pick, (0, k - pick.shape[-1]), value=-1))
        s["blocks"] = torch.stack(lists).to(torch.int32)
    return s


def _visible(s, N, device):
    """[B or 1, N, N]: which new token (last axis) each new token sees."""
    if s["parents"] is None:
        i = torch.arange(N, device=device)
        return (i[None, :] <= i[:, None])[None]
    parents = s["parents"].long()
    step = torch.nn.functional.one_hot(parents.clamp(min=0), N).float() * (parents >= 0)[..., None]
    # (a token reaches its ancestors in at most N steps, each up the tree or in place)
    return torch.linalg.matrix_power(step + torch.eye(N, device=device), N) > 0


def _softmax(logits, mask):
    """exp(logits - max), their sum and the max over the last axis, of what the mask leaves."""
    logits = logits.masked_fill(~mask, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - top.clamp(min=-1e30))
    return p, p.sum(-1, keepdim=True), top


def _attend_plain(s):
    case, q, K, V = s["case"], s["q"], s["K"].float(), s["V"].float()
    B, H, G, N, D, T = (case[x] for x in ("B", "H", "G", "N", "D", "T"))
    dev, dt = q.device, q.dtype
    qf = q.float().reshape(B, H, G * N, D)
    row = torch.arange(T, device=dev)
    mask = (row[None] < s["lengths"][:, None] if s["lengths"] is not None else torch.ones(1, T, dtype=torch.bool, device=dev))
    mask = mask[:, None, None, None].expand(B, 1, 1, N, T)
    if s["K_new"] is not None:
        K, V = torch.cat([K, s["K_new"].float()], 2), torch.cat([V, s["V_new"].float()], 2)
        mask = torch.cat([mask, _visible(s, N, dev).expand(B, N, N)[:, None, None]], -1)
    logits = (qf @ K.transpose(2, 3) * s["scale"]).unflatten(2, (G, N))
    p, total, top = _softmax(logits, mask)
    out = (p.flatten(2, 3) @ V).unflatten(2, (G, N)) / total.clamp(min=1e-30)
    lse = (top + torch.log(total))[..., 0]
    return out.to(dt).reshape(B, H * G, N, D), lse.reshape(B, H * G, N)


def _attend_blocks_plain(s):
    case, q, blocks = s["case"], s["q"], s["blocks"].long()
    B, H, G, N, D, T = (case[x] for x in ("B", "H", "G", "N", "D", "T"))
    block, k, dev = case["block"], case["k"], q.device
    rows = (blocks[..., None] * block + torch.arange(block, device=dev)).flatten(-2)      # [B,H,N,k*block]
    length = s["lengths"].long()[:, None, None, None] if s["lengths"] is not None else T
    mask = (rows < length) & (blocks >= 0).repeat_interleave(block, -1)
    at = rows.clamp(0, T - 1).reshape(B, H, -1, 1).expand(-1, -1, -1, D)
    K, V = (x.gather(2, at).float().unflatten(2, (N, k * block)) for x in (s["K"], s["V"]))
    mask = mask[:, :, :, None]
    qf = q.float().reshape(B, H, G, N, D).transpose(2, 3)                                   # [B,H,N,G,D]
    logits = qf @ K.transpose(3, 4) * s["scale"]
    mask = mask.expand_as(logits)
    if s["K_new"] is not None:
        fresh = (qf.flatten(2, 3) @ s["K_new"].float().transpose(2, 3) * s["scale"]).unflatten(2, (N, G))
        logits = torch.cat([logits, fresh], -1)
        mask = torch.cat([mask, _visible(s, N, dev).expand(B, N, N)[:, None, :, None].expand_as(fresh)], -1)
    p, total, top = _softmax(logits, mask)
    out = p[..., :k * block] @ V
    if s["K_new"] is not None:
        out = out + (p[..., k * block:].flatten(2, 3) @ s["V_new"].float()).unflatten(2, (N, G))
    out = (out / total.clamp(min=1e-30)).to(q.dtype).transpose(2, 3)
    lse = (top + torch.log(total))[..., 0].transpose(2, 3)
    return out.reshape(B, H * G, N, D), lse.reshape(B, H * G, N)


def _bounds_plain(s):
    case, K = s["case"], s["K"]
    block, T, at = case["block"], case["T"], case["start"] // case["block"]
    K = K[:, :, at * block:]
    whole = K.shape[2] // block * block
    for out, f in ((s["lo"], torch.amin), (s["hi"], torch.amax)):
        if whole:
            out[:, :, at:T // block] = f(K[:, :, :whole].unflatten(2, (-1, block)), 3)
        if whole < K.shape[2]:
            out[:, :, T // block] = f(K[:, :, whole:], 2)
    return s["lo"], s["hi"]


def _select_plain(s):
    # (64 bits: which of two blocks next to the border is taken must not depend on the order of a sum)
    case, dev = s["case"], s["q"].device
    B, H, G, N, D, k, block = (case[x] for x in ("B", "H", "G", "N", "D", "k", "block"))
    q = s["q"].double().reshape(B, H, G, N, D)
    score = q.clamp(min=0).sum(2) @ s["hi"].double().transpose(2, 3) + q.clamp(max=0).sum(2) @ s["lo"].double().transpose(2, 3)
    lengths = s["lengths"].long() if s["lengths"] is not None else torch.full((1,), case["T"], device=dev)
    i, nb = torch.arange(score.shape[-1], device=dev), ((lengths + block - 1) // block)[:, None]
    always = ((i < case["first"]) | (i >= nb - case["last"])) & (i < nb)
    score = score.masked_fill(always[:, None, None], math.inf).masked_fill((i >= nb)[:, None, None], -math.inf)
    top = score.sort(dim=-1, descending=True, stable=True)
    pick = top.indices[..., :k].masked_fill(top.values[..., :k] == -math.inf, score.shape[-1]).sort(-1).values
    return pick.masked_fill(pick == score.shape[-1], -1).to(torch.int32)


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        from paper_2504_04704_amd import lagkv
        if op == "attend":
            a = lagkv.attend(s["q"], s["K"], s["V"], K_new=s["K_new"], V_new=s["V_new"], parents=s["parents"],
                             lengths=s["lengths"], want_lse=True)
            return a.out, a.lse
        if op == "attend_blocks":
            a = lagkv.attend_blocks(s["q"], s["K"], s["V"], s["blocks"], case["block"], K_new=s["K_new"], V_new=s["V_new"],
                                    parents=s["parents"], lengths=s["lengths"], want_lse=True)
            return a.out, a.lse
        if op == "block_bounds":
            return lagkv.block_bounds(s["K"], case["block"], start=case["start"], out=(s["lo"], s["hi"]))
        return lagkv.select_blocks(s["q"], s["lo"], s["hi"], case["T"], case["block"], case["k"], first=case["first"],
                                   last=case["last"], lengths=s["lengths"])
    return {"attend": _attend_plain, "attend_blocks": _attend_blocks_plain, "block_bounds": _bounds_plain,
            "select_blocks": _select_plain}[op](s)


def _ancestors(parents, N):
    """For each new token the tokens that it sees, itself among them."""
    if parents is None:
        return [list(range(n + 1)) for n in range(N)]
    got = []
    for n in range(N):
        path, at = [], n
        while at >= 0:
            path.append(at)
            at = parents[at]
        got.append(sorted(path))
    return got


def exact(case, seed):
    """The definitions in 64 bits, one batch entry at a time."""
    s = prepare(case, seed)
    B, H, G, N, D, T, block = (case[x] for x in ("B", "H", "G", "N", "D", "T", "block"))
    if case["op"] == "block_bounds":
        K, at = s["K"].double(), case["start"] // block
        got = [torch.zeros(B, H, -(-T // block), D, dtype=torch.float64, device=K.device) for _ in range(2)]
        fill = -T % block
        for out, f, edge in ((got[0], torch.amin, math.inf), (got[1], torch.amax, -math.inf)):
            for b in range(B):
                padded = torch.nn.functional.pad(K[b], (0, 0, 0, fill), value=edge)
                out[b, :, at:] = f(padded.reshape(H, -1, block, D), 2)[:, at:]
        return tuple(got)
    lengths = _lengths(case)
    q = s["q"].double()
    if case["op"] == "select_blocks":
        lo, hi, k = s["lo"].double(), s["hi"].double(), case["k"]
        picks = torch.full((B, H, N, k), -1, dtype=torch.int32)
        for b in range(B):
            nb = -(-lengths[b] // block)
            for n in range(N):
                x = q[b, :, n].reshape(H, G, 1, D)
                # of two channels' products the larger one bounds what any row of the block can give
                score = torch.maximum(x * lo[b, :, None, :nb], x * hi[b, :, None, :nb]).sum((1, 3)).cpu()
                for h in range(H):
                    j = np.arange(nb)
                    free = ~((j < case["first"]) | (j >= nb - case["last"]))
                    order = np.sort(np.lexsort((j, -score[h].numpy(), free))[:k])
                    picks[b, h, n, :len(order)] = torch.from_numpy(order)
        return picks.to(q.device)
    out = torch.zeros(B, H * G, N, D, dtype=torch.float64, device=q.device)
    lse = torch.full((B, H * G, N), -math.inf, dtype=torch.float64, device=q.device)
    for b in range(B):
        tree = None if s["parents"] is None else s["parents"][b].tolist()
        sees = None
        if s["K_new"] is not None:
            sees = torch.zeros(N, N, dtype=torch.bool)
            for n, path in enumerate(_ancestors(tree, N)):
                sees[n, path] = True
            sees = sees.to(q.device)
        x = q[b].reshape(H, G, N, D)
        for h in range(H):
            K, V = s["K"][b, h, :lengths[b]].double(), s["V"][b, h, :lengths[b]].double()
            allowed = torch.ones(N, lengths[b], dtype=torch.bool, device=q.device)
            if case["op"] == "attend_blocks":
                of = torch.arange(lengths[b], device=q.device) // block
                allowed = torch.zeros(N, -(-lengths[b] // block) + 1, dtype=torch.bool, device=q.device)
                allowed.scatter_(1, s["blocks"][b, h].long().clamp(min=-1) % allowed.shape[1], True)
                allowed = allowed[:, of]
            if sees is not None:
                K, V = torch.cat([K, s["K_new"][b, h].double()]), torch.cat([V, s["V_new"][b, h].double()])
                allowed = torch.cat([allowed, sees], 1)
            logits = torch.where(allowed[None], torch.matmul(x[h], K.T.contiguous()) / math.sqrt(D), -math.inf)
            total = torch.logsumexp(logits, -1)
            lse[b, h * G:(h + 1) * G] = total
            out[b, h * G:(h + 1) * G] = torch.matmul(torch.exp(logits - total[..., None]), V)
    return out, lse
