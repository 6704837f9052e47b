"""Performance cases of a KV cache held in 8 bits, through the entry points a program calls:

  quantize          rows as 8-bit codes (int8, or floating point with 4 exponent and 3 mantissa bits) with one scale for
                    every block of rows and head, as the cache is written
  dequantize        the rows back in 16 or 32 bits
  attend_quantized  attention of one or more new tokens over such a cache, over rows behind it that are not quantised
                    yet (a tail), and over themselves

A case is a dict of plain values.  `B` holds the batch (layers folded in), `H` the KV heads, `G` the query heads that
share one, `N` the new tokens, `D` the channels, `T` the rows in 8 bits, `R` those of the tail, `block` the rows of a
scale.  `ragged` gives each batch entry lengths of its own.  `new` says what the tokens see of each other: "none" (only
the cache is read), "chain" (each the ones before it and itself), "tree" (each its ancestors and itself).
"""
from __future__ import annotations

import math
import random

import torch

own = False
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def _case(name, op, **kw):
    c = dict(name=name, op=op, B=1, H=8, G=1, N=0, D=128, T=0, R=0, dtype="bf16", code="int8", block=64, new="none",
             ragged=False, start=0)
    c.update(kw)
    return c


def listed():
    return [
        # The last block of a request's cache, one layer, behind appended rows: a call's own latency.
        _case("write_block", "quantize", T=4288, start=4224),
        # All layers of a 128K request, compressed to a quarter: the cache is written once after its prompt.
        _case("write_128k", "quantize", B=32, T=33536),
        # A ragged batch of fp16 heads of 100 channels, in blocks of 32 rows, as floating-point codes.
        _case("write_head100_f16", "quantize", B=6, H=4, T=20011, D=100, dtype="f16", code="e4m3", block=32, ragged=True),
        # fp32 rows behind the first half, blocks of 128.
        _case("write_half_f32", "quantize", B=8, H=4, T=8461, D=96, dtype="f32", block=128, start=4261),
        # One layer of four 128K requests read back, for a program that needs the rows themselves.
        _case("read_128k", "dequantize", B=4, T=33536),
        # A small ragged read, heads of 80 channels, fp32.
        _case("read_head80_f32", "dequantize", B=3, H=2, T=1503, D=80, dtype="f32", code="e4m3", block=16, ragged=True, start=200),
        # One token over a short fp32 cache: a call's own latency.
        _case("token_tiny_f32", "attend_quantized", H=2, G=2, N=1, D=64, T=512, R=128, dtype="f32", new="chain"),
        # One layer of one request in decode, its 16K prompt compressed to a quarter, the last rows not quantised yet.
        _case("token_16k", "attend_quantized", G=4, N=1, T=4032, R=256, new="chain"),
        # One layer of 32 requests in decode, each with a length of its own.
        _case("token_b32", "attend_quantized", B=32, G=4, N=1, T=8128, R=256, new="chain", ragged=True),
        # 64 drafted tokens of four requests, over caches compressed from 128K.
        _case("tree64_128k", "attend_quantized", B=4, G=4, N=64, T=33280, R=256, code="e4m3", new="tree"),
        # A small tree, seven query heads of 80 channels in fp16, odd lengths.
        _case("tree21_head80_f16", "attend_quantized", B=2, H=4, G=7, N=21, D=80, T=2999, R=77, dtype="f16", code="e4m3",
              block=32, new="tree", ragged=True),
        # A chunk of 512 prompt tokens over what a 64K prompt left of itself: bound by the products.
        _case("chunk512_64k", "attend_quantized", G=4, N=512, T=8448, R=192, new="chain"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    op = rng.choice(["quantize"] * 2 + ["dequantize"] + ["attend_quantized"] * 4)
    c = _case("", op, B=_log(rng, 1, 32), H=rng.choice([1, 2, 4, 8]), D=rng.choice([128, 128, 128, 64, 80, 96, 256, 100]),
              T=_log(rng, 16, 65536), dtype=rng.choice(["bf16", "bf16", "bf16", "f16", "f32"]), code=rng.choice(["int8", "int8", "e4m3"]),
              block=rng.choice([16, 32, 64, 64, 128]), ragged=rng.random() < 0.4)
    if op == "attend_quantized":
        kind = rng.choice(["token", "token", "tree", "tree", "chunk"])
        c["G"] = rng.choice([1, 2, 4, 4, 5, 7, 8])
        c["N"] = 1 if kind == "token" else _log(rng, 2, 64) if kind == "tree" else _log(rng, 16, 512)
        c["new"] = "none" if kind == "token" and rng.random() < 0.3 else "tree" if kind == "tree" else "chain"
        c["R"] = 0 if rng.random() < 0.2 else _log(rng, 1, 2048)
    else:
        c["start"] = 0 if rng.random() < 0.6 else rng.randrange(c["T"])
    return c


def draw(rng):
    """One more case: the sizes spread over what the listed ones span."""
    most = {o: max(work(x)["bytes"] for x in listed() if x["op"] == o) for o in {x["op"] for x in listed()}}
    flops = max(work(x)["flops"] for x in listed())
    while True:
        c = _draw(rng)
        w = work(c)
        # (the last: the logits that the plain form holds)
        if 0 < w["bytes"] <= most[c["op"]] and w["flops"] <= flops and c["B"] * c["H"] * c["G"] * c["N"] * (c["T"] + c["R"] + c["N"]) <= 2.8e8:
            del c["name"]
            return c


def _lengths(case, rows):
    B = case["B"]
    return [rows - (b * rows) // (2 * B) if case["ragged"] else rows for b in range(B)]


def work(case):
    """What one pass cannot do without: each input read once, each output written once."""
    B, H, G, N, D, T, block = (case[x] for x in ("B", "H", "G", "N", "D", "T", "block"))
    e, start = BYTES[case["dtype"]], case["start"]
    lengths, tail = _lengths(case, T), sum(_lengths(case, case["R"]))
    if case["op"] != "attend_quantized":
        at = start // block * block if case["op"] == "quantize" else start
        rows = sum(max(0, x - at) for x in lengths)
        blocks = sum(max(0, -(-x // block) - at // block) for x in lengths)
        return {"bytes": 2 * H * (rows * D * (e + 1) + blocks * 4), "flops": 0}
    rows, blocks = sum(lengths), sum(-(-x // block) for x in lengths)
    new = 0 if case["new"] == "none" else N
    pairs = 0 if new == 0 else B * H * G * (N * (N + 1) // 2 if case["new"] == "chain" else N)
    io = 2 * B * H * G * N * D * e + B * H * G * N * 4 + 2 * B * H * new * D * e
    return {"bytes": io + 2 * H * (rows * D + blocks * 4 + tail * D * e), "flops": 4 * D * (H * G * N * (rows + tail) + pairs)}


def _scaled(x, case):
    """x as codes of the case's kind with a scale for each block of rows, for what prepare() has in hand."""
    B, H, T, D = x.shape
    block = case["block"]
    x = torch.nn.functional.pad(x, (0, 0, 0, -T % block)).unflatten(2, (-1, block)).float()
    most = 127.0 if case["code"] == "int8" else 448.0
    scale = x.abs().amax((3, 4)) / most
    x = (x / scale[..., None, None]).flatten(2, 3)[:, :, :T]
    return (x.round() if case["code"] == "int8" else x.clamp(-448, 448)).to(CODES[case["code"]]), scale


def prepare(case, seed):
    """Rows as a model leaves them: keys with a scale for each channel and a few strong channels, values with a scale for
    each row; queries, drafted tokens and their tree; the cache in 8 bits, or room for it."""
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + 29)
    rng = random.Random(seed)
    B, H, G, N, D, T, R, block = (case[x] for x in ("B", "H", "G", "N", "D", "T", "R", "block"))
    dt = DTYPES[case["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=g, device=dev, dtype=dtype)

    channel = torch.exp(0.5 * normal(1, H, 1, D, dtype=torch.float32))
    channel[..., torch.randperm(D, generator=g, device=dev)[:max(1, D // 32)]] *= 6.0

    def keys(rows):
        return normal(B, H, rows, D).mul_(channel.to(dt))

    def values(rows):
        return normal(B, H, rows, D).mul_(torch.exp(0.3 * normal(B, H, rows, 1, dtype=torch.float32)).to(dt))

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev) if case["ragged"] else None

    s = dict(case=dict(case), lengths=ints(_lengths(case, T)), scale=1.0 / math.sqrt(D))
    s["K"], s["V"] = keys(T), values(T)
    if case["op"] == "quantize":
        for x in ("K", "V"):
            s[x + "q"] = torch.zeros(B, H, T, D, dtype=torch.int8, device=dev).view(CODES[case["code"]])
            s[x + "s"] = torch.zeros(B, H, -(-T // block), dtype=torch.float32, device=dev)
        return s
    for x in ("K", "V"):
        s[x + "q"], s[x + "s"] = _scaled(s[x], case)
    if case["op"] == "dequantize":
        s["K"], s["V"] = s["K"].zero_(), s["V"].zero_()
        return s
    del s["K"], s["V"]
    # queries come from a projection as [B, N, heads, D]
    s["q"] = normal(B, N, H * G, D).transpose(1, 2)
    s["K_tail"], s["V_tail"] = (keys(R), values(R)) if R else (None, None)
    s["tail_lengths"] = ints(_lengths(case, R)) if R else None
    s["K_new"], s["V_new"] = (keys(N), values(N)) if case["new"] != "none" else (None, None)
    s["parents"] = None
    if case["new"] == "tree":
        # each token drafted behind one of the eight before it, or behind the cache
        s["parents"] = torch.tensor([[rng.randrange(max(-1, n - 8), n) for n in range(N)] for _ in range(B)],
                                    dtype=torch.int32, device=dev)
    return s


def _block_rows(case, lengths, at, device):
    """[B or 1, blocks, block]: rows that are there, of the blocks from the one `at` on."""
    i = torch.arange(at * case["block"], -(-case["T"] // case["block"]) * case["block"], device=device)
    n = lengths.long()[:, None] if lengths is not None else torch.full((1, 1), case["T"], device=device)
    return (i[None] < n).unflatten(1, (-1, case["block"]))


def _quantize_plain(s):
    case = s["case"]
    block, T, at = case["block"], case["T"], case["start"] // case["block"]
    for x in ("K", "V"):
        rows, codes, scales = s[x][:, :, at * block:], s[x + "q"][:, :, at * block:], s[x + "s"][:, :, at:]
        there = _block_rows(case, s["lengths"], at, rows.device)
        y = torch.nn.functional.pad(rows, (0, 0, 0, -T % block)).unflatten(2, (-1, block)).float()
        y = torch.where(there[:, None, ..., None], y, 0.0)
        most = y.abs().amax((3, 4))
        fine = torch.isfinite(most)
        use = torch.where(fine & (most > 0), most, 1.0)[..., None, None]
        if case["code"] == "int8":
            scale = most / 127.0
            # (64 bits: which of two codes next to the border is taken must not depend on how the quotient is rounded)
            y = ((y.double() * 127.0) / use.double()).round()
        else:
            m, e = torch.frexp(use)
            e = torch.clamp(e - 8 - (m <= 0.875).int(), min=-126)
            scale = torch.where(most > 0, ((e + 127) << 23).view(torch.float32)[..., 0, 0], 0.0)
            y = y * ((127 - e) << 23).view(torch.float32)
        scale = torch.where(fine, scale, math.nan)
        y = torch.where(fine[..., None, None], y, 0.0).flatten(2, 3)[:, :, :rows.shape[2]].to(codes.dtype)
        there = there.flatten(1)[:, None, :rows.shape[2], None]
        codes.copy_(torch.where(there, y.view(torch.int8), codes.view(torch.int8)).view(codes.dtype))
        scales.copy_(torch.where(there[:, :, ::block, 0], scale, scales))
    return s["Kq"], s["Vq"], s["Ks"], s["Vs"]


def _values(s, x, first=0):
    """The rows from `first` on that the codes of x stand for, in 32 bits."""
    codes, scale = s[x + "q"][:, :, first:], s[x + "s"]
    row = torch.arange(first, first + codes.shape[2], device=codes.device) // s["case"]["block"]
    return codes.float() * scale[:, :, row, None]


def _dequantize_plain(s):
    case = s["case"]
    i = torch.arange(case["start"], case["T"], device=s["K"].device)
    for x in ("K", "V"):
        y, out = _values(s, x, case["start"]).to(s[x].dtype), s[x][:, :, case["start"]:]
        if s["lengths"] is not None:
            y = torch.where((i[None] < s["lengths"][:, None])[:, None, :, None], y, out)
        out.copy_(y)
    return s["K"], s["V"]


def _visible(s, N, device):
    """[B or 1, N, N]: which new token (last axis) each new token sees."""
    if s["parents"] is None:
        i = torch.arange(N, device=device)
        return (i[None, :] <= i[:, None])[None]
    parents = s["parents"].long()
    step = torch.nn.functional.one_hot(parents.clamp(min=0), N).float() * (parents >= 0)[..., None]
    # (a token reaches its ancestors in at most N steps, each up the tree or in place)
    return torch.linalg.matrix_power(step + torch.eye(N, device=device), N) > 0


def _attend_plain(s):
    case, q = s["case"], s["q"]
    B, H, G, N, D = (case[x] for x in ("B", "H", "G", "N", "D"))
    dev = q.device

    def held(rows, lengths):
        i = torch.arange(rows, device=dev)
        m = i[None] < lengths[:, None] if lengths is not None else torch.ones(1, rows, dtype=torch.bool, device=dev)
        return m[:, None, None, None].expand(B, 1, 1, N, rows)

    K, V, mask = [_values(s, "K")], [_values(s, "V")], [held(case["T"], s["lengths"])]
    if s["K_tail"] is not None:
        K, V, mask = K + [s["K_tail"].float()], V + [s["V_tail"].float()], mask + [held(case["R"], s["tail_lengths"])]
    if s["K_new"] is not None:
        K, V, mask = K + [s["K_new"].float()], V + [s["V_new"].float()], mask + [_visible(s, N, dev).expand(B, N, N)[:, None, None]]
    K, V, mask = torch.cat(K, 2), torch.cat(V, 2), torch.cat(mask, -1)
    logits = (q.float().reshape(B, H, G * N, D) @ K.transpose(2, 3) * s["scale"]).unflatten(2, (G, N))
    logits = logits.masked_fill(~mask, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - top.clamp(min=-1e30))
    total = p.sum(-1, keepdim=True)
    out = (p.flatten(2, 3) @ V).unflatten(2, (G, N)) / total.clamp(min=1e-30)
    lse = (top + torch.log(total))[..., 0]
    return out.to(q.dtype).reshape(B, H * G, N, D), lse.reshape(B, H * G, N)


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        from paper_2504_04704_amd import lagkv
        x = lagkv.Quantized(s["Kq"], s["Vq"], s["Ks"], s["Vs"], case["block"])
        if op == "quantize":
            lagkv.quantize(s["K"], s["V"], case["block"], lengths=s["lengths"], start=case["start"], out=x)
            return x.K, x.V, x.K_scale, x.V_scale
        if op == "dequantize":
            return lagkv.dequantize(x, lengths=s["lengths"], start=case["start"], out=(s["K"], s["V"]))
        a = lagkv.attend_quantized(s["q"], x, s["K_tail"], s["V_tail"], s["K_new"], s["V_new"], s["parents"], lengths=s["lengths"],
                                   tail_lengths=s["tail_lengths"], want_lse=True)
        return a.out, a.lse
    return {"quantize": _quantize_plain, "dequantize": _dequantize_plain, "attend_quantized": _attend_plain}[op](s)


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


def _nearest_e4m3(x):
    """The nearest number with 4 exponent and 3 mantissa bits, of two the one whose last bit is 0."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    # (log2 next to a power of two may be off by its last bit)
    e = torch.where(torch.exp2(e + 1) <= x.abs(), e + 1, torch.where(torch.exp2(e) > x.abs().clamp(min=2.0 ** -6), e - 1, e))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    """The definitions in 64 bits, one batch entry at a time."""
    s = prepare(case, seed)
    B, H, G, N, D, T, R, block, start = (case[x] for x in ("B", "H", "G", "N", "D", "T", "R", "block", "start"))
    lengths, dev = _lengths(case, T), s["Kq"].device
    f64 = torch.float64
    if case["op"] == "quantize":
        if B * H * T * D > 1.5e9:
            return None
        at, nb = start // block, -(-T // block)
        codes, scales = [], []
        for x in ("K", "V"):
            c, f = torch.zeros(B, H, T, D, dtype=f64 if case["code"] != "int8" else torch.int8, device=dev), torch.zeros(B, H, nb, dtype=f64, device=dev)
            for b in range(B):
                n = lengths[b]
                if n <= at * block:
                    continue
                y = s[x][b, :, at * block:n].double()
                end = -(-n // block)
                most = torch.nn.functional.pad(y, (0, 0, 0, -n % block)).reshape(H, end - at, block * D).abs().amax(2)
                if case["code"] == "int8":
                    f[b, :, at:end] = most / 127
                    each = most.repeat_interleave(block, 1)[:, :y.shape[1], None]
                    c[b, :, at * block:n] = torch.round(127 * y / each).to(torch.int8)
                else:
                    e = torch.ceil(torch.log2(most / 448))
                    e = torch.where(448 * torch.exp2(e - 1) >= most, e - 1, torch.where(448 * torch.exp2(e) < most, e + 1, e))
                    f[b, :, at:end] = torch.exp2(e)
                    each = torch.exp2(e).repeat_interleave(block, 1)[:, :y.shape[1], None]
                    c[b, :, at * block:n] = _nearest_e4m3(y / each)
            codes.append(c)
            scales.append(f)
        return (*codes, *scales)
    if case["op"] == "dequantize":
        got = []
        for x in ("K", "V"):
            y = torch.zeros(B, H, T, D, dtype=f64, device=dev)
            for b in range(B):
                n = lengths[b]
                each = s[x + "s"][b].double().repeat_interleave(block, 1)[:, start:max(n, start), None]
                y[b, :, start:max(n, start)] = s[x + "q"][b, :, start:max(n, start)].float().double() * each
            got.append(y)
        return tuple(got)
    tails = _lengths(case, R)
    out = torch.zeros(B, H * G, N, D, dtype=f64, device=dev)
    lse = torch.full((B, H * G, N), -math.inf, dtype=f64, device=dev)
    for b in range(B):
        allowed = torch.ones(N, lengths[b] + tails[b], dtype=torch.bool)
        if s["K_new"] is not None:
            sees = torch.zeros(N, N, dtype=torch.bool)
            for n, path in enumerate(_ancestors(None if s["parents"] is None else s["parents"][b].tolist(), N)):
                sees[n, path] = True
            allowed = torch.cat([allowed, sees], 1)
        allowed = allowed.to(dev)
        for h in range(H):
            rows = []
            for x in ("K", "V"):
                each = s[x + "s"][b, h].double().repeat_interleave(block)[:lengths[b], None]
                y = [s[x + "q"][b, h, :lengths[b]].float().double() * each]
                if R:
                    y.append(s[x + "_tail"][b, h, :tails[b]].double())
                if s["K_new"] is not None:
                    y.append(s[x + "_new"][b, h].double())
                rows.append(torch.cat(y))
            for i in range(h * G, (h + 1) * G):
                logits = torch.matmul(s["q"][b, i].double(), rows[0].T.contiguous()) / math.sqrt(D)
                logits = torch.where(allowed, logits, -math.inf)
                lse[b, i] = torch.logsumexp(logits, -1)
                out[b, i] = torch.matmul(torch.exp(logits - lse[b, i, :, None]), rows[1])
    return out, lse
