"""Plain 64-bit forms of the operators of a cache in 8 bits, and how far a kernel may be from them."""
import math

import torch

import attend_util as A

F64 = torch.float64
E4M3 = torch.float8_e4m3fn


def nearest_e4m3(x):
    """Of the numbers with 4 exponent (bias 7) and 3 mantissa bits the nearest to each x, of two the even one."""
    small, rest = [m * 2.0 ** -9 for m in range(8)], [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)]
    grid = torch.tensor((small + rest)[:-1], dtype=F64)  # (the last would be 480: no number)
    a = x.abs().clamp(max=448.0)
    hi = torch.searchsorted(grid, a).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - a, a - grid[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.copysign(grid[pick], x)


def quantize(K, block, code, lengths=None):
    """Codes (64 bits) and scales of rows [B,H,T,D]; NaN for codes and scales that are not written."""
    K = K.detach().cpu()
    B, H, T, D = K.shape
    nb = -(-T // block)
    codes, scales = torch.full((B, H, T, D), math.nan, dtype=F64), torch.full((B, H, nb), math.nan, dtype=F64)
    written = torch.zeros(B, H, T, dtype=torch.bool)
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        for h in range(H):
            for j in range(-(-n // block)):
                at = slice(j * block, min((j + 1) * block, n))
                x = K[b, h, at].to(F64)
                a = float(x.abs().max())
                written[b, h, at] = True
                if not math.isfinite(a):
                    codes[b, h, at], scales[b, h, j] = 0, math.nan
                elif a == 0:
                    codes[b, h, at], scales[b, h, j] = 0, 0
                elif code == torch.int8:
                    codes[b, h, at] = torch.round(127 * x / a)  # (to even)
                    scales[b, h, j] = float(torch.tensor(a, dtype=torch.float32) / torch.tensor(127.0, dtype=torch.float32))
                else:
                    e = -126
                    while a > 448 * 2.0 ** e:
                        e += 1
                    codes[b, h, at], scales[b, h, j] = nearest_e4m3(x / 2.0 ** e), 2.0 ** e
    return codes, scales, written


def values(codes, scale, block):
    """Rows [B,H,T,D] in 64 bits."""
    T = codes.shape[2]
    s = scale.detach().cpu().to(F64).repeat_interleave(block, 2)[:, :, :T, None]
    return codes.detach().cpu().float().to(F64) * s


def attend(q, x, K_tail=None, V_tail=None, K_new=None, V_new=None, parents=None, lengths=None, tail_lengths=None, scale=None):
    """out, lse and their bounds: attend_util's of the rows that the codes stand for with the tail behind them, and what the operands
    of the products add to its bounds."""
    K, V = values(x.K, x.K_scale, x.block), values(x.V, x.V_scale, x.block)
    B, H, T, D = K.shape
    parts = []
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        k, v = K[b:b + 1, :, :n], V[b:b + 1, :, :n]
        # Errors of the operands: the elements of q by c of the row's largest (the logits by its products with the rows' sums), and weights
        # as two numbers of 11 bits, the second rounded: 2^-22 of each, and half of binary16's smallest, times 2^-14 and the
        # largest scale's power of two, that is 2^-38 of the largest value for each row.
        c = {torch.float16: 0.0, torch.bfloat16: 2.0 ** -25, torch.float32: 2.0 ** -23}[q.dtype]
        most_k = float(k.abs().sum(-1).max()) if n else 0.0
        most_v = float(v.abs().max()) if n else 0.0
        if K_tail is not None:
            R = K_tail.shape[2]
            r = R if tail_lengths is None else min(max(int(tail_lengths[b]), 0), R)
            k = torch.cat([k, K_tail[b:b + 1, :, :r].detach().cpu().to(F64)], 2)
            v = torch.cat([v, V_tail[b:b + 1, :, :r].detach().cpu().to(F64)], 2)
        at = lambda t: None if t is None else t[b:b + 1]  # noqa: E731
        par = parents if parents is None or parents.dim() == 1 else parents[b:b + 1]
        out, lse, tol, tol_lse = A.attend(q[b:b + 1], k, v, at(K_new), at(V_new), par, scale=scale)
        s = 1 / math.sqrt(D) if scale is None else abs(scale)
        d = c * q[b].detach().cpu().to(F64).abs().amax(-1) * most_k * s           # [Hq, N]
        top = max([float(t.abs().max()) for t in (v, at(V_new)) if t is not None and t.numel()] or [0.0])
        tol = tol + ((2 * d[None, ..., None] + 2.0 ** -22) * top + n * 2.0 ** -38 * most_v)
        parts.append((out, lse, tol, tol_lse + 2 * d[None]))
    return tuple(torch.cat(p) for p in zip(*parts))
