"""Plain 64-bit forms of the operators that read a cache, and how far a kernel may be from them."""
import math

import torch

F64 = torch.float64


def tree_visible(parents, N):
    """[N, N] bool: which new tokens token n sees; a value that is no earlier token and not -1 is no token."""
    see = torch.zeros(N, N, dtype=torch.bool)
    for n in range(N):
        at = n
        while at >= 0:
            up = int(parents[at])
            if up < -1 or up >= at:
                break
            see[n, at] = True
            at = up
    return see


def attend(q, K, V, K_new=None, V_new=None, parents=None, lengths=None, scale=None, blocks=None, block=0):
    """out, lse and the bound on |kernel - out| in 64 bits, on the CPU."""
    dt = q.dtype
    q, K, V = (x.detach().cpu().to(F64) for x in (q, K, V))
    B, H, T, D = K.shape
    Hq, N = q.shape[1], q.shape[2]
    G = Hq // H
    scale = 1 / math.sqrt(D) if scale is None else scale
    if K_new is not None:
        K_new, V_new = K_new.detach().cpu().to(F64), V_new.detach().cpu().to(F64)
    u = torch.finfo(dt).eps / 2
    out = torch.zeros(B, Hq, N, D, dtype=F64)
    lse = torch.full((B, Hq, N), -math.inf, dtype=F64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        n_rows = T if lengths is None else min(max(int(lengths[b]), 0), T)
        par = None if parents is None else (parents[b] if parents.dim() == 2 else parents).cpu()
        see = None
        if K_new is not None:
            see = tree_visible(par, N) if par is not None else torch.ones(N, N).tril().bool()
        for hq in range(Hq):
            h = hq // G
            for n in range(N):
                if par is not None and (int(par[n]) < -1 or int(par[n]) >= n):
                    continue
                if blocks is None:
                    rows = torch.arange(n_rows)
                else:
                    nb = -(-n_rows // block)
                    rows = [torch.arange(j * block, min((j + 1) * block, n_rows)) for j in blocks[b, h, n].tolist() if 0 <= j < nb]
                    rows = torch.cat(rows) if rows else torch.arange(0)
                k, v = K[b, h][rows], V[b, h][rows]
                if see is not None:
                    k, v = torch.cat([k, K_new[b, h][see[n]]]), torch.cat([v, V_new[b, h][see[n]]])
                if k.shape[0] == 0:
                    continue
                x = (k @ q[b, hq, n]) * scale
                top = x.max()
                e = torch.exp(x - top)
                p = e / e.sum()
                out[b, hq, n] = p @ v
                lse[b, hq, n] = top + torch.log(e.sum())
                # A logit is a sum of D products in fp32, each step off by up to 2^-23 of what is summed, times scale and
                # in units of its distance from the maximum; an error d of the logits moves every weight by 2d at most,
                # the sums over the rows by one rounding each.  The weights are put in as two numbers of the type, or as
                # one (u); the output is rounded once (u).
                d = (abs(k) @ abs(q[b, hq, n])).max() * abs(scale) * (D + 4) * 2.0 ** -23 + abs(x).max() * 2.0 ** -21
                s = (len(x) + 64) * 2.0 ** -24
                tol[b, hq, n] = u * abs(out[b, hq, n]) + (u * 1.01 + 2 * d + 2 * s) * (p @ abs(v)) + torch.finfo(dt).tiny
                tol_lse[b, hq, n] = d + s + 2.0 ** -23 * (abs(lse[b, hq, n]) + 1)
    return out, lse, tol, tol_lse


def check(got, want, where=""):
    out, lse, tol, tol_lse = want
    g = got.out.detach().cpu().to(F64)
    assert g.shape == out.shape
    assert bool(torch.isfinite(g).all()), where
    off = abs(g - out)
    assert bool((off <= tol).all()), f"{where}: {float((off - tol).max()):.3e} over, off {float(off.max()):.3e}"
    if got.lse is not None:
        gl = got.lse.cpu().to(F64)
        seen = torch.isfinite(lse)
        assert torch.equal(torch.isfinite(gl), seen) and bool((gl[~seen] == -math.inf).all()), where
        assert bool((abs(gl - lse)[seen] <= tol_lse[seen]).all()), f"{where}: lse off {float(abs(gl - lse)[seen].max()):.3e}"


def bounds(K, block, lengths=None):
    B, H, T, D = K.shape
    nb = -(-T // block)
    lo, hi = torch.full((B, H, nb, D), math.inf, dtype=K.dtype), torch.full((B, H, nb, D), -math.inf, dtype=K.dtype)
    K = K.cpu()
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        for j in range(-(-n // block)):
            rows = K[b, :, j * block:min((j + 1) * block, n)]
            lo[b, :, j], hi[b, :, j] = rows.amin(1), rows.amax(1)
    return lo, hi


def select(q, lo, hi, T, block, k, first=0, last=0, lengths=None):
    q, lo, hi = (x.cpu().to(F64) for x in (q, lo, hi))
    B, H, _, D = lo.shape
    G, N = q.shape[1] // H, q.shape[2]
    got = torch.full((B, H, N, k), -1, dtype=torch.int32)
    for b in range(B):
        n_rows = T if lengths is None else min(max(int(lengths[b]), 0), T)
        nb = -(-n_rows // block)
        for h in range(H):
            for n in range(N):
                x = q[b, h * G:(h + 1) * G, n][:, None]
                s = torch.maximum(x * lo[b, h, None, :nb], x * hi[b, h, None, :nb]).sum((0, 2)).tolist()
                order = sorted(range(nb), key=lambda j: (not (j < first or j >= nb - last), -s[j], j))[:k]
                got[b, h, n, :len(order)] = torch.tensor(sorted(order), dtype=torch.int32)
    return got
