"""Attention in 64 bits with a bound on what the kernels' roundings may do to every element.  No arithmetic of the library here."""
import math

import numpy as np
import torch


def attend(q, k, v, limit, fp16):
    """q [rows][H][hd], k, v [keys][Hkv][hd] (any type), row r sees the keys up to limit[r].  Returns (out, bound), [rows][H * hd]
    in fp64.

    The bound, with p the probabilities, A = sum p |v| / sum p and n the number of keys:
      scores    hd products of exact factors summed in fp32, then scaled: off by at most hd 2^-24 sum |q||k| / sqrt(hd) + 2^-22 |s|;
                a relative error of a probability, so at most twice that times A in the quotient; exp2 itself: 2^-22;
      sums      n fp32 additions, their rescalings and the quotient: (n + 64) 2^-23 A for numerator and denominator together;
      fp16 only a probability is off by half a step, 2^-11 of it, or by 2^-25 where it is subnormal (the largest one is at least 1):
                2 2^-11 A + 2 n 2^-25 max|v|;  the result by 2^-11 |o| + 2^-25."""
    rows, H, hd = q.shape
    n, hk = k.shape[0], k.shape[1]
    G = H // hk
    q, k, v = q.double(), k.double(), v.double()
    out = torch.empty((rows, H, hd), dtype=torch.float64, device=q.device)
    bound = torch.empty_like(out)
    key = torch.arange(n, device=q.device)
    step = max(1, (1 << 24) // max(1, n))
    for h in range(H):
        kh, vh = k[:, h // G], v[:, h // G]
        for r in range(0, rows, step):
            x = q[r:r + step, h]
            hidden = key[None, :] > limit[r:r + step, None]
            s = (x @ kh.t().contiguous()) / math.sqrt(hd)
            mag = (x.abs() @ kh.abs().t().contiguous()) / math.sqrt(hd)
            err = hd * 2.0 ** -24 * mag + 2.0 ** -22 * s.abs()
            err = err.masked_fill(hidden, 0).amax(dim=1, keepdim=True) + 2.0 ** -22
            p = torch.softmax(s.masked_fill(hidden, -math.inf), dim=1)
            clean = torch.where(torch.isfinite(vh), vh, 0.0)
            o, A = p @ clean, p @ clean.abs()
            b = (2 * err + (n + 64) * 2.0 ** -23) * A
            if fp16:
                b += 2 * 2.0 ** -11 * A + 2 * n * 2.0 ** -25 * clean.abs().max() + 2.0 ** -11 * o.abs() + 2.0 ** -25
            else:
                b += 2.0 ** -24 * o.abs()
            out[r:r + step, h], bound[r:r + step, h] = o, b
    return out.reshape(rows, -1), bound.reshape(rows, -1)


def check(got, want, bound):
    got = got.double()
    assert torch.isfinite(got).all()
    over = (got - want).abs() - bound
    worst = int(over.argmax())
    assert over.max() <= 0, "row %d column %d: %g instead of %g, off by more than %g" % (
        worst // got.shape[1], worst % got.shape[1], got.flatten()[worst], want.flatten()[worst], bound.flatten()[worst])


def ties(q, k, v, limit):
    """Scores so far apart that a row's weight is all on the keys that attain its largest, in equal shares (or, with a query of zeros, on
    all).  Equal keys give equal scores whatever the roundings, every other probability is 0: what is left are the sums and the
    quotient, and the rounding of the result."""
    rows, H, hd = q.shape
    G = H // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, bound = [], []
    for h in range(H):
        s = (q[:, h] @ k[:, h // G].t().contiguous()) / math.sqrt(hd)
        s = s.masked_fill(torch.arange(len(k), device=q.device)[None, :] > limit[:, None], -math.inf)
        top = s.amax(dim=1, keepdim=True)
        assert ((s == top) | (top - s > 64)).all()
        p = (s == top).double()
        p /= p.sum(dim=1, keepdim=True)
        out.append(p @ v[:, h // G])
        bound.append((len(k) + 64) * 2.0 ** -23 * (p @ v[:, h // G].abs()))
    return torch.stack(out, 1).reshape(rows, -1), torch.stack(bound, 1).reshape(rows, -1)


def levels(n, shape, seed):
    g = np.random.default_rng(seed)
    x = g.integers(1, 9, n)
    return torch.tensor(np.sort(x) if shape == "rising" else np.sort(x)[::-1].copy() if shape == "falling" else x, device="cuda")


def factors(n, kind, seed):
    """One factor per row: the largest that the type's scores stand, ordinary ones, none, and negative ones."""
    far = 65504.0 if kind == "f16" else 2.0 ** 53
    return torch.tensor(np.random.default_rng(seed).choice([far, -far, far / 16, 8.0, -2.0, 0.0], n), device="cuda")
