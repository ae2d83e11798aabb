"""The paged key/value cache, its attention and the verification of drafts from their definitions, in 64 bits on the CPU: what
the GPU tests of siso_kv.h compare with.  Shares no code with the library."""

import math

import numpy as np
import torch


def held(x: torch.Tensor, dtype: str) -> torch.Tensor:
    """The values that the cache holds for bfloat16 vectors (last axis), as float64.  8 bits: the scale and the quotient are
    numbers of 32 bits by definition (a quotient of two such numbers formed in 64 bits and rounded is the correctly rounded one)."""
    x = x.double().cpu()
    if dtype == "bf16":
        return x
    fine = torch.isfinite(x).all(-1, keepdim=True)
    y = torch.where(fine, x, torch.zeros_like(x))
    s = (y.abs().amax(-1, keepdim=True) / 448.0).float().double()
    quotient = torch.where(s > 0, y / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(y)).float().double()
    a = quotient.abs()
    exponent = torch.clamp(torch.frexp(torch.clamp(a, min=2.0 ** -6))[1] - 1, min=-6).double()
    step = torch.exp2(exponent - 3)
    code = torch.sign(quotient) * torch.clamp(torch.round(a / step) * step, max=448.0)
    return torch.where(fine, code * s, torch.full_like(x, math.nan))


def attend(q, k, v, length, new, scale, window=0, hidden=()):
    """One sequence: q [new, heads, d], k and v [length, kv_heads, d] float64, `hidden`: positions that nobody sees.
    Returns out, sum p |v| / sum p (what errors of p scale with), lse, and scale * max_j sum_d |q_d k_jd| per row and head."""
    m, heads, d = q.shape
    group = heads // k.shape[1]
    out, mag = torch.zeros(m, heads, d, dtype=torch.float64), torch.zeros(m, heads, d, dtype=torch.float64)
    lse, size = torch.full((m, heads), -math.inf, dtype=torch.float64), torch.zeros(m, heads, dtype=torch.float64)
    q = q.double().cpu()
    for i in range(m):
        pos = length - m + i
        seen = [j for j in range(max(0, pos - window + 1) if window else 0, pos + 1) if j not in hidden]
        if not seen:
            continue
        for h in range(heads):
            kk, vv = k[seen, h // group], v[seen, h // group]
            s = scale * (kk @ q[i, h])
            top = s.max()
            p = torch.exp(s - top)
            total = p.sum()
            out[i, h] = (p @ vv) / total
            mag[i, h] = (p @ vv.abs()) / total
            lse[i, h] = top + torch.log(total)
            size[i, h] = abs(scale) * (kk.abs() @ q[i, h].abs()).max()
    return out, mag, lse, size


def check_attend(got_out, got_lse, want, d, label):
    """The bar.  out: rounded to 8 significant bits (half a unit of the last: 2^-8 of itself), each p rounded to as many (2^-8 of sum p |v| / sum p), and the
    errors of single precision: the scores' (d additions of products, bounded by size, and three roundings), exp's and the sums'.
    lse: the scores' error and that of exp, the sum and log."""
    out, mag, lse, size = want
    score = (d + 4) * 2.0 ** -24 * size
    empty = torch.isneginf(lse)
    g, gl = got_out.double().cpu(), got_lse.double().cpu()
    assert torch.equal(torch.isneginf(gl), empty), f"{label}: rows that see nothing"
    assert (g[empty] == 0).all(), f"{label}: rows that see nothing are zeros"
    tol = 1.02 * 2.0 ** -8 * (out.abs() + mag) + (2 * score[..., None] + 2.0 ** -16) * mag + 1e-37
    err = (g - out).abs()
    assert torch.isfinite(g).all() and (err <= tol).all(), f"{label}: out {float((err - tol).max()):.3e} beyond the bar"
    fin = ~empty
    err = (gl - lse)[fin].abs()
    tol = (score + 2.0 ** -20 * (1 + lse.abs()))[fin]
    assert (err <= tol).all(), f"{label}: lse {float((err - tol).max()):.3e} beyond the bar"


def verify(tokens, rows, target, draft=None, u_accept=None, u_sample=None):
    """Sequence by sequence; numpy float64 arrays [rows, vocab].  Returns accepted, tokens."""
    accepted, out, at = [], [], 0
    vocab = target.shape[1]
    for b, m in enumerate(rows):
        if m == 0:
            accepted.append(-1)
            continue
        kept = 0
        while kept < m - 1:
            r, x = at + kept, int(tokens[at + kept + 1])
            if u_accept is None:
                row = np.where(np.isnan(target[r]), -np.inf, target[r])
                real = ~np.isnan(target[r])
                best = int(np.argmax(np.where(real, row, -np.inf))) if real.any() else -1
                if best >= 0 and not real[best]:
                    best = int(np.nonzero(real)[0][0])
                if best < 0 or best != x:
                    break
            else:
                if not 0 <= x < vocab:
                    break
                c = 1.0 if draft is None else draft[r, x]
                if not float(u_accept[r]) * c < target[r, x]:
                    break
            kept += 1
        r = at + kept
        if u_accept is None:
            real = ~np.isnan(target[r])
            if not real.any():
                nxt = -1
            else:
                best = np.max(target[r][real])
                nxt = int(np.nonzero(real & (target[r] == best))[0][0])
        else:
            w = target[r].copy()
            if kept < m - 1:
                if draft is not None:
                    w = w - draft[r]
                elif 0 <= int(tokens[r + 1]) < vocab:
                    w[int(tokens[r + 1])] = 0.0
            w = np.where(w > 0, w, 0.0)
            if w.sum() == 0:
                w = np.where(target[r] > 0, target[r], 0.0)
            sums = np.cumsum(w)
            over = np.nonzero(sums > float(u_sample[b]) * sums[-1])[0]
            nxt = int(over[0]) if len(over) else -1
        accepted.append(kept)
        out += [int(x) for x in tokens[at + 1:at + 1 + kept]] + [nxt] + [-1] * (m - 1 - kept)
        at += m
    return accepted, out
