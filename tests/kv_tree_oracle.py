"""Trees of drafted tokens over the paged cache, and eviction by attention weight, from their definitions in 64 bits on the CPU.
Shares no code with the library."""

import math

import numpy as np
import torch


def ancestors(parents):
    """Of every row the row itself and its ancestors, ascending."""
    lists = []
    for i, p in enumerate(parents):
        lists.append((lists[p] if 0 <= p < i else []) + [i])
    return lists


def words(lists):
    """Rows' lists as masks of 256 bits, int32 [rows, 8]."""
    out = np.zeros((len(lists), 8), np.uint32)
    for i, rows in enumerate(lists):
        for j in rows:
            out[i, j // 32] |= np.uint32(1 << (j % 32))
    return torch.from_numpy(out.view(np.int32))


def seen_by(lists, length, window=0, hidden=()):
    """[rows, length]: which positions the rows see; `lists`: of every row, ascending, those of the rows that it may see."""
    m = len(lists)
    seen = torch.zeros(m, length, dtype=torch.bool)
    for i, rows in enumerate(lists):
        rows = [j for j in rows if j <= i]
        here = length - m + max(0, len(rows) - 1)
        seen[i, max(0, here - window + 1) if window else 0:max(0, length - m)] = True
        for j in rows[-window:] if window else rows:
            if length - m + j >= 0:
                seen[i, length - m + j] = True
    seen[:, list(hidden)] = False
    return seen


def attend(q, k, v, seen, scale):
    """What kv_oracle.attend returns, for rows that see any positions."""
    m, heads, d = q.shape
    group = heads // k.shape[1]
    out, mag = torch.zeros(m, heads, d, dtype=torch.float64), torch.zeros(m, heads, d, dtype=torch.float64)
    lse, size = torch.full((m, heads), -math.inf, dtype=torch.float64), torch.zeros(m, heads, dtype=torch.float64)
    some = seen.any(1)
    if not bool(some.any()):
        return out, mag, lse, size
    used = seen.any(0)  # what nobody sees may be anything
    for h in range(heads):
        for rows in [torch.nonzero(some).squeeze(1)]:
            at = seen[rows][:, used]
            kk, vv, qq = k[used, h // group], v[used, h // group], q[rows, h].double()
            bad = ~torch.isfinite(kk).all(1) | ~torch.isfinite(vv).all(1)
            if bool(bad.any()):  # row by row: what a row does not see must not touch it
                for r in range(len(rows)):
                    kr, vr = kk[at[r]], vv[at[r]]
                    s = scale * (kr @ qq[r])
                    top = s.max()
                    p = torch.exp(s - top)
                    out[rows[r], h], mag[rows[r], h] = (p @ vr) / p.sum(), (p @ vr.abs()) / p.sum()
                    lse[rows[r], h] = top + torch.log(p.sum())
                    size[rows[r], h] = abs(scale) * (kr.abs() @ qq[r].abs()).max()
                continue
            s = torch.where(at, scale * (qq @ kk.t()), torch.full((), -math.inf, dtype=torch.float64))
            top = s.amax(1, keepdim=True)
            p = torch.exp(s - top)
            total = p.sum(1, keepdim=True)
            out[rows, h], mag[rows, h] = (p @ vv) / total, (p @ vv.abs()) / total
            lse[rows, h] = (top + torch.log(total)).squeeze(1)
            size[rows, h] = torch.where(at, abs(scale) * (qq.abs() @ kk.abs().t()), torch.zeros((), dtype=torch.float64)).amax(1)
    return out, mag, lse, size


def verify(parents, tokens, target, u=None):
    """One sequence; target numpy float64 [rows, vocab].  Returns accepted, rows, tokens."""
    m = len(parents)
    if m == 0:
        return -1, [], []
    row, rows, out = 0, [], []
    while True:
        p = target[row]
        if u is None:
            real = ~np.isnan(p)
            x = int(np.nonzero(real & (p == p[real].max()))[0][0]) if real.any() else -1
        else:
            w = np.where(p > 0, p, 0.0)
            sums = np.cumsum(w)
            over = np.nonzero((sums > float(u[row]) * sums[-1]) & (w > 0))[0]
            x = int(over[0]) if len(over) else -1
        rows.append(row)
        out.append(x)
        nxt = [c for c in range(row + 1, m) if parents[c] == row and tokens[c] == x and x >= 0]
        if not nxt:
            return len(rows) - 1, rows + [-1] * (m - len(rows)), out + [-1] * (m - len(out))
        row = nxt[0]


def weigh(q, k, lse, length, window, scale):
    """One sequence: sums [kv_heads, length] of the rows' weights, and how far single precision may be off: every score by its d additions and
    four roundings (bounded by size), the exponent by its own rounding and that of lse (2^-22 of 1 + |lse| + |score - lse|), the sum by
    one rounding for each term, 2^-24 of the whole."""
    m, heads, d = q.shape
    kvh = k.shape[1]
    group = heads // kvh
    sums, tol = torch.zeros(kvh, length, dtype=torch.float64), torch.zeros(kvh, length, dtype=torch.float64)
    pos, row = torch.arange(length)[None], torch.arange(length - m, length)[:, None]
    seen = (pos <= row) & ((pos > row - window) if window else (pos >= 0)) & (row >= 0)
    for h in range(heads):
        kk, qq, ll = k[:, h // group], q[:, h].double(), lse[:, h].double()[:, None]
        use = seen & ~torch.isneginf(ll)
        s = scale * (qq @ kk.t())
        size = abs(scale) * (qq.abs() @ kk.abs().t())
        x = torch.where(use, s - ll, torch.full_like(s, -math.inf))
        w = torch.exp(x)
        off = (d + 4) * 2.0 ** -24 * size + 2.0 ** -22 * (1 + ll.abs() + torch.where(use, x.abs(), torch.zeros_like(x)))
        sums[h // group] += w.sum(0)
        tol[h // group] += torch.where(use, w * off, torch.zeros_like(w)).sum(0)
    return sums, tol + (m * group + 4) * 2.0 ** -24 * sums + m * group * 2.0 ** -126


def evict(mass, born, keep, recent, early):
    """One sequence and head, lists of its slots' numbers: from which slot what stands in each of the first min(length, keep) comes."""
    length = len(mass)
    stay = min(length, keep)
    born = list(range(length)) if born is None else born
    newest = max(born, default=0)
    safe = [b > newest - recent or b < early for b in born]
    key = [math.inf if s else (-math.inf if math.isnan(w) else w) for w, s in zip(mass, safe)]
    rank = [2 if s else 0 if math.isnan(w) else 1 for w, s in zip(mass, safe)]
    order = sorted(range(length), key=lambda i: (-rank[i], -key[i], i))
    kept = set(order[:stay])
    later = iter(sorted(i for i in kept if i >= stay))
    return [i if i in kept else next(later) for i in range(stay)]
