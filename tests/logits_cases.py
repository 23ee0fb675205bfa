"""What the tests of the operators on rows of logits share: inputs and tolerances.

Tolerances, u = 2^-24, x = scale (z - max) of a column, E a mean under the row's p:
  y = log2(e) x takes a difference, the constant's and two products' roundings: 4 u |x|; its power of
  two that much relatively and 2 u of its own.  Each time a lane, a wave or a row is measured from a
  new largest logit its sums move by such a power and a product, and these distances add up to |x| at
  most: in all 4 u |x| + 3 u a move.  A lane adds at most d / 64 columns one after the other, or
  d / 256 of a row longer than 6,144 (768 chunks of 8 are the most that a wave has alone), and at most 64 sums of lanes, waves and parts follow; it moves no more often.  So S is off by
  sum_error(), relatively, log S by that and its own rounding; a term of sum p x by its p's share and
  that of x; outputs are then rounded to their type (half a step, UNIT).  Powers below 2^-126 are 0.
"""

import numpy as np

from oracle import logits as L
from rows_cases import DEV, LEAST, TYPES, U, UNIT, blank, close, gaps_untouched, host, rows, torch  # noqa: F401

INTS = {32: torch.int32, 64: torch.int64}


def steps(d):
    """Roundings that one sum of a row goes through, moves included (3 each)."""
    lane = d / 64 if d <= 6144 else d / 256
    return 4 * (lane + 64)


class Soft:
    """The oracle's softmax of each row, and what binary32 may make of it."""

    def __init__(self, Z, scale):
        self.Z, self.scale, self.d = Z, scale, Z.shape[1]
        both = [L.log_softmax(z, scale) for z in Z]
        self.log_p = np.stack([b[0] for b in both])
        self.lse = np.array([b[1] for b in both])
        self.p = np.exp(self.log_p)
        m = Z.max(axis=1, keepdims=True)
        with np.errstate(invalid="ignore", over="ignore"):
            x = np.where(Z > -np.inf, scale * (Z - np.where(m > -np.inf, m, 0)), -np.inf)
        self.x = np.maximum(x, -200.0)              # (its power of two is 0 long before)
        self.m = np.where(m > -np.inf, m, 0)[:, 0]
        self.live = m[:, 0] > -np.inf
        self.mean_x = (self.p * np.abs(self.x)).sum(1)
        self.mean_x2 = (self.p * self.x ** 2).sum(1)
        self.sum_error = U * (4 * self.mean_x + steps(self.d)) + 2.0 ** -100
        self.log_s = np.where(self.live, np.log(np.maximum(np.exp(np.where(self.live[:, None], x, -np.inf)).sum(1), 1)), 0)
        self.log_s_error = self.sum_error + 4 * U * self.log_s + U
        # sum p x: each term's power, x and the running sum; and the division by S
        self.mean_error = U * (4 * self.mean_x2 + (steps(self.d) + 8) * self.mean_x) + self.mean_x * self.sum_error

    def logp_tol(self, columns):
        at = np.clip(columns, 0, self.d - 1)
        x = np.abs(np.take_along_axis(self.x, at, 1))
        # (a log p of -2.7e38, of a logit at the type's lowest value, has a rounding of u times that)
        lp = np.abs(np.take_along_axis(self.log_p, at, 1))
        return self.log_s_error[:, None] + 2 * U * x + 2 * U * np.where(np.isfinite(lp), lp, 0)

    def lse_tol(self):
        return self.log_s_error + 2 * U * np.abs(self.scale * self.m) + 2 * U * np.abs(np.where(self.live, self.lse, 0))

    def entropy_tol(self):
        return self.log_s_error + self.mean_error + 4 * U * (self.log_s + self.mean_x)

    def p_error(self):
        """Of each p_j, relatively."""
        return U * (4 * np.abs(self.x) + 6) + self.sum_error[:, None]


def grad_tol(s, want, kind, gl, gs, ge, given):
    """Tolerance of toc_logprob_grad's dZ; gl, gs, ge: absolute values per row, given: n x d, whether
    a column is the given token."""
    gl, gs, ge = (np.abs(np.broadcast_to(g, s.lse.shape))[:, None] for g in (gl, gs, ge))
    p = s.p * (s.p_error() + 8 * U)
    tol = p * (gl + gs)
    tol += ge * (p * (s.mean_x[:, None] + np.abs(s.x)) + s.p * s.mean_error[:, None])
    tol += 4 * U * (gl * given) + 2.0 ** -120 * (gl + gs + ge)
    return s.scale * tol + UNIT[kind] * np.abs(want) + LEAST[kind]


def taught_tol(s, ids, t, scale, lse):
    """(tolerance of the loss, of each entry's q, relatively)."""
    n, k = ids.shape
    loss, rel = np.zeros(n), np.zeros((n, k))
    for i in range(n):
        log_q, q = L.teacher(ids[i], t[i], s.d, scale, None if lse is None else float(lse[i]))
        real = q > 0
        if not real.any():
            continue
        # the difference, the product, exp; the sum of at most 256 entries: 4 of a lane, 6 of a wave, 16 waves; its log
        size = np.abs(scale * t[i]) + (0 if lse is None else abs(float(lse[i])))
        size = np.where(real, size + np.max(np.where(real, np.abs(scale * t[i]), 0)), 0)
        rel[i] = U * (4 * size + 40 + 4 * np.abs(np.where(real, log_q, 0)))
        if lse is None:
            rel[i] += (q * rel[i]).sum() * 2
        at = np.where(real, ids[i], 0)
        lp = np.where(real, s.log_p[i, at], 0)
        size = np.abs(np.where(real, log_q, 0)) + np.abs(np.where(np.isfinite(lp), lp, 0))
        e = s.log_s_error[i] + 2 * U * np.abs(s.x[i, at]) + 2 * U * size + rel[i] + size * (rel[i] + 40 * U)
        loss[i] = (q * np.where(real, e, 0)).sum()
    return loss, rel


def logits(rng, n, d, kind, gap=0, shift=0, spread=3.0, masked=0.0, low=False):
    """(device tensor, its float64 values); a share of the columns at minus infinity or at the type's
    lowest value."""
    t, _ = rows(rng, n, d, kind, spread, gap, shift)
    if masked:
        at = torch.from_numpy(rng.random((n, d)) < masked).to(DEV)
        t[at] = torch.finfo(TYPES[kind]).min if low else -float("inf")
    return t, t.double().cpu().numpy()


def given(rng, n, d, bits):
    """Token numbers, some that are none, on the host and the device."""
    ids = rng.integers(0, d, n)
    ids[rng.random(n) < 0.15] = -1
    if n > 4:
        ids[:5] = [d - 1, d, -1, 0, (1 << (bits - 1)) - 1]
    return ids, torch.from_numpy(ids.astype(np.int32 if bits == 32 else np.int64)).to(DEV)


def vec(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(DEV)


def workspace(n, d, k=0):
    """Exactly the bytes asked for, or None."""
    size = __import__("paper_1702_06943_amd").toc_logits_workspace_size(n, d, k)
    return torch.full((size,), 0xA5, dtype=torch.uint8, device=DEV) if size else None


def saved(rng, n, d, k, bits, kind, repeats=False, none=0.1):
    """A teacher's rows: (columns, their device tensor, logits' float64 values, their tensor)."""
    if repeats:
        ids = rng.integers(0, max(1, min(d, k // 2)), (n, k))
    else:
        ids = np.stack([rng.permutation(max(d, k))[:k] for _ in range(n)])
    ids[rng.random((n, k)) < none] = -1
    t = torch.from_numpy(rng.standard_normal((n, k)) * 2 + 3).to(TYPES[kind]).to(DEV)
    return ids, torch.from_numpy(ids).to(INTS[bits]).to(DEV), t.double().cpu().numpy(), t
