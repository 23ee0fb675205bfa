"""What the tests of the row operators share: inputs on the GPU with their float64 values,
and unit roundoffs.

Tolerances.  u = 2^-24 bounds the relative error of a binary32 operation, UNIT[type] that of
the one rounding to an output, LEAST[type] half the type's smallest number (results near zero
are rounded to a multiple of it).  Products and sums of a fixed few operations are given one u
each and a few more; the sum over a row runs through at most TREE additions one after the
other (32 of a lane's octets, 6 of a wave, 16 of the waves), so its error is at most TREE u
times the sum of its terms' absolute values."""

import numpy as np

torch = __import__("pytest").importorskip("torch")

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}
TREE = 64


def rows(rng, n, d, kind, scale=1.0, gap=0, shift=0):
    """(n x d device tensor whose rows are `gap` columns apart and start `shift` elements
    into their allocation, its values in float64)."""
    t = torch.from_numpy(rng.standard_normal((n, d)) * scale).to(TYPES[kind])
    buf = torch.full((n * (d + gap) + shift,), float("nan"), dtype=TYPES[kind], device=DEV)
    out = buf[shift:].view(n, d + gap)[:, :d]
    out.copy_(t)
    return out, t.double().numpy()


def blank(n, d, kind, gap=0, shift=0):
    buf = torch.full((n * (d + gap) + shift,), 7.0, device=DEV).to(
        TYPES[kind] if isinstance(kind, str) else kind)
    return buf[shift:].view(n, d + gap)[:, :d]


def gaps_untouched(t, value=7.0):
    """The elements between t's rows still hold what blank() put there."""
    if t.shape[0] == 0 or t.stride(0) == t.shape[1]:
        return True
    between = torch.as_strided(t, (t.shape[0], t.stride(0) - t.shape[1]), t.stride(),
                               t.storage_offset() + t.shape[1])
    return bool((between.float() == value).all())


def host(t):
    return t.detach().double().cpu().numpy()


def vec(rng, d):
    w = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32)
    return torch.from_numpy(w).to(DEV), w.astype(np.float64)


def close(got, want, tol, what):
    got = host(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, what
    err = np.abs(got - want)
    worst = float(np.max(err / np.maximum(tol, 1e-300), initial=0.0))
    assert np.all(err <= tol), f"{what}: worst error {worst:.3g} of the tolerance"
