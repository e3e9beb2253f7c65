"""Inputs of a product in microscaled 4 bits that show P = x L_B^T alone, with all 24 bits of each of its numbers (test infrastructure, NumPy).

The weights are zeros (of gates: one 64 against a one of every token), so the outputs are P L_A^T (64 times that).  A rank has three channels, of 8 bits each and 2^-8 apart, against
+-2^s of the token: P has 24 bits, and sums of any order are exact.  The first of them is the same for all ranks.  An output has one rank, or the difference
of two, which is 2^-8 of them, times a power of two."""
import numpy as np

from oracle import mx4_oracle as orc

ENDS = {"middle": ((0, -20, 30), -2), "small": ((0, -60, -100, -112, -118, -122), 20), "large": ((0, 60, 118, 126, 127), -14)}


def ranks_alone(rng, rows, n, m, r, end, swiglu=False, tokens=None):
    """(codes and scales of x, of w, L_A, L_B, P, outputs, sum of their magnitudes); m: outputs; the arrays float64.  The last row is NaN if there are more than two.
    tokens: codes and scales of x instead of new ones."""
    exps, by = ENDS[end]
    width = orc.width(n)
    last = (n + 31) // 32 - 1                                      # the block of the ones
    assert last > 0
    xc = np.where(rng.random((rows, width)) < 0.5, 2, 10).astype(np.uint8)       # +-1
    xc[::5] = 2
    xc[:, 32 * last:] = 0
    xc[:, 32 * last] = 2
    xs = np.zeros((rows, width // 32), np.uint8)
    xs[:, :last] = (127 + rng.choice(exps, rows))[:, None]
    xs[:, last] = 127
    if rows > 2:
        xs[-1, 0] = 255
    gates = m if swiglu else 0
    xc, xs = tokens or (xc, xs)
    wc, ws = np.zeros((gates + m, width), np.uint8), np.full((gates + m, width // 32), 127, np.uint8)
    wc[:gates, 32 * last] = 6
    ws[:gates, last] = 131                                         # 4 2^4
    L_B = np.zeros((r, n))
    channels = np.stack([7 + rng.permutation(32 * last - 7)[:3] for _ in range(r)])
    for j in range(3):
        bits = 1.0 + rng.integers(0, 128, r) / 128.0
        bits[0] = 255.0 / 128.0
        if j == 0:                                                 # at the end the largest of 8 bits: most sums have no nearest number of 8 bits but an infinity
            channels[:, 0], bits[:] = 3, 255.0 / 128.0 if end == "large" else 181.0 / 128.0
        L_B[np.arange(r), channels[:, j]] = bits * 2.0 ** (-8 * j)
    L_A = np.zeros((gates + m, r))
    o = np.arange(m)
    size = 2.0 ** (by + o % 3)
    L_A[gates + o, o % r] = size
    if r > 1:
        two = o[(o // r) % 2 == 0]
        L_A[gates + two, (two + 1) % r] = -size[two]
    P = orc.values(xc, xs)[:, :n] @ L_B.T
    Z, S = P @ L_A[gates:].T, np.abs(P) @ np.abs(L_A[gates:]).T
    if swiglu:
        Z, S = 64.0 * Z, 64.0 * S
    return (xc, xs), (wc, ws), L_A, L_B, P, Z, S


def off(S, Z, bf16, many, swiglu):
    """What an output may be off: three products of P and twice three or fewer of the output, each addition 2^-23 of the magnitudes; bf16 outputs of many rows have P as two
    terms, which leave 2^-17 (2^-8, and of the rest, at most half the next binade, 2^-8 again); gates 2^-21; half a step of the result."""
    unit = 10 * 2.0 ** -23 + (2.0 ** -17 if bf16 and many else 0.0) + (2.0 ** -21 if swiglu else 0.0)
    return unit * S + (np.abs(Z) + unit * S) * (2.0 ** -8 if bf16 else 2.0 ** -24)


def terms(P, count):
    """P as so many bf16 terms, each the rounded rest, added up again: what they hold."""
    rest, held = P.astype(np.float32), np.zeros_like(P)
    for _ in range(count):
        u = rest.view(np.uint32)
        with np.errstate(all="ignore"):
            term = ((u + np.uint32(0x7FFF) + ((u >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)
            held = held + term.astype(np.float64)
            rest = rest - term
    return held
