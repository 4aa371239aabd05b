"""The gated linear recurrence in 64 bits, token by token, with the error bounds that fp32 arithmetic gives."""
import numpy as np

from .layers_util import U, sigmoid


def gate_error(g):
    """How far, relative to the gate's own slope, sigma(g) and 1 - sigma(g) are off: as if g were moved by this.
    The exponential's argument is rounded (|g| 2^-23 with the product by log2 e), the exponential is within 2
    units in the last place, sum, reciprocal and product round or are within one: (4 + |g|) 2^-23 covers them."""
    return (4 + np.abs(g)) * 2.0 ** -23


def forward(g, v, initial=None, begins=None, lengths=None):
    """(h, last) and their bounds before the outputs' rounding.

    A state is off by what the one before it was, times f; by its gate's error, f (1 - f) times the spread
    between state and value; and by roundings, each at most U times the sum H of the magnitudes that make it
    up: a product and an addition for the token, the same again where its stretch is joined to others, whose
    factors are products of as many roundings (one a token): 8 U H a token covers them."""
    n, T, d = g.shape
    f, rest = sigmoid(g), sigmoid(-g)
    h = np.zeros((n, d)) if initial is None else initial.astype(np.float64)
    H, E = np.abs(h), np.zeros((n, d))
    out, bound = np.zeros((n, T, d)), np.zeros((n, T, d))
    ends = np.full(n, T) if lengths is None else np.clip(lengths, 0, T)
    for t in range(T):
        new = np.zeros((n, 1), bool) if begins is None else begins[:, t, None] != 0
        used = (t < ends)[:, None]
        h0, H0, E0 = (np.where(new, 0, x) for x in (h, H, E))
        h1 = f[:, t] * h0 + rest[:, t] * v[:, t]
        H1 = f[:, t] * H0 + rest[:, t] * np.abs(v[:, t])
        slope = gate_error(g[:, t]) * (f[:, t] * rest[:, t] * (H0 + np.abs(v[:, t])))
        E1 = f[:, t] * E0 + slope + 8 * U * H1
        h, H, E = np.where(used, h1, h), np.where(used, H1, H), np.where(used, E1, E)
        out[:, t], bound[:, t] = np.where(used, h, 0), np.where(used, E, 0)
    return out, h, bound, E


def backward(dout, g, v, h, initial=None, dlast=None, begins=None, lengths=None):
    """(dgate, dvalue, dinitial) and their bounds: the same recurrence from the other end."""
    n, T, d = g.shape
    f, rest = sigmoid(g), sigmoid(-g)
    m = np.zeros((n, d)) if dlast is None else dlast.astype(np.float64)
    M, E = np.abs(m), np.zeros((n, d))
    first = np.zeros((n, d)) if initial is None else initial.astype(np.float64)
    dg, dv, bg, bv = (np.zeros((n, T, d)) for _ in range(4))
    ends = np.full(n, T) if lengths is None else np.clip(lengths, 0, T)
    for t in range(T - 1, -1, -1):
        new = np.zeros((n, 1), bool) if begins is None else begins[:, t, None] != 0
        used = (t < ends)[:, None]
        F, R, off = f[:, t], rest[:, t], gate_error(g[:, t])
        d_t = np.where(used, dout[:, t], 0)
        l, L = d_t + m, np.abs(d_t) + M
        El = E + 4 * U * L
        h0 = np.where(new, 0, first if t == 0 else h[:, t - 1])
        spread = np.abs(h0) + np.abs(np.where(used, v[:, t], 0))
        dv[:, t], bv[:, t] = np.where(used, l * R, 0), np.where(used, R * El + (off + 2 * U) * R * L, 0)
        with np.errstate(invalid="ignore"):
            dg[:, t] = np.where(used, l * R * F * (h0 - v[:, t]), 0)
        bg[:, t] = np.where(used, F * R * spread * (El + (2 * off + 6 * U) * L), 0)
        m1, M1, E1 = F * l, F * L, F * El + (off * R + 8 * U) * F * L
        m, M, E = (np.where(used, np.where(new, 0, x1), x) for x1, x in ((m1, m), (M1, M), (E1, E)))
    return dg, dv, m, bg, bv, E
