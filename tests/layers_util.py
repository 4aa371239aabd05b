"""The layer operators' definitions in 64 bits, their 8-bit format, the inputs
of their tests and the error bounds that the arithmetic gives."""
import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
#: half a unit in the last place, relative, and half the spacing of the smallest numbers
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}
U = 2.0 ** -24  # fp32's rounding
#: terms that a row's fp32 sum adds in a chain at most: 32 in a thread, 5 across a warp, 32 warps, and a few more
CHAIN = 80


def pitch(d):
    return (d + 127) // 128 * 128


def scale_bytes(most):
    """The scale byte of blocks with the largest magnitudes `most` (float64 array), by search:
    the least c in 7..254 for which the largest code is at most 127; 255 where there is none."""
    out = np.full(most.shape, 255, np.int64)
    for c in range(254, 6, -1):
        fits = np.rint(np.ldexp(most, 133 - c)) <= 127
        out[fits] = c
    out[~np.isfinite(most)] = 255
    return out


def pack(x):
    """(codes int8 [..][pitch], scales uint8 [..][pitch / 32]) of x (float64 array)."""
    d = x.shape[-1]
    p = pitch(d)
    b = np.zeros(x.shape[:-1] + (p,))
    b[..., :d] = x
    b = b.reshape(x.shape[:-1] + (p // 32, 32))
    most = np.abs(b).max(-1) if b.size else np.zeros(b.shape[:-1])
    most = np.where(np.isnan(b).any(-1), np.nan, most)
    c = scale_bytes(most)
    with np.errstate(invalid="ignore"):
        q = np.rint(np.ldexp(b, 133 - c[..., None]))
    q = np.where(c[..., None] == 255, 0, q).astype(np.int8)
    return q.reshape(x.shape[:-1] + (p,)), c.astype(np.uint8)


def held(codes, scales, d):
    """The values of a checkpoint, float64."""
    c = np.repeat(scales.astype(np.int64), 32, axis=-1)[..., :d]
    v = np.ldexp(codes[..., :d].astype(np.float64), np.maximum(c, 7) - 133)
    return np.where(c == 255, np.nan, v)


def half_step(x):
    """Half of the format's step for each value of x (float64): the largest of its block is at
    least 63.75 steps, or the step is 2^-126."""
    d = x.shape[-1]
    b = np.zeros(x.shape[:-1] + (pitch(d),))
    b[..., :d] = np.abs(x)
    most = b.reshape(x.shape[:-1] + (-1, 32)).max(-1)
    return np.repeat(np.maximum(most / 127.5, 2.0 ** -127), 32, axis=-1)[..., :d]


def rows(values, dtype, layout, device="cuda", fill=None):
    """`values` (float64 [n][T][d] array) as a tensor of the type in a layout, and the whole buffer:
    dense; wide (rows apart, 16-byte aligned); odd (nothing aligned); tokens (token by token, the
    workers of one next to one another).  `fill`: what the rest of the buffer holds."""
    n, T, d = values.shape
    gap, first = {"dense": (0, 0), "wide": (16, 32), "odd": (3, 1), "tokens": (0, 0)}[layout]
    shape = (T, n, d + gap) if layout == "tokens" else (n, T, d + gap)
    buf = torch.full((first + int(np.prod(shape)) + 64,), float("nan") if fill is None else fill, dtype=dtype,
                     device=device)
    v = buf[first:first + int(np.prod(shape))].view(shape)
    v = v.transpose(0, 1) if layout == "tokens" else v
    v = v[..., :d]
    v.copy_(torch.from_numpy(values))
    return v, buf


def empty_rows(n, T, d, dtype, layout):
    """An output of a layout, filled with 77, and its buffer."""
    return rows(np.full((n, T, d), 77.0), dtype, layout, fill=77.0)


def only_rows_written(view, buf):
    """Whether nothing of `buf` outside of the view differs from 77."""
    seen = torch.zeros_like(buf, dtype=torch.bool)
    seen.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(True)
    return bool((buf[~seen] == 77).all())


def np64(t):
    return t.detach().double().cpu().numpy()


def within(got, want, bound):
    """got and want agree within bound, NaN with NaN."""
    got = np64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (got.shape, want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bad = np.abs(got - want) > bound
    bad &= ~np.isnan(want)
    assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4], np.broadcast_to(bound, got.shape)[bad][:4])


# ------------------------------------------------------------------ definitions


def norm(x, r, w, eps):
    h = x if r is None else x + r
    s = 1 / np.sqrt((h * h).mean(-1) + eps)
    xhat = h * s[..., None]
    return h, s, xhat, xhat * w[:, None, :]


def norm_backward(dy, w, s, xhat, dh, used):
    """(dx, dw) and their error bounds in fp32, without the outputs' rounding."""
    d = dy.shape[-1]
    dy, xhat, s = np.where(used, dy, 0), np.where(used, xhat, 0), np.where(used, s[..., None], 0)
    dh = np.zeros_like(dy) if dh is None else np.where(used, dh, 0)
    u = dy * w[:, None, :]
    along = (u * xhat).sum(-1, keepdims=True) / d
    dx = s * (u - xhat * along) + dh
    spread = np.abs(u * xhat).sum(-1, keepdims=True) / d
    dx_bound = U * (8 * (s * (np.abs(u) + np.abs(xhat * along)) + np.abs(dh)) + CHAIN * s * np.abs(xhat) * spread)
    dw = (dy * xhat).sum(1)
    dw_bound = (dy.shape[1] + 64) * U * np.abs(dy * xhat).sum(1)
    return dx, dw, dx_bound, dw_bound


def sigmoid(g):
    e = np.exp(-np.abs(g))
    return np.where(g < 0, e, 1) / (1 + e)


def gated_backward(da, g, u):
    s, r = sigmoid(g), sigmoid(-g)
    return da * u * (s + g * s * r), da * g * s


def used_rows(lengths, n, T):
    m = np.full(n, T) if lengths is None else np.clip(lengths, 0, T)
    return (np.arange(T)[None, :] < m[:, None])[..., None]
