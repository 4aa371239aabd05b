"""The backward step between blocks where a wait for a row ran out, on the CPU: the kernels' own arithmetic of a row's
features, with whatever lay in shared memory in place of the row.  Its gradients and the sums of the weights' gradients that
it goes into, all of them, have to be NaN."""
import ctypes

import numpy as np
import pytest

from tests.device_text import compiled

D = 64

PAIR = """
struct Pair {
    float2 v;
    Pair() {}
    Pair(float a, float b) : v{a, b} {}
    explicit Pair(float both) : v{both, both} {}
    float sum() const { return v.x + v.y; }
};
inline Pair operator*(Pair a, Pair b) { return Pair(a.v.x * b.v.x, a.v.y * b.v.y); }
inline Pair fma(Pair a, Pair b, Pair c) { return Pair(std::fmaf(a.v.x, b.v.x, c.v.x), std::fmaf(a.v.y, b.v.y, c.v.y)); }
template <typename T>
struct Gate {
    float at, rest;
    explicit Gate(float g) : at(1.0f / (1.0f + std::exp(-g))), rest(1.0f / (1.0f + std::exp(g))) {}
};
"""

BODY = """
constexpr int kD = 64, kPairs = kD / 2;
static void pairs(const float* from, Pair (&to)[kPairs]) {
    for (int k = 0; k < kPairs; ++k) to[k] = Pair(from[2 * k], from[2 * k + 1]);
}
static void numbers(const Pair (&from)[kPairs], float* to) {
    for (int k = 0; k < kPairs; ++k) to[2 * k] = from[k].v.x, to[2 * k + 1] = from[k].v.y;
}

// A row as relay_block_norm_backward_rows_kernel takes it.  rows: x, residual, gate, dy, dtotal; weights: post, pre, scale;
// out: dx, dresidual, dgate; sums: of post, pre, scale.
void row(bool came, bool gated, float row_x, float row_h, const float* rows, const float* weights, float* out, float* sums) {
    const float sx = factor_of(came, row_x), sh = factor_of(came, row_h);
    Features<float, kPairs> o;
    Pair w[kPairs], pre[kPairs], rho[kPairs], u[kPairs], over[kPairs], dz[kPairs], dr[kPairs], dpost[kPairs], dpre[kPairs], dscale[kPairs];
    pairs(rows, o.xhat), pairs(rows + kD, o.r), pairs(rows + 2 * kD, o.p), pairs(rows + 3 * kD, u), pairs(rows + 4 * kD, over);
    pairs(weights, w), pairs(weights + kD, pre), pairs(weights + 2 * kD, rho);
    for (int k = 0; k < kPairs; ++k) dpost[k] = dpre[k] = dscale[k] = Pair(0.0f);
    Pair three[3] = {Pair(0.0f), Pair(0.0f), Pair(0.0f)};
    o.make(w, rho, gated, sx, sh);
    o.add(u, pre, over, sh, three, dpre);
    const float along = three[0].sum() / kD, along_x = three[1].sum() / kD - sh * along * (three[2].sum() / kD);
    o.leave(u, pre, over, w, rho, sx, sh, along, along_x, dz, dr, dpost, dscale);
    numbers(u, out), numbers(dr, out + kD), numbers(dz, out + 2 * kD);
    numbers(dpost, sums), numbers(dpre, sums + kD), numbers(dscale, sums + 2 * kD);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    here = "block_norm.cu"
    return compiled(tmp_path_factory.mktemp("block"), [PAIR, (here, "factor_of"), (here, "Features")], BODY)


def _p(a):
    return a.ctypes.data_as(ctypes.c_void_p)


def _row(lib, came, gated, rows, weights, sx=0.8, sh=1.3):
    out, sums = np.zeros((3, D), np.float32), np.zeros((3, D), np.float32)
    lib.row(ctypes.c_bool(came), ctypes.c_bool(gated), ctypes.c_float(sx), ctypes.c_float(sh), _p(rows), _p(weights), _p(out), _p(sums))
    return out, sums


@pytest.mark.parametrize("gated", [False, True])
def test_a_row_that_came(lib, gated):
    r = np.random.default_rng(0)
    rows, weights = r.standard_normal((5, D)).astype(np.float32), r.standard_normal((3, D)).astype(np.float32)
    out, sums = _row(lib, True, gated, rows, weights)
    x, res, z, dy, over = rows.astype(np.float64)
    post, pre, rho = weights.astype(np.float64)
    p = 1 / (1 + np.exp(-z)) if gated else np.ones(D)
    xhat, sh = x * np.float64(np.float32(0.8)), np.float64(np.float32(1.3))
    hhat = (rho * res + p * xhat * post) * sh
    dh = sh * (dy * pre - hhat * (dy * pre * hhat).mean()) + over
    v = dh * p * post
    # mean(v xhat) as the kernel has it, for the factors here are not those of these rows: over the h that they give
    along_x = (p * xhat * post * (sh * dy * pre + over)).mean() - sh * (dy * pre * hhat).mean() * (p * xhat * post * hhat).mean()
    want = [np.float64(np.float32(0.8)) * (v - xhat * along_x), rho * dh, dh * xhat * post * p * (1 - p)]
    # sums of 64 fp32 products in some order: 64 roundings of 2^-24 of the terms' sizes and a few more, far below 1e-4 here
    for got, exact in zip(out, want):
        np.testing.assert_allclose(got, exact, rtol=1e-4, atol=1e-4)
    for got, exact in zip(sums, [dh * p * xhat, dy * hhat, dh * res]):
        np.testing.assert_allclose(got, exact, rtol=1e-4, atol=1e-4)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("stale", ["numbers", "zeros", "large", "infinite"])
def test_a_row_that_did_not(lib, gated, stale):
    r = np.random.default_rng(1)
    rows = r.standard_normal((5, D)).astype(np.float32) * np.float32(dict(numbers=1, zeros=0, large=1e18, infinite=np.inf)[stale])
    weights = r.standard_normal((3, D)).astype(np.float32)
    weights[:, ::7] = 0
    for factors in ((0.8, 1.3), (0.0, 0.0)):
        out, sums = _row(lib, False, gated, rows, weights, *factors)
        assert np.isnan(out[:2]).all() and np.isnan(sums).all()
        assert not gated or np.isnan(out[2]).all()
