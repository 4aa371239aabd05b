"""The recurrence where a wait for rows ran out, on the CPU: the kernels' own arithmetic, a strip's runs one behind the other,
one of them made of rows that never came.  All that it made has to be NaN, whatever begins in it, and what went through it up
to the next beginning behind it; the rest is what it would have been."""
import ctypes
import math

import numpy as np
import pytest

from tests.device_text import compiled

RUN, RUNS = 4, 5
TOKENS = RUN * RUNS

BODY = """
constexpr int kRun = 4, kRuns = 5;

// f (-0 at beginnings) and b of the tokens; `lost`: the run whose rows did not come, from `from` tokens on
// padding.  rows[t] and last as relay_recurrence_tiles_kernel makes them, a run a warp.
void forward(const float* f, const float* b, float initial, int lost, int tokens, float* rows, float* last) {
    float h = initial;
    for (int run = 0; run < kRuns; ++run) {
        float fr[kRun][2], br[kRun][2];
        const int counts = tokens - run * kRun;
        for (int r = 0; r < kRun; ++r)
            for (int k = 0; k < 2; ++k) fr[r][k] = f[run * kRun + r], br[r][k] = b[run * kRun + r];
        if (run == lost) lose(br);
        for (int r = 0; r < kRun; ++r)
            if (r >= counts) fr[r][0] = fr[r][1] = 1.0f, br[r][0] = br[r][1] = 0.0f;
        float a = fr[0][0], e = br[0][0], x = h;
        for (int r = 1; r < kRun; ++r) join<true>(a, e, fr[r][0], br[r][0]);
        for (int r = 0; r < kRun; ++r) {
            x = carry<true>(x, fr[r][0], br[r][0]);
            if (r < counts) rows[run * kRun + r] = x;
        }
        h = carry<true>(h, a, e);
    }
    *last = h;
}

// The same of relay_recurrence_backward_tiles_kernel, from the last run to the first.
void backward(const float* f, const uint8_t* begins, const float* dout, const float* before, const float* value, float dlast,
              int lost, int tokens, float* dg, float* dv, float* dinitial) {
    float m = dlast;
    for (int run = kRuns - 1; run >= 0; --run) {
        float at[kRun][2], rest[kRun][2], ends[4] = {1.0f, 1.0f, 0.0f, 0.0f}, x = m;
        const int counts = tokens - run * kRun, first = run * kRun;
        for (int r = kRun - 1; r >= 0; --r)
            for (int k = 0; k < 2; ++k) {
                at[r][k] = f[first + r], rest[r][k] = 1.0f - f[first + r];
                if (r < counts) back_join(begins[first + r], at[r][k], dout[first + r], ends[k], ends[2 + k]);
            }
        if (run == lost && counts > 0) lose(at, rest, ends);
        for (int r = kRun - 1; r >= 0; --r)
            if (r < counts)
                back_step(begins[first + r], at[r][0], rest[r][0], dout[first + r], begins[first + r] ? 0.0f : before[first + r],
                          value[first + r], x, dg[first + r], dv[first + r]);
        m = carry<true>(m, ends[0], ends[2]);
    }
    *dinitial = m;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    here = "recurrence.cu"
    return compiled(tmp_path_factory.mktemp("recurrence"),
                    [(here, name) for name in ("starts", "carry", "join", "lose", "back_step", "back_join")], BODY)


def _p(a):
    return a.ctypes.data_as(ctypes.c_void_p)


def _inputs(begins, seed=3):
    r = np.random.default_rng(seed)
    f = r.uniform(0.2, 0.9, TOKENS).astype(np.float32)
    rows = [r.standard_normal(TOKENS).astype(np.float32) for _ in range(4)]
    marks = np.zeros(TOKENS, np.uint8)
    marks[list(begins)] = 1
    return f, marks, rows


def _forward(lib, f, marks, add, lost, tokens):
    rows, last = np.zeros(TOKENS, np.float32), ctypes.c_float()
    factor = np.where(marks, np.float32(-0.0), f).astype(np.float32)
    lib.forward(_p(factor), _p(add), ctypes.c_float(0.7), lost, tokens, _p(rows), ctypes.byref(last))
    return rows, last.value


def _backward(lib, f, marks, dout, before, value, lost, tokens):
    dg, dv, first = np.zeros(TOKENS, np.float32), np.zeros(TOKENS, np.float32), ctypes.c_float()
    lib.backward(_p(f), _p(marks), _p(dout), _p(before), _p(value), ctypes.c_float(0.3), lost, tokens, _p(dg), _p(dv),
                 ctypes.byref(first))
    return dg, dv, first.value


BEGINS = [(), (8,), (9,), (10, 11), (8, 9, 10, 11), (11,), (9, 14), (0, 9, 16)]


@pytest.mark.parametrize("tokens", [TOKENS, 11, 10, 8])
@pytest.mark.parametrize("begins", BEGINS)
def test_forward(lib, begins, tokens):
    f, marks, (add, *_) = _inputs(begins)
    good, good_last = _forward(lib, f, marks, add, -1, tokens)
    rows, last = _forward(lib, f, marks, add, 2, tokens)
    gone, off = np.zeros(TOKENS + 1, bool), False  # the last one: the state behind the tokens
    for t in range(tokens):
        off = t // RUN == 2 or (off and not marks[t])
        gone[t] = off
    gone[TOKENS] = off
    assert np.array_equal(np.isnan(np.append(rows, last)), gone)
    assert np.array_equal(np.append(rows, last)[~gone], np.append(good, np.float32(good_last))[~gone])


@pytest.mark.parametrize("tokens", [TOKENS, 11, 10, 8])
@pytest.mark.parametrize("begins", BEGINS)
def test_backward(lib, begins, tokens):
    f, marks, (dout, before, value, _) = _inputs(begins)
    good = _backward(lib, f, marks, dout, before, value, -1, tokens)
    here = _backward(lib, f, marks, dout, before, value, 2, tokens)
    # a token's gradients: gone in the run that is, and before it where no sequence begins in between; what goes on
    # before token t is gone with it unless t begins one, and out of the run itself it always is
    gone, off = np.zeros(TOKENS, bool), False
    for t in range(tokens - 1, -1, -1):
        gone[t] = off or t // RUN == 2
        off = t // RUN == 2 or (off and not marks[t])
    for a, b in zip(here[:2], good[:2]):
        assert np.array_equal(np.isnan(a), gone)
        assert np.array_equal(a[~gone], b[~gone])
    assert math.isnan(here[2]) == off and (off or here[2] == good[2])
