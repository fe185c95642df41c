"""How many draws of actions 32 bits leave undecided, and that those they decide are right: the
decision itself, compiled for the host (no GPU needed)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from paper_2602_01665_amd import build as hip_build
from tests import learner_reference as R

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def pick(tmp_path_factory):
    from paper_2602_01665_amd.binding import TabxSampling
    lib = tmp_path_factory.mktemp("pick") / "learner_pick.so"
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc] + hip_build.HIPCC_FLAGS + ["-I", os.path.dirname(hip_build.SOURCES[0]), "-x", "hip",
                                                      os.path.join(HERE, "learner_pick.cpp"), "-o", str(lib)],
                   check=True, capture_output=True)
    rows_of = C.CDLL(str(lib)).pick_rows
    rows_of.argtypes = [C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]

    def go(logits, u, *how):
        n = len(u)
        choice, close = np.empty(n, np.int32), np.empty(n, np.uint8)
        s = TabxSampling(*how)
        rows_of(n, logits.ctypes.data, u.ctypes.data, C.addressof(s), choice.ctypes.data, close.ctypes.data)
        return choice, close != 0
    return go


def _rows(rng, n):
    """Logits of a trained team, the combat action barred for most."""
    l = rng.normal(size=(n, 8)).astype(np.float32) * 2
    l[rng.random(n) < 0.6, R.ATTACK] = -np.inf
    l[rng.random((n, 8)) < 0.01] = -np.inf
    l[:, 0] = np.where(np.isinf(l).all(1), 0.0, l[:, 0])
    return l, rng.random(n).astype(np.float32)


# (temperature, top_k, top_p, min_p)
SETTINGS = [(1.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 1e-5), (0.3, 0, 1.0, 1e-5), (1.0, 0, 1.0, 1e-7), (1.0, 4, 1.0, 1e-30),
            (0.3, 0, 0.99999, 0.0), (1.0, 0, 0.9999, 0.0), (0.3, 0, 0.9999, 0.0), (1.0, 0, 1 - 2.0 ** -24, 0.0),
            (1.0, 0, 1e-6, 0.0), (0.8, 5, 0.9, 0.02), (0.8, 5, 0.9999, 1e-6), (2.0, 0, 0.5, 1.0), (0.02, 0, 0.95, 1e-4)]


@pytest.mark.parametrize("how", SETTINGS)
def test_few_rows_are_left_undecided(pick, how):
    """A draw is within 2^-16 of one of seven borders with a probability of at most 7 * 2^-15 (the sum
    of all is one or more), four of 20000 rows; a filter's comparison within 2^-16 of itself is one
    of seven logarithms within 2^-16 of a given one, which is no likelier.  50 rows are six times both."""
    l, u = _rows(np.random.default_rng(1), 20000)
    _, close = pick(l, u, *how)
    print(how, int(close.sum()))
    assert close.sum() <= 50, close.mean()


@pytest.mark.parametrize("how", SETTINGS)
def test_what_is_decided_is_right(pick, how):
    rng = np.random.default_rng(2)
    l, u = _rows(rng, 3000)
    l[1000:2000] = np.round(l[1000:2000])                      # many equal scores
    u[:5] = 0.0, 2.0 ** -30, 0.5, 1 - 2.0 ** -24, 1e-6
    choice, close = pick(l, u, *how)
    want = np.array([R.choose(row.astype(np.float64), *how, x) for row, x in zip(l, u)])
    assert np.array_equal(choice[~close], want[~close])


def test_scores_next_to_a_border_are_left_undecided(pick):
    """Weights moved by less than 32 bits tell apart from min_p, and from a share of top_p."""
    n = 4000
    l = np.zeros((n, 8), np.float32)
    l[:, 2:] = -np.inf
    u = np.full(n, 0.999, np.float32)
    for top_p, min_p in ((1.0, 0.01), (1 / 1.01, 0.0), (1 / 1.01, 0.01)):
        l[:, 1] = np.float32(np.log(0.01)) + np.linspace(-2e-5, 2e-5, n).astype(np.float32)
        choice, close = pick(l, u, 1.0, 0, top_p, min_p)
        want = np.array([R.choose(row.astype(np.float64), 1.0, 0, top_p, min_p, x) for row, x in zip(l, u)])
        assert np.array_equal(choice[~close], want[~close])
        assert close.any() and not close.all()
