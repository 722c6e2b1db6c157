"""Orthogonalisation of matrices of few directions, of singular values over many orders and of few different elements, in few steps and in many, against the same iteration in
64 bits: within a figure that is the same for all of them, whatever a model of the roundings would lose.

Bound, of the result's norm.  What enters the products is rounded to fp16, half a step 2^-11 of each element.  Independent roundings average over the elements of a row and leave 3e-3
at most; where elements are few different ones the roundings are too, and move the singular values themselves: a step multiplies X by a polynomial P of A = X X^T, of which A's
rounding (twice X's), O's, P's and X's again make 2^-11 (2 + 1 + 1 + 1) |P X|, with |b + c| = 2.7 up to 7e-3 of a singular value of 1, of which the next steps leave some 0.7 each (their
slope near 1): 1e-2 for roundings that do not all have the same sign.  To that comes what no form with X in fp32 is without: directions that are not there at first
receive the sums' and the iterate's rounding, some 2^-24 for each of its four operations, and every step multiplies it by a: 2^-22 |a|^steps in all, relative to X's norm.  Where many directions are equally strong and as many are not there, what a
step adds is 2^-12 / sqrt(3) (a rounding's root mean square) of |P X| = 2.7 for each of the four roundings, 8e-4 by their squares, and no step takes it away: 8e-4 steps."""
import numpy as np
import pytest

from oracle import update as orc
import test_gpu_newton_schulz as common

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = common.ah

DEFAULT = (3.4445, -4.7750, 2.0315)


def matrix(kind, m, n):
    r = np.random.default_rng([m, n])
    u, v = r.normal(size=m), r.normal(size=n)
    if kind == "one":
        return np.outer(u, v)
    if kind == "sixteen":
        return r.normal(size=(m, 16)) @ r.normal(size=(16, n))
    if kind == "graded":  # singular values from 1 to 1e-6
        k = min(m, n)
        return (np.linalg.qr(r.normal(size=(m, k)))[0] * 10.0 ** -np.linspace(0, 6, k)) @ np.linalg.qr(r.normal(size=(n, k)))[0].T
    if kind == "half":    # of all directions, equally strong
        k = min(m, n)
        return np.linalg.qr(r.normal(size=(m, k)))[0][:, :k // 2] @ np.linalg.qr(r.normal(size=(n, k)))[0].T[:k // 2]
    if kind == "two values":
        return np.outer(np.where(r.random(m) < 0.5, 1.0, 0.37), np.where(r.random(n) < 0.5, 1.0, 0.41))
    if kind == "equal rows":
        return np.outer(np.ones(m), v)
    return r.normal(size=(m, n))


def most(kind, steps, coefficients, want):
    return (8e-4 * steps if kind == "half" else 1e-2 if kind in ("two values", "equal rows") else 3e-3) + 2.0 ** -22 * abs(coefficients[0]) ** steps / np.linalg.norm(want)


SIZES = [(64, 300), (128, 128), (129, 129), (255, 129), (160, 200), (129, 4000), (400, 300), (1000, 600)]


@pytest.mark.parametrize("kind", ["one", "sixteen", "graded", "half", "two values", "equal rows", "plain"])
@pytest.mark.parametrize("m,n", SIZES)
def test_few_directions(ah, m, n, kind):
    g = common.up(matrix(kind, m, n), f32=True)
    u = common.down(g)
    for steps, coefficients in ((5, DEFAULT), (6, DEFAULT), (8, DEFAULT), (10, DEFAULT), (1, DEFAULT), (8, (1.875, -1.25, 0.375)), (20, (1.5, -0.5, 0.0))):
        common.say("few directions", m, n, kind, steps, coefficients)
        want = orc.newton_schulz(u, steps=steps, coefficients=coefficients)
        got = common.down(ah.adahop_orthogonalize(g, dtype=torch.float32, steps=steps, coefficients=coefficients))
        off = common.distance(got, want)
        print("   off", off, flush=True)
        assert off <= most(kind, steps, coefficients, want), (steps, coefficients)


@pytest.mark.parametrize("kind", ["one", "sixteen"])
def test_update_along_few_directions(ah, kind):
    """A weight of 160 x 200 that has seen few tokens, eight steps."""
    common.say("update", kind)
    g = common.up(matrix(kind, 160, 200), f32=True)
    w, mom = (torch.zeros(160, 200, device="cuda") for _ in range(2))
    ah.adahop_muon_update(w, g, mom, 1.0, scale=1.0, steps=8)
    want = -orc.newton_schulz(common.down(g) * 1.95, steps=8)
    assert common.distance(common.down(w), want) <= most(kind, 8, DEFAULT, want) + 2.0 ** -23
