"""Which kernels the operators behind the last block take for which sizes (no GPU): what the queries refuse, and that the tests of the kernels have a size for each one that any
size reaches."""
import random

import pytest

pytest.importorskip("torch")

from paper_2604_02525_amd import binding as ah  # noqa: E402
import test_gpu_linear_ce_kernels as loss  # noqa: E402
import test_gpu_newton_schulz_kernels as updates  # noqa: E402


def test_refused():
    for call in (lambda *a: ah.adahop_debug_linear_ce_plan(*a), lambda *a: ah.adahop_debug_newton_schulz_plan(a[0], *a[2:])):
        for a in ((-1, 5, 5, 0), (5, 5, 0, 1), (5, 5, 5, 3), (5, 5, 5, -1), (1 << 22, 5, 5, 0)):
            with pytest.raises(ah.AdahopError):
                call(*a)


def of_loss(T, D, V):
    """The kernels: product, tile, alone, slices or not"""
    return {(i, tile, alone, slices > 1) for i in range(3) for tile, alone, slices in [ah.adahop_debug_linear_ce_plan(T, V, D, i)]}


def of_update(m, n):
    """The same, and from which side and with how many numbers the iterate enters A and the step"""
    how = ("wide" if m <= n else "tall", min(m, n) <= 128)
    return {(i, tile, alone, slices > 1, how if i != 1 else ()) for i in range(3) for tile, alone, slices in [ah.adahop_debug_newton_schulz_plan(m, n, i)]}


def log_uniform(r, low, high):
    return int(round(low * (high / low) ** r.random()))


def test_the_tests_of_the_kernels_have_a_size_for_each():
    for T, D, V, *wanted in loss.SIZES:
        loss.check_plan(ah, T, D, V, wanted)
    for m, n, *wanted in updates.SIZES:
        updates.check_plan(ah, m, n, wanted)
    tested = set.union(*(of_loss(T, D, V) for T, D, V, *_ in loss.SIZES))
    r = random.Random(0)
    for _ in range(4000):
        T, D, V = log_uniform(r, 1, 20000), log_uniform(r, 1, 10000), log_uniform(r, 1, 140000)
        assert of_loss(T, D, V) <= tested, (T, D, V, of_loss(T, D, V) - tested)
    tested = set.union(*(of_update(m, n) for m, n, *_ in updates.SIZES))
    for _ in range(4000):
        m, n = log_uniform(r, 1, 32000), log_uniform(r, 1, 65536)
        assert of_update(m, n) <= tested, (m, n, of_update(m, n) - tested)
        assert of_update(n, m) <= tested, (n, m, of_update(n, m) - tested)
