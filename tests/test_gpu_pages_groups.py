"""Attention over the paged 4-bit cache where the channel groups of V, or the keys, are of very different sizes."""
import numpy as np
import pytest
import torch

from paper_2411_10803_b200 import build as md_build
from test_gpu_pages import Case, queries

pytestmark = pytest.mark.gpu

ROWS = [(1, 1), (2, 1), (3, 1), (1, 5), (8, 1), (4, 4), (3, 9)]     # query heads to a K / V head, query tokens


@pytest.fixture(scope="module", autouse=True)
def _built():
    md_build.build()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,n_q", ROWS)
@pytest.mark.parametrize("power", [14, 20, 26, 60, -20, -60])
def test_groups_of_v_do_not_set_what_other_groups_are_rounded_to(d, group, n_q, power):
    """One group of 32 channels 2^power times the others: each is as exact as if it were alone."""
    rng = np.random.default_rng(power + 100)
    lens = [300, 0, 17, 1]
    v = rng.standard_normal((4, 2, 300, d))
    v[:, 0, :, :32] *= 2.0 ** power
    v[:, 1, :, -32:] *= 2.0 ** power
    c = Case(rng, lens, heads=2, d=d, k=rng.standard_normal(v.shape), v=v)
    c.check(queries(rng, 4, n_q, 2 * group, d))


@pytest.mark.parametrize("group,n_q", ROWS)
@pytest.mark.parametrize("d", [64, 128])
def test_groups_of_v_that_grow_and_fade_at_different_keys(d, group, n_q):
    """Every group has a hump of 2^40 at keys of its own, and every query row attends to another hump."""
    rng = np.random.default_rng(7)
    n, groups = 500, d // 32
    at = np.arange(n)[:, None] - (np.arange(groups) + 0.5) * n / groups
    v = rng.standard_normal((1, 1, n, d)) * np.repeat(np.exp2(np.clip(40 - np.abs(at) / 2, -40, 40)), 32, -1)
    # queries: one direction of K per hump, so that row i sits on hump i mod groups
    k = 0.2 * rng.standard_normal((1, 1, n, d))
    for g in range(groups):
        k[0, 0, np.abs(at[:, g]) < 40, g * 32] += 12
    q = 0.3 * np.random.default_rng(8).standard_normal((1, n_q, group, d))
    for i in range(n_q * group):
        q[0, i // group, i % group, (i % groups) * 32] = 6
    c = Case(rng, [n], heads=1, d=d, k=k, v=v)
    c.check(torch.from_numpy(q).cuda().bfloat16(), causal=False)


@pytest.mark.parametrize("group,n_q", [(1, 1), (4, 1), (2, 6)])
def test_groups_of_v_far_apart_in_a_sequence_that_many_ctas_share(group, n_q):
    rng = np.random.default_rng(9)
    v = rng.standard_normal((1, 1, 7001, 128)) * np.repeat(np.exp2([0, 24, -24, 48]), 32)
    c = Case(rng, [7001], heads=1, page=64, k=rng.standard_normal(v.shape), v=v)
    c.check(queries(rng, 1, n_q, group, 128))
