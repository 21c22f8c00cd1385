"""Attention over the paged 4-bit cache where the channel groups of V, or the keys, are of very different sizes."""
import numpy as np
import pytest
import torch

from oracle import pages
from paper_2411_10803_b200 import build as md_build
from test_gpu_pages import BF16, FP16, Case, f64, queries

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


def bounds(c, q, causal):
    """-> (out in 64 bits, how far a result may be off): half a step of the result; P s in fp16 times the codes; P in 11 bits times the
    centres (it has 16, which leaves room for fp32 sums over a few hundred keys); and what a logit's error makes of the probabilities,
    24 roundings of at most 2^-22 of its magnitudes."""
    q = f64(q)
    n, n_q, q_heads, d = q.shape
    group = q_heads // c.heads
    k, v = pages.values(c.ck, c.sk, c.zk), pages.values(c.cv, c.sv, c.zv)
    z = np.repeat(np.abs(c.zv), 32, -1)
    codes = np.abs(v - np.repeat(c.zv, 32, -1))
    kz = np.repeat(np.abs(c.zk), 32, -1)
    mass = np.abs(k - np.repeat(c.zk, 32, -1)) + kz
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for s, t, j in np.ndindex(n, n_q, q_heads):
        h, seen = j // group, int(c.lens[s]) - (n_q - 1 - t if causal else 0)
        if seen <= 0:
            continue
        x = k[s, h, :seen] @ q[s, t, j] * d ** -0.5
        p = np.exp(x - x.max())
        p /= p.sum()
        dz = 24 * 2.0 ** -22 * (mass[s, h, :seen] @ np.abs(q[s, t, j])).max() * d ** -0.5 + 2.0 ** -20
        out[s, t, j] = p @ v[s, h, :seen]
        tol[s, t, j] = BF16 * np.abs(out[s, t, j]) + (FP16 + 2 * dz) * (1 + BF16) * (p @ (codes[s, h, :seen] + z[s, h, :seen])) + 1e-30
    return out, tol


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,n_q", ROWS)
def test_centres_far_from_zero_that_cancel(group, n_q, d, causal):
    """Values of +300 and -300 in turn with a spread of one: the centres are the result, and what P loses before it meets them is not
    made up for by its sum."""
    rng = np.random.default_rng(n_q * group)
    lens = [2, 3, 5, 8, 13, 40, 300, 1, 0]
    v = rng.standard_normal((9, 2, 300, d)) + 300.0 * (-1.0) ** np.arange(300)[:, None]
    c = Case(rng, lens, heads=2, d=d, k=0.3 * rng.standard_normal(v.shape), v=v)
    q = queries(rng, 9, n_q, 2 * group, d)
    out, code = c.attend(q, causal)
    want, tol = bounds(c, q, causal)
    off = np.abs(f64(out) - want)
    assert code == [0, 0] and (off <= tol).all(), (off / np.maximum(tol, 1e-30)).max()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,n_q", ROWS)
def test_products_of_keys_that_cancel(group, n_q, d):
    """Channel pairs with one value of K and opposite values of q: thousands of nats of products, of which nothing is left but the last
    group's ordinary logits.  Beside that of the result's type the error is that of fp32 sums: some 2^-23 of 15 scales times q, 10^-3 nats."""
    rng = np.random.default_rng(d + group)
    n = 400
    k = np.repeat(rng.standard_normal((2, 1, n, d // 2)), 2, -1)
    q = np.empty((2, n_q, group, d))
    q[..., 0::2] = 1000 * rng.standard_normal((2, n_q, group, d // 2))
    q[..., 1::2] = -q[..., 0::2]
    q[..., -32:] = rng.standard_normal((2, n_q, group, 32))
    c = Case(rng, [n, n], heads=1, d=d, k=k, v=rng.standard_normal((2, 1, n, d)))
    q = torch.from_numpy(q).cuda().bfloat16()
    out, code = c.attend(q, causal=False)
    want, _ = bounds(c, q, False)
    rounding = np.linalg.norm(pages.to_bf16(want) - want)
    assert code == [0, 0] and np.linalg.norm(f64(out) - want) <= 1.15 * rounding, np.linalg.norm(f64(out) - want) / rounding


@pytest.mark.parametrize("group,n_q", ROWS)
def test_keys_of_the_largest_numbers_there_are(group, n_q):
    """Keys of 10^37 and queries of 10^-33: logits of some 10^4, so that nearly all of a row's share is one key's."""
    rng = np.random.default_rng(6)
    v = rng.standard_normal((2, 1, 200, 128))
    c = Case(rng, [200, 7], heads=1, k=2e37 * rng.standard_normal(v.shape).clip(-3, 3), v=v)
    q = queries(rng, 2, n_q, group, 128, 1e-33)
    got = f64(c.check(q, causal=False))
    k, v = pages.values(c.ck, c.sk, c.zk)[:, 0], pages.values(c.cv, c.sv, c.zv)[:, 0]
    x = np.einsum("bthd,bjd->bthj", f64(q), k) * 128 ** -0.5
    x[1, ..., 7:] = -np.inf
    best = np.sort(x, -1)
    sure = best[..., -1] - best[..., -2] > 1e-3 * np.abs(best[..., -1])      # (what fp32 sums tell apart, and tens of nats)
    want = np.stack([v[b][x[b].argmax(-1)] for b in range(2)])
    tol = BF16 * np.abs(want) + FP16 * (np.abs(c.zv).max() + 8 * c.sv.max())
    assert sure.any() and (np.abs(got - want) <= tol)[sure].all()
