"""The paged 4-bit cache where a call meets its limits: waits that run out, other streams, kept status words."""
import numpy as np
import pytest
import torch

from oracle import pages
from paper_2411_10803_b200 import binding as md
from paper_2411_10803_b200 import build as md_build
from test_gpu_pages import Case, f64, i32, queries, status, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    md_build.build()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,heads,group,n_q", [
    ([0, 40, 700, 3, 0], 3, 1, 1), ([2600], 1, 2, 1), ([9000, 40], 1, 4, 1), ([300] * 9, 2, 3, 5), (list(range(0, 90)), 2, 1, 1),
])
def test_a_wait_that_runs_out_in_some_lanes_ends_the_call(d, lens, heads, group, n_q):
    """The lanes of a warp each have a clock to give up by, so one may while another's copy lands: the warp gives up as one, the call
    comes back and says so, and the same call with ordinary waits on a zeroed workspace is right."""
    c = Case(np.random.default_rng(len(lens)), lens, heads=heads, d=d, page=32)
    q = queries(np.random.default_rng(d), len(lens), n_q, heads * group, d)
    sizes = dict(q_heads=heads * group, n_q=n_q, causal=1, **c.base)
    cfg, bad = md.PageConfig(**sizes), md.PageConfig(flags=md.MUSTDROP_PAGE_FLAG_DEBUG_TIMEOUT, **sizes)
    ws, out, table, n = workspace(cfg), torch.full_like(q, 77.0), i32(c.table), i32(c.lens)
    assert md.mustdrop_page_workspace_bytes(bad) == ws.numel()
    for _ in range(3):
        assert md.mustdrop_page_attend(bad, q, c.pool, table, n, out, ws) == md.MUSTDROP_OK
        assert status(ws)[0] == md.MUSTDROP_ERR_TIMEOUT
        empty = torch.from_numpy(c.lens == 0).cuda()
        assert not out[empty].any()                 # (zeros of sequences without keys wait for nothing)
        ws.zero_()
        c.check(q, ws=ws)


@pytest.mark.parametrize("scale", [1e-7, 1e-12, 1e-25, 1e-38, 1e-44])
@pytest.mark.parametrize("group,n_q", [(1, 1), (2, 1), (4, 1), (3, 5)])
def test_scales_down_to_the_smallest_there_is(scale, group, n_q):
    """Every visible key has the same share, hidden ones none - for queries of zeros (a padded row) as well."""
    c = Case(np.random.default_rng(3), [37, 5, 0, 600], heads=2, d=128)
    q = queries(np.random.default_rng(4), 4, n_q, 2 * group, 128)
    q[:, :, ::2] = 0
    c.check(q, scale=scale)
    c.check(torch.zeros_like(q), scale=scale, causal=False)


def test_the_largest_scale_over_keys_of_zeros():
    rng = np.random.default_rng(5)
    c = Case(rng, [50], heads=1, d=64, k=np.zeros((1, 1, 50, 64)), v=rng.standard_normal((1, 1, 50, 64)))
    for rows in (1, 2, 5):
        c.check(queries(rng, 1, 2, rows, 64, 3e7), scale=1e37)


LONG = 40_000_000      # clock cycles that hold a stream up: some 20 ms


def filled(n, heads=2, rows=40):
    cache = md.PagedCache(n_seq=n, n_heads=heads, n_pages=8 * n, max_pages=8, max_q=2)
    gen = torch.Generator(device="cuda").manual_seed(n)
    k, v = (torch.randn((n, heads, rows, 128), device="cuda", generator=gen).bfloat16() for _ in range(2))
    cache.store(cache.extend(torch.full((n,), rows, dtype=torch.int32, device="cuda"), rows), k, v)
    cache.attend(torch.zeros((n, 1, heads, 128), dtype=torch.bfloat16, device="cuda"))     # (first calls take longer than the delay)
    torch.cuda._sleep(1000)
    return cache


class Held:
    """A stream of another library: something with a raw handle."""

    def __init__(self, stream):
        self.cuda_stream = stream.cuda_stream


KINDS = {"torch": lambda s: s, "raw": lambda s: s.cuda_stream, "held": Held}


@pytest.mark.parametrize("kind", sorted(KINDS))
def test_results_of_a_call_on_another_stream_are_not_handed_out_again(kind):
    cache = filled(64)
    q = queries(np.random.default_rng(1), 64, 1, 2, 128)
    side = torch.cuda.Stream()
    on = KINDS[kind](side)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    out = cache.attend(q, stream=on)                   # pending behind the delay, and dropped
    slots = cache.extend(torch.zeros(64, dtype=torch.int32, device="cuda"), 37, stream=on)
    del out, slots
    ours = [torch.full((64, 1, 2, 128), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    more = [torch.full((64, 37), 9, dtype=torch.int32, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert all((x == 5).all() for x in ours) and all((x == 9).all() for x in more)
    assert cache.device_status() == (0, 0)


def test_results_of_a_call_on_another_stream_use_no_memory_still_read_on_this_one():
    cache = filled(64)
    q = queries(np.random.default_rng(1), 64, 1, 2, 128)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    before, copy = torch.full((64, 1, 2, 128), 3.0, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(q)
    torch.cuda.synchronize()
    torch.cuda._sleep(LONG)
    copy.copy_(before)                                 # pending on the current stream, and its source dropped
    del before
    out = cache.attend(q, stream=side)
    torch.cuda.synchronize()
    assert (copy == 3).all()
    assert torch.equal(out, cache.attend(q))


def test_arguments_of_a_call_on_another_stream_may_be_dropped():
    cache = filled(64)
    q = queries(np.random.default_rng(1), 64, 1, 2, 128)
    want = cache.attend(q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    out, mine = torch.zeros_like(q), q.clone()
    side.wait_stream(torch.cuda.current_stream())
    cache.attend(mine, out=out, stream=side)
    del mine
    others = [torch.full_like(q, 50.0) for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(out, want) and all((x == 50).all() for x in others)


@pytest.mark.parametrize("raw", [False, True])
def test_the_status_of_another_stream_is_read_behind_its_calls(raw):
    cache = filled(3)
    side = torch.cuda.Stream()
    on = side.cuda_stream if raw else side
    add, slots = torch.tensor([1, 9, 1], dtype=torch.int32, device="cuda"), torch.empty((3, 1), dtype=torch.int32, device="cuda")
    assert cache.device_status() == cache.device_status(on) == (0, 0)
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    cache.extend(add, 1, slots, stream=on)             # more tokens than rows for sequence 1
    assert cache.device_status(on) == (md.MUSTDROP_ERR_BAD_LENGTH, 1)
    assert cache.device_status() == (md.MUSTDROP_ERR_BAD_LENGTH, 1) and cache.len.tolist() == [41, 40, 41]


def test_a_status_that_was_cleared_does_not_hide_the_next():
    cache = md.PagedCache(n_seq=3, n_heads=2, n_pages=4, max_pages=8, max_q=2)
    i = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    rows = queries(np.random.default_rng(2), 3, 2, 16, 128)
    cache.store(cache.extend(i(16, 16, 16), 16), rows, rows)
    cache.extend(i(0, 33, 0), 40)                      # two pages asked for, one is free
    assert cache.device_status() == (md.MUSTDROP_ERR_NO_PAGES, 1) and cache.len.tolist() == [16, 16, 16]
    cache.extend(i(0, 0, 41), 40)                      # more tokens than rows: hidden behind the first
    assert cache.device_status(clear=True) == (md.MUSTDROP_ERR_NO_PAGES, 1)
    assert cache.device_status() == (0, 0)
    cache.extend(i(0, 0, 41), 40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert cache.device_status(side, clear=True) == (md.MUSTDROP_ERR_BAD_LENGTH, 2)
    torch.cuda.current_stream().wait_stream(side)
    q = queries(np.random.default_rng(1), 3, 1, 2, 128)
    out = cache.attend(q)
    assert cache.device_status(clear=True) == cache.device_status() == (0, 0)
    cache.workspace[:1024] = 255                       # what a call that timed out may leave: a status and counters
    assert cache.device_status(clear=True)[0] != 0
    assert torch.equal(out, cache.attend(q)) and cache.device_status() == (0, 0)


@pytest.mark.parametrize("group,n_q", [(1, 1), (4, 1)])
def test_the_longest_sequence_there_can_be(group, n_q):
    """2^30 - 5 tokens over eight pages that the table names again and again: the attention over those pages' 1024 tokens.  Beside the result
    type's half step, a warp's sums are cut at each of its 38 thousand chunks, by 2^-23 at most and half of that on average: 5e-3 of the values."""
    rng = np.random.default_rng(group)
    d, page, n_pages, length = 64, 128, 8, 2 ** 30 - 5
    sizes = dict(n_seq=1, n_heads=1, head_dim=d, page=page, n_pages=n_pages)
    k, v = queries(rng, 1, 1, 1024, d), queries(rng, 1, 1, 1024, d)
    store = md.PageConfig(rows=1024, **sizes)
    pool = torch.empty(md.mustdrop_page_pool_bytes(store), dtype=torch.uint8, device="cuda")
    assert md.mustdrop_page_store(store, i32(np.arange(1024))[None], k, v, pool) == md.MUSTDROP_OK
    cfg = md.PageConfig(q_heads=group, n_q=n_q, max_pages=2 ** 23, **sizes)
    table = torch.arange(2 ** 23, dtype=torch.int32, device="cuda") % n_pages
    q, ws = queries(rng, 1, n_q, group, d), workspace(cfg)
    out = torch.zeros_like(q)
    assert md.mustdrop_page_attend(cfg, q, pool, table, i32([length]), out, ws) == md.MUSTDROP_OK
    assert status(ws) == [0, 0]
    kk, vv = (pages.values(*pages.quantise(f64(x)))[0, 0] for x in (k, v))
    x = f64(q)[0, 0] @ kk.T * d ** -0.5
    p = np.exp(x - x.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    assert (np.abs(f64(out)[0, 0] - p @ vv) <= 2.0 ** -8 * np.abs(p @ vv) + 5e-3 * (p @ np.abs(vv)) + 2.0 ** -11 * np.abs(vv).max()).all()
