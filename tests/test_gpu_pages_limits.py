"""The paged 4-bit cache where a call meets its limits: waits that run out, other streams, kept status words."""
import numpy as np
import pytest
import torch

from paper_2411_10803_b200 import binding as md
from paper_2411_10803_b200 import build as md_build
from test_gpu_pages import Case, i32, queries, status, workspace

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
