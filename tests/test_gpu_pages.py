"""The paged 4-bit cache on the GPU against its plain statement in 64 bits (oracle/pages.py)."""
import numpy as np
import pytest
import torch

from oracle import pages
from paper_2411_10803_b200 import binding as md
from paper_2411_10803_b200 import build as md_build

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8      # half a step, relative
FP16 = 2.0 ** -11


@pytest.fixture(scope="module", autouse=True)
def _built():
    md_build.build()


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().bfloat16()


def f64(t):
    return t.double().cpu().numpy()


def status(ws):
    torch.cuda.synchronize()
    return ws[:8].view(torch.int32).tolist()


def workspace(cfg):
    return torch.zeros(md.mustdrop_page_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------ tables

def run_tables(add, lens, state, ring, table, page, rows, in_place=False, ws=None):
    cfg = md.PageConfig(n_seq=len(add), page=page, n_pages=len(ring), max_pages=table.shape[1], rows=rows)
    ws = workspace(cfg) if ws is None else ws
    d_len, d_state, d_ring, d_table = i32(lens), i32(state), i32(ring), i32(table)
    len_out, state_out = (d_len, d_state) if in_place else (torch.full_like(d_len, -7), torch.full_like(d_state, -7))
    slots = torch.full((len(add), rows), -9, dtype=torch.int32, device="cuda")
    assert md.mustdrop_page_tables(cfg, i32(add), d_len, d_state, len_out, state_out, d_ring, d_table, slots, ws) == md.MUSTDROP_OK
    code = status(ws)
    return [x.cpu().numpy() for x in (len_out, state_out, d_ring, d_table, slots)], code


def table_case(rng, n, page, wide, rows, free, grow, shrink):
    lens = rng.integers(0, wide * page + 1, n).astype(np.int32)
    lens = np.minimum(lens, wide * page - rows if wide * page > rows else 0).astype(np.int32)
    used = -(-lens // page)
    n_pages = int(used.sum()) + free
    ids = rng.permutation(n_pages).astype(np.int32)
    table = np.full((n, wide), -1, np.int32)
    table[np.arange(wide)[None] < used[:, None]] = ids[free:]
    head = int(rng.integers(0, n_pages))
    ring = np.full(n_pages, -1, np.int32)
    ring[(head + np.arange(free)) % n_pages] = ids[:free]
    add = rng.integers(0, rows + 1, n)
    add = np.where(rng.random(n) < shrink, -rng.integers(0, 2 * wide * page, n), np.where(rng.random(n) < grow, add, 0))
    return add.astype(np.int32), lens, np.array([head, free], np.int32), ring, table


@pytest.mark.parametrize("n,page,wide,rows,free", [
    (1, 16, 3, 1, 1), (1, 128, 70, 4097, 60), (3, 16, 8, 17, 2), (240, 16, 30, 1, 250), (513, 32, 9, 8, 300), (1025, 16, 4, 1, 500),
    (1531, 64, 12, 300, 3000), (97, 16, 700, 9000, 40000), (3000, 16, 5, 3, 3000),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_tables_are_the_plain_ones(n, page, wide, rows, free, in_place):
    rng = np.random.default_rng(n + page)
    for grow, shrink in ((1.0, 0.0), (0.7, 0.4)):
        case = table_case(rng, n, page, wide, rows, free, grow, shrink)
        *want, bad, short = pages.tables(*case, page, rows)
        got, code = run_tables(*case, page, rows, in_place)
        for name, a, b in zip(("len", "state", "ring", "table", "slots"), got, want):
            assert np.array_equal(a, b), name
        assert code[0] == (md.MUSTDROP_ERR_NO_PAGES if short else md.MUSTDROP_OK)
        assert not short or code[1] in short


def test_tables_in_a_long_run_of_calls_that_share_a_workspace():
    rng = np.random.default_rng(2)
    n, page, wide, n_pages = 1300, 16, 6, 3000
    state, lens = np.array([17, n_pages], np.int32), np.zeros(n, np.int32)
    ring, table = rng.permutation(n_pages).astype(np.int32), np.full((n, wide), -1, np.int32)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    for rows in (40, 1, 40, 7, 33, 40, 1, 40):
        add = rng.integers(-40, rows + 1, n).astype(np.int32)
        want = pages.tables(add, lens, state, ring, table, page, rows)
        got, _ = run_tables(add, lens, state, ring, table, page, rows, True, ws)
        for a, b in zip(got, want):
            assert np.array_equal(a, b)
        lens, state, ring, table = got[:4]


def test_tables_refuse_lengths_and_states_that_cannot_be():
    rng = np.random.default_rng(0)
    add, lens, state, ring, table = table_case(rng, 6, 16, 5, 20, 12, 1.0, 0.0)
    lens[1], add[2], lens[3], add[4] = -5, 21, 5 * 16 + 1, 2 ** 31 - 1
    *want, bad, short = pages.tables(add, lens, state, ring, table, 16, 20)
    got, code = run_tables(add, lens, state, ring, table, 16, 20)
    assert bad == [1, 2, 3, 4] and code[0] == md.MUSTDROP_ERR_BAD_LENGTH and code[1] in bad
    for a, b in zip(got, want):
        assert np.array_equal(a, b)
    for broken in ([-1, 3], [len(ring), 3], [0, -1], [0, len(ring) + 1]):
        add, lens = np.array([20, -3, 1], np.int32), np.array([0, 17, 1], np.int32)
        table3 = np.array([[0, 0], [1, 2], [3, 0]], np.int32)
        got, code = run_tables(add, lens, np.array(broken, np.int32), ring, table3, 16, 20)
        assert code[0] != md.MUSTDROP_OK
        assert got[0].tolist() == [0, 14, 2] and got[1].tolist() == broken          # no pages without a ring; none lost into it
        assert np.array_equal(got[2], ring) and np.array_equal(got[3], table3)
        assert (got[4][:2] == -1).all() and got[4][2, 0] == 3 * 16 + 1


def test_a_page_id_that_is_none_gives_no_slot():
    table = np.array([[99, -1]], np.int32)
    got, code = run_tables(np.array([3]), np.array([2]), np.array([0, 2]), np.array([0, 1]), table, 16, 4)
    assert got[4].tolist() == [[-1] * 4] and code == [md.MUSTDROP_ERR_BAD_PAGE, 0]


# ------------------------------------------------------------------ store and load

def rows_case(rng, n, heads, rows, d, token_major):
    shape = (n, rows, heads, d) if token_major else (n, heads, rows, d)
    out = []
    for _ in range(2):
        x = rng.standard_normal(shape) * np.exp2(rng.integers(-3, 4, shape[:-1] + (1,)))
        x[..., 3] *= 20
        t = bf16(x)
        out.append(t.transpose(1, 2) if token_major else t)
    return out


@pytest.mark.parametrize("n,heads,rows,d,page,begin,token_major", [
    (1, 1, 1, 128, 16, 0, False), (2, 3, 1, 64, 32, 13, True), (3, 2, 33, 128, 32, 5, True), (2, 5, 70, 64, 64, 3, False),
    (1, 2, 129, 128, 128, 2, False), (4, 1, 16, 128, 16, 0, True), (2, 40, 7, 128, 16, 9, False),
])
def test_store_writes_the_described_bytes_and_load_reads_them(n, heads, rows, d, page, begin, token_major):
    rng = np.random.default_rng(rows + d)
    k, v = rows_case(rng, n, heads, rows, d, token_major)
    wide = -(-(begin + rows) // page)
    n_pages = n * wide + 2
    ids = rng.permutation(n_pages)[:n * wide].reshape(n, wide)
    pos = begin + np.arange(rows)
    slots = (ids[:, pos // page] * page + pos % page).astype(np.int32)
    slots[-1, rows // 2] = -1 if rows > 2 else slots[-1, rows // 2]
    pool = torch.from_numpy(rng.integers(0, 256, (n_pages, heads, page // 16, 20 * d)).astype(np.uint8)).cuda()
    want = pool.cpu().numpy().copy()
    ks, vs = k.stride(), v.stride()
    cfg = md.PageConfig(n_seq=n, n_heads=heads, head_dim=d, page=page, n_pages=n_pages, rows=rows, k_stride_s=ks[0], k_stride_h=ks[1],
                        k_stride_r=ks[2], v_stride_s=vs[0], v_stride_h=vs[1], v_stride_r=vs[2])
    ws = workspace(cfg)
    assert md.mustdrop_page_store(cfg, i32(slots), k, v, pool, ws) == md.MUSTDROP_OK
    assert status(ws) == [0, 0]
    pages.store(want, slots, f64(k), f64(v))
    assert np.array_equal(pool.cpu().numpy(), want)        # bytes of other tokens included

    k_out, v_out = (torch.full((n, heads, rows, d), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert md.mustdrop_page_load(cfg, i32(slots), pool, k_out, v_out, ws) == md.MUSTDROP_OK
    wk, wv = (np.full((n, heads, rows, d), 3.0) for _ in range(2))
    pages.load(want, slots, wk, wv)
    # values are centre + scale * code in one fp32 rounding, then bf16: the same numbers
    assert np.array_equal(f64(k_out), pages.to_bf16(wk)) and np.array_equal(f64(v_out), pages.to_bf16(wv))
    only = torch.zeros_like(v_out)
    assert md.mustdrop_page_load(cfg, i32(slots), pool, None, only, None) == md.MUSTDROP_OK
    there = torch.from_numpy(slots >= 0).cuda()[:, None, :, None]
    assert torch.equal(only, torch.where(there, v_out, 0))


def test_slots_in_no_order_and_outside_the_pool():
    rng = np.random.default_rng(4)
    n, heads, rows, d, page, n_pages = 2, 2, 23, 128, 32, 3
    k, v = rows_case(rng, n, heads, rows, d, False)
    slots = rng.permutation(n_pages * page)[:n * rows].reshape(n, rows).astype(np.int32)
    slots[1, 3], slots[1, 9], slots[0, 5] = n_pages * page, 2 ** 31 - 1, -2 ** 31
    pool = torch.zeros((n_pages, heads, page // 16, 20 * d), dtype=torch.uint8, device="cuda")
    want = pool.cpu().numpy().copy()
    cfg = md.PageConfig(n_seq=n, n_heads=heads, head_dim=d, page=page, n_pages=n_pages, rows=rows)
    ws = workspace(cfg)
    assert md.mustdrop_page_store(cfg, i32(slots), k, v, pool, ws) == md.MUSTDROP_OK
    assert status(ws) == [md.MUSTDROP_ERR_BAD_PAGE, 1]
    pages.store(want, slots, f64(k), f64(v))
    assert np.array_equal(pool.cpu().numpy(), want)
    ws.zero_()
    out = torch.zeros((n, heads, rows, d), dtype=torch.bfloat16, device="cuda")
    assert md.mustdrop_page_load(cfg, i32(slots), pool, out, None, ws) == md.MUSTDROP_OK
    assert status(ws) == [md.MUSTDROP_ERR_BAD_PAGE, 1]
    assert not out[1, :, 3].any() and not out[1, :, 9].any() and not out[0, :, 5].any() and out[1, :, 4].any()


def test_values_at_the_ends_of_the_type():
    d, x = 128, np.zeros((1, 1, 10, 128))
    big = 3.3895314e38
    x[0, 0, 0] = -2.5                                   # one value throughout
    x[0, 0, 1, ::2] = big                               # the widest range there is
    x[0, 0, 1, 1::2] = -big
    x[0, 0, 2, :32] = np.inf                            # groups that hold what is no number
    x[0, 0, 3, 33] = np.nan
    x[0, 0, 4, 64:] = -np.inf
    x[0, 0, 5] = 1e-30 * np.arange(128)
    x[0, 0, 6] = 100 + np.arange(128) % 2 * 0.5         # a range of one step of the type
    x[0, 0, 7, 5] = 1.0
    x[0, 0, 8] = np.arange(128) - 64
    t = bf16(x)
    slots = np.arange(10, dtype=np.int32)[None]
    cfg = md.PageConfig(n_seq=1, n_heads=1, head_dim=d, page=16, n_pages=1, rows=10)
    pool = torch.zeros(md.mustdrop_page_pool_bytes(cfg), dtype=torch.uint8, device="cuda")
    out = [torch.zeros_like(t) for _ in range(2)]
    assert md.mustdrop_page_store(cfg, i32(slots), t, t, pool) == md.MUSTDROP_OK
    assert md.mustdrop_page_load(cfg, i32(slots), pool, *out) == md.MUSTDROP_OK
    want = pages.to_bf16(pages.values(*pages.quantise(f64(t))))
    for o in out:
        assert np.array_equal(f64(o), want, equal_nan=True)
    assert np.isnan(want[0, 0, 2, :32]).all() and np.isfinite(want[0, 0, 2, 32:]).all() and np.isfinite(want[0, 0, 1]).all()


def test_codes_of_groups_of_every_magnitude():
    # members that are near whole and half steps of their group's scale, which runs over the exponents of the type
    rng = np.random.default_rng(31)
    n, rows, d = 8, 128, 128
    step = 2.0 ** rng.integers(-133, 124, (n, 1, rows, 4, 1)) * (1 + rng.integers(0, 128, (n, 1, rows, 4, 1)) / 128)
    off = rng.integers(-12, 12, (n, 1, rows, 4, 1)) * step * rng.integers(0, 2, (n, 1, rows, 4, 1)) / 4
    x = np.clip(rng.integers(0, 31, (n, 1, rows, 4, 32)) / 2 * step - 7.5 * step + off, -3.3e38, 3.3e38)
    x[..., 5] *= 2.0 ** -18
    t = bf16(x.reshape(n, 1, rows, d))
    slots = np.arange(n * rows, dtype=np.int32).reshape(n, rows)
    for first in (0, 1):                                 # many rows of a sequence; one row of each
        s, y = (slots, t) if first == 0 else (slots.reshape(-1, 1), t.reshape(n * rows, 1, 1, d))
        cfg = md.PageConfig(n_seq=s.shape[0], n_heads=1, head_dim=d, page=16, n_pages=n * rows // 16, rows=s.shape[1])
        pool = torch.zeros((n * rows // 16, 1, 1, 20 * d), dtype=torch.uint8, device="cuda")
        want = pool.cpu().numpy().copy()
        assert md.mustdrop_page_store(cfg, i32(s), y, y, pool) == md.MUSTDROP_OK
        pages.store(want, s, f64(y), f64(y))
        assert np.array_equal(pool.cpu().numpy(), want)


# ------------------------------------------------------------------ attend

class Case:
    """A filled cache, and what it stands for in 64 bits."""

    def __init__(self, rng, lens, heads=2, d=128, page=16, garbage=255, k_scale=1.0, k=None, v=None):
        self.lens, self.heads, self.d, self.page = np.asarray(lens, np.int32), heads, d, page
        n, rows = len(lens), max(1, max(lens))
        if k is None:
            k, v = rng.standard_normal((n, heads, rows, d)) * k_scale, rng.standard_normal((n, heads, rows, d))
            k[..., 7] *= 4
        k, v = bf16(k), bf16(v)
        used = -(-self.lens // page)
        wide = max(1, int(used.max())) + 1
        self.n_pages = int(used.sum()) + 3
        ids = rng.permutation(self.n_pages)[:int(used.sum())]
        self.table = np.full((n, wide), -1, np.int32)
        self.table[np.arange(wide)[None] < used[:, None]] = ids
        pos = np.arange(rows)
        slots = np.where(pos[None] < self.lens[:, None], self.table[:, np.minimum(pos // page, wide - 1)].astype(np.int64) * page + pos % page, -1)
        self.base = dict(n_seq=n, n_heads=heads, head_dim=d, page=page, n_pages=self.n_pages, max_pages=wide)
        cfg = md.PageConfig(rows=rows, **self.base)
        self.pool = torch.full((md.mustdrop_page_pool_bytes(cfg),), garbage, dtype=torch.uint8, device="cuda")
        assert md.mustdrop_page_store(cfg, i32(slots), k, v, self.pool) == md.MUSTDROP_OK
        self.ck, self.sk, self.zk = pages.quantise(f64(k))
        self.cv, self.sv, self.zv = pages.quantise(f64(v))

    def attend(self, q, causal=True, scale=0.0, lens=None, table=None, ws=None, **strides):
        n, n_q, q_heads, d = q.shape
        cfg = md.PageConfig(q_heads=q_heads, n_q=n_q, causal=int(causal), scale=scale, **strides, **self.base)
        ws = workspace(cfg) if ws is None else ws
        out = torch.full((n, n_q, q_heads, d), 77.0, dtype=torch.bfloat16, device="cuda")
        st = md.mustdrop_page_attend(cfg, q, self.pool, i32(self.table if table is None else table), i32(self.lens if lens is None else lens), out, ws)
        assert st == md.MUSTDROP_OK
        return out, status(ws)

    def want(self, q, causal=True, scale=None, hidden=None):
        """-> (out in 64 bits, how far a result may be off)."""
        q = f64(q)
        n, n_q, q_heads, d = q.shape
        group = q_heads // self.heads
        scale = scale or d ** -0.5
        k, v = pages.values(self.ck, self.sk, self.zk), pages.values(self.cv, self.sv, self.zv)
        zv, vc = np.repeat(np.abs(self.zv), 32, -1), np.abs(v - np.repeat(self.zv, 32, -1))
        out, tol = np.zeros(q.shape), np.zeros(q.shape)
        for s in range(n):
            L = int(self.lens[s])
            for t in range(n_q):
                lim = L - n_q + 1 + t if causal else L
                seen = [x for x in range(max(0, lim)) if hidden is None or not hidden[s][x]]
                if not seen:
                    continue
                for j in range(q_heads):
                    h = j // group
                    kk, vv = k[s, h, seen], v[s, h, seen]
                    z = kk @ q[s, t, j] * scale
                    p = np.exp(z - z.max())
                    p /= p.sum()
                    o = p @ vv
                    # products of a logit: at most 24 additions of at most 2^-22 of the sum of magnitudes (codes, then centres)
                    mass = (np.abs(kk - np.repeat(self.zk[s, h, seen], 32, -1)) + np.repeat(np.abs(self.zk[s, h, seen]), 32, -1)) @ np.abs(q[s, t, j]) * scale
                    dz = 24 * 2.0 ** -22 * mass.max() + 2.0 ** -20
                    tol[s, t, j] = BF16 * np.abs(o) + p @ (FP16 * vc[s, h, seen] + BF16 * zv[s, h, seen]) * (1 + BF16) + \
                        2 * dz * (p @ (vc[s, h, seen] + zv[s, h, seen])) + 1e-30
                    out[s, t, j] = o
        return out, tol

    def check(self, q, causal=True, scale=0.0, **kw):
        out, code = self.attend(q, causal, scale, **kw)
        assert code == [0, 0]
        want, tol = self.want(q, causal, scale)
        off = np.abs(f64(out) - want)
        assert np.isfinite(f64(out)).all()
        assert (off <= tol).all(), (off / tol).max()
        return out


def queries(rng, n, n_q, q_heads, d, size=1.0):
    return bf16(rng.standard_normal((n, n_q, q_heads, d)) * size)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_attend_lengths_around_chunks_and_pages(d, page):
    rng = np.random.default_rng(d + page)
    lens = [0, 1, 2, 15, 16, 17, 31, 33, page - 1, page, page + 1, 2 * page + 5, 0, 300]
    c = Case(rng, lens, heads=2, d=d, page=page)
    c.check(queries(rng, len(lens), 1, 2, d))


@pytest.mark.parametrize("d,heads,group,n_q", [
    (128, 1, 1, 1), (128, 3, 2, 1), (64, 1, 8, 1), (128, 2, 1, 5), (128, 2, 3, 3), (128, 1, 4, 4), (64, 2, 2, 7), (128, 1, 8, 5),
    (64, 1, 1, 37), (128, 2, 1, 128), (128, 1, 71, 1),
])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_query_tokens_and_shared_heads(d, heads, group, n_q, causal):
    rng = np.random.default_rng(heads * group * n_q)
    lens = [0, 1, 3, 40, 133]
    c = Case(rng, lens, heads=heads, d=d, page=32)
    c.check(queries(rng, len(lens), n_q, heads * group, d), causal)


def test_attend_one_long_sequence_is_split_over_the_gpu():
    rng = np.random.default_rng(9)
    c = Case(rng, [20011], heads=1, d=128, page=64)
    c.check(queries(rng, 1, 1, 1, 128))
    c.check(queries(rng, 1, 2, 7, 128))


@pytest.mark.parametrize("lens,heads,group,n_q,d", [
    ([3000], 2, 4, 1, 128), ([2500], 8, 1, 1, 64), ([9000], 1, 1, 1, 128), ([1300, 0, 4100], 2, 2, 1, 128), ([0, 5, 2600, 700], 3, 8, 2, 64),
    ([700 + 90 * i for i in range(32)], 1, 1, 1, 128), ([700 + 90 * i for i in range(33)], 1, 1, 1, 128), ([2100] * 4, 4, 3, 1, 64),
    ([40, 6000], 1, 9, 1, 128), ([1700] * 37, 4, 1, 1, 64),
])
def test_attend_few_units_get_whole_numbers_of_ctas(lens, heads, group, n_q, d):
    rng = np.random.default_rng(len(lens) * heads)
    c = Case(rng, lens, heads=heads, d=d, page=64)
    c.check(queries(rng, len(lens), n_q, heads * group, d))


def test_attend_many_ragged_sequences():
    rng = np.random.default_rng(10)
    lens = rng.integers(0, 90, 700)
    lens[5:60] = 0
    c = Case(rng, lens, heads=3, d=64, page=16)
    c.check(queries(rng, 700, 1, 3, 64))


def test_attend_more_sequences_than_threads_scan_at_once():
    rng = np.random.default_rng(11)
    c = Case(rng, rng.integers(0, 4, 4096), heads=1, d=64, page=16)
    c.check(queries(rng, 4096, 1, 1, 64))


@pytest.mark.parametrize("size,k_scale", [(60.0, 1.0), (1e-6, 1.0), (1.0, 30.0), (3e4, 1e-4), (1e-20, 1e20)])
def test_attend_logits_and_queries_of_any_size(size, k_scale):
    rng = np.random.default_rng(12)
    c = Case(rng, [200, 17, 1], heads=2, d=128, k_scale=k_scale)
    c.check(queries(rng, 3, 2, 2, 128, size))


def test_attend_logits_that_grow_along_the_keys():
    rng = np.random.default_rng(13)
    n = 400
    q = np.ones((1, 1, 1, 128))
    k = 0.05 * rng.standard_normal((1, 1, n, 128)) + (np.arange(n) * 0.02)[None, None, :, None]
    c = Case(rng, [n], heads=1, k=k, v=rng.standard_normal((1, 1, n, 128)))
    c.check(bf16(q))


def test_attend_scales_of_v_that_grow_and_shrink_along_the_keys():
    rng = np.random.default_rng(14)
    n = 300
    v = rng.standard_normal((1, 1, n, 128)) * np.exp2(np.clip(np.abs(np.arange(n) - 150) - 75, -60, 75))[None, None, :, None]
    c = Case(rng, [n], heads=1, k=rng.standard_normal((1, 1, n, 128)), v=v)
    c.check(queries(rng, 1, 1, 1, 128))
    v = rng.standard_normal((1, 1, n, 128)) + 300.0          # far from zero
    c = Case(rng, [n], heads=1, k=rng.standard_normal((1, 1, n, 128)), v=v)
    c.check(queries(rng, 1, 1, 1, 128))


@pytest.mark.parametrize("n_q", [1, 2, 5])
@pytest.mark.parametrize("where", [0, 100, 299])
def test_attend_a_large_value_that_nobody_attends_to_costs_no_precision(n_q, where):
    """Keys with a scale of V 2^20 times the others' and a logit 60 below: their share is nothing, and they must not set what the
    others are rounded to.  And the other way round: the others' share is nothing beside one key's."""
    rng = np.random.default_rng(where + n_q)
    n, q = 300, np.ones((1, n_q, 1, 128))
    k, v = 0.3 * rng.standard_normal((1, 1, n, 128)), rng.standard_normal((1, 1, n, 128))
    k[0, 0, where] = -60 / 128 ** 0.5
    v[0, 0, where] *= 2.0 ** 20
    c = Case(rng, [n], heads=1, k=k, v=v)
    c.check(bf16(q), causal=False)
    k[0, 0, where] = 30 / 128 ** 0.5
    v[0, 0, where] *= 2.0 ** -40
    c = Case(rng, [n], heads=1, k=k, v=v)
    c.check(bf16(q), causal=False)


def values64(x):
    """What stored rows stand for, float64 on the GPU (the statement of oracle/pages.py)."""
    g = x.double().unflatten(-1, (-1, 32))
    low, high = g.amin(-1), g.amax(-1)
    s = ((high / 2 - low / 2) / 7.5).float().bfloat16().double()[..., None]
    z = (low[..., None] + 8 * s).float().bfloat16().double()
    return (z + s * (torch.round((g - z) / s) + 8).clamp(0, 15) - 8 * s).flatten(-2)


@pytest.mark.parametrize("heads,n,L", [(2, 6, 3000), (32, 24, 1100)])
@pytest.mark.parametrize("group,n_q", [(1, 1), (2, 1), (4, 1), (3, 4)])
@pytest.mark.parametrize("size", [0.0, 1.0, 4.0])
def test_attend_is_as_exact_as_its_result_type(heads, n, L, group, n_q, size):
    """The error's norm over many rows against that of rounding the exact result to bf16, 1.15 times at most: the next terms are
    P in bf16 times centres (a third of the values, and not all of one sign) and P s in fp16 - (1 + 0.35^2 / 2 + 2^-6)^0.5 = 1.04.
    Sums that lose bits, or lose them to one side, show here and not in the bound of a single element; in the large case a
    warp adds up several hundred keys of one sequence."""
    gen = torch.Generator(device="cuda").manual_seed(heads + group)
    rng = np.random.default_rng(heads + group)
    d, page = 64, 64
    k, v = (torch.randn((n, heads, L, d), device="cuda", generator=gen).bfloat16() for _ in range(2))
    lens = i32(rng.integers(L // 3, L + 1, n))
    cache = md.PagedCache(n_seq=n, n_heads=heads, n_pages=n * (L // page + 2), max_pages=L // page + 2, head_dim=d, page=page,
                          q_heads=heads * group, max_q=n_q, causal=0)
    cache.store(cache.extend(lens, L), k, v)
    q = (torch.randn((n, n_q, heads * group, d), device="cuda", generator=gen) * size).bfloat16()
    out = cache.attend(q)
    z = torch.einsum("bthgd,bhjd->bhgtj", q.double().unflatten(2, (heads, group)), values64(k)) * d ** -0.5
    z = z.masked_fill(torch.arange(L, device="cuda") >= lens[:, None, None, None, None], -np.inf)
    want = torch.einsum("bhgtj,bhjd->bthgd", torch.softmax(z, -1), values64(v)).flatten(2, 3)
    own, rounding = (out.double() - want).norm(), (want.bfloat16().double() - want).norm()
    assert cache.device_status() == (0, 0) and own <= 1.15 * rounding, (own / rounding)


def test_attend_keys_of_one_value_and_zero_queries():
    rng = np.random.default_rng(15)
    k, v = np.full((1, 2, 50, 128), 0.75), np.full((1, 2, 50, 128), -1.5)
    c = Case(rng, [50], heads=2, k=k, v=v)
    out = c.check(queries(rng, 1, 1, 2, 128))
    assert (out == -1.5).all()
    c.check(torch.zeros((1, 1, 2, 128), dtype=torch.bfloat16, device="cuda"))


def test_attend_numbers_that_are_none_stay_with_who_sees_them():
    rng = np.random.default_rng(16)
    n = 40
    k, v = rng.standard_normal((2, 1, n, 128)), rng.standard_normal((2, 1, n, 128))
    v[0, 0, n - 1, 40] = np.nan              # the last key: query token 1 sees it, query token 0 does not
    k[1, 0, n - 1, 3] = np.inf
    c = Case(rng, [n, n], heads=1, k=k, v=v)
    q = queries(rng, 2, 2, 1, 128)
    out, code = c.attend(q)
    got = f64(out)
    assert code == [0, 0] and np.isfinite(got[0, 0]).all() and np.isfinite(got[1, 0]).all()
    assert np.isnan(got[0, 1, 0, 32:64]).all() and np.isfinite(got[0, 1, 0, :32]).all() and np.isfinite(got[0, 1, 0, 64:]).all()
    assert np.isnan(got[1, 1]).all()
    q2 = q.clone()
    q2[0, 0, 0, 5] = float("nan")
    got = f64(c.attend(q2)[0])
    assert np.isnan(got[0, 0]).all() and np.isfinite(got[1, 0]).all()


def test_attend_strided_queries_and_a_scale():
    rng = np.random.default_rng(17)
    c = Case(rng, [70, 9], heads=2, d=128)
    wide = queries(rng, 2, 6, 3, 256)                     # [n_seq, q_heads = 6, n_q = 3, 256]: head-major, half of every row
    q = wide[..., 128:].transpose(1, 2)
    want = c.check(q.contiguous(), scale=0.2)
    out, code = c.attend(q, scale=0.2, q_stride_s=q.stride(0), q_stride_t=q.stride(1), q_stride_h=q.stride(2))
    assert code == [0, 0] and torch.equal(out, want)


def test_attend_pages_that_are_none_and_lengths_that_cannot_be():
    rng = np.random.default_rng(18)
    c = Case(rng, [100, 60, 80], heads=2, d=128, page=16)
    table = c.table.copy()
    table[0, 2], table[1, 0], table[1, 1], table[1, 2], table[1, 3] = c.n_pages, -1, -2 ** 31, 2 ** 31 - 1, -1
    q = queries(rng, 3, 2, 4, 128)
    out, code = c.attend(q, table=table)
    assert code[0] == md.MUSTDROP_ERR_BAD_PAGE
    hidden = [[x // 16 < table.shape[1] and not 0 <= table[s, x // 16] < c.n_pages for x in range(100)] for s in range(3)]
    want, tol = c.want(q, hidden=hidden)
    assert (np.abs(f64(out) - want) <= tol).all()
    assert not out[1].any()                              # no page at all: no key
    lens = c.lens.copy()
    lens[1], lens[2] = -4, 80
    c.lens[1] = 0
    out, code = c.attend(q, lens=lens)
    want, tol = c.want(q)
    assert code == [md.MUSTDROP_ERR_BAD_LENGTH, 1] and (np.abs(f64(out) - want) <= tol).all()


def test_attend_more_keys_than_the_table_holds_are_left_out():
    rng = np.random.default_rng(19)
    c = Case(rng, [64], heads=1, d=64, page=16)
    c.table, c.base["max_pages"] = c.table[:, :4].copy(), 4
    out, code = c.attend(queries(np.random.default_rng(1), 1, 1, 1, 64), lens=np.array([2 ** 31 - 1]))
    assert code == [md.MUSTDROP_ERR_BAD_LENGTH, 0]
    want, tol = c.want(queries(np.random.default_rng(1), 1, 1, 1, 64))
    assert (np.abs(f64(out) - want) <= tol).all()


def test_attend_gives_the_same_bits_and_leaves_the_workspace_ready():
    rng = np.random.default_rng(20)
    c = Case(rng, rng.integers(0, 500, 23), heads=4, d=128, page=32)
    q = queries(rng, 23, 1, 8, 128)
    cfg = md.PageConfig(q_heads=8, n_q=1, **c.base)
    ws = workspace(cfg)
    first, _ = c.attend(q, ws=ws)
    for _ in range(20):
        again, code = c.attend(q, ws=ws)
        assert torch.equal(first, again) and code == [0, 0]


def test_a_pool_of_more_than_four_gigabytes():
    rng = np.random.default_rng(21)
    heads, page, n_pages = 32, 128, 7000                # 32 * 128 * 160 = 640 KB a page
    cfg = md.PageConfig(n_seq=1, n_heads=heads, page=page, n_pages=n_pages, max_pages=2, rows=200, q_heads=heads, n_q=1)
    pool = torch.empty(md.mustdrop_page_pool_bytes(cfg), dtype=torch.uint8, device="cuda")
    assert pool.numel() > 1 << 32
    table = np.array([[n_pages - 1, 6700]], np.int32)
    pos = np.arange(200)
    slots = i32(table[0, pos // page] * page + pos % page)[None]
    k, v = rows_case(rng, 1, heads, 200, 128, False)
    assert md.mustdrop_page_store(cfg, slots, k, v, pool) == md.MUSTDROP_OK
    got = [torch.zeros_like(k) for _ in range(2)]
    assert md.mustdrop_page_load(cfg, slots, pool, *got) == md.MUSTDROP_OK
    for x, y in zip((k, v), got):
        assert np.array_equal(f64(y), pages.to_bf16(pages.values(*pages.quantise(f64(x)))))
    q = queries(rng, 1, 1, heads, 128)
    out, ws = torch.zeros_like(q), workspace(cfg)
    assert md.mustdrop_page_attend(cfg, q, pool, i32(table), i32([200]), out, ws) == md.MUSTDROP_OK
    assert status(ws) == [0, 0]
    kk, vv = (torch.from_numpy(pages.values(*pages.quantise(f64(x))))[0] for x in (k, v))
    p = torch.softmax(torch.einsum("hjd,hd->hj", kk, q.double().cpu()[0, 0]) * 128 ** -0.5, -1)
    want = torch.einsum("hj,hjd->hd", p, vv)
    # half a step of the result, and of P s (fp16) and P (bf16) times the largest value and centre there is
    tol = BF16 * want.abs() + (2 * FP16 + BF16) * vv.abs().amax()
    assert ((out.double().cpu()[0, 0] - want).abs() <= tol).all()


# ------------------------------------------------------------------ together, as they are used

def test_a_pruned_prompt_and_its_decoded_tokens():
    """One pruning layer on a ragged batch, its kept rows into the cache, then tokens one by one - captured and replayed -
    with drafts of three taken back in between."""
    from paper_2411_10803_b200 import synth
    w = synth.WORKLOADS["c1_tiny"].with_(batch=3, n_vis=96, n_txt=12, n_heads=4, hidden=512, key_cnt=4, budget=24)
    d = synth.make_batch(w)
    up = lambda a: torch.from_numpy(a.view(np.int16)).cuda().view(torch.bfloat16)  # noqa: E731
    f = md.Filter(md.config_for(w, flags=md.MUSTDROP_FLAG_REBUILD_SEQUENCE))
    f.filter(up(d["q_text"]), up(d["k"]), up(d["v"]), up(d["hidden"]), i32(d["key_idx"]), i32(d["key_cnt"]))
    rng = np.random.default_rng(3)
    B, H, rows = 3, 4, f.config.out_rows
    cache = md.PagedCache(n_seq=B, n_heads=H, n_pages=40, max_pages=8, q_heads=8, max_q=3)
    cache.pool.fill_(255)
    cache.store(cache.extend(f.kept_cnt + (w.vis_start + w.n_txt), rows), f.k_out, f.v_out)
    keep = [f.k_out.clone(), f.v_out.clone()]             # the rows of every sequence so far
    f.close()

    def reference(q):
        n_q = q.shape[1]
        k, v = (torch.from_numpy(pages.values(*pages.quantise(f64(x)))) for x in keep)
        L = k.shape[2]
        z = torch.einsum("bthgd,bhjd->bhgtj", q.double().cpu().unflatten(2, (H, 2)), k) * 128 ** -0.5
        z = z.masked_fill(torch.arange(L)[None] > (L - n_q + torch.arange(n_q))[:, None], -np.inf)
        return torch.einsum("bhgtj,bhjd->bthgd", torch.softmax(z, -1), v).flatten(2, 3), v.abs().amax()

    def compare(out, q):
        want, top = reference(q)
        assert ((out.double().cpu() - want).abs() <= BF16 * want.abs() + (2 * FP16 + BF16) * top).all()

    assert cache.len.tolist() == [rows] * B
    k1, v1, q1 = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((B, 1, H, 128), (B, 1, H, 128), (B, 1, 8, 128)))
    one, slots, out = torch.ones(B, dtype=torch.int32, device="cuda"), torch.empty((B, 1), dtype=torch.int32, device="cuda"), torch.empty_like(q1)

    def decode():
        cache.extend(one, 1, slots)
        cache.store(slots, k1.transpose(1, 2), v1.transpose(1, 2))
        cache.attend(q1, out=out)

    def token():
        for x in (k1, v1, q1):
            x.copy_(bf16(rng.standard_normal(x.shape)))
        for i, x in enumerate((k1, v1)):
            keep[i] = torch.cat([keep[i], x.transpose(1, 2)], 2)

    token()
    decode()
    compare(out, q1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        decode()
    for step in range(20):
        token()
        graph.replay()
        compare(out, q1)
        if step % 6 == 5:                                 # three drafted tokens at once; two are taken back
            k3, v3, q3 = (bf16(rng.standard_normal((B, 3, n, 128))) for n in (H, H, 8))
            cache.store(cache.extend(one * 3, 3), k3.transpose(1, 2), v3.transpose(1, 2))
            held = list(keep)
            keep = [torch.cat([a, b.transpose(1, 2)], 2) for a, b in zip(held, (k3, v3))]
            compare(cache.attend(q3), q3)
            cache.extend(one * -2, 1)
            keep = [torch.cat([a, b.transpose(1, 2)[:, :, :1]], 2) for a, b in zip(held, (k3, v3))]
    assert cache.device_status() == (0, 0)
    cache.extend(one * -10000, 1)
    assert cache.len.tolist() == [0] * B and cache.ring_state.tolist()[1] == 40
    assert not cache.attend(q1).any()


def test_two_caches_on_two_streams():
    rng = np.random.default_rng(30)
    cases = [Case(rng, rng.integers(1, 900, 9), heads=8, d=128, page=16) for _ in range(2)]
    qs = [queries(rng, 9, 1, 8, 128) for _ in range(2)]
    alone = [c.attend(q)[0] for c, q in zip(cases, qs)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    cfgs = [md.PageConfig(q_heads=8, n_q=1, **c.base) for c in cases]
    ws, outs = [workspace(c) for c in cfgs], [torch.zeros_like(q) for q in qs]
    tables, lens = [i32(c.table) for c in cases], [i32(c.lens) for c in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, s in enumerate(streams):
            assert md.mustdrop_page_attend(cfgs[i], qs[i], cases[i].pool, tables[i], lens[i], outs[i], ws[i], s) == md.MUSTDROP_OK
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))


def test_the_owner_refuses_what_it_cannot_hand_on():
    cache = md.PagedCache(n_seq=2, n_heads=2, n_pages=8, max_pages=4)
    good = torch.zeros((2, 2, 3, 128), dtype=torch.bfloat16, device="cuda")
    add = torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    slots = cache.extend(add, 3)
    with pytest.raises(ValueError):
        cache.extend(add.long(), 3)
    with pytest.raises(ValueError):
        cache.extend(add.cpu(), 3)
    with pytest.raises(ValueError):
        cache.store(slots, good.float(), good)
    with pytest.raises(ValueError):
        cache.store(slots, good[:, :1], good)
    with pytest.raises(ValueError):
        cache.attend(good.transpose(1, 2)[:, :2])
    with pytest.raises(md.MustDropError):
        cache.store(slots, torch.zeros((2, 2, 3, 132), dtype=torch.bfloat16, device="cuda")[..., :128], good)   # rows of 264 bytes
    with pytest.raises(md.MustDropError):
        md.PagedCache(n_seq=2, n_heads=2, n_pages=8, max_pages=4, page=20)
    cache.store(slots, good, good)
    assert cache.device_status() == (0, 0)


def test_the_owner_takes_axes_of_one_element_and_refuses_expanded_ones():
    rng = np.random.default_rng(40)
    cache = md.PagedCache(n_seq=6, n_heads=2, n_pages=12, max_pages=2, max_q=2)
    k = queries(rng, 6, 2, 1, 128).as_strided((6, 2, 1, 128), (256, 128, 7, 1))       # a row axis whose stride says nothing
    slots = cache.extend(torch.ones(6, dtype=torch.int32, device="cuda"), 1)
    cache.store(slots, k, k)
    out = [torch.zeros((6, 2, 1, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache.load(slots, *out)
    want = pages.to_bf16(pages.values(*pages.quantise(f64(k))))
    assert np.array_equal(f64(out[0]), want) and np.array_equal(f64(out[1]), want)
    with pytest.raises(ValueError):
        cache.store(slots, k[:, :1].expand(6, 2, 1, 128), k)
    with pytest.raises(ValueError):
        cache.attend(queries(rng, 1, 1, 2, 128).expand(6, 1, 2, 128))
    # one layer's sequences: a slice of the tables (lengths and tables then begin at any four bytes)
    q = queries(rng, 3, 1, 2, 128)
    got = cache.attend(q, first=3)
    assert torch.equal(got.transpose(1, 2), out[1][3:])                               # one key each: its value
    assert cache.device_status() == (0, 0)


def test_the_first_calls_of_a_process_can_be_captured(tmp_path):
    """Kernels are loaded and set up by their first call, which may happen while a graph is recorded."""
    import subprocess
    import sys
    code = """
import torch
from paper_2411_10803_b200 import binding as md
cache = md.PagedCache(n_seq=2, n_heads=2, n_pages=8, max_pages=4, q_heads=2)
one = torch.ones(2, dtype=torch.int32, device="cuda")
slots = torch.empty((2, 1), dtype=torch.int32, device="cuda")
k = torch.randn((2, 2, 1, 128), device="cuda").bfloat16()
q, out, back = torch.randn((2, 1, 2, 128), device="cuda").bfloat16(), torch.zeros((2, 1, 2, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros_like(k)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    cache.extend(one, 1, slots)
    cache.store(slots, k, k)
    cache.load(slots, back, None)
    cache.attend(q, out=out)
assert cache.len.tolist() == [0, 0]
g.replay()
torch.cuda.synchronize()
assert cache.len.tolist() == [1, 1] and cache.device_status() == (0, 0)
assert torch.equal(out.transpose(1, 2), back) and back.any()
print("fine")
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]


def test_two_graphs_with_workspaces_of_their_own_replay_side_by_side():
    rng = np.random.default_rng(41)
    caches, graphs, outs, streams = [], [], [], [torch.cuda.Stream() for _ in range(2)]
    lens = [rng.integers(1, 400, 20) for _ in range(2)]
    for i in range(2):
        cache = md.PagedCache(n_seq=20, n_heads=4, n_pages=600, max_pages=26, q_heads=4)
        rows = int(lens[i].max())
        k, v = queries(rng, 20, 4, rows, 128), queries(rng, 20, 4, rows, 128)
        cache.store(cache.extend(i32(lens[i]), rows), k, v)
        caches.append(cache)
    qs = [queries(rng, 20, 1, 4, 128) for _ in range(2)]
    want = [c.attend(q) for c, q in zip(caches, qs)]
    torch.cuda.synchronize()
    for i in range(2):
        g, out = torch.cuda.CUDAGraph(), torch.zeros_like(qs[i])
        with torch.cuda.graph(g):
            for _ in range(5):
                caches[i].attend(qs[i], out=out)
        graphs.append(g)
        outs.append(out)
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], want[i]) and caches[i].device_status() == (0, 0)
