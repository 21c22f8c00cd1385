"""The paged 4-bit cache without a GPU: the plain statement against hand-made values and against itself, and every refusal
that the host makes."""
import numpy as np
import pytest

from oracle import pages
from paper_2411_10803_b200 import binding as md
from paper_2411_10803_b200 import build as md_build

A = 256     # an address that is aligned and never read: refused calls launch nothing


@pytest.fixture(scope="module", autouse=True)
def _built():
    md_build.build()


def test_a_group_by_hand():
    # -7.5 .. 7.5 in steps of one: scale (7.5 / 2 + 7.5 / 2) / 7.5 = 1, centre -7.5 + 8 = 0.5, codes 0 .. 15 twice
    x = np.concatenate([np.arange(16) - 7.5, np.arange(16) - 7.5])[None]
    c, s, z = pages.quantise(x)
    assert s.tolist() == [[1.0]] and z.tolist() == [[0.5]]
    assert c.tolist() == [list(range(16)) * 2]
    assert np.array_equal(pages.values(c, s, z), x)
    # one value throughout: no scale, the value itself is the centre
    c, s, z = pages.quantise(np.full((1, 32), -3.25))
    assert s.tolist() == [[0.0]] and z.tolist() == [[-3.25]] and set(c.reshape(-1).tolist()) == {8}
    # the largest numbers bf16 has: nothing overflows
    big = float(np.float32(3.3895314e38))
    c, s, z = pages.quantise(np.array([[-big] + [big] * 31]))
    assert np.isfinite(pages.values(c, s, z)).all() and np.isfinite(s).all()
    # an infinity or a NaN takes its group with it, and no other
    x = np.ones((1, 64))
    x[0, 40] = np.inf
    v = pages.values(*pages.quantise(x))
    assert np.array_equal(v[0, :32], x[0, :32]) and np.isnan(v[0, 32:]).all()


@pytest.mark.parametrize("spread,centre", [(1.0, 0.0), (1e-3, 0.0), (1e4, 0.0), (1.0, 5.0)])
def test_a_value_is_off_by_half_a_step_and_the_rounding_of_scale_and_centre(spread, centre):
    x = pages.to_bf16(centre + spread * np.random.default_rng(1).standard_normal((400, 128)))
    c, s, z = pages.quantise(x)
    off = np.abs(pages.values(c, s, z) - x).reshape(400, 4, 32)
    # half a step; at the ends of the range 8 steps' rounding of the scale and the centre's rounding (each half a bf16
    # ulp, 2^-9 relative at most times a factor of two inside a binade), which the clamped codes cannot make up for
    bound = s / 2 + 8 * s * 2.0 ** -8 + np.abs(z) * 2.0 ** -8
    assert (off <= bound[..., None] * (1 + 1e-9)).all()


def test_every_byte_of_a_chunk_has_one_owner():
    for d in (64, 128):
        k, v, meta = pages._places(d)
        owned = [tuple(x) for x in k.reshape(-1, 2)] + [tuple(x) for x in v.reshape(-1, 2)]
        owned += [(b + i, h) for b in meta.reshape(-1) for i in (0, 1) for h in (0, 1)]
        assert len(owned) == len(set(owned)) == 2 * 20 * d


@pytest.mark.parametrize("d", [64, 128])
def test_stored_tokens_read_back(d):
    rng = np.random.default_rng(d)
    k, v = (pages.to_bf16(rng.standard_normal((2, 3, 21, d))) for _ in range(2))
    pool = rng.integers(0, 256, (6, 3, 2, 20 * d)).astype(np.uint8)
    slots = rng.permutation(6 * 32)[:42].reshape(2, 21)
    slots[0, 4] = -1
    pages.store(pool, slots, k, v)
    got = [np.full(k.shape, 9.0) for _ in range(2)]
    pages.load(pool, slots, *got)
    for x, y in zip((k, v), got):
        want = pages.values(*pages.quantise(x))
        want[0, :, 4] = 9.0
        assert np.array_equal(y, want)


def test_tables_keep_every_page_exactly_once():
    rng = np.random.default_rng(5)
    n, page, wide, n_pages = 9, 16, 12, 30
    ring, table = rng.permutation(n_pages).astype(np.int32), np.full((n, wide), -1, np.int32)
    lens, state = np.zeros(n, np.int32), np.array([13, n_pages], np.int32)
    refused = 0
    for step in range(60):
        add = rng.integers(-60, 60, n).astype(np.int32)
        lens, state, ring, table, slots, bad, short = pages.tables(add, lens, state, ring, table, page, 60)
        refused += len(short)
        held = [int(p) for s in range(n) for p in table[s, :-(-lens[s] // page)]]
        free = [int(ring[(state[0] + i) % n_pages]) for i in range(state[1])]
        assert sorted(held + free) == list(range(n_pages))
        used = slots[slots >= 0]
        assert len(used) == len(set(used.tolist()))
    assert refused > 0


GOOD = dict(n_seq=3, n_heads=2, head_dim=128, page=16, n_pages=40, max_pages=10, rows=8, q_heads=4, n_q=2)


def _call(name, cfg, **swap):
    args = {"tables": ["add", "len", "ring_state", "len_out", "ring_state_out", "ring", "page_table", "slots", "workspace"],
            "store": ["slots", "k", "v", "pool", "workspace"], "load": ["slots", "pool", "k_out", "v_out", "workspace"],
            "attend": ["q", "pool", "page_table", "len", "out", "workspace"]}[name]
    return getattr(md, "mustdrop_page_" + name)(cfg, *[swap.get(a, A) for a in args], stream=0)


@pytest.mark.parametrize("bad,code", [
    (dict(n_seq=0), md.MUSTDROP_ERR_INVALID_ARG), (dict(n_pages=0), md.MUSTDROP_ERR_INVALID_ARG),
    (dict(flags=1), md.MUSTDROP_ERR_INVALID_ARG), (dict(page=24), md.MUSTDROP_ERR_UNSUPPORTED),
    (dict(page=256), md.MUSTDROP_ERR_UNSUPPORTED), (dict(n_seq=65536), md.MUSTDROP_ERR_UNSUPPORTED),
    (dict(n_pages=1 << 27), md.MUSTDROP_ERR_UNSUPPORTED),
])
def test_sizes_every_call_refuses(bad, code):
    cfg = md.PageConfig(**{**GOOD, **bad})
    for name in ("tables", "store", "load", "attend"):
        assert _call(name, cfg) == code, name
    assert md.mustdrop_page_pool_bytes(cfg) == 0 and md.mustdrop_page_workspace_bytes(cfg) == 0


@pytest.mark.parametrize("name,bad,code", [
    ("tables", dict(rows=0), md.MUSTDROP_ERR_INVALID_ARG), ("tables", dict(max_pages=0), md.MUSTDROP_ERR_INVALID_ARG),
    ("tables", dict(max_pages=1 << 27), md.MUSTDROP_ERR_UNSUPPORTED),
    ("store", dict(rows=0), md.MUSTDROP_ERR_INVALID_ARG), ("store", dict(n_heads=0), md.MUSTDROP_ERR_INVALID_ARG),
    ("store", dict(head_dim=96), md.MUSTDROP_ERR_UNSUPPORTED), ("store", dict(k_stride_h=12), md.MUSTDROP_ERR_UNSUPPORTED),
    ("store", dict(v_stride_r=130), md.MUSTDROP_ERR_UNSUPPORTED),
    ("load", dict(rows=-1), md.MUSTDROP_ERR_INVALID_ARG), ("load", dict(head_dim=32), md.MUSTDROP_ERR_UNSUPPORTED),
    ("attend", dict(q_heads=3), md.MUSTDROP_ERR_INVALID_ARG), ("attend", dict(q_heads=0), md.MUSTDROP_ERR_INVALID_ARG),
    ("attend", dict(n_q=0), md.MUSTDROP_ERR_INVALID_ARG), ("attend", dict(n_q=129), md.MUSTDROP_ERR_UNSUPPORTED),
    ("attend", dict(causal=2), md.MUSTDROP_ERR_INVALID_ARG), ("attend", dict(scale=-1.0), md.MUSTDROP_ERR_INVALID_ARG),
    ("attend", dict(scale=float("nan")), md.MUSTDROP_ERR_INVALID_ARG), ("attend", dict(n_seq=4097), md.MUSTDROP_ERR_UNSUPPORTED),
    ("attend", dict(scale=float("inf")), md.MUSTDROP_ERR_INVALID_ARG),
    ("attend", dict(q_stride_t=4), md.MUSTDROP_ERR_UNSUPPORTED), ("attend", dict(max_pages=0), md.MUSTDROP_ERR_INVALID_ARG),
    ("attend", dict(n_seq=4096, max_pages=1 << 20), md.MUSTDROP_ERR_UNSUPPORTED),
    ("attend", dict(max_pages=(1 << 26) + 1), md.MUSTDROP_ERR_UNSUPPORTED), ("tables", dict(n_seq=65535, max_pages=1 << 16), md.MUSTDROP_ERR_UNSUPPORTED),
    ("attend", dict(scale=1e38), md.MUSTDROP_ERR_INVALID_ARG),
])
def test_sizes_one_call_refuses(name, bad, code):
    assert _call(name, md.PageConfig(**{**GOOD, **bad})) == code


@pytest.mark.parametrize("name,swap,code", [
    ("tables", dict(add=None), 1), ("tables", dict(ring=None), 1), ("tables", dict(slots=A + 2), 1), ("tables", dict(workspace=None), 4),
    ("tables", dict(workspace=A + 4), 1),
    ("store", dict(k=None), 1), ("store", dict(v=A + 8), 1), ("store", dict(pool=None), 1), ("store", dict(slots=A + 1), 1),
    ("load", dict(pool=A + 8), 1), ("load", dict(k_out=A + 2), 1), ("load", dict(slots=None), 1),
    ("attend", dict(q=None), 1), ("attend", dict(out=A + 4), 1), ("attend", dict(page_table=None), 1), ("attend", dict(len=A + 1), 1),
    ("attend", dict(workspace=None), 4),
])
def test_pointers_that_are_refused(name, swap, code):
    assert _call(name, md.PageConfig(**GOOD), **swap) == code


def test_load_of_nothing_is_fine_without_a_launch():
    assert _call("load", md.PageConfig(**GOOD), k_out=None, v_out=None) == md.MUSTDROP_OK


def test_sizes_of_pool_and_workspace():
    cfg = md.PageConfig(**GOOD)
    assert md.mustdrop_page_pool_bytes(cfg) == 40 * 2 * 1 * 20 * 128
    assert md.mustdrop_page_workspace_bytes(cfg) % 256 == 0 and md.mustdrop_page_workspace_bytes(cfg) > 256
    assert md.mustdrop_page_workspace_bytes(md.PageConfig(n_seq=1, page=16, n_pages=1, max_pages=1, rows=1)) == 256
    with pytest.raises(TypeError):
        md.PageConfig(pages=3)


@pytest.mark.parametrize("bad", [
    dict(n_q=129), dict(n_q=200), dict(n_q=-1), dict(q_heads=3), dict(q_heads=0), dict(q_heads=-4), dict(n_heads=0), dict(head_dim=96),
    dict(n_heads=1, q_heads=129, n_q=128), dict(n_heads=1, q_heads=65536, n_q=1),
])
def test_no_workspace_for_queries_that_the_attention_refuses(bad):
    cfg = md.PageConfig(**{**GOOD, **bad})
    assert _call("attend", cfg) in (md.MUSTDROP_ERR_INVALID_ARG, md.MUSTDROP_ERR_UNSUPPORTED)
    assert md.mustdrop_page_workspace_bytes(cfg) == 0


def test_a_workspace_serves_every_smaller_number_of_queries():
    for heads, q_heads in ((2, 2), (2, 4), (1, 71), (8, 64)):
        sizes = [md.mustdrop_page_workspace_bytes(md.PageConfig(**{**GOOD, "n_heads": heads, "q_heads": q_heads, "n_q": n_q})) for n_q in range(1, 129)]
        assert sizes[0] > 256 and sizes == sorted(sizes)


@pytest.mark.parametrize("bad", [dict(max_q=129), dict(max_q=-1), dict(q_heads=3), dict(max_q=128, q_heads=258)])
def test_the_owner_refuses_queries_without_a_workspace(bad):
    with pytest.raises(md.MustDropError):      # (before anything is allocated: there is no device here)
        md.PagedCache(**{**dict(n_seq=2, n_heads=2, n_pages=8, max_pages=4, device="cuda:0"), **bad})


def test_the_owner_keeps_a_bounded_number_of_descriptors():
    cache = object.__new__(md.PagedCache)
    cache._configs = {}
    for rows in list(range(1, 2000)) * 2:
        c = cache._config(("extend", rows), n_seq=3, rows=rows, n_pages=4)
        assert c.c.rows == rows and c is cache._config(("extend", rows), n_seq=3, rows=rows, n_pages=4)
    assert len(cache._configs) <= 256
