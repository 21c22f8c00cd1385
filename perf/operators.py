"""Operators of the decoding-stage cache held in pages of 4-bit values, as cases that can be timed and compared.

  tables   pages and slots for the tokens that sequences gain or give back, from lengths on the GPU
  store    rows of keys and values quantised into the pages (and read back: what the pages now stand for)
  load     the values of stored tokens as bf16 rows
  attend   attention of one or a few query tokens per sequence over its pages

A sequence is one request's cache at one layer.  Sizes are those of the library's own workloads (576 vision tokens pruned to
192 / 128 / 64, 64 text tokens, 32 or 40 heads of 128, 30 later layers) and generic ones that no tile divides.

One page of one head holds page / 16 chunks of 16 tokens.  With D = head_dim and G = D / 32 groups of 32 channels, a chunk is
20 D bytes; token k of it has the row r(k) = k / 2 + 8 (k mod 2), and, bytes in this order,
  [16 r][4 t][G g][4 b]                        K codes: channel 32 g + 8 t + 2 b in the low half of the byte, the next one in the high half
  [D/64 a][8 i][4 t][4 = (2 h, 2 e)][4 b]      V codes of token 4 t + b: channel 32 (2 a + h) + 4 i + 2 e low, the next one high
  [16 r][G scale, G centre] bf16               K: value = centre + scale (code - 8)
  [16 r][G] bf16                               V scales
  [G][16 r] bf16                               V centres
"""
import math

import numpy as np
import torch

own = False

GROUP = 32
MOST_BYTES = 330e6      # what a drawn case may move


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # one decoded token of 8 requests in the 30 layers that keep only the last set: the smallest call, all latency
        {"name": "tables_one_token", "op": "tables", "n_seq": 240, "page": 16, "len_lo": 100, "len_hi": 400, "add_lo": 1,
         "add_hi": 1, "rows": 1, "release": 0.0, "short": False},
        # 64 requests after the last pruning layer, all 32 layers at once: 64 + 64 to 192 + 64 rows each
        {"name": "tables_after_prune", "op": "tables", "n_seq": 2048, "page": 32, "len_lo": 0, "len_hi": 0, "add_lo": 128,
         "add_hi": 256, "rows": 256, "release": 0.0, "short": False},
        # a server's churn: some requests end, some are admitted, the pool runs out for the last ones
        {"name": "tables_churn", "op": "tables", "n_seq": 1531, "page": 64, "len_lo": 1, "len_hi": 2500, "add_lo": 0,
         "add_hi": 700, "rows": 700, "release": 0.3, "short": True},
        # the decoded token of the same 240 sequences
        {"name": "store_one_token", "op": "store", "n_seq": 240, "n_heads": 32, "head_dim": 128, "page": 16, "rows": 1,
         "cnt_lo": 1, "at_hi": 400, "token_major": True},
        # the pruned prompts of 32 requests at one layer: 192 vision rows and 64 text rows at most
        {"name": "store_pruned_prompt", "op": "store", "n_seq": 32, "n_heads": 32, "head_dim": 128, "page": 16, "rows": 256,
         "cnt_lo": 128, "at_hi": 0, "token_major": False},
        # odd counts behind a prefix that ends inside a chunk
        {"name": "store_odd", "op": "store", "n_seq": 13, "n_heads": 5, "head_dim": 64, "page": 32, "rows": 777,
         "cnt_lo": 0, "at_hi": 90, "token_major": True},
        # an earlier turn's cache read back for another pruning layer
        {"name": "load_prompt", "op": "load", "n_seq": 32, "n_heads": 32, "head_dim": 128, "page": 64, "rows": 640,
         "cnt_lo": 576, "at_hi": 0, "token_major": False},
        {"name": "load_odd", "op": "load", "n_seq": 21, "n_heads": 3, "head_dim": 64, "page": 16, "rows": 351, "cnt_lo": 0,
         "at_hi": 77, "token_major": False},
        # one request, one token, an image's tokens unpruned in the first layers: latency
        {"name": "attend_one_request", "op": "attend", "n_seq": 1, "n_heads": 32, "group": 1, "head_dim": 128, "page": 16,
         "len_lo": 640, "len_hi": 640, "n_q": 1, "causal": True},
        # a full batch after many decoded tokens, ragged: the throughput point
        {"name": "attend_batch64", "op": "attend", "n_seq": 64, "n_heads": 32, "group": 1, "head_dim": 128, "page": 32,
         "len_lo": 200, "len_hi": 1800, "n_q": 1, "causal": True},
        # hours of video in two requests, four query heads to a K / V head
        {"name": "attend_long", "op": "attend", "n_seq": 2, "n_heads": 8, "group": 4, "head_dim": 128, "page": 64,
         "len_lo": 90001, "len_hi": 131071, "n_q": 1, "causal": True},
        # five drafted tokens at once, small heads, some sequences shorter than the drafts or empty
        {"name": "attend_draft_odd", "op": "attend", "n_seq": 37, "n_heads": 4, "group": 3, "head_dim": 64, "page": 16,
         "len_lo": 0, "len_hi": 1451, "n_q": 5, "causal": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(["tables", "store", "load", "attend"], [20, 20, 15, 45])[0]
    page = rng.choice([16, 32, 64, 128])
    if op == "tables":
        rows = _log(rng, 1, 900)
        return {"op": op, "n_seq": _log(rng, 1, 2500), "page": page, "len_lo": 0, "len_hi": _log(rng, 1, 3000),
                "add_lo": rng.randint(0, rows), "add_hi": rows, "rows": rows, "release": rng.choice([0.0, 0.0, 0.2, 0.5]),
                "short": rng.random() < 0.25}
    case = {"op": op, "n_seq": _log(rng, 1, 64), "n_heads": rng.choice([1, 2, 3, 5, 8, 16, 32, 40]),
            "head_dim": rng.choice([64, 128, 128]), "page": page}
    if op == "attend":
        group = rng.choice([1, 1, 1, 2, 3, 4, 8])
        hi = _log(rng, 1, 130000)
        n_q = rng.choice([1, 1, 1, 2, 5, 8, rng.randint(1, 40)])
        case.update(group=group, len_lo=rng.choice([0, hi // 8, hi // 2, hi]), len_hi=hi, n_q=n_q, causal=rng.random() < 0.9)
        while case["n_seq"] * case["n_heads"] * hi * case["head_dim"] * 1.25 * max(1, n_q * group / 8) > MOST_BYTES:
            if case["n_seq"] > 1:
                case["n_seq"] //= 2
            elif case["n_heads"] > 1:
                case["n_heads"] //= 2
            else:
                hi //= 2
                case.update(len_lo=min(case["len_lo"], hi), len_hi=hi)
    else:
        rows = _log(rng, 1, 1500)
        case.update(rows=rows, cnt_lo=rng.choice([0, rows // 2, rows]), at_hi=rng.choice([0, 0, rng.randint(1, 500)]),
                    token_major=rng.random() < 0.5)
        while case["n_seq"] * case["n_heads"] * rows * case["head_dim"] * 5.25 > MOST_BYTES:
            if case["n_seq"] > 1:
                case["n_seq"] //= 2
            else:
                rows //= 2
                case.update(rows=rows, cnt_lo=min(case["cnt_lo"], rows))
    return case


# ------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _layout(case, lens, rng):
    """Page table of the given lengths over a pool whose pages lie in no order: (table with -1 behind, pages of the pool)."""
    page = case["page"]
    used = -(-lens // page)
    wide = max(1, int(used.max()))
    total = max(1, int(used.sum()))
    pages = total + 3 + total // 8
    ids = rng.permutation(pages)[:int(used.sum())]
    table = np.full((len(lens), wide), -1, dtype=np.int32)
    table[np.arange(wide)[None, :] < used[:, None]] = ids
    return table, pages


def _rows(gen, case, rows):
    """Keys with a few strong channels, values without: bf16 [n_seq, n_heads, rows, head_dim] (strides as the case says)."""
    shape = (case["n_seq"], rows, case["n_heads"], case["head_dim"]) if case.get("token_major") else \
        (case["n_seq"], case["n_heads"], rows, case["head_dim"])
    k, v = (torch.randn(shape, device="cuda", generator=gen) for _ in range(2))
    k[..., ::29] *= 5
    k, v = k.bfloat16(), v.bfloat16()
    return (k.transpose(1, 2), v.transpose(1, 2)) if case.get("token_major") else (k, v)


def _slots(case, rng, gen):
    """Slots of `rows` new tokens per sequence (-1 behind its count) that begin at an earlier length: (slots, pages)."""
    n, rows, page = case["n_seq"], case["rows"], case["page"]
    at = rng.randint(0, case["at_hi"] + 1, n)
    cnt = rng.randint(case["cnt_lo"], rows + 1, n)
    table, pages = _layout(case, at + cnt, rng)
    pos = at[:, None] + np.arange(rows)[None, :]
    entry = np.take_along_axis(table, np.minimum(pos // page, table.shape[1] - 1), 1)
    slots = np.where(np.arange(rows)[None, :] < cnt[:, None], entry.astype(np.int64) * page + pos % page, -1)
    return torch.from_numpy(slots.astype(np.int32)).cuda(), pages


def _new_pool(case, pages):
    """A pool (and one page more, which nothing of the library is told of) with bits nobody has written yet."""
    return torch.full((pages + 1, case["n_heads"], case["page"] // 16, 20 * case["head_dim"]), 255, dtype=torch.uint8, device="cuda")


def _prepare_tables(case, rng):
    n, page, rows = case["n_seq"], case["page"], case["rows"]
    lens = rng.randint(case["len_lo"], case["len_hi"] + 1, n)
    add = rng.randint(case["add_lo"], case["add_hi"] + 1, n)
    ends = rng.random_sample(n) < case["release"]
    add = np.where(ends, -lens, add)
    used = -(-lens // page)
    need = np.maximum(-(-(lens + add) // page) - used, 0)
    wide = -(-(case["len_hi"] + rows) // page)
    free = int(need.sum()) * (3 if case["short"] else 5) // 4 + 2
    pages = n * wide + 2            # other sequences hold the rest
    free = min(free, pages - int(used.sum()))
    ids = rng.permutation(pages)
    table = np.full((n, wide), -1, dtype=np.int32)
    table[np.arange(wide)[None, :] < used[:, None]] = ids[free:free + int(used.sum())]
    ring = np.full(pages, -1, dtype=np.int32)
    head = rng.randint(0, pages)
    ring[(head + np.arange(free)) % pages] = ids[:free]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    state = {"add": dev(add), "len": dev(lens), "ring_state": dev([head, free]), "table": dev(table), "ring": dev(ring), "pages": pages}
    state["len_out"], state["ring_state_out"] = torch.empty_like(state["len"]), torch.empty_like(state["ring_state"])
    state["slots"] = torch.empty((n, rows), dtype=torch.int32, device="cuda")
    return state


def prepare(case, seed):
    rng, gen = np.random.RandomState(seed % (1 << 31)), _generator(seed)
    op, page = case["op"], case["page"]
    if op == "tables":
        state = _prepare_tables(case, rng)
        sizes = {"n_seq": case["n_seq"], "page": page, "n_pages": state["pages"], "max_pages": state["table"].shape[1], "rows": case["rows"]}
    elif op in ("store", "load"):
        slots, pages = _slots(case, rng, gen)
        state = {"slots": slots, "pool": _new_pool(case, pages)}
        k, v = _rows(gen, case, case["rows"])
        shape = (case["n_seq"], case["n_heads"], case["rows"], case["head_dim"])
        state["k_out"], state["v_out"] = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        if op == "store":
            state["k"], state["v"] = k, v
        else:
            _put(state["pool"], slots, *_quantise(k), *_quantise(v))
        sizes = {"n_seq": case["n_seq"], "n_heads": case["n_heads"], "head_dim": case["head_dim"], "page": page,
                 "n_pages": pages, "rows": case["rows"]}
        if op == "store":
            sizes.update({"%s_stride_%s" % (x, a): state[x].stride(d) for x in "kv" for d, a in enumerate("shr")})
    else:
        lens = rng.randint(case["len_lo"], case["len_hi"] + 1, case["n_seq"])
        if case["n_seq"] > 2 and case["len_lo"] < 4:
            lens[1:3] = case["len_lo"], min(3, case["len_hi"])
        table, pages = _layout(case, lens, rng)
        rows = max(1, int(lens.max()))
        k, v = _rows(gen, case, rows)
        pos = np.arange(rows)[None, :]
        entry = np.take_along_axis(table, np.minimum(np.broadcast_to(pos // page, (len(lens), rows)), table.shape[1] - 1), 1)
        slots = np.where(pos < lens[:, None], entry.astype(np.int64) * page + pos % page, -1).astype(np.int32)
        state = {"pool": _new_pool(case, pages), "table": torch.from_numpy(table).cuda(), "len": torch.from_numpy(lens.astype(np.int32)).cuda()}
        _put(state["pool"], torch.from_numpy(slots).cuda(), *_quantise(k), *_quantise(v))
        q_heads = case["n_heads"] * case["group"]
        state["q"] = torch.randn((case["n_seq"], case["n_q"], q_heads, case["head_dim"]), device="cuda", generator=gen).bfloat16()
        state["out"] = torch.empty_like(state["q"])
        sizes = {"n_seq": case["n_seq"], "n_heads": case["n_heads"], "q_heads": q_heads, "head_dim": case["head_dim"], "page": page,
                 "n_pages": pages, "max_pages": table.shape[1], "n_q": case["n_q"], "causal": int(case["causal"])}
    state["case"], state["sizes"] = case, sizes
    if own:  # the descriptor and the workspace that a program keeps
        from paper_2411_10803_b200 import binding as md
        state["md"], state["config"] = md, md.PageConfig(**sizes)
        state["workspace"] = torch.zeros(md.mustdrop_page_workspace_bytes(state["config"]), dtype=torch.uint8, device="cuda")
    return state


# ------------------------------------------------------------------ the operators

def run(state):
    op = state["case"]["op"]
    if not own:
        return {"tables": _tables, "store": _store, "load": _load, "attend": _attend}[op](state)
    md, c, ws = state["md"], state["config"], state["workspace"]
    if op == "tables":
        _ok(md, md.mustdrop_page_tables(c, state["add"], state["len"], state["ring_state"], state["len_out"], state["ring_state_out"],
                                        state["ring"], state["table"], state["slots"], ws))
        return {x: state[x] for x in ("len_out", "ring_state_out", "ring", "table", "slots")}
    if op == "attend":
        _ok(md, md.mustdrop_page_attend(c, state["q"], state["pool"], state["table"], state["len"], state["out"], ws))
        return state["out"]
    if op == "store":
        _ok(md, md.mustdrop_page_store(c, state["slots"], state["k"], state["v"], state["pool"], ws))
    _ok(md, md.mustdrop_page_load(c, state["slots"], state["pool"], state["k_out"], state["v_out"], ws))
    return state["k_out"], state["v_out"]


def _ok(md, status):
    if status != md.MUSTDROP_OK:
        raise md.MustDropError(status, "page operator")


def _tables(state):
    page, rows, pages = state["case"]["page"], state["case"]["rows"], state["pages"]
    add, lens, table, ring = state["add"].long(), state["len"].long(), state["table"].clone(), state["ring"].clone()
    n, wide = table.shape
    head, count = state["ring_state"].long().unbind()
    new = (lens + add).clamp(min=0)
    had, want = -(-lens // page), -(-new // page)
    need, back = (want - had).clamp(min=0), (had - want).clamp(min=0)
    before = need.cumsum(0) - need
    granted = (need == 0) | (before + need <= count)
    taken = torch.where(granted, need, 0).sum()
    entry = torch.arange(wide, device="cuda")[None, :]
    # pages given back go to the end of the ring, in order
    gone = (entry >= want[:, None]) & (entry < had[:, None])
    to = (head + count + (back.cumsum(0) - back)[:, None] + entry - want[:, None]) % pages
    ring = torch.cat([ring, ring[:1]]).scatter_(0, torch.where(gone, to, pages).reshape(-1), table.reshape(-1))[:pages]
    # pages taken come from its head, in order
    fresh = (entry >= had[:, None]) & (entry < want[:, None]) & granted[:, None]
    at = (head + before[:, None] + entry - had[:, None]) % pages
    table = torch.where(fresh, state["ring"][torch.where(fresh, at, 0)], table)
    len_out = torch.where(granted, new, lens)
    t = torch.arange(rows, device="cuda")[None, :]
    pos = lens[:, None] + t
    there = granted[:, None] & (t < add[:, None])
    slots = table.long().gather(1, (pos // page).clamp(max=wide - 1)) * page + pos % page
    slots = torch.where(there, slots, -1).int()
    state_out = torch.stack([(head + taken) % pages, count - taken + back.sum()]).int()
    return {"len_out": len_out.int(), "ring_state_out": state_out, "ring": ring, "table": table, "slots": slots}


def _quantise(x):
    """Codes, scales and centres of bf16 rows [..., D]."""
    x = x.float().unflatten(-1, (-1, GROUP))
    low, high = x.amin(-1), x.amax(-1)
    scale = ((high * 0.5 - low * 0.5) / 7.5).bfloat16()
    centre = (low + 8 * scale.float()).bfloat16()
    s = scale.float()[..., None]
    code = torch.where(s > 0, torch.round((x - centre.float()[..., None]) / torch.where(s > 0, s, 1)) + 8, 8).clamp(0, 15)
    return code.to(torch.uint8).flatten(-2), scale, centre


def _parts(pool):
    """Views of a pool [pages, heads, chunks, 20 D]: K codes, V codes, K scales and centres, V scales, V centres."""
    d = pool.shape[-1] // 20
    g = d // GROUP
    half = pool.view(torch.bfloat16)
    return (pool[..., :8 * d].unflatten(-1, (16, 4, g, 4)), pool[..., 8 * d:16 * d].unflatten(-1, (d // 64, 8, 4, 4, 4)),
            half[..., 8 * d:9 * d].unflatten(-1, (16, 2, g)), half[..., 9 * d:9 * d + d // 2].unflatten(-1, (16, g)),
            half[..., 9 * d + d // 2:].unflatten(-1, (g, 16)))


def _put(pool, slots, kc, ks, kz, vc, vs, vz):
    """Writes rows [n_seq, heads, rows, ...] to their slots; those without one go to the pool's spare last page."""
    page, d = 16 * pool.shape[2], pool.shape[-1] // 20
    slots = slots.long().reshape(-1)
    at = torch.where(slots >= 0, slots // page, pool.shape[0] - 1)
    off = torch.where(slots >= 0, slots % page, 0)
    ch, key = off // 16, off % 16
    r = key // 2 + 8 * (key % 2)
    rows = lambda a: a.transpose(1, 2).flatten(0, 1)  # noqa: E731
    kc, vc = rows(kc), rows(vc)
    kc = kc[..., 0::2] | (kc[..., 1::2] << 4)                                 # [n, heads, D / 2], bytes in channel order
    vc = vc[..., 0::2] | (vc[..., 1::2] << 4)
    kp, vp, ksz, vsp, vzp = _parts(pool)
    kp[at, :, ch, r] = kc.unflatten(-1, (-1, 4, 4)).transpose(-3, -2)         # [g, t, b] -> [t, g, b]
    # bytes of V by channel pair (a, h, i, e) -> [a, i, (h, e)]
    vp[at, :, ch, :, :, key // 4, :, key % 4] = vc.unflatten(-1, (d // 64, 2, 8, 2)).transpose(-3, -2).flatten(-2)
    ksz[at, :, ch, r, 0], ksz[at, :, ch, r, 1] = rows(ks), rows(kz)
    vsp[at, :, ch, r] = rows(vs)
    vzp[at, :, ch, :, r] = rows(vz)


def _bits(x, dim):
    """The two codes of every byte, along a new axis."""
    return torch.stack([x & 15, x >> 4], dim)


def _values(chunks):
    """fp32 K and V [..., 16, D] of chunks [..., 20 D]."""
    d = chunks.shape[-1] // 20
    kc, vc, ksz, vs, vz = _parts(chunks)
    key = torch.arange(16, device="cuda")
    r = key // 2 + 8 * (key % 2)
    k = _bits(kc.transpose(-3, -2), -1).flatten(-3).float() - 8               # [r, g, 32]
    k = ksz[..., 1, :, None].float() + ksz[..., 0, :, None].float() * k
    v = _bits(vc, -1).unflatten(-3, (2, 2))                                   # [a, i, t, h, e, b, n]
    lead = list(range(v.dim() - 7))
    n = len(lead)
    v = v.permute(lead + [n + 2, n + 5, n + 0, n + 3, n + 1, n + 4, n + 6]).reshape(*v.shape[:n], 16, d // GROUP, GROUP).float() - 8
    v = vz.transpose(-2, -1)[..., r, :, None].float() + vs[..., r, :, None].float() * v
    return k.flatten(-2)[..., r, :], v.flatten(-2)


def _store(state):
    pool = state["pool"]
    _put(pool, state["slots"], *_quantise(state["k"]), *_quantise(state["v"]))
    return _load(state)


def _load(state):
    pool, slots = state["pool"], state["slots"].long()
    page = 16 * pool.shape[2]
    safe = slots.clamp(min=0)
    at, ch, key = safe // page, safe % page // 16, safe % 16
    r = key // 2 + 8 * (key % 2)
    kc, vc, ksz, vs, vz = _parts(pool)
    k = _bits(kc[at, :, ch, r].transpose(-3, -2), -1).flatten(-3).float() - 8
    k = ksz[at, :, ch, r, 1].float()[..., None] + ksz[at, :, ch, r, 0].float()[..., None] * k
    v = _bits(vc[at, :, ch, :, :, key // 4, :, key % 4].unflatten(-1, (2, 2)).transpose(-3, -2), -1)
    v = v.flatten(-5).unflatten(-1, (-1, GROUP)).float() - 8
    v = vz[at, :, ch, :, r].float()[..., None] + vs[at, :, ch, r].float()[..., None] * v
    there = (slots >= 0)[:, None, :, None]
    out = lambda x, old: torch.where(there, x.flatten(-2).transpose(1, 2).bfloat16(), old)  # noqa: E731
    return out(k, state["k_out"]), out(v, state["v_out"])


def _attend(state):
    case, pool, lens, q = state["case"], state["pool"], state["len"].long(), state["q"]
    n, n_q, q_heads, d = q.shape
    heads, group = case["n_heads"], case["group"]
    chunks = pool[state["table"].clamp(min=0).long()].transpose(1, 2).flatten(2, 3)       # [n, heads, chunks, 20 D]
    k, v = (x.flatten(2, 3) for x in _values(chunks))
    pos = torch.arange(k.shape[2], device="cuda")
    here = pos[None, :] < lens[:, None]
    k, v = (torch.where(here[:, None, :, None], x, 0) for x in (k, v))
    x = q.float().unflatten(2, (heads, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)       # [n, heads, n_q * group, D]
    z = (x @ k.transpose(2, 3)) * d ** -0.5
    limit = lens[:, None].expand(n, n_q)
    if case["causal"]:
        limit = limit - n_q + 1 + torch.arange(n_q, device="cuda")[None, :]
    seen = (pos[None, None, :] < limit[:, :, None]).repeat_interleave(group, 1)[:, None]
    z = torch.where(seen, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(z - torch.where(top > -math.inf, top, 0)), 0)
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(total > 0, total, 1)
    return o.unflatten(2, (n_q, group)).permute(0, 2, 1, 3, 4).flatten(2, 3).bfloat16()


# ------------------------------------------------------------------ what cannot be left out

def work(case):
    n, page = case["n_seq"], case["page"]
    if case["op"] == "tables":
        new = 0.5 * (case["add_lo"] + case["add_hi"]) * (1 - case["release"])
        return {"bytes": 4.0 * n * (3 + case["rows"] + 2 * new / page), "flops": 0.0}
    d, h = case["head_dim"], case["n_heads"]
    if case["op"] == "attend":
        mean = 0.5 * (case["len_lo"] + case["len_hi"])
        r = case["n_q"] * case["group"]
        return {"bytes": n * h * (1.25 * d * mean + 4.0 * d * r) + 4.0 * n * mean / page, "flops": 4.0 * n * h * r * d * mean}
    tokens = n * 0.5 * (case["cnt_lo"] + case["rows"])
    moved = {"store": 4 + 1.25 + 1.25 + 4, "load": 1.25 + 4}[case["op"]]
    return {"bytes": tokens * h * d * moved + 4.0 * n * case["rows"] * (2 if case["op"] == "store" else 1),
            "flops": tokens * h * d * 4.0}


# ------------------------------------------------------------------ the same from the definition, in 64 bits

def _byte_of(d):
    """Where a chunk keeps its values: K and V byte offsets [16, D] and half (0 low, 1 high), scale and centre offsets in
    16-bit units [16, D]."""
    key, ch = np.arange(16)[:, None], np.arange(d)[None, :]
    r, g, w = key // 2 + 8 * (key % 2), ch // 32, ch % 32
    groups = d // 32
    k = r * (d // 2) + (w // 8) * 4 * groups + 4 * g + w % 8 // 2
    v = 8 * d + (g // 2) * 512 + (w // 4) * 64 + (key // 4) * 16 + 8 * (g % 2) + 4 * (w % 4 // 2) + key % 4
    ks = 8 * d + r * 2 * groups + g
    vs = 9 * d + r * groups + g
    vz = 9 * d + d // 2 + g * 16 + r
    both = lambda a: torch.from_numpy(np.array(np.broadcast_to(a, (16, d)))).cuda()  # noqa: E731
    return [both(a) for a in (k, v, ch % 2, ks, ks + groups, vs, vz)]


def _exact_chunks(chunks, d):
    """Float64 K, V [..., 16, D]."""
    k, v, half, ks, kz, vs, vz = _byte_of(d)
    wide = chunks.view(torch.bfloat16)
    code = lambda at: ((chunks[..., at] >> (4 * half).to(torch.uint8)) & 15).double() - 8  # noqa: E731
    return wide[..., kz].double() + wide[..., ks].double() * code(k), wide[..., vz].double() + wide[..., vs].double() * code(v)


def _exact_rows(x):
    """Float64 values that stored rows [..., D] stand for."""
    x = x.double().reshape(*x.shape[:-1], -1, 32)
    low, high = x.min(-1).values, x.max(-1).values
    s = ((high - low) / 15).to(torch.bfloat16).double()
    z = (low + 8 * s).to(torch.bfloat16).double()[..., None]
    s = s[..., None]
    c = torch.clamp(torch.round((x - z) / torch.where(s == 0, 1.0, s)), -8, 7)
    return (z + torch.where(s == 0, 0.0, s * c)).reshape(*x.shape[:-2], -1)


def exact(case, seed):
    if case["op"] == "tables":
        return None
    state = prepare(case, seed)
    if case["op"] == "store":
        there = (state["slots"] >= 0)[:, None, :, None]
        return tuple(torch.where(there, _exact_rows(state[x]), 0.0) for x in "kv")
    pool, d, page = state["pool"], case["head_dim"], case["page"]
    if case["op"] == "load":
        slots = state["slots"].long()
        k, v = torch.zeros(state["k_out"].shape, dtype=torch.float64, device="cuda"), torch.zeros(state["k_out"].shape, dtype=torch.float64, device="cuda")
        for b in range(case["n_seq"]):
            at = torch.nonzero(slots[b] >= 0)[:, 0]
            s = slots[b, at]
            for h in range(case["n_heads"]):
                ek, ev = _exact_chunks(pool[s // page, h, s % page // 16], d)
                pick = (s % 16)[:, None, None].expand(-1, 1, d)
                k[b, h, at], v[b, h, at] = ek.gather(1, pick)[:, 0], ev.gather(1, pick)[:, 0]
        return k, v
    lens = state["len"].tolist()
    n_q, group = case["n_q"], case["group"]
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda")
    for b, length in enumerate(lens):
        pages = state["table"][b, :-(-length // page)].long()
        for h in range(case["n_heads"] if length else 0):
            k, v = (x.reshape(-1, d)[:length] for x in _exact_chunks(pool[pages, h].reshape(-1, 20 * d), d))
            q = state["q"][b, :, h * group:(h + 1) * group].double()                       # [n_q, group, D]
            z = torch.einsum("tgd,jd->tgj", q, k) / math.sqrt(d)
            if case["causal"]:
                limit = length - n_q + 1 + torch.arange(n_q, device="cuda")
                z = z.masked_fill(torch.arange(length, device="cuda") >= limit[:, None, None], -math.inf)
            p = torch.softmax(z, -1).nan_to_num(0.0)
            out[b, :, h * group:(h + 1) * group] = torch.einsum("tgj,jd->tgd", p, v)
    return out
