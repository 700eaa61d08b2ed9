"""The paged key/value cache operators: measured cases, plain forms and definitions.

Four operators let a request's sequences grow over a cache of fixed-size pages instead of being recomputed:

* append   pages for every sequence's new tokens: block tables, row offsets, positions and the slot of every new row
           (``prism_op_page_append``);
* release  the pages of the candidates that left go back to the pool, the survivors' tables move together
           (``prism_op_page_release``);
* rope     per-head RMSNorm of queries and keys, rotary position, and the rows' keys and values into their cache slots,
           in one pass (``prism_op_qknorm_rope_paged``);
* attn     attention of every sequence's new tokens over its cached and new keys, through the block table
           (``prism_op_attention_paged``).

A case is a dict of plain values; the lengths inside a case follow from its own ``mix`` number, the data from the seed.
``run`` takes the plain forms below (elementary torch operations, fp32, rounded once) while ``own`` is false, and the
library's entry points when it is true.  ``exact`` is each operator's definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # twenty candidates of about 500 tokens enter behind a cached query of 32 tokens
        {"name": "append_20_docs", "op": "append", "n": 20, "new_min": 440, "new_max": 480, "cached_min": 32,
         "cached_max": 32, "page": 16, "mix": 1},
        # a large request: a thousand candidates of ragged length behind a cached prompt of 256
        {"name": "append_1000_docs", "op": "append", "n": 1000, "new_min": 32, "new_max": 1024, "cached_min": 256,
         "cached_max": 256, "page": 16, "mix": 2},
        # a probe on a hundred candidates keeps forty; the query's two pages are shared and stay
        {"name": "release_100", "op": "release", "n": 100, "keep": 40, "cached_min": 160, "cached_max": 544,
         "page": 16, "shared": 2, "mix": 3},
        # the same on a thousand candidates, 250 of which stay
        {"name": "release_1000", "op": "release", "n": 1000, "keep": 250, "cached_min": 64, "cached_max": 1056,
         "page": 16, "shared": 2, "mix": 4},
        # one new token for each of twenty sequences: latency
        {"name": "rope_20_tokens", "op": "rope", "rows": 20, "hq": 16, "hkv": 8, "dh": 128, "dtype": "bf16",
         "norm": True, "page": 16, "far": 512, "theta": 1e6, "mix": 5},
        # all rows of a hundred candidates
        {"name": "rope_35200_rows", "op": "rope", "rows": 35200, "hq": 16, "hkv": 8, "dh": 128, "dtype": "bf16",
         "norm": True, "page": 16, "far": 1024, "theta": 1e6, "mix": 6},
        # the small fp32 model, without head norms, an odd number of rows
        {"name": "rope_773_rows_fp32", "op": "rope", "rows": 773, "hq": 4, "hkv": 2, "dh": 64, "dtype": "fp32",
         "norm": False, "page": 16, "far": 64, "theta": 1e4, "mix": 7},
        # one new token for each of twenty candidates of about 500 tokens: latency
        {"name": "attn_20_tokens", "op": "attn", "n": 20, "new_min": 1, "new_max": 1, "cached_min": 440,
         "cached_max": 512, "shared": 32, "hq": 16, "hkv": 8, "dh": 128, "dtype": "bf16", "causal": True, "page": 16,
         "mix": 8},
        # one new token for each of a hundred sequences, lengths from hundreds to tens of thousands of tokens
        {"name": "attn_100_tokens_long", "op": "attn", "n": 100, "new_min": 1, "new_max": 1, "cached_min": 500,
         "cached_max": 32768, "shared": 0, "hq": 32, "hkv": 8, "dh": 128, "dtype": "bf16", "causal": True, "page": 16,
         "mix": 9},
        # a hundred candidates of 128 to 512 tokens behind one cached prompt of 512 tokens that all of them read
        {"name": "attn_100_docs", "op": "attn", "n": 100, "new_min": 128, "new_max": 512, "cached_min": 512,
         "cached_max": 512, "shared": 512, "hq": 16, "hkv": 8, "dh": 128, "dtype": "bf16", "causal": True, "page": 16,
         "mix": 10},
        # one chunk of 1024 tokens behind 64 thousand cached ones: few rows, a long axis
        {"name": "attn_chunk_64k", "op": "attn", "n": 1, "new_min": 1024, "new_max": 1024, "cached_min": 65536,
         "cached_max": 65536, "shared": 0, "hq": 32, "hkv": 8, "dh": 128, "dtype": "bf16", "causal": True, "page": 64,
         "mix": 11},
        # the small fp32 model: sixteen documents of 16 to 48 tokens behind a query of 16
        {"name": "attn_16_docs_fp32", "op": "attn", "n": 16, "new_min": 16, "new_max": 48, "cached_min": 16,
         "cached_max": 16, "shared": 16, "hq": 4, "hkv": 2, "dh": 64, "dtype": "fp32", "causal": True, "page": 16,
         "mix": 12},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _draw_once(rng):
    op = rng.choice(["append", "release", "rope", "rope", "attn", "attn", "attn", "attn"])
    mix = rng.randrange(1 << 30)
    page = rng.choice([16, 16, 32, 64, 128])
    if op == "append":
        hi = _log_int(rng, 1, 1024)
        c = _log_int(rng, 1, 4096) - 1
        return {"op": op, "n": _log_int(rng, 1, 2000), "new_min": rng.choice([0, 1, (hi + 1) // 2]) if hi > 1 else hi,
                "new_max": hi, "cached_min": c // 2, "cached_max": c, "page": page, "mix": mix}
    if op == "release":
        n = _log_int(rng, 1, 2000)
        shared = rng.choice([0, 0, 1, 3])
        lo = shared * page
        return {"op": op, "n": n, "keep": rng.randint(0, n), "cached_min": lo, "cached_max": lo + _log_int(rng, 1, 2048),
                "page": page, "shared": shared, "mix": mix}
    heads = rng.choice([(16, 8), (32, 8), (16, 16), (12, 4), (28, 4), (8, 1)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    dh = rng.choice([64, 128, 128])
    if op == "rope":
        return {"op": op, "rows": _log_int(rng, 1, 40000), "hq": heads[0], "hkv": heads[1], "dh": dh, "dtype": dtype,
                "norm": rng.random() < 0.7, "page": page, "far": _log_int(rng, 1, 1 << 20),
                "theta": rng.choice([1e4, 1e6]), "mix": mix}
    kind = rng.choice(["token", "token", "docs", "chunk"])
    shared = 0
    if kind == "token":
        n, new = _log_int(rng, 1, 400), (1, rng.choice([1, 1, 1, 2, 5]))
        far = _log_int(rng, 1, 40000)
        cached = far // rng.choice([1, 2, 30]), far
    elif kind == "docs":
        hi = _log_int(rng, 3, 900)
        n, new = _log_int(rng, 1, 200), (rng.choice([1, hi // 3, hi // 2]), hi)
        shared = page * rng.choice([0, 1, 2, 5])
        cached = shared, shared + rng.choice([0, 0, 77])
    else:
        n, hi = rng.randint(1, 4), _log_int(rng, 20, 2000)
        new, far = (hi, hi), _log_int(rng, 1, 60000)
        cached = far // 2, far
    return {"op": op, "n": n, "new_min": new[0], "new_max": new[1], "cached_min": cached[0], "cached_max": cached[1],
            "shared": shared, "hq": heads[0], "hkv": heads[1], "dh": dh,
            "dtype": dtype, "causal": rng.random() < 0.8, "page": page, "mix": mix}


# Costs of the largest listed cases: a drawn one stays below them (fp32 has a tenth of the matrix rate, so a tenth of
# the operations).
_MAX_BYTES = 3.2e9
_MAX_FLOPS = 1.0e12


def draw(rng):
    while True:
        case = _draw_once(rng)
        w = work(case)
        room = 0.1 if case.get("dtype") == "fp32" else 1.0
        if w["bytes"] <= room * _MAX_BYTES and w["flops"] <= room * _MAX_FLOPS:
            return case


def _between(g, lo, hi, n):
    """n whole numbers in [lo, hi]; over their logarithm where the range spans more than a factor of ten."""
    if lo > 0 and hi > 10 * lo:
        return np.minimum(hi, np.exp(g.uniform(math.log(lo), math.log(hi + 1), size=n)).astype(np.int64))
    return g.integers(lo, hi + 1, size=n)


def _lengths(case):
    g = np.random.default_rng(case["mix"])
    cached = _between(g, case["cached_min"], case["cached_max"], case["n"])
    new = _between(g, case["new_min"], case["new_max"], case["n"]) if "new_max" in case else None
    return cached, new


def _pages(tokens, page):
    return -(-tokens // page)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    """What a pass cannot do without: inputs read once, outputs written once."""
    op = case["op"]
    if op == "append":
        cached, new = _lengths(case)
        need = _pages(cached + new, case["page"]) - _pages(cached, case["page"])
        total = int(new.sum())
        # lengths in and out, offsets, two words a row, a page id read and written for every new page
        return {"bytes": 4 * (4 * case["n"] + 1 + 2 * total + 2 * int(need.sum()) + 2), "flops": 0}
    if op == "release":
        cached, _ = _lengths(case)
        pages = _pages(cached, case["page"])
        # every page id is read once and written once: to the survivor's new row or to the pool
        return {"bytes": 4 * (2 * int(pages.sum()) + 2 * case["n"] + case["keep"] + 2), "flops": 0}
    b = 2 if case["dtype"] == "bf16" else 4
    if op == "rope":
        per_row = (case["hq"] + 2 * case["hkv"]) * case["dh"]
        rows = case["rows"]
        return {"bytes": 2 * rows * per_row * b + 8 * rows, "flops": rows * (case["hq"] + case["hkv"]) * case["dh"] * 7}
    cached, new = _lengths(case)
    kv = cached + new
    keys = int(kv.sum()) - (case["n"] - 1) * case["shared"]  # a shared prefix is read once
    rows = int(new.sum())
    if case["causal"]:
        pairs = int((new * cached + new * (new + 1) // 2).sum())
    else:
        pairs = int((new * kv).sum())
    return {"bytes": b * case["dh"] * (2 * keys * case["hkv"] + 2 * rows * case["hq"]) + 4 * 2 * case["n"],
            "flops": 4 * pairs * case["hq"] * case["dh"]}


# ------------------------------------------------------------------------------------------------ inputs
def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _tables(g, lens, page, max_pages, shared_pages, perm):
    """A block table for sequences of these lengths out of a shuffled pool: rows [n, max_pages] and the pages left over.
    The first shared_pages entries of every row are the same pages; entries behind a row's last page are -1."""
    n = len(lens)
    table = np.full((n, max_pages), -1, np.int64)
    own_pages = np.maximum(_pages(lens, page) - shared_pages, 0)
    ends = np.cumsum(own_pages) + shared_pages
    for s in range(n):
        have = int(_pages(lens[s], page))
        k = min(have, shared_pages)
        table[s, :k] = perm[:k]
        table[s, k:have] = perm[ends[s] - own_pages[s]:ends[s]]
    return table, perm[(ends[-1] if n else shared_pages):]


def prepare(case, seed):
    g = np.random.default_rng([seed, case["mix"]])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(g.integers(1 << 62)))
    st = {"case": case}
    op = case["op"]
    page = case["page"]
    i32 = dict(dtype=torch.int32, device="cuda")
    if op == "append":
        cached, new = _lengths(case)
        tot = _pages(cached + new, page)
        pool = int(tot.sum()) + 16
        max_pages = int(tot.max()) + 3
        table, left = _tables(g, cached, page, max_pages, 0, g.permutation(pool))
        free = np.zeros(pool, np.int64)
        free[:len(left)] = left
        total = int(new.sum())
        st.update(new=_i32(new), kv=_i32(cached), table=_i32(table), free=_i32(free), n_free=_i32([len(left)]),
                  pool=pool, total=total, err=torch.zeros(1, **i32), kv_out=torch.empty(case["n"], **i32),
                  n_free_out=torch.empty(1, **i32), cu=torch.empty(case["n"] + 1, **i32), pos=torch.empty(total, **i32),
                  slot=torch.empty(total, **i32))
        return st
    if op == "release":
        cached, _ = _lengths(case)
        tot = _pages(cached, page)
        pool = int(tot.sum()) + 16
        max_pages = int(tot.max()) + 3
        table, left = _tables(g, cached, page, max_pages, case["shared"], g.permutation(pool))
        free = np.zeros(pool, np.int64)
        free[:len(left)] = left
        keep = np.sort(g.permutation(case["n"])[:case["keep"]])
        st.update(keep=_i32(keep), kv=_i32(cached), table=_i32(table), free=_i32(free), n_free=_i32([len(left)]),
                  pool=pool, err=torch.zeros(1, **i32), kv_out=torch.empty(case["n"], **i32), n_free_out=torch.empty(1, **i32),
                  table_out=torch.empty(case["n"], max_pages, **i32))
        return st
    dt = DTYPES[case["dtype"]]
    hq, hkv, dh = case["hq"], case["hkv"], case["dh"]
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda", dtype=dt)
    if op == "rope":
        rows = case["rows"]
        pool = int(_pages(rows, page)) + 8
        run_pages = g.permutation(pool)[:_pages(rows, page)]
        slot = run_pages[np.arange(rows) // page] * page + np.arange(rows) % page
        st.update(qkv=rand(rows, (hq + 2 * hkv) * dh), pos=_i32(g.integers(0, case["far"], size=rows)), slot=_i32(slot),
                  g_q=1 + 0.1 * rand(dh), g_k=1 + 0.1 * rand(dh), k=rand(pool, hkv, page, dh),
                  v=rand(pool, hkv, page, dh), q=torch.empty(rows, hq * dh, dtype=dt, device="cuda"), err=torch.zeros(1, **i32))
        return st
    cached, new = _lengths(case)
    kv = cached + new
    tot = _pages(kv, page)
    shared_pages = case["shared"] // page
    pool = int(tot.sum()) - (case["n"] - 1) * shared_pages + 8
    max_pages = int(tot.max())
    table, _ = _tables(g, kv, page, max_pages, shared_pages, g.permutation(pool))
    cu = np.concatenate([[0], np.cumsum(new)])
    rows = int(cu[-1])
    st.update(q=rand(rows, hq * dh), k=rand(pool, hkv, page, dh), v=rand(pool, hkv, page, dh), table=_i32(table),
              cu=_i32(cu), kv=_i32(kv), out=torch.empty(rows, hq * dh, dtype=dt, device="cuda"), err=torch.zeros(1, **i32),
              max_q=int(new.max()), host=(cached, new))
    if own:
        # A program lays the attention's work out once a step and uses it in every layer of the model.
        from paper_2510_15620_b200 import ops
        shape = (case["n"], rows, st["max_q"], hq, hkv, dh, 1 if case["dtype"] == "bf16" else 0)
        plan_bytes, ws_bytes = ops.prism_op_attention_paged_bytes(*shape)
        st["plan"] = torch.empty(plan_bytes, dtype=torch.uint8, device="cuda")
        st["ws"] = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
        ops.prism_op_attention_paged_plan(st["cu"], st["kv"], rows, st["max_q"], hq, hkv, dh, shape[-1],
                                          int(case["causal"]), st["plan"], st["err"])
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    from paper_2510_15620_b200 import ops
    case = st["case"]
    op = case["op"]
    if op == "append":
        ops.prism_op_page_append(st["new"], st["kv"], st["kv_out"], case["page"], st["pool"], st["table"], st["free"],
                                 st["n_free"], st["n_free_out"], st["cu"], st["pos"], st["slot"], st["err"])
        return {"kv": st["kv_out"], "table": st["table"], "n_free": st["n_free_out"], "cu": st["cu"], "pos": st["pos"],
                "slot": st["slot"]}
    if op == "release":
        ops.prism_op_page_release(st["keep"], st["kv"], st["kv_out"], case["page"], st["pool"], case["shared"],
                                  st["table"], st["table_out"], st["free"], st["n_free"], st["n_free_out"], st["err"])
        return {"kv": st["kv_out"], "table": st["table_out"], "free": st["free"], "n_free": st["n_free_out"]}
    dtype = 1 if case["dtype"] == "bf16" else 0
    if op == "rope":
        ops.prism_op_qknorm_rope_paged(st["qkv"], dtype, st["pos"], st["slot"], case["hq"], int(case["norm"]),
                                       st["g_q"], st["g_k"], 1e-6, case["theta"], st["q"], st["k"], st["v"], st["err"])
        return {"q": st["q"], "k": st["k"], "v": st["v"]}
    ops.prism_op_attention_paged(st["q"], st["k"], st["v"], st["table"], st["plan"], case["n"], st["max_q"], case["hq"],
                                 dtype, st["out"], st["ws"], st["err"])
    return st["out"]


def _run_plain(st):
    return {"append": _append, "release": _release, "rope": _rope, "attn": _attention}[st["case"]["op"]](st)


def _append(st):
    page, table = st["case"]["page"], st["table"]
    n, width = table.shape
    kv, new = st["kv"].long(), st["new"].long()
    have = (kv + page - 1) // page
    want = (kv + new + page - 1) // page
    need = want - have
    first = need.cumsum(0) - need
    j = torch.arange(width, device="cuda")
    k = first[:, None] + j - have[:, None]
    take = (j >= have[:, None]) & (j < want[:, None])
    n_free = st["n_free"].long()
    ids = st["free"][(n_free - 1 - k).clamp(0, st["free"].numel() - 1)]
    table.copy_(torch.where(take, ids, table))
    ends = new.cumsum(0)
    cu = torch.cat([ends.new_zeros(1), ends])
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), new, output_size=st["total"])
    pos = kv[seq] + torch.arange(st["total"], device="cuda") - cu[seq]
    slot = table[seq, pos // page].long() * page + pos % page
    return {"kv": (kv + new).int(), "table": table, "n_free": (n_free - need.sum()).int(), "cu": cu.int(),
            "pos": pos.int(), "slot": slot.int()}


def _release(st):
    case = st["case"]
    page, table = case["page"], st["table"]
    n, width = table.shape
    kv = st["kv"].long()
    have = (kv + page - 1) // page
    j = torch.arange(width, device="cuda")
    stays = torch.zeros(n, dtype=torch.bool, device="cuda")
    stays[st["keep"].long()] = True
    leaves = ~stays[:, None] & (j >= case["shared"]) & (j < have[:, None])
    order = leaves.flatten().cumsum(0) - 1 + st["n_free"].long()
    size = st["free"].numel()
    spot = torch.where(leaves.flatten(), order, torch.full_like(order, size))
    free = torch.cat([st["free"], st["free"].new_zeros(1)])
    free[spot] = table.flatten()
    st["free"].copy_(free[:size])
    rows = torch.full_like(table, -1)
    kept = st["keep"].long()
    rows[:kept.numel()] = torch.where(j < have[kept][:, None], table[kept], torch.full_like(table[kept], -1))
    kv_out = torch.zeros_like(kv)
    kv_out[:kept.numel()] = kv[kept]
    return {"kv": kv_out.int(), "table": rows, "free": st["free"], "n_free": (st["n_free"].long() + leaves.sum()).int()}


def _rope(st):
    case = st["case"]
    hq, hkv, dh, rows, page = case["hq"], case["hkv"], case["dh"], case["rows"], case["page"]
    x = st["qkv"].float().view(rows, hq + 2 * hkv, dh)
    j = torch.arange(dh // 2, device="cuda", dtype=torch.float64)
    angle = st["pos"].double()[:, None] * torch.pow(torch.tensor(case["theta"], dtype=torch.float64, device="cuda"),
                                                    -2 * j / dh)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turn(u, gain):
        if case["norm"]:
            u = u * torch.rsqrt((u * u).mean(-1, keepdim=True) + 1e-6) * gain.float()
        a, b = u[..., :dh // 2], u[..., dh // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(st["qkv"].dtype)

    st["q"].copy_(turn(x[:, :hq], st["g_q"]).view(rows, hq * dh))
    where, off = st["slot"].long() // page, st["slot"].long() % page
    st["k"][where, :, off] = turn(x[:, hq:hq + hkv], st["g_k"])
    st["v"][where, :, off] = x[:, hq + hkv:].to(st["qkv"].dtype)
    return {"q": st["q"], "k": st["k"], "v": st["v"]}


def _attention(st):
    """Sequences side by side, padded to the longest of their group; one key/value head after the other where the scores
    of all heads would be too many to hold."""
    case = st["case"]
    hq, hkv, dh, page = case["hq"], case["hkv"], case["dh"], case["page"]
    group = hq // hkv
    cached, new = st["host"]
    starts = np.concatenate([[0], np.cumsum(new)])
    room = 1 << 28
    q_all = st["q"].view(-1, hq, dh)
    out = st["out"].view(-1, hq, dh)
    s0 = 0
    while s0 < case["n"]:
        s1, mq, mk = s0, 0, 0
        while s1 < case["n"]:
            a, b = max(mq, int(new[s1])), max(mk, int(cached[s1] + new[s1]))
            if s1 > s0 and (s1 + 1 - s0) * b * max(a * hq, hkv * dh) > room:
                break
            s1, mq, mk = s1 + 1, a, b
        nb = s1 - s0
        if mq == 0:
            s0 = s1
            continue
        pages = int(_pages(mk, page))
        tab = st["table"][s0:s1, :pages].clamp(min=0).long()
        kv, cu = st["kv"][s0:s1].long(), st["cu"][s0:s1 + 1].long()
        t = torch.arange(mq, device="cuda")
        rows = (cu[:-1, None] + t).clamp(max=q_all.shape[0] - 1)
        live_row = t < (cu[1:] - cu[:-1])[:, None]
        key = torch.arange(pages * page, device="cuda")
        seen = (key < kv[:, None])[:, None, :].expand(nb, mq, -1)
        if case["causal"]:
            position = (kv - (cu[1:] - cu[:-1]))[:, None] + t
            seen = seen & (key <= position[:, :, None])
        per = hkv if nb * mq * mk * hq <= room else 1
        for h0 in range(0, hkv, per):
            h1 = h0 + per
            k = st["k"][tab, h0:h1] if per < hkv else st["k"][tab]
            v = st["v"][tab, h0:h1] if per < hkv else st["v"][tab]
            k = k.float().permute(0, 2, 1, 3, 4).reshape(nb, per, pages * page, dh)
            v = v.float().permute(0, 2, 1, 3, 4).reshape(nb, per, pages * page, dh)
            v = torch.where((key < kv[:, None])[:, None, :, None], v, torch.zeros((), device="cuda"))
            q = q_all[rows][:, :, h0 * group:h1 * group].float().view(nb, mq, per, group, dh)
            q = q.permute(0, 2, 1, 3, 4).reshape(nb, per, mq * group, dh)
            s = (torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(dh))).view(nb, per, mq, group, -1)
            s = s.masked_fill(~seen[:, None, :, None], -math.inf)
            top = s.amax(-1, keepdim=True)
            p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
            del s
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p.view(nb, per, mq * group, -1), v).view(nb, per, mq, group, dh)
            del p
            o = o / torch.where(total == 0, torch.ones_like(total), total)
            o = o.permute(0, 2, 1, 3, 4).reshape(nb, mq, per * group, dh)
            out[st["cu"][s0].long() + torch.arange(int(starts[s1] - starts[s0]), device="cuda"),
                h0 * group:h1 * group] = o[live_row].to(out.dtype)
        s0 = s1
    return st["out"]


# ------------------------------------------------------------------------------------------------ definitions, 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "release": _exact_release, "rope": _exact_rope,
            "attn": _exact_attention}[case["op"]](st)


def _exact_append(st):
    page = st["case"]["page"]
    kv, new = st["kv"].cpu().numpy().astype(np.int64), st["new"].cpu().numpy().astype(np.int64)
    table, free = st["table"].cpu().numpy().copy(), list(st["free"].cpu().numpy()[:int(st["n_free"])])
    pos, slot = [], []
    for s in range(len(kv)):
        for t in range(int(kv[s]), int(kv[s] + new[s])):
            if t % page == 0:
                table[s, t // page] = free.pop()
            pos.append(t)
            slot.append(int(table[s, t // page]) * page + t % page)
    return {"kv": _i32(kv + new), "table": _i32(table), "n_free": _i32([len(free)]),
            "cu": _i32(np.concatenate([[0], np.cumsum(new)])), "pos": _i32(np.array(pos, np.int64)),
            "slot": _i32(np.array(slot, np.int64))}


def _exact_release(st):
    case = st["case"]
    kv, table = st["kv"].cpu().numpy(), st["table"].cpu().numpy()
    keep = st["keep"].cpu().numpy()
    free, n_free = st["free"].cpu().numpy().copy(), int(st["n_free"])
    rows, lens = np.full_like(table, -1), np.zeros_like(kv)
    for s in sorted(set(range(len(kv))) - set(int(i) for i in keep)):
        for j in range(case["shared"], -(-int(kv[s]) // case["page"])):
            free[n_free] = table[s, j]
            n_free += 1
    for i, s in enumerate(keep):
        have = -(-int(kv[s]) // case["page"])
        rows[i, :have] = table[s, :have]
        lens[i] = kv[s]
    return {"kv": _i32(lens), "table": _i32(rows), "free": _i32(free), "n_free": _i32([n_free])}


def _exact_rope(st):
    case = st["case"]
    hq, hkv, dh, rows = case["hq"], case["hkv"], case["dh"], case["rows"]
    half = dh // 2
    freq = case["theta"] ** (-np.arange(half, dtype=np.float64) * 2.0 / dh)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       torch.outer(st["pos"].double(), torch.from_numpy(freq).cuda()))[:, None, :]
    x = st["qkv"].double().view(rows, hq + 2 * hkv, dh)
    parts = []
    for lo, hi, gain in ((0, hq, st["g_q"]), (hq, hq + hkv, st["g_k"])):
        u = x[:, lo:hi]
        if case["norm"]:
            u = u / torch.sqrt((u ** 2).sum(-1, keepdim=True) / dh + 1e-6) * gain.double()
        z = torch.complex(u[..., :half].contiguous(), u[..., half:].contiguous()) * turn
        parts.append(torch.cat([z.real, z.imag], -1))
    k, v = st["k"].double(), st["v"].double()
    page, off = st["slot"].long() // case["page"], st["slot"].long() % case["page"]
    k.transpose(1, 2)[page, off] = parts[1]
    v.transpose(1, 2)[page, off] = x[:, hq + hkv:]
    return {"q": parts[0].reshape(rows, hq * dh), "k": k, "v": v}


def _exact_attention(st):
    case = st["case"]
    hq, hkv, dh, page = case["hq"], case["hkv"], case["dh"], case["page"]
    group = hq // hkv
    cached, new = st["host"]
    out = torch.zeros(st["q"].shape[0], hq, dh, dtype=torch.float64, device="cuda")
    q_all = st["q"].view(-1, hq, dh)
    row = 0
    for s in range(case["n"]):
        lq, lk = int(new[s]), int(cached[s] + new[s])
        ids = st["table"][s, :_pages(lk, page)].long()
        for h in range(hkv if lq else 0):
            k = st["k"][ids, h].reshape(-1, dh)[:lk].double()
            v = st["v"][ids, h].reshape(-1, dh)[:lk].double()
            step = max(1, (1 << 27) // (lk * group))
            for t0 in range(0, lq, step):
                t1 = min(lq, t0 + step)
                q = q_all[row + t0:row + t1, h * group:(h + 1) * group].double()
                s_ = torch.einsum("tgd,kd->tgk", q, k) / math.sqrt(dh)
                if case["causal"]:
                    ahead = torch.arange(lk, device="cuda") > (lk - lq + torch.arange(t0, t1, device="cuda"))[:, None]
                    s_.masked_fill_(ahead[:, None], -math.inf)
                p = torch.softmax(s_, -1)
                out[row + t0:row + t1, h * group:(h + 1) * group] = torch.einsum("tgk,kd->tgd", p, v)
        row += lq
    return out.view(-1, hq * dh)
