"""What is measured of the paged cache and of attention over bf16 rows: block tables and slot maps from lengths
(`gvote_page_tables`), rows into pages (`gvote_page_write`), attention over pages (`gvote_page_attend`) and over
slabs (`gvote_attend`).

`run` computes the plain forms in torch, or, with `own` set, calls the library.  A case names its operator, the head
layout, the lengths of its requests and how full each head is; what else a layout needs (rows per head, pages, kept
rows) is drawn from the case's own values, the data from the seed.
"""
import math
import random

import torch

own = False

DEV = "cuda"
RAGGED = "880,4580,321,5252,393,8178,438,9418,395,11730,872,9983,924,7349,703,6059"   # short and long requests mixed


# ----------------------------------------------------------------------------- cases
def listed():
    return [
        # a serving batch's step: rejected draft tokens leave the cache, one to four new ones get their places
        dict(name="tables_step", op="tables", hq=32, hkv=8, d=128, lens=",".join(["1100", "3700", "250", "2050"] * 64), page=16,
             fill_lo=10, fill_hi=90, n_new_lo=1, n_new_hi=4, drop=3, mask=False),
        # sixteen finished requests' pages go to the rows that a keep mask leaves of sixteen new prompts
        dict(name="tables_prompt", op="tables", hq=32, hkv=8, d=128, lens=RAGGED, page=16, fill_lo=10, fill_hi=90,
             keep_lo=5, keep_hi=90, mask=True),
        # one new row per head of 64 requests: latency
        dict(name="write_step", op="write", hq=32, hkv=8, d=128, lens=",".join(["1"] * 64), page=16, keep_lo=100, keep_hi=100),
        # the rows that the pass keeps of a 32K prompt, uneven over the heads
        dict(name="write_prompt", op="write", hq=32, hkv=8, d=128, lens="32768", page=64, keep_lo=5, keep_hi=100),
        # the smallest decode step: latency
        dict(name="decode_small", op="pages", hq=8, hkv=2, d=64, lens="512", page=16, fill_lo=90, fill_hi=100, n_q=1),
        # a decode step of the ragged batch over pruned heads of different length, small pages
        dict(name="decode_ragged", op="pages", hq=32, hkv=8, d=128, lens=RAGGED, page=16, fill_lo=5, fill_hi=90, n_q=1),
        # one token against 128K cached rows, seven query heads to a KV head
        dict(name="decode_long", op="pages", hq=28, hkv=4, d=128, lens="131072", page=64, fill_lo=100, fill_hi=100, n_q=1),
        # the next turn of a conversation: 500 new tokens behind a pruned 32K cache
        dict(name="chunk_pages", op="pages", hq=32, hkv=8, d=128, lens="32768", page=32, fill_lo=20, fill_hi=60, n_q=500),
        # the smallest prompt
        dict(name="prompt_small", op="slabs", hq=8, hkv=2, d=64, lens="512", fill_lo=100, fill_hi=100, n_q=512),
        # sixteen prompts of different length, packed
        dict(name="prompt_ragged", op="slabs", hq=32, hkv=8, d=128, lens=RAGGED, fill_lo=100, fill_hi=100, n_q=1 << 20),
        # a whole 32K prompt
        dict(name="prompt_long", op="slabs", hq=32, hkv=8, d=128, lens="32768", fill_lo=100, fill_hi=100, n_q=1 << 20),
        # a decode step over slabs that the pass has compacted in place
        dict(name="slab_step", op="slabs", hq=32, hkv=8, d=128, lens=RAGGED, fill_lo=5, fill_hi=90, n_q=1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tables", "write", "pages", "pages", "slabs", "slabs"])
    hq, hkv, d = rng.choice([(8, 2, 64), (32, 8, 128), (28, 4, 128), (6, 3, 80), (5, 5, 128), (24, 2, 64), (16, 1, 96)])
    batch = _log_int(rng, 1, 64 if op in ("tables", "write") else 16)
    lens = [_log_int(rng, 1, 65536 // batch) for _ in range(batch)]
    c = dict(op=op, hq=hq, hkv=hkv, d=d)
    if op != "slabs":
        c["page"] = rng.choice([16, 32, 64, 128])
    lo = rng.choice([0, 5, 30, 90])
    hi = rng.randint(max(lo, 50), 100)
    keep = rng.randint(0, 90)
    if op == "tables":
        mask = rng.random() < 0.5
        c.update(lens=",".join(map(str, lens)), fill_lo=lo, fill_hi=hi, mask=mask)
        if mask:
            c.update(keep_lo=keep, keep_hi=rng.randint(keep, 100))
        else:
            new = _log_int(rng, 1, 200)
            c.update(n_new_lo=rng.randint(0, new), n_new_hi=new, drop=rng.randint(0, 8))
        return c
    if op == "write":
        lens = [min(n, 32768) for n in lens]
        c.update(lens=",".join(map(str, lens)), keep_lo=keep, keep_hi=rng.randint(keep, 100))
        return c
    n_q = _log_int(rng, 1, 4096)
    if n_q > 64:
        lens = [min(n, 16384) for n in lens]
    c.update(lens=",".join(map(str, lens)), fill_lo=lo, fill_hi=hi, n_q=n_q)
    return c


def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def _rng(case, what):
    return random.Random(what + repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _fill(case):
    """Rows each head of each request holds, [batch][hkv]."""
    rng = _rng(case, "fill")
    return [[int(round(n * rng.uniform(case["fill_lo"], case["fill_hi"]) / 100)) for _ in range(case["hkv"])] for n in _lens(case)]


def _kept(case):
    """New rows each head of each request keeps, [batch][hkv]."""
    rng = _rng(case, "keep")
    return [[int(n * rng.uniform(case["keep_lo"], case["keep_hi"]) / 100) for _ in range(case["hkv"])] for n in _new(case)]


def _new(case):
    """New tokens of each request."""
    if case["op"] == "write" or case.get("mask"):
        return _lens(case)
    rng = _rng(case, "new")
    return [rng.randint(case["n_new_lo"], case["n_new_hi"]) for _ in _lens(case)]


def _n_q(case):
    """Query tokens of each request: never more than the request has."""
    return [min(case["n_q"], n) for n in _lens(case)]


def _pages_of(rows, page):
    return -(-rows // page)


def _sums(xs):
    out = [0]
    for x in xs:
        out.append(out[-1] + x)
    return out


def work(case):
    """Bytes that have to be read and written once, and the multiply-adds of the definition."""
    hkv, hq, d, op = case["hkv"], case["hq"], case["d"], case["op"]
    if op == "tables":
        new = _new(case)
        got = _kept(case) if case["mask"] else [[n] * hkv for n in new]
        entries, slots, rows = len(new) * hkv, sum(new) * hkv, sum(map(sum, got))
        return {"bytes": 12 * entries + 4 * slots + (slots // 8 if case["mask"] else 0) + 8 * _pages_of(rows, case["page"]),
                "flops": slots + entries}
    if op == "write":
        rows = sum(map(sum, _kept(case)))
        return {"bytes": 8 * d * rows + 4 * hkv * sum(_lens(case)), "flops": 2 * d * rows}
    nq, fill = _n_q(case), _fill(case)
    rows = sum(map(sum, fill))
    pairs = sum(sum(max(0, f - n + i + 1) for i in range(n)) if f < n else n * f - n * (n - 1) // 2
                for n, fr in zip(nq, fill) for f in fr)
    return {"bytes": 4 * d * rows + sum(nq) * hq * (4 * d + 4), "flops": pairs * (hq // hkv) * 4 * d}


# ----------------------------------------------------------------------------- inputs
def _keys(g, hkv, n, d):
    """Cached rows: a few channels much larger than the rest, some rows much larger than the others."""
    x = torch.randn(hkv, n, d, generator=g, device=DEV)
    x[:, :, torch.randperm(d, generator=g, device=DEV)[:4]] *= 8.0
    heavy = torch.rand(hkv, n, 1, generator=g, device=DEV) < 0.02
    return torch.where(heavy, x * 2.5, x).bfloat16()


def _ints(xs):
    return torch.tensor(xs, dtype=torch.int32, device=DEV)


def _pool(g, case, rows, capacity, spare):
    """Pages in disorder: tables [batch, hkv, max_pages] for entries of `rows` rows, the other pages on the free stack."""
    page, hkv = case["page"], case["hkv"]
    counts = [[_pages_of(x, page) for x in xs] for xs in rows]
    most = max(1, _pages_of(capacity, page))
    used = sum(map(sum, counts))
    n_pages = used + spare
    perm = torch.randperm(n_pages, generator=g, device=DEV).int()
    take = torch.arange(most, device=DEV) < torch.tensor(counts, device=DEV).view(-1, 1)
    tables = torch.zeros(len(rows) * hkv, most, dtype=torch.int32, device=DEV)
    tables[take] = perm[:used]
    free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    free[:spare] = perm[used:]
    return dict(tables=tables.view(len(rows), hkv, most), kv_len=_ints(rows).view(len(rows), hkv), free=free,
                n_free=_ints([spare]), n_pages=n_pages)


def _masks(g, case):
    """Keep flags [hkv, total] of the new tokens, and the same as mask words (each request starts on a word)."""
    new, kept, hkv = _new(case), _kept(case), case["hkv"]
    cu = _sums(new)
    keep = torch.zeros(hkv, cu[-1], dtype=torch.bool, device=DEV)
    words = torch.zeros(hkv, cu[-1] // 32 + len(new), dtype=torch.int32, device=DEV)
    weight = torch.tensor([1 << i for i in range(31)] + [-(1 << 31)], dtype=torch.int32, device=DEV)
    for r, n in enumerate(new):
        order = torch.rand(hkv, n, generator=g, device=DEV).argsort(dim=1).argsort(dim=1)
        flags = order < _ints(kept[r])[:, None]
        keep[:, cu[r]:cu[r] + n] = flags
        w = -(-n // 32)
        bits = torch.zeros(hkv, w * 32, dtype=torch.int32, device=DEV)
        bits[:, :n] = flags.int()
        at = cu[r] // 32 + r
        words[:, at:at + w] = (bits.view(hkv, w, 32) * weight).sum(dim=2, dtype=torch.int32)
    return keep, words


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op, hq, hkv, d, lens = case["op"], case["hq"], case["hkv"], case["d"], _lens(case)
    batch = len(lens)
    st = dict(case=case)
    tq = mq = 0
    if op == "tables":
        new, fill = _new(case), _fill(case)
        if case["mask"]:
            keep = [[0] * hkv for _ in lens]                  # the requests that had these entries have ended
            grow = _kept(case)
            st["flags"], st["mask"] = _masks(g, case)
        else:
            rng = _rng(case, "drop")
            keep = [[max(0, f - k) for f in fr] for fr in fill for k in [rng.randint(0, case["drop"])]]
            grow = [[n] * hkv for n in new]
            st["mask"] = None
        cap = max(max(lens), max(f + x for fr, xr in zip(fill, grow) for f, x in zip(fr, xr)))
        need = sum(_pages_of(x, case["page"]) + 1 for xr in grow for x in xr)
        st.update(_pool(g, case, fill, cap, need + 5))
        st.update(new=new, keep=_ints(keep).view(batch, hkv), cu_new=_ints(_sums(new)), total_new=sum(new),
                  slots=torch.zeros(hkv, sum(new), dtype=torch.int32, device=DEV))
        st["K"] = st["V"] = torch.zeros(st["n_pages"], case["page"], d, dtype=torch.bfloat16, device=DEV)
    elif op == "write":
        total, kept = sum(lens), _kept(case)
        st.update(_pool(g, case, kept, max(map(max, kept)), 7))
        keep, _ = _masks(g, case)
        slots = torch.full((hkv, total), -1, dtype=torch.int32, device=DEV)
        cu = _sums(lens)
        for r in range(batch):
            for h in range(hkv):
                at = keep[h, cu[r]:cu[r + 1]].nonzero()[:, 0]
                i = torch.arange(kept[r][h], device=DEV)
                slots[h, cu[r] + at] = (st["tables"][r, h, i // case["page"]] * case["page"] + i % case["page"]).int()
        st["slots"] = slots
        st["K_new"], st["V_new"] = _keys(g, hkv, total, d), torch.randn(hkv, total, d, generator=g, device=DEV).bfloat16()
        st["K"], st["V"] = (torch.zeros(st["n_pages"], case["page"], d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    else:
        nq, fill = _n_q(case), _fill(case)
        tq, mq = sum(nq), max(nq)
        st.update(nq=nq, fill=fill, cu_q=_ints(_sums(nq)), max_q=mq)
        st["Q"] = (torch.randn(tq, hq, d, generator=g, device=DEV) * 1.5).bfloat16()
        st["out"] = torch.zeros(tq, hq, d, dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.zeros(tq, hq, device=DEV)
        if op == "pages":
            st.update(_pool(g, case, fill, max(lens), 11))
            n, page = st["n_pages"], case["page"]
            st["K"] = _keys(g, 1, n * page, d).view(n, page, d)
            st["V"] = torch.randn(n, page, d, generator=g, device=DEV).bfloat16()
        else:
            total = sum(lens)
            st["K"], st["V"] = _keys(g, hkv, total, d), torch.randn(hkv, total, d, generator=g, device=DEV).bfloat16()
            st["cu"], st["geom"] = _ints(_sums(lens)), (batch, total, max(lens))
            st["kv_len"] = None if case["fill_lo"] == 100 else _ints(fill).view(batch, hkv)
    if own:
        from paper_2509_03136_b200 import gvote as gv
        st["gv"] = gv
        st["p"] = gv.make_params(d_h=64, n_q_heads=hq, n_kv_heads=hkv, d_k=d, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1,
                                 n_s=4, seed=0)
        st["ws"] = gv.alloc_attend_workspace(st["p"], batch, tq, mq)
        if op != "slabs":
            st["pages"] = gv.PageCache(st["K"], st["V"], st["tables"], st["kv_len"], st["free"], st["n_free"])
    return st


# ----------------------------------------------------------------------------- one pass
def _run_own(st):
    gv, p, ws, op = st["gv"], st["p"], st["ws"], st["case"]["op"]
    if op == "tables":
        gv.gvote_page_tables(p, st["pages"], ws, keep=st["keep"], cu_new=st["cu_new"], max_new=max(st["new"]),
                             slots=st["slots"], mask=st["mask"])
        return [st["tables"], st["kv_len"], st["free"], st["n_free"], st["slots"]]
    if op == "write":
        gv.gvote_page_write(p, st["K_new"], st["V_new"], st["slots"], st["pages"], ws)
        return [st["K"], st["V"]]
    if op == "pages":
        gv.gvote_page_attend(p, st["Q"], st["cu_q"], st["max_q"], st["pages"], st["out"], ws, lse=st["lse"])
    else:
        gv.gvote_attend(p, st["Q"], st["cu_q"], st["max_q"], st["K"], st["V"], st["cu"], st["geom"], st["out"], ws,
                        lse=st["lse"], kv_len=st["kv_len"])
    return [st["out"], st["lse"]]


def _plain_tables(st):
    """Cut, give pages back, take pages, place the new rows: cumulative sums and scatters (a spare last element takes
    what goes nowhere)."""
    page, hkv = st["case"]["page"], st["case"]["hkv"]
    batch, _, most = st["tables"].shape
    new = st["cu_new"][1:] - st["cu_new"][:-1]
    request = torch.repeat_interleave(torch.arange(batch, device=DEV), new, output_size=st["total_new"])
    if st["mask"] is None:
        keep = torch.ones(hkv, st["total_new"], dtype=torch.int64, device=DEV)
    else:
        t = torch.arange(st["total_new"], device=DEV) - st["cu_new"][request]
        word = (st["cu_new"][request] >> 5) + request + (t >> 5)
        keep = ((st["mask"][:, word] >> (t & 31).int()) & 1).long()
    before = torch.cat([torch.zeros(hkv, 1, dtype=torch.int64, device=DEV), keep.cumsum(dim=1)], dim=1)
    at = before[:, st["cu_new"].long()]                                       # kept rows before each request
    held = st["kv_len"].clamp(0, most * page).long().view(-1)
    cut = torch.minimum(held, st["keep"].clamp_min(0).long().view(-1))
    grown = cut + (at[:, 1:] - at[:, :-1]).t().reshape(-1)
    n_held, n_cut, n_grown = (-(-x // page) for x in (held, cut, grown))
    column = torch.arange(most, device=DEV)
    tables, spare = st["tables"].long().view(-1, most), st["free"].numel()

    gone = (column >= n_cut[:, None]) & (column < n_held[:, None])
    n_gone = (n_held - n_cut).clamp_min(0).sum()
    rank = gone.view(-1).long().cumsum(0).view(gone.shape) - 1
    stack = torch.cat([st["free"].long(), torch.zeros(1, dtype=torch.int64, device=DEV)])
    top = st["n_free"].long() + n_gone
    stack.index_put_((torch.where(gone, top - 1 - rank, spare),), tables)

    want = (column >= n_cut[:, None]) & (column < n_grown[:, None])
    rank = want.view(-1).long().cumsum(0).view(want.shape) - 1
    tables = torch.where(want, stack[torch.where(want, top - 1 - rank, spare)], tables)
    n_free = top - want.sum()

    place = cut.view(batch, hkv).t()[:, request] + before[:, :-1] - at[:, :-1][:, request]
    entry = request[None, :] * hkv + torch.arange(hkv, device=DEV)[:, None]
    slot = tables[entry, (place // page).clamp_max(most - 1)] * page + place % page
    slots = torch.where(keep > 0, slot, -1)
    return [tables.int().view(batch, hkv, most), grown.int().view(batch, hkv), stack[:-1].int(), n_free.int(), slots.int()]


def _plain_write(st):
    out = []
    last = st["n_pages"] * st["case"]["page"]
    at = torch.where(st["slots"] < 0, last, st["slots"]).long().view(-1)
    for pool, rows in ((st["K"], st["K_new"]), (st["V"], st["V_new"])):
        buf = torch.cat([pool.view(last, -1), pool.new_zeros(1, pool.shape[2])])
        buf.index_copy_(0, at, rows.reshape(-1, rows.shape[2]))
        out.append(buf[:last].view(pool.shape))
    return out


def _request_rows(st, r):
    """Keys and values of one request, [hkv, longest head, d] (rows behind a shorter head's last are anything)."""
    case = st["case"]
    longest = max(1, max(st["fill"][r]))
    if case["op"] == "slabs":
        a = _sums(_lens(case))[r]
        return st["K"][:, a:a + longest], st["V"][:, a:a + longest]
    i = torch.arange(longest, device=DEV)
    at = st["tables"][r][:, i // case["page"]].long() * case["page"] + i % case["page"]
    return st["K"].view(-1, case["d"])[at], st["V"].view(-1, case["d"])[at]


def _plain_attend(st):
    case = st["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    out, lse = torch.empty(st["Q"].shape, device=DEV), torch.empty(st["Q"].shape[:2], device=DEV)
    q0 = 0
    for r, n in enumerate(st["nq"]):
        held = st["fill"][r]
        rows = _ints(held).view(hkv, 1)
        k, v = (x.float() for x in _request_rows(st, r))
        v = torch.where((torch.arange(v.shape[1], device=DEV) < rows)[:, :, None], v, 0.0)
        step = max(1, (1 << 27) // (hq * k.shape[1]))
        for a in range(0, n, step):
            b = min(n, a + step)
            seen = max(1, max(held) - n + b)                                  # the keys that the last of these tokens sees
            q = st["Q"][q0 + a:q0 + b].float().view(b - a, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
            logit = torch.matmul(q, k[:, :seen].transpose(1, 2)).view(hkv, -1, b - a, seen) / math.sqrt(d)
            limit = rows - n + 1 + torch.arange(a, b, device=DEV)
            logit.masked_fill_(~(torch.arange(seen, device=DEV) < limit[:, None, :, None]), -math.inf)
            top = logit.amax(dim=-1, keepdim=True)
            top = torch.where(top == -math.inf, 0.0, top)
            weight = torch.exp(logit - top)
            total = weight.sum(dim=-1, keepdim=True)
            o = torch.matmul(weight.view(hkv, -1, seen), v[:, :seen]).view(hkv, -1, b - a, d)
            o = torch.where(total > 0, o / total, 0.0)
            out[q0 + a:q0 + b] = o.permute(2, 0, 1, 3).reshape(b - a, hq, d)
            lse[q0 + a:q0 + b] = (top + torch.log(total)).squeeze(-1).permute(2, 0, 1).reshape(b - a, hq)
        q0 += n
    return [out.bfloat16(), lse]


def run(st):
    if own:
        return _run_own(st)
    op = st["case"]["op"]
    return _plain_tables(st) if op == "tables" else _plain_write(st) if op == "write" else _plain_attend(st)


# ----------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    if case["op"] == "tables":
        return None                                                           # whole numbers only
    st = prepare(case, seed)
    if case["op"] == "write":
        pools = [torch.zeros(st["n_pages"] * case["page"], case["d"], dtype=torch.float64, device=DEV) for _ in range(2)]
        for h, slots in enumerate(st["slots"]):
            kept = (slots >= 0).nonzero()[:, 0]
            for pool, rows in zip(pools, (st["K_new"], st["V_new"])):
                pool[slots[kept].long()] = rows[h, kept].double()
        return [pool.view(st["n_pages"], case["page"], case["d"]) for pool in pools]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    group = hq // hkv
    out = torch.zeros(st["Q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(st["Q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    first = 0
    for r, n in enumerate(st["nq"]):
        for h in range(hkv):
            held = st["fill"][r][h]
            if case["op"] == "slabs":
                start = sum(_lens(case)[:r])
                k, v = st["K"][h, start:start + held].double(), st["V"][h, start:start + held].double()
            else:
                ids = st["tables"][r, h, :_pages_of(held, case["page"])].long()
                k, v = (st[x][ids].flatten(0, 1)[:held].double() for x in "KV")
            begin = max(0, n - held)                                          # the tokens before see nothing
            step = max(1, (1 << 26) // (group * max(1, held)))
            for a in range(begin, n, step):
                b = min(n, a + step)
                seen = held - n + b
                q = st["Q"][first + a:first + b, h * group:(h + 1) * group].double()
                l = torch.einsum("tgd,nd->gtn", q, k[:seen]) * d ** -0.5
                last = torch.arange(held - n + a, held - n + b, device=DEV)
                l = l.masked_fill(torch.arange(seen, device=DEV)[None, :] > last[:, None], -math.inf)
                z = torch.logsumexp(l, dim=2)
                out[first + a:first + b, h * group:(h + 1) * group] = torch.einsum("gtn,nd->tgd", torch.exp(l - z[:, :, None]), v[:seen])
                lse[first + a:first + b, h * group:(h + 1) * group] = z.t()
        first += n
    return [out, lse]
