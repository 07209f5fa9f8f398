"""What is measured of the pruned-cache operators: an 8-bit cache that takes the rows a pass keeps
(`gvote_store8`, `gvote_prune8`), grows by new tokens (`gvote_append8`) and is attended to
(`gvote_attend8`), and eviction by accumulated attention weight (`gvote_accumulate`, `gvote_evict`).

`run` computes the plain forms in torch (fp32), or, with `own` set, calls the library.  A case names its
operator, the head layout, the slab lengths of its requests and how full each head's slab is.  The
lengths are drawn from the case's own values, the data from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 64                      # rows of one head that share a scale
E4M3_MAX = 448.0
DEV = "cuda"


# ----------------------------------------------------------------------------- cases
RAGGED = "880,4580,321,5252,393,8178,438,9418,395,11730,872,9983,924,7349,703,6059"   # short and long requests mixed


def listed():
    return [
        # the end of a 32K prompt: the rows a keep mask leaves go to the 8-bit cache, uneven over the heads
        dict(name="store_prompt", op="store", hq=32, hkv=8, d=128, lens="32768", fill_lo=100, fill_hi=100,
             keep_lo=5, keep_hi=100),
        # a serving batch whose 8-bit cache is pruned once more
        dict(name="prune_ragged", op="prune", hq=32, hkv=8, d=128, lens=RAGGED, fill_lo=30, fill_hi=90,
             keep_lo=30, keep_hi=70),
        # one new token for each request of the batch
        dict(name="append_step", op="append", hq=32, hkv=8, d=128, lens=RAGGED, fill_lo=30, fill_hi=90, n_new=1),
        # three draft tokens of a small model's only request
        dict(name="append_small", op="append", hq=8, hkv=2, d=64, lens="512", fill_lo=60, fill_hi=90, n_new=3),
        # the smallest decode step: latency
        dict(name="attend_small", op="attend", hq=8, hkv=2, d=64, lens="512", fill_lo=90, fill_hi=100, n_q=1, acc=False),
        # a decode step of the ragged batch over pruned heads of different length, weights accumulated
        dict(name="attend_ragged", op="attend", hq=32, hkv=8, d=128, lens=RAGGED, fill_lo=5, fill_hi=90, n_q=1, acc=True),
        # five draft tokens checked against a 32K request, weights accumulated
        dict(name="attend_draft", op="attend", hq=32, hkv=8, d=128, lens="32768", fill_lo=20, fill_hi=100, n_q=5, acc=True),
        # one token against 128K cached tokens, seven query heads to a KV head
        dict(name="attend_long", op="attend", hq=28, hkv=4, d=128, lens="131072", fill_lo=100, fill_hi=100, n_q=1, acc=False),
        # the weights all tokens of a 32K prompt give to its keys
        dict(name="accumulate_prompt", op="accumulate", hq=32, hkv=8, d=128, lens="32768", n_q=32768),
        # the weights the last 32 tokens of a 128K prompt give to its keys
        dict(name="accumulate_window", op="accumulate", hq=28, hkv=4, d=128, lens="131072", n_q=32),
        # which rows of the ragged batch stay: half of the slab's size, sinks and a recent window among them
        dict(name="evict_ragged", op="evict", hq=32, hkv=8, d=128, lens=RAGGED, fill_lo=30, fill_hi=100, keep_lo=10,
             keep_hi=60, n_recent=32),
        # which of 128K rows stay
        dict(name="evict_long", op="evict", hq=28, hkv=4, d=128, lens="131072", fill_lo=100, fill_hi=100, keep_lo=5,
             keep_hi=20, n_recent=512),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["store", "prune", "append", "attend", "attend", "accumulate", "evict"])
    hq, hkv, d = rng.choice([(8, 2, 64), (32, 8, 128), (28, 4, 128), (6, 3, 80), (5, 5, 128), (24, 2, 64)])
    batch = _log_int(rng, 1, 16)
    top = 65536 // batch
    lens = [_log_int(rng, 1, top) for _ in range(batch)]
    c = dict(op=op, hq=hq, hkv=hkv, d=d)
    if op == "accumulate":
        n_q = _log_int(rng, 1, 4096)
        lens = [min(n, 16384) for n in lens]
        c.update(lens=",".join(map(str, lens)), n_q=n_q)
        return c
    lo = rng.choice([0, 5, 30, 90])
    c.update(lens=",".join(map(str, lens)), fill_lo=lo, fill_hi=rng.randint(max(lo, 50), 100))
    if op in ("store", "prune", "evict"):
        k = rng.randint(0, 90)
        c.update(keep_lo=k, keep_hi=rng.randint(k, 100))
    if op == "evict":
        c["n_recent"] = rng.choice([0, 1, 32, 500])
    if op == "append":
        c["n_new"] = _log_int(rng, 1, 80)
    if op == "attend":
        c.update(n_q=_log_int(rng, 1, 8), acc=rng.random() < 0.5)
    return c


def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def _fill(case):
    """Rows each head of each request holds, [batch][hkv]: from the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    lo, hi = case.get("fill_lo", 100), case.get("fill_hi", 100)
    return [[int(round(n * rng.uniform(lo, hi) / 100)) for _ in range(case["hkv"])] for n in _lens(case)]


def _shares(case):
    """Share of its rows each head keeps, [batch][hkv]: from the case alone."""
    rng = random.Random("keep" + repr(sorted((k, v) for k, v in case.items() if k != "name")))
    return [[rng.uniform(case["keep_lo"], case["keep_hi"]) / 100 for _ in range(case["hkv"])] for _ in _lens(case)]


def _n_q(case, n):
    """Query tokens of a request with n rows: a window is never longer than the prompt."""
    return min(case["n_q"], n) if case["op"] == "accumulate" else case["n_q"]


def work(case):
    """Bytes that have to be read and written once, and the multiply-adds of the definition."""
    lens, fill, d, hkv, hq = _lens(case), _fill(case), case["d"], case["hkv"], case["hq"]
    op = case["op"]
    rows = sum(map(sum, fill))
    if op in ("store", "prune"):
        share = _shares(case)
        kept = sum(int(f * s) for fr, sr in zip(fill, share) for f, s in zip(fr, sr))
        src = 2 * d * (2 if op == "store" else 1)
        return {"bytes": kept * (src + 2 * d + 16) + rows // 8, "flops": kept * 2 * d}
    if op == "append":
        touched = sum(min(f % BLOCK, f) + case["n_new"] for fr in fill for f in fr)
        new = len(lens) * hkv * case["n_new"]
        return {"bytes": new * 2 * d * 3 + 8 * len(lens) * hkv, "flops": touched * 2 * d}
    if op == "attend":
        g = hq // hkv
        q = len(lens) * case["n_q"] * hq * d * 2
        return {"bytes": rows * (2 * d + (8 if case["acc"] else 0)) + rows // BLOCK * 8 + 2 * q,
                "flops": rows * case["n_q"] * g * 4 * d}
    if op == "accumulate":
        pairs = sum(_n_q(case, n) * (n - (_n_q(case, n) - 1) / 2) for n in lens)
        q = sum(_n_q(case, n) for n in lens) * hq * d * 2
        return {"bytes": int(sum(lens) * hkv * (2 * d + 8) + q), "flops": int(pairs * hq * 2 * d)}
    return {"bytes": rows * 4 + rows // 8 + 8 * len(lens) * hkv, "flops": rows}


# ----------------------------------------------------------------------------- inputs
def _keys(g, hkv, n, d):
    """Cached rows: a few channels much larger than the rest, some rows much larger than the others."""
    x = torch.randn(hkv, n, d, generator=g, device=DEV)
    chan = torch.randperm(d, generator=g, device=DEV)[:4]
    x[:, :, chan] *= 8.0
    heavy = torch.rand(hkv, n, 1, generator=g, device=DEV) < 0.02
    return torch.where(heavy, x * 2.5, x).bfloat16()


def _scale_of(amax):
    """The smallest power of two s >= 2^-126 with amax <= 448 s (448 = 0.875 * 2^9)."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(amax > 0, e, torch.full_like(e, -126)).clamp_min(-126)
    return torch.ldexp(torch.ones_like(amax), e)


def _quantise(x):
    """Rows [n, d] fp32 -> (e4m3 codes, one scale per 64 rows)."""
    n, d = x.shape
    nb = (n + BLOCK - 1) // BLOCK
    pad = torch.zeros(nb * BLOCK, d, device=x.device)
    pad[:n] = x
    pad = pad.view(nb, BLOCK * d)
    s = _scale_of(pad.abs().amax(dim=1)) if nb else torch.empty(0, device=x.device)
    codes = (pad / s[:, None]).to(torch.float8_e4m3fn).view(nb * BLOCK, d)[:n]
    return codes, s


def _block_off(cu_r, r):
    return (cu_r // BLOCK) + r


class _Cache:
    """An 8-bit cache in the layout the library uses: codes [hkv, total, d], scales [hkv, blocks]."""

    def __init__(self, case, fill):
        lens, hkv, d = _lens(case), case["hkv"], case["d"]
        self.cu = [0]
        for n in lens:
            self.cu.append(self.cu[-1] + n)
        total, batch = self.cu[-1], len(lens)
        self.codes = [torch.zeros(hkv, total, d, dtype=torch.uint8, device=DEV) for _ in range(2)]
        self.scale = [torch.zeros(hkv, total // BLOCK + batch, device=DEV) for _ in range(2)]
        self.kv_len = torch.tensor(fill, dtype=torch.int32, device=DEV).view(batch, hkv)
        self.cu_dev = torch.tensor(self.cu, dtype=torch.int32, device=DEV)
        self.geom = (batch, total, max(lens))

    def put(self, which, r, h, rows):
        codes, s = _quantise(rows)
        a = self.cu[r]
        self.codes[which][h, a:a + codes.shape[0]] = codes.view(torch.uint8)
        b = _block_off(a, r)
        self.scale[which][h, b:b + s.numel()] = s

    def rows(self, which, r, h, n):
        a, b = self.cu[r], _block_off(self.cu[r], r)
        s = self.scale[which][h, b:b + (n + BLOCK - 1) // BLOCK].repeat_interleave(BLOCK)[:n]
        return self.codes[which][h, a:a + n].view(torch.float8_e4m3fn).float() * s[:, None]

    def outputs(self):
        return [c.view(torch.float8_e4m3fn) for c in self.codes] + self.scale


def _pack_mask(keep, cu, words):
    """Keep flags [hkv, total] -> mask words [hkv, words] (each request starts on a word)."""
    hkv = keep.shape[0]
    mask = torch.zeros(hkv, words, dtype=torch.int32, device=keep.device)
    weights = torch.tensor([1 << i for i in range(31)] + [-(1 << 31)], dtype=torch.int32, device=keep.device)
    for r in range(len(cu) - 1):
        n = cu[r + 1] - cu[r]
        w = (n + 31) // 32
        bits = torch.zeros(hkv, w * 32, dtype=torch.int32, device=keep.device)
        bits[:, :n] = keep[:, cu[r]:cu[r + 1]].int()
        off = cu[r] // 32 + r
        mask[:, off:off + w] = (bits.view(hkv, w, 32) * weights).sum(dim=2, dtype=torch.int32)
    return mask


def _unpack_mask(mask, cu, total):
    bit = torch.arange(32, device=mask.device, dtype=torch.int32)
    keep = torch.zeros(mask.shape[0], total, dtype=torch.bool, device=mask.device)
    for r in range(len(cu) - 1):
        n = cu[r + 1] - cu[r]
        off = cu[r] // 32 + r
        w = mask[:, off:off + (n + 31) // 32]
        keep[:, cu[r]:cu[r + 1]] = ((w[:, :, None] >> bit) & 1).bool().flatten(1)[:, :n]
    return keep


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    lens, fill, hkv, hq, d, op = _lens(case), _fill(case), case["hkv"], case["hq"], case["d"], case["op"]
    batch = len(lens)
    cache = _Cache(case, fill)
    cu, total = cache.cu, cache.cu[-1]
    st = dict(case=case, cache=cache, cu=cu, lens=lens, fill=fill)
    words = total // 32 + batch
    full = _keys(g, hkv, total, d), torch.randn(hkv, total, d, generator=g, device=DEV).bfloat16()
    if op in ("prune", "append", "attend"):
        for r in range(batch):
            for h in range(hkv):
                for w in range(2):
                    cache.put(w, r, h, full[w][h, cu[r]:cu[r] + fill[r][h]].float())
    if op in ("store", "prune", "evict", "append") or case.get("acc"):
        # weights collected so far: a few rows hold most, rows not looked at yet hold none
        acc = torch.exp(2.5 * torch.randn(hkv, total, generator=g, device=DEV)) * 0.01
        st["acc"] = torch.where(torch.rand(hkv, total, generator=g, device=DEV) < 0.05, torch.zeros_like(acc), acc)
    if op in ("store", "prune"):
        keep = torch.zeros(hkv, total, dtype=torch.bool, device=DEV)
        share = _shares(case)
        for r in range(batch):
            for h in range(hkv):
                n = fill[r][h]
                pick = torch.randperm(n, generator=g, device=DEV)[:int(n * share[r][h])]
                keep[h, cu[r] + pick] = True
        st["mask"] = _pack_mask(keep, cu, words)
        st["out"] = _Cache(case, [[0] * hkv for _ in lens])
        st["token_pos"] = (torch.arange(total, device=DEV, dtype=torch.int32).expand(hkv, total) * 2).contiguous()
        st["acc_out"] = torch.zeros(hkv, total, device=DEV)
        st["pos_out"] = torch.zeros(hkv, total, dtype=torch.int32, device=DEV)
        if op == "store":
            st["K"], st["V"] = full
    if op == "append":
        n_new = case["n_new"]
        st["n_new"] = [min(n_new, n - max(f)) for n, f in zip(lens, fill)]
        tot_new = sum(st["n_new"])
        st["K_new"], st["V_new"] = _keys(g, hkv, max(tot_new, 1), d)[:, :tot_new].contiguous(), torch.randn(
            hkv, tot_new, d, generator=g, device=DEV).bfloat16()
        st["cu_new"] = torch.tensor(np.concatenate([[0], np.cumsum(st["n_new"])]), dtype=torch.int32, device=DEV)
        st["kv_len_out"] = torch.zeros_like(cache.kv_len)
    if op in ("attend", "accumulate"):
        nq = [_n_q(case, n) for n in lens]
        st["nq"], tq = nq, sum(nq)
        st["Q"] = (torch.randn(tq, hq, d, generator=g, device=DEV) * 1.5).bfloat16()
        st["cu_q"] = torch.tensor(np.concatenate([[0], np.cumsum(nq)]), dtype=torch.int32, device=DEV)
        if op == "accumulate":
            st["K"] = full[0]
            st["acc_out"] = torch.zeros(hkv, total, device=DEV)
        else:
            st["o"] = torch.zeros(tq, hq, d, dtype=torch.bfloat16, device=DEV)
            st["lse"] = torch.zeros(tq, hq, device=DEV)
            if case["acc"]:
                st["acc_out"] = torch.zeros(hkv, total, device=DEV)
    if op == "evict":
        share = _shares(case)
        st["keep"] = torch.tensor([[int(n * s) for s in sr] for n, sr in zip(lens, share)], dtype=torch.int32,
                                  device=DEV).view(batch, hkv)
        st["mask"] = torch.zeros(hkv, words, dtype=torch.int32, device=DEV)
        st["budget"] = torch.zeros(batch, hkv, dtype=torch.int32, device=DEV)
    if own:
        from paper_2509_03136_b200 import gvote as gv
        st["gv"] = gv
        st["p"] = gv.make_params(d_h=64, n_q_heads=hq, n_kv_heads=hkv, d_k=d, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1,
                                 n_s=4, seed=0)
        tq, mq = (sum(st["nq"]), max(st["nq"])) if "nq" in st else (0, 0)
        st["max_q"] = mq
        st["ws"] = gv.alloc_cache_workspace(st["p"], *cache.geom, tq, mq)
        st["cache8"] = gv.Cache8(*cache.codes, *cache.scale, cache.cu_dev, cache.kv_len, cache.geom)
        if "out" in st:
            o = st["out"]
            st["out8"] = gv.Cache8(*o.codes, *o.scale, o.cu_dev, o.kv_len, o.geom)
    return st


# ----------------------------------------------------------------------------- one pass
def _run_own(st):
    gv, p, ws, c, op = st["gv"], st["p"], st["ws"], st["cache8"], st["case"]["op"]
    if op == "store":
        gv.gvote_store8(p, st["K"], st["V"], c.cu_seqlens, c.geom, st["out8"], ws, mask=st["mask"], kv_len=c.kv_len,
                        acc=st["acc"], acc_out=st["acc_out"], token_pos=st["token_pos"], token_pos_out=st["pos_out"])
    elif op == "prune":
        gv.gvote_prune8(p, c, st["mask"], st["out8"], ws, acc=st["acc"], acc_out=st["acc_out"],
                        token_pos=st["token_pos"], token_pos_out=st["pos_out"])
    elif op == "append":
        gv.gvote_append8(p, st["K_new"], st["V_new"], st["cu_new"], max(st["n_new"]), c, st["kv_len_out"], ws,
                         acc=st["acc"])
    elif op == "attend":
        gv.gvote_attend8(p, st["Q"], st["cu_q"], st["max_q"], c, st["o"], ws, lse=st["lse"], acc=st.get("acc"),
                         acc_out=st.get("acc_out"))
    elif op == "accumulate":
        gv.gvote_accumulate(p, st["Q"], st["cu_q"], st["max_q"], st["K"], c.cu_seqlens, c.geom, st["acc_out"], ws)
    else:
        gv.gvote_evict(p, st["acc"], c.cu_seqlens, c.geom, st["keep"], st["case"]["n_recent"], st["mask"],
                       st["budget"], ws, kv_len=c.kv_len)


def _results(st):
    op = st["case"]["op"]
    if op in ("store", "prune"):
        return st["out"].outputs() + [st["out"].kv_len, st["acc_out"], st["pos_out"]]
    if op == "append":
        return st["cache"].outputs() + [st["kv_len_out"], st["acc"]]
    if op == "attend":
        return [st["o"], st["lse"]] + ([st["acc_out"]] if st["case"]["acc"] else [])
    if op == "accumulate":
        return [st["acc_out"]]
    return [st["mask"], st["budget"]]


def _plain_store(st):
    cache, out, cu, fill = st["cache"], st["out"], st["cu"], st["fill"]
    hkv, total = cache.codes[0].shape[:2]
    keep = _unpack_mask(st["mask"], cu, total)
    lens = []
    for r in range(len(cu) - 1):
        for h in range(hkv):
            idx = keep[h, cu[r]:cu[r] + fill[r][h]].nonzero()[:, 0]
            m = idx.numel()
            for w in range(2):
                rows = (st["K"], st["V"])[w][h, cu[r] + idx].float() if "K" in st else cache.rows(w, r, h, fill[r][h])[idx]
                out.put(w, r, h, rows)
            st["acc_out"][h, cu[r]:cu[r] + m] = st["acc"][h, cu[r] + idx]
            st["pos_out"][h, cu[r]:cu[r] + m] = st["token_pos"][h, cu[r] + idx]
            lens.append(m)
    out.kv_len.copy_(torch.tensor(lens, dtype=torch.int32, device=DEV).view_as(out.kv_len))


def _plain_append(st):
    cache, cu, fill = st["cache"], st["cu"], st["fill"]
    hkv = cache.codes[0].shape[0]
    at = 0
    lens = []
    for r in range(len(cu) - 1):
        n_new = st["n_new"][r]
        for h in range(hkv):
            n = fill[r][h]
            for w in range(2):
                new = (st["K_new"], st["V_new"])[w][h, at:at + n_new].float()
                codes, scale = cache.codes[w][h], cache.scale[w][h]
                done = 0
                while done < n_new:
                    row = n + done
                    first = row - row % BLOCK
                    take = min(BLOCK - row % BLOCK, n_new - done)
                    x = new[done:done + take]
                    b = _block_off(cu[r], r) + first // BLOCK
                    s = _scale_of(x.abs().amax()[None])
                    a, m = cu[r] + first, row - first
                    if m:                                      # rows the block holds already
                        s = torch.maximum(s, scale[b:b + 1])
                        old = codes[a:a + m].view(torch.float8_e4m3fn).float() * (scale[b] / s)
                        codes[a:a + m] = old.to(torch.float8_e4m3fn).view(torch.uint8)
                    codes[a + m:a + m + take] = (x / s).to(torch.float8_e4m3fn).view(torch.uint8)
                    scale[b:b + 1] = s
                    done += take
            st["acc"][h, cu[r] + n:cu[r] + n + n_new] = 0
            lens.append(n + n_new)
        at += n_new
    st["kv_len_out"].copy_(torch.tensor(lens, dtype=torch.int32, device=DEV).view_as(st["kv_len_out"]))


def _seen(n, n_q, first, count):
    """Rows the query tokens first .. first+count-1 of n_q see among n rows, [count, 1]."""
    return n - (n_q - 1 - torch.arange(first, first + count, device=DEV))[:, None]


def _plain_attend(st):
    cache, case, cu, fill = st["cache"], st["case"], st["cu"], st["fill"]
    hkv, d, g, nq = case["hkv"], case["d"], case["hq"] // case["hkv"], case["n_q"]
    if case["acc"]:
        st["acc_out"].zero_()
    for r in range(len(cu) - 1):
        for h in range(hkv):
            n = fill[r][h]
            q = st["Q"][r * nq:(r + 1) * nq, h * g:(h + 1) * g].float()                    # [nq, g, d]
            k, v = cache.rows(0, r, h, n), cache.rows(1, r, h, n)
            logit = (q.reshape(nq * g, d) @ k.T).view(nq, g, n) / math.sqrt(d)
            hide = torch.arange(n, device=DEV)[None, :] >= _seen(n, nq, 0, nq)             # [nq, n]
            logit = logit.masked_fill(hide[:, None, :], -math.inf)
            top = logit.amax(dim=2, keepdim=True) if n else torch.full((nq, g, 1), -math.inf, device=DEV)
            e = torch.exp(logit - torch.where(top == -math.inf, torch.zeros_like(top), top))
            z = e.sum(dim=2, keepdim=True)
            w = e / torch.where(z == 0, torch.ones_like(z), z)
            st["o"][r * nq:(r + 1) * nq, h * g:(h + 1) * g] = (w.view(nq * g, n) @ v).view(nq, g, d).bfloat16()
            st["lse"][r * nq:(r + 1) * nq, h * g:(h + 1) * g] = (top + torch.log(z))[:, :, 0]
            if case["acc"]:
                st["acc_out"][h, cu[r]:cu[r] + n] = st["acc"][h, cu[r]:cu[r] + n] + w.sum(dim=(0, 1))


def _plain_accumulate(st):
    case, cu = st["case"], st["cu"]
    hkv, d, g = case["hkv"], case["d"], case["hq"] // case["hkv"]
    at = 0
    for r in range(len(cu) - 1):
        n, nq = cu[r + 1] - cu[r], st["nq"][r]
        chunk = max(1, min(nq, (1 << 27) // max(1, n * g)))
        for h in range(hkv):
            k = st["K"][h, cu[r]:cu[r + 1]].float()
            total = torch.zeros(n, dtype=torch.float64, device=DEV)
            for a in range(0, nq, chunk):
                c = min(chunk, nq - a)
                q = st["Q"][at + a:at + a + c, h * g:(h + 1) * g].float().reshape(c * g, d)
                logit = (q @ k.T).view(c, g, n) / math.sqrt(d)
                hide = torch.arange(n, device=DEV)[None, :] >= _seen(n, nq, a, c)
                logit = logit.masked_fill_(hide[:, None, :], -math.inf)
                e = torch.exp_(logit.sub_(logit.amax(dim=2, keepdim=True)))
                total += e.div_(e.sum(dim=2, keepdim=True)).view(c * g, n).sum(dim=0).double()
            st["acc_out"][h, cu[r]:cu[r + 1]] = total.float()
        at += nq


def _plain_evict(st):
    case, cu, fill = st["case"], st["cu"], st["fill"]
    hkv = case["hkv"]
    want = st["keep"].tolist()
    keep = torch.zeros(hkv, cu[-1], dtype=torch.bool, device=DEV)
    budget = []
    for r in range(len(cu) - 1):
        for h in range(hkv):
            n = fill[r][h]
            k = min(want[r][h], n)
            recent = min(case["n_recent"], k)
            sink = min(4, k - recent)
            row = keep[h, cu[r]:cu[r] + n]
            row[n - recent:] = True
            row[:sink] = True
            mid = st["acc"][h, cu[r] + sink:cu[r] + n - recent]
            order = torch.sort(mid, descending=True, stable=True).indices[:k - recent - sink]
            row[sink + order] = True
            budget.append(k)
    st["mask"].copy_(_pack_mask(keep, cu, st["mask"].shape[1]))
    st["budget"].copy_(torch.tensor(budget, dtype=torch.int32, device=DEV).view_as(st["budget"]))


def run(state):
    """One pass through the case's operator; its outputs, whole."""
    if own:
        _run_own(state)
    else:
        {"store": _plain_store, "prune": _plain_store, "append": _plain_append, "attend": _plain_attend,
         "accumulate": _plain_accumulate, "evict": _plain_evict}[state["case"]["op"]](state)
    return _results(state)


# ----------------------------------------------------------------------------- the definitions in 64 bits
def _exact_round(y):
    """Nearest e4m3 value, ties to the even code: steps of 2^(exponent - 3), exponent at least -6."""
    mag = y.abs()
    e = torch.floor(torch.log2(mag.clamp_min(2.0 ** -30))).clamp_min(-6.0)
    e = torch.where(mag >= torch.exp2(e + 1), e + 1, e)                     # log2 rounded down past a power of two
    e = torch.where((mag < torch.exp2(e)) & (e > -6), e - 1, e)
    step = torch.exp2(e - 3)
    return torch.round(y / step) * step


def _exact_scale(amax):
    e = -126
    if amax > 0:
        e = max(-126, math.frexp(amax)[1] - 10)
        while amax > E4M3_MAX * 2.0 ** e:
            e += 1
    return 2.0 ** e


def _exact_blocks(rows, codes, scale, a, b):
    """Quantises rows (fp64) block by block into codes[a:], scale[b:]."""
    n = rows.shape[0]
    tops = [float(x) for x in torch.stack([rows[i:i + BLOCK].abs().max() for i in range(0, n, BLOCK)]).cpu()] if n else []
    for j, top in enumerate(tops):
        s = _exact_scale(top)
        scale[b + j] = s
        codes[a + j * BLOCK:a + min(n, (j + 1) * BLOCK)] = _exact_round(rows[j * BLOCK:(j + 1) * BLOCK] / s)


def _values(cache, which, r, h, n):
    """Rows a head holds, in 64 bits."""
    c = cache.codes[which][h, cache.cu[r]:cache.cu[r] + n].view(torch.float8_e4m3fn).double()
    off = cache.cu[r] // BLOCK + r
    block = torch.arange(n, device=DEV) // BLOCK
    return c * cache.scale[which][h].double()[off + block][:, None]


def exact(case, seed):
    st = prepare(case, seed)
    cache, cu, fill, op = st["cache"], st["cu"], st["fill"], case["op"]
    hkv, hq, d = case["hkv"], case["hq"], case["d"]
    g, batch, total = hq // hkv, len(cu) - 1, cu[-1]
    f64 = torch.float64
    if op in ("store", "prune"):
        codes = [torch.zeros(hkv, total, d, dtype=f64, device=DEV) for _ in range(2)]
        scale = [torch.zeros_like(s, dtype=f64) for s in cache.scale]
        kv, acc, pos = st["out"].kv_len.clone(), torch.zeros(hkv, total, dtype=f64, device=DEV), torch.zeros_like(st["pos_out"])
        words = st["mask"].cpu().numpy().view(np.uint32)
        for r in range(batch):
            for h in range(hkv):
                n = np.arange(fill[r][h])
                idx = torch.from_numpy(n[(words[h, cu[r] // 32 + r + n // 32] >> (n % 32)) & 1 == 1]).to(DEV)
                m = idx.numel()
                for w in range(2):
                    rows = (st["K"], st["V"])[w][h, cu[r] + idx].double() if op == "store" else _values(
                        cache, w, r, h, fill[r][h])[idx]
                    _exact_blocks(rows, codes[w][h], scale[w][h], cu[r], cu[r] // BLOCK + r)
                acc[h, cu[r]:cu[r] + m] = st["acc"][h, cu[r] + idx].double()
                pos[h, cu[r]:cu[r] + m] = st["token_pos"][h, cu[r] + idx]
                kv[r, h] = m
        return codes + scale + [kv, acc, pos]
    if op == "append":
        codes = [c.view(torch.float8_e4m3fn).double() for c in cache.codes]
        scale = [s.double() for s in cache.scale]
        kv, acc = cache.kv_len.clone(), st["acc"].double()
        at = np.concatenate([[0], np.cumsum(st["n_new"])])
        for r in range(batch):
            for h in range(hkv):
                n, m = fill[r][h], st["n_new"][r]
                for w in range(2):
                    new = (st["K_new"], st["V_new"])[w][h, at[r]:at[r] + m].double()
                    for first in range(n - n % BLOCK, n + m, BLOCK):
                        have = max(0, n - first)                            # rows of this block already there
                        x = new[max(0, first - n):max(0, first - n) + min(BLOCK, n + m - first) - have]
                        if not x.shape[0]:
                            continue
                        b = cu[r] // BLOCK + r + first // BLOCK
                        s = _exact_scale(float(x.abs().max()))
                        a = cu[r] + first
                        if have:
                            s = max(s, float(scale[w][h, b]))
                            codes[w][h, a:a + have] = _exact_round(codes[w][h, a:a + have] * (float(scale[w][h, b]) / s))
                        codes[w][h, a + have:a + have + x.shape[0]] = _exact_round(x / s)
                        scale[w][h, b] = s
                acc[h, cu[r] + n:cu[r] + n + m] = 0
                kv[r, h] = n + m
        return codes + scale + [kv, acc]
    if op == "attend":
        nq = case["n_q"]
        o = torch.zeros(batch * nq, hq, d, dtype=f64, device=DEV)
        lse = torch.full((batch * nq, hq), -math.inf, dtype=f64, device=DEV)
        acc = torch.zeros(hkv, total, dtype=f64, device=DEV)
        for r in range(batch):
            for h in range(hkv):
                n = fill[r][h]
                if case["acc"]:
                    acc[h, cu[r]:cu[r] + n] = st["acc"][h, cu[r]:cu[r] + n].double()
                k, v = _values(cache, 0, r, h, n), _values(cache, 1, r, h, n)
                for i in range(nq):
                    see = n - (nq - 1 - i)
                    if see <= 0:
                        continue
                    t = r * nq + i
                    logit = st["Q"][t, h * g:(h + 1) * g].double() @ k[:see].T / math.sqrt(d)
                    lse[t, h * g:(h + 1) * g] = torch.logsumexp(logit, dim=1)
                    w = torch.softmax(logit, dim=1)
                    o[t, h * g:(h + 1) * g] = w @ v[:see]
                    acc[h, cu[r]:cu[r] + see] += w.sum(dim=0) if case["acc"] else 0
        return [o, lse] + ([acc] if case["acc"] else [])
    if op == "accumulate":
        acc = torch.zeros(hkv, total, dtype=f64, device=DEV)
        at = 0
        for r in range(batch):
            n, nq = cu[r + 1] - cu[r], st["nq"][r]
            step = max(1, (1 << 26) // max(1, n))
            for head in range(hq):
                k = st["K"][head // g, cu[r]:cu[r + 1]].double()
                for a in range(0, nq, step):
                    c = min(step, nq - a)
                    logit = st["Q"][at + a:at + a + c, head].double() @ k.T / math.sqrt(d)
                    limit = n - nq + 1 + torch.arange(a, a + c, device=DEV)
                    logit[torch.arange(n, device=DEV)[None, :] >= limit[:, None]] = -math.inf
                    acc[head // g, cu[r]:cu[r + 1]] += torch.softmax(logit, dim=1).sum(dim=0)
            at += nq
        return [acc]
    mask = np.zeros(st["mask"].shape, dtype=np.uint32)
    budget = np.zeros((batch, hkv), dtype=np.int32)
    score = st["acc"].cpu().numpy()
    want = st["keep"].cpu().numpy()
    for r in range(batch):
        for h in range(hkv):
            n = fill[r][h]
            k = min(int(want[r, h]), n)
            i = np.arange(n)
            recent = min(case["n_recent"], k)
            sink = min(4, k - recent)
            cls = np.where(i >= n - recent, 0, np.where(i < sink, 1, 2))
            chosen = np.lexsort((i, -score[h, cu[r]:cu[r] + n].astype(np.float64), cls))[:k]
            np.bitwise_or.at(mask[h], cu[r] // 32 + r + chosen // 32, np.uint32(1) << (chosen % 32).astype(np.uint32))
            budget[r, h] = k
    return [torch.from_numpy(mask.view(np.int32)), torch.from_numpy(budget)]
