"""Cases of the attention over bf16 rows: what a user holds, with everything that must not be read poisoned."""
import numpy as np
import torch

from oracle import attend_oracle as ao


def cu_of(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def dev(x):
    return torch.tensor(np.asarray(x), device="cuda")


def params(gv, hq, hkv, d):
    return gv.make_params(d_h=64, n_q_heads=hq, n_kv_heads=hkv, d_k=d, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1, n_s=4, seed=0)


def poison(shape, seed):
    """bf16 values that must not be read: NaN, infinities, the lowest value."""
    g = torch.Generator().manual_seed(seed)
    pick = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(torch.bfloat16).min]).bfloat16()
    return pick[torch.randint(0, 4, shape, generator=g)]


class Case:
    """rows[r][h] cached rows, nq[r] query tokens; K, V [r][h] lists of bf16 arrays [rows, d]."""

    def __init__(self, hq, hkv, d, rows, nq, seed=0, scale=1.5, outliers=True, lead=0, trail=0):
        g = torch.Generator().manual_seed(seed)
        self.hq, self.hkv, self.d, self.rows, self.nq = hq, hkv, d, rows, nq
        self.lead, self.trail, self.seed = lead, trail, seed
        boost = torch.ones(d)
        if outliers:
            boost[torch.randperm(d, generator=g)[:4]] = 6.0
        self.K = [[(torch.randn(n, d, generator=g) * boost).bfloat16() for n in rr] for rr in rows]
        self.V = [[torch.randn(n, d, generator=g).bfloat16() for n in rr] for rr in rows]
        self.Q = (torch.randn(lead + sum(nq) + trail, hq, d, generator=g) * scale).bfloat16()
        self.cu_q = cu_of(nq) + lead

    def geom(self):
        return len(self.nq), self.Q.shape[0], max(max(self.nq), 1)

    def oracle(self, weight_err):
        n = self.Q.shape[0]
        res = [np.full((n, self.hq, self.d), np.nan), np.full((n, self.hq), np.nan), np.zeros((n, self.hq, self.d)), np.zeros((n, self.hq))]
        g = self.hq // self.hkv
        q = self.Q.double().numpy()
        for r, c in enumerate(self.nq):
            a = self.cu_q[r]
            for h in range(self.hkv):
                got = ao.attend(q[a:a + c, h * g:(h + 1) * g], self.K[r][h].double().numpy(), self.V[r][h].double().numpy(), weight_err)
                for x, y in zip(res, got):
                    x[a:a + c, h * g:(h + 1) * g] = y
        return res

    def outputs(self, head_pad=0):
        """out and lse full of a mark; out with room between its rows."""
        n = self.Q.shape[0]
        wide = torch.full((n, self.hq, self.d + head_pad), 7.0, dtype=torch.bfloat16, device="cuda")
        return wide, wide[:, :, :self.d], torch.full((n, self.hq), 7.0, device="cuda")

    def check(self, wide, out, lse, weight_err, lse_given=True):
        want, want_lse, tol, tol_lse = self.oracle(weight_err)
        a, b = int(self.cu_q[0]), int(self.cu_q[-1])
        o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
        assert np.all(o[:a] == 7) and np.all(o[b:] == 7) and np.all(l[:a] == 7) and np.all(l[b:] == 7)
        assert bool((wide[:, :, self.d:] == 7).all())
        compare(o[a:b], want[a:b], tol[a:b], "out")
        if lse_given:
            compare(l[a:b], want_lse[a:b], tol_lse[a:b], "lse")

    # ------------------------------------------------------------------ pages
    def pages(self, gv, page_rows, spare=3, split=False, extra=0):
        """A PageCache of these rows: pages in disorder, everything else poisoned."""
        B, H, d = len(self.rows), self.hkv, self.d
        need = [[-(-n // page_rows) for n in rr] for rr in self.rows]
        n_pages = sum(map(sum, need)) + spare
        g = torch.Generator().manual_seed(self.seed + 1)
        order = torch.randperm(n_pages, generator=g).tolist()
        shape = (n_pages, 2, page_rows, d + 8) if split else (2, n_pages, page_rows, d)
        mem = poison(shape, self.seed + 2)
        K, V = (mem[:, 0, :, :d], mem[:, 1, :, :d]) if split else (mem[0], mem[1])
        most = max(1, max(map(max, need))) + extra
        tab = torch.full((B, H, most), 0x7fffffff, dtype=torch.int32)      # entries behind the last page are not read
        at = 0
        for r in range(B):
            for h in range(H):
                for j in range(need[r][h]):
                    page, n = order[at], min(page_rows, self.rows[r][h] - j * page_rows)
                    at += 1
                    tab[r, h, j] = page
                    K[page, :n] = self.K[r][h][j * page_rows:j * page_rows + n]
                    V[page, :n] = self.V[r][h][j * page_rows:j * page_rows + n]
        m = mem.cuda()
        K, V = (m[:, 0, :, :d], m[:, 1, :, :d]) if split else (m[0], m[1])
        free = torch.zeros(n_pages, dtype=torch.int32)
        free[:spare] = torch.tensor(order[at:], dtype=torch.int32)
        return gv.PageCache(K, V, tab.cuda(), torch.tensor(self.rows, dtype=torch.int32, device="cuda").view(B, H), free.cuda(),
                            torch.tensor([spare], dtype=torch.int32, device="cuda"))

    # ------------------------------------------------------------------ slabs
    def slabs(self, room=5, tokens_outer=False, width=0):
        """K, V, cu, kv_len, geom: slabs with poisoned room behind each head's rows."""
        lens = [max(rr) + room for rr in self.rows]
        cu = cu_of(lens)
        total, d = int(cu[-1]), self.d
        mem = poison((2, total, self.hkv, d + width) if tokens_outer else (2, self.hkv, total, d + width), self.seed + 3)
        view = lambda m: (m.transpose(1, 2) if tokens_outer else m)[..., :d]
        x = view(mem)
        for r, rr in enumerate(self.rows):
            for h, n in enumerate(rr):
                x[0, h, cu[r]:cu[r] + n] = self.K[r][h]
                x[1, h, cu[r]:cu[r] + n] = self.V[r][h]
        y = view(mem.cuda())
        return y[0], y[1], dev(cu), torch.tensor(self.rows, dtype=torch.int32, device="cuda").view(len(lens), self.hkv), (len(lens), total, max(lens))


def compare(got, want, tol, what):
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), f"{what}: infinities differ"
    off = np.abs(got[fine] - want[fine])
    bad = off > tol[fine]
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, the worst {np.max(off / np.maximum(tol[fine], 1e-300)):.3g} times its tolerance"
