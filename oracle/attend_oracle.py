"""Attention over cached rows, block tables and slot maps in plain loops and 64 bits: what gvote_attend, gvote_page_attend,
gvote_page_tables and gvote_page_write are held to.  Shares no code with the library."""
import numpy as np

U = 2.0 ** -24                     # half a step of a 32-bit float


def attend(q, k, v, weight_err):
    """q [n, g, d], k, v [rows, d] float64 of one KV head; token i of n sees rows 0 .. rows - n + i.
    Returns out [n, g, d], lse [n, g] and bounds of their errors: `weight_err` is the rounding of a weight on its way into the
    product with the values; a logit is a sum of d products in 32 bits times a rounded factor, its error at most
    (d + 3) U sum|q_i k_i| / sqrt(d); exponentials and sums of them in 32 bits add 2^-18; the output is rounded to bf16."""
    n, g, d = q.shape
    rows = k.shape[0]
    out, lse = np.zeros((n, g, d)), np.full((n, g), -np.inf)
    out_tol, lse_tol = np.zeros((n, g, d)), np.zeros((n, g))
    with np.errstate(all="ignore"):
        for i in range(n):
            seen = rows - n + i + 1
            if seen <= 0:
                continue
            l = (q[i] @ k[:seen].T) / np.sqrt(d)
            top = l.max(axis=1, keepdims=True)
            none = np.isneginf(top)                                   # logits that are all -inf: as if there were no rows
            w = np.exp(l - np.where(none, 0.0, top))
            z = w.sum(axis=1, keepdims=True)
            w = np.where(none, 0.0, w / z)
            lse[i] = (top + np.log(z))[:, 0]
            out[i] = np.where(none, 0.0, _weighted(w, v[:seen]))
            size = np.where(np.isneginf(l), 0.0, (np.abs(q[i]) @ np.abs(k[:seen]).T) / np.sqrt(d))
            dl = np.nan_to_num((d + 3) * U * size.max(axis=1, keepdims=True), posinf=0.0) + 2.0 ** -18
            spread = _weighted(w, np.abs(np.where(np.isfinite(v[:seen]), v[:seen], 0.0)))
            out_tol[i] = 2.0 ** -8 * np.abs(out[i]) + spread * (weight_err + 2 * dl) * 1.01 + 1e-30
            lse_tol[i] = dl[:, 0] + 4 * U * np.abs(lse[i])
    return out, lse, out_tol, lse_tol


def _weighted(w, v):
    """w @ v; a value that is not finite counts whatever its row's weight, zero (a logit of -inf) among them."""
    if np.isfinite(v).all():
        return w @ v
    o = w @ np.where(np.isfinite(v), v, 0.0)
    for j, c in zip(*np.nonzero(~np.isfinite(v))):
        o[:, c] += v[j, c]
    return o


def tables(tabs, kv_len, free, n_free, page_rows, keep=None, cu_new=None, kept=None):
    """kept: bool [hkv, total_new] or None for all.  Returns the new (tables, kv_len, free, n_free, slots), or None where the
    call has to refuse."""
    tabs, kv_len, free = tabs.copy(), kv_len.copy(), free.copy()
    B, H, M = tabs.shape
    P = page_rows
    total = 0 if cu_new is None else int(cu_new[-1])
    slots = np.full((H, total), -1, np.int32)
    pages = lambda x: -(-x // P)
    held = np.clip(kv_len, 0, M * P)
    cut = held if keep is None else np.minimum(held, np.maximum(keep, 0))
    gone = [tabs[r, h, j] for r in range(B) for h in range(H) for j in range(pages(cut[r, h]), pages(held[r, h]))]
    rows = {}
    for r in range(B):
        for h in range(H):
            if cu_new is None:
                rows[r, h] = []
            else:
                rows[r, h] = [t for t in range(cu_new[r], cu_new[r + 1]) if kept is None or kept[h, t]]
    if any(cut[r, h] + len(x) > M * P for (r, h), x in rows.items()):
        return None
    need = sum(pages(cut[r, h] + len(x)) - pages(cut[r, h]) for (r, h), x in rows.items())
    top = int(n_free) + len(gone)
    if not 0 <= n_free <= len(free) or top > len(free) or need > top:
        return None
    moved = gone + free[top - max(need, len(gone)):int(n_free)].tolist()
    if any(not 0 <= page < len(free) for page in moved):
        return None
    for i, page in enumerate(gone):
        free[top - 1 - i] = page
    for r in range(B):
        for h in range(H):
            new = cut[r, h] + len(rows[r, h])
            for j in range(pages(cut[r, h]), pages(new)):
                top -= 1
                tabs[r, h, j] = free[top]
            for i, t in enumerate(rows[r, h]):
                at = cut[r, h] + i
                slots[h, t] = tabs[r, h, at // P] * P + at % P
            kv_len[r, h] = new
    return tabs, kv_len, free, np.int32(top), slots
