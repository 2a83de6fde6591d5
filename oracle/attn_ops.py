"""Plain fp64 forms of the full-attention layer's operators and of linear attention
(torch, any device): what the GPU calls are compared with.  Where sums are formed,
the same sums over magnitudes come with them, against which an error bound is
stated element by element."""
from __future__ import annotations

import torch

MOST = 2 ** 31 - 1


def extend_pages(table, lens, cu, free, page_size, first=0, taken=0):
    """Lists in, lists out: table, lens, taken, slots, positions."""
    table, out_lens, slots, positions = [list(r) for r in table], [], [], []
    taken = max(taken, 0)
    for n, row in enumerate(table):
        held, q = max(lens[n], 0), cu[n + 1] - cu[n]
        total = min(held + q, MOST)
        for c in range(min(-(-held // page_size), len(row)), min(-(-total // page_size), len(row))):
            row[c] = free[taken] if taken < len(free) else -1
            taken += 1
        for i in range(held, held + q):
            page = row[i // page_size] if i // page_size < len(row) else -1
            slot = page * page_size + i % page_size
            slots.append(slot if page >= 0 and slot <= MOST else -1)
            positions.append(min(first + i, MOST))
        out_lens.append(total)
    return table, out_lens, taken, slots, positions


def qk_rows(x, positions, cos_sin, weight=None, eps=1e-6, interleaved=False):
    """Normed and rotated rows of x [T, H, D] and the magnitudes of their sums."""
    x, R = x.double(), cos_sin.shape[1]
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    cs = cos_sin.double()[positions.long()]
    y, mag = x.clone(), x.abs()
    for p in range(R // 2):
        a, b = (2 * p, 2 * p + 1) if interleaved else (p, p + R // 2)
        c, s = cs[:, None, p], cs[:, None, R // 2 + p]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        mag[..., a] = (x[..., a] * c).abs() + (x[..., b] * s).abs()
        mag[..., b] = (x[..., b] * c).abs() + (x[..., a] * s).abs()
    return y, mag


def attention(q, k_cache, v_cache, table, lens, cu, prefix_pages=None, prefix_len=0, scale=None, max_len=None):
    """out [T, Hq, D]; sum w |v| / sum w; per query and head the largest |scale| sum |q k| and the range of the
    scores; the keys that it sees.  Pages outside the cache hold nothing."""
    T, H, D = q.shape
    pages, ps, Hk = k_cache.shape[:3]
    scale = D ** -0.5 if scale is None else scale
    dev = q.device
    out = torch.zeros(T, H, D, dtype=torch.float64, device=dev)
    mag = torch.zeros_like(out)
    size = torch.zeros(T, H, dtype=torch.float64, device=dev)
    spread = torch.zeros_like(size)
    count = torch.zeros(T, dtype=torch.int64, device=dev)
    room = table.shape[1] * ps if max_len is None else max_len

    def rows(list_, n):
        at = torch.arange(n, device=dev)
        page = list_.long()[at // ps] if n else at
        return torch.where((page >= 0) & (page < pages), page * ps + at % ps, -1)
    flat = lambda c: c.reshape(pages * ps, Hk, D)
    kf, vf = flat(k_cache), flat(v_cache)
    for s in range(len(cu) - 1):
        L = cu[s + 1] - cu[s]
        m = min(max(int(lens[s]), 0), room)
        at = torch.cat([rows(prefix_pages, prefix_len) if prefix_len else torch.empty(0, dtype=torch.int64, device=dev),
                        rows(table[s], m)])
        there = at >= 0
        own = torch.arange(len(at), device=dev) - prefix_len
        for i in range(L):
            t = cu[s] + i
            see = there & (own <= max(m - L + i, -1))   # (the prefix is below 0: seen by all)
            r = at[see]
            count[t] = len(r)
            if len(r) == 0:
                continue
            k = kf[r].double().repeat_interleave(H // Hk, 1)
            v = vf[r].double().repeat_interleave(H // Hk, 1)
            x = (q[t].double() * k).sum(-1) * scale                # [keys, H]
            size[t] = (q[t].double() * k).abs().sum(-1).amax(0) * abs(scale)
            spread[t] = x.amax(0) - x.amin(0)
            w = torch.softmax(x, 0)
            out[t], mag[t] = (w[..., None] * v).sum(0), (w[..., None] * v.abs()).sum(0)
    return out, mag, size, spread, count


def linear(q, k, v, g, cu, scale=1.0, state=None):
    """o [T, Hv, d_v], states [N, Hv, d_k, d_v], and the magnitudes of both."""
    k, v = k.double(), v.double()
    T, H, V = v.shape
    Hk, K = k.shape[1:]
    n = len(cu) - 1
    alpha = torch.exp(g.double())[:, None, None]
    grp = torch.arange(H, device=v.device) // (H // Hk)
    o, omag = torch.zeros_like(v), torch.zeros_like(v)
    st = torch.zeros(n, H, K, V, dtype=torch.float64, device=v.device) if state is None else state.double().clone()
    mag = st.abs()
    for s in range(n):
        m, mm = st[s], mag[s]
        for t in range(cu[s], cu[s + 1]):
            add = k[t, grp][:, :, None] * v[t][:, None, :]
            m, mm = alpha * m + add, alpha * mm + add.abs()
            if q is not None:
                x = q[t].double()[grp][:, :, None]
                o[t], omag[t] = (x * m).sum(1) * scale, (x.abs() * mm).sum(1) * abs(scale)
        st[s], mag[s] = m, mm
    return o, st, omag, mag
