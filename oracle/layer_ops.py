"""Plain fp64 forms of the recurrent layer's operators, token by token (torch,
any device): what the GPU calls are compared with.  Each also returns the same
sums over magnitudes, against which an error bound is stated element by
element: an operator that adds n products in fp32 is off by at most about
n * 2^-24 times them."""
from __future__ import annotations

import torch


def causal_conv(x, w, cu, bias=None, history=None, silu=True):
    """y [T, C], the histories after each sequence, and sum |w x| + |bias|."""
    x, w = x.double(), w.double()
    C, W = w.shape
    n = len(cu) - 1
    y, mag = torch.zeros_like(x), torch.zeros_like(x)
    before = torch.zeros(n, W - 1, C, dtype=torch.float64, device=x.device) if history is None else history.double()
    after = torch.empty_like(before)
    for s in range(n):
        rows = torch.cat([before[s], x[cu[s]:cu[s + 1]]])
        L = cu[s + 1] - cu[s]
        acc = torch.zeros(L, C, dtype=torch.float64, device=x.device)
        m = torch.zeros_like(acc)
        for j in range(W):
            acc = acc + rows[j:j + L] * w[:, j]
            m = m + (rows[j:j + L] * w[:, j]).abs()
        if bias is not None:
            acc, m = acc + bias.double(), m + bias.double().abs()
        y[cu[s]:cu[s + 1]] = acc * torch.sigmoid(acc) if silu else acc
        mag[cu[s]:cu[s + 1]] = m
        after[s] = rows[L:]
    return y, after, mag


def ssm(x, dt, a_log, B, C, cu, d_skip=None, dt_bias=None, state=None):
    """y [T, H, P], states [n, H, N, P], and the magnitudes of both."""
    x, B, C = x.double(), B.double(), C.double()
    T, H, P = x.shape
    G, N = B.shape[1:]
    n = len(cu) - 1
    z = dt.double() + (0.0 if dt_bias is None else dt_bias.double())
    delta = torch.logaddexp(z, torch.zeros_like(z))
    alpha = torch.exp(-torch.exp(a_log.double()) * delta)
    grp = torch.arange(H, device=x.device) // (H // G)
    y, ymag = torch.zeros_like(x), torch.zeros_like(x)
    st = torch.zeros(n, H, N, P, dtype=torch.float64, device=x.device) if state is None else state.double().clone()
    mag = st.abs()
    for s in range(n):
        m, mm = st[s], mag[s]
        for t in range(cu[s], cu[s + 1]):
            add = B[t, grp][:, :, None] * (delta[t][:, None] * x[t])[:, None, :]
            m = alpha[t][:, None, None] * m + add
            mm = alpha[t][:, None, None] * mm + add.abs()
            y[t] = (C[t, grp][:, :, None] * m).sum(1)
            ymag[t] = (C[t, grp][:, :, None].abs() * mm).sum(1)
        st[s], mag[s] = m, mm
    if d_skip is not None:
        y = y + d_skip.double()[:, None] * x
        ymag = ymag + (d_skip.double()[:, None] * x).abs()
    return y, st, ymag, mag


def lora(base, x, a, b, adapters, cu, scales=None):
    """out [T, M] and |base| + |scale| |x| |A|^T |B|^T."""
    out, mag = base.double().clone(), base.double().abs()
    for s, i in enumerate(adapters):
        rows = slice(cu[s], cu[s + 1])
        if i < 0 or cu[s] == cu[s + 1]:
            continue
        k = 1.0 if scales is None else float(scales[i])
        out[rows] += k * (x[rows].double() @ a[i].double().t()) @ b[i].double().t()
        mag[rows] += abs(k) * (x[rows].double().abs() @ a[i].double().abs().t()) @ b[i].double().abs().t()
    return out, mag
