"""The operators around a recurrent layer's state, as measurable cases: the short causal convolution, the selective
state space scan, both for prompts and for single tokens, and low-rank adapters beside a shared projection.

Where `own` is false each operator is computed in its plain form, from elementary torch operations in 32 bits; where it
is true, by the package's public calls.  Inputs are laid out as a layer has them: the convolution reads columns of the
in-projection's rows, the scan reads x, B and C as columns of the convolution's rows and dt as columns of the
in-projection's.
"""
import math
import random

import torch

DEVICE = "cuda:0"
own = False

# the package's hybrid layer (16 key and 32 value heads of 128: 8192 convolved of 12352 projected columns)
LAYER = dict(chans=8192, ld=12352, taps=4, dtype="bf16")
# a state space layer of 64 heads of 64 with 128 state rows, B and C shared by all heads
SSM = dict(heads=64, groups=1, dstate=128, headdim=64, dtype="bf16")
# the same width in the package's head layout: 16 B/C groups, 32 heads of 128
SSM_WIDE = dict(heads=32, groups=16, dstate=128, headdim=128, dtype="bf16")
SSM_SMALL = dict(heads=4, groups=2, dstate=64, headdim=64, dtype="f32")
LORA = dict(hidden=2048, width=12352, dtype="bf16")


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # the convolution over a prompt of the hybrid layer
        dict(LAYER, name="conv_prompt_8k", kind="conv", n=1, lo=8192, hi=8192, lens=0, history=False, bias=False),
        # seven ragged continuations of a small fp32 layer, each from the inputs before it; odd channel count
        dict(name="conv_ragged_f32", kind="conv", chans=771, ld=771, taps=4, dtype="f32", n=7, lo=1, hi=700, lens=5,
             history=True, bias=True),
        # one token of one conversation: the smallest call, all latency
        dict(LAYER, name="conv_step_1", kind="conv_step", n=1, bias=False),
        # one token for every conversation of a serving batch
        dict(LAYER, name="conv_step_256", kind="conv_step", n=256, bias=True),
        # the state rebuilt from 10 % of 8192 matched tokens, one conversation
        dict(SSM, name="scan_819", kind="scan", n=1, lo=819, hi=819, lens=0, state=False),
        # the longest prompt that the package's benchmark knows
        dict(SSM, name="scan_32k", kind="scan", n=1, lo=32768, hi=32768, lens=0, state=False),
        # 16 concurrent suffixes, each from its own state, in the package's head layout
        dict(SSM_WIDE, name="scan_16_ragged", kind="scan", n=16, lo=128, hi=2048, lens=3, state=True),
        # a small fp32 layer: 2048 tokens
        dict(SSM_SMALL, name="scan_small_f32", kind="scan", n=1, lo=2048, hi=2048, lens=0, state=True),
        # one token of one conversation
        dict(SSM, name="step_1", kind="step", n=1),
        # one token for every conversation of a serving batch
        dict(SSM, name="step_128", kind="step", n=128),
        # one token for each of 64 conversations with 32 adapters beside the in-projection
        dict(LORA, name="lora_decode_64", kind="lora", n=64, lo=1, hi=1, lens=0, rank=16, adapters=32),
        # the tails of 8 requests replayed in one call, each with an adapter of its own or none
        dict(LORA, name="lora_tails_8", kind="lora", n=8, lo=200, hi=819, lens=2, rank=64, adapters=6),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["conv", "conv_step", "scan", "scan", "scan", "step", "lora", "lora"])
    lens = rng.randrange(1 << 20)
    if kind == "conv":
        chans = rng.choice([_log_int(rng, 16, 8192), 8 * _log_int(rng, 2, 1024)])
        n = _log_int(rng, 1, 32)
        hi = _log_int(rng, 1, max(1, 16384 // n))
        return dict(kind="conv", chans=chans, ld=chans + rng.choice([0, 0, 8, 72, 5]), taps=rng.choice([4, 4, 3, 2]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), n=n, lo=rng.choice([0, 1, hi]) if n > 1 else hi, hi=hi,
                    lens=lens, history=rng.random() < 0.5, bias=rng.random() < 0.5)
    if kind == "conv_step":
        chans = rng.choice([_log_int(rng, 16, 8192), 8 * _log_int(rng, 2, 1024)])
        return dict(kind="conv_step", chans=chans, ld=chans + rng.choice([0, 8, 72, 5]), taps=rng.choice([4, 4, 3, 2]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), n=_log_int(rng, 1, 256), bias=rng.random() < 0.5)
    if kind in ("scan", "step"):
        heads = rng.choice([SSM, SSM, SSM_WIDE, SSM_SMALL, dict(SSM, groups=8), dict(SSM, dstate=64),
                            dict(SSM, heads=24, groups=3), dict(SSM_WIDE, dstate=64),
                            dict(SSM_SMALL, heads=7, groups=1), dict(SSM_WIDE, heads=16, groups=2, dtype="f32")])
        if kind == "step":
            return dict(heads, kind="step", n=_log_int(rng, 1, 128))
        n = rng.choice([1, 1, 2, 5, _log_int(rng, 2, 64)])
        hi = _log_int(rng, 16, (8192 if heads["dtype"] == "f32" else 32768) // n)
        return dict(heads, kind="scan", n=n, lo=rng.choice([0, 1, hi]) if n > 1 else hi, hi=hi, lens=lens,
                    state=rng.random() < 0.5)
    n = _log_int(rng, 1, 64)
    hi = 1 if rng.random() < 0.4 else _log_int(rng, 1, max(1, 4096 // n))
    return dict(kind="lora", hidden=8 * _log_int(rng, 16, 512), width=rng.choice([8, 1]) * _log_int(rng, 64, 1544),
                dtype=rng.choice(["bf16", "bf16", "f32"]), n=n, lo=rng.choice([0, 1, hi]) if n > 1 else hi, hi=hi,
                lens=lens, rank=rng.choice([8, 16, 16, 32, 40, 64, 128]), adapters=_log_int(rng, 1, 32))


def _lengths(case):
    """The lengths of a batch's sequences: `n` of them between the two bounds, by the case alone."""
    rng = random.Random("%d" % case["lens"])
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["n"])]
    lens[-1] = case["hi"]
    return lens


def _sizes(case):
    """(rows of tokens, sequences)."""
    return (case["n"] if "lo" not in case else sum(_lengths(case))), case["n"]


# ------------------------------------------------------------------ inputs
def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _offsets(lens):
    cu = torch.zeros(len(lens) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor(lens, dtype=torch.int64), 0).to(torch.int32)
    return cu.to(DEVICE), cu


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    rn = lambda *s: torch.randn(*s, device=DEVICE, generator=gen)
    ru = lambda *s: torch.rand(*s, device=DEVICE, generator=gen)
    kind, dt, n = case["kind"], _dt(case), case["n"]
    st = dict(case=case)
    if "lo" in case:
        st["cu"], st["cu_host"] = _offsets(_lengths(case))
    T = _sizes(case)[0]
    if kind in ("conv", "conv_step"):
        C, W = case["chans"], case["taps"]
        st.update(x=rn(T, case["ld"]).to(dt)[:, :C], w=ru(C, W) - 0.5, bias=0.1 * rn(C) if case["bias"] else None,
                  y=torch.empty(T, C, dtype=dt, device=DEVICE))
        st["history"] = rn(n, W - 1, C).to(dt) if kind == "conv_step" or case["history"] else None
        st["history_out"] = torch.empty(n, W - 1, C, dtype=dt, device=DEVICE)
    elif kind in ("scan", "step"):
        H, G, N, P = (case[k] for k in ("heads", "groups", "dstate", "headdim"))
        # x, B and C as the convolution leaves them (after SiLU), dt as columns of the projection's rows
        xbc = torch.nn.functional.silu(rn(T, H * P + 2 * G * N)).to(dt)
        step = torch.exp(math.log(1e-3) + ru(H) * math.log(100.0))   # time steps of 0.001 to 0.1 where dt is zero
        st.update(x=xbc[:, :H * P].unflatten(1, (H, P)), B=xbc[:, H * P:H * P + G * N].unflatten(1, (G, N)),
                  C=xbc[:, H * P + G * N:].unflatten(1, (G, N)), dt=rn(T, H + 8).to(dt)[:, 8:],
                  a_log=torch.log(1 + 15 * ru(H)), d=0.5 + ru(H), dt_bias=step + torch.log(-torch.expm1(-step)),
                  y=torch.empty(T, H, P, dtype=dt, device=DEVICE),
                  state=rn(n, H, N, P) * 0.5 if kind == "step" or case["state"] else None,
                  state_out=torch.empty(n, H, N, P, dtype=torch.float32, device=DEVICE))
    else:
        K, M, R, A = case["hidden"], case["width"], case["rank"], case["adapters"]
        ids = torch.randint(-1, A, (n,), generator=torch.Generator().manual_seed(case["lens"] + 1), dtype=torch.int32)
        st.update(x=rn(T, K).to(torch.bfloat16), a=(rn(A, R, K) / K ** 0.5).to(torch.bfloat16),
                  b=(rn(A, M, R) / R ** 0.5).to(torch.bfloat16), scales=0.25 + ru(A), base=rn(T, M).to(dt),
                  ids=ids.to(DEVICE), ids_host=ids, out=torch.empty(T, M, dtype=dt, device=DEVICE))
    return st


# ------------------------------------------------------------------ the calls
def run(st):
    kind = st["case"]["kind"]
    if own:
        import paper_2608_30310_amd as gdn
        if kind == "conv":
            y, h = gdn.causal_conv(st["x"], st["w"], st["cu"], st["cu_host"], bias=st["bias"],
                                   history_in=st["history"], activation="silu", out=st["y"],
                                   history_out=st["history_out"])
            return dict(y=y, history=h)
        if kind == "conv_step":
            y, h = gdn.causal_conv_step(st["x"], st["w"], st["history"], bias=st["bias"], activation="silu",
                                        out=st["y"], history_out=st["history_out"])
            return dict(y=y, history=h)
        if kind == "scan":
            y, s = gdn.ssm_scan(st["x"], st["dt"], st["a_log"], st["B"], st["C"], st["cu"], st["cu_host"],
                                d_skip=st["d"], dt_bias=st["dt_bias"], state_in=st["state"], out=st["y"],
                                state_out=st["state_out"])
            return dict(y=y, state=s)
        if kind == "step":
            y, s = gdn.ssm_step(st["x"], st["dt"], st["a_log"], st["B"], st["C"], d_skip=st["d"],
                                dt_bias=st["dt_bias"], state_in=st["state"], out=st["y"], state_out=st["state_out"])
            return dict(y=y, state=s)
        return dict(out=gdn.lora_add(st["base"], st["x"], st["a"], st["b"], st["ids"], st["cu"], st["cu_host"],
                                     adapters_host=st["ids_host"], scales=st["scales"], out=st["out"]))
    if kind == "conv":
        return _plain_conv(st)
    if kind == "conv_step":
        return _plain_conv_step(st)
    if kind == "scan":
        return _plain_scan(st)
    if kind == "step":
        return _plain_step(st)
    return _plain_lora(st)


def _silu(x):
    return x / (1.0 + torch.exp(-x))


def _softplus(x):
    """log(1 + e^x), in 64 bits (its sums over many tokens go into exponents), without overflow."""
    x = x.double()
    return torch.clamp(x, min=0.0) + torch.log1p(torch.exp(-x.abs()))


def _plain_conv(st):
    case = st["case"]
    W, C, n = case["taps"], case["chans"], case["n"]
    x, cu = st["x"].float(), st["cu"].long()
    T = x.shape[0]
    hist = torch.zeros(n, W - 1, C, device=x.device) if st["history"] is None else st["history"].float()
    # every sequence's rows behind its history: row t of sequence s stands at t + (W - 1)(s + 1)
    seq = torch.searchsorted(cu[1:], torch.arange(T, device=x.device), right=True)
    at = torch.arange(T, device=x.device) + (W - 1) * (seq + 1)
    head = cu[:-1, None] + (W - 1) * torch.arange(n, device=x.device)[:, None] + torch.arange(W - 1, device=x.device)
    rows = torch.empty(T + n * (W - 1), C, device=x.device)
    rows[at] = x
    rows[head.reshape(-1)] = hist.reshape(-1, C)
    taps = torch.stack([at - (W - 1) + j for j in range(W)])                     # [W, T]
    acc = (rows[taps] * st["w"].t()[:, None, :]).sum(0)
    if st["bias"] is not None:
        acc = acc + st["bias"]
    last = cu[1:, None] + (W - 1) * torch.arange(n, device=x.device)[:, None] + torch.arange(W - 1, device=x.device)
    dt = st["y"].dtype
    return dict(y=_silu(acc).to(dt), history=rows[last.reshape(-1)].view(n, W - 1, C).to(dt))


def _plain_conv_step(st):
    rows = torch.cat([st["history"].float(), st["x"].float()[:, None]], 1)       # [n, W, C]
    acc = (rows * st["w"].t()).sum(1)
    if st["bias"] is not None:
        acc = acc + st["bias"]
    dt = st["y"].dtype
    return dict(y=_silu(acc).to(dt), history=rows[:, 1:].to(dt))


def _plain_scan(st):
    """Chunks of 64 tokens, all at once: products inside the chunks, then every chunk's start as the sum of the chunks
    before it in its sequence, each by its decay."""
    case = st["case"]
    H, G, N, P, n, Q = case["heads"], case["groups"], case["dstate"], case["headdim"], case["n"], 64
    dev = st["x"].device
    lens = st["cu_host"][1:].long() - st["cu_host"][:-1].long()
    per = (lens + Q - 1) // Q
    nc = int(per.sum())
    seq = torch.repeat_interleave(torch.arange(n), per)                          # [nc]: each chunk's sequence
    first = torch.cumsum(per, 0) - per
    start = (torch.arange(nc) - first[seq]) * Q
    off = start[:, None] + torch.arange(Q)                                       # [nc, Q]
    there = off < lens[seq][:, None]
    spots = there.reshape(-1).nonzero()[:, 0].to(dev)                            # the places that hold a token, in order
    tok = torch.where(there, st["cu_host"].long()[seq][:, None] + off, 0).to(dev)
    seq, there, lens = seq.to(dev), there.to(dev), lens.to(dev)
    take = lambda t: torch.where(there[..., None, None], t.float()[tok], 0.0).transpose(1, 2)   # [nc, heads, Q, d]
    x = take(st["x"])
    B, C = (take(st[k])[:, :, None].expand(nc, G, H // G, Q, N).reshape(nc, H, Q, N) for k in ("B", "C"))
    delta = torch.where(there[..., None], _softplus(st["dt"].float()[tok] + st["dt_bias"]), 0.0).transpose(1, 2)
    cum = torch.cumsum(-torch.exp(st["a_log"].double())[:, None] * delta, -1)    # [nc, H, Q], 64 bits
    delta = delta.float()
    lower = torch.ones(Q, Q, dtype=torch.bool, device=dev).tril()
    L = torch.exp(torch.where(lower, cum[..., :, None] - cum[..., None, :], -math.inf)).float()
    P_ = (C @ B.transpose(-1, -2)) * L * delta[..., None, :]
    w = torch.exp(cum[..., -1:] - cum).float() * delta
    own_state = (B * w[..., None]).transpose(-1, -2) @ x                         # [nc, H, N, P]
    # start of chunk c: sum over the chunks e < c of its sequence, decayed over the chunks between, and the first state
    total = cum[..., -1]                                                         # [nc, H]
    run_ = torch.cumsum(total, 0)
    same = seq[:, None] == seq[None, :]
    before = same & (torch.arange(nc, device=dev)[:, None] > torch.arange(nc, device=dev)[None, :])
    decay = torch.exp(torch.where(before[..., None], (run_ - total)[:, None] - run_[None, :], -math.inf)).float()
    flat = own_state.transpose(0, 1).reshape(H, nc, N * P)
    begin = (decay.permute(2, 0, 1) @ flat).view(H, nc, N, P).transpose(0, 1)
    state = torch.zeros(n, H, N, P, device=dev) if st["state"] is None else st["state"]
    if nc:
        base = run_ - total                                                      # decays before each chunk, all sequences
        f = first.to(dev).clamp(max=nc - 1)
        since = torch.exp(base - base[f[seq]]).float()
        begin = begin + since[..., None, None] * state[seq]
        end = torch.exp(total).float()[..., None, None] * begin + own_state
        last = (first.to(dev) + per.to(dev) - 1).clamp(min=0)
        state = torch.where((lens > 0)[:, None, None, None], end[last], state)
    y = P_ @ x + torch.exp(cum).float()[..., None] * (C @ begin) + st["d"][:, None, None] * x
    y = y.transpose(1, 2).reshape(nc * Q, H, P)[spots]                           # chunks follow the packed order
    return dict(y=y.to(st["y"].dtype), state=state)


def _plain_step(st):
    case = st["case"]
    per = case["heads"] // case["groups"]
    delta = _softplus(st["dt"].float() + st["dt_bias"]).float()                  # [n, H]
    alpha = torch.exp(-torch.exp(st["a_log"]) * delta)
    x = st["x"].float()
    B, C = (st[k].float().repeat_interleave(per, 1) for k in ("B", "C"))
    state = alpha[..., None, None] * st["state"] + B[..., None] * (delta[..., None] * x)[..., None, :]
    y = (C[..., None] * state).sum(2) + st["d"][:, None] * x
    return dict(y=y.to(st["y"].dtype), state=state)


def _plain_lora(st):
    """The sequences padded to the longest, one batched product each way."""
    cu = st["cu_host"].long()
    lens = cu[1:] - cu[:-1]
    off = torch.arange(int(lens.max()))
    there = (off < lens[:, None]) & (st["ids_host"] >= 0)[:, None]
    tok = torch.where(there, cu[:-1, None] + off, 0)
    spots = there.reshape(-1).nonzero()[:, 0]
    rows, spots, tok = tok.reshape(-1)[spots].to(DEVICE), spots.to(DEVICE), tok.to(DEVICE)
    ids = st["ids"].long().clamp(min=0)
    u = st["x"].float()[tok] @ st["a"].float()[ids].transpose(1, 2)              # [n, longest, R]
    add = (u * st["scales"][ids][:, None, None]) @ st["b"].float()[ids].transpose(1, 2)
    out = st["base"].float()
    out[rows] += add.reshape(-1, add.shape[-1])[spots]
    return dict(out=out.to(st["out"].dtype))


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("conv", "conv_step"):
        W, C, n = case["taps"], case["chans"], case["n"]
        x, w = st["x"].double(), st["w"].double()
        cuts = st["cu_host"].tolist() if kind == "conv" else list(range(n + 1))
        y = torch.empty(x.shape[0], C, dtype=torch.float64, device=DEVICE)
        hist = torch.zeros(n, W - 1, C, dtype=torch.float64, device=DEVICE)
        if st["history"] is not None:
            hist = st["history"].double()
        after = torch.empty_like(hist)
        for s in range(n):
            rows = torch.cat([hist[s], x[cuts[s]:cuts[s + 1]]])
            L = cuts[s + 1] - cuts[s]
            acc = torch.zeros(L, C, dtype=torch.float64, device=DEVICE)
            for j in range(W):
                acc += rows[j:j + L] * w[:, j]
            if st["bias"] is not None:
                acc += st["bias"].double()
            y[cuts[s]:cuts[s + 1]] = acc * torch.sigmoid(acc)
            after[s] = rows[L:]
        return dict(y=y, history=after)
    if kind in ("scan", "step"):
        H, G, n = case["heads"], case["groups"], case["n"]
        if kind == "scan" and max(_lengths(case)) * n * H > 1 << 22:
            return None
        cuts = st["cu_host"].tolist() if kind == "scan" else list(range(n + 1))
        state = torch.zeros(n, H, case["dstate"], case["headdim"], dtype=torch.float64, device=DEVICE)
        if st["state"] is not None:
            state = st["state"].double()
        group = torch.arange(H, device=DEVICE) // (H // G)
        x = st["x"].double()
        z = st["dt"].double() + st["dt_bias"].double()
        delta = torch.logaddexp(z, torch.zeros_like(z))
        alpha = torch.exp(-torch.exp(st["a_log"].double()) * delta)
        B, C = st["B"].double(), st["C"].double()
        y = torch.empty(x.shape[0], H, case["headdim"], dtype=torch.float64, device=DEVICE)
        first = torch.tensor(cuts[:-1], device=DEVICE)
        lens = torch.tensor(cuts[1:], device=DEVICE) - first
        # the recurrence itself, one token of every sequence at a time, the longest sequences first
        order = torch.argsort(lens, descending=True, stable=True)
        first, ordered = first[order], lens[order].tolist()
        state = state[order].contiguous()
        m = n
        for t in range(ordered[0] if ordered else 0):
            while ordered[m - 1] <= t:
                m -= 1
            i = first[:m] + t
            state[:m] *= alpha[i][:, :, None, None]
            state[:m].addcmul_(B[i][:, group][..., None], (delta[i][..., None] * x[i])[:, :, None])
            y[i] = (state[:m] * C[i][:, group][..., None]).sum(2)
        y += st["d"].double()[:, None] * x
        back = torch.empty_like(state)
        back[order] = state
        return dict(y=y, state=back)
    out = st["base"].double()
    cuts = st["cu_host"].tolist()
    for s, a in enumerate(st["ids_host"].tolist()):
        if a >= 0 and cuts[s + 1] > cuts[s]:
            u = st["x"][cuts[s]:cuts[s + 1]].double() @ st["a"][a].double().t()
            out[cuts[s]:cuts[s + 1]] += st["scales"][a].double() * (u @ st["b"][a].double().t())
    return dict(out=out)


# ------------------------------------------------------------------ the least work of a pass
def work(case):
    """Bytes: every input read once, every output written once.  Flops: the products of the formulas (for the scan the
    token-by-token form's: two multiply-adds per state element and token)."""
    T, n = _sizes(case)
    e = 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if kind in ("conv", "conv_step"):
        C, W = case["chans"], case["taps"]
        reads_history = kind == "conv_step" or case["history"]
        hist = n * (W - 1) * C * e
        return dict(bytes=2 * T * C * e + hist * (2 if reads_history else 1) + C * W * 4, flops=2 * W * T * C)
    if kind in ("scan", "step"):
        H, G, N, P = (case[k] for k in ("heads", "groups", "dstate", "headdim"))
        reads_state = kind == "step" or case["state"]
        return dict(bytes=T * (2 * H * P + 2 * G * N + H) * e + n * H * N * P * 4 * (2 if reads_state else 1),
                    flops=4 * T * H * N * P)
    K, M, R = case["hidden"], case["width"], case["rank"]
    ids = torch.randint(-1, case["adapters"], (n,), generator=torch.Generator().manual_seed(case["lens"] + 1),
                        dtype=torch.int32).tolist()
    lens = _lengths(case)
    adapted = sum(L for L, a in zip(lens, ids) if a >= 0)
    used = len({a for L, a in zip(lens, ids) if a >= 0 and L > 0})
    return dict(bytes=adapted * K * 2 + 2 * T * M * e + used * R * (K + M) * 2, flops=2 * adapted * R * (K + M))
