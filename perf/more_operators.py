"""The operators of a hybrid model's other layers at a prefix hit, as measurable cases: pages and slots from lengths,
norm and rotation of queries and keys on their way into the pages, attention of a batch that shares a prefix, and linear
attention with a fixed decay for each head.

Where `own` is false each operator is computed in its plain form, from elementary torch operations in 32 bits; where it
is true, by the package's public calls.  Inputs are laid out as a layer has them: q, k and v are columns of a
projection's rows, the caches are pages in a shuffled order, of which every sequence has a table.
"""
import math
import random

import torch

DEVICE = "cuda:0"
own = False

# a full-attention layer of grouped heads, in pages of 64 tokens
ATTN = dict(heads=32, kv_heads=4, dim=128, page=64, dtype="bf16")
ATTN_SMALL = dict(heads=8, kv_heads=8, dim=64, page=16, dtype="f32")
# the package's head layout (16 key heads, 32 value heads of 128) and one with a key head for each value head
LINEAR = dict(key_heads=16, heads=32, d_k=128, d_v=128, dtype="bf16")
LINEAR_EVEN = dict(key_heads=20, heads=20, d_k=128, d_v=64, dtype="bf16")


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one generated token of every conversation of a serving batch
        dict(name="pages_step_256", kind="pages", n=256, lo=1, hi=1, lens=1, held=4096, width=80, page=64),
        # 48 prompts arrive at once
        dict(name="pages_prompts_48", kind="pages", n=48, lo=64, hi=2048, lens=2, held=0, width=160, page=16),
        # one token of one conversation: the smallest call, all latency
        dict(ATTN, name="rope_step_1", kind="rope", tokens=1, rotary=64, interleaved=False, norm=True),
        # a prompt of 8192 tokens
        dict(ATTN, name="rope_prompt_8k", kind="rope", tokens=8192, rotary=128, interleaved=False, norm=True),
        # one token of one conversation of 819 tokens, nothing shared
        dict(ATTN, name="attn_step_1", kind="attn", n=1, lo=1, hi=1, lens=0, prefix=0, before=818),
        # one token for each of 128 conversations behind the same 8192 tokens
        dict(ATTN, name="attn_step_128", kind="attn", n=128, lo=1, hi=1, lens=1, prefix=8192, before=2047),
        # the new suffixes of 16 hits of one prefix of 8192 tokens: the largest case
        dict(ATTN, name="attn_suffixes_16", kind="attn", n=16, lo=128, hi=2048, lens=3, prefix=8192, before=0),
        # a prompt of 8192 tokens that nobody shares
        dict(ATTN, name="attn_prompt_8k", kind="attn", n=1, lo=8192, hi=8192, lens=0, prefix=0, before=0),
        # seven ragged continuations of a small fp32 layer, a prefix that ends inside a page
        dict(ATTN_SMALL, name="attn_ragged_f32", kind="attn", n=7, lo=1, hi=200, lens=4, prefix=1001, before=90),
        # the states rebuilt from 10 % of 8192 matched tokens
        dict(LINEAR, name="linear_tail_819", kind="linear", n=1, lo=819, hi=819, lens=0, state=False, outputs=False),
        # 16 concurrent suffixes, each from its own state
        dict(LINEAR, name="linear_suffixes_16", kind="linear", n=16, lo=128, hi=2048, lens=3, state=True, outputs=True),
        # one token for every conversation of a serving batch
        dict(LINEAR, name="linear_step_128", kind="linear_step", n=128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["pages", "rope", "attn", "attn", "attn", "attn", "linear", "linear", "linear_step"])
    lens = rng.randrange(1 << 20)
    if kind == "pages":
        n = _log_int(rng, 1, 512)
        hi = 1 if rng.random() < 0.4 else _log_int(rng, 1, max(1, 65536 // n))
        page = rng.choice([16, 64, 128, 1, 7, 48])
        held = rng.choice([0, _log_int(rng, 1, 4096 * min(page, 16) // 16 + 1)])
        return dict(kind="pages", n=n, lo=rng.choice([0, 1, hi]), hi=hi, lens=lens, held=held,
                    width=(held + hi) // page + _log_int(rng, 1, 64), page=page)
    if kind == "rope":
        heads = rng.choice([dict(ATTN), dict(ATTN, heads=16, kv_heads=16), dict(ATTN, heads=20, kv_heads=4),
                            dict(ATTN, heads=14, kv_heads=2, dim=64), dict(ATTN, heads=5, kv_heads=1),
                            dict(ATTN_SMALL), dict(ATTN_SMALL, heads=6, kv_heads=3, dim=128)])
        return dict(heads, kind="rope", tokens=_log_int(rng, 1, 8192),
                    rotary=rng.choice([16, 32, 48, 64]) * heads["dim"] // 64,
                    page=rng.choice([16, 64, 128, 1, 7, 48]), interleaved=rng.random() < 0.3, norm=rng.random() < 0.8)
    if kind == "attn":
        heads = rng.choice([dict(ATTN), dict(ATTN), dict(ATTN, heads=16, kv_heads=16), dict(ATTN, heads=20, kv_heads=4),
                            dict(ATTN, heads=28, kv_heads=4, dim=64), dict(ATTN, heads=5, kv_heads=1),
                            dict(ATTN_SMALL), dict(ATTN_SMALL, heads=6, kv_heads=2, dim=128)])
        heads["page"] = rng.choice([16, 64, 64, 128, 1, 7, 48])
        small = heads["dtype"] == "f32"
        prefix = rng.choice([0, 0, _log_int(rng, 1, 1024 if small else 12288)])
        if rng.random() < 0.45:
            n = _log_int(rng, 1, 32 if small else 128)
            hi, lo = rng.choice([1, 1, 1, 2, 5]), 1
            before = rng.choice([0, _log_int(rng, 1, 512 if small else 4096)])
        else:
            n = rng.choice([1, 1, 2, 5, _log_int(rng, 2, 32)])
            hi = _log_int(rng, 2, (1024 if small else 8192) // n)
            lo, before = rng.choice([0, 1, hi]) if n > 1 else hi, rng.choice([0, _log_int(rng, 1, 512)])
        return dict(heads, kind="attn", n=n, lo=lo, hi=hi, lens=lens, prefix=prefix, before=before)
    heads = rng.choice([LINEAR, LINEAR, LINEAR_EVEN, dict(LINEAR, d_k=64),
                        dict(LINEAR, key_heads=8, heads=8, d_k=64, d_v=64), dict(LINEAR, key_heads=5, heads=15), dict(LINEAR, key_heads=4, heads=8, d_k=64, dtype="f32"),
                        dict(LINEAR, key_heads=3, heads=3, d_v=64, dtype="f32")])
    if kind == "linear_step":
        return dict(heads, kind="linear_step", n=_log_int(rng, 1, 128))
    n = rng.choice([1, 1, 2, 5, _log_int(rng, 2, 64)])
    hi = _log_int(rng, 16, (4096 if heads["dtype"] == "f32" else 32768) // n)
    return dict(heads, kind="linear", n=n, lo=rng.choice([0, 1, hi]) if n > 1 else hi, hi=hi, lens=lens,
                state=rng.random() < 0.5, outputs=rng.random() < 0.7)


def _lengths(case):
    """The lengths of a batch's sequences: `n` of them between the two bounds, by the case alone."""
    rng = random.Random("%d" % case["lens"])
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["n"])]
    lens[-1] = case["hi"]
    return lens


def _held(case):
    """The tokens that each sequence holds before the call: between a half and all of the bound."""
    rng = random.Random("held %d" % case["lens"])
    most = case["held"] if case["kind"] == "pages" else case["before"]
    return [rng.randint((most + 1) // 2, most) for _ in range(case["n"])]


# ------------------------------------------------------------------ inputs
def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _offsets(lens):
    cu = torch.zeros(len(lens) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor(lens, dtype=torch.int64), 0).to(torch.int32)
    return cu.to(DEVICE), cu


def _tables(lens, page, width, pages):
    """A table of `width` pages for each sequence, filled as far as its tokens go, from the shuffled `pages`."""
    need = torch.tensor([(n + page - 1) // page for n in lens])
    first = torch.cumsum(need, 0) - need
    at = torch.arange(width)
    there = at < need[:, None]
    return torch.where(there, pages[torch.where(there, first[:, None] + at, 0)], -1).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, device=DEVICE, generator=gen)
    ru = lambda *s: torch.rand(*s, device=DEVICE, generator=gen)
    kind = case["kind"]
    st = dict(case=case)
    if "lo" in case:
        st["cu"], st["cu_host"] = _offsets(_lengths(case))
    if kind == "pages":
        held, page, n, W = _held(case), case["page"], case["n"], case["width"]
        total = sum((a + b + page - 1) // page for a, b in zip(held, _lengths(case)))
        pages = torch.randperm(total + 8, generator=host, dtype=torch.int64)
        table = _tables(held, page, W, pages)
        used = sum((a + page - 1) // page for a in held)
        T = int(st["cu_host"][-1])
        new = lambda *s: torch.empty(*s, dtype=torch.int32, device=DEVICE)
        st.update(table=table.to(DEVICE), held=torch.tensor(held, dtype=torch.int32, device=DEVICE),
                  free=pages.to(torch.int32).to(DEVICE), taken=torch.tensor([used], dtype=torch.int32, device=DEVICE),
                  table_out=new(n, W), lens_out=new(n), taken_out=new(1), slots=new(T), positions=new(T))
        return st
    dt = _dt(case)
    if kind == "rope":
        T, H, Hk, D, R, page = (case[k] for k in ("tokens", "heads", "kv_heads", "dim", "rotary", "page"))
        row = rn(T, (H + 2 * Hk) * D).to(dt)
        far = 2 * T + 64                                         # the table's positions
        angle = torch.arange(far, dtype=torch.float64, device=DEVICE)[:, None] * 10000.0 ** (
            -torch.arange(0, R, 2, dtype=torch.float64, device=DEVICE) / R)
        pages = T // page + 2
        st.update(q=row[:, :H * D].unflatten(1, (H, D)), k=row[:, H * D:(H + Hk) * D].unflatten(1, (Hk, D)),
                  v=row[:, (H + Hk) * D:].unflatten(1, (Hk, D)), cos_sin=torch.cat([angle.cos(), angle.sin()], 1).float(),
                  positions=torch.arange(T, dtype=torch.int32, device=DEVICE) + int(torch.randint(T + 64, (1,), generator=host)),
                  q_weight=0.5 + ru(D) if case["norm"] else None, k_weight=0.5 + ru(D) if case["norm"] else None,
                  k_cache=torch.zeros(pages, page, Hk, D, dtype=dt, device=DEVICE),
                  v_cache=torch.zeros(pages, page, Hk, D, dtype=dt, device=DEVICE),
                  slots=(torch.randperm(pages, device=DEVICE, generator=gen, dtype=torch.int32)[:, None] * page
                         + torch.arange(page, dtype=torch.int32, device=DEVICE)).reshape(-1)[:T],
                  q_out=torch.empty(T, H, D, dtype=dt, device=DEVICE))
        return st
    if kind == "attn":
        H, Hk, D, page, n, P = (case[k] for k in ("heads", "kv_heads", "dim", "page", "n", "prefix"))
        T = int(st["cu_host"][-1])
        total = [a + b for a, b in zip(_held(case), _lengths(case))]
        shared = (P + page - 1) // page
        count = shared + sum((m + page - 1) // page for m in total) + 3
        pages = torch.randperm(count, generator=host)
        width = max(1, (max(total) + page - 1) // page)
        # queries and keys as after the norms: scores of a few units
        st.update(q=rn(T, (H + 2 * Hk) * D).to(dt)[:, :H * D].unflatten(1, (H, D)),
                  k_cache=rn(count, page, Hk, D).to(dt), v_cache=rn(count, page, Hk, D).to(dt),
                  table=_tables(total, page, width, pages[shared:]).to(DEVICE),
                  lens=torch.tensor(total, dtype=torch.int32, device=DEVICE), lens_host=total,
                  prefix_pages=pages[:shared].to(torch.int32).to(DEVICE) if P else None,
                  out=torch.empty(T, H, D, dtype=dt, device=DEVICE))
        return st
    Hk, H, K, V, n = (case[k] for k in ("key_heads", "heads", "d_k", "d_v", "n"))
    T = n if kind == "linear_step" else int(st["cu_host"][-1])
    row = torch.nn.functional.silu(rn(T, 2 * Hk * K + H * V)).to(dt)
    st.update(q=row[:, :Hk * K].unflatten(1, (Hk, K)), k=row[:, Hk * K:2 * Hk * K].unflatten(1, (Hk, K)),
              v=row[:, 2 * Hk * K:].unflatten(1, (H, V)),
              g=-torch.exp(math.log(0.002) + ru(H) * math.log(350.0)),         # decays of 0.998 to 0.5 a token
              state=rn(n, H, K, V) if kind == "linear_step" or case["state"] else None,
              state_out=torch.empty(n, H, K, V, dtype=torch.float32, device=DEVICE))
    st["out"] = torch.empty(T, H, V, dtype=dt, device=DEVICE) if case.get("outputs", True) else None
    return st


# ------------------------------------------------------------------ the calls
def run(st):
    case = st["case"]
    kind = case["kind"]
    if own:
        import paper_2608_30310_amd as gdn
        if kind == "pages":
            table, lens, taken, slots, positions = gdn.extend_pages(
                st["table"], st["held"], st["cu"], st["free"], case["page"], st["cu_host"], taken=st["taken"],
                table_out=st["table_out"], lens_out=st["lens_out"], taken_out=st["taken_out"], slots=st["slots"],
                positions=st["positions"])
            return dict(table=table, lens=lens, taken=taken, slots=slots, positions=positions)
        if kind == "rope":
            q, _ = gdn.qk_norm_rope(st["q"], st["k"], st["positions"], st["cos_sin"], st["q_weight"], st["k_weight"],
                                    eps=1e-6, interleaved=case["interleaved"], v=st["v"], k_cache=st["k_cache"],
                                    v_cache=st["v_cache"], slots=st["slots"], q_out=st["q_out"])
            return dict(q=q, k_cache=st["k_cache"], v_cache=st["v_cache"])
        if kind == "attn":
            return dict(out=gdn.prefix_attention(st["q"], st["k_cache"], st["v_cache"], st["table"], st["lens"], st["cu"],
                                                 st["cu_host"], prefix_pages=st["prefix_pages"], prefix_len=case["prefix"],
                                                 out=st["out"]))
        scale = case["d_k"] ** -0.5
        if kind == "linear":
            o, s = gdn.linear_attention(st["q"], st["k"], st["v"], st["g"], st["cu"], st["cu_host"], scale=scale,
                                        state_in=st["state"], outputs=case["outputs"], out=st["out"],
                                        state_out=st["state_out"])
        else:
            o, s = gdn.linear_attention_step(st["q"], st["k"], st["v"], st["g"], state_in=st["state"], scale=scale,
                                             out=st["out"], state_out=st["state_out"])
        return dict(out=o, state=s)
    return dict(pages=_plain_pages, rope=_plain_rope, attn=_plain_attn, linear=_plain_linear,
                linear_step=_plain_linear_step)[kind](st)


def _plain_pages(st):
    case = st["case"]
    page, W = case["page"], case["width"]
    held, cu, free = st["held"].long(), st["cu"].long(), st["free"]
    lens = held + cu[1:] - cu[:-1]
    have = torch.clamp((held + page - 1) // page, max=W)
    need = torch.clamp((lens + page - 1) // page, max=W)
    ends = torch.cumsum(need - have, 0) + st["taken"].long()
    at = torch.arange(W, device=cu.device)
    index = (ends - need)[:, None] + at                             # of page `at` in the free list
    new = torch.where(index < free.numel(), free[index.clamp(0, free.numel() - 1)], -1)
    table = torch.where((at >= have[:, None]) & (at < need[:, None]), new, st["table"])
    token = torch.arange(st["slots"].numel(), device=cu.device)
    seq = torch.searchsorted(cu[1:], token, right=True)
    position = held[seq] + token - cu[seq]
    of = position // page
    number = torch.where(of < W, table[seq, of.clamp(max=W - 1)].long(), -1)
    slots = torch.where(number >= 0, number * page + position % page, -1)
    return dict(table=table, lens=lens.to(torch.int32), taken=ends[-1:].to(torch.int32), slots=slots.to(torch.int32),
                positions=position.to(torch.int32))


def _rotated(x, cos, sin, R, interleaved):
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    c, d = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([c, d], -1).flatten(-2) if interleaved else torch.cat([c, d], -1)
    return torch.cat([turned, x[..., R:]], -1)


def _plain_rope(st):
    case = st["case"]
    R, dt = case["rotary"], st["q_out"].dtype
    rows = st["cos_sin"][st["positions"].long()]
    cos, sin = rows[:, None, :R // 2], rows[:, None, R // 2:]

    def one(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
        return _rotated(x, cos, sin, R, case["interleaved"]).to(dt)
    slots = st["slots"].long()
    st["k_cache"].flatten(0, 1)[slots] = one(st["k"], st["k_weight"])
    st["v_cache"].flatten(0, 1)[slots] = st["v"]
    return dict(q=one(st["q"], st["q_weight"]), k_cache=st["k_cache"], v_cache=st["v_cache"])


def _plain_attn(st):
    """Scores of all tokens against the prefix by one product, those against the own keys in sequences padded to the
    longest, one softmax over both."""
    case = st["case"]
    H, Hk, D, page, P = (case[k] for k in ("heads", "kv_heads", "dim", "page", "prefix"))
    G, dev = H // Hk, st["q"].device
    cu, total = st["cu_host"].long(), torch.tensor(st["lens_host"])
    new = cu[1:] - cu[:-1]
    n, Lq, Lk = len(new), int(new.max()), int(total.max())
    off = torch.arange(Lq)
    there = off < new[:, None]
    tok = torch.where(there, cu[:-1, None] + off, 0).to(dev)                     # [n, Lq]
    spots = there.reshape(-1).nonzero()[:, 0].to(dev)
    q = st["q"].float() * D ** -0.5
    keys = torch.arange(Lk, device=dev)
    row = st["table"].long()[:, keys // page].clamp(min=0) * page + keys % page  # [n, Lk]
    total, new = total.to(dev), new.to(dev)
    take = lambda c, r: c.flatten(0, 1)[r].float()
    inside = (keys < total[:, None])[..., None, None]
    k = torch.where(inside, take(st["k_cache"], row), 0.0).permute(0, 2, 1, 3)   # [n, Hk, Lk, D]
    v = torch.where(inside, take(st["v_cache"], row), 0.0).permute(0, 2, 1, 3)
    qo = q[tok].view(n, Lq, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(n, Hk, G * Lq, D)
    last = (total - new)[:, None] + torch.arange(Lq, device=dev)                 # [n, Lq]: the last key that a query sees
    seen = (keys <= last[..., None])[:, None, None]                              # [n, 1, 1, Lq, Lk]
    s = (qo @ k.transpose(-1, -2)).view(n, Hk, G, Lq, Lk).masked_fill(~seen, -math.inf)
    top = s.amax(-1)                                                             # [n, Hk, G, Lq]
    if P:
        at = torch.arange(P, device=dev)
        rows = st["prefix_pages"].long()[at // page] * page + at % page
        kp, vp = (take(st[c], rows).transpose(0, 1) for c in ("k_cache", "v_cache"))   # [Hk, P, D]
        qp = q.view(-1, Hk, G, D).permute(1, 2, 0, 3).reshape(Hk, -1, D)         # [Hk, G T, D]
        sp = (qp @ kp.transpose(-1, -2)).view(Hk, G, -1, P)
        tp = sp.amax(-1)[:, :, tok].permute(2, 0, 1, 3)                          # [n, Hk, G, Lq]
        top = torch.maximum(top, tp)
        by_token = top.permute(1, 2, 0, 3).reshape(Hk, G, -1)[:, :, spots]       # [Hk, G, T]
        sp = torch.exp(sp - by_token[..., None])
        sum_p = sp.sum(-1)
        out_p = (sp.view(Hk, -1, P) @ vp).view(Hk, G, -1, D)
    s = torch.exp(s - top[..., None])
    weight = s.sum(-1)
    out = (s.view(n, Hk, G * Lq, Lk) @ v).view(n, Hk, G, Lq, D)
    weight = weight.permute(0, 3, 1, 2).reshape(n * Lq, Hk, G)[spots]
    out = out.permute(0, 3, 1, 2, 4).reshape(n * Lq, Hk, G, D)[spots]            # packed order
    if P:
        weight = weight + sum_p.permute(2, 0, 1)
        out = out + out_p.permute(2, 0, 1, 3)
    return dict(out=(out / weight[..., None]).reshape(-1, H, D).to(st["out"].dtype))


def _plain_linear(st):
    """Chunks of 64 tokens, all at once: products inside the chunks, then every chunk's start as the sum of the chunks
    before it in its sequence, each by its decay."""
    case = st["case"]
    Hk, H, K, V, n, Q = (*(case[k] for k in ("key_heads", "heads", "d_k", "d_v", "n")), 64)
    dev = st["v"].device
    lens = st["cu_host"][1:].long() - st["cu_host"][:-1].long()
    per = (lens + Q - 1) // Q
    nc = int(per.sum())
    seq = torch.repeat_interleave(torch.arange(n), per)                          # [nc]: each chunk's sequence
    first = torch.cumsum(per, 0) - per
    start = (torch.arange(nc) - first[seq]) * Q
    off = start[:, None] + torch.arange(Q)
    there = off < lens[seq][:, None]
    spots = there.reshape(-1).nonzero()[:, 0].to(dev)
    tok = torch.where(there, st["cu_host"].long()[seq][:, None] + off, 0).to(dev)
    count = (lens[seq] - start).clamp(max=Q).to(dev)                             # tokens of each chunk
    seq, there, lens = seq.to(dev), there.to(dev), lens.to(dev)
    take = lambda t: torch.where(there[..., None, None], t.float()[tok], 0.0).transpose(1, 2)   # [nc, heads, Q, d]
    wide = lambda t: take(t)[:, :, None].expand(nc, Hk, H // Hk, Q, K).reshape(nc, H, Q, K)
    v, k = take(st["v"]), wide(st["k"])
    g = st["g"].double()
    at = torch.arange(Q, device=dev, dtype=torch.float64)
    left = (count[:, None] - 1 - at).clamp(min=0)                                # [nc, Q]: tokens behind
    w = torch.exp(g[:, None] * left[:, None]).float()                            # [nc, H, Q]
    own_state = (k * w[..., None]).transpose(-1, -2) @ v                         # [nc, H, K, V]
    total = g * count[:, None]                                                   # [nc, H]
    ends = torch.cumsum(total, 0)
    before = (seq[:, None] == seq[None, :]) & (torch.arange(nc, device=dev)[:, None] > torch.arange(nc, device=dev))
    decay = torch.exp(torch.where(before[..., None], (ends - total)[:, None] - ends[None, :], -math.inf)).float()
    begin = (decay.permute(2, 0, 1) @ own_state.transpose(0, 1).reshape(H, nc, K * V)).view(H, nc, K, V).transpose(0, 1)
    state = torch.zeros(n, H, K, V, device=dev) if st["state"] is None else st["state"]
    if nc:
        base = ends - total
        f = first.to(dev).clamp(max=nc - 1)
        begin = begin + torch.exp(base - base[f[seq]]).float()[..., None, None] * state[seq]
        end = torch.exp(total).float()[..., None, None] * begin + own_state
        last = (first.to(dev) + per.to(dev) - 1).clamp(min=0)
        state = torch.where((lens > 0)[:, None, None, None], end[last], state)
    if not case["outputs"]:
        return dict(out=None, state=state)
    q = wide(st["q"]) * K ** -0.5
    gap = at[:, None] - at
    L = torch.exp(torch.where(gap >= 0, g[:, None, None] * gap, -math.inf)).float()
    pre = torch.exp(g[:, None] * (at + 1)).float()                               # [H, Q]
    o = ((q @ k.transpose(-1, -2)) * L) @ v + pre[..., None] * (q @ begin)
    return dict(out=o.transpose(1, 2).reshape(nc * Q, H, V)[spots].to(st["v"].dtype), state=state)


def _plain_linear_step(st):
    case = st["case"]
    per = case["heads"] // case["key_heads"]
    q, k = (st[x].float().repeat_interleave(per, 1) for x in ("q", "k"))
    state = torch.exp(st["g"])[:, None, None] * st["state"] + k[..., None] * st["v"].float()[..., None, :]
    o = (q[..., None] * state).sum(2) * case["d_k"] ** -0.5
    return dict(out=o.to(st["out"].dtype), state=state)


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    kind = case["kind"]
    if kind == "pages":
        return None
    st = prepare(case, seed)
    if kind == "rope":
        T, R = case["tokens"], case["rotary"]
        angle = st["cos_sin"].double()[st["positions"].long()]
        turn = torch.complex(angle[:, :R // 2], angle[:, R // 2:])[:, None]      # [T, 1, R / 2]

        def one(x, w):
            x = x.double()
            if w is not None:
                x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6) * w.double()
            y = x.clone()
            even, odd = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
            z = torch.complex(x[..., even].contiguous(), x[..., odd].contiguous()) * turn
            y[..., even], y[..., odd] = z.real, z.imag
            return y
        kc, vc = st["k_cache"].double(), st["v_cache"].double()
        kc.flatten(0, 1)[st["slots"].long()] = one(st["k"], st["k_weight"])
        vc.flatten(0, 1)[st["slots"].long()] = st["v"].double()
        return dict(q=one(st["q"], st["q_weight"]), k_cache=kc, v_cache=vc)
    if kind == "attn":
        H, Hk, D, page, P = (case[k] for k in ("heads", "kv_heads", "dim", "page", "prefix"))
        G = H // Hk
        out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEVICE)
        cuts, at = st["cu_host"].tolist(), torch.arange(P, device=DEVICE)
        head = [] if P == 0 else [st["prefix_pages"].long()[at // page] * page + at % page]
        for s, m in enumerate(st["lens_host"]):
            L = cuts[s + 1] - cuts[s]
            at = torch.arange(m, device=DEVICE)
            rows = torch.cat(head + [st["table"][s].long()[at // page] * page + at % page])
            for h in range(Hk if L else 0):
                k, v = (st[c].flatten(0, 1)[rows, h].double() for c in ("k_cache", "v_cache"))
                for a in range(0, L, 1024):                                     # queries a .. b of the sequence
                    b = min(L, a + 1024)
                    q = st["q"][cuts[s] + a:cuts[s] + b, h * G:(h + 1) * G].double()
                    w = torch.einsum("tgd,kd->gtk", q, k) / math.sqrt(D)
                    hidden = torch.arange(P + m, device=DEVICE) > P + m - L + torch.arange(a, b, device=DEVICE)[:, None]
                    w = torch.softmax(w.masked_fill(hidden, -math.inf), -1)
                    out[cuts[s] + a:cuts[s] + b, h * G:(h + 1) * G] = (w @ v).transpose(0, 1)
        return dict(out=out)
    H, n = case["heads"], case["n"]
    if kind == "linear" and max(_lengths(case)) * n * H > 1 << 21:
        return None
    cuts = st["cu_host"].tolist() if kind == "linear" else list(range(n + 1))
    state = torch.zeros(n, H, case["d_k"], case["d_v"], dtype=torch.float64, device=DEVICE)
    if st["state"] is not None:
        state = st["state"].double()
    group = torch.arange(H, device=DEVICE) // (H // case["key_heads"])
    q, k, v = (st[x].double() for x in ("q", "k", "v"))
    alpha = torch.exp(st["g"].double())[:, None, None]
    out = torch.empty(v.shape, dtype=torch.float64, device=DEVICE)
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
        state[:m] *= alpha
        state[:m].addcmul_(k[i][:, group][..., None], v[i][:, :, None])
        out[i] = (state[:m] * q[i][:, group][..., None]).sum(2) * case["d_k"] ** -0.5
    back = torch.empty_like(state)
    back[order] = state
    return dict(out=out if case.get("outputs", True) else None, state=back)


# ------------------------------------------------------------------ the least work of a pass
def work(case):
    """Bytes: every input read once, every output written once, a shared prefix once for all.  Flops: the products of the
    formulas (linear attention: the token-by-token form's, two multiply-adds per state element and token)."""
    kind, n = case["kind"], case.get("n", 0)
    if kind == "pages":
        T = sum(_lengths(case))
        return dict(bytes=4 * (2 * n * case["width"] + 3 * n + 3 + 2 * T), flops=0)
    e = 2 if case["dtype"] == "bf16" else 4
    if kind == "rope":
        T, H, Hk, D, R = (case[k] for k in ("tokens", "heads", "kv_heads", "dim", "rotary"))
        return dict(bytes=T * (2 * (H + 2 * Hk) * D * e + 4 * R + 8), flops=T * (H + Hk) * (4 * D + 3 * R))
    if kind == "attn":
        H, Hk, D, P = (case[k] for k in ("heads", "kv_heads", "dim", "prefix"))
        pairs = keys = 0
        for L, b in zip(_lengths(case), _held(case)):
            pairs += L * (P + b) + L * (L + 1) // 2
            keys += b + L
        return dict(bytes=2 * sum(_lengths(case)) * H * D * e + 2 * (P + keys) * Hk * D * e, flops=4 * D * H * pairs)
    Hk, H, K, V = (case[k] for k in ("key_heads", "heads", "d_k", "d_v"))
    T = n if kind == "linear_step" else sum(_lengths(case))
    outputs, reads = case.get("outputs", True), kind == "linear_step" or case["state"]
    return dict(bytes=T * ((Hk * K + H * V) * (2 if outputs else 1)) * e + n * H * K * V * 4 * (2 if reads else 1),
                flops=(4 if outputs else 2) * T * H * K * V)
