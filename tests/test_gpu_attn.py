"""Attention over a shared prefix and own pages against fp64, query by query.

Bounds.  A score is an fp32 sum of D products, within (D + 2) 2^-24 of |scale| sum
|q k| =: S, and its distance from the maximum, at most R, is rounded when it goes
into the exponent, 2^-23 R; so a weight is off by e = (D + 2) 2^-24 S + 2^-23 R + 2^-22
relative, in numerator and denominator.  n weights are added in fp32, n 2^-24.  With
bf16 the weights enter the second product rounded, by 2^-8 each.  So outputs are
within 2 e + n 2^-23 (+ 2^-8) of sum w |v| / sum w, and a bf16 output is rounded once
more, by 2^-8 of itself.
"""
import ctypes
import threading

import pytest
import torch

import paper_2608_30310_amd as gdn
from oracle import attn_ops as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    gdn.load_library()


def case(new, before=0, prefix=0, H=4, Hk=2, D=64, ps=16, dtype="bf16", seed=0, layout="pages", pad=0, spare=0, size=1.0,
         junk=float("nan")):
    """Sequences of `before` held and `new` query tokens; whatever no table names is `junk`."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    rn = lambda *s: torch.randn(*s, device=DEV, generator=g)
    dt = BF if dtype == "bf16" else torch.float32
    before = [before] * len(new) if isinstance(before, int) else before
    lens = [b + q for b, q in zip(before, new)]
    shared = -(-prefix // ps)
    need = [-(-m // ps) for m in lens]
    pages = shared + sum(need) + 2
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    W = max(need + [1]) + 1
    table, at = torch.full((len(new), W), -1, dtype=torch.int32), shared
    rows = [p * ps + r for p in perm[:shared] for r in range(ps)][:prefix]
    for n, (c, m) in enumerate(zip(need, lens)):
        table[n, :c] = torch.tensor(perm[at:at + c], dtype=torch.int32)
        rows += [p * ps + r for p in perm[at:at + c] for r in range(ps)][:m]
        at += c
    shape = dict(pages=(pages, ps, Hk, D), heads=(pages, Hk, ps, D), both=(pages, 2, ps, Hk, D), rows=(pages, ps, 2, Hk, D))[layout]

    def cache(kv):
        c = torch.full(shape, junk, dtype=dt, device=DEV) if kv == 0 or layout in ("pages", "heads") else kc_all
        c0 = c.transpose(1, 2) if layout == "heads" else c[:, kv] if layout == "both" else c[:, :, kv] if layout == "rows" else c
        flat = torch.full((pages * ps, Hk, D), junk, dtype=dt, device=DEV)
        flat[torch.tensor(rows, dtype=torch.int64, device=DEV)] = (rn(len(rows), Hk, D) * (size if kv == 0 else 1.0)).to(dt)
        c0.copy_(flat.view(pages, ps, Hk, D))
        return c, c0
    kc_all, kc = cache(0)
    _, vc = cache(1)
    cu = torch.tensor([0] + list(torch.tensor(new).cumsum(0)), dtype=torch.int32)
    T = sum(new) + spare
    q = rn(T, H * D + pad).to(dt)[:, :H * D].unflatten(1, (H, D))
    return dict(q=q, k_cache=kc, v_cache=vc, table=table.to(DEV), lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
                cu=cu.to(DEV), cu_host=cu, prefix_pages=torch.tensor(perm[:shared], dtype=torch.int32, device=DEV) if prefix else None,
                prefix_len=prefix)


def call(c, **kw):
    kw = dict(dict(prefix_pages=c["prefix_pages"], prefix_len=c["prefix_len"]), **kw)
    return gdn.prefix_attention(c["q"], c["k_cache"], c["v_cache"], c["table"], c["lens"], c["cu"], c["cu_host"], **kw)


def check(c, out, rows=None, **kw):
    T, D = int(c["cu_host"][-1]), c["q"].shape[2]
    want, mag, S, R, n = ref.attention(c["q"][:T], c["k_cache"], c["v_cache"], c["table"], c["lens"], c["cu_host"].tolist(),
                                       c["prefix_pages"], c["prefix_len"], **kw)
    bf = out.dtype == BF
    e = (D + 2) * 2.0 ** -24 * S + 2.0 ** -23 * R + 2.0 ** -22
    bound = (2 * e + (n * 2.0 ** -23)[:, None])[..., None] + (2.0 ** -8 if bf else 0.0)
    allowed = bound * mag + (2.0 ** -8 * want.abs() * (1 + bound) if bf else 0.0) + 1e-37
    got = out[:T].double()
    pick = slice(None) if rows is None else rows
    assert torch.isfinite(got[pick]).all()
    worst = float(((got - want).abs() / allowed)[pick].max()) if T else 0.0
    print(f"[attn] worst {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0


DT = pytest.mark.parametrize("dtype", ["bf16", "f32"])


@DT
@pytest.mark.parametrize("prefix", [0, 1, 40, 130])
@pytest.mark.parametrize("new", [[1], [2], [31], [33], [64], [65], [130], [1, 0, 17, 70], [0, 0, 3]], ids=str)
def test_prompts(dtype, new, prefix):
    c = case(new, prefix=prefix, dtype=dtype, seed=prefix + len(new))
    check(c, call(c))


@DT
@pytest.mark.parametrize("prefix", [0, 100, 1500])
@pytest.mark.parametrize("n,before", [(1, 0), (1, 15), (1, 700), (1, 3000), (7, [0, 1, 15, 16, 63, 64, 1000]), (40, 33)], ids=str)
def test_single_tokens(dtype, n, before, prefix):
    c = case([1] * n, before, prefix, H=8, Hk=2, D=128, dtype=dtype, seed=n)
    check(c, call(c))


@DT
@pytest.mark.parametrize("ps", [1, 3, 7, 16, 48, 64, 100, 1000])
def test_page_sizes(dtype, ps):
    c = case([40, 1, 5], [10, 200, 0], 90, ps=ps, dtype=dtype, seed=ps)
    check(c, call(c))


@DT
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Hk", [(1, 1), (3, 3), (5, 1), (8, 1), (28, 4), (40, 1)])
def test_heads(dtype, D, H, Hk):
    c = case([20, 1, 3], [0, 90, 7], 70, H=H, Hk=Hk, D=D, dtype=dtype, seed=H)
    check(c, call(c))


@DT
@pytest.mark.parametrize("layout", ["heads", "both", "rows"])
def test_layouts(dtype, layout):
    c = case([20, 1, 70], [0, 90, 7], 70, dtype=dtype, seed=2, layout=layout, pad=16)
    check(c, call(c))


@DT
@pytest.mark.parametrize("new,before,prefix", [([700], 0, 0), ([400, 300], [0, 50], 600), ([2, 3, 5] * 12, 100, 900), ([200], 0, 4000)], ids=str)
def test_long(dtype, new, before, prefix):
    c = case(new, before, prefix, H=4, Hk=1, D=128, dtype=dtype, seed=9)
    check(c, call(c))


@DT
def test_large_scores(dtype):
    """Scores of hundreds, so that a key's weight is one or nothing, and the maximum moves late."""
    c = case([70, 1, 1], [0, 300, 64], 200, dtype=dtype, seed=3, size=30.0)
    check(c, call(c))
    c = case([130], 0, 100, dtype=dtype, seed=4)
    flat = c["k_cache"].reshape(-1, 2, 64)
    ps, at = 16, torch.arange(130, device=DEV)
    rows = c["table"][0].long()[at // ps] * ps + at % ps
    flat[rows] = (flat[rows].float() * torch.linspace(0.01, 20, 130, device=DEV)[:, None, None]).to(flat.dtype)
    check(c, call(c))


@DT
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0, 3.0])
def test_scales(dtype, scale):
    c = case([30, 1], [0, 90], 50, dtype=dtype, seed=5)
    check(c, call(c, scale=scale), scale=scale)


@DT
def test_queries_that_see_nothing(dtype):
    """Lengths that are less than the queries, zero or negative; lengths behind the table and behind max_len."""
    c = case([10, 4, 3, 2, 1, 5], [0, 0, 0, 0, 0, 60], dtype=dtype, seed=6)
    c["lens"] = torch.tensor([4, 0, -7, 2, 1, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    c["k_cache"][torch.isnan(c["k_cache"])] = 1.0   # (the last sequence's length takes it behind what was filled)
    c["v_cache"][torch.isnan(c["v_cache"])] = 1.0
    out = call(c)
    check(c, out)
    assert (out[:6] == 0).all() and (out[10:17] == 0).all()
    check(c, call(c, max_len=50), max_len=50)
    check(c, call(c, max_len=1), max_len=1)


@DT
def test_pages_that_are_none(dtype):
    """Entries outside the cache, in the table and in the prefix: their tokens are not seen."""
    c = case([40, 1, 1], [30, 200, 16], 100, dtype=dtype, seed=7)
    pages = c["k_cache"].shape[0]
    c["table"][0, 1], c["table"][1, 3], c["table"][1, 12], c["table"][2, :2] = -1, pages, 2 ** 31 - 1, -2 ** 31
    c["prefix_pages"][2] = -5
    check(c, call(c))
    c["prefix_pages"][:] = pages
    out = call(c)
    check(c, out)
    assert (out[41] == 0).all()


@DT
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("which", ["k_cache", "v_cache"])
@pytest.mark.parametrize("prefix,before", [(0, 0), (70, 40)])
def test_values_that_are_not_finite_reach_those_who_see_them(dtype, value, which, prefix, before):
    c = case([90, 20, 1], [before, 3, 50], prefix, dtype=dtype, seed=8)
    want = call(c)
    at = before + 37   # the first query that sees it is number 37
    slot = int(c["table"][0, at // 16]) * 16 + at % 16
    c[which][slot // 16, slot % 16, 1, 5] = value
    out = call(c)
    heads = torch.tensor([0, 1])
    assert torch.equal(out[:37], want[:37]) and torch.equal(out[90:], want[90:]) and torch.equal(out[:, heads], want[:, heads])
    if which == "v_cache":
        assert not torch.isfinite(out[37:90, 2:, 5].float()).any()
        rest = [d for d in range(64) if d != 5]
        assert torch.equal(out[37:90, 2:, rest], want[37:90, 2:, rest])
    elif value != value:
        assert torch.isnan(out[37:90, 2:].float()).all()


# Sequences of such batches take each of the ways: rows of their own, with and without a prefix that all rows share
# out, single tokens of one line with and without a prefix, few rows of too many sequences for a line.
WAYS = pytest.mark.parametrize("new,before,prefix", [([70, 1], 0, 0), ([150, 40], [30, 7], 70), ([1, 1, 1], [0, 40, 300], 0), ([1, 2], [3, 90], 130),
                                                     ([1, 2] + [1] * 1030, 3, 0), ([3], 0, 0)], ids=["rows", "shared", "line", "behind", "many", "few"])


def formula(c, out_head, t, n, i):
    """The formula for query i of sequence n (packed row t) and a head, its pieces in fp64: the output, the weighted
    magnitudes, and S, R and the keys seen over the scores that are finite."""
    ps, Hk = c["k_cache"].shape[1:3]
    q = c["q"][t, out_head].double()
    kvh = out_head // (c["q"].shape[1] // Hk)
    m = int(c["lens"][n])
    own = torch.arange(max(0, m - (int(c["cu_host"][n + 1]) - int(c["cu_host"][n])) + i + 1), device=DEV)
    at = torch.arange(c["prefix_len"], device=DEV)
    rows = c["table"][n].long()[own // ps] * ps + own % ps
    if c["prefix_len"]:
        rows = torch.cat([c["prefix_pages"].long()[at // ps] * ps + at % ps, rows])
    k, v = (c[x].reshape(-1, *c[x].shape[2:])[rows, kvh].double() for x in ("k_cache", "v_cache"))
    x = (q * k).sum(1) * len(q) ** -0.5
    w = torch.exp(x - x.max())
    w = w / w.sum()
    fin = torch.isfinite(x)
    S = float((q * k)[fin].abs().sum(1).max()) * len(q) ** -0.5 if fin.any() else 0.0
    R = float(x[fin].max() - x[fin].min()) if fin.any() else 0.0
    return (w[:, None] * v).sum(0), (w[:, None] * v.abs()).sum(0), S, R, len(rows)


@DT
@WAYS
@pytest.mark.parametrize("value", [1.0, float("nan")])
def test_scores_of_minus_infinity(dtype, new, before, prefix, value):
    """Keys whose score is -inf weigh nothing beside others, and a query that sees no other has no output: 0 / 0.  The
    first 37 tokens, and the prefix, have such keys for head 2, whose scores for head 3 are +inf.  A value of theirs
    that is not finite reaches those who see it at a weight of nothing too."""
    c = case(new, before, prefix, dtype=dtype, seed=19)
    c["q"][:, 2, 5], c["q"][:, 3, 5] = c["q"][:, 2, 5].abs() + 0.1, -c["q"][:, 3, 5].abs() - 0.1
    ps = 16
    first = min(37, int(c["lens"][0]))
    slots = [int(c["table"][0, j // ps]) * ps + j % ps for j in range(first)]
    slots += [int(c["prefix_pages"][j // ps]) * ps + j % ps for j in range(prefix)]
    for s in slots:
        c["k_cache"][s // ps, s % ps, 1, 5] = float("-inf")
    c["v_cache"][slots[-1] // ps, slots[-1] % ps, 1, 9] = value
    out = call(c)
    D, bf, nans, worst = 64, dtype == "bf16", 0, 0.0
    for n in range(min(len(new), 3)):
        for i in range(new[n]):
            t = int(c["cu_host"][n]) + i
            for h in range(4):
                want, mag, S, R, keys = formula(c, h, t, n, i)
                got, none = out[t, h].double(), torch.isnan(want)
                assert torch.equal(torch.isnan(got), none), (n, i, h)
                nans += int(none.all())
                e = (D + 2) * 2.0 ** -24 * S + 2.0 ** -23 * R + 2.0 ** -22
                bound = 2 * e + keys * 2.0 ** -23 + (2.0 ** -8 if bf else 0.0)
                allowed = bound * mag + (2.0 ** -8 * want.abs() * (1 + bound) if bf else 0.0) + 1e-37
                if not none.all():
                    worst = max(worst, float(((got - want).abs() / allowed)[~none].max()))
    print(f"[attn] worst {worst:.3f} of the bound, {nans} rows without an output", flush=True)
    assert nans > 0 and worst <= 1.0


@DT
def test_rows_left_alone_and_out(dtype):
    c = case([20, 5], [0, 30], 20, dtype=dtype, seed=10, spare=6, pad=8)
    rows = torch.full((31, 4 * 64 + 24), 7.0, dtype=c["q"].dtype, device=DEV)
    out = rows[:, 8:264].unflatten(1, (4, 64))
    assert call(c, out=out) is out
    assert torch.equal(out[:25], call(c)[:25])
    assert (rows[25:] == 7).all() and (rows[:, :8] == 7).all() and (rows[:, 264:] == 7).all()


@DT
def test_prefix_is_the_same_as_own_tokens(dtype):
    """A prefix that is given as such, and as the first pages of the one sequence."""
    c = case([33], 0, 96, dtype=dtype, seed=11)
    own = dict(c, table=torch.cat([c["prefix_pages"], c["table"][0]])[None].contiguous(), lens=c["lens"] + 96, prefix_pages=None,
               prefix_len=0)
    a, b = call(c), call(own)
    check(c, a)
    check(own, b)


@DT
def test_captured_steps_advance(dtype):
    """A step of single tokens, captured once: lengths, tables and caches move on between the replays."""
    c = case([1] * 6, [3, 14, 15, 16, 200, 90], 120, dtype=dtype, seed=12, junk=1.0)
    out = torch.empty_like(c["q"]).contiguous()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call(c, out=out)
    spare = c["k_cache"].shape[0] - 1
    for step in range(4):
        c["lens"] += 1
        full = c["lens"] > (c["table"] >= 0).sum(1) * 16
        c["table"][full, (c["table"] >= 0).sum(1)[full]] = spare   # (all may share it: only reads)
        c["q"].copy_(torch.randn(c["q"].shape, device=DEV))
        eager = call(c)
        call(case([300], 0, 50, seed=13))   # another call's workspace between
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        check(c, out)


def test_two_graphs_and_an_eager_call_share_nothing():
    cs = [case([1] * 20, 200, 700, H=8, Hk=1, D=128, seed=s) for s in (1, 2)]
    want, outs, graphs = [call(c) for c in cs], [torch.empty_like(c["q"]).contiguous() for c in cs], []
    for c, o in zip(cs, outs):
        g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=side):
            call(c, out=o)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(3):
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = call(cs[0])
        torch.cuda.synchronize()
        assert torch.equal(eager, want[0]) and all(torch.equal(o, w) for o, w in zip(outs, want))


def test_streams_and_threads():
    ins = [case([30, 1, 1], [0, 400, 100], 500, seed=30 + k) for k in range(3)]
    want = [call(c) for c in ins]
    torch.cuda.synchronize()
    got = [None] * 3

    def work(k):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(5):
                got[k] = call(ins[k])
        s.synchronize()
    ts = [threading.Thread(target=work, args=(k,)) for k in range(3)]
    [t.start() for t in ts]
    [t.join(60) for t in ts]
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_no_sequences_and_no_queries():
    c = case([0, 0], [5, 6], seed=14)
    assert call(c).shape == (0, 4, 64)
    c = case([3], seed=15)
    none = dict(c, q=c["q"][:0], table=c["table"][:0], lens=c["lens"][:0], cu=c["cu"][:1], cu_host=c["cu_host"][:1])
    assert call(none).shape == (0, 4, 64)


def test_a_step_as_it_is_used():
    """Prompts, then a captured step that is replayed: pages taken, rows normed, rotated and written, attention, with all
    of it against one fp64 attention over whole sequences."""
    H, Hk, D, ps, P, n, W = 8, 2, 64, 16, 70, 4, 8
    g = torch.Generator(device=DEV).manual_seed(1)
    rn = lambda *s: torch.randn(*s, device=DEV, generator=g)
    pages = 60
    kc, vc = (torch.zeros(pages, ps, Hk, D, dtype=BF, device=DEV) for _ in range(2))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    free = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).to(torch.int32).to(DEV)
    angle = torch.arange(300, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, device=DEV) / D)
    cos_sin, wq, wk = torch.cat([angle.cos(), angle.sin()], 1).float(), 0.5 + rn(D).abs(), 0.5 + rn(D).abs()
    lens, taken, table = i32([0] * n), i32([0]), torch.full((n, W), -1, dtype=torch.int32, device=DEV)
    rows = []   # every token's q, k, v by sequence: the prefix under -1

    def layer(qkv, table, lens, taken, cu, host, first, **attn):
        q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([H * D, Hk * D, Hk * D], 1))
        _, _, _, slots, positions = gdn.extend_pages(table, lens, cu, free, ps, host, first=first, taken=taken, table_out=table,
                                                     lens_out=lens, taken_out=taken)
        q, _ = gdn.qk_norm_rope(q, k, positions, cos_sin, wq, wk, v=v, k_cache=kc, v_cache=vc, slots=slots)
        return gdn.prefix_attention(q, kc, vc, table, lens, cu, host, **attn)

    width = (H + 2 * Hk) * D
    prefix, ptable, plens = rn(P, width).to(BF), torch.full((1, W), -1, dtype=torch.int32, device=DEV), i32([0])
    layer(prefix, ptable, plens, taken, i32([0, P]), torch.tensor([0, P], dtype=torch.int32), 0)
    shared = ptable[0, :-(-P // ps)].clone()
    new = [20, 0, 33, 1]
    host = torch.tensor([0, 20, 20, 53, 54], dtype=torch.int32)
    own = rn(54, width).to(BF)
    outs = [layer(own, table, lens, taken, host.to(DEV), host, P, prefix_pages=shared, prefix_len=P)]
    tokens = [[own[host[s]:host[s + 1]]] for s in range(n)]
    one = torch.arange(n + 1, dtype=torch.int32)
    qkv, dev = torch.zeros(n, width, dtype=BF, device=DEV), one.to(DEV)
    saved = [t.clone() for t in (table, lens, taken, kc, vc)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        res = layer(qkv, table, lens, taken, dev, one, P, prefix_pages=shared, prefix_len=P)
    torch.cuda.synchronize()
    for t, s in zip((table, lens, taken, kc, vc), saved):
        assert torch.equal(t, s)   # capturing ran nothing
    for _ in range(20):
        qkv.copy_(rn(n, width))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for s in range(n):
            tokens[s].append(qkv[s:s + 1].clone())
        outs.append(res.clone())
    assert lens.tolist() == [40, 20, 53, 21] and int(taken) == 5 + 3 + 2 + 4 + 2
    for s in range(n):
        seq = torch.cat([prefix] + tokens[s])
        q, k, v = (x.unflatten(1, (-1, D)) for x in seq.split([H * D, Hk * D, Hk * D], 1))
        pos = torch.arange(len(seq), device=DEV)
        # keys and queries are rounded to bf16 between the operators, as their types say
        q = ref.qk_rows(q, pos, cos_sin, wq)[0].to(BF)
        k = ref.qk_rows(k, pos, cos_sin, wk)[0].to(BF)
        m = len(seq)
        got = torch.cat([outs[0][host[s]:host[s + 1]]] + [o[s:s + 1] for o in outs[1:]]).double()
        want, mag, S, R, cnt = ref.attention(q[P:], k[None], v[None], torch.zeros(1, 1, dtype=torch.int32, device=DEV),
                                             [m], [0, m - P])
        # a bf16 rounding of q and k may fall the other way than the oracle's: then both are 2^-7 of themselves apart
        # (two halves of a step), and a score by 2 x 2^-7 S
        bound = 2 * (2 * 2.0 ** -7 * S + 2.0 ** -16)[..., None] + 2.0 ** -8 + cnt[:, None, None] * 2.0 ** -23
        allowed = bound * mag + 2.0 ** -8 * want.abs() * (1 + bound)
        assert float(((got - want).abs() / allowed).max()) <= 1.0


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes whose last pages are used."""
    free = torch.cuda.mem_get_info()[0]
    pages, ps, Hk, D = 17000, 1024, 1, 128   # 4.4 GB each
    if free < 24 << 30:
        pytest.skip("needs 24 GB")
    kc, vc = (torch.zeros(pages, ps, Hk, D, dtype=BF, device=DEV) for _ in range(2))
    c = case([3, 1], [700, 2000], 1500, H=2, Hk=1, D=D, ps=ps, seed=16, junk=1.0)
    count = c["k_cache"].shape[0]
    kc[-count:], vc[-count:] = c["k_cache"], c["v_cache"]
    far = dict(c, k_cache=kc, v_cache=vc, table=torch.where(c["table"] >= 0, c["table"] + pages - count, -1),
               prefix_pages=c["prefix_pages"] + pages - count)
    assert torch.equal(call(far), call(c))
    slots = torch.tensor([pages * ps - 1, (pages - 1) * ps], dtype=torch.int32, device=DEV)
    k = torch.randn(2, 1, D, device=DEV).to(BF)
    gdn.qk_norm_rope(k, k, torch.zeros(2, dtype=torch.int32, device=DEV), torch.cat([torch.ones(1, 64), torch.zeros(1, 64)], 1).to(DEV),
                     v=k, k_cache=kc, v_cache=vc, slots=slots)
    assert torch.equal(kc[-1, -1], k[0]) and torch.equal(vc[-1, 0], k[1])


def test_refusals():
    c = case([20, 5], [0, 30], 20, seed=17)
    bad = lambda err, **kw: pytest.raises(err, call, dict(c, **{k: kw.pop(k) for k in list(kw) if k in c}), **kw)
    bad(ValueError, q=c["q"].cpu())
    bad(ValueError, q=c["q"].half())
    bad(ValueError, k_cache=c["k_cache"].float())
    bad(ValueError, v_cache=c["v_cache"][1:])
    bad(ValueError, v_cache=c["v_cache"][:, :, :1])
    bad(ValueError, v_cache=c["v_cache"].transpose(2, 3).contiguous().transpose(2, 3))
    bad(ValueError, table=c["table"].long())
    bad(ValueError, table=c["table"][:1])
    bad(ValueError, lens=c["lens"][:1])
    bad(ValueError, prefix_pages=c["prefix_pages"][:1])
    bad(TypeError, prefix_pages=None)
    bad(ValueError, cu_host=torch.tensor([0, 20, 26], dtype=torch.int32))
    bad(ValueError, max_len=0)
    bad(ValueError, out=torch.empty(24, 4, 64, dtype=BF, device=DEV))
    bad(ValueError, workspace=torch.empty(8))
    bad(gdn.GDNError, cu_host=torch.tensor([0, 30, 25], dtype=torch.int32))
    bad(gdn.GDNError, max_len=1000)
    bad(gdn.GDNError, scale=float("nan"))
    bad(gdn.GDNError, scale=float("inf"))
    bad(gdn.GDNError, prefix_len=-1)
    bad(gdn.GDNError, out=c["q"])
    bad(gdn.GDNError, out=c["k_cache"].flatten(0, 1)[:50].reshape(-1)[:25 * 256].view(25, 4, 64))
    bad(gdn.GDNError, q=torch.empty(25, 3, 64, dtype=BF, device=DEV))
    bad(gdn.GDNError, q=torch.empty(25 * 256 + 1, dtype=BF, device=DEV)[1:].view(25, 4, 64))
    bad(gdn.GDNError, k_cache=c["k_cache"][:, :1].expand(-1, 16, -1, -1))
    bad(gdn.GDNError, q=torch.empty(25, 4, 96, dtype=BF, device=DEV), k_cache=torch.empty(9, 16, 2, 96, dtype=BF, device=DEV),
        v_cache=torch.empty(9, 16, 2, 96, dtype=BF, device=DEV))
    big = case([1], 3000, 5000, H=2, Hk=1, seed=18)
    need = torch.empty(1, dtype=torch.uint8, device=DEV)
    try:
        call(big, workspace=need)
    except gdn.GDNError as e:
        assert e.status == 5


@pytest.mark.parametrize("new,before,prefix", [([1], 3000, 5000), ([300], 0, 2000)], ids=["line", "shared"])
def test_a_workspace_that_is_too_small_is_refused(new, before, prefix):
    """Before anything runs; one of the size that is asked for is enough."""
    c = case(new, before, prefix, H=2, Hk=1, seed=18)
    want = call(c)
    shape = gdn.binding.AttnShape(len(new), 2, 1, 64, 1, *c["k_cache"].shape[:2], c["table"].shape[1], prefix, 0, 0.125, 128, 128,
                                  *c["k_cache"].stride()[:3], *c["v_cache"].stride()[:3])
    size = ctypes.c_size_t(0)
    lib = gdn.load_library()
    assert lib.gdn_prefix_attention_workspace_size(ctypes.byref(shape), c["cu_host"].data_ptr(), ctypes.byref(size)) == 0
    assert size.value > 256
    for few in (1, 255, size.value - 256, size.value - 1):
        out = torch.full_like(want, 7.0)
        with pytest.raises(gdn.GDNError) as e:
            call(c, out=out, workspace=torch.empty(few, dtype=torch.uint8, device=DEV))
        assert e.value.status == 5 and (out == 7).all()
    assert torch.equal(call(c, workspace=torch.empty(size.value, dtype=torch.uint8, device=DEV)), want)


@pytest.mark.parametrize("x", [2 ** 31, 2 ** 32, 2 ** 32 + 40, -2 ** 32 + 40, 2 ** 63])
def test_numbers_past_32_bits_are_refused(x):
    """Not taken for what their low bits are (40 tokens, pages of 40)."""
    c = case([20, 5], [0, 30], 40, seed=17)
    with pytest.raises(ValueError):
        call(c, max_len=x)
    with pytest.raises(ValueError):
        call(c, prefix_len=x)
    free = torch.arange(8, dtype=torch.int32, device=DEV)
    for kw in (dict(page_size=x), dict(page_size=16, first=x)):
        with pytest.raises(ValueError, match="32 bits"):
            gdn.extend_pages(c["table"], c["lens"], c["cu"], free, cu_seqlens_host=c["cu_host"], **kw)
