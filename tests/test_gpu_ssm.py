"""The selective state space scan and its single-token step against the fp64
token-by-token form.

Bounds.  Everything is summed in fp32: an element of a state or an output is a
sum of at most d_state + 64 products a chunk, whose factors (decays, steps)
carry a few roundings, so it is within N32 = (d_state + 3 x 64) 2^-24 of the
same sum over magnitudes.  With bf16 inputs the fp32 factors go through the
matrix cores in bf16 parts: in the states three of them (24 bits, nothing
added), in the outputs two (within 2^-16 each for the state and for the decayed
products, so 2^-15).  A bf16 output is rounded once more, by 2^-8 of itself.
"""
import threading

import pytest
import torch

import paper_2608_30310_amd as gdn
from oracle import layer_ops as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    gdn.load_library()


def inputs(lens, H=4, G=2, N=64, P=64, dtype="bf16", seed=0, state=True, dt32=False, pad=0, spare=0):
    """A layer's tensors as views of the rows they stand in; `spare` rows behind the last sequence."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt_ = torch.bfloat16 if dtype == "bf16" else torch.float32
    rn = lambda *s: torch.randn(*s, device=DEV, generator=g)
    T = sum(lens) + spare
    row = rn(T, H * P + 2 * G * N + pad).to(dt_)
    x = row[:, :H * P].unflatten(1, (H, P))
    B = row[:, H * P:H * P + G * N].unflatten(1, (G, N))
    C = row[:, H * P + G * N:H * P + 2 * G * N].unflatten(1, (G, N))
    dt = rn(T, H + 3).to(torch.float32 if dt32 else dt_)[:, 1:1 + H]
    cu = torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32)
    return dict(x=x, dt=dt, B=B, C=C, a_log=torch.log(1 + 15 * torch.rand(H, device=DEV, generator=g)),
                d_skip=rn(H), dt_bias=rn(H) * 0.5 - 3.0, cu=cu.to(DEV), cu_host=cu,
                state=rn(len(lens), H, N, P) if state else None)


def scan(i, **kw):
    kw = dict(dict(d_skip=i["d_skip"], dt_bias=i["dt_bias"], state_in=i["state"]), **kw)
    return gdn.ssm_scan(i["x"], i["dt"], i["a_log"], i["B"], i["C"], i["cu"], i["cu_host"], **kw)


def want(i, **kw):
    kw = dict(dict(d_skip=i["d_skip"], dt_bias=i["dt_bias"], state=i["state"]), **kw)
    return ref.ssm(i["x"], i["dt"], i["a_log"], i["B"], i["C"], i["cu_host"].tolist(), **kw)


def n32(i):
    return (i["B"].shape[2] + 3 * 64) * 2.0 ** -24


def close(got, exact, mag, bound, rounding=0.0):
    """|got - exact| <= bound mag + rounding |exact|, element by element."""
    off = (got.double() - exact).abs()
    allowed = bound * mag + rounding * exact.abs() * (1 + bound) + 1e-37
    worst = float((off / allowed).max()) if off.numel() else 0.0
    print(f"[ssm] worst {worst:.3f} of the bound", flush=True)
    assert torch.isfinite(got.double()).all()
    assert worst <= 1.0


def check(i, y, st):
    ey, es, my, ms = want(i)
    T = int(i["cu_host"][-1])
    bf = i["x"].dtype == torch.bfloat16
    if st is not None:
        close(st, es, ms, n32(i))
    if y is not None:
        close(y[:T], ey[:T], my[:T], n32(i) + (2.0 ** -15 if bf else 0.0), 2.0 ** -8 if bf else 0.0)


LENS = [[1], [2], [63], [64], [65], [130, 0, 1, 77], [0, 0, 5], [256, 3, 64]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", LENS, ids=lambda l: "-".join(map(str, l)))
def test_lengths(dtype, lens):
    i = inputs(lens, dtype=dtype, seed=len(lens))
    check(i, *scan(i))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,P", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("H,G", [(1, 1), (3, 1), (8, 1), (8, 8), (12, 3), (6, 2)])
def test_heads(dtype, N, P, H, G):
    i = inputs([70, 9], H=H, G=G, N=N, P=P, dtype=dtype, seed=H, dt32=dtype == "bf16" and H == 3)
    check(i, *scan(i))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_state_no_skip_no_bias(dtype):
    i = inputs([100, 33], dtype=dtype, seed=3, state=False)
    i.update(d_skip=None, dt_bias=None)
    check(i, *scan(i))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,H,G,N,P", [([1500], 2, 1, 64, 64), ([2300, 0, 40], 8, 1, 128, 64), ([1200, 1], 4, 2, 128, 128)])
def test_long(dtype, lens, H, G, N, P):
    """Sequences long enough to be worked on in several pieces."""
    i = inputs(lens, H=H, G=G, N=N, P=P, dtype=dtype, seed=8)
    check(i, *scan(i))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slow_decay_carries_the_first_state_to_the_end(dtype):
    """Steps so small that a piece's start still weighs at its end."""
    i = inputs([1700], H=4, G=1, N=128, P=64, dtype=dtype, seed=9)
    i["dt_bias"] = torch.full((4,), -9.0, device=DEV)
    i["a_log"] = torch.zeros(4, device=DEV)
    ey, es, my, ms = want(i)
    rest = want(dict(i, state=None))[1]
    assert float((es - rest).norm() / es.norm()) > 0.2
    check(i, *scan(i))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_that_forget_everything(dtype):
    """Steps of up to 200 (decays far below the least fp32 value) beside tiny ones."""
    i = inputs([150], H=4, G=2, dtype=dtype, seed=4, dt32=True)
    i["dt"] = torch.where(torch.rand(150, 4, device=DEV, generator=torch.Generator(DEV).manual_seed(1)) < 0.1, 200.0, -8.0)
    i["dt_bias"] = None
    check(i, *scan(i))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("steps", ["3 each", "10 each", "8 of 5", 7, 12, 15])
@pytest.mark.parametrize("length,N,P", [(200, 64, 64), (200, 128, 128), (1500, 128, 64)])
def test_short_decays_after_long_ones(dtype, steps, length, N, P):
    """Tokens that forget nearly everything, and ordinary ones behind them in the
    same 16 tokens: the decays between the ordinary ones are sums of few short
    steps, whatever came before.  x, B and C are positive, so that every output is
    its own sum over magnitudes and the bound is one on its relative error.
    `steps`: softplus(dt) of about 3 or 10 everywhere (a decay of e^-48 or e^-160 a
    token); of each 16 tokens the first 8 of about 5; the first 7, 12 or 15 of 200."""
    i = inputs([length], H=4, G=2, N=N, P=P, dtype=dtype, seed=28, state=False, dt32=True)
    noise = torch.randn(length, 4, device=DEV, generator=torch.Generator(DEV).manual_seed(29))
    place = (torch.arange(length, device=DEV) % 16)[:, None]
    if isinstance(steps, int):
        dt = torch.where(place < steps, 200.0, noise - 1.5)
    elif steps == "8 of 5":
        dt = torch.where(place < 8, noise + 5.0, noise - 3.0)
    else:
        dt = noise + float(steps.split()[0])
    i.update(x=i["x"].abs(), B=i["B"].abs(), C=i["C"].abs(), dt=dt, dt_bias=None, d_skip=None,
             a_log=torch.full((4,), 16.0, device=DEV).log())
    y, st = scan(i)
    ey, _, my, _ = want(i)
    assert torch.allclose(ey, my, rtol=1e-12)
    check(i, y, st)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [150, 1500])
def test_steps_of_nothing_and_of_everything(dtype, length):
    """Tokens whose step is masked out (dt of -infinity or near it: delta is zero)
    beside ones with enormous steps; one head has no other tokens than masked ones."""
    i = inputs([length, 3], H=4, G=2, dtype=dtype, seed=30, dt32=True)
    g = torch.Generator(DEV).manual_seed(31)
    kinds = torch.tensor([-float("inf"), -1e30, -90.0, 0.0, 90.0, 1e4], device=DEV)
    i["dt"] = kinds[torch.randint(0, 6, (length + 3, 4), device=DEV, generator=g)]
    i["dt"][:, 1] = -float("inf")
    y, st = scan(i)
    check(i, y, st)
    assert torch.equal(st[:, 1], i["state"][:, 1])
    one = dict(i, x=i["x"][:2], B=i["B"][:2], C=i["C"][:2], dt=i["dt"][:2], cu_host=torch.tensor([0, 1, 2]))
    check(one, *gdn.ssm_step(one["x"], one["dt"], i["a_log"], one["B"], one["C"], d_skip=i["d_skip"], dt_bias=i["dt_bias"],
                             state_in=i["state"]))


def test_all_outputs_choices_agree():
    """Outputs alone, states alone and both are the same numbers; so is a state updated in place."""
    for lens in ([100, 65], [1500]):
        i = inputs(lens, H=4, G=1, N=128, seed=6)
        y, st = scan(i)
        assert torch.equal(scan(i, write_state=False)[0], y)
        none, st2 = gdn.ssm_scan(i["x"], i["dt"], i["a_log"], i["B"], None, i["cu"], i["cu_host"],
                                 dt_bias=i["dt_bias"], state_in=i["state"], outputs=False)
        assert none is None
        check(i, None, st2)
        s = i["state"].clone()
        y3, st3 = scan(i, state_in=s, state_out=s)
        assert st3 is s and torch.equal(y3, y) and torch.equal(st3, st)


def test_repeats_bitwise_and_sequences_do_not_meet():
    i = inputs([90, 200, 31], H=6, G=2, seed=7)
    y, st = scan(i)
    for _ in range(3):
        y2, st2 = scan(i)
        assert torch.equal(y, y2) and torch.equal(st, st2)
    # the middle sequence ruined: its neighbours keep every bit
    bad = dict(i, x=i["x"].clone(), B=i["B"].clone(), C=i["C"].clone(), dt=i["dt"].clone(), state=i["state"].clone())
    for k in ("x", "B", "C", "dt"):
        bad[k][90:290] = float("nan")
    bad["x"][95] = float("inf")
    bad["state"][1] = float("nan")
    y3, st3 = scan(bad)
    for a, b in ((y, y3),):
        assert torch.equal(a[:90], b[:90]) and torch.equal(a[290:], b[290:])
    assert torch.equal(st[0], st3[0]) and torch.equal(st[2], st3[2])
    assert torch.isnan(y3[90:290]).all()


def test_rows_behind_the_last_sequence_are_left():
    i = inputs([70, 30], seed=5, spare=37, pad=24)
    for k in ("x", "B", "C", "dt"):
        i[k][100:] = float("nan")
    rows = torch.full((137, 4 * 64 + 40), 3.0, dtype=torch.bfloat16, device=DEV)
    y, st = scan(i, out=rows[:, 16:16 + 256].unflatten(1, (4, 64)))
    check(i, y, st)
    assert (rows[100:] == 3.0).all() and (rows[:, :16] == 3.0).all() and (rows[:, 272:] == 3.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cut", [1, 64, 100])
def test_continues_from_its_state(dtype, cut):
    i = inputs([200], H=4, G=2, N=128, dtype=dtype, seed=11)
    part = lambda a, b, st: gdn.ssm_scan(i["x"][a:b], i["dt"][a:b], i["a_log"], i["B"][a:b], i["C"][a:b], [0, b - a],
                                         d_skip=i["d_skip"], dt_bias=i["dt_bias"], state_in=st)
    y1, s1 = part(0, cut, i["state"])
    y2, s2 = part(cut, 200, s1)
    check(i, torch.cat([y1, y2]), s2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,P", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("H,G", [(1, 1), (6, 2)])
def test_step(dtype, N, P, H, G):
    """One token per sequence is the scan of sequences of one token."""
    i = inputs([1] * 5, H=H, G=G, N=N, P=P, dtype=dtype, seed=12)
    y, st = gdn.ssm_step(i["x"], i["dt"], i["a_log"], i["B"], i["C"], d_skip=i["d_skip"], dt_bias=i["dt_bias"],
                         state_in=i["state"])
    check(i, y, st)
    s = i["state"].clone()
    y2, s2 = gdn.ssm_step(i["x"], i["dt"], i["a_log"], i["B"], i["C"], d_skip=i["d_skip"], dt_bias=i["dt_bias"],
                          state_in=s, state_out=s)
    assert s2 is s and torch.equal(y2, y) and torch.equal(s2, st)
    i.update(state=None, d_skip=None, dt_bias=None)
    check(i, *gdn.ssm_step(i["x"], i["dt"], i["a_log"], i["B"], i["C"]))


def test_steps_after_a_scan():
    i = inputs([80], H=4, G=1, N=128, seed=13)
    y, st = gdn.ssm_scan(i["x"][:70], i["dt"][:70], i["a_log"], i["B"][:70], i["C"][:70], [0, 70], d_skip=i["d_skip"],
                         dt_bias=i["dt_bias"], state_in=i["state"])
    ys = [y]
    for t in range(70, 80):
        r = slice(t, t + 1)
        y, st = gdn.ssm_step(i["x"][r], i["dt"][r], i["a_log"], i["B"][r], i["C"][r], d_skip=i["d_skip"],
                             dt_bias=i["dt_bias"], state_in=st, state_out=st)
        ys.append(y)
    check(i, torch.cat(ys), st)


@pytest.mark.parametrize("lens", [[90, 40], [1500]])
def test_graph_replays(lens):
    """A captured scan and step, replayed between eager work of other sizes."""
    i = inputs(lens, H=4, G=1, N=128, seed=14)
    y0, s0 = scan(i)
    y, st = torch.empty_like(y0), torch.empty_like(s0)
    one = inputs([1] * 3, H=4, G=1, N=128, seed=15)
    step = lambda **kw: gdn.ssm_step(one["x"], one["dt"], one["a_log"], one["B"], one["C"], state_in=one["state"], **kw)
    sy0, ss0 = step()
    sy, ss = torch.empty_like(sy0), torch.empty_like(ss0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        scan(i, out=y, state_out=st)
        step(out=sy, state_out=ss)
    for k in range(3):
        for t in (y, st, sy, ss):
            t.zero_()
        graph.replay()
        other = inputs([3000 + 100 * k], H=4, G=1, N=128, seed=20 + k)
        scan(other)
        torch.cuda.synchronize()
        assert torch.equal(y, y0) and torch.equal(st, s0) and torch.equal(sy, sy0) and torch.equal(ss, ss0)


def test_two_streams_at_once():
    """Calls on two streams keep to workspaces of their own."""
    a, b = inputs([1500], H=4, G=1, N=128, seed=16), inputs([1800], H=4, G=1, N=128, seed=17)
    ya, sa = scan(a)
    yb, sb = scan(b)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(4):
        with torch.cuda.stream(s1):
            got.append((scan(a), ya, sa))
        with torch.cuda.stream(s2):
            got.append((scan(b), yb, sb))
    torch.cuda.synchronize()
    for (y, s), wy, ws in got:
        assert torch.equal(y, wy) and torch.equal(s, ws)


def test_two_threads_on_one_stream():
    """Launches of two threads' calls may take turns on a stream: each has a workspace of its own."""
    both = [inputs([1500], H=4, G=1, N=128, seed=26), inputs([1800], H=4, G=1, N=128, seed=27)]
    want_ = [scan(i) for i in both]
    torch.cuda.synchronize()
    got = [[], []]

    def work(k):
        for _ in range(40):
            got[k].append(scan(both[k]))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    torch.cuda.synchronize()
    for k in range(2):
        assert len(got[k]) == 40
        for y, s in got[k]:
            assert torch.equal(y, want_[k][0]) and torch.equal(s, want_[k][1])


def test_many_sequences():
    """More sequences than a wave has lanes, with one long enough for segments among them."""
    i = inputs([3] * 100 + [1500] + [0] * 40 + [200, 1], H=4, G=1, N=64, seed=19)
    check(i, *scan(i))


@pytest.mark.parametrize("N", [64, 128])
def test_as_many_sequences_as_places(N):
    """Heads of a workgroup by fours where there are enough sequences, by twos where there are few."""
    i = inputs([70] * 39 + [130], H=16, G=2, N=N, seed=23)
    y, st = scan(i)
    check(i, y, st)
    one = inputs([130], H=16, G=2, N=N, seed=24)
    check(one, *scan(one))


@pytest.mark.parametrize("n", [13, 20, 64, 65])
@pytest.mark.parametrize("H,G,P", [(64, 1, 64), (32, 8, 64), (32, 16, 128)])
def test_more_sequences_than_places(n, H, G, P):
    """Ragged batches whose workgroups do not fit at once: the longest start first."""
    some = [200, 3, 0, 64, 65, 1, 130, 17, 2, 80, 5, 9, 33]
    lens = [some[k % 13] if k < 13 else (7 * k) % 40 for k in range(n)]
    i = inputs(lens, H=H, G=G, N=64, P=P, seed=n, spare=2)
    check(i, *scan(i))


def test_arguments_by_name():
    i = inputs([40, 30], seed=25)
    y, st = scan(i)
    y2, st2 = gdn.ssm_scan(cu_seqlens=i["cu"], C=i["C"], B=i["B"], a_log=i["a_log"], dt=i["dt"], x=i["x"], d_skip=i["d_skip"],
                           dt_bias=i["dt_bias"], state_in=i["state"])
    assert torch.equal(y, y2) and torch.equal(st, st2)


def test_a_head_without_a_number():
    """A decay that is not a number makes that head's outputs and states so, and no other's."""
    i = inputs([70, 1500], H=4, G=2, seed=21)
    y, st = scan(i)
    bad = dict(i, a_log=i["a_log"].clone())
    bad["a_log"][2] = float("nan")
    y2, st2 = scan(bad)
    keep = [0, 1, 3]
    assert torch.equal(y[:, keep], y2[:, keep]) and torch.equal(st[:, keep], st2[:, keep])
    assert torch.isnan(st2[:, 2]).all() and torch.isnan(y2[1:, 2][:60]).all()
    y3, st3 = gdn.ssm_step(i["x"][:2], i["dt"][:2], bad["a_log"], i["B"][:2], i["C"][:2], state_in=i["state"])
    assert torch.isnan(st3[:, 2]).all() and torch.isfinite(st3[:, keep]).all()


def test_refuses():
    i = inputs([5, 3], seed=22)
    x, dt, a, B, C = (i[k] for k in ("x", "dt", "a_log", "B", "C"))
    for bad in (dict(x=x[:, :3]), dict(B=B[:, :1]), dict(C=C[:7]), dict(dt=dt.double()), dict(dt=dt[:, :3]), dict(a_log=a[:3]),
                dict(x=x.half()), dict(d_skip=a.bfloat16()), dict(dt_bias=a[:1]), dict(state_in=torch.zeros(2, 4, 64, 32, device=DEV)),
                dict(state_in=torch.zeros(3, 4, 64, 64, device=DEV)), dict(cu=[0, 5, 9]), dict(out=torch.empty(8, 4, 64, device=DEV)),
                dict(out=torch.empty(7, 4, 64, dtype=x.dtype, device=DEV)), dict(x=x.cpu()), dict(a_log=a.cpu()), dict(C=None),
                dict(outputs=False, out=torch.empty_like(x)), dict(workspace=torch.empty(8))):
        kw = dict(dict(x=x, dt=dt, a_log=a, B=B, C=C, cu=i["cu_host"].tolist()), **bad)
        first = [kw.pop(k) for k in ("x", "dt", "a_log", "B", "C", "cu")]
        with pytest.raises((ValueError, TypeError)):
            gdn.ssm_scan(*first, **kw)
    for cu in ([1, 5, 8], [0, 6, 3, 8]):
        with pytest.raises(gdn.GDNError):
            gdn.ssm_scan(x, dt, a, B, C, cu)
    with pytest.raises(gdn.GDNError):   # rows that do not start at 16 bytes
        big = torch.zeros(8, 4 * 64 + 8, dtype=x.dtype, device=DEV)
        gdn.ssm_scan(big[:, 4:260].unflatten(1, (4, 64)), dt, a, B, C, i["cu"])
    with pytest.raises(gdn.GDNError):   # in place over x
        y = x.contiguous()
        gdn.ssm_scan(y, dt, a, B, C, i["cu"], out=y)


def test_no_tokens():
    i = inputs([0, 0], seed=18)
    y, st = scan(i)
    assert y.shape == (0, 4, 64) and torch.equal(st, i["state"])
    i = inputs([0, 0], seed=18, state=False)
    assert not scan(i)[1].any()


def test_outputs_of_no_tokens_alone():
    i = inputs([0, 0], seed=18)
    y, st = scan(i, write_state=False)
    assert y.shape == (0, 4, 64) and st is None
