"""Linear attention with a decay for each head, and its single-token step, against
the fp64 token-by-token form.

Bounds, as for the state space scan whose kernels these are: an element is a sum of
at most d_k + 64 products a chunk of factors that carry a few roundings, within
N32 = (d_k + 3 x 64) 2^-24 of the same sum over magnitudes; a decay over n tokens
has its exponent in 64 bits, so it is within 2^-22 at any n.  bf16 inputs go
through the matrix cores in bf16 parts: three for the states (24 bits), two for the
outputs (2^-16 each for state and products, so 2^-15).  A bf16 output is rounded
once more, by 2^-8 of itself.
"""
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


def inputs(lens, Hk=2, Hv=4, K=64, V=64, dtype="bf16", seed=0, state=True, pad=0, spare=0, slow=0.002):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rn = lambda *s: torch.randn(*s, device=DEV, generator=g)
    T = sum(lens) + spare
    row = rn(T, 2 * Hk * K + Hv * V + pad).to(BF if dtype == "bf16" else torch.float32)
    cu = torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32)
    return dict(q=row[:, :Hk * K].unflatten(1, (Hk, K)), k=row[:, Hk * K:2 * Hk * K].unflatten(1, (Hk, K)),
                v=row[:, 2 * Hk * K:2 * Hk * K + Hv * V].unflatten(1, (Hv, V)),
                g=-torch.exp(torch.linspace(0, 1, Hv, device=DEV) * 6.0) * slow, cu=cu.to(DEV), cu_host=cu,
                state=rn(len(lens), Hv, K, V) if state else None)


def call(i, **kw):
    kw = dict(dict(scale=0.3, state_in=i["state"]), **kw)
    return gdn.linear_attention(i["q"], i["k"], i["v"], i["g"], i["cu"], i["cu_host"], **kw)


def close(got, exact, mag, bound, rounding=0.0):
    off = (got.double() - exact).abs()
    allowed = bound * mag + rounding * exact.abs() * (1 + bound) + 1e-37
    worst = float((off / allowed).max()) if off.numel() else 0.0
    print(f"[linear] worst {worst:.3f} of the bound", flush=True)
    assert torch.isfinite(got.double()).all()
    assert worst <= 1.0


def check(i, o, st, scale=0.3, state="state"):
    eo, es, mo, ms = ref.linear(i["q"], i["k"], i["v"], i["g"], i["cu_host"].tolist(), scale, i[state])
    bf, T = i["v"].dtype == BF, int(i["cu_host"][-1])
    n32 = (i["k"].shape[2] + 3 * 64) * 2.0 ** -24
    if st is not None:
        close(st, es, ms, n32)
    if o is not None:
        close(o[:T], eo[:T], mo[:T], n32 + (2.0 ** -15 if bf else 0.0), 2.0 ** -8 if bf else 0.0)


LENS = [[1], [2], [15], [16], [17], [63], [64], [65], [130, 0, 1, 77], [0, 0, 5], [256, 3, 64], [33, 47, 48, 49]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", LENS, ids=lambda l: "-".join(map(str, l)))
def test_lengths(dtype, lens):
    i = inputs(lens, dtype=dtype, seed=len(lens))
    check(i, *call(i))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,V", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("Hv,Hk", [(1, 1), (3, 1), (8, 1), (8, 8), (12, 3), (6, 2)])
def test_heads(dtype, K, V, Hv, Hk):
    i = inputs([70, 9], Hk=Hk, Hv=Hv, K=K, V=V, dtype=dtype, seed=Hv)
    check(i, *call(i))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,Hv,Hk,K,V", [([1500], 2, 1, 64, 64), ([2300, 0, 40], 8, 1, 128, 64), ([1203, 1], 4, 2, 128, 128)])
def test_long(dtype, lens, Hv, Hk, K, V):
    """Sequences long enough to be worked on in several pieces, with a state that reaches the end."""
    i = inputs(lens, Hk=Hk, Hv=Hv, K=K, V=V, dtype=dtype, seed=8, slow=0.0004)
    rest = ref.linear(None, i["k"], i["v"], i["g"], i["cu_host"].tolist())[1]
    es = ref.linear(None, i["k"], i["v"], i["g"], i["cu_host"].tolist(), state=i["state"])[1]
    assert float((es - rest)[0, 0].norm() / es[0, 0].norm()) > 0.005
    check(i, *call(i))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_states_alone(dtype):
    i = inputs([300, 0, 77], dtype=dtype, seed=5, state=False)
    o, st = gdn.linear_attention(None, i["k"], i["v"], i["g"], i["cu"], i["cu_host"], outputs=False)
    assert o is None
    check(i, None, st)
    i = inputs([900, 65], dtype=dtype, seed=6)
    o, st = call(i, outputs=False)
    check(i, None, st)
    assert torch.equal(st, call(i, outputs=False)[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g", [0.0, -1e-7, -3.0, -40.0, -200.0, float("-inf")])
@pytest.mark.parametrize("lens", [[70], [1300]], ids=str)
def test_decays(dtype, g, lens):
    """No decay at all, and ones that forget everything at once (2^-150 is the least there is)."""
    i = inputs(lens, dtype=dtype, seed=7)
    i["g"] = torch.full((4,), g, device=DEV)
    check(i, *call(i))


def test_a_decay_that_is_not_a_number_stays_in_its_head():
    i = inputs([100], seed=9)
    want = call(i)
    i["g"][1] = float("nan")
    o, st = call(i)
    assert torch.isnan(st[:, 1]).all() and torch.isnan(o[:, 1].float()).all()
    for h in (0, 2, 3):
        assert torch.equal(o[:, h], want[0][:, h]) and torch.equal(st[:, h], want[1][:, h])


def test_scales():
    i = inputs([90, 20], seed=10)
    for scale in (0.0, -1.5, 1e20):
        o, st = call(i, scale=scale)
        check(i, o, st, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_spare_rows_and_in_place(dtype):
    i = inputs([100, 30], dtype=dtype, seed=11, pad=24, spare=7)
    want_o, want_s = call(i)
    rows = torch.full((137, 4 * 64 + 40), 7.0, dtype=i["v"].dtype, device=DEV)
    out = rows[:, 16:16 + 256].unflatten(1, (4, 64))
    st = i["state"].clone()
    o, s = call(i, out=out, state_in=st, state_out=st)
    assert o is out and s is st
    assert torch.equal(out[:130], want_o[:130]) and torch.equal(st, want_s)
    assert (rows[:, :16] == 7).all() and (rows[:, 272:] == 7).all() and (rows[130:] == 7).all()


def test_write_state_false_and_empty():
    i = inputs([50, 60], seed=12)
    o, st = call(i, write_state=False)
    assert st is None and torch.equal(o, call(i)[0])
    i = inputs([0, 0], seed=13)
    o, st = call(i)
    assert torch.equal(st, i["state"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,V,Hk,Hv", [(64, 64, 2, 4), (64, 128, 1, 3), (128, 64, 4, 4), (128, 128, 16, 32)])
@pytest.mark.parametrize("n", [1, 5])
def test_step(dtype, K, V, Hk, Hv, n):
    i = inputs([1] * n, Hk=Hk, Hv=Hv, K=K, V=V, dtype=dtype, seed=n, pad=8)
    o, st = gdn.linear_attention_step(i["q"], i["k"], i["v"], i["g"], state_in=i["state"], scale=0.3)
    check(i, o, st)
    s = i["state"].clone()
    o2, s2 = gdn.linear_attention_step(i["q"], i["k"], i["v"], i["g"], state_in=s, scale=0.3, state_out=s)
    assert s2 is s and torch.equal(s, st) and torch.equal(o, o2)
    o, st = gdn.linear_attention_step(i["q"], i["k"], i["v"], i["g"], scale=0.3)
    check(dict(i, state=None), o, st)


def test_a_prompt_then_tokens_is_one_sequence():
    """A tail replayed from zero, its suffix, then single tokens: the states and outputs of the whole."""
    i = inputs([150], Hk=2, Hv=4, K=128, V=128, seed=14, state=False, slow=0.01)
    cut = lambda a, b: (i["q"][a:b], i["k"][a:b], i["v"][a:b], i["g"])
    cu = lambda n: (torch.tensor([0, n], dtype=torch.int32, device=DEV), torch.tensor([0, n], dtype=torch.int32))
    q, k, v, g = cut(0, 100)
    _, st = gdn.linear_attention(None, k, v, g, *cu(100), outputs=False)
    o1, st = gdn.linear_attention(*cut(100, 140), *cu(40), scale=0.3, state_in=st)
    outs = [o1]
    for t in range(140, 150):
        o, st = gdn.linear_attention_step(*cut(t, t + 1), state_in=st, scale=0.3, state_out=st)
        outs.append(o)
    eo, es, mo, ms = ref.linear(i["q"], i["k"], i["v"], g, [0, 150], 0.3)
    n32 = 3 * (128 + 3 * 64) * 2.0 ** -24   # three calls
    close(st, es, ms, n32)
    close(torch.cat(outs), eo[100:], mo[100:], n32 + 2.0 ** -15, 2.0 ** -8)


@pytest.mark.parametrize("lens", [[200, 10], [1900]], ids=str)
def test_captured(lens):
    i = inputs(lens, Hk=4, Hv=4, K=128, seed=15)
    st, out = i["state"].clone(), torch.empty_like(i["v"]).contiguous()
    work = dict(i, state=st)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call(work, state_out=st, out=out)
        step = gdn.linear_attention_step(i["q"][:len(lens)], i["k"][:len(lens)], i["v"][:len(lens)], i["g"], state_in=st,
                                         state_out=st)[0]
    st.copy_(i["state"])
    for _ in range(3):
        o, s = call(dict(i, state=st.clone()))
        s1, s2 = gdn.linear_attention_step(i["q"][:len(lens)], i["k"][:len(lens)], i["v"][:len(lens)], i["g"], state_in=s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(st, s2) and torch.equal(step, s1)


def test_streams_and_threads():
    want, ins = [], [inputs([700, 40], seed=20 + k) for k in range(3)]
    for i in ins:
        want.append(call(i))
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
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_refusals():
    i = inputs([20, 5], seed=16)
    bad = lambda err, **kw: pytest.raises(err, call, dict(i, **{k: kw.pop(k) for k in list(kw) if k in i}), **kw)
    bad(TypeError, q=None)
    bad(TypeError, g=None)
    bad(ValueError, g=i["g"][:3])
    bad(ValueError, g=i["g"].double())
    bad(ValueError, k=i["k"][:-1])
    bad(ValueError, k=i["k"].float())
    bad(ValueError, q=i["q"].cpu())
    bad(ValueError, v=i["v"].half(), k=i["k"].half(), q=i["q"].half())
    bad(ValueError, state=i["state"][:1])
    bad(ValueError, outputs=False, out=torch.empty(25, 4, 64, dtype=BF, device=DEV))
    bad(ValueError, outputs=False, write_state=False)
    bad(ValueError, cu_host=torch.tensor([0, 20, 26], dtype=torch.int32))
    bad(gdn.GDNError, cu_host=torch.tensor([0, 30, 25], dtype=torch.int32))
    bad(gdn.GDNError, scale=float("nan"))
    bad(gdn.GDNError, scale=float("inf"))
    bad(gdn.GDNError, out=i["v"])
    wide = torch.empty(3, 4, 64, 64, device=DEV)
    bad(gdn.GDNError, state=wide[:2], state_out=wide[1:])
    bad(ValueError, workspace=torch.empty(8))
    big = inputs([3000], seed=17)
    with pytest.raises(gdn.GDNError):
        call(big, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    odd = torch.empty(25 * 4 * 64 + 1, dtype=BF, device=DEV)[1:].view(25, 4, 64)
    bad(gdn.GDNError, v=odd)
    k3 = torch.empty(25, 3, 64, dtype=BF, device=DEV)
    bad(gdn.GDNError, k=k3, q=k3)
    k48 = torch.empty(25, 2, 48, dtype=BF, device=DEV)
    bad(gdn.GDNError, k=k48, q=k48, state=None)
    with pytest.raises(ValueError):
        gdn.linear_attention_step(None, i["k"], i["v"], i["g"])
