"""Calls that bring no workspace, captured into a HIP graph: the graph's memory
is its own, whatever the binding keeps, frees or replaces for eager calls
afterwards, and whatever becomes of the thread that captured it."""
import threading

import numpy as np
import pytest
import torch

import paper_2608_30310_amd as gdn
import synth
from paper_2608_30310_amd import binding
from synth.layer import LayerDims, hiddens, layer_weights, pack_hiddens
from tests.gpu_util import device_inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPE = synth.Shape(hk=2, hv=4, dk=128, dv=128, dtype="bf16")
DIMS = LayerDims(hidden=256, hk=2, hv=4, dk=64, dv=64)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    gdn.load_library()


def _tokens(seed, lens):
    return device_inputs(synth.pack([synth.tokens(600 + seed, 0, i, 0, n, SHAPE) for i, n in enumerate(lens)]))


def _layer(lens):
    x, cu = pack_hiddens([hiddens(61, 0, i, 0, n, DIMS.hidden) for i, n in enumerate(lens)], DIMS.hidden)
    bf = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16).to(DEV)
    w = {k: bf(a) if a.dtype == np.uint16 else torch.from_numpy(a).to(DEV) for k, a in layer_weights(61, 0, DIMS).items()}
    cu = torch.from_numpy(cu)
    return bf(x), w, cu.to(DEV), cu


def _calls(lens):
    """Every call that takes a workspace, each as (call(out tensors), fresh out tensors)."""
    t, s = _tokens(1, lens), _tokens(2, [n // 2 + 1 for n in lens])
    n, x, w, cu, cu_host = (len(lens),) + _layer(lens)
    states = lambda: torch.empty((n, 4, 128, 128), device=DEV)
    tail = lambda st: gdn.tail_replay(t["k"], t["v"], t["g"], t["beta"], t["cu"], t["cu_host"], state_out=st)
    fwd = lambda o, st: gdn.chunk_forward(t["q"], t["k"], t["v"], t["g"], t["beta"], t["cu"], t["cu_host"], o=o, state_out=st)
    both = lambda mid, o, st: gdn.replay_forward(
        t["k"], t["v"], t["g"], t["beta"], t["cu"], s["q"], s["k"], s["v"], s["g"], s["beta"], s["cu"],
        cu_tail_host=t["cu_host"], cu_suf_host=s["cu_host"], state_mid=mid, o=o, state_out=st)
    layer = lambda st, out: gdn.la_block_replay(x, w, cu, 2, 4, 64, 64, 0.7, cu_seqlens_host=cu_host, state_out=st, out=out)
    return [(tail, lambda: [states()]), (fwd, lambda: [torch.empty_like(t["v"]), states()]),
            (both, lambda: [states(), torch.empty_like(s["v"]), states()]),
            (layer, lambda: [torch.empty((n, 4, 64, 64), device=DEV), torch.empty_like(x)])]


@pytest.mark.parametrize("thread", [False, True])
def test_captured_calls_without_a_workspace(thread):
    small, large = _calls([150, 70]), _calls([1700, 900])
    want = []
    for call, outs in small:
        want.append(outs())
        call(*want[-1])
    torch.cuda.synchronize()
    got = [outs() for _, outs in small]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kept = []

    def capture():
        with torch.cuda.graph(graph, stream=side):
            for (call, _), out in zip(small, got):
                call(*out)
        kept.append(dict(binding._WORKSPACES.kept))

    if thread:
        t = threading.Thread(target=capture)
        t.start()
        t.join(60)
    else:
        capture()
    assert len(kept) == 1 and (0, side.cuda_stream) not in kept[0]
    for _ in range(3):
        for outs in got:
            for o in outs:
                o.zero_()
        # on the graph's stream and here: larger workspaces, and tensors where smaller ones were
        for stream in (side, torch.cuda.current_stream()):
            with torch.cuda.stream(stream):
                for call, outs in large:
                    call(*outs())
                junk = [torch.full((1 << 20,), float("nan"), device=DEV) for _ in range(8)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        del junk
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
