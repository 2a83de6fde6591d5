"""The layer operators' C ABI on the host: what they refuse before anything is
enqueued, their workspace sizes, the scan's choice of segments and the overlap
rules (no GPU).

Device pointers are placeholders that are never dereferenced: every call
carries at least one invalid argument, and the cases that reach past the
validation of shapes are skipped where a GPU is.
"""
import ctypes
import os
import shutil
import subprocess
import threading

import pytest
import torch

import paper_2608_30310_amd as gdn
from paper_2608_30310_amd import binding
from paper_2608_30310_amd.binding import ConvShape, GDN_BF16, GDN_F32, LAAdapters, LoraShape, SSMShape

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, SEQLENS, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5
needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(),
                                  reason="placeholder pointers are only used without a GPU")


def P(at):
    return ctypes.c_void_p(at) if at is not None else None


def cu_of(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return (ctypes.c_int32 * len(cu))(*cu)


def conv(lens=(5, 3), host="lens", x=0x100000, w=0x1000, bias=None, hin=None, y=0x200000, hout=None, cu=0x3000, **kw):
    s = dict(num_seqs=len(lens), channels=64, taps=4, dtype=GDN_BF16, activation=1, ld_x=64, ld_y=64)
    s.update(kw)
    c = cu_of(lens) if host == "lens" else host
    return gdn.load_library().gdn_causal_conv(ctypes.byref(ConvShape(**s)), c and ctypes.cast(c, ctypes.c_void_p), P(cu),
                                              P(x), P(w), P(bias), P(hin), P(y), P(hout), None)


def conv_step(x=0x100000, w=0x1000, hin=None, y=0x200000, hout=0x300000, **kw):
    s = dict(num_seqs=2, channels=64, taps=4, dtype=GDN_BF16, activation=1, ld_x=64, ld_y=64)
    s.update(kw)
    return gdn.load_library().gdn_causal_conv_step(ctypes.byref(ConvShape(**s)), P(x), P(w), None, P(hin), P(y), P(hout),
                                                   None)


def ssm_shape(n, **kw):
    s = dict(num_seqs=n, num_heads=4, num_groups=2, d_state=64, head_dim=64, dtype=GDN_BF16, dt_dtype=GDN_BF16, ld_x=256,
             ld_dt=4, ld_b=128, ld_c=128, ld_y=256)
    s.update(kw)
    return SSMShape(**s)


def scan(lens=(5, 3), host="lens", x=0x100000, dt=0x1000, a_log=0x2000, B=0x200000, C=0x300000, sin=None, y=0x400000,
         sout=0x500000, cu=0x3000, ws=None, wsb=0, **kw):
    c = cu_of(lens) if host == "lens" else host
    return gdn.load_library().gdn_ssm_scan(ctypes.byref(ssm_shape(len(lens), **kw)), c and ctypes.cast(c, ctypes.c_void_p),
                                           P(cu), P(x), P(dt), P(a_log), P(B), P(C), None, None, P(sin), P(y), P(sout),
                                           P(ws), wsb, None)


def step(x=0x100000, dt=0x1000, a_log=0x2000, B=0x200000, C=0x300000, sin=None, y=0x400000, sout=0x500000, **kw):
    return gdn.load_library().gdn_ssm_step(ctypes.byref(ssm_shape(2, **kw)), P(x), P(dt), P(a_log), P(B), P(C), None, None,
                                           P(sin), P(y), P(sout), None)


def lora(lens=(5, 3), host="lens", ids=(0, 1), cu=0x3000, dev_ids=0x4000, base=0x100000, x=0x200000, a=0x300000,
         b=0x400000, out=0x500000, ws=0x600000, wsb=1 << 20, **kw):
    s = dict(num_seqs=len(lens), num_adapters=2, hidden=64, width=96, rank=16, out_dtype=GDN_BF16, ld_x=64, ld_base=96,
             ld_out=96)
    s.update(kw)
    c = cu_of(lens) if host == "lens" else host
    i = (ctypes.c_int32 * len(ids))(*ids) if ids is not None else None
    return gdn.load_library().gdn_lora_add(ctypes.byref(LoraShape(**s)), c and ctypes.cast(c, ctypes.c_void_p), P(cu),
                                           i and ctypes.cast(i, ctypes.c_void_p), P(dev_ids), P(base), P(x), P(a), P(b),
                                           None, P(out), P(ws), wsb, None)


@needs_no_gpu
@pytest.mark.parametrize("status,kw", [
    (SHAPE, dict(num_seqs=-1)), (SHAPE, dict(channels=0)), (UNSUPPORTED, dict(taps=1)), (UNSUPPORTED, dict(taps=5)),
    (UNSUPPORTED, dict(dtype=2)), (UNSUPPORTED, dict(activation=2)), (SHAPE, dict(ld_x=63)), (SHAPE, dict(ld_y=63)),
    (UNSUPPORTED, dict(ld_x=(1 << 23) + 1)), (NULL, dict(host=None)), (NULL, dict(cu=None)), (NULL, dict(x=None)),
    (NULL, dict(y=None)), (NULL, dict(w=None)), (UNSUPPORTED, dict(x=0x100001)), (UNSUPPORTED, dict(hout=0x300001)),
    (SEQLENS, dict(host=(ctypes.c_int32 * 3)(1, 5, 8))), (SEQLENS, dict(host=(ctypes.c_int32 * 3)(0, 5, 3))),
    (SHAPE, dict(y=0x100000)), (SHAPE, dict(y=0x100000 + 64, ld_x=128, ld_y=128)), (SHAPE, dict(hout=0x100000)),
    (SHAPE, dict(hout=0x200000)), (SHAPE, dict(hin=0x300000, hout=0x300000 + 128)), (SHAPE, dict(hin=0x200000)),
])
def test_conv_refuses(status, kw):
    assert conv(**kw) == status, gdn.load_library().gdn_last_error().decode()
    assert gdn.load_library().gdn_last_error()


@needs_no_gpu
@pytest.mark.parametrize("status,kw", [
    (NULL, dict(x=None)), (NULL, dict(y=None)), (NULL, dict(w=None)), (NULL, dict(hout=None)),
    (UNSUPPORTED, dict(taps=8)), (SHAPE, dict(ld_x=3)), (SHAPE, dict(hin=0x300000 + 2)), (SHAPE, dict(y=0x300000)),
])
def test_conv_step_refuses(status, kw):
    assert conv_step(**kw) == status, gdn.load_library().gdn_last_error().decode()


@needs_no_gpu
@pytest.mark.parametrize("status,kw", [
    (SHAPE, dict(num_heads=0)), (SHAPE, dict(num_groups=3)), (UNSUPPORTED, dict(d_state=96)),
    (UNSUPPORTED, dict(head_dim=32)), (UNSUPPORTED, dict(dtype=3)), (UNSUPPORTED, dict(dtype=GDN_F32)),
    (SHAPE, dict(ld_x=255)), (UNSUPPORTED, dict(ld_x=257)), (UNSUPPORTED, dict(ld_b=132)), (SHAPE, dict(ld_c=64)),
    (SHAPE, dict(ld_dt=3)), (UNSUPPORTED, dict(ld_y=1 << 24)), (NULL, dict(host=None)), (NULL, dict(cu=None)),
    (NULL, dict(x=None)), (NULL, dict(dt=None)), (NULL, dict(a_log=None)), (NULL, dict(B=None)), (NULL, dict(C=None)),
    (NULL, dict(y=None, sout=None)), (UNSUPPORTED, dict(x=0x100008)), (UNSUPPORTED, dict(dt=0x1001)),
    (UNSUPPORTED, dict(sout=0x500008)), (SEQLENS, dict(host=(ctypes.c_int32 * 3)(0, 5, 3))),
    (SHAPE, dict(sin=0x500000 + 256)), (SHAPE, dict(y=0x100000)), (SHAPE, dict(y=0x200000)), (SHAPE, dict(y=0x300000)),
    (SHAPE, dict(y=0x500000)), (SHAPE, dict(sout=0x100000)), (SHAPE, dict(sout=0x200000)),
    (WORKSPACE, dict(lens=(2000,))), (WORKSPACE, dict(lens=(2000,), ws=0x600000, wsb=1000)),
    (WORKSPACE, dict(lens=(2000,), ws=0x600080, wsb=1 << 30)),
])
def test_scan_refuses(status, kw):
    assert scan(**kw) == status, gdn.load_library().gdn_last_error().decode()


@needs_no_gpu
@pytest.mark.parametrize("bad", [dict(ld_c=0), dict(ld_y=0), dict(ld_c=0, ld_y=0), dict(ld_c=132, ld_y=257), dict(ld_y=1 << 24)])
def test_scan_of_states_alone_has_no_rows_of_C_and_y(bad):
    """Their strides are not looked at without y: such a call is refused for its
    workspace alone, whose size does not ask for them either."""
    need = ctypes.c_size_t(0)
    size = lambda **kw: gdn.load_library().gdn_ssm_workspace_size(ctypes.byref(ssm_shape(1, **kw)), ctypes.cast(
        cu_of((2000,)), ctypes.c_void_p), ctypes.byref(need))
    assert size() == 0 and need.value > 0
    whole = need.value
    assert size(**bad) == 0 and need.value == whole
    assert scan(lens=(2000,), C=None, y=None, **bad) == WORKSPACE
    assert scan(lens=(2000,), **bad) in (SHAPE, UNSUPPORTED)
    assert step(**bad) in (SHAPE, UNSUPPORTED)
    assert scan(lens=(2000,), C=None, y=None, **dict(bad, ld_b=64)) == SHAPE


@needs_no_gpu
@pytest.mark.parametrize("kw", [dict(sin=0x600004), dict(sout=0x500008), dict(sin=0x600004, y=None, C=None)])
def test_scan_refuses_states_off_16_bytes(kw):
    assert scan(**kw) == UNSUPPORTED


@needs_no_gpu
@pytest.mark.parametrize("status,kw", [
    (NULL, dict(x=None)), (NULL, dict(y=None)), (NULL, dict(sout=None)), (NULL, dict(C=None)), (NULL, dict(a_log=None)),
    (UNSUPPORTED, dict(sin=0x500004)), (SHAPE, dict(sin=0x500010)), (SHAPE, dict(y=0x100000)),
])
def test_step_refuses(status, kw):
    assert step(**kw) == status, gdn.load_library().gdn_last_error().decode()


@needs_no_gpu
@pytest.mark.parametrize("status,kw", [
    (SHAPE, dict(num_adapters=-1)), (SHAPE, dict(width=0)), (UNSUPPORTED, dict(hidden=60)), (UNSUPPORTED, dict(rank=12)),
    (UNSUPPORTED, dict(rank=136)), (UNSUPPORTED, dict(out_dtype=5)), (SHAPE, dict(ld_x=56)), (UNSUPPORTED, dict(ld_x=68)),
    (SHAPE, dict(ld_base=95)), (SHAPE, dict(ld_out=95)), (NULL, dict(host=None)), (NULL, dict(ids=None)),
    (NULL, dict(cu=None)), (NULL, dict(dev_ids=None)), (NULL, dict(base=None)), (NULL, dict(out=None)),
    (NULL, dict(x=None)), (NULL, dict(a=None)), (NULL, dict(b=None)), (SHAPE, dict(ids=(0, 2))), (SHAPE, dict(ids=(-2, 0))),
    (UNSUPPORTED, dict(x=0x200002)), (UNSUPPORTED, dict(b=0x400008)), (UNSUPPORTED, dict(base=0x100001)),
    (SHAPE, dict(out=0x100000 + 2)), (SHAPE, dict(out=0x100000, ld_out=104)), (SHAPE, dict(out=0x200000)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(wsb=16)), (WORKSPACE, dict(ws=0x600010)),
    (SEQLENS, dict(host=(ctypes.c_int32 * 3)(0, 5, 3))),
])
def test_lora_refuses(status, kw):
    assert lora(**kw) == status, gdn.load_library().gdn_last_error().decode()


def test_nothing_to_do_is_no_error():
    """No sequences; no tokens and no history wanted; no tokens for the adapters."""
    assert conv(lens=(), cu=None, x=None, y=None, w=None) == 0
    assert conv(lens=(0, 0), cu=None, x=None, y=None, w=None) == 0
    assert scan(lens=(), cu=None, x=None) == 0
    assert lora(lens=(0, 0), base=None, x=None, out=None, ws=None) == 0
    assert lora(lens=(0, 0), ids=None, dev_ids=None, base=None, x=None, out=None, ws=None) == 0
    assert lora(lens=(), ids=(), host="lens") == 0


def test_outputs_of_no_tokens_alone_are_no_error():
    """An empty tensor of outputs has no address; without tokens there is nothing to write."""
    assert scan(lens=(0, 0), cu=None, x=None, dt=None, B=None, C=None, y=None, sout=None) == 0
    assert scan(lens=(0, 0), cu=None, x=None, dt=None, B=None, C=None, sout=None) == 0


def test_adapted_layer_workspace():
    """The adapters' workspace lies behind the layer's own."""
    lib = gdn.load_library()
    shp = binding.LAShape(1, 128, 2, 4, 64, 64, 4, GDN_BF16, 1.0, 0.0, 0.0)
    cu = cu_of([100])
    plain, adapted = ctypes.c_size_t(0), ctypes.c_size_t(0)
    c = ctypes.cast(cu, ctypes.c_void_p)
    assert lib.gdn_la_block_workspace_size(ctypes.byref(shp), c, 1, ctypes.byref(plain)) == 0
    ad = LAAdapters(2, 16, 8)
    assert lib.gdn_la_block_adapted_workspace_size(ctypes.byref(shp), ctypes.byref(ad), c, 1, ctypes.byref(adapted)) == 0
    assert adapted.value == plain.value + 100 * 16 * 4 // 256 * 256 + (256 if 100 * 16 * 4 % 256 else 0)
    for bad in (LAAdapters(2, 12, 8), LAAdapters(2, 16, 200), LAAdapters(-1, 16, 8)):
        assert lib.gdn_la_block_adapted_workspace_size(ctypes.byref(shp), ctypes.byref(bad), c, 1, ctypes.byref(adapted))
    assert lib.gdn_la_block_adapted_workspace_size(ctypes.byref(shp), None, c, 1, ctypes.byref(adapted)) == NULL


def adapted(ids=(-1, -1), ws=None, out=0x700000, **kw):
    shp = binding.LAShape(2, 128, 2, 4, 64, 64, 4, GDN_BF16, 1.0, 0.0, 0.0)
    w = binding.LAWeights(0x100000, 0x200000, 0x300000, 0x400000, 0x500000, 0x600000)
    host = (ctypes.c_int32 * 2)(*ids)
    ad = LAAdapters(**dict(dict(num_adapters=0, rank_in=16, rank_out=8, adapters_host=ctypes.addressof(host), adapters=0x800000),
                           **kw))
    return gdn.load_library().gdn_la_block_replay_adapted(
        ctypes.byref(shp), ctypes.byref(w), ctypes.byref(ad), ctypes.cast(cu_of((5, 3)), ctypes.c_void_p), P(0x900000),
        P(0xa00000), P(0xb00000), P(out), P(ws), 1 << 30, None)


@needs_no_gpu
def test_adapted_layer_looks_at_the_matrices_in_use():
    """Refused for the missing workspace alone: no adapters and no request that has
    one; matrices of a projection that is not adapted, or not run."""
    mats = dict(a_in=0x10000, b_in=0x20000, a_out=0x30000, b_out=0x40000)
    assert adapted() == WORKSPACE
    assert adapted(num_adapters=2) == WORKSPACE
    assert adapted(rank_in=0, rank_out=0, a_in=2, b_out=8) == WORKSPACE
    assert adapted(ids=(1, -1), out=None, num_adapters=2, **dict(mats, a_out=None, b_out=2)) == WORKSPACE
    assert adapted(ids=(1, -1), num_adapters=2, **mats) == WORKSPACE
    # and those that are
    assert adapted(ids=(1, -1), num_adapters=2, **dict(mats, a_in=None)) == NULL
    assert adapted(ids=(1, -1), num_adapters=2, **dict(mats, b_out=None)) == NULL
    assert adapted(ids=(1, -1), num_adapters=2, **dict(mats, b_in=0x20008)) == UNSUPPORTED
    assert adapted(ids=(0, -1)) == SHAPE
    assert adapted(adapters=None) == NULL


def test_workspaces_are_a_threads_own():
    seen = []
    t = threading.Thread(target=lambda: seen.append(binding._WORKSPACES.kept))
    t.start()
    t.join()
    assert seen[0] == {} and seen[0] is not binding._WORKSPACES.kept


def test_a_captured_call_takes_memory_of_its_own(monkeypatch):
    """Neither the workspace that is kept, which a later call or the end of its
    thread would free under the graph, nor one that is kept from then on."""
    def aligned(n, dtype, device):
        t = torch.zeros(n + 256, dtype=dtype, device=device)
        return t[-t.data_ptr() % 256:][:n]
    monkeypatch.setattr(torch, "empty", aligned)
    capturing = [False]
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: capturing[0])
    monkeypatch.setattr(binding._WORKSPACES, "kept", {})
    cpu = torch.device("cpu")
    kept = binding._workspace(1000, cpu, 7)
    assert binding._workspace(500, cpu, 7) is kept
    capturing[0] = True
    for n in (500, 1000, 5000):
        ws = binding._workspace(n, cpu, 7)
        assert ws.numel() >= n and ws is not kept
        assert binding._WORKSPACES.kept == {(None, 7): kept}
    assert binding._workspace(300, cpu, 8).numel() >= 300 and (None, 8) not in binding._WORKSPACES.kept
    capturing[0] = False
    assert binding._workspace(1000, cpu, 7) is kept


def test_adapter_indices():
    """Integers that fit 32 bits, however they come; what is rounded, cut off or contradicts itself is refused."""
    cpu = torch.device("cpu")
    ids = lambda a, host=None: binding._adapter_ids(a, host, 2, cpu)
    i32 = torch.tensor([1, -1], dtype=torch.int32)
    for a, host in ((i32, None), (i32, i32), ([1, -1], None), ((1, -1), i32), ([1, -1], torch.tensor([1, -1])), (i32, [1, -1])):
        dev, back = ids(a, host)
        assert dev.dtype == back.dtype == torch.int32 and dev.tolist() == back.tolist() == [1, -1]
    assert binding._adapter_ids([], None, 0, cpu)[1].numel() == 0
    for a, host in (([0.0, 1.9], None), ([True, False], None), ([0, 2 ** 32], None), ([0, 1], torch.tensor([2 ** 32, 1])),
                    ([0, 1], [0.5, 1]), (i32, torch.tensor([1.0, -1.0])), ([0, 1], [1, 0]), ([0, 1], i32), ([0], None),
                    (i32, [1]), ([0, -2 ** 31 - 1], None), (torch.tensor([[1, -1]]), None)):
        with pytest.raises((ValueError, TypeError)):
            ids(a, host)


def test_calls_refuse_host_tensors():
    x, w = torch.zeros(2, 8), torch.zeros(8, 4)
    for call in (lambda: gdn.causal_conv(x, w, [0, 2]), lambda: gdn.causal_conv_step(x, w),
                 lambda: gdn.ssm_scan(x, x, x, x, x, [0, 2]), lambda: gdn.ssm_step(x, x, x, x, x),
                 lambda: gdn.lora_add(x, x, x, x, [0], [0, 2]), lambda: gdn.causal_conv(None, w, [0, 2]),
                 lambda: gdn.causal_conv(weight=w, x=x, cu_seqlens=[0, 2]), lambda: gdn.causal_conv_step(weight=w)):
        with pytest.raises(ValueError, match="GPU memory"):
            call()


def test_row_checks():
    """Strides of token rows as the binding reads them."""
    from paper_2608_30310_amd.layer_ops import _rows
    cpu, f = torch.device("cpu"), torch.float32
    big = torch.zeros(6, 40)
    assert _rows(big, "x", f, cpu, (40,)) == 40
    assert _rows(big[:, 3:35], "x", f, cpu, (32,)) == 40
    assert _rows(big[:, 8:].unflatten(1, (4, 8)), "x", f, cpu, (4, 8)) == 40
    assert _rows(big[::2], "x", f, cpu, (40,)) == 80
    assert _rows(big[:1, :8], "x", f, cpu, (8,)) == 8 and _rows(big[:0, :8], "x", f, cpu, (8,)) == 8
    assert _rows(big[:, 8:16].unflatten(1, (1, 8)), "x", f, cpu, (1, 8)) == 40
    assert _rows(big[:, ::8].unsqueeze(2)[:, :1], "x", f, cpu, (1, 1)) == 40
    for t, shape in ((big[:, ::2], (20,)), (big.t(), (6,)), (big[:1].expand(6, 40), (40,)),
                     (big[:, :32].unflatten(1, (8, 4)).transpose(1, 2), (4, 8)), (big, (41,)), (big.double(), (40,))):
        with pytest.raises(ValueError):
            _rows(t, "x", f, cpu, shape)
    with pytest.raises(TypeError):
        _rows([1.0], "x", f, cpu, (1,))


# ---------------------------------------------------------------- the plan, built here with the host compiler
SHIM = r"""
#include "gdn_layer_plan.h"
extern "C" int64_t seg_tokens(const gdn_ssm_shape* s, const int32_t* cu) {
  gdn::SsmPlan p;
  std::string err;
  return gdn::make_ssm_plan(s, cu, &p, &err) == GDN_OK ? p.seg_tokens : -1;
}
extern "C" int meet(int64_t a, int64_t wa, int64_t lda, int64_t b, int64_t wb, int64_t ldb, int64_t rows) {
  return gdn::rows_overlap(reinterpret_cast<void*>(a), wa, lda, reinterpret_cast<void*>(b), wb, ldb, rows);
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("layer_plan")
    src, lib = d / "shim.cpp", d / "libplan.so"
    src.write_text(SHIM)
    csrc = os.path.join(ROOT, "paper_2608_30310_amd", "csrc")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"),
                    "-I", csrc, "-o", str(lib), str(src), os.path.join(csrc, "gdn_layer_plan.cpp"),
                    os.path.join(csrc, "gdn_plan.cpp")], check=True)
    lib = ctypes.CDLL(str(lib))
    lib.seg_tokens.restype = ctypes.c_int64
    lib.meet.argtypes = [ctypes.c_int64] * 7
    return lib


def test_segments_only_where_places_are_free(plan):
    big = dict(num_heads=64, num_groups=1, d_state=128, ld_x=4096, ld_dt=64, ld_b=128, ld_c=128, ld_y=4096)
    seg = lambda lens, **kw: plan.seg_tokens(ctypes.byref(ssm_shape(len(lens), **dict(big, **kw))), cu_of(lens))
    assert seg([819]) == 64                    # 13 chunks x 16 workgroups fit beside each other
    assert seg([32768]) == 64 * 32
    assert seg([64]) == 0 and seg([128]) == 0  # too short to pay for the states' way through memory
    assert seg([256]) == 0                     # measured: 24 us with two heads a workgroup, 28 in segments
    assert seg([512]) == 64                    # 37 us against 45
    assert seg([2048] * 16) == 0               # as many sequences as places
    assert seg([]) == 0 and seg([0, 0]) == 0
    small = dict(num_heads=4, num_groups=2, d_state=64, ld_x=256, ld_dt=4, ld_b=128, ld_c=128, ld_y=256)
    assert seg([2048], **small) == 64


def test_rows_overlap(plan):
    m = plan.meet
    assert not m(0, 100, 100, 1000, 100, 100, 10) and m(0, 100, 100, 999, 100, 100, 10)
    # columns of the same rows
    assert not m(0, 40, 100, 40, 60, 100, 10) and m(0, 40, 100, 39, 60, 100, 10)
    assert not m(40, 60, 100, 0, 40, 100, 10) and m(40, 61, 100, 0, 40, 100, 10)
    assert not m(0, 40, 100, 240, 60, 100, 10) and m(0, 41, 100, 240, 60, 100, 10)
    assert m(0, 10, 100, 50, 10, 90, 10)       # other strides: extents decide
    assert not m(0, 10, 100, 50, 10, 100, 0)
