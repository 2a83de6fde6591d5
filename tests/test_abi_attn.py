"""The C ABI of the full-attention layer's operators and of linear attention on the
host: what they refuse before anything is enqueued, their workspace sizes, the
attention's plan and which caches share memory (no GPU).

Device pointers are placeholders that are never dereferenced: every call carries at
least one invalid argument, or has nothing to do.
"""
import ctypes
import os
import random
import shutil
import subprocess

import pytest
import torch

import paper_2608_30310_amd as gdn
from paper_2608_30310_amd.binding import AttnShape, GDN_BF16, GDN_F32, LinearShape, PagesShape, QkShape

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, SEQLENS, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5
needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(),
                                  reason="placeholder pointers are only used without a GPU")


def P(at):
    return ctypes.c_void_p(at) if at is not None else None


def ints(*x):
    return (ctypes.c_int32 * len(x))(*x)


def cu_of(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return ints(*cu)


def host_of(lens, host):
    c = cu_of(lens) if host == "lens" else host
    return c and ctypes.cast(c, ctypes.c_void_p)


def refused(status, got):
    assert got == status, gdn.load_library().gdn_last_error().decode()
    assert gdn.load_library().gdn_last_error()


# ---------------------------------------------------------------- pages
def pages_shape(n, **kw):
    return PagesShape(**dict(dict(num_seqs=n, table_width=8, page_size=16, num_free=10, first=0), **kw))


def pages(lens=(5, 3), host="lens", cu=0x1000, table=0x2000, held=0x3000, free=0x4000, taken=0x5000, table_out=0x6000,
          lens_out=0x7000, taken_out=0x8000, slots=0x9000, positions=0xa000, ws=0x10000, wsb=1 << 20, **kw):
    return gdn.load_library().gdn_extend_pages(
        ctypes.byref(pages_shape(len(lens), **kw)), host_of(lens, host), P(cu), P(table), P(held), P(free), P(taken),
        P(table_out), P(lens_out), P(taken_out), P(slots), P(positions), P(ws), wsb, None)


@needs_no_gpu
@pytest.mark.parametrize("status,kw", [
    (SHAPE, dict(num_seqs=-1)), (SHAPE, dict(num_free=-1)), (SHAPE, dict(first=-1)), (SHAPE, dict(table_width=0)),
    (SHAPE, dict(page_size=0)), (UNSUPPORTED, dict(table_width=1 << 30)), (NULL, dict(host=None)),
    (SEQLENS, dict(host=ints(0, 5, 3))), (SEQLENS, dict(host=ints(1, 5, 8))), (NULL, dict(cu=None)),
    (NULL, dict(table=None)), (NULL, dict(held=None)), (NULL, dict(free=None)), (NULL, dict(table_out=None)),
    (NULL, dict(lens_out=None)), (NULL, dict(taken_out=None)), (NULL, dict(slots=None)), (NULL, dict(positions=None)),
    (UNSUPPORTED, dict(table=0x2002)), (UNSUPPORTED, dict(taken=0x5001)), (UNSUPPORTED, dict(slots=0x9003)),
    (SHAPE, dict(table_out=0x2004)), (SHAPE, dict(lens_out=0x3004)), (SHAPE, dict(lens_out=0x2000)),
    (SHAPE, dict(taken_out=0x4000)), (SHAPE, dict(taken_out=0x1008)), (SHAPE, dict(slots=0x1000)),
    (SHAPE, dict(slots=0xa000 - 4)), (SHAPE, dict(positions=0x6000)), (SHAPE, dict(taken_out=0x7004)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(wsb=255)), (WORKSPACE, dict(ws=0x10080)),
])
def test_pages_refuse(status, kw):
    refused(status, pages(**kw))


def test_pages_workspace():
    need = ctypes.c_size_t(7)
    size = lambda lens, **kw: gdn.load_library().gdn_extend_pages_workspace_size(
        ctypes.byref(pages_shape(len(lens), **kw)), host_of(lens, "lens"), ctypes.byref(need))
    assert size(()) == 0 and need.value == 0
    assert size((1,) * 21) == 0 and need.value == 256
    assert size((0,) * 1000) == 0 and need.value == 12032
    assert size((1,), page_size=0) == SHAPE
    assert gdn.load_library().gdn_extend_pages_workspace_size(None, None, ctypes.byref(need)) == NULL
    assert gdn.load_library().gdn_extend_pages_workspace_size(ctypes.byref(pages_shape(0)), None, None) == NULL


# ---------------------------------------------------------------- norm and rotation
CACHE = dict(k_page=16 * 2 * 64, k_token=2 * 64, k_head=64, v_page=16 * 2 * 64, v_token=2 * 64, v_head=64)


def qk(q=0x1000000, k=0x2000000, v=0x3000000, positions=0x1000, cos_sin=0x100000, qw=0x2000, kw_=0x3000, slots=0x4000,
       q_out=0x4000000, k_out=0x5000000, k_cache=0x6000000, v_cache=0x7000000, null=False, **kw):
    s = dict(dict(num_tokens=9, num_heads=4, num_kv_heads=2, head_dim=64, dtype=GDN_BF16, rotary_dim=32, interleaved=0,
                  num_positions=100, eps=1e-6, num_pages=10, page_size=16, ld_q=256, ld_k=128, ld_v=128, ld_q_out=256,
                  ld_k_out=128, **CACHE), **kw)
    return gdn.load_library().gdn_qk_norm_rope(None if null else ctypes.byref(QkShape(**s)), P(q), P(k), P(v), P(positions),
                                               P(cos_sin), P(qw), P(kw_), P(slots), P(q_out), P(k_out), P(k_cache),
                                               P(v_cache), None)


@needs_no_gpu
@pytest.mark.parametrize("status,kw", [
    (NULL, dict(null=True)), (SHAPE, dict(num_tokens=-1)), (SHAPE, dict(num_heads=0)), (SHAPE, dict(num_kv_heads=0)),
    (UNSUPPORTED, dict(num_heads=70000, ld_q=1 << 23)), (UNSUPPORTED, dict(head_dim=96)), (UNSUPPORTED, dict(dtype=2)),
    (UNSUPPORTED, dict(rotary_dim=8)), (UNSUPPORTED, dict(rotary_dim=40)), (UNSUPPORTED, dict(rotary_dim=80)),
    (SHAPE, dict(interleaved=2)), (SHAPE, dict(num_positions=0)), (SHAPE, dict(eps=-1.0)), (SHAPE, dict(eps=float("nan"))),
    (SHAPE, dict(eps=float("inf"))), (SHAPE, dict(ld_q=255)), (UNSUPPORTED, dict(ld_q=257)), (UNSUPPORTED, dict(ld_k=132)),
    (UNSUPPORTED, dict(ld_v=(1 << 23) + 8)), (SHAPE, dict(ld_q_out=0)), (SHAPE, dict(ld_k_out=64)), (SHAPE, dict(num_pages=0)),
    (SHAPE, dict(page_size=0)), (UNSUPPORTED, dict(num_pages=1 << 28)), (SHAPE, dict(k_page=-64)), (SHAPE, dict(k_head=32)),
    (SHAPE, dict(k_token=64)), (SHAPE, dict(v_token=0)), (UNSUPPORTED, dict(v_page=16 * 2 * 64 + 4)),
    (UNSUPPORTED, dict(k_page=1 << 34)), (UNSUPPORTED, dict(num_pages=1 << 20, v_page=1 << 33)), (NULL, dict(q=None)), (NULL, dict(k=None)),
    (NULL, dict(positions=None)), (NULL, dict(cos_sin=None)), (NULL, dict(q_out=None)), (NULL, dict(k_out=None, k_cache=None, v=None, v_cache=None)),
    (NULL, dict(v=None)), (NULL, dict(v_cache=None)), (NULL, dict(k_cache=None)), (NULL, dict(slots=None)), (NULL, dict(qw=None)),
    (NULL, dict(kw_=None)), (UNSUPPORTED, dict(q=0x1000008)), (UNSUPPORTED, dict(v_cache=0x7000002)), (UNSUPPORTED, dict(qw=0x2004)),
    (UNSUPPORTED, dict(positions=0x1001)), (UNSUPPORTED, dict(slots=0x4002)),
    (SHAPE, dict(q_out=0x1000010)), (SHAPE, dict(q_out=0x1000000, ld_q_out=264)), (SHAPE, dict(q_out=0x2000000)),
    (SHAPE, dict(q_out=0x3000000)), (SHAPE, dict(q_out=0x100000)), (SHAPE, dict(k_out=0x1000000)), (SHAPE, dict(k_out=0x3000000)),
    (SHAPE, dict(k_out=0x4000000)), (SHAPE, dict(k_cache=0x3000000)), (SHAPE, dict(v_cache=0x1000000 - 32)),
    (SHAPE, dict(v_cache=0x6000000)), (SHAPE, dict(v_cache=0x6000000 + 64)), (SHAPE, dict(k_cache=0x5000000)),
])
def test_norm_and_rotation_refuse(status, kw):
    refused(status, qk(**kw))


def test_norm_and_rotation_of_no_tokens():
    """An empty tensor has no address."""
    assert qk(num_tokens=0, q=None, k=None, v=None, positions=None, slots=None, q_out=None, k_out=None) == 0


# ---------------------------------------------------------------- attention
def attn_shape(n, **kw):
    return AttnShape(**dict(dict(num_seqs=n, num_heads=4, num_kv_heads=2, head_dim=64, dtype=GDN_BF16, num_pages=10,
                                 page_size=16, table_width=8, prefix_len=40, max_len=0, scale=0.125, ld_q=256, ld_out=256,
                                 **CACHE), **kw))


def attn(lens=(5, 3), host="lens", cu=0x1000, q=0x1000000, k=0x2000000, v=0x3000000, table=0x2000, held=0x3000, prefix=0x4000,
         out=0x5000000, ws=0x8000000, wsb=1 << 30, **kw):
    return gdn.load_library().gdn_prefix_attention(
        ctypes.byref(attn_shape(len(lens), **kw)), host_of(lens, host), P(cu), P(q), P(k), P(v), P(table), P(held),
        P(prefix), P(out), P(ws), wsb, None)


@needs_no_gpu
@pytest.mark.parametrize("status,kw", [
    (SHAPE, dict(num_seqs=-1)), (SHAPE, dict(num_heads=0)), (SHAPE, dict(num_kv_heads=0)), (SHAPE, dict(num_kv_heads=3)),
    (UNSUPPORTED, dict(num_heads=1 << 17, ld_q=1 << 23, ld_out=1 << 23)), (UNSUPPORTED, dict(head_dim=32)),
    (UNSUPPORTED, dict(dtype=7)), (SHAPE, dict(table_width=0)), (SHAPE, dict(prefix_len=-1)), (SHAPE, dict(max_len=-1)),
    (SHAPE, dict(max_len=129)), (SHAPE, dict(scale=float("inf"))), (SHAPE, dict(scale=float("nan"))), (SHAPE, dict(ld_q=248)),
    (UNSUPPORTED, dict(ld_out=260)), (SHAPE, dict(num_pages=0)), (SHAPE, dict(page_size=0)), (UNSUPPORTED, dict(num_pages=1 << 28)),
    (UNSUPPORTED, dict(table_width=1 << 27)), (UNSUPPORTED, dict(prefix_len=1 << 30)), (SHAPE, dict(k_token=64)),
    (SHAPE, dict(v_head=0)), (UNSUPPORTED, dict(k_page=16 * 2 * 64 + 4)), (UNSUPPORTED, dict(num_pages=1 << 20, k_page=1 << 33)),
    (SEQLENS, dict(host=ints(0, 5, 3))), (SEQLENS, dict(host=ints(1, 5, 8))), (NULL, dict(host=None)), (NULL, dict(cu=None)),
    (NULL, dict(q=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(table=None)), (NULL, dict(held=None)),
    (NULL, dict(prefix=None)), (NULL, dict(out=None)), (UNSUPPORTED, dict(q=0x1000008)), (UNSUPPORTED, dict(k=0x2000004)),
    (UNSUPPORTED, dict(out=0x5000001)), (UNSUPPORTED, dict(held=0x3002)), (SHAPE, dict(out=0x1000000)),
    (SHAPE, dict(out=0x1000000 + 256)), (SHAPE, dict(out=0x2000000)), (SHAPE, dict(out=0x3000000 - 16)), (SHAPE, dict(out=0x2000 - 64)),
    (SHAPE, dict(out=0x3000)), (SHAPE, dict(out=0x4000)), (UNSUPPORTED, dict(lens=(1 << 29, 1))),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(wsb=1000)), (WORKSPACE, dict(ws=0x8000080)),
])
def test_attention_refuses(status, kw):
    refused(status, attn(**kw))


def test_attention_of_nothing():
    assert attn(lens=(), cu=None, q=None, k=None, v=None, table=None, held=None, prefix=None, out=None, ws=None) == 0
    assert attn(lens=(0, 0), q=None, out=None, ws=None) == 0


# ---------------------------------------------------------------- linear attention
def linear_shape(n, **kw):
    return LinearShape(**dict(dict(num_seqs=n, num_k_heads=2, num_v_heads=4, d_k=64, d_v=128, dtype=GDN_BF16, scale=1.0, ld_q=128,
                                   ld_k=128, ld_v=512, ld_o=512), **kw))


def linear(lens=(5, 3), host="lens", cu=0x1000, q=0x100000, k=0x200000, v=0x300000, g=0x2000, sin=None, o=0x400000,
           sout=0x500000, ws=None, wsb=0, **kw):
    return gdn.load_library().gdn_linear_attention(
        ctypes.byref(linear_shape(len(lens), **kw)), host_of(lens, host), P(cu), P(q), P(k), P(v), P(g), P(sin), P(o), P(sout),
        P(ws), wsb, None)


def linear_step(q=0x100000, k=0x200000, v=0x300000, g=0x2000, sin=None, o=0x400000, sout=0x500000, **kw):
    return gdn.load_library().gdn_linear_attention_step(ctypes.byref(linear_shape(2, **kw)), P(q), P(k), P(v), P(g), P(sin), P(o),
                                                        P(sout), None)


BAD_LINEAR = [
    (SHAPE, dict(num_k_heads=0)), (SHAPE, dict(num_v_heads=0)), (SHAPE, dict(num_k_heads=3)), (UNSUPPORTED, dict(d_k=96)),
    (UNSUPPORTED, dict(d_v=32)), (UNSUPPORTED, dict(dtype=5)), (SHAPE, dict(scale=float("nan"))), (SHAPE, dict(scale=float("-inf"))),
    (SHAPE, dict(ld_q=120)), (SHAPE, dict(ld_k=64)), (SHAPE, dict(ld_v=256)), (SHAPE, dict(ld_o=256)), (UNSUPPORTED, dict(ld_k=132)),
    (UNSUPPORTED, dict(ld_v=(1 << 23) + 8)), (UNSUPPORTED, dict(num_v_heads=1 << 17, num_k_heads=1, ld_v=1 << 23)),
    (NULL, dict(q=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(g=None)), (UNSUPPORTED, dict(k=0x200008)),
    (UNSUPPORTED, dict(o=0x400002)), (UNSUPPORTED, dict(sin=0x600004)), (UNSUPPORTED, dict(g=0x2002)),
    (SHAPE, dict(sin=0x500100)), (SHAPE, dict(o=0x100000)), (SHAPE, dict(o=0x200010)), (SHAPE, dict(o=0x300000)),
    (SHAPE, dict(o=0x500000)), (SHAPE, dict(sin=0x400000)), (SHAPE, dict(sout=0x100000)), (SHAPE, dict(sout=0x300000)),
    (SHAPE, dict(g=0x500010)), (SHAPE, dict(g=0x400010)),
]


@needs_no_gpu
@pytest.mark.parametrize("status,kw", BAD_LINEAR + [
    (SHAPE, dict(num_seqs=-1)), (NULL, dict(host=None)), (NULL, dict(cu=None)), (NULL, dict(o=None, sout=None)),
    (SEQLENS, dict(host=ints(0, 5, 3))), (WORKSPACE, dict(lens=(2000,))), (WORKSPACE, dict(lens=(2000,), ws=0x1000000, wsb=1000)),
    (WORKSPACE, dict(lens=(2000,), ws=0x1000080, wsb=1 << 30)),
])
def test_linear_attention_refuses(status, kw):
    refused(status, linear(**kw))


@needs_no_gpu
@pytest.mark.parametrize("status,kw", BAD_LINEAR + [(NULL, dict(o=None)), (NULL, dict(sout=None))])
def test_linear_step_refuses(status, kw):
    refused(status, linear_step(**kw))


@needs_no_gpu
def test_linear_states_alone_have_no_queries():
    """Without o neither q nor the strides of q and o are looked at: refused for the workspace alone."""
    assert linear(lens=(2000,), o=None, q=None, ld_q=0, ld_o=3) == WORKSPACE
    assert linear(lens=(), cu=None, k=None) == 0
    assert linear(lens=(0, 0), cu=None, k=None, v=None, q=None, o=None, sout=None) == 0


def test_calls_refuse_host_tensors():
    x = torch.zeros(2, 4, 64)
    for call in (lambda: gdn.extend_pages(x, x, [0, 2], x, 16), lambda: gdn.qk_norm_rope(x, x, x, x),
                 lambda: gdn.prefix_attention(x, x, x, x, x, [0, 2]), lambda: gdn.linear_attention(x, x, x, x, [0, 2]),
                 lambda: gdn.linear_attention_step(x, x, x, x, x), lambda: gdn.qk_norm_rope(k=x, q=x, positions=x, cos_sin=x)):
        with pytest.raises(ValueError, match="GPU memory"):
            call()


@pytest.mark.parametrize("x", [2 ** 31, 2 ** 32, 2 ** 32 + 40, -2 ** 31 - 1, -2 ** 32 + 40, 2 ** 63])
def test_numbers_are_not_cut_to_32_bits(x):
    """A field of a shape would keep the low bits of them."""
    from paper_2608_30310_amd.attn_ops import _int32
    assert AttnShape(max_len=x).max_len != x
    with pytest.raises(ValueError, match="max_len must fit 32 bits"):
        _int32(x, "max_len")
    assert [_int32(y, "max_len") for y in (-2 ** 31, 0, 2 ** 31 - 1)] == [-2 ** 31, 0, 2 ** 31 - 1]


# ---------------------------------------------------------------- the plan, built here with the host compiler
SHIM = r"""
#include "gdn_attn_plan.h"
extern "C" int attn_plan(const gdn_attn_shape* s, const int32_t* cu, int64_t* out) {
  gdn::AttnPlan p;
  std::string err;
  const int st = gdn::make_attn_plan(s, cu, &p, &err);
  const int64_t v[] = {p.rows, p.shared_splits, p.shared_chunk, p.shared_tiles, p.shared_items, p.shared_wt, p.own_tile,
                       p.own_splits, p.own_chunk, p.own_slots, p.own_items, p.stream, p.stream_first, p.stream_waves, p.grid,
                       p.joined, static_cast<int64_t>(p.off_ml), static_cast<int64_t>(p.off_line),
                       static_cast<int64_t>(p.bytes), p.max_len};
  for (unsigned i = 0; i < sizeof(v) / sizeof(v[0]); ++i) out[i] = v[i];
  return st;
}
extern "C" int apart(int64_t a, int64_t b, int64_t e, int32_t pages, int32_t ps, int32_t heads, int32_t dim, int64_t pg,
                     int64_t tk, int64_t hd) {
  return gdn::caches_apart(reinterpret_cast<void*>(a), reinterpret_cast<void*>(b), e, pages, ps, heads, dim, pg, tk, hd);
}
"""
FIELDS = ("rows shared_splits shared_chunk shared_tiles shared_items shared_wt own_tile own_splits own_chunk own_slots own_items "
          "stream stream_first stream_waves grid joined off_ml off_line bytes max_len").split()


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("attn_plan")
    src, so = d / "shim.cpp", d / "libplan.so"
    src.write_text(SHIM)
    csrc = os.path.join(ROOT, "paper_2608_30310_amd", "csrc")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"),
                    "-I", csrc, "-o", str(so), str(src)] + [os.path.join(csrc, f"gdn_{n}.cpp") for n in
                                                            ("attn_plan", "layer_plan", "plan")], check=True)
    so = ctypes.CDLL(str(so))
    so.apart.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int32] * 4 + [ctypes.c_int64] * 3
    return so


def plan_of(lib, lens, **kw):
    out = (ctypes.c_int64 * len(FIELDS))()
    s = attn_shape(len(lens), **kw)
    st = lib.attn_plan(ctypes.byref(s), cu_of(lens), out)
    return st, dict(zip(FIELDS, out)), s


@pytest.mark.parametrize("seed", range(400))
def test_plan_covers_every_key_of_every_row(lib, seed):
    """Pieces cover the prefix and the own tokens once each, the grid all items, the workspace all partial results."""
    rng = random.Random(seed)
    Hk = rng.choice([1, 2, 4, 8])
    H, D = Hk * rng.choice([1, 3, 8, 16]), rng.choice([64, 128])
    n = rng.choice([1, 2, 7, 40, 300, 1024, 1025])
    lens = [rng.choice([0, 1, 1, rng.randrange(2000 if n < 100 else 4)]) if rng.random() < 0.7 else 1 for _ in range(n)]
    if rng.random() < 0.5:
        lens = [min(x, 1) for x in lens]
    ps, width = rng.choice([1, 7, 16, 64]), rng.choice([1, 33, 500])
    prefix = rng.choice([0, 1, 63, 1000, 8192, 200000])
    st, p, s = plan_of(lib, lens, num_heads=H, num_kv_heads=Hk, head_dim=D, dtype=rng.choice([GDN_BF16, GDN_F32]), page_size=ps,
                       table_width=width, prefix_len=prefix, ld_q=H * D, ld_out=H * D, k_page=ps * Hk * D, k_token=Hk * D, k_head=D,
                       v_page=ps * Hk * D, v_token=Hk * D, v_head=D, max_len=rng.choice([0, min(width * ps, 100)]))
    assert st == 0
    G, T = H // Hk, sum(lens)
    assert p["rows"] == T * G and p["own_tile"] in (32, 128)
    if p["shared_items"]:
        assert p["shared_items"] == p["shared_tiles"] * Hk * p["shared_splits"]
        assert (p["shared_splits"] - 1) * p["shared_chunk"] < prefix <= p["shared_splits"] * p["shared_chunk"]
        assert p["shared_chunk"] % 32 == 0 and p["shared_tiles"] * 128 >= p["rows"] > (p["shared_tiles"] - 1) * 128
        assert p["shared_wt"] == 4 or (p["stream"] and p["rows"] <= 32)
    parts = p["shared_items"] * p["shared_wt"]
    if p["stream"]:
        # at most 32 rows a sequence: one wave's; every workgroup of the line is in the grid
        assert max(lens) * G <= 32 and n <= 1024 and p["joined"] and p["stream_waves"] >= Hk
        assert p["grid"] >= p["stream_first"] + -(-p["stream_waves"] // 4)
        if p["stream_first"]:
            assert p["stream_first"] * (4 if p["shared_wt"] == 1 else 1) >= p["shared_items"]
        assert prefix == 0 or T == 0 or p["shared_items"] > 0   # the line's items have no prefix (without tokens nothing runs)
        parts += 2 * p["stream_waves"] + n * Hk
        assert p["bytes"] >= p["off_line"] + 4 * (n + 1 + T)
    else:
        assert p["own_splits"] * p["own_chunk"] >= p["max_len"] and p["own_chunk"] % 64 == 0
        assert p["own_slots"] >= sum(max(1, -(-x * G // p["own_tile"])) for x in lens)
        assert p["own_items"] == p["own_slots"] * Hk * p["own_splits"] and p["grid"] == p["shared_items"] + p["own_items"]
        # the whole prefix lies before one piece of own tokens, or with the shared items
        assert p["own_splits"] == 1 or prefix == 0 or p["shared_items"] > 0
        assert p["joined"] == (p["shared_items"] > 0 or p["own_splits"] > 1)
        parts += p["own_items"] * (p["own_tile"] // 32)
    if p["joined"]:
        assert p["off_ml"] == parts * 32 * D * 4 and p["off_line"] == p["off_ml"] + parts * 32 * 8 and p["bytes"] >= p["off_line"]
    else:
        assert p["bytes"] == 0
    assert p["bytes"] % 256 == 0
    need = ctypes.c_size_t(0)
    assert gdn.load_library().gdn_prefix_attention_workspace_size(ctypes.byref(s), host_of(lens, "lens"), ctypes.byref(need)) == 0
    assert need.value == p["bytes"]


@pytest.mark.parametrize("dtype", [GDN_BF16, GDN_F32])
@pytest.mark.parametrize("n,heads,kw", [(1025, 4, {}), (4, 1025, {}), (64, 4, dict(table_width=1 << 24)), (1, 1, {}), (1024, 4, {}), (0, 4, {})],
                         ids=lambda x: str(x))
@pytest.mark.parametrize("prefix", [0, 1, 100, 200000])
def test_batches_without_queries_are_planned(lib, prefix, n, heads, kw, dtype):
    """Sequences without new tokens behind a prefix, also too many (or too many heads, or too wide a table) for a line:
    nothing to run, and no error."""
    strides = dict(k_page=16 * heads * 64, k_token=heads * 64, k_head=64, v_page=16 * heads * 64, v_token=heads * 64, v_head=64)
    kw = dict(num_heads=heads, num_kv_heads=heads, ld_q=heads * 64, ld_out=heads * 64, prefix_len=prefix, dtype=dtype, **strides, **kw)
    st, p, s = plan_of(lib, (0,) * n, **kw)
    assert st == 0 and p["rows"] == p["shared_items"] == 0
    need = ctypes.c_size_t(7)
    assert gdn.load_library().gdn_prefix_attention_workspace_size(ctypes.byref(s), host_of((0,) * n, "lens"), ctypes.byref(need)) == 0
    assert need.value == p["bytes"]
    assert attn(lens=(0,) * n, cu=None, q=None, out=None, prefix=None, ws=None, **kw) == 0


def test_caches_that_share_an_allocation(lib):
    """Two caches of the same strides: keys and values by turns, at each of the strides; and such that do meet."""
    ap = lib.apart
    shape = (10, 16, 4, 64)                       # pages, page size, heads, dim
    n = 16 * 4 * 64
    assert ap(0, 2 * 10 * n, 2, *shape, n, 256, 64)                # one behind the other
    assert not ap(0, 2 * 10 * n - 16, 2, *shape, n, 256, 64)
    assert ap(0, 2 * n, 2, *shape, 2 * n, 256, 64)                 # page by page
    assert not ap(0, 2 * n - 16, 2, *shape, 2 * n, 256, 64)
    assert ap(0, 2 * 256, 2, *shape, 2 * n, 512, 64)               # token by token
    assert ap(0, 2 * 64, 2, *shape, 2 * n, 512, 128)               # head by head
    assert not ap(0, 2 * 32, 2, *shape, 2 * n, 512, 128)
    assert not ap(0, 0, 2, *shape, n, 256, 64)
    assert ap(1 << 40, (1 << 40) + 2 * 64, 2, *shape, 2 * n, 512, 128) and ap((1 << 40) + 2 * 64, 1 << 40, 2, *shape, 2 * n, 512, 128)


@pytest.mark.parametrize("seed", range(200))
def test_caches_apart_never_share_a_byte(lib, seed):
    """Against all addresses of small caches: never apart where they meet."""
    rng = random.Random(seed)
    pages, ps, heads, dim = rng.choice([1, 2, 3]), rng.choice([1, 2, 4]), rng.choice([1, 2, 3]), 8
    order = [("p", pages), ("t", ps), ("h", heads)]
    rng.shuffle(order)
    st, at = {}, dim
    for name, count in order:
        st[name] = at * rng.choice([1, 1, 2, 3]) + 8 * rng.choice([0, 0, 1])
        at = st[name] * count
    rows = {2 * (p * st["p"] + t * st["t"] + h * st["h"] + d) for p in range(pages) for t in range(ps) for h in range(heads)
            for d in range(dim)}
    for off in range(0, 2 * at + 32, 16):
        if lib.apart(0, off, 2, pages, ps, heads, dim, st["p"], st["t"], st["h"]):
            assert not rows & {r + off for r in rows}, off
        else:
            assert off < 2 * at


def test_states_alone_need_no_more_workspace():
    """They are walked in other segments than with outputs, for which the size is given."""
    for lens in ((500,), (819,), (2048,), (1200, 64), (8192,), (819,) * 4, (64,) * 3):
        for H in (4, 32):
            need = ctypes.c_size_t(0)
            s = linear_shape(len(lens), num_v_heads=H, num_k_heads=H // 2, ld_q=64 * H // 2, ld_k=64 * H // 2, ld_v=128 * H, ld_o=128 * H)
            assert gdn.load_library().gdn_linear_attention_workspace_size(ctypes.byref(s), host_of(lens, "lens"), ctypes.byref(need)) == 0
            call = lambda wsb: gdn.load_library().gdn_linear_attention(
                ctypes.byref(s), host_of(lens, "lens"), P(0x1000), None, P(0x200000), P(0x300000), None, None, None, P(0x500000),
                P(0x1000000) if wsb else None, wsb, None)
            assert call(need.value) == NULL   # for g, which is looked at behind the workspace
