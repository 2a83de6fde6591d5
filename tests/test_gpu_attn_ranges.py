"""The full-attention layer's operators at the ends of their ranges: many rows and many
sequences, batches of both kinds, outputs that are an input in part, caches whose rows lie
far apart, values near the largest (bounds as in the tests of each operator).
"""
import random

import pytest
import torch

import paper_2608_30310_amd as gdn
from tests import test_gpu_attn as attn
from tests import test_gpu_pages as pages

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
DT = pytest.mark.parametrize("dtype", ["bf16", "f32"])


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    gdn.load_library()


@DT
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R,T", [(64, 64, 4000), (128, 96, 2000)])
def test_qk_of_many_rows(dtype, interleaved, D, R, T):
    """So many that a wave takes several rows of a token; 43 head rows are no multiple of them."""
    c = pages.qk_case(T, 33, 5, D, R, dtype, seed=R)
    q, _ = pages.into(c, interleaved=interleaved)
    pages.check_qk(c, q, interleaved=interleaved)
    args = (c["positions"], c["cos_sin"], c["q_weight"], c["k_weight"])
    q2, k2 = gdn.qk_norm_rope(c["q"], c["k"], *args, interleaved=interleaved)   # no values: 38 rows
    assert torch.equal(q, q2) and torch.equal(k2, pages.flat(c["k_cache"])[c["slots"].long()])
    c["positions"][::3] = -1   # rows of tokens that are skipped stay
    keep = q2.clone()
    out, _ = gdn.qk_norm_rope(c["q"], c["k"], *args, interleaved=interleaved, q_out=torch.zeros_like(q2))
    assert (out[::3] == 0).all() and torch.equal(out[1::3], keep[1::3])


@pytest.mark.parametrize("which", ["table_out", "lens_out", "taken_out"])
@pytest.mark.parametrize("n", [5, 700, 1024])
def test_pages_with_one_output_in_place(which, n):
    gen = torch.Generator().manual_seed(n)
    held, new = torch.randint(0, 100, (n,), generator=gen).tolist(), torch.randint(0, 4, (n,), generator=gen).tolist()
    c = pages.pages_case(held, new, 16, 8, seed=n, taken=3)
    t = torch.tensor(c["table"], dtype=torch.int32, device=DEV)
    ins = dict(table_out=t, lens_out=pages.i32(c["lens"]), taken_out=pages.i32([3]))
    got = gdn.extend_pages(t, ins["lens_out"], pages.i32(c["cu"]), pages.i32(c["free"]), 16,
                           torch.tensor(c["cu"], dtype=torch.int32), taken=ins["taken_out"], **{which: ins[which]})
    pages.check_pages(c, got)
    if which != "lens_out":
        assert ins["lens_out"].tolist() == c["lens"]
    if which != "taken_out":
        assert ins["taken_out"].tolist() == [3]


@DT
@pytest.mark.parametrize("n", [1024, 1025, 2000])
@pytest.mark.parametrize("prefix", [0, 100])
def test_single_tokens_of_many_sequences(dtype, n, prefix):
    c = attn.case([1] * n, [i * 7 % 50 for i in range(n)], prefix, dtype=dtype, seed=n)
    attn.check(c, attn.call(c))


@DT
def test_prompts_and_single_tokens_in_one_batch(dtype):
    c = attn.case([1, 300, 1, 1, 0, 40, 1], [2000, 0, 5, 0, 9, 700, 33], 260, H=8, Hk=2, D=128, dtype=dtype, seed=1)
    attn.check(c, attn.call(c))


@DT
@pytest.mark.parametrize("ps", [8, 24, 32, 112])
@pytest.mark.parametrize("D", [64, 128])
def test_page_sizes_beside_the_tiles(dtype, ps, D):
    """Pages that hold whole DMAs of rows but not a wave's part of a tile, and such that do; tiles over several pages."""
    c = attn.case([70, 1, 130], [10, 200, 0], 200, ps=ps, D=D, dtype=dtype, seed=ps)
    attn.check(c, attn.call(c))
    c = attn.case([1, 1, 1], [10, 200, 700], 200, ps=ps, D=D, dtype=dtype, seed=ps)
    attn.check(c, attn.call(c))


@DT
def test_invalid_pages_in_prompts(dtype):
    """Some of a tile's pages are none: each wave's part, the first, the last, all of a tile."""
    c = attn.case([150, 90], [100, 0], 300, ps=16, dtype=dtype, seed=3)
    for n, at in ((0, 0), (0, 3), (0, 5), (0, 8), (0, 9), (0, 10), (0, 11), (1, 1)):
        c["table"][n, at] = [-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1][at % 4]
    c["prefix_pages"][[0, 7, 18]] = torch.tensor([-1, 10 ** 6, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    attn.check(c, attn.call(c))


@DT
def test_scores_that_rise_all_the_way(dtype):
    """Every tile's scores lie above the last one's: small steps, which leave the maximum behind by less than the
    bound that it is kept to, and large ones."""
    for top in (2.0, 12.0, 60.0):
        c = attn.case([64, 1], [1500, 1500], 500, dtype=dtype, seed=5)
        c["q"].copy_(torch.ones_like(c["q"]) * 0.25)
        ps, k = 16, c["k_cache"].reshape(-1, 2, 64)
        order = [c["prefix_pages"].long()[torch.arange(500, device=DEV) // ps] * ps + torch.arange(500, device=DEV) % ps]
        own = torch.arange(1501, device=DEV)
        for n, m in ((0, 1564), (1, 1501)):
            own = torch.arange(m, device=DEV)
            rows = torch.cat(order + [c["table"][n].long()[own // ps] * ps + own % ps])
            k[rows] = (torch.linspace(0, top, len(rows), device=DEV)[:, None, None] / 2).expand(-1, 2, 64).to(k.dtype)
        c["k_cache"].copy_(k.view_as(c["k_cache"]))
        attn.check(c, attn.call(c))


@DT
@pytest.mark.parametrize("low", [3.0, 5.4, 7.0, 40.0])
def test_a_first_tile_far_below_the_rest(dtype, low):
    """All other scores lie `low` above the first tile's (5.5: 2^8 of its weights), in some rows alone."""
    c = attn.case([100, 1, 1], [700, 900, 3], 200, dtype=dtype, seed=8)
    c["q"].mul_(0.02)
    c["q"][..., 0] = torch.where(torch.arange(102, device=DEV) % 3 > 0, 8.0, 0.0)[:, None].to(c["q"].dtype)   # scale 2^-3
    rows = torch.arange(64, device=DEV)
    flat = c["k_cache"].reshape(-1, 2, 64)
    flat[..., 0] = low
    flat[c["prefix_pages"].long()[rows // 16] * 16 + rows % 16, :, 0] = 0.0
    c["k_cache"].copy_(flat.view_as(c["k_cache"]))
    attn.check(c, attn.call(c))


@DT
def test_values_near_the_largest(dtype):
    """Weights stay below 2^8, so values of 2^100 do not leave the range."""
    for new, before in (([100], 900), ([1, 1], 900)):
        c = attn.case(new, before, 300, dtype=dtype, seed=6, size=3.0)
        c["v_cache"].mul_(2.0 ** 100)
        attn.check(c, attn.call(c))


@pytest.mark.parametrize("new", [[70], [1, 1]])
def test_rows_of_a_page_far_apart(new):
    """Token strides of 2^28 bytes: the offset of a DMA's rows does not fit 32 bits."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    c = attn.case(new, [20] * len(new), 30, H=4, Hk=2, D=64, ps=16, seed=7)
    count, step = c["k_cache"].shape[0], 2 ** 27   # elements
    assert 16 * count <= 4096
    big = torch.zeros(15 * step + count * 4 * 64, dtype=BF, device=DEV)
    far = lambda kv: torch.as_strided(big, (count, 16, 2, 64), (256, step, 64, 1), kv * 128)
    far(0).copy_(c["k_cache"])
    far(1).copy_(c["v_cache"])
    assert torch.equal(attn.call(dict(c, k_cache=far(0), v_cache=far(1))), attn.call(c))


@pytest.mark.parametrize("seed", range(40))
def test_whatever_the_workspace_held(seed):
    """Batches drawn over the ranges, on a workspace full of NaN; some entries of the tables are no pages."""
    rng = random.Random(seed)
    Hk = rng.choice([1, 2, 3, 4, 8])
    H, D = Hk * rng.choice([1, 2, 5, 8]), rng.choice([64, 128])
    n = rng.choice([1, 2, 5, 30])
    new = [rng.choice([0, 1, 1, 2, rng.randrange(1, 150)]) for _ in range(n)] if rng.random() < 0.6 else [1] * n
    before = [rng.choice([0, 1, 31, 64, rng.randrange(600)]) for _ in range(n)]
    dtype, ps = rng.choice(["bf16", "f32"]), rng.choice([1, 5, 16, 24, 64, 128])
    c = attn.case(new, before, rng.choice([0, 0, 1, 100, 640]), H=H, Hk=Hk, D=D, ps=ps, dtype=dtype, seed=seed,
                  layout=rng.choice(["pages", "heads", "both", "rows"]), pad=rng.choice([0, 8]), spare=rng.choice([0, 3]))
    if rng.random() < 0.4:
        for _ in range(3):
            c["table"][rng.randrange(n), rng.randrange(c["table"].shape[1])] = rng.choice([-1, 2 ** 31 - 1])
    kw = dict(scale=rng.choice([None, 0.05, -0.3]))
    if rng.random() < 0.3:
        kw["max_len"] = rng.randrange(1, c["table"].shape[1] * ps + 1)
        c["lens"].clamp_(max=kw["max_len"])   # (a bound that holds)
    ws = torch.full((64 << 20,), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.full_like(c["q"], 7.0).contiguous()
    attn.check(c, attn.call(c, workspace=ws, out=out, **kw), **kw)
    assert (out[sum(new):] == 7).all()


@DT
@pytest.mark.parametrize("new,before,prefix,H,Hk", [([200, 20], [300, 480], 0, 4, 2), ([150, 3], [120, 30], 230, 4, 2),
                                                    ([1] * 300, 499, 0, 8, 8), ([1] * 300, 249, 250, 8, 8)],
                         ids=["rows", "shared", "line", "behind"])
@pytest.mark.parametrize("rise", [2.0, 5.0])
def test_sums_of_large_values_stay_finite(dtype, rise, new, before, prefix, H, Hk):
    """All scores but the first 48 tokens' are higher by less than moves the running maximum at once (weights of e^2 and
    e^5).  Values below 2^118 of 500 tokens at most: sums of values below 2^127, as they are of weights up to one."""
    c = attn.case(new, before, prefix, H=H, Hk=Hk, dtype=dtype, seed=5)
    assert int(c["lens"].max()) + prefix <= 500
    c["q"].zero_()
    c["q"][..., 0] = 1.0
    c["k_cache"].copy_(torch.where(torch.isnan(c["k_cache"]), c["k_cache"], 0.0))   # (unused rows stay NaN)
    c["k_cache"][..., 0] += rise
    low = (c["prefix_pages"][:3] if prefix else c["table"][:, :3].reshape(-1)).long()
    c["k_cache"][low, :, :, 0] -= rise
    c["v_cache"].copy_((c["v_cache"].float().abs().clamp(0.5, 0.99) * 2.0 ** 118).to(c["v_cache"].dtype))
    out = attn.call(c, scale=1.0)
    attn.check(c, out, scale=1.0)
