"""The fp64 forms of the full-attention layer's operators and of linear attention
against other ways of computing the same: library attention over gathered rows,
complex multiplication, the closed form of the recurrence, counting (CPU)."""
import random

import pytest
import torch

from oracle import attn_ops as ref

F64 = torch.float64


@pytest.mark.parametrize("prefix,new,held", [(0, [4, 1], [0, 9]), (7, [3, 0, 2], [0, 5, 11]), (12, [1], [0])])
def test_attention_is_library_attention_of_the_gathered_rows(prefix, new, held):
    torch.manual_seed(len(new) + prefix)
    H, Hk, D, ps, pages = 6, 2, 8, 4, 40
    kc, vc = torch.randn(pages, ps, Hk, D, dtype=F64), torch.randn(pages, ps, Hk, D, dtype=F64)
    perm = torch.randperm(pages)
    W = 5
    table = perm[:len(new) * W].reshape(len(new), W).int()
    pre = perm[len(new) * W:][:-(-prefix // ps)].int()
    lens = torch.tensor([a + b for a, b in zip(new, held)], dtype=torch.int32)
    cu = [0]
    for x in new:
        cu.append(cu[-1] + x)
    q = torch.randn(cu[-1], H, D, dtype=F64)
    out, mag, _, _, count = ref.attention(q, kc, vc, table, lens, cu, pre, prefix, scale=0.3)
    for n, L in enumerate(new):
        m = int(lens[n])
        own = lambda c: c[table[n].long()].reshape(-1, Hk, D)[:m]
        k, v = (torch.cat([c[pre.long()].reshape(-1, Hk, D)[:prefix], own(c)]).repeat_interleave(H // Hk, 1) for c in (kc, vc))
        see = torch.arange(prefix + m)[None] <= prefix + m - L + torch.arange(L)[:, None]
        want = torch.nn.functional.scaled_dot_product_attention(
            q[cu[n]:cu[n + 1]].transpose(0, 1), k.transpose(0, 1), v.transpose(0, 1), attn_mask=see, scale=0.3).transpose(0, 1)
        torch.testing.assert_close(out[cu[n]:cu[n + 1]], want, rtol=1e-12, atol=1e-12)
        assert count[cu[n]:cu[n + 1]].tolist() == see.sum(1).tolist()
    assert (mag >= out.abs() - 1e-12).all()


def test_attention_of_pages_that_are_none_and_of_nothing():
    kc = vc = torch.ones(3, 2, 1, 4, dtype=F64)
    vc = vc.clone()
    vc[1] = 5.0
    table = torch.tensor([[-1, 1], [3, -1]], dtype=torch.int32)
    out, _, _, _, count = ref.attention(torch.ones(3, 1, 4), kc, vc, table, torch.tensor([4, 2]), [0, 1, 3])
    assert (out[0] == 5.0).all() and (out[1:] == 0).all() and count.tolist() == [2, 0, 0]


def test_queries_before_the_own_tokens_see_the_prefix_alone():
    kc = torch.ones(4, 2, 1, 4, dtype=F64)
    vc = torch.arange(4, dtype=F64)[:, None, None, None].expand(4, 2, 1, 4)
    out, _, _, _, count = ref.attention(torch.ones(3, 1, 4), kc, vc, torch.tensor([[3]], dtype=torch.int32), torch.tensor([1]),
                                        [0, 3], torch.tensor([1, 2], dtype=torch.int32), 4)
    assert count.tolist() == [4, 4, 5] and (out[:2] == 1.5).all() and torch.allclose(out[2], torch.tensor(9 / 5, dtype=F64))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_complex_multiplication(interleaved):
    torch.manual_seed(1)
    x, cs = torch.randn(5, 3, 16, dtype=F64), torch.randn(9, 8)
    pos = torch.tensor([0, 8, 3, 3, 1])
    w = torch.randn(16, dtype=F64)
    y, _ = ref.qk_rows(x, pos, cs, w, eps=0.1, interleaved=interleaved)
    n = torch.nn.functional.rms_norm(x, (16,), w, eps=0.1)
    a, b = (n[..., 0:8:2], n[..., 1:8:2]) if interleaved else (n[..., :4], n[..., 4:8])
    c = cs.double()[pos][:, None]
    z = torch.complex(a.contiguous(), b.contiguous()) * torch.complex(c[..., :4].contiguous(), c[..., 4:].contiguous())
    re, im = (y[..., 0:8:2], y[..., 1:8:2]) if interleaved else (y[..., :4], y[..., 4:8])
    torch.testing.assert_close(re, z.real, rtol=1e-12, atol=1e-12)
    torch.testing.assert_close(im, z.imag, rtol=1e-12, atol=1e-12)
    torch.testing.assert_close(y[..., 8:], n[..., 8:], rtol=1e-12, atol=1e-12)


def test_linear_attention_is_its_closed_form():
    """o_t = scale sum_{s <= t} exp((t - s) g) (q_t . k_s) v_s, and the state's part exp((t + 1) g)."""
    torch.manual_seed(2)
    L, Hk, H, K, V = 6, 2, 4, 3, 5
    q, k, v = torch.randn(L, Hk, K, dtype=F64), torch.randn(L, Hk, K, dtype=F64), torch.randn(L, H, V, dtype=F64)
    g, s0 = -torch.rand(H), torch.randn(1, H, K, V, dtype=F64)
    o, st, _, _ = ref.linear(q, k, v, g, [0, L], scale=0.7, state=s0)
    for h in range(H):
        d = torch.arange(L, dtype=F64)[:, None] - torch.arange(L, dtype=F64)[None]
        a = torch.where(d >= 0, torch.exp(d * g[h].double()), 0.0) * (q[:, h // 2] @ k[:, h // 2].T)
        first = torch.exp(torch.arange(1, L + 1, dtype=F64) * g[h].double())[:, None] * (q[:, h // 2] @ s0[0, h])
        torch.testing.assert_close(o[:, h], 0.7 * (a @ v[:, h] + first), rtol=1e-12, atol=1e-12)
    one = ref.linear(None, k[:L - 1], v[:L - 1], g, [0, L - 1], state=s0)[1]
    two = ref.linear(None, k[L - 1:], v[L - 1:], g, [0, 1], state=one)[1]
    torch.testing.assert_close(two, st, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("seed", range(30))
def test_pages_are_taken_once_and_in_order(seed):
    rng = random.Random(seed)
    n, ps, W = rng.randrange(1, 6), rng.choice([1, 3, 16]), 12
    held = [rng.randrange(0, W * ps // 2) for _ in range(n)]
    new = [rng.randrange(0, W * ps // 2) for _ in range(n)]
    cu = [0]
    for x in new:
        cu.append(cu[-1] + x)
    table, free = [[1000 + 100 * i + c for c in range(W)] for i in range(n)], list(range(500))
    out, lens, taken, slots, positions = ref.extend_pages(table, held, cu, free, ps, first=7, taken=3)
    assert lens == [a + b for a, b in zip(held, new)]
    fresh = [p for r in out for p in r if p < 1000]
    assert fresh == list(range(3, taken))
    for i in range(n):
        old = -(-held[i] // ps)
        assert out[i][:old] == table[i][:old] and len([p for p in out[i] if p < 1000]) == -(-lens[i] // ps) - old
        for j in range(new[i]):
            t = held[i] + j
            assert slots[cu[i] + j] == out[i][t // ps] * ps + t % ps and positions[cu[i] + j] == 7 + t
    assert len(set(slots)) == len(slots)


def test_the_free_list_and_the_table_end():
    table, lens, taken, slots, _ = ref.extend_pages([[9, -5], [-5, -5]], [2, 0], [0, 3, 6], [4], 2)
    assert table == [[9, 4], [-1, -1]] and lens == [5, 3] and taken == 3
    assert slots == [8, 9, -1, -1, -1, -1]
