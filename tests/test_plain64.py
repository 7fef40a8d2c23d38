"""The plain 64-bit implementations that the GPU tests compare with: against torch's automatic differentiation, differences of the
loss, and the 4-bit format's closed forms (CPU only)."""
import math

import pytest
import torch

import plain64 as P64


def _case(seed, q_lens, k_lens, m_lens, H, H_kv, d_h):
    g = torch.Generator().manual_seed(seed)
    mk = lambda n, h: torch.randn((n, h, d_h), generator=g, dtype=torch.float64)
    return dict(Q=mk(sum(q_lens), H), Kn=mk(sum(k_lens), H_kv), Vn=mk(sum(k_lens), H_kv), Kl=mk(sum(m_lens), H_kv),
                Vl=mk(sum(m_lens), H_kv)), mk(sum(q_lens), H)


CASES = [
    ([5], [3], [7], 2, 2, 4), ([4, 0, 1, 6], [2, 3, 0, 5], [6, 2, 1, 4], 4, 2, 4),  # (the last: rows that see no local key)
    ([3], [0], [2], 1, 1, 4),  # a row that sees nothing at all
]


@pytest.mark.parametrize("q_lens,k_lens,m_lens,H,H_kv,d_h", CASES)
def test_gradients_are_those_of_automatic_differentiation(q_lens, k_lens, m_lens, H, H_kv, d_h):
    t, dO = _case(1, q_lens, k_lens, m_lens, H, H_kv, d_h)
    entries, scale = P64.entries_of(q_lens, k_lens, m_lens), 0.6
    leaves = {n: v.clone().requires_grad_() for n, v in t.items()}
    loss = 0.0
    for e in entries:
        for h in range(H):
            kv = h // (H // H_kv)
            K = torch.cat((leaves["Kn"][e[2]:e[2] + e[3], kv], leaves["Kl"][e[4]:e[4] + e[5], kv]))
            V = torch.cat((leaves["Vn"][e[2]:e[2] + e[3], kv], leaves["Vl"][e[4]:e[4] + e[5], kv]))
            for i in range(e[1]):
                see = [j for j in range(e[3] + e[5]) if j < e[3] or j - e[3] <= e[5] - e[1] + i]
                if see:
                    p = torch.softmax(scale * (K[see] @ leaves["Q"][e[0] + i, h]), 0)
                    loss = loss + (p @ V[see]) @ dO[e[0] + i, h]
    want = torch.autograd.grad(loss, [leaves[n] for n in ("Q", "Kn", "Vn", "Kl", "Vl")], allow_unused=True)
    O, lse = P64.attention(*t.values(), entries, scale)
    got, near, wide, _ = P64.attention_grad(*t.values(), dO, O, lse, entries, scale)
    for a, b, n, w in zip(got, want, near, wide):
        b = torch.zeros_like(a) if b is None else b
        assert torch.allclose(a, b, rtol=1e-11, atol=1e-12)
        assert bool((n >= a.abs() - 1e-12).all()) and bool((w >= n - 1e-12).all())


@pytest.mark.parametrize("q_lens,k_lens,m_lens,H,H_kv,d_h", CASES)
def test_gradients_are_differences_of_the_loss(q_lens, k_lens, m_lens, H, H_kv, d_h):
    t, dO = _case(2, q_lens, k_lens, m_lens, H, H_kv, d_h)
    entries, scale, step = P64.entries_of(q_lens, k_lens, m_lens), 0.6, 1e-5
    O, lse = P64.attention(*t.values(), entries, scale)
    got = dict(zip(t, P64.attention_grad(*t.values(), dO, O, lse, entries, scale)[0]))
    g = torch.Generator().manual_seed(3)
    for name in t:
        way = torch.randn(t[name].shape, generator=g, dtype=torch.float64)
        loss = [float((P64.attention(*dict(t, **{name: t[name] + s * step * way}).values(), entries, scale)[0] * dO).sum()) for s in (1, -1)]
        # (the difference's own error: step^2 times a third derivative of a few tens, and 2^-52 / step)
        assert abs((loss[0] - loss[1]) / (2 * step) - float((got[name] * way).sum())) <= 1e-7 * (1 + float((got[name] * way).abs().sum()))


def test_shared_rows_add_up():
    # two entries over the same nuggets and overlapping local rows: the sum of the two alone
    t, dO = _case(4, [4, 3], [5], [9], 2, 1, 4)
    entries = [(0, 4, 0, 2, 0, 5), (4, 3, 0, 5, 3, 6)]
    O, lse = P64.attention(*t.values(), entries, 0.5)
    both = P64.attention_grad(*t.values(), dO, O, lse, entries, 0.5)[0]
    alone = [P64.attention_grad(*t.values(), dO, O, lse, [e], 0.5)[0] for e in entries]
    for a, b, c in zip(both, *alone):
        assert torch.allclose(a, b + c, rtol=1e-13, atol=1e-13)


def test_four_bit_values():
    x = torch.zeros(2, 64, dtype=torch.float64)
    x[0, :8] = torch.tensor([0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])  # ties go to the even code
    x[0, 8:12] = torch.tensor([-0.0, -0.2, -6.0, 7.0])                       # 7 is the largest that a scale of 1 takes
    x[1, 0], x[1, 1] = 7.0001, -0.5
    codes, scales = P64.quantise_q4(x)
    n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    assert n[0, :12].tolist() == [0, 0, 2, 2, 4, 4, 6, 6, 8, 8, 15, 7]
    assert scales[0].tolist() == [127, 2] and scales[1].tolist() == [128, 2]  # (a block of zeros has the least scale)
    assert P64.values_q4(codes, scales)[1, :2].tolist() == [8.0, 0.0]
    x[1, 40] = math.inf
    codes, scales = P64.quantise_q4(x)
    assert scales[1].tolist() == [128, 255] and int(codes[1, 16:].max()) == 0
    assert torch.isnan(P64.values_q4(codes, scales)[1, 32:]).all() and torch.isfinite(P64.values_q4(codes, scales)[1, :32]).all()
    # no value is off by more than half of the step where it lies, relative to the block's largest
    g = torch.Generator().manual_seed(5)
    y = torch.randn(50, 128, generator=g, dtype=torch.float64) * torch.exp(3 * torch.randn(50, 1, generator=g, dtype=torch.float64))
    v = P64.values_q4(*P64.quantise_q4(y))
    top = y.abs().reshape(50, 4, 32).amax(-1).repeat_interleave(32, -1)
    assert bool(((y - v).abs() <= top / 3.5).all())  # a step of 2 / 2 over a scale with top > 3.5
