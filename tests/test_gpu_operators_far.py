"""Gradients and 4-bit caches where the rows lie behind 2^31 elements and 2^32 bytes: the same bits as for the rows by themselves."""
import pytest
import torch

import paper_2310_02409_amd as D

pytestmark = pytest.mark.gpu
H, H_kv, d_h = 16, 8, 128
K_B, Q_B = 200, 40


def cu(*lens):
    return torch.tensor((0,) + lens).cumsum(0).to(torch.int32).cuda()


def randn(*shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=torch.Generator().manual_seed(sum(shape))).to(dtype).cuda()


@pytest.mark.parametrize("layout", [D.TOKEN_MAJOR, D.HEAD_MAJOR])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_gradients(dtype, layout):
    far = 2_200_000  # rows of a first sequence, which no query row asks for
    Q, dO, Kl, Vl = (randn(Q_B, h, d_h, dtype=dtype) for h in (H, H, H_kv, H_kv))
    near = [randn(K_B, H_kv, d_h, dtype=dtype) for _ in range(2)]
    if layout == D.HEAD_MAJOR:
        near = [x.transpose(0, 1).contiguous() for x in near]
    rows = lambda x: x[far:] if layout == D.TOKEN_MAJOR else x[:, far:]
    whole = [torch.empty((far + K_B, H_kv, d_h) if layout == D.TOKEN_MAJOR else (H_kv, far + K_B, d_h), dtype=dtype, device="cuda") for _ in range(2)]
    for x, y in zip(whole, near):
        rows(x).copy_(y)
    a = (Kl, Vl, cu(Q_B), cu(K_B), cu(Q_B), Q_B, K_B, Q_B, d_h ** -0.5, layout)
    O, lse = D.dodo_nugget_attention(Q, *near, *a, want_lse=True)
    want = D.dodo_nugget_attention_grad(Q, *near, Kl, Vl, dO, O, lse, *a[2:])
    # the larger bounds may choose other workgroups, and with them another order of the sums
    tol = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -17
    got = D.dodo_nugget_attention_grad(Q, *whole, Kl, Vl, dO, O, lse, cu(0, Q_B), cu(far, K_B), cu(0, Q_B), Q_B, far, Q_B, d_h ** -0.5, layout)
    for i, (x, y) in enumerate(zip(got, want)):
        x = rows(x) if i in (1, 2) else x
        assert (x.float() - y.float()).abs().max() <= tol * y.float().abs().max()
    for x in got[1:3]:
        first = x[:far] if layout == D.TOKEN_MAJOR else x[:, :far]
        assert all(not bool(part.any()) for part in first.split(1 << 19, dim=0 if layout == D.TOKEN_MAJOR else 1))


@pytest.mark.parametrize("layout", [D.TOKEN_MAJOR, D.HEAD_MAJOR])
@pytest.mark.parametrize("q", [1, 4, 40])
def test_attention_over_4_bits(q, layout):
    far = 9_000_000
    Q, Kl, Vl = randn(q, H, d_h), randn(q + 9, H_kv, d_h), randn(q + 9, H_kv, d_h)
    idx, cu_s = torch.arange(K_B, dtype=torch.int32, device="cuda"), cu(K_B)
    near = D.dodo_gather_nuggets_q4(randn(K_B, H_kv, d_h), randn(K_B, H_kv, d_h).flip(0), idx, cu_s, cu(K_B), K_B, layout)
    rows = lambda x: x[far:] if layout == D.TOKEN_MAJOR else x[:, far:]
    lead = (far + K_B, H_kv) if layout == D.TOKEN_MAJOR else (H_kv, far + K_B)
    whole = [torch.empty(lead + x.shape[2:], dtype=torch.uint8, device="cuda") for x in near]
    for x, y in zip(whole, near):
        rows(x).copy_(y)
    want = D.dodo_nugget_attention_q4(Q, *near, Kl, Vl, cu(q), cu(K_B), cu(q + 9), q, K_B, q + 9, layout=layout)[0]
    got = D.dodo_nugget_attention_q4(Q, *whole, Kl, Vl, cu(0, q), cu(far, K_B), cu(0, q + 9), q, K_B, q + 9, layout=layout)[0]
    # (two sequences may be shared out otherwise than one: another order of the sums, O rounded once)
    assert (got.float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()


def test_gather_and_its_gradient():
    far = 2_200_000  # tokens of a first sequence
    idx = torch.cat((torch.tensor([3, far - 1]), torch.arange(0, 2 * K_B, 2))).to(torch.int32).cuda()
    K = torch.zeros(far + 2 * K_B, H_kv, d_h, dtype=torch.bfloat16, device="cuda")
    K[far:] = randn(2 * K_B, H_kv, d_h)
    V = K.flip(2)
    near = D.dodo_gather_nuggets_q4(K[far:].clone(), V[far:].clone(), idx[2:].clone(), cu(2 * K_B), cu(K_B), K_B)
    got = D.dodo_gather_nuggets_q4(K, V, idx, cu(far, 2 * K_B), cu(2, K_B), K_B + 2)
    assert all(torch.equal(x[2:], y) for x, y in zip(got, near))
    plain = D.dodo_unpack_nuggets_q4(*got)
    assert not bool(plain[0][:2].any())
    dKn, dVn = randn(K_B + 2, H_kv, d_h), randn(K_B + 2, H_kv, d_h).flip(0)
    dK, dV = D.dodo_gather_nuggets_grad(dKn, dVn, idx, cu(far, 2 * K_B), cu(2, K_B), far + 2 * K_B)
    for g, x in ((dKn, dK), (dVn, dV)):
        assert torch.equal(x[far::2], g[2:]) and torch.equal(x[3], g[0]) and torch.equal(x[far - 1], g[1])
        assert not bool(x[far + 1::2].any()) and sum(int(part.flatten(1).any(1).sum()) for part in x.split(1 << 19)) == K_B + 2
