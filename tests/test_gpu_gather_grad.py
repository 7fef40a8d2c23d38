"""GPU parity: the gradient of the gather, alone and after the forward calls that made its index lists."""
import pytest
import torch

import plain64 as P64
import workloads as W
from gpu_util import dev

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def D():
    import paper_2310_02409_amd as D
    return D


def lists_of(seed, n_lens, k_lens):
    """Ascending distinct indices per sequence."""
    out = []
    for b, (n, k) in enumerate(zip(n_lens, k_lens)):
        order = torch.argsort(W.uniform_bits(seed + b, 0, 0, n, "cpu"))[:k]
        out.append(sorted(int(i) for i in order))
    return out


def tokens_of(lists, n_lens):
    first, out = 0, []
    for l, n in zip(lists, n_lens):
        out += [first + i for i in l]
        first += n
    return torch.tensor(out, dtype=torch.long)


def check(got, ref, dtype, parts):
    """fp32 sums of `parts` rows at most, rounded once: copies are exact."""
    got = got.detach().cpu().double()
    if parts == 1:
        assert torch.equal(got, ref)
    else:
        assert bool(((got - ref).abs() <= P64.half_step(dtype) * ref.abs() + parts * 2.0 ** -24 * 16 + 1e-30).all())


CASES = [([1], [1]), ([1], [0]), ([9, 8, 1], [3, 0, 1]), ([64, 7, 0, 100], [64, 1, 0, 33]), ([4097], [411]), ([700, 33], [10, 30])]


@pytest.mark.parametrize("dtype,H_kv,d_h", [(BF16, 2, 128), (BF16, 1, 64), (F32, 3, 64), (F32, 1, 4), (BF16, 40, 128)])
@pytest.mark.parametrize("n_lens,k_lens", CASES)
def test_rows_go_back(D, n_lens, k_lens, dtype, H_kv, d_h):
    N, Kt = sum(n_lens), sum(k_lens)
    lists = lists_of(5, n_lens, k_lens)
    tokens = tokens_of(lists, n_lens)
    idx = torch.tensor([i for l in lists for i in l], dtype=torch.int32, device=dev())
    cu_n, cu_k = W.cumulative(n_lens, dev()), W.cumulative(k_lens, dev())
    rows = [W.normal(6, i, (Kt, H_kv, d_h), 1.0, dtype) for i in range(2)]
    base = [W.normal(6, 2 + i, (N, H_kv, d_h), 1.0, dtype) for i in range(2)]
    for layout in (0, 1):
        src = [(r if layout == 0 else r.permute(1, 0, 2)).contiguous().to(dev()) for r in rows]
        out = D.dodo_gather_nuggets_grad(*src, idx, cu_n, cu_k, N, layout)
        for x, r in zip(out, rows):
            check(x, P64.gather_grad(r, tokens, N), dtype, 1)
        # into the caller's rows of a wider buffer, which stays as it is around them
        wide = [torch.full((N + 2, 2 * H_kv, d_h), 7.0, dtype=dtype, device=dev()) for _ in range(2)]
        D.dodo_gather_nuggets_grad(*src, idx, cu_n, cu_k, N, layout, wide[0][1:N + 1, :H_kv], wide[1][1:N + 1, :H_kv])
        for w, x in zip(wide, out):
            assert torch.equal(w[1:N + 1, :H_kv], x) and bool((w[:, H_kv:] == 7).all()) and bool((w[0] == 7).all()) and bool((w[-1] == 7).all())
        # added to gradients that are there
        added = [b.to(dev()) for b in base]
        back = D.dodo_gather_nuggets_grad(*src, idx, cu_n, cu_k, N, layout, *added, accumulate=True)
        for x, a, b, r in zip(back, added, base, rows):
            assert x is a
            check(x, P64.gather_grad(r, tokens, N, b), dtype, 2)
            others = torch.ones(N, dtype=torch.bool)
            others[tokens] = False
            assert torch.equal(x.cpu()[others], b[others])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_repeated_indices_are_summed(D, dtype):
    # runs within 64 entries, one of more than 64 that crosses them, at a sequence's first and last token, and in two sequences
    lists = [[0, 0, 3, 3, 3, 9] + [12] * 150 + [13, 20, 20], [0] * 70 + [1, 1]]
    n_lens, k_lens = [21, 2], [len(l) for l in lists]
    tokens = tokens_of(lists, n_lens)
    idx = torch.tensor([i for l in lists for i in l], dtype=torch.int32, device=dev())
    cu_n, cu_k = W.cumulative(n_lens, dev()), W.cumulative(k_lens, dev())
    rows = [W.normal(7, i, (sum(k_lens), 2, 64), 1.0, dtype) for i in range(2)]
    src = [r.to(dev()) for r in rows]
    out = D.dodo_gather_nuggets_grad(*src, idx, cu_n, cu_k, 23)
    for x, r in zip(out, rows):
        check(x, P64.gather_grad(r, tokens, 23), dtype, 150)
    base = W.normal(7, 4, (23, 2, 64), 1.0, dtype)
    added = [base.to(dev()), base.to(dev())]
    D.dodo_gather_nuggets_grad(*src, idx, cu_n, cu_k, 23, 0, *added, accumulate=True)
    for x, r in zip(added, rows):
        check(x, P64.gather_grad(r, tokens, 23, base), dtype, 151)


def test_indices_outside_and_rows_behind(D):
    # an index below 0 or past its sequence gives no row; rows behind the last sequence and list entries behind the last nugget are not touched
    idx = torch.tensor([-3, 2, 5, 900, 1, 77, 78], dtype=torch.int32, device=dev())
    cu_n, cu_k = W.cumulative([6, 4], dev()), W.cumulative([4, 1], dev())
    src = [W.normal(8, i, (7, 1, 64), 1.0, F32, dev()) for i in range(2)]
    for accumulate in (False, True):
        out = [torch.full((13, 1, 64), 4.0, device=dev()) for _ in range(2)]
        D.dodo_gather_nuggets_grad(*src, idx, cu_n, cu_k, 13, 0, *out, accumulate=accumulate)
        for x, r in zip(out, src):
            want = torch.full((13, 1, 64), 4.0) if accumulate else torch.cat((torch.zeros(10, 1, 64), torch.full((3, 1, 64), 4.0)))
            for tok, row in ((2, 1), (5, 2), (7, 4)):
                want[tok] = r[row].cpu() + (4.0 if accumulate else 0.0)
            assert torch.equal(x.cpu(), want)


def test_many_sequences(D):
    n_lens = [(11 * b) % 23 for b in range(150)]
    k_lens = [(3 * b) % (n + 1) for b, n in enumerate(n_lens)]
    lists = lists_of(9, n_lens, k_lens)
    tokens, N = tokens_of(lists, n_lens), sum(n_lens)
    idx = torch.tensor([i for l in lists for i in l], dtype=torch.int32, device=dev())
    r = W.normal(10, 0, (sum(k_lens), 2, 64), 1.0, BF16)
    out = D.dodo_gather_nuggets_grad(r.to(dev()), r.to(dev()), idx, W.cumulative(n_lens, dev()), W.cumulative(k_lens, dev()), N)
    check(out[0], P64.gather_grad(r, tokens, N), BF16, 1)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("accumulate", [False, True])
def test_layers_are_that_many_calls(D, layout, accumulate):
    n_lens, k_lens, L = [50, 31], [7, 30], 3
    lists = lists_of(11, n_lens, k_lens)
    idx = torch.tensor([i for l in lists for i in l], dtype=torch.int32, device=dev())
    cu_n, cu_k = W.cumulative(n_lens, dev()), W.cumulative(k_lens, dev())
    shape = (L, 37, 2, 64) if layout == 0 else (L, 2, 37, 64)
    src = [W.normal(12, i, shape, 1.0, BF16, dev()) for i in range(2)]
    base = [W.normal(12, 2 + i, (L, 81, 2, 64), 1.0, BF16, dev()) for i in range(2)]
    out = D.dodo_gather_nuggets_grad_layers(*src, idx, cu_n, cu_k, 81, layout, *([b.clone() for b in base] if accumulate else (None, None)),
                                            accumulate)
    for l in range(L):
        one = D.dodo_gather_nuggets_grad(src[0][l], src[1][l], idx, cu_n, cu_k, 81, layout, *([b[l].clone() for b in base] if accumulate else (None, None)),
                                         accumulate)
        assert torch.equal(out[0][l], one[0]) and torch.equal(out[1][l], one[1])


def test_gather_then_its_gradient(D):
    # scores -> selection -> gather -> gradient: <gather(K), G> = <K, gather_grad(G)> exactly where the sums are of the same numbers
    n_lens = [700, 333]
    cu_n = W.cumulative(n_lens, dev())
    cu_k, ks = D.cu_nuggets_from_lengths(n_lens, 1, 10, dev())
    hidden, w = W.normal(13, 0, (1033, 64), 1.0, BF16, dev()), W.normal(13, 1, (64,), 0.1, BF16, dev())
    idx = D.dodo_select_topk(D.dodo_score(hidden, w), cu_n, cu_k, 700, max(ks), sum(ks))
    K, V = (W.normal(13, 2 + i, (1033, 2, 64), 1.0, F32, dev()) for i in range(2))
    Kn, Vn = D.dodo_gather_nuggets(K, V, idx, cu_n, cu_k, sum(ks))
    G = W.normal(13, 4, Kn.shape, 1.0, F32, dev())
    dK, dV = D.dodo_gather_nuggets_grad(G, Kn, idx, cu_n, cu_k, 1033)
    assert torch.equal(dV[dV.abs().sum((1, 2)) > 0], Vn * 0 + Kn)
    assert abs(float((Kn.double() * G.double()).sum() - (K.double() * dK.double()).sum())) <= 1e-9
    assert int((dK.abs().sum((1, 2)) > 0).sum()) == sum(ks)


def test_refusals(D):
    idx, cu = torch.zeros(3, dtype=torch.int32, device=dev()), W.cumulative([4], dev())
    cu_k = W.cumulative([3], dev())
    src = torch.zeros(3, 1, 64, device=dev())
    out = torch.zeros(4, 1, 64, device=dev())
    with pytest.raises(ValueError):
        D.dodo_gather_nuggets_grad(src, src, idx, cu, cu_k, 4, accumulate=True)
    with pytest.raises(ValueError):
        D.dodo_gather_nuggets_grad(src, src, idx, cu, cu_k, 4, 0, out)
    with pytest.raises(ValueError):
        D.dodo_gather_nuggets_grad(src, src, idx[:2], cu, cu_k, 4)
    with pytest.raises(ValueError):
        D.dodo_gather_nuggets_grad(src, src, idx, cu, cu_k, 4, 0, out, out.bfloat16())
    with pytest.raises(TypeError):
        D.dodo_gather_nuggets_grad(src, src, idx.long(), cu, cu_k, 4)
    with pytest.raises(ValueError):
        D.dodo_gather_nuggets_grad(src, src.cpu(), idx, cu, cu_k, 4)
