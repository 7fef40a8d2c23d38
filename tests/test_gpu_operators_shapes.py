"""Gradients of the attention and 4-bit caches: group sizes and grids that choose other workgroups, bounds far above the lengths, capture
without a workspace of the caller's, and a training step from the context's K and V on."""
import pytest
import torch

import plain64 as P64
import test_gpu_attention_grad as G
import test_gpu_q4 as Q4
import workloads as W
from gpu_util import dev

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def D():
    import paper_2310_02409_amd as D
    return D


@pytest.mark.parametrize("lens", [([1, 2], [300, 40], [60, 2]), ([3], [70], [9]), ([16, 5], [100, 33], [40, 5]), ([25], [65], [90])])
@pytest.mark.parametrize("H,H_kv,d_h", [(10, 2, 128), (21, 3, 64), (24, 2, 128), (40, 2, 64), (24, 1, 64), (32, 1, 128), (33, 1, 64)])
def test_attention_over_4_bits_group_sizes(D, H, H_kv, d_h, lens):
    t = Q4.attention_case(40, *lens, H, H_kv, d_h, BF16)
    for layout in (0, 1):
        O, lse = Q4.attend(D, t, lens, d_h ** -0.5, layout, want_lse=True)
        Q4.check(D, t, lens, d_h ** -0.5, BF16, O, lse)


@pytest.mark.parametrize("q,H,H_kv,d_h", [(32, 16, 16, 64), (33, 16, 16, 128), (9, 32, 8, 64), (2, 64, 4, 128), (1, 32, 32, 64)])
def test_attention_over_4_bits_many_sequences(D, q, H, H_kv, d_h):
    lens = ([q - b % 2 for b in range(24)], [(37 * b) % 150 for b in range(24)], [q + (11 * b) % 40 for b in range(24)])
    t = Q4.attention_case(41, *lens, H, H_kv, d_h, BF16)
    O, lse = Q4.attend(D, t, lens, d_h ** -0.5, want_lse=True)
    Q4.check(D, t, lens, d_h ** -0.5, BF16, O, lse)


@pytest.mark.parametrize("H,H_kv", [(4, 4), (8, 1)])
@pytest.mark.parametrize("bounds", [(15, 9000, 3000), (64, 100000, 40), (1000, 1, 9)])
def test_bounds_above_the_lengths(D, bounds, H, H_kv):
    lens, d_h = ([1, 0, 9], [70, 5, 0], [4, 3, 9]), 64
    bounds = tuple(max(b, max(x)) for b, x in zip(bounds, lens))
    t = Q4.attention_case(42, *lens, H, H_kv, d_h, BF16)
    d, cu = {n: v.to(dev()) for n, v in t.items()}, [W.cumulative(x, dev()) for x in lens]
    O, lse = D.dodo_nugget_attention_q4(d["Q"], d["Kc"], d["Ks"], d["Vc"], d["Vs"], d["Kl"], d["Vl"], *cu, *bounds, 0.125, want_lse=True)
    Q4.check(D, t, lens, 0.125, BF16, O, lse)
    entries = P64.entries_of(*lens)
    for dtype in (BF16, F32):
        t = G.make(43, 10, 75, 16, H, H_kv, d_h, dtype, entries, 0.125)
        d = {n: v.to(dev()) for n, v in t.items()}
        got = D.dodo_nugget_attention_grad(*(d[n] for n in ("Q", "Kn", "Vn", "Kl", "Vl", "dO", "O", "lse")), *cu, *bounds, 0.125)
        G.check(got, G.reference(t, entries, 0.125), 100, d_h, dtype)


# (a grid of many workgroups: 128 owned rows each)
@pytest.mark.parametrize("H,H_kv,d_h", [(16, 16, 64), (16, 16, 128), (40, 8, 64), (21, 3, 128)])
def test_gradients_of_many_sequences(D, H, H_kv, d_h):
    B = 40 if H == H_kv else 16
    lens = ([1 + (29 * b) % 170 for b in range(B)], [(17 * b) % 140 for b in range(B)], [1 + (29 * b) % 170 + b % 5 for b in range(B)])
    scale, entries = d_h ** -0.5, P64.entries_of(*lens)
    t = G.make(44, *(sum(x) for x in lens), H, H_kv, d_h, BF16, entries, scale)
    G.check(G.call(D, t, lens, scale), G.reference(t, entries, scale), max(170 * (H // H_kv), 320), d_h, BF16)


# (few key rows, and walks of 16 and more tiles of query rows: four wavefronts for 32 keys, two tiles at a time, odd ends)
@pytest.mark.parametrize("H,H_kv,d_h", [(8, 1, 64), (8, 1, 128), (16, 2, 64), (1, 1, 128)])
@pytest.mark.parametrize("lens", [([1100], [70], [1100]), ([1025, 3], [0, 65], [1090, 1]), ([1200], [33], [900])])
def test_gradients_of_long_walks(D, lens, H, H_kv, d_h):
    scale, entries = d_h ** -0.5, P64.entries_of(*lens)
    t = G.make(48, *(sum(x) for x in lens), H, H_kv, d_h, BF16, entries, scale)
    G.check(G.call(D, t, lens, scale), G.reference(t, entries, scale), max(1200 * (H // H_kv), 1200), d_h, BF16)


@pytest.mark.parametrize("H,H_kv", [(16, 16), (32, 16)])
def test_gradients_of_long_texts_in_segments(D, H, H_kv):
    N, seg, tau, every = 4300, 500, 60, 40
    entries = [(s, min(seg, N - s), 0, max(0, s - tau) // every, max(0, s - tau), min(N, s + seg) - max(0, s - tau)) for s in range(0, N, seg)]
    Kt, d_h = N // every, 64
    t = G.make(45, N, Kt, N, H, H_kv, d_h, BF16, entries, 0.125)
    d = {n: v.to(dev()) for n, v in t.items()}
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev())
    plan = [i32([e[0] for e in entries] + [N])] + [i32([e[i] for e in entries]) for i in (2, 3, 4, 5)]
    got = D.dodo_nugget_attention_segments_grad(*(d[n] for n in ("Q", "Kn", "Vn", "Kl", "Vl", "dO", "O", "lse")), *plan, seg, Kt, seg + tau, 0.125)
    G.check(got, G.reference(t, entries, 0.125), N * (H // H_kv), d_h, BF16)


@pytest.mark.parametrize("q,k", [(1, 2000), (40, 60), (300, 60)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_captured_without_a_workspace(D, dtype, q, k):
    """The binding's own workspaces live in the graph: replays, with eager calls in between, give the eager result."""
    lens, H, H_kv, d_h = ([q], [k], [q + 7]), 8, 2, 64
    t = Q4.attention_case(46, *lens, H, H_kv, d_h, dtype)
    d, cu = {n: v.to(dev()) for n, v in t.items()}, [W.cumulative(x, dev()) for x in lens]
    dO = W.normal(46, 9, (q, H, d_h), 1.0, dtype, dev())

    def step():
        cache = [d[n] for n in ("Kc", "Ks", "Vc", "Vs")]
        O, lse = D.dodo_nugget_attention_q4(d["Q"], *cache, d["Kl"], d["Vl"], *cu, q, k, q + 7, 0.125, want_lse=True)
        Kn, Vn = D.dodo_unpack_nuggets_q4(*cache, dtype)
        return (O, lse) + D.dodo_nugget_attention_grad(d["Q"], Kn, Vn, d["Kl"], d["Vl"], dO, O, lse, *cu, q, k, q + 7, 0.125)

    want = [x.clone() for x in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(4):
        for x in got:
            x.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        assert all(torch.equal(x, y) for x, y in zip(step(), want))
        torch.cuda.synchronize()


def test_calls_at_once_on_two_streams(D):
    lens, H, H_kv, d_h = ([3, 1], [900, 2000], [40, 90]), 16, 4, 128
    cases = [Q4.attention_case(47 + i, *lens, H, H_kv, d_h, BF16) for i in range(2)]
    want = [Q4.attend(D, t, lens, 0.1)[0] for t in cases]
    sets, cu = [{n: v.to(dev()) for n, v in t.items()} for t in cases], [W.cumulative(x, dev()) for x in lens]
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, (s, d) in enumerate(zip(streams, sets)):
            with torch.cuda.stream(s):
                got[i].append(D.dodo_nugget_attention_q4(d["Q"], d["Kc"], d["Ks"], d["Vc"], d["Vs"], d["Kl"], d["Vl"], *cu, 3, 2000, 90, 0.1)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[i]) for i in range(2) for x in got[i])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_training_step_from_the_context_on(D, dtype):
    """gather -> attention -> gradients -> gather's gradient: those of the context's K and V, against the formulas in 64 bits fed with the
    library's O and log-sum-exp."""
    n_lens, q_lens, H, H_kv, d_h = [330, 200], [48, 31], 4, 2, 64
    scale, N = d_h ** -0.5, sum(n_lens)
    cu_n, cu_q = W.cumulative(n_lens, dev()), W.cumulative(q_lens, dev())
    cu_k, ks = D.cu_nuggets_from_lengths(n_lens, 1, 10, dev())
    mk = lambda i, n, h: W.normal(60, i, (n, h, d_h), 1.0, dtype, dev())
    K, V, Q, dO, Kl, Vl = mk(0, N, H_kv), mk(1, N, H_kv), mk(2, 79, H), mk(3, 79, H), mk(4, 79, H_kv), mk(5, 79, H_kv)
    scores = W.normal(60, 6, (N,), 1.0, F32, dev())
    idx = D.dodo_select_topk(scores, cu_n, cu_k, max(n_lens), max(ks), sum(ks))
    Kn, Vn = D.dodo_gather_nuggets(K, V, idx, cu_n, cu_k, sum(ks))
    a = (cu_q, cu_k, cu_q, max(q_lens), max(ks), max(q_lens), scale)
    O, lse = D.dodo_nugget_attention(Q, Kn, Vn, Kl, Vl, *a, want_lse=True)
    got = D.dodo_nugget_attention_grad(Q, Kn, Vn, Kl, Vl, dO, O, lse, *a)
    entries = P64.entries_of(q_lens, ks, q_lens)
    t = {n: x.cpu() for n, x in dict(Q=Q, Kn=Kn, Vn=Vn, Kl=Kl, Vl=Vl, dO=dO, O=O, lse=lse).items()}
    G.check(got, G.reference(t, entries, scale), 200, d_h, dtype)
    dK, dV = D.dodo_gather_nuggets_grad(got[1], got[2], idx, cu_n, cu_k, N)
    tok = idx.long() + torch.repeat_interleave(cu_n[:-1].long(), torch.tensor(ks, device=dev()))
    for x, g in ((dK, got[1]), (dV, got[2])):
        rest = torch.ones(N, dtype=torch.bool, device=dev())
        rest[tok] = False
        assert torch.equal(x[tok], g) and not bool(x[rest].any())


def test_packing_of_more_sequences_than_lanes(D):
    n_lens = [1 + (13 * b) % 40 for b in range(90)]
    k_lens = [min(n, b % 4) for b, n in enumerate(n_lens)]
    K, V = W.normal(61, 0, (sum(n_lens), 2, 64), 1.0, BF16, dev()), W.normal(61, 1, (sum(n_lens), 2, 64), 1.0, BF16, dev())
    lists = [sorted((7 * i + b) % n for i in range(k)) for b, (n, k) in enumerate(zip(n_lens, k_lens))]
    idx = torch.tensor([i for l in lists for i in l], dtype=torch.int32, device=dev())
    got = D.dodo_gather_nuggets_q4(K, V, idx, W.cumulative(n_lens, dev()), W.cumulative(k_lens, dev()), sum(k_lens))
    starts = W.cumulative(n_lens, dev()).tolist()
    tokens = [starts[b] + i for b, l in enumerate(lists) for i in l]
    want = [x for t in (K, V) for x in P64.quantise_q4(t.cpu()[tokens])]
    assert all(torch.equal(x.cpu(), y) for x, y in zip(got, want))
