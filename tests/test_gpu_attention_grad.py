"""GPU parity: the backward pass of nugget attention against the formulas in 64 bits, fed with the same O and log-sum-exp."""
import pytest
import torch

import plain64 as P64
import workloads as W
from gpu_util import dev

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
NAMES = ("dQ", "dKn", "dVn", "dKl", "dVl")


@pytest.fixture(scope="module")
def D():
    import paper_2310_02409_amd as D
    return D


def make(seed, Sq, Kt, Sm, H, H_kv, d_h, dtype, entries, scale, dO_std=1.0):
    mk = lambda tid, n, h, std=1.0: W.normal(seed, tid, (n, h, d_h), std, dtype)
    t = dict(Q=mk(0, Sq, H), Kn=mk(1, Kt, H_kv), Vn=mk(2, Kt, H_kv), Kl=mk(3, Sm, H_kv), Vl=mk(4, Sm, H_kv), dO=mk(5, Sq, H, dO_std))
    O, lse = P64.attention(t["Q"], t["Kn"], t["Vn"], t["Kl"], t["Vl"], entries, scale)
    t["O"], t["lse"] = O.to(dtype), lse.float()
    return t


def reference(t, entries, scale):
    return P64.attention_grad(*(t[n] for n in ("Q", "Kn", "Vn", "Kl", "Vl", "dO", "O", "lse")), entries, scale)


def check(got, ref, terms, d_h, dtype, layout=0):
    for name, x, r, near, wide in zip(NAMES, got, ref[0], ref[1], ref[2]):
        x = x.detach().cpu().double()
        if layout == 1 and name in ("dKn", "dVn"):
            x = x.permute(1, 0, 2)
        assert torch.isfinite(x).all(), name
        over = (x - r).abs() - P64.grad_tolerance(r, near, wide, ref[3], terms, d_h, dtype)
        assert over.numel() == 0 or float(over.max()) <= 0, f"{name}: {float(over.max()):.3e} beyond the bound"


def call(D, t, lens, scale, layout=0, **kw):
    d = {n: v.to(dev()) for n, v in t.items()}
    if layout == 1:
        d["Kn"], d["Vn"] = d["Kn"].permute(1, 0, 2).contiguous(), d["Vn"].permute(1, 0, 2).contiguous()
    cu = [W.cumulative(x, dev()) for x in lens]
    return D.dodo_nugget_attention_grad(d["Q"], d["Kn"], d["Vn"], d["Kl"], d["Vl"], d["dO"], d["O"], d["lse"], *cu, *(max(x) for x in lens),
                                        scale, layout, **kw)


HEADS = [(2, 2, 128), (4, 2, 64), (4, 1, 128), (3, 3, 64)]
LENS = [
    ([1], [1], [1]), ([1, 3], [0, 5], [2, 3]), ([33], [31], [40]), ([64, 1], [65, 7], [64, 1]), ([32, 31], [32, 33], [32, 95]),
    ([100, 0, 37, 5], [13, 4, 200, 0], [130, 9, 37, 6]),
    ([129], [127], [129]), ([70, 40], [129, 300], [200, 41]),
    ([6, 3], [2, 0], [3, 1]),   # more query rows than local rows: the first of them see nuggets alone, or nothing
    ([5, 9], [0, 3], [0, 0]),   # no local rows; a sequence without any key
    ([3], [0], [70]),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,H_kv,d_h", HEADS)
@pytest.mark.parametrize("q_lens,k_lens,m_lens", LENS)
def test_gradients(D, q_lens, k_lens, m_lens, H, H_kv, d_h, dtype):
    scale, entries = d_h ** -0.5, P64.entries_of(q_lens, k_lens, m_lens)
    t = make(10 + len(q_lens), sum(q_lens), sum(k_lens), sum(m_lens), H, H_kv, d_h, dtype, entries, scale)
    ref, terms = reference(t, entries, scale), max(max(q_lens) * (H // H_kv), max(k_lens) + max(m_lens))
    got = call(D, t, (q_lens, k_lens, m_lens), scale)
    check(got, ref, terms, d_h, dtype)
    again = call(D, t, (q_lens, k_lens, m_lens), scale, layout=1)
    check(again, ref, terms, d_h, dtype, layout=1)
    for a, b in zip(got, again):  # the same sums
        assert torch.equal(a if a.shape == b.shape else a.permute(1, 0, 2), b) or torch.equal(a.permute(1, 0, 2), b)


# longer ones: several tiles of rows and of keys per workgroup, ragged ends
@pytest.mark.parametrize("q_lens,k_lens,m_lens,H,H_kv,d_h", [
    ([300, 515], [410, 103], [428, 515], 2, 2, 128), ([1025], [64], [1030], 2, 1, 128), ([257, 40], [520, 700], [290, 600], 4, 2, 64),
])
def test_longer_sequences(D, q_lens, k_lens, m_lens, H, H_kv, d_h):
    scale, entries = d_h ** -0.5, P64.entries_of(q_lens, k_lens, m_lens)
    for dtype in (BF16, F32):
        t = make(40, sum(q_lens), sum(k_lens), sum(m_lens), H, H_kv, d_h, dtype, entries, scale)
        terms = max(max(q_lens) * (H // H_kv), max(k_lens) + max(m_lens))
        check(call(D, t, (q_lens, k_lens, m_lens), scale), reference(t, entries, scale), terms, d_h, dtype)


def test_many_short_sequences(D):
    q_lens = [(7 * b) % 19 for b in range(90)]
    k_lens = [(5 * b) % 13 for b in range(90)]
    m_lens = [q + b % 4 for b, q in enumerate(q_lens)]
    scale, entries = 0.3, P64.entries_of(q_lens, k_lens, m_lens)
    for dtype in (BF16, F32):
        t = make(50, sum(q_lens), sum(k_lens), sum(m_lens), 2, 2, 64, dtype, entries, scale)
        check(call(D, t, (q_lens, k_lens, m_lens), scale), reference(t, entries, scale), 40, 64, dtype)


@pytest.mark.parametrize("scale", [-0.2, 0.0, 2.5])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scales(D, scale, dtype):
    # (2.5: nearly all of a row's weight on one key, most weights underflow)
    lens = ([40], [35], [50])
    entries = P64.entries_of(*lens)
    t = make(60, 40, 35, 50, 2, 2, 64, dtype, entries, scale)
    check(call(D, t, lens, scale), reference(t, entries, scale), 90, 64, dtype)


def test_rows_behind_the_last_sequence_are_left_alone(D):
    lens = ([33, 20], [40, 9], [50, 30])
    for dtype in (BF16, F32):
        entries = P64.entries_of(*lens)
        t = make(70, 53 + 5, 49 + 5, 80 + 5, 2, 2, 128, dtype, entries, 0.1)
        outs = {n: torch.full_like(t[m], 7.0).to(dev()) for n, m in zip(NAMES, ("Q", "Kn", "Vn", "Kl", "Vl"))}
        got = call(D, t, lens, 0.1, **outs)
        ref = reference(t, entries, 0.1)
        for name, x, end in zip(NAMES, got, (53, 49, 49, 80, 80)):
            assert x is outs[name] and bool((x[end:] == 7.0).all()), name
        check([x[:e] for x, e in zip(got, (53, 49, 49, 80, 80))], tuple([y[:e] for y, e in zip(r, (53, 49, 49, 80, 80))] for r in ref[:3]) + (ref[3],),
              90, 128, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_bad_row_stays_in_its_sequence(D, dtype, value):
    lens = ([40, 37, 20], [20, 21, 50], [60, 45, 20])
    entries = P64.entries_of(*lens)
    t = make(80, 97, 91, 125, 2, 2, 64, dtype, entries, 0.125)
    good = call(D, t, lens, 0.125)
    for name in ("Q", "Kn", "Vn", "Kl", "Vl", "dO"):
        bad = {n: v.clone() for n, v in t.items()}
        e = entries[1]
        first, count = (e[0], e[1]) if name in ("Q", "dO") else (e[2], e[3]) if name in ("Kn", "Vn") else (e[4], e[5])
        bad[name][first:first + count] = value
        got = call(D, bad, lens, 0.125)
        for out, (lo, hi) in zip(range(5), ((40, 77), (20, 41), (20, 41), (60, 105), (60, 105))):
            assert torch.equal(got[out][:lo], good[out][:lo]) and torch.equal(got[out][hi:], good[out][hi:]), (name, NAMES[out])


# segments: a plan's ranges, ranges with gaps that no entry holds, entries without rows or keys
SEGMENTS = [
    [(0, 20, 0, 0, 0, 20), (20, 20, 0, 3, 12, 28), (40, 7, 0, 5, 30, 17), (47, 20, 5, 0, 47, 20), (67, 13, 5, 4, 60, 20)],
    [(0, 64, 0, 0, 0, 64), (64, 64, 0, 9, 40, 88), (128, 33, 0, 17, 100, 61)],
    [(0, 10, 3, 4, 20, 12), (10, 0, 0, 8, 0, 5), (10, 50, 2, 6, 25, 60), (60, 5, 7, 0, 90, 0)],
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("entries", SEGMENTS)
@pytest.mark.parametrize("H,H_kv,d_h", [(2, 2, 128), (4, 2, 64)])
def test_segments(D, entries, H, H_kv, d_h, dtype):
    Sq, Kt, N, scale = entries[-1][0] + entries[-1][1], 20, 170, d_h ** -0.5
    t = make(90, Sq, Kt, N, H, H_kv, d_h, dtype, entries, scale)
    ref = reference(t, entries, scale)
    d = {n: v.to(dev()) for n, v in t.items()}
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev())
    plan = [i32([e[0] for e in entries] + [Sq])] + [i32([e[i] for e in entries]) for i in (2, 3, 4, 5)]
    bounds = [max(e[i] for e in entries) for i in (1, 3, 5)]
    for layout in (0, 1):
        Kn, Vn = (d[n] if layout == 0 else d[n].permute(1, 0, 2).contiguous() for n in ("Kn", "Vn"))
        outs = [torch.full_like(x, float("nan")) for x in (d["Q"], Kn, Vn, d["Kl"], d["Vl"])]
        got = D.dodo_nugget_attention_segments_grad(d["Q"], Kn, Vn, d["Kl"], d["Vl"], d["dO"], d["O"], d["lse"], *plan, *bounds, scale, layout, *outs)
        check(got, ref, len(entries) * 300, d_h, dtype, layout)


def test_more_segments_than_lanes(D):
    # 100 texts of one to four segments of 5 tokens: entries are looked for 64 at a time
    entries, q, k = [], 0, 0
    for b in range(100):
        n = 3 + (7 * b) % 18
        nug = b % 4
        for s in range(0, n, 5):
            first = max(0, s - 2)
            entries.append((q + s, min(5, n - s), k, min(nug, first), q + first, min(n, s + 5) - first))
        q, k = q + n, k + nug
    t = make(95, q, k, q, 2, 1, 64, BF16, entries, 0.125)
    d = {n: v.to(dev()) for n, v in t.items()}
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev())
    plan = [i32([e[0] for e in entries] + [q])] + [i32([e[i] for e in entries]) for i in (2, 3, 4, 5)]
    got = D.dodo_nugget_attention_segments_grad(d["Q"], d["Kn"], d["Vn"], d["Kl"], d["Vl"], d["dO"], d["O"], d["lse"], *plan, 5, 3, 7, 0.125)
    check(got, reference(t, entries, 0.125), 40, 64, BF16)


def test_no_segments_and_no_queries_give_zeros(D):
    for dtype in (BF16, F32):
        t = make(96, 4, 6, 9, 2, 2, 64, dtype, [(0, 4, 0, 6, 0, 9)], 0.1)
        d = {n: v.to(dev()) for n, v in t.items()}
        none = torch.zeros(0, dtype=torch.int32, device=dev())
        got = D.dodo_nugget_attention_segments_grad(d["Q"], d["Kn"], d["Vn"], d["Kl"], d["Vl"], d["dO"], d["O"], d["lse"],
                                                    torch.zeros(1, dtype=torch.int32, device=dev()), none, none, none, none, 4, 6, 9, 0.1)
        assert all(float(x.float().abs().max()) == 0 for x in got[1:])
        empty = {n: d[n][:0].contiguous() for n in ("Q", "dO", "O", "lse")}
        cu = [W.cumulative([n], dev()) for n in (0, 6, 9)]
        got = D.dodo_nugget_attention_grad(empty["Q"], d["Kn"], d["Vn"], d["Kl"], d["Vl"], empty["dO"], empty["O"], empty["lse"], *cu, 0, 6, 9, 0.1)
        assert all(float(x.float().abs().max()) == 0 for x in got[1:])


def test_forward_and_backward_together_against_differences(D):
    # the library's own forward pass in fp32, then its gradients, against differences of the loss in 64 bits
    lens = ([30, 21], [25, 40], [44, 21])
    entries, scale, step = P64.entries_of(*lens), 64 ** -0.5, 1e-4
    t = make(97, 51, 65, 65, 4, 2, 64, F32, entries, scale)
    d = {n: v.to(dev()) for n, v in t.items()}
    cu = [W.cumulative(x, dev()) for x in lens]
    O, lse = D.dodo_nugget_attention(d["Q"], d["Kn"], d["Vn"], d["Kl"], d["Vl"], *cu, 30, 40, 44, scale, want_lse=True)
    got = D.dodo_nugget_attention_grad(d["Q"], d["Kn"], d["Vn"], d["Kl"], d["Vl"], d["dO"], O, lse, *cu, 30, 40, 44, scale)
    inputs = {n: t[n].double() for n in ("Q", "Kn", "Vn", "Kl", "Vl")}
    for name, x in zip(inputs, got):
        way = W.normal(98, 1, t[name].shape, 1.0, F32).double()
        loss = [float((P64.attention(*dict(inputs, **{name: inputs[name] + s * step * way}).values(), entries, scale)[0] * t["dO"].double()).sum())
                for s in (1, -1)]
        terms = x.cpu().double() * way
        # a difference is off by step^2 times a third derivative (1e-8 of the terms' magnitudes); fp32 terms by some 2^-24 each
        assert abs((loss[0] - loss[1]) / (2 * step) - float(terms.sum())) <= 2e-6 * float(terms.abs().sum())


def test_deterministic_captured_and_on_another_stream(D):
    lens = ([200, 90], [70, 130], [260, 90])
    t = make(99, 290, 200, 350, 4, 2, 128, BF16, P64.entries_of(*lens), 128 ** -0.5)
    first = [x.clone() for x in call(D, t, lens, 128 ** -0.5)]
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, call(D, t, lens, 128 ** -0.5)))
    d = {n: v.to(dev()) for n, v in t.items()}
    cu = [W.cumulative(x, dev()) for x in lens]
    outs = [torch.empty_like(d[n]) for n in ("Q", "Kn", "Vn", "Kl", "Vl")]
    ws = torch.empty(D.dodo_nugget_attention_grad_workspace_bytes(2, 4, 2, 128, 200, 130, 260, 290, 200, 350, D.BF16), dtype=torch.uint8,
                     device=dev())
    go = lambda: D.dodo_nugget_attention_grad(d["Q"], d["Kn"], d["Vn"], d["Kl"], d["Vl"], d["dO"], d["O"], d["lse"], *cu, 200, 130, 260,
                                              128 ** -0.5, 0, *outs, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    other = [x.clone() for x in (d["Q"], d["dO"])]
    for turn in range(3):
        for x in outs:
            x.fill_(3.0)
        ws.fill_(255)
        if turn == 1:  # other values at the same addresses
            d["Q"].mul_(0.5)
        elif turn == 2:
            d["Q"].copy_(other[0])
        graph.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in outs]
        go()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs)), turn
        assert turn == 1 or all(torch.equal(a, b) for a, b in zip(first, outs))


def test_refusals(D):
    lens = ([4], [5], [6])
    t = make(100, 4, 5, 6, 2, 2, 64, F32, P64.entries_of(*lens), 0.1)
    with pytest.raises(ValueError):
        call(D, dict(t, O=t["O"].bfloat16()), lens, 0.1)
    with pytest.raises(ValueError):
        call(D, dict(t, dO=t["dO"][:3]), lens, 0.1)
    with pytest.raises(ValueError):
        call(D, dict(t, Vn=t["Vn"][:4]), lens, 0.1)
    with pytest.raises(D.DodoError):
        call(D, t, lens, 0.1, ws=torch.empty(16, dtype=torch.uint8, device=dev()))
    with pytest.raises(ValueError):
        call(D, t, lens, 0.1, dQ=torch.empty((4, 2, 32), device=dev()))
