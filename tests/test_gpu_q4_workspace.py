"""Attention over 4-bit caches: one workspace for calls of different sizes and routes, and the routes that unpack the cache under kept
workspaces, streams, graphs and rows behind 2^31 elements."""
import pytest
import torch

import test_gpu_q4 as Q4
import workloads as W
from gpu_util import dev

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# (type, heads, K/V heads, channels, lengths): codes read in place in several shares, in one, and unpacked for either attention kernel
CALLS = [(BF16, 8, 8, 128, ([1], [1500], [300])), (F32, 8, 2, 64, ([1, 2], [700, 90], [80, 5])), (BF16, 16, 2, 128, ([1, 1, 1], [3000, 2500, 40], [100, 90, 7])),
         (BF16, 4, 2, 128, ([140], [900], [200])), (BF16, 8, 1, 64, ([9], [2000], [30])), (BF16, 40, 1, 64, ([2], [800], [40])),
         (BF16, 4, 4, 64, ([64, 3], [200, 900], [70, 3])), (F32, 2, 2, 128, ([33], [1200], [64])), (BF16, 2, 1, 128, ([1], [3], [2]))]
ZEROED = 65536


@pytest.fixture(scope="module")
def D():
    import paper_2310_02409_amd as D
    return D


def on_device(seed, dtype, H, H_kv, d_h, lens):
    t = Q4.attention_case(seed, *lens, H, H_kv, d_h, dtype)
    return {n: v.to(dev()) for n, v in t.items()}, [W.cumulative(x, dev()) for x in lens], [max(x) for x in lens]


def need_of(D, dtype, H, H_kv, d_h, lens):
    return D.dodo_nugget_attention_q4_workspace_bytes(len(lens[0]), H, H_kv, d_h, *(max(x) for x in lens), sum(lens[1]), D.F32 if dtype == F32 else D.BF16)


def attend(D, d, cu, bounds, **kw):
    return D.dodo_nugget_attention_q4(d["Q"], d["Kc"], d["Ks"], d["Vc"], d["Vs"], d["Kl"], d["Vl"], *cu, *bounds, 0.1, **kw)


def test_one_workspace_for_calls_of_all_sizes_and_routes(D):
    needs = [need_of(D, *c) for c in CALLS]
    assert min(needs) == 0 and sum(n > ZEROED for n in needs) >= 6
    ws = torch.full((max(needs),), 255, dtype=torch.uint8, device=dev())
    ws[:ZEROED] = 0
    cases = [on_device(80 + i, *c) for i, c in enumerate(CALLS)]
    want = [attend(D, *c, want_lse=True) for c in cases]
    for step in (1, 2, 4, 5, 7):  # (orders in which different calls follow one another)
        for i in range(len(cases)):
            at = (step * i) % len(cases)
            got = attend(D, *cases[at], want_lse=True, ws=ws)
            assert torch.equal(got[0], want[at][0]) and torch.equal(got[1], want[at][1]), (step, CALLS[at])
            assert not bool(ws[:ZEROED].any()), (step, CALLS[at])


@pytest.mark.parametrize("dtype,H,H_kv,d_h,lens", [CALLS[1], CALLS[3], CALLS[5], CALLS[7], (BF16, 2, 2, 64, ([300], [200], [310]))])
def test_unpacked_caches_streams_and_graphs(D, dtype, H, H_kv, d_h, lens):
    case = on_device(90, dtype, H, H_kv, d_h, lens)
    ws = torch.zeros(max(16, need_of(D, dtype, H, H_kv, d_h, lens)), dtype=torch.uint8, device=dev())
    O, lse = torch.empty_like(case[0]["Q"]), torch.empty(case[0]["Q"].shape[:2], device=dev())
    go = lambda: attend(D, *case, O=O, lse=lse, ws=ws)
    go()
    first = O.clone(), lse.clone()

    def again(run):
        O.fill_(float("nan"))
        lse.fill_(float("nan"))
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        assert torch.equal(O, first[0]) and torch.equal(lse, first[1])

    for _ in range(5):
        again(go)
    side = torch.cuda.Stream()

    def beside():
        with torch.cuda.stream(side):
            go()
    again(beside)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for _ in range(4):
        again(graph.replay)
        again(go)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype,q", [(BF16, 140), (F32, 1), (F32, 3)])
def test_unpacked_rows_behind_2_to_31_elements(D, dtype, q, layout):
    far, H, H_kv, d_h, k = 2_200_000, 16, 8, 128, 200
    lens = ([q], [k], [q + 9])
    d, cu, bounds = on_device(95, dtype, H, H_kv, d_h, lens)
    if layout == 1:
        for n in ("Kc", "Ks", "Vc", "Vs"):
            d[n] = d[n].permute(1, 0, 2).contiguous()
    d["Ks"][(k - 1, H_kv - 1) if layout == 0 else (H_kv - 1, k - 1)] = 255  # the last row's key, in the last head
    want = attend(D, d, cu, bounds, layout=layout, want_lse=True)
    whole = dict(d)
    for n in ("Kc", "Ks", "Vc", "Vs"):
        lead = (far + k, H_kv) if layout == 0 else (H_kv, far + k)
        whole[n] = torch.zeros(lead + d[n].shape[2:], dtype=torch.uint8, device=dev())
        (whole[n][far:] if layout == 0 else whole[n][:, far:]).copy_(d[n])
    two = lambda *x: W.cumulative(x, dev())
    got = attend(D, whole, (two(0, q), two(far, k), two(0, q + 9)), (q, far, q + 9), layout=layout, want_lse=True)
    G, hit = H // H_kv, torch.zeros(q, H, dtype=torch.bool, device=dev())
    hit[:, H - G:] = True
    for O, lse in (want, got):
        assert torch.equal(torch.isnan(O).all(-1), hit) and torch.equal(torch.isnan(O).any(-1), hit) and torch.equal(torch.isnan(lse), hit)
    # (two sequences may be shared out otherwise than one: another order of the sums, O rounded once)
    tol = 2.0 ** -7 if dtype == BF16 else 2.0 ** -17
    x, y = got[0][~hit].float(), want[0][~hit].float()
    assert (x - y).abs().max() <= tol * y.abs().max()
    assert (got[1][~hit] - want[1][~hit]).abs().max() <= 2.0 ** -17 * want[1][~hit].abs().max()
