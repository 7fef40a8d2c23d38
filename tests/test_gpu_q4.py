"""GPU parity: nugget caches in 4 bits -- packing, reading back, and attention over them."""
import math

import pytest
import torch

import plain64 as P64
import workloads as W
from gpu_util import dev
from test_gpu_gather_grad import lists_of, tokens_of

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def D():
    import paper_2310_02409_amd as D
    return D


def special_rows(d, dtype):
    """Rows in which a block's largest magnitude lies around a scale's limits, halves of steps, zeros of both signs, numbers at
    the ends of the range, and NaN and infinities."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn(60, d, generator=g).clamp(-3, 3)
    steps = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.0, -0.0, -0.25, -0.75, -5.0, -3.5, 0.2500001, 0.7499999, 4.9999995])
    for r, (top, factor) in enumerate([(6.0, 1.0), (7.0, 1.0), (7.03125, 1.0), (4.0, 1.0), (3.5, 1.0), (3.515625, 1.0), (6.0, 2.0 ** -20),
                                       (7.0, 2.0 ** 90), (6.0, 2.0 ** -124), (7.0, 2.0 ** -126), (1.0, 2.0 ** -130), (7.5, 2.0 ** 125)]):
        x[r] = 0
        x[r, :16] = steps
        x[r, 16] = top
        x[r, 32:48] = -steps
        x[r, 50] = -top
        x[r] *= factor if factor > 2.0 ** -127 else 1
        if factor < 2.0 ** -127:
            x[r] = x[r] * 2.0 ** -100 * 2.0 ** -30
    x[20] = 0
    x[21, 5], x[22, 40], x[23, 63], x[24, 31] = math.nan, math.inf, -math.inf, math.nan
    x[25] = torch.finfo(dtype).max
    x[26] = -torch.finfo(dtype).tiny
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H_kv,d_h", [(2, 64), (1, 128), (3, 32), (5, 128)])
def test_packing_is_the_formats(D, dtype, H_kv, d_h):
    n_lens, k_lens = [40, 0, 20], [33, 0, 20]
    K = special_rows(H_kv * d_h, dtype).view(60, H_kv, d_h) if H_kv * d_h >= 64 else special_rows(96, dtype)[:, :H_kv * d_h].reshape(60, H_kv, d_h)
    V = W.normal(2, 1, (60, H_kv, d_h), 3.0, dtype)
    lists = lists_of(4, n_lens, k_lens)
    lists[0] = [i for i in range(40) if i not in (0, 1, 13, 27, 33, 34, 39)]
    tokens = tokens_of(lists, n_lens)
    idx = torch.tensor([i for l in lists for i in l], dtype=torch.int32, device=dev())
    cu_n, cu_k = W.cumulative(n_lens, dev()), W.cumulative(k_lens, dev())
    for layout in (0, 1):
        q4 = D.dodo_gather_nuggets_q4(K.to(dev()), V.to(dev()), idx, cu_n, cu_k, 53, layout)
        back = {t: D.dodo_unpack_nuggets_q4(*q4, dtype=t) for t in (BF16, F32)}
        for i, src in ((0, K), (1, V)):
            rows = src[tokens]
            codes, scales = P64.quantise_q4(rows)
            if layout == 1:
                codes, scales = codes.permute(1, 0, 2), scales.permute(1, 0, 2)
            assert torch.equal(q4[2 * i + 1].cpu(), scales)
            assert torch.equal(q4[2 * i].cpu(), codes)
            want = P64.values_q4(codes, scales)
            for t, x in back.items():
                assert torch.equal(torch.isnan(x[i].cpu()), torch.isnan(want)) and torch.equal(torch.nan_to_num(x[i].cpu().double()), torch.nan_to_num(want))


@pytest.mark.parametrize("layout", [0, 1])
def test_layers_strides_and_an_upper_bound_of_the_count(D, layout):
    n_lens, k_lens, L = [50, 31], [7, 30], 3
    lists = lists_of(11, n_lens, k_lens)
    idx = torch.tensor([i for l in lists for i in l] + [0, 0], dtype=torch.int32, device=dev())
    cu_n, cu_k = W.cumulative(n_lens, dev()), W.cumulative(k_lens, dev())
    K, V = (W.normal(12, i, (L, 81, 4, 64), 1.0, BF16, dev())[:, :, 1:3] for i in range(2))  # rows apart by twice their size
    out = D.dodo_gather_nuggets_q4_layers(K, V, idx, cu_n, cu_k, 37, layout)
    for l in range(L):
        one = D.dodo_gather_nuggets_q4(K[l].contiguous(), V[l].contiguous(), idx, cu_n, cu_k, 37, layout)
        assert all(torch.equal(a[l], b) for a, b in zip(out, one))
    plain = D.dodo_gather_nuggets(K[0].contiguous(), V[0].contiguous(), idx, cu_n, cu_k, 37, layout)
    codes, scales = P64.quantise_q4(plain[0].cpu())
    assert torch.equal(out[0][0].cpu(), codes) and torch.equal(out[1][0].cpu(), scales)
    if layout == 0:  # 39 rows of room, 37 nuggets: the rest stays as it is
        room = [torch.full((39, 2, n), 9, dtype=torch.uint8, device=dev()) for n in (32, 2, 32, 2)]
        D.dodo_gather_nuggets_q4(K[0], V[0], idx, cu_n, cu_k, 39, layout, *room)
        for r, o in zip(room, out):
            assert torch.equal(r[:37], o[0]) and bool((r[37:] == 9).all())


def attention_case(seed, q_lens, k_lens, m_lens, H, H_kv, d_h, dtype):
    mk = lambda tid, n, h: W.normal(seed, tid, (n, h, d_h), 1.0, dtype)
    t = dict(Q=mk(0, sum(q_lens), H), Kl=mk(3, sum(m_lens), H_kv), Vl=mk(4, sum(m_lens), H_kv))
    t["Kc"], t["Ks"] = P64.quantise_q4(mk(1, sum(k_lens), H_kv))
    t["Vc"], t["Vs"] = P64.quantise_q4(mk(2, sum(k_lens), H_kv))
    return t


def attend(D, t, lens, scale, layout=0, **kw):
    d = {n: v.to(dev()) for n, v in t.items()}
    if layout == 1:
        for n in ("Kc", "Ks", "Vc", "Vs"):
            d[n] = d[n].permute(1, 0, 2).contiguous()
    cu = [W.cumulative(x, dev()) for x in lens]
    return D.dodo_nugget_attention_q4(d["Q"], d["Kc"], d["Ks"], d["Vc"], d["Vs"], d["Kl"], d["Vl"], *cu, *(max(x) for x in lens), scale, layout,
                                      **kw)


def check(D, t, lens, scale, dtype, O, lse):
    """Against 64 bits: O is rounded once, and with bf16 the weights may be rounded to it before they meet V (half a step of each
    term); fp32 sums of the d_h products of a logit (of magnitude `most`), of the weights and of their products with V."""
    entries, d_h = P64.entries_of(*lens), t["Q"].shape[2]
    Kn, Vn = P64.values_q4(t["Kc"], t["Ks"]), P64.values_q4(t["Vc"], t["Vs"])
    ref, lse_ref = P64.attention(t["Q"], Kn, Vn, t["Kl"], t["Vl"], entries, scale)
    size, _ = P64.attention(t["Q"], Kn, Vn.abs(), t["Kl"], t["Vl"].abs(), entries, scale)
    most = 0.0
    for e in entries:
        K = torch.cat((Kn[e[2]:e[2] + e[3]], t["Kl"][e[4]:e[4] + e[5]].double())).abs()
        q = t["Q"][e[0]:e[0] + e[1]].double().abs()
        if e[1] and len(K):
            G = q.shape[1] // K.shape[1]
            most = max(most, float(torch.matmul(q.permute(1, 0, 2), K.repeat_interleave(G, 1).permute(1, 2, 0)).max()) * abs(scale))
    fp32 = 2.0 ** -24 * (max(lens[1]) + max(lens[2]) + (d_h + 64) * (1 + most))
    tol = P64.half_step(dtype) * ref.abs() + (2 * fp32 + (2 * P64.half_step(BF16) if dtype == BF16 else 0)) * size + 1e-30
    got = O.detach().cpu().double()
    assert torch.isfinite(got).all()
    over = (got - ref).abs() - tol
    assert float(over.max()) <= 0, f"{float(over.max()):.3e} beyond the bound"
    if lse is not None:
        x = lse.detach().cpu().double()
        assert torch.equal(torch.isneginf(x), torch.isneginf(lse_ref))
        fin = torch.isfinite(lse_ref)
        # (the sum of the weights may be that of the rounded ones)
        assert bool(((x - lse_ref).abs()[fin] <= 2 * fp32 * (1 + lse_ref.abs()[fin]) + (P64.half_step(BF16) if dtype == BF16 else 0)).all())


LENS = [
    ([1], [1], [1]), ([1, 1, 1], [410, 33, 0], [257, 0, 5]), ([1], [0], [40]), ([1] * 5, [31, 32, 33, 64, 65], [31, 32, 33, 64, 65]),
    ([1], [3277], [300]), ([1], [2000], [0]), ([4, 2], [100, 37], [90, 3]), ([15], [200], [15]), ([16], [40], [16]), ([33, 0, 70], [64, 9, 129], [40, 2, 70]),
    ([7, 3], [2, 0], [4, 1]),  # rows that see no local row, or nothing
    ([130], [700], [200]),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,H_kv,d_h", [(4, 4, 128), (8, 1, 128), (4, 2, 64), (3, 3, 64), (40, 1, 64)])
@pytest.mark.parametrize("lens", LENS)
def test_attention(D, lens, H, H_kv, d_h, dtype):
    scale = d_h ** -0.5
    t = attention_case(20, *lens, H, H_kv, d_h, dtype)
    O, lse = attend(D, t, lens, scale, want_lse=True)
    check(D, t, lens, scale, dtype, O, lse)
    O1, lse1 = attend(D, t, lens, scale, layout=1, want_lse=True)
    assert torch.equal(O, O1) and torch.equal(lse, lse1)


def test_wide_scales_and_large_logits(D):
    # scales from 2^-125 to 2^40 side by side, and logits of several hundred
    lens, H, d_h = ([1, 20], [200, 90], [30, 40]), 2, 128
    t = attention_case(21, *lens, H, H, d_h, BF16)
    for b, f in enumerate((2, 60, 100, 126, 129, 131)):
        t["Ks"][b::7] = f
        t["Vs"][b + 1::9] = min(f, 130)
    for scale in (d_h ** -0.5, -0.05, 0.0, 0.9):
        O, lse = attend(D, t, lens, scale, want_lse=True)
        check(D, t, lens, scale, BF16, O, lse)


@pytest.mark.parametrize("q", [1, 5, 40])
def test_a_bad_block_reaches_its_own_head_and_channels(D, q):
    lens, H, d_h = ([q, q], [70, 40], [q + 3, q]), 2, 128
    t = attention_case(22, *lens, H, H, d_h, BF16)
    good, _ = attend(D, t, lens, d_h ** -0.5)
    bad = {n: v.clone() for n, v in t.items()}
    bad["Ks"][75, 1, 2] = 255  # a key of the second sequence, head 1
    O, _ = attend(D, bad, lens, d_h ** -0.5)
    assert torch.equal(O[:q], good[:q]) and torch.equal(O[q:, 0], good[q:, 0]) and torch.isnan(O[q:, 1]).all()
    bad = {n: v.clone() for n, v in t.items()}
    bad["Vs"][75, 1, 2] = 255  # a value: its 32 channels
    O, _ = attend(D, bad, lens, d_h ** -0.5)
    keep = [c for c in range(d_h) if c // 32 != 2]
    assert torch.equal(O[:q], good[:q]) and torch.equal(O[q:, 0], good[q:, 0])
    assert torch.isnan(O[q:, 1, 64:96]).all() and torch.equal(O[q:, 1][:, keep], good[q:, 1][:, keep])


@pytest.mark.parametrize("H,H_kv,lens", [(8, 8, ([1], [1500], [300])), (16, 2, ([1, 1], [3000, 2500], [100, 90])), (4, 4, ([64], [900], [70]))])
def test_a_kept_workspace_streams_and_graphs(D, H, H_kv, lens):
    t = attention_case(23, *lens, H, H_kv, 128, BF16)
    d = {n: v.to(dev()) for n, v in t.items()}
    cu = [W.cumulative(x, dev()) for x in lens]
    B, (mq, mk, mm), Kt = len(lens[0]), [max(x) for x in lens], sum(lens[1])
    need = D.dodo_nugget_attention_q4_workspace_bytes(B, H, H_kv, 128, mq, mk, mm, Kt, D.BF16)
    ws = torch.zeros(max(16, need), dtype=torch.uint8, device=dev())
    O = torch.empty_like(d["Q"])
    go = lambda: D.dodo_nugget_attention_q4(d["Q"], d["Kc"], d["Ks"], d["Vc"], d["Vs"], d["Kl"], d["Vl"], *cu, mq, mk, mm, 0.088, O=O, ws=ws)
    go()
    first = O.clone()
    for _ in range(20):
        O.fill_(float("nan"))
        go()
        assert torch.equal(O, first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    O.fill_(float("nan"))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        go()
    torch.cuda.synchronize()
    assert torch.equal(O, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for _ in range(4):
        O.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, first)
        O.fill_(float("nan"))
        go()  # an eager call between the replays, on the same workspace
        torch.cuda.synchronize()
        assert torch.equal(O, first)


def test_pack_then_attend_as_a_server_does(D):
    # a context compressed into a 4-bit cache, a prompt over it, then single tokens as the window grows
    n_lens, H, H_kv, d_h = [600, 411], 8, 2, 64
    cu_n = W.cumulative(n_lens, dev())
    cu_k, ks = D.cu_nuggets_from_lengths(n_lens, 1, 10, dev())
    hidden, w = W.normal(30, 0, (1011, 512), 1.0, BF16, dev()), W.normal(30, 1, (512,), 0.05, BF16, dev())
    K, V = (W.normal(30, 2 + i, (1011, H_kv, d_h), 1.0, BF16, dev()) for i in range(2))
    idx = D.dodo_select_topk(D.dodo_score(hidden, w), cu_n, cu_k, 600, max(ks), sum(ks))
    q4 = D.dodo_gather_nuggets_q4(K, V, idx, cu_n, cu_k, sum(ks))
    tokens = tokens_of([idx.cpu()[:ks[0]].tolist(), idx.cpu()[ks[0]:].tolist()], n_lens)
    assert torch.equal(q4[0].cpu(), P64.quantise_q4(K.cpu()[tokens])[0])
    for q, m in ((20, 20), (1, 21), (1, 22)):
        lens = ([q, q], ks, [m, m])
        t = dict(zip(("Kc", "Ks", "Vc", "Vs"), (x.cpu() for x in q4)), Q=W.normal(31, m, (2 * q, H, d_h), 1.0, BF16),
                 Kl=W.normal(32, m, (2 * m, H_kv, d_h), 1.0, BF16), Vl=W.normal(33, m, (2 * m, H_kv, d_h), 1.0, BF16))
        O, lse = attend(D, t, lens, d_h ** -0.5, want_lse=True)
        check(D, t, lens, d_h ** -0.5, BF16, O, lse)


def test_refusals(D):
    lens = ([1], [8], [4])
    t = attention_case(24, *lens, 2, 2, 64, BF16)
    with pytest.raises(ValueError):
        attend(D, dict(t, Ks=t["Ks"][:, :, :1]), lens, 0.1)
    with pytest.raises(ValueError):
        attend(D, dict(t, Kc=t["Kc"].to(torch.int32)), lens, 0.1)
    with pytest.raises(ValueError):
        attend(D, dict(t, Kl=t["Kl"].float()), lens, 0.1)
    with pytest.raises(ValueError):
        attend(D, t, lens, 0.1, lse=torch.empty(3, device=dev()))
    with pytest.raises(ValueError):
        D.dodo_unpack_nuggets_q4(t["Kc"].to(dev()), t["Ks"].to(dev()), t["Vc"].to(dev()), t["Vs"][:4].to(dev()))
    K, idx, cu = torch.zeros(9, 2, 64, dtype=BF16, device=dev()), torch.zeros(3, dtype=torch.int32, device=dev()), W.cumulative([9], dev())
    with pytest.raises(ValueError):
        D.dodo_gather_nuggets_q4(K, K, idx, cu, W.cumulative([3], dev()), 4)
    with pytest.raises(ValueError):
        D.dodo_gather_nuggets_q4(K, K, idx, cu, W.cumulative([3], dev()), 3, 0, torch.empty(3, 2, 32, dtype=torch.uint8, device=dev()))
    with pytest.raises(D.DodoError):  # blocks of 32 channels
        D.dodo_gather_nuggets_q4(K[:, :, :48].contiguous(), K[:, :, :48].contiguous(), idx, cu, W.cumulative([3], dev()), 3)
