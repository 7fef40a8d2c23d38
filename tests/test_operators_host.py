"""Host-only checks of the calls around nugget attention -- gradients, 4-bit caches: exported, and bad arguments refused before
anything is launched (no GPU)."""
import pytest
import torch

OK, INVALID, UNSUPPORTED, SMALL = 0, -1, -2, -3
P = 0x1000  # any non-null, 16-byte aligned fake pointer: validation must fail before it is used
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def D():
    import paper_2310_02409_amd as D
    return D


def grad(D, seg=False, ptr=None, B=2, H=4, H_kv=2, d_h=64, mq=8, mk=4, mm=9, Sq=16, Kt=8, Sm=18, scale=0.1, dtype=BF16, layout=0, ws=P,
         ws_bytes=1 << 20):
    names = ["Q", "Kn", "Vn", "Kl", "Vl", "dO", "O", "lse"] + (["cu_q", "ns", "nl", "ls", "ll"] if seg else ["cu_q", "cu_k", "cu_l"])
    outs = ["dQ", "dKn", "dVn", "dKl", "dVl"]
    ptr = ptr or {}
    f = D.lib.dodo_nugget_attention_segments_grad if seg else D.lib.dodo_nugget_attention_grad
    return f(*(ptr.get(n, P) for n in names), B, H, H_kv, d_h, mq, mk, mm, Sq, Kt, Sm, scale, dtype, layout, *(ptr.get(n, P) for n in outs), ws,
             ws_bytes, 0)


@pytest.mark.parametrize("seg", [False, True])
def test_attention_grad_refusals(D, seg):
    for bad in (dict(B=-1), dict(H=0), dict(H=3), dict(H_kv=0), dict(d_h=0), dict(mq=-1), dict(mk=-1), dict(mm=-1), dict(Sq=-1), dict(Kt=-1),
                dict(Sm=-1), dict(scale=float("nan")), dict(layout=2)):
        assert grad(D, seg, **bad) == INVALID, bad
    for name in ["Q", "Kn", "Vn", "Kl", "Vl", "dO", "O", "lse", "cu_q", "dQ", "dKn", "dVn", "dKl", "dVl"] + (["ns", "nl", "ls", "ll"] if seg else
                                                                                                          ["cu_k", "cu_l"]):
        assert grad(D, seg, ptr={name: 0}) == INVALID, name
    for name in ("Q", "Kn", "Vn", "Kl", "Vl", "dO", "O", "dQ", "dKn", "dVn", "dKl", "dVl"):
        assert grad(D, seg, ptr={name: P + 8}) == UNSUPPORTED, name
    for bad in (dict(dtype=2), dict(d_h=32), dict(d_h=96), dict(d_h=256), dict(ws=P + 4), dict(Sq=1 << 31), dict(Kt=1 << 31), dict(Sm=1 << 31)):
        assert grad(D, seg, **bad) == UNSUPPORTED, bad
    need = D.dodo_nugget_attention_grad_workspace_bytes(2, 4, 2, 64, 8, 4, 9, 16, 8, 18, BF16)
    assert need > 0 and grad(D, seg, ws_bytes=need - 1) == SMALL and grad(D, seg, ws=0) == SMALL
    # nothing to do
    assert grad(D, seg, B=0, Kt=0, Sm=0) == OK
    if not seg:
        assert grad(D, B=0) == OK
    assert grad(D, seg, mq=0, mk=0, mm=0, Kt=0, Sm=0) == OK


def test_grad_workspace_sizes(D):
    f = D.dodo_nugget_attention_grad_workspace_bytes
    assert f(0, 4, 2, 64, 8, 4, 9, 16, 8, 18, BF16) == 0 and f(2, 4, 2, 64, 8, 4, 9, 0, 8, 18, BF16) == 0
    assert f(2, 4, 2, 64, 8, 4, 9, 16, 8, 18, BF16) >= 2 * 4 * 16 * 4


def gather_grad(D, layers=False, ptr=None, dtype=BF16, B=2, Kt=8, N=20, L=3, H_kv=2, d_h=64, tok=128, src=8 * 128, dst=20 * 128, acc=0, layout=0):
    p = lambda n: (ptr or {}).get(n, P)
    if layers:
        return D.lib.dodo_gather_nuggets_grad_layers(p("dKn"), p("dVn"), dtype, p("idx"), p("cu"), p("cu_k"), B, Kt, N, L, H_kv, d_h, tok, src, dst,
                                                     acc, p("dK"), p("dV"), layout, 0)
    return D.lib.dodo_gather_nuggets_grad(p("dKn"), p("dVn"), dtype, p("idx"), p("cu"), p("cu_k"), B, Kt, N, H_kv, d_h, tok, acc, p("dK"), p("dV"),
                                          layout, 0)


@pytest.mark.parametrize("layers", [False, True])
def test_gather_grad_refusals(D, layers):
    for bad in (dict(B=-1), dict(Kt=-1), dict(N=-1), dict(H_kv=0), dict(d_h=0), dict(tok=127), dict(layout=5)):
        assert gather_grad(D, layers, **bad) == INVALID, bad
    for name in ("dKn", "dVn", "idx", "cu", "cu_k", "dK", "dV"):
        assert gather_grad(D, layers, ptr={name: 0}) == INVALID, name
    for bad in (dict(dtype=3), dict(tok=132, dst=20 * 136), dict(d_h=12, tok=128), dict(ptr={"dK": P + 8}), dict(ptr={"dVn": P + 2}), dict(N=1 << 31, dst=1 << 40),
                dict(Kt=1 << 31, src=1 << 40)):
        assert gather_grad(D, layers, **bad) == UNSUPPORTED, bad
    for nothing in (dict(B=0), dict(N=0), dict(Kt=0, acc=1)):
        assert gather_grad(D, layers, **nothing) == OK, nothing
    if layers:
        assert gather_grad(D, True, L=-1) == INVALID and gather_grad(D, True, L=0) == OK and gather_grad(D, True, L=70000) == UNSUPPORTED
        assert gather_grad(D, True, src=8 * 128 - 8) == INVALID and gather_grad(D, True, dst=19 * 128) == INVALID
        assert gather_grad(D, True, src=8 * 128 + 4) == UNSUPPORTED and gather_grad(D, True, dst=20 * 128 + 4) == UNSUPPORTED


def gather_q4(D, layers=False, ptr=None, dtype=BF16, B=2, Kt=8, L=3, H_kv=2, d_h=64, tok=128, src=20 * 128, layout=0):
    p = lambda n: (ptr or {}).get(n, P)
    tail = (p("Kc"), p("Ks"), p("Vc"), p("Vs"), layout, 0)
    if layers:
        return D.lib.dodo_gather_nuggets_q4_layers(p("K"), p("V"), dtype, p("idx"), p("cu"), p("cu_k"), B, Kt, L, H_kv, d_h, tok, src, *tail)
    return D.lib.dodo_gather_nuggets_q4(p("K"), p("V"), dtype, p("idx"), p("cu"), p("cu_k"), B, Kt, H_kv, d_h, tok, *tail)


@pytest.mark.parametrize("layers", [False, True])
def test_gather_q4_refusals(D, layers):
    for bad in (dict(B=-1), dict(Kt=-1), dict(H_kv=0), dict(d_h=0), dict(tok=127), dict(layout=-1)):
        assert gather_q4(D, layers, **bad) == INVALID, bad
    for name in ("K", "V", "idx", "cu", "cu_k", "Kc", "Ks", "Vc", "Vs"):
        assert gather_q4(D, layers, ptr={name: 0}) == INVALID, name
    for bad in (dict(dtype=2), dict(d_h=48, tok=128), dict(tok=132), dict(ptr={"K": P + 8}), dict(ptr={"Kc": P + 8}), dict(ptr={"Vs": P + 2}),
                dict(Kt=1 << 30)):
        assert gather_q4(D, layers, **bad) == UNSUPPORTED, bad
    assert gather_q4(D, layers, B=0) == OK and gather_q4(D, layers, Kt=0) == OK
    if layers:
        assert gather_q4(D, True, L=-1) == INVALID and gather_q4(D, True, src=-8) == INVALID
        assert gather_q4(D, True, L=0) == OK and gather_q4(D, True, L=70000) == UNSUPPORTED and gather_q4(D, True, src=20 * 128 + 4) == UNSUPPORTED


def test_unpack_refusals(D):
    f = lambda rows=8, d_h=64, dtype=BF16, **ptr: D.lib.dodo_unpack_nuggets_q4(*(ptr.get(n, P) for n in ("Kc", "Ks", "Vc", "Vs")), rows, d_h, dtype,
                                                                             ptr.get("Kn", P), ptr.get("Vn", P), 0)
    assert f(rows=-1) == INVALID and f(d_h=0) == INVALID and f(rows=0) == OK
    for name in ("Kc", "Ks", "Vc", "Vs", "Kn", "Vn"):
        assert f(**{name: 0}) == INVALID
    assert f(dtype=9) == UNSUPPORTED and f(d_h=40) == UNSUPPORTED and f(Kn=P + 8) == UNSUPPORTED and f(Vc=P + 4) == UNSUPPORTED
    assert f(rows=1 << 40) == UNSUPPORTED


def attention_q4(D, ptr=None, B=2, H=4, H_kv=2, d_h=64, mq=1, mk=40, mm=9, Kt=80, scale=0.1, dtype=BF16, layout=0, ws=P, ws_bytes=1 << 30):
    p = lambda n: (ptr or {}).get(n, P)
    return D.lib.dodo_nugget_attention_q4(*(p(n) for n in ("Q", "Kc", "Ks", "Vc", "Vs", "Kl", "Vl", "cu_q", "cu_k", "cu_l")), B, H, H_kv, d_h, mq, mk,
                                          mm, Kt, scale, dtype, layout, p("O"), p("lse"), ws, ws_bytes, 0)


def test_attention_q4_refusals(D):
    for bad in (dict(B=-1), dict(H=0), dict(H=3), dict(H_kv=0), dict(d_h=0), dict(mq=-1), dict(mk=-1), dict(mm=-1), dict(Kt=-1),
                dict(scale=float("nan")), dict(layout=2)):
        assert attention_q4(D, **bad) == INVALID, bad
    for name in ("Q", "Kc", "Ks", "Vc", "Vs", "Kl", "Vl", "cu_q", "cu_k", "cu_l", "O"):
        assert attention_q4(D, ptr={name: 0}) == INVALID, name
    for bad in (dict(dtype=2), dict(d_h=32), dict(ws=P + 8), dict(ptr={"Q": P + 8}), dict(ptr={"Vc": P + 8}), dict(ptr={"Ks": P + 1})):
        assert attention_q4(D, **bad) == UNSUPPORTED, bad
    assert attention_q4(D, B=0) == OK and attention_q4(D, mq=0) == OK
    for shape in (dict(mq=1, mk=3000, Kt=6000), dict(mq=64), dict(dtype=F32)):
        a = dict(dict(B=2, H=4, H_kv=2, d_h=64, mq=1, mk=40, mm=9, Kt=80, dtype=BF16), **shape)
        need = D.dodo_nugget_attention_q4_workspace_bytes(*(a[n] for n in ("B", "H", "H_kv", "d_h", "mq", "mk", "mm", "Kt", "dtype")))
        if need:
            assert attention_q4(D, ws_bytes=need - 1, **a) == SMALL and attention_q4(D, ws=0, ws_bytes=0, **a) == SMALL


def test_the_binding_refuses_host_tensors(D):
    t = torch.zeros(4, 2, 64)
    cu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        D.dodo_nugget_attention_grad(t, t, t, t, t, t, t, t[:, :, 0], cu, cu, cu, 4, 4, 4)
    with pytest.raises(ValueError):
        D.dodo_gather_nuggets_grad(t, t, cu, cu, cu, 4)
    with pytest.raises(ValueError):
        D.dodo_gather_nuggets_q4(t, t, cu, cu, cu, 2)
