"""Gradients of nugget attention and of the gather, and 4-bit caches, through the binding's native calls (csrc/dodo_torch.cpp) and
through ctypes: the same results, returned objects and refusals."""
import types

import pytest
import torch

import paper_2310_02409_amd.binding as B

pytestmark = pytest.mark.gpu
NAMES = ("nugget_attention_grad", "nugget_attention_segments_grad", "gather_nuggets_grad", "gather_nuggets_q4", "unpack_nuggets_q4",
         "nugget_attention_q4")


@pytest.fixture
def native(monkeypatch):
    """The module with a note of the calls that it did itself; `native(False)` declines them all."""
    module, done = B._native, []

    def noting(name):
        f = getattr(module, name)

        def call(*a):
            r = f(*a)
            if r is not None:
                done.append(name)
            return r
        return call

    def switch(on):
        done.clear()
        new = types.SimpleNamespace(**{n: getattr(module, n) for n in dir(module) if not n.startswith("__")})
        for n in NAMES:
            setattr(new, n, noting(n) if on else (lambda *a: None))
        monkeypatch.setattr(B, "_native", new)
        return done
    return switch


def inputs(dtype):
    g = torch.Generator().manual_seed(7)
    r = lambda *s: torch.randn(s, generator=g).to(dtype).cuda()
    cu = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    t = dict(K=r(300, 2, 64), V=r(300, 2, 64), Q=r(40, 4, 64), dO=r(40, 4, 64), Kl=r(60, 2, 64), Vl=r(60, 2, 64), Kn=r(30, 2, 64), Vn=r(30, 2, 64),
             cu_s=cu(0, 100, 300), cu_k=cu(0, 10, 30), cu_q=cu(0, 20, 40), cu_l=cu(0, 25, 60), ns=cu(0, 5), nl=cu(10, 25), ls=cu(0, 25), ll=cu(25, 35),
             idx=torch.cat((torch.arange(0, 100, 10), torch.arange(0, 200, 10))).to(torch.int32).cuda())
    t["O"], t["lse"] = B.dodo_nugget_attention(t["Q"], t["Kn"], t["Vn"], t["Kl"], t["Vl"], t["cu_q"], t["cu_k"], t["cu_l"], 20, 20, 35, want_lse=True)
    return t


def calls(t):
    """Every function in the forms that programs use: results allocated or given, optional arguments named or left out."""
    out = {}
    a = tuple(t[n] for n in ("Q", "Kn", "Vn", "Kl", "Vl", "dO", "O", "lse"))
    cu = (t["cu_q"], t["cu_k"], t["cu_l"])
    out["grad"] = B.dodo_nugget_attention_grad(*a, *cu, 20, 20, 35)
    given = [torch.empty_like(t[n]) for n in ("Q", "Kn", "Vn", "Kl", "Vl")]
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    got = out["grad given"] = B.dodo_nugget_attention_grad(*a, *cu, 20, 20, 35, 0.125, B.TOKEN_MAJOR, *given, ws=ws)
    assert all(x is y for x, y in zip(got, given))
    hm = [x.transpose(0, 1).contiguous() for x in (t["Kn"], t["Vn"])]
    out["grad head"] = B.dodo_nugget_attention_grad(a[0], *hm, *a[3:], *cu, 20, 20, 35, layout=B.HEAD_MAJOR)
    assert out["grad head"][1].shape == (2, 30, 64)
    seg = (t["cu_q"], t["ns"], t["nl"], t["ls"], t["ll"])
    out["segments"] = B.dodo_nugget_attention_segments_grad(*a, *seg, 20, 25, 35, 0.125)
    given = [torch.empty_like(x) for x in a[:5]]
    got = out["segments given"] = B.dodo_nugget_attention_segments_grad(*a, *seg, 20, 25, 35, 0.125, 0, *given, ws=ws)
    assert all(x is y for x, y in zip(got, given))
    g = (t["Kn"], t["Vn"], t["idx"], t["cu_s"], t["cu_k"], 300)
    out["gather grad"] = B.dodo_gather_nuggets_grad(*g)
    dK, dV = t["K"].clone(), t["V"].clone()
    got = out["gather grad added"] = B.dodo_gather_nuggets_grad(*g, 0, dK, dV, True)
    assert got[0] is dK and got[1] is dV
    out["gather grad head"] = B.dodo_gather_nuggets_grad(*hm, *g[2:], layout=B.HEAD_MAJOR)
    p = (t["K"], t["V"], t["idx"], t["cu_s"], t["cu_k"], 30)
    cache = out["pack"] = B.dodo_gather_nuggets_q4(*p)
    mine = [torch.empty_like(x) for x in cache]
    got = out["pack given"] = B.dodo_gather_nuggets_q4(*p, 0, *mine)
    assert all(x is y for x, y in zip(got, mine))
    head = out["pack head"] = B.dodo_gather_nuggets_q4(*p, B.HEAD_MAJOR)
    out["unpack"] = B.dodo_unpack_nuggets_q4(*cache, t["K"].dtype)
    given = [torch.empty(30, 2, 64, device="cuda") for _ in range(2)]
    got = out["unpack given"] = B.dodo_unpack_nuggets_q4(*cache, torch.float32, *given)
    assert got[0] is given[0] and got[1] is given[1]
    q = (t["Kl"], t["Vl"], *cu, 20, 20, 35)
    out["attention"] = B.dodo_nugget_attention_q4(t["Q"], *cache, *q)[:1]
    O = torch.empty_like(t["Q"])
    got = out["attention lse"] = B.dodo_nugget_attention_q4(t["Q"], *cache, *q, 0.2, 0, O, want_lse=True)
    assert got[0] is O and got[1].shape == (40, 4)
    lse = torch.empty(40, 4, device="cuda")
    zeros = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    got = out["attention head"] = B.dodo_nugget_attention_q4(t["Q"], *head, *q, 0.2, B.HEAD_MAJOR, lse=lse, ws=zeros)
    assert got[1] is lse
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_same_results_as_through_ctypes(dtype, native):
    t = inputs(dtype)
    done = native(True)
    fast = calls(t)
    assert set(done) == set(NAMES)
    native(False)
    slow = calls(t)
    for name in slow:
        for x, y in zip(fast[name], slow[name], strict=True):
            assert x.shape == y.shape and x.dtype == y.dtype and torch.equal(x, y), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_apart(dtype, native):
    """K and V (or their gradients) as two halves of one tensor, and K alone with another stride, which is refused."""
    t = inputs(dtype)
    for on in (True, False):
        native(on)
        both = torch.full((300, 2, 2, 64), 7.0, dtype=dtype, device="cuda")
        got = B.dodo_gather_nuggets_grad(t["Kn"], t["Vn"], t["idx"], t["cu_s"], t["cu_k"], 300, 0, both[:, 0], both[:, 1])
        want = B.dodo_gather_nuggets_grad(t["Kn"], t["Vn"], t["idx"], t["cu_s"], t["cu_k"], 300)
        assert torch.equal(both[:, 0], want[0]) and torch.equal(both[:, 1], want[1]) and got[0].data_ptr() == both.data_ptr()
        kv = torch.stack((t["K"], t["V"]), 1)
        cache = B.dodo_gather_nuggets_q4(kv[:, 0], kv[:, 1], t["idx"], t["cu_s"], t["cu_k"], 30)
        assert all(torch.equal(x, y) for x, y in zip(cache, B.dodo_gather_nuggets_q4(t["K"], t["V"], t["idx"], t["cu_s"], t["cu_k"], 30)))
        with pytest.raises(ValueError):
            B.dodo_gather_nuggets_grad(t["Kn"], t["Vn"], t["idx"], t["cu_s"], t["cu_k"], 300, 0, both[:, 0], t["V"])
        with pytest.raises(ValueError):
            B.dodo_gather_nuggets_q4(kv[:, 0], t["V"], t["idx"], t["cu_s"], t["cu_k"], 30)


def test_refusals_are_the_same(native):
    t = inputs(torch.bfloat16)
    a = {n: t[n] for n in ("Q", "Kn", "Vn", "Kl", "Vl", "dO", "O", "lse")}
    cu = (t["cu_q"], t["cu_k"], t["cu_l"])
    native(False)
    cache = B.dodo_gather_nuggets_q4(t["K"], t["V"], t["idx"], t["cu_s"], t["cu_k"], 30)
    wrong = {"Q": t["Q"].float(), "dO": t["dO"][:-1], "O": t["O"].float(), "lse": t["lse"].double(), "Kn": t["Kn"].transpose(0, 1), "Vl": t["Vl"].cpu()}
    said = {}
    for on in (False, True):
        native(on)

        def refused(key, f, *args, **kw):
            with pytest.raises((ValueError, RuntimeError, TypeError)) as e:
                f(*args, **kw)
            assert said.setdefault(key, (type(e.value), str(e.value))) == (type(e.value), str(e.value)), key

        for name, x in wrong.items():
            refused(("grad", name), B.dodo_nugget_attention_grad, *{**a, name: x}.values(), *cu, 20, 20, 35)
        refused("cu", B.dodo_nugget_attention_grad, *a.values(), t["cu_q"], t["cu_k"][:-1], t["cu_l"], 20, 20, 35)
        refused("cu int64", B.dodo_nugget_attention_grad, *a.values(), t["cu_q"].long(), *cu[1:], 20, 20, 35)
        refused("ws", B.dodo_nugget_attention_grad, *a.values(), *cu, 20, 20, 35, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
        refused("dQ", B.dodo_nugget_attention_grad, *a.values(), *cu, 20, 20, 35, dQ=torch.empty(40, 4, 32, dtype=torch.bfloat16, device="cuda"))
        refused("max", B.dodo_nugget_attention_grad, *a.values(), *cu, -1, 20, 35)
        refused("heads", B.dodo_nugget_attention_grad, *{**a, **{n: a[n][:, :3].contiguous() for n in ("Q", "dO", "O", "lse")}}.values(), *cu, 20, 20, 35)
        refused("lens", B.dodo_nugget_attention_segments_grad, *a.values(), t["cu_q"], t["ns"], t["nl"], t["ls"], t["ll"][:-1], 20, 25, 35)
        refused("rows", B.dodo_gather_nuggets_grad, t["Kn"], t["Vn"], t["idx"][:20], t["cu_s"], t["cu_k"], 300)
        refused("one", B.dodo_gather_nuggets_grad, t["Kn"], t["Vn"], t["idx"], t["cu_s"], t["cu_k"], 300, 0, t["K"])
        refused("nothing to add to", B.dodo_gather_nuggets_grad, t["Kn"], t["Vn"], t["idx"], t["cu_s"], t["cu_k"], 300, accumulate=True)
        refused("pack one", B.dodo_gather_nuggets_q4, t["K"], t["V"], t["idx"], t["cu_s"], t["cu_k"], 30, 0, cache[0])
        refused("unpack type", B.dodo_unpack_nuggets_q4, *cache, torch.float16)
        refused("codes", B.dodo_unpack_nuggets_q4, cache[0], cache[1][:-1], *cache[2:])
        q = (t["Kl"], t["Vl"], *cu, 20, 20, 35)
        refused("scales", B.dodo_nugget_attention_q4, t["Q"], cache[0], cache[1].float(), *cache[2:], *q)
        refused("layout", B.dodo_nugget_attention_q4, t["Q"], *cache, *q, layout=2)
        refused("O", B.dodo_nugget_attention_q4, t["Q"], *cache, *q, O=t["Q"].float())
        refused("host", B.dodo_nugget_attention_q4, t["Q"].cpu(), *cache, *q)
