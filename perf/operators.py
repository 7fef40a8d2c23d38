"""Training and small-cache operators around nugget attention, as cases to be timed.

A case is a dict of plain values; its ``op`` names one operator:

``attention_grad``  the backward pass of nugget attention: dQ, dKn, dVn, dKl, dVl from dO, O and the log-sum-exp of the
                    forward pass, the probabilities recomputed.  With ``seg`` the ranges are the segments of the
                    autoregressive objective (Sec. 2.4) over whole texts, which share nuggets and local rows, and the cache's
                    gradient is added to the texts' own (``gather_grad`` in its accumulating form).
``gather_grad``     the gradient of the gather (Eq. 5): the cache's gradient rows go back to the tokens they came from.
``cache_q4``        the chosen tokens' K/V rows into a nugget cache held in 4 bits, and the same cache read back.
``attention_q4``    nugget attention (Eq. 9, Eq. 13) over such a cache.

Where ``own`` is false, ``run`` computes the operators in elementary torch operations.  Ragged lengths are a function of the
case alone, tensor values of the seed.

The 4-bit cache: 32 consecutive channels of a row and head share a scale 2^e, held as the byte e + 127, where e is the least
whole number with max|x| <= 7 * 2^e, between -125 and 125; a channel is a sign and one of the magnitudes 0, 0.5, 1, 1.5, 2, 3,
4, 6 (their index in 3 bits) of x / 2^e, the nearest, ties to the even index; channel 2i sits in the lower half of byte i.
A block with a NaN or an infinity has the scale byte 255 and reads as NaN.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_DEFAULTS = dict(dtype="bf16", H=32, H_kv=32, d_h=128, den=10, tau=0, q=1, q_lo=0, seg=0, head_major=False, layers=1)
_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # backward of one layer of a toy model in fp32: launches are all there is
        dict(name="grad_tiny_fp32", op="attention_grad", dtype="fp32", B=1, n_lo=512, n_hi=512, H=4, H_kv=4, d_h=64, q=32, tau=16),
        # training step of one 7B-shaped layer in the compressor mode: 8 contexts of 4096 tokens at 10x, 512 query rows
        dict(name="grad_prefill_7b", op="attention_grad", B=8, n_lo=4096, n_hi=4096, q=512, tau=128),
        # autoencoding of one 13B-shaped layer: 16 contexts of 2048 tokens at 20x, every token decoded again (the largest)
        dict(name="grad_autoencode_13b", op="attention_grad", B=16, n_lo=2048, n_hi=2048, H=40, H_kv=40, den=20, q=2048),
        # ragged documents under grouped-query heads, cache by heads: sequences of a few rows up to several hundred
        dict(name="grad_gqa_ragged", op="attention_grad", B=5, n_lo=500, n_hi=4100, H=64, H_kv=8, q=777, q_lo=3, tau=33, head_major=True),
        # the autoregressive objective over whole texts, up to the gradient of every token's K and V: segments of 512 tokens,
        # 128 tokens of overlap
        dict(name="grad_segments_7b", op="attention_grad", B=4, n_lo=3500, n_hi=4096, seg=512, tau=128),
        # the gradient of prefill's cache on its way to the context's K and V: mostly zeros are written
        dict(name="gather_grad_7b", op="gather_grad", B=8, n_lo=4096, n_hi=4096),
        # three layers of short ragged documents, cache by heads
        dict(name="gather_grad_layers", op="gather_grad", B=4, n_lo=320, n_hi=1280, layers=3, head_major=True),
        # the caches of prefill in 4 bits
        dict(name="cache_q4_7b", op="cache_q4", B=8, n_lo=4096, n_hi=4096),
        # a single short document, heads of 64, cache by heads
        dict(name="cache_q4_short", op="cache_q4", B=1, n_lo=878, n_hi=878, H=16, H_kv=16, d_h=64, head_major=True),
        # one user's decode step
        dict(name="attention_q4_one", op="attention_q4", B=1, n_lo=4099, n_hi=4099, tau=256),
        # a serving batch's decode step: long ragged contexts, grouped-query heads
        dict(name="attention_q4_batch", op="attention_q4", B=32, n_lo=16384, n_hi=32768, H=64, H_kv=8, tau=256),
        # a prompt read over the compressed contexts of prefill
        dict(name="attention_q4_prefill", op="attention_q4", B=8, n_lo=4096, n_hi=4096, q=512, tau=128),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm; odd sizes come as often as they do."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 5e14


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("attention_grad", "gather_grad", "cache_q4", "attention_q4")}
    while True:
        op = rng.choice(["attention_grad", "attention_grad", "attention_grad", "gather_grad", "cache_q4", "attention_q4", "attention_q4",
                         "attention_q4"])
        H, H_kv, d_h = rng.choice([(32, 32, 128), (32, 32, 128), (40, 40, 128), (64, 8, 128), (32, 8, 128), (16, 16, 64), (8, 2, 64)])
        c = dict(op=op, H=H, H_kv=H_kv, d_h=d_h, den=rng.choice([5, 10, 20]), head_major=rng.random() < 0.3)
        if rng.random() < 0.15:  # toy models, fp32
            H = rng.choice([2, 4, 8])
            c.update(dtype="fp32", H=H, H_kv=H // rng.choice([1, 2]), d_h=64)
        toy = "dtype" in c
        if op == "attention_grad":
            if rng.random() < 0.25:
                c.update(B=_log(rng, 1, 4), n_hi=_log(rng, 200, 1500 if toy else 6000), seg=rng.choice([64, 100, 256, 512]),
                         tau=rng.randint(0, 200))
            else:
                c.update(B=_log(rng, 1, 3 if toy else 16), n_hi=_log(rng, 64, 1500 if toy else 16384), q=_log(rng, 1, 64 if toy else 2048),
                         tau=rng.randint(0, 200))
                c["q_lo"] = rng.randint(1, c["q"]) if rng.random() < 0.5 else 0
        elif op in ("gather_grad", "cache_q4"):
            c.update(B=_log(rng, 1, 16), n_hi=_log(rng, 64, 16384), layers=rng.choice([1, 1, 1, 3]))
        else:
            c.update(B=_log(rng, 1, 64), n_hi=_log(rng, 100, 32768), tau=_log(rng, 1, 1200), q=rng.choice([1, 1, 1, 1, 4, _log(rng, 2, 1024)]))
        # ragged batches as often as even ones
        c["n_lo"] = max(1, int(c["n_hi"] * rng.uniform(0.3, 1.0))) if rng.random() < 0.5 else c["n_hi"]
        if _cost(c) <= most[op]:
            return c


def _ragged(tag, lo, hi, count):
    """`count` whole numbers between lo and hi: a function of its arguments alone."""
    r = random.Random("%s %d %d %d" % (tag, lo, hi, count))
    return [r.randint(lo, hi) for _ in range(count)]


def _full(case):
    """The case with its defaults, and its entries: (query rows, nugget rows, local rows) as ranges (first, length)."""
    c = dict(_DEFAULTS, **case)
    c["lens"] = _ragged("tokens", c["n_lo"], c["n_hi"], c["B"])
    c["ks"] = [max(1, -(-n // c["den"])) for n in c["lens"]]
    c["N"], c["Kt"] = sum(c["lens"]), sum(c["ks"])
    c["G"] = c["H"] // c["H_kv"]
    if c["seg"]:
        c["q_lens"] = c["m_lens"] = c["lens"]
    else:
        c["q_lens"] = _ragged("queries", c["q_lo"], c["q"], c["B"]) if c["q_lo"] else [c["q"]] * c["B"]
        c["m_lens"] = [q + c["tau"] for q in c["q_lens"]]
    c["Sq"], c["Sm"] = sum(c["q_lens"]), sum(c["m_lens"])
    return c


def _starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _index_lists(c):
    """Ascending nugget indices of every sequence (host lists, a function of the case)."""
    r = random.Random("nuggets %d %d %d" % (c["N"], c["Kt"], c["B"]))
    return [sorted(r.sample(range(n), k)) for n, k in zip(c["lens"], c["ks"])]


def _entries(c):
    """(first query row, rows, first nugget, nuggets, first local row, local rows) of every sequence or segment."""
    q, k, m = _starts(c["q_lens"]), _starts(c["ks"]), _starts(c["m_lens"])
    if not c["seg"]:
        return [(q[b], c["q_lens"][b], k[b], c["ks"][b], m[b], c["m_lens"][b]) for b in range(c["B"])]
    out, lists = [], _index_lists(c)
    for b, n in enumerate(c["lens"]):
        for s in range(0, n, c["seg"]):
            t, e = max(0, s - c["tau"]), min(n, s + c["seg"])
            out.append((q[b] + s, e - s, k[b], sum(1 for i in lists[b] if i < t), q[b] + t, e - t))
    return out


def _pairs(q, k, m):
    """Visible (query row, key) pairs: all nuggets, local row j of m for query row i of q if j <= m - q + i."""
    return q * k + sum(max(0, min(m, m - q + i + 1)) for i in range(q))


def work(case):
    c = _full(case)
    es = 4 if c["dtype"] == "fp32" else 2
    d_h, L = c["d_h"], c["layers"]
    kv_row, q_row = 2 * c["H_kv"] * d_h * es, c["H"] * d_h * es  # K and V of a token; a query row
    q4_row = 2 * c["H_kv"] * (d_h // 2 + d_h // 32)
    if c["op"] == "attention_grad":
        pairs = sum(_pairs(q, k, m) for _, q, _, k, _, m in _entries(c))
        return {"bytes": 4 * c["Sq"] * q_row + 4 * c["Sq"] * c["H"] + 2 * (c["Kt"] + c["Sm"]) * kv_row, "flops": 10 * d_h * c["H"] * pairs}
    if c["op"] == "gather_grad":
        return {"bytes": L * (c["Kt"] + c["N"]) * kv_row + 4 * c["Kt"], "flops": 0}
    if c["op"] == "cache_q4":
        return {"bytes": L * c["Kt"] * (2 * kv_row + 2 * q4_row) + 4 * c["Kt"], "flops": 0}
    pairs = sum(_pairs(q, k, m) for _, q, _, k, _, m in _entries(c))
    return {"bytes": c["Kt"] * q4_row + c["Sm"] * kv_row + 2 * c["Sq"] * q_row, "flops": 4 * d_h * c["H"] * pairs}


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _quantise(x):
    """Codes [..., d/2] and scale bytes [..., d/32] of x [..., d]."""
    blocks = x.float().unflatten(-1, (-1, 32))
    top = blocks.abs().amax(-1)
    bad = ~torch.isfinite(blocks).all(-1)
    mant, exp = torch.frexp(torch.where(bad, torch.ones_like(top), top))  # top = mant * 2^exp, mant in [0.5, 1)
    e = torch.where(mant <= 0.875, exp - 3, exp - 2)
    e = torch.where(top == 0, torch.full_like(e, -125), e).clamp(-125, 125)
    a = torch.ldexp(blocks.abs().double(), -e.unsqueeze(-1)).float()
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() +
            (a > 5.0).int())
    code = (code + 8 * torch.signbit(blocks).int()).flatten(-2)
    scale = torch.where(bad, torch.full_like(e, 255), e + 127)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), scale.to(torch.uint8)


def _dequantise(codes, scales):
    """fp32 values of codes [..., d/2] under scale bytes [..., d/32]."""
    grid = torch.tensor(_MAGNITUDES + tuple(-m for m in _MAGNITUDES), device=codes.device)
    nibbles = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    scale = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127)
    scale = torch.where(scales == 255, torch.full_like(scale, float("nan")), scale)
    return (grid[nibbles].unflatten(-1, (-1, 32)) * scale.unsqueeze(-1)).flatten(-2)


def _by_head(x, G=1):
    """[rows, H, d] -> [H / G, G * rows, d] in fp32: the heads that share a K/V head side by side."""
    rows, H, d = x.shape
    return x.float().transpose(0, 1).reshape(H // G, G * rows, d)


def _rows(x, G=1):
    """The reverse of _by_head."""
    return x.reshape(x.shape[0] * G, -1, x.shape[2]).transpose(0, 1)


def _visible(q, k, m, G, device):
    """[G * q, k + m]: query row i sees all nuggets, and local row j if j <= m - q + i."""
    i, j = torch.arange(q, device=device), torch.arange(m, device=device)
    local = j[None, :] <= (m - q + i)[:, None]
    return torch.cat((torch.ones((q, k), dtype=torch.bool, device=device), local), 1).repeat(G, 1)


def _plain_attention(Q, Kn, Vn, Kl, Vl, entries, scale, G):
    """Token-major caches in fp32; O [Sq, H, d] and lse [Sq, H] in fp32."""
    O = torch.zeros(Q.shape, dtype=torch.float32, device=Q.device)
    lse = torch.full(Q.shape[:2], -math.inf, dtype=torch.float32, device=Q.device)
    for q0, q, k0, k, l0, m in entries:
        if q == 0 or k + m == 0:
            continue
        Qe = _by_head(Q[q0:q0 + q], G)
        K = _by_head(torch.cat((Kn[k0:k0 + k].float(), Kl[l0:l0 + m].float())))
        V = _by_head(torch.cat((Vn[k0:k0 + k].float(), Vl[l0:l0 + m].float())))
        S = torch.matmul(Qe, K.transpose(1, 2).contiguous()) * scale
        S.masked_fill_(~_visible(q, k, m, G, Q.device), -math.inf)
        top = S.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        P = torch.exp(S.sub_(top))
        total = P.sum(-1, keepdim=True)
        out = torch.matmul(P, V) / torch.where(total == 0, torch.ones_like(total), total)
        O[q0:q0 + q] = _rows(out, G)
        lse[q0:q0 + q] = _rows(top + torch.log(total), G)[..., 0]
    return O, lse


def _plain_attention_grad(s):
    c, G, scale = s["c"], s["c"]["G"], s["scale"]
    Kn, Vn = _token_major(s, "Kn"), _token_major(s, "Vn")
    dQ = torch.zeros(s["Q"].shape, dtype=torch.float32, device="cuda")
    dKn, dVn = (torch.zeros(Kn.shape, dtype=torch.float32, device="cuda") for _ in range(2))
    dKl, dVl = (torch.zeros(s["Kl"].shape, dtype=torch.float32, device="cuda") for _ in range(2))
    for q0, q, k0, k, l0, m in s["entries"]:
        if q == 0 or k + m == 0:
            continue
        rows = slice(q0, q0 + q)
        Qe, dOe, Oe = (_by_head(s[name][rows], G) for name in ("Q", "dO", "O"))
        K = _by_head(torch.cat((Kn[k0:k0 + k].float(), s["Kl"][l0:l0 + m].float())))
        V = _by_head(torch.cat((Vn[k0:k0 + k].float(), s["Vl"][l0:l0 + m].float())))
        lse = s["lse"][rows].t().reshape(c["H_kv"], G * q, 1)
        D = (dOe * Oe).sum(-1, keepdim=True)
        P = torch.matmul(Qe, K.transpose(1, 2).contiguous()).mul_(scale).sub_(lse).exp_()
        P.masked_fill_(~_visible(q, k, m, G, "cuda"), 0.0)
        dS = torch.matmul(dOe, V.transpose(1, 2).contiguous()).sub_(D).mul_(P)
        dV = _rows(torch.matmul(P.transpose(1, 2).contiguous(), dOe))
        dK = _rows(torch.matmul(dS.transpose(1, 2).contiguous(), Qe)) * scale
        dQ[rows] = _rows(torch.matmul(dS, K), G) * scale
        dKn[k0:k0 + k] += dK[:k]
        dVn[k0:k0 + k] += dV[:k]
        dKl[l0:l0 + m] += dK[k:]
        dVl[l0:l0 + m] += dV[k:]
    dQ, dKn, dVn, dKl, dVl = (t.to(s["Q"].dtype) for t in (dQ, dKn, dVn, dKl, dVl))
    if c["seg"]:
        for total, part in ((dKl, dKn), (dVl, dVn)):
            total[s["tokens"]] = (total[s["tokens"]].float() + part.float()).to(total.dtype)
    if c["head_major"]:
        dKn, dVn = dKn.transpose(0, 1).contiguous(), dVn.transpose(0, 1).contiguous()
    return [dQ, dKn, dVn, dKl, dVl]


def _plain_gather_grad(s):
    c = s["c"]
    out = []
    for name in ("K", "V"):
        d = s["d" + name + "n"].float()
        if c["head_major"]:
            d = d.transpose(1, 2)
        full = torch.zeros((c["layers"], c["N"], c["H_kv"], c["d_h"]), dtype=torch.float32, device="cuda")
        full[:, s["tokens"]] = d
        out.append(full.to(_DTYPES[c["dtype"]]))
    return out


def _plain_cache_q4(s):
    out = []
    for name in ("K", "V"):
        rows = s[name][:, s["tokens"]]
        if s["c"]["head_major"]:
            rows = rows.transpose(1, 2)
        out.append(_dequantise(*_quantise(rows)).to(s[name].dtype))
    return out


def _plain_attention_q4(s):
    c = s["c"]
    Kn, Vn = _dequantise(s["Kc"], s["Ks"]), _dequantise(s["Vc"], s["Vs"])
    if c["head_major"]:
        Kn, Vn = Kn.transpose(0, 1), Vn.transpose(0, 1)
    O, _ = _plain_attention(s["Q"], Kn, Vn, s["Kl"], s["Vl"], s["entries"], s["scale"], c["G"])
    return O.to(s["Q"].dtype)


def _token_major(s, name):
    return s[name].transpose(0, 1) if s["c"]["head_major"] else s[name]


# ---- the framework's operators ---------------------------------------------------------------------------------------

def _own_attention_grad(s):
    import paper_2310_02409_amd as D
    if s["c"]["seg"]:
        dQ, dKn, dVn, dK, dV = D.dodo_nugget_attention_segments_grad(
            s["Q"], s["Kn"], s["Vn"], s["Kl"], s["Vl"], s["dO"], s["O"], s["lse"], *s["plan"], s["max_q"], s["max_k"], s["max_m"], s["scale"],
            s["layout"], ws=s["ws"])
        D.dodo_gather_nuggets_grad(dKn, dVn, s["idx"], s["cu_seqlens"], s["cu_nuggets"], s["c"]["N"], s["layout"], dK, dV, True)
        return dQ, dKn, dVn, dK, dV
    return D.dodo_nugget_attention_grad(s["Q"], s["Kn"], s["Vn"], s["Kl"], s["Vl"], s["dO"], s["O"], s["lse"], s["cu_q"], s["cu_nuggets"],
                                        s["cu_local"], s["max_q"], s["max_k"], s["max_m"], s["scale"], s["layout"], ws=s["ws"])


def _own_gather_grad(s):
    import paper_2310_02409_amd as D
    c = s["c"]
    if c["layers"] == 1:
        dK, dV = D.dodo_gather_nuggets_grad(s["dKn"][0], s["dVn"][0], s["idx"], s["cu_seqlens"], s["cu_nuggets"], c["N"], s["layout"])
        return [dK[None], dV[None]]
    return list(D.dodo_gather_nuggets_grad_layers(s["dKn"], s["dVn"], s["idx"], s["cu_seqlens"], s["cu_nuggets"], c["N"], s["layout"]))


def _own_cache_q4(s):
    import paper_2310_02409_amd as D
    if s["c"]["layers"] == 1:
        q4 = D.dodo_gather_nuggets_q4(s["K"][0], s["V"][0], s["idx"], s["cu_seqlens"], s["cu_nuggets"], s["c"]["Kt"], s["layout"])
    else:
        q4 = D.dodo_gather_nuggets_q4_layers(s["K"], s["V"], s["idx"], s["cu_seqlens"], s["cu_nuggets"], s["c"]["Kt"], s["layout"])
    Kn, Vn = D.dodo_unpack_nuggets_q4(*q4, dtype=s["K"].dtype)
    return [t.view((s["c"]["layers"],) + tuple(t.shape[-3:])) for t in (Kn, Vn)]


def _own_attention_q4(s):
    import paper_2310_02409_amd as D
    O, _ = D.dodo_nugget_attention_q4(s["Q"], s["Kc"], s["Ks"], s["Vc"], s["Vs"], s["Kl"], s["Vl"], s["cu_q"], s["cu_nuggets"], s["cu_local"],
                                      s["max_q"], s["max_k"], s["max_m"], s["scale"], s["layout"], ws=s["ws"])
    return O


_PLAIN = dict(attention_grad=_plain_attention_grad, gather_grad=_plain_gather_grad, cache_q4=_plain_cache_q4, attention_q4=_plain_attention_q4)
_OWN = dict(attention_grad=_own_attention_grad, gather_grad=_own_gather_grad, cache_q4=_own_cache_q4, attention_q4=_own_attention_q4)


def prepare(case, seed):
    c = _full(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, H, H_kv, d_h, L = _DTYPES[c["dtype"]], c["H"], c["H_kv"], c["d_h"], c["layers"]
    normal = lambda *shape: torch.randn(shape, generator=g, dtype=dt, device="cuda")
    ints = lambda values: torch.tensor(values, dtype=torch.int32, device="cuda")
    s = dict(c=c, scale=d_h ** -0.5, layout=1 if c["head_major"] else 0, cu_nuggets=ints(_starts(c["ks"])))
    if c["op"] in ("gather_grad", "cache_q4") or c["seg"]:
        lists, first = _index_lists(c), _starts(c["lens"])
        s.update(idx=ints([i for l in lists for i in l]), cu_seqlens=ints(first),
                 tokens=torch.tensor([first[b] + i for b, l in enumerate(lists) for i in l], device="cuda"))
    if c["op"] in ("gather_grad", "cache_q4"):
        cache = (L, H_kv, c["Kt"], d_h) if c["head_major"] else (L, c["Kt"], H_kv, d_h)
        if c["op"] == "cache_q4":
            # keys have a few channels that are much larger than the rest, in every token alike
            spread = torch.exp(torch.randn((H_kv, d_h), generator=g, device="cuda")).to(dt)
            s.update(K=normal(L, c["N"], H_kv, d_h) * spread, V=normal(L, c["N"], H_kv, d_h))
        else:
            s.update(dKn=normal(*cache), dVn=normal(*cache))
        return s
    s["entries"] = _entries(c)
    s.update(max_q=max(e[1] for e in s["entries"]), max_k=max(c["ks"]), max_m=max(e[5] for e in s["entries"]),
             cu_q=ints(_starts(c["q_lens"])), cu_local=ints(_starts(c["m_lens"])), Q=normal(c["Sq"], H, d_h),
             Kl=normal(c["Sm"], H_kv, d_h), Vl=normal(c["Sm"], H_kv, d_h))
    Kn, Vn = normal(c["Kt"], H_kv, d_h), normal(c["Kt"], H_kv, d_h)
    by_head = (lambda t: t.transpose(0, 1).contiguous()) if c["head_major"] else (lambda t: t)
    if c["op"] == "attention_q4":
        s["Kc"], s["Ks"] = (by_head(t) for t in _quantise(Kn))
        s["Vc"], s["Vs"] = (by_head(t) for t in _quantise(Vn))
    else:
        s.update(Kn=by_head(Kn), Vn=by_head(Vn), dO=normal(c["Sq"], H, d_h))
        O, s["lse"] = _plain_attention(s["Q"], Kn, Vn, s["Kl"], s["Vl"], s["entries"], s["scale"], c["G"])
        s["O"] = O.to(dt)
        if c["seg"]:
            s["plan"] = (ints([e[0] for e in s["entries"]] + [c["Sq"]]),) + tuple(ints([e[i] for e in s["entries"]]) for i in (2, 3, 4, 5))
    s["ws"] = None
    if own:  # a training or serving loop keeps its workspace
        import paper_2310_02409_amd as D
        code, n = D.F32 if c["dtype"] == "fp32" else D.BF16, len(s["entries"])
        if c["op"] == "attention_q4":
            need = D.dodo_nugget_attention_q4_workspace_bytes(n, H, H_kv, d_h, s["max_q"], s["max_k"], s["max_m"], c["Kt"], code)
        else:
            need = D.dodo_nugget_attention_grad_workspace_bytes(n, H, H_kv, d_h, s["max_q"], s["max_k"], s["max_m"], c["Sq"], c["Kt"], c["Sm"],
                                                                code)
        s["ws"] = torch.zeros(max(16, need), dtype=torch.uint8, device="cuda")
    return s


def run(state):
    return (_OWN if own else _PLAIN)[state["c"]["op"]](state)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _values64(codes, scales):
    """What a 4-bit cache stands for, element by element: (-1)^s * 2^(E - 1) * (1 + M / 2), or M / 2 where E is 0."""
    n = torch.stack((codes.bitwise_and(15), codes.bitwise_right_shift(4)), dim=-1).reshape(*codes.shape[:-1], -1).double()
    sign = torch.where(n >= 8, -1.0, 1.0).double()
    n = n % 8
    E, M = torch.div(n, 2, rounding_mode="floor"), n % 2
    mag = torch.where(E == 0, M / 2, torch.pow(2.0, E - 1) * (1 + M / 2))
    scale = torch.pow(2.0, scales.double() - 127)
    scale[scales == 255] = math.nan
    return sign * mag * scale.repeat_interleave(32, dim=-1)


def _nearest64(x):
    """The 4-bit value of every element of x [..., d] in 64 bits, by the distance to each magnitude."""
    x = x.double()
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = b.abs().max(dim=-1, keepdim=True).values
    e = torch.full_like(top, -125.0)
    for step in range(-124, 126):  # the least e with top <= 7 * 2^e
        e = torch.where(top > 7 * 2.0 ** (step - 1), torch.full_like(e, float(step)), e)
    a = b.abs() / torch.pow(2.0, e)
    grid = (0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0)  # even indices first: they win ties
    best, dist = torch.zeros_like(a), torch.full_like(a, math.inf)
    for v in grid:
        d = (a - v).abs()
        best, dist = torch.where(d < dist, torch.full_like(best, v), best), torch.minimum(d, dist)
    return (torch.sign(b) * best * torch.pow(2.0, e)).reshape(x.shape)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = s["c"]
    if c["op"] == "cache_q4":
        out = []
        for name in ("K", "V"):
            v = _nearest64(torch.index_select(s[name], 1, s["tokens"]))
            out.append(v.permute(0, 2, 1, 3) if c["head_major"] else v)
        return out
    if c["op"] == "gather_grad":
        out = []
        for name in ("K", "V"):
            d = s["d" + name + "n"].double()
            if c["head_major"]:
                d = d.permute(0, 2, 1, 3)
            full = torch.zeros((c["layers"], c["N"], c["H_kv"], c["d_h"]), dtype=torch.float64, device="cuda")
            out.append(full.index_add_(1, s["tokens"], d.contiguous()))
        return out
    head = 0 if c["head_major"] else 1
    if c["op"] == "attention_q4":
        Kn, Vn = _values64(s["Kc"], s["Ks"]), _values64(s["Vc"], s["Vs"])
        O = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    else:
        Kn, Vn = s["Kn"].double(), s["Vn"].double()
        dQ = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
        dKn, dVn = torch.zeros_like(Kn), torch.zeros_like(Vn)
        dKl, dVl = (torch.zeros(s["Kl"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
    for q0, q, k0, k, l0, m in s["entries"]:
        hidden = torch.arange(m, device="cuda")[None, :] > torch.arange(m - q, m, device="cuda")[:, None]
        for h in range(c["H"]):  # one query head at a time
            kv = h * c["H_kv"] // c["H"]
            Kh = torch.cat((Kn.select(head, kv)[k0:k0 + k], s["Kl"][l0:l0 + m, kv].double()))
            Vh = torch.cat((Vn.select(head, kv)[k0:k0 + k], s["Vl"][l0:l0 + m, kv].double()))
            Qh = s["Q"][q0:q0 + q, h].double()
            xi = s["scale"] * (Qh @ Kh.T)
            xi[:, k:] = torch.where(hidden, -math.inf, xi[:, k:])
            if c["op"] == "attention_q4":
                O[q0:q0 + q, h] = torch.softmax(xi, -1) @ Vh
                continue
            dOh, lse = s["dO"][q0:q0 + q, h].double(), s["lse"][q0:q0 + q, h].double()
            p = torch.exp(xi - lse[:, None])
            p = torch.where(torch.isneginf(lse)[:, None], torch.zeros_like(p), p)
            back = p * (dOh @ Vh.T - (dOh * s["O"][q0:q0 + q, h].double()).sum(1)[:, None])
            dQ[q0:q0 + q, h] = s["scale"] * (back @ Kh)
            dK, dV = s["scale"] * (back.T @ Qh), p.T @ dOh
            dKn.select(head, kv)[k0:k0 + k] += dK[:k]
            dVn.select(head, kv)[k0:k0 + k] += dV[:k]
            dKl[l0:l0 + m, kv] += dK[k:]
            dVl[l0:l0 + m, kv] += dV[k:]
    if c["op"] == "attention_q4":
        return O
    if c["seg"]:
        for total, part in ((dKl, dKn), (dVl, dVn)):
            total.index_add_(0, s["tokens"], (part.permute(1, 0, 2) if c["head_major"] else part).contiguous())
    return [dQ, dKn, dVn, dKl, dVl]
