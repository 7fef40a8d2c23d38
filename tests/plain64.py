"""Plain implementations in 64 bits (torch on the CPU) of the operators around nugget attention: what the GPU tests compare with.

Entries are (first query row, rows, first nugget, nuggets, first local row, local rows); caches are token-major."""
import math

import torch

MAGNITUDES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def entries_of(q_lens, k_lens, m_lens):
    out, q, k, m = [], 0, 0, 0
    for a, b, c in zip(q_lens, k_lens, m_lens):
        out.append((q, a, k, b, m, c))
        q, k, m = q + a, k + b, m + c
    return out


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def _keys(Kn, Kl, e, kv):
    return torch.cat((Kn[e[2]:e[2] + e[3], kv], Kl[e[4]:e[4] + e[5], kv])).double()


def _mask(e):
    """[q, k + m]: query row i sees all nuggets, and local row j if j <= m - q + i."""
    q, k, m = e[1], e[3], e[5]
    local = torch.arange(m)[None, :] <= (m - q + torch.arange(q))[:, None]
    return torch.cat((torch.ones((q, k), dtype=torch.bool), local), 1)


def attention(Q, Kn, Vn, Kl, Vl, entries, scale):
    """O [Sq, H, d_h] and lse [Sq, H] in 64 bits; a row that sees nothing gives 0 and -inf."""
    Sq, H, _ = Q.shape
    O, lse = torch.zeros(Q.shape, dtype=torch.float64), torch.full((Sq, H), -math.inf, dtype=torch.float64)
    for e in entries:
        rows = slice(e[0], e[0] + e[1])
        for h in range(H):
            kv = h // (H // Kl.shape[1])
            x = (Q[rows, h].double() @ _keys(Kn, Kl, e, kv).T) * scale
            x = torch.where(_mask(e), x, -math.inf)
            if x.shape[1] == 0:
                continue
            lse[rows, h] = torch.logsumexp(x, 1)
            P = torch.exp(x - torch.where(torch.isinf(lse[rows, h]), 0.0, lse[rows, h])[:, None])
            O[rows, h] = P @ _keys(Vn, Vl, e, kv)
    return O, lse


def attention_grad(Q, Kn, Vn, Kl, Vl, dO, O, lse, entries, scale):
    """(dQ, dKn, dVn, dKl, dVl) in 64 bits, and for each the sums of the same terms' magnitudes that its error is measured by: with
    the factor P or dS of a term as it is, and with dS's two parts added in magnitude (what cancels in dS is rounded too); and the
    largest sum of magnitudes in a logit."""
    H, H_kv = Q.shape[1], Kl.shape[1]
    z = lambda t: torch.zeros(t.shape, dtype=torch.float64)
    g = [z(Q), z(Kn), z(Vn), z(Kl), z(Vl)]
    near = [z(Q), z(Kn), z(Vn), z(Kl), z(Vl)]
    wide = [z(Q), z(Kn), z(Vn), z(Kl), z(Vl)]
    most = 0.0
    for e in entries:
        rows, nug, loc, k = slice(e[0], e[0] + e[1]), slice(e[2], e[2] + e[3]), slice(e[4], e[4] + e[5]), e[3]
        if e[1] == 0 or e[3] + e[5] == 0:
            continue
        for h in range(H):
            kv = h // (H // H_kv)
            K, V = _keys(Kn, Kl, e, kv), _keys(Vn, Vl, e, kv)
            q, do, o, l = Q[rows, h].double(), dO[rows, h].double(), O[rows, h].double(), lse[rows, h].double()
            x = (q @ K.T) * scale
            most = max(most, float(((q.abs() @ K.abs().T) * abs(scale)).max()))
            P = torch.where(_mask(e) & ~torch.isneginf(l)[:, None], torch.exp(x - l[:, None]), 0.0)
            dS = P * (do @ V.T - (do * o).sum(1)[:, None])
            dS_wide = P * (do.abs() @ V.abs().T + (do * o).abs().sum(1)[:, None])
            for out, s, p, K_, q_, do_ in ((g, dS, P, K, q, do), (near, dS.abs(), P, K.abs(), q.abs(), do.abs()),
                                           (wide, dS_wide, P, K.abs(), q.abs(), do.abs())):
                c = scale if out is g else abs(scale)
                out[0][rows, h] += c * (s @ K_)
                dK, dV = c * (s.T @ q_), p.T @ do_
                out[1][nug, kv] += dK[:k]
                out[2][nug, kv] += dV[:k]
                out[3][loc, kv] += dK[k:]
                out[4][loc, kv] += dV[k:]
    return g, near, wide, most


def grad_tolerance(ref, near, wide, most, terms, d_h, dtype):
    """What a gradient computed as the library does may be off by, element by element.  The result is rounded once; with bf16
    inputs P and dS are rounded to bf16 before the second product (half a step of each term).  fp32 sums: a chain of `terms`
    additions, the d_h products of a logit (relative to its magnitudes, at most `most`, whose error is P's relative error), of
    dP and of D, each with d_h roundings, and 64 for exponentials and scales."""
    fp32 = 2.0 ** -24 * (terms + (d_h + 64) * (1 + most))
    tol = half_step(dtype) * ref.abs() + fp32 * wide
    if dtype == torch.bfloat16:
        tol = tol + half_step(dtype) * (1 + half_step(dtype)) * near
    return tol + 1e-30


def gather_grad(dKn, tokens, N, base=None):
    """Rows of dKn [Kt, H_kv, d_h] summed into their tokens' rows of base (zeros)."""
    out = torch.zeros((N,) + tuple(dKn.shape[1:]), dtype=torch.float64) if base is None else base.double()
    return out.index_add(0, tokens, dKn.double())


def quantise_q4(x):
    """Codes [..., d/2] and scale bytes [..., d/32] (uint8) of x [..., d], by the format's definition, element by element."""
    b = x.double().unflatten(-1, (x.shape[-1] // 32, 32))
    top = b.abs().amax(-1)
    bad = ~torch.isfinite(b).all(-1)
    safe = torch.where(bad, torch.ones_like(top), top)
    e = torch.full_like(safe, -125.0)
    for step in range(-124, 126):
        e = torch.where(safe > 7 * 2.0 ** (step - 1), torch.full_like(e, float(step)), e)
    a = torch.where(bad[..., None], torch.zeros_like(b), b.abs() / torch.pow(2.0, e)[..., None])
    best, dist = torch.zeros_like(a), torch.full_like(a, math.inf)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):  # (even codes first: they win ties)
        d = (a - MAGNITUDES[code]).abs()
        best, dist = torch.where(d < dist, torch.full_like(best, code), best), torch.minimum(d, dist)
    code = (best + torch.where(torch.signbit(b) & ~bad[..., None], 8.0, 0.0)).to(torch.int32).flatten(-2)
    scale = torch.where(bad, torch.full_like(e, 255.0), e + 127)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), scale.to(torch.uint8)


def values_q4(codes, scales):
    """What codes [..., d/2] under scale bytes [..., d/32] stand for, in 64 bits."""
    n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    v = torch.where(n >= 8, -1.0, 1.0).double() * MAGNITUDES[n % 8]
    s = torch.where(scales == 255, math.nan, torch.pow(2.0, scales.double() - 127))
    return v * s.repeat_interleave(32, -1)
