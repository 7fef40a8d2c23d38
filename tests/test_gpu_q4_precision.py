"""Attention over 4-bit caches where the codes are read in place: weights count with two bf16 parts, within a bound that one part breaks.

Queries and keys are small whole numbers (and halves), whose products fp32 sums exactly, so that a bound of a few roundings holds."""
import math

import pytest
import torch

import plain64 as P64
import test_gpu_q4 as Q4

BF16 = torch.bfloat16
# up to 15 rows, or up to 128 query vectors a K/V head, and up to 32 heads a K/V head: 16 and 32 vectors at a time, in one share and several
CASES = [(([1], [60], [40]), 16, 16, 128), (([1, 1, 1], [100, 33, 0], [57, 0, 5]), 16, 2, 64), (([1], [410], [120]), 64, 8, 128),
         (([15, 9], [100, 70], [15, 60]), 8, 4, 64), (([40, 17], [120, 100], [90, 17]), 6, 2, 128), (([128], [65], [100]), 2, 2, 64),
         (([4], [300], [40]), 32, 1, 128), (([1], [700], [60]), 32, 2, 64), (([20], [500], [70]), 8, 4, 128)]


def inputs(lens, H, H_kv, d_h):
    t = Q4.attention_case(75, *lens, H, H_kv, d_h, BF16)
    whole = lambda x, most: torch.clamp(torch.round(x.float()), -most, most).to(BF16)
    t["Q"], t["Kl"] = whole(t["Q"], 2), whole(t["Kl"], 3)
    t["Ks"][:] = 127
    t["Kc"] &= 0xbb  # (magnitudes up to 1.5)
    return t


def reference(t, lens, scale, as_kept=lambda w: w):
    """O in 64 bits (its weights as `as_kept` has them when they meet V), and its bound.  A weight's upper part keeps 8 of its bits, so the rest
    is below 2^-7 of it, and rounds to bf16 by half a step, 2^-8: 2^-15 of each term.  fp32: a chain of additions as long as there are
    keys, at most 8 roundings of a logit and its offset (exact sums times a scale, in base 2), 64 for the exponential, the merges and the
    division, of the weights and of their sum.  The result is rounded once."""
    entries, H = P64.entries_of(*lens), t["Q"].shape[1]
    Kn, Vn = P64.values_q4(t["Kc"], t["Ks"]), P64.values_q4(t["Vc"], t["Vs"])
    O, size = torch.zeros(t["Q"].shape, dtype=torch.float64), torch.zeros(t["Q"].shape, dtype=torch.float64)
    logit = 0.0
    for e in entries:
        rows = slice(e[0], e[0] + e[1])
        for h in range(H):
            kv = h // (H // t["Kl"].shape[1])
            K, V = P64._keys(Kn, t["Kl"], e, kv), P64._keys(Vn, t["Vl"], e, kv)
            x = (t["Q"][rows, h].double() @ K.T) * scale
            logit = max(logit, float(x.abs().max()))
            x = torch.where(P64._mask(e), x, -math.inf)
            w = torch.exp(x - x.amax(1, keepdim=True))
            total = w.sum(1, keepdim=True)
            O[rows, h], size[rows, h] = as_kept(w) @ V / total, w @ V.abs() / total
    fp32 = 2.0 ** -24 * (max(lens[1]) + max(lens[2]) + 64 + 8 * logit / math.log(2))
    err = (2.0 ** -15 + 2 * fp32) * size
    return O, P64.half_step(BF16) * (O.abs() + err) + err + 1e-30


@pytest.mark.gpu
@pytest.mark.parametrize("lens,H,H_kv,d_h", CASES)
def test_weights_have_two_parts(lens, H, H_kv, d_h):
    import paper_2310_02409_amd as D
    t = inputs(lens, H, H_kv, d_h)
    ref, tol = reference(t, lens, d_h ** -0.5)
    for layout in (0, 1):
        O, _ = Q4.attend(D, t, lens, d_h ** -0.5, layout)
        assert float(((O.cpu().double() - ref).abs() - tol).max()) <= 0


@pytest.mark.parametrize("lens,H,H_kv,d_h", CASES)
def test_the_bound_sees_one_part(lens, H, H_kv, d_h):
    """(On the CPU.)  Weights of one bf16 part, rounded or cut off, are beyond the bound; of two parts they are within."""
    t = inputs(lens, H, H_kv, d_h)
    ref, tol = reference(t, lens, d_h ** -0.5)
    cut = lambda w: (w.float().view(torch.int32) & -65536).view(torch.float32)
    one, upper = (lambda w: w.float().bfloat16().double()), (lambda w: cut(w).double())
    two = lambda w: upper(w) + (w.float() - cut(w)).bfloat16().double()
    beyond = lambda kept: int((((reference(t, lens, d_h ** -0.5, kept)[0].to(BF16).double() - ref).abs() - tol) > 0).sum())
    assert beyond(one) > 0 and beyond(upper) > 0 and beyond(two) == 0, (beyond(one), beyond(upper), beyond(two))
