"""GPU: blocks of a 4-bit cache with the scale byte 255, on every route that attention over such a cache takes."""
import pytest
import torch

import test_gpu_q4 as Q4

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# (type, heads, K/V heads, query rows): codes read in place (up to 128 vectors a K/V head); unpacked for the split-K kernel (fp32; more
# than 32 heads a K/V head) and for the query-block kernel
ROUTES = [(BF16, 4, 2, 1), (BF16, 8, 2, 32), (F32, 4, 2, 1), (F32, 2, 2, 5), (F32, 8, 2, 40), (BF16, 80, 2, 1), (BF16, 80, 2, 7), (BF16, 2, 2, 140),
          (BF16, 24, 2, 33), (F32, 16, 16, 1)]


@pytest.fixture(scope="module")
def D():
    import paper_2310_02409_amd as D
    return D


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("k", [3, 70, 1500])
@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("dtype,H,H_kv,q", ROUTES)
def test_a_bad_block_on_every_route(D, dtype, H, H_kv, q, d_h, k, layout):
    """A key makes NaN of the rows and log-sum-exps of its K/V head in its sequence; a value of 32 channels of these rows, and of no log-sum-exp;
    everything else has the bits that it has without them."""
    lens, scale = ([q, q, q], [5, k, 40], [q + 3, q, 0]), d_h ** -0.5
    t = Q4.attention_case(70, *lens, H, H_kv, d_h, dtype)
    good, good_lse = Q4.attend(D, t, lens, scale, layout, want_lse=True)
    assert torch.isfinite(good.float()).all() and torch.isfinite(good_lse).all()
    G, at = H // H_kv, 5 + k - 2  # the nugget before the second sequence's last one
    head = slice((H_kv - 1) * G, H)
    hit = torch.zeros_like(good, dtype=torch.bool)
    hit[q:2 * q, head] = True
    for block in range(d_h // 32):
        for names in (("Ks",), ("Vs",), ("Ks", "Vs")):
            bad = {n: v.clone() for n, v in t.items()}
            for n in names:
                bad[n][at, H_kv - 1, block] = 255
            O, lse = Q4.attend(D, bad, lens, scale, layout, want_lse=True)
            want = hit.clone()
            if "Ks" not in names:
                want[..., :32 * block] = False
                want[..., 32 * block + 32:] = False
            assert torch.equal(torch.isnan(O), want), (names, block)
            assert torch.equal(O[~want], good[~want]), (names, block)
            rows = hit[..., 0] if "Ks" in names else torch.zeros_like(hit[..., 0])
            assert torch.equal(torch.isnan(lse), rows), (names, block)
            assert torch.equal(lse[~rows], good_lse[~rows]), (names, block)


@pytest.mark.parametrize("dtype,H,H_kv,q", ROUTES)
def test_a_whole_sequence_of_bad_keys(D, dtype, H, H_kv, q):
    lens, d_h = ([q, q], [40, 33], [0, q]), 64
    t = Q4.attention_case(71, *lens, H, H_kv, d_h, dtype)
    good, good_lse = Q4.attend(D, t, lens, 0.125, want_lse=True)
    t["Ks"][:40] = 255
    O, lse = Q4.attend(D, t, lens, 0.125, want_lse=True)
    assert torch.isnan(O[:q].float()).all() and torch.isnan(lse[:q]).all()
    assert torch.equal(O[q:], good[q:]) and torch.equal(lse[q:], good_lse[q:])
    assert torch.equal(torch.isnan(Q4.attend(D, t, lens, 0.125)[0]), torch.isnan(O))


def test_reading_back_a_bad_key_leaves_its_value(D):
    t = Q4.attention_case(72, [1], [9], [1], 2, 2, 64, BF16)
    t["Ks"][4, 1, 0] = 255
    cache = [t[n].cuda() for n in ("Kc", "Ks", "Vc", "Vs")]
    for dtype in (BF16, F32):
        Kn, Vn = D.dodo_unpack_nuggets_q4(*cache, dtype)
        want = torch.zeros(9, 2, 64, dtype=torch.bool, device="cuda")
        want[4, 1, :32] = True
        assert torch.equal(torch.isnan(Kn), want) and not bool(torch.isnan(Vn).any())


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("H,H_kv,q,m", [(4, 2, 1, 40), (8, 2, 9, 50), (2, 2, 60, 100)])
def test_a_local_row_that_is_not_finite(D, H, H_kv, q, m, value):
    """Codes read in place: it reaches the rows of its sequence and K/V head that see it, and no other sequence's or head's."""
    lens, d_h, at = ([q, q, q], [70, 300, 40], [m, m, m]), 64, m - 1 - q // 2  # (a row that the later half of the query rows sees)
    t = Q4.attention_case(73, *lens, H, H_kv, d_h, BF16)
    t["Q"][..., 3] = t["Q"][..., 3].abs() + 0.5  # (an infinite channel of K makes an infinite logit, of one sign)
    good, good_lse = Q4.attend(D, t, lens, 0.125, want_lse=True)
    G, first = H // H_kv, 2 * q - 1 - q // 2  # of the second sequence's query rows, the first one that sees it
    for name in ("Kl", "Vl"):
        bad = {n: v.clone() for n, v in t.items()}
        bad[name][m + at, 1, 3] = value
        O, lse = Q4.attend(D, bad, lens, 0.125, want_lse=True)
        rows, other = torch.zeros_like(lse, dtype=torch.bool), torch.ones_like(lse, dtype=torch.bool)
        rows[first:2 * q, G:2 * G] = True
        other[q:2 * q, G:2 * G] = False
        assert torch.equal(O[other], good[other]) and torch.equal(lse[other], good_lse[other]), name
        if name == "Kl":
            assert torch.isnan(O[rows].float()).all() and not torch.isfinite(lse[rows]).any()
        else:
            assert not torch.isfinite(O[rows].float())[:, 3].any() and torch.equal(lse[rows], good_lse[rows])
