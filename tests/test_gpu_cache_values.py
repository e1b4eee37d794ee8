"""Attention over a paged cache whose values differ by many binades from token to token, and tokens that a row does not see:
against the definition in 64 bits, in both kernels."""
import math

import pytest
import torch

from cache_cases import Case, Device, quantise

pytestmark = pytest.mark.gpu

D = 128


@pytest.fixture(scope="module")
def heart():
    from paper_2605_14513_b200 import heart as h

    return h


def bits(x):
    return x.contiguous().view(torch.uint8).cpu()


def e4m3_case(lens, new, edit, seed=0, **kw):
    """A Case whose keys and values are edit(case, k, v, generator) of normal ones, as e4m3: [n_pages, Hkv, page, D] pools, fp32."""
    c = Case(lens, new, garbage=False, seed=seed, pad=kw.pop("pad", 40), **kw)
    k, v = c.k.float(), c.v.float()
    edit(c, k, v, torch.Generator().manual_seed(1000 + seed))
    c.kind = "e4m3"
    (c.k, c.k_scale), (c.v, c.v_scale) = (quantise(x.to(torch.bfloat16)) for x in (k, v))
    return c


def slots(c, s, tokens):
    """Pages and slots of tokens of sequence s."""
    j = torch.as_tensor(tokens)
    return c.table[s].long()[j // c.page], j % c.page


def product_bound(c):
    """For each row: the largest product of a weight and its value's scale, times sum_j |code_j| over the keys that it sees."""
    k, v = c.values()
    scale = torch.where(c.v_scale == 255, 0.0, torch.exp2(c.v_scale.double() - 127))
    codes = c.v.double().nan_to_num(0.0).abs()
    B = torch.zeros((c.T, c.Hq, D), dtype=torch.float64)
    factor, G = (c.scale if c.scale > 0 else 1 / math.sqrt(D)), c.Hq // c.Hkv
    for s in range(c.S):
        r0, n = int(c.row_start[s]), c.new[s]
        if not c.lens[s] or not n:
            continue
        ks, cs, ok = c.tokens(k, s), c.tokens(codes, s), c.seen(s)
        es = c.tokens(scale[..., None], s)[..., 0]
        for h in range(c.Hq):
            logits = torch.where(ok, c.Q[r0:r0 + n, h].double() @ ks[:, h // G].T * factor, torch.tensor(-math.inf, dtype=torch.float64))
            w = torch.nan_to_num(torch.softmax(logits, -1), 0.0)
            B[r0:r0 + n, h] = (w * es[:, h // G]).amax(-1, keepdim=True) * (ok.double() @ cs[:, h // G])
    return B


def check(c, O, lse, rows=None):
    """As cache_cases.check_attention, with one term more: a weight of f16 is off by 2^-25 at most where it is below 2^-14, and the row's largest
    product of a weight and a scale is held as 1 at least (2^6 by rows; by tiles 2^8, of which up to 2^8 is the span of a step's
    scales): each key's part is off by 2^-25 of that product times its code."""
    want, want_lse = c.attention()
    n = int(c.row_start[-1])
    O, lse = O.cpu(), lse.cpu()
    assert (O[n:] == 77).all() and (lse[n:] == 55).all()
    at = torch.arange(n) if rows is None else rows
    got, want = O[at].double(), want[at]
    bound = (2 ** -8 + 2 ** -12) * c.weight_bound()[at] + 2 ** -8 * want.abs() + 2 ** -25 * product_bound(c)[at] + 1e-30
    worst = (got - want).abs() / bound
    empty = want_lse[at] == -math.inf
    assert (got[empty] == 0).all() and (lse[at][empty] == -math.inf).all()
    assert worst[~empty].max() <= 1.0, float(worst[~empty].max())
    off = (lse[at].double() - want_lse[at])[~empty].abs()
    assert off.max() <= 2 ** -14, float(off.max())


def attend(heart, c, **kw):
    d = Device(heart, c, **kw)
    out = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    return out


BOTH = pytest.mark.parametrize("max_new", [1], ids=["rows"])


def scatter(lo, hi):
    def edit(c, k, v, g):
        v *= torch.exp2(torch.randint(lo, hi + 1, v.shape[:3], generator=g).float())[..., None]

    return edit


@BOTH
@pytest.mark.parametrize("seed", range(10))
def test_value_scales_far_apart(heart, seed, max_new):
    """Token by token up to 2^40, and 2^80, apart."""
    for spread in (20, 40):
        c = e4m3_case([300, 40], [3, 40], scatter(-spread, spread), seed, Hq=4, Hkv=2, causal=1)
        check(c, *attend(heart, c, max_new=max_new))


@BOTH
@pytest.mark.parametrize("span", [2, 6, 7, 8, 9, 12, 15, 16, 25])
def test_value_scales_some_binades_apart(heart, span, max_new):
    c = e4m3_case([500, 300, 140], [200, 7, 140], scatter(0, span), span, Hq=6, Hkv=2, page=32, causal=1, window=150, sink=3)
    check(c, *attend(heart, c, max_new=max_new))


@BOTH
@pytest.mark.parametrize("gain", [20, 26, 40, 90])
def test_large_values_of_tokens_that_come_later(heart, gain, max_new):
    """The last token's values are 2^gain times the others: the rows before it know nothing of it."""
    def edit(c, k, v, g):
        for s in range(c.S):
            page, slot = slots(c, s, c.lens[s] - 1)
            v[page, :, slot] *= 2.0 ** gain

    c = e4m3_case([2, 60, 131], [2, 9, 5], edit, gain, Hq=4, Hkv=2, causal=1)
    check(c, *attend(heart, c, max_new=max_new))


@BOTH
@pytest.mark.parametrize("seed", range(3))
def test_tokens_before_a_window_hold_anything(heart, seed, max_new):
    """Any scale byte in tokens of the sequence that no new one sees: the same bits as without them."""
    for page in (16, 64, 128):
        c = Case([700, 90, 400], [5, 20, 1], Hq=4, Hkv=2, page=page, kind="e4m3", causal=1, window=60 + 17 * seed, sink=3, garbage=False, seed=seed, pad=40)
        want = attend(heart, c, max_new=max_new)
        g = torch.Generator().manual_seed(seed)
        for s in range(c.S):
            first = c.lens[s] - c.new[s] + 1 - c.window
            page_, slot = slots(c, s, torch.arange(3, max(3, first)))
            n = page_.numel()
            for x in (c.k_scale, c.v_scale):
                x[page_, :, slot] = torch.randint(0, 256, (n, c.Hkv), generator=g, dtype=torch.uint8)
        got = attend(heart, c, max_new=max_new)
        assert torch.equal(bits(got[0]), bits(want[0])) and torch.equal(bits(got[1]), bits(want[1]))


@BOTH
@pytest.mark.parametrize("gain", [24, 40, 80])
def test_a_large_value_of_no_weight(heart, gain, max_new):
    """Every row sees a token whose values are 2^gain times the others', with a logit far below theirs (2^-150 of a weight)."""
    def edit(c, k, v, g):
        c.Q = (c.Q.float() * 0.1 + 1.0).to(torch.bfloat16)
        for s in range(c.S):
            page, slot = slots(c, s, c.lens[s] // 2)
            k[page, :, slot] = -9.0
            v[page, :, slot] *= 2.0 ** gain

    c = e4m3_case([30, 300], [30, 130], edit, gain, Hq=4, Hkv=2, page=64)
    check(c, *attend(heart, c, max_new=max_new))


@BOTH
@pytest.mark.parametrize("zeros", ["the first steps", "single tokens", "the last steps", "all but one"])
@pytest.mark.parametrize("gain", [0, 17, 24, 60])
def test_zero_values_beside_others(heart, gain, zeros, max_new):
    """Tokens of weight whose values are zero count in the denominator, whatever the others' scales are."""
    def edit(c, k, v, g):
        v *= 2.0 ** gain
        for s in range(c.S):
            L = c.lens[s]
            at = {"the first steps": torch.arange(min(L - 1, 256)), "single tokens": torch.arange(0, L, 7), "the last steps": torch.arange(min(L - 1, 128), L),
                  "all but one": torch.arange(1, L)}[zeros]
            page, slot = slots(c, s, at)
            v[page, :, slot] = 0.0

    c = e4m3_case([390, 300], [3, 140], edit, gain, Hq=4, Hkv=2, page=64)
    check(c, *attend(heart, c, max_new=max_new))
