"""Attention over a paged cache whose values differ by many binades from token to token, and tokens that a row does not see:
against the definition in 64 bits, in both kernels."""
import math

import pytest
import torch

from cache_cases import Case, Device, check_attention, quantise

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
    product of a weight and a scale is held as 2^-2 at least (2^6, by tiles less the span of a step's scales, up to 2^8): each
    key's part is off by 2^-23 of that product times its code."""
    want, want_lse = c.attention()
    n = int(c.row_start[-1])
    O, lse = O.cpu(), lse.cpu()
    assert (O[n:] == 77).all() and (lse[n:] == 55).all()
    at = torch.arange(n) if rows is None else rows
    got, want = O[at].double(), want[at]
    bound = (2 ** -8 + 2 ** -12) * c.weight_bound()[at] + 2 ** -8 * want.abs() + 2 ** -23 * product_bound(c)[at] + 1e-30
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


BOTH = pytest.mark.parametrize("max_new", [1, 0], ids=["rows", "tiles"])


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
    """Any code, any scale byte, in tokens of the sequence that no new one sees: the same bits as without them."""
    for page in (16, 64, 128):
        c = Case([700, 90, 400], [5, 20, 1], Hq=4, Hkv=2, page=page, kind="e4m3", causal=1, window=60 + 17 * seed, sink=3, garbage=False, seed=seed, pad=40)
        want = attend(heart, c, max_new=max_new)
        g = torch.Generator().manual_seed(seed)
        for s in range(c.S):
            first = c.lens[s] - c.new[s] + 1 - c.window
            page_, slot = slots(c, s, torch.arange(3, max(3, first)))
            n = page_.numel()
            for x in (c.k, c.v):
                b = torch.randint(0, 256, (n, c.Hkv, D), generator=g, dtype=torch.uint8)
                x.view(torch.uint8)[page_, :, slot] = b | (torch.rand(b.shape, generator=g) < 0.2).to(torch.uint8) * 0x7f
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


@pytest.mark.parametrize("how", ["zeros first", "zeros at times", "rising", "falling", "rising far", "falling far", "far apart", "one without weight"])
@pytest.mark.parametrize("gain", [-40, 0, 20, 60])
def test_parts_of_many_steps(heart, gain, how):
    """As many heads as give a CTA several steps of a tile."""
    def edit(c, k, v, g):
        v *= 2.0 ** gain
        L = c.lens[0]
        page, slot = slots(c, 0, torch.arange(L))
        step = torch.arange(L) // 128
        if how == "zeros first":
            v[page[:300], :, slot[:300]] = 0.0
        elif how == "zeros at times":
            v[page[::50], :, slot[::50]] = 0.0
            v[page[640:768], :, slot[640:768]] = 0.0
        elif how == "far apart":
            scatter(-30, 30)(c, k, v, g)
        elif how == "one without weight":
            c.Q = (c.Q.float() * 0.1 + 1.0).to(torch.bfloat16)
            k[page[200], :, slot[200]] = -9.0
            v[page[200], :, slot[200]] *= 2.0 ** 30
        else:
            by = {"rising": 3, "falling": -3, "rising far": 6, "falling far": -6}[how]
            v[page, :, slot] *= torch.exp2((by * step).float().clamp(max=85 - gain))[:, None, None]

    c = e4m3_case([1500], [290], edit, gain, Hq=48, Hkv=24, page=64, causal=1)
    check(c, *attend(heart, c))


@BOTH
@pytest.mark.parametrize("pool", ["k", "v"])
def test_codes_that_are_no_numbers(heart, pool, max_new):
    """A code of 0x7f in a token: rows before it are what they are without it, rows that see it are no numbers."""
    for new in (6, 140):
        c, without = (Case([new + 50], [new], Hq=2, kind="e4m3", causal=1, page=16, garbage=False, pad=40) for _ in range(2))
        clean = attend(heart, without, max_new=max_new)
        page, slot = slots(c, 0, 50 + new // 2)
        getattr(c, pool).view(torch.uint8)[page, :, slot, 77] = 0x7f
        O, lse = attend(heart, c, max_new=max_new)
        n = new // 2
        # (by tiles another kernel may have brought them: both are within the bound)
        check(without, *(torch.cat([x[:n], y[n:]]) for x, y in zip((O, lse), clean)), rows=torch.arange(n))
        assert torch.isfinite(O[:n]).all() and torch.isfinite(lse[:n]).all()
        assert not torch.isfinite(O[n:new].float()).all(-1).any()


@pytest.mark.parametrize("S", [3, 40])
def test_other_heads_keep_their_bits(heart, S):
    """Scales far apart in one sequence and key head: what the others get does not change by a bit, now or in the next call."""
    lens = [200 + 31 * (i % 5) for i in range(S)]
    new = [60 + 13 * (i % 4) for i in range(S)]
    for G in (1, 3, 8):
        c = e4m3_case(lens, new, lambda *a: None, G, Hq=3 * G, Hkv=3, causal=1, page=32, pad=40)
        d = Device(heart, c, max_new=0)
        want = d.attention()
        far = e4m3_case(lens, new, lambda *a: None, G, Hq=3 * G, Hkv=3, causal=1, page=32, pad=40)
        page, slot = slots(far, 2, torch.arange(0, lens[2], 3))
        far.v_scale[page, 1, slot] += 40
        e = Device(heart, far, max_new=0)
        e.ws = d.ws
        O, lse = e.attention()
        r0, n = int(c.row_start[2]), new[2]
        rows = torch.zeros((c.T, 3 * G), dtype=torch.bool)
        rows[r0:r0 + n, G:2 * G] = True
        assert torch.equal(bits(O.cpu()[~rows]), bits(want[0].cpu()[~rows])) and torch.equal(lse.cpu()[~rows], want[1].cpu()[~rows])
        check(far, O, lse)
        again = e.attention()
        assert torch.equal(bits(O), bits(again[0])) and torch.equal(bits(lse), bits(again[1]))
        after = d.attention()
        assert torch.equal(bits(after[0]), bits(want[0])) and torch.equal(bits(after[1]), bits(want[1]))
        assert heart.heart_get_status(d.ws) == 0


def test_captured_calls_with_scales_far_apart(heart):
    """One captured call, replayed over a cache whose scales are alike, far apart, and alike again."""
    near = e4m3_case([300, 140], [150, 140], lambda *a: None, 1, Hq=4, Hkv=2, causal=1)
    far = e4m3_case([300, 140], [150, 140], scatter(-30, 30), 1, Hq=4, Hkv=2, causal=1)
    d = Device(heart, near)
    want = d.attention()
    O, lse = torch.full_like(d.Q, 77.0), torch.full((near.T, 4), 55.0, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        heart.heart_cache_attn(d.cfg, d.Q, d.cache, *d.where, O, d.ws, lse=lse)
    for c in (near, far, near, far):
        d.cache.v.view(torch.uint8).copy_(c.v.view(torch.uint8))
        d.cache.v_scale.copy_(c.v_scale)
        graph.replay()
        if c is near:
            assert torch.equal(bits(O), bits(want[0])) and torch.equal(bits(lse), bits(want[1]))
        else:
            check(c, O, lse)
    assert heart.heart_get_status(d.ws) == 0


@BOTH
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 64])
def test_tokens_of_pages_that_there_are_not_count_as_zeros(heart, page, kind, max_new):
    """An entry out of range: its tokens are keys and values of zero, whatever the scales of the pool's last page are."""
    for gone in (2, -1):
        c = Case([200, 150], [5, 40], Hq=4, Hkv=2, page=page, kind=kind, causal=1, garbage=False, pad=40, spare=3)
        used = set(c.table.flatten().tolist())
        zeros, = [p for p in range(c.n_pages - 1) if p not in used][:1]
        c.table[0, 1] = zeros
        for x in (c.k, c.v):
            x.view(torch.uint8 if kind == "e4m3" else torch.bfloat16)[zeros] = 0
        if kind == "e4m3":
            c.k_scale[zeros], c.v_scale[zeros] = 127, 127
        d = Device(heart, c, max_new=max_new)
        d.where[0][0, 1] = c.n_pages if gone == 2 else gone
        if kind == "e4m3":
            d.cache.v_scale[-1], d.cache.k_scale[-1] = 250, 255
            c.v_scale[-1], c.k_scale[-1] = 250, 255
        if c.n_pages - 1 in used:  # the last page is to be nobody's: its tokens go to a free one
            free = [p for p in range(c.n_pages - 1) if p not in used and p != zeros][0]
            c.table[c.table == c.n_pages - 1] = free
            d.where[0][d.where[0] == c.n_pages - 1] = free
        O, lse = d.attention()
        assert heart.heart_get_status(d.ws) == heart.ERR_DEVICE_CHECK
        if kind == "e4m3":
            check(c, O, lse)
        else:
            check_attention(c, O, lse)


@BOTH
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e-10])
def test_queries_of_zeros_and_a_small_scale(heart, scale, kind, max_new):
    """The mean of the values that a row sees: a query's own scale times the call's is below the 32-bit numbers."""
    c = Case([200, 30], [40, 30], Hq=4, Hkv=2, page=16, kind=kind, causal=1, scale=scale, garbage=False, pad=40)
    c.Q[::2] = 0.0
    c.Q[1::4] = (c.Q[1::4].float() * 2.0 ** -100).to(torch.bfloat16)
    O, lse = attend(heart, c, max_new=max_new)
    if kind == "e4m3":
        check(c, O, lse)
    else:
        check_attention(c, O, lse)


@BOTH
@pytest.mark.parametrize("which", ["one", "all"])
def test_keys_of_infinity(heart, which, max_new):
    """A bf16 key with an infinity: rows whose logit it makes -inf are as if they did not see it (zeros where they see nothing else), rows whose logit it makes
    +inf are no numbers."""
    new = 20
    c = Case([60], [new], Hq=4, Hkv=2, page=16, pad=40, garbage=False, window=0 if which == "one" else 1)
    bad = 30 if which == "one" else 59  # (a window of one, no order: all rows see the last token alone)
    page, slot = slots(c, 0, bad)
    c.k[page, 0, slot, 5] = math.inf
    sign = torch.where(torch.arange(new) % 2 == 0, 1.0, -1.0)
    c.Q[:new, :, 5] = (c.Q[:new, :, 5].float().abs() + 0.5).mul(sign[:, None]).to(torch.bfloat16)
    O, lse = (x.cpu() for x in attend(heart, c, max_new=max_new))
    plus = torch.zeros((c.T, 4), dtype=torch.bool)
    plus[:new:2, :2] = True  # (the heads of the first key head)
    assert not torch.isfinite(O[plus].float()).any() and not torch.isfinite(lse[plus]).any()
    minus, other = torch.zeros_like(plus), torch.zeros_like(plus)
    minus[1:new:2, :2] = True
    other[:new, 2:] = True

    def agree(rows):  # (the bound of cache_cases.check_attention)
        want, want_lse = c.attention()
        assert ((O.double() - want).abs() <= (2 ** -8 + 2 ** -12) * c.weight_bound() + 2 ** -8 * want.abs())[rows].all()
        assert ((lse.double() - want_lse).abs() <= 2 ** -14)[rows].all()

    agree(other)
    if which == "all":
        assert (O[minus] == 0).all() and (lse[minus] == -math.inf).all()
    else:
        c.k[page, 0, slot] = 0.0
        c.seen = lambda s: (torch.arange(60) != bad).expand(new, 60)
        agree(minus)


@pytest.mark.parametrize("heads", [1, 2, 8])
def test_one_token_of_a_long_context(heart, heads):
    """A large value of no weight, wherever it is: several CTAs look at the scales of a key head."""
    for at in (5, 127, 15000, 29999):
        def edit(c, k, v, g):
            c.Q = (c.Q.float() * 0.1 + 1.0).to(torch.bfloat16)
            page, slot = slots(c, 0, at)
            k[page, heads - 1, slot] = -9.0
            v[page, heads - 1, slot] *= 2.0 ** 30

        c = e4m3_case([30000], [20], edit, at, Hq=heads, Hkv=heads, page=128)
        check(c, *attend(heart, c, max_new=0))


@pytest.mark.parametrize("S,heads", [(200, 1), (640, 8)])
def test_one_token_of_many_sequences(heart, S, heads):
    """More sequences and key heads than CTAs, and than warps that look at once."""
    lens = [10 + s % 9 for s in range(S)]

    def edit(c, k, v, g):
        for s in (0, S // 2 + 1, S - 1):
            page, slot = slots(c, s, lens[s] - 1)
            v[page, heads - 1, slot] *= 2.0 ** 30

    c = e4m3_case(lens, [1 + s % 3 for s in range(S)], edit, S, Hq=heads, Hkv=heads, causal=1, page=16)
    check(c, *attend(heart, c, max_new=0))
