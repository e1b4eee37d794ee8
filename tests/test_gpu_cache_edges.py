"""A paged cache of keys and values on the GPU: what pages may hold besides tokens, extreme scales, shared pages, streams, captured
graphs, and waits that run out."""
import math
import time

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


@pytest.mark.parametrize("max_new", [1, 0])
@pytest.mark.parametrize("seed", range(3))
def test_pages_hold_anything_behind_a_sequence(heart, seed, max_new):
    """e4m3: any code and any scale byte, NaN codes among them, in slots without a token and in pages of no sequence."""
    g = torch.Generator().manual_seed(seed)
    c = Case([40 + 37 * seed, 129, 5], [3, 40, 5], Hq=4, Hkv=2, page=(16, 32, 64)[seed], kind="e4m3", causal=1, pad=40, seed=seed)
    used = torch.zeros((c.n_pages, c.page), dtype=torch.bool)
    for s in range(c.S):
        j = torch.arange(c.lens[s])
        used[c.table[s].long()[j // c.page], j % c.page] = True
    free = ~used[:, None, :].expand(-1, c.Hkv, -1)
    for x in (c.k, c.v):
        x.view(torch.uint8)[free] = torch.randint(0, 256, (int(free.sum()), D), generator=g, dtype=torch.uint8)
        x.view(torch.uint8)[free] |= (torch.rand((int(free.sum()), D), generator=g) < 0.2).to(torch.uint8) * 0x7f
    for x in (c.k_scale, c.v_scale):
        x[free] = torch.randint(0, 256, (int(free.sum()),), generator=g, dtype=torch.uint8)
    d = Device(heart, c, max_new=max_new)
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    check_attention(c, O, lse)


@pytest.mark.parametrize("max_new", [1, 0])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("what", ["zero values", "tiny and large values", "tiny", "large", "zero keys", "zero queries", "one token of weight"])
def test_extreme_values(heart, what, kind, max_new):
    c = Case([300, 40], [3, 40], Hq=4, Hkv=2, page=16, causal=1, pad=40, garbage=False, seed=len(what))
    k, v = c.k.float(), c.v.float()
    g = torch.Generator().manual_seed(7)
    if what == "zero values":
        v.zero_()
    elif what == "tiny and large values":  # token by token, scales 2^40 apart
        v *= torch.exp2(torch.randint(-20, 21, v.shape[:3], generator=g).float())[..., None]
    elif what == "tiny":
        v *= 2.0 ** -60
        k *= 2.0 ** -40
        c.Q = (c.Q.float() * 2.0 ** 40).to(torch.bfloat16)
    elif what == "large":
        v *= 2.0 ** 60
        k *= 2.0 ** 40
        c.Q = (c.Q.float() * 2.0 ** -40).to(torch.bfloat16)
    elif what == "zero keys":
        k.zero_()
    elif what == "zero queries":
        c.Q.zero_()
    else:
        k[:, :, 3] *= 30
    k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
    if kind == "e4m3":
        c.kind = kind
        (c.k, c.k_scale), (c.v, c.v_scale) = quantise(k), quantise(v)
    else:
        c.k, c.v = k, v
    if what == "one token of weight":  # (logits up to some 10^2: 32-bit sums of products are off by 2^-20 of that and more; here only what is finite)
        O, lse = Device(heart, c, max_new=max_new).attention()
        n = int(c.row_start[-1])
        want, want_lse = c.attention()
        assert torch.isfinite(O[:n]).all() and ((lse[:n].cpu() - want_lse[:n]).abs() < 2 ** -10).all()
        return
    d = Device(heart, c, max_new=max_new)
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    check_attention(c, O, lse)


@pytest.mark.parametrize("max_new", [1, 0])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_queries_that_are_not_finite(heart, kind, max_new):
    """A query of NaN or infinity makes its own row of its own head no numbers; one without keys still gives zeros."""
    c = Case([3, 200], [6, 40], Hq=4, Hkv=2, kind=kind, causal=1, page=16, pad=40)
    want = Device(heart, c, max_new=max_new).attention()[0]
    c.Q[1, 2, 5], c.Q[20, 1, 7], c.Q[30, 3] = math.nan, math.inf, math.nan  # row 1: no token (six new ones of three)
    O, lse = Device(heart, c, max_new=max_new).attention()
    assert (O[:3] == 0).all() and (lse[:3] == -math.inf).all()
    clean = torch.ones((c.T, 4), dtype=torch.bool)
    clean[20, 1] = clean[30, 3] = clean[1, 2] = False
    assert torch.equal(bits(O.cpu()[clean]), bits(want.cpu()[clean]))
    assert not torch.isfinite(O[20, 1].float()).any() and not torch.isfinite(O[30, 3].float()).any()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_pages_shared_by_sequences(heart, kind):
    """A common prefix in common pages, the same page twice in one table."""
    c = Case([150, 170, 64], [2, 30, 1], Hq=4, Hkv=2, kind=kind, page=32, causal=1, pad=40)
    c.table[1, :4] = c.table[0, :4]
    c.table[2, 1] = c.table[2, 0]
    for max_new in (1, 0):
        O, lse = Device(heart, c, max_new=max_new).attention()
        check_attention(c, O, lse)


def test_two_streams_at_a_time(heart):
    """Calls with a workspace each, side by side; and calls that share one, in a row without a wait between them."""
    cases = [Case([3000, 700], [40, 3], Hq=8, Hkv=4, page=64, causal=1, kind=k, garbage=False, seed=i) for i, k in enumerate(("bf16", "e4m3"))]
    singles = [Case([5000, 40, 900], [1, 1, 1], Hq=8, Hkv=4, page=32, kind=k, garbage=False, seed=i) for i, k in enumerate(("bf16", "e4m3"))]
    devices = [Device(heart, c) for c in cases + singles]
    want = [d.attention() for d in devices]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in devices]
    got = []
    for _ in range(10):
        for d, s in zip(devices, streams):
            with torch.cuda.stream(s):
                got.append(d.attention())
    torch.cuda.synchronize()
    for i, (O, lse) in enumerate(got):
        assert torch.equal(bits(O), bits(want[i % 4][0])) and torch.equal(lse, want[i % 4][1])
    ws = max((d.ws for d in devices), key=lambda x: x.numel()).clone().zero_()
    for d in devices:
        d.ws = ws
    got = [d.attention() for _ in range(5) for d in devices]
    for i, (O, lse) in enumerate(got):
        assert torch.equal(bits(O), bits(want[i % 4][0])) and torch.equal(lse, want[i % 4][1])
    assert heart.heart_get_status(ws) == 0


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_captured_tiles_follow_the_lengths(heart, kind):
    """The kernel for many rows, captured once and replayed over other lengths and rows; two graphs in one workspace."""
    first = Case([300, 60, 140], [200, 60, 7], Hq=4, Hkv=2, kind=kind, causal=1, page=16, garbage=False, seed=1, pad=0)
    d = Device(heart, first)
    full = [sum(1 for p in first.table[s].tolist() if p >= 0) * 16 for s in range(3)]
    outs = [(torch.zeros_like(d.Q), torch.zeros((first.T, 4), device="cuda")) for _ in range(2)]
    graphs = []
    for O, lse in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            heart.heart_cache_attn(d.cfg, d.Q, d.cache, *d.where, O, d.ws, lse=lse)
        graphs.append(graph)
    for new, lens in (([200, 60, 7], [300, 60, 140]), ([1, 50, 0], [290, 50, 3]), ([0, 0, 144], [1, 1, 144]), ([90, 1, 100], [90, 33, 101])):
        assert all(a <= b for a, b in zip(lens, full)) and sum(new) <= first.T
        c = Case(lens, new, Hq=4, Hkv=2, kind=kind, causal=1, page=16, garbage=False, pad=first.T - sum(new))
        c.table, c.n_pages, c.width, c.Q = first.table, first.n_pages, first.width, first.Q
        c.k, c.v, c.k_scale, c.v_scale = first.k, first.v, first.k_scale, first.v_scale
        for to, x in zip(d.where[1:], (c.row_start, c.kv_len)):
            to.copy_(x)
        for O, lse in outs:
            O.fill_(77)
            lse.fill_(55)
        for graph in graphs:
            graph.replay()
        for O, lse in outs:
            check_attention(c, O, lse)
    assert heart.heart_get_status(d.ws) == 0


def test_long_tiles_of_many_parts(heart):
    """A tile that most of the chip shares, many short tiles beside a long one, more tiles than CTAs."""
    for kw in (dict(lens=[6000], new=[60], Hq=1, Hkv=1), dict(lens=[6000, 30, 30, 500], new=[90, 30, 30, 300], Hq=2, Hkv=2),
               dict(lens=[700, 900], new=[700, 500], Hq=24, Hkv=24, causal=1)):
        for kind in ("bf16", "e4m3"):
            c = Case(**kw, page=64, kind=kind, seed=3)
            d = Device(heart, c)
            O, lse = d.attention()
            check_attention(c, O, lse)
            assert heart.heart_get_status(d.ws) == 0


def test_dealt_tiles(heart):
    """Keys and values beyond what stays in L2: tiles are dealt in turn.  The same pages over and over stand for a long context."""
    H, page, n_pages, L, new = 12, 128, 4, 16384 + 77, 1500  # 202 MB of keys and values, 12 tiles a head
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn((n_pages, H, page, D), generator=g).to(torch.bfloat16) for _ in range(2))
    width = -(-L // page)
    table = (torch.arange(width) % n_pages).to(torch.int32)[None]
    cfg = heart.make_cache_config(1, new, H, H, page, n_pages, width, causal=1)
    Q = torch.randn((new, H, D), generator=g).to(torch.bfloat16)
    O, lse = torch.zeros_like(Q).cuda(), torch.zeros((new, H), device="cuda")
    ws = heart.new_cache_workspace(cfg)
    heart.heart_cache_attn(cfg, Q.cuda(), heart.Cache(cfg, k.cuda(), v.cuda()), table.cuda(), torch.tensor([0, new], dtype=torch.int32, device="cuda"),
                           torch.tensor([L], dtype=torch.int32, device="cuda"), O, ws, lse=lse)
    assert heart.heart_get_status(ws) == 0
    j = torch.arange(L, device="cuda")
    for h in (0, 5, 11):
        ks, vs = (x[table[0].long()[torch.arange(L) // page], h, torch.arange(L) % page].cuda().double() for x in (k, v))
        logits = Q[:, h].cuda().double() @ ks.T / math.sqrt(D)
        logits.masked_fill_(j[None] > torch.arange(L - new, L, device="cuda")[:, None], -math.inf)
        w = torch.softmax(logits, -1)
        want, most = w @ vs, w @ vs.abs()
        # (as check_attention: a weight is rounded once, the result once)
        assert ((O[:, h].double() - want).abs() <= (2 ** -8 + 2 ** -12) * most + 2 ** -8 * want.abs()).all()
        assert ((lse[:, h].double() - torch.logsumexp(logits, -1)).abs() <= 2 ** -14).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("name", ["ragged prompts", "more sequences", "one long among short", "short among long"])
def test_several_tiles_a_cta(heart, name, kind):
    """Tiles of unlike cost: masked and whole steps, long and short, sequences by the lane and by the thread."""
    g = torch.Generator().manual_seed(11)
    if name == "ragged prompts":
        new = torch.randint(1, 700, (6,), generator=g).tolist()
        kw = dict(new=new, lens=[n + int(torch.randint(0, 500, (1,), generator=g)) for n in new], Hq=24, Hkv=8, causal=1, window=256, sink=4)
    elif name == "more sequences":
        new = torch.randint(0, 90, (50,), generator=g).tolist()
        kw = dict(new=new, lens=[n + int(torch.randint(0, 300, (1,), generator=g)) for n in new], Hq=12, Hkv=6, causal=16, page=32)
    elif name == "one long among short":
        kw = dict(new=[60] + [40] * 60, lens=[6000] + [40] * 60, Hq=8, Hkv=8, causal=1, page=64)
    else:
        kw = dict(new=[40] * 41, lens=[900] * 20 + [40] + [900] * 20, Hq=10, Hkv=10, page=128)
    c = Case(**kw, kind=kind, pad=9, seed=3)
    d = Device(heart, c)
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    check_attention(c, O, lse)
    again = d.attention()
    assert torch.equal(bits(O), bits(again[0])) and torch.equal(bits(lse), bits(again[1]))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("name", ["rows", "tiles"])
def test_a_wait_that_runs_out_is_reported(heart, name, kind):
    """In the test-hook build a flag makes one CTA leave out a copy: its waits run out after a millisecond, the status tells, and the next
    call in the same workspace is right."""
    from paper_2605_14513_b200 import build

    product = heart.lib()
    c = Case([8192], [1], kind=kind, page=64, garbage=False) if name == "rows" else Case([4000], [200], kind=kind, page=64, garbage=False)
    try:
        heart._lib = heart.load(build.build_test_hooks())
        d = Device(heart, c)
        want = d.attention()
        assert heart.heart_get_status(d.ws) == 0
        d.cfg.flags = 0x80000000
        t0 = time.perf_counter()
        d.attention()
        assert heart.heart_get_status(d.ws) == heart.ERR_DEVICE_CHECK
        assert time.perf_counter() - t0 < 5.0
        d.cfg.flags = 0
        for _ in range(3):
            O, lse = d.attention()
            assert heart.heart_get_status(d.ws) == 0
            assert torch.equal(bits(O), bits(want[0])) and torch.equal(lse, want[1])
    finally:
        heart._lib = product
