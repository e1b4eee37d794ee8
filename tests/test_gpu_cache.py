"""A paged cache of keys and values on the GPU, against the definition in 64 bits (tests/cache_cases.py)."""
import math

import pytest
import torch

from cache_cases import Case, Device, check_attention, dequantise, quantise

pytestmark = pytest.mark.gpu

D = 128


@pytest.fixture(scope="module")
def heart():
    from paper_2605_14513_b200 import heart as h

    return h


def same(a, b):
    a, b = a.cpu(), b.cpu()
    if a.dtype == torch.float8_e4m3fn:
        a, b = a.view(torch.uint8), b.view(torch.uint8)
    elif a.dtype == torch.bfloat16:
        a, b = a.contiguous().view(torch.int16), b.contiguous().view(torch.int16)
    return torch.equal(a, b)


COPIES = [
    dict(lens=[5], new=[5]), dict(lens=[1], new=[1], Hkv=3, Hq=3), dict(lens=[100, 0, 17, 64], new=[1, 0, 17, 33], Hkv=2),
    dict(lens=[300, 299], new=[129, 300], page=128, Hkv=5, Hq=5),  # (the second has more new tokens than tokens: its first one has no place)
    dict(lens=[33] * 40, new=[1] * 40, page=32, Hkv=9, Hq=9, pad=0), dict(lens=[4000], new=[2111], page=64, Hkv=4, Hq=4),
    dict(lens=[70, 1, 1, 2000], new=[0, 1, 0, 1999], page=16, pad=70),
]


@pytest.mark.parametrize("layout", ["head", "token"])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", range(len(COPIES)))
def test_write_and_read(heart, shape, kind, layout):
    c = Case(**COPIES[shape], kind=kind, layout=layout, seed=shape)
    d = Device(heart, c)
    want = [x.clone() if x is not None else None for x in (c.k, c.v, c.k_scale, c.v_scale)]
    for x, y, given in ((0, 2, c.K), (1, 3, c.V)):
        rows = quantise(given) if kind == "e4m3" else (given, None)
        for s in range(c.S):
            for i in range(c.new[s]):
                j = c.lens[s] - c.new[s] + i
                if j < 0:
                    continue
                page, slot = int(c.table[s, j // c.page]), j % c.page
                r = int(c.row_start[s]) + i
                (want[x].view(torch.uint8) if kind == "e4m3" else want[x])[page, :, slot] = rows[0].view(torch.uint8)[r] if kind == "e4m3" else rows[0][r]
                if kind == "e4m3":
                    want[y][page, :, slot] = rows[1][r]
    heart.heart_cache_write(d.cfg, d.K, d.V, d.cache, *d.where, d.ws)
    assert heart.heart_get_status(d.ws) == 0
    for a, b in zip((d.cache.k, d.cache.v, d.cache.k_scale, d.cache.v_scale), want):
        assert b is None or same(a, b)
    # and back: the rows as they were written, zeros for tokens that there are not, other rows as they are
    K, V = torch.full_like(d.K, 3.0), torch.full_like(d.V, 4.0)
    heart.heart_cache_read(d.cfg, d.cache, *d.where, K, V, d.ws)
    assert heart.heart_get_status(d.ws) == 0
    for got, given, fill in ((K, c.K, 3.0), (V, c.V, 4.0)):
        want_rows = torch.full((c.T, c.Hkv, D), fill, dtype=torch.bfloat16)
        back = dequantise(*quantise(given)).to(torch.bfloat16) if kind == "e4m3" else given
        for s in range(c.S):
            r, n, lost = int(c.row_start[s]), c.new[s], max(0, c.new[s] - c.lens[s])
            want_rows[r:r + n] = back[r:r + n]
            want_rows[r:r + lost] = 0
        assert same(got, want_rows)
    if kind == "e4m3":  # off by at most half a step of the code: 2^-4 of the value, 2^-10 of the scale
        err = (dequantise(*quantise(c.K)) - c.K.double()).abs()
        unit = torch.exp2(quantise(c.K)[1].double() - 127)[..., None]
        assert (err <= torch.maximum(2.0 ** -4 * c.K.double().abs(), 2.0 ** -10 * unit)).all()


def test_write_odd_values(heart):
    """Scales at both ends, rows of zeros, subnormal numbers, rows that are not finite."""
    c = Case([200], [200], kind="e4m3", Hkv=2, page=64, pad=0)
    x = c.K.float()
    for i in range(200):
        x[i] *= 2.0 ** (i - 126 if i < 196 else 100)
    x[150], x[151, 0], x[152, 1, 7], x[153, 0, 127], x[154] = 0.0, 0.0, math.inf, math.nan, -math.inf
    x[155, :, 0], x[156, :, 0] = 448.0 * 2.0 ** 30, 450.0 * 2.0 ** 30
    c.K, c.V = x.to(torch.bfloat16), x.flip(0).to(torch.bfloat16)
    d = Device(heart, c)
    heart.heart_cache_write(d.cfg, d.K, d.V, d.cache, *d.where, d.ws)
    j = torch.arange(200)
    for got, scale, given in ((d.cache.k, d.cache.k_scale, c.K), (d.cache.v, d.cache.v_scale, c.V)):
        codes, scales = quantise(given)
        page, slot = c.table[0].long()[j // 64], j % 64
        assert torch.equal(scale.cpu()[page, :, slot], scales)
        assert torch.equal(got.view(torch.uint8).cpu()[page, :, slot], codes.view(torch.uint8))
    K, V = torch.zeros_like(d.K), torch.zeros_like(d.V)
    heart.heart_cache_read(d.cfg, d.cache, *d.where, K, V, d.ws)
    want = dequantise(*quantise(c.K))
    assert torch.equal(torch.nan_to_num(K.cpu().double(), 7.0), torch.nan_to_num(want, 7.0))
    assert torch.equal(want.to(torch.bfloat16).double().nan_to_num(7.0), want.nan_to_num(7.0))  # (bf16 holds them)


def test_read_into_head_major_tensors(heart):
    """The layout of the calls that take whole tensors."""
    c = Case([150], [150], Hkv=3, Hq=3, page=32, kind="e4m3", pad=0)
    d = Device(heart, c, kv_strides=(D, 150 * D))
    K, V = (torch.zeros((1, 3, 150, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    heart.heart_cache_read(d.cfg, d.cache, *d.where, K, V, d.ws)
    for got, pool in zip((K, V), c.values()):
        assert torch.equal(got.cpu()[0].double(), c.tokens(pool, 0).transpose(0, 1))


ATTENTION = {
    "one token": dict(lens=[1], new=[1]),
    "one token, one key head of eight": dict(lens=[300], new=[1], Hq=8),
    "no token": dict(lens=[0, 40], new=[0, 1]),
    "more new tokens than tokens": dict(lens=[3, 20], new=[5, 20], causal=1),
    "only such": dict(lens=[0], new=[4]),
    "ends in a page": dict(lens=[17, 31, 129], new=[1, 1, 1], Hq=4, Hkv=2, page=16),
    "pages of 128": dict(lens=[127, 128, 129, 1000], new=[1, 2, 1, 1], Hq=4, Hkv=4, page=128),
    "causal": dict(lens=[40, 200, 7], new=[9, 16, 7], causal=1, Hq=3, Hkv=1),
    "causal by groups": dict(lens=[100, 131], new=[64, 100], causal=24, Hq=2, Hkv=2, page=64),
    "window": dict(lens=[500, 90], new=[5, 60], causal=1, window=33, Hq=2, Hkv=2),
    "window of one": dict(lens=[300], new=[20], causal=1, window=1),
    "window and sinks": dict(lens=[700, 20], new=[3, 11], causal=1, window=100, sink=5, Hq=6, Hkv=2, page=32),
    "sinks longer than a step": dict(lens=[900], new=[7], causal=1, window=64, sink=200),
    "window without order": dict(lens=[600], new=[12], window=150, sink=1),
    "groups and window": dict(lens=[400], new=[120], causal=50, window=70, sink=3, page=64),
    "many rows": dict(lens=[300, 260], new=[200, 130], causal=1, Hq=6, Hkv=2, page=32),
    "128 query heads a key head": dict(lens=[150, 33], new=[3, 1], Hq=128, Hkv=1, causal=1),
    "five and seven query heads": dict(lens=[150, 33], new=[30, 33], Hq=35, Hkv=7, page=64, causal=1),
    "a long one": dict(lens=[5000, 3, 2100], new=[1, 1, 1], Hq=4, Hkv=1, page=64),
    "large logits": dict(lens=[400], new=[20], gain=20.0, causal=1, scale=0.05),
    "small scale": dict(lens=[400], new=[2], scale=1e-6),
    "a chunk": dict(lens=[700], new=[300], Hq=2, Hkv=2, page=64),
    "whole tiles": dict(lens=[512, 384], new=[256, 128], Hq=2, Hkv=2, page=128, pad=0),
    "many sequences": dict(lens=[(i * 37) % 90 for i in range(300)], new=[min(1, (i * 37) % 90) for i in range(300)], Hq=2, Hkv=1, page=16),
}


@pytest.mark.parametrize("layout", ["head", "token"])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("name", ATTENTION)
def test_attention(heart, name, kind, layout):
    c = Case(**ATTENTION[name], kind=kind, layout=layout, seed=len(name))
    d = Device(heart, c)
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    check_attention(c, O, lse)
    # once more in the same workspace, without lse, and with no word of how many tokens are new: all kernels
    for max_new in {0, 1, c.T}:
        d.cfg.max_new = max_new
        P, _ = d.attention(lse=False)
        check_attention(c, P, lse)
    assert heart.heart_get_status(d.ws) == 0


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("name", ATTENTION)
def test_attention_by_tiles(heart, name, kind):
    """The kernel for many rows, which a call takes that does not say how few there are, and the same bits every time."""
    c = Case(**{**ATTENTION[name], "pad": 140}, kind=kind, seed=len(name) + 1)
    d = Device(heart, c, max_new=0)
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    check_attention(c, O, lse)
    P, l2 = d.attention()
    assert same(O, P) and same(lse, l2)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_strided_rows(heart, kind):
    """Q and O inside larger tensors, as a fused projection leaves them."""
    c = Case([200, 90], [40, 3], Hq=4, Hkv=2, kind=kind, causal=1)
    d = Device(heart, c, q_strides=(7 * D, D))
    Q, O = (torch.full((c.T, 7, D), 77.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    Q[:, 2:6] = d.Q
    L = torch.full((c.T, c.Hq), 55.0, device="cuda")
    heart.heart_cache_attn(d.cfg, Q[:, 2:6], d.cache, *d.where, O[:, 2:6], d.ws, lse=L)
    check_attention(c, O[:, 2:6].contiguous(), L)
    assert (O[:, :2] == 77).all() and (O[:, 6:] == 77).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_only_rows_that_see_a_nan_get_one(heart, kind):
    for new, max_new in ((6, 6), (6, 0), (140, 140)):
        c = Case([new + 50], [new], Hq=2, kind=kind, causal=1, page=16)
        bad = 50 + new // 2  # a token in the middle of the new ones
        for pool, scale, what in ((c.k, c.k_scale, math.nan), (c.v, c.v_scale, math.inf)):
            page, slot = int(c.table[0, bad // 16]), bad % 16
            if kind == "e4m3":
                scale[page, :, slot] = 255
            else:
                pool[page, :, slot, 5] = what
        d = Device(heart, c, max_new=max_new)
        O, lse = d.attention()
        n = new // 2
        assert torch.isfinite(O[:n]).all() and torch.isfinite(lse[:n]).all()
        assert not torch.isfinite(O[n:new].float()).all(-1).any()
        clean = Case([new + 50], [new], Hq=2, kind=kind, causal=1, page=16)
        want = Device(heart, clean, max_new=max_new).attention()[0]
        assert same(O[:n], want[:n])


def test_bad_arrays_are_reported(heart):
    """Entries out of range: nothing is touched outside the tensors, the status tells, the other sequences are right."""
    for kind in ("bf16", "e4m3"):
        for what in ("page", "negative page", "length", "negative length", "starts", "end"):
            c = Case([100, 80], [3, 2], Hq=2, Hkv=2, kind=kind, causal=1, pad=0)
            d = Device(heart, c)
            table, row_start, kv_len = d.where
            if what == "page":
                table[0, 2] = c.n_pages
            elif what == "negative page":
                table[0, 2] = -1
            elif what == "length":
                kv_len[0] = c.width * c.page + 1
            elif what == "negative length":
                kv_len[0] = -5
            elif what == "starts":
                row_start[0] = -2
            else:
                row_start[2] = c.T + 1
            table[0, 6:] = 0
            O, lse = d.attention()
            assert heart.heart_get_status(d.ws) == heart.ERR_DEVICE_CHECK, what
            assert heart.heart_get_status(d.ws) == 0
            if what not in ("starts", "end"):
                want, _ = c.attention()
                got = O[3:5].cpu().double()
                assert (got - want[3:5]).abs().max() < 0.05
            if what in ("page", "negative page"):
                table[0, -1] = 0
                table[0, 6] = c.n_pages + 5  # the page of the new tokens
            heart.heart_cache_write(d.cfg, d.K, d.V, d.cache, *d.where, d.ws)
            assert heart.heart_get_status(d.ws) == heart.ERR_DEVICE_CHECK, what
            K, V = torch.zeros_like(d.K), torch.zeros_like(d.V)
            heart.heart_cache_read(d.cfg, d.cache, *d.where, K, V, d.ws)
            assert heart.heart_get_status(d.ws) == heart.ERR_DEVICE_CHECK, what


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_run_of_steps(heart, kind):
    """A prompt, then chunks and single tokens, written and attended to, as a program goes: each step against the definition,
    and the context read back at the end into a dense layer-step."""
    g = torch.Generator().manual_seed(3)
    H, page, steps = 2, 16, [37, 1, 1, 20, 1]
    total = sum(steps)
    n_pages, width = 9, 6
    table = torch.randperm(n_pages, generator=g)[:width].to(torch.int32).cuda()[None]
    cache = None
    K, V, Q = (torch.randn((total, H, D), generator=g).to(torch.bfloat16) for _ in range(3))
    at = 0
    for n in steps:
        cfg = heart.make_cache_config(1, n, H, H, page, n_pages, width, kind=heart.CACHE_E4M3 if kind == "e4m3" else heart.CACHE_BF16, max_new=n, causal=1)
        cache = cache or heart.Cache(cfg)
        ws = heart.new_cache_workspace(cfg)
        where = table, torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.tensor([at + n], dtype=torch.int32, device="cuda")
        heart.heart_cache_write(cfg, K[at:at + n].cuda(), V[at:at + n].cuda(), cache, *where, ws)
        O = torch.zeros((n, H, D), dtype=torch.bfloat16, device="cuda")
        heart.heart_cache_attn(cfg, Q[at:at + n].cuda(), cache, *where, O, ws)
        at += n
        assert heart.heart_get_status(ws) == 0
        k, v = ((dequantise(*quantise(x)) if kind == "e4m3" else x.double())[:at].transpose(0, 1) for x in (K, V))
        logits = Q[at - n:at].double().transpose(0, 1) @ k.transpose(1, 2) / math.sqrt(D)
        logits.masked_fill_(torch.arange(at)[None] > torch.arange(at - n, at)[:, None], -math.inf)
        want = (torch.softmax(logits, -1) @ v).transpose(0, 1)
        # (weights and the result rounded once each, 2^-8; |v| below 5 here)
        assert ((O.cpu().double() - want).abs() <= 2 ** -8 * want.abs() + 2 ** -8 * 5).all()
    cfg = heart.make_cache_config(1, total, H, H, page, n_pages, width, kind=heart.CACHE_E4M3 if kind == "e4m3" else heart.CACHE_BF16,
                                  kv_strides=(D, total * D))
    ws = heart.new_cache_workspace(cfg)
    Kr, Vr = (torch.zeros((1, H, total, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    heart.heart_cache_read(cfg, cache, table, torch.tensor([0, total], dtype=torch.int32, device="cuda"),
                           torch.tensor([total], dtype=torch.int32, device="cuda"), Kr, Vr, ws)
    step = heart.make_config(1, H, total, 64, flags=heart.FORCE_DENSE)
    O = torch.zeros_like(Kr)
    Qh = Q.transpose(0, 1).contiguous().cuda()[None]
    heart.heart_block_sparse_attn(step, Qh, Kr, Vr, None, None, O, heart.new_workspace(step))
    want = torch.softmax(Qh.cpu().double() @ Kr.cpu().double().transpose(2, 3) / math.sqrt(D), -1) @ Vr.cpu().double()
    assert ((O.cpu().double() - want).abs() <= 2 ** -8 * want.abs() + 2 ** -8 * 5).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_captured_calls_follow_the_lengths(heart, kind):
    """Write and attention captured once and replayed over other lengths, pages and rows."""
    first = Case([130, 60, 9], [2, 1, 1], Hq=8, Hkv=2, kind=kind, causal=1, garbage=False, seed=1)
    d = Device(heart, first)
    O, lse = torch.zeros_like(d.Q), torch.zeros((first.T, 8), device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        heart.heart_cache_write(d.cfg, d.K, d.V, d.cache, *d.where, d.ws)
        heart.heart_cache_attn(d.cfg, d.Q, d.cache, *d.where, O, d.ws, lse=lse)
    for new, lens, seed in (([2, 1, 1], [130, 60, 9], 5), ([0, 4, 0], [50, 144, 3], 6), ([1, 0, 2], [1, 7, 100], 7)):
        c = Case(lens, new, Hq=8, Hkv=2, kind=kind, causal=1, garbage=False, seed=seed)
        T = first.T
        c.table = torch.randperm(first.n_pages, generator=torch.Generator().manual_seed(seed))[:3 * first.width].reshape(3, -1)[:, :first.width].to(torch.int32) \
            if 3 * first.width <= first.n_pages else first.table.clamp(min=0)
        if 3 * first.width > first.n_pages:  # too few pages for tables of their own: the first sequence's pages in turn
            c.lens = lens = [min(x, len([p for p in first.table[s].tolist() if p >= 0]) * first.page) for s, x in enumerate(lens)]
            c.kv_len = torch.tensor(lens, dtype=torch.int32)
        for to, x in zip(d.where, (c.table, c.row_start, c.kv_len)):
            to.copy_(x)
        rows = min(T, c.T)
        for to, x in ((d.Q, c.Q), (d.K, c.K), (d.V, c.V)):
            to[:rows] = x[:rows].cuda()
        O.fill_(77)
        lse.fill_(55)
        graph.replay()
        torch.cuda.synchronize()
        assert heart.heart_get_status(d.ws) == 0
        c.T, c.Q = T, d.Q.cpu()
        c.k, c.v = d.cache.k.cpu(), d.cache.v.cpu()
        c.k_scale, c.v_scale = (None if x is None else x.cpu() for x in (d.cache.k_scale, d.cache.v_scale))
        check_attention(c, O, lse)


def test_results_repeat(heart):
    """The same bits every time: parts of tiles are put together in order."""
    c = Case([9000, 4000], [1, 1], Hq=4, Hkv=1, page=64, garbage=False)
    d = Device(heart, c)
    O, lse = d.attention()
    for _ in range(20):
        P, l2 = d.attention()
        assert same(O, P) and torch.equal(lse, l2)


def test_offsets_beyond_32_bits(heart):
    """Pools of more than 2^32 bytes: pages at both ends."""
    page, Hkv = 128, 8
    n_pages = (1 << 32) // (page * Hkv * D) + 40  # elements of a pool beyond 2^32
    cfg = heart.make_cache_config(2, 5, 16, Hkv, page, n_pages, 2, causal=1, max_new=3)
    k, v = (torch.empty((n_pages, Hkv, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache, ws = heart.Cache(cfg, k, v), heart.new_cache_workspace(cfg)
    c = Case([200, 140], [3, 2], Hq=16, Hkv=Hkv, page=page, causal=1, pad=0, spare=0)
    pages = torch.tensor([n_pages - 1, 0, n_pages - 2, 7], dtype=torch.int64)
    k[pages.cuda()], v[pages.cuda()] = c.k.cuda(), c.v.cuda()
    table = torch.where(c.table >= 0, pages[c.table.clamp(min=0).long()].to(torch.int32), c.table).cuda()
    O, lse = torch.full_like(c.Q, 77.0).cuda(), torch.full((5, 16), 55.0, device="cuda")
    where = table, c.row_start.cuda(), c.kv_len.cuda()
    heart.heart_cache_attn(cfg, c.Q.cuda(), cache, *where, O, ws, lse=lse)
    check_attention(c, O, lse)
    heart.heart_cache_write(cfg, c.K.cuda(), c.V.cuda(), cache, *where, ws)
    K, V = torch.zeros_like(c.K).cuda(), torch.zeros_like(c.V).cuda()
    heart.heart_cache_read(cfg, cache, *where, K, V, ws)
    assert same(K, c.K) and same(V, c.V)
    assert heart.heart_get_status(ws) == 0


def test_wrong_tensors_are_refused(heart):
    c = Case([50, 20], [2, 1], Hq=4, Hkv=2)
    d = Device(heart, c)
    ok = dict(Q=d.Q, table=d.where[0], row_start=d.where[1], kv_len=d.where[2], O=torch.zeros_like(d.Q), ws=d.ws)

    def call(**kw):
        a = dict(ok, **kw)
        heart.heart_cache_attn(d.cfg, a["Q"], d.cache, a["table"], a["row_start"], a["kv_len"], a["O"], a["ws"], lse=a.get("lse"))

    call()
    for kw in (dict(Q=d.Q.half()), dict(Q=d.Q[1:]), dict(O=d.Q.float()), dict(Q=d.Q.cpu()), dict(table=d.where[0].long()), dict(row_start=d.where[1][1:]),
               dict(kv_len=d.where[2].cpu()), dict(ws=d.ws[:1024]), dict(lse=torch.zeros((c.T, 4), device="cuda", dtype=torch.float64)),
               dict(lse=torch.zeros((c.T, 3), device="cuda")), dict(table=d.where[0].t().contiguous().t()) if c.width > 1 else dict(Q=d.Q.half()),
               dict(Q=torch.zeros((c.T, D, 4), dtype=torch.bfloat16, device="cuda").transpose(1, 2))):
        with pytest.raises(ValueError):
            call(**kw)
    for k in (d.cache.k.half(), d.cache.k[1:], d.cache.k.transpose(1, 2)):
        with pytest.raises(ValueError):
            heart.Cache(d.cfg, k, d.cache.v)
    with pytest.raises(ValueError):
        heart.heart_cache_write(d.cfg, d.K.float(), d.V, d.cache, *d.where, d.ws)
    with pytest.raises(ValueError):
        heart.heart_cache_read(d.cfg, d.cache, *d.where, d.K[:, :1], d.V, d.ws)
