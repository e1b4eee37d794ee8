"""Cross attention on the GPU, against the definition in 64 bits."""
import math
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

D = 128


@pytest.fixture(scope="module")
def heart():
    from paper_2605_14513_b200 import heart as h

    return h


class Case:
    """q, k: queries and states of each sequence.  layout of the states: packed in order, "padded" (a constant pitch), "shuffled" (packed in another order),
    "shared" (all sequences begin at row 1), or "fused" (halves of one projection's rows).  What is no sequence's holds no numbers."""

    def __init__(self, q, k, Hq=2, Hkv=1, layout="packed", scale=0.0, pad=3, seed=0, gain=1.3, fused_q=False, pad_k=0):
        self.q, self.k, self.Hq, self.Hkv, self.scale = list(q), list(k), Hq, Hkv, scale
        g = torch.Generator().manual_seed(seed)
        S = self.S = len(self.q)
        self.T, self.rows = sum(q) + pad, sum(q)
        if layout == "padded":
            first = [s * (max(k) + 2) for s in range(S)]
        elif layout == "shared":
            first = [1] * S
        else:
            order = torch.randperm(S, generator=g).tolist() if layout == "shuffled" else list(range(S))
            first, at = [0] * S, 0
            for s in order:
                first[s] = at
                at += k[s]
        self.first = first
        self.Tk = max(max(f + n for f, n in zip(first, k)), 1) + (2 if layout in ("padded", "shuffled") else 0) + pad_k

        def normal(*shape, k=1.0):
            return (torch.randn(shape, generator=g) * k).to(torch.bfloat16)

        self.fused_q, self.fused_k = fused_q, layout == "fused"
        self.Q, self.K, self.V = normal(self.T, Hq, D, k=gain), normal(self.Tk, Hkv, D), normal(self.Tk, Hkv, D)
        used = torch.zeros(self.Tk, dtype=torch.bool)
        for f, n in zip(first, k):
            used[f:f + n] = True
        for x in (self.K, self.V):
            x[~used] = torch.tensor([math.nan, math.inf, -math.inf, 1e30] * 32, dtype=torch.bfloat16)
        i32 = dict(dtype=torch.int32)
        self.q_start = torch.tensor([sum(self.q[:s]) for s in range(S + 1)], **i32)
        self.k_start, self.k_len = torch.tensor(first, **i32), torch.tensor(self.k, **i32)

    def attention(self):
        """O, lse, and sum_j w_j |v_j|, which roundings of the weights are relative to, of the sequences' rows."""
        O, B = torch.zeros((self.rows, self.Hq, D), dtype=torch.float64), torch.zeros((self.rows, self.Hq, D), dtype=torch.float64)
        lse = torch.full((self.rows, self.Hq), -math.inf, dtype=torch.float64)
        scale = self.scale if self.scale > 0 else 1 / math.sqrt(D)
        for s in range(self.S):
            r0, n, f, L = int(self.q_start[s]), self.q[s], self.first[s], self.k[s]
            for h in range(self.Hq if n and L else 0):
                k, v = (x[f:f + L, h // (self.Hq // self.Hkv)].double() for x in (self.K, self.V))
                logits = self.Q[r0:r0 + n, h].double() @ k.T * scale
                lse[r0:r0 + n, h] = torch.logsumexp(logits, -1)
                w = torch.softmax(logits, -1)
                O[r0:r0 + n, h], B[r0:r0 + n, h] = w @ v, w @ v.abs()
        return O, lse, B


class Device:
    def __init__(self, heart, c, device="cuda", **kw):
        self.c, self.heart = c, heart
        kw.setdefault("max_q", max(c.q))
        if c.fused_q:
            kw["q_strides"] = (3 * c.Hq * D, D)
        if c.fused_k:
            kw["kv_strides"] = (2 * c.Hkv * D, D)
        self.cfg = heart.make_cross_config(c.S, c.T, c.Tk, c.Hq, c.Hkv, scale=c.scale, **kw)
        if c.fused_k:
            both = torch.stack((c.K, c.V), 1).to(device)
            self.K, self.V = both[:, 0], both[:, 1]
        else:
            self.K, self.V = c.K.to(device), c.V.to(device)
        self.Q = self._rows(c.Q.to(device))
        self.where = c.q_start.to(device), c.k_start.to(device), c.k_len.to(device)
        self.ws = heart.new_cross_workspace(self.cfg, device=device)

    def _rows(self, x):
        if not self.c.fused_q:
            return x
        wide = torch.full((self.c.T, 3, self.c.Hq, D), 77.0, dtype=torch.bfloat16, device=x.device)
        wide[:, 1] = x
        return wide[:, 1]

    def attention(self, lse=True):
        O = self._rows(torch.full((self.c.T, self.c.Hq, D), 77.0, dtype=torch.bfloat16, device=self.Q.device))
        L = torch.full((self.c.T, self.c.Hq), 55.0, device=self.Q.device) if lse else None
        self.heart.heart_cross_attn(self.cfg, self.Q, self.K, self.V, *self.where, O, self.ws, lse=L)
        return O, L


def same(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16)) if a.dtype == torch.bfloat16 else torch.equal(a, b)


def check(c, O, lse):
    """Rows of no sequence are as they were (77, 55)."""
    want, want_lse, weights = c.attention()
    if c.fused_q:
        wide = O._base if O._base is not None else O
        assert (wide[:, 0] == 77).all() and (wide[:, 2] == 77).all()
    O = O.cpu()
    assert (O[c.rows:] == 77).all()
    got = O[:c.rows].double()
    empty = want_lse == -math.inf
    assert (got[empty] == 0).all()
    # A weight is rounded to bf16 once (half a step: 2^-8 of it), the result once more; products are exact in 32 bits, their sums off by less than
    # 2^-17 of the sum of magnitudes (128 to some 10^4 terms, each sum rounded by 2^-24; the exponent's argument, up to 2^6, by 2^-18 of one:
    # weights by as much).
    bound = (2 ** -8 + 2 ** -12) * weights + 2 ** -8 * want.abs() + 1e-30
    worst = ((got - want).abs() / bound)[~empty]
    assert worst.numel() == 0 or worst.max() <= 1.0, float(worst.max())
    if lse is not None:
        lse = lse.cpu()
        assert (lse[c.rows:] == 55).all() and (lse[:c.rows][empty] == -math.inf).all()
        off = (lse[:c.rows].double() - want_lse)[~empty].abs()
        assert off.numel() == 0 or off.max() <= 2 ** -14, float(off.max())  # (logits up to 2^6, 32-bit sums of 128 products)


CASES = {
    "one token over one state": dict(q=[1], k=[1]),
    "one token": dict(q=[1], k=[300], Hq=8, Hkv=2),
    "no state": dict(q=[1, 5], k=[0, 7]),
    "no state at all": dict(q=[4], k=[0]),
    "no query": dict(q=[0, 3, 0, 1], k=[5, 0, 9, 77], Hq=4, Hkv=4),
    "tokens": dict(q=[1] * 9, k=[3, 16, 17, 128, 129, 127, 1000, 1, 64], Hq=3, Hkv=3, layout="padded"),
    "drafted tokens": dict(q=[4, 1, 8], k=[200, 33, 515], Hq=2, Hkv=1, layout="fused"),
    "77 states": dict(q=[130], k=[77], Hq=4, Hkv=4),
    "a chunk over a text": dict(q=[300, 257], k=[512, 226], Hq=2, Hkv=2, layout="shuffled"),
    "whole tiles": dict(q=[256, 128], k=[256, 128], Hq=2, Hkv=2, pad=0),
    "shared states": dict(q=[140, 3, 60], k=[300, 300, 11], Hq=4, Hkv=2, layout="shared"),
    "five and seven query heads": dict(q=[31, 140], k=[150, 33], Hq=35, Hkv=7, layout="fused"),
    "three query heads": dict(q=[200], k=[140], Hq=6, Hkv=2, fused_q=True),
    "128 query heads a key head": dict(q=[3, 1], k=[150, 33], Hq=128, Hkv=1),
    "100 query heads a key head": dict(q=[3, 2], k=[150, 33], Hq=100, Hkv=1),
    "long states": dict(q=[20, 1], k=[9000, 2100], Hq=2, Hkv=1),
    "one step of 16": dict(q=[500], k=[16], Hq=3, Hkv=3),
    "tokens among rows": dict(q=[1, 400, 1, 1], k=[300, 1, 0, 129], Hq=6, Hkv=2),
    "no state of many rows": dict(q=[300, 200], k=[0, 0], Hq=2, Hkv=2),
    "no query of many": dict(q=[0, 300, 0, 1], k=[5, 0, 9, 77], Hq=4, Hkv=4),
    "a step and a state": dict(q=[140, 140], k=[129, 1], layout="shuffled"),
    "long states of several": dict(q=[200, 70, 300], k=[3000, 2200, 5000], Hq=6, Hkv=2, layout="shuffled"),
    "large logits": dict(q=[140], k=[400], gain=20.0, scale=0.05),
    "large logits of many": dict(q=[240], k=[400], gain=20.0, scale=0.05),
    "small scale of many": dict(q=[420], k=[400], scale=1e-6),
    "small scale": dict(q=[20], k=[400], scale=1e-6),
    "tokens of short and long states": dict(q=[1, 0, 1, 1, 1, 0, 1, 1], k=[2000, 5, 1, 0, 130, 700, 90, 1500], Hq=24, Hkv=24, layout="shuffled"),
    "tokens of short states": dict(q=[(i * 5 + 1) % 4 for i in range(20)], k=[(i * 137 + 60) % 512 for i in range(20)], Hq=24, Hkv=12, layout="shuffled"),
    "tokens of middling states": dict(q=[(i * 5 + 1) % 3 for i in range(30)], k=[(i * 137 + 60) % 1000 for i in range(30)], Hq=24, Hkv=24, layout="fused"),
    "batch of tokens": dict(q=[(i * 5) % 3 for i in range(400)], k=[(i * 137) % 600 for i in range(400)], Hq=8, Hkv=4),
    "many sequences": dict(q=[(i * 7) % 5 for i in range(700)], k=[(i * 37) % 90 for i in range(700)]),
    "40 sequences": dict(q=[(i * 53) % 150 for i in range(40)], k=[(i * 37) % 190 for i in range(40)], layout="shuffled", Hq=3, Hkv=3),
    "many tiles": dict(q=[2500, 4], k=[200, 300], Hq=12, Hkv=12, fused_q=True),
}


@pytest.mark.parametrize("name", CASES)
def test_attention(heart, name):
    c = Case(**CASES[name], seed=len(name))
    d = Device(heart, c)
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    check(c, O, lse)
    # the kernel for the other number of rows, without lse, in the same workspace; the same bits every time
    for max_q in (1, 0):
        d.cfg.max_q = max_q
        P, _ = d.attention(lse=False)
        check(c, P, None)
        R, _ = d.attention()
        assert same(P, R)
    assert heart.heart_get_status(d.ws) == 0


PAIRS = ("77 states", "a chunk over a text", "whole tiles", "shared states", "five and seven query heads", "three query heads", "long states", "long states of several", "one step of 16",
         "a step and a state", "large logits", "many sequences", "40 sequences")


@pytest.mark.parametrize("name", PAIRS)
def test_large_tensors_of_states(heart, name):
    """More than 64 MB of keys and values, most of them no sequence's: two CTAs share what they read."""
    c = Case(**CASES[name], seed=len(name), pad_k=140000 // CASES[name].get("Hkv", 1))
    d = Device(heart, c, max_q=0)
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    check(c, O, lse)
    P, _ = d.attention(lse=False)
    assert same(O, P)


@pytest.mark.parametrize("q,k", [([4700, 0, 130, 4700], [70, 9, 1, 300]), ([9500], [33]), ([19100], [33])])
def test_many_tiles_a_cta(heart, q, k):
    c = Case(q, k, Hq=32, Hkv=32, layout="fused", seed=sum(q))
    d = Device(heart, c)
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    check(c, O, lse)


@pytest.mark.parametrize("name", ["rows", "tiles", "shared tiles", "pairs", "shared tiles of pairs"])
def test_a_wait_that_runs_out_is_reported(heart, name):
    """In the test-hook build a flag makes one CTA leave out a copy: its waits run out after a millisecond, the status tells, and the next
    call in the same workspace is right."""
    from paper_2605_14513_b200 import build

    product = heart.lib()
    q, k = {"rows": ([1], [8192])}.get(name, ([200, 700], [600, 300]) if "shared" not in name else ([300], [4000]))
    c = Case(q, k, Hq=2, Hkv=2, pad_k=70000 if "pairs" in name else 0)
    try:
        heart._lib = heart.load(build.build_test_hooks())
        d = Device(heart, c)
        want = d.attention()
        assert heart.heart_get_status(d.ws) == 0
        check(c, *want)
        d.cfg.flags = 0x80000000
        t0 = time.perf_counter()
        d.attention()
        assert heart.heart_get_status(d.ws) == heart.ERR_DEVICE_CHECK
        assert time.perf_counter() - t0 < 5.0
        d.cfg.flags = 0
        for _ in range(3):
            O, lse = d.attention()
            assert heart.heart_get_status(d.ws) == 0
            assert same(O, want[0]) and same(lse, want[1])
    finally:
        heart._lib = product


@pytest.mark.parametrize("q,max_q", [(6, 6), (6, 0), (140, 140)])
def test_only_rows_that_see_a_nan_get_one(heart, q, max_q):
    """A state that is not finite is one of the second sequence's; the first one's rows are as they are without it, bit by bit."""
    clean = Case([q, q], [50, 70], Hq=2)
    want, _ = Device(heart, clean, max_q=max_q).attention()
    for what, where in ((math.nan, "K"), (math.inf, "V"), (-math.inf, "V"), (math.nan, "V")):
        c = Case([q, q], [50, 70], Hq=2)
        getattr(c, where)[50 + 13, 0, 5] = what
        O, lse = Device(heart, c, max_q=max_q).attention()
        assert same(O[:q], want[:q]) and torch.isfinite(lse[:q]).all()
        assert not torch.isfinite(O[q:2 * q].float()).all(-1).any()
    # a logit of -inf has no weight
    c, d = Case([q], [60], Hq=1), Case([q], [60], Hq=1)
    for x in (c, d):
        x.Q[:, :, 5] = x.Q[:, :, 5].abs() + 1
    c.K[59, 0, 5] = -math.inf
    d.k_len[0], d.k[0] = 59, 59
    a, b = Device(heart, c, max_q=max_q).attention()[0], Device(heart, d, max_q=max_q).attention()[0]
    assert torch.isfinite(a[:q].float()).all()
    assert (a[:q].float() - b[:q].float()).abs().max() <= 2 ** -7 * 5


@pytest.mark.parametrize("max_q,many", [(1, 1), (0, 1), (0, 60)])
def test_bad_arrays_are_reported(heart, max_q, many):
    """Entries out of range: nothing is touched outside the tensors, the status tells, the other sequence is right."""
    for what in ("starts", "end", "descending", "length", "negative length", "first", "negative first"):
        c = Case([4 * many, 3 * many], [100, 80], Hq=2, Hkv=2, pad=0)
        d = Device(heart, c, max_q=max_q)
        q_start, k_start, k_len = d.where
        if what == "starts":
            q_start[0] = -2
        elif what == "end":
            q_start[2] = c.T + 1
        elif what == "descending":
            q_start[1] = c.T + 2
        elif what == "length":
            k_len[0] = c.Tk + 1
        elif what == "negative length":
            k_len[0] = -5
        elif what == "first":
            k_start[0] = c.Tk - 99
        else:
            k_start[0] = -1
        O, _ = d.attention()
        assert heart.heart_get_status(d.ws) == heart.ERR_DEVICE_CHECK, what
        assert heart.heart_get_status(d.ws) == 0
        if what not in ("starts", "end", "descending"):
            want, _, _ = c.attention()
            assert (O[4 * many:].cpu().double() - want[4 * many:]).abs().max() < 0.05, what
    # of a sequence without states it does not matter where they begin
    c = Case([4 * many, 3 * many], [0, 80], Hq=2, Hkv=2)
    d = Device(heart, c, max_q=max_q)
    d.where[1][0] = -9
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    check(c, O, lse)


@pytest.mark.parametrize("max_q", [3, 200])
def test_captured_calls_follow_the_lengths(heart, max_q):
    first = Case([max_q, 2, 1], [130, 60, 9], Hq=4, Hkv=2, seed=1, pad=9)
    d = Device(heart, first, max_q=max_q)
    O, lse = torch.zeros_like(d.Q), torch.zeros((first.T, 4), device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        heart.heart_cross_attn(d.cfg, d.Q, d.K, d.V, *d.where, O, d.ws, lse=lse)
    for q, k in (([max_q, 2, 1], [130, 60, 9]), ([0, 3, 2], [1, 190, 8]), ([1, 0, 2], [0, 100, 99])):
        c = Case(q, k, Hq=4, Hkv=2, seed=5, pad=first.T - sum(q))
        for to, x in ((d.Q, c.Q), (d.K, c.K), (d.V, c.V), *zip(d.where, (c.q_start, c.k_start, c.k_len))):
            to[:min(len(to), len(x))].copy_(x[:min(len(to), len(x))])
        O.fill_(77)
        lse.fill_(55)
        graph.replay()
        torch.cuda.synchronize()
        assert heart.heart_get_status(d.ws) == 0
        check(c, O, lse)


@pytest.mark.parametrize("max_q", [4, 200])
def test_two_graphs_share_a_workspace(heart, max_q):
    """One after the other, in any order, between plain calls; shared tiles among them."""
    cases = [Case([max_q, 1], [3000, 20], Hq=2, Hkv=2, seed=1), Case([2, max_q], [5000, 2300], Hq=2, Hkv=1, seed=2)]
    devices = [Device(heart, c, max_q=max_q) for c in cases]
    ws = devices[0].ws
    want = []
    for d in devices:
        d.ws = ws
        want.append(d.attention())
    for c, w in zip(cases, want):
        check(c, *w)
    graphs, out = [], []
    for d in devices:
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        O, lse = torch.zeros_like(d.Q), torch.zeros((d.c.T, d.c.Hq), device="cuda")
        with torch.cuda.graph(graph, stream=stream):
            heart.heart_cross_attn(d.cfg, d.Q, d.K, d.V, *d.where, O, ws, lse=lse)
        graphs.append(graph)
        out.append((O, lse))
    for i in (0, 1, 1, 0, 0, 1):
        for x in out[i]:
            x.fill_(9)
        graphs[i].replay()
        other = devices[1 - i].attention()
        rows = cases[i].rows
        assert same(out[i][0][:rows], want[i][0][:rows]) and same(out[i][1][:rows], want[i][1][:rows])
        assert same(other[0], want[1 - i][0]) and same(other[1], want[1 - i][1])
    assert heart.heart_get_status(ws) == 0


@pytest.mark.parametrize("q,k", [([3, 1], [40, 170]), ([150, 60], [200, 33])])
def test_heads_first_and_rows_ahead(heart, q, k):
    """Heads are the outer dimension of all tensors; rows before the first sequence are left as they are."""
    c = Case(q, k, Hq=6, Hkv=2, seed=7)
    ahead = 5
    want, want_lse, _ = c.attention()
    O = torch.full((c.Hq, c.T + ahead, D), 77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.T + ahead, c.Hq), 55.0, device="cuda")
    Q = torch.full_like(O, math.nan)
    Q[:, ahead:] = c.Q.transpose(0, 1).cuda()
    K, V = (x.transpose(0, 1).contiguous().cuda() for x in (c.K, c.V))
    cfg = heart.make_cross_config(c.S, c.T + ahead, c.Tk, c.Hq, c.Hkv, max_q=max(q), q_strides=(D, (c.T + ahead) * D), kv_strides=(D, c.Tk * D))
    ws = heart.new_cross_workspace(cfg)
    heart.heart_cross_attn(cfg, Q, K, V, (c.q_start + ahead).cuda(), c.k_start.cuda(), c.k_len.cuda(), O, ws, lse=lse)
    assert heart.heart_get_status(ws) == 0
    assert (O[:, :ahead] == 77).all() and (lse[:ahead] == 55).all()
    check(c, O[:, ahead:].transpose(0, 1).contiguous(), lse[ahead:])


def test_two_streams_with_workspaces_of_their_own(heart):
    cases = [Case([300, 40], [900, 70], Hq=4, Hkv=2, seed=i) for i in range(2)]
    devices = [Device(heart, c) for c in cases]
    want = [d.attention() for d in devices]
    streams = [torch.cuda.Stream() for _ in devices]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for d, s in zip(devices, streams):
            with torch.cuda.stream(s):
                got.append((d, d.attention()))
    torch.cuda.synchronize()
    for d, (O, lse) in got:
        O2, lse2 = want[devices.index(d)]
        assert same(O, O2) and same(lse, lse2)
    for c, (O, lse) in zip(cases, want):
        check(c, O, lse)


@pytest.mark.parametrize("max_q,Hq,Hkv", [(1, 2, 1), (0, 2, 1), (0, 10, 5)])
def test_offsets_beyond_32_bits(heart, max_q, Hq, Hkv):
    """K, V, Q and O of more than 2^32 elements, by their strides."""
    rows, far = 40, 1 << 27  # (elements between rows)
    c = Case([rows], [rows], Hq=Hq, Hkv=Hkv, pad=0)
    room = (rows - 1) * far + Hq * D
    Q, O, K, V = (torch.empty(room, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    view = [x.as_strided((rows, h, D), (far, D, 1)) for x, h in ((Q, Hq), (O, Hq), (K, Hkv), (V, Hkv))]
    for to, x in zip(view, (c.Q, c.Q, c.K, c.V)):
        to.copy_(x)
    cfg = heart.make_cross_config(1, rows, rows, Hq, Hkv, max_q=max_q, q_strides=(far, D), kv_strides=(far, D))
    ws = heart.new_cross_workspace(cfg)
    heart.heart_cross_attn(cfg, view[0], view[2], view[3], c.q_start.cuda(), c.k_start.cuda(), c.k_len.cuda(), view[1], ws)
    assert heart.heart_get_status(ws) == 0
    check(c, view[1].contiguous(), None)


def test_wrong_tensors_are_refused(heart):
    c = Case([5, 2], [50, 20], Hq=4, Hkv=2)
    d = Device(heart, c)
    ok = dict(Q=d.Q, K=d.K, V=d.V, q_start=d.where[0], k_start=d.where[1], k_len=d.where[2], O=torch.zeros_like(d.Q), ws=d.ws)

    def call(**kw):
        a = dict(ok, **kw)
        heart.heart_cross_attn(d.cfg, a["Q"], a["K"], a["V"], a["q_start"], a["k_start"], a["k_len"], a["O"], a["ws"], lse=a.get("lse"))

    call()
    for kw in (dict(Q=d.Q.half()), dict(Q=d.Q[1:]), dict(O=d.Q.float()), dict(Q=d.Q.cpu()), dict(K=d.K.cpu()), dict(V=d.V[:-1]), dict(q_start=d.where[0].long()),
               dict(q_start=d.where[0][1:]), dict(k_len=d.where[2].cpu()), dict(k_start=d.where[0]), dict(ws=d.ws[:1024]), dict(ws=d.ws.cpu()),
               dict(lse=torch.zeros((c.T, 4), device="cuda", dtype=torch.float64)), dict(lse=torch.zeros((c.T, 3), device="cuda")),
               dict(K=torch.zeros((c.Tk, D, 2), dtype=torch.bfloat16, device="cuda").transpose(1, 2))):
        with pytest.raises(ValueError):
            call(**kw)
